// Whole prompts: causal attention of packed sequences with grouped heads, and the
// attention weight that each position received from the last rows of its sequence.
// Contract: include/oilbird.h.
//
// attend: the rows of a (sequence, key/value head) are its tokens' queries of the G
// heads that share it, row = token * G + g, so that short sequences fill tiles and a
// tile's tokens lie close together.  A workgroup takes a tile of rows, 32 a wave, and
// passes over the keys once, 64 at a time, from LDS: S^T = K Q^T on matrix cores (a
// lane's column is one row of queries, so that the softmax's statistics are its own),
// the running maximum m and sum l in binary32, P = exp2(S c - m) rounded to bf16 where
// it lies (the registers of S^T are the operand's, under the order of the keys that
// V's transposing reads give), O^T += V^T P.  m is the largest score of the first tile
// and stays, unseen, until a lane's weights of a tile pass kMost, when m rises, they are
// made anew, and sums and outputs are scaled.
// c is log2 e times the scale, rounded, and so is m, while S c is exact: where scores are
// so large that this tells (kFar), and wherever else a result is not finite, a second pass
// makes the row from (S - max S) scale.
// Bound by matrix cores, exponentials and LDS, which overlap in part: at 128 columns a wave's
// tile of 64 keys is 32 matrix instructions of 32 cycles, some 560 cycles of exponentials,
// scaling and sums, and 256 cycles of LDS, which the CU's eight waves share.  So the matrix
// cores are busy 0.65 of the cycles of 16,384 rows (0.41 of 48 short sequences'); a library
// product of 16,384^3 on the same card keeps them busy 0.90 of the cycles at the same clock, 1.7 GHz.
// 16,384 rows, 32 heads over 8 of 128 columns: 1,895 to 2,060 us on different cards, 1,070 to
// 1,160 TFLOP/s (the library product: 1,586); 8,191 rows 497 to 537 us; 65,533 rows, 2
// heads over 1: 1,950 to 2,110 us; 48 sequences of 390 to 1,500 rows 585 to 630 us, 720 to 780: a
// workgroup passes over some ten tiles there, and 6 of its 20 us are its first loads and its end.
// 8,191 rows of 64 columns 292 us; 72 to 120 columns are made as 128 are (72: 440 us, 96: 460).
//
// weigh: a lane's column is a key, S = Q K^T, and the sums of exp2(S c - lse) stay in
// registers: no two workgroups add to one sum, so the result does not depend on the order
// in which they run.  Bound by exponentials beside the products, of which there is one a
// score here: without either the other alone takes three quarters of the time.  8,192 rows
// over themselves, 32 heads over 8 of 128 columns: 302 to 312 us, 880 to 910 TFLOP/s; four sequences
// of 2,866 to 8,191 rows, their last 64 rows: 26 us, of which the list 4; the keys are 45 MB.
#include "common.hpp"
#include "internal.hpp"

#include <type_traits>

namespace oil {

namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef float floatx2 __attribute__((ext_vector_type(2)));
typedef short shortx4 __attribute__((ext_vector_type(4)));

#define LDS_PTR(T, p) ((T __attribute__((address_space(3)))*)(p))

constexpr int kKeys = 64;       // keys of a tile
constexpr int kWeighKeys = 64;   // keys of a wave
constexpr int kWeighRows = 128;  // rows of a tile
constexpr int kMaxSeqs = 512;
// The most that a lane's 32 weights of a tile may add up to: what is rounded to bf16 keeps its relative
// precision whatever m is, and sums of 2^30 such weights stay within binary32.  Their products with values need
// not, though what they are divided to does: such results are made again with weights that add up to less than 1.
constexpr float kMost = 256.f;
// Scores in base 2 from which on, in size, binary32 holds m with an error that matters beside them.
constexpr float kFar = 0x1p24f;
// An lse from which on, in size, weights are not taken from S c - lse log2 e: its roundings are some 2.5 x 2^-24
// of lse, 2^-10.7 of a weight here.
constexpr float kFarLse = 0x1p12f;
constexpr float kLargest = 0x1.FEp127f;  // of bf16
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
// A byte offset past every buffer's end (128 rows of 2^25 bytes at most): reads as zero.
constexpr uint32_t kOutside = 0xFFFFFF00u;

union Operand {
    u32x4 w;
    bf16x8 b;
    shortx4 h[2];
};

// The larger of each two 16-bit whole numbers.
__device__ __forceinline__ uint32_t max_u16(uint32_t a, uint32_t b)
{
    typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b)));
}

__device__ __forceinline__ uint32_t pack2(float a, float b)
{
    const floatx2 x = {a, b};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(x, bf16x2));
}

// bf16 values times zero, without the sign: NaN where they are not finite (all bits of the exponent set).
__device__ __forceinline__ u32x4 times_zero(u32x4 w)
{
#pragma unroll
    for (int e = 0; e < 4; e++)
        w[e] = (((w[e] & 0x7F807F80u) + 0x00800080u) >> 15 & 0x00010001u) * 0x7FC0u;
    return w;
}

// A value beside its counterpart 32 lanes away.
__device__ __forceinline__ void swap32(float x, float* a, float* b)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    *a = __uint_as_float(r[0]);
    *b = __uint_as_float(r[1]);
}

// A workgroup's share of the work: tile `tile` of the sequence of rows first .. first +
// len - 1; none with len 0.
struct Tile {
    int first, len, tile, pad;
};

template <int kControl>
__device__ __forceinline__ int add_moved(int x)
{
    return x + __builtin_amdgcn_update_dpp(0, x, kControl, 0xF, 0xF, true);
}

// The sum over a wave, in every lane.
__device__ __forceinline__ int wave_sum(int x)
{
    x = add_moved<0xB1>(x);   // lane ^ 1
    x = add_moved<0x4E>(x);   // lane ^ 2
    x = add_moved<0x141>(x);  // mirrored in 8
    x = add_moved<0x140>(x);  // mirrored in 16
    auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    x = r[0] + r[1];
    r = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    return __builtin_amdgcn_readfirstlane(r[0] + r[1]);
}

// The tiles of all sequences, (len * per + rows - 1) / rows of each: the longest sequence
// first (ties by number), of each the tiles of the largest number first.  So the
// workgroups that run at one time read the keys of few sequences, from L2, and the last
// ones are short.  (The largest numbers of all sequences first: 48 sequences of up to
// 1,500 tokens took 1.13 times as long; their keys came from memory again and again.  A search in
// every workgroup instead of the list: 3.3 us of 28.)  A wave takes every so many sequences.
constexpr int kListWaves = 128;

__global__ __launch_bounds__(256) void prompt_list_kernel(const int32_t* __restrict__ starts, int32_t B, int32_t T,
                                                          int32_t per, int32_t rows, Tile* __restrict__ list,
                                                          int32_t places)
{
    const int lane = threadIdx.x & 63, wave = blockIdx.x * 4 + (threadIdx.x >> 6);
    auto tiles = [&](int s, int* from, int* size) {
        *from = seq_first(starts, T, s);
        *size = seq_end(starts, T, s) - *from;
        return (int)(((int64_t)*size * per + rows - 1) / rows);
    };
    int n[kMaxSeqs / 64], all = 0, from, size;
#pragma unroll
    for (int i = 0; i < kMaxSeqs / 64; i++) {
        n[i] = i * 64 + lane < B ? tiles(i * 64 + lane, &from, &size) : 0;
        all += n[i];
    }
    all = wave_sum(all);
    // starts that do not ascend can name more tiles than there are places, or than 31 bits hold
    all = (uint32_t)all > (uint32_t)places ? places : all;
    for (int s = wave; s < B; s += kListWaves) {
        const int mine = tiles(s, &from, &size);
        int before = 0;
#pragma unroll
        for (int i = 0; i < kMaxSeqs / 64; i++)
            before += n[i] > mine || (n[i] == mine && i * 64 + lane < s) ? n[i] : 0;
        before = wave_sum(before);
        for (int t = lane; t < mine; t += 64)
            if ((uint32_t)(before + mine - 1 - t) < (uint32_t)places)
                list[before + mine - 1 - t] = Tile{from, size, t, 0};
    }
    for (int i = all + wave * 64 + lane; i < places; i += kListWaves * 64)
        list[i] = Tile{0, 0, 0, 0};
}

// Workgroup `rank`'s tile; of one sequence it is known without a list.
__device__ __forceinline__ Tile tile_of(const Tile* list, const int32_t* starts, int32_t T, int rank, int per, int rows)
{
    if (list)
        return list[rank];
    Tile r;
    r.first = seq_first(starts, T, 0);
    r.len = seq_end(starts, T, 0) - r.first;
    r.tile = (int)(((int64_t)r.len * per + rows - 1) / rows) - 1 - rank;
    if (r.tile < 0)
        r.len = 0;
    return r;
}

// A buffer's descriptor: address, bytes (reads past them give zeros), raw 32-bit data.
__device__ __forceinline__ u32x4 rows_at(uint64_t a, uint32_t bytes)
{
    return u32x4{(uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)a),
                 (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)(a >> 32)) & 0xFFFFu,
                 (uint32_t)__builtin_amdgcn_readfirstlane(bytes), 0x00020000u};
}

// 16 bytes a lane, at byte `from` of the buffer (zeros past its end), straight to LDS:
// one KiB from `to` on, lane by lane.  In asm because the compiler would wait for all of
// them before any later read of LDS, the other half of a double buffer's among them; it
// has no output registers, and loads_done() comes before what it loads is read.
__device__ __forceinline__ void load_kib(u32x4 r, uint8_t* to, uint32_t from)
{
    const uint32_t at = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)LDS_PTR(uint8_t, to));
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
                 :
                 : "s"(at), "v"(from), "s"(r)
                 : "m0", "memory");
}

// Of 64 values that 16 lanes hold the addresses of, four each (a matrix of four rows of
// 16): lane i's column i.
__device__ __forceinline__ shortx4 column_of(const uint8_t* p)
{
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16(LDS_PTR(shortx4, p));
}

// Waits until none of the wave's loads is in flight.
__device__ __forceinline__ void loads_done()
{
    __builtin_amdgcn_s_waitcnt((7 << 4) | (15 << 8));
    __builtin_amdgcn_sched_barrier(0);
}

// Where 16-byte chunk `chunk` of row `row` of a tile of rows of W values lies in LDS:
// permuted so that 16 consecutive rows' like chunks lie in 16 different places (keys;
// read 16 bytes a lane, a row a lane) or that four consecutive rows' like 64 bytes do
// (values, whose transposing reads take 8 bytes a lane of four rows).
template <int W>
__device__ __forceinline__ int key_place(int row, int chunk)
{
    return row * (W / 8) + (W == 128 ? chunk ^ (row & 15) : chunk ^ ((row >> 1) & 7));
}
template <int W>
__device__ __forceinline__ int value_place(int row, int chunk)
{
    return row * (W / 8) + (W == 128 ? chunk ^ ((row & 3) << 2) : chunk ^ ((row & 2) << 1));
}

struct Attend {
    const Tile* list;
    const int32_t* starts;
    const uint16_t *q, *k, *v;
    int64_t q_ld, ld;
    uint16_t* out;
    float* lse;
    int32_t T, G, H, D;
    float scale;
};

template <int W, int NW>
__global__ __launch_bounds__(NW * 64, 2) void prompt_attend_kernel(Attend)
{
    constexpr int kTile = kKeys * W * 2;          // bytes
    constexpr int kLoads = kTile / 1024 / NW;     // 1 KiB loads of a wave, a side
    constexpr int kRows = 32 * NW;
    __shared__ __align__(1024) uint8_t key_lds[2][kTile];
    __shared__ __align__(1024) uint8_t value_lds[2][kTile];
    __shared__ int odd_lds[2][NW];                // whether a wave's part of the values is not finite
    const int lane = threadIdx.x & 63, col = lane & 31, half = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // The arguments, read where they are used: held throughout they would take the scalar
    // registers that the loop over the keys needs.
    auto args = [&]() {
        const Attend __attribute__((address_space(4)))* p =
            (const Attend __attribute__((address_space(4)))*)__builtin_amdgcn_kernarg_segment_ptr();
        asm volatile("" : "+s"(p));
        return p;
    };

    // loads: chunk `lane` of each KiB from where its place in LDS says
    uint32_t key_from[kLoads], value_from[kLoads];
    const uint32_t row_bytes = (uint32_t)args()->ld * 2, value_bytes = args()->D * 2;
#pragma unroll
    for (int i = 0; i < kLoads; i++) {
        const int at = (wave * kLoads + i) * 64 + lane, r = at / (W / 8);
        const int kc = key_place<W>(r, at % (W / 8)) - r * (W / 8), vc = value_place<W>(r, at % (W / 8)) - r * (W / 8);
        key_from[i] = kc * 16 < (int)value_bytes ? r * row_bytes + kc * 16 : kOutside;
        value_from[i] = vc * 16 < (int)value_bytes ? r * row_bytes + vc * 16 : kOutside;
    }
    int key_at[W / 16], value_at[W / 32];
#pragma unroll
    for (int i = 0; i < W / 16; i++)
        key_at[i] = key_place<W>(col, 2 * i + half) * 16;
#pragma unroll
    for (int i = 0; i < W / 32; i++)
        value_at[i] = value_place<W>(4 * half + (lane & 15) / 4, i * 4 + 2 * (col >> 4) + ((lane & 3) >> 1)) * 16 +
                      (lane & 1) * 8;
    const float scale = args()->scale, c = scale == 0.f ? 1.f : fabsf(scale) * kLog2e;

    // its sequence's rows and where its keys and values begin, the lane's token,
    // tiles of keys that the workgroup sees, and how many of them every row of it sees whole
    int len, token, tiles, whole;
    uint64_t key_base, value_base;
    int to;  // the row and head of the outputs, -1 past the sequence
    // rows t kKeys .. of a side; none past the sequence
    auto tile_rows = [&](uint64_t side, int t) {
        const int left = len - t * kKeys < kKeys ? len - t * kKeys : kKeys;
        return rows_at(side + (uint64_t)(t * kKeys) * row_bytes, left > 0 ? (left - 1) * row_bytes + value_bytes : 0u);
    };
    auto load_keys = [&](int t) {
        const u32x4 r = tile_rows(key_base, t);
#pragma unroll
        for (int i = 0; i < kLoads; i++)
            load_kib(r, &key_lds[t & 1][(wave * kLoads + i) * 1024], key_from[i]);
    };
    auto load_values = [&](int t) {
        const u32x4 r = tile_rows(value_base, t);
#pragma unroll
        for (int i = 0; i < kLoads; i++)
            load_kib(r, &value_lds[t & 1][(wave * kLoads + i) * 1024], value_from[i]);
    };
    Operand qs[W / 16];  // queries: an operand of 16 columns each
    {
        const auto* a = args();
        const int H = a->H, G = a->G, D = a->D, h = blockIdx.x % H;
        const Tile mine = tile_of(a->list, a->starts, a->T, blockIdx.x / H, G, kRows);
        const int first = __builtin_amdgcn_readfirstlane(mine.first), tile = __builtin_amdgcn_readfirstlane(mine.tile);
        len = __builtin_amdgcn_readfirstlane(mine.len);
        if (len == 0)
            return;
        const int64_t base = ((int64_t)first * a->ld + (int64_t)h * D) * 2;
        key_base = (uint64_t)a->k + base;
        value_base = (uint64_t)a->v + base;
        load_keys(0);
        load_values(0);
        load_keys(1);
        const int rows = len * G, row0 = tile * kRows + wave * 32;  // len * G <= T * Hq <= 2^30
        const int row = row0 + col < rows ? row0 + col : rows - 1;
        token = row / G;
        const int head = h * G + row - token * G;
        const uint16_t* from = a->q + ((int64_t)first + token) * a->q_ld + (int64_t)head * D;
#pragma unroll
        for (int i = 0; i < W / 16; i++) {
            const int d = i * 16 + half * 8;
            qs[i].w = d < D ? *(const u32x4*)(from + d) : u32x4{0, 0, 0, 0};
        }
        to = row0 + col < rows ? (first + token) * (H * G) + head : -1;
        const int end_row = (tile + 1) * kRows - 1;
        const int first_token = tile * kRows / G, last_token = (end_row < rows ? end_row : rows - 1) / G;
        tiles = last_token / kKeys + 1;
        whole = (first_token + 1) / kKeys;
        // a negative scale turns the signs; one of zero is zeros in the queries' place, as
        // 0 * -inf would not keep a key unseen
        if (scale < 0.f) {
#pragma unroll
            for (int i = 0; i < W / 16; i++)
                qs[i].w ^= 0x80008000u;
        } else if (scale == 0.f) {
#pragma unroll
            for (int i = 0; i < W / 16; i++)
                qs[i].w = times_zero(qs[i].w);
        }
    }

    floatx16 o[W / 32];
    float top, l;      // the score, unscaled, that m is made of
    float less, most;  // what scores add for m, and kMost, or -1 until m is a number
    floatx16 s[2];
    Operand p[4];
    // S^T of tile t
    auto scores = [&](int t) {
        const uint8_t* keys = key_lds[t & 1];
#pragma unroll
        for (int b = 0; b < 2; b++)
#pragma unroll
            for (int r = 0; r < 16; r++)
                s[b][r] = 0.f;
#pragma unroll
        for (int i = 0; i < W / 16; i++)
#pragma unroll
            for (int b = 0; b < 2; b++) {
                const bf16x8 a = *(const bf16x8*)(keys + key_at[i] + b * 32 * W * 2);
                s[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, qs[i].b, s[b], 0, 0, 0);
            }
    };
    // P of the scores and the lane's part of their sum
    auto relative = [&]() {
        float sum[2] = {0.f, 0.f};
#pragma unroll
        for (int b = 0; b < 2; b++)
#pragma unroll
            for (int r = 0; r < 16; r += 2) {
                float x[2];
#pragma unroll
                for (int e = 0; e < 2; e++) {
                    x[e] = __builtin_amdgcn_exp2f(fmaf(s[b][r + e], c, less));
                    sum[e] += x[e];
                }
                p[2 * b + r / 8].w[(r % 8) / 2] = pack2(x[0], x[1]);
            }
        return sum[0] + sum[1];
    };
    // the row's largest score, unscaled
    auto largest = [&]() {
        float most = s[0][0];
#pragma unroll
        for (int b = 0; b < 2; b++)
#pragma unroll
            for (int r = 0; r < 16; r++)
                most = fmaxf(most, s[b][r]);
        float x, y;
        swap32(most, &x, &y);
        return fmaxf(x, y);
    };
    // m = top c, rounded.  The product of scores and c is not: past kFar what m lacks is no small part of a
    // weight, and the row becomes NaN here, to be made again.
    auto set_m = [&](float now) {
        top = now;
        less = now == -INFINITY ? 0.f : fabsf(now * c) < kFar ? -(now * c) : __builtin_nanf("");
        most = now == -INFINITY ? -1.f : kMost;
    };
    // Keys of tile t that a row does not see have no part in its scores.
    auto mask = [&](int t) {
        const int seen = token - t * kKeys - 4 * half;
#pragma unroll
        for (int b = 0; b < 2; b++)
#pragma unroll
            for (int r = 0; r < 16; r++)
                s[b][r] = b * 32 + 8 * (r / 4) + r % 4 <= seen ? s[b][r] : -INFINITY;
    };
    // P of a tile's scores: m stays where it is, and the scores' maximum is not sought, unless
    // they turn out too large (sought in every tile: 16,384 rows 1.03 times as long).
    auto weights = [&]() {
        float sum = relative();
        const uint64_t over = __ballot(sum > most);
        if (over) {
            // only of such rows: what other rows of the wave hold changes no bit of a row
            const float high = largest(), now = (over >> col | over >> (col + 32)) & 1 ? fmaxf(top, high) : top;
            const float was = less, none = most;
            set_m(now);
            const float f = none < 0.f ? 0.f : exp2f(less - was);
#pragma unroll
            for (int i = 0; i < W / 32; i++)
#pragma unroll
                for (int r = 0; r < 16; r++)
                    o[i][r] *= f;
            l *= f;
            sum = relative();
        }
        l += sum;
    };
    // 16 keys j, columns 32 i .. 32 i + 31 of V^T
    auto value_part = [&](const uint8_t* values, int j, int i) {
        Operand a;
#pragma unroll
        for (int e = 0; e < 2; e++)
            a.h[e] = column_of(values + value_at[i] + (16 * j + 8 * e) * W * 2);
        return a;
    };
    // O^T += V^T P of tile t
    auto products = [&](int t, auto edge) {
        const uint8_t* values = value_lds[t & 1];
        bool odd = false;
        if (decltype(edge)::value) {
            // a value that is not finite must not reach rows that do not see it through a
            // product with zero: where the tile has one, it leaves the products and is
            // added to the rows that see it
            int any = 0;
#pragma unroll
            for (int i = 0; i < NW; i++)
                any |= odd_lds[t & 1][i];
            odd = __builtin_amdgcn_readfirstlane(any) != 0;
        }
        if (decltype(edge)::value && __builtin_expect(odd, 0)) {
#pragma unroll 1
            for (int key = 0; key < kKeys; key++)
#pragma unroll
                for (int i = 0; i < W / 32; i++)
#pragma unroll
                    for (int r = 0; r < 16; r += 4) {
                        const uint32_t* at = (const uint32_t*)(values + value_place<W>(key, 4 * i + r / 4) * 16 + 8 * half);
#pragma unroll
                        for (int e = 0; e < 4; e++) {
                            const uint32_t u = e & 1 ? at[e / 2] & 0xFFFF0000u : at[e / 2] << 16;
                            if ((u & 0x7F800000u) == 0x7F800000u && t * kKeys + key <= token)
                                o[i][r + e] += __uint_as_float(u);
                        }
                    }
#pragma unroll
            for (int j = 0; j < 4; j++)
#pragma unroll
                for (int i = 0; i < W / 32; i++) {
                    Operand a = value_part(values, j, i);
#pragma unroll
                    for (int e = 0; e < 4; e++) {
                        a.w[e] = (a.w[e] & 0x7F80u) == 0x7F80u ? a.w[e] & 0xFFFF0000u : a.w[e];
                        a.w[e] = (a.w[e] & 0x7F800000u) == 0x7F800000u ? a.w[e] & 0xFFFFu : a.w[e];
                    }
                    o[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.b, p[j].b, o[i], 0, 0, 0);
                }
        } else {
#pragma unroll
            for (int j = 0; j < 4; j++)
#pragma unroll
                for (int i = 0; i < W / 32; i++)
                    o[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(value_part(values, j, i).b, p[j].b, o[i], 0, 0, 0);
        }
    };

    // Products and scores beside each other: reads of LDS four matrix instructions ahead.
    auto pipeline = [&]() {
        constexpr int kEach = W / 8, kMatrix = 0x8, kRead = 0x100;  // matrix instructions of each; 2 reads and 1
        __builtin_amdgcn_sched_group_barrier(kRead, 8, 0);
#pragma unroll
        for (int i = 0; i < kEach - 4; i++) {
            __builtin_amdgcn_sched_group_barrier(kMatrix, 1, 0);
            __builtin_amdgcn_sched_group_barrier(kRead, 2, 0);
        }
#pragma unroll
        for (int i = 0; i < kEach; i++) {
            __builtin_amdgcn_sched_group_barrier(kMatrix, 1, 0);
            __builtin_amdgcn_sched_group_barrier(kRead, 1, 0);
        }
        __builtin_amdgcn_sched_group_barrier(kMatrix, 4, 0);
    };

    // Whether the wave's part of the values of tile t, which it loaded itself, is finite; asked
    // of tiles whose products are made at the edge.
    auto look = [&](int t) {
        u32x4 most = {0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < kLoads; i++) {
            const u32x4 w = *(const u32x4*)&value_lds[t & 1][((wave * kLoads + i) * 64 + lane) * 16];
#pragma unroll
            for (int e = 0; e < 4; e++)
                most[e] = max_u16(most[e], w[e] & 0x7FFF7FFFu);
        }
        const uint32_t m2 = max_u16(max_u16(most[0], most[1]), max_u16(most[2], most[3]));
        const bool odd = (m2 & 0xFFFFu) >= 0x7F80u || m2 >= 0x7F800000u;
        const int any = __ballot(odd) != 0;
        if (lane == 0)
            odd_lds[t & 1][wave] = any;
    };

    // Between two barriers a wave makes the products of tile t, then the scores and the
    // weights of tile t + 1.
    auto next = [&](int t) {
        __syncthreads();
        load_values(t + 1);
        load_keys(t + 2);
    };
    const std::false_type inner;
    const std::true_type edge;
#pragma unroll
    for (int i = 0; i < W / 32; i++)
#pragma unroll
        for (int r = 0; r < 16; r++)
            o[i][r] = 0.f;
    loads_done();
    if (whole == 0 || tiles == 1)
        look(0);
    __syncthreads();
    scores(0);
    if (whole == 0)
        mask(0);
    set_m(largest());
    l = relative();
    // products of tiles that every row sees, the scores of the next beside them
    int t = 0;
    for (; t < whole && t + 1 < tiles; t++) {
        loads_done();
        next(t);
        products(t, inner);
        scores(t + 1);
        pipeline();
        __builtin_amdgcn_sched_barrier(0);  // exponentials among the last products: 1 to 2% more
        if (t + 1 == whole)
            mask(whole);
        weights();
    }
    for (; t < tiles; t++) {
        loads_done();
        if (t > 0)
            look(t);
        next(t);
        products(t, edge);
        if (t + 1 < tiles) {
            scores(t + 1);
            mask(t + 1);
            weights();
        }
    }
    loads_done();  // none is in flight when the buffers go to another workgroup

    // what a second pass's weights are multiplied by: a power of two below half of one over the keys that the row
    // sees (not over all of its sequence: later keys change no bit of a row)
    const float small = __uint_as_float((uint32_t)(127 - 33 + __builtin_clz(token + 1)) << 23);
    // Writes the row; `again`: where what is there is not finite.  Whether anything written is not finite, but
    // for rows that a score of NaN makes NaN.
    auto store = [&](auto again) {
        float x, y;
        swap32(l, &x, &y);
        const float sum = x + y;
        const float inv = sum == 0.f ? 0.f : (decltype(again)::value ? 1.f / small : 1.f) / sum;  // scores of -inf alone give zeros
        const auto* a = args();
        if (to >= 0 && a->lse && half == 0) {
            // with the score itself, not with m: to the last place of what the score alone has
            const float lacks = decltype(again)::value ? 0.f : fmaf(top, c, less);
            const float lse = sum == 0.f ? -INFINITY
                                         : fmaf(top, fabsf(a->scale), (__builtin_amdgcn_logf(sum) - lacks) * kLn2);
            if (!decltype(again)::value || isnan(a->lse[to]))
                a->lse[to] = lse;
        }
        const int D = a->D;
        uint16_t* const out = a->out + (int64_t)to * D;
        uint32_t size = 0;
        // a lane has columns 8 j + 4 half .. + 3 of its row; halves trade so that it writes
        // eight in a row: the even j's or the odd ones
#pragma unroll
        for (int i = 0; i < W / 32; i++)
#pragma unroll
            for (int r = 0; r < 16; r += 8) {
                uint32_t w[4];
#pragma unroll
                for (int e = 0; e < 4; e++) {
                    float z[2];
#pragma unroll
                    for (int n = 0; n < 2; n++) {
                        const float u = o[i][r + 2 * e + n];
                        z[n] = u * inv;
                        // no mean is past all values, which a weight's rounding can bring it
                        if (decltype(again)::value && __builtin_isfinite(u))
                            z[n] = fminf(fmaxf(z[n], -kLargest), kLargest);
                    }
                    w[e] = pack2(z[0], z[1]);
                }
                const auto even = __builtin_amdgcn_permlane32_swap(w[0], w[2], false, false);
                const auto odd = __builtin_amdgcn_permlane32_swap(w[1], w[3], false, false);
                const int d = i * 32 + 2 * r + 8 * half;
                if (to < 0 || d >= D)
                    continue;
                u32x4 now = {even[0], odd[0], even[1], odd[1]};
                if (decltype(again)::value) {
                    const u32x4 was = *(const u32x4*)(out + d);
#pragma unroll
                    for (int e = 0; e < 4; e++) {
                        const uint32_t low = (was[e] & 0x7F80u) == 0x7F80u ? 0xFFFFu : 0u;
                        const uint32_t high = (was[e] & 0x7F800000u) == 0x7F800000u ? 0xFFFF0000u : 0u;
                        now[e] = (now[e] & (low | high)) | (was[e] & ~(low | high));
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 4; e++)
                        size = max_u16(size, now[e] & 0x7FFF7FFFu);
                }
                *(u32x4*)(out + d) = now;
            }
        return ((size & 0xFFFFu) >= 0x7F80u || size >= 0x7F800000u) &&
               !(isnan(sum) && (isnan(top) || !isnan(less)));
    };
    if (!__ballot(store(std::false_type())))
        return;

    // Results that are not finite are made again, with the largest score sought in every tile, unscaled, and
    // taken from the others before they are scaled: exact where it matters, whatever the scores.  Rare, so made
    // simply, by each wave that has some, from memory; what is finite stays as it was, so that a row's bits do
    // not depend on those beside it.
    const float by = scale == 0.f ? 1.f : fabsf(scale);
    const int D = args()->D;
#pragma unroll
    for (int i = 0; i < W / 32; i++)
#pragma unroll
        for (int r = 0; r < 16; r++)
            o[i][r] = 0.f;
    l = 0.f;
    top = -INFINITY;
#pragma unroll 1
    for (int t = 0; t < tiles; t++) {
#pragma unroll
        for (int b = 0; b < 2; b++) {
            const int key = t * kKeys + b * 32 + col;
            const uint16_t* from = (const uint16_t*)(key_base + (uint64_t)(key < len ? key : len - 1) * row_bytes);
#pragma unroll
            for (int r = 0; r < 16; r++)
                s[b][r] = 0.f;
#pragma unroll
            for (int i = 0; i < W / 16; i++) {
                Operand a;
                a.w = 16 * i + 8 * half < D ? *(const u32x4*)(from + 16 * i + 8 * half) : u32x4{0, 0, 0, 0};
                s[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.b, qs[i].b, s[b], 0, 0, 0);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        mask(t);
        __builtin_amdgcn_sched_barrier(0);
        const float now = fmaxf(top, largest()), most = now * by;
        // a score past binary32's range makes the row NaN, below it all weigh nothing
        const float base = most == INFINITY ? __builtin_nanf("") : most == -INFINITY ? INFINITY : now;
        const float f = top == now ? 1.f : __builtin_amdgcn_exp2f((top - now) * by * kLog2e);
#pragma unroll
        for (int i = 0; i < W / 32; i++)
#pragma unroll
            for (int r = 0; r < 16; r++)
                o[i][r] *= __builtin_isfinite(o[i][r]) ? f : 1.f;
        l *= f;
        top = now;
        uint32_t counts = 0;  // keys, in the order of s, of scores above -inf
#pragma unroll
        for (int b = 0; b < 2; b++)
#pragma unroll
            for (int r = 0; r < 16; r += 2) {
                float x[2];
#pragma unroll
                for (int e = 0; e < 2; e++) {
                    x[e] = __builtin_amdgcn_exp2f((s[b][r + e] - base) * by * kLog2e);
                    l += x[e];
                    counts |= (uint32_t)!(s[b][r + e] * by == -INFINITY) << (16 * b + r + e);
                }
                p[2 * b + r / 8].w[(r % 8) / 2] = pack2(x[0] * small, x[1] * small);
            }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < W / 32; i++) {
            // the lane's column of V^T; columns past D are not written, keys past the sequence do not count
            const uint64_t from = value_base + (32 * i + col < D ? 32 * i + col : 0) * 2;
            Operand values[2];  // of two j: more loads in flight at once take a wave from a SIMD at 64 columns
#pragma unroll
            for (int j = 0; j < 4; j++) {
                if (j % 2 == 0) {
                    int first_key = t * kKeys + 16 * j + 4 * half;
                    asm volatile("" : "+v"(first_key));  // addresses are made here, not held for every i
#pragma unroll
                    for (int e = 0; e < 8; e++) {
                        uint32_t u[2];
#pragma unroll
                        for (int z = 0; z < 2; z++) {
                            const int key = first_key + 8 * (e / 2) + 2 * (e % 2) + z;
                            u[z] = *(const uint16_t*)(from + (uint64_t)(key < len ? key : len - 1) * row_bytes);
                        }
                        values[e / 4].w[e % 4] = u[0] | u[1] << 16;
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
                Operand a = values[j % 2];
                uint32_t size = 0;
#pragma unroll
                for (int e = 0; e < 4; e++)
                    size = max_u16(size, a.w[e] & 0x7FFF7FFFu);
                asm volatile("" : "+v"(counts));  // nor what is made of this
                if (__ballot((size & 0xFFFFu) >= 0x7F80u || size >= 0x7F800000u)) {
                    // a value that is not finite counts wherever the score is above -inf, even if the weight is 0
                    // in binary32, so that tiles and the order of keys decide nothing: how many infinities of
                    // either sign do, NaN as both
                    Operand up, down, count;
#pragma unroll
                    for (int e = 0; e < 4; e++) {
                        up.w[e] = down.w[e] = count.w[e] = 0;
#pragma unroll
                        for (int z = 0; z < 2; z++) {
                            const uint32_t u = a.w[e] >> (16 * z) & 0xFFFFu, one = 0x3F80u << (16 * z);
                            const bool odd = (u & 0x7F80u) == 0x7F80u;
                            up.w[e] |= odd && u != 0xFF80u ? one : 0u;
                            down.w[e] |= odd && u != 0x7F80u ? one : 0u;
                            count.w[e] |= counts >> (8 * j + 2 * e + z) & 1 ? one : 0u;
                            a.w[e] &= odd ? ~(0xFFFFu << (16 * z)) : ~0u;
                        }
                    }
                    floatx16 n;
#pragma unroll
                    for (int r = 0; r < 16; r++)
                        n[r] = 0.f;
                    n = __builtin_amdgcn_mfma_f32_32x32x16_bf16(up.b, count.b, n, 0, 0, 0);
#pragma unroll
                    for (int r = 0; r < 16; r++) {
                        o[i][r] += n[r] > 0.f ? INFINITY : 0.f;
                        n[r] = 0.f;
                    }
                    n = __builtin_amdgcn_mfma_f32_32x32x16_bf16(down.b, count.b, n, 0, 0, 0);
#pragma unroll
                    for (int r = 0; r < 16; r++)
                        o[i][r] -= n[r] > 0.f ? INFINITY : 0.f;
                }
                o[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.b, p[j].b, o[i], 0, 0, 0);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
    }
    store(std::true_type());
}

// kWeighKeys keys a wave, NW waves; rows kWeighRows at a time from LDS (64 at a time, which
// lets three workgroups into a CU: 1.16 times as long, registers spill; with 128 all 256 are used at
// 128 columns and two spilled), 32 of them multiplied while the exponentials of the 32
// before are made.  Of the rows that count for a tile of keys the workgroup takes
// blockIdx.y's `chunk` tokens' and writes part blockIdx.y of the sum (a plane of n_heads x
// T), so that the first keys, which most rows see, do not take longest.
template <int W, int NW>
__global__ __launch_bounds__(NW * 64, 2) void prompt_weigh_kernel(
    const Tile* __restrict__ list, const int32_t* __restrict__ starts, int32_t T, const uint16_t* __restrict__ q,
    int64_t q_ld, int32_t G, const float* __restrict__ lse, const uint16_t* __restrict__ k, int64_t ld, int32_t H,
    int32_t D, int32_t last, int32_t chunk, float scale, float* __restrict__ weight)
{
    constexpr int kTile = kWeighRows * W * 2, kLoads = kTile / 1024 / NW, kBlock = kWeighKeys * NW;
    constexpr int kParts = kWeighRows / 32;
    static_assert(NW * 64 >= kWeighRows, "a thread brings a row's lse");
    __shared__ __align__(1024) uint8_t row_lds[2][kTile];
    __shared__ __align__(16) float less_lds[2][kWeighRows];
    __shared__ __align__(16) int token_lds[2][kWeighRows];  // -1: the row counts nowhere
    __shared__ int odd_lds[2][NW];  // whether the wave brought such a row or one past kFarLse (then + 2)
    const int lane = threadIdx.x & 63, col = lane & 31, half = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int h = blockIdx.x % H;
    const Tile mine = tile_of(list, starts, T, blockIdx.x / H, 1, kBlock);
    const int first = mine.first, len = mine.len;
    if (len == 0)
        return;
    const int key0 = ((len + kBlock - 1) / kBlock - 1 - mine.tile) * kBlock;  // the lowest keys, which most rows see, first
    const int all_from = len - last > key0 ? len - last : key0;  // the first token whose rows count here
    if ((int64_t)blockIdx.y * chunk >= len - all_from)
        return;
    const int seen_from = all_from + blockIdx.y * chunk;
    const int seen_to = len - seen_from < chunk ? len : seen_from + chunk;
    const int rows = (seen_to - seen_from) * G;  // len * G <= T * Hq <= 2^30
    const int turns = (rows + kWeighRows - 1) / kWeighRows;
    const float by = fabsf(scale), c = by * kLog2e;
    const uint32_t magic = 65536 / G + 1;  // x / G = x magic >> 16 for x < 64 + kWeighRows, G <= 64

    // A tile's rows are read from its first token's base: row x = rem + i is token x / G,
    // head x % G.  Rows past the last token's lie past the buffer's end.
    uint32_t from[kLoads];
    int from_rem = -1;
    float next_lse = 0.f;  // of row threadIdx.x, looked at once the tile is there: not to wait for it here
    int next_token = 0;
    // the tile's first token and its first row's place in it, from tile to tile
    int token0 = seen_from, rem = 0;
    const int more_tokens = kWeighRows / G, more_rem = kWeighRows - more_tokens * G;
    auto load = [&](int t) {
        const int here = rows - t * kWeighRows < kWeighRows ? rows - t * kWeighRows : kWeighRows;
        const int tokens = (int)((rem + here - 1) * magic >> 16);
        if (rem != from_rem) {
            from_rem = rem;
#pragma unroll
            for (int i = 0; i < kLoads; i++) {
                const int at = (wave * kLoads + i) * 64 + lane, r = at / (W / 8);
                const int qc = key_place<W>(r, at % (W / 8)) - r * (W / 8);
                const uint32_t x = rem + r, d = x * magic >> 16;
                from[i] = qc * 8 < D ? (uint32_t)(d * q_ld * 2) + (x - d * G) * D * 2 + qc * 16 : kOutside;
            }
        }
        const u32x4 r = rows_at((uint64_t)(q + ((int64_t)first + token0) * q_ld + (int64_t)h * G * D),
                                (uint32_t)(tokens * q_ld * 2 + G * D * 2));
#pragma unroll
        for (int i = 0; i < kLoads; i++)
            load_kib(r, &row_lds[t & 1][(wave * kLoads + i) * 1024], from[i]);
        if ((int)threadIdx.x < kWeighRows) {
            const uint32_t x = rem + threadIdx.x, d = x * magic >> 16;
            next_lse = -INFINITY;
            if ((int)threadIdx.x < here)
                next_lse = lse[((int64_t)first + token0 + d) * (H * G) + h * G + (x - d * G)];
            next_token = (int)(token0 + d);
        }
    };
    load(0);
    int first_token = seen_from;  // of the tile at work

    // the wave's keys: operands of 16 columns
    Operand ks[2][W / 16];
    const uint32_t turn = scale < 0.f ? 0x80008000u : 0u;
    int key[2];
#pragma unroll
    for (int b = 0; b < 2; b++) {
        key[b] = key0 + wave * kWeighKeys + b * 32 + col;
        const int at = key[b] < len ? key[b] : len - 1;
        const uint16_t* row = k + ((int64_t)first + at) * ld + (int64_t)h * D;
#pragma unroll
        for (int i = 0; i < W / 16; i++) {
            const int d = i * 16 + half * 8;
            ks[b][i].w = d < D ? *(const u32x4*)(row + d) : u32x4{0, 0, 0, 0};
            ks[b][i].w ^= turn;
        }
    }
    if (scale == 0.f) {
        // as in attention, so that a product past binary32's range does not become NaN
#pragma unroll
        for (int b = 0; b < 2; b++)
#pragma unroll
            for (int i = 0; i < W / 16; i++)
                ks[b][i].w = times_zero(ks[b][i].w);
    }
    int row_at[W / 16];
#pragma unroll
    for (int i = 0; i < W / 16; i++)
        row_at[i] = key_place<W>(col, 2 * i + half) * 16;

    // S of the tile's rows 32 a .. 32 a + 31
    typedef floatx16 Scores[2];
    auto scores = [&](int t, int a, Scores& s) {
#pragma unroll
        for (int b = 0; b < 2; b++)
#pragma unroll
            for (int r = 0; r < 16; r++)
                s[b][r] = 0.f;
#pragma unroll
        for (int i = 0; i < W / 16; i++) {
            const bf16x8 x = *(const bf16x8*)(row_lds[t & 1] + row_at[i] + a * 32 * W * 2);
#pragma unroll
            for (int b = 0; b < 2; b++)
                s[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, ks[b][i].b, s[b], 0, 0, 0);
        }
    };
    float total[2] = {0.f, 0.f}, part[2][2] = {};  // parts of 16 tiles, so that long sums lose little
    // edge: rows count for the keys that they see; far: by (S scale - lse) log2 e, whose product is exact
    // beside lse, so that weights are right wherever lse is
    auto add = [&](int t, int a, Scores& s, auto edge, auto far) __attribute__((always_inline)) {
#pragma unroll
        for (int r = 0; r < 16; r += 4) {
            const floatx4 less = *(const floatx4*)&less_lds[t & 1][a * 32 + 2 * r + 4 * half];
#pragma unroll
            for (int e = 0; e < 4; e++)
#pragma unroll
                for (int b = 0; b < 2; b++) {
                    float x = fmaf(s[b][r + e], decltype(far)::value ? by : c, less[e]);
                    x = __builtin_amdgcn_exp2f(decltype(far)::value ? x * kLog2e : x);
                    if (decltype(edge)::value)
                        x = key[b] <= token_lds[t & 1][a * 32 + 2 * r + 4 * half + e] ? x : 0.f;
                    part[b][e & 1] += x;
                }
        }
    };

    const int wave_key = key0 + wave * kWeighKeys + kWeighKeys - 1;  // the wave's last
    for (int t = 0; t < turns; t++) {
        loads_done();
        // rows past kFarLse, and all where c is past binary32's range, which the scale need not be
        const bool mine_too = (int)threadIdx.x < kWeighRows;
        float less = next_lse * -kLog2e;
        int odd = __ballot(mine_too && !(fabsf(next_lse) < kFarLse && c < INFINITY)) != 0;
        if (odd && __ballot(mine_too && !(fabsf(next_lse) < kFarLse && c < INFINITY) && next_lse != -INFINITY)) {
            odd = 3;
            less = -next_lse;  // of all the wave's rows
        }
        if (mine_too) {
            less_lds[t & 1][threadIdx.x] = less;
            token_lds[t & 1][threadIdx.x] = next_lse == -INFINITY ? -1 : next_token;
        }
        if (lane == 0)
            odd_lds[t & 1][wave] = odd;
        __syncthreads();
        const int least = first_token;
        if (t + 1 < turns) {
            token0 += more_tokens;
            rem += more_rem;
            if (rem >= G) {
                rem -= G;
                token0++;
            }
            first_token = token0;
            load(t + 1);
        }
        int any = 0;
#pragma unroll
        for (int i = 0; i < kWeighRows / 64; i++)
            any |= odd_lds[t & 1][i] << (2 * i);
        any = __builtin_amdgcn_readfirstlane(any);
        Scores s[2];
        const std::true_type yes;
        const std::false_type no;
        if (least < wave_key || any) {
#pragma unroll 1
            for (int a = 0; a < kParts; a++) {
                scores(t, a, s[0]);
                if (any >> (2 * (a / 2)) & 2)
                    add(t, a, s[0], yes, yes);
                else
                    add(t, a, s[0], yes, no);
            }
        } else {
            scores(t, 0, s[0]);
#pragma unroll
            for (int a = 0; a < kParts; a++) {
                if (a + 1 < kParts)
                    scores(t, a + 1, s[(a + 1) & 1]);
                add(t, a, s[a & 1], no, no);
            }
            // At 128 columns reads of LDS eight ahead, which leaves the exponentials where they
            // are beside products: 16 + 32 + 16 matrix instructions, 48 reads.  (Without: 8,192
            // rows 1.03 times as long; at 64 columns the compiler's own order is as fast.)
            constexpr int kMatrix = 0x8, kRead = 0x100;
            if (W == 128) {
                __builtin_amdgcn_sched_group_barrier(kRead, 8, 0);
#pragma unroll
                for (int i = 0; i < 8; i++) {
                    __builtin_amdgcn_sched_group_barrier(kMatrix, 2, 0);
                    __builtin_amdgcn_sched_group_barrier(kRead, 1, 0);
                }
#pragma unroll
                for (int i = 0; i < 16; i++) {
                    __builtin_amdgcn_sched_group_barrier(kMatrix, 2, 0);
                    __builtin_amdgcn_sched_group_barrier(kRead, 2, 0);
                }
                __builtin_amdgcn_sched_group_barrier(kMatrix, 16, 0);
            }
        }
        if ((t & 15) == 15) {
#pragma unroll
            for (int b = 0; b < 2; b++) {
                total[b] += part[b][0] + part[b][1];
                part[b][0] = part[b][1] = 0.f;
            }
        }
    }
#pragma unroll
    for (int b = 0; b < 2; b++) {
        float x, y;
        swap32(total[b] + (part[b][0] + part[b][1]), &x, &y);
        if (half == 0 && key[b] < len)
            weight[((int64_t)blockIdx.y * H + h) * T + first + key[b]] = x + y;
    }
}

// The parts of every position's weight, added in order.
__global__ __launch_bounds__(256) void prompt_weigh_join_kernel(const int32_t* __restrict__ starts, int32_t B, int32_t T,
                                                                int32_t H, int32_t last, int32_t chunk,
                                                                const float* __restrict__ parts,
                                                                float* __restrict__ weight, int32_t block)
{
    const int s = blockIdx.y, first = seq_first(starts, T, s), len = seq_end(starts, T, s) - first;
    const int64_t plane = (int64_t)H * T;
    for (int64_t i = blockIdx.x * 256ll + threadIdx.x; i < (int64_t)len * H; i += gridDim.x * 256ll) {
        const int h = (int)(i / len), j = (int)(i - (int64_t)h * len), key0 = j / block * block;
        const int from = len - last > key0 ? len - last : key0, n = (len - from + chunk - 1) / chunk;
        const int64_t at = (int64_t)h * T + first + j;
        float x = parts[at];
        for (int p = 1; p < n; p++)
            x += parts[p * plane + at];
        weight[at] = x;
    }
}

// Tiles of `rows` rows that sequences of T rows in all, times `per`, have at most.
int64_t most_tiles(int64_t T, int32_t per, int32_t rows, int32_t B) { return T * per / rows + B; }

// Fills the list of a call's tiles, where it takes one.
const Tile* make_list(const int32_t* starts, int32_t B, int32_t T, int32_t per, int32_t rows, void* workspace,
                      hipStream_t stream)
{
    if (B == 1)
        return nullptr;
    hipLaunchKernelGGL(prompt_list_kernel, dim3(kListWaves / 4), dim3(256), 0, stream, starts, B, T, per, rows,
                       (Tile*)workspace, (int32_t)most_tiles(T, per, rows, B));
    return (const Tile*)workspace;
}

constexpr int kWeighBlock = kWeighKeys * 4;
// Workgroups that leave no CU idle long, whatever their shares (4,096: 8,192 rows 1.05 times as
// long, 65,536 rows of one head 0.97 times).
constexpr int64_t kWeighWork = 2048;

// Chunks that the rows of a call are cut into, and their tokens.
int32_t weigh_chunks(int32_t B, int32_t T, int32_t G, int32_t H, int32_t last, int32_t* chunk)
{
    const int64_t n = kWeighWork / (most_tiles(T, 1, kWeighBlock, B) * H);
    // eight tiles of rows to a chunk, but one where there is little to do
    const int32_t most = last < T ? last : T, least = ((n > 4 ? 1 : 8) * kWeighRows + G - 1) / G;
    const int64_t want = n < 1 ? most : (most + n - 1) / n;
    *chunk = (int32_t)(want < least ? least : want);
    return (most + *chunk - 1) / *chunk;
}

// A list's bytes: 256 without one, more with one.
size_t list_bytes(int32_t B, int64_t tiles)
{
    return B == 1 ? 256 : 256 + (size_t)(tiles * sizeof(Tile) + 255) / 256 * 256;
}

// Waves of a workgroup of attention: two where four would leave CUs without one, 256 of 128 rows.
int attend_waves(int64_t T, int32_t Hq) { return T * Hq >= 128 * 256 ? 4 : 2; }

}  // namespace

size_t prompt_attend_workspace_bytes(int32_t B, int32_t T, int32_t Hq, int32_t H)
{
    return list_bytes(B, most_tiles(T, Hq / H, 32 * attend_waves(T, Hq), B));
}

size_t prompt_weigh_workspace_bytes(int32_t B, int32_t T, int32_t Hq, int32_t H, int32_t last)
{
    int32_t chunk;
    const int32_t chunks = weigh_chunks(B, T, Hq / H, H, last, &chunk);
    return list_bytes(B, most_tiles(T, 1, kWeighBlock, B)) + (chunks > 1 ? (size_t)chunks * H * T * 4 : 0);
}

hipError_t launch_prompt_attend(const int32_t* starts, int32_t B, int32_t T, const void* q, int64_t q_ld, int32_t Hq,
                                const void* k, const void* v, int64_t ld, int32_t H, int32_t D, float scale,
                                void* workspace, void* out, float* lse, hipStream_t stream)
{
    const int32_t G = Hq / H, waves = attend_waves(T, Hq);
    const Tile* list = make_list(starts, B, T, G, 32 * waves, workspace, stream);
    const Attend a = {list, starts, (const uint16_t*)q, (const uint16_t*)k, (const uint16_t*)v, q_ld, ld,
                      (uint16_t*)out, lse, T, G, H, D, scale};
    const dim3 grid((uint32_t)(most_tiles(T, G, 32 * waves, B) * H));
#define OIL_PROMPT_ATTEND(W, NW) \
    hipLaunchKernelGGL((prompt_attend_kernel<W, NW>), grid, dim3(NW * 64), 0, stream, a)
    if (D <= 64 && waves == 4)
        OIL_PROMPT_ATTEND(64, 4);
    else if (D <= 64)
        OIL_PROMPT_ATTEND(64, 2);
    else if (waves == 4)
        OIL_PROMPT_ATTEND(128, 4);
    else
        OIL_PROMPT_ATTEND(128, 2);
#undef OIL_PROMPT_ATTEND
    return hipGetLastError();
}

hipError_t launch_prompt_weigh(const int32_t* starts, int32_t B, int32_t T, const void* q, int64_t q_ld, int32_t Hq,
                               const float* lse, const void* k, int64_t ld, int32_t H, int32_t D, int32_t last,
                               float scale, void* workspace, float* weight, hipStream_t stream)
{
    const int32_t G = Hq / H;
    int32_t chunk;
    const int32_t chunks = weigh_chunks(B, T, G, H, last, &chunk);
    const int64_t tiles = most_tiles(T, 1, kWeighBlock, B);
    const Tile* list = make_list(starts, B, T, 1, kWeighBlock, workspace, stream);
    float* parts = chunks > 1 ? (float*)((uint8_t*)workspace + list_bytes(B, tiles)) : weight;
#define OIL_PROMPT_WEIGH(W)                                                                                         \
    hipLaunchKernelGGL((prompt_weigh_kernel<W, kWeighBlock / kWeighKeys>), dim3((uint32_t)(tiles * H), chunks),    \
                       dim3(kWeighBlock), 0, stream, list, starts, T, (const uint16_t*)q, q_ld, G, lse,            \
                       (const uint16_t*)k, ld, H, D, last, chunk, scale, parts)
    if (D <= 64)
        OIL_PROMPT_WEIGH(64);
    else
        OIL_PROMPT_WEIGH(128);
#undef OIL_PROMPT_WEIGH
    if (chunks > 1) {
        const int64_t blocks = ((int64_t)T * H / B + 255) / 256;
        hipLaunchKernelGGL(prompt_weigh_join_kernel, dim3((uint32_t)(blocks < 1 ? 1 : blocks > 1024 ? 1024 : blocks), B),
                           dim3(256), 0, stream, starts, B, T, H, last, chunk, parts, weight, kWeighBlock);
    }
    return hipGetLastError();
}

}  // namespace oil
