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
// V's transposing reads give), O^T += V^T P.  m follows the largest score only when
// that passes it by 2^8: sums and outputs are then scaled; below, P is at most 2^8.
//
// weigh: a lane's column is a key, S = Q K^T, and the sums of exp2(S c - lse) stay in
// registers: no two workgroups add to one position, so the result does not depend on
// any order.
#include "common.hpp"
#include "internal.hpp"

namespace oil {

namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef float floatx2 __attribute__((ext_vector_type(2)));
typedef short shortx4 __attribute__((ext_vector_type(4)));

#define LDS_PTR(T, p) ((T __attribute__((address_space(3)))*)(p))

constexpr int kKeys = 64;       // keys of a tile
constexpr int kWeighKeys = 64;  // keys of a wave
constexpr int kMaxSeqs = 512;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr uint32_t kOutside = 0xF0000000u;  // a byte offset past every buffer's end: reads as zero

union Operand {
    u32x4 w;
    bf16x8 b;
    shortx4 h[2];
};

__device__ __forceinline__ uint32_t pack2(float a, float b)
{
    const floatx2 x = {a, b};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(x, bf16x2));
}

// A value beside its counterpart 32 lanes away.
__device__ __forceinline__ void swap32(float x, float* a, float* b)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    *a = __uint_as_float(r[0]);
    *b = __uint_as_float(r[1]);
}

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

// Workgroup `rank` of those that the sequences need, `per(length)` tiles each, the
// tiles of the largest number first (the heaviest: theirs is the longest pass).  A
// wave as a whole finds it: N(t) = sum of max(0, tiles - t) counts the tiles numbered
// t and up.  False past the last one.
template <typename F>
__device__ __forceinline__ bool find_tile(const int32_t* starts, int32_t B, int32_t T, int rank, F per, int* seq,
                                          int* tile)
{
    if (B == 1) {
        const int n = per(seq_end(starts, T, 0) - seq_first(starts, T, 0));
        *seq = 0;
        *tile = n - 1 - rank;
        return rank < n;
    }
    const int lane = threadIdx.x & 63;
    int n[kMaxSeqs / 64], all = 0, most = 0;
#pragma unroll
    for (int i = 0; i < kMaxSeqs / 64; i++) {
        const int s = i * 64 + lane;
        n[i] = 0;
        if (i * 64 < B && s < B)
            n[i] = per(seq_end(starts, T, s) - seq_first(starts, T, s));
        all += n[i];
        most = n[i] > most ? n[i] : most;
    }
    if (rank >= wave_sum(all))
        return false;
    // N(low) > rank >= N(high), N(high) = 0 where every lane's most is at or below it
    int low = 0, high = 1, above = 0;
    auto count = [&](int t) {
        int c = 0;
#pragma unroll
        for (int i = 0; i < kMaxSeqs / 64; i++)
            if (i * 64 < B)
                c += n[i] > t ? n[i] - t : 0;
        return wave_sum(c);
    };
    while (true) {  // doubles until it passes: at most 31 turns, as tiles are below 2^30
        const int c = count(high);
        if (c <= rank) {
            above = c;
            break;
        }
        low = high;
        high *= 2;
    }
    while (high - low > 1) {
        const int mid = low + (high - low) / 2, c = count(mid);
        if (c > rank) {
            low = mid;
        } else {
            high = mid;
            above = c;
        }
    }
    int at = rank - above;  // among the sequences of more than `low` tiles
    *tile = low;
#pragma unroll
    for (int i = 0; i < kMaxSeqs / 64; i++) {
        if (i * 64 >= B)
            break;
        const uint64_t has = __ballot(n[i] > low);
        const int c = __popcll(has);
        if (at >= 0 && at < c) {
            const int before = __builtin_amdgcn_mbcnt_hi((uint32_t)(has >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)has, 0));
            const uint64_t mine = __ballot(n[i] > low && before == at);
            *seq = i * 64 + __builtin_ctzll(mine);
        }
        at -= c;
    }
    return true;
}

__device__ __forceinline__ __amdgpu_buffer_rsrc_t rows_at(const uint16_t* p, int64_t bytes)
{
    const uint64_t a = (uint64_t)p;
    const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)a), hi = __builtin_amdgcn_readfirstlane((uint32_t)(a >> 32));
    const int n = __builtin_amdgcn_readfirstlane((int)(uint32_t)bytes);
    return __builtin_amdgcn_make_buffer_rsrc((void*)((uint64_t)hi << 32 | lo), (short)0, n, 0x00020000);
}

// 16 bytes a lane, at byte `from` of the buffer (zeros past its end), straight to LDS:
// one KiB from `to` on, lane by lane.
__device__ __forceinline__ void load_kib(__amdgpu_buffer_rsrc_t r, uint8_t* to, uint32_t from)
{
    __builtin_amdgcn_raw_ptr_buffer_load_lds(r, LDS_PTR(void, to), 16, from, 0, 0, 0);
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

template <int W, int NW>
__global__ __launch_bounds__(NW * 64, 2) void prompt_attend_kernel(
    const int32_t* __restrict__ starts, int32_t B, int32_t T, const uint16_t* __restrict__ q, int64_t q_ld, int32_t G,
    const uint16_t* __restrict__ k, const uint16_t* __restrict__ v, int64_t ld, int32_t H, int32_t D, float scale,
    uint16_t* __restrict__ out, float* __restrict__ lse)
{
    constexpr int kTile = kKeys * W * 2;          // bytes
    constexpr int kLoads = kTile / 1024 / NW;     // 1 KiB loads of a wave, a side
    constexpr int kRows = 32 * NW;
    __shared__ __align__(1024) uint8_t key_lds[2][kTile];
    __shared__ __align__(1024) uint8_t value_lds[2][kTile];
    const int lane = threadIdx.x & 63, col = lane & 31, half = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int h = blockIdx.x % H;
    int seq, tile;
    if (!find_tile(starts, B, T, blockIdx.x / H, [&](int n) { return (int)(((int64_t)n * G + kRows - 1) / kRows); }, &seq,
                   &tile))
        return;
    const int first = seq_first(starts, T, seq), len = seq_end(starts, T, seq) - first;
    const int64_t rows = (int64_t)len * G, row0 = (int64_t)tile * kRows + wave * 32;
    const int64_t row = row0 + col < rows ? row0 + col : rows - 1;
    const int token = (int)(row / G), head = h * G + (int)(row % G);
    // tokens of the workgroup's last row, of the wave's first and last
    const int64_t end_row = (int64_t)(tile + 1) * kRows - 1;
    const int last_token = __builtin_amdgcn_readfirstlane((int)((end_row < rows ? end_row : rows - 1) / G));
    const int wave_first = __builtin_amdgcn_readfirstlane(token), wave_last = __builtin_amdgcn_readlane(token, 31);
    const int tiles = last_token / kKeys + 1, wave_tiles = row0 < rows ? wave_last / kKeys + 1 : 0;

    // loads: chunk `lane` of each KiB from where its place in LDS says
    uint32_t key_from[kLoads], value_from[kLoads];
#pragma unroll
    for (int i = 0; i < kLoads; i++) {
        const int at = (wave * kLoads + i) * 64 + lane, r = at / (W / 8);
        const int kc = key_place<W>(r, at % (W / 8)) - r * (W / 8), vc = value_place<W>(r, at % (W / 8)) - r * (W / 8);
        key_from[i] = kc * 8 < D ? (uint32_t)(r * ld * 2) + kc * 16 : kOutside;
        value_from[i] = vc * 8 < D ? (uint32_t)(r * ld * 2) + vc * 16 : kOutside;
    }
    const int64_t base = (int64_t)first * ld + (int64_t)h * D;
    auto load = [&](int t) {
        const int left = len - t * kKeys < kKeys ? len - t * kKeys : kKeys;
        const int64_t bytes = (left - 1) * ld * 2 + D * 2, at = base + (int64_t)t * kKeys * ld;
        const __amdgpu_buffer_rsrc_t kr = rows_at(k + at, bytes), vr = rows_at(v + at, bytes);
#pragma unroll
        for (int i = 0; i < kLoads; i++)
            load_kib(kr, &key_lds[t & 1][(wave * kLoads + i) * 1024], key_from[i]);
#pragma unroll
        for (int i = 0; i < kLoads; i++)
            load_kib(vr, &value_lds[t & 1][(wave * kLoads + i) * 1024], value_from[i]);
    };
    load(0);

    // queries: an operand of 16 columns each.  A negative scale turns their signs; one of
    // zero is zeros in their place, as 0 * -inf would not keep a key unseen.
    const float c = scale == 0.f ? 1.f : fabsf(scale) * kLog2e;
    Operand qs[W / 16];
    {
        const uint16_t* from = q + ((int64_t)first + token) * q_ld + (int64_t)head * D;
        const uint32_t turn = scale < 0.f ? 0x80008000u : 0u;
#pragma unroll
        for (int i = 0; i < W / 16; i++) {
            const int d = i * 16 + half * 8;
            qs[i].w = d < D ? *(const u32x4*)(from + d) : u32x4{0, 0, 0, 0};
            qs[i].w ^= turn;
            if (scale == 0.f)
#pragma unroll
                for (int e = 0; e < 4; e++) {
                    const uint32_t w = qs[i].w[e];
                    qs[i].w[e] = ((w & 0x7F80u) == 0x7F80u ? 0x7FC0u : 0u) |
                                 ((w & 0x7F800000u) == 0x7F800000u ? 0x7FC00000u : 0u);
                }
        }
    }
    int key_at[W / 16], value_at[W / 32];
#pragma unroll
    for (int i = 0; i < W / 16; i++)
        key_at[i] = key_place<W>(col, 2 * i + half) * 16;
#pragma unroll
    for (int i = 0; i < W / 32; i++)
        value_at[i] = value_place<W>(4 * half + (lane & 15) / 4, i * 4 + 2 * (col >> 4) + ((lane & 3) >> 1)) * 16 +
                      (lane & 1) * 8;

    floatx16 o[W / 32];
#pragma unroll
    for (int i = 0; i < W / 32; i++)
#pragma unroll
        for (int r = 0; r < 16; r++)
            o[i][r] = 0.f;
    float m = -INFINITY, l = 0.f;

    for (int t = 0; t < tiles; t++) {
        loads_done();
        __syncthreads();
        if (t + 1 < tiles)
            load(t + 1);
        if (t >= wave_tiles)
            continue;
        const uint8_t* keys = key_lds[t & 1];
        const uint8_t* values = value_lds[t & 1];
        floatx16 s[2];
#pragma unroll
        for (int b = 0; b < 2; b++) {
#pragma unroll
            for (int r = 0; r < 16; r++)
                s[b][r] = 0.f;
#pragma unroll
            for (int i = 0; i < W / 16; i++) {
                const bf16x8 a = *(const bf16x8*)(keys + key_at[i] + b * 32 * W * 2);
                s[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, qs[i].b, s[b], 0, 0, 0);
            }
        }
        const bool edge = t * kKeys + kKeys - 1 > wave_first;  // some row does not see some key
        if (edge) {
            const int seen = token - t * kKeys - 4 * half;
#pragma unroll
            for (int b = 0; b < 2; b++)
#pragma unroll
                for (int r = 0; r < 16; r++)
                    s[b][r] = b * 32 + 8 * (r / 4) + r % 4 <= seen ? s[b][r] : -INFINITY;
        }
        float top = s[0][0];
#pragma unroll
        for (int b = 0; b < 2; b++)
#pragma unroll
            for (int r = 0; r < 16; r++)
                top = fmaxf(top, s[b][r]);
        float x, y;
        swap32(top, &x, &y);
        top = fmaxf(x, y) * c;
        if (__ballot(top > m + 8.f)) {
            const float now = fmaxf(m, top), f = exp2f(m - (now == -INFINITY ? 0.f : now));
#pragma unroll
            for (int i = 0; i < W / 32; i++)
#pragma unroll
                for (int r = 0; r < 16; r++)
                    o[i][r] *= f;
            l *= f;
            m = now;
        }
        const float less = m == -INFINITY ? 0.f : -m;
        Operand p[4];
        float sum[2] = {0.f, 0.f};
#pragma unroll
        for (int b = 0; b < 2; b++) {
#pragma unroll
            for (int r = 0; r < 16; r++) {
                s[b][r] = __builtin_amdgcn_exp2f(fmaf(s[b][r], c, less));
                sum[r & 1] += s[b][r];
            }
#pragma unroll
            for (int r = 0; r < 16; r += 2)
                p[2 * b + r / 8].w[(r % 8) / 2] = pack2(s[b][r], s[b][r + 1]);
        }
        l += sum[0] + sum[1];
        if (edge) {
            // a value that is not finite must not reach rows that do not see it through a
            // product with zero: such values leave the products, and how many of each sign
            // a row sees is counted by products of ones
            uint32_t odd = 0;
#pragma unroll
            for (int j = 0; j < 4; j++)
#pragma unroll
                for (int i = 0; i < W / 32; i++) {
                    const u32x4 w = *(const u32x4*)(values + ((j * W / 32 + i) * 64 + lane) * 16);
#pragma unroll
                    for (int e = 0; e < 4; e++)
                        odd |= (w[e] & 0x7F80u) == 0x7F80u || (w[e] & 0x7F800000u) == 0x7F800000u;
                }
            if (__builtin_expect(__ballot(odd) != 0, 0)) {
                const int seen = token - t * kKeys - 4 * half;
#pragma unroll
                for (int i = 0; i < W / 32; i++) {
                    floatx16 up, down;
#pragma unroll
                    for (int r = 0; r < 16; r++)
                        up[r] = down[r] = 0.f;
#pragma unroll
                    for (int j = 0; j < 4; j++) {
                        Operand a, plus, minus, sees;
#pragma unroll
                        for (int e = 0; e < 2; e++)
                            a.h[e] = column_of(values + value_at[i] + (16 * j + 8 * e) * W * 2);
#pragma unroll
                        for (int e = 0; e < 4; e++) {
                            uint32_t pl = 0, mi = 0, se = 0;
#pragma unroll
                            for (int g = 0; g < 2; g++) {
                                const uint32_t u = (a.w[e] >> (16 * g)) & 0xFFFFu;
                                const bool wild = (u & 0x7F80u) == 0x7F80u, nan = wild && (u & 0x7Fu);
                                pl |= (wild && (nan || !(u >> 15)) ? 0x3F80u : 0u) << (16 * g);
                                mi |= (wild && (nan || (u >> 15)) ? 0x3F80u : 0u) << (16 * g);
                                if (wild)
                                    a.w[e] &= ~(0xFFFFu << (16 * g));
                                const int key = 16 * j + 8 * (e / 2) + 2 * (e % 2) + g;
                                se |= (key <= seen ? 0x3F80u : 0u) << (16 * g);
                            }
                            plus.w[e] = pl;
                            minus.w[e] = mi;
                            sees.w[e] = se;
                        }
                        o[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.b, p[j].b, o[i], 0, 0, 0);
                        up = __builtin_amdgcn_mfma_f32_32x32x16_bf16(plus.b, sees.b, up, 0, 0, 0);
                        down = __builtin_amdgcn_mfma_f32_32x32x16_bf16(minus.b, sees.b, down, 0, 0, 0);
                    }
#pragma unroll
                    for (int r = 0; r < 16; r++) {
                        o[i][r] += up[r] > 0.f ? INFINITY : 0.f;
                        o[i][r] -= down[r] > 0.f ? INFINITY : 0.f;
                    }
                }
                continue;
            }
        }
#pragma unroll
        for (int j = 0; j < 4; j++)
#pragma unroll
            for (int i = 0; i < W / 32; i++) {
                Operand a;
#pragma unroll
                for (int e = 0; e < 2; e++)
                    a.h[e] = column_of(values + value_at[i] + (16 * j + 8 * e) * W * 2);
                o[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.b, p[j].b, o[i], 0, 0, 0);
            }
    }

    if (row0 + col >= rows)
        return;
    float x, y;
    swap32(l, &x, &y);
    l = x + y;
    const float inv = l == 0.f ? 0.f : 1.f / l;  // scores of -inf alone give zeros
    const int64_t at = ((int64_t)first + token) * (H * G) + head;
    if (lse && half == 0)
        lse[at] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * kLn2;
#pragma unroll
    for (int i = 0; i < W / 32; i++)
#pragma unroll
        for (int r = 0; r < 16; r += 4) {
            const int d = i * 32 + 2 * r + 4 * half;
            if (d < D) {
                typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
                *(u32x2*)(out + at * D + d) = u32x2{pack2(o[i][r] * inv, o[i][r + 1] * inv),
                                                   pack2(o[i][r + 2] * inv, o[i][r + 3] * inv)};
            }
        }
}

// kWeighKeys keys a wave, NW waves; rows 64 at a time from LDS.
template <int W, int NW>
__global__ __launch_bounds__(NW * 64, 2) void prompt_weigh_kernel(
    const int32_t* __restrict__ starts, int32_t B, int32_t T, const uint16_t* __restrict__ q, int64_t q_ld, int32_t G,
    const float* __restrict__ lse, const uint16_t* __restrict__ k, int64_t ld, int32_t H, int32_t D, int32_t last,
    float scale, float* __restrict__ weight)
{
    constexpr int kRowTile = 64, kTile = kRowTile * W * 2, kLoads = kTile / 1024 / NW, kBlock = kWeighKeys * NW;
    __shared__ __align__(1024) uint8_t row_lds[2][kTile];
    __shared__ __align__(16) float less_lds[2][kRowTile];
    __shared__ __align__(16) int token_lds[2][kRowTile];  // -1: the row counts nowhere
    __shared__ int none_lds[2];                           // whether the tile has such a row
    const int lane = threadIdx.x & 63, col = lane & 31, half = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int h = blockIdx.x % H;
    auto per = [&](int n) { return (n + kBlock - 1) / kBlock; };
    int seq, tile;
    if (!find_tile(starts, B, T, blockIdx.x / H, per, &seq, &tile))
        return;
    const int first = seq_first(starts, T, seq), len = seq_end(starts, T, seq) - first;
    const int key0 = (per(len) - 1 - tile) * kBlock;  // the lowest keys, which most rows see, first
    const int seen_from = len - last > key0 ? len - last : key0;  // the first token whose rows count here
    const int64_t row_begin = (int64_t)seen_from * G, rows = (int64_t)len * G - row_begin;
    const int turns = (int)((rows + kRowTile - 1) / kRowTile);
    const float c = fabsf(scale) * kLog2e;
    const uint32_t magic = 65536 / G + 1;  // x / G = x magic >> 16 for x < 128, G <= 64

    // rows: token seen_from + x / G, head x % G; a tile's are at its first token's base
    uint32_t chunk_from[kLoads];
    int row_of[kLoads];
#pragma unroll
    for (int i = 0; i < kLoads; i++) {
        const int at = (wave * kLoads + i) * 64 + lane, r = at / (W / 8);
        const int qc = key_place<W>(r, at % (W / 8)) - r * (W / 8);
        row_of[i] = r;
        chunk_from[i] = qc * 8 < D ? qc * 16 : kOutside;
    }
    float next_less = 0.f;
    int next_token = 0;
    auto load = [&](int t) {
        const int64_t row0 = row_begin + (int64_t)t * kRowTile;
        const int token0 = (int)(row0 / G), rem = (int)(row0 % G);
        const int here = rows - (int64_t)t * kRowTile < kRowTile ? (int)(rows - (int64_t)t * kRowTile) : kRowTile;
        const int tokens = ((rem + here - 1) / G);
        const __amdgpu_buffer_rsrc_t r = rows_at(q + ((int64_t)first + token0) * q_ld + (int64_t)h * G * D,
                                                 tokens * q_ld * 2 + (int64_t)G * D * 2);
#pragma unroll
        for (int i = 0; i < kLoads; i++) {
            const uint32_t x = rem + row_of[i], d = x * magic >> 16;
            const uint32_t from = row_of[i] < here && chunk_from[i] != kOutside
                                      ? (uint32_t)(d * q_ld * 2) + (x - d * G) * D * 2 + chunk_from[i]
                                      : kOutside;
            load_kib(r, &row_lds[t & 1][(wave * kLoads + i) * 1024], from);
        }
        if (wave == 0) {
            const uint32_t x = rem + lane, d = x * magic >> 16;
            float y = -INFINITY;
            if (lane < here)
                y = lse[((int64_t)first + token0 + d) * (H * G) + h * G + (x - d * G)];
            next_less = y * kLog2e;
            next_token = y == -INFINITY ? -1 : (int)(token0 + d);
        }
    };
    load(0);

    // the wave's keys: operands of 16 columns
    Operand ks[2][W / 16];
    const uint32_t turn = scale < 0.f ? 0x80008000u : 0u;
    int key[2];
#pragma unroll
    for (int b = 0; b < 2; b++) {
        key[b] = key0 + wave * kWeighKeys + b * 32 + col;
        const int at = key[b] < len ? key[b] : len - 1;
        const uint16_t* from = k + ((int64_t)first + at) * ld + (int64_t)h * D;
#pragma unroll
        for (int i = 0; i < W / 16; i++) {
            const int d = i * 16 + half * 8;
            ks[b][i].w = d < D ? *(const u32x4*)(from + d) : u32x4{0, 0, 0, 0};
            ks[b][i].w ^= turn;
        }
    }
    int row_at[W / 16];
#pragma unroll
    for (int i = 0; i < W / 16; i++)
        row_at[i] = key_place<W>(col, 2 * i + half) * 16;

    const int wave_key = key0 + wave * kWeighKeys + kWeighKeys - 1;  // the wave's last
    float total[2] = {0.f, 0.f}, part[2] = {0.f, 0.f};  // parts of 32 tiles, so that long sums lose little
    for (int t = 0; t < turns; t++) {
        loads_done();
        if (wave == 0) {
            less_lds[t & 1][lane] = next_less;
            token_lds[t & 1][lane] = next_token;
            const bool none = __ballot(next_token < 0) != 0;
            if (lane == 0)
                none_lds[t & 1] = none;
        }
        __syncthreads();
        if (t + 1 < turns)
            load(t + 1);
        const int token0 = (int)((row_begin + (int64_t)t * kRowTile) / G);
        const bool edge = token0 < wave_key || none_lds[t & 1];
#pragma unroll
        for (int a = 0; a < 2; a++) {
            floatx16 s[2];
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
#pragma unroll
            for (int r = 0; r < 16; r += 4) {
                const floatx4 less = *(const floatx4*)&less_lds[t & 1][a * 32 + 2 * r + 4 * half];
#pragma unroll
                for (int b = 0; b < 2; b++)
#pragma unroll
                    for (int e = 0; e < 4; e++)
                        s[b][r + e] = __builtin_amdgcn_exp2f(fmaf(s[b][r + e], c, -less[e]));
            }
            if (edge) {
#pragma unroll
                for (int r = 0; r < 16; r++) {
                    const int token = token_lds[t & 1][a * 32 + 8 * (r / 4) + 4 * half + r % 4];
#pragma unroll
                    for (int b = 0; b < 2; b++)
                        s[b][r] = key[b] <= token ? s[b][r] : 0.f;
                }
            }
#pragma unroll
            for (int b = 0; b < 2; b++) {
                float two[2] = {0.f, 0.f};
#pragma unroll
                for (int r = 0; r < 16; r++)
                    two[r & 1] += s[b][r];
                part[b] += two[0] + two[1];
            }
        }
        if ((t & 31) == 31) {
#pragma unroll
            for (int b = 0; b < 2; b++) {
                total[b] += part[b];
                part[b] = 0.f;
            }
        }
    }
#pragma unroll
    for (int b = 0; b < 2; b++) {
        float x, y;
        swap32(total[b] + part[b], &x, &y);
        if (half == 0 && key[b] < len)
            weight[(int64_t)h * T + first + key[b]] = x + y;
    }
}

// Workgroups that sequences of T rows in all, times G, need at most, at `per` rows each.
int64_t most_tiles(int64_t rows, int64_t per, int32_t B) { return rows / per + B; }

}  // namespace

hipError_t launch_prompt_attend(const int32_t* starts, int32_t B, int32_t T, const void* q, int64_t q_ld, int32_t Hq,
                                const void* k, const void* v, int64_t ld, int32_t H, int32_t D, float scale, void* out,
                                float* lse, hipStream_t stream)
{
    const int32_t G = Hq / H;
#define OIL_PROMPT_ATTEND(W, NW)                                                                                   \
    hipLaunchKernelGGL((prompt_attend_kernel<W, NW>),                                                              \
                       dim3((uint32_t)(most_tiles((int64_t)T * G, 32 * NW, B) * H)), dim3(NW * 64), 0, stream, starts, \
                       B, T, (const uint16_t*)q, q_ld, G, (const uint16_t*)k, (const uint16_t*)v, ld, H, D, scale, \
                       (uint16_t*)out, lse)
    const bool wide = (int64_t)T * Hq >= 256 * 512;
    if (D <= 64 && wide)
        OIL_PROMPT_ATTEND(64, 8);
    else if (D <= 64)
        OIL_PROMPT_ATTEND(64, 2);
    else if (wide)
        OIL_PROMPT_ATTEND(128, 8);
    else
        OIL_PROMPT_ATTEND(128, 2);
#undef OIL_PROMPT_ATTEND
    return hipGetLastError();
}

hipError_t launch_prompt_weigh(const int32_t* starts, int32_t B, int32_t T, const void* q, int64_t q_ld, int32_t Hq,
                               const float* lse, const void* k, int64_t ld, int32_t H, int32_t D, int32_t last,
                               float scale, float* weight, hipStream_t stream)
{
    const int32_t G = Hq / H;
#define OIL_PROMPT_WEIGH(W, NW)                                                                                   \
    hipLaunchKernelGGL((prompt_weigh_kernel<W, NW>), dim3((uint32_t)(most_tiles(T, kWeighKeys * NW, B) * H)),     \
                       dim3(NW * 64), 0, stream, starts, B, T, (const uint16_t*)q, q_ld, G, lse, (const uint16_t*)k, \
                       ld, H, D, last, scale, weight)
    if (D <= 64)
        OIL_PROMPT_WEIGH(64, 4);
    else
        OIL_PROMPT_WEIGH(128, 4);
#undef OIL_PROMPT_WEIGH
    return hipGetLastError();
}

}  // namespace oil
