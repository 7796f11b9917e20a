// The verifier's 4-bit key/value cache: clearing, appending (quantising),
// reading back and eviction.  Layout and contract: include/oilbird.h; the
// attention that reads it: kvattend.hip.
//
// append: one workgroup per touched 32-position tile of a (request, head).  A
// row is quantised by 8 lanes: extremes by shuffles, s = bf16 at or above (max -
// min) / 15, z = bf16 at or below min, c = round((x - z) / s).  The tile's codes
// are put together in LDS as they are stored and leave 16 bytes a lane; where the
// tile also holds earlier positions, a value dword (8 positions of a column) is
// read and merged.  The workgroup owns the tile, so there is no race on a dword.
// Bound by memory and by the VALU (18 instructions a value, 0.8 of its issue) alike:
// 4 prompts of 8,191 rows, 8 heads of 128 columns in bf16: 136 MB in and 38 MB out in
// 45 us, 3.9 TB/s, from memory, 37 from the last-level cache; in binary32 64 us (306
// MB, 4.8 TB/s); 16 requests of 4,097 rows 69 us (5.0 TB/s; a copy reaches 4.9).  Small
// appends by their latencies, 6 us; the committed paths of 32 trees 8 us.
//
// read: a tile's codes to LDS, y = z + s c, 16 bytes a lane; the same rows in 27 us
// (36 MB in, 134 MB out, 6.4 TB/s).
//
// evict: a row kept above the budget moves into a hole below it, so sources
// and destinations are disjoint and every move is independent.  One workgroup
// per (request, head) finds the budget-th largest weight by radix selection
// and lists the moves with their positions and weights; a second kernel owns
// one destination tile per workgroup.  16 requests of 8 heads, 20,481 rows to
// 16,384: 44 us to select (128 workgroups for 256 CUs: a head's three passes over
// LDS, one after the other, are the time) and 129 to move (a nibble of every dword of
// the values changes with a row, so nearly every tile below the budget is read and
// written: 430 MB in, 169 out, 4.6 TB/s; turn after turn fewer rows move, 106 us).
// A head's ranks fit LDS up to 36,864 rows.  Past that each pass reads weights and
// positions again (from the caches), through one workgroup a head still: of one
// request, 8 heads, 36,864 rows take 62 us, 40,960 118, 147,456 411, 393,216 1,200.
//
// A slot's length changes when the last workgroup of the request has read it:
// each takes a ticket when it is done, or, where they are many, by a launch of its
// own.
#include "kv.hpp"

namespace oil {

namespace {

constexpr int64_t kMaxGridTiles = 16384;  // workgroups a (request, head); past that they take turns

__global__ __launch_bounds__(256) void kv_clear_kernel(KvView c)
{
    const int64_t n = (int64_t)c.n_slots * c.H * c.cap;
    for (int64_t i = blockIdx.x * 256ll + threadIdx.x; i < n; i += gridDim.x * 256ll) {
        c.pos[i] = -1;
        c.weight[i] = 0.f;
    }
    if (blockIdx.x == 0)
        for (int64_t i = threadIdx.x; i < 4ll * c.n_slots; i += 256)
            c.state[i] = 0;
}

// Workgroups of a request up to which the last one writes the slot's state
// (each takes a ticket, so it has read the state before): past that the tickets,
// one address over all XCDs, cost more than a launch of their own, 4 us.
constexpr int kTickets = 64;

// Whether this workgroup is the last of `total` of its request to be done; the
// ticket is left at zero then.  Nothing is published by it but the order of the
// state's reads and its write, so it needs no fence over the data.
__device__ __forceinline__ bool kv_last(const KvView& c, int slot, int total)
{
    __shared__ int last;
    __syncthreads();
    if (threadIdx.x == 0) {
        int32_t* ticket = c.state + 4 * (int64_t)slot + kKvTicket;
        last = __hip_atomic_fetch_add(ticket, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == total - 1;
        if (last)
            __hip_atomic_store(ticket, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    __syncthreads();
    return last;
}

__device__ __forceinline__ void kv_advance(const KvView& c, int slot, int32_t len, int cnt)
{
    int32_t* st = c.state + 4 * (int64_t)slot;
    const int64_t end = len + (int64_t)cnt, next = st[kKvNext] + (int64_t)cnt;
    st[kKvLen] = (int32_t)(end < c.cap ? end : c.cap);
    st[kKvNext] = next < INT32_MAX ? (int32_t)next : INT32_MAX;
}

// The state after an append (rows of max_rows, nodes, count) or, with max_rows
// 0, a reset; one workgroup per request.
__global__ __launch_bounds__(64) void kv_state_kernel(KvView c, const int32_t* __restrict__ slots, int32_t max_rows,
                                                      const int32_t* __restrict__ nodes,
                                                      const int32_t* __restrict__ count)
{
    __shared__ int bound;
    const int b = blockIdx.x, slot = kv_slot(c, slots, b);
    if (slot < 0)
        return;
    const int cnt = max_rows ? kv_count(nodes, count, b, max_rows, &bound) : 0;
    if (threadIdx.x != 0)
        return;
    if (max_rows)
        kv_advance(c, slot, kv_len(c, slot), cnt);
    else
        c.state[4 * (int64_t)slot + kKvLen] = c.state[4 * (int64_t)slot + kKvNext] = 0;
}

__global__ __launch_bounds__(256) void kv_reset_kernel(KvView c, const int32_t* __restrict__ slots)
{
    const int b = blockIdx.z, h = blockIdx.y;
    const int slot = kv_slot(c, slots, b);
    if (slot < 0)
        return;
    const int32_t n = kv_len(c, slot);
    const int64_t row = kv_row(c, slot, h);
    for (int64_t i = blockIdx.x * 256ll + threadIdx.x; i < n; i += gridDim.x * 256ll) {
        c.pos[row + i] = -1;
        c.weight[row + i] = 0.f;
    }
    if (gridDim.x * gridDim.y <= kTickets && kv_last(c, slot, gridDim.x * gridDim.y) && threadIdx.x == 0)
        c.state[4 * (int64_t)slot + kKvLen] = c.state[4 * (int64_t)slot + kKvNext] = 0;
}

// x / s to the nearest, as the binary32 division has it, for an s of 8 significant
// bits and inv within a few units of 1 / s: x * inv is within a few units, its
// remainder exact (a small multiple of the last places of s and q), and the sum
// corrected by it is off by less than 2^-20 of a unit before it is rounded, while a
// quotient by 8 bits lies at least 1 / 512 of a unit from where rounding turns.
__device__ __forceinline__ float kv_quotient(float x, float s, float inv)
{
    const float q = x * inv;
    return fmaf(fmaf(-s, q, x), inv, q);
}

// The least s that codes are made with this way: no remainder that matters
// underflows.
constexpr float kLeastScale = 0x1p-90f;

// (s, z) of a row with extremes lo, hi; `fine`: every value is finite.
__device__ __forceinline__ uint32_t kv_pair(float lo, float hi, bool fine)
{
    const uint32_t u = __float_as_uint(lo);
    const uint32_t z = (u >> 31 ? u + 0xFFFFu : u) & 0xFFFF0000u;
    const float q = kv_quotient(hi - __uint_as_float(z), 15.f, 1.f / 15.f);
    const uint32_t s = (__float_as_uint(q) + 0xFFFFu) >> 16;  // q >= 0
    if (!fine || (z & 0x7F800000u) == 0x7F800000u || s >= 0x7F80u)
        return 0x7FC0u;
    return s | z;
}

// Eight values that lie on [z, z + 15 s] as whole numbers 0 .. 15 in the low bits of
// 0x4B400000: adding 1.5 2^23 rounds to the nearest, ties to even.
__device__ __forceinline__ void kv_quantise(const float* x, float s, float z, float inv, uint32_t (&c)[8])
{
    float q[8];
#pragma unroll
    for (int e = 0; e < 8; e++)
        q[e] = kv_quotient(x[e] - z, s, inv);
    if (!(s >= kLeastScale))
        for (int e = 0; e < 8; e++)
            q[e] = s > 0.f ? (x[e] - z) / s : 0.f;
#pragma unroll
    for (int e = 0; e < 8; e++)
        c[e] = __float_as_uint(q[e] + 12582912.f);
}

// Their dword of nibbles (element e in nibble e / 2 + 4 (e % 2)); the sum of the
// 0x4B400000 at their places goes, modulo 2^32.
__device__ __forceinline__ uint32_t kv_nibbles(const uint32_t (&c)[8])
{
    uint32_t w = c[7];
    w = (w << 4) + c[5];
    w = (w << 4) + c[3];
    w = (w << 4) + c[1];
    w = (w << 4) + c[6];
    w = (w << 4) + c[4];
    w = (w << 4) + c[2];
    w = (w << 4) + c[0];
    return w - (0x4B400000u * 0x11111111u);
}

// Four of them in bytes.
__device__ __forceinline__ uint32_t kv_bytes(const uint32_t* c)
{
    return (((((c[3] << 8) + c[2]) << 8) + c[1]) << 8) + c[0] - 0x4B400000u * 0x01010101u;
}

template <int W, typename T>
struct KvRowRegs {
    u32x4 w[W / 64][sizeof(T) / 2];  // 8 values each

    __device__ __forceinline__ void load(const T* row, int part, int D)
    {
#pragma unroll
        for (int i = 0; i < W / 64; i++) {
            const int d = part * (W / 8) + 8 * i;
#pragma unroll
            for (int j = 0; j < (int)sizeof(T) / 2; j++)
                w[i][j] = d < D ? ((const u32x4*)(row + d))[j] : u32x4{0, 0, 0, 0};
        }
    }
    __device__ __forceinline__ float at(int i, int e) const
    {
        if (sizeof(T) == 4)
            return __uint_as_float(w[i][e >> 2][e & 3]);
        return __uint_as_float(e & 1 ? w[i][0][e >> 1] & 0xFFFF0000u : w[i][0][e >> 1] << 16);
    }
};

// Packed sequences: the place of a request's first workgroup.  It has at least as many
// as its n rows touch tiles, n / 32 + 2 whatever the slot's length, and the places
// ascend without a sum over the requests.
__device__ __forceinline__ int64_t kv_packed_place(const int32_t* starts, int32_t total, int b)
{
    return seq_first(starts, total, b) / kKvTile + 2ll * b;
}

// The tiles that its n rows can touch.
__device__ __forceinline__ int64_t kv_packed_tiles(int n) { return n > 0 ? n / kKvTile + 2ll : 0; }

// The state after an append of packed sequences, a thread a request.  Starts that do not ascend can leave a
// request without its workgroups: then no request has got rows, and what the append wrote past the slots'
// lengths is cleared.
__global__ __launch_bounds__(256) void kv_packed_state_kernel(KvView c, const int32_t* __restrict__ slots, int32_t B,
                                                              const int32_t* __restrict__ starts, int32_t total)
{
    __shared__ int short_of;
    if (threadIdx.x == 0)
        short_of = 0;
    __syncthreads();
    for (int b = threadIdx.x; b < B; b += 256) {
        const int64_t next = b + 1 < B ? kv_packed_place(starts, total, b + 1) : total / kKvTile + 2ll * B;
        if (next - kv_packed_place(starts, total, b) <
            kv_packed_tiles(seq_end(starts, total, b) - seq_first(starts, total, b)))
            short_of = 1;
    }
    __syncthreads();
    if (short_of) {
        for (int b = blockIdx.x * 256; b < B && b < (int)blockIdx.x * 256 + 256; b++) {
            const int slot = kv_slot(c, slots, b);
            if (slot < 0)
                continue;
            const int64_t len = kv_len(c, slot), past = len + seq_end(starts, total, b) - seq_first(starts, total, b);
            const int64_t end = past < c.cap ? past : c.cap;
            for (int h = 0; h < c.H; h++)
                for (int64_t i = kv_row(c, slot, h) + len + threadIdx.x; i < kv_row(c, slot, h) + end; i += 256) {
                    c.pos[i] = -1;
                    c.weight[i] = 0.f;
                }
        }
        return;
    }
    const int b = blockIdx.x * 256 + threadIdx.x;
    const int slot = b < B ? kv_slot(c, slots, b) : -1;
    if (slot >= 0)
        kv_advance(c, slot, kv_len(c, slot), seq_end(starts, total, b) - seq_first(starts, total, b));
}

// kPacked: `starts` tells the rows of each of the B requests (oil_kv_append_packed), of
// max_rows in all; a workgroup finds its request by bisection and has one tile.
// (Six workgroups a CU: 4 x 8,191 rows in bf16 37 us, at five 39, at four 42; at
// eight, or six with binary32 rows, registers spill.)
template <int W, typename T, bool kPacked>
__global__ __launch_bounds__(256, sizeof(T) == 2 ? 6 : 5) void kv_append_kernel(KvView c, const int32_t* __restrict__ slots,
                                                        const T* __restrict__ k, const T* __restrict__ v, int64_t ld,
                                                        int32_t max_rows, const int32_t* __restrict__ nodes,
                                                        const int32_t* __restrict__ count,
                                                        const float* __restrict__ weight,
                                                        const int32_t* __restrict__ starts, int32_t B)
{
    constexpr int kRow = W / 4 + 1;  // dwords of a row of value codes in LDS
    __shared__ __align__(16) uint32_t image[2 * KvTile<W>::kWords];  // the tile's codes as they are stored
    __shared__ uint32_t vcode[kKvTile][kRow];
    __shared__ int bound;
    const int h = blockIdx.y, tid = threadIdx.x;
    int b = blockIdx.z;
    int64_t turn = blockIdx.x;
    if (kPacked) {
        int past = B;
        while (past - b > 1) {
            const int mid = b + (past - b) / 2;
            if (kv_packed_place(starts, max_rows, mid) <= turn)
                b = mid;
            else
                past = mid;
        }
        turn -= kv_packed_place(starts, max_rows, b);
        if (turn < 0)
            return;
    }
    const int slot = kv_slot(c, slots, b);
    if (slot < 0)
        return;
    const int32_t len = kv_len(c, slot), next = c.state[4 * (int64_t)slot + kKvNext];
    const int row0 = kPacked ? seq_first(starts, max_rows, b) : 0;
    const int cnt = kPacked ? seq_end(starts, max_rows, b) - row0 : kv_count(nodes, count, b, max_rows, &bound);
    const int64_t end = len + (int64_t)cnt < c.cap ? len + (int64_t)cnt : c.cap;
    for (int64_t first = (len / kKvTile + turn) * kKvTile; first < end;
         first += (int64_t)gridDim.x * kKvTile) {  // of the tile
        uint8_t* tile = kv_tiles(c, slot, h) + first / kKvTile * c.tile_bytes;
        const int key = tid >> 3, part = tid & 7;
        const int64_t j = first + key;
        if (j >= len && j < end) {  // the 8 lanes of a row alike
            const int r = (int)(j - len), src = kPacked ? row0 + r : kv_source(nodes, b, max_rows, r);
            const int64_t at = ((kPacked ? 0 : (int64_t)b * max_rows) + src) * ld + (int64_t)h * c.D;
            KvRowRegs<W, T> rows[2];
            rows[0].load(k + at, part, c.D);
            rows[1].load(v + at, part, c.D);
#pragma unroll
            for (int side = 0; side < 2; side++) {
                float x[W / 8];
                float lo = INFINITY, hi = -INFINITY;
                float none[2] = {0.f, 0.f};  // not 0 once a value is not finite
#pragma unroll
                for (int i = 0; i < W / 64; i++) {
                    const bool in = part * (W / 8) + 8 * i < c.D;
                    float l = INFINITY, m = -INFINITY;
#pragma unroll
                    for (int e = 0; e < 8; e++) {
                        x[8 * i + e] = rows[side].at(i, e);
                        l = fminf(l, x[8 * i + e]);
                        m = fmaxf(m, x[8 * i + e]);
                    }
#pragma unroll
                    for (int e = 0; e < 8; e++)
                        none[e & 1] = fmaf(x[8 * i + e], 0.f, none[e & 1]);
                    lo = in ? fminf(lo, l) : lo;
                    hi = in ? fmaxf(hi, m) : hi;
                }
#pragma unroll
                for (int o = 1; o < 8; o <<= 1) {
                    lo = fminf(lo, __shfl_xor(lo, o, 8));
                    hi = fmaxf(hi, __shfl_xor(hi, o, 8));
                }
                const uint64_t odds = __ballot(!(none[0] + none[1] == 0.f));
                const uint32_t pair = kv_pair(lo, hi, ((odds >> (tid & 56)) & 255) == 0);
                const float s = kv_s(pair), z = kv_z(pair), inv = __builtin_amdgcn_rcpf(s);
#pragma unroll
                for (int i = 0; i < W / 64; i++) {
                    const int d = part * (W / 8) + 8 * i;
                    uint32_t codes[8];
#pragma unroll
                    for (int e = 0; e < 8; e++)
                        codes[e] = 0x4B400000u;
                    if (d < c.D)
                        kv_quantise(x + 8 * i, s, z, inv, codes);
                    if (side == 0) {
                        image[kv_word_at((key >> 4) * (W / 32) + (d >> 5), (key & 15) + 16 * ((d & 31) >> 3))] =
                            kv_nibbles(codes);
                    } else {
                        vcode[key][d / 4] = kv_bytes(codes);
                        vcode[key][d / 4 + 1] = kv_bytes(codes + 4);
                    }
                }
                if (part == 0)
                    *(uint32_t*)(tile + (side ? KvTile<W>::kValueScales : KvTile<W>::kKeyScales) + key * 4) = pair;
            }
            if (part == 0) {
                const int64_t at_row = kv_row(c, slot, h) + j;
                const int64_t pos = next + (int64_t)r;
                c.pos[at_row] = pos < INT32_MAX ? (int32_t)pos : INT32_MAX;
                c.weight[at_row] = weight ? weight[((kPacked ? 0 : (int64_t)b * c.H) + h) * max_rows + src] : 0.f;
            }
        }
        __syncthreads();
        const bool full = first >= len && first + kKvTile <= end;
        // four columns' value dwords a thread: eight positions' bytes, two to a byte,
        // and the four by four bytes turned
        if (tid < W) {
            const int g = tid / (W / 4), d4 = tid % (W / 4);
            uint32_t w[8];
#pragma unroll
            for (int e = 0; e < 8; e++)
                w[kv_nibble(e)] = vcode[16 * (e >> 2) + 4 * g + (e & 3)][d4];
            if (!full)
#pragma unroll
                for (int e = 0; e < 8; e++) {
                    const int64_t jj = first + 16 * (e >> 2) + 4 * g + (e & 3);
                    w[kv_nibble(e)] = jj >= len && jj < end ? w[kv_nibble(e)] : 0u;
                }
            uint32_t two[4];
#pragma unroll
            for (int i = 0; i < 4; i++)
                two[i] = w[2 * i] | w[2 * i + 1] << 4;
            // bytes 0 and 1 (2 and 3) of a pair, side by side
            const uint32_t left = __builtin_amdgcn_perm(two[1], two[0], 0x05010400u);
            const uint32_t right = __builtin_amdgcn_perm(two[3], two[2], 0x05010400u);
            const uint32_t left2 = __builtin_amdgcn_perm(two[1], two[0], 0x07030602u);
            const uint32_t right2 = __builtin_amdgcn_perm(two[3], two[2], 0x07030602u);
            const uint32_t word[4] = {(left & 0xFFFFu) | right << 16, left >> 16 | (right & 0xFFFF0000u),
                                      (left2 & 0xFFFFu) | right2 << 16, left2 >> 16 | (right2 & 0xFFFF0000u)};
#pragma unroll
            for (int i = 0; i < 4; i++) {
                const int d = 4 * d4 + i;
                image[KvTile<W>::kWords + kv_word_at(d >> 4, (d & 15) + 16 * g)] = word[i];
            }
        }
        __syncthreads();
        if (full) {
            for (int i = tid; i < KvTile<W>::kWords / 2; i += 256)
                ((u32x4*)tile)[i] = ((const u32x4*)image)[i];
        } else {
            uint32_t* to = (uint32_t*)tile;
            for (int w = tid; w < KvTile<W>::kWords; w += 256) {
                int Q, lane;
                kv_word(w, &Q, &lane);
                const int64_t jj = first + (lane & 15) + 16 * (Q / (W / 32));
                if (jj >= len && jj < end)
                    to[w] = image[w];
                uint32_t keep = 0;
                bool any = false;
#pragma unroll
                for (int e = 0; e < 8; e++) {
                    const int64_t kk = first + 16 * (e >> 2) + 4 * (lane >> 4) + (e & 3);
                    any = any || (kk >= len && kk < end);
                    if (kk < len)
                        keep |= 15u << (4 * kv_nibble(e));
                }
                if (any)
                    to[KvTile<W>::kWords + w] =
                        image[KvTile<W>::kWords + w] | (keep ? to[KvTile<W>::kWords + w] & keep : 0u);
            }
        }
        __syncthreads();
        if (kPacked)
            return;
    }
    if (!kPacked && gridDim.x * gridDim.y <= kTickets && kv_last(c, slot, gridDim.x * gridDim.y) && tid == 0)
        kv_advance(c, slot, len, cnt);
}

// z + s c for eight codes c, as they leave (16-byte stores).
__device__ __forceinline__ void kv_put(float* to, const float (&x)[8])
{
#pragma unroll
    for (int i = 0; i < 2; i++)
        ((floatx4*)to)[i] = floatx4{x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]};
}
__device__ __forceinline__ void kv_put(uint16_t* to, const float (&x)[8])
{
    u32x4 w;
#pragma unroll
    for (int i = 0; i < 4; i++)
        w[i] = pack_bf16(x[2 * i], x[2 * i + 1]);
    *(u32x4*)to = w;
}

// One workgroup per tile of a (request, head): codes to LDS, then eight columns a
// thread, of a key's one dword, or of two neighbouring positions' eight dwords (whose
// nibbles lie 16 bits apart).
template <int W, typename T>
__global__ __launch_bounds__(256) void kv_read_kernel(KvView c, const int32_t* __restrict__ slots, int64_t first,
                                                      int64_t n, T* __restrict__ k_out, T* __restrict__ v_out)
{
    constexpr int kUnits = W / 8, kRows = 256 / kUnits;
    __shared__ __align__(16) uint32_t buf[KvTile<W>::kBytes / 4];
    const int b = blockIdx.z, h = blockIdx.y, tid = threadIdx.x, d = tid % kUnits * 8, row = tid / kUnits;
    const int slot = kv_slot(c, slots, b);
    const int32_t len = slot < 0 ? 0 : kv_len(c, slot);
    const int64_t out = ((int64_t)b * c.H + h) * n - first;
    for (int64_t t0 = (first / kKvTile + (int64_t)blockIdx.x) * kKvTile; t0 < first + n;
         t0 += (int64_t)gridDim.x * kKvTile) {
        if (t0 < len) {
            const u32x4* tile = (const u32x4*)(kv_tiles(c, slot, h) + t0 / kKvTile * c.tile_bytes);
            for (int i = tid; i < KvTile<W>::kBytes / 16; i += 256)
                ((u32x4*)buf)[i] = tile[i];
        }
        __syncthreads();
        auto put = [&](T* to, int key, int scales, float (&x)[8]) {
            const int64_t j = t0 + key;
            if (j < first || j >= first + n || d >= c.D)
                return;
            const uint32_t pair = buf[scales / 4 + key];
            const float s = kv_s(pair), z = kv_z(pair);
#pragma unroll
            for (int i = 0; i < 8; i++)
                x[i] = j < len ? fmaf(s, x[i], z) : 0.f;
            kv_put(to + (out + j) * c.D + d, x);
        };
        for (int key = row; key < kKvTile; key += kRows) {
            const uint32_t w = buf[kv_word_at((key >> 4) * (W / 32) + (d >> 5), (key & 15) + 16 * ((d & 31) >> 3))];
            float x[8];
#pragma unroll
            for (int e = 0; e < 8; e++)
                x[e] = (float)kv_code(w, e);
            put(k_out, key, KvTile<W>::kKeyScales, x);
        }
        for (int two = row; two < kKvTile / 2; two += kRows) {
            const int key = 2 * two, e = 4 * (key >> 4) + (key & 3);
            float x[8], y[8];
#pragma unroll
            for (int i = 0; i < 8; i++) {
                const uint32_t w = buf[KvTile<W>::kValues / 4 +
                                       kv_word_at(d >> 4, (d & 15) + i + 16 * ((key & 15) >> 2))] >> (4 * (e >> 1));
                x[i] = (float)(w & 15u);
                y[i] = (float)(w >> 16 & 15u);
            }
            put(v_out, key, KvTile<W>::kValueScales, x);
            put(v_out, key + 1, KvTile<W>::kValueScales, y);
        }
        __syncthreads();
    }
}

// ---------------------------------------------------------------- eviction
// A row that moves, with what else it carries.
struct KvMove {
    int32_t dst, src, pos;
    float weight;
};

struct KvMoves {
    int32_t n;      // rows before (0: nothing to do)
    int32_t count;  // moves
    int32_t pad[2];
};

// A head's part of the workspace: KvMoves, the tile that the budget ends in as
// it was, the first move into each tile below the budget (and one past), the moves.
struct KvMovesAt {
    int64_t tile, first, moves, stride;
};

__host__ __device__ __forceinline__ KvMovesAt kv_moves_at(const KvView& c, int64_t keep)
{
    KvMovesAt at;
    const int64_t most = keep < c.cap - keep ? keep : c.cap - keep;
    at.tile = sizeof(KvMoves);
    at.first = at.tile + c.tile_bytes;
    at.moves = at.first + (keep / kKvTile + 5) / 4 * 16;
    at.stride = at.moves + most * (int64_t)sizeof(KvMove);
    return at;
}

// Rank of a row: recent rows above every weight, NaN below.
__device__ __forceinline__ uint32_t kv_rank(float w, bool young)
{
    if (young)
        return 0xFFFFFFFFu;
    return w != w ? 0u : score_code(w);
}

constexpr int kSelect = 1024, kSelectWaves = kSelect / 64;
constexpr int kDigit = 11, kBins = 1 << kDigit;
constexpr int32_t kHeldRanks = 36864;  // ranks that fit LDS beside the bins

// Sums of `mine` over the waves before this one, and over all (each wave's lanes alike).
__device__ __forceinline__ int kv_before(int mine, int* waves, int* total)
{
    const int wave = threadIdx.x >> 6;
    __syncthreads();
    if ((threadIdx.x & 63) == 0)
        waves[wave] = mine;
    __syncthreads();
    int before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < kSelectWaves; w++) {
        before += w < wave ? waves[w] : 0;
        all += waves[w];
    }
    *total = all;
    return before;
}

// One workgroup per (request, head).  The keep-th largest rank by three digits
// of 11 bits; then, each wave over a stretch of its own in chunks of 64 rows,
// ranks among ties, holes and late rows by ballots, with one exchange between the waves each.
__global__ __launch_bounds__(kSelect) void kv_select_kernel(KvView c, const int32_t* __restrict__ slots, int64_t keep,
                                                            int64_t recent, uint8_t* __restrict__ work)
{
    __shared__ uint32_t held[kHeldRanks];
    __shared__ uint32_t hist[kBins];
    __shared__ int waves[kSelectWaves];
    __shared__ uint32_t digit, above;
    const int b = blockIdx.y, h = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const KvMovesAt at = kv_moves_at(c, keep);
    uint8_t* mine = work + ((int64_t)b * c.H + h) * at.stride;
    KvMoves* head = (KvMoves*)mine;
    const int slot = kv_slot(c, slots, b);
    const int32_t n = slot < 0 ? 0 : kv_len(c, slot);
    if (n <= keep) {
        if (tid == 0) {
            head->n = 0;
            head->count = 0;
        }
        return;
    }
    KvMove* moves = (KvMove*)(mine + at.moves);
    int32_t* first = (int32_t*)(mine + at.first);
    const int64_t row = kv_row(c, slot, h);
    const int64_t young = c.state[4 * (int64_t)slot + kKvNext] - recent;
    const bool holds = n <= kHeldRanks;
    auto rank = [&](int32_t i) {
        return holds ? held[i] : kv_rank(c.weight[row + i], c.pos[row + i] >= young);
    };
    if (holds)
        for (int32_t i0 = 0; i0 < n; i0 += 8 * kSelect) {  // eight rows' loads of a thread at once
            float w[8];
            int32_t p[8];
#pragma unroll
            for (int x = 0; x < 8; x++) {
                const int32_t i = i0 + x * kSelect + tid, at = i < n ? i : n - 1;
                w[x] = c.weight[row + at];
                p[x] = c.pos[row + at];
            }
#pragma unroll
            for (int x = 0; x < 8; x++)
                if (i0 + x * kSelect + tid < n)
                    held[i0 + x * kSelect + tid] = kv_rank(w[x], p[x] >= young);
        }
    uint32_t prefix = 0, need = (uint32_t)keep;  // rows still to take at the prefix
    for (int shift = 21; ; shift = shift > 10 ? shift - kDigit : 0) {
        // digits of bits 31 .. 21, 20 .. 10, 9 .. 0
        const int width = shift ? kDigit : 10;
        for (int i = tid; i < kBins; i += kSelect)
            hist[i] = 0;
        __syncthreads();
#pragma unroll 4
        for (int32_t i = tid; i < n; i += kSelect) {
            const uint32_t r = rank(i);
            const bool counts = shift == 21 || (r >> (shift + width)) == (prefix >> (shift + width));
            // recent rows share one rank: one lane adds them all
            const uint64_t same = __ballot(counts && r == 0xFFFFFFFFu);
            if (counts && (r != 0xFFFFFFFFu || lane == __ffsll((unsigned long long)same) - 1))
                atomicAdd(&hist[(r >> shift) & ((1u << width) - 1)], r != 0xFFFFFFFFu ? 1u : (uint32_t)__popcll(same));
        }
        __syncthreads();
        // the digit: bins from the top until `need` rows are reached; a thread holds two
        const int bin = kBins - 1 - 2 * tid;
        const uint32_t x0 = hist[bin], x1 = hist[bin - 1];
        uint32_t sum = x0 + x1;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const uint32_t y = __shfl_up(sum, o, 64);
            sum += lane >= o ? y : 0;
        }
        int all;
        const uint32_t before = (uint32_t)kv_before((int)__shfl(sum, 63, 64), waves, &all) + sum - x0 - x1;
        if (before < need && before + x0 >= need) {
            digit = (uint32_t)bin;
            above = before;
        } else if (before + x0 < need && before + x0 + x1 >= need) {
            digit = (uint32_t)bin - 1;
            above = before + x0;
        }
        __syncthreads();
        prefix |= digit << shift;
        need -= above;
        __syncthreads();
        if (shift == 0)
            break;
    }
    // rows above the rank stay, and the first `need` at it
    const int32_t span = ((n + kSelect - 1) / kSelect) * 64, i0 = wave * span, i1 = min(i0 + span, n);
    int count = 0, total;
    for (int32_t i = i0; i < i1; i += 64)
        count += __popcll(__ballot(i + lane < i1 && rank(i + lane) == prefix));
    const int tied = kv_before(count, waves, &total);
    const uint64_t below = (1ull << lane) - 1;
    // a chunk's masks of rows that stay, given the ties before it
    auto stays = [&](int32_t i, int* ties, uint32_t* r) {
        const bool in = i + lane < i1;
        *r = in ? rank(i + lane) : 0;
        const uint64_t eq = __ballot(in && *r == prefix);
        const bool yes = in && (*r > prefix || (*r == prefix && *ties + __popcll(eq & below) < (int)need));
        *ties += __popcll(eq);
        return yes;
    };
    int ties = tied, holes = 0, late = 0;
    uint32_t r;
    for (int32_t i = i0; i < i1; i += 64) {
        const bool yes = stays(i, &ties, &r);
        holes += __popcll(__ballot(i + lane < i1 && i + lane < keep && !yes));
        late += __popcll(__ballot(i + lane >= keep && yes));
    }
    int moving;
    int hole = kv_before(holes, waves, &moving);
    int from = kv_before(late, waves, &total);
    ties = tied;
    for (int32_t i = i0; i < i1; i += 64) {
        const int32_t x = i + lane;
        const bool yes = stays(i, &ties, &r);
        const bool open = x < i1 && x < keep && !yes, moves_in = x >= keep && yes;
        const uint64_t mo = __ballot(open), mf = __ballot(moves_in);
        const int at_hole = hole + __popcll(mo & below);
        if (open)
            moves[at_hole].dst = x;
        if (x < i1 && x < keep && (x & (kKvTile - 1)) == 0)
            first[x / kKvTile] = at_hole;
        if (moves_in)
            moves[from + __popcll(mf & below)].src = x;
        hole += __popcll(mo);
        from += __popcll(mf);
    }
    // (the late rows are a few waves' stretches: all waves fetch what they carry)
    __syncthreads();
    for (int i = tid; i < moving; i += kSelect) {
        const int32_t x = moves[i].src;
        moves[i].pos = c.pos[row + x];
        moves[i].weight = c.weight[row + x];
    }
    if (tid == 0) {
        head->n = n;
        head->count = moving;
        first[(keep + kKvTile - 1) / kKvTile] = moving;
    }
    if (keep % kKvTile) {
        const u32x4* tile = (const u32x4*)(kv_tiles(c, slot, h) + keep / kKvTile * c.tile_bytes);
        for (int i = tid; i < c.tile_bytes / 16; i += kSelect)
            ((u32x4*)(mine + at.tile))[i] = tile[i];
    }
}

// A workgroup per destination tile, of one wave where there are many (a tile's
// dependent loads are the time, and tiles in flight cover it: 65,536 tiles 116 us,
// with two waves 136, with four 188), of four where there are few (1,024 tiles 6.4 us,
// with one 9.3).  Rows that move out of the tile that the budget ends in are read
// from its copy: that tile may be written meanwhile.
template <int W>
__global__ __launch_bounds__(256) void kv_move_kernel(KvView c, const int32_t* __restrict__ slots, int64_t keep,
                                                      const uint8_t* __restrict__ work)
{
    __shared__ int32_t source[kKvTile];
    const int b = blockIdx.z, h = blockIdx.y, tid = threadIdx.x;
    const int slot = kv_slot(c, slots, b);
    if (slot < 0)
        return;
    const KvMovesAt at = kv_moves_at(c, keep);
    const uint8_t* mine = work + ((int64_t)b * c.H + h) * at.stride;
    const int32_t n = ((const KvMoves*)mine)->n;
    if (n == 0)
        return;
    const KvMove* moves = (const KvMove*)(mine + at.moves);
    const int32_t* first = (const int32_t*)(mine + at.first);
    const int64_t row = kv_row(c, slot, h);
    // rows past the budget leave
    for (int64_t i = keep + (int64_t)blockIdx.x * blockDim.x + tid; i < n;
         i += (int64_t)gridDim.x * blockDim.x) {
        c.pos[row + i] = -1;
        c.weight[row + i] = 0.f;
    }
    if (blockIdx.x == 0 && h == 0 && tid == 0)
        c.state[4 * (int64_t)slot + kKvLen] = (int32_t)keep;
    uint8_t* tiles = kv_tiles(c, slot, h);
    const int32_t edge = keep % kKvTile ? (int32_t)(keep / kKvTile) : -1;
    auto from = [&](int32_t src) -> const uint8_t* {
        return (src >> 5) == edge ? mine + at.tile : tiles + (int64_t)(src >> 5) * c.tile_bytes;
    };
    for (int32_t t = blockIdx.x; (int64_t)t * kKvTile < keep; t += gridDim.x) {
        const int m0 = first[t], m1 = first[t + 1];
        if (m0 == m1)
            continue;
        __syncthreads();
        if (tid < kKvTile)
            source[tid] = -1;
        __syncthreads();
        if (tid < m1 - m0) {
            const KvMove m = moves[m0 + tid];
            source[m.dst & 31] = m.src;
            c.pos[row + m.dst] = m.pos;
            c.weight[row + m.dst] = m.weight;
        }
        __syncthreads();
        uint8_t* tile = tiles + (int64_t)t * c.tile_bytes;
        // a lane's loads are made wherever its row comes from, its own place for one that
        // does not move, so that none waits for another's condition (the keys' own places
        // are a quarter of what is read; without them 1 to 2% slower all the same, for
        // lines that are then written in part)
        typedef uint32_t quarter __attribute__((ext_vector_type(W / 32)));
        quarter code[2];
        uint32_t* to[2];
        bool on[2];
#pragma unroll
        for (int i = 0; i < 2; i++) {  // keys: a quarter of a row a lane
            const int x = tid + i * (int)blockDim.x, key = (x >> 2) & 31, g = x & 3;
            const int32_t src = source[key];
            on[i] = src >= 0 && x < 4 * kKvTile;
            to[i] = (uint32_t*)tile + kv_word_at((key >> 4) * (W / 32), (key & 15) + 16 * g);
            const uint32_t* at_src = (const uint32_t*)from(src) + kv_word_at(((src >> 4) & 1) * (W / 32), (src & 15) + 16 * g);
            code[i] = *(const quarter*)(on[i] ? at_src : to[i]);
        }
        const int32_t its = source[tid & 31];  // scales
        const int pairs = ((tid >> 5) & 1 ? KvTile<W>::kValueScales : KvTile<W>::kKeyScales) / 4;
        uint32_t* pair_to = (uint32_t*)tile + pairs + (tid & 31);
        const uint32_t pair = *(its >= 0 ? (const uint32_t*)from(its) + pairs + (its & 31) : pair_to);
#pragma unroll 2
        for (int w = tid; w < KvTile<W>::kWords; w += blockDim.x) {  // values: a nibble of each dword a row
            int Q, lane;
            kv_word(w, &Q, &lane);
            uint32_t* word_to = (uint32_t*)(tile + KvTile<W>::kValues) + w;
            uint32_t clear = 0, got[8];
            int32_t src[8];
#pragma unroll
            for (int e = 0; e < 8; e++) {  // (one group of positions a wave)
                src[e] = __builtin_amdgcn_readfirstlane(source[16 * (e >> 2) + 4 * (lane >> 4) + (e & 3)]);
                clear |= src[e] >= 0 ? 15u << (4 * kv_nibble(e)) : 0u;
            }
            if (!clear)
                continue;
#pragma unroll
            for (int e = 0; e < 8; e++)
                got[e] = *(src[e] < 0 ? word_to
                                      : (const uint32_t*)(from(src[e]) + KvTile<W>::kValues) +
                                            kv_word_at(Q, (lane & 15) + 16 * ((src[e] & 15) >> 2)));
            uint32_t word = *word_to & ~clear;
#pragma unroll
            for (int e = 0; e < 8; e++)
                if (src[e] >= 0)
                    word |= (uint32_t)kv_code(got[e], 4 * ((src[e] >> 4) & 1) + (src[e] & 3)) << (4 * kv_nibble(e));
            *word_to = word;
        }
#pragma unroll
        for (int i = 0; i < 2; i++)
            if (on[i])
                *(quarter*)to[i] = code[i];
        if (tid < 64 && its >= 0)
            *pair_to = pair;
    }
}

}  // namespace

hipError_t launch_kv_clear(const KvView& c, hipStream_t stream)
{
    const int64_t n = (int64_t)c.n_slots * c.H * c.cap;
    const int64_t blocks = (n + 2047) / 2048 < 2048 ? (n + 2047) / 2048 : 2048;
    hipLaunchKernelGGL(kv_clear_kernel, dim3((unsigned)blocks), dim3(256), 0, stream, c);
    return hipGetLastError();
}

hipError_t launch_kv_reset(const KvView& c, const int32_t* slots, int32_t B, hipStream_t stream)
{
    const int64_t blocks = (c.cap + 4095) / 4096 < 64 ? (c.cap + 4095) / 4096 : 64;
    hipLaunchKernelGGL(kv_reset_kernel, dim3((unsigned)blocks, c.H, B), dim3(256), 0, stream, c, slots);
    if (blocks * c.H > kTickets)
        hipLaunchKernelGGL(kv_state_kernel, dim3(B), dim3(64), 0, stream, c, slots, 0, nullptr, nullptr);
    return hipGetLastError();
}

hipError_t launch_kv_append(const KvView& c, const int32_t* slots, int32_t B, const void* k, const void* v,
                            int dtype, int64_t ld, int32_t max_rows, const int32_t* nodes, const int32_t* count,
                            const float* weight, hipStream_t stream)
{
    // tiles that max_rows rows can touch from any length on
    int64_t tiles = ((int64_t)max_rows + kKvTile - 1 + kKvTile - 1) / kKvTile;
    tiles = tiles < c.tiles ? tiles : c.tiles;
    const dim3 grid((unsigned)(tiles < kMaxGridTiles ? tiles : kMaxGridTiles), c.H, B), block(256);
#define OIL_KV_APPEND(W, T)                                                                                       \
    hipLaunchKernelGGL((kv_append_kernel<W, T, false>), grid, block, 0, stream, c, slots, (const T*)k, (const T*)v, \
                       ld, max_rows, nodes, count, weight, nullptr, 0)
    if (c.W == 64 && dtype == 0)
        OIL_KV_APPEND(64, float);
    else if (c.W == 64)
        OIL_KV_APPEND(64, uint16_t);
    else if (dtype == 0)
        OIL_KV_APPEND(128, float);
    else
        OIL_KV_APPEND(128, uint16_t);
#undef OIL_KV_APPEND
    if ((int64_t)grid.x * c.H > kTickets)
        hipLaunchKernelGGL(kv_state_kernel, dim3(B), dim3(64), 0, stream, c, slots, max_rows, nodes, count);
    return hipGetLastError();
}

hipError_t launch_kv_append_packed(const KvView& c, const int32_t* slots, int32_t B, const int32_t* starts,
                                   int32_t total, const void* k, const void* v, int dtype, int64_t ld,
                                   const float* weight, hipStream_t stream)
{
    const dim3 grid((unsigned)(total / kKvTile + 2ll * B), c.H), block(256);
#define OIL_KV_APPEND(W, T)                                                                                      \
    hipLaunchKernelGGL((kv_append_kernel<W, T, true>), grid, block, 0, stream, c, slots, (const T*)k, (const T*)v, \
                       ld, total, nullptr, nullptr, weight, starts, B)
    if (c.W == 64 && dtype == 0)
        OIL_KV_APPEND(64, float);
    else if (c.W == 64)
        OIL_KV_APPEND(64, uint16_t);
    else if (dtype == 0)
        OIL_KV_APPEND(128, float);
    else
        OIL_KV_APPEND(128, uint16_t);
#undef OIL_KV_APPEND
    hipLaunchKernelGGL(kv_packed_state_kernel, dim3((B + 255) / 256), dim3(256), 0, stream, c, slots, B, starts, total);
    return hipGetLastError();
}

hipError_t launch_kv_read(const KvView& c, const int32_t* slots, int32_t B, int64_t first, int64_t n, void* k_out,
                          void* v_out, int dtype, hipStream_t stream)
{
    const int64_t tiles = (first + n - 1) / kKvTile - first / kKvTile + 1;
    const dim3 grid((unsigned)(tiles < kMaxGridTiles ? tiles : kMaxGridTiles), c.H, B), block(256);
#define OIL_KV_READ(W, T)                                                                                 \
    hipLaunchKernelGGL((kv_read_kernel<W, T>), grid, block, 0, stream, c, slots, first, n, (T*)k_out, (T*)v_out)
    if (c.W == 64 && dtype == 0)
        OIL_KV_READ(64, float);
    else if (c.W == 64)
        OIL_KV_READ(64, uint16_t);
    else if (dtype == 0)
        OIL_KV_READ(128, float);
    else
        OIL_KV_READ(128, uint16_t);
#undef OIL_KV_READ
    return hipGetLastError();
}

size_t kv_evict_workspace_bytes(const KvView& c, int32_t B, int64_t keep)
{
    return (size_t)B * c.H * (size_t)kv_moves_at(c, keep).stride;
}

hipError_t launch_kv_evict(const KvView& c, const int32_t* slots, int32_t B, int64_t keep, int64_t recent,
                           void* workspace, hipStream_t stream)
{
    hipLaunchKernelGGL(kv_select_kernel, dim3(c.H, B), dim3(kSelect), 0, stream, c, slots, keep, recent,
                       (uint8_t*)workspace);
    const int64_t tiles = (keep + kKvTile - 1) / kKvTile;
    const dim3 grid((unsigned)(tiles < 4096 ? tiles : 4096), c.H, B), block(tiles * c.H * B > 8192 ? 64 : 256);
    if (c.W == 64)
        hipLaunchKernelGGL(kv_move_kernel<64>, grid, block, 0, stream, c, slots, keep, (const uint8_t*)workspace);
    else
        hipLaunchKernelGGL(kv_move_kernel<128>, grid, block, 0, stream, c, slots, keep,
                           (const uint8_t*)workspace);
    return hipGetLastError();
}

}  // namespace oil
