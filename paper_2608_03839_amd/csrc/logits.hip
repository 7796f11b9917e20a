// Log probabilities of tokens from rows of logits, with the entropy and the most
// likely tokens.  Contract: include/oilbird.h.
//
// One pass over a row: with m the running maximum, z = (x - m) log2 e, a lane keeps
//     s = sum 2^z,  t = sum z 2^z,
// both rescaled when m rises.  Then
//     log p = (x - m) - ln s,      H = ln s - ln 2 t / s,
// where both terms of H are at least 0, so that nothing cancels.  9 instructions a value,
// one of them an exponential; the pass over many rows is bound by memory: 4,054 rows of
// 50,021 binary32 values 143 us (5.7 TB/s), 1,635 of 131,072 bf16 values with
// eight alternatives 98 us (4.4 TB/s, and the VALU 0.77 of the cycles).
//
// The k best tokens (logit descending, token ascending: one 64-bit key a token) are a
// list over the lanes of a wave, which a step of values enters only where some lane's
// largest reaches a bound: at first the k-th largest of the lanes' own maxima, then the
// list's last or that of another wave of the workgroup.  A few keys enter one after the other, more
// are sorted and joined with the list; so are the waves' lists, in pairs.
//
// Where rows are few, a row is cut among workgroups, and a second launch joins: 61 rows of
// 131,072 bf16 values 8.6 and 3.6 us.  A row of up to 160 KiB stays one wide workgroup's, as
// a second launch costs more: one of 32,003 binary32 values 12.4 us, two rounds of loads.
#include "common.hpp"
#include "internal.hpp"

namespace oil {

namespace {

constexpr int kDeep = 4;  // loads of a lane in flight
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kLeast = -2000.f;  // below any z whose power of two is not 0
constexpr float kLowest = -3.4028234663852886e38f;

// m, and the sums relative to it; m is -FLT_MAX at first.
struct Sums {
    float m, s, t;
};

__device__ __forceinline__ Sums join(Sums a, Sums b)
{
    Sums r;
    r.m = fmaxf(a.m, b.m);
    const float ya = fmaxf((a.m - r.m) * kLog2e, kLeast), yb = fmaxf((b.m - r.m) * kLog2e, kLeast);
    const float fa = __builtin_amdgcn_exp2f(ya), fb = __builtin_amdgcn_exp2f(yb);
    r.s = a.s * fa + b.s * fb;
    r.t = fmaf(ya, a.s, a.t) * fa + fmaf(yb, b.s, b.t) * fb;
    return r;
}

template <int kControl>
__device__ __forceinline__ float moved(float x)
{
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), kControl, 0xF, 0xF, true));
}

// Over a wave, in every lane: neighbours by lane moves, then halves of 16 and 32.
__device__ __forceinline__ Sums join_wave(Sums a)
{
    a = join(a, Sums{moved<0xB1>(a.m), moved<0xB1>(a.s), moved<0xB1>(a.t)});
    a = join(a, Sums{moved<0x4E>(a.m), moved<0x4E>(a.s), moved<0x4E>(a.t)});
    a = join(a, Sums{moved<0x141>(a.m), moved<0x141>(a.s), moved<0x141>(a.t)});
    a = join(a, Sums{moved<0x140>(a.m), moved<0x140>(a.s), moved<0x140>(a.t)});
    a = join(a, Sums{__shfl_xor(a.m, 16), __shfl_xor(a.s, 16), __shfl_xor(a.t, 16)});
    return join(a, Sums{__shfl_xor(a.m, 32), __shfl_xor(a.s, 32), __shfl_xor(a.t, 32)});
}

// A token's key: larger is better; 0: not a candidate (-inf, NaN).
__device__ __forceinline__ uint64_t token_key(float x, uint32_t token)
{
    return x > -INFINITY ? rank_key(x, token) : 0ull;
}

__device__ __forceinline__ uint64_t lane_key(uint64_t k, int lane)
{
    return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(k >> 32), lane) << 32 |
           (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)k, lane);
}

// The key of the lane before.
__device__ __forceinline__ uint64_t key_before(uint64_t k)
{
    const uint32_t hi = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)(k >> 32), 0x138, 0xF, 0xF, true);
    const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)k, 0x138, 0xF, 0xF, true);
    return (uint64_t)hi << 32 | lo;
}

template <int kControl>
__device__ __forceinline__ uint64_t moved_key(uint64_t k)
{
    const uint32_t hi = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)(k >> 32), kControl, 0xF, 0xF, true);
    const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)k, kControl, 0xF, 0xF, true);
    return (uint64_t)hi << 32 | lo;
}

// The larger (or smaller) of a lane's key and that of lane ^ kFar.
template <int kFar>
__device__ __forceinline__ uint64_t exchanged(uint64_t k, bool larger)
{
    uint64_t a = k, b;
    if (kFar == 1)
        b = moved_key<0xB1>(k);
    else if (kFar == 2)
        b = moved_key<0x4E>(k);
    else if (kFar == 4)
        b = moved_key<0x1B>(moved_key<0x141>(k));  // mirrored in 8, then in 4
    else if (kFar == 8)
        b = moved_key<0x128>(k);  // turned by 8 in 16
    else {
        // the two lanes' keys in both
        const auto lo = kFar == 16 ? __builtin_amdgcn_permlane16_swap((uint32_t)k, (uint32_t)k, false, false)
                                   : __builtin_amdgcn_permlane32_swap((uint32_t)k, (uint32_t)k, false, false);
        const auto hi = kFar == 16
                            ? __builtin_amdgcn_permlane16_swap((uint32_t)(k >> 32), (uint32_t)(k >> 32), false, false)
                            : __builtin_amdgcn_permlane32_swap((uint32_t)(k >> 32), (uint32_t)(k >> 32), false, false);
        a = (uint64_t)hi[0] << 32 | lo[0];
        b = (uint64_t)hi[1] << 32 | lo[1];
    }
    return (a > b) == larger ? a : b;
}

// Sorts keys that rise and then fall, or the other way round, by lane (or kSize lanes each):
// the largest first where `falling`.
template <int kSize>
__device__ __forceinline__ uint64_t merged(uint64_t k, int lane, bool falling)
{
    if (kSize >= 64)
        k = exchanged<32>(k, ((lane & 32) == 0) == falling);
    if (kSize >= 32)
        k = exchanged<16>(k, ((lane & 16) == 0) == falling);
    if (kSize >= 16)
        k = exchanged<8>(k, ((lane & 8) == 0) == falling);
    if (kSize >= 8)
        k = exchanged<4>(k, ((lane & 4) == 0) == falling);
    if (kSize >= 4)
        k = exchanged<2>(k, ((lane & 2) == 0) == falling);
    return exchanged<1>(k, ((lane & 1) == 0) == falling);
}

// A wave's keys, the smallest first.
__device__ __forceinline__ uint64_t rising(uint64_t k, int lane)
{
    k = merged<2>(k, lane, (lane & 2) != 0);
    k = merged<4>(k, lane, (lane & 4) != 0);
    k = merged<8>(k, lane, (lane & 8) != 0);
    k = merged<16>(k, lane, (lane & 16) != 0);
    k = merged<32>(k, lane, (lane & 32) != 0);
    return merged<64>(k, lane, false);
}

// The best keys a wave has seen, best first by lane; k of them count.  kMany: more than kSerial keys
// that are to enter are sorted first (2 x 82 rows of 1,279 values, k = 64: 56 us without, 15 with; k = 8
// has few such steps, and 32 trees of 131,072 values 101 us with, 98 without, in registers that leave
// room for fewer waves).
constexpr int kSerial = 6, kFewKeys = 16;

template <bool kMany>
struct Best {
    uint64_t mine = 0, last = 0;  // last: the k-th

    // The best of two lists, the other's lanes turned round.
    __device__ __forceinline__ void join(uint64_t other, int lane, int k)
    {
        mine = merged<64>(mine > other ? mine : other, lane, true);
        last = lane_key(mine, k - 1);
    }

    // Enters one key a lane; 0 enters nothing.
    __device__ __forceinline__ void add(uint64_t key, int lane, int k)
    {
        uint64_t who = __ballot(key > last);
        if (kMany && __popcll(who) > kSerial) {
            join(rising(key > last ? key : 0ull, lane), lane, k);
            return;
        }
        while (who) {
            const int from = __builtin_ctzll(who);
            const uint64_t x = lane_key(key, from);
            const int place = __popcll(__ballot(mine > x));
            const uint64_t up = key_before(mine);
            mine = lane < place ? mine : lane == place ? x : up;
            last = lane_key(mine, k - 1);
            who &= ~(1ull << from) & __ballot(key > last);
        }
    }
};

template <int kControl>
__device__ __forceinline__ uint32_t max_moved(uint32_t x)
{
    const uint32_t y = __builtin_amdgcn_update_dpp(0, (int)x, kControl, 0xF, 0xF, true);
    return x > y ? x : y;
}

// At most the k-th largest of the lanes' codes (0 where fewer lanes have one): with k = 1
// the largest, else its first 16 bits.
__device__ __forceinline__ uint32_t kth_code(uint32_t code, int k)
{
    if (k == 1) {
        code = max_moved<0x140>(max_moved<0x141>(max_moved<0x4E>(max_moved<0xB1>(code))));
        auto r = __builtin_amdgcn_permlane16_swap(code, code, false, false);
        code = r[0] > r[1] ? r[0] : r[1];
        r = __builtin_amdgcn_permlane32_swap(code, code, false, false);
        return r[0] > r[1] ? r[0] : r[1];
    }
    uint32_t at = 0;
#pragma unroll
    for (int bit = 31; bit >= 16; bit--) {
        const uint32_t up = at | 1u << bit;
        at = __popcll(__ballot(code >= up)) >= k ? up : at;
    }
    return at;
}

// A row as loads of 16 bytes, aligned; `off` values of the first lie before it.
template <typename X>
struct Row {
    static constexpr int E = 16 / sizeof(X);
    const X* x;
    int V, off;

    __device__ __forceinline__ Row(const X* row, int v)
        : x(row), V(v), off((int)((uintptr_t)row % 16) / (int)sizeof(X))
    {
    }
    __device__ __forceinline__ int64_t loads() const { return ((int64_t)V + off + E - 1) / E; }
    // The first token of load g.
    __device__ __forceinline__ int64_t token(int64_t g) const { return g * E - off; }
    // Whether all values of load g are the row's.
    __device__ __forceinline__ bool whole(int64_t g) const { return token(g) >= 0 && token(g) + E <= V; }
    static __device__ __forceinline__ float value(float v) { return v; }
    static __device__ __forceinline__ float value(uint16_t v) { return bf16_bits_to_float(v); }
    __device__ __forceinline__ float one(int64_t token) const { return value(x[token]); }
    __device__ __forceinline__ u32x4 load(int64_t g) const { return *(const u32x4*)(x + token(g)); }
    static __device__ __forceinline__ float of(const u32x4& w, int e)
    {
        if (E == 4)
            return __uint_as_float(w[e & 3]);
        return __uint_as_float(e & 1 ? w[e >> 1 & 3] & 0xFFFF0000u : w[e >> 1 & 3] << 16);
    }
    // -inf in every place.
    static __device__ __forceinline__ u32x4 none()
    {
        const uint32_t w = E == 4 ? 0xFF800000u : 0xFF80FF80u;
        return u32x4{w, w, w, w};
    }
    // Load g with -inf where it leaves the row.
    __device__ __forceinline__ u32x4 part(int64_t g) const
    {
        u32x4 w = none();
#pragma unroll
        for (int e = 0; e < E; e++)
            if (token(g) + e >= 0 && token(g) + e < V) {
                if (E == 4)
                    w[e & 3] = __float_as_uint(one(token(g) + e));
                else
                    w[e >> 1 & 3] = e & 1 ? (w[e >> 1 & 3] & 0xFFFFu) | __float_as_uint(one(token(g) + e))
                                          : (w[e >> 1 & 3] & 0xFFFF0000u) | __float_as_uint(one(token(g) + e)) >> 16;
            }
        return w;
    }
};

// LDS of a workgroup of NT threads.
template <int NT>
struct Shared {
    uint64_t keys[NT / 64 * OIL_TOPK_MAX];
    Sums sums[NT / 64];
    uint32_t bound;
};

// The part [g0, g1) of a row's loads by NT threads: in the first wave, the part's sums in
// every lane, and the i-th best key in lane i (0 past the k).
template <typename X, int NT, bool kMany>
__device__ __forceinline__ void scan_part(const Row<X>& row, int64_t g0, int64_t g1, int k, Shared<NT>& lds, Sums* sums,
                                          uint64_t* key)
{
    constexpr int E = Row<X>::E;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    Sums a = {kLowest, 0.f, 0.f};
    Best<kMany> best;
    uint32_t bound = 0;  // code below which nothing enters
    if (threadIdx.x == 0)
        lds.bound = 0;
    __syncthreads();
    bool begun = false;
    for (int64_t g = g0 + wave * 64; g < g1; g += NT * kDeep) {
        u32x4 w[kDeep];
        const bool inner = row.whole(g) && g + NT * (kDeep - 1) + 64 <= g1 && row.whole(g + NT * (kDeep - 1) + 63);
        int n = kDeep;  // loads of this step
        if (inner) {
#pragma unroll
            for (int i = 0; i < kDeep; i++)
                w[i] = row.load(g + i * NT + lane);
        } else {
            n = 0;
#pragma unroll
            for (int i = 0; i < kDeep; i++) {
                const int64_t at = g + i * NT + lane;
                w[i] = Row<X>::none();
                if (at < g1)
                    w[i] = row.whole(at) ? row.load(at) : row.part(at);
                n += g + i * NT < g1;
            }
        }
        float top[kDeep], most = kLowest;
#pragma unroll
        for (int i = 0; i < kDeep; i++) {
            top[i] = Row<X>::of(w[i], 0);
#pragma unroll
            for (int e = 1; e < E; e++)
                top[i] = fmaxf(top[i], Row<X>::of(w[i], e));
            most = fmaxf(most, top[i]);
        }
        const float m = fmaxf(a.m, most);
        const float y = fmaxf((a.m - m) * kLog2e, kLeast), f = __builtin_amdgcn_exp2f(y);
        a.t = fmaf(y, a.s, a.t) * f;
        a.s *= f;
        a.m = m;
#pragma unroll
        for (int i = 0; i < kDeep; i++) {
            if (i >= n)
                break;
            float s[2] = {0.f, 0.f}, t[2] = {0.f, 0.f};
#pragma unroll
            for (int e = 0; e < E; e++) {
                const float z = (Row<X>::of(w[i], e) - m) * kLog2e, p = __builtin_amdgcn_exp2f(z);
                s[e & 1] += p;
                t[e & 1] = fmaf(fmaxf(z, kLeast), p, t[e & 1]);
            }
            a.s += s[0] + s[1];
            a.t += t[0] + t[1];
        }
        if (k == 0)
            continue;
        const uint32_t code = score_code(most);
        if (!begun) {
            begun = true;
            const uint32_t c = kth_code(code, k);
            bound = c > bound ? c : bound;
        }
        const uint32_t others = *(volatile uint32_t*)&lds.bound;
        bound = others > bound ? others : bound;
        if (!__ballot(code >= bound))
            continue;
#pragma unroll
        for (int i = 0; i < kDeep; i++) {
            if (!__ballot(score_code(top[i]) >= bound))
                continue;
#pragma unroll
            for (int e = 0; e < E; e++) {
                const float x = Row<X>::of(w[i], e);
                const bool enters = score_code(x) >= bound;
                if (__ballot(enters))
                    best.add(enters ? token_key(x, (uint32_t)(row.token(g + i * NT + lane) + e)) : 0ull, lane, k);
            }
        }
        const uint32_t mine = (uint32_t)(best.last >> 32);
        if (mine > bound) {
            bound = mine;
            if (lane == 0)
                atomicMax(&lds.bound, mine);
        }
    }
    a = join_wave(a);
    if (lane == 0)
        lds.sums[wave] = a;
    // waves' lists in pairs
    if (lane < k)
        lds.keys[wave * k + lane] = best.mine;
    for (int n = NT / 128; n >= 1; n /= 2) {
        __syncthreads();
        if (k > 0 && wave < n) {
            best.mine = lane < k ? best.mine : 0ull;
            best.join(63 - lane < k ? lds.keys[(wave + n) * k + 63 - lane] : 0ull, lane, k);
            if (lane < k)
                lds.keys[wave * k + lane] = best.mine;
        }
    }
    if (wave == 0) {
        a = lane < NT / 64 ? lds.sums[lane] : Sums{kLowest, 0.f, 0.f};
        *sums = join_wave(a);
        *key = lane < k ? best.mine : 0ull;
    }
}

// What a row of which a is known gives; by one wave, whose lane i has the i-th best key.
template <typename X>
__device__ __forceinline__ void write_row(const Row<X>& row, int64_t r, Sums a, uint64_t key, const int32_t* tokens,
                                          int M, int k, float* logprob, float* entropy, int32_t* top_tokens,
                                          float* top_logprobs)
{
    const int lane = threadIdx.x & 63;
    const float log_s = logf(a.s);
    const bool none = a.s == 0.f;  // every logit is -inf
    for (int i = lane; i < M; i += 64) {
        const int token = tokens[r * M + i];
        const bool in = token >= 0 && token < row.V;
        const float x = in ? row.one(token) : -INFINITY;
        logprob[r * M + i] = !in || none ? -INFINITY : x - a.m - log_s;
    }
    if (entropy && lane == 0)
        entropy[r] = none ? 0.f : fmaf(-kLn2, a.t / a.s, log_s);
    if (lane < k) {
        const float x = code_score((uint32_t)(key >> 32));
        top_tokens[r * k + lane] = key ? (int32_t)key_pos(key) : -1;
        top_logprobs[r * k + lane] = key ? x - a.m - log_s : -INFINITY;
    }
}

__device__ __forceinline__ void write_none(int64_t r, int M, int k, float* logprob, float* entropy,
                                           int32_t* top_tokens, float* top_logprobs)
{
    for (int i = threadIdx.x; i < M; i += (int)blockDim.x)
        logprob[r * M + i] = -INFINITY;
    if (entropy && threadIdx.x == 0)
        entropy[r] = 0.f;
    if ((int)threadIdx.x < k) {
        top_tokens[r * k + threadIdx.x] = -1;
        top_logprobs[r * k + threadIdx.x] = -INFINITY;
    }
}

struct Call {
    int64_t ld;
    int32_t V, max_rows, M, k, parts;
    const int32_t* n_rows;
    const int32_t* tokens;
    Sums* part;       // parts a row
    uint64_t* keys;   // k a part
    float *logprob, *entropy, *top_logprobs;
    int32_t* top_tokens;

    __device__ __forceinline__ bool none(int64_t r) const
    {
        return n_rows && (int)(r % max_rows) >= n_rows[r / max_rows];
    }
};

// One workgroup a (row, part); with one part the row's outputs, else its sums and keys.
template <typename X, int NT, bool kMany>
__global__ __launch_bounds__(NT) void logprobs_kernel(const X* __restrict__ logits, Call c)
{
    __shared__ Shared<NT> lds;
    const int64_t r = blockIdx.x / c.parts;
    const int p = blockIdx.x % c.parts, lane = threadIdx.x & 63;
    if (c.none(r)) {
        if (c.parts == 1)
            write_none(r, c.M, c.k, c.logprob, c.entropy, c.top_tokens, c.top_logprobs);
        return;
    }
    const Row<X> row(logits + r * c.ld, c.V);
    const int64_t all = row.loads(), per = (all + c.parts - 1) / c.parts;
    const int64_t g0 = p * per, g1 = g0 + per < all ? g0 + per : all;
    Sums a;
    uint64_t key;
    scan_part<X, NT, kMany>(row, g0, g1, c.k, lds, &a, &key);
    if (threadIdx.x >= 64)
        return;
    if (c.parts == 1) {
        write_row(row, r, a, key, c.tokens, c.M, c.k, c.logprob, c.entropy, c.top_tokens, c.top_logprobs);
        return;
    }
    if (lane == 0)
        c.part[r * c.parts + p] = a;
    if (lane < c.k)
        c.keys[(r * c.parts + p) * c.k + lane] = key;
}

// One wave a row; parts' lists by depth, so that what comes later seldom enters.
template <typename X>
__global__ __launch_bounds__(64) void logprobs_join_kernel(const X* __restrict__ logits, Call c)
{
    const int64_t r = blockIdx.x;
    const int lane = threadIdx.x;
    if (c.none(r)) {
        write_none(r, c.M, c.k, c.logprob, c.entropy, c.top_tokens, c.top_logprobs);
        return;
    }
    const Row<X> row(logits + r * c.ld, c.V);
    Best<true> best;
    for (int i = 0; i < c.parts * c.k; i += 64) {
        const int at = i + lane, depth = at / c.parts, p = at - depth * c.parts;
        best.add(at < c.parts * c.k ? c.keys[(r * c.parts + p) * c.k + depth] : 0ull, lane, c.k);
    }
    const Sums a = join_wave(lane < c.parts ? c.part[r * c.parts + lane] : Sums{kLowest, 0.f, 0.f});
    write_row(row, r, a, best.mine, c.tokens, c.M, c.k, c.logprob, c.entropy, c.top_tokens, c.top_logprobs);
}

constexpr int kThreads = 256, kWideThreads = 1024;  // of a workgroup
constexpr int64_t kFewBytes = 160 << 10;            // of a row that one wide workgroup reads

// Workgroups a row is cut among, 16 KiB each at least (a step of their loads): one where
// rows fill the chip with four a CU.
int32_t row_parts(int64_t rows, int32_t V, int size)
{
    const int64_t bytes = (int64_t)V * size, most = (bytes + (16 << 10) - 1) / (16 << 10), want = 1024 / rows;
    if (bytes <= kFewBytes && rows <= 512)
        return 1;
    const int64_t n = want < most ? want : most;
    return (int32_t)(n < 1 ? 1 : n > 64 ? 64 : n);
}

// Whether a row's one workgroup is wide: where rows leave CUs without one otherwise.
bool wide(int64_t rows, int32_t parts) { return parts == 1 && rows <= 512; }

}  // namespace

size_t logprobs_workspace_bytes(int64_t rows, int32_t V, int dtype, int32_t k)
{
    const int64_t parts = row_parts(rows, V, dtype == 0 ? 4 : 2);
    return parts == 1 ? 256 : (size_t)(rows * parts) * (8 * (size_t)k + sizeof(Sums)) + 256;
}

hipError_t launch_logprobs(int64_t rows, int32_t max_rows, const int32_t* n_rows, const void* logits, int dtype,
                           int32_t V, int64_t ld, const int32_t* tokens, int32_t M, int32_t k, void* workspace,
                           float* logprob, float* entropy, int32_t* top_tokens, float* top_logprobs,
                           hipStream_t stream)
{
    const int32_t parts = row_parts(rows, V, dtype == 0 ? 4 : 2);
    uint64_t* keys = (uint64_t*)workspace;
    const Call c = {ld,     V,    max_rows, M,       k,       parts,        n_rows,
                    tokens, (Sums*)(keys + rows * parts * k), keys, logprob, entropy, top_logprobs, top_tokens};
#define OIL_LOGPROBS_OF(X, NT, MANY)                                                                      \
    hipLaunchKernelGGL((logprobs_kernel<X, NT, MANY>), dim3((uint32_t)(rows * parts)), dim3(NT), 0, stream, \
                       (const X*)logits, c)
#define OIL_LOGPROBS(X)                             \
    if (wide(rows, parts) && k > kFewKeys)          \
        OIL_LOGPROBS_OF(X, kWideThreads, true);     \
    else if (wide(rows, parts))                     \
        OIL_LOGPROBS_OF(X, kWideThreads, false);    \
    else if (k > kFewKeys)                          \
        OIL_LOGPROBS_OF(X, kThreads, true);         \
    else                                            \
        OIL_LOGPROBS_OF(X, kThreads, false);        \
    if (parts > 1)                                  \
    hipLaunchKernelGGL(logprobs_join_kernel<X>, dim3((uint32_t)rows), dim3(64), 0, stream, (const X*)logits, c)
    if (dtype == 0) {
        OIL_LOGPROBS(float);
    } else {
        OIL_LOGPROBS(uint16_t);
    }
#undef OIL_LOGPROBS
#undef OIL_LOGPROBS_OF
    return hipGetLastError();
}

}  // namespace oil
