// Log probabilities of tokens from rows of logits, with the entropy and the most
// likely tokens.  Contract: include/oilbird.h.
//
// One pass over a row: with m the running maximum, y = (x - m) log2 e, a lane keeps
// s = sum 2^y and t = sum y 2^y, both rescaled when m rises.  Then
//     log p = (x - m) - ln s,      H = ln s - ln 2 t / s,
// where both terms of H are at least 0, so that nothing cancels.  The k best (logit
// descending, token ascending: one 64-bit key a token) are a list over the lanes of a
// wave, which a step of values enters only where some lane's largest reaches the
// list's last; waves of a workgroup share the highest such bound.  The first step's
// bound is the k-th largest of the lanes' own maxima.
//
// Where rows are few, a row is cut among workgroups, and a second launch joins.
#include "common.hpp"
#include "internal.hpp"

namespace oil {

namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kDeep = 4;  // loads of a lane in flight
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kLeast = -2000.f;  // below any y whose power of two is not 0
constexpr float kLowest = -3.4028234663852886e38f;

struct Sums {
    float m, s, t;
};

// What a workgroup found of its part of a row.
struct Part {
    Sums sums;
    float pad;
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

__device__ __forceinline__ Sums join_wave(Sums a)
{
#pragma unroll
    for (int o = 32; o; o >>= 1)
        a = join(a, Sums{__shfl_xor(a.m, o), __shfl_xor(a.s, o), __shfl_xor(a.t, o)});
    return a;
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

// The best k keys a wave has seen, best first by lane (0 past them).
struct Best {
    uint64_t mine = 0, last = 0;  // last: the k-th

    // Enters one key a lane; 0 enters nothing.
    __device__ __forceinline__ void add(uint64_t key, int lane, int k)
    {
        uint64_t who = __ballot(key > last);
        while (who) {
            const int from = __builtin_ctzll(who);
            const uint64_t x = lane_key(key, from);
            const int place = __popcll(__ballot(mine > x));
            const uint64_t up = __shfl_up((unsigned long long)mine, 1);
            mine = lane < place ? mine : lane == place ? x : up;
            last = lane_key(mine, k - 1);
            who &= ~(1ull << from) & __ballot(key > last);
        }
    }
};

// The k-th largest of the lanes' codes (0 where fewer lanes have one).
__device__ __forceinline__ uint32_t kth_code(uint32_t code, int k)
{
    uint32_t at = 0;
    for (int bit = 31; bit >= 0; bit--) {
        const uint32_t up = at | 1u << bit;
        if (__popcll(__ballot(code >= up)) >= k)
            at = up;
    }
    return at;
}

template <typename X>
struct Row {
    static constexpr int E = 16 / sizeof(X);  // values of a 16-byte load
    const X* x;
    int V, off;  // off: values before the row in its first 16 bytes

    __device__ __forceinline__ Row(const X* row, int v) : x(row), V(v), off((int)((uintptr_t)row % 16) / (int)sizeof(X)) {}
    __device__ __forceinline__ int64_t loads() const { return ((int64_t)V + off + E - 1) / E; }
    // The first token of load g.
    __device__ __forceinline__ int64_t token(int64_t g) const { return g * E - off; }
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
};

// The part [g0, g1) of a row's loads: the workgroup's sums (in thread 0) and, with k,
// its best k keys in lds_keys[0 .. k) (0 past them).
template <typename X>
__device__ __forceinline__ Sums scan_part(const Row<X>& row, int64_t g0, int64_t g1, int k, uint64_t* lds_keys,
                                          Sums* lds_sums, uint32_t* lds_bound)
{
    constexpr int E = Row<X>::E;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    Sums a = {kLowest, 0.f, 0.f};
    Best best;
    uint32_t bound = 0;  // code below which nothing enters
    if (threadIdx.x == 0)
        *lds_bound = 0;
    __syncthreads();
    bool begun = false;
    for (int64_t g = g0 + wave * (64 * kDeep); g < g1; g += kThreads * kDeep) {
        float x[kDeep][E];
        const bool whole = g + 64 * kDeep <= g1 && row.token(g) >= 0 && row.token(g + 64 * kDeep) <= row.V;
        if (whole) {
            u32x4 w[kDeep];
#pragma unroll
            for (int i = 0; i < kDeep; i++)
                w[i] = row.load(g + i * 64 + lane);
#pragma unroll
            for (int i = 0; i < kDeep; i++)
#pragma unroll
                for (int e = 0; e < E; e++)
                    x[i][e] = Row<X>::of(w[i], e);
        } else {
#pragma unroll
            for (int i = 0; i < kDeep; i++)
#pragma unroll
                for (int e = 0; e < E; e++) {
                    const int64_t at = g + i * 64 + lane, token = row.token(at) + e;
                    x[i][e] = at < g1 && token >= 0 && token < row.V ? row.one(token) : -INFINITY;
                }
        }
        float top[kDeep];
        float most = kLowest;
#pragma unroll
        for (int i = 0; i < kDeep; i++) {
            top[i] = x[i][0];
#pragma unroll
            for (int e = 1; e < E; e++)
                top[i] = fmaxf(top[i], x[i][e]);
            most = fmaxf(most, top[i]);
        }
        const float m = fmaxf(a.m, most);
        const float y = fmaxf((a.m - m) * kLog2e, kLeast), f = __builtin_amdgcn_exp2f(y);
        a.t = fmaf(y, a.s, a.t) * f;
        a.s *= f;
        a.m = m;
        float s[2] = {0.f, 0.f}, t[2] = {0.f, 0.f};
#pragma unroll
        for (int i = 0; i < kDeep; i++)
#pragma unroll
            for (int e = 0; e < E; e++) {
                const float z = (x[i][e] - m) * kLog2e, p = __builtin_amdgcn_exp2f(z);
                s[e & 1] += p;
                t[e & 1] = fmaf(fmaxf(z, kLeast), p, t[e & 1]);
            }
        a.s += s[0] + s[1];
        a.t += t[0] + t[1];
        if (k == 0)
            continue;
        uint32_t code = score_code(most);
        if (!begun) {
            begun = true;
            const uint32_t c = kth_code(code, k);
            bound = c > bound ? c : bound;
        }
        const uint32_t others = *(volatile uint32_t*)lds_bound;
        bound = others > bound ? others : bound;
        if (!__ballot(code >= bound))
            continue;
#pragma unroll
        for (int i = 0; i < kDeep; i++) {
            if (!__ballot(score_code(top[i]) >= bound))
                continue;
#pragma unroll
            for (int e = 0; e < E; e++) {
                const uint64_t key = token_key(x[i][e], (uint32_t)(row.token(g + i * 64 + lane) + e));
                best.add((uint32_t)(key >> 32) >= bound ? key : 0ull, lane, k);
            }
        }
        const uint32_t mine = (uint32_t)(best.last >> 32);
        if (mine > bound) {
            bound = mine;
            if (lane == 0)
                atomicMax(lds_bound, mine);
        }
    }
    a = join_wave(a);
    if (lane == 0)
        lds_sums[wave] = a;
    if (lane < k)
        lds_keys[wave * k + lane] = best.mine;
    __syncthreads();
    if (wave == 0) {
        for (int i = 1; i < kWaves; i++) {
            a = join(a, lds_sums[i]);
            if (k)
                best.add(lane < k ? lds_keys[i * k + lane] : 0ull, lane, k);
        }
        if (lane < k)
            lds_keys[lane] = best.mine;
    }
    return a;
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
        top_tokens[r * k + lane] = key ? (int32_t)key_pos(key) : -1;
        top_logprobs[r * k + lane] = key ? code_score((uint32_t)(key >> 32)) - a.m - log_s : -INFINITY;
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

// One workgroup a (row, part); with one part the row's outputs, else a Part and keys.
template <typename X>
__global__ __launch_bounds__(kThreads) void logprobs_kernel(const X* __restrict__ logits, int64_t ld, int32_t V,
                                                            int32_t max_rows, const int32_t* __restrict__ n_rows,
                                                            const int32_t* __restrict__ tokens, int32_t M, int32_t k,
                                                            int32_t parts, Part* __restrict__ part,
                                                            uint64_t* __restrict__ part_keys,
                                                            float* __restrict__ logprob, float* __restrict__ entropy,
                                                            int32_t* __restrict__ top_tokens,
                                                            float* __restrict__ top_logprobs)
{
    __shared__ uint64_t lds_keys[kWaves * OIL_TOPK_MAX];
    __shared__ Sums lds_sums[kWaves];
    __shared__ uint32_t lds_bound;
    const int64_t r = blockIdx.x / parts;
    const int p = blockIdx.x % parts, lane = threadIdx.x & 63;
    if (n_rows && (int)(r % max_rows) >= n_rows[r / max_rows]) {
        if (parts == 1)
            write_none(r, M, k, logprob, entropy, top_tokens, top_logprobs);
        return;
    }
    const Row<X> row(logits + r * ld, V);
    const int64_t all = row.loads(), per = (all + parts - 1) / parts;
    const int64_t g0 = p * per, g1 = g0 + per < all ? g0 + per : all;
    const Sums a = scan_part(row, g0, g1, k, lds_keys, lds_sums, &lds_bound);
    if (threadIdx.x >= 64)
        return;
    const uint64_t key = lane < k ? lds_keys[lane] : 0ull;
    if (parts == 1) {
        write_row(row, r, a, key, tokens, M, k, logprob, entropy, top_tokens, top_logprobs);
    } else {
        if (lane == 0)
            part[r * parts + p] = Part{a, 0.f};
        if (lane < k)
            part_keys[(r * parts + p) * k + lane] = key;
    }
}

// One wave a row.
template <typename X>
__global__ __launch_bounds__(64) void logprobs_join_kernel(const X* __restrict__ logits, int64_t ld, int32_t V,
                                                           int32_t max_rows, const int32_t* __restrict__ n_rows,
                                                           const int32_t* __restrict__ tokens, int32_t M, int32_t k,
                                                           int32_t parts, const Part* __restrict__ part,
                                                           const uint64_t* __restrict__ part_keys,
                                                           float* __restrict__ logprob, float* __restrict__ entropy,
                                                           int32_t* __restrict__ top_tokens,
                                                           float* __restrict__ top_logprobs)
{
    const int64_t r = blockIdx.x;
    const int lane = threadIdx.x;
    if (n_rows && (int)(r % max_rows) >= n_rows[r / max_rows]) {
        write_none(r, M, k, logprob, entropy, top_tokens, top_logprobs);
        return;
    }
    const Row<X> row(logits + r * ld, V);
    Sums a = {kLowest, 0.f, 0.f};
    for (int p = lane; p < parts; p += 64)
        a = join(a, part[r * parts + p].sums);
    a = join_wave(a);
    Best best;
    for (int i = 0; i < parts * k; i += 64)
        best.add(i + lane < parts * k ? part_keys[r * parts * k + i + lane] : 0ull, lane, k);
    write_row(row, r, a, best.mine, tokens, M, k, logprob, entropy, top_tokens, top_logprobs);
}

constexpr int64_t kWorkgroups = 2048;  // 8 a CU

// Workgroups a row of V logits is cut among where there are `rows` of them: as many as
// fill the chip, each with one step of its loads at least.
int32_t row_parts(int64_t rows, int32_t V, int size)
{
    const int64_t steps = ((int64_t)V * size / 16 + kThreads * kDeep) / (kThreads * kDeep);
    const int64_t want = (kWorkgroups + rows - 1) / rows;
    const int64_t n = want < steps ? want : steps;
    return (int32_t)(n < 1 ? 1 : n > 64 ? 64 : n);
}

}  // namespace

size_t logprobs_workspace_bytes(int64_t rows, int32_t V, int dtype, int32_t k)
{
    const int64_t parts = row_parts(rows, V, dtype == 0 ? 4 : 2);
    return parts == 1 ? 256 : (size_t)(rows * parts) * (sizeof(Part) + 8 * (size_t)k) + 256;
}

hipError_t launch_logprobs(int64_t rows, int32_t max_rows, const int32_t* n_rows, const void* logits, int dtype,
                           int32_t V, int64_t ld, const int32_t* tokens, int32_t M, int32_t k, void* workspace,
                           float* logprob, float* entropy, int32_t* top_tokens, float* top_logprobs,
                           hipStream_t stream)
{
    const int32_t parts = row_parts(rows, V, dtype == 0 ? 4 : 2);
    Part* part = (Part*)workspace;
    uint64_t* keys = (uint64_t*)(part + rows * parts);
#define OIL_LOGPROBS(X)                                                                                             \
    hipLaunchKernelGGL(logprobs_kernel<X>, dim3((uint32_t)(rows * parts)), dim3(kThreads), 0, stream,              \
                       (const X*)logits, ld, V, max_rows, n_rows, tokens, M, k, parts, part, keys, logprob, entropy, \
                       top_tokens, top_logprobs);                                                                  \
    if (parts > 1)                                                                                                 \
    hipLaunchKernelGGL(logprobs_join_kernel<X>, dim3((uint32_t)rows), dim3(64), 0, stream, (const X*)logits, ld, V, \
                       max_rows, n_rows, tokens, M, k, parts, part, keys, logprob, entropy, top_tokens, top_logprobs)
    if (dtype == 0) {
        OIL_LOGPROBS(float);
    } else {
        OIL_LOGPROBS(uint16_t);
    }
#undef OIL_LOGPROBS
    return hipGetLastError();
}

}  // namespace oil
