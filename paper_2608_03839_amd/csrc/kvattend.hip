// Attention over the verifier's 4-bit cache and the nodes of a draft tree, and
// the attention weight that committed rows give to cached positions.
#include "kv.hpp"

namespace oil {

namespace {

constexpr int kChunk = 256;

template <int W>
__device__ __forceinline__ float kv_key_dot(const uint8_t* tile, int key, const float* q)
{
    float dot = 0.f, sum = 0.f;
    for (int ks = 0; ks < W / 32; ks++)
        for (int g = 0; g < 4; g++) {
            const uint32_t w = ((const uint32_t*)tile)[kv_word_at((key >> 4) * (W / 32) + ks, (key & 15) + 16 * g)];
            for (int e = 0; e < 8; e++) {
                const float x = q[32 * ks + 8 * g + e];
                dot += x * (float)kv_code(w, e);
                sum += x;
            }
        }
    const uint32_t pair = *(const uint32_t*)(tile + KvTile<W>::kKeyScales + key * 4);
    return kv_s(pair) * dot + kv_z(pair) * sum;
}

template <int W>
__device__ __forceinline__ float kv_value_at(const uint8_t* tile, int key, int d)
{
    const uint32_t w = ((const uint32_t*)(tile + KvTile<W>::kValues))[kv_word_at(d >> 4, (d & 15) + 16 * ((key & 15) >> 2))];
    const uint32_t pair = *(const uint32_t*)(tile + KvTile<W>::kValueScales + key * 4);
    return kv_z(pair) + kv_s(pair) * (float)kv_code(w, 4 * (key >> 4) + (key & 3));
}

// One workgroup per row: chunks of 256 positions, a score a thread, then the
// values by column with the running maximum and sum of the softmax.
template <int W>
__global__ __launch_bounds__(256) void kv_attend_kernel(KvView c, const int32_t* __restrict__ slots,
                                                        const uint16_t* __restrict__ q, int64_t q_ld, int32_t Hq,
                                                        const uint16_t* __restrict__ k,
                                                        const uint16_t* __restrict__ v, int64_t ld,
                                                        const int32_t* __restrict__ n_nodes,
                                                        const uint32_t* __restrict__ mask, int32_t max_nodes,
                                                        float scale, uint16_t* __restrict__ out,
                                                        float* __restrict__ lse)
{
    __shared__ float qs[W], p[kChunk], red[8];
    __shared__ float half[W];
    const int a = blockIdx.x, i = blockIdx.y, b = blockIdx.z, tid = threadIdx.x;
    const int h = a / (Hq / c.H), D = c.D;
    const int slot = kv_slot(c, slots, b);
    int m = n_nodes ? n_nodes[b] : max_nodes;
    m = m < 0 ? 0 : m > max_nodes ? max_nodes : m;
    const bool live = slot >= 0 && i < m;
    const int32_t len = live ? kv_len(c, slot) : 0;
    const int extra = live && k ? m : 0;
    const int64_t row = ((int64_t)b * max_nodes + i) * q_ld + (int64_t)a * D;
    if (tid < W)
        qs[tid] = live && tid < D ? bf16_bits_to_float(q[row + tid]) : 0.f;
    __syncthreads();
    float top = -INFINITY, total = 0.f, acc = 0.f;
    const int d = tid % W, part = tid / W;  // column, and share of the chunk
    const uint8_t* tiles = slot < 0 ? nullptr : kv_tiles(c, slot, h);
    for (int64_t j0 = 0; j0 < (int64_t)len + extra; j0 += kChunk) {
        const int64_t j = j0 + tid;
        float s = -INFINITY;
        if (j < len) {
            s = scale * kv_key_dot<W>(tiles + j / kKvTile * c.tile_bytes, (int)(j % kKvTile), qs);
        } else if (j < (int64_t)len + extra) {
            const int u = (int)(j - len);
            const uint32_t* bits = mask ? mask + ((int64_t)b * max_nodes + i) * ((max_nodes + 31) / 32) : nullptr;
            if (bits ? (bits[u >> 5] >> (u & 31)) & 1 : u <= i) {
                const uint16_t* kr = k + ((int64_t)b * max_nodes + u) * ld + (int64_t)h * D;
                float dot = 0.f;
                for (int e = 0; e < D; e++)
                    dot += qs[e] * bf16_bits_to_float(kr[e]);
                s = scale * dot;
            }
        }
        float t = s;
        bool nan = s != s;
        for (int o = 32; o >= 1; o >>= 1)
            t = fmaxf(t, __shfl_xor(t, o, 64));
        if ((tid & 63) == 0)
            red[tid >> 6] = t;
        __syncthreads();
        const float m_new = fmaxf(fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3])), top);
        const float base = m_new == -INFINITY ? 0.f : m_new;
        float e = s == -INFINITY ? 0.f : nan ? s : expf(s - base);
        p[tid] = e;
        for (int o = 32; o >= 1; o >>= 1)
            e += __shfl_xor(e, o, 64);
        if ((tid & 63) == 0)
            red[4 + (tid >> 6)] = e;
        __syncthreads();
        const float fade = top == -INFINITY ? 0.f : expf(top - base);
        total = total * fade + (red[4] + red[5] + red[6] + red[7]);
        top = m_new;
        acc *= fade;
        for (int x = part; x < kChunk; x += 256 / W) {
            const int64_t jj = j0 + x;
            const float px = p[x];
            if (d >= D || px == 0.f)
                continue;
            if (jj < len)
                acc += px * kv_value_at<W>(tiles + jj / kKvTile * c.tile_bytes, (int)(jj % kKvTile), d);
            else if (jj < (int64_t)len + extra)
                acc += px * bf16_bits_to_float(v[((int64_t)b * max_nodes + (jj - len)) * ld + (int64_t)h * D + d]);
        }
        __syncthreads();
    }
    // the column's shares
    for (int s = 1; s < 256 / W; s++) {
        if (part == s)
            half[d] = acc;
        __syncthreads();
        if (part == 0)
            acc += half[d];
        __syncthreads();
    }
    const int64_t at = ((int64_t)b * max_nodes + i) * Hq + a;
    if (part == 0 && d < D)
        out[at * D + d] = total == 0.f ? (uint16_t)0 : float_to_bf16_rne(acc / total);
    if (tid == 0 && lse)
        lse[at] = total == 0.f ? -INFINITY : top + logf(total);
}

// One thread per position: every committed row's probability at it.
template <int W>
__global__ __launch_bounds__(256) void kv_weigh_kernel(KvView c, const int32_t* __restrict__ slots,
                                                       const uint16_t* __restrict__ q, int64_t q_ld, int32_t Hq,
                                                       const float* __restrict__ lse, int32_t max_nodes,
                                                       const int32_t* __restrict__ nodes,
                                                       const int32_t* __restrict__ count, float scale)
{
    __shared__ float qs[W];
    __shared__ int bound;
    const int b = blockIdx.z, h = blockIdx.y, tid = threadIdx.x, G = Hq / c.H;
    const int slot = kv_slot(c, slots, b);
    if (slot < 0)
        return;
    const int32_t len = kv_len(c, slot);
    const int rows = kv_count(nodes, count, b, max_nodes, &bound);
    const uint8_t* tiles = kv_tiles(c, slot, h);
    for (int64_t j0 = blockIdx.x * 256ll; j0 < len; j0 += gridDim.x * 256ll) {
        const int64_t j = j0 + tid;
        float sum = 0.f;
        for (int r = 0; r < rows; r++)
            for (int g = 0; g < G; g++) {
                const int64_t at = (int64_t)b * max_nodes + kv_source(nodes, b, max_nodes, r);
                __syncthreads();
                if (tid < W)
                    qs[tid] = tid < c.D ? bf16_bits_to_float(q[at * q_ld + (int64_t)(h * G + g) * c.D + tid]) : 0.f;
                __syncthreads();
                const float l = lse[at * Hq + h * G + g];
                if (j < len && l != -INFINITY)
                    sum += expf(scale * kv_key_dot<W>(tiles + j / kKvTile * c.tile_bytes, (int)(j % kKvTile), qs) - l);
            }
        if (j < len)
            c.weight[kv_row(c, slot, h) + j] += sum;
    }
}

}  // namespace

size_t kv_attend_workspace_bytes(const KvView&, int32_t, int32_t, int32_t) { return 256; }

hipError_t launch_kv_attend(const KvView& c, const int32_t* slots, int32_t B, const void* q, int64_t q_ld,
                            int32_t Hq, const void* k, const void* v, int64_t ld, const int32_t* n_nodes,
                            const uint32_t* mask, int32_t max_nodes, float scale, void*, void* out, float* lse,
                            hipStream_t stream)
{
    const dim3 grid(Hq, max_nodes, B);
#define OIL_KV_ATTEND(W)                                                                                          \
    hipLaunchKernelGGL(kv_attend_kernel<W>, grid, dim3(256), 0, stream, c, slots, (const uint16_t*)q, q_ld, Hq, \
                       (const uint16_t*)k, (const uint16_t*)v, ld, n_nodes, mask, max_nodes, scale,             \
                       (uint16_t*)out, lse)
    if (c.W == 64)
        OIL_KV_ATTEND(64);
    else
        OIL_KV_ATTEND(128);
#undef OIL_KV_ATTEND
    return hipGetLastError();
}

hipError_t launch_kv_weigh(const KvView& c, const int32_t* slots, int32_t B, const void* q, int64_t q_ld,
                           int32_t Hq, const float* lse, int32_t max_nodes, const int32_t* nodes,
                           const int32_t* count, float scale, hipStream_t stream)
{
    const int64_t blocks = (c.cap + 255) / 256;
    const dim3 grid((unsigned)(blocks < 4096 ? blocks : 4096), c.H, B);
#define OIL_KV_WEIGH(W)                                                                                            \
    hipLaunchKernelGGL(kv_weigh_kernel<W>, grid, dim3(256), 0, stream, c, slots, (const uint16_t*)q, q_ld, Hq, lse, \
                       max_nodes, nodes, count, scale)
    if (c.W == 64)
        OIL_KV_WEIGH(64);
    else
        OIL_KV_WEIGH(128);
#undef OIL_KV_WEIGH
    return hipGetLastError();
}

}  // namespace oil
