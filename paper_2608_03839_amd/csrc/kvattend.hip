// Attention over the verifier's 4-bit cache and the nodes of a draft tree, and
// the attention weight that committed rows give to cached positions.
//
// attend: a wave streams 32-position tiles of one head straight into registers
// in MFMA operand order and multiplies them with 16 NT rows (node, query head)
// at once: S^T = K Q^T puts a row's scores into one lane column, and the
// probabilities of a lane are, as they are, the operand of O^T = V^T P^T.  No
// tile passes through LDS and nothing in the loop waits for another wave.
//
// A code c of a 4-bit row enters the product as the binary16 subnormal c 2^-24
// (its nibble is the mantissa; the MFMA takes subnormals as they are) or, for
// every other pair, as 16 c 2^-24: eight codes cost four ANDs and a shift.
// Queries are scaled to binary16 by a power of two per row, so every product is
// exact and sums are binary32; z enters as z sum(q), and the values' z as
// sum(p z), both in binary32.
//
// The softmax keeps, per row, a reference m and sums relative to it (base 2).
// m moves only when a score passes it by 2^15, to 11 below the maximum: then
// p <= 2^15 fits binary16, and a p below 2^-32 of the largest is the first that
// rounds to nothing.  p times the value row's s, over a power of two E at or above every s
// so far, is what the second product takes, rounded to binary16 (2^-12
// relative).  z and s c may be far larger than the value they add up to, so that
// rounding must not reach s c alone: with one row tile a second operand takes
// what the first leaves (the product has time to spare there); with more, z is
// weighted by the rounded p (z / s times the operand).  Tiles in which some s is
// below a bound times E, where operands would lose bits, take two bf16 operands.
//
// The tree's nodes come as further tiles in bf16 (p rounded to 2^-9).
#include "kv.hpp"

namespace oil {

namespace {

typedef _Float16 h16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 h16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float floatx2 __attribute__((ext_vector_type(2)));

constexpr float kLog2e = 1.44269504088896341f, kLn2 = 0.693147180559945309f;
constexpr float kLow = -1e38f;      // m of a row that has seen nothing
constexpr float kHead = 11.f;       // the maximum's place above m
constexpr float kRoom = 15.f;       // and the most a score may pass m by

// How the rounding of a value operand is met (see the top), and the smallest
// s / E it is met by.
template <int NT>
struct KvRounding {
    static constexpr bool kTwo = NT == 1;
    static constexpr float kLeast = kTwo ? 0x1p-16f : 0x1p-6f;
};

struct KvAttend {
    KvView c;
    const int32_t* slots;
    const uint16_t* q;
    const uint16_t *k, *v;
    const int32_t* n_nodes;
    const uint32_t* mask;
    uint16_t* out;
    float* lse;
    int64_t* start;  // per request (and one past): units before it,
    int64_t* items;  // items before it,
    int64_t* shares; // (one word) shares the units are cut into;
    float* part_o;   // per cut of an item: unnormalised rows,
    float* part_ml;  // and each one's (m, sum)
    int64_t q_ld, ld;
    int32_t B, Hq, G, max_nodes;
    float scale;
};

union Frag {
    u32x4 w;
    h16x8 h;
    bf16x8 b;
};

// A dword's eight codes as binary16 subnormals: pairs 1 and 3 are 16 times too large.
__device__ __forceinline__ h16x8 kv_codes(uint32_t w)
{
    Frag f;
    const uint32_t x = w >> 8;
    f.w[0] = w & 0x000F000Fu;
    f.w[1] = w & 0x00F000F0u;
    f.w[2] = x & 0x000F000Fu;
    f.w[3] = x & 0x00F000F0u;
    return f.h;
}

__device__ __forceinline__ uint32_t pack_f16(float a, float b)
{
    const floatx2 x = {a, b};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(x, h16x2));
}

__device__ __forceinline__ uint32_t pack_bf16(float a, float b)
{
    const floatx2 x = {a, b};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(x, bf16x2));
}

// A dword's eight codes in bf16, without the factors.
__device__ __forceinline__ bf16x8 kv_codes_bf16(uint32_t w)
{
    Frag f;
#pragma unroll
    for (int p = 0; p < 4; p++)
        f.w[p] = pack_bf16((float)kv_code(w, 2 * p), (float)kv_code(w, 2 * p + 1));
    return f.b;
}

// A value beside its counterpart 32 (16) lanes away.
__device__ __forceinline__ void swap32(float x, float* a, float* b)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    *a = __uint_as_float(r[0]);
    *b = __uint_as_float(r[1]);
}
__device__ __forceinline__ void swap16(float x, float* a, float* b)
{
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    *a = __uint_as_float(r[0]);
    *b = __uint_as_float(r[1]);
}

// Over the four lanes that share lane % 16.
__device__ __forceinline__ float quad_max(float x)
{
    float a, b;
    swap16(x, &a, &b);
    swap32(fmaxf(a, b), &a, &b);
    return fmaxf(a, b);
}
__device__ __forceinline__ float quad_sum(float x)
{
    float a, b;
    swap16(x, &a, &b);
    swap32(a + b, &a, &b);
    return a + b;
}

// The largest of a wave.
__device__ __forceinline__ float wave_max(float x)
{
    x = quad_max(x);
    x = fmaxf(x, __uint_as_float(__builtin_amdgcn_ds_swizzle(__float_as_uint(x), 0x201F)));
    x = fmaxf(x, __uint_as_float(__builtin_amdgcn_ds_swizzle(__float_as_uint(x), 0x101F)));
    x = fmaxf(x, __uint_as_float(__builtin_amdgcn_ds_swizzle(__float_as_uint(x), 0x081F)));
    return fmaxf(x, __uint_as_float(__builtin_amdgcn_ds_swizzle(__float_as_uint(x), 0x041F)));
}

// Raw bf16 operand of a row for columns 32 ks + 8 g ..; zeros past D or for no row.
__device__ __forceinline__ u32x4 kv_raw(const uint16_t* row, int d, int D)
{
    u32x4 z = {0, 0, 0, 0};
    return row && d < D ? *(const u32x4*)(row + d) : z;
}

// Scaled binary16 operands of a row, and the factors of its scores in base 2:
// x = c1 (s dot) + c2 z.
template <int W>
__device__ __forceinline__ void kv_query(const uint16_t* row, int g, int D, float scale, Frag (&f)[W / 32], float* c1,
                                         float* c2)
{
    u32x4 raw[W / 32];
    uint32_t top = 0;
    float sum = 0.f;
#pragma unroll
    for (int ks = 0; ks < W / 32; ks++) {
        raw[ks] = kv_raw(row, 32 * ks + 8 * g, D);
#pragma unroll
        for (int j = 0; j < 4; j++) {
            const uint32_t lo = raw[ks][j] & 0x7FFFu, hi = (raw[ks][j] >> 16) & 0x7FFFu;
            top = max(top, max(lo, hi));
            sum += __uint_as_float(raw[ks][j] << 16) + __uint_as_float(raw[ks][j] & 0xFFFF0000u);
        }
    }
    top = (uint32_t)quad_max((float)top);
    const int e = max((int)(top >> 7) - 127, -112);
    const float by = __uint_as_float((uint32_t)(127 + 14 - e) << 23);  // the largest value to [2^14, 2^15)
#pragma unroll
    for (int ks = 0; ks < W / 32; ks++)
#pragma unroll
        for (int j = 0; j < 4; j++) {
            const float m = j & 1 ? by * 0.0625f : by;
            f[ks].w[j] = pack_f16(__uint_as_float(raw[ks][j] << 16) * m,
                                  __uint_as_float(raw[ks][j] & 0xFFFF0000u) * m);
        }
    *c1 = scale * kLog2e * __uint_as_float((uint32_t)min(127 + 24 - 14 + e, 254) << 23);
    *c2 = scale * kLog2e * quad_sum(sum);
}

// One tile of the cache in registers: its codes, and one (s, z) pair a lane (the
// keys' in lanes 0 .. 31, the values' in the others).
template <int W>
struct KvTileRegs {
    u32x4 k[W / 64], v[W / 64];
    uint32_t pair;

    __device__ __forceinline__ void load_keys(const uint8_t* tile, int lane)
    {
#pragma unroll
        for (int p = 0; p < W / 64; p++)
            k[p] = *(const u32x4*)(tile + p * 1024 + lane * 16);
        pair = *(const uint32_t*)(tile + KvTile<W>::kKeyScales + lane * 4);
    }
    __device__ __forceinline__ void load_values(const uint8_t* tile, int lane)
    {
#pragma unroll
        for (int p = 0; p < W / 64; p++)
            v[p] = *(const u32x4*)(tile + KvTile<W>::kValues + p * 1024 + lane * 16);
    }
    __device__ __forceinline__ uint32_t key_word(int Q) const { return k[Q >> 2][Q & 3]; }
    __device__ __forceinline__ uint32_t value_word(int Q) const { return v[Q >> 2][Q & 3]; }
};

// LDS of a wave for the scales of its tile: s of the 32 keys, the factors of the
// 32 value operands; then z of the keys, and what z of the values enters by.
struct KvScales {
    float s[64], z[64];
};

// The running state of a wave's 16 NT rows; a lane's column is row lane % 16 of
// each 16.
template <int W, int NT>
struct KvRows {
    floatx4 o[NT][W / 16];  // O^T / (E 2^24)
    float m[NT], l[NT], w[NT];
    float E;

    __device__ __forceinline__ void init()
    {
#pragma unroll
        for (int t = 0; t < NT; t++) {
            m[t] = kLow;
            l[t] = w[t] = 0.f;
#pragma unroll
            for (int mt = 0; mt < W / 16; mt++)
                o[t][mt] = floatx4{0.f, 0.f, 0.f, 0.f};
        }
        E = 0x1p-100f;
    }
    __device__ __forceinline__ void fade(int t, float by)
    {
        l[t] *= by;
        w[t] *= by;
#pragma unroll
        for (int mt = 0; mt < W / 16; mt++)
            o[t][mt] *= by;
    }
    // m of row t up to `top` (any lane's; the row's lanes agree afterwards).
    __device__ __forceinline__ void raise(int t, float top)
    {
        const float m_new = fmaxf(m[t], quad_max(top) - kHead);
        fade(t, __builtin_amdgcn_exp2f(m[t] - m_new));
        m[t] = m_new;
    }
    // E up to a power of two at or above `top` (any lane's).
    __device__ __forceinline__ void widen(float top)
    {
        top = wave_max(top);
        const float up = __uint_as_float((__float_as_uint(top) + 0x7FFFFFu) & 0x7F800000u);
        if (up > E) {
            const float by = E * (1.f / up);
#pragma unroll
            for (int t = 0; t < NT; t++)
#pragma unroll
                for (int mt = 0; mt < W / 16; mt++)
                    o[t][mt] *= by;
            E = up;
        }
    }
};

// A tile of `valid` cached positions (32, or fewer at the end of a slot).  Each
// lane prepares one pair; the eight of its rows' scores come back through LDS.
// The wave's next tile is loaded into the same registers, the keys when the first
// product has taken them, the values after the second.
template <int W, int NT, bool END>
__device__ __forceinline__ void kv_tile(KvTileRegs<W>& T, const uint8_t* next, int valid, int lane, KvScales& L,
                                        const u32x4 (*q)[W / 32][64], const float (&c1)[NT], const float (&c2)[NT],
                                        KvRows<W, NT>& R)
{
    constexpr bool kTwo = KvRounding<NT>::kTwo;
    const int g = lane >> 4;
    const bool on = !END || (lane & 31) < valid, value = lane >= 32;
    float s = on ? kv_s(T.pair) : 0.f, z = on ? kv_z(T.pair) : 0.f;
    if (__any(value && s > R.E))
        R.widen(value ? s : 0.f);
    const bool rare = __any(value && on && s < R.E * KvRounding<NT>::kLeast);
    if (value) {
        const float by = 1.f / R.E;
        s *= lane & 2 ? by * 0.0625f : by;
        if (!kTwo && !rare)
            z = on ? z * __builtin_amdgcn_rcpf(s) : 0.f;
    }
    L.s[lane] = s;
    L.z[lane] = z;
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    asm volatile("" ::: "memory");  // the queries are read from LDS tile by tile: their registers are wanted
    floatx4 S[NT][2];
#pragma unroll
    for (int t = 0; t < NT; t++)
        S[t][0] = S[t][1] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int s = 0; s < W / 32; s++) {
        const h16x8 k0 = kv_codes(T.key_word(s)), k1 = kv_codes(T.key_word(W / 32 + s));
#pragma unroll
        for (int t = 0; t < NT; t++) {
            Frag qf;
            qf.w = q[t][s][lane];
            S[t][0] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k0, qf.h, S[t][0], 0, 0, 0);
            S[t][1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k1, qf.h, S[t][1], 0, 0, 0);
        }
    }
    if (!END)
        T.load_keys(next, lane);
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    float ks[8], kz[8], vs[8], vz[8];
    bool in[8];
#pragma unroll
    for (int a = 0; a < 2; a++) {
        const floatx4 x0 = *(const floatx4*)&L.s[16 * a + 4 * g], x1 = *(const floatx4*)&L.z[16 * a + 4 * g];
        const floatx4 x2 = *(const floatx4*)&L.s[32 + 16 * a + 4 * g], x3 = *(const floatx4*)&L.z[32 + 16 * a + 4 * g];
#pragma unroll
        for (int i = 0; i < 4; i++) {
            ks[4 * a + i] = x0[i];
            kz[4 * a + i] = x1[i];
            vs[4 * a + i] = x2[i];
            vz[4 * a + i] = x3[i];
            in[4 * a + i] = !END || 16 * a + 4 * g + i < valid;
        }
    }
    __builtin_amdgcn_wave_barrier();
    Frag p[NT], low[kTwo ? NT : 1];  // low: what the first operands leave
#pragma unroll
    for (int t = 0; t < NT; t++) {
        float x[8];
        float top = -INFINITY;
#pragma unroll
        for (int e = 0; e < 8; e++) {
            x[e] = fmaf(ks[e] * S[t][e >> 2][e & 3], c1[t], fmaf(kz[e], c2[t], -R.m[t]));
            if (END)
                x[e] = in[e] ? x[e] : -INFINITY;
            top = fmaxf(top, x[e]);
        }
        if (__any(top > kRoom)) {
            top = -INFINITY;
#pragma unroll
            for (int e = 0; e < 8; e++) {
                x[e] = fmaf(ks[e] * S[t][e >> 2][e & 3], c1[t], kz[e] * c2[t]);
                if (END)
                    x[e] = in[e] ? x[e] : -INFINITY;
                top = fmaxf(top, x[e]);
            }
            R.raise(t, top);
#pragma unroll
            for (int e = 0; e < 8; e++)
                x[e] = fmaf(ks[e] * S[t][e >> 2][e & 3], c1[t], fmaf(kz[e], c2[t], -R.m[t]));
            if (END)
#pragma unroll
                for (int e = 0; e < 8; e++)
                    x[e] = in[e] ? x[e] : -INFINITY;
        }
#pragma unroll
        for (int e = 0; e < 8; e++) {
            x[e] = __builtin_amdgcn_exp2f(x[e]);
            R.l[t] += x[e];
            if (kTwo || rare)
                R.w[t] = fmaf(x[e], vz[e], R.w[t]);
            x[e] *= vs[e];
        }
        if (rare) {
#pragma unroll
            for (int e = 0; e < 8; e++)
                x[e] *= e & 2 ? 0x1p-20f : 0x1p-24f;
#pragma unroll
            for (int j = 0; j < 4; j++) {
                p[t].w[j] = pack_bf16(x[2 * j], x[2 * j + 1]);
                low[0].w[j] = pack_bf16(x[2 * j] - __uint_as_float(p[t].w[j] << 16),
                                        x[2 * j + 1] - __uint_as_float(p[t].w[j] & 0xFFFF0000u));
            }
#pragma unroll
            for (int mt = 0; mt < W / 16; mt++) {
                const bf16x8 vf = kv_codes_bf16(T.value_word(mt));
                R.o[t][mt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, low[0].b, R.o[t][mt], 0, 0, 0);
                R.o[t][mt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, p[t].b, R.o[t][mt], 0, 0, 0);
            }
        } else {
#pragma unroll
            for (int j = 0; j < 4; j++)
                p[t].w[j] = pack_f16(x[2 * j], x[2 * j + 1]);
            if (kTwo) {
#pragma unroll
                for (int j = 0; j < 4; j++)
                    low[t].w[j] = pack_f16(x[2 * j] - (float)p[t].h[2 * j], x[2 * j + 1] - (float)p[t].h[2 * j + 1]);
            } else {
#pragma unroll
                for (int e = 0; e < 8; e++)
                    R.w[t] = fmaf((float)p[t].h[e], vz[e], R.w[t]);
            }
        }
    }
    if (!rare) {
#pragma unroll
        for (int mt = 0; mt < W / 16; mt++) {
            const h16x8 vf = kv_codes(T.value_word(mt));
#pragma unroll
            for (int t = 0; t < NT; t++) {
                if (kTwo)
                    R.o[t][mt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vf, low[t].h, R.o[t][mt], 0, 0, 0);
                R.o[t][mt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vf, p[t].h, R.o[t][mt], 0, 0, 0);
            }
        }
    }
    if (!END)
        T.load_values(next, lane);
}

// The node of row r of a head, -1 for none, and the row's queries.
__device__ __forceinline__ int kv_row_of(const KvAttend& A, int b, int h, int m, int r, const uint16_t** row)
{
    if (r >= m * A.G) {
        *row = nullptr;
        return -1;
    }
    const int node = r / A.G;
    *row = A.q + ((int64_t)b * A.max_nodes + node) * A.q_ld + (int64_t)(h * A.G + r - node * A.G) * A.c.D;
    return node;
}

// A tile of the tree: nodes n0 .. n0 + 31 of m, for rows r0 ...
template <int W, int NT>
__device__ __forceinline__ void kv_nodes(const KvAttend& A, int b, int h, int n0, int m, int lane, int r0,
                                         KvRows<W, NT>& R)
{
    const int g = lane >> 4, r = lane & 15, D = A.c.D;
    int node[NT];
    const uint16_t* row[NT];
#pragma unroll
    for (int t = 0; t < NT; t++)
        node[t] = kv_row_of(A, b, h, m, r0 + 16 * t + r, &row[t]);
    uint32_t sees[NT], any = 0;
    const uint32_t live = m - n0 >= 32 ? 0xFFFFFFFFu : (1u << (m - n0)) - 1;
#pragma unroll
    for (int t = 0; t < NT; t++) {
        sees[t] = 0;
        if (node[t] >= 0) {
            if (A.mask)
                sees[t] = A.mask[((int64_t)b * A.max_nodes + node[t]) * ((A.max_nodes + 31) / 32) + n0 / 32] & live;
            else if (node[t] >= n0)
                sees[t] = (node[t] - n0 >= 31 ? 0xFFFFFFFFu : (2u << (node[t] - n0)) - 1) & live;
        }
        any |= sees[t];
    }
    if (!__any(any != 0))
        return;
    const int64_t base = ((int64_t)b * A.max_nodes + n0) * A.ld + (int64_t)h * D;
    if (R.E < 1.f)
        R.widen(1.f);
    const float by = 0x1p-24f / R.E;
    floatx4 S[NT][2];
#pragma unroll
    for (int t = 0; t < NT; t++)
        S[t][0] = S[t][1] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int s = 0; s < W / 32; s++) {
        Frag kf[2];
#pragma unroll
        for (int a = 0; a < 2; a++)
            kf[a].w = kv_raw(n0 + 16 * a + r < m ? A.k + base + (int64_t)(16 * a + r) * A.ld : nullptr,
                             32 * s + 8 * g, D);
#pragma unroll
        for (int t = 0; t < NT; t++) {
            Frag qf;
            qf.w = kv_raw(row[t], 32 * s + 8 * g, D);
#pragma unroll
            for (int a = 0; a < 2; a++)
                S[t][a] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[a].b, qf.b, S[t][a], 0, 0, 0);
        }
    }
    Frag p[NT];
#pragma unroll
    for (int t = 0; t < NT; t++) {
        float x[8], top = -INFINITY;
#pragma unroll
        for (int e = 0; e < 8; e++) {
            const bool on = (sees[t] >> (16 * (e >> 2) + 4 * g + (e & 3))) & 1;
            x[e] = on ? S[t][e >> 2][e & 3] * (A.scale * kLog2e) : -INFINITY;
            top = fmaxf(top, x[e]);
        }
        if (__any(top - R.m[t] > kRoom))
            R.raise(t, top);
#pragma unroll
        for (int e = 0; e < 8; e++) {
            x[e] = __builtin_amdgcn_exp2f(x[e] - R.m[t]);
            R.l[t] += x[e];
            x[e] *= by;
        }
#pragma unroll
        for (int j = 0; j < 4; j++)
            p[t].w[j] = pack_bf16(x[2 * j], x[2 * j + 1]);
    }
    bool odd = false;
#pragma unroll
    for (int mt = 0; mt < W / 16; mt++) {
        const int d = 16 * mt + r;
        Frag vf;
#pragma unroll
        for (int j = 0; j < 4; j++) {
            uint32_t two = 0;
#pragma unroll
            for (int x = 0; x < 2; x++) {
                const int e = 2 * j + x, key = 16 * (e >> 2) + 4 * g + (e & 3);
                uint32_t u = n0 + key < m && d < D ? A.v[base + (int64_t)key * A.ld + d] : 0;
                if ((u & 0x7F80u) == 0x7F80u) {  // not finite: added below, to the rows that see it
                    odd = true;
                    u = 0;
                }
                two |= u << (16 * x);
            }
            vf.w[j] = two;
        }
#pragma unroll
        for (int t = 0; t < NT; t++)
            R.o[t][mt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf.b, p[t].b, R.o[t][mt], 0, 0, 0);
    }
    if (__any(odd)) {
        for (int key = 0; key < 32 && n0 + key < m; key++)
#pragma unroll
            for (int mt = 0; mt < W / 16; mt++)
#pragma unroll
                for (int i = 0; i < 4; i++) {
                    const int d = 16 * mt + 4 * g + i;
                    const uint32_t u = d < D ? A.v[base + (int64_t)key * A.ld + d] : 0;
                    if ((u & 0x7F80u) == 0x7F80u)
#pragma unroll
                        for (int t = 0; t < NT; t++)
                            if ((sees[t] >> key) & 1)
                                R.o[t][mt][i] += bf16_bits_to_float(u);
                }
    }
}

constexpr int kAttendWaves = 4;
constexpr int kMaxB = 512;

__device__ __forceinline__ int kv_live_nodes(const KvAttend& A, int b, int slot)
{
    if (slot < 0)
        return 0;
    const int m = A.n_nodes ? A.n_nodes[b] : A.max_nodes;
    return m < 0 ? 0 : m > A.max_nodes ? A.max_nodes : m;
}

// Tiles that a live row of a request goes through: the cache's, then the tree's.
__device__ __forceinline__ int64_t kv_units(const KvAttend& A, int32_t len, int m)
{
    return ((int64_t)len + kKvTile - 1) / kKvTile + (A.k ? (m + 31) / 32 : 0);
}

// The work of a call is one list of units: requests, in each its heads, in each
// its blocks of 16 NT rows (an item), in each the tiles.  Equal shares of it go
// to the workgroups, whatever the lengths; a share that begins or ends inside an
// item leaves a part of it, numbered share + item (which no two parts have in
// common), for the join.
// Least units of a share: two tiles a wave.
constexpr int64_t kLeastShare = 2 * kAttendWaves;

// A value that all lanes hold alike, as a scalar.
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ int64_t uniform(int64_t x)
{
    return (int64_t)((uint64_t)(uint32_t)uniform((int)(x >> 32)) << 32 | (uint32_t)uniform((int)x));
}

__device__ __forceinline__ int64_t kv_cut(int64_t total, int64_t shares, int64_t w)
{
    return total / shares * w + (total % shares) * w / shares;
}

template <int W, int NT>
__global__ __launch_bounds__(256, NT == 1 ? 3 : 2) void kv_attend_kernel(KvAttend A)
{
    constexpr int kRows = 16 * NT;
    __shared__ int64_t start[kMaxB + 1], items[kMaxB + 1];
    __shared__ int64_t sums[2][kAttendWaves];
    __shared__ float sm[kAttendWaves][kRows], sl[kAttendWaves][kRows];
    __shared__ floatx4 so[kAttendWaves / 2][NT][W / 16][64];
    __shared__ u32x4 sq[NT][W / 32][64];
    __shared__ __align__(16) KvScales scales[kAttendWaves];
    const int lane0 = threadIdx.x & 63, wave = uniform((int)(threadIdx.x >> 6)), D = A.c.D;
    // units and items before each request
    int64_t before[2] = {0, 0};
    for (int b0 = 0; b0 < A.B; b0 += 256) {
        const int b = b0 + (int)threadIdx.x;
        int64_t x[2] = {0, 0};
        if (b < A.B) {
            const int slot = kv_slot(A.c, A.slots, b), m = kv_live_nodes(A, b, slot);
            x[1] = (int64_t)A.c.H * ((m * A.G + kRows - 1) / kRows);
            x[0] = m ? x[1] * kv_units(A, kv_len(A.c, slot), m) : 0;
        }
#pragma unroll
        for (int y = 0; y < 2; y++) {
            int64_t run = x[y];
#pragma unroll
            for (int o = 1; o < 64; o <<= 1) {
                const int64_t z = __shfl_up(run, o, 64);
                run += lane0 >= o ? z : 0;
            }
            if (lane0 == 63)
                sums[y][wave] = run;
            x[y] = run;
        }
        __syncthreads();
#pragma unroll
        for (int y = 0; y < 2; y++) {
            int64_t all = 0, mine = before[y];
            for (int w = 0; w < kAttendWaves; w++) {
                mine += w < wave ? sums[y][w] : 0;
                all += sums[y][w];
            }
            if (b < A.B)
                (y ? items : start)[b + 1] = mine + x[y];
            before[y] += all;
        }
        __syncthreads();
    }
    if (threadIdx.x == 0)
        start[0] = items[0] = 0;
    __syncthreads();
    const int64_t total = uniform(before[0]), most = (total + kLeastShare - 1) / kLeastShare;
    const int64_t shares = most < 1 ? 1 : most < gridDim.x ? most : gridDim.x;
    if (blockIdx.x == 0) {
        for (int b = threadIdx.x; b <= A.B; b += 256) {
            A.start[b] = start[b];
            A.items[b] = items[b];
        }
        if (threadIdx.x == 0)
            *A.shares = shares;
    }
    // neighbouring shares on one XCD: the row blocks of a head read the same tiles
    const int64_t per_xcd = (shares + 7) / 8, share = (int64_t)(blockIdx.x & 7) * per_xcd + (blockIdx.x >> 3);
    if ((int64_t)(blockIdx.x >> 3) >= per_xcd || share >= shares)
        return;
    int64_t at = kv_cut(total, shares, share);
    const int64_t end = kv_cut(total, shares, share + 1);
    int b = 0;
    for (int hi = A.B; hi - b > 1;) {  // the last request that begins at or before `at`
        const int mid = (b + hi) >> 1;
        if (uniform(start[mid]) <= at)
            b = mid;
        else
            hi = mid;
    }
    while (at < end) {
        // what follows from the lane is worked out anew for each item: kept over all
        // of them it would take the registers that the tiles need
        int lane = lane0;
        asm volatile("" : "+v"(lane));
        const int r16 = lane & 15, g = lane >> 4;
        while (uniform(start[b + 1]) <= at)
            b++;
        const int slot = uniform(kv_slot(A.c, A.slots, b)), m = uniform(kv_live_nodes(A, b, slot));
        const int32_t len = uniform(kv_len(A.c, slot));
        const int64_t begin = uniform(start[b]);
        const int64_t cached = ((int64_t)len + kKvTile - 1) / kKvTile, units = kv_units(A, len, m);
        const int64_t item = (at - begin) / units, row_blocks = (m * A.G + kRows - 1) / kRows;
        const int h = (int)(item / row_blocks), rb = (int)(item % row_blocks);
        const int64_t u0 = at - begin - item * units;
        const int64_t u1 = end - at < units - u0 ? u0 + (end - at) : units;
        const bool whole = u0 == 0 && u1 == units;
        const int64_t part = share + uniform(items[b]) + item;
        at += u1 - u0;
        float c1[NT], c2[NT];
#pragma unroll
        for (int t = 0; t < NT; t++) {
            Frag q[W / 32];
            const uint16_t* row;
            kv_row_of(A, b, h, m, rb * kRows + 16 * t + r16, &row);
            kv_query<W>(row, g, D, A.scale, q, &c1[t], &c2[t]);
            if (wave == 0)
#pragma unroll
                for (int s = 0; s < W / 32; s++)
                    sq[t][s][lane] = q[s].w;
        }
        __syncthreads();
        KvRows<W, NT> R;
        R.init();
        const uint8_t* tiles = kv_tiles(A.c, slot, h);
        const int64_t last = cached < u1 ? cached : u1, full = len / kKvTile < last ? len / kKvTile : last;
        int64_t u = u0 + wave;
        if (u < last) {
            KvTileRegs<W> T;
            T.load_keys(tiles + u * KvTile<W>::kBytes, lane);
            T.load_values(tiles + u * KvTile<W>::kBytes, lane);
            for (; u < full; u += kAttendWaves) {
                const int64_t next = u + kAttendWaves < last ? u + kAttendWaves : u;
                kv_tile<W, NT, false>(T, tiles + next * KvTile<W>::kBytes, 32, lane, scales[wave], sq, c1, c2, R);
            }
            if (u < last) {  // the slot's last tile, with fewer than 32 positions
                kv_tile<W, NT, true>(T, nullptr, (int)(len - u * kKvTile), lane, scales[wave], sq, c1, c2, R);
                u += kAttendWaves;
            }
        }
        for (; u < u1; u += kAttendWaves)
            kv_nodes<W, NT>(A, b, h, (int)(u - cached) * 32, m, lane, rb * kRows, R);
        // the waves' shares, relative to the largest m
#pragma unroll
        for (int t = 0; t < NT; t++) {
            R.l[t] = quad_sum(R.l[t]);
            R.w[t] = quad_sum(R.w[t]);
            if (g == 0) {
                sm[wave][16 * t + r16] = R.m[t];
                sl[wave][16 * t + r16] = R.l[t];
            }
        }
        __syncthreads();
        float top[NT], sum[NT];
#pragma unroll
        for (int t = 0; t < NT; t++) {
            top[t] = kLow;
#pragma unroll
            for (int x = 0; x < kAttendWaves; x++)
                top[t] = fmaxf(top[t], sm[x][16 * t + r16]);
            sum[t] = 0.f;
#pragma unroll
            for (int x = 0; x < kAttendWaves; x++)
                sum[t] += sl[x][16 * t + r16] * __builtin_amdgcn_exp2f(sm[x][16 * t + r16] - top[t]);
            const float f = __builtin_amdgcn_exp2f(R.m[t] - top[t]), of = R.E * 0x1p24f;
#pragma unroll
            for (int mt = 0; mt < W / 16; mt++)
#pragma unroll
                for (int i = 0; i < 4; i++)
                    R.o[t][mt][i] = R.l[t] == 0.f ? 0.f : fmaf(R.o[t][mt][i], of, R.w[t]) * f;
        }
#pragma unroll
        for (int half = kAttendWaves / 2; half >= 1; half >>= 1) {
            if (wave >= half && wave < 2 * half)
#pragma unroll
                for (int t = 0; t < NT; t++)
#pragma unroll
                    for (int mt = 0; mt < W / 16; mt++)
                        so[wave - half][t][mt][lane] = R.o[t][mt];
            __syncthreads();
            if (wave < half)
#pragma unroll
                for (int t = 0; t < NT; t++)
#pragma unroll
                    for (int mt = 0; mt < W / 16; mt++)
                        R.o[t][mt] += so[wave][t][mt][lane];
            __syncthreads();
        }
        if (wave != 0)
            continue;
#pragma unroll
        for (int t = 0; t < NT; t++) {
            const int r = rb * kRows + 16 * t + r16;
            if (r >= m * A.G)
                continue;
            if (!whole) {
                const int64_t to = part * kRows + 16 * t + r16;
                if (g == 0)
                    ((floatx2*)A.part_ml)[to] = floatx2{top[t], sum[t]};
#pragma unroll
                for (int mt = 0; mt < W / 16; mt++)
                    *(floatx4*)(A.part_o + to * W + 16 * mt + 4 * g) = R.o[t][mt];
            } else {
                const int node = r / A.G;
                const int64_t to = ((int64_t)b * A.max_nodes + node) * A.Hq + h * A.G + (r - node * A.G);
                const bool none = sum[t] == 0.f;
                const float by = none ? 0.f : 1.f / sum[t];
                if (g == 0 && A.lse)
                    A.lse[to] = none ? -INFINITY : kLn2 * (top[t] + __builtin_amdgcn_logf(sum[t]));
#pragma unroll
                for (int mt = 0; mt < W / 16; mt++)
                    if (16 * mt + 4 * g < D) {
                        uint2 o;
                        o.x = none ? 0u : pack_bf16(R.o[t][mt][0] * by, R.o[t][mt][1] * by);
                        o.y = none ? 0u : pack_bf16(R.o[t][mt][2] * by, R.o[t][mt][3] * by);
                        *(uint2*)(A.out + to * D + 16 * mt + 4 * g) = o;
                    }
            }
        }
    }
}

// The parts of a row joined, by WR waves (4, or 1 where an item has few parts);
// rows that no share covered whole, and rows that see nothing.
constexpr int kMaxShares = 768;

template <int W, int WR>
__global__ __launch_bounds__(256) void kv_join_kernel(KvAttend A, int kRows)
{
    __shared__ float f[4 / WR][kMaxShares];
    __shared__ float red[2][4];
    __shared__ floatx2 so[4][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, b = blockIdx.z, h = blockIdx.y, D = A.c.D;
    const int mine = WR == 4 ? 0 : wave, r = blockIdx.x * (4 / WR) + mine;
    if (r >= A.max_nodes * A.G)
        return;
    const int slot = kv_slot(A.c, A.slots, b), m = kv_live_nodes(A, b, slot);
    const int node = r / A.G, d = W == 128 ? 2 * lane : lane;
    const int64_t to = ((int64_t)b * A.max_nodes + node) * A.Hq + h * A.G + (r - node * A.G);
    float total = 0.f, top = kLow;
    floatx2 o = {0.f, 0.f};
    if (r < m * A.G) {
        const int64_t row_blocks = (m * A.G + kRows - 1) / kRows, in_b = h * row_blocks + r / kRows;
        const int64_t item = A.items[b] + in_b, all = A.start[A.B], shares = *A.shares;
        const int64_t units = (A.start[b + 1] - A.start[b]) / (A.items[b + 1] - A.items[b]);
        const int64_t g0 = A.start[b] + in_b * units, g1 = g0 + units;
        if (units > 0) {
            // the shares that hold g0 and g1 - 1
            int64_t w0 = (int64_t)((double)g0 * (double)shares / (double)all);
            int64_t w1 = (int64_t)((double)(g1 - 1) * (double)shares / (double)all);
            w0 = w0 < shares ? w0 : shares - 1;
            w1 = w1 < shares ? w1 : shares - 1;
            while (kv_cut(all, shares, w0) > g0)
                w0--;
            while (kv_cut(all, shares, w0 + 1) <= g0)
                w0++;
            while (kv_cut(all, shares, w1) > g1 - 1)
                w1--;
            while (kv_cut(all, shares, w1 + 1) <= g1 - 1)
                w1++;
            if (w0 == w1)
                return;  // one share wrote the row
            const int parts = (int)(w1 - w0) + 1;
            const int64_t first = (w0 + item) * kRows + r % kRows;  // parts are kRows apart
            const floatx2* ml = (const floatx2*)A.part_ml;
            const int t0 = WR == 4 ? threadIdx.x : lane, dt = 64 * WR;
            for (int p = t0; p < parts; p += dt)
                top = fmaxf(top, ml[first + (int64_t)p * kRows][0]);
            top = wave_max(top);
            if (WR == 4) {
                if (lane == 0)
                    red[0][wave] = top;
                __syncthreads();
                top = fmaxf(fmaxf(red[0][0], red[0][1]), fmaxf(red[0][2], red[0][3]));
            }
            for (int p = t0; p < parts; p += dt) {
                const floatx2 x = ml[first + (int64_t)p * kRows];
                const float by = x[1] == 0.f ? 0.f : __builtin_amdgcn_exp2f(x[0] - top);
                f[mine][p] = by;
                total += x[1] * by;
            }
#pragma unroll
            for (int x = 1; x < 64; x <<= 1)
                total += __shfl_xor(total, x, 64);
            if (WR == 4) {
                if (lane == 0)
                    red[1][wave] = total;
                __syncthreads();
                total = red[1][0] + red[1][1] + red[1][2] + red[1][3];
            }
#pragma unroll 8
            for (int p = WR == 4 ? wave : 0; p < parts; p += WR) {
                const float by = f[mine][p];
                const float* from = A.part_o + (first + (int64_t)p * kRows) * W + d;
                if (W == 128) {
                    const floatx2 x = *(const floatx2*)from;
                    o[0] = by == 0.f ? o[0] : fmaf(by, x[0], o[0]);
                    o[1] = by == 0.f ? o[1] : fmaf(by, x[1], o[1]);
                } else {
                    o[0] = by == 0.f ? o[0] : fmaf(by, from[0], o[0]);
                }
            }
            if (WR == 4) {
                so[wave][lane] = o;
                __syncthreads();
                if (wave != 0)
                    return;
#pragma unroll
                for (int w = 1; w < 4; w++)
                    o += so[w][lane];
            }
        }
    }
    if (WR == 4 && wave != 0)
        return;
    const bool none = total == 0.f;
    const float by = none ? 0.f : 1.f / total;
    if (d < D) {
        if (W == 128)
            *(uint32_t*)(A.out + to * D + d) = none ? 0u : pack_bf16(o[0] * by, o[1] * by);
        else
            A.out[to * D + d] = none ? (uint16_t)0 : (uint16_t)pack_bf16(o[0] * by, 0.f);
    }
    if (lane == 0 && A.lse)
        A.lse[to] = none ? -INFINITY : kLn2 * (top + __builtin_amdgcn_logf(total));
}

// A workgroup's waves stream tiles of keys; up to 64 rows at a time stand in LDS
// as operands.  S = Q K^T puts a position into a lane column, so a position's sum
// over rows is over a lane's registers and four lanes.  ONE: at most 16 rows,
// whose operands stay in registers.
template <int W, bool ONE>
__global__ __launch_bounds__(256) void kv_weigh_kernel(KvView c, const int32_t* __restrict__ slots,
                                                       const uint16_t* __restrict__ q, int64_t q_ld, int32_t Hq,
                                                       const float* __restrict__ lse, int32_t max_nodes,
                                                       const int32_t* __restrict__ nodes,
                                                       const int32_t* __restrict__ count, float scale)
{
    constexpr int kTiles = ONE ? 1 : 4;
    __shared__ u32x4 sq[kTiles][W / 32][64];
    __shared__ floatx4 sc[kTiles][3][4];  // c1, c2 and lse (base 2) of a tile's rows
    __shared__ int bound, some;
    const int b = blockIdx.z, h = blockIdx.y, G = Hq / c.H;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r16 = lane & 15, g = lane >> 4;
    const int slot = kv_slot(c, slots, b);
    if (slot < 0)
        return;
    const int32_t len = kv_len(c, slot);
    const int64_t u0 = (int64_t)blockIdx.x * 4 + wave, du = (int64_t)gridDim.x * 4;
    const int64_t units = ((int64_t)len + kKvTile - 1) / kKvTile;
    if ((int64_t)blockIdx.x * 4 >= units)
        return;
    const int rows = kv_count(nodes, count, b, max_nodes, &bound) * G;
    const uint8_t* tiles = kv_tiles(c, slot, h);
    float* weight = c.weight + kv_row(c, slot, h);
    for (int r0 = 0; r0 < rows; r0 += 16 * kTiles) {
        __syncthreads();
        if (threadIdx.x == 0)
            some = 0;
        __syncthreads();
        if (wave < kTiles) {
            const int r = r0 + 16 * wave + r16;
            const uint16_t* row = nullptr;
            float l = -INFINITY;
            if (r < rows) {
                const int64_t at = (int64_t)b * max_nodes + kv_source(nodes, b, max_nodes, r / G);
                l = lse[at * Hq + h * G + r % G];
                if (l != -INFINITY)
                    row = q + at * q_ld + (int64_t)(h * G + r % G) * c.D;
            }
            Frag f[W / 32];
            float c1, c2;
            kv_query<W>(row, g, c.D, scale, f, &c1, &c2);
#pragma unroll
            for (int s = 0; s < W / 32; s++)
                sq[wave][s][lane] = f[s].w;
            if (g == 0) {
                ((float*)sc[wave][0])[r16] = c1;
                ((float*)sc[wave][1])[r16] = c2;
                ((float*)sc[wave][2])[r16] = row ? l * kLog2e : INFINITY;  // no row: exp2 gives 0
            }
            if (row)
                some = 1;
        }
        __syncthreads();
        if (!some)
            continue;
        const int left = (rows - r0 + 15) / 16, tiles_now = left < kTiles ? left : kTiles;
        u32x4 k[W / 64];
        uint32_t pair[2];
        float w = 0.f;
        auto load = [&](int64_t u) {
            const uint8_t* tile = tiles + u * KvTile<W>::kBytes;
#pragma unroll
            for (int p = 0; p < W / 64; p++)
                k[p] = *(const u32x4*)(tile + p * 1024 + lane * 16);
#pragma unroll
            for (int a = 0; a < 2; a++)
                pair[a] = *(const uint32_t*)(tile + KvTile<W>::kKeyScales + 64 * a + 4 * r16);
            if (lane < 32 && u * kKvTile + lane < len)
                w = weight[u * kKvTile + lane];
        };
        if (u0 < units)
            load(u0);
        for (int64_t u = u0; u < units; u += du) {
            h16x8 kf[2][W / 32];
#pragma unroll
            for (int a = 0; a < 2; a++)
#pragma unroll
                for (int s = 0; s < W / 32; s++) {
                    const int Q = a * (W / 32) + s;
                    kf[a][s] = kv_codes(k[Q >> 2][Q & 3]);
                }
            const float ks[2] = {kv_s(pair[0]), kv_s(pair[1])}, kz[2] = {kv_z(pair[0]), kv_z(pair[1])};
            const float before = w;
            if (u + du < units)
                load(u + du);
            float sum[2] = {0.f, 0.f};
            for (int t = 0; t < tiles_now; t++) {
                floatx4 S[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
                for (int s = 0; s < W / 32; s++) {
                    Frag qf;
                    qf.w = sq[t][s][lane];
#pragma unroll
                    for (int a = 0; a < 2; a++)
                        S[a] = __builtin_amdgcn_mfma_f32_16x16x32_f16(qf.h, kf[a][s], S[a], 0, 0, 0);
                }
                const floatx4 c1 = sc[t][0][g], c2 = sc[t][1][g], l = sc[t][2][g];
#pragma unroll
                for (int a = 0; a < 2; a++)
#pragma unroll
                    for (int i = 0; i < 4; i++)
                        sum[a] += __builtin_amdgcn_exp2f(fmaf(ks[a] * S[a][i], c1[i], fmaf(kz[a], c2[i], -l[i])));
            }
            sum[0] = quad_sum(sum[0]);
            sum[1] = quad_sum(sum[1]);
            if (lane < 32 && u * kKvTile + lane < len)
                weight[u * kKvTile + lane] = before + (lane < 16 ? sum[0] : sum[1]);
        }
    }
}

}  // namespace

// Rows a workgroup takes (16 nt), its items at most, and the workgroups that
// share the work: as many as the chip holds at once (3 a CU with one row tile, 2
// with more), fewer where the slots cannot hold so many units.
struct KvPlan {
    int nt, wgs;
    int64_t items;
};

static KvPlan kv_plan(const KvView& c, int32_t B, int32_t max_nodes, int32_t Hq)
{
    KvPlan p;
    const int rows = max_nodes * (Hq / c.H);
    p.nt = rows <= 16 ? 1 : rows <= 32 ? 2 : 3;
    p.items = (int64_t)B * c.H * ((rows + 16 * p.nt - 1) / (16 * p.nt));
    const int64_t units = p.items * (c.tiles + (max_nodes + 31) / 32);
    const int64_t most = ((units + kLeastShare - 1) / kLeastShare + 7) / 8 * 8;
    const int64_t chip = p.nt == 1 ? kMaxShares : 512;
    p.wgs = (int)(most < chip ? most : chip);
    return p;
}

static size_t kv_part_rows(const KvPlan& p) { return (size_t)(p.wgs + p.items) * 16 * p.nt; }

size_t kv_attend_workspace_bytes(const KvView& c, int32_t B, int32_t max_nodes, int32_t Hq)
{
    const size_t n = kv_part_rows(kv_plan(c, B, max_nodes, Hq));
    return (2 * (size_t)(B + 1) + 2) * sizeof(int64_t) + 16 + n * (c.W + 2) * sizeof(float);
}

template <int W>
static void kv_attend_launch(const KvAttend& A, const KvPlan& p, hipStream_t stream)
{
    const dim3 grid(p.wgs), block(64 * kAttendWaves);
    if (p.nt == 1)
        hipLaunchKernelGGL((kv_attend_kernel<W, 1>), grid, block, 0, stream, A);
    else if (p.nt == 2)
        hipLaunchKernelGGL((kv_attend_kernel<W, 2>), grid, block, 0, stream, A);
    else
        hipLaunchKernelGGL((kv_attend_kernel<W, 3>), grid, block, 0, stream, A);
    const int rows = A.max_nodes * A.G;
    if (p.wgs >= 8 * p.items)
        hipLaunchKernelGGL((kv_join_kernel<W, 4>), dim3(rows, A.c.H, A.B), dim3(256), 0, stream, A, 16 * p.nt);
    else
        hipLaunchKernelGGL((kv_join_kernel<W, 1>), dim3((rows + 3) / 4, A.c.H, A.B), dim3(256), 0, stream, A,
                           16 * p.nt);
}

hipError_t launch_kv_attend(const KvView& c, const int32_t* slots, int32_t B, const void* q, int64_t q_ld,
                            int32_t Hq, const void* k, const void* v, int64_t ld, const int32_t* n_nodes,
                            const uint32_t* mask, int32_t max_nodes, float scale, void* workspace, void* out,
                            float* lse, hipStream_t stream)
{
    const KvPlan p = kv_plan(c, B, max_nodes, Hq);
    KvAttend A;
    A.c = c;
    A.slots = slots;
    A.q = (const uint16_t*)q;
    A.k = (const uint16_t*)k;
    A.v = (const uint16_t*)v;
    A.n_nodes = n_nodes;
    A.mask = mask;
    A.out = (uint16_t*)out;
    A.lse = lse;
    A.start = (int64_t*)workspace;
    A.items = A.start + B + 1;
    A.shares = A.items + B + 1;
    A.part_o = (float*)(A.shares + 2);  // 16-byte aligned: an even number of words before
    A.part_ml = A.part_o + kv_part_rows(p) * c.W;
    A.q_ld = q_ld;
    A.ld = ld;
    A.B = B;
    A.Hq = Hq;
    A.G = Hq / c.H;
    A.max_nodes = max_nodes;
    A.scale = scale;
    if (c.W == 64)
        kv_attend_launch<64>(A, p, stream);
    else
        kv_attend_launch<128>(A, p, stream);
    return hipGetLastError();
}

hipError_t launch_kv_weigh(const KvView& c, const int32_t* slots, int32_t B, const void* q, int64_t q_ld,
                           int32_t Hq, const float* lse, int32_t max_nodes, const int32_t* nodes,
                           const int32_t* count, float scale, hipStream_t stream)
{
    // two tiles a wave at least, and enough workgroups for the chip's 1,024 SIMDs
    const int64_t heads = (int64_t)B * c.H, most = (c.tiles + 7) / 8;
    int64_t blocks = (2048 + heads - 1) / heads;
    blocks = blocks < most ? blocks : most;
    const dim3 grid((unsigned)blocks, c.H, B), block(256);
    const bool one = max_nodes * (Hq / c.H) <= 16;
#define OIL_KV_WEIGH(W, ONE)                                                                                      \
    hipLaunchKernelGGL((kv_weigh_kernel<W, ONE>), grid, block, 0, stream, c, slots, (const uint16_t*)q, q_ld, Hq, \
                       lse, max_nodes, nodes, count, scale)
    if (c.W == 64 && one)
        OIL_KV_WEIGH(64, true);
    else if (c.W == 64)
        OIL_KV_WEIGH(64, false);
    else if (one)
        OIL_KV_WEIGH(128, true);
    else
        OIL_KV_WEIGH(128, false);
#undef OIL_KV_WEIGH
    return hipGetLastError();
}

}  // namespace oil
