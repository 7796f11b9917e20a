// Attention over the verifier's 4-bit cache and the nodes of a draft tree, and
// the attention weight that committed rows give to cached positions.
//
// attend: a wave streams 32-position tiles of one head, stored in MFMA operand
// order, and multiplies them with 16 NT rows (node, query head) at once: S^T =
// K Q^T puts a row's scores into one lane column, and the probabilities of a lane
// are, as they are, the operand of O^T = V^T P^T.  Tiles are loaded straight to
// LDS, two a wave in flight (a lane reads back what it loaded; in registers one
// tile fits beside the sums), and nothing in the loop waits for another wave.
//
// A code c of a 4-bit row enters the product as the binary16 subnormal c 2^-24
// (its nibble is the mantissa) or, for every other pair, as 16 c 2^-24: eight
// codes cost four ANDs and a shift.  The MFMA cuts a subnormal product's low bits,
// by the place that its exponent would have: scores differ from exact ones by 2e-7 of
// sum |q|(|z| + s c) where 128 columns share it (normal operands: 1e-8), by up to
// 5e-6 where one or two hold it, and sums p s c by 2^-18 of themselves, at most 2^-14
// (measured over equal value rows): outputs are bf16, 2^-8.  Queries are scaled to binary16 by
// a power of two per row, exactly for values within 2^-28 of the row's largest;
// sums are binary32.  The keys' codes are taken from their middle: the
// product starts at -7.5 sum(q) and y = z + 7.5 s enters as y sum(q), two small
// terms where s c and z would be large ones that cancel.  The values' z enters as
// sum(p z), in binary32.
//
// The softmax keeps, per row, a reference m and sums relative to it (base 2).
// m moves only when a score passes it by 2^15, to 11 below the maximum: then
// p <= 2^15 fits binary16, and a p below 2^-31 of the largest (2^-26 where s is far
// below E) is the first that rounds to nothing.  p times the value row's s, over a
// power of two E at or above every s so far, is what the second product takes,
// rounded to binary16 (2^-11 of it).  z and s c may be far larger than the value
// they add up to, so that rounding must not reach s c alone: z is weighted by the
// rounded p too (z / s times the operand).  Tiles in which some s is below 2^-6 E,
// where operands would lose bits, take two bf16 operands, the second what the first
// leaves.  Sums are kept over E 2^24, E also at or above every |z| 2^-64, and a
// wave's become a mean before they are multiplied by E: nothing passes binary32
// that the values do not, and what lies within 2^90 of the largest value counts.
//
// The tree's nodes come as further tiles in bf16, p as two operands, the second
// what the first leaves (2^-16 of p: one alone, 2^-8, would show in outputs of
// bf16 where the nodes hold the weight).
//
// What bounds it, at 8 key/value heads of 128 columns.  Single tokens: the stream
// of tiles (32 requests of up to 16,384 positions, 32 query heads: 364 MB in 75
// us, 4.9 TB/s; one slot of 262,149, 40 query heads: 286 MB in 58 us; the tiles by
// themselves stream at 7 TB/s, the rest is the share, the queries and the joining
// of the waves).  Many rows: the softmax's instructions between the products
// (about 330 VALU and 24 exponentials for 32 positions by 48 rows, two waves a
// SIMD; calls with their join: 32 trees of up to 65 nodes over up to 8,192
// positions, 32 query heads, 343 us, 443 TFLOP/s; 4 chunks of 256 nodes over
// 16,001, 64 query heads, 790 us, 685 TFLOP/s).  Few positions: the launch and five
// dependent steps of 1 to 2 us each (2,047 positions, one token: 11 us; 61 nodes
// over empty slots, 32 requests: 46 us, most of it the nodes' own tiles).
//
// weigh: below.
#include "kv.hpp"

namespace oil {

namespace {

typedef _Float16 h16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 h16x2 __attribute__((ext_vector_type(2)));

constexpr double kLog2eDouble = 1.44269504088896340736;
constexpr float kLog2e = (float)kLog2eDouble, kLn2 = 0.693147180559945309f;
constexpr float kLow = -1e38f;      // m of a row that has seen nothing
constexpr float kHead = 11.f;       // the maximum's place above m
constexpr float kRoom = 15.f;       // and the most a score may pass m by
constexpr float kLeast = 0x1p-6f;    // the smallest s / E that binary16 operands are taken at
constexpr float kOffset = 0x1p-64f;  // E / |z| at least
constexpr float kUnit = 0x1p-24f;    // of sums, times 1 / E: a code's place in binary16

// The item that a share begins inside (parts 0: at one's start).
struct KvCut {
    int32_t b, h, row_block;
    int32_t nth;     // share since the item's first
    int32_t parts;   // of the item
    int32_t first;   // the item's first share
    int32_t pad[2];
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
    KvCut* cuts;     // where each share begins
    float* part_o;   // per part of an item: its rows' means of the values,
    float* part_ml;  // and each one's (m, sum)
    int64_t q_ld, ld;
    int32_t B, Hq, G, max_nodes;
    int32_t shift;   // a unit is 2^shift tiles
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

// A dword's eight codes less 8, as they are: exact, and normal numbers, whose
// products the MFMA sums to 1e-8 of their size (subnormals, whose low bits it
// cuts, to 2e-7; measured over 128 columns).  A weight is a sum of exponentials of
// such scores, in binary32: there the difference shows.
__device__ __forceinline__ h16x8 kv_codes_less_8(uint32_t w)
{
    union {
        h16x2 p[4];
        h16x8 h;
    } f;
    const uint32_t x = w >> 8;
    const h16x2 sixteenth = {(_Float16)0.0625f, (_Float16)0.0625f}, less = {(_Float16)-72.f, (_Float16)-72.f};
    const h16x2 off = {(_Float16)-1032.f, (_Float16)-1032.f};
    // 1024 + c and 1024 + 16 c; the masks in registers, so that and-or is one instruction
    uint32_t low = 0x000F000Fu, high = 0x00F000F0u;
    asm("" : "+v"(low), "+v"(high));
    f.p[0] = __builtin_bit_cast(h16x2, (w & low) | 0x64006400u) + off;
    f.p[1] = __builtin_elementwise_fma(__builtin_bit_cast(h16x2, (w & high) | 0x64006400u), sixteenth, less);
    f.p[2] = __builtin_bit_cast(h16x2, (x & low) | 0x64006400u) + off;
    f.p[3] = __builtin_elementwise_fma(__builtin_bit_cast(h16x2, (x & high) | 0x64006400u), sixteenth, less);
    return f.h;
}

__device__ __forceinline__ uint32_t pack_f16(float a, float b)
{
    const floatx2 x = {a, b};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(x, h16x2));
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

// What memory holds is read again after this: no load moves past it.
__device__ __forceinline__ void read_anew() { asm volatile("" ::: "memory"); }

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

// The sum over a wave.
__device__ __forceinline__ float wave_sum(float x)
{
    x = quad_sum(x);
    x += __uint_as_float(__builtin_amdgcn_ds_swizzle(__float_as_uint(x), 0x201F));
    x += __uint_as_float(__builtin_amdgcn_ds_swizzle(__float_as_uint(x), 0x101F));
    x += __uint_as_float(__builtin_amdgcn_ds_swizzle(__float_as_uint(x), 0x081F));
    return x + __uint_as_float(__builtin_amdgcn_ds_swizzle(__float_as_uint(x), 0x041F));
}

// Raw bf16 operand of a row for columns d .. d + 7; zeros past D or where it is
// not wanted (the load is made all the same, inside the row, so that loads do not
// wait for each other's conditions).
__device__ __forceinline__ u32x4 kv_raw(const uint16_t* row, int d, int D, bool wanted = true)
{
    const u32x4 x = *(const u32x4*)(row + (d < D ? d : 0)), z = {0, 0, 0, 0};
    return wanted && d < D ? x : z;
}

// Of a row's scores in base 2, x = c1 (s dot) + c2 y, with dot starting at `from`.
struct KvFactors {
    float c1, c2, from;
};

// Scaled binary16 operands of a row and its factors, for codes as subnormals or
// (EXACT) codes less 8, which begin at 0 and take y = z + 8 s.  sum(q) is taken in binary64:
// its error would be a row's alone, and grow by y.
template <int W, bool EXACT>
__device__ __forceinline__ KvFactors kv_query(const uint16_t* row, bool live, int g, int D, float scale,
                                              Frag (&f)[W / 32])
{
    u32x4 raw[W / 32];
    uint32_t top = 0;
    double sum = 0.0;
#pragma unroll
    for (int ks = 0; ks < W / 32; ks++) {
        raw[ks] = kv_raw(row, 32 * ks + 8 * g, D, live);
#pragma unroll
        for (int j = 0; j < 4; j++) {
            const uint32_t lo = raw[ks][j] & 0x7FFFu, hi = (raw[ks][j] >> 16) & 0x7FFFu;
            top = max(top, max(lo, hi));
            sum += (double)__uint_as_float(raw[ks][j] << 16) + (double)__uint_as_float(raw[ks][j] & 0xFFFF0000u);
        }
    }
    top = (uint32_t)quad_max((float)top);
    const int e = max((int)(top >> 7) - 127, -112);
    const float by = __uint_as_float((uint32_t)(127 + 14 - e) << 23);  // the largest value to [2^14, 2^15)
#pragma unroll
    for (int ks = 0; ks < W / 32; ks++)
#pragma unroll
        for (int j = 0; j < 4; j++) {
            const float m = (j & 1) && !EXACT ? by * 0.0625f : by;
            f[ks].w[j] = pack_f16(__uint_as_float(raw[ks][j] << 16) * m,
                                  __uint_as_float(raw[ks][j] & 0xFFFF0000u) * m);
        }
    sum += __shfl_xor(sum, 16, 64);
    sum += __shfl_xor(sum, 32, 64);
    const double in2 = (double)scale * kLog2eDouble;
    KvFactors x;
    x.c1 = __builtin_ldexpf((float)in2, (EXACT ? 0 : 24) - 14 + e);
    x.c2 = (float)(in2 * sum);
    x.from = EXACT ? 0.f : (float)(-7.5 * 0x1p-24 * sum * (double)by);
    return x;
}

// The halves of a tile of the cache in LDS, as they are stored.
template <int W>
struct KvKeys {
    u32x4 code[W / 64][64];
    uint32_t pair[64];  // the keys' (s, z), the values'
};
template <int W>
struct KvValues {
    u32x4 code[W / 64][64];
};

// Loads of a wave straight to LDS (buffer loads: the compiler counts what is in
// flight exactly, where it takes global ones to LDS for flat accesses).
template <int W>
struct KvLoads {
    static constexpr int kAll = W / 32 + 1;  // of a tile

    static __device__ __forceinline__ __amdgpu_buffer_rsrc_t at(const uint8_t* tile)
    {
        return __builtin_amdgcn_make_buffer_rsrc((void*)tile, (short)0, KvTile<W>::kBytes, 0x00020000);
    }
    static __device__ __forceinline__ void keys(KvKeys<W>& to, const uint8_t* tile, int lane)
    {
        const __amdgpu_buffer_rsrc_t r = at(tile);
#pragma unroll
        for (int p = 0; p < W / 64; p++)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (void __attribute__((address_space(3)))*)&to.code[p][0], 16,
                                                     lane * 16, p * 1024, 0, 0);
        __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (void __attribute__((address_space(3)))*)&to.pair[0], 4, lane * 4,
                                                 KvTile<W>::kKeyScales, 0, 0);
    }
    static __device__ __forceinline__ void values(KvValues<W>& to, const uint8_t* tile, int lane)
    {
        const __amdgpu_buffer_rsrc_t r = at(tile);
#pragma unroll
        for (int p = 0; p < W / 64; p++)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (void __attribute__((address_space(3)))*)&to.code[p][0], 16,
                                                     lane * 16, KvTile<W>::kValues + p * 1024, 0, 0);
    }
};

// Waits until at most N of the wave's loads are in flight (expcnt and lgkmcnt as
// they are).
template <int N>
__device__ __forceinline__ void loads_at_most()
{
    __builtin_amdgcn_s_waitcnt((N & 15) | (7 << 4) | (15 << 8) | ((N >> 4) << 14));
    __builtin_amdgcn_sched_barrier(0);
}

// LDS of a wave for the scales of its tile: s of the 32 keys, the factors of the
// 32 value operands; then z of the keys, and what z of the values enters by.
struct KvScales {
    float s[64], z[64];
};

// The running state of a wave's 16 NT rows; a lane's column is row lane % 16 of
// each 16.
template <int W, int NT>
struct KvRows {
    floatx4 o[NT][W / 16];  // of O^T / (E 2^24) the codes' and the nodes' part
    float m[NT], l[NT], w[NT];  // w: the part of z, over E 2^24 too
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
            for (int t = 0; t < NT; t++) {
                w[t] *= by;
#pragma unroll
                for (int mt = 0; mt < W / 16; mt++)
                    o[t][mt] *= by;
            }
            E = up;
        }
    }
};

// A tile of `valid` cached positions (32, or fewer at the end of a slot).  Each
// lane prepares one pair; the eight of its rows' scores come back through LDS.
// The tile after the wave's next goes to the same place, the keys when the first
// product has taken them, the values after the second.
template <int W, int NT, bool END>
__device__ __forceinline__ void kv_tile(KvKeys<W>& K, KvValues<W>& V, const uint8_t* later, int valid, int lane, KvScales& L,
                                        const u32x4 (*q)[W / 32][64], const float (*factors)[3][16],
                                        KvRows<W, NT>& R)
{
    const int g = lane >> 4;
    const bool on = !END || (lane & 31) < valid, value = lane >= 32;
    const uint32_t pair = K.pair[lane];
    float s = on ? kv_s(pair) : 0.f, z = on ? kv_z(pair) : 0.f;
    u32x4 code[W / 64];
#pragma unroll
    for (int p = 0; p < W / 64; p++)
        code[p] = K.code[p][lane];
    const float least = value ? fmaxf(s, fabsf(z) * kOffset) : 0.f;
    if (__builtin_expect(__any(least > R.E), 0))
        R.widen(least);
    const bool rare = __any(value && on && s < R.E * kLeast);
    if (value) {
        const float by = 1.f / R.E;
        s *= lane & 2 ? by * 0.0625f : by;
        z *= by * kUnit;
        if (!rare)
            z = on ? z * __builtin_amdgcn_rcpf(s) : 0.f;
    }
    L.s[lane] = s;
    L.z[lane] = value ? z : fmaf(7.5f, s, z);
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    read_anew();  // the queries are read from LDS tile by tile: their registers are wanted
    floatx4 S[NT][2];
#pragma unroll
    for (int t = 0; t < NT; t++) {
        const float from = factors[t][2][lane & 15];
        S[t][0] = S[t][1] = floatx4{from, from, from, from};
    }
#pragma unroll
    for (int s = 0; s < W / 32; s++) {
        const int Q0 = s, Q1 = W / 32 + s;
        const h16x8 k0 = kv_codes(code[Q0 >> 2][Q0 & 3]), k1 = kv_codes(code[Q1 >> 2][Q1 & 3]);
#pragma unroll
        for (int t = 0; t < NT; t++) {
            Frag qf;
            qf.w = q[t][s][lane];
            S[t][0] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k0, qf.h, S[t][0], 0, 0, 0);
            S[t][1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k1, qf.h, S[t][1], 0, 0, 0);
        }
    }
    if (!END) {
        __builtin_amdgcn_sched_barrier(0);
        KvLoads<W>::keys(K, later, lane);
    }
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
    // (the values' codes follow while the scores are made)
#pragma unroll
    for (int p = 0; p < W / 64; p++)
        code[p] = V.code[p][lane];
    Frag p[NT];
#pragma unroll
    for (int t = 0; t < NT; t++) {
        const float c1 = factors[t][0][lane & 15], c2 = factors[t][1][lane & 15];
        float x[8];
        float top = -INFINITY;
#pragma unroll
        for (int e = 0; e < 8; e++) {
            x[e] = fmaf(ks[e] * S[t][e >> 2][e & 3], c1, fmaf(kz[e], c2, -R.m[t]));
            if (END)
                x[e] = in[e] ? x[e] : -INFINITY;
            top = fmaxf(top, x[e]);
        }
        if (__builtin_expect(__any(top > kRoom), 0)) {
            top = -INFINITY;
#pragma unroll
            for (int e = 0; e < 8; e++) {
                x[e] = fmaf(ks[e] * S[t][e >> 2][e & 3], c1, kz[e] * c2);
                if (END)
                    x[e] = in[e] ? x[e] : -INFINITY;
                top = fmaxf(top, x[e]);
            }
            R.raise(t, top);
#pragma unroll
            for (int e = 0; e < 8; e++)
                x[e] = fmaf(ks[e] * S[t][e >> 2][e & 3], c1, fmaf(kz[e], c2, -R.m[t]));
            if (END)
#pragma unroll
                for (int e = 0; e < 8; e++)
                    x[e] = in[e] ? x[e] : -INFINITY;
        }
        if (__builtin_expect(rare, 0)) {
#pragma unroll
            for (int e = 0; e < 8; e++) {
                x[e] = __builtin_amdgcn_exp2f(x[e]);
                R.l[t] += x[e];
                R.w[t] = fmaf(x[e], vz[e], R.w[t]);
                x[e] *= vs[e] * (e & 2 ? 0x1p-20f : 0x1p-24f);
            }
            Frag low;
#pragma unroll
            for (int j = 0; j < 4; j++) {
                p[t].w[j] = pack_bf16(x[2 * j], x[2 * j + 1]);
                low.w[j] = pack_bf16(x[2 * j] - __uint_as_float(p[t].w[j] << 16),
                                        x[2 * j + 1] - __uint_as_float(p[t].w[j] & 0xFFFF0000u));
            }
#pragma unroll
            for (int mt = 0; mt < W / 16; mt++) {
                __builtin_amdgcn_sched_barrier(0);  // one after the other: registers, not time, are short
                const bf16x8 vf = kv_codes_bf16(code[mt >> 2][mt & 3]);
                R.o[t][mt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, low.b, R.o[t][mt], 0, 0, 0);
                R.o[t][mt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, p[t].b, R.o[t][mt], 0, 0, 0);
            }
        } else {
#pragma unroll
            for (int e = 0; e < 8; e++) {
                x[e] = __builtin_amdgcn_exp2f(x[e]);
                R.l[t] += x[e];
                x[e] *= vs[e];
            }
#pragma unroll
            for (int j = 0; j < 4; j++)
                p[t].w[j] = pack_f16(x[2 * j], x[2 * j + 1]);
#pragma unroll
            for (int e = 0; e < 8; e++)
                R.w[t] = fmaf((float)p[t].h[e], vz[e], R.w[t]);
        }
    }
    if (__builtin_expect(!rare, 1)) {
#pragma unroll
        for (int mt = 0; mt < W / 16; mt++) {
            const h16x8 vf = kv_codes(code[mt >> 2][mt & 3]);
#pragma unroll
            for (int t = 0; t < NT; t++)
                R.o[t][mt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vf, p[t].h, R.o[t][mt], 0, 0, 0);
        }
    }
    if (!END) {
        __builtin_amdgcn_sched_barrier(0);
        KvLoads<W>::values(V, later, lane);
    }
}

// The node of row r of a head, -1 for none, and the row's queries (for none:
// those of row 0).
__device__ __forceinline__ int kv_row_of(const KvAttend& A, int b, int h, int m, int r, const uint16_t** row)
{
    const bool live = r < m * A.G;
    r = live ? r : 0;
    const int node = r / A.G;
    *row = A.q + ((int64_t)b * A.max_nodes + node) * A.q_ld + (int64_t)(h * A.G + r - node * A.G) * A.c.D;
    return live ? node : -1;
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
    // p / (E 2^24), or where that leaves bf16's range, part of it with the values
    const bool far = R.E > 0x1p56f;
    const float by = far ? 0x1p-80f : kUnit / R.E;
    floatx4 S[NT][2];
#pragma unroll
    for (int t = 0; t < NT; t++)
        S[t][0] = S[t][1] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int s = 0; s < W / 32; s++) {
        Frag kf[2];
#pragma unroll
        for (int a = 0; a < 2; a++)
            kf[a].w = kv_raw(A.k + base + (int64_t)(n0 + 16 * a + r < m ? 16 * a + r : 0) * A.ld, 32 * s + 8 * g, D);
#pragma unroll
        for (int t = 0; t < NT; t++) {
            Frag qf;
            qf.w = kv_raw(row[t], 32 * s + 8 * g, D);
#pragma unroll
            for (int a = 0; a < 2; a++)
                S[t][a] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[a].b, qf.b, S[t][a], 0, 0, 0);
        }
    }
    Frag p[NT], low[NT];
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
        for (int j = 0; j < 4; j++) {
            p[t].w[j] = pack_bf16(x[2 * j], x[2 * j + 1]);
            low[t].w[j] = pack_bf16(x[2 * j] - __uint_as_float(p[t].w[j] << 16),
                                    x[2 * j + 1] - __uint_as_float(p[t].w[j] & 0xFFFF0000u));
        }
    }
    // the values, columns in lanes: two bytes a load, from eight rows at fixed distances
    const uint16_t* from[8];
#pragma unroll
    for (int e = 0; e < 8; e++) {
        const int key = 16 * (e >> 2) + 4 * g + (e & 3);
        from[e] = A.v + base + (int64_t)(n0 + key < m ? key : 0) * A.ld;
    }
    bool odd = false;
    constexpr int kGroup = NT == 1 ? 4 : 2;  // column tiles whose loads are in flight together
#pragma unroll
    for (int m0 = 0; m0 < W / 16; m0 += kGroup) {
        read_anew();  // the next group's loads would take registers that the rows need
        uint32_t raw[kGroup][8];
#pragma unroll
        for (int i = 0; i < kGroup; i++) {
            // past D nothing is wanted; half a column tile repeats itself
            const int at = D == W || 16 * (m0 + i) + 16 <= D ? 16 * (m0 + i) + r
                                                             : 16 * (m0 + i) < D ? 16 * (m0 + i) + (r & 7) : 0;
#pragma unroll
            for (int e = 0; e < 8; e++)
                raw[i][e] = from[e][at];
        }
        Frag vf[kGroup];
        typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
        u16x2 top = {0, 0};
#pragma unroll
        for (int i = 0; i < kGroup; i++)
#pragma unroll
            for (int j = 0; j < 4; j++) {
                vf[i].w[j] = raw[i][2 * j] | raw[i][2 * j + 1] << 16;
                top = __builtin_elementwise_max(top, __builtin_bit_cast(u16x2, vf[i].w[j] & 0x7FFF7FFFu));
            }
        if (__builtin_expect(__any(top[0] >= 0x7F80 || top[1] >= 0x7F80) || far, 0)) {
            // not finite: nothing here, and added below to the rows that see it
            odd = true;
            const float rest = far ? 0x1p56f / R.E : 1.f;
#pragma unroll
            for (int i = 0; i < kGroup; i++)
#pragma unroll
                for (int j = 0; j < 4; j++) {
                    const uint32_t lo = vf[i].w[j] << 16, hi = vf[i].w[j] & 0xFFFF0000u;
                    vf[i].w[j] = pack_bf16((lo & 0x7F800000u) == 0x7F800000u ? 0.f : __uint_as_float(lo) * rest,
                                           (hi & 0x7F800000u) == 0x7F800000u ? 0.f : __uint_as_float(hi) * rest);
                }
        }
#pragma unroll
        for (int i = 0; i < kGroup; i++)
#pragma unroll
            for (int t = 0; t < NT; t++) {
                R.o[t][m0 + i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf[i].b, low[t].b, R.o[t][m0 + i], 0, 0, 0);
                R.o[t][m0 + i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf[i].b, p[t].b, R.o[t][m0 + i], 0, 0, 0);
            }
    }
    if (__builtin_expect(odd, 0)) {
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

// The same for one row tile and the few nodes of single tokens: lane by lane, in
// binary32, a node at a time (at one node, a decode step's, 1 us where the
// products above and their operands take 8).
constexpr int kFewNodes = 4;

template <int W>
__device__ __forceinline__ void kv_few_nodes(const KvAttend& A, int b, int h, int m, int lane, KvRows<W, 1>& R)
{
    const int g = lane >> 4, D = A.c.D;
    const uint16_t* row;
    const int node = kv_row_of(A, b, h, m, lane & 15, &row);
    u32x4 q[W / 32];
#pragma unroll
    for (int s = 0; s < W / 32; s++)
        q[s] = kv_raw(row, 32 * s + 8 * g, D);
    uint32_t sees = node < 0 ? 0 : (2u << node) - 1;
    if (A.mask && node >= 0)
        sees = A.mask[((int64_t)b * A.max_nodes + node) * ((A.max_nodes + 31) / 32)];
    if (R.E < 1.f)
        R.widen(1.f);
    const float by = 1.f / R.E;
    for (int u = 0; u < m; u++) {
        const int64_t at = ((int64_t)b * A.max_nodes + u) * A.ld + (int64_t)h * D;
        u32x4 k[W / 32];
        uint2 v[W / 16];
#pragma unroll
        for (int s = 0; s < W / 32; s++)
            k[s] = kv_raw(A.k + at, 32 * s + 8 * g, D);
#pragma unroll
        for (int mt = 0; mt < W / 16; mt++)
            v[mt] = *(const uint2*)(A.v + at + (16 * mt + 4 * g < D ? 16 * mt + 4 * g : 0));
        float dot = 0.f;
#pragma unroll
        for (int s = 0; s < W / 32; s++)
#pragma unroll
            for (int j = 0; j < 4; j++) {
                dot = fmaf(__uint_as_float(q[s][j] << 16), __uint_as_float(k[s][j] << 16), dot);
                dot = fmaf(__uint_as_float(q[s][j] & 0xFFFF0000u), __uint_as_float(k[s][j] & 0xFFFF0000u), dot);
            }
        dot = quad_sum(dot);
        const bool on = (sees >> u) & 1;
        const float x = on ? dot * (A.scale * kLog2e) : -INFINITY;
        if (__any(x - R.m[0] > kRoom))
            R.raise(0, x);
        const float p = on ? __builtin_amdgcn_exp2f(x - R.m[0]) : 0.f;
        R.l[0] += g == 0 ? p : 0.f;
#pragma unroll
        for (int mt = 0; mt < W / 16; mt++)
#pragma unroll
            for (int i = 0; i < 4; i++) {
                const uint32_t w = i < 2 ? v[mt].x : v[mt].y;
                const uint32_t y = i & 1 ? w & 0xFFFF0000u : w << 16;
                // not finite: itself, whatever p rounds to
                const float f = (y & 0x7F800000u) == 0x7F800000u ? 1.f : p * kUnit;
                R.o[0][mt][i] = on ? fmaf(f, __uint_as_float(y) * by, R.o[0][mt][i]) : R.o[0][mt][i];
            }
    }
}

constexpr int kAttendWaves = 4;

__device__ __forceinline__ int kv_live_nodes(const KvAttend& A, int b, int slot)
{
    if (slot < 0)
        return 0;
    const int m = A.n_nodes ? A.n_nodes[b] : A.max_nodes;
    return m < 0 ? 0 : m > A.max_nodes ? A.max_nodes : m;
}

// Tiles that a live row of a request goes through: the cache's, then the tree's.
__device__ __forceinline__ int kv_row_tiles(const KvAttend& A, int32_t len, int m)
{
    return (len + kKvTile - 1) / kKvTile + (A.k ? (m + 31) / 32 : 0);
}

// The work of a call is one list of units: requests, in each its heads, in each
// its blocks of 16 NT rows (an item), in each the tiles (a unit is one, or so many
// that there are fewer than 2^31).  Equal shares of it go
// to the workgroups, whatever the lengths; a share that begins or ends inside an
// item leaves a part of it for the join: one that begins inside one as part 2 share,
// one that starts an item and ends inside it as 2 share + 1.  So the workspace grows
// with the workgroups alone.

// Where part p of the item whose first share is `first` stands.
__device__ __forceinline__ int kv_part_at(int first, int p) { return 2 * (first + p) + (p == 0); }

// Least units of a share: two tiles a wave (or what an item has, if less).
constexpr int kLeastShare = 2 * kAttendWaves;
constexpr int kMaxShares = 768;

// A value that all lanes hold alike, as a scalar.
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ const uint8_t* uniform(const uint8_t* p)
{
    const uint64_t x = (uint64_t)p;
    return (const uint8_t*)((uint64_t)(uint32_t)uniform((int)(x >> 32)) << 32 | (uint32_t)uniform((int)x));
}

// total units in `shares` equal ones: share w begins at each * w + left * w / shares.
struct KvShares {
    int total, shares, each, left;

    __device__ __forceinline__ int cut(int w) const
    {
        return each * w + (int)((uint32_t)left * (uint32_t)w / (uint32_t)shares);
    }
    // The share that holds unit x.
    __device__ __forceinline__ int of(int x) const
    {
        int w = (int)((float)x * (float)shares / (float)total);
        w = w < shares ? w : shares - 1;
        while (w > 0 && cut(w) > x)
            w--;
        while (w + 1 < shares && cut(w + 1) <= x)
            w++;
        return w;
    }
};

// Sums over the lanes up to and with this one (rows of 16 by shifts, then the
// last lane of each row to the rows after it).
__device__ __forceinline__ int wave_scan(int x)
{
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xF, 0xF, false);  // row_shr:1
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xF, 0xF, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xF, 0xF, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xF, 0xF, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xA, 0xF, false);  // row_bcast:15
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xC, 0xF, false);  // row_bcast:31
    return x;
}

// A request's part of the list.
template <int NT>
struct KvRequest {
    int slot, len, m, items, units;  // m: live nodes (0 without a tile); units of an item

    __device__ __forceinline__ void load(const KvAttend& A, int b)
    {
        m = A.max_nodes;
        slot = len = items = units = 0;
        if (b >= A.B)
            return;
        slot = kv_slot(A.c, A.slots, b);
        m = kv_live_nodes(A, b, slot);
        len = m ? kv_len(A.c, slot) : 0;
        const int tiles = m ? kv_row_tiles(A, len, m) : 0;
        units = (tiles + (1 << A.shift) - 1) >> A.shift;
        m = tiles ? m : 0;
        items = A.c.H * ((m * A.G + 16 * NT - 1) / (16 * NT));
    }
};

// 64 requests in LDS: read once an item, they would take registers that the tiles
// need.
struct KvRequestTable {
    int slot[64], len[64], m[64], units[64], items[64], upto[64];

    template <int NT>
    __device__ __forceinline__ int put(const KvRequest<NT>& r, int lane)
    {
        const int sum = wave_scan(r.items * r.units);
        slot[lane] = r.slot;
        len[lane] = r.len;
        m[lane] = r.m;
        units[lane] = r.units;
        items[lane] = r.items;
        upto[lane] = sum;
        return __builtin_amdgcn_readlane(sum, 63);
    }
};

// Rows that see nothing (past a request's nodes, or without a tile) are cleared
// by the first waves of all workgroups together.
template <int NT>
__device__ __forceinline__ void kv_clear_dead(const KvAttend& A, int b0, int m, int lane)
{
    const int D = A.c.D;
    for (uint64_t some = __ballot(m < A.max_nodes); some; some &= some - 1) {
        const int l = __ffsll((unsigned long long)some) - 1, live = __builtin_amdgcn_readlane(m, l);
        const int64_t n = (int64_t)(A.max_nodes - live) * A.Hq;
        const int64_t first = ((int64_t)(b0 + l) * A.max_nodes + live) * A.Hq;
        for (int64_t i = blockIdx.x * 64ll + lane; i < n * (D / 8); i += gridDim.x * 64ll)
            ((u32x4*)(A.out + first * D))[i] = u32x4{0, 0, 0, 0};
        if (A.lse)
            for (int64_t i = blockIdx.x * 64ll + lane; i < n; i += gridDim.x * 64ll)
                A.lse[first + i] = -INFINITY;
    }
}

// The part of an item in hand and where the share goes on: kept in LDS while the
// tiles have the registers (scalar ones too: they spill into vector ones).
struct KvPart {
    int more;                          // whether there is one
    int at, end, base, b0;             // the rest of the share; requests in the table
    int b, h, row_block, m, len;
    int part, whole, t0, t1;           // its number; tiles
    const uint8_t* tiles;
};

// The kernel's arguments, read where they are wanted.
__device__ __forceinline__ KvAttend kv_args()
{
    auto p = (const __attribute__((address_space(4))) KvAttend*)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(p));
    return *(const KvAttend*)p;
}

// The next part of a share, if there is one (a wave for its workgroup).
template <int NT>
__device__ __forceinline__ void kv_next_part(const KvAttend& A, KvPart& P, KvRequestTable& table, const KvShares& S, int share,
                                             int lane)
{
    int at = uniform(P.at), end = uniform(P.end), base = uniform(P.base), b0 = uniform(P.b0);
    P.more = 0;
    if (at >= end)
        return;
    uint64_t past;
    while (!(past = __ballot(table.upto[lane] > at - base))) {
        base += uniform(table.upto[63]);
        b0 += 64;
        if (b0 >= A.B)
            return;
        KvRequest<NT> more;
        more.load(A, b0 + lane);
        table.put(more, lane);
    }
    const int l = __ffsll((unsigned long long)past) - 1, b = b0 + l;
    const int m = uniform(table.m[l]), units = uniform(table.units[l]), items = uniform(table.items[l]);
    const int begin = base + uniform(table.upto[l]) - items * units;
    const int slot = uniform(table.slot[l]), len = uniform(table.len[l]), row_tiles = kv_row_tiles(A, len, m);
    const int row_blocks = (uint32_t)items / (uint32_t)A.c.H, item = (uint32_t)(at - begin) / (uint32_t)units;
    const int h = (uint32_t)item / (uint32_t)row_blocks;
    const int u0 = at - begin - item * units, u1 = end - at < units - u0 ? u0 + (end - at) : units;
    if (u0 != 0 && lane == 0) {  // the first of a share's parts at most
        const int w0 = S.of(at - u0), w1 = S.of(at - u0 + units - 1);
        KvCut cut;
        cut.b = b;
        cut.h = h;
        cut.row_block = item - h * row_blocks;
        cut.nth = share - w0;
        cut.parts = w1 - w0 + 1;
        cut.first = w0;
        A.cuts[share] = cut;
    }
    P.more = 1;
    P.at = at + u1 - u0;
    P.base = base;
    P.b0 = b0;
    P.b = b;
    P.h = h;
    P.row_block = item - h * row_blocks;
    P.m = m;
    P.len = len;
    P.part = 2 * share + (u0 == 0);
    P.whole = u0 == 0 && u1 == units;
    P.t0 = u0 << A.shift;
    P.t1 = (u1 << A.shift) < row_tiles ? u1 << A.shift : row_tiles;
    P.tiles = kv_tiles(A.c, slot, h);
}

template <int W, int NT>
__global__ __launch_bounds__(256, NT == 1 ? 3 : 2) void kv_attend_kernel(KvAttend)
{
    constexpr int kRows = 16 * NT;
    __shared__ float sm[kAttendWaves][kRows], sl[kAttendWaves][kRows];
    // the waves' tiles, two each (objects of their own, so that what a read waits for
    // is known), and after them the waves' sums
    __shared__ KvKeys<W> keys0[kAttendWaves], keys1[kAttendWaves];
    __shared__ KvValues<W> values0[kAttendWaves], values1[kAttendWaves];
    constexpr int kSums = (W / 16) * 64;
    static_assert(kSums * sizeof(floatx4) <= sizeof(values0), "sums of a row tile");
    floatx4 *const so0 = (floatx4*)&values0[0], *const so1 = (floatx4*)&values1[0];
    __shared__ u32x4 sq[NT][W / 32][64];
    __shared__ float factors[NT][3][16];
    __shared__ __align__(16) KvScales scales[kAttendWaves];
    __shared__ KvRequestTable table;
    __shared__ KvPart P;
    __shared__ KvShares shares;
    const int wave = uniform((int)(threadIdx.x >> 6));
    if (wave == 0) {
        const KvAttend A = kv_args();
        const int lane = threadIdx.x;
        KvShares S;
        int items;
        {
            KvRequest<NT> first;
            first.load(A, lane);
            S.total = table.put(first, lane);
            items = __builtin_amdgcn_readlane(wave_scan(first.items), 63);
            kv_clear_dead<NT>(A, 0, first.m, lane);
        }
        for (int b0 = 64; b0 < A.B; b0 += 64) {
            KvRequest<NT> more;
            more.load(A, b0 + lane);
            kv_clear_dead<NT>(A, b0, more.m, lane);
            S.total += __builtin_amdgcn_readlane(wave_scan(more.items * more.units), 63);
            items += __builtin_amdgcn_readlane(wave_scan(more.items), 63);
        }
        const int fine = (int)(((uint32_t)S.total + kLeastShare - 1) / kLeastShare), most = fine < items ? items : fine;
        S.shares = most < 1 ? 1 : most < (int)gridDim.x ? most : (int)gridDim.x;
        // as many to each item, where there are more: items of one length then end
        // with a share, and no workgroup has two parts
        if (S.shares > items)
            S.shares = items ? (int)((uint32_t)S.shares / (uint32_t)items * (uint32_t)items) : 1;
        S.each = (int)((uint32_t)S.total / (uint32_t)S.shares);
        S.left = S.total - S.each * S.shares;
        // neighbouring shares on one XCD: the row blocks of a head read the same tiles
        const int per_xcd = (S.shares + 7) / 8, share = (blockIdx.x & 7) * per_xcd + (blockIdx.x >> 3);
        const bool mine = (int)(blockIdx.x >> 3) < per_xcd && share < S.shares;
        if ((int)blockIdx.x >= S.shares && lane == 0)
            A.cuts[blockIdx.x].parts = 0;  // no such share
        if (mine && lane == 0)
            A.cuts[share].parts = 0;
        shares = S;
        P.at = mine ? S.cut(share) : 0;
        P.end = mine ? S.cut(share + 1) : 0;
        P.base = P.b0 = 0;
    }
    while (true) {
        // what follows from the lane is worked out anew for each part: kept over all
        // of them it would take the registers that the tiles need
        int lane = threadIdx.x & 63;
        asm volatile("" : "+v"(lane));
        const int r16 = lane & 15, g = lane >> 4;
        {
            const KvAttend A = kv_args();
            if (wave == 0) {
                const int per_xcd = (uniform(shares.shares) + 7) / 8;
                kv_next_part<NT>(A, P, table, shares, (blockIdx.x & 7) * per_xcd + (blockIdx.x >> 3), lane);
            }
            __syncthreads();
            if (!uniform(P.more))
                break;
            {  // the wave's first two tiles are on their way while the queries come
                const int cached = (uniform(P.len) + kKvTile - 1) / kKvTile, t1 = uniform(P.t1);
                const int last = cached < t1 ? cached : t1, u = uniform(P.t0) + wave;
                const int v = u + kAttendWaves < last ? u + kAttendWaves : u;
                if (u < last) {
                    const uint8_t* tiles = uniform(P.tiles);
                    KvLoads<W>::keys(keys0[wave], tiles + (int64_t)u * KvTile<W>::kBytes, lane);
                    KvLoads<W>::values(values0[wave], tiles + (int64_t)u * KvTile<W>::kBytes, lane);
                    KvLoads<W>::keys(keys1[wave], tiles + (int64_t)v * KvTile<W>::kBytes, lane);
                    KvLoads<W>::values(values1[wave], tiles + (int64_t)v * KvTile<W>::kBytes, lane);
                }
            }
            const int b = uniform(P.b), h = uniform(P.h), m = uniform(P.m), r0 = uniform(P.row_block) * kRows;
            if (wave < NT) {  // a row tile a wave
                Frag q[W / 32];
                const uint16_t* row;
                const int node = kv_row_of(A, b, h, m, r0 + 16 * wave + r16, &row);
                const KvFactors f = kv_query<W, false>(row, node >= 0, g, A.c.D, A.scale, q);
#pragma unroll
                for (int s = 0; s < W / 32; s++)
                    sq[wave][s][lane] = q[s].w;
                factors[wave][0][r16] = f.c1;  // the four lanes of a row alike
                factors[wave][1][r16] = f.c2;
                factors[wave][2][r16] = f.from;
            }
        }
        __syncthreads();
        KvRows<W, NT> R;
        R.init();
        int u;
        {
            const int len = uniform(P.len), cached = (len + kKvTile - 1) / kKvTile, t1 = uniform(P.t1);
            const int last = cached < t1 ? cached : t1, full = len / kKvTile < last ? len / kKvTile : last;
            const uint8_t* tiles = uniform(P.tiles);
            u = uniform(P.t0) + wave;
            if (u < last) {
                auto tile = [&](int x) { return tiles + (int64_t)(x < last ? x : last - 1) * KvTile<W>::kBytes; };
                bool second = false;
                while (u < full) {
                    loads_at_most<KvLoads<W>::kAll>();
                    kv_tile<W, NT, false>(keys0[wave], values0[wave], tile(u + 2 * kAttendWaves), 32, lane,
                                          scales[wave], sq, factors, R);
                    u += kAttendWaves;
                    second = u >= full;
                    if (second)
                        break;
                    loads_at_most<KvLoads<W>::kAll>();
                    kv_tile<W, NT, false>(keys1[wave], values1[wave], tile(u + 2 * kAttendWaves), 32, lane,
                                          scales[wave], sq, factors, R);
                    u += kAttendWaves;
                }
                loads_at_most<0>();
                if (__builtin_expect(u < last, 0)) {  // the slot's last tile, with fewer than 32 positions
                    kv_tile<W, NT, true>(second ? keys1[wave] : keys0[wave], second ? values1[wave] : values0[wave],
                                         nullptr, uniform(P.len) - u * kKvTile, lane, scales[wave], sq, factors, R);
                    u += kAttendWaves;
                }
            }
        }
        read_anew();
        if (__builtin_expect(u < uniform(P.t1), 0)) {
            const KvAttend A = kv_args();
            const int cached = (uniform(P.len) + kKvTile - 1) / kKvTile, t1 = uniform(P.t1);
            if constexpr (NT == 1) {
                if (uniform(P.m) <= kFewNodes) {
                    kv_few_nodes<W>(A, uniform(P.b), uniform(P.h), uniform(P.m), lane, R);
                    u = t1;
                }
            }
            for (; u < t1; u += kAttendWaves)
                kv_nodes<W, NT>(A, uniform(P.b), uniform(P.h), (u - cached) * 32, uniform(P.m), lane,
                                uniform(P.row_block) * kRows, R);
        }
        // the waves' shares of the mean, relative to the largest m
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
            const float f = __builtin_amdgcn_exp2f(R.m[t] - top[t]) / (sum[t] * kUnit);
#pragma unroll
            for (int mt = 0; mt < W / 16; mt++)
#pragma unroll
                for (int i = 0; i < 4; i++)
                    R.o[t][mt][i] = R.l[t] == 0.f ? 0.f : (R.o[t][mt][i] + R.w[t]) * f * R.E;
        }
#pragma unroll
        for (int t = 0; t < NT; t++)
#pragma unroll
            for (int half = kAttendWaves / 2; half >= 1; half >>= 1) {
                if (wave >= half && wave < 2 * half)
#pragma unroll
                    for (int mt = 0; mt < W / 16; mt++)
                        (wave == half ? so0 : so1)[mt * 64 + lane] = R.o[t][mt];
                __syncthreads();
                if (wave < half)
#pragma unroll
                    for (int mt = 0; mt < W / 16; mt++)
                        R.o[t][mt] += (wave == 0 ? so0 : so1)[mt * 64 + lane];
                __syncthreads();
            }
        if (wave != 0)
            continue;
        const KvAttend A = kv_args();
        const int b = uniform(P.b), h = uniform(P.h), D = A.c.D, r0 = uniform(P.row_block) * kRows;
        const int live = uniform(P.m) * A.G;
        const bool whole = uniform(P.whole);
#pragma unroll
        for (int t = 0; t < NT; t++) {
            const int r = r0 + 16 * t + r16;
            if (r >= live)
                continue;
            if (!whole) {
                const int64_t to = (int64_t)uniform(P.part) * kRows + 16 * t + r16;
                if (g == 0)
                    ((floatx2*)A.part_ml)[to] = floatx2{top[t], sum[t]};
#pragma unroll
                for (int mt = 0; mt < W / 16; mt++)
                    *(floatx4*)(A.part_o + to * W + 16 * mt + 4 * g) = R.o[t][mt];
            } else {
                const int node = r / A.G;
                const int64_t to = ((int64_t)b * A.max_nodes + node) * A.Hq + h * A.G + (r - node * A.G);
                const bool none = sum[t] == 0.f;
                if (g == 0 && A.lse)
                    A.lse[to] = none ? -INFINITY : kLn2 * (top[t] + __builtin_amdgcn_logf(sum[t]));
#pragma unroll
                for (int mt = 0; mt < W / 16; mt++)
                    if (16 * mt + 4 * g < D) {
                        uint2 o;
                        o.x = pack_bf16(R.o[t][mt][0], R.o[t][mt][1]);
                        o.y = pack_bf16(R.o[t][mt][2], R.o[t][mt][3]);
                        *(uint2*)(A.out + to * D + 16 * mt + 4 * g) = o;
                    }
            }
        }
    }
}

// The parts of the items that shares cut, joined: o = sum o_p l_p 2^(m_p - m) over
// sum l_p 2^(m_p - m), m the largest.  The workgroup of each share that begins
// inside an item takes its part of that item's rows, with four waves a row where
// the parts are many (past 16 a wave's loads would follow each other), else one.
// Latencies bound it: a launch, a table entry, (m, l), rows: 4 to 6 us, 19 us where
// 512 shares of 48 rows by 128 columns are joined (23 MB).  Factors of parts go from
// lane to lane by reads of a lane and sums by swaps and swizzles: as LDS shuffles they
// stood before the rows' loads could be used (23 us).
template <int W>
__global__ __launch_bounds__(256) void kv_join_kernel(KvAttend A, int rows_per_item)
{
    constexpr int kFew = 16;
    __shared__ float f[kMaxShares];
    __shared__ float red[2][4];
    __shared__ floatx2 so[4][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, D = A.c.D, d = W == 128 ? 2 * lane : lane;
    const KvCut cut = A.cuts[blockIdx.x];
    if (cut.parts < 2 || cut.nth < 1)
        return;
    const int b = cut.b, m = kv_live_nodes(A, b, kv_slot(A.c, A.slots, b)), left = m * A.G - cut.row_block * rows_per_item;
    const int rows = left < rows_per_item ? left : rows_per_item;
    const bool few = cut.parts <= kFew;
    const int step = few ? 4 * (cut.parts - 1) : cut.parts - 1;
    for (int r = few ? 4 * (cut.nth - 1) + wave : cut.nth - 1; r < rows; r += step) {
        auto at = [&](int p) { return (int64_t)kv_part_at(cut.first, p) * rows_per_item + r; };  // part p's row
        const floatx2* ml = (const floatx2*)A.part_ml;
        const float* from = A.part_o + d;
        float top = kLow, total = 0.f;
        floatx2 o = {0.f, 0.f};
        if (few) {
            const floatx2 mine = ml[at(lane < cut.parts ? lane : 0)];
            top = wave_max(mine[0]);
            float part = lane >= cut.parts || mine[1] == 0.f ? 0.f : mine[1] * __builtin_amdgcn_exp2f(mine[0] - top);
            total = wave_sum(part);
            part = total == 0.f ? 0.f : part / total;
            for (int p0 = 0; p0 < cut.parts; p0 += 4) {
                floatx2 y[4];
#pragma unroll
                for (int p = 0; p < 4; p++) {
                    const float* row = from + at(p0 + p < cut.parts ? p0 + p : 0) * W;
                    if (W == 128)
                        y[p] = *(const floatx2*)row;
                    else
                        y[p] = floatx2{row[0], 0.f};
                }
#pragma unroll
                for (int p = 0; p < 4; p++) {
                    const float by = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(part), p0 + p));
                    // (a part that weighs nothing is added too: its rows may be NaN)
                    const bool real = p0 + p < cut.parts;
                    o[0] = real ? fmaf(by, y[p][0], o[0]) : o[0];
                    o[1] = real ? fmaf(by, y[p][1], o[1]) : o[1];
                }
            }
        } else {
            for (int p = threadIdx.x; p < cut.parts; p += 256)
                top = fmaxf(top, ml[at(p)][0]);
            top = wave_max(top);
            __syncthreads();
            if (lane == 0)
                red[0][wave] = top;
            __syncthreads();
            top = fmaxf(fmaxf(red[0][0], red[0][1]), fmaxf(red[0][2], red[0][3]));
            for (int p = threadIdx.x; p < cut.parts; p += 256) {
                const floatx2 x = ml[at(p)];
                f[p] = x[1] == 0.f ? 0.f : x[1] * __builtin_amdgcn_exp2f(x[0] - top);
                total += f[p];
            }
            total = wave_sum(total);
            if (lane == 0)
                red[1][wave] = total;
            __syncthreads();
            total = red[1][0] + red[1][1] + red[1][2] + red[1][3];
            const float each = total == 0.f ? 0.f : 1.f / total;
#pragma unroll 8
            for (int p = wave; p < cut.parts; p += 4) {
                const float by = f[p] * each;
                const float* part = from + at(p) * W;
                floatx2 y = {part[0], 0.f};
                if (W == 128)
                    y = *(const floatx2*)part;
                o[0] = fmaf(by, y[0], o[0]);
                o[1] = fmaf(by, y[1], o[1]);
            }
            so[wave][lane] = o;
            __syncthreads();
#pragma unroll
            for (int w = 1; w < 4; w++)
                o += so[(wave + w) & 3][lane];
            __syncthreads();
            if (wave != 0)
                continue;
        }
        const int row = cut.row_block * rows_per_item + r, node = row / A.G;
        const int64_t to = ((int64_t)b * A.max_nodes + node) * A.Hq + cut.h * A.G + (row - node * A.G);
        const bool none = total == 0.f;
        if (d < D) {
            if (W == 128)
                *(uint32_t*)(A.out + to * D + d) = pack_bf16(o[0], o[1]);
            else
                A.out[to * D + d] = (uint16_t)pack_bf16(o[0], 0.f);
        }
        if (lane == 0 && A.lse)
            A.lse[to] = none ? -INFINITY : kLn2 * (top + __builtin_amdgcn_logf(total));
    }
}

// w[j] += sum over rows of exp(scale q.k_j - lse): the keys' half of each tile and
// the weights are read once for up to 64 rows, which stand in LDS as operands.
// S = Q K^T puts a position into a lane column, so a position's sum over rows is
// over a lane's registers and four lanes; a wave owns its tiles' weights, so there
// are no atomics and one result.  Bound by tiles in flight: with one in flight a
// wave 32 requests of up to 16,384 positions took 51.5 us, with two 47.7 (205 MB,
// 4.3 TB/s; the longest requests' waves run on alone at the end); 8 requests of up
// to 32,768 and up to 56 rows a head 33 us, much of it the exponentials' instructions.
// ONE: at most 16 rows, whose loop over row tiles is gone.
template <int W, bool ONE>
__global__ __launch_bounds__(256, 4) void kv_weigh_kernel(KvView c, const int32_t* __restrict__ slots,
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
    const int units = (int)(((int64_t)len + kKvTile - 1) / kKvTile);
    const int u0 = (int)blockIdx.x * 4 + uniform(wave), du = (int)gridDim.x * 4;
    if ((int)blockIdx.x * 4 >= units)
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
            const int rr = r < rows ? r : 0, a = h * G + rr % G;
            const int64_t at = (int64_t)b * max_nodes + kv_source(nodes, b, max_nodes, rr / G);
            const float l = lse[at * Hq + a];
            const bool row = r < rows && l != -INFINITY;
            Frag f[W / 32];
            const KvFactors x = kv_query<W, true>(q + at * q_ld + (int64_t)a * c.D, row, g, c.D, scale, f);
#pragma unroll
            for (int s = 0; s < W / 32; s++)
                sq[wave][s][lane] = f[s].w;
            if (g == 0) {
                ((float*)sc[wave][0])[r16] = x.c1;
                ((float*)sc[wave][1])[r16] = x.c2;
                ((float*)sc[wave][2])[r16] = row ? (float)((double)l * kLog2eDouble) : INFINITY;  // no row: exp2 gives 0
            }
            if (row)
                some = 1;
        }
        __syncthreads();
        if (!some)
            continue;
        const int left = (rows - r0 + 15) / 16, tiles_now = left < kTiles ? left : kTiles;
        struct Tile {
            u32x4 k[W / 64];
            uint32_t pair[2];
            float w;  // of position `mine`
        };
        const int mine = r16 + 16 * (g >> 1);  // whose sum this lane has in the end (odd g: a copy)
        auto load = [&](Tile& x, int u) {
            u = u < units ? u : units - 1;
            const uint8_t* tile = tiles + (int64_t)u * KvTile<W>::kBytes;
#pragma unroll
            for (int p = 0; p < W / 64; p++)
                x.k[p] = *(const u32x4*)(tile + p * 1024 + lane * 16);
#pragma unroll
            for (int a = 0; a < 2; a++)
                x.pair[a] = *(const uint32_t*)(tile + KvTile<W>::kKeyScales + 64 * a + 4 * r16);
            const int left = len - u * kKvTile;
            x.w = (weight + (int64_t)u * kKvTile)[mine < left ? mine : 0];
        };
        auto add = [&](Tile& x, int u) {
            h16x8 kf[2][W / 32];
#pragma unroll
            for (int a = 0; a < 2; a++)
#pragma unroll
                for (int s = 0; s < W / 32; s++) {
                    const int Q = a * (W / 32) + s;
                    kf[a][s] = kv_codes_less_8(x.k[Q >> 2][Q & 3]);
                }
            const float ks[2] = {kv_s(x.pair[0]), kv_s(x.pair[1])};
            const float kz[2] = {fmaf(8.f, ks[0], kv_z(x.pair[0])), fmaf(8.f, ks[1], kv_z(x.pair[1]))};
            const float before = x.w;
            load(x, u + 2 * du);
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
            // over the four lanes of a column, those of the second 16 columns to the upper half
            const auto halves = __builtin_amdgcn_permlane32_swap(__float_as_uint(sum[0]), __float_as_uint(sum[1]),
                                                                 false, false);
            float p, q;
            swap16(__uint_as_float(halves[0]) + __uint_as_float(halves[1]), &p, &q);
            if (!(g & 1) && mine < len - u * kKvTile)
                (weight + (int64_t)u * kKvTile)[mine] = before + (p + q);
        };
        // two tiles of a wave in flight
        Tile x, y;
        load(x, u0);
        __builtin_amdgcn_sched_barrier(0);
        load(y, u0 + du);
        __builtin_amdgcn_sched_barrier(0);
        for (int u = u0; u < units; u += 2 * du) {
            add(x, u);
            if (u + du < units)
                add(y, u + du);
        }
    }
}

}  // namespace

// Rows a workgroup takes (16 nt: three row tiles share a tile's unpacking; a fourth
// would spill), its items at most, and the workgroups that share the work: as many
// as the chip holds at once (3 a CU with one row tile, whose registers at 4 would
// spill, 2 with more), fewer where the slots cannot hold so many units.
struct KvPlan {
    int nt, wgs, shift;
    int64_t items;
};

static KvPlan kv_plan(const KvView& c, int32_t B, int32_t max_nodes, int32_t Hq)
{
    KvPlan p;
    const int rows = max_nodes * (Hq / c.H);
    p.nt = rows <= 16 ? 1 : rows <= 32 ? 2 : 3;
    p.items = (int64_t)B * c.H * ((rows + 16 * p.nt - 1) / (16 * p.nt));
    int64_t units = p.items * (c.tiles + (max_nodes + 31) / 32);
    for (p.shift = 0; units >= 0x7FFFFFFF; p.shift++)
        units = p.items * (((c.tiles + (max_nodes + 31) / 32) >> (p.shift + 1)) + 1);
    const int64_t fine = (units + kLeastShare - 1) / kLeastShare, most = ((fine < p.items ? p.items : fine) + 7) / 8 * 8;
    const int64_t chip = p.nt == 1 ? kMaxShares : 512;
    p.wgs = (int)(most < chip ? most : chip);
    return p;
}

static size_t kv_part_rows(const KvPlan& p) { return (size_t)(2 * p.wgs) * 16 * p.nt; }

size_t kv_attend_workspace_bytes(const KvView& c, int32_t B, int32_t max_nodes, int32_t Hq)
{
    const size_t n = kv_part_rows(kv_plan(c, B, max_nodes, Hq));
    return kMaxShares * sizeof(KvCut) + n * (c.W + 2) * sizeof(float);
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
    hipLaunchKernelGGL(kv_join_kernel<W>, grid, dim3(256), 0, stream, A, 16 * p.nt);
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
    A.cuts = (KvCut*)workspace;
    A.part_o = (float*)(A.cuts + kMaxShares);
    A.part_ml = A.part_o + kv_part_rows(p) * c.W;
    A.q_ld = q_ld;
    A.ld = ld;
    A.B = B;
    A.Hq = Hq;
    A.G = Hq / c.H;
    A.max_nodes = max_nodes;
    A.shift = p.shift;
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
    // two tiles a wave at least, and as many workgroups as the chip holds at once (4 a
    // CU: 2,048 take 1.03 to 1.13 of the time, equal shares of all tiles whatever the
    // lengths 0.95 to 1.12)
    const int64_t heads = (int64_t)B * c.H, most = (c.tiles + 7) / 8;
    int64_t blocks = (1024 + heads - 1) / heads;
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
