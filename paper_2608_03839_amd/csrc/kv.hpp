// The 4-bit key/value cache: layout and helpers shared by its kernels
// (internal only).  The buffer layout is described in include/oilbird.h.
#pragma once

#include "common.hpp"
#include "internal.hpp"

namespace oil {

constexpr int kKvTile = 32;  // positions per tile

// Geometry of a tile for heads padded to W values (64 or 128).
template <int W>
struct KvTile {
    static constexpr int kValues = W * 16;            // byte offset of the values' codes
    static constexpr int kKeyScales = W * 32;         // (s, z) bf16 pairs of the keys
    static constexpr int kValueScales = W * 32 + 128; // and of the values
    static constexpr int kBytes = W * 32 + 256;
    static constexpr int kWords = W * 4;              // dwords of codes a side
};

// Words of a slot's state.
enum { kKvLen = 0, kKvNext = 1, kKvTicket = 2 };

// The slot that request b of a call is held in, or -1.
__device__ __forceinline__ int kv_slot(const KvView& c, const int32_t* slots, int b)
{
    const int s = slots ? slots[b] : b;
    return s >= 0 && s < c.n_slots ? s : -1;
}

__device__ __forceinline__ int32_t kv_len(const KvView& c, int slot)
{
    const int32_t n = c.state[4 * (int64_t)slot + kKvLen];
    return n < 0 ? 0 : n > c.cap ? (int32_t)c.cap : n;
}

__device__ __forceinline__ uint8_t* kv_tiles(const KvView& c, int slot, int h)
{
    return c.codes + ((int64_t)slot * c.H + h) * c.tiles * c.tile_bytes;
}

__device__ __forceinline__ int64_t kv_row(const KvView& c, int slot, int h)
{
    return ((int64_t)slot * c.H + h) * c.cap;
}

// Rows a request names (see oil_kv_append): how many, and the r-th.  `ids` and
// `bound` are LDS of the block, which calls this as a whole.
__device__ __forceinline__ int kv_count(const int32_t* nodes, const int32_t* count, int b, int max_rows, int* bound)
{
    if (!count)
        return max_rows;
    int n = count[b];
    if (!nodes)
        return n < 0 ? 0 : n > max_rows ? max_rows : n;
    n = n < 0 ? 0 : n > max_rows - 1 ? max_rows - 1 : n;
    if (threadIdx.x == 0)
        *bound = n;
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += blockDim.x) {
        const int id = nodes[(int64_t)b * max_rows + i];
        if (id < 0 || id >= max_rows)
            atomicMin(bound, i);
    }
    __syncthreads();
    return 1 + *bound;
}

__device__ __forceinline__ int kv_source(const int32_t* nodes, int b, int max_rows, int r)
{
    return !nodes || r == 0 ? r : nodes[(int64_t)b * max_rows + r - 1];
}

// The dword of the codes (either side) at linear dword w: its 16-byte plane,
// lane and place give dword Q of the lane.
__device__ __forceinline__ void kv_word(int w, int* Q, int* lane)
{
    *Q = (w >> 8) * 4 + (w & 3);
    *lane = (w >> 2) & 63;
}

__device__ __forceinline__ int kv_word_at(int Q, int lane) { return (Q >> 2) * 256 + lane * 4 + (Q & 3); }

// Nibble of element e of a dword.
__device__ __forceinline__ int kv_nibble(int e) { return (e >> 1) + 4 * (e & 1); }

__device__ __forceinline__ int kv_code(uint32_t word, int e) { return (word >> (4 * kv_nibble(e))) & 15; }

__device__ __forceinline__ float kv_s(uint32_t pair) { return __uint_as_float(pair << 16); }
__device__ __forceinline__ float kv_z(uint32_t pair) { return __uint_as_float(pair & 0xFFFF0000u); }

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float floatx2 __attribute__((ext_vector_type(2)));

// Two values in bf16, to the nearest even.
__device__ __forceinline__ uint32_t pack_bf16(float a, float b)
{
    const floatx2 x = {a, b};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(x, bf16x2));
}

}  // namespace oil
