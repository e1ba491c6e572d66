/*
 * Tiles in LDS for the matrix instructions, shared by the products and the weight gradient.
 *
 * The products' rows, and those of the weight gradient in parts, are 64 bytes of the summed dimension (spot), else 128 (place).  Measured here for accesses of 16
 * bytes per lane: a read takes 16 lanes a cycle (lanes 0-3, 12-15, 20-23 and 24-27, and so on) and a write eight neighbouring
 * ones, over 256 and 128 bytes of banks.  So the chunks of 16 bytes lie within 256 bytes in an order that differs from pair (place) or
 * four (spot) of rows to the next, such that reads of the same chunk of 32 rows, and writes of the same chunk of
 * consecutive rows, meet no bank twice.  Rows 32 apart have the same order: one address per operand does for all blocks.
 */
#ifndef NSML_LAYER8_TILES_HPP
#define NSML_LAYER8_TILES_HPP

#include "layer8.hpp"

namespace {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef int v16i __attribute__((ext_vector_type(16)));
typedef float v16f __attribute__((ext_vector_type(16)));
typedef __bf16 v8bf __attribute__((ext_vector_type(8)));

/* Words at an address of any alignment. */
typedef uint32_t Loose2 __attribute__((ext_vector_type(2), aligned(1)));
typedef uint32_t Loose4 __attribute__((ext_vector_type(4), aligned(1)));

/* Longest row stride: the rows of a tile lie within 32 bits of its first. */
constexpr uint64_t MAX_LD = 1u << 22;

__device__ __forceinline__ uint32_t place(uint32_t row, uint32_t chunk)
{
    return row / 2u * 256u + ((row % 2u * 12u ^ chunk ^ row / 2u % 8u) * 16u);
}
__device__ __forceinline__ uint32_t spot(uint32_t row, uint32_t chunk)
{
    return row / 4u * 256u + (((row % 4u * 4u + chunk) ^ (row / 4u % 4u)) * 16u);
}

/* What a lane gives a matrix instruction of 32 x 32: 16 bytes of one row of a block. */
__device__ __forceinline__ v4i frag(const uint8_t *at) { return *reinterpret_cast<const v4i *>(at); }
/* The row of a 32 x 32 result that register r of a lane holds; its column is lane % 32. */
__device__ __forceinline__ uint32_t acc_row(int r, uint32_t lane) { return (uint32_t)(r % 4 + r / 4 * 8) + lane / 32u * 4u; }

/* Until this wavefront's reads of LDS are done. */
__device__ __forceinline__ void wait_lds() { __builtin_amdgcn_s_waitcnt(0xC07F); }
/* Until at most N of this wavefront's loads are on their way, and its accesses to LDS are done; then until all wavefronts are here.
 * (__syncthreads would wait for every load that goes straight to LDS.) */
template <int N> __device__ __forceinline__ void loads_sync()
{
    static_assert(N < 64, "six bits");
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0x0070 | (N & 15) | (N >> 4 << 14));
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

/* The first n bytes of a chunk, zeros after them. */
__device__ __forceinline__ v4i first_bytes(v4i v, int n)
{
#pragma unroll
    for (int i = 0; i < 4; i++) {
        const int have = n - i * 4;
        v[i] = have >= 4 ? v[i] : have <= 0 ? 0 : (int)((uint32_t)v[i] & ((1u << (8 * have)) - 1u));
    }
    return v;
}

/* Which tile a workgroup takes.  Workgroups go round the eight dies; each die gets a run of neighbouring tiles, in bands of
 * four tile rows, so that what its 32 workgroups read at the same time is shared in its cache (bands of 8 and 16: 1 and 2 % more time). */
struct Tile { uint32_t row, col; };
__device__ __forceinline__ Tile tile_of(uint32_t id, uint32_t rows, uint32_t cols)
{
    const uint32_t total = rows * cols, per = total / 8u, more = total % 8u, die = id % 8u;
    const uint32_t i = die * per + min(die, more) + id / 8u;
    const uint32_t band = i / (4u * cols), first = band * 4u, high = min(rows - first, 4u), in = i - band * 4u * cols;
    return {first + in % high, in / high};
}

}  // namespace

#endif
