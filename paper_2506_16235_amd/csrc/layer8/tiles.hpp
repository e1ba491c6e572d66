/*
 * Tiles in LDS for the matrix instructions, shared by the products and the weight gradient.
 *
 * A tile's row is 128 bytes of the summed dimension (128 codes, or 64 bfloat16) in eight chunks of 16 bytes.  Two neighbouring
 * rows share 256 bytes, all the banks of LDS once, and their sixteen chunks lie there in an order that is another one for each
 * of 16 neighbouring pairs, so that the same chunk of 32 rows, which is what a matrix instruction reads, meets every bank equally
 * often.  Rows 32 apart have the same order: one address per operand and chunk does for all of a wavefront's blocks.
 */
#ifndef NSML_LAYER8_TILES_HPP
#define NSML_LAYER8_TILES_HPP

#include "layer8.hpp"

namespace {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef int v16i __attribute__((ext_vector_type(16)));
typedef float v16f __attribute__((ext_vector_type(16)));
typedef __bf16 v8bf __attribute__((ext_vector_type(8)));

/* Longest row stride: the rows of a tile lie within 32 bits of its first. */
constexpr uint64_t MAX_LD = 1u << 22;

__device__ __forceinline__ uint32_t place(uint32_t row, uint32_t chunk)
{
    return row / 2u * 256u + ((((row % 2u) * 8u + chunk) ^ (row / 2u % 16u)) * 16u);
}
constexpr uint32_t BLOCK = 32 * 128;                 /* bytes from one block of 32 rows to the next */

/* What a lane gives a matrix instruction of 32 x 32: 16 bytes of one row of a block. */
__device__ __forceinline__ v4i frag(const uint8_t *at) { return *reinterpret_cast<const v4i *>(at); }
/* The row of a 32 x 32 result that register r of a lane holds; its column is lane % 32. */
__device__ __forceinline__ uint32_t acc_row(int r, uint32_t lane) { return (uint32_t)(r % 4 + r / 4 * 8) + lane / 32u * 4u; }

__device__ __forceinline__ void wait_loads() { __builtin_amdgcn_s_waitcnt(0x0F70); }       /* vmcnt(0) */

/* ROWS x 128 bytes from memory straight into LDS by W wavefronts: eight rows per instruction, lanes permuted within their row.
 * Rows beyond `rows` are given the last one's contents. */
template <int ROWS, int W>
__device__ __forceinline__ void load_tile(const int8_t *from, uint64_t ld, uint32_t rows, uint8_t *to, uint32_t wave, uint32_t lane)
{
#pragma unroll
    for (int i = 0; i < ROWS / 8 / W; i++) {
        const uint32_t r0 = (i * W + wave) * 8u, pair = r0 / 2u + lane / 16u, at = (lane % 16u) ^ (pair % 16u);
        const uint32_t off = min(pair * 2u + at / 8u, rows - 1) * (uint32_t)ld + at % 8u * 16u;
        __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)(from + off),
                                         (__attribute__((address_space(3))) void *)(to + r0 * 128u), 16, 0, 0);
    }
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

/* The last stage of rows that end within it, `bytes` (< 128) of each: through registers, with zeros from there on.  Nothing is
 * read beyond the chunk of 16 bytes that a row ends in. */
template <int ROWS, int W>
__device__ __forceinline__ void load_tail(const int8_t *from, uint64_t ld, uint32_t rows, uint32_t bytes, uint8_t *to, uint32_t thread)
{
#pragma unroll
    for (uint32_t i = thread; i < ROWS * 8u; i += W * 64u) {
        const uint32_t row = i / 8u, chunk = i % 8u;
        v4i v = {};
        if (chunk * 16u < bytes) v = first_bytes(*reinterpret_cast<const v4i *>(from + min(row, rows - 1) * (uint32_t)ld + chunk * 16u), (int)(bytes - chunk * 16u));
        *reinterpret_cast<v4i *>(to + place(row, chunk)) = v;
    }
}

/* Which tile a workgroup takes.  Workgroups go round the eight dies; each die gets a run of neighbouring tiles, in bands of
 * eight tile rows, so that what its workgroups read at the same time is shared in its cache. */
struct Tile { uint32_t row, col; };
__device__ __forceinline__ Tile tile_of(uint32_t id, uint32_t rows, uint32_t cols)
{
    const uint32_t total = rows * cols, per = total / 8u, more = total % 8u, die = id % 8u;
    const uint32_t i = die * per + min(die, more) + id / 8u;
    const uint32_t band = i / (8u * cols), first = band * 8u, high = min(rows - first, 8u), in = i - band * 8u * cols;
    return {first + in % high, in / high};
}

}  // namespace

#endif
