/*
 * What the kernels of the 8-bit layer share: loads and stores of any alignment, reductions, the two codings.
 * Included by rows.hip, products.hip and wgrad.hip; not a public header.
 */
#ifndef NSML_LAYER8_HPP
#define NSML_LAYER8_HPP

#include <hip/hip_runtime.h>

#include <cstdint>
#include <initializer_list>

#include "nsml.h"

namespace {

typedef __bf16 bf16;
typedef _Float16 f16;

/* Rows of odd widths start anywhere: 16 bytes at an address of any alignment are one instruction on this
 * GPU, as aligned ones are. */
template <int N> struct __attribute__((packed, aligned(1))) Bytes { uint32_t w[N]; };

/* Barrier of a workgroup with the wait for this wavefront's own LDS accesses written out: the compiler has
 * dropped that wait where the accesses come over a loop's back edge. */
__device__ __forceinline__ void wg_sync()
{
    __builtin_amdgcn_s_waitcnt(0xC07F);              /* lgkmcnt(0) */
    __syncthreads();
}

__device__ __forceinline__ float from_bits(uint32_t u) { return __builtin_bit_cast(float, u); }
__device__ __forceinline__ uint32_t to_bits(float f) { return __builtin_bit_cast(uint32_t, f); }

/* Eight neighbours of a row as they are in memory; the ones from n on are 0 and not read. */
template <typename T> using Raw = Bytes<sizeof(T) * 2>;
template <typename T> __device__ __forceinline__ Raw<T> load_raw(const T *p, int n)
{
    if (n >= 8) return *reinterpret_cast<const Raw<T> *>(p);
    T x[8];
#pragma unroll
    for (int i = 0; i < 8; i++) x[i] = i < n ? p[i] : (T)0.0f;
    Raw<T> r;
    __builtin_memcpy(&r, x, sizeof x);
    return r;
}
template <typename T> __device__ __forceinline__ void from_raw(const Raw<T> &r, float (&v)[8])
{
    T x[8];
    __builtin_memcpy(x, &r, sizeof x);
#pragma unroll
    for (int i = 0; i < 8; i++) v[i] = (float)x[i];
}

/* Eight neighbours of a row as binary32; the ones from n on are 0 and not read. */
template <typename T> __device__ __forceinline__ void load8(const T *p, int n, float (&v)[8])
{
    if (n >= 8) {
        const auto b = *reinterpret_cast<const Bytes<sizeof(T) * 2> *>(p);
        T x[8];
        __builtin_memcpy(x, &b, sizeof x);
#pragma unroll
        for (int i = 0; i < 8; i++) v[i] = (float)x[i];
    } else {
#pragma unroll
        for (int i = 0; i < 8; i++) v[i] = i < n ? (float)p[i] : 0.0f;
    }
}
template <typename T> __device__ __forceinline__ void store8(T *p, int n, const float (&v)[8])
{
    T x[8];
#pragma unroll
    for (int i = 0; i < 8; i++) x[i] = (T)v[i];
    if (n >= 8) {
        Bytes<sizeof(T) * 2> b;
        __builtin_memcpy(&b, x, sizeof x);
        *reinterpret_cast<Bytes<sizeof(T) * 2> *>(p) = b;
    } else {
#pragma unroll
        for (int i = 0; i < 8; i++)
            if (i < n) p[i] = x[i];
    }
}

/* Four, the ones from n on left alone. */
__device__ __forceinline__ void load4(const float *p, int n, float (&v)[4])
{
    if (n == 4) {
        const auto b = *reinterpret_cast<const Bytes<4> *>(p);
        __builtin_memcpy(v, &b, 16);
    } else {
#pragma unroll
        for (int i = 0; i < 4; i++) v[i] = i < n ? p[i] : 0.0f;
    }
}
template <typename T> __device__ __forceinline__ void store4(T *p, int n, const float (&v)[4])
{
    T x[4];
#pragma unroll
    for (int i = 0; i < 4; i++) x[i] = (T)v[i];
    if (n == 4) {
        Bytes<sizeof(T)> b;
        __builtin_memcpy(&b, x, sizeof x);
        *reinterpret_cast<Bytes<sizeof(T)> *>(p) = b;
    } else {
#pragma unroll
        for (int i = 0; i < 4; i++)
            if (i < n) p[i] = x[i];
    }
}

/* Magnitudes are compared as bit patterns: an infinity or NaN comes out on top, where fmax would drop it. */
__device__ __forceinline__ uint32_t mag(float v) { return to_bits(v) & 0x7FFFFFFFu; }
constexpr uint32_t MAG_INF = 0x7F800000u;
constexpr uint32_t MAG_TINY = 15u << 23;             /* 2^-112 */

/* Nearest whole number of |v| < 2^22, ties to even: its low byte in two's complement is the sum's low byte. */
__device__ __forceinline__ uint32_t code(float v) { return to_bits(v + 12582912.0f); }
__device__ __forceinline__ uint32_t pack4(uint32_t a, uint32_t b, uint32_t c, uint32_t d)
{
    const uint32_t ab = __builtin_amdgcn_perm(b, a, 0x0C0C0400u), cd = __builtin_amdgcn_perm(d, c, 0x0C0C0400u);
    return __builtin_amdgcn_perm(cd, ab, 0x05040100u);
}

/* Scale of a row of absmax `m` and what its values are multiplied by for their codes. */
struct RowCode { float scale, inv; };
__device__ __forceinline__ RowCode row_code(uint32_t m)
{
    if (m >= MAG_INF) return {from_bits(0x7FC00000u), 0.0f};
    if (m < MAG_TINY) return {0.0f, 0.0f};
    return {from_bits(m) / 127.0f, 127.0f / from_bits(m)};
}
/* Codes of eight values; inv == 0 gives zeros whatever the values are. */
__device__ __forceinline__ uint2 row_codes8(const float (&t)[8], float inv)
{
    if (inv == 0.0f) return make_uint2(0, 0);
    uint32_t c[8];
#pragma unroll
    for (int i = 0; i < 8; i++) c[i] = code(t[i] * inv);
    return make_uint2(pack4(c[0], c[1], c[2], c[3]), pack4(c[4], c[5], c[6], c[7]));
}

/* Exponent byte of a checkpoint's block of absmax `m`.  2^(e - 127) <= absmax / 64, so codes stay below 128. */
__device__ __forceinline__ uint32_t ckpt_exp(uint32_t m)
{
    const int e = (int)(m >> 23) - 6;                /* floor(log2) + 127 - 6; subnormals count as 2^-127 */
    return m >= MAG_INF ? 255u : (uint32_t)(e < 1 ? 1 : e);
}
__device__ __forceinline__ float ckpt_scale(uint32_t e) { return from_bits(e << 23); }      /* 2^(e - 127); e = 255: infinity */
/* Codes of eight values of a block: held to 127 steps, divided by the step (exact: powers of two) and rounded, the last two in one
 * instruction whose sum has the code in its low byte. */
__device__ __forceinline__ uint2 ckpt_codes8(const float (&x)[8], uint32_t e)
{
    if (e == 255u) return make_uint2(0, 0);
    const float inv = from_bits((254u - e) << 23), most = 127.0f * ckpt_scale(e);
    uint32_t c[8];
#pragma unroll
    for (int i = 0; i < 8; i++) c[i] = to_bits(__builtin_fmaf(__builtin_amdgcn_fmed3f(x[i], -most, most), inv, 12582912.0f));
    return make_uint2(pack4(c[0], c[1], c[2], c[3]), pack4(c[4], c[5], c[6], c[7]));
}
__device__ __forceinline__ void codes8(uint2 w, float (&v)[8])
{
#pragma unroll
    for (int i = 0; i < 4; i++) {
        v[i] = (float)(int8_t)(w.x >> (8 * i));
        v[4 + i] = (float)(int8_t)(w.y >> (8 * i));
    }
}
__device__ __forceinline__ uint32_t max8(const float (&v)[8], uint32_t m)
{
#pragma unroll
    for (int i = 0; i < 8; i++) m = max(m, mag(v[i]));
    return m;
}

/* Most of what the four lanes of a quad have: a checkpoint's block is four lanes with eight values each. */
__device__ __forceinline__ uint32_t quad_max(uint32_t m)
{
    m = max(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0xB1, 0xF, 0xF, true));       /* lanes 1 0 3 2 */
    return max(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0x4E, 0xF, 0xF, true));    /* lanes 2 3 0 1 */
}

/* One matrix in a kernel's arguments. */
template <typename T> struct Mat {
    T *p;
    uint64_t ld;
    __device__ __forceinline__ T *at(uint64_t row, uint32_t col) const { return p + row * ld + col; }
};
struct Ckpt {
    int8_t *q;
    uint8_t *e;
    uint64_t ldq, lde;
};
/* Eight neighbours from column c (a multiple of 8) of a checkpoint's row. */
__device__ __forceinline__ void ckpt_load8(const Ckpt &k, uint64_t row, uint32_t c, float (&v)[8])
{
    codes8(*reinterpret_cast<const uint2 *>(k.q + row * k.ldq + c), v);
    const float s = ckpt_scale(k.e[row * k.lde + c / 32u]);
#pragma unroll
    for (int i = 0; i < 8; i++) v[i] *= s;
}
/* A lane's eight neighbours into a checkpoint; the lanes of a quad hold a block between them (zeros beyond the row)
 * and all come here. */
__device__ __forceinline__ void ckpt_store8(const Ckpt &k, uint64_t row, uint32_t c, uint32_t cols, const float (&v)[8])
{
    const uint32_t e = ckpt_exp(quad_max(max8(v, 0u)));
    const uint2 w = ckpt_codes8(v, e);
    if (c < cols) {
        *reinterpret_cast<uint2 *>(k.q + row * k.ldq + c) = w;
        if (c % 32u == 0) k.e[row * k.lde + c / 32u] = (uint8_t)e;
    }
}

/* ---------------------------------------------------------------- host */

constexpr uint32_t MAX_COLS = 0x7FFFFF00u;          /* so that column numbers rounded up to a tile stay below 2^31 */
inline bool at_multiple(const void *p, uintptr_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }
inline bool whole_lines(const void *p, uint64_t row_bytes) { return at_multiple(p, 128) && row_bytes % 128 == 0; }
inline uint32_t type_bytes(int type) { return type == NSML_F32 ? 4u : 2u; }
inline bool bad_type(int type) { return type != NSML_F32 && type != NSML_BF16 && type != NSML_F16; }
inline bool bad_mat(const void *p, int type, uint64_t ld, uint32_t cols)
{
    return !p || ld < cols || !at_multiple(p, type_bytes(type));
}
inline bool bad_f32(const void *p) { return !p || !at_multiple(p, 4); }
inline bool bad_codes(const void *p, uint64_t ld, uint32_t cols) { return !p || ld < cols || ld % 16 != 0 || !at_multiple(p, 16); }
inline bool bad_ckpt(const nsml_ckpt8 *k, uint32_t cols)
{
    return !k || !k->e || k->lde < (cols + 31u) / 32u || bad_codes(k->q, k->ldq, cols);
}
inline Ckpt ckpt_of(const nsml_ckpt8 *k) { return k ? Ckpt{k->q, k->e, k->ldq, k->lde} : Ckpt{nullptr, nullptr, 0, 0}; }

/* The bytes of a matrix: `rows` times `width`, `pitch` from row to row. */
struct Area { uintptr_t at; uint64_t rows, pitch, width; };
inline Area area(const void *p, uint64_t rows, uint64_t pitch, uint64_t width) { return {reinterpret_cast<uintptr_t>(p), p ? rows : 0, pitch, width}; }
inline Area area(const void *p, int type, uint64_t rows, uint64_t ld, uint32_t cols) { return area(p, rows, ld * type_bytes(type), (uint64_t)cols * type_bytes(type)); }
inline Area floats(const float *p, uint64_t n) { return area(p, 1, n * 4u, n * 4u); }
inline Area codes_area(const int8_t *p, uint64_t rows, uint64_t ld, uint32_t cols) { return area(p, rows, ld, ((uint64_t)cols + 15u) / 16u * 16u); }
inline Area exps_area(const nsml_ckpt8 *k, uint64_t rows, uint32_t cols) { return area(k ? k->e : nullptr, rows, k ? k->lde : 0, (cols + 31u) / 32u); }
inline Area codes_area(const nsml_ckpt8 *k, uint64_t rows, uint32_t cols) { return codes_area(k ? k->q : nullptr, rows, k ? k->ldq : 0, cols); }
/* Whether two matrices have a byte in common.  Matrices side by side in one (the same pitch) do not. */
inline bool meet(Area a, Area b)
{
    if (a.rows == 0 || b.rows == 0 || a.width == 0 || b.width == 0) return false;
    if (b.at < a.at) {
        const Area c = a;
        a = b, b = c;
    }
    if (b.at >= a.at + (a.rows - 1) * a.pitch + a.width) return false;
    if (a.rows == 1) return true;
    const uint64_t in = (b.at - a.at) % a.pitch;
    if (in < a.width) return true;
    if (b.rows == 1 || b.pitch == a.pitch) return in + b.width > a.pitch;        /* the row of a behind it is there: b begins before a ends */
    uint64_t i = (b.at - a.at) / a.pitch + 1, j = 0;
    while (i < a.rows && j < b.rows) {
        const uintptr_t x = a.at + i * a.pitch, y = b.at + j * b.pitch;
        if (x + a.width <= y) i++;
        else if (y + b.width <= x) j++;
        else return true;
    }
    return false;
}
/* Whether one that is written meets another, or one that is read. */
inline bool clash(std::initializer_list<Area> written, std::initializer_list<Area> read)
{
    for (const Area *w = written.begin(); w != written.end(); w++) {
        for (const Area *o = written.begin(); o != w; o++)
            if (meet(*w, *o)) return true;
        for (const Area &r : read)
            if (meet(*w, r)) return true;
    }
    return false;
}
/* What is read, but nothing where it is the very matrix that is written: where every thread reads an element before it writes it. */
inline Area apart(Area read, const Area &written)
{
    if (read.at == written.at && read.rows == written.rows && read.width == written.width && (read.pitch == written.pitch || read.rows == 1)) read.rows = 0;
    return read;
}
inline int launched() { return hipGetLastError() == hipSuccess ? NSML_OK : NSML_EHIP; }
template <typename T> Mat<T> mat(void *p, uint64_t ld) { return {static_cast<T *>(p), ld}; }
template <typename T> Mat<const T> mat(const void *p, uint64_t ld) { return {static_cast<const T *>(p), ld}; }

}  // namespace

#endif
