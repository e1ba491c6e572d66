/*
 * The 8-bit layer's passes over rows: coding by rows, the norm and its gradient, the gated activation and its
 * gradient, checkpoints written and read.
 *
 * All of them are bound by memory (1 to 6 operations per byte): every element is read once, what a row's absmax,
 * sum or mean is needed for waits in registers, and what is written goes out in the same kernel.
 */
#include "layer8.hpp"

#include <cfloat>

namespace {

/* ---------------------------------------------------------------- reductions */

template <int CTRL> __device__ __forceinline__ uint32_t dpp(uint32_t v)
{
    return (uint32_t)__builtin_amdgcn_mov_dpp((int)v, CTRL, 0xF, 0xF, true);
}
/* Over the 64 lanes, in one order: neighbours, pairs, halves and mirror images of 16, then the four sixteens. */
template <typename F> __device__ __forceinline__ uint32_t wave_all(uint32_t v, F f)
{
    v = f(v, dpp<0xB1>(v));
    v = f(v, dpp<0x4E>(v));
    v = f(v, dpp<0x141>(v));
    v = f(v, dpp<0x140>(v));
    const uint32_t a = __builtin_amdgcn_readlane(v, 0), b = __builtin_amdgcn_readlane(v, 16);
    const uint32_t c = __builtin_amdgcn_readlane(v, 32), d = __builtin_amdgcn_readlane(v, 48);
    return f(f(a, b), f(c, d));
}
__device__ __forceinline__ uint32_t max_of(uint32_t a, uint32_t b) { return max(a, b); }
__device__ __forceinline__ uint32_t sum_of(uint32_t a, uint32_t b) { return to_bits(from_bits(a) + from_bits(b)); }

/* ---------------------------------------------------------------- rows that are coded as a whole */

/* T threads hold a row, V times eight neighbours each; V == 0: rows wider than registers hold are read twice.
 * OP: load() gives the values to code and adds to the row's sum (SUMS; again() once more, in another unit), done() gets the sum and
 * the row's code, store() writes beside the codes.  SHORT: two times eight per thread at most. */
template <int T, int V, typename OP>
__global__ void __launch_bounds__(T < 256 ? 256 : T) k_rows(OP op, uint64_t rows, uint32_t cols)
{
    constexpr int B = T < 256 ? 256 : T, R = B / T, W = T / 64, N = V ? V : 1;
    __shared__ uint32_t part[2][2][W > 1 ? W : 1];
    const uint32_t t = threadIdx.x % T;
    uint32_t turn = 0;
    for (uint64_t row = (uint64_t)blockIdx.x * R + threadIdx.x / T; row < rows; row += (uint64_t)gridDim.x * R, turn ^= 1u) {
        typename OP::Reg reg[N];
        uint32_t m = 0;
        float sum = 0.0f;
        auto at = [&](uint32_t i) { return (i * T + t) * 8u; };
        auto left = [&](uint32_t c) { return c < cols ? (int)min(cols - c, 8u) : 0; };
        const uint32_t steps = V ? V : (cols + T * 8u - 1u) / (T * 8u);
        if (V) {
#pragma unroll
            for (int i = 0; i < N; i++) op.load(row, at(i), left(at(i)), reg[i], m, sum, true);
        } else {
            for (uint32_t i = 0; i < steps; i++) op.load(row, at(i), left(at(i)), reg[0], m, sum, true);
        }
        m = wave_all(m, max_of);
        if (OP::SUMS) sum = from_bits(wave_all(to_bits(sum), sum_of));
        if (W > 1) {
            if (threadIdx.x % 64 == 0) {
                part[turn][0][threadIdx.x / 64] = m;
                if (OP::SUMS) part[turn][1][threadIdx.x / 64] = to_bits(sum);
            }
            wg_sync();                       /* the other half of `part` is this one's past: one barrier per row does */
            m = 0;
            sum = 0.0f;
#pragma unroll
            for (int i = 0; i < W; i++) {
                m = max(m, part[turn][0][i]);
                if (OP::SUMS) sum += from_bits(part[turn][1][i]);
            }
        }
        if constexpr (OP::SUMS) {
            /* The same for all threads of a row. */
            if (__builtin_expect(op.left_range(sum), 0)) {
                const float unit = sum > 1.0f ? 0x1p-75f : 0x1p+75f;
                uint32_t thread = threadIdx.x;
                asm volatile("" : "+v"(thread));     /* nothing of this is kept in registers where it is not needed */
                sum = 0.0f;
#pragma unroll
                for (int i = 0; i < N; i++) sum = op.again(reg[i], unit, sum);
                sum = from_bits(wave_all(to_bits(sum), sum_of));
                if (W > 1) {
                    wg_sync();               /* the first sum's parts have been read */
                    if (thread % 64 == 0) part[turn][1][thread / 64] = to_bits(sum);
                    wg_sync();
                    sum = 0.0f;
#pragma unroll 1
                    for (int i = 0; i < W; i++) sum += from_bits(part[turn][1][i]);
                }
                op.mean(sum, cols, unit);
            } else {
                op.mean(sum, cols, 1.0f);
            }
        }
        const RowCode rc = row_code(m);
        op.done(row, t == 0, rc);
        if (V) {
#pragma unroll
            for (int i = 0; i < N; i++) {
                const uint32_t c = at(i);
                if (c < cols) *reinterpret_cast<uint2 *>(op.q.at(row, c)) = row_codes8(reg[i].t, rc.inv);
                op.store(row, c, cols, reg[i]);
            }
        } else {
            for (uint32_t i = 0; i < steps; i++) {
                const uint32_t c = at(i);
                uint32_t m2 = 0;
                float s2 = 0.0f;
                op.load(row, c, left(c), reg[0], m2, s2, false);
                if (c < cols) *reinterpret_cast<uint2 *>(op.q.at(row, c)) = row_codes8(reg[0].t, rc.inv);
                op.store(row, c, cols, reg[0]);
            }
        }
    }
}

template <int T, int V, typename OP> int go_rows(const OP &op, uint64_t rows, uint32_t cols, hipStream_t st)
{
    constexpr uint64_t R = T < 256 ? 256 / T : 1;
    const uint64_t blocks = (rows + R - 1) / R;
    k_rows<T, V, OP><<<(uint32_t)(blocks < (1u << 20) ? blocks : 1u << 20), T < 256 ? 256 : T, 0, st>>>(op, rows, cols);
    return launched();
}
/* A wavefront holds rows of up to 1024 columns, four up to 4096, eight up to 8192; beyond that as many as the operator's registers make
 * best: with few registers each, workgroups share a compute unit and one reads while the other computes, with more, less of them wait
 * at a row's barrier (rows of 11008 bfloat16 from memory, us for 1024 x 2, 768 x 2, 512 x 3, 256 x 6 threads times eights: gated activation of 4096 with
 * checkpoints 106, 80, 87, 125, of 8192 without 144, 97, 110, 168; q8_rows of 8192 with col_scale 70, 69, 67, 70; norm of 8192 with its checkpoint
 * 208, 151, 173, 199: there 512 was chosen when the norm took more registers). */
template <typename OP> int launch_rows(const OP &op, uint64_t rows, uint32_t cols, hipStream_t st)
{
    if (rows == 0) return NSML_OK;
    if (cols <= 512) return go_rows<64, 1>(op, rows, cols, st);
    if (cols <= 1024) return go_rows<64, 2>(op, rows, cols, st);
    if (cols <= 2048) return go_rows<256, 1>(op, rows, cols, st);
    if (cols <= 4096) return go_rows<256, 2>(op, rows, cols, st);
    if (cols <= 8192) return go_rows<512, 2>(op, rows, cols, st);
    if (cols <= 12288) return go_rows<OP::SHORT ? 768 : 512, OP::SHORT ? 2 : 3>(op, rows, cols, st);
    if (cols <= 16384) return go_rows<OP::SHORT ? 1024 : 512, OP::SHORT ? 2 : 4>(op, rows, cols, st);
    if constexpr (OP::SUMS) return go_rows<1024, 4>(op, rows, cols, st);          /* up to 32768 columns */
    else return cols <= 32768 ? go_rows<1024, 4>(op, rows, cols, st) : go_rows<1024, 0>(op, rows, cols, st);
}

template <typename T> struct OpRows {
    static constexpr bool SUMS = false, SHORT = false;
    struct Reg { float t[8]; };
    Mat<const T> x;
    const float *col;
    Mat<int8_t> q;
    float *scale;
    __device__ __forceinline__ void load(uint64_t row, uint32_t c, int n, Reg &r, uint32_t &m, float &, bool) const
    {
        load8(x.at(row, c), n, r.t);
        if (col) {
            float f[8];
            load8(col + c, n, f);
#pragma unroll
            for (int i = 0; i < 8; i++) r.t[i] *= f[i];
        }
        m = max8(r.t, m);
    }
    __device__ __forceinline__ void done(uint64_t row, bool first, RowCode rc) const
    {
        if (first) scale[row] = rc.scale;
    }
    __device__ __forceinline__ void store(uint64_t, uint32_t, uint32_t, const Reg &) const {}
};

/* The norm: codes are those of gamma * h, so that they wait for the absmax alone; the mean of h^2, which comes out of
 * the same reduction, goes into the scale. */
template <typename T> struct OpNorm {
    static constexpr bool SUMS = true, SHORT = false;
    struct Reg { float t[8], h[8]; };
    Mat<const T> x, res;
    const float *gamma;
    float eps;
    Mat<T> h;
    Mat<int8_t> q;
    float *scale, *rstd;
    Ckpt xhat;
    float r = 0.0f;                          /* the row's 1 / rms */
    __device__ __forceinline__ void load(uint64_t row, uint32_t c, int n, Reg &g, uint32_t &m, float &sum, bool first) const
    {
        load8(x.at(row, c), n, g.h);
        if (res.p) {
            float f[8];
            load8(res.at(row, c), n, f);
#pragma unroll
            for (int i = 0; i < 8; i++) g.h[i] = (float)(T)(g.h[i] + f[i]);
            if (first && n) store8(h.at(row, c), n, g.h);
        }
#pragma unroll
        for (int i = 0; i < 8; i++) {
            sum = __builtin_fmaf(g.h[i], g.h[i], sum);
            g.t[i] = g.h[i];
        }
        if (gamma) {
            float f[8];
            load8(gamma + c, n, f);
#pragma unroll
            for (int i = 0; i < 8; i++) g.t[i] *= f[i];
        }
        m = max8(g.t, m);
    }
    /* Whether the sum of squares has left binary32's range, or squares that count may have: they are then added once more in a unit, a
     * power of two, that brings them back (a sum below 2^-75 to one below 2^75; an infinity among the values stays one). */
    __device__ __forceinline__ bool left_range(float sum) const { return sum > FLT_MAX || (sum < 0x1p-75f && eps < 0x1p-90f); }
    __device__ __forceinline__ float again(const Reg &g, float unit, float sum) const
    {
#pragma unroll
        for (int i = 0; i < 8; i++) {
            const float v = g.h[i] * unit;
            sum = __builtin_fmaf(v, v, sum);
        }
        return sum;
    }
    __device__ __forceinline__ void mean(float sum, uint32_t cols, float unit)
    {
        r = rsqrtf(sum / (float)cols + eps * unit * unit) * unit;
        if (r > FLT_MAX) r = FLT_MAX;        /* a row of zeros without eps: what it is multiplied by stays 0 */
    }
    __device__ __forceinline__ void done(uint64_t row, bool first, RowCode rc) const
    {
        if (first) {
            rstd[row] = r;
            scale[row] = rc.scale * r;
        }
    }
    __device__ __forceinline__ void store(uint64_t row, uint32_t c, uint32_t cols, const Reg &g) const
    {
        if (!xhat.q) return;
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; i++) v[i] = g.h[i] * r;
        ckpt_store8(xhat, row, c, cols, v);
    }
};

/* 1 / (1 + exp(-x)) by the GPU's exponential of two and reciprocal (a unit in the last place each); 0 and 1 at the infinities, 0 below 2^-126.
 * What is lost in rounding x log2(e), and what log2(e) lacks as binary32, the exponential turns into 1.25 |x| units of 2^-24: this one is within
 * (5 + 1.25 |x|) 2^-24 of the value, enough for what becomes codes (half a step is 2^-8 of a row's absmax).  Measured at -20: 14.2 units, by `sigmoid` 3.1. */
__device__ __forceinline__ float sigmoid_rough(float x)
{
    return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(x * -0x1.715476p+0f));
}
/* For gradients, which may be binary32: the rest of that product goes into a factor 1 + rest * ln 2.  Within 7 * 2^-24, for four
 * instructions more (the gradient takes no longer for them; the activation by the rough one, 4096 x 11008 without checkpoints, 52.0 us, by this 53.6). */
__device__ __forceinline__ float sigmoid(float x)
{
    const float v = __builtin_amdgcn_fmed3f(x, -200.0f, 200.0f);
    const float t = v * -0x1.715476p+0f;             /* log2(e) = 0x1.715476p+0 + 1.925963e-8 */
    const float f = __builtin_fmaf(__builtin_fmaf(v, -0x1.715476p+0f, -t), 0.693147181f, __builtin_fmaf(v, -1.334976e-8f, 1.0f));
    return __builtin_amdgcn_rcpf(__builtin_fmaf(__builtin_amdgcn_exp2f(t), f, 1.0f));
}

template <typename T> struct OpGlu {
    static constexpr bool SUMS = false, SHORT = true;
    struct Reg { float t[8]; };
    Mat<const T> gate, up;
    Mat<int8_t> q;
    float *scale;
    Ckpt kg, ku, ka;
    uint32_t cols;
    __device__ __forceinline__ void load(uint64_t row, uint32_t c, int n, Reg &r, uint32_t &m, float &, bool first) const
    {
        float g[8], u[8];
        load8(gate.at(row, c), n, g);
        load8(up.at(row, c), n, u);
        if (first && kg.q) ckpt_store8(kg, row, c, cols, g);
        if (first && ku.q) ckpt_store8(ku, row, c, cols, u);
#pragma unroll
        for (int i = 0; i < 8; i++) r.t[i] = g[i] * sigmoid_rough(g[i]) * u[i];
        m = max8(r.t, m);
    }
    __device__ __forceinline__ void done(uint64_t row, bool first, RowCode rc) const
    {
        if (first) scale[row] = rc.scale;
    }
    __device__ __forceinline__ void store(uint64_t row, uint32_t c, uint32_t n, const Reg &r) const
    {
        if (ka.q) ckpt_store8(ka, row, c, n, r.t);
    }
};

/* ---------------------------------------------------------------- elements and blocks */

/* Eight neighbours per thread, L threads side by side in a row, 256 / L rows per workgroup; workgroups side by side cover
 * a window that moves through memory. */
template <typename OP> __global__ void __launch_bounds__(256) k_each(OP op, uint64_t rows, uint32_t cols, uint32_t log2l)
{
    const uint32_t c = ((blockIdx.x << log2l) + (threadIdx.x & ((1u << log2l) - 1u))) * 8u;
    const uint32_t per = 256u >> log2l;
    const int n = c < cols ? (int)min(cols - c, 8u) : 0;
    for (uint64_t row = (uint64_t)blockIdx.y * per + (threadIdx.x >> log2l); row < rows; row += (uint64_t)gridDim.y * per)
        op.run(row, c, n, cols);
}
template <typename OP> int launch_each(const OP &op, uint64_t rows, uint32_t cols, hipStream_t st)
{
    if (rows == 0) return NSML_OK;
    const uint32_t vecs = (cols + 31u) / 32u * 4u;
    uint32_t log2l = 2;
    while (log2l < 8u && (1u << log2l) < vecs) log2l++;
    const uint64_t groups = (rows + (256u >> log2l) - 1) / (256u >> log2l);
    k_each<OP><<<dim3((vecs + (1u << log2l) - 1u) >> log2l, (uint32_t)(groups < 65535u ? groups : 65535u)), 256, 0, st>>>(op, rows, cols, log2l);
    return launched();
}

template <typename T> struct OpPack {
    Mat<const T> x;
    Ckpt k;
    __device__ __forceinline__ void run(uint64_t row, uint32_t c, int n, uint32_t cols) const
    {
        float v[8];
        load8(x.at(row, c), n, v);
        ckpt_store8(k, row, c, cols, v);
    }
};
template <typename T> struct OpUnpack {
    Ckpt k;
    Mat<T> out;
    __device__ __forceinline__ void run(uint64_t row, uint32_t c, int n, uint32_t) const
    {
        if (!n) return;
        float v[8];
        ckpt_load8(k, row, c, v);
        store8(out.at(row, c), n, v);
    }
};
template <typename T> struct OpValues {
    Mat<const int8_t> q;
    const float *scale;
    Mat<T> out;
    __device__ __forceinline__ void run(uint64_t row, uint32_t c, int n, uint32_t) const
    {
        if (!n) return;
        float v[8];
        codes8(*reinterpret_cast<const uint2 *>(q.at(row, c)), v);
        const float s = scale ? scale[row] : 1.0f;
#pragma unroll
        for (int i = 0; i < 8; i++) v[i] *= s;
        store8(out.at(row, c), n, v);
    }
};
template <typename T> struct OpGluBack {
    Mat<const T> da;
    Ckpt kg, ku;
    Mat<T> dg, du;
    __device__ __forceinline__ void run(uint64_t row, uint32_t c, int n, uint32_t) const
    {
        if (!n) return;
        float a[8], g[8], u[8];
        load8(da.at(row, c), n, a);
        ckpt_load8(kg, row, c, g);
        ckpt_load8(ku, row, c, u);
#pragma unroll
        for (int i = 0; i < 8; i++) {
            const float s = sigmoid(g[i]), d = a[i] * s;
            u[i] = d * u[i] * __builtin_fmaf(g[i], 1.0f - s, 1.0f);
            a[i] = d * g[i];
        }
        store8(dg.at(row, c), n, u);
        store8(du.at(row, c), n, a);
    }
};

/* ---------------------------------------------------------------- codes the other way round */

/* out[c, r] = q[r, c] by tiles of 128 x 128: 16 bytes of a row per lane into LDS, then 16 rows of four columns per thread, turned round by
 * permutations of bytes, and 16 bytes of a row out.  Eight lanes read, and write, a line of 128 bytes.  Rows of LDS are 33 words apart, the second
 * 64 eight words further, so that the 64 words that a wavefront reads lie in as many banks.  Bound by memory (11008 x 4096: 22.0 us
 * from memory, 4.1 TB/s, 15.0 where the codes are still in the last cache). */
__global__ void __launch_bounds__(256) k_turn(const int8_t *q, uint64_t ldq, int8_t *out, uint64_t ldo, uint32_t rows, uint32_t cols)
{
    __shared__ uint32_t tile[128 * 33 + 8];
    const uint32_t across = (cols + 127u) / 128u;
    const uint64_t tiles = (uint64_t)across * ((rows + 127u) / 128u);
    for (uint64_t id = blockIdx.x; id < tiles; id += gridDim.x) {
        const uint32_t r0 = (uint32_t)(id / across) * 128u, c0 = (uint32_t)(id % across) * 128u;
#pragma unroll
        for (uint32_t i = 0; i < 4; i++) {
            const uint32_t r = i * 32u + threadIdx.x / 8u, c = threadIdx.x % 8u * 16u;
            uint4 v = make_uint4(0, 0, 0, 0);
            if (r0 + r < rows && c0 + c < cols) v = *reinterpret_cast<const uint4 *>(q + (r0 + r) * ldq + c0 + c);
            uint32_t *to = tile + r * 33u + r / 64u * 8u + c / 4u;
            to[0] = v.x, to[1] = v.y, to[2] = v.z, to[3] = v.w;
        }
        wg_sync();
        const uint32_t part = threadIdx.x % 8u, four = threadIdx.x / 8u;
        const uint32_t *from = tile + part * 16u * 33u + part / 4u * 8u + four;
        uint32_t o[4][4];
#pragma unroll
        for (int g = 0; g < 4; g++) {
            uint32_t w[4];
#pragma unroll
            for (int i = 0; i < 4; i++) w[i] = from[(g * 4 + i) * 33];
            const uint32_t a = __builtin_amdgcn_perm(w[1], w[0], 0x05010400u), b = __builtin_amdgcn_perm(w[1], w[0], 0x07030602u);
            const uint32_t c = __builtin_amdgcn_perm(w[3], w[2], 0x05010400u), d = __builtin_amdgcn_perm(w[3], w[2], 0x07030602u);
            o[0][g] = __builtin_amdgcn_perm(c, a, 0x05040100u), o[1][g] = __builtin_amdgcn_perm(c, a, 0x07060302u);
            o[2][g] = __builtin_amdgcn_perm(d, b, 0x05040100u), o[3][g] = __builtin_amdgcn_perm(d, b, 0x07060302u);
        }
        if (r0 + part * 16u < rows)
#pragma unroll
            for (uint32_t j = 0; j < 4; j++) {
                const uint32_t c = c0 + four * 4u + j;
                if (c < cols) *reinterpret_cast<uint4 *>(out + c * ldo + r0 + part * 16u) = make_uint4(o[j][0], o[j][1], o[j][2], o[j][3]);
            }
        wg_sync();                           /* before the next tile goes to the same place */
    }
}

/* ---------------------------------------------------------------- gradient of the norm */

/* T threads hold a row; a workgroup takes every so many rows and keeps its share of dgamma in registers, one row of
 * `part` for each T threads at the end, which k_norm_sum adds up in order. */
template <typename X, int T, int V>
__global__ void __launch_bounds__(T < 256 ? 256 : T)
k_norm_back(Mat<const X> dy, Ckpt xhat, const float *rstd, const float *gamma, Mat<const X> dres, Mat<X> dx, float *part,
            uint64_t rows, uint32_t cols)
{
    constexpr int B = T < 256 ? 256 : T, R = B / T, W = T / 64;
    __shared__ uint32_t sums[2][W > 1 ? W : 1];
    const uint32_t t = threadIdx.x % T;
    const uint64_t first = (uint64_t)blockIdx.x * R + threadIdx.x / T, step = (uint64_t)gridDim.x * R;
    auto at = [&](int i) { return (i * T + t) * 8u; };
    auto left = [&](int i) { return at(i) < cols ? (int)min(cols - at(i), 8u) : 0; };
    /* Where registers are short (1024 threads) gamma is read for each row, and the next row is not asked for early. */
    constexpr bool EARLY = T < 1024;
    float g[EARLY ? V : 1][8], dg[V][8];
    auto gammas = [&](int i, float (&v)[8]) {
#pragma unroll
        for (int j = 0; j < 8; j++) v[j] = 1.0f;
        if (gamma && left(i)) load8(gamma + at(i), left(i), v);
    };
#pragma unroll
    for (int i = 0; i < V; i++) {
#pragma unroll
        for (int j = 0; j < 8; j++) dg[i][j] = 0.0f;
        if constexpr (EARLY) gammas(i, g[i]);
    }
    /* The next row is asked for before this one is worked on. */
    Raw<X> dn[V], rn[V];
    uint2 qn[V];
    uint32_t en[V];
    float sn;
    auto ask = [&](uint64_t row) {
        row = min(row, rows - 1);
#pragma unroll
        for (int i = 0; i < V; i++) {
            if (left(i)) {
                dn[i] = load_raw(dy.at(row, at(i)), left(i));
                if (dres.p) rn[i] = load_raw(dres.at(row, at(i)), left(i));
                qn[i] = *reinterpret_cast<const uint2 *>(xhat.q + row * xhat.ldq + at(i));
                en[i] = xhat.e[row * xhat.lde + at(i) / 32u];
            }
        }
        sn = rstd[row];
    };
    uint32_t turn = 0;
    if (EARLY && first < rows) ask(first);
    for (uint64_t row = first; row < rows; row += step, turn ^= 1u) {
        if (!EARLY) ask(row);
        float d[V][8], x[V][8];
        Raw<X> res[V];
        const float r = sn;
#pragma unroll
        for (int i = 0; i < V; i++) {
            if (left(i) == 0) continue;
            from_raw<X>(dn[i], d[i]);
            codes8(qn[i], x[i]);
            const float s = ckpt_scale(en[i]);
#pragma unroll
            for (int j = 0; j < 8; j++) x[i][j] = at(i) + j < cols ? x[i][j] * s : 0.0f;    /* codes beyond the row are not values */
            res[i] = rn[i];
        }
        if (EARLY) ask(row + step);
        float dot = 0.0f;
#pragma unroll
        for (int i = 0; i < V; i++) {
            if (left(i) == 0) continue;
            if constexpr (!EARLY) gammas(i, g[0]);
#pragma unroll
            for (int j = 0; j < 8; j++) {
                dg[i][j] = __builtin_fmaf(d[i][j], x[i][j], dg[i][j]);
                d[i][j] *= g[EARLY ? i : 0][j];
                dot = __builtin_fmaf(d[i][j], x[i][j], dot);
            }
        }
        dot = from_bits(wave_all(to_bits(dot), sum_of));
        if (W > 1) {
            if (threadIdx.x % 64 == 0) sums[turn][threadIdx.x / 64] = to_bits(dot);
            wg_sync();
            dot = 0.0f;
#pragma unroll
            for (int i = 0; i < W; i++) dot += from_bits(sums[turn][i]);
        }
        const float mean = dot / (float)cols;
#pragma unroll
        for (int i = 0; i < V; i++) {
            if (left(i) == 0) continue;
            float v[8] = {};
            if (dres.p) from_raw<X>(res[i], v);
#pragma unroll
            for (int j = 0; j < 8; j++) v[j] = __builtin_fmaf(r, d[i][j] - x[i][j] * mean, v[j]);
            store8(dx.at(row, at(i)), left(i), v);
        }
    }
    if (!part || first >= rows) return;
#pragma unroll
    for (int i = 0; i < V; i++) {
        if (left(i)) store8(part + first * cols + at(i), left(i), dg[i]);
    }
}

/* dgamma[i] = sum of part[0..groups)[i]: 16 columns (a 64-byte line) by 64 slices per workgroup, the slices added in order. */
__global__ void __launch_bounds__(1024) k_norm_sum(const float *part, uint32_t groups, uint32_t cols, float *dgamma)
{
    __shared__ float s[64][17];
    const uint32_t lane = threadIdx.x % 16, slice = threadIdx.x / 16, c = blockIdx.x * 16u + lane;
    float sum = 0.0f;
    if (c < cols)
        for (uint32_t g = slice; g < groups; g += 64) sum += part[(uint64_t)g * cols + c];
    s[slice][lane] = sum;
    wg_sync();
    if (threadIdx.x < 16 && c < cols) {
        sum = 0.0f;
        for (int i = 0; i < 64; i++) sum += s[i][lane];
        dgamma[c] = sum;
    }
}

/* Threads per row, and how many rows are worked on at the same time (each leaves a row of partial sums). */
struct BackShape { uint32_t threads, groups; };
BackShape back_shape(uint64_t rows, uint32_t cols)
{
    const uint32_t threads = cols <= 1024 ? 64 : cols <= 2048 ? 256 : cols <= 16384 ? 512 : 1024;
    const uint32_t most = threads == 64 ? 1024u : threads == 1024 ? 256u : 512u;
    return {threads, (uint32_t)(rows < most ? rows : most)};
}

template <typename X, int T, int V, typename... A>
int go_back(uint32_t groups, hipStream_t st, A... a)
{
    constexpr uint32_t R = T < 256 ? 256 / T : 1;
    k_norm_back<X, T, V><<<(groups + R - 1) / R, T < 256 ? 256 : T, 0, st>>>(a...);
    return launched();
}
template <typename X, typename... A> int launch_back(uint32_t cols, uint32_t groups, hipStream_t st, A... a)
{
    if (cols <= 512) return go_back<X, 64, 1>(groups, st, a...);
    if (cols <= 1024) return go_back<X, 64, 2>(groups, st, a...);
    if (cols <= 2048) return go_back<X, 256, 1>(groups, st, a...);
    if (cols <= 4096) return go_back<X, 512, 1>(groups, st, a...);
    if (cols <= 8192) return go_back<X, 512, 2>(groups, st, a...);
    if (cols <= 12288) return go_back<X, 512, 3>(groups, st, a...);
    if (cols <= 16384) return go_back<X, 512, 4>(groups, st, a...);
    return go_back<X, 1024, 4>(groups, st, a...);
}

template <typename F> int by_type(int type, F f)
{
    if (type == NSML_F32) return f(float{});
    if (type == NSML_BF16) return f(bf16{});
    return f(f16{});
}

}  // namespace

extern "C" {

int nsml_q8_rows(const void *x, int type, uint64_t ldx, uint64_t rows, uint32_t cols, const float *col_scale,
                 int8_t *q, uint64_t ldq, float *scale, void *stream)
{
    if (cols == 0 || bad_type(type) || (col_scale && bad_f32(col_scale)) ||
        (rows && (bad_mat(x, type, ldx, cols) || bad_codes(q, ldq, cols) || bad_f32(scale))))
        return NSML_EINVAL;
    if (cols > NSML_Q8_MAX_COLS) return NSML_ECAP;
    if (clash({codes_area(q, rows, ldq, cols), floats(scale, rows)}, {area(x, type, rows, ldx, cols), floats(col_scale, cols)})) return NSML_EINVAL;
    return by_type(type, [&](auto v) {
        using T = decltype(v);
        return launch_rows(OpRows<T>{mat<T>(x, ldx), col_scale, mat<int8_t>((void *)q, ldq), scale}, rows, cols, (hipStream_t)stream);
    });
}

int nsml_q8_values(const int8_t *q, uint64_t ldq, const float *scale, uint64_t rows, uint32_t cols,
                   void *out, int type, uint64_t ldo, void *stream)
{
    if (cols == 0 || bad_type(type) || (rows && (bad_codes(q, ldq, cols) || (scale && bad_f32(scale)) || bad_mat(out, type, ldo, cols))))
        return NSML_EINVAL;
    if (cols > MAX_COLS) return NSML_ECAP;
    if (clash({area(out, type, rows, ldo, cols)}, {codes_area(q, rows, ldq, cols), floats(scale, rows)})) return NSML_EINVAL;
    return by_type(type, [&](auto v) {
        using T = decltype(v);
        return launch_each(OpValues<T>{mat<int8_t>((const void *)q, ldq), scale, mat<T>(out, ldo)}, rows, cols, (hipStream_t)stream);
    });
}

int nsml_q8_transpose(const int8_t *q, uint64_t ldq, uint64_t rows, uint32_t cols, int8_t *out, uint64_t ldo, void *stream)
{
    if (cols == 0 || (rows && bad_codes(q, ldq, cols))) return NSML_EINVAL;
    if (cols > MAX_COLS || rows > MAX_COLS) return NSML_ECAP;
    if (rows == 0) return NSML_OK;
    if (bad_codes(out, ldo, (uint32_t)rows) || clash({codes_area(out, cols, ldo, (uint32_t)rows)}, {codes_area(q, rows, ldq, cols)})) return NSML_EINVAL;
    const uint64_t tiles = (rows + 127u) / 128u * ((cols + 127u) / 128u);
    k_turn<<<(uint32_t)(tiles < (1u << 20) ? tiles : 1u << 20), 256, 0, (hipStream_t)stream>>>(q, ldq, out, ldo, (uint32_t)rows, cols);
    return launched();
}

int nsml_ckpt8_pack(const void *x, int type, uint64_t ldx, uint64_t rows, uint32_t cols, const nsml_ckpt8 *out, void *stream)
{
    if (cols == 0 || bad_type(type) || (rows && (bad_mat(x, type, ldx, cols) || bad_ckpt(out, cols)))) return NSML_EINVAL;
    if (cols > MAX_COLS) return NSML_ECAP;
    if (clash({codes_area(out, rows, cols), exps_area(out, rows, cols)}, {area(x, type, rows, ldx, cols)})) return NSML_EINVAL;
    return by_type(type, [&](auto v) {
        using T = decltype(v);
        return launch_each(OpPack<T>{mat<T>(x, ldx), ckpt_of(out)}, rows, cols, (hipStream_t)stream);
    });
}

int nsml_ckpt8_unpack(const nsml_ckpt8 *x, uint64_t rows, uint32_t cols, void *out, int type, uint64_t ldo, void *stream)
{
    if (cols == 0 || bad_type(type) || (rows && (bad_ckpt(x, cols) || bad_mat(out, type, ldo, cols)))) return NSML_EINVAL;
    if (cols > MAX_COLS) return NSML_ECAP;
    if (clash({area(out, type, rows, ldo, cols)}, {codes_area(x, rows, cols), exps_area(x, rows, cols)})) return NSML_EINVAL;
    return by_type(type, [&](auto v) {
        using T = decltype(v);
        return launch_each(OpUnpack<T>{ckpt_of(x), mat<T>(out, ldo)}, rows, cols, (hipStream_t)stream);
    });
}

int nsml_rmsnorm_q8(const void *x, uint64_t ldx, const void *residual, uint64_t ldr, const float *gamma, float eps,
                    int type, uint64_t rows, uint32_t cols, void *h, uint64_t ldh, int8_t *q, uint64_t ldq,
                    float *scale, float *rstd, const nsml_ckpt8 *xhat, void *stream)
{
    if (cols == 0 || bad_type(type) || !(eps >= 0.0f) || (gamma && bad_f32(gamma)) ||
        (rows && (bad_mat(x, type, ldx, cols) || !residual != !h ||
                  (residual && (bad_mat(residual, type, ldr, cols) || bad_mat(h, type, ldh, cols))) ||
                  bad_codes(q, ldq, cols) || bad_f32(scale) || bad_f32(rstd) || (xhat && bad_ckpt(xhat, cols)))))
        return NSML_EINVAL;
    if (cols > NSML_NORM_MAX_COLS) return NSML_ECAP;
    const Area sum = area(h, type, rows, ldh, cols);
    if (clash({sum, codes_area(q, rows, ldq, cols), floats(scale, rows), floats(rstd, rows), codes_area(xhat, rows, cols), exps_area(xhat, rows, cols)},
              {apart(area(x, type, rows, ldx, cols), sum), apart(area(residual, type, rows, ldr, cols), sum), floats(gamma, cols)}))
        return NSML_EINVAL;
    return by_type(type, [&](auto v) {
        using T = decltype(v);
        return launch_rows(OpNorm<T>{mat<T>(x, ldx), mat<T>(residual, ldr), gamma, eps, mat<T>(h, ldh),
                                     mat<int8_t>((void *)q, ldq), scale, rstd, ckpt_of(xhat)}, rows, cols, (hipStream_t)stream);
    });
}

uint64_t nsml_rmsnorm_backward_work(uint64_t rows, uint32_t cols)
{
    return (uint64_t)back_shape(rows, cols).groups * cols * 4u;
}

int nsml_rmsnorm_backward(const void *dy, uint64_t lddy, const nsml_ckpt8 *xhat, const float *rstd, const float *gamma,
                          const void *dres, uint64_t lddres, int type, uint64_t rows, uint32_t cols,
                          void *dx, uint64_t lddx, float *dgamma, void *work, uint64_t work_bytes, void *stream)
{
    if (cols == 0 || bad_type(type) || (gamma && bad_f32(gamma)) ||
        (rows && (bad_mat(dy, type, lddy, cols) || bad_ckpt(xhat, cols) || bad_f32(rstd) ||
                  (dres && bad_mat(dres, type, lddres, cols)) || bad_mat(dx, type, lddx, cols))))
        return NSML_EINVAL;
    if (cols > NSML_NORM_MAX_COLS) return NSML_ECAP;
    const BackShape s = back_shape(rows, cols);
    float *part = nullptr;
    if (dgamma) {
        if (bad_f32(dgamma)) return NSML_EINVAL;
        if (rows && (!work || !at_multiple(work, 16) || work_bytes < nsml_rmsnorm_backward_work(rows, cols))) return NSML_EINVAL;
        part = static_cast<float *>(work);
    }
    const Area out = area(dx, type, rows, lddx, cols);
    if (clash({out, floats(dgamma, cols), area(part, 1, 0, nsml_rmsnorm_backward_work(rows, cols))},
              {apart(area(dy, type, rows, lddy, cols), out), apart(area(dres, type, rows, lddres, cols), out), codes_area(xhat, rows, cols),
               exps_area(xhat, rows, cols), floats(rstd, rows), floats(gamma, cols)}))
        return NSML_EINVAL;
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (rows) {
        const int rc = by_type(type, [&](auto v) {
            using T = decltype(v);
            return launch_back<T>(cols, s.groups, st, mat<T>(dy, lddy), ckpt_of(xhat), rstd, gamma, mat<T>(dres, lddres),
                                  mat<T>(dx, lddx), part, rows, cols);
        });
        if (rc) return rc;
    }
    if (dgamma) {
        k_norm_sum<<<(cols + 15u) / 16u, 1024, 0, st>>>(part, s.groups, cols, dgamma);
        return launched();
    }
    return NSML_OK;
}

int nsml_swiglu_q8(const void *gate, uint64_t ldg, const void *up, uint64_t ldu, int type, uint64_t rows, uint32_t cols,
                   int8_t *q, uint64_t ldq, float *scale, const nsml_ckpt8 *gate_ckpt, const nsml_ckpt8 *up_ckpt,
                   const nsml_ckpt8 *act_ckpt, void *stream)
{
    if (cols == 0 || bad_type(type) ||
        (rows && (bad_mat(gate, type, ldg, cols) || bad_mat(up, type, ldu, cols) || bad_codes(q, ldq, cols) || bad_f32(scale) ||
                  (gate_ckpt && bad_ckpt(gate_ckpt, cols)) || (up_ckpt && bad_ckpt(up_ckpt, cols)) || (act_ckpt && bad_ckpt(act_ckpt, cols)))))
        return NSML_EINVAL;
    if (cols > NSML_Q8_MAX_COLS) return NSML_ECAP;
    if (clash({codes_area(q, rows, ldq, cols), floats(scale, rows), codes_area(gate_ckpt, rows, cols), exps_area(gate_ckpt, rows, cols),
               codes_area(up_ckpt, rows, cols), exps_area(up_ckpt, rows, cols), codes_area(act_ckpt, rows, cols), exps_area(act_ckpt, rows, cols)},
              {area(gate, type, rows, ldg, cols), area(up, type, rows, ldu, cols)}))
        return NSML_EINVAL;
    return by_type(type, [&](auto v) {
        using T = decltype(v);
        return launch_rows(OpGlu<T>{mat<T>(gate, ldg), mat<T>(up, ldu), mat<int8_t>((void *)q, ldq), scale, ckpt_of(gate_ckpt),
                                    ckpt_of(up_ckpt), ckpt_of(act_ckpt), cols}, rows, cols, (hipStream_t)stream);
    });
}

int nsml_swiglu_backward(const void *da, uint64_t ldda, const nsml_ckpt8 *gate, const nsml_ckpt8 *up, int type,
                         uint64_t rows, uint32_t cols, void *dgate, uint64_t lddg, void *dup, uint64_t lddu, void *stream)
{
    if (cols == 0 || bad_type(type) ||
        (rows && (bad_mat(da, type, ldda, cols) || bad_ckpt(gate, cols) || bad_ckpt(up, cols) ||
                  bad_mat(dgate, type, lddg, cols) || bad_mat(dup, type, lddu, cols))))
        return NSML_EINVAL;
    if (cols > MAX_COLS) return NSML_ECAP;
    const Area g = area(dgate, type, rows, lddg, cols), u = area(dup, type, rows, lddu, cols);
    if (clash({g, u}, {apart(apart(area(da, type, rows, ldda, cols), g), u), codes_area(gate, rows, cols), exps_area(gate, rows, cols),
                       codes_area(up, rows, cols), exps_area(up, rows, cols)}))
        return NSML_EINVAL;
    return by_type(type, [&](auto v) {
        using T = decltype(v);
        return launch_each(OpGluBack<T>{mat<T>(da, ldda), ckpt_of(gate), ckpt_of(up), mat<T>(dgate, lddg), mat<T>(dup, lddu)}, rows, cols,
                           (hipStream_t)stream);
    });
}

}  // extern "C"
