/*
 * Products of matrices in 8 bits: c[i, j] = a_scale[i] * b_scale[j] * sum_k a[i, k] * b[j, k] + bias[j].
 *
 * Both operands have k side by side, which is what the matrix instructions take: 16 bytes of a row per lane.  The sum is a
 * whole number below 2^31 (k <= 131072), so any order and any split of k give the same result.
 */
#include "tiles.hpp"

namespace {

/* What becomes of a sum. */
template <typename T> struct Out {
    T *c;
    uint64_t ldc;
    const float *as, *bs, *bias;
    __device__ __forceinline__ T value(int sum, float a, uint32_t j) const
    {
        float v = (float)sum * a;
        if (bs) v *= bs[j];
        if (bias) v += bias[j];
        return (T)v;
    }
};

/* ---------------------------------------------------------------- tiles */

/* A tile of BM x BN by WM x WN wavefronts; k in stages of 128 bytes, loaded straight into LDS one stage ahead.
 * The matrix instructions of the last quarter of a stage run while the first quarter of the next is read from LDS: the barrier
 * between stages stands before them, when all of the stage is in registers. */
template <typename T, int BM, int BN, int WM, int WN>
__global__ void __launch_bounds__(WM * WN * 64)
k_product(const int8_t *a, uint64_t lda, const int8_t *b, uint64_t ldb, uint64_t m, uint32_t n, uint32_t k, Out<T> out)
{
    constexpr int W = WM * WN, TM = BM / WM / 32, TN = BN / WN / 32;
    constexpr int STAGE = (BM + BN) * 128;
    __shared__ __align__(16) uint8_t lds[2 * STAGE];
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64;
    const Tile tile = tile_of(blockIdx.x, (uint32_t)((m + BM - 1) / BM), (n + BN - 1) / BN);
    const uint64_t m0 = (uint64_t)tile.row * BM;
    const uint32_t n0 = tile.col * BN;
    const uint32_t rows_a = (uint32_t)min<uint64_t>(m - m0, BM), rows_b = min(n - n0, (uint32_t)BN);
    const uint32_t wm = wave / WN * (BM / WM), wn = wave % WN * (BN / WN);
    v16i acc[TM][TN] = {};
    v4i fa[2][TM], fb[2][TN];
    const int8_t *pa = a + m0 * lda, *pb = b + (uint64_t)n0 * ldb;
    auto fetch = [&](uint32_t k0, uint8_t *to) {
        if (k - k0 >= 128u) {
            load_tile<BM, W>(pa + k0, lda, rows_a, to, wave, lane);
            load_tile<BN, W>(pb + k0, ldb, rows_b, to + BM * 128, wave, lane);
        } else {
            load_tail<BM, W>(pa + k0, lda, rows_a, k - k0, to, threadIdx.x);
            load_tail<BN, W>(pb + k0, ldb, rows_b, k - k0, to + BM * 128, threadIdx.x);
        }
    };
    /* Chunk 2s + lane / 32 of a lane's row: the place of chunk lane / 32 with two bits turned. */
    const uint32_t ra = place(wm + lane % 32, lane / 32), rb = BM * 128 + place(wn + lane % 32, lane / 32);
    auto read = [&](uint32_t from, int s) {
        const uint8_t *at_a = lds + ((ra + from) ^ (s * 32u)), *at_b = lds + ((rb + from) ^ (s * 32u));
#pragma unroll
        for (int j = 0; j < TN; j++) fb[s & 1][j] = frag(at_b + j * BLOCK);
#pragma unroll
        for (int i = 0; i < TM; i++) fa[s & 1][i] = frag(at_a + i * BLOCK);
    };
    /* Rows of a result are columns of c, so that a lane holds four neighbours of a row of c. */
    auto multiply = [&](int s, int from, int to) {
#pragma unroll
        for (int t = from; t < to; t++)
            acc[t / TN][t % TN] = __builtin_amdgcn_mfma_i32_32x32x32_i8(fb[s & 1][t % TN], fa[s & 1][t / TN], acc[t / TN][t % TN], 0, 0, 0);
    };
    fetch(0, lds);
    wait_loads();
    wg_sync();
    if (k > 128u) fetch(128u, lds + STAGE);
    read(0, 0);
    for (uint32_t k0 = 0, at = 0; k0 < k; k0 += 128u, at ^= STAGE) {
#pragma unroll
        for (int s = 0; s < 3; s++) {
            multiply(s, 0, 1);               /* waits for what it multiplies, so the next reads come after it: they are on their way */
            __builtin_amdgcn_sched_barrier(0);       /* behind the other products */
            read(at, s + 1);
            __builtin_amdgcn_sched_barrier(0);
            multiply(s, 1, TM * TN);
            __builtin_amdgcn_sched_barrier(0);
        }
        wait_loads();
        wg_sync();                           /* the next stage is there, and this one is in registers everywhere */
        multiply(3, 0, 1);
        __builtin_amdgcn_sched_barrier(0);
        if (k0 + 256u < k) fetch(k0 + 256u, lds + at);
        read(at ^ STAGE, 0);                 /* behind the last stage: old contents, not used */
        __builtin_amdgcn_sched_barrier(0);
        multiply(3, 1, TM * TN);
    }
    wg_sync();
    /* Out through LDS, 32 rows of a wavefront's part at a time, so that lines are written whole. */
    constexpr int COLS = TN * 32, PITCH = COLS * (int)sizeof(T) + 16, LANES = COLS * (int)sizeof(T) / 16, PER = 16 / (int)sizeof(T);
    static_assert(32 * PITCH * W <= 2 * STAGE, "room for every wavefront");
    uint8_t *mine = lds + wave * (32 * PITCH);
#pragma unroll
    for (int i = 0; i < TM; i++) {
        const uint32_t row = wm + i * 32 + lane % 32;
        const float as = out.as[m0 + min(row, rows_a - 1)];
#pragma unroll
        for (int j = 0; j < TN; j++)
#pragma unroll
            for (int q = 0; q < 4; q++) {
                const uint32_t col = j * 32 + q * 8 + lane / 32 * 4;
                T v[4];
#pragma unroll
                for (int e = 0; e < 4; e++) v[e] = out.value(acc[i][j][q * 4 + e], as, min(n0 + wn + col + e, n - 1));
                __builtin_memcpy(__builtin_assume_aligned(mine + lane % 32 * PITCH + col * sizeof(T), sizeof v), v, sizeof v);
            }
#pragma unroll
        for (int s = 0; s < 32 * LANES / 64; s++) {
            const uint32_t r = s * (64 / LANES) + lane / LANES, c = lane % LANES * PER, at = wn + c, to = wm + i * 32 + r;
            T v[PER];
            __builtin_memcpy(v, __builtin_assume_aligned(mine + r * PITCH + c * sizeof(T), 16), 16);
            if (to < rows_a) {
                T *p = out.c + (m0 + to) * out.ldc + n0 + at;
                if (at + PER <= rows_b) {
                    Bytes<4> x;
                    __builtin_memcpy(&x, v, 16);
                    *reinterpret_cast<Bytes<4> *>(p) = x;
                } else {
#pragma unroll
                    for (int e = 0; e < PER; e++)
                        if (at + e < rows_b) p[e] = v[e];
                }
            }
        }
    }
}

/* ---------------------------------------------------------------- few rows */

/* Up to 16 * MR rows of a against 16 * NC rows of b, k split over the wavefronts in runs of 256 bytes: the weights are read
 * once, each row's run by one wavefront, straight into registers.  The parts meet in LDS. */
template <typename T, int MR, int NC, int W>
__global__ void __launch_bounds__(W * 64)
k_product_few(const int8_t *a, uint64_t lda, const int8_t *b, uint64_t ldb, uint64_t m, uint32_t n, uint32_t k, Out<T> out)
{
    __shared__ int sums[MR * 16][NC * 16 + 4];
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64;
    const uint32_t n0 = blockIdx.x * (NC * 16u);
    const uint64_t m0 = (uint64_t)blockIdx.y * (MR * 16u);
    const uint32_t r = lane % 16, part = lane / 16 * 16;
    for (uint32_t i = threadIdx.x; i < sizeof sums / 4; i += W * 64) (&sums[0][0])[i] = 0;
    v4i acc[MR][NC] = {};
    const int8_t *pa[MR], *pb[NC];
#pragma unroll
    for (int i = 0; i < MR; i++) pa[i] = a + min<uint64_t>(m0 + i * 16 + r, m - 1) * lda;
#pragma unroll
    for (int j = 0; j < NC; j++) pb[j] = b + (uint64_t)min(n0 + j * 16 + r, n - 1) * ldb;
    for (uint32_t k0 = wave * 256u; k0 < k; k0 += W * 256u) {
        v4i fa[4][MR], fb[4][NC];
#pragma unroll
        for (int s = 0; s < 4; s++) {
            const uint32_t at = k0 + s * 64u + part;
#pragma unroll
            for (int j = 0; j < NC; j++) fb[s][j] = at < k ? *reinterpret_cast<const v4i *>(pb[j] + at) : v4i{};
#pragma unroll
            for (int i = 0; i < MR; i++)
                fa[s][i] = at < k && m0 + i * 16 + r < m ? *reinterpret_cast<const v4i *>(pa[i] + at) : v4i{};
        }
        if (k0 + 256u > k)
#pragma unroll
            for (int s = 0; s < 4; s++)
#pragma unroll
                for (int i = 0; i < MR; i++) fa[s][i] = first_bytes(fa[s][i], (int)k - (int)(k0 + s * 64u + part));
#pragma unroll
        for (int s = 0; s < 4; s++)
#pragma unroll
            for (int i = 0; i < MR; i++)
#pragma unroll
                for (int j = 0; j < NC; j++) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fb[s][j], fa[s][i], acc[i][j], 0, 0, 0);
    }
    wg_sync();
#pragma unroll
    for (int i = 0; i < MR; i++)
#pragma unroll
        for (int j = 0; j < NC; j++)
#pragma unroll
            for (int e = 0; e < 4; e++) atomicAdd(&sums[i * 16 + r][j * 16 + lane / 16 * 4 + e], acc[i][j][e]);
    wg_sync();
    for (uint32_t i = threadIdx.x; i < MR * NC * 256u; i += W * 64) {
        const uint32_t row = i / (NC * 16u), col = i % (NC * 16u);
        if (m0 + row < m && n0 + col < n) out.c[(m0 + row) * out.ldc + n0 + col] = out.value(sums[row][col], out.as[m0 + row], n0 + col);
    }
}

template <typename T>
int launch_product(const int8_t *a, uint64_t lda, const int8_t *b, uint64_t ldb, uint64_t m, uint32_t n, uint32_t k, const Out<T> &out, hipStream_t st)
{
    if (m <= 64) {
        if (m <= 16)
            k_product_few<T, 1, 1, 16><<<dim3((n + 15) / 16, 1), 1024, 0, st>>>(a, lda, b, ldb, m, n, k, out);
        else if (m <= 32)
            k_product_few<T, 2, 2, 8><<<dim3((n + 31) / 32, 1), 512, 0, st>>>(a, lda, b, ldb, m, n, k, out);
        else
            k_product_few<T, 4, 2, 8><<<dim3((n + 31) / 32, 1), 512, 0, st>>>(a, lda, b, ldb, m, n, k, out);
        return launched();
    }
    const auto tiles = [&](uint64_t s) { return ((m + s - 1) / s) * ((n + s - 1) / s); };
    if (tiles(256) >= (1u << 24)) return NSML_ECAP;
    if (tiles(256) >= 256)
        k_product<T, 256, 256, 2, 4><<<(uint32_t)tiles(256), 512, 0, st>>>(a, lda, b, ldb, m, n, k, out);
    else if (tiles(128) >= 256)
        k_product<T, 128, 128, 2, 2><<<(uint32_t)tiles(128), 256, 0, st>>>(a, lda, b, ldb, m, n, k, out);
    else
        k_product<T, 64, 64, 2, 2><<<(uint32_t)tiles(64), 256, 0, st>>>(a, lda, b, ldb, m, n, k, out);
    return launched();
}

}  // namespace

extern "C" int nsml_q8_matmul(const int8_t *a, uint64_t lda, const float *a_scale, const int8_t *b, uint64_t ldb,
                              const float *b_scale, const float *bias, uint64_t m, uint32_t n, uint32_t k,
                              void *c, int type, uint64_t ldc, void *stream)
{
    if (n == 0 || k == 0 || bad_type(type) || bad_codes(b, ldb, k) || (b_scale && bad_f32(b_scale)) || (bias && bad_f32(bias)) ||
        (m && (bad_codes(a, lda, k) || bad_f32(a_scale) || bad_mat(c, type, ldc, n))))
        return NSML_EINVAL;
    if (k > NSML_Q8_MAX_COLS || lda > MAX_LD || ldb > MAX_LD) return NSML_ECAP;
    if (m == 0) return NSML_OK;
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (type == NSML_F32) return launch_product(a, lda, b, ldb, m, n, k, Out<float>{static_cast<float *>(c), ldc, a_scale, b_scale, bias}, st);
    if (type == NSML_BF16) return launch_product(a, lda, b, ldb, m, n, k, Out<bf16>{static_cast<bf16 *>(c), ldc, a_scale, b_scale, bias}, st);
    return launch_product(a, lda, b, ldb, m, n, k, Out<f16>{static_cast<f16 *>(c), ldc, a_scale, b_scale, bias}, st);
}
