/*
 * Products of matrices in 8 bits: c[i, j] = a_scale[i] * b_scale[j] * sum_k a[i, k] * b[j, k] + bias[j].
 *
 * Both operands have k side by side, which is what the matrix instructions take: 16 bytes of a row per lane.  The sum is a
 * whole number below 2^31 (k <= 131072), so any order and any split of k give the same result.
 */
#include "tiles.hpp"

namespace {

/* What becomes of the sums. */
template <typename T> struct Out {
    T *c;
    uint64_t ldc;
    const float *as, *bs, *bias;
    bool past;                   /* past the caches */
};

/* ---------------------------------------------------------------- tiles */

constexpr uint32_t DEPTH = 64;               /* bytes of k to a stage */

/* A tile of BM x BN by WM x WN wavefronts.  Stages go from memory straight into a ring of places in LDS, all but one ahead; a wavefront's
 * requests are spread between its matrix instructions, as one that waits to make a request multiplies nothing.  The matrix instructions of
 * a stage's second half run while the next stage's first half is read from LDS: the barrier between stages stands before them,
 * when all of the stage is in registers. */
template <typename T, int BM, int BN, int WM, int WN, int RING>
__device__ __forceinline__ void product_tile(uint8_t *lds, uint64_t m0, uint32_t n0, const int8_t *a, uint64_t lda, const int8_t *b, uint64_t ldb,
                                             uint64_t m, uint32_t n, uint32_t k, const Out<T> &out)
{
    constexpr int W = WM * WN, TM = BM / WM / 32, TN = BN / WN / 32, LA = BM / 16 / W, LB = BN / 16 / W, L = LA + LB;
    constexpr uint32_t STAGE = (BM + BN) * DEPTH;
    static_assert(LA >= 1 && LB >= 1 && (TM * TN >= L || TM * TN == 1), "a request between two matrix instructions");
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64;
    const uint32_t rows_a = (uint32_t)min<uint64_t>(m - m0, BM), rows_b = min(n - n0, (uint32_t)BN);
    const uint32_t wm = wave / WN * (BM / WM), wn = wave % WN * (BN / WN);
    const int8_t *pa = a + m0 * lda, *pb = b + (uint64_t)n0 * ldb;
    v16i acc[TM][TN] = {};
    v4i fa[2][TM], fb[2][TN];

    /* A request brings 16 rows; rows beyond the matrix are its last one again.  Chunks beyond a row's end (in the last stage) are the
     * stage's first again: what they hold is multiplied by zeros. */
    uint32_t off[L], chunk[L];
#pragma unroll
    for (int l = 0; l < L; l++) {
        const uint32_t four = ((l < LA ? l : l - LA) * W + wave) * 4u + lane / 16u, at = (lane % 16u) ^ (four % 4u);
        const uint32_t row = min(four * 4u + at / 4u, (l < LA ? rows_a : rows_b) - 1u);
        chunk[l] = at % 4u * 16u;
        off[l] = row * (uint32_t)(l < LA ? lda : ldb);
    }
    /* The scales are asked for before they are needed, those of a before anything else. */
    float as[TM];
#pragma unroll
    for (int i = 0; i < TM; i++) as[i] = out.as[m0 + min(wm + i * 32 + lane % 32, rows_a - 1)];
    const uint32_t stages = (k + DEPTH - 1) / DEPTH;
    auto request = [&](uint32_t stage, uint32_t ring, int l) {
        const uint32_t k0 = min(stage, stages - 1u) * DEPTH;
        const uint32_t at = off[l] + (k0 + chunk[l] < k ? chunk[l] : 0u);
        uint8_t *to = lds + ring + (l < LA ? 0u : BM * DEPTH) + ((l < LA ? l : l - LA) * W + wave) * 1024u;
        __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)((l < LA ? pa : pb) + k0 + at),
                                         (__attribute__((address_space(3))) void *)to, 16, 0, 0);
    };
    /* Chunk 2s + lane / 32 of a lane's row: the place of chunk lane / 32 with a bit turned. */
    const uint32_t ra = spot(wm + lane % 32, lane / 32), rb = BM * DEPTH + spot(wn + lane % 32, lane / 32);
    auto read = [&](uint32_t from, int s) {
        const uint8_t *at_a = lds + ((ra + from) ^ (s * 32u)), *at_b = lds + ((rb + from) ^ (s * 32u));
#pragma unroll
        for (int j = 0; j < TN; j++) fb[s][j] = frag(at_b + j * (32 * DEPTH));
#pragma unroll
        for (int i = 0; i < TM; i++) fa[s][i] = frag(at_a + i * (32 * DEPTH));
    };
    /* Rows of a result are columns of c, so that a lane holds four neighbours of a row of c. */
    auto multiply = [&](int s, int t) {
        acc[t / TN][t % TN] = __builtin_amdgcn_mfma_i32_32x32x32_i8(fb[s][t % TN], fa[s][t / TN], acc[t / TN][t % TN], 0, 0, 0);
    };
    auto cut = [&](int s) {                  /* the last stage: zeros from k on */
#pragma unroll
        for (int i = 0; i < TM; i++) fa[s][i] = first_bytes(fa[s][i], (int)(k - (stages - 1u) * DEPTH) - (int)(s * 32u + lane / 32u * 16u));
    };

#pragma unroll
    for (uint32_t r = 0; r < RING - 1; r++)
#pragma unroll
        for (int l = 0; l < L; l++) request(r, r * STAGE, l);
    constexpr int LATER = (RING - 2) * L;    /* requests that may be on their way when the next stage has to be there */
    loads_sync<LATER>();
    read(0, 0);
    uint32_t here = 0, there = (RING - 1) * STAGE;       /* the stage's place, and the one before it, which is free */
    for (uint32_t stage = 0; stage < stages; stage++) {
        const uint32_t next = here + STAGE == RING * STAGE ? 0u : here + STAGE;
        const bool ends = stage + 1 == stages && k % DEPTH;
        wait_lds();
        if (ends) cut(0);
        multiply(0, 0);
        __builtin_amdgcn_sched_barrier(0);
        read(here, 1);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int t = 1; t < TM * TN; t++) {
            multiply(0, t);
            if (t - 1 < L) request(stage + RING - 1, there, t - 1);
            __builtin_amdgcn_sched_barrier(0);
        }
        if (TM * TN - 1 < L)
#pragma unroll
            for (int l = TM * TN - 1; l < L; l++) request(stage + RING - 1, there, l);
        loads_sync<LATER>();                 /* the next stage is there, and this one is in registers everywhere */
        if (ends) cut(1);
        multiply(1, 0);
        __builtin_amdgcn_sched_barrier(0);
        read(next, 0);                       /* behind the last stage: its contents again, not used */
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int t = 1; t < TM * TN; t++) multiply(1, t);
        __builtin_amdgcn_sched_barrier(0);
        there = here;
        here = next;
    }
    float bs[TN][16];
#pragma unroll
    for (int j = 0; j < TN; j++)
#pragma unroll
        for (int e = 0; e < 16; e++) bs[j][e] = out.bs ? out.bs[min(n0 + wn + j * 32 + acc_row(e, lane), n - 1)] : 1.0f;
    loads_sync<0>();
    /* Out through LDS, 32 rows of a wavefront's part at a time, so that lines are written whole. */
    constexpr int COLS = TN * 32, PITCH = COLS * (int)sizeof(T) + 16, LANES = COLS * (int)sizeof(T) / 16, PER = 16 / (int)sizeof(T);
    static_assert(32 * PITCH * W <= RING * STAGE, "room for every wavefront");
    uint8_t *mine = lds + wave * (32 * PITCH);
    float bias[TN][16];
#pragma unroll
    for (int j = 0; j < TN; j++)
#pragma unroll
        for (int e = 0; e < 16; e++) bias[j][e] = out.bias ? out.bias[min(n0 + wn + j * 32 + acc_row(e, lane), n - 1)] : 0.0f;
#pragma unroll
    for (int i = 0; i < TM; i++) {
#pragma unroll
        for (int j = 0; j < TN; j++)
#pragma unroll
            for (int q = 0; q < 4; q++) {
                const uint32_t col = j * 32 + q * 8 + lane / 32 * 4;
                T v[4];
#pragma unroll
                for (int e = 0; e < 4; e++) v[e] = (T)((float)acc[i][j][q * 4 + e] * as[i] * bs[j][q * 4 + e] + bias[j][q * 4 + e]);
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
                    Loose4 x;
                    __builtin_memcpy(&x, v, 16);
                    if (out.past) __builtin_nontemporal_store(x, reinterpret_cast<Loose4 *>(p));
                    else *reinterpret_cast<Loose4 *>(p) = x;
                } else {
#pragma unroll
                    for (int e = 0; e < PER; e++)
                        if (at + e < rows_b) p[e] = v[e];
                }
            }
        }
    }
}

template <typename T, int SIDE, int RING>
__global__ void __launch_bounds__(256)
k_product(const int8_t *a, uint64_t lda, const int8_t *b, uint64_t ldb, uint64_t m, uint32_t n, uint32_t k, Out<T> out)
{
    __shared__ __align__(16) uint8_t lds[RING * 2 * SIDE * DEPTH];
    const Tile tile = tile_of(blockIdx.x, (uint32_t)((m + SIDE - 1) / SIDE), (n + SIDE - 1) / SIDE);
    product_tile<T, SIDE, SIDE, 2, 2, RING>(lds, (uint64_t)tile.row * SIDE, tile.col * SIDE, a, lda, b, ldb, m, n, k, out);
}

/* Tiles of 256 x 256, one workgroup a compute unit.  Those from `whole` on, which would leave half of the chip or more without work
 * in the last round, are two workgroups each, 128 x 256. */
template <typename T>
__global__ void __launch_bounds__(512, 2)
k_product_large(const int8_t *a, uint64_t lda, const int8_t *b, uint64_t ldb, uint64_t m, uint32_t n, uint32_t k, Out<T> out, uint32_t whole)
{
    __shared__ __align__(16) uint8_t lds[4 * 512 * DEPTH];
    const uint32_t id = blockIdx.x, rows = (uint32_t)((m + 255) / 256), cols = (n + 255) / 256;
    if (id < whole) {
        const Tile tile = tile_of(id, rows, cols);
        product_tile<T, 256, 256, 2, 4, 4>(lds, (uint64_t)tile.row * 256, tile.col * 256u, a, lda, b, ldb, m, n, k, out);
    } else {
        const Tile tile = tile_of(whole + (id - whole) / 2u, rows, cols);
        const uint64_t m0 = (uint64_t)tile.row * 256 + (id - whole) % 2u * 128u;
        if (m0 < m) product_tile<T, 128, 256, 2, 4, 4>(lds, m0, tile.col * 256u, a, lda, b, ldb, m, n, k, out);
    }
}

/* ---------------------------------------------------------------- few rows */

/* The same for results whose type is looked up once they are there: few, so that it costs nothing, and a third of the kernels. */
struct AnyOut {
    void *c;
    uint64_t ldc;
    const float *as, *bs, *bias;
    int type;
};

/* 16 * MR rows of a against 16 * NC rows of b, k split over W wavefronts in runs of 256 or 512 bytes, straight into registers: a compute unit
 * reads its rows of b once, and those of a once for all of them.  Bound by memory, so all that matters is that a wavefront's
 * requests are on their way together.  The parts meet in LDS. */
template <int MR, int NC, int W>
__global__ void __launch_bounds__(W * 64, W / 4)
k_product_few(const int8_t *a, uint64_t lda, const int8_t *b, uint64_t ldb, uint64_t m, uint32_t n, uint32_t k, AnyOut out)
{
    constexpr uint32_t RUN = W == 16 ? 256 : 512;
    __shared__ int sums[MR * NC][4][64];             /* as a wavefront holds them: additions of 64 lanes meet no bank twice */
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64;
    const uint32_t n0 = blockIdx.x * (NC * 16u);
    const uint64_t m0 = (uint64_t)blockIdx.y * (MR * 16u);
    const uint32_t r = lane % 16, part = lane / 16 * 16;
    for (uint32_t i = threadIdx.x; i < sizeof sums / 4; i += W * 64) (&sums[0][0][0])[i] = 0;
    v4i acc[MR][NC] = {};
    const int8_t *pa[MR], *pb[NC];
#pragma unroll
    for (int i = 0; i < MR; i++) pa[i] = a + min<uint64_t>(m0 + i * 16 + r, m - 1) * lda;
#pragma unroll
    for (int j = 0; j < NC; j++) pb[j] = b + (uint64_t)min(n0 + j * 16 + r, n - 1) * ldb;
    /* All of a run's rows of b are asked for at once, those of a, which other compute units have read too, half a run at a time. */
    for (uint32_t k0 = wave * RUN; k0 < k; k0 += W * RUN) {
        v4i fb[RUN / 64][NC];
#pragma unroll
        for (int s = 0; s < (int)RUN / 64; s++)
#pragma unroll
            for (int j = 0; j < NC; j++) {
                const uint32_t at = k0 + s * 64u + part;
                fb[s][j] = at < k ? *reinterpret_cast<const v4i *>(pb[j] + at) : v4i{};
            }
#pragma unroll
        for (int h = 0; h < (int)RUN / 64; h += 4) {
            v4i fa[4][MR];
#pragma unroll
            for (int s = 0; s < 4; s++)
#pragma unroll
                for (int i = 0; i < MR; i++) {
                    const uint32_t at = k0 + (h + s) * 64u + part;
                    fa[s][i] = at < k && m0 + i * 16 + r < m ? *reinterpret_cast<const v4i *>(pa[i] + at) : v4i{};
                }
            if (k0 + RUN > k)
#pragma unroll
                for (int s = 0; s < 4; s++)
#pragma unroll
                    for (int i = 0; i < MR; i++) fa[s][i] = first_bytes(fa[s][i], (int)k - (int)(k0 + (h + s) * 64u + part));
#pragma unroll
            for (int s = 0; s < 4; s++)
#pragma unroll
                for (int i = 0; i < MR; i++)
#pragma unroll
                    for (int j = 0; j < NC; j++) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fb[h + s][j], fa[s][i], acc[i][j], 0, 0, 0);
        }
    }
    wg_sync();
    if (wave * RUN < k)
#pragma unroll
        for (int i = 0; i < MR; i++)
#pragma unroll
            for (int j = 0; j < NC; j++)
#pragma unroll
                for (int e = 0; e < 4; e++) atomicAdd(&sums[i * NC + j][e][lane], acc[i][j][e]);
    wg_sync();
    for (uint32_t i = threadIdx.x; i < MR * NC * 64u; i += W * 64) {
        const uint32_t block = i / 64u, row = block / NC * 16u + lane % 16u, col = n0 + block % NC * 16u + lane / 16u * 4u;
        if (m0 + row >= m || col >= n) continue;
        const float as = out.as[m0 + row];
        float v[4];
#pragma unroll
        for (int e = 0; e < 4; e++) {
            const uint32_t at = min(col + e, n - 1);
            v[e] = (float)sums[block][e][lane] * as;
            if (out.bs) v[e] *= out.bs[at];
            if (out.bias) v[e] += out.bias[at];
        }
        const uint64_t to = (m0 + row) * out.ldc + col;
        const int have = (int)min(n - col, 4u);
        if (out.type == NSML_F32) store4(static_cast<float *>(out.c) + to, have, v);
        else if (out.type == NSML_BF16) store4(static_cast<bf16 *>(out.c) + to, have, v);
        else store4(static_cast<f16 *>(out.c) + to, have, v);
    }
}

/* 16 wavefronts where what they hold fits the 128 registers that are left for each, else eight. */
template <int MR, int NC> int go_few(const int8_t *a, uint64_t lda, const int8_t *b, uint64_t ldb, uint64_t m, uint32_t n, uint32_t k, const AnyOut &out, hipStream_t st)
{
    constexpr int W = 16 * (MR + NC) + 4 * MR * NC <= 100 ? 16 : 8;
    k_product_few<MR, NC, W><<<dim3((n + NC * 16 - 1) / (NC * 16), (uint32_t)((m + MR * 16 - 1) / (MR * 16))), W * 64, 0, st>>>(a, lda, b, ldb, m, n, k, out);
    return launched();
}
/* As many rows of b to a workgroup as give every compute unit one workgroup (us for 16, 32, 48 and 64 rows, k = 4096: 1 x 4096 7.1, 8.7, 10.7, 13.2;
 * 48 x 4096 12.8, 14.5; 1 x 11008 13.2, 15.6, 13.4, 15.5).  More than 32 rows of a come here only where 32 of b do.  These figures and those below:
 * both operands of so many matrices in turn that they come from memory, results in bfloat16, 24 calls in a graph (weights that stay in the last cache:
 * 1 x 11008 10.7, 48 x 11008 in tiles 15.2). */
template <int MR, typename... A> int few_cols(uint64_t nc, A... x)
{
    if (nc <= 1) return go_few<MR, 1>(x...);
    if constexpr (MR <= 2) {
        if (nc == 3) return go_few<MR, 3>(x...);
        if (nc > 3) return go_few<MR, 4>(x...);
    }
    return go_few<MR, 2>(x...);
}
int launch_few(const int8_t *a, uint64_t lda, const int8_t *b, uint64_t ldb, uint64_t m, uint32_t n, uint32_t k, const AnyOut &out, hipStream_t st)
{
    const uint64_t groups = (m + 63) / 64 * ((n + 15) / 16), nc = (groups + 255) / 256;
    if (m <= 16) return few_cols<1>(nc, a, lda, b, ldb, m, n, k, out, st);
    if (m <= 32) return few_cols<2>(nc, a, lda, b, ldb, m, n, k, out, st);
    if (m <= 48) return few_cols<3>(nc, a, lda, b, ldb, m, n, k, out, st);
    return few_cols<4>(nc, a, lda, b, ldb, m, n, k, out, st);
}

/* Whether k is split over the wavefronts of a workgroup.  Up to 64 rows, unless there are so many rows of b that tiles fill the chip and
 * their ring in LDS keeps more on its way (us, split and in tiles; k = 4096: 1 x 11008 13.4, 15.3; 48 x 11008 28.5, 17.3; 64 x 4096 15.1, 16.6;
 * 16 x 32000 36.0, 31.4; 64 x 32000 68, 37.5).  Beyond that where there are few tiles (512 x 512 x 4096 12.4, 14.3; 128 x 768 x 11008 26.9, 32.0;
 * 171 x 1500 x 5184 14.5, 17.2; 1868 x 179 x 2112, 90 tiles, 8.9, 9.5; 6000 x 64 x 4096, 94, 19.0, 19.6; 128 x 4096 x 4096, 128, 16.8, 19.6, but 15
 * and 14 with a in the caches) and k is not short (623 x 384 x 517 4.7, 5.4; 152 x 1939 x 80 5.8, 3.9; 83 x 3060 x 256 5.9, 4.6). */
bool by_few(uint64_t m, uint32_t n, uint32_t k)
{
    const uint64_t tiles = ((m + 63) / 64) * ((n + 63) / 64);
    return m <= 64 ? tiles < (m <= 32 ? 384u : 128u) : k > 384 && tiles <= 90;
}

/* A launch has fewer than 2^32 threads: 256 for each tile of 64, which results of up to 64 rows or columns take, else at most 512 for each of 256. */
bool beyond_a_launch(uint64_t m, uint32_t n)
{
    const auto tiles = [&](uint64_t s) { return ((m + s - 1) / s) * ((n + s - 1) / s); };
    return (m <= 64 ? tiles(64) / 2u : tiles(256)) >= (1u << 23) - 256u || (n <= 64 && tiles(64) >= (1u << 24));
}

template <typename T>
int launch_product(const int8_t *a, uint64_t lda, const int8_t *b, uint64_t ldb, uint64_t m, uint32_t n, uint32_t k, Out<T> out, hipStream_t st)
{
    const auto tiles = [&](uint64_t s) { return ((m + s - 1) / s) * ((n + s - 1) / s); };
    const uint32_t large = (uint32_t)tiles(256), rest = large % 256u, whole = rest <= 128u ? large - rest : large;
    /* Large results go past the caches, where the operands are read from, if their rows are whole lines: 8192 x 11008 x 1024 131 -> 124 us,
     * but 8192 x 5001 x 512 40 -> 56. */
    out.past = m > 64 && large >= 96 && whole_lines(out.c, out.ldc * sizeof(T));
    /* The largest tiles that still give work to most compute units (us by tiles of 256, halved where they are few, 128 and 64: 2048 x 4096 x 4096
     * 46.5, 51, 85; 1024 x 4096 x 4096 41.5, 29.5, 43.8; 4096 x 768 x 768 11.2, 9.4, 10.0; 1024 x 1536 x 1536 15.6, 11.8, 10.1; 6459 x 768 x 2877, 78
     * of 256, 35.9, 35.1, 43; 5579 x 617 x 1792, 66, 20.2, 17.0, 21.0).  Where k is short, those of 64 as long as the chip holds all of them at a time
     * (5596 x 704 x 97 8.8, 8.9, 6.4; 279 x 6592 x 640 10.8, 9.3, 7.7; 4715 x 768 x 768 11.5, 9.9, 11.9; 7819 x 779 x 192 9.6, 10.3, 10.3;
     * 6463 x 896 x 576 12.2, 12.4, 14.0).  Where the weights are read once, from memory, the ring is twice as long (48 x 11008 x 4096 20.7 -> 17.3).
     * No side is longer than the matrix needs (100 x 32000 x 4096 48.6, 34.2, 51.1; 40000 x 128 x 4096 63.6, 59.1, 66.4; 100000 x 64 x 1024 50.8,
     * 37.1, 33.8). */
    const bool wide = m > 128 && n > 128 && large >= 76;
    if (m <= 64)
        k_product<T, 64, 8><<<(uint32_t)tiles(64), 256, 0, st>>>(a, lda, b, ldb, m, n, k, out);
    else if (n <= 64 || (!wide && tiles(128) < 150) || (k <= 640 && tiles(64) <= 1024))
        k_product<T, 64, 4><<<(uint32_t)tiles(64), 256, 0, st>>>(a, lda, b, ldb, m, n, k, out);
    else if (!wide)
        k_product<T, 128, 4><<<(uint32_t)tiles(128), 256, 0, st>>>(a, lda, b, ldb, m, n, k, out);
    else
        k_product_large<T><<<whole + (large - whole) * 2u, 512, 0, st>>>(a, lda, b, ldb, m, n, k, out, whole);
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
    if (k > NSML_Q8_MAX_COLS || n > MAX_COLS || (m && lda > MAX_LD) || ldb > MAX_LD || beyond_a_launch(m, n)) return NSML_ECAP;
    if (m == 0) return NSML_OK;
    if (clash({area(c, type, m, ldc, n)}, {codes_area(a, m, lda, k), codes_area(b, n, ldb, k), floats(a_scale, m), floats(b_scale, n), floats(bias, n)}))
        return NSML_EINVAL;
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (by_few(m, n, k)) return launch_few(a, lda, b, ldb, m, n, k, AnyOut{c, ldc, a_scale, b_scale, bias, type}, st);
    if (type == NSML_F32) return launch_product(a, lda, b, ldb, m, n, k, Out<float>{static_cast<float *>(c), ldc, a_scale, b_scale, bias, false}, st);
    if (type == NSML_BF16) return launch_product(a, lda, b, ldb, m, n, k, Out<bf16>{static_cast<bf16 *>(c), ldc, a_scale, b_scale, bias, false}, st);
    return launch_product(a, lda, b, ldb, m, n, k, Out<f16>{static_cast<f16 *>(c), ldc, a_scale, b_scale, bias, false}, st);
}
