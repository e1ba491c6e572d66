/*
 * Weight gradient from a checkpoint: dw[j, i] = add[j, i] + col_scale[i] * sum over rows t of dy[t, j] * x[t, i].
 *
 * The summed dimension runs down the columns of both operands, and the matrix instructions want it side by side: eight rows of
 * eight neighbours are turned round in registers on their way to LDS, one byte permutation per two values.  There the codes
 * become bfloat16, which holds them exactly (the scale is a power of two).  dy is exact as well: bfloat16 as it is, float16 as
 * the sum of two bfloat16, binary32 of three, each a product of its own, so that the binary32 sum is all that rounds.
 */
#include "tiles.hpp"

namespace {

template <typename T> constexpr int PARTS = sizeof(T) == 4 ? 3 : 2;
template <> constexpr int PARTS<bf16> = 1;

/* Words of eight neighbours of dy. */
template <typename T> constexpr int WORDS = (int)sizeof(T) * 2;

/* Upper halves of two binary32 side by side: bfloat16 where the lower halves are 0, else cut off. */
__device__ __forceinline__ uint32_t upper2(float lo, float hi) { return __builtin_amdgcn_perm(to_bits(hi), to_bits(lo), 0x07060302u); }
/* What a bfloat16 cut off from v leaves; nothing of an infinity. */
__device__ __forceinline__ float left_of(float v)
{
    const float h = from_bits(to_bits(v) & 0xFFFF0000u);
    return h == v ? 0.0f : v - h;
}

template <typename T> struct Wgrad {
    Mat<const T> dy;
    Ckpt x;
    const float *col, *add;
    float *dw, *part;            /* part: sums of the slices when there is more than one */
    uint64_t lddw, rows;
    uint32_t n, k, slices;
};

/* A tile of BN x BK of dw by WM x WN wavefronts, one slice of the rows, 64 rows to a stage.  Half of the wavefronts bring dy, the
 * other half the codes: the next stage's are on their way to registers while this one's are multiplied. */
template <typename T, int BN, int BK, int WM, int WN>
__global__ void __launch_bounds__(WM * WN * 64)
k_wgrad(Wgrad<T> g)
{
    constexpr int P = PARTS<T>, W = WM * WN, TM = BN / WM / 32, TN = BK / WN / 32, HALF = W * 32;
    constexpr int STAGE = (P * BN + BK) * 128;
    static_assert(BN == HALF && BK == HALF, "a unit of 8 x 8 per thread");
    __shared__ __align__(16) uint8_t lds[2 * STAGE];
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64;
    const Tile tile = tile_of(blockIdx.x, (g.n + BN - 1) / BN, (g.k + BK - 1) / BK);
    const uint32_t n0 = tile.row * BN, k0 = tile.col * BK;
    const uint64_t stages = (g.rows + 63) / 64;
    const uint64_t from = stages * blockIdx.y / g.slices, to = stages * (blockIdx.y + 1) / g.slices;
    const uint32_t wm = wave / WN * (BN / WM), wn = wave % WN * (BK / WN);
    const bool brings_dy = wave < W / 2;
    const uint32_t unit = threadIdx.x % HALF, group = unit % (HALF / 8), chunk = unit / (HALF / 8);
    uint32_t raw[8][WORDS<T>];

    auto fetch = [&](uint64_t stage) {
        const uint64_t row0 = stage * 64 + chunk * 8;
        if (brings_dy) {
            const uint32_t c = n0 + group * 8;
            const int have = c < g.n ? (int)min(g.n - c, 8u) : 0;
#pragma unroll
            for (int i = 0; i < 8; i++) {
                if (row0 + i < g.rows && have == 8) {
                    const auto b = *reinterpret_cast<const Bytes<WORDS<T>> *>(g.dy.at(row0 + i, c));
#pragma unroll
                    for (int w = 0; w < WORDS<T>; w++) raw[i][w] = b.w[w];
                } else {
                    T v[8];
#pragma unroll
                    for (int e = 0; e < 8; e++) v[e] = row0 + i < g.rows && e < have ? *g.dy.at(row0 + i, c + e) : (T)0.0f;
                    __builtin_memcpy(raw[i], v, sizeof v);
                }
            }
        } else {
            const uint32_t c = k0 + group * 8;
#pragma unroll
            for (int i = 0; i < 8; i++) {
                uint2 q = make_uint2(0, 0);
                uint32_t e = 0;
                if (row0 + i < g.rows && c < g.k) {
                    q = *reinterpret_cast<const uint2 *>(g.x.q + (row0 + i) * g.x.ldq + c);
                    e = g.x.e[(row0 + i) * g.x.lde + c / 32u];
                }
                raw[i][0] = q.x, raw[i][1] = q.y, raw[i][2] = e;
            }
        }
    };
    auto put = [&](uint8_t *stage) {
        if (brings_dy) {
#pragma unroll
            for (int j = 0; j < 8; j++) {
                v4i p[P];
                if constexpr (P == 1) {
#pragma unroll
                    for (int i = 0; i < 4; i++)
                        p[0][i] = (int)__builtin_amdgcn_perm(raw[2 * i + 1][j / 2], raw[2 * i][j / 2], j % 2 ? 0x07060302u : 0x05040100u);
                } else {
#pragma unroll
                    for (int i = 0; i < 4; i++) {
                        float v[2];
#pragma unroll
                        for (int h = 0; h < 2; h++) {
                            if constexpr (P == 2) v[h] = (float)__builtin_bit_cast(f16, (uint16_t)(raw[2 * i + h][j / 2] >> (j % 2 * 16)));
                            else v[h] = from_bits(raw[2 * i + h][j]);
                        }
#pragma unroll
                        for (int s = 0; s < P; s++) {
                            p[s][i] = (int)upper2(v[0], v[1]);
                            v[0] = left_of(v[0]), v[1] = left_of(v[1]);
                        }
                    }
                }
#pragma unroll
                for (int s = 0; s < P; s++) *reinterpret_cast<v4i *>(stage + s * BN * 128 + place(group * 8 + j, chunk)) = p[s];
            }
        } else {
            float s[8];
#pragma unroll
            for (int i = 0; i < 8; i++) s[i] = ckpt_scale(raw[i][2]);
#pragma unroll
            for (int j = 0; j < 8; j++) {
                v4i p;
#pragma unroll
                for (int i = 0; i < 4; i++)
                    p[i] = (int)upper2((float)(int8_t)(raw[2 * i][j / 4] >> (j % 4 * 8)) * s[2 * i],
                                       (float)(int8_t)(raw[2 * i + 1][j / 4] >> (j % 4 * 8)) * s[2 * i + 1]);
                *reinterpret_cast<v4i *>(stage + P * BN * 128 + place(group * 8 + j, chunk)) = p;
            }
        }
    };

    v16f acc[TM][TN] = {};
    auto step = [&](const uint8_t *stage) {
#pragma unroll
        for (int s = 0; s < 4; s++) {
            v8bf fb[TN];
#pragma unroll
            for (int j = 0; j < TN; j++) fb[j] = __builtin_bit_cast(v8bf, frag(stage + P * BN * 128, wn + j * 32 + lane % 32, s * 2 + lane / 32));
#pragma unroll
            for (int p = P - 1; p >= 0; p--)
#pragma unroll
                for (int i = 0; i < TM; i++) {
                    const v8bf fa = __builtin_bit_cast(v8bf, frag(stage + p * BN * 128, wm + i * 32 + lane % 32, s * 2 + lane / 32));
#pragma unroll
                    for (int j = 0; j < TN; j++) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fa, fb[j], acc[i][j], 0, 0, 0);
                }
        }
    };
    if (from < to) fetch(from);
    uint32_t at = 0;
    for (uint64_t stage = from; stage < to; stage++, at ^= STAGE) {
        put(lds + at);
        wg_sync();                           /* this stage is there; the other half is read by nobody: all came here after it */
        if (stage + 1 < to) fetch(stage + 1);
        step(lds + at);
    }
    const uint64_t base = (uint64_t)blockIdx.y * g.n;
#pragma unroll
    for (int j = 0; j < TN; j++) {
        const uint32_t c = k0 + wn + j * 32 + lane % 32;
        if (c >= g.k) continue;
        const float s = g.col ? g.col[c] : 1.0f;
#pragma unroll
        for (int i = 0; i < TM; i++)
#pragma unroll
            for (int r = 0; r < 16; r++) {
                const uint32_t row = n0 + wm + i * 32 + acc_row(r, lane);
                if (row >= g.n) continue;
                if (g.slices > 1) g.part[(base + row) * g.k + c] = acc[i][j][r];
                else {
                    const float v = acc[i][j][r] * s;
                    g.dw[row * g.lddw + c] = g.add ? g.add[row * g.lddw + c] + v : v;
                }
            }
    }
}

/* The slices' sums added up in order. */
__global__ void __launch_bounds__(256) k_wgrad_sum(const float *part, const float *col, const float *add, float *dw, uint64_t lddw,
                                                   uint32_t n, uint32_t k, uint32_t slices)
{
    const uint32_t c = blockIdx.x * 256u + threadIdx.x;
    if (c >= k) return;
    for (uint32_t row = blockIdx.y; row < n; row += gridDim.y) {
        float v = 0.0f;
        for (uint32_t s = 0; s < slices; s++) v += part[((uint64_t)s * n + row) * k + c];
        if (col) v *= col[c];
        dw[row * lddw + c] = add ? add[row * lddw + c] + v : v;
    }
}

constexpr uint32_t SIDE = 128;
/* Rows are cut into slices where there are fewer tiles than the chip has room for at two a compute unit, but no slice is shorter than two stages. */
uint32_t slices_of(uint64_t rows, uint32_t n, uint32_t k)
{
    const uint64_t tiles = (uint64_t)((n + SIDE - 1) / SIDE) * ((k + SIDE - 1) / SIDE), stages = (rows + 63) / 64;
    uint64_t s = 512 / tiles;
    if (s > stages / 2) s = stages / 2;
    return s < 2 ? 1u : (uint32_t)s;
}

template <typename T> int launch_wgrad(const Wgrad<T> &g, hipStream_t st)
{
    const uint64_t tiles = (uint64_t)((g.n + SIDE - 1) / SIDE) * ((g.k + SIDE - 1) / SIDE);
    k_wgrad<T, 128, 128, 2, 2><<<dim3((uint32_t)tiles, g.slices), 256, 0, st>>>(g);
    const int rc = launched();
    if (rc || g.slices == 1) return rc;
    k_wgrad_sum<<<dim3((g.k + 255u) / 256u, g.n < 65535u ? g.n : 65535u), 256, 0, st>>>(g.part, g.col, g.add, g.dw, g.lddw, g.n, g.k, g.slices);
    return launched();
}

}  // namespace

extern "C" {

uint64_t nsml_ckpt8_wgrad_work(uint64_t rows, uint32_t n, uint32_t k)
{
    if (n == 0 || k == 0) return 0;
    const uint32_t s = slices_of(rows, n, k);
    return s > 1 ? (uint64_t)s * n * k * 4u : 0u;
}

int nsml_ckpt8_wgrad(const void *dy, int type, uint64_t lddy, const nsml_ckpt8 *x, const float *col_scale,
                     uint64_t rows, uint32_t n, uint32_t k, const float *add, float *dw, uint64_t lddw,
                     void *work, uint64_t work_bytes, void *stream)
{
    if (n == 0 || k == 0 || bad_type(type) || (rows && (bad_mat(dy, type, lddy, n) || bad_ckpt(x, k))) ||
        (col_scale && bad_f32(col_scale)) || (add && bad_f32(add)) || bad_mat(dw, NSML_F32, lddw, k))
        return NSML_EINVAL;
    const uint64_t need = nsml_ckpt8_wgrad_work(rows, n, k);
    if (need && (!work || !at_multiple(work, 16) || work_bytes < need)) return NSML_EINVAL;
    if ((uint64_t)((n + SIDE - 1) / SIDE) * ((k + SIDE - 1) / SIDE) >= (1u << 24)) return NSML_ECAP;
    hipStream_t st = static_cast<hipStream_t>(stream);
    const uint32_t slices = slices_of(rows, n, k);
    const auto go = [&](auto v) {
        using T = decltype(v);
        return launch_wgrad(Wgrad<T>{mat<T>(dy, lddy), ckpt_of(x), col_scale, add, dw, static_cast<float *>(work), lddw, rows, n, k, slices}, st);
    };
    if (type == NSML_F32) return go(float{});
    if (type == NSML_BF16) return go(bf16{});
    return go(f16{});
}

}  // extern "C"
