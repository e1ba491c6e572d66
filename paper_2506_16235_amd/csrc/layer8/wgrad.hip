/*
 * Weight gradient from a checkpoint: dw[j, i] = add[j, i] + col_scale[i] * sum over rows t of dy[t, j] * x[t, i].
 *
 * The summed dimension runs down the columns of both operands, and the matrix instructions want it side by side: eight rows of
 * eight neighbours are turned round in registers on their way to LDS, one byte permutation per two values.  There the codes
 * become bfloat16, which holds them exactly (the scale is a power of two).  dy is exact as well: bfloat16 as it is, float16 as
 * the sum of two bfloat16, binary32 of three, each a product of its own, so that the binary32 sum is all that rounds.
 */
#include "tiles.hpp"

#include <algorithm>
#include <cmath>
#include <type_traits>

namespace {

template <typename T> constexpr int PARTS = sizeof(T) == 4 ? 3 : 2;
template <> constexpr int PARTS<bf16> = 1;

/* Words of four neighbours of dy. */
template <typename T> constexpr int WORDS = (int)sizeof(T);

/* Upper halves of two binary32 side by side: bfloat16 where the lower halves are 0, else cut off. */
__device__ __forceinline__ uint32_t upper2(float lo, float hi) { return __builtin_amdgcn_perm(to_bits(hi), to_bits(lo), 0x07060302u); }
/* What a bfloat16 cut off from v leaves, exactly (of an infinity NaN: what it makes is not finite either way). */
__device__ __forceinline__ float left_of(float v) { return v - from_bits(to_bits(v) & 0xFFFF0000u); }

typedef const __attribute__((address_space(1))) uint8_t *Global;
template <int N> using Loose = std::conditional_t<N == 2, Loose2, Loose4>;

template <typename T> struct Wgrad {
    Mat<const T> dy;
    Ckpt x;
    const float *col, *add;
    float *dw, *part;            /* part: sums of the slices when there is more than one */
    uint64_t lddw, rows;
    uint32_t n, k, slices;
    bool past;                   /* dw past the caches */
};

/* Rows of a stage.  With parts half as many: two stages of a tile of 256 then fit LDS, and two workgroups with tiles of 128 a compute unit
 * (us with 64 rows, for which only tiles of 128 fit, and with 32: 8192 x 4096 x 4096 float16 743, 447, binary32 939, 619; 4096 x 2048 x 4096
 * by tiles of 128 both 188, 156 and 235, 208). */
template <typename T> constexpr int ROWS = PARTS<T> == 1 ? 64 : 32;
/* Where chunk c (eight rows of the stage) of a row of LDS lies. */
template <int N> __device__ __forceinline__ uint32_t spot_of(uint32_t row, uint32_t c) { return N == 64 ? place(row, c) : spot(row, c); }

/* A tile of BN x BK of dw by WM x WN wavefronts, one slice of the rows, ROWS to a stage.  Every thread brings an eighth of a stage's rows of
 * four neighbours of both operands: the next stage's wait in registers while this one is multiplied and go to the other half of LDS
 * between its matrix instructions, which leave the vector unit three quarters of its time.  Neighbour j of the four goes to row
 * j * BN / 4 + group of LDS: a wavefront whose blocks are the four neighbours of 32 groups holds four neighbours of dw in a lane.
 * NARROW: n < 4. */
template <typename T, int BN, int BK, int WM, int WN, bool NARROW>
__global__ void __launch_bounds__(WM * WN * 64)
k_wgrad(Wgrad<T> g)
{
    constexpr int P = PARTS<T>, N = ROWS<T>, R = N / 8, LINE = N * 2, W = WM * WN, TM = BN / WM / 32, TN = 4, WD = WORDS<T>;
    constexpr int STAGE = (P * BN + BK) * LINE;
    static_assert(BN == W * 32 && BK == BN && BK == WN * 128, "a unit of an eighth x 4 of both operands per thread, 128 columns per wavefront");
    __shared__ __align__(16) uint8_t lds[2 * STAGE];
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64;
    const Tile tile = tile_of(blockIdx.x, (g.n + BN - 1) / BN, (g.k + BK - 1) / BK);
    const uint32_t n0 = tile.row * BN, k0 = tile.col * BK;
    const uint64_t stages = (g.rows + N - 1) / N;
    const uint64_t from = stages * blockIdx.y / g.slices, to = stages * (blockIdx.y + 1) / g.slices;
    const uint32_t wm = wave / WN * (BN / WM), wn = wave % WN * 32u;        /* rows of LDS */
    const uint32_t group = threadIdx.x % (BN / 4), part = threadIdx.x / (BN / 4);
    /* Columns beyond the matrices: any that are there, as what comes of them is not stored.  The four that a row of dy ends in are read
     * from the last four, and moved (n >= 4), or one by one. */
    const uint32_t cd = n0 + group * 4u, cx = k0 + group * 4u;
    const bool ends = !NARROW && cd < g.n && cd + 4u > g.n;
    const uint32_t at_d = (cd + 4u <= g.n ? cd : NARROW ? 0u : g.n - 4u) * (uint32_t)sizeof(T);
    const uint32_t at_x = cx < g.k ? cx : 0u, at_e = at_x / 32u;
    const uint32_t ld_d = (uint32_t)g.dy.ld * (uint32_t)sizeof(T), ld_x = (uint32_t)g.x.ldq, ld_e = (uint32_t)g.x.lde;
    uint32_t d[R][WD], q[R], e[R];

    /* Where a thread's first row lies; the others are whole rows away, which is the same for all threads. */
    const uint32_t to_d = __umul24(part * R, ld_d) + at_d, to_x = __umul24(part * R, ld_x) + at_x, to_e = __umul24(part * R, ld_e) + at_e;
    auto fetch = [&](uint64_t stage, auto edge) {
        const uint64_t row0 = stage * N;
        const uint8_t *pd = reinterpret_cast<const uint8_t *>(g.dy.p) + row0 * ld_d;
        const uint8_t *px = reinterpret_cast<const uint8_t *>(g.x.q) + row0 * ld_x;
        const uint8_t *pe = g.x.e + row0 * ld_e;
        const uint32_t last = (uint32_t)min<uint64_t>(g.rows - row0, N) - 1u;
#pragma unroll
        for (int i = 0; i < R; i++) {
            Global rd = (Global)(pd + i * ld_d), rx = (Global)(px + i * ld_x), re = (Global)(pe + i * ld_e);
            if constexpr (!edge.value) {
                uint32_t od = to_d, ox = to_x, oe = to_e;
                asm("" : "+s"(rd), "+s"(rx), "+s"(re));      /* a row's address is the same for all threads, and what a thread adds fits */
                asm("" : "+v"(od), "+v"(ox), "+v"(oe));      /* the load itself: no addition of 64 bits per load */
                rd += od, rx += ox, re += oe;
            } else {                         /* rows beyond the matrix: its last one */
                const uint32_t row = min(part * R + i, last);
                rd = (Global)pd + (__umul24(row, ld_d) + at_d), rx = (Global)px + (__umul24(row, ld_x) + at_x), re = (Global)pe + (__umul24(row, ld_e) + at_e);
            }
            q[i] = *(const __attribute__((address_space(1))) uint32_t *)rx;
            e[i] = *re;
            if constexpr (!NARROW) {
                const Loose<WD> b = *(const __attribute__((address_space(1))) Loose<WD> *)rd;
#pragma unroll
                for (int w = 0; w < WD; w++) d[i][w] = b[w];
            } else {
                T v[4];
#pragma unroll
                for (uint32_t c = 0; c < 4; c++) v[c] = *(const __attribute__((address_space(1))) T *)(rd + min(c, g.n - 1) * (uint32_t)sizeof(T));
                __builtin_memcpy(d[i], v, sizeof v);
            }
        }
    };
    /* What was read where a matrix ends: rows beyond it become zeros, the four that a row of dy ends in were read with those before. */
    auto mend = [&](uint64_t stage) {
        const uint64_t have = g.rows - stage * N;
        if (have < N) {
#pragma unroll
            for (int i = 0; i < R; i++)
                if (part * R + i >= have) {
                    q[i] = e[i] = 0;
#pragma unroll
                    for (int w = 0; w < WD; w++) d[i][w] = 0;
                }
        }
        if (ends)
            for (uint32_t s = g.n % 4u; s < 4u; s++)
#pragma unroll
                for (int i = 0; i < R; i++) {
                    if constexpr (sizeof(T) == 2) {
                        d[i][0] = __builtin_amdgcn_alignbit(d[i][1], d[i][0], 16);
                        d[i][1] >>= 16;
                    } else {
                        d[i][0] = d[i][1], d[i][1] = d[i][2], d[i][2] = d[i][3];
                    }
                }
    };
    /* Neighbour j of the four, of both operands, as rows side by side: a chunk, or half of one. */
    auto put = [&](uint8_t *stage, int j) {
        typedef int Out __attribute__((ext_vector_type(R / 2)));
        Out p[P], x;
#pragma unroll
        for (int i = 0; i < R / 2; i++) {
            if constexpr (P == 1) {
                p[0][i] = (int)__builtin_amdgcn_perm(d[2 * i + 1][j / 2], d[2 * i][j / 2], j % 2 ? 0x07060302u : 0x05040100u);
            } else {
                float v[2];
#pragma unroll
                for (int h = 0; h < 2; h++) {
                    if constexpr (P == 2) v[h] = (float)__builtin_bit_cast(f16, (uint16_t)(d[2 * i + h][j / 2] >> (j % 2 * 16)));
                    else v[h] = from_bits(d[2 * i + h][j]);
                }
#pragma unroll
                for (int s = 0; s < P; s++) {
                    p[s][i] = (int)upper2(v[0], v[1]);
                    v[0] = left_of(v[0]), v[1] = left_of(v[1]);
                }
            }
            x[i] = (int)upper2((float)(int8_t)(q[2 * i] >> (j * 8)) * ckpt_scale(e[2 * i]),
                               (float)(int8_t)(q[2 * i + 1] >> (j * 8)) * ckpt_scale(e[2 * i + 1]));
        }
        const uint32_t row = j * (BN / 4) + group, at = N == 64 ? spot_of<N>(row, part) : spot_of<N>(row, part / 2) + part % 2 * 8u;
#pragma unroll
        for (int s = 0; s < P; s++) *reinterpret_cast<Out *>(stage + s * BN * LINE + at) = p[s];
        *reinterpret_cast<Out *>(stage + P * BN * LINE + at) = x;
    };

    v16f acc[TM][TN] = {};
    const uint32_t ra = spot_of<N>(wm + lane % 32, lane / 32), rb = P * BN * LINE + spot_of<N>(wn + lane % 32, lane / 32);
    /* A stage is multiplied in U turns, 16 rows of one part of dy each, the smallest part first. */
    constexpr int U = N / 16 * P, ALL = TM * TN;
    static_assert(U % 2 == 0 && U >= 4, "two sets of registers by turns");
    v8bf fa[2][TM], fb[2][TN];
    auto read = [&](uint32_t stage, int u) {
        const int s = u / P, p = P - 1 - u % P;
        const uint8_t *at_a = lds + ((ra + stage) ^ (s * 32u)), *at_b = lds + ((rb + stage) ^ (s * 32u));
        if (u % P == 0)
#pragma unroll
            for (int j = 0; j < TN; j++) fb[s & 1][j] = __builtin_bit_cast(v8bf, frag(at_b + j * (BK / 4 * LINE)));
#pragma unroll
        for (int i = 0; i < TM; i++) fa[u & 1][i] = __builtin_bit_cast(v8bf, frag(at_a + p * BN * LINE + i * 32 * LINE));
    };
    auto multiply = [&](int u, int from, int to) {
#pragma unroll
        for (int t = from; t < to; t++)
            acc[t / TN][t % TN] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fa[u & 1][t / TN], fb[u / P & 1][t % TN], acc[t / TN][t % TN], 0, 0, 0);
    };
    /* One turn: its first product waits for what it multiplies, the next turn's is read behind the others, with
     * `work` for the vector unit between them. */
    auto turn = [&](uint32_t next, int u, auto work) {
        wait_lds();
        multiply(u, 0, 1);
        __builtin_amdgcn_sched_barrier(0);
        read(next, (u + 1) % U);
        __builtin_amdgcn_sched_barrier(0);
        multiply(u, 1, ALL);
        work();
    };
    /* What the vector unit does in a turn goes between its products, some instructions behind each. */
    auto between = [&]() {
#pragma unroll
        for (int t = 1; t < ALL; t++) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x002, 7, 0);
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    /* The turn in which neighbour j is put: the last ones before the barrier, as what was asked for has then had the longest time to come. */
    constexpr auto turn_of = [](int j) { return U == 4 ? (j ? 2 : 1) : U - 5 + j; };
    /* edge: the tile or the slice holds an end of the matrices. */
    auto all = [&](auto edge) {
        fetch(from, edge);
        if constexpr (edge.value) mend(from);
#pragma unroll
        for (int j = 0; j < 4; j++) put(lds, j);
        /* Behind the last stage it is read again, and put where nobody looks: one copy of everything. */
        fetch(min(from + 1, to - 1), edge);
        wg_sync();
        read(0, 0);
        uint32_t at = 0;
        for (uint64_t stage = from; stage < to; stage++, at ^= STAGE) {
#pragma unroll
            for (int u = 0; u < U - 1; u++) {
                if constexpr (edge.value)
                    if (u == turn_of(0)) mend(min(stage + 1, to - 1));
                turn(at, u, [&] {
#pragma unroll
                    for (int j = 0; j < 4; j++)
                        if (turn_of(j) == u) put(lds + (at ^ STAGE), j);
                });
                if (u >= turn_of(0)) between();
                else __builtin_amdgcn_sched_barrier(0);
            }
            wg_sync();                       /* the next stage is there, and this one is in registers everywhere */
            fetch(min(stage + 2, to - 1), edge);         /* (between the products: the same within 2 %) */
            __builtin_amdgcn_sched_barrier(0);
            turn(at ^ STAGE, U - 1, [] {});
        }
    };
    if (from < to) {
        if (NARROW || n0 + BN > g.n || to * N > g.rows) all(std::true_type{});
        else all(std::false_type{});
    }
    const uint32_t c = k0 + (wn + lane % 32) * 4u;
    const int have = c < g.k ? (int)min(g.k - c, 4u) : 0;
    if (have == 0) return;
    float s[4] = {1.0f, 1.0f, 1.0f, 1.0f};
    if (g.col && g.slices == 1)
#pragma unroll
        for (int j = 0; j < 4; j++) s[j] = g.col[min(c + j, g.k - 1)];
    float *to_dw = g.slices > 1 ? g.part + (uint64_t)blockIdx.y * g.n * g.k : g.dw;
    const float *add = g.slices > 1 ? nullptr : g.add;
    const uint64_t ld = g.slices > 1 ? g.k : g.lddw;
#pragma unroll
    for (int i = 0; i < TM; i++)
#pragma unroll
        for (int r = 0; r < 16; r++) {
            const uint32_t at_row = wm + i * 32 + acc_row(r, lane), row = n0 + at_row % (BN / 4) * 4u + at_row / (BN / 4);
            if (row >= g.n) continue;
            float v[4], old[4] = {};
            if (add) load4(add + row * ld + c, have, old);
#pragma unroll
            for (int j = 0; j < 4; j++) v[j] = old[j] + acc[i][j][r] * s[j];
            if (g.past && have == 4) {
                Loose4 x;
                __builtin_memcpy(&x, v, 16);
                __builtin_nontemporal_store(x, reinterpret_cast<Loose4 *>(to_dw + row * ld + c));
            } else {
                store4(to_dw + row * ld + c, have, v);
            }
        }
}

/* The slices' sums added up in order, four columns a thread. */
__global__ void __launch_bounds__(256) k_wgrad_sum(const float *part, const float *col, const float *add, float *dw, uint64_t lddw,
                                                   uint32_t n, uint32_t k, uint32_t slices, uint32_t log2l)
{
    const uint32_t c = ((blockIdx.x << log2l) + (threadIdx.x & ((1u << log2l) - 1u))) * 4u, per = 256u >> log2l;
    if (c >= k) return;
    const int have = (int)min(k - c, 4u);
    const uint64_t slice = (uint64_t)n * k;
    float f[4] = {1.0f, 1.0f, 1.0f, 1.0f};
    if (col) load4(col + c, have, f);
    for (uint32_t row = blockIdx.y * per + (threadIdx.x >> log2l); row < n; row += gridDim.y * per) {
        const float *p = part + (uint64_t)row * k + c;
        float v[4] = {}, old[4] = {};
        if (add) load4(add + row * lddw + c, have, old);
#pragma unroll 4
        for (uint32_t s = 0; s < slices; s++) {
            float x[4];
            load4(p + s * slice, have, x);
#pragma unroll
            for (int i = 0; i < 4; i++) v[i] += x[i];
        }
#pragma unroll
        for (int i = 0; i < 4; i++) v[i] = old[i] + v[i] * f[i];
        store4(dw + row * lddw + c, have, v);
    }
}

/* Side of the tiles and number of slices of the rows: what is least by the time that it should take, of what fills one, two or three rounds of
 * 256 compute units, what balances the rows' time with that of joining the slices, and one slice.  Per 64 rows of a round, tiles of 256 take
 * `large` us, tiles of 128 `alone` where a compute unit has one of them and `two` where it has two; a round takes 1.3 us to begin and end;
 * joining takes 3 us, and for each slice 0.1 us and 8 bytes more for each element of dw (at 7 TB/s, part of them from caches).  Against the
 * least of all sides and slices, measured for 60 sizes of three types, what is taken was 1 % slower in the mean and 15 % at most (us of the
 * side / slices taken, and of others: bfloat16 8000 x 5000 x 1000 256/3 109, 128/1 201, 256/1 234; 8192 x 2048 x 2048 256/4 88, 256/3 96,
 * 128/1 139; 600 x 1200 x 1200 128/1 18, 128/4 24; float16 1027 x 768 x 768 128/5 21, 128/1 32; 4000 x 300 x 11008 256/5 105, 128/1 150).  A
 * side of 128 or less has tiles of 128, which hold it; those of fewer than four columns have no other kernel. */
struct Shape { uint32_t side, slices; uint64_t tiles; };
struct Rates { double large, alone, two; };
Shape shape_of(uint64_t rows, uint32_t n, uint32_t k, int type)
{
    const Rates r = type == NSML_BF16 ? Rates{1.9, 0.95, 1.25} : type == NSML_F16 ? Rates{2.95, 1.45, 1.95} : Rates{3.8, 1.9, 2.5};
    const uint64_t stages = (rows + 63) / 64;
    const double slice = 0.1 + (double)n * k * 1.15e-6;
    Shape best{};
    double least = 0.0;
    for (uint32_t side : {128u, 256u}) {
        if (side == 256 && (n <= 128 || k <= 128)) continue;
        const uint64_t tiles = ((uint64_t)n + side - 1) / side * (((uint64_t)k + side - 1) / side);
        const uint64_t even = (uint64_t)std::sqrt((side == 256 ? r.large : r.alone) * (double)stages / slice);
        for (uint64_t s : {uint64_t(1), 256 / tiles, 512 / tiles, 768 / tiles, std::min(even, 512 / tiles)}) {
            if (s == 0 || (s > 1 && s > stages)) continue;
            const uint64_t groups = tiles * s, per = (stages + s - 1) / s;
            const uint64_t full = groups / (side == 256 ? 256 : 512), rest = groups % (side == 256 ? 256 : 512);
            const double one = side == 256 ? r.large : r.two, last = side == 128 && rest <= 256 ? r.alone : one;
            const double join = s > 1 ? 3.0 + (double)s * slice : 0.0;
            const double us = (double)full * ((double)per * one + 1.3) + (rest ? (double)per * last + 1.3 : 0.0) + join;
            if (best.side == 0 || us < least) best = {side, (uint32_t)s, tiles}, least = us;
        }
    }
    return best;
}

template <typename T> int launch_wgrad(const Wgrad<T> &g, const Shape &s, hipStream_t st)
{
    const dim3 grid((uint32_t)s.tiles, s.slices);
    if (s.side == 256) k_wgrad<T, 256, 256, 4, 2, false><<<grid, 512, 0, st>>>(g);
    else if (g.n < 4) k_wgrad<T, 128, 128, 4, 1, true><<<grid, 256, 0, st>>>(g);
    else k_wgrad<T, 128, 128, 4, 1, false><<<grid, 256, 0, st>>>(g);
    const int rc = launched();
    if (rc || s.slices == 1) return rc;
    uint32_t log2l = 0;
    while (log2l < 8u && (4u << log2l) < g.k) log2l++;
    const uint32_t rows = (g.n + (256u >> log2l) - 1u) / (256u >> log2l);
    k_wgrad_sum<<<dim3((g.k + (4u << log2l) - 1u) / (4u << log2l), rows < 65535u ? rows : 65535u), 256, 0, st>>>(g.part, g.col, g.add, g.dw, g.lddw, g.n, g.k, g.slices, log2l);
    return launched();
}

}  // namespace

extern "C" {

uint64_t nsml_ckpt8_wgrad_work(uint64_t rows, uint32_t n, uint32_t k)
{
    if (n == 0 || k == 0) return 0;
    /* enough for every type */
    uint32_t s = 1;
    for (int type : {NSML_F32, NSML_BF16, NSML_F16}) s = std::max(s, shape_of(rows, n, k, type).slices);
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
    if (n > MAX_COLS || k > MAX_COLS) return NSML_ECAP;
    const Shape s = shape_of(rows, n, k, type);
    /* A launch has fewer than 2^32 threads: 512 for each tile of 256, 256 for each of 128. */
    if (s.tiles >= (s.side == 256 ? 1u << 23 : 1u << 24) || (rows && (lddy >= MAX_LD || x->ldq >= MAX_LD || x->lde >= MAX_LD))) return NSML_ECAP;
    const Area out = area(dw, NSML_F32, n, lddw, k);
    if (clash({out, area(need ? work : nullptr, 1, 0, need)},
              {area(dy, type, rows, lddy, n), codes_area(x, rows, k), exps_area(x, rows, k), floats(col_scale, k), apart(area(add, NSML_F32, n, lddw, k), out)}))
        return NSML_EINVAL;
    hipStream_t st = static_cast<hipStream_t>(stream);
    /* Large results past the caches, where dy and x are read from, if their rows are whole lines (8192 x 11008 x 4096: 764 -> 728 us; see
     * the products for rows that are not). */
    const bool past = s.side == 256 && s.slices == 1 && whole_lines(dw, lddw * 4u);
    const auto go = [&](auto v) {
        using T = decltype(v);
        return launch_wgrad(Wgrad<T>{mat<T>(dy, lddy), ckpt_of(x), col_scale, add, dw, static_cast<float *>(work), lddw, rows, n, k, s.slices, past}, s, st);
    };
    if (type == NSML_F32) return go(float{});
    if (type == NSML_BF16) return go(bf16{});
    return go(f16{});
}

}  // extern "C"
