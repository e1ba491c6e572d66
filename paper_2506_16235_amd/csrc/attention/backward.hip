/*
 * Gradients of attention from its result: p = exp(s - lse), delta = do o, dp = do v, ds = p (dp - delta),
 *   dq = scale ds k      dk = scale ds^T q      dv = p^T do
 *
 * Kernels that make the scores anew: one goes through the keys for a tile of queries (dq), one or two through the queries of all heads for a tile of
 * keys (dk, dv).  Seven products up to 64 elements a head, eight beyond, in place of five, but every sum is one wavefront's in an order that
 * sizes alone decide: no atomics.  With few keys the queries are split, each split writes its sums in 32 bits, and k_grad_join adds them in order.
 *
 * Bound by the matrix instructions and what stands between them, two wavefronts on a SIMD at most (8192 tokens in documents of 351 to 4509, 32 heads of 128 over 8,
 * bfloat16: dq 317 us, dk and dv 611, join 30; 16 x 512 tokens, 12 heads of 64: dq 44, dk with dv 53).
 */
#include "attention.hpp"

namespace {

template <typename T> struct Grad {
    Heads<const T> q, k, v, o, d;        /* d: gradient of the result */
    const float *lse;
    Heads<T> dq, dk, dv;
    float *delta, *part;         /* part: sums of the splits when there is more than one, for dq of the keys, then for dk and dv of the queries */
    Seqs seqs;
    Group group;
    Reach reach;
    uint32_t heads, kv, dim, slots, splits, key_splits;
    float scale;
    int rest;                    /* rows of no sequence become zeros, of dq (1), dk (2) and dv (4) */
};

/* A split's part of a key's gradients: dk, then dv. */
__device__ __forceinline__ uint64_t part_at(uint64_t rows, uint32_t kv, uint32_t dim, uint32_t split, uint64_t row, uint32_t head)
{
    return ((split * rows + row) * kv + head) * (2u * dim);
}

/* A split's part of a query's gradient. */
__device__ __forceinline__ uint64_t query_part_at(uint64_t rows, uint32_t heads, uint32_t dim, uint32_t split, uint64_t row, uint32_t head)
{
    return ((split * rows + row) * heads + head) * dim;
}

/* float16 has few exponents: ds is brought to a power of two that its column's largest value so far decides, and the sums with it, so that what
 * is lost lies far below that.  The other types need none. */
template <typename T> struct Level {
    float up = 1.0f;
    template <int N, int DB> __device__ __forceinline__ void take(const float (&)[N], v16f (&)[DB]) {}
};
template <> struct Level<f16> {
    float up = from_bits(227u << 23);                /* 2^100 */
    template <int N, int DB> __device__ __forceinline__ void take(const float (&ds)[N], v16f (&acc)[DB])
    {
        float most = 0.0f;
#pragma unroll
        for (int e = 0; e < N; e++) most = fmaxf(most, fabsf(ds[e]));
        most = half_max(most);
        if (__ballot(most * up > 32768.0f)) {
            /* the largest to 2^7, so that few that are larger follow; what is lost lies 2^-32 below it, where a sum in binary32 holds nothing of it */
            const float now = most * up > 32768.0f ? from_bits((261u - min(to_bits(most) >> 23, 254u)) << 23) : up;
            const float f = now / up;
            up = now;
#pragma unroll
            for (int b = 0; b < DB; b++) acc[b] *= f;
        }
    }
};
/* Weights p as powers of two too large, for the same reason. */
template <typename T> constexpr float LIFT = 0.0f;
template <> constexpr float LIFT<f16> = 14.0f;
__device__ __forceinline__ float power(float e) { return __builtin_amdgcn_exp2f(e); }

/* ---------------------------------------------------------------- dq, and delta for the other kernel
 *
 * delta = do o has the rounding of o in it, which the gradient shows where a query's weight is on few keys.  The sum of ds over a query's keys is 0 but for what
 * delta is off by, so it is made beside ds, and dk always gets a delta without that.  dq is off by as much times the sum of p k.  MEND: that sum is made too, a
 * product that reads nothing more, and taken off at the end.  AGAIN, where registers do not last for it (dim beyond 64 in 16 bits): a tile of queries that see
 * EXACT keys at most goes through them for delta alone first.  One that sees more makes dq, and its wavefronts make theirs anew where delta is off by more
 * than STEPS, two steps of the type, of the root of the sum of ds^2 for some row.  Rounding o and weights alone makes 0.3 steps in the mean square of keys with
 * normal scores, and one row in 60000 comes to two (dq of 1200 tokens in bfloat16 is off by 0.24 % either way; 0.37 % in place of 0.29 where keys have
 * a mean as large as their deviation).  Those of a key with all but 0.001 of the weight come far beyond: off by 133 % with a delta that is never mended, 0.28 % so.  The
 * sums take 1 % of a step of 8192 tokens; one tile that goes through its keys twice ends last where all are long (4096 tokens, 32 heads of 128: 790 -> 840 us). */
constexpr uint32_t EXACT = 512;
template <typename T> constexpr float STEPS = 0.015625f;         /* 2^-6 */
template <> constexpr float STEPS<f16> = 0.001953125f;           /* 2^-9 */

template <typename T, int D, int W, int KB, Rows R>
__global__ void __launch_bounds__(W * 64, sizeof(T) == 2 ? 2 : 1)
k_attend_dq(Grad<T> g)
{
    typedef TileOf<T, D> L;
    constexpr int ROWS = W * 32, TILE = KB * L::ROW, DB = D / 32;
    constexpr bool MEND = sizeof(T) == 2 && D == 64, AGAIN = sizeof(T) == 2 && D > 64;      /* binary32 rounds o no more than anything else */
    typedef Cleaner<T, D, KB, W * 64> Clean;
    __shared__ __align__(16) uint8_t lds[4 * TILE + Clean::BYTES];
    const uint32_t wave = uniform(threadIdx.x / 64u), lane = threadIdx.x % 64u;
    const bool parts = sizeof(T) == 4 && g.key_splits > 1u;
    const Job job = job_of(blockIdx.x, g.kv, parts ? g.key_splits : 1u);
    uint32_t which, tile;
    find_tile<ROWS, false>(g.seqs.q_off, g.seqs.n, g.seqs.q_rows, g.group.n, job.slot, g.slots, which, tile);
    if (tile == 0xFFFFFFFFu) return;
    const Seq s = seq_of(g.seqs, which);
    const uint32_t head0 = job.head * g.group.n, r0 = tile * ROWS, rows = s.m * g.group.n;
    if (g.rest & 1 && job.split == 0) {
        const uint32_t room = s.q_room * g.group.n;
        for (uint32_t r = max(r0, rows) + threadIdx.x / 32u; r < min(r0 + ROWS, room); r += W * 2) {
            const uint32_t at = g.group.div(r);
            const float none[4] = {};
            for (uint32_t c = threadIdx.x % 32u * 4u; c < g.dim; c += 128u) put4<R>(g.dq.at((uint64_t)s.q0 + at, head0 + r - at * g.group.n), c, g.dim, none);
        }
    }
    if (r0 >= rows) return;
    const uint32_t wr = r0 + wave * 32u, last = rows - 1u;
    const uint32_t r = min(wr + lane % 32u, last), query = g.group.div(r), head = head0 + r - query * g.group.n;
    const Seen seen = seen_by(g.reach, s, query);
    const Seen first = seen_by(g.reach, s, g.group.div(r0)), end = seen_by(g.reach, s, g.group.div(min(r0 + ROWS - 1u, last)));
    const Seen wave_first = seen_by(g.reach, s, g.group.div(min(wr, last))), wave_end = seen_by(g.reach, s, g.group.div(min(wr + 31u, last)));
    uint32_t from = first.lo / KB, to = end.count ? (end.lo + end.count + KB - 1u) / KB : from;
    if (parts && to > from) {
        const uint32_t per = (to - from + g.key_splits - 1u) / g.key_splits;
        from = min(from + job.split * per, to), to = min(from + per, to);
    }
    const uint64_t row = (uint64_t)s.q0 + query;
    Frag<T> q[D / 16], d[D / 16];
    v16f square = {};
#pragma unroll
    for (int i = 0; i < D / 16; i++) {
        q[i] = frag_at<T, R>(g.q.at(row, head), i * 16u + lane / 32u * 8u, g.dim);
        d[i] = frag_at<T, R>(g.d.at(row, head), i * 16u + lane / 32u * 8u, g.dim);
        /* delta by the instruction that makes dp, so that a query of one key has ds = 0 exactly */
        mma(frag_at<T, R>(g.o.at(row, head), i * 16u + lane / 32u * 8u, g.dim), d[i], square);
        if constexpr (sizeof(T) == 4) q[i] *= g.scale * LOG2E;
    }
    float delta = 0.0f;
#pragma unroll
    for (int e = 0; e < 16; e++) delta = acc_row(e, lane) == lane % 32u ? square[e] : delta;
    {
        const float other = __shfl_xor(delta, 32);
        delta = (lane / 32u == lane / 4u % 2u) ? delta : other;
    }
    const float c = sizeof(T) == 4 ? 1.0f : g.scale * LOG2E, off = LIFT<T> - g.lse[row * g.heads + head] * LOG2E;

    const Loader<T, D, KB, W * 64, R> load;
    const RowLane<T, D> at_row(lane);
    const ColLane<T, D> at_col(lane);
    const T *k = g.k.at(s.k0, job.head), *v = g.v.at(s.k0, job.head);
    auto fetch = [&](uint32_t t, uint8_t *in) INLINE {
        load.keys(in, k, g.k.ld, t * KB, s.n, g.dim);
        load.keys(in + TILE, v, g.v.ld, t * KB, s.n, g.dim);
    };
    Clean cleaner(lds + 4 * TILE);
    float over = 0.0f;                               /* this lane's part of the sum of ds */
    uint64_t none = 0;                               /* lanes whose row sees a key of which an element was made zero in LDS */
    /* Weights and ds of 32 keys. */
    auto scores = [&](uint32_t t, const uint8_t *in, int b, bool all, float (&w)[16], float (&ds)[16]) INLINE {
        v16f p = {}, dp = {};
#pragma unroll
        for (int i = 0; i < D / 16; i++)
            if (used<T, D, R>(i * 16, g.dim)) mma(at_row(shared(in), b * 32u, i), q[i], p);
#pragma unroll
        for (int i = 0; i < D / 16; i++)
            if (used<T, D, R>(i * 16, g.dim)) mma(at_row(shared(in) + TILE, b * 32u, i), d[i], dp);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int e = 0; e < 16; e++) {
            w[e] = power(__builtin_fmaf(p[e], c, off));
            ds[e] = w[e] * (dp[e] - delta);
        }
        if (!all) {
            uint32_t here = t * KB + b * 32u + lane / 32u * 4u - seen.lo;
            asm("" : "+v"(here));                    /* one register and what a row adds, not a register for each row */
#pragma unroll
            for (int e = 0; e < 16; e++) {
                const bool sees = here + acc_row(e, 0) < seen.count;
                w[e] = sees ? w[e] : 0.0f;
                ds[e] = sees ? ds[e] : 0.0f;
            }
        }
    };
    bool idle = wr > last;                           /* this wavefront only brings what the others work on */
    /* All tiles by turns in both halves of LDS: work(tile, where it is, whether every row of the wavefront sees all of it). */
    auto tiles = [&](auto work) INLINE {
        auto turn = [&](uint32_t t, uint8_t *in, uint8_t *other) INLINE {
            tile_sync();
            if (t + 1u < to) fetch(t + 1u, other);
            const uint32_t a = t * KB, z = a + KB;
            const bool mixed = a < end.lo || z > first.lo + first.count, marked = mixed && cleaner.template clean<1>(in);
            if (idle || z <= wave_first.lo || a >= wave_end.lo + wave_end.count) return;
            if (marked)
#pragma unroll
                for (int b = 0; b < KB / 32; b++) none |= cleaner.seen(b * 32u, seen.lo - a - b * 32u, seen.lo + seen.count - a - b * 32u);
            work(t, in, a >= wave_end.lo && z <= wave_first.lo + wave_first.count);
        };
        if (from < to) fetch(from, lds);
        for (uint32_t t = from; t < to; t += 2u) {
            turn(t, lds, lds + 2 * TILE);
            if (t + 1u < to) turn(t + 1u, lds + 2 * TILE, lds);
        }
    };
    const float low = power(-LIFT<T>);
    /* Where this lane's row lies, made where it is needed, not kept in registers from tile to tile. */
    const auto own_row = [&](uint32_t &own_head) INLINE {
        uint32_t in = threadIdx.x % 32u;
        asm("" : "+v"(in));
        const uint32_t own = min(wr + in, last), at = g.group.div(own);
        own_head = head0 + own - at * g.group.n;
        return (uint64_t)s.q0 + at;
    };
    const bool few = end.lo + end.count <= first.lo + EXACT;
    v16f acc[DB] = {}, mean[MEND ? DB : 1] = {};
    Level<T> level;
    float squares = 0.0f;                            /* this lane's part of the sum of ds^2 */
    if (AGAIN && few) {
        tiles([&](uint32_t t, const uint8_t *in, bool all) INLINE {
#pragma unroll 1
            for (int b = 0; b < KB / 32; b++) {
                float w[16], ds[16];
                scores(t, in, b, all, w, ds);
#pragma unroll
                for (int e = 0; e < 16; e++) over += ds[e];
            }
        });
        delta += half_sum(over) * low;
        wg_sync();
    }
    auto pass = [&]() INLINE {
        tiles([&](uint32_t t, const uint8_t *in, bool all) INLINE {
#pragma unroll
            for (int b = 0; b < KB / 32; b++) {
                float w[16], ds[16];
                scores(t, in, b, all, w, ds);
                if constexpr (MEND || AGAIN)
#pragma unroll
                    for (int e = 0; e < 16; e++) over += ds[e];
                if constexpr (AGAIN)
#pragma unroll
                    for (int e = 0; e < 16; e++) squares = __builtin_fmaf(ds[e], ds[e], squares);
                level.take(ds, acc);
                Frag<T> fd[2], fw[2];
#pragma unroll
                for (int h = 0; h < 2; h++) {
                    float x[8];
#pragma unroll
                    for (int e = 0; e < 8; e++) x[e] = ds[h * 8 + e] * level.up;
                    fd[h] = rounded<T>(x);
                    fw[h] = rounded<T>(w + h * 8);
                }
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int h = 0; h < 2; h++)
#pragma unroll
                    for (int x = 0; x < DB; x++) {
                        if (!used<T, D, R>(x * 32, g.dim)) continue;
                        const Frag<T> f = at_col(shared(in), b * 32u + h * 16u, x);
                        mma(f, fd[h], acc[x]);
                        if constexpr (MEND) mma(f, fw[h], mean[x]);
                    }
            }
        });
    };
    pass();
    if (AGAIN && !few) {
        /* A row that has no need stays as it is or makes the same bits once more, so that none depends on its neighbours. */
        over = half_sum(over) * low;
        const bool off = fabsf(over) > STEPS<T> * low * __builtin_sqrtf(half_sum(squares));
        wg_sync();                                   /* nobody reads LDS any more */
        uint32_t *const any = reinterpret_cast<uint32_t *>(lds);
        const bool some = __ballot(off) != 0;
        any[wave] = some;
        wg_sync();
        uint32_t somebody = 0;
#pragma unroll
        for (int w = 0; w < W; w++) somebody |= any[w];
        wg_sync();
        uint32_t own_head;
        const uint64_t own = own_row(own_head) * g.heads + own_head;
        if (lane < 32u && wr + lane <= last) g.delta[own] = delta + over + Clean::none(none);
        if (uniform(somebody)) {
            delta = off ? delta + over : delta;
            idle |= !some;
            if (!idle) {
#pragma unroll
                for (int b = 0; b < DB; b++) acc[b] = v16f{};
                level = Level<T>{};
            }
            pass();
        }
    }
    if (none)
#pragma unroll
        for (int b = 0; b < DB; b++) acc[b] += Clean::none(none);
    const float r_off = MEND ? half_sum(over) * low : 0.0f;
    if (wr + lane % 32u > last) return;
    uint32_t own_head;
    const uint64_t own = own_row(own_head);
    if ((!AGAIN || few) && lane < 32u && job.split == 0) g.delta[own * g.heads + own_head] = delta + r_off + (MEND || AGAIN ? Clean::none(none) : 0.0f);
    const float f = g.scale * low / level.up, fm = g.scale * low * r_off;
    T *dq = g.dq.at(own, own_head);
    if constexpr (sizeof(T) == 4)
        if (parts) dq = g.part + query_part_at(g.seqs.q_rows, g.heads, g.dim, job.split, own, own_head);
#pragma unroll
    for (int b = 0; b < DB; b++)
#pragma unroll
        for (int e = 0; e < 4; e++) {
            float x[4];
#pragma unroll
            for (int i = 0; i < 4; i++) x[i] = acc[b][e * 4 + i] * f - (MEND ? mean[MEND ? b : 0][e * 4 + i] * fm : 0.0f);
            put4<R>(dq, b * 32u + e * 8u + lane / 32u * 4u, g.dim, x);
        }
}

/* The parts of dq added up in order, 32 threads to a row. */
template <typename T, int ROWS> __global__ void __launch_bounds__(256) k_query_join(Grad<T> g)
{
    const uint32_t head_of_keys = blockIdx.x / g.slots, c = threadIdx.x % 32u * 4u;
    uint32_t which, tile;
    find_slot<ROWS>(g.seqs.q_off, g.seqs.n, g.seqs.q_rows, g.group.n, blockIdx.x % g.slots, which, tile);
    if (tile == 0xFFFFFFFFu || c >= g.dim) return;
    const Seq s = seq_of(g.seqs, which);
    const uint64_t step = query_part_at(g.seqs.q_rows, g.heads, g.dim, 1, 0, 0);
    const int have = (int)min(g.dim - c, 4u);
    for (uint32_t r = tile * ROWS + threadIdx.x / 32u; r < min((tile + 1u) * ROWS, s.m * g.group.n); r += 8u) {
        const uint32_t query = g.group.div(r), head = head_of_keys * g.group.n + r - query * g.group.n;
        const uint64_t row = (uint64_t)s.q0 + query;
        const float *part = g.part + query_part_at(g.seqs.q_rows, g.heads, g.dim, 0, row, head) + c;
        float sum[4] = {};
#pragma unroll 4
        for (uint32_t i = 0; i < g.key_splits; i++) {
            float x[4];
            load4(part + i * step, have, x);
#pragma unroll
            for (int e = 0; e < 4; e++) sum[e] += x[e];
        }
        store4(g.dq.at(row, head) + c, have, sum);
    }
}

/* ---------------------------------------------------------------- dk and dv
 *
 * DK, DV: what is made.  Both at a time where registers last for both sums and two wavefronts on a SIMD; else each by a workgroup of its own, which
 * makes the scores once more. */

template <typename T, int D, int QB> constexpr int GRAD_STAGE = 2 * QB * TileOf<T, D>::ROW + 2 * QB * 4;
template <typename T, int D, int QB> constexpr int GRAD_LDS = 2 * GRAD_STAGE<T, D, QB> + Cleaner<T, D, QB, 64>::BYTES;

template <typename T, int D, int W, int QB, Rows R, bool DK, bool DV>
__device__ __forceinline__ void grad_keys(const Grad<T> &g, const Job &job, uint8_t *lds)
{
    typedef TileOf<T, D> L;
    constexpr int KEYS = W * 32, TILE = QB * L::ROW, DB = D / 32, STAGE = GRAD_STAGE<T, D, QB>;
    static_assert(QB <= W * 64, "");
    const uint32_t wave = uniform(threadIdx.x / 64u), lane = threadIdx.x % 64u;
    uint32_t which, tile;
    find_tile<KEYS, true>(g.seqs.k_off, g.seqs.n, g.seqs.k_rows, 1, job.slot, g.slots, which, tile);
    if (tile == 0xFFFFFFFFu) return;
    const Seq s = seq_of(g.seqs, which);
    const uint32_t k0 = tile * KEYS, head0 = job.head * g.group.n, rows = s.m * g.group.n;
    if (g.rest & 6 && job.split == 0) {
        for (uint32_t r = max(k0, s.n) + threadIdx.x / 32u; r < min(k0 + KEYS, s.k_room); r += W * 2) {
            const float none[4] = {};
            for (uint32_t c = threadIdx.x % 32u * 4u; c < g.dim; c += 128u) {
                if (DK && g.rest & 2) put4<R>(g.dk.at((uint64_t)s.k0 + r, job.head), c, g.dim, none);
                if (DV && g.rest & 4) put4<R>(g.dv.at((uint64_t)s.k0 + r, job.head), c, g.dim, none);
            }
        }
    }
    if (k0 >= s.n) return;
    const uint32_t wk = k0 + wave * 32u, key = min(wk + lane % 32u, s.n - 1u);
    /* The rows of queries that see a key: of the first and the last of the workgroup's and the wavefront's, and of this lane's. */
    const int64_t shift = (int64_t)s.n - s.m;
    const auto lo_of = [&](uint32_t j) { return (uint32_t)(g.reach.right < 0 ? 0 : within(j - shift - g.reach.right, s.m)) * g.group.n; };
    const auto hi_of = [&](uint32_t j) { return (uint32_t)(g.reach.left < 0 ? s.m : within(j - shift + g.reach.left + 1, s.m)) * g.group.n; };
    const uint32_t lo = lo_of(k0), hi = hi_of(min(k0 + KEYS, s.n) - 1u), wk_last = min(wk + 31u, s.n - 1u);
    const uint32_t first_all = lo_of(min(k0 + KEYS, s.n) - 1u), end_all = hi_of(k0);
    const uint32_t any_lo = lo_of(min(wk, wk_last)), any_hi = hi_of(wk_last), all_lo = lo_of(wk_last), all_hi = hi_of(min(wk, wk_last));
    const uint32_t my_lo = lo_of(key), my_hi = hi_of(key), my_count = my_hi > my_lo ? my_hi - my_lo : 0u;
    uint32_t from = lo / QB, to = hi > lo ? (hi + QB - 1u) / QB : from;
    if (g.splits > 1u) {
        const uint32_t per = (to - from + g.splits - 1u) / g.splits;
        from = min(from + job.split * per, to), to = min(from + per, to);
    }
    const uint64_t row = (uint64_t)s.k0 + key;
    Frag<T> k[D / 16], v[DK ? D / 16 : 1];
#pragma unroll
    for (int i = 0; i < D / 16; i++) {
        k[i] = frag_at<T, R>(g.k.at(row, job.head), i * 16u + lane / 32u * 8u, g.dim);
        if constexpr (DK) v[i] = frag_at<T, R>(g.v.at(row, job.head), i * 16u + lane / 32u * 8u, g.dim);
        if constexpr (sizeof(T) == 4) k[i] *= g.scale * LOG2E;
    }
    const float c = sizeof(T) == 4 ? 1.0f : g.scale * LOG2E;

    v16f ak[DK ? DB : 1] = {}, av[DV ? DB : 1] = {};
    Level<T> level;
    const Loader<T, D, QB, W * 64, R> load;
    const RowLane<T, D> at_row(lane);
    const ColLane<T, D> at_col(lane);
    const T *pq = g.q.at(s.q0, head0), *pd = g.d.at(s.q0, head0);
    const float *lse = g.lse + (uint64_t)s.q0 * g.heads + head0, *delta = g.delta + (uint64_t)s.q0 * g.heads + head0;
    auto fetch = [&](uint32_t t, uint8_t *in) INLINE {
        load.queries(in, pq, g.q.ld, g.q.hs, g.group, t * QB, rows, g.dim);
        load.queries(in + TILE, pd, g.d.ld, g.d.hs, g.group, t * QB, rows, g.dim);
        {
            /* every thread, so that none branches: several bring the same.  The stores wait for all that was asked for before. */
            const uint32_t own = threadIdx.x % QB, r = min(t * QB + own, rows - 1u), at = g.group.div(r);
            const uint64_t i = (uint64_t)at * g.heads + r - at * g.group.n;
            float *side = reinterpret_cast<float *>(in + 2 * TILE);
            side[own] = LIFT<T> - lse[i] * LOG2E;
            if (DK) side[QB + own] = delta[i];
        }
    };
    typedef Cleaner<T, D, QB, W * 64> Clean;
    Clean cleaner(lds + 2 * STAGE);
    uint64_t none = 0;                               /* lanes whose key is seen by a query of which a value was made zero in LDS */
    auto work = [&](uint32_t t, const uint8_t *in, bool all) INLINE {
        const Shared in_q = shared(in), in_d = in_q + TILE, side = in_d + TILE + lane / 32u * 16u;
#pragma unroll
        for (int b = 0; b < QB / 32; b++) {
            v16f p = {}, dp = {};
#pragma unroll
            for (int i = 0; i < D / 16; i++)
                if (used<T, D, R>(i * 16, g.dim)) mma(at_row(in_q, b * 32u, i), k[i], p);
            if constexpr (DK)
#pragma unroll
                for (int i = 0; i < D / 16; i++)
                    if (used<T, D, R>(i * 16, g.dim)) mma(at_row(in_d, b * 32u, i), v[i], dp);
            __builtin_amdgcn_sched_barrier(0);
            float w[16], ds[16];
#pragma unroll
            for (int x = 0; x < 4; x++) {
                typedef __attribute__((ext_vector_type(4))) float v4f;
                const v4f a = *reinterpret_cast<const __attribute__((address_space(3))) v4f *>(side + (b * 32 + x * 8) * 4);
                const v4f z = *reinterpret_cast<const __attribute__((address_space(3))) v4f *>(side + (QB + b * 32 + x * 8) * 4);
#pragma unroll
                for (int e = 0; e < 4; e++) {
                    w[x * 4 + e] = power(__builtin_fmaf(p[x * 4 + e], c, a[e]));
                    if constexpr (DK) ds[x * 4 + e] = w[x * 4 + e] * (dp[x * 4 + e] - z[e]);
                }
            }
            if (!all) {
                uint32_t here = t * QB + b * 32u + lane / 32u * 4u - my_lo;
                asm("" : "+v"(here));
#pragma unroll
                for (int e = 0; e < 16; e++) {
                    const bool sees = here + acc_row(e, 0) < my_count;
                    if constexpr (DV) w[e] = sees ? w[e] : 0.0f;
                    if constexpr (DK) ds[e] = sees ? ds[e] : 0.0f;
                }
            }
            if constexpr (DK) level.take(ds, ak);
            Frag<T> fd[2], fw[2];
#pragma unroll
            for (int h = 0; h < 2; h++) {
                if constexpr (DK) {
                    float x[8];
#pragma unroll
                    for (int e = 0; e < 8; e++) x[e] = ds[h * 8 + e] * level.up;
                    fd[h] = rounded<T>(x);
                }
                if constexpr (DV) fw[h] = rounded<T>(w + h * 8);
            }
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int h = 0; h < 2; h++)
#pragma unroll
                for (int x = 0; x < DB; x++) {
                    if (!used<T, D, R>(x * 32, g.dim)) continue;
                    if constexpr (DK) mma(at_col(in_q, b * 32u + h * 16u, x), fd[h], ak[x]);
                    if constexpr (DV) mma(at_col(in_d, b * 32u + h * 16u, x), fw[h], av[x]);
                }
        }
    };
    auto turn = [&](uint32_t t, uint8_t *in, uint8_t *other) INLINE {
        tile_sync();
        if (t + 1u < to) fetch(t + 1u, other);
        const uint32_t a = t * QB, z = a + QB;
        const bool mixed = a < first_all || z > end_all, marked = mixed && cleaner.template clean<2>(in);
        if (wk >= s.n || z <= any_lo || a >= any_hi) return;
        if (marked)
#pragma unroll
            for (int b = 0; b < QB / 32; b++) none |= cleaner.seen(b * 32u, my_lo - a - b * 32u, my_lo + my_count - a - b * 32u);
        work(t, in, a >= all_lo && z <= all_hi);
    };
    if (from < to) fetch(from, lds);
    for (uint32_t t = from; t < to; t += 2u) {
        turn(t, lds, lds + STAGE);
        if (t + 1u < to) turn(t + 1u, lds + STAGE, lds);
    }
    if (none)
#pragma unroll
        for (int b = 0; b < DB; b++) {
            if constexpr (DK) ak[b] += Clean::none(none);
            if constexpr (DV) av[b] += Clean::none(none);
        }
    if (wk + lane % 32u >= s.n) return;
    /* q was not scaled; in binary32 k was, but q is what dk is made of */
    const float fk = g.scale * power(-LIFT<T>) / level.up, fv = power(-LIFT<T>);
    float *part = g.splits > 1u ? g.part + part_at(g.seqs.k_rows, g.kv, g.dim, job.split, row, job.head) : nullptr;
#pragma unroll
    for (int b = 0; b < DB; b++)
#pragma unroll
        for (int e = 0; e < 4; e++) {
            const uint32_t at = b * 32u + e * 8u + lane / 32u * 4u;
            if constexpr (DK) {
                const float x[4] = {ak[b][e * 4] * fk, ak[b][e * 4 + 1] * fk, ak[b][e * 4 + 2] * fk, ak[b][e * 4 + 3] * fk};
                if (part) put4<R>(part, at, g.dim, x);
                else put4<R>(g.dk.at(row, job.head), at, g.dim, x);
            }
            if constexpr (DV) {
                const float y[4] = {av[b][e * 4] * fv, av[b][e * 4 + 1] * fv, av[b][e * 4 + 2] * fv, av[b][e * 4 + 3] * fv};
                if (part) put4<R>(part + g.dim, at, g.dim, y);
                else put4<R>(g.dv.at(row, job.head), at, g.dim, y);
            }
        }
}

template <typename T, int D, int W, int QB, Rows R>
__global__ void __launch_bounds__(W * 64, sizeof(T) == 2 ? 2 : 1)
k_attend_dkv(Grad<T> g)
{
    __shared__ __align__(16) uint8_t lds[GRAD_LDS<T, D, QB>];
    grad_keys<T, D, W, QB, R, true, true>(g, job_of(blockIdx.x, g.kv, g.splits), lds);
}
/* dk and dv of a tile by two workgroups of the same die, one after the other in the order of work. */
template <typename T, int D, int W, int QB, Rows R>
__global__ void __launch_bounds__(W * 64, sizeof(T) == 2 ? 2 : 1)
k_attend_dk_dv(Grad<T> g)
{
    __shared__ __align__(16) uint8_t lds[GRAD_LDS<T, D, QB>];
    const uint32_t half = gridDim.x / 2u, whole = half / 8u * 8u, id = blockIdx.x, left = half - whole;
    const bool paired = id < 2u * whole;
    const uint32_t idx = paired ? id / 16u * 8u + id % 8u : whole + (id - 2u * whole) % max(left, 1u);
    const bool dv = paired ? id / 8u % 2u : id - 2u * whole >= left;
    const Job job = job_of(idx, g.kv, g.splits);
    if (dv) grad_keys<T, D, W, QB, R, false, true>(g, job, lds);
    else grad_keys<T, D, W, QB, R, true, false>(g, job, lds);
}

/* The splits' parts added up in order, four neighbours a thread: 32 threads to a key up to 64 elements, else 64. */
template <typename T, int ROWS> __global__ void __launch_bounds__(256) k_grad_join(Grad<T> g)
{
    const uint32_t head = blockIdx.x / g.slots, across = g.dim <= 64u ? 32u : 64u;
    uint32_t which, tile;
    find_slot<ROWS>(g.seqs.k_off, g.seqs.n, g.seqs.k_rows, 1, blockIdx.x % g.slots, which, tile);
    if (tile == 0xFFFFFFFFu) return;
    const Seq s = seq_of(g.seqs, which);
    const uint32_t k0 = tile * ROWS, c = threadIdx.x % across * 4u, end = min(k0 + ROWS, s.n);
    const uint64_t step = part_at(g.seqs.k_rows, g.kv, g.dim, 1, 0, 0);
    const int have = c < 2u * g.dim ? (int)min(2u * g.dim - c, 4u) : 0;
    if (have == 0) return;
    for (uint32_t j = k0 + threadIdx.x / across; j < end; j += 256u / across) {
        const uint64_t row = (uint64_t)s.k0 + j;
        const float *part = g.part + part_at(g.seqs.k_rows, g.kv, g.dim, 0, row, head) + c;
        float sum[4] = {};
#pragma unroll 4
        for (uint32_t i = 0; i < g.splits; i++) {
            float x[4];
            load4(part + i * step, have, x);
#pragma unroll
            for (int e = 0; e < 4; e++) sum[e] += x[e];
        }
        T *dk = g.dk.at(row, head), *dv = g.dv.at(row, head);
        if (c + 4u <= g.dim) store4(dk + c, 4, sum);
        else if (c >= g.dim) store4(dv + (c - g.dim), have, sum);
        else                                         /* where one ends and the other begins */
#pragma unroll
            for (uint32_t e = 0; e < 4u; e++)
                if ((int)e < have) (c + e < g.dim ? dk[c + e] : dv[c + e - g.dim]) = (T)sum[e];
    }
}

/* ---------------------------------------------------------------- launches */

constexpr int WAVES = 4, TILE_ROWS = WAVES * 32, JOINED = 32;
/* Queries split over workgroups where there are too few tiles of keys to fill the chip, as where many heads share few heads of keys, and where those that
 * there are differ too much in what they cost: the first tiles of a long sequence are seen by all of it, twice what a tile is seen by in the mean, so
 * that 1024 workgroups are wanted where 512 run at a time; of several sequences, whose lengths are not known here, half as many again (us for 1024 and 1536:
 * 8192 tokens in documents of 351 to 4509, 32 heads over 8 1093, 942; 16 x 1024, 16 over 4 411, 485; 4096, 32 over 8 670, 655, unsplit 880; 2048 226, 235;
 * heads of 64, which make dk and dv at once, 4096, 32 over 32 327, 365). */
uint32_t splits_of(uint64_t q_rows, uint64_t k_rows, uint32_t seqs, uint32_t kv, uint32_t group, uint32_t dim)
{
    const uint64_t groups = std::max<uint64_t>(k_rows / TILE_ROWS, seqs) * kv * (dim > 64 ? 2u : 1u), tiles = q_rows * group / seqs / 64u;
    const uint64_t wanted = seqs > 1 && dim > 64 ? 1536 : 1024;
    const uint64_t s = std::min<uint64_t>(std::max(std::min(512 / groups, tiles / 2), std::min((wanted + groups - 1) / groups, tiles / 16)), 32);
    return s > 1 ? (uint32_t)s : 1u;
}

/* Keys split over workgroups for dq in binary32, whose products take sixteen times those of 16 bits: where half of the chip would idle, or a long
 * sequence's last tiles see far more than its first (us of a whole gradient, unsplit and split: 1031 tokens of five sequences, 6 heads of 72 over 2 131, 107;
 * 512 tokens, 8 heads of 128 159, 90; 2087 of two sequences, 4 heads of 128 319, 203; 4096, 8 heads of 128 1700, 1390; four of 512, 12 heads of 64, which
 * fill three quarters of it, 162, 174, so not there). */
uint32_t key_splits_of(int type, uint64_t q_rows, uint64_t k_rows, uint32_t seqs, uint32_t kv, uint32_t group, uint32_t dim)
{
    if (type != NSML_F32) return 1;
    const uint64_t groups = std::max<uint64_t>(q_rows * group / TILE_ROWS, seqs) * kv, tiles = k_rows / seqs / (dim > 64 ? 32u : 64u);
    const uint64_t s = std::max(groups <= 128 ? std::min(512 / groups, tiles / 2) : 1, std::min(1024 / groups, tiles / 16));
    return s > 1 ? (uint32_t)std::min<uint64_t>(s, 16) : 1u;
}

template <typename T, int D, Rows R> int launch(Grad<T> g, uint32_t q_slots, uint32_t k_slots, hipStream_t st)
{
    constexpr int B = D * sizeof(T) > 256 ? 32 : 64;
    if (q_slots) {
        g.slots = q_slots;
        k_attend_dq<T, D, WAVES, B, R><<<q_slots * g.kv * g.key_splits, WAVES * 64, 0, st>>>(g);
        if (const int rc = launched()) return rc;
        if constexpr (sizeof(T) == 4)
            if (g.key_splits > 1u) {
                g.slots = (uint32_t)(g.seqs.q_rows * g.group.n / JOINED) + g.seqs.n + 1u;
                k_query_join<T, JOINED><<<g.slots * g.kv, 256, 0, st>>>(g);
                if (const int rc = launched()) return rc;
            }
    }
    if (!k_slots) return NSML_OK;
    g.slots = k_slots;
    if constexpr (D > 64) k_attend_dk_dv<T, D, WAVES, B, R><<<2u * k_slots * g.kv * g.splits, WAVES * 64, 0, st>>>(g);
    else k_attend_dkv<T, D, WAVES, B, R><<<k_slots * g.kv * g.splits, WAVES * 64, 0, st>>>(g);
    const int rc = launched();
    if (rc || g.splits == 1u) return rc;
    g.slots = g.seqs.k_rows / JOINED + g.seqs.n + 1u;
    k_grad_join<T, JOINED><<<g.slots * g.kv, 256, 0, st>>>(g);
    return launched();
}

}  // namespace

static uint64_t delta_bytes(uint64_t q_rows, uint32_t heads) { return (q_rows * heads * 4u + 15u) / 16u * 16u; }

extern "C" {

uint64_t nsml_attention_backward_work(int type, uint64_t q_rows, uint64_t k_rows, uint32_t seqs, uint32_t heads, uint32_t kv_heads, uint32_t dim)
{
    if (bad_type(type) || bad_shape(q_rows, k_rows, seqs, heads, kv_heads, dim)) return 0;
    const uint32_t splits = splits_of(q_rows, k_rows, seqs, kv_heads, heads / kv_heads, dim);
    const uint32_t key_splits = key_splits_of(type, q_rows, k_rows, seqs, kv_heads, heads / kv_heads, dim);
    return delta_bytes(q_rows, heads) + std::max(splits > 1u ? splits * k_rows * kv_heads * dim * 8u : 0u, key_splits > 1u ? key_splits * q_rows * heads * dim * 4u : 0u);
}

int nsml_attention_backward(const nsml_heads *dout, const nsml_heads *q, const nsml_heads *k, const nsml_heads *v, const nsml_heads *o, const float *lse, int type,
                            const nsml_seqs *seqs, uint32_t heads, uint32_t kv_heads, uint32_t dim, int32_t left, int32_t right, float scale,
                            const nsml_heads *dq, const nsml_heads *dk, const nsml_heads *dv, int rest, void *work, uint64_t work_bytes, void *stream)
{
    if (!seqs || bad_type(type) || !(scale > 0.0f) || !(scale <= 2.0e38f) || bad_seqs(seqs)) return NSML_EINVAL;
    const uint64_t m = seqs->q_rows, n = seqs->k_rows;
    if (const int rc = bad_shape(m, n, seqs->n, heads, kv_heads, dim)) return rc;
    if ((m && (bad_heads(dout, type) || bad_heads(q, type) || bad_heads(o, type) || bad_f32(lse) || bad_results(dq, type, m, heads, dim))) ||
        (n && (bad_heads(k, type) || bad_heads(v, type) || bad_results(dk, type, n, kv_heads, dim) || bad_results(dv, type, n, kv_heads, dim))))
        return NSML_EINVAL;
    const uint64_t need = nsml_attention_backward_work(type, m, n, seqs->n, heads, kv_heads, dim);
    if (need && (!work || !at_multiple(work, 16) || work_bytes < need)) return NSML_EINVAL;
    const uint32_t q_slots = m ? (uint32_t)(m * (heads / kv_heads) / TILE_ROWS) + seqs->n + 1u : 0u, k_slots = n ? (uint32_t)(n / TILE_ROWS) + seqs->n + 1u : 0u;
    const uint32_t splits = splits_of(m, n, seqs->n, kv_heads, heads / kv_heads, dim);
    const uint32_t key_splits = key_splits_of(type, m, n, seqs->n, kv_heads, heads / kv_heads, dim);
    if (std::max<uint64_t>({q_slots * (uint64_t)key_splits, key_splits > 1u ? m * (heads / kv_heads) / JOINED + seqs->n + 1u : 0u, 2u * splits * (uint64_t)k_slots, splits > 1u ? n / JOINED + seqs->n + 1u : 0u}) * kv_heads >= 1u << 24) return NSML_ECAP;
    const auto at = [&](const nsml_heads *h) { return head_area(h, type, m, heads, dim); };
    const auto kt = [&](const nsml_heads *h) { return head_area(h, type, n, kv_heads, dim); };
    if (clash({at(dq), kt(dk), kt(dv), one_area(area(need ? work : nullptr, 1, 0, need))},
              {at(dout), at(q), at(o), kt(k), kt(v), one_area(area(lse, 1, 0, m * heads * 4u)), int_area(seqs->q_off, seqs->n + 1ull), int_area(seqs->k_off, seqs->n + 1ull),
               int_area(seqs->q_len, seqs->n), int_area(seqs->k_len, seqs->n)}))
        return NSML_EINVAL;
    const Rows like = rows_of((m == 0 || (fast_heads(q, type) && fast_heads(dout, type))) && (n == 0 || (fast_heads(k, type) && fast_heads(v, type))), type, dim);
    hipStream_t st = static_cast<hipStream_t>(stream);
    const auto go = [&](auto t) {
        using T = decltype(t);
        const Grad<T> g{heads_of<const T>(q), heads_of<const T>(k), heads_of<const T>(v), heads_of<const T>(o), heads_of<const T>(dout), lse, heads_of<T>(dq),
                        heads_of<T>(dk), heads_of<T>(dv), static_cast<float *>(work),
                        reinterpret_cast<float *>(static_cast<uint8_t *>(work) + delta_bytes(m, heads)), seqs_of(seqs), group_of(heads / kv_heads), Reach{left, right},
                        heads, kv_heads, dim, 0u, splits, key_splits, scale, rest};
        const auto with = [&](auto l) { return dim <= 64 ? launch<T, 64, decltype(l)::value>(g, q_slots, k_slots, st) : launch<T, 128, decltype(l)::value>(g, q_slots, k_slots, st); };
        if (like == WHOLE) return with(std::integral_constant<Rows, WHOLE>{});
        return like == CHUNKS ? with(std::integral_constant<Rows, CHUNKS>{}) : with(std::integral_constant<Rows, ANY>{});
    };
    if (type == NSML_F32) return go(float{});
    if (type == NSML_BF16) return go(bf16{});
    return go(f16{});
}

}  // extern "C"
