/*
 * Attention of packed sequences: s = scale q k, p = softmax over the keys that a query sees, o = p v, lse = log of the sum of exp s.
 *
 * One pass over the keys with a running maximum and sum.  Scores come with keys as rows and queries as columns, so that a query's maximum and sum are a
 * lane's own and its other half's; p leaves the registers as the operand of the second product.
 *
 * Prompts are bound by the matrix instructions, which wait while maxima and exponentials are made unless the other wavefront of the SIMD has products (8192 causal
 * tokens, 32 heads of 128 in bfloat16: 549 us, 1.0 Pflop/s; 32768 over 8 heads of keys 8.2 ms, 1.07); single tokens by memory (16 over 4096 to 16384 keys, 32
 * heads of 128 over 8: 135 us, 4.3 TB/s) or, when few, by a chain of dependent loads (one over 777 keys, 12 heads of 64: 8 us and 4 to join).
 */
#include "attention.hpp"

namespace {

template <typename T> struct Attend {
    Heads<const T> q, k, v;
    Heads<T> o;
    float *lse, *part;           /* part: sums of the splits when there is more than one */
    Seqs seqs;
    Group group;
    Reach reach;
    uint32_t heads, kv, dim, slots, splits;
    float scale;
    int rest;                    /* rows of no sequence become zeros, of the result (1) and of lse (2) */
};

constexpr uint32_t FEW_ROWS = 32, MOST_SPLITS = 64;

/* A split's part of a row: dim sums, the maximum in powers of two and the sum of weights. */
__device__ __forceinline__ uint64_t part_at(uint64_t rows, uint32_t heads, uint32_t dim, uint32_t split, uint64_t row, uint32_t head)
{
    return ((split * rows + row) * heads + head) * (dim + 2u);
}

/* W wavefronts, KB keys to a tile.  FEW = false: 32 rows to each wavefront, which all read the same keys.  FEW: 32 rows for all of them, each takes 32
 * keys of a tile, and what they have is joined through LDS.  Two tiles in LDS: more of them, and fewer workgroups beside each other, were slower (us for
 * 16 tokens, 32 heads over 8, up to 16384 keys: two wavefronts with two tiles 141, with four 196; four with two 160). */
template <typename T, int D, int W, int KB, bool FEW, Rows R>
__global__ void __launch_bounds__(W * 64, sizeof(T) == 2 ? 2 : 1)
k_attend(Attend<T> g)
{
    typedef TileOf<T, D> L;
    constexpr int ROWS = FEW ? 32 : W * 32, BLOCKS = FEW ? 1 : KB / 32, TILE = KB * L::ROW, DB = D / 32;
    static_assert(!FEW || KB == W * 32, "a block of keys to each wavefront");
    typedef Cleaner<T, D, KB, W * 64> Clean;
    __shared__ __align__(16) uint8_t lds[4 * TILE + Clean::BYTES];
    static_assert(!FEW || W * (DB * 16 * 64 + 64) * 4 <= 4 * TILE, "room for the join");
    const uint32_t wave = uniform(threadIdx.x / 64u), lane = threadIdx.x % 64u;
    const Job job = job_of(blockIdx.x, g.kv, g.splits);
    uint32_t which, tile;
    if constexpr (FEW) find_slot<ROWS>(g.seqs.q_off, g.seqs.n, g.seqs.q_rows, g.group.n, job.slot, which, tile);
    else find_tile<ROWS, false>(g.seqs.q_off, g.seqs.n, g.seqs.q_rows, g.group.n, job.slot, g.slots, which, tile);
    if (tile == 0xFFFFFFFFu) return;
    const Seq s = seq_of(g.seqs, which);
    const uint32_t head0 = job.head * g.group.n, r0 = tile * ROWS, rows = s.m * g.group.n;

    /* Rows of the room that hold no query. */
    if (g.rest && job.split == 0) {
        const uint32_t room = s.q_room * g.group.n;
        for (uint32_t r = max(r0, rows) + threadIdx.x / 32u; r < min(r0 + ROWS, room); r += W * 2) {
            const uint32_t at = g.group.div(r), head = head0 + r - at * g.group.n;
            const float none[4] = {};
            if (g.rest & 1)
                for (uint32_t c = threadIdx.x % 32u * 4u; c < g.dim; c += 128u) put4<R>(g.o.at((uint64_t)s.q0 + at, head), c, g.dim, none);
            if (g.rest & 2 && threadIdx.x % 32u == 0) g.lse[((uint64_t)s.q0 + at) * g.heads + head] = from_bits(0xFF800000u);
        }
    }
    if (r0 >= rows) return;

    /* The rows of this wavefront, and the keys that the workgroup and it go through. */
    const uint32_t wr = r0 + (FEW ? 0u : wave * 32u), last = rows - 1u;
    const uint32_t r = min(wr + lane % 32u, last), query = g.group.div(r), head = head0 + r - query * g.group.n;
    const Seen seen = seen_by(g.reach, s, query);
    const Seen first = seen_by(g.reach, s, g.group.div(r0)), end = seen_by(g.reach, s, g.group.div(min(r0 + ROWS - 1u, last)));
    const Seen wave_first = seen_by(g.reach, s, g.group.div(min(wr, last))), wave_end = seen_by(g.reach, s, g.group.div(min(wr + 31u, last)));
    uint32_t from = first.lo / KB, to = (end.lo + end.count + KB - 1u) / KB;
    if (end.count == 0) to = from;
    if (g.splits > 1u && to > from) {
        const uint32_t per = (to - from + g.splits - 1u) / g.splits;
        from = min(from + job.split * per, to), to = min(from + per, to);
    }
    const float c = sizeof(T) == 4 ? 1.0f : g.scale * LOG2E;
    Frag<T> q[D / 16];
#pragma unroll
    for (int i = 0; i < D / 16; i++) {
        q[i] = frag_at<T, R>(g.q.at((uint64_t)s.q0 + query, head), i * 16u + lane / 32u * 8u, g.dim);
        if constexpr (sizeof(T) == 4) q[i] *= g.scale * LOG2E;       /* so that the largest score's weight is 1 exactly */
    }

    v16f o[DB] = {};
    float top = LOWEST, sum = 0.0f;              /* the maximum times c, in powers of two; the sum of this lane's weights */
    const Loader<T, D, KB, W * 64, R> load;
    const RowLane<T, D> at_k(lane);
    const ColLane<T, D> at_v(lane);
    const T *k = g.k.at(s.k0, job.head), *v = g.v.at(s.k0, job.head);
    auto fetch = [&](uint32_t t, uint8_t *in) INLINE {
        load.keys(in, k, g.k.ld, t * KB, s.n, g.dim);
        load.keys(in + TILE, v, g.v.ld, t * KB, s.n, g.dim);
    };
    const uint32_t block0 = FEW ? wave * 32u : 0u;
    Clean cleaner(lds + 4 * TILE);
    uint64_t none = 0;                           /* lanes whose row sees a value that was made zero in LDS */
    /* all: every row of the wavefront sees every key of its blocks. */
    auto work = [&](uint32_t t, const uint8_t *in, bool all) INLINE {
        const uint32_t key0 = t * KB + block0;
        const Shared in_k = shared(in) + block0 * L::ROW, in_v = in_k + TILE;
        v16f p[BLOCKS] = {};
#pragma unroll
        for (int b = 0; b < BLOCKS; b++)
#pragma unroll
            for (int i = 0; i < D / 16; i++)
                if (used<T, D, R>(i * 16, g.dim)) mma(at_k(in_k, b * 32u, i), q[i], p[b]);
        __builtin_amdgcn_sched_barrier(0);
        if (!all) {
            uint32_t first = key0 + lane / 32u * 4u - seen.lo;
            asm("" : "+v"(first));               /* one register and what a row adds, not a register for each row */
#pragma unroll
            for (int b = 0; b < BLOCKS; b++)
#pragma unroll
                for (int e = 0; e < 16; e++) p[b][e] = first + (b * 32u + acc_row(e, 0)) < seen.count ? p[b][e] : from_bits(0xFF800000u);
        }
        float most = LOWEST;
#pragma unroll
        for (int b = 0; b < BLOCKS; b++)
#pragma unroll
            for (int e = 0; e < 16; e++) most = fmaxf(most, p[b][e]);
        most = half_max(most) * c;
        /* Weights up to 2^8 do no harm, so the sums are seldom brought to another maximum, each row's by what it alone holds. */
        if (__ballot(most > top + 8.0f)) {
            const float now = most > top + 8.0f ? most : top, f = __builtin_amdgcn_exp2f(top - now);
            top = now;
            sum *= f;
#pragma unroll
            for (int b = 0; b < DB; b++) o[b] *= f;
        }
        const float off = OFFSET<T> - top;
        Frag<T> w[BLOCKS * 2];
#pragma unroll
        for (int b = 0; b < BLOCKS; b++)
#pragma unroll
            for (int h = 0; h < 2; h++) {
                float x[8];
#pragma unroll
                for (int e = 0; e < 8; e++) {
                    x[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(p[b][h * 8 + e], c, off));
                    sum += x[e];
                }
                w[b * 2 + h] = rounded<T>(x);
            }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int b = 0; b < BLOCKS * 2; b++)
#pragma unroll
            for (int d = 0; d < DB; d++)
                if (used<T, D, R>(d * 32, g.dim)) mma(at_v(in_v, b * 16u, d), w[b], o[d]);
    };
    /* One tile in the half of LDS that `in` is; the next one is asked for as soon as nobody reads the other half.  In 16 bits the compiler waits for it before the
     * transposing reads of this one. */
    auto turn = [&](uint32_t t, uint8_t *in, uint8_t *other) INLINE {
        tile_sync();
        if (t + 1u < to) fetch(t + 1u, other);
        const bool mixed = t * KB < end.lo || (t + 1u) * KB > first.lo + first.count, marked = mixed && cleaner.template clean<1>(in + TILE);
        const uint32_t a = t * KB + block0, z = a + BLOCKS * 32u;
        if (wr > last || z <= wave_first.lo || a >= wave_end.lo + wave_end.count) return;
        if (marked)
#pragma unroll
            for (int b = 0; b < BLOCKS; b++) none |= cleaner.seen(block0 + b * 32u, seen.lo - a - b * 32u, seen.lo + seen.count - a - b * 32u);
        work(t, in, a >= wave_end.lo && z <= wave_first.lo + wave_first.count);
    };
    if (from < to) fetch(from, lds);
    for (uint32_t t = from; t < to; t += 2u) {
        turn(t, lds, lds + 2 * TILE);
        if (t + 1u < to) turn(t + 1u, lds + 2 * TILE, lds);
    }
    sum = half_sum(sum);
    if (none)
#pragma unroll
        for (int b = 0; b < DB; b++) o[b] += Clean::none(none);

    if constexpr (FEW) {
        /* Everybody's maximum and sums, then the sums brought to the largest and added up in the order of the wavefronts, each by one for its columns. */
        wg_sync();
        float *m = reinterpret_cast<float *>(lds), *z = m + W * 32, *acc = z + W * 32 + lane;
        if (lane < 32u) m[wave * 32u + lane] = top, z[wave * 32u + lane] = sum;
#pragma unroll
        for (int b = 0; b < DB; b++)
#pragma unroll
            for (int e = 0; e < 16; e++) acc[((wave * DB + b) * 16 + e) * 64] = o[b][e];
        wg_sync();
        float now = LOWEST, f[W];
#pragma unroll
        for (int w = 0; w < W; w++) now = fmaxf(now, m[w * 32 + lane % 32u]);
        sum = 0.0f, top = now;
#pragma unroll
        for (int w = 0; w < W; w++) f[w] = __builtin_amdgcn_exp2f(m[w * 32 + lane % 32u] - now), sum += z[w * 32 + lane % 32u] * f[w];
#pragma unroll
        for (int b = 0; b < DB; b++) {
            if (wave != (uint32_t)b % W) continue;
#pragma unroll
            for (int e = 0; e < 16; e++) {
                float v = 0.0f;
#pragma unroll
                for (int w = 0; w < W; w++) v += acc[((w * DB + b) * 16 + e) * 64] * f[w];
                o[b][e] = v;
            }
        }
    }
    if (wr + lane % 32u > last) return;
    const uint64_t row = (uint64_t)s.q0 + query;
    if (g.splits > 1u) {
        float *part = g.part + part_at(g.seqs.q_rows, g.heads, g.dim, job.split, row, head);
#pragma unroll
        for (int b = 0; b < DB; b++) {
            if (FEW && wave != (uint32_t)b % W) continue;
#pragma unroll
            for (int e = 0; e < 4; e++) {
                const float v[4] = {o[b][e * 4], o[b][e * 4 + 1], o[b][e * 4 + 2], o[b][e * 4 + 3]};
                put4<R>(part, b * 32u + e * 8u + lane / 32u * 4u, g.dim, v);
            }
        }
        if (lane < 32u && (!FEW || wave == 0)) part[g.dim] = top, part[g.dim + 1u] = sum;
    } else {
        const float f = sum == 0.0f ? 0.0f : 1.0f / sum;
#pragma unroll
        for (int b = 0; b < DB; b++) {
            if (FEW && wave != (uint32_t)b % W) continue;
#pragma unroll
            for (int e = 0; e < 4; e++) {
                const float v[4] = {o[b][e * 4] * f, o[b][e * 4 + 1] * f, o[b][e * 4 + 2] * f, o[b][e * 4 + 3] * f};
                put4<R>(g.o.at(row, head), b * 32u + e * 8u + lane / 32u * 4u, g.dim, v);
            }
        }
        if (lane < 32u && (!FEW || wave == 0)) g.lse[row * g.heads + head] = sum == 0.0f ? from_bits(0xFF800000u) : (top + __log2f(sum) - OFFSET<T>) * LN2;
    }
}

/* The splits' parts of a row joined, a workgroup per query and head: 32 threads to a part, eight parts at a time, then the eight sums in order (a wavefront
 * that went through 62 parts one after the other took 25 us, these 5). */
template <typename T> __global__ void __launch_bounds__(256) k_attend_join(Attend<T> g)
{
    __shared__ float sums[8][128], factors[MOST_SPLITS];
    const uint32_t lane = threadIdx.x % 64u, head_of_keys = blockIdx.x / g.slots;
    uint32_t which, r;
    find_slot<1>(g.seqs.q_off, g.seqs.n, g.seqs.q_rows, g.group.n, blockIdx.x % g.slots, which, r);
    if (r == 0xFFFFFFFFu) return;
    const Seq s = seq_of(g.seqs, which);
    if (r >= s.m * g.group.n) return;
    const uint32_t query = g.group.div(r), head = head_of_keys * g.group.n + r - query * g.group.n;
    const uint64_t row = (uint64_t)s.q0 + query, step = part_at(g.seqs.q_rows, g.heads, g.dim, 1, 0, 0);
    const float *part = g.part + part_at(g.seqs.q_rows, g.heads, g.dim, 0, row, head);
    const uint32_t own = threadIdx.x / 32u, c = threadIdx.x % 32u * 4u;
    /* every wavefront finds the maximum and what each part is multiplied by; one of them keeps it for all */
    const bool has = lane < g.splits;
    const float mine = has ? part[lane * step + g.dim] : LOWEST, weight = has ? part[lane * step + g.dim + 1u] : 0.0f;
    float top = mine;
#pragma unroll
    for (int d = 32; d; d /= 2) top = fmaxf(top, __shfl_xor(top, d));
    const float factor = __builtin_amdgcn_exp2f(mine - top);
    float sum = weight * factor;
#pragma unroll
    for (int d = 32; d; d /= 2) sum += __shfl_xor(sum, d);
    if (threadIdx.x < MOST_SPLITS) factors[threadIdx.x] = factor;
    wg_sync();
    float v[4] = {};
    const int have = c < g.dim ? (int)min(g.dim - c, 4u) : 0;
    if (have)
#pragma unroll 4
        for (uint32_t i = own; i < g.splits; i += 8u) {
            float x[4];
            load4(part + i * step + c, have, x);
#pragma unroll
            for (int e = 0; e < 4; e++) v[e] += x[e] * factors[i];
        }
#pragma unroll
    for (int e = 0; e < 4; e++) sums[own][c + e] = v[e];
    wg_sync();
    if (threadIdx.x < g.dim) {
        float total = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; i++) total += sums[i][threadIdx.x];
        /* no weight at all: 0, or NaN if a value that is seen is not finite, as without splits */
        g.o.at(row, head)[threadIdx.x] = (T)(sum == 0.0f ? total * 0.0f : total / sum);
    }
    if (threadIdx.x == 0) g.lse[row * g.heads + head] = sum == 0.0f ? from_bits(0xFF800000u) : (top + __log2f(sum) - OFFSET<T>) * LN2;
}

/* The same where rows are many and parts few: eight rows a workgroup, 32 threads to each, a part after the other (us, a workgroup a row and this: 3020 tokens,
 * 4 heads of 120 20.6, 7.8; but 12 tokens of 2000 keys, 12 heads of 64 2.9, 3.7). */
constexpr uint32_t FEW_PARTS = 8, MANY_ROWS = 1024, JOINED = 8;
template <typename T> __global__ void __launch_bounds__(256) k_attend_join_few(Attend<T> g)
{
    const uint32_t head_of_keys = blockIdx.x / g.slots, c = threadIdx.x % 32u * 4u;
    uint32_t which, tile;
    find_slot<JOINED>(g.seqs.q_off, g.seqs.n, g.seqs.q_rows, g.group.n, blockIdx.x % g.slots, which, tile);
    if (tile == 0xFFFFFFFFu) return;
    const Seq s = seq_of(g.seqs, which);
    const uint32_t r = tile * JOINED + threadIdx.x / 32u;
    if (r >= s.m * g.group.n) return;
    const uint32_t query = g.group.div(r), head = head_of_keys * g.group.n + r - query * g.group.n;
    const uint64_t row = (uint64_t)s.q0 + query, step = part_at(g.seqs.q_rows, g.heads, g.dim, 1, 0, 0);
    const float *part = g.part + part_at(g.seqs.q_rows, g.heads, g.dim, 0, row, head);
    const int have = c < g.dim ? (int)min(g.dim - c, 4u) : 0;
    float top = LOWEST, sum = 0.0f, v[4] = {};
#pragma unroll 4
    for (uint32_t i = 0; i < g.splits; i++) top = fmaxf(top, part[i * step + g.dim]);
#pragma unroll 4
    for (uint32_t i = 0; i < g.splits; i++) {
        const float factor = __builtin_amdgcn_exp2f(part[i * step + g.dim] - top);
        float x[4] = {};
        load4(part + i * step + c, have, x);
        sum += part[i * step + g.dim + 1u] * factor;
#pragma unroll
        for (int e = 0; e < 4; e++) v[e] += x[e] * factor;
    }
    if (have) {
        const float f = sum == 0.0f ? 0.0f : 1.0f / sum;
#pragma unroll
        for (int e = 0; e < 4; e++) v[e] *= f;
        store4(g.o.at(row, head) + c, have, v);
    }
    if (c == 0) g.lse[row * g.heads + head] = sum == 0.0f ? from_bits(0xFF800000u) : (top + __log2f(sum) - OFFSET<T>) * LN2;
}

/* ---------------------------------------------------------------- launches */

/* FEW where a sequence's queries and their heads fill a tile of 32 rows at most, in the mean; not where heads of more than 64 elements in 16 bits have keys
 * for few workgroups, each of which then waits less where four wavefronts fetch (us, FEW and not: one token, 32 heads of 128 over 8, 300, 2000 and 8000 keys
 * 12.4, 11.1; 14.7, 11.6; 16.8, 15.5; two tokens of 8000 22.1, 23.3; four of 2000 15.8, 13.2, six 19.1, 21.1; sixteen of 4096 to 16384 140, 172; twelve
 * heads of 64, 300 keys 8.4, 9.9; twelve tokens of 2000 19.7, 26.1).  The keys are split over workgroups where there are too few of those to fill the chip,
 * four tiles of 64 to each at least (one token, 32 heads over 8, 4000 and 32000 keys: 15.5, 32.0; in eights 23, 32, in twos 15.2, 31.8; 777 keys of 12
 * heads of 64 in fours 11.0, in twos 9.8). */
constexpr uint64_t KEYS_FOR_FEW = 65536;
template <typename T, int D> struct Shape {
    static constexpr int W = 4, ROWS = W * 32, KEYS = D * sizeof(T) > 256 ? 32 : 64;
    static constexpr int FEW_W = 2, FEW_KEYS = FEW_W * 32;
};
struct Plan { bool few; uint32_t rows, slots, splits; };
Plan plan_of(int type, uint64_t q_rows, uint64_t k_rows, uint32_t seqs, uint32_t kv, uint32_t group, uint32_t dim)
{
    Plan p;
    p.few = q_rows * group <= (uint64_t)FEW_ROWS * seqs && (dim <= 64 || type == NSML_F32 || k_rows * kv > KEYS_FOR_FEW);
    p.rows = p.few ? FEW_ROWS : 128u;
    p.slots = (uint32_t)(q_rows * group / p.rows) + seqs + 1u;
    const uint32_t keys = p.few ? 64u : dim > 64 && type == NSML_F32 ? 32u : 64u;
    const uint64_t groups = (uint64_t)std::max<uint64_t>(p.few ? seqs : q_rows * group / p.rows, 1) * kv, tiles = (k_rows / seqs + keys - 1) / keys;
    p.splits = (uint32_t)std::min<uint64_t>({512 / groups, tiles / (p.few ? 4u : 2u), MOST_SPLITS});
    if (p.splits < 1u) p.splits = 1u;
    return p;
}

template <typename T, int D, Rows R> int launch(const Attend<T> &g, const Plan &p, hipStream_t st)
{
    typedef Shape<T, D> S;
    const uint32_t groups = p.slots * g.kv;
    if (p.few) k_attend<T, D, S::FEW_W, S::FEW_KEYS, true, R><<<groups * p.splits, S::FEW_W * 64, 0, st>>>(g);
    else k_attend<T, D, S::W, S::KEYS, false, R><<<groups * p.splits, S::W * 64, 0, st>>>(g);
    const int rc = launched();
    if (rc || p.splits == 1u) return rc;
    Attend<T> j = g;
    const bool some = p.splits <= FEW_PARTS && g.seqs.q_rows * g.heads >= MANY_ROWS;
    j.slots = g.seqs.q_rows * g.group.n / (some ? JOINED : 1u) + g.seqs.n + 1u;
    if (some) k_attend_join_few<T><<<j.slots * g.kv, 256, 0, st>>>(j);
    else k_attend_join<T><<<j.slots * g.kv, 256, 0, st>>>(j);
    return launched();
}

}  // namespace

extern "C" {

uint64_t nsml_attention_work(int type, uint64_t q_rows, uint64_t k_rows, uint32_t seqs, uint32_t heads, uint32_t kv_heads, uint32_t dim)
{
    if (bad_type(type) || bad_shape(q_rows, k_rows, seqs, heads, kv_heads, dim) || q_rows == 0) return 0;
    const Plan p = plan_of(type, q_rows, k_rows, seqs, kv_heads, heads / kv_heads, dim);
    return p.splits > 1u ? (uint64_t)p.splits * q_rows * heads * (dim + 2u) * 4u : 0u;
}

int nsml_attention(const nsml_heads *q, const nsml_heads *k, const nsml_heads *v, int type, const nsml_seqs *seqs, uint32_t heads,
                   uint32_t kv_heads, uint32_t dim, int32_t left, int32_t right, float scale, const nsml_heads *o, float *lse, int rest,
                   void *work, uint64_t work_bytes, void *stream)
{
    if (!seqs || bad_type(type) || !(scale > 0.0f) || !(scale <= 2.0e38f) || bad_seqs(seqs)) return NSML_EINVAL;
    const uint64_t m = seqs->q_rows, n = seqs->k_rows;
    if (const int rc = bad_shape(m, n, seqs->n, heads, kv_heads, dim)) return rc;
    if ((m && (bad_heads(q, type) || bad_results(o, type, m, heads, dim) || bad_f32(lse))) || (n && (bad_heads(k, type) || bad_heads(v, type)))) return NSML_EINVAL;
    const uint64_t need = nsml_attention_work(type, m, n, seqs->n, heads, kv_heads, dim);
    if (need && (!work || !at_multiple(work, 16) || work_bytes < need)) return NSML_EINVAL;
    if (m == 0) return NSML_OK;
    const Plan p = plan_of(type, m, n, seqs->n, kv_heads, heads / kv_heads, dim);
    if (std::max<uint64_t>((uint64_t)p.slots * p.splits, p.splits > 1u ? m * (heads / kv_heads) + seqs->n + 1u : 0u) * kv_heads >= 1u << 24) return NSML_ECAP;
    const HeadArea out = head_area(o, type, m, heads, dim), sums = one_area(area(lse, 1, 0, m * heads * 4u)), parts = one_area(area(need ? work : nullptr, 1, 0, need));
    if (clash({out, sums, parts}, {head_area(q, type, m, heads, dim), head_area(k, type, n, kv_heads, dim), head_area(v, type, n, kv_heads, dim),
                                   int_area(seqs->q_off, seqs->n + 1ull), int_area(seqs->k_off, seqs->n + 1ull), int_area(seqs->q_len, seqs->n), int_area(seqs->k_len, seqs->n)}))
        return NSML_EINVAL;
    const Rows like = rows_of((n == 0 || (fast_heads(k, type) && fast_heads(v, type))), type, dim);
    hipStream_t st = static_cast<hipStream_t>(stream);
    const auto go = [&](auto t) {
        using T = decltype(t);
        const Attend<T> g{heads_of<const T>(q), heads_of<const T>(k), heads_of<const T>(v), heads_of<T>(o), lse,
                          static_cast<float *>(work), seqs_of(seqs), group_of(heads / kv_heads), Reach{left, right}, heads, kv_heads, dim, p.slots, p.splits, scale, rest};
        if (dim <= 64) return like == WHOLE ? launch<T, 64, WHOLE>(g, p, st) : like == CHUNKS ? launch<T, 64, CHUNKS>(g, p, st) : launch<T, 64, ANY>(g, p, st);
        return like == WHOLE ? launch<T, 128, WHOLE>(g, p, st) : like == CHUNKS ? launch<T, 128, CHUNKS>(g, p, st) : launch<T, 128, ANY>(g, p, st);
    };
    if (type == NSML_F32) return go(float{});
    if (type == NSML_BF16) return go(bf16{});
    return go(f16{});
}

}  // extern "C"
