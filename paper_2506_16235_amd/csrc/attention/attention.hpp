/*
 * What the attention kernels share: sequences, tiles in LDS, the matrix instructions' operands, what a query sees.
 * Included by forward.hip and backward.hip; not a public header.
 *
 * Every product is made so that what varies over the registers of a result is summed over by the next one.  A 32 x 32 result has one
 * column per lane of half a wavefront and 16 of its rows in registers: rows r % 4 + 8 (r / 4) + 4 (lane / 32).  Scores with keys as rows and
 * queries as columns leave a query's softmax in one lane and its other half; registers 8 s to 8 s + 7 of them are, in this order of rows,
 * the operand of the product over 16 keys.  The other operand, which has its rows in memory and is wanted by columns, is read from LDS by
 * the transposing read in the same order of rows.
 *
 * The query heads that share a head of keys are rows of one matrix: row r of a sequence is query r / group of head r % group, so that keys
 * are read once for all of them and a single token fills a tile as far as there are heads.
 */
#ifndef NSML_ATTENTION_HPP
#define NSML_ATTENTION_HPP

#include "../layer8/layer8.hpp"

#include <algorithm>
#include <type_traits>

/* Of a kernel's parts that are named: a call would keep its registers in memory. */
#define INLINE __attribute__((always_inline))

namespace {

typedef float v16f __attribute__((ext_vector_type(16)));
typedef int v4i __attribute__((ext_vector_type(4)));
typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef float v8f __attribute__((ext_vector_type(8)));
typedef short v4s __attribute__((ext_vector_type(4)));

template <typename T> struct Operand;
template <> struct Operand<bf16> { typedef v8bf V; };
template <> struct Operand<f16> { typedef v8h V; };
template <> struct Operand<float> { typedef v8f V; };
/* What a lane gives a product over 16: eight neighbours of a row (or of a column). */
template <typename T> using Frag = typename Operand<T>::V;

/* c += a b over 16.  binary32: eight products over 2, an element of each lane half at a time. */
__device__ __forceinline__ void mma(const v8bf &a, const v8bf &b, v16f &c) { c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ void mma(const v8h &a, const v8h &b, v16f &c) { c = __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ void mma(const v8f &a, const v8f &b, v16f &c)
{
#pragma unroll
    for (int e = 0; e < 8; e++) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[e], b[e], c, 0, 0, 0);
}
/* The row of a 32 x 32 result that register r of a lane holds; its column is lane % 32. */
__device__ __forceinline__ uint32_t acc_row(int r, uint32_t lane) { return (uint32_t)(r % 4 + r / 4 * 8) + lane / 32u * 4u; }

/* Sum and maximum of what the two lanes of a column hold. */
__device__ __forceinline__ float half_max(float v)
{
    const auto s = __builtin_amdgcn_permlane32_swap(to_bits(v), to_bits(v), false, false);
    return fmaxf(from_bits(s[0]), from_bits(s[1]));
}
__device__ __forceinline__ float half_sum(float v)
{
    const auto s = __builtin_amdgcn_permlane32_swap(to_bits(v), to_bits(v), false, false);
    return from_bits(s[0]) + from_bits(s[1]);
}

/* Eight registers of a result as an operand, each rounded once. */
template <typename T> __device__ __forceinline__ Frag<T> rounded(const float *p)
{
    Frag<T> f;
#pragma unroll
    for (int i = 0; i < 8; i++) f[i] = (T)p[i];
    return f;
}

/* ---------------------------------------------------------------- tiles in LDS
 *
 * Rows of D elements in chunks of 16 bytes, which lie within 256 bytes in an order that differs from row to row such that the same chunk of 16
 * rows, and four neighbouring chunks of four rows (what the transposing read takes), meet no bank twice. */
template <typename T, int D> struct TileOf {
    static constexpr int ROW = D * (int)sizeof(T), CHUNKS = ROW / 16, E = 16 / (int)sizeof(T);
    static_assert(ROW == 128 || ROW == 256 || ROW == 512, "");
    static __device__ __forceinline__ uint32_t turn(uint32_t row) { return row % 4u * 4u + row / 4u % 4u; }
    static __device__ __forceinline__ uint32_t place(uint32_t row, uint32_t chunk)
    {
        if constexpr (ROW == 128) return row / 2u * 256u + (((row % 2u * 8u + chunk) ^ (row / 2u % 2u * 4u + row / 4u % 4u)) * 16u);
        else return row * ROW + ((chunk ^ turn(row)) * 16u);
    }
    /* Which row and chunk lie at the slot-th 16 bytes. */
    static __device__ __forceinline__ void at_slot(uint32_t slot, uint32_t &row, uint32_t &chunk)
    {
        if constexpr (ROW == 128) {
            const uint32_t p = slot / 16u, x = slot % 16u ^ (p % 2u * 4u + p / 2u % 4u);
            row = p * 2u + x / 8u, chunk = x % 8u;
        } else {
            row = slot / CHUNKS, chunk = slot % CHUNKS ^ turn(row);
        }
    }
};

/* Where a lane's operands lie in a tile: what is added for other rows (multiples of 32, of 16 for columns) and other tiles is the same for all lanes, and
 * part of the instruction where it is known at compile time. */
typedef const __attribute__((address_space(3))) uint8_t *Shared;
__device__ __forceinline__ Shared shared(const uint8_t *p) { return (Shared)p; }

/* Elements 16 i + 8 (lane / 32) and the seven after them of row lane % 32 of a block of 32 rows. */
template <typename T, int D> struct RowLane {
    typedef TileOf<T, D> L;
    static constexpr int N = D / 16, H = sizeof(T) / 2;      /* chunks to an operand */
    uint32_t at[N * H];
    __device__ __forceinline__ explicit RowLane(uint32_t lane)
    {
#pragma unroll
        for (int i = 0; i < N * H; i++) at[i] = L::place(lane % 32u, i / H * (2u * H) + lane / 32u * H + i % H);
    }
    __device__ __forceinline__ Frag<T> operator()(Shared tile, uint32_t first_row, int i) const
    {
        struct { v4i v[H]; } x;
#pragma unroll
        for (int h = 0; h < H; h++) x.v[h] = *reinterpret_cast<const __attribute__((address_space(3))) v4i *>(tile + at[i * H + h] + first_row * L::ROW);
        return __builtin_bit_cast(Frag<T>, x);
    }
};
/* Column 32 b + lane % 32, rows first_row + 4 (lane / 32) + {0, 1, 2, 3, 8, 9, 10, 11}; first_row a multiple of 16. */
template <typename T, int D> struct ColLane {
    typedef TileOf<T, D> L;
    static constexpr int N = sizeof(T) == 2 ? 2 : 8;         /* reads to an operand */
    uint32_t at[D / 32][N];
    __device__ __forceinline__ explicit ColLane(uint32_t lane)
    {
#pragma unroll
        for (int b = 0; b < D / 32; b++)
#pragma unroll
            for (int j = 0; j < N; j++) {
                /* Sixteen lanes read four rows of 16 neighbours, eight bytes each, and get a column each. */
                if constexpr (sizeof(T) == 2)
                    at[b][j] = L::place(j * 8u + lane / 32u * 4u + lane % 16u / 4u, b * 4u + lane / 16u % 2u * 2u + lane % 4u / 2u) + lane % 2u * 8u;
                else
                    at[b][j] = L::place(j / 4 * 8u + lane / 32u * 4u + j % 4u, b * 8u + lane % 32u / 4u) + lane % 4u * 4u;
            }
    }
    __device__ __forceinline__ Frag<T> operator()(Shared tile, uint32_t first_row, int b) const
    {
        if constexpr (sizeof(T) == 2) {
            struct { v4s v[2]; } two;
#pragma unroll
            for (int j = 0; j < 2; j++) two.v[j] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s *)(tile + at[b][j] + first_row * L::ROW));
            return __builtin_bit_cast(Frag<T>, two);
        } else {
            Frag<T> f;
#pragma unroll
            for (int e = 0; e < 8; e++) f[e] = *reinterpret_cast<const __attribute__((address_space(3))) float *>(tile + at[b][e] + first_row * L::ROW);
            return f;
        }
    }
};

__device__ __forceinline__ uint32_t uniform(uint32_t v) { return __builtin_amdgcn_readfirstlane(v); }

/* ---------------------------------------------------------------- heads in memory */

template <typename T> struct Heads {
    T *p;
    uint64_t ld, hs;             /* elements from row to row and from head to head */
    __device__ __forceinline__ T *at(uint64_t row, uint32_t head) const { return p + row * ld + head * hs; }
};

/* What the rows of a call's heads are like.  WHOLE: as many elements as a tile has, at multiples of 16 bytes.  CHUNKS: fewer, but whole chunks of 16
 * bytes, at multiples of them.  ANY: neither. */
enum Rows { ANY, CHUNKS, WHOLE };
/* Whether products over the elements from c on are needed: of heads that are shorter than a tile's rows, the last quarter of them is left out where it
 * is all beyond them; in binary32, whose products take eight times as long, every sixteen. */
template <typename T, int D, Rows R> __device__ __forceinline__ bool used(uint32_t c, uint32_t dim)
{
    if (R == WHOLE) return true;
    return sizeof(T) == 4 ? c < dim : c < D * 3 / 4 || dim > D * 3 / 4;
}
/* Read where a chunk lies beyond a row. */
__device__ const uint32_t ZEROS[4] = {};

/* Lanes take no branches of their own around what is kept for long: this compiler has been seen to copy a register into an accumulation register while only
 * some lanes were active (the copy went before the instruction that brings them back), and what the others held was lost. */

/* E neighbours from element c of a row, those from dim on zero. */
template <typename T, Rows R, int E> __device__ __forceinline__ void load_some(const T *row, uint32_t c, uint32_t dim, T (&x)[E])
{
    static_assert(E * sizeof(T) % 16 == 0, "");
    if (R == WHOLE || dim % E == 0) {
        const bool in = R == WHOLE || c < dim;
        const auto b = *reinterpret_cast<const Bytes<E * sizeof(T) / 4> *>(row + (in ? c : 0u));
        __builtin_memcpy(x, &b, sizeof x);
        if (R != WHOLE)
#pragma unroll
            for (int i = 0; i < E; i++) x[i] = in ? x[i] : (T)0.0f;
    } else {
#pragma unroll
        for (uint32_t i = 0; i < (uint32_t)E; i++) {
            const T v = row[min(c + i, dim - 1u)];
            x[i] = c + i < dim ? v : (T)0.0f;
        }
    }
}
/* Eight of them as an operand straight from memory. */
template <typename T, Rows R> __device__ __forceinline__ Frag<T> frag_at(const T *row, uint32_t c, uint32_t dim)
{
    T x[8];
    load_some<T, R>(row, c, dim, x);
    Frag<T> f;
#pragma unroll
    for (int i = 0; i < 8; i++) f[i] = x[i];
    return f;
}
/* Four neighbours of a row's result. */
template <Rows R, typename T> __device__ __forceinline__ void put4(T *row, uint32_t c, uint32_t dim, const float (&v)[4])
{
    if (R == WHOLE) store4(row + c, 4, v);
    else if (c < dim) store4(row + c, (int)min(dim - c, 4u), v);
}

/* Division by the number of query heads to a head of keys, for numerators below 2^31: high half of a product (host: group_of). */
struct Group {
    uint32_t n, magic, shift;
    __device__ __forceinline__ uint32_t div(uint32_t x) const { return n == 1u ? x : __umulhi(x, magic) >> shift; }
};

/* Rows of a tile on their way to LDS, a thread's chunks THREADS apart, which are whole rows: the same chunk of each.  WHOLE and CHUNKS: straight there (a
 * wavefront's chunks are side by side, as that needs), zeros from memory where a row has no such chunk; ANY: through registers. */
template <typename T, int D, int ROWS, int THREADS, Rows R> struct Loader {
    typedef TileOf<T, D> L;
    typedef const __attribute__((address_space(1))) uint8_t *Global;
    static constexpr int N = ROWS * L::CHUNKS / THREADS, STEP = THREADS / L::CHUNKS, E = L::E;
    static_assert(N * THREADS == ROWS * L::CHUNKS, "");
    uint32_t row, chunk0;
    __device__ __forceinline__ Loader() { L::at_slot(threadIdx.x, row, chunk0); }
    /* The order within 256 bytes comes again every 16 rows. */
    __device__ __forceinline__ uint32_t chunk(int i) const
    {
        if (STEP % 16 == 0) return chunk0;
        uint32_t r, c;
        L::at_slot(i * THREADS + threadIdx.x, r, c);
        return c;
    }
    __device__ __forceinline__ void straight(uint8_t *tile, int i, Global from) const
    {
        uint8_t *to = tile + (i * THREADS + uniform(threadIdx.x)) * 16u;         /* the first lane's place; the others' follow by themselves */
        __builtin_amdgcn_global_load_lds(from, (__attribute__((address_space(3))) void *)to, 16, 0, 0);
    }
    /* The same for an address that is alike for all threads and what a thread adds to it: kept apart, as sums of them would fill the registers. */
    __device__ __forceinline__ void straight(uint8_t *tile, int i, const uint8_t *base, uint32_t own) const
    {
        const uint64_t at = reinterpret_cast<uint64_t>(base);
        uint32_t lo = uniform((uint32_t)at), hi = uniform((uint32_t)(at >> 32));
        asm("" : "+s"(lo), "+s"(hi));
        asm("" : "+v"(own));
        straight(tile, i, (Global)((uint64_t)hi << 32 | lo) + own);
    }
    __device__ __forceinline__ void chunk_of(uint8_t *tile, int i, const T *from, uint32_t dim) const
    {
        if constexpr (R == WHOLE) {
            straight(tile, i, (Global)(from + chunk(i) * E));
        } else if constexpr (R == CHUNKS) {
            straight(tile, i, chunk(i) * E < dim ? (Global)(from + chunk(i) * E) : (Global)ZEROS);
        } else {
            T x[E];
            load_some<T, ANY>(from, chunk(i) * E, dim, x);
            *reinterpret_cast<v4i *>(tile + (i * THREADS + threadIdx.x) * 16u) = __builtin_bit_cast(v4i, x);
        }
    }
    /* Rows of keys or values from row `first` of a sequence's n on (p: its first one); rows from n on are its last one again. */
    __device__ __forceinline__ void keys(uint8_t *tile, const T *p, uint64_t ld, uint32_t first, uint32_t n, uint32_t dim) const
    {
        if (R == WHOLE && first + ROWS <= n) {
            const uint8_t *base = reinterpret_cast<const uint8_t *>(p + first * ld);
#pragma unroll
            for (int i = 0; i < N; i++) {
                const uint32_t off = (row * (uint32_t)ld + chunk(i) * E) * (uint32_t)sizeof(T);     /* fits (fast_heads) */
                straight(tile, i, base + (uint64_t)(i * STEP) * ld * sizeof(T), off);
            }
        } else {
            uint32_t r = row;
            asm("" : "+v"(r));                   /* made here, not kept in registers from tile to tile */
#pragma unroll
            for (int i = 0; i < N; i++) chunk_of(tile, i, p + min(first + i * STEP + r, n - 1u) * ld, dim);
        }
    }
    /* Rows of queries (or of their gradients), as query and head in the group; p: the first query's first head of the group. */
    __device__ __forceinline__ void queries(uint8_t *tile, const T *p, uint64_t ld, uint64_t hs, const Group &group, uint32_t first, uint32_t rows, uint32_t dim) const
    {
        if (R == WHOLE && STEP % group.n == 0 && first + ROWS <= rows) {
            /* a thread's rows are the same head of queries that lie the same way apart for all threads */
            const uint32_t at = group.div(row);
            const T *mine = p + at * ld + (row - at * group.n) * hs;
#pragma unroll
            for (int i = 0; i < N; i++) straight(tile, i, (Global)(mine + chunk(i) * E + group.div(first + i * STEP) * ld));
        } else {
            uint32_t own = row;
            asm("" : "+v"(own));
#pragma unroll
            for (int i = 0; i < N; i++) {
                const uint32_t r = min(first + i * STEP + own, rows - 1u), at = group.div(r);
                chunk_of(tile, i, p + at * ld + (r - at * group.n) * hs, dim);
            }
        }
    }
};

/* Until the tile that this wavefront asked for is there and its accesses to LDS are done, then until all wavefronts are here. */
__device__ __forceinline__ void tile_sync()
{
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0x0070);              /* vmcnt(0) lgkmcnt(0) */
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

/* ---------------------------------------------------------------- sequences */

struct Seqs {
    const int32_t *q_off, *k_off, *q_len, *k_len;
    uint32_t n;
    uint32_t q_rows, k_rows;
};
/* One sequence: where its queries and keys begin, how many there are, how many rows its room has. */
struct Seq {
    uint32_t q0, m, q_room, k0, n, k_room;
};
__device__ __forceinline__ uint32_t held(int32_t v, uint32_t lo, uint32_t hi) { return v < 0 || (uint32_t)v < lo ? lo : min((uint32_t)v, hi); }
/* Offsets and lengths are read on the GPU, so whatever they hold is held to the rows that there are.  i == s.n: the rows behind the last one. */
__device__ __forceinline__ Seq seq_of(const Seqs &s, uint32_t i)
{
    Seq q;
    q.q0 = s.q_off ? held(s.q_off[i], 0, s.q_rows) : i ? s.q_rows : 0u;
    q.k0 = s.k_off ? held(s.k_off[i], 0, s.k_rows) : i ? s.k_rows : 0u;
    if (i >= s.n) {
        q.q_room = s.q_rows - q.q0, q.k_room = s.k_rows - q.k0;
        q.m = q.n = 0;
    } else {
        q.q_room = (s.q_off ? held(s.q_off[i + 1], q.q0, s.q_rows) : s.q_rows) - q.q0;
        q.k_room = (s.k_off ? held(s.k_off[i + 1], q.k0, s.k_rows) : s.k_rows) - q.k0;
        q.m = s.q_len ? held(s.q_len[i], 0, q.q_room) : q.q_room;
        q.n = s.k_len ? held(s.k_len[i], 0, q.k_room) : q.k_room;
    }
    q.q0 = uniform(q.q0), q.m = uniform(q.m), q.q_room = uniform(q.q_room);
    q.k0 = uniform(q.k0), q.n = uniform(q.n), q.k_room = uniform(q.k_room);
    return q;
}
/* Which sequence a slot belongs to, and the tile of it: sequence i has the slots from off[i] * per / SIZE + i on, which are enough for its rows
 * (per of them to a row of off) and one more at most.  64 sequences are looked at a time. */
template <uint32_t SIZE> __device__ __forceinline__ void find_slot(const int32_t *off, uint32_t seqs, uint32_t rows, uint32_t per, uint32_t slot, uint32_t &seq, uint32_t &tile)
{
    const uint32_t lane = threadIdx.x % 64u;
    uint32_t lo = 0, count = seqs + 1u;              /* with the rows behind the last one */
    const auto first = [&](uint32_t i) -> uint64_t {
        const uint32_t at = off ? held(off[i], 0, rows) : i ? rows : 0u;
        return (uint64_t)at * per / SIZE + i;
    };
    while (count > 1u) {
        const uint32_t step = (count + 63u) / 64u, i = lane * step;
        const uint64_t before = __ballot(i < count && first(lo + i) <= slot);
        const uint32_t c = before ? __popcll(before) - 1u : 0u;
        lo += c * step;
        count = min(step, count - c * step);
    }
    seq = uniform(lo);
    const uint64_t f = first(seq);
    tile = uniform(slot < f ? 0xFFFFFFFFu : (uint32_t)(slot - f));
}

__device__ __forceinline__ uint32_t wave_sum(uint32_t v)
{
#define FROM(ctrl, rows) v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, ctrl, rows, 0xF, false)
    FROM(0x111, 0xF);                                /* from one, two, four and eight lanes before, in rows of 16 */
    FROM(0x112, 0xF);
    FROM(0x114, 0xF);
    FROM(0x118, 0xF);
    FROM(0x142, 0xA);                                /* a row's last to the next row, the second row's to the last two */
    FROM(0x143, 0xC);
#undef FROM
    return (uint32_t)__builtin_amdgcn_readlane((int)v, 63);
}
/* The tile that stands idx-th in the order of work.  Long sequences' tiles differ in what they cost, the last ones most where keys ahead are hidden, so the
 * order is by a tile's number in its sequence, over all sequences at once: from the first up (UP, for keys) or from the last down (8192 tokens in seven
 * documents, heads of 128: gradient of keys 864 -> 740 us).  Up to 63 sequences; of more, one after the other. */
template <uint32_t SIZE, bool UP>
__device__ __forceinline__ void find_tile(const int32_t *off, uint32_t seqs, uint32_t rows, uint32_t per, uint32_t idx, uint32_t slots, uint32_t &seq, uint32_t &tile)
{
    if (seqs > 63u) {
        find_slot<SIZE>(off, seqs, rows, per, UP ? idx : slots - 1u - idx, seq, tile);
        return;
    }
    const uint32_t lane = threadIdx.x % 64u;
    uint32_t begin = rows, end = rows;               /* the last one: the rows behind the sequences */
    if (lane <= seqs) begin = off ? held(off[lane], 0, rows) : lane ? rows : 0u;
    if (lane < seqs) end = off ? held(off[lane + 1], begin, rows) : rows;
    const uint32_t tiles = ((end - begin) * per + SIZE - 1u) / SIZE, total = wave_sum(tiles);
    seq = 0, tile = 0xFFFFFFFFu;
    if (idx >= total) return;
    const uint32_t s = UP ? idx : total - 1u - idx;
    const uint64_t some = __ballot(tiles != 0);
    uint32_t lo = 0, hi = s + 1u, before = 0;        /* the most tiles of each sequence that are s or fewer together */
    if (__popcll(some) == 1u) {
        lo = before = s;
    } else {
        while (hi - lo > 1u) {
            const uint32_t mid = lo + (hi - lo) / 2u, sum = wave_sum(min(tiles, mid));
            if (sum <= s) lo = mid, before = sum;
            else hi = mid;
        }
    }
    const uint64_t here = __ballot(tiles > lo);
    const uint32_t rank = __popcll(here & ((1ull << lane) - 1ull));
    const uint64_t mine = __ballot(tiles > lo && rank == s - before);
    if (mine == 0) return;                           /* offsets that descend */
    seq = uniform((uint32_t)__builtin_ctzll(mine)), tile = uniform(lo);
}

/* Which tile in the order of work, head of keys and split a workgroup takes: heads by turns, so that what workgroups of one die (every eighth) take is of
 * few heads, whose keys they read together, and every die has long tiles and short ones alike (us with a run of tiles to each die: gradient of 8192 tokens,
 * 16 heads over 2, 2244). */
struct Job { uint32_t slot, head, split; };
__device__ __forceinline__ Job job_of(uint32_t id, uint32_t heads, uint32_t splits)
{
    const uint32_t in = id / heads, slot = in / splits;
    return {slot, id - in * heads, in - slot * splits};
}

/* What a query sees: keys from lo on, `count` of them. */
struct Reach {
    int32_t left, right;         /* how far back and ahead; below 0: all */
};
struct Seen { uint32_t lo, count; };
__device__ __forceinline__ int64_t within(int64_t v, int64_t most) { return v < 0 ? 0 : v < most ? v : most; }
__device__ __forceinline__ Seen seen_by(const Reach &r, const Seq &s, uint32_t query)
{
    const int64_t at = (int64_t)query + s.n - s.m;
    const int64_t hi = r.right < 0 ? (int64_t)s.n : within(at + r.right + 1, s.n), lo = r.left < 0 ? 0 : within(at - r.left, s.n);
    return {(uint32_t)lo, hi > lo ? (uint32_t)(hi - lo) : 0u};
}

/* ---------------------------------------------------------------- values that are not finite where nobody sees them
 *
 * A product over rows takes a row that somebody does not see with weight 0, and 0 times an infinity is NaN.  So in tiles of which not everybody sees
 * everything such values become zeros in LDS, for all wavefronts, and their rows are marked: whoever sees one of those, in a wavefront that sees all of the tile
 * or not, has its result made NaN at the end. */
template <typename T, int D, int ROWS, int THREADS> struct Cleaner {
    typedef TileOf<T, D> L;
    static constexpr int BYTES = ROWS * 4 + 16;
    float *mark;                 /* of each row: 0, or NaN; then whether any is; then what nobody reads */
    bool dirty;
    __device__ __forceinline__ Cleaner(uint8_t *lds) : mark(reinterpret_cast<float *>(lds)), dirty(true) {}
    /* TILES tiles of ROWS rows, one after the other; all of the workgroup comes here.  -> whether a row is marked. */
    template <int TILES> __device__ __forceinline__ bool clean(uint8_t *tile)
    {
        static_assert(THREADS > ROWS && TILES * ROWS * L::CHUNKS % THREADS == 0, "");
        if (dirty) {
            mark[min(threadIdx.x, (uint32_t)ROWS)] = 0.0f;
            wg_sync();
        }
        constexpr bool ONE = sizeof(T) == 4;
        constexpr uint32_t X = ONE ? 0x7F800000u : std::is_same_v<T, bf16> ? 0x7F80u : 0x7C00u;
#pragma unroll 1
        for (uint32_t i = 0; i < (uint32_t)(TILES * ROWS * L::CHUNKS / THREADS); i++) {
            const uint32_t slot = i * THREADS + threadIdx.x;
            v4i *at = reinterpret_cast<v4i *>(tile + slot * 16u);
            v4i v = *at;
            uint32_t any = 0;
#pragma unroll
            for (int e = 0; e < 4; e++) {
                const uint32_t lo = ((uint32_t)v[e] & X) == X ? (ONE ? 0xFFFFFFFFu : 0xFFFFu) : 0u, hi = !ONE && ((uint32_t)v[e] >> 16 & X) == X ? 0xFFFF0000u : 0u;
                any |= lo | hi;
                v[e] &= ~(lo | hi);
            }
            if (__ballot(any != 0)) {
                uint32_t row, chunk;
                L::at_slot(slot % (uint32_t)(ROWS * L::CHUNKS), row, chunk);
                *at = v;
                mark[any ? row : ROWS + 1u] = from_bits(0x7FC00000u);
                mark[ROWS] = 1.0f;
            }
        }
        wg_sync();
        dirty = uniform(to_bits(mark[ROWS])) != 0;
        return dirty;
    }
    /* The lanes that see a marked one of the 32 rows from `first` on, a bit each: a lane sees those from lo up to hi, which may lie outside.  By itself, apart
     * from the products, and in a scalar register: marks among the weights took 27 registers of a prompt's loop. */
    __device__ __forceinline__ uint64_t seen(uint32_t first, int32_t lo, int32_t hi) const
    {
        const uint32_t marked = (uint32_t)__ballot(mark[first + threadIdx.x % 32u] != 0.0f);
        const uint32_t below = (1ull << max(0, min(hi, 32))) - 1ull, before = (1ull << max(0, min(lo, 32))) - 1ull;
        return __ballot((marked & below & ~before) != 0);
    }
    /* What such a lane's result becomes by addition. */
    static __device__ __forceinline__ float none(uint64_t lanes) { return lanes >> threadIdx.x % 64u & 1u ? from_bits(0x7FC00000u) : 0.0f; }
};

/* ---------------------------------------------------------------- softmax */

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f, LOWEST = -3.0e38f;
/* Weights are made as powers of two 2^OFFSET times too large where the type has few exponents: float16 holds what lies 2^-14 below 1 with fewer bits. */
template <typename T> constexpr float OFFSET = 0.0f;
template <> constexpr float OFFSET<f16> = 7.0f;

/* ---------------------------------------------------------------- host */

/* A matrix of heads that is read may have any strides; one that is written holds each of its elements once. */
inline bool bad_heads(const nsml_heads *h, int type) { return !h || !h->p || !at_multiple(h->p, type_bytes(type)); }
inline bool bad_results(const nsml_heads *h, int type, uint64_t rows, uint32_t heads, uint32_t dim)
{
    if (bad_heads(h, type) || (rows > 1 && h->ld < dim) || (heads > 1 && h->hs < dim)) return true;
    if (rows < 2 || heads < 2) return false;
    /* all heads of a row before the next row, or all rows of a head before the next head */
    return (h->ld - dim) / (heads - 1u) < h->hs && (h->hs - dim) / (rows - 1u) < h->ld;
}
inline bool bad_offsets(const int32_t *p) { return p && !at_multiple(p, 4); }
inline bool bad_seqs(const nsml_seqs *s)
{
    return s->n == 0 || (s->n > 1 && (!s->q_off || !s->k_off)) || bad_offsets(s->q_off) || bad_offsets(s->k_off) || bad_offsets(s->q_len) || bad_offsets(s->k_len);
}
inline int bad_shape(uint64_t q_rows, uint64_t k_rows, uint32_t seqs, uint32_t heads, uint32_t kv, uint32_t dim)
{
    if (heads == 0 || kv == 0 || heads % kv || dim == 0 || seqs == 0) return NSML_EINVAL;
    if (dim > NSML_HEAD_MAX_DIM || heads > NSML_MAX_HEADS || seqs > NSML_MAX_SEQS || k_rows > NSML_MAX_TOKENS || q_rows > NSML_MAX_TOKENS / (heads / kv)) return NSML_ECAP;
    return NSML_OK;
}
inline Seqs seqs_of(const nsml_seqs *s) { return {s->q_off, s->k_off, s->q_len, s->k_len, s->n, (uint32_t)s->q_rows, (uint32_t)s->k_rows}; }

/* The bytes of a matrix of heads: one area, or one for each head where rows and heads go through each other. */
struct HeadArea { Area first; uint32_t count; uint64_t step; };
inline HeadArea one_area(const Area &a) { return {a, 1, 0}; }
inline HeadArea head_area(const nsml_heads *h, int type, uint64_t rows, uint32_t heads, uint32_t dim)
{
    if (!h || rows == 0) return one_area(area(nullptr, 0, 0, 0));
    const uint64_t b = type_bytes(type), ld = h->ld * b, hs = h->hs * b, width = dim * b;
    if (ld == 0) rows = 1;       /* one row, or one head, for all */
    if (hs == 0) heads = 1;
    if (heads == 1 || hs == width) return one_area(area(h->p, rows, ld, heads * width));
    if (rows == 1 || ld == width) return one_area(area(h->p, heads, hs, rows * width));
    if (ld == heads * hs) return one_area(area(h->p, rows * heads, hs, width));
    return {area(h->p, rows, ld, width), heads, hs};
}
inline HeadArea int_area(const int32_t *p, uint64_t n) { return one_area(area(p, 1, 0, n * 4u)); }
inline bool meet(const HeadArea &a, const HeadArea &b)
{
    if (a.first.rows == 0 || b.first.rows == 0) return false;
    const auto end = [](const HeadArea &x) { return x.first.at + (x.count - 1u) * x.step + (x.first.rows - 1u) * x.first.pitch + x.first.width; };
    if (end(a) <= b.first.at || end(b) <= a.first.at) return false;
    for (uint32_t i = 0; i < a.count; i++)
        for (uint32_t j = 0; j < b.count; j++) {
            Area x = a.first, y = b.first;
            x.at += i * a.step, y.at += j * b.step;
            if (meet(x, y)) return true;
        }
    return false;
}
/* What is read, but nothing where it is the very matrix that is written. */
inline HeadArea apart(HeadArea read, const HeadArea &written)
{
    if (read.count == written.count && read.step == written.step) read.first = apart(read.first, written.first);
    return read;
}
inline bool clash(std::initializer_list<HeadArea> written, std::initializer_list<HeadArea> read)
{
    for (const HeadArea *w = written.begin(); w != written.end(); w++) {
        for (const HeadArea *o = written.begin(); o != w; o++)
            if (meet(*w, *o)) return true;
        for (const HeadArea &r : read)
            if (meet(*w, r)) return true;
    }
    return false;
}
template <typename T> Heads<T> heads_of(const nsml_heads *h) { return h ? Heads<T>{static_cast<T *>(h->p), h->ld, h->hs} : Heads<T>{nullptr, 0, 0}; }
inline bool fast_heads(const nsml_heads *h, int type)
{
    /* at multiples of 16 bytes, and the rows of a tile within 32 bits of its first */
    return at_multiple(h->p, 16) && h->ld * type_bytes(type) % 16 == 0 && h->hs * type_bytes(type) % 16 == 0 && h->ld <= 1u << 22;
}
/* What a call's rows are like, `fast` being fast_heads of what goes to LDS. */
inline Rows rows_of(bool fast, int type, uint32_t dim)
{
    return !fast || dim * type_bytes(type) % 16 != 0 ? ANY : dim == 64 || dim == 128 ? WHOLE : CHUNKS;
}
inline Group group_of(uint32_t n)
{
    uint32_t s = 0;
    while ((1ull << s) < n) s++;
    /* floor(x / n) = floor(x m / 2^(32 + s - 1)) for x below 2^31, m = ceil(2^(31 + s) / n) */
    const uint64_t m = n > 1 ? ((1ull << (31 + s)) + n - 1) / n : 0;
    return {n, (uint32_t)m, s ? s - 1 : 0};
}

}  // namespace

#endif
