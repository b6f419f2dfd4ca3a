// A cache in pages (the layout is in include/ra.h): attention over all tokens (ra_full_attention_paged), over the retrieved set Omega and
// the static set W of Sec. 3.3 with their combination by Eq. 4-5 (ra_attend_paged), and rows side by side again (ra_gather_paged).
// What puts tokens into pages is with the other calls that append (kv4.hip).
//
// Rows are cut into parts; a workgroup turns one part into a record (128 weighted sums, the maximum of <q, k>, the sum of weights), and a
// head's records are combined by a second kernel. Weights are powers of two, p = 2^(c (<q, k> - m)) with c = log2(e) / sqrt(d) and m the running
// maximum of <q, k>: the difference first, here and where records and sets are combined, so that its rounding goes by the difference and equal
// logits have equal weights however large they are and wherever their rows were. (A maximum may lag behind its rows' by PG_LAG. With
// records' maxima multiplied by c first, means over 131072 rows whose products are 2^24 were off by up to 1.8 %.)
#include "common.h"
#include "records.h"

#define PG_WAVES 8                  // wavefronts of a workgroup over all tokens
#define PG_GATHER_THREADS 256
#define PG_HEADS 16                 // query heads of a tile: columns of the matrix instructions
#define PG_C ((float)(1.4426950408889634 / 11.313708498984761))
#define PG_LOWEST (-3.402823466e38f)        // no logit is below it: a maximum that nothing has moved yet
#define PG_LAG (8.f / PG_C)         // by how much a product may exceed it, a weight of 2^8

template <int DT> constexpr int PG_ROW = RA_D * (DT == RA_BF16 ? 2 : 4);         // bytes of a row
template <int DT> constexpr int PG_PIECES = PG_ROW<DT> / 64;                     // of 16 bytes that a lane has of a chunk's keys, and of its values
#define PG_CHUNK 16                 // rows that a wavefront takes at a time

typedef __bf16 pg_bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 pg_bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 pg_f16x2 __attribute__((ext_vector_type(2)));
typedef short pg_s16x4 __attribute__((ext_vector_type(4)));
typedef float pg_f32x4 __attribute__((ext_vector_type(4), may_alias));
typedef uint32_t pg_u32x4 __attribute__((ext_vector_type(4), may_alias));

// ---- chunks of rows on the matrix cores --------------------------------------------------------
// A wavefront takes a chunk of rows for up to 16 query heads of one KV head, two products with nothing in between but registers:
//   logits  S[row][head]. Lane (kg, r) = (lane / 16, lane % 16) wants a quarter of row r, in pieces of 16 bytes that alternate between
//           the four kg, and ends with rows 4 kg + i of head r.
//   sums    O[dimension][head] += V^T P. The lane's weights are of rows 4 kg + i, so they go in as they come out; V^T wants the same rows:
//           lane (kg, r) has 16 bytes of each (16 lanes read a row, or half of a float32 one).
// Keys are read like values, whole lines an instruction, and turn into the first product's layout through shared memory of the wavefront's
// own, a piece p of row r at place p ^ r of the row, so that neither side meets in a bank (no conflicts counted). Read in that layout from memory, 64
// bytes of each of 16 rows an instruction, half of a line is fetched again where rows are not kept (65536 float32 rows of 8 heads 124 us a call,
// this way 103; bfloat16 96, 94).
// bfloat16: v_mfma_f32_16x16x32_bf16 for the logits, sums of exact products, and v_mfma_f32_16x16x16_bf16 for the sums. A float32 weight
// goes in as three terms of bfloat16, the first as rounded, the next what the rounding left: all of its 24 bits. Infinite values meet the first
// alone, or zero times infinity, or infinities of both signs, would be what is added up. Whether a chunk has one is asked with eight instructions: what has all bits of a
// bfloat16 exponent set is no number when it is read as float16 (so are values above 2^121, which lose nothing), and the maximum of float16 keeps that. (It costs 0 to 2 %; with
// masks and integer maxima, 31 instructions, 1 to 4 %; all rows again where a sum is no number, by a flag, 0 to 20 %, as registers run out.)
// float32: v_mfma_f32_16x16x4_f32, products and sums in float32.
// The running maximum of a head moves only when a logit exceeds it by more than 8 (in powers of two), which keeps the
// lanes' exchange and the scaling of sums out of nearly every chunk.
// What bounds it is the memory: of a dispatch of 84 us over 131072 rows of 8 heads the vector instructions take a fifth and the matrix
// instructions less; the same loads without the products take as long. One compute unit by itself takes in 57 GB a second: 9 ns a row, whatever
// is on its way (the next chunk, or two, asked for ahead: 93.6 and 94.4 us a call, as it is 91.6).
template <int DT>
struct PgChunk {
    pg_u32x4 k[PG_PIECES<DT>], v[PG_PIECES<DT>];             // piece r of rows 4 kg + i at [i], float32: pieces r and 16 + r at [2 i] and [2 i + 1]
    uint32_t there;             // bit j: the lane's row j of v is one that is attended
    uint64_t at[4];             // where the lane's rows of v are: bytes from the first, or (consecutive rows) the address of the first and bytes from there
};

// between what lanes of a wavefront store and others of it read, and the next stores there: the hardware keeps the wavefront's order, this keeps
// the compiler's
__device__ __forceinline__ void pg_wave_sync() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

template <int DT>
struct PgWave {
    static constexpr int PIECES = PG_PIECES<DT>;
    pg_u32x4 q[PIECES];
    pg_f32x4 acc[8];            // bfloat16: [m][x] is dimension 8 (4 kg + x) + m; float32: [4 h + c][x] is 64 h + 4 (4 kg + x) + c
    float m, l;                 // the maximum of <q, k>, and the weights' sum, of the lane's own rows

    // queries of heads 0 .. n - 1 of a tile, 128 values each; columns past them are the first one's, and nobody asks for them
    __device__ __forceinline__ void start(const void* q0, int n, int lane) {
        const int kg = lane >> 4, h = lane & 15;
        const char* at = reinterpret_cast<const char*>(q0) + (size_t)(h < n ? h : 0) * PG_ROW<DT> + 16 * kg;
#pragma unroll
        for (int i = 0; i < PIECES; ++i) q[i] = *reinterpret_cast<const pg_u32x4*>(at + 64 * i);
#pragma unroll
        for (int d = 0; d < 8; ++d) acc[d] = pg_f32x4{0.f, 0.f, 0.f, 0.f};
        m = PG_LOWEST;
        l = 0.f;
    }

    // `stage`: a chunk's keys in shared memory. `values` asks for the chunk's, with the keys, or (LATE) when these are in shared memory
    // (us, with the keys and later: 65536 float32 rows of 8 heads 106, 102, 128 float32 jobs of 1000 rows 33.7, 32.2, 128 sparse float32 jobs 39.4, 37.4; 64
    // and 128 bfloat16 jobs whose static rows' values come so 13.9, 13.6 and 18.6, 18.0, but 8 with 30000 static rows 36.4, 40.1). ONE: the rows are head
    // `head`'s alone, and other heads' sums stay as they are, whatever the rows hold.
    template <bool ONE, bool LATE, class F>
    __device__ __forceinline__ void add(PgChunk<DT>& c, F values, pg_u32x4* stage, int lane, int head = 0) {
        const int kg = lane >> 4, r = lane & 15;
        if (!LATE) values(c);
        pg_wave_sync();                                     // (the chunk before has been read)
#pragma unroll
        for (int j = 0; j < PIECES; ++j) {
            const int row = 4 * kg + j / (PIECES / 4), piece = 16 * (j % (PIECES / 4)) + r;
            stage[row * (PG_ROW<DT> / 16) + (piece ^ row)] = c.k[j];
        }
        pg_wave_sync();
        if (LATE) values(c);
        pg_f32x4 S[PIECES / 2] = {};        // (several sums: fewer roundings one after another, and an instruction waits for the one before it)
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            const pg_u32x4 k = stage[r * (PG_ROW<DT> / 16) + ((4 * i + kg) ^ r)];
            if constexpr (DT == RA_BF16)
                S[i & 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(pg_bf16x8, k), __builtin_bit_cast(pg_bf16x8, q[i]), S[i & 1], 0, 0, 0);
            else
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    S[e] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(k[e]), __uint_as_float(q[i][e]), S[e], 0, 0, 0);
        }
        const bool mine = !ONE || r == head;
        float z[4], top = -INFINITY;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            z[j] = DT == RA_BF16 ? S[0][j] + S[1][j] : (S[0][j] + S[1][j]) + (S[PIECES / 2 - 2][j] + S[PIECES / 2 - 1][j]);
            z[j] = mine && (c.there >> j) & 1u ? z[j] : -INFINITY;
            top = fmaxf(top, z[j]);
        }
        if (__builtin_amdgcn_ballot_w64(top > m + PG_LAG) != 0ull) {
            top = fmaxf(top, __uint_as_float(lane_xor32<16>(__float_as_uint(top), lane)));
            top = fmaxf(top, __uint_as_float(lane_xor32<32>(__float_as_uint(top), lane)));
            const float now = fmaxf(m, top), corr = __builtin_amdgcn_exp2f((m - now) * PG_C);
            m = now;
            l *= corr;
#pragma unroll
            for (int d = 0; d < 8; ++d) acc[d] *= corr;
        }
        float x[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            x[j] = __builtin_amdgcn_exp2f((z[j] - m) * PG_C);
            l += x[j];
        }
        if constexpr (DT == RA_BF16) {
            pg_s16x4 P[3];
#pragma unroll
            for (int t = 0; t < 3; ++t) {
                uint32_t pair[2];
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const pg_bf16x2 b = {(__bf16)x[2 * j], (__bf16)x[2 * j + 1]};
                    pair[j] = __builtin_bit_cast(uint32_t, b);
                    if (t < 2) { x[2 * j] -= bf16_lo(pair[j]); x[2 * j + 1] -= bf16_hi(pair[j]); }
                }
                P[t] = __builtin_bit_cast(pg_s16x4, (uint64_t)pair[1] << 32 | pair[0]);
            }
            uint32_t a[8][2];                                // dimension i of the lane's 8, of rows 0 and 1, 2 and 3
            pg_f16x2 odd = {0, 0};                           // no number in a half: values may be infinite
#pragma unroll
            for (int y = 0; y < 4; ++y) {                    // dimensions 2 y and 2 y + 1 share a word of every row
                uint32_t w[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) w[j] = (c.there >> j) & 1u ? c.v[j][y] : 0u;          // (0 * NaN is not 0)
#pragma unroll
                for (int j = 0; j < 4; ++j) odd = __builtin_elementwise_maximum(odd, __builtin_bit_cast(pg_f16x2, w[j]));
#pragma unroll
                for (int i = 0; i < 4; ++i) a[2 * y + i / 2][i % 2] = __builtin_amdgcn_perm(w[i % 2 * 2 + 1], w[i % 2 * 2], i / 2 ? 0x07060302u : 0x05040100u);
            }
            auto rows = [&](int i) { return __builtin_bit_cast(pg_s16x4, (uint64_t)a[i][1] << 32 | a[i][0]); };
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const pg_f32x4 sum = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(rows(i), P[0], acc[i], 0, 0, 0);
                acc[i] = mine ? sum : acc[i];
            }
            // what is infinite or no number has met the first terms
            if (__builtin_amdgcn_ballot_w64(odd[0] != odd[0] || odd[1] != odd[1]) != 0ull) {
#pragma unroll
                for (int i = 0; i < 8; ++i)
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        if ((a[i][j] & 0x7f80u) == 0x7f80u) a[i][j] &= 0xffff0000u;
                        if ((a[i][j] & 0x7f800000u) == 0x7f800000u) a[i][j] &= 0xffffu;
                    }
            }
#pragma unroll
            for (int i = 0; i < 8; ++i)                      // (of heads that are not `mine` these terms are zero)
#pragma unroll
                for (int t = 1; t < 3; ++t) acc[i] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(rows(i), P[t], acc[i], 0, 0, 0);
        } else {
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    pg_f32x4 sum = acc[4 * h + e];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const float w = (c.there >> j) & 1u ? __uint_as_float(c.v[PIECES / 4 * j + h][e]) : 0.f;
                        sum = __builtin_amdgcn_mfma_f32_16x16x4f32(w, x[j], sum, 0, 0, 0);
                    }
                    acc[4 * h + e] = mine ? sum : acc[4 * h + e];
                }
        }
    }
};

#define PG_PAD (RA_D + 4)
template <int WAVES>
struct PgLds {
    float a[WAVES][PG_HEADS][PG_PAD], m[WAVES][PG_HEADS], l[WAVES][PG_HEADS];
    int row[WAVES][PG_CHUNK], page[WAVES][PG_CHUNK];         // the sparse set's: rows and pages of Omega's first chunks
    // (a wavefront's keys and later its sums lie in the same place)
    __device__ __forceinline__ pg_u32x4* stage(int wv) { return reinterpret_cast<pg_u32x4*>(&a[wv][0][0]); }
};
static_assert(sizeof(float[PG_HEADS][PG_PAD]) >= PG_CHUNK * PG_ROW<RA_BF16> && sizeof(float[PG_HEADS][PG_PAD]) >= PG_CHUNK * PG_ROW<RA_F32> &&
              sizeof(float[PG_HEADS][PG_PAD]) % 16 == 0, "a chunk of keys fits");

// A wavefront's state for the first n heads into shared memory; a head without rows has the maximum -infinity.
template <int DT, int WAVES>
__device__ __forceinline__ void pg_leave(const PgWave<DT>& s, PgLds<WAVES>& lds, int n, int wv, int lane) {
    const int kg = lane >> 4, col = lane & 15;
    float l = s.l + __uint_as_float(lane_xor32<16>(__float_as_uint(s.l), lane));
    l += __uint_as_float(lane_xor32<32>(__float_as_uint(l), lane));
    pg_wave_sync();                                         // (the last chunk's keys, in whose place the sums go, have been read)
    if (col >= n) return;
    // a sum that is not a number keeps a maximum that is one, or it would count as empty
    if (kg == 0) {
        lds.m[wv][col] = l != l ? 0.f : l > 0.f ? s.m : -INFINITY;
        lds.l[wv][col] = l;
    }
#pragma unroll
    for (int x = 0; x < 4; ++x)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            float* to = &lds.a[wv][col][DT == RA_BF16 ? 8 * (4 * kg + x) + 4 * h : 64 * h + 4 * (4 * kg + x)];
            *reinterpret_cast<pg_f32x4*>(to) = pg_f32x4{s.acc[4 * h][x], s.acc[4 * h + 1][x], s.acc[4 * h + 2][x], s.acc[4 * h + 3][x]};
        }
}
// dimension d of head h from the states of the first `of_w` wavefronts, and of the others. No branches: all that is read is on its way at once.
template <int WAVES>
__device__ __forceinline__ void pg_together(const PgLds<WAVES>& lds, int of_w, int h, int d, RecSum (&x)[2]) {
    float m[WAVES], l[WAVES], a[WAVES];
#pragma unroll
    for (int w = 0; w < WAVES; ++w) { m[w] = lds.m[w][h]; l[w] = lds.l[w][h]; a[w] = lds.a[w][h][d]; }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        x[i] = RecSum{-INFINITY, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < WAVES; ++w) x[i].m = fmaxf(x[i].m, (w < of_w) == (i == 0) ? m[w] : -INFINITY);
        const float base = x[i].m > -INFINITY ? x[i].m : 0.f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {                // (a wavefront without rows has sums of zero)
            const bool is = (w < of_w) == (i == 0);
            const float wt = is ? __builtin_amdgcn_exp2f((m[w] - base) * PG_C) : 0.f;
            x[i].a = fmaf(is ? a[w] : 0.f, wt, x[i].a);
            x[i].l = fmaf(is ? l[w] : 0.f, wt, x[i].l);
        }
    }
}

// ---- where rows are --------------------------------------------------------------------------
// Rows of one KV head of one sequence. All rows of a pool are counted through, in 31 bits; a row without a page is number -1.
template <int DT>
struct PgRows {
    const char *k, *v;
    const int32_t* table;
    int page_log2, last, n_pages, n_kv, kv;

    // (the table comes as a kernel's argument of its own, which the compiler knows not to be written to: uniform entries are scalar loads)
    __device__ __forceinline__ PgRows(const PgCache& c, const int32_t* tab, int seq, int kv_head, int n_kv_heads)
        : k((const char*)c.k), v((const char*)c.v), table(tab + (size_t)seq * c.table_stride), page_log2(c.page_log2), last(c.table_pages - 1),
          n_pages(c.n_pages), n_kv(n_kv_heads), kv(kv_head) {}
    // the table's entry for a row (of rows past the table: the last)
    __device__ __forceinline__ int page_of(int row) const {
        const int p = row >> page_log2;
        return table[p < last ? p : last];
    }
    __device__ __forceinline__ int number(int page, int row) const {
        return (uint32_t)page < (uint32_t)n_pages ? ((page * n_kv + kv) << page_log2) + (row & ((1 << page_log2) - 1)) : -1;
    }
};

// A chunk of rows whose numbers the lanes hold, row j that of lane j. Loads are not branched around: a row that is not there is row 0. ONCE:
// non-temporal.
template <bool ONCE>
__device__ __forceinline__ pg_u32x4 pg_load(const char* at) {
    if constexpr (ONCE) return __builtin_nontemporal_load(reinterpret_cast<const pg_u32x4*>(at));
    else return *reinterpret_cast<const pg_u32x4*>(at);
}
template <bool ONCE, int DT>
__device__ __forceinline__ void pg_fetch(PgChunk<DT>& c, const PgRows<DT>& src, int number, int lane) {
    const int kg = lane >> 4, r = lane & 15;
    auto row = [](int n) { return (uint64_t)(uint32_t)(n < 0 ? 0 : n) * PG_ROW<DT>; };
    c.there = 0u;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int n = __shfl(number, 4 * kg + j);
        c.at[j] = row(n) + 16 * r;
        c.there |= (n >= 0 ? 1u : 0u) << j;
#pragma unroll
        for (int h = 0; h < PG_PIECES<DT> / 4; ++h) c.k[PG_PIECES<DT> / 4 * j + h] = pg_load<ONCE>(src.k + c.at[j] + 256 * h);
    }
}
template <bool ONCE, int DT>
__device__ __forceinline__ void pg_values(PgChunk<DT>& c, const PgRows<DT>& src) {
#pragma unroll
    for (int j = 0; j < PG_PIECES<DT>; ++j) c.v[j] = pg_load<ONCE>(src.v + c.at[j / (PG_PIECES<DT> / 4)] + j % (PG_PIECES<DT> / 4) * 256);
}

// a lane's pieces of consecutive rows, its first `by` behind the scalar `base`
template <int DT>
__device__ __forceinline__ void pg_consecutive(pg_u32x4 (&x)[PG_PIECES<DT>], uint64_t base, uint32_t by) {
    typedef const __attribute__((address_space(1))) char* at_t;
#pragma unroll
    for (int j = 0; j < PG_PIECES<DT>; ++j)
        x[j] = __builtin_nontemporal_load(reinterpret_cast<const __attribute__((address_space(1))) pg_u32x4*>(
            reinterpret_cast<at_t>(base) + (by + j / (PG_PIECES<DT> / 4) * PG_ROW<DT> + j % (PG_PIECES<DT> / 4) * 256)));
}

// A chunk of consecutive rows from `row` on, a multiple of 16 and the same in all lanes, in a page of 16 rows or more: what differs
// from lane to lane never changes. `page`: its entry of the table, `to`: rows that there are. Rows are read once, non-temporal.
template <int DT>
__device__ __forceinline__ void pg_fetch(PgChunk<DT>& c, const PgRows<DT>& src, int page, int row, int to, int lane) {
    const int kg = lane >> 4, r = lane & 15, n = src.number(page, row);
    const uint32_t mine = 4 * kg * PG_ROW<DT> + 16 * r;
    const uint64_t at = (uint64_t)(uint32_t)(n < 0 ? 0 : n) * PG_ROW<DT>;
    uint64_t k_at = (uint64_t)src.k + at, v_at = (uint64_t)src.v + at;
    asm("" : "+s"(k_at), "+s"(v_at));                        // (a scalar base and a lane's place: left to itself the compiler adds them up in vector registers)
    c.at[0] = v_at;
    c.at[1] = mine;
    c.there = 0u;
    pg_consecutive<DT>(c.k, k_at, mine);
#pragma unroll
    for (int j = 0; j < 4; ++j) c.there |= (n >= 0 && row + 4 * kg + j < to ? 1u : 0u) << j;
}

// ---- attention over all tokens -----------------------------------------------------------------
// The work is a list: per sequence, KV head and tile of its query heads (a job) the job's rows in units of 64, of 128 (a round of a workgroup's
// wavefronts) where there are more than that for each, or, for lists that would be too long for 32 bits, a power of two of these. Workgroups
// take equal stretches of that list, whatever the lengths of the sequences are, and leave a record per job they touched, at place
// (workgroup + job): going along the list, one or the other grows by one at a time. One workgroup of eight wavefronts per compute unit (us a call,
// 131072 rows of 8 heads and 16 sequences of up to 32768: 91.5, 170.6; two of eight 93.2, 173.2, one of 16 93.2, 172.9, two, three and four of
// four wavefronts 92.0, 93.9 and 94.5, 170.7, 172 and 176.3).
// Records lie per head of a tile, then place: sums [16][places][128], then maxima and sums of weights [16][places][2], so that
// what is combined lies in a row.
// A launch of as many workgroups as jobs (`whole`) gives each its job, and the workgroup writes the result.
#define PG_UNIT 64
#define PG_MOST_UNITS (1u << 21)    // times the workgroups, below 2^32
#define PG_MOST_WORKGROUPS 256      // one per compute unit

template <int DT, bool SMALL>
__global__ __launch_bounds__(PG_WAVES * RA_WAVE, DT == RA_BF16 ? 4 : 2) void pg_full_kernel(
    const void* __restrict__ q, PgCache c, const int32_t* __restrict__ table, int n_seq, int n_q, int n_kv, int N, const int32_t* __restrict__ n_tokens,
    int tiles, int unit_log2, int whole, float* __restrict__ partials, float* __restrict__ out, float* __restrict__ lse) {
    extern __shared__ __align__(16) char pg_lds[];
    PgLds<PG_WAVES>& lds = *reinterpret_cast<PgLds<PG_WAVES>*>(pg_lds);
    const int jobs = n_kv * tiles, group = n_q / n_kv, wg = blockIdx.x;
    uint32_t at = 0, end = 1, first = 0;
    int seq = wg / jobs;
    RowList x;
    if (!whole) {
        x = row_list(n_tokens, n_seq, 0, N, unit_log2, jobs, gridDim.x);
        if ((uint32_t)wg >= x.workgroups) return;
        at = x.from(wg);
        end = x.from(wg + 1);
        seq = row_seq_of(x, n_tokens, n_seq, N, unit_log2, jobs, at, &first);
    }
    const int tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid / RA_WAVE);
    while (at < end) {
        const int n = whole || seq >= RA_WAVE ? seq_rows(n_tokens, seq, N) : __builtin_amdgcn_readlane(x.rows, seq);
        const uint32_t units = row_units(n, unit_log2);
        int job = wg % jobs;
        uint32_t unit0 = 0, unit1 = units;
        if (!whole) {
            if (at >= first + units * jobs) {                // (the stretch goes on in the next sequence that has rows)
                first += units * jobs;
                ++seq;
                continue;
            }
            job = (int)((at - first) / units);
            unit0 = at - first - (uint32_t)job * units;
            unit1 = unit0 + (end - at) < units ? unit0 + (end - at) : units;
        }
        const int head_in_group = job % tiles * PG_HEADS, heads = group - head_in_group < PG_HEADS ? group - head_in_group : PG_HEADS;
        const size_t head0 = (size_t)seq * n_q + (size_t)(job / tiles) * group + head_in_group;
        const int64_t upto = (int64_t)unit1 << unit_log2;
        const int from = (int)((int64_t)unit0 << unit_log2), to = (int)(upto < n ? upto : n);
        const PgRows<DT> src(c, table, seq, job / tiles, n_kv);
        PgWave<DT> s;
        s.start(reinterpret_cast<const char*>(q) + head0 * PG_ROW<DT>, heads, lane);
        // The next chunk's entries of the table are on their way while the current one is worked on.
        constexpr int step = PG_WAVES * PG_CHUNK;
        int row = from + wv * PG_CHUNK;
        PgChunk<DT> a;
        if constexpr (SMALL) {
            auto number = [&](int at) {
                const int mine = at + (lane & (PG_CHUNK - 1)), n = src.number(src.page_of(mine), mine);
                return mine < to ? n : -1;
            };
            for (int number_of = number(row); row < to; row += step) {
                const int next = number(row + step);         // (asked for first: loads come back in order)
                pg_fetch<true>(a, src, number_of, lane);
                s.template add<false, DT == RA_F32>(a, [&](PgChunk<DT>& c) { pg_values<true>(c, src); }, lds.stage(wv), lane);
                number_of = next;
            }
        } else {
            for (int next = src.page_of(row); row < to; row += step) {
                pg_fetch(a, src, next, row, to, lane);
                next = src.page_of(row + step);
                s.template add<false, DT == RA_F32>(a, [](PgChunk<DT>& c) { pg_consecutive<DT>(c.v, c.at[0], (uint32_t)c.at[1]); }, lds.stage(wv), lane);
            }
        }
        const size_t places = (size_t)gridDim.x + (size_t)n_seq * jobs, place = (size_t)wg + (size_t)seq * jobs + job;
        pg_leave(s, lds, heads, wv, lane);
        __syncthreads();
        for (int y = tid; y < heads * RA_D; y += PG_WAVES * RA_WAVE) {
            const int hd = y / RA_D, d = y % RA_D;
            RecSum x[2];
            pg_together(lds, PG_WAVES, hd, d, x);
            const RecSum& all = x[0];
            if (!whole) {
                partials[(hd * places + place) * RA_D + d] = all.a;
                if (d == 0) reinterpret_cast<float2*>(partials + PG_HEADS * places * RA_D)[hd * places + place] = make_float2(all.m, all.l);
            } else {
                out[(head0 + hd) * RA_D + d] = all.m > -INFINITY ? all.a / all.l : 0.f;
                if (d == 0) lse[head0 + hd] = all.m > -INFINITY ? all.m * PG_C * REC_LN2 + logf(all.l) : -INFINITY;
            }
        }
        if (whole) return;
        at += unit1 - unit0;
        if (at < end) __syncthreads();                       // (the next job's sums go through the same LDS)
    }
}

// grid: x = head (with its sequence); SLICES threads per dimension take the records in turn, eight each on their way at a time: with 17 to 32 records
// a head (8 jobs over 256 workgroups) one trip and one exchange. (us a call, this and what combines other numbers of records, q4_full_merge_kernel: 8 heads of
// 4096 rows 9.3, 10.1, of 32768 28.6, 29.9; 8 records a head 8.2, 7.9; one KV head, 256 records, 96.5, 93.2.)
#define PG_MERGE_FEW 16
#define PG_MERGE_SLICES 4
__global__ __launch_bounds__(RA_D * PG_MERGE_SLICES) void pg_full_merge_kernel(const float* __restrict__ partials, int n_seq, int n_q, int n_kv, int N,
                                                                      const int32_t* __restrict__ n_tokens, int tiles, int unit_log2, int grid,
                                                                      float* __restrict__ out, float* __restrict__ lse) {
    constexpr int FLY = 8, SLICES = PG_MERGE_SLICES;
    __shared__ RecSum s_part[SLICES][RA_D];
    const int d = threadIdx.x % RA_D, slice = threadIdx.x / RA_D;
    const size_t head = blockIdx.x;
    const FullRecords y = full_records(partials, head, n_seq, n_q, n_kv, N, n_tokens, tiles, unit_log2, PG_HEADS, grid);
    RecSum x{-INFINITY, 0.f, 0.f};
    for (int i0 = slice; i0 < y.have; i0 += FLY * SLICES) {
        float m[FLY], l[FLY], a[FLY], mx = x.m;
#pragma unroll
        for (int u = 0; u < FLY; ++u) {
            const int i = i0 + u * SLICES, at = i < y.have ? i : i0;
            const float2 ml = y.ml[at];
            m[u] = i < y.have ? ml.x : -INFINITY;
            l[u] = ml.y;
            a[u] = y.sums[(size_t)at * RA_D + d];
        }
#pragma unroll
        for (int u = 0; u < FLY; ++u) mx = fmaxf(mx, m[u]);
        if (mx == -INFINITY) continue;
        const float corr = __builtin_amdgcn_exp2f((x.m - mx) * PG_C);
        x.a *= corr;
        x.l *= corr;
#pragma unroll
        for (int u = 0; u < FLY; ++u) {
            const bool is = m[u] > -INFINITY;
            const float w = __builtin_amdgcn_exp2f((m[u] - mx) * PG_C);
            x.a = fmaf(is ? a[u] : 0.f, w, x.a);
            x.l = fmaf(is ? l[u] : 0.f, w, x.l);
        }
        x.m = mx;
    }
    s_part[slice][d] = x;
    __syncthreads();
    if (slice) return;
    x = RecSum{-INFINITY, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < SLICES; ++i) x.m = fmaxf(x.m, s_part[i][d].m);
    const float base = x.m > -INFINITY ? x.m : 0.f;
#pragma unroll
    for (int i = 0; i < SLICES; ++i) {
        const float w = __builtin_amdgcn_exp2f((s_part[i][d].m - base) * PG_C);
        x.a = fmaf(s_part[i][d].a, w, x.a);
        x.l = fmaf(s_part[i][d].l, w, x.l);
    }
    out[head * RA_D + d] = x.m > -INFINITY ? x.a / x.l : 0.f;
    if (d == 0) lse[head] = x.m > -INFINITY ? x.m * PG_C * REC_LN2 + logf(x.l) : -INFINITY;
}

// How a call is cut. Each job is one workgroup's, and there is no second launch, where its rows are few or the jobs many enough to fill the part: by
// themselves and shared out, us, bfloat16: 8 jobs of 250 rows 5.3, 7.8, of 500 7.5, 7.8, of 1000 11.1, 8.0; 128 of 500 9.3, 12.5, of 1000 16.3, 18.7,
// of 2000 27.5, 28.3; 512 of 500 24.5, 31.2, of 2000 86.3, 91.2; float32: 8 of 250 8.8, 9.5, of 400 12.2, 11.1; 128 of 250 11.0, 13.3, of 500 19.5,
// 19.2, of 1000 32.3, 29.5; 512 of 500 54.8, 59.3, of 2000 185, 191. No more than 2048 rows: the lengths are known on the device only, and what a
// job that is longer than the others takes alone is 9 ns a row (float32: 26).
#define PG_MOST_ROWS (1 << 24)      // of one job that a workgroup takes alone
struct PgCut { int tiles, workgroups, unit_log2; bool whole; const char* refused; };       // refused: why, or null
static PgCut pg_cut(ra_dtype dt, int n_seq, int n_q, int n_kv, int64_t N) {
    PgCut x;
    x.tiles = (int)(((int64_t)(n_q / n_kv) + PG_HEADS - 1) / PG_HEADS);
    const int64_t jobs = (int64_t)n_seq * n_kv * x.tiles;
    // (from PG_MOST_UNITS jobs on there is no list: its units, and the threads of the second kernel, 128 for each of up to 16 heads, fit 32 bits)
    const int64_t few = dt == RA_BF16 ? 640 : 320, per_job = dt == RA_BF16 ? 16 : 4;
    x.whole = N <= few || (N <= 2048 && N <= per_job * jobs) || (jobs >= PG_MOST_UNITS && N <= PG_MOST_ROWS);
    x.unit_log2 = jobs * N <= 2 * PG_UNIT * PG_MOST_WORKGROUPS ? 6 : 7;
    static_assert(PG_UNIT == 1 << 6, "rows of a unit");
    x.refused = x.whole && jobs >= 1 << 23 ? "too many heads for one launch: 2^23 tiles of up to 16 query heads"
                : !x.whole && jobs >= PG_MOST_UNITS ? "too many heads for one launch: 2^21 tiles of up to 16 query heads over more than 2^24 tokens" : nullptr;
    x.workgroups = (int)jobs;
    if (x.whole || x.refused) return x;
    auto units = [&] { return jobs * ((N + ((int64_t)1 << x.unit_log2) - 1) >> x.unit_log2); };
    while (units() > PG_MOST_UNITS) ++x.unit_log2;
    const int64_t most = (units() + ROW_LEAST_UNITS - 1) / ROW_LEAST_UNITS;           // (with more, some would have nothing to do)
    x.workgroups = (int)(most < PG_MOST_WORKGROUPS ? most : PG_MOST_WORKGROUPS);
    return x;
}

size_t ra_full_paged_partial_floats(ra_dtype dt, int n_seq, int n_q, int n_kv, int64_t N) {
    const PgCut x = pg_cut(dt, n_seq, n_q, n_kv, N);
    return x.whole || x.refused ? 0 : ((size_t)x.workgroups + (size_t)n_seq * n_kv * x.tiles) * PG_HEADS * (RA_D + 2);
}

ra_status ra_launch_full_paged(const void* q, ra_dtype dt, const PgCache& c, int n_seq, int n_q, int n_kv, int64_t N, const int32_t* n_tokens,
                               float* partials, hipStream_t st, float* out, float* lse) {
    const PgCut x = pg_cut(dt, n_seq, n_q, n_kv, N);
    if (x.refused) RA_FAIL(RA_EUNSUP, "%s", x.refused);
#define PG_GO(DTV, SMALL)                                                                                                                             \
    do {                                                                                                                                              \
        constexpr auto kernel = &pg_full_kernel<DTV, SMALL>;                                                                                          \
        RA_LDS_OPT_IN(*kernel, sizeof(PgLds<PG_WAVES>));                                                                                              \
        hipLaunchKernelGGL(*kernel, dim3(x.workgroups), dim3(PG_WAVES * RA_WAVE), sizeof(PgLds<PG_WAVES>), st, q, c, c.table, n_seq, n_q, n_kv, (int)N, \
                           n_tokens, x.tiles, x.unit_log2, (int)x.whole, partials, out, lse);                                                         \
    } while (0)
    if (c.page_log2 < 4) { if (dt == RA_BF16) PG_GO(RA_BF16, true); else PG_GO(RA_F32, true); }
    else if (dt == RA_BF16) PG_GO(RA_BF16, false);
    else PG_GO(RA_F32, false);
#undef PG_GO
    RA_HIP(hipGetLastError());
    if (x.whole) return RA_OK;
    // records per head, were all sequences as long as the longest
    const int records = x.workgroups / (n_seq * n_kv * x.tiles);
    if (records <= PG_MERGE_FEW || records > 8 * PG_MERGE_SLICES)
        return ra_launch_full_merge(partials, n_seq, n_q, n_kv, N, n_tokens, x.tiles, x.unit_log2, PG_HEADS, x.workgroups, PG_C, st, out, lse);
    hipLaunchKernelGGL(pg_full_merge_kernel, dim3(n_seq * n_q), dim3(RA_D * PG_MERGE_SLICES), 0, st, partials, n_seq, n_q, n_kv, (int)N, n_tokens,
                       x.tiles, x.unit_log2, x.workgroups, out, lse);
    RA_HIP(hipGetLastError());
    return RA_OK;
}

// ---- the retrieved set and the static set -------------------------------------------------------
// W of a sequence, [0, s) u [w, n); ranges that meet make everything static. The host knows neither n nor how many tokens came after
// the index was built; what the parts of a job take is worked out here.
struct PgSets { int s, w, count; };         // count: rows of W
// lens: n_tokens[seq] in lane 0 and n_indexed[seq] in lane 1
__device__ __forceinline__ PgSets pg_sets(int lens, bool has_tokens, bool has_indexed, int N, int sink, int window) {
    PgSets x;
    const int given = __builtin_amdgcn_readlane(lens, 0), given_indexed = __builtin_amdgcn_readlane(lens, 1);
    auto upto = [](int v, int most) { return v < 0 ? 0 : v < most ? v : most; };
    const int n = has_tokens ? upto(given, N) : N, indexed = has_indexed ? upto(given_indexed, n) : n;
    x.s = sink < n ? sink : n;
    const int w = window < n ? n - window : 0, late = w < indexed ? w : indexed;
    x.w = late > x.s ? late : x.s;
    x.count = x.s + n - x.w;
    return x;
}

// A job is a KV head of a sequence, and up to 16 of its query heads: chunks of W, for all of the heads, and of each head's Omega. It is cut into
// `parts` workgroups, each of which takes an equal stretch of either list and shares its wavefronts out between the two.
// They leave a record of each set per head, or, where a job is one workgroup's, the results. grid: x = part, y = KV head (with its tile), z = sequence. What bounds it is the way from the
// lengths and ids to the table and from there to the rows, three trips, and the second launch; where jobs are many, the same way of each, as a
// workgroup has a compute unit to itself (bfloat16: 139 KB of shared memory; float32: registers for two wavefronts a SIMD) and nothing runs beside its
// start and end (256 jobs of 644 static rows and 4 x 100 ids, 137 MB, 32 to 34 us, 128 float32 ones, 137 MB, 38).
template <int DT, int WAVES>
__global__ __launch_bounds__(WAVES * RA_WAVE, DT == RA_BF16 ? 4 : 2) void pg_attend_kernel(
    const void* __restrict__ q, PgCache c, const int32_t* __restrict__ table, int group, int n_kv, int N, const int32_t* __restrict__ n_tokens,
    const int32_t* __restrict__ n_indexed, int sink, int window, int topk, int per_head, const int32_t* __restrict__ ids, int tiles,
    float* __restrict__ partials, SetOut o) {
    extern __shared__ __align__(16) char pg_lds[];
    PgLds<WAVES>& lds = *reinterpret_cast<PgLds<WAVES>*>(pg_lds);
    const int tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid / RA_WAVE), r = lane & 15;
    const int part = blockIdx.x, parts = gridDim.x, seq = blockIdx.z;
    const int kv_head = tiles == 1 ? (int)blockIdx.y : (int)blockIdx.y / tiles, first = tiles == 1 ? 0 : (int)blockIdx.y % tiles * PG_HEADS;
    const int heads = group - first < PG_HEADS ? group - first : PG_HEADS;
    const size_t head0 = ((size_t)seq * n_kv + kv_head) * group + first;
    const PgRows<DT> src(c, table, seq, kv_head, n_kv);
    // the lengths, one lane's load each; the table's first entry where one is not given
    const int32_t *at_tokens = n_tokens ? n_tokens + seq : table, *at_indexed = n_indexed ? n_indexed + seq : table;
    const int lens = *(lane & 1 ? at_indexed : at_tokens);
    // the part's stretch of a list
    auto cut = [&](uint32_t chunks, int& from, int& many) {
        const uint32_t each = chunks / (uint32_t)parts, more = chunks - each * parts;
        from = (int)(each * part + min((uint32_t)part, more));
        many = (int)(each + ((uint32_t)part < more ? 1u : 0u));
    };
    int w0, ws, g0, gs;
    const int in_om = heads * per_head;
    cut(in_om, g0, gs);
    // chunk i of the part's Omega: row r of it (-1 past a head's list)
    auto id_of = [&](int i) {
        const uint32_t x = g0 + i < in_om ? g0 + i : in_om - 1, h = x / (uint32_t)per_head;
        const int j = (int)(x - h * per_head) * PG_CHUNK + r, id = ids[(head0 + h) * topk + (j < topk ? j : topk - 1)];
        return j < topk ? id : -1;
    };
    // (a row's page is asked for before it is known whether the row is one)
    auto page_of = [&](int row) { return src.page_of(row < 0 ? 0 : row); };
    // What Omega's wavefronts begin with is asked for by all, while the lengths that say which these are are on their way (one sequence of 8 KV heads
    // 8.9 -> 8.5 us; where a job is one workgroup's of 16 wavefronts, all of which would wait for it, 17.9 -> 18.9).
    constexpr bool EARLY = WAVES == PG_WAVES;
    if (EARLY && wv < gs) {
        const int row = id_of(wv), page = page_of(row);
        if (lane < PG_CHUNK) {
            lds.row[wv][r] = row;
            lds.page[wv][r] = page;
        }
    }
    const PgSets set = pg_sets(lens, n_tokens != nullptr, n_indexed != nullptr, N, sink, window);
    cut((set.count + PG_CHUNK - 1) / PG_CHUNK, w0, ws);
    // wavefronts of W's chunks; the others have Omega's
    int of_w = (int)((uint32_t)(WAVES * ws + (ws + gs) / 2) / (uint32_t)(ws + gs > 0 ? ws + gs : 1));
    if (of_w < 1 && ws > 0) of_w = 1;
    if (of_w > WAVES - 1 && gs > 0) of_w = WAVES - 1;
    const bool om = wv >= of_w;
    const int step = om ? WAVES - of_w : of_w, chunks = om ? gs : ws;
    auto w_row_of = [&](int i) {
        const int j = (w0 + i) * PG_CHUNK + r;
        return j < set.s ? j : set.w - set.s + j;
    };
    int i = om ? wv - of_w : wv, row = om ? 0 : w_row_of(i), page = om ? 0 : src.page_of(row);
    PgWave<DT> st;
    st.start(reinterpret_cast<const char*>(q) + head0 * PG_ROW<DT>, heads, lane);
    if (EARLY) __syncthreads();
    PgChunk<DT> a;
    auto values = [&](PgChunk<DT>& c) { pg_values<false>(c, src); };
    // What leads to the next chunk's rows, their entries of the table and before these the ids, is asked for ahead of the current chunk's rows:
    // loads come back in order, and who waits for one behind the rows waits for the rows.
    if (!om) {
        for (; i < chunks; i += step) {
            const int next = w_row_of(i + step), next_page = src.page_of(next);
            pg_fetch<false>(a, src, (w0 + i) * PG_CHUNK + r < set.count ? src.number(page, row) : -1, lane);
            st.template add<false, true>(a, values, lds.stage(wv), lane);
            row = next;
            page = next_page;
        }
    } else if (i < chunks) {
        row = EARLY ? lds.row[i][r] : id_of(i);
        page = EARLY ? lds.page[i][r] : page_of(row);
        for (int next = i + step < chunks ? id_of(i + step) : -1; i < chunks; i += step) {
            const int next_page = page_of(next), after = id_of(i + 2 * step);
            pg_fetch<false>(a, src, row >= set.s && row < set.w ? src.number(page, row) : -1, lane);      // (members of W are attended there)
            st.template add<true, DT == RA_F32>(a, values, lds.stage(wv), lane, (g0 + i) / per_head);
            row = next;
            next = after;
            page = next_page;
        }
    }
    pg_leave(st, lds, heads, wv, lane);
    __syncthreads();
    for (int y = tid; y < heads * RA_D; y += WAVES * RA_WAVE) {
        const int hd = y / RA_D, d = y % RA_D;
        RecSum both[2];
        pg_together(lds, of_w, hd, d, both);
        if (parts == 1) {
            rec_write(both, head0 + hd, d, PG_C, o);
            continue;
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            float* rec = partials + ((head0 + hd) * 2 + i) * parts * REC_FLOATS + (size_t)part * REC_FLOATS;
            rec[d] = both[i].a;
            if (d == 0) { rec[RA_D] = both[i].m; rec[RA_D + 1] = both[i].l; }
        }
    }
}

// grid: x = head (with its sequence); for each set SLICES threads per dimension take the records in turn
template <int SLICES>
__global__ __launch_bounds__(2 * RA_D * SLICES) void pg_merge_kernel(const float* __restrict__ partials, int parts, SetOut o) {
    __shared__ RecSum s_part[SLICES][2][RA_D];
    const size_t head = blockIdx.x;
    const int d = threadIdx.x % RA_D, i = threadIdx.x / RA_D % 2, slice = threadIdx.x / (2 * RA_D);
    s_part[slice][i][d] = rec_add_up<false>(partials + (head * 2 + i) * parts * REC_FLOATS, slice, parts, SLICES, d, PG_C);
    __syncthreads();
    if (threadIdx.x >= RA_D) return;
    RecSum set[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        RecSum x{-INFINITY, 0.f, 0.f};
#pragma unroll
        for (int y = 0; y < SLICES; ++y) x.m = fmaxf(x.m, s_part[y][k][d].m);
        const float base = x.m > -INFINITY ? x.m : 0.f;
#pragma unroll
        for (int y = 0; y < SLICES; ++y) {
            const float w = __builtin_amdgcn_exp2f((s_part[y][k][d].m - base) * PG_C);
            x.a = fmaf(s_part[y][k][d].a, w, x.a);
            x.l = fmaf(s_part[y][k][d].l, w, x.l);
        }
        set[k] = x;
    }
    rec_write(set, head, d, PG_C, o);
}

// How a job is cut: half a round of chunks for a workgroup's wavefronts each, up to so many workgroups that each has a compute unit to itself
// (us, a whole round and half of one: 8 jobs of 644 static rows and 4 x 100 ids 9.8, 9.7, with 2000 static rows 12.6, 10.6, with 30000
// 59.5, 41.5, float32 13.9, 12.6; 16 query heads of one KV head 12.0, 13.1). Tokens that have come since the index was built are not counted, as the host does
// not know how many they are: a job that has grown by 30000 rows is cut by its window and ids alone (one KV head, window 0, one id, one workgroup 197 us;
// eight, window 64, 16 ids 150, window 640, 100 ids 40; one sequence of 16, in bfloat16 a workgroup for each KV head, 286).
// Many jobs are one workgroup's each (128 of them, bfloat16, by themselves with 16 wavefronts 18.2, with eight 19.9, in two 19.6 and a launch more;
// 64 14.8, in four 13.5; float32, which has registers for eight wavefronts: 128 48, in two 40).
static int pg_parts(ra_dtype dt, int n_seq, int n_q, int n_kv, int64_t N, int sink, int window, int topk, int* tiles) {
    const int group = n_q / n_kv, heads = group < PG_HEADS ? group : PG_HEADS;
    *tiles = (group + PG_HEADS - 1) / PG_HEADS;
    const int64_t both = (int64_t)sink + window, rows = both < N ? both : N, jobs = (int64_t)n_seq * n_kv * *tiles;
    const int64_t chunks = (rows + PG_CHUNK - 1) / PG_CHUNK + (int64_t)heads * ((topk + PG_CHUNK - 1) / PG_CHUNK);
    const int64_t rounds = (chunks + PG_WAVES / 2 - 1) / (PG_WAVES / 2), most = jobs >= (dt == RA_BF16 ? 128 : 256) ? 1 : PG_MOST_WORKGROUPS / jobs;
    return (int)(rounds < most ? rounds : most);
}

size_t ra_attend_paged_partial_floats(ra_dtype dt, int n_seq, int n_q, int n_kv, int64_t N, int sink, int window, int topk) {
    int tiles;
    const int parts = pg_parts(dt, n_seq, n_q, n_kv, N, sink, window, topk, &tiles);
    return parts == 1 ? 0 : (size_t)n_seq * n_q * 2 * parts * REC_FLOATS;
}

ra_status ra_launch_attend_paged(const void* q, ra_dtype dt, const PgCache& c, int n_seq, int n_q, int n_kv, int64_t N, const int32_t* n_tokens,
                                 const int32_t* n_indexed, int sink, int window, int topk, const int32_t* ids, float* partials, hipStream_t st,
                                 float* out, float* lse, float* o_omega, float* lse_omega, float* o_w, float* lse_w) {
    int tiles;
    const int parts = pg_parts(dt, n_seq, n_q, n_kv, N, sink, window, topk, &tiles);
    const int64_t per_seq = (int64_t)n_kv * tiles;
    if (n_seq > 65535 || per_seq > 65535 || n_seq * per_seq * parts > (1 << 22) - 1) RA_FAIL(RA_EUNSUP, "too many heads for one launch");
    const SetOut o{nullptr, out, lse, o_omega, lse_omega, o_w, lse_w};
#define PG_GO(DTV, W)                                                                                                                           \
    do {                                                                                                                                        \
        constexpr auto kernel = &pg_attend_kernel<DTV, W>;                                                                                      \
        RA_LDS_OPT_IN(*kernel, sizeof(PgLds<W>));                                                                                               \
        hipLaunchKernelGGL(*kernel, dim3(parts, (unsigned)per_seq, n_seq), dim3(W * RA_WAVE), sizeof(PgLds<W>), st, q, c, c.table, n_q / n_kv,  \
                           n_kv, (int)N, n_tokens, n_indexed, sink, window, topk, (topk + PG_CHUNK - 1) / PG_CHUNK, ids, tiles, partials, o);   \
    } while (0)
    if (dt == RA_F32) PG_GO(RA_F32, PG_WAVES);
    else if (parts == 1) PG_GO(RA_BF16, 2 * PG_WAVES);
    else PG_GO(RA_BF16, PG_WAVES);
#undef PG_GO
    RA_HIP(hipGetLastError());
    if (parts == 1) return RA_OK;
    if (parts <= 8) hipLaunchKernelGGL(pg_merge_kernel<1>, dim3(n_seq * n_q), dim3(2 * RA_D), 0, st, partials, parts, o);
    else hipLaunchKernelGGL(pg_merge_kernel<4>, dim3(n_seq * n_q), dim3(2 * RA_D * 4), 0, st, partials, parts, o);
    RA_HIP(hipGetLastError());
    return RA_OK;
}

// ---- rows side by side ------------------------------------------------------------------------
// A group of lanes takes a row, 16 bytes a lane: its entry of the table, then the row. What hides the two trips is how many rows are on their way: a
// group with two or four of them is slower (131072 rows of 8 heads 89 and 90 us, 4096 rows 3.6 and 3.7, one each 88 and 3.5). Written
// once, non-temporal (91.6 us; 100 with plain stores). Read so, too, where that is more than a quarter of what the memory side keeps: what a call reads
// may have just been made (us, plain and non-temporal loads: 8192 rows of 8 heads, 17 MB, 6.6, 7.5; 32768, 67 MB, 22.1, 25.0, where nothing
// of them is kept 25.4, 23.4; 131072, 268 MB, 91.6, 88.0).
#define PG_KEPT (1 << 26)
template <int DT, bool ONCE>
__global__ __launch_bounds__(PG_GATHER_THREADS) void pg_gather_kernel(const char* __restrict__ pages, PgCache c, const int32_t* __restrict__ table,
                                                                      int n_kv, int64_t T, uint32_t blocks, const int32_t* __restrict__ first,
                                                                      char* __restrict__ X) {
    constexpr int LANES = PG_ROW<DT> / 16, GROUPS = PG_GATHER_THREADS / LANES;
    const int l = threadIdx.x % LANES;
    const uint32_t head = blockIdx.x / blocks, seq = head / n_kv;
    const int64_t t = (int64_t)(blockIdx.x % blocks) * GROUPS + threadIdx.x / LANES, at = (first ? first[seq] : 0) + t;
    if (t >= T) return;
    const PgRows<DT> src(c, table, seq, head % n_kv, n_kv);
    const bool in = at >= 0 && at < ((int64_t)src.last + 1) << src.page_log2;
    const int row = in ? (int)at : 0, n = src.number(src.page_of(row), row);
    pg_u32x4 x = pg_load<ONCE>(pages + (uint64_t)(uint32_t)(n < 0 ? 0 : n) * PG_ROW<DT> + 16 * l);
    if (!in || n < 0) x = pg_u32x4{0u, 0u, 0u, 0u};
    __builtin_nontemporal_store(x, reinterpret_cast<pg_u32x4*>(X + ((uint64_t)head * T + t) * PG_ROW<DT> + 16 * l));
}

ra_status ra_launch_gather_paged(const PgCache& c, const void* pages, ra_dtype dt, int n_seq, int n_kv, int64_t T, const int32_t* first,
                                 hipStream_t st, void* X) {
    const int64_t heads = (int64_t)n_seq * n_kv, row = dt == RA_BF16 ? PG_ROW<RA_BF16> : PG_ROW<RA_F32>;
    const int64_t rows = PG_GATHER_THREADS * 16 / row, blocks = (T + rows - 1) / rows;
    if (heads > (1 << 24) - 1 || heads * blocks > (1 << 24) - 1) RA_FAIL(RA_EUNSUP, "too many rows for one launch");
#define PG_GO(DTV, ONCE)                                                                                                                             \
    hipLaunchKernelGGL((pg_gather_kernel<DTV, ONCE>), dim3((unsigned)(heads * blocks)), dim3(PG_GATHER_THREADS), 0, st, (const char*)pages, c, c.table, \
                       n_kv, T, (uint32_t)blocks, first, (char*)X)
    if (heads * T * row > PG_KEPT) { if (dt == RA_BF16) PG_GO(RA_BF16, true); else PG_GO(RA_F32, true); }
    else if (dt == RA_BF16) PG_GO(RA_BF16, false);
    else PG_GO(RA_F32, false);
#undef PG_GO
    RA_HIP(hipGetLastError());
    return RA_OK;
}
