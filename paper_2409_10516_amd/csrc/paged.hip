// A cache in pages (the layout is in include/ra.h): attention over all tokens (ra_full_attention_paged), over the retrieved set Omega and
// the static set W of Sec. 3.3 with their combination by Eq. 4-5 (ra_attend_paged), and rows side by side again (ra_gather_paged).
// What puts tokens into pages is with the other calls that append (kv4.hip).
//
// Rows are cut into parts; a workgroup turns one part into a record (128 weighted sums, the running maximum of
// z log2(e), the sum of weights), and a head's records are combined by a second kernel. Weights are powers of two,
// p = 2^(c <q, k> - m) with c = log2(e) / sqrt(d): one multiply-add and one instruction each.
#include "common.h"
#include "records.h"

#define PG_THREADS 256
#define PG_WAVES (PG_THREADS / RA_WAVE)
#define PG_HEADS 16                 // query heads of a tile: columns of the matrix instructions
#define PG_PART 128                 // rows of a part of the sparse set
#define PG_C ((float)(1.4426950408889634 / 11.313708498984761))
#define PG_LOWEST (-1.7e38f)        // below every logit: a maximum that nothing has moved yet

template <int DT> constexpr int PG_ROW = RA_D * (DT == RA_BF16 ? 2 : 4);         // bytes of a row
template <int DT> constexpr int PG_CHUNK = DT == RA_BF16 ? 32 : 16;             // rows that a wavefront takes at a time

typedef __bf16 pg_bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 pg_bf16x8 __attribute__((ext_vector_type(8)));
typedef float pg_f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t pg_u32x4 __attribute__((ext_vector_type(4)));

// ---- chunks of rows on the matrix cores --------------------------------------------------------
// A wavefront takes a chunk of rows for up to 16 query heads of one KV head, two products with nothing in between but registers:
//   logits  S[row][head]. Lane (kg, r) = (lane / 16, lane % 16) holds a quarter of row r, in pieces of 16 bytes that alternate between
//           the four kg, so that an instruction reads 64 bytes of each of 16 rows. It ends with rows 4 kg + i of head r.
//   sums    O[dimension][head] += V^T P. The lane's weights are of rows 4 kg + i, so they go in as they come out; V^T wants the same rows:
//           lane (kg, r) reads 16 bytes of each (16 lanes read a row, or half of a float32 one).
// bfloat16: v_mfma_f32_16x16x32_bf16, 32 rows. Logits are sums of exact products. A float32 weight goes in as three terms of
// bfloat16, the first as rounded, the next what the rounding left: all of its 24 bits. (An infinite value times the lesser terms is not a number.)
// float32: v_mfma_f32_16x16x4_f32, 16 rows, products and sums in float32.
// The running maximum of a head moves only when a logit exceeds it by more than 8 (in powers of two), which keeps the
// lanes' exchange and the scaling of sums out of nearly every chunk.
template <int DT>
struct PgChunk {
    pg_u32x4 k[8], v[8];        // bfloat16: pieces 64 i + 16 kg of row 16 t + r at [4 t + i], rows 16 t + 4 kg + i at [4 t + i]
                                // float32: pieces 64 i + 16 kg of row r at [i], halves h of rows 4 kg + i at [2 i + h]
    uint32_t there;             // bit j: the lane's row j of v is one that is attended
};

template <int DT>
struct PgWave {
    static constexpr int MINE = PG_CHUNK<DT> / 4;            // rows of a lane
    pg_u32x4 q[DT == RA_BF16 ? 4 : 8];
    pg_f32x4 acc[8];            // bfloat16: [m][x] is dimension 8 (4 kg + x) + m; float32: [4 h + c][x] is 64 h + 4 (4 kg + x) + c
    float m, l;                 // l: of the lane's own rows

    // queries of heads 0 .. n - 1 of a tile, 128 values each; columns past them are the first one's, and nobody asks for them
    __device__ __forceinline__ void start(const void* q0, int n, int lane) {
        const int kg = lane >> 4, h = lane & 15;
        const char* at = reinterpret_cast<const char*>(q0) + (size_t)(h < n ? h : 0) * PG_ROW<DT> + 16 * kg;
#pragma unroll
        for (int i = 0; i < (DT == RA_BF16 ? 4 : 8); ++i) q[i] = *reinterpret_cast<const pg_u32x4*>(at + 64 * i);
#pragma unroll
        for (int d = 0; d < 8; ++d) acc[d] = pg_f32x4{0.f, 0.f, 0.f, 0.f};
        m = PG_LOWEST;
        l = 0.f;
    }

    __device__ __forceinline__ void add(const PgChunk<DT>& c, int lane) {
        float z[MINE], top = PG_LOWEST;
        if constexpr (DT == RA_BF16) {
            pg_f32x4 S[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int t = 0; t < 2; ++t)
                    S[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(pg_bf16x8, c.k[4 * t + i]),
                                                                   __builtin_bit_cast(pg_bf16x8, q[i]), S[t], 0, 0, 0);
#pragma unroll
            for (int j = 0; j < 8; ++j) z[j] = S[j / 4][j & 3];
        } else {
            pg_f32x4 S[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};       // (two sums side by side: an instruction waits for the one before it)
#pragma unroll
            for (int i = 0; i < 8; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    S[e & 1] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(c.k[i][e]), __uint_as_float(q[i][e]), S[e & 1], 0, 0, 0);
#pragma unroll
            for (int j = 0; j < 4; ++j) z[j] = S[0][j] + S[1][j];
        }
#pragma unroll
        for (int j = 0; j < MINE; ++j) {
            z[j] = (c.there >> j) & 1u ? z[j] : -INFINITY;
            top = fmaxf(top, z[j]);
        }
        if (__builtin_amdgcn_ballot_w64(top * PG_C > m + 8.f) != 0ull) {
            top = fmaxf(top, __uint_as_float(lane_xor32<16>(__float_as_uint(top), lane)));
            top = fmaxf(top, __uint_as_float(lane_xor32<32>(__float_as_uint(top), lane)));
            const float now = fmaxf(m, top * PG_C), corr = __builtin_amdgcn_exp2f(m - now);
            m = now;
            l *= corr;
#pragma unroll
            for (int d = 0; d < 8; ++d) acc[d] *= corr;
        }
        float x[MINE];
#pragma unroll
        for (int j = 0; j < MINE; ++j) {
            x[j] = __builtin_amdgcn_exp2f(fmaf(z[j], PG_C, -m));
            l += x[j];
        }
        if constexpr (DT == RA_BF16) {
            pg_bf16x8 P[3];
#pragma unroll
            for (int t = 0; t < 3; ++t) {
                uint32_t pair[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const pg_bf16x2 b = {(__bf16)x[2 * j], (__bf16)x[2 * j + 1]};
                    pair[j] = __builtin_bit_cast(uint32_t, b);
                    if (t < 2) { x[2 * j] -= bf16_lo(pair[j]); x[2 * j + 1] -= bf16_hi(pair[j]); }
                }
                P[t] = __builtin_bit_cast(pg_bf16x8, pg_u32x4{pair[0], pair[1], pair[2], pair[3]});
            }
#pragma unroll
            for (int y = 0; y < 4; ++y) {                    // dimensions 2 y and 2 y + 1 of the lane's 8, which share a word of every row
                uint32_t w[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) w[j] = (c.there >> j) & 1u ? c.v[j][y] : 0u;          // (0 * NaN is not 0)
#pragma unroll
                for (int o = 0; o < 2; ++o) {
                    const uint32_t half = o ? 0x07060302u : 0x05040100u;
                    const pg_u32x4 a = {__builtin_amdgcn_perm(w[1], w[0], half), __builtin_amdgcn_perm(w[3], w[2], half),
                                        __builtin_amdgcn_perm(w[5], w[4], half), __builtin_amdgcn_perm(w[7], w[6], half)};
#pragma unroll
                    for (int t = 2; t >= 0; --t)
                        acc[2 * y + o] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(pg_bf16x8, a), P[t], acc[2 * y + o], 0, 0, 0);
                }
            }
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const bool have = (c.there >> j) & 1u;
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float w = have ? __uint_as_float(c.v[2 * j + h][e]) : 0.f;
                        acc[4 * h + e] = __builtin_amdgcn_mfma_f32_16x16x4f32(w, x[j], acc[4 * h + e], 0, 0, 0);
                    }
            }
        }
    }
};

#define PG_PAD (RA_D + 4)
struct PgLds { float a[PG_WAVES][PG_HEADS][PG_PAD], m[PG_WAVES][PG_HEADS], l[PG_WAVES][PG_HEADS]; };

// The states of the wavefronts -> one per head: f(head of the tile, dimension, sum, maximum, sum of weights), called by
// one thread for each; a head without rows has the maximum -infinity.
template <int DT, class Fn>
__device__ __forceinline__ void pg_close(const PgWave<DT>& s, PgLds& lds, int n, int tid, Fn f) {
    const int wv = tid / RA_WAVE, lane = tid & 63, kg = lane >> 4, col = lane & 15;
    float l = s.l + __uint_as_float(lane_xor32<16>(__float_as_uint(s.l), lane));
    l += __uint_as_float(lane_xor32<32>(__float_as_uint(l), lane));
    if (col < n) {
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
                *reinterpret_cast<float4*>(to) = make_float4(s.acc[4 * h][x], s.acc[4 * h + 1][x], s.acc[4 * h + 2][x], s.acc[4 * h + 3][x]);
            }
    }
    __syncthreads();
    for (int x = tid; x < n * RA_D; x += PG_THREADS) {
        const int h = x / RA_D, d = x % RA_D;
        float m[PG_WAVES], mx = -INFINITY, a = 0.f, ll = 0.f;
#pragma unroll
        for (int w = 0; w < PG_WAVES; ++w) mx = fmaxf(mx, m[w] = lds.m[w][h]);
        const float base = mx > -INFINITY ? mx : 0.f;
#pragma unroll
        for (int w = 0; w < PG_WAVES; ++w) {                // (a wavefront without rows has sums of zero)
            const float wt = __builtin_amdgcn_exp2f(m[w] - base);
            a = fmaf(lds.a[w][h][d], wt, a);
            ll = fmaf(lds.l[w][h], wt, ll);
        }
        f(h, d, a, mx, ll);
    }
}

// ---- where rows are --------------------------------------------------------------------------
// Rows of one KV head of one sequence. All rows of a pool are counted through, in 31 bits; a row without a page is number -1.
template <int DT>
struct PgRows {
    const char *k, *v;
    const int32_t* table;
    int page_log2, last, n_pages, n_kv, kv;

    __device__ __forceinline__ PgRows(const PgCache& c, int seq, int kv_head, int n_kv_heads)
        : k((const char*)c.k), v((const char*)c.v), table(c.table + (size_t)seq * c.table_stride), page_log2(c.page_log2), last(c.table_pages - 1),
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

// A chunk of rows whose numbers the lanes hold, row j that of lane j. Loads are not branched around: a row that is not there is row 0.
template <int DT>
__device__ __forceinline__ void pg_fetch(PgChunk<DT>& c, const PgRows<DT>& src, int number, int lane) {
    const int kg = lane >> 4, r = lane & 15;
    auto row = [](int n) { return (uint64_t)(uint32_t)(n < 0 ? 0 : n) * PG_ROW<DT>; };
    c.there = 0u;
#pragma unroll
    for (int t = 0; t < (DT == RA_BF16 ? 2 : 1); ++t) {
        const char* at = src.k + row(__shfl(number, 16 * t + r)) + 16 * kg;
#pragma unroll
        for (int i = 0; i < (DT == RA_BF16 ? 4 : 8); ++i) c.k[4 * t + i] = *reinterpret_cast<const pg_u32x4*>(at + 64 * i);
    }
#pragma unroll
    for (int j = 0; j < PG_CHUNK<DT> / 4; ++j) {
        const int n = __shfl(number, 16 * (j / 4) + 4 * kg + (j & 3));
        const char* at = src.v + row(n) + 16 * r;
        c.there |= (n >= 0 ? 1u : 0u) << j;
        if constexpr (DT == RA_BF16) c.v[j] = *reinterpret_cast<const pg_u32x4*>(at);
        else {
            c.v[2 * j] = *reinterpret_cast<const pg_u32x4*>(at);
            c.v[2 * j + 1] = *reinterpret_cast<const pg_u32x4*>(at + 256);
        }
    }
}

// ---- attention over all tokens -----------------------------------------------------------------
// The work is a list: per sequence, KV head and tile of its query heads (a job) the job's rows in units of 128 or, for lists that
// would be too long for 32 bits, a power of two of these. Workgroups
// take equal stretches of that list, whatever the lengths of the sequences are, and leave a record per job they touched, at place
// (workgroup + job): going along the list, one or the other grows by one at a time.
// Records lie per head of a tile, then place: sums [16][places][128], then maxima and sums of weights [16][places][2], so that
// what is combined lies in a row.
// A launch of as many workgroups as jobs (`whole`) gives each its job, and the workgroup writes the result.
#define PG_UNIT 128
#define PG_MOST_UNITS (1u << 21)    // times the workgroups, below 2^32

template <int DT>
__global__ __launch_bounds__(PG_THREADS, 2) void pg_full_kernel(const void* __restrict__ q, PgCache c, int n_seq, int n_q, int n_kv, int N,
                                                                const int32_t* __restrict__ n_tokens, int tiles, int unit_log2, int whole,
                                                                float* __restrict__ partials, float* __restrict__ out, float* __restrict__ lse) {
    __shared__ PgLds lds;
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
        const PgRows<DT> src(c, seq, job / tiles, n_kv);
        PgWave<DT> s;
        s.start(reinterpret_cast<const char*>(q) + head0 * PG_ROW<DT>, heads, lane);
        for (int row = from + wv * PG_CHUNK<DT>; row < to; row += PG_WAVES * PG_CHUNK<DT>) {
            const int mine = row + (lane & (PG_CHUNK<DT> - 1));
            PgChunk<DT> a;
            pg_fetch(a, src, mine < to ? src.number(src.page_of(mine), mine) : -1, lane);
            s.add(a, lane);
        }
        const size_t places = (size_t)gridDim.x + (size_t)n_seq * jobs, place = (size_t)wg + (size_t)seq * jobs + job;
        pg_close(s, lds, heads, tid, [&](int hd, int d, float sum, float mx, float l) {
            if (!whole) {
                partials[(hd * places + place) * RA_D + d] = sum;
                if (d == 0) reinterpret_cast<float2*>(partials + PG_HEADS * places * RA_D)[hd * places + place] = make_float2(mx, l);
            } else {
                out[(head0 + hd) * RA_D + d] = mx > -INFINITY ? sum / l : 0.f;
                if (d == 0) lse[head0 + hd] = mx > -INFINITY ? mx * REC_LN2 + logf(l) : -INFINITY;
            }
        });
        if (whole) return;
        at += unit1 - unit0;
        if (at < end) __syncthreads();                       // (the next job's sums go through the same LDS)
    }
}

#define PG_MOST_ROWS (1 << 24)      // of one job that a workgroup takes alone
struct PgCut { int tiles, workgroups, unit_log2; bool whole; const char* refused; };       // refused: why, or null
static PgCut pg_cut(int n_seq, int n_q, int n_kv, int64_t N) {
    PgCut x;
    x.tiles = (int)(((int64_t)(n_q / n_kv) + PG_HEADS - 1) / PG_HEADS);
    const int64_t jobs = (int64_t)n_seq * n_kv * x.tiles;
    // (from PG_MOST_UNITS jobs on there is no list: its units, and the threads of the second kernel, 128 for each of up to 16 heads, fit 32 bits)
    x.whole = N <= 256 || (jobs >= PG_MOST_UNITS && N <= PG_MOST_ROWS);
    x.unit_log2 = 7;
    static_assert(PG_UNIT == 1 << 7, "rows of a unit");
    x.refused = x.whole && jobs >= 1 << 24 ? "too many heads for one launch: 2^24 tiles of up to 16 query heads"
                : !x.whole && jobs >= PG_MOST_UNITS ? "too many heads for one launch: 2^21 tiles of up to 16 query heads over more than 2^24 tokens" : nullptr;
    x.workgroups = (int)jobs;
    if (x.whole || x.refused) return x;
    auto units = [&] { return jobs * ((N + ((int64_t)1 << x.unit_log2) - 1) >> x.unit_log2); };
    while (units() > PG_MOST_UNITS) ++x.unit_log2;
    const int most = ROW_MOST_WORKGROUPS / 3 * 2;
    x.workgroups = (int)(units() < most ? units() : most);
    return x;
}

size_t ra_full_paged_partial_floats(int n_seq, int n_q, int n_kv, int64_t N) {
    const PgCut x = pg_cut(n_seq, n_q, n_kv, N);
    return x.whole || x.refused ? 0 : ((size_t)x.workgroups + (size_t)n_seq * n_kv * x.tiles) * PG_HEADS * (RA_D + 2);
}

ra_status ra_launch_full_paged(const void* q, ra_dtype dt, const PgCache& c, int n_seq, int n_q, int n_kv, int64_t N, const int32_t* n_tokens,
                               float* partials, hipStream_t st, float* out, float* lse) {
    const PgCut x = pg_cut(n_seq, n_q, n_kv, N);
    if (x.refused) RA_FAIL(RA_EUNSUP, "%s", x.refused);
#define PG_GO(DTV)                                                                                                                        \
    hipLaunchKernelGGL((pg_full_kernel<DTV>), dim3(x.workgroups), dim3(PG_THREADS), 0, st, q, c, n_seq, n_q, n_kv, (int)N, n_tokens, x.tiles, \
                       x.unit_log2, (int)x.whole, partials, out, lse)
    if (dt == RA_BF16) PG_GO(RA_BF16); else PG_GO(RA_F32);
#undef PG_GO
    RA_HIP(hipGetLastError());
    if (x.whole) return RA_OK;
    return ra_launch_full_merge(partials, n_seq, n_q, n_kv, N, n_tokens, x.tiles, x.unit_log2, PG_HEADS, x.workgroups, st, out, lse);
}

// ---- the retrieved set and the static set -------------------------------------------------------
// W of a sequence, [0, s) u [w, n); ranges that meet make everything static. The host knows neither n nor how many tokens came after
// the index was built, so it fixes the number of W's parts, and what each of them takes is worked out here.
struct PgSets {
    int n, s, w, count, span, parts;        // rows of W, of a part of it, and parts that have rows
};
__device__ __forceinline__ PgSets pg_sets(const int32_t* n_tokens, const int32_t* n_indexed, int seq, int N, int sink, int window, int nS) {
    PgSets x;
    x.n = seq_rows(n_tokens, seq, N);
    const int indexed = n_indexed ? seq_rows(n_indexed, seq, x.n) : x.n;
    x.s = sink < x.n ? sink : x.n;
    const int w = window < x.n ? x.n - window : 0, late = w < indexed ? w : indexed;
    x.w = late > x.s ? late : x.s;
    x.count = x.s + x.n - x.w;
    const int least = nS > 0 ? (x.count + nS - 1) / nS : 0;
    x.span = least < PG_PART ? PG_PART : (least + PG_PART - 1) / PG_PART * PG_PART;
    x.parts = (x.count + x.span - 1) / x.span;
    return x;
}

// grid: per (sequence, KV head) the parts of each of its query heads' Omega (their loads wait for ids, so they start first), then
// the parts of the static set per tile of heads.
template <int DT>
__global__ __launch_bounds__(PG_THREADS, 2) void pg_attend_kernel(const void* __restrict__ q, PgCache c, int n_q, int n_kv, int N,
                                                                  const int32_t* __restrict__ n_tokens, const int32_t* __restrict__ n_indexed,
                                                                  int sink, int window, int topk, const int32_t* __restrict__ ids, int nS, int nG,
                                                                  int spanG, int tiles, float* __restrict__ partials) {
    __shared__ PgLds lds;
    const int tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid / RA_WAVE);
    const int group = n_q / n_kv, per = tiles * nS + group * nG, P = nS + nG;
    const int kv_head = blockIdx.x / per, x = blockIdx.x % per, seq = kv_head / n_kv;
    const bool om = x < group * nG;
    const int first = om ? x / nG : (x - group * nG) / nS * PG_HEADS;        // of the group's heads
    const int part = om ? x % nG : (x - group * nG) % nS, slot = om ? nS + part : part;
    const int heads = om ? 1 : group - first < PG_HEADS ? group - first : PG_HEADS;
    const size_t head0 = (size_t)seq * n_q + (size_t)(kv_head % n_kv) * group + first;
    const PgSets set = pg_sets(n_tokens, n_indexed, seq, N, sink, window, nS);
    if (!om && part >= set.parts) return;
    const PgRows<DT> src(c, seq, kv_head % n_kv, n_kv);
    const int count = om ? topk : set.count, span = om ? spanG : set.span, from = part * span, to = from + span < count ? from + span : count;
    const int32_t* list = ids + head0 * topk;
    PgWave<DT> st;
    st.start(reinterpret_cast<const char*>(q) + head0 * PG_ROW<DT>, heads, lane);
    for (int at = from + wv * PG_CHUNK<DT>; at < to; at += PG_WAVES * PG_CHUNK<DT>) {
        const int mine = at + (lane & (PG_CHUNK<DT> - 1)), j = mine < to ? mine : to - 1;
        int row = om ? list[j] : j < set.s ? j : set.w - set.s + j;
        bool is = mine < to;
        if (om) {
            is = is && row >= set.s && row < set.w;          // (members of W are attended there)
            row = is ? row : 0;
        }
        const int number = src.number(src.page_of(row), row);
        PgChunk<DT> a;
        pg_fetch(a, src, is ? number : -1, lane);
        st.add(a, lane);
    }
    pg_close(st, lds, heads, tid, [&](int hd, int d, float sum, float mx, float l) {
        float* rec = partials + ((head0 + hd) * P + slot) * REC_FLOATS;
        rec[d] = sum;
        if (d == 0) { rec[RA_D] = mx; rec[RA_D + 1] = l; }
    });
}

// grid: x = head (with its sequence); SLICES threads per dimension take the records in turn
template <int SLICES>
__global__ __launch_bounds__(RA_D * SLICES) void pg_merge_kernel(const float* __restrict__ partials, int n_q, int N, const int32_t* __restrict__ n_tokens,
                                                                 const int32_t* __restrict__ n_indexed, int sink, int window, int nS, int nG, SetOut o) {
    const size_t head = blockIdx.x;
    const float* rec = partials + head * (nS + nG) * REC_FLOATS;
    const int d = threadIdx.x % RA_D, slice = threadIdx.x / RA_D;
    const int have = pg_sets(n_tokens, n_indexed, (int)(head / n_q), N, sink, window, nS).parts;
    RecSum set[2] = {rec_add_up<false>(rec, slice, have, SLICES, d), rec_add_up<false>(rec, nS + slice, nS + nG, SLICES, d)};
    if constexpr (SLICES > 1) {
        __shared__ RecSum s_part[SLICES][2][RA_D];
        s_part[slice][0][d] = set[0];
        s_part[slice][1][d] = set[1];
        __syncthreads();
        if (slice) return;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            RecSum x{-INFINITY, 0.f, 0.f};
#pragma unroll
            for (int y = 0; y < SLICES; ++y) x.m = fmaxf(x.m, s_part[y][i][d].m);
            const float base = x.m > -INFINITY ? x.m : 0.f;
#pragma unroll
            for (int y = 0; y < SLICES; ++y) {
                const float w = __builtin_amdgcn_exp2f(s_part[y][i][d].m - base);
                x.a = fmaf(s_part[y][i][d].a, w, x.a);
                x.l = fmaf(s_part[y][i][d].l, w, x.l);
            }
            set[i] = x;
        }
    }
    rec_write(set, head, d, o);
}

// parts of the two sets: 128 rows each, a chunk for each wavefront of a workgroup; longer ones where they would be very many
struct PgParts { int nS, nG, spanG, tiles; };
static PgParts pg_parts(int n_seq, int n_q, int n_kv, int64_t most_static, int topk) {
    PgParts p;
    p.tiles = (n_q / n_kv + PG_HEADS - 1) / PG_HEADS;
    p.spanG = PG_PART;
    while (p.spanG < topk && (int64_t)n_seq * n_q * ((topk + p.spanG - 1) / p.spanG) > 2048) p.spanG *= 2;
    p.nG = (topk + p.spanG - 1) / p.spanG;
    const int64_t jobs = (int64_t)n_seq * n_kv * p.tiles, rest = (512 - (int64_t)n_seq * n_q * p.nG) / jobs;
    int64_t most = rest >= 1 && rest < 512 / jobs ? rest : 512 / jobs, nS = (most_static + PG_PART - 1) / PG_PART;
    if (most < 1) most = 1;
    p.nS = (int)(nS > most ? most : nS);
    return p;
}
// the most rows W can have
static int64_t pg_most_static(int64_t N, bool grows, int sink, int window) {
    const int64_t both = (int64_t)sink + window;
    return grows || both > N ? N : both;
}

size_t ra_attend_paged_partial_floats(int n_seq, int n_q, int n_kv, int64_t N, bool grows, int sink, int window, int topk) {
    const PgParts p = pg_parts(n_seq, n_q, n_kv, pg_most_static(N, grows, sink, window), topk);
    return (size_t)n_seq * n_q * (p.nS + p.nG) * REC_FLOATS;
}

ra_status ra_launch_attend_paged(const void* q, ra_dtype dt, const PgCache& c, int n_seq, int n_q, int n_kv, int64_t N, const int32_t* n_tokens,
                                 const int32_t* n_indexed, int sink, int window, int topk, const int32_t* ids, float* partials, hipStream_t st,
                                 float* out, float* lse, float* o_omega, float* lse_omega, float* o_w, float* lse_w) {
    const PgParts p = pg_parts(n_seq, n_q, n_kv, pg_most_static(N, n_indexed != nullptr, sink, window), topk);
    const int64_t blocks = (int64_t)n_seq * n_kv * ((int64_t)p.tiles * p.nS + (int64_t)(n_q / n_kv) * p.nG);
    if (blocks > (1 << 24) - 1) RA_FAIL(RA_EUNSUP, "too many heads for one launch");
    const SetOut o{nullptr, out, lse, o_omega, lse_omega, o_w, lse_w};
#define PG_GO(DTV)                                                                                                                               \
    hipLaunchKernelGGL((pg_attend_kernel<DTV>), dim3((unsigned)blocks), dim3(PG_THREADS), 0, st, q, c, n_q, n_kv, (int)N, n_tokens, n_indexed, sink, \
                       window, topk, ids, p.nS, p.nG, p.spanG, p.tiles, partials)
    if (dt == RA_BF16) PG_GO(RA_BF16); else PG_GO(RA_F32);
#undef PG_GO
    RA_HIP(hipGetLastError());
#define PG_MERGE(SLICES)                                                                                                                         \
    hipLaunchKernelGGL(pg_merge_kernel<SLICES>, dim3(n_seq * n_q), dim3(RA_D * SLICES), 0, st, partials, n_q, (int)N, n_tokens, n_indexed, sink, \
                       window, p.nS, p.nG, o)
    if ((p.nS + 7) / 8 + (p.nG + 7) / 8 <= 3) PG_MERGE(1); else PG_MERGE(8);
#undef PG_MERGE
    RA_HIP(hipGetLastError());
    return RA_OK;
}

// ---- rows side by side ------------------------------------------------------------------------
// A group of lanes takes FLY rows, 16 bytes a lane, whose table entries are all on their way before the first is used, and then the rows.
template <int DT, int FLY>
__global__ __launch_bounds__(PG_THREADS) void pg_gather_kernel(const char* __restrict__ pages, PgCache c, int n_kv, int64_t T, uint32_t blocks,
                                                               const int32_t* __restrict__ first, char* __restrict__ X) {
    constexpr int LANES = PG_ROW<DT> / 16, GROUPS = PG_THREADS / LANES;
    const int l = threadIdx.x % LANES;
    const uint32_t head = blockIdx.x / blocks, seq = head / n_kv;
    const int64_t t0 = (int64_t)(blockIdx.x % blocks) * (GROUPS * FLY) + threadIdx.x / LANES, at0 = first ? first[seq] : 0;
    const PgRows<DT> src(c, seq, head % n_kv, n_kv);
    const int64_t room = ((int64_t)src.last + 1) << src.page_log2;
    int number[FLY];
#pragma unroll
    for (int u = 0; u < FLY; ++u) {
        const int64_t at = at0 + t0 + GROUPS * u;
        const bool in = at >= 0 && at < room;
        const int row = in ? (int)at : 0, n = src.number(src.page_of(row), row);
        number[u] = in ? n : -1;
    }
    pg_u32x4 x[FLY];
#pragma unroll
    for (int u = 0; u < FLY; ++u)
        x[u] = *reinterpret_cast<const pg_u32x4*>(pages + (uint64_t)(uint32_t)(number[u] < 0 ? 0 : number[u]) * PG_ROW<DT> + 16 * l);
#pragma unroll
    for (int u = 0; u < FLY; ++u) {
        const int64_t t = t0 + GROUPS * u;
        if (t >= T) continue;
        if (number[u] < 0) x[u] = pg_u32x4{0u, 0u, 0u, 0u};
        *reinterpret_cast<pg_u32x4*>(X + ((uint64_t)head * T + t) * PG_ROW<DT> + 16 * l) = x[u];
    }
}

ra_status ra_launch_gather_paged(const PgCache& c, const void* pages, ra_dtype dt, int n_seq, int n_kv, int64_t T, const int32_t* first,
                                 hipStream_t st, void* X) {
    const int64_t heads = (int64_t)n_seq * n_kv;
    constexpr int FLY = 4;
    const int64_t rows = PG_THREADS * FLY * 16 / (dt == RA_BF16 ? PG_ROW<RA_BF16> : PG_ROW<RA_F32>), blocks = (T + rows - 1) / rows;
    if (heads * blocks > (1 << 24) - 1) RA_FAIL(RA_EUNSUP, "too many rows for one launch");
#define PG_GO(DTV)                                                                                                                         \
    hipLaunchKernelGGL((pg_gather_kernel<DTV, FLY>), dim3((unsigned)(heads * blocks)), dim3(PG_THREADS), 0, st, (const char*)pages, c, n_kv, T, \
                       (uint32_t)blocks, first, (char*)X)
    if (dt == RA_BF16) PG_GO(RA_BF16); else PG_GO(RA_F32);
#undef PG_GO
    RA_HIP(hipGetLastError());
    return RA_OK;
}
