// What the attention kernels over whole caches share (q4.hip, paged.hip): the list of rows that their workgroups take stretches of,
// and what becomes of the records of a head's two sets, Omega and W.
#pragma once
#include "common.h"

#define REC_FLOATS (RA_D + 4)           // floats of a record of a set's part: sums, maximum, sum of weights, 2 pad
// A record's maximum is in units whose multiple by `unit` is z log2(e): those of z log2(e) itself (1), or of the products <q, k>. What is combined takes
// differences of maxima first and then the multiple, so that in units of exact products equal logits have equal weights however large they are.
#define REC_LN2 0.6931471805599453f
#define ROW_LEAST_UNITS 2u           // units that are worth a workgroup
#define ROW_MOST_WORKGROUPS 768      // three per compute unit

// over the 64 lanes: the sum, in all of them, and the sums up to each
__device__ __forceinline__ uint32_t sum64(uint32_t x, int lane) {
    x += lane_xor32<1>(x, lane); x += lane_xor32<2>(x, lane); x += lane_xor32<4>(x, lane);
    x += lane_xor32<8>(x, lane); x += lane_xor32<16>(x, lane); x += lane_xor32<32>(x, lane);
    return (uint32_t)__builtin_amdgcn_readfirstlane((int)x);
}
__device__ __forceinline__ uint32_t scan64(uint32_t x) {
#define ROW_STEP(CTRL, ROWS) x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, ROWS, 0xF, ROWS == 0xF)
    ROW_STEP(0x111, 0xF); ROW_STEP(0x112, 0xF); ROW_STEP(0x114, 0xF); ROW_STEP(0x118, 0xF);     // within rows of 16
    ROW_STEP(0x142, 0xA); ROW_STEP(0x143, 0xC);           // the row before's last to every second row, then the half before's
#undef ROW_STEP
    return x;
}
struct RowList {
    uint32_t units, first;          // of the whole list; before a sequence's jobs
    int n;                          // rows of the sequence
    uint32_t workgroups;            // that have a stretch
    int rows;                       // rows of sequence `lane`

    __device__ __forceinline__ uint32_t from(uint32_t wg) const { return units * wg / workgroups; }
    __device__ __forceinline__ uint32_t owner(uint32_t unit) const { return ((unit + 1) * workgroups - 1) / units; }
};
__device__ __forceinline__ int seq_rows(const int32_t* n_tokens, int seq, int N) {
    const int n = n_tokens ? n_tokens[seq] : N;
    return n < 0 ? 0 : n < N ? n : N;
}
__device__ __forceinline__ uint32_t row_units(int rows, int unit_log2) { return ((uint32_t)rows + (1u << unit_log2) - 1u) >> unit_log2; }
// the list, and where sequence `seq`'s part of it begins; called by whole wavefronts, the same in all lanes
__device__ __forceinline__ RowList row_list(const int32_t* n_tokens, int n_seq, int seq, int N, int unit_log2, uint32_t jobs, uint32_t grid) {
    RowList x;
    x.rows = N;
    if (!n_tokens) {
        x.units = row_units(N, unit_log2) * n_seq * jobs;
        x.first = row_units(N, unit_log2) * seq * jobs;
        x.n = N;
    } else if (n_seq == 1) {        // (a scalar load, and nothing to add up)
        x.n = x.rows = seq_rows(n_tokens, 0, N);
        x.units = row_units(x.n, unit_log2) * jobs;
        x.first = 0;
    } else {
        uint32_t all = 0, before = 0, mine = 0;
        const int lane = threadIdx.x & 63;
        for (int s0 = 0; s0 < n_seq; s0 += RA_WAVE) {
            const int s = s0 + lane, rows = s < n_seq ? seq_rows(n_tokens, s, N) : 0;
            const uint32_t u = row_units(rows, unit_log2);
            if (s0 == 0) x.rows = rows;
            all += u;
            before += s < seq ? u : 0u;
            mine += s == seq ? (uint32_t)rows : 0u;
        }
        x.units = sum64(all, lane) * jobs;
        x.first = sum64(before, lane) * jobs;
        x.n = (int)sum64(mine, lane);
    }
    const uint32_t most = (x.units + ROW_LEAST_UNITS - 1u) / ROW_LEAST_UNITS;
    x.workgroups = most < grid ? most : grid;
    return x;
}
// the sequence that has unit `unit` (one of the list's), and where its part begins
__device__ __forceinline__ int row_seq_of(const RowList& x, const int32_t* n_tokens, int n_seq, int N, int unit_log2, uint32_t jobs,
                                         uint32_t unit, uint32_t* first) {
    if (n_seq == 1) {
        *first = 0;
        return 0;
    }
    if (!n_tokens) {
        const uint32_t per = row_units(N, unit_log2) * jobs, seq = unit / per;
        *first = seq * per;
        return (int)seq;
    }
    const int lane = threadIdx.x & 63;
    uint32_t at = 0;
    for (int s0 = 0;; s0 += RA_WAVE) {
        const int s = s0 + lane;
        const uint32_t u = row_units(s0 == 0 ? x.rows : s < n_seq ? seq_rows(n_tokens, s, N) : 0, unit_log2);
        const uint32_t upto = scan64(u);
        const unsigned long long past = __ballot(at + upto * jobs > unit);
        if (past != 0ull || s0 + RA_WAVE >= n_seq) {
            const int l = past != 0ull ? __ffsll(past) - 1 : 63;
            *first = at + (uint32_t)__builtin_amdgcn_readlane((int)(upto - u), l) * jobs;
            return s0 + l;
        }
        at += (uint32_t)__builtin_amdgcn_readlane((int)upto, 63) * jobs;
    }
}

// A head's records, those of a row of workgroups: their sums, their maxima and sums of weights, and how many.
struct FullRecords { const float* sums; const float2* ml; int have; };
__device__ __forceinline__ FullRecords full_records(const float* partials, size_t head, int n_seq, int n_q, int n_kv, int N,
                                                const int32_t* n_tokens, int tiles, int unit_log2, int heads, int grid) {
    const int seq = (int)(head / n_q), group = n_q / n_kv, h = (int)(head % n_q), jobs = n_kv * tiles;
    const int job = h / group * tiles + h % group / heads;
    const RowList x = row_list(n_tokens, n_seq, seq, N, unit_log2, jobs, grid);
    const uint32_t units = row_units(x.n, unit_log2);
    int have = 0, wg0 = 0;
    if (units) {
        const uint32_t unit0 = x.first + job * units;
        wg0 = (int)x.owner(unit0);
        have = (int)x.owner(unit0 + units - 1) - wg0 + 1;
    }
    const size_t places = (size_t)grid + (size_t)n_seq * jobs, at = h % group % heads * places + (size_t)wg0 + (size_t)seq * jobs + job;
    return {partials + at * RA_D, reinterpret_cast<const float2*>(partials + heads * places * RA_D) + at, have};
}

// ---- records of two sets ----------------------------------------------------------------
struct SetOut {
    uint32_t* tickets;                  // one word per query head (ticket.h), or null
    float *out, *lse, *o_om, *lse_om, *o_w, *lse_w;
};

template <bool COHERENT>
__device__ __forceinline__ void rec_put(float* p, float v) {
    if (COHERENT) __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    else *p = v;
}
template <bool COHERENT>
__device__ __forceinline__ float rec_get(const float* p) {
    return COHERENT ? __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : *p;
}

// Dimension d of a head's records [first, last), every `by`th: their maximum, sum of weights and weighted sum.
struct RecSum { float m, l, a; };
template <bool COHERENT>
__device__ __forceinline__ RecSum rec_add_up(const float* rec, int first, int last, int by, int d, float unit) {
    constexpr int FLY = 8;
    RecSum x{-INFINITY, 0.f, 0.f};
    for (int i0 = first; i0 < last; i0 += FLY * by) {
        float m[FLY], l[FLY], a[FLY], mx = x.m;
#pragma unroll
        for (int u = 0; u < FLY; ++u) {
            const float* y = rec + (size_t)(i0 + u * by < last ? i0 + u * by : i0) * REC_FLOATS;
            m[u] = rec_get<COHERENT>(y + RA_D);
            l[u] = rec_get<COHERENT>(y + RA_D + 1);
            a[u] = rec_get<COHERENT>(y + d);
        }
#pragma unroll
        for (int u = 0; u < FLY; ++u) mx = fmaxf(mx, m[u]);
        if (mx == -INFINITY) continue;
        const float corr = __builtin_amdgcn_exp2f((x.m - mx) * unit);
        x.a *= corr;
        x.l *= corr;
#pragma unroll
        for (int u = 0; u < FLY; ++u) {
            const bool is = i0 + u * by < last;             // (a trip that is not full reads its first record again, whose sum may be infinite)
            const float w = __builtin_amdgcn_exp2f((m[u] - mx) * unit);
            x.a = fmaf(is ? a[u] : 0.f, w, x.a);
            x.l = fmaf(is ? l[u] : 0.f, w, x.l);
        }
        x.m = mx;
    }
    return x;
}
// Eq. 4 for the static set and for Omega, Eq. 5 for both
__device__ __forceinline__ void rec_write(const RecSum (&set)[2], size_t head, int d, float unit, const SetOut& o) {
    float* o_set[2] = {o.o_w, o.o_om};
    float* l_set[2] = {o.lse_w, o.lse_om};
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const bool empty = set[i].m == -INFINITY;
        if (o_set[i]) o_set[i][head * RA_D + d] = empty ? 0.f : set[i].a / set[i].l;
        if (l_set[i] && d == 0) l_set[i][head] = empty ? -INFINITY : set[i].m * unit * REC_LN2 + logf(set[i].l);
    }
    const float mx = fmaxf(set[0].m, set[1].m);
    float out = 0.f, lse = -INFINITY;
    if (mx > -INFINITY) {
        const float e0 = __builtin_amdgcn_exp2f((set[0].m - mx) * unit), e1 = __builtin_amdgcn_exp2f((set[1].m - mx) * unit);
        const float l = set[0].l * e0 + set[1].l * e1;
        out = (set[0].a * e0 + set[1].a * e1) / l;
        lse = mx * unit * REC_LN2 + logf(l);
    }
    o.out[head * RA_D + d] = out;
    if (d == 0) o.lse[head] = lse;
}
// dimension d of a head from its records, nS of the static set and nG of Omega
template <bool COHERENT>
__device__ __forceinline__ void rec_finish(const float* rec, int nS, int nG, size_t head, int d, float unit, const SetOut& o) {
    const RecSum set[2] = {rec_add_up<COHERENT>(rec, 0, nS, 1, d, unit), rec_add_up<COHERENT>(rec, nS, nS + nG, 1, d, unit)};
    rec_write(set, head, d, unit, o);
}
