// Attention over a cache in 4 bits: all tokens (ra_full_attention_q4), and the retrieved set Omega and the static set W of
// Sec. 3.3 with their combination by Eq. 4-5 (ra_attend_q4).
//
// Rows are cut into parts; a workgroup turns one part into a record (128 weighted sums, the running maximum of
// z log2(e), the sum of weights), and a head's records are combined by a second kernel or by whoever stores the last. Weights are powers of two,
// p = 2^(c <q, k> - m) with c = log2(e) / sqrt(d): one multiply-add and one instruction each.
#include "q4_dev.h"
#include "ticket.h"

#define Q4_THREADS 256
#define Q4_REC (RA_D + 4)           // floats of a record: sums, maximum, sum of weights, 2 pad
#define Q4_PART 128                 // rows of a part of the sparse set
#define Q4_C ((float)(1.4426950408889634 / 11.313708498984761))
#define Q4_LN2 0.6931471805599453f

// ---- chunks of 32 rows on the matrix cores ---------------------------------------------------
// A wavefront takes 32 rows at a time for a tile of query heads of one KV head, two products of v_mfma_f32_16x16x32_bf16
// with nothing in between but registers:
//   logits  S[row][column] = <k_row, q_column>. Lane (kg, r) = (lane / 16, lane % 16) holds 32 dimensions of key r of each half of
//           the chunk: 16 bytes of codes, one block, one scale. The four instructions of a half take 8 of them each, in whatever
//           order as long as the query's lanes have the same. Lane (kg, c) ends with rows 4 kg + i of column c.
//   sums    O[dimension][column] += V^T P. The lane's weights of the two halves are 8 consecutive slots of the contraction, so
//           they go in as they come out; V^T wants for them, per dimension, the same 8 rows. Lane (kg, r) reads codes 8 r .. 8 r + 7 of
//           these rows, four bytes each (16 lanes read a row): instruction m takes the m-th of each, dimension 8 r + m.
// Codes become bfloat16 exactly. A float32 weight goes in as three terms of bfloat16, the first as rounded, the next what the rounding
// left, an instruction for each: all of its 24 bits. Two (16 bits) are not enough: with a flat softmax (logits of deviation 1, bfloat16 queries) outputs
// over 200, 2000 and 131072 tokens were 1.6, 1.8 and 2.2e-6 off (2-norm), with three 0.15, 0.18 and 0.50e-6; with logits of deviation 5, 0.42, 0.18
// and 0.24e-6 and now 0.11, 0.18 and 0.21e-6; a sparse set, a few rows with all the weight, up to 1.2e-6 and now 0.2e-6. The third costs 2 to 4 % over all
// tokens (131072 of 8 heads, 32 query heads, 31.8 -> 32.9 us, 16 sequences of up to 32768 61.6 -> 63.3), where 16 query heads share a KV head 7 % (a million tokens
// 33.7 -> 36.0), and 2 % for a sparse set. Float32 queries are three terms too. The sum of the weights is that of the terms (an
// instruction with a row of ones), so that what their rounding does to a weight that has nearly everything cancels.
// Columns are heads, HEADS of them; where that is 8 or 4, two or four groups of columns have the same heads, and a lane makes the weights of
// half or a quarter of its rows only (the others are zero): exponentials and splits are what vector instructions are short of,
// not matrix instructions. Every column has a maximum and sums of its own; they are put together at the end.
// The running maximum of a column moves only when a logit exceeds it by more than 8 (in powers of two), which keeps the
// lanes' exchange and the scaling of sums out of nearly every chunk.
typedef __bf16 q4_bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 q4_bf16x8 __attribute__((ext_vector_type(8)));
typedef float q4_f32x4 __attribute__((ext_vector_type(4)));
#define Q4_CHUNK 32
#define Q4_LOWEST (-1.7e38f)        // below every logit: a maximum that nothing has moved yet

struct Q4Chunk {
    uint4 k[2];
    uint32_t ks[2], v[8], vs[8];
};

template <int DT, int HEADS>
struct Q4Wave {
    static constexpr int TERMS = 3, QTERMS = DT == RA_BF16 ? 1 : 3;        // of weights and of queries
    static constexpr int SHARES = 16 / HEADS, MINE = 8 / SHARES;        // groups of columns; rows of a lane's 8 that are its own
    q4_bf16x8 q[QTERMS][4];
    q4_f32x4 acc[8], sum;       // weighted sums, and the sum of the weights as they went in, the same in all rows
    float m;
    uint32_t turn;              // by how much a word of four scale bytes turns for the lane's to lie at the exponent

    // queries of heads 0 .. n - 1 of a tile, 128 values each; columns past them are the first one's, and nobody asks for them
    __device__ __forceinline__ void start(const void* q0, int n, int lane) {
        const int kg = lane >> 4, h = (lane & 15) % HEADS;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const size_t at = (size_t)(h < n ? h : 0) * RA_D + 32 * kg + 8 * i;
            if constexpr (DT == RA_BF16) {
                q[0][i] = __builtin_bit_cast(q4_bf16x8, *reinterpret_cast<const uint4*>(reinterpret_cast<const uint16_t*>(q0) + at));
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    float x = reinterpret_cast<const float*>(q0)[at + e];
#pragma unroll
                    for (int t = 0; t < QTERMS; ++t) {
                        q[t][i][e] = (__bf16)x;
                        x -= (float)q[t][i][e];
                    }
                }
            }
        }
#pragma unroll
        for (int d = 0; d < 8; ++d) acc[d] = q4_f32x4{0.f, 0.f, 0.f, 0.f};
        sum = q4_f32x4{0.f, 0.f, 0.f, 0.f};
        m = Q4_LOWEST;
        turn = (8 * ((lane & 15) / 4) + 9) & 31;
    }

    // `there`: bit j says whether the lane's row j is one (rows 4 kg + j of the first half, j < 4, then of the second); ALL: all are
    template <bool ALL>
    __device__ __forceinline__ void add(const Q4Chunk& c, uint32_t there, int lane) {
        // (the lesser terms of a float32 query have a sum of their own, so that the first one's is rounded four times, not twelve)
        q4_f32x4 S[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}}, less[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const float unit = q4_unit(c.ks[t]);
            const uint32_t w[4] = {c.k[t].x, c.k[t].y, c.k[t].z, c.k[t].w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                uint4 b;
                b.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[i], unit, 0));
                b.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[i], unit, 1));
                b.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[i], unit, 2));
                b.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[i], unit, 3));
#pragma unroll
                for (int x = QTERMS - 1; x >= 1; --x)
                    less[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(q4_bf16x8, b), q[x][i], less[t], 0, 0, 0);
                S[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(q4_bf16x8, b), q[0][i], S[t], 0, 0, 0);
            }
            if (QTERMS > 1) S[t] += less[t];
        }
        // the lane's own rows: MINE from g MINE on
        const int g = (lane & 15) / HEADS;
        float z[MINE], top = Q4_LOWEST;
#pragma unroll
        for (int j = 0; j < MINE; ++j) {
            z[j] = S[j / 4][j & 3];
            if (SHARES == 2) z[j] = g ? S[1][j & 3] : z[j];
            if (SHARES == 4) {
                z[j] = g & 1 ? S[0][2 + (j & 1)] : z[j];
                const float far = g & 1 ? S[1][2 + (j & 1)] : S[1][j & 1];
                z[j] = g & 2 ? far : z[j];
            }
            if (!ALL) z[j] = (there >> (g * MINE + j)) & 1u ? z[j] : -INFINITY;
            top = fmaxf(top, z[j]);
        }
        if (__builtin_amdgcn_ballot_w64(top * Q4_C > m + 8.f) != 0ull) {
            top = fmaxf(top, __uint_as_float(lane_xor32<16>(__float_as_uint(top), lane)));
            top = fmaxf(top, __uint_as_float(lane_xor32<32>(__float_as_uint(top), lane)));
            const float now = fmaxf(m, top * Q4_C), corr = __builtin_amdgcn_exp2f(m - now);
            m = now;
            sum *= corr;
#pragma unroll
            for (int d = 0; d < 8; ++d) acc[d] *= corr;
        }
        q4_bf16x8 P[TERMS];
        {
            float x[MINE];
#pragma unroll
            for (int j = 0; j < MINE; ++j) x[j] = __builtin_amdgcn_exp2f(fmaf(z[j], Q4_C, -m));
#pragma unroll
            for (int t = 0; t < TERMS; ++t) {
                uint32_t pair[MINE / 2], w[4];
#pragma unroll
                for (int j = 0; j < MINE / 2; ++j) {
                    const q4_bf16x2 b = {(__bf16)x[2 * j], (__bf16)x[2 * j + 1]};
                    pair[j] = __builtin_bit_cast(uint32_t, b);
                    if (t + 1 < TERMS) { x[2 * j] -= bf16_lo(pair[j]); x[2 * j + 1] -= bf16_hi(pair[j]); }
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) w[i] = SHARES == 1 || g == i / (MINE / 2) ? pair[i % (MINE / 2)] : 0u;
                P[t] = __builtin_bit_cast(q4_bf16x8, make_uint4(w[0], w[1], w[2], w[3]));
            }
        }
        const q4_bf16x8 ones = __builtin_bit_cast(q4_bf16x8, make_uint4(0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u));
#pragma unroll
        for (int t = TERMS - 1; t >= 0; --t) sum = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, P[t], sum, 0, 0, 0);
        float unit[8];                                       // the scale byte of the lane's block, where its exponent goes
        uint32_t w[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            unit[j] = __uint_as_float(__builtin_amdgcn_alignbit(c.vs[j], c.vs[j], turn));
            w[j] = c.v[j];
            if (!ALL) {                                      // (0 * NaN is not 0)
                const bool have = (there >> j) & 1u;
                unit[j] = have ? unit[j] : 1.f;
                w[j] = have ? w[j] : 0u;
            }
        }
        sums<0>(w, unit, P);
        sums<1>(w, unit, P);
        sums<2>(w, unit, P);
        sums<3>(w, unit, P);
    }
    // dimensions 2 Y and 2 Y + 1 of the lane's 8, which share a byte of every row's codes
    template <int Y>
    __device__ __forceinline__ void sums(const uint32_t (&w)[8], const float (&unit)[8], const q4_bf16x8 (&P)[TERMS]) {
        uint32_t p[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) p[j] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[j], unit[j], Y));
#pragma unroll
        for (int o = 0; o < 2; ++o) {
            const uint32_t half = o ? 0x07060302u : 0x05040100u;
            uint4 a;
            a.x = __builtin_amdgcn_perm(p[1], p[0], half);
            a.y = __builtin_amdgcn_perm(p[3], p[2], half);
            a.z = __builtin_amdgcn_perm(p[5], p[4], half);
            a.w = __builtin_amdgcn_perm(p[7], p[6], half);
#pragma unroll
            for (int t = TERMS - 1; t >= 0; --t)
                acc[2 * Y + o] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(q4_bf16x8, a), P[t], acc[2 * Y + o], 0, 0, 0);
        }
    }
};

// Rows of one head from `first` on, read through buffer descriptors: a lane's places in a chunk never change, and what moves
// from chunk to chunk is one scalar, so that no vector instruction is spent on addresses. Codes of keys are non-temporal: of a
// cache that is read again before long, or is larger than what the memory side keeps, the values' half stays (three caches of 131072 rows
// in turn 37.9 -> 33.1 us a call, of 303 MB 63.2 -> 61.5; both halves 35.5 and 59.6).
#define Q4_RSRC 0x00020000          // raw buffer, no format
#define Q4_NT 2                     // non-temporal
struct Q4Stream {
    __amdgpu_buffer_rsrc_t k, ks, v, vs;
    int at_k, at_ks, at_v, at_vs;

    __device__ __forceinline__ void start(const Q4Cache& h, int64_t first, int64_t rows, int lane) {
        const int kg = lane >> 4, r = lane & 15;
        auto rsrc = [&](const uint8_t* p, int row) {
            return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(p) + first * row, 0, (int)(rows * row), Q4_RSRC);
        };
        k = rsrc(h.k, Q4_ROW); ks = rsrc(h.ks, Q4_BLOCKS); v = rsrc(h.v, Q4_ROW); vs = rsrc(h.vs, Q4_BLOCKS);
        at_k = r * Q4_ROW + 16 * kg; at_ks = r * Q4_BLOCKS + kg; at_v = 4 * kg * Q4_ROW + 4 * r; at_vs = 4 * kg * Q4_BLOCKS;
    }
    // rows [row, row + 32), all of which there are; `row` is the same in all lanes
    __device__ __forceinline__ void fetch(Q4Chunk& c, int row) const {
        const int by = row * Q4_ROW, bys = row * Q4_BLOCKS;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            c.k[t] = __builtin_bit_cast(uint4, __builtin_amdgcn_raw_buffer_load_b128(k, at_k, by + 16 * t * Q4_ROW, Q4_NT));
            c.ks[t] = __builtin_amdgcn_raw_buffer_load_b8(ks, at_ks, bys + 16 * t * Q4_BLOCKS, 0);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j)
            c.v[j] = __builtin_amdgcn_raw_buffer_load_b32(v, at_v, by + ((j & 4) * 4 + (j & 3)) * Q4_ROW, 0);
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const uint4 w = __builtin_bit_cast(uint4, __builtin_amdgcn_raw_buffer_load_b128(vs, at_vs, bys + 16 * t * Q4_BLOCKS, 0));
            c.vs[4 * t] = w.x; c.vs[4 * t + 1] = w.y; c.vs[4 * t + 2] = w.z; c.vs[4 * t + 3] = w.w;
        }
    }
};
// rows [from, from + 32) of a head; past the last row, n - 1, that one
__device__ __forceinline__ void q4_fetch_last(Q4Chunk& c, const Q4Cache& h, int64_t from, int64_t n, int lane) {
    const int kg = lane >> 4, r = lane & 15, last = (int)(n - 1 - from);
    const uint8_t *k = h.k + from * Q4_ROW, *ks = h.ks + from * Q4_BLOCKS, *v = h.v + from * Q4_ROW, *vs = h.vs + from * Q4_BLOCKS;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        const int row = min(16 * t + r, last);
        c.k[t] = *reinterpret_cast<const uint4*>(k + row * Q4_ROW + 16 * kg);
        c.ks[t] = ks[row * Q4_BLOCKS + kg];
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int row = min((j & 4) * 4 + 4 * kg + (j & 3), last);
        c.v[j] = *reinterpret_cast<const uint32_t*>(v + row * Q4_ROW + 4 * r);
        c.vs[j] = *reinterpret_cast<const uint32_t*>(vs + row * Q4_BLOCKS);
    }
}
// which of the lane's rows of [from, from + 32) are below n
__device__ __forceinline__ uint32_t q4_there(int64_t from, int64_t n, int lane) {
    uint32_t there = 0u;
#pragma unroll
    for (int j = 0; j < 8; ++j) there |= (from + (j & 4) * 4 + 4 * (lane >> 4) + (j & 3) < n ? 1u : 0u) << j;
    return there;
}

#define Q4_WAVES (Q4_THREADS / RA_WAVE)
#define Q4_PAD (RA_D + 4)
struct Q4Lds { float a[Q4_WAVES][16][Q4_PAD], m[Q4_WAVES][16], l[Q4_WAVES][16]; };

// The states of the wavefronts' columns -> one per head: f(head of the tile, dimension, sum, maximum, sum of weights), called by
// one thread for each; a head without rows has the maximum -infinity.
template <int DT, int HEADS, class Fn>
__device__ __forceinline__ void q4_close(Q4Wave<DT, HEADS>& s, Q4Lds& lds, int n, int tid, Fn f) {
    constexpr int SHARES = 16 / HEADS;
    const int wv = tid / RA_WAVE, lane = tid & 63, kg = lane >> 4, col = lane & 15;
    const float l = s.sum[0];
    // a sum that is not a number keeps a maximum that is one, or it would count as empty
    if (kg == 0) {
        lds.m[wv][col] = l != l ? 0.f : l > 0.f ? s.m : -INFINITY;
        lds.l[wv][col] = l;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float* to = &lds.a[wv][col][8 * (4 * kg + i)];
        *reinterpret_cast<float4*>(to) = make_float4(s.acc[0][i], s.acc[1][i], s.acc[2][i], s.acc[3][i]);
        *reinterpret_cast<float4*>(to + 4) = make_float4(s.acc[4][i], s.acc[5][i], s.acc[6][i], s.acc[7][i]);
    }
    __syncthreads();
    for (int x = tid; x < n * RA_D; x += Q4_THREADS) {
        const int h = x / RA_D, d = x % RA_D;
        float m[Q4_WAVES][SHARES], mx = -INFINITY, a = 0.f, ll = 0.f;
#pragma unroll
        for (int w = 0; w < Q4_WAVES; ++w)
#pragma unroll
            for (int g = 0; g < SHARES; ++g) mx = fmaxf(mx, m[w][g] = lds.m[w][g * HEADS + h]);
        const float base = mx > -INFINITY ? mx : 0.f;
#pragma unroll
        for (int w = 0; w < Q4_WAVES; ++w)
#pragma unroll
            for (int g = 0; g < SHARES; ++g) {              // (a column without rows has sums of zero)
                const float wt = __builtin_amdgcn_exp2f(m[w][g] - base);
                a = fmaf(lds.a[w][g * HEADS + h][d], wt, a);
                ll = fmaf(lds.l[w][g * HEADS + h], wt, ll);
            }
        f(h, d, a, mx, ll);
    }
}

// Attention over all tokens. The work is a list: per sequence, KV head and tile of its query heads (a job) the job's rows in units of
// 128 (a chunk for each wavefront of a workgroup) or, for lists that would be too long for 32 bits, a power of two of these. Workgroups
// take equal stretches of that list, whatever the lengths of the sequences are, and leave a record per job they touched, at place
// (workgroup + job): going along the list, one or the other grows by one at a time.
// Records lie per head of a tile, then place: sums [HEADS][places][128], then maxima and sums of weights [HEADS][places][2], so that
// what is combined lies in a row.
// A launch of as many workgroups as jobs (`whole`) gives each its job, and the workgroup writes the result.
#define Q4_UNIT (Q4_WAVES * Q4_CHUNK)
#define Q4_MOST_UNITS (1u << 21)    // times the workgroups, below 2^32
#define Q4_LEAST_UNITS 2u           // units that are worth a workgroup
#define Q4_MOST_WORKGROUPS 768      // three per compute unit
// over the 64 lanes: the sum, in all of them, and the sums up to each
__device__ __forceinline__ uint32_t q4_sum64(uint32_t x, int lane) {
    x += lane_xor32<1>(x, lane); x += lane_xor32<2>(x, lane); x += lane_xor32<4>(x, lane);
    x += lane_xor32<8>(x, lane); x += lane_xor32<16>(x, lane); x += lane_xor32<32>(x, lane);
    return (uint32_t)__builtin_amdgcn_readfirstlane((int)x);
}
__device__ __forceinline__ uint32_t q4_scan64(uint32_t x) {
#define Q4_STEP(CTRL, ROWS) x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, ROWS, 0xF, ROWS == 0xF)
    Q4_STEP(0x111, 0xF); Q4_STEP(0x112, 0xF); Q4_STEP(0x114, 0xF); Q4_STEP(0x118, 0xF);     // within rows of 16
    Q4_STEP(0x142, 0xA); Q4_STEP(0x143, 0xC);           // the row before's last to every second row, then the half before's
#undef Q4_STEP
    return x;
}
struct Q4List {
    uint32_t units, first;          // of the whole list; before a sequence's jobs
    int n;                          // rows of the sequence
    uint32_t workgroups;            // that have a stretch
    int rows;                       // rows of sequence `lane`

    __device__ __forceinline__ uint32_t from(uint32_t wg) const { return units * wg / workgroups; }
    __device__ __forceinline__ uint32_t owner(uint32_t unit) const { return ((unit + 1) * workgroups - 1) / units; }
};
__device__ __forceinline__ int q4_rows_of(const int32_t* n_tokens, int seq, int N) {
    const int n = n_tokens ? n_tokens[seq] : N;
    return n < 0 ? 0 : n < N ? n : N;
}
__device__ __forceinline__ uint32_t q4_units(int rows, int unit_log2) { return ((uint32_t)rows + (1u << unit_log2) - 1u) >> unit_log2; }
// the list, and where sequence `seq`'s part of it begins; called by whole wavefronts, the same in all lanes
__device__ __forceinline__ Q4List q4_list(const int32_t* n_tokens, int n_seq, int seq, int N, int unit_log2, uint32_t jobs, uint32_t grid) {
    Q4List x;
    x.rows = N;
    if (!n_tokens) {
        x.units = q4_units(N, unit_log2) * n_seq * jobs;
        x.first = q4_units(N, unit_log2) * seq * jobs;
        x.n = N;
    } else if (n_seq == 1) {        // (a scalar load, and nothing to add up)
        x.n = x.rows = q4_rows_of(n_tokens, 0, N);
        x.units = q4_units(x.n, unit_log2) * jobs;
        x.first = 0;
    } else {
        uint32_t all = 0, before = 0, mine = 0;
        const int lane = threadIdx.x & 63;
        for (int s0 = 0; s0 < n_seq; s0 += RA_WAVE) {
            const int s = s0 + lane, rows = s < n_seq ? q4_rows_of(n_tokens, s, N) : 0;
            const uint32_t u = q4_units(rows, unit_log2);
            if (s0 == 0) x.rows = rows;
            all += u;
            before += s < seq ? u : 0u;
            mine += s == seq ? (uint32_t)rows : 0u;
        }
        x.units = q4_sum64(all, lane) * jobs;
        x.first = q4_sum64(before, lane) * jobs;
        x.n = (int)q4_sum64(mine, lane);
    }
    const uint32_t most = (x.units + Q4_LEAST_UNITS - 1u) / Q4_LEAST_UNITS;
    x.workgroups = most < grid ? most : grid;
    return x;
}
// the sequence that has unit `unit` (one of the list's), and where its part begins
__device__ __forceinline__ int q4_seq_of(const Q4List& x, const int32_t* n_tokens, int n_seq, int N, int unit_log2, uint32_t jobs,
                                         uint32_t unit, uint32_t* first) {
    if (n_seq == 1) {
        *first = 0;
        return 0;
    }
    if (!n_tokens) {
        const uint32_t per = q4_units(N, unit_log2) * jobs, seq = unit / per;
        *first = seq * per;
        return (int)seq;
    }
    const int lane = threadIdx.x & 63;
    uint32_t at = 0;
    for (int s0 = 0;; s0 += RA_WAVE) {
        const int s = s0 + lane;
        const uint32_t u = q4_units(s0 == 0 ? x.rows : s < n_seq ? q4_rows_of(n_tokens, s, N) : 0, unit_log2);
        const uint32_t upto = q4_scan64(u);
        const unsigned long long past = __ballot(at + upto * jobs > unit);
        if (past != 0ull || s0 + RA_WAVE >= n_seq) {
            const int l = past != 0ull ? __ffsll(past) - 1 : 63;
            *first = at + (uint32_t)__builtin_amdgcn_readlane((int)(upto - u), l) * jobs;
            return s0 + l;
        }
        at += (uint32_t)__builtin_amdgcn_readlane((int)upto, 63) * jobs;
    }
}

template <int DT, int HEADS>
__global__ __launch_bounds__(Q4_THREADS, DT == RA_BF16 ? 3 : 2) void q4_full_kernel(const void* __restrict__ q, Q4Cache c, int n_seq, int n_q,
                                                                                  int n_kv, int N, const int32_t* __restrict__ n_tokens,
                                                                                  int tiles, int unit_log2, int whole, float* __restrict__ partials,
                                                                                  float* __restrict__ out, float* __restrict__ lse) {
    __shared__ Q4Lds lds;
    const int jobs = n_kv * tiles, group = n_q / n_kv, wg = blockIdx.x;
    uint32_t at = 0, end = 1, first = 0;
    int seq = wg / jobs;
    Q4List x;
    if (!whole) {
        x = q4_list(n_tokens, n_seq, 0, N, unit_log2, jobs, gridDim.x);
        if ((uint32_t)wg >= x.workgroups) return;
        at = x.from(wg);
        end = x.from(wg + 1);
        seq = q4_seq_of(x, n_tokens, n_seq, N, unit_log2, jobs, at, &first);
    }
    while (at < end) {
        // (what depends on the thread alone is worked out anew for each job: kept over the loop it takes 80 registers)
        int tid = threadIdx.x;
        asm volatile("" : "+v"(tid));
        const int lane = tid & 63, wv = tid / RA_WAVE;
        const int n = whole || seq >= RA_WAVE ? q4_rows_of(n_tokens, seq, N) : __builtin_amdgcn_readlane(x.rows, seq);
        const uint32_t units = q4_units(n, unit_log2);
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
        const size_t kv_head = (size_t)seq * n_kv + job / tiles;
        const int head_in_group = job % tiles * HEADS, heads = group - head_in_group < HEADS ? group - head_in_group : HEADS;
        const size_t head0 = (size_t)seq * n_q + (size_t)(job / tiles) * group + head_in_group;
        const int64_t from = (int64_t)unit0 << unit_log2, upto = (int64_t)unit1 << unit_log2, to = upto < n ? upto : n;
        const Q4Cache h{c.k + kv_head * c.kv_stride * Q4_ROW, c.ks + kv_head * c.kv_stride * Q4_BLOCKS,
                        c.v + kv_head * c.kv_stride * Q4_ROW, c.vs + kv_head * c.kv_stride * Q4_BLOCKS, c.kv_stride};
        // whole chunks, then the last, if it is not. Loads are not branched around (the counts of what is on its way would have to
        // hold for both ways, and every chunk would wait for the next one's loads): past the end it is the last chunk again. That is so for
        // bfloat16. With float32 queries the compiler puts the next chunk's loads behind the first products of the current one and a wait for all of
        // that one's, values included, and a head's queries, split into terms, are waited for in two groups before its first rows are asked for.
        const int step = Q4_UNIT, rows = (int)(to - from);
        int row = __builtin_amdgcn_readfirstlane(wv) * Q4_CHUNK;
        const int last = row + (rows - Q4_CHUNK - row) / step * step;
        Q4Wave<DT, HEADS> s;
        Q4Chunk a, b;
        s.start(reinterpret_cast<const char*>(q) + head0 * RA_D * (DT == RA_BF16 ? 2 : 4), heads, lane);
        if (row + Q4_CHUNK <= rows) {
            Q4Stream rd;
            rd.start(h, from, rows, lane);
            rd.fetch(a, row);
            while (true) {
                rd.fetch(b, row + step < last ? row + step : last);
                s.template add<true>(a, 255u, lane);
                row += step;
                if (row > last) break;
                rd.fetch(a, row + step < last ? row + step : last);
                s.template add<true>(b, 255u, lane);
                row += step;
                if (row > last) break;
            }
        }
        if (row < rows) {
            q4_fetch_last(a, h, from + row, to, lane);
            s.template add<false>(a, q4_there(from + row, to, lane), lane);
        }
        const size_t places = (size_t)gridDim.x + (size_t)n_seq * jobs, place = (size_t)wg + (size_t)seq * jobs + job;
        q4_close(s, lds, heads, tid, [&](int hd, int d, float sum, float mx, float l) {
            if (!whole) {
                partials[(hd * places + place) * RA_D + d] = sum;
                if (d == 0) reinterpret_cast<float2*>(partials + HEADS * places * RA_D)[hd * places + place] = make_float2(mx, l);
            } else {
                out[(head0 + hd) * RA_D + d] = mx > -INFINITY ? sum / l : 0.f;
                if (d == 0) lse[head0 + hd] = mx > -INFINITY ? mx * Q4_LN2 + logf(l) : -INFINITY;
            }
        });
        if (whole) return;
        at += unit1 - unit0;
        if (at < end) __syncthreads();                       // (the next job's sums go through the same LDS)
    }
}

// A head's records, those of a row of workgroups: their sums, their maxima and sums of weights, and how many.
struct Q4Records { const float* sums; const float2* ml; int have; };
__device__ __forceinline__ Q4Records q4_records(const float* partials, size_t head, int n_seq, int n_q, int n_kv, int N,
                                                const int32_t* n_tokens, int tiles, int unit_log2, int heads, int grid) {
    const int seq = (int)(head / n_q), group = n_q / n_kv, h = (int)(head % n_q), jobs = n_kv * tiles;
    const int job = h / group * tiles + h % group / heads;
    const Q4List x = q4_list(n_tokens, n_seq, seq, N, unit_log2, jobs, grid);
    const uint32_t units = q4_units(x.n, unit_log2);
    int have = 0, wg0 = 0;
    if (units) {
        const uint32_t unit0 = x.first + job * units;
        wg0 = (int)x.owner(unit0);
        have = (int)x.owner(unit0 + units - 1) - wg0 + 1;
    }
    const size_t places = (size_t)grid + (size_t)n_seq * jobs, at = h % group % heads * places + (size_t)wg0 + (size_t)seq * jobs + job;
    return {partials + at * RA_D, reinterpret_cast<const float2*>(partials + heads * places * RA_D) + at, have};
}

// What is combined: grid: x = DIMS dimensions of a head. One record or a few (of most heads, in a batch): a thread per dimension, all records
// on their way at once. More: groups of DIMS threads take records in turn, the first of which are on their way before the weights are known.
// Workgroups of 32 dimensions where few heads have many records each (131072 tokens of 8 KV heads: with 1024 threads 32.5 us a
// call, 512 31.9, 256 32.0), else of all 128: of 512 threads, for a batch's one long sequence (32 of one KV head, one of 262144 tokens and the
// others 500: with 128 threads 61 us, 512 32), and where the heads are many, of 128 (1024 jobs of 2500 rows: with 512 threads 69, 128 61).
#define Q4_MERGE_FEW 16
template <int THREADS, int DIMS>
__global__ __launch_bounds__(THREADS) void q4_full_merge_kernel(const float* __restrict__ partials, int n_seq, int n_q, int n_kv,
                                                                         int N, const int32_t* __restrict__ n_tokens, int tiles,
                                                                         int unit_log2, int heads, int grid, float* __restrict__ out,
                                                                         float* __restrict__ lse) {
    constexpr int WAVES = THREADS / RA_WAVE, SL = THREADS / DIMS, FLY = DIMS == RA_D ? 16 : 32;
    constexpr int MOST = DIMS == RA_D ? Q4_MOST_WORKGROUPS : Q4_MOST_WORKGROUPS / 3 * 2;       // records of a head
    constexpr int MINE = (MOST + THREADS - 1) / THREADS;                     // that a thread makes the weight of
    __shared__ float s_w[MINE * THREADS], s_m[WAVES], s_l[WAVES], s_a[SL][DIMS];
    const int tid = threadIdx.x, t = tid % DIMS, slice = tid / DIMS, lane = tid & 63;
    const size_t head = blockIdx.x / (RA_D / DIMS);
    const int dim = blockIdx.x % (RA_D / DIMS) * DIMS + t;
    const Q4Records x = q4_records(partials, head, n_seq, n_q, n_kv, N, n_tokens, tiles, unit_log2, heads, grid);
    const int have = x.have;
    float mx = -INFINITY, ll = 0.f, a = 0.f;
    if (DIMS == RA_D && have <= Q4_MERGE_FEW) {
        if (slice) return;
        float m[Q4_MERGE_FEW], l[Q4_MERGE_FEW], r[Q4_MERGE_FEW];
#pragma unroll
        for (int u = 0; u < Q4_MERGE_FEW; ++u) {
            const bool is = u < have;
            const float2 ml = is ? x.ml[u] : make_float2(-INFINITY, 0.f);
            m[u] = ml.x;
            l[u] = ml.y;
            r[u] = is ? x.sums[(size_t)u * RA_D + dim] : 0.f;
        }
#pragma unroll
        for (int u = 0; u < Q4_MERGE_FEW; ++u) mx = fmaxf(mx, m[u]);
        const float base = mx > -INFINITY ? mx : 0.f;
#pragma unroll
        for (int u = 0; u < Q4_MERGE_FEW; ++u) {
            const float w = __builtin_amdgcn_exp2f(m[u] - base);
            a = fmaf(r[u], w, a);
            ll = fmaf(l[u], w, ll);
        }
    } else {
        float r[FLY], m[MINE], l[MINE];
#pragma unroll
        for (int u = 0; u < FLY; ++u) r[u] = slice + u * SL < have ? x.sums[(size_t)(slice + u * SL) * RA_D + dim] : 0.f;
#pragma unroll
        for (int i = 0; i < MINE; ++i) {
            const int rec = tid + i * THREADS;
            const float2 ml = rec < have ? x.ml[rec] : make_float2(-INFINITY, 0.f);
            m[i] = ml.x;
            l[i] = ml.y;
            mx = fmaxf(mx, m[i]);
        }
#pragma unroll
        for (int d = 1; d < RA_WAVE; d <<= 1) mx = fmaxf(mx, __shfl_xor(mx, d));
        if (lane == 0) s_m[tid / RA_WAVE] = mx;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < WAVES; ++w) mx = fmaxf(mx, s_m[w]);
#pragma unroll
        for (int i = 0; i < MINE; ++i) {
            const float w = mx > -INFINITY ? __builtin_amdgcn_exp2f(m[i] - mx) : 0.f;
            s_w[tid + i * THREADS] = w;
            ll = fmaf(l[i], w, ll);
        }
#pragma unroll
        for (int d = 1; d < RA_WAVE; d <<= 1) ll += __shfl_xor(ll, d);
        if (lane == 0) s_l[tid / RA_WAVE] = ll;
        __syncthreads();
        for (int first = slice;;) {
#pragma unroll
            for (int u = 0; u < FLY; ++u)
                if (first + u * SL < have) a = fmaf(r[u], s_w[first + u * SL], a);
            first += FLY * SL;
            if (FLY * SL >= MOST || first - slice >= have) break;
#pragma unroll
            for (int u = 0; u < FLY; ++u) r[u] = first + u * SL < have ? x.sums[(size_t)(first + u * SL) * RA_D + dim] : 0.f;
        }
        s_a[slice][t] = a;
        __syncthreads();
        if (slice) return;
        ll = 0.f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) ll += s_l[w];
#pragma unroll
        for (int i = 1; i < SL; ++i) a += s_a[i][t];
    }
    out[head * RA_D + dim] = mx > -INFINITY ? a / ll : 0.f;
    if (dim == 0) lse[head] = mx > -INFINITY ? mx * Q4_LN2 + logf(ll) : -INFINITY;
}

// ---- the retrieved set and the static set -------------------------------------------------------
struct Q4Out {
    uint32_t* tickets;                  // one word per query head (ticket.h), or null
    float *out, *lse, *o_om, *lse_om, *o_w, *lse_w;
};

// the rows of a job: ids of a head, or [0, s) and then from `w` on
struct Q4Rows {
    const int32_t* ids;
    int64_t N, s, w;
    int count;
};
__device__ __forceinline__ int q4_row(const Q4Rows& src, int r) {
    if (src.ids) {
        const int id = src.ids[r < src.count ? r : src.count - 1];
        return r < src.count && id < src.N ? id : -1;
    }
    return r >= src.count ? -1 : r < src.s ? r : (int)(src.w - src.s) + r;
}
// rows [at, at + 32) of a job; returns which of the lane's rows there are. Loads of rows are not branched around: a row that is
// not there is row 0. (Its ids are: as compiled, a lane's ten are read and waited for one after another, nearly all from the nearest cache.)
__device__ __forceinline__ uint32_t q4_gather(Q4Chunk& c, const Q4Cache& h, const Q4Rows& src, int at, int lane) {
    const int kg = lane >> 4, r = lane & 15;
    int kr[2], vr[8];
#pragma unroll
    for (int t = 0; t < 2; ++t) kr[t] = q4_row(src, at + 16 * t + r);
#pragma unroll
    for (int j = 0; j < 8; ++j) vr[j] = q4_row(src, at + (j & 4) * 4 + 4 * kg + (j & 3));
    uint32_t there = 0u;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        const size_t row = kr[t] >= 0 ? kr[t] : 0;
        c.k[t] = *reinterpret_cast<const uint4*>(h.k + row * Q4_ROW + 16 * kg);
        c.ks[t] = h.ks[row * Q4_BLOCKS + kg];
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const size_t row = vr[j] >= 0 ? vr[j] : 0;
        c.v[j] = *reinterpret_cast<const uint32_t*>(h.v + row * Q4_ROW + 4 * r);
        c.vs[j] = *reinterpret_cast<const uint32_t*>(h.vs + row * Q4_BLOCKS);
        there |= (vr[j] >= 0 ? 1u : 0u) << j;
    }
    return there;
}

template <bool COHERENT>
__device__ __forceinline__ void q4_store(float* p, float v) {
    if (COHERENT) __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    else *p = v;
}
template <bool COHERENT>
__device__ __forceinline__ float q4_load(const float* p) {
    return COHERENT ? __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : *p;
}

// Dimension d of a head's records [first, last), every `by`th: their maximum, sum of weights and weighted sum.
struct Q4Sum { float m, l, a; };
template <bool COHERENT>
__device__ __forceinline__ Q4Sum q4_add_up(const float* rec, int first, int last, int by, int d) {
    constexpr int FLY = 8;
    Q4Sum x{-INFINITY, 0.f, 0.f};
    for (int i0 = first; i0 < last; i0 += FLY * by) {
        float m[FLY], l[FLY], a[FLY], mx = x.m;
#pragma unroll
        for (int u = 0; u < FLY; ++u) {
            const float* y = rec + (size_t)(i0 + u * by < last ? i0 + u * by : i0) * Q4_REC;
            m[u] = q4_load<COHERENT>(y + RA_D);
            l[u] = q4_load<COHERENT>(y + RA_D + 1);
            a[u] = q4_load<COHERENT>(y + d);
        }
#pragma unroll
        for (int u = 0; u < FLY; ++u) mx = fmaxf(mx, m[u]);
        if (mx == -INFINITY) continue;
        const float corr = __builtin_amdgcn_exp2f(x.m - mx);
        x.a *= corr;
        x.l *= corr;
#pragma unroll
        for (int u = 0; u < FLY; ++u) {
            const float w = i0 + u * by < last ? __builtin_amdgcn_exp2f(m[u] - mx) : 0.f;
            x.a = fmaf(a[u], w, x.a);
            x.l = fmaf(l[u], w, x.l);
        }
        x.m = mx;
    }
    return x;
}
// Eq. 4 for the static set and for Omega, Eq. 5 for both
__device__ __forceinline__ void q4_write(const Q4Sum (&set)[2], size_t head, int d, const Q4Out& o) {
    float* o_set[2] = {o.o_w, o.o_om};
    float* l_set[2] = {o.lse_w, o.lse_om};
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const bool empty = set[i].m == -INFINITY;
        if (o_set[i]) o_set[i][head * RA_D + d] = empty ? 0.f : set[i].a / set[i].l;
        if (l_set[i] && d == 0) l_set[i][head] = empty ? -INFINITY : set[i].m * Q4_LN2 + logf(set[i].l);
    }
    const float mx = fmaxf(set[0].m, set[1].m);
    float out = 0.f, lse = -INFINITY;
    if (mx > -INFINITY) {
        const float e0 = __builtin_amdgcn_exp2f(set[0].m - mx), e1 = __builtin_amdgcn_exp2f(set[1].m - mx);
        const float l = set[0].l * e0 + set[1].l * e1;
        out = (set[0].a * e0 + set[1].a * e1) / l;
        lse = mx * Q4_LN2 + logf(l);
    }
    o.out[head * RA_D + d] = out;
    if (d == 0) o.lse[head] = lse;
}
// dimension d of a head from its records, nS of the static set and nG of Omega
template <bool COHERENT>
__device__ __forceinline__ void q4_finish(const float* rec, int nS, int nG, size_t head, int d, const Q4Out& o) {
    const Q4Sum set[2] = {q4_add_up<COHERENT>(rec, 0, nS, 1, d), q4_add_up<COHERENT>(rec, nS, nS + nG, 1, d)};
    q4_write(set, head, d, o);
}

// grid: per (sequence, KV head) the parts of each of its query heads' Omega (their loads wait for ids, so they start first), then
// the parts of the static set per tile of heads. `spanS`, `spanG`: rows of a part. TICKETS: the workgroup that stores a head's last
// record combines them all (ticket.h), which saves a launch.
template <int DT, int HEADS, bool TICKETS>
__global__ __launch_bounds__(Q4_THREADS, 3) void q4_attend_kernel(const void* __restrict__ q, Q4Cache c, int n_q, int n_kv, int64_t N,
                                                               int64_t s, int64_t w, int topk, const int32_t* __restrict__ ids, int nS,
                                                               int nG, int spanS, int spanG, int tiles, float* partials, Q4Out o) {
    __shared__ Q4Lds lds;
    __shared__ uint32_t s_last[HEADS];
    const int tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid / RA_WAVE);
    const int group = n_q / n_kv, per = tiles * nS + group * nG, P = nS + nG;
    const size_t kv_head = blockIdx.x / per;
    const int x = blockIdx.x % per;
    const size_t group0 = kv_head / n_kv * n_q + kv_head % n_kv * group;
    const bool om = x < group * nG;
    const int first = om ? x / nG : (x - group * nG) / nS * HEADS;        // of the group's heads
    const int part = om ? x % nG : (x - group * nG) % nS, slot = om ? nS + part : part;
    const int heads = om ? 1 : group - first < HEADS ? group - first : HEADS;
    const size_t head0 = group0 + first;
    const Q4Cache h{c.k + kv_head * c.kv_stride * Q4_ROW, c.ks + kv_head * c.kv_stride * Q4_BLOCKS, c.v + kv_head * c.kv_stride * Q4_ROW,
                    c.vs + kv_head * c.kv_stride * Q4_BLOCKS, c.kv_stride};
    const Q4Rows src = om ? Q4Rows{ids + head0 * topk, N, 0, 0, topk} : Q4Rows{nullptr, N, s, w, (int)(s + N - w)};
    const int span = om ? spanG : spanS, from = part * span, to = from + span < src.count ? from + span : src.count;
    Q4Wave<DT, HEADS> st;
    st.start(reinterpret_cast<const char*>(q) + head0 * RA_D * (DT == RA_BF16 ? 2 : 4), heads, lane);
    // Whole chunks of W's rows behind the sink lie side by side, [lo, hi) in steps, and are read as over all tokens, the next one always on
    // its way (with float32 queries asked for as late as in q4_full_kernel); then all others (us, one sequence of 32 + 8 heads with 8644,
    // 30644 and 100644 static rows 15.0, 19.9, 36 without, 11.4, 14.6, 28). Where everything is static there is no such part: all rows are others.
    const int step = Q4_WAVES * Q4_CHUNK, mine = from + wv * Q4_CHUNK;
    int lo = mine, hi = mine;
    if (!om) {
        if (lo < s) lo += ((int)s - lo + step - 1) / step * step;
        hi = lo;
        if (lo + Q4_CHUNK <= to) {
            Q4Chunk a, b;
            Q4Stream rd;
            const int last = (to - Q4_CHUNK - lo) / step * step;
            rd.start(h, w - s + lo, last + Q4_CHUNK, lane);
            hi = lo + last + step;
            int row = 0;
            rd.fetch(a, 0);
            while (true) {
                rd.fetch(b, row + step < last ? row + step : last);
                st.template add<true>(a, 255u, lane);
                row += step;
                if (row > last) break;
                rd.fetch(a, row + step < last ? row + step : last);
                st.template add<true>(b, 255u, lane);
                row += step;
                if (row > last) break;
            }
        }
    }
    for (int at = mine == lo ? hi : mine; at < to; at = at + step == lo ? hi : at + step) {
        Q4Chunk ch;
        const uint32_t there = q4_gather(ch, h, src, at, lane);
        st.template add<false>(ch, there, lane);
    }
    q4_close(st, lds, heads, tid, [&](int hd, int d, float sum, float mx, float l) {
        float* rec = partials + ((head0 + hd) * P + slot) * Q4_REC;
        q4_store<TICKETS>(rec + d, sum);
        if (d == 0) { q4_store<TICKETS>(rec + RA_D, mx); q4_store<TICKETS>(rec + RA_D + 1, l); }
    });
    if constexpr (TICKETS) {
        __builtin_amdgcn_s_waitcnt(0x0F70);     // vmcnt(0): this wavefront's record stores have completed
        __syncthreads();                        // ... and every other's
        if (tid < heads) {
            const uint32_t step = ticket_step(slot, P);
            s_last[tid] = ticket_last(__hip_atomic_fetch_add(o.tickets + head0 + tid, step, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT), step);
        }
        __syncthreads();
        for (int y = tid; y < heads * RA_D; y += Q4_THREADS)
            if (s_last[y / RA_D]) q4_finish<true>(partials + (head0 + y / RA_D) * P * Q4_REC, nS, nG, head0 + y / RA_D, y % RA_D, o);
    }
}

// grid: x = head (with its sequence); SLICES threads per dimension take the records in turn
template <int SLICES>
__global__ __launch_bounds__(RA_D * SLICES) void q4_merge_kernel(const float* __restrict__ partials, int nS, int nG, Q4Out o) {
    const size_t head = blockIdx.x;
    const float* rec = partials + head * (nS + nG) * Q4_REC;
    const int d = threadIdx.x % RA_D, slice = threadIdx.x / RA_D;
    if constexpr (SLICES == 1) {
        q4_finish<false>(rec, nS, nG, head, d, o);
    } else {
        __shared__ Q4Sum s_part[SLICES][2][RA_D];
        s_part[slice][0][d] = q4_add_up<false>(rec, slice, nS, SLICES, d);
        s_part[slice][1][d] = q4_add_up<false>(rec, nS + slice, nS + nG, SLICES, d);
        __syncthreads();
        if (slice) return;
        Q4Sum set[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            Q4Sum x{-INFINITY, 0.f, 0.f};
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
        q4_write(set, head, d, o);
    }
}

// query heads of a tile (columns of the matrix instructions)
static int q4_heads(int group) { return group <= 4 ? 4 : group <= 8 ? 8 : 16; }
#define Q4_HEADS_GO(GO, DTV)                            \
    do {                                                \
        const int hv_ = q4_heads(n_q / n_kv);           \
        if (hv_ == 4) GO(DTV, 4);                       \
        else if (hv_ == 8) GO(DTV, 8);                  \
        else GO(DTV, 16);                               \
    } while (0)

// How a call is cut: tiles of query heads per KV head, workgroups, and whether each has a job of its own. That is so where a head's rows are
// few or the jobs many. Shared out and by themselves, us: 512 rows of 8 jobs 8.8, 7.0, 1000 rows 9.0, 9.8 (and a launch less on the host's
// side), 2000 rows 8.9, 15.2; 128 jobs of 2000 rows 17.3, 16.5, of 4000 22.1, 26.7, of 8000 32.1, 47.8; 512 of 8000 107, 99.5, of 0 to 8000 70, 67; 1024
// of 16000 388, 375, of 0 to 16000 235, 244; 2048 of 20000 927, 886. The price is what a job costs that is longer than the others: it takes 5 ns a
// row alone, hence the limit however many there are. 8 jobs of 8000 rows (one sequence) beside 504 of 200 take 18.8 shared out and 47 by themselves: the
// lengths are known on the device only, and this goes by the capacity.
// Otherwise three workgroups of bfloat16 fit a compute unit, two of float32; where few jobs share them, two leave fewer records to
// combine (us, two and three: 8 jobs of 131072 rows 32.9, 33.9, one of a million 36.0, 40.3, 64 of 20011 38.1, 38.5, 128 of up to
// 32768 64.5, 62.8).
#define Q4_MOST_ROWS (1 << 24)      // of one job in a stretch: places in its codes fit 31 bits
struct Q4Cut { int tiles, workgroups, unit_log2; bool whole; const char* refused; };       // refused: why, or null
static Q4Cut q4_cut(ra_dtype dt, int n_seq, int n_q, int n_kv, int64_t N) {
    Q4Cut x;
    const int heads = q4_heads(n_q / n_kv);
    x.tiles = (int)(((int64_t)(n_q / n_kv) + heads - 1) / heads);
    const int64_t jobs = (int64_t)n_seq * n_kv * x.tiles;
    // (from Q4_MOST_UNITS jobs on there is no list: its units, and the threads of the second kernel, 128 for each of up to 16 heads, fit 32 bits)
    x.whole = N <= 1024 || N <= (jobs < 2048 ? 16 * jobs : 32768) || (jobs >= Q4_MOST_UNITS && N <= Q4_MOST_ROWS);
    x.unit_log2 = 7;
    static_assert(Q4_UNIT == 1 << 7, "rows of a unit");
    x.refused = x.whole && jobs >= 1 << 24 ? "too many heads for one launch: 2^24 tiles of up to 16 query heads"
                : !x.whole && jobs >= Q4_MOST_UNITS ? "too many heads for one launch: 2^21 tiles of up to 16 query heads over more than 2^24 tokens" : nullptr;
    x.workgroups = (int)jobs;
    if (x.whole || x.refused) return x;
    auto units = [&] { return jobs * ((N + ((int64_t)1 << x.unit_log2) - 1) >> x.unit_log2); };
    while (units() > Q4_MOST_UNITS) ++x.unit_log2;
    const int most = jobs <= 64 || dt == RA_F32 ? Q4_MOST_WORKGROUPS / 3 * 2 : Q4_MOST_WORKGROUPS;
    x.workgroups = (int)(units() < most ? units() : most);
    // (a stretch is longest with all sequences at their longest; only very many query heads of one KV head get here)
    if (N > Q4_MOST_ROWS && ((units() / x.workgroups + 1) << x.unit_log2) > Q4_MOST_ROWS)
        x.refused = "too many heads for one launch: a workgroup's part of one would pass 2^24 rows";
    return x;
}

size_t ra_full_q4_partial_floats(ra_dtype dt, int n_seq, int n_q, int n_kv, int64_t N) {
    const Q4Cut x = q4_cut(dt, n_seq, n_q, n_kv, N);
    return x.whole || x.refused ? 0 : ((size_t)x.workgroups + (size_t)n_seq * n_kv * x.tiles) * q4_heads(n_q / n_kv) * (RA_D + 2);
}

#define Q4_FEW_RECORDS 32
ra_status ra_launch_full_q4(const void* q, ra_dtype dt, const Q4Cache& c, int n_seq, int n_q, int n_kv, int64_t N,
                            const int32_t* n_tokens, float* partials, hipStream_t st, float* out, float* lse) {
    const Q4Cut x = q4_cut(dt, n_seq, n_q, n_kv, N);
    if (x.refused) RA_FAIL(RA_EUNSUP, "%s", x.refused);
#define Q4_GO(DTV, HV)                                                                                                         \
    hipLaunchKernelGGL((q4_full_kernel<DTV, HV>), dim3(x.workgroups), dim3(Q4_THREADS), 0, st, q, c, n_seq, n_q, n_kv, (int)N, n_tokens, \
                       x.tiles, x.unit_log2, (int)x.whole, partials, out, lse)
    if (dt == RA_BF16) Q4_HEADS_GO(Q4_GO, RA_BF16); else Q4_HEADS_GO(Q4_GO, RA_F32);
#undef Q4_GO
    RA_HIP(hipGetLastError());
    if (x.whole) return RA_OK;
#define Q4_MERGE(THREADS, DIMS)                                                                                                                  \
    hipLaunchKernelGGL((q4_full_merge_kernel<THREADS, DIMS>), dim3(n_seq * n_q * (RA_D / DIMS)), dim3(THREADS), 0, st, partials, n_seq, n_q, n_kv, \
                       (int)N, n_tokens, x.tiles, x.unit_log2, q4_heads(n_q / n_kv), x.workgroups, out, lse)
    // records per head, were all sequences as long as the longest
    if (x.workgroups / (n_seq * n_kv * x.tiles) > Q4_FEW_RECORDS) Q4_MERGE(512, 32);
    else if ((int64_t)n_seq * n_q <= 1024) Q4_MERGE(512, RA_D);
    else Q4_MERGE(128, RA_D);
#undef Q4_MERGE
    RA_HIP(hipGetLastError());
    return RA_OK;
}

// W = [0, s) u [w, N) of Sec. 3.3, with what came after the index was built; ranges that meet make everything static
static void q4_static(int64_t N, int64_t Ng, int sink, int window, int64_t* s, int64_t* w) {
    *s = sink < N ? sink : N;
    *w = N - window < Ng ? N - window : Ng;
    if (*w <= *s) { *s = N; *w = N; }
}

// Columns of the sparse set's tiles: a wavefront has a chunk or two, and what counts is the way to its end, which is longer the more
// columns a head has.
#define Q4_ATTEND_HEADS 16
// parts of the two sets: 128 rows each, a chunk for each wavefront of a workgroup; longer ones where they would be very many
struct Q4Parts { int nS, nG, spanS, spanG, tiles; };
static Q4Parts q4_parts(int n_seq, int n_q, int n_kv, int64_t n_static, int topk) {
    const int heads = Q4_ATTEND_HEADS;
    Q4Parts p;
    p.tiles = (n_q / n_kv + heads - 1) / heads;
    p.spanG = Q4_PART;
    while (p.spanG < topk && (int64_t)n_seq * n_q * ((topk + p.spanG - 1) / p.spanG) > 2048) p.spanG *= 2;
    p.nG = (topk + p.spanG - 1) / p.spanG;
    // Of the static set so many that all workgroups are there at once, three per compute unit, where Omega's leave room for some (us, 16
    // sequences of 32 + 8 heads, 8 static parts of 512 rows each in 128: 512 workgroups at most 18.4 float32, 14.7 bfloat16, the rest of 768 15.6
    // and 14.5; where Omega leaves none, one part 26.5, up to 512 workgroups 23.4).
    const int64_t jobs = (int64_t)n_seq * n_kv * p.tiles, rest = (768 - (int64_t)n_seq * n_q * p.nG) / jobs;
    int64_t most = rest >= 1 && rest < 512 / jobs ? rest : 512 / jobs;
    if (most < 1) most = 1;
    int64_t nS = (n_static + Q4_PART - 1) / Q4_PART;
    if (nS > most) nS = most;
    if (nS < (n_static + Q4_MOST_ROWS - 1) / Q4_MOST_ROWS) nS = (n_static + Q4_MOST_ROWS - 1) / Q4_MOST_ROWS;
    p.spanS = nS ? (int)((n_static + nS - 1) / nS + Q4_PART - 1) / Q4_PART * Q4_PART : Q4_PART;
    p.nS = (int)((n_static + p.spanS - 1) / p.spanS);
    return p;
}

size_t ra_attend_q4_partial_floats(ra_dtype, int n_seq, int n_q, int n_kv, int64_t N, int64_t Ng, int sink, int window, int topk) {
    int64_t s, w;
    q4_static(N, Ng, sink, window, &s, &w);
    const Q4Parts p = q4_parts(n_seq, n_q, n_kv, s + N - w, topk);
    return (size_t)n_seq * n_q * (p.nS + p.nG) * Q4_REC;
}

// Whether a head's last workgroup combines its records, or a second launch, which costs 1 us, does. That workgroup reads past the L2, eight
// records at a time and two heads side by side, for all heads of a tile that it was the last of; and storing and drawing tickets costs each
// workgroup something. So: up to 4 heads to a tile, three trips of eight records, fewer than 2048 records in all (us, second launch and
// tickets. 32 + 8 heads, 7 records a head, of 1, 4 and 8 sequences 8.2, 7.3, 10.5, 9.8, 12.3, 11.4; 13 records, of 1 and 4 sequences 8.9, 7.9, 11.7, 10.4; 3 or 4
// records, of 12, 16, 24 and 32 sequences 13.1, 12.5, 14.2, 13.8, 18.9, 19.6, 22.2, 24.0; 4 heads of one KV head, 13, 21, 29, 41, 64 and 127 records 8.5,
// 7.7, 8.3, 8.2, 8.3, 8.8, 8.4, 9.3, 8.4, 11.0, 9.3, 16.4; 32 + 8 heads, 21 and 29 records 8.8, 9.2, 9.0, 12.9; 8 heads of one KV head, 7
// records, of 1 and 16 sequences 7.9, 7.4 to 8.4, 9.1, 9.7 to 10.6; 16 of one, 7 and 64 records 8.7, 18.5, 9.4, 50.9).
#define Q4_TICKET_HEADS 4
#define Q4_TICKET_TRIPS 3
#define Q4_TICKET_RECORDS 2048

ra_status ra_launch_attend_q4(const void* q, ra_dtype dt, const Q4Cache& c, int n_seq, int n_q, int n_kv, int64_t N, int64_t Ng,
                              int sink, int window, int topk, const int32_t* ids, float* partials, uint32_t* tickets,
                              hipStream_t st, float* out, float* lse, float* o_omega, float* lse_omega, float* o_w, float* lse_w) {
    int64_t s, w;
    q4_static(N, Ng, sink, window, &s, &w);
    const Q4Parts p = q4_parts(n_seq, n_q, n_kv, s + N - w, topk);
    const int64_t blocks = (int64_t)n_seq * n_kv * (p.tiles * p.nS + n_q / n_kv * p.nG);
    if (blocks > (1 << 24) - 1) RA_FAIL(RA_EUNSUP, "too many heads for one launch");
    const int trips = (p.nS + 7) / 8 + (p.nG + 7) / 8;
    if (n_q / n_kv > Q4_TICKET_HEADS || trips > Q4_TICKET_TRIPS || (int64_t)n_seq * n_q * (p.nS + p.nG) >= Q4_TICKET_RECORDS) tickets = nullptr;
    const Q4Out o{tickets, out, lse, o_omega, lse_omega, o_w, lse_w};
#define Q4_GO(DTV, TK)                                                                                                          \
    hipLaunchKernelGGL((q4_attend_kernel<DTV, Q4_ATTEND_HEADS, TK>), dim3((unsigned)blocks), dim3(Q4_THREADS), 0, st, q, c, n_q, n_kv, N, s, w, \
                       topk, ids, p.nS, p.nG, p.spanS, p.spanG, p.tiles, partials, o)
    if (dt == RA_BF16) { if (tickets) Q4_GO(RA_BF16, true); else Q4_GO(RA_BF16, false); }
    else { if (tickets) Q4_GO(RA_F32, true); else Q4_GO(RA_F32, false); }
#undef Q4_GO
    RA_HIP(hipGetLastError());
    if (tickets) return RA_OK;
    // (eight records are on their way at a time. 16 heads of one KV head, 100640 static rows in 394 records: 44 us with one thread per
    // dimension, 19 with eight; 24 records 26.7 and 27.3)
    if (trips <= 3) hipLaunchKernelGGL(q4_merge_kernel<1>, dim3(n_seq * n_q), dim3(RA_D), 0, st, partials, p.nS, p.nG, o);
    else hipLaunchKernelGGL(q4_merge_kernel<8>, dim3(n_seq * n_q), dim3(RA_D * 8), 0, st, partials, p.nS, p.nG, o);
    RA_HIP(hipGetLastError());
    return RA_OK;
}
