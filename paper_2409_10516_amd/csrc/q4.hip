// Attention over a cache in 4 bits: all tokens (ra_full_attention_q4), and the retrieved set Omega and the static set W of
// Sec. 3.3 with their combination by Eq. 4-5 (ra_attend_q4).
//
// Rows are cut into parts; a workgroup turns one part into a record (128 weighted sums, the running maximum of
// z log2(e), the sum of weights), and a second kernel combines a head's records. Weights are powers of two,
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
// Codes become bfloat16 exactly. The columns are terms of weights: a bfloat16 weight has 8 bits, so column c holds term c / H of head
// c % H, the first as rounded, the next what the rounding left; 2 terms of 8 heads (bfloat16), 3 of 4 (float32, whose queries are
// three bfloat16 terms too, in three instructions). The terms of a head are added at the end. The sum of the weights is that of the
// terms (an instruction with a row of ones), so that what their rounding does to a weight that has nearly everything cancels.
// The running maximum of a column moves only when a logit exceeds it by more than 8 (in powers of two), which keeps the
// lanes' exchange and the scaling of sums out of nearly every chunk.
typedef __bf16 q4_bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 q4_bf16x8 __attribute__((ext_vector_type(8)));
typedef float q4_f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t q4_u32x4 __attribute__((ext_vector_type(4), aligned(4)));
#define Q4_CHUNK 32
#define Q4_LOWEST (-1.7e38f)        // below every logit: a maximum that nothing has moved yet

template <int DT> struct Q4Form;
template <> struct Q4Form<RA_BF16> { enum { HEADS = 8, TERMS = 2, Q = 1 }; };
template <> struct Q4Form<RA_F32> { enum { HEADS = 4, TERMS = 3, Q = 3 }; };

struct Q4Chunk {
    uint4 k[2];
    uint32_t ks[2], v[8], vs[8];
};

template <int DT>
struct Q4Wave {
    typedef Q4Form<DT> F;
    q4_bf16x8 q[F::Q][4];
    q4_f32x4 acc[8], sum;      // weighted sums, and the sum of the weights as they went in, the same in all rows
    float m;

    // queries of heads 0 .. n - 1 of a tile, 128 values each; columns past them are zero
    __device__ __forceinline__ void start(const void* q0, int n, int lane) {
        const int kg = lane >> 4, h = (lane & 15) % F::HEADS;
        const bool have = h < n;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const size_t at = (size_t)(have ? h : 0) * RA_D + 32 * kg + 8 * i;
            if constexpr (DT == RA_BF16) {
                const uint4 u = *reinterpret_cast<const uint4*>(reinterpret_cast<const uint16_t*>(q0) + at);
                q[0][i] = __builtin_bit_cast(q4_bf16x8, have ? u : make_uint4(0u, 0u, 0u, 0u));
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    float x = have ? reinterpret_cast<const float*>(q0)[at + e] : 0.f;
#pragma unroll
                    for (int t = 0; t < F::Q; ++t) {
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
    }

    // `there`: bit j says whether the lane's row j is one (rows 4 kg + j of the first half, j < 4, then of the second); ALL: all are
    template <bool ALL>
    __device__ __forceinline__ void add(const Q4Chunk& c, uint32_t there, int lane) {
        q4_f32x4 S[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
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
                for (int x = F::Q - 1; x >= 0; --x)         // (the smallest term first)
                    S[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(q4_bf16x8, b), q[x][i], S[t], 0, 0, 0);
            }
        }
        float z[8], top = Q4_LOWEST;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            z[j] = S[j / 4][j & 3];
            if (!ALL) z[j] = (there >> j) & 1u ? z[j] : -INFINITY;
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
        // weights, and this column's term of them
        const int term = (lane & 15) / F::HEADS;
        q4_bf16x8 P;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            float x = __builtin_amdgcn_exp2f(fmaf(z[j], Q4_C, -m));
#pragma unroll
            for (int t = 1; t < F::TERMS; ++t) x = fmaf(term >= t ? -1.f : 0.f, (float)(__bf16)x, x);
            P[j] = (__bf16)x;
        }
        sum = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(q4_bf16x8, make_uint4(0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u)),
                                                      P, sum, 0, 0, 0);
        uint32_t pair[4][8];                                 // [dimensions 2 y, 2 y + 1][row]
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            float unit = q4_unit((c.vs[j] >> (8 * ((lane & 15) / 4))) & 255u);
            uint32_t w = c.v[j];
            if (!ALL) {                                      // (0 * NaN is not 0)
                const bool have = (there >> j) & 1u;
                unit = have ? unit : 1.f;
                w = have ? w : 0u;
            }
            pair[0][j] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, unit, 0));
            pair[1][j] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, unit, 1));
            pair[2][j] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, unit, 2));
            pair[3][j] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, unit, 3));
        }
#pragma unroll
        for (int d = 0; d < 8; ++d) {
            const uint32_t half = d & 1 ? 0x07060302u : 0x05040100u;
            const uint32_t(&p)[8] = pair[d / 2];
            uint4 a;
            a.x = __builtin_amdgcn_perm(p[1], p[0], half);
            a.y = __builtin_amdgcn_perm(p[3], p[2], half);
            a.z = __builtin_amdgcn_perm(p[5], p[4], half);
            a.w = __builtin_amdgcn_perm(p[7], p[6], half);
            acc[d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(q4_bf16x8, a), P, acc[d], 0, 0, 0);
        }
    }
};

// rows [from, from + 32) of a head (`from` the same in all lanes); past the last row, n - 1, that one
template <bool ALL>
__device__ __forceinline__ void q4_fetch(Q4Chunk& c, const Q4Cache& h, int64_t from, int64_t n, int lane) {
    const int kg = lane >> 4, r = lane & 15;
    const uint8_t *k = h.k + from * Q4_ROW, *ks = h.ks + from * Q4_BLOCKS, *v = h.v + from * Q4_ROW, *vs = h.vs + from * Q4_BLOCKS;
    const int last = ALL ? 31 : (int)(n - 1 - from);
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        const int row = ALL ? 16 * t + r : min(16 * t + r, last);
        c.k[t] = *reinterpret_cast<const uint4*>(k + row * Q4_ROW + 16 * kg);
        c.ks[t] = ks[row * Q4_BLOCKS + kg];
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int row = (j & 4) * 4 + 4 * kg + (j & 3);
        c.v[j] = *reinterpret_cast<const uint32_t*>(v + (ALL ? row : min(row, last)) * Q4_ROW + 4 * r);
        if (!ALL) c.vs[j] = *reinterpret_cast<const uint32_t*>(vs + min(row, last) * Q4_BLOCKS);
    }
    if (ALL)
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const q4_u32x4 w = *reinterpret_cast<const q4_u32x4*>(vs + (16 * t + 4 * kg) * Q4_BLOCKS);
            c.vs[4 * t] = w.x; c.vs[4 * t + 1] = w.y; c.vs[4 * t + 2] = w.z; c.vs[4 * t + 3] = w.w;
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

// The wavefronts' states -> one per head: f(head of the tile, dimension, sum, maximum, sum of weights), called by one thread
// for each; a head without rows has the maximum -infinity.
template <int DT, class Fn>
__device__ __forceinline__ void q4_close(Q4Wave<DT>& s, Q4Lds& lds, int n, Fn f) {
    typedef Q4Form<DT> F;
    const int tid = threadIdx.x, wv = tid / RA_WAVE, lane = tid & 63, kg = lane >> 4, col = lane & 15;
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
        float mx = -INFINITY, a = 0.f, ll = 0.f;
#pragma unroll
        for (int w = 0; w < Q4_WAVES; ++w) mx = fmaxf(mx, lds.m[w][h]);
        if (mx > -INFINITY)
#pragma unroll
            for (int w = 0; w < Q4_WAVES; ++w) {
                const float wt = __builtin_amdgcn_exp2f(lds.m[w][h] - mx);
                float sum = lds.a[w][h][d];
#pragma unroll
                for (int t = 1; t < F::TERMS; ++t) sum += lds.a[w][h + t * F::HEADS][d];
                float l = lds.l[w][h];
#pragma unroll
                for (int t = 1; t < F::TERMS; ++t) l += lds.l[w][h + t * F::HEADS];
                if (lds.m[w][h] > -INFINITY) {
                    a = fmaf(sum, wt, a);
                    ll = fmaf(l, wt, ll);
                }
            }
        f(h, d, a, mx, ll);
    }
}

// Attention over all tokens. A workgroup takes `span` rows of a KV head for a tile of its query heads, its wavefronts
// chunks in turn, the next one's loads before the present one's work. grid: per (KV head, tile of heads, part), eight parts side by side,
// then the next tile of the same ones, which then find their rows in the L2 of their XCD. A launch of one part per head writes
// the results; otherwise parts with rows leave records.
template <int DT>
__global__ __launch_bounds__(Q4_THREADS) void q4_full_kernel(const void* __restrict__ q, Q4Cache c, int n_q, int n_kv, int64_t N,
                                                             const int32_t* __restrict__ n_tokens, int span, int parts, int tiles,
                                                             float* __restrict__ partials, float* __restrict__ out,
                                                             float* __restrict__ lse) {
    typedef Q4Form<DT> F;
    __shared__ Q4Lds lds;
    const int rows8 = (parts + 7) / 8, lane = threadIdx.x & 63, wv = threadIdx.x / RA_WAVE;
    const int part = (blockIdx.x / (8 * tiles)) % rows8 * 8 + blockIdx.x % 8, tile = blockIdx.x / 8 % tiles;
    const size_t kv_head = blockIdx.x / (8u * tiles * rows8);
    const int seq = (int)(kv_head / n_kv), group = n_q / n_kv;
    int64_t n = n_tokens ? n_tokens[seq] : N;
    n = n < 0 ? 0 : n < N ? n : N;
    if (part >= parts || (parts > 1 && (int64_t)part * span >= n)) return;
    const int64_t from = (int64_t)part * span, to = from + span < n ? from + span : n;
    const size_t head0 = (size_t)seq * n_q + (kv_head % n_kv) * group + tile * F::HEADS;
    const int heads = group - tile * F::HEADS < F::HEADS ? group - tile * F::HEADS : F::HEADS;
    const Q4Cache h{c.k + kv_head * c.kv_stride * Q4_ROW, c.ks + kv_head * c.kv_stride * Q4_BLOCKS, c.v + kv_head * c.kv_stride * Q4_ROW,
                    c.vs + kv_head * c.kv_stride * Q4_BLOCKS, c.kv_stride};
    Q4Wave<DT> s;
    s.start(reinterpret_cast<const char*>(q) + head0 * RA_D * (DT == RA_BF16 ? 2 : 4), heads, lane);
    const int wave_first = __builtin_amdgcn_readfirstlane(wv) * Q4_CHUNK;
    int64_t at = from + wave_first;
    const int64_t step = Q4_WAVES * Q4_CHUNK;
    Q4Chunk a, b;
    if (at + Q4_CHUNK <= to) {
        q4_fetch<true>(a, h, at, to, lane);
        while (true) {
            const bool more = at + step + Q4_CHUNK <= to;
            if (more) q4_fetch<true>(b, h, at + step, to, lane);
            s.template add<true>(a, 255u, lane);
            at += step;
            if (!more) break;
            const bool more2 = at + step + Q4_CHUNK <= to;
            if (more2) q4_fetch<true>(a, h, at + step, to, lane);
            s.template add<true>(b, 255u, lane);
            at += step;
            if (!more2) break;
        }
    }
    if (at < to) {
        q4_fetch<false>(a, h, at, to, lane);
        s.template add<false>(a, q4_there(at, to, lane), lane);
    }
    q4_close<DT>(s, lds, heads, [&](int hd, int d, float sum, float mx, float l) {
        if (parts > 1) {
            float* rec = partials + ((head0 + hd) * parts + part) * Q4_REC;
            rec[d] = sum;
            if (d == 0) { rec[RA_D] = mx; rec[RA_D + 1] = l; }
        } else {
            out[(head0 + hd) * RA_D + d] = mx > -INFINITY ? sum / l : 0.f;
            if (d == 0) lse[head0 + hd] = mx > -INFINITY ? mx * Q4_LN2 + logf(l) : -INFINITY;
        }
    });
}

// The records of a head of all tokens. grid: x = head (with its sequence)
#define Q4_MAX_PARTS 512
#define Q4_MERGE_THREADS 512
__global__ __launch_bounds__(Q4_MERGE_THREADS) void q4_full_merge_kernel(const float* __restrict__ partials, int n_q, int64_t N,
                                                                         const int32_t* __restrict__ n_tokens, int span, int parts,
                                                                         float* __restrict__ out, float* __restrict__ lse) {
    __shared__ float s_w[Q4_MAX_PARTS], s_x[Q4_MERGE_THREADS / RA_WAVE], s_a[Q4_MERGE_THREADS / RA_D][RA_D];
    const int tid = threadIdx.x, t = tid % RA_D, slice = tid / RA_D, lane = tid & 63;
    const size_t head = blockIdx.x;
    int64_t n = n_tokens ? n_tokens[head / n_q] : N;
    n = n < 0 ? 0 : n < N ? n : N;
    const int have = (int)((n + span - 1) / span);           // parts with rows
    const float* rec = partials + head * parts * Q4_REC;
    const float m = tid < have ? rec[(size_t)tid * Q4_REC + RA_D] : -INFINITY, l = tid < have ? rec[(size_t)tid * Q4_REC + RA_D + 1] : 0.f;
    float mx = m;
#pragma unroll
    for (int d = 1; d < RA_WAVE; d <<= 1) mx = fmaxf(mx, __shfl_xor(mx, d));
    if (lane == 0) s_x[tid / RA_WAVE] = mx;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < Q4_MERGE_THREADS / RA_WAVE; ++w) mx = fmaxf(mx, s_x[w]);
    const float w = mx > -INFINITY ? __builtin_amdgcn_exp2f(m - mx) : 0.f;
    s_w[tid] = w;
    float ll = l * w;
#pragma unroll
    for (int d = 1; d < RA_WAVE; d <<= 1) ll += __shfl_xor(ll, d);
    __syncthreads();
    if (lane == 0) s_x[tid / RA_WAVE] = ll;
    float a = 0.f;
    constexpr int SL = Q4_MERGE_THREADS / RA_D;
#pragma unroll 8
    for (int i = slice; i < have; i += SL) a = fmaf(rec[(size_t)i * Q4_REC + t], s_w[i], a);
    s_a[slice][t] = a;
    __syncthreads();
    if (slice) return;
    ll = 0.f;
#pragma unroll
    for (int x = 0; x < Q4_MERGE_THREADS / RA_WAVE; ++x) ll += s_x[x];
#pragma unroll
    for (int x = 1; x < SL; ++x) a += s_a[x][t];
    out[head * RA_D + t] = mx > -INFINITY ? a / ll : 0.f;
    if (t == 0) lse[head] = mx > -INFINITY ? mx * Q4_LN2 + logf(ll) : -INFINITY;
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
// rows [at, at + 32) of a job; returns which of the lane's rows there are. Loads are never branched around: a row that is
// not there is row 0.
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

// Dimension d of a head from its records, nS of the static set and nG of Omega: Eq. 4 for each, Eq. 5 for both.
template <bool COHERENT>
__device__ __forceinline__ void q4_finish(const float* rec, int nS, int nG, size_t head, int d, const Q4Out& o) {
    float M[2] = {-INFINITY, -INFINITY}, L[2] = {0.f, 0.f}, A[2] = {0.f, 0.f};
    constexpr int FLY = 8;
#pragma unroll
    for (int set = 0; set < 2; ++set) {
        const int first = set ? nS : 0, last = set ? nS + nG : nS;
        for (int i0 = first; i0 < last; i0 += FLY) {
            float m[FLY], l[FLY], a[FLY];
#pragma unroll
            for (int u = 0; u < FLY; ++u) {
                const float* x = rec + (size_t)(i0 + u < last ? i0 + u : last - 1) * Q4_REC;
                m[u] = q4_load<COHERENT>(x + RA_D);
                l[u] = q4_load<COHERENT>(x + RA_D + 1);
                a[u] = q4_load<COHERENT>(x + d);
            }
            float mx = M[set];
#pragma unroll
            for (int u = 0; u < FLY; ++u) mx = fmaxf(mx, m[u]);
            if (mx == -INFINITY) continue;
            const float corr = __builtin_amdgcn_exp2f(M[set] - mx);
            A[set] *= corr;
            L[set] *= corr;
#pragma unroll
            for (int u = 0; u < FLY; ++u) {
                const float w = i0 + u < last ? __builtin_amdgcn_exp2f(m[u] - mx) : 0.f;
                A[set] = fmaf(a[u], w, A[set]);
                L[set] = fmaf(l[u], w, L[set]);
            }
            M[set] = mx;
        }
    }
    float* o_set[2] = {o.o_w, o.o_om};
    float* l_set[2] = {o.lse_w, o.lse_om};
#pragma unroll
    for (int set = 0; set < 2; ++set) {
        const bool empty = M[set] == -INFINITY;
        if (o_set[set]) o_set[set][head * RA_D + d] = empty ? 0.f : A[set] / L[set];
        if (l_set[set] && d == 0) l_set[set][head] = empty ? -INFINITY : M[set] * Q4_LN2 + logf(L[set]);
    }
    const float mx = fmaxf(M[0], M[1]);
    float out = 0.f, lse = -INFINITY;
    if (mx > -INFINITY) {
        const float e0 = __builtin_amdgcn_exp2f(M[0] - mx), e1 = __builtin_amdgcn_exp2f(M[1] - mx), l = L[0] * e0 + L[1] * e1;
        out = (A[0] * e0 + A[1] * e1) / l;
        lse = mx * Q4_LN2 + logf(l);
    }
    o.out[head * RA_D + d] = out;
    if (d == 0) o.lse[head] = lse;
}

// grid: per (sequence, KV head) the parts of each of its query heads' Omega (their loads wait for ids, so they start first), then
// the parts of the static set per tile of heads. `spanS`, `spanG`: rows of a part. TICKETS: the workgroup that stores a head's last
// record combines them all (ticket.h), which saves a launch.
template <int DT, bool TICKETS>
__global__ __launch_bounds__(Q4_THREADS) void q4_attend_kernel(const void* __restrict__ q, Q4Cache c, int n_q, int n_kv, int64_t N,
                                                               int64_t s, int64_t w, int topk, const int32_t* __restrict__ ids, int nS,
                                                               int nG, int spanS, int spanG, int tiles, float* partials, Q4Out o) {
    typedef Q4Form<DT> F;
    __shared__ Q4Lds lds;
    __shared__ uint32_t s_last[F::HEADS];
    const int tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid / RA_WAVE);
    const int group = n_q / n_kv, per = tiles * nS + group * nG, P = nS + nG;
    const size_t kv_head = blockIdx.x / per;
    const int x = blockIdx.x % per;
    const size_t group0 = kv_head / n_kv * n_q + kv_head % n_kv * group;
    const bool om = x < group * nG;
    const int first = om ? x / nG : (x - group * nG) / nS * F::HEADS;        // of the group's heads
    const int part = om ? x % nG : (x - group * nG) % nS, slot = om ? nS + part : part;
    const int heads = om ? 1 : group - first < F::HEADS ? group - first : F::HEADS;
    const size_t head0 = group0 + first;
    const Q4Cache h{c.k + kv_head * c.kv_stride * Q4_ROW, c.ks + kv_head * c.kv_stride * Q4_BLOCKS, c.v + kv_head * c.kv_stride * Q4_ROW,
                    c.vs + kv_head * c.kv_stride * Q4_BLOCKS, c.kv_stride};
    const Q4Rows src = om ? Q4Rows{ids + head0 * topk, N, 0, 0, topk} : Q4Rows{nullptr, N, s, w, (int)(s + N - w)};
    const int span = om ? spanG : spanS, from = part * span, to = from + span < src.count ? from + span : src.count;
    Q4Wave<DT> st;
    st.start(reinterpret_cast<const char*>(q) + head0 * RA_D * (DT == RA_BF16 ? 2 : 4), heads, lane);
    for (int at = from + wv * Q4_CHUNK; at < to; at += Q4_WAVES * Q4_CHUNK) {
        Q4Chunk ch;
        const uint32_t there = q4_gather(ch, h, src, at, lane);
        st.template add<false>(ch, there, lane);
    }
    q4_close<DT>(st, lds, heads, [&](int hd, int d, float sum, float mx, float l) {
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

// grid: x = head (with its sequence)
__global__ __launch_bounds__(RA_D) void q4_merge_kernel(const float* __restrict__ partials, int nS, int nG, Q4Out o) {
    const size_t head = blockIdx.x;
    q4_finish<false>(partials + head * (nS + nG) * Q4_REC, nS, nG, head, threadIdx.x, o);
}

// Rows of a part of all tokens, a multiple of what a workgroup's wavefronts take at once: parts for about four workgroups
// per compute unit, at least 256 rows each.
static int full_span(ra_dtype dt, int n_seq, int n_q, int n_kv, int64_t N, int* parts, int* tiles) {
    const int heads = dt == RA_BF16 ? Q4Form<RA_BF16>::HEADS : Q4Form<RA_F32>::HEADS;
    *tiles = (n_q / n_kv + heads - 1) / heads;
    const int64_t jobs = (int64_t)n_seq * n_kv * *tiles, unit = Q4_WAVES * Q4_CHUNK;
    int64_t want = (1024 + jobs - 1) / jobs;
    if (want > N / 256) want = N / 256;
    if (want > Q4_MAX_PARTS) want = Q4_MAX_PARTS;
    if (want < 1) want = 1;
    const int64_t span = ((N + want - 1) / want + unit - 1) / unit * unit;
    *parts = (int)((N + span - 1) / span);
    return (int)span;
}

size_t ra_full_q4_partial_floats(ra_dtype dt, int n_seq, int n_q, int n_kv, int64_t N) {
    int parts, tiles;
    full_span(dt, n_seq, n_q, n_kv, N, &parts, &tiles);
    return parts > 1 ? (size_t)n_seq * n_q * parts * Q4_REC : 0;
}

ra_status ra_launch_full_q4(const void* q, ra_dtype dt, const Q4Cache& c, int n_seq, int n_q, int n_kv, int64_t N,
                            const int32_t* n_tokens, float* partials, hipStream_t st, float* out, float* lse) {
    int parts, tiles;
    const int span = full_span(dt, n_seq, n_q, n_kv, N, &parts, &tiles);
    const int64_t blocks = (int64_t)n_seq * n_kv * tiles * ((parts + 7) / 8 * 8);
    if (blocks > (1 << 24) - 1) RA_FAIL(RA_EUNSUP, "too many (sequence, KV head) pairs for one launch");
    if (dt == RA_BF16)
        hipLaunchKernelGGL(q4_full_kernel<RA_BF16>, dim3((unsigned)blocks), dim3(Q4_THREADS), 0, st, q, c, n_q, n_kv, N, n_tokens, span,
                           parts, tiles, partials, out, lse);
    else
        hipLaunchKernelGGL(q4_full_kernel<RA_F32>, dim3((unsigned)blocks), dim3(Q4_THREADS), 0, st, q, c, n_q, n_kv, N, n_tokens, span,
                           parts, tiles, partials, out, lse);
    RA_HIP(hipGetLastError());
    if (parts == 1) return RA_OK;
    hipLaunchKernelGGL(q4_full_merge_kernel, dim3(n_seq * n_q), dim3(Q4_MERGE_THREADS), 0, st, partials, n_q, N, n_tokens, span, parts, out,
                       lse);
    RA_HIP(hipGetLastError());
    return RA_OK;
}

// W = [0, s) u [w, N) of Sec. 3.3, with what came after the index was built; ranges that meet make everything static
static void q4_static(int64_t N, int64_t Ng, int sink, int window, int64_t* s, int64_t* w) {
    *s = sink < N ? sink : N;
    *w = N - window < Ng ? N - window : Ng;
    if (*w <= *s) { *s = N; *w = N; }
}

// parts of the two sets: 128 rows each, a chunk for each wavefront of a workgroup; longer ones where they would be very many
struct Q4Parts { int nS, nG, spanS, spanG, tiles; };
static Q4Parts q4_parts(ra_dtype dt, int n_seq, int n_q, int n_kv, int64_t n_static, int topk) {
    const int heads = dt == RA_BF16 ? Q4Form<RA_BF16>::HEADS : Q4Form<RA_F32>::HEADS;
    Q4Parts p;
    p.tiles = (n_q / n_kv + heads - 1) / heads;
    p.spanG = Q4_PART;
    p.nG = (topk + p.spanG - 1) / p.spanG;
    int64_t most = 2048 / ((int64_t)n_seq * n_kv * p.tiles);
    if (most < 1) most = 1;
    int64_t nS = (n_static + Q4_PART - 1) / Q4_PART;
    if (nS > most) nS = most;
    if (nS < 1) nS = n_static > 0;
    p.spanS = nS ? (int)((n_static + nS - 1) / nS + Q4_PART - 1) / Q4_PART * Q4_PART : Q4_PART;
    p.nS = (int)((n_static + p.spanS - 1) / p.spanS);
    return p;
}

size_t ra_attend_q4_partial_floats(ra_dtype dt, int n_seq, int n_q, int n_kv, int64_t N, int64_t Ng, int sink, int window, int topk) {
    int64_t s, w;
    q4_static(N, Ng, sink, window, &s, &w);
    const Q4Parts p = q4_parts(dt, n_seq, n_q, n_kv, s + N - w, topk);
    return (size_t)n_seq * n_q * (p.nS + p.nG) * Q4_REC;
}

#define Q4_TICKET_RECORDS 512

ra_status ra_launch_attend_q4(const void* q, ra_dtype dt, const Q4Cache& c, int n_seq, int n_q, int n_kv, int64_t N, int64_t Ng,
                              int sink, int window, int topk, const int32_t* ids, float* partials, uint32_t* tickets,
                              hipStream_t st, float* out, float* lse, float* o_omega, float* lse_omega, float* o_w, float* lse_w) {
    int64_t s, w;
    q4_static(N, Ng, sink, window, &s, &w);
    const Q4Parts p = q4_parts(dt, n_seq, n_q, n_kv, s + N - w, topk);
    const int64_t blocks = (int64_t)n_seq * n_kv * (p.tiles * p.nS + n_q / n_kv * p.nG);
    if (blocks > (1 << 24) - 1) RA_FAIL(RA_EUNSUP, "too many heads for one launch");
    if ((int64_t)n_seq * n_q * (p.nS + p.nG) > Q4_TICKET_RECORDS) tickets = nullptr;
    const Q4Out o{tickets, out, lse, o_omega, lse_omega, o_w, lse_w};
#define Q4_GO(DTV, TK)                                                                                                       \
    hipLaunchKernelGGL((q4_attend_kernel<DTV, TK>), dim3((unsigned)blocks), dim3(Q4_THREADS), 0, st, q, c, n_q, n_kv, N, s, w, topk, ids, \
                       p.nS, p.nG, p.spanS, p.spanG, p.tiles, partials, o)
    if (dt == RA_BF16) { if (tickets) Q4_GO(RA_BF16, true); else Q4_GO(RA_BF16, false); }
    else { if (tickets) Q4_GO(RA_F32, true); else Q4_GO(RA_F32, false); }
#undef Q4_GO
    RA_HIP(hipGetLastError());
    if (tickets) return RA_OK;
    hipLaunchKernelGGL(q4_merge_kernel, dim3(n_seq * n_q), dim3(RA_D), 0, st, partials, p.nS, p.nG, o);
    RA_HIP(hipGetLastError());
    return RA_OK;
}
