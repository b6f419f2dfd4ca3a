// Attention over a cache in 4 bits: all tokens (ra_full_attention_q4), and the retrieved set Omega and the static set W of
// Sec. 3.3 with their combination by Eq. 4-5 (ra_attend_q4).
//
// Rows are cut into parts; a workgroup turns one part into a record (128 weighted sums, the running maximum of
// z log2(e), the sum of weights), and a second kernel combines a head's records. Weights are powers of two,
// p = 2^(c <q, k> - m) with c = log2(e) / sqrt(d): one multiply-add and one instruction each.
#include "q4_dev.h"

#define Q4_THREADS 256
#define Q4_GROUPS (Q4_THREADS / 16)
#define Q4_REC (RA_D + 4)           // floats of a record: sums, maximum, sum of weights, 2 pad
#define Q4_PART 128                 // rows of a part of the sparse set
#define Q4_LONG 1024                // rows of a part of all tokens
#define Q4_C (1.4426950408889634f * 0.08838834764831845f)
#define Q4_LN2 0.6931471805599453f

// the rows of a job: ids of a head, or [0, s) and then from `w` on
struct Q4Rows {
    const int32_t* ids;
    int64_t N, s, w, count;
};
__device__ __forceinline__ int64_t q4_row(const Q4Rows& src, int64_t r) {
    if (src.ids) {
        const int64_t id = src.ids[r];
        return id < src.N ? id : -1;
    }
    return r < src.s ? r : src.w + (r - src.s);
}

template <int DT>
__device__ __forceinline__ void q4_part(const void* q, const Q4Cache& c, size_t kv_head, const Q4Rows& src, int64_t from, int64_t to,
                                        float* rec) {
    __shared__ float s_m[Q4_GROUPS], s_l[Q4_GROUPS], s_a[Q4_GROUPS][RA_D];
    const int tid = threadIdx.x, grp = tid >> 4, l16 = tid & 15;
    float qv[8];
#pragma unroll
    for (int e = 0; e < 8; ++e)
        qv[e] = DT == RA_BF16 ? bf16_lo(reinterpret_cast<const uint16_t*>(q)[8 * l16 + e]) : reinterpret_cast<const float*>(q)[8 * l16 + e];
    float m = -INFINITY, l = 0.f, acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    for (int64_t r = from + grp; r < to; r += Q4_GROUPS) {
        const int64_t id = q4_row(src, r);
        if (id < 0) continue;
        const size_t row = kv_head * c.kv_stride + id;
        float k[8], v[8];
        q4_values(reinterpret_cast<const uint32_t*>(c.k + row * Q4_ROW)[l16], q4_unit(c.ks[row * Q4_BLOCKS + l16 / 4]), k);
        q4_values(reinterpret_cast<const uint32_t*>(c.v + row * Q4_ROW)[l16], q4_unit(c.vs[row * Q4_BLOCKS + l16 / 4]), v);
        float dot = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) dot = fmaf(qv[e], k[e], dot);
#pragma unroll
        for (int d = 1; d < 16; d <<= 1) dot += __shfl_xor(dot, d);
        const float z = dot * Q4_C, mn = fmaxf(m, z), base = mn == -INFINITY ? 0.f : mn;
        const float corr = exp2f(m - base), p = exp2f(z - base);
        m = mn;
        l = l * corr + p;
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[e] = fmaf(p, v[e], acc[e] * corr);
    }
    // (a sum that is not a number keeps a maximum that is one, or its record would count as empty)
    if (l != l) m = 0.f;
    if (l16 == 0) { s_m[grp] = m; s_l[grp] = l; }
#pragma unroll
    for (int e = 0; e < 8; ++e) s_a[grp][8 * l16 + e] = acc[e];
    __syncthreads();
    if (tid < RA_D) {
        float mx = -INFINITY, a = 0.f, ll = 0.f;
        for (int g = 0; g < Q4_GROUPS; ++g) mx = fmaxf(mx, s_m[g]);
        for (int g = 0; g < Q4_GROUPS; ++g)
            if (s_m[g] > -INFINITY) {
                const float w = exp2f(s_m[g] - mx);
                a = fmaf(s_a[g][tid], w, a);
                ll = fmaf(s_l[g], w, ll);
            }
        rec[tid] = a;
        if (tid == 0) { rec[RA_D] = mx; rec[RA_D + 1] = ll; }
    }
}

// grid: x = part, y = query head, z = sequence
template <int DT>
__global__ __launch_bounds__(Q4_THREADS) void q4_full_kernel(const void* __restrict__ q, Q4Cache c, int n_q, int n_kv, int64_t N,
                                                             const int32_t* __restrict__ n_tokens, float* __restrict__ partials) {
    const int x = blockIdx.x, h = blockIdx.y, seq = blockIdx.z;
    int64_t n = n_tokens ? n_tokens[seq] : N;
    n = n < 0 ? 0 : n < N ? n : N;
    const size_t head = (size_t)seq * n_q + h;
    const int64_t from = (int64_t)x * Q4_LONG, to = from + Q4_LONG < n ? from + Q4_LONG : n;
    q4_part<DT>(reinterpret_cast<const char*>(q) + head * RA_D * (DT == RA_BF16 ? 2 : 4), c, (size_t)seq * n_kv + h / (n_q / n_kv),
                Q4Rows{nullptr, N, N, 0, n}, from, to, partials + (head * gridDim.x + x) * Q4_REC);
}

template <int DT>
__global__ __launch_bounds__(Q4_THREADS) void q4_attend_kernel(const void* __restrict__ q, Q4Cache c, int n_q, int n_kv, int64_t N,
                                                               int64_t s, int64_t w, int topk, const int32_t* __restrict__ ids, int nS,
                                                               float* __restrict__ partials) {
    const int x = blockIdx.x, h = blockIdx.y, seq = blockIdx.z;
    const size_t head = (size_t)seq * n_q + h;
    const Q4Rows src = x < nS ? Q4Rows{nullptr, N, s, w, s + N - w} : Q4Rows{ids + head * topk, N, 0, 0, topk};
    const int64_t from = (int64_t)(x < nS ? x : x - nS) * Q4_PART, to = from + Q4_PART < src.count ? from + Q4_PART : src.count;
    q4_part<DT>(reinterpret_cast<const char*>(q) + head * RA_D * (DT == RA_BF16 ? 2 : 4), c, (size_t)seq * n_kv + h / (n_q / n_kv), src,
                from, to, partials + (head * gridDim.x + x) * Q4_REC);
}

struct Q4Out { float *out, *lse, *o_om, *lse_om, *o_w, *lse_w; };

// grid: x = head (with its sequence); records of the static set (0) and then of Omega (1)
__global__ __launch_bounds__(RA_D) void q4_merge_kernel(const float* __restrict__ partials, int nS, int nG, Q4Out o) {
    const size_t head = blockIdx.x;
    const int t = threadIdx.x;
    const float* rec = partials + head * (nS + nG) * Q4_REC;
    float M[2] = {-INFINITY, -INFINITY}, L[2] = {0.f, 0.f}, A[2] = {0.f, 0.f};
#pragma unroll
    for (int set = 0; set < 2; ++set)
        for (int i = set ? nS : 0; i < (set ? nS + nG : nS); ++i) {
            const float m = rec[(size_t)i * Q4_REC + RA_D];
            if (m == -INFINITY) continue;
            const float mx = fmaxf(M[set], m), c0 = exp2f(M[set] - mx), c1 = exp2f(m - mx);
            A[set] = A[set] * c0 + rec[(size_t)i * Q4_REC + t] * c1;
            L[set] = L[set] * c0 + rec[(size_t)i * Q4_REC + RA_D + 1] * c1;
            M[set] = mx;
        }
    float* o_set[2] = {o.o_w, o.o_om};
    float* l_set[2] = {o.lse_w, o.lse_om};
#pragma unroll
    for (int set = 0; set < 2; ++set) {
        const bool empty = M[set] == -INFINITY;
        if (o_set[set]) o_set[set][head * RA_D + t] = empty ? 0.f : A[set] / L[set];
        if (l_set[set] && t == 0) l_set[set][head] = empty ? -INFINITY : M[set] * Q4_LN2 + logf(L[set]);
    }
    const float mx = fmaxf(M[0], M[1]);
    float out = 0.f, lse = -INFINITY;
    if (mx > -INFINITY) {
        const float e0 = exp2f(M[0] - mx), e1 = exp2f(M[1] - mx), l = L[0] * e0 + L[1] * e1;
        out = (A[0] * e0 + A[1] * e1) / l;
        lse = mx * Q4_LN2 + logf(l);
    }
    o.out[head * RA_D + t] = out;
    if (t == 0) o.lse[head] = lse;
}

size_t ra_full_q4_partial_floats(ra_dtype, int n_seq, int n_q, int, int64_t N) {
    return (size_t)n_seq * n_q * ((N + Q4_LONG - 1) / Q4_LONG) * Q4_REC;
}

ra_status ra_launch_full_q4(const void* q, ra_dtype dt, const Q4Cache& c, int n_seq, int n_q, int n_kv, int64_t N,
                            const int32_t* n_tokens, float* partials, hipStream_t st, float* out, float* lse) {
    const int parts = (int)((N + Q4_LONG - 1) / Q4_LONG);
    const dim3 grid(parts, n_q, n_seq);
    if (dt == RA_BF16) hipLaunchKernelGGL(q4_full_kernel<RA_BF16>, grid, dim3(Q4_THREADS), 0, st, q, c, n_q, n_kv, N, n_tokens, partials);
    else hipLaunchKernelGGL(q4_full_kernel<RA_F32>, grid, dim3(Q4_THREADS), 0, st, q, c, n_q, n_kv, N, n_tokens, partials);
    RA_HIP(hipGetLastError());
    hipLaunchKernelGGL(q4_merge_kernel, dim3(n_seq * n_q), dim3(RA_D), 0, st, partials, parts, 0,
                       Q4Out{out, lse, nullptr, nullptr, nullptr, nullptr});
    RA_HIP(hipGetLastError());
    return RA_OK;
}

// W = [0, s) u [w, N) of Sec. 3.3, with what came after the index was built; ranges that meet make everything static
static void q4_static(int64_t N, int64_t Ng, int sink, int window, int64_t* s, int64_t* w) {
    *s = sink < N ? sink : N;
    *w = N - window < Ng ? N - window : Ng;
    if (*w <= *s) { *s = N; *w = N; }
}

size_t ra_attend_q4_partial_floats(ra_dtype, int n_seq, int n_q, int, int64_t N, int64_t Ng, int sink, int window, int topk) {
    int64_t s, w;
    q4_static(N, Ng, sink, window, &s, &w);
    return (size_t)n_seq * n_q * ((s + N - w + Q4_PART - 1) / Q4_PART + (topk + Q4_PART - 1) / Q4_PART) * Q4_REC;
}

ra_status ra_launch_attend_q4(const void* q, ra_dtype dt, const Q4Cache& c, int n_seq, int n_q, int n_kv, int64_t N, int64_t Ng,
                              int sink, int window, int topk, const int32_t* ids, float* partials, uint32_t* tickets,
                              hipStream_t st, float* out, float* lse, float* o_omega, float* lse_omega, float* o_w, float* lse_w) {
    (void)tickets;
    int64_t s, w;
    q4_static(N, Ng, sink, window, &s, &w);
    const int nS = (int)((s + N - w + Q4_PART - 1) / Q4_PART), nG = (topk + Q4_PART - 1) / Q4_PART;
    const dim3 grid(nS + nG, n_q, n_seq);
    if (dt == RA_BF16)
        hipLaunchKernelGGL(q4_attend_kernel<RA_BF16>, grid, dim3(Q4_THREADS), 0, st, q, c, n_q, n_kv, N, s, w, topk, ids, nS, partials);
    else
        hipLaunchKernelGGL(q4_attend_kernel<RA_F32>, grid, dim3(Q4_THREADS), 0, st, q, c, n_q, n_kv, N, s, w, topk, ids, nS, partials);
    RA_HIP(hipGetLastError());
    hipLaunchKernelGGL(q4_merge_kernel, dim3(n_seq * n_q), dim3(RA_D), 0, st, partials, nS, nG,
                       Q4Out{out, lse, o_omega, lse_omega, o_w, lse_w});
    RA_HIP(hipGetLastError());
    return RA_OK;
}
