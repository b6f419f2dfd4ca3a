// Tokens that enter a cache: norms of queries and keys per head, position rotation, the new rows (ra_append_tokens), and
// rows into 4 bits and back (ra_quantize_kv4, ra_dequantize_kv4). All of it moves rows: 16 lanes hold one row of 128 values, 8
// each, so a block of 32 dimensions is four lanes and the partner of a half-split rotation (a multiple of 8 dimensions away,
// rot_dim being one of 16) is 8 values of one other lane.
#include "q4_dev.h"

#define KV_THREADS 256
#define KV_GROUPS (KV_THREADS / 16)

// values [8 l16, 8 l16 + 8) of a row
template <int DT>
__device__ __forceinline__ void kv_load8(const void* row, int l16, float (&v)[8]) {
    if constexpr (DT == RA_BF16) {
        const uint4 u = reinterpret_cast<const uint4*>(row)[l16];
        v[0] = bf16_lo(u.x); v[1] = bf16_hi(u.x); v[2] = bf16_lo(u.y); v[3] = bf16_hi(u.y);
        v[4] = bf16_lo(u.z); v[5] = bf16_hi(u.z); v[6] = bf16_lo(u.w); v[7] = bf16_hi(u.w);
    } else {
        const float4 a = reinterpret_cast<const float4*>(row)[2 * l16], b = reinterpret_cast<const float4*>(row)[2 * l16 + 1];
        v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
    }
}
typedef __bf16 kv_bf16x8 __attribute__((ext_vector_type(8)));
// stores them, rounded to DT; v becomes what was stored
template <int DT>
__device__ __forceinline__ void kv_round8(float (&v)[8]) {
    if constexpr (DT == RA_BF16)
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = (float)(__bf16)v[e];
}
template <int DT>
__device__ __forceinline__ void kv_store8(void* row, int l16, const float (&v)[8]) {
    if constexpr (DT == RA_BF16) {
        kv_bf16x8 b;
#pragma unroll
        for (int e = 0; e < 8; ++e) b[e] = (__bf16)v[e];
        reinterpret_cast<uint4*>(row)[l16] = __builtin_bit_cast(uint4, b);
    } else {
        reinterpret_cast<float4*>(row)[2 * l16] = make_float4(v[0], v[1], v[2], v[3]);
        reinterpret_cast<float4*>(row)[2 * l16 + 1] = make_float4(v[4], v[5], v[6], v[7]);
    }
}
// A row of 16 lanes x 8 values into 4 bits. Called by whole groups of 16 lanes.
__device__ __forceinline__ void kv_store4(uint8_t* codes, uint8_t* scale, int l16, int lane, const float (&v)[8]) {
    uint32_t m = 0u;                                   // magnitudes compare like their bits, a NaN above all
#pragma unroll
    for (int e = 0; e < 8; ++e) m = max(m, __float_as_uint(v[e]) & 0x7fffffffu);
    m = max(m, lane_xor32<1>(m, lane));
    m = max(m, lane_xor32<2>(m, lane));
    const uint32_t byte = q4_scale_byte(m);
    reinterpret_cast<uint32_t*>(codes)[l16] = q4_codes(v, byte);
    if ((l16 & 3) == 0) scale[l16 / 4] = (uint8_t)byte;
}

// One workgroup per token: the sines and cosines of its angles, then its heads' rows, one per 16 lanes.
template <int DT>
__global__ __launch_bounds__(KV_THREADS) void append_kernel(AppendArgs a) {
    __shared__ float2 s_cs[RA_D / 2];
    const int tid = threadIdx.x, lane = tid & (RA_WAVE - 1), l16 = tid & 15, grp = tid >> 4;
    const size_t esz = DT == RA_BF16 ? 2 : 4;
    const int64_t tok = blockIdx.x, seq = tok / a.T, t = tok % a.T;
    if (a.n_new && t >= a.n_new[seq]) return;                       // (uniform)
    const int64_t pos = (a.first ? a.first[seq] : 0) + t;
    const int rot = a.rot, half = rot / 2;
    if (tid < half) {
        double s, c;
        sincos((double)pos * (double)a.inv_freq[tid], &s, &c);
        s_cs[tid] = make_float2((float)c, (float)s);
    }
    __syncthreads();
    const int n_rows = a.n_q + 2 * a.n_kv;
    for (int r = grp; r < n_rows; r += KV_GROUPS) {
        const int which = r < a.n_q ? 0 : r < a.n_q + a.n_kv ? 1 : 2;
        const int h = which == 0 ? r : which == 1 ? r - a.n_q : r - a.n_q - a.n_kv;
        const char* in = reinterpret_cast<const char*>(a.in[which]);
        const bool row_there = pos >= 0 && pos < a.stride[0], row4_there = pos >= 0 && pos < a.stride[1];
        if (!in || (which && !row_there && !row4_there)) continue;
        float v[8];
        kv_load8<DT>(in + ((size_t)tok * a.row[which] + (size_t)h * RA_D) * esz, l16, v);
        if (which < 2) {
            if (const void* weight = a.weight[which]) {
                double sum = 0.;
#pragma unroll
                for (int e = 0; e < 8; ++e) sum += (double)v[e] * (double)v[e];
#pragma unroll
                for (int d = 1; d < 16; d <<= 1) sum += __shfl_xor(sum, d);
                const float rinv = (float)(1.0 / sqrt(sum / RA_D + a.eps));
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int d = 8 * l16 + e;
                    const float w = DT == RA_BF16 ? bf16_lo(reinterpret_cast<const uint16_t*>(weight)[d])
                                                  : reinterpret_cast<const float*>(weight)[d];
                    v[e] = v[e] * rinv * w;
                }
            }
            if (a.interleaved) {
                if (8 * l16 < rot)
#pragma unroll
                    for (int e = 0; e < 8; e += 2) {
                        const float2 cs = s_cs[4 * l16 + e / 2];
                        const float x = v[e], y = v[e + 1];
                        v[e] = x * cs.x - y * cs.y;
                        v[e + 1] = y * cs.x + x * cs.y;
                    }
            } else if (rot) {
                const int step = half / 8;
                const bool low = l16 < step, in_rot = l16 < 2 * step;
                const int from = (lane & ~15) + (low ? l16 + step : in_rot ? l16 - step : l16);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float other = __shfl(v[e], from);
                    if (in_rot) {
                        const float2 cs = s_cs[8 * (low ? l16 : l16 - step) + e];
                        v[e] = low ? v[e] * cs.x - other * cs.y : v[e] * cs.x + other * cs.y;
                    }
                }
            }
            kv_round8<DT>(v);
        }
        if (which == 0) {
            kv_store8<DT>(reinterpret_cast<char*>(a.out[0]) + (((size_t)seq * a.n_q + h) * a.T + t) * RA_D * esz, l16, v);
        } else {
            const size_t head = (size_t)seq * a.n_kv + h, row = head * a.stride[0] + pos, row4 = head * a.stride[1] + pos;
            if (a.out[which] && row_there) kv_store8<DT>(reinterpret_cast<char*>(a.out[which]) + row * RA_D * esz, l16, v);
            if (a.codes[which - 1] && row4_there)
                kv_store4(a.codes[which - 1] + row4 * Q4_ROW, a.scale[which - 1] + row4 * Q4_BLOCKS, l16, lane, v);
        }
    }
}

ra_status ra_launch_append(const AppendArgs& a, ra_dtype dt, hipStream_t st) {
    const int64_t blocks = a.T * a.n_seq;
    if (blocks > (1u << 24) - 1) RA_FAIL(RA_EUNSUP, "more than 2^24 - 1 tokens in a call");
    if (dt == RA_BF16) hipLaunchKernelGGL(append_kernel<RA_BF16>, dim3((unsigned)blocks), dim3(KV_THREADS), 0, st, a);
    else hipLaunchKernelGGL(append_kernel<RA_F32>, dim3((unsigned)blocks), dim3(KV_THREADS), 0, st, a);
    RA_HIP(hipGetLastError());
    return RA_OK;
}

// grid: x = rows of a head, 16 to a workgroup, y = head (with its sequence)
template <int DT>
__global__ __launch_bounds__(KV_THREADS) void quantize_kv4_kernel(const void* __restrict__ X, int n_kv, int64_t T,
                                                                  const int32_t* __restrict__ first, const int32_t* __restrict__ n_new,
                                                                  int64_t kv_stride, uint8_t* __restrict__ codes,
                                                                  uint8_t* __restrict__ scale) {
    const int tid = threadIdx.x, lane = tid & (RA_WAVE - 1), l16 = tid & 15;
    const size_t head = blockIdx.y;
    const int seq = (int)(head / n_kv);
    const int64_t t = (int64_t)blockIdx.x * KV_GROUPS + (tid >> 4), at = t + (first ? first[seq] : 0);
    if (t >= T || (n_new && t >= n_new[seq]) || at < 0 || at >= kv_stride) return;
    float v[8];
    kv_load8<DT>(reinterpret_cast<const char*>(X) + (head * T + t) * RA_D * (DT == RA_BF16 ? 2 : 4), l16, v);
    const size_t row = head * kv_stride + at;
    kv_store4(codes + row * Q4_ROW, scale + row * Q4_BLOCKS, l16, lane, v);
}

template <int DT>
__global__ __launch_bounds__(KV_THREADS) void dequantize_kv4_kernel(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scale,
                                                                    int n_kv, int64_t T, const int32_t* __restrict__ first,
                                                                    int64_t kv_stride, void* __restrict__ X) {
    const int tid = threadIdx.x, l16 = tid & 15;
    const size_t head = blockIdx.y;
    const int seq = (int)(head / n_kv);
    const int64_t t = (int64_t)blockIdx.x * KV_GROUPS + (tid >> 4), at = t + (first ? first[seq] : 0);
    if (t >= T) return;
    float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (at >= 0 && at < kv_stride) {
        const size_t row = head * kv_stride + at;
        q4_values(reinterpret_cast<const uint32_t*>(codes + row * Q4_ROW)[l16], q4_unit(scale[row * Q4_BLOCKS + l16 / 4]), v);
    }
    kv_store8<DT>(reinterpret_cast<char*>(X) + (head * T + t) * RA_D * (DT == RA_BF16 ? 2 : 4), l16, v);
}

static ra_status rows_grid(int n_seq, int n_kv, int64_t T, dim3* grid) {
    const int64_t heads = (int64_t)n_seq * n_kv, blocks = (T + KV_GROUPS - 1) / KV_GROUPS;
    if (heads > 65535) RA_FAIL(RA_EUNSUP, "more than 65535 (sequence, KV head) pairs");
    if (blocks > (1 << 24) - 1) RA_FAIL(RA_EUNSUP, "T too large");
    *grid = dim3((unsigned)blocks, (unsigned)heads);
    return RA_OK;
}

ra_status ra_launch_quantize_kv4(const void* X, ra_dtype dt, int n_seq, int n_kv, int64_t T, const int32_t* first,
                                 const int32_t* n_new, int64_t kv_stride, hipStream_t st, uint8_t* codes, uint8_t* scale) {
    dim3 grid;
    const ra_status rc = rows_grid(n_seq, n_kv, T, &grid);
    if (rc != RA_OK) return rc;
    if (dt == RA_BF16)
        hipLaunchKernelGGL(quantize_kv4_kernel<RA_BF16>, grid, dim3(KV_THREADS), 0, st, X, n_kv, T, first, n_new, kv_stride, codes, scale);
    else
        hipLaunchKernelGGL(quantize_kv4_kernel<RA_F32>, grid, dim3(KV_THREADS), 0, st, X, n_kv, T, first, n_new, kv_stride, codes, scale);
    RA_HIP(hipGetLastError());
    return RA_OK;
}

ra_status ra_launch_dequantize_kv4(const uint8_t* codes, const uint8_t* scale, ra_dtype dt, int n_seq, int n_kv, int64_t T,
                                   const int32_t* first, int64_t kv_stride, hipStream_t st, void* X) {
    dim3 grid;
    const ra_status rc = rows_grid(n_seq, n_kv, T, &grid);
    if (rc != RA_OK) return rc;
    if (dt == RA_BF16)
        hipLaunchKernelGGL(dequantize_kv4_kernel<RA_BF16>, grid, dim3(KV_THREADS), 0, st, codes, scale, n_kv, T, first, kv_stride, X);
    else
        hipLaunchKernelGGL(dequantize_kv4_kernel<RA_F32>, grid, dim3(KV_THREADS), 0, st, codes, scale, n_kv, T, first, kv_stride, X);
    RA_HIP(hipGetLastError());
    return RA_OK;
}
