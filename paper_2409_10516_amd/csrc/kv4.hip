// Tokens that enter a cache: norms of queries and keys per head, position rotation, the new rows (ra_append_tokens), and
// rows into 4 bits and back (ra_quantize_kv4, ra_dequantize_kv4). All of it moves rows: a lane has 16 bytes of one, 8 values of bfloat16 in
// 16 lanes or 4 of float32 in 32, so that an instruction reads or writes whole lines (float32 rows in 16 lanes, two instructions
// for halves of a line's every 32 bytes: 32674 x 5 x 2 of them into 4 bits and back 99.7 us). A block of 32 dimensions is four or eight lanes, and
// the partner of a half-split rotation (a multiple of 8 dimensions away, rot_dim being one of 16) is the same value of another lane.
#include "q4_dev.h"

#define KV_THREADS 256
template <int DT> constexpr int KV_VALS = DT == RA_BF16 ? 8 : 4;        // of a lane
template <int DT> constexpr int KV_LANES = RA_D / KV_VALS<DT>;          // of a row

// A lane's values of a row, as loaded. Rows are written once: non-temporal (131072 rows of 8 heads into 4 bits and back 116 -> 107
// us, a 32K prompt's rows 159 -> 154, 2000 tokens 15.1 -> 13.5). They are read once, too, but what a call reads has just been made, and up to a
// quarter of what the memory side keeps is taken from there (us with ONCE and without: 5105 tokens of 10 float32 heads, 26 MB, 15.5,
// 13.5, 32768 rows of 8 heads, 64 MB, 30.9, 28.2, 8000 tokens of 48 heads, 98 MB, 42.5, 44.8, a 32K prompt 154, 157; as a choice at
// run time it costs the large ones 3 %).
#define KV_KEPT (1 << 26)           // bytes read
typedef uint32_t kv_u32x4 __attribute__((ext_vector_type(4)));
template <bool ONCE>
__device__ __forceinline__ kv_u32x4 kv_load(const void* row, int l) {
    const kv_u32x4* from = reinterpret_cast<const kv_u32x4*>(row) + l;
    if constexpr (ONCE) return __builtin_nontemporal_load(from);
    else return *from;
}
__device__ __forceinline__ void kv_store(void* row, int l, kv_u32x4 x) {
    __builtin_nontemporal_store(x, reinterpret_cast<kv_u32x4*>(row) + l);
}
template <int DT>
__device__ __forceinline__ void kv_floats(kv_u32x4 x, float (&v)[KV_VALS<DT>]) {
#pragma unroll
    for (int e = 0; e < KV_VALS<DT>; ++e) {
        if constexpr (DT == RA_BF16) v[e] = e & 1 ? bf16_hi(x[e / 2]) : bf16_lo(x[e / 2]);
        else v[e] = __uint_as_float(x[e]);
    }
}
typedef __bf16 kv_bf16x8 __attribute__((ext_vector_type(8)));
// rounded to DT
template <int DT>
__device__ __forceinline__ kv_u32x4 kv_pack(const float (&v)[KV_VALS<DT>]) {
    if constexpr (DT == RA_BF16) {
        kv_bf16x8 b;
#pragma unroll
        for (int e = 0; e < 8; ++e) b[e] = (__bf16)v[e];
        return __builtin_bit_cast(kv_u32x4, b);
    } else {
        return kv_u32x4{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
    }
}
// A row into 4 bits. Called by all of its lanes.
template <int DT>
__device__ __forceinline__ void kv_store4(uint8_t* codes, uint8_t* scale, int l, int lane, const float (&v)[KV_VALS<DT>]) {
    uint32_t m = 0u;                                   // magnitudes compare like their bits, a NaN above all
#pragma unroll
    for (int e = 0; e < KV_VALS<DT>; ++e) m = max(m, __float_as_uint(v[e]) & 0x7fffffffu);
    m = max(m, lane_xor32<1>(m, lane));
    m = max(m, lane_xor32<2>(m, lane));
    if constexpr (DT == RA_F32) m = max(m, lane_xor32<4>(m, lane));
    const uint32_t byte = q4_scale_byte(m), w = q4_codes(v, byte);
    if constexpr (DT == RA_F32) reinterpret_cast<uint16_t*>(codes)[l] = (uint16_t)w;
    else reinterpret_cast<uint32_t*>(codes)[l] = w;
    uint32_t all = byte << (8 * (l / (32 / KV_VALS<DT>)));       // the four blocks' bytes, in one word
    if constexpr (DT == RA_BF16) all |= lane_xor32<4>(all, lane);
    all |= lane_xor32<8>(all, lane);
    if constexpr (DT == RA_F32) all |= lane_xor32<16>(all, lane);
    if (l == 0) *reinterpret_cast<uint32_t*>(scale) = all;
}

__device__ __forceinline__ double xor_add(double x, uint32_t lo, uint32_t hi) {
    return x + __hiloint2double((int)hi, (int)lo);
}
// sum over a row's lanes, the same in all of them
template <int LANES>
__device__ __forceinline__ double row_sum(double x, int lane) {
    uint32_t lo, hi;
#define KV_STEP(J)                                                                             \
    lo = (uint32_t)__double2loint(x); hi = (uint32_t)__double2hiint(x);                        \
    x = xor_add(x, lane_xor32<J>(lo, lane), lane_xor32<J>(hi, lane));
    KV_STEP(1) KV_STEP(2) KV_STEP(4) KV_STEP(8)
    if constexpr (LANES == 32) { KV_STEP(16) }
#undef KV_STEP
    return x;
}

// 1 / sqrt(x) to the last few bits of a double: the hardware's estimate and one step of Newton's method
__device__ __forceinline__ double rsqrt64(double x) {
    const double y = __builtin_amdgcn_rsq(x), z = y * fma(-0.5 * x * y, y, 1.5);
    return y > 0. && y < INFINITY ? z : y;               // (zero and infinity are their own)
}

// The sine and cosine of x, to float32: x less the nearest multiple of pi / 2, in two parts, and the series of both about zero,
// to terms below 2^-44 of the result at pi / 4.
__device__ __forceinline__ float2 cos_sin64(double x) {
    const double n = rint(x * 0.63661977236758134308);
    const double r = fma(-n, 6.123233995736766036e-17, fma(-n, 1.57079632679489655800, x)), t = r * r;
    double s = fma(t, 1. / 6227020800., -1. / 39916800.), c = fma(t, -1. / 87178291200., 1. / 479001600.);
    s = fma(t, s, 1. / 362880.); c = fma(t, c, -1. / 3628800.);
    s = fma(t, s, -1. / 5040.); c = fma(t, c, 1. / 40320.);
    s = fma(t, s, 1. / 120.); c = fma(t, c, -1. / 720.);
    s = fma(t, s, -1. / 6.); c = fma(t, c, 1. / 24.);
    s = fma(t * r, s, r); c = fma(t, c, -0.5);
    c = fma(t, c, 1.);
    const int k = (int)((long long)n & 3);               // quarter turns
    const float fs = (float)(k & 1 ? c : s), fc = (float)(k & 1 ? s : c);
    return make_float2(k == 1 || k == 2 ? -fc : fc, k & 2 ? -fs : fs);
}

// Rotation of a row: a value times its cosine plus its pair's other value times its sine, which is negative for a pair's first. The other
// value is in the same lane for neighbouring pairs, else STEP lanes away (0: in lane `from`).
template <int STEP, int VALS>
__device__ __forceinline__ void turn(float (&v)[VALS], const float2 (&cs)[VALS], bool in_rot, int lane, int from) {
    float other[VALS];
#pragma unroll
    for (int e = 0; e < VALS; ++e) {
        if constexpr (STEP < 0) other[e] = v[e ^ 1];
        else if constexpr (STEP == 0) other[e] = __shfl(v[e], from);
        else other[e] = __uint_as_float(lane_xor32<STEP>(__float_as_uint(v[e]), lane));
    }
#pragma unroll
    for (int e = 0; e < VALS; ++e) {
        float x = v[e] * cs[e].x + other[e] * cs[e].y;
        asm("" : "+v"(x));                                         // (not to be worked out behind a branch)
        v[e] = in_rot ? x : v[e];
    }
}

// A workgroup takes a token, or with few tokens, one of `split` parts of its heads: the sines and cosines of the token's angles, one
// per lane of its first wavefront, then the heads' rows, one per group of lanes. What bounds it is how many rows are on their way, hence
// registers for eight wavefronts per SIMD and nothing asked for ahead, and next the vector instructions of a row.
// A 32K prompt of 32 + 8 + 8 normed heads, 150 us (5.4 TB/s; without norm and rotation 145). Held to seven wavefronts, six, five or four
// 206, 223, 248, 283 of then 192; that 192 had a branch and a wait for shared memory per rotated value, with a branch around
// both sides of a rotation it was 165. Two, four, eight or 16 tokens side by side in a workgroup 197, 200, 200, 205 of 192. With 512
// threads 211, 768 273 (a turn that is not full is a longer one).
template <int DT, int THREADS, bool ONCE>
__global__ __launch_bounds__(THREADS, 8) void append_kernel(AppendArgs a, int split) {
    __shared__ float2 s_cs[RA_D / 2];
    __shared__ float4 s_w[2][RA_D / 4];
    constexpr int VALS = KV_VALS<DT>, LANES = KV_LANES<DT>, GROUPS = THREADS / LANES;
    const int tid = threadIdx.x, lane = tid & (RA_WAVE - 1), l = tid % LANES, grp = tid / LANES;
    const size_t esz = DT == RA_BF16 ? 2 : 4;
    const int T = (int)a.T, tok = blockIdx.x / split, seq = tok / T, t = tok % T;
    if (a.n_new && t >= a.n_new[seq]) return;                       // (uniform)
    const int64_t pos = (int64_t)(a.first ? a.first[seq] : 0) + t;
    const bool there[2] = {pos >= 0 && pos < a.stride[0], pos >= 0 && pos < a.stride[1]};
    const int n_rows = a.n_q + 2 * a.n_kv, step = GROUPS * split, rot = a.rot, half = rot / 2;
    // where the token's rows are, head 0's (none: no such input or output)
    auto at = [&](const void* p, size_t row) { return p ? reinterpret_cast<char*>(const_cast<void*>(p)) + row * esz : nullptr; };
    const char *in_q = at(a.in[0], tok * a.row[0]), *in_k = at(a.in[1], tok * a.row[1]), *in_v = at(a.in[2], tok * a.row[2]);
    char* out_q = at(a.out[0], ((size_t)seq * a.n_q * T + t) * RA_D);
    const size_t row0 = (size_t)seq * a.n_kv * a.stride[0] + pos, head4 = (size_t)seq * a.n_kv * a.stride[1] + pos;
    char *out_k = at(a.out[1], row0 * RA_D), *out_v = at(a.out[2], row0 * RA_D);
    if (tid < half) s_cs[tid] = cos_sin64((double)pos * (double)a.inv_freq[tid]);
#pragma unroll
    for (int i = 0; i < 2; ++i)
        if (a.weight[i])                                           // (the last wavefronts first: the angles are the first one's)
            for (int d = THREADS - 1 - tid; d < RA_D; d += THREADS)
                reinterpret_cast<float*>(s_w[i])[d] = DT == RA_BF16 ? bf16_lo(reinterpret_cast<const uint16_t*>(a.weight[i])[d])
                                                                    : reinterpret_cast<const float*>(a.weight[i])[d];
    __syncthreads();
    const int near = half / VALS;                                  // lanes of a half
    const bool low = l < near, in_rot = l < 2 * near;
    const int from = lane - l + (low ? l + near : in_rot ? l - near : l);
    float2 cs[VALS];                                               // of the lane's dimensions, whatever the row
    if (rot) {
        const float2* at = s_cs + (!in_rot ? 0 : a.interleaved ? VALS / 2 * l : VALS * (low ? l : l - near));
#pragma unroll
        for (int e = 0; e < VALS; ++e) {
            cs[e] = at[a.interleaved ? e / 2 : e];
            if (a.interleaved ? !(e & 1) : low) cs[e].y = -cs[e].y;
        }
    }
    for (int r = grp + (int)(blockIdx.x % split) * GROUPS; r < n_rows; r += step) {
        const int which = r < a.n_q ? 0 : r < a.n_q + a.n_kv ? 1 : 2;
        const int h = which == 0 ? r : which == 1 ? r - a.n_q : r - a.n_q - a.n_kv;
        const char* in = which == 0 ? in_q : which == 1 ? in_k : in_v;
        if (!in || (which && !there[0] && !there[1])) continue;
        kv_u32x4 row = kv_load<ONCE>(in + (uint64_t)(uint32_t)h * (RA_D * esz), l);
        if (which < 2) {
            float v[VALS];
            kv_floats<DT>(row, v);
            if (a.weight[which]) {
                double sum = 0.;
#pragma unroll
                for (int e = 0; e < VALS; ++e) sum = fma((double)v[e], (double)v[e], sum);
                double r64 = rsqrt64(row_sum<LANES>(sum, lane) * (1. / RA_D) + a.eps);
                if (r64 > 0x1p100 || r64 < 0x1p-100) {             // (near or past float32's ends: the values take a part of it, exactly)
                    const bool tiny = r64 > 1.;
#pragma unroll
                    for (int e = 0; e < VALS; ++e) v[e] *= tiny ? 0x1p64f : 0x1p-64f;
                    r64 *= tiny ? 0x1p-64 : 0x1p64;
                }
                const float rinv = (float)r64;
#pragma unroll
                for (int f = 0; f < VALS / 4; ++f) {
                    const float4 w = s_w[which][VALS / 4 * l + f];
                    v[4 * f] = v[4 * f] * rinv * w.x;
                    v[4 * f + 1] = v[4 * f + 1] * rinv * w.y;
                    v[4 * f + 2] = v[4 * f + 2] * rinv * w.z;
                    v[4 * f + 3] = v[4 * f + 3] * rinv * w.w;
                }
            }
            if (rot) {
                if (a.interleaved) turn<-1>(v, cs, in_rot, lane, from);
                else if (near == LANES / 2) turn<LANES / 2>(v, cs, in_rot, lane, from);
                else if (near == LANES / 4) turn<LANES / 4>(v, cs, in_rot, lane, from);
                else turn<0>(v, cs, in_rot, lane, from);
            }
            row = kv_pack<DT>(v);
        }
        if (which == 0) {
            kv_store(out_q + (uint64_t)(uint32_t)h * (uint32_t)T * (RA_D * esz), l, row);
        } else {
            // (capacities are below 2^30 rows)
            char* out = which == 1 ? out_k : out_v;
            if (out && there[0]) kv_store(out + (uint64_t)(uint32_t)h * (uint32_t)a.stride[0] * (RA_D * esz), l, row);
            if (a.codes[which - 1] && there[1]) {
                float v[VALS];
                kv_floats<DT>(row, v);
                const uint64_t row4 = head4 + (uint64_t)(uint32_t)h * (uint32_t)a.stride[1];
                kv_store4<DT>(a.codes[which - 1] + row4 * Q4_ROW, a.scale[which - 1] + row4 * Q4_BLOCKS, l, lane, v);
            }
        }
    }
}

ra_status ra_launch_append(const AppendArgs& a, ra_dtype dt, hipStream_t st) {
    const int64_t tokens = a.T * a.n_seq;
    if (tokens > (1 << 24) - 1) RA_FAIL(RA_EUNSUP, "more than 2^24 - 1 tokens in a call");
    if ((int64_t)a.n_q + 2 * (int64_t)a.n_kv > (1 << 24) - 1) RA_FAIL(RA_EUNSUP, "too many heads for one launch");
    // where a workgroup per token leaves compute units idle, a workgroup for as many heads of one as it takes at a time
    const int groups = dt == RA_BF16 ? KV_THREADS / KV_LANES<RA_BF16> : KV_THREADS / KV_LANES<RA_F32>;
    const int heads = a.n_q + 2 * a.n_kv, split = tokens <= 128 ? (heads + groups - 1) / groups : 1;
    const int64_t blocks = tokens * split;
    if (blocks > (1 << 24) - 1) RA_FAIL(RA_EUNSUP, "too many heads for one launch");
#define KV_GO_1(DTV, THREADS, ONCE) hipLaunchKernelGGL((append_kernel<DTV, THREADS, ONCE>), dim3((unsigned)blocks), dim3(THREADS), 0, st, a, split)
#define KV_GO_T(DTV, THREADS)                                                                                        \
    do {                                                                                                             \
        if (tokens * bytes > KV_KEPT) KV_GO_1(DTV, THREADS, true); else KV_GO_1(DTV, THREADS, false);                \
    } while (0)
    // Tokens of little data want small workgroups, which wait for less at a time, where there are enough of them to fill the part (us
    // with 64, 128 and 256 threads, bfloat16: 20000 of 6 + 2 + 2 heads 30, 35, 45; 16384 of 16 + 2 + 2 36, 39, 47; 32768 of 28 + 4 + 4
    // 123, 113, 125; 16384 of 64 + 8 + 8 135, 129, 122; float32, 16384 of 6 + 2 + 2 38, 41, 47, of 16 + 2 + 2 67, 69, 71; 2500 of 16 + 2 + 2 11.7, 10.8, 11.6;
    // 1000 of 32 + 8 + 8 17.5, 11.5, 9.4, of 4 + 1 + 1 6.1, 5.0, 5.4).
    const int64_t bytes = (int64_t)heads * RA_D * (dt == RA_BF16 ? 2 : 4);
#define KV_GO(DTV)                                                                                    \
    do {                                                                                              \
        if (bytes <= 1024 || (tokens >= 8192 && bytes <= 6144)) KV_GO_T(DTV, 64);                     \
        else if (bytes <= 2048 || (tokens >= 2048 && bytes <= 10240)) KV_GO_T(DTV, 128);                 \
        else KV_GO_T(DTV, KV_THREADS);                                                                \
    } while (0)
    if (dt == RA_BF16) KV_GO(RA_BF16); else KV_GO(RA_F32);
#undef KV_GO_T
#undef KV_GO_1
#undef KV_GO
    RA_HIP(hipGetLastError());
    return RA_OK;
}

// grid: x = rows of a head, GROUPS x FLY to a workgroup, y = head (with its sequence). A group of lanes takes FLY rows, whose
// loads are all on their way before the first is worked on; a row that is not there is loaded as another one that is. Four rows where
// there are many, else one (us into 4 bits and back, four and one: 8 heads of 131072 bfloat16 rows 103, 109, of 4096 7.1, 6.8; 6 heads
// of 1003 float32 rows 5.7, 5.3).
template <int DT, int FLY, bool ONCE>
__global__ __launch_bounds__(KV_THREADS) void quantize_kv4_kernel(const void* __restrict__ X, int n_kv, int64_t T,
                                                                  const int32_t* __restrict__ first, const int32_t* __restrict__ n_new,
                                                                  int64_t kv_stride, uint8_t* __restrict__ codes,
                                                                  uint8_t* __restrict__ scale) {
    constexpr int LANES = KV_LANES<DT>, GROUPS = KV_THREADS / LANES;
    const int tid = threadIdx.x, lane = tid & (RA_WAVE - 1), l = tid % LANES;
    const size_t head = blockIdx.y;
    const int seq = (int)(head / n_kv);
    const int64_t t0 = (int64_t)blockIdx.x * (GROUPS * FLY) + tid / LANES, at0 = first ? first[seq] : 0;
    const int64_t n = n_new && n_new[seq] < T ? n_new[seq] : T;
    const char* rows = reinterpret_cast<const char*>(X) + head * T * RA_D * (DT == RA_BF16 ? 2 : 4);
    kv_u32x4 raw[FLY];
#pragma unroll
    for (int u = 0; u < FLY; ++u) {
        const int64_t t = t0 + GROUPS * u;
        raw[u] = kv_load<ONCE>(rows + (t < T ? t : T - 1) * RA_D * (DT == RA_BF16 ? 2 : 4), l);
    }
#pragma unroll
    for (int u = 0; u < FLY; ++u) {
        const int64_t t = t0 + GROUPS * u, at = at0 + t;
        if (t >= n || at < 0 || at >= kv_stride) continue;
        float v[KV_VALS<DT>];
        kv_floats<DT>(raw[u], v);
        const size_t row = head * kv_stride + at;
        kv_store4<DT>(codes + row * Q4_ROW, scale + row * Q4_BLOCKS, l, lane, v);
    }
}

template <int DT, int FLY>
__global__ __launch_bounds__(KV_THREADS) void dequantize_kv4_kernel(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scale,
                                                                    int n_kv, int64_t T, const int32_t* __restrict__ first,
                                                                    int64_t kv_stride, void* __restrict__ X) {
    constexpr int LANES = KV_LANES<DT>, GROUPS = KV_THREADS / LANES;
    const int tid = threadIdx.x, l = tid % LANES;
    const size_t head = blockIdx.y;
    const int seq = (int)(head / n_kv);
    const int64_t t0 = (int64_t)blockIdx.x * (GROUPS * FLY) + tid / LANES, at0 = first ? first[seq] : 0;
    uint32_t c[FLY], b[FLY];
    bool there[FLY];
#pragma unroll
    for (int u = 0; u < FLY; ++u) {
        const int64_t at = at0 + t0 + GROUPS * u;
        there[u] = at >= 0 && at < kv_stride;
        const size_t row = head * kv_stride + (there[u] ? at : 0);
        if constexpr (DT == RA_F32) c[u] = reinterpret_cast<const uint16_t*>(codes + row * Q4_ROW)[l];
        else c[u] = reinterpret_cast<const uint32_t*>(codes + row * Q4_ROW)[l];
        b[u] = scale[row * Q4_BLOCKS + l / (LANES / Q4_BLOCKS)];
    }
#pragma unroll
    for (int u = 0; u < FLY; ++u) {
        const int64_t t = t0 + GROUPS * u;
        if (t >= T) continue;
        float v[KV_VALS<DT>];
        q4_values(there[u] ? c[u] : 0u, q4_unit(there[u] ? b[u] : 127u), v);
        kv_store(reinterpret_cast<char*>(X) + (head * T + t) * RA_D * (DT == RA_BF16 ? 2 : 4), l, kv_pack<DT>(v));
    }
}

// what both launch: rows per group of lanes, and the grid
static ra_status rows_grid(ra_dtype dt, int n_seq, int n_kv, int64_t T, bool* four, dim3* grid) {
    const int64_t heads = (int64_t)n_seq * n_kv;
    *four = heads * T >= 1 << 16;
    const int64_t rows = KV_THREADS / (dt == RA_BF16 ? KV_LANES<RA_BF16> : KV_LANES<RA_F32>) * (*four ? 4 : 1), blocks = (T + rows - 1) / rows;
    if (heads > 65535) RA_FAIL(RA_EUNSUP, "more than 65535 (sequence, KV head) pairs");
    if (blocks > (1 << 24) - 1) RA_FAIL(RA_EUNSUP, "T too large");
    *grid = dim3((unsigned)blocks, (unsigned)heads);
    return RA_OK;
}
#define KV_ROWS_GO(KERNEL, ...) hipLaunchKernelGGL((KERNEL), grid, dim3(KV_THREADS), 0, st, __VA_ARGS__)

ra_status ra_launch_quantize_kv4(const void* X, ra_dtype dt, int n_seq, int n_kv, int64_t T, const int32_t* first,
                                 const int32_t* n_new, int64_t kv_stride, hipStream_t st, uint8_t* codes, uint8_t* scale) {
    dim3 grid;
    bool four;
    const ra_status rc = rows_grid(dt, n_seq, n_kv, T, &four, &grid);
    if (rc != RA_OK) return rc;
    const bool once = (int64_t)n_seq * n_kv * T * RA_D * (dt == RA_BF16 ? 2 : 4) > KV_KEPT;      // (never so few that each takes one row)
#define KV_GO(DTV)                                                                                                              \
    do {                                                                                                                        \
        if (once) KV_ROWS_GO((quantize_kv4_kernel<DTV, 4, true>), X, n_kv, T, first, n_new, kv_stride, codes, scale);           \
        else if (four) KV_ROWS_GO((quantize_kv4_kernel<DTV, 4, false>), X, n_kv, T, first, n_new, kv_stride, codes, scale);     \
        else KV_ROWS_GO((quantize_kv4_kernel<DTV, 1, false>), X, n_kv, T, first, n_new, kv_stride, codes, scale);               \
    } while (0)
    if (dt == RA_BF16) KV_GO(RA_BF16); else KV_GO(RA_F32);
#undef KV_GO
    RA_HIP(hipGetLastError());
    return RA_OK;
}

ra_status ra_launch_dequantize_kv4(const uint8_t* codes, const uint8_t* scale, ra_dtype dt, int n_seq, int n_kv, int64_t T,
                                   const int32_t* first, int64_t kv_stride, hipStream_t st, void* X) {
    dim3 grid;
    bool four;
    const ra_status rc = rows_grid(dt, n_seq, n_kv, T, &four, &grid);
    if (rc != RA_OK) return rc;
#define KV_GO(DTV)                                                                                                              \
    do {                                                                                                                        \
        if (four) KV_ROWS_GO((dequantize_kv4_kernel<DTV, 4>), codes, scale, n_kv, T, first, kv_stride, X);                      \
        else KV_ROWS_GO((dequantize_kv4_kernel<DTV, 1>), codes, scale, n_kv, T, first, kv_stride, X);                           \
    } while (0)
    if (dt == RA_BF16) KV_GO(RA_BF16); else KV_GO(RA_F32);
#undef KV_GO
    RA_HIP(hipGetLastError());
    return RA_OK;
}
