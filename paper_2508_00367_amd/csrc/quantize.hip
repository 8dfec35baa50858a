// Symmetric quantization to 8-bit integers with one scale a row (activations) or a column (weights):
//   scale = max(amax * fl(1/127), FLT_MIN),  q = rint(x * fl(1/scale)),  half to even, |q| <= 127
// every step rounded to fp32 once, so that the integers are the same bits wherever they are formed (quant_scale, quant8).
// FLT_MIN keeps the reciprocal finite; a row of zeros gives zeros.  A row that holds an infinity or a NaN gets the scale NaN and
// zeros: what is computed from it is NaN, as it would be without quantization.
#include "quantize.hpp"

namespace rs {

// 16 values of a row from column k on, k a multiple of 16; zeros from column K on.  VEC: rows are whole 16-byte pieces and start
// 16-byte aligned, and a resource ends with the row.
template <typename T, bool VEC>
__device__ __forceinline__ void load16(__amdgpu_buffer_rsrc_t row, const T* p, int k, int K, float (&v)[16]) {
    if constexpr (VEC) {
#pragma unroll
        for (int h = 0; h < (int)sizeof(T); ++h) {
            const u32x4 w = __builtin_amdgcn_raw_buffer_load_b128(row, k * (int)sizeof(T) + h * 16, 0, 0);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if constexpr (sizeof(T) == 4) {
                    v[h * 4 + i] = __uint_as_float(w[i]);
                } else {
                    v[h * 8 + 2 * i] = __uint_as_float(w[i] << 16);
                    v[h * 8 + 2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
                }
            }
        }
    } else if (k + 16 <= K) {  // aligned to its elements only (the hardware takes that in its stride)
        struct __attribute__((packed, aligned(sizeof(T)))) { T e[16]; } raw;
        __builtin_memcpy(&raw, p + k, sizeof(raw));
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] = Elem<T>::ld(&raw.e[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] = k + i < K ? Elem<T>::ld(p + k + i) : 0.f;
    }
}

__device__ __forceinline__ u32x4 pack16(const float (&v)[16], QuantScale s) {
    u32x4 b;
#pragma unroll
    for (int i = 0; i < 4; ++i) b[i] = quant8x4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3], s);
    return b;
}

// G lanes per row (16, 32, 64 or a workgroup of 256), MAXC pieces of 16 values per lane in registers: rows of up to 16 G MAXC values
// are read once.  LONG: longer rows in pieces of 16 G, read twice (the second time from the caches).
// Bound by memory, M K (e + 1) bytes: 16388 x 4096 bf16 36 us, 5.5 TB/s, fp32 59 us, 5.6 (a copy: 5.1); 50432 x 768 21-29 us with the rows in the
// caches or not.  Two or more pieces a lane measured slower up to 1024 columns (768: 21.4 -> 25.8 us) and beyond but for bf16 of 1025 .. 2048
// columns (16388 x 1536 14.8 -> 13.1).
template <typename T, int G, int MAXC, bool VEC, bool LONG>
__global__ __launch_bounds__(256) void quantize_rows_kernel(const T* __restrict__ x, int64_t ldx, int8_t* __restrict__ q,
                                                            int64_t ldq, float* __restrict__ scale, int64_t M, int K) {
    constexpr int RPB = 256 / G;
    __shared__ float s_max[4];
    const int sub = threadIdx.x % G;
    const int64_t row = (int64_t)blockIdx.x * RPB + (G == 64 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : G < 64 ? threadIdx.x / G : 0);
    const bool on = row < M;  // lanes of rows past the last stay for the reductions
    const T* xr = x + (on ? row : 0) * ldx;
    const __amdgpu_buffer_rsrc_t rs_x = row_rsrc(G >= 64 ? xr : x, VEC && G >= 64 ? K * (int)sizeof(T) : 0);
    auto load = [&](int k, float(&v)[16]) {
        if constexpr (VEC && G < 64) {  // several rows per wave: no common resource
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                float t[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
                if (on && k + h * 8 < K) Elem<T>::load8(xr + k + h * 8, t);
#pragma unroll
                for (int i = 0; i < 8; ++i) v[h * 8 + i] = t[i];
            }
        } else {
            load16<T, VEC>(rs_x, xr, k, K, v);
        }
    };
    float v[MAXC][16], amax = 0.f;
    const int trips = LONG ? (K + 16 * G - 1) / (16 * G) : MAXC;
    if constexpr (LONG) {
        for (int c = 0; c < trips; ++c) {
            load((c * G + sub) * 16, v[0]);
#pragma unroll
            for (int i = 0; i < 16; ++i) amax = amax_step(amax, v[0][i]);
        }
    } else {
#pragma unroll
        for (int c = 0; c < MAXC; ++c) load((c * G + sub) * 16, v[c]);
#pragma unroll
        for (int c = 0; c < MAXC; ++c)
#pragma unroll
            for (int i = 0; i < 16; ++i) amax = amax_step(amax, v[c][i]);
    }
    amax = lanes_reduce<(G < 64 ? G : 64)>(amax, [](float a, float b) { return amax_step(a, b); });
    if constexpr (G == 256) {
        if ((threadIdx.x & 63) == 0) s_max[threadIdx.x >> 6] = amax;
        __syncthreads();
        amax = amax_step(amax_step(s_max[0], s_max[1]), amax_step(s_max[2], s_max[3]));
    }
    if (!on) return;
    const QuantScale qs = quant_scale(amax);
    int8_t* qr = q + row * ldq;
    if constexpr (LONG) {
        for (int c = 0; c < trips; ++c) {
            const int k = (c * G + sub) * 16;
            load(k, v[0]);
            if (k < K) *reinterpret_cast<u32x4*>(qr + k) = pack16(v[0], qs);
        }
    } else {
#pragma unroll
        for (int c = 0; c < MAXC; ++c) {
            const int k = (c * G + sub) * 16;
            if (k < K) *reinterpret_cast<u32x4*>(qr + k) = pack16(v[c], qs);
        }
    }
    if (sub == 0) scale[row] = qs.scale;
}

template <typename T, int G, int MAXC, bool VEC, bool LONG>
static void go(const void* x, int64_t ldx, int8_t* q, int64_t ldq, float* scale, int64_t M, int K, hipStream_t s) {
    constexpr int RPB = 256 / G;
    constexpr int64_t most = (int64_t)1 << 23;  // workgroups of a launch: fewer than 2^32 threads
    for (int64_t r = 0; r < M; r += most * RPB) {
        const int64_t m = M - r < most * RPB ? M - r : most * RPB;
        hipLaunchKernelGGL((quantize_rows_kernel<T, G, MAXC, VEC, LONG>), dim3((unsigned)((m + RPB - 1) / RPB)), dim3(256), 0, s,
                           (const T*)x + r * ldx, ldx, q + r * ldq, ldq, scale + r, m, K);
    }
}

template <typename T>
static void by_width(const void* x, int64_t ldx, int8_t* q, int64_t ldq, float* scale, int64_t M, int K, hipStream_t s) {
#define RS_Q(G_, C_, VEC_, LONG_) go<T, G_, C_, VEC_, LONG_>(x, ldx, q, ldq, scale, M, K, s)
    if (K % 8 == 0 && ldx * (int64_t)sizeof(T) % 16 == 0) {
        if (K <= 256) RS_Q(16, 1, true, false);
        else if (K <= 512) RS_Q(32, 1, true, false);
        else if (K <= 1024) RS_Q(64, 1, true, false);
        else if (K <= 2048 && sizeof(T) == 2 && M >= 4096) RS_Q(64, 2, true, false);
        else if (K <= 4096) RS_Q(256, 1, true, false);
        else if (K <= 16384) RS_Q(256, 4, true, false);
        else RS_Q(256, 1, true, true);
    } else {
        if (K <= 1024) RS_Q(64, 1, false, false);
        else if (K <= 4096) RS_Q(256, 1, false, false);
        else RS_Q(256, 1, false, true);
    }
#undef RS_Q
}

hipError_t launch_quantize_rows(rs_dtype dt, const void* x, int64_t ldx, int8_t* q, int64_t ldq, float* scale, int64_t M, int K,
                                hipStream_t s) {
    if (dt == RS_F32) by_width<float>(x, ldx, q, ldq, scale, M, K, s);
    else by_width<bf16raw>(x, ldx, q, ldq, scale, M, K, s);
    return M ? hipGetLastError() : hipSuccess;
}

// Columns of w [K, N] (weights, one-off work): 32 columns per workgroup, 32 threads down each.
template <typename T>
__global__ __launch_bounds__(1024) void quantize_columns_kernel(const T* __restrict__ w, int8_t* __restrict__ q,
                                                                float* __restrict__ scale, int K, int N) {
    __shared__ float s_max[32][33];
    const int tx = threadIdx.x & 31, ty = threadIdx.x >> 5;
    const int n = blockIdx.x * 32 + tx;
    float amax = 0.f;
    if (n < N)
        for (int k = ty; k < K; k += 32) amax = amax_step(amax, Elem<T>::ld(w + (int64_t)k * N + n));
    s_max[ty][tx] = amax;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 32; ++i) amax = amax_step(amax, s_max[i][tx]);
    const QuantScale qs = quant_scale(amax);
    if (n >= N) return;
    for (int k = ty; k < K; k += 32) q[(int64_t)k * N + n] = (int8_t)quant8(Elem<T>::ld(w + (int64_t)k * N + n), qs);
    if (ty == 0) scale[n] = qs.scale;
}

hipError_t launch_quantize_columns(rs_dtype dt, const void* w, int8_t* q, float* scale, int K, int N, hipStream_t s) {
    const dim3 grid((unsigned)((N + 31) / 32));
    if (dt == RS_F32) hipLaunchKernelGGL(quantize_columns_kernel<float>, grid, dim3(1024), 0, s, (const float*)w, q, scale, K, N);
    else hipLaunchKernelGGL(quantize_columns_kernel<bf16raw>, grid, dim3(1024), 0, s, (const bf16raw*)w, q, scale, K, N);
    return hipGetLastError();
}

}  // namespace rs
