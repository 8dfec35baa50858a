// Symmetric quantization to 8-bit integers with one scale a row (activations) or a column (weights):
//   scale = max(amax * fl(1/127), FLT_MIN),  q = rint(x * fl(1/scale)),  half to even, |q| <= 127
// every step rounded to fp32 once, so that the integers are the same bits wherever they are formed (quant_scale, quant8).
// FLT_MIN keeps the reciprocal finite; a row of zeros gives zeros.  A row that holds an infinity or a NaN gets the scale NaN and
// zeros: what is computed from it is NaN, as it would be without quantization.
#include "quantize.hpp"

namespace rs {

// One workgroup per row, two passes over it.
template <typename T>
__global__ __launch_bounds__(256) void quantize_rows_kernel(const T* __restrict__ x, int64_t ldx, int8_t* __restrict__ q,
                                                            int64_t ldq, float* __restrict__ scale, int64_t M, int K) {
    __shared__ float s_max[4];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    for (int64_t row = blockIdx.x; row < M; row += gridDim.x) {
        const T* xr = x + row * ldx;
        float amax = 0.f;
        for (int k = tid; k < K; k += 256) amax = amax_step(amax, Elem<T>::ld(xr + k));
        amax = wave_amax(amax);
        if (lane == 0) s_max[wave] = amax;
        __syncthreads();
        const QuantScale qs = quant_scale(amax_step(amax_step(s_max[0], s_max[1]), amax_step(s_max[2], s_max[3])));
        __syncthreads();
        const int padded = (K + 15) / 16 * 16;
        for (int k = tid; k < padded; k += 256) q[row * ldq + k] = k < K ? (int8_t)quant8(Elem<T>::ld(xr + k), qs) : (int8_t)0;
        if (tid == 0) scale[row] = qs.scale;
    }
}

hipError_t launch_quantize_rows(rs_dtype dt, const void* x, int64_t ldx, int8_t* q, int64_t ldq, float* scale, int64_t M, int K,
                                hipStream_t s) {
    if (M == 0) return hipSuccess;
    const dim3 grid((unsigned)(M < 1 << 20 ? M : 1 << 20));
    if (dt == RS_F32)
        hipLaunchKernelGGL(quantize_rows_kernel<float>, grid, dim3(256), 0, s, (const float*)x, ldx, q, ldq, scale, M, K);
    else
        hipLaunchKernelGGL(quantize_rows_kernel<bf16raw>, grid, dim3(256), 0, s, (const bf16raw*)x, ldx, q, ldq, scale, M, K);
    return hipGetLastError();
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
