// Linear layers in 8-bit integers (W8A8): out = epi((sum_k a[m,k] w[k,n]) a_scale[m] w_scale[n] + bias[n]), the sums exact in
// int32 (v_mfma_i32_32x32x32_i8), everything behind them in fp32, rounded once.
//
// Weights are packed in fragment order, [Np / 32][Kp / 32] fragments of 32 features x 32 k, 1 KB each, lane l's 16 bytes in
// a row: feature l & 31, k 16 (l >> 5) .. + 15; Np and Kp are N and K rounded up to 64 and 128, the rest is zeros.  A byte of
// `a` behind column K (up to the row's pitch, or of the next row) is multiplied by such a zero: being an integer it adds nothing.
#include "gemm_tile.hpp"

namespace rs {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x16 __attribute__((ext_vector_type(16)));

size_t packed_i8_size(int K, int N) { return align_up((size_t)N, 64) * align_up((size_t)K, 128); }

__device__ __forceinline__ float gelu_of(float x, const float*) { return gelu_erf(x); }
__device__ __forceinline__ float gelu_of(float x, const bf16raw*) { return gelu_sp(x); }

// Four waves of 32 rows x 64 features, operands straight from memory.
template <typename T, int EPI>
__global__ __launch_bounds__(256) void gemm_i8_kernel(const int8_t* __restrict__ a, int64_t lda, const float* __restrict__ a_scale,
                                                      const int8_t* __restrict__ w, const float* __restrict__ w_scale,
                                                      const T* __restrict__ bias, const T* __restrict__ res, T* __restrict__ out,
                                                      int64_t M, int N, int K, int tiles_n) {
    const int lane = threadIdx.x & 63, l32 = lane & 31, g = lane >> 5;
    const int64_t m = (int64_t)(blockIdx.x / tiles_n) * 128 + (threadIdx.x >> 6) * 32 + l32;
    const int n0 = (int)(blockIdx.x % tiles_n) * 64;
    const int steps = (K + 31) / 32;
    const int64_t frag_row = (int64_t)((K + 127) / 128 * 128) * 32;
    const int8_t* ar = a + (m < M ? m : M - 1) * lda + g * 16;
    const int8_t* wr = w + (n0 / 32) * frag_row + lane * 16;
    i32x16 acc[2];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[i][r] = 0;
    for (int t = 0; t < steps; ++t) {
        i32x4 av{0, 0, 0, 0};
        if (t * 32 + g * 16 < K) av = *reinterpret_cast<const i32x4*>(ar + t * 32);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const i32x4 wv = *reinterpret_cast<const i32x4*>(wr + i * frag_row + (int64_t)t * 1024);
            acc[i] = __builtin_amdgcn_mfma_i32_32x32x32_i8(wv, av, acc[i], 0, 0, 0);
        }
    }
    if (m >= M) return;
    const float as = a_scale[m];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const int n = n0 + i * 32 + (r >> 2) * 8 + g * 4 + (r & 3);
            if (n >= N) continue;
            float v = fmaf((float)acc[i][r], as * w_scale[n], bias ? Elem<T>::ld(bias + n) : 0.f);
            if (EPI == EPI_BIAS_GELU) v = gelu_of(v, bias);
            if (EPI == EPI_BIAS_RES) v += Elem<T>::ld(res + m * N + n);
            Elem<T>::st(out + m * N + n, v);
        }
}

template <typename T, int EPI>
static hipError_t launch_i8(const GemmI8Args& g, hipStream_t s) {
    const int tiles_n = (g.N + 63) / 64;
    const int64_t rows = ((int64_t)1 << 23) / tiles_n * 128;  // of one launch
    for (int64_t r = 0; r < g.M; r += rows) {
        const int64_t M = g.M - r < rows ? g.M - r : rows;
        const T* res = (const T*)g.res;
        hipLaunchKernelGGL((gemm_i8_kernel<T, EPI>), dim3((unsigned)((M + 127) / 128 * tiles_n)), dim3(256), 0, s, g.a + r * g.lda,
                           g.lda, g.a_scale + r, (const int8_t*)g.w, g.w_scale, (const T*)g.bias, res ? res + r * g.N : nullptr,
                           (T*)g.out + r * g.N, M, g.N, g.K, tiles_n);
    }
    return hipGetLastError();
}

hipError_t launch_gemm_i8(rs_dtype dt, GemmEpilogue epi, const GemmI8Args& g, hipStream_t s) {
    if (epi == EPI_BIAS) return dt == RS_F32 ? launch_i8<float, EPI_BIAS>(g, s) : launch_i8<bf16raw, EPI_BIAS>(g, s);
    if (epi == EPI_BIAS_GELU) return dt == RS_F32 ? launch_i8<float, EPI_BIAS_GELU>(g, s) : launch_i8<bf16raw, EPI_BIAS_GELU>(g, s);
    return dt == RS_F32 ? launch_i8<float, EPI_BIAS_RES>(g, s) : launch_i8<bf16raw, EPI_BIAS_RES>(g, s);
}

// [K, N] row-major -> fragment order: 64 x 64 bytes through LDS, 2 x 2 fragments, written 16 bytes per lane.
__global__ __launch_bounds__(256) void pack_i8_kernel(const int8_t* __restrict__ q, int8_t* __restrict__ wf, int K, int N, int steps) {
    __shared__ int8_t tile[64][68];
    const int k0 = blockIdx.y * 64, n0 = blockIdx.x * 64;
    const int tx = threadIdx.x & 63, ty = threadIdx.x >> 6;
    for (int r = ty; r < 64; r += 4) {
        const int k = k0 + r, n = n0 + tx;
        tile[r][tx] = k < K && n < N ? q[(int64_t)k * N + n] : (int8_t)0;
    }
    __syncthreads();
    const int f = ty & 1, kk = ty >> 1, n = f * 32 + (tx & 31), k = kk * 32 + (tx >> 5) * 16;
    uint32_t v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[i] = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[i] |= (uint32_t)(uint8_t)tile[k + 4 * i + e][n] << (8 * e);
    }
    const int64_t at = ((int64_t)(n0 / 32 + f) * steps + k0 / 32 + kk) * 1024 + tx * 16;
    *reinterpret_cast<uint4*>(wf + at) = make_uint4(v[0], v[1], v[2], v[3]);
}

hipError_t launch_pack_i8(const int8_t* q, void* packed, int K, int N, hipStream_t s) {
    const int kp = (K + 127) / 128 * 128;
    hipLaunchKernelGGL(pack_i8_kernel, dim3((N + 63) / 64, kp / 64), dim3(256), 0, s, q, (int8_t*)packed, K, N, kp / 32);
    return hipGetLastError();
}

}  // namespace rs
