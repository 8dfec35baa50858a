// The step between two halves of an encoder block: the branch's own norm, gate and scale, the residual add, and the norm and
// modulation in front of the next branch, whose rows may leave in 8 bits:
//   y = x_scale x + f_scale gate . Norm_post(f),   u = Norm_pre(y) . (1 + mod_scale) + mod_shift
// A row's f, then y, then u stay in registers between the steps; y goes into the second norm as it is in fp32, unrounded.
// Variances are taken over the deviations from the mean.  Bound by reading x and f and writing y and u once.
#include "quantize.hpp"

namespace rs {

// Sum over the WPR waves of a row (wave order), or the largest magnitude.
template <int WPR, bool MAX>
__device__ __forceinline__ float row_reduce(float v, float* s) {
    v = MAX ? wave_amax(v) : wave_sum(v);
    if constexpr (WPR > 1) {
        __syncthreads();
        if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
        __syncthreads();
        v = s[0];
#pragma unroll
        for (int i = 1; i < WPR; ++i) v = MAX ? amax_step(v, s[i]) : v + s[i];
    }
    return v;
}

// v = Norm(v); chunks past the row's end hold zeros before and after, and the deviations leave them out.
template <int MAXC, int WPR>
__device__ __forceinline__ void row_norm(float (&v)[MAXC][8], rs_norm kind, float eps, int D, int t, float* s) {
    if (kind == RS_NORM_NONE) return;
    const int nchunk = D >> 3;
    float mean = 0.f;
    if (kind == RS_NORM_LAYER) {
        float sum = 0.f;
#pragma unroll
        for (int c = 0; c < MAXC; ++c)
#pragma unroll
            for (int i = 0; i < 8; ++i) sum += v[c][i];
        mean = row_reduce<WPR, false>(sum, s) / (float)D;
    }
    float sq = 0.f;
#pragma unroll
    for (int c = 0; c < MAXC; ++c) {
        const float q = chunk_sq(v[c], mean, sq);
        sq = t + c * (64 * WPR) < nchunk ? q : sq;
    }
    const float r = rsqrtf(row_reduce<WPR, false>(sq, s) / (float)D + eps);
#pragma unroll
    for (int c = 0; c < MAXC; ++c)
#pragma unroll
        for (int i = 0; i < 8; ++i) v[c][i] = t + c * (64 * WPR) < nchunk ? (v[c][i] - mean) * r : 0.f;
}

template <typename T, int MAXC, int WPR>
__global__ __launch_bounds__(256) void residual_norm_kernel(ResidualNormArgs p) {
    __shared__ float s_red[WPR > 1 ? WPR : 1];
    constexpr int RPB = 4 / WPR;  // rows of a workgroup
    const int t = threadIdx.x & (64 * WPR - 1), D = p.D, nchunk = D >> 3;
    const T *xp = (const T*)p.x, *fp = (const T*)p.f, *post_g = (const T*)p.post_g, *post_b = (const T*)p.post_b;
    const T *pre_g = (const T*)p.pre_g, *pre_b = (const T*)p.pre_b;
    for (int64_t row = (int64_t)blockIdx.x * RPB + (WPR == 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : 0); row < p.rows; row += (int64_t)gridDim.x * RPB) {
        const int64_t img = row / p.N;
        const T* gate = p.gate ? (const T*)p.gate + img * p.gate_stride : nullptr;
        const T* ms = p.mod_scale ? (const T*)p.mod_scale + img * p.mod_stride : nullptr;
        const T* mt = p.mod_shift ? (const T*)p.mod_shift + img * p.mod_stride : nullptr;
        float v[MAXC][8], w[8];
#pragma unroll
        for (int c = 0; c < MAXC; ++c) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[c][i] = 0.f;
            const int ch = t + c * (64 * WPR);
            if (fp && ch < nchunk) Elem<T>::load8(fp + row * D + ch * 8, v[c]);
        }
        row_norm<MAXC, WPR>(v, p.post, p.post_eps, D, t, s_red);
#pragma unroll
        for (int c = 0; c < MAXC; ++c) {
            const int ch = t + c * (64 * WPR);
            if (ch >= nchunk) continue;
            if (post_g) {
                Elem<T>::load8(post_g + ch * 8, w);
#pragma unroll
                for (int i = 0; i < 8; ++i) v[c][i] *= w[i];
            }
            if (post_b) {
                Elem<T>::load8(post_b + ch * 8, w);
#pragma unroll
                for (int i = 0; i < 8; ++i) v[c][i] += w[i];
            }
            if (gate) {
                Elem<T>::load8(gate + ch * 8, w);
#pragma unroll
                for (int i = 0; i < 8; ++i) v[c][i] *= w[i];
            }
            Elem<T>::load8(xp + row * D + ch * 8, w);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[c][i] = fp ? fmaf(p.x_scale, w[i], p.f_scale * v[c][i]) : p.x_scale * w[i];
            if (p.y) Elem<T>::store8((T*)p.y + row * D + ch * 8, v[c]);
        }
        if (!p.u && !p.u_q) continue;
        row_norm<MAXC, WPR>(v, p.pre, p.pre_eps, D, t, s_red);
        float amax = 0.f;
#pragma unroll
        for (int c = 0; c < MAXC; ++c) {
            const int ch = t + c * (64 * WPR);
            if (ch >= nchunk) continue;
            if (pre_g) {
                Elem<T>::load8(pre_g + ch * 8, w);
#pragma unroll
                for (int i = 0; i < 8; ++i) v[c][i] *= w[i];
            }
            if (pre_b) {
                Elem<T>::load8(pre_b + ch * 8, w);
#pragma unroll
                for (int i = 0; i < 8; ++i) v[c][i] += w[i];
            }
            if (ms) {
                Elem<T>::load8(ms + ch * 8, w);
#pragma unroll
                for (int i = 0; i < 8; ++i) v[c][i] = fmaf(v[c][i], w[i], v[c][i]);
            }
            if (mt) {
                Elem<T>::load8(mt + ch * 8, w);
#pragma unroll
                for (int i = 0; i < 8; ++i) v[c][i] += w[i];
            }
            if (p.u) Elem<T>::store8((T*)p.u + row * D + ch * 8, v[c]);
#pragma unroll
            for (int i = 0; i < 8; ++i) amax = amax_step(amax, v[c][i]);
        }
        if (p.u_q) {
            const QuantScale qs = quant_scale(row_reduce<WPR, true>(amax, s_red));
            const int npad = (D + 15) / 16 * 2;
#pragma unroll
            for (int c = 0; c < MAXC; ++c) {
                const int ch = t + c * (64 * WPR);
                uint32_t b[2] = {0, 0};
                if (ch < nchunk) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) b[i >> 2] |= (uint32_t)(quant8(v[c][i], qs) & 255) << (8 * (i & 3));
                }
                if (ch < npad) *reinterpret_cast<uint2*>(p.u_q + row * p.ldq + ch * 8) = make_uint2(b[0], b[1]);
            }
            if (t == 0) p.u_scale[row] = qs.scale;
        }
    }
}

template <typename T, int MAXC, int WPR>
static hipError_t go(const ResidualNormArgs& p, hipStream_t s) {
    constexpr int RPB = 4 / WPR;
    const int64_t blocks = (p.rows + RPB - 1) / RPB;
    hipLaunchKernelGGL((residual_norm_kernel<T, MAXC, WPR>), dim3((unsigned)(blocks < 1 << 20 ? blocks : 1 << 20)), dim3(256), 0, s, p);
    return hipGetLastError();
}

template <typename T>
static hipError_t launch_rn(const ResidualNormArgs& p, hipStream_t s) {
    if (p.D <= 512) return go<T, 1, 1>(p, s);
    if (p.D <= 1024) return go<T, 2, 1>(p, s);
    if (p.D <= 2048) return go<T, 4, 1>(p, s);
    if (p.D <= 4096) return go<T, 2, 4>(p, s);
    if (p.D <= 8192) return go<T, 4, 4>(p, s);
    return go<T, 8, 4>(p, s);
}

hipError_t launch_residual_norm(rs_dtype dt, const ResidualNormArgs& p, hipStream_t s) {
    if (p.rows == 0) return hipSuccess;
    return dt == RS_F32 ? launch_rn<float>(p, s) : launch_rn<bf16raw>(p, s);
}

}  // namespace rs
