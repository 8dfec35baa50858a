// The step between two halves of an encoder block: the branch's own norm, gate and scale, the residual add, and the norm and
// modulation in front of the next branch, whose rows may leave in 8 bits:
//   y = x_scale x + f_scale gate . Norm_post(f),   u = Norm_pre(y) . (1 + mod_scale) + mod_shift
// A row's f, then y, then u stay in registers between the steps; y goes into the second norm as it is in fp32, unrounded.
// Variances are taken over the deviations from the mean.  Bound by reading x and f and writing y and u once.
#include "quantize.hpp"

namespace rs {

// 8 elements as they are in memory.
template <typename T> struct Raw8 { u32x4 w[sizeof(T) / 2]; };

// `off`: byte offset, or one past the resource's end (zeros).
template <typename T>
__device__ __forceinline__ Raw8<T> raw_load(__amdgpu_buffer_rsrc_t r, int off) {
    Raw8<T> v;
#pragma unroll
    for (int h = 0; h < (int)sizeof(T) / 2; ++h) v.w[h] = __builtin_amdgcn_raw_buffer_load_b128(r, off + h * 16, 0, 0);
    return v;
}
template <typename T>
__device__ __forceinline__ Raw8<T> raw_load(const T* p) {
    Raw8<T> v;
#pragma unroll
    for (int h = 0; h < (int)sizeof(T) / 2; ++h) v.w[h] = reinterpret_cast<const u32x4*>(p)[h];
    return v;
}
template <typename T>
__device__ __forceinline__ float at(const Raw8<T>& v, int i) {
    if constexpr (sizeof(T) == 4) return __uint_as_float(v.w[i >> 2][i & 3]);
    else return __uint_as_float((i & 1) ? (v.w[0][i >> 1] & 0xffff0000u) : (v.w[0][i >> 1] << 16));
}

// Sum, or the largest magnitude, over the G lanes of a row (256: the four waves of a workgroup, in wave order).
template <int G, bool MAX>
__device__ __forceinline__ float row_reduce(float v, float* s) {
    auto op = [](float a, float b) { return MAX ? amax_step(a, b) : a + b; };
    v = lanes_reduce<(G < 64 ? G : 64)>(v, op);
    if constexpr (G == 256) {
        __syncthreads();
        if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
        __syncthreads();
        v = op(op(op(s[0], s[1]), s[2]), s[3]);
    }
    return v;
}

// v = Norm(v); chunks past the row's end hold zeros before and after, and the deviations leave them out.
template <int G, int MAXC>
__device__ __forceinline__ void row_norm(float (&v)[MAXC][8], rs_norm kind, float eps, float inv_d, int nchunk, int sub, float* s) {
    if (kind == RS_NORM_NONE) return;
    float mean = 0.f;
    if (kind == RS_NORM_LAYER) {
        float sum = 0.f;
#pragma unroll
        for (int c = 0; c < MAXC; ++c)
#pragma unroll
            for (int i = 0; i < 8; ++i) sum += v[c][i];
        mean = row_reduce<G, false>(sum, s) * inv_d;
#pragma unroll
        for (int c = 0; c < MAXC; ++c)
#pragma unroll
            for (int i = 0; i < 8; ++i) v[c][i] = sub + c * G < nchunk ? v[c][i] - mean : 0.f;
    }
    float sq = 0.f;
#pragma unroll
    for (int c = 0; c < MAXC; ++c)
#pragma unroll
        for (int i = 0; i < 8; ++i) sq = fmaf(v[c][i], v[c][i], sq);
    const float r = rsqrtf(fmaf(row_reduce<G, false>(sq, s), inv_d, eps));
#pragma unroll
    for (int c = 0; c < MAXC; ++c)
#pragma unroll
        for (int i = 0; i < 8; ++i) v[c][i] *= r;
}

// G lanes per row (8 .. 64, or a workgroup of 256), MAXC chunks of 8 channels per lane: lane l has chunks l, l + G, ...
// The rows of a wave are neighbours: one resource holds them, and what lies past the last row or the end of a row is aimed
// past its end.
template <typename T, int G, int MAXC>
__global__ __launch_bounds__(256) void residual_norm_kernel(ResidualNormArgs p) {
    __shared__ float s_red[4];
    constexpr int RPW = G < 64 ? 64 / G : 1, RPB = G == 256 ? 1 : 4 * RPW;  // rows of a wave, of a workgroup
    constexpr int ES = sizeof(T);
    const int D = p.D, nchunk = D >> 3, sub = threadIdx.x % G;
    const float inv_d = 1.0f / (float)D;
    const bool has_f = p.f != nullptr;
    const T *post_g = (const T*)p.post_g, *post_b = (const T*)p.post_b, *pre_g = (const T*)p.pre_g, *pre_b = (const T*)p.pre_b;
    const int64_t wave0 = (int64_t)blockIdx.x * RPB + (G == 256 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) * RPW);
    for (int64_t row0 = wave0; row0 < p.rows; row0 += (int64_t)gridDim.x * RPB) {
        const int my = G < 64 ? (threadIdx.x & 63) / G : 0;
        const int64_t left = p.rows - row0;
        const int bytes = (int)(left < RPW ? left : RPW) * D * ES;
        const __amdgpu_buffer_rsrc_t rs_x = row_rsrc((const T*)p.x + row0 * D, bytes);
        const __amdgpu_buffer_rsrc_t rs_f = row_rsrc(has_f ? (const T*)p.f + row0 * D : nullptr, has_f ? bytes : 0);
        int off[MAXC];
#pragma unroll
        for (int c = 0; c < MAXC; ++c) off[c] = sub + c * G < nchunk ? (my * D + (sub + c * G) * 8) * ES : 0x7fffff00;
        Raw8<T> rx[MAXC], w[MAXC];
        float v[MAXC][8];
#pragma unroll
        for (int c = 0; c < MAXC; ++c) w[c] = raw_load<T>(rs_f, off[c]);
#pragma unroll
        for (int c = 0; c < MAXC; ++c) rx[c] = raw_load<T>(rs_x, off[c]);
        // a vector's chunks of this lane; past the row's end its first one, of which nothing is used
        auto vec = [&](const T* q) {
#pragma unroll
            for (int c = 0; c < MAXC; ++c) w[c] = raw_load<T>(q + (sub + c * G < nchunk ? sub + c * G : 0) * 8);
        };
        int64_t img = 0;
        if (p.gate_stride | p.mod_stride) {
            const int64_t row = row0 + my < p.rows ? row0 + my : p.rows - 1;
            img = (uint32_t)row / (uint32_t)p.N;
        }
#pragma unroll
        for (int c = 0; c < MAXC; ++c)
#pragma unroll
            for (int i = 0; i < 8; ++i) v[c][i] = at<T>(w[c], i);
        row_norm<G, MAXC>(v, p.post, p.post_eps, inv_d, nchunk, sub, s_red);
#define RS_EACH(expr_)                                        \
    _Pragma("unroll") for (int c = 0; c < MAXC; ++c)          \
        _Pragma("unroll") for (int i = 0; i < 8; ++i) { const float t = at<T>(w[c], i); v[c][i] = (expr_); }
        if (post_g) { vec(post_g); RS_EACH(v[c][i] * t) }
        if (post_b) { vec(post_b); RS_EACH(v[c][i] + t) }
        if (p.gate) { vec((const T*)p.gate + img * p.gate_stride); RS_EACH(v[c][i] * t) }
#pragma unroll
        for (int c = 0; c < MAXC; ++c)
#pragma unroll
            for (int i = 0; i < 8; ++i) v[c][i] = sub + c * G < nchunk ? fmaf(p.x_scale, at<T>(rx[c], i), p.f_scale * v[c][i]) : 0.f;
        const bool on = row0 + my < p.rows;
        const int64_t row = row0 + my;
        if (p.y) {
#pragma unroll
            for (int c = 0; c < MAXC; ++c)
                if (on && sub + c * G < nchunk) Elem<T>::store8((T*)p.y + row * D + (sub + c * G) * 8, v[c]);
        }
        if (!p.u && !p.u_q) continue;
        row_norm<G, MAXC>(v, p.pre, p.pre_eps, inv_d, nchunk, sub, s_red);
        if (pre_g) { vec(pre_g); RS_EACH(v[c][i] * t) }
        if (pre_b) { vec(pre_b); RS_EACH(v[c][i] + t) }
        if (p.mod_scale) { vec((const T*)p.mod_scale + img * p.mod_stride); RS_EACH(fmaf(v[c][i], t, v[c][i])) }
        if (p.mod_shift) { vec((const T*)p.mod_shift + img * p.mod_stride); RS_EACH(v[c][i] + t) }
#undef RS_EACH
        if (p.u) {
#pragma unroll
            for (int c = 0; c < MAXC; ++c)
                if (on && sub + c * G < nchunk) Elem<T>::store8((T*)p.u + row * D + (sub + c * G) * 8, v[c]);
        }
        if (p.u_q) {
            float amax = 0.f;
#pragma unroll
            for (int c = 0; c < MAXC; ++c)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    v[c][i] = sub + c * G < nchunk ? v[c][i] : 0.f;
                    amax = amax_step(amax, v[c][i]);
                }
            const QuantScale qs = quant_scale(row_reduce<G, true>(amax, s_red));
            const int npad = (D + 15) / 16 * 2;  // zeros up to a multiple of 16
#pragma unroll
            for (int c = 0; c < MAXC; ++c) {
                const int ch = sub + c * G;
                const uint2 b = make_uint2(quant8x4(v[c][0], v[c][1], v[c][2], v[c][3], qs), quant8x4(v[c][4], v[c][5], v[c][6], v[c][7], qs));
                if (on && ch < npad) *reinterpret_cast<uint2*>(p.u_q + row * p.ldq + ch * 8) = b;
            }
            if (on && sub == 0) p.u_scale[row] = qs.scale;
        }
    }
}

template <typename T, int G, int MAXC>
static hipError_t go(const ResidualNormArgs& p, hipStream_t s) {
    constexpr int RPB = G == 256 ? 1 : 256 / G;
    const int64_t blocks = (p.rows + RPB - 1) / RPB;
    hipLaunchKernelGGL((residual_norm_kernel<T, G, MAXC>), dim3((unsigned)(blocks < 1 << 20 ? blocks : 1 << 20)), dim3(256), 0, s, p);
    return hipGetLastError();
}

// The fewest lanes that hold a row in up to four chunks each: every lane busy at 192, 384 and 768 channels, where a wave per
// row leaves a quarter to five eighths of its lanes without work.
template <typename T>
static hipError_t launch_rn(const ResidualNormArgs& p, hipStream_t s) {
    const int D = p.D;
    if (D <= 128) return go<T, 8, 2>(p, s);
    if (D <= 192) return go<T, 8, 3>(p, s);
    if (D <= 256) return go<T, 8, 4>(p, s);
    if (D <= 384) return go<T, 16, 3>(p, s);
    if (D <= 512) return go<T, 16, 4>(p, s);
    if (D <= 768) return go<T, 32, 3>(p, s);
    if (D <= 1024) return go<T, 32, 4>(p, s);
    if (D <= 1536) return go<T, 64, 3>(p, s);
    if (D <= 2048) return go<T, 64, 4>(p, s);
    if (D <= 4096) return go<T, 256, 2>(p, s);
    if (D <= 8192) return go<T, 256, 4>(p, s);
    return go<T, 256, 8>(p, s);
}

hipError_t launch_residual_norm(rs_dtype dt, const ResidualNormArgs& p, hipStream_t s) {
    if (p.rows == 0) return hipSuccess;
    return dt == RS_F32 ? launch_rn<float>(p, s) : launch_rn<bf16raw>(p, s);
}

}  // namespace rs
