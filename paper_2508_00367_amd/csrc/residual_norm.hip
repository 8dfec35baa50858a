// The step between two halves of an encoder block: the branch's own norm, gate and scale, the residual add, and the norm and
// modulation in front of the next branch, whose rows may leave in 8 bits:
//   y = x_scale x + f_scale gate . Norm_post(f),   u = Norm_pre(y) . (1 + mod_scale) + mod_shift
// A row's f, then y, then u stay in registers between the steps; y goes into the second norm as it is in fp32, unrounded.
// Variances are taken over the deviations from the mean.
// Bound by reading x and f and writing y and u once, at the rate of a copy (5.1 TB/s): 4 x 4097 x 1024 fp32 with every vector 51 us, 5.3 TB/s; 256 x
// 197 x 768 bf16 with one norm or two 61 us, 5.1 TB/s; with two norms and 8-bit rows (a third of the stores) 57 us, 4.7 TB/s, one call behind the other, and
// 69-72 between the products of 8-bit layers, whose output is still on its way to memory: about 40 ALU instructions
// a value then.  What it took: x and f requested together before anything is summed; every lane with work (below); vectors
// through resources, whose scalar addresses leave the registers to the rows (bf16 in three pieces 161 -> 125, four waves per SIMD; forced lower, they
// spill: 107 us); fp32 in pieces of 4 channels, so that neighbouring lanes' pieces lie side by side (58 -> 51); stores through the L2 where rows are whole
// lines (4 us of 60), and left to the L2 to join where they are not (8 x 4097 x 4040 fp32 474 -> 389, x 1000 bf16 65 -> 58).
// What it costs: up to eleven resources of four scalars each, 20 to 64 of which go to lanes of vector registers and back; four pieces a lane take 131
// registers and more, three waves per SIMD.  fp32 rows of more than 8192 channels, 1024 lanes to a row, have 128 registers and keep
// 80 bytes a lane in scratch memory: 4097 x 16384 242 us, 4.4 TB/s (bf16 into 8-bit rows, 512 lanes, 151 us, 3.1 TB/s).
#include "quantize.hpp"

namespace rs {

// 16 bytes of a row, 8 or 4 channels: what a lane loads and stores at a time, its neighbours the ones beside it.
template <typename T> constexpr int kE = 16 / (int)sizeof(T);

template <typename T>
__device__ __forceinline__ float at(u32x4 w, int i) {
    if constexpr (sizeof(T) == 4) return __uint_as_float(w[i]);
    else return __uint_as_float((i & 1) ? (w[i >> 1] & 0xffff0000u) : (w[i >> 1] << 16));
}
template <typename T>
__device__ __forceinline__ u32x4 piece(const float (&v)[kE<T>]) {
    if constexpr (sizeof(T) == 4) return __builtin_bit_cast(u32x4, f32x4{v[0], v[1], v[2], v[3]});
    else return u32x4{pack2bf(v[0], v[1]), pack2bf(v[2], v[3]), pack2bf(v[4], v[5]), pack2bf(v[6], v[7])};
}

// The largest magnitude over the G lanes of a row (more than 64: the waves of a workgroup).
template <int G>
__device__ __forceinline__ float row_amax(float v, float* s) {
    auto op = [](float a, float b) { return amax_step(a, b); };
    v = lanes_reduce<(G < 64 ? G : 64)>(v, op);
    if constexpr (G > 64) {
        __syncthreads();
        if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
        __syncthreads();
        v = s[0];
#pragma unroll
        for (int i = 1; i < G / 64; ++i) v = op(v, s[i]);
    }
    return v;
}

// The sum over a row of what its pieces add up to, t[c] piece lane + c G of it.  Rows of up to 256 pieces have one order of additions
// whatever G and P are: pieces 128 apart first, then 64, and so on down to neighbours, absent ones being zeros.  So a row's bits do not depend on
// how many rows there are, by which the lanes are chosen.  (Longer rows have one G and P each: the waves' sums are added in wave order.)
template <int G, int P>
__device__ __forceinline__ float row_sum(const float (&t)[P], float* s) {
    float v = t[0];
    if constexpr (P == 2) v = t[0] + t[1];
    if constexpr (P == 3) v = (t[0] + t[2]) + t[1];
    if constexpr (P == 4) v = (t[0] + t[2]) + (t[1] + t[3]);
    if constexpr (G > 64 && P == 1) {
        static_assert(G == 256, "four waves: 128 and 64 pieces apart");
        const int lane = threadIdx.x & 63;
        __syncthreads();
        s[threadIdx.x] = v;
        __syncthreads();
        v = (s[lane] + s[lane + 128]) + (s[lane + 64] + s[lane + 192]);
    }
    v = lanes_sum<(G < 64 ? G : 64)>(v);
    if constexpr (G > 64 && P > 1) {
        __syncthreads();
        if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
        __syncthreads();
        v = s[0];
#pragma unroll
        for (int i = 1; i < G / 64; ++i) v += s[i];
    }
    return v;
}

// v = Norm(v); pieces past the row's end (`n` of them are inside) hold zeros before and after, and the deviations leave them out.
template <int G, int P, int E>
__device__ __forceinline__ void row_norm(float (&v)[P][E], rs_norm kind, float eps, float inv_d, int n, int sub, float* s) {
#pragma clang fp contract(off)  // the same operations whatever G and P are
    if (kind == RS_NORM_NONE) return;
    float t[P];
    if (kind == RS_NORM_LAYER) {
#pragma unroll
        for (int c = 0; c < P; ++c) {
            t[c] = v[c][0];
#pragma unroll
            for (int i = 1; i < E; ++i) t[c] += v[c][i];
        }
        const float mean = row_sum<G, P>(t, s) * inv_d;
#pragma unroll
        for (int c = 0; c < P; ++c) {
            const float m = sub + c * G < n ? mean : 0.f;
#pragma unroll
            for (int i = 0; i < E; ++i) v[c][i] -= m;
        }
    }
#pragma unroll
    for (int c = 0; c < P; ++c) {
        t[c] = v[c][0] * v[c][0];
#pragma unroll
        for (int i = 1; i < E; ++i) t[c] = fmaf(v[c][i], v[c][i], t[c]);
    }
    const float r = rsqrtf(fmaf(row_sum<G, P>(t, s), inv_d, eps));
#pragma unroll
    for (int c = 0; c < P; ++c)
#pragma unroll
        for (int i = 0; i < E; ++i) v[c][i] *= r;
}

// G lanes per row (8 .. 64, or a workgroup of 256 .. 1024), P pieces per lane: lane l has pieces l, l + G, ...
// The rows of a wave are neighbours: one resource holds them, and what lies past the last row or the end of a row is aimed
// past its end.
template <typename T, int G, int P>
__global__ __launch_bounds__(G > 256 ? G : 256) void residual_norm_kernel(ResidualNormArgs p) {
#pragma clang fp contract(off)  // as in row_norm
    __shared__ float s_red[G <= 64 ? 1 : P == 1 ? G : G / 64];
    constexpr int RPW = G < 64 ? 64 / G : 1, RPB = G > 64 ? 1 : 4 * RPW;  // rows of a wave, of a workgroup
    constexpr int ES = sizeof(T), E = kE<T>;
    const int D = p.D, n = D / E, sub = threadIdx.x % G;
    const float inv_d = 1.0f / (float)D;
    const bool lines = D * ES % 128 == 0;
    auto put = [&](__amdgpu_buffer_rsrc_t r, int at, u32x4 v) {
        if (lines) store16_wt(r, at, v);
        else __builtin_amdgcn_raw_buffer_store_b128(v, r, at, 0, 0);
    };
    const int64_t wave0 = (int64_t)blockIdx.x * RPB + (G > 64 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) * RPW);
    for (int64_t row0 = wave0; row0 < p.rows; row0 += (int64_t)gridDim.x * RPB) {
        const int my = G < 64 ? (threadIdx.x & 63) / G : 0;
        const int64_t left = p.rows - row0, row = row0 + my;
        const bool on = my < left;
        const int bytes = (int)(left < RPW ? left : RPW) * D * ES;
        auto rsrc = [&](const void* q) { return row_rsrc(q ? (const T*)q + row0 * D : nullptr, q ? bytes : 0); };
        const __amdgpu_buffer_rsrc_t rs_x = rsrc(p.x), rs_f = rsrc(p.f), rs_y = rsrc(p.y), rs_u = rsrc(p.u);
        int off[P];
#pragma unroll
        for (int c = 0; c < P; ++c) off[c] = sub + c * G < n ? my * D * ES + (sub + c * G) * 16 : 0x7fffff00;
        u32x4 rx[P], w[P], va[P], vb[P], vc[P], vd[P];
        float v[P][E];
#pragma unroll
        for (int c = 0; c < P; ++c) w[c] = __builtin_amdgcn_raw_buffer_load_b128(rs_f, off[c], 0, 0);
#pragma unroll
        for (int c = 0; c < P; ++c) rx[c] = __builtin_amdgcn_raw_buffer_load_b128(rs_x, off[c], 0, 0);
        // Vectors: this lane's pieces (past the row's end the first one, of which nothing is used), the image's by their distance from
        // those of the wave's first row.
        int64_t img0 = 0;
        int at_gate = 0, at_mod = 0;
        if (p.gate_stride | p.mod_stride) {
            img0 = (uint32_t)row0 / (uint32_t)p.N;
            if constexpr (G < 64) {
                const int d = (int)((uint32_t)(on ? row : p.rows - 1) / (uint32_t)p.N) - (int)img0;
                at_gate = d * (int)p.gate_stride * ES;
                at_mod = d * (int)p.mod_stride * ES;
            }
        }
        auto vec = [&](auto& r, const void* q, int64_t first, int by) {
            const __amdgpu_buffer_rsrc_t rs = row_rsrc((const T*)q + first, 0x7fffffff);
#pragma unroll
            for (int c = 0; c < P; ++c) r[c] = __builtin_amdgcn_raw_buffer_load_b128(rs, (sub + c * G < n ? (sub + c * G) * 16 : 0) + by, 0, 0);
        };
#define RS_VEC(r_, name_) if (p.name_) vec(r_, p.name_, 0, 0)
#define RS_VEC_GATE(r_) if (p.gate) vec(r_, p.gate, img0 * p.gate_stride, at_gate)
#define RS_VEC_MOD(r_, name_) if (p.name_) vec(r_, p.name_, img0 * p.mod_stride, at_mod)
// each of the lane's values with its place t in a vector
#define RS_EACH(cond_, r_, expr_)                                                                        \
    if (cond_) {                                                                                          \
        _Pragma("unroll") for (int c = 0; c < P; ++c)                                                     \
            _Pragma("unroll") for (int i = 0; i < E; ++i) {                                               \
                const float t = at<T>(r_[c], i);                                                          \
                v[c][i] = (expr_);                                                                        \
            }                                                                                             \
    }
// v . g + b, each where there is one
#define RS_AFFINE(g_, b_)                                                                                 \
    if (g_ && b_) {                                                                                       \
        _Pragma("unroll") for (int c = 0; c < P; ++c)                                                     \
            _Pragma("unroll") for (int i = 0; i < E; ++i) v[c][i] = fmaf(v[c][i], at<T>(va[c], i), at<T>(vb[c], i)); \
    } else {                                                                                              \
        RS_EACH(g_, va, v[c][i] * t)                                                                      \
        RS_EACH(b_, vb, v[c][i] + t)                                                                      \
    }
        RS_VEC(va, post_g);
        RS_VEC(vb, post_b);
        RS_VEC_GATE(vc);
#pragma unroll
        for (int c = 0; c < P; ++c)
#pragma unroll
            for (int i = 0; i < E; ++i) v[c][i] = at<T>(w[c], i);
        row_norm<G, P, E>(v, p.post, p.post_eps, inv_d, n, sub, s_red);
        RS_AFFINE(p.post_g, p.post_b)
        RS_EACH(p.gate, vc, v[c][i] * t)
#pragma unroll
        for (int c = 0; c < P; ++c) {
#pragma unroll
            for (int i = 0; i < E; ++i) v[c][i] = sub + c * G < n ? fmaf(p.x_scale, at<T>(rx[c], i), p.f_scale * v[c][i]) : 0.f;
            if (p.y) put(rs_y, off[c], piece<T>(v[c]));
        }
        if (!p.u && !p.u_q) continue;
        RS_VEC(va, pre_g);
        RS_VEC(vb, pre_b);
        RS_VEC_MOD(vc, mod_scale);
        RS_VEC_MOD(vd, mod_shift);
        row_norm<G, P, E>(v, p.pre, p.pre_eps, inv_d, n, sub, s_red);
        RS_AFFINE(p.pre_g, p.pre_b)
        RS_EACH(p.mod_scale, vc, fmaf(v[c][i], t, v[c][i]))
        RS_EACH(p.mod_shift, vd, v[c][i] + t)
#undef RS_EACH
#undef RS_AFFINE
#undef RS_VEC
#undef RS_VEC_GATE
#undef RS_VEC_MOD
        if (p.u) {
#pragma unroll
            for (int c = 0; c < P; ++c) put(rs_u, off[c], piece<T>(v[c]));
        }
        if (p.u_q) {
            float amax = 0.f;
#pragma unroll
            for (int c = 0; c < P; ++c)
#pragma unroll
                for (int i = 0; i < E; ++i) {
                    v[c][i] = sub + c * G < n ? v[c][i] : 0.f;
                    amax = amax_step(amax, v[c][i]);
                }
            const QuantScale qs = quant_scale(row_amax<G>(amax, s_red));
            const int npad = (D + 15) / 16 * 16 / E;  // zeros up to a multiple of 16
#pragma unroll
            for (int c = 0; c < P; ++c) {
                uint32_t b[E / 4];
#pragma unroll
                for (int h = 0; h < E / 4; ++h) b[h] = quant8x4(v[c][4 * h], v[c][4 * h + 1], v[c][4 * h + 2], v[c][4 * h + 3], qs);
                if (on && sub + c * G < npad) {
                    int8_t* q = p.u_q + row * p.ldq + (sub + c * G) * E;
                    if constexpr (E == 8) *reinterpret_cast<uint2*>(q) = make_uint2(b[0], b[E / 4 - 1]);
                    else *reinterpret_cast<uint32_t*>(q) = b[0];
                }
            }
            if (on && sub == 0) p.u_scale[row] = qs.scale;
        }
    }
}

template <typename T, int G, int P>
static hipError_t go(const ResidualNormArgs& p, hipStream_t s) {
    constexpr int RPB = G > 64 ? 1 : 256 / G;
    const int64_t blocks = (p.rows + RPB - 1) / RPB;
    hipLaunchKernelGGL((residual_norm_kernel<T, G, P>), dim3((unsigned)(blocks < 1 << 20 ? blocks : 1 << 20)), dim3(G > 256 ? G : 256), 0, s, p);
    return hipGetLastError();
}

// The fewest lanes that hold a row in up to four pieces each: every lane busy at 192, 384 and 768 channels, where a wave per row
// leaves a quarter to five eighths of its lanes without work (512 x 197 x 192 bf16 79 -> 34 us, 256 x 197 x 768 97 -> 61).
// Where rows are too few to fill the chip so, one piece per lane: the way through is shorter.  Two LayerNorms, us, four pieces / one: 512
// channels at 1 row 5.2 / 3.4, at 2000 6.6 / 4.5; 256 at 4000 6.5 / 4.6; 1024 at 197 6.1 / 4.4, at 1000 6.6 / 6.0.
template <typename T>
static hipError_t launch_rn(const ResidualNormArgs& p, hipStream_t s) {
    const int n = p.D / kE<T>;
    const int64_t cus = device_cus();
    if (n <= 32 && p.rows <= 16 * cus) return go<T, 32, 1>(p, s);
    if (n > 32 && n <= 64 && p.rows <= 8 * cus) return go<T, 64, 1>(p, s);
    if (n > 64 && n <= 256 && p.rows <= 4 * cus) return go<T, 256, 1>(p, s);
    if (n <= 16) return go<T, 8, 2>(p, s);
    if (n <= 24) return go<T, 8, 3>(p, s);
    if (n <= 32) return go<T, 8, 4>(p, s);
    if (n <= 48) return go<T, 16, 3>(p, s);
    if (n <= 64) return go<T, 16, 4>(p, s);
    if (n <= 96) return go<T, 32, 3>(p, s);
    if (n <= 128) return go<T, 32, 4>(p, s);
    if (n <= 192) return go<T, 64, 3>(p, s);
    if (n <= 256) return go<T, 64, 4>(p, s);
    if (n <= 512) return go<T, 256, 2>(p, s);
    if (n <= 1024) return go<T, 256, 4>(p, s);
    if constexpr (sizeof(T) == 4)  // D > 8192
        if (n > 2048) return go<T, 1024, 4>(p, s);
    return go<T, 512, 4>(p, s);
}

hipError_t launch_residual_norm(rs_dtype dt, const ResidualNormArgs& p, hipStream_t s) {
    if (p.rows == 0) return hipSuccess;
    return dt == RS_F32 ? launch_rn<float>(p, s) : launch_rn<bf16raw>(p, s);
}

}  // namespace rs
