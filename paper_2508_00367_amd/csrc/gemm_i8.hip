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

// ---------------------------------------------------------------------------
// Epilogue in the accumulator layout, as in the bf16 kernels (gemm_tile.hpp): lane (l32, g) holds, for row 32 j + l32, features
// 32 i + 8 q + 4 g + e in register 4 q + e of acc[i][j].  Only the traffic with memory goes through LDS, one 4 KB region (32 rows of
// 128 bytes) per 32-row group: residual rows arrive there by direct copies, a lane picks up its 4 features and puts the result
// back in place, the group leaves as 16 bytes per lane in whole row segments.  In bf16 a region holds the wave's 64 features, in
// fp32 32 of them, and the features go in two passes.  Rows of `out` that are not whole 16-byte pieces (RAGGED) are
// read and written an element per lane.
// ---------------------------------------------------------------------------
template <typename T> struct EpiI8 {
    static constexpr int PASSES = sizeof(T) / 2;        // over the wave's 64 features
    static constexpr int F = 64 / PASSES;               // features of a region
};

// w_scale, bias and a_scale of a tile in LDS: 256 features in fp32, 256 of T, 256 rows.
constexpr int kVecBias = 1024, kVecRows = 2048, kVecBytes = 3072;

// Requests the vectors of a tile of BM rows and BN features with the first waves; past M and N zeros (nothing of it is stored).
template <typename T, int BM, int BN>
__device__ __forceinline__ void i8_request_vecs(unsigned char* s, const float* a_scale, const float* w_scale, const T* bias, int64_t rows,
                                                int N, int n0, int wave, int lane) {
    static_assert(BM <= 256 && BN <= 256, "vectors of a tile");
    const int f = max(min(N - n0, BN), 0);
    if (wave == 0) dma16(make_rsrc(w_scale + n0, f * 4), s, lane * 16, 0);
    // the range check goes by whole words: an odd count of bf16 reads the word that holds its last one
    if (wave == 1) dma16(make_rsrc(bias ? bias + n0 : bias, bias ? (f * (int)sizeof(T) + 3) & ~3 : 0), s + kVecBias, lane * 16, 0);
    // row scales need only be 4-byte aligned
    const __amdgpu_buffer_rsrc_t rs_s = make_rsrc(a_scale, rows * 4);
#pragma unroll
    for (int i = 0; i < BM / 64; ++i)
        if (wave == 2 + (i & 1)) __builtin_amdgcn_raw_ptr_buffer_load_lds(rs_s, (lds_ptr)(s + kVecRows + i * 256), 4, lane * 4, i * 256, 0, 0);
}

template <typename T>
__device__ __forceinline__ int region_at(int r, int f) {  // byte of feature f (of the region's) of row r
    const int b = f * (int)sizeof(T);
    return r * 128 + (((b >> 4) ^ epi_swz(r)) << 4) + (b & 15);
}

// Residual rows of one pass into the regions; rows past M read as zeros, pieces past N are of the next row and not used.
template <typename T, int TM, bool RAGGED>
__device__ __forceinline__ void i8_request_res(const EpiRegions<TM>& reg, const T* res, int64_t M, int N, int64_t m_base, int n,
                                               int lane) {
    const int64_t left = M - m_base;
    if (n >= N || left <= 0) return;
    const int rows = (int)(left < 32 * TM ? left : 32 * TM);
    const T* base = res + m_base * N + n;
    if constexpr (RAGGED) {
        constexpr int F = EpiI8<T>::F, RPI = 64 / F;
        const int f = lane % F;
        for (int r = lane / F; r < rows; r += RPI)
            if (n + f < N) *reinterpret_cast<T*>(reg.r[0] + (r >> 5) * 4096 + region_at<T>(r & 31, f)) = base[(int64_t)r * N + f];
    } else {
        const int64_t bytes = ((int64_t)(rows - 1) * N + min(N - n, EpiI8<T>::F)) * (int)sizeof(T);
        const __amdgpu_buffer_rsrc_t rs_res = make_rsrc(base, bytes);
#pragma unroll
        for (int p = 0; p < 4; ++p) {
            const int r = p * 8 + (lane >> 3);
            const int voff = r * N * (int)sizeof(T) + (((lane & 7) ^ epi_swz(r)) << 4);
#pragma unroll
            for (int j = 0; j < TM; ++j) dma16(rs_res, reg.r[j] + p * 1024, voff, j * 32 * N * (int)sizeof(T));
        }
    }
}

__device__ __forceinline__ void res_add(float (&v)[4], const unsigned char* at, const bf16raw*) {
    const uint2 r = *reinterpret_cast<const uint2*>(at);
    v[0] += __uint_as_float(r.x << 16); v[1] += __uint_as_float(r.x & 0xffff0000u);
    v[2] += __uint_as_float(r.y << 16); v[3] += __uint_as_float(r.y & 0xffff0000u);
}
__device__ __forceinline__ void res_add(float (&v)[4], const unsigned char* at, const float*) {
    const f32x4 r = *reinterpret_cast<const f32x4*>(at);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] += r[e];
}
__device__ __forceinline__ void put4(unsigned char* at, const float (&v)[4], bf16raw*) {
    *reinterpret_cast<uint2*>(at) = make_uint2(pack2bf(v[0], v[1]), pack2bf(v[2], v[3]));
}
__device__ __forceinline__ void put4(unsigned char* at, const float (&v)[4], float*) {
    *reinterpret_cast<f32x4*>(at) = f32x4{v[0], v[1], v[2], v[3]};
}
__device__ __forceinline__ f32x4 bias4(const unsigned char* at, const bf16raw*) {
    const uint2 r = *reinterpret_cast<const uint2*>(at);
    return f32x4{__uint_as_float(r.x << 16), __uint_as_float(r.x & 0xffff0000u), __uint_as_float(r.y << 16), __uint_as_float(r.y & 0xffff0000u)};
}
__device__ __forceinline__ f32x4 bias4(const unsigned char* at, const float*) { return *reinterpret_cast<const f32x4*>(at); }

// `vec`: the tile's vectors (landed); row0 and f0: the wave's first row and feature inside the tile.  The regions are this wave's
// own and consecutive 4 KB apart (one array per wave).
template <typename T, int EPI, int TM, bool RAGGED>
__device__ __forceinline__ void i8_epilogue(const i32x16 (&acc)[2][TM], const EpiRegions<TM>& reg, const unsigned char* vec, const T* res, T* out, int64_t M, int N, int64_t m_base, int n_base, int row0, int f0, int lane) {
    constexpr int P = EpiI8<T>::PASSES, F = EpiI8<T>::F;
    const int l32 = lane & 31, g = lane >> 5;
    if (n_base >= N || m_base >= M) return;
    float as[TM];
#pragma unroll
    for (int j = 0; j < TM; ++j) as[j] = *reinterpret_cast<const float*>(vec + kVecRows + (row0 + j * 32 + l32) * 4);
    const int rows = (int)(M - m_base < 32 * TM ? M - m_base : 32 * TM);
#pragma unroll
    for (int p = 0; p < P; ++p) {
        const int n = n_base + p * F;
        if (n >= N) break;
        if (EPI == EPI_BIAS_RES) {
            if (p > 0) __builtin_amdgcn_s_waitcnt(0xC07F);  // what the last pass reads from the regions has been read
            i8_request_res<T, TM, RAGGED>(reg, res, M, N, m_base, n, lane);
            __builtin_amdgcn_s_waitcnt(vmcnt_imm(0) & 0xC07F);  // every residual row of the pass has landed
        }
        f32x4 ws[2 / P][4], bv[2 / P][4];
#pragma unroll
        for (int i = 0; i < 2 / P; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int f = f0 + p * F + i * 32 + q * 8 + g * 4;
                ws[i][q] = *reinterpret_cast<const f32x4*>(vec + f * 4);
                bv[i][q] = bias4(vec + kVecBias + f * (int)sizeof(T), (const T*)nullptr);
            }
        const __amdgpu_buffer_rsrc_t rs_out = make_rsrc(out + m_base * N + n, ((int64_t)(rows - 1) * N + min(N - n, F)) * (int)sizeof(T));
#pragma unroll
        for (int j = 0; j < TM; ++j) {
            unsigned char* buf = reg.r[j];
#pragma unroll
            for (int i = 0; i < 2 / P; ++i)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    unsigned char* at = buf + region_at<T>(l32, i * 32 + q * 8 + g * 4);
                    float v[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        v[e] = fmaf((float)acc[P == 2 ? p : i][j][4 * q + e], as[j] * ws[i][q][e], bv[i][q][e]);
                        if (EPI == EPI_BIAS_GELU) v[e] = gelu_of(v[e], (const T*)nullptr);
                    }
                    if (EPI == EPI_BIAS_RES) res_add(v, at, (const T*)nullptr);
                    put4(at, v, (T*)nullptr);  // in place: this lane alone reads and writes these bytes
                }
            // the group leaves (LDS accesses of one wave are served in order)
            if constexpr (RAGGED) {
                constexpr int RPI = 64 / F;
                const int f = lane % F;
                for (int r = lane / F; r < 32 && j * 32 + r < rows; r += RPI) {
                    const T v = *reinterpret_cast<const T*>(buf + region_at<T>(r, f));
                    if (n + f < N) out[(m_base + j * 32 + r) * N + n + f] = v;
                }
            } else {
#pragma unroll
                for (int s = 0; s < 4; ++s) {
                    const int r = s * 8 + (lane >> 3), c = lane & 7;
                    const u32x4 o4 = *reinterpret_cast<const u32x4*>(buf + r * 128 + ((c ^ epi_swz(r)) << 4));
                    const bool in = j * 32 + r < rows && n + c * (16 / (int)sizeof(T)) < N;
                    store16_wt(rs_out, in ? ((j * 32 + r) * N) * (int)sizeof(T) + c * 16 : kPastEnd, o4);
                }
            }
        }
    }
}

// ---------------------------------------------------------------------------
// Direct kernel: workgroup tile 128 rows x 256 features, four waves of 128 x 64, two workgroups per CU.  Weights go from memory
// straight into the registers of the one wave that needs them, the activations through a ring of four LDS stages of 128 k, copied
// three slices ahead, as in gemm_bf16_direct_kernel, whose slices hold as many bytes.
// ---------------------------------------------------------------------------
template <typename T, int EPI, bool RAGGED>
__global__ __launch_bounds__(256, 2) void gemm_i8_direct_kernel(const int8_t* __restrict__ a, int lda, const float* __restrict__ a_scale,
                                                                const int8_t* __restrict__ w, const float* __restrict__ w_scale,
                                                                const T* __restrict__ bias, const T* res, T* out, int64_t M, int N, int K,
                                                                int tiles_m, int tiles_n, int gm) {
    constexpr int TM = 4, TN = 2, BM = 128, BN = 256, RB = 128, STAGE = BM * RB;
    __shared__ __attribute__((aligned(1024))) unsigned char st0[STAGE];
    __shared__ __attribute__((aligned(1024))) unsigned char st1[STAGE];
    __shared__ __attribute__((aligned(1024))) unsigned char st2[STAGE];
    __shared__ __attribute__((aligned(1024))) unsigned char st3[STAGE];
    __shared__ __attribute__((aligned(1024))) unsigned char s_vec[kVecBytes];

    const int nblk = tiles_m * tiles_n;
    const int xcd = blockIdx.x & 7;
    const int xq = nblk >> 3, xr = nblk & 7;
    const int x_cnt = xq + (xcd < xr ? 1 : 0), x_start = xcd * xq + (xcd < xr ? xcd : xr);
    const int seq = blockIdx.x >> 3;
    if (seq >= x_cnt) return;  // whole workgroup, before any barrier
    int64_t m0;
    int n0;
    {
        const int bid = x_start + seq;
        const int per_group = gm * tiles_n;
        const int grp = bid / per_group, rem = bid - grp * per_group;
        const int first_m = grp * gm;
        const int gsz = min(tiles_m - first_m, gm);
        const int tn = rem / gsz;
        n0 = tn * BN;
        m0 = (int64_t)(first_m + rem - tn * gsz) * BM;
    }

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l32 = lane & 31, g = lane >> 5;
    const int n_base = n0 + wave * 64;
    const int S = (K + 127) >> 7, frag_row = S * 4096;  // bytes of a row of fragments

    const int64_t rows = M - m0 < BM ? M - m0 : BM;
    const __amdgpu_buffer_rsrc_t rs_a = make_rsrc(a + m0 * lda, rows * lda);
    const __amdgpu_buffer_rsrc_t rs_w = make_rsrc(n_base < N ? w + (int64_t)(n_base >> 5) * frag_row : w, n_base < N ? 2 * frag_row : 0);
    const int ld_r = lane >> 3, ld_p = lane & 7;
    const int voff = (wave * 8 + ld_r) * lda + ((ld_p ^ ld_r ^ (wave & 1)) << 4);
    const int pass_bytes = 32 * lda;
    const int sw = (l32 & 7) ^ ((l32 >> 3) & 1);
    const int woff0 = lane * 16, woff1 = woff0 + frag_row;

#define RS_I8_DMA(stage_, t_)                                                                             \
    {                                                                                                     \
        const bool real_ = (t_) < S;                                                                      \
        const int kb_ = (t_) * RB;                                                                        \
        _Pragma("unroll") for (int i = 0; i < 4; ++i)                                                     \
            dma16(rs_a, (stage_) + (i * 4 + wave) * 1024, voff, real_ ? i * pass_bytes + kb_ : kPastEnd); \
    }
// weights of K step kk_ of slice t_
#define RS_I8_W(kk_, t_)                                                                                  \
    {                                                                                                     \
        const int so_ = (t_) < S ? ((t_) * 4 + (kk_)) * 1024 : kPastEnd;                                  \
        wf[kk_][0] = __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(rs_w, woff0, so_, 0)); \
        wf[kk_][1] = __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(rs_w, woff1, so_, 0)); \
    }
#define RS_I8_FRAGS(f_, stage_, kk_)                                                                      \
    {                                                                                                     \
        const int co_ = ((((kk_) * 2 + g) ^ sw) << 4);                                                    \
        _Pragma("unroll") for (int j = 0; j < TM; ++j)                                                    \
            f_[j] = *reinterpret_cast<const i32x4*>((stage_) + (l32 + j * 32) * RB + co_);                \
    }
#define RS_I8_MFMA(f_, kk_)                                                                               \
    {                                                                                                     \
        _Pragma("unroll") for (int i = 0; i < TN; ++i)                                                    \
            _Pragma("unroll") for (int j = 0; j < TM; ++j)                                                \
                acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(wf[kk_][i], f_[j], acc[i][j], 0, 0, 0); \
    }
// one K step: an LDS read of the next step's rows, two MFMAs, a request
#define RS_I8_INTERLEAVE()                                                                                \
    {                                                                                                     \
        _Pragma("unroll") for (int s_ = 0; s_ < TM; ++s_) {                                               \
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);                                            \
            __builtin_amdgcn_sched_group_barrier(0x008, TN, 0);                                           \
            __builtin_amdgcn_sched_group_barrier(0x020, 1, 0);                                            \
        }                                                                                                 \
        __builtin_amdgcn_sched_barrier(0);                                                                \
    }
// Everything but the newest n_ requests has been answered, and this wave's LDS reads all have.
#define RS_I8_WAIT(n_)                                                                                    \
    {                                                                                                     \
        __builtin_amdgcn_s_waitcnt(((n_) & 15) | (((n_) >> 4) << 14) | 0x0070);                           \
        __builtin_amdgcn_s_barrier();                                                                     \
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup"); /* LDS reads stay below the barrier */     \
        __builtin_amdgcn_sched_barrier(0);                                                                \
    }
// Slice t from cur_ (its first fragments are in f0).  fre_ held slice t - 1, which every wave has read before the last
// barrier: the copies of slice t + 3 go there.  At this slice's barrier those of slice t + 1 must have landed: behind them
// lie at least the copies of slices t + 2 and t + 3 and this slice's 6 weight loads.
#define RS_I8_SLICE(cur_, nxt_, fre_, t_)                                                                 \
    {                                                                                                     \
        RS_I8_DMA(fre_, (t_) + 3)                                                                         \
        RS_I8_FRAGS(f1, cur_, 1)                                                                          \
        RS_I8_MFMA(f0, 0)                                                                                 \
        RS_I8_INTERLEAVE()                                                                                \
        RS_I8_W(0, (t_) + 1)                                                                              \
        RS_I8_FRAGS(f0, cur_, 2)                                                                          \
        RS_I8_MFMA(f1, 1)                                                                                 \
        RS_I8_INTERLEAVE()                                                                                \
        RS_I8_W(1, (t_) + 1)                                                                              \
        RS_I8_FRAGS(f1, cur_, 3)                                                                          \
        RS_I8_MFMA(f0, 2)                                                                                 \
        RS_I8_INTERLEAVE()                                                                                \
        RS_I8_W(2, (t_) + 1)                                                                              \
        RS_I8_WAIT(14)                                                                                    \
        RS_I8_FRAGS(f0, nxt_, 0)                                                                          \
        RS_I8_MFMA(f1, 3)                                                                                 \
        RS_I8_INTERLEAVE()                                                                                \
        RS_I8_W(3, (t_) + 1)                                                                              \
    }

    i32x4 wf[4][TN], f0[TM], f1[TM];
    i32x16 acc[TN][TM];
#pragma unroll
    for (int i = 0; i < TN; ++i)
#pragma unroll
        for (int j = 0; j < TM; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][j][r] = 0;
    RS_I8_DMA(st0, 0)
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int kk = 0; kk < 4; ++kk) RS_I8_W(kk, 0)
    __builtin_amdgcn_sched_barrier(0);
    RS_I8_DMA(st1, 1)
    RS_I8_DMA(st2, 2)
    i8_request_vecs<T, BM, BN>(s_vec, a_scale + m0, w_scale, bias, rows, N, n0, wave, lane);
    RS_I8_WAIT(16)  // slice 0 has landed: behind it at least 8 weight loads and two slices' copies
    RS_I8_FRAGS(f0, st0, 0)
    const int full = S & ~3, left = S & 3;
    for (int t = 0; t < full; t += 4) {
        RS_I8_SLICE(st0, st1, st3, t)
        RS_I8_SLICE(st1, st2, st0, t + 1)
        RS_I8_SLICE(st2, st3, st1, t + 2)
        RS_I8_SLICE(st3, st0, st2, t + 3)
    }
    if (left > 0) {
        RS_I8_SLICE(st0, st1, st3, full)
        if (left > 1) RS_I8_SLICE(st1, st2, st0, full + 1)
        if (left > 2) RS_I8_SLICE(st2, st3, st1, full + 2)
    }
    RS_I8_WAIT(0)  // trailing (empty) copies: the stages get reused
#undef RS_I8_DMA
#undef RS_I8_W
#undef RS_I8_FRAGS
#undef RS_I8_MFMA
#undef RS_I8_INTERLEAVE
#undef RS_I8_WAIT
#undef RS_I8_SLICE

    EpiRegions<TM> reg;
    unsigned char* const base = wave == 0 ? st0 : wave == 1 ? st1 : wave == 2 ? st2 : st3;
#pragma unroll
    for (int j = 0; j < TM; ++j) reg.r[j] = base + j * 4096;
    i8_epilogue<T, EPI, TM, RAGGED>(acc, reg, s_vec, res, out, M, N, m0, n_base, 0, wave * 64, lane);
}

template <typename T, int EPI, bool RAGGED>
static void launch_i8_direct(const GemmI8Args& g, hipStream_t s) {
    const int tiles_m = (int)((g.M + 127) / 128), tiles_n = (g.N + 255) / 256, nblk = tiles_m * tiles_n;
    hipLaunchKernelGGL((gemm_i8_direct_kernel<T, EPI, RAGGED>), dim3(8 * ((nblk + 7) / 8)), dim3(256), 0, s, g.a, (int)g.lda, g.a_scale,
                       (const int8_t*)g.w, g.w_scale, (const T*)g.bias, (const T*)g.res, (T*)g.out, g.M, g.N, g.K, tiles_m, tiles_n, 16);
}

// Rows in parts of at most 2^22 tiles of 128 x 64 (a launch holds fewer than 2^32 threads).
template <typename T, int EPI>
static hipError_t launch_i8(const GemmI8Args& g, hipStream_t s) {
    const int64_t rows = ((int64_t)1 << 22) / ((g.N + 63) / 64) * 128;
    for (int64_t r = 0; r < g.M; r += rows) {
        GemmI8Args p = g;
        p.a = g.a + r * g.lda;
        p.a_scale = g.a_scale + r;
        p.res = g.res ? (const T*)g.res + r * g.N : nullptr;
        p.out = (T*)g.out + r * g.N;
        p.M = g.M - r < rows ? g.M - r : rows;
        if ((int64_t)g.N * sizeof(T) % 16) launch_i8_direct<T, EPI, true>(p, s);
        else launch_i8_direct<T, EPI, false>(p, s);
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
