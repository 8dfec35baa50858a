// Linear layers in 8-bit integers (W8A8): out = epi((sum_k a[m,k] w[k,n]) (a_scale[m] w_scale[n]) + bias[n]), the sums exact in
// int32 (v_mfma_i32_32x32x32_i8), everything behind them in fp32, rounded once.
//
// Weights are packed in fragment order, [Np / 32][Kp / 32] fragments of 32 features x 32 k, 1 KB each, lane l's 16 bytes in
// a row: feature l & 31, k 16 (l >> 5) .. + 15; Np and Kp are N and K rounded up to 64 and 128, the rest is zeros.  A byte of
// `a` behind column K (up to the row's pitch, or of the next row) is multiplied by such a zero: being an integer it adds nothing.
#include <float.h>

#include <type_traits>

#include "gemm_i8_choice.hpp"
#include "gemm_tile.hpp"

namespace rs {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x16 __attribute__((ext_vector_type(16)));

size_t packed_i8_size(int K, int N) { return align_up((size_t)N, 64) * align_up((size_t)K, 128); }

// x Phi(x) for bf16 outputs: max(x, 0) - |x| Phi(-|x|), where nothing cancels, with Phi(-a) = 2^q(a) and q a polynomial fitted to
// log2 Phi(-a) over 0 <= a <= 9 (minimax, with weights 1000 times smaller at 9 than at 0).  At most 6.2e-7 off; of Phi(-a), 8e-6 up to
// a = 2, 2e-5 to 4, 1.4e-4 to 6, 1.7e-3 to 9: under half a step of bf16 (2^-9 .. 2^-8) wherever |x| Phi(-|x|) >= 1e-18.  Beyond, q only falls, and
// the product goes to 0 as it should.  A NaN stays one; the largest finite number in |x|'s place keeps an infinity from meeting the 0.
// 16388 x 1024 -> 4096 takes 86-91 us by the run, and 84-89 with the sigmoid that the bf16 layers of gemm.hip have (2.6e-5 off: at -4 3.6 % of the value,
// at -6 as much as the value); degree 10 (1.2e-7 off) takes 4 us more.
__device__ __forceinline__ float gelu_tail(float x) {
    const float a = fabsf(x);
    float q = fmaf(-1.480356e-6f, a, 5.4427055e-5f);
    q = fmaf(q, a, -8.753758e-4f);
    q = fmaf(q, a, 8.305447e-3f);
    q = fmaf(q, a, -5.359435e-2f);
    q = fmaf(q, a, -0.458766f);
    q = fmaf(q, a, -1.15116f);
    q = fmaf(q, a, -1.0000006f);
    return fmaf(-fminf(a, FLT_MAX), __builtin_amdgcn_exp2f(q), fmaxf(x, 0.f));
}
__device__ __forceinline__ float gelu_of(float x, const float*) { return gelu_erf(x); }
__device__ __forceinline__ float gelu_of(float x, const bf16raw*) { return gelu_tail(x); }

// ---------------------------------------------------------------------------
// Epilogue in the accumulator layout, as in the bf16 kernels (gemm_tile.hpp): lane (l32, g) holds, for row 32 j + l32, features
// 32 i + 8 q + 4 g + e in register 4 q + e of acc[i][j].  Only the traffic with memory goes through LDS, one 4 KB region (32 rows of
// 128 bytes) per 32-row group: residual rows arrive there by direct copies, a lane picks up its 4 features and puts the result
// back in place, the group leaves as 16 bytes per lane in whole row segments.  In bf16 a region holds the wave's 64 features, in
// fp32 32 of them, and a group goes in two passes.  Waves that store whole lines do so through the L2 (store16_wt); of other rows, and of half-filled
// regions, a line is written in parts, which only the L2 can join (fp32 43814 x 128 -> 6228 555 us written through, pass by pass; so 330.  Half-filled
// regions: the same either way, 788 x 768 -> 768 4.2 us, 50432 x 768 -> 64 12.0).  RAGGED: rows of `out` are no whole 16-byte pieces, so that they start
// anywhere; their pieces go at addresses aligned to the element (2013 x 64 -> 1356 with residual an element per lane 18.9 us, so 9.4).
// ---------------------------------------------------------------------------
template <typename T, int TN> struct EpiI8 {              // a wave of 32 TN features
    static constexpr int F = sizeof(T) == 4 ? 32 : 32 * TN;  // features of a region
    static constexpr int PASSES = 32 * TN / F;
    static constexpr int PIECES = F * (int)sizeof(T) / 16;   // of a row: 8, or 4 in half-filled regions (bf16, TN = 1)
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

// Piece c of a row that starts anywhere, of which `n` elements are inside: 16 bytes at an address aligned to the element only (which
// the hardware takes), the last elements one by one.
template <typename T> struct __attribute__((packed, aligned(sizeof(T)))) Piece16 { u32x4 v; };
template <typename T>
__device__ __forceinline__ u32x4 load_piece(const T* row, int c, int n) {
    constexpr int E = 16 / (int)sizeof(T);
    if ((c + 1) * E <= n) return reinterpret_cast<const Piece16<T>*>(row + c * E)->v;
    struct { T e[E]; } w;
#pragma unroll
    for (int i = 0; i < E; ++i) w.e[i] = c * E + i < n ? row[c * E + i] : T{};
    return __builtin_bit_cast(u32x4, w);
}
template <typename T>
__device__ __forceinline__ void store_piece(T* row, int c, int n, u32x4 v) {
    constexpr int E = 16 / (int)sizeof(T);
    if ((c + 1) * E <= n) {
        reinterpret_cast<Piece16<T>*>(row + c * E)->v = v;
        return;
    }
    struct W { T e[E]; };
    const W w = __builtin_bit_cast(W, v);
#pragma unroll
    for (int i = 0; i < E; ++i)
        if (c * E + i < n) row[c * E + i] = w.e[i];
}

// F features from n on of 32 residual rows into a region, and no more: the next ones are another wave's, which may be writing them by now (out
// may be res).  Rows past M read as zeros (or stay what they are), pieces past N are of the next row and not used.
template <typename T, bool RAGGED, int F>
__device__ __forceinline__ void i8_request_res(unsigned char* region, const T* res, int64_t M, int N, int64_t m, int n, int lane) {
    constexpr int PIECES = F * (int)sizeof(T) / 16;
    const int rows = (int)min(M - m, (int64_t)32);
    if (n >= N || rows <= 0) return;
    const T* base = res + m * N + n;
    if constexpr (RAGGED) {
#pragma unroll
        for (int p = 0; p < 4; ++p) {
            const int r = p * 8 + (lane >> 3), c = lane & 7;
            if (r < rows && c < PIECES) *reinterpret_cast<u32x4*>(region + r * 128 + ((c ^ epi_swz(r)) << 4)) = load_piece(base + (int64_t)r * N, c, N - n);
        }
    } else {
        const __amdgpu_buffer_rsrc_t rs_res = make_rsrc(base, ((int64_t)(rows - 1) * N + min(N - n, F)) * (int)sizeof(T));
#pragma unroll
        for (int p = 0; p < 4; ++p) {
            const int r = p * 8 + (lane >> 3), c = (lane & 7) ^ epi_swz(r);
            dma16(rs_res, region + p * 1024, c < PIECES ? r * N * (int)sizeof(T) + (c << 4) : kPastEnd, 0);
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
template <typename T, int EPI, int TM, bool RAGGED, int TN>
__device__ __forceinline__ void i8_epilogue(const i32x16 (&acc)[TN][TM], const EpiRegions<TM>& reg, const unsigned char* vec, const T* res, T* out,
                                            int64_t M, int N, int64_t m_base, int n_base, int row0, int f0, int lane) {
    constexpr int P = EpiI8<T, TN>::PASSES, F = EpiI8<T, TN>::F, NI = TN / P, PIECES = EpiI8<T, TN>::PIECES;
    const int l32 = lane & 31, g = lane >> 5;
    if (n_base >= N || m_base >= M) return;
    float as[TM];
#pragma unroll
    for (int j = 0; j < TM; ++j) as[j] = *reinterpret_cast<const float*>(vec + kVecRows + (row0 + j * 32 + l32) * 4);
    const int rows = (int)(M - m_base < 32 * TM ? M - m_base : 32 * TM);
    const bool lines = PIECES == 8 && (int64_t)N * sizeof(T) % 128 == 0;
    f32x4 ws[TN][4], bv[TN][4];
#pragma unroll
    for (int i = 0; i < TN; ++i)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int f = f0 + i * 32 + q * 8 + g * 4;
            ws[i][q] = *reinterpret_cast<const f32x4*>(vec + f * 4);
            bv[i][q] = bias4(vec + kVecBias + f * (int)sizeof(T), (const T*)nullptr);
        }
    // 32-row group j, features p F .. of the wave's, through the region at buf
    auto group = [&](int p, int j, unsigned char* buf) {
        const int n = n_base + p * F;
        if (n >= N) return;
#pragma unroll
        for (int i = 0; i < NI; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                unsigned char* at = buf + region_at<T>(l32, i * 32 + q * 8 + g * 4);
                float v[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int fi = P > 1 ? p : i;
                    v[e] = fmaf((float)acc[fi][j][4 * q + e], as[j] * ws[fi][q][e], bv[fi][q][e]);
                    if (EPI == EPI_BIAS_GELU) v[e] = gelu_of(v[e], (const T*)nullptr);
                }
                if (EPI == EPI_BIAS_RES) res_add(v, at, (const T*)nullptr);
                put4(at, v, (T*)nullptr);  // in place: this lane alone reads and writes these bytes
            }
        // the group leaves (LDS accesses of one wave are served in order)
        const __amdgpu_buffer_rsrc_t rs_out = make_rsrc(out + m_base * N + n, ((int64_t)(rows - 1) * N + min(N - n, F)) * (int)sizeof(T));
#pragma unroll
        for (int s = 0; s < PIECES / 2; ++s) {
            const int r = s * (64 / PIECES) + lane / PIECES, c = lane % PIECES;
            const u32x4 o4 = *reinterpret_cast<const u32x4*>(buf + r * 128 + ((c ^ epi_swz(r)) << 4));
            if constexpr (RAGGED) {
                if (j * 32 + r < rows) store_piece(out + (m_base + j * 32 + r) * N + n, c, N - n, o4);
            } else {
                const bool in = j * 32 + r < rows && n + c * (16 / (int)sizeof(T)) < N;
                const int at = in ? ((j * 32 + r) * N) * (int)sizeof(T) + c * 16 : kPastEnd;
                if (lines) store16_wt(rs_out, at, o4);
                else __builtin_amdgcn_raw_buffer_store_b128(o4, rs_out, at, 0, 0);
            }
        }
    };
    if (P > 1 && EPI != EPI_BIAS_RES && !RAGGED && lines) {
#pragma unroll
        for (int p = 0; p < P; ++p)
#pragma unroll
            for (int j = 0; j < TM; ++j) group(p, j, reg.r[j]);
        return;
    }
    // A row's passes one behind the other, so that a line they share is written at about one time (rows of whole lines: above, 16388 x 1024 ->
    // 4096 106 -> 102 us).  With a residual TM / P groups at a time, each pass in a region of its own.
    constexpr int GROUPS = EPI == EPI_BIAS_RES ? TM / P : TM;
#pragma unroll
    for (int j0 = 0; j0 < TM; j0 += GROUPS) {
        if constexpr (EPI == EPI_BIAS_RES) {
            if (j0 > 0) __builtin_amdgcn_s_waitcnt(0xC07F);  // what the last groups read from the regions has been read
#pragma unroll
            for (int j = 0; j < GROUPS; ++j)
#pragma unroll
                for (int p = 0; p < P; ++p) i8_request_res<T, RAGGED, F>(reg.r[j * P + p], res, M, N, m_base + (j0 + j) * 32, n_base + p * F, lane);
            __builtin_amdgcn_s_waitcnt(vmcnt_imm(0) & 0xC07F);  // all of them have landed
        }
#pragma unroll
        for (int j = 0; j < GROUPS; ++j)
#pragma unroll
            for (int p = 0; p < P; ++p) group(p, j0 + j, reg.r[EPI == EPI_BIAS_RES ? j * P + p : j]);
    }
}

// ---------------------------------------------------------------------------
// Direct kernel: workgroup tile 32 TM rows x 256 features, four waves of 32 TM x 64, two workgroups per CU.  Weights go from memory
// straight into the registers of the one wave that needs them, the activations through a ring of four LDS stages of 128 k, copied
// three slices ahead, as in gemm_bf16_direct_kernel, whose slices hold as many bytes.  TM = 8, one workgroup per CU with 256
// accumulator registers a lane: the weights of a slice serve twice the rows.
// What bounds the large layers is power first: 32768 x 4096 -> 4096 runs at 1.7 GHz with the matrix cores busy 70 % of the cycles (2.45
// POPS; a loop of nothing but these matrix instructions reaches 4.3), and a layer's time is the sum of what its products and its
// bytes cost (50432 x K -> 2304: 42 us + 0.088 us per k; stores and loads overlap in time but not in power; starting the second workgroup
// of a CU half a tile later changes nothing).  So the kernel with the fewest bytes moved per product wins where it fills the chip.
// 8192^3: 420 us, without the copies in the loop 390, without the weight loads 392, without both 363.  No better: waves of 128 x 128 in a 256 x 256
// tile (half the LDS reads, weights loaded by two waves each) 447; weights two slices ahead 429; the slices of neighbouring row
// panels in rotated order, for layers whose weights all panels read at once (no change).
// ---------------------------------------------------------------------------
template <typename T, int EPI, bool RAGGED, int TM>
__global__ __launch_bounds__(256, TM == 8 ? 1 : 2) void gemm_i8_direct_kernel(const int8_t* __restrict__ a, int lda, const float* __restrict__ a_scale,
                                                                const int8_t* __restrict__ w, const float* __restrict__ w_scale,
                                                                const T* __restrict__ bias, const T* res, T* out, int64_t M, int N, int K,
                                                                int tiles_m, int tiles_n, int gm) {
    constexpr int TN = 2, BM = 32 * TM, BN = 256, RB = 128, STAGE = BM * RB;
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
        _Pragma("unroll") for (int i = 0; i < TM; ++i)                                                    \
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
            __builtin_amdgcn_sched_group_barrier(0x020, TM == 2 ? 2 : 1, 0);                              \
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
        RS_I8_WAIT(2 * TM + 6)                                                                                    \
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
    RS_I8_WAIT(2 * TM + 8)  // slice 0 has landed: behind it at least 8 weight loads and two slices' copies
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
    i8_epilogue<T, EPI, TM, RAGGED, TN>(acc, reg, s_vec, res, out, M, N, m0, n_base, 0, wave * 64, lane);
}

// ---------------------------------------------------------------------------
// Split kernel, for the smallest problems: 32 rows x 32 TN features, the slices of K dealt out to the eight waves, two of them at a
// time in registers straight from memory, the partial sums added in LDS by integer atomics, whose order does not matter.
// What bounds such a call is the way to memory and back, once or twice, not bytes: no barrier before the sums meet, everything
// the epilogue reads requested behind the first slices.  (Slices past K requested and multiplied as zeros, without the peeled
// tail: 1 x 768 -> 2304 3.4 -> 4.1 us.)
// ---------------------------------------------------------------------------
template <typename T>
__device__ __forceinline__ void ld4(const T* p, int n, bool vec, float (&v)[4]) {  // n of 4 values
    if (vec) {
        if constexpr (sizeof(T) == 4) {
            const f32x4 r = *reinterpret_cast<const f32x4*>(p);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = r[e];
        } else {
            const uint2 r = *reinterpret_cast<const uint2*>(p);
            v[0] = __uint_as_float(r.x << 16); v[1] = __uint_as_float(r.x & 0xffff0000u);
            v[2] = __uint_as_float(r.y << 16); v[3] = __uint_as_float(r.y & 0xffff0000u);
        }
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = e < n ? Elem<T>::ld(p + e) : 0.f;
    }
}

template <typename T, int EPI, int TN>
__global__ __launch_bounds__(512, TN > 1 ? 2 : 4) void gemm_i8_split_kernel(
    const int8_t* __restrict__ a, int lda, const float* __restrict__ a_scale, const int8_t* __restrict__ w,
    const float* __restrict__ w_scale, const T* __restrict__ bias, const T* res, T* out, int64_t M, int N, int K, int tiles_n) {
    constexpr int W = 8, BM = 32, BN = 32 * TN, LD = BN + 1;
    __shared__ int s_sum[BM * LD];
    const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, g = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int64_t m0 = (int64_t)(blockIdx.x / tiles_n) * BM;
    const int n0 = (int)(blockIdx.x % tiles_n) * BN;
    const int S = (K + 127) >> 7, frag_row = S * 4096;
    const int rows = (int)(M - m0 < BM ? M - m0 : BM);
    const __amdgpu_buffer_rsrc_t rs_a = make_rsrc(a + m0 * lda, (int64_t)rows * lda);
    // rows of fragments: Np / 32 of them, an even number
    const __amdgpu_buffer_rsrc_t rs_w = make_rsrc(w + (int64_t)(n0 >> 5) * frag_row, (int64_t)TN * frag_row);
    const int aoff = l32 * lda + g * 16, woff = lane * 16;

    i32x4 av[2][4], wv[2][4][TN];
    i32x16 acc[TN];
    auto request = [&](int b, int kk, int t) {  // K step kk of slice t
#pragma unroll
        for (int j = 0; j < TN; ++j)
            wv[b][kk][j] = __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(rs_w, woff, j * frag_row + t * 4096 + kk * 1024, 0));
        av[b][kk] = __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(rs_a, aoff, t * 128 + kk * 32, 0));
    };
    // the products of a slice; more: each step's registers requested again for this wave's slice after next
    auto slice = [&](int b, int t, auto more) {
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) {
#pragma unroll
            for (int j = 0; j < TN; ++j) acc[j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(wv[b][kk][j], av[b][kk], acc[j], 0, 0, 0);
            if constexpr (decltype(more)::value) {
                request(b, kk, t + 2 * W);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
    };
#pragma unroll
    for (int b = 0; b < 2; ++b)
        if (wave + b * W < S) {
#pragma unroll
            for (int kk = 0; kk < 4; ++kk) request(b, kk, wave + b * W);
        }
    // Thread t writes features 4 (t % (BN / 4)) .. + 3 of row t / (BN / 4); the first 32 BN / 4 of the 512.
    constexpr int PER_ROW = BN / 4;
    const int ec = n0 + (tid % PER_ROW) * 4, er = tid / PER_ROW;
    const int ne = er < rows ? min(N - ec, 4) : 0;
    const bool vec = N % 4 == 0;
    float ws[4] = {0.f, 0.f, 0.f, 0.f}, bv[4] = {0.f, 0.f, 0.f, 0.f}, rv[4] = {0.f, 0.f, 0.f, 0.f}, as = 0.f;
    if (ne > 0) {
        ld4(w_scale + ec, ne, ne == 4, ws);
        if (bias) ld4(bias + ec, ne, ne == 4, bv);
        as = a_scale[m0 + er];
        if (EPI == EPI_BIAS_RES) ld4(res + (m0 + er) * N + ec, ne, vec, rv);
    }
    for (int i = tid; i < BM * LD; i += 64 * W) s_sum[i] = 0;
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[j][r] = 0;
    int t = wave;
    for (; t + 3 * W < S; t += 2 * W) {
        slice(0, t, std::true_type{});
        slice(1, t + W, std::true_type{});
    }
    if (t + 2 * W < S) {  // three slices left, two of them in registers
        slice(0, t, std::true_type{});
        slice(1, t + W, std::false_type{});
        slice(0, t + 2 * W, std::false_type{});
    } else {
        if (t < S) slice(0, t, std::false_type{});
        if (t + W < S) slice(1, t + W, std::false_type{});
    }
    __syncthreads();  // the sums are zero
    if (wave < S) {
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) atomicAdd(&s_sum[l32 * LD + j * 32 + (r >> 2) * 8 + g * 4 + (r & 3)], acc[j][r]);
    }
    __syncthreads();
    if (ne <= 0) return;
    float v[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        v[e] = fmaf((float)s_sum[er * LD + ec - n0 + e], as * ws[e], bv[e]);
        if (EPI == EPI_BIAS_GELU) v[e] = gelu_of(v[e], (const T*)nullptr);
        if (EPI == EPI_BIAS_RES) v[e] += rv[e];
    }
    T* o = out + (m0 + er) * N + ec;
    if (vec) {
        put4((unsigned char*)o, v, (T*)nullptr);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < ne) Elem<T>::st(o + e, v[e]);
    }
}

// ---------------------------------------------------------------------------
// Private kernel, for grids in between: 64 rows x 64 features, the slices of K dealt out to four waves, each with two stages of
// its own for the rows (whole lines by direct copies) and its weights in registers: no barrier before the sums meet.  They
// do so in LDS, where each wave collects the 32 x 32 block that it then writes (two waves, 32 rows each: 1003 x 588 -> 1000 fp32 with
// GELU 8.8 us, so 7.1).  Two workgroups per CU.
// (128 rows, one workgroup per CU: 512 x 4096 -> 4096 15.2 -> 13.9 us, where every CU has one such tile, elsewhere slower: 788 x 768 -> 2304
// 6.4 -> 6.8, 1576 x 4096 -> 1024 the same.)
// ---------------------------------------------------------------------------
template <typename T, int EPI, bool RAGGED>
__global__ __launch_bounds__(256, 2) void gemm_i8_private_kernel(
    const int8_t* __restrict__ a, int lda, const float* __restrict__ a_scale, const int8_t* __restrict__ w,
    const float* __restrict__ w_scale, const T* __restrict__ bias, const T* res, T* out, int64_t M, int N, int K, int tiles_m,
    int tiles_n, int gm) {
    constexpr int W = 4, TM = 2, TN = 2, BM = 32 * TM, BN = 64, RB = 128, STAGE = BM * RB;
    __shared__ __attribute__((aligned(1024))) unsigned char st0[W * STAGE];
    __shared__ __attribute__((aligned(1024))) unsigned char st1[W * STAGE];
    __shared__ __attribute__((aligned(1024))) unsigned char s_vec[kVecBytes];
    int64_t m0;
    int n0;
    {
        const int nblk = tiles_m * tiles_n;
        const int xcd = blockIdx.x & 7;
        const int xq = nblk >> 3, xr = nblk & 7;
        const int x_cnt = xq + (xcd < xr ? 1 : 0), x_start = xcd * xq + (xcd < xr ? xcd : xr);
        const int seq = blockIdx.x >> 3;
        if (seq >= x_cnt) return;  // whole workgroup, before any barrier
        const int bid = x_start + seq;
        const int per_group = gm * tiles_n;
        const int grp = bid / per_group, rem = bid - grp * per_group;
        const int first_m = grp * gm;
        const int gsz = min(tiles_m - first_m, gm);
        const int tn = rem / gsz;
        n0 = tn * BN;
        m0 = (int64_t)(first_m + rem - tn * gsz) * BM;
    }
    const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, g = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int S = (K + 127) >> 7, frag_row = S * 4096;
    const int64_t rows = M - m0 < BM ? M - m0 : BM;
    const __amdgpu_buffer_rsrc_t rs_a = make_rsrc(a + m0 * lda, rows * lda);
    const __amdgpu_buffer_rsrc_t rs_w = make_rsrc(w + (int64_t)(n0 >> 5) * frag_row, 2 * frag_row);
    const int ld_r = lane >> 3, ld_p = lane & 7;
    // copy i takes rows 8 i .. + 7; chunk c of row r in slot c ^ (r & 7) ^ ((r >> 3) & 1)
    const int voff0 = ld_r * lda + ((ld_p ^ ld_r) << 4), voff1 = (8 + ld_r) * lda + ((ld_p ^ ld_r ^ 1) << 4);
    const int sw = (l32 & 7) ^ ((l32 >> 3) & 1);
    const int woff0 = lane * 16, woff1 = woff0 + frag_row;
    const int mine = wave * STAGE;

    i32x4 wf[2][4][TN], f0[TM], f1[TM];
    i32x16 acc[TN][TM];
#define RS_I8_ROWS(stage_, t_)                                                                            \
    {                                                                                                     \
        const int kb_ = (t_) * RB;                                                                        \
        _Pragma("unroll") for (int i = 0; i < BM / 16; ++i) {                                             \
            dma16(rs_a, (stage_) + mine + i * 2048, voff0, i * 16 * lda + kb_);                           \
            dma16(rs_a, (stage_) + mine + i * 2048 + 1024, voff1, i * 16 * lda + kb_);                    \
        }                                                                                                 \
    }
#define RS_I8_W(b_, t_)                                                                                   \
    {                                                                                                     \
        _Pragma("unroll") for (int kk = 0; kk < 4; ++kk) {                                                \
            const int so_ = ((t_) * 4 + kk) * 1024;                                                       \
            wf[b_][kk][0] = __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(rs_w, woff0, so_, 0)); \
            wf[b_][kk][1] = __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(rs_w, woff1, so_, 0)); \
        }                                                                                                 \
    }
#define RS_I8_FRAGS(f_, stage_, kk_)                                                                      \
    {                                                                                                     \
        const int co_ = ((((kk_) * 2 + g) ^ sw) << 4);                                                    \
        _Pragma("unroll") for (int j = 0; j < TM; ++j)                                                    \
            f_[j] = *reinterpret_cast<const i32x4*>((stage_) + mine + (l32 + j * 32) * RB + co_);         \
    }
#define RS_I8_MFMA(f_, b_, kk_)                                                                           \
    {                                                                                                     \
        _Pragma("unroll") for (int i = 0; i < TN; ++i)                                                    \
            _Pragma("unroll") for (int j = 0; j < TM; ++j)                                                \
                acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(wf[b_][kk_][i], f_[j], acc[i][j], 0, 0, 0); \
    }
// A slice from stage_ and wf[b_]; what it has been waited for is the caller's
#define RS_I8_COMPUTE(stage_, b_)                                                                         \
    {                                                                                                     \
        RS_I8_FRAGS(f0, stage_, 0)                                                                        \
        RS_I8_FRAGS(f1, stage_, 1)                                                                        \
        RS_I8_MFMA(f0, b_, 0)                                                                             \
        RS_I8_FRAGS(f0, stage_, 2)                                                                        \
        RS_I8_MFMA(f1, b_, 1)                                                                             \
        RS_I8_FRAGS(f1, stage_, 3)                                                                        \
        RS_I8_MFMA(f0, b_, 2)                                                                             \
        RS_I8_MFMA(f1, b_, 3)                                                                             \
    }
    constexpr int SLICE_LOADS = BM / 8 + 8;
#define RS_I8_WAIT(n_)                                                                                    \
    {                                                                                                     \
        __builtin_amdgcn_s_waitcnt(((n_) & 15) | (((n_) >> 4) << 14) | 0x0070); /* and every LDS read */  \
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");                                            \
        __builtin_amdgcn_sched_barrier(0);                                                                \
    }
#pragma unroll
    for (int i = 0; i < TN; ++i)
#pragma unroll
        for (int j = 0; j < TM; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][j][r] = 0;
    i8_request_vecs<T, BM, BN>(s_vec, a_scale + m0, w_scale, bias, rows, N, n0, wave, lane);
    if (wave < S) {
        RS_I8_ROWS(st0, wave)
        RS_I8_W(0, wave)
    }
    __builtin_amdgcn_sched_barrier(0);
    int t = wave;
    for (; t + 2 * W < S; t += 2 * W) {  // a stage is free once its slice has been read: the next but one goes there
        RS_I8_ROWS(st1, t + W)
        RS_I8_W(1, t + W)
        RS_I8_WAIT(SLICE_LOADS)
        RS_I8_COMPUTE(st0, 0)
        RS_I8_WAIT(SLICE_LOADS)
        RS_I8_ROWS(st0, t + 2 * W)
        RS_I8_W(0, t + 2 * W)
        RS_I8_WAIT(SLICE_LOADS)
        RS_I8_COMPUTE(st1, 1)
        RS_I8_WAIT(SLICE_LOADS)
    }
    if (t + W < S) {
        RS_I8_ROWS(st1, t + W)
        RS_I8_W(1, t + W)
        RS_I8_WAIT(SLICE_LOADS)
        RS_I8_COMPUTE(st0, 0)
        RS_I8_WAIT(0)
        RS_I8_COMPUTE(st1, 1)
    } else if (t < S) {
        RS_I8_WAIT(0)
        RS_I8_COMPUTE(st0, 0)
    }
#undef RS_I8_ROWS
#undef RS_I8_W
#undef RS_I8_FRAGS
#undef RS_I8_MFMA
#undef RS_I8_COMPUTE
#undef RS_I8_WAIT
    // Wave f collects 32 x 32 block f, features 32 (f / 2) .. of rows 32 (f % 2) ..: the others leave theirs in slots of
    // 4 KB, [block][other wave], 16 bytes per lane.
    __builtin_amdgcn_s_waitcnt(vmcnt_imm(0) & 0xC07F);  // the vectors have landed
    __syncthreads();  // every wave has read its stages
    static_assert(TM * TN == W && W * (W - 1) * 4096 <= 2 * W * STAGE, "a block for each wave, slots in the stages");
    constexpr int PER = W * STAGE / 4096;  // slots of a stage array
    auto slot = [&](int f, int from) {
        const int at = f * (W - 1) + from;
        return (at < PER ? st0 + at * 4096 : st1 + (at - PER) * 4096) + lane * 16;
    };
    i32x16 sum[1][1];
#pragma unroll
    for (int f = 0; f < W; ++f) {
        const i32x16& own = acc[f >> 1][f & 1];
        if (f == wave) {
#pragma unroll
            for (int r = 0; r < 16; ++r) sum[0][0][r] = own[r];
        } else {
            unsigned char* s = slot(f, wave - (wave > f ? 1 : 0));
#pragma unroll
            for (int q = 0; q < 4; ++q) *reinterpret_cast<i32x4*>(s + q * 1024) = i32x4{own[4 * q], own[4 * q + 1], own[4 * q + 2], own[4 * q + 3]};
        }
    }
    __syncthreads();
#pragma unroll
    for (int o = 0; o < W - 1; ++o) {
        const unsigned char* s = slot(wave, o);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const i32x4 v = *reinterpret_cast<const i32x4*>(s + q * 1024);
#pragma unroll
            for (int e = 0; e < 4; ++e) sum[0][0][4 * q + e] += v[e];
        }
    }
    EpiRegions<1> reg;
    reg.r[0] = slot(wave, 0) - lane * 16;  // read by this wave alone, and it has been read
    __builtin_amdgcn_s_waitcnt(0xC07F);
    const int fo = (wave >> 1) * 32, ro = (wave & 1) * 32;
    i8_epilogue<T, EPI, 1, RAGGED, 1>(sum, reg, s_vec, res, out, M, N, m0 + ro, n0 + fo, ro, fo, lane);
}

template <typename T, int EPI, bool RAGGED, int TM>
static void launch_i8_direct(const GemmI8Args& g, hipStream_t s) {
    const int tiles_m = (int)((g.M + 32 * TM - 1) / (32 * TM)), tiles_n = (g.N + 255) / 256, nblk = tiles_m * tiles_n;
    hipLaunchKernelGGL((gemm_i8_direct_kernel<T, EPI, RAGGED, TM>), dim3(8 * ((nblk + 7) / 8)), dim3(256), 0, s, g.a, (int)g.lda, g.a_scale,
                       (const int8_t*)g.w, g.w_scale, (const T*)g.bias, (const T*)g.res, (T*)g.out, g.M, g.N, g.K, tiles_m, tiles_n, TM == 8 ? 8 : 16);  // row panels that pass together
}

template <typename T, int EPI, bool RAGGED>
static void launch_i8_private(const GemmI8Args& g, hipStream_t s) {
    const int tiles_m = (int)((g.M + 63) / 64), tiles_n = (g.N + 63) / 64, nblk = tiles_m * tiles_n;
    hipLaunchKernelGGL((gemm_i8_private_kernel<T, EPI, RAGGED>), dim3(8 * ((nblk + 7) / 8)), dim3(256), 0, s, g.a, (int)g.lda, g.a_scale,
                       (const int8_t*)g.w, g.w_scale, (const T*)g.bias, (const T*)g.res, (T*)g.out, g.M, g.N, g.K, tiles_m, tiles_n, 16);
}

template <typename T, int EPI, int TN>
static void launch_i8_split(const GemmI8Args& g, hipStream_t s) {
    const int tiles_n = (g.N + 32 * TN - 1) / (32 * TN), tiles = (int)((g.M + 31) / 32 * tiles_n);
    hipLaunchKernelGGL((gemm_i8_split_kernel<T, EPI, TN>), dim3(tiles), dim3(512), 0, s, g.a, (int)g.lda, g.a_scale, (const int8_t*)g.w,
                       g.w_scale, (const T*)g.bias, (const T*)g.res, (T*)g.out, g.M, g.N, g.K, tiles_n);
}

template <typename T, int EPI, bool RAGGED>
static void launch_i8_part(const GemmI8Args& g, hipStream_t s) {
    switch (gemm_i8_choose(g.M, g.N, g.K, device_cus())) {
        case GemmI8Tile::Split32x32: launch_i8_split<T, EPI, 1>(g, s); break;
        case GemmI8Tile::Split32x64: launch_i8_split<T, EPI, 2>(g, s); break;
        case GemmI8Tile::Private64x64: launch_i8_private<T, EPI, RAGGED>(g, s); break;
        case GemmI8Tile::Direct64x256: launch_i8_direct<T, EPI, RAGGED, 2>(g, s); break;
        case GemmI8Tile::Direct128x256: launch_i8_direct<T, EPI, RAGGED, 4>(g, s); break;
        case GemmI8Tile::Direct256x256: launch_i8_direct<T, EPI, RAGGED, 8>(g, s); break;
    }
}

// Rows in parts of at most 2^22 tiles of 128 x 64: 2^23 workgroups of the smallest tile that takes so many rows (a launch holds fewer than 2^32
// threads).
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
        if ((int64_t)g.N * sizeof(T) % 16) launch_i8_part<T, EPI, true>(p, s);
        else launch_i8_part<T, EPI, false>(p, s);
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
