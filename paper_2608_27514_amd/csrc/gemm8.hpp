// Matrix product with 8-bit operands (fp8.hpp): D[M,N] = A[M,K] W[K,N] (+ D).  W comes in e4m3 with a scale per block of
// 128 x 128, A in bf16 and is taken to e4m3 with a scale per row and 128 of k; fp32 accumulation on the matrix core, whose
// 8-bit products take both scales, one bf16 rounding of each result.
//   quantize8_kernel       W to 8 bits, once
//   quantize8_rows_kernel  A to 8 bits, into the workspace
//   gemm8_ring_kernel      the product
//
// Operands lie in slabs of 64 of k: [k / 64][row][k % 64], rows being rows of A and columns of W, and K padded with zeros
// to a multiple of 128.  So what a workgroup needs of a slab is contiguous, whole lines however few of k a stage holds, and
// both operands are k-contiguous: a fragment (32 of k of a row) is two 16-byte LDS reads, with no transposition.
#pragma once

#include "fp8.hpp"
#include "gemm.hpp"

namespace trajspec {

constexpr int kG8Block = 128;  // of k (and of columns of W) per scale
constexpr int kG8Slab = 64;
constexpr int64_t kG8MaxK = 65536;

typedef int i32x8_t __attribute__((ext_vector_type(8)));

// ------------------------------------------------------------------ W
// A workgroup per 128 x 128 block: 4 x 8 values (4 of k, 8 columns) per thread and turn, whose bytes go through LDS, so that
// both sides move whole lines.  Bound by the copy.
// grid: x = blocks of columns, y = blocks of k
constexpr int kQ8Row = 132;  // LDS bytes per column: the 32 words that half a wave writes lie in banks of their own
__global__ __launch_bounds__(256) void quantize8_kernel(const uint16_t* __restrict__ w, uint8_t* __restrict__ w8, uint8_t* __restrict__ scale,
                                                        int K, int N) {
    __shared__ __align__(16) uint8_t lds[kG8Block * kQ8Row];
    __shared__ uint32_t sh_max[4];
    const int tid = threadIdx.x, c = tid & 15, rg = tid >> 4;
    const int64_t n0 = (int64_t)blockIdx.x * kG8Block;
    const int k0 = blockIdx.y * kG8Block;
    u32x4_t x[2][4];
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int k = k0 + 4 * (rg + 16 * i) + j;
            x[i][j] = u32x4_t{};
            if (k < K && n0 + 8 * c < N) x[i][j] = ldg16(w + (int64_t)k * N + n0 + 8 * c);
#pragma unroll
            for (int e = 0; e < 4; ++e) m = max(m, max(magnitude_bits(bf16_lo(x[i][j][e])), magnitude_bits(bf16_hi(x[i][j][e]))));
        }
#pragma unroll
    for (int t = 0; t < 6; ++t) {
        uint32_t a, b;
        lane_pair(t, m, a, b);
        m = max(a, b);
    }
    if ((tid & 63) == 0) sh_max[tid >> 6] = m;
    __syncthreads();
    const uint32_t byte = scale_byte(max(max(sh_max[0], sh_max[1]), max(sh_max[2], sh_max[3])));
    if (tid == 0) scale[(int64_t)blockIdx.x * gridDim.y + blockIdx.y] = (uint8_t)byte;
    const float inv = scale_inverse(byte);
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            float v[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = (e % 2 == 0 ? bf16_lo(x[i][j][e / 2]) : bf16_hi(x[i][j][e / 2])) * inv;
            *reinterpret_cast<uint32_t*>(lds + (8 * c + e) * kQ8Row + 4 * (rg + 16 * i)) = pack_e4m3(v[0], v[1], v[2], v[3]);
        }
    __syncthreads();
    // a column's 64 bytes of a slab by 16 threads
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const int q = tid + 256 * i, word = q & 15, n = q / 16 & 127, slab = q / 2048;
        if (n0 + n < N)
            *reinterpret_cast<uint32_t*>(w8 + ((int64_t)(2 * blockIdx.y + slab) * N + n0 + n) * kG8Slab + 4 * word) =
                *reinterpret_cast<const uint32_t*>(lds + n * kQ8Row + slab * kG8Slab + 4 * word);
    }
}

// ------------------------------------------------------------------ A
// The scale byte of row r in block kb, in the order that the product reads: a word holds those of rows r, r + 32, r + 64 and
// r + 96 of 128.
__device__ __forceinline__ int64_t g8_scale_at(int64_t r, int kb, int blocks) {
    return (((r >> 7) * blocks + kb) * 32 + (r & 31)) * 4 + ((r >> 5) & 3);
}

// 16 lanes per row and block of 128, 8 values each.  grid: x = groups of 16 rows, y = blocks of k
__global__ __launch_bounds__(256) void quantize8_rows_kernel(const uint16_t* __restrict__ x, uint8_t* __restrict__ x8, uint8_t* __restrict__ scale,
                                                             int M, int K) {
    const int lane = threadIdx.x & 15, kb = blockIdx.y;
    const int64_t r = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4);
    const int k = kb * kG8Block + 8 * lane;
    u32x4_t v = {};
    if (r < M && k < K) v = ldg16(x + r * K + k);
    uint32_t m = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) m = max(m, max(magnitude_bits(bf16_lo(v[e])), magnitude_bits(bf16_hi(v[e]))));
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        uint32_t a, b;
        lane_pair(t, m, a, b);
        m = max(a, b);
    }
    if (r >= M) return;
    const uint32_t byte = scale_byte(m);
    const float inv = scale_inverse(byte);
    u32x2_t o;
#pragma unroll
    for (int e = 0; e < 2; ++e)
        o[e] = pack_e4m3(bf16_lo(v[2 * e]) * inv, bf16_hi(v[2 * e]) * inv, bf16_lo(v[2 * e + 1]) * inv, bf16_hi(v[2 * e + 1]) * inv);
    *reinterpret_cast<u32x2_t*>(x8 + ((int64_t)(2 * kb + (lane >> 3)) * M + r) * kG8Slab + 8 * (lane & 7)) = o;
    if (lane == 0) scale[g8_scale_at(r, kb, gridDim.y)] = (uint8_t)byte;
}

// ------------------------------------------------------------------ product
struct Gemm8Params : GemmParams {  // A and W of the base unused; K a multiple of 128
    const uint8_t *A8, *W8;        // slabs
    const uint8_t *a_scale;        // g8_scale_at
    const uint8_t *w_scale;        // [ceil(N / 128)][K / 128]
};

// A wave-wide 4-byte-per-lane load from a buffer straight into LDS (as gemm_dma16).
__device__ __forceinline__ void gemm8_dma4(const gemm_i32x4_t& rsrc, unsigned voffset, unsigned lds) {
    unsigned saved;
    asm volatile(
        "s_mov_b32 %0, m0\n\t"
        "s_mov_b32 m0, %1\n\t"
        "s_nop 0\n\t"
        "buffer_load_dword %2, %3, 0 offen lds\n\t"
        "s_mov_b32 m0, %0"
        : "=&s"(saved)
        : "s"(lds), "v"(voffset), "s"(rsrc)
        : "memory");
}

// BM x BN tiles by WM x WN waves, k in stages of 64 (a slab) through a ring of S.  LDS rows are 64 bytes, chunk c of row r at
// c ^ ((r >> 2) & 3): the 16 rows that a quarter of a wave reads cover all 64 banks.  A stage also brings the scales of
// each wave's 128 rows (a word per lane); those of W's columns are in lanes from the start, one per 128 of k.
// While a stage multiplies, the next one's fragments are read and the loads of the one S behind go out between the MFMAs.
template <int BM, int BN, int WM, int WN, int S, int EPI>
__global__ __launch_bounds__(WM* WN * 64, 1) void gemm8_ring_kernel(Gemm8Params P) {
    constexpr int NW = WM * WN, RM = BM / WM, RN = BN / WN, MB = RM / 32, NB = RN / 32;
    constexpr int AB = BM * kG8Slab, WB = BN * kG8Slab, SB = AB + WB + NW * 256;  // bytes of A, W, a stage
    constexpr int LA = BM / 16 / NW, LW = BN / 16 / NW, LS = LA + LW + 1;       // wave-wide loads per wave and stage
    static_assert(BM % (16 * NW) == 0 && BN % (16 * NW) == 0, "whole wave loads");
    static_assert(RM % 32 == 0 && RN % 32 == 0 && (128 % RM == 0 || RM % 128 == 0) && RM <= 128 && 128 % RN == 0, "scales of a wave");
    static_assert((S - 2) * LS < 64, "vmcnt has 6 bits");
    constexpr int kLds = S * SB > BM * BN * 2 ? S * SB : BM * BN * 2;
    static_assert(kLds <= 160 * 1024, "LDS");
    __shared__ __attribute__((aligned(1024))) uint8_t lds[kLds];
    const int tid = threadIdx.x;
    const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    int m0, n0;
    gemm_tile_origin(P, BM, BN, m0, n0);
    const int M = P.M, N = P.N, K = P.K, blocks = K / kG8Block;
    const int kb0 = EPI == kEpiPartial ? (int)blockIdx.y * (P.k_split / kG8Block) : 0;  // this workgroup's blocks of k
    const int kb1 = EPI == kEpiPartial ? min(blocks, kb0 + P.k_split / kG8Block) : blocks;
    const unsigned lds0 = (unsigned)(size_t)((gemm_lds_void_t*)lds);
    const int wm = wave / WN, wn = wave % WN, r32 = lane & 31, h = lane >> 5;

    // 16 rows per load; slot chunk lane & 3 of a row holds chunk (lane & 3) ^ ((row >> 2) & 3)
    const unsigned off = (unsigned)((lane >> 2) * kG8Slab + 16 * ((lane & 3) ^ ((lane >> 4) & 3)));
    const uint8_t* a_ptr = P.A8 + ((int64_t)2 * kb0 * M + m0) * kG8Slab;
    const uint8_t* w_ptr = P.W8 + ((int64_t)2 * kb0 * N + n0) * kG8Slab;
    const unsigned a_rec = (unsigned)min(M - m0, BM) * kG8Slab, w_rec = (unsigned)min(N - n0, BN) * kG8Slab;
    const int group = (m0 + wm * RM) >> 7;  // the wave's 128 rows, which may lie behind the last
    const uint8_t* s_ptr = P.a_scale + ((int64_t)min(group, (M - 1) >> 7) * blocks + kb0) * 128;
    int l_k = 2 * kb0;       // the next slab to load
    unsigned l_dst = lds0;   // its LDS slot
    gemm_i32x4_t ars, wrs, srs;
    auto begin_stage = [&]() {
        const bool in = l_k < 2 * kb1;  // past the range: zeros, into slots that are not multiplied
        ars = gemm_descriptor(a_ptr, in ? a_rec : 0u);
        wrs = gemm_descriptor(w_ptr, in ? w_rec : 0u);
        srs = gemm_descriptor(s_ptr, in ? 128u : 0u);
    };
    auto load_one = [&](int i) {
        if (i < LA)
            gemm_dma16<false>(ars, off + 1024u * (unsigned)(wave * LA + i), l_dst + 1024u * (unsigned)(wave * LA + i));
        else if (i < LA + LW)
            gemm_dma16<false>(wrs, off + 1024u * (unsigned)(wave * LW + i - LA), l_dst + (unsigned)AB + 1024u * (unsigned)(wave * LW + i - LA));
        else
            gemm8_dma4(srs, 4u * (unsigned)r32, l_dst + (unsigned)(AB + WB) + 256u * (unsigned)wave);
    };
    auto end_stage = [&]() {
        a_ptr += (int64_t)M * kG8Slab;
        w_ptr += (int64_t)N * kG8Slab;
        s_ptr += (l_k & 1) != 0 ? 128 : 0;
        ++l_k;
        l_dst += SB;
        if (l_dst == lds0 + S * SB) l_dst = lds0;
    };

    // scale bytes of the wave's columns: block kb0 + 64 i + lane in byte i % 4 of word i / 4
    uint32_t w_scales[2] = {};
    {
        const int64_t nb = min(n0 + wn * RN, N - 1) >> 7;
        const int count = kb1 - kb0;
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (64 * i + lane < count) w_scales[i / 4] |= (uint32_t)P.w_scale[nb * blocks + kb0 + 64 * i + lane] << (8 * (i % 4));
    }
    int a_at[MB], b_at[NB];  // of chunk 2 h; chunk 2 h + 1 is at ^ 16
#pragma unroll
    for (int i = 0; i < MB; ++i) {
        const int r = wm * RM + 32 * i + r32;
        a_at[i] = r * kG8Slab + 16 * ((2 * h) ^ ((r >> 2) & 3));
    }
#pragma unroll
    for (int i = 0; i < NB; ++i) {
        const int r = wn * RN + 32 * i + r32;
        b_at[i] = AB + r * kG8Slab + 16 * ((2 * h) ^ ((r >> 2) & 3));
    }
    f32x16_t acc[MB][NB];
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j) acc[i][j] = f32x16_t{};
    i32x8_t af[2][MB], bf[2][NB];
    uint32_t as[2];
    const int shift = RM == 128 ? 0 : 8 * (((m0 + wm * RM) & 127) / 32);  // the wave's bytes of a scale word

    constexpr int FR = MB + NB + 1;
    auto read16 = [&](int at, const uint8_t* st) { return *reinterpret_cast<const u32x4_t*>(st + at); };
    auto read_frag = [&](auto set_tag, const uint8_t* st, int f) {
        constexpr int SET = decltype(set_tag)::value;
        if (f == 0) {
            as[SET] = *reinterpret_cast<const uint32_t*>(st + AB + WB + 256 * wave + 4 * lane) >> shift;
        } else if (f <= NB) {
            const int at = b_at[f >= 1 && f <= NB ? f - 1 : 0];
            bf[SET][f >= 1 && f <= NB ? f - 1 : 0] =
                __builtin_bit_cast(i32x8_t, __builtin_shufflevector(read16(at, st), read16(at ^ 16, st), 0, 1, 2, 3, 4, 5, 6, 7));
        } else {
            const int at = a_at[f > NB ? f - NB - 1 : 0];
            af[SET][f > NB ? f - NB - 1 : 0] =
                __builtin_bit_cast(i32x8_t, __builtin_shufflevector(read16(at, st), read16(at ^ 16, st), 0, 1, 2, 3, 4, 5, 6, 7));
        }
    };
    // MFMAs of a stage from set CUR; the next stage's fragments and this step's loads go between them
    auto multiply = [&](auto cur_tag, const uint8_t* nxt, int ws) {
        constexpr int CUR = decltype(cur_tag)::value;
        constexpr int NM = MB * NB;
#pragma unroll
        for (int i = 0; i < NM; ++i) {
            const int am = i / NB, bn = i % NB;
#define TRAJ_G8_MFMA(SEL) __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(af[CUR][am], bf[CUR][bn], acc[am][bn], 0, 0, SEL, (int)as[CUR], 0, ws)
            acc[am][bn] = am == 0 ? TRAJ_G8_MFMA(0) : am == 1 ? TRAJ_G8_MFMA(1) : am == 2 ? TRAJ_G8_MFMA(2) : TRAJ_G8_MFMA(3);
#undef TRAJ_G8_MFMA
#pragma unroll
            for (int f = FR * i / NM; f < FR * (i + 1) / NM; ++f) read_frag(std::integral_constant<int, CUR ^ 1>{}, nxt, f);
#pragma unroll
            for (int l = LS * i / NM; l < LS * (i + 1) / NM; ++l) load_one(l);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    auto meet = [&]() {  // the wave's fragment reads are done, its loads of the next stage have landed
        __builtin_amdgcn_s_waitcnt(wait_vmcnt_imm((S - 2) * LS) & ~0x0F00);
        ring_barrier();
    };
    using Z = std::integral_constant<int, 0>;
    using O = std::integral_constant<int, 1>;
#pragma unroll
    for (int i = 0; i < S - 1; ++i) {
        begin_stage();
#pragma unroll
        for (int l = 0; l < LS; ++l) load_one(l);
        end_stage();
    }
    meet();
#pragma unroll
    for (int f = 0; f < FR; ++f) read_frag(Z{}, lds, f);
    begin_stage();
#pragma unroll
    for (int l = 0; l < LS; ++l) load_one(l);
    end_stage();
    int slot = 0;  // being read
    auto next_slot = [&]() {
        slot = slot == S - 1 ? 0 : slot + 1;
        return lds + slot * SB;
    };
    for (int i = 0; i < kb1 - kb0; ++i) {
        const uint32_t word = i < 256 ? w_scales[0] : w_scales[1];
        const int ws = (int)((uint32_t)__builtin_amdgcn_readlane((int)word, i & 63) >> (8 * ((i >> 6) & 3)));
        meet();
        begin_stage();
        multiply(Z{}, next_slot(), ws);
        end_stage();
        meet();
        begin_stage();
        multiply(O{}, next_slot(), ws);
        end_stage();
    }
    __builtin_amdgcn_s_waitcnt(wait_vmcnt_imm(0) & ~0x0F00);  // the loads past the k range have landed too
    ring_barrier();
    if (EPI == kEpiPartial) {
        float* out = P.partial + (int64_t)blockIdx.y * M * N;
#pragma unroll
        for (int am = 0; am < MB; ++am)
#pragma unroll
            for (int bn = 0; bn < NB; ++bn) {
                const int col = n0 + wn * RN + bn * 32 + r32;
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int row = m0 + wm * RM + am * 32 + 8 * (e >> 2) + 4 * h + (e & 3);
                    if (row < M && col < N) out[(int64_t)row * N + col] = acc[am][bn][e];
                }
            }
        return;
    }
    gemm_epilogue<BM, BN, WM, WN, EPI>(P, acc, reinterpret_cast<uint16_t*>(lds), m0, n0);
}

}  // namespace trajspec
