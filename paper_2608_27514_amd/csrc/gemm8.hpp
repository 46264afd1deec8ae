// Matrix product with 8-bit operands (fp8.hpp): D[M,N] = A[M,K] W[K,N] (+ D).  W comes in e4m3 with a scale per block of
// 128 x 128, A in bf16 and is taken to e4m3 with a scale per row and 128 of k; fp32 accumulation on the matrix core, whose
// 8-bit products take both scales, one bf16 rounding of each result.
//   quantize8_kernel       W to 8 bits, once
//   quantize8_rows_kernel  A to 8 bits, into the workspace
//   gemm8_ring_kernel      the product
//   gemm8_rows_kernel      the product of few rows, A taken to 8 bits on the way where it is small
//
// Operands lie in slabs of 64 of k: [k / 64][row][k % 64], rows being rows of A and columns of W, and K padded with zeros
// to a multiple of 128.  So what a workgroup needs of a slab is contiguous, whole lines however few of k a stage holds, and
// both operands are k-contiguous: a fragment (32 of k of a row) is two 16-byte LDS reads, with no transposition.
#pragma once

#include "fp8.hpp"
#include "gemm.hpp"
#include "verify_attn16.hpp"

namespace trajspec {

constexpr int kG8Block = 128;  // of k (and of columns of W) per scale
constexpr int kG8Slab = 64;
constexpr int64_t kG8MaxK = 65536;

typedef int i32x8_t __attribute__((ext_vector_type(8)));

// ------------------------------------------------------------------ W
// A workgroup per 128 x 128 block: 4 x 8 values (4 of k, 8 columns) per thread and turn, whose bytes go through LDS, so that
// both sides move whole lines.  Bound by the copy: 4096 x 12288 (151 MB) 27 us in a row of calls = 5.6 TB/s, where a copy of
// as much moves 5.2; 1000 x 712 4.7 us, its latencies.
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

// 16 lanes per row and block of 128, 8 values each, kG8RowBlocks blocks per workgroup with their loads requested together.
// Bound by the copy: 4096 x 4096 11 us (50 MB, 9.8 at the copy's rate); 96 x 3584 3.2, a launch.
// grid: x = groups of 16 rows, y = groups of blocks of k
constexpr int kG8RowBlocks = 4;
__global__ __launch_bounds__(256) void quantize8_rows_kernel(const uint16_t* __restrict__ x, uint8_t* __restrict__ x8, uint8_t* __restrict__ scale,
                                                             int M, int K, int blocks) {
    const int lane = threadIdx.x & 15, kb0 = blockIdx.y * kG8RowBlocks;
    const int64_t r = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4);
    u32x4_t v[kG8RowBlocks];
#pragma unroll
    for (int i = 0; i < kG8RowBlocks; ++i) {
        const int k = (kb0 + i) * kG8Block + 8 * lane;
        v[i] = u32x4_t{};
        if (r < M && k < K) v[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(x + r * K + k));
    }
#pragma unroll
    for (int i = 0; i < kG8RowBlocks; ++i) {
        const int kb = kb0 + i;
        if (kb >= blocks) break;  // uniform
        const uint32_t word[4] = {v[i][0], v[i][1], v[i][2], v[i][3]};
        uint32_t m = magnitude_of(word);
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            uint32_t a, b;
            lane_pair(t, m, a, b);
            m = max(a, b);
        }
        const uint32_t byte = scale_byte(m);
        if (r >= M) continue;
        *reinterpret_cast<u32x2_t*>(x8 + ((int64_t)(2 * kb + (lane >> 3)) * M + r) * kG8Slab + 8 * (lane & 7)) =
            u32x2_t{pack_e4m3(word[0], word[1], scale_value(byte)), pack_e4m3(word[2], word[3], scale_value(byte))};
        if (lane == 0) scale[g8_scale_at(r, kb, blocks)] = (uint8_t)byte;
    }
}

// ------------------------------------------------------------------ product
struct Gemm8Params : GemmParams {  // K padded to a multiple of 128; W unused, A where the kernel takes it to 8 bits itself
    const uint8_t *A8, *W8;        // slabs
    const uint8_t *a_scale;        // g8_scale_at
    const uint8_t* w_scale;        // [ceil(N / 128)][K / 128]
    int k_rows;                    // K as A has it
};

// BM x BN tiles by WM x WN waves, k in stages of KS slabs through a ring of S.  LDS rows are 64 bytes, chunk c of row r at
// c ^ ((r >> 2) & 3): the 16 rows that a quarter of a wave reads cover all 64 banks.
// While a slab multiplies, the next one's fragments are read, and the loads of the stage S behind go out between the MFMAs.
// Where a wave has few MFMAs per slab, a stage holds two, which halves the meetings.
// What bounds it is the way from the L2 to LDS and the meetings, not the matrix core and not HBM: 4096 x 4096 x 12288, normal
// values, takes 164 us by itself = 2.5 PFLOP/s (8192 x 8192 x 8192 403 = 2.73), 117 with the loads left out (266), and 174 .. 181
// (446) behind quantize8_rows_kernel, whose 11 us (40) are in it.  With that kernel, rings of four stages of one slab 177 (476)
// and tiles of 256 x 128 205 (503); other cache policies change nothing.  Fewer rows run through their k at some
// 0.32 us per 128 at any depth of the ring: 96 x 3584 x 4608 14.8 us with a ring of 5 and 15.3 with one of 9, 14.1 in tiles
// of 32 x 64, which take 19.2 for 17.2 at 64 x 4096 x 12288.
// Scales: those of each wave's 128 rows come as a kilobyte for 8 blocks of k, into one of two places of the wave's own, a
// turn ahead; those of W's columns are in lanes from the start, one per block.
template <int BM, int BN, int WM, int WN, int KS, int S, int EPI>
__global__ __launch_bounds__(WM* WN * 64, 1) void gemm8_ring_kernel(Gemm8Params P) {
    constexpr int NW = WM * WN, RM = BM / WM, RN = BN / WN, MB = RM / 32, NB = RN / 32;
    constexpr int AB = BM * kG8Slab, WB = BN * kG8Slab, SB = KS * (AB + WB);    // bytes of a slab of A, of W, of a stage
    constexpr int LA = BM / 16 / NW, LW = BN / 16 / NW, LS = KS * (LA + LW);  // wave-wide loads per wave: of a slab, of a stage
    static_assert(BM % (16 * NW) == 0 && BN % (16 * NW) == 0, "whole wave loads");
    static_assert(RM % 32 == 0 && RN % 32 == 0 && 128 % RM == 0 && 128 % RN == 0, "scales of a wave");
    static_assert((S - 2) * LS < 64, "vmcnt has 6 bits");
    static_assert(KS == 1 || KS == 2, "a block of k is two slabs");
    constexpr int kScales = S * SB, kRing = kScales + NW * 2048;
    constexpr int kLds = kRing > BM * BN * 2 ? kRing : BM * BN * 2;
    static_assert(kLds <= 160 * 1024, "LDS");
    __shared__ __attribute__((aligned(1024))) uint8_t lds[kLds];
    const int tid = threadIdx.x;
    const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    int m0, n0;
    gemm_tile_origin(P, BM, BN, m0, n0);
    const int M = P.M, N = P.N, blocks = P.K / kG8Block;
    const int kb0 = EPI == kEpiPartial ? (int)blockIdx.y * (P.k_split / kG8Block) : 0;  // this workgroup's blocks of k
    const int count = (EPI == kEpiPartial ? min(blocks, kb0 + P.k_split / kG8Block) : blocks) - kb0;
    const unsigned lds0 = (unsigned)(size_t)((gemm_lds_void_t*)lds);
    const int wm = wave / WN, wn = wave % WN, r32 = lane & 31, h = lane >> 5;

    // 16 rows per load; slot chunk lane & 3 of a row holds chunk (lane & 3) ^ ((row >> 2) & 3)
    const unsigned off = (unsigned)((lane >> 2) * kG8Slab + 16 * ((lane & 3) ^ ((lane >> 4) & 3)));
    const uint8_t* a_ptr = P.A8 + ((int64_t)2 * kb0 * M + m0) * kG8Slab;
    const uint8_t* w_ptr = P.W8 + ((int64_t)2 * kb0 * N + n0) * kG8Slab;
    const unsigned a_rec = (unsigned)min(M - m0, BM) * kG8Slab, w_rec = (unsigned)min(N - n0, BN) * kG8Slab;
    int left = 2 * count;    // slabs to load
    unsigned l_dst = lds0;   // the next stage's LDS slot
    gemm_i32x4_t ars, wrs;
    auto begin_slab = [&]() {  // past the range: zeros, into slots that are not multiplied
        ars = gemm_descriptor(a_ptr, left > 0 ? a_rec : 0u);
        wrs = gemm_descriptor(w_ptr, left > 0 ? w_rec : 0u);
    };
    auto end_slab = [&]() {
        a_ptr += (int64_t)M * kG8Slab;
        w_ptr += (int64_t)N * kG8Slab;
        --left;
    };
    auto load_one = [&](int i) {  // load i of a stage
        const int s = i / (LA + LW), j = i % (LA + LW);
        if (j == 0) begin_slab();
        if (j < LA)
            gemm_dma16<false>(ars, off + 1024u * (unsigned)(wave * LA + j), l_dst + (unsigned)(s * AB) + 1024u * (unsigned)(wave * LA + j));
        else
            gemm_dma16<false>(wrs, off + 1024u * (unsigned)(wave * LW + j - LA),
                              l_dst + (unsigned)(KS * AB + s * WB) + 1024u * (unsigned)(wave * LW + j - LA));
        if (j == LA + LW - 1) end_slab();
    };
    auto end_stage = [&]() {
        l_dst += SB;
        if (l_dst == lds0 + S * SB) l_dst = lds0;
    };
    // scales of the wave's rows, which may lie behind the last, for the blocks from c on
    const uint8_t* s_ptr = P.a_scale + ((int64_t)min((m0 + wm * RM) >> 7, (M - 1) >> 7) * blocks + kb0) * 128;
    auto load_scales = [&](int c) {
        const gemm_i32x4_t rs = gemm_descriptor(s_ptr + 128 * c, c < count ? 128u * (unsigned)min(count - c, 8) : 0u);
        gemm_dma16<false>(rs, 16u * (unsigned)lane, lds0 + (unsigned)kScales + 2048u * (unsigned)wave + 1024u * (unsigned)((c >> 3) & 1));
    };

    // scale bytes of the wave's columns: block 64 i + lane in byte i % 4 of word i / 4
    uint32_t w_scales[2] = {};
    {
        const int64_t nb = min(n0 + wn * RN, N - 1) >> 7;
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
        b_at[i] = KS * AB + r * kG8Slab + 16 * ((2 * h) ^ ((r >> 2) & 3));
    }
    f32x16_t acc[MB][NB];
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j) acc[i][j] = f32x16_t{};
    i32x8_t af[2][MB], bf[2][NB];
    const int shift = RM == 128 ? 0 : 8 * (((m0 + wm * RM) & 127) / 32);  // the wave's bytes of a scale word
    const uint8_t* scales = lds + kScales + 2048 * wave + 4 * r32;

    constexpr int FR = MB + NB;
    auto read32 = [&](const uint8_t* st, int at) {
        return __builtin_bit_cast(i32x8_t, __builtin_shufflevector(*reinterpret_cast<const u32x4_t*>(st + at),
                                                                  *reinterpret_cast<const u32x4_t*>(st + (at ^ 16)), 0, 1, 2, 3, 4, 5, 6, 7));
    };
    // fragment f of slab s of the stage at st, into set SET; in the order of use: A block 0, the W blocks, the other A blocks
    auto read_frag = [&](auto set_tag, const uint8_t* st, int s, int f) {
        constexpr int SET = decltype(set_tag)::value;
        if (f >= 1 && f <= NB)
            bf[SET][f >= 1 && f <= NB ? f - 1 : 0] = read32(st + s * WB, b_at[f >= 1 && f <= NB ? f - 1 : 0]);
        else
            af[SET][f == 0 ? 0 : f - NB] = read32(st + s * AB, a_at[f == 0 ? 0 : f - NB]);
    };
    // MFMAs of a slab from set CUR; the fragments of slab s of the stage at st and loads of a stage from L0 on go between them
    auto multiply = [&](auto cur_tag, const uint8_t* st, int s, auto l0_tag, auto l1_tag, int as, int ws) {
        constexpr int CUR = decltype(cur_tag)::value, L0 = decltype(l0_tag)::value, NL = decltype(l1_tag)::value - L0;
        constexpr int NM = MB * NB;
#pragma unroll
        for (int i = 0; i < NM; ++i) {
            const int am = i / NB, bn = i % NB;
#define TRAJ_G8_MFMA(SEL) __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(af[CUR][am], bf[CUR][bn], acc[am][bn], 0, 0, SEL, as, 0, ws)
            acc[am][bn] = am == 0 ? TRAJ_G8_MFMA(0) : am == 1 ? TRAJ_G8_MFMA(1) : am == 2 ? TRAJ_G8_MFMA(2) : TRAJ_G8_MFMA(3);
#undef TRAJ_G8_MFMA
#pragma unroll
            for (int f = FR * i / NM; f < FR * (i + 1) / NM; ++f) read_frag(std::integral_constant<int, CUR ^ 1>{}, st, s, f);
#pragma unroll
            for (int l = NL * i / NM; l < NL * (i + 1) / NM; ++l) load_one(L0 + l);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    auto meet = [&]() {  // the wave's fragment reads are done, its loads of the next stage have landed
        __builtin_amdgcn_s_waitcnt(wait_vmcnt_imm((S - 2) * LS) & ~0x0F00);
        ring_barrier();
    };
    using Z = std::integral_constant<int, 0>;
    using O = std::integral_constant<int, 1>;
    using LEnd = std::integral_constant<int, LS>;
    load_scales(0);
#pragma unroll
    for (int i = 0; i < S - 1; ++i) {
#pragma unroll
        for (int l = 0; l < LS; ++l) load_one(l);
        end_stage();
    }
    meet();
#pragma unroll
    for (int f = 0; f < FR; ++f) read_frag(Z{}, lds, 0, f);
#pragma unroll
    for (int l = 0; l < LS; ++l) load_one(l);
    end_stage();
    int slot = 0;  // being read
    auto next_slot = [&]() {
        slot = slot == S - 1 ? 0 : slot + 1;
        return lds + slot * SB;
    };
    for (int i = 0; i < count; ++i) {
        const uint32_t word = i < 256 ? w_scales[0] : w_scales[1];
        const int ws = (int)((uint32_t)__builtin_amdgcn_readlane((int)word, i & 63) >> (8 * ((i >> 6) & 3)));
        const int as = (int)(*reinterpret_cast<const uint32_t*>(scales + 128 * (i & 15)) >> shift);
        if ((i & 7) == 0) load_scales(i + 8);  // read from two blocks on at the earliest: waits count it as one more of the ring's
        if constexpr (KS == 1) {
            meet();
            multiply(Z{}, next_slot(), 0, Z{}, LEnd{}, as, ws);
            end_stage();
            meet();
            multiply(O{}, next_slot(), 0, Z{}, LEnd{}, as, ws);
            end_stage();
        } else {
            multiply(Z{}, lds + slot * SB, 1, Z{}, Z{}, as, ws);
            meet();
            multiply(O{}, next_slot(), 0, Z{}, LEnd{}, as, ws);
            end_stage();
        }
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

// ---------------------------------------------------------------- few rows
// Up to 16 MR rows: the stream of W bounds the call, so nothing but W passes through memory at length.  A workgroup takes
// 16 NB columns, its waves the blocks of 128 of k in turn, DEPTH of them in flight; W's fragments (16 columns, 2 KB) come
// straight into registers, each load 1 KB in a row, and the waves' sums meet in LDS in the waves' order.
// The k order within a block is the same for both operands but not the memory's: lane l has 16 of each slab, from 16 (l / 16).
// LDSX 0: A comes in 8 bits from the workspace; otherwise (M K at most LDSX) every workgroup takes A to 8 bits itself, into LDS
// in the order of the fragments, while its first loads of W are on their way: one launch for the whole call.
//   MI355X: 1 x 4096 x 12288 (50 MB of W) 10.0 .. 10.7 us, where the read takes 8.1; with A taken to 8 bits first and
//   through the ring kernel 15.5.
template <int MR, int NB, int WAVES, int DEPTH, int LDSX, int EPI>
__global__ __launch_bounds__(WAVES * 64, WAVES == 16 ? 4 : 2) void gemm8_rows_kernel(Gemm8Params P) {
    constexpr bool X8 = LDSX == 0;
    constexpr int kSums = WAVES * NB * MR * 1024, kX = LDSX + LDSX / kG8Block;
    static_assert((kSums > kX ? kSums : kX) <= 160 * 1024, "LDS");
    __shared__ __attribute__((aligned(16))) uint8_t lds[kSums > kX ? kSums : kX];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int row = lane & 15, q = lane >> 4;
    const int n0 = (int)blockIdx.x * 16 * NB, M = P.M, N = P.N, blocks = P.K / kG8Block;
    u32x4_t w[DEPTH][NB][2], x[X8 ? DEPTH : 1][MR][2];
    uint32_t xs[X8 ? DEPTH : 1][MR], scales[NB];
    f32x4_t acc[NB][MR];
    // Blocks behind the last read nothing and count as 0.
    auto request = [&](auto slot, int kb) {
        constexpr int u = decltype(slot)::value;
        const bool in = kb < blocks;
        const int64_t at = in ? kb : 0;
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const auto rs = __builtin_amdgcn_make_buffer_rsrc((void*)(P.W8 + ((2 * at + s) * N + n0) * kG8Slab), (short)0,
                                                              in ? min(N - n0, 16 * NB) * kG8Slab : 0, kGemmBufferFlags);
#pragma unroll
            for (int j = 0; j < NB; ++j) w[u][j][s] = __builtin_amdgcn_raw_buffer_load_b128(rs, 1024 * j + kG8Slab * row + 16 * q, 0, 2);
        }
        if constexpr (X8) {
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                const auto rs = __builtin_amdgcn_make_buffer_rsrc((void*)(P.A8 + (2 * at + s) * M * kG8Slab), (short)0, in ? M * kG8Slab : 0,
                                                                  kGemmBufferFlags);
#pragma unroll
                for (int i = 0; i < MR; ++i) x[u][i][s] = __builtin_amdgcn_raw_buffer_load_b128(rs, 1024 * i + kG8Slab * row + 16 * q, 0, 0);
            }
#pragma unroll
            for (int i = 0; i < MR; ++i) xs[u][i] = P.a_scale[g8_scale_at(min(16 * i + row, M - 1), (int)at, blocks)];
        }
    };
    auto multiply = [&](auto slot, int t) {
        constexpr int u = decltype(slot)::value, ux = X8 ? u : 0;
        if constexpr (!X8) {
            const int kb = min(wave + WAVES * t, blocks - 1);
#pragma unroll
            for (int i = 0; i < MR; ++i) {
                const int m = min(16 * i + row, M - 1);
#pragma unroll
                for (int s = 0; s < 2; ++s) x[0][i][s] = *reinterpret_cast<const u32x4_t*>(lds + (((2 * kb + s) * 4 + q) * M + m) * 16);
                xs[0][i] = lds[P.K * M + kb * M + m];
            }
        }
#pragma unroll
        for (int j = 0; j < NB; ++j) {
            const int ws = __builtin_amdgcn_readlane((int)scales[j], t & 63);
            const i32x8_t wf = __builtin_bit_cast(i32x8_t, __builtin_shufflevector(w[u][j][0], w[u][j][1], 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
            for (int i = 0; i < MR; ++i) {
                const i32x8_t xf = __builtin_bit_cast(i32x8_t, __builtin_shufflevector(x[ux][i][0], x[ux][i][1], 0, 1, 2, 3, 4, 5, 6, 7));
                acc[j][i] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wf, xf, acc[j][i], 0, 0, 0, ws, 0, (int)xs[ux][i]);
            }
        }
    };
    const int turns = (blocks - wave + WAVES - 1) / WAVES;  // blocks of this wave
    auto each = [&](auto&& f) {  // f(slot) for every slot of the ring
        f(std::integral_constant<int, 0>{});
        if constexpr (DEPTH > 1) f(std::integral_constant<int, (DEPTH > 1 ? 1 : 0)>{});
        if constexpr (DEPTH > 2) f(std::integral_constant<int, (DEPTH > 2 ? 2 : 0)>{});
        if constexpr (DEPTH > 3) f(std::integral_constant<int, (DEPTH > 3 ? 3 : 0)>{});
    };
    each([&](auto slot) { request(slot, wave + WAVES * decltype(slot)::value); });
    // block wave + WAVES i of the scales of W's columns is in lane i
#pragma unroll
    for (int j = 0; j < NB; ++j) {
        const int64_t nb = min(n0 + 16 * j, N - 1) >> 7;
        scales[j] = wave + WAVES * lane < blocks ? P.w_scale[nb * blocks + wave + WAVES * lane] : kScaleOne;
#pragma unroll
        for (int i = 0; i < MR; ++i) acc[j][i] = f32x4_t{};
    }
    if constexpr (!X8) {
        // 16 lanes per row and block, 8 values each
        const int part = tid & 15;
        constexpr int STEP = WAVES * 4, U = 4;
        for (int at0 = tid >> 4; at0 < M * blocks; at0 += U * STEP) {
            u32x4_t v[U];
#pragma unroll
            for (int i = 0; i < U; ++i) {
                const int at = at0 + i * STEP, kb = at / M, m = at - kb * M, k = kb * kG8Block + 8 * part;
                v[i] = u32x4_t{};
                if (at < M * blocks && k < P.k_rows) v[i] = ldg16(P.A + (int64_t)m * P.k_rows + k);
            }
#pragma unroll
            for (int i = 0; i < U; ++i) {
                const int at = at0 + i * STEP, kb = at / M, m = at - kb * M;
                const uint32_t word[4] = {v[i][0], v[i][1], v[i][2], v[i][3]};
                uint32_t top = magnitude_of(word);
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    uint32_t a, b;
                    lane_pair(t, top, a, b);
                    top = max(a, b);
                }
                if (at >= M * blocks) break;
                const uint32_t byte = scale_byte(top);
                *reinterpret_cast<u32x2_t*>(lds + ((8 * kb + part / 2) * M + m) * 16 + 8 * (part & 1)) =
                    u32x2_t{pack_e4m3(word[0], word[1], scale_value(byte)), pack_e4m3(word[2], word[3], scale_value(byte))};
                if (part == 0) lds[P.K * M + kb * M + m] = (uint8_t)byte;
            }
        }
        __syncthreads();
    }
    for (int t = 0; t < turns; t += DEPTH)
        each([&](auto slot) {
            constexpr int u = decltype(slot)::value;
            multiply(slot, t + u);
            request(slot, wave + WAVES * (t + u + DEPTH));
        });
    if (!X8) __syncthreads();
    f32x4_t(*sums)[NB * MR][64] = reinterpret_cast<f32x4_t(*)[NB * MR][64]>(lds);
#pragma unroll
    for (int j = 0; j < NB; ++j)
#pragma unroll
        for (int i = 0; i < MR; ++i) sums[wave][j * MR + i][lane] = acc[j][i];
    __syncthreads();
    for (int at = tid; at < NB * MR * 64; at += WAVES * 64) {
        const int f = at >> 6, l = at & 63;
        f32x4_t v = sums[0][f][l];
#pragma unroll
        for (int s = 1; s < WAVES; ++s) v += sums[s][f][l];
        // the lane's result: row l % 16 of A, columns 4 (l / 16) .. + 4
        const int m = 16 * (f % MR) + (l & 15), n = n0 + 16 * (f / MR) + 4 * (l >> 4);
        if (m >= M || n >= N) continue;
        u32x2_t* dst = reinterpret_cast<u32x2_t*>(P.D + (int64_t)m * N + n);
        if (EPI == kEpiAccumulate) {
            const u32x2_t d = *dst;
            v += f32x4_t{bf16_lo(d[0]), bf16_hi(d[0]), bf16_lo(d[1]), bf16_hi(d[1])};
        }
        u32x2_t o;
#pragma unroll
        for (int e = 0; e < 2; ++e)
            o[e] = (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)v[2 * e]) | ((uint32_t)__builtin_bit_cast(uint16_t, (__bf16)v[2 * e + 1]) << 16);
        *dst = o;
    }
}

}  // namespace trajspec
