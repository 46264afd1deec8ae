// The paged key-value cache in 8 bits (fp8.hpp): pages of e4m3 values and, for keys and for values, a scale byte per
// block of `sb` tokens of a page and kv head, [num_pages][page_size / sb][Hkv].
//   paged8_append_kernel   rotates new tokens' queries and keys, takes keys and values to 8 bits
//   paged8_attn_kernel     attention over the cached keys, up to 32 rows per kv head
//   paged8_rows_kernel     more rows
// Ranges, row state, partial results and their join are the bf16 cache's (paged.hpp).
#pragma once

#include "fp8.hpp"
#include "paged.hpp"

namespace trajspec {

constexpr int kScaleTokens = 64;  // tokens of a scale at most

struct Paged8Cache {
    uint8_t *k, *v, *k_scale, *v_scale;
    int sb, blocks, Hkv;  // tokens of a scale, scales of a page and head
    FastDiv by_block;
};

// ------------------------------------------------------------------ append
struct Append8Params {
    const uint16_t *q, *k, *v;            // token rows of contiguous heads; q may be null
    int64_t q_row, k_row, v_row;          // elements from one token's row to the next
    uint16_t* q_out;                      // [B, T, Hq, D]
    PagedCache cache;                     // strides in values; k and v unused
    Paged8Cache c8;
    const int32_t *start, *n_new, *pos0;  // [B]; n_new null: T, pos0 null: start
    int T, Hq, Hkv, rotate;
    int tokens;                           // cache rows of a workgroup: whole blocks
    double turns[kAppendMaxHalf];         // rotation per position of pair d in turns: theta^(-2d/D) / 2 pi
    const int32_t* lens;                  // [B]; WITHIN: the sequences' tokens, those behind the call's among them
};

// A workgroup takes `tokens` cache rows (whole scale blocks) of a sequence, of which at most ROWS are the call's: their places
// and angles' sines and cosines go to LDS once, then each wave takes a head of q, K or V at a time, the next one's loads under
// way.  A lane holds 8 values of a row's first half and the matching 8 of its second, a wave all rows; a block's largest
// magnitude is found by lane exchanges and an LDS maximum per wave.  Rows that the first block held before are rounded
// again if the block's scale grows (rare: read only then).  WITHIN: so are the rows that its last block holds behind the
// call's (a kernel of its own, so that other calls pay nothing for it: one token 5.1 us for 4.6, 4 x 4096 62.9 for 62.4).
// Bound by the copy, (4 Hq + 6 Hkv) D bytes per token, and in small calls by a chain of loads, angles, rows and stores, where
// every workgroup that shares a group of rows computes all its angles and waits for them, also one of V heads alone.
//   MI355X: 4 x 4096 tokens, 28 over 4 heads of 128 62.1 us (289 MB, 55.9 at the copy's rate), blocks of 64 tokens 52.7 (8192
//   tokens, 32 over 8 heads, copy 36.2; with the rotated values kept and a head ahead 256 registers and 70.9); one token 4.7,
//   16 blocks of up to 32 tokens of 32 heads 7.7, 64 sequences' tokens 5.2.
// grid: x = groups of cache rows from the block that holds the first token, y shares the heads out, z = sequence.
template <int D, int ROWS, bool WITHIN>
__global__ __launch_bounds__(kAppendThreads) void paged8_append_kernel(Append8Params P) {
    constexpr int HALF = D / 2, LPR = D / 16, RPS = 64 / LPR, STEPS = ROWS / RPS, WAVES = kAppendThreads / 64;
    // Registers: long blocks keep their rows as loaded and rotate them twice, and request no head ahead.
    constexpr bool AHEAD = STEPS <= 4;
    static_assert(STEPS * RPS == ROWS && kAppendThreads % HALF == 0, "whole steps");
    __shared__ __align__(16) float cs[ROWS][HALF], sn[ROWS][HALF];
    __shared__ int64_t sh_row[ROWS];    // the row's place in the pools; -1: none
    __shared__ int64_t sh_scale[ROWS];  // of the row's block, head 0
    __shared__ uint32_t sh_max[WAVES][kScaleTokens];
    const int b = blockIdx.z, tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int start = P.start[b];
    int n = P.n_new != nullptr ? P.n_new[b] : P.T;
    const bool report = blockIdx.x == 0 && blockIdx.y == 0 && tid == 0;
    if (n < 0 || n > P.T) {
        if (report) flag_device_status(kDevBadLength);
        n = n < 0 ? 0 : P.T;
    }
    if (n == 0) return;
    if ((start < 0 || (int64_t)start + n > P.cache.capacity) && report) flag_device_status(kDevBadLength);
    int lead = start % P.c8.sb;  // rows of the first block before the call's tokens
    if (lead < 0) lead += P.c8.sb;
    const int t0 = max((int)blockIdx.x * P.tokens - lead, 0);  // the workgroup's first token of the call
    if (t0 >= n) return;
    lead = blockIdx.x == 0 ? lead : 0;
    const int rows = min(P.tokens - lead, n - t0);
    int behind = 0;  // rows behind the call's last token that its block holds
    const int last = WITHIN ? P.c8.by_block.div(lead + rows - 1) : 0;  // that block, where this is the last workgroup
    if constexpr (WITHIN) {
        int len = P.lens[b];
        if (len < 0 || len > P.cache.capacity) {
            if (report) flag_device_status(kDevBadLength);
            len = len < 0 ? 0 : P.cache.capacity;
        }
        const int64_t more = (int64_t)len - ((int64_t)start + n);
        if (t0 + rows == n && more > 0) behind = (int)min(more, (int64_t)((last + 1) * P.c8.sb - (lead + rows)));
    }
    const int qh = P.q != nullptr ? P.Hq : 0, units = qh + 2 * P.Hkv;
    const int row0 = lane / LPR, d0 = 8 * (lane % LPR);
    const int64_t token0 = (int64_t)b * P.T + t0;
    u32x4_t lo[STEPS], hi[STEPS];
    auto fetch = [&](int unit) {
        const bool query = unit < qh, key = unit < qh + P.Hkv;
        const int head = query ? unit : unit - qh - (key ? 0 : P.Hkv);
        const uint16_t* src = (query ? P.q : key ? P.k : P.v) + head * D + d0;
        const int64_t src_row = query ? P.q_row : key ? P.k_row : P.v_row;
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
            const int r = s * RPS + row0;
            lo[s] = hi[s] = u32x4_t{};
            if (r < rows) {
                const uint16_t* p = src + (token0 + r) * src_row;
                lo[s] = ldg16(p);
                hi[s] = ldg16(p + HALF);
            }
        }
    };
    const int unit0 = (int)blockIdx.y * WAVES + wave;
    if (AHEAD && unit0 < units) fetch(unit0);
    if (tid < rows) {
        const int64_t at = (int64_t)start + t0 + tid;
        int64_t row = -1, scale = 0;
        if (at >= 0 && at < P.cache.capacity) {
            const int col = P.cache.by_page.div((int)at), in = (int)at - col * P.cache.page_size;
            const int page = P.cache.table[b * P.cache.table_stride + col];
            if (page >= 0 && page < P.cache.num_pages) {
                row = page * P.cache.page_stride + in * P.cache.token_stride;
                scale = ((int64_t)page * P.c8.blocks + P.c8.by_block.div(in)) * P.Hkv;
            } else if (blockIdx.y == 0) {
                flag_device_status(kDevBadPage);
            }
        }
        sh_row[tid] = row;
        sh_scale[tid] = scale;
    }
    if (P.rotate) {
        const int64_t pos0 = (int64_t)(P.pos0 != nullptr ? P.pos0[b] : start) + t0;
        const int d = tid % HALF;
        const double per = P.turns[d];
        for (int r = tid / HALF; r < rows; r += kAppendThreads / HALF) {
            double turn = (double)(pos0 + r) * per;
            turn -= rint(turn);
            // 32 bits hold it to 2^-25, 0.2 millionths of a radian, which would show where a key lies next to the middle
            // between two codes: what they leave is added to the angle to first order
            const float near = (float)turn, rest = (float)(turn - near) * 6.2831853f;
            float s, c;
            sincospif(2.0f * near, &s, &c);
            sn[r][d] = s + c * rest;
            cs[r][d] = c - s * rest;
        }
    }
    __syncthreads();
    for (int unit = unit0; unit < units; unit += (int)gridDim.y * WAVES) {
        if (!AHEAD) fetch(unit);
        const bool query = unit < qh, key = unit < qh + P.Hkv;
        const int head = query ? unit : unit - qh - (key ? 0 : P.Hkv);
        // the scales of the first and the last block where they hold rows that stay
        uint8_t* scales = (key ? P.c8.k_scale : P.c8.v_scale) + head;
        auto scale_of = [&](int r) { return min(max((uint32_t)scales[sh_scale[r]], kScaleLowest), kScaleHighest); };
        const bool kept = !query && lead > 0 && sh_row[0] >= 0;
        const uint32_t old = kept ? scale_of(0) : 0u;
        const bool kept_behind = WITHIN && !query && behind > 0 && sh_row[rows - 1] >= 0;
        const uint32_t old_behind = kept_behind ? scale_of(rows - 1) : 0u;
        auto rotated = [&](int s, float(&v)[16]) {  // the lane's values of step s
            const int r = s * RPS + row0;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                v[e] = e % 2 == 0 ? bf16_lo(lo[s][e / 2]) : bf16_hi(lo[s][e / 2]);
                v[8 + e] = e % 2 == 0 ? bf16_lo(hi[s][e / 2]) : bf16_hi(hi[s][e / 2]);
            }
            if (P.rotate && key) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float a = v[e], c = v[8 + e], co = cs[r][d0 + e], si = sn[r][d0 + e];
                    v[e] = a * co - c * si;
                    v[8 + e] = c * co + a * si;
                }
            }
        };
        float x[AHEAD ? STEPS : 1][16];
#pragma unroll
        for (int s = 0; s < (AHEAD ? STEPS : 0); ++s) {
            if (s * RPS >= rows) break;  // uniform
            rotated(s, x[AHEAD ? s : 0]);
        }
        const int next = unit + (int)gridDim.y * WAVES;
        if (AHEAD && next < units) fetch(next);
        if (query) {
#pragma unroll
            for (int s = 0; s < STEPS; ++s) {
                const int r = s * RPS + row0;
                if (r >= rows) continue;
                float(&v)[16] = x[AHEAD ? s : 0];
                if (!AHEAD) rotated(s, v);
                u32x4_t o[2];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const f32x2_t pair = {v[2 * e], v[2 * e + 1]};
                    o[e / 4][e % 4] = __builtin_bit_cast(uint32_t, __builtin_convertvector(pair, bf16x2_t));
                }
                uint16_t* dst = P.q_out + ((token0 + r) * P.Hq + head) * D + d0;
                *reinterpret_cast<u32x4_t*>(dst) = o[0];
                *reinterpret_cast<u32x4_t*>(dst + HALF) = o[1];
            }
            continue;
        }
        uint32_t* most = sh_max[wave];
        most[lane] = 0u;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
            if (s * RPS >= rows) break;
            const int r = s * RPS + row0;
            float(&v)[16] = x[AHEAD ? s : 0];
            if (!AHEAD) rotated(s, v);
            uint32_t m = 0u;
#pragma unroll
            for (int e = 0; e < 16; ++e) m = max(m, magnitude_bits(v[e]));
#pragma unroll
            for (int t = 0; t < (LPR == 8 ? 3 : 2); ++t) m = max(m, (uint32_t)__shfl_xor((int)m, 1 << t));
            if (lane % LPR == 0 && r < rows) atomicMax(&most[P.c8.by_block.div(lead + r)], m);
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        uint8_t* pool = (key ? P.c8.k : P.c8.v) + head * P.cache.head_stride + d0;
        // the two are the same block where the call lies in one
        const uint32_t first_byte = max(scale_byte(most[0]), WITHIN && last == 0 ? max(old, old_behind) : old);
        const uint32_t last_byte = last == 0 ? first_byte : max(scale_byte(most[last]), old_behind);
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
            const int r = s * RPS + row0;
            if (r >= rows || sh_row[r] < 0) continue;
            const int block = P.c8.by_block.div(lead + r);
            const uint32_t byte = block == 0 ? first_byte : WITHIN && block == last ? last_byte : scale_byte(most[block]);
            const float inv = scale_inverse(byte);
            float(&v)[16] = x[AHEAD ? s : 0];
            if (!AHEAD) rotated(s, v);
            u32x2_t a, c;
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                a[e] = pack_e4m3(v[4 * e] * inv, v[4 * e + 1] * inv, v[4 * e + 2] * inv, v[4 * e + 3] * inv);
                c[e] = pack_e4m3(v[8 + 4 * e] * inv, v[9 + 4 * e] * inv, v[10 + 4 * e] * inv, v[11 + 4 * e] * inv);
            }
            uint8_t* dst = pool + sh_row[r];
            *reinterpret_cast<u32x2_t*>(dst) = a;
            *reinterpret_cast<u32x2_t*>(dst + HALF) = c;
            if (lane % LPR == 0 && r == max(0, block * P.c8.sb - lead)) scales[sh_scale[r]] = (uint8_t)byte;
        }
        // rows that stay, those before `end`: by 2^(was - byte), exact but for what falls into the subnormals, or below them
        auto move = [&](uint8_t* end, int count, uint32_t was, uint32_t byte) {
            const float down = byte - was < kScaleOne ? scale_value(kScaleOne - (byte - was)) : 0.f;
            for (int r = row0; r < count; r += RPS) {
                uint8_t* dst = end - (int64_t)(count - r) * P.cache.token_stride;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    u32x2_t a = *reinterpret_cast<const u32x2_t*>(dst + h * HALF);
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const auto p = __builtin_amdgcn_cvt_pk_f32_fp8((int)a[e], false), o = __builtin_amdgcn_cvt_pk_f32_fp8((int)a[e], true);
                        a[e] = pack_e4m3(p[0] * down, p[1] * down, o[0] * down, o[1] * down);
                    }
                    *reinterpret_cast<u32x2_t*>(dst + h * HALF) = a;
                }
            }
        };
        if (kept && first_byte > old) move(pool + sh_row[0], lead, old, first_byte);
        if (kept_behind && last_byte > old_behind)
            move(pool + sh_row[rows - 1] + (behind + 1) * P.cache.token_stride, behind, old_behind, last_byte);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
}

// ------------------------------------------------------------------ attention
// Up to 16 rows chunks make twice the bf16 cache's workgroups: two or three fit a CU, and half the bytes take half as long
// (4 x 16384 keys x 8 heads 25.2 -> 22.4 us, 2 x 16384 x 16 heads of 64 24.3 -> 20.6; 768 24.0 and 21.2).  More rows leave
// more partial results behind each (32 rows: 15.5 us, 17.8 with 512; blocks of 32 tokens 29.9 and 32.3).
constexpr int kPaged8FillWgs = 512;
constexpr int kPaged8FillRows = 16;

struct Paged8AttnParams : PagedAttnParams {
    Paged8Cache c8;
};

// paged_place, but where a head's row of a token is half a line two heads follow each other on an XCD, whose L2 then has the
// other half (16384 and 10323 keys of 16 heads of 64, [page, token, head] pools: 22.8 us with the heads on XCDs of their own).
template <int D>
__device__ __forceinline__ PagedPlace paged8_place(const PagedAttnParams& P) {
    if (D == 128 || P.Hkv % 2 != 0) return paged_place(P);
    PagedPlace w;
    const int turn = blockIdx.x / 8 / P.tiles, pair = turn / 2 * 8 + blockIdx.x % 8;  // of two heads
    w.row_tile = blockIdx.x / 8 - turn * P.tiles;
    w.slot = pair / (P.Hkv / 2);
    w.g = 2 * (pair - w.slot * (P.Hkv / 2)) + (turn & 1);
    w.unit = w.g * P.tiles + w.row_tile;
    return w;
}

// Where 16 BLK keys lie, as PagedTile, and their scales: lane l has those of key l % (16 BLK).
template <bool UNIFORM, int BLK>
struct Paged8Tile {
    int64_t at[UNIFORM ? BLK : 1];
    uint64_t vis;
    uint32_t ks, vs;
};

template <bool UNIFORM, int BLK>
__device__ __forceinline__ Paged8Tile<UNIFORM, BLK> paged8_tile(const Paged8AttnParams& P, const PagedPages<UNIFORM, BLK>& p, int g, int key0,
                                                                int first, int end, bool& bad) {
    const PagedCache& C = P.cache;
    constexpr int KEYS = 16 * BLK;
    constexpr uint64_t kAll = KEYS == 64 ? ~0ull : (1ull << (KEYS & 63)) - 1ull;
    const int64_t head = g * C.head_stride;
    const int mine = threadIdx.x & (KEYS - 1);
    Paged8Tile<UNIFORM, BLK> t;
    t.vis = 0;
    int64_t block = 0;  // of this lane's key
#pragma unroll
    for (int j = 0; j < (UNIFORM ? BLK : 1); ++j) {
        const int key = UNIFORM ? key0 + 16 * j : key0 + mine;
        const int at = key < end ? key : first;
        const bool good = p.page[j] >= 0 && p.page[j] < C.num_pages;
        bad |= !good && key < end;
        const int page = good ? p.page[j] : 0, in = at - C.by_page.div(at) * C.page_size;
        t.at[j] = page * C.page_stride + in * C.token_stride + head;
        if constexpr (UNIFORM) {
            const int n = key < end && good ? (end - key < 16 ? end - key : 16) : 0;
            t.vis |= (uint64_t)((1u << n) - 1u) << (16 * j);
            t.at[j] = uniform64(t.at[j]);
            if (j == 0 || mine / 16 == j) block = (int64_t)page * P.c8.blocks + P.c8.by_block.div(in - in % 16 + mine % 16);
        } else {
            t.vis = ballot64(good && key < end) & kAll;
            block = (int64_t)page * P.c8.blocks + P.c8.by_block.div(in);
        }
    }
    block = block * P.c8.Hkv + g;
    t.ks = P.c8.k_scale[block];
    t.vs = P.c8.v_scale[block];
    return t;
}

// What a lane multiplies its key's values by: 1 for an invisible one, whose scale may be anything.
__device__ __forceinline__ uint32_t paged8_scale(uint32_t byte, uint64_t vis, int key) {
    return ((vis >> key) & 1ull) != 0ull ? byte : kScaleOne;
}

// A tile's rows of K or V: a wave-wide load takes 1024 / D rows.  UNIFORM: buffers of the visible rows, so that rows
// behind them read as 0.
template <int D, bool UNIFORM, int BLK, bool ONCE>
__device__ __forceinline__ void paged8_load(u32x4_t (&x)[BLK * D / 64], const uint8_t* pool, const Paged8Tile<UNIFORM, BLK>& t, int token_stride) {
    constexpr int RPI = 1024 / D;
    const int lane = threadIdx.x & 63, vrow = lane / (D / 16), vchunk = lane % (D / 16);
#pragma unroll
    for (int i = 0; i < BLK * D / 64; ++i) {
        if constexpr (UNIFORM) {
            const int j = i * RPI / 16, rows = __popc((uint32_t)(t.vis >> (16 * j)) & 0xffffu);
            const auto rs = __builtin_amdgcn_make_buffer_rsrc((void*)(pool + t.at[j]), (short)0, rows * token_stride, kBufferFlags);
            x[i] = __builtin_amdgcn_raw_buffer_load_b128(rs, ((i * RPI) % 16 + vrow) * token_stride + 16 * vchunk, 0, ONCE ? 2 : 0);
        } else {
            const u32x4_t* p = reinterpret_cast<const u32x4_t*>(pool + __shfl(t.at[0], i * RPI + vrow) + 16 * vchunk);
            x[i] = ONCE ? __builtin_nontemporal_load(p) : *p;
        }
    }
}

// Loaded rows to LDS as bf16, times their scales (lane l of `scale` has key l's, that of an invisible one being 1).  Rows that
// are not in vis may hold anything and count as 0; those of a buffer (UNIFORM) read as 0 anyway.
template <int D, bool UNIFORM, int BLK, int ROW>
__device__ __forceinline__ void paged8_put(uint16_t* to, const u32x4_t (&x)[BLK * D / 64], uint64_t vis, uint32_t scale) {
    constexpr int RPI = 1024 / D;
    const int lane = threadIdx.x & 63, vrow = lane / (D / 16), vchunk = lane % (D / 16);
#pragma unroll
    for (int i = 0; i < BLK * D / 64; ++i) {
        const int row = i * RPI + vrow;
        u32x4_t v = x[i], lo, hi;
        if (!UNIFORM) v = ((vis >> row) & 1ull) != 0ull ? v : u32x4_t{};
        unpack_e4m3(v, scale_value((uint32_t)__shfl((int)scale, row)), lo, hi);
        uint16_t* p = to + row * ROW + 16 * vchunk;
        *reinterpret_cast<u32x4_t*>(p) = lo;
        *reinterpret_cast<u32x4_t*>(p + 8) = hi;
    }
}

// PagedRows::weights with the first operand cut to 16 bits rather than rounded, a pair in one instruction: the second one takes
// what is left, so that the product has the weights to 2^-16.
template <int D, int NR, int NK, bool PAIRED>
__device__ __forceinline__ void paged8_weights(PagedRows<D, NR, PAIRED>& st, const f32x4_t (&s)[NR][2 * NK], float c, bf16x8_t (&pf)[2][NR][NK]) {
#pragma unroll
    for (int f = 0; f < NR; ++f) {
        float mx = s[f][0][0];
#pragma unroll
        for (int v = 1; v < 8 * NK; ++v) mx = __builtin_elementwise_maximum(mx, s[f][v >> 2][v & 3]);
        st.raise(f, quad_max(mx), c);
        u32x4_t first[NK], rest[NK];
#pragma unroll
        for (int v = 0; v < 8 * NK; v += 2) {
            const float a = fast_exp2(__builtin_fmaf(s[f][v >> 2][v & 3], c, st.neg_mc[f]));
            const float b = fast_exp2(__builtin_fmaf(s[f][v >> 2][(v & 3) + 1], c, st.neg_mc[f]));
            st.lsum[f] += a;
            st.lsum[f] += b;
            const uint32_t ua = __builtin_bit_cast(uint32_t, a), ub = __builtin_bit_cast(uint32_t, b);
            first[v / 8][v % 8 / 2] = __builtin_amdgcn_perm(ub, ua, 0x07060302u);
            const bf16x2_t left = {(__bf16)(a - __builtin_bit_cast(float, ua & 0xffff0000u)), (__bf16)(b - __builtin_bit_cast(float, ub & 0xffff0000u))};
            rest[v / 8][v % 8 / 2] = __builtin_bit_cast(uint32_t, left);
        }
#pragma unroll
        for (int i = 0; i < NK; ++i) {
            pf[0][f][i] = __builtin_bit_cast(bf16x8_t, first[i]);
            pf[1][f][i] = __builtin_bit_cast(bf16x8_t, rest[i]);
        }
    }
}

// Up to 32 rows: the waves take the range's 32-key tiles in turn, the next one in flight.  K passes through LDS as it was
// loaded, in whole lines where the matrix core wants 16 values of each of 16 rows, and becomes bf16 on the way to the matrix
// core; V becomes bf16 before LDS, whose transposing reads take 16-bit values, while the scores are multiplied.
//   MI355X, one token a sequence, K from memory in the operand's order (no LDS) / as bf16 through LDS / as here: 32
//   sequences of up to 8192 keys x 32 heads of 128 222 / 213 / 210 us, 65536 keys x 8 heads 30.5 / 34.7 / 31.1, 4 x 16384
//   24.0 / 28.8 / 25.6; with two or three tiles in flight no faster (210.9, 33.3, 27.4), as 12 waves a CU hold enough loads.
template <int D, int NR, bool UNIFORM>
__global__ __launch_bounds__(kPagedThreads, 2) void paged8_attn_kernel(Paged8AttnParams P) {
    using L = PagedLds<D>;
    constexpr int ROWS = 16 * NR, BLK = 2, NVL = BLK * D / 64, RPI = 1024 / D;
    constexpr int kTileBytes = kPagedTile * L::kVRow * 2, kMergeBytes = ROWS * L::kMergeRow * 4;
    constexpr int kTiles = kPagedWaves * kTileBytes, kMerge = kPagedWaves * kMergeBytes;
    constexpr int kRow8 = D + 16;  // LDS bytes per row of K: the 16 rows of a fragment read start 4 banks apart
    __shared__ __align__(16) char lds[kTiles > kMerge ? kTiles : kMerge];
    __shared__ float sh_m[kPagedWaves * ROWS], sh_l[kPagedWaves * ROWS];

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const PagedPlace w = paged8_place<D>(P);
    PagedRange r;
    if (!paged_range<ROWS <= kPaged8FillRows ? kPaged8FillWgs : kPagedFillWgs>(P, w, r)) return;
    const int len = r.len;
    const int begin = r.split * r.chunk, end = len - begin > r.chunk ? begin + r.chunk : len;
    const int n_new = paged_new(P, r.b, w.unit == 0 && r.split == 0 && threadIdx.x == 0);
    const int min_limit = P.causal ? len - n_new + 1 : len;  // of a row that is not padding

    uint16_t* tile = reinterpret_cast<uint16_t*>(lds + wave * kTileBytes);  // K's and then V's
    uint8_t* kwrite = reinterpret_cast<uint8_t*>(tile) + lane / (D / 16) * kRow8 + 16 * (lane % (D / 16));
    const uint8_t* kread = reinterpret_cast<const uint8_t*>(tile) + (lane & 15) * kRow8 + 16 * (lane >> 4);
    const PagedCache& C = P.cache;
    const int ts = (int)C.token_stride;
    const int32_t* row = C.table + r.b * C.table_stride;
    const float c = P.scale_log2;
    const int first = begin + wave * kPagedTile;
    u32x4_t kr[NVL], vr[NVL];
    uint32_t vis = 0, ks = 0, vs = 0;
    bool bad = false;
    PagedRows<D, NR, true> st;
    PagedPages<UNIFORM, BLK> pages;  // of the tile to load next
    auto fetch = [&](int key0) { pages = paged_pages<UNIFORM, BLK>(C, row, key0, first, end); };
    auto load = [&](int key0) {
        const Paged8Tile<UNIFORM, BLK> t = paged8_tile<UNIFORM, BLK>(P, pages, w.g, key0, first, end, bad);
        paged8_load<D, UNIFORM, BLK, true>(kr, P.c8.k, t, ts);
        paged8_load<D, UNIFORM, BLK, true>(vr, P.c8.v, t, ts);
        vis = (uint32_t)t.vis;
        ks = t.ks;
        vs = t.vs;
    };
    // The tile at key0; with `more` also the loads of the next one.
    auto step = [&](int key0, bool more) {
#pragma unroll
        for (int i = 0; i < NVL; ++i) *reinterpret_cast<u32x4_t*>(kwrite + i * RPI * kRow8) = kr[i];
        u32x4_t k[BLK][D / 64];
#pragma unroll
        for (int j = 0; j < BLK; ++j)
#pragma unroll
            for (int i = 0; i < D / 64; ++i) k[j][i] = *reinterpret_cast<const u32x4_t*>(kread + 16 * j * kRow8 + 64 * i);
        // The scale of the row that the lane has of each block (an invisible row's score is replaced, so its scale may be
        // anything).  Lanes have a block's by rows of 16, which are exchanged in pairs.
        uint32_t scale[BLK];
        lane_pair(4, ks, scale[0], scale[1]);
        f32x4_t s[NR][BLK];
#pragma unroll
        for (int j = 0; j < BLK; ++j) {
#pragma unroll
            for (int f = 0; f < NR; ++f) s[f][j] = f32x4_t{};
#pragma unroll
            for (int i = 0; i < D / 64; ++i) {
                u32x4_t half[2];
                unpack_e4m3(k[j][i], scale_value(scale[j]), half[0], half[1]);
#pragma unroll
                for (int e = 0; e < 2; ++e)
#pragma unroll
                    for (int f = 0; f < NR; ++f)
                        s[f][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, half[e]), st.qf[f][2 * i + e], s[f][j], 0, 0, 0);
            }
        }
        const uint32_t seen = vis;
        paged8_put<D, UNIFORM, BLK, L::kVRow>(tile, vr, seen, paged8_scale(vs, seen, lane & 31));
        if (more) {
            load(key0 + kPagedGranule);
            fetch(key0 + 2 * kPagedGranule);
        }
        if (seen != ~0u || key0 + kPagedTile > min_limit) st.template mask<1>(s, seen, key0);  // rare: a sequence's last tile
        bf16x8_t pf[2][NR][1];
        paged8_weights<D, NR, 1>(st, s, c, pf);
        __builtin_amdgcn_sched_barrier(0);  // the next tile's products stay behind this one's: registers
        st.template values<1>(tile, pf);
        __builtin_amdgcn_sched_barrier(0);
    };
    if (first < end) fetch(first);
    st.init(P, r.b, w.g, len, n_new, w.row_tile * ROWS);
    if (first < end) {
        load(first);
        fetch(first + kPagedGranule);
        int key0 = first;
        for (; end - key0 > kPagedGranule; key0 += kPagedGranule) step(key0, true);
        step(key0, false);
        if (ballot64(bad) != 0ull && lane == 0) flag_device_status(kDevBadPage);
    }

    __syncthreads();
    float* buf = reinterpret_cast<float*>(lds);
    st.leave(buf + wave * ROWS * L::kMergeRow, sh_m + wave * ROWS, sh_l + wave * ROWS);
    __syncthreads();
    paged_store<D, ROWS, kPagedWaves>(P, r, w, n_new, buf, sh_m, sh_l);
}

// More rows: RW waves of 32 rows each share the stages of 16 RW keys that they load into LDS together, as bf16 (the stage is
// read once per 32 rows, taken from 8 bits once); 4 / RW such groups of waves take the range's stages in turn.  While a stage
// is multiplied the next one lies in registers on its way to the other buffer.
// A long call is bound by the products and the vector instructions beside them (4 x 512 tokens, 32 over 8 heads, 4096 keys:
// 251 us = 0.82 PFLOP/s with both parts of the weights); a short one by the latency of one wave a SIMD: 2.2 us a stage (2.5
// the first) and 4.2 before it (the range from the lengths 1.3, queries 1.5, the first stage's loads 1.4).  With a stamp
// behind every part, which costs a third more, a stage is scores 0.45, weights 0.8, values 0.75, to LDS 0.35, next loads 0.25,
// what is visible 0.2.  The states go to memory from the registers, 64 bytes of a row at once, in 1.9 us; in whole rows,
// through LDS, 4 us.
//   MI355X: 8 blocks of 32 tokens, 28 over 4 heads, up to 2048 keys 28.1 us (30.1 through LDS and with rounded weights); a
//   block over 4096 keys, 32 over 8 heads, 17.8 (19.1).  Workgroups of eight waves, two ranges of keys each: 28.0 and 19.3,
//   8 x 4096 keys 43.0 for 46.4, but 64 rows of 256 keys 13.3 for 12.3 and of 4096 51.7 .. 64 for 54.  Pages of bf16 take
//   as long (27.4, 19.0, 46.5) and the long call 233: here the 8 bits save memory, not time.
template <int D, int RW, bool UNIFORM, bool ONCE>
__global__ __launch_bounds__(kPagedThreads, 2) void paged8_rows_kernel(Paged8AttnParams P) {
    using L = PagedLds<D>;
    constexpr int NR = 2, KW = kPagedWaves / RW, ROWS = 32 * RW, STAGE = 16 * RW, NK = STAGE / 32, NVL = D / 64;
    constexpr int kStage = STAGE * (L::kKRow + L::kVRow);  // elements
    constexpr int kStages = KW * 2 * kStage * 2, kMerge = (KW - 1) * ROWS * L::kMergeRow * 4;
    __shared__ __align__(16) char lds[kStages > kMerge ? kStages : kMerge];
    __shared__ float sh_m[KW > 1 ? (KW - 1) * ROWS : 1], sh_l[KW > 1 ? (KW - 1) * ROWS : 1];
    __shared__ uint32_t sh_vis[KW][2][RW];

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int kg = wave / RW, rw = wave % RW;
    const PagedPlace w = paged8_place<D>(P);
    PagedRange r;
    if (!paged_range(P, w, r)) return;
    const int len = r.len;
    const int begin = r.split * r.chunk, end = len - begin > r.chunk ? begin + r.chunk : len;
    const int n_new = paged_new(P, r.b, w.unit == 0 && r.split == 0 && threadIdx.x == 0);
    const int min_limit = P.causal ? len - n_new + 1 : len;  // of a row that is not padding

    uint16_t* stage = reinterpret_cast<uint16_t*>(lds) + kg * 2 * kStage;  // two of them, K rows then V rows
    const PagedCache& C = P.cache;
    const int ts = (int)C.token_stride;
    const int32_t* row = C.table + r.b * C.table_stride;
    const float c = P.scale_log2;
    u32x4_t kr[NVL], vr[NVL];  // this wave's 16 keys of the next stage
    uint64_t vis = 0;
    uint32_t ks = 0, vs = 0;
    bool bad = false;
    const int rounds = (end - begin + KW * STAGE - 1) / (KW * STAGE);
    auto stage_key = [&](int n) { return begin + (n * KW + kg) * STAGE; };
    PagedPages<UNIFORM, 1> pages;
    auto fetch = [&](int n) { pages = paged_pages<UNIFORM, 1>(C, row, stage_key(n) + 16 * rw, begin, end); };
    auto request = [&](int n) {
        const Paged8Tile<UNIFORM, 1> t = paged8_tile<UNIFORM, 1>(P, pages, w.g, stage_key(n) + 16 * rw, begin, end, bad);
        fetch(n + 1);
        paged8_load<D, UNIFORM, 1, ONCE>(kr, P.c8.k, t, ts);
        paged8_load<D, UNIFORM, 1, ONCE>(vr, P.c8.v, t, ts);
        vis = t.vis;
        ks = t.ks;
        vs = t.vs;
    };
    auto put = [&](int n) {
        uint16_t* k = stage + (n & 1) * kStage;
        paged8_put<D, UNIFORM, 1, L::kKRow>(k + 16 * rw * L::kKRow, kr, vis, paged8_scale(ks, vis, lane & 15));
        paged8_put<D, UNIFORM, 1, L::kVRow>(k + STAGE * L::kKRow + 16 * rw * L::kVRow, vr, vis, paged8_scale(vs, vis, lane & 15));
        if (lane == 0) sh_vis[kg][n & 1][rw] = (uint32_t)vis;
    };
    PagedRows<D, NR> st;
    if (rounds > 0) fetch(0);
    st.init(P, r.b, w.g, len, n_new, w.row_tile * ROWS + 32 * rw);
    if (rounds > 0) {
        request(0);
        put(0);
        request(1);  // past the end: the range's first row, not visible
        __syncthreads();
        for (int n = 0; n < rounds; ++n) {
            const uint16_t* k = stage + (n & 1) * kStage;
            uint32_t seen[NK];
#pragma unroll
            for (int i = 0; i < NK; ++i)
                seen[i] = __builtin_amdgcn_readfirstlane(sh_vis[kg][n & 1][2 * i] | sh_vis[kg][n & 1][2 * i + 1] << 16);
            put(n + 1);
            request(n + 2);
            f32x4_t s[NR][2 * NK];
            st.template scores<NK>(k, s);
            const uint64_t all = NK == 1 ? seen[0] : seen[0] | (uint64_t)seen[NK - 1] << 32;
            const int key0 = stage_key(n);
            if (all != (NK == 1 ? 0xffffffffull : ~0ull) || key0 + STAGE > min_limit) st.template mask<NK>(s, all, key0);
            bf16x8_t pf[2][NR][NK];
            paged8_weights<D, NR, NK>(st, s, c, pf);
            st.template values<NK>(k + STAGE * L::kKRow, pf);
            __syncthreads();
        }
        if (ballot64(bad) != 0ull && lane == 0) flag_device_status(kDevBadPage);
    }

    // the first group takes in what the others leave, in their order, and writes the result or its part of one
    float* buf = reinterpret_cast<float*>(lds);
    if (KW > 1) {
        const int set = (kg - 1) * ROWS + 32 * rw;
        if (kg > 0) st.leave(buf + set * L::kMergeRow, sh_m + set, sh_l + set);
        __syncthreads();
        if (kg > 0) return;
    }
    if (!P.single && w.unit == 0 && r.split == 0 && threadIdx.x == 0) P.ranges[r.b] = make_int2(r.n, r.slot0);
    const int l16 = lane & 15, q4 = lane >> 4;
#pragma unroll
    for (int f = 0; f < NR; ++f) {
        const int rr = 32 * rw + 16 * f + l16, qrow = w.row_tile * ROWS + rr;
        float M = st.m[f], l = quad_sum(st.lsum[f]);
#pragma unroll
        for (int e = 0; e < KW - 1; ++e) {
            const float m = sh_m[e * ROWS + rr], top = fmaxf(M, m), base = top == kNegInf ? 0.f : top;
            const float a = fast_exp2((M - base) * c), b = fast_exp2((m - base) * c);  // 0 for a state without keys
            l = a * l + b * sh_l[e * ROWS + rr];
#pragma unroll
            for (int db = 0; db < D / 16; ++db)
                st.o[f][db] = a * st.o[f][db] + b * *reinterpret_cast<const f32x4_t*>(buf + (e * ROWS + rr) * L::kMergeRow + 16 * db + 4 * q4);
            M = top;
        }
        const int t = P.by_group.div(qrow), h = w.g * P.group + qrow - t * P.group;
        const bool pad = t >= n_new;  // whose query may hold anything
        if (qrow >= P.rows) continue;
        if (r.n == 1) {
            const float inv = l > 0.f && !pad ? 1.0f / l : 0.f;  // a row that sees nothing: 0
            uint16_t* out = P.out + (((int64_t)r.b * P.T + t) * P.Hq + h) * D + 4 * q4;
#pragma unroll
            for (int db = 0; db < D / 16; ++db) {
                const f32x4_t o = pad ? f32x4_t{} : st.o[f][db];
                u32x2_t x;
                x[0] = (uint32_t)f2bf(o[0] * inv) | ((uint32_t)f2bf(o[1] * inv) << 16);
                x[1] = (uint32_t)f2bf(o[2] * inv) | ((uint32_t)f2bf(o[3] * inv) << 16);
                *reinterpret_cast<u32x2_t*>(out + 16 * db) = x;
            }
        } else {
            const int64_t at = ((int64_t)w.slot * P.units + w.unit) * ROWS + rr;
#pragma unroll
            for (int db = 0; db < D / 16; ++db)
                *reinterpret_cast<f32x4_t*>(P.part_o + at * D + 16 * db + 4 * q4) = pad ? f32x4_t{} : st.o[f][db];
            if (q4 == 0) *reinterpret_cast<float2*>(P.part_ml + 2 * at) = pad ? make_float2(kNegInf, 0.f) : make_float2(M, l);
        }
    }
}

}  // namespace trajspec
