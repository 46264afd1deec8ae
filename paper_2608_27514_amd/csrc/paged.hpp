// The paged key-value cache: pages of `page_size` tokens in one pool, a table of page numbers per
// sequence (token s of sequence b lies in page table[b][s / page_size], row s % page_size), and per-sequence
// lengths that only the device knows.
//   paged_append_kernel   rotates the new tokens' queries and keys by position and writes keys and values
//                         into the pages
//   paged_attn_kernel     attention of the new tokens over their sequences' cached keys
//   paged_join_kernel     joins the partial results of sequences whose keys were split over workgroups
#pragma once

#include <type_traits>

#include "conf_topk.hpp"
#include "layer.hpp"
#include "verify_attn16.hpp"

namespace trajspec {

constexpr int kDevBadLength = 0x10;  // TRAJ_DEV_BAD_LENGTH
constexpr int kDevBadPage = 0x20;    // TRAJ_DEV_BAD_PAGE

// n / d for 0 <= n < 2^31 as a multiplication: with 2^(s-1) < d <= 2^s and m = ceil(2^(31+s) / d) < 2^32
// the error m d - 2^(31+s) < 2^s adds less than 1 / d to the quotient of any such n.
struct FastDiv {
    uint32_t mul;
    int shift;
    __device__ __forceinline__ int div(int n) const { return (int)(((uint64_t)(uint32_t)n * mul) >> shift); }
};

struct PagedCache {
    uint16_t *k, *v;
    const int32_t* table;
    int64_t table_stride, page_stride, token_stride, head_stride;  // elements
    int num_pages, page_size, capacity;  // capacity: tokens of a row of the table
    FastDiv by_page;
};

// ------------------------------------------------------------------ append
constexpr int kAppendThreads = 256;
constexpr int kAppendMaxHalf = 64;  // D / 2
constexpr int kAppendTokens = 4;    // tokens a workgroup takes where there are many

struct AppendParams {
    const uint16_t *q, *k, *v;            // token rows of contiguous heads; q may be null
    int64_t q_row, k_row, v_row;          // elements from one token's row to the next
    uint16_t* q_out;                      // [B, T, Hq, D]
    PagedCache cache;
    const int32_t *start, *n_new, *pos0;  // [B]; n_new null: T, pos0 null: start
    int T, Hq, Hkv, rotate;
    int per_token;  // chunk pairs of a token
    FastDiv by_token;
    double turns[kAppendMaxHalf];  // rotation per position of pair d in turns: theta^(-2d/D) / 2 pi
};

// A pair of 16-byte chunks (8 values of a head's first half and the matching 8 of its second) per thread and
// step.  The angle pos * theta^(-2d/D) is reduced to a turn's fraction in 64 bits (in 32 a position of 10^5
// would be off by 2^-8 of a radian) and its sine and cosine, computed once per token, pass through LDS.
// Bound by the copy (2 (Hq + 2 Hkv) D bytes read and written per token).
// grid: x = groups of TOK tokens of a sequence (one token: y shares its chunks out), z = sequence.
template <int D, int TOK>
__global__ __launch_bounds__(kAppendThreads) void paged_append_kernel(AppendParams P) {
    constexpr int HALF = D / 2, CPR = HALF / 8;
    __shared__ float cs[TOK][HALF], sn[TOK][HALF];
    const int b = blockIdx.z, p0 = blockIdx.x * TOK;
    const int start = P.start[b];
    int n = P.n_new != nullptr ? P.n_new[b] : P.T;
    const bool report = blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0;
    if (n < 0 || n > P.T) {
        if (report) flag_device_status(kDevBadLength);
        n = n < 0 ? 0 : P.T;
    }
    if (p0 >= n) return;
    if (start < 0 || (int64_t)start + n > P.cache.capacity) {
        if (report) flag_device_status(kDevBadLength);
    }
    const int qh = P.q != nullptr ? P.Hq : 0;
    const int tasks = min(n - p0, TOK) * P.per_token;
    if (P.rotate) {
        const int64_t pos0 = (int64_t)(P.pos0 != nullptr ? P.pos0[b] : start) + p0;
        for (int i = threadIdx.x; i < TOK * HALF; i += kAppendThreads) {
            const int tok = i / HALF, d = i % HALF;
            const double turn = (double)(pos0 + tok) * P.turns[d];
            sincospif(2.0f * (float)(turn - floor(turn)), &sn[tok][d], &cs[tok][d]);
        }
        __syncthreads();
    }
    const int64_t t0 = (int64_t)b * P.T + p0;
    for (int i = blockIdx.y * kAppendThreads + threadIdx.x; i < tasks; i += gridDim.y * kAppendThreads) {
        const int tok = P.by_token.div(i), r = i - tok * P.per_token;
        const int head = r / CPR, d0 = 8 * (r % CPR);  // q heads, k heads, v heads
        const int64_t t = t0 + tok;
        const uint16_t* src = head < qh           ? P.q + t * P.q_row + head * D
                              : head < qh + P.Hkv ? P.k + t * P.k_row + (head - qh) * D
                                                  : P.v + t * P.v_row + (head - qh - P.Hkv) * D;
        u32x4_t lo = ldg16(src + d0), hi = ldg16(src + d0 + HALF);
        uint16_t* dst;
        if (head < qh) {
            dst = P.q_out + (t * P.Hq + head) * D;
        } else {
            const int64_t at = (int64_t)start + p0 + tok;
            if (at < 0 || at >= P.cache.capacity) continue;
            const int col = P.cache.by_page.div((int)at);
            const int page = P.cache.table[b * P.cache.table_stride + col];
            if (page < 0 || page >= P.cache.num_pages) {
                if (r == qh * CPR) flag_device_status(kDevBadPage);
                continue;
            }
            const bool key = head < qh + P.Hkv;
            dst = (key ? P.cache.k : P.cache.v) + page * P.cache.page_stride + ((int)at - col * P.cache.page_size) * P.cache.token_stride +
                  (head - qh - (key ? 0 : P.Hkv)) * P.cache.head_stride;
        }
        if (P.rotate && head < qh + P.Hkv) {
            const u32x4_t a = lo, c = hi;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int d = d0 + 2 * e;
                const float x1a = bf16_lo(a[e]), x1b = bf16_hi(a[e]);
                const float x2a = bf16_lo(c[e]), x2b = bf16_hi(c[e]);
                const float ca = cs[tok][d], cb = cs[tok][d + 1], sa = sn[tok][d], sb = sn[tok][d + 1];
                lo[e] = (uint32_t)f2bf(x1a * ca - x2a * sa) | ((uint32_t)f2bf(x1b * cb - x2b * sb) << 16);
                hi[e] = (uint32_t)f2bf(x2a * ca + x1a * sa) | ((uint32_t)f2bf(x2b * cb + x1b * sb) << 16);
            }
        }
        *reinterpret_cast<u32x4_t*>(dst + d0) = lo;
        *reinterpret_cast<u32x4_t*>(dst + d0 + HALF) = hi;
    }
}

// ------------------------------------------------------------------ attention
// Every cached key and value is read once and takes T Hq / Hkv multiply-adds per element, so up to some hundreds of
// rows (row = new token * group + head in group of one kv head) the stream of K and V bounds the call: rows are padded
// to 16 for the matrix core, which idles either way, and what counts is how the loads are issued.
//   * Whole 128-byte lines per load: a wave takes 4 (D = 128) or 8 rows of K or V per instruction, not the 16 rows of
//     32 values that the K operand wants; both pass through LDS, which also does V's transposition
//     (65536 keys, 8 heads, non-temporal: 66.8 -> 59.8 us).
//   * Page numbers come by scalar loads and are requested a tile before they are needed.  Loaded like the keys they
//     drained the wave's whole queue once per tile.
//   * Two tiles in flight per wave where the registers hold them; buffers for 16 visible rows each give uniform
//     bases and zeros behind the last key.
//   * Each weight takes part in two products, as bf16 and as what that leaves: up to 32 rows this costs under 1%.
//   S^T = K Q^T, weights in the lane that has the scores, O^T += V^T P^T: layouts of the 16-row verification kernel.
//
// Splits: the device computes from the lengths how many keys a workgroup takes (`chunk`).  A slot is a (sequence, range)
// pair in order; the partial results of a sequence in several ranges are joined by a second kernel.
//   MI355X: 32 sequences of up to 8192 keys x 32 heads of 128 (2.2 GB) 359 us = 6.2 TB/s, one of 2^20 keys x 8 heads
//   6.7 TB/s, one of 65536 49.2 us = 5.5 TB/s (the read-only logit pass streams 6.2 TB/s).
constexpr int kPagedWaves = 4;
constexpr int kPagedThreads = kPagedWaves * 64;
constexpr int kPagedTile = 32;
constexpr int kPagedGranule = kPagedWaves * kPagedTile;
// Chunks make about kPagedFillWgs workgroups at least (one per CU), then stay at kPagedChunk keys, under which filling and
// joining costs more than the shorter chain saves (65536 keys x 8 heads: 512 keys take 1.5 us longer than 1024), and grow once
// there are kPagedMostWgs of them: finer ones balance lengths and CUs better (32 sequences of up to 8192 keys: 4224 keys
// 377 us, 2112 keys 359).  All three were measured on calls of one token a sequence and hold for the kernels of more rows too.
constexpr int kPagedFillWgs = 256, kPagedChunk = 1024, kPagedMostWgs = 2048;
// More sequences than this fill the chip by themselves and are never split: every workgroup of a split call looks at all
// lengths.
constexpr int kPagedSplitBatch = 2048;
// Nor are batches of so many query rows, of which a wave each would not go into the joining launch.
constexpr int64_t kPagedSplitRows = 1 << 26;
// Caches up to this many keys are never split: a join takes longer.  One token each, whole and split: 192 keys 4.2 and 7.4 us
// (4 heads of 64), 5.4 and 7.6 (32 over 8 of 128); 272 keys 5.0 and 6.4, 6.6 and 7.1; 512 keys 5.9 and 6.6, 8.2 and 7.2.
// Blocks of 32 tokens, 28 over 4 heads: 192 keys 12.5 and 13.9, 272 keys 16.9 and 14.8.  `capacity` decides, as the launch
// knows no length: short sequences in a wide table pay the split's price.
constexpr int kPagedWhole = 256;

struct PagedAttnParams {
    const uint16_t* q;
    PagedCache cache;
    const int32_t *lens, *n_new;  // [B]; n_new null: T
    uint16_t* out;
    float *part_o, *part_ml;  // partial results per (slot, unit, row): D values; maximum and sum
    int2* ranges;             // [B] number of ranges, first slot
    int B, T, Hq, Hkv, group, rows;  // rows = T * group
    FastDiv by_group;
    int tile_rows, tiles, units;     // rows per tile; tiles; units = Hkv * tiles
    int single, causal;              // single: no sequence can be split
    float scale_log2;
};

struct PagedRange {
    int b, split, n, slot0, len, chunk;  // n: ranges of sequence b, the first at slot0
};

__device__ __forceinline__ int paged_length(const PagedAttnParams& P, int b, bool report) {
    const int len = P.lens[b];
    if (len < 0 || len > P.cache.capacity) {
        if (report) flag_device_status(kDevBadLength);
        return len < 0 ? 0 : P.cache.capacity;
    }
    return len;
}

// New tokens of a sequence; the rows behind them are padding.
__device__ __forceinline__ int paged_new(const PagedAttnParams& P, int b, bool report) {
    if (P.n_new == nullptr) return P.T;
    const int n = P.n_new[b];
    if (n < 0 || n > P.T) {
        if (report) flag_device_status(kDevBadLength);
        return n < 0 ? 0 : P.T;
    }
    return n;
}

// Keys per workgroup.  Every wave computes the same from the same lengths (whole numbers, quotients by powers of two).
__device__ __forceinline__ int paged_chunk(int64_t total, int units, int capacity) {
    const double work = (double)total * (double)units / kPagedGranule;
    double per = fmax(work / kPagedMostWgs, fmin(work / kPagedFillWgs, (double)(kPagedChunk / kPagedGranule)));
    per = fmin(per, (double)(capacity / kPagedGranule + 1));
    const int granules = (int)ceil(per);
    return kPagedGranule * (granules < 1 ? 1 : granules);
}

// Workgroup i runs on XCD i % 8.  The row tiles of one (slot, kv head) follow each other on one XCD, whose L2
// they share; the (slot, kv head) pairs go round the XCDs in order, so that slots without work, the last ones,
// leave none of them idle.
struct PagedPlace {
    int slot, g, unit, row_tile;
};
__device__ __forceinline__ PagedPlace paged_place(const PagedAttnParams& P) {
    PagedPlace w;
    const int turn = blockIdx.x / 8 / P.tiles, pair = turn * 8 + blockIdx.x % 8;
    w.row_tile = blockIdx.x / 8 - turn * P.tiles;
    w.slot = pair / P.Hkv;
    w.g = pair - w.slot * P.Hkv;
    w.unit = w.g * P.tiles + w.row_tile;
    return w;
}

// The range that the workgroup's slot stands for; false where the batch has fewer.  All lanes of the wave take part.
// Lengths out of range are reported once per sequence where each workgroup looks at its own alone, else by workgroup 0.
__device__ __forceinline__ bool paged_range(const PagedAttnParams& P, const PagedPlace& w, PagedRange& r) {
    const int lane = threadIdx.x & 63, slot = w.slot;
    if (P.single) {
        if (slot >= P.B) return false;
        r = PagedRange{slot, 0, 1, slot, paged_length(P, slot, w.unit == 0 && threadIdx.x == 0), P.cache.capacity};
        return true;
    }
    const bool report = blockIdx.x == 0;
    const int len0 = lane < P.B ? paged_length(P, lane, report) : 0;
    uint64_t total = len0;
    for (int i = lane + 64; i < P.B; i += 64) total += paged_length(P, i, report);
#pragma unroll
    for (int t = 0; t < 6; ++t) {
        uint64_t x, y;
        lane_pair64(t, total, x, y);
        total = x + y;
    }
    const int chunk = __builtin_amdgcn_readfirstlane(paged_chunk((int64_t)total, P.units, P.cache.capacity));
    int base = 0;
    for (int i0 = 0; i0 < P.B; i0 += 64) {
        const int i = i0 + lane;
        const int len = i0 == 0 ? len0 : i < P.B ? paged_length(P, i, false) : 0;
        int n = (int)(((uint32_t)len + (uint32_t)chunk - 1u) / (uint32_t)chunk);
        n = i < P.B ? (n < 1 ? 1 : n) : 0;  // an empty sequence still has rows to write
        const int incl = wave_prefix(n), lo = base + incl - n;
        const uint64_t hit = ballot64(slot >= lo && slot < lo + n);
        if (hit != 0ull) {
            const int src = __builtin_ctzll(hit);
            r.b = i0 + src;
            r.n = __builtin_amdgcn_readlane(n, src);
            r.slot0 = __builtin_amdgcn_readlane(lo, src);
            r.len = __builtin_amdgcn_readlane(len, src);
            r.split = slot - r.slot0;
            r.chunk = chunk;
            return true;
        }
        base += __builtin_amdgcn_readlane(incl, 63);
    }
    return false;
}

// Where a tile of 16 BLK keys lies.  UNIFORM (page_size % 16 == 0): each 16-key block within one page, so its page
// comes by a scalar load and its base is uniform; otherwise lane l holds the page and the offset of key l % (16 BLK).
// vis: visible keys (inside the range, on a good page).
template <bool UNIFORM, int BLK>
struct PagedTile {
    int64_t at[UNIFORM ? BLK : 1];
    uint32_t vis;
};
template <bool UNIFORM, int BLK>
struct PagedPages {
    int page[UNIFORM ? BLK : 1];
};
typedef const __attribute__((address_space(4))) int32_t const_i32_t;  // read by scalar loads where uniform

// Page numbers of the tile at key0: only requested here, looked at a tile later.  Keys at or behind `end`
// take the place of `first`, which lies before it.
template <bool UNIFORM, int BLK>
__device__ __forceinline__ PagedPages<UNIFORM, BLK> paged_pages(const PagedCache& C, const int32_t* row, int key0, int first, int end) {
    PagedPages<UNIFORM, BLK> p;
    if constexpr (UNIFORM) {
        const_i32_t* table = (const_i32_t*)(uintptr_t)row;
#pragma unroll
        for (int j = 0; j < BLK; ++j) p.page[j] = table[C.by_page.div(key0 + 16 * j < end ? key0 + 16 * j : first)];
    } else {
        const int key = key0 + (threadIdx.x & (16 * BLK - 1));
        p.page[0] = row[C.by_page.div(key < end ? key : first)];
    }
    return p;
}

__device__ __forceinline__ int64_t uniform64(int64_t x) {
    const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)x), hi = __builtin_amdgcn_readfirstlane((uint32_t)((uint64_t)x >> 32));
    return (int64_t)(((uint64_t)hi << 32) | lo);
}

template <bool UNIFORM, int BLK>
__device__ __forceinline__ PagedTile<UNIFORM, BLK> paged_tile(const PagedCache& C, const PagedPages<UNIFORM, BLK>& p, int64_t head, int key0,
                                                              int first, int end, bool& bad) {
    PagedTile<UNIFORM, BLK> t;
    t.vis = 0;
#pragma unroll
    for (int j = 0; j < (UNIFORM ? BLK : 1); ++j) {
        const int key = UNIFORM ? key0 + 16 * j : key0 + (int)(threadIdx.x & (16 * BLK - 1));
        const int at = key < end ? key : first;
        const bool good = p.page[j] >= 0 && p.page[j] < C.num_pages;
        bad |= !good && key < end;
        t.at[j] = (good ? p.page[j] : 0) * C.page_stride + (at - C.by_page.div(at) * C.page_size) * C.token_stride + head;
        if constexpr (UNIFORM) {
            const int n = key < end && good ? (end - key < 16 ? end - key : 16) : 0;
            t.vis |= ((1u << n) - 1u) << (16 * j);
            t.at[j] = uniform64(t.at[j]);
        } else {
            t.vis = (uint32_t)ballot64(good && key < end) & (BLK == 2 ? 0xffffffffu : 0xffffu);
        }
    }
    return t;
}

// A tile's rows of K or V, whole 128-byte lines per wave-wide load (512 / D rows).  UNIFORM: a buffer of each block's
// visible rows with 32-bit lane offsets, so that rows behind its end read as 0.  ONCE: nothing reads them again.
template <int D, bool UNIFORM, int BLK, bool ONCE>
__device__ __forceinline__ void paged_load(u32x4_t (&x)[BLK * D / 32], const uint16_t* pool, const PagedTile<UNIFORM, BLK>& t, int token_stride) {
    constexpr int RPI = 512 / D;
    const int lane = threadIdx.x & 63, vrow = lane / (D / 8), vchunk = lane % (D / 8);
#pragma unroll
    for (int i = 0; i < BLK * D / 32; ++i) {
        if constexpr (UNIFORM) {
            const int j = i * RPI / 16, rows = __popc(t.vis >> (16 * j) & 0xffffu);
            const auto rs = __builtin_amdgcn_make_buffer_rsrc((void*)(pool + t.at[j]), (short)0, rows * 2 * token_stride, kBufferFlags);
            x[i] = __builtin_amdgcn_raw_buffer_load_b128(rs, 2 * (((i * RPI) % 16 + vrow) * token_stride + 8 * vchunk), 0, ONCE ? 2 : 0);
        } else {
            const u32x4_t* p = reinterpret_cast<const u32x4_t*>(pool + __shfl(t.at[0], i * RPI + vrow) + 8 * vchunk);
            x[i] = ONCE ? __builtin_nontemporal_load(p) : *p;
        }
    }
}

// LDS rows: elements per row of a K tile (the 16 rows of a fragment read start 4 banks apart), of a V tile (the 8 rows
// that half a wave reads of a transposing load start 8 banks apart, 72 and 40 words a row, and each takes 8 of the
// 64), and floats per row of the merge buffers.
template <int D>
struct PagedLds {
    static constexpr int kKRow = D + 8, kVRow = D + 16, kMergeRow = D + 4;
};

// A wave's query rows: 16 NR of them, row 16 f + lane % 16 in fragment f.
template <int D, int NR>
struct PagedRows {
    bf16x8_t qf[NR][D / 32];     // head dims 32 ks + 8 (lane / 16) ..
    int limit[NR];               // keys that the row sees
    f32x4_t o[NR][D / 16];       // O^T: head dims 16 db + 4 (lane / 16) ..
    float m[NR], neg_mc[NR], lsum[NR];  // the reference is the maximum itself: the largest weight is 1 and exact in bf16

    __device__ __forceinline__ void init(const PagedAttnParams& P, int b, int g, int len, int n_new, int row0) {
        const int lane = threadIdx.x & 63;
#pragma unroll
        for (int f = 0; f < NR; ++f) {
            const int row = min(row0 + 16 * f + (lane & 15), P.rows - 1);  // rows past the last repeat it and are not stored
            const int t = P.by_group.div(row), h = g * P.group + row - t * P.group;
            limit[f] = P.causal ? len - n_new + t + 1 : len;
#pragma unroll
            for (int ks = 0; ks < D / 32; ++ks)
                qf[f][ks] = __builtin_bit_cast(bf16x8_t, ldg16(P.q + (((int64_t)b * P.T + t) * P.Hq + h) * D + 32 * ks + 8 * (lane >> 4)));
            m[f] = kNegInf;
            neg_mc[f] = 0.f;
            lsum[f] = 0.f;
#pragma unroll
            for (int db = 0; db < D / 16; ++db) o[f][db] = f32x4_t{};
        }
    }

    // S^T = K Q^T of the 32 NK keys whose LDS rows start at k
    template <int NK>
    __device__ __forceinline__ void scores(const uint16_t* k, f32x4_t (&s)[NR][2 * NK]) const {
        const int lane = threadIdx.x & 63;
        const uint16_t* kread = k + (lane & 15) * PagedLds<D>::kKRow + 8 * (lane >> 4);
#pragma unroll
        for (int f = 0; f < NR; ++f)
#pragma unroll
            for (int j = 0; j < 2 * NK; ++j) s[f][j] = f32x4_t{};
#pragma unroll
        for (int ks = 0; ks < D / 32; ++ks)
#pragma unroll
            for (int j = 0; j < 2 * NK; ++j) {
                const bf16x8_t kf = lds16(kread + 16 * j * PagedLds<D>::kKRow + 32 * ks);
#pragma unroll
                for (int f = 0; f < NR; ++f) s[f][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[f][ks], s[f][j], 0, 0, 0);
            }
    }

    // scores of keys key0 .. that are not in vis or behind the row's last key
    template <int NK>
    __device__ __forceinline__ void mask(f32x4_t (&s)[NR][2 * NK], uint64_t vis, int key0) const {
#pragma unroll
        for (int f = 0; f < NR; ++f)
#pragma unroll
            for (int v = 0; v < 8 * NK; ++v) {
                const int k = 16 * (v >> 2) + 4 * ((threadIdx.x & 63) >> 4) + (v & 3);
                const bool seen = ((vis >> k) & 1ull) != 0ull && key0 + k < limit[f];
                s[f][v >> 2][v & 3] = seen ? s[f][v >> 2][v & 3] : kNegInf;
            }
    }

    // Weights of the keys against the running reference, in the operand order of values().  What rounding to bf16 leaves
    // goes into a second operand, so that the product has the weights to 16 bits.
    template <int NK>
    __device__ __forceinline__ void weights(const f32x4_t (&s)[NR][2 * NK], float c, bf16x8_t (&pf)[2][NR][NK]) {
#pragma unroll
        for (int f = 0; f < NR; ++f) {
            float mx = s[f][0][0];
#pragma unroll
            for (int v = 1; v < 8 * NK; ++v) mx = __builtin_elementwise_maximum(mx, s[f][v >> 2][v & 3]);
            mx = quad_max(mx);
            const bool up = mx > m[f];
            if (ballot64(up) != 0ull) {  // rare after the first tiles
                const float m_new = up ? mx : m[f];
                const float alpha = up ? fast_exp2((m[f] - m_new) * c) : 1.0f;  // 0 at the first reference
                lsum[f] *= alpha;
#pragma unroll
                for (int db = 0; db < D / 16; ++db) o[f][db] *= alpha;
                m[f] = m_new;
                neg_mc[f] = m_new == kNegInf ? 0.f : -m_new * c;
            }
#pragma unroll
            for (int v = 0; v < 8 * NK; ++v) {
                const float p = fast_exp2(__builtin_fmaf(s[f][v >> 2][v & 3], c, neg_mc[f]));
                lsum[f] += p;
                pf[0][f][v / 8][v % 8] = (__bf16)p;
                pf[1][f][v / 8][v % 8] = (__bf16)(p - (float)(__bf16)p);
            }
        }
    }

    // O^T += V^T P^T over the 32 NK keys whose LDS rows start at v
    template <int NK>
    __device__ __forceinline__ void values(const uint16_t* v, const bf16x8_t (&pf)[2][NR][NK]) {
        const int lane = threadIdx.x & 63;
        const uint16_t* vread = v + (4 * (lane >> 4) + ((lane & 15) >> 2)) * PagedLds<D>::kVRow + 4 * (lane & 3);
#pragma unroll
        for (int i = 0; i < NK; ++i)
#pragma unroll
            for (int db = 0; db < D / 16; ++db) {
                const bf16x4_t a0 = lds_read_tr(vread + 16 * db + 32 * i * PagedLds<D>::kVRow);
                const bf16x4_t a1 = lds_read_tr(vread + 16 * db + (32 * i + 16) * PagedLds<D>::kVRow);
                const bf16x8_t va = __builtin_shufflevector(a0, a1, 0, 1, 2, 3, 4, 5, 6, 7);
#pragma unroll
                for (int e = 0; e < 2; ++e)
#pragma unroll
                    for (int f = 0; f < NR; ++f) o[f][db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va, pf[e][f][i], o[f][db], 0, 0, 0);
            }
    }

    // this wave's state into its rows of a merge buffer
    __device__ __forceinline__ void leave(float* buf, float* sm, float* sl) const {
        const int lane = threadIdx.x & 63, q4 = lane >> 4, l16 = lane & 15;
#pragma unroll
        for (int f = 0; f < NR; ++f) {
            const float l = quad_sum(lsum[f]);
            if (q4 == 0) {
                sm[16 * f + l16] = m[f];
                sl[16 * f + l16] = l;
            }
#pragma unroll
            for (int db = 0; db < D / 16; ++db)
                *reinterpret_cast<f32x4_t*>(buf + (16 * f + l16) * PagedLds<D>::kMergeRow + 16 * db + 4 * q4) = o[f][db];
        }
    }
};

// Joins the SETS states of each of a workgroup's ROWS rows and writes the result, or its part of a sequence in several
// ranges.
template <int D, int ROWS, int SETS>
__device__ __forceinline__ void paged_store(const PagedAttnParams& P, const PagedRange& r, const PagedPlace& w, int n_new, const float* buf,
                                            const float* sm, const float* sl) {
    constexpr int kRow = PagedLds<D>::kMergeRow, LPR = D / 4, STEP = kPagedThreads / LPR;
    const int d = 4 * (threadIdx.x % LPR), first = threadIdx.x / LPR;
    if (!P.single && w.unit == 0 && r.split == 0 && threadIdx.x == 0) P.ranges[r.b] = make_int2(r.n, r.slot0);
#pragma unroll
    for (int i = 0; i < ROWS / STEP; ++i) {
        const int rr = first + i * STEP, qrow = w.row_tile * ROWS + rr;
        float M = kNegInf;
#pragma unroll
        for (int e = 0; e < SETS; ++e) M = fmaxf(M, sm[e * ROWS + rr]);
        const float Ms = M == kNegInf ? 0.f : M;
        f32x4_t acc = {};
        float l = 0.f;
#pragma unroll
        for (int e = 0; e < SETS; ++e) {
            const float scale = SETS == 1 ? 1.0f : fast_exp2((sm[e * ROWS + rr] - Ms) * P.scale_log2);  // 0 for a state without keys
            l += scale * sl[e * ROWS + rr];
            acc += scale * *reinterpret_cast<const f32x4_t*>(buf + (e * ROWS + rr) * kRow + d);
        }
        const int t = P.by_group.div(qrow), h = w.g * P.group + qrow - t * P.group;
        if (t >= n_new) {  // padding, whose query may hold anything
            M = kNegInf;
            l = 0.f;
            acc = f32x4_t{};
        }
        if (r.n == 1) {
            const float inv = l > 0.f ? 1.0f / l : 0.f;  // a row that sees nothing: 0
            u32x2_t x;
            x[0] = (uint32_t)f2bf(acc[0] * inv) | ((uint32_t)f2bf(acc[1] * inv) << 16);
            x[1] = (uint32_t)f2bf(acc[2] * inv) | ((uint32_t)f2bf(acc[3] * inv) << 16);
            if (qrow < P.rows) *reinterpret_cast<u32x2_t*>(P.out + (((int64_t)r.b * P.T + t) * P.Hq + h) * D + d) = x;
        } else if (qrow < P.rows) {
            const int64_t at = ((int64_t)w.slot * P.units + w.unit) * ROWS + rr;
            *reinterpret_cast<f32x4_t*>(P.part_o + at * D + d) = acc;
            if (d == 0) *reinterpret_cast<float2*>(P.part_ml + 2 * at) = make_float2(M, l);
        }
    }
}

// Up to 32 rows: the waves take the range's 32-key tiles in turn.
template <int D, int NR, bool UNIFORM, int DEPTH>
__global__ __launch_bounds__(kPagedThreads, 2) void paged_attn_kernel(PagedAttnParams P) {
    using L = PagedLds<D>;
    constexpr int ROWS = 16 * NR, NVL = D / 16, RPI = 512 / D;
    constexpr int kTileBytes = kPagedTile * L::kVRow * 2, kMergeBytes = ROWS * L::kMergeRow * 4;
    constexpr int kTiles = kPagedWaves * kTileBytes, kMerge = kPagedWaves * kMergeBytes;
    __shared__ __align__(16) char lds[kTiles > kMerge ? kTiles : kMerge];
    __shared__ float sh_m[kPagedWaves * ROWS], sh_l[kPagedWaves * ROWS];

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const PagedPlace w = paged_place(P);
    PagedRange r;
    if (!paged_range(P, w, r)) return;
    const int len = r.len;
    const int begin = r.split * r.chunk, end = len - begin > r.chunk ? begin + r.chunk : len;
    const int n_new = paged_new(P, r.b, w.unit == 0 && r.split == 0 && threadIdx.x == 0);
    const int min_limit = P.causal ? len - n_new + 1 : len;  // of a row that is not padding

    // one LDS tile per wave, K's and then V's
    uint16_t* tile = reinterpret_cast<uint16_t*>(lds + wave * kTileBytes);
    const int vrow = lane / (D / 8), vchunk = lane % (D / 8);  // of a load
    uint16_t* kwrite = tile + vrow * L::kKRow + 8 * vchunk;
    uint16_t* vwrite = tile + vrow * L::kVRow + 8 * vchunk;

    const PagedCache& C = P.cache;
    const int ts = (int)C.token_stride;
    const int32_t* row = C.table + r.b * C.table_stride;
    const int64_t head = w.g * C.head_stride;
    const float c = P.scale_log2;
    const int first = begin + wave * kPagedTile;
    u32x4_t kr[DEPTH][NVL], vr[DEPTH][NVL];
    uint32_t vis[DEPTH];
    bool bad = false;
    using Tile = PagedTile<UNIFORM, 2>;
    using Pages = PagedPages<UNIFORM, 2>;
    PagedRows<D, NR> st;
    Pages pages;  // of the tile after those in flight
    // The tile at key0, held in ring slot u; with `more` also the loads of the tile DEPTH rounds behind it.
    auto step = [&](auto slot, int key0, bool more) {
        constexpr int u = decltype(slot)::value;
#pragma unroll
        for (int i = 0; i < NVL; ++i) *reinterpret_cast<u32x4_t*>(kwrite + i * RPI * L::kKRow) = kr[u][i];
        f32x4_t s[NR][2];
        st.template scores<1>(tile, s);
        if (!UNIFORM) __builtin_amdgcn_sched_barrier(0);  // lane addresses only while they are needed
        Tile next;
        if (more) {
            next = paged_tile<UNIFORM, 2>(C, pages, head, key0 + DEPTH * kPagedGranule, first, end, bad);
            pages = paged_pages<UNIFORM, 2>(C, row, key0 + (DEPTH + 1) * kPagedGranule, first, end);
            paged_load<D, UNIFORM, 2, true>(kr[u], C.k, next, ts);
        }
        if (!UNIFORM) __builtin_amdgcn_sched_barrier(0);
        if (vis[u] != 0xffffffffu || key0 + kPagedTile > min_limit) {  // rare: a sequence's last tile
            st.template mask<1>(s, vis[u], key0);
            // V rows that are not visible may hold anything and count as 0 (a block's buffer ends before them)
            if constexpr (!UNIFORM) {
#pragma unroll
                for (int i = 0; i < NVL; ++i)
                    if (((vis[u] >> (i * RPI + vrow)) & 1u) == 0u) vr[u][i] = u32x4_t{};
            }
        }
        bf16x8_t pf[2][NR][1];
        st.template weights<1>(s, c, pf);
#pragma unroll
        for (int i = 0; i < NVL; ++i) *reinterpret_cast<u32x4_t*>(vwrite + i * RPI * L::kVRow) = vr[u][i];
        if (!UNIFORM) __builtin_amdgcn_sched_barrier(0);
        if (more) {
            paged_load<D, UNIFORM, 2, true>(vr[u], C.v, next, ts);
            vis[u] = next.vis;
        }
        __builtin_amdgcn_sched_barrier(0);  // the next tile's products stay behind this one's: registers
        st.template values<1>(tile, pf);
        __builtin_amdgcn_sched_barrier(0);
    };

    auto fetch = [&](int u) { return paged_pages<UNIFORM, 2>(C, row, first + u * kPagedGranule, first, end); };
    Pages p0{}, p1{};
    if (first < end) {
        p0 = fetch(0);
        p1 = fetch(DEPTH - 1);
        pages = fetch(DEPTH);
    }
    st.init(P, r.b, w.g, len, n_new, w.row_tile * ROWS);
    int left = first < end ? (end - first + kPagedGranule - 1) / kPagedGranule : 0;  // tiles of this wave
    if (left > 0) {
        using Slot0 = std::integral_constant<int, 0>;
        using Slot1 = std::integral_constant<int, DEPTH - 1>;
        auto request = [&](auto slot, const Pages& p) {
            constexpr int u = decltype(slot)::value;
            const Tile t = paged_tile<UNIFORM, 2>(C, p, head, first + u * kPagedGranule, first, end, bad);
            vis[u] = t.vis;
            paged_load<D, UNIFORM, 2, true>(kr[u], C.k, t, ts);
            paged_load<D, UNIFORM, 2, true>(vr[u], C.v, t, ts);
        };
        int key0 = first;
        // No load under a condition ahead of the loop: the compiler's waits count the loads that every path issued.
        if constexpr (DEPTH == 1) {
            request(Slot0{}, p0);
            for (; left > 1; --left, key0 += kPagedGranule) step(Slot0{}, key0, true);
            step(Slot0{}, key0, false);
        } else if (left == 1) {
            request(Slot0{}, p0);
            step(Slot0{}, key0, false);
        } else {
            request(Slot0{}, p0);
            request(Slot1{}, p1);
            for (; left > 3; left -= 2, key0 += 2 * kPagedGranule) {
                step(Slot0{}, key0, true);
                step(Slot1{}, key0 + kPagedGranule, true);
            }
            if (left > 2) {
                step(Slot0{}, key0, true);
                step(Slot1{}, key0 + kPagedGranule, false);
                step(Slot0{}, key0 + 2 * kPagedGranule, false);
            } else {
                step(Slot0{}, key0, false);
                step(Slot1{}, key0 + kPagedGranule, false);
            }
        }
        if (ballot64(bad) != 0ull && lane == 0) flag_device_status(kDevBadPage);
    }

    __syncthreads();
    float* buf = reinterpret_cast<float*>(lds);
    st.leave(buf + wave * ROWS * L::kMergeRow, sh_m + wave * ROWS, sh_l + wave * ROWS);
    __syncthreads();
    paged_store<D, ROWS, kPagedWaves>(P, r, w, n_new, buf, sh_m, sh_l);
}

// More rows: RW waves of 32 rows each share the stages of 16 RW keys that they load into LDS together (a stage's K and
// V would otherwise pass from the L2 once per 32 rows); 4 / RW such groups of waves take the range's stages in turn.
// While a stage is multiplied the next one lies in registers on its way to the other buffer.  Here the matrix products
// and the LDS reads that feed them count too; the weights' second part costs 12% of the blocks below and 23% of 2 x 512
// tokens over 4096 keys (104 us without it), where the products bound the call.  Without it the error against 64 bits is
// 2.2e-3 of the output, with it 1.7e-3, which is the output's own rounding.
//   MI355X: 8 blocks of 32 tokens, 28 over 4 heads, up to 2048 keys 28.3 us; 2 of 64 tokens over 10000 keys 66.
template <int D, int RW, bool UNIFORM, bool ONCE>
__global__ __launch_bounds__(kPagedThreads, 2) void paged_rows_kernel(PagedAttnParams P) {
    using L = PagedLds<D>;
    constexpr int NR = 2, KW = kPagedWaves / RW, ROWS = 32 * RW, STAGE = 16 * RW, NK = STAGE / 32, NVL = D / 32, RPI = 512 / D;
    constexpr int kStage = STAGE * (L::kKRow + L::kVRow);  // elements
    constexpr int kStages = KW * 2 * kStage * 2, kMerge = KW * ROWS * L::kMergeRow * 4;
    __shared__ __align__(16) char lds[kStages > kMerge ? kStages : kMerge];
    __shared__ float sh_m[KW * ROWS], sh_l[KW * ROWS];
    __shared__ uint32_t sh_vis[KW][2][RW];

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int kg = wave / RW, rw = wave % RW;
    const PagedPlace w = paged_place(P);
    PagedRange r;
    if (!paged_range(P, w, r)) return;
    const int len = r.len;
    const int begin = r.split * r.chunk, end = len - begin > r.chunk ? begin + r.chunk : len;
    const int n_new = paged_new(P, r.b, w.unit == 0 && r.split == 0 && threadIdx.x == 0);
    const int min_limit = P.causal ? len - n_new + 1 : len;  // of a row that is not padding

    uint16_t* stage = reinterpret_cast<uint16_t*>(lds) + kg * 2 * kStage;  // two of them, K rows then V rows
    const int vrow = lane / (D / 8), vchunk = lane % (D / 8);
    const PagedCache& C = P.cache;
    const int ts = (int)C.token_stride;
    const int32_t* row = C.table + r.b * C.table_stride;
    const int64_t head = w.g * C.head_stride;
    const float c = P.scale_log2;
    u32x4_t kr[NVL], vr[NVL];  // this wave's 16 keys of the next stage
    uint32_t vis = 0;
    bool bad = false;
    const int rounds = (end - begin + KW * STAGE - 1) / (KW * STAGE);
    auto stage_key = [&](int n) { return begin + (n * KW + kg) * STAGE; };
    PagedPages<UNIFORM, 1> pages;
    auto fetch = [&](int n) { pages = paged_pages<UNIFORM, 1>(C, row, stage_key(n) + 16 * rw, begin, end); };
    auto request = [&](int n) {
        const PagedTile<UNIFORM, 1> t = paged_tile<UNIFORM, 1>(C, pages, head, stage_key(n) + 16 * rw, begin, end, bad);
        fetch(n + 1);
        paged_load<D, UNIFORM, 1, ONCE>(kr, C.k, t, ts);
        paged_load<D, UNIFORM, 1, ONCE>(vr, C.v, t, ts);
        vis = t.vis;
    };
    auto put = [&](int n) {
        uint16_t* k = stage + (n & 1) * kStage;
        uint16_t* kwrite = k + (16 * rw + vrow) * L::kKRow + 8 * vchunk;
        uint16_t* vwrite = k + STAGE * L::kKRow + (16 * rw + vrow) * L::kVRow + 8 * vchunk;
#pragma unroll
        for (int i = 0; i < NVL; ++i) {
            *reinterpret_cast<u32x4_t*>(kwrite + i * RPI * L::kKRow) = kr[i];
            u32x4_t x = vr[i];
            // rows that are not visible may hold anything and count as 0 (a block's buffer ends before them)
            if (!UNIFORM) x = ((vis >> (i * RPI + vrow)) & 1u) != 0u ? x : u32x4_t{};
            *reinterpret_cast<u32x4_t*>(vwrite + i * RPI * L::kVRow) = x;
        }
        if (lane == 0) sh_vis[kg][n & 1][rw] = vis;
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
            if (n + 1 < rounds) {
                put(n + 1);
                request(n + 2);
            }
            const uint16_t* k = stage + (n & 1) * kStage;
            uint32_t seen[NK];
#pragma unroll
            for (int i = 0; i < NK; ++i)
                seen[i] = __builtin_amdgcn_readfirstlane(sh_vis[kg][n & 1][2 * i] | sh_vis[kg][n & 1][2 * i + 1] << 16);
            const uint64_t all = NK == 1 ? seen[0] : seen[0] | (uint64_t)seen[NK - 1] << 32;
            if (all != 0ull) {
                f32x4_t s[NR][2 * NK];
                st.template scores<NK>(k, s);
                const int key0 = stage_key(n);
                if (all != (NK == 1 ? 0xffffffffull : ~0ull) || key0 + STAGE > min_limit) st.template mask<NK>(s, all, key0);
                bf16x8_t pf[2][NR][NK];
                st.template weights<NK>(s, c, pf);
                st.template values<NK>(k + STAGE * L::kKRow, pf);
            }
            __syncthreads();
        }
        if (ballot64(bad) != 0ull && lane == 0) flag_device_status(kDevBadPage);
    }

    float* buf = reinterpret_cast<float*>(lds);
    const int set = kg * ROWS + 32 * rw;
    st.leave(buf + set * L::kMergeRow, sh_m + set, sh_l + set);
    __syncthreads();
    paged_store<D, ROWS, KW>(P, r, w, n_new, buf, sh_m, sh_l);
}

// THREADS threads per (sequence, new token, query head): each range by D / 4 lanes, THREADS * 4 / D ranges at a time,
// every group with its own running maximum, joined through LDS in the groups' order.  Sequences in one range were
// written by the attention itself.
template <int D, int THREADS>
__global__ __launch_bounds__(THREADS < 256 ? 256 : THREADS) void paged_join_kernel(PagedAttnParams P) {
    constexpr int LPR = D / 4, GR = THREADS / LPR, ROWS = THREADS < 256 ? 256 / THREADS : 1, U = 4;
    static_assert(THREADS >= 64, "a row's lanes of a wave have one sequence");
    __shared__ f32x4_t sh_o[ROWS][GR][LPR];
    __shared__ float sh_m[ROWS][GR], sh_l[ROWS][GR];
    const int mine = threadIdx.x / THREADS, tid = threadIdx.x % THREADS;
    const int64_t rows = (int64_t)P.B * P.T * P.Hq;
    const int64_t orow = min((int64_t)blockIdx.x * ROWS + mine, rows - 1);
    const int h = (int)(orow % P.Hq);
    const int64_t bt = orow / P.Hq;
    const int b = (int)(bt / P.T), t = (int)(bt - (int64_t)b * P.T);
    const int2 r = P.ranges[b];
    const int g = h / P.group, qrow = t * P.group + h - g * P.group;
    const int unit = g * P.tiles + qrow / P.tile_rows, rr = qrow % P.tile_rows;
    const int64_t at0 = ((int64_t)r.y * P.units + unit) * P.tile_rows + rr, step = (int64_t)P.units * P.tile_rows;
    const int grp = tid / LPR, d = tid % LPR;
    const int n = r.x > 1 ? r.x : 0;
    f32x4_t acc = {};
    float m = kNegInf, l = 0.f;
    for (int s0 = grp; s0 < n; s0 += U * GR) {
        f32x4_t x[U];
        float xm[U], xl[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t a = at0 + min(s0 + u * GR, n - 1) * step;
            x[u] = *reinterpret_cast<const f32x4_t*>(P.part_o + a * D + 4 * d);
            xm[u] = s0 + u * GR < n ? P.part_ml[2 * a] : kNegInf;
            xl[u] = P.part_ml[2 * a + 1];
        }
        float top = m;
#pragma unroll
        for (int u = 0; u < U; ++u) top = fmaxf(top, xm[u]);
        const float ref = top == kNegInf ? 0.f : top;
        const float keep = fast_exp2((m - ref) * P.scale_log2);
        acc *= keep;
        l *= keep;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const float e = fast_exp2((xm[u] - ref) * P.scale_log2);
            acc += e * x[u];
            l += e * xl[u];
        }
        m = top;
    }
    sh_o[mine][grp][d] = acc;
    if (d == 0) {
        sh_m[mine][grp] = m;
        sh_l[mine][grp] = l;
    }
    __syncthreads();
    if (grp != 0 || n == 0 || (int64_t)blockIdx.x * ROWS + mine >= rows) return;
    float top = kNegInf;
#pragma unroll
    for (int w = 0; w < GR; ++w) top = fmaxf(top, sh_m[mine][w]);
    const float ref = top == kNegInf ? 0.f : top;
    l = 0.f;
    acc = f32x4_t{};
#pragma unroll
    for (int w = 0; w < GR; ++w) {
        const float e = fast_exp2((sh_m[mine][w] - ref) * P.scale_log2);
        l += e * sh_l[mine][w];
        acc += e * sh_o[mine][w][d];
    }
    const float inv = l > 0.f ? 1.0f / l : 0.f;
    u32x2_t w2;
    w2[0] = (uint32_t)f2bf(acc[0] * inv) | ((uint32_t)f2bf(acc[1] * inv) << 16);
    w2[1] = (uint32_t)f2bf(acc[2] * inv) | ((uint32_t)f2bf(acc[3] * inv) << 16);
    *reinterpret_cast<u32x2_t*>(P.out + orow * D + 4 * d) = w2;
}

}  // namespace trajspec
