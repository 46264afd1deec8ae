// The paged key-value cache: pages of `page_size` tokens in one pool, a table of page numbers per
// sequence (token s of sequence b lies in page table[b][s / page_size], row s % page_size), and per-sequence
// lengths that only the device knows.
//   paged_append_kernel   rotates the new tokens' queries and keys by position and writes keys and values
//                         into the pages
//   paged_attn_kernel     attention of the new tokens over their sequences' cached keys
//   paged_join_kernel     joins the partial results of sequences whose keys were split over workgroups
#pragma once

#include <type_traits>

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
// Work: a workgroup takes `16 NR` query rows of one (sequence, kv head) (row = new token * group + head in
// group) and a range of the sequence's keys; its 4 waves take 32-key tiles of the range in turn, each with its own
// running softmax state, merged through LDS at the end.  The call reads every cached key and value once and does
// T Hq / Hkv multiply-adds per element read, so up to some hundreds of rows the stream of K and V bounds it:
// rows are padded to 16 for the matrix core, which idles either way.
//   S^T = K Q^T with K fragments loaded straight from the pages into the A operand (no wave shares another's
//   keys); V goes through the wave's own LDS tile for the transposing reads of O^T += V^T P^T (layouts of
//   the 16-row verification kernel).  DEPTH tiles are held in registers: a tile's K registers are requested anew
//   behind its score MFMAs and its V registers behind the LDS writes; page numbers are requested a tile earlier.
//
// Splits: the device computes from the lengths how many keys a workgroup takes (`chunk`), so that the batch makes
// about kPagedTargetWgs workgroups whatever the lengths are; slot = index of a (sequence, range) pair in order.
constexpr int kPagedWaves = 4;
constexpr int kPagedThreads = kPagedWaves * 64;
constexpr int kPagedTile = 32;
constexpr int kPagedGranule = kPagedWaves * kPagedTile;
#ifndef X_TARGET
#define X_TARGET 2048
#endif
#ifndef X_FILL
#define X_FILL 512
#endif
#ifndef X_CHUNK
#define X_CHUNK 512
#endif
#ifndef X_NT
#define X_NT 1
#endif
constexpr int kPagedFillWgs = X_FILL, kPagedMostWgs = X_TARGET, kPagedChunk = X_CHUNK;
constexpr int kPagedWhole = 256;

struct PagedAttnParams {
    const uint16_t* q;
    PagedCache cache;
    const int32_t* lens;
    uint16_t* out;
    float *part_o, *part_ml;  // partial results per (slot, unit, row): D values; maximum and sum
    int B, T, Hq, Hkv, group, rows;  // rows = T * group
    int tiles, units;                // row tiles; units = Hkv * tiles
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

// Keys per workgroup.  Every wave computes the same from the same lengths (whole numbers, quotients by powers of two).
__device__ __forceinline__ int paged_chunk(int64_t total, int units, int capacity) {
    const double work = (double)total * (double)units / kPagedGranule;  // of all workgroups together
    double per = fmax(work / kPagedMostWgs, fmin(work / kPagedFillWgs, (double)(kPagedChunk / kPagedGranule)));
    per = fmin(per, (double)(capacity / kPagedGranule + 1));
    const int granules = (int)ceil(per);
    return kPagedGranule * (granules < 1 ? 1 : granules);
}

// The range that `slot` stands for (by == false), or the ranges of sequence `slot` (by == true); false where
// the batch has fewer.  All lanes of the wave take part.
__device__ __forceinline__ bool paged_range(const PagedAttnParams& P, int slot, bool by, bool report, PagedRange& r) {
    const int lane = threadIdx.x & 63;
    if (P.single) {
        if (slot >= P.B) return false;
        r = PagedRange{slot, 0, 1, slot, paged_length(P, slot, report), P.cache.capacity};
        return true;
    }
    int64_t total = 0;
    for (int i = lane; i < P.B; i += 64) total += paged_length(P, i, report);
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) total += __shfl_xor(total, off);
    const int chunk = __builtin_amdgcn_readfirstlane(paged_chunk(total, P.units, P.cache.capacity));
    int base = 0;
    for (int i0 = 0; i0 < P.B; i0 += 64) {
        const int i = i0 + lane;
        const int len = i < P.B ? paged_length(P, i, false) : 0;
        int n = (int)(((uint32_t)len + (uint32_t)chunk - 1u) / (uint32_t)chunk);
        n = i < P.B ? (n < 1 ? 1 : n) : 0;  // an empty sequence still has rows to write
        int incl = n;
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
            const int o = __shfl_up(incl, off);
            if (lane >= off) incl += o;
        }
        const int lo = base + incl - n;
        const uint64_t hit = by ? ballot64(i == slot && i < P.B) : ballot64(slot >= lo && slot < lo + n);
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

// Where a tile's 32 keys lie.  UNIFORM (page_size % 16 == 0): each 16-key block within one page, so its page
// comes by a scalar load and its base is uniform; otherwise lane l holds the page and the offset of key l % 32.
// vis: visible keys (inside the range, on a good page).
template <bool UNIFORM>
struct PagedTile {
    int64_t at[UNIFORM ? 2 : 1];
    uint32_t vis;
};
template <bool UNIFORM>
struct PagedPages {
    int page[UNIFORM ? 2 : 1];
};
typedef const __attribute__((address_space(4))) int32_t const_i32_t;  // read by scalar loads where uniform

// Page numbers of the tile at key0: only requested here, looked at a tile later.  Keys at or behind `end`
// take the place of `first`, which lies before it.
template <bool UNIFORM>
__device__ __forceinline__ PagedPages<UNIFORM> paged_pages(const PagedCache& C, const int32_t* row, int key0, int first, int end) {
    PagedPages<UNIFORM> p;
    if constexpr (UNIFORM) {
        const_i32_t* table = (const_i32_t*)(uintptr_t)row;
#pragma unroll
        for (int j = 0; j < 2; ++j) p.page[j] = table[C.by_page.div(key0 + 16 * j < end ? key0 + 16 * j : first)];
    } else {
        const int key = key0 + (threadIdx.x & 31);
        p.page[0] = row[C.by_page.div(key < end ? key : first)];
    }
    return p;
}

__device__ __forceinline__ int64_t uniform64(int64_t x) {
    const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)x), hi = __builtin_amdgcn_readfirstlane((uint32_t)((uint64_t)x >> 32));
    return (int64_t)(((uint64_t)hi << 32) | lo);
}

template <bool UNIFORM>
__device__ __forceinline__ PagedTile<UNIFORM> paged_tile(const PagedCache& C, const PagedPages<UNIFORM>& p, int64_t head, int key0,
                                                         int first, int end, bool& bad) {
    PagedTile<UNIFORM> t;
    t.vis = 0;
#pragma unroll
    for (int j = 0; j < (UNIFORM ? 2 : 1); ++j) {
        const int key = UNIFORM ? key0 + 16 * j : key0 + (int)(threadIdx.x & 31);
        const int at = key < end ? key : first;
        const bool good = p.page[j] >= 0 && p.page[j] < C.num_pages;
        bad |= !good && key < end;
        if constexpr (UNIFORM) {
            const int n = key < end && good ? (end - key < 16 ? end - key : 16) : 0;
            t.vis |= ((1u << n) - 1u) << (16 * j);
        } else {
            t.vis = (uint32_t)ballot64(good && key < end);
        }
        t.at[j] = (good ? p.page[j] : 0) * C.page_stride + (at - C.by_page.div(at) * C.page_size) * C.token_stride + head;
        if (UNIFORM) t.at[j] = uniform64(t.at[j]);
    }
    return t;
}

template <int D, int NR>
struct PagedGeom {
    static constexpr int kRows = 16 * NR;
    static constexpr int kRowF = D + 4;  // floats per row of the merge buffers: rows start 4 banks apart
    static constexpr int kKRow = D + 8;   // elements per row of a K tile: the 16 rows of a fragment read start 4 banks apart
    static constexpr int kVRow = D + 16;  // elements per row of a V tile: the 8 rows that half a wave reads of a transposing
                                          // load start 8 banks apart (72 and 40 words a row) and each takes 8 of the 64
    static constexpr int kTileBytes = kPagedTile * kVRow * 2;
    static constexpr int kMergeBytes = kRows * kRowF * 4;
    static constexpr int kWaveBytes = kTileBytes > kMergeBytes ? kTileBytes : kMergeBytes;
};

template <int D, int NR, bool UNIFORM, int DEPTH, bool ONCE>
__global__ __launch_bounds__(kPagedThreads, 2) void paged_attn_kernel(PagedAttnParams P) {
    using G = PagedGeom<D, NR>;
    constexpr int KS = D / 32;       // k steps of the scores
    constexpr int NDB = D / 16;      // head-dim blocks of the output
    constexpr int RPI = 512 / D;     // V rows per wave-wide 16-byte load
    constexpr int NVL = kPagedTile / RPI;
    __shared__ __align__(16) char lds[kPagedWaves * G::kWaveBytes];
    __shared__ float sh_m[kPagedWaves][G::kRows], sh_l[kPagedWaves][G::kRows];

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int q4 = lane >> 4, l16 = lane & 15;
    // Workgroup i runs on XCD i % 8.  The row tiles of one (slot, kv head) follow each other on one XCD, whose L2
    // they share; the (slot, kv head) pairs go round the XCDs in order, so that slots without work, the last ones,
    // leave none of them idle.
    const int turn = blockIdx.x / 8 / P.tiles, row_tile = blockIdx.x / 8 - turn * P.tiles;
    const int pair = turn * 8 + blockIdx.x % 8, slot = pair / P.Hkv, g = pair - slot * P.Hkv;
    const int unit = g * P.tiles + row_tile, tile_row = row_tile * G::kRows;
    PagedRange r;
    if (!paged_range(P, slot, false, blockIdx.x == 0, r)) return;
    const int b = r.b, len = r.len;
    const int begin = r.split * r.chunk, end = len - begin > r.chunk ? begin + r.chunk : len;

    // query fragments: row tile_row + 16 f + l16, head dims 32 ks + 8 q4 ..
    bf16x8_t qf[NR][KS];
    int limit[NR];  // keys that the row sees
#pragma unroll
    for (int f = 0; f < NR; ++f) {
        const int row = min(tile_row + 16 * f + l16, P.rows - 1);  // rows past the last repeat it and are not stored
        const int t = row / P.group, h = g * P.group + row - t * P.group;
        limit[f] = P.causal ? len - P.T + t + 1 : len;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
            qf[f][ks] = __builtin_bit_cast(bf16x8_t, ldg16(P.q + (((int64_t)b * P.T + t) * P.Hq + h) * D + 32 * ks + 8 * q4));
    }
    const int min_limit = P.causal ? len - P.T + 1 : len;

    f32x4_t o[NR][NDB];
    float m[NR], thr[NR], neg_mc[NR], lsum[NR];
#pragma unroll
    for (int f = 0; f < NR; ++f) {
        m[f] = kNegInf;
        thr[f] = kNegInf;
        neg_mc[f] = 0.f;
        lsum[f] = 0.f;
#pragma unroll
        for (int db = 0; db < NDB; ++db) o[f][db] = f32x4_t{};
    }

    uint16_t* vt = reinterpret_cast<uint16_t*>(lds + wave * G::kWaveBytes);
    const uint16_t* kread = vt + l16 * G::kKRow + 8 * q4;
    const uint16_t* vread = vt + (4 * q4 + (l16 >> 2)) * G::kVRow + 4 * (l16 & 3);
    const int vrow = lane / (D / 8), vchunk = lane % (D / 8);  // of a V load
    uint16_t* kwrite = vt + vrow * G::kKRow + 8 * vchunk;
    uint16_t* vwrite = vt + vrow * G::kVRow + 8 * vchunk;

    const PagedCache& C = P.cache;
    const int32_t* row = C.table + b * C.table_stride;
    const int64_t head = g * C.head_stride;
    const float c = P.scale_log2, lazy = kLazyLog2 / c;
    const int first = begin + wave * kPagedTile;
    u32x4_t kr[DEPTH][NVL], vr[DEPTH][NVL];
    uint32_t vis[DEPTH];
    bool bad = false;

    int voff[16 / RPI];
#pragma unroll
    for (int i = 0; i < 16 / RPI; ++i) voff[i] = 2 * ((i * RPI + vrow) * (int)C.token_stride + 8 * vchunk);
    // A tile's rows of K or V, whole 128-byte lines per load.  UNIFORM: a buffer of each block's visible rows with
    // 32-bit lane offsets, so that rows behind its end read as 0.
    auto load = [&](u32x4_t (&x)[NVL], const uint16_t* pool, const PagedTile<UNIFORM>& t) {
#pragma unroll
        for (int i = 0; i < NVL; ++i) {
            if constexpr (UNIFORM) {
                const int j = i * RPI / 16, rows = __popc(t.vis >> (16 * j) & 0xffffu);
                const auto rs = __builtin_amdgcn_make_buffer_rsrc((void*)(pool + t.at[j]), (short)0, rows * 2 * (int)C.token_stride, kBufferFlags);
                x[i] = __builtin_amdgcn_raw_buffer_load_b128(rs, voff[i % (16 / RPI)], 0, ONCE ? 2 : 0);
            } else {
                const u32x4_t* p = reinterpret_cast<const u32x4_t*>(pool + __shfl(t.at[0], i * RPI + vrow) + 8 * vchunk);
                x[i] = ONCE ? __builtin_nontemporal_load(p) : *p;
            }
        }
    };
    PagedPages<UNIFORM> pages;  // of the tile after those in flight
    // The tile at key0, held in ring slot u; with `more` also the loads of the tile DEPTH rounds behind it.
    auto step = [&](auto slot, int key0, bool more) {
        constexpr int u = decltype(slot)::value;
#pragma unroll
        for (int i = 0; i < NVL; ++i) *reinterpret_cast<u32x4_t*>(kwrite + i * RPI * G::kKRow) = kr[u][i];
        f32x4_t s[NR][2];
#pragma unroll
        for (int f = 0; f < NR; ++f)
#pragma unroll
            for (int j = 0; j < 2; ++j) s[f][j] = f32x4_t{};
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const bf16x8_t kf = lds16(kread + 16 * j * G::kKRow + 32 * ks);
#pragma unroll
                for (int f = 0; f < NR; ++f) s[f][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[f][ks], s[f][j], 0, 0, 0);
            }
        PagedTile<UNIFORM> next;
        if (more) {
            next = paged_tile<UNIFORM>(C, pages, head, key0 + DEPTH * kPagedGranule, first, end, bad);
            pages = paged_pages<UNIFORM>(C, row, key0 + (DEPTH + 1) * kPagedGranule, first, end);
            load(kr[u], C.k, next);
        }
        if (vis[u] != 0xffffffffu || key0 + kPagedTile > min_limit) {  // rare: a sequence's last tile
#pragma unroll
            for (int f = 0; f < NR; ++f)
#pragma unroll
                for (int v = 0; v < 8; ++v) {
                    const int k = 16 * (v >> 2) + 4 * q4 + (v & 3);
                    const bool seen = ((vis[u] >> k) & 1u) != 0u && key0 + k < limit[f];
                    s[f][v >> 2][v & 3] = seen ? s[f][v >> 2][v & 3] : kNegInf;
                }
            // V rows that are not visible may hold anything and count as 0 (a block's buffer ends before them)
            if constexpr (!UNIFORM) {
#pragma unroll
                for (int i = 0; i < NVL; ++i)
                    if (((vis[u] >> (i * RPI + vrow)) & 1u) == 0u) vr[u][i] = u32x4_t{};
            }
        }
        bf16x8_t pf[NR];
#pragma unroll
        for (int f = 0; f < NR; ++f) {
            float mx = s[f][0][0];
#pragma unroll
            for (int v = 1; v < 8; ++v) mx = __builtin_elementwise_maximum(mx, s[f][v >> 2][v & 3]);
            mx = quad_max(mx);
            const bool up = mx > thr[f];
            if (ballot64(up) != 0ull) {  // the reference follows the maximum in steps of at least 2^8
                const float m_new = up ? mx : m[f];
                const float alpha = up ? fast_exp2((m[f] - m_new) * c) : 1.0f;  // 0 at the first reference
                lsum[f] *= alpha;
#pragma unroll
                for (int db = 0; db < NDB; ++db) o[f][db] *= alpha;
                m[f] = m_new;
                thr[f] = m_new + lazy;
                neg_mc[f] = m_new == kNegInf ? 0.f : -m_new * c;
            }
#pragma unroll
            for (int v = 0; v < 8; ++v) {
                const float p = fast_exp2(__builtin_fmaf(s[f][v >> 2][v & 3], c, neg_mc[f]));
                lsum[f] += p;
                pf[f][v] = (__bf16)p;
            }
        }
#pragma unroll
        for (int i = 0; i < NVL; ++i) {
            *reinterpret_cast<u32x4_t*>(vwrite + i * RPI * G::kVRow) = vr[u][i];
        }
        if (more) {
            load(vr[u], C.v, next);
            vis[u] = next.vis;
        }
#pragma unroll
        for (int db = 0; db < NDB; ++db) {
            const bf16x4_t a0 = lds_read_tr(vread + 16 * db);
            const bf16x4_t a1 = lds_read_tr(vread + 16 * db + 16 * G::kVRow);
            const bf16x8_t va = __builtin_shufflevector(a0, a1, 0, 1, 2, 3, 4, 5, 6, 7);
#pragma unroll
            for (int f = 0; f < NR; ++f) o[f][db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va, pf[f], o[f][db], 0, 0, 0);
        }
    };

    int left = first < end ? (end - first + kPagedGranule - 1) / kPagedGranule : 0;  // tiles of this wave
    if (left > 0) {
        using Slot0 = std::integral_constant<int, 0>;
        using Slot1 = std::integral_constant<int, DEPTH - 1>;
        auto fetch = [&](int u) { return paged_pages<UNIFORM>(C, row, first + u * kPagedGranule, first, end); };
        auto request = [&](auto slot, const PagedPages<UNIFORM>& p) {
            constexpr int u = decltype(slot)::value;
            const PagedTile<UNIFORM> t = paged_tile<UNIFORM>(C, p, head, first + u * kPagedGranule, first, end, bad);
            vis[u] = t.vis;
            load(kr[u], C.k, t);
            load(vr[u], C.v, t);
        };
        const PagedPages<UNIFORM> p0 = fetch(0), p1 = fetch(DEPTH - 1);
        pages = fetch(DEPTH);
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

    // waves -> workgroup
    __syncthreads();
    float* mine = reinterpret_cast<float*>(lds + wave * G::kWaveBytes);
#pragma unroll
    for (int f = 0; f < NR; ++f) {
        const float l = quad_sum(lsum[f]);
        if (q4 == 0) {
            sh_m[wave][16 * f + l16] = m[f];
            sh_l[wave][16 * f + l16] = l;
        }
#pragma unroll
        for (int db = 0; db < NDB; ++db) *reinterpret_cast<f32x4_t*>(mine + (16 * f + l16) * G::kRowF + 16 * db + 4 * q4) = o[f][db];
    }
    __syncthreads();
    for (int i = threadIdx.x; i < G::kRows * (D / 4); i += kPagedThreads) {
        const int rr = i / (D / 4), d = 4 * (i % (D / 4));
        const int qrow = tile_row + rr;
        if (qrow >= P.rows) continue;
        float M = kNegInf;
#pragma unroll
        for (int w = 0; w < kPagedWaves; ++w) M = fmaxf(M, sh_m[w][rr]);
        const float Ms = M == kNegInf ? 0.f : M;
        f32x4_t acc = {};
        float l = 0.f;
#pragma unroll
        for (int w = 0; w < kPagedWaves; ++w) {
            const float e = fast_exp2((sh_m[w][rr] - Ms) * c);  // 0 for a wave without keys
            l += e * sh_l[w][rr];
            acc += e * *reinterpret_cast<const f32x4_t*>(lds + w * G::kWaveBytes + (rr * G::kRowF + d) * 4);
        }
        if (r.n == 1) {
            const float inv = l > 0.f ? 1.0f / l : 0.f;  // a row that sees nothing: 0
            const int t = qrow / P.group, h = g * P.group + qrow - t * P.group;
            u32x2_t w2;
            w2[0] = (uint32_t)f2bf(acc[0] * inv) | ((uint32_t)f2bf(acc[1] * inv) << 16);
            w2[1] = (uint32_t)f2bf(acc[2] * inv) | ((uint32_t)f2bf(acc[3] * inv) << 16);
            *reinterpret_cast<u32x2_t*>(P.out + (((int64_t)b * P.T + t) * P.Hq + h) * D + d) = w2;
        } else {
            const int64_t at = ((int64_t)slot * P.units + unit) * G::kRows + rr;
            *reinterpret_cast<f32x4_t*>(P.part_o + at * D + d) = acc;
            if (d == 0) {
                P.part_ml[2 * at] = M;
                P.part_ml[2 * at + 1] = l;
            }
        }
    }
}

// THREADS threads per (sequence, new token, query head): each range by D / 4 lanes, THREADS * 4 / D ranges at a time,
// every group with its own running maximum, joined through LDS in the groups' order.  Sequences in one range were
// written by the attention itself.
template <int D, int NR, int THREADS>
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
    PagedRange r{};
    paged_range(P, b, true, false, r);
    const int g = h / P.group, qrow = t * P.group + h - g * P.group;
    const int unit = g * P.tiles + qrow / (16 * NR), rr = qrow % (16 * NR);
    const int64_t at0 = ((int64_t)r.slot0 * P.units + unit) * (16 * NR) + rr, step = (int64_t)P.units * (16 * NR);
    const int grp = tid / LPR, d = tid % LPR;
    const int n = r.n > 1 ? r.n : 0;
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
