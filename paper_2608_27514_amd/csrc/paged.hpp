// The paged key-value cache: pages of `page_size` tokens in one pool, a table of page numbers per
// sequence (token s of sequence b lies in page table[b][s / page_size], row s % page_size), and per-sequence
// lengths that only the device knows.
//   paged_append_kernel   rotates the new tokens' queries and keys by position and writes keys and values
//                         into the pages
//   paged_attn_kernel     attention of the new tokens over their sequences' cached keys
//   paged_join_kernel     joins the partial results of sequences whose keys were split over workgroups
#pragma once

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
// running softmax state, merged through LDS at the end.  A step reads every cached key and value once and does
// T Hq / Hkv multiply-adds per element read, so up to some hundreds of rows the stream of K and V bounds it:
// rows are padded to 16 for the matrix core, which idles either way.
//   S^T = K Q^T with K fragments loaded straight from the pages into the A operand (no wave shares another's
//   keys); V goes through the wave's own LDS tile for the transposing reads of O^T += V^T P^T (layouts of
//   the 16-row verification kernel).  The next tile's K loads are issued behind the score MFMAs and its V
//   loads behind the LDS writes, so one tile of each is always in flight; page numbers are fetched a tile earlier.
//
// Splits: the device computes from the lengths how many keys a workgroup takes (`chunk`), so that the batch makes
// about kPagedTargetWgs workgroups whatever the lengths are; slot = index of a (sequence, range) pair in order.
constexpr int kPagedWaves = 4;
constexpr int kPagedThreads = kPagedWaves * 64;
constexpr int kPagedTile = 32;
constexpr int kPagedChunkMin = kPagedWaves * kPagedTile;
constexpr int kPagedTargetWgs = 1024;

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

// Keys per workgroup: the batch's keys times units over the target, in whole rounds of the waves' tiles.
// Every wave computes the same from the same lengths (whole numbers; the quotient by a power of two is exact).
__device__ __forceinline__ int paged_chunk(int64_t total, int units, int capacity) {
    const double per = (double)total * (double)units / (double)(kPagedTargetWgs * kPagedChunkMin);
    const double most = (double)(capacity / kPagedChunkMin + 1);
    const int rounds = (int)ceil(per < most ? per : most);
    return kPagedChunkMin * (rounds < 1 ? 1 : rounds);
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

// Where a tile's 32 keys lie.  UNIFORM (page_size % 16 == 0): each 16-key block within one page, so its base is
// uniform; otherwise lane l holds the offset of key l % 32.  vis: visible keys (inside the range, on a good page).
template <bool UNIFORM>
struct PagedTile;
template <>
struct PagedTile<true> {
    int64_t base[2];
    uint32_t vis;
};
template <>
struct PagedTile<false> {
    int64_t off;
    uint32_t vis;
};

template <bool UNIFORM>
__device__ __forceinline__ PagedTile<UNIFORM> paged_tile(const PagedCache& C, const int32_t* row, int64_t head, int key0, int end) {
    PagedTile<UNIFORM> t;
    if constexpr (UNIFORM) {
        t.vis = 0;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int key = key0 + 16 * j;
            const int at = key < end ? key : key0;  // a block behind the end reads the first one's rows
            const int col = C.by_page.div(at);
            int page = __builtin_amdgcn_readfirstlane(row[col]);
            const bool good = page >= 0 && page < C.num_pages;
            if (!good) page = 0;
            const int n = key < end && good ? (end - key < 16 ? end - key : 16) : 0;
            t.vis |= ((1u << n) - 1u) << (16 * j);
            if (!good && key < end && (threadIdx.x & 63) == 0) flag_device_status(kDevBadPage);
            t.base[j] = page * C.page_stride + (at - col * C.page_size) * C.token_stride + head;
        }
    } else {
        const int key = key0 + (threadIdx.x & 31);
        const int at = key < end ? key : key0;
        const int col = C.by_page.div(at);
        int page = row[col];
        const bool good = page >= 0 && page < C.num_pages;
        if (!good) page = 0;
        if (!good && key < end) flag_device_status(kDevBadPage);
        t.vis = (uint32_t)ballot64(good && key < end);
        t.off = page * C.page_stride + (at - col * C.page_size) * C.token_stride + head;
    }
    return t;
}

template <int D, int NR>
struct PagedGeom {
    static constexpr int kRows = 16 * NR;
    static constexpr int kRowF = D + 4;  // floats per row of the merge buffers: rows start 4 banks apart
    static constexpr int kTileBytes = kPagedTile * D * 2;
    static constexpr int kMergeBytes = kRows * kRowF * 4;
    static constexpr int kWaveBytes = kTileBytes > kMergeBytes ? kTileBytes : kMergeBytes;
};

template <int D, int NR, bool UNIFORM>
__global__ __launch_bounds__(kPagedThreads) void paged_attn_kernel(PagedAttnParams P) {
    using G = PagedGeom<D, NR>;
    using AG = AttnGeom<D, 16>;
    constexpr int KS = D / 32;       // k steps of the scores
    constexpr int NDB = D / 16;      // head-dim blocks of the output
    constexpr int RPI = 512 / D;     // V rows per wave-wide 16-byte load
    constexpr int NVL = kPagedTile / RPI;
    __shared__ __align__(16) char lds[kPagedWaves * G::kWaveBytes];
    __shared__ float sh_m[kPagedWaves][G::kRows], sh_l[kPagedWaves][G::kRows];

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int q4 = lane >> 4, l16 = lane & 15;
    const int id = xcd_logical_id(blockIdx.x, gridDim.x);
    const int slot = id / P.units, unit = id - slot * P.units;
    const int g = unit / P.tiles, tile_row = (unit - g * P.tiles) * G::kRows;
    PagedRange r;
    if (!paged_range(P, slot, false, id == 0, r)) return;
    const int b = r.b, len = r.len;
    const int begin = r.split * r.chunk, end = len - begin > r.chunk ? begin + r.chunk : len;

    // query fragments: row tile_row + 16 f + l16, head dims 32 ks + 8 q4 ..
    bf16x8_t qf[NR][KS];
    int limit[NR];  // keys that the row sees
#pragma unroll
    for (int f = 0; f < NR; ++f) {
        const int row = tile_row + 16 * f + l16;
        const int t = row / P.group, h = g * P.group + row - t * P.group;
        limit[f] = P.causal ? len - P.T + t + 1 : len;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            qf[f][ks] = bf16x8_t{};
            if (row < P.rows) qf[f][ks] = __builtin_bit_cast(bf16x8_t, ldg16(P.q + (((int64_t)b * P.T + t) * P.Hq + h) * D + 32 * ks + 8 * q4));
        }
    }
    const int min_limit = P.causal ? len - P.T + 1 : len;

    f32x4_t o[NR][NDB];
    float m[NR], neg_mc[NR], lsum[NR];
#pragma unroll
    for (int f = 0; f < NR; ++f) {
        m[f] = kNegInf;
        neg_mc[f] = 0.f;
        lsum[f] = 0.f;
#pragma unroll
        for (int db = 0; db < NDB; ++db) o[f][db] = f32x4_t{};
    }

    uint16_t* vt = reinterpret_cast<uint16_t*>(lds + wave * G::kWaveBytes);
    int vq[NDB];
    {
        const int vr = 4 * q4 + (l16 >> 2);
#pragma unroll
        for (int db = 0; db < NDB; ++db) {
            const int chunk = 2 * db + ((l16 & 3) >> 1);
            vq[db] = vr * D + ((chunk ^ AG::v_rot(vr)) << 3) + (l16 & 1) * 4;
        }
    }
    const int vrow = lane / (D / 8), vchunk = lane % (D / 8);  // of a V load

    const PagedCache& C = P.cache;
    const int32_t* row = C.table + b * C.table_stride;
    const int64_t head = g * C.head_stride;
    const float c = P.scale_log2;
    u32x4_t kr[2][KS], vr[NVL];

    auto load_k = [&](const PagedTile<UNIFORM>& t) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const uint16_t* p;
            if constexpr (UNIFORM)
                p = C.k + t.base[j] + (l16 * (int)C.token_stride + 8 * q4);
            else
                p = C.k + __shfl(t.off, 16 * j + l16) + 8 * q4;
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) kr[j][ks] = ldg16(p + 32 * ks);
        }
    };
    auto load_v = [&](const PagedTile<UNIFORM>& t) {
#pragma unroll
        for (int i = 0; i < NVL; ++i) {
            if constexpr (UNIFORM)
                vr[i] = ldg16(C.v + t.base[i * RPI / 16] + (((i * RPI) % 16 + vrow) * (int)C.token_stride + 8 * vchunk));
            else
                vr[i] = ldg16(C.v + __shfl(t.off, i * RPI + vrow) + 8 * vchunk);
        }
    };
    // one tile; `next`: the tile whose loads it issues, if there is one
    auto step = [&](int key0, uint32_t vis, bool more, const PagedTile<UNIFORM>& next) {
        f32x4_t s[NR][2];
#pragma unroll
        for (int f = 0; f < NR; ++f)
#pragma unroll
            for (int j = 0; j < 2; ++j) s[f][j] = f32x4_t{};
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int f = 0; f < NR; ++f)
                    s[f][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, kr[j][ks]), qf[f][ks], s[f][j], 0, 0, 0);
        if (more) load_k(next);
        const bool whole = vis == 0xffffffffu && key0 + kPagedTile <= min_limit;
        bf16x8_t pf[NR];
#pragma unroll
        for (int f = 0; f < NR; ++f) {
            if (!whole) {
#pragma unroll
                for (int v = 0; v < 8; ++v) {
                    const int k = 16 * (v >> 2) + 4 * q4 + (v & 3);
                    const bool seen = ((vis >> k) & 1u) != 0u && key0 + k < limit[f];
                    s[f][v >> 2][v & 3] = seen ? s[f][v >> 2][v & 3] : kNegInf;
                }
            }
            float mx = kNegInf;
#pragma unroll
            for (int v = 0; v < 8; ++v) mx = fmaxf(mx, s[f][v >> 2][v & 3]);
            mx = quad_max(mx);
            const bool up = mx > m[f];
            if (ballot64(up) != 0ull) {
                const float m_new = up ? mx : m[f];
                const float alpha = up ? fast_exp2((m[f] - m_new) * c) : 1.0f;  // 0 from the first reference on
                lsum[f] *= alpha;
#pragma unroll
                for (int db = 0; db < NDB; ++db) o[f][db] *= alpha;
                m[f] = m_new;
                neg_mc[f] = m_new == kNegInf ? 0.f : -m_new * c;
            }
#pragma unroll
            for (int v = 0; v < 8; ++v) {
                const float p = fast_exp2(__builtin_fmaf(s[f][v >> 2][v & 3], c, neg_mc[f]));
                lsum[f] += p;
                pf[f][v] = (__bf16)p;
            }
        }
        // V into the wave's tile; rows that are not visible may hold anything and count as 0
#pragma unroll
        for (int i = 0; i < NVL; ++i) {
            const int rr = i * RPI + vrow;
            u32x4_t x = vr[i];
            if (vis != 0xffffffffu && ((vis >> rr) & 1u) == 0u) x = u32x4_t{};
            *reinterpret_cast<u32x4_t*>(vt + rr * D + ((vchunk ^ AG::v_rot(rr & 15)) << 3)) = x;
        }
        if (more) load_v(next);
#pragma unroll
        for (int db = 0; db < NDB; ++db) {
            const bf16x4_t a0 = lds_read_tr(vt + vq[db]);
            const bf16x4_t a1 = lds_read_tr(vt + vq[db] + 16 * D);
            const bf16x8_t va = __builtin_shufflevector(a0, a1, 0, 1, 2, 3, 4, 5, 6, 7);
#pragma unroll
            for (int f = 0; f < NR; ++f) o[f][db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va, pf[f], o[f][db], 0, 0, 0);
        }
    };

    int key0 = begin + wave * kPagedTile;
    if (key0 < end) {
        PagedTile<UNIFORM> cur = paged_tile<UNIFORM>(C, row, head, key0, end);
        load_k(cur);
        load_v(cur);
        PagedTile<UNIFORM> nxt = cur;
        if (key0 + kPagedChunkMin < end) nxt = paged_tile<UNIFORM>(C, row, head, key0 + kPagedChunkMin, end);
        while (key0 + kPagedChunkMin < end) {
            const PagedTile<UNIFORM> now = cur;
            cur = nxt;
            if (key0 + 2 * kPagedChunkMin < end) nxt = paged_tile<UNIFORM>(C, row, head, key0 + 2 * kPagedChunkMin, end);
            step(key0, now.vis, true, cur);
            key0 += kPagedChunkMin;
        }
        step(key0, cur.vis, false, cur);
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

// One workgroup per (sequence, new token, query head): 8 (D = 128) or 16 (D = 64) ranges at a time, each by D / 4
// lanes, joined through LDS.  Sequences in one range were written by the attention itself.
template <int D, int NR>
__global__ __launch_bounds__(kPagedThreads) void paged_join_kernel(PagedAttnParams P) {
    constexpr int LPR = D / 4, GR = kPagedThreads / LPR;
    __shared__ f32x4_t sh_o[GR][LPR];
    __shared__ float sh_w[kPagedWaves][2];
    __shared__ float sh_l[GR];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t orow = blockIdx.x;
    const int h = (int)(orow % P.Hq);
    const int64_t bt = orow / P.Hq;
    const int b = (int)(bt / P.T), t = (int)(bt - (int64_t)b * P.T);
    PagedRange r;
    if (!paged_range(P, b, true, false, r) || r.n <= 1) return;
    const int g = h / P.group, qrow = t * P.group + h - g * P.group;
    const int unit = g * P.tiles + qrow / (16 * NR), rr = qrow % (16 * NR);
    auto at = [&](int s) { return ((int64_t)(r.slot0 + s) * P.units + unit) * (16 * NR) + rr; };
    // the joint maximum
    float M = kNegInf;
    for (int s = threadIdx.x; s < r.n; s += kPagedThreads) M = fmaxf(M, P.part_ml[2 * at(s)]);
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) M = fmaxf(M, __shfl_xor(M, off));
    if (lane == 0) sh_w[wave][0] = M;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kPagedWaves; ++w) M = fmaxf(M, sh_w[w][0]);
    const float Ms = M == kNegInf ? 0.f : M;
    const int grp = threadIdx.x / LPR, d = threadIdx.x % LPR;
    f32x4_t acc = {};
    float l = 0.f;
    for (int s = grp; s < r.n; s += GR) {
        const int64_t a = at(s);
        const float e = fast_exp2((P.part_ml[2 * a] - Ms) * P.scale_log2);
        l += e * P.part_ml[2 * a + 1];
        acc += e * *reinterpret_cast<const f32x4_t*>(P.part_o + a * D + 4 * d);
    }
    sh_o[grp][d] = acc;
    if (d == 0) sh_l[grp] = l;
    __syncthreads();
    if (grp != 0) return;
    l = 0.f;
    acc = f32x4_t{};
#pragma unroll
    for (int w = 0; w < GR; ++w) {
        l += sh_l[w];
        acc += sh_o[w][d];
    }
    const float inv = l > 0.f ? 1.0f / l : 0.f;
    u32x2_t w2;
    w2[0] = (uint32_t)f2bf(acc[0] * inv) | ((uint32_t)f2bf(acc[1] * inv) << 16);
    w2[1] = (uint32_t)f2bf(acc[2] * inv) | ((uint32_t)f2bf(acc[3] * inv) << 16);
    *reinterpret_cast<u32x2_t*>(P.out + orow * D + 4 * d) = w2;
}

}  // namespace trajspec
