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
};

// A workgroup takes `tokens` cache rows (whole scale blocks, at most ROWS) of a sequence: page numbers, angles' sines and
// cosines go to LDS once, then each wave takes a head of q, K or V at a time.  A lane holds 8 values of a row's first half
// and the matching 8 of its second, a wave ROWS rows; a block's largest magnitude is found by lane exchanges and an LDS
// maximum per wave.  Rows that the first block held before are rounded again if the block's scale grows (rare: read only
// then).  Bound by the copy: (4 Hq + 6 Hkv) D bytes per token.
// grid: x = groups of rows from the block that holds the first token, y shares the heads out, z = sequence.
template <int D, int ROWS>
__global__ __launch_bounds__(kAppendThreads) void paged8_append_kernel(Append8Params P) {
    constexpr int HALF = D / 2, LPR = D / 16, RPS = 64 / LPR, STEPS = ROWS / RPS, WAVES = kAppendThreads / 64;
    __shared__ float cs[ROWS][HALF], sn[ROWS][HALF];
    __shared__ int64_t sh_row[ROWS];    // the row's place in the pools; -1: none
    __shared__ int64_t sh_scale[ROWS];  // of the row's block, head 0
    __shared__ uint32_t sh_max[WAVES][ROWS];
    const int b = blockIdx.z, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
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
    const int t0 = (int)blockIdx.x * P.tokens - lead;  // of the workgroup's first row, as a token of the call
    if (t0 >= n) return;
    const int rows = min(P.tokens, n - t0);
    const int first = t0 < 0 ? -t0 : 0;  // the first row that is the call's
    if (tid < rows) {
        const int64_t at = (int64_t)start + t0 + tid;
        int64_t row = -1, scale = 0;
        if (at >= 0 && at < P.cache.capacity) {
            const int col = P.cache.by_page.div((int)at), in = (int)at - col * P.cache.page_size;
            const int page = P.cache.table[b * P.cache.table_stride + col];
            if (page >= 0 && page < P.cache.num_pages) {
                row = page * P.cache.page_stride + in * P.cache.token_stride;
                scale = ((int64_t)page * P.c8.blocks + P.c8.by_block.div(in)) * P.Hkv;
            } else if (blockIdx.y == 0 && tid >= first) {
                flag_device_status(kDevBadPage);
            }
        }
        sh_row[tid] = row;
        sh_scale[tid] = scale;
    }
    if (P.rotate) {
        const int64_t pos0 = (int64_t)(P.pos0 != nullptr ? P.pos0[b] : start) + t0;
        for (int i = first * HALF + tid; i < rows * HALF; i += kAppendThreads) {
            const int r = i / HALF, d = i % HALF;
            const double turn = (double)(pos0 + r) * P.turns[d];
            sincospif(2.0f * (float)(turn - floor(turn)), &sn[r][d], &cs[r][d]);
        }
    }
    __syncthreads();
    const int qh = P.q != nullptr ? P.Hq : 0;
    const int d0 = 8 * (lane % LPR);
    const int64_t token0 = (int64_t)b * P.T + t0;
    for (int unit = (int)blockIdx.y * WAVES + wave; unit < qh + 2 * P.Hkv; unit += (int)gridDim.y * WAVES) {
        const bool query = unit < qh, key = unit < qh + P.Hkv;
        const int head = query ? unit : unit - qh - (key ? 0 : P.Hkv);
        const uint16_t* src = (query ? P.q : key ? P.k : P.v) + head * D + d0;
        const int64_t src_row = query ? P.q_row : key ? P.k_row : P.v_row;
        uint8_t* scales = (key ? P.c8.k_scale : P.c8.v_scale) + head;
        u32x4_t lo[STEPS], hi[STEPS];
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
            const int r = s * RPS + lane / LPR;
            const bool mine = r >= first && r < rows;
            lo[s] = hi[s] = u32x4_t{};
            if (mine) {
                const uint16_t* p = src + (token0 + r) * src_row;
                lo[s] = ldg16(p);
                hi[s] = ldg16(p + HALF);
            }
        }
        // the first block's scale where it holds rows from before
        const bool kept = !query && first > 0 && sh_row[0] >= 0;
        const uint32_t old = kept ? min(max((uint32_t)scales[sh_scale[0]], kScaleLowest), kScaleHighest) : 0u;
        float x[STEPS][16];
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
            const int r = s * RPS + lane / LPR;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float a = e % 2 == 0 ? bf16_lo(lo[s][e / 2]) : bf16_hi(lo[s][e / 2]);
                const float c = e % 2 == 0 ? bf16_lo(hi[s][e / 2]) : bf16_hi(hi[s][e / 2]);
                x[s][e] = a;
                x[s][8 + e] = c;
                if (P.rotate && key) {
                    const float co = cs[r][d0 + e], si = sn[r][d0 + e];
                    x[s][e] = a * co - c * si;
                    x[s][8 + e] = c * co + a * si;
                }
            }
        }
        if (query) {
#pragma unroll
            for (int s = 0; s < STEPS; ++s) {
                const int r = s * RPS + lane / LPR;
                if (r < first || r >= rows) continue;
                u32x4_t o[2];
#pragma unroll
                for (int e = 0; e < 8; ++e) o[e / 4][e % 4] = (uint32_t)f2bf(x[s][2 * e]) | ((uint32_t)f2bf(x[s][2 * e + 1]) << 16);
                uint16_t* dst = P.q_out + ((token0 + r) * P.Hq + head) * D + d0;
                *reinterpret_cast<u32x4_t*>(dst) = o[0];
                *reinterpret_cast<u32x4_t*>(dst + HALF) = o[1];
            }
            continue;
        }
        uint32_t* most = sh_max[wave];
        if (lane < ROWS) most[lane] = 0u;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
            const int r = s * RPS + lane / LPR;
            uint32_t m = 0u;
#pragma unroll
            for (int e = 0; e < 16; ++e) m = max(m, magnitude_bits(x[s][e]));
#pragma unroll
            for (int t = 0; t < (LPR == 8 ? 3 : 2); ++t) m = max(m, (uint32_t)__shfl_xor((int)m, 1 << t));
            if (lane % LPR == 0 && r >= first && r < rows) atomicMax(&most[P.c8.by_block.div(r)], m);
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        uint8_t* pool = (key ? P.c8.k : P.c8.v) + head * P.cache.head_stride + d0;
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
            const int r = s * RPS + lane / LPR;
            if (r >= rows || sh_row[r] < 0) continue;
            const int block = P.c8.by_block.div(r);
            uint32_t byte = scale_byte(most[block]);
            if (block == 0) byte = max(byte, old);
            uint8_t* dst = pool + sh_row[r];
            if (r >= first) {
                const float inv = scale_inverse(byte);
                u32x2_t a, c;
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    a[e] = pack_e4m3(x[s][4 * e] * inv, x[s][4 * e + 1] * inv, x[s][4 * e + 2] * inv, x[s][4 * e + 3] * inv);
                    c[e] = pack_e4m3(x[s][8 + 4 * e] * inv, x[s][9 + 4 * e] * inv, x[s][10 + 4 * e] * inv, x[s][11 + 4 * e] * inv);
                }
                *reinterpret_cast<u32x2_t*>(dst) = a;
                *reinterpret_cast<u32x2_t*>(dst + HALF) = c;
                if (lane % LPR == 0 && r == max(first, block * P.c8.sb)) scales[sh_scale[r]] = (uint8_t)byte;
            } else if (byte > old) {
                // 2^(old - byte): exact but for what falls into the subnormals, or below them
                const float down = byte - old < kScaleOne ? scale_value(kScaleOne - (byte - old)) : 0.f;
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
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
}

// ------------------------------------------------------------------ attention
struct Paged8AttnParams : PagedAttnParams {
    Paged8Cache c8;
};

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

// Loaded rows to LDS as bf16, times their scales (lane l of `scale` has key l's).  Rows that are not in vis count as 0:
// neither their values nor their scales need to be anything.
template <int D, int BLK, int ROW>
__device__ __forceinline__ void paged8_put(uint16_t* to, const u32x4_t (&x)[BLK * D / 64], uint64_t vis, uint32_t scale) {
    constexpr int RPI = 1024 / D;
    const int lane = threadIdx.x & 63, vrow = lane / (D / 16), vchunk = lane % (D / 16);
#pragma unroll
    for (int i = 0; i < BLK * D / 64; ++i) {
        const int row = i * RPI + vrow;
        const bool seen = ((vis >> row) & 1ull) != 0ull;
        const uint32_t byte = (uint32_t)__shfl((int)scale, row);
        u32x4_t lo, hi;
        unpack_e4m3(seen ? x[i] : u32x4_t{}, scale_value(seen ? byte : kScaleOne), lo, hi);
        uint16_t* p = to + row * ROW + 16 * vchunk;
        *reinterpret_cast<u32x4_t*>(p) = lo;
        *reinterpret_cast<u32x4_t*>(p + 8) = hi;
    }
}

// Up to 32 rows: the waves take the range's tiles of 32 NK keys in turn, DEPTH tiles in flight each.
template <int D, int NR, bool UNIFORM, int NK, int DEPTH>
__global__ __launch_bounds__(kPagedThreads, 2) void paged8_attn_kernel(Paged8AttnParams P) {
    using L = PagedLds<D>;
    constexpr int ROWS = 16 * NR, KEYS = 32 * NK, BLK = 2 * NK, NVL = BLK * D / 64, ROUND = kPagedWaves * KEYS;
    constexpr int kTileBytes = KEYS * L::kVRow * 2, kMergeBytes = ROWS * L::kMergeRow * 4;
    constexpr int kTiles = kPagedWaves * kTileBytes, kMerge = kPagedWaves * kMergeBytes;
    constexpr uint64_t kAll = KEYS == 64 ? ~0ull : (1ull << (KEYS & 63)) - 1ull;
    __shared__ __align__(16) char lds[kTiles > kMerge ? kTiles : kMerge];
    __shared__ float sh_m[kPagedWaves * ROWS], sh_l[kPagedWaves * ROWS];

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const PagedPlace w = paged_place(P);
    PagedRange r;
    if (!paged_range<ROUND>(P, w, r)) return;
    const int len = r.len;
    const int begin = r.split * r.chunk, end = len - begin > r.chunk ? begin + r.chunk : len;
    const int n_new = paged_new(P, r.b, w.unit == 0 && r.split == 0 && threadIdx.x == 0);
    const int min_limit = P.causal ? len - n_new + 1 : len;  // of a row that is not padding

    uint16_t* tile = reinterpret_cast<uint16_t*>(lds + wave * kTileBytes);  // K's and then V's
    const PagedCache& C = P.cache;
    const int ts = (int)C.token_stride;
    const int32_t* row = C.table + r.b * C.table_stride;
    const float c = P.scale_log2;
    const int first = begin + wave * KEYS;
    u32x4_t kr[DEPTH][NVL], vr[DEPTH][NVL];
    uint64_t vis[DEPTH];
    uint32_t ks[DEPTH], vs[DEPTH];
    bool bad = false;
    using Tile = Paged8Tile<UNIFORM, BLK>;
    using Pages = PagedPages<UNIFORM, BLK>;
    PagedRows<D, NR> st;
    Pages pages;  // of the tile after those in flight
    // The tile at key0, held in ring slot u; with `more` also the loads of the tile DEPTH rounds behind it.
    auto step = [&](auto slot, int key0, bool more) {
        constexpr int u = decltype(slot)::value;
        paged8_put<D, BLK, L::kKRow>(tile, kr[u], vis[u], ks[u]);
        f32x4_t s[NR][2 * NK];
        st.template scores<NK>(tile, s);
        Tile next;
        if (more) {
            next = paged8_tile<UNIFORM, BLK>(P, pages, w.g, key0 + DEPTH * ROUND, first, end, bad);
            pages = paged_pages<UNIFORM, BLK>(C, row, key0 + (DEPTH + 1) * ROUND, first, end);
            paged8_load<D, UNIFORM, BLK, true>(kr[u], P.c8.k, next, ts);
        }
        if (vis[u] != kAll || key0 + KEYS > min_limit) st.template mask<NK>(s, vis[u], key0);  // rare: a sequence's last tile
        bf16x8_t pf[2][NR][NK];
        st.template weights<NK>(s, c, pf);
        paged8_put<D, BLK, L::kVRow>(tile, vr[u], vis[u], vs[u]);
        if (more) {
            paged8_load<D, UNIFORM, BLK, true>(vr[u], P.c8.v, next, ts);
            vis[u] = next.vis;
            ks[u] = next.ks;
            vs[u] = next.vs;
        }
        __builtin_amdgcn_sched_barrier(0);  // the next tile's products stay behind this one's: registers
        st.template values<NK>(tile, pf);
        __builtin_amdgcn_sched_barrier(0);
    };

    auto fetch = [&](int u) { return paged_pages<UNIFORM, BLK>(C, row, first + u * ROUND, first, end); };
    Pages p0{}, p1{};
    if (first < end) {
        p0 = fetch(0);
        p1 = fetch(DEPTH - 1);
        pages = fetch(DEPTH);
    }
    st.init(P, r.b, w.g, len, n_new, w.row_tile * ROWS);
    int left = first < end ? (end - first + ROUND - 1) / ROUND : 0;  // tiles of this wave
    if (left > 0) {
        using Slot0 = std::integral_constant<int, 0>;
        using Slot1 = std::integral_constant<int, DEPTH - 1>;
        auto request = [&](auto slot, const Pages& p) {
            constexpr int u = decltype(slot)::value;
            const Tile t = paged8_tile<UNIFORM, BLK>(P, p, w.g, first + u * ROUND, first, end, bad);
            vis[u] = t.vis;
            ks[u] = t.ks;
            vs[u] = t.vs;
            paged8_load<D, UNIFORM, BLK, true>(kr[u], P.c8.k, t, ts);
            paged8_load<D, UNIFORM, BLK, true>(vr[u], P.c8.v, t, ts);
        };
        int key0 = first;
        // No load under a condition ahead of the loop: the compiler's waits count the loads that every path issued.
        if constexpr (DEPTH == 1) {
            request(Slot0{}, p0);
            for (; left > 1; --left, key0 += ROUND) step(Slot0{}, key0, true);
            step(Slot0{}, key0, false);
        } else if (left == 1) {
            request(Slot0{}, p0);
            step(Slot0{}, key0, false);
        } else {
            request(Slot0{}, p0);
            request(Slot1{}, p1);
            for (; left > 3; left -= 2, key0 += 2 * ROUND) {
                step(Slot0{}, key0, true);
                step(Slot1{}, key0 + ROUND, true);
            }
            if (left > 2) {
                step(Slot0{}, key0, true);
                step(Slot1{}, key0 + ROUND, false);
                step(Slot0{}, key0 + 2 * ROUND, false);
            } else {
                step(Slot0{}, key0, false);
                step(Slot1{}, key0 + ROUND, false);
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

// More rows: RW waves of 32 rows each share the stages of 16 RW keys that they load into LDS together; 4 / RW such groups
// of waves take the range's stages in turn.  While a stage is multiplied the next one lies in registers on its way to the
// other buffer.
template <int D, int RW, bool UNIFORM, bool ONCE>
__global__ __launch_bounds__(kPagedThreads, 2) void paged8_rows_kernel(Paged8AttnParams P) {
    using L = PagedLds<D>;
    constexpr int NR = 2, KW = kPagedWaves / RW, ROWS = 32 * RW, STAGE = 16 * RW, NK = STAGE / 32, NVL = D / 64;
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
        paged8_put<D, 1, L::kKRow>(k + 16 * rw * L::kKRow, kr, vis, ks);
        paged8_put<D, 1, L::kVRow>(k + STAGE * L::kKRow + 16 * rw * L::kVRow, vr, vis, vs);
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

}  // namespace trajspec
