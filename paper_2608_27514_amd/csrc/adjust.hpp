// Confidences and top-k candidates of logits under each request's penalties, biases and grammar mask, without
// writing the adjusted logits anywhere.  For the row's sequence, token v and c = times v occurs in its history:
//     x = logit;  c > 0: x = (x > 0 ? x / r : x * r) - (f c + p);  x += sum of v's biases;  forbidden: x = -inf
// then the maximum, the sum of exp(x - max) and the k largest of x as in conf_topk.hpp.
//
// Few tokens of the vocabulary are in a history or a bias list (at most H + NB of V).  adjust_prepare_kernel
// turns a sequence's lists into a bitmap of these "special" tokens and, in the order of their ids, one
// record each of whether the token was seen and of what is added to it.  adjust_topk_kernel streams a row with
// the special and the forbidden tokens masked out (one bit per token, staged in LDS), then gathers the special
// ones by their records.  So the stream's cost does not depend on the lists, and every sum runs in a fixed order.
#pragma once

#include <algorithm>

#include "conf_topk.hpp"
#include "layer.hpp"

namespace trajspec {

constexpr int kDevBadMask = 0x40;    // TRAJ_DEV_BAD_MASK
constexpr int kDevBadHistory = 0x80; // TRAJ_DEV_BAD_HISTORY

constexpr int kAdjustMaxVocab = 1 << 19;  // a bit per token and two bytes per 32 of them in LDS: 96 KB
constexpr int kAdjustPrepThreads = 1024;
constexpr int kAdjustGroup = 512;         // tokens per popcount prefix
constexpr int kAdjustLds = 144 << 10;      // of adjust_prepare_kernel, beside 8.2 KB of fixed size
constexpr int kAdjustRounds = 4;          // entries per token of a part of a bias list that are added by all threads together
constexpr int kAdjustScan = 16;           // entries that a thread looks at together
constexpr uint32_t kAdjustSeen = 0x80000000u;
constexpr uint32_t kFloorFinite = 0x00800000u;  // order_bits of the lowest finite value: -inf is no candidate

struct AdjustRecord {
    uint32_t id;  // | kAdjustSeen
    float add;
};

struct AdjustParams {
    // per sequence
    const int32_t *history, *history_len;  // [n_seq, H], [n_seq] (null: H)
    const float *repetition, *frequency, *presence;  // [n_seq], null: 1, 0, 0
    const int32_t* bias_ids;               // [n_seq, NB]
    const float* bias;
    int H, NB, rows_per_seq, max_records;
    // per row
    const uint32_t* mask;        // [n_masks, mask_stride]
    const int32_t* mask_index;   // [rows], null: the row itself
    int64_t mask_stride;
    int n_masks;
    // what adjust_prepare_kernel leaves (null: no special tokens)
    uint32_t* special;           // [n_seq, words]
    AdjustRecord* records;       // [n_seq, max_records], in the order of their ids
    int32_t* before;             // [n_seq, groups + 1]: records before each group of kAdjustGroup tokens
    int V, words, groups, window;  // window: records counted at a time
};

// bias - (f c + p), each operation rounded by itself.
__device__ __forceinline__ float adjust_add(float bias, float f, float p, int c) {
#pragma clang fp contract(off)
    const float penalty = f * (float)c + p;
    return bias - penalty;
}

// One workgroup per sequence.  LDS: the bitmap (words), a prefix of popcounts per group of 512 tokens, and a window
// of counts and biases.  A record's place is its token's rank among the set bits, so no order of atomics shows.
// A chain of LDS latencies between barriers (a sequence of 500 ids 5.2 us, 64 of 2048 ids 7.8).
// A bias list is taken in parts of an entry per thread, so that its cost goes by its length whatever it names: a round adds
// each token's first entry of the part that is not in its sum, and what a token has left after kAdjustRounds of them is added
// by one thread each, from LDS (8 rows of 126464: 300 biases distinct 24 us, 250 of them one token's 41; 16384 distinct 54, one
// token five times 76, one token in every second 402).
__global__ __launch_bounds__(kAdjustPrepThreads) void adjust_prepare_kernel(AdjustParams P) {
    extern __shared__ uint32_t prep_lds[];
    __shared__ int sh_wave[kAdjustPrepThreads / 64];
    constexpr int WPG = kAdjustGroup / 32;
    const int words = P.words, groups = P.groups;
    uint32_t* bits = prep_lds;
    uint16_t* inside = reinterpret_cast<uint16_t*>(prep_lds + groups * WPG);             // set bits of the group before the word
    int* prefix = reinterpret_cast<int*>(prep_lds + groups * WPG + groups * (WPG / 2));  // and before the group
    int* count = prefix + groups;                       // times seen
    int* turn = count + P.window;                       // the thread whose entry is next
    float* bias_sum = reinterpret_cast<float*>(turn + P.window);
    __shared__ int sh_more;
    __shared__ __align__(16) int sh_rank[kAdjustPrepThreads];  // of a part of the bias list
    __shared__ __align__(16) float sh_bias[kAdjustPrepThreads];
    const int seq = blockIdx.x, tid = threadIdx.x;
    const int32_t* history = P.history + (int64_t)seq * P.H;
    const int32_t* ids = P.bias_ids + (int64_t)seq * P.NB;
    const float* bias = P.bias + (int64_t)seq * P.NB;
    int hl = P.H;
    if (P.history_len != nullptr && P.H > 0) {
        hl = P.history_len[seq];
        if (hl < 0 || hl > P.H) {
            if (tid == 0) flag_device_status(kDevBadHistory);
            hl = hl < 0 ? 0 : P.H;
        }
    }
    // the first entries are requested before anything waits
    const int h0 = tid < P.H ? history[tid] : -1, b0 = tid < P.NB ? ids[tid] : -1;
    const float y0 = tid < P.NB ? bias[tid] : 0.f;
    const float f = P.frequency != nullptr ? P.frequency[seq] : 0.f;
    const float p = P.presence != nullptr ? P.presence[seq] : 0.f;
    auto seen_at = [&](int i) { return i < kAdjustPrepThreads ? h0 : history[i]; };
    auto in_vocab = [&](int id) { return id >= 0 && id < P.V; };

    for (int w = tid; w < groups * (WPG / 4); w += kAdjustPrepThreads) reinterpret_cast<u32x4_t*>(bits)[w] = u32x4_t{};
    auto clear_window = [&] {
        for (int i = tid; i < P.window; i += kAdjustPrepThreads) {
            count[i] = 0;
            turn[i] = INT32_MAX;
            bias_sum[i] = -0.f;  // plus any value: that value
        }
    };
    clear_window();
    __syncthreads();
    for (int i = tid; i < hl; i += kAdjustPrepThreads) {
        const int id = seen_at(i);
        if (in_vocab(id)) atomicOr(&bits[id >> 5], 1u << (id & 31));
    }
    for (int j = tid; j < P.NB; j += kAdjustPrepThreads) {
        const int id = j < kAdjustPrepThreads ? b0 : ids[j];
        if (in_vocab(id)) atomicOr(&bits[id >> 5], 1u << (id & 31));
    }
    __syncthreads();
    // prefixes of the words' popcounts: a group per thread
    static_assert(kAdjustMaxVocab / kAdjustGroup <= kAdjustPrepThreads, "a group per thread");
    int own = 0;
    if (tid < groups) {
        const u32x4_t* x = reinterpret_cast<const u32x4_t*>(bits + tid * WPG);
#pragma unroll
        for (int i = 0; i < WPG / 4; ++i) {
            const u32x4_t v = x[i];
            u32x2_t two;
            two[0] = (uint32_t)own;
            own += __popc(v[0]);
            two[0] |= (uint32_t)own << 16;
            own += __popc(v[1]);
            two[1] = (uint32_t)own;
            own += __popc(v[2]);
            two[1] |= (uint32_t)own << 16;
            own += __popc(v[3]);
            reinterpret_cast<u32x2_t*>(inside + tid * WPG)[i] = two;
        }
    }
    const int incl = wave_prefix(own);
    if ((tid & 63) == 63) sh_wave[tid >> 6] = incl;
    __syncthreads();
    int excl = incl - own, total = 0;
#pragma unroll
    for (int w = 0; w < kAdjustPrepThreads / 64; ++w) {
        excl += w < (tid >> 6) ? sh_wave[w] : 0;
        total += sh_wave[w];
    }
    int32_t* before = P.before + (int64_t)seq * (groups + 1);
    if (tid < groups) {
        prefix[tid] = excl;
        before[tid] = excl;
    }
    if (tid == 0) before[groups] = total;
    uint32_t* special = P.special + (int64_t)seq * words;
    for (int w = tid; w < words; w += kAdjustPrepThreads) special[w] = bits[w];
    __syncthreads();

    auto rank = [&](int id) -> int {
        return prefix[id / kAdjustGroup] + (int)inside[id >> 5] + __popc(bits[id >> 5] & ((1u << (id & 31)) - 1u));
    };
    AdjustRecord* records = P.records + (int64_t)seq * P.max_records;
    for (int w0 = 0; w0 < total; w0 += P.window) {
        if (w0 > 0) {
            __syncthreads();
            clear_window();
            __syncthreads();
        }
        for (int i = tid; i < hl; i += kAdjustPrepThreads) {
            const int id = seen_at(i);
            if (!in_vocab(id)) continue;
            const int r = rank(id) - w0;
            if (r >= 0 && r < P.window) atomicAdd(&count[r], 1);
        }
        // Biases of one token add up in the order of the list.
        int id = b0;
        float y = y0;
        for (int j0 = 0; j0 < P.NB; j0 += kAdjustPrepThreads) {
            int r = tid < P.NB - j0 && in_vocab(id) ? rank(id) - w0 : -1;
            if (r >= P.window) r = -1;
            bool open = r >= 0;
            sh_rank[tid] = r;
            sh_bias[tid] = y;
            const int next = j0 + kAdjustPrepThreads + tid;
            if (next < P.NB) {
                id = ids[next];
                y = bias[next];
            }
            bool more = true;
            for (int round = 0; more && round <= kAdjustRounds; ++round) {
                if (tid == 0) sh_more = 0;
                if (open) atomicMin(&turn[r], tid);
                __syncthreads();
                const bool mine = open && turn[r] == tid;
                if (mine) {
                    float sum = bias_sum[r] + sh_bias[tid];
                    if (round == kAdjustRounds) {
                        for (int i = tid & ~(kAdjustScan - 1); i < kAdjustPrepThreads; i += kAdjustScan) {
                            u32x4_t rank4[kAdjustScan / 4];
                            u32x4_t bias4[kAdjustScan / 4];
#pragma unroll
                            for (int e = 0; e < kAdjustScan / 4; ++e) {
                                rank4[e] = *reinterpret_cast<const u32x4_t*>(sh_rank + i + 4 * e);
                                bias4[e] = *reinterpret_cast<const u32x4_t*>(sh_bias + i + 4 * e);
                            }
#pragma unroll
                            for (int e = 0; e < kAdjustScan; ++e) {
                                const uint32_t other = rank4[e / 4][e % 4], add = bias4[e / 4][e % 4];
                                sum = other == (uint32_t)r && i + e > tid ? sum + __builtin_bit_cast(float, add) : sum;
                            }
                        }
                    }
                    bias_sum[r] = sum;
                } else if (open) {
                    sh_more = 1;
                }
                __syncthreads();
                more = sh_more != 0;
                if (mine) {
                    turn[r] = INT32_MAX;
                    open = false;
                }
                __syncthreads();
            }
        }
        if (P.NB == 0) __syncthreads();
        for (int w = tid; w < words; w += kAdjustPrepThreads) {
            uint32_t x = bits[w];
            if (x == 0u) continue;
            int r = rank(w * 32) - w0;
            for (; x != 0u; x &= x - 1u, ++r) {
                if (r < 0 || r >= P.window) continue;
                const int c = count[r];
                const float y = bias_sum[r];
                records[w0 + r] = AdjustRecord{(uint32_t)(w * 32 + __builtin_ctz(x)) | (c > 0 ? kAdjustSeen : 0u), c > 0 ? adjust_add(y, f, p, c) : y};
            }
        }
    }
}

// Absorbs NV values x (-inf: forbidden) of vocabulary indices id0 .. whose maximum is vmax, as absorb() does, but the sum is
// kept relative to 2^(-nrl), nrl being the rounded product, which lane_sum() corrects once at the end: no error grows
// with the logits' size.
template <int K, int NV>
__device__ __forceinline__ void adjust_absorb(const float (&x)[NV], float vmax, int id0, TopkLane<K>& st, uint32_t floor_bits) {
    const bool up = vmax > st.rthr;
    if (ballot64(up) != 0ull) {  // wave-uniform branch, rare after the first vectors
        const float ref = fmaxf(vmax, kRefFloor);
        const float nr = -ref * kLog2e;
        st.s = up && st.s != 0.f ? st.s * fast_exp2(nr - st.nrl) : st.s;
        st.ref = up ? ref : st.ref;
        st.nrl = up ? nr : st.nrl;
        st.rthr = up ? ref + kTopkLazyLog2 / kLog2e : st.rthr;
    }
    st.lmax = __builtin_elementwise_maximum(st.lmax, vmax);
    float acc = fast_exp2(__builtin_fmaf(x[0], kLog2e, st.nrl));
#pragma unroll
    for (int j = 1; j < NV; ++j) acc += fast_exp2(__builtin_fmaf(x[j], kLog2e, st.nrl));
    st.s += acc;
    if (vmax >= st.ins) {
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            if (x[j] >= st.ins) {
                const uint64_t key = make_key(x[j], id0 + j);
                if (key > st.tl.key[K - 1]) st.tl.insert(key);
            }
        }
        st.refresh(floor_bits);
    }
}
// The lane's sum relative to its reference itself.
template <int K>
__device__ __forceinline__ float lane_sum(const TopkLane<K>& st) {
    return st.s != 0.f ? st.s * fast_exp2(-__builtin_fmaf(st.ref, kLog2e, st.nrl)) : 0.f;
}

// conf / idx of a row from its (reference, sum) and its keys; a slot without a candidate: 0 and -1.
template <int K>
__device__ __forceinline__ void adjust_finish(const uint64_t (&key)[K], float m, float s, int row, int k, float* conf, int32_t* idx) {
    const float inv = 1.0f / s;
#pragma unroll
    for (int j = 0; j < K; ++j) {
        if (j < k) {
            const bool some = key[j] != 0ull;
            conf[(int64_t)row * k + j] = some ? fast_exp2((key_value(key[j]) - m) * kLog2e) * inv : 0.f;
            idx[(int64_t)row * k + j] = some ? key_index(key[j]) : -1;
        }
    }
}

// grid.x = rows * splits, slices and register ring as conf_topk_kernel.  LDS: the slice's allowed bits, and the list of
// a slice with few allowed tokens.
//   * Vectors without an allowed token are not read (their lanes load the slice's first vector), and a slice with at
//     most kAdjustList allowed ones gathers just those (256 rows of 126464 under masks of 250 tokens: 22.5 -> 10.0 us).
//   * The special tokens are gathered behind the stream, several per lane at a time.  Each costs a 64-byte sector of
//     its row: 2048 rows of 126464 bf16 take 87 us with nothing to adjust (6.0 TB/s), 100 with a mask of 97%, 129 with
//     1800 special tokens each besides (222 MB of sectors).  Gathered along the way, with the lines just streamed, they
//     took as long: the registers cost a wave per SIMD, and the XCD's 4 MB L2 does not hold its 256 rows' windows.
constexpr int kAdjustList = 512;

template <typename T, int K, int THREADS, int U, int DEPTH>
__global__ __launch_bounds__(THREADS) void adjust_topk_kernel(AdjustParams A, const T* __restrict__ logits, int64_t row_stride, int k,
                                                              int splits, int chunk, float* __restrict__ conf,
                                                              int32_t* __restrict__ idx, float* __restrict__ partial) {
    constexpr int NV = VecOf<T>::n;
    constexpr int SW = THREADS * U;
    constexpr int NW = THREADS / 64;
    static_assert(NW > 1 && NW <= 16, "the row reduction covers at most 16 waves");
    constexpr uint32_t kAll = (1u << NV) - 1u;
    extern __shared__ uint32_t allowed[];
    __shared__ uint32_t sh_floor[NW];
    __shared__ int sh_count[NW];
    const int row = blockIdx.x / splits;
    const int split = blockIdx.x - row * splits;
    const int begin = split * chunk;  // a multiple of kAdjustGroup
    const int end = min(A.V, begin + chunk);
    const T* base = logits + (int64_t)row * row_stride;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int seq = row / A.rows_per_seq;

    const uint32_t* mrow = nullptr;
    bool forbidden = false;
    if (A.mask != nullptr) {
        const int mi = A.mask_index != nullptr ? A.mask_index[row] : row;
        if (mi >= 0 && mi < A.n_masks) {
            mrow = A.mask + mi * A.mask_stride;
        } else if (mi != -1) {  // not a mask: nothing is allowed
            if (split == 0 && tid == 0) flag_device_status(kDevBadMask);
            forbidden = true;
        }
    }
    const bool masked = mrow != nullptr || forbidden;

    const int lead = (int)((0u - (unsigned)(reinterpret_cast<uintptr_t>(base + begin) / sizeof(T))) % NV);
    const int head = min(lead, end - begin);
    const int vbegin = begin + head;
    const int nvec = (end - vbegin) / NV;
    const u32x4_t* vp = reinterpret_cast<const u32x4_t*>(base + vbegin);
    u32x4_t buf[DEPTH][U];
    if (!masked && nvec > 0) {  // the first sweeps are on their way while the special tokens' bits arrive
#pragma unroll
        for (int d = 0; d + 1 < DEPTH; ++d)
#pragma unroll
            for (int u = 0; u < U; ++u) buf[d][u] = __builtin_nontemporal_load(vp + min(d * SW + u * THREADS + tid, nvec - 1));
    }

    // the slice's special tokens
    const int32_t* before = A.before + (int64_t)seq * (A.groups + 1);
    const AdjustRecord* rec = A.records + (int64_t)seq * A.max_records;
    const bool specials = A.special != nullptr && !forbidden;
    const int first_special = specials ? before[begin / kAdjustGroup] : 0;
    const int last_special = specials ? before[(end + kAdjustGroup - 1) / kAdjustGroup] : 0;
    const float r = A.repetition != nullptr ? A.repetition[seq] : 1.0f;
    auto special_value = [&](const AdjustRecord& a, float l, uint32_t m) {
        if (a.id & kAdjustSeen) l = l > 0.f ? l / r : l * r;
        return ((m >> (a.id & 31)) & 1u) != 0u ? l + a.add : kNegInf;
    };

    const int nw = (end - begin + 31) / 32;
    int n_allowed = 0;
    for (int w = tid; w < nw; w += THREADS) {
        uint32_t x = forbidden ? 0u : 0xffffffffu;
        if (mrow != nullptr) x = mrow[begin / 32 + w];
        if (A.special != nullptr) x &= ~A.special[(int64_t)seq * A.words + begin / 32 + w];
        if (w == nw - 1 && (end & 31) != 0) x &= (1u << (end & 31)) - 1u;  // only the row's last word is not whole
        allowed[w] = x;
        n_allowed += __popc(x);
    }
    const int before_lane = wave_prefix(n_allowed) - n_allowed;
    if (lane == 63) sh_count[wave] = before_lane + n_allowed;
    if (lane == 0) sh_floor[wave] = 0u;
    __syncthreads();
    int list_at = before_lane, listed = 0;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
        list_at += w < wave ? sh_count[w] : 0;
        listed += sh_count[w];
    }

    TopkLane<K> st;
    st.init();
    uint32_t floor_bits = kFloorFinite;
    st.refresh(floor_bits);

    const bool few = listed <= kAdjustList;
    int32_t* list = reinterpret_cast<int32_t*>(allowed + (chunk + 31) / 32 + 1);
    if (few) {
        for (int w = tid; w < nw; w += THREADS)
            for (uint32_t x = allowed[w]; x != 0u; x &= x - 1u) list[list_at++] = begin + 32 * w + __builtin_ctz(x);
        __syncthreads();
        for (int i = tid; i < listed; i += THREADS) {
            const int id = list[i];
            const float x[1] = {load_scalar(base + id)};
            adjust_absorb<K, 1>(x, x[0], id, st, floor_bits);
        }
    } else {
        // The waves of a workgroup share their floors through LDS, as in conf_topk_kernel.
        auto share_floor = [&](uint32_t fb) {
            if (lane == 0) __hip_atomic_store(&sh_floor[wave], fb, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
#pragma unroll
            for (int w = 0; w < NW; ++w) {
                const uint32_t o = __hip_atomic_load(&sh_floor[w], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
                fb = o > fb ? o : fb;
            }
            return fb;
        };
        // Allowed bits of this lane's vector in a sweep, 0 past the slice.  A vector's first bit has the same place in its
        // byte in every sweep (THREADS * NV is a multiple of 8); bits behind a byte come from the next (the LDS holds a
        // word more).
        const uint8_t* bytes = reinterpret_cast<const uint8_t*>(allowed) + ((head + tid * NV) >> 3);
        const int shift = (head + tid * NV) & 7;
        const bool any_bits = masked || A.special != nullptr;
        auto vec_bits = [&](int v) -> uint32_t {  // v: of lane 0
            const int at = v + tid < nvec ? v * NV / 8 : 0;
            uint32_t x = bytes[at];
            if (head != 0) x |= (uint32_t)bytes[at + 1] << 8;  // uniform
            return v + tid < nvec ? x >> shift & kAll : 0u;
        };
        auto load = [&](int sweep, u32x4_t (&b)[U]) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int v0 = sweep * SW + u * THREADS, v = min(v0 + tid, nvec - 1);
                b[u] = __builtin_nontemporal_load(vp + (!masked || vec_bits(v0) != 0u ? v : 0));
            }
        };
        // the values of a vector, forbidden ones -inf; false where the wave has none
        auto values = [&](int v0, const u32x4_t& b, float (&x)[NV]) {
            const uint32_t ok = any_bits ? vec_bits(v0) : v0 + tid < nvec ? kAll : 0u;
            if (ballot64(ok != 0u) == 0ull) return false;
            unpack(b, x);
            if (ballot64(ok != kAll) != 0ull) {
#pragma unroll
                for (int j = 0; j < NV; ++j) {
                    const int m = (int)(ok << (31 - j)) >> 31;
                    const int xi = __builtin_bit_cast(int, x[j]);
                    x[j] = __builtin_bit_cast(float, (xi & m) | ((int)0xff800000 & ~m));
                }
            }
            return true;
        };
        auto absorb_sweep = [&](int sweep, const u32x4_t (&b)[U]) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int v0 = sweep * SW + u * THREADS;
                float x[NV];
                if (!values(v0, b[u], x)) continue;
                adjust_absorb<K, NV>(x, vec_max<NV>(x), vbegin + (v0 + tid) * NV, st, floor_bits);
            }
            if (sweep != 0 && (sweep & (sweep + 1)) == 0) {
                const uint32_t own = wave_kth_floor<K>(st.lmax, k);
                floor_bits = share_floor(own > floor_bits ? own : floor_bits);
                st.refresh(floor_bits);
            } else {
                const uint32_t f = share_floor(floor_bits);
                if (f != floor_bits) {  // wave-uniform
                    floor_bits = f;
                    st.refresh(floor_bits);
                }
            }
        };
        const int nsw = (nvec + SW - 1) / SW;
        if (nsw > 0) {
            if (masked) {
#pragma unroll
                for (int d = 0; d + 1 < DEPTH; ++d) load(d, buf[d]);
            }
            {  // a first floor from sweep 0's lane maxima, so that sweep 0 already inserts rarely
                float lm = kNegInf;
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    float x[NV];
                    if (values(u * THREADS, buf[0][u], x)) lm = __builtin_elementwise_maximum(lm, vec_max<NV>(x));
                }
                const uint32_t own = wave_kth_floor<K>(lm, k);
                floor_bits = share_floor(own > floor_bits ? own : floor_bits);
                st.refresh(floor_bits);
            }
            for (int it = 0; it < nsw; it += DEPTH) {
#pragma unroll
                for (int j = 0; j < DEPTH; ++j) {
                    load(it + j + DEPTH - 1, buf[(j + DEPTH - 1) % DEPTH]);
                    __builtin_amdgcn_sched_barrier(0);
                    absorb_sweep(it + j, buf[j]);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
        }
        const int tail = vbegin + nvec * NV;  // values before and behind the vectors
        for (int i = tid; i < head + (end - tail); i += THREADS) {
            const int e = i < head ? begin + i : tail + (i - head);
            const bool ok = ((allowed[(e - begin) >> 5] >> (e & 31)) & 1u) != 0u;
            const float l = load_scalar(base + e);
            const float x[1] = {ok ? l : kNegInf};
            adjust_absorb<K, 1>(x, x[0], e, st, floor_bits);
        }
    }
    // The special tokens, several per lane at a time: records, then logits, then values.
    constexpr int G = 4;
    for (int i0 = first_special + tid; i0 < last_special; i0 += G * THREADS) {
        AdjustRecord a[G];
        float l[G];
        uint32_t m[G];
#pragma unroll
        for (int e = 0; e < G; ++e) a[e] = rec[min(i0 + e * THREADS, last_special - 1)];
#pragma unroll
        for (int e = 0; e < G; ++e) {
            const int id = (int)(a[e].id & ~kAdjustSeen);
            l[e] = load_scalar(base + id);
            m[e] = mrow != nullptr ? mrow[id >> 5] : 0xffffffffu;
        }
#pragma unroll
        for (int e = 0; e < G; ++e) {
            const float x[1] = {i0 + e * THREADS < last_special ? special_value(a[e], l[e], m[e]) : kNegInf};
            adjust_absorb<K, 1>(x, x[0], (int)(a[e].id & ~kAdjustSeen), st, floor_bits);
        }
    }

    // lanes -> wave -> workgroup, as conf_topk_kernel
    float m = st.ref, s = lane_sum(st);
    lanes_merge_ms<6>(m, s);
    uint64_t best[K];
    wave_top_keys<K>(st.tl, best, k);
    TopList<K> tl;
    __shared__ float sh_m[NW], sh_s[NW];
    __shared__ uint64_t sh_k[NW][K];
    __shared__ float sh_max;
    if (lane == 0) {
        sh_m[wave] = m;
        sh_s[wave] = s;
#pragma unroll
        for (int j = 0; j < K; ++j) sh_k[wave][j] = best[j];
    }
    __syncthreads();
    if (wave == 0) {
        tl.clear();
        m = kNegInf;
        s = 0.f;
        if (lane < NW) {
            m = sh_m[lane];
            s = sh_s[lane];
#pragma unroll
            for (int j = 0; j < K; ++j) tl.key[j] = sh_k[lane][j];
        }
        constexpr int STEPS = NW <= 2 ? 1 : NW <= 4 ? 2 : 4;
        lanes_merge_ms<STEPS>(m, s);
#pragma unroll
        for (int t = 0; t < STEPS; ++t) {
            uint64_t b[K];
#pragma unroll
            for (int j = 0; j < K; ++j) lane_pair64(t, tl.key[j], tl.key[j], b[j]);
            tl.merge(b);
        }
        // a slice with candidates whose weights came to nothing: see below
        if (lane == 0) sh_max = tl.key[0] != 0ull && !(s > 0.f && s < -kNegInf) ? key_value(tl.key[0]) : kNegInf;
    }
    __syncthreads();
    // All of the slice's values are at the lowest end of their type (or its maximum at the highest), where a product
    // with log2(e) overflows: the sum is taken again, relative to the maximum and subtracting first.
    const float top = sh_max;
    if (top != kNegInf) {
        float acc = 0.f;
        for (int e = begin + tid; e < end; e += THREADS)
            if ((allowed[(e - begin) >> 5] >> (e & 31)) & 1u) acc += fast_exp2((load_scalar(base + e) - top) * kLog2e);
        for (int i = first_special + tid; i < last_special; i += THREADS) {
            const AdjustRecord a = rec[i];
            const int id = (int)(a.id & ~kAdjustSeen);
            acc += fast_exp2((special_value(a, load_scalar(base + id), mrow != nullptr ? mrow[id >> 5] : 0xffffffffu) - top) * kLog2e);
        }
        m = top;
        s = block_sum<THREADS>(acc, sh_s);
    }
    if (tid != 0) return;
    if (partial != nullptr) {
        float* rec = partial + ((int64_t)row * splits + split) * kTopkRecord;
        rec[0] = m;
        rec[1] = s;
        uint64_t* rk = reinterpret_cast<uint64_t*>(rec + 2);
#pragma unroll
        for (int j = 0; j < 8; ++j) rk[j] = j < K ? tl.key[j] : 0ull;
        return;
    }
    adjust_finish<K>(tl.key, m, s, row, k, conf, idx);
}

// One wave per row merges `splits` partial records.
template <int K>
__global__ __launch_bounds__(64) void adjust_merge_kernel(const float* __restrict__ partial, int splits, int k, float* __restrict__ conf,
                                                          int32_t* __restrict__ idx) {
    const int row = blockIdx.x;
    const int lane = threadIdx.x;
    float m = kNegInf, s = 0.f;
    TopList<K> tl;
    tl.clear();
    for (int sp = lane; sp < splits; sp += 64) {
        const float* rec = partial + ((int64_t)row * splits + sp) * kTopkRecord;
        merge_ms(m, s, rec[0], rec[1]);
        const uint64_t* rk = reinterpret_cast<const uint64_t*>(rec + 2);
        uint64_t o[K];
#pragma unroll
        for (int j = 0; j < K; ++j) o[j] = rk[j];
        tl.merge(o);
    }
    float top = m;
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) top = fmaxf(top, __shfl_xor(top, off));
    s *= fast_exp2((m - (top == kNegInf ? 0.f : top)) * kLog2e);
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) s += __shfl_xor(s, off);
    uint64_t best[K];
    wave_top_keys<K>(tl, best, k);
    m = top;
    if (lane == 0) adjust_finish<K>(best, m, s, row, k, conf, idx);
}

inline size_t adjust_lds(int chunk) { return ((size_t)(chunk + 31) / 32 + 1 + kAdjustList) * sizeof(uint32_t); }
// LDS of adjust_prepare_kernel: bits and prefixes, then 12 bytes per record of the window.
inline size_t adjust_prepare_fixed(int groups) { return (size_t)groups * (kAdjustGroup / 32 * 6 + 4); }
inline int adjust_window(int groups, int max_records) {
    const int most = (int)((kAdjustLds - adjust_prepare_fixed(groups)) / 12);
    return max_records < most ? max_records : most;
}

// Launch shape: threads per row slice and its register ring, slices per row (as plan_conf_topk; one wave per row
// would hold the allowed bits of a row per wave in LDS, so rows take 4 waves at least).
constexpr int64_t kAdjustFewRows = 64, kAdjustSlices = 256;
inline TopkPlan plan_adjust(int64_t rows, int64_t vocab, int vec) {
    TopkPlan p = plan_conf_topk(rows, vocab, vec);
    if (p.threads == 64) p = TopkPlan{256, 2, 2, 1, (int)vocab};
    // Few rows that are split are split further, down to two vectors per lane: a slice is a chain of latencies beside its
    // stream (1 row of 126464 16.3 -> 15.4 us, 32 rows 20.1 -> 17.7; 100 rows 31.6 against 32.4, so not those; rows
    // that one workgroup takes in four vectors per lane stay whole, 5 of 9000 12.0 against 13.8).
    if (p.splits > 1 && rows <= kAdjustFewRows) {
        const int64_t align = (int64_t)p.threads * vec;
        int64_t splits = std::min<int64_t>((kAdjustSlices + rows - 1) / rows, (vocab + 2 * align - 1) / (2 * align));
        splits = std::min<int64_t>(splits, 64);
        p.chunk = (int)(((vocab + splits - 1) / splits + align - 1) / align * align);
        p.splits = (int)((vocab + p.chunk - 1) / p.chunk);
    }
    return p;
}

}  // namespace trajspec
