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

#include "conf_topk.hpp"
#include "layer.hpp"

namespace trajspec {

constexpr int kDevBadMask = 0x40;    // TRAJ_DEV_BAD_MASK
constexpr int kDevBadHistory = 0x80; // TRAJ_DEV_BAD_HISTORY

constexpr int kAdjustMaxVocab = 1 << 20;  // one bit per token in LDS: 128 KB
constexpr int kAdjustPrepThreads = 1024;
constexpr int kAdjustGroup = 512;         // tokens per popcount prefix
constexpr int kAdjustWindow = 2048;       // records counted at a time
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
    AdjustRecord* records;       // [n_seq, max_records]
    int32_t* n_records;          // [n_seq]
    int V, words;
};

// bias - (f c + p), each operation rounded by itself.
__device__ __forceinline__ float adjust_add(float bias, float f, float p, int c) {
#pragma clang fp contract(off)
    const float penalty = f * (float)c + p;
    return bias - penalty;
}

// One workgroup per sequence.  LDS: the bitmap (words), a prefix of popcounts per group of 512 tokens, and a window
// of counts and biases.  A record's place is its token's rank among the set bits, so no order of atomics shows.
__global__ __launch_bounds__(kAdjustPrepThreads) void adjust_prepare_kernel(AdjustParams P) {
    extern __shared__ uint32_t prep_lds[];
    __shared__ int sh_wave[kAdjustPrepThreads / 64];
    __shared__ int sh_dup;
    constexpr int WPG = kAdjustGroup / 32;
    const int words = P.words, groups = (words + WPG - 1) / WPG;
    uint32_t* bits = prep_lds;
    int* prefix = reinterpret_cast<int*>(prep_lds + groups * WPG);
    int* count = prefix + groups;
    float* bias_sum = reinterpret_cast<float*>(count + kAdjustWindow);
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
    auto in_vocab = [&](int id) { return id >= 0 && id < P.V; };

    for (int w = tid; w < groups * WPG; w += kAdjustPrepThreads) bits[w] = 0u;
    if (tid == 0) sh_dup = 0;
    __syncthreads();
    for (int j = tid; j < P.NB; j += kAdjustPrepThreads) {
        const int id = ids[j];
        if (in_vocab(id) && ((atomicOr(&bits[id >> 5], 1u << (id & 31)) >> (id & 31)) & 1u)) sh_dup = 1;
    }
    __syncthreads();
    for (int i = tid; i < hl; i += kAdjustPrepThreads) {
        const int id = history[i];
        if (in_vocab(id)) atomicOr(&bits[id >> 5], 1u << (id & 31));
    }
    __syncthreads();
    // exclusive prefix of the groups' popcounts: two consecutive groups per thread (2048 groups at most)
    static_assert(kAdjustMaxVocab / kAdjustGroup <= 2 * kAdjustPrepThreads, "two groups per thread");
    int own[2] = {0, 0};
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        const int gidx = 2 * tid + e;
        if (gidx < groups)
            for (int w = 0; w < WPG; ++w) own[e] += __popc(bits[gidx * WPG + w]);
    }
    int incl = own[0] + own[1];
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const int o = __shfl_up(incl, off);
        if ((tid & 63) >= off) incl += o;
    }
    if ((tid & 63) == 63) sh_wave[tid >> 6] = incl;
    __syncthreads();
    int before = 0, total = 0;
    for (int w = 0; w < kAdjustPrepThreads / 64; ++w) {
        if (w < (tid >> 6)) before += sh_wave[w];
        total += sh_wave[w];
    }
    const int excl = before + incl - own[0] - own[1];
    if (2 * tid < groups) prefix[2 * tid] = excl;
    if (2 * tid + 1 < groups) prefix[2 * tid + 1] = excl + own[0];
    uint32_t* special = P.special + (int64_t)seq * words;
    for (int w = tid; w < words; w += kAdjustPrepThreads) special[w] = bits[w];
    if (tid == 0) P.n_records[seq] = total;
    __syncthreads();

    auto rank = [&](int id) {
        int r = prefix[id / kAdjustGroup];
        const int w1 = id >> 5;
        for (int w = id / kAdjustGroup * WPG; w < w1; ++w) r += __popc(bits[w]);
        return r + __popc(bits[w1] & ((1u << (id & 31)) - 1u));
    };
    const float f = P.frequency != nullptr ? P.frequency[seq] : 0.f;
    const float p = P.presence != nullptr ? P.presence[seq] : 0.f;
    AdjustRecord* records = P.records + (int64_t)seq * P.max_records;
    for (int w0 = 0; w0 < total; w0 += kAdjustWindow) {
        for (int i = tid; i < kAdjustWindow; i += kAdjustPrepThreads) {
            count[i] = 0;
            bias_sum[i] = 0.f;
        }
        __syncthreads();
        for (int i = tid; i < hl; i += kAdjustPrepThreads) {
            const int id = history[i];
            if (!in_vocab(id)) continue;
            const int r = rank(id) - w0;
            if (r >= 0 && r < kAdjustWindow) atomicAdd(&count[r], 1);
        }
        for (int j = tid; j < P.NB; j += kAdjustPrepThreads) {
            const int id = ids[j];
            if (!in_vocab(id)) continue;
            const int r = rank(id) - w0;
            if (r < 0 || r >= kAdjustWindow) continue;
            float sum = bias[j];
            bool owner = true;
            if (sh_dup) {  // biases of one token add up in the order of the list
                for (int i = 0; i < P.NB && owner; ++i) {
                    if (ids[i] != id) continue;
                    if (i < j) owner = false;
                    if (i > j) sum += bias[i];
                }
            }
            if (owner) bias_sum[r] = sum;
        }
        __syncthreads();
        for (int w = tid; w < words; w += kAdjustPrepThreads) {
            uint32_t x = bits[w];
            if (x == 0u) continue;
            int r = rank(w * 32) - w0;
            for (; x != 0u; x &= x - 1u, ++r) {
                if (r < 0 || r >= kAdjustWindow) continue;
                const int c = count[r];
                const float add = c > 0 ? adjust_add(bias_sum[r], f, p, c) : bias_sum[r];
                records[w0 + r] = AdjustRecord{(uint32_t)(w * 32 + __builtin_ctz(x)) | (c > 0 ? kAdjustSeen : 0u), add};
            }
        }
        __syncthreads();
    }
}

// Absorbs NV values x (-inf: forbidden) of vocabulary indices id0 .. whose maximum is vmax, as absorb() does, with two
// differences.  A lane's reference stays at or above kRefFloor, so that values at the type's lowest add 0 and not NaN
// (a row of nothing else is summed again).  And the sum is kept relative to 2^(-nrl), nrl being the
// rounded product, which lane_sum() corrects once at the end: no error grows with the logits' size.
constexpr float kRefFloor = -1e30f;
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

// Two (reference, sum) pairs whose references may be of any finite size; -inf: nothing.
__device__ __forceinline__ void adjust_merge_ms(float& m, float& s, float m2, float s2) {
    const float M = fmaxf(m, m2), Ms = M == kNegInf ? 0.f : M;
    s = s * fast_exp2((m - Ms) * kLog2e) + s2 * fast_exp2((m2 - Ms) * kLog2e);
    m = M;
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

// grid.x = rows * splits, slices and register ring as conf_topk_kernel.  LDS: the slice's allowed bits.
template <typename T, int K, int THREADS, int U, int DEPTH>
__global__ __launch_bounds__(THREADS) void adjust_topk_kernel(AdjustParams A, const T* __restrict__ logits, int64_t row_stride, int k,
                                                              int splits, int chunk, float* __restrict__ conf,
                                                              int32_t* __restrict__ idx, float* __restrict__ partial) {
    constexpr int NV = VecOf<T>::n;
    constexpr int SW = THREADS * U;
    constexpr uint32_t kAll = (1u << NV) - 1u;
    extern __shared__ uint32_t allowed[];
    const int row = blockIdx.x / splits;
    const int split = blockIdx.x - row * splits;
    const int begin = split * chunk;  // a multiple of 32
    const int end = min(A.V, begin + chunk);
    const T* base = logits + (int64_t)row * row_stride;
    const int tid = threadIdx.x;
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
    const int nw = (end - begin + 31) / 32;
    for (int w = tid; w < nw; w += THREADS) {
        uint32_t x = forbidden ? 0u : 0xffffffffu;
        if (mrow != nullptr) x = mrow[begin / 32 + w];
        if (A.special != nullptr) x &= ~A.special[(int64_t)seq * A.words + begin / 32 + w];
        allowed[w] = x;
    }
    __syncthreads();

    TopkLane<K> st;
    st.init();
    uint32_t floor_bits = kFloorFinite;
    st.refresh(floor_bits);

    const int lead = (int)((0u - (unsigned)(reinterpret_cast<uintptr_t>(base + begin) / sizeof(T))) % NV);
    const int head = min(lead, end - begin);
    const int vbegin = begin + head;
    const int nvec = (end - vbegin) / NV;
    // allowed bits of vector v
    const uint8_t* bytes = reinterpret_cast<const uint8_t*>(allowed);
    auto vec_bits = [&](int v) -> uint32_t {
        const int at = head + v * NV;
        uint32_t x = bytes[at >> 3];
        if (head != 0) x |= (uint32_t)bytes[(at >> 3) + 1] << 8;  // uniform; the LDS holds a word more
        return (x >> (at & 7)) & kAll;
    };
    {
        const int nsw = (nvec + SW - 1) / SW;
        const u32x4_t* vp = reinterpret_cast<const u32x4_t*>(base + vbegin);
        // Vectors without an allowed value (and those past the slice) load its first vector instead: one cache line.
        auto load = [&](int sweep, u32x4_t (&b)[U]) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int v = sweep * SW + u * THREADS + tid;
                const bool some = v < nvec && vec_bits(v < nvec ? v : 0) != 0u;
                b[u] = __builtin_nontemporal_load(vp + (some ? v : 0));
            }
        };
        auto absorb_sweep = [&](int sweep, const u32x4_t (&b)[U]) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int v = sweep * SW + u * THREADS + tid;
                const uint32_t bits = v < nvec ? vec_bits(v) : 0u;
                if (ballot64(bits != 0u) == 0ull) continue;
                float x[NV];
                unpack(b[u], x);
                if (ballot64(bits != kAll) != 0ull) {
#pragma unroll
                    for (int j = 0; j < NV; ++j) {
                        const int m = (int)(bits << (31 - j)) >> 31;
                        const int xi = __builtin_bit_cast(int, x[j]);
                        x[j] = __builtin_bit_cast(float, (xi & m) | ((int)0xff800000 & ~m));
                    }
                }
                adjust_absorb<K, NV>(x, vec_max<NV>(x), vbegin + v * NV, st, floor_bits);
            }
            if ((sweep & (sweep + 1)) == 0) {
                const uint32_t own = wave_kth_floor<K>(st.lmax, k);
                floor_bits = own > floor_bits ? own : floor_bits;
                st.refresh(floor_bits);
            }
        };
        if (nsw > 0) {
            u32x4_t buf[DEPTH][U];
#pragma unroll
            for (int d = 0; d + 1 < DEPTH; ++d) load(d, buf[d]);
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
    }
    const int tail = vbegin + nvec * NV;
    const int lone = head + (end - tail);  // values before and behind the vectors
    auto lone_value = [&](int i, int& e) {
        e = i < head ? begin + i : tail + (i - head);
        const float l = load_scalar(base + e);
        return ((allowed[(e - begin) >> 5] >> (e & 31)) & 1u) != 0u ? l : kNegInf;
    };
    for (int i = tid; i < lone; i += THREADS) {
        int e;
        const float x[1] = {lone_value(i, e)};
        adjust_absorb<K, 1>(x, x[0], e, st, floor_bits);
    }
    // the special tokens, shared out over the row's slices
    const int specials = A.special != nullptr && !forbidden ? A.n_records[seq] : 0;
    const float r = A.repetition != nullptr ? A.repetition[seq] : 1.0f;
    const AdjustRecord* rec = A.records + (int64_t)seq * A.max_records;
    auto special_value = [&](int i, int& id) {
        const AdjustRecord a = rec[i];
        id = (int)(a.id & ~kAdjustSeen);
        const bool ok = mrow == nullptr || ((mrow[id >> 5] >> (id & 31)) & 1u) != 0u;
        float l = load_scalar(base + id);
        if (a.id & kAdjustSeen) l = l > 0.f ? l / r : l * r;
        return ok ? l + a.add : kNegInf;
    };
    for (int i = split * THREADS + tid; i < specials; i += splits * THREADS) {
        int id;
        const float x[1] = {special_value(i, id)};
        adjust_absorb<K, 1>(x, x[0], id, st, floor_bits);
    }

    // lanes -> wave -> workgroup, as conf_topk_kernel
    float m = st.ref, s = lane_sum(st);
    lanes_merge_ms<6>(m, s);
    uint64_t best[K];
    wave_top_keys<K>(st.tl, best, k);
    constexpr int NW = THREADS / 64;
    static_assert(NW > 1 && NW <= 16, "the row reduction covers at most 16 waves");
    TopList<K> tl;
    const int lane = tid & 63, wave = tid >> 6;
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
        for (int i = split * THREADS + tid; i < specials; i += splits * THREADS) {
            int id;
            acc += fast_exp2((special_value(i, id) - top) * kLog2e);
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
        adjust_merge_ms(m, s, rec[0], rec[1]);
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

// Launch shape: threads per row slice and its register ring, slices per row (as plan_conf_topk; a wave per row
// would hold the allowed bits of one row per wave in LDS, so rows take 4 waves at least).
inline TopkPlan plan_adjust(int64_t rows, int64_t vocab, int vec) {
    TopkPlan p = plan_conf_topk(rows, vocab, vec);
    if (p.threads == 64) p = TopkPlan{256, 2, 2, 1, (int)vocab};
    return p;
}

}  // namespace trajspec
