// Log probabilities of given tokens, the entropy of every row of logits and its most probable tokens; the logits' gradient.
//
// With t_j = scale (x_j - max x), S = sum_j e^t_j, p_j = e^t_j / S and i the row's given token:
//
//   logp = t_i - log S,   H = -sum_j p_j log p_j = log S - (sum_j e^t_j t_j) / S
//   dx_j = scale (g ([j = i] - p_j) - h p_j (log p_j + H))        with g, h the gradients of logp and H
//
// Differences to the largest logit are formed before they are scaled, so a row far from zero loses nothing.  Both are bound
// by memory: the forward reads every logit once (maximum and sums run together, rescaled where the maximum grows), the
// gradient reads and writes each once.  Both terms of H are of one sign: nothing cancels.
// Times below: one B200, device time per call in a row of calls on three sets of arrays.
#include <cmath>
#include <cooperative_groups.h>
#include <cuda_runtime.h>
#include <new>
#include <string>
#include <type_traits>

#include "baoc_device.cuh"

namespace baoc {

constexpr int kLogpMaxTop = 32;
constexpr int kLogpBatch = 4;                  // 16-byte loads a thread has in flight
constexpr int kLogpMostCtas = 8;               // CTAs (a cluster) that share a row where there are few rows,
constexpr int kLogpCtaLogits = 4096;           // each with at least so many logits
constexpr int kLogpShort = 64;                  // vectors a thread for which a row is given to fewer threads
constexpr int64_t kLogpMaxStride = int64_t(1) << 32;
constexpr float kLogpMaxScale = 1.7014118346046923e38f;      // 2^127: scale log2(e) stays finite
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kLeastExponent = -10000.f;     // 2^this is zero; it keeps 0 * -inf out of the entropy's sum

__device__ __forceinline__ float exp2_approx(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
// Maxima that keep a NaN.
__device__ __forceinline__ float max_nan(float a, float b) {
    float d;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
    return d;
}

template <int DT>
struct Logits {
    static constexpr int kSize = DT == BAOC_BF16 ? 2 : 4;
    static constexpr int kVec = 16 / kSize;
    static __device__ __forceinline__ float one(const char* row, int64_t j) {
        if constexpr (DT == BAOC_BF16) return bf16_bits_to_float(*reinterpret_cast<const uint16_t*>(row + 2 * j));
        else return *reinterpret_cast<const float*>(row + 4 * j);
    }
    static __device__ __forceinline__ void vec(const uint4& w, float (&x)[kVec]) {
        if constexpr (DT == BAOC_BF16) {
            unpack8(w, x);
        } else {
            x[0] = __uint_as_float(w.x); x[1] = __uint_as_float(w.y); x[2] = __uint_as_float(w.z); x[3] = __uint_as_float(w.w);
        }
    }
    // Numbers in the order of their values, all of them above 0; NaNs are alike and above infinity, -0 is 0.  The key of a
    // bf16 number has its upper 16 bits alone.
    static constexpr int kKeyBit = DT == BAOC_BF16 ? 16 : 0;
    static constexpr uint32_t kKeyMask = 0xffffffffu << kKeyBit;
    static __device__ __forceinline__ uint32_t key(float x) {
        if (x != x) return kKeyMask;
        const uint32_t u = __float_as_uint(x == 0.f ? 0.f : x);
        return (u & 0x80000000u ? ~u : u | 0x80000000u) & kKeyMask;
    }
    static __device__ __forceinline__ float value(uint32_t k) {
        return __uint_as_float((k & 0x80000000u ? k & 0x7fffffffu : ~k) & kKeyMask);
    }
    // larger logit, then lower token
    static __device__ __forceinline__ uint64_t key(float x, uint32_t token) { return uint64_t(key(x)) << 32 | uint32_t(~token); }
};

// A row as 16-byte vectors that start at its first aligned element, and the elements before and behind them.
struct RowSplit {
    int head;                // elements before the vectors
    int64_t vecs;
    int tail;
    template <int DT>
    __device__ __forceinline__ static RowSplit of(const char* row, int64_t vocab) {
        constexpr int kSize = Logits<DT>::kSize, kVec = Logits<DT>::kVec;
        RowSplit r;
        r.head = int(min64(vocab, int64_t((16 - (reinterpret_cast<uintptr_t>(row) & 15)) & 15) / kSize));
        r.vecs = (vocab - r.head) / kVec;
        r.tail = int(vocab - r.head - r.vecs * kVec);
        return r;
    }
    // the i-th element that no vector holds
    __device__ __forceinline__ int64_t edge(int64_t vocab, int i) const { return i < head ? i : vocab - tail + (i - head); }
};

// A maximum m, and the sums of 2^u and 2^u u over elements x with u = a (x - m), a = scale log2(e).
__device__ __forceinline__ float finite_ref(float m) { return fmaxf(m, -3.402823466e38f); }    // (where nothing but -inf has been seen)
struct Sums {
    float m, s, q;
    __device__ __forceinline__ void raise(float to, float a) {
        const float d = fmaxf(a * (finite_ref(m) - finite_ref(to)), kLeastExponent), f = exp2_approx(d);
        q = f * (q + d * s);
        s *= f;
        m = to;
    }
    __device__ __forceinline__ void join(Sums o, float a) {
        const float to = max_nan(m, o.m);
        raise(to, a);
        o.raise(to, a);
        s += o.s;
        q += o.q;
    }
};

// A thread's sums, two of each side by side, and the largest and smallest of a few vectors in front of them.
template <int DT>
struct ThreadSums {
    static constexpr int kVec = Logits<DT>::kVec;
    float m = -INFINITY;
    f32x2 s = 0, q = 0;

    __device__ __forceinline__ void raise(float to, float a) {
        const float d = fmaxf(a * (finite_ref(m) - finite_ref(to)), kLeastExponent);
        const f32x2 f = splat2(exp2_approx(d));
        q = mul2(f, fma2(splat2(d), s, q));
        s = mul2(f, s);
        m = to;
    }
    __device__ __forceinline__ void one(float x, float a) {
        const float to = max_nan(m, x);
        if (!(to <= m)) raise(to, a);
        const float u = fmaxf(a * (x - finite_ref(m)), kLeastExponent), e = exp2_approx(u);
        s = add2(s, pack2(e, 0.f));
        q = add2(q, pack2(e * u, 0.f));
    }
    // kClamp: some exponents are out of reach (a masked logit's is -inf, and 0 * -inf has no place in q)
    template <bool kClamp>
    __device__ __forceinline__ void vector(const uint4& w, f32x2 minus_ref, f32x2 a) {
        float x[kVec];
        Logits<DT>::vec(w, x);
#pragma unroll
        for (int j = 0; j < kVec; j += 2) {
            const f32x2 u2 = mul2(a, add2(pack2(x[j], x[j + 1]), minus_ref));
            float u, v;
            unpack2(u2, u, v);
            if constexpr (kClamp) {
                u = fmaxf(u, kLeastExponent);
                v = fmaxf(v, kLeastExponent);
            }
            const f32x2 e = pack2(exp2_approx(u), exp2_approx(v));
            s = add2(s, e);
            q = fma2(e, kClamp ? pack2(u, v) : u2, q);
        }
    }
    // n of the vectors count, the others repeat one of those; returns the largest
    __device__ __forceinline__ float batch(const uint4 (&w)[kLogpBatch], int n, float a) {
        float most, least;
        if constexpr (DT == BAOC_BF16) {
            uint32_t hi = w[0].x, lo = w[0].x;
#pragma unroll
            for (int u = 0; u < kLogpBatch; ++u)
#pragma unroll
                for (int i = u == 0 ? 1 : 0; i < 4; ++i) {
                    const uint32_t x = i == 0 ? w[u].x : (i == 1 ? w[u].y : (i == 2 ? w[u].z : w[u].w));
                    asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(hi) : "r"(hi), "r"(x));
                    asm("min.bf16x2 %0, %1, %2;" : "=r"(lo) : "r"(lo), "r"(x));
                }
            most = max_nan(bf16_lo(hi), bf16_hi(hi));
            least = fminf(bf16_lo(lo), bf16_hi(lo));
        } else {
            most = least = __uint_as_float(w[0].x);
#pragma unroll
            for (int u = 0; u < kLogpBatch; ++u) {
                float x[kVec];
                Logits<DT>::vec(w[u], x);
#pragma unroll
                for (int j = 0; j < kVec; ++j) {
                    most = max_nan(most, x[j]);
                    least = fminf(least, x[j]);
                }
            }
        }
        if (!(most <= m)) raise(max_nan(most, m), a);
        const float ref = finite_ref(m);
        const f32x2 minus_ref = splat2(-ref), a2 = splat2(a);
        if (a * (least - ref) >= kLeastExponent) {
#pragma unroll
            for (int u = 0; u < kLogpBatch; ++u)
                if (u < n) vector<false>(w[u], minus_ref, a2);
        } else {
#pragma unroll
            for (int u = 0; u < kLogpBatch; ++u)
                if (u < n) vector<true>(w[u], minus_ref, a2);
        }
        return most;
    }
    __device__ __forceinline__ Sums total() const {
        float s0, s1, q0, q1;
        unpack2(s, s0, s1);
        unpack2(q, q0, q1);
        return Sums{m, s0 + s1, q0 + q1};
    }
};

struct LogpArgs {
    const char* logits;
    const void* ids;
    int id_bits, top;
    int64_t vocab, step;         // step: bytes from row to row
    float scale;
    float *logp, *entropy, *stats;
    int32_t* top_ids;
    float* top_logp;
};

__device__ __forceinline__ int64_t given_token(const void* ids, int id_bits, int64_t row) {
    return id_bits == 64 ? static_cast<const int64_t*>(ids)[row] : static_cast<const int32_t*>(ids)[row];
}

// The largest value that at least `need` of the warp's values reach (kPer per lane); zero where fewer are above zero.
template <int kPer>
__device__ __forceinline__ uint32_t reached_by(const uint32_t (&v)[kPer], int need, int low_bit) {
    uint32_t t = 0;
    for (int bit = 31; bit >= low_bit; --bit) {
        const uint32_t c = t | (1u << bit);
        int n = 0;
#pragma unroll
        for (int i = 0; i < kPer; ++i) n += v[i] >= c;
        if (__reduce_add_sync(0xffffffffu, n) >= need) t = c;
    }
    return t;
}

// The same by taking the largest `need` times: a maximum and a ballot each, against 16 or 32 steps of a sum each above.
constexpr int kTopByMaxima = 8;
template <int kPer>
__device__ __forceinline__ uint32_t reached_by_maxima(uint32_t (&v)[kPer], int need) {
    const int lane = threadIdx.x & 31;
    for (;;) {
        uint32_t own = v[0];
#pragma unroll
        for (int i = 1; i < kPer; ++i) own = max(own, v[i]);
        const uint32_t most = __reduce_max_sync(0xffffffffu, own);
        if (--need == 0 || most == 0) return most;
        if (lane == __ffs(int(__ballot_sync(0xffffffffu, own == most))) - 1) {       // one of the largest goes
            bool gone = false;
#pragma unroll
            for (int i = 0; i < kPer; ++i)
                if (!gone && v[i] == most) {
                    v[i] = 0;
                    gone = true;
                }
        }
    }
}

// The most probable tokens of a CTA's share of a row, in two looks.  Every thread knows its largest logit from the sums' pass.
// The `top` groups of threads with the largest ones hold `top` tokens at least as large as the last of those, so all tokens
// looked for reach it: only the batches whose largest does are looked through again (a few in the hundred, from L2, or from
// registers where a thread had one batch), and what reaches it is ranked.  Where that is more than shared memory holds (many equal
// logits, or a few threads with most of the large ones), the threads' largest are told apart by their tokens, and then the tokens
// themselves are counted bit by bit.  Order: larger logit, then lower token; a token and its logit make one 64-bit key.
constexpr int kTopGroups = 64, kTopSlots = 16;               // slots: runs of a thread's batches whose largest is noted
template <int kT>
struct TopShared {
    static constexpr int kFound = kT >= 256 ? 1024 : 256;        // candidates that it holds
    uint32_t key[kT], first[kT];             // the threads' (first: groups') largest; the lowest tokens that have it
    uint32_t last, last_first;               // the last of the chosen threads' maxima, and the token up to which equal ones count
    int ties, need, n_chosen, n_found;
    uint16_t chosen[kT];                     // threads (up to 512), or slot * kT + thread
    float slot[kTopSlots][kT];
    uint64_t found[kFound], best[kLogpMaxTop];
};

template <int DT, int kT>
struct TopFinder {
    const char* row;
    RowSplit split;
    int64_t lo, hi, vocab;                   // the CTA's vectors
    bool edges;                              // the CTA has the elements outside the vectors
    uint32_t run;                            // batches of a slot
    TopShared<kT>* sh;

    // f(logit, token) for every element of thread t, the elements dealt to the lanes of the calling warp
    template <typename F>
    __device__ __forceinline__ void each(int t, F f) const {
        constexpr int kVec = Logits<DT>::kVec;
        const int lane = threadIdx.x & 31;
        const char* body = row + int64_t(split.head) * Logits<DT>::kSize;
        for (int64_t v = lo + t + int64_t(lane) * kT; v < hi; v += 32 * kT) {
            float x[kVec];
            Logits<DT>::vec(*reinterpret_cast<const uint4*>(body + v * 16), x);
#pragma unroll
            for (int j = 0; j < kVec; ++j) f(x[j], uint32_t(split.head + v * kVec + j));
        }
        if (edges && t < split.head + split.tail && lane == 0) {
            const int64_t j = split.edge(vocab, t);
            f(Logits<DT>::one(row, j), uint32_t(j));
        }
    }
    // of the CTA's chosen threads' elements, how many reach a key (all threads call it)
    __device__ __forceinline__ int count(uint64_t key) const {
        int n = 0;
        for (int c = threadIdx.x >> 5; c < sh->n_chosen; c += kT / 32)
            each(sh->chosen[c], [&](float x, uint32_t j) { n += Logits<DT>::key(x, j) >= key; });
        n = __reduce_add_sync(0xffffffffu, n);
        __syncthreads();
        if (threadIdx.x == 0) sh->n_found = 0;
        __syncthreads();
        if ((threadIdx.x & 31) == 0) atomicAdd(&sh->n_found, n);
        __syncthreads();
        return sh->n_found;
    }
    // their keys that reach `least` into found (all threads call it; n_found is zero): the vectors dealt out to all threads, four
    // in flight each
    __device__ __forceinline__ void take(float x, uint32_t j, uint64_t least) const {
        const uint64_t k = Logits<DT>::key(x, j);
        if (k >= least) {
            const int at = atomicAdd(&sh->n_found, 1);
            if (at < TopShared<kT>::kFound) sh->found[at] = k;
        }
    }
    __device__ __forceinline__ void take(const uint4& w, int64_t v, uint64_t least) const {
        constexpr int kVec = Logits<DT>::kVec;
        float x[kVec];
        Logits<DT>::vec(w, x);
#pragma unroll
        for (int j = 0; j < kVec; ++j) take(x[j], uint32_t(split.head + v * kVec + j), least);
    }
    __device__ __forceinline__ void take_edges(uint64_t least) const {
        if (edges && int(threadIdx.x) < split.head + split.tail) {
            const int64_t j = split.edge(vocab, threadIdx.x);
            take(Logits<DT>::one(row, j), uint32_t(j), least);
        }
    }
    template <bool kSlots>
    __device__ __forceinline__ void collect(uint64_t least) const {
        const char* body = row + int64_t(split.head) * Logits<DT>::kSize;
        const uint32_t per = kSlots ? run * kLogpBatch : uint32_t((hi - lo + kT - 1) / kT), all = uint32_t(sh->n_chosen) * per;
        for (uint32_t i = threadIdx.x; i < all; i += 4 * kT) {
            uint4 w[4];
            int64_t v[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const uint32_t at = i + u * kT, c = at / per;
                v[u] = hi;
                if (at < all) {
                    const uint32_t which = sh->chosen[c];
                    v[u] = lo + (which & (kT - 1)) + (int64_t(at - c * per) + (kSlots ? int64_t(which / kT) * per : 0)) * kT;
                }
                if (v[u] < hi) w[u] = *reinterpret_cast<const uint4*>(body + v[u] * 16);
            }
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (v[u] < hi) take(w[u], v[u], least);
        }
        take_edges(least);
        __syncthreads();
    }
    // n keys of `from` (n <= kFound), the largest `top` of them in descending order into best; zeros behind the last
    __device__ __forceinline__ static void rank(TopShared<kT>* sh, const uint64_t* from, int n, int top) {
        for (int i = threadIdx.x; i < top; i += kT)
            if (i >= n) sh->best[i] = 0;
        for (int i = threadIdx.x; i < n; i += kT) {
            const uint64_t k = from[i];
            int r = 0;
            for (int j = 0; j < n; ++j) r += from[j] > k;
            if (r < top) sh->best[r] = k;
        }
        __syncthreads();
    }
    // The keys that reach `least` of the chosen threads into found; all threads call it.
    __device__ __forceinline__ void gather(bool chosen, uint64_t least, const uint4 (&w)[kLogpBatch]) const {
        const int tid = threadIdx.x;
        if (hi - lo <= kLogpBatch * kT) {
            if (chosen) {
#pragma unroll
                for (int u = 0; u < kLogpBatch; ++u)
                    if (lo + tid + u * kT < hi) take(w[u], lo + tid + u * kT, least);
            }
            take_edges(least);
            __syncthreads();
        } else {
            if (chosen) {
                const uint32_t slots = (uint32_t((hi - lo - tid + kT - 1) / kT) + run * kLogpBatch - 1) / (run * kLogpBatch);
                for (uint32_t i = 0; i < slots; ++i)
                    if (Logits<DT>::key(sh->slot[i][tid]) >= uint32_t(least >> 32)) {
                        const int at = atomicAdd(&sh->n_chosen, 1);
                        if (at < kT) sh->chosen[at] = uint16_t(i * kT + tid);
                    }
            }
            __syncthreads();
            if (sh->n_chosen <= kT) collect<true>(least);
            else if (tid == 0) sh->n_found = TopShared<kT>::kFound + 1;      // (more than the list holds: the same as too many found)
            __syncthreads();
        }
    }
    // own: the thread's largest logit, has: it had any; w: its last vectors, which are all it had where the share has one batch of
    // them.  All threads call it; best is filled behind it.
    __device__ __forceinline__ void find(float own, bool has, int top, const uint4 (&w)[kLogpBatch]) const {
        constexpr int kGroups = kT < kTopGroups ? kT : kTopGroups, kMembers = kT / kGroups;
        const int tid = threadIdx.x, lane = tid & 31;
        const uint32_t mine = has ? Logits<DT>::key(own) : 0u;
        uint32_t group = mine;
#pragma unroll
        for (int o = 1; o < kMembers; o <<= 1) group = max(group, __shfl_xor_sync(0xffffffffu, group, o));
        if (tid % kMembers == 0) sh->first[tid / kMembers] = group;
        if (tid == 0) sh->n_chosen = sh->n_found = 0;
        __syncthreads();
        if (tid < 32) {
            uint32_t v[kGroups / 32];
#pragma unroll
            for (int i = 0; i < kGroups / 32; ++i) v[i] = sh->first[i * 32 + lane];
            const uint32_t last = top <= kTopByMaxima ? reached_by_maxima(v, top) : reached_by(v, top, Logits<DT>::kKeyBit);
            if (lane == 0) sh->last = last;
        }
        __syncthreads();
        const uint32_t bound = sh->last;
        gather(has && mine >= bound, uint64_t(bound) << 32, w);
        if (sh->n_found > TopShared<kT>::kFound) find_exact(mine, has, top);
        rank(sh, sh->found, min(sh->n_found, TopShared<kT>::kFound), top);
    }
    // As few threads as tokens are looked for, and then, if some hold many, the exact key of the last of these.
    __device__ __noinline__ void find_exact(uint32_t mine, bool has, int top) const {
        const int tid = threadIdx.x, lane = tid & 31;
        __syncthreads();
        sh->key[tid] = mine;
        sh->first[tid] = 0;
        if (tid == 0) sh->n_chosen = sh->n_found = 0;
        __syncthreads();
        if (tid < 32) {
            uint32_t v[kT / 32];
#pragma unroll
            for (int i = 0; i < kT / 32; ++i) v[i] = sh->key[i * 32 + lane];
            const uint32_t last = reached_by(v, top, Logits<DT>::kKeyBit);
            int above = 0, equal = 0;
#pragma unroll
            for (int i = 0; i < kT / 32; ++i) {
                above += v[i] > last;
                equal += v[i] == last;
            }
            above = __reduce_add_sync(0xffffffffu, above);
            equal = __reduce_add_sync(0xffffffffu, equal);
            if (lane == 0) {
                sh->last = last;
                sh->need = top - above;
                sh->ties = last != 0 && above + equal > top;
                sh->last_first = 0xffffffffu;
            }
        }
        __syncthreads();
        const uint32_t last = sh->last;
        const int ties = sh->ties;
        if (ties) {                          // more threads than looked for: of the equal ones, those with the lowest tokens
            for (int t = tid >> 5; t < kT; t += kT / 32) {
                if (sh->key[t] != last) continue;
                uint32_t first = 0xffffffffu;
                each(t, [&](float x, uint32_t j) { if (Logits<DT>::key(x) == last) first = min(first, j); });
                first = __reduce_min_sync(0xffffffffu, first);
                if (lane == 0) sh->first[t] = ~first;
            }
            __syncthreads();
            if (tid < 32) {
                uint32_t v[kT / 32];
#pragma unroll
                for (int i = 0; i < kT / 32; ++i) v[i] = sh->first[i * 32 + lane];
                const uint32_t f = reached_by(v, sh->need, 0);
                if (lane == 0) sh->last_first = ~f;
            }
            __syncthreads();
        }
        const bool chosen = has && (mine > last || (mine == last && (!ties || ~sh->first[tid] <= sh->last_first)));
        if (chosen) sh->chosen[atomicAdd(&sh->n_chosen, 1)] = uint16_t(tid);
        __syncthreads();
        collect<false>(last == 0 ? 0 : uint64_t(last) << 32 | uint32_t(~sh->last_first));
        if (sh->n_found > TopShared<kT>::kFound) {
            uint64_t t = 0;
            for (int bit = 63; bit >= 0; --bit)
                if (count(t | uint64_t(1) << bit) >= top) t |= uint64_t(1) << bit;
            __syncthreads();
            if (tid == 0) sh->n_found = 0;
            __syncthreads();
            collect<false>(t);
        }
    }
};

// One row per cluster of kC CTAs, kT threads each.
template <int DT, int kC, int kT, bool kTop>
__global__ void __launch_bounds__(kT) logp_kernel(const LogpArgs g) {
    namespace cg = cooperative_groups;
    __shared__ Sums warp_sums[kT / 32], cta_sums;
    __shared__ typename std::conditional<kTop, TopShared<kT>, int>::type top_shared;
    begin_in_row();
    const int tid = threadIdx.x, lane = tid & 31, part = kC > 1 ? int(blockIdx.x % kC) : 0;
    const int64_t row = blockIdx.x / kC, vocab = g.vocab;
    const char* x = g.logits + row * g.step;
    const RowSplit split = RowSplit::of<DT>(x, vocab);
    const int64_t lo = split.vecs * part / kC, hi = split.vecs * (part + 1) / kC;
    const char* body = x + int64_t(split.head) * Logits<DT>::kSize;
    const int64_t id = given_token(g.ids, g.id_bits, row);
    if (id < 0 || id >= vocab) {             // (alike in all CTAs of the cluster)
        if (part == 0) {
            if (tid == 0) g.logp[row] = g.entropy[row] = 0.f;
            if (tid < 3) g.stats[row * 3 + tid] = 0.f;
            if (tid < g.top) { g.top_ids[row * g.top + tid] = -1; g.top_logp[row * g.top + tid] = 0.f; }
        }
        return;
    }
    const float a = g.scale * kLog2e;
    ThreadSums<DT> own;
    bool has = lo + tid < hi;
    if (part == 0 && tid < split.head + split.tail) {
        has = true;
        own.one(Logits<DT>::one(x, split.edge(vocab, tid)), a);
    }
    // whole batches, one requested while the one before is summed; the last one may have fewer vectors
    const int64_t left = hi - lo - tid;
    int64_t batches = left > 0 ? (left + kT - 1) / kT : 0;       // (vectors of this thread)
    const int last = batches == 0 ? 0 : int((batches - 1) % kLogpBatch) + 1;
    batches = (batches + kLogpBatch - 1) / kLogpBatch;
    uint4 w[kLogpBatch];
    const char* at = body + (lo + tid) * 16;
    auto load = [&](uint4 (&to)[kLogpBatch], int n) {
#pragma unroll
        for (int u = 0; u < kLogpBatch; ++u) to[u] = ld_stream_u4(at + (u < n ? u : 0) * (kT * 16));
        at += kLogpBatch * kT * 16;
    };
    // (the largest of every run of batches is noted where the most probable tokens are looked for)
    const uint32_t run = uint32_t((hi - lo + int64_t(kLogpBatch * kTopSlots) * kT - 1) / (int64_t(kLogpBatch * kTopSlots) * kT));
    uint32_t in_run = 0, slot = 0;
    float slot_max = -INFINITY;
    auto sum_up = [&](int n, bool end) {
        const float most = own.batch(w, n, a);
        if constexpr (kTop) {
            slot_max = max_nan(slot_max, most);
            if (++in_run == run || end) {
                top_shared.slot[slot++][tid] = slot_max;
                slot_max = -INFINITY;
                in_run = 0;
            }
        }
    };
    if (batches > 0) load(w, batches == 1 ? last : kLogpBatch);
    for (int64_t i = 1; i < batches; ++i) {
        uint4 next[kLogpBatch];
        load(next, i == batches - 1 ? last : kLogpBatch);
        sum_up(kLogpBatch, false);
#pragma unroll
        for (int u = 0; u < kLogpBatch; ++u) w[u] = next[u];
    }
    if (batches > 0) sum_up(last, true);
    Sums sum = own.total();
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
        sum.join(Sums{__shfl_xor_sync(0xffffffffu, sum.m, o), __shfl_xor_sync(0xffffffffu, sum.s, o), __shfl_xor_sync(0xffffffffu, sum.q, o)}, a);
    if (lane == 0) warp_sums[tid >> 5] = sum;
    if constexpr (kTop) {
        TopFinder<DT, kT>{x, split, lo, hi, vocab, part == 0, run, &top_shared}.find(own.m, has, g.top, w);
    } else {
        __syncthreads();
    }
    if (tid == 0) {
        Sums all = warp_sums[0];
        for (int w = 1; w < kT / 32; ++w) all.join(warp_sums[w], a);
        cta_sums = all;
    }
    if constexpr (kC > 1) {
        cg::cluster_group cluster = cg::this_cluster();
        cluster.sync();
        if (part == 0) {
            if (tid == 0)
                for (int c = 1; c < kC; ++c) cta_sums.join(*cluster.map_shared_rank(&cta_sums, c), a);
            if constexpr (kTop) {
                for (int i = tid; i < kC * g.top; i += kT) top_shared.found[i] = cluster.map_shared_rank(&top_shared, i / g.top)->best[i % g.top];
                __syncthreads();
                TopFinder<DT, kT>::rank(&top_shared, top_shared.found, kC * g.top, g.top);
            }
        }
        cluster.sync();                      // (the others' shared memory is read up to here)
        if (part) return;
    }
    __syncthreads();
    const Sums all = cta_sums;
    const bool empty = all.m == -INFINITY, broken = !(all.m < INFINITY);    // nothing but -inf; a NaN or an infinite logit
    const float log_sum = empty ? 0.f : (broken ? NAN : logf(all.s));
    if (tid == 0) {
        const float h = empty ? 0.f : (broken ? NAN : log_sum - kLn2 * (all.q / all.s));
        g.logp[row] = empty ? -INFINITY : g.scale * (Logits<DT>::one(x, id) - all.m) - log_sum;
        g.entropy[row] = h;
        g.stats[row * 3] = all.m;
        g.stats[row * 3 + 1] = log_sum;
        g.stats[row * 3 + 2] = h;
    }
    if constexpr (kTop) {
        if (tid < g.top) {
            const uint64_t k = top_shared.best[tid];
            g.top_ids[row * g.top + tid] = int32_t(~uint32_t(k));
            g.top_logp[row * g.top + tid] = empty ? -INFINITY : g.scale * (Logits<DT>::value(uint32_t(k >> 32)) - all.m) - log_sum;
        }
    }
}

struct LogpGradArgs {
    const char* logits;
    const void* ids;
    const float *stats, *dlogp, *dentropy;
    char* out;
    int id_bits, segments;
    int64_t vocab, step, out_step;
    float scale;
};

// One segment of kLogpBatch vectors per thread of one row per CTA.  kWide: logits and their gradient lie alike to 16 bytes.
template <int DT, bool kWide>
__global__ void __launch_bounds__(kThreads) logp_grad_kernel(const LogpGradArgs g) {
    constexpr int kVec = Logits<DT>::kVec, kSize = Logits<DT>::kSize;
    begin_in_row();
    const int tid = threadIdx.x;
    const int64_t row = blockIdx.x / g.segments;
    const int seg = int(blockIdx.x - row * g.segments);
    const char* x = g.logits + row * g.step;
    char* out = g.out + row * g.out_step;
    RowSplit split = RowSplit::of<DT>(x, g.vocab);
    const int64_t first = int64_t(seg) * kLogpBatch * kThreads + tid;
    const int64_t id = given_token(g.ids, g.id_bits, row);
    const bool kept = id >= 0 && id < g.vocab;
    const char* body = x + int64_t(split.head) * kSize;
    uint4 w[kLogpBatch];
    if (kWide && kept) {
#pragma unroll
        for (int u = 0; u < kLogpBatch; ++u)
            if (first + u * kThreads < split.vecs) w[u] = ld_stream_u4(body + (first + u * kThreads) * 16);
    }
    const float most = g.stats[row * 3], log_sum = g.stats[row * 3 + 1], gl = g.dlogp[row] * g.scale;
    const float gh = g.dentropy ? g.dentropy[row] * g.scale : 0.f;
    const bool empty = most == -INFINITY || !kept;
    const float a = g.scale * kLog2e, b = log_sum * kLog2e;
    // -p (g + h (H + log p)) as p (c0 + c1 u) with u = log2 p
    const float c0 = gh != 0.f ? -(gl + gh * g.stats[row * 3 + 2]) : -gl, c1 = -gh * kLn2;
    auto one = [&](float y) {
        if (empty) return 0.f;
        float u = a * (y - most) - b;
        u = u < kLeastExponent ? kLeastExponent : u;            // (a NaN stays)
        return exp2_approx(u) * (c0 + c1 * u);
    };
    auto store = [&](int64_t j, float r) {
        if constexpr (DT == BAOC_BF16) {
            uint16_t h;
            asm("cvt.rn.bf16.f32 %0, %1;" : "=h"(h) : "f"(r));
            *reinterpret_cast<uint16_t*>(out + 2 * j) = h;
        } else {
            *reinterpret_cast<float*>(out + 4 * j) = r;
        }
    };
    if constexpr (kWide) {
        char* to = out + int64_t(split.head) * kSize;
#pragma unroll
        for (int u = 0; u < kLogpBatch; ++u) {
            const int64_t v = first + u * kThreads;
            if (v >= split.vecs) break;
            float y[kVec];
            if (!kept) w[u] = make_uint4(0, 0, 0, 0);
            Logits<DT>::vec(w[u], y);
#pragma unroll
            for (int j = 0; j < kVec; ++j) y[j] = one(y[j]);
            const int64_t d = id - split.head - v * kVec;
            if (d >= 0 && d < kVec && !empty) {
#pragma unroll
                for (int j = 0; j < kVec; ++j) y[j] += j == d ? gl : 0.f;
            }
            uint4 r;
            if constexpr (DT == BAOC_BF16) {
                asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r.x) : "f"(y[1]), "f"(y[0]));
                asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r.y) : "f"(y[3]), "f"(y[2]));
                asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r.z) : "f"(y[5]), "f"(y[4]));
                asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r.w) : "f"(y[7]), "f"(y[6]));
            } else {
                r = make_uint4(__float_as_uint(y[0]), __float_as_uint(y[1]), __float_as_uint(y[2]), __float_as_uint(y[3]));
            }
            st_stream_u4(to + v * 16, r);
        }
        if (seg == 0 && tid < split.head + split.tail) {
            const int64_t j = split.edge(g.vocab, tid);
            store(j, (kept ? one(Logits<DT>::one(x, j)) : 0.f) + (j == id && !empty ? gl : 0.f));
        }
    } else {
        const int64_t lo = int64_t(seg) * kLogpBatch * kThreads * kVec;
        const int64_t hi = min64(g.vocab, lo + int64_t(kLogpBatch) * kThreads * kVec);
        for (int64_t j = lo + tid; j < hi; j += kThreads)
            store(j, (kept ? one(Logits<DT>::one(x, j)) : 0.f) + (j == id && !empty ? gl : 0.f));
    }
}

namespace {

thread_local std::string g_logp_err;

int fail_logp(int code, const std::string& msg) {
    g_logp_err = msg;
    return code;
}
int64_t elem_bytes(int dtype) { return dtype == BAOC_F32 ? 4 : 2; }
bool aligned(const void* p, int64_t bytes) { return (reinterpret_cast<uintptr_t>(p) & uintptr_t(bytes - 1)) == 0; }

int check_logp(const baoc_logp_t* e, int64_t n, const std::string& what) {
    if (!e) return fail_logp(BAOC_E_INVALID, what + ": null descriptor");
    if (e->vocab < 1 || e->vocab > 0x7fffffff) return fail_logp(BAOC_E_INVALID, what + ": vocab must be in 1 .. 2^31 - 1");
    if (e->dtype != BAOC_BF16 && e->dtype != BAOC_F32) return fail_logp(BAOC_E_INVALID, what + ": dtype must be BAOC_BF16 or BAOC_F32");
    if (e->id_bits != 32 && e->id_bits != 64) return fail_logp(BAOC_E_INVALID, what + ": id_bits must be 32 or 64");
    if (!(e->scale > 0.f) || !(e->scale <= kLogpMaxScale)) return fail_logp(BAOC_E_INVALID, what + ": scale must be above zero and at most 2^127");
    if (e->top < 0 || e->top > kLogpMaxTop || e->top > e->vocab) return fail_logp(BAOC_E_INVALID, what + ": top must be in 0 .. 32 and at most vocab");
    for (int64_t s : {e->stride, e->grad_stride})
        if (s && (s < e->vocab || s > kLogpMaxStride)) return fail_logp(BAOC_E_INVALID, what + ": a row stride must be 0 or in vocab .. 2^32");
    if (n < 0 || n > 0x7fffffff) return fail_logp(BAOC_E_INVALID, what + ": n_tokens must be in 0 .. 2^31 - 1");
    return BAOC_OK;
}

// n rows of `row` bytes, `step` bytes apart.
struct Extent {
    const void* p;
    int64_t n, step, row;
};
Extent vector_of(const void* p, int64_t n, int64_t elem) { return Extent{p, 1, n * elem, n * elem}; }
// Whether two arrays share bytes.  (Rows of one buffer may lie between each other's, a vector behind the columns of a row.)
bool overlap(const Extent& a, const Extent& b) {
    if (!a.p || !b.p || a.n == 0 || b.n == 0) return false;
    if (a.n == 1 && b.n > 1) return overlap(b, a);
    const char *x = static_cast<const char*>(a.p), *y = static_cast<const char*>(b.p);
    if (x >= y + (b.n - 1) * b.step + b.row || y >= x + (a.n - 1) * a.step + a.row) return false;
    if (b.n > 1 && a.step != b.step) return true;
    const int64_t off = ((y - x) % a.step + a.step) % a.step;
    return off < a.row || off + b.row > a.step;
}

template <int DT, int kC, int kT>
int launch_logp(const LogpArgs& a, int64_t n, cudaStream_t s) {
    if (n * kC > 0x7fffffff) return fail_logp(BAOC_E_INVALID, "baoc_logp: too many rows for one launch");
    const cudaError_t ce = launch_in_row(a.top ? logp_kernel<DT, kC, kT, true> : logp_kernel<DT, kC, kT, false>, dim3(unsigned(n * kC)), kT, 0, kC, s, a);
    return ce == cudaSuccess ? BAOC_OK : fail_logp(BAOC_E_CUDA, std::string("logp_kernel: ") + cudaGetErrorString(ce));
}

// Few rows: each is shared by a cluster.  Else one CTA a row, of fewer threads where rows are short: a CTA's barriers and the
// search for the most probable tokens cost the same for any row (65536 x 1000 with five of them: 128 us with a warp each, 650 with 256 threads; 8192 x 50257, a third masked: 146 us with 128
// threads, 165 with 256).
template <int DT>
int logp_of(const LogpArgs& a, int64_t n, cudaStream_t s) {
    int c = 1;
    while (c < kLogpMostCtas && n * c * 2 <= 2 * 148 && a.vocab >= int64_t(c) * 2 * kLogpCtaLogits) c *= 2;
    switch (c) {
        case 2: return launch_logp<DT, 2, 512>(a, n, s);
        case 4: return launch_logp<DT, 4, 512>(a, n, s);
        case 8: return launch_logp<DT, 8, 512>(a, n, s);
        default: break;
    }
    const int64_t vecs = a.vocab / Logits<DT>::kVec;
    if (vecs <= kLogpShort * 32) return launch_logp<DT, 1, 32>(a, n, s);
    if (vecs <= kLogpShort * 128) return launch_logp<DT, 1, 128>(a, n, s);
    return launch_logp<DT, 1, 256>(a, n, s);
}

}  // namespace

}  // namespace baoc

using namespace baoc;

extern "C" {

const char* baoc_logp_last_error(void) { return g_logp_err.c_str(); }

int baoc_logp(const baoc_logp_t* e, const void* logits, const void* ids, int64_t n_tokens, float* logp, float* entropy, float* stats,
              int32_t* top_ids, float* top_logp, baoc_stream_t stream) try {
    const int rc = check_logp(e, n_tokens, "baoc_logp");
    if (rc) return rc;
    if (n_tokens == 0) return BAOC_OK;
    if (!logits || !ids || !logp || !entropy || !stats || (e->top && (!top_ids || !top_logp))) return fail_logp(BAOC_E_INVALID, "baoc_logp: null pointer");
    const int64_t eb = elem_bytes(e->dtype), stride = e->stride ? e->stride : e->vocab;
    if (!aligned(logits, eb) || !aligned(ids, e->id_bits / 8) || !aligned(logp, 4) || !aligned(entropy, 4) || !aligned(stats, 4) ||
        (e->top && (!aligned(top_ids, 4) || !aligned(top_logp, 4))))
        return fail_logp(BAOC_E_ALIGN, "baoc_logp: a pointer is not aligned to its elements");
    const Extent ins[] = {{logits, n_tokens, stride * eb, e->vocab * eb}, vector_of(ids, n_tokens, e->id_bits / 8)},
                 outs[] = {vector_of(logp, n_tokens, 4), vector_of(entropy, n_tokens, 4), vector_of(stats, n_tokens * 3, 4),
                           vector_of(e->top ? top_ids : nullptr, n_tokens * e->top, 4), vector_of(e->top ? top_logp : nullptr, n_tokens * e->top, 4)};
    for (const Extent& o : outs) {
        for (const Extent& i : ins)
            if (overlap(o, i)) return fail_logp(BAOC_E_INVALID, "baoc_logp: an output overlaps another array");
        for (const Extent* q = outs; q != &o; ++q)
            if (overlap(o, *q)) return fail_logp(BAOC_E_INVALID, "baoc_logp: an output overlaps another array");
    }
    const LogpArgs a{static_cast<const char*>(logits), ids, e->id_bits, e->top, e->vocab, stride * eb, e->scale, logp, entropy, stats, top_ids, top_logp};
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    return e->dtype == BAOC_BF16 ? logp_of<BAOC_BF16>(a, n_tokens, s) : logp_of<BAOC_F32>(a, n_tokens, s);
} catch (const std::bad_alloc&) {
    return BAOC_E_INVALID;
}

int baoc_logp_grad(const baoc_logp_t* e, const void* logits, const void* ids, const float* stats, const float* dlogp, const float* dentropy,
                   int64_t n_tokens, void* dlogits, baoc_stream_t stream) try {
    const int rc = check_logp(e, n_tokens, "baoc_logp_grad");
    if (rc) return rc;
    if (n_tokens == 0) return BAOC_OK;
    if (!logits || !ids || !stats || !dlogp || !dlogits) return fail_logp(BAOC_E_INVALID, "baoc_logp_grad: null pointer");
    const int64_t eb = elem_bytes(e->dtype), step = (e->stride ? e->stride : e->vocab) * eb, out_step = (e->grad_stride ? e->grad_stride : e->vocab) * eb;
    if (!aligned(logits, eb) || !aligned(dlogits, eb) || !aligned(ids, e->id_bits / 8) || !aligned(stats, 4) || !aligned(dlogp, 4) || !aligned(dentropy, 4))
        return fail_logp(BAOC_E_ALIGN, "baoc_logp_grad: a pointer is not aligned to its elements");
    const char* x = static_cast<const char*>(logits);
    char* d = static_cast<char*>(dlogits);
    const int64_t row = e->vocab * eb;
    const Extent to{d, n_tokens, out_step, row};
    if (overlap(to, Extent{x, n_tokens, step, row}) && !(x == d && (step == out_step || n_tokens == 1)))
        return fail_logp(BAOC_E_INVALID, "baoc_logp_grad: dlogits overlaps logits and is not the same array");
    for (const Extent& v : {vector_of(ids, n_tokens, e->id_bits / 8), vector_of(stats, n_tokens * 3, 4), vector_of(dlogp, n_tokens, 4), vector_of(dentropy, n_tokens, 4)})
        if (overlap(to, v)) return fail_logp(BAOC_E_INVALID, "baoc_logp_grad: dlogits overlaps an array of one value per token");
    const int64_t segments = ceil_div(row, int64_t(16) * kLogpBatch * kThreads);
    if (n_tokens * segments > 0x7fffffff) return fail_logp(BAOC_E_INVALID, "baoc_logp_grad: too many logits for one launch");
    const LogpGradArgs a{x, ids, stats, dlogp, dentropy, d, e->id_bits, int(segments), e->vocab, step, out_step, e->scale};
    const bool wide = ((d - x) & 15) == 0 && ((out_step - step) & 15) == 0;
    const unsigned grid = unsigned(n_tokens * segments);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const auto kernel = e->dtype == BAOC_BF16 ? (wide ? logp_grad_kernel<BAOC_BF16, true> : logp_grad_kernel<BAOC_BF16, false>)
                                              : (wide ? logp_grad_kernel<BAOC_F32, true> : logp_grad_kernel<BAOC_F32, false>);
    const cudaError_t ce = launch_in_row(kernel, dim3(grid), kThreads, 0, 1, s, a);
    return ce == cudaSuccess ? BAOC_OK : fail_logp(BAOC_E_CUDA, std::string("logp_grad_kernel: ") + cudaGetErrorString(ce));
} catch (const std::bad_alloc&) {
    return BAOC_E_INVALID;
}

}  // extern "C"
