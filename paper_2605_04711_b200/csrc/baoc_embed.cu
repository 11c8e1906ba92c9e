// The token table: row lookup with scaling, and its gradient by grouped tokens.
//
//   out[t, :]    = scale * table[ids[t], :]
//   dtable[v, :] = scale * sum over t with ids[t] = v of dout[t, :]
//
// Both move rows and compute next to nothing, so memory bounds them: the lookup reads the distinct rows and writes n rows, the
// gradient reads the named rows of dout once and writes every row of dtable once.  The gradient has no atomics on data: the
// tokens are first grouped by id (integers only), then every row is summed in a fixed order, so equal inputs give equal bits.
// Times below: one B200, device time per call in a row of calls on three sets of arrays.
#include <algorithm>
#include <atomic>
#include <cmath>
#include <cooperative_groups.h>
#include <cuda_runtime.h>
#include <new>
#include <string>

#include "baoc_device.cuh"

namespace baoc {

constexpr int kGroupCtas = 128;        // id classes (one CTA each) of the grouping; doubled while a class has over kGroupBins ids
constexpr int kGroupBins = 768;        // most ids of a class: one thread of the CTA per id, and what shared memory holds
constexpr int kGroupWarps = 32;
constexpr int kGroupSplit = 4;         // CTAs that share the reading of the ids,
constexpr int64_t kSplitTokens = 32768; // from this many tokens on
constexpr int kIdLoads = 16;           // ids a lane of the grouping has in flight
constexpr int kListed = 512;           // tokens a warp of the grouping can list; when it finds more it reads the ids again
constexpr int kSeen = 256;             // the same for what a warp finds of all classes of a cluster
constexpr int kListBits = 22;          // bits of a token's offset in a list entry (the id of the class, below kGroupBins, has the others)
constexpr int kShortRow = 32;          // tokens of a row that one warp sums by itself; longer rows are cut into chunks
constexpr int kMostChunks = 512;
constexpr int kJoin = 16;              // chunks whose partial sums one warp adds; a longer row's are added in two levels
constexpr int kSlotWarps = 16;         // warps that share a run of 32 slots
constexpr int kSlotTokens = 16;        // places of the grouped order per slot of the chunk list
constexpr int kSegShift = 5;           // log2 of the rows and tokens, together, of a segment of the sums: one row per lane at most,
constexpr int kSegShiftLeast = 3;      // fewer while there are not
constexpr int kSegWarps = 24 * 148;    // as many segments' slabs as warps that the GPU holds
// The one-kernel gradient takes at most one token per thread of a CTA, and at most so many bytes of dout: one CTA may have to
// add them all up.  Against two kernels: 256 tokens x 256 into 4096 rows 3.4 us (8.5), 64 x 257 fp32 into 1000 rows 2.9 (9.4),
// 4 x 1280 into 41212 rows 16.4 (25.1), 64 x 2048 into 32000 rows 20.9 (25.9); all tokens alike it loses from 128 tokens on
// (128 x 2048 into 32000 rows 27.3 against 25.6, 256 x 256 into 4096 rows 19.9 against 11.6).  Large tables want their rows
// dealt to more CTAs than find room at once (64 x 2048 into 32000 rows: 20.9 us, 24.6 with kFewCtas), small ones do not
// (256 x 512 into 16384 rows: 6.2 us, 8.9 with kFewCtasLarge).
constexpr int kFewTokens = kThreads;
constexpr int64_t kFewBytes = 512 << 10;
constexpr int64_t kFewLargeTable = 32 << 20;           // bytes of dtable from which the rows are dealt to more CTAs
constexpr int kFewCtas = 8 * 148, kFewCtasLarge = 24 * 148;
constexpr int kEmbedMaxDim = 1 << 24;
constexpr int64_t kEmbedMaxStride = 1 << 28;           // (row products stay far inside 64 bits)

__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

// Loads of rows, requested ahead of their use.  Their uses below stand on every path that follows: a use behind a test of
// its own would let the compiler move the request behind that test.
__device__ __forceinline__ uint4 ld_row_u4(const void* p) {
    uint4 r;
    asm volatile("ld.global.nc.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "l"(p));
    return r;
}
__device__ __forceinline__ uint2 ld_row_u2(const void* p) {
    uint2 r;
    asm volatile("ld.global.nc.v2.u32 {%0,%1}, [%2];" : "=r"(r.x), "=r"(r.y) : "l"(p));
    return r;
}
__device__ __forceinline__ uint32_t ld_row_u1(const void* p) {
    uint32_t r;
    asm volatile("ld.global.nc.u32 %0, [%1];" : "=r"(r) : "l"(p));
    return r;
}
__device__ __forceinline__ uint32_t ld_row_bf16(const void* p) {
    uint16_t r;
    asm volatile("ld.global.nc.u16 %0, [%1];" : "=h"(r) : "l"(p));
    return r;
}

// What the kernels take of a descriptor.  Row strides in bytes: 32 bits hold them, and a row's offset is one product.
struct EmbedArgs {
    uint32_t src_step, dst_step;
    int dim;
    float scale;
};

// A warp works on 32 * V columns (a slab) of a row.  How a lane's V columns lie depends on what base, row stride and dim of
// both arrays allow: kWide, V neighbours (16-byte accesses); kPairs, V / 2 pairs that are 64 columns apart; kSingles, V columns
// that are 32 apart.  V = 8 for dim > 128, 4 for dim > 64, else 2: a narrower table leaves fewer lanes idle.
enum Access : int { kSingles = 0, kPairs = 1, kWide = 2 };
template <int V, int M>
__device__ __forceinline__ constexpr int column_of(int j) { return M == kWide ? j : (M == kPairs ? 64 * (j / 2) + j % 2 : 32 * j); }

template <int DT, int V, int M>
struct Part {
    static constexpr int kSize = DT == BAOC_BF16 ? 2 : 4;
    static constexpr int kWords = M == kSingles ? V : V * kSize / 4;
    uint32_t w[kWords];

    // p: the lane's first column; last: bytes from there to the last column (pair) that the row can be read at
    __device__ __forceinline__ void load(const char* p, int last) {
        if constexpr (M == kWide) {
            if constexpr (kWords == 1) w[0] = ld_row_u1(p);
            if constexpr (kWords == 2) { const uint2 a = ld_row_u2(p); w[0] = a.x; w[1] = a.y; }
            if constexpr (kWords >= 4) { const uint4 a = ld_row_u4(p); w[0] = a.x; w[1] = a.y; w[2] = a.z; w[3] = a.w; }
            if constexpr (kWords == 8) { const uint4 a = ld_row_u4(p + 16); w[4] = a.x; w[5] = a.y; w[6] = a.z; w[7] = a.w; }
        } else if constexpr (M == kPairs) {
#pragma unroll
            for (int j = 0; j < V / 2; ++j) {
                const char* q = p + min(j * 64 * kSize, last);
                if constexpr (DT == BAOC_BF16) {
                    w[j] = ld_row_u1(q);
                } else {
                    const uint2 a = ld_row_u2(q);
                    w[2 * j] = a.x;
                    w[2 * j + 1] = a.y;
                }
            }
        } else {
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const char* q = p + min(j * 32 * kSize, last);
                if constexpr (DT == BAOC_BF16) w[j] = ld_row_bf16(q) << 16;
                else w[j] = ld_row_u1(q);
            }
        }
    }
    __device__ __forceinline__ float at(int j) const {
        if constexpr (M != kSingles && DT == BAOC_BF16) return (j & 1) ? bf16_hi(w[j >> 1]) : bf16_lo(w[j >> 1]);
        else return __uint_as_float(w[j]);
    }
};

// The lane's first column, and the one that it reads from: columns beyond the row read its last ones instead.
template <int V, int M>
__device__ __forceinline__ int lane_col(int slab, int lane) { return slab * 32 * V + lane * (M == kWide ? V : (M == kPairs ? 2 : 1)); }
template <int V, int M>
__device__ __forceinline__ constexpr int run_of() { return M == kWide ? V : (M == kPairs ? 2 : 1); }      // neighbours that are read together
template <int V, int M>
__device__ __forceinline__ int read_col(int col, int dim) { return min(col, dim - run_of<V, M>()); }
template <int V, int M>
__device__ __forceinline__ int last_read(int rc, int dim, int size) { return (dim - run_of<V, M>() - rc) * size; }

// V values of a lane into a row (p: the lane's first column).
template <int DT, int V, int M>
__device__ __forceinline__ void store_part(char* p, int col, int dim, const float (&y)[V]) {
    if constexpr (M == kWide) {
        if (col >= dim) return;
        if constexpr (DT == BAOC_BF16) {
            if constexpr (V == 8) st_stream_u4(p, make_uint4(bf16_pair(y[0], y[1]), bf16_pair(y[2], y[3]), bf16_pair(y[4], y[5]), bf16_pair(y[6], y[7])));
            if constexpr (V == 4) st_stream_u2(p, make_uint2(bf16_pair(y[0], y[1]), bf16_pair(y[2], y[3])));
            if constexpr (V == 2) *reinterpret_cast<uint32_t*>(p) = bf16_pair(y[0], y[1]);
        } else {
            if constexpr (V >= 4) st_stream_f4(p, make_float4(y[0], y[1], y[2], y[3]));
            if constexpr (V == 8) st_stream_f4(p + 16, make_float4(y[4], y[5], y[6], y[7]));
            if constexpr (V == 2) *reinterpret_cast<float2*>(p) = make_float2(y[0], y[1]);
        }
    } else if constexpr (M == kPairs) {
#pragma unroll
        for (int j = 0; j < V / 2; ++j) {
            if (col + 64 * j < dim) {
                if constexpr (DT == BAOC_BF16) reinterpret_cast<uint32_t*>(p)[32 * j] = bf16_pair(y[2 * j], y[2 * j + 1]);
                else reinterpret_cast<float2*>(p)[32 * j] = make_float2(y[2 * j], y[2 * j + 1]);
            }
        }
    } else {
#pragma unroll
        for (int j = 0; j < V; ++j) {
            if (col + 32 * j < dim) {
                if constexpr (DT == BAOC_BF16) reinterpret_cast<uint16_t*>(p)[32 * j] = uint16_t(bf16_pair(y[j], 0.f));
                else reinterpret_cast<float*>(p)[32 * j] = y[j];
            }
        }
    }
}

// A token id's low word, and whether it names a row.
__device__ __forceinline__ bool is_row(int32_t id, uint32_t vocab) { return uint32_t(id) < vocab; }
__device__ __forceinline__ bool is_row(int64_t id, uint32_t vocab) { return uint32_t(uint64_t(id) >> 32) == 0u && uint32_t(id) < vocab; }

// ---- lookup: one warp per slab of kTokens tokens, all of their loads in flight -----------------------------------------
// Two rows of fp32 or four of bf16 are 2 KB in flight per warp, in as many warps as an SM holds: with one load per thread and a
// division per element the same calls took 10.9 us (16384 x 768 of fp32, now 9.0: 4.9 TB/s of the distinct rows and the
// output), 175 us (131072 x 2048 of fp32, now 125: 5.6 TB/s) and 81 us (65536 x 2048 of bf16, now 53: 6.1 TB/s).  Twice the
// tokens in half the warps: 127 us for the second, 65 us instead of 54 for 32768 x 2047 (element by element); half the tokens:
// 160 and 57 us.  The fp32 table's repeated rows cross L2 once per use, which is what is left there.  One token: 1.9 us, a launch.
template <int SRC, int DST, int V, int M, typename Id>
__global__ void __launch_bounds__(kThreads, M == kWide ? 8 : 6)
embed_kernel(const char* __restrict__ table, const Id* __restrict__ ids, char* __restrict__ out, uint32_t vocab, int64_t n, int slabs,
             const EmbedArgs a) {
    using P = Part<SRC, V, M>;
    constexpr int kTokens = P::kWords == 8 ? 2 : 4;
    const int lane = threadIdx.x & 31;
    const uint32_t item = blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5);
    // fp32 tables go through slab by slab: a frequent row's kilobyte is then found in L1 (131072 tokens x 2048 of a Zipf-like
    // stream, four tokens a warp: 128 us, 140 token by token); rows of half that size go token by token (65536 x 2048 of bf16: 54 us, 58 slab by slab).
    constexpr bool kBySlab = SRC == BAOC_F32 && M == kWide;
    const uint32_t groups = uint32_t((n + kTokens - 1) / kTokens), per = kBySlab ? groups : uint32_t(slabs), q = item / per, r = item - q * per;
    const int slab = int(kBySlab ? q : r);
    const int64_t t0 = int64_t(kBySlab ? r : q) * kTokens;
    if (slab >= slabs || t0 >= n) return;
    const int m = int(min64(n - t0, kTokens));
    const Id own = __ldg(ids + t0 + min(lane, m - 1));
    const uint32_t row = is_row(own, vocab) ? uint32_t(own) : 0u, named = __ballot_sync(0xffffffffu, is_row(own, vocab));
    const int col = lane_col<V, M>(slab, lane), rc = read_col<V, M>(col, a.dim), last = last_read<V, M>(rc, a.dim, P::kSize);
    const char* src = table + int64_t(rc) * P::kSize;
    P x[kTokens];
#pragma unroll
    for (int i = 0; i < kTokens; ++i) x[i].load(src + uint64_t(__shfl_sync(0xffffffffu, row, i)) * a.src_step, last);
    char* dst = out + int64_t(col) * (DST == BAOC_BF16 ? 2 : 4) + t0 * a.dst_step;
#pragma unroll
    for (int i = 0; i < kTokens; ++i) {
        if (i >= m) break;
        float y[V];
#pragma unroll
        for (int j = 0; j < V; ++j) y[j] = named >> i & 1u ? x[i].at(j) * a.scale : 0.f;
        store_part<DST, V, M>(dst + int64_t(i) * a.dst_step, col, a.dim, y);
    }
}

// A row that `count` > kShortRow tokens name is cut into chunks of kShortRow tokens, or of the next power of two that leaves
// about kMostChunks of them; a rest of less than half a chunk goes to the last one.  Chunk k of a row takes slot
// ceil(start / kSlotTokens) + k * len / kSlotTokens: that slot begins inside the row, as the last chunk has at least
// len / 2 >= kSlotTokens tokens, so no two rows share a slot.
__host__ __device__ __forceinline__ int chunk_tokens(int count) {
    int len = kShortRow;
    while (int64_t(len) * kMostChunks < count) len <<= 1;
    return len;
}
__host__ __device__ __forceinline__ int chunks_of(int count, int len) { return int((int64_t(count) + len / 2) / len); }

// ---- gradient, first kernel: group the tokens by id -----------------------------------------------------------------
// Bound by instructions and latency, not by bytes (the ids come from L2): this kernel alone, launches in a row, takes 7.2 us
// for 16384 tokens, 11.3 us for 65536, 16.2 us for 131072 (ncu: issue slots half busy, DRAM idle).  Reading the ids by every
// class instead of sorting in passes over the GPU saves the grid-wide steps in between; a cluster of four shares the reading
// from kSplitTokens tokens on (8192: 7.4 us against 5.8 without, 16384: 7.7 against 7.2, 24576: 8.3 against 9.5, 32768: 9.0
// against 10.3, 65536: 11.3 against 15.3, 131072: 16.2 against 25.1), clusters of eight do not all find room at once (+ 18 us).
// These hold up to 128 * kGroupBins = 98304 rows (16384 tokens: 7.9 us there).  Beyond, the classes double and no longer run
// all at once: 16384 tokens into 128256 rows 12.5 us, into 256000 rows 22.1; 65536 tokens 18.5 and 32.8 (12.0 at 98304).
// The ids fall into 2^shift classes by their low bits; CTA c lists the tokens of class c, grouped by id.  Every CTA reads
// all ids and counts those of lower classes too, which is where its part of the order begins: no CTA waits for another,
// nothing is left to chance, and frequent neighbouring ids fall into different classes.
//
// Left for the sums, all in the workspace (a row's index is class * bins + id of the class):
struct GradBufs {
    int32_t* start;      // per row index: its first place in perm; one more at the end
    int32_t* perm;       // the tokens, grouped by id
    uint2* segs;         // per segment: {first row index, its start}; one more at the end
    int2* slots;         // chunks of the long rows: {row index, chunk}, or {-1, 0}
    uint32_t* tickets;   // [slot][slab][2]: chunks done of the kJoin whose first slot this is; such groups done of the row
    float* partial;      // [slot][slab][32 V]: a chunk's sum
    int shift, bins, slabs, seg_shift, n_segs, n_slots;
};

// Index of the last entry of the ascending a[0 .. n] that is <= x (a[0] <= x).
__device__ __forceinline__ int last_not_above(const int32_t* a, int n, int32_t x) {
    int lo = 0, hi = n;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (a[mid] <= x) lo = mid; else hi = mid - 1;
    }
    return lo;
}

// kSplit > 1: the CTAs of a cluster, kSplit neighbouring classes, read one part of the ids each for all of them and
// exchange what they have found through distributed shared memory.
template <typename Id, int kSplit>
__global__ void __launch_bounds__(kGroupWarps * 32)
embed_group_kernel(const Id* __restrict__ ids, int n, uint32_t vocab, uint32_t pad, const GradBufs b BAOC_CHECK_PARAM) {
    constexpr int kOffBits = kSplit > 1 ? kListBits - 3 : kListBits;      // a list entry: {id of the class, part or class, offset of the token}
    constexpr uint32_t kOffMask = (1u << kOffBits) - 1u;
    static_assert(kSplit <= 8, "three bits of a list entry");
    extern __shared__ int32_t smem[];
    let_later_kernel_start();
    int32_t* hist = smem;                                                        // [warps][bins]
    int32_t* begin = hist + kGroupWarps * b.bins;                                // [bins + 1]: start of the class's rows
    uint32_t* list = reinterpret_cast<uint32_t*>(begin + b.bins + 1);            // [warps][kListed] of the class; kSplit > 1: [warps][kSeen] of all
    __shared__ int32_t s_warp[kGroupWarps], s_found[kGroupWarps];
    __shared__ int32_t s_less, s_below;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, bins = b.bins, shift = b.shift;
    const uint32_t cls = blockIdx.x, mask = (1u << shift) - 1u, below = (1u << lane) - 1u;
    const uint32_t rank = kSplit > 1 ? cls % kSplit : 0u, cls0 = cls - rank;
    const int64_t row0 = int64_t(cls) * bins;
#ifdef BAOC_CHECKED
    // (the same ranges in every CTA: if one leaves, all of a cluster do)
    if (!check_range(ck, kKerEmbedGroup, b.start, 4 * ((int64_t(bins) << shift) + 1), 0) || !check_range(ck, kKerEmbedGroup, b.perm, 4ll * n, 1) ||
        !check_range(ck, kKerEmbedGroup, b.slots, 8ll * b.n_slots, 2) || !check_range(ck, kKerEmbedGroup, b.segs, 8ll * (b.n_segs + 1), 3) ||
        !check_range(ck, kKerEmbedGroup, b.tickets, 8ll * b.n_slots * b.slabs, 4))
        return;
#endif
    // part r of the tokens begins at r * part; of each, warp w has the stretch that begins w * seg further on
    const int part = (n + kSplit * 32 - 1) / (kSplit * 32) * 32;
    const int warps = max(1, min(kGroupWarps, (part + 32 * kIdLoads - 1) / (32 * kIdLoads)));
    const int seg = (part + warps * 32 - 1) / (warps * 32) * 32;
    auto stretch = [&](int r, int& t0, int& t1) {
        const int end = int(min64(int64_t(r + 1) * part, n));
        t0 = int(min64(int64_t(r) * part + int64_t(warp) * seg, end));
        t1 = warp < warps ? min(t0 + seg, end) : t0;
    };
    for (int i = threadIdx.x; i < warps * bins; i += blockDim.x) hist[i] = 0;
    if (threadIdx.x == 0) { s_less = 0; s_below = 0; }
    __syncthreads();
    int32_t* mine = hist + warp * bins;
    uint32_t* found = list + warp * kListed;
    // A warp's pass over a stretch, kIdLoads ids per lane at a time: take(class, id of the class, token, place) for every id
    // with want(class), where place numbers them from `from` on.  Returns the number behind the last one.
    auto pass = [&](int t0, int t1, int from, auto want, auto take) {
        for (int tb = t0; tb < t1; tb += 32 * kIdLoads) {
            Id id[kIdLoads];
            if (tb + 32 * kIdLoads <= t1) {
#pragma unroll
                for (int u = 0; u < kIdLoads; ++u) id[u] = __ldg(ids + tb + lane + 32 * u);
            } else {
#pragma unroll
                for (int u = 0; u < kIdLoads; ++u) id[u] = tb + lane + 32 * u < t1 ? __ldg(ids + tb + lane + 32 * u) : Id(-1);
            }
            uint32_t hits = 0;
#pragma unroll
            for (int u = 0; u < kIdLoads; ++u) {
                if (is_row(id[u], vocab) && uint32_t(id[u]) != pad && want(uint32_t(id[u]) & mask)) hits |= 1u << u;
            }
            if (!__any_sync(0xffffffffu, hits != 0u)) continue;
            const int k = __popc(hits);
            int upto = k;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int y = __shfl_up_sync(0xffffffffu, upto, o);
                if (lane >= o) upto += y;
            }
            int at = from + upto - k;
#pragma unroll
            for (int u = 0; u < kIdLoads; ++u)
                if (hits >> u & 1u) take(uint32_t(id[u]) & mask, uint32_t(id[u]) >> shift, tb + 32 * u + lane, at++);
            from += __shfl_sync(0xffffffffu, upto, 31);
        }
        return from;
    };
    int less = 0, n_found = 0, t0, t1;
    if constexpr (kSplit == 1) {
        stretch(0, t0, t1);
        n_found = pass(t0, t1, 0, [&](uint32_t c) { less += c < cls; return c == cls; },
                       [&](uint32_t, uint32_t bin, int t, int at) {
                           if (at < kListed) found[at] = bin << kListBits | uint32_t(t - t0);
                           atomicAdd(&mine[bin], 1);
                       });
    } else {
        namespace cg = cooperative_groups;
        cg::cluster_group cluster = cg::this_cluster();
        uint32_t* all = list + kGroupWarps * kListed + warp * kSeen;
        stretch(int(rank), t0, t1);
        const int seen = pass(t0, t1, 0, [&](uint32_t c) { less += c < cls0; return c - cls0 < uint32_t(kSplit); },
                              [&](uint32_t c, uint32_t bin, int t, int at) {
                                  if (at < kSeen) all[at] = bin << kListBits | (c - cls0) << kOffBits | uint32_t(t - t0);
                              });
        if (lane == 0) s_found[warp] = seg <= 1 << kOffBits ? seen : kSeen + 1;
        less = __reduce_add_sync(0xffffffffu, less);
        if (lane == 0 && less) atomicAdd(&s_below, less);
        less = 0;
        cluster.sync();
        // what all CTAs of the cluster have listed for this class; tokens of the cluster's lower classes count as less
        const int theirs = lane < kSplit ? *cluster.map_shared_rank(s_found + warp, lane) : 0;
        if (warp == 0 && lane < kSplit) less = *cluster.map_shared_rank(&s_below, lane);
        if (!__any_sync(0xffffffffu, theirs > kSeen)) {
            const int most = __reduce_max_sync(0xffffffffu, theirs);
            for (int i = 0; i < most; i += 32) {
                uint32_t x[kSplit];
#pragma unroll
                for (int r = 0; r < kSplit; ++r) {
                    const bool in = i + lane < __shfl_sync(0xffffffffu, theirs, r);
                    x[r] = in ? cluster.map_shared_rank(all, r)[i + lane] : 0xffffffffu;
                }
#pragma unroll
                for (int r = 0; r < kSplit; ++r) {
                    const bool in = i + lane < __shfl_sync(0xffffffffu, theirs, r);
                    const uint32_t d = x[r] >> kOffBits & 7u;
                    less += in && d < rank;
                    const bool hit = in && d == rank;
                    const uint32_t who = __ballot_sync(0xffffffffu, hit);
                    const int at = n_found + __popc(who & below);
                    if (hit) {
                        if (at < kListed) found[at] = (x[r] & ~(7u << kOffBits)) | uint32_t(r) << kOffBits;
                        atomicAdd(&mine[x[r] >> kListBits], 1);
                    }
                    n_found += __popc(who);
                }
            }
        } else {
            for (int r = 0; r < kSplit; ++r) {
                stretch(r, t0, t1);
                n_found = pass(t0, t1, n_found, [&](uint32_t c) { less += c >= cls0 && c < cls; return c == cls; },
                               [&](uint32_t, uint32_t bin, int t, int at) {
                                   if (at < kListed) found[at] = bin << kListBits | uint32_t(r) << kOffBits | (uint32_t(t - t0) & kOffMask);
                                   atomicAdd(&mine[bin], 1);
                               });
            }
        }
        cluster.sync();                                 // (nobody's lists are needed any more)
    }
    less = __reduce_add_sync(0xffffffffu, less);
    if (lane == 0 && less) atomicAdd(&s_less, less);
    __syncthreads();
    // one thread per id: the warps' counts become offsets within the id, the ids' totals offsets within the order
    int total = 0;
    if (int(threadIdx.x) < bins) {
#pragma unroll 8
        for (int w = 0; w < warps; ++w) {
            const int x = hist[w * bins + threadIdx.x];
            hist[w * bins + threadIdx.x] = total;
            total += x;
        }
    }
    int incl = total;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += y;
    }
    if (lane == 31) s_warp[warp] = incl;
    __syncthreads();
    const int first = s_less + __reduce_add_sync(0xffffffffu, lane < warp ? s_warp[lane] : 0) + incl - total;
    if (int(threadIdx.x) < bins) {
        begin[threadIdx.x] = first;
        b.start[row0 + threadIdx.x] = first;
        if (int(threadIdx.x) == bins - 1) {
            begin[bins] = first + total;
            if (cls == mask) b.start[row0 + bins] = first + total;
        }
    }
    __syncthreads();
    // Segments of the sums: row index + start grows by one per row and one per token; segment j begins with the first row
    // where it has reached j segment lengths.  This class names the segments that begin behind one of its rows.
    const int end = begin[bins];
    const int seg_lo = int((row0 + begin[0]) >> b.seg_shift) + 1, seg_hi = cls == mask ? b.n_segs : int((row0 + bins + end) >> b.seg_shift);
    if (cls == 0u && threadIdx.x == 0) b.segs[0] = make_uint2(0u, 0u);
    for (int j = seg_lo + threadIdx.x; j <= seg_hi; j += blockDim.x) {
        int lo = 0, hi = bins;                          // the first row of the class (bins: the next class's) that has reached it
        while (lo < hi) {
            const int mid = (lo + hi) >> 1;
            if (row0 + mid + begin[mid] >= int64_t(j) << b.seg_shift) hi = mid; else lo = mid + 1;
        }
        b.segs[j] = make_uint2(uint32_t(row0 + lo), uint32_t(begin[lo]));
    }
    // Chunk list: the slots that begin in this class's part of the order (the last class: all that follow, too).
    const int slot_lo = (begin[0] + kSlotTokens - 1) / kSlotTokens, slot_hi = cls == mask ? b.n_slots : (end + kSlotTokens - 1) / kSlotTokens;
    for (int j = slot_lo + int(blockDim.x - 1 - threadIdx.x); j < slot_hi; j += blockDim.x) {      // (other warps than the segments')
        int2 d = make_int2(-1, 0);
        if (j * kSlotTokens < end) {
            const int r = last_not_above(begin, bins, j * kSlotTokens), count = begin[r + 1] - begin[r];
            if (count > kShortRow) {
                const int len = chunk_tokens(count), at = j - (begin[r] + kSlotTokens - 1) / kSlotTokens, k = at / (len / kSlotTokens);
                if (at == k * (len / kSlotTokens) && k < chunks_of(count, len)) d = make_int2(int(row0 + r), k);
            }
        }
        b.slots[j] = d;
    }
    for (int64_t i = int64_t(slot_lo) * b.slabs * 2 + threadIdx.x; i < int64_t(slot_hi) * b.slabs * 2; i += blockDim.x) b.tickets[i] = 0u;

    // places: equal ids among a warp's 32 candidates take consecutive ones, in the order of the lanes
    auto place = [&](bool in, uint32_t bin, int t) {
        const uint32_t who = __ballot_sync(0xffffffffu, in);
        if (in) {
            const uint32_t peers = __match_any_sync(who, bin);
            const int rank = __popc(peers & below);
            const int at = mine[bin];
            __syncwarp(who);
            if (rank == 0) mine[bin] = at + __popc(peers);
            b.perm[begin[bin] + at + rank] = t;
        }
        __syncwarp();
    };
    if (n_found <= kListed && seg <= 1 << kOffBits) {
        __syncwarp();
        for (int i = 0; i < n_found; i += 32) {
            const bool in = i + lane < n_found;
            const uint32_t x = in ? found[i + lane] : 0u;
            const int r = kSplit > 1 ? int(x >> kOffBits & 7u) : 0;
            place(in, x >> kListBits, r * part + warp * seg + int(x & kOffMask));
        }
    } else {
        for (int r = 0; r < kSplit; ++r) {
            stretch(r, t0, t1);
            for (int tb = t0; tb < t1; tb += 32 * kIdLoads) {
                Id id[kIdLoads];
#pragma unroll
                for (int u = 0; u < kIdLoads; ++u) id[u] = tb + lane + 32 * u < t1 ? __ldg(ids + tb + lane + 32 * u) : Id(-1);
#pragma unroll
                for (int u = 0; u < kIdLoads; ++u)
                    place(is_row(id[u], vocab) && uint32_t(id[u]) != pad && (uint32_t(id[u]) & mask) == cls, uint32_t(id[u]) >> shift, tb + 32 * u + lane);
            }
        }
    }
}

// ---- gradient, second kernel: sums of the grouped tokens ----------------------------------------------------------------
// A warp's window of 32 places of perm, passed from lane to lane.
struct Window {
    int32_t at, mine;
    __device__ __forceinline__ void open(const int32_t* perm, int32_t p, int32_t end, int lane) {
        at = p;
        mine = p + lane < end ? __ldg(perm + p + lane) : 0;
    }
    __device__ __forceinline__ uint32_t token(int32_t p) const { return uint32_t(__shfl_sync(0xffffffffu, mine, p - at)); }
};

template <int V>
__device__ __forceinline__ void load_partial(const float* p, float (&x)[V]) {
    if constexpr (V == 2) { const float2 a = __ldcg(reinterpret_cast<const float2*>(p)); x[0] = a.x; x[1] = a.y; }
    if constexpr (V >= 4) { const float4 a = __ldcg(reinterpret_cast<const float4*>(p)); x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; }
    if constexpr (V == 8) { const float4 a = __ldcg(reinterpret_cast<const float4*>(p) + 1); x[4] = a.x; x[5] = a.y; x[6] = a.z; x[7] = a.w; }
}
template <int V>
__device__ __forceinline__ void store_partial(float* p, const float (&x)[V]) {
    if constexpr (V == 2) __stcg(reinterpret_cast<float2*>(p), make_float2(x[0], x[1]));
    if constexpr (V >= 4) __stcg(reinterpret_cast<float4*>(p), make_float4(x[0], x[1], x[2], x[3]));
    if constexpr (V == 8) __stcg(reinterpret_cast<float4*>(p) + 1, make_float4(x[4], x[5], x[6], x[7]));
}

// After this warp has stored a sum: whether it is the last of n to come to the ticket (then it may read the others' sums).
__device__ __forceinline__ bool last_to_come(uint32_t* ticket, int n, int lane) {
    __syncwarp();
    uint32_t before = 0;
    if (lane == 0) before = take_ticket(ticket);
    before = __shfl_sync(0xffffffffu, before, 0);
    __syncwarp();
    return before == uint32_t(n - 1);
}

template <int V>
__device__ __forceinline__ void join_partials(const float* part, size_t step, int n, float (&sum)[V]) {
#pragma unroll
    for (int j = 0; j < V; ++j) sum[j] = 0.f;
#pragma unroll 8
    for (int k = 0; k < n; ++k) {
        float x[V];
        load_partial<V>(part + size_t(k) * step, x);
#pragma unroll
        for (int j = 0; j < V; ++j) sum[j] += x[j];
    }
}

// The finished sum of one row's slab: scaled, added to what is there or not, rounded once.
template <int GRAD, int V, int M>
__device__ __forceinline__ void write_row(char* p, int col, const float (&sum)[V], int accumulate, const EmbedArgs& a) {
    float y[V];
#pragma unroll
    for (int j = 0; j < V; ++j) y[j] = sum[j] * a.scale;
    if (accumulate) {
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const int k = column_of<V, M>(j);
            if (col + k < a.dim) {
                if constexpr (GRAD == BAOC_BF16) y[j] += bf16_bits_to_float(reinterpret_cast<const uint16_t*>(p)[k]);
                else y[j] += reinterpret_cast<const float*>(p)[k];
            }
        }
    }
    store_part<GRAD, V, M>(p, col, a.dim, y);
}

// The sums move all of the bytes.  65536 tokens x 2048 of bf16 into 32000 rows, ids uniform: 66 us for 400 MB = 6.1 TB/s, at the
// copy bandwidth; Zipf-like ids with a tenth padding: 67 us for 373 MB; 16384 x 768 into 50257 rows: 24 us for 102 MB, two
// waves of warps whose start and end weigh.  A warp per row took 1558 us (a frequent row is one warp's work), rows without
// regard to their tokens 82 us more than segments of equal rows + tokens.  Segments end where rows do, so only long rows need
// partial sums; those of 32 tokens a chunk cost 1/8 of their tokens' bytes in L2.
//
// One warp works on one slab of
//   - some of 32 slots of the chunk list: each chunk's tokens are summed into the slot's partial sum;
//   - or one segment, neighbours of the grouped order: its unnamed rows are zeroed, the tokens of its short rows stream
//     through, kBatch of them in flight whatever rows they belong to, and a row is written after its last token.
template <int ACT, int GRAD, int V, int M>
__global__ void __launch_bounds__(kThreads, M == kWide && ACT == BAOC_BF16 && V == 8 ? 4 : 3)
embed_grad_kernel(const char* __restrict__ dout, char* dtable, const GradBufs b, uint32_t vocab, int n, int accumulate,
                  const EmbedArgs a BAOC_CHECK_PARAM) {
    using P = Part<ACT, V, M>;
    constexpr int kBatch = P::kWords >= 8 ? 4 : (P::kWords == 4 ? 8 : 16);
    const int lane = threadIdx.x & 31;
    const uint32_t item = blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5);
    wait_for_earlier_kernel();
    const int slab = int(item % uint32_t(b.slabs));
    int work = int(item / uint32_t(b.slabs));
    const int col = lane_col<V, M>(slab, lane), rc = read_col<V, M>(col, a.dim), last = last_read<V, M>(rc, a.dim, P::kSize);
    const char* src = dout + int64_t(rc) * P::kSize;
    char* dst = dtable + int64_t(col) * (GRAD == BAOC_BF16 ? 2 : 4);
    float acc[V];
#pragma unroll
    for (int j = 0; j < V; ++j) acc[j] = 0.f;

    const int slot_work = b.n_slots / 32 * kSlotWarps;
    if (work < slot_work) {
        const int run = work / kSlotWarps * 32;
#ifdef BAOC_CHECKED
        if (!check_range(ck, kKerEmbedGrad, b.slots + run, 8ll * 32, 3)) return;
#endif
        const int2 listed = b.slots[run + lane];
        const uint32_t used = __ballot_sync(0xffffffffu, listed.x >= 0);
        // the warps of a run take its chunks in turn
        uint32_t todo = __ballot_sync(0xffffffffu, listed.x >= 0 && __popc(used & ((1u << lane) - 1u)) % kSlotWarps == work % kSlotWarps);
#pragma unroll 1
        for (; todo; todo &= todo - 1u) {
            const int at = __ffs(todo) - 1, slot = run + at;
            const int2 d = make_int2(__shfl_sync(0xffffffffu, listed.x, at), __shfl_sync(0xffffffffu, listed.y, at));
#ifdef BAOC_CHECKED
            if (d.x >= int64_t(b.bins) << b.shift) { check_fail(kChkBlockIndex, kKerEmbedGrad, d.x, int64_t(b.bins) << b.shift, slot, 0); return; }
#endif
            const int32_t s0 = b.start[d.x], count = b.start[d.x + 1] - s0;
            const int len = chunk_tokens(count), chunks = chunks_of(count, len), apart = len / kSlotTokens, first = slot - d.y * apart;
            const int32_t p0 = s0 + d.y * len, p1 = d.y == chunks - 1 ? s0 + count : p0 + len;
#ifdef BAOC_CHECKED
            if (!check_range(ck, kKerEmbedGrad, b.perm + p0, 4ll * (p1 - p0), 1) ||
                !check_range(ck, kKerEmbedGrad, b.partial + size_t(first) * b.slabs * 32 * V, 4ll * ((chunks - 1) * apart + 1) * b.slabs * 32 * V, 4) ||
                !check_range(ck, kKerEmbedGrad, b.tickets + size_t(first) * b.slabs * 2, 8ll * ((chunks - 1) * apart + 1) * b.slabs, 5))
                return;
            for (int32_t p = p0; p < p1; ++p)
                if (b.perm[p] < 0 || b.perm[p] >= n) { check_fail(kChkTileIndex, kKerEmbedGrad, b.perm[p], n, p, 2); return; }
#endif
            Window win;
#pragma unroll 1
            for (int32_t p = p0; p < p1; p += kBatch) {
                if (((p - p0) & 31) == 0) win.open(b.perm, p, p1, lane);
                P x[kBatch];
#pragma unroll
                for (int i = 0; i < kBatch; ++i) x[i].load(src + uint64_t(win.token(min(p + i, p1 - 1))) * a.src_step, last);
#pragma unroll
                for (int i = 0; i < kBatch; ++i)
                    if (p + i < p1) {
#pragma unroll
                        for (int j = 0; j < V; ++j) acc[j] += x[i].at(j);
                    }
            }
            // the slot's partial sum; whoever brings the last of kJoin neighbours adds them up, and whoever brings the last
            // of those sums writes the row.  Nobody waits, and each sum has its fixed order.
            const size_t step = size_t(apart) * b.slabs * (32 * V);
            float* part = b.partial + (size_t(first) * b.slabs + slab) * (32 * V) + lane * V;
            uint32_t* tickets = b.tickets + (size_t(first) * b.slabs + slab) * 2;
            store_partial<V>(part + size_t(d.y) * step, acc);
            const int group = d.y / kJoin, in_group = min(kJoin, chunks - group * kJoin), groups = (chunks + kJoin - 1) / kJoin;
            bool mine = last_to_come(tickets + size_t(group) * kJoin * apart * b.slabs * 2, in_group, lane);
            if (mine) {
                join_partials<V>(part + size_t(group) * kJoin * step, step, in_group, acc);
                if (groups > 1) {
                    store_partial<V>(part + size_t(group) * kJoin * step, acc);
                    mine = last_to_come(tickets + 1, groups, lane);
                    if (mine) join_partials<V>(part, size_t(kJoin) * step, groups, acc);
                }
            }
            if (mine) {
                const uint32_t cls = uint32_t(d.x) / uint32_t(b.bins), bin = uint32_t(d.x) - cls * uint32_t(b.bins);
                write_row<GRAD, V, M>(dst + uint64_t((bin << b.shift) + cls) * a.dst_step, col, acc, accumulate, a);
            }
#pragma unroll
            for (int j = 0; j < V; ++j) acc[j] = 0.f;
        }
        return;
    }
    work -= slot_work;
    if (work >= b.n_segs) return;
#ifdef BAOC_CHECKED
    if (!check_range(ck, kKerEmbedGrad, b.segs + work, 16, 6)) return;
#endif
    const uint2 d0 = b.segs[work], d1 = b.segs[work + 1];
    const int rows = int(d1.x - d0.x);                  // at most one per lane
    const int32_t end = int32_t(d1.y);
#ifdef BAOC_CHECKED
    if (rows < 0 || rows > 32 || !check_range(ck, kKerEmbedGrad, b.start + size_t(d0.x), 4ll * rows, 0) ||
        !check_range(ck, kKerEmbedGrad, b.perm + d0.y, 4ll * (end - int32_t(d0.y)), 1)) {
        check_fail(kChkBlockIndex, kKerEmbedGrad, d0.x, d1.x, work, 0);
        return;
    }
    for (int32_t p = int32_t(d0.y); p < end; ++p)
        if (b.perm[p] < 0 || b.perm[p] >= n) { check_fail(kChkTileIndex, kKerEmbedGrad, b.perm[p], n, p, 2); return; }
#endif
    Window win;
    win.open(b.perm, int32_t(d0.y), end, lane);
    // lane r has row r of the segment: the table's row, its first place and its number of tokens
    const int32_t st = lane < rows ? b.start[size_t(d0.x) + lane] : end;
    const uint32_t idx = d0.x + uint32_t(lane), cls = idx / uint32_t(b.bins);
    const uint32_t row = ((idx - cls * uint32_t(b.bins)) << b.shift) + cls;
    const int32_t up = __shfl_down_sync(0xffffffffu, st, 1);
    const int count = lane < rows ? (lane == 31 ? end : up) - st : 0;
    const uint32_t longs = __ballot_sync(0xffffffffu, count > kShortRow);
    if (!accumulate) {
        float zero[V];
#pragma unroll
        for (int j = 0; j < V; ++j) zero[j] = 0.f;
        uint32_t unnamed = __ballot_sync(0xffffffffu, lane < rows && count == 0 && row < vocab);
        while (unnamed) {
            const int r = __ffs(unnamed) - 1;
            unnamed &= unnamed - 1u;
            store_part<GRAD, V, M>(dst + uint64_t(__shfl_sync(0xffffffffu, row, r)) * a.dst_step, col, a.dim, zero);
        }
    }
    // the runs of short rows between the long ones (which their chunks write)
    int32_t p0 = int32_t(d0.y);
    for (uint32_t rest = longs;; rest &= rest - 1u) {
        const int next = rest ? __ffs(rest) - 1 : 0;
        const int32_t p1 = rest ? __shfl_sync(0xffffffffu, st, next) : end;
        if (p0 < p1) {
            // the row of a place: the last one that begins at it or before
            int r = __popc(__ballot_sync(0xffffffffu, lane < rows && st <= p0)) - 1;
            int32_t row_end = __shfl_sync(0xffffffffu, st + count, r);
#pragma unroll
            for (int j = 0; j < V; ++j) acc[j] = 0.f;
#pragma unroll 1
            for (int32_t p = p0; p < p1; p += kBatch) {
                if (((p - p0) & 31) == 0 && p != win.at) win.open(b.perm, p, p1, lane);
                P x[kBatch];
#pragma unroll
                for (int i = 0; i < kBatch; ++i) x[i].load(src + uint64_t(win.token(min(p + i, p1 - 1))) * a.src_step, last);
#pragma unroll
                for (int i = 0; i < kBatch; ++i) {
                    // (what a last batch adds behind p1 belongs to no row: no row ends within a batch behind p1)
#pragma unroll
                    for (int j = 0; j < V; ++j) acc[j] += x[i].at(j);
                    if (p + i + 1 == row_end) {
                        write_row<GRAD, V, M>(dst + uint64_t(__shfl_sync(0xffffffffu, row, r)) * a.dst_step, col, acc, accumulate, a);
#pragma unroll
                        for (int j = 0; j < V; ++j) acc[j] = 0.f;
                        r = __popc(__ballot_sync(0xffffffffu, lane < rows && st <= row_end)) - 1;
                        row_end = __shfl_sync(0xffffffffu, st + count, r);
                    }
                }
            }
        }
        if (rest == 0u) break;
        p0 = __shfl_sync(0xffffffffu, st + count, next);
    }
}

// ---- gradient of a few tokens: one kernel ---------------------------------------------------------------------------
// CTA c has the rows c, c + gridDim, ..; its threads look at one id each, list those of its rows in the tokens' order, and
// its warps take (row, slab) pairs in turn: a row's tokens are found in the list by a vote.
template <int ACT, int GRAD, int V, int M>
__global__ void __launch_bounds__(kThreads)
embed_grad_few_kernel(const void* __restrict__ ids, int id_bits, int n, const char* __restrict__ dout, char* dtable, uint32_t vocab, uint32_t pad,
                      int slabs, int accumulate, const EmbedArgs a) {
    using P = Part<ACT, V, M>;
    constexpr int kBatch = P::kWords >= 8 ? 4 : 8;
    __shared__ uint32_t list_row[kFewTokens];
    __shared__ int32_t list_token[kFewTokens];
    __shared__ int found[kThreads / 32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint32_t step = gridDim.x;
    uint32_t k = 0;
    bool in = false;
    if (int(threadIdx.x) < n) {
        const int64_t id = id_bits == 64 ? __ldg(static_cast<const int64_t*>(ids) + threadIdx.x) : int64_t(__ldg(static_cast<const int32_t*>(ids) + threadIdx.x));
        if (is_row(id, vocab) && uint32_t(id) != pad) {
            k = uint32_t(id) / step;
            in = uint32_t(id) - k * step == blockIdx.x;
        }
    }
    const uint32_t who = __ballot_sync(0xffffffffu, in);
    if (lane == 0) found[warp] = __popc(who);
    __syncthreads();
    int before = 0, listed = 0;
#pragma unroll
    for (int w = 0; w < kThreads / 32; ++w) {
        before += w < warp ? found[w] : 0;
        listed += found[w];
    }
    if (in) {
        const int at = before + __popc(who & ((1u << lane) - 1u));
        list_row[at] = k;
        list_token[at] = int32_t(threadIdx.x);
    }
    __syncthreads();
    const uint32_t rows = (vocab - blockIdx.x + step - 1) / step;
    // the next pair of a warp is kThreads / 32 further on
    const uint32_t row_step = uint32_t(kThreads / 32) / uint32_t(slabs);
    const int slab_step = kThreads / 32 - int(row_step) * slabs;
    uint32_t r = uint32_t(warp) / uint32_t(slabs);
    int slab = warp - int(r) * slabs;
    auto next = [&]() {
        r += row_step;
        slab += slab_step;
        if (slab >= slabs) { slab -= slabs; ++r; }
    };
    if (listed == 0) {                                  // most CTAs: nothing but zeros to write
        if (accumulate) return;
        float zero[V];
#pragma unroll
        for (int j = 0; j < V; ++j) zero[j] = 0.f;
        for (; r < rows; next()) {
            const int col = lane_col<V, M>(slab, lane);
            store_part<GRAD, V, M>(dtable + uint64_t(blockIdx.x + r * step) * a.dst_step + int64_t(col) * (GRAD == BAOC_BF16 ? 2 : 4), col, a.dim, zero);
        }
        return;
    }
    for (; r < rows; next()) {
        const int col = lane_col<V, M>(slab, lane), rc = read_col<V, M>(col, a.dim), last = last_read<V, M>(rc, a.dim, P::kSize);
        const char* src = dout + int64_t(rc) * P::kSize;
        float acc[V];
#pragma unroll
        for (int j = 0; j < V; ++j) acc[j] = 0.f;
        bool named = false;
        for (int l0 = 0; l0 < listed; l0 += 32) {
            uint32_t hits = __ballot_sync(0xffffffffu, l0 + lane < listed && list_row[l0 + lane] == r);
            named |= hits != 0u;
            while (hits) {
                const int m = min(__popc(hits), kBatch);
                P x[kBatch];
#pragma unroll
                for (int i = 0; i < kBatch; ++i) {      // (behind the m-th token it is read again, and not added)
                    x[i].load(src + uint64_t(uint32_t(list_token[l0 + __ffs(hits) - 1])) * a.src_step, last);
                    if (i + 1 < m) hits &= hits - 1u;
                }
                hits &= hits - 1u;
#pragma unroll
                for (int i = 0; i < kBatch; ++i)
                    if (i < m) {
#pragma unroll
                        for (int j = 0; j < V; ++j) acc[j] += x[i].at(j);
                    }
            }
        }
        if (named || !accumulate)
            write_row<GRAD, V, M>(dtable + uint64_t(blockIdx.x + r * step) * a.dst_step + int64_t(col) * (GRAD == BAOC_BF16 ? 2 : 4), col, acc, accumulate, a);
    }
}

namespace {

thread_local std::string g_embed_err;

int fail_embed(int code, const std::string& msg) {
    g_embed_err = msg;
    return code;
}

int64_t elem_bytes(int dtype) { return dtype == BAOC_F32 ? 4 : 2; }
int64_t stride_of(int64_t stride, int dim) { return stride ? stride : dim; }

int check_embed(const baoc_embed_t* e, const char* what) {
    if (!e) return fail_embed(BAOC_E_INVALID, std::string(what) + ": null descriptor");
    if (e->vocab < 1 || e->vocab > int64_t(0x7fffffff) || e->dim < 1 || e->dim > kEmbedMaxDim)
        return fail_embed(BAOC_E_INVALID, std::string(what) + ": vocab must be in 1 .. 2^31 - 1 and dim in 1 .. 2^24");
    for (int dt : {e->table_dtype, e->act_dtype, e->grad_dtype})
        if (dt != BAOC_F32 && dt != BAOC_BF16) return fail_embed(BAOC_E_INVALID, std::string(what) + ": unknown dtype");
    if (e->id_bits != 32 && e->id_bits != 64) return fail_embed(BAOC_E_INVALID, std::string(what) + ": id_bits must be 32 or 64");
    if (!std::isfinite(e->scale)) return fail_embed(BAOC_E_INVALID, std::string(what) + ": scale must be finite");
    if (e->pad_id < -1 || e->pad_id >= e->vocab) return fail_embed(BAOC_E_INVALID, std::string(what) + ": pad_id must be -1 or a row of the table");
    for (int64_t st : {e->table_stride, e->act_stride, e->grad_stride})
        if (st != 0 && (st < e->dim || st > kEmbedMaxStride)) return fail_embed(BAOC_E_INVALID, std::string(what) + ": a row stride must be in dim .. 2^28 (0 stands for dim)");
    return BAOC_OK;
}

bool aligned(const void* p, int64_t bytes) { return (reinterpret_cast<uintptr_t>(p) & uintptr_t(bytes - 1)) == 0; }

// What rows of an array allow (eb: bytes of an element).
int access_of(const void* p, int64_t stride, int64_t eb, int dim) {
    if (dim % 8 == 0 && aligned(p, 16) && (stride * eb) % 16 == 0) return kWide;
    return dim % 2 == 0 && aligned(p, 2 * eb) && stride % 2 == 0 ? kPairs : kSingles;
}

bool overlap(const void* a, int64_t abytes, const void* b, int64_t bbytes) {
    const char* x = static_cast<const char*>(a);
    const char* y = static_cast<const char*>(b);
    return x < y + bbytes && y < x + abytes;
}

// The classes of the grouping for a vocabulary, and the ids per class.
void group_geometry(int64_t vocab, int* shift, int* bins) {
    int s = 0;
    while ((1 << s) < kGroupCtas || ceil_div(vocab, int64_t(1) << s) > kGroupBins) ++s;
    *shift = s;
    *bins = int(ceil_div(vocab, int64_t(1) << s));
}

int columns_per_warp(int dim) { return dim > 128 ? 256 : (dim > 64 ? 128 : 64); }
int group_smem(int bins, int split) { return 4 * (kGroupWarps * bins + bins + 1 + kGroupWarps * (kListed + (split > 1 ? kSeen : 0))); }

// The grouping's shared memory is above the default limit; the permission is per device and lasts.
template <typename Id, int kSplit>
cudaError_t allow_group_smem() {
    static std::atomic<uint64_t> done{0};               // one bit per device
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    const uint64_t bit = dev < 64 ? uint64_t(1) << dev : 0;
    if (done.load(std::memory_order_relaxed) & bit) return cudaSuccess;
    e = cudaFuncSetAttribute(embed_group_kernel<Id, kSplit>, cudaFuncAttributeMaxDynamicSharedMemorySize, group_smem(kGroupBins, kSplit));
    if (e == cudaSuccess) done.fetch_or(bit, std::memory_order_relaxed);
    return e;
}

struct EmbedLayout { size_t start, perm, segs, slots, tickets, partial, total; int shift, bins, slabs, seg_shift, n_segs, n_slots; };

EmbedLayout embed_layout(const baoc_embed_t* e, int64_t n) {
    EmbedLayout L{};
    L.slabs = int(ceil_div(e->dim, columns_per_warp(e->dim)));
    group_geometry(e->vocab, &L.shift, &L.bins);
    L.start = 0;
    L.perm = size_t(round_up(4 * ((int64_t(L.bins) << L.shift) + 1), 256));
    L.n_slots = int(round_up(ceil_div(n, kSlotTokens), 32));
    const int64_t length = (int64_t(L.bins) << L.shift) + n;
    L.seg_shift = kSegShift;
    while (L.seg_shift > kSegShiftLeast && (length >> L.seg_shift) * L.slabs < kSegWarps) --L.seg_shift;
    L.n_segs = int(ceil_div(length, int64_t(1) << L.seg_shift));
    // The segment table's size must not fall as n grows (a workspace serves every smaller batch), though n_segs halves where
    // the segments get longer: a shift below kSegShift is taken only while the next one leaves fewer than ceil(kSegWarps /
    // slabs) segments, so it has at most twice as many.
    const int64_t most_segs = std::min(ceil_div(length, int64_t(1) << kSegShiftLeast),
                                       std::max(ceil_div(length, int64_t(1) << kSegShift), 2 * ceil_div(int64_t(kSegWarps), L.slabs)));
    L.segs = L.perm + size_t(round_up(4 * n, 256));
    L.slots = L.segs + size_t(round_up(8 * (most_segs + 1), 256));
    L.tickets = L.slots + size_t(round_up(8 * int64_t(L.n_slots), 256));
    L.partial = L.tickets + size_t(round_up(8 * int64_t(L.n_slots) * L.slabs, 256));
    L.total = L.partial + size_t(4 * int64_t(L.n_slots) * L.slabs * columns_per_warp(e->dim));
    return L;
}

// f(source type, destination type, V, access) for the types, the row length and the alignment of a call, as constants.
template <int S, int D, int V, typename F>
int with_access(int access, F f) {
    using std::integral_constant;
    const integral_constant<int, S> s{};
    const integral_constant<int, D> d{};
    const integral_constant<int, V> v{};
    if (access == kWide) return f(s, d, v, integral_constant<int, kWide>{});
    if (access == kPairs) return f(s, d, v, integral_constant<int, kPairs>{});
    return f(s, d, v, integral_constant<int, kSingles>{});
}
template <int S, int D, typename F>
int with_shape(int dim, int access, F f) {
    if (dim > 128) return with_access<S, D, 8>(access, f);
    if (dim > 64) return with_access<S, D, 4>(access, f);
    return with_access<S, D, 2>(access, f);
}
template <typename F>
int with_types(int a, int b, int dim, int access, F f) {
    if (a == BAOC_F32) return b == BAOC_F32 ? with_shape<BAOC_F32, BAOC_F32>(dim, access, f) : with_shape<BAOC_F32, BAOC_BF16>(dim, access, f);
    return b == BAOC_F32 ? with_shape<BAOC_BF16, BAOC_F32>(dim, access, f) : with_shape<BAOC_BF16, BAOC_BF16>(dim, access, f);
}

int launched(const char* kernel) {
    const cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? BAOC_OK : fail_embed(BAOC_E_CUDA, std::string(kernel) + ": " + cudaGetErrorString(e));
}

}  // namespace

BAOC_DEFINE_CHECK_FETCH(embed_check_fetch)

}  // namespace baoc

using namespace baoc;

extern "C" {

const char* baoc_embed_last_error(void) { return g_embed_err.c_str(); }

int baoc_embed(const baoc_embed_t* e, const void* table, const void* ids, int64_t n_tokens, void* out, baoc_stream_t stream) try {
    const char* what = "baoc_embed";
    int rc = check_embed(e, what);
    if (rc) return rc;
    if (n_tokens < 0) return fail_embed(BAOC_E_INVALID, "baoc_embed: n_tokens must not be negative");
    if (n_tokens == 0) return BAOC_OK;
    if (!table || !ids || !out) return fail_embed(BAOC_E_INVALID, "baoc_embed: null pointer");
    const int64_t tb = elem_bytes(e->table_dtype), ob = elem_bytes(e->act_dtype);
    const int64_t ts = stride_of(e->table_stride, e->dim), os = stride_of(e->act_stride, e->dim);
    if (!aligned(table, tb) || !aligned(out, ob) || !aligned(ids, e->id_bits / 8)) return fail_embed(BAOC_E_ALIGN, "baoc_embed: a pointer is not aligned to its elements");
    if (n_tokens > (int64_t(1) << 40) / os) return fail_embed(BAOC_E_INVALID, "baoc_embed: too many tokens");
    if (ts == e->dim && os == e->dim && overlap(table, e->vocab * ts * tb, out, n_tokens * os * ob))
        return fail_embed(BAOC_E_INVALID, "baoc_embed: out overlaps the table");
    const EmbedArgs a{uint32_t(ts * tb), uint32_t(os * ob), e->dim, e->scale};
    const int slabs = int(ceil_div(e->dim, columns_per_warp(e->dim)));
    const int access = std::min(access_of(table, ts, tb, e->dim), access_of(out, os, ob, e->dim));
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    return with_types(e->table_dtype, e->act_dtype, e->dim, access, [&](auto S, auto D, auto V, auto M) {
        constexpr int kTokens = Part<S(), V(), M()>::kWords == 8 ? 2 : 4;
        const int64_t items = ceil_div(n_tokens, kTokens) * slabs, blocks = ceil_div(items, kThreads / 32);
        if (items > int64_t(0x7fffffff)) return fail_embed(BAOC_E_INVALID, "baoc_embed: too many elements for one launch");
        const char* tab = static_cast<const char*>(table);
        char* o = static_cast<char*>(out);
        if (e->id_bits == 64)
            embed_kernel<S(), D(), V(), M(), int64_t><<<unsigned(blocks), kThreads, 0, s>>>(tab, static_cast<const int64_t*>(ids), o, uint32_t(e->vocab), n_tokens, slabs, a);
        else
            embed_kernel<S(), D(), V(), M(), int32_t><<<unsigned(blocks), kThreads, 0, s>>>(tab, static_cast<const int32_t*>(ids), o, uint32_t(e->vocab), n_tokens, slabs, a);
        return launched("embed_kernel");
    });
} catch (const std::bad_alloc&) {
    return BAOC_E_INVALID;
}

int baoc_embed_grad_workspace_bytes(const baoc_embed_t* e, int64_t n_tokens, size_t* bytes) try {
    const int rc = check_embed(e, "baoc_embed_grad_workspace_bytes");
    if (rc) return rc;
    if (!bytes || n_tokens < 0 || n_tokens > (int64_t(1) << 30)) return fail_embed(BAOC_E_INVALID, "baoc_embed_grad_workspace_bytes: n_tokens must be in 0 .. 2^30");
    *bytes = embed_layout(e, n_tokens).total;
    return BAOC_OK;
} catch (const std::bad_alloc&) {
    return BAOC_E_INVALID;
}

int baoc_embed_grad(const baoc_embed_t* e, const void* ids, const void* dout, int64_t n_tokens, void* dtable, int accumulate, void* ws,
                    size_t ws_bytes, baoc_stream_t stream) try {
    const char* what = "baoc_embed_grad";
    int rc = check_embed(e, what);
    if (rc) return rc;
    if (n_tokens < 0 || n_tokens > (int64_t(1) << 30)) return fail_embed(BAOC_E_INVALID, "baoc_embed_grad: n_tokens must be in 0 .. 2^30");
    if (!dtable || !ws || (n_tokens > 0 && (!ids || !dout))) return fail_embed(BAOC_E_INVALID, "baoc_embed_grad: null pointer");
    const int64_t ab = elem_bytes(e->act_dtype), gb = elem_bytes(e->grad_dtype);
    const int64_t as = stride_of(e->act_stride, e->dim), gs = stride_of(e->grad_stride, e->dim);
    if (!aligned(dout, ab) || !aligned(dtable, gb) || !aligned(ids, e->id_bits / 8)) return fail_embed(BAOC_E_ALIGN, "baoc_embed_grad: a pointer is not aligned to its elements");
    if (!aligned(ws, 256)) return fail_embed(BAOC_E_ALIGN, "baoc_embed_grad: workspace not 256-byte aligned");
    const EmbedLayout L = embed_layout(e, n_tokens);
    if (ws_bytes < L.total) return fail_embed(BAOC_E_WORKSPACE, "baoc_embed_grad: workspace too small");
    if (overlap(ws, int64_t(L.total), dtable, ((e->vocab - 1) * gs + e->dim) * gb)) return fail_embed(BAOC_E_INVALID, "baoc_embed_grad: dtable overlaps the workspace");
    if (n_tokens > 0 && as == e->dim && gs == e->dim && overlap(dout, n_tokens * as * ab, dtable, e->vocab * gs * gb))
        return fail_embed(BAOC_E_INVALID, "baoc_embed_grad: dtable overlaps dout");
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    char* w = static_cast<char*>(ws);
    const GradBufs b{reinterpret_cast<int32_t*>(w + L.start), reinterpret_cast<int32_t*>(w + L.perm), reinterpret_cast<uint2*>(w + L.segs),
                     reinterpret_cast<int2*>(w + L.slots), reinterpret_cast<uint32_t*>(w + L.tickets), reinterpret_cast<float*>(w + L.partial),
                     L.shift, L.bins, L.slabs, L.seg_shift, L.n_segs, L.n_slots};
    const CheckCtx ck{w, w + L.total, 0, 0, 0};
    (void)ck;
    const EmbedArgs a{uint32_t(as * ab), uint32_t(gs * gb), e->dim, e->scale};
    const int access = std::min(access_of(dout, as, ab, e->dim), access_of(dtable, gs, gb, e->dim));
    if (n_tokens <= kFewTokens && n_tokens * e->dim * ab <= kFewBytes) {
        const int64_t pairs = e->vocab * L.slabs;
        const unsigned ctas = unsigned(std::min<int64_t>(std::min<int64_t>(e->vocab, e->vocab * e->dim * gb < kFewLargeTable ? kFewCtas : kFewCtasLarge), ceil_div(pairs, kThreads / 32)));
        return with_types(e->act_dtype, e->grad_dtype, e->dim, access, [&](auto A, auto G, auto V, auto M) {
            embed_grad_few_kernel<A(), G(), V(), M()><<<ctas, kThreads, 0, s>>>(ids, e->id_bits, int(n_tokens), static_cast<const char*>(dout),
                                                                                 static_cast<char*>(dtable), uint32_t(e->vocab), uint32_t(e->pad_id),
                                                                                 L.slabs, accumulate, a);
            return launched("embed_grad_few_kernel");
        });
    }
    const int64_t items = (int64_t(L.n_slots / 32) * kSlotWarps + L.n_segs) * L.slabs;
    if (items > int64_t(0x7fffffff)) return fail_embed(BAOC_E_INVALID, "baoc_embed_grad: too many elements for one launch");
    auto group = [&](auto id, auto split) {
        using Id = decltype(id);
        constexpr int kSplit = decltype(split)::value;
        cudaError_t ce = allow_group_smem<Id, kSplit>();
        if (ce == cudaSuccess) {
            cudaLaunchAttribute at{};
            at.id = cudaLaunchAttributeClusterDimension;
            at.val.clusterDim.x = kSplit; at.val.clusterDim.y = 1; at.val.clusterDim.z = 1;
            cudaLaunchConfig_t cfg{};
            cfg.gridDim = dim3(1u << L.shift); cfg.blockDim = dim3(kGroupWarps * 32); cfg.dynamicSmemBytes = size_t(group_smem(L.bins, kSplit)); cfg.stream = s;
            cfg.attrs = &at; cfg.numAttrs = kSplit > 1 ? 1 : 0;
            ce = cudaLaunchKernelEx(&cfg, embed_group_kernel<Id, kSplit>, static_cast<const Id*>(ids), int(n_tokens), uint32_t(e->vocab),
                                    uint32_t(e->pad_id), b BAOC_CHECK_ARG(ck));
        }
        return ce == cudaSuccess ? BAOC_OK : fail_embed(BAOC_E_CUDA, std::string("embed_group_kernel: ") + cudaGetErrorString(ce));
    };
    const std::integral_constant<int, 1> alone{};
    const std::integral_constant<int, kGroupSplit> shared{};
    if (n_tokens < kSplitTokens) rc = e->id_bits == 64 ? group(int64_t(0), alone) : group(int32_t(0), alone);
    else rc = e->id_bits == 64 ? group(int64_t(0), shared) : group(int32_t(0), shared);
    if (rc) return rc;
    const unsigned grid = unsigned(ceil_div(items, kThreads / 32));
    return with_types(e->act_dtype, e->grad_dtype, e->dim, access, [&](auto A, auto G, auto V, auto M) {
        const cudaError_t ce = launch_behind(embed_grad_kernel<A(), G(), V(), M()>, grid, kThreads, s, static_cast<const char*>(dout),
                                             static_cast<char*>(dtable), b, uint32_t(e->vocab), int(n_tokens), accumulate, a BAOC_CHECK_ARG(ck));
        return ce == cudaSuccess ? BAOC_OK : fail_embed(BAOC_E_CUDA, std::string("embed_grad_kernel: ") + cudaGetErrorString(ce));
    });
} catch (const std::bad_alloc&) {
    return BAOC_E_INVALID;
}

}  // extern "C"
