// Global gradient norm over the handle's blocks, and clipping by it.
//
//   n_i = ||g_i||,  n = sqrt(sum_i n_i^2),  dst_i = min(1, max_norm / (n + 1e-6)) * src_i.
//
// Memory bounds both: the norm reads every gradient once, the clip reads it again (the factor exists only after the last
// element has been read) and writes it.  Times below: one B200, device time per call in a row of calls on three sets of arrays.
#include <algorithm>
#include <cmath>
#include <cstring>
#include <cuda_runtime.h>
#include <new>

#include "baoc_device.cuh"

namespace baoc {

constexpr double kClipEps = 1e-6;
// A thread's fp32 sum of up to 32 squares (bf16; 16 of fp32) is taken as it is inside this range: no square has overflowed,
// and what squares below the smallest fp32 number have lost is under 32 * 2^-150 of at least 1e-30.
constexpr float kSquaresLo = 1e-30f, kSquaresHi = 1e30f;

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

// Elements of one 16-byte load, as floats.
template <int DT> struct Vec;
template <> struct Vec<BAOC_BF16> {
    static constexpr int kN = 8;
    using Elem = uint16_t;
    static __device__ __forceinline__ void floats(const uint4& w, float (&x)[8]) { unpack8(w, x); }
    static __device__ __forceinline__ float one(const Elem* p) { return bf16_bits_to_float(*p); }
};
template <> struct Vec<BAOC_F32> {
    static constexpr int kN = 4;
    using Elem = float;
    static __device__ __forceinline__ void floats(const uint4& w, float (&x)[4]) {
        x[0] = __uint_as_float(w.x); x[1] = __uint_as_float(w.y); x[2] = __uint_as_float(w.z); x[3] = __uint_as_float(w.w);
    }
    static __device__ __forceinline__ float one(const Elem* p) { return *p; }
};

constexpr int kNormLoads = 4;          // 16-byte loads a thread of the norm has in flight

// The squares of n 16-byte words, kThreads apart, in double throughout.  Called where fp32 squares would leave their range
// (infinities and NaN end there too and pass through); the words are read again, so that the usual path keeps none.
template <int DT>
__device__ __noinline__ double squares_in_double(const uint4* q, int n) {
    double d = 0.0;
    for (int k = 0; k < n; ++k) {
        float x[Vec<DT>::kN];
        Vec<DT>::floats(ld_stream_u4(q + k * kThreads), x);
        for (int j = 0; j < Vec<DT>::kN; ++j) d = fma(double(x[j]), double(x[j]), d);
    }
    return d;
}

// The squares of K 16-byte words that a thread has loaded from q on, kThreads apart.
template <int DT, int K>
__device__ __forceinline__ double sum_squares(const uint4 (&w)[K], const uint4* q) {
    float a[4] = {0.f, 0.f, 0.f, 0.f};
    uint32_t any = 0;
#pragma unroll
    for (int k = 0; k < K; ++k) {
        float x[Vec<DT>::kN];
        Vec<DT>::floats(w[k], x);
#pragma unroll
        for (int j = 0; j < Vec<DT>::kN; ++j) a[j & 3] = fmaf(x[j], x[j], a[j & 3]);
        any |= w[k].x | w[k].y | w[k].z | w[k].w;
    }
    const float s = (a[0] + a[1]) + (a[2] + a[3]);
    if (s >= kSquaresLo && s <= kSquaresHi) return double(s);
    return (any & (DT == BAOC_BF16 ? 0x7fff7fffu : 0x7fffffffu)) ? squares_in_double<DT>(q, K) : 0.0;
}

#ifdef BAOC_CHECKED
__device__ __forceinline__ bool check_segment(const CheckCtx& ck, unsigned kernel, const ClipBufs& c, int s) {
    if (s < 0 || s >= ck.n_tiles) return check_fail(kChkTileIndex, kernel, s, ck.n_tiles, 0, 0);
    if (!check_range(ck, kernel, c.segs + s, sizeof(ClipSeg), 9)) return false;
    const int b = c.segs[s].block;
    if (b < 0 || b >= ck.n_blocks) return check_fail(kChkBlockIndex, kernel, b, ck.n_blocks, s, 0);
    return c.segs[s].count > 0 && s >= c.block_seg[b] && s < c.block_seg[b + 1] ? true : check_fail(kChkTileStart, kernel, s, c.block_seg[b], b, 0);
}
#endif

// Blocks of at most this many segments are added by one thread each at the end of the norm, the others by a warp.
constexpr int kThreadSegs = 32;
constexpr int kStagedSegs = 4096;      // partial sums that the last CTA takes into shared memory first

__device__ __forceinline__ double warp_sum(double x) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}

// The last CTA: per block and over all, the sums of the segments' partial sums in a fixed order.
__device__ __forceinline__ void finish_norm(const ClipBufs& c, double max_norm, float* norms) {
    __shared__ double stage[kStagedSegs];
    __shared__ double sum;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const bool staged = c.n_segs <= kStagedSegs;
    // neighbouring blocks go to different warps: the large ones are often next to each other
    constexpr int kWarps = kThreads / 32;
    int b = warp + lane * kWarps;
    int lo = b < c.n_blocks ? c.block_seg[b] : 0, hi = b < c.n_blocks ? c.block_seg[b + 1] : 0;
    double acc[1] = {0.0};
#pragma unroll 4
    for (int i = threadIdx.x; i < c.n_segs; i += kThreads) {
        const double x = __ldcg(c.partials + i);         // (past L1, which may hold a line from before)
        if (staged) stage[i] = x;
        acc[0] += x;
    }
    cta_reduce_store<1>(acc, &sum);                     // (its barriers also close the stage)
    if (threadIdx.x == 0) {
        const double n = sqrt(sum), f = max_norm / (n + kClipEps);
        norms[0] = float(n);
        *c.factor = f < 1.0 ? float(f) : (f >= 1.0 ? 1.0f : float(n));      // (a NaN norm is a NaN factor)
        *c.ticket = 0u;
    }
    auto part = [&](int i) { return staged ? stage[i] : __ldcg(c.partials + i); };
    for (int b0 = warp; b0 < c.n_blocks; b0 += kThreads) {
        if (b0 > warp) {
            b = b0 + lane * kWarps;
            lo = b < c.n_blocks ? c.block_seg[b] : 0;
            hi = b < c.n_blocks ? c.block_seg[b + 1] : 0;
        }
        if (hi - lo <= kThreadSegs && b < c.n_blocks) {
            double s = 0.0;
            for (int i = lo; i < hi; ++i) s += part(i);
            norms[1 + b] = float(sqrt(s));
        }
        uint32_t many = __ballot_sync(0xffffffffu, hi - lo > kThreadSegs);
        for (; many; many &= many - 1u) {
            const int k = __ffs(many) - 1, l = __shfl_sync(0xffffffffu, lo, k), h = __shfl_sync(0xffffffffu, hi, k);
            double s = 0.0;
            for (int i = l + lane; i < h; i += 32) s += part(i);
            s = warp_sum(s);
            if (lane == 0) norms[1 + b0 + k * kWarps] = float(sqrt(s));
        }
    }
}

// A CTA per share.  Each segment's sum of squares goes to the segment's slot; the last CTA to end adds the slots.
// One read of everything: 1.14 G bf16 elements in 316 us = 7.2 TB/s, 124 M in 43 us (bf16) and 78 us (fp32, 6.4 TB/s); 2.4 M
// in 7.3 us, of which 2.6 us are the reading, 2.2 us the joint finish and the rest the launch.  A CTA per tile took 418 and
// 53 us: its registers (eight loads held for the wide-range path) left three CTAs on an SM, and each ended in a reduction, a
// fence and a ticket.  Equal shares end once, but all wait for their loads together: without the second round in flight
// they took 392 and 52 us.  The values' squares are checked per round, not per element, and a round that leaves the fp32
// range is read again.
template <int DT>
__global__ void __launch_bounds__(kThreads, kNormCtasPerSm)
grad_norm_kernel(const ClipBufs c, double max_norm, float* __restrict__ norms BAOC_CHECK_PARAM) {
    constexpr int V = Vec<DT>::kN;
    using E = typename Vec<DT>::Elem;
    const ClipCta share = c.ctas[blockIdx.x];
    ClipSeg g = share.seg;
    for (int s = share.seg0; s < share.seg1; ++s) {
        if (s > share.seg0) g = c.segs[s];
#ifdef BAOC_CHECKED
        if (!check_segment(ck, kKerGradNorm, c, s) || !check_range(ck, kKerGradNorm, c.partials + s, 8, 0) ||
            !check_caller_ptr(kKerGradNorm, c.src[c.segs[s].block], 1))
            return;
#endif
        const E* __restrict__ p = static_cast<const E*>(c.src[g.block]) + g.first;
        const int64_t words = g.count / V, rounds = words / (kThreads * kNormLoads);
        const uint4* q = reinterpret_cast<const uint4*>(p) + threadIdx.x;
        double acc[1] = {0.0};
        if (rounds > 0) {                               // a round is requested while the one before it is summed
            constexpr int kRound = kThreads * kNormLoads;
            uint4 w[kNormLoads], next[kNormLoads];
#pragma unroll
            for (int k = 0; k < kNormLoads; ++k) w[k] = ld_stream_u4(q + k * kThreads);
#pragma unroll 1
            for (int64_t r = 1; r < rounds; ++r, q += kRound) {
#pragma unroll
                for (int k = 0; k < kNormLoads; ++k) next[k] = ld_stream_u4(q + kRound + k * kThreads);
                acc[0] += sum_squares<DT, kNormLoads>(w, q);
#pragma unroll
                for (int k = 0; k < kNormLoads; ++k) w[k] = next[k];
            }
            acc[0] += sum_squares<DT, kNormLoads>(w, q);
            q += kRound;
        }
        const int rest = int(words - rounds * (kThreads * kNormLoads));
        for (int e = threadIdx.x; e < rest; e += kThreads, q += kThreads) {
            const uint4 w[1] = {ld_stream_u4(q)};
            acc[0] += sum_squares<DT, 1>(w, q);
        }
        if (threadIdx.x < g.count - words * V) {
            const double x = double(Vec<DT>::one(p + words * V + threadIdx.x));
            acc[0] = fma(x, x, acc[0]);
        }
        cta_reduce_store<1>(acc, c.partials + s);
    }
    let_later_kernel_start();
    __shared__ bool last;
    if (threadIdx.x == 0) last = take_ticket(c.ticket) == uint32_t(c.n_ctas - 1);      // (thread 0 has written the CTA's partial sums)
    __syncthreads();
    if (!last) return;
    finish_norm(c, max_norm, norms);
}

// Eight elements: two 16-byte loads of fp32, one of bf16.
template <int SRC>
__device__ __forceinline__ void load8(const typename Vec<SRC>::Elem* p, uint4& a, uint4& b) {
    a = ld_stream_u4(p);
    if constexpr (SRC == BAOC_F32) b = ld_stream_u4(p + 4);
}

// 1.14 G bf16 elements: 690 us behind the norm = 6.6 TB/s of one read and one write, the copy bandwidth; 124 M from fp32 to bf16:
// 117 us = 6.4 TB/s.  Tiles of 4096 elements (both kernels, bf16): 9.0 us at 2 Mi elements against 9.8 with 16384, 10.3 against 12.2
// at 4 Mi; from 8 Mi to 32 Mi = kClipSmallTotal the two stay within 4 % of one another, and above it 16384 leads: 71.4 against
// 72.7 us at 64 Mi, 133 against 139 at 128 Mi (fp32 to bf16: 109 against 114 and 211 against 215).  Policies that keep the
// norm's last bytes in L2 for this read, and orders that go with them, were measured and make no difference.
//
// dst = factor * src, one CTA per tile (last tiles first: any order takes the same time).  All but the factor is there before the norm has ended: a CTA
// that finds a place by then has its first elements in hand when the factor comes.
template <int SRC, int DST>
__global__ void __launch_bounds__(kThreads)
grad_clip_kernel(const ClipBufs c BAOC_CHECK_PARAM) {
    using ES = typename Vec<SRC>::Elem;
    using ED = typename Vec<DST>::Elem;
#ifdef BAOC_CHECKED
    {
        if (!check_range(ck, kKerGradClip, c.tiles + blockIdx.x, sizeof(Tile), 0)) return;
        const Tile ct = c.tiles[blockIdx.x];
        if (ct.block >= unsigned(ck.n_blocks)) { check_fail(kChkBlockIndex, kKerGradClip, ct.block, ck.n_blocks, blockIdx.x, 0); return; }
        if (!check_tile(ck, kKerGradClip, 0, ct.block, int64_t(ct.piece) * c.clip_tile, c.numel[ct.block]) ||
            !check_caller_ptr(kKerGradClip, c.src[ct.block], 1) || !check_caller_ptr(kKerGradClip, c.dst[ct.block], 2))
            return;
    }
#endif
    const Tile t = c.tiles[blockIdx.x];
    const int64_t base = int64_t(t.piece) * c.clip_tile;
    const int left = int(min64(c.numel[t.block] - base, c.clip_tile)), whole = left / 8 * 8;
    const ES* src = static_cast<const ES*>(c.src[t.block]) + base;
    ED* dst = static_cast<ED*>(c.dst[t.block]) + base;
    int e = int(threadIdx.x) * 8;
    uint4 a{}, b{};
    if (e < whole) load8<SRC>(src + e, a, b);
    wait_for_earlier_kernel();
    const float f = *c.factor;
    if (f == 1.0f && static_cast<const void*>(src) == static_cast<const void*>(dst)) return;
    while (e < whole) {
        float x[8];
        if constexpr (SRC == BAOC_BF16) {
            unpack8(a, x);
        } else {
            x[0] = __uint_as_float(a.x); x[1] = __uint_as_float(a.y); x[2] = __uint_as_float(a.z); x[3] = __uint_as_float(a.w);
            x[4] = __uint_as_float(b.x); x[5] = __uint_as_float(b.y); x[6] = __uint_as_float(b.z); x[7] = __uint_as_float(b.w);
        }
        ED* to = dst + e;
        e += kThreads * 8;
        if (e < whole) load8<SRC>(src + e, a, b);
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] *= f;
        if constexpr (DST == BAOC_BF16) {
            st_stream_u4(to, make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7])));
        } else {
            st_stream_f4(to, make_float4(x[0], x[1], x[2], x[3]));
            st_stream_f4(to + 4, make_float4(x[4], x[5], x[6], x[7]));
        }
    }
    if (int(threadIdx.x) < left - whole) {
        const float y = Vec<SRC>::one(src + whole + threadIdx.x) * f;
        if constexpr (DST == BAOC_BF16) dst[whole + threadIdx.x] = uint16_t(pack_bf16(y, 0.f));
        else dst[whole + threadIdx.x] = y;
    }
}

// Pointers into a device table, by value: ordered on the stream like the kernels that read them, also in a captured graph.
__global__ void clip_ptrs_kernel(const ClipPtrs p, const void** table, int n) {
    if (int(threadIdx.x) < n) table[threadIdx.x] = p.p[threadIdx.x];
}

namespace {

struct ClipLayout { size_t tile_list, numel, segs, cta_list, block_seg, src, dst, partials, ticket, factor, total; int64_t tiles, clip_tiles, max_segs; int ctas, clip_tile; };

ClipLayout clip_layout(const Handle* h) {
    ClipLayout L{};
    for (const baoc_block_t& b : h->blocks) L.tiles += ceil_div(b.numel, kNormTile);
    L.clip_tile = h->numel < kClipSmallTotal ? kClipTileSmall : kClipTile;
    for (const baoc_block_t& b : h->blocks) L.clip_tiles += ceil_div(b.numel, L.clip_tile);
    L.ctas = int(std::min<int64_t>(L.tiles, kNormCtas));
    const size_t n = size_t(h->n_blocks);
    L.max_segs = int64_t(n) + L.ctas - 1;              // a cut between two shares adds at most one
    size_t cur = 0;
    auto take = [&cur](size_t bytes) { const size_t o = cur; cur = size_t(round_up(int64_t(cur + bytes), 256)); return o; };
    L.tile_list = take(sizeof(Tile) * size_t(L.clip_tiles));
    L.numel = take(8 * n);
    L.segs = take(sizeof(ClipSeg) * size_t(L.max_segs));
    L.cta_list = take(sizeof(ClipCta) * size_t(L.ctas));
    L.block_seg = take(4 * (n + 1));
    L.src = take(8 * n);
    L.dst = take(8 * n);
    L.partials = take(8 * size_t(L.max_segs));
    L.ticket = take(4);
    L.factor = take(4);
    L.total = cur;
    return L;
}

int cuda_error(const Handle* h, const char* what, cudaError_t e) {
    return fail(h, BAOC_E_CUDA, std::string(what) + ": " + cudaGetErrorString(e));
}

// Check a host array of device pointers and bring the device table up to date: the upload is left out when the same
// pointers were last uploaded on the same stream and no graph that was captured from this handle can have replaced them.
int clip_pointers(Handle* h, const void* const* ptrs, std::vector<const void*>* cache, const void** table, cudaStream_t s,
                  const char* what) {
    const int n = h->n_blocks;
    for (int i = 0; i < n; ++i) {
        if (!ptrs[i]) return fail(h, BAOC_E_INVALID, std::string(what) + ": null block pointer");
        if (reinterpret_cast<uintptr_t>(ptrs[i]) & 15u) return fail(h, BAOC_E_ALIGN, std::string(what) + ": block pointer not 16-byte aligned");
    }
    if (cache->size() == size_t(n) && std::memcmp(cache->data(), ptrs, sizeof(void*) * size_t(n)) == 0) return BAOC_OK;
    cache->clear();
    for (int i = 0; i < n; i += kClipPtrChunk) {
        ClipPtrs p;
        const int m = n - i < kClipPtrChunk ? n - i : kClipPtrChunk;
        std::memcpy(p.p, ptrs + i, sizeof(void*) * size_t(m));
        clip_ptrs_kernel<<<1, kClipPtrChunk, 0, s>>>(p, table + i, m);
        const cudaError_t e = cudaGetLastError();
        if (e != cudaSuccess) return cuda_error(h, what, e);
        h->launches += 1;
    }
    if (!h->clip_captured) cache->assign(ptrs, ptrs + n);
    return BAOC_OK;
}

[[maybe_unused]] CheckCtx clip_ctx(const Handle* h) { return CheckCtx{h->cw, h->cw + h->cw_bytes, (long long)h->clip.n_segs, h->n_blocks, 0}; }

// What both calls do: checks, pointer tables, the norm kernel.
int clip_norm(Handle* h, const void* const* src, int src_dtype, void* const* dst, double max_norm, float* norms, cudaStream_t s,
              const char* what) {
    cudaStreamCaptureStatus cap = cudaStreamCaptureStatusNone;
    cudaError_t e = cudaStreamIsCapturing(s, &cap);
    if (e != cudaSuccess) return cuda_error(h, what, e);
    if (cap != cudaStreamCaptureStatusNone) h->clip_captured = true;
    if (h->clip_captured || h->last_clip_stream != s) { h->last_clip_src.clear(); h->last_clip_dst.clear(); }
    h->last_clip_stream = s;
    int rc = clip_pointers(h, src, &h->last_clip_src, h->clip.src, s, what);
    if (rc) return rc;
    if (dst) {
        rc = clip_pointers(h, const_cast<const void* const*>(dst), &h->last_clip_dst, const_cast<const void**>(h->clip.dst), s,
                           what);
        if (rc) return rc;
    }
    const unsigned grid = unsigned(h->clip.n_ctas);
    if (src_dtype == BAOC_BF16) grad_norm_kernel<BAOC_BF16><<<grid, kThreads, 0, s>>>(h->clip, max_norm, norms BAOC_CHECK_ARG(clip_ctx(h)));
    else grad_norm_kernel<BAOC_F32><<<grid, kThreads, 0, s>>>(h->clip, max_norm, norms BAOC_CHECK_ARG(clip_ctx(h)));
    e = cudaGetLastError();
    if (e != cudaSuccess) return cuda_error(h, "grad_norm_kernel", e);
    h->launches += 1;
    return BAOC_OK;
}

int check_call(Handle* h, const void* const* grads, int dtype, const float* norms, const char* what) {
    if (!grads || !norms) return fail(h, BAOC_E_INVALID, std::string(what) + ": null argument");
    if (dtype != BAOC_BF16 && dtype != BAOC_F32) return fail(h, BAOC_E_INVALID, std::string(what) + ": unknown dtype");
    if (reinterpret_cast<uintptr_t>(norms) & 3u) return fail(h, BAOC_E_ALIGN, std::string(what) + ": norms not 4-byte aligned");
    if (!h->cw) return fail(h, BAOC_E_STATE, std::string(what) + ": no clip workspace bound");
    return BAOC_OK;
}

}  // namespace

BAOC_DEFINE_CHECK_FETCH(clip_check_fetch)

}  // namespace baoc

using namespace baoc;

extern "C" {

int baoc_clip_workspace_bytes(const baoc_t* h, size_t* bytes) {
    if (!h || !bytes) return BAOC_E_INVALID;
    *bytes = clip_layout(h).total;
    return BAOC_OK;
}

int baoc_bind_clip_workspace(baoc_t* h, void* dev, size_t bytes, baoc_stream_t stream) try {
    if (!h) return BAOC_E_INVALID;
    if (!dev) return fail(h, BAOC_E_INVALID, "baoc_bind_clip_workspace: null workspace");
    if (reinterpret_cast<uintptr_t>(dev) & 255u) return fail(h, BAOC_E_ALIGN, "baoc_bind_clip_workspace: workspace not 256-byte aligned");
    const ClipLayout L = clip_layout(h);
    if (bytes < L.total) return fail(h, BAOC_E_WORKSPACE, "baoc_bind_clip_workspace: workspace too small");
    if (L.clip_tiles > int64_t(0x7fffffff)) return fail(h, BAOC_E_INVALID, "baoc_bind_clip_workspace: too many elements for one launch");
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    // (a captured upload would read the vectors below when the graph is replayed, long after they are gone)
    cudaStreamCaptureStatus cap = cudaStreamCaptureStatusNone;
    cudaError_t e = cudaStreamIsCapturing(s, &cap);
    if (e != cudaSuccess) return cuda_error(h, "baoc_bind_clip_workspace", e);
    if (cap != cudaStreamCaptureStatusNone) return fail(h, BAOC_E_STATE, "baoc_bind_clip_workspace: the stream is capturing; bind before the capture");
    char* ws = static_cast<char*>(dev);
    // share i: the tiles [i * tiles / ctas, (i + 1) * tiles / ctas) of all blocks in a row
    std::vector<ClipSeg> segs;
    std::vector<ClipCta> ctas;
    std::vector<int32_t> block_seg;
    segs.reserve(size_t(L.max_segs));
    int64_t tile = 0, cut = 0;                          // tiles dealt so far; where the present share ends
    for (int i = 0; i < h->n_blocks; ++i) {
        const int64_t n = h->blocks[i].numel, k = ceil_div(n, kNormTile);
        block_seg.push_back(int32_t(segs.size()));
        for (int64_t j = 0; j < k;) {
            if (tile + j == cut) {
                ctas.push_back(ClipCta{int32_t(segs.size()), 0, ClipSeg{}});
                cut = int64_t(ctas.size()) * L.tiles / L.ctas;
            }
            const int64_t m = std::min(k - j, cut - tile - j);
            segs.push_back(ClipSeg{j * kNormTile, std::min(n, (j + m) * kNormTile) - j * kNormTile, i, 0});
            j += m;
        }
        tile += k;
    }
    block_seg.push_back(int32_t(segs.size()));
    for (size_t c = 0; c < ctas.size(); ++c) {
        ctas[c].seg1 = c + 1 < ctas.size() ? ctas[c + 1].seg0 : int32_t(segs.size());
        ctas[c].seg = segs[size_t(ctas[c].seg0)];
    }
    auto up = [&](size_t at, const void* data, size_t size) { return cudaMemcpyAsync(ws + at, data, size, cudaMemcpyHostToDevice, s); };
    // the clip's tiles, last first
    std::vector<Tile> tiles;
    tiles.reserve(size_t(L.clip_tiles));
    for (int i = h->n_blocks - 1; i >= 0; --i)
        for (int64_t j = ceil_div(h->blocks[i].numel, L.clip_tile) - 1; j >= 0; --j) tiles.push_back(Tile{uint32_t(i), uint32_t(j)});
    std::vector<int64_t> numel;
    for (const baoc_block_t& b : h->blocks) numel.push_back(b.numel);
    e = up(L.segs, segs.data(), sizeof(ClipSeg) * segs.size());
    if (e == cudaSuccess) e = up(L.tile_list, tiles.data(), sizeof(Tile) * tiles.size());
    if (e == cudaSuccess) e = up(L.numel, numel.data(), 8 * numel.size());
    if (e == cudaSuccess) e = up(L.cta_list, ctas.data(), sizeof(ClipCta) * ctas.size());
    if (e == cudaSuccess) e = up(L.block_seg, block_seg.data(), 4 * block_seg.size());
    if (e == cudaSuccess) e = cudaMemsetAsync(ws + L.ticket, 0, 4, s);
    if (e != cudaSuccess) return cuda_error(h, "baoc_bind_clip_workspace", e);
    h->cw = ws; h->cw_bytes = bytes;
    h->clip = ClipBufs{reinterpret_cast<const Tile*>(ws + L.tile_list), reinterpret_cast<const int64_t*>(ws + L.numel), reinterpret_cast<const ClipSeg*>(ws + L.segs), reinterpret_cast<const ClipCta*>(ws + L.cta_list),
                       reinterpret_cast<const int32_t*>(ws + L.block_seg), reinterpret_cast<const void**>(ws + L.src),
                       reinterpret_cast<void**>(ws + L.dst), reinterpret_cast<double*>(ws + L.partials),
                       reinterpret_cast<uint32_t*>(ws + L.ticket), reinterpret_cast<float*>(ws + L.factor), int(L.clip_tiles), L.clip_tile, L.ctas, int(segs.size()), h->n_blocks};
    h->last_clip_src.clear(); h->last_clip_dst.clear();
    return BAOC_OK;
} catch (const std::bad_alloc&) {
    return BAOC_E_INVALID;
}

int baoc_grad_norm(baoc_t* h, const void* const* grads, int dtype, float* norms, baoc_stream_t stream) try {
    if (!h) return BAOC_E_INVALID;
    const int rc = check_call(h, grads, dtype, norms, "baoc_grad_norm");
    if (rc) return rc;
    return clip_norm(h, grads, dtype, nullptr, 0.0, norms, static_cast<cudaStream_t>(stream), "baoc_grad_norm");
} catch (const std::bad_alloc&) {
    return BAOC_E_INVALID;
}

int baoc_clip_grads(baoc_t* h, const void* const* src, int src_dtype, void* const* dst, int dst_dtype, double max_norm,
                    float* norms, baoc_stream_t stream) try {
    if (!h) return BAOC_E_INVALID;
    const char* what = "baoc_clip_grads";
    int rc = check_call(h, src, src_dtype, norms, what);
    if (rc) return rc;
    if (!dst) return fail(h, BAOC_E_INVALID, "baoc_clip_grads: null argument");
    if (!(dst_dtype == src_dtype || (src_dtype == BAOC_F32 && dst_dtype == BAOC_BF16)))
        return fail(h, BAOC_E_INVALID, "baoc_clip_grads: offered types are bf16 -> bf16, fp32 -> fp32 and fp32 -> bf16");
    if (!(std::isfinite(max_norm) && max_norm >= 0.0)) return fail(h, BAOC_E_INVALID, "baoc_clip_grads: max_norm must be finite and >= 0");
    const int64_t es = src_dtype == BAOC_F32 ? 4 : 2, ed = dst_dtype == BAOC_F32 ? 4 : 2;
    for (int i = 0; i < h->n_blocks; ++i) {
        const char* a = static_cast<const char*>(src[i]);
        const char* b = static_cast<const char*>(dst[i]);
        if (a == b && es == ed) continue;
        if (a < b + ed * h->blocks[i].numel && b < a + es * h->blocks[i].numel)
            return fail(h, BAOC_E_INVALID, "baoc_clip_grads: a destination overlaps its source without being it");
    }
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    rc = clip_norm(h, src, src_dtype, dst, max_norm, norms, s, what);
    if (rc) return rc;
    const unsigned grid = unsigned(h->clip.n_tiles);
    auto launch = [&](auto kernel) { return launch_behind(kernel, grid, kThreads, s, h->clip BAOC_CHECK_ARG(clip_ctx(h))); };
    const cudaError_t e = dst_dtype == BAOC_F32 ? launch(grad_clip_kernel<BAOC_F32, BAOC_F32>)
                          : (src_dtype == BAOC_F32 ? launch(grad_clip_kernel<BAOC_F32, BAOC_BF16>) : launch(grad_clip_kernel<BAOC_BF16, BAOC_BF16>));
    if (e != cudaSuccess) return cuda_error(h, "grad_clip_kernel", e);
    h->launches += 1;
    return BAOC_OK;
} catch (const std::bad_alloc&) {
    return BAOC_E_INVALID;
}

}  // extern "C"
