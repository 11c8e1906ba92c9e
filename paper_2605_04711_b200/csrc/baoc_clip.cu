// Global gradient norm over the handle's blocks, and clipping by it.
//
//   n_i = ||g_i||,  n = sqrt(sum_i n_i^2),  dst_i = min(1, max_norm / (n + 1e-6)) * src_i.
#include <cmath>
#include <cstring>
#include <cuda_runtime.h>
#include <new>

#include "baoc_device.cuh"

namespace baoc {

constexpr double kClipEps = 1e-6;
// A thread's fp32 sum of up to 64 squares is taken as it is inside this range: no square has overflowed, and what
// squares below the smallest fp32 number have lost is under 64 * 2^-150 of at least 1e-30.
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

// Sum of squares of the elements held in K 16-byte words of one thread: fp32, or double where fp32 squares would leave
// their range (infinities and NaN end there too and pass through).
template <int DT, int K>
__device__ __forceinline__ double sum_squares(const uint4 (&w)[K]) {
    float a[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < K; ++k) {
        float x[Vec<DT>::kN];
        Vec<DT>::floats(w[k], x);
#pragma unroll
        for (int j = 0; j < Vec<DT>::kN; ++j) a[j & 3] = fmaf(x[j], x[j], a[j & 3]);
    }
    const float s = (a[0] + a[1]) + (a[2] + a[3]);
    if (s >= kSquaresLo && s <= kSquaresHi) return double(s);
    uint32_t any = 0;
#pragma unroll
    for (int k = 0; k < K; ++k) any |= w[k].x | w[k].y | w[k].z | w[k].w;
    if ((any & (DT == BAOC_BF16 ? 0x7fff7fffu : 0x7fffffffu)) == 0u) return 0.0;
    double d = 0.0;
#pragma unroll
    for (int k = 0; k < K; ++k) {
        float x[Vec<DT>::kN];
        Vec<DT>::floats(w[k], x);
#pragma unroll
        for (int j = 0; j < Vec<DT>::kN; ++j) d = fma(double(x[j]), double(x[j]), d);
    }
    return d;
}

// Sum of n doubles that other CTAs have written, in a fixed order.  Loaded past L1, which may hold a line from before.
__device__ __forceinline__ void sum_slots(const double* slots, int n, double* out) {
    double acc[1] = {0.0};
#pragma unroll 4
    for (int i = threadIdx.x; i < n; i += kThreads) acc[0] += __ldcg(slots + i);
    cta_reduce_store<1>(acc, out);
}

// One CTA per tile.  Its sum of squares goes to the tile's slot; the last CTA of a block adds the block's slots, the
// last block's CTA adds the blocks, each in a fixed order.
template <int DT>
__global__ void __launch_bounds__(kThreads)
grad_norm_kernel(const ClipBufs c, double max_norm, float* __restrict__ norms BAOC_CHECK_PARAM) {
    constexpr int V = Vec<DT>::kN, kLoads = 8;
    using E = typename Vec<DT>::Elem;
#ifdef BAOC_CHECKED
    {
        if (int64_t(blockIdx.x) >= ck.n_tiles) { check_fail(kChkTileIndex, kKerGradNorm, blockIdx.x, ck.n_tiles, 0, 0); return; }
        const Tile ct = c.tiles[blockIdx.x];
        if (ct.block >= unsigned(ck.n_blocks)) { check_fail(kChkBlockIndex, kKerGradNorm, ct.block, ck.n_blocks, blockIdx.x, 0); return; }
        const ClipBlock& cb = c.blocks[ct.block];
        if (!check_tile(ck, kKerGradNorm, blockIdx.x, ct.block, int64_t(ct.piece) * kClipTile, cb.numel) ||
            !check_range(ck, kKerGradNorm, c.partials + cb.tile0, 8ll * cb.ntiles, 0) ||
            !check_range(ck, kKerGradNorm, c.bsq, 8ll * c.n_blocks, 1) ||
            !check_range(ck, kKerGradNorm, c.tickets, 4ll * (c.n_blocks + 1), 2) ||
            !check_caller_ptr(kKerGradNorm, c.src[ct.block], 3))
            return;
    }
#endif
    const Tile t = c.tiles[blockIdx.x];
    const ClipBlock b = c.blocks[t.block];
    const E* __restrict__ g = static_cast<const E*>(c.src[t.block]);
    const int64_t base = int64_t(t.piece) * kClipTile;
    const int64_t left = b.numel - base;
    double acc[1] = {0.0};
    if (left >= kClipTile) {
#pragma unroll 1
        for (int r = 0; r < kClipTile / (kThreads * V * kLoads); ++r) {
            uint4 w[kLoads];
#pragma unroll
            for (int k = 0; k < kLoads; ++k)
                w[k] = ld_stream_u4(g + base + (int64_t(r * kLoads + k) * kThreads + threadIdx.x) * V);
            acc[0] += sum_squares<DT, kLoads>(w);
        }
    } else {
        for (int64_t e = int64_t(threadIdx.x) * V; e < left; e += kThreads * V) {
            if (e + V <= left) {
                uint4 w[1] = {ld_stream_u4(g + base + e)};
                acc[0] += sum_squares<DT, 1>(w);
            } else {
                for (int64_t j = e; j < left; ++j) {
                    const double x = double(Vec<DT>::one(g + base + j));
                    acc[0] = fma(x, x, acc[0]);
                }
            }
        }
    }
    cta_reduce_store<1>(acc, c.partials + blockIdx.x);

    __shared__ bool last;
    __shared__ double sum;
    if (threadIdx.x == 0) {
        __threadfence();
        last = atomicAdd(c.tickets + t.block, 1u) == uint32_t(b.ntiles - 1);
    }
    __syncthreads();
    if (!last) return;
    __threadfence();
    sum_slots(c.partials + b.tile0, b.ntiles, &sum);
    if (threadIdx.x == 0) {
        c.bsq[t.block] = sum;
        norms[1 + t.block] = float(sqrt(sum));
        c.tickets[t.block] = 0u;
        __threadfence();
        last = atomicAdd(c.tickets + c.n_blocks, 1u) == uint32_t(c.n_blocks - 1);
    }
    __syncthreads();
    if (!last) return;
    __threadfence();
    sum_slots(c.bsq, c.n_blocks, &sum);
    if (threadIdx.x == 0) {
        const double n = sqrt(sum);
        norms[0] = float(n);
        const double f = max_norm / (n + kClipEps);
        *c.factor = f < 1.0 ? float(f) : (f >= 1.0 ? 1.0f : float(n));      // (a NaN norm is a NaN factor)
        c.tickets[c.n_blocks] = 0u;
    }
}

// dst = factor * src, one CTA per tile, the last tiles first: they are what the norm has just read, and what the L2
// cache still holds.
template <int SRC, int DST>
__global__ void __launch_bounds__(kThreads)
grad_clip_kernel(const ClipBufs c BAOC_CHECK_PARAM) {
    using ES = typename Vec<SRC>::Elem;
    using ED = typename Vec<DST>::Elem;
    const int64_t tile = c.n_tiles - 1 - int64_t(blockIdx.x);
#ifdef BAOC_CHECKED
    {
        if (int64_t(blockIdx.x) >= ck.n_tiles) { check_fail(kChkTileIndex, kKerGradClip, blockIdx.x, ck.n_tiles, 0, 0); return; }
        const Tile ct = c.tiles[tile];
        if (ct.block >= unsigned(ck.n_blocks)) { check_fail(kChkBlockIndex, kKerGradClip, ct.block, ck.n_blocks, tile, 0); return; }
        if (!check_tile(ck, kKerGradClip, tile, ct.block, int64_t(ct.piece) * kClipTile, c.blocks[ct.block].numel) ||
            !check_caller_ptr(kKerGradClip, c.src[ct.block], 0) || !check_caller_ptr(kKerGradClip, c.dst[ct.block], 1))
            return;
    }
#endif
    const Tile t = c.tiles[tile];
    const ES* src = static_cast<const ES*>(c.src[t.block]);
    ED* dst = static_cast<ED*>(c.dst[t.block]);
    const int64_t base = int64_t(t.piece) * kClipTile;
    const int64_t left = min64(c.blocks[t.block].numel - base, kClipTile);
    const float f = *c.factor;
    if (f == 1.0f && static_cast<const void*>(src) == static_cast<const void*>(dst)) return;
    for (int64_t e = int64_t(threadIdx.x) * 8; e < left; e += kThreads * 8) {
        if (e + 8 <= left) {
            float x[8];
            if (SRC == BAOC_BF16) unpack8(ld_stream_u4(src + base + e), x);
            else f4_to8(ld_stream_f4(src + base + e), ld_stream_f4(src + base + e + 4), x);
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] *= f;
            if (DST == BAOC_BF16) {
                st_stream_u4(dst + base + e, make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7])));
            } else {
                st_stream_f4(dst + base + e, make_float4(x[0], x[1], x[2], x[3]));
                st_stream_f4(dst + base + e + 4, make_float4(x[4], x[5], x[6], x[7]));
            }
        } else {
            for (int64_t j = base + e; j < base + left; ++j) {
                const float y = Vec<SRC>::one(src + j) * f;
                if constexpr (DST == BAOC_BF16) dst[j] = uint16_t(pack_bf16(y, 0.f));
                else dst[j] = y;
            }
        }
    }
}

// Pointers into a device table, by value: ordered on the stream like the kernels that read them, also in a captured graph.
__global__ void clip_ptrs_kernel(const ClipPtrs p, const void** table, int n) {
    if (int(threadIdx.x) < n) table[threadIdx.x] = p.p[threadIdx.x];
}

namespace {

struct ClipLayout { size_t blocks, tiles, src, dst, partials, bsq, tickets, factor, total; int64_t n_tiles; };

ClipLayout clip_layout(const Handle* h) {
    ClipLayout L{};
    for (const baoc_block_t& b : h->blocks) L.n_tiles += ceil_div(b.numel, kClipTile);
    const size_t n = size_t(h->n_blocks);
    size_t cur = 0;
    auto take = [&cur](size_t bytes) { const size_t o = cur; cur = size_t(round_up(int64_t(cur + bytes), 256)); return o; };
    L.blocks = take(sizeof(ClipBlock) * n);
    L.tiles = take(sizeof(Tile) * size_t(L.n_tiles));
    L.src = take(8 * n);
    L.dst = take(8 * n);
    L.partials = take(8 * size_t(L.n_tiles));
    L.bsq = take(8 * n);
    L.tickets = take(4 * (n + 1));
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

[[maybe_unused]] CheckCtx clip_ctx(const Handle* h) { return CheckCtx{h->cw, h->cw + h->cw_bytes, (long long)h->clip.n_tiles, h->n_blocks, 0}; }

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
    const unsigned grid = unsigned(h->clip.n_tiles);
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
    if (L.n_tiles > int64_t(0x7fffffff)) return fail(h, BAOC_E_INVALID, "baoc_bind_clip_workspace: too many tiles for one launch");
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    char* ws = static_cast<char*>(dev);
    std::vector<ClipBlock> cb(size_t(h->n_blocks));
    std::vector<Tile> tiles;
    tiles.reserve(size_t(L.n_tiles));
    for (int i = 0; i < h->n_blocks; ++i) {
        const int64_t n = h->blocks[i].numel, k = ceil_div(n, kClipTile);
        cb[i] = ClipBlock{n, int64_t(tiles.size()), int32_t(k), 0};
        for (int64_t j = 0; j < k; ++j) tiles.push_back(Tile{uint32_t(i), uint32_t(j)});
    }
    cudaError_t e = cudaMemcpyAsync(ws + L.blocks, cb.data(), sizeof(ClipBlock) * cb.size(), cudaMemcpyHostToDevice, s);
    if (e == cudaSuccess) e = cudaMemcpyAsync(ws + L.tiles, tiles.data(), sizeof(Tile) * tiles.size(), cudaMemcpyHostToDevice, s);
    if (e == cudaSuccess) e = cudaMemsetAsync(ws + L.tickets, 0, 4 * (size_t(h->n_blocks) + 1), s);
    if (e != cudaSuccess) return cuda_error(h, "baoc_bind_clip_workspace", e);
    h->cw = ws; h->cw_bytes = bytes;
    h->clip = ClipBufs{reinterpret_cast<const ClipBlock*>(ws + L.blocks), reinterpret_cast<const Tile*>(ws + L.tiles),
                       reinterpret_cast<const void**>(ws + L.src), reinterpret_cast<void**>(ws + L.dst),
                       reinterpret_cast<double*>(ws + L.partials), reinterpret_cast<double*>(ws + L.bsq),
                       reinterpret_cast<uint32_t*>(ws + L.tickets), reinterpret_cast<float*>(ws + L.factor), L.n_tiles, h->n_blocks};
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
    if (dst_dtype == BAOC_F32) grad_clip_kernel<BAOC_F32, BAOC_F32><<<grid, kThreads, 0, s>>>(h->clip BAOC_CHECK_ARG(clip_ctx(h)));
    else if (src_dtype == BAOC_F32) grad_clip_kernel<BAOC_F32, BAOC_BF16><<<grid, kThreads, 0, s>>>(h->clip BAOC_CHECK_ARG(clip_ctx(h)));
    else grad_clip_kernel<BAOC_BF16, BAOC_BF16><<<grid, kThreads, 0, s>>>(h->clip BAOC_CHECK_ARG(clip_ctx(h)));
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return cuda_error(h, "grad_clip_kernel", e);
    h->launches += 1;
    return BAOC_OK;
} catch (const std::bad_alloc&) {
    return BAOC_E_INVALID;
}

}  // extern "C"
