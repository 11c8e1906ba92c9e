// The token table: row lookup with scaling, and its gradient by grouped tokens.
//
//   out[t, :]    = scale * table[ids[t], :]
//   dtable[v, :] = scale * sum over t with ids[t] = v of dout[t, :]
#include <cmath>
#include <cuda_runtime.h>
#include <new>
#include <string>

#include "baoc_device.cuh"

namespace baoc {

constexpr int kGroupCtas = 128;        // id classes (one CTA each) of the grouping; doubled while a class has over kGroupBins ids
constexpr int kGroupBins = 1024;       // most ids of a class: one thread of the CTA per id
constexpr int kGroupWarps = 32;
constexpr int kEmbedMaxDim = 1 << 24;
constexpr int64_t kEmbedMaxStride = 1 << 28;           // (row products stay far inside 64 bits)

__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

// V consecutive elements of a bf16 or fp32 row, as floats.
template <int DT, int V>
__device__ __forceinline__ void load_row(const void* row, int64_t e, float (&x)[V]) {
    if constexpr (DT == BAOC_BF16) {
        const uint16_t* p = static_cast<const uint16_t*>(row) + e;
        if constexpr (V == 8) unpack8(__ldg(reinterpret_cast<const uint4*>(p)), x);
        else x[0] = bf16_bits_to_float(__ldg(p));
    } else {
        const float* p = static_cast<const float*>(row) + e;
        if constexpr (V == 8) f4_to8(__ldg(reinterpret_cast<const float4*>(p)), __ldg(reinterpret_cast<const float4*>(p) + 1), x);
        else x[0] = __ldg(p);
    }
}
template <int DT, int V>
__device__ __forceinline__ void store_row(void* row, int64_t e, const float (&x)[V]) {
    if constexpr (DT == BAOC_BF16) {
        uint16_t* p = static_cast<uint16_t*>(row) + e;
        if constexpr (V == 8) st_stream_u4(p, make_uint4(bf16_pair(x[0], x[1]), bf16_pair(x[2], x[3]), bf16_pair(x[4], x[5]), bf16_pair(x[6], x[7])));
        else *p = uint16_t(bf16_pair(x[0], 0.f));
    } else {
        float* p = static_cast<float*>(row) + e;
        if constexpr (V == 8) {
            st_stream_f4(p, make_float4(x[0], x[1], x[2], x[3]));
            st_stream_f4(p + 4, make_float4(x[4], x[5], x[6], x[7]));
        } else {
            *p = x[0];
        }
    }
}

// What the kernels take of a descriptor.  Strides in elements.
struct EmbedArgs {
    int64_t vocab, n, pad;
    int64_t src_stride, dst_stride;
    int dim;
    float scale;
};

// ---- lookup: one thread per V elements of a row -----------------------------------------------------------------
template <int SRC, int DST, int V, typename Id>
__global__ void __launch_bounds__(kThreads)
embed_kernel(const void* __restrict__ table, const Id* __restrict__ ids, void* __restrict__ out, const EmbedArgs a) {
    constexpr int ss = SRC == BAOC_BF16 ? 2 : 4, ds = DST == BAOC_BF16 ? 2 : 4;
    const int per_row = a.dim / V;
    const int64_t k = int64_t(blockIdx.x) * kThreads + threadIdx.x;
    const int64_t t = k / per_row;
    if (t >= a.n) return;
    const int64_t e = (k - t * per_row) * V;
    const int64_t id = int64_t(ids[t]);
    float x[V];
    if (id >= 0 && id < a.vocab) {
        load_row<SRC, V>(static_cast<const char*>(table) + id * a.src_stride * ss, e, x);
#pragma unroll
        for (int j = 0; j < V; ++j) x[j] *= a.scale;
    } else {
#pragma unroll
        for (int j = 0; j < V; ++j) x[j] = 0.f;
    }
    store_row<DST, V>(static_cast<char*>(out) + t * a.dst_stride * ds, e, x);
}

// ---- gradient, first kernel: group the tokens by id -----------------------------------------------------------------
// The ids fall into n_ctas = 2^shift classes by their low bits; CTA c lists the tokens of class c, ordered by id and
// within an id by token.  Every CTA reads all ids and counts those of lower classes too, which is where its part of the
// list begins: no CTA waits for another.  start[] has one entry per (class, id of the class) and one more, perm[] one
// per listed token.
template <typename Id>
__global__ void __launch_bounds__(kGroupWarps * 32)
embed_group_kernel(const Id* __restrict__ ids, int n, int64_t vocab, int64_t pad, int shift, int bins, int32_t* __restrict__ start,
                   int32_t* __restrict__ perm BAOC_CHECK_PARAM) {
    extern __shared__ int32_t hist[];                   // [warps][bins]
    __shared__ int32_t s_warp[kGroupWarps];
    __shared__ int32_t s_less;
#ifdef BAOC_CHECKED
    if (!check_range(ck, kKerEmbedGroup, start + size_t(blockIdx.x) * bins, 4ll * (bins + 1), 0) ||
        !check_range(ck, kKerEmbedGroup, perm, 4ll * n, 1))
        return;
#endif
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint32_t cls = blockIdx.x, mask = (1u << shift) - 1u;
    for (int i = threadIdx.x; i < kGroupWarps * bins; i += blockDim.x) hist[i] = 0;
    if (threadIdx.x == 0) s_less = 0;
    __syncthreads();
    // a warp takes one stretch of the tokens, so that its list is in their order
    const int seg = ((n + kGroupWarps - 1) / kGroupWarps + 31) / 32 * 32;
    const int t0 = min(n, warp * seg), t1 = min(n, t0 + seg);
    int32_t* mine = hist + warp * bins;
    int less = 0;
    for (int t = t0 + lane; t < t1; t += 32) {
        const int64_t id = int64_t(ids[t]);
        if (id < 0 || id >= vocab || id == pad) continue;
        const uint32_t c = uint32_t(id) & mask;
        less += c < cls;
        if (c == cls) atomicAdd(&mine[uint32_t(id) >> shift], 1);
    }
    less = __reduce_add_sync(0xffffffffu, less);
    if (lane == 0 && less) atomicAdd(&s_less, less);
    __syncthreads();
    // one thread per id: the warps' counts become offsets within the id, the ids' totals offsets within the list
    int total = 0;
    if (int(threadIdx.x) < bins) {
        for (int w = 0; w < kGroupWarps; ++w) {
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
    int before = s_less;
    for (int w = 0; w < warp; ++w) before += s_warp[w];
    const int first = before + incl - total;
    if (int(threadIdx.x) < bins) {
        for (int w = 0; w < kGroupWarps; ++w) hist[w * bins + threadIdx.x] += first;
        start[size_t(cls) * bins + threadIdx.x] = first;
        if (int(threadIdx.x) == bins - 1 && cls == mask) start[size_t(cls + 1) * bins] = first + total;
    }
    __syncthreads();
    for (int tb = t0; tb < t1; tb += 32) {
        const int t = tb + lane;
        const int64_t id = t < t1 ? int64_t(ids[t]) : -1;
        const bool in = id >= 0 && id < vocab && id != pad && (uint32_t(id) & mask) == cls;
        const uint32_t who = __ballot_sync(0xffffffffu, in);
        if (in) {
            const uint32_t bin = uint32_t(id) >> shift;
            const uint32_t peers = __match_any_sync(who, bin);
            const int rank = __popc(peers & ((1u << lane) - 1u));
            const int at = mine[bin];
            __syncwarp(who);
            if (rank == 0) mine[bin] = at + __popc(peers);
            perm[at + rank] = t;
        }
        __syncwarp();
    }
}

// ---- gradient, second kernel: one warp per row and 32 V columns -------------------------------------------------------
template <int ACT, int GRAD, int V>
__global__ void __launch_bounds__(kThreads)
embed_grad_kernel(const void* __restrict__ dout, void* dtable, const int32_t* __restrict__ start, const int32_t* __restrict__ perm,
                  int shift, int bins, int slabs, int accumulate, const EmbedArgs a BAOC_CHECK_PARAM) {
    constexpr int as = ACT == BAOC_BF16 ? 2 : 4, gs = GRAD == BAOC_BF16 ? 2 : 4;
    const int lane = threadIdx.x & 31;
    const int64_t item = (int64_t(blockIdx.x) * kThreads + threadIdx.x) >> 5;
    const int64_t v = item / slabs;
    const int e = int(item - v * slabs) * 32 * V + lane * V;
    if (v >= a.vocab) return;
    const size_t slot = size_t(v & ((1 << shift) - 1)) * bins + size_t(v >> shift);
#ifdef BAOC_CHECKED
    if (!check_range(ck, kKerEmbedGrad, start + slot, 8, 0)) return;
#endif
    const int32_t p0 = start[slot], p1 = start[slot + 1];
    if (e >= a.dim || (accumulate && p0 == p1)) return;
    float acc[V];
#pragma unroll
    for (int j = 0; j < V; ++j) acc[j] = 0.f;
    for (int32_t p = p0; p < p1; ++p) {
#ifdef BAOC_CHECKED
        if (!check_range(ck, kKerEmbedGrad, perm + p, 4, 1)) return;
        if (perm[p] < 0 || perm[p] >= a.n) { check_fail(kChkTileIndex, kKerEmbedGrad, perm[p], a.n, p, 2); return; }
#endif
        float x[V];
        load_row<ACT, V>(static_cast<const char*>(dout) + int64_t(perm[p]) * a.src_stride * as, e, x);
#pragma unroll
        for (int j = 0; j < V; ++j) acc[j] += x[j];
    }
    char* row = static_cast<char*>(dtable) + v * a.dst_stride * gs;
#pragma unroll
    for (int j = 0; j < V; ++j) acc[j] *= a.scale;
    if (accumulate) {
#pragma unroll
        for (int j = 0; j < V; ++j) {
            if constexpr (GRAD == BAOC_BF16) acc[j] += bf16_bits_to_float(reinterpret_cast<const uint16_t*>(row)[e + j]);
            else acc[j] += reinterpret_cast<const float*>(row)[e + j];
        }
    }
    store_row<GRAD, V>(row, e, acc);
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

// Whether rows of this array can be read and written 8 elements at a time.
bool wide(const void* p, int64_t stride, int64_t eb, int dim) { return dim % 8 == 0 && aligned(p, 16) && (stride * eb) % 16 == 0; }

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

struct EmbedLayout { size_t start, perm, total; int shift, bins; };

EmbedLayout embed_layout(const baoc_embed_t* e, int64_t n) {
    EmbedLayout L{};
    group_geometry(e->vocab, &L.shift, &L.bins);
    L.start = 0;
    L.perm = size_t(round_up(4 * ((int64_t(L.bins) << L.shift) + 1), 256));
    L.total = L.perm + size_t(round_up(4 * n, 256));
    return L;
}

template <typename F>
int with_types(int a, int b, F f) {
    if (a == BAOC_F32) return b == BAOC_F32 ? f(std::integral_constant<int, BAOC_F32>{}, std::integral_constant<int, BAOC_F32>{})
                                            : f(std::integral_constant<int, BAOC_F32>{}, std::integral_constant<int, BAOC_BF16>{});
    return b == BAOC_F32 ? f(std::integral_constant<int, BAOC_BF16>{}, std::integral_constant<int, BAOC_F32>{})
                         : f(std::integral_constant<int, BAOC_BF16>{}, std::integral_constant<int, BAOC_BF16>{});
}

int launched(const char* kernel) {
    const cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? BAOC_OK : fail_embed(BAOC_E_CUDA, std::string(kernel) + ": " + cudaGetErrorString(e));
}

template <int S, int D, int V, typename Id>
int launch_embed(const void* table, const void* ids, void* out, const EmbedArgs& a, cudaStream_t s) {
    const int64_t blocks = ceil_div(a.n * (a.dim / V), kThreads);
    if (blocks > int64_t(0x7fffffff)) return fail_embed(BAOC_E_INVALID, "baoc_embed: too many elements for one launch");
    embed_kernel<S, D, V, Id><<<unsigned(blocks), kThreads, 0, s>>>(table, static_cast<const Id*>(ids), out, a);
    return launched("embed_kernel");
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
    const EmbedArgs a{e->vocab, n_tokens, e->pad_id, ts, os, e->dim, e->scale};
    const bool w = wide(table, ts, tb, e->dim) && wide(out, os, ob, e->dim);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    return with_types(e->table_dtype, e->act_dtype, [&](auto S, auto D) {
        if (w) return e->id_bits == 64 ? launch_embed<S(), D(), 8, int64_t>(table, ids, out, a, s) : launch_embed<S(), D(), 8, int32_t>(table, ids, out, a, s);
        return e->id_bits == 64 ? launch_embed<S(), D(), 1, int64_t>(table, ids, out, a, s) : launch_embed<S(), D(), 1, int32_t>(table, ids, out, a, s);
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
    int32_t* start = reinterpret_cast<int32_t*>(w + L.start);
    int32_t* perm = reinterpret_cast<int32_t*>(w + L.perm);
    const CheckCtx ck{w, w + L.total, 0, 0, 0};
    (void)ck;
    const int smem = 4 * kGroupWarps * L.bins;
    const void* group = e->id_bits == 64 ? reinterpret_cast<const void*>(embed_group_kernel<int64_t>) : reinterpret_cast<const void*>(embed_group_kernel<int32_t>);
    cudaError_t ce = cudaFuncSetAttribute(group, cudaFuncAttributeMaxDynamicSharedMemorySize, 4 * kGroupWarps * kGroupBins);
    if (ce != cudaSuccess) return fail_embed(BAOC_E_CUDA, std::string("embed_group_kernel: ") + cudaGetErrorString(ce));
    if (e->id_bits == 64)
        embed_group_kernel<int64_t><<<1u << L.shift, kGroupWarps * 32, smem, s>>>(static_cast<const int64_t*>(ids), int(n_tokens), e->vocab, e->pad_id, L.shift, L.bins, start, perm BAOC_CHECK_ARG(ck));
    else
        embed_group_kernel<int32_t><<<1u << L.shift, kGroupWarps * 32, smem, s>>>(static_cast<const int32_t*>(ids), int(n_tokens), e->vocab, e->pad_id, L.shift, L.bins, start, perm BAOC_CHECK_ARG(ck));
    rc = launched("embed_group_kernel");
    if (rc) return rc;
    const EmbedArgs a{e->vocab, n_tokens, e->pad_id, as, gs, e->dim, e->scale};
    const bool wd = wide(dout, as, ab, e->dim) && wide(dtable, gs, gb, e->dim);
    const int slabs = int(ceil_div(e->dim, 32 * (wd ? 8 : 1)));
    const int64_t blocks = ceil_div(e->vocab * slabs * 32, kThreads);
    if (blocks > int64_t(0x7fffffff)) return fail_embed(BAOC_E_INVALID, "baoc_embed_grad: too many elements for one launch");
    return with_types(e->act_dtype, e->grad_dtype, [&](auto A, auto G) {
        if (wd) embed_grad_kernel<A(), G(), 8><<<unsigned(blocks), kThreads, 0, s>>>(dout, dtable, start, perm, L.shift, L.bins, slabs, accumulate, a BAOC_CHECK_ARG(ck));
        else embed_grad_kernel<A(), G(), 1><<<unsigned(blocks), kThreads, 0, s>>>(dout, dtable, start, perm, L.shift, L.bins, slabs, accumulate, a BAOC_CHECK_ARG(ck));
        return launched("embed_grad_kernel");
    });
} catch (const std::bad_alloc&) {
    return BAOC_E_INVALID;
}

}  // extern "C"
