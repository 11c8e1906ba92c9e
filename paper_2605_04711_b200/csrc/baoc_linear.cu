// A matrix product with bias, activation and residual in its epilogue, and its gradient, on the tensor cores.
//
//   z = x w^T + b,   pre = z,   out = act(z) + residual
//   dz = dout * act'(pre),   dx = dz w,   dw = dz^T x,   db = sum over rows of dz
//
// One kernel forms all three products, D[m, n] = sum_k A[m, k] B[n, k]: which of an operand's dimensions lies contiguous is a
// flag of its descriptor, so neither w nor x nor dz is ever transposed in memory.  Operands are bf16, sums fp32 in tensor memory.
// A CTA works through tiles of 128 x kN: one thread keeps tiled copies of 64 k in flight through a ring of stages, one issues
// the products, and eight warps write the last tile out while the next one's products run into the other half of the
// accumulators.  Edges come from the copies' zero fill; only the stores look at the true sizes.
// Times below: one B200, device time per call in a row of calls on three sets of arrays.
#include <algorithm>
#include <atomic>
#include <cmath>
#include <cuda_runtime.h>
#include <new>
#include <string>

#include "baoc_tensor.cuh"

namespace baoc {

constexpr int kTileM = 128, kTileK = 64;
constexpr int kRowBytes = 128;                       // of a stage's operand: 64 bf16
constexpr int kLinearMaxDim = 1 << 24;
constexpr int64_t kLinearMaxTokens = int64_t(1) << 30, kLinearMaxStride = int64_t(1) << 28;
constexpr int kWriters = 8;                          // warps of the epilogue
constexpr int kProductThreads = 128 + 32 * kWriters;
constexpr int kBand = 16;                            // tiles along m that are worked on side by side: their operands stay in L2
constexpr int kStageBudget = 200 * 1024;             // shared memory of the ring

template <int kN>
struct TileShape {
    static constexpr int kABytes = kTileM * kRowBytes, kBBytes = kN * kRowBytes, kStage = kABytes + kBBytes;
    static constexpr int kStages = kStageBudget / kStage > 8 ? 8 : kStageBudget / kStage;
    static constexpr int kSmem = kStages * kStage + 1024;
    static constexpr int kColumns = 2 * kN;          // of tensor memory: two accumulators
};

__device__ unsigned int g_gave_up;                   // CTAs in which a wait ran out

struct ProductArgs {
    int m, n, k_tiles, passes;       // passes: products of as many operand pairs are added up
    int a_mn, b_mn;                  // the operand's m (n) lies contiguous, not its k
    int act, out_f32;
    char *out, *pre;
    const char* residual;
    const float* bias;
    int64_t out_step, pre_step, residual_step;      // bytes
    int out_wide, pre_wide, residual_wide;           // 16-byte accesses fit
};

struct Maps { CUtensorMap a[3], b[3]; };

__device__ __forceinline__ float sigmoid(float z) { return __fdividef(1.f, 1.f + __expf(-z)); }

template <int kAct>
__device__ __forceinline__ float act_of(float z) {
    if constexpr (kAct == BAOC_ACT_RELU) return z > 0.f || z != z ? z : 0.f;
    if constexpr (kAct == BAOC_ACT_GELU) return 0.5f * z * erfcf(-0.70710678118654752f * z);
    if constexpr (kAct == BAOC_ACT_GELU_TANH) return __fdividef(z, 1.f + __expf(-1.5957691216057308f * (z + 0.044715f * z * z * z)));
    if constexpr (kAct == BAOC_ACT_SILU) return __fdividef(z, 1.f + __expf(-z));
    return z;
}
template <int kAct>
__device__ __forceinline__ void act_all(float (&v)[32]) {
#pragma unroll
    for (int i = 0; i < 32; ++i) v[i] = act_of<kAct>(v[i]);
}
__device__ __forceinline__ void apply_act(float (&v)[32], int act) {
    switch (act) {
        case BAOC_ACT_RELU: act_all<BAOC_ACT_RELU>(v); break;
        case BAOC_ACT_GELU: act_all<BAOC_ACT_GELU>(v); break;
        case BAOC_ACT_GELU_TANH: act_all<BAOC_ACT_GELU_TANH>(v); break;
        case BAOC_ACT_SILU: act_all<BAOC_ACT_SILU>(v); break;
        default: break;
    }
}
// (past the ends below the derivative is 0 or 1 to all bits, and its formula would form inf * 0)
__device__ __forceinline__ float act_slope(float z, int act) {
    switch (act) {
        case BAOC_ACT_RELU: return z > 0.f ? 1.f : (z != z ? z : 0.f);
        case BAOC_ACT_GELU: return fabsf(z) > 15.f ? (z > 0.f ? 1.f : 0.f) : 0.5f * erfcf(-0.70710678118654752f * z) + 0.3989422804014327f * z * __expf(-0.5f * z * z);
        case BAOC_ACT_GELU_TANH: {
            if (fabsf(z) > 15.f) return z > 0.f ? 1.f : 0.f;
            const float s = sigmoid(1.5957691216057308f * (z + 0.044715f * z * z * z));
            return s + z * s * (1.f - s) * 1.5957691216057308f * (1.f + 0.134145f * z * z);
        }
        case BAOC_ACT_SILU: {
            if (fabsf(z) > 90.f) return z > 0.f ? 1.f : 0.f;
            const float s = sigmoid(z);
            return s * (1.f + z * (1.f - s));
        }
        default: return 1.f;
    }
}

__device__ __forceinline__ uint32_t pair_bf16(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ uint16_t one_bf16(float x) {
    uint16_t h;
    asm("cvt.rn.bf16.f32 %0, %1;" : "=h"(h) : "f"(x));
    return h;
}

// `count` of a row's 32 columns from column col on
__device__ __forceinline__ void store_columns(char* row, int64_t col, int count, int f32, int wide, const float (&v)[32]) {
    if (f32) {
        float* p = reinterpret_cast<float*>(row) + col;
        if (wide && count == 32) {
#pragma unroll
            for (int i = 0; i < 32; i += 4) *reinterpret_cast<float4*>(p + i) = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
        } else {
#pragma unroll
            for (int i = 0; i < 32; ++i)
                if (i < count) p[i] = v[i];
        }
    } else {
        uint16_t* p = reinterpret_cast<uint16_t*>(row) + col;
        if (wide && count == 32) {
#pragma unroll
            for (int i = 0; i < 32; i += 8)
                *reinterpret_cast<uint4*>(p + i) = make_uint4(pair_bf16(v[i], v[i + 1]), pair_bf16(v[i + 2], v[i + 3]), pair_bf16(v[i + 4], v[i + 5]), pair_bf16(v[i + 6], v[i + 7]));
        } else {
#pragma unroll
            for (int i = 0; i < 32; ++i)
                if (i < count) p[i] = one_bf16(v[i]);
        }
    }
}
__device__ __forceinline__ void add_columns(const char* row, int64_t col, int count, int f32, int wide, float (&v)[32]) {
    if (f32) {
        const float* p = reinterpret_cast<const float*>(row) + col;
        if (wide && count == 32) {
#pragma unroll
            for (int i = 0; i < 32; i += 4) {
                const float4 a = *reinterpret_cast<const float4*>(p + i);
                v[i] += a.x; v[i + 1] += a.y; v[i + 2] += a.z; v[i + 3] += a.w;
            }
        } else {
#pragma unroll
            for (int i = 0; i < 32; ++i)
                if (i < count) v[i] += p[i];
        }
    } else {
        const uint16_t* p = reinterpret_cast<const uint16_t*>(row) + col;
        if (wide && count == 32) {
#pragma unroll
            for (int i = 0; i < 32; i += 8) {
                float x[8];
                unpack8(*reinterpret_cast<const uint4*>(p + i), x);
#pragma unroll
                for (int j = 0; j < 8; ++j) v[i + j] += x[j];
            }
        } else {
#pragma unroll
            for (int i = 0; i < 32; ++i)
                if (i < count) v[i] += bf16_bits_to_float(p[i]);
        }
    }
}

// Tile number to its place: bands of kBand tiles along m, each worked through column by column.
__device__ __forceinline__ void tile_place(int tile, int m_tiles, int n_tiles, int* mt, int* nt) {
    const int band = tile / (kBand * n_tiles), first = band * kBand, height = min(kBand, m_tiles - first), in = tile - band * kBand * n_tiles;
    *nt = in / height;
    *mt = first + in - *nt * height;
}

template <int kN>
__global__ void __launch_bounds__(kProductThreads, 1) product_kernel(const __grid_constant__ Maps maps, const ProductArgs g) {
    using T = TileShape<kN>;
    constexpr int kS = T::kStages;
    extern __shared__ char raw[];
    __shared__ uint64_t bars[2 * kS + 5];
    __shared__ uint32_t acc_at;
    __shared__ int failed;
    const uint32_t ring = (smem_addr(raw) + 1023) & ~1023u, bar0 = smem_addr(bars);
    auto full = [&](int s) { return bar0 + 8 * s; };
    auto empty = [&](int s) { return bar0 + 8 * (kS + s); };
    auto acc_full = [&](int a) { return bar0 + 8 * (2 * kS + a); };
    auto acc_empty = [&](int a) { return bar0 + 8 * (2 * kS + 2 + a); };
    const uint32_t drained = bar0 + 8 * (2 * kS + 4);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int m_tiles = (g.m + kTileM - 1) / kTileM, n_tiles = (g.n + kN - 1) / kN, tiles = m_tiles * n_tiles, steps = g.k_tiles * g.passes;
    if (threadIdx.x == 0) {
        for (int s = 0; s < kS; ++s) { bar_init(full(s), 1); bar_init(empty(s), 1); }
        for (int a = 0; a < 2; ++a) { bar_init(acc_full(a), 1); bar_init(acc_empty(a), kWriters); }
        bar_init(drained, 1);
        failed = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 2) acc_alloc(smem_addr(&acc_at), T::kColumns);
    acc_fence_before();
    __syncthreads();
    acc_fence_after();
    const uint32_t acc = acc_at;

    if (warp == 0 && lane == 0) {                     // copies
        int s = 0, round = 0, issued = 0;
        bool ok = true;
        for (int tile = blockIdx.x; ok && tile < tiles; tile += gridDim.x) {
            int mt, nt;
            tile_place(tile, m_tiles, n_tiles, &mt, &nt);
            for (int i = 0; i < steps; ++i) {
                if (!(ok = bar_wait(empty(s), (round & 1) ^ 1))) break;
                bar_expect(full(s), T::kStage);
                const int pass = (i >= g.k_tiles) + (i >= 2 * g.k_tiles), k = (i - pass * g.k_tiles) * kTileK;
                const uint32_t a = ring + s * T::kStage, b = a + T::kABytes;
                if (g.a_mn) {
#pragma unroll
                    for (int c = 0; c < kTileM / 64; ++c) copy_tile(a + c * 64 * kRowBytes, &maps.a[pass], mt * kTileM + c * 64, k, full(s));
                } else {
                    copy_tile(a, &maps.a[pass], k, mt * kTileM, full(s));
                }
                if (g.b_mn) {
#pragma unroll
                    for (int c = 0; c < kN / 64; ++c) copy_tile(b + c * 64 * kRowBytes, &maps.b[pass], nt * kN + c * 64, k, full(s));
                } else {
                    copy_tile(b, &maps.b[pass], k, nt * kN, full(s));
                }
                ++issued;
                if (++s == kS) { s = 0; ++round; }
            }
        }
        if (!ok) {
            failed = 1;
            // this CTA's copies have to have landed before its shared memory goes: stage j was filled (issued - 1 - j) / kS + 1 times
            for (int j = 0; j < min(issued, kS); ++j) bar_wait(full(j), ((issued - 1 - j) / kS) & 1);
        }
    } else if (warp == 1 && lane == 0) {              // products
        const uint32_t desc = product_desc(kTileM, kN, g.a_mn, g.b_mn);
        const uint32_t a_step = g.a_mn ? 16 * kRowBytes : 32, b_step = g.b_mn ? 16 * kRowBytes : 32;    // bytes per 16 k
        int s = 0, round = 0, count = 0;
        bool ok = true;
        for (int tile = blockIdx.x; ok && tile < tiles; tile += gridDim.x, ++count) {
            const int half = count & 1;
            if (!(ok = bar_wait(acc_empty(half), ((count >> 1) & 1) ^ 1))) break;
            acc_fence_after();
            const uint32_t d = acc + half * kN;
            for (int i = 0; i < steps; ++i) {
                if (!(ok = bar_wait(full(s), round & 1))) break;
                const uint32_t a = ring + s * T::kStage, b = a + T::kABytes;
#pragma unroll
                for (int k = 0; k < kTileK / 16; ++k)
                    product(d, operand_desc(a + k * a_step, 64 * kRowBytes), operand_desc(b + k * b_step, 64 * kRowBytes), desc, i > 0 || k > 0);
                product_commit(empty(s));
                if (++s == kS) { s = 0; ++round; }
            }
            product_commit(acc_full(half));
        }
        if (!ok) {                                    // (products in flight read shared and write tensor memory)
            failed = 1;
            product_commit(drained);
            bar_wait(drained, 0);
        }
    } else if (warp >= 4) {                           // write out
        const int quarter = warp & 3, side = (warp - 4) >> 2;       // a warp reads its quarter of the lanes alone
        int count = 0;
        for (int tile = blockIdx.x; tile < tiles; tile += gridDim.x, ++count) {
            const int half = count & 1;
            int mt, nt;
            tile_place(tile, m_tiles, n_tiles, &mt, &nt);
            if (!bar_wait(acc_full(half), (count >> 1) & 1)) { failed = 1; break; }
            acc_fence_after();
            const int64_t row = int64_t(mt) * kTileM + quarter * 32 + lane;
            for (int c = side * (kN / 2); c < (side + 1) * (kN / 2); c += 32) {
                const int col = nt * kN + c, left = min(32, g.n - col);
                if (left <= 0) break;                 // (alike in the warp)
                float v[32];
                acc_load(acc + half * kN + (uint32_t(quarter * 32) << 16) + c, v);
                if (row < g.m) {
                    if (g.bias) {
#pragma unroll
                        for (int i = 0; i < 32; ++i) v[i] += i < left ? __ldg(g.bias + col + i) : 0.f;
                    }
                    if (g.pre) store_columns(g.pre + row * g.pre_step, col, left, 0, g.pre_wide, v);
                    apply_act(v, g.act);
                    if (g.residual) add_columns(g.residual + row * g.residual_step, col, left, g.out_f32, g.residual_wide, v);
                    store_columns(g.out + row * g.out_step, col, left, g.out_f32, g.out_wide, v);
                }
                __syncwarp();                         // (the next load is the whole warp's)
            }
            acc_fence_before();
            __syncwarp();
            if (lane == 0) bar_arrive(acc_empty(half));
        }
    }
    __syncwarp();
    acc_fence_before();
    __syncthreads();
    if (warp == 2) {
        acc_fence_after();
        acc_free(acc, T::kColumns);
    }
    if (threadIdx.x == 0 && failed) atomicAdd(&g_gave_up, 1u);
}

// ---- what goes in front of the products ---------------------------------------------------------------------------
// Rows copied to where a tiled copy can read them: base and row stride multiples of 16 bytes.
struct Repack { const char* from; char* to; int64_t from_step, to_step, rows; int cols; };
struct Repacks { Repack r[3]; int64_t ends[3]; int n; };       // ends: running counts of 8-column pieces

__global__ void __launch_bounds__(kThreads) repack_kernel(const Repacks g) {
    for (int64_t i = int64_t(blockIdx.x) * kThreads + threadIdx.x; i < g.ends[g.n - 1]; i += int64_t(gridDim.x) * kThreads) {
        int which = 0;
        while (i >= g.ends[which]) ++which;
        const Repack& r = g.r[which];
        const int64_t at = i - (which ? g.ends[which - 1] : 0);
        const int pieces = (r.cols + 7) / 8;
        const int64_t row = at / pieces;
        const int col = int(at - row * pieces) * 8;
        const uint16_t* p = reinterpret_cast<const uint16_t*>(r.from + row * r.from_step) + col;
        uint16_t v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = col + j < r.cols ? p[j] : uint16_t(0);
        uint4 w;
        w.x = v[0] | uint32_t(v[1]) << 16; w.y = v[2] | uint32_t(v[3]) << 16; w.z = v[4] | uint32_t(v[5]) << 16; w.w = v[6] | uint32_t(v[7]) << 16;
        *reinterpret_cast<uint4*>(r.to + row * r.to_step + 2 * col) = w;
    }
}

// dz = dout * act'(pre) as bf16 (and what the rounding left, as two bf16 more, where dw is wanted in fp32), and its column sums.
// A CTA has 256 columns and rows_per_part rows: a lane 8 columns, a warp every eighth row.
struct SlopeArgs {
    const char *dout, *pre;
    char *dz, *dz_mid, *dz_low;      // null: not wanted
    float* part;                     // [part][n]; null: no column sums
    int64_t dout_step, pre_step, dz_step, rows, rows_per_part;
    int n, act, wide;
};

__device__ __forceinline__ void load8(const char* row, int col, int n, int wide, float (&x)[8]) {
    if (wide && col + 8 <= n) {
        unpack8(ld_stream_u4(row + 2 * int64_t(col)), x);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = col + j < n ? bf16_bits_to_float(reinterpret_cast<const uint16_t*>(row)[col + j]) : 0.f;
    }
}

__global__ void __launch_bounds__(kThreads) slope_kernel(const SlopeArgs g) {
    __shared__ float sh[8][256];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, col = int(blockIdx.x) * 256 + lane * 8;
    const int64_t first = int64_t(blockIdx.y) * g.rows_per_part, end = min64(g.rows, first + g.rows_per_part);
    float sum[8] = {};
    let_later_kernel_start();
    if (col < g.n)
        for (int64_t row = first + warp; row < end; row += 8) {
            float d[8];
            load8(g.dout + row * g.dout_step, col, g.n, g.wide, d);
            if (g.act != BAOC_ACT_NONE) {
                float z[8];
                load8(g.pre + row * g.pre_step, col, g.n, g.wide, z);
#pragma unroll
                for (int j = 0; j < 8; ++j) d[j] *= act_slope(z[j], g.act);
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) sum[j] += d[j];
            if (g.dz) {
                const uint4 w = make_uint4(pair_bf16(d[0], d[1]), pair_bf16(d[2], d[3]), pair_bf16(d[4], d[5]), pair_bf16(d[6], d[7]));
                *reinterpret_cast<uint4*>(g.dz + row * g.dz_step + 2 * int64_t(col)) = w;
                if (g.dz_mid) {
                    float h[8];
                    unpack8(w, h);
#pragma unroll
                    for (int j = 0; j < 8; ++j) d[j] -= h[j];
                    const uint4 m = make_uint4(pair_bf16(d[0], d[1]), pair_bf16(d[2], d[3]), pair_bf16(d[4], d[5]), pair_bf16(d[6], d[7]));
                    *reinterpret_cast<uint4*>(g.dz_mid + row * g.dz_step + 2 * int64_t(col)) = m;
                    unpack8(m, h);
#pragma unroll
                    for (int j = 0; j < 8; ++j) d[j] -= h[j];
                    *reinterpret_cast<uint4*>(g.dz_low + row * g.dz_step + 2 * int64_t(col)) =
                        make_uint4(pair_bf16(d[0], d[1]), pair_bf16(d[2], d[3]), pair_bf16(d[4], d[5]), pair_bf16(d[6], d[7]));
                }
            }
        }
    if (!g.part) return;
#pragma unroll
    for (int j = 0; j < 8; ++j) sh[warp][lane * 8 + j] = sum[j];
    __syncthreads();
    const int c = int(blockIdx.x) * 256 + int(threadIdx.x);
    if (c < g.n) {
        float s = sh[0][threadIdx.x];
        for (int w = 1; w < 8; ++w) s += sh[w][threadIdx.x];
        g.part[int64_t(blockIdx.y) * g.n + c] = s;
    }
}

// The parts' column sums, 32 columns per CTA: every warp adds each 32nd part, then the warps' sums are added in order.
__global__ void __launch_bounds__(1024) slope_sums_kernel(const float* __restrict__ part, int parts, int n, char* db, int f32) {
    __shared__ float sh[32][33];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, col = int(blockIdx.x) * 32 + lane;
    wait_for_earlier_kernel();
    float s = 0.f;
    if (col < n)
        for (int p = warp; p < parts; p += 32) s += part[int64_t(p) * n + col];
    sh[warp][lane] = s;
    __syncthreads();
    if (warp == 0 && col < n) {
        for (int w = 1; w < 32; ++w) s += sh[w][lane];
        if (f32) reinterpret_cast<float*>(db)[col] = s;
        else reinterpret_cast<uint16_t*>(db)[col] = one_bf16(s);
    }
}

namespace {

thread_local std::string g_linear_err;

int fail_linear(int code, const std::string& msg) {
    g_linear_err = msg;
    return code;
}
int64_t elem_bytes(int dtype) { return dtype == BAOC_F32 ? 4 : 2; }
bool aligned(const void* p, int64_t bytes) { return (reinterpret_cast<uintptr_t>(p) & uintptr_t(bytes - 1)) == 0; }
int launched(cudaError_t ce, const char* kernel) {
    return ce == cudaSuccess ? BAOC_OK : fail_linear(BAOC_E_CUDA, std::string(kernel) + ": " + cudaGetErrorString(ce));
}

int check_linear(const baoc_linear_t* e, int64_t tokens, const std::string& what) {
    if (!e) return fail_linear(BAOC_E_INVALID, what + ": null descriptor");
    if (e->n_in < 1 || e->n_in > kLinearMaxDim || e->n_out < 1 || e->n_out > kLinearMaxDim) return fail_linear(BAOC_E_INVALID, what + ": n_in and n_out must be in 1 .. 2^24");
    if (e->act < BAOC_ACT_NONE || e->act > BAOC_ACT_SILU) return fail_linear(BAOC_E_INVALID, what + ": unknown activation");
    if (e->layout != BAOC_OUT_IN && e->layout != BAOC_IN_OUT) return fail_linear(BAOC_E_INVALID, what + ": layout must be BAOC_OUT_IN or BAOC_IN_OUT");
    for (int t : {e->out_dtype, e->grad_dtype})
        if (t != BAOC_BF16 && t != BAOC_F32) return fail_linear(BAOC_E_INVALID, what + ": dtypes must be BAOC_BF16 or BAOC_F32");
    const int64_t w_cols = e->layout == BAOC_OUT_IN ? e->n_in : e->n_out;
    const int64_t strides[][2] = {{e->x_stride, e->n_in}, {e->w_stride, w_cols}, {e->out_stride, e->n_out}, {e->residual_stride, e->n_out}, {e->pre_stride, e->n_out},
                                  {e->dout_stride, e->n_out}, {e->dx_stride, e->n_in}, {e->dw_stride, w_cols}};
    for (const auto& s : strides)
        if (s[0] && (s[0] < s[1] || s[0] > kLinearMaxStride)) return fail_linear(BAOC_E_INVALID, what + ": a row stride must be 0 or from the row's length to 2^28");
    if (tokens < 0 || tokens > kLinearMaxTokens) return fail_linear(BAOC_E_INVALID, what + ": tokens must be in 0 .. 2^30");
    return BAOC_OK;
}

// A bf16 or fp32 matrix in memory.
struct Matrix {
    const char* p;
    int64_t rows, cols, step, eb;        // bytes from row to row, of an element
    Matrix(const void* p, int64_t rows, int64_t cols, int64_t stride, int dtype)
        : p(static_cast<const char*>(p)), rows(rows), cols(cols), step((stride ? stride : cols) * elem_bytes(dtype)), eb(elem_bytes(dtype)) {}
    bool wide() const { return aligned(p, 16) && step % 16 == 0; }
    bool fits() const { return aligned(p, eb); }
    int64_t end() const { return (rows - 1) * step + cols * eb; }
};
bool overlap(const Matrix& a, const Matrix& b) {
    if (!a.p || !b.p || !a.rows || !b.rows || a.p >= b.p + b.end() || b.p >= a.p + a.end()) return false;
    if (a.step != b.step) return true;
    const int64_t off = ((b.p - a.p) % a.step + a.step) % a.step;    // (rows of one buffer may lie between each other's)
    return off < a.cols * a.eb || off + b.cols * b.eb > a.step;
}

int64_t packed_step(int64_t cols) { return round_up(cols, 8) * 2; }
int64_t packed_bytes(int64_t rows, int64_t cols) { return round_up(rows * packed_step(cols), 256); }

using EncodeFn = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*, const cuuint32_t*,
                              CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeFn encode_fn() {
    static std::atomic<void*> found{nullptr};
    void* f = found.load(std::memory_order_acquire);
    if (!f) {
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &q) != cudaSuccess || q != cudaDriverEntryPointSuccess) return nullptr;
        found.store(f, std::memory_order_release);
    }
    return reinterpret_cast<EncodeFn>(f);
}

// Boxes of 64 contiguous elements by box_rows rows, laid out with the 128-byte swizzle; zeros outside.
bool encode(CUtensorMap* map, const Matrix& t, int box_rows) {
    EncodeFn f = encode_fn();
    if (!f) return false;
    const cuuint64_t dims[2] = {cuuint64_t(t.cols), cuuint64_t(t.rows)}, strides[1] = {cuuint64_t(t.step)};
    const cuuint32_t box[2] = {64, cuuint32_t(box_rows)}, unit[2] = {1, 1};
    return f(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<char*>(t.p), dims, strides, box, unit, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
             CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// A product's operands: a as [m][k] or, a_mn, as [k][m]; b as [n][k] or [k][n]; up to three pairs whose products are added.
struct Operands { const Matrix *a[3], *b[3]; };

template <int kN>
int launch_product(const Operands& o, ProductArgs g, cudaStream_t s) {
    using T = TileShape<kN>;
    static std::atomic<uint64_t> allowed{0};         // the permission for large shared memory is per device and lasts
    int dev = 0;
    cudaError_t ce = cudaGetDevice(&dev);
    if (ce != cudaSuccess) return launched(ce, "product_kernel");
    const uint64_t bit = dev < 64 ? uint64_t(1) << dev : 0;
    if (!(allowed.load(std::memory_order_relaxed) & bit)) {
        ce = cudaFuncSetAttribute(product_kernel<kN>, cudaFuncAttributeMaxDynamicSharedMemorySize, T::kSmem);
        if (ce != cudaSuccess) return launched(ce, "product_kernel");
        allowed.fetch_or(bit, std::memory_order_relaxed);
    }
    Maps maps;
    for (int i = 0; i < g.passes; ++i)
        if (!encode(&maps.a[i], *o.a[i], g.a_mn ? kTileK : kTileM) || !encode(&maps.b[i], *o.b[i], g.b_mn ? kTileK : kN))
            return fail_linear(BAOC_E_CUDA, "the driver refused a tensor map");
    const int64_t tiles = ceil_div(g.m, kTileM) * ceil_div(g.n, kN);
    if (tiles > 0x7fffffff - 148) return fail_linear(BAOC_E_INVALID, "too many tiles for one launch");
    product_kernel<kN><<<unsigned(std::min<int64_t>(tiles, 148)), kProductThreads, T::kSmem, s>>>(maps, g);
    return launched(cudaGetLastError(), "product_kernel");
}

int form_product(const Operands& o, const ProductArgs& g, cudaStream_t s) {
    const int64_t m_tiles = ceil_div(g.m, kTileM);
    if (m_tiles * ceil_div(g.n, 256) >= 148) return launch_product<256>(o, g, s);
    if (m_tiles * ceil_div(g.n, 128) >= 148) return launch_product<128>(o, g, s);
    return launch_product<64>(o, g, s);
}

// Matrices that a tiled copy cannot read go through the workspace: `at` is where the next one may lie.
struct Packer {
    char *at, *end;
    Repacks todo{};
    bool fits = true;
    Packer(void* ws, size_t bytes) : at(static_cast<char*>(ws)), end(static_cast<char*>(ws) + bytes) {}
    char* take(int64_t bytes) {
        char* p = at;
        if (bytes > end - at) { fits = false; return nullptr; }
        at += bytes;
        return p;
    }
    Matrix operand(const Matrix& t) {
        if (t.wide()) return t;
        char* p = take(packed_bytes(t.rows, t.cols));
        if (p) {
            const int64_t before = todo.n ? todo.ends[todo.n - 1] : 0;
            todo.r[todo.n] = Repack{t.p, p, t.step, packed_step(t.cols), t.rows, int(t.cols)};
            todo.ends[todo.n++] = before + t.rows * ceil_div(t.cols, 8);
        }
        return Matrix(p, t.rows, t.cols, packed_step(t.cols) / 2, BAOC_BF16);
    }
    int launch(cudaStream_t s) const {
        if (!todo.n) return BAOC_OK;
        const unsigned grid = unsigned(std::min<int64_t>(ceil_div(todo.ends[todo.n - 1], kThreads), 148 * 16));
        repack_kernel<<<grid, kThreads, 0, s>>>(todo);
        return launched(cudaGetLastError(), "repack_kernel");
    }
};

// Rows per part of the slope kernel: enough CTAs for the GPU, at least 8 rows (one per warp).
int64_t slope_parts(int64_t tokens, int64_t n, int64_t* rows_per_part) {
    const int64_t want = ceil_div(int64_t(148) * 8, ceil_div(n, 256));
    *rows_per_part = std::max<int64_t>(8, round_up(ceil_div(tokens, want), 8));
    return ceil_div(tokens, *rows_per_part);
}
// (most parts that so many tokens or fewer can get)
int64_t slope_bytes(int64_t tokens, int64_t n) {
    const int64_t want = ceil_div(int64_t(148) * 8, ceil_div(n, 256));
    return round_up(std::min(want, ceil_div(tokens, 8)) * n * 4, 256);
}

bool off_grid(int64_t stride, int64_t cols, int anywhere) { return anywhere || (stride ? stride : cols) % 8; }

}  // namespace

}  // namespace baoc

using namespace baoc;

extern "C" {

const char* baoc_linear_last_error(void) { return g_linear_err.c_str(); }

int baoc_linear_status(int32_t* gave_up) try {
    if (!gave_up) return fail_linear(BAOC_E_INVALID, "baoc_linear_status: null pointer");
    unsigned int n = 0;
    cudaError_t ce = cudaDeviceSynchronize();
    if (ce == cudaSuccess) ce = cudaMemcpyFromSymbol(&n, g_gave_up, sizeof n);
    if (ce == cudaSuccess && n) {
        const unsigned int zero = 0;
        ce = cudaMemcpyToSymbol(g_gave_up, &zero, sizeof zero);
    }
    if (ce != cudaSuccess) return launched(ce, "baoc_linear_status");
    *gave_up = int32_t(std::min<unsigned>(n, 0x7fffffff));
    return BAOC_OK;
} catch (const std::bad_alloc&) {
    return BAOC_E_INVALID;
}

int baoc_linear_workspace_bytes(const baoc_linear_t* e, int64_t tokens, int anywhere, size_t* bytes) try {
    const int rc = check_linear(e, tokens, "baoc_linear_workspace_bytes");
    if (rc) return rc;
    if (!bytes) return fail_linear(BAOC_E_INVALID, "baoc_linear_workspace_bytes: null pointer");
    const int64_t w_rows = e->layout == BAOC_OUT_IN ? e->n_out : e->n_in, w_cols = e->layout == BAOC_OUT_IN ? e->n_in : e->n_out;
    int64_t n = 0;
    if (off_grid(e->x_stride, e->n_in, anywhere)) n += packed_bytes(tokens, e->n_in);
    if (off_grid(e->w_stride, w_cols, anywhere)) n += packed_bytes(w_rows, w_cols);
    *bytes = size_t(n);
    return BAOC_OK;
} catch (const std::bad_alloc&) {
    return BAOC_E_INVALID;
}

int baoc_linear(const baoc_linear_t* e, const void* x, const void* w, const float* bias, const void* residual, int64_t tokens, void* out, void* pre,
                void* ws, size_t ws_bytes, baoc_stream_t stream) try {
    int rc = check_linear(e, tokens, "baoc_linear");
    if (rc) return rc;
    if (tokens == 0) return BAOC_OK;
    if (!x || !w || !out || (!ws && ws_bytes)) return fail_linear(BAOC_E_INVALID, "baoc_linear: null pointer");
    const bool out_in = e->layout == BAOC_OUT_IN;
    const Matrix mx(x, tokens, e->n_in, e->x_stride, BAOC_BF16), mw(w, out_in ? e->n_out : e->n_in, out_in ? e->n_in : e->n_out, e->w_stride, BAOC_BF16),
        mo(out, tokens, e->n_out, e->out_stride, e->out_dtype), mr(residual, tokens, e->n_out, e->residual_stride, e->out_dtype), mp(pre, tokens, e->n_out, e->pre_stride, BAOC_BF16);
    for (const Matrix* t : {&mx, &mw, &mo, &mr, &mp})
        if (!t->fits()) return fail_linear(BAOC_E_ALIGN, "baoc_linear: a pointer is not aligned to its elements");
    if (!aligned(bias, 4)) return fail_linear(BAOC_E_ALIGN, "baoc_linear: a pointer is not aligned to its elements");
    if (!aligned(ws, 256)) return fail_linear(BAOC_E_ALIGN, "baoc_linear: workspace not 256-byte aligned");
    const Matrix space(ws, 1, int64_t(ws_bytes) / 2, 0, BAOC_BF16);
    if (overlap(mo, mx) || overlap(mo, mw) || overlap(mp, mx) || overlap(mp, mw) || overlap(mo, mp) || overlap(mp, mr) ||
        (overlap(mo, mr) && !(mo.p == mr.p && (mo.step == mr.step || tokens == 1))))
        return fail_linear(BAOC_E_INVALID, "baoc_linear: out may be residual; outputs overlap nothing else");
    if (ws_bytes)
        for (const Matrix* t : {&mx, &mw, &mo, &mr, &mp})
            if (overlap(space, *t)) return fail_linear(BAOC_E_INVALID, "baoc_linear: the workspace overlaps an array");
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    Packer pack(ws, ws_bytes);
    const Matrix a = pack.operand(mx), b = pack.operand(mw);
    if (!pack.fits) return fail_linear(BAOC_E_WORKSPACE, "baoc_linear: workspace too small");
    if ((rc = pack.launch(s))) return rc;
    ProductArgs g{};
    g.m = int(tokens); g.n = e->n_out; g.k_tiles = int(ceil_div(e->n_in, kTileK)); g.passes = 1;
    g.b_mn = !out_in;
    g.act = e->act; g.out_f32 = e->out_dtype == BAOC_F32;
    g.out = static_cast<char*>(out); g.pre = static_cast<char*>(pre); g.residual = mr.p; g.bias = bias;
    g.out_step = mo.step; g.pre_step = mp.step; g.residual_step = mr.step;
    g.out_wide = mo.wide(); g.pre_wide = mp.wide(); g.residual_wide = mr.wide();
    return form_product(Operands{{&a}, {&b}}, g, s);
} catch (const std::bad_alloc&) {
    return BAOC_E_INVALID;
}

int baoc_linear_grad_workspace_bytes(const baoc_linear_t* e, int64_t tokens, int anywhere, size_t* bytes) try {
    const int rc = check_linear(e, tokens, "baoc_linear_grad_workspace_bytes");
    if (rc) return rc;
    if (!bytes) return fail_linear(BAOC_E_INVALID, "baoc_linear_grad_workspace_bytes: null pointer");
    const int64_t w_rows = e->layout == BAOC_OUT_IN ? e->n_out : e->n_in, w_cols = e->layout == BAOC_OUT_IN ? e->n_in : e->n_out;
    int64_t n = slope_bytes(tokens, e->n_out);
    if (off_grid(e->x_stride, e->n_in, anywhere)) n += packed_bytes(tokens, e->n_in);
    if (off_grid(e->w_stride, w_cols, anywhere)) n += packed_bytes(w_rows, w_cols);
    if (e->act != BAOC_ACT_NONE || off_grid(e->dout_stride, e->n_out, anywhere)) n += packed_bytes(tokens, e->n_out);
    if (e->act != BAOC_ACT_NONE && e->grad_dtype == BAOC_F32) n += 2 * packed_bytes(tokens, e->n_out);
    *bytes = size_t(n);
    return BAOC_OK;
} catch (const std::bad_alloc&) {
    return BAOC_E_INVALID;
}

int baoc_linear_grad(const baoc_linear_t* e, const void* x, const void* w, const void* dout, const void* pre, int64_t tokens, void* dx, void* dw,
                     void* db, void* ws, size_t ws_bytes, baoc_stream_t stream) try {
    const char* what = "baoc_linear_grad";
    int rc = check_linear(e, tokens, what);
    if (rc) return rc;
    const bool out_in = e->layout == BAOC_OUT_IN, act = e->act != BAOC_ACT_NONE;
    if (tokens && (!dout || (act && !pre) || (dx && !w) || (dw && !x) || (!ws && ws_bytes))) return fail_linear(BAOC_E_INVALID, "baoc_linear_grad: null pointer");
    const int64_t w_rows = out_in ? e->n_out : e->n_in, w_cols = out_in ? e->n_in : e->n_out;
    const Matrix mx(dw ? x : nullptr, tokens, e->n_in, e->x_stride, BAOC_BF16), mw(dx ? w : nullptr, w_rows, w_cols, e->w_stride, BAOC_BF16),
        md(dout, tokens, e->n_out, e->dout_stride, BAOC_BF16), mp(act ? pre : nullptr, tokens, e->n_out, e->pre_stride, BAOC_BF16),
        mdx(dx, tokens, e->n_in, e->dx_stride, BAOC_BF16), mdw(dw, w_rows, w_cols, e->dw_stride, e->grad_dtype), mdb(db, 1, e->n_out, 0, e->grad_dtype);
    for (const Matrix* t : {&mx, &mw, &md, &mp, &mdx, &mdw, &mdb})
        if (!t->fits()) return fail_linear(BAOC_E_ALIGN, "baoc_linear_grad: a pointer is not aligned to its elements");
    if (!aligned(ws, 256)) return fail_linear(BAOC_E_ALIGN, "baoc_linear_grad: workspace not 256-byte aligned");
    const Matrix space(ws_bytes ? ws : nullptr, 1, int64_t(ws_bytes) / 2, 0, BAOC_BF16);
    const Matrix* ins[] = {&mx, &mw, &md, &mp, &space};
    const Matrix* outs[] = {&mdx, &mdw, &mdb};
    for (int i = 0; i < 3; ++i) {
        for (const Matrix* t : ins)
            if (overlap(*outs[i], *t)) return fail_linear(BAOC_E_INVALID, "baoc_linear_grad: an output overlaps another array");
        for (int j = 0; j < i; ++j)
            if (overlap(*outs[i], *outs[j])) return fail_linear(BAOC_E_INVALID, "baoc_linear_grad: an output overlaps another array");
    }
    for (int i = 0; i < 4; ++i)
        if (overlap(space, *ins[i])) return fail_linear(BAOC_E_INVALID, "baoc_linear_grad: the workspace overlaps an array");
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (tokens == 0) {                               // sums over nothing
        cudaError_t ce = cudaSuccess;
        if (dw) ce = cudaMemset2DAsync(dw, size_t(mdw.step), 0, size_t(mdw.cols * mdw.eb), size_t(mdw.rows), s);
        if (ce == cudaSuccess && db) ce = cudaMemsetAsync(db, 0, size_t(mdb.cols * mdb.eb), s);
        return launched(ce, "baoc_linear_grad");
    }
    Packer pack(ws, ws_bytes);
    const Matrix bx = dw ? pack.operand(mx) : mx, bw = dx ? pack.operand(mw) : mw;
    // dz: dout itself where nothing changes it and a tiled copy can read it
    SlopeArgs g{};
    Matrix dz = md, mid = md, low = md;
    const bool split = act && dw && e->grad_dtype == BAOC_F32;
    if ((act || !md.wide()) && (dx || dw)) {
        g.dz = pack.take(packed_bytes(tokens, e->n_out));
        dz = Matrix(g.dz, tokens, e->n_out, packed_step(e->n_out) / 2, BAOC_BF16);
        if (split) {
            g.dz_mid = pack.take(packed_bytes(tokens, e->n_out));
            g.dz_low = pack.take(packed_bytes(tokens, e->n_out));
            mid = Matrix(g.dz_mid, tokens, e->n_out, packed_step(e->n_out) / 2, BAOC_BF16);
            low = Matrix(g.dz_low, tokens, e->n_out, packed_step(e->n_out) / 2, BAOC_BF16);
        }
    }
    const int64_t parts = slope_parts(tokens, e->n_out, &g.rows_per_part);
    if (db) g.part = reinterpret_cast<float*>(pack.take(slope_bytes(tokens, e->n_out)));
    if (!pack.fits) return fail_linear(BAOC_E_WORKSPACE, "baoc_linear_grad: workspace too small");
    if ((rc = pack.launch(s))) return rc;
    if (g.dz || g.part) {
        g.dout = md.p; g.pre = mp.p; g.dout_step = md.step; g.pre_step = mp.step; g.dz_step = packed_step(e->n_out);
        g.rows = tokens; g.n = e->n_out; g.act = e->act; g.wide = md.wide() && (!act || mp.wide());
        slope_kernel<<<dim3(unsigned(ceil_div(e->n_out, 256)), unsigned(parts)), kThreads, 0, s>>>(g);
        if ((rc = launched(cudaGetLastError(), "slope_kernel"))) return rc;
        if (g.part && (rc = launched(launch_behind(slope_sums_kernel, unsigned(ceil_div(e->n_out, 32)), 1024, s, static_cast<const float*>(g.part), int(parts), int(e->n_out),
                                                   static_cast<char*>(db), int(e->grad_dtype == BAOC_F32)), "slope_sums_kernel")))
            return rc;
    }
    if (dx) {
        ProductArgs p{};
        p.m = int(tokens); p.n = e->n_in; p.k_tiles = int(ceil_div(e->n_out, kTileK)); p.passes = 1;
        p.b_mn = out_in;
        p.out = static_cast<char*>(dx); p.out_step = mdx.step; p.out_wide = mdx.wide();
        if ((rc = form_product(Operands{{&dz}, {&bw}}, p, s))) return rc;
    }
    if (dw) {
        ProductArgs p{};
        p.m = int(w_rows); p.n = int(w_cols); p.k_tiles = int(ceil_div(tokens, kTileK)); p.passes = split ? 3 : 1;
        p.a_mn = p.b_mn = 1;
        p.out = static_cast<char*>(dw); p.out_step = mdw.step; p.out_wide = mdw.wide(); p.out_f32 = e->grad_dtype == BAOC_F32;
        const Operands o = out_in ? Operands{{&dz, &mid, &low}, {&bx, &bx, &bx}} : Operands{{&bx, &bx, &bx}, {&dz, &mid, &low}};
        if ((rc = form_product(o, p, s))) return rc;
    }
    return BAOC_OK;
} catch (const std::bad_alloc&) {
    return BAOC_E_INVALID;
}

}  // extern "C"
