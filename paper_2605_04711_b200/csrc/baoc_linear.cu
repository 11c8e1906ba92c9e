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
constexpr int kSmemMost = 226 * 1024;                // shared memory of a CTA: the ring of stages, outputs on their way
constexpr int kChunk = 8;                            // steps of 64 k

// kCtas CTAs (a pair shares the tensor cores' work on a tile of 256 rows: each holds its 128 rows of A, half the columns' rows
// of B, and its rows' accumulators, so that a stage of both feeds twice the products of one CTA's).
// kChunked, for fp32 outputs: the tensor cores cut an accumulator's low bits off at every addition (2^-25 of it on average, always
// towards zero; at k = 8192 random products the result is off by 9e-6, at 16384 positive ones by 8e-5), so every
// kChunk steps the sums so far are added up in registers, rounded to nearest, and the accumulator starts again (5e-7).
template <int kCtas, int kN, bool kChunked>
struct TileShape {
    static constexpr int kBRows = kN / kCtas;
    static constexpr int kABytes = kTileM * kRowBytes, kBBytes = kBRows * kRowBytes, kStage = kABytes + kBBytes;
    static constexpr int kOutBytes = kChunked ? 4096 : 2048;         // 32 x 32 outputs of a writing warp, two of them
    static constexpr int kOuts = kWriters * 2 * kOutBytes;
    static constexpr int kStages = (kSmemMost - 1024 - kOuts) / kStage > 8 ? 8 : (kSmemMost - 1024 - kOuts) / kStage;
    static constexpr int kSmem = kStages * kStage + kOuts + 1024;
    static constexpr int kColumns = 2 * kN;          // of tensor memory: two accumulators
};

__device__ unsigned int g_gave_up;                   // CTAs in which a wait ran out

struct ProductArgs {
    int m, n, k_tiles, passes;       // passes: products of as many operand pairs are added up
    int a_mn, b_mn;                  // the operand's m (n) lies contiguous, not its k
    int a_rows;                      // rows of A that a copy brings: fewer than a tile's where m is smaller
    int act, out_f32;
    char *out, *pre;
    const char* residual;
    const float* bias;
    int64_t out_step, pre_step, residual_step;      // bytes
    int out_wide, pre_wide, residual_wide;           // 16-byte accesses fit; out and pre are then stored by tiled copies
};

struct Maps { CUtensorMap a[3], b[3], out, pre; };

__device__ __forceinline__ float exp2_approx(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
constexpr float kLog2e = 1.4426950408889634f;

// The normal distribution below -|z|, as e^(-z^2/2) times a polynomial in t = 1 / (1 + 0.35 |z|): erfc(x) e^(x^2) is smooth in
// such a t.  The coefficients are a least-maximum fit of the relative error over |z| <= 15 (3.2e-8 in exact arithmetic, 5 2^-24
// with the coefficients and every step in fp32); two approximate functions against some forty instructions of erfcf.
// Returns it and, in *density, e^(-z^2/2).
__device__ __forceinline__ float lower_tail(float z, float* density) {
    const float t = rcp_approx(fmaf(0.35f, fabsf(z), 1.f));
    float p = -0.02916380763053894f;
    p = fmaf(p, t, 0.14406023919582367f);
    p = fmaf(p, t, -0.2559007406234741f);
    p = fmaf(p, t, 0.15939167141914368f);
    p = fmaf(p, t, -0.02326301671564579f);
    p = fmaf(p, t, 0.10557447373867035f);
    p = fmaf(p, t, 0.11981557309627533f);
    p = fmaf(p, t, 0.13986432552337646f);
    p = fmaf(p, t, 0.13962125778198242f);
    *density = exp2_approx(-0.5f * kLog2e * (z * z));
    return p * t * *density;
}
__device__ __forceinline__ float sigmoid(float z) { return rcp_approx(1.f + exp2_approx(-kLog2e * z)); }

template <int kAct>
__device__ __forceinline__ float act_of(float z) {
    if constexpr (kAct == BAOC_ACT_RELU) return z > 0.f || z != z ? z : 0.f;
    if constexpr (kAct == BAOC_ACT_GELU) {
        float d;
        const float tail = lower_tail(z, &d);
        return z * (z > 0.f ? 1.f - tail : tail);
    }
    if constexpr (kAct == BAOC_ACT_GELU_TANH) return z * sigmoid(1.5957691216057308f * (z + 0.044715f * z * z * z));
    if constexpr (kAct == BAOC_ACT_SILU) return z * sigmoid(z);
    return z;
}
template <int kAct>
__device__ __forceinline__ void act_all(float* v, int n) {
#pragma unroll
    for (int i = 0; i < n; ++i) v[i] = act_of<kAct>(v[i]);
}
template <int kCount>
__device__ __forceinline__ void apply_act(float (&v)[kCount], int act) {
    switch (act) {
        case BAOC_ACT_RELU: act_all<BAOC_ACT_RELU>(v, kCount); break;
        case BAOC_ACT_GELU: act_all<BAOC_ACT_GELU>(v, kCount); break;
        case BAOC_ACT_GELU_TANH: act_all<BAOC_ACT_GELU_TANH>(v, kCount); break;
        case BAOC_ACT_SILU: act_all<BAOC_ACT_SILU>(v, kCount); break;
        default: break;
    }
}
// (past the ends below the derivative is 0 or 1 to all bits, and its formula would form inf * 0)
template <int kAct>
__device__ __forceinline__ float act_slope(float z) {
    if constexpr (kAct == BAOC_ACT_RELU) {
        return z > 0.f ? 1.f : (z != z ? z : 0.f);
    } else if constexpr (kAct == BAOC_ACT_GELU) {
        float d;
        const float y = fminf(fmaxf(z, -15.f), 15.f), tail = lower_tail(y, &d), r = (y > 0.f ? 1.f - tail : tail) + 0.3989422804014327f * y * d;
        return z != z ? z : r;
    } else if constexpr (kAct == BAOC_ACT_GELU_TANH) {
        const float y = fminf(fmaxf(z, -15.f), 15.f), s = sigmoid(1.5957691216057308f * (y + 0.044715f * y * y * y));
        const float r = s + y * s * (1.f - s) * 1.5957691216057308f * (1.f + 0.134145f * y * y);
        return z != z ? z : r;
    } else if constexpr (kAct == BAOC_ACT_SILU) {
        const float y = fminf(fmaxf(z, -90.f), 90.f), s = sigmoid(y), r = s * (1.f + y * (1.f - s));
        return z != z ? z : r;
    }
    return 1.f;
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

__device__ __forceinline__ void store4(char* row, int64_t col, int count, int f32, int wide, const float (&v)[4]) {
    if (f32) {
        float* p = reinterpret_cast<float*>(row) + col;
        if (wide && count == 4) *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
        else
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (i < count) p[i] = v[i];
    } else {
        uint16_t* p = reinterpret_cast<uint16_t*>(row) + col;
        if (wide && count == 4) *reinterpret_cast<uint2*>(p) = make_uint2(pair_bf16(v[0], v[1]), pair_bf16(v[2], v[3]));
        else
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (i < count) p[i] = one_bf16(v[i]);
    }
}

// Tile number to its place: bands of kBand tiles along m, each worked through column by column.
__device__ __forceinline__ void tile_place(int tile, int m_tiles, int n_tiles, int* mt, int* nt) {
    const int band = tile / (kBand * n_tiles), first = band * kBand, height = min(kBand, m_tiles - first), in = tile - band * kBand * n_tiles;
    *nt = in / height;
    *mt = first + in - *nt * height;
}

// What a writing warp does with 32 columns of its 32 rows.
struct Writer {
    const ProductArgs& g;
    const Maps& maps;
    uint32_t buf;                    // two buffers of `bytes`
    uint32_t bytes;
    int lane, turn = 0;

    // a thread's row of 32 values into the warp's buffer, as a tiled copy with swizzled rows expects it, and off
    __device__ __forceinline__ void send(const CUtensorMap* map, int f32, int col, int row0, const float (&v)[32]) {
        const uint32_t to = buf + turn * bytes;
        turn ^= 1;
        if (lane == 0) stores_read<1>();                   // (the store before last has left this buffer)
        __syncwarp();
        if (f32) {
#pragma unroll
            for (int c = 0; c < 8; ++c)
                asm volatile("st.shared.v4.f32 [%0], {%1,%2,%3,%4};" ::"r"(to + lane * 128 + ((c ^ (lane & 7)) << 4)), "f"(v[4 * c]), "f"(v[4 * c + 1]), "f"(v[4 * c + 2]),
                             "f"(v[4 * c + 3]) : "memory");
        } else {
#pragma unroll
            for (int c = 0; c < 4; ++c)
                asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(to + lane * 64 + ((c ^ ((lane >> 1) & 3)) << 4)), "r"(pair_bf16(v[8 * c], v[8 * c + 1])),
                             "r"(pair_bf16(v[8 * c + 2], v[8 * c + 3])), "r"(pair_bf16(v[8 * c + 4], v[8 * c + 5])), "r"(pair_bf16(v[8 * c + 6], v[8 * c + 7])) : "memory");
        }
        shared_to_async();
        __syncwarp();
        if (lane == 0) store_tile(map, to, col, row0);
    }
    // row0: the warp's first row (below m); the whole warp calls it
    __device__ __forceinline__ void write(int64_t row0, int col, float (&v)[32]) {
        const int left = min(32, g.n - col);
        const int64_t row = row0 + lane;
        const bool mine = row < g.m;
        if (g.bias) {
            if (left == 32 && (reinterpret_cast<uintptr_t>(g.bias) & 15) == 0) {
#pragma unroll
                for (int i = 0; i < 32; i += 4) {
                    const float4 b = __ldg(reinterpret_cast<const float4*>(g.bias + col + i));
                    v[i] += b.x; v[i + 1] += b.y; v[i + 2] += b.z; v[i + 3] += b.w;
                }
            } else {
#pragma unroll
                for (int i = 0; i < 32; ++i) v[i] += i < left ? __ldg(g.bias + col + i) : 0.f;
            }
        }
        if (g.pre) {
            if (g.pre_wide) send(&maps.pre, 0, col, int(row0), v);
            else if (mine) store_columns(g.pre + row * g.pre_step, col, left, 0, 0, v);
        }
        apply_act(v, g.act);
        if (g.residual && mine) add_columns(g.residual + row * g.residual_step, col, left, g.out_f32, g.residual_wide, v);
        if (g.out_wide) send(&maps.out, g.out_f32, col, int(row0), v);
        else if (mine) store_columns(g.out + row * g.out_step, col, left, g.out_f32, 0, v);
        __syncwarp();
    }
};

template <int kCtas, int kN, bool kChunked>
__global__ void __launch_bounds__(kProductThreads, 1) product_kernel(const __grid_constant__ Maps maps, const ProductArgs g) {
    using T = TileShape<kCtas, kN, kChunked>;
    constexpr int kS = T::kStages;
    extern __shared__ char raw[];
    __shared__ uint64_t bars[2 * kS + 5];
    __shared__ uint32_t acc_at;
    __shared__ int failed;
    const uint32_t ring = (smem_addr(raw) + 1023) & ~1023u, outs = ring + kS * T::kStage, bar0 = smem_addr(bars);
    auto full = [&](int s) { return bar0 + 8 * s; };
    auto empty = [&](int s) { return bar0 + 8 * (kS + s); };
    auto acc_full = [&](int a) { return bar0 + 8 * (2 * kS + a); };
    auto acc_empty = [&](int a) { return bar0 + 8 * (2 * kS + 2 + a); };
    const uint32_t drained = bar0 + 8 * (2 * kS + 4);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, rank = kCtas == 2 ? int(cluster_rank()) : 0;
    const int worker = int(blockIdx.x) / kCtas, workers = int(gridDim.x) / kCtas;
    const int m_tiles = (g.m + kTileM * kCtas - 1) / (kTileM * kCtas), n_tiles = (g.n + kN - 1) / kN, tiles = m_tiles * n_tiles, steps = g.k_tiles * g.passes;
    const int chunk = kChunked ? kChunk : steps, chunks = (steps + chunk - 1) / chunk;
    if (threadIdx.x == 0) {
        for (int s = 0; s < kS; ++s) { bar_init(full(s), 1); bar_init(empty(s), 1); }
        for (int a = 0; a < 2; ++a) { bar_init(acc_full(a), 1); bar_init(acc_empty(a), kWriters * kCtas); }
        bar_init(drained, 1);
        failed = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        shared_to_async();
    }
    if (warp == 2) acc_alloc<kCtas>(smem_addr(&acc_at), T::kColumns);
    acc_fence_before();
    if constexpr (kCtas == 2) cluster_barrier();
    else __syncthreads();
    acc_fence_after();
    begin_in_row();
    const uint32_t acc = acc_at;

    if (warp == 0 && lane == 0) {                     // copies: each CTA its own operands, a pair's bytes counted by its first CTA
        int s = 0, round = 0, issued = 0;
        bool ok = true;
        for (int tile = worker; ok && tile < tiles; tile += workers) {
            int mt, nt;
            tile_place(tile, m_tiles, n_tiles, &mt, &nt);
            const int m0 = (mt * kCtas + rank) * kTileM, n0 = nt * kN + rank * T::kBRows;
            for (int i = 0; i < steps; ++i) {
                if (!(ok = bar_wait(empty(s), (round & 1) ^ 1))) break;
                if (rank == 0) bar_expect(full(s), (g.a_rows * kRowBytes + T::kBBytes) * kCtas);
                const uint32_t bar = kCtas == 2 ? at_rank(full(s), 0) : full(s);
                const int pass = (i >= g.k_tiles) + (i >= 2 * g.k_tiles), k = (i - pass * g.k_tiles) * kTileK;
                const uint32_t a = ring + s * T::kStage, b = a + T::kABytes;
                if (g.a_mn) {
#pragma unroll
                    for (int c = 0; c < kTileM / 64; ++c) copy_tile<kCtas>(a + c * 64 * kRowBytes, &maps.a[pass], m0 + c * 64, k, bar);
                } else {
                    copy_tile<kCtas>(a, &maps.a[pass], k, m0, bar);
                }
                if (g.b_mn) {
#pragma unroll
                    for (int c = 0; c < T::kBRows / 64; ++c) copy_tile<kCtas>(b + c * 64 * kRowBytes, &maps.b[pass], n0 + c * 64, k, bar);
                } else {
                    copy_tile<kCtas>(b, &maps.b[pass], k, n0, bar);
                }
                ++issued;
                if (++s == kS) { s = 0; ++round; }
            }
        }
        if (!ok) {
            failed = 1;
            // this CTA's copies have to have landed before its shared memory goes: the j-th last one was fill (issued - 1 - j) of the ring
            if (rank == 0)
                for (int j = 0; j < min(issued, kS); ++j) bar_wait(full((issued - 1 - j) % kS), ((issued - 1 - j) / kS) & 1);
        }
    } else if (warp == 1 && lane == 0 && rank == 0) { // products
        const uint32_t desc = product_desc(kTileM * kCtas, kN, g.a_mn, g.b_mn);
        const uint32_t a_step = g.a_mn ? 16 * kRowBytes : 32, b_step = g.b_mn ? 16 * kRowBytes : 32;    // bytes per 16 k
        int s = 0, round = 0, count = 0;
        bool ok = true;
        for (int tile = worker; ok && tile < tiles; tile += workers) {
            for (int first = 0; ok && first < steps; first += chunk, ++count) {
                const int half = count & 1, last = min(steps, first + chunk);
                if (!(ok = bar_wait(acc_empty(half), ((count >> 1) & 1) ^ 1))) break;
                acc_fence_after();
                const uint32_t d = acc + half * kN;
                for (int i = first; i < last; ++i) {
                    if (!(ok = bar_wait(full(s), round & 1))) break;
                    acc_fence_after();
                    const uint32_t a = ring + s * T::kStage, b = a + T::kABytes;
#pragma unroll
                    for (int k = 0; k < kTileK / 16; ++k)
                        product<kCtas>(d, operand_desc(a + k * a_step, 64 * kRowBytes), operand_desc(b + k * b_step, 64 * kRowBytes), desc, i > first || k > 0);
                    product_commit<kCtas>(empty(s));
                    if (++s == kS) { s = 0; ++round; }
                }
                product_commit<kCtas>(acc_full(half));
            }
        }
        if (!ok) {                                    // (products in flight read shared and write tensor memory)
            failed = 1;
            product_commit<kCtas>(drained);
            bar_wait(drained, 0);
        }
    } else if (warp >= 4) {                           // write out
        const int quarter = warp & 3, side = (warp - 4) >> 2;       // a warp reads its quarter of the lanes alone
        constexpr int kCols = kN / 2;
        Writer writer{g, maps, outs + (warp - 4) * 2 * T::kOutBytes, T::kOutBytes, lane};
        int count = 0;
        bool ok = true;
        for (int tile = worker; ok && tile < tiles; tile += workers) {
            int mt, nt;
            tile_place(tile, m_tiles, n_tiles, &mt, &nt);
            const int64_t row0 = (int64_t(mt) * kCtas + rank) * kTileM + quarter * 32;
            const int col0 = nt * kN + side * kCols;
            float total[kChunked ? kCols / 32 : 1][32];
            for (int c = 0; c < chunks; ++c, ++count) {
                const int half = count & 1;
                if (!(ok = bar_wait(acc_full(half), (count >> 1) & 1))) break;
                acc_fence_after();
                const uint32_t at = acc + half * kN + (uint32_t(quarter * 32) << 16) + side * kCols;
                if constexpr (kChunked) {
#pragma unroll
                    for (int p = 0; p < kCols / 32; ++p) {
                        float v[32];
                        acc_load(at + p * 32, v);
#pragma unroll
                        for (int i = 0; i < 32; ++i) total[p][i] = c == 0 ? v[i] : total[p][i] + v[i];
                    }
                } else {
                    for (int p = 0; p < kCols && col0 + p < g.n && row0 < g.m; p += 32) {      // (alike in the warp)
                        acc_load(at + p, total[0]);
                        writer.write(row0, col0 + p, total[0]);
                    }
                }
                acc_fence_before();
                __syncwarp();
                if (lane == 0) {
                    if constexpr (kCtas == 2) bar_arrive_at(acc_empty(half), 0);
                    else bar_arrive(acc_empty(half));
                }
            }
            if constexpr (kChunked) {
                if (ok && row0 < g.m) {
#pragma unroll
                    for (int p = 0; p < kCols / 32; ++p)
                        if (col0 + p * 32 < g.n) writer.write(row0, col0 + p * 32, total[p]);
                }
            }
        }
        if (!ok) failed = 1;
        if (lane == 0) stores_read<0>();
    }
    __syncwarp();
    acc_fence_before();
    if constexpr (kCtas == 2) cluster_barrier();      // (the first CTA's products read the second one's shared memory)
    else __syncthreads();
    if (warp == 2) {
        acc_fence_after();
        acc_free<kCtas>(acc, T::kColumns);
    }
    if (threadIdx.x == 0 && failed) atomicAdd(&g_gave_up, 1u);
}

// ---- few tiles: the sum over k is split --------------------------------------------------------------------------------
// A cluster of CTAs shares one tile of 128 x 64, each a run of the steps over k; their sums meet in shared memory, where every
// CTA reads its part of the tile from all of them, adds in order of rank and writes it out.  One tile of few rows is bound by the
// reading of B: two CTAs per SM keep 64 KB of it in flight.
constexpr int kSplitN = 64, kSplitStages = 4, kSplitWriters = 4, kSplitMost = 8;
constexpr int kSplitThreads = 128 + 32 * kSplitWriters;
constexpr int kSplitStage = (kTileM + kSplitN) * kRowBytes, kSplitSmem = kSplitStages * kSplitStage + 1024;

__device__ __forceinline__ float4 load_at_rank(uint32_t addr, uint32_t rank) {
    float4 v;
    asm volatile("ld.shared::cluster.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(at_rank(addr, rank)) : "memory");
    return v;
}
// where 16 bytes (4 sums) of the tile lie: rows of 256 bytes, spread over the banks
__device__ __forceinline__ uint32_t sum_place(int row, int four) { return uint32_t(row * 256 + ((four ^ (row & 15)) << 4)); }

__global__ void __launch_bounds__(kSplitThreads, 2) product_split_kernel(const __grid_constant__ Maps maps, const ProductArgs g, int parts) {
    constexpr int kS = kSplitStages;
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
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, rank = int(cluster_rank()), tile = int(blockIdx.x) / parts;
    const int n_tiles = (g.n + kSplitN - 1) / kSplitN, mt = tile / n_tiles, nt = tile - mt * n_tiles;
    const int total_steps = g.k_tiles * g.passes, from = int(int64_t(total_steps) * rank / parts), to = int(int64_t(total_steps) * (rank + 1) / parts);
    if (threadIdx.x == 0) {
        for (int s = 0; s < kS; ++s) { bar_init(full(s), 1); bar_init(empty(s), 1); }
        for (int a = 0; a < 2; ++a) { bar_init(acc_full(a), 1); bar_init(acc_empty(a), kSplitWriters); }
        bar_init(drained, 1);
        failed = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        shared_to_async();
    }
    if (warp == 2) acc_alloc<1>(smem_addr(&acc_at), 2 * kSplitN);
    acc_fence_before();
    __syncthreads();
    acc_fence_after();
    begin_in_row();
    const uint32_t acc = acc_at;
    if (warp == 0 && lane == 0) {
        bool ok = true;
        int issued = 0;
        for (int i = from; i < to; ++i, ++issued) {
            const int s = issued % kS;
            if (!(ok = bar_wait(empty(s), (issued / kS & 1) ^ 1))) break;
            bar_expect(full(s), (g.a_rows + kSplitN) * kRowBytes);
            const int pass = (i >= g.k_tiles) + (i >= 2 * g.k_tiles), k = (i - pass * g.k_tiles) * kTileK;
            const uint32_t a = ring + s * kSplitStage, b = a + kTileM * kRowBytes;
            if (g.a_mn) {
#pragma unroll
                for (int c = 0; c < kTileM / 64; ++c) copy_tile<1>(a + c * 64 * kRowBytes, &maps.a[pass], mt * kTileM + c * 64, k, full(s));
            } else {
                copy_tile<1>(a, &maps.a[pass], k, mt * kTileM, full(s));
            }
            if (g.b_mn) copy_tile<1>(b, &maps.b[pass], nt * kSplitN, k, full(s));
            else copy_tile<1>(b, &maps.b[pass], k, nt * kSplitN, full(s));
        }
        if (!ok) {
            failed = 1;
            for (int j = 0; j < min(issued, kS); ++j) bar_wait(full((issued - 1 - j) % kS), ((issued - 1 - j) / kS) & 1);
        }
    } else if (warp == 1 && lane == 0) {
        const uint32_t desc = product_desc(kTileM, kSplitN, g.a_mn, g.b_mn);
        const uint32_t a_step = g.a_mn ? 16 * kRowBytes : 32, b_step = g.b_mn ? 16 * kRowBytes : 32;
        bool ok = true;
        for (int i = 0; ok && i < to - from; ++i) {
            const int s = i % kS, half = (i / kChunk) & 1;
            if (i % kChunk == 0) {
                if (!(ok = bar_wait(acc_empty(half), (i / kChunk >> 1 & 1) ^ 1))) break;
                acc_fence_after();
            }
            if (!(ok = bar_wait(full(s), i / kS & 1))) break;
            acc_fence_after();
            const uint32_t a = ring + s * kSplitStage, b = a + kTileM * kRowBytes;
#pragma unroll
            for (int k = 0; k < kTileK / 16; ++k)
                product<1>(acc + half * kSplitN, operand_desc(a + k * a_step, 64 * kRowBytes), operand_desc(b + k * b_step, 64 * kRowBytes), desc, i % kChunk > 0 || k > 0);
            product_commit<1>(empty(s));
            if (i % kChunk == kChunk - 1 || i == to - from - 1) product_commit<1>(acc_full(half));
        }
        if (!ok) {
            failed = 1;
            product_commit<1>(drained);
            bar_wait(drained, 0);
        }
    } else if (warp >= 4) {
        const int quarter = warp & 3, row = quarter * 32 + lane;
        float total[2][32];
        bool ok = true;
        for (int c = 0; c * kChunk < to - from; ++c) {
            if (!(ok = bar_wait(acc_full(c & 1), c >> 1 & 1))) break;
            acc_fence_after();
#pragma unroll
            for (int p = 0; p < 2; ++p) {
                float v[32];
                acc_load(acc + (c & 1) * kSplitN + (uint32_t(quarter * 32) << 16) + p * 32, v);
#pragma unroll
                for (int i = 0; i < 32; ++i) total[p][i] = c == 0 ? v[i] : total[p][i] + v[i];
            }
            acc_fence_before();
            __syncwarp();
            if (lane == 0) bar_arrive(acc_empty(c & 1));
        }
        if (!ok) failed = 1;
        // (the last product is done: the ring's stages are free)
        if (mt * kTileM + row < g.m)
#pragma unroll
            for (int f = 0; f < 16; ++f)
                asm volatile("st.shared.v4.f32 [%0], {%1,%2,%3,%4};" ::"r"(ring + sum_place(row, f)), "f"(total[f / 8][f % 8 * 4]), "f"(total[f / 8][f % 8 * 4 + 1]),
                             "f"(total[f / 8][f % 8 * 4 + 2]), "f"(total[f / 8][f % 8 * 4 + 3]) : "memory");
    }
    __syncwarp();
    acc_fence_before();
    cluster_barrier();
    if (warp == 2) {
        acc_fence_after();
        acc_free<1>(acc, 2 * kSplitN);
    }
    const int rows = min(kTileM, g.m - mt * kTileM);
    for (int i = rank * kSplitThreads + int(threadIdx.x); i < rows * 16; i += parts * kSplitThreads) {
        const int r = i >> 4, f = i & 15, col = nt * kSplitN + f * 4;
        if (col >= g.n) continue;
        float v[4] = {0.f, 0.f, 0.f, 0.f};
        float4 p[kSplitMost];
#pragma unroll
        for (int q = 0; q < kSplitMost; ++q)
            if (q < parts) p[q] = load_at_rank(ring + sum_place(r, f), q);
#pragma unroll
        for (int q = 0; q < kSplitMost; ++q)
            if (q < parts) { v[0] += p[q].x; v[1] += p[q].y; v[2] += p[q].z; v[3] += p[q].w; }
        const int64_t row = int64_t(mt) * kTileM + r;
        const int left = min(4, g.n - col);
        if (g.bias)
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] += j < left ? __ldg(g.bias + col + j) : 0.f;
        if (g.pre) store4(g.pre + row * g.pre_step, col, left, 0, g.pre_wide, v);
        apply_act(v, g.act);
        if (g.residual)
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (j < left) {
                    const char* at = g.residual + row * g.residual_step;
                    v[j] += g.out_f32 ? reinterpret_cast<const float*>(at)[col + j] : bf16_bits_to_float(reinterpret_cast<const uint16_t*>(at)[col + j]);
                }
        store4(g.out + row * g.out_step, col, left, g.out_f32, g.out_wide, v);
    }
    __syncwarp();
    cluster_barrier();                                // (its sums have been read)
    if (threadIdx.x == 0 && failed) atomicAdd(&g_gave_up, 1u);
}

// ---- what goes in front of the products ---------------------------------------------------------------------------
// Rows copied to where a tiled copy can read them: base and row stride multiples of 16 bytes.
struct Repack { const char* from; char* to; int64_t from_step, to_step, rows; int cols; };
struct Repacks { Repack r[3]; int64_t ends[3]; int n; };       // ends: running counts of 8-column pieces

__global__ void __launch_bounds__(kThreads) repack_kernel(const Repacks g) {
    begin_in_row();
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
constexpr int kSlopeRows = 4;        // rows a warp has in flight
struct SlopeArgs {
    const char *dout, *pre;
    char *dz, *dz_mid, *dz_low;      // null: not wanted
    float* part;                     // [part][n]; null: no column sums
    int64_t dout_step, pre_step, dz_step, rows, rows_per_part;
    int n;
};

template <bool kWide>
__device__ __forceinline__ void load8(const char* row, int col, int n, float (&x)[8]) {
    if constexpr (kWide) {
        unpack8(ld_stream_u4(row + 2 * int64_t(col)), x);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = col + j < n ? bf16_bits_to_float(reinterpret_cast<const uint16_t*>(row)[col + j]) : 0.f;
    }
}

// kWide: n is a multiple of 8, and the rows of dout and pre start on 16-byte boundaries.
template <int kAct, bool kWide>
__global__ void __launch_bounds__(kThreads) slope_kernel(const SlopeArgs g) {
    constexpr bool kPre = kAct != BAOC_ACT_NONE;
    __shared__ float sh[8][256];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, col = int(blockIdx.x) * 256 + lane * 8;
    const int64_t first = int64_t(blockIdx.y) * g.rows_per_part, end = min64(g.rows, first + g.rows_per_part);
    float sum[8] = {};
    begin_in_row();
    auto one_row = [&](int64_t row, float (&d)[8], const float (&z)[8]) {
        if constexpr (kPre) {
#pragma unroll
            for (int j = 0; j < 8; ++j) d[j] *= act_slope<kAct>(z[j]);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) sum[j] += d[j];
        if (!g.dz) return;
        const uint4 w = make_uint4(pair_bf16(d[0], d[1]), pair_bf16(d[2], d[3]), pair_bf16(d[4], d[5]), pair_bf16(d[6], d[7]));
        const int64_t at = row * g.dz_step + 2 * int64_t(col);
        *reinterpret_cast<uint4*>(g.dz + at) = w;
        if (!kPre || !g.dz_mid) return;
        float h[8];
        unpack8(w, h);
#pragma unroll
        for (int j = 0; j < 8; ++j) d[j] -= h[j];
        const uint4 m = make_uint4(pair_bf16(d[0], d[1]), pair_bf16(d[2], d[3]), pair_bf16(d[4], d[5]), pair_bf16(d[6], d[7]));
        *reinterpret_cast<uint4*>(g.dz_mid + at) = m;
        unpack8(m, h);
#pragma unroll
        for (int j = 0; j < 8; ++j) d[j] -= h[j];
        *reinterpret_cast<uint4*>(g.dz_low + at) = make_uint4(pair_bf16(d[0], d[1]), pair_bf16(d[2], d[3]), pair_bf16(d[4], d[5]), pair_bf16(d[6], d[7]));
    };
    if (col < g.n)
        for (int64_t row = first + warp; row < end; row += 8 * kSlopeRows) {
            float d[kSlopeRows][8], z[kPre ? kSlopeRows : 1][8];
#pragma unroll
            for (int r = 0; r < kSlopeRows; ++r) {
                const int64_t at = min64(row + 8 * r, end - 1);          // (a row too many is read, not used)
                load8<kWide>(g.dout + at * g.dout_step, col, g.n, d[r]);
                if constexpr (kPre) load8<kWide>(g.pre + at * g.pre_step, col, g.n, z[r]);
            }
#pragma unroll
            for (int r = 0; r < kSlopeRows; ++r)
                if (row + 8 * r < end) one_row(row + 8 * r, d[r], z[kPre ? r : 0]);
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
    begin_in_row();
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

// Boxes of box_cols contiguous elements (64 or 128 bytes, laid out with the swizzle of that width) by box_rows rows; zeros outside.
bool encode(CUtensorMap* map, const Matrix& t, int box_rows, int box_cols = 64) {
    EncodeFn f = encode_fn();
    if (!f) return false;
    const cuuint64_t dims[2] = {cuuint64_t(t.cols), cuuint64_t(t.rows)}, strides[1] = {cuuint64_t(t.step)};
    const cuuint32_t box[2] = {cuuint32_t(box_cols), cuuint32_t(box_rows)}, unit[2] = {1, 1};
    return f(map, t.eb == 4 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<char*>(t.p), dims, strides, box, unit,
             CU_TENSOR_MAP_INTERLEAVE_NONE, box_cols * t.eb == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
             CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// A product's operands: a as [m][k] or, a_mn, as [k][m]; b as [n][k] or [k][n]; up to three pairs whose products are added.
struct Operands { const Matrix *a[3], *b[3]; };

template <int kCtas, int kN, bool kChunked>
int launch_product(const Operands& o, const Matrix& out, const Matrix& pre, const ProductArgs& g, cudaStream_t s) {
    using T = TileShape<kCtas, kN, kChunked>;
    static_assert(T::kStages >= 4 && T::kSmem <= 227 * 1024 - 512, "the ring, the outputs and the barriers share 227 KB");
    auto kernel = product_kernel<kCtas, kN, kChunked>;
    static std::atomic<uint64_t> allowed{0};         // the permission for large shared memory is per device and lasts
    int dev = 0;
    cudaError_t ce = cudaGetDevice(&dev);
    if (ce != cudaSuccess) return launched(ce, "product_kernel");
    const uint64_t bit = dev < 64 ? uint64_t(1) << dev : 0;
    if (!(allowed.load(std::memory_order_relaxed) & bit)) {
        ce = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, T::kSmem);
        if (ce != cudaSuccess) return launched(ce, "product_kernel");
        allowed.fetch_or(bit, std::memory_order_relaxed);
    }
    Maps maps;
    bool ok = true;
    for (int i = 0; i < g.passes; ++i) ok = ok && encode(&maps.a[i], *o.a[i], g.a_mn ? kTileK : g.a_rows) && encode(&maps.b[i], *o.b[i], g.b_mn ? kTileK : T::kBRows);
    if (g.out_wide) ok = ok && encode(&maps.out, out, 32, 32);
    if (g.pre && g.pre_wide) ok = ok && encode(&maps.pre, pre, 32, 32);
    if (!ok) return fail_linear(BAOC_E_CUDA, "the driver refused a tensor map");
    const int64_t tiles = ceil_div(g.m, kTileM * kCtas) * ceil_div(g.n, kN);
    if (tiles > 0x7fffffff - 148) return fail_linear(BAOC_E_INVALID, "too many tiles for one launch");
    return launched(launch_in_row(kernel, dim3(unsigned(std::min<int64_t>(tiles, 148 / kCtas) * kCtas)), kProductThreads, T::kSmem, kCtas, s, maps, g), "product_kernel");
}

int launch_split(const Operands& o, const ProductArgs& g, int64_t tiles, int parts, cudaStream_t s) {
    static std::atomic<uint64_t> allowed{0};
    int dev = 0;
    cudaError_t ce = cudaGetDevice(&dev);
    if (ce != cudaSuccess) return launched(ce, "product_split_kernel");
    const uint64_t bit = dev < 64 ? uint64_t(1) << dev : 0;
    if (!(allowed.load(std::memory_order_relaxed) & bit)) {
        ce = cudaFuncSetAttribute(product_split_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSplitSmem);
        if (ce != cudaSuccess) return launched(ce, "product_split_kernel");
        allowed.fetch_or(bit, std::memory_order_relaxed);
    }
    Maps maps;
    for (int i = 0; i < g.passes; ++i)
        if (!encode(&maps.a[i], *o.a[i], g.a_mn ? kTileK : g.a_rows) || !encode(&maps.b[i], *o.b[i], g.b_mn ? kTileK : kSplitN))
            return fail_linear(BAOC_E_CUDA, "the driver refused a tensor map");
    return launched(launch_in_row(product_split_kernel, dim3(unsigned(tiles * parts)), kSplitThreads, kSplitSmem, unsigned(parts), s, maps, g, parts), "product_split_kernel");
}

// The largest tiles that still give every CTA one; where the smallest do not, the sum over k is split among two CTAs per SM, at
// least four steps each.  g has its sizes and flags, out and pre are where it goes.
int form_product(const Operands& o, const Matrix& out, const Matrix& pre, ProductArgs g, cudaStream_t s) {
    g.out = const_cast<char*>(out.p); g.out_step = out.step; g.out_f32 = out.eb == 4; g.out_wide = out.wide();
    g.pre = const_cast<char*>(pre.p); g.pre_step = pre.step; g.pre_wide = pre.wide();
    g.a_rows = g.a_mn ? kTileM : std::min(kTileM, int(round_up(g.m, 8)));
    const int64_t pairs = ceil_div(g.m, 2 * kTileM), ones = ceil_div(g.m, kTileM), smallest = ones * ceil_div(g.n, kSplitN);
    int parts = 1;
    while (parts < kSplitMost && smallest * parts * 2 <= 2 * 148 && int64_t(g.k_tiles) * g.passes >= 8 * parts) parts *= 2;
    if (parts > 1) return launch_split(o, g, smallest, parts, s);
    if (g.out_f32) {
        if (pairs * ceil_div(g.n, 128) >= 74) return launch_product<2, 128, true>(o, out, pre, g, s);
        return launch_product<1, 64, true>(o, out, pre, g, s);
    }
    if (pairs * ceil_div(g.n, 256) >= 74) return launch_product<2, 256, false>(o, out, pre, g, s);
    if (ones * ceil_div(g.n, 128) >= 148) return launch_product<1, 128, false>(o, out, pre, g, s);
    return launch_product<1, 64, false>(o, out, pre, g, s);
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
        return launched(launch_in_row(repack_kernel, dim3(grid), kThreads, 0, 1, s, todo), "repack_kernel");
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
    g.act = e->act; g.bias = bias;
    g.residual = mr.p; g.residual_step = mr.step; g.residual_wide = mr.wide();
    return form_product(Operands{{&a}, {&b}}, mo, mp, g, s);
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
        g.rows = tokens; g.n = e->n_out;
        const dim3 grid(unsigned(ceil_div(e->n_out, 256)), unsigned(parts));
        const bool wide = e->n_out % 8 == 0 && md.wide() && (!act || mp.wide());
        auto go = [&](auto a) {
            return launched(launch_in_row(wide ? slope_kernel<decltype(a)::value, true> : slope_kernel<decltype(a)::value, false>, grid, kThreads, 0, 1, s, g), "slope_kernel");
        };
        using std::integral_constant;
        switch (e->act) {
            case BAOC_ACT_RELU: rc = go(integral_constant<int, BAOC_ACT_RELU>{}); break;
            case BAOC_ACT_GELU: rc = go(integral_constant<int, BAOC_ACT_GELU>{}); break;
            case BAOC_ACT_GELU_TANH: rc = go(integral_constant<int, BAOC_ACT_GELU_TANH>{}); break;
            case BAOC_ACT_SILU: rc = go(integral_constant<int, BAOC_ACT_SILU>{}); break;
            default: rc = go(integral_constant<int, BAOC_ACT_NONE>{}); break;
        }
        if (rc) return rc;
        if (g.part && (rc = launched(launch_in_row(slope_sums_kernel, dim3(unsigned(ceil_div(e->n_out, 32))), 1024, 0, 1, s, static_cast<const float*>(g.part), int(parts),
                                                   int(e->n_out), static_cast<char*>(db), int(e->grad_dtype == BAOC_F32)), "slope_sums_kernel")))
            return rc;
    }
    const Matrix none(nullptr, 0, 0, 0, BAOC_BF16);
    if (dx) {
        ProductArgs p{};
        p.m = int(tokens); p.n = e->n_in; p.k_tiles = int(ceil_div(e->n_out, kTileK)); p.passes = 1;
        p.b_mn = out_in;
        if ((rc = form_product(Operands{{&dz}, {&bw}}, mdx, none, p, s))) return rc;
    }
    if (dw) {
        ProductArgs p{};
        p.m = int(w_rows); p.n = int(w_cols); p.k_tiles = int(ceil_div(tokens, kTileK)); p.passes = split ? 3 : 1;
        p.a_mn = p.b_mn = 1;
        const Operands o = out_in ? Operands{{&dz, &mid, &low}, {&bx, &bx, &bx}} : Operands{{&bx, &bx, &bx}, {&dz, &mid, &low}};
        if ((rc = form_product(o, mdw, none, p, s))) return rc;
    }
    return BAOC_OK;
} catch (const std::bad_alloc&) {
    return BAOC_E_INVALID;
}

}  // extern "C"
