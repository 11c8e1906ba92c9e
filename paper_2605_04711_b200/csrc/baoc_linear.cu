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
#include <utility>

#include "baoc_check.cuh"
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
constexpr int kLongSum = 1024;                       // steps: positive sums of 65536 products are off by 3e-4, a tenth of half a bf16 step

// kCtas CTAs (a pair shares the tensor cores' work on a tile of 256 rows: each holds its 128 rows of A, half the columns' rows
// of B, and its rows' accumulators, so that a stage of both feeds twice the products of one CTA's).
// kChunked, for fp32 outputs and for sums over more than kLongSum steps: the tensor cores cut an accumulator's low bits off at
// every addition (2^-25 of it on average, always towards zero; at k = 8192 random products the result is off by 9e-6, at 16384
// positive ones by 8e-5), so every kChunk steps the sums so far are added up in registers, rounded to nearest, and the accumulator
// starts again (5e-7).
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
    int m_tiles, n_tiles;
    int a_mn, b_mn;                  // the operand's m (n) lies contiguous, not its k
    int a_rows;                      // rows of A that a copy brings: fewer than a tile's where m is smaller
    int act, out_f32;
    char *out, *pre;
    const char* residual;
    const float* bias;
    int64_t out_step, pre_step, residual_step;      // bytes
    int out_wide, pre_wide, residual_wide;           // 16-byte accesses fit; kTiled (out, pre): tiled copies store it
};

constexpr int kTiled = 2;

struct Maps { CUtensorMap a[3], b[3], out, pre; };

// One or two products of one launch (two where a gradient's both are formed: the second's tiles fill the places that the first's
// last round leaves empty).
struct Problem {
    Maps maps;
    ProductArgs g;
};
struct Problems {
    Problem p[2];
    int tiles[2];
    int fewer;                       // tiles of the second that the workers take which have one more of the first's (see Walk)
};
static_assert(sizeof(Problems) <= 4096, "a kernel's parameters");

__device__ __forceinline__ float exp2_approx(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
constexpr float kLog2e = 1.4426950408889634f;

// The normal distribution below -|z|, as e^(-z^2/2) times a polynomial in t = 1 / (1 + 0.35 |z|): erfc(x) e^(x^2) is smooth in
// such a t.  The coefficients are a least-maximum fit of the relative error over |z| <= 15 (3.2e-8 in exact arithmetic, 5 2^-24
// with the coefficients and every step in fp32); two approximate functions against some forty instructions of erfcf.  Two at a
// time.  Returns it and, in *density, e^(-z^2/2).
__device__ __forceinline__ f32x2 exp2_pair(f32x2 x) {
    float a, b;
    unpack2(x, a, b);
    return pack2(exp2_approx(a), exp2_approx(b));
}
__device__ __forceinline__ f32x2 rcp_pair(f32x2 x) {
    float a, b;
    unpack2(x, a, b);
    return pack2(rcp_approx(a), rcp_approx(b));
}
__device__ __forceinline__ f32x2 lower_tail(f32x2 z, f32x2* density) {
    float a, b;
    unpack2(z, a, b);
    const f32x2 t = rcp_pair(fma2(splat2(0.35f), pack2(fabsf(a), fabsf(b)), splat2(1.f)));
    f32x2 p = splat2(-0.02916380763053894f);
    p = fma2(p, t, splat2(0.14406023919582367f));
    p = fma2(p, t, splat2(-0.2559007406234741f));
    p = fma2(p, t, splat2(0.15939167141914368f));
    p = fma2(p, t, splat2(-0.02326301671564579f));
    p = fma2(p, t, splat2(0.10557447373867035f));
    p = fma2(p, t, splat2(0.11981557309627533f));
    p = fma2(p, t, splat2(0.13986432552337646f));
    p = fma2(p, t, splat2(0.13962125778198242f));
    *density = exp2_pair(mul2(splat2(-0.5f * kLog2e), mul2(z, z)));
    return mul2(mul2(p, t), *density);
}
// the normal distribution below z from its tail below -|z|
__device__ __forceinline__ f32x2 below(f32x2 z, f32x2 tail) {
    float a, b, s, t;
    unpack2(z, a, b);
    unpack2(tail, s, t);
    return pack2(a > 0.f ? 1.f - s : s, b > 0.f ? 1.f - t : t);
}
__device__ __forceinline__ f32x2 sigmoid(f32x2 z) { return rcp_pair(add2(splat2(1.f), exp2_pair(mul2(splat2(-kLog2e), z)))); }
// the exponent of gelu's tanh form, 2 sqrt(2 / pi) (z + 0.044715 z^3)
__device__ __forceinline__ f32x2 tanh_form(f32x2 z) { return mul2(splat2(1.5957691216057308f), fma2(mul2(mul2(splat2(0.044715f), z), z), z, z)); }

template <int kAct>
__device__ __forceinline__ f32x2 act_of(f32x2 z) {
    if constexpr (kAct == BAOC_ACT_RELU) {
        float a, b;
        unpack2(z, a, b);
        return pack2(a > 0.f || a != a ? a : 0.f, b > 0.f || b != b ? b : 0.f);
    }
    if constexpr (kAct == BAOC_ACT_GELU) {
        f32x2 d;
        return mul2(z, below(z, lower_tail(z, &d)));
    }
    if constexpr (kAct == BAOC_ACT_GELU_TANH) return mul2(z, sigmoid(tanh_form(z)));
    if constexpr (kAct == BAOC_ACT_SILU) return mul2(z, sigmoid(z));
    return z;
}
template <int kAct>
__device__ __forceinline__ void act_all(float* v, int n) {
#pragma unroll
    for (int i = 0; i < n; i += 2) unpack2(act_of<kAct>(pack2(v[i], v[i + 1])), v[i], v[i + 1]);
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
__device__ __forceinline__ f32x2 act_slope(f32x2 z) {
    float a, b;
    unpack2(z, a, b);
    if constexpr (kAct == BAOC_ACT_RELU) {
        auto one = [](float x) { return x > 0.f ? 1.f : (x != x ? x : 0.f); };
        return pack2(one(a), one(b));
    }
    constexpr float kEnd = kAct == BAOC_ACT_SILU ? 90.f : 15.f;
    auto clamp = [](float x) { return x != x ? x : fminf(fmaxf(x, -kEnd), kEnd); };
    const f32x2 y = pack2(clamp(a), clamp(b));
    if constexpr (kAct == BAOC_ACT_GELU) {
        f32x2 d;
        const f32x2 p = below(y, lower_tail(y, &d));
        return fma2(mul2(splat2(0.3989422804014327f), y), d, p);
    }
    if constexpr (kAct == BAOC_ACT_GELU_TANH) {
        const f32x2 s = sigmoid(tanh_form(y)), rest = fma2(mul2(splat2(-1.f), s), s, s);      // s (1 - s)
        return fma2(mul2(y, rest), mul2(splat2(1.5957691216057308f), fma2(mul2(splat2(0.134145f), y), y, splat2(1.f))), s);
    }
    if constexpr (kAct == BAOC_ACT_SILU) {
        const f32x2 s = sigmoid(y);
        return mul2(s, fma2(y, add2(splat2(1.f), mul2(splat2(-1.f), s)), splat2(1.f)));
    }
    return splat2(1.f);
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

// The tiles of a worker, in the order that all of its roles go through them: the first product's every workers-th, then the
// second's.  Workers that the first left with a tile more take `fewer` of the second's, the others go on until all are taken.
struct Walk {
    int worker, workers, longer, fewer, problem = 0, i = -1;
    __device__ __forceinline__ Walk(const Problems& all, int worker, int workers)
        : worker(worker), workers(workers), longer(all.tiles[0] % workers), fewer(all.fewer) {}
    __device__ __forceinline__ bool next(const Problems& all, int* tile) {
        ++i;
        if (problem == 0) {
            *tile = worker + i * workers;
            if (*tile < all.tiles[0]) return true;
            problem = 1;
            i = 0;
        }
        if (i < fewer) *tile = i * workers + worker;
        else if (worker >= longer) *tile = fewer * workers + (i - fewer) * (workers - longer) + worker - longer;
        else return false;
        return *tile < all.tiles[1];
    }
};

// What a writing warp does with 32 columns of its 32 rows.
struct Writer {
    const ProductArgs& g;
    const Maps& maps;
    uint32_t buf;                    // two buffers of `bytes`
    uint32_t bytes;
    int lane, turn;

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
    // Arrays that no tiled copy fits (rows off the 16-byte grid): the warp's 32 x 32 values pass through both buffers, so that its
    // lanes go along the columns of a row outside and along the rows inside.
    __device__ __forceinline__ uint32_t cell(int row, int col) const { return buf + (row * 32 + (col ^ row)) * 4; }
    __device__ __forceinline__ void store_rows(char* to, int64_t step, int f32, int64_t row0, int col, int left, const float (&v)[32]) {
        if (lane == 0) stores_read<0>();
        __syncwarp();
#pragma unroll
        for (int c = 0; c < 32; ++c) asm volatile("st.shared.f32 [%0], %1;" ::"r"(cell(lane, c)), "f"(v[c]) : "memory");
        __syncwarp();
        const int rows = int(min64(32, g.m - row0));
        if (lane < left)
#pragma unroll 8
            for (int r = 0; r < 32; ++r) {
                if (r >= rows) break;
                float x;
                asm volatile("ld.shared.f32 %0, [%1];" : "=f"(x) : "r"(cell(r, lane)) : "memory");
                char* p = to + (row0 + r) * step;
                if (f32) reinterpret_cast<float*>(p)[col + lane] = x;
                else reinterpret_cast<uint16_t*>(p)[col + lane] = one_bf16(x);
            }
        __syncwarp();
    }
    __device__ __forceinline__ void add_rows(const char* from, int64_t step, int f32, int64_t row0, int col, int left, float (&v)[32]) {
        if (lane == 0) stores_read<0>();
        __syncwarp();
        const int rows = int(min64(32, g.m - row0));
#pragma unroll 8
        for (int r = 0; r < 32; ++r) {
            const char* p = from + (row0 + r) * step;
            float x = 0.f;
            if (r < rows && lane < left) x = f32 ? reinterpret_cast<const float*>(p)[col + lane] : bf16_bits_to_float(reinterpret_cast<const uint16_t*>(p)[col + lane]);
            asm volatile("st.shared.f32 [%0], %1;" ::"r"(cell(r, lane)), "f"(x) : "memory");
        }
        __syncwarp();
#pragma unroll
        for (int c = 0; c < 32; ++c) {
            float x;
            asm volatile("ld.shared.f32 %0, [%1];" : "=f"(x) : "r"(cell(lane, c)) : "memory");
            v[c] += x;
        }
        __syncwarp();
    }
    // a thread's row of a residual on the 16-byte grid, all 32 columns there
    __device__ __forceinline__ void add_wide(const char* p, int f32, float (&v)[32]) {
        if (f32) {
#pragma unroll
            for (int i = 0; i < 32; i += 4) {
                const float4 a = reinterpret_cast<const float4*>(p)[i / 4];
                v[i] += a.x; v[i + 1] += a.y; v[i + 2] += a.z; v[i + 3] += a.w;
            }
        } else {
#pragma unroll
            for (int i = 0; i < 32; i += 8) {
                float x[8];
                unpack8(reinterpret_cast<const uint4*>(p)[i / 8], x);
#pragma unroll
                for (int j = 0; j < 8; ++j) v[i + j] += x[j];
            }
        }
    }
    // row0: the warp's first row (below m); the whole warp calls it
    __device__ __forceinline__ void write(int64_t row0, int col, float (&v)[32]) {
        const int left = min(32, g.n - col);
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
            if (g.pre_wide == kTiled) send(&maps.pre, 0, col, int(row0), v);
            else store_rows(g.pre, g.pre_step, 0, row0, col, left, v);
        }
        apply_act(v, g.act);
        if (g.residual) {
            if (!g.residual_wide || left < 32) add_rows(g.residual, g.residual_step, g.out_f32, row0, col, left, v);
            else if (row0 + lane < g.m) add_wide(g.residual + (row0 + lane) * g.residual_step + int64_t(col) * (g.out_f32 ? 4 : 2), g.out_f32, v);
            __syncwarp();
        }
        if (g.out_wide == kTiled) send(&maps.out, g.out_f32, col, int(row0), v);
        else store_rows(g.out, g.out_step, g.out_f32, row0, col, left, v);
        __syncwarp();
    }
};

template <int kCtas, int kN, bool kChunked>
__global__ void __launch_bounds__(kProductThreads, 1) product_kernel(const __grid_constant__ Problems all) {
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
    const int warp = uniform_warp(), lane = threadIdx.x & 31, rank = kCtas == 2 ? int(cluster_rank()) : 0;
    Walk walk(all, int(blockIdx.x) / kCtas, int(gridDim.x) / kCtas);
    int tile;
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

    if (warp == 0) {                                  // copies: each CTA its own operands, a pair's bytes counted by its first CTA
        const uint32_t first_full = kCtas == 2 ? at_rank(full(0), 0) : full(0);
        int s = 0, round = 0, issued = 0;
        bool ok = true;
        while (ok && walk.next(all, &tile)) {
            const ProductArgs& g = all.p[walk.problem].g;
            const Maps& maps = all.p[walk.problem].maps;
            int mt, nt;
            tile_place(tile, g.m_tiles, g.n_tiles, &mt, &nt);
            const int m0 = (mt * kCtas + rank) * kTileM, n0 = nt * kN + rank * T::kBRows, k_tiles = g.k_tiles, steps = k_tiles * g.passes, a_mn = g.a_mn, b_mn = g.b_mn;
            const uint32_t bytes = (g.a_rows * kRowBytes + T::kBBytes) * kCtas;
            for (int i = 0; i < steps; ++i) {
                if (!(ok = warp_wait(empty(s), (round & 1) ^ 1))) break;
                const uint32_t bar = first_full + 8 * s;
                const int pass = (i >= k_tiles) + (i >= 2 * k_tiles), k = (i - pass * k_tiles) * kTileK;
                const uint32_t a = ring + s * T::kStage, b = a + T::kABytes;
                if (elected()) {
                    if (rank == 0) bar_expect(full(s), bytes);
                    if (a_mn) {
#pragma unroll
                        for (int c = 0; c < kTileM / 64; ++c) copy_tile<kCtas>(a + c * 64 * kRowBytes, &maps.a[pass], m0 + c * 64, k, bar);
                    } else {
                        copy_tile<kCtas>(a, &maps.a[pass], k, m0, bar);
                    }
                    if (b_mn) {
#pragma unroll
                        for (int c = 0; c < T::kBRows / 64; ++c) copy_tile<kCtas>(b + c * 64 * kRowBytes, &maps.b[pass], n0 + c * 64, k, bar);
                    } else {
                        copy_tile<kCtas>(b, &maps.b[pass], k, n0, bar);
                    }
                }
                __syncwarp();
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
    } else if (warp == 1 && rank == 0) {              // products: what is computed for each is an addition to a descriptor
        const uint64_t first_a = operand_desc(ring, 64 * kRowBytes);
        int s = 0, round = 0, count = 0;
        bool ok = true;
        while (ok && walk.next(all, &tile)) {
            const ProductArgs& g = all.p[walk.problem].g;
            const uint32_t desc = product_desc(kTileM * kCtas, kN, g.a_mn, g.b_mn);
            const uint32_t a_step = (g.a_mn ? 16 * kRowBytes : 32) >> 4, b_step = (g.b_mn ? 16 * kRowBytes : 32) >> 4;    // per 16 k, in units of 16 bytes
            const int steps = g.k_tiles * g.passes, chunk = kChunked ? kChunk : steps;
            for (int first = 0; ok && first < steps; first += chunk, ++count) {
                const int half = count & 1, last = min(steps, first + chunk);
                if (!(ok = warp_wait(acc_empty(half), ((count >> 1) & 1) ^ 1))) break;
                acc_fence_after();
                const uint32_t d = acc + half * kN;
                for (int i = first; i < last; ++i) {
                    if (!(ok = warp_wait(full(s), round & 1))) break;
                    const uint64_t a = first_a + uint32_t(s) * (T::kStage >> 4), b = a + (T::kABytes >> 4);
                    if (elected()) {
                        product<kCtas>(d, a, b, desc, i > first);
#pragma unroll
                        for (uint32_t k = 1; k < kTileK / 16; ++k) product<kCtas>(d, a + k * a_step, b + k * b_step, desc, 1);
                        product_commit<kCtas>(empty(s));
                        if (i == last - 1) product_commit<kCtas>(acc_full(half));
                    }
                    __syncwarp();
                    if (++s == kS) { s = 0; ++round; }
                }
            }
        }
        if (!ok) {                                    // (products in flight read shared and write tensor memory)
            failed = 1;
            if (elected()) product_commit<kCtas>(drained);
            bar_wait(drained, 0);
        }
    } else if (warp >= 4) {                           // write out
        const int quarter = warp & 3, side = (warp - 4) >> 2;       // a warp reads its quarter of the lanes alone
        constexpr int kCols = kN / 2;
        int count = 0, turn = 0;
        bool ok = true;
        while (ok && walk.next(all, &tile)) {
            const ProductArgs& g = all.p[walk.problem].g;
            Writer writer{g, all.p[walk.problem].maps, outs + (warp - 4) * 2 * T::kOutBytes, T::kOutBytes, lane, turn};
            int mt, nt;
            tile_place(tile, g.m_tiles, g.n_tiles, &mt, &nt);
            const int64_t row0 = (int64_t(mt) * kCtas + rank) * kTileM + quarter * 32;
            const int col0 = nt * kN + side * kCols, chunks = kChunked ? (g.k_tiles * g.passes + kChunk - 1) / kChunk : 1;
            float total[kChunked ? kCols / 32 : 1][32];
            for (int c = 0; c < chunks; ++c, ++count) {
                const int half = count & 1;
                if (!(ok = warp_wait(acc_full(half), (count >> 1) & 1))) break;
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
            turn = writer.turn;
        }
        if (!ok) failed = 1;
        if (lane == 0) stores_done();
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
// A cluster of CTAs shares one tile of 128 x kN, each a run of the steps over k; their sums meet in shared memory, where every
// CTA reads its part of the tile from all of them, adds in order of rank and writes it out.  One tile of few rows is bound by the
// reading of B: two CTAs per SM, of 64 columns each, keep 64 KB of it in flight.  Sums over many rows (a narrow layer's dw) are bound by what
// L2 gives an SM: 256 columns, and one CTA per SM, need half the bytes a product.
constexpr int kSplitMost = 8;
template <int kN>
struct SplitShape {
    static constexpr int kStages = 4, kWriters = kN == 64 ? 4 : 8, kThreads = 128 + 32 * kWriters;
    static constexpr int kStage = (kTileM + kN) * kRowBytes, kSmem = kStages * kStage + 1024;
    static constexpr int kOwn = kN * 4 / kWriters, kPiece = kN == 64 ? 32 : 16;      // columns of a writing thread, and at a time
};

__device__ __forceinline__ float4 load_at_rank(uint32_t addr, uint32_t rank) {
    float4 v;
    asm volatile("ld.shared::cluster.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(at_rank(addr, rank)) : "memory");
    return v;
}
// where 16 bytes (4 sums) of the tile lie: a row's are spread over the banks
template <int kN>
__device__ __forceinline__ uint32_t sum_place(int row, int four) { return uint32_t(row * kN * 4 + ((four ^ (row & 15)) << 4)); }

template <int kN>
__global__ void __launch_bounds__(SplitShape<kN>::kThreads, kN == 64 ? 2 : 1) product_split_kernel(const __grid_constant__ Problems all, int parts) {
    using T = SplitShape<kN>;
    static_assert(kTileM * kN * 4 <= T::kStages * T::kStage, "the sums lie where the ring was");
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
    const int warp = uniform_warp(), lane = threadIdx.x & 31, rank = int(cluster_rank()), number = int(blockIdx.x) / parts;
    const int which = number >= all.tiles[0], tile = number - (which ? all.tiles[0] : 0);
    const ProductArgs& g = all.p[which].g;
    const Maps& maps = all.p[which].maps;
    const int n_tiles = g.n_tiles, mt = tile / n_tiles, nt = tile - mt * n_tiles;
    const int total_steps = g.k_tiles * g.passes, from = int(int64_t(total_steps) * rank / parts), to = int(int64_t(total_steps) * (rank + 1) / parts);
    if (threadIdx.x == 0) {
        for (int s = 0; s < kS; ++s) { bar_init(full(s), 1); bar_init(empty(s), 1); }
        for (int a = 0; a < 2; ++a) { bar_init(acc_full(a), 1); bar_init(acc_empty(a), T::kWriters); }
        bar_init(drained, 1);
        failed = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        shared_to_async();
    }
    if (warp == 2) acc_alloc<1>(smem_addr(&acc_at), 2 * kN);
    acc_fence_before();
    __syncthreads();
    acc_fence_after();
    begin_in_row();
    const uint32_t acc = acc_at;
    if (warp == 0) {
        bool ok = true;
        int issued = 0;
        for (int i = from; i < to; ++i, ++issued) {
            const int s = issued % kS;
            if (!(ok = warp_wait(empty(s), (issued / kS & 1) ^ 1))) break;
            const int pass = (i >= g.k_tiles) + (i >= 2 * g.k_tiles), k = (i - pass * g.k_tiles) * kTileK;
            const uint32_t a = ring + s * T::kStage, b = a + kTileM * kRowBytes;
            if (elected()) {
                bar_expect(full(s), (g.a_rows + kN) * kRowBytes);
                if (g.a_mn) {
#pragma unroll
                    for (int c = 0; c < kTileM / 64; ++c) copy_tile<1>(a + c * 64 * kRowBytes, &maps.a[pass], mt * kTileM + c * 64, k, full(s));
                } else {
                    copy_tile<1>(a, &maps.a[pass], k, mt * kTileM, full(s));
                }
                if (g.b_mn) {
#pragma unroll
                    for (int c = 0; c < kN / 64; ++c) copy_tile<1>(b + c * 64 * kRowBytes, &maps.b[pass], nt * kN + c * 64, k, full(s));
                } else {
                    copy_tile<1>(b, &maps.b[pass], k, nt * kN, full(s));
                }
            }
            __syncwarp();
        }
        if (!ok) {
            failed = 1;
            for (int j = 0; j < min(issued, kS); ++j) bar_wait(full((issued - 1 - j) % kS), ((issued - 1 - j) / kS) & 1);
        }
    } else if (warp == 1) {
        const uint32_t desc = product_desc(kTileM, kN, g.a_mn, g.b_mn);
        const uint32_t a_step = (g.a_mn ? 16 * kRowBytes : 32) >> 4, b_step = (g.b_mn ? 16 * kRowBytes : 32) >> 4;
        const uint64_t first_a = operand_desc(ring, 64 * kRowBytes);
        bool ok = true;
        for (int i = 0; ok && i < to - from; ++i) {
            const int s = i % kS, half = (i / kChunk) & 1;
            if (i % kChunk == 0) {
                if (!(ok = warp_wait(acc_empty(half), (i / kChunk >> 1 & 1) ^ 1))) break;
                acc_fence_after();
            }
            if (!(ok = warp_wait(full(s), i / kS & 1))) break;
            const uint64_t a = first_a + uint32_t(s) * (T::kStage >> 4), b = a + (kTileM * kRowBytes >> 4);
            if (elected()) {
                product<1>(acc + half * kN, a, b, desc, i % kChunk > 0);
#pragma unroll
                for (uint32_t k = 1; k < kTileK / 16; ++k) product<1>(acc + half * kN, a + k * a_step, b + k * b_step, desc, 1);
                product_commit<1>(empty(s));
                if (i % kChunk == kChunk - 1 || i == to - from - 1) product_commit<1>(acc_full(half));
            }
            __syncwarp();
        }
        if (!ok) {
            failed = 1;
            if (elected()) product_commit<1>(drained);
            bar_wait(drained, 0);
        }
    } else if (warp >= 4) {
        const int quarter = warp & 3, row = quarter * 32 + lane, own = (warp - 4) / 4 * T::kOwn;
        float total[T::kOwn] = {};
        bool ok = true;
        for (int c = 0; c * kChunk < to - from; ++c) {
            if (!(ok = warp_wait(acc_full(c & 1), c >> 1 & 1))) break;
            acc_fence_after();
#pragma unroll
            for (int p = 0; p < T::kOwn; p += T::kPiece) {
                float v[T::kPiece];
                acc_load(acc + (c & 1) * kN + (uint32_t(quarter * 32) << 16) + own + p, v);
#pragma unroll
                for (int i = 0; i < T::kPiece; ++i) total[p + i] += v[i];
            }
            acc_fence_before();
            __syncwarp();
            if (lane == 0) bar_arrive(acc_empty(c & 1));
        }
        if (!ok) failed = 1;
        // (the last product is done: the ring's stages are free)
        if (mt * kTileM + row < g.m)
#pragma unroll
            for (int f = 0; f < T::kOwn / 4; ++f)
                asm volatile("st.shared.v4.f32 [%0], {%1,%2,%3,%4};" ::"r"(ring + sum_place<kN>(row, own / 4 + f)), "f"(total[4 * f]), "f"(total[4 * f + 1]), "f"(total[4 * f + 2]),
                             "f"(total[4 * f + 3]) : "memory");
    }
    __syncwarp();
    acc_fence_before();
    cluster_barrier();
    if (warp == 2) {
        acc_fence_after();
        acc_free<1>(acc, 2 * kN);
    }
    const int rows = min(kTileM, g.m - mt * kTileM);
    for (int i = rank * T::kThreads + int(threadIdx.x); i < rows * (kN / 4); i += parts * T::kThreads) {
        const int r = i / (kN / 4), f = i % (kN / 4), col = nt * kN + f * 4;
        if (col >= g.n) continue;
        float v[4] = {0.f, 0.f, 0.f, 0.f};
        float4 p[kSplitMost];
#pragma unroll
        for (int q = 0; q < kSplitMost; ++q)
            if (q < parts) p[q] = load_at_rank(ring + sum_place<kN>(r, f), q);
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

__global__ void __launch_bounds__(kThreads) repack_kernel(const Repacks g BAOC_CHECK_PARAM) {
    begin_in_row();
    for (int64_t i = int64_t(blockIdx.x) * kThreads + threadIdx.x; i < g.ends[g.n - 1]; i += int64_t(gridDim.x) * kThreads) {
        int which = 0;
        while (i >= g.ends[which]) ++which;
        const Repack& r = g.r[which];
        const int64_t at = i - (which ? g.ends[which - 1] : 0);
        const int pieces = (r.cols + 7) / 8;
        const int64_t row = at / pieces;
        const int col = int(at - row * pieces) * 8;
#ifdef BAOC_CHECKED
        if (!check_range(ck, kKerLinearRepack, r.to + row * r.to_step + 2 * col, 16, which)) return;
#endif
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

// a thread's 8 of 256 columns: neighbours (kWide), or 32 apart
template <bool kWide>
__device__ __forceinline__ int slope_column(int lane, int j) { return kWide ? lane * 8 + j : j * 32 + lane; }
template <bool kWide>
__device__ __forceinline__ void load8(const char* row, int base, int lane, int n, float (&x)[8]) {
    if constexpr (kWide) {
        unpack8(ld_stream_u4(row + 2 * int64_t(base + lane * 8)), x);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int c = base + slope_column<false>(lane, j);
            x[j] = c < n ? bf16_bits_to_float(reinterpret_cast<const uint16_t*>(row)[c]) : 0.f;
        }
    }
}
// as bf16 into a row, and what the rounding left into d
template <bool kWide>
__device__ __forceinline__ void store8(char* row, int base, int lane, int n, float (&d)[8]) {
    const uint4 w = make_uint4(pair_bf16(d[0], d[1]), pair_bf16(d[2], d[3]), pair_bf16(d[4], d[5]), pair_bf16(d[6], d[7]));
    float h[8];
    unpack8(w, h);
    if constexpr (kWide) {
        *reinterpret_cast<uint4*>(row + 2 * int64_t(base + lane * 8)) = w;
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int c = base + slope_column<false>(lane, j);
            if (c < n) reinterpret_cast<uint16_t*>(row)[c] = uint16_t(__float_as_uint(h[j]) >> 16);
        }
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) d[j] -= h[j];
}

// kWide: n is a multiple of 8, and the rows of dout and pre start on 16-byte boundaries.
template <int kAct, bool kWide>
__global__ void __launch_bounds__(kThreads) slope_kernel(const SlopeArgs g BAOC_CHECK_PARAM) {
    constexpr bool kPre = kAct != BAOC_ACT_NONE;
    __shared__ float sh[8][256];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, base = int(blockIdx.x) * 256;
    const int64_t first = int64_t(blockIdx.y) * g.rows_per_part, end = min64(g.rows, first + g.rows_per_part);
    float sum[8] = {};
    begin_in_row();
#ifdef BAOC_CHECKED
    {
        const int cols = min(256, g.n - base);
        int what = 0;
        for (char* dz : {g.dz, g.dz_mid, g.dz_low}) {
            if (dz && first < end && !check_range(ck, kKerLinearSlope, dz + first * g.dz_step + 2 * base, (end - 1 - first) * g.dz_step + 2 * cols, what)) return;
            ++what;
        }
        if (g.part && !check_range(ck, kKerLinearSlope, g.part + int64_t(blockIdx.y) * g.n + base, 4ll * cols, 3)) return;
    }
#endif
    auto one_row = [&](int64_t row, float (&d)[8], const float (&z)[8]) {
        if constexpr (kPre) {
#pragma unroll
            for (int j = 0; j < 8; j += 2) unpack2(mul2(pack2(d[j], d[j + 1]), act_slope<kAct>(pack2(z[j], z[j + 1]))), d[j], d[j + 1]);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) sum[j] += d[j];
        if (!g.dz) return;
        store8<kWide>(g.dz + row * g.dz_step, base, lane, g.n, d);
        if (!kPre || !g.dz_mid) return;
        store8<kWide>(g.dz_mid + row * g.dz_step, base, lane, g.n, d);
        store8<kWide>(g.dz_low + row * g.dz_step, base, lane, g.n, d);
    };
    if (base + slope_column<kWide>(lane, 0) < g.n)
        for (int64_t row = first + warp; row < end; row += 8 * kSlopeRows) {
            float d[kSlopeRows][8], z[kPre ? kSlopeRows : 1][8];
            auto load = [&](int64_t at, int r) {
                load8<kWide>(g.dout + at * g.dout_step, base, lane, g.n, d[r]);
                if constexpr (kPre) load8<kWide>(g.pre + at * g.pre_step, base, lane, g.n, z[r]);
            };
            if (row + 8 >= end) {                    // a warp's last row (of few, its only one) alone
                load(row, 0);
                one_row(row, d[0], z[0]);
                break;
            }
#pragma unroll
            for (int r = 0; r < kSlopeRows; ++r) load(min64(row + 8 * r, end - 1), r);       // (a row too many is read, not used)
#pragma unroll
            for (int r = 0; r < kSlopeRows; ++r)
                if (row + 8 * r < end) one_row(row + 8 * r, d[r], z[kPre ? r : 0]);
        }
    if (!g.part) return;
#pragma unroll
    for (int j = 0; j < 8; ++j) sh[warp][slope_column<kWide>(lane, j)] = sum[j];
    __syncthreads();
    const int c = base + int(threadIdx.x);
    if (c < g.n) {
        float s = sh[0][threadIdx.x];
        for (int w = 1; w < 8; ++w) s += sh[w][threadIdx.x];
        g.part[int64_t(blockIdx.y) * g.n + c] = s;
    }
}

// The parts' column sums, 32 columns per CTA: every warp adds each 32nd part, then the warps' sums are added in order.
__global__ void __launch_bounds__(1024) slope_sums_kernel(const float* __restrict__ part, int parts, int n, char* db, int f32 BAOC_CHECK_PARAM) {
    __shared__ float sh[32][33];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, col = int(blockIdx.x) * 32 + lane;
    begin_in_row();
#ifdef BAOC_CHECKED
    if (!check_range(ck, kKerLinearSlope, part, 4ll * parts * n, 4)) return;
#endif
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
    // A tiled store writes whole units of 16 bytes: rows that end inside one, in a buffer of wider rows, would lose what lies behind them.
    int width() const { return !wide() ? 0 : (cols * eb % 16 ? 1 : kTiled); }
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

// A product to be formed: sizes, flags and the epilogue in g, where it goes in out and pre.
struct Product {
    Operands o;
    Matrix out, pre;
    ProductArgs g;
    int64_t tiles(int m, int n) const { return ceil_div(g.m, m) * ceil_div(g.n, n); }
    int64_t steps() const { return int64_t(g.k_tiles) * g.passes; }
    bool chunked() const { return out.eb == 4 || steps() > kLongSum; }
};

// A product as a kernel with tiles of m x n takes it (b_rows: of a CTA's copy of B).
int fill_problem(const Product& d, int m, int n, int b_rows, bool stores, Problem* p, int* tiles) {
    p->g = d.g;
    p->g.m_tiles = int(ceil_div(d.g.m, m));
    p->g.n_tiles = int(ceil_div(d.g.n, n));
    const int64_t t = d.tiles(m, n);
    if (t > 0x7fffffff / 4) return fail_linear(BAOC_E_INVALID, "too many tiles for one launch");
    *tiles = int(t);
    bool ok = true;
    for (int i = 0; i < d.g.passes; ++i) ok = ok && encode(&p->maps.a[i], *d.o.a[i], d.g.a_mn ? kTileK : d.g.a_rows) && encode(&p->maps.b[i], *d.o.b[i], d.g.b_mn ? kTileK : b_rows);
    if (stores && d.g.out_wide == kTiled) ok = ok && encode(&p->maps.out, d.out, 32, 32);
    if (stores && d.g.pre && d.g.pre_wide == kTiled) ok = ok && encode(&p->maps.pre, d.pre, 32, 32);
    return ok ? BAOC_OK : fail_linear(BAOC_E_CUDA, "the driver refused a tensor map");
}

// The permission for large shared memory is per kernel and device and lasts.
template <typename K>
int allow_shared(K kernel, int bytes, std::atomic<uint64_t>* allowed) {
    int dev = 0;
    cudaError_t ce = cudaGetDevice(&dev);
    const uint64_t bit = dev < 64 ? uint64_t(1) << dev : 0;
    if (ce == cudaSuccess && !(allowed->load(std::memory_order_relaxed) & bit)) {
        ce = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
        if (ce == cudaSuccess) allowed->fetch_or(bit, std::memory_order_relaxed);
    }
    return launched(ce, "product_kernel");
}

template <int kCtas, int kN, bool kChunked>
int launch_product(const Product* d, int count, cudaStream_t s) {
    using T = TileShape<kCtas, kN, kChunked>;
    static_assert(T::kStages >= 4 && T::kSmem <= 227 * 1024 - 512, "the ring, the outputs and the barriers share 227 KB");
    auto kernel = product_kernel<kCtas, kN, kChunked>;
    static std::atomic<uint64_t> allowed{0};
    int rc = allow_shared(kernel, T::kSmem, &allowed);
    Problems all;
    all.tiles[1] = all.fewer = 0;
    for (int i = 0; i < count && !rc; ++i) rc = fill_problem(d[i], kTileM * kCtas, kN, T::kBRows, true, &all.p[i], &all.tiles[i]);
    if (rc) return rc;
    const int workers = int(std::min<int64_t>(int64_t(all.tiles[0]) + all.tiles[1], 148 / kCtas));
    if (count == 2) {                                // the share of the second that ends soonest (see Walk)
        const int64_t longer = all.tiles[0] % workers, rounds = all.tiles[0] / workers, s0 = d[0].steps(), s1 = d[1].steps();
        int64_t best = -1;
        for (int q = 0; q <= ceil_div(all.tiles[1], workers); ++q) {
            const int64_t rest = std::max<int64_t>(0, all.tiles[1] - int64_t(q) * workers);
            const int64_t end = std::max((rounds + (longer > 0)) * s0 + q * s1, rounds * s0 + (q + ceil_div(rest, workers - longer)) * s1);
            if (best < 0 || end < best) { best = end; all.fewer = q; }
        }
    }
    return launched(launch_in_row(kernel, dim3(unsigned(workers * kCtas)), kProductThreads, T::kSmem, kCtas, s, all), "product_kernel");
}

template <int kN>
int launch_split(const Product* d, int count, int parts, cudaStream_t s) {
    using T = SplitShape<kN>;
    static std::atomic<uint64_t> allowed{0};
    int rc = allow_shared(product_split_kernel<kN>, T::kSmem, &allowed);
    Problems all;
    all.tiles[1] = all.fewer = 0;
    for (int i = 0; i < count && !rc; ++i) rc = fill_problem(d[i], kTileM, kN, kN, false, &all.p[i], &all.tiles[i]);
    if (rc) return rc;
    return launched(launch_in_row(product_split_kernel<kN>, dim3(unsigned((all.tiles[0] + all.tiles[1]) * parts)), T::kThreads, T::kSmem, unsigned(parts), s, all, parts),
                    "product_split_kernel");
}

// The kernel for a product: the one that is expected to end first.  A step (64 k of a tile) takes the tensor cores 4 products'
// time or the copies their bytes at 64 a clock and SM (what L2 gives one), and no less than a copy's way (2800 clocks) over the
// stages in flight; steps follow one another in every CTA, rounds of tiles too, and everything together takes at least the
// operands' bytes at 3400 a clock (HBM).  Rows off the 16-byte grid are written by the warps themselves, 32 clocks a column.
// Against the largest tiles that give every CTA one: 512 x 4096 into 4096 47 -> 18 us, the gradient of 4096 x 768 into 2304
// 74 -> 36 us.  A split's sums meet at 6000 clocks.  Tiles of 256 columns are charged more: their sums take longer to meet, and they
// have an SM to themselves.  How much is fitted to 800 calls (products and gradients of 1 to 16384 tokens, 48 to 8192 columns, drawn
// evenly over the logarithms, where these tiles are within reach): the mean time over that of each call's best choice is 1.9 % with
// 9000 clocks, 0.9 with 14000 to 16000, 1.0 with 18000, 1.5 with 24000 and 2.8 without such tiles.  dw of 16384 x 768 into 768, split
// six ways, takes 26 us instead of 41, of 16384 x 1024 into 1024 33 instead of 56.
enum Kind : int { kPairs256, kPairs128, kOnes128, kOnes64, kSplit64, kSplit256 };
struct Choice {
    Kind kind;
    int parts;
};
Choice choose(const Product& d, int split_most) {
    const ProductArgs& g = d.g;
    const int64_t steps = d.steps(), a_bytes = int64_t(g.a_rows) * kRowBytes, bytes = 2 * (int64_t(g.m) + g.n) * 64 * steps;
    Choice best{kSplit64, 0};
    int64_t least = 0;
    auto consider = [&](Kind kind, int parts, int64_t rounds, int64_t own_steps, int64_t step, int64_t fixed) {
        const int64_t cost = std::max(rounds * own_steps * step, bytes / 3400) + fixed;
        if (best.parts == 0 || cost < least) { best = Choice{kind, parts}; least = cost; }
    };
    auto whole = [&](Kind kind, int ctas, int n, int64_t products) {
        consider(kind, 1, ceil_div(d.tiles(kTileM * ctas, n), 148 / ctas), steps, std::max<int64_t>({products, (a_bytes + n / ctas * kRowBytes) / 64, 2800 / 6}), 3000 + (g.out_wide == kTiled ? 0 : 32 * n));
    };
    if (!d.chunked()) whole(kPairs256, 2, 256, 512);
    whole(kPairs128, 2, 128, 256);
    if (!d.chunked()) whole(kOnes128, 1, 128, 256);
    whole(kOnes64, 1, 64, 128);
    const int64_t tiles = d.tiles(kTileM, 64), step = (a_bytes + 64 * kRowBytes) / 64;
    for (int parts = 2; parts <= kSplitMost && tiles * parts <= split_most && steps >= 4 * parts; parts *= 2)
        consider(kSplit64, parts, 1, ceil_div(steps, parts), std::max<int64_t>(tiles * parts > 148 ? 2 * step : step, 2800 / SplitShape<64>::kStages), 6000);
    constexpr int kClusters[kSplitMost + 1] = {0, 148, 74, 45, 33, 26, 22, 15, 15};      // that find room at once with an SM per CTA
    const int64_t wide_tiles = d.tiles(kTileM, 256);
    for (int parts = 2; parts <= kSplitMost && steps >= 4 * parts; ++parts)
        if (wide_tiles <= kClusters[parts])
            consider(kSplit256, parts, 1, ceil_div(steps, parts), std::max<int64_t>((a_bytes + 256 * kRowBytes) / 64, 2800 / SplitShape<256>::kStages), 16000);
    return best;
}

// split_most: CTAs (of which an SM holds two) that one product's sums may be split among: by it, not by what else is formed, so
// that a product's bits do not depend on that.
int form_products(Product* d, int count, int split_most, cudaStream_t s) {
    Kind kind[2];
    int parts[2];
    for (int i = 0; i < count; ++i) {
        ProductArgs& g = d[i].g;
        g.out = const_cast<char*>(d[i].out.p); g.out_step = d[i].out.step; g.out_f32 = d[i].out.eb == 4; g.out_wide = d[i].out.width();
        g.pre = const_cast<char*>(d[i].pre.p); g.pre_step = d[i].pre.step; g.pre_wide = d[i].pre.width();
        g.a_rows = g.a_mn ? kTileM : std::min(kTileM, int(round_up(g.m, 8)));
        const Choice c = choose(d[i], split_most);
        kind[i] = c.kind;
        parts[i] = c.parts;
    }
    // two of one kind in one launch (chunked and other sums are two kinds)
    const bool alike = count == 2 && kind[0] == kind[1] && parts[0] == parts[1] && (kind[0] >= kSplit64 || d[0].chunked() == d[1].chunked());
    const int step = alike ? 2 : 1;
    for (int i = 0; i < count; i += step) {
        int rc;
        switch (kind[i]) {
            case kSplit64: rc = launch_split<64>(d + i, step, parts[i], s); break;
            case kSplit256: rc = launch_split<256>(d + i, step, parts[i], s); break;
            case kPairs256: rc = launch_product<2, 256, false>(d + i, step, s); break;
            case kPairs128: rc = d[i].chunked() ? launch_product<2, 128, true>(d + i, step, s) : launch_product<2, 128, false>(d + i, step, s); break;
            case kOnes128: rc = launch_product<1, 128, false>(d + i, step, s); break;
            default: rc = d[i].chunked() ? launch_product<1, 64, true>(d + i, step, s) : launch_product<1, 64, false>(d + i, step, s); break;
        }
        if (rc) return rc;
    }
    return BAOC_OK;
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
    int launch(cudaStream_t s, const CheckCtx& ck) const {
        (void)ck;
        if (!todo.n) return BAOC_OK;
        const unsigned grid = unsigned(std::min<int64_t>(ceil_div(todo.ends[todo.n - 1], kThreads), 148 * 16));
        return launched(launch_in_row(repack_kernel, dim3(grid), kThreads, 0, 1, s, todo BAOC_CHECK_ARG(ck)), "repack_kernel");
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

BAOC_DEFINE_CHECK_FETCH(linear_check_fetch)

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
        mo(out, tokens, e->n_out, e->out_stride, e->out_dtype), mr(residual, tokens, e->n_out, e->residual_stride, e->out_dtype), mp(pre, tokens, e->n_out, e->pre_stride, BAOC_BF16),
        mb(bias, 1, e->n_out, 0, BAOC_F32);
    for (const Matrix* t : {&mx, &mw, &mo, &mr, &mp, &mb})
        if (!t->fits()) return fail_linear(BAOC_E_ALIGN, "baoc_linear: a pointer is not aligned to its elements");
    if (!aligned(ws, 256)) return fail_linear(BAOC_E_ALIGN, "baoc_linear: workspace not 256-byte aligned");
    const Matrix space(ws, 1, int64_t(ws_bytes) / 2, 0, BAOC_BF16);
    if (overlap(mo, mx) || overlap(mo, mw) || overlap(mp, mx) || overlap(mp, mw) || overlap(mo, mp) || overlap(mp, mr) || overlap(mo, mb) ||
        overlap(mp, mb) || (overlap(mo, mr) && !(mo.p == mr.p && (mo.step == mr.step || tokens == 1))))
        return fail_linear(BAOC_E_INVALID, "baoc_linear: out may be residual; outputs overlap nothing else");
    if (ws_bytes)
        for (const Matrix* t : {&mx, &mw, &mo, &mr, &mp, &mb})
            if (overlap(space, *t)) return fail_linear(BAOC_E_INVALID, "baoc_linear: the workspace overlaps an array");
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    Packer pack(ws, ws_bytes);
    const Matrix a = pack.operand(mx), b = pack.operand(mw);
    if (!pack.fits) return fail_linear(BAOC_E_WORKSPACE, "baoc_linear: workspace too small");
    const CheckCtx ck{static_cast<char*>(ws), static_cast<char*>(ws) + ws_bytes, 0, 0, 0};
    if ((rc = pack.launch(s, ck))) return rc;
    Product d{Operands{{&a}, {&b}}, mo, mp, {}};
    ProductArgs& g = d.g;
    g.m = int(tokens); g.n = e->n_out; g.k_tiles = int(ceil_div(e->n_in, kTileK)); g.passes = 1;
    g.b_mn = !out_in;
    g.act = e->act; g.bias = bias;
    g.residual = mr.p; g.residual_step = mr.step; g.residual_wide = mr.wide();
    return form_products(&d, 1, 2 * 148, s);
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
    const CheckCtx ck{static_cast<char*>(ws), static_cast<char*>(ws) + ws_bytes, 0, 0, 0};
    if ((rc = pack.launch(s, ck))) return rc;
    if (g.dz || g.part) {
        g.dout = md.p; g.pre = mp.p; g.dout_step = md.step; g.pre_step = mp.step; g.dz_step = packed_step(e->n_out);
        g.rows = tokens; g.n = e->n_out;
        const dim3 grid(unsigned(ceil_div(e->n_out, 256)), unsigned(parts));
        const bool wide = e->n_out % 8 == 0 && md.wide() && (!act || mp.wide());
        auto go = [&](auto a) {
            return launched(launch_in_row(wide ? slope_kernel<decltype(a)::value, true> : slope_kernel<decltype(a)::value, false>, grid, kThreads, 0, 1, s, g BAOC_CHECK_ARG(ck)), "slope_kernel");
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
                                                   int(e->n_out), static_cast<char*>(db), int(e->grad_dtype == BAOC_F32) BAOC_CHECK_ARG(ck)), "slope_sums_kernel")))
            return rc;
    }
    // (the longer sums first: what the second product's shorter ones leave uneven is less)
    const Matrix none(nullptr, 0, 0, 0, BAOC_BF16);
    Product d[2]{{{}, none, none, {}}, {{}, none, none, {}}};
    int count = 0;
    if (dw) {
        Product& q = d[count++];
        q.o = out_in ? Operands{{&dz, &mid, &low}, {&bx, &bx, &bx}} : Operands{{&bx, &bx, &bx}, {&dz, &mid, &low}};
        q.out = mdw;
        q.g.m = int(w_rows); q.g.n = int(w_cols); q.g.k_tiles = int(ceil_div(tokens, kTileK)); q.g.passes = split ? 3 : 1;
        q.g.a_mn = q.g.b_mn = 1;
    }
    if (dx) {
        Product& q = d[count++];
        q.o = Operands{{&dz}, {&bw}};
        q.out = mdx;
        q.g.m = int(tokens); q.g.n = e->n_in; q.g.k_tiles = int(ceil_div(e->n_out, kTileK)); q.g.passes = 1;
        q.g.b_mn = out_in;
    }
    if (count == 2 && d[0].steps() < d[1].steps()) std::swap(d[0], d[1]);
    if (count) return form_products(d, count, 148, s);
    return BAOC_OK;
} catch (const std::bad_alloc&) {
    return BAOC_E_INVALID;
}

}  // extern "C"
