// The join of a block's branch into the residual stream, with the norm behind the branch and the norm before the next block.
//
//   y = c x + g * post(f),   h = pre(y)
//
// post and pre are an RMS norm (n(v) = v / sqrt(mean(v^2) + eps)) or a layer norm (the same of v - mean(v)), each with a weight
// and, for layer norms, a bias per column; g is nothing, a vector or a vector per group of rows.  Backwards, with
// n = n(v) and r = 1 / sqrt(..) of a norm, dn = dout * w:
//
//   dv = r (dn - n mean(dn n) [- mean(dn) for a layer norm]),  dw = sum over rows of dout * n,  db = sum over rows of dout
//   Dy = dy + (dv of pre, from dh),  dx = c Dy,  du = g * Dy,  dg = sum over the group's rows of Dy * post(f),  df = (dv of post, from du)
//
// Memory bounds both ways: x and f in, y and h out; y, f, dy and dh in, dx and df out, and nothing else moves but the column
// sums.  A row lies in the registers of its threads (a team: 8 columns each) from its load to its store, so statistics need no
// second pass, and the mean is taken out before the squares are summed.  The gradient's column sums stay with the team's threads
// over all rows of a CTA; the CTAs' sums are joined by a second kernel in a fixed order.  All arithmetic is fp32; y, h, dx and df
// are rounded once, and h comes from the unrounded y.
// Times below: one B200, device time per call in a row of calls on three sets of arrays.
#include <algorithm>
#include <cmath>
#include <cuda_runtime.h>
#include <new>
#include <string>

#include "baoc_device.cuh"

namespace baoc {

constexpr int kJoinMaxDim = 8192;
constexpr int64_t kJoinMaxStride = int64_t(1) << 28;
constexpr int kJoinCols = 8;                   // columns of a thread
constexpr int kSoloWarps = 4;                  // rows that a warp takes alone: so many warps per CTA
constexpr int kJoinWarps = 32, kJoinGradWarps = 16;    // warps per SM of the other rows' kernels
constexpr int kFewRows = 592;                  // few rows: up to 4 per SM
constexpr int kJoinSums = 5;                   // column sums of the gradient: weight and bias of pre, of post, and the gate

// How a row is spread.  Classes 1 to 3: one warp, each lane 1 to 3 times 8 columns (no barrier, and a sum's shuffles are paid
// once a row: 65536 x 768 bf16 layer norms forwards 110 -> 73 us against three warps).  Classes 4, 5 and 6: a CTA of as many warps as the row
// needs, up to 8, 16 and 32, 8 columns a thread (what differs is the registers that a thread may have).  Few rows of 2 or 3 times
// 256 columns are of class 4 too: with one row a warp at most there is nothing to pay shuffles for, and a lane's loads wait for one another
// (one bf16 row of 768, layer norms: 4.9 -> 3.3 us, its gradient 8.3 -> 6.1, of 296 rows 10.8 -> 9.4; at 592 both ways take as long).
__host__ __device__ constexpr bool solo(int c) { return c <= 3; }
__host__ __device__ constexpr int chunks_of(int c) { return c <= 3 ? c : 1; }
__host__ __device__ constexpr int class_threads(int c) { return c <= 3 ? 32 * kSoloWarps : (c == 4 ? 256 : (c == 5 ? 512 : 1024)); }
// warps per SM that the registers (and, backwards, the shared memory) allow
__host__ __device__ constexpr int class_warps(int c) { return c == 1 ? 32 : (c == 2 ? 24 : (c == 3 ? 16 : kJoinWarps)); }
__host__ __device__ constexpr int class_grad_warps(int c) { return c <= 2 ? 12 : (c == 3 ? 8 : kJoinGradWarps); }
__host__ __device__ constexpr int class_blocks(int c, int warps) { return c == 6 ? 1 : warps * 32 / class_threads(c); }
// Threads of a team as the columns are counted: a lane with several times 8 columns counts as so many threads.
template <int kClass>
__device__ __forceinline__ int team_size() { return solo(kClass) ? 32 * chunks_of(kClass) : int(blockDim.x); }

template <int DT, int kClass, bool kWide>
struct RowPart {
    // a thread's 8 columns: neighbours, or a team's size apart
    static constexpr int kSize = DT == BAOC_BF16 ? 2 : 4;
    static constexpr int kWords = kWide ? 2 * kSize : 8;
    uint32_t w[kWords];
    static __device__ __forceinline__ int column(int t, int j) { return kWide ? t * kJoinCols + j : j * team_size<kClass>() + t; }

    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int i = 0; i < kWords; ++i) w[i] = 0;
    }
    __device__ __forceinline__ void load(const char* row, int t, int dim) {
        if constexpr (kWide) {
            clear();
            if (t * kJoinCols < dim) {
                const char* p = row + t * kJoinCols * kSize;
                if constexpr (DT == BAOC_F32) {
                    ld_stream_u8(p, w);
                } else {
                    const uint4 a = ld_stream_u4(p);
                    w[0] = a.x; w[1] = a.y; w[2] = a.z; w[3] = a.w;
                }
            }
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int c = column(t, j);
                if constexpr (DT == BAOC_BF16) w[j] = c < dim ? *reinterpret_cast<const uint16_t*>(row + 2 * c) : 0;
                else w[j] = c < dim ? *reinterpret_cast<const uint32_t*>(row + 4 * c) : 0;
            }
        }
    }
    // The same of a bf16 row by way of shared memory: requested ahead, without a register.  A thread reads back what it requested
    // itself.
    static __device__ __forceinline__ void request(uint32_t slot, const char* row, int t) { cp_async16(slot + t * 16, row + t * 16); }
    __device__ __forceinline__ void take(uint32_t slot, int t) {
        asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(slot + t * 16) : "memory");
    }
    __device__ __forceinline__ void get(f32x2 (&x)[4]) const {
        if constexpr (DT == BAOC_F32) {
#pragma unroll
            for (int j = 0; j < 4; ++j) x[j] = pack2(__uint_as_float(w[2 * j]), __uint_as_float(w[2 * j + 1]));
        } else if constexpr (kWide) {
#pragma unroll
            for (int j = 0; j < 4; ++j) x[j] = pack2(bf16_lo(w[j]), bf16_hi(w[j]));
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) x[j] = pack2(bf16_lo(w[2 * j]), bf16_lo(w[2 * j + 1]));
        }
    }
    static __device__ __forceinline__ void store(char* row, int t, int dim, const f32x2 (&v)[4]) {
        float x[8];
#pragma unroll
        for (int j = 0; j < 4; ++j) unpack2(v[j], x[2 * j], x[2 * j + 1]);
        if constexpr (kWide) {
            if (t * kJoinCols >= dim) return;
            char* p = row + t * kJoinCols * kSize;
            if constexpr (DT == BAOC_F32) {
                st_stream_f8(p, x);
            } else {
                uint4 r;
                asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r.x) : "f"(x[1]), "f"(x[0]));
                asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r.y) : "f"(x[3]), "f"(x[2]));
                asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r.z) : "f"(x[5]), "f"(x[4]));
                asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r.w) : "f"(x[7]), "f"(x[6]));
                st_stream_u4(p, r);
            }
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int c = column(t, j);
                if (c >= dim) continue;
                if constexpr (DT == BAOC_F32) {
                    *reinterpret_cast<float*>(row + 4 * c) = x[j];
                } else {
                    uint16_t h;
                    asm("cvt.rn.bf16.f32 %0, %1;" : "=h"(h) : "f"(x[j]));
                    *reinterpret_cast<uint16_t*>(row + 2 * c) = h;
                }
            }
        }
    }
    // v less m, and zero where there is no column.  (kWide: a thread has all of its columns or none; one without any leaves the
    // sums at zero and the rest alone.)
    static __device__ __forceinline__ void centre(f32x2 (&v)[4], float m, int t, int dim) {
        const f32x2 m2 = splat2(-m);
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = add2(v[j], m2);
        if constexpr (!kWide) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                float a, b;
                unpack2(v[j], a, b);
                v[j] = pack2(column(t, 2 * j) < dim ? a : 0.f, column(t, 2 * j + 1) < dim ? b : 0.f);
            }
        }
    }
};

__device__ __forceinline__ float sum8(const f32x2 (&v)[4]) {
    float a, b;
    unpack2(add2(add2(v[0], v[1]), add2(v[2], v[3])), a, b);
    return a + b;
}
__device__ __forceinline__ float dot8(const f32x2 (&v)[4], const f32x2 (&w)[4]) {
    float a, b;
    unpack2(fma2(v[3], w[3], fma2(v[2], w[2], fma2(v[1], w[1], mul2(v[0], w[0])))), a, b);
    return a + b;
}

// A thread's 8 values of a vector per column (fp32, 4-byte aligned); `other` where there is none.
template <int kClass, bool kWide>
__device__ __forceinline__ void per_column(const float* v, int t, int dim, float other, f32x2 (&x)[4]) {
    using P = RowPart<BAOC_F32, kClass, kWide>;
    if (kWide && v && t * kJoinCols < dim) {
        const float4 a = __ldg(reinterpret_cast<const float4*>(v + t * kJoinCols)), b = __ldg(reinterpret_cast<const float4*>(v + t * kJoinCols) + 1);
        x[0] = pack2(a.x, a.y); x[1] = pack2(a.z, a.w); x[2] = pack2(b.x, b.y); x[3] = pack2(b.z, b.w);
        return;
    }
    auto one = [&](int j) { return v && P::column(t, j) < dim ? __ldg(v + P::column(t, j)) : other; };
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = pack2(one(2 * j), one(2 * j + 1));
}

// The same, read row after row: kept in shared memory, every thread its own (from L1 or L2 each would cost its latency in every
// row, and registers have the row).  Warps that work alone share one copy, but for the gate.
template <int kClass>
struct Kept {
    float4* at;                      // [vector][2][team's threads]
    __device__ __forceinline__ float4* place(int which, int t) const { return at + which * 2 * team_size<kClass>() + t; }
    __device__ __forceinline__ void put(int which, int t, const f32x2 (&x)[4]) const {
        float v[8];
#pragma unroll
        for (int j = 0; j < 4; ++j) unpack2(x[j], v[2 * j], v[2 * j + 1]);
        float4* p = place(which, t);
        p[0] = make_float4(v[0], v[1], v[2], v[3]);
        p[team_size<kClass>()] = make_float4(v[4], v[5], v[6], v[7]);
    }
    __device__ __forceinline__ void get(int which, int t, f32x2 (&x)[4]) const {
        const float4* p = place(which, t);
        const float4 a = p[0], b = p[team_size<kClass>()];
        x[0] = pack2(a.x, a.y); x[1] = pack2(a.z, a.w); x[2] = pack2(b.x, b.y); x[3] = pack2(b.z, b.w);
    }
};
enum Vector : int { kVPreW = 0, kVPostW = 1, kVGate = 2, kVPreB = 2, kVPostB = 3 };      // (forwards every team keeps a gate of its own, behind these)

// Sums of K = 1, 2 or 4 values over a team, the same in all of its threads.  In a warp the lanes first share the values out (a
// lane keeps half of them and adds its neighbour's half, so 4 values cost 6 shuffles and not 20).  A CTA's warps take turns of
// two buffers, so that one barrier a round is enough; all of its threads call it.
template <int kClass>
struct TeamSum {
    float4 (*buf)[32];               // [2][warps]
    int turn = 0;
    template <int K>
    __device__ __forceinline__ void operator()(float (&v)[K]) {
        static_assert(K == 1 || K == 2 || K == 4, "");
        constexpr uint32_t kAll = 0xffffffffu;
        const int lane = threadIdx.x & 31;
        float r = v[0];
        int at = 0;                  // which of the values this lane ends up with
        if constexpr (K == 4) {
            const bool odd = lane & 1;
            const float a = (odd ? v[2] : v[0]) + __shfl_xor_sync(kAll, odd ? v[0] : v[2], 1), b = (odd ? v[3] : v[1]) + __shfl_xor_sync(kAll, odd ? v[1] : v[3], 1);
            const bool up = lane & 2;
            r = (up ? b : a) + __shfl_xor_sync(kAll, up ? a : b, 2);
            at = (odd ? 2 : 0) + (up ? 1 : 0);
        } else if constexpr (K == 2) {
            const bool odd = lane & 1;
            r = (odd ? v[1] : v[0]) + __shfl_xor_sync(kAll, odd ? v[0] : v[1], 1);
            at = odd;
        }
#pragma unroll
        for (int o = K; o < 32; o <<= 1) r += __shfl_xor_sync(kAll, r, o);
        if constexpr (solo(kClass)) {
            v[0] = r;
            if constexpr (K > 1) {
                constexpr int kFrom[4] = {0, K == 4 ? 2 : 1, 1, 3};      // a lane that has value k
#pragma unroll
                for (int k = 0; k < K; ++k) v[k] = __shfl_sync(kAll, r, kFrom[k]);
            }
        } else {
            const int warps = int(blockDim.x) >> 5;
            if (lane < K) reinterpret_cast<float*>(&buf[turn][threadIdx.x >> 5])[at] = r;
            __syncthreads();
            float4 s;
            if constexpr (kClass == 4) {             // up to 8 warps: every thread adds them up
                s = buf[turn][0];
                for (int w = 1; w < warps; ++w) {
                    const float4 o = buf[turn][w];
                    s.x += o.x; s.y += o.y; s.z += o.z; s.w += o.w;
                }
            } else {
                s = lane < warps ? buf[turn][lane] : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) {
                    s.x += __shfl_xor_sync(kAll, s.x, o);
                    if constexpr (K > 1) s.y += __shfl_xor_sync(kAll, s.y, o);
                    if constexpr (K > 2) { s.z += __shfl_xor_sync(kAll, s.z, o); s.w += __shfl_xor_sync(kAll, s.w, o); }
                }
            }
            const float all[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
            for (int k = 0; k < K; ++k) v[k] = all[k];
            turn ^= 1;
        }
    }
};

struct JoinArgs {
    const char *x, *f;
    char *y, *h;
    const float *post_w, *post_b, *gate, *pre_w, *pre_b;
    int64_t x_step, f_step, y_step, h_step, rows, rows_per_gate, rows_per_cta;
    int dim, layer;
    float scale, eps;
};

template <int S, int B, int kClass, bool kWide>
__global__ void __launch_bounds__(class_threads(kClass), class_blocks(kClass, class_warps(kClass))) join_kernel(const JoinArgs g) {
    constexpr bool kSolo = solo(kClass);
    constexpr int kTeams = kSolo ? kSoloWarps : 1, kC = chunks_of(kClass);
    using Stream = RowPart<S, kClass, kWide>;
    using Branch = RowPart<B, kClass, kWide>;
    __shared__ float4 buf[kSolo ? 1 : 2][32];
    TeamSum<kClass> sum{buf};
    begin_in_row();
    const int t = kSolo ? int(threadIdx.x & 31) : int(threadIdx.x), team = kSolo ? int(threadIdx.x >> 5) : 0, dim = g.dim;
    const float over = 1.f / float(dim);
    const int64_t end = min64(g.rows, (int64_t(blockIdx.x) + 1) * g.rows_per_cta);
    extern __shared__ float4 dynamic4[];             // the vectors, then a gate per team
    const Kept<kClass> kept{dynamic4}, gates{dynamic4 + ((g.layer ? 4 : 2) + team) * 2 * team_size<kClass>()};
    auto keep = [&](const Kept<kClass>& to, int which, const float* v) {
#pragma unroll
        for (int c = 0; c < kC; ++c) {
            f32x2 x[4];
            per_column<kClass, kWide>(v, t + 32 * c, dim, 0.f, x);
            to.put(which, t + 32 * c, x);
        }
    };
    // v without its mean (layer norm), times 1 / sqrt(mean square + eps) * w + b
    auto norm = [&](f32x2 (&v)[kC][4], int weight, int bias) {
        float s[1] = {0.f};
        if (g.layer) {
#pragma unroll
            for (int c = 0; c < kC; ++c) s[0] += sum8(v[c]);
            sum(s);
#pragma unroll
            for (int c = 0; c < kC; ++c) Stream::centre(v[c], s[0] * over, t + 32 * c, dim);
        }
        s[0] = 0.f;
#pragma unroll
        for (int c = 0; c < kC; ++c) s[0] += !kWide || (t + 32 * c) * kJoinCols < dim ? dot8(v[c], v[c]) : 0.f;
        sum(s);
        const f32x2 k = splat2(rsqrtf(s[0] * over + g.eps));
#pragma unroll
        for (int c = 0; c < kC; ++c) {
            f32x2 w[4];
            kept.get(weight, t + 32 * c, w);
#pragma unroll
            for (int j = 0; j < 4; ++j) v[c][j] = mul2(mul2(v[c][j], k), w[j]);
            if (g.layer) {
                kept.get(bias, t + 32 * c, w);
#pragma unroll
                for (int j = 0; j < 4; ++j) v[c][j] = add2(v[c][j], w[j]);
            }
        }
    };
    Stream next_x[kC];
    Branch next_f[kC];
    auto fetch = [&](int64_t row) {
        if (row < end)
#pragma unroll
            for (int c = 0; c < kC; ++c) {
                next_f[c].load(g.f + row * g.f_step, t + 32 * c, dim);
                if (g.x) next_x[c].load(g.x + row * g.x_step, t + 32 * c, dim);
            }
    };
#pragma unroll
    for (int c = 0; c < kC; ++c) next_x[c].clear();
    int64_t row = int64_t(blockIdx.x) * g.rows_per_cta + team, gate_row = 0;       // gate_row: the first that the kept gate is not for
    fetch(row);
    if (team == 0) {
        keep(kept, kVPreW, g.pre_w);
        if (g.post_w) keep(kept, kVPostW, g.post_w);
        if (g.layer) {
            keep(kept, kVPreB, g.pre_b);
            if (g.post_w) keep(kept, kVPostB, g.post_b);
        }
    }
    if (g.gate && !g.rows_per_gate) {
        keep(gates, 0, g.gate);
        gate_row = g.rows;
    }
    if (kSolo) __syncthreads();
    const f32x2 scale = splat2(g.scale);
    for (; row < end; row += kTeams) {               // (alike in a team)
        f32x2 x[kC][4], u[kC][4];
#pragma unroll
        for (int c = 0; c < kC; ++c) {
            next_x[c].get(x[c]);
            next_f[c].get(u[c]);
        }
        fetch(row + kTeams);                         // (the next row is on its way while this one is reduced)
        if (g.post_w) norm(u, kVPostW, kVPostB);
        if (g.gate) {
            if (row >= gate_row) {
                const int64_t group = uint32_t(row) / uint32_t(g.rows_per_gate);
                gate_row = (group + 1) * g.rows_per_gate;
                keep(gates, 0, g.gate + group * dim);
            }
#pragma unroll
            for (int c = 0; c < kC; ++c) {
                f32x2 w[4];
                gates.get(0, t + 32 * c, w);
#pragma unroll
                for (int j = 0; j < 4; ++j) u[c][j] = mul2(w[j], u[c][j]);
            }
        }
#pragma unroll
        for (int c = 0; c < kC; ++c) {
#pragma unroll
            for (int j = 0; j < 4; ++j) u[c][j] = fma2(scale, x[c][j], u[c][j]);
            Stream::store(g.y + row * g.y_step, t + 32 * c, dim, u[c]);
        }
        norm(u, kVPreW, kVPreB);
#pragma unroll
        for (int c = 0; c < kC; ++c) Branch::store(g.h + row * g.h_step, t + 32 * c, dim, u[c]);
    }
}

// ---- gradient ---------------------------------------------------------------------------------------------------
enum Sum : int { kPreW = 0, kPostW = 1, kGate = 2, kPreB = 3, kPostB = 4 };
// What is summed row by row.  A gate is the same for all rows of its group, so its gradient and those of post's weight and bias follow
// from two sums a column at the group's end: with A = sum of Dy n(f) and B = sum of Dy, dgate = w A + b B, dw = g A, db = g B.  (Without
// post A is the sum of Dy f, and dgate.)
enum Running : int { kDhN = 0, kDyN = 1, kDh = 2, kDy = 3 };

struct JoinGradArgs {
    const char *y, *f, *dy, *dh;
    char *dx, *df;
    const float *post_w, *post_b, *gate, *pre_w;
    char* out[kJoinSums];          // the sums' destinations; null: not wanted
    float* part;                   // [CTA][kJoinSums + 1][dim]; a gate per group: slots kGate and kJoinSums, see below
    int64_t y_step, f_step, dy_step, dh_step, dx_step, df_step, rows, rows_per_gate, rows_per_cta;
    int dim, grad_dtype;
    float scale, eps;
};

__device__ __forceinline__ void store_grad(char* out, int dtype, int64_t i, float v) {
    if (dtype == BAOC_F32) {
        reinterpret_cast<float*>(out)[i] = v;
    } else {
        uint16_t h;
        asm("cvt.rn.bf16.f32 %0, %1;" : "=h"(h) : "f"(v));
        reinterpret_cast<uint16_t*>(out)[i] = h;
    }
}

// A CTA takes rows_per_cta rows in order.  A gate per group: its sums are handed out at the end of every group.  A group whose
// rows all belong to this CTA is finished here; of the others a CTA has two at most, the one its first row is in (slot kGate)
// and the one its last row is in (slot kJoinSums).
template <int S, int B, bool kLayer, int kClass, bool kWide>
__global__ void __launch_bounds__(class_threads(kClass), class_blocks(kClass, class_grad_warps(kClass))) join_grad_kernel(const JoinGradArgs g BAOC_CHECK_PARAM) {
    constexpr bool kSolo = solo(kClass);
    constexpr int kTeams = kSolo ? kSoloWarps : 1, kC = chunks_of(kClass), kSums = kLayer ? 4 : 2;
    // The sums lie in shared memory where the registers have a row of several chunks, or are few (65536 x 512 bf16 layer norms with a
    // gate: 109 us against 126 in registers, 95 with what came later), else in registers (65536 x 256 bf16 layer norms: 56 us, in shared memory 68).
    constexpr bool kShared = kClass == 2 || kClass == 3 || kClass == 6;
    constexpr bool kAhead = kClass == 4 || kClass == 5;      // the next row is fetched into registers,
    constexpr bool kStaged = (kSolo || kClass == 6) && kWide && S == BAOC_BF16 && B == BAOC_BF16;     // or into shared memory (16 bytes a thread and array)
    // Kept vectors: the weights and the gate (of a segment); pre's weight alone where shared memory has no room for all of them, the sums and a
    // staged row (8192 x 8192 bf16 layer norms: 312 us, 357 with the vectors and no staged row).
    constexpr int kVectors = kClass == 6 && kLayer ? 1 : 3;
    using Stream = RowPart<S, kClass, kWide>;
    using Branch = RowPart<B, kClass, kWide>;
    extern __shared__ float4 dynamic4[];             // the vectors; kShared or kSolo: the sums, [team][sum][2][team's threads]; kStaged: a row per team
    __shared__ float4 buf[kSolo ? 1 : 2][32];
    TeamSum<kClass> sum{buf};
    begin_in_row();
    const int size = team_size<kClass>(), t = kSolo ? int(threadIdx.x & 31) : int(threadIdx.x), team = kSolo ? int(threadIdx.x >> 5) : 0, dim = g.dim;
    const Kept<kClass> kept{dynamic4};
    float4* sums = dynamic4 + kVectors * 2 * size;
    const float over = 1.f / float(dim);
    const int64_t begin = int64_t(blockIdx.x) * g.rows_per_cta, end = min64(g.rows, begin + g.rows_per_cta);
    float* part = g.part + int64_t(blockIdx.x) * (kJoinSums + 1) * dim;
#ifdef BAOC_CHECKED
    if (!check_range(ck, kKerJoinGrad, part, int64_t(kJoinSums + 1) * dim * 4, 0)) return;
#endif
    const bool need_f = g.post_w || g.gate;
    f32x2 acc[kShared ? 1 : kSums][4] = {};
    // a * b to the sums k of a thread's columns
    auto add = [&](int k, int c, const f32x2 (&a)[4], const f32x2 (&b)[4]) {
        if constexpr (kShared) {
            float4* p = sums + (team * kSums + k) * 2 * size + t + 32 * c;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                float4 v = p[h * size];
                unpack2(fma2(a[2 * h], b[2 * h], pack2(v.x, v.y)), v.x, v.y);
                unpack2(fma2(a[2 * h + 1], b[2 * h + 1], pack2(v.z, v.w)), v.z, v.w);
                p[h * size] = v;
            }
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[k][j] = fma2(a[j], b[j], acc[k][j]);
        }
    };
    auto zero = [&](int k) {
#pragma unroll
        for (int c = 0; c < kC; ++c) {
            if constexpr (kShared) {
                float4* p = sums + (team * kSums + k) * 2 * size + t + 32 * c;
                p[0] = p[size] = make_float4(0.f, 0.f, 0.f, 0.f);
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[k][j] = 0;
            }
        }
    };
    // At a group's end and a CTA's: the sums of all teams, each column's in one thread (half_sum, over `places`), behind a barrier that
    // follows what the teams have added and publish() of sums in registers.
    auto publish = [&](auto which) {
        if constexpr (kSolo && !kShared) {
            constexpr int k = decltype(which)::value;
            float v[8];
#pragma unroll
            for (int j = 0; j < 4; ++j) unpack2(acc[k][j], v[2 * j], v[2 * j + 1]);
            float4* p = sums + (team * kSums + k) * 2 * size + t;
            p[0] = make_float4(v[0], v[1], v[2], v[3]);
            p[size] = make_float4(v[4], v[5], v[6], v[7]);
        }
    };
    // (four neighbours in one access where that can be: one by one, a CTA's sums of 768 columns took as long as a row)
    auto store4 = [&](char* to, int dtype, int of, int j, float4 v, bool add) {        // columns j to j + 3 of place `of`
        if (kWide && dtype == BAOC_F32 && (reinterpret_cast<uintptr_t>(to) & 15) == 0) {
            if (Stream::column(of, j) >= dim) return;
            float4* p = reinterpret_cast<float4*>(to + 4 * Stream::column(of, j));
            if (add) { const float4 o = *p; v.x += o.x; v.y += o.y; v.z += o.z; v.w += o.w; }
            *p = v;
            return;
        }
        const float x[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int c = Stream::column(of, j + i);
            if (c < dim) store_grad(to, dtype, c, add ? reinterpret_cast<const float*>(to)[c] + x[i] : x[i]);      // (add: fp32)
        }
    };
    auto half_sum = [&](auto which, int i) {         // sum `which`, float4 i of its 2 * size
        constexpr int k = decltype(which)::value;
        float4 v;
        if constexpr (kSolo || kShared) {
            v = sums[k * 2 * size + i];
            for (int o = 1; o < kTeams; ++o) {
                const float4 w = sums[(o * kSums + k) * 2 * size + i];
                v.x += w.x; v.y += w.y; v.z += w.z; v.w += w.w;
            }
        } else {
            const int j = i == t ? 0 : 2;
            unpack2(j ? acc[k][2] : acc[k][0], v.x, v.y);
            unpack2(j ? acc[k][3] : acc[k][1], v.z, v.w);
        }
        return v;
    };
    auto places = [&](auto f) {                      // f(i) for this thread's share of the 2 * size
        if constexpr (kSolo) {
            for (int i = int(threadIdx.x); i < 2 * size; i += int(blockDim.x)) f(i);
        } else {
            f(t);
            f(size + t);
        }
    };
    auto columns_of = [&](const float* v, int i) {
        auto one = [&](int e) {
            const int c = Stream::column(i % size, 4 * (i / size) + e);
            return v && c < dim ? __ldg(v + c) : 0.f;
        };
        return make_float4(one(0), one(1), one(2), one(3));
    };
    auto four_of = [&](int which, const float* v, int i) { return which < kVectors ? kept.at[which * 2 * size + i] : columns_of(v, i); };
    auto times = [](float4 a, float4 b) { return make_float4(a.x * b.x, a.y * b.y, a.z * b.z, a.w * b.w); };
    auto plus = [](float4 a, float4 b) { return make_float4(a.x + b.x, a.y + b.y, a.z + b.z, a.w + b.w); };
    auto in = [&](int c) { return !kWide || (t + 32 * c) * kJoinCols < dim; };
    auto keep = [&](int which, const float* v) {
#pragma unroll
        for (int c = 0; c < kC; ++c) {
            f32x2 x[4];
            per_column<kClass, kWide>(v, t + 32 * c, dim, 0.f, x);
            kept.put(which, t + 32 * c, x);
        }
    };
    auto vector = [&](int which, const float* v, int c, f32x2 (&x)[4]) {
        if (which < kVectors) kept.get(which, t + 32 * c, x);
        else per_column<kClass, kWide>(v, t + 32 * c, dim, 0.f, x);
    };
    Stream next_y[kC], next_dy[kC];
    Branch next_f[kC], next_dh[kC];
    auto fetch = [&](int64_t row) {
        if (row < end)
#pragma unroll
            for (int c = 0; c < kC; ++c) {
                next_y[c].load(g.y + row * g.y_step, t + 32 * c, dim);
                next_dh[c].load(g.dh + row * g.dh_step, t + 32 * c, dim);
                if (g.dy) next_dy[c].load(g.dy + row * g.dy_step, t + 32 * c, dim);
                if (need_f) next_f[c].load(g.f + row * g.f_step, t + 32 * c, dim);
            }
    };
    // The staged row: y, dy, dh, f.  What a thread has taken may be overwritten once it has gone into something that is done before
    // the request: y, dh and f into the row's sums, dy into a store of dx or df (see below), which is why it is requested later.
    const uint32_t ahead = smem_addr(sums + kTeams * kSums * 2 * size) + team * 4 * 16 * size;
    const uint32_t at_dy = ahead + 16 * size, at_dh = ahead + 32 * size, at_f = ahead + 48 * size;
    auto request = [&](int64_t row) {
        (void)at_f;
        if (row < end)
#pragma unroll
            for (int c = 0; c < kC; ++c) {
                if (!in(c)) continue;
                Stream::request(ahead, g.y + row * g.y_step, t + 32 * c);
                Branch::request(at_dh, g.dh + row * g.dh_step, t + 32 * c);
                if (need_f) Branch::request(at_f, g.f + row * g.f_step, t + 32 * c);
            }
        cp_async_commit();
    };
    auto request_dy = [&](int64_t row) {
        (void)at_dy;
        if (!g.dy) return;
        if (row < end)
#pragma unroll
            for (int c = 0; c < kC; ++c)
                if (in(c)) Stream::request(at_dy, g.dy + row * g.dy_step, t + 32 * c);
        cp_async_commit();
    };
#pragma unroll
    for (int c = 0; c < kC; ++c) {
        next_y[c].clear();
        next_dh[c].clear();
        next_dy[c].clear();
        next_f[c].clear();
    }
    int64_t row = begin + team;
    if constexpr (kStaged) {
        request(row);
        request_dy(row);
    } else {
        fetch(row);
    }
    if (team == 0) {
        keep(kVPreW, g.pre_w);
        if (kVectors == 3 && g.post_w) keep(kVPostW, g.post_w);
        if (kVectors == 3 && g.gate && !g.rows_per_gate) keep(kVGate, g.gate);
    }
    if constexpr (kShared)
        for (int k = 0; k < kSums; ++k) zero(k);
    if (kSolo) __syncthreads();
    const f32x2 ones[4] = {splat2(1.f), splat2(1.f), splat2(1.f), splat2(1.f)};
    for (int64_t seg = begin; seg < end;) {
        const int64_t group = g.rows_per_gate ? seg / g.rows_per_gate : 0;
        const int64_t seg_end = g.rows_per_gate ? min64(end, (group + 1) * g.rows_per_gate) : end;
        const float* gate = g.gate ? g.gate + group * dim : nullptr;
        if (kVectors == 3 && g.rows_per_gate) {
            if (kSolo) __syncthreads();              // (no warp reads the last group's any more)
            if (team == 0) keep(kVGate, gate);
            if (kSolo) __syncthreads();
        }
        for (; row < seg_end; row += kTeams) {       // (alike in a team)
            f32x2 y[kC][4], d[kC][4], f[kC][4], dy[kC][4];       // d: from dh to Dy
            if constexpr (kStaged) {
                cp_async_wait<0>();
#pragma unroll
                for (int c = 0; c < kC; ++c) {
                    if (!in(c)) continue;
                    next_y[c].take(ahead, t + 32 * c);
                    if (g.dy) next_dy[c].take(at_dy, t + 32 * c);
                    next_dh[c].take(at_dh, t + 32 * c);
                    if (need_f) next_f[c].take(at_f, t + 32 * c);
                }
            }
#pragma unroll
            for (int c = 0; c < kC; ++c) {
                next_y[c].get(y[c]);
                next_dh[c].get(d[c]);
                next_f[c].get(f[c]);
                next_dy[c].get(dy[c]);
            }
            if (kAhead) fetch(row + kTeams);
            if constexpr (kLayer) {
                float s[2] = {0.f, 0.f};
#pragma unroll
                for (int c = 0; c < kC; ++c) {
                    s[0] += sum8(y[c]);
                    s[1] += sum8(f[c]);
                }
                sum(s);
#pragma unroll
                for (int c = 0; c < kC; ++c) {
                    Stream::centre(y[c], s[0] * over, t + 32 * c, dim);
                    if (g.post_w) Stream::centre(f[c], s[1] * over, t + 32 * c, dim);        // (post(f) is f itself without a norm)
                }
            }
            float r_f;
            {
                float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int c = 0; c < kC; ++c) {
                    f32x2 w[4];
                    vector(kVPreW, g.pre_w, c, w);
#pragma unroll
                    for (int j = 0; j < 4; ++j) w[j] = mul2(d[c][j], w[j]);
                    s[0] += in(c) ? dot8(y[c], y[c]) : 0.f;
                    s[1] += in(c) ? dot8(f[c], f[c]) : 0.f;
                    s[2] += dot8(w, y[c]);
                    if (kLayer) s[3] += sum8(w);
                }
                sum(s);
                if constexpr (kStaged) request(row + kTeams);       // (the sums are made of all of y, dh and f: their places are free)
                const float r_y = rsqrtf(s[0] * over + g.eps);
                r_f = rsqrtf(s[1] * over + g.eps);
                const f32x2 r2 = splat2(r_y), slope = splat2(-r_y * r_y * s[2] * over), mean = splat2(-s[3] * over);
#pragma unroll
                for (int c = 0; c < kC; ++c) {
                    f32x2 w[4], n[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) n[j] = mul2(y[c][j], r2);
                    add(kDhN, c, d[c], n);
                    if (kLayer) add(kDh, c, d[c], ones);
                    vector(kVPreW, g.pre_w, c, w);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const f32x2 dn = mul2(d[c][j], w[j]);
                        d[c][j] = fma2(r2, kLayer ? add2(fma2(y[c][j], slope, dn), mean) : fma2(y[c][j], slope, dn), dy[c][j]);
                    }
                }
            }
            if (g.dx) {
                const f32x2 scale = splat2(g.scale);
#pragma unroll
                for (int c = 0; c < kC; ++c) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) dy[c][j] = mul2(scale, d[c][j]);
                    Stream::store(g.dx + row * g.dx_step, t + 32 * c, dim, dy[c]);
                }
                if constexpr (kStaged) request_dy(row + kTeams);    // (dy has left in dx)
            }
            if (g.post_w) {
                const f32x2 r2 = splat2(r_f);
                float s[2] = {0.f, 0.f};
#pragma unroll
                for (int c = 0; c < kC; ++c) {
                    f32x2 w[4], b[4];
                    vector(kVPostW, g.post_w, c, w);
#pragma unroll
                    for (int j = 0; j < 4; ++j) f[c][j] = mul2(f[c][j], r2);
                    add(kDyN, c, d[c], f[c]);
                    if (kLayer) add(kDy, c, d[c], ones);
                    if (gate) {
                        vector(kVGate, gate, c, b);
#pragma unroll
                        for (int j = 0; j < 4; ++j) d[c][j] = mul2(d[c][j], b[j]);
                    }
#pragma unroll
                    for (int j = 0; j < 4; ++j) d[c][j] = mul2(d[c][j], w[j]);
                    s[0] += dot8(d[c], f[c]);
                    if (kLayer) s[1] += sum8(d[c]);
                }
                sum(s);
                const f32x2 slope = splat2(-s[0] * over), mean = splat2(-s[1] * over);
#pragma unroll
                for (int c = 0; c < kC; ++c)
#pragma unroll
                    for (int j = 0; j < 4; ++j) d[c][j] = mul2(r2, kLayer ? add2(fma2(f[c][j], slope, d[c][j]), mean) : fma2(f[c][j], slope, d[c][j]));
            } else if (gate) {
#pragma unroll
                for (int c = 0; c < kC; ++c) {
                    f32x2 w[4];
                    vector(kVGate, gate, c, w);
                    add(kDyN, c, d[c], f[c]);
#pragma unroll
                    for (int j = 0; j < 4; ++j) d[c][j] = mul2(d[c][j], w[j]);
                }
            }
#pragma unroll
            for (int c = 0; c < kC; ++c) Branch::store(g.df + row * g.df_step, t + 32 * c, dim, d[c]);
            if constexpr (kStaged)
                if (!g.dx) request_dy(row + kTeams);                // (without dx it has left in df)
            if (!kAhead && !kStaged) fetch(row + kTeams);
        }
        if (g.out[kGate] || g.out[kPostW] || g.out[kPostB]) {
            const bool whole = g.rows_per_gate && group * g.rows_per_gate >= begin && min64(g.rows, (group + 1) * g.rows_per_gate) <= end;
            float* slot = part + int64_t(!g.rows_per_gate || group == begin / g.rows_per_gate ? kGate : kJoinSums) * dim;
            publish(std::integral_constant<int, kDyN>{});
            if constexpr (kLayer) publish(std::integral_constant<int, kDy>{});
            if (kSolo) __syncthreads();
            places([&](int i) {
                float4 a = half_sum(std::integral_constant<int, kDyN>{}, i), b = make_float4(0.f, 0.f, 0.f, 0.f);
                if constexpr (kLayer) b = half_sum(std::integral_constant<int, kDy>{}, i);
                const int of = i % size, j = 4 * (i / size);
                if (g.out[kGate]) {
                    float4 v = a;
                    if (g.post_w) v = times(v, four_of(kVPostW, g.post_w, i));
                    if (kLayer && g.post_w) v = plus(v, times(b, columns_of(g.post_b, i)));
                    if (whole) store4(g.out[kGate] + group * dim * (g.grad_dtype == BAOC_F32 ? 4 : 2), g.grad_dtype, of, j, v, false);
                    else store4(reinterpret_cast<char*>(slot), BAOC_F32, of, j, v, false);
                }
                if (gate) {
                    const float4 w = four_of(kVGate, gate, i);
                    a = times(a, w);
                    b = times(b, w);
                }
                if (g.out[kPostW]) store4(reinterpret_cast<char*>(part + int64_t(kPostW) * dim), BAOC_F32, of, j, a, seg != begin);
                if (kLayer && g.out[kPostB]) store4(reinterpret_cast<char*>(part + int64_t(kPostB) * dim), BAOC_F32, of, j, b, seg != begin);
            });
            if (kSolo) __syncthreads();
            zero(kDyN);
            if constexpr (kLayer) zero(kDy);
        }
        seg = seg_end;
    }
    publish(std::integral_constant<int, kDhN>{});
    if constexpr (kLayer) publish(std::integral_constant<int, kDh>{});
    if (kSolo) __syncthreads();
    places([&](int i) {
        const int of = i % size, j = 4 * (i / size);
        if (g.out[kPreW]) store4(reinterpret_cast<char*>(part + int64_t(kPreW) * dim), BAOC_F32, of, j, half_sum(std::integral_constant<int, kDhN>{}, i), false);
        if constexpr (kLayer)
            if (g.out[kPreB]) store4(reinterpret_cast<char*>(part + int64_t(kPreB) * dim), BAOC_F32, of, j, half_sum(std::integral_constant<int, kDh>{}, i), false);
    });
}

// The CTAs' sums, 32 columns per CTA: every warp adds each 32nd CTA's, then the warps' sums are added in order.
// blockIdx.y: which sum; from kJoinSums on, groups of a gate that several CTAs have rows of.
__global__ void __launch_bounds__(1024) join_sums_kernel(const JoinGradArgs g, int ctas, int64_t groups BAOC_CHECK_PARAM) {
    __shared__ float sh[32][33];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int col = int(blockIdx.x) * 32 + lane;
    begin_in_row();
    auto total = [&](int64_t c0, int64_t c1, int64_t group, int k, int64_t at) {
        float s = 0.f;
#ifdef BAOC_CHECKED
        if (c0 <= c1 && !check_range(ck, kKerJoinGrad, g.part + c0 * (kJoinSums + 1) * g.dim, 4 * (c1 - c0 + 1) * (kJoinSums + 1) * g.dim, 1)) return;
#endif
        if (col < g.dim)
#pragma unroll 8
            for (int64_t c = c0 + warp; c <= c1; c += 32) {
                const int slot = group < 0 || group == c * g.rows_per_cta / g.rows_per_gate ? k : kJoinSums;
                s += g.part[(c * (kJoinSums + 1) + slot) * g.dim + col];
            }
        sh[warp][lane] = s;
        __syncthreads();
        if (warp == 0 && col < g.dim) {
            for (int w = 1; w < 32; ++w) s += sh[w][lane];
            store_grad(g.out[k], g.grad_dtype, at + col, s);
        }
        __syncthreads();
    };
    const int k = int(blockIdx.y);
    if (k < kJoinSums) {
        if (!g.out[k] || (k == kGate && g.rows_per_gate)) return;
        total(0, ctas - 1, -1, k, 0);
        return;
    }
    for (int64_t group = k - kJoinSums; group < groups; group += gridDim.y - kJoinSums) {
        const int64_t c0 = group * g.rows_per_gate / g.rows_per_cta, c1 = (min64(g.rows, (group + 1) * g.rows_per_gate) - 1) / g.rows_per_cta;
        if (c0 == c1) continue;                  // (that CTA has written it)
        total(c0, c1, group, kGate, group * g.dim);
    }
}

namespace {

thread_local std::string g_join_err;

int fail_join(int code, const std::string& msg) {
    g_join_err = msg;
    return code;
}
int64_t elem_bytes(int dtype) { return dtype == BAOC_F32 ? 4 : 2; }
bool aligned(const void* p, int64_t bytes) { return (reinterpret_cast<uintptr_t>(p) & uintptr_t(bytes - 1)) == 0; }

int check_join(const baoc_join_t* e, int64_t rows, const std::string& what) {
    if (!e) return fail_join(BAOC_E_INVALID, what + ": null descriptor");
    if (e->dim < 1 || e->dim > kJoinMaxDim) return fail_join(BAOC_E_INVALID, what + ": dim must be in 1 .. 8192");
    if (e->kind != BAOC_NORM_RMS && e->kind != BAOC_NORM_LAYER) return fail_join(BAOC_E_INVALID, what + ": kind must be BAOC_NORM_RMS or BAOC_NORM_LAYER");
    for (int t : {e->stream_dtype, e->branch_dtype, e->grad_dtype})
        if (t != BAOC_BF16 && t != BAOC_F32) return fail_join(BAOC_E_INVALID, what + ": dtypes must be BAOC_BF16 or BAOC_F32");
    if (e->stream_dtype == BAOC_BF16 && e->branch_dtype == BAOC_F32) return fail_join(BAOC_E_INVALID, what + ": an fp32 branch needs an fp32 stream");
    if (!std::isfinite(e->scale)) return fail_join(BAOC_E_INVALID, what + ": scale must be finite");
    if (!std::isfinite(e->eps) || !(e->eps > 0.f)) return fail_join(BAOC_E_INVALID, what + ": eps must be finite and above zero");
    if (e->rows_per_gate < 0) return fail_join(BAOC_E_INVALID, what + ": rows_per_gate must not be negative");
    for (int64_t s : {e->x_stride, e->f_stride, e->y_stride, e->h_stride})
        if (s && (s < e->dim || s > kJoinMaxStride)) return fail_join(BAOC_E_INVALID, what + ": a row stride must be 0 or in dim .. 2^28");
    if (rows < 0 || rows > (int64_t(1) << 31)) return fail_join(BAOC_E_INVALID, what + ": rows must be in 0 .. 2^31");
    return BAOC_OK;
}

// An array of rows (or a vector per column: one row) as the kernels see it.
struct Rows {
    const void* p;
    int64_t step, width, eb, n;     // bytes from row to row, of a row, of an element; rows
    Rows(const void* p, int64_t stride, int dtype, int dim, int64_t n)
        : p(p), step((stride ? stride : dim) * elem_bytes(dtype)), width(dim * elem_bytes(dtype)), eb(elem_bytes(dtype)), n(n) {}
    bool wide() const { return !p || (aligned(p, kJoinCols * eb) && step % (kJoinCols * eb) == 0); }     // a thread's columns in one access
    bool fits() const { return aligned(p, eb); }
};
// Whether the rows of two arrays share bytes.  (Rows of one buffer may lie between each other's.)
bool overlap(const Rows& a, const Rows& b) {
    if (!a.p || !b.p || a.n == 0 || b.n == 0) return false;
    const char *x = static_cast<const char*>(a.p), *y = static_cast<const char*>(b.p);
    if (x >= y + (b.n - 1) * b.step + b.width || y >= x + (a.n - 1) * a.step + a.width) return false;
    if (a.step != b.step) return true;
    const int64_t off = ((y - x) % a.step + a.step) % a.step;
    return off < a.width || off + b.width > a.step;
}
bool same(const Rows& a, const Rows& b) { return a.p == b.p && a.width == b.width && (a.step == b.step || a.n == 1); }
// An output, and the input that it may be (null: none).
struct Written {
    const Rows* out;
    const Rows* instead_of;
};
// Whether an output shares bytes with an input or another output in a way that is not allowed.
template <int kOuts, int kIns>
bool collide(const Written (&outs)[kOuts], const Rows* const (&ins)[kIns]) {
    for (int i = 0; i < kOuts; ++i) {
        for (const Rows* in : ins)
            if (overlap(*outs[i].out, *in) && !(in == outs[i].instead_of && same(*outs[i].out, *in))) return true;
        for (int j = 0; j < i; ++j)
            if (overlap(*outs[i].out, *outs[j].out)) return true;
    }
    return false;
}
int64_t gates_of(int64_t rows, int64_t rows_per_gate) { return rows_per_gate > 0 && rows_per_gate < rows ? ceil_div(rows, rows_per_gate) : 1; }

// How rows are spread over threads: their class, and what follows from it.  alone: a warp may take a row of 2 or 3 times 256 columns alone.
struct Spread {
    int c, cta, team, rows;         // class, threads of a CTA, columns' threads of a team (see team_size), rows that a CTA works on at a time
    Spread(int dim, int64_t n_rows, bool alone) {
        const int w = int(ceil_div(dim, 32 * kJoinCols));
        c = w == 1 || (w <= 3 && alone && n_rows > kFewRows) ? w : (w <= 8 ? 4 : (w <= 16 ? 5 : 6));
        cta = solo(c) ? 32 * kSoloWarps : 32 * w;
        team = solo(c) ? 32 * c : cta;
        rows = solo(c) ? kSoloWarps : 1;
    }
    int64_t at_once(int sm_warps) const { return int64_t(148) * std::max(1, sm_warps * 32 / cta); }     // CTAs that find room, sm_warps per SM
};

// f(class, wide) as constants.
template <int kClass, typename F>
int with_width(bool wide, F f) {
    std::integral_constant<int, kClass> c{};
    return wide ? f(c, std::true_type{}) : f(c, std::false_type{});
}
template <typename F>
int with_class(int c, bool wide, F f) {
    switch (c) {
        case 1: return with_width<1>(wide, f);
        case 2: return with_width<2>(wide, f);
        case 3: return with_width<3>(wide, f);
        case 4: return with_width<4>(wide, f);
        case 5: return with_width<5>(wide, f);
        default: return with_width<6>(wide, f);
    }
}
template <typename F>
int with_types(int stream, int branch, F f) {
    using std::integral_constant;
    if (stream == BAOC_BF16) return f(integral_constant<int, BAOC_BF16>{}, integral_constant<int, BAOC_BF16>{});
    return branch == BAOC_BF16 ? f(integral_constant<int, BAOC_F32>{}, integral_constant<int, BAOC_BF16>{})
                               : f(integral_constant<int, BAOC_F32>{}, integral_constant<int, BAOC_F32>{});
}

// The gradient's rows per CTA and CTAs: whole rounds of a CTA's teams, all CTAs at once.
void grad_shape(const Spread& d, int64_t rows, int64_t* per_cta, int* ctas) {
    *per_cta = std::max<int64_t>(d.rows, round_up(ceil_div(rows, d.at_once(class_grad_warps(d.c))), d.rows));
    *ctas = int(ceil_div(rows, *per_cta));
}
// Backwards a row of the wide path is not taken alone where the stream is fp32: its lanes' loads fill their sectors as they are, and a
// CTA's sums stay in registers (65536 x 768: 158 -> 152 us, 64 gates of 1024 x 640: 166 -> 148; bf16 streams 144 -> 166, rows
// element by element 302 -> 359 at 513 columns).
constexpr bool grad_alone(int stream, bool wide) { return !wide || stream == BAOC_BF16; }
// (By the most CTAs that so many rows or fewer can get in any type: whole rounds leave fewer of them for some larger numbers of rows.)
int64_t grad_ws(int dim, int64_t rows) {
    int64_t ctas = 0;
    for (bool alone : {true, false}) {
        const Spread d(dim, rows, alone);
        ctas = std::max(ctas, std::min(ceil_div(rows, d.rows), d.at_once(class_grad_warps(d.c))));
    }
    return std::max<int64_t>(256, round_up(ctas * (kJoinSums + 1) * dim * 4, 256));
}

int launched(cudaError_t ce, const char* kernel) {
    return ce == cudaSuccess ? BAOC_OK : fail_join(BAOC_E_CUDA, std::string(kernel) + ": " + cudaGetErrorString(ce));
}

}  // namespace

BAOC_DEFINE_CHECK_FETCH(join_check_fetch)

}  // namespace baoc

using namespace baoc;

extern "C" {

const char* baoc_join_last_error(void) { return g_join_err.c_str(); }

int baoc_join(const baoc_join_t* e, const void* x, const void* f, const float* post_w, const float* post_b, const float* gate,
              const float* pre_w, const float* pre_b, int64_t rows, void* y, void* h, baoc_stream_t stream) try {
    const int rc = check_join(e, rows, "baoc_join");
    if (rc) return rc;
    if (rows == 0) return BAOC_OK;
    if (!f || !pre_w || !y || !h) return fail_join(BAOC_E_INVALID, "baoc_join: null pointer");
    if ((post_b && !post_w) || (e->kind == BAOC_NORM_RMS && (post_b || pre_b))) return fail_join(BAOC_E_INVALID, "baoc_join: biases belong to layer norms");
    const Rows rx(x, e->x_stride, e->stream_dtype, e->dim, rows), rf(f, e->f_stride, e->branch_dtype, e->dim, rows), ry(y, e->y_stride, e->stream_dtype, e->dim, rows),
        rh(h, e->h_stride, e->branch_dtype, e->dim, rows);
    auto vector = [&](const float* p) { return Rows(p, 0, BAOC_F32, e->dim, 1); };
    const Rows rpost_w = vector(post_w), rpost_b = vector(post_b), rpre_w = vector(pre_w), rpre_b = vector(pre_b), rgate(gate, 0, BAOC_F32, e->dim, gates_of(rows, e->rows_per_gate));
    bool wide = e->dim % kJoinCols == 0;
    for (const Rows* r : {&rx, &rf, &ry, &rh}) {
        if (!r->fits()) return fail_join(BAOC_E_ALIGN, "baoc_join: a pointer is not aligned to its elements");
        wide = wide && r->wide();
    }
    for (const Rows* r : {&rpost_w, &rpost_b, &rgate, &rpre_w, &rpre_b}) {
        if (!r->fits()) return fail_join(BAOC_E_ALIGN, "baoc_join: a pointer is not aligned to its elements");
        wide = wide && aligned(r->p, 16);
    }
    if (collide({{&ry, &rx}, {&rh, &rf}}, {&rx, &rf, &rpost_w, &rpost_b, &rgate, &rpre_w, &rpre_b}))
        return fail_join(BAOC_E_INVALID, "baoc_join: y may be x and h may be f; outputs overlap nothing else");
    JoinArgs a{static_cast<const char*>(x), static_cast<const char*>(f), static_cast<char*>(y), static_cast<char*>(h), post_w, post_b, gate, pre_w, pre_b,
                     rx.step, rf.step, ry.step, rh.step, rows, e->rows_per_gate < rows ? e->rows_per_gate : 0, 0, e->dim, e->kind == BAOC_NORM_LAYER, e->scale, e->eps};
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    return with_types(e->stream_dtype, e->branch_dtype, [&](auto S, auto B) {
        const Spread d(e->dim, rows, true);
        return with_class(d.c, wide, [&](auto C, auto W) {
            const int bytes = ((a.layer ? 4 : 2) + d.rows) * 8 * d.team * 4;
            a.rows_per_cta = round_up(ceil_div(rows, d.at_once(class_warps(C()))), d.rows);      // all CTAs at once
            auto kernel = join_kernel<S(), B(), C(), W()>;
            if (bytes > 40 * 1024) {             // (48 KB go without asking, the kernel's own arrays included)
                const cudaError_t ce = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
                if (ce != cudaSuccess) return launched(ce, "join_kernel");
            }
            return launched(launch_in_row(kernel, dim3(unsigned(ceil_div(rows, a.rows_per_cta))), unsigned(d.cta), size_t(bytes), 1, s, a), "join_kernel");
        });
    });
} catch (const std::bad_alloc&) {
    return BAOC_E_INVALID;
}

int baoc_join_grad_workspace_bytes(const baoc_join_t* e, int64_t rows, size_t* bytes) try {
    const int rc = check_join(e, rows, "baoc_join_grad_workspace_bytes");
    if (rc) return rc;
    if (!bytes) return fail_join(BAOC_E_INVALID, "baoc_join_grad_workspace_bytes: null pointer");
    *bytes = size_t(grad_ws(e->dim, rows));
    return BAOC_OK;
} catch (const std::bad_alloc&) {
    return BAOC_E_INVALID;
}

int baoc_join_grad(const baoc_join_t* e, const void* y, const void* f, const void* dy, const void* dh, const float* post_w, const float* post_b,
                   const float* gate, const float* pre_w, int64_t rows, void* dx, void* df, void* dpost_w, void* dpost_b, void* dgate,
                   void* dpre_w, void* dpre_b, void* ws, size_t ws_bytes, baoc_stream_t stream) try {
    const char* what = "baoc_join_grad";
    int rc = check_join(e, rows, what);
    if (rc) return rc;
    for (int64_t s : {e->dy_stride, e->dh_stride, e->dx_stride, e->df_stride})
        if (s && (s < e->dim || s > kJoinMaxStride)) return fail_join(BAOC_E_INVALID, "baoc_join_grad: a row stride must be 0 or in dim .. 2^28");
    const bool layer = e->kind == BAOC_NORM_LAYER;
    if (!pre_w || !ws || (rows && (!y || !dh || !df || ((post_w || gate) && !f)))) return fail_join(BAOC_E_INVALID, "baoc_join_grad: null pointer");
    if (((post_b || dpost_w || dpost_b) && !post_w) || (dgate && !gate) || (!layer && (post_b || dpost_b || dpre_b)))
        return fail_join(BAOC_E_INVALID, "baoc_join_grad: a bias or a gradient of something that is not there");
    const Rows ry(y, e->y_stride, e->stream_dtype, e->dim, rows), rf(post_w || gate ? f : nullptr, e->f_stride, e->branch_dtype, e->dim, rows),
        rdy(dy, e->dy_stride, e->stream_dtype, e->dim, rows), rdh(dh, e->dh_stride, e->branch_dtype, e->dim, rows), rdx(dx, e->dx_stride, e->stream_dtype, e->dim, rows),
        rdf(df, e->df_stride, e->branch_dtype, e->dim, rows);
    const int64_t gates = gates_of(rows, e->rows_per_gate);
    auto vector = [&](const void* p, int dtype) { return Rows(p, 0, dtype, e->dim, 1); };
    const Rows rpost_w = vector(post_w, BAOC_F32), rpost_b = vector(post_b, BAOC_F32), rpre_w = vector(pre_w, BAOC_F32), rgate(gate, 0, BAOC_F32, e->dim, gates),
        rdpost_w = vector(dpost_w, e->grad_dtype), rdpost_b = vector(dpost_b, e->grad_dtype), rdpre_w = vector(dpre_w, e->grad_dtype), rdpre_b = vector(dpre_b, e->grad_dtype),
        rdgate(dgate, 0, e->grad_dtype, e->dim, gates);
    bool wide = e->dim % kJoinCols == 0;
    for (const Rows* r : {&ry, &rf, &rdy, &rdh, &rdx, &rdf}) {
        if (!r->fits()) return fail_join(BAOC_E_ALIGN, "baoc_join_grad: a pointer is not aligned to its elements");
        wide = wide && r->wide();
    }
    for (const Rows* r : {&rpost_w, &rpost_b, &rgate, &rpre_w}) {
        if (!r->fits()) return fail_join(BAOC_E_ALIGN, "baoc_join_grad: a pointer is not aligned to its elements");
        wide = wide && aligned(r->p, 16);
    }
    void* outs[kJoinSums] = {};
    outs[kPreW] = dpre_w; outs[kPreB] = dpre_b; outs[kPostW] = dpost_w; outs[kPostB] = dpost_b; outs[kGate] = dgate;
    for (const Rows* r : {&rdpost_w, &rdpost_b, &rdgate, &rdpre_w, &rdpre_b})
        if (!r->fits()) return fail_join(BAOC_E_ALIGN, "baoc_join_grad: a pointer is not aligned to its elements");
    if (!aligned(ws, 256)) return fail_join(BAOC_E_ALIGN, "baoc_join_grad: workspace not 256-byte aligned");
    const int64_t need = grad_ws(e->dim, rows);
    if (ws_bytes < size_t(need)) return fail_join(BAOC_E_WORKSPACE, "baoc_join_grad: workspace too small");
    const Rows space(ws, 0, BAOC_F32, int(need / 4), 1);
    if (collide({{&rdx, &rdy}, {&rdf, &rdh}, {&rdpost_w, nullptr}, {&rdpost_b, nullptr}, {&rdgate, nullptr}, {&rdpre_w, nullptr}, {&rdpre_b, nullptr}, {&space, nullptr}},
                {&ry, &rf, &rdy, &rdh, &rpost_w, &rpost_b, &rgate, &rpre_w}))
        return fail_join(BAOC_E_INVALID, "baoc_join_grad: dx may be dy and df may be dh; outputs and the workspace overlap nothing else");
    JoinGradArgs a{static_cast<const char*>(y), static_cast<const char*>(rf.p), static_cast<const char*>(dy), static_cast<const char*>(dh), static_cast<char*>(dx),
                   static_cast<char*>(df), post_w, post_b, gate, pre_w, {}, static_cast<float*>(ws), ry.step, rf.step, rdy.step, rdh.step, rdx.step, rdf.step, rows,
                   gate && e->rows_per_gate < rows ? e->rows_per_gate : 0, 0, e->dim, e->grad_dtype, e->scale, e->eps};
    for (int k = 0; k < kJoinSums; ++k) a.out[k] = static_cast<char*>(outs[k]);
    int ctas;
    const Spread d(e->dim, rows, grad_alone(e->stream_dtype, wide));
    grad_shape(d, std::max<int64_t>(rows, 1), &a.rows_per_cta, &ctas);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const CheckCtx ck{static_cast<char*>(ws), static_cast<char*>(ws) + need, 0, 0, 0};
    (void)ck;
    if (rows) {
        rc = with_types(e->stream_dtype, e->branch_dtype, [&](auto S, auto B) {
            return with_class(d.c, wide, [&](auto C, auto W) {
                auto go = [&](auto L) {
                    const int sums = solo(C()) || C() == 6 ? d.rows * (L() ? 4 : 2) : 0;
                    const int staged = (solo(C()) || C() == 6) && W() && S() == BAOC_BF16 && B() == BAOC_BF16 ? d.rows * 4 / 2 : 0;        // four rows of 2 bytes a column, counted as vectors of 4
                    const int bytes = (sums + (C() == 6 && L() ? 1 : 3) + staged) * 8 * d.team * 4;
                    constexpr int kClass = (C() == 2 || C() == 3) && !grad_alone(S(), W()) ? 4 : C();      // (one that no call has is not made)
                    auto kernel = join_grad_kernel<S(), B(), L(), kClass, W()>;
                    if (bytes > 40 * 1024) {
                        const cudaError_t ce = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
                        if (ce != cudaSuccess) return launched(ce, "join_grad_kernel");
                    }
                    return launched(launch_in_row(kernel, dim3(unsigned(ctas)), unsigned(d.cta), size_t(bytes), 1, s, a BAOC_CHECK_ARG(ck)), "join_grad_kernel");
                };
                return layer ? go(std::true_type{}) : go(std::false_type{});
            });
        });
        if (rc) return rc;
    } else {
        ctas = 0;
    }
    bool any = false;
    for (const void* p : outs) any = any || p;
    if (!any) return BAOC_OK;
    const int64_t groups = a.rows_per_gate && dgate ? ceil_div(rows, a.rows_per_gate) : 0;
    const dim3 grid(unsigned(ceil_div(e->dim, 32)), unsigned(kJoinSums + std::min<int64_t>(groups, 1024)));
    return launched(launch_in_row(join_sums_kernel, grid, 1024, 0, 1, s, a, ctas, groups BAOC_CHECK_ARG(ck)), "join_sums_kernel");
} catch (const std::bad_alloc&) {
    return BAOC_E_INVALID;
}

}  // extern "C"
