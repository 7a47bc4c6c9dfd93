// Layer norm over the rows of a matrix, forward and backward, and straight to the int8 codes that a ternary
// projection reads:
//     mean = sum x / n,  var = sum (x - mean)^2 / n,  rstd = 1 / sqrt(var + eps),  y = (x - mean) rstd w + b
//     g = dy w,  xh = (x - mean) rstd,  dx = rstd (g - sum(g) / n - xh sum(g xh) / n),  dw = sum_r dy xh,  db = sum_r dy
//     gamma = max |y|,  scale = 127 / max(gamma, 1e-5),  q = clip(round(y scale), -128, 127)      (as in actquant.cuh)
// All three are bound by their bytes: x is read once and a row's statistics are taken from the registers that hold it.
//
// Forward: a warp takes a row of up to 128 accesses of 16 bytes, a block a longer one, up to four accesses a thread; the loads
// of a row are in flight together and several rows share an SM.  Statistics in binary32, the variance from the
// differences to the mean (a sum of squares would cancel).  For codes the statistics are taken in binary64 and
// rounded once, and every step behind them is a single binary32 operation, so that a code does not depend on the
// order of a sum.
//
// Backward: one block per SM walks over its rows, in groups of threads that each take a row at a time.  A row of x
// and dy comes through a ring of bulk copies, a few rows ahead, and the column sums dw and db stay in registers
// until the block has seen its last row: one partial sum per block, added up by a second kernel in a fixed order
// (no atomics: the same inputs give the same bits).  Rows that are not made of whole 16-byte pieces are read element
// by element, and rows too long for the registers take plain loops.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <type_traits>

#include "actquant.cuh"
#include "common.cuh"
#include "ptx.cuh"

namespace prom { namespace norm {

// ---- values of the three types, E to an access: 16 bytes, or one element -------------------------
template <class T> __device__ __forceinline__ float to_float(T v);
template <> __device__ __forceinline__ float to_float<float>(float v) { return v; }
template <> __device__ __forceinline__ float to_float<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }
template <> __device__ __forceinline__ float to_float<__half>(__half v) { return __half2float(v); }
template <class T> __device__ __forceinline__ T from_float(float v);
template <> __device__ __forceinline__ float from_float<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_float<__half>(float v) { return __float2half_rn(v); }

template <class T> constexpr int kWide = 16 / (int)sizeof(T);      // elements of a 16-byte access

template <class T, int E> struct Piece {
    union { uint4 raw; T v[kWide<T>]; };
    __device__ __forceinline__ Piece() : raw(make_uint4(0u, 0u, 0u, 0u)) {}
    __device__ __forceinline__ void load(const T *p) { raw = *reinterpret_cast<const uint4 *>(p); }
    __device__ __forceinline__ void store(T *p) const { *reinterpret_cast<uint4 *>(p) = raw; }
    __device__ __forceinline__ float get(int e) const { return to_float<T>(v[e]); }
    __device__ __forceinline__ void set(int e, float f) { v[e] = from_float<T>(f); }
};
template <class T> struct Piece<T, 1> {
    T v;
    __device__ __forceinline__ Piece() : v(from_float<T>(0.0f)) {}
    __device__ __forceinline__ void load(const T *p) { v = *p; }
    __device__ __forceinline__ void store(T *p) const { *p = v; }
    __device__ __forceinline__ float get(int) const { return to_float<T>(v); }
    __device__ __forceinline__ void set(int, float f) { v = from_float<T>(f); }
};

// A vector of parameters (weight or bias) of any of the types; absent: `otherwise`.
struct Vector {
    const void *p;
    int type;           // prom_type
    __device__ __forceinline__ float at(int i, float otherwise) const
    {
        if (!p) return otherwise;
        if (type == PROM_TYPE_F32) return __ldg(static_cast<const float *>(p) + i);
        if (type == PROM_TYPE_BF16) return to_float(__ldg(static_cast<const __nv_bfloat16 *>(p) + i));
        return to_float(__ldg(static_cast<const __half *>(p) + i));
    }
    // E neighbours from a multiple of E; the base is 16-byte aligned
    template <int E> __device__ __forceinline__ void get(int i, float otherwise, float (&f)[E]) const
    {
        if constexpr (E == 1) {
            f[0] = at(i, otherwise);
        } else {
            if (!p) {
#pragma unroll
                for (int e = 0; e < E; ++e) f[e] = otherwise;
            } else if (type == PROM_TYPE_F32) {
#pragma unroll
                for (int e = 0; e < E; e += 4) {
                    const float4 v = __ldg(reinterpret_cast<const float4 *>(static_cast<const float *>(p) + i + e));
                    f[e] = v.x; f[e + 1] = v.y; f[e + 2] = v.z; f[e + 3] = v.w;
                }
            } else {
                uint32_t w[E / 2];
                const uint2 *src = reinterpret_cast<const uint2 *>(static_cast<const uint16_t *>(p) + i);
#pragma unroll
                for (int e = 0; e < E / 4; ++e) {
                    const uint2 v = __ldg(src + e);
                    w[2 * e] = v.x; w[2 * e + 1] = v.y;
                }
#pragma unroll
                for (int e = 0; e < E / 2; ++e) {
                    if (type == PROM_TYPE_BF16) {
                        f[2 * e] = __uint_as_float(w[e] << 16); f[2 * e + 1] = __uint_as_float(w[e] & 0xFFFF0000u);
                    } else {
                        const float2 v = __half22float2(*reinterpret_cast<const __half2 *>(&w[e]));
                        f[2 * e] = v.x; f[2 * e + 1] = v.y;
                    }
                }
            }
        }
    }
};

struct Fwd {
    const void *x;
    long long m, x_pitch, y_pitch;
    int n;
    Vector w, b;
    double eps;
    void *y;                // nullptr for codes
    int8_t *q;              // [m][n]
    float *mean, *rstd;     // may be nullptr
    float *gamma, *scale;   // with q
};

// ---- sums over the threads that share a row --------------------------------------------------------
template <class A> __device__ __forceinline__ A warp_sum(A v)
{
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
    return v;
}
// Maxima that keep a NaN: a row with one has no codes that mean anything, and its gamma says so.
__device__ __forceinline__ float max_nan(float a, float b) { return b > a || b != b ? b : a; }
__device__ __forceinline__ float warp_max(float v)
{
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) v = max_nan(v, __shfl_xor_sync(0xFFFFFFFFu, v, d));
    return v;
}
// Over the block, in `red` (a slot per warp, not used for another purpose until the next barrier behind this one).
template <class A> __device__ __forceinline__ A block_sum(A v, A *red)
{
    v = warp_sum(v);
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
    __syncthreads();
    const int warps = (int)blockDim.x >> 5;
    A r = (int)(threadIdx.x & 31) < warps ? red[threadIdx.x & 31] : (A)0;
    return warp_sum(r);
}
__device__ __forceinline__ float block_max(float v, float *red)
{
    v = warp_max(v);
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
    __syncthreads();
    const int warps = (int)blockDim.x >> 5;
    const float r = (int)(threadIdx.x & 31) < warps ? red[threadIdx.x & 31] : 0.0f;
    return warp_max(r);
}

// The affine step behind the statistics, each operation rounded on its own (not fused): what a code depends on.
__device__ __forceinline__ float affine_exact(float x, float mean, float rstd, float w, float b)
{
    return __fadd_rn(__fmul_rn(__fmul_rn(__fsub_rn(x, mean), rstd), w), b);
}

// E codes of neighbouring columns in one store (E is 1, 4 or 8; the row's codes are E-aligned).
template <int E> __device__ __forceinline__ void store_codes(int8_t *q, const float (&y)[E], float scale)
{
    if constexpr (E == 1) {
        *q = actq::quantise_one(y[0], scale);
    } else {
        uint32_t w[E / 4];
#pragma unroll
        for (int e = 0; e < E / 4; ++e) w[e] = actq::quantise_four(make_float4(y[4 * e], y[4 * e + 1], y[4 * e + 2], y[4 * e + 3]), scale);
        if constexpr (E == 4) *reinterpret_cast<uint32_t *>(q) = w[0];
        else *reinterpret_cast<uint2 *>(q) = make_uint2(w[0], w[1]);
    }
}

// ---- forward: the row in registers ------------------------------------------------------------------
// WARP: a warp per row, else a block.  V accesses of E elements a thread, thread t takes accesses t, t + threads, ...
template <class T, int E, int V, bool CODES, bool WARP>
__global__ void __launch_bounds__(WARP ? 256 : 1024)
forward_kernel(const Fwd p)
{
    using Sum = typename std::conditional<CODES, double, float>::type;
    __shared__ Sum red[2][32];
    __shared__ float red_max[32];
    const int threads = WARP ? 32 : (int)blockDim.x, t = WARP ? (int)threadIdx.x & 31 : (int)threadIdx.x;
    const long long r = WARP ? (long long)blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5) : (long long)blockIdx.x;
    ptx::grid_dep_wait();
    ptx::grid_dep_launch();
    if (r >= p.m) return;               // whole warps; blocks have exactly their rows
    const int pieces = p.n / E;
    const T *row = static_cast<const T *>(p.x) + r * p.x_pitch;
    Piece<T, E> v[V];
#pragma unroll
    for (int i = 0; i < V; ++i)
        if (t + i * threads < pieces) v[i].load(row + (size_t)(t + i * threads) * E);

    Sum s = 0;
#pragma unroll
    for (int i = 0; i < V; ++i)
#pragma unroll
        for (int e = 0; e < E; ++e) s += (Sum)v[i].get(e);          // what lies past the row is zero
    if constexpr (WARP) s = warp_sum(s); else s = block_sum(s, red[0]);
    const Sum mean = s / (Sum)p.n;
    s = 0;
#pragma unroll
    for (int i = 0; i < V; ++i)
        if (t + i * threads < pieces) {
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const Sum d = (Sum)v[i].get(e) - mean;
                s += d * d;
            }
        }
    if constexpr (WARP) s = warp_sum(s); else s = block_sum(s, red[1]);
    float rstd;
    if constexpr (CODES) rstd = (float)(1.0 / sqrt(s / (double)p.n + p.eps));
    else rstd = 1.0f / sqrtf(s / (float)p.n + (float)p.eps);
    const float mu = (float)mean;
    if (t == 0) {
        if (p.mean) p.mean[r] = mu;
        if (p.rstd) p.rstd[r] = rstd;
    }
    if constexpr (!CODES) {
        T *out = static_cast<T *>(p.y) + r * p.y_pitch;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int c = (t + i * threads) * E;
            if (t + i * threads >= pieces) break;
            float w[E], b[E];
            p.w.get<E>(c, 1.0f, w);
            p.b.get<E>(c, 0.0f, b);
            Piece<T, E> o;
#pragma unroll
            for (int e = 0; e < E; ++e) o.set(e, (v[i].get(e) - mu) * rstd * w[e] + b[e]);
            o.store(out + c);
        }
    } else {
        float y[V][E], top = 0.0f;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int c = (t + i * threads) * E;
            if (t + i * threads >= pieces) break;
            float w[E], b[E];
            p.w.get<E>(c, 1.0f, w);
            p.b.get<E>(c, 0.0f, b);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                y[i][e] = affine_exact(v[i].get(e), mu, rstd, w[e], b[e]);
                top = max_nan(top, fabsf(y[i][e]));
            }
        }
        if constexpr (WARP) top = warp_max(top); else top = block_max(top, red_max);
        const float sc = actq::scale_of(top, 1e-5f);
        if (t == 0) { p.gamma[r] = top; p.scale[r] = sc; }
        int8_t *out = p.q + r * p.n;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            if (t + i * threads >= pieces) break;
            store_codes<E>(out + (size_t)(t + i * threads) * E, y[i], sc);
        }
    }
}

// Rows of any length: a block reads its row once per step (from L2 after the first).
template <class T, bool CODES>
__global__ void __launch_bounds__(1024)
forward_long_kernel(const Fwd p)
{
    using Sum = typename std::conditional<CODES, double, float>::type;
    __shared__ Sum red[2][32];
    __shared__ float red_max[32];
    ptx::grid_dep_wait();
    ptx::grid_dep_launch();
    const long long r = blockIdx.x;
    const T *row = static_cast<const T *>(p.x) + r * p.x_pitch;
    Sum s = 0;
    for (int c = threadIdx.x; c < p.n; c += blockDim.x) s += (Sum)to_float(row[c]);
    const Sum mean = block_sum(s, red[0]) / (Sum)p.n;
    s = 0;
    for (int c = threadIdx.x; c < p.n; c += blockDim.x) {
        const Sum d = (Sum)to_float(row[c]) - mean;
        s += d * d;
    }
    s = block_sum(s, red[1]);
    float rstd;
    if constexpr (CODES) rstd = (float)(1.0 / sqrt(s / (double)p.n + p.eps));
    else rstd = 1.0f / sqrtf(s / (float)p.n + (float)p.eps);
    const float mu = (float)mean;
    if (threadIdx.x == 0) {
        if (p.mean) p.mean[r] = mu;
        if (p.rstd) p.rstd[r] = rstd;
    }
    if constexpr (!CODES) {
        T *out = static_cast<T *>(p.y) + r * p.y_pitch;
        for (int c = threadIdx.x; c < p.n; c += blockDim.x)
            out[c] = from_float<T>((to_float(row[c]) - mu) * rstd * p.w.at(c, 1.0f) + p.b.at(c, 0.0f));
    } else {
        float top = 0.0f;
        for (int c = threadIdx.x; c < p.n; c += blockDim.x)
            top = max_nan(top, fabsf(affine_exact(to_float(row[c]), mu, rstd, p.w.at(c, 1.0f), p.b.at(c, 0.0f))));
        top = block_max(top, red_max);
        const float sc = actq::scale_of(top, 1e-5f);
        if (threadIdx.x == 0) { p.gamma[r] = top; p.scale[r] = sc; }
        for (int c = threadIdx.x; c < p.n; c += blockDim.x)
            p.q[r * p.n + c] = actq::quantise_one(affine_exact(to_float(row[c]), mu, rstd, p.w.at(c, 1.0f), p.b.at(c, 0.0f)), sc);
    }
}

// ---- backward ----------------------------------------------------------------------------------------
struct Bwd {
    const void *dy, *x;
    long long m, dy_pitch, x_pitch, dx_pitch;
    int n;
    Vector w;
    const float *mean, *rstd;
    void *dx;               // may be nullptr
    float *part;            // [blocks][2][n_pad]: sums of dy xh, then of dy; nullptr: not wanted
    int n_pad;              // n rounded up to a multiple of 4
    int group;              // threads that share a row
    int groups;             // of them in a block
    int stages;             // rows of each group's ring
};

// Threads of a block, by the registers that a thread's columns take (2 V E sums, and the weights where they fit beside).
template <int E, int V> constexpr bool kHeavy = V * E >= 32 || V >= 16;
template <int E, int V> constexpr int kBwdThreads = kHeavy<E, V> ? 512 : 768;
constexpr int kMaxGroups = 768 / 32;
constexpr int kMaxStages = 8;

__device__ __forceinline__ void group_barrier(int g, int threads) { ptx::named_sync(1u + (uint32_t)g, (uint32_t)threads); }

// RING: rows come through shared memory by bulk copies (whole 16-byte pieces), else by plain loads.
// Shared memory: the rings ([groups][stages][2][row bytes]), used again at the end for the groups' column sums.
template <class T, int E, int V, bool RING>
__global__ void __launch_bounds__(kBwdThreads<E, V>, 1)
backward_kernel(const Bwd p)
{
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ __align__(8) uint64_t bars[kMaxGroups * kMaxStages];
    __shared__ float2 red[2][kMaxGroups];
    __shared__ volatile int failed;
    const int g = (int)threadIdx.x / p.group, t = (int)threadIdx.x - g * p.group;
    const int lane = threadIdx.x & 31, warps = p.group >> 5, first_warp = g * warps;
    const int pieces = p.n / E;
    const uint32_t row_bytes = (uint32_t)p.n * (uint32_t)sizeof(T);
    const uint32_t ring = ptx::smem_u32(smem) + (uint32_t)g * p.stages * 2u * row_bytes;
    const uint32_t bar0 = ptx::smem_u32(bars) + 8u * (uint32_t)(g * p.stages);
    const long long step = (long long)gridDim.x * p.groups, r0 = (long long)blockIdx.x * p.groups + g;
    const T *x = static_cast<const T *>(p.x), *dy = static_cast<const T *>(p.dy);

    if (RING) {
        if (t < p.stages) ptx::mbar_init(bar0 + 8u * t, 1);
        ptx::mbar_init_fence();
    }
    if (threadIdx.x == 0) failed = 0;
    __syncthreads();
    ptx::grid_dep_wait();
    ptx::grid_dep_launch();
    auto fetch = [&](int s, long long r) {      // by one thread of the group
        ptx::mbar_expect_tx(bar0 + 8u * s, 2u * row_bytes);
        ptx::bulk_load(ring + (uint32_t)s * 2u * row_bytes, x + r * p.x_pitch, row_bytes, bar0 + 8u * s);
        ptx::bulk_load(ring + (uint32_t)s * 2u * row_bytes + row_bytes, dy + r * p.dy_pitch, row_bytes, bar0 + 8u * s);
    };
    long long ahead = r0;                       // the next row to fetch (kept by that thread)
    if (RING && t == 0)
        for (int s = 0; s < p.stages && ahead < p.m; ++s, ahead += step) fetch(s, ahead);

    constexpr bool kHoldW = !kHeavy<E, V>;
    float held[kHoldW ? V : 1][E], dw[V][E], db[V][E];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        if constexpr (kHoldW)
            if (t + i * p.group < pieces) p.w.get<E>((t + i * p.group) * E, 1.0f, held[i]);
#pragma unroll
        for (int e = 0; e < E; ++e) dw[i][e] = db[i][e] = 0.0f;
    }
    const float inv_n = 1.0f / (float)p.n;
    int s = 0, which = 0;
    uint32_t phase = 0;
    for (long long r = r0; r < p.m; r += step) {
        const float mean = __ldg(p.mean + r), rstd = __ldg(p.rstd + r);
        Piece<T, E> vx[V], vd[V];
        if constexpr (RING) {
            // A wait that runs out is the last one: the block goes on without waiting, so that its barriers stay in
            // step, fetches nothing more and reports at the end.
            const unsigned long long t0 = ptx::globaltimer();
            while (!ptx::mbar_try_wait(bar0 + 8u * s, phase))
                if (failed || ptx::globaltimer() - t0 > actq::kWaitLimitNs) { failed = 1; break; }
            const T *sx = reinterpret_cast<const T *>(smem + (size_t)(g * p.stages + s) * 2 * row_bytes);
            const T *sd = reinterpret_cast<const T *>(smem + (size_t)(g * p.stages + s) * 2 * row_bytes + row_bytes);
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (t + i * p.group < pieces) {
                    vx[i].load(sx + (size_t)(t + i * p.group) * E);
                    vd[i].load(sd + (size_t)(t + i * p.group) * E);
                }
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (t + i * p.group < pieces) {
                    vx[i].load(x + r * p.x_pitch + (size_t)(t + i * p.group) * E);
                    vd[i].load(dy + r * p.dy_pitch + (size_t)(t + i * p.group) * E);
                }
        }
        float2 sum = make_float2(0.0f, 0.0f);       // of g and of g xh
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (t + i * p.group < pieces) {
                float w[E];
                if constexpr (!kHoldW) p.w.get<E>((t + i * p.group) * E, 1.0f, w);
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const float we = kHoldW ? held[kHoldW ? i : 0][e] : w[e];
                    const float d = vd[i].get(e), xh = (vx[i].get(e) - mean) * rstd, gr = d * we;
                    sum.x += gr;
                    sum.y += gr * xh;
                    dw[i][e] += d * xh;
                    db[i][e] += d;
                }
            }
        sum.x = warp_sum(sum.x);
        sum.y = warp_sum(sum.y);
        if (warps > 1) {
            if (lane == 0) red[which][threadIdx.x >> 5] = sum;
            group_barrier(g, p.group);
            // every thread of the group has read its part of the stage, so it can be filled again
            float2 a = lane < warps ? red[which][first_warp + lane] : make_float2(0.0f, 0.0f);
            sum.x = warp_sum(a.x);
            sum.y = warp_sum(a.y);
            which ^= 1;                         // the next row's sums go elsewhere: these may still be read
        } else {
            __syncwarp();
        }
        if (RING) {
            if (t == 0 && ahead < p.m && !failed) { fetch(s, ahead); ahead += step; }
            if (++s == p.stages) { s = 0; phase ^= 1u; }
        }
        if (p.dx) {
            const float c1 = sum.x * inv_n, c2 = sum.y * inv_n;
            T *out = static_cast<T *>(p.dx) + r * p.dx_pitch;
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (t + i * p.group < pieces) {
                    Piece<T, E> o;
                    float w[E];
                    if constexpr (!kHoldW) p.w.get<E>((t + i * p.group) * E, 1.0f, w);
#pragma unroll
                    for (int e = 0; e < E; ++e) {
                        const float we = kHoldW ? held[kHoldW ? i : 0][e] : w[e];
                        const float xh = (vx[i].get(e) - mean) * rstd;
                        o.set(e, rstd * (vd[i].get(e) * we - c1 - xh * c2));
                    }
                    o.store(out + (size_t)(t + i * p.group) * E);
                }
        }
    }
    __syncthreads();
    if (RING && failed) {
        // copies may be in flight yet: outwait them before the shared memory goes
        const unsigned long long t0 = ptx::globaltimer();
        while (ptx::globaltimer() - t0 < actq::kWaitLimitNs) {}
        if (threadIdx.x == 0) raise_status(PROM_ERR_TIMEOUT);
        return;
    }
    if (!p.part) return;

    // The groups' column sums, added in the order of the groups; all copies have landed and been read.
    float *acc = reinterpret_cast<float *>(smem);       // [2][n_pad]
    for (int k = 0; k < p.groups; ++k) {
        if (g == k) {
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (t + i * p.group < pieces) {
                    const int c = (t + i * p.group) * E;
#pragma unroll
                    for (int e = 0; e < E; ++e) {
                        acc[c + e] = dw[i][e] + (k ? acc[c + e] : 0.0f);
                        acc[p.n_pad + c + e] = db[i][e] + (k ? acc[p.n_pad + c + e] : 0.0f);
                    }
                }
        }
        __syncthreads();
    }
    float *mine = p.part + (size_t)blockIdx.x * 2 * p.n_pad;
    for (int c = threadIdx.x; c < 2 * p.n_pad; c += blockDim.x)
        mine[c] = c % p.n_pad < p.n ? acc[c] : 0.0f;
}

// Rows of any length: dx by a block per row, and the column sums of a slice of rows by a block per 256 columns.
template <class T>
__global__ void __launch_bounds__(1024)
backward_long_kernel(const Bwd p)
{
    __shared__ float red[2][32];
    ptx::grid_dep_wait();
    ptx::grid_dep_launch();
    const long long r = blockIdx.x;
    const T *x = static_cast<const T *>(p.x) + r * p.x_pitch, *dy = static_cast<const T *>(p.dy) + r * p.dy_pitch;
    T *dx = static_cast<T *>(p.dx) + r * p.dx_pitch;
    const float mean = p.mean[r], rstd = p.rstd[r];
    float s1 = 0.0f, s2 = 0.0f;
    for (int c = threadIdx.x; c < p.n; c += blockDim.x) {
        const float gr = to_float(dy[c]) * p.w.at(c, 1.0f);
        s1 += gr;
        s2 += gr * ((to_float(x[c]) - mean) * rstd);
    }
    const float c1 = block_sum(s1, red[0]) / (float)p.n, c2 = block_sum(s2, red[1]) / (float)p.n;
    for (int c = threadIdx.x; c < p.n; c += blockDim.x)
        dx[c] = from_float<T>(rstd * (to_float(dy[c]) * p.w.at(c, 1.0f) - c1 - (to_float(x[c]) - mean) * rstd * c2));
}

// Launched behind backward_long_kernel without overlap: with dx == dy the column sums would read what that one wrote, so it
// goes first (see the host code).
template <class T>
__global__ void __launch_bounds__(256)
column_sums_kernel(const Bwd p, long long rows_per_block)
{
    ptx::grid_dep_wait();
    ptx::grid_dep_launch();
    const int c = blockIdx.x * 256 + threadIdx.x;
    const long long r0 = (long long)blockIdx.y * rows_per_block, r1 = r0 + rows_per_block < p.m ? r0 + rows_per_block : p.m;
    if (c >= p.n_pad) return;
    float dw = 0.0f, db = 0.0f;
    if (c < p.n)
        for (long long r = r0; r < r1; ++r) {
            const float d = to_float(static_cast<const T *>(p.dy)[r * p.dy_pitch + c]);
            dw += d * ((to_float(static_cast<const T *>(p.x)[r * p.x_pitch + c]) - __ldg(p.mean + r)) * __ldg(p.rstd + r));
            db += d;
        }
    float *mine = p.part + (size_t)blockIdx.y * 2 * p.n_pad;
    mine[c] = dw;
    mine[p.n_pad + c] = db;
}

// The sums over the blocks' partial sums: eight warps share 128 columns, each every eighth block, then one adds the eight.
__global__ void __launch_bounds__(256)
backward_sum_kernel(const float *__restrict__ part, int blocks, int n, int n_pad, void *dw, void *db, int type)
{
    __shared__ float4 s[8][32];
    ptx::grid_dep_wait();
    ptx::grid_dep_launch();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int c = blockIdx.x * 128 + lane * 4;          // of the 2 n_pad columns
    float4 a = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    if (c < 2 * n_pad) {
#pragma unroll 4
        for (int k = warp; k < blocks; k += 8) {
            const float4 v = *reinterpret_cast<const float4 *>(part + (size_t)k * 2 * n_pad + c);
            a.x += v.x; a.y += v.y; a.z += v.z; a.w += v.w;
        }
    }
    s[warp][lane] = a;
    __syncthreads();
    if (warp || c >= 2 * n_pad) return;
#pragma unroll
    for (int k = 1; k < 8; ++k) { const float4 v = s[k][lane]; a.x += v.x; a.y += v.y; a.z += v.z; a.w += v.w; }
    void *out = c < n_pad ? dw : db;
    if (!out) return;
    const int c0 = c < n_pad ? c : c - n_pad;
    const float f[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        if (c0 + e >= n) break;
        if (type == PROM_TYPE_F32) static_cast<float *>(out)[c0 + e] = f[e];
        else if (type == PROM_TYPE_BF16) static_cast<__nv_bfloat16 *>(out)[c0 + e] = __float2bfloat16_rn(f[e]);
        else static_cast<__half *>(out)[c0 + e] = __float2half_rn(f[e]);
    }
}

// dw and db of no rows.
__global__ void zero_kernel(int n, void *dw, void *db, int type)
{
    ptx::grid_dep_wait();
    ptx::grid_dep_launch();
    const int c = blockIdx.x * blockDim.x + threadIdx.x;
    if (c >= n) return;
    for (int k = 0; k < 2; ++k) {
        void *out = k ? db : dw;
        if (!out) continue;
        if (type == PROM_TYPE_F32) static_cast<float *>(out)[c] = 0.0f;
        else static_cast<uint16_t *>(out)[c] = 0;
    }
}

}}  // namespace prom::norm
