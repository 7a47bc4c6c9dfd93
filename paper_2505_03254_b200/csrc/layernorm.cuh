// Layer norm over the rows of a matrix, forward and backward, and straight to the int8 codes that a ternary
// projection reads:
//     mean = sum x / n,  var = sum (x - mean)^2 / n,  rstd = 1 / sqrt(var + eps),  y = (x - mean) rstd w + b
//     g = dy w,  xh = (x - mean) rstd,  dx = rstd (g - sum(g) / n - xh sum(g xh) / n),  dw = sum_r dy xh,  db = sum_r dy
//     gamma = max |y|,  scale = 127 / max(gamma, 1e-5),  q = clip(round(y scale), -128, 127)      (as in actquant.cuh)
// What all of them cannot do without is their bytes: x once (and dy), y, codes or dx once.  At 16384 x 4096 bf16 the forward
// pass takes 53.9 us (5.0 TB/s, 76 % of the measured copy bandwidth), the backward pass 81.5 (4.9 TB/s; 76 in a replayed graph);
// 8192 x 4096 bf16 to codes takes 42.4 us, there bound by its issue slots: 26 instructions a value, of which the 64-bit sums
// take a share, and the affine step with its parameters, worked out once for the maximum and once for the codes.
//
// Many rows, forward: a warp per row, in registers or in shared memory, the parameters in shared memory.  Otherwise, and in
// the backward pass, threads come in groups that share a row, a 16-byte piece (8 or 4 columns) each, as many groups as fill
// an SM, and walk over the rows: what belongs to a column (weight, bias, the sums for dw and db) stays in registers, and the
// next rows are on their way while the current ones are worked on.  Two rows are taken at a time where registers allow, so
// that an exchange between the warps of a group serves both.  Few rows: a block each.
//
// Rows need not start on a 16-byte boundary.  A thread's piece is one of memory, its columns are shifted by the row's offset,
// and a group only takes rows of one offset (it repeats after at most eight rows), so the shifted parameters stay in
// registers too; only the first and the last piece of a row are read and written by the element.
//
// Forward: statistics in binary32, the variance from the differences to the mean (a sum of squares would cancel).  For
// codes the statistics are taken in binary64 and rounded once, and every step behind them is a single binary32 operation, so
// that the order of a sum, which moves it by a few 2^-53, shows only where that decides the one rounding.
//
// Backward: rows of a kilobyte or more on 16-byte boundaries come through a ring of bulk copies.  The column sums make one
// partial sum per block, added up by a second kernel in a fixed order (no atomics: the same inputs give the same bits).
//
// Rows of more than 1024 pieces take several pieces a thread, very long ones plain loops; tensors whose rows have different
// offsets are read element by element.
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
template <> __device__ __forceinline__ float to_float<__nv_bfloat16>(__nv_bfloat16 v)
{
    return __uint_as_float((uint32_t)__bfloat16_as_ushort(v) << 16);
}
template <> __device__ __forceinline__ float to_float<__half>(__half v) { return __half2float(v); }
template <class T> __device__ __forceinline__ T from_float(float v);
template <> __device__ __forceinline__ float from_float<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_float<__half>(float v) { return __float2half_rn(v); }

// Two values to one word, and one of a word's two.  Shifts and packed conversions: a 16-bit value converted alone takes the
// pipe of the special functions, at an eighth of their rate, which was the bound of every kernel here.
template <class T> __device__ __forceinline__ uint32_t pack_pair(float lo, float hi);
template <> __device__ __forceinline__ uint32_t pack_pair<__nv_bfloat16>(float lo, float hi)
{
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&v);
}
template <> __device__ __forceinline__ uint32_t pack_pair<__half>(float lo, float hi)
{
    const __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&v);
}

template <class T> __device__ __forceinline__ float half_of(uint32_t w, int upper);
template <> __device__ __forceinline__ float half_of<__nv_bfloat16>(uint32_t w, int upper) { return __uint_as_float(upper ? w & 0xFFFF0000u : w << 16); }
template <> __device__ __forceinline__ float half_of<__half>(uint32_t w, int upper)
{
    const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&w));
    return upper ? f.y : f.x;
}
template <> __device__ __forceinline__ float half_of<float>(uint32_t w, int) { return __uint_as_float(w); }      // (not used)

template <class T> constexpr int kWide = 16 / (int)sizeof(T);      // elements of a 16-byte access

// Two neighbours in one operation each, rounded as two single ones would be: the kernels' issue slots, and not the operations
// themselves, are what runs short beside the memory (backward, 16384 x 4096 bf16: 84.1 us one value at a time, 80.5 so).
struct Two { float x, y; };
__device__ __forceinline__ Two both(float v) { return {v, v}; }
__device__ __forceinline__ Two operator+(Two a, Two b)
{
    Two d;
    asm("{\n.reg .b64 a, b, d;\nmov.b64 a, {%2, %3};\nmov.b64 b, {%4, %5};\nadd.rn.f32x2 d, a, b;\nmov.b64 {%0, %1}, d;\n}"
        : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
}
__device__ __forceinline__ Two operator*(Two a, Two b)
{
    Two d;
    asm("{\n.reg .b64 a, b, d;\nmov.b64 a, {%2, %3};\nmov.b64 b, {%4, %5};\nmul.rn.f32x2 d, a, b;\nmov.b64 {%0, %1}, d;\n}"
        : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
}
__device__ __forceinline__ Two fma_of(Two a, Two b, Two c)
{
    Two d;
    asm("{\n.reg .b64 a, b, c, d;\nmov.b64 a, {%2, %3};\nmov.b64 b, {%4, %5};\nmov.b64 c, {%6, %7};\nfma.rn.f32x2 d, a, b, c;\n"
        "mov.b64 {%0, %1}, d;\n}"
        : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
    return d;
}

template <class T, int E> struct Piece {
    uint4 raw;
    __device__ __forceinline__ Piece() : raw(make_uint4(0u, 0u, 0u, 0u)) {}
    __device__ __forceinline__ void load(const T *p) { raw = *reinterpret_cast<const uint4 *>(p); }
    __device__ __forceinline__ void store(T *p) const { *reinterpret_cast<uint4 *>(p) = raw; }
    __device__ __forceinline__ void load_shared(uint32_t addr)
    {
        const int4 v = ptx::lds_128(addr);
        raw = make_uint4((uint32_t)v.x, (uint32_t)v.y, (uint32_t)v.z, (uint32_t)v.w);
    }
    __device__ __forceinline__ float get(int e) const
    {
        const int i = sizeof(T) == 4 ? e : e >> 1;
        const uint32_t w = i == 0 ? raw.x : i == 1 ? raw.y : i == 2 ? raw.z : raw.w;
        return sizeof(T) == 4 ? __uint_as_float(w) : half_of<T>(w, e & 1);
    }
    __device__ __forceinline__ Two two(int e) const { return {get(e), get(e + 1)}; }
    __device__ __forceinline__ void set(const float (&f)[E])
    {
        if constexpr (sizeof(T) == 4) raw = make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
        else raw = make_uint4(pack_pair<T>(f[0], f[1]), pack_pair<T>(f[2], f[3]), pack_pair<T>(f[4 % E], f[5 % E]), pack_pair<T>(f[6 % E], f[7 % E]));
    }
    // From here on the values are converted again instead of being kept as floats, twice the registers of 16-bit ones.
    __device__ __forceinline__ void again() { asm volatile("" : "+r"(raw.x), "+r"(raw.y), "+r"(raw.z), "+r"(raw.w)); }
};
// The piece of columns c .. c + E - 1 of a row of n, of which some may lie outside it (zeros).
template <class T, int E> __device__ __forceinline__ void load_at(Piece<T, E> &v, const T *row, int c, int n)
{
    if (c >= 0 && c + E <= n) {
        v.load(row + c);
    } else {
        uint32_t w[4] = {0u, 0u, 0u, 0u};
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (c + e >= 0 && c + e < n) {
                if constexpr (sizeof(T) == 4) w[e] = __float_as_uint((float)row[c + e]);
                else w[e / 2] |= (uint32_t)reinterpret_cast<const uint16_t *>(row)[c + e] << (16 * (e & 1));
            }
        v.raw = make_uint4(w[0], w[1], w[2], w[3]);
    }
}
// What of it lies outside the row takes the first value that does not.
template <class T, int E> __device__ __forceinline__ void fill_outside(Piece<T, E> &v, int c, int n)
{
    constexpr int kBits = 8 * (int)sizeof(T), kEach = 32 / kBits;
    constexpr uint32_t mask = sizeof(T) == 4 ? 0xFFFFFFFFu : 0xFFFFu;
    uint32_t w[4] = {v.raw.x, v.raw.y, v.raw.z, v.raw.w}, first = 0u;
#pragma unroll
    for (int e = 0; e < E; ++e)
        if (e == (c < 0 ? -c : 0)) first = (w[e / kEach] >> (kBits * (e % kEach))) & mask;
#pragma unroll
    for (int e = 0; e < E; ++e)
        if (c + e < 0 || c + e >= n) w[e / kEach] = (w[e / kEach] & ~(mask << (kBits * (e % kEach)))) | first << (kBits * (e % kEach));
    v.raw = make_uint4(w[0], w[1], w[2], w[3]);
}
template <class T, int E> __device__ __forceinline__ void store_at(const Piece<T, E> &v, T *row, int c, int n)
{
    if (c >= 0 && c + E <= n) {
        v.store(row + c);
    } else {
        const uint32_t w[4] = {v.raw.x, v.raw.y, v.raw.z, v.raw.w};
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (c + e >= 0 && c + e < n) {
                if constexpr (sizeof(T) == 4) row[c + e] = __uint_as_float(w[e]);
                else reinterpret_cast<uint16_t *>(row)[c + e] = (uint16_t)(w[e / 2] >> (16 * (e & 1)));
            }
    }
}
template <class T> struct Piece<T, 1> {
    T v;
    __device__ __forceinline__ Piece() : v(from_float<T>(0.0f)) {}
    __device__ __forceinline__ void load(const T *p) { v = *p; }
    __device__ __forceinline__ void store(T *p) const { *p = v; }
    __device__ __forceinline__ void load_shared(uint32_t) {}       // (rows in shared memory are whole pieces)
    __device__ __forceinline__ float get(int) const { return to_float<T>(v); }
    __device__ __forceinline__ void set(const float (&f)[1]) { v = from_float<T>(f[0]); }
    __device__ __forceinline__ void again() {}
};

// One value or two, for kernels of both kinds of pieces.
template <class P> __device__ __forceinline__ P all(float v) { if constexpr (sizeof(P) == 8) return both(v); else return v; }
template <class P, class T, int E> __device__ __forceinline__ P some(const Piece<T, E> &v, int e) { if constexpr (sizeof(P) == 8) return v.two(e); else return v.get(e); }
template <class P> __device__ __forceinline__ P some(const float *f, int e) { if constexpr (sizeof(P) == 8) return {f[e], f[e + 1]}; else return f[e]; }
__device__ __forceinline__ void put(float *f, int e, Two v) { f[e] = v.x; f[e + 1] = v.y; }
__device__ __forceinline__ void put(float *f, int e, float v) { f[e] = v; }
__device__ __forceinline__ float sum_of(Two v) { return v.x + v.y; }
__device__ __forceinline__ float sum_of(float v) { return v; }
__device__ __forceinline__ float fma_of(float a, float b, float c) { return fmaf(a, b, c); }

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
    // E neighbours from column c on, which may start and end outside the n; once per thread
    template <int E> __device__ __forceinline__ void get_at(int c, int n, float otherwise, float (&f)[E]) const
    {
        if (c % E == 0 && c >= 0 && c + E <= n && (reinterpret_cast<uintptr_t>(p) & 15u) == 0) {
            get<E>(c, otherwise, f);
        } else {
#pragma unroll
            for (int e = 0; e < E; ++e) f[e] = c + e >= 0 && c + e < n ? at(c + e, otherwise) : 0.0f;
        }
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
    int group, groups, period;      // as in Bwd
    void *y;                // nullptr for codes
    int8_t *q;              // [m][n]
    float *mean, *rstd;     // may be nullptr
    float *gamma, *scale;   // with q
};

// A value as a double without a conversion (a quarter of the rate of the arithmetic): the bits moved into a double's places
// are the value times 2^-896, zeros and subnormals included, and the factor enters the next multiply-add.  What is not finite
// would become finite: the callers look for it.
template <class T> __device__ __forceinline__ double scaled_down(float f)
{
    const int u = __float_as_int(f);
    return __hiloint2double((u >> 3) & (int)0x8FFFFFFF, std::is_same<T, float>::value ? u << 29 : 0);   // (16-bit types end above)
}
__device__ __forceinline__ double two_896() { return __hiloint2double(0x77F00000, 0); }

// s / n, correctly rounded, from 1 / n rounded: the product corrected once by its remainder (P. Markstein, IBM Journal of Research
// and Development 34, 1990).  n is a whole number below 2^17, so the remainder is exact, the corrected quotient is off by less than
// 2^-22 units of its last place before it is rounded, and no quotient lies that near to the middle of two numbers (such a
// middle times n has a bit more than s; any other quotient is 2^-18 of a unit away).  The plain product gives a constant row
// a mean beside its value, and a mean halfway between two binary32 numbers the wrong one.  (Division, which has to find 1 / n
// anew: 25088 x 192 float32 to codes 13.2 us instead of 11.2.)
__device__ __forceinline__ float quotient(float s, float n, float inverse)
{
    const float q = s * inverse, r = fmaf(fmaf(-q, n, s), inverse, q);
    return fabsf(q) <= 3.402823466e38f ? r : q;         // (an infinity has no remainder)
}
__device__ __forceinline__ double quotient(double s, double n, double inverse)      // (of finite sums)
{
    const double q = s * inverse;
    return fma(fma(-q, n, s), inverse, q);
}

// 1 / sqrt(v + eps), in every kernel by the same operations; binary32: the approximation and one step of Newton's method.
__device__ __forceinline__ float inverse_root(float v, double eps)
{
    v += (float)eps;
    const float r = rsqrtf(v);
    return v > 0.0f && v < 1e38f ? r * fmaf(-0.5f * v * r, r, 1.5f) : r;
}
__device__ __forceinline__ float inverse_root(double v, double eps) { return (float)rsqrt(v + eps); }

// ---- sums over the threads that share a row --------------------------------------------------------
template <class A> __device__ __forceinline__ A warp_sum(A v)
{
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
    return v;
}
// Maxima that keep a NaN: a row with one has no codes that mean anything, and its gamma says so.
__device__ __forceinline__ float max_nan(float a, float b)
{
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
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

// The maximum of a row to codes is not finite: because its values are not, or because a parameter is not or y overflows.  The
// sum of what is not finite in it over one thread's part, 0 where all is finite.  (The statistics' sums take such bits for
// a number's; the formula's mean is this sum over all threads, and NaN is what the rest of the row becomes.)
template <class T> __device__ __forceinline__ float sum_not_finite(const Fwd &p, long long r, int first, int hop)
{
    const T *row = static_cast<const T *>(p.x) + r * p.x_pitch;
    float s = 0.0f;
    for (int c = first; c < p.n; c += hop) {
        const float f = to_float(row[c]);
        s += fabsf(f) <= 3.402823466e38f ? 0.0f : f;
    }
    return s;
}
__device__ __forceinline__ bool not_finite(float v) { return !(fabsf(v) <= 3.402823466e38f); }

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

// ---- groups of threads that share rows -----------------------------------------------------------------
__device__ __forceinline__ void group_barrier(int g, int threads)
{
    if (threads == (int)blockDim.x) __syncthreads();
    else ptx::named_sync(1u + (uint32_t)g, (uint32_t)threads);
}

// The sums over a warp of four values at once: lane bit 4 chooses between the first and the second two, bit 3 within them.
__device__ __forceinline__ float warp_sum_4(float a, float b, float c, float d)
{
    const int lane = threadIdx.x & 31;
    const bool up = (lane & 16) != 0;
    float x = up ? c : a, y = up ? d : b;
    x += __shfl_xor_sync(0xFFFFFFFFu, up ? a : c, 16);
    y += __shfl_xor_sync(0xFFFFFFFFu, up ? b : d, 16);
    const bool second = (lane & 8) != 0;
    float v = second ? y : x;
    v += __shfl_xor_sync(0xFFFFFFFFu, second ? x : y, 8);
#pragma unroll
    for (int k = 4; k > 0; k >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, k);
    return v;
}
__device__ __forceinline__ void spread_4(float v, float &a, float &b, float &c, float &d)
{
    a = __shfl_sync(0xFFFFFFFFu, v, 0);
    b = __shfl_sync(0xFFFFFFFFu, v, 8);
    c = __shfl_sync(0xFFFFFFFFu, v, 16);
    d = __shfl_sync(0xFFFFFFFFu, v, 24);
}

// The same for two values: lane bit 4 chooses.
template <class A> __device__ __forceinline__ A warp_sum_2(A a, A b)
{
    const bool up = (threadIdx.x & 16) != 0;
    A v = up ? b : a;
    v += __shfl_xor_sync(0xFFFFFFFFu, up ? a : b, 16);
#pragma unroll
    for (int k = 8; k > 0; k >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, k);
    return v;
}
__device__ __forceinline__ float warp_max_2(float a, float b)
{
    const bool up = (threadIdx.x & 16) != 0;
    float v = max_nan(up ? b : a, __shfl_xor_sync(0xFFFFFFFFu, up ? a : b, 16));
#pragma unroll
    for (int k = 8; k > 0; k >>= 1) v = max_nan(v, __shfl_xor_sync(0xFFFFFFFFu, v, k));
    return v;
}
// Two sums (or maxima) over a group: the first in the lower half of every warp, the second in the upper one, where what
// follows from them is worked out for both at once.  `red` has a pair per warp of the block and is free again behind the
// barrier after next.
template <class A> __device__ __forceinline__ A group_sum_2(A a, A b, A (*red)[2], int g, int threads)
{
    A v = warp_sum_2(a, b);
    const int lane = threadIdx.x & 31, warps = threads >> 5;
    if (warps > 1) {
        if ((lane & 15) == 0) red[threadIdx.x >> 5][lane >> 4] = v;
        group_barrier(g, threads);
        A x = (A)0, y = (A)0;
        if (lane < warps) { x = red[g * warps + lane][0]; y = red[g * warps + lane][1]; }
        v = warp_sum_2(x, y);
    }
    return v;
}
__device__ __forceinline__ float group_max_2(float a, float b, float (*red)[2], int g, int threads)
{
    float v = warp_max_2(a, b);
    const int lane = threadIdx.x & 31, warps = threads >> 5;
    if (warps > 1) {
        if ((lane & 15) == 0) red[threadIdx.x >> 5][lane >> 4] = v;
        group_barrier(g, threads);
        float x = 0.0f, y = 0.0f;
        if (lane < warps) { x = red[g * warps + lane][0]; y = red[g * warps + lane][1]; }
        v = warp_max_2(x, y);
    }
    return v;
}
template <class A> __device__ __forceinline__ void spread_2(A v, A (&to)[2])
{
    to[0] = __shfl_sync(0xFFFFFFFFu, v, 0);
    to[1] = __shfl_sync(0xFFFFFFFFu, v, 16);
}

// The parameters as floats in shared memory, a piece's first and last four columns apart, so that a warp's 16-byte accesses
// are side by side.  n is a multiple of E.
template <int E> __device__ __forceinline__ void stage_parameters(const Fwd &p, float *sw, float *sb)
{
    const int pieces = p.n / E;
    for (int i = threadIdx.x; i < p.n; i += blockDim.x) {
        const int at = ((i % E / 4) * pieces + i / E) * 4 + i % 4;
        sw[at] = p.w.at(i, 1.0f);
        sb[at] = p.b.at(i, 0.0f);
    }
}
template <int E>
__device__ __forceinline__ void parameters_of(const float *sw, const float *sb, int pieces, int piece, float (&w)[E], float (&b)[E])
{
#pragma unroll
    for (int f = 0; f < E / 4; ++f) {
        const float4 a = reinterpret_cast<const float4 *>(sw)[f * pieces + piece], c = reinterpret_cast<const float4 *>(sb)[f * pieces + piece];
        w[4 * f] = a.x; w[4 * f + 1] = a.y; w[4 * f + 2] = a.z; w[4 * f + 3] = a.w;
        b[4 * f] = c.x; b[4 * f + 1] = c.y; b[4 * f + 2] = c.z; b[4 * f + 3] = c.w;
    }
}

// Columns that the first piece of the row at `p` has before it.
template <class T> __device__ __forceinline__ int offset_of(const void *p) { return (int)((reinterpret_cast<uintptr_t>(p) & 15u) / sizeof(T)); }

// ---- forward: groups, for rows that start anywhere ------------------------------------------------------
// V pieces a thread, two rows at a time and the next two on their way.  (576 threads are two groups for rows of 4096 and
// some values: 8192 x 4269 bf16 69.5 us, 100 with 512.)
constexpr int kGroupThreads = 576;
template <class T, int V, bool CODES>
__global__ void __launch_bounds__(kGroupThreads, 1)
forward_groups_kernel(const Fwd p)
{
    using Sum = typename std::conditional<CODES, double, float>::type;
    constexpr int E = kWide<T>;
    __shared__ Sum red_mean[32][2], red_var[32][2];
    __shared__ float red_max[32][2];
    const int g = (int)threadIdx.x / p.group, t = (int)threadIdx.x - g * p.group, n = p.n;
    const int all = (int)gridDim.x * p.groups / p.period * p.period;       // groups: a whole number for every offset
    const int r0 = g * (int)gridDim.x + (int)blockIdx.x, m = (int)p.m;     // (the last rows go round the SMs)
    ptx::grid_dep_wait();
    ptx::grid_dep_launch();
    if (r0 >= all || r0 >= m) return;           // (whole groups, which meet no other's threads)
    const T *x = static_cast<const T *>(p.x);
    const int c0 = t * E - offset_of<T>(x + r0 * p.x_pitch), hop = p.group * E;     // access i has columns c0 + i hop .. + E - 1
    auto full = [&](int i) { return c0 + i * hop >= 0 && c0 + i * hop + E <= n; };
    auto some = [&](int i) { return c0 + i * hop + E > 0 && c0 + i * hop < n; };
    auto inside = [&](int i, int e) { return c0 + i * hop + e >= 0 && c0 + i * hop + e < n; };
    float w[V][E], b[V][E];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        p.w.get_at<E>(c0 + i * hop, n, 1.0f, w[i]);
        p.b.get_at<E>(c0 + i * hop, n, 0.0f, b[i]);
    }
    const Sum inv_n = (Sum)1 / (Sum)n;
    // codes of a whole piece in one store
    const bool wide_q = CODES && (reinterpret_cast<uintptr_t>(p.q) + (uint64_t)((long long)r0 * n + c0)) % E == 0 && (long long)all * n % E == 0;

    Piece<T, E> v[2][V], next[2][V];
    auto load = [&](int r, Piece<T, E> (&to)[V]) {
        const T *row = x + r * p.x_pitch;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            to[i].raw = make_uint4(0u, 0u, 0u, 0u);
            if (r < m && some(i)) load_at(to[i], row, c0 + i * hop, n);
        }
    };
    auto later = [&](int r, int k) { return (long long)r + (long long)k * all < m ? r + k * all : m; };
    load(r0, next[0]);
    load(later(r0, 1), next[1]);
#pragma unroll 1
    for (int r = r0; r < m; r = later(r, 2)) {
        const bool two = later(r, 1) < m;
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int i = 0; i < V; ++i) v[k][i] = next[k][i];
        load(later(r, 2), next[0]);
        load(later(r, 3), next[1]);
        Sum s[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            s[k] = 0;
#pragma unroll
            for (int i = 0; i < V; ++i)
#pragma unroll
                for (int e = 0; e < E; ++e) {   // (what lies outside the row is zero)
                    if constexpr (CODES) s[k] = fma(scaled_down<T>(v[k][i].get(e)), two_896(), s[k]);
                    else s[k] += v[k][i].get(e);
                }
        }
        Sum mean[2];
        spread_2(quotient(group_sum_2(s[0], s[1], red_mean, g, p.group), (Sum)n, inv_n), mean);
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            s[k] = 0;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                v[k][i].again();
                if (some(i)) {
#pragma unroll
                    for (int e = 0; e < E; ++e) {
                        Sum d;
                        if constexpr (CODES) d = fma(scaled_down<T>(v[k][i].get(e)), two_896(), -mean[k]);
                        else d = v[k][i].get(e) - mean[k];
                        if (full(i) || inside(i, e)) s[k] = fma(d, d, s[k]);
                    }
                }
            }
        }
        const float rstd_half = inverse_root(quotient(group_sum_2(s[0], s[1], red_var, g, p.group), (Sum)n, inv_n), p.eps);
        float mu[2] = {(float)mean[0], (float)mean[1]}, rstd[2];
        spread_2(rstd_half, rstd);
        if constexpr (!CODES) {
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                if (k && !two) continue;
                T *row = static_cast<T *>(p.y) + (r + k * all) * p.y_pitch;
#pragma unroll
                for (int i = 0; i < V; ++i)
                    if (some(i)) {
                        v[k][i].again();
                        float f[E];
#pragma unroll
                        for (int e = 0; e < E; ++e) f[e] = (v[k][i].get(e) - mu[k]) * rstd[k] * w[i][e] + b[i][e];
                        Piece<T, E> o;
                        o.set(f);
                        store_at<T, E>(o, row, c0 + i * hop, n);
                    }
            }
        } else {
            float top[2], scale[2];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                top[k] = 0.0f;
#pragma unroll
                for (int i = 0; i < V; ++i)
                    if (some(i)) {
                        v[k][i].again();
#pragma unroll
                        for (int e = 0; e < E; ++e)
                            if (full(i) || inside(i, e))
                                top[k] = max_nan(top[k], fabsf(affine_exact(v[k][i].get(e), mu[k], rstd[k], w[i][e], b[i][e])));
                    }
            }
            float top_half = group_max_2(top[0], top[1], red_max, g, p.group);
            spread_2(top_half, top);
            if (not_finite(top[0]) || not_finite(top[1])) {         // (the same for all of the group)
                float odd[2];
                odd[0] = sum_not_finite<T>(p, r, t, p.group);
                odd[1] = two ? sum_not_finite<T>(p, r + all, t, p.group) : 0.0f;
                Sum all_odd[2];
                spread_2(group_sum_2((Sum)odd[0], (Sum)odd[1], red_var, g, p.group), all_odd);     // (read before the barrier behind the maximum)
#pragma unroll
                for (int k = 0; k < 2; ++k)
                    if (all_odd[k] != (Sum)0) { mu[k] = (float)all_odd[k]; rstd[k] = top[k] = __int_as_float(0x7FC00000); }
                top_half = (threadIdx.x & 16) ? top[1] : top[0];
            }
            spread_2(actq::scale_of(top_half, 1e-5f), scale);
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                if (k && !two) continue;
                if (t == 0) { p.gamma[r + k * all] = top[k]; p.scale[r + k * all] = scale[k]; }
#pragma unroll
                for (int i = 0; i < V; ++i)
                    if (some(i)) {
                        v[k][i].again();        // computed again: kept, the values would take more registers than there are
                        float f[E];
#pragma unroll
                        for (int e = 0; e < E; ++e) f[e] = affine_exact(v[k][i].get(e), mu[k], rstd[k], w[i][e], b[i][e]);
                        int8_t *out = p.q + (long long)(r + k * all) * n + c0 + i * hop;
                        if (full(i) && wide_q) {
                            store_codes<E>(out, f, scale[k]);
                        } else {
#pragma unroll
                            for (int e = 0; e < E; ++e)
                                if (inside(i, e)) out[e] = actq::quantise_one(f[e], scale[k]);
                        }
                    }
            }
        }
        if (t == 0) {
#pragma unroll
            for (int k = 0; k < 2; ++k)
                if (k == 0 || two) {
                    if (p.mean) p.mean[r + k * all] = mu[k];
                    if (p.rstd) p.rstd[r + k * all] = rstd[k];
                }
        }
    }
}

// ---- forward: a warp per short row ----------------------------------------------------------------------------
// V pieces a lane, in registers, and with up to two the next row's too (25088 x 192 float32 9.7 us, 11.3 without; 16384 x 1024
// float16, where four run out of registers, 16.6, 14.2 without); the parameters in shared memory as in the next kernel.  (A bulk
// copy of a row of a kilobyte costs more than its loads: 25088 x 192 float32, 14.3 us through shared memory.)
template <class T, int V, bool CODES>
__global__ void __launch_bounds__(1024, 1)
forward_short_kernel(const Fwd p)
{
    using Sum = typename std::conditional<CODES, double, float>::type;
    constexpr int E = kWide<T>;
    constexpr bool kAhead = V <= 2;
    extern __shared__ __align__(16) float short_params[];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, n = p.n, m = (int)p.m, pieces = n / E;
    float *sw = short_params, *sb = short_params + n;
    ptx::grid_dep_wait();
    ptx::grid_dep_launch();
    const Sum inv_n = (Sum)1 / (Sum)n;
    Piece<T, E> next[V];
    auto load = [&](long long r) {
        const T *row = static_cast<const T *>(p.x) + r * p.x_pitch;
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (r < m && lane + 32 * i < pieces) next[i].load(row + (lane + 32 * i) * E);
    };
    if constexpr (kAhead) load((long long)warp * gridDim.x + blockIdx.x);
    stage_parameters<E>(p, sw, sb);
    __syncthreads();
#pragma unroll 1
    for (long long r = (long long)warp * gridDim.x + blockIdx.x; r < m; r += 32ll * gridDim.x) {
        Piece<T, E> v[V];
        if constexpr (!kAhead) load(r);
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = next[i];
        if constexpr (kAhead) load(r + 32ll * gridDim.x);
        Sum s = 0;
        Two t = both(0.0f);
#pragma unroll
        for (int i = 0; i < V; ++i)
#pragma unroll
            for (int e = 0; e < E; e += 2) {    // (what lies past the row is zero)
                if constexpr (CODES) s = fma(scaled_down<T>(v[i].get(e + 1)), two_896(), fma(scaled_down<T>(v[i].get(e)), two_896(), s));
                else t = t + v[i].two(e);
            }
        if constexpr (!CODES) s = t.x + t.y;
        const Sum mean = quotient(warp_sum(s), (Sum)n, inv_n);
        s = 0;
        t = both(0.0f);
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (lane + 32 * i < pieces) {
                v[i].again();
#pragma unroll
                for (int e = 0; e < E; e += 2) {
                    if constexpr (CODES) {
                        const double d = fma(scaled_down<T>(v[i].get(e)), two_896(), -mean), d2 = fma(scaled_down<T>(v[i].get(e + 1)), two_896(), -mean);
                        s = fma(d2, d2, fma(d, d, s));
                    } else {
                        const Two d = v[i].two(e) + both(-mean);
                        t = fma_of(d, d, t);
                    }
                }
            }
        if constexpr (!CODES) s = t.x + t.y;
        float mu = (float)mean, rstd = inverse_root(quotient(warp_sum(s), (Sum)n, inv_n), p.eps);
        if constexpr (!CODES) {
            T *out = static_cast<T *>(p.y) + r * p.y_pitch;
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (lane + 32 * i < pieces) {
                    float w[E], b[E];
                    parameters_of<E>(sw, sb, pieces, lane + 32 * i, w, b);
                    v[i].again();
#pragma unroll
                    for (int e = 0; e < E; e += 2) {
                        const Two y = fma_of((v[i].two(e) + both(-mu)) * both(rstd), Two{w[e], w[e + 1]}, Two{b[e], b[e + 1]});
                        w[e] = y.x;
                        w[e + 1] = y.y;
                    }
                    v[i].set(w);
                    v[i].store(out + (lane + 32 * i) * E);
                }
        } else {
            float y[V][E], top = 0.0f;
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (lane + 32 * i < pieces) {
                    float w[E], b[E];
                    parameters_of<E>(sw, sb, pieces, lane + 32 * i, w, b);
#pragma unroll
                    for (int e = 0; e < E; ++e) {
                        y[i][e] = affine_exact(v[i].get(e), mu, rstd, w[e], b[e]);
                        top = max_nan(top, fabsf(y[i][e]));
                    }
                }
            top = warp_max(top);
            if (not_finite(top)) {
                const float odd = warp_sum(sum_not_finite<T>(p, r, lane, 32));
                if (odd != 0.0f) { mu = odd; rstd = top = __int_as_float(0x7FC00000); }
            }
            const float sc = actq::scale_of(top, 1e-5f);
            if (lane == 0) { p.gamma[r] = top; p.scale[r] = sc; }
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (lane + 32 * i < pieces) store_codes<E>(p.q + r * n + (lane + 32 * i) * E, y[i], sc);
        }
        if (lane == 0) {
            if (p.mean) p.mean[r] = mu;
            if (p.rstd) p.rstd[r] = rstd;
        }
    }
}

// ---- forward: a warp per row ------------------------------------------------------------------------------
// For many rows of whole pieces.  No exchange between warps, and what belongs to a row worked out once for all of it.  A bulk
// copy brings the row into shared memory, where the warp passes over it three times (four for codes): in registers the
// longer rows leave none for the arithmetic (16 pieces a lane with the next row's copy beside all of it: 62 us against 53.9,
// in spilled registers).  As many warps as there is room for rows; while one waits for its row the
// others work, and the row behind comes to L2 meanwhile (8192 x 4096 bf16 30.8 us, 33.9 without; to codes 42.4, 45.7).
template <class T, bool CODES>
__global__ void __launch_bounds__(1024, 1)
forward_warps_kernel(const Fwd p)
{
    using Sum = typename std::conditional<CODES, double, float>::type;
    constexpr int E = kWide<T>;
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ __align__(8) uint64_t bars[32];
    __shared__ volatile int failed;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, n = p.n, m = (int)p.m, pieces = n / E;
    const int own = (int)blockDim.x >> 5, warps = (int)gridDim.x * own;
    const uint32_t row_bytes = (uint32_t)n * (uint32_t)sizeof(T);
    float *sw = reinterpret_cast<float *>(smem), *sb = sw + n;      // (n is a multiple of E: both 16-byte aligned)
    const uint4 *mine = reinterpret_cast<const uint4 *>(smem + (size_t)n * 8 + (size_t)warp * row_bytes);
    const uint32_t mine_addr = ptx::smem_u32(mine), bar = ptx::smem_u32(bars) + 8u * warp;
    if (lane == 0) { ptx::mbar_init(bar, 1); ptx::mbar_init_fence(); }
    if (threadIdx.x == 0) failed = 0;
    ptx::grid_dep_wait();
    ptx::grid_dep_launch();
    const T *x = static_cast<const T *>(p.x);
    auto fetch = [&](long long r) {
        ptx::mbar_expect_tx(bar, row_bytes);
        ptx::bulk_load(mine_addr, x + r * p.x_pitch, row_bytes, bar);
    };
    long long r = (long long)warp * gridDim.x + blockIdx.x;        // (the last rows go round the SMs)
    if (lane == 0 && r < m) fetch(r);
    stage_parameters<E>(p, sw, sb);
    __syncthreads();
    auto parameters = [&](int piece, float (&w)[E], float (&b)[E]) { parameters_of<E>(sw, sb, pieces, piece, w, b); };
    const Sum inv_n = (Sum)1 / (Sum)n;
    uint32_t phase = 0;
#pragma unroll 1
    for (; r < m; r += warps, phase ^= 1u) {
        if (!ptx::mbar_try_wait(bar, phase)) {
            const unsigned long long t0 = ptx::globaltimer();
            while (!ptx::mbar_try_wait(bar, phase))
                if (failed || ptx::globaltimer() - t0 > actq::kWaitLimitNs) { failed = 1; break; }
        }
        if (__any_sync(0xFFFFFFFFu, failed)) break;
        if (lane == 0 && r + warps < m) ptx::bulk_prefetch(x + (r + warps) * p.x_pitch, row_bytes);
        Piece<T, E> v;
        Sum s = 0, s2 = 0;
        [[maybe_unused]] Sum sq = 0, sq2 = 0;
        Two t = both(0.0f);
#pragma unroll 4
        for (int i = lane; i < pieces; i += 32) {
            v.raw = mine[i];
#pragma unroll
            for (int e = 0; e < E; e += 2) {
                if constexpr (CODES) {
                    const double d = scaled_down<T>(v.get(e)) * two_896(), d2 = scaled_down<T>(v.get(e + 1)) * two_896();
                    s += d;
                    s2 += d2;
                    sq = fma(d, d, sq);
                    sq2 = fma(d2, d2, sq2);
                } else {
                    t = t + v.two(e);
                }
            }
        }
        if constexpr (!CODES) s = t.x + t.y;
        const Sum mean = quotient(warp_sum(s + s2), (Sum)n, inv_n);
        // In 64 bits the squares of the values can be summed on the same pass: what their difference to the mean's square loses is
        // seen, and where it is more than two or three bits the differences are taken after all, so that rstd is as near to its
        // value as every other kernel's.  (With twelve bits allowed, one row in a million of offsets of 20 to 60 spreads got
        // the neighbouring rstd.)
        Sum var = 0;
        bool again = true;
        if constexpr (CODES) {
            var = fma(-mean, mean, quotient(warp_sum(sq + sq2), (Sum)n, inv_n));
            again = !(var * 4.0 >= mean * mean);
        }
        if (again) {
            s = s2 = 0;
            t = both(0.0f);
#pragma unroll 4
            for (int i = lane; i < pieces; i += 32) {
                v.raw = mine[i];
#pragma unroll
                for (int e = 0; e < E; e += 2) {
                    if constexpr (CODES) {
                        const double d = fma(scaled_down<T>(v.get(e)), two_896(), -mean), d2 = fma(scaled_down<T>(v.get(e + 1)), two_896(), -mean);
                        s = fma(d, d, s);
                        s2 = fma(d2, d2, s2);
                    } else {
                        const Two d = v.two(e) + both(-mean);
                        t = fma_of(d, d, t);
                    }
                }
            }
            if constexpr (!CODES) s = t.x + t.y;
            var = quotient(warp_sum(s + s2), (Sum)n, inv_n);
        }
        float mu = (float)mean, rstd = inverse_root(var, p.eps);
        if constexpr (!CODES) {
            T *out = static_cast<T *>(p.y) + r * p.y_pitch;
#pragma unroll 2
            for (int i = lane; i < pieces; i += 32) {
                float w[E], b[E];
                parameters(i, w, b);
                v.raw = mine[i];
#pragma unroll
                for (int e = 0; e < E; e += 2) {
                    const Two y = fma_of((v.two(e) + both(-mu)) * both(rstd), Two{w[e], w[e + 1]}, Two{b[e], b[e + 1]});
                    w[e] = y.x;
                    w[e + 1] = y.y;
                }
                v.set(w);
                v.store(out + i * E);
            }
        } else {
            float top = 0.0f;
#pragma unroll 2
            for (int i = lane; i < pieces; i += 32) {
                float w[E], b[E];
                parameters(i, w, b);
                v.raw = mine[i];
#pragma unroll
                for (int e = 0; e < E; ++e) top = max_nan(top, fabsf(affine_exact(v.get(e), mu, rstd, w[e], b[e])));
            }
            top = warp_max(top);
            if (not_finite(top)) {
                const float odd = warp_sum(sum_not_finite<T>(p, r, lane, 32));
                if (odd != 0.0f) { mu = odd; rstd = top = __int_as_float(0x7FC00000); }
            }
            const float sc = actq::scale_of(top, 1e-5f);
            if (lane == 0) { p.gamma[r] = top; p.scale[r] = sc; }
            int8_t *out = p.q + r * n;
#pragma unroll 2
            for (int i = lane; i < pieces; i += 32) {
                float w[E], b[E];
                parameters(i, w, b);
                v.raw = mine[i];
#pragma unroll
                for (int e = 0; e < E; ++e) w[e] = affine_exact(v.get(e), mu, rstd, w[e], b[e]);
                store_codes<E>(out + i * E, w, sc);
            }
        }
        if (lane == 0) {
            if (p.mean) p.mean[r] = mu;
            if (p.rstd) p.rstd[r] = rstd;
        }
        __syncwarp();                           // the row has been read
        if (lane == 0 && r + warps < m) fetch(r + warps);
    }
    __syncthreads();
    if (failed) {
        // copies may be in flight yet: outwait them before the shared memory goes
        const unsigned long long t0 = ptx::globaltimer();
        while (ptx::globaltimer() - t0 < actq::kWaitLimitNs) {}
        if (threadIdx.x == 0) raise_status(PROM_ERR_TIMEOUT);
    }
}

// ---- forward: a block per row ---------------------------------------------------------------------------
// V accesses of E elements a thread, thread t takes accesses t, t + threads, ...
template <class T, int E, int V, bool CODES>
__global__ void __launch_bounds__(1024)
forward_kernel(const Fwd p)
{
    using Sum = typename std::conditional<CODES, double, float>::type;
    __shared__ Sum red[2][32];
    __shared__ float red_max[32];
    const int threads = (int)blockDim.x, t = (int)threadIdx.x;
    const long long r = blockIdx.x;
    ptx::grid_dep_wait();
    ptx::grid_dep_launch();
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
        for (int e = 0; e < E; ++e) {   // (what lies past the row is zero)
            if constexpr (CODES) s = fma(scaled_down<T>(v[i].get(e)), two_896(), s);
            else s += v[i].get(e);
        }
    s = block_sum(s, red[0]);
    const Sum mean = s / (Sum)p.n;
    s = 0;
#pragma unroll
    for (int i = 0; i < V; ++i)
        if (t + i * threads < pieces) {
            v[i].again();
#pragma unroll
            for (int e = 0; e < E; ++e) {
                Sum d;
                if constexpr (CODES) d = fma(scaled_down<T>(v[i].get(e)), two_896(), -mean);
                else d = v[i].get(e) - mean;
                s = fma(d, d, s);
            }
        }
    s = block_sum(s, red[1]);
    float rstd = inverse_root(s / (Sum)p.n, p.eps), mu = (float)mean;
    if constexpr (!CODES) {
        T *out = static_cast<T *>(p.y) + r * p.y_pitch;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int c = (t + i * threads) * E;
            if (t + i * threads < pieces) {
                float w[E], b[E];
                p.w.get<E>(c, 1.0f, w);
                p.b.get<E>(c, 0.0f, b);
                v[i].again();
#pragma unroll
                for (int e = 0; e < E; ++e) w[e] = (v[i].get(e) - mu) * rstd * w[e] + b[e];
                Piece<T, E> o;
                o.set(w);
                o.store(out + c);
            }
        }
    } else {
        // few values a thread are kept between the maximum and the codes, many are computed again
        constexpr bool kKeep = V * E <= 16;
        float y[kKeep ? V : 1][E], top = 0.0f;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int c = (t + i * threads) * E;
            if (t + i * threads < pieces) {
                float w[E], b[E];
                p.w.get<E>(c, 1.0f, w);
                p.b.get<E>(c, 0.0f, b);
                v[i].again();
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const float f = affine_exact(v[i].get(e), mu, rstd, w[e], b[e]);
                    if constexpr (kKeep) y[i][e] = f;
                    top = max_nan(top, fabsf(f));
                }
            }
        }
        top = block_max(top, red_max);
        if (not_finite(top)) {
            const Sum odd = block_sum((Sum)sum_not_finite<T>(p, r, t, threads), red[0]);       // (read before the last two barriers)
            if (odd != (Sum)0) { mu = (float)odd; rstd = top = __int_as_float(0x7FC00000); }
        }
        const float sc = actq::scale_of(top, 1e-5f);
        if (t == 0) { p.gamma[r] = top; p.scale[r] = sc; }
        int8_t *out = p.q + r * p.n;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int c = (t + i * threads) * E;
            if (t + i * threads < pieces) {
                if constexpr (kKeep) {
                    store_codes<E>(out + c, y[i], sc);
                } else {
                    float w[E], b[E], f[E];
                    p.w.get<E>(c, 1.0f, w);
                    p.b.get<E>(c, 0.0f, b);
                    v[i].again();
#pragma unroll
                    for (int e = 0; e < E; ++e) f[e] = affine_exact(v[i].get(e), mu, rstd, w[e], b[e]);
                    store_codes<E>(out + c, f, sc);
                }
            }
        }
    }
    if (t == 0) {
        if (p.mean) p.mean[r] = mu;
        if (p.rstd) p.rstd[r] = rstd;
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
    const float rstd = inverse_root(s / (Sum)p.n, p.eps);
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
    int period;             // rows after which the offset from a 16-byte boundary repeats
    int stages;             // rows of each group's ring
};

constexpr int kMaxGroups = 32;
constexpr int kMaxStages = 16;              // rows of a group's ring
// Two pieces a thread, and two rows at a time out of the ring (one, with the next one on its way, without it): what a row costs
// beside its values, the exchange and the addresses, is then spread over 16 or 32 of them, and the column sums (2 V E),
// weights and rows still fit the registers.  More pieces: one row at a time.
constexpr int kBwdThreads = 512;             // (768 with fewer registers: 25088 x 960 float32 72 us instead of 52)
template <int V, bool RING> constexpr int kBwdRows = V <= 2 && RING ? 2 : 1;

// RING: rows come through shared memory by bulk copies (whole 16-byte pieces), else by plain loads.
// Shared memory: the rings ([groups][stages][2][row bytes]), used again at the end for the groups' column sums.
template <class T, int E, int V, bool RING>
__global__ void __launch_bounds__(kBwdThreads, 1)
backward_kernel(const Bwd p)
{
    constexpr int R = kBwdRows<V, RING>;
    constexpr bool kShift = !RING && E > 1;     // rows may start anywhere
    constexpr bool kHoldW = V * E <= 16;
    constexpr int kStep = E > 1 ? 2 : 1;
    using Some = typename std::conditional<(E > 1), Two, float>::type;
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ __align__(8) uint64_t bars[RING ? kMaxGroups * kMaxStages : 1];
    __shared__ float4 red[2][32];
    __shared__ volatile int failed;
    const int g = (int)threadIdx.x / p.group, t = (int)threadIdx.x - g * p.group;
    const int lane = threadIdx.x & 31, warps = p.group >> 5, first_warp = g * warps;
    const int n = p.n, m = (int)p.m;
    const uint32_t row_bytes = (uint32_t)n * (uint32_t)sizeof(T);
    const uint32_t ring = ptx::smem_u32(smem) + (uint32_t)(g * p.stages) * 2u * row_bytes + (uint32_t)t * 16u;
    const uint32_t bar0 = ptx::smem_u32(bars) + 8u * (uint32_t)(g * p.stages);
    const int step = (int)gridDim.x * p.groups / p.period * p.period;
    const int r0 = g * (int)gridDim.x + (int)blockIdx.x < step ? g * (int)gridDim.x + (int)blockIdx.x : m;      // (the last rows go round the SMs)
    const T *x = static_cast<const T *>(p.x), *dy = static_cast<const T *>(p.dy);
    const int c0 = t * E - (kShift && r0 < m ? offset_of<T>(x + r0 * p.x_pitch) : 0), hop = p.group * E;
    // access i has columns c0 + i hop .. + E - 1
    auto in_row = [&](int i) { return kShift ? c0 + i * hop + E > 0 && c0 + i * hop < n : c0 + i * hop < n; };

    if (RING) {
        if (t < p.stages) ptx::mbar_init(bar0 + 8u * t, 1);
        ptx::mbar_init_fence();
    }
    if (threadIdx.x == 0) failed = 0;
    __syncthreads();
    ptx::grid_dep_wait();
    ptx::grid_dep_launch();
    auto fetch = [&](uint32_t s, long long r) {      // by one thread of the group (t == 0)
        ptx::mbar_expect_tx(bar0 + 8u * s, 2u * row_bytes);
        ptx::bulk_load(ring + s * 2u * row_bytes, x + r * p.x_pitch, row_bytes, bar0 + 8u * s);
        ptx::bulk_load(ring + s * 2u * row_bytes + row_bytes, dy + r * p.dy_pitch, row_bytes, bar0 + 8u * s);
    };
    long long ahead = r0;                       // the next row to fetch (kept by that thread)
    if (RING && t == 0)
        for (int s = 0; s < p.stages && ahead < m; ++s, ahead += step) fetch((uint32_t)s, ahead);

    float held[kHoldW ? V : 1][E], dw[V][E], db[V][E];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        if constexpr (kHoldW) p.w.get_at<E>(c0 + i * hop, n, 1.0f, held[i]);
#pragma unroll
        for (int e = 0; e < E; ++e) dw[i][e] = db[i][e] = 0.0f;
    }
    const float inv_n = 1.0f / (float)n;
    float next_mean[R], next_rstd[R];           // of the rows behind the current ones: not waited for
    auto statistics = [&](int r) {
#pragma unroll
        for (int k = 0; k < R; ++k) {
            const bool there = k == 0 ? r < m : step < m - r;
            next_mean[k] = there ? __ldg(p.mean + r + k * step) : 0.0f;
            next_rstd[k] = there ? __ldg(p.rstd + r + k * step) : 0.0f;
        }
    };
    statistics(r0);
    Piece<T, E> next_x[RING ? 1 : V], next_d[RING ? 1 : V];
    auto load = [&](int r) {
#pragma unroll
        for (int i = 0; i < (RING ? 1 : V); ++i)
            if (r < m && in_row(i)) {
                const T *xr = x + r * p.x_pitch, *dr = dy + r * p.dy_pitch;
                if constexpr (kShift) {
                    load_at(next_x[i], xr, c0 + i * hop, n);
                    load_at(next_d[i], dr, c0 + i * hop, n);
                } else {
                    next_x[i].load(xr + c0 + i * hop);
                    next_d[i].load(dr + c0 + i * hop);
                }
            }
    };
    if constexpr (!RING) load(r0);
    uint32_t s = 0, phase = 0;                  // the ring's stage of the first row
    int which = 0;
    T *out = static_cast<T *>(p.dx) + (r0 < m ? r0 * p.dx_pitch : 0) + c0;
    const long long out_step = (long long)step * p.dx_pitch;
#pragma unroll 1
    for (int r = r0; r < m;) {
        const bool two = R == 2 && step < m - r;
        const int after = (R == 2 ? two && step < m - r - step : step < m - r) ? r + R * step : m;
        float mean[R], rstd[R], s1[R], s2[R];   // sums of g and of g xh
        Piece<T, E> vx[R][V], vd[R][V];
#pragma unroll
        for (int k = 0; k < R; ++k) { mean[k] = next_mean[k]; rstd[k] = next_rstd[k]; }
        statistics(after);
        if constexpr (RING) {
#pragma unroll
            for (int k = 0; k < R; ++k)
                if (k == 0 || two) {
                    // A wait that runs out is the last one: the block goes on without waiting, so that its barriers stay in
                    // step, fetches nothing more and reports at the end.
                    const uint32_t st = s + k < (uint32_t)p.stages ? s + k : 0u, ph = s + k < (uint32_t)p.stages ? phase : phase ^ 1u;
                    if (!ptx::mbar_try_wait(bar0 + 8u * st, ph)) {
                        const unsigned long long t0 = ptx::globaltimer();
                        while (!ptx::mbar_try_wait(bar0 + 8u * st, ph))
                            if (failed || ptx::globaltimer() - t0 > actq::kWaitLimitNs) { failed = 1; break; }
                    }
                    const uint32_t at = ring + st * 2u * row_bytes;
#pragma unroll
                    for (int i = 0; i < V; ++i)
                        if (in_row(i)) {
                            vx[k][i].load_shared(at + (uint32_t)(i * p.group) * 16u);
                            vd[k][i].load_shared(at + row_bytes + (uint32_t)(i * p.group) * 16u);
                        }
                }
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i) { vx[0][i] = next_x[RING ? 0 : i]; vd[0][i] = next_d[RING ? 0 : i]; }
            load(after);
        }
        // Columns beside the row have a zero gradient and, as they were loaded, zero as x.  Where a large mean makes their xh infinite
        // the product of both would be NaN: such a row's take one of its values.
        if constexpr (kShift)
            if (!(fabsf(mean[0] * rstd[0]) <= 3.402823466e38f)) {
#pragma unroll
                for (int i = 0; i < V; ++i)
                    if (in_row(i)) fill_outside(vx[0][i], c0 + i * hop, n);
            }
#pragma unroll
        for (int k = 0; k < R; ++k) {
            Some t1 = all<Some>(0.0f), t2 = t1;
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (in_row(i)) {
                    float w[E];
                    if constexpr (!kHoldW) p.w.get_at<E>(c0 + i * hop, n, 1.0f, w);
#pragma unroll
                    for (int e = 0; e < E; e += kStep) {       // (a row that is not there is one of zeros, as is dy outside a row)
                        const Some we = some<Some>(kHoldW ? held[kHoldW ? i : 0] : w, e);
                        const Some d = some<Some>(vd[k][i], e), xh = (some<Some>(vx[k][i], e) + all<Some>(-mean[k])) * all<Some>(rstd[k]), gr = d * we;
                        t1 = t1 + gr;
                        t2 = fma_of(gr, xh, t2);
                        put(dw[i], e, fma_of(d, xh, some<Some>(dw[i], e)));
                        put(db[i], e, some<Some>(db[i], e) + d);
                    }
                }
            s1[k] = sum_of(t1);
            s2[k] = sum_of(t2);
        }
        float v = R == 2 ? warp_sum_4(s1[0], s2[0], s1[R - 1], s2[R - 1]) : warp_sum_2(s1[0], s2[0]);
        constexpr int kValues = 2 * R, kSpan = 32 / kValues;
        if (warps > 1) {
            if ((lane & (kSpan - 1)) == 0) reinterpret_cast<float *>(&red[which][threadIdx.x >> 5])[lane / kSpan] = v;
            group_barrier(g, p.group);
            // every thread of the group has read its part of the stages, so they can be filled again
            const float4 a = lane < warps ? red[which][first_warp + lane] : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            v = R == 2 ? warp_sum_4(a.x, a.y, a.z, a.w) : warp_sum_2(a.x, a.y);
            which ^= 1;                         // the next rows' sums go elsewhere: these may still be read
        } else {
            __syncwarp();
        }
        v = quotient(v, (float)n, inv_n);
#pragma unroll
        for (int k = 0; k < R; ++k) {
            s1[k] = __shfl_sync(0xFFFFFFFFu, v, 2 * k * kSpan);
            s2[k] = __shfl_sync(0xFFFFFFFFu, v, (2 * k + 1) * kSpan);
        }
        if (RING) {
            if (t == 0 && !failed) {
#pragma unroll
                for (int k = 0; k < R; ++k)
                    if (ahead < m) { fetch(s + k < (uint32_t)p.stages ? s + k : 0u, ahead); ahead += step; }
            }
            s += R;
            if (s >= (uint32_t)p.stages) { s -= (uint32_t)p.stages; phase ^= 1u; }
        }
        if (p.dx) {
#pragma unroll
            for (int k = 0; k < R; ++k)
                if (k == 0 || two) {
#pragma unroll
                    for (int i = 0; i < V; ++i)
                        if (in_row(i)) {
                            float w[E];
                            if constexpr (!kHoldW) p.w.get_at<E>(c0 + i * hop, n, 1.0f, w);
                            vx[k][i].again();
                            vd[k][i].again();
#pragma unroll
                            for (int e = 0; e < E; e += kStep) {
                                const Some we = some<Some>(kHoldW ? held[kHoldW ? i : 0] : w, e);
                                const Some xh = (some<Some>(vx[k][i], e) + all<Some>(-mean[k])) * all<Some>(rstd[k]);
                                put(w, e, all<Some>(rstd[k]) * fma_of(xh, all<Some>(-s2[k]), fma_of(some<Some>(vd[k][i], e), we, all<Some>(-s1[k]))));
                            }
                            Piece<T, E> o;
                            o.set(w);
                            if constexpr (kShift) store_at<T, E>(o, out + k * out_step - c0, c0 + i * hop, n);
                            else o.store(out + k * out_step + i * hop);
                        }
                }
            out += R * out_step;
        }
        r = after;
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

    // The groups' column sums side by side ([groups][2][n_pad]), then added in the order of the groups; all copies have landed
    // and been read.
    float *acc = reinterpret_cast<float *>(smem), *own = acc + (size_t)g * 2 * p.n_pad;
#pragma unroll
    for (int i = 0; i < V; ++i)
        if (g < p.groups && in_row(i)) {
            const int c = c0 + i * hop;
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (!kShift || (c + e >= 0 && c + e < n)) {
                    own[c + e] = dw[i][e];
                    own[p.n_pad + c + e] = db[i][e];
                }
        }
    __syncthreads();
    float *mine = p.part + (size_t)blockIdx.x * 2 * p.n_pad;
    for (int c = threadIdx.x; c < 2 * p.n_pad; c += blockDim.x) {
        float a = 0.0f;
        if ((c < p.n_pad ? c : c - p.n_pad) < n)
            for (int k = 0; k < p.groups; ++k) a += acc[(size_t)k * 2 * p.n_pad + c];
        mine[c] = a;
    }
}

// Rows of any length: dx by a block per row, behind the column sums of a slice of rows by a block per 256 columns.
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

// The column sums of such rows, launched in front of backward_long_kernel, which may write dx in the place of dy or x: that one
// waits for this one's end.
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

// The sums over the blocks' partial sums: 32 warps share 128 columns, each every 32nd block, then one adds the 32.
constexpr int kSumWarps = 32;
__global__ void __launch_bounds__(32 * kSumWarps)
backward_sum_kernel(const float *__restrict__ part, int blocks, int n, int n_pad, void *dw, void *db, int type)
{
    __shared__ float4 s[kSumWarps][32];
    ptx::grid_dep_wait();
    ptx::grid_dep_launch();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int c = blockIdx.x * 128 + lane * 4;          // of the 2 n_pad columns
    float4 a = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    if (c < 2 * n_pad) {
#pragma unroll 8
        for (int k = warp; k < blocks; k += kSumWarps) {
            const float4 v = *reinterpret_cast<const float4 *>(part + (size_t)k * 2 * n_pad + c);
            a.x += v.x; a.y += v.y; a.z += v.z; a.w += v.w;
        }
    }
    s[warp][lane] = a;
    __syncthreads();
    if (warp || c >= 2 * n_pad) return;
#pragma unroll
    for (int k = 1; k < kSumWarps; ++k) { const float4 v = s[k][lane]; a.x += v.x; a.y += v.y; a.z += v.z; a.w += v.w; }
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
