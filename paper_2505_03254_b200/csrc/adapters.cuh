// A ternary projection with the low-rank adapters of many requests beside it: for row r of sample s,
//     f = max(gamma[s], 1e-5) / 127,  a = adapter_of_sample[s],
//     y[r][o] = (sum_k x[r][k] W-hat[o][k]) alpha[o] f  +  scale[a] f sum_j B[a][o][j] (sum_k A[a][j][k] x[r][k])
// The weights are frozen 2-bit codes, so what differs between requests is a product of two thin matrices.  The inner
// products t[r][j] = sum_k A[a][j][k] x[r][k] come from a kernel of their own in front, the projection adds the
// outer ones in its epilogue: y is written once, and the adapters' part is never a tensor of y's size.
#pragma once

#include "common.cuh"
#include "layernorm.cuh"
#include "ptx.cuh"

namespace prom { namespace lora {

struct Params {
    const int8_t *x;
    long long m, rows_per_sample;
    int cin, cout;
    const uint8_t *w;
    const float *alpha, *gamma;
    const void *a, *b;              // nullptr: no adapters
    const float *scale;             // [n] or nullptr: 1
    const int32_t *which;           // [batch]
    int n, rank;
    void *y;
    long long y_pitch;
    float *t;                       // [m][rank] inner products (few rows)
    int chained;                    // a kernel of the same call is in front: only what that one writes is waited for
};

__device__ __forceinline__ float row_factor(const Params &p, long long s)
{
    const float g = __ldg(p.gamma + s);
    return __fdiv_rn(g < 1e-5f ? 1e-5f : g, 127.0f);        // (a NaN stays one)
}

// The adapter of a sample, -1 for none.  An index that is outside the table counts as none and is reported.
__device__ __forceinline__ int adapter_of(const Params &p, long long s)
{
    if (!p.a) return -1;
    const int a = __ldg(p.which + s);
    if (a >= -1 && a < p.n) return a;
    raise_status(PROM_ERR_RANGE);
    return -1;
}

// Two neighbouring 16-bit values of one word.
template <class H> __device__ __forceinline__ float2 unpack_2(uint32_t w);
template <> __device__ __forceinline__ float2 unpack_2<__nv_bfloat16>(uint32_t w)
{
    return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
}
template <> __device__ __forceinline__ float2 unpack_2<__half>(uint32_t w) { return __half22float2(*reinterpret_cast<const __half2 *>(&w)); }

// The i-th signed byte of a word as a float.
__device__ __forceinline__ float byte_float(uint32_t w, int i) { return (float)(int8_t)(w >> (8 * i)); }

// ---- few rows: inner products, a warp per (row, j) -------------------------------------------------------
// Bound by latency: a row's A is rank x cin 16-bit values out of L2 or HBM.
template <class H>
__global__ void __launch_bounds__(256)
inner_rows_kernel(const Params p)
{
    ptx::grid_dep_wait();
    ptx::grid_dep_launch();
    const long long r = blockIdx.x;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, j = blockIdx.y * 8 + warp;
    const int a = adapter_of(p, r / p.rows_per_sample);
    if (a < 0 || j >= p.rank) return;
    const uint4 *x = reinterpret_cast<const uint4 *>(p.x + r * p.cin);
    const uint4 *av = reinterpret_cast<const uint4 *>(static_cast<const H *>(p.a) + ((size_t)a * p.rank + j) * p.cin);
    float sum = 0.0f;
#pragma unroll 4
    for (int k = lane; k < p.cin / 16; k += 32) {
        const uint4 xv = __ldg(x + k), a0 = __ldg(av + 2 * k), a1 = __ldg(av + 2 * k + 1);
        const uint32_t xw[4] = {xv.x, xv.y, xv.z, xv.w}, aw[8] = {a0.x, a0.y, a0.z, a0.w, a1.x, a1.y, a1.z, a1.w};
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float2 f = unpack_2<H>(aw[i]);
            sum = fmaf(f.x, byte_float(xw[i >> 1], 2 * (i & 1)), sum);
            sum = fmaf(f.y, byte_float(xw[i >> 1], 2 * (i & 1) + 1), sum);
        }
    }
    sum = norm::warp_sum(sum);
    if (lane == 0) p.t[r * p.rank + j] = sum;
}

// sum_j B[a][o][j] t[j].  A value of B that is not finite counts as zero and is reported (many rows share a tile of B,
// where infinity times another row's zero would spread).
template <class H> __device__ __forceinline__ float finite(float v, bool &bad)
{
    const bool ok = fabsf(v) <= 3.402823466e38f;
    bad |= !ok;
    return ok ? v : 0.0f;
}
template <class H>
__device__ __forceinline__ float outer(const Params &p, int a, int o, const float *t, bool &bad)
{
    const H *b = static_cast<const H *>(p.b) + ((size_t)a * p.cout + o) * p.rank;
    float s = 0.0f;
    if ((p.rank & 7) == 0) {
        for (int j = 0; j < p.rank; j += 8) {
            const uint4 v = __ldg(reinterpret_cast<const uint4 *>(b + j));
            const float4 t0 = *reinterpret_cast<const float4 *>(t + j), t1 = *reinterpret_cast<const float4 *>(t + j + 4);
            const uint32_t w[4] = {v.x, v.y, v.z, v.w};
            const float tt[8] = {t0.x, t0.y, t0.z, t0.w, t1.x, t1.y, t1.z, t1.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float2 f = unpack_2<H>(w[i]);
                s = fmaf(finite<H>(f.x, bad), tt[2 * i], s);
                s = fmaf(finite<H>(f.y, bad), tt[2 * i + 1], s);
            }
        }
    } else {
        for (int j = 0; j < p.rank; ++j) s = fmaf(finite<H>(norm::to_float(b[j]), bad), t[j], s);
    }
    return s;
}

// ---- few rows: the projection -------------------------------------------------------------------------------
// D[16 outputs][8 rows] += W[16][32] x[32][8] with the warp-level int8 MMA: the weights' bytes, a quarter of one per
// product, are what has to be read, and with few rows the tensor memory path has nothing to amortise its set-up on.
// A block takes 16 MO outputs and 8 MT rows, its eight warps share K in pieces of 256.
// Codes become operands in three operations per 16: two's complement codes with the upper bit flipped are w + 2, and
// (word >> 2 j) & 0x03030303 are the values k = j, 4 + j, 8 + j, 12 + j of the word's 16.  The rows' bytes are put in the same
// order by transposing their 4 x 4 blocks, and 2 sum_k x is taken off at the end.
__device__ __forceinline__ void mma_u8s8(int (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k32.row.col.s32.u8.s8.s32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+r"(d[0]), "+r"(d[1]), "+r"(d[2]), "+r"(d[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// Byte i of word j of `v` to byte j of word i.
__device__ __forceinline__ void transpose_4x4(const uint4 &v, uint32_t (&o)[4])
{
    const uint32_t lo01 = __byte_perm(v.x, v.y, 0x5140), hi01 = __byte_perm(v.x, v.y, 0x7362);
    const uint32_t lo23 = __byte_perm(v.z, v.w, 0x5140), hi23 = __byte_perm(v.z, v.w, 0x7362);
    o[0] = __byte_perm(lo01, lo23, 0x5410);
    o[1] = __byte_perm(lo01, lo23, 0x7632);
    o[2] = __byte_perm(hi01, hi23, 0x5410);
    o[3] = __byte_perm(hi01, hi23, 0x7632);
}

constexpr int kRowWarps = 8;

template <class H, class Y, int MO, int MT>
__global__ void __launch_bounds__(32 * kRowWarps)
proj_rows_kernel(const Params p)
{
    __shared__ int acc_s[kRowWarps][16 * MO][8 * MT + 1];
    __shared__ int sum_s[kRowWarps][8 * MT];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int o0 = blockIdx.x * 16 * MO;
    const long long r0 = (long long)blockIdx.y * 8 * MT;
    const int rowb = p.cin >> 2;
    const bool wide = (rowb & 15) == 0;
    if (!p.chained) ptx::grid_dep_wait();
    ptx::grid_dep_launch();

    int d[MO][MT][4], sx[MT];
#pragma unroll
    for (int i = 0; i < MT; ++i) {
        sx[i] = 0;
#pragma unroll
        for (int o = 0; o < MO; ++o)
#pragma unroll
            for (int e = 0; e < 4; ++e) d[o][i][e] = 0;
    }
    uint32_t invalid = 0;
    for (int k0 = warp * 256; k0 < p.cin; k0 += 256 * kRowWarps) {
        const int k = k0 + 64 * t;              // this thread's 64 of the piece
        uint32_t w[MO][2][4];
#pragma unroll
        for (int o = 0; o < MO; ++o)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int row = o0 + 16 * o + 8 * h + g;
                const uint8_t *src = p.w + (size_t)row * rowb + (k >> 2);
                if (row < p.cout && wide && k < p.cin) {
                    const uint4 v = __ldg(reinterpret_cast<const uint4 *>(src));
                    w[o][h][0] = v.x; w[o][h][1] = v.y; w[o][h][2] = v.z; w[o][h][3] = v.w;
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        w[o][h][i] = row < p.cout && k + 16 * i < p.cin ? __ldg(reinterpret_cast<const uint32_t *>(src) + i) : 0u;
                }
            }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint32_t b[MT][4];
#pragma unroll
            for (int c = 0; c < MT; ++c) {
                const long long r = r0 + 8 * c + g;
                uint4 v = make_uint4(0u, 0u, 0u, 0u);
                if (r < p.m && k + 16 * i < p.cin) v = __ldg(reinterpret_cast<const uint4 *>(p.x + r * p.cin + k + 16 * i));
                transpose_4x4(v, b[c]);
#pragma unroll
                for (int j = 0; j < 4; ++j) sx[c] = __dp4a((int)b[c][j], 0x01010101, sx[c]);
            }
#pragma unroll
            for (int o = 0; o < MO; ++o) {
                invalid |= ((w[o][0][i] >> 1) & ~w[o][0][i] & 0x55555555u) | ((w[o][1][i] >> 1) & ~w[o][1][i] & 0x55555555u);
                const uint32_t lo = w[o][0][i] ^ 0xAAAAAAAAu, hi = w[o][1][i] ^ 0xAAAAAAAAu;
                uint32_t al[4], ah[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) { al[j] = (lo >> (2 * j)) & 0x03030303u; ah[j] = (hi >> (2 * j)) & 0x03030303u; }
#pragma unroll
                for (int c = 0; c < MT; ++c) {
                    mma_u8s8(d[o][c], al[0], ah[0], al[1], ah[1], b[c][0], b[c][1]);
                    mma_u8s8(d[o][c], al[2], ah[2], al[3], ah[3], b[c][2], b[c][3]);
                }
            }
        }
    }
    if (invalid && blockIdx.y == 0) raise_status(PROM_ERR_BAD_WEIGHT);
#pragma unroll
    for (int c = 0; c < MT; ++c) {
        sx[c] += __shfl_xor_sync(0xFFFFFFFFu, sx[c], 1);
        sx[c] += __shfl_xor_sync(0xFFFFFFFFu, sx[c], 2);
        if (t == 0) sum_s[warp][8 * c + g] = sx[c];
#pragma unroll
        for (int o = 0; o < MO; ++o)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc_s[warp][16 * o + g + 8 * (e >> 1)][8 * c + 2 * t + (e & 1)] = d[o][c][e];
    }
    __syncthreads();
    if (p.chained) ptx::grid_dep_wait();        // for the inner products
    bool bad = false;
    for (int i = threadIdx.x; i < 16 * MO * 8 * MT; i += 32 * kRowWarps) {
        const int o = i % (16 * MO), c = i / (16 * MO);
        const long long r = r0 + c;
        if (r >= p.m || o0 + o >= p.cout) continue;
        int acc = 0;
#pragma unroll
        for (int w = 0; w < kRowWarps; ++w) acc += acc_s[w][o][c] - 2 * sum_s[w][c];
        const long long s = r / p.rows_per_sample;
        const float f = row_factor(p, s);
        float y = (float)acc * __ldg(p.alpha + o0 + o) * f;
        const int a = adapter_of(p, s);
        if (a >= 0) y += (p.scale ? __ldg(p.scale + a) : 1.0f) * f * outer<H>(p, a, o0 + o, p.t + r * p.rank, bad);
        static_cast<Y *>(p.y)[r * p.y_pitch + o0 + o] = norm::from_float<Y>(y);
    }
    if (bad) raise_status(PROM_ERR_BAD_WEIGHT);
}

}}  // namespace prom::lora
