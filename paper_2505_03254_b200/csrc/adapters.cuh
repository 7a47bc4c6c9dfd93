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
#include "wide.cuh"

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
    // Many rows: the inner products as sums of `terms` 16-bit values, [m][terms][pitch] (pitch: rank rounded up to 16, zeros
    // behind it), divided by a power of two per row; the rows' adapters; and per tile of 256 rows the number of its adapters
    // and these.
    void *t16;
    float *power;
    int *list, *row_adapter;
    int pitch, terms;
    int chained;                    // a kernel of the same call is in front: only what that one writes is waited for
};

__device__ __forceinline__ int sample_of(const Params &p, long long r)     // (both below 2^31)
{
    return p.rows_per_sample == 1 ? (int)r : (int)((uint32_t)r / (uint32_t)p.rows_per_sample);
}
__device__ __forceinline__ float factor_of(float gamma) { return __fdiv_rn(gamma < 1e-5f ? 1e-5f : gamma, 127.0f); }     // (a NaN stays one)

// The adapter of a sample, -1 for none.  An index that is outside the table counts as none and is reported.
__device__ __forceinline__ int adapter_of(const Params &p, int s)
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
// Bound by latency: a row's A is rank x cin 16-bit values out of L2 or HBM (32 rows 4096 -> 4096, rank 16: the call takes 9.2 us
// with the kernel below, that one alone 5.9; their bytes, 2 us).
template <class H>
__global__ void __launch_bounds__(1024)
inner_rows_kernel(const Params p)
{
    ptx::grid_dep_wait();
    ptx::grid_dep_launch();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const long long i = (long long)blockIdx.x * (blockDim.x >> 5) + warp, r = i / p.rank;
    const int j = (int)(i - r * p.rank);
    if (r >= p.m) return;
    const int a = adapter_of(p, sample_of(p, r));
    if (a < 0) return;
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
// The first sixteen values of a row of B, which can be on their way before the inner products are there.
struct Ahead {
    uint4 v[2];
    template <class H> __device__ __forceinline__ void load(const Params &p, int a, int o)
    {
        if (p.rank & 7) return;
        const uint4 *b = reinterpret_cast<const uint4 *>(static_cast<const H *>(p.b) + ((size_t)a * p.cout + o) * p.rank);
        v[0] = __ldg(b);
        if (p.rank > 8) v[1] = __ldg(b + 1);
    }
};
template <class H> __device__ __forceinline__ float outer_8(const uint4 &v, const float *t, float s, bool &bad)
{
    const float4 t0 = *reinterpret_cast<const float4 *>(t), t1 = *reinterpret_cast<const float4 *>(t + 4);
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    const float tt[8] = {t0.x, t0.y, t0.z, t0.w, t1.x, t1.y, t1.z, t1.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = unpack_2<H>(w[i]);
        s = fmaf(finite<H>(f.x, bad), tt[2 * i], s);
        s = fmaf(finite<H>(f.y, bad), tt[2 * i + 1], s);
    }
    return s;
}
template <class H>
__device__ __forceinline__ float outer(const Params &p, int a, int o, const float *t, const Ahead &ahead, bool &bad)
{
    const H *b = static_cast<const H *>(p.b) + ((size_t)a * p.cout + o) * p.rank;
    float s = 0.0f;
    if ((p.rank & 7) == 0) {
        s = outer_8<H>(ahead.v[0], t, s, bad);
        if (p.rank > 8) s = outer_8<H>(ahead.v[1], t + 8, s, bad);
#pragma unroll 4
        for (int j = 16; j < p.rank; j += 8) s = outer_8<H>(__ldg(reinterpret_cast<const uint4 *>(b + j)), t + j, s, bad);
    } else {
        for (int j = 0; j < p.rank; ++j) s = fmaf(finite<H>(norm::to_float(b[j]), bad), t[j], s);
    }
    return s;
}

// ---- few rows: the projection -------------------------------------------------------------------------------
// D[16 outputs][8 rows] += W[16][32] x[32][8] with the warp-level int8 MMA: the weights' bytes, a quarter of one per
// product, are what has to be read, and with few rows the tensor memory path has nothing to amortise its set-up on.
// A block takes 16 MO outputs and 8 MT rows; its warps split K into pieces of 64 PW values.  Latency is the bound, so there
// are as many of them as leave a piece or two to each, and what the epilogue needs beside the sums is loaded in front of them.
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

// PW: words of 16 codes that a thread takes of each weight row.  The four threads of a fragment's row lie side by side in
// memory, 64 values of k apart from one word to the next.
template <class H, class Y, int MO, int MT, int PW, int WARPS>
__global__ void __launch_bounds__(32 * WARPS, (MT == 1 ? 2 : 1) * (WARPS == 8 ? 2 : 1))
proj_rows_kernel(const Params p)
{
    constexpr int kPitch = 16 * MO + 4;         // of a row's outputs: a warp's additions fall into different banks
    __shared__ int acc_s[8 * MT * kPitch], sum_s[8 * MT];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int o0 = blockIdx.x * 16 * MO;
    const long long r0 = (long long)blockIdx.y * 8 * MT;
    const int rowb = p.cin >> 2;
    for (int i = threadIdx.x; i < 8 * MT * kPitch; i += 32 * WARPS) acc_s[i] = 0;
    if (threadIdx.x < 8 * MT) sum_s[threadIdx.x] = 0;
    if (!p.chained) ptx::grid_dep_wait();
    ptx::grid_dep_launch();
    __syncthreads();

    // what an output needs beside the sums, on its way before them
    constexpr int kEach = (128 * MO * MT + 32 * WARPS - 1) / (32 * WARPS);      // outputs of a thread
    float alpha[kEach], gamma[kEach];
    int a[kEach];
    auto output = [&](int q, int &o, long long &r) {
        const int i = threadIdx.x + q * 32 * WARPS;
        o = o0 + i % (16 * MO);
        r = r0 + i / (16 * MO);
        return i < 128 * MO * MT && r < p.m && o < p.cout;
    };
#pragma unroll
    for (int q = 0; q < kEach; ++q) {
        int o;
        long long r;
        a[q] = -1;
        alpha[q] = gamma[q] = 0.0f;
        if (output(q, o, r)) {
            const int s = sample_of(p, r);
            alpha[q] = __ldg(p.alpha + o);
            gamma[q] = __ldg(p.gamma + s);
            a[q] = adapter_of(p, s);
        }
    }

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
    for (int k0 = warp * 64 * PW; k0 < p.cin; k0 += 64 * PW * WARPS) {
        const int k = k0 + 16 * t;              // this thread's words: k, k + 64, ...
        uint32_t w[MO][2][PW];
#pragma unroll
        for (int o = 0; o < MO; ++o)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int row = o0 + 16 * o + 8 * h + g;
                const uint8_t *src = p.w + (size_t)row * rowb + (k >> 2);
#pragma unroll
                for (int i = 0; i < PW; ++i)
                    w[o][h][i] = row < p.cout && k + 64 * i < p.cin ? __ldg(reinterpret_cast<const uint32_t *>(src + 16 * i)) : 0u;
            }
        uint4 v[MT][PW];
#pragma unroll
        for (int c = 0; c < MT; ++c) {
            const long long r = r0 + 8 * c + g;
            const int8_t *src = p.x + r * p.cin + k;
#pragma unroll
            for (int i = 0; i < PW; ++i) {
                v[c][i] = make_uint4(0u, 0u, 0u, 0u);
                if (r < p.m && k + 64 * i < p.cin) v[c][i] = __ldg(reinterpret_cast<const uint4 *>(src + 64 * i));
            }
        }
#pragma unroll
        for (int i = 0; i < PW; ++i) {
            uint32_t b[MT][4];
#pragma unroll
            for (int c = 0; c < MT; ++c) {
                transpose_4x4(v[c][i], b[c]);
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
    // B while the warps' sums are added (whole numbers: in any order)
    Ahead ahead[kEach];
#pragma unroll
    for (int q = 0; q < kEach; ++q) {
        int o;
        long long r;
        if (a[q] >= 0 && output(q, o, r)) ahead[q].template load<H>(p, a[q], o);
    }
#pragma unroll
    for (int c = 0; c < MT; ++c) {
        sx[c] += __shfl_xor_sync(0xFFFFFFFFu, sx[c], 1);
        sx[c] += __shfl_xor_sync(0xFFFFFFFFu, sx[c], 2);
        if (t == 0) atomicAdd(&sum_s[8 * c + g], sx[c]);
#pragma unroll
        for (int o = 0; o < MO; ++o)
#pragma unroll
            for (int e = 0; e < 4; ++e) atomicAdd(&acc_s[(8 * c + 2 * t + (e & 1)) * kPitch + 16 * o + g + 8 * (e >> 1)], d[o][c][e]);
    }
    __syncthreads();
    if (p.chained) ptx::grid_dep_wait();        // for the inner products
    bool bad = false;
#pragma unroll
    for (int q = 0; q < kEach; ++q) {
        int o;
        long long r;
        if (!output(q, o, r)) continue;
        const int c = (int)(r - r0), acc = acc_s[c * kPitch + o - o0] - 2 * sum_s[c];
        const float f = factor_of(gamma[q]);
        float y = (float)acc * alpha[q] * f;
        if (a[q] >= 0) y += (p.scale ? __ldg(p.scale + a[q]) * f : f) * outer<H>(p, a[q], o, p.t + r * p.rank, ahead[q], bad);
        static_cast<Y *>(p.y)[r * p.y_pitch + o] = norm::from_float<Y>(y);
    }
    if (bad) raise_status(PROM_ERR_BAD_WEIGHT);
}

// ---- many rows: inner products ----------------------------------------------------------------------------------
// Rows in tiles of 256.  A block sorts the tile's rows by their adapter (a row's place is the number of smaller keys), so
// that rows of one adapter need not stand side by side: an item is up to 32 of the tile's rows of one adapter, and the items go
// round the blocks of a tile.  What counts is the adapters in a tile, here and in the projection behind.  K comes in stages of 256 (128 from 48 ranks on) by asynchronous copies of 16 bytes (a bulk copy
// per row and rank took twice as long: they are a few hundred bytes each); each of the eight warps multiplies an eighth of
// them with the warp-level 16-bit MMA, rows as A (int8 values are exact in both 16-bit types) and the adapter as B, and the
// warps' sums are added at the end.  A thread's 4 KS bytes of a row and 8 KS of the adapter are neighbouring values of k,
// whose order inside the MMAs is free.  The sums are then split into 16-bit values once, for all the projection's tiles of outputs.
constexpr int kTile = 256;
constexpr int kItemRows = 32;
constexpr int kListInts = kTile + 1;
constexpr int kInnerWarps = 8;
constexpr int kRankPart = 64;               // ranks of one pass over K
constexpr int kInnerThreads = 32 * kInnerWarps;
constexpr int kInnerStages = 4;
// KS: MMA steps (16 values of k) per warp and stage.
static __host__ __device__ constexpr int inner_ks(int r) { return r >= 48 ? 1 : 2; }
static __host__ __device__ constexpr uint32_t x_pitch(int ks) { return 144u * ks; }     // bytes: a warp's accesses fall into
static __host__ __device__ constexpr uint32_t a_pitch(int ks) { return 288u * ks; }     // different banks

// Four int8 values (one word) to two words of 16-bit values: 0, 1 and 2, 3.
template <class H> __device__ __forceinline__ void widen_4(uint32_t w, uint32_t &lo, uint32_t &hi);
template <> __device__ __forceinline__ void widen_4<__half>(uint32_t w, uint32_t &lo, uint32_t &hi)
{
    // 1024 + u has u = x + 128 in its low byte
    const uint32_t u = w ^ 0x80808080u, base = 0x64646464u;
    const uint32_t a = __byte_perm(u, base, 0x4140), b = __byte_perm(u, base, 0x4342), off = 0x64806480u;     // 1024 + 128
    const __half2 x = __hsub2(*reinterpret_cast<const __half2 *>(&a), *reinterpret_cast<const __half2 *>(&off));
    const __half2 y = __hsub2(*reinterpret_cast<const __half2 *>(&b), *reinterpret_cast<const __half2 *>(&off));
    lo = *reinterpret_cast<const uint32_t *>(&x);
    hi = *reinterpret_cast<const uint32_t *>(&y);
}
template <> __device__ __forceinline__ void widen_4<__nv_bfloat16>(uint32_t w, uint32_t &lo, uint32_t &hi)
{
    // 128 + (x & 127) minus 128, or minus 256 where the sign is set: all three are bfloat16 values
    const uint32_t base = 0x43434343u;
    const uint32_t a = __byte_perm(w, base, 0x4140), b = __byte_perm(w, base, 0x4342);
    const uint32_t an = a & 0xFF7FFF7Fu, as = a & 0xFF80FF80u, bn = b & 0xFF7FFF7Fu, bs = b & 0xFF80FF80u;
    const __nv_bfloat162 x = __hsub2(*reinterpret_cast<const __nv_bfloat162 *>(&an), *reinterpret_cast<const __nv_bfloat162 *>(&as));
    const __nv_bfloat162 y = __hsub2(*reinterpret_cast<const __nv_bfloat162 *>(&bn), *reinterpret_cast<const __nv_bfloat162 *>(&bs));
    lo = *reinterpret_cast<const uint32_t *>(&x);
    hi = *reinterpret_cast<const uint32_t *>(&y);
}
template <class H> __device__ __forceinline__ void mma_16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1);
template <> __device__ __forceinline__ void mma_16<__nv_bfloat16>(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
template <> __device__ __forceinline__ void mma_16<__half>(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// The power of two by which a row's inner products are divided, so that the largest lies in [2^13, 2^14): far from both ends
// of the 16-bit types.  1 for a row of (nearly) zeros or one that has a value which is not finite.
__device__ __forceinline__ float row_power(float top, float &inverse)
{
    const uint32_t e = (__float_as_uint(top) >> 23) & 0xFFu;
    const bool plain = e <= 14u || e == 255u;
    inverse = plain ? 1.0f : __uint_as_float((267u - e) << 23);        // 2^(13 + 127 - e), down to 2^-113
    return plain ? 1.0f : __uint_as_float((e - 13u) << 23);
}

// Shared memory: the stages (rows, then ranks), afterwards the warps' sums [warp][row][kPartPitch]; behind them the item's
// sums [row][pitch].
constexpr int kPartPitch = kRankPart + 1;
static __host__ __device__ constexpr uint32_t inner_stage(int r) { return kItemRows * x_pitch(inner_ks(r)) + (uint32_t)r * a_pitch(inner_ks(r)); }
static __host__ __device__ constexpr uint32_t inner_sums_at(int r)
{
    return kInnerStages * inner_stage(r) > kInnerWarps * kItemRows * kPartPitch * 4u ? kInnerStages * inner_stage(r)
                                                                                    : kInnerWarps * kItemRows * kPartPitch * 4u;
}
static constexpr size_t inner_smem(int r, int pitch) { return inner_sums_at(r) + (size_t)kItemRows * pitch * sizeof(float); }

// R: ranks of a pass, the pitch up to 64.
template <class H, int R>
__global__ void __launch_bounds__(kInnerThreads, 2)
inner_tiles_kernel(const Params p)
{
    extern __shared__ __align__(16) uint8_t smem[];
    float *part = reinterpret_cast<float *>(smem), *sums = reinterpret_cast<float *>(smem + inner_sums_at(R));
    __shared__ __align__(16) int key_s[kTile];
    __shared__ int sorted_s[kTile + 1];         // adapter << 8 | row
    __shared__ unsigned start_s[kTile / 32];    // places where another adapter begins
    __shared__ int item_s[kTile];               // first place | rows << 16
    __shared__ int warp_items[kTile / 32], warp_lists[kTile / 32];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
    const long long tile = blockIdx.x, first = tile * kTile;
    ptx::grid_dep_wait();
    ptx::grid_dep_launch();

    // rows without an adapter come last (adapters are below 2^20)
    constexpr int kNone = 1 << 20;
    const int mine = first + tid < p.m ? adapter_of(p, sample_of(p, first + tid)) : -1;
    const int key = (mine < 0 ? kNone : mine) << 8 | tid;
    key_s[tid] = key;
    if (blockIdx.y == 0 && first + tid < p.m) p.row_adapter[first + tid] = mine;
    __syncthreads();
    int place = 0;
#pragma unroll 8
    for (int i = 0; i < kTile; i += 4) {
        const int4 k = *reinterpret_cast<const int4 *>(key_s + i);
        place += (k.x < key) + (k.y < key) + (k.z < key) + (k.w < key);
    }
    sorted_s[place] = key;
    if (tid == 0) sorted_s[kTile] = -1;         // (an adapter that no row has)
    __syncthreads();
    // from here on a thread is a place
    const int a_here = sorted_s[tid] >> 8;
    const bool start = tid == 0 || (sorted_s[tid - 1] >> 8) != a_here;
    const unsigned starts = __ballot_sync(0xFFFFFFFFu, start);
    if (lane == 0) start_s[warp] = starts;
    __syncthreads();
    const unsigned upto = 0xFFFFFFFFu >> (31 - lane), below = upto >> 1;
    int begin;                                  // of this place's adapter
    {
        int w = warp;
        unsigned mask = starts & upto;
        while (!mask) mask = start_s[--w];      // (place 0 is a start)
        begin = 32 * w + 31 - __clz(mask);
    }
    const bool real = a_here != kNone, head = real && (tid - begin) % kItemRows == 0, newcomer = real && start;
    const unsigned heads = __ballot_sync(0xFFFFFFFFu, head), news = __ballot_sync(0xFFFFFFFFu, newcomer);
    if (lane == 0) { warp_items[warp] = __popc(heads); warp_lists[warp] = __popc(news); }
    __syncthreads();
    int items = 0, before = 0, adapters = 0, list_before = 0;
    for (int w = 0; w < kTile / 32; ++w) {
        if (w == warp) { before = items; list_before = adapters; }
        items += warp_items[w];
        adapters += warp_lists[w];
    }
    if (head) {
        int n = 1;
        while (n < kItemRows && (sorted_s[tid + n] >> 8) == a_here) ++n;
        item_s[before + __popc(heads & below)] = tid | (n << 16);
    }
    if (blockIdx.y == 0) {
        int *list = p.list + tile * kListInts;
        if (newcomer) list[1 + list_before + __popc(news & below)] = a_here;
        if (tid == 0) list[0] = adapters;
    }
    __syncthreads();

    constexpr int KS = inner_ks(R), kInnerK = 16 * KS * kInnerWarps, kXRows = 32 / KS, kARows = 16 / KS, kACopies = R / kARows;
    constexpr uint32_t kXPitch = x_pitch(KS), kAPitch = a_pitch(KS), stage_bytes = inner_stage(R);
    const uint32_t base = ptx::smem_u32(smem);
    const int steps = (p.cin + kInnerK - 1) / kInnerK;
    for (int it = blockIdx.y; it < items; it += gridDim.y) {
        const int at = item_s[it] & 0xFFFF, count = item_s[it] >> 16;
        const int a = sorted_s[at] >> 8;
        for (int j0 = 0; j0 < p.pitch; j0 += R) {
            // Copies: KS pieces of 16 bytes of the rows and R KS / 16 of the ranks per thread and stage, zeros past cin.  Rows past
            // the item's and ranks past the adapter's repeat the last one: they end in sums that are not used.
            const int xk = 16 * (tid % (8 * KS)), ak = 8 * (tid % (16 * KS)), xrow = tid / (8 * KS), arow = tid / (16 * KS);
            const int8_t *xsrc[KS];
            const H *asrc[kACopies];
#pragma unroll
            for (int i = 0; i < KS; ++i) {
                const int row = xrow + kXRows * i;
                xsrc[i] = p.x + (first + (sorted_s[at + (row < count ? row : count - 1)] & 255)) * p.cin + xk;
            }
#pragma unroll
            for (int i = 0; i < kACopies; ++i) {
                const int j = j0 + arow + kARows * i;
                asrc[i] = static_cast<const H *>(p.a) + ((size_t)a * p.rank + (j < p.rank ? j : p.rank - 1)) * p.cin + ak;
            }
            const uint32_t xdst = base + (uint32_t)xrow * kXPitch + (uint32_t)xk;
            const uint32_t adst = base + kItemRows * kXPitch + (uint32_t)arow * kAPitch + 2u * ak;
            int k_next = 0;
            uint32_t to = 0;
            auto fetch = [&] {
                if (k_next + kInnerK <= p.cin) {
#pragma unroll
                    for (int i = 0; i < KS; ++i) ptx::cp_async_16(xdst + to + (uint32_t)(kXRows * i) * kXPitch, xsrc[i] + k_next);
#pragma unroll
                    for (int i = 0; i < kACopies; ++i) ptx::cp_async_16(adst + to + (uint32_t)(kARows * i) * kAPitch, asrc[i] + k_next);
                } else if (k_next < p.cin) {
                    const bool xin = k_next + xk < p.cin, ain = k_next + ak < p.cin;
#pragma unroll
                    for (int i = 0; i < KS; ++i)
                        ptx::cp_async_16_or_zero(xdst + to + (uint32_t)(kXRows * i) * kXPitch, xin ? xsrc[i] + k_next : p.x, xin);
#pragma unroll
                    for (int i = 0; i < kACopies; ++i)
                        ptx::cp_async_16_or_zero(adst + to + (uint32_t)(kARows * i) * kAPitch, ain ? (const void *)(asrc[i] + k_next) : p.a, ain);
                }
                k_next += kInnerK;
                to = to + stage_bytes == kInnerStages * stage_bytes ? 0u : to + stage_bytes;
                ptx::cp_async_commit();         // (an empty group where there is no stage: the waits count groups)
            };
            float acc[2][R / 8][4];             // [16 rows][8 ranks][...]
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < R / 8; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[i][j][e] = 0.0f;
#pragma unroll
            for (int i = 0; i < kInnerStages - 1; ++i) fetch();
            uint32_t st = 0;
            for (int step = 0; step < steps; ++step) {
                ptx::cp_async_wait<kInnerStages - 2>();
                __syncthreads();                // the stage is there, and the one before it has been read
                fetch();
                const uint8_t *sx = smem + st * stage_bytes + KS * (16 * warp + 4 * t);
                const uint8_t *sa = smem + st * stage_bytes + kItemRows * kXPitch + KS * (32 * warp + 8 * t);
                uint2 b[R / 8][KS];
#pragma unroll
                for (int j = 0; j < R / 8; ++j) {
                    if constexpr (KS == 2) {
                        const uint4 v = *reinterpret_cast<const uint4 *>(sa + (uint32_t)(8 * j + g) * kAPitch);
                        b[j][0] = make_uint2(v.x, v.y);
                        b[j][1] = make_uint2(v.z, v.w);
                    } else {
                        b[j][0] = *reinterpret_cast<const uint2 *>(sa + (uint32_t)(8 * j + g) * kAPitch);
                    }
                }
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    uint32_t xv[2][KS];
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const uint8_t *src = sx + (uint32_t)(16 * i + 8 * h + g) * kXPitch;
                        if constexpr (KS == 2) {
                            const uint2 v = *reinterpret_cast<const uint2 *>(src);
                            xv[h][0] = v.x;
                            xv[h][1] = v.y;
                        } else {
                            xv[h][0] = *reinterpret_cast<const uint32_t *>(src);
                        }
                    }
#pragma unroll
                    for (int s = 0; s < KS; ++s) {
                        uint32_t f[4];
                        widen_4<H>(xv[0][s], f[0], f[2]);
                        widen_4<H>(xv[1][s], f[1], f[3]);
#pragma unroll
                        for (int j = 0; j < R / 8; ++j) mma_16<H>(acc[i][j], f, b[j][s].x, b[j][s].y);
                    }
                }
                st = (st + 1) % kInnerStages;
            }
            ptx::cp_async_wait<0>();
            __syncthreads();                    // the sums take the stages' place
            float *own = part + (size_t)warp * kItemRows * kPartPitch;
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < R / 8; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) own[(16 * i + g + 8 * (e >> 1)) * kPartPitch + 8 * j + 2 * t + (e & 1)] = acc[i][j][e];
            __syncthreads();
            for (int i = tid; i < count * R; i += kInnerThreads) {
                const int k = i / R, j = i % R;
                float s = 0.0f;
#pragma unroll
                for (int w = 0; w < kInnerWarps; ++w) s += part[(w * kItemRows + k) * kPartPitch + j];
                if (j0 + j < p.pitch) sums[k * p.pitch + j0 + j] = j0 + j < p.rank ? s : 0.0f;
            }
            __syncthreads();
        }
        // eight lanes a row: the power, and the 16-bit values
        const int k = tid >> 3, q = tid & 7;
        const float *v = sums + (k < count ? k : 0) * p.pitch;
        float top = 0.0f;
        for (int j = q; j < p.pitch; j += 8) top = norm::max_nan(top, fabsf(v[j]));
#pragma unroll
        for (int d = 4; d > 0; d >>= 1) top = norm::max_nan(top, __shfl_xor_sync(0xFFFFFFFFu, top, d));
        if (k < count) {
            float by;
            const float power = row_power(top, by);
            const long long r = first + (sorted_s[at + k] & 255);
            if (q == 0) p.power[r] = power;
            uint32_t *out = static_cast<uint32_t *>(p.t16) + (size_t)r * p.terms * (p.pitch / 2);
            for (int j = q; j < p.pitch / 2; j += 8) {
                float lo = v[2 * j] * by, hi = v[2 * j + 1] * by;
                for (int m = 0; m < p.terms; ++m) {
                    out[m * (p.pitch / 2) + j] = norm::pack_pair<H>(lo, hi);
                    lo -= norm::to_float(norm::from_float<H>(lo));
                    hi -= norm::to_float(norm::from_float<H>(hi));
                }
            }
        }
        __syncthreads();
    }
}

// ---- many rows: the projection -------------------------------------------------------------------------------------
// Tiles of 256 rows x nt outputs by pairs of CTAs (cta_group::2, 128 rows of x and half of the tile's weights in each),
// accumulators of two kinds in tensor memory: int32 for the projection, binary32 for the adapters, which the epilogue joins;
// two of each where they fit (without adapters, and up to 128 outputs), so that a tile is read out beside the next one's MMAs.
// x comes by TMA.  The weights never exist as bytes in memory: eight warps expand the 2-bit codes into the swizzled
// operand layout on their way into shared memory (four pairs of warps take the stages in turn), so a stage takes 4 KB of
// weights from L2 instead of 16 (a pair's SM would need 64 bytes a clock of both operands at the MMAs' rate, of the 58 that L2
// gives it; this way it is 40).
// 8192 rows 4096 -> 4096 with adapters of rank 64 take 148 us (170 in long runs, under the power cap), of which the inner
// products in front take 29; without adapters 98 (2.8 POPS of 4.56).  Bound by the stages' rate, 0.4 us each where their MMAs
// take 0.3; which part of a stage holds it there has not been measured by itself.  Narrower tiles with two accumulators of
// each kind take longer (160 outputs 201 us, 128 outputs 223, when 256 took 154), and twice as many fillers on half as
// many epilogue warps gain 2 % there, so that the expansion is not all of it, and lose 10 % at 1024 -> 4096.
// Behind the chunks of K come those of the adapters: for each adapter of the tile the rows' inner products (zero for rows of
// other adapters), as sums of 16-bit values (three, or two float16 ones for 16-bit outputs) side by side along K, against B
// repeated as often.  An adapter costs the tile that many stages however few of its rows have it: 512 rows 4096 -> 4096 of rank
// 16 take 33 us with two adapters and 40 with eight, of rank 64 50 and 74.
constexpr int kFillGroups = 4, kGroupWarps = 2, kFillWarps = kFillGroups * kGroupWarps;
constexpr int kEpiGroups = 4, kEpiWarps = 4 * kEpiGroups;
constexpr int kFill0 = 2, kEpi0 = kFill0 + kFillWarps;
constexpr int kTileThreads = 32 * (kEpi0 + kEpiWarps);
constexpr uint32_t kHalfStage = 128u * 128u, kStage = 2u * kHalfStage;      // rows of x, rows of weights: 128 bytes of K each
// As many stages as fit beside the epilogue warps' slabs of 32 rows x 32 outputs.  A group of fillers that has entered a stage
// knows that the one kStages before it is done: its next one, kFillGroups further, must not lie a whole round beyond that,
// or its wait could not tell the phase before from the one it needs.
template <class Y> struct TileLayout {
    static constexpr int kStages = sizeof(Y) == 4 ? 5 : 6;
    static constexpr uint32_t kSlab = 32u * 32u * (uint32_t)sizeof(Y);
    static constexpr uint32_t kOffSlab = kStages * kStage;
    static constexpr uint32_t kOffBars = kOffSlab + kEpiWarps * kSlab;
    static constexpr size_t kSmem = 1024 + kOffBars + 256;
    static_assert(kFillGroups <= kStages, "waits of the fillers");
    static_assert(kSmem <= 227 * 1024, "shared memory");
};

struct Tiles {
    Params p;
    int kc, ksteps_last;        // chunks of 128 bytes of K; MMA steps in the last one
    int n_mtiles, n_ctiles, nt;
    int depth;                  // accumulators of each kind, nt columns each: the projection's, then the adapters'
    int store;                  // y has a tensor map
};

// 16 codes to 16 bytes in order (invalid ones become -2).
__device__ __forceinline__ uint4 expand_16(uint32_t w)
{
    const uint32_t even = w & 0x33333333u, odd = (w >> 2) & 0x33333333u, lut = 0xFFFE0100u;
    const uint32_t e0 = __byte_perm(lut, 0u, even), e1 = __byte_perm(lut, 0u, even >> 16);
    const uint32_t o0 = __byte_perm(lut, 0u, odd), o1 = __byte_perm(lut, 0u, odd >> 16);
    return make_uint4(__byte_perm(e0, o0, 0x5140), __byte_perm(e0, o0, 0x7362), __byte_perm(e1, o1, 0x5140), __byte_perm(e1, o1, 0x7362));
}

template <class H, class Y>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kTileThreads, 1)
proj_tiles_kernel(const __grid_constant__ CUtensorMap xmap, const __grid_constant__ CUtensorMap ymap, const Tiles q)
{
    constexpr int kStages = TileLayout<Y>::kStages;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = smem_raw + ((1024u - (ptx::smem_u32(smem_raw) & 1023u)) & 1023u);
    const uint32_t base = ptx::smem_u32(smem);
    const int warp = ptx::warp_index(), lane = threadIdx.x & 31;
    const uint32_t rank = ptx::cluster_rank();
    const Params &p = q.p;

    // In the first CTA: full (its loader's arrival, both CTAs' fillers and both loads' bytes) and tempty (both read-outs).
    // In each: empty and tfull, by the MMAs' completion.
    uint64_t *bars = reinterpret_cast<uint64_t *>(smem + TileLayout<Y>::kOffBars);
    const uint32_t bar_full = ptx::smem_u32(bars), bar_empty = bar_full + 8 * kStages;
    const uint32_t bar_tfull = bar_empty + 8 * kStages, bar_tempty = bar_tfull + 16, bar_drain = bar_tempty + 16;      // (two accumulators)
    volatile uint32_t *tmem_slot = reinterpret_cast<volatile uint32_t *>(bars + 2 * kStages + 5);
    volatile int *flags = reinterpret_cast<volatile int *>(bars + 2 * kStages + 6);

    const int pair = (int)blockIdx.x >> 1, pairs = (int)gridDim.x >> 1;
    const long long units = (long long)q.n_mtiles * q.n_ctiles;
    auto width = [&](int ct) { const int left = p.cout - ct * q.nt; return left >= q.nt ? q.nt : (left + 31) & ~31; };
    const int k2 = p.terms * p.pitch, per_adapter = (k2 + 63) >> 6;    // chunks of 64 values

    if (warp == 0) {
        if (lane < kStages) {
            ptx::mbar_init(bar_full + 8 * lane, 1 + 2 * kFillWarps);
            ptx::mbar_init(bar_empty + 8 * lane, 1);
        } else if (lane == 31) {
            for (int i = 0; i < 2; ++i) {
                ptx::mbar_init(bar_tfull + 8 * i, 1);
                ptx::mbar_init(bar_tempty + 8 * i, 2 * kEpiWarps);
            }
            ptx::mbar_init(bar_drain, 1);
            flags[0] = 0;
            ptx::tma_prefetch_desc(&xmap);
            if (q.store) ptx::tma_prefetch_desc(&ymap);
        }
        ptx::mbar_init_fence();
    }
    if (warp == 1) ptx::tmem_alloc_pair(ptx::smem_u32((const void *)tmem_slot), 512u);
    ptx::tc_fence_before_sync();
    __syncthreads();
    ptx::cluster_sync();
    ptx::tc_fence_after_sync();
    const uint32_t tmem = *tmem_slot;
    // What a kernel in front of this call wrote: with inner_tiles_kernel in between it is complete already.
    if (!p.chained) ptx::grid_dep_wait();
    ptx::grid_dep_launch();
    auto adapters_of_tile = [&](int mt) { return p.a ? __ldcg(p.list + (size_t)mt * kListInts) : 0; };

    if (warp == 0) {
        // ---- loader of x ----------------------------------------------------------------------------------
        const bool leader = ptx::elect_one();
        const uint32_t full = ptx::map_to_rank(bar_full, 0);
        uint32_t st = 0, ph = 0;
        bool ok = true, waited = !p.chained;
        for (long long u = pair; u < units && ok; u += pairs) {
            const int mt = (int)(u / q.n_ctiles);
            for (int c = 0; c < q.kc; ++c) {
                if (!tc::wait_bar_warp(bar_empty + 8 * st, ph ^ 1u, flags)) { ok = false; break; }
                if (leader) {
                    if (rank == 0) ptx::mbar_expect_tx(bar_full + 8 * st, 2u * kHalfStage);
                    ptx::tma_load_2d_pair(base + st * kStage, &xmap, c * 128, mt * kTile + (int)rank * 128, full + 8 * st);
                }
                if (++st == kStages) { st = 0; ph ^= 1u; }
            }
            if (!ok || !p.a) continue;
            // The adapters' stages are the fillers' alone, but each is waited for: a wait for a phase can not be told
            // from one for the phase two before it.
            if (!waited) { ptx::grid_dep_wait(); waited = true; }
            for (int c = adapters_of_tile(mt) * per_adapter; c > 0 && ok; --c) {
                ok = tc::wait_bar_warp(bar_empty + 8 * st, ph ^ 1u, flags);
                if (++st == kStages) { st = 0; ph ^= 1u; }
            }
        }
        // the completions of the last MMAs arrive here before the CTA may go away
        for (int s = 0; s < kStages && ok; ++s) {
            ok = tc::wait_bar_warp(bar_empty + 8 * st, ph ^ 1u, flags);
            if (++st == kStages) { st = 0; ph ^= 1u; }
        }
        if (!ok) wide::outwait_copies();
        __syncwarp();
    } else if (warp == 1) {
        // ---- MMA issuer: the first CTA's, for both ----------------------------------------------------------
        if (rank == 0) {
            const bool leader = ptx::elect_one();
            const uint64_t d_128 = tc::smem_desc(0u, 128u);
            const uint32_t a_lo0 = base >> 4, step = kStage >> 4, half = kHalfStage >> 4;
            constexpr uint32_t f16_types = std::is_same<H, __nv_bfloat16>::value ? (1u << 7) | (1u << 10) : 0u;
            uint32_t st = 0, ph = 0, done = 0;
            bool ok = true, waited = !p.chained;
            auto wait_full = [&] { return tc::wait_bar_warp(bar_full + 8 * st, ph, flags); };
            // for the read-out of the `n`-th unit of an accumulator, counted from 1 (0: returns at once)
            auto wait_read = [&](uint32_t buf, uint32_t n) { return tc::wait_bar_warp(bar_tempty + 8 * buf, (n & 1u) ^ 1u, flags); };
            for (long long u = pair; u < units && ok; u += pairs, ++done) {
                const int mt = (int)(u / q.n_ctiles), ct = (int)(u % q.n_ctiles);
                const uint32_t shape = (((uint32_t)width(ct) >> 3) << 17) | ((256u >> 4) << 24);
                const uint32_t id_i8 = (2u << 4) | (1u << 7) | (1u << 10) | shape, id_f16 = (1u << 4) | f16_types | shape;
                const uint32_t buf = q.depth == 2 ? done & 1u : 0u, use = q.depth == 2 ? done >> 1 : done;
                const uint32_t d1 = tmem + buf * (uint32_t)q.nt, d2 = d1 + (uint32_t)(q.depth * q.nt);
                if (!wait_read(buf, use)) { ok = false; break; }
                ptx::tc_fence_after_sync();
                for (int c = 0; c < q.kc; ++c) {
                    if (!wait_full()) { ok = false; break; }
                    ptx::tc_fence_after_sync();
                    const uint32_t a_lo = a_lo0 + st * step, b_lo = a_lo + half;
                    const int nks = c == q.kc - 1 ? q.ksteps_last : 4;
                    if (leader) {
                        if (c == 0) ptx::mma_i8_pair<false>(d1, d_128 | (uint64_t)a_lo, d_128 | (uint64_t)b_lo, id_i8);
                        else ptx::mma_i8_pair<true>(d1, d_128 | (uint64_t)a_lo, d_128 | (uint64_t)b_lo, id_i8);
#pragma unroll
                        for (int ks = 1; ks < 4; ++ks)
                            if (ks < nks)
                                ptx::mma_i8_pair<true>(d1, d_128 | (uint64_t)(a_lo + 2 * ks), d_128 | (uint64_t)(b_lo + 2 * ks), id_i8);
                        ptx::mma_commit_pair(bar_empty + 8 * st);
                    }
                    if (++st == kStages) { st = 0; ph ^= 1u; }
                }
                if (ok && p.a) {
                    if (!waited) { ptx::grid_dep_wait(); waited = true; }
                    const int chunks = adapters_of_tile(mt) * per_adapter;
                    for (int c = 0, part = 0; c < chunks; ++c) {
                        if (!wait_full()) { ok = false; break; }
                        ptx::tc_fence_after_sync();
                        const uint32_t a_lo = a_lo0 + st * step, b_lo = a_lo + half;
                        const int left = (k2 - 64 * part) >> 4, nks = left < 4 ? left : 4;
                        if (leader) {
                            for (int ks = 0; ks < nks; ++ks)
                                ptx::mma_f16_pair(d2, d_128 | (uint64_t)(a_lo + 2 * ks), d_128 | (uint64_t)(b_lo + 2 * ks), id_f16,
                                                  c || ks ? 1u : 0u);
                            ptx::mma_commit_pair(bar_empty + 8 * st);
                        }
                        if (++part == per_adapter) part = 0;
                        if (++st == kStages) { st = 0; ph ^= 1u; }
                    }
                }
                if (ok && leader) ptx::mma_commit_pair(bar_tfull + 8 * buf);
            }
            // the second CTA's read-outs arrive here
            for (uint32_t b = 0; ok && b < (uint32_t)q.depth; ++b) ok = wait_read(b, q.depth == 2 ? (done + 1u - b) >> 1 : done);
            if (leader) ptx::mma_commit_own(bar_drain);
            const unsigned long long t0 = ptx::globaltimer();
            while (!ptx::mbar_try_wait(bar_drain, 0) && ptx::globaltimer() - t0 < tc::kWaitLimitNs) {}
        }
        __syncwarp();
    } else if (warp < kEpi0) {
        // ---- fillers: weights, then the adapters' operands ----------------------------------------------------
        // The stages of all units are numbered through.  A group takes every fourth of those with weights (its arrival counts
        // for the others'), a thread four half rows of 64 bytes: rows row0, row0 + 32, ...  Those of the adapters, of which
        // there are few, all groups fill together, a group 32 rows.
        const int f = threadIdx.x - 32 * kFill0, grp = f / (32 * kGroupWarps), ft = f % (32 * kGroupWarps);
        const int row0 = ft >> 1, half = ft & 1;
        constexpr int kHop = 16 * kGroupWarps, kRows = 128 / kHop;          // weights: between a thread's rows, their number
        constexpr int kPerRow = kFillWarps / 4, kPieces = 8 / kPerRow;      // adapters: threads of a row, 16-byte pieces of each
        const uint32_t full = ptx::map_to_rank(bar_full, 0);
        const int rowb = p.cin >> 2;
        const bool wide_codes = (rowb & 15) == 0;
        uint32_t seq = 0, invalid = 0;          // number of the unit's first stage
        bool ok = true, waited = !p.chained, bad = false;
        auto enter = [&](uint32_t n) {
            return tc::wait_bar_warp(bar_empty + 8 * (n % kStages), ((n / kStages) & 1u) ^ 1u, flags);
        };
        // The operands that the arrival announces are read by the tensor cores of the SM that wrote them, and this SM's fence
        // stands before it: what crosses to the first CTA is the signal alone (mbar_arrive_cluster_n).  An arrival with
        // release.cluster orders the writes for the other CTA's threads too, which read none of them, and waits about a
        // microsecond: 8192 rows 4096 -> 4096 took 148 us instead of 115 with one in every filler, and 274 instead of 96 with
        // one warp that passed the fillers' word on.
        auto publish = [&](uint32_t n, uint32_t arrivals) {
            ptx::fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive_cluster_n(full + 8 * (n % kStages), arrivals);
        };
        for (long long u = pair; u < units && ok; u += pairs) {
            const int mt = (int)(u / q.n_ctiles), ct = (int)(u % q.n_ctiles);
            const int rows = width(ct) / 2, o0 = ct * q.nt + (int)rank * rows;
            uint32_t code[kRows][4];
            auto fetch = [&](int c) {
                const int k = c * 128 + half * 64;
#pragma unroll
                for (int i = 0; i < kRows; ++i) {
                    const int row = row0 + kHop * i;
                    const bool there = row < rows && o0 + row < p.cout;
                    const uint8_t *src = p.w + (size_t)(there ? o0 + row : 0) * rowb + c * 32 + half * 16;
                    if (wide_codes) {
                        uint4 w = make_uint4(0u, 0u, 0u, 0u);
                        if (there && k < p.cin) w = __ldg(reinterpret_cast<const uint4 *>(src));
                        code[i][0] = w.x; code[i][1] = w.y; code[i][2] = w.z; code[i][3] = w.w;
                    } else {
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            code[i][j] = there && k + 16 * j < p.cin ? __ldg(reinterpret_cast<const uint32_t *>(src) + j) : 0u;
                    }
                }
            };
            // the tile's adapters and this thread's row's own, looked up a whole pass over K before they are needed
            const int *list = p.list + (size_t)mt * kListInts;
            int chunks = 0, mine = -1, held[2];
            auto look = [&] {
                chunks = __ldcg(list) * per_adapter;
                held[0] = __ldcg(list + 1);         // (what lies past the number is not used)
                held[1] = __ldcg(list + 2);
                const long long r = (long long)mt * kTile + (int)rank * 128 + f / kPerRow;
                mine = r < p.m ? __ldcg(p.row_adapter + r) : -1;
            };
            if (p.a && waited) look();
            int c = (int)(((uint32_t)grp - seq) % kFillGroups);
            if (c < q.kc) fetch(c);
            for (; c < q.kc; c += kFillGroups) {
                const uint32_t n = seq + (uint32_t)c;
                if (!enter(n)) { ok = false; break; }
                uint8_t *dst = smem + (n % kStages) * kStage + kHalfStage;
#pragma unroll
                for (int i = 0; i < kRows; ++i)
                    if (row0 + kHop * i < rows) {
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            if (mt == 0) invalid |= (code[i][j] >> 1) & ~code[i][j] & 0x55555555u;     // (every tile of rows sees the same)
                            *reinterpret_cast<uint4 *>(dst + tc::swz_offset((uint32_t)(row0 + kHop * i), (uint32_t)(half * 4 + j), 128u)) = expand_16(code[i][j]);
                        }
                    }
                if (c + kFillGroups < q.kc) fetch(c + kFillGroups);
                publish(n, kFillGroups);
            }
            seq += (uint32_t)q.kc;
            if (!ok || !p.a) continue;
            if (!waited) { ptx::grid_dep_wait(); waited = true; look(); }
            const int row = f / kPerRow, first = f % kPerRow * kPieces;
            const long long r = (long long)mt * kTile + (int)rank * 128 + row;
            const bool there = row < rows && o0 + row < p.cout, wide_b = (p.rank & 7) == 0;
            const uint32_t off0 = tc::swz_offset((uint32_t)row, (uint32_t)first, 128u);       // piece k: off0 ^ 16 k
            // a chunk is announced while the next two's copies are on their way
            auto land = [&](uint32_t n) {
#pragma unroll
                for (int k = 0; k < kPieces; ++k) {       // what is not finite in B counts as zero
                    const uint32_t at = base + (n % kStages) * kStage + kHalfStage + (off0 ^ (16u * k));
                    const int4 v = ptx::lds_128(at);
                    uint32_t w[4] = {(uint32_t)v.x, (uint32_t)v.y, (uint32_t)v.z, (uint32_t)v.w};
                    constexpr uint32_t top = std::is_same<H, __nv_bfloat16>::value ? 0x7F80u : 0x7C00u;    // its exponent
                    bool hit = false;
#pragma unroll
                    for (int s = 0; s < 4; ++s) {
                        if ((w[s] & top) == top) { w[s] &= 0xFFFF0000u; hit = true; }
                        if (((w[s] >> 16) & top) == top) { w[s] &= 0x0000FFFFu; hit = true; }
                    }
                    if (hit) { bad = true; ptx::sts_128(at, w[0], w[1], w[2], w[3]); }
                }
                publish(n, f < 32 && rank == 0 ? 2u : 1u);      // (the loader's arrival among them)
            };
            for (int i_ad = 0, part = 0, c2 = 0; c2 < chunks; ++c2) {
                const uint32_t n = seq + (uint32_t)c2;
                const int a = i_ad == 0 ? held[0] : (i_ad == 1 ? held[1] : __ldcg(list + 1 + i_ad));
                const int e0 = part * 64 + first * 8;
                if (!enter(n)) { ok = false; break; }
                const uint32_t dst = base + (n % kStages) * kStage;
                const H *t16 = static_cast<const H *>(p.t16) + (size_t)(mine == a ? r : 0) * k2;
                const H *b = static_cast<const H *>(p.b) + ((size_t)a * p.cout + (there ? o0 + row : 0)) * p.rank;
#pragma unroll
                for (int k = 0; k < kPieces; ++k) {
                    const int e = e0 + 8 * k, j = e - (e >= p.pitch ? p.pitch : 0) - (e >= 2 * p.pitch ? p.pitch : 0);
                    const uint32_t off = off0 ^ (16u * k);
                    const bool t_in = e < k2 && mine == a, b_in = e < k2 && there && j < p.rank;
                    ptx::cp_async_16_or_zero(dst + off, t16 + (t_in ? e : 0), t_in);
                    if (wide_b) {
                        ptx::cp_async_16_or_zero(dst + kHalfStage + off, b + (b_in ? j : 0), b_in);
                    } else {
                        uint32_t w[4] = {0u, 0u, 0u, 0u};
#pragma unroll
                        for (int s = 0; s < 8; ++s)
                            if (b_in && j + s < p.rank) w[s >> 1] |= (uint32_t)__ldg(reinterpret_cast<const unsigned short *>(b) + j + s) << (16 * (s & 1));
                        ptx::sts_128(dst + kHalfStage + off, w[0], w[1], w[2], w[3]);
                    }
                }
                ptx::cp_async_commit();
                if (c2 > 1) {
                    ptx::cp_async_wait<2>();
                    land(n - 2);
                }
                if (++part == per_adapter) { part = 0; ++i_ad; }
            }
            ptx::cp_async_wait_all();
            if (ok && chunks > 1) land(seq + (uint32_t)chunks - 2);
            if (ok && chunks) land(seq + (uint32_t)chunks - 1);
            seq += (uint32_t)chunks;
        }
        if (invalid || bad) raise_status(PROM_ERR_BAD_WEIGHT);
        __syncwarp();
    } else {
        // ---- epilogue --------------------------------------------------------------------------------------------
        // Four groups of four warps, a warp per quarter of the rows: pieces of 32 outputs, every fourth one a group's.
        const int e = warp - kEpi0, quarter = warp & 3, grp = e >> 2;
        uint8_t *slab = smem + TileLayout<Y>::kOffSlab + (size_t)e * TileLayout<Y>::kSlab;
        const uint32_t slab_addr = ptx::smem_u32(slab);
        const uint32_t t_lane = tmem + ((uint32_t)(quarter * 32) << 16);
        const uint32_t tempty = ptx::map_to_rank(bar_tempty, 0);
        constexpr uint32_t kRowBytes = 32u * (uint32_t)sizeof(Y);
        const bool alpha_wide = (reinterpret_cast<uintptr_t>(p.alpha) & 15u) == 0;
        if (p.chained) ptx::grid_dep_wait();
        uint32_t done = 0;
        for (long long u = pair; u < units; u += pairs, ++done) {
            const int mt = (int)(u / q.n_ctiles), ct = (int)(u % q.n_ctiles), pieces = width(ct) / 32;
            const long long row0 = (long long)mt * kTile + (int)rank * 128 + quarter * 32, r = row0 + lane;
            const int adapters = adapters_of_tile(mt);
            float fac = 0.0f, ad = 0.0f;
            bool with = false;
            if (r < p.m) {
                const int s = sample_of(p, r);
                fac = factor_of(__ldg(p.gamma + s));
                if (adapters) {
                    const int a = __ldcg(p.row_adapter + r);
                    with = a >= 0;
                    if (with) ad = (p.scale ? __ldg(p.scale + a) : 1.0f) * fac * __ldcg(p.power + r);
                }
            }
            const uint32_t buf = q.depth == 2 ? done & 1u : 0u, use = q.depth == 2 ? done >> 1 : done;
            const uint32_t d1 = t_lane + buf * (uint32_t)q.nt, d2 = d1 + (uint32_t)(q.depth * q.nt);
            if (!tc::wait_bar<true>(bar_tfull + 8 * buf, use & 1u, flags)) break;
            ptx::tc_fence_after_sync();
            auto release = [&] {
                ptx::tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive_cluster(tempty + 8 * buf);
            };
            if (grp >= pieces) release();
#pragma unroll 1
            for (int pc = grp; pc < pieces; pc += kEpiGroups) {
                const int at = ct * q.nt + pc * 32;
                ptx::bulk_wait_read0();             // the previous store has read the slab
                __syncwarp();
#pragma unroll
                for (int h = 0; h < 32; h += 16) {
                    uint32_t v[16], w[16];
                    ptx::tmem_ld_x16(d1 + (uint32_t)(pc * 32 + h), v);
                    if (adapters) ptx::tmem_ld_x16(d2 + (uint32_t)(pc * 32 + h), w);
                    float al[16];
#pragma unroll
                    for (int i = 0; i < 16; i += 4) {
                        float4 a4 = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                        if (at + h + i < p.cout) {          // (whole groups of eight outputs)
                            const float *src = p.alpha + at + h + i;
                            if (alpha_wide) a4 = __ldg(reinterpret_cast<const float4 *>(src));
                            else a4 = make_float4(__ldg(src), __ldg(src + 1), __ldg(src + 2), __ldg(src + 3));
                        }
                        al[i] = a4.x; al[i + 1] = a4.y; al[i + 2] = a4.z; al[i + 3] = a4.w;
                    }
                    ptx::tmem_wait_ld();
                    if (h && pc + kEpiGroups >= pieces) release();
                    float y[16];
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        y[i] = (float)(int)v[i] * al[i] * fac;
                        if (with) y[i] += ad * __uint_as_float(w[i]);
                    }
                    if constexpr (sizeof(Y) == 4) {
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            *reinterpret_cast<float4 *>(slab + tc::swz_offset((uint32_t)lane, (uint32_t)(h / 4 + j), 128u)) =
                                make_float4(y[4 * j], y[4 * j + 1], y[4 * j + 2], y[4 * j + 3]);
                    } else {
#pragma unroll
                        for (int j = 0; j < 2; ++j)
                            *reinterpret_cast<uint4 *>(slab + tc::swz_offset((uint32_t)lane, (uint32_t)(h / 8 + j), 64u)) =
                                make_uint4(norm::pack_pair<Y>(y[8 * j], y[8 * j + 1]), norm::pack_pair<Y>(y[8 * j + 2], y[8 * j + 3]),
                                           norm::pack_pair<Y>(y[8 * j + 4], y[8 * j + 5]), norm::pack_pair<Y>(y[8 * j + 6], y[8 * j + 7]));
                    }
                }
                if (q.store) {
                    ptx::fence_proxy_async_smem();
                    __syncwarp();
                    if (lane == 0 && row0 < p.m) {
                        ptx::tma_store_2d(&ymap, at, (int)row0, slab_addr);
                        ptx::bulk_commit();
                    }
                } else {
                    __syncwarp();
                    constexpr uint32_t per = 16u / (uint32_t)sizeof(Y);
                    if (at + lane < p.cout)
                        for (int i = 0; i < 32 && row0 + i < p.m; ++i)
                            static_cast<Y *>(p.y)[(row0 + i) * p.y_pitch + at + lane] =
                                *reinterpret_cast<const Y *>(slab + tc::swz_offset((uint32_t)i, (uint32_t)lane / per, kRowBytes) + (lane % per) * sizeof(Y));
                    __syncwarp();
                }
            }
        }
        ptx::bulk_wait_all();
    }

    // neither CTA may go while the other can still reach its shared memory
    ptx::tc_fence_before_sync();
    __syncthreads();
    ptx::cluster_sync();
    if (warp == 1) {
        ptx::tc_fence_after_sync();
        ptx::tmem_dealloc_pair(tmem, 512u);
    }
}

}}  // namespace prom::lora
