// Counter-based random numbers of the dropout: Philox-4x32-10 (Salmon, Moraes, Dror, Shaw, "Parallel random
// numbers: as easy as 1, 2, 3", SC 2011), and the row layout that the kernels with dropout share.
//
// Eight columns of a row take one 128-bit block: key = the 64-bit seed, counter = (column / 8, row, site, offset).
// Column c keeps its value if the (c mod 8)-th 16-bit half word (low half first) is >= t = round(65536 p) and is then
// scaled by 65536 / (65536 - t), the reciprocal of the probability that it is kept with.  16 bits a value and not 32:
// the generator is then forty instructions for eight values, which a pass over bf16 rows hides behind its memory traffic.
#pragma once
#include <cuda_bf16.h>
#include <stdint.h>

namespace hdt {

struct Drop {
    const unsigned long long *rng;   // device: seed, offset (the low 32 bits count); nullptr: nothing is dropped
    uint32_t site, t;
    float scale;
};

struct PhiloxKey { uint32_t k0, k1, offset; };
__device__ __forceinline__ PhiloxKey philox_key(const Drop &d) {
    const unsigned long long seed = d.rng[0];
    return PhiloxKey{(uint32_t)seed, (uint32_t)(seed >> 32), (uint32_t)d.rng[1]};
}
__device__ __forceinline__ uint4 philox(PhiloxKey k, uint32_t block, uint32_t row, uint32_t site) {
    uint32_t a = block, b = row, c = site, d = k.offset, k0 = k.k0, k1 = k.k1;
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const unsigned long long p = 0xD2511F53ull * a, q = 0xCD9E8D57ull * c;
        a = (uint32_t)(q >> 32) ^ b ^ k0;
        c = (uint32_t)(p >> 32) ^ d ^ k1;
        b = (uint32_t)q;
        d = (uint32_t)p;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return make_uint4(a, b, c, d);
}

// A row lies on LPR neighbouring lanes (of WPR warps, where one has not enough), each with eight columns of every
// chunk of 8 LPR: neighbouring ones where rows are 16-byte aligned (VEC; one 16-byte access of bf16, two of fp32),
// else one of every LPR, so that unaligned rows are read in coalesced pieces too.
template <int LPR, bool VEC>
__device__ __forceinline__ int col_of(int chunk, int l, int e) { return chunk * 8 * LPR + (VEC ? l * 8 + e : e * LPR + l); }

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ void from_f32(float &d, float x) { d = x; }
__device__ __forceinline__ void from_f32(__nv_bfloat16 &d, float x) { d = __float2bfloat16(x); }

// A lane's eight columns of a chunk as they are in memory: what has been requested and is not needed yet takes half of
// the registers of its values in fp32 (bf16).  Columns that the row does not have read as 0.  (VEC rows have a
// multiple of eight columns.)
template <typename T, bool VEC>
struct Raw8;
template <>
struct Raw8<__nv_bfloat16, true> {
    uint4 x;
    template <int LPR>
    __device__ __forceinline__ void load(const __nv_bfloat16 *row, int chunk, int l, int cols) {
        const int c = col_of<LPR, true>(chunk, l, 0);
        x = c < cols ? *reinterpret_cast<const uint4 *>(row + c) : make_uint4(0, 0, 0, 0);
    }
    __device__ __forceinline__ void get(float (&v)[8]) const {
        const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            v[2 * e] = __uint_as_float(w[e] << 16);
            v[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
        }
    }
};
template <>
struct Raw8<float, true> {
    float4 x, y;
    template <int LPR>
    __device__ __forceinline__ void load(const float *row, int chunk, int l, int cols) {
        const int c = col_of<LPR, true>(chunk, l, 0);
        x = y = make_float4(0.f, 0.f, 0.f, 0.f);
        if (c < cols) {
            x = *reinterpret_cast<const float4 *>(row + c);
            y = *reinterpret_cast<const float4 *>(row + c + 4);
        }
    }
    __device__ __forceinline__ void get(float (&v)[8]) const {
        v[0] = x.x; v[1] = x.y; v[2] = x.z; v[3] = x.w;
        v[4] = y.x; v[5] = y.y; v[6] = y.z; v[7] = y.w;
    }
};
template <typename T>
struct Raw8<T, false> {
    T x[8];
    template <int LPR>
    __device__ __forceinline__ void load(const T *row, int chunk, int l, int cols) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int c = col_of<LPR, false>(chunk, l, e);
            if (c < cols) x[e] = row[c];
            else from_f32(x[e], 0.f);
        }
    }
    __device__ __forceinline__ void get(float (&v)[8]) const {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = to_f32(x[e]);
    }
};
template <int LPR, bool VEC, typename T>
__device__ __forceinline__ void load8(const T *row, int chunk, int l, int cols, float (&v)[8]) {
    Raw8<T, VEC> r;
    r.template load<LPR>(row, chunk, l, cols);
    r.get(v);
}
template <int LPR, bool VEC, typename T>
__device__ __forceinline__ void store8(T *row, int chunk, int l, int cols, const float (&v)[8]) {
    if constexpr (VEC) {
        const int c = col_of<LPR, true>(chunk, l, 0);
        if (c >= cols) return;
        if constexpr (sizeof(T) == 2) {
            uint32_t w[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const __nv_bfloat162 p = __floats2bfloat162_rn(v[2 * e], v[2 * e + 1]);
                w[e] = *reinterpret_cast<const uint32_t *>(&p);
            }
            *reinterpret_cast<uint4 *>(row + c) = make_uint4(w[0], w[1], w[2], w[3]);
        } else {
            *reinterpret_cast<float4 *>(row + c) = make_float4(v[0], v[1], v[2], v[3]);
            *reinterpret_cast<float4 *>(row + c + 4) = make_float4(v[4], v[5], v[6], v[7]);
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int c = col_of<LPR, false>(chunk, l, e);
            if (c < cols) from_f32(row[c], v[e]);
        }
    }
}
// The lane's eight columns of a chunk times their keep mask; what is dropped is 0 whatever it was.  All lanes of the warp call it.
template <int LPR, bool VEC>
__device__ __forceinline__ void drop8(const PhiloxKey &k, const Drop &d, uint32_t row, int chunk, int l, float (&v)[8]) {
    const uint4 x = philox(k, (uint32_t)(chunk * LPR + l), row, d.site);
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
    if constexpr (VEC) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint32_t u = e & 1 ? w[e >> 1] >> 16 : w[e >> 1] & 0xffffu;
            v[e] = u >= d.t ? v[e] * d.scale : 0.f;
        }
    } else {      // column e LPR + l of the chunk is in the block of lane (e LPR + l) / 8 of the row's lanes
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int at = e * LPR + l, src = at >> 3, word = (at & 7) >> 1;
            uint32_t u = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t y = __shfl_sync(0xffffffffu, w[i], src, LPR);
                if (word == i) u = y;
            }
            u = at & 1 ? u >> 16 : u & 0xffffu;
            v[e] = u >= d.t ? v[e] * d.scale : 0.f;
        }
    }
}

}  // namespace hdt
