// Dropout, and layer norm with the residual sum and the dropout in front of it: the junction of two sub-layers
// of an encoder or decoder block.  One pass over the data each: everything here is bound by HBM (and, in the smallest
// calls, by the launch).
//
//   D        scaled keep mask of the counter-based generator in hdt_philox.cuh, never stored
//   dropout  y = residual + D o x
//   forward  h = residual + D o x;  mean, var over the row's columns;  y = (h - mean) rstd weight + bias
//   backward xhat = (h - mean) rstd, g = dY weight:
//            dResidual = rstd (g - mean(g) - xhat mean(g xhat)) + dH,   dX = D o dResidual
//            dWeight = sum over rows of dY xhat,   dBias = sum over rows of dY
//
// A row lies in the registers of its lanes from the load to the store, so the variance is the mean square of the
// differences from the mean (a second pass, in registers) and nothing is read twice.  All arithmetic in fp32; each
// output is rounded once.  mean and rstd belong to h before its rounding.
// The column sums of the backward: every CTA walks rows with a stride of the grid and keeps its columns' sums in
// registers, adds its warps' sums in a fixed order and leaves one partial row per CTA, which k_norm_columns adds up in a
// fixed order too: no atomics, the same bits every run.
//
// Measured, bf16: dropout and residual on 65536 x 1024 61 us, 6.6 TB/s; forward with both on 32768 x 768 37 us, 5.5 TB/s; its
// backward with dH 53 us, 4.8 TB/s, and 6 us for the last sum of the columns.  The backward is held up by HBM's latency and not by its
// rate: 168 registers a thread leave twelve warps to an SM, each with one row of dY and h in flight (without dropout and dH
// 32768 x 768 36 us, 4.2 TB/s, 16384 x 2048 65 us, 3.1; issue slots 49 and 35 %, loads the longest stall).
#include "hdt_internal.cuh"
#include "hdt_philox.cuh"

namespace hdt {
namespace {

constexpr int THREADS = 128;
__host__ __device__ constexpr int cta_threads(int wpr) { return wpr > 1 ? 32 * wpr : THREADS; }      // WPR > 1: a row to a CTA
// CTAs of the backward that are resident on an SM, by what a warp keeps of a row.
__host__ __device__ constexpr int bwd_ctas(int wpr, int nv) { return wpr == 16 ? 1 : wpr == 2 ? 7 : nv == 1 ? 5 : 3; }

struct NormArgs {
    const void *x, *residual, *weight, *bias;
    void *h, *y;
    float *mean, *rstd;
    // backward
    const void *dy, *dh, *hin;
    const float *mean_in, *rstd_in;
    void *dres, *dx;
    float *part;                 // [grid, 2, cols]
    int rows, cols;
    float eps;
    Drop drop;
};

// Sum over the lanes of a row; every lane gets it.  WPR > 1: over the CTA's warps too (one row per CTA).
template <int LPR, int WPR>
__device__ __forceinline__ float row_sum(float v, float *s) {
#pragma unroll
    for (int o = LPR / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if constexpr (WPR > 1) {
        if ((threadIdx.x & 31) == 0) s[threadIdx.x >> 5] = v;
        __syncthreads();
        v = 0.f;
#pragma unroll
        for (int w = 0; w < WPR; ++w) v += s[w];
        __syncthreads();
    }
    return v;
}

// Two sums at once; `turn` alternates from call to call, so that one barrier is enough.
template <int LPR, int WPR>
__device__ __forceinline__ void row_sums(float &a, float &b, float2 (&s)[2][WPR], int turn) {
#pragma unroll
    for (int o = LPR / 2; o > 0; o >>= 1) {
        a += __shfl_xor_sync(0xffffffffu, a, o);
        b += __shfl_xor_sync(0xffffffffu, b, o);
    }
    if constexpr (WPR > 1) {
        if ((threadIdx.x & 31) == 0) s[turn][threadIdx.x >> 5] = make_float2(a, b);
        __syncthreads();
        a = b = 0.f;
#pragma unroll
        for (int w = 0; w < WPR; ++w) {
            a += s[turn][w].x;
            b += s[turn][w].y;
        }
    }
}

template <typename T, typename W, bool VEC, int LPR, int WPR, int NV>
__global__ void __launch_bounds__(cta_threads(WPR)) k_norm_fwd(const NormArgs a) {
    __shared__ float s_sum[WPR];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, l = lane % LPR;
    const int first = WPR > 1 ? blockIdx.x : (blockIdx.x * (THREADS / 32) + warp) * (32 / LPR) + lane / LPR;
    const int w0 = WPR > 1 ? warp : 0;
    const bool on = first < a.rows;
    const int row = on ? first : a.rows - 1;
    const size_t at = (size_t)row * a.cols;
    float v[NV][8];
#pragma unroll
    for (int i = 0; i < NV; ++i) load8<LPR, VEC>((const T *)a.x + at, w0 + i * WPR, l, a.cols, v[i]);
    if (a.residual != nullptr) {
        float r[NV][8];
#pragma unroll
        for (int i = 0; i < NV; ++i) load8<LPR, VEC>((const T *)a.residual + at, w0 + i * WPR, l, a.cols, r[i]);
        if (a.drop.rng != nullptr) {
            const PhiloxKey k = philox_key(a.drop);
#pragma unroll
            for (int i = 0; i < NV; ++i) drop8<LPR, VEC>(k, a.drop, row, w0 + i * WPR, l, v[i]);
        }
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) v[i][e] += r[i][e];
    } else if (a.drop.rng != nullptr) {
        const PhiloxKey k = philox_key(a.drop);
#pragma unroll
        for (int i = 0; i < NV; ++i) drop8<LPR, VEC>(k, a.drop, row, w0 + i * WPR, l, v[i]);
    }
    if (a.h != nullptr && on)
#pragma unroll
        for (int i = 0; i < NV; ++i) store8<LPR, VEC>((T *)a.h + at, w0 + i * WPR, l, a.cols, v[i]);
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) sum += v[i][e];
    const float inv = 1.f / (float)a.cols, mean = row_sum<LPR, WPR>(sum, s_sum) * inv;
    sum = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            v[i][e] -= mean;
            if (col_of<LPR, VEC>(w0 + i * WPR, l, e) < a.cols) sum = fmaf(v[i][e], v[i][e], sum);
        }
    const float rstd = rsqrtf(fmaf(row_sum<LPR, WPR>(sum, s_sum), inv, a.eps));
    if (!on) return;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        float w[8], b[8];
        load8<LPR, VEC>((const W *)a.weight, w0 + i * WPR, l, a.cols, w);
        load8<LPR, VEC>((const W *)a.bias, w0 + i * WPR, l, a.cols, b);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[i][e] = fmaf(v[i][e] * rstd, w[e], b[e]);
        store8<LPR, VEC>((T *)a.y + at, w0 + i * WPR, l, a.cols, v[i]);
    }
    if (l == 0 && w0 == 0) {
        a.mean[row] = mean;
        a.rstd[row] = rstd;
    }
}

template <typename T, typename W, bool VEC, int LPR, int WPR, int NV>
__global__ void __launch_bounds__(cta_threads(WPR), bwd_ctas(WPR, NV)) k_norm_bwd(const NormArgs a) {
    constexpr int NW = cta_threads(WPR) / 32, RPC = WPR > 1 ? 1 : NW * (32 / LPR);   // rows of a CTA at a time
    __shared__ float2 s_sum[2][WPR];
    __shared__ float s_col[WPR > 1 ? 1 : NW * 8 * 32];
    pdl_launch_dependents();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, l = lane % LPR;
    const int sub = WPR > 1 ? 0 : warp * (32 / LPR) + lane / LPR, w0 = WPR > 1 ? warp : 0;
    const float inv = 1.f / (float)a.cols;
    float dw[NV][8], db[NV][8];
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) dw[i][e] = db[i][e] = 0.f;
    PhiloxKey key{0, 0, 0};
    if (a.drop.rng != nullptr) key = philox_key(a.drop);
    // the next row's dY and h are requested before this one's are looked at
    Raw8<T, VEC> ng[NV], nx[NV];
    auto request = [&](int r0) {
        const size_t at = (size_t)min(r0 + sub, a.rows - 1) * a.cols;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            ng[i].template load<LPR>((const T *)a.dy + at, w0 + i * WPR, l, a.cols);
            nx[i].template load<LPR>((const T *)a.hin + at, w0 + i * WPR, l, a.cols);
        }
    };
    const int stride = gridDim.x * RPC;
    int r0 = blockIdx.x * RPC, turn = 0;
    if (r0 < a.rows) request(r0);
    for (; r0 < a.rows; r0 += stride) {
        const bool on = r0 + sub < a.rows;
        const int row = on ? r0 + sub : a.rows - 1;
        const size_t at = (size_t)row * a.cols;
        const float mean = a.mean_in[row], rstd = a.rstd_in[row];
        float g[NV][8], x[NV][8];
        Raw8<T, VEC> d[NV];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if (a.dh != nullptr) d[i].template load<LPR>((const T *)a.dh + at, w0 + i * WPR, l, a.cols);
            ng[i].get(g[i]);
            nx[i].get(x[i]);
        }
        if (r0 + stride < a.rows) request(r0 + stride);
        float s1 = 0.f, s2 = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            float w[8];
            load8<LPR, VEC>((const W *)a.weight, w0 + i * WPR, l, a.cols, w);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                // (a column that the row does not have has dY = 0 and weight 0: it adds nothing to any sum)
                x[i][e] = (x[i][e] - mean) * rstd;
                if (on) {
                    dw[i][e] = fmaf(g[i][e], x[i][e], dw[i][e]);
                    db[i][e] += g[i][e];
                }
                g[i][e] *= w[e];
                s1 += g[i][e];
                s2 = fmaf(g[i][e], x[i][e], s2);
            }
        }
        row_sums<LPR, WPR>(s1, s2, s_sum, turn);
        turn ^= 1;
        const float m1 = s1 * inv, m2 = s2 * inv;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            float y[8];
            if (a.dh != nullptr) d[i].get(y);
#pragma unroll
            for (int e = 0; e < 8; ++e) g[i][e] = fmaf(g[i][e] - m1 - x[i][e] * m2, rstd, a.dh != nullptr ? y[e] : 0.f);
            if (on) store8<LPR, VEC>((T *)a.dres + at, w0 + i * WPR, l, a.cols, g[i]);
            if (a.drop.rng != nullptr) drop8<LPR, VEC>(key, a.drop, row, w0 + i * WPR, l, g[i]);
            if (a.dx != nullptr && on) store8<LPR, VEC>((T *)a.dx + at, w0 + i * WPR, l, a.cols, g[i]);
        }
    }
    // the CTA's column sums: over the row groups of a warp by shuffles, over the warps through shared memory
    float *out = a.part + (size_t)blockIdx.x * 2 * a.cols;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            float v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                v[e] = t == 0 ? dw[i][e] : db[i][e];
#pragma unroll
                for (int o = LPR; o < 32; o <<= 1) v[e] += __shfl_xor_sync(0xffffffffu, v[e], o);
            }
            if constexpr (WPR == 1) {
                __syncthreads();
#pragma unroll
                for (int e = 0; e < 8; ++e) s_col[(warp * 8 + e) * 32 + lane] = v[e];
                __syncthreads();
                if (warp != 0) continue;
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    for (int w = 1; w < NW; ++w) v[e] += s_col[(w * 8 + e) * 32 + lane];
                if (lane >= LPR) continue;
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int c = col_of<LPR, VEC>(w0 + i * WPR, l, e);
                if (c < a.cols) out[t * a.cols + c] = v[e];
            }
        }
}

// Sums of the partial rows, 32 columns a CTA, its 32 warps a stride of 32 partial rows each.
template <typename W>
__global__ void __launch_bounds__(1024) k_norm_columns(const float *part, int n, int cols, W *dw, W *db) {
    __shared__ float s[32][33];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
    pdl_wait();
    float v = 0.f;
    if (c < 2 * cols)
#pragma unroll 4
        for (int i = warp; i < n; i += 32) v += part[(size_t)i * 2 * cols + c];
    s[warp][lane] = v;
    __syncthreads();
    v = s[lane][warp];              // lane = which sum of column `warp`
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if (lane == 0) {
        const int x = blockIdx.x * 32 + warp;
        if (x < cols) from_f32(dw[x], v);
        else if (x < 2 * cols) from_f32(db[x - cols], v);
    }
}

// Four pieces of a lane at a time: four chunks of a row, or, where a row is one chunk (ONE), four rows.
template <typename T, bool VEC, int LPR, bool ONE>
__global__ void __launch_bounds__(256, 4) k_dropout(const T *x, const T *residual, T *y, int rows, int cols, const Drop d) {
    constexpr int U = 4, RPW = 32 / LPR;
    const int lane = threadIdx.x & 31, l = lane % LPR;
    const int first = (blockIdx.x * 8 + (threadIdx.x >> 5)) * RPW * (ONE ? U : 1) + lane / LPR;
    const int chunks = ONE ? U : (cols + 8 * LPR - 1) / (8 * LPR);
    const PhiloxKey k = philox_key(d);
    for (int c0 = 0; c0 < chunks; c0 += U) {
        Raw8<T, VEC> rx[U], rr[U];
#pragma unroll
        for (int i = 0; i < U; ++i) {      // (a chunk behind the row's end reads as zeros, a row behind the last as the last)
            const size_t at = (size_t)min(first + (ONE ? i * RPW : 0), rows - 1) * cols;
            rx[i].template load<LPR>(x + at, ONE ? 0 : c0 + i, l, cols);
            if (residual != nullptr) rr[i].template load<LPR>(residual + at, ONE ? 0 : c0 + i, l, cols);
        }
#pragma unroll
        for (int i = 0; i < U; ++i) {
            if (!ONE && c0 + i >= chunks) break;
            const int row = first + (ONE ? i * RPW : 0), c = ONE ? 0 : c0 + i;
            float v[8], r[8];
            rx[i].get(v);
            drop8<LPR, VEC>(k, d, row, c, l, v);
            if (residual != nullptr) {
                rr[i].get(r);
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] += r[e];
            }
            if (row < rows) store8<LPR, VEC>(y + (size_t)row * cols, c, l, cols, v);
        }
    }
}

bool aligned16(const void *p) { return ((uintptr_t)p & 15) == 0; }

int make_drop(Drop *d, const int64_t *rng, int32_t site, float p, bool wanted, const char *who) {
    *d = Drop{nullptr, (uint32_t)site, 0, 1.f};
    if (!(p >= 0.f && p < 1.f)) return set_error(HDT_ERR_INVALID_ARG, "%s: p must be in [0, 1)", who);
    int t = (int)(65536.0 * (double)p + 0.5);
    if (t > 65535) t = 65535;
    if (t == 0 && !wanted) return HDT_OK;
    if (!rng) return set_error(HDT_ERR_INVALID_ARG, "%s: p > 0 needs the generator's state", who);
    if ((uintptr_t)rng & 7) return set_error(HDT_ERR_INVALID_ARG, "%s: the generator's state must be 8-byte aligned", who);
    d->rng = (const unsigned long long *)rng;
    d->t = (uint32_t)t;
    d->scale = (float)(65536.0 / (65536 - t));
    return HDT_OK;
}

int norm_check(int64_t rows, int32_t cols, int32_t dtype, int32_t w_dtype, const char *who) {
    if (rows < 0 || cols < 1) return set_error(HDT_ERR_INVALID_ARG, "%s: negative number of rows or no column", who);
    if (rows > 0x7fff0000LL || cols > 8192) return set_error(HDT_ERR_UNSUPPORTED, "%s: at most 2^31 - 2^16 rows and 8192 columns", who);
    if (dtype != HDT_F32 && dtype != HDT_BF16) return set_error(HDT_ERR_UNSUPPORTED, "%s: unknown dtype %d", who, dtype);
    if (w_dtype != HDT_F32 && w_dtype != dtype) return set_error(HDT_ERR_UNSUPPORTED, "%s: weights must be fp32 or of the rows' type", who);
    return HDT_OK;
}

// How a row lies on lanes: LPR lanes with up to NV x 8 columns each, the smallest that hold it (a warp for up to 1024
// columns); beyond that all warps of a CTA.
template <template <typename, typename, bool, int, int, int> class K, typename T, typename W, bool VEC>
int norm_pick(const NormArgs &a, cudaStream_t st) {
    const int c = a.cols;
    if (c <= 32) return K<T, W, VEC, 4, 1, 1>::go(a, st);
    if (c <= 64) return K<T, W, VEC, 8, 1, 1>::go(a, st);
    if (c <= 128) return K<T, W, VEC, 16, 1, 1>::go(a, st);
    if (c <= 256) return K<T, W, VEC, 32, 1, 1>::go(a, st);
    if (c <= 512) return K<T, W, VEC, 32, 1, 2>::go(a, st);
    if (c <= 768) return K<T, W, VEC, 32, 1, 3>::go(a, st);
    if (c <= 1024) return K<T, W, VEC, 32, 1, 4>::go(a, st);
    if (c <= 2048) return K<T, W, VEC, 32, 4, 2>::go(a, st);
    if (c <= 4096) return K<T, W, VEC, 32, 4, 4>::go(a, st);
    return K<T, W, VEC, 32, 16, 2>::go(a, st);
}
template <template <typename, typename, bool, int, int, int> class K>
int norm_types(const NormArgs &a, int dtype, int w_dtype, bool vec, cudaStream_t st) {
    if (dtype == HDT_F32) return vec ? norm_pick<K, float, float, true>(a, st) : norm_pick<K, float, float, false>(a, st);
    if (w_dtype == HDT_F32) return vec ? norm_pick<K, __nv_bfloat16, float, true>(a, st) : norm_pick<K, __nv_bfloat16, float, false>(a, st);
    return vec ? norm_pick<K, __nv_bfloat16, __nv_bfloat16, true>(a, st) : norm_pick<K, __nv_bfloat16, __nv_bfloat16, false>(a, st);
}

// The backward keeps two sums a column and the next row besides, so a warp holds a row of up to 768 (aligned bf16) or 512 columns, two
// (aligned bf16) or four warps one of up to 1024, four one of up to 2048, sixteen up to 8192 (1024 columns on one warp spilled 500 bytes a thread).
template <template <typename, typename, bool, int, int, int> class K, typename T, typename W, bool VEC>
int norm_pick_bwd(const NormArgs &a, cudaStream_t st) {
    const int c = a.cols;
    if (c <= 32) return K<T, W, VEC, 4, 1, 1>::go(a, st);
    if (c <= 64) return K<T, W, VEC, 8, 1, 1>::go(a, st);
    if (c <= 128) return K<T, W, VEC, 16, 1, 1>::go(a, st);
    if (c <= 256) return K<T, W, VEC, 32, 1, 1>::go(a, st);
    if (c <= 512) return K<T, W, VEC, 32, 1, 2>::go(a, st);
    if constexpr (sizeof(T) == 2 && VEC)
        if (c <= 768) return K<T, W, VEC, 32, 1, 3>::go(a, st);
    if constexpr (sizeof(T) == 2 && VEC)
        if (c <= 1024) return K<T, W, VEC, 32, 2, 2>::go(a, st);
    if (c <= 1024) return K<T, W, VEC, 32, 4, 1>::go(a, st);
    if (c <= 2048) return K<T, W, VEC, 32, 4, 2>::go(a, st);
    if (c <= 4096) return K<T, W, VEC, 32, 16, 1>::go(a, st);
    return K<T, W, VEC, 32, 16, 2>::go(a, st);
}
template <template <typename, typename, bool, int, int, int> class K>
int norm_types_bwd(const NormArgs &a, int dtype, int w_dtype, bool vec, cudaStream_t st) {
    if (dtype == HDT_F32) return vec ? norm_pick_bwd<K, float, float, true>(a, st) : norm_pick_bwd<K, float, float, false>(a, st);
    if (w_dtype == HDT_F32) return vec ? norm_pick_bwd<K, __nv_bfloat16, float, true>(a, st) : norm_pick_bwd<K, __nv_bfloat16, float, false>(a, st);
    return vec ? norm_pick_bwd<K, __nv_bfloat16, __nv_bfloat16, true>(a, st) : norm_pick_bwd<K, __nv_bfloat16, __nv_bfloat16, false>(a, st);
}

// An upper limit of the backward's CTAs, and so of its partial rows.
int64_t bwd_most(int64_t rows, int cols) {
    const int at_once = cols > 512 ? 1 : cols > 128 ? 4 : cols > 64 ? 8 : cols > 32 ? 16 : 32;
    const int64_t need = (rows + at_once - 1) / at_once, most = (int64_t)PLAN_SMS * bwd_ctas(2, 2);
    return need < most ? need : most;
}

template <typename T, typename W, bool VEC, int LPR, int WPR, int NV>
struct Fwd {
    static int go(const NormArgs &a, cudaStream_t st) {
        const int per = WPR > 1 ? 1 : THREADS / LPR;
        HDT_CUDA_CHECK(launch_dependent(k_norm_fwd<T, W, VEC, LPR, WPR, NV>, false, dim3((a.rows + per - 1) / per), cta_threads(WPR), 0, st, a));
        return HDT_OK;
    }
};
template <typename T, typename W, bool VEC, int LPR, int WPR, int NV>
struct Bwd {      // returns the number of CTAs (all resident at once), or an error
    static int go(const NormArgs &a, cudaStream_t st) {
        const int at_once = WPR > 1 ? 1 : THREADS / LPR, need = (a.rows + at_once - 1) / at_once, most = PLAN_SMS * bwd_ctas(WPR, NV), n = need < most ? need : most;
        HDT_CUDA_CHECK(launch_dependent(k_norm_bwd<T, W, VEC, LPR, WPR, NV>, false, dim3(n), cta_threads(WPR), 0, st, a));
        return n;
    }
};

template <typename T, bool VEC>
int dropout_pick(const void *x, const void *res, void *y, int rows, int cols, const Drop &d, cudaStream_t st) {
    auto go = [&](auto *kern, int rows_of_warp) -> int {
        const int per = 8 * rows_of_warp;
        HDT_CUDA_CHECK(launch_dependent(kern, false, dim3((rows + per - 1) / per), 256, 0, st, (const T *)x, (const T *)res, (T *)y, rows, cols, d));
        return HDT_OK;
    };
    if (cols <= 32) return go(k_dropout<T, VEC, 4, true>, 32);
    if (cols <= 64) return go(k_dropout<T, VEC, 8, true>, 16);
    if (cols <= 128) return go(k_dropout<T, VEC, 16, true>, 8);
    if (cols <= 256) return go(k_dropout<T, VEC, 32, true>, 4);
    return go(k_dropout<T, VEC, 32, false>, 1);
}

}  // namespace
}  // namespace hdt

using namespace hdt;

extern "C" int hdt_dropout(const void *x, const void *residual, const int64_t *rng, int32_t site, int64_t rows, int32_t cols, int32_t dtype, float p, void *y,
                           void *stream) {
    if (const int rc = norm_check(rows, cols, dtype, dtype, "hdt_dropout")) return rc;
    Drop d;
    if (const int rc = make_drop(&d, rng, site, p, true, "hdt_dropout")) return rc;
    if (rows == 0) return HDT_OK;
    if (!x || !y) return set_error(HDT_ERR_INVALID_ARG, "hdt_dropout: null tensor pointer");
    const uintptr_t el = dtype == HDT_F32 ? 3 : 1;
    if (((uintptr_t)x | (uintptr_t)residual | (uintptr_t)y) & el) return set_error(HDT_ERR_INVALID_ARG, "hdt_dropout: misaligned tensor");
    const bool vec = cols % 8 == 0 && aligned16(x) && aligned16(residual) && aligned16(y);
    cudaStream_t st = (cudaStream_t)stream;
    if (dtype == HDT_F32) return vec ? dropout_pick<float, true>(x, residual, y, (int)rows, cols, d, st) : dropout_pick<float, false>(x, residual, y, (int)rows, cols, d, st);
    return vec ? dropout_pick<__nv_bfloat16, true>(x, residual, y, (int)rows, cols, d, st) : dropout_pick<__nv_bfloat16, false>(x, residual, y, (int)rows, cols, d, st);
}

extern "C" int hdt_layer_norm_fwd(const void *x, const void *residual, const void *weight, const void *bias, const int64_t *rng, int32_t site, float p, int64_t rows,
                                  int32_t cols, int32_t dtype, int32_t w_dtype, float eps, void *h, void *y, float *mean, float *rstd, void *stream) {
    if (const int rc = norm_check(rows, cols, dtype, w_dtype, "hdt_layer_norm_fwd")) return rc;
    if (!(eps >= 0.f)) return set_error(HDT_ERR_INVALID_ARG, "hdt_layer_norm_fwd: eps must not be negative");
    NormArgs a{};
    if (const int rc = make_drop(&a.drop, rng, site, p, false, "hdt_layer_norm_fwd")) return rc;
    if (rows == 0) return HDT_OK;
    if (!x || !weight || !bias || !y || !mean || !rstd) return set_error(HDT_ERR_INVALID_ARG, "hdt_layer_norm_fwd: null tensor pointer");
    if (!h && (residual || p > 0.f)) return set_error(HDT_ERR_INVALID_ARG, "hdt_layer_norm_fwd: with a residual or dropout h has to be written");
    const uintptr_t el = dtype == HDT_F32 ? 3 : 1, wl = w_dtype == HDT_F32 ? 3 : 1;
    if ((((uintptr_t)x | (uintptr_t)residual | (uintptr_t)h | (uintptr_t)y) & el) || (((uintptr_t)weight | (uintptr_t)bias) & wl) ||
        (((uintptr_t)mean | (uintptr_t)rstd) & 3))
        return set_error(HDT_ERR_INVALID_ARG, "hdt_layer_norm_fwd: misaligned tensor");
    a.x = x; a.residual = residual; a.weight = weight; a.bias = bias; a.h = h; a.y = y; a.mean = mean; a.rstd = rstd;
    a.rows = (int)rows; a.cols = cols; a.eps = eps;
    const bool vec = cols % 8 == 0 && aligned16(x) && aligned16(residual) && aligned16(weight) && aligned16(bias) && aligned16(h) && aligned16(y);
    return norm_types<Fwd>(a, dtype, w_dtype, vec, (cudaStream_t)stream);
}

extern "C" size_t hdt_layer_norm_workspace_bytes(int64_t rows, int32_t cols) {
    if (rows < 0 || rows > 0x7fff0000LL || cols < 1 || cols > 8192) return 0;
    const int64_t n = bwd_most(rows, cols);
    return ((size_t)(n > 0 ? n : 1) * 2 * cols * 4 + 255) / 256 * 256;
}

extern "C" int hdt_layer_norm_bwd(const void *d_y, const void *d_h, const void *h, const float *mean, const float *rstd, const void *weight, const int64_t *rng,
                                  int32_t site, float p, int64_t rows, int32_t cols, int32_t dtype, int32_t w_dtype, void *d_residual, void *d_x, void *d_weight,
                                  void *d_bias, void *workspace, size_t workspace_bytes, void *stream) {
    if (const int rc = norm_check(rows, cols, dtype, w_dtype, "hdt_layer_norm_bwd")) return rc;
    NormArgs a{};
    if (const int rc = make_drop(&a.drop, rng, site, p, false, "hdt_layer_norm_bwd")) return rc;
    if (!d_weight || !d_bias) return set_error(HDT_ERR_INVALID_ARG, "hdt_layer_norm_bwd: null tensor pointer");
    if (rows > 0 && (!d_y || !h || !mean || !rstd || !weight || !d_residual || (p > 0.f && !d_x)))
        return set_error(HDT_ERR_INVALID_ARG, "hdt_layer_norm_bwd: null tensor pointer");
    if (rows > 0 && p > 0.f && d_x == d_residual) return set_error(HDT_ERR_INVALID_ARG, "hdt_layer_norm_bwd: with dropout d_x and d_residual are two tensors");
    const size_t need = hdt_layer_norm_workspace_bytes(rows, cols);
    if (!workspace || workspace_bytes < need) return set_error(HDT_ERR_WORKSPACE, "hdt_layer_norm_bwd: workspace %zu < required %zu", workspace_bytes, need);
    if ((uintptr_t)workspace & 255) return set_error(HDT_ERR_INVALID_ARG, "hdt_layer_norm_bwd: workspace must be 256-byte aligned");
    const uintptr_t el = dtype == HDT_F32 ? 3 : 1, wl = w_dtype == HDT_F32 ? 3 : 1;
    if ((((uintptr_t)d_y | (uintptr_t)d_h | (uintptr_t)h | (uintptr_t)d_residual | (uintptr_t)d_x) & el) || (((uintptr_t)weight | (uintptr_t)d_weight | (uintptr_t)d_bias) & wl) ||
        (((uintptr_t)mean | (uintptr_t)rstd) & 3))
        return set_error(HDT_ERR_INVALID_ARG, "hdt_layer_norm_bwd: misaligned tensor");
    a.dy = d_y; a.dh = d_h; a.hin = h; a.mean_in = mean; a.rstd_in = rstd; a.weight = weight; a.dres = d_residual;
    a.dx = d_x != d_residual ? d_x : nullptr;      // (a buffer of the caller's is written with and without dropout)
    a.part = (float *)workspace; a.rows = (int)rows; a.cols = cols;
    cudaStream_t st = (cudaStream_t)stream;
    int n = 0;
    if (rows > 0) {
        const bool vec = cols % 8 == 0 && aligned16(d_y) && aligned16(d_h) && aligned16(h) && aligned16(weight) && aligned16(d_residual) && aligned16(d_x);
        n = norm_types_bwd<Bwd>(a, dtype, w_dtype, vec, st);
        if (n < 0) return n;
    }
    const int ctas = (2 * cols + 31) / 32;
    if (w_dtype == HDT_F32) HDT_CUDA_CHECK(launch_dependent(k_norm_columns<float>, rows > 0, dim3(ctas), 1024, 0, st, a.part, n, cols, (float *)d_weight, (float *)d_bias));
    else HDT_CUDA_CHECK(launch_dependent(k_norm_columns<__nv_bfloat16>, rows > 0, dim3(ctas), 1024, 0, st, a.part, n, cols, (__nv_bfloat16 *)d_weight, (__nv_bfloat16 *)d_bias));
    return HDT_OK;
}
