// Self-attention with a relative position bias in fp32, forward and backward (there is no tcgen05 product of fp32
// operands: the products run on the FMA pipe).  256 threads take 64 rows of one side, resident in shared memory, and walk
// the other side in tiles of 64; a thread has a 4 x 4 piece of the tile (rows ty + 16 i, columns tx + 16 j, so that the 16-byte
// reads of neighbouring threads lie in different banks) and 4 rows x D / 16 columns of a result (rows 4 ty + i, columns
// 4 tx + 64 j).  A 64 x 64 product matrix goes from the one layout to the other through shared memory, transposed.
// Bound by the shared-memory reads (two of 16 bytes for 16 fma) and, in short calls, by the longest document's last block: 2 x 777
// tokens, 12 x 64, forward 98 us and backward 270, 19 and 17 TFLOP/s.  Rows behind a document's end are stored as zeros.
//
// Forward: running maximum and sum of the softmax, O rescaled at every tile.  Backward as in bf16: once with keys resident
// (dK, dV), once with rows resident (dQ, and the bias' gradient: the sums along the diagonals of the tile's dS, then by
// bucket), no atomics.
#include "hdt_rows.cuh"
#include "hdt_self.cuh"

namespace hdt {
namespace {

constexpr long long MOST_CTAS = 1 << 20;          // (a CTA walks units with the grid's stride beyond that; the host's limits of sizes leave room for one in 32 bits)
constexpr int R = SELF_F32_ROWS, PS = R + 4;      // row stride of a transposed 64 x 64 matrix
template <int D>
struct Shape { static constexpr int XS = D + 4, X = R * XS; };

// 64 rows of [T, H, D] from `row` on, those behind `n` as zeros: requested here, there after `arrived`.
template <int D>
__device__ __forceinline__ void request_rows(float *dst, const float *src, int row, int n, int h, int H) {
#pragma unroll
    for (int i = threadIdx.x; i < R * (D / 4); i += 256) {
        const int r = i / (D / 4), c = 4 * (i % (D / 4));
        const uint32_t to = (uint32_t)__cvta_generic_to_shared(dst + r * Shape<D>::XS + c);
        const float *from = src + ((size_t)(row + min(r, n - 1)) * H + h) * D + c;      // (n > 0)
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(r < n ? 16 : 0) : "memory");
    }
}
__device__ __forceinline__ void requested() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int LEFT>
__device__ __forceinline__ void arrived() { asm volatile("cp.async.wait_group %0;" ::"n"(LEFT) : "memory"); }
// s[i][j] = a row (ty + 16 i) . b row (tx + 16 j), even and odd columns in the halves of packed sums
template <int D>
__device__ __forceinline__ void dots(const float *a, const float *b, int ty, int tx, float (&s)[4][4]) {
    f2 t[4][4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) t[i][j] = pack2(0.f, 0.f);
#pragma unroll 4
    for (int c = 0; c < D; c += 4) {
        f2 x[4][2], y[4][2];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float4 u = *reinterpret_cast<const float4 *>(a + (ty + 16 * i) * Shape<D>::XS + c), v = *reinterpret_cast<const float4 *>(b + (tx + 16 * i) * Shape<D>::XS + c);
            x[i][0] = pack2(u.x, u.y); x[i][1] = pack2(u.z, u.w);
            y[i][0] = pack2(v.x, v.y); y[i][1] = pack2(v.z, v.w);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) t[i][j] = fma2(x[i][1], y[j][1], fma2(x[i][0], y[j][0], t[i][j]));
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            float u, v;
            unpack2(t[i][j], u, v);
            s[i][j] = u + v;
        }
}
// One column of the sums below; ONLY: for the rows of `rows` (bit i: row 4 ty + i).
template <int D, bool ONLY>
__device__ __forceinline__ void accumulate_column(const float *p, const float *v, int c, int ty, int tx, f2 (&acc)[4][D / 32], unsigned rows) {
    const float4 x = *reinterpret_cast<const float4 *>(p + c * PS + 4 * ty);
    const f2 xs[4] = {pack2(x.x, x.x), pack2(x.y, x.y), pack2(x.z, x.z), pack2(x.w, x.w)};
#pragma unroll
    for (int j = 0; j < D / 64; ++j) {
        const float4 y = *reinterpret_cast<const float4 *>(v + c * Shape<D>::XS + 4 * tx + 64 * j);
        const f2 y0 = pack2(y.x, y.y), y1 = pack2(y.z, y.w);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (!ONLY || (rows >> i & 1u)) {
                acc[i][2 * j] = fma2(xs[i], y0, acc[i][2 * j]);
                acc[i][2 * j + 1] = fma2(xs[i], y1, acc[i][2 * j + 1]);
            }
    }
}
// acc[i][..] += sum over columns c of p[c][4 ty + i] v[c][4 tx + 64 j ..]
template <int D>
__device__ __forceinline__ void accumulate(const float *p, const float *v, int ty, int tx, f2 (&acc)[4][D / 32]) {
#pragma unroll 4
    for (int c = 0; c < R; ++c) accumulate_column<D, false>(p, v, c, ty, tx, acc, 15u);
}
// The same in a tile that causality cuts: row r has the columns c with c - r < edge (BELOW) or >= edge, and only those are added.  p of the
// others is 0, but 0 times what is not finite is no number, and their rows must not reach this one.  (The four rows of a thread
// differ in three columns; it skips what none of them has.)
template <int D, bool BELOW>
__device__ __forceinline__ void accumulate_cut(const float *p, const float *v, int ty, int tx, f2 (&acc)[4][D / 32], int edge) {
    const int e = edge + 4 * ty, mid0 = min(max(e, 0), R), mid1 = min(max(e + 3, 0), R);      // between them not all four
#pragma unroll 4
    for (int c = BELOW ? 0 : mid1; c < (BELOW ? mid0 : R); ++c) accumulate_column<D, false>(p, v, c, ty, tx, acc, 15u);
    for (int c = mid0; c < mid1; ++c) {
        const unsigned above = 15u << (c - e + 1) & 15u;      // rows i with c < e + i (c - e is 0, 1 or 2)
        accumulate_column<D, true>(p, v, c, ty, tx, acc, BELOW ? above : ~above);
    }
}
template <int N>
__device__ __forceinline__ void scale_by(f2 (&acc)[N], float f) {
#pragma unroll
    for (int c = 0; c < N; ++c) acc[c] = mul2(acc[c], pack2(f, f));
}
// bias' by distance of a tile: entry 63 + (distance - base)
__device__ __forceinline__ void load_near(float *nb, const SelfDist &d, int h, int base) {
    if (threadIdx.x < 2 * R) nb[threadIdx.x] = d.bias[(size_t)h * d.n + self_dist_at(d, base + (int)threadIdx.x - (R - 1))];
}
template <int D>
__device__ __forceinline__ void store_rows(float *dst, const f2 (&acc)[4][D / 32], int row, int n, int h, int H, int ty, int tx) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (4 * ty + i < n)
#pragma unroll
            for (int j = 0; j < D / 64; ++j) {
                float4 y;
                unpack2(acc[i][2 * j], y.x, y.y);
                unpack2(acc[i][2 * j + 1], y.z, y.w);
                *reinterpret_cast<float4 *>(dst + ((size_t)(row + 4 * ty + i) * H + h) * D + 4 * tx + 64 * j) = y;
            }
}

template <int D>
__global__ void __launch_bounds__(256, D == 64 ? 2 : 1) k_self_fwd_f32(const SelfFwdArgs a) {
    extern __shared__ float sm[];
    constexpr int X = Shape<D>::X;
    float *sQ = sm, *sKV = sQ + X, *sP = sKV + 4 * X, *sF = sP + R * PS, *sNb = sF + R;      // K and V twice
    const int ty = threadIdx.x >> 4, tx = threadIdx.x & 15, H = a.H;
    pdl_wait();
    const int n_units = *a.q.count * H;
    for (int u = blockIdx.x; u < n_units; u += gridDim.x) {
        const SelfBlk b = a.q.blk[u / H];
        const int h = u % H, rows = min(R, b.nq - b.r0), keys = self_keys_of(a.causal, b.r0, R, b.nq, b.nk);
        auto request = [&](int k, int to) {
            request_rows<D>(sKV + 2 * to * X, (const float *)a.kp, b.k0 + k, b.nk - k, h, H);
            request_rows<D>(sKV + (2 * to + 1) * X, (const float *)a.vp, b.k0 + k, b.nk - k, h, H);
            requested();
        };
        __syncthreads();
        if (keys > 0) {
            request_rows<D>(sQ, (const float *)a.qp, b.q0 + b.r0, rows, h, H);
            request(0, 0);
        }
        f2 acc[4][D / 32];
        float m[4], l[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            m[i] = -INFINITY;
            l[i] = 0.f;
#pragma unroll
            for (int c = 0; c < D / 32; ++c) acc[i][c] = pack2(0.f, 0.f);
        }
        for (int k = 0, at = 0; k < keys; k += R, at ^= 1) {
            const float *sK = sKV + 2 * at * X, *sV = sK + X;
            __syncthreads();                    // (the other buffer, P and the bias have been read)
            if (a.bias_on) load_near(sNb, a.dist, h, b.off + b.r0 - k);
            if (k + R < keys) {
                request(k + R, at ^ 1);
                arrived<1>();
            } else arrived<0>();
            __syncthreads();
            float s[4][4];
            dots<D>(sQ, sK, ty, tx, s);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int r = ty + 16 * i, lim = a.causal ? b.off + b.r0 + r + 1 : b.nk;
                float top = m[i];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int c = tx + 16 * j;
                    s[i][j] = fmaf(s[i][j], a.scale_log2, a.bias_on ? sNb[R - 1 + r - c] : 0.f);
                    if (k + c >= min(lim, b.nk)) s[i][j] = -INFINITY;
                    top = fmaxf(top, s[i][j]);
                }
#pragma unroll
                for (int o = 8; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
                const float use = top == -INFINITY ? 0.f : top, f = exp2f(m[i] - use);
                m[i] = top;
                float sum = 0.f;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float p = exp2f(s[i][j] - use);
                    sum += p;
                    sP[(tx + 16 * j) * PS + r] = p;
                }
#pragma unroll
                for (int o = 8; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
                l[i] = l[i] * f + sum;
                if (tx == 0) sF[r] = f;
            }
            __syncthreads();
#pragma unroll
            for (int i = 0; i < 4; ++i) scale_by(acc[i], sF[4 * ty + i]);
            const int edge = b.off + b.r0 - k + 1;      // (causal: row r sees the columns below edge + r)
            if (!a.causal || edge >= R) accumulate<D>(sP, sV, ty, tx, acc);
            else accumulate_cut<D, true>(sP, sV, ty, tx, acc, edge);
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (tx == 0) {
                const int r = ty + 16 * i;
                sF[r] = l[i] == 0.f ? 0.f : 1.f / l[i];
                if (r < rows) a.lse[(size_t)h * a.Tq + b.q0 + b.r0 + r] = l[i] == 0.f ? -INFINITY : (m[i] + log2f(l[i])) * 0.6931471805599453f;
            }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 4; ++i) scale_by(acc[i], sF[4 * ty + i]);
        store_rows<D>((float *)a.o, acc, b.q0 + b.r0, rows, h, H, ty, tx);
    }
}

// Unit u of ROWS: resident Q, dO, walked K, V: dQ and the sums of dS by bucket.  Else resident K, V, walked Q, dO: dK, dV.
template <int D, bool ROWS>
__device__ __forceinline__ void bwd_unit(const SelfBwdArgs &a, int u, float *sm) {
    constexpr int X = Shape<D>::X, NBUF = D == 64 ? 2 : 1;      // (two buffers of walked tiles do not fit at head_dim 128)
    float *sA = sm, *sB = sA + X, *sXY = sB + X, *sP = sXY + 2 * NBUF * X, *sD = sP + (ROWS ? 0 : R * PS);
    float *sL = sD + R * PS, *sDel = sL + R, *sNb = sDel + R, *sDiag = sNb + 2 * R;
    int *sBk = (int *)(sDiag + 2 * R);
    const int t = threadIdx.x, ty = t >> 4, tx = t & 15, H = a.H;
    const float LOG2E = 1.4426950408889634f;
    const SelfBlk b = a.blk.blk[u / H];
    const int h = u % H, rows = min(R, (ROWS ? b.nq : b.nk) - b.r0);
    const int c0 = ROWS ? 0 : self_first_row(a.causal, b.r0, b.nq, b.nk), c1 = ROWS ? self_keys_of(a.causal, b.r0, R, b.nq, b.nk) : b.nq;
    const int a0 = (ROWS ? b.q0 : b.k0) + b.r0, x0 = ROWS ? b.k0 : b.q0;
    auto request = [&](int c, int to) {
        request_rows<D>(sXY + 2 * to * X, (const float *)(ROWS ? a.kp : a.qp), x0 + c, c1 - c, h, H);
        request_rows<D>(sXY + (2 * to + 1) * X, (const float *)(ROWS ? a.vp : a.dop), x0 + c, c1 - c, h, H);
        requested();
    };
    __syncthreads();
    if (c0 < c1) {
        request_rows<D>(sA, (const float *)(ROWS ? a.qp : a.kp), a0, rows, h, H);
        request_rows<D>(sB, (const float *)(ROWS ? a.dop : a.vp), a0, rows, h, H);
        request(c0, 0);
    }
    auto stats = [&](int row, int n) {      // LSE' and delta of 64 query rows
        if (t >= R) return;
        const size_t r = (size_t)h * a.Tq + row + t;
        const float L = t < n ? a.lse[r] : -INFINITY;
        sL[t] = L == -INFINITY ? INFINITY : L * LOG2E;
        sDel[t] = t < n ? a.delta[r] : 0.f;
    };
    if (ROWS) stats(a0, rows);
    f2 acc1[4][D / 32], acc2[4][ROWS ? 1 : D / 32];
    float by_bucket = 0.f, far_sum[2] = {0.f, 0.f};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
#pragma unroll
        for (int c = 0; c < D / 32; ++c) acc1[i][c] = pack2(0.f, 0.f);
#pragma unroll
        for (int c = 0; c < (ROWS ? 1 : D / 32); ++c) acc2[i][c] = pack2(0.f, 0.f);
    }
    for (int c = c0, at = 0; c < c1; c += R, at ^= NBUF - 1) {
        const float *sX = sXY + 2 * at * X, *sY = sX + X;
        const int base = ROWS ? b.off + b.r0 - c : b.off + c - b.r0;      // distance of row 0 and column 0
        const int side = !a.bias_on ? 2 : base - (R - 1) >= a.dist.far ? 1 : base + (R - 1) <= -a.dist.far ? -1 : 0;
        __syncthreads();
        if (!ROWS) stats(x0 + c, c1 - c);
        if (a.bias_on) load_near(sNb, a.dist, h, base);
        if (ROWS && a.part != nullptr && side == 0 && t < 2 * R) sBk[t] = a.dist.bucket[self_dist_at(a.dist, base + t - (R - 1))];
        // (one buffer and two CTAs an SM instead at head_dim 64: slower, 345 us against 297 at 2 x 777 tokens: shared memory is what both want)
        if (NBUF == 2 && c + R < c1) {
            request(c + R, at ^ 1);
            arrived<1>();
        } else {
            if (NBUF == 1 && c > c0) request(c, 0);
            arrived<0>();
        }
        __syncthreads();
        float s[4][4], d[4][4];
        dots<D>(sA, sX, ty, tx, s);
        dots<D>(sB, sY, ty, tx, d);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int r = ty + 16 * i, k = tx + 16 * j, q = ROWS ? r : k, step = ROWS ? r - k : k - r;
                const bool keep = r < rows && c + k < c1 && (!a.causal || base + step >= 0);
                const float y = fmaf(s[i][j], a.scale_log2, a.bias_on ? sNb[R - 1 + step] : 0.f) - sL[q];
                const float p = keep ? exp2f(y) : 0.f, ds = keep ? p * (d[i][j] - sDel[q]) : 0.f;
                if (!ROWS) sP[k * PS + r] = p;
                else if (side == 1 || side == -1) far_sum[side == -1] += ds;
                sD[k * PS + r] = ds;
            }
        __syncthreads();
        if (!a.causal || base >= R - 1) {      // all pairs of the tile
            accumulate<D>(sD, sX, ty, tx, acc1);
            if constexpr (!ROWS) accumulate<D>(sP, sY, ty, tx, acc2);
        } else {      // rows: row r sees column c for base + r - c >= 0; keys: column c sees row r for base + c - r >= 0
            accumulate_cut<D, ROWS>(sD, sX, ty, tx, acc1, ROWS ? base + 1 : -base);
            if constexpr (!ROWS) accumulate_cut<D, ROWS>(sP, sY, ty, tx, acc2, -base);
        }
        if (ROWS && a.part != nullptr && side == 0) {
            if (t < 2 * R - 1) {      // the diagonal row - column = t - 63
                float v = 0.f;
                for (int r = max(0, t - (R - 1)); r < min(R, t + 1); ++r) v += sD[(r - (t - (R - 1))) * PS + r];
                sDiag[t] = v;
            }
            __syncthreads();
            if (t < a.buckets)
#pragma unroll 4
                for (int i = 0; i < 2 * R - 1; ++i) by_bucket += sBk[i] == t ? sDiag[i] : 0.f;
        }
    }
    if (ROWS && a.part != nullptr) {      // the sums beyond the last borders: over the warps in order
        __syncthreads();
#pragma unroll
        for (int g = 0; g < 2; ++g) {
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) far_sum[g] += __shfl_xor_sync(0xffffffffu, far_sum[g], o);
            if ((t & 31) == 0) sDiag[8 * g + (t >> 5)] = far_sum[g];
        }
        __syncthreads();
        for (int g = 0; g < 2; ++g)
            if (t == a.dist.bucket[g == 0 ? a.dist.n - 1 : 0])
                for (int i = 0; i < 8; ++i) by_bucket += sDiag[8 * g + i];
    }
    const float scale = a.scale;
#pragma unroll
    for (int i = 0; i < 4; ++i) scale_by(acc1[i], scale);
    if constexpr (ROWS) {
        store_rows<D>((float *)a.dq, acc1, a0, rows, h, H, ty, tx);
        if (a.part != nullptr && t < a.buckets) a.part[((size_t)b.id * H + h) * a.buckets + t] = by_bucket;
    } else {
        store_rows<D>((float *)a.dk, acc1, a0, rows, h, H, ty, tx);
        store_rows<D>((float *)a.dv, acc2, a0, rows, h, H, ty, tx);
    }
}

// Both in one launch, the units of either by turns, dearest first: they fill each other's last waves.
template <int D>
__global__ void __launch_bounds__(256, 1) k_self_bwd_f32(const __grid_constant__ SelfBwdArgs keys, const __grid_constant__ SelfBwdArgs rows) {
    extern __shared__ float sm[];
    pdl_wait();
    pdl_launch_dependents();
    const int nk = *keys.blk.count * keys.H, nq = *rows.blk.count * rows.H, both = min(nk, nq);
    for (int c = blockIdx.x; c < nk + nq; c += gridDim.x) {
        const bool is_rows = c < 2 * both ? (c & 1) != 0 : nq > nk;
        const int u = c < 2 * both ? c >> 1 : c - both;
        if (is_rows) bwd_unit<D, true>(rows, u, sm);
        else bwd_unit<D, false>(keys, u, sm);
    }
}

template <int D>
int fwd(const SelfFwdArgs &a, cudaStream_t st) {
    constexpr int smem = (5 * Shape<D>::X + R * PS + R + 2 * R) * 4;
    static DevOnce attr;
    if (!attr.done()) {
        HDT_CUDA_CHECK(cudaFuncSetAttribute(k_self_fwd_f32<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
        attr.set();
    }
    const long long units = (long long)a.q.most * a.H;
    HDT_CUDA_CHECK(launch_dependent(k_self_fwd_f32<D>, true, dim3((unsigned)(units < MOST_CTAS ? units : MOST_CTAS)), 256, smem, st, a));
    return HDT_OK;
}
template <int D>
int bwd(const SelfBwdArgs &keys, const SelfBwdArgs &rows, cudaStream_t st) {
    constexpr int smem = ((D == 64 ? 6 : 4) * Shape<D>::X + 2 * R * PS + 2 * R + 2 * R + 2 * R + 2 * R) * 4;
    static DevOnce attr;
    if (!attr.done()) {
        HDT_CUDA_CHECK(cudaFuncSetAttribute(k_self_bwd_f32<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
        attr.set();
    }
    // (a CTA per unit, dearest first: one goes to the SM that is free first.  148 CTAs with units dealt to them: 326 us against 271 at 2 x 777 tokens, 12 x 64)
    const long long units = ((long long)keys.blk.most + rows.blk.most) * keys.H;
    HDT_CUDA_CHECK(launch_dependent(k_self_bwd_f32<D>, true, dim3((unsigned)(units < MOST_CTAS ? units : MOST_CTAS)), 256, smem, st, keys, rows));
    return HDT_OK;
}

}  // namespace

int launch_self_fwd_f32(const SelfFwdArgs &a, int head_dim, cudaStream_t st) { return head_dim == 64 ? fwd<64>(a, st) : fwd<128>(a, st); }
int launch_self_bwd_f32(const SelfBwdArgs &keys, const SelfBwdArgs &rows, int head_dim, cudaStream_t st) {
    return head_dim == 64 ? bwd<64>(keys, rows, st) : bwd<128>(keys, rows, st);
}

}  // namespace hdt
