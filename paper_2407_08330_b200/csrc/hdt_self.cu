// Self-attention with a learned relative position bias: C entry points, what a call prepares on the device, the step of
// autoregressive decoding, and the last sum of the bias' gradient.
//
// Preparation (one launch): the documents' blocks of rows, ordered by cost (a persistent kernel takes the dearest
// first), from offsets that only the device knows; and the bias by distance, [heads][distances], so that a tile reads a
// vector of it and nobody looks for buckets again.  Latency: 4 x 4096 tokens about 5 us.
//
// Decoding (few rows per document): bound by HBM, the keys and values once.  A warp takes a piece of a document's keys for
// one head and up to four rows; every lane group has a softmax of its own, joined at the piece's end, the pieces by
// k_self_join (8 documents of 4096 keys, 12 x 64, caches that L2 does not hold, with both launches: bf16 23 us, 4.4 TB/s, fp32 36, 5.6; four
// rows each 45 and 52; a cache of bf16 that L2 holds for the most part 18).  A document with more rows takes longer pieces, so that the number of pieces is bounded by the keys.
#include <math.h>

#include <type_traits>

#include "hdt_rows.cuh"
#include "hdt_self.cuh"

namespace hdt {
namespace {

struct PrepList { SelfBlk *raw, *out; int *count; int rows, of_keys, most; };
struct PrepArgs {
    const int32_t *cu_q, *cu_k, *len_k;
    int B, Tq, Tk, H, n_lists;
    PrepList list[2];
    int behind;               // launched as a programmatic dependent of a kernel of which it reads nothing: it ends behind it
    SelfRel rel;
    const void *table;
    int dtype;
    float *bias;
    unsigned char *bucket;
    int lo, n;
};
// A document's rows, whatever the arrays hold: inside the tensors, never negative.
struct Doc { int q0, nq, k0, nk; };
__device__ __forceinline__ Doc document(const int32_t *cu_q, const int32_t *cu_k, const int32_t *len_k, int b, int Tq, int Tk) {
    Doc d;
    d.q0 = min(max(cu_q[b], 0), Tq);
    d.nq = min(max(cu_q[b + 1], d.q0), Tq) - d.q0;
    d.k0 = min(max(cu_k[b], 0), Tk);
    d.nk = min(max(cu_k[b + 1], d.k0), Tk) - d.k0;
    if (len_k != nullptr) d.nk = min(max(len_k[b], 0), d.nk);
    return d;
}
__device__ __forceinline__ float load_f32(const void *p, size_t i, int dtype) {
    return dtype == HDT_F32 ? ((const float *)p)[i] : __bfloat162float(((const __nv_bfloat16 *)p)[i]);
}
__device__ __forceinline__ float bias_base2(const void *table, size_t i, int dtype) {
    const float v = load_f32(table, i, dtype);
    return (isfinite(v) ? fminf(fmaxf(v, -SELF_MAX_BIAS), SELF_MAX_BIAS) : v) * 1.4426950408889634f;
}

// x + y of numbers that are not negative, at most the largest of them: documents that overlap may have any number of blocks.
__host__ __device__ __forceinline__ int add_up_to_most(int x, int y) {
    const unsigned v = (unsigned)x + (unsigned)y;
    return v > 0x7fffffffu ? 0x7fffffff : (int)v;
}
// Inclusive scan over the CTA's 1024 threads, of such sums.
__device__ __forceinline__ int scan1024(int v, int *s_warp) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, v, o);
        if (lane >= o) v = add_up_to_most(v, y);
    }
    if (lane == 31) s_warp[warp] = v;
    __syncthreads();
    if (warp == 0) {
        int w = s_warp[lane];
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, w, o);
            if (lane >= o) w = add_up_to_most(w, y);
        }
        s_warp[lane] = w;
    }
    __syncthreads();
    if (warp > 0) v = add_up_to_most(v, s_warp[warp - 1]);
    __syncthreads();
    return v;
}

__global__ void __launch_bounds__(1024) k_self_prep(const __grid_constant__ PrepArgs a) {
    constexpr int BINS = 1024;
    __shared__ int s_warp[32], s_pre[1024], s_bin[BINS];
    __shared__ Doc s_doc[1024];
    const int t = threadIdx.x;
    pdl_launch_dependents();
    if ((int)blockIdx.x >= a.n_lists) {      // the bias by distance
        const int i = ((int)blockIdx.x - a.n_lists) * 1024 + t;
        if (i >= a.n) {
            if (a.behind) pdl_wait();
            return;
        }
        const int bk = self_bucket(a.rel, a.lo + i);
        a.bucket[i] = (unsigned char)bk;
        for (int h = 0; h < a.H; ++h) a.bias[(size_t)h * a.n + i] = bias_base2(a.table, (size_t)bk * a.H + h, a.dtype);
        if (a.behind) pdl_wait();
        return;
    }
    const PrepList L = a.list[blockIdx.x];
    s_bin[t] = 0;
    int total = 0;
    SelfBlk mine{};      // block number t, where this thread comes to it, stays in registers; the others take the way through `raw`
    bool have = false;
    for (int b0 = 0; b0 < a.B; b0 += 1024) {
        int nb = 0;
        if (b0 + t < a.B) {
            const Doc d = document(a.cu_q, a.cu_k, a.len_k, b0 + t, a.Tq, a.Tk);
            s_doc[t] = d;
            nb = ((L.of_keys ? d.nk : d.nq) + L.rows - 1) / L.rows;
        }
        s_pre[t] = scan1024(nb, s_warp);
        __syncthreads();
        const int n = s_pre[1023];
        for (int i = t; i < n; i += 1024) {
            int lo = 0, hi = 1023;           // first document whose blocks end behind i
            while (lo < hi) {
                const int mid = (lo + hi) >> 1;
                if (s_pre[mid] > i) hi = mid;
                else lo = mid + 1;
            }
            const Doc d = s_doc[lo];
            SelfBlk x;
            x.q0 = d.q0; x.nq = d.nq; x.k0 = d.k0; x.nk = d.nk; x.off = d.nk - d.nq;
            x.r0 = (i - (lo > 0 ? s_pre[lo - 1] : 0)) * L.rows;
            x.tiles = L.of_keys ? (d.nq - self_first_row(a.rel.causal, x.r0, d.nq, d.nk) + 127) >> 7 : (self_keys_of(a.rel.causal, x.r0, L.rows, d.nq, d.nk) + 127) >> 7;
            x.id = total + i;
            if (x.id >= L.most) break;       // (documents that overlap: there is room for those that do not)
            if (x.id == t) {
                mine = x;
                have = true;
            } else L.raw[x.id] = x;
            atomicAdd(&s_bin[BINS - 1 - min(x.tiles, BINS - 1)], 1);
        }
        total = min(add_up_to_most(total, n), L.most);      // (so that the next documents' numbers stay inside 32 bits)
        __syncthreads();
    }
    const int n_bin = s_bin[t];
    const int start = scan1024(n_bin, s_warp) - n_bin;      // (its barriers lie between the last read and the next write)
    s_bin[t] = start;
    __syncthreads();
    for (int i = t; i < total; i += 1024) {
        const SelfBlk x = i == t && have ? mine : L.raw[i];
        L.out[atomicAdd(&s_bin[BINS - 1 - min(x.tiles, BINS - 1)], 1)] = x;
    }
    if (t == 0) *L.count = total;
    if (a.behind) pdl_wait();
}

// Sums of the blocks' partial sums, a CTA per head; threads of one bucket take every G-th block, then meet in order.
__global__ void __launch_bounds__(1024) k_self_dbias(const float *part, const int *count, int H, int buckets, int dtype, void *out) {
    __shared__ float s[1024];
    const int h = blockIdx.x, G = 1024 / buckets, b = threadIdx.x % buckets, g = threadIdx.x / buckets;
    pdl_wait();
    const int n = part != nullptr ? *count : 0;
    float v = 0.f;
    if (g < G)
#pragma unroll 4
        for (int i = g; i < n; i += G) v += part[((size_t)i * H + h) * buckets + b];
    s[threadIdx.x] = v;
    __syncthreads();
    if (g != 0) return;
    for (int i = 1; i < G; ++i) v += s[i * buckets + b];
    if (dtype == HDT_F32) ((float *)out)[(size_t)b * H + h] = v;
    else ((__nv_bfloat16 *)out)[(size_t)b * H + h] = __float2bfloat16(v);
}

// ---- decoding -----------------------------------------------------------------------------------
struct StepArgs {
    const int32_t *cu_q, *cu_k, *len_k;
    int B, Tq, Tk, H, piece, dtype, items;      // items: an upper limit
    const void *q, *k, *v, *table;
    void *o;
    float *lse, *part_o, *part_ml;      // [slot][H][D], [slot][H][2]; a slot per (item, row of its group)
    float scale_log2;
    int *before;                        // [B]: items of the documents before (many documents), [B] of all, and [B + 1] whether any has several
                                        // pieces; or nullptr: every warp counts them itself
    SelfRel rel;
};
template <int RG>
struct StepDoc {      // how a document's work is cut: row groups x pieces of keys
    int groups, per, pieces;
    __device__ __forceinline__ StepDoc(const Doc &d, int piece) {
        groups = (d.nq + RG - 1) / RG;
        per = (int)max(1ll, min((long long)piece * groups, (long long)d.nk));
        pieces = groups == 0 ? 0 : max(1, d.nk / per + (d.nk % per > 0));
    }
    __device__ __forceinline__ int items() const { return groups * pieces; }
};
// Items before every document, and whether there is anything to join.
template <int RG>
__global__ void __launch_bounds__(1024) k_self_items(const __grid_constant__ StepArgs a) {
    __shared__ int s_warp[32], s_sum;
    pdl_launch_dependents();
    int base = 0, several = 0;
    for (int b0 = 0; b0 < a.B; b0 += 1024) {
        const int b = b0 + (int)threadIdx.x;
        int n = 0;
        if (b < a.B) {
            const StepDoc<RG> cut(document(a.cu_q, a.cu_k, a.len_k, b, a.Tq, a.Tk), a.piece);
            n = cut.items();
            several |= cut.pieces > 1;
        }
        const int pre = scan1024(n, s_warp);
        if (b < a.B) a.before[b] = add_up_to_most(base, pre - n);
        if (threadIdx.x == 1023) s_sum = pre;
        __syncthreads();
        base = add_up_to_most(base, s_sum);
        __syncthreads();
    }
    several = __syncthreads_or(several);
    if (threadIdx.x == 0) {
        a.before[a.B] = base;
        a.before[a.B + 1] = several;
    }
}
// The last of n ascending numbers that is at most x (-1: none), by a whole warp, thirty-two at a time.
template <class F>
__device__ __forceinline__ int last_at_most(int n, int x, F get) {
    const int lane = threadIdx.x & 31;
    int lo = 0, len = n;
    while (len > 0) {
        const int step = (len + 31) / 32, i = lo + lane * step;
        const unsigned m = __ballot_sync(0xffffffffu, lane * step < len && get(i) <= x);
        if (m == 0) return lo - 1;
        const int k = 31 - __clz(m);
        if (step == 1) return lo + k;
        const int end = lo + len;
        lo += k * step;
        len = min(step, end - lo);
    }
    return -1;
}
// The document that item x, or row x, lies in, and how many items come before the document (whole warp).  Up to 64 documents, whose
// loads are two rounds, every warp counts; beyond, k_self_items has, and the document is searched for.  12 x 64 bf16, counted and
// searched: 32 x 100 keys 9.8 and 12.1 us, 64 x 500 23.0 and 25.6, 65 x 500 23.9 and 25.2, 128 x 100 18.2 and 16.2, 128 x 500 44.7 and
// 42.8, 1000 x 100 330 and 73, 4000 x 50 4014 and 180.
template <int RG, bool BY_ROW>
__device__ __forceinline__ bool find_doc(const StepArgs &a, int x, Doc &d, int &before) {
    if (a.before != nullptr) {
        const int b = BY_ROW ? last_at_most(a.B, x, [&](int i) { return a.cu_q[i]; }) : last_at_most(a.B, x, [&](int i) { return a.before[i]; });
        if (b < 0) return false;
        d = document(a.cu_q, a.cu_k, a.len_k, b, a.Tq, a.Tk);
        before = a.before[b];
        return BY_ROW ? x >= d.q0 && x < d.q0 + d.nq : (unsigned)x - (unsigned)before < (unsigned)StepDoc<RG>(d, a.piece).items();
    }
    const int lane = threadIdx.x & 31;
    int base = 0;
    for (int b0 = 0; b0 < a.B; b0 += 32) {
        Doc m{0, 0, 0, 0};
        if (b0 + lane < a.B) m = document(a.cu_q, a.cu_k, a.len_k, b0 + lane, a.Tq, a.Tk);
        const int n = StepDoc<RG>(m, a.piece).items();
        int pre = n;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, pre, o);
            if (lane >= o) pre += y;
        }
        const int first = base + pre - n;
        const unsigned hit = __ballot_sync(0xffffffffu, n > 0 && (BY_ROW ? x >= m.q0 && x < m.q0 + m.nq : x >= first && x < first + n));
        if (hit) {
            const int src = __ffs(hit) - 1;
            d.q0 = __shfl_sync(0xffffffffu, m.q0, src);
            d.nq = __shfl_sync(0xffffffffu, m.nq, src);
            d.k0 = __shfl_sync(0xffffffffu, m.k0, src);
            d.nk = __shfl_sync(0xffffffffu, m.nk, src);
            before = __shfl_sync(0xffffffffu, first, src);
            return true;
        }
        base += __shfl_sync(0xffffffffu, pre, 31);
    }
    return false;
}
// A key's row lies on D / 8 lanes, a lane group has four keys at a time (and, one row, bf16, the next four in flight); each lane keeps the
// score of one of them, so an exponential is computed twice or four times and not by every lane.
template <int D, bool BF16, int RG>
__global__ void __launch_bounds__(128, RG == 1 ? 4 : 3) k_self_step(const __grid_constant__ StepArgs a) {
    constexpr int LPK = D / 8, KPI = 32 / LPK, C = 4;
    using W = Raw<BF16, LPK>;
    constexpr size_t ROW = D * (BF16 ? 2 : 4);
    pdl_launch_dependents();
    const int lane = threadIdx.x & 31, l = lane % LPK, slot = lane / LPK, src = lane - l;
    const unsigned mask = 0xffffffffu;
    const int wid = blockIdx.x * 4 + (threadIdx.x >> 5), item = wid / a.H, h = wid % a.H;
    const float far_bias = a.rel.on ? bias_base2(a.table, (size_t)self_bucket(a.rel, a.rel.far) * a.H + h, a.dtype) : 0.f;
    Doc d;
    int before;
    pdl_wait();
    if (item >= (a.before != nullptr ? min(a.items, a.before[a.B]) : a.items) || !find_doc<RG, false>(a, item, d, before)) return;
    const StepDoc<RG> cut(d, a.piece);
    const int g = (item - before) / cut.pieces, pc = (item - before) % cut.pieces, r0 = g * RG, nr = min(RG, d.nq - r0);
    const int pos0 = d.nk - d.nq + r0;                                  // position of the group's first row
    const int kb = min(pc * cut.per, d.nk);
    int ke = min(kb + cut.per, d.nk);
    if (a.rel.causal) ke = max(kb, min(ke, pos0 + nr));
    constexpr bool AHEAD = RG == 1 && BF16;      // (else the registers do not hold the next four keys)
    W q[RG], x[C], y[C], x1[AHEAD ? C : 1], y1[AHEAD ? C : 1];
    RowSoftmax S[RG];
    const char *kp = (const char *)a.k + ((size_t)d.k0 * a.H + h) * ROW, *vp = (const char *)a.v + ((size_t)d.k0 * a.H + h) * ROW;
    auto request = [&](int k0, W (&kx)[C], W (&vx)[C]) {
#pragma unroll
        for (int c = 0; c < C; ++c) {      // (past the end: the last key, weight 0)
            const size_t o = (size_t)min(k0 + slot * C + c, ke - 1) * a.H * ROW;
            kx[c].load(kp + o, 0u, l);
            vx[c].load(vp + o, 0u, l);
        }
    };
    if constexpr (AHEAD)
        if (kb < ke) request(kb, x1, y1);
#pragma unroll
    for (int r = 0; r < RG; ++r) {
        q[r].load((const char *)a.q + ((size_t)(d.q0 + r0 + min(r, nr - 1)) * a.H + h) * ROW, 0u, l);
        S[r].clear();
    }
    auto chunk = [&](int k0, auto cut) {      // cut: the first row does not see all of these keys
        if constexpr (AHEAD) {
#pragma unroll
            for (int c = 0; c < C; ++c) {
                x[c] = x1[c];
                y[c] = y1[c];
            }
            if (k0 + KPI * C < ke) request(k0 + KPI * C, x1, y1);
        } else request(k0, x, y);
        const int key = k0 + slot * C + (l & (C - 1));                  // the key whose score this lane keeps
#pragma unroll
        for (int i = 0; i < RG; ++i) {
            const int r = decltype(cut)::value ? RG - 1 - i : i;
            if constexpr (decltype(cut)::value)      // last row first: the values that a row does not see are taken out for it and those before it (0 times what is not finite is no number)
#pragma unroll
                for (int c = 0; c < C; ++c)
                    if (k0 + slot * C + c > pos0 + r) y[c].clear();
            float sc[C];
            dots<C>(q[r], x, sc);
            float s = reduce_scatter<C, LPK>(sc, l, mask) * a.scale_log2;
            const int dist = pos0 + r - key;
            if (a.rel.on) s += dist >= a.rel.far ? far_bias : bias_base2(a.table, (size_t)self_bucket(a.rel, dist) * a.H + h, a.dtype);
            if (key >= ke || (a.rel.causal && dist < 0)) s = -INFINITY;
            const float p = S[r].template add<C>(s, mask);
            axpys<C>(S[r].acc, p, y, mask, src);
        }
    };
    // (the last keys apart: the loop over the others has nothing to look at.  In one loop: four rows each of 8 caches of 1024 to 4096 keys 33 -> 38 us)
    const int end = RG > 1 && a.rel.causal ? min(ke, pos0 + 2 - KPI * C) : ke;
    int k0 = kb;
    for (; k0 < end; k0 += KPI * C) chunk(k0, std::false_type{});
    if constexpr (RG > 1)
        for (; k0 < ke; k0 += KPI * C) chunk(k0, std::true_type{});
#pragma unroll
    for (int r = 0; r < RG; ++r) {
        if (r > 0 && r >= nr) break;
#pragma unroll
        for (int o = 1; o < C; o *= 2) S[r].l += __shfl_xor_sync(mask, S[r].l, o);
#pragma unroll
        for (int o = LPK; o < 32; o <<= 1) {      // the lane groups' softmaxes
            f2 z[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) z[u] = __shfl_xor_sync(mask, S[r].acc[u], o);
            const float m2 = __shfl_xor_sync(mask, S[r].m, o), l2 = __shfl_xor_sync(mask, S[r].l, o);
            S[r].merge(m2, l2, z);
        }
        if (lane >= LPK) continue;
        const int row = d.q0 + r0 + r;
        if (cut.pieces == 1) {
            // (a sum that is no number stays one)
            const float inv = S[r].l == 0.f ? 0.f : 1.f / S[r].l;
#pragma unroll
            for (int u = 0; u < 4; ++u) S[r].acc[u] = mul2(S[r].acc[u], pack2(inv, inv));
            W::store((char *)a.o + ((size_t)row * a.H + h) * ROW, 0u, l, S[r].acc);
            if (l == 0) a.lse[(size_t)h * a.Tq + row] = S[r].l == 0.f ? -INFINITY : (S[r].m + log2f(S[r].l)) * 0.6931471805599453f;
        } else {
            const size_t at = ((size_t)item * RG + r) * a.H + h;
            Raw<BF16, LPK>::store_f32(a.part_o + at * D, 0, l, S[r].acc);
            if (l == 0) *reinterpret_cast<float2 *>(a.part_ml + at * 2) = make_float2(S[r].m, S[r].l);
        }
    }
}

// The pieces of a row, a CTA: its four warps take every fourth piece, four of them in flight, and meet in order.
template <int D, bool BF16, int RG>
__device__ __forceinline__ void join_row(const StepArgs &a, int row, int h, float (*s_acc)[D], float (*s_ml)[2]) {
    constexpr int E = D / 32;
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    Doc d;
    int before;
    // (before the wait where every warp counts: the kernel in front does not write the offsets, and began behind what did)
    const bool found = find_doc<RG, true>(a, row, d, before);
    pdl_wait();
    if (!found) return;
    const StepDoc<RG> cut(d, a.piece);
    const int r = row - d.q0, first = before + (r / RG) * cut.pieces;
    if (cut.pieces == 1 || first < 0 || cut.pieces > a.items - first) return;      // written by the one warp that had the row (or no valid offsets)
    auto at = [&](int i) { return ((size_t)(first + i) * RG + r % RG) * a.H + h; };
    float m = -INFINITY, l = 0.f, acc[E];
#pragma unroll
    for (int e = 0; e < E; ++e) acc[e] = 0.f;
    for (int i0 = w; i0 < cut.pieces; i0 += 16) {
        float2 ml[4];
        float x[4][E];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int i = min(i0 + 4 * u, cut.pieces - 1);
            ml[u] = *reinterpret_cast<const float2 *>(a.part_ml + at(i) * 2);
#pragma unroll
            for (int e = 0; e < E; ++e) x[u][e] = a.part_o[at(i) * D + lane * E + e];
        }
        float top = m;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            if (i0 + 4 * u >= cut.pieces) ml[u] = make_float2(-INFINITY, 0.f);
            top = fmaxf(top, ml[u].x);
        }
        const float use = top == -INFINITY ? 0.f : top, f = exp2f(m - use);
        m = top;
        l *= f;
#pragma unroll
        for (int e = 0; e < E; ++e) acc[e] *= f;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const float f = exp2f(ml[u].x - use);
            l += ml[u].y * f;
#pragma unroll
            for (int e = 0; e < E; ++e) acc[e] = fmaf(x[u][e], f, acc[e]);
        }
    }
#pragma unroll
    for (int e = 0; e < E; ++e) s_acc[w][lane * E + e] = acc[e];
    if (lane == 0) { s_ml[w][0] = m; s_ml[w][1] = l; }
    __syncthreads();
    if (threadIdx.x >= D) return;
    float top = -INFINITY, y = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) top = fmaxf(top, s_ml[i][0]);
    const float use = top == -INFINITY ? 0.f : top;
    l = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float f = exp2f(s_ml[i][0] - use);
        l += s_ml[i][1] * f;
        y = fmaf(s_acc[i][threadIdx.x], f, y);
    }
    y *= l == 0.f ? 0.f : 1.f / l;
    const size_t out = ((size_t)row * a.H + h) * D + threadIdx.x;
    if constexpr (BF16) ((__nv_bfloat16 *)a.o)[out] = __float2bfloat16(y);
    else ((float *)a.o)[out] = y;
    if (threadIdx.x == 0) a.lse[(size_t)h * a.Tq + row] = l == 0.f ? -INFINITY : (top + log2f(l)) * 0.6931471805599453f;
}
template <int D, bool BF16, int RG>
__global__ void __launch_bounds__(128) k_self_join(const __grid_constant__ StepArgs a) {
    __shared__ float s_acc[4][D], s_ml[4][2];
    if (a.before != nullptr) {
        pdl_wait();
        if (a.before[a.B + 1] == 0) return;
    }
    const int n = a.Tq * a.H;
    for (int x = blockIdx.x; x < n; x += gridDim.x) {      // (the host sees to it that this ends inside 32 bits)
        if (x != (int)blockIdx.x) __syncthreads();
        join_row<D, BF16, RG>(a, x / a.H, x % a.H, s_acc, s_ml);
    }
}

// ---- host ---------------------------------------------------------------------------------------
// Whether the distance d has passed the border far^(k/m) e^(1 - k/m), i.e. d^m e^k >= far^k e^m.  The difference of
// the logarithms is known to about 1e-15 of their size; where it is that small, the two products are compared by their prime
// factors.
bool same_product(int d, int m, int far, int k, int e) {      // d^m e^(k - m) == far^k ?
    for (int p = 2; d > 1 || far > 1 || e > 1; ++p) {
        if ((long long)p * p > (d > far ? (d > e ? d : e) : (far > e ? far : e))) p = d > 1 ? d : far > 1 ? far : e;
        long long n = 0;
        while (d % p == 0) { d /= p; n += m; }
        while (e % p == 0) { e /= p; n += k - m; }
        while (far % p == 0) { far /= p; n -= k; }
        if (n != 0) return false;
    }
    return true;
}
bool passed(int d, int m, int far, int k, int e) {
    const double x = m * log((double)d) + (k - m) * log((double)e) - k * log((double)far);
    return x > 1e-9 || (x > -1e-9 && (same_product(d, m, far, k, e) || x > 0));
}
// The buckets of one direction: one per distance below half of them, then logarithmic up to max_distance.
void rel_fill(SelfRel *r, int buckets, int max_distance, int causal) {
    static thread_local SelfRel last{};
    static thread_local int last_far = -1;
    if (last_far == max_distance && last.buckets == buckets && last.causal == causal) { *r = last; return; }
    SelfRel x{};
    x.on = 1; x.causal = causal; x.buckets = buckets; x.one_way = causal ? buckets : buckets / 2;
    const int e = x.one_way / 2, m = x.one_way - e;
    for (int b = 0; b <= e; ++b) x.first[b] = b;
    for (int k = 1; k < m; ++k) {
        int d = (int)(e * pow((double)max_distance / e, (double)k / m)) - 1;
        if (d < x.first[e + k - 1]) d = x.first[e + k - 1];
        while (!passed(d, m, max_distance, k, e)) ++d;
        x.first[e + k] = d;
    }
    x.far = x.first[x.one_way - 1];
    last = *r = x;
    last_far = max_distance;
}

size_t al(size_t n) { return (n + 255) / 256 * 256; }
constexpr int STEP_COUNTED = 64;  // documents up to which every warp of a step counts their items itself
constexpr int JOIN_CTAS = 16;      // CTAs of a join to an SM (all at once; more rows: one after the other)
constexpr int STEP_ROWS = 4;      // rows per document, on average, up to which a call is a step of decoding
bool is_step(int B, int Tq) { return B > 0 && Tq <= STEP_ROWS * (long long)B; }
// Keys of a piece, for documents of one length (the host knows no other): a piece is a warp, `most` of them are resident at once and
// take turns in waves, and a warp takes about as long to begin as for 32 keys.  Of the pieces that fill 1 .. 8 waves, those that
// are done first.  (Against one wave of fourteen warps to an SM: 8 x 4096 keys, which L2 held for the most part, 19.4 -> 18.0 us, 128 x 500
// 48 -> 42, 100 x 3000 209 -> 155; at most 256 keys: 100 x 3000 157, but 64 x 2000 72 -> 66 here, 128 x 500 50.)  The documents' room is
// what the host knows: where a third of a cache is unused, a third of the warps has nothing to do.
int step_piece(int B, int Tk, int H, int rg) {
    const long long most = (rg == 1 ? 16 : 12) * PLAN_SMS, b = B > 0 ? B : 1, keys = (Tk + b - 1) / b;
    long long best = 0, piece = 64;
    for (int w = 1; w <= 8; ++w) {
        const long long p = most * w / (b * H), most_p = (keys + 63) / 64, n = p < 1 ? 1 : p > most_p && most_p > 0 ? most_p : p;
        const long long per = ((keys + n - 1) / n + 15) / 16 * 16, waves = (b * H * ((keys + per - 1) / (per > 0 ? per : 1)) + most - 1) / most, cost = waves * (per + 32);
        if (w == 1 || cost < best) {
            best = cost;
            piece = per;
        }
    }
    return (int)(piece < 64 ? 64 : piece);
}
// (a document of g row groups has at most keys / piece + g items)
long long step_items(int B, int Tq, int Tk, int H, int rg) { return (long long)Tk / step_piece(B, Tk, H, rg) + Tq / rg + B + 2; }
int step_group(int B, int Tq) { return Tq <= B ? 1 : STEP_ROWS; }

struct Layout {
    int rows_q, most_q, most_k, n;
    size_t count, raw, q, k, bias, bucket, delta, part, part_o, part_ml, before, total;
};
long long blocks(int T, int B, int rows) { return (long long)T / rows + B; }
Layout layout(int B, int Tq, int Tk, int H, int D, int buckets, int max_distance, int causal, int dtype, int bwd) {
    Layout L{};
    size_t at = 0;
    auto take = [&](size_t n) { const size_t x = at; at += al(n); return x; };
    if (!bwd && is_step(B, Tq)) {
        const int rg = step_group(B, Tq);
        const long long slots = step_items(B, Tq, Tk, H, rg) * rg;
        L.part_o = take((size_t)slots * H * D * 4);
        L.part_ml = take((size_t)slots * H * 8);
        if (B > STEP_COUNTED) L.before = take(((size_t)B + 2) * 4);
    } else {
        L.rows_q = dtype == HDT_F32 ? SELF_F32_ROWS : 128;
        // two row tiles to a unit (they share the K and V tiles) where that leaves a unit for every SM
        if (!bwd && dtype == HDT_BF16 && blocks(Tq, B, 256) * H >= PLAN_SMS) L.rows_q = 256;
        L.most_q = (int)blocks(Tq, B, L.rows_q);
        L.most_k = bwd ? (int)blocks(Tk, B, dtype == HDT_F32 ? SELF_F32_ROWS : 128) : 0;
        L.count = take(8);
        L.raw = take((size_t)(L.most_q + L.most_k) * sizeof(SelfBlk));
        L.q = take((size_t)L.most_q * sizeof(SelfBlk));
        L.k = take((size_t)L.most_k * sizeof(SelfBlk));
        if (buckets > 0) {
            L.n = causal ? max_distance + 1 : 2 * max_distance + 1;      // (an upper limit: the last border may lie before max_distance)
            L.bias = take((size_t)L.n * H * 4);
            L.bucket = take((size_t)L.n);
        }
        if (bwd) {
            L.delta = take((size_t)H * Tq * 4);
            if (buckets > 0) L.part = take((size_t)(dtype == HDT_F32 ? L.most_q : L.most_k) * H * buckets * 4);
        }
    }
    L.total = at > 0 ? at : 256;
    return L;
}
int sizes_check(int B, int Tq, int Tk, int H, int D, int buckets, int max_distance, int causal, int dtype, const char *who) {
    if (B < 0 || Tq < 0 || Tk < 0 || H < 1 || buckets < 0) return set_error(HDT_ERR_INVALID_ARG, "%s: negative size or no head", who);
    if (D != 64 && D != 128) return set_error(HDT_ERR_UNSUPPORTED, "%s: head_dim %d not supported (64 or 128)", who, D);
    if (dtype != HDT_F32 && dtype != HDT_BF16) return set_error(HDT_ERR_UNSUPPORTED, "%s: unknown dtype %d", who, dtype);
    if (H > 65535 || (long long)(Tq > Tk ? Tq : Tk) + B > 0x7ffff000LL) return set_error(HDT_ERR_UNSUPPORTED, "%s: more rows or heads than the kernels' grids hold", who);
    // (documents that overlap may fill the lists of both sides, and the fp32 kernels walk both with a stride of up to 2^20)
    if ((blocks(Tq, B, SELF_F32_ROWS) + blocks(Tk, B, SELF_F32_ROWS)) * H > 0x7fe00000LL || step_items(B, Tq, Tk, H, step_group(B, Tq)) * H > 0x7ffff000LL || (is_step(B, Tq) && (long long)Tq * H > 0x7fff0000LL))
        return set_error(HDT_ERR_UNSUPPORTED, "%s: more blocks than the kernels' grids hold", who);
    if (buckets > 0) {
        const int one = causal ? buckets : buckets / 2;
        if (buckets > SELF_MAX_BUCKETS) return set_error(HDT_ERR_UNSUPPORTED, "%s: at most %d buckets", who, SELF_MAX_BUCKETS);
        if (one < 2 || (!causal && buckets % 2 != 0)) return set_error(HDT_ERR_INVALID_ARG, "%s: at least two buckets a direction, the same number both ways", who);
        if (max_distance <= one / 2) return set_error(HDT_ERR_INVALID_ARG, "%s: max_distance must exceed half of a direction's buckets", who);
        if (max_distance > SELF_MAX_DISTANCE) return set_error(HDT_ERR_UNSUPPORTED, "%s: max_distance at most %d", who, SELF_MAX_DISTANCE);
    }
    return HDT_OK;
}
int ptr_check(const void *p, const char *who) {
    if (!p) return set_error(HDT_ERR_INVALID_ARG, "%s: null tensor pointer", who);
    if ((uintptr_t)p & 15) return set_error(HDT_ERR_INVALID_ARG, "%s: tensors must be 16-byte aligned", who);
    return HDT_OK;
}
int ws_check(const void *ws, size_t n, size_t need, const char *who) {
    if (!ws || n < need) return set_error(HDT_ERR_WORKSPACE, "%s: workspace %zu < required %zu", who, n, need);
    if ((uintptr_t)ws & 255) return set_error(HDT_ERR_INVALID_ARG, "%s: workspace must be 256-byte aligned", who);
    return HDT_OK;
}

template <int D, bool BF16, int RG>
int step_go(StepArgs a, cudaStream_t st) {
    a.items = (int)step_items(a.B, a.Tq, a.Tk, a.H, RG);
    if (a.before != nullptr) HDT_CUDA_CHECK(launch_dependent(k_self_items<RG>, false, dim3(1), 1024, 0, st, a));
    HDT_CUDA_CHECK(launch_dependent(k_self_step<D, BF16, RG>, a.before != nullptr, dim3((unsigned)(((long long)a.items * a.H + 3) / 4)), 128, 0, st, a));
    if (a.Tk <= a.piece) return HDT_OK;      // no document of several pieces
    const long long rows = (long long)a.Tq * a.H, most = JOIN_CTAS * PLAN_SMS;
    HDT_CUDA_CHECK(launch_dependent(k_self_join<D, BF16, RG>, true, dim3((unsigned)(rows < most ? rows : most)), 128, 0, st, a));
    return HDT_OK;
}
template <int D, bool BF16>
int step_rows(const StepArgs &a, cudaStream_t st) {
    return step_group(a.B, a.Tq) == 1 ? step_go<D, BF16, 1>(a, st) : step_go<D, BF16, STEP_ROWS>(a, st);
}

struct Prepared { SelfLists q, k; SelfDist dist; };
int prepare(const Layout &L, char *ws, const int32_t *cu_q, const int32_t *cu_k, const int32_t *len_k, int B, int Tq, int Tk, int H, int buckets, int max_distance,
            int causal, const void *table, int dtype, int bwd, cudaStream_t st, Prepared *out) {
    PrepArgs p{};
    p.cu_q = cu_q; p.cu_k = cu_k; p.len_k = len_k; p.B = B; p.Tq = Tq; p.Tk = Tk; p.H = H;
    p.n_lists = bwd ? 2 : 1;
    int *count = (int *)(ws + L.count);
    SelfBlk *raw = (SelfBlk *)(ws + L.raw);
    p.list[0] = PrepList{raw, (SelfBlk *)(ws + L.q), count, L.rows_q, 0, L.most_q};
    p.list[1] = PrepList{raw + L.most_q, (SelfBlk *)(ws + L.k), count + 1, dtype == HDT_F32 ? SELF_F32_ROWS : 128, 1, L.most_k};
    p.rel.causal = causal;
    p.dtype = dtype;
    *out = Prepared{};
    if (buckets > 0) {
        rel_fill(&p.rel, buckets, max_distance, causal);
        p.table = table;
        p.lo = causal ? 0 : -p.rel.far;
        p.n = p.rel.far - p.lo + 1;
        p.bias = (float *)(ws + L.bias);
        p.bucket = (unsigned char *)(ws + L.bucket);
        out->dist = SelfDist{p.bias, p.bucket, p.lo, p.rel.far, p.n};
    }
    out->q = SelfLists{p.list[0].out, count, L.most_q};
    out->k = SelfLists{p.list[1].out, count + 1, L.most_k};
    p.behind = bwd && Tq > 0;      // (delta's kernel, which is not a dependent itself)
    HDT_CUDA_CHECK(launch_dependent(k_self_prep, p.behind != 0, dim3((unsigned)(p.n_lists + (p.n + 1023) / 1024)), 1024, 0, st, p));
    return HDT_OK;
}

}  // namespace
}  // namespace hdt

using namespace hdt;

extern "C" size_t hdt_self_workspace_bytes(int32_t batch, int32_t total_q, int32_t total_k, int32_t heads, int32_t head_dim, int32_t num_buckets,
                                           int32_t max_distance, int32_t causal, int32_t dtype, int32_t bwd) {
    if (sizes_check(batch, total_q, total_k, heads, head_dim, num_buckets, max_distance, causal, dtype, "hdt_self_workspace_bytes")) return 0;
    return layout(batch, total_q, total_k, heads, head_dim, num_buckets, max_distance, causal ? 1 : 0, dtype, bwd).total;
}

extern "C" int hdt_self_bucket_borders(int32_t num_buckets, int32_t max_distance, int32_t causal, int32_t *first) {
    if (num_buckets < 1 || !first) return set_error(HDT_ERR_INVALID_ARG, "hdt_self_bucket_borders: no bucket or a null pointer");
    if (const int rc = sizes_check(0, 0, 0, 1, 64, num_buckets, max_distance, causal, HDT_F32, "hdt_self_bucket_borders")) return rc;
    SelfRel r;
    rel_fill(&r, num_buckets, max_distance, causal ? 1 : 0);
    for (int b = 0; b < r.one_way; ++b) first[b] = r.first[b];
    return HDT_OK;
}

extern "C" int hdt_self_attn_fwd(const int32_t *cu_seqlens_q, const int32_t *cu_seqlens_k, const int32_t *seqlens_k, int32_t batch, int32_t total_q,
                                 int32_t total_k, const void *q, const void *k, const void *v, const void *bias, int32_t num_buckets, int32_t max_distance,
                                 int32_t causal, void *o, float *lse, int32_t heads, int32_t head_dim, int32_t dtype, float softmax_scale, void *workspace,
                                 size_t workspace_bytes, void *stream) {
    const char *who = "hdt_self_attn_fwd";
    if (!bias) num_buckets = 0;
    causal = causal ? 1 : 0;
    if (const int rc = sizes_check(batch, total_q, total_k, heads, head_dim, num_buckets, max_distance, causal, dtype, who)) return rc;
    if (bias && num_buckets == 0) return set_error(HDT_ERR_INVALID_ARG, "%s: a bias without buckets", who);
    const Layout L = layout(batch, total_q, total_k, heads, head_dim, num_buckets, max_distance, causal, dtype, 0);
    if (const int rc = ws_check(workspace, workspace_bytes, L.total, who)) return rc;
    if (total_q == 0 || batch == 0) return HDT_OK;
    if (!cu_seqlens_q || !cu_seqlens_k) return set_error(HDT_ERR_INVALID_ARG, "%s: null structure pointer", who);
    if (total_k == 0) { if (!k) k = q; if (!v) v = q; }      // (never read)
    for (const void *p : {q, k, v, (const void *)o})
        if (const int rc = ptr_check(p, who)) return rc;
    if (!lse || ((uintptr_t)lse & 3) || ((uintptr_t)bias & (dtype == HDT_F32 ? 3 : 1))) return set_error(HDT_ERR_INVALID_ARG, "%s: null or misaligned tensor", who);
    const float scale = softmax_scale > 0.f ? softmax_scale : 1.0f / sqrtf((float)head_dim), LOG2E = 1.4426950408889634f;
    cudaStream_t st = (cudaStream_t)stream;
    char *ws = (char *)workspace;
    if (is_step(batch, total_q)) {
        StepArgs s{};
        s.cu_q = cu_seqlens_q; s.cu_k = cu_seqlens_k; s.len_k = seqlens_k; s.B = batch; s.Tq = total_q; s.Tk = total_k; s.H = heads;
        s.piece = step_piece(batch, total_k, heads, step_group(batch, total_q)); s.dtype = dtype;
        s.q = q; s.k = k; s.v = v; s.table = bias; s.o = o; s.lse = lse; s.part_o = (float *)(ws + L.part_o); s.part_ml = (float *)(ws + L.part_ml);
        s.scale_log2 = scale * LOG2E;
        s.before = batch > STEP_COUNTED ? (int *)(ws + L.before) : nullptr;
        s.rel.causal = causal;
        if (num_buckets > 0) rel_fill(&s.rel, num_buckets, max_distance, causal);
        if (head_dim == 64) return dtype == HDT_BF16 ? step_rows<64, true>(s, st) : step_rows<64, false>(s, st);
        return dtype == HDT_BF16 ? step_rows<128, true>(s, st) : step_rows<128, false>(s, st);
    }
    int *const status = device_status_ptr();
    if (!status) return HDT_ERR_CUDA;
    Prepared p;
    if (const int rc = prepare(L, ws, cu_seqlens_q, cu_seqlens_k, seqlens_k, batch, total_q, total_k, heads, num_buckets, max_distance, causal, bias, dtype, 0, st, &p)) return rc;
    SelfFwdArgs a{};
    a.q = p.q; a.block_rows = L.rows_q; a.dist = p.dist; a.H = heads; a.Tq = total_q; a.Tk = total_k; a.causal = causal; a.bias_on = num_buckets > 0;
    a.qp = q; a.kp = k; a.vp = v; a.o = o; a.lse = lse; a.scale_log2 = scale * LOG2E;
    a.status = status;
    return dtype == HDT_BF16 ? launch_self_fwd_tc(a, head_dim, st) : launch_self_fwd_f32(a, head_dim, st);
}

extern "C" int hdt_self_attn_bwd(const int32_t *cu_seqlens_q, const int32_t *cu_seqlens_k, const int32_t *seqlens_k, int32_t batch, int32_t total_q,
                                 int32_t total_k, const void *q, const void *k, const void *v, const void *bias, int32_t num_buckets, int32_t max_distance,
                                 int32_t causal, const void *o, const float *lse, const void *d_o, void *dq, void *dk, void *dv, void *d_bias, int32_t heads,
                                 int32_t head_dim, int32_t dtype, float softmax_scale, void *workspace, size_t workspace_bytes, void *stream) {
    const char *who = "hdt_self_attn_bwd";
    if (!bias) num_buckets = 0;
    causal = causal ? 1 : 0;
    if (const int rc = sizes_check(batch, total_q, total_k, heads, head_dim, num_buckets, max_distance, causal, dtype, who)) return rc;
    if (bias && (num_buckets == 0 || !d_bias)) return set_error(HDT_ERR_INVALID_ARG, "%s: a bias without buckets or without room for its gradient", who);
    const Layout L = layout(batch, total_q, total_k, heads, head_dim, num_buckets, max_distance, causal, dtype, 1);
    if (const int rc = ws_check(workspace, workspace_bytes, L.total, who)) return rc;
    const uintptr_t el = dtype == HDT_F32 ? 3 : 1;
    if (((uintptr_t)bias | (bias ? (uintptr_t)d_bias : 0)) & el) return set_error(HDT_ERR_INVALID_ARG, "%s: misaligned bias", who);
    cudaStream_t st = (cudaStream_t)stream;
    char *ws = (char *)workspace;
    const bool none = batch == 0 || (total_q == 0 && total_k == 0);
    Prepared p{};
    if (!none) {
        if (!cu_seqlens_q || !cu_seqlens_k) return set_error(HDT_ERR_INVALID_ARG, "%s: null structure pointer", who);
        if (total_k == 0) { if (!k) k = q; if (!v) v = q; if (!dk) dk = dq; if (!dv) dv = dq; }      // (never read or written)
        if (total_q == 0) { if (!q) q = k; if (!o) o = k; if (!d_o) d_o = k; if (!dq) dq = dk; if (!lse) lse = (const float *)k; }
        for (const void *x : {q, k, v, o, d_o, (const void *)dq, (const void *)dk, (const void *)dv})
            if (const int rc = ptr_check(x, who)) return rc;
        if (!lse || ((uintptr_t)lse & 3)) return set_error(HDT_ERR_INVALID_ARG, "%s: null or misaligned tensor", who);
        int *const status = device_status_ptr();
        if (!status) return HDT_ERR_CUDA;
        // (delta first: the preparation runs beside it)
        if (const int rc = launch_delta(o, d_o, (float *)(ws + L.delta), total_q, heads, head_dim, dtype, st)) return rc;
        if (const int rc = prepare(L, ws, cu_seqlens_q, cu_seqlens_k, seqlens_k, batch, total_q, total_k, heads, num_buckets, max_distance, causal, bias, dtype, 1, st, &p)) return rc;
        const float scale = softmax_scale > 0.f ? softmax_scale : 1.0f / sqrtf((float)head_dim);
        SelfBwdArgs a{};
        a.dist = p.dist; a.H = heads; a.Tq = total_q; a.Tk = total_k; a.causal = causal; a.bias_on = num_buckets > 0; a.buckets = num_buckets;
        a.qp = q; a.kp = k; a.vp = v; a.dop = d_o; a.lse = lse; a.delta = (float *)(ws + L.delta); a.dq = dq; a.dk = dk; a.dv = dv;
        a.scale = scale; a.scale_log2 = scale * 1.4426950408889634f; a.status = status;
        SelfBwdArgs keys = a, rows = a;
        keys.blk = p.k;
        rows.blk = p.q;
        (dtype == HDT_F32 ? rows : keys).part = num_buckets > 0 ? (float *)(ws + L.part) : nullptr;
        if (const int rc = dtype == HDT_BF16 ? launch_self_bwd_tc(keys, rows, head_dim, st) : launch_self_bwd_f32(keys, rows, head_dim, st)) return rc;
    }
    if (num_buckets > 0) {
        const bool any = !none && total_q > 0;
        HDT_CUDA_CHECK(launch_dependent(k_self_dbias, any, dim3((unsigned)heads), 1024, 0, st, any ? (const float *)(ws + L.part) : (const float *)nullptr,
                                        dtype == HDT_F32 ? p.q.count : p.k.count, heads,
                                        num_buckets, dtype, d_bias));
    }
    return HDT_OK;
}
