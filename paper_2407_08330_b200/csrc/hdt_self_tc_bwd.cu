// Self-attention with a relative position bias, backward in bf16 (TMA + tcgen05), head_dim 64 and 128: one kernel in
// two forms, each with a block of 128 rows of one side in the TMEM lanes, which walks the other side in tiles of 128:
//
//   rows (dQ), first   resident Q, dO; walked K, V:  S = Q K^T, dP = dO V^T;      dQ += dS K, W += P K
//   keys (dK, dV)      resident K, V; walked Q, dO:  S^T = K Q^T, dP^T = V dO^T;  dK += dS^T Q, dV += P^T dO
//   P = exp2(S scale' + bias' - LSE'),   dS = scale P o (dP - delta)
//
// Both forms compute S and dP (eight products of a tile pair in all, one walk would need five), and in exchange nothing is
// added up across CTAs: no fp32 buffer for dQ, no atomics, the same bits every run; and every operand that the tensor
// pipe reads is where TMA or the compute warps put it, P and dS in TMEM.  That also is what fits at head_dim 128,
// where two accumulators take half of TMEM.
//
// delta.  rowsum(dO o O) with the O that was rounded to bf16 is off by e = dO . (rounding of O), in every dS of the row by P e:
// in rows of few keys as much as all other roundings together.  But the exact dS of a row add up to 0, so the row
// sum of the computed ones, in fp32, IS -scale e.  The rows form takes it: dQ loses r W at the end (r the row sum, W = P K),
// and delta is put right for the keys form.
//
// A unit is (block, head).  One CTA of 768 threads per SM walks units, dearest first:
//   warps 0-7, 8-15   compute, 64 of a tile's columns each (a step): a warp has a TMEM lane quarter and 32 columns, a thread
//                     a lane; P from S, then dS from dP.  (Half the warps with 64 columns a thread: 2950 cycles a
//                     step, whose exponentials take 512: two warps to a scheduler do not hide each other's latencies.)
//   warps 16-19       bring the resident tiles from shared memory into TMEM (head_dim 64); drain the accumulators at a
//                     unit's end: bf16 rows through a staging tile and TMA stores
//   warp 20           requests the tiles (TMA); LSE and delta (keys) and the bias of the tile's distances
//   warp 21           issues the MMAs; warps 22 and 23 fill the warp group
// What bounds it is the tensor pipe's operand reads: a product of M = 128, N = 64, K = 16 takes about 75 cycles with both
// operands in shared memory and 40 with A in TMEM.  So at head_dim 64 the resident tiles lie in TMEM too.
// 4 x 4096 tokens, causal: 12 heads of 64 584 us with all launches (rows 235, keys 332), 16 heads of 128 1144.
// TMEM: S of either step 64 columns (P over it), dP 64 (dS over it), the accumulators 2 x 64 or 2 x 128, at head_dim 64 the
// resident tiles of two units, 2 x 32 each.  One buffer of each is enough: S of a step's next tile is computed, behind the product that reads P,
// while the compute warps are at dS, and dP, behind the one that reads dS, while they are at the next P.
//
// Rows that are not the document's (the walked tile's tail) are set to zero in shared memory: their P and dS are 0, but
// another document's rows, or unused ones, may hold NaN.
//
// The bias' gradient (keys form): the sum of dS over the pairs of a bucket.  In a tile whose distances are all beyond the
// last border a thread adds its dS up in a register.  Elsewhere the sums run along the diagonals of a warp's 32 x 32
// piece: column by column, each lane passes its sum to the next lane (one shuffle and one addition an entry),
// so that a sum always stays with its distance; then neighbouring distances of one bucket are joined by a segmented
// reduction.  All in fp32, from dS before its rounding, in an order that depends on nothing but the shapes.
#include "hdt_rows.cuh"
#include "hdt_self.cuh"
#include "hdt_sm100.cuh"
#include "hdt_tmap.cuh"

namespace hdt {
using namespace sm100;

namespace {
constexpr int SUB = 16384;                        // [128 rows x 64] bf16
constexpr long long WAIT_CYCLES = 400000000LL;
constexpr int KID = 10;                           // kernel id in the device status word
__device__ __forceinline__ uint32_t swz(int r, int c) { return (uint32_t)(r * 128 + ((c ^ (r & 7)) << 4)); }

__device__ __forceinline__ bool group_all(bool pred, int id, int n) {      // barrier over a warp group: did all of them pass `pred`?
    uint32_t r;
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t"
        "setp.ne.b32 p, %1, 0;\n\t"
        "bar.red.and.pred q, %2, %3, p;\n\t"
        "selp.u32 %0, 1, 0, q;\n\t}"
        : "=r"(r)
        : "r"((uint32_t)pred), "r"(id), "r"(n)
        : "memory");
    return r != 0;
}

template <int D, bool ROWS>
struct BwdShape {
    static constexpr int NS = D / 64, TILE = SUB * NS, ST = D == 64 ? 4 : 2;
    static constexpr bool RTM = D == 64;                      // the resident tiles are read from TMEM
    static constexpr uint32_t TM_S = 0, TM_P = 128, TM_ACC = 256, TM_R = 384;
    static constexpr int STAT = 128 * 8 + 256 * 4 + 256;      // -LSE', -delta' by column; bias' and bucket by distance
    static constexpr int SUMS = ROWS ? 4 * 128 * 4 : 16 * (SELF_MAX_BUCKETS + 32) * 4;
    static constexpr int SMEM = (2 + ST * 2) * TILE + SUB + ST * STAT + SUMS + 512;
};
}  // namespace

// P from S (in place, 32 columns of a lane's row), then dS from dP and P (in place, 16 columns at a time: with 32 the registers do not
// hold them, and a spilled word is a trip to L2: 1500 cycles more a step).  NEAR: a bias by distance (nr, step +-1 per
// column); MASK: only the columns of `keep`.
template <bool ROWS, bool NEAR, bool MASK>
__device__ __forceinline__ void probabilities(uint32_t *x, const float *neg_l, const float *nr, float row_l, float scale_log2, uint32_t keep) {
#pragma unroll
    for (int e = 0; e < 32; e += 4) {
        f2 l[2] = {pack2(row_l, row_l), pack2(row_l, row_l)};
        if constexpr (!ROWS) {
            const float4 z = *reinterpret_cast<const float4 *>(neg_l + e);
            l[0] = pack2(z.x, z.y);
            l[1] = pack2(z.z, z.w);
        }
#pragma unroll
        for (int f = 0; f < 4; f += 2) {
            const int k = e + f;
            f2 y = fma2(pack2(__uint_as_float(x[k]), __uint_as_float(x[k + 1])), pack2(scale_log2, scale_log2), l[f >> 1]);
            if constexpr (NEAR) y = add2(y, pack2(nr[ROWS ? -k : k], nr[ROWS ? -(k + 1) : k + 1]));
            float y0, y1;
            unpack2(y, y0, y1);
            y0 = exp2f(y0);
            y1 = exp2f(y1);
            if constexpr (MASK) {
                if (!(keep >> k & 1u)) y0 = 0.f;
                if (!(keep >> k & 2u)) y1 = 0.f;
            }
            x[k] = __float_as_uint(y0);
            x[k + 1] = __float_as_uint(y1);
        }
    }
}
template <bool ROWS, bool MASK>
__device__ __forceinline__ void gradients(uint32_t (&x)[16], const uint32_t *p, const float *neg_d, float row_d, float scale, uint32_t keep) {
#pragma unroll
    for (int e = 0; e < 16; e += 4) {
        f2 l[2] = {pack2(row_d, row_d), pack2(row_d, row_d)};
        if constexpr (!ROWS) {
            const float4 z = *reinterpret_cast<const float4 *>(neg_d + e);
            l[0] = pack2(z.x, z.y);
            l[1] = pack2(z.z, z.w);
        }
#pragma unroll
        for (int f = 0; f < 4; f += 2) {
            const int k = e + f;
            const f2 g = mul2(pack2(__uint_as_float(p[k]), __uint_as_float(p[k + 1])),
                              fma2(pack2(__uint_as_float(x[k]), __uint_as_float(x[k + 1])), pack2(scale, scale), l[f >> 1]));
            float y0, y1;
            unpack2(g, y0, y1);
            if constexpr (MASK) {      // (0 x NaN: a lane that is no row of the document may hold anything)
                if (!(keep >> k & 1u)) y0 = 0.f;
                if (!(keep >> k & 2u)) y1 = 0.f;
            }
            x[k] = __float_as_uint(y0);
            x[k + 1] = __float_as_uint(y1);
        }
    }
}

template <int D, bool ROWS>
__global__ void __launch_bounds__(768, 1) k_self_bwd(const __grid_constant__ CUtensorMap tm_r1, const __grid_constant__ CUtensorMap tm_r2,
                                                     const __grid_constant__ CUtensorMap tm_s1, const __grid_constant__ CUtensorMap tm_s2,
                                                     const __grid_constant__ StoreMaps sm_out, const SelfBwdArgs a) {
    using Sh = BwdShape<D, ROWS>;
    constexpr int NS = Sh::NS, TILE = Sh::TILE, ST = Sh::ST;
    constexpr uint32_t TM_S = Sh::TM_S, TM_P = Sh::TM_P, TM_ACC = Sh::TM_ACC, TM_R = Sh::TM_R, TM_COLS = 512;
    constexpr bool RTM = Sh::RTM;
    constexpr int W_DRAIN = 16, W_LOAD = 20, W_MMA = 21;
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    uint8_t *sR = smem_raw;                       // R1, R2: K, V or Q, dO
    uint8_t *sS = sR + 2 * TILE;                  // [ST] x {S1, S2}: Q, dO or K, V
    uint8_t *sStg = sS + ST * 2 * TILE;           // staging of 64 columns of a result
    uint8_t *sStat = sStg + SUB;                  // [ST] x STAT
    float *sSum = (float *)(sStat + ST * Sh::STAT);        // rows: [4][128] row sums of dS; keys: per compute warp [buckets] and [32] of scratch
    uint64_t *bars = (uint64_t *)((uint8_t *)sSum + Sh::SUMS);
    // resident tiles: loaded, free, in TMEM, read for the last time; walked tiles; S, dP; P, dS; accumulators; the rest
    uint64_t *r_full = bars, *r_empty = bars + 1, *r_ready = bars + 2, *r_free = bars + 4, *s_full = bars + 6, *dp_full = bars + 8, *p_ready = bars + 10, *ds_ready = bars + 12;
    uint64_t *acc_full = bars + 14, *acc_free = bars + 15, *fix = bars + 16, *sum_full = bars + 17, *sum_free = bars + 18;
    uint64_t *t_full = bars + 19, *t_empty = t_full + ST;
    uint32_t *slot = (uint32_t *)(t_empty + ST);
    volatile int *abort_flag = (volatile int *)(slot + 1);

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, H = a.H;
    const float LOG2E = 1.4426950408889634f;
    if ((smem_u32(smem_raw) & 1023u) != 0u) {
        if (tid == 0) atomicCAS(a.status, 0, HDT_ERR_CUDA);
        return;
    }
    if (tid == 0) {
        mbar_init(r_full, 1);
        mbar_init(r_empty, RTM ? 128 : 1);
        for (int i = 0; i < 2; ++i) {
            mbar_init(&r_ready[i], 128);
            mbar_init(&r_free[i], 1);
            mbar_init(&s_full[i], 1);
            mbar_init(&p_ready[i], 256);
            mbar_init(&dp_full[i], 1);
            mbar_init(&ds_ready[i], 256);
        }
        for (int i = 0; i < ST; ++i) {
            mbar_init(&t_full[i], 2);      // the tile's bytes; its statistics
            mbar_init(&t_empty[i], 1);
        }
        mbar_init(acc_full, 1);
        mbar_init(acc_free, 128);
        mbar_init(fix, 1);
        mbar_init(sum_full, 512);
        mbar_init(sum_free, 128);
        *abort_flag = (*a.status != 0);
        fence_mbar_init();
    }
    for (int i = tid; i < Sh::SUMS / 4; i += 768) sSum[i] = 0.f;
    if (warp == 0) tmem_alloc(slot, TM_COLS);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *slot;
    const uint32_t lane_base = (uint32_t)((warp & 3) * 32) << 16;
    const bool dead = (*abort_flag != 0);
    bool ok = true;
    int fail_site = 0;
    pdl_wait();
    pdl_launch_dependents();
    const int n_units = *a.blk.count * H;
    const bool sums = !ROWS && a.part != nullptr;

#define HDT_AGREE() (ok = __all_sync(0xffffffffu, ok))
#define HDT_WAIT(bar, parity, site)                                                   \
    do {                                                                              \
        if (ok && !mbar_wait((bar), (uint32_t)(parity), abort_flag, WAIT_CYCLES)) {   \
            ok = false;                                                               \
            fail_site = (site);                                                       \
        }                                                                             \
    } while (0)

    // What a unit walks: columns [c0, c1) of the other side (document numbers), in nt tiles.
    struct Unit { SelfBlk b; int h, c0, c1, nt; };
    auto unit = [&](int u) {
        Unit x;
        x.b = a.blk.blk[u / H];
        x.h = u % H;
        x.c0 = ROWS ? 0 : self_first_row(a.causal, x.b.r0, x.b.nq, x.b.nk);
        x.c1 = ROWS ? self_keys_of(a.causal, x.b.r0, 128, x.b.nq, x.b.nk) : x.b.nq;
        x.nt = (max(x.c1 - x.c0, 0) + 127) >> 7;
        return x;
    };
    // Distance of lane 0 and column 0 of tile j; it grows by 1 per row and falls by 1 per key.
    auto base_of = [&](const Unit &x, int j) { return ROWS ? x.b.off + x.b.r0 - 128 * j : x.b.off + x.c0 + 128 * j - x.b.r0; };
    // -1, 1: all distances of the tile lie beyond the last border behind / before the query; 0: they do not
    auto far_side = [&](int base) { return !a.bias_on ? 2 : base - 127 >= a.dist.far ? 1 : base + 127 <= -a.dist.far ? -1 : 0; };

    // 80 registers a thread at launch (768 threads): the compute warps take what the others do not need
    // (512 x 88 + 256 x 64 = 768 x 80)
    if (warp < W_DRAIN) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 88;");
        if (!dead) {
            // ================= compute: columns c0 .. c0 + 31 of every tile =================
            const int x = warp >> 3, qh = (warp >> 2) & 1, rl = (warp & 3) * 32 + lane, c0 = 64 * x + 32 * qh;
            float *sum = sSum + warp * (SELF_MAX_BUCKETS + 32), *scratch = sum + SELF_MAX_BUCKETS;      // (keys)
            const uint32_t tm_s = tmem + TM_S + 64u * x + 32u * qh + lane_base, tm_dp = tmem + TM_P + 64u * x + 32u * qh + lane_base;
            int st = 0, uc = 0, par = 0;
            auto flush = [&](float v, int at) {      // a warp's sum beyond the borders, to the bucket of distance number `at`
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
                if (lane == 0) sum[a.dist.bucket[at]] += v;
                __syncwarp();
            };
            for (int k = 0, u; ok && (u = self_unit(k, blockIdx.x, gridDim.x)) < n_units; ++k) {
                // (what a unit needs in its loop, and no more: p and d fill the registers)
                int nt, first, end;            // tiles; columns that this lane's row pairs with, from c0 on
                int whole0, whole1;            // tiles in which every lane of the warp keeps all its columns
                int near0 = 0, near1 = 0;      // tiles with distances inside the borders; those before and behind lie beyond them
                float row_l = 0.f, row_d = 0.f, by_side[2];      // rows: -LSE' and -delta'; -LSE' with the bias of the tiles before and behind the near ones
                {
                    const Unit U = unit(u);
                    if (U.nt == 0) continue;
                    nt = U.nt;
                    const int base = base_of(U, 0);
                    if (a.bias_on) {
                        near0 = max(((ROWS ? base - 127 - a.dist.far : -a.dist.far - 127 - base) >> 7) + 1, 0);
                        near1 = max(((ROWS ? base + 127 + a.dist.far : a.dist.far + 127 - base) + 127) >> 7, near0);
                    }
                    const int row = U.b.r0 + rl;
                    first = end = 0;
                    if (row < (ROWS ? U.b.nq : U.b.nk)) {
                        if (ROWS) {
                            const size_t r = (size_t)U.h * a.Tq + U.b.q0 + row;
                            const float L = a.lse[r];
                            row_l = L == -INFINITY ? -INFINITY : -L * LOG2E;
                            row_d = -a.delta[r] * a.scale;
                            end = a.causal ? min(max(U.b.off + row + 1, 0), U.b.nk) : U.b.nk;
                        } else {
                            first = self_first_row(a.causal, row, U.b.nq, U.b.nk);
                            end = U.b.nq;
                        }
                    }
                    first -= U.c0 + c0;
                    end -= U.c0 + c0;
                    whole0 = (max(__reduce_max_sync(0xffffffffu, first), 0) + 127) >> 7;
                    whole1 = (__reduce_min_sync(0xffffffffu, end) - 32 + 128) >> 7;
                    by_side[0] = by_side[1] = row_l;
                    if (ROWS && a.bias_on) {      // (keys behind the query come last)
                        by_side[0] += a.dist.bias[(size_t)(U.h + 1) * a.dist.n - 1];
                        by_side[1] += a.dist.bias[(size_t)U.h * a.dist.n];
                    }
                }
                float far_sum = 0.f;
                f2 row_sum = pack2(0.f, 0.f);
                for (int j = 0; j < nt; ++j) {
                    const bool near = j >= near0 && j < near1;
                    if (sums && j == near0 && j > 0) {      // what was summed so far lies behind the query, what comes after the near tiles before it
                        flush(far_sum, 0);
                        far_sum = 0.f;
                    }
                    const uint8_t *stat = sStat + st * Sh::STAT;
                    uint32_t keep = 0xffffffffu;
                    const bool all = j >= whole0 && j < whole1;
                    bool any = true;
                    if (!all) {
                        const int jl = max(first, 0), jh = min(end, 32);
                        keep = jh <= jl ? 0u : (jh >= 32 ? 0xffffffffu : (1u << jh) - 1u) & ~((1u << jl) - 1u);
                        any = __any_sync(0xffffffffu, keep != 0u);
                    }
                    first -= 128;
                    end -= 128;
                    const float l = !ROWS || near ? row_l : by_side[j >= near1];
                    if (j == 0 && uc > 0) HDT_WAIT(sum_free, (uc - 1) & 1, 18);      // the drain group has read the last unit's sums
                    HDT_WAIT(&s_full[x], par, 12);      // (a wait that ran out changes nothing in what the warp does before the tile's end)
                    tc_fence_after();
                    uint32_t p[32], d2[2][16];
                    if (any) {
                        tmem_ld32(tm_s, p);
                        tmem_wait_ld();
                        const float *neg_l = reinterpret_cast<const float *>(stat) + c0;
                        // entry (row, column) of a tile with near distances: + 1 per row, - 1 per key
                        const float *n = reinterpret_cast<const float *>(stat + 1024) + 127 + (ROWS ? rl - c0 : c0 - rl);
                        if (near) {
                            if (all) probabilities<ROWS, true, false>(p, neg_l, n, l, a.scale_log2, keep);
                            else probabilities<ROWS, true, true>(p, neg_l, n, l, a.scale_log2, keep);
                        } else if (all) probabilities<ROWS, false, false>(p, neg_l, n, l, a.scale_log2, keep);
                        else probabilities<ROWS, false, true>(p, neg_l, n, l, a.scale_log2, keep);
                    } else {
#pragma unroll
                        for (int e = 0; e < 32; ++e) p[e] = 0u;
                    }
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        uint32_t y[8];
#pragma unroll
                        for (int e = 0; e < 8; ++e) y[e] = pack_bf16(__uint_as_float(p[16 * i + 2 * e]), __uint_as_float(p[16 * i + 2 * e + 1]));
                        tmem_st8(tm_s + 8u * i, y);      // (inside the columns that this warp alone reads)
                    }
                    tmem_wait_st();
                    tc_fence_before();
                    mbar_arrive(&p_ready[x]);
                    HDT_WAIT(&dp_full[x], par, 15);
                    tc_fence_after();
                    float diag = 0.f;
                    if (any && !ROWS) tmem_ld16(tm_dp, d2[0]);      // (rows: no room for a second load in flight)
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        uint32_t (&d)[16] = d2[i], y[8];
                        if (any) {
                            if (ROWS) tmem_ld16(tm_dp + 16u * i, d);
                            tmem_wait_ld();
                            if (!ROWS && i == 0) tmem_ld16(tm_dp + 16u, d2[1]);
                            const float *neg_d = reinterpret_cast<const float *>(stat) + 128 + c0 + 16 * i;
                            if (all) gradients<ROWS, false>(d, p + 16 * i, neg_d, row_d, a.scale, 0u);
                            else gradients<ROWS, true>(d, p + 16 * i, neg_d, row_d, a.scale, keep >> (16 * i));
                        } else {
#pragma unroll
                            for (int e = 0; e < 16; ++e) d[e] = 0u;
                        }
#pragma unroll
                        for (int e = 0; e < 8; ++e) y[e] = pack_bf16(__uint_as_float(d[2 * e]), __uint_as_float(d[2 * e + 1]));
                        tmem_st8(tm_dp + 8u * i, y);
                        if (ROWS || (sums && !near)) {
                            f2 v = pack2(0.f, 0.f);
#pragma unroll
                            for (int e = 0; e < 16; e += 2) v = add2(v, pack2(__uint_as_float(d[e]), __uint_as_float(d[e + 1])));
                            if (ROWS) row_sum = add2(row_sum, v);
                            else {
                                float v0, v1;
                                unpack2(v, v0, v1);
                                far_sum += v0 + v1;
                            }
                        } else if (sums && any) {
#pragma unroll
                            for (int e = 0; e < 16; ++e) {
                                // the sums move on by a lane; the last lane's is complete: distance k - 32 from lane 0 and column 0
                                const int k = 16 * i + e;
                                if (k > 0) {
                                    diag = __shfl_sync(0xffffffffu, diag, (lane + 31) & 31);
                                    if (lane == 0) {
                                        scratch[k] = diag;
                                        diag = 0.f;
                                    }
                                }
                                diag += __uint_as_float(d[e]);
                            }
                        }
                    }
                    // distances 31 - lane (this lane's sum) and lane - 32 (in scratch, lanes 1..31) from the piece's corner: their buckets,
                    // before the arrival that lets the load warp use the stage again
                    int bks[2] = {255, 255};
                    if (sums && near && any) {
                        const uint8_t *at = stat + 2048 + 127 + c0 - (warp & 3) * 32;
                        bks[0] = at[31 - lane];
                        if (lane > 0) bks[1] = at[lane - 32];
                    }
                    tmem_wait_st();
                    tc_fence_before();
                    mbar_arrive(&ds_ready[x]);
                    if (++st == ST) st = 0;
                    par ^= 1;
                    if (!HDT_AGREE()) break;
                    if (!(sums && near && any)) continue;
                    __syncwarp();
#pragma unroll
                    for (int g = 0; g < 2; ++g) {
                        const bool have = g == 0 || lane > 0;
                        float y = g == 0 ? diag : have ? scratch[lane] : 0.f;
                        const int bk = bks[g];
#pragma unroll
                        for (int o = 1; o < 32; o <<= 1) {      // sum of the lanes of one bucket from here on
                            const float y1 = __shfl_down_sync(0xffffffffu, y, o);
                            const int z = __shfl_down_sync(0xffffffffu, bk, o);
                            if (lane + o < 32 && z == bk) y += y1;
                        }
                        const int before = __shfl_up_sync(0xffffffffu, bk, 1);
                        if (have && (lane == 0 || before != bk)) sum[bk] += y;
                        __syncwarp();
                    }
                }
                if (!ok) break;
                if (ROWS) {
                    float v0, v1;
                    unpack2(row_sum, v0, v1);
                    sSum[(2 * x + qh) * 128 + rl] = v0 + v1;
                } else if (sums) flush(far_sum, nt > near0 ? a.dist.n - 1 : 0);
                mbar_arrive(sum_full);
                ++uc;
            }
        }
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
        if (dead) {
        } else if (warp == W_LOAD) {
            // ================= load warp =================
            int t = 0, uc = 0, nfix = 0;
            for (int k = 0, u; ok && (u = self_unit(k, blockIdx.x, gridDim.x)) < n_units; ++k) {
                const Unit x = unit(u);
                if (x.nt == 0) continue;
                if (uc > 0) HDT_WAIT(r_empty, (uc - 1) & 1, 1);
                if (!HDT_AGREE()) break;
                if (lane == 0) {
                    const int row = (ROWS ? x.b.q0 : x.b.k0) + x.b.r0;
                    mbar_expect_tx(r_full, 2u * TILE);
#pragma unroll
                    for (int s = 0; s < NS; ++s) {
                        tma_load_3d(sR + s * SUB, &tm_r1, 64 * s, x.h, row, r_full);
                        tma_load_3d(sR + TILE + s * SUB, &tm_r2, 64 * s, x.h, row, r_full);
                    }
                }
                ++uc;
                const float *bias = a.dist.bias + (size_t)x.h * a.dist.n;
                for (int j = 0; j < x.nt && ok; ++j, ++t) {
                    const int s = t % ST, round = t / ST, col = x.c0 + 128 * j, rows = x.c1 - col, base = base_of(x, j), side = far_side(base);
                    // requested before the wait for the ring stage, all at once, and not looked at before the tile is
                    float L[4], dl[4], c = 0.f, nb[8];
                    unsigned char bk[8];
                    if (!ROWS) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const size_t r = (size_t)x.h * a.Tq + x.b.q0 + col + min(lane + 32 * i, rows - 1);
                            L[i] = a.lse[r];
                            dl[i] = a.delta[r];
                        }
                        if (side == 1 || side == -1) c = bias[side == 1 ? a.dist.n - 1 : 0];
                    }
                    if (side == 0) {
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            const int at = self_dist_at(a.dist, base + lane + 32 * i - 127);
                            nb[i] = bias[at];
                            bk[i] = sums ? a.dist.bucket[at] : 0;
                        }
                    }
                    if (round > 0) HDT_WAIT(&t_empty[s], (round - 1) & 1, 2);
                    if (!HDT_AGREE()) break;
                    uint8_t *d = sS + s * 2 * TILE;
                    uint64_t *bar = rows >= 128 ? &t_full[s] : fix;
                    if (lane == 0) {
                        const int row = (ROWS ? x.b.k0 : x.b.q0) + col;
                        mbar_expect_tx(bar, 2u * TILE);
#pragma unroll
                        for (int c = 0; c < NS; ++c) {
                            tma_load_3d(d + c * SUB, &tm_s1, 64 * c, x.h, row, bar);
                            tma_load_3d(d + TILE + c * SUB, &tm_s2, 64 * c, x.h, row, bar);
                        }
                    }
                    uint8_t *stat = sStat + s * Sh::STAT;
                    if (!ROWS)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            // (a row without keys: every exponential is 0; one number for the tile's bias goes into the LSE; columns
                            // behind the last are masked, but must be finite)
                            const bool in = lane + 32 * i < rows;
                            reinterpret_cast<float *>(stat)[lane + 32 * i] = !in ? 0.f : L[i] == -INFINITY ? -INFINITY : c - L[i] * LOG2E;
                            reinterpret_cast<float *>(stat)[128 + lane + 32 * i] = in ? -dl[i] * a.scale : 0.f;
                        }
                    if (side == 0)
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            reinterpret_cast<float *>(stat + 1024)[lane + 32 * i] = nb[i];
                            stat[2048 + lane + 32 * i] = bk[i];
                        }
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&t_full[s]);
                    if (rows < 128) {
                        HDT_WAIT(fix, nfix & 1, 3);
                        ++nfix;
                        if (!HDT_AGREE()) break;
                        for (int i = lane; i < (128 - rows) * 8; i += 32)
#pragma unroll
                            for (int c = 0; c < 2 * NS; ++c) *reinterpret_cast<uint4 *>(d + c * SUB + rows * 128 + i * 16) = make_uint4(0, 0, 0, 0);
                        fence_proxy_async_smem();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(&t_full[s]);
                    }
                }
            }
        } else if (warp == W_MMA) {
            // ================= MMA warp =================
            const uint32_t id_s = idesc_bf16(64, false, false), id_a = idesc_bf16(D, false, true), leader = elect_one() ? 1u : 0u;
            const uint64_t d_r = smem_desc(smem_u32(sR), 0, 1024), d_sk = smem_desc(smem_u32(sS), 0, 1024), d_sm = smem_desc(smem_u32(sS), SUB, 1024);
            const uint32_t r_hi = (uint32_t)(d_r >> 32), sk_hi = (uint32_t)(d_sk >> 32), sm_hi = (uint32_t)(d_sm >> 32);
            constexpr uint32_t T16 = TILE >> 4, S16 = SUB >> 4;
            // (TMEM is allocated whole, its addresses begin at 0)
            auto issue_sdp = [&](uint32_t q, uint32_t dst, uint32_t x, uint32_t s, uint32_t rb) {      // S (q = 0) or dP (1) of columns 64 x ..
                const uint32_t r_lo = (uint32_t)d_r + q * T16, s_lo = (uint32_t)d_sk + (s * 2u + q) * T16 + x * (8192u >> 4);
#pragma unroll
                for (uint32_t kk = 0; kk < D / 16; ++kk) {
                    const uint32_t o = (kk >> 2) * S16 + 2u * (kk & 3u);
                    if (RTM) mma_ts_p(leader, dst, TM_R + 64u * rb + 32u * q + 8u * kk, s_lo + o, sk_hi, id_s, kk > 0);
                    else mma_ss_p(leader, dst, r_lo + o, r_hi, s_lo + o, sk_hi, id_s, kk > 0);
                }
            };
            auto issue_acc = [&](uint32_t acc_at, uint32_t src, uint32_t q, uint32_t x, uint32_t s, uint32_t acc) {      // (columns 0..31 of P or dS in 16 of TMEM, 32..63 from 32 on)
                const uint32_t b_lo = (uint32_t)d_sm + (s * 2u + q) * T16 + x * (8192u >> 4);
#pragma unroll
                for (uint32_t kk = 0; kk < 4; ++kk) mma_ts_p(leader, acc_at, src + (kk < 2 ? 8u * kk : 32u + 8u * (kk - 2)), b_lo + 128u * kk, sm_hi, id_a, acc | (kk > 0));
            };
            // Tile by tile: this one's products with P and dS, and between them S and dP of the tiles behind it.  What this warp
            // keeps is counted: every instruction of it is on the critical chain.
            int k_next = 0;
            auto next_nt = [&]() {      // tiles of the next unit that has any, 0 behind the last
                for (int u; (u = self_unit(k_next, blockIdx.x, gridDim.x)) < n_units;) {
                    ++k_next;
                    const int n = __shfl_sync(0xffffffffu, unit(u).nt, 0);
                    if (n > 0) return n;
                }
                return 0;
            };
            auto wait = [&](uint64_t *bar, uint32_t parity, int site) {      // (the whole warp knows whether it ended well)
                HDT_WAIT(bar, parity, site);
                return HDT_AGREE();
            };
            int nt = next_nt(), nt_n = nt > 0 ? next_nt() : 0, j = 0;
            uint32_t uc = 0, st = 0, tp = 0, par = 0;      // unit; ring stage of this tile and parity of its use; parity of the tile number
            // rb: which of the two units in TMEM (head_dim 64)
            auto put_s = [&](uint32_t x, uint32_t s_, uint32_t rb) {
                issue_sdp(0, TM_S + 64u * x, x, s_, rb);
                mma_commit_p(leader, &s_full[x]);
            };
            auto put_dp = [&](uint32_t x, uint32_t s_, uint32_t rb, bool last_of_unit) {
                issue_sdp(1, TM_P + 64u * x, x, s_, rb);
                mma_commit_p(leader, &dp_full[x]);
                if (x == 1 && last_of_unit) mma_commit_p(leader, RTM ? &r_free[rb] : r_empty);      // the last that reads the resident tiles
            };
            auto resident = [&](uint32_t unit_no) {      // the unit's resident tiles are there
                return RTM ? wait(&r_ready[unit_no & 1u], (unit_no >> 1) & 1u, 4) : wait(r_full, unit_no & 1u, 4);
            };
            bool go = nt > 0 && resident(0) && wait(&t_full[0], 0, 5);
            if (go) {
                tc_fence_after();
                put_s(0, 0, 0);
                put_s(1, 0, 0);
                put_dp(0, 0, 0, false);
                put_dp(1, 0, 0, nt == 1);
            }
            while (go && nt > 0) {
                const bool last = j + 1 == nt, opens = last && nt_n > 0, more = !last || opens;      // the next tile: opens a unit, is there
                const bool last1 = last ? nt_n == 1 : j + 2 == nt;                                      // is its unit's last
                // resident tiles in shared memory, one buffer: the next unit's come when this unit's last S and dP are through
                const bool defer = !RTM && opens;
                const uint32_t s1 = st + 1 == ST ? 0 : st + 1, tp1 = st + 1 == ST ? tp ^ 1u : tp, acc = j == 0 ? 0u : 1u, rb1 = (uc + (last ? 1u : 0u)) & 1u;
#pragma unroll
                for (uint32_t x = 0; x < 2; ++x) {
                    go = wait(&p_ready[x], par, 7);
                    if (go && x == 0 && j == 0 && uc > 0) go = wait(acc_free, (uc - 1) & 1u, 6);
                    if (!go) break;
                    tc_fence_after();
                    issue_acc(TM_ACC + D, TM_S + 64u * x, ROWS ? 0 : 1, x, st, x == 0 ? acc : 1u);
                    if (more && !defer) {
                        if (x == 0) {
                            go = (!opens || resident(uc + 1)) && wait(&t_full[s1], tp1, 5);
                            if (!go) break;
                            tc_fence_after();
                        }
                        put_s(x, s1, rb1);
                    }
                    go = wait(&ds_ready[x], par, 8);
                    if (!go) break;
                    tc_fence_after();
                    issue_acc(TM_ACC, TM_P + 64u * x, 0, x, st, x == 0 ? acc : 1u);
                    if (x == 1) mma_commit_p(leader, &t_empty[st]);
                    if (more && !defer) put_dp(x, s1, rb1, last1);
                }
                if (!go) break;
                if (last) {
                    mma_commit_p(leader, acc_full);
                    if (defer) {
                        go = resident(uc + 1) && wait(&t_full[s1], tp1, 5);
                        if (!go) break;
                        tc_fence_after();
                        put_s(0, s1, 0);
                        put_s(1, s1, 0);
                        put_dp(0, s1, 0, false);
                        put_dp(1, s1, 0, last1);
                    }
                    nt = nt_n;
                    nt_n = nt > 0 ? next_nt() : 0;
                    j = 0;
                    ++uc;
                } else ++j;
                st = s1;
                tp = tp1;
                par ^= 1u;
            }
        } else if (warp < W_LOAD) {
            // ================= drain group =================
            const int rl = tid & 127;
            int uc = 0, um = 0, k_move = 0;
            // the resident tiles of the next unit that has any: from shared memory into TMEM, once the last products with those
            // of two units before are through
            auto move_next = [&]() {
                if (!RTM) return;
                int u;
                while ((u = self_unit(k_move, blockIdx.x, gridDim.x)) < n_units && unit(u).nt == 0) ++k_move;
                if (u >= n_units) return;
                ++k_move;
                HDT_WAIT(r_full, um & 1, 16);
                if (um > 1) HDT_WAIT(&r_free[um & 1], ((um >> 1) - 1) & 1, 17);
                if (!HDT_AGREE()) return;
                tc_fence_after();
#pragma unroll
                for (int q = 0; q < 4; ++q) {      // 32 columns of R1 or R2 at a time
                    uint32_t y[16];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const uint4 z = *reinterpret_cast<const uint4 *>(sR + (q >> 1) * TILE + swz(rl, 4 * (q & 1) + e));
                        y[4 * e] = z.x; y[4 * e + 1] = z.y; y[4 * e + 2] = z.z; y[4 * e + 3] = z.w;
                    }
                    tmem_st16(tmem + TM_R + 64u * (um & 1) + 16u * q + lane_base, y);
                }
                tmem_wait_st();
                tc_fence_before();
                mbar_arrive(r_empty);
                mbar_arrive(&r_ready[um & 1]);
                ++um;
            };
            move_next();
            move_next();
            for (int k = 0, u; (u = self_unit(k, blockIdx.x, gridDim.x)) < n_units; ++k) {
                const Unit U = unit(u);
                const int nrows = min(128, (ROWS ? U.b.nq : U.b.nk) - U.b.r0);
                float r = 0.f;
                if (U.nt > 0) HDT_WAIT(sum_full, uc & 1, 13);
                if (HDT_AGREE()) {
                    if (ROWS && U.nt > 0) {
#pragma unroll
                        for (int w = 0; w < 4; ++w) r += sSum[w * 128 + rl];
                        if (rl < nrows) a.delta[(size_t)U.h * a.Tq + U.b.q0 + U.b.r0 + rl] += r / a.scale;
                    } else if (sums && rl < a.buckets) {
                        float v = 0.f;
                        if (U.nt > 0)
#pragma unroll
                            for (int w = 0; w < 16; ++w) {
                                float *p = sSum + w * (SELF_MAX_BUCKETS + 32) + rl;
                                v += *p;
                                *p = 0.f;
                            }
                        a.part[((size_t)U.b.id * H + U.h) * a.buckets + rl] = v / a.scale;
                    }
                    if (U.nt > 0) mbar_arrive(sum_free);
                }
                const int bx = max(__clz(nrows) - 25, 0), bbox = 64 >> bx;
                if (U.nt > 0) {
                    HDT_WAIT(acc_full, uc & 1, 14);
                    ++uc;
                }
                bool go = group_all(ok, 1, 128);
                if (!go) break;
                tc_fence_after();
#pragma unroll 1
                for (int c = 0; c < (ROWS ? 1 : 2) * NS; ++c) {      // 64 columns of a result at a time
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        uint32_t y[16], w[16];
                        if (U.nt > 0) {
                            tmem_ld16(tmem + TM_ACC + 64u * c + lane_base + 16u * q, y);
                            if (ROWS) tmem_ld16(tmem + TM_ACC + D + 64u * c + lane_base + 16u * q, w);
                            tmem_wait_ld();
                            if (ROWS)
#pragma unroll
                                for (int e = 0; e < 16; ++e) y[e] = __float_as_uint(fmaf(-r, __uint_as_float(w[e]), __uint_as_float(y[e])));
                        } else {
#pragma unroll
                            for (int e = 0; e < 16; ++e) y[e] = 0u;
                        }
                        if (c == (ROWS ? 1 : 2) * NS - 1 && q == 3 && U.nt > 0) {      // the accumulators have been read
                            tc_fence_before();
                            mbar_arrive(acc_free);
                        }
#pragma unroll
                        for (int e = 0; e < 16; e += 8)
                            *reinterpret_cast<uint4 *>(sStg + swz(rl, (16 * q + e) >> 3)) =
                                make_uint4(pack_bf16(__uint_as_float(y[e]), __uint_as_float(y[e + 1])), pack_bf16(__uint_as_float(y[e + 2]), __uint_as_float(y[e + 3])),
                                           pack_bf16(__uint_as_float(y[e + 4]), __uint_as_float(y[e + 5])), pack_bf16(__uint_as_float(y[e + 6]), __uint_as_float(y[e + 7])));
                    }
                    fence_proxy_async_smem();
                    group_all(true, 1, 128);
                    // rows [0, nrows) as at most two boxes of b rows, b the largest power of two <= min(nrows, 64); where they
                    // overlap the same values are written twice
                    if (rl == 0) {
                        const int which = ROWS ? 0 : 1 + c / NS, at = (ROWS ? U.b.q0 : U.b.k0) + U.b.r0;
                        tma_store_3d(&sm_out.m[which][bx], 64 * (c % NS), U.h, at, sStg);
                        if (nrows > bbox) tma_store_3d(&sm_out.m[which][bx], 64 * (c % NS), U.h, at + nrows - bbox, sStg + (nrows - bbox) * 128);
                        bulk_commit();
                        bulk_wait_read();
                    }
                    group_all(true, 1, 128);      // (the staging tile has been read)
                }
                if (U.nt > 0) move_next();      // (the unit after the next, where this one's was)
            }
            if (rl == 0) bulk_wait_all();
        }
    }
    if (!ok) {
        if (atomicCAS(a.status, 0, HDT_ERR_TIMEOUT) == 0) {
            a.status[1] = (KID << 8) | fail_site;
            a.status[2] = (int)blockIdx.x;
        }
    }
#undef HDT_WAIT
#undef HDT_AGREE
    tc_fence_before();
    __syncthreads();
    if (warp == 0) tmem_dealloc(tmem, TM_COLS);
}

template <int D, bool ROWS>
static int go(const SelfBwdArgs &a, cudaStream_t st) {
    static DevOnce attr;
    using Sh = BwdShape<D, ROWS>;
    if (!attr.done()) {
        HDT_CUDA_CHECK(cudaFuncSetAttribute(k_self_bwd<D, ROWS>, cudaFuncAttributeMaxDynamicSharedMemorySize, Sh::SMEM));
        attr.set();
    }
    int n_sm = 0;
    if (const int rc = sm_count(&n_sm)) return rc;
    CUtensorMap tq, tk, tv, tdo;
    if (const int rc = make_tmap_bf16(&tq, a.qp, D, a.H, a.Tq, 128)) return rc;
    if (const int rc = make_tmap_bf16(&tk, a.kp, D, a.H, a.Tk, 128)) return rc;
    if (const int rc = make_tmap_bf16(&tv, a.vp, D, a.H, a.Tk, 128)) return rc;
    if (const int rc = make_tmap_bf16(&tdo, a.dop, D, a.H, a.Tq, 128)) return rc;
    StoreMaps outs;
    void *const dst[3] = {a.dq, a.dk, a.dv};
    for (int i = 0; i < 3; ++i) {
        if (ROWS != (i == 0)) continue;
        for (int b = 0; b < 7; ++b)
            if (const int rc = make_tmap_bf16(&outs.m[i][b], dst[i], D, a.H, i == 0 ? a.Tq : a.Tk, 64 >> b)) return rc;
    }
    const long long units = (long long)a.blk.most * a.H;
    const dim3 grid((unsigned)(units < n_sm ? units : n_sm));
    if (ROWS) HDT_CUDA_CHECK(launch_dependent(k_self_bwd<D, ROWS>, true, grid, 768, Sh::SMEM, st, tq, tdo, tk, tv, outs, a));
    else HDT_CUDA_CHECK(launch_dependent(k_self_bwd<D, ROWS>, true, grid, 768, Sh::SMEM, st, tk, tv, tq, tdo, outs, a));
    return HDT_OK;
}
int launch_self_bwd_tc(const SelfBwdArgs &keys, const SelfBwdArgs &rows, int head_dim, cudaStream_t st) {
    if (rows.Tq > 0)
        if (const int rc = head_dim == 64 ? go<64, true>(rows, st) : go<128, true>(rows, st)) return rc;
    if (keys.Tk > 0)
        if (const int rc = head_dim == 64 ? go<64, false>(keys, st) : go<128, false>(keys, st)) return rc;
    return HDT_OK;
}

}  // namespace hdt
