// Self-attention with a relative position bias, forward in bf16 (TMA + tcgen05), head_dim 64 and 128.
//
// A unit is (256 query rows of a document, head): two tiles of 128 rows that share every K and V tile.  One CTA of 384
// threads per SM walks units, dearest first:
//   warps 0-3, 4-7   softmax of one row tile each, a thread per row: S (128 keys) from TMEM into registers, bias, mask,
//                    running maximum, P (bf16) back over the S columns, O rescaled where the maximum grew
//   warp 8           requests Q per unit, K and V per key tile (TMA, rings of their own barriers)
//   warp 9           issues S = Q K^T and O += P V (A operand from TMEM); warps 10 and 11 fill the warp group
// While one tile's softmax runs, the tensor pipe works for the other.  TMEM: S0 0..127, S1 128..255, O0 256.., O1 256 + D..
//
// Scaling, bias and maximum in base 2: p = exp2(s scale' + (bias' - m)), one fma and one exponential where the tile's
// bias is one number, which it is beyond the distance where the buckets end; else the row's entries of the vector
// bias'[r - c] are added first (neighbouring lanes read neighbouring words of it).  The maximum that p refers to moves only when
// a tile's exceeds it by more than 8 (a factor of 256 that fp32 sums and bf16 P both have room for), so O is rescaled on few
// tiles.  P is rounded to bf16 for the product (8 significant bits, relative, as V has); the row sum adds it unrounded.
//
// At head_dim 64 a pair of tiles needs 1024 cycles of products, 2048 of exponentials, and takes 3660 (1 x 16384 tokens, 12 heads, both
// ways 1237 us, 667 TFLOP/s; causal 4 x 4096 182 us, 567 of unmasked pairs, and with 16 heads of 128 278 us, 989).  No unit is full there:
// exponentials 67 % of the time on the SMs with the most units (768 units on 148 SMs: six at most, 5.2 on average), tensor pipe 34 %
// and issue slots 38 % of active cycles.  What takes the time is a tile's chain (S, maximum, exponentials, P stored and fenced as a
// whole, product), which two row tiles cover in part; an SM's TMEM has no room for a third.
//
// The rows of V behind a document's last key are set to zero in shared memory: P is 0 there, but another document's rows,
// or a cache's unused ones, may hold NaN.
#include "hdt_rows.cuh"
#include "hdt_self.cuh"
#include "hdt_sm100.cuh"
#include "hdt_tmap.cuh"

namespace hdt {
using namespace sm100;

namespace {
constexpr int SUB = 16384;                        // [128 rows x 64] bf16
constexpr long long WAIT_CYCLES = 400000000LL;
constexpr int KID = 9;                            // kernel id in the device status word

template <int D>
struct FwdShape {
    static constexpr int ST = D == 64 ? 3 : 2, TILE = SUB * (D / 64), NS = D / 64;
    static constexpr int SMEM = (2 + 2 * ST) * TILE + 4 * 256 * 4 + 256;
    // At head_dim 128 the bias vector of the next near tile is requested a tile ahead, and the softmax warps have the registers for
    // it (4 x 4096 tokens 309 -> 295 us, borders up to 2000 340 -> 318).  At 64, where the two row tiles' exponentials
    // have to take turns, the same slows far tiles (1 x 16384 both ways 1237 -> 1308 us, 16 x 512 36.5 -> 34.2).
    static constexpr bool NEAR_AHEAD = D == 128;
};
}  // namespace

template <int D>
__global__ void __launch_bounds__(384, 1) k_self_fwd(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k,
                                                     const __grid_constant__ CUtensorMap tm_v, const SelfFwdArgs a) {
    using Sh = FwdShape<D>;
    constexpr int ST = Sh::ST, TILE = Sh::TILE, NS = Sh::NS;
    constexpr uint32_t TM_O = 256, TM_COLS = 512;
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    uint8_t *sQ = smem_raw, *sK = sQ + 2 * TILE, *sV = sK + ST * TILE;
    float *sNb = (float *)(sV + ST * TILE);       // [2 row tiles][2][256]
    uint64_t *bars = (uint64_t *)(sNb + 4 * 256);
    uint64_t *q_full = bars, *q_empty = bars + 2, *s_full = bars + 4, *p_ready = bars + 6, *o_full = bars + 8, *fix = bars + 10;
    uint64_t *k_full = bars + 11, *k_empty = k_full + ST, *v_full = k_empty + ST, *v_empty = v_full + ST;
    uint64_t *nb_full = v_empty + ST;
    uint32_t *slot = (uint32_t *)(nb_full + 2);
    volatile int *abort_flag = (volatile int *)(slot + 1);

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, H = a.H;
    if ((smem_u32(smem_raw) & 1023u) != 0u) {     // the swizzled tiles need 1024-byte alignment
        if (tid == 0) atomicCAS(a.status, 0, HDT_ERR_CUDA);
        return;
    }
    if (tid == 0) {
        for (int i = 0; i < 2; ++i) {
            mbar_init(&q_full[i], 1);
            mbar_init(&q_empty[i], 1);
            mbar_init(&s_full[i], 1);
            mbar_init(&p_ready[i], 128);
            mbar_init(&o_full[i], 1);
            mbar_init(&nb_full[i], 128);
        }
        mbar_init(fix, 1);
        for (int i = 0; i < 4 * ST; ++i) mbar_init(k_full + i, 1);
        *abort_flag = (*a.status != 0);
        fence_mbar_init();
    }
    if (warp == 0) tmem_alloc(slot, TM_COLS);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *slot;
    const bool dead = (*abort_flag != 0);
    bool ok = true;
    int fail_site = 0;
    pdl_wait();
    const int n_units = *a.q.count * H;

#define HDT_AGREE() (ok = __all_sync(0xffffffffu, ok))
#define HDT_WAIT(bar, parity, site)                                                   \
    do {                                                                              \
        if (ok && !mbar_wait((bar), (uint32_t)(parity), abort_flag, WAIT_CYCLES)) {   \
            ok = false;                                                               \
            fail_site = (site);                                                       \
        }                                                                             \
    } while (0)

    auto key_tiles = [&](const SelfBlk &b, int w) {
        const int r = b.r0 + 128 * w;
        if (128 * w >= a.block_rows || r >= b.nq) return 0;
        return (self_keys_of(a.causal, r, 128, b.nq, b.nk) + 127) >> 7;
    };

    // 168 registers a thread at launch (384 threads): the softmax warps take what the others do not need
    // (256 x 208 + 128 x 88 = 384 x 168, or 256 x 224 + 128 x 56)
    if (warp < 8) {
        if constexpr (D == 64) asm volatile("setmaxnreg.inc.sync.aligned.u32 208;");
        else asm volatile("setmaxnreg.inc.sync.aligned.u32 224;");
        if (!dead) {
            // ================= softmax: row tile w, a thread per row =================
            const int w = warp >> 2, rl = tid & 127;
            const uint32_t lane_base = (uint32_t)((warp & 3) * 32) << 16, tm_s = tmem + 128u * w + lane_base, tm_o = tmem + TM_O + D * w + lane_base;
            int ns = 0, near_no = 0, nu = 0;
            for (int k = 0, u; ok && (u = self_unit(k, blockIdx.x, gridDim.x)) < n_units; ++k) {
                const SelfBlk b = a.q.blk[u / H];
                const int h = u % H, nt = key_tiles(b, w), row = b.r0 + 128 * w + rl;
                const bool valid = 128 * w < a.block_rows && row < b.nq;
                const int first = b.off + b.r0 + 128 * w;      // position of the tile's first row
                const int lim0 = !valid ? 0 : a.causal ? min(max(b.off + row + 1, 0), b.nk) : b.nk;
                const float *bias = a.dist.bias + (size_t)h * a.dist.n;
                const int whole = __reduce_min_sync(0xffffffffu, lim0) >> 7;      // tiles that every row of the warp sees whole
                float m = -INFINITY, l = 0.f, ahead[2] = {0.f, 0.f};
                auto request_near = [&](int base) {      // this thread's two entries of a tile's bias vector
                    ahead[0] = bias[self_dist_at(a.dist, base + rl - 127)];
                    ahead[1] = bias[self_dist_at(a.dist, base + rl + 1)];
                };
                for (int j = 0; j < nt; ++j, ++ns) {
                    const int base = first - 128 * j, lim = lim0 - 128 * j;
                    float c = 0.f;
                    bool near = false;
                    float *nb = sNb + (w * 2 + (near_no & 1)) * 256;
                    if (a.bias_on) {
                        if (base - 127 >= a.dist.far) c = bias[a.dist.n - 1];
                        else if (base + 127 <= -a.dist.far) c = bias[0];
                        else {
                            near = true;
                            if (!Sh::NEAR_AHEAD || j == 0) request_near(base);
                            nb[rl] = ahead[0];
                            nb[rl + 128] = ahead[1];
                            mbar_arrive(&nb_full[w]);      // (an mbarrier, whose wait is bounded, and not a CTA barrier)
                        }
                        if (Sh::NEAR_AHEAD && j + 1 < nt && base - 128 - 127 < a.dist.far && base - 128 + 127 > -a.dist.far) request_near(base - 128);
                        if (near) {
                            HDT_WAIT(&nb_full[w], near_no & 1, 12);
                            ++near_no;
                        }
                    }
                    HDT_WAIT(&s_full[w], ns & 1, 10);
                    if (!HDT_AGREE()) break;
                    tc_fence_after();
                    float s[128];
#pragma unroll
                    for (int i = 0; i < 4; ++i) tmem_ld32(tm_s + 32u * i, reinterpret_cast<uint32_t(&)[32]>(s[32 * i]));
                    tmem_wait_ld();
                    float sl = a.scale_log2;
                    if (near) {
                        const float *nr = nb + rl + 127;
#pragma unroll
                        for (int i = 0; i < 128; i += 2) {
                            const f2 x = fma2(pack2(s[i], s[i + 1]), pack2(sl, sl), pack2(nr[-i], nr[-i - 1]));
                            unpack2(x, s[i], s[i + 1]);
                        }
                        sl = 1.f;
                    }
                    if (j >= whole) {      // (a row of the warp does not see the whole tile)
#pragma unroll
                        for (int i = 0; i < 128; ++i) s[i] = i < lim ? s[i] : -INFINITY;
                    }
                    float x[4] = {s[0], s[1], s[2], s[3]};
#pragma unroll
                    for (int i = 4; i < 128; ++i) x[i & 3] = fmaxf(x[i & 3], s[i]);
                    const float top = fmaf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), sl, c);
                    if (j == 0) m = top;
                    else if (__any_sync(0xffffffffu, top > m + 8.f)) {
                        const float m1 = top > m + 8.f ? top : m, f = m1 == m ? 1.f : exp2f(m - m1);
                        m = m1;
                        l *= f;
#pragma unroll
                        for (int i = 0; i < D / 32; ++i) {
                            uint32_t o[32];
                            tmem_ld32(tm_o + 32u * i, o);
                            tmem_wait_ld();
#pragma unroll
                            for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
                            tmem_st32(tm_o + 32u * i, o);
                        }
                    }
                    const float cm = m == -INFINITY ? c : c - m;      // (no key so far: all of s, or c, is -inf, and exp2(-inf) = 0)
                    f2 sum[2] = {pack2(0.f, 0.f), pack2(0.f, 0.f)};
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        uint32_t p[32];
#pragma unroll
                        for (int i = 0; i < 32; ++i) {
                            float p0, p1;
                            unpack2(fma2(pack2(s[64 * half + 2 * i], s[64 * half + 2 * i + 1]), pack2(sl, sl), pack2(cm, cm)), p0, p1);
                            p0 = exp2f(p0);
                            p1 = exp2f(p1);
                            sum[i & 1] = add2(sum[i & 1], pack2(p0, p1));
                            p[i] = pack_bf16(p0, p1);
                        }
                        tmem_st32(tm_s + 32u * half, p);
                    }
                    float sum0, sum1;
                    unpack2(add2(sum[0], sum[1]), sum0, sum1);
                    l += sum0 + sum1;
                    tmem_wait_st();
                    tc_fence_before();
                    mbar_arrive(&p_ready[w]);
                }
                if (!ok) break;
                if (nt > 0) {
                    HDT_WAIT(&o_full[w], nu & 1, 11);
                    ++nu;
                    if (!HDT_AGREE()) break;
                    tc_fence_after();
                }
                const float inv = l == 0.f ? 0.f : 1.f / l;
                __nv_bfloat16 *out = (__nv_bfloat16 *)a.o + ((size_t)(b.q0 + row) * H + h) * D;
#pragma unroll
                for (int i = 0; i < D / 32; ++i) {
                    uint32_t o[32];
                    if (nt > 0) {
                        tmem_ld32(tm_o + 32u * i, o);
                        tmem_wait_ld();
                    } else {
#pragma unroll
                        for (int e = 0; e < 32; ++e) o[e] = 0u;
                    }
                    if (valid)
#pragma unroll
                        for (int e = 0; e < 32; e += 8) {
                            uint32_t y[4];
#pragma unroll
                            for (int t = 0; t < 4; ++t) y[t] = pack_bf16(__uint_as_float(o[e + 2 * t]) * inv, __uint_as_float(o[e + 2 * t + 1]) * inv);
                            *reinterpret_cast<uint4 *>(out + 32 * i + e) = make_uint4(y[0], y[1], y[2], y[3]);
                        }
                }
                tc_fence_before();      // (the next unit's first product over O comes behind this thread's next arrival at p_ready)
                if (valid) a.lse[(size_t)h * a.Tq + b.q0 + row] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
            }
        }
    } else {
        if constexpr (D == 64) asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
        else asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
        if (dead) {
        } else if (warp == 8) {
            // ================= load warp =================
            int uq[2] = {0, 0}, kt = 0, nfix = 0;
            for (int k = 0, u; ok && (u = self_unit(k, blockIdx.x, gridDim.x)) < n_units; ++k) {
                const SelfBlk b = a.q.blk[u / H];
                const int h = u % H, nt[2] = {key_tiles(b, 0), key_tiles(b, 1)}, n = max(nt[0], nt[1]);
                auto load = [&](uint8_t *dst, const CUtensorMap *tm, int row, uint64_t *bar) {
                    mbar_expect_tx(bar, (uint32_t)TILE);
#pragma unroll
                    for (int s = 0; s < NS; ++s) tma_load_3d(dst + s * SUB, tm, 64 * s, h, row, bar);
                };
                auto load_q = [&](int w) {
                    if (nt[w] == 0) return;
                    if (uq[w] > 0) HDT_WAIT(&q_empty[w], (uq[w] - 1) & 1, 1);
                    ++uq[w];
                    if (!HDT_AGREE()) return;
                    if (lane == 0) load(sQ + w * TILE, &tm_q, b.q0 + b.r0 + 128 * w, &q_full[w]);
                };
                load_q(0);
                for (int j = 0; j < n && ok; ++j, ++kt) {
                    const int s = kt % ST, round = kt / ST;
                    if (round > 0) HDT_WAIT(&k_empty[s], (round - 1) & 1, 2);
                    if (!HDT_AGREE()) break;
                    if (lane == 0) load(sK + s * TILE, &tm_k, b.k0 + 128 * j, &k_full[s]);
                    if (j == 0) load_q(1);
                    if (round > 0) HDT_WAIT(&v_empty[s], (round - 1) & 1, 3);
                    if (!HDT_AGREE()) break;
                    const int rows = b.nk - 128 * j;      // rows of the tile that are the document's
                    if (rows >= 128) {
                        if (lane == 0) load(sV + s * TILE, &tm_v, b.k0 + 128 * j, &v_full[s]);
                    } else {
                        if (lane == 0) load(sV + s * TILE, &tm_v, b.k0 + 128 * j, fix);
                        HDT_WAIT(fix, nfix & 1, 4);
                        ++nfix;
                        ok = __all_sync(0xffffffffu, ok);
                        if (!ok) break;
                        for (int x = lane; x < (128 - rows) * 8; x += 32)
#pragma unroll
                            for (int t = 0; t < NS; ++t) *reinterpret_cast<uint4 *>(sV + s * TILE + t * SUB + rows * 128 + x * 16) = make_uint4(0, 0, 0, 0);
                        fence_proxy_async_smem();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(&v_full[s]);
                    }
                }
            }
        } else if (warp == 9) {
            // ================= MMA warp =================
            const uint32_t id_s = idesc_bf16(128, false, false), id_o = idesc_bf16(D, false, true);
            const uint64_t d_q = smem_desc(smem_u32(sQ), 0, 1024), d_k = smem_desc(smem_u32(sK), 0, 1024), d_v = smem_desc(smem_u32(sV), SUB, 1024);
            const uint32_t q_hi = (uint32_t)(d_q >> 32), k_hi = (uint32_t)(d_k >> 32), v_hi = (uint32_t)(d_v >> 32);
            const uint32_t leader = elect_one() ? 1u : 0u;
            // (TMEM is allocated whole, its addresses begin at 0)
            auto issue_s = [&](uint32_t w, uint32_t s) {
                const uint32_t q_lo = (uint32_t)d_q + w * (TILE >> 4), k_lo = (uint32_t)d_k + s * (TILE >> 4);
#pragma unroll
                for (uint32_t kk = 0; kk < D / 16; ++kk)
                    mma_ss_p(leader, 128u * w, q_lo + (kk >> 2) * (SUB >> 4) + 2u * (kk & 3u), q_hi, k_lo + (kk >> 2) * (SUB >> 4) + 2u * (kk & 3u), k_hi, id_s, kk > 0);
                mma_commit_p(leader, &s_full[w]);
            };
            auto issue_o = [&](uint32_t w, uint32_t s, uint32_t acc) {
                const uint32_t v_lo = (uint32_t)d_v + s * (TILE >> 4);
#pragma unroll
                for (uint32_t kk = 0; kk < 8; ++kk) mma_ts_p(leader, TM_O + D * w, 128u * w + 8u * kk, v_lo + 128u * kk, v_hi, id_o, acc | (kk > 0));
            };
            auto wait = [&](uint64_t *bar, uint32_t parity, int site) {      // (the whole warp knows whether it ended well)
                HDT_WAIT(bar, parity, site);
                return HDT_AGREE();
            };
            uint32_t uq[2] = {0, 0}, np[2] = {0, 0}, st = 0, round = 0;      // ring stage of this tile and parity of its use
            bool go = true;
            for (int k = 0, u; go && (u = self_unit(k, blockIdx.x, gridDim.x)) < n_units; ++k) {
                const SelfBlk b = a.q.blk[u / H];
                const int nt[2] = {__shfl_sync(0xffffffffu, key_tiles(b, 0), 0), __shfl_sync(0xffffffffu, key_tiles(b, 1), 0)}, n = max(nt[0], nt[1]);
                if (n == 0) continue;
                go = wait(&k_full[st], round, 5);
#pragma unroll
                for (uint32_t w = 0; w < 2; ++w)
                    if (go && nt[w] > 0) {
                        go = wait(&q_full[w], uq[w] & 1u, 6);
                        ++uq[w];
                        if (!go) break;
                        tc_fence_after();
                        issue_s(w, st);
                        if (nt[w] == 1) mma_commit_p(leader, &q_empty[w]);
                    }
                if (!go) break;
                mma_commit_p(leader, &k_empty[st]);
                for (int j = 0; j < n && go; ++j) {
                    const uint32_t s1 = st + 1 == ST ? 0 : st + 1, round1 = st + 1 == ST ? round ^ 1u : round;
                    go = wait(&v_full[st], round, 7) && (j + 1 >= n || wait(&k_full[s1], round1, 8));
#pragma unroll
                    for (uint32_t w = 0; w < 2; ++w)
                        if (go && j < nt[w]) {
                            go = wait(&p_ready[w], np[w] & 1u, 9);
                            ++np[w];
                            if (!go) break;
                            tc_fence_after();
                            issue_o(w, st, j > 0 ? 1u : 0u);
                            if (j + 1 < nt[w]) {
                                issue_s(w, s1);      // (over P, which the products before it have read)
                                if (j + 2 == nt[w]) mma_commit_p(leader, &q_empty[w]);
                            } else mma_commit_p(leader, &o_full[w]);
                        }
                    if (!go) break;
                    mma_commit_p(leader, &v_empty[st]);
                    if (j + 1 < n) mma_commit_p(leader, &k_empty[s1]);
                    st = s1;
                    round = round1;
                }
            }
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

template <int D>
static int go(const SelfFwdArgs &a, cudaStream_t st) {
    static DevOnce attr;
    if (!attr.done()) {
        HDT_CUDA_CHECK(cudaFuncSetAttribute(k_self_fwd<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, FwdShape<D>::SMEM));
        attr.set();
    }
    int n_sm = 0;
    if (const int rc = sm_count(&n_sm)) return rc;
    CUtensorMap tq, tk, tv;
    if (const int rc = make_tmap_bf16(&tq, a.qp, D, a.H, a.Tq, 128)) return rc;
    if (const int rc = make_tmap_bf16(&tk, a.kp, D, a.H, a.Tk, 128)) return rc;
    if (const int rc = make_tmap_bf16(&tv, a.vp, D, a.H, a.Tk, 128)) return rc;
    const long long units = (long long)a.q.most * a.H;
    HDT_CUDA_CHECK(launch_dependent(k_self_fwd<D>, true, dim3((unsigned)(units < n_sm ? units : n_sm)), 384, FwdShape<D>::SMEM, st, tq, tk, tv, a));
    return HDT_OK;
}
int launch_self_fwd_tc(const SelfFwdArgs &a, int head_dim, cudaStream_t st) { return head_dim == 64 ? go<64>(a, st) : go<128>(a, st); }

}  // namespace hdt
