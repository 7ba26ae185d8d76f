// Self-attention of packed documents with a learned relative position bias: what its kernels share.
//
//   pos_i = (n_k - n_q) + i for row i of a document's queries, d = pos_i - j for key j,
//   A_ij = scale q_i . k_j + bias[bucket(d)][head]   (causal: d >= 0 only),   O = softmax(A) V.
//
// bucket(d) is monotone in d on either side of 0 and constant beyond `far`, so a tile of 128 x 128 pairs whose
// distances are all beyond it takes one number, and another tile a vector of 255: entry (r, c) depends on r - c.
#pragma once
#include <cuda_bf16.h>

#include "hdt_internal.cuh"

namespace hdt {

constexpr int SELF_MAX_BUCKETS = 128, SELF_MAX_DISTANCE = 32768;
// A finite bias beyond this counts as this: fp32 logits of that size have lost the products they are added to, and
// the difference of a logit and its row's LSE has to stay exact to a few thousandths.
constexpr float SELF_MAX_BIAS = 32768.f;

// Buckets of one direction: bucket b holds the distances [first[b], first[b + 1]).
struct SelfRel {
    int on;            // 0: no bias
    int causal;
    int buckets;       // all
    int one_way;       // of one direction: all, or half of them (then the second half is that of keys behind the query)
    int far;           // first[one_way - 1]: from here on everything is in the last bucket
    int first[SELF_MAX_BUCKETS];
};
__host__ __device__ __forceinline__ int self_bucket_one_way(const SelfRel &r, int d) {      // d >= 0
    int b = 0;
    for (int s = 64; s > 0; s >>= 1)
        if (b + s < r.one_way && r.first[b + s] <= d) b += s;
    return b;
}
__host__ __device__ __forceinline__ int self_bucket(const SelfRel &r, int d) {
    if (r.causal) return self_bucket_one_way(r, d > 0 ? d : 0);
    return d < 0 ? r.one_way + self_bucket_one_way(r, -d) : self_bucket_one_way(r, d);
}
// The bias by distance, expanded once per call (in base-2 logarithms): distances lo .. far, lo = 0 or -far.
struct SelfDist {
    const float *bias;               // [heads][n]
    const unsigned char *bucket;     // [n]
    int lo, far, n;
};
__device__ __forceinline__ int self_dist_at(const SelfDist &s, int d) { return min(max(d, s.lo), s.far) - s.lo; }

struct SelfBlk {
    int q0, nq, k0, nk;      // the document's rows in q and in k
    int r0;                  // first row of the block (in the document), of q or of k
    int off;                 // n_k - n_q
    int tiles, id;           // cost; number of the block before the list was ordered by cost
};
struct SelfLists {
    const SelfBlk *blk;      // ordered by cost, dearest first
    const int *count;
    int most;                // an upper limit that the host knows
};
// Keys that rows [r0, r0 + rows) of a document see at most, and the first row that sees a key of [k, ...).
__host__ __device__ __forceinline__ int self_keys_of(int causal, int r0, int rows, int nq, int nk) {
    const int last = r0 + rows < nq ? r0 + rows : nq, k = causal ? nk - nq + last : nk;
    return k < 0 ? 0 : k > nk ? nk : k;
}
__host__ __device__ __forceinline__ int self_first_row(int causal, int k, int nq, int nk) {
    const int r = causal ? k - (nk - nq) : 0;
    return r < 0 ? 0 : r > nq ? nq : r;
}

// The k-th unit of CTA `cta` of `ctas`, from a list ordered by cost: there and back again, so that who begins with the dearest
// goes on with the cheapest (1 x 4096 tokens, 12 heads: a CTA's most tiles 40 -> 32).  Grows with k.
__device__ __forceinline__ int self_unit(int k, int cta, int ctas) { return k * ctas + (k & 1 ? ctas - 1 - cta : cta); }

struct SelfFwdArgs {
    SelfLists q;             // blocks of block_rows rows
    int block_rows;
    SelfDist dist;
    int H, Tq, Tk, causal, bias_on;
    const void *qp, *kp, *vp;
    void *o;
    float *lse;
    float scale_log2;
    int *status;
};
struct SelfBwdArgs {
    SelfLists blk;           // of q (dQ and the bias) or of k (dK, dV)
    SelfDist dist;
    int H, Tq, Tk, causal, bias_on, buckets;
    const void *qp, *kp, *vp, *dop;
    const float *lse;
    float *delta;            // rowsum(dO o O); bf16: put right by dQ's pass for that of dK and dV
    void *dq, *dk, *dv;
    float scale, scale_log2;
    float *part;             // [block id][head][buckets]: sums of dS by bucket (the pass that is given it), or nullptr
    int *status;
};
int launch_self_fwd_tc(const SelfFwdArgs &a, int head_dim, cudaStream_t st);
int launch_self_bwd_tc(const SelfBwdArgs &keys, const SelfBwdArgs &rows, int head_dim, cudaStream_t st);
int launch_self_fwd_f32(const SelfFwdArgs &a, int head_dim, cudaStream_t st);
int launch_self_bwd_f32(const SelfBwdArgs &keys, const SelfBwdArgs &rows, int head_dim, cudaStream_t st);
constexpr int SELF_F32_ROWS = 64;      // rows of a block in the fp32 kernels

}  // namespace hdt
