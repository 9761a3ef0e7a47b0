// What the attention kernels have in common: arguments, the sequences of a call, the split of the work among the
// CTAs, which key a row sees, and the slow path for rows that need care.
//
// Rows.  Query heads of one key/value head share its keys, so a row of the product is a (token, query head of the
// group) pair: row r of a sequence is token r / group, head h * group + r % group.  An ITEM is a block of
// `rows_tile` rows of one sequence and key/value head against all keys that block sees; keys come in tiles of
// `key_tile`.
//
// Split of the work (tree attention).  A tree has few rows and a long context: one CTA per item would leave most of
// the GPU idle and follow the longest context.  So all key tiles of all items are laid end to end (sequence, head,
// row block, tile) and cut into equal ranges, one per CTA, whatever the lengths: a CTA holds at most one item that
// began before it and one that goes on behind it, whose running maximum, sum and unnormalised product go to the
// workspace; whole items are written out.  The cut depends on the lengths alone, so results do not depend on timing.
#pragma once

#include <math_constants.h>

#include "common.cuh"

namespace s2moe {

constexpr int kAttnMaxNodes = 64;         // nodes of a tree with parents: one bit each

struct AttnArgs {
    const void *q;               // [n_tokens][Hq][D], q_stride elements from token to token
    const void *k, *v;           // prompts: [n_tokens][Hk][D] with strides; trees: the layer's pages [n_pages][Hk][page][D]
    void *out;                   // [n_tokens][Hq][D]
    long long q_stride, k_stride, v_stride;
    const int32_t *seq_start;    // [n_seq + 1] first token of every sequence
    const int32_t *node_start;   // [n_seq + 1] first node of every tree, or NULL: the tokens are the nodes
    const int32_t *context;      // [n_seq] committed tokens
    const int32_t *parent;       // [n_nodes], or NULL: chains
    const int32_t *page_table;   // [n_seq][table_width]
    int n_seq, n_tokens, n_nodes, Hk, group, table_width, page_shift, n_pages;
    int rows_tile;               // rows of an item
    int min_units;               // split: tiles that a CTA takes at least
    float scale_log2;            // scale * log2(e): exponentials are taken to base 2
    float *part_o;               // split: [CTA][2][rows_tile][D] unnormalised product
    float *part_ml;              // split: [CTA][2][rows_tile][2] maximum (times scale_log2) and sum
    int *status;                 // device word: a bounded wait gave up
};

struct AttnSeq {
    int tok0, n;                 // tokens (rows of q)
    int node0, nodes;            // tree; the tokens are its last n nodes
    int ctx, total;              // committed keys, keys in all
    bool bad;                    // more tokens than nodes, or a tree too large for its masks: rows become NaN
};

// Device arrays can hold anything, so every value is brought into range here: nothing outside the arrays is read.
template <bool PAGED>
__device__ __forceinline__ AttnSeq attn_seq(const AttnArgs &a, int s)
{
    AttnSeq q;
    q.tok0 = min(max(__ldg(a.seq_start + s), 0), a.n_tokens);
    q.n = min(max(__ldg(a.seq_start + s + 1), q.tok0), a.n_tokens) - q.tok0;
    q.node0 = q.tok0;
    q.nodes = q.n;
    q.ctx = 0;
    q.total = q.n;
    q.bad = false;
    if (PAGED) {
        if (a.node_start) {
            q.node0 = min(max(__ldg(a.node_start + s), 0), a.n_nodes);
            q.nodes = min(max(__ldg(a.node_start + s + 1), q.node0), a.n_nodes) - q.node0;
        }
        const int cap = a.table_width << a.page_shift;
        q.ctx = min(max(__ldg(a.context + s), 0), cap);
        q.total = q.ctx + min(q.nodes, cap - q.ctx);
        q.bad = q.n > q.nodes || (a.parent && q.nodes > kAttnMaxNodes);
    }
    return q;
}

// ancestors of node i, itself among them, as bits; a parent that does not come before its child counts as none
__device__ __forceinline__ unsigned long long attn_ancestors(const AttnArgs &a, const AttnSeq &q, int i)
{
    unsigned long long m = 0;
    while (i >= 0 && i < kAttnMaxNodes) {
        m |= 1ull << i;
        const int p = __ldg(a.parent + q.node0 + i);
        i = p < i ? p : -1;
    }
    return m;
}

// first key behind those that token t of the sequence sees, ancestry aside
template <bool PAGED>
__device__ __forceinline__ int attn_limit(const AttnSeq &q, int t)
{
    const int lim = PAGED ? q.ctx + max(q.nodes - q.n + t, 0) + 1 : t + 1;
    return min(lim, q.total);
}

// does a row see the key; lim from attn_limit, anc from attn_ancestors (all ones for chains)
__device__ __forceinline__ bool attn_sees(int key, int ctx, int lim, unsigned long long anc)
{
    return key < lim && (key < ctx || key - ctx >= kAttnMaxNodes || ((anc >> (key - ctx)) & 1ull));
}

// element offset of a key's row in k and v; false: its page is none of the cache's
template <bool PAGED, int D>
__device__ __forceinline__ bool attn_key(const AttnArgs &a, const AttnSeq &q, int s, int h, int key, long long &ko, long long &vo)
{
    if (PAGED) {
        const int page = __ldg(a.page_table + (long long)s * a.table_width + (key >> a.page_shift));
        if ((unsigned)page >= (unsigned)a.n_pages) return false;
        ko = vo = ((((long long)page * a.Hk + h) << a.page_shift) + (key & ((1 << a.page_shift) - 1))) * D;
    } else {
        ko = (long long)(q.tok0 + key) * a.k_stride + h * D;
        vo = (long long)(q.tok0 + key) * a.v_stride + h * D;
    }
    return true;
}

// ---- the split ---------------------------------------------------------------------------------------------------

template <int KEY_TILE>
struct AttnCut {
    __device__ static int tiles(const AttnSeq &q) { return max(1, (q.total + KEY_TILE - 1) / KEY_TILE); }
    __device__ static int row_tiles(const AttnArgs &a, const AttnSeq &q)
    {
        return (int)(((long long)q.n * a.group + a.rows_tile - 1) / a.rows_tile);
    }
};

struct AttnPiece {
    int s, h, rt;                // sequence, key/value head, block of rows
    int t0, t1;                  // key tiles
    int slot;                    // place in the workspace, or -1: whole item, written out
    AttnSeq q;
};

// Walks the pieces of one CTA; every warp that needs them walks for itself, all 32 lanes together.
// SPLIT: units are key tiles and a CTA takes one range of them; otherwise units are items and a CTA takes every
// gridDim.x-th (prompts: the blocks of a sequence with the most keys first, its heads side by side).
template <bool PAGED, bool SPLIT, int KEY_TILE>
struct AttnIter {
    using Cut = AttnCut<KEY_TILE>;
    const AttnArgs &a;
    const int lane;
    int s = -1;
    long long base = 0, units = 0;       // first unit and units of sequence s
    long long u = 0, u_end = 0;
    AttnSeq q{};
    bool first = true;

    __device__ AttnIter(const AttnArgs &args, int lane_) : a(args), lane(lane_) {}

    __device__ long long units_of(int i) const
    {
        const AttnSeq x = attn_seq<PAGED>(a, i);
        return (long long)a.Hk * Cut::row_tiles(a, x) * (SPLIT ? Cut::tiles(x) : 1);
    }
    __device__ bool seek(long long unit)
    {
        if (unit < base + units) return true;
        long long b = base + units;
        for (int s0 = s + 1; s0 < a.n_seq; s0 += 32) {
            const int mine = s0 + lane;
            const long long un = mine < a.n_seq ? units_of(mine) : 0;
            long long inc = un;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const long long t = __shfl_up_sync(0xffffffffu, inc, o);
                if (lane >= o) inc += t;
            }
            const unsigned hit = __ballot_sync(0xffffffffu, b + inc > unit);
            if (hit) {
                const int l = __ffs((int)hit) - 1;
                s = s0 + l;
                base = b + __shfl_sync(0xffffffffu, inc - un, l);
                units = __shfl_sync(0xffffffffu, un, l);
                q = attn_seq<PAGED>(a, s);
                return true;
            }
            b += __shfl_sync(0xffffffffu, inc, 31);
        }
        return false;
    }
    __device__ long long total_units() const
    {
        long long w = 0;
        for (int i = lane; i < a.n_seq; i += 32) w += units_of(i);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) w += __shfl_xor_sync(0xffffffffu, w, o);
        return w;
    }
    // CTAs that take part in a split of w units
    __device__ static long long ctas(const AttnArgs &a, long long w, int grid)
    {
        return max(1ll, min((long long)grid, w / a.min_units));
    }
    __device__ void begin()
    {
        if (SPLIT) {
            const long long w = total_units(), g = ctas(a, w, (int)gridDim.x);
            if (blockIdx.x < g) {
                u = w * blockIdx.x / g;
                u_end = w * (blockIdx.x + 1) / g;
            }
        } else {
            u = blockIdx.x;
            u_end = 1ll << 62;
        }
    }
    __device__ bool next(AttnPiece &p)
    {
        if (u >= u_end || !seek(u)) return false;
        p.s = s;
        p.q = q;
        const int rts = Cut::row_tiles(a, q);
        if (SPLIT) {
            const int tiles = Cut::tiles(q);
            const int rel = (int)(u - base), item = rel / tiles;
            p.h = item / rts;
            p.rt = item - p.h * rts;
            p.t0 = rel - item * tiles;
            p.t1 = (int)min((long long)tiles, p.t0 + (u_end - u));
            // an unfinished item is the CTA's first (place 0) or its last (place 1)
            p.slot = p.t0 == 0 && p.t1 == tiles ? -1 : 2 * (int)blockIdx.x + (first ? 0 : 1);
            first = false;
            u += p.t1 - p.t0;
        } else {
            const int rel = (int)(u - base), r = rel / a.Hk;
            p.h = rel - r * a.Hk;
            p.rt = PAGED ? r : rts - 1 - r;
            p.t0 = 0;
            // no key behind the last row's own is needed
            const int last = min(q.n, ((p.rt + 1) * a.rows_tile + a.group - 1) / a.group) - 1;
            p.t1 = max(1, (attn_limit<PAGED>(q, last) + KEY_TILE - 1) / KEY_TILE);
            p.slot = -1;
            u += gridDim.x;
        }
        return true;
    }
};

// ---- rows that need care --------------------------------------------------------------------------------------------

template <typename T>
__device__ __forceinline__ float attn_float(T x);
template <>
__device__ __forceinline__ float attn_float<float>(float x) { return x; }
template <>
__device__ __forceinline__ float attn_float<__nv_bfloat16>(__nv_bfloat16 x) { return __bfloat162float(x); }

__device__ __forceinline__ bool attn_finite(float x) { return fabsf(x) <= CUDART_MAX_NORMAL_F; }

// A product with a weight of zero is no zero where the value is infinite or NaN: a key that a row must not see can
// so reach it through the tiles it shares with others.  A row whose result is not finite, or that has no weight at
// all, comes here: one warp looks whether an unseen key between the row's limit and `kend` (the end of what its item
// went through) could have done it, and if so takes the row's keys one by one.  All lanes return with lane l's
// values of columns l, l + 32, ...; false: the result at hand stands.
// Cost: nothing where results are finite; otherwise the unseen keys of one tile, rarely a whole row.
template <typename T, int D, bool PAGED>
__device__ __noinline__ bool attn_row_again(const AttnArgs &a, const AttnSeq &q, int s, int h, int token, int head, int kend,
                                            bool no_weight, float (&o)[D / 32])
{
    const int lane = threadIdx.x & 31;
    const T *kp = reinterpret_cast<const T *>(a.k), *vp = reinterpret_cast<const T *>(a.v);
    const int lim = attn_limit<PAGED>(q, token);
    const unsigned long long anc = PAGED && a.parent && !q.bad ? attn_ancestors(a, q, q.nodes - q.n + token) : ~0ull;
    long long ko, vo;
    if (!no_weight) {
        bool found = false;
        for (int key = PAGED ? q.ctx : lim; key < min(kend, q.total); ++key) {
            if (attn_sees(key, q.ctx, lim, anc) || !attn_key<PAGED, D>(a, q, s, h, key, ko, vo)) continue;
#pragma unroll
            for (int i = 0; i < D / 32; ++i) found |= !attn_finite(attn_float(vp[vo + lane + 32 * i]));
            if (__any_sync(0xffffffffu, found)) { found = true; break; }
        }
        if (!__any_sync(0xffffffffu, found)) return false;
    }
    const T *qp = reinterpret_cast<const T *>(a.q) + (long long)(q.tok0 + token) * a.q_stride + (long long)head * D;
    float x[D / 32], m = -CUDART_INF_F, l = 0.f;
    bool any = false;
#pragma unroll
    for (int i = 0; i < D / 32; ++i) {
        x[i] = attn_float(qp[lane + 32 * i]);
        o[i] = 0.f;
    }
    for (int key = 0; key < lim; ++key) {
        if (!attn_sees(key, q.ctx, lim, anc) || !attn_key<PAGED, D>(a, q, s, h, key, ko, vo)) continue;
        any = true;
        float dot = 0.f;
#pragma unroll
        for (int i = 0; i < D / 32; ++i) dot = fmaf(x[i], attn_float(kp[ko + lane + 32 * i]), dot);
#pragma unroll
        for (int w = 16; w > 0; w >>= 1) dot += __shfl_xor_sync(0xffffffffu, dot, w);
        dot *= a.scale_log2;
        if (dot != dot) l = dot;                       // one NaN score makes the row NaN
        const float mn = fmaxf(m, dot);
        if (mn == -CUDART_INF_F) continue;
        const float f = m == -CUDART_INF_F ? 0.f : exp2f(m - mn), p = exp2f(dot - mn);
        m = mn;
        l = l * f + p;
        bool all_nan = true;
#pragma unroll
        for (int i = 0; i < D / 32; ++i) {
            const float val = attn_float(vp[vo + lane + 32 * i]);
            o[i] = (o[i] == 0.f ? 0.f : o[i] * f) + p * val;
            all_nan &= o[i] != o[i];
        }
        if (l != l || __all_sync(0xffffffffu, all_nan)) break;
    }
#pragma unroll
    for (int i = 0; i < D / 32; ++i) o[i] = any ? (l != l ? l : l == 0.f ? CUDART_NAN_F : o[i] / l) : 0.f;
    return true;
}

}  // namespace s2moe
