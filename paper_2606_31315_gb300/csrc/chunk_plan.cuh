// How the work of a chunk attention is laid out: what chunk_attention.cu (a bf16 cache) and chunk_attention_fp8.cu (a cache
// in 8 bits) share.  The work tiles of all sequences and heads lie on one line, measured in keys; every CTA takes an equal
// stretch of it, and what a cut leaves in parts is merged by a second kernel (chunk_merge_kernel, in chunk_attention.cu).
// Whoever includes this has defined bp::kTileCost, a work tile's fixed cost (queries in, output out) in keys.
#pragma once

#include <cuda_bf16.h>

#include "common.cuh"
#include "ptx_sm103.cuh"

namespace bp {

constexpr int kTileM = 128;                      // rows of one stream's query tile
constexpr int kKeys = 128;                       // keys per K/V tile

constexpr int kLeastCost = 2 * kKeys;            // of a CTA's stretch: below it, fewer CTAs take part
constexpr int kLeastCut = 2;                     // key tiles on either side of a cut

struct ChunkParams {
    __nv_bfloat16* o;
    float* lse;
    const int32_t* cu_q;
    const int32_t* cu_kv;
    const int32_t* block_table;
    int num_seqs, total_q, num_q_heads, num_kv_heads, group;
    int tokens;  // of one stream's tile: floor(128 / group)
    int pages_per_seq, page_shift, num_pages;
    int max_q, max_kv;  // of a sequence: the merge's launch rests on them
    int causal, window;
    float scale_log2;
    float* part_o;   // [grid][2][D / 8][256][8] (part_at): the first stretch's part (it began in an earlier CTA) and the last one's
    float2* part_ml; // [grid][2][256]
    unsigned long long grid_inverse;  // 2^64 / the grid, rounded down
    int4* info;      // [grid]: flags; of the tile that the CTA began and did not end, its first token's row among the
                     // queries, its tokens and its KV head
    unsigned int* err;
};
enum : int { kHasTail = 1, kHasHead = 2, kHeadEnds = 4 };

namespace {  // (each translation unit has its own)

// Where column `col` (a multiple of 8) of row `row` of a part lies: 8 columns of all rows together, so that the threads of
// a warp, a row each, write whole lines.
template <int D>
__device__ __forceinline__ size_t part_at(size_t slot, int row, int col) {
    return ((slot * (D / 8) + col / 8) * (2 * kTileM) + row) * 8;
}

__device__ __forceinline__ float chunk_exp2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// What a row's maximum and sum say of it.  A row saw no key where its maximum is still -inf and its sum 0 (the least sum
// otherwise is the weight of the maximum); all others are divided by what was summed, so that a NaN or an overflow, which
// makes the sum a NaN, shows in the output and in the log-sum-exp.
__device__ __forceinline__ bool saw_no_key(float m, float l) { return m == -INFINITY && l == 0.f; }
__device__ __forceinline__ float row_inverse(float m, float l) { return saw_no_key(m, l) ? 0.f : 1.f / l; }
__device__ __forceinline__ float row_lse(float m, float l) {
    return saw_no_key(m, l) ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
}

// A sequence of B new tokens that ends n keys; tile t holds the tokens [t * Q, (t + 1) * Q).
struct Seq {
    int B, n, Q;
    int causal, window;
    __device__ __forceinline__ int tiles() const { return (B + Q - 1) / Q; }
    __device__ __forceinline__ int hi(int tok_end) const { return causal ? max(0, n - B + tok_end) : n; }  // tok_end <= B
    __device__ __forceinline__ int lo(int tok) const { return window > 0 ? min(n, max(0, n - B + tok + 1 - window)) : 0; }
    __device__ __forceinline__ int keys(int t) const { return max(0, hi(min(B, (t + 1) * Q)) - lo(t * Q)); }
    // sum over t < x of max(0, a + t * Q)
    __device__ __forceinline__ long long ramp(int a, int x) const {
        const int t0 = a >= 0 ? 0 : min(x, (-a + Q - 1) / Q);
        const long long c = x - t0;
        return c * a + Q * ((c * (t0 + x - 1)) >> 1);
    }
    // keys (and fixed costs) of the tiles before x, 0 <= x <= tiles(): cost(t + 1) - cost(t) is kTileCost + keys(t)
    __device__ __forceinline__ long long cost(int x) const {
        long long w = (long long)x * kTileCost;
        const int T = tiles();
        if (causal) {
            w += ramp(n - B + Q, x == T ? x - 1 : x);
            if (x == T && x > 0) w += n;
        } else {
            w += (long long)x * n;
        }
        if (window > 0) w -= ramp(max(n - B + 1 - window, -(1 << 30)), x);
        return w;
    }
};

// A place on the line of all work: key tile j of tile t of head h of sequence s.
struct Place {
    int s, h, t, j;
    __device__ __forceinline__ bool same_tile(const Place& o) const { return s == o.s && h == o.h && t == o.t; }
};

// One CTA's run of key tiles of one work tile.
struct Job {
    int s, h, t;       // sequence (-1: no more jobs), KV head, work tile
    int q0, B, n;      // the sequence's first query row, its new tokens and keys
    int j0, j1;        // key tiles, counted from key 0
    int a[2], b[2];    // those that some row of stream 0's / 1's tile sees (a = b: none)
    int first, last;   // it holds the work tile's first / last key tile
};

__device__ __forceinline__ Seq load_seq(const ChunkParams& p, int s) {
    const int q0 = __ldg(p.cu_q + s), q1 = __ldg(p.cu_q + s + 1), k0 = __ldg(p.cu_kv + s), k1 = __ldg(p.cu_kv + s + 1);
    // (a sequence whose rows are not all among the call's is left out: they would be written behind the outputs' ends)
    const bool there = q0 >= 0 && q1 <= p.total_q;
    if (!there) raise_error(p.err, kErrDeviceArg);
    return Seq{there ? q1 - q0 : 0, k1 - k0, 2 * p.tokens, p.causal, p.window};
}
// Key tiles [first, first + count) under tile t.
__device__ __forceinline__ void tile_span(const Seq& q, int t, int& first, int& count) {
    const int lo = q.lo(t * q.Q), hi = q.hi(min(q.B, (t + 1) * q.Q));
    first = lo / kKeys;
    count = hi > lo ? (hi + kKeys - 1) / kKeys - first : 0;
}
// A sequence's whole part of the line.
__device__ __forceinline__ long long seq_cost(const ChunkParams& p, const Seq& q) {
    if (q.B <= 0) return 0;
    return (q.B <= q.Q ? kTileCost + q.keys(0) : q.cost(q.tiles())) * p.num_kv_heads;
}
// The place at `rem` of that part.
__device__ __forceinline__ Place place_in(const ChunkParams& p, int s, const Seq& q, long long rem) {
    const int T = q.B <= q.Q ? 1 : q.tiles();
    const long long all = T == 1 ? kTileCost + q.keys(0) : q.cost(T);
    Place at;
    at.s = s;
    at.h = min((int)__fdividef((float)rem, (float)all), p.num_kv_heads - 1);  // rem / all, put right below
    rem -= at.h * all;
    while (rem < 0) rem += all, --at.h;
    while (rem >= all) rem -= all, ++at.h;
    at.t = 0;
    for (int hi = T; hi - at.t > 1;) {  // the largest t with cost(t) <= rem
        const int mid = (at.t + hi) >> 1;
        if (q.cost(mid) <= rem) at.t = mid; else hi = mid;
    }
    const int off = (int)(at.t > 0 ? rem - q.cost(at.t) : rem), w = kTileCost + q.keys(at.t);
    int first, count;
    tile_span(q, at.t, first, count);
    at.j = off <= kTileCost ? 0 : min(count, (off - kTileCost + kKeys / 2) / kKeys);
    const bool whole = count < 2 * kLeastCut;  // not to be cut: the nearer end
    if (whole ? 2 * off >= w : count - at.j < kLeastCut) at.j = 0, ++at.t;
    else if (whole || at.j < kLeastCut) at.j = 0;
    if (at.t == T) at.t = 0, ++at.h;
    if (at.h == p.num_kv_heads) at.h = 0, ++at.s;
    return at;
}

// Works through the jobs between two places.
struct Walk {
    const ChunkParams& p;
    Place at, end;
    int known;  // the sequence that `q` and `q0` are of
    Seq q;
    int q0;
    __device__ __forceinline__ bool next(Job& g) {
        while (at.s < end.s || (at.s == end.s && (at.h < end.h || (at.h == end.h && (at.t < end.t || (at.t == end.t && at.j < end.j)))))) {
            if (at.s != known) {
                q = load_seq(p, at.s);
                q0 = __ldg(p.cu_q + at.s);
                known = at.s;
                if (q.B > p.max_q || (q.B > 0 && q.n > p.max_kv)) raise_error(p.err, kErrDeviceArg);
            }
            const int T = q.tiles();
            if (T <= 0) {
                at = Place{at.s + 1, 0, 0, 0};
                continue;
            }
            int first, count;
            tile_span(q, at.t, first, count);
            const bool cut = at.same_tile(end);
            g.s = at.s; g.h = at.h; g.t = at.t; g.q0 = q0; g.B = q.B; g.n = q.n;
            g.j0 = first + at.j;
            g.j1 = first + (cut ? end.j : count);
            g.first = at.j == 0;
            g.last = !cut;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int tok = g.t * q.Q + i * p.tokens, tok_end = min(g.B, tok + p.tokens);
                const int lo = q.lo(tok), hi = q.hi(max(tok_end, 0));
                const int a = max(g.j0, lo / kKeys), b = min(g.j1, (hi + kKeys - 1) / kKeys);
                const bool some = tok < g.B && hi > lo && a < b;
                g.a[i] = some ? a : g.j0;
                g.b[i] = some ? b : g.j0;
            }
            if (cut) {
                at = end;
            } else {
                at.j = 0;
                if (++at.t == T) {
                    at.t = 0;
                    if (++at.h == p.num_kv_heads) at.h = 0, ++at.s;
                }
            }
            return true;
        }
        return false;
    }
};

// This CTA's part of the line, by one warp: [place[0], place[1]).
__device__ __forceinline__ void find_places(const ChunkParams& p, int lane, Place (&place)[2]) {
    const int c = blockIdx.x, mine = lane & 1;  // even lanes find this CTA's begin, odd ones the next one's
    auto take = [&](int s) { return s < p.num_seqs ? load_seq(p, s) : Seq{}; };
    auto scan = [&](long long w) {
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long y = __shfl_up_sync(0xffffffffu, w, o);
            if (lane >= o) w += y;
        }
        return w;
    };
    Seq q = take(lane);
    long long w = seq_cost(p, q), incl = scan(w), total = __shfl_sync(0xffffffffu, incl, 31);
    for (int base = 32; base < p.num_seqs; base += 32) {
        long long more = seq_cost(p, take(base + lane));
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) more += __shfl_xor_sync(0xffffffffu, more, o);
        total += more;
    }
    // the cuts lie at total * c / parts
    const int parts = (int)min((long long)gridDim.x, max(1ll, total / kLeastCost));
    const long long cut = c + mine >= parts               ? total
                          : parts == (int)gridDim.x ? (long long)__umul64hi(total * (c + mine), p.grid_inverse)
                                                    : (long long)((unsigned)total * (unsigned)(c + mine) / (unsigned)parts);
    Seq my_q = q;
    int my_s = p.num_seqs;
    long long my_rem = 0, before = 0;
    for (int base = 0; c < parts && base < p.num_seqs; base += 32) {
        if (base > 0) {
            q = take(base + lane);
            w = seq_cost(p, q);
            incl = before + scan(w);
        }
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const long long at = __shfl_sync(0xffffffffu, cut, e);
            const unsigned hit = __ballot_sync(0xffffffffu, w > 0 && incl - w <= at && at < incl);
            if (hit) {
                const int l = __ffs(hit) - 1;
                const int B = __shfl_sync(0xffffffffu, q.B, l), n = __shfl_sync(0xffffffffu, q.n, l);
                const long long rem = at - __shfl_sync(0xffffffffu, incl - w, l);
                if (mine == e) my_s = base + l, my_q = Seq{B, n, 2 * p.tokens, p.causal, p.window}, my_rem = rem;
            }
        }
        before = __shfl_sync(0xffffffffu, incl, 31);
    }
    Place at = Place{p.num_seqs, 0, 0, 0};
    if (my_s < p.num_seqs) at = place_in(p, my_s, my_q, my_rem);
    __syncwarp();
#pragma unroll
    for (int e = 0; e < 2; ++e)
        place[e] = Place{__shfl_sync(0xffffffffu, at.s, e), __shfl_sync(0xffffffffu, at.h, e),
                         __shfl_sync(0xffffffffu, at.t, e), __shfl_sync(0xffffffffu, at.j, e)};
}

}  // namespace

// Merges what the cuts left (chunk_attention.cu); `few`: every sequence has one tile of one stream.
int launch_chunk_merge(const ChunkParams& p, int head_dim, int grid, int max_q_len, cudaStream_t stream);
// The fields of ChunkParams that both kernels take alike.
ChunkParams chunk_params(const ChunkAttentionArgs& a, int grid);

}  // namespace bp
