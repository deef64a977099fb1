// Attention of chunks of new tokens over a paged KV cache: the prefill of prompts, whole or in chunks, and decoding
// sequences in the same call.
//
//   O_i = sum_j softmax_j(scale <q_i, k_j>) v_j   over lo_i <= j < hi_i
//
// with p_i = n - B + i the position of new token i among its sequence's n keys, hi_i = p_i + 1 (causal) or n, lo_i =
// p_i + 1 - window or 0.  A row that sees no key is 0, its log-sum-exp -inf.
//
//   * The G = Hq / Hkv query heads of a KV head are rows of one tile, token-major: floor(128 / G) tokens are an M = 128
//     tile, two tiles are a work tile that reads every K/V tile once.  Each of the two has eight softmax warps (two
//     threads a row) and its own S, P and O in tensor memory, so that the tensor cores work on one while the other's
//     weights are formed.  A key tile (128 keys) is S = Q K^T, the online softmax in fp32 (base 2, the accumulator
//     rescaled only where a row's maximum grew by more than 2^8), P in bf16 over S, O += P V with P from tensor memory.
//   * The work tiles of all sequences and heads lie on one line, measured in keys; every CTA (one an SM) takes an equal
//     stretch of it and works through its tiles.  Where a cut falls inside a tile, the two CTAs leave (O, m, l) in the
//     workspace and a second kernel merges them, in the order of the keys.  So one long context, a ragged batch and a
//     mix of prompts and decoding sequences all fill the GPU, and no order of arrival enters the result.
//   * Roles: warps 0-7 and 8-15 softmax of stream 0 and 1, warp 16 lays out the CTA's jobs and issues the TMA copies (its
//     lanes the boxes of a tile's pages), warps 17 and 18 issue the streams' MMAs, warp 19 clears the rows of V behind a
//     sequence's last key (a page's unused rows may hold anything; their weight is 0, but 0 times a NaN is none).
//
// What bounds it: of a pair of key tiles' 2 x 16 MMAs, 2,048 cycles at D = 128, about 2,950 are taken: a stream's softmax
// (1,050), its MMAs (1,024) and the hand-overs between them follow one another, with two streams in turn.  2048 tokens
// over 32768 keys, 32 query and 8 KV heads: 706 to 726 us in short runs, 744 to 775 in long ones, as the clock drops (1.37 to
// 1.51 PFLOP/s); a prompt of 8192: 363 to 371 and 389 to 400 us; one token over 2048 keys: 16.5 us, a chain of latencies
// (9 over 100 keys, which need no merge).  How the MMA loops are
// unrolled counts: over the ring's slots as well they took 20 % more, not at all 50 %.
#include <cuda_bf16.h>

#include <algorithm>
#include <mutex>

#include "common.cuh"
#include "ptx_sm103.cuh"

namespace bp {
namespace {

constexpr int kTileM = 128;                      // rows of one stream's query tile
constexpr int kKeys = 128;                       // keys per K/V tile
constexpr int kHalfBytes = kKeys * 128;          // 128 rows of 64 columns, 128-byte swizzle
constexpr int kSoftmaxWarps = 16;                // two threads a row, 64 keys each
constexpr int kProducerWarp = 16, kMmaWarp = 17, kTailWarp = 19;  // (a stream's MMA warp: kMmaWarp + stream)
constexpr int kChunkThreads = 32 * 20;
// Registers: 96 a thread at launch; the softmax warps take 104, the other warpgroup keeps 64 (512 x 104 + 128 x 64 =
// 640 x 96).  The compiler spills 108 bytes a thread at D = 128, 92 at 64, of all roles together.
constexpr int kSoftmaxRegs = 104, kOtherRegs = 64;
constexpr uint32_t kChunkTmem = 512;
// A work tile's fixed cost (queries in, output out), in keys: a prompt of 8192 takes 399 us with 192, 372 with 320, 368
// with 448, 374 with 640.  Heads of 64 and tiles of one stream take the same number; it was not fitted to them.
constexpr int kTileCost = 400;
constexpr int kLeastCost = 2 * kKeys;            // of a CTA's stretch: below it, fewer CTAs take part
constexpr int kLeastCut = 2;                     // key tiles on either side of a cut
constexpr int kJobs = 4;                         // jobs laid out ahead

template <int D>
struct Shape {
    static constexpr int halves = D / 64;
    static constexpr int tile_bytes = halves * kHalfBytes;      // one K, V or Q tile
    static constexpr int slots = D == 128 ? 5 : 12;             // ring of K and V tiles
    static constexpr int tiles = (2 + slots) * tile_bytes;      // the two Q tiles, the ring
    static constexpr uint32_t col_o = 256;                      // O of stream i: columns col_o + i * D
};
static_assert(Shape<128>::tiles >= tmem_smem_share((int)kChunkTmem, 228 * 1024) &&
                  Shape<64>::tiles >= tmem_smem_share((int)kChunkTmem, 228 * 1024),
              "leaves no other CTA's tensor memory room");

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

// Shared memory behind the tiles.
template <int SLOTS>
struct Shared {
    uint64_t full[SLOTS], empty[SLOTS], raw[SLOTS];  // the ring; raw: a V tile that the tail warp hands on
    uint64_t q_full, q_empty, drain[2], turn[2];
    uint64_t s[2], p[2], o[2];                       // of a stream: scores, weights, the accumulator
    uint64_t job_full[kJobs], job_empty[kJobs];
    Job job[kJobs];                                  // what the producer warp has laid out for the others
    uint32_t tmem;
    int pair_failed[8];
    float row[2][2][kTileM];                         // [stream][half]: row maxima, at the end row sums
};
template <int D>
constexpr int chunk_smem() { return Shape<D>::tiles + (int)sizeof(Shared<Shape<D>::slots>); }
static_assert(chunk_smem<128>() <= 227 * 1024 && chunk_smem<64>() <= 227 * 1024, "a block's shared memory");

template <int D>
__global__ void __launch_bounds__(kChunkThreads, 1)
chunk_attention_kernel(const __grid_constant__ ChunkParams p, const __grid_constant__ CUtensorMap qmap,
                       const __grid_constant__ CUtensorMap kmap, const __grid_constant__ CUtensorMap vmap) {
    using S = Shape<D>;
    extern __shared__ __align__(1024) uint8_t smem[];
    uint8_t* const sQ = smem;                           // two tiles
    uint8_t* const sKV = smem + 2 * S::tile_bytes;      // the ring
    Shared<S::slots>& sh = *reinterpret_cast<Shared<S::slots>*>(smem + S::tiles);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int G = p.group;
    if (smem_addr(smem) & 1023) {  // (the swizzled tiles' alignment: dynamic shared memory starts on such a boundary)
        if (tid == 0) raise_error(p.err, kErrDeviceArg);
        return;
    }

    if (tid < 8) sh.pair_failed[tid] = 0;
    if (tid == 0) {
        for (int i = 0; i < S::slots; ++i) {
            mbar_init(&sh.full[i], 1);
            mbar_init(&sh.empty[i], 2);
            mbar_init(&sh.raw[i], 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&sh.s[i], 1);
            mbar_init(&sh.p[i], 256);
            mbar_init(&sh.o[i], 1);
            mbar_init(&sh.drain[i], 1);
            mbar_init(&sh.turn[i], 1);
        }
        for (int i = 0; i < kJobs; ++i) {
            mbar_init(&sh.job_full[i], 1);
            mbar_init(&sh.job_empty[i], kSoftmaxWarps + 3);
        }
        mbar_init(&sh.q_full, 1);
        mbar_init(&sh.q_empty, 2);
        fence_mbar_init();
    }
    if (warp == kMmaWarp) {
        tmem_alloc(&sh.tmem, kChunkTmem);
        tmem_relinquish();
    }
    if (warp == kProducerWarp && lane < 3) prefetch_tensormap(lane == 0 ? &qmap : lane == 1 ? &kmap : &vmap);
    griddep_wait();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    griddep_launch_dependents();
    const uint32_t tmem = sh.tmem;
    // The next job, for a warp that has had `nj` of them; none if there are no more (or a wait was given up: ok is false).
    // The warp reads what it needs and calls had_job.
    auto next_job = [&](unsigned nj, bool& ok) -> const Job* {
        ok = __all_sync(0xffffffffu, mbar_wait(&sh.job_full[nj % kJobs], (nj / kJobs) & 1, kWaitBudget));
        if (!ok) return nullptr;
        const Job* g = &sh.job[nj % kJobs];
        return g->s >= 0 ? g : nullptr;
    };
    auto had_job = [&](unsigned& nj) {
        __syncwarp();
        if (lane == 0) mbar_arrive(&sh.job_empty[nj % kJobs]);
        ++nj;
    };

    if (warp < kSoftmaxWarps) {
        regs_inc<kSoftmaxRegs>();
        // ================= softmax of stream i: two threads a row, each 64 of a tile's keys and half of O's columns.  The
        // two warps that share 32 rows ask each other once a tile whether a row of theirs has outgrown its maximum; where
        // one has, they exchange their halves' maxima and go on with the same numbers.
        const int i = warp >> 3, half = (warp >> 2) & 1, quad = warp & 3;
        const int r = quad * 32 + lane, pair = i * 4 + quad;
        const uint32_t lanes = tmem + (static_cast<uint32_t>(quad * 32) << 16);
        const uint32_t s_addr = lanes + i * 128 + half * 64;  // P comes over this half's own scores
        const uint32_t o_addr = lanes + S::col_o + i * D + half * (D / 2);
        const int my_tok = r / G, my_head = r - my_tok * G;
        unsigned ns = 0, no = 0;
        bool failed = false;
        // what the other half has for this row, given what this one has; false: one of the two warps gave up a wait
        // (the other warp has read the last tile's before this one writes: its weights were waited for since)
        auto meet = [&](float mine, float& theirs) {
            sh.row[i][half][r] = mine;
            if (failed) sh.pair_failed[pair] = 1;
            named_barrier(1 + pair, 64);
            theirs = sh.row[i][half ^ 1][r];
            return *const_cast<volatile int*>(&sh.pair_failed[pair]) == 0;
        };
        unsigned nj = 0;
        for (;;) {
            bool ok;
            const Job* g = next_job(nj, ok);
            // (a warp that gave up a wait takes its partner along, here and wherever they meet: neither waits alone)
            failed = named_barrier_or(1 + pair, 64, !ok);
            if (failed || !g) break;
            const int a = g->a[i], b = g->b[i];
            const int tok = g->t * 2 * p.tokens + i * p.tokens + my_tok;
            const bool active = my_tok < p.tokens && tok < g->B;
            const int pos = g->n - g->B + tok;
            const int hi = !active ? 0 : p.causal ? max(0, pos + 1) : g->n;
            const int lo = p.window > 0 ? max(0, pos + 1 - p.window) : 0;
            const bool first = g->first, whole = first && g->last;
            // the query row's number among all, in the output (-1: none)
            const long long orow = active ? (long long)(g->q0 + tok) * p.num_q_heads + g->h * G + my_head : -1;
            had_job(nj);
            float m = -INFINITY, l = 0.f;
            for (int j = a; j < b; ++j, ++ns) {
                const int from = lo - j * kKeys - half * 64, to = hi - j * kKeys - half * 64;  // visible columns
                const bool full = __all_sync(0xffffffffu, from <= 0 && to >= 64);
                failed = !__all_sync(0xffffffffu, mbar_wait(&sh.s[i], ns & 1, kWaitBudget));
                tc_fence_after();
                uint32_t x[2][32];
                float mine;
                if (full) {
                    float m0, m1;
                    tmem_ld32_max(s_addr, x[0], m0);
                    tmem_ld32_max(s_addr + 32, x[1], m1);
                    tmem_ld_wait();
                    mine = fmaxf(m0, m1);
                } else {
                    tmem_ld32(s_addr, x[0]);
                    tmem_ld32(s_addr + 32, x[1]);
                    tmem_ld_wait();
                    float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                    for (int c = 0; c < 2; ++c)
#pragma unroll
                        for (int e = 0; e < 32; ++e) {
                            if (c * 32 + e < from || c * 32 + e >= to) x[c][e] = 0xff800000u;  // -inf
                            mx[e & 3] = fmaxf(mx[e & 3], __uint_as_float(x[c][e]));
                        }
                    mine = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3]));
                }
                // weights 2^(scale * score - m) of columns [32 c, 32 c + 32), as packed pairs; their sum
                const uint64_t scale2 = pack_f32x2(p.scale_log2, p.scale_log2);
                uint32_t pk[16];
                auto weigh = [&](int c) {
                    const float negm = m == -INFINITY ? 0.f : -m;
                    const uint64_t negm2 = pack_f32x2(negm, negm);
                    uint64_t sum2[2] = {0ull, 0ull};
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        float u, w;
                        unpack_f32x2(fma_f32x2(pack_f32x2(__uint_as_float(x[c][2 * e]), __uint_as_float(x[c][2 * e + 1])), scale2, negm2), u, w);
                        u = chunk_exp2(u);
                        w = chunk_exp2(w);
                        sum2[e & 1] = add_f32x2(sum2[e & 1], pack_f32x2(u, w));
                        // bf16: the type of V, which P multiplies; against 64 bits o is off by 0.0021 to 0.0023 of its
                        // size, with weights in fp32 by 0.0016 to 0.0017 (o's own rounding)
                        pk[e] = pack_bf16x2(u, w);
                    }
                    float u, w;
                    unpack_f32x2(add_f32x2(sum2[0], sum2[1]), u, w);
                    return u + w;
                };
                // the first half of them with the maximum so far, which is rarely outgrown; then again if it was
                float sum = 0.f;
#pragma unroll 1
                for (bool once = true, again = true; again; once = false) {
                    sum = weigh(0);
                    again = false;
                    if (!once) break;
                    // (m is the same in both warps; with it 2^(score - m) stays below 2^8)
                    if (!named_barrier_or(1 + pair, 64, failed || mine * p.scale_log2 > m + 8.f)) break;
                    float theirs;
                    if (!meet(mine, theirs)) {
                        failed = true;
                        break;
                    }
                    const float top = fmaxf(mine, theirs) * p.scale_log2;
                    const bool grew = top > m + 8.f;
                    const float alpha = grew ? chunk_exp2(m - top) : 1.f;
                    // (this tile's scores are complete, so the MMAs before them, the last P V among them, are too)
                    if (j > a && __any_sync(0xffffffffu, grew && m != -INFINITY)) {
#pragma unroll
                        for (int c = 0; c < D / 32; ++c) {
                            uint32_t v[16];
                            tmem_ld16(o_addr + c * 16, v);
                            tmem_ld_wait();
#pragma unroll
                            for (int e = 0; e < 16; ++e) v[e] = __float_as_uint(__uint_as_float(v[e]) * alpha);
                            tmem_st16(o_addr + c * 16, v);
                        }
                    }
                    if (grew) {
                        l *= alpha;
                        m = top;
                    }
                    again = true;
                }
                if (failed) break;
                tmem_st16(s_addr, pk);
                sum += weigh(1);
                tmem_st16(s_addr + 16, pk);
                l += sum;
                tmem_st_wait();
                tc_fence_before();
                mbar_arrive(&sh.p[i]);
            }
            if (failed) break;
            if (b > a) {
                failed = !__all_sync(0xffffffffu, mbar_wait(&sh.o[i], no & 1, kWaitBudget));
                ++no;
                tc_fence_after();
            }
            float others;
            if (!meet(l, others)) {
                failed = true;
                break;
            }
            named_barrier(1 + pair, 64);  // both have read it before the next job's first tile writes there
            l = half ? others + l : l + others;
            const float inv = whole ? row_inverse(m, l) : 1.f;
            const size_t slot = (size_t)blockIdx.x * 2 + (first ? 1 : 0);
            // the rows of this lane's group of four, each of which the four store together
            long long rows[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) rows[k] = __shfl_sync(0xffffffffu, orow, (lane & ~3) + k);
#pragma unroll
            for (int c = 0; c < D / 64; ++c) {
                uint32_t v[32];
                if (b > a) {
                    tmem_ld32(o_addr + c * 32, v);
                    tmem_ld_wait();
                } else {
#pragma unroll
                    for (int e = 0; e < 32; ++e) v[e] = 0u;
                }
                if (whole) {
                    // 4 lanes' 4 pieces of 8 columns (16 bytes) transposed among them, so that a store's 4 lanes write 64
                    // consecutive bytes of one row: 8 lines a store instead of 32
                    uint32_t w[4][4];
#pragma unroll
                    for (int k = 0; k < 16; ++k)
                        w[k >> 2][k & 3] = pack_bf16x2(__uint_as_float(v[2 * k]) * inv, __uint_as_float(v[2 * k + 1]) * inv);
#pragma unroll
                    for (int o = 1; o < 4; o <<= 1)
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            if (!(k & o)) {
#pragma unroll
                                for (int e = 0; e < 4; ++e) {
                                    const bool up = lane & o;
                                    const uint32_t got = __shfl_xor_sync(0xffffffffu, up ? w[k][e] : w[k | o][e], o);
                                    if (up) w[k][e] = got; else w[k | o][e] = got;
                                }
                            }
#pragma unroll
                    for (int k = 0; k < 4; ++k)  // piece lane & 3 of the row of lane (lane & ~3) + k
                        if (rows[k] >= 0)
                            *reinterpret_cast<uint4*>(p.o + rows[k] * D + half * (D / 2) + c * 32 + (lane & 3) * 8) =
                                make_uint4(w[k][0], w[k][1], w[k][2], w[k][3]);
                } else if (active) {
#pragma unroll
                    for (int e = 0; e < 32; e += 8)
                        st_global_f32x8(p.part_o + part_at<D>(slot, i * kTileM + r, half * (D / 2) + c * 32 + e), reinterpret_cast<const float*>(&v[e]));
                }
                __syncwarp();
            }
            if (active && half == 0) {
                if (!whole) p.part_ml[slot * (2 * kTileM) + i * kTileM + r] = make_float2(m, l);
                else if (p.lse) p.lse[orow] = row_lse(m, l);
            }
            tc_fence_before();
        }
        if (failed && lane == 0) raise_error(p.err, kErrTimeout);
    } else {
        regs_dec<kOtherRegs>();
        if (warp == kProducerWarp) {
            // ================= this CTA's part of the line, laid out in jobs; their queries, then K and V tiles through
            // the ring, K first
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
            Place place[2];
#pragma unroll
            for (int e = 0; e < 2; ++e)
                place[e] = Place{__shfl_sync(0xffffffffu, at.s, e), __shfl_sync(0xffffffffu, at.h, e),
                                 __shfl_sync(0xffffffffu, at.t, e), __shfl_sync(0xffffffffu, at.j, e)};
            Walk walk{p, place[0], place[1], -1, Seq{}, 0};
            unsigned nj = 0;
            bool ok = true;
            // lays out the next job, or the end of them
            auto lay_out = [&](Job& g) {
                if (!walk.next(g)) g.s = -1;
                const int e = nj % kJobs;
                if (nj >= kJobs && !__all_sync(0xffffffffu, mbar_wait(&sh.job_empty[e], ((nj / kJobs) - 1) & 1, kWaitBudget))) {
                    ok = false;
                    return;
                }
                if (lane == 0) {
                    sh.job[e] = g;
                    mbar_arrive(&sh.job_full[e]);
                }
                ++nj;
            };
            const int rows = min(kKeys, 1 << p.page_shift);  // of a box
            const int nbox = kKeys / rows;
            const int box = lane / S::halves, half = lane % S::halves;
            unsigned x = 0;  // ring position
            int nq = 0;
            unsigned on_raw = 0, raw_phase = 0;  // per slot: whether its last use is on raw; that barrier's uses, mod 2
            Job g, after;
            for (bool have = false; ; have = true) {
                lay_out(after);  // one ahead of the copies
                if (!ok) break;
                if (have && g.j1 > g.j0) {
                    const int tok = g.t * 2 * p.tokens;
                    if (nq > 0 && !__all_sync(0xffffffffu, mbar_wait(&sh.q_empty, (nq - 1) & 1, kWaitBudget))) {
                        ok = false;
                        break;
                    }
                    const bool two = tok + p.tokens < g.B;
                    if (lane == 0) {
                        const uint32_t bytes = (uint32_t)(p.tokens * G) * 128 * S::halves;
                        mbar_arrive_expect_tx(&sh.q_full, two ? 2 * bytes : bytes);
#pragma unroll
                        for (int i = 0; i < 2; ++i)
                            if (i == 0 || two)
#pragma unroll
                                for (int hh = 0; hh < S::halves; ++hh)
                                    tma_load_3d(sQ + i * S::tile_bytes + hh * kHalfBytes, &qmap, &sh.q_full, 64 * hh, g.h * G,
                                                g.q0 + tok + i * p.tokens);
                    }
                    ++nq;
                    const int32_t* table = p.block_table + (size_t)g.s * p.pages_per_seq;
                    const int last_page = (g.n - 1) >> p.page_shift;
                    // the pool row of this lane's box of key tile j (-1: past the sequence's last page)
                    auto pool_row = [&](int j) {
                        const int key = j * kKeys + box * rows, pg = key >> p.page_shift;
                        if (box >= nbox || pg > last_page) return -1;
                        int id = pg < p.pages_per_seq ? __ldg(table + pg) : -1;
                        if ((unsigned)id >= (unsigned)p.num_pages) {
                            raise_error(p.err, kErrDeviceArg);
                            id = 0;
                        }
                        return (id << p.page_shift) + (key & ((1 << p.page_shift) - 1));
                    };
                    int row = pool_row(g.j0);
                    for (int j = g.j0; j < g.j1 && ok; ++j) {
                        const int row_next = j + 1 < g.j1 ? pool_row(j + 1) : -1;
                        const int boxes = min(nbox, ((g.n - j * kKeys) + rows - 1) / rows);
#pragma unroll
                        for (int kv = 0; kv < 2; ++kv, ++x) {
                            const int slot = x % S::slots;
                            const unsigned use = x / S::slots;
                            if (use > 0 && !__all_sync(0xffffffffu, mbar_wait(&sh.empty[slot], (use - 1) & 1, kWaitBudget))) {
                                ok = false;
                                break;
                            }
                            // a V tile with rows past the last key goes through the tail warp
                            const bool raw = kv == 1 && (j + 1) * kKeys > g.n;
                            uint64_t* bar = raw ? &sh.raw[slot] : &sh.full[slot];
                            on_raw = raw ? on_raw | 1u << slot : on_raw & ~(1u << slot);
                            if (raw) raw_phase ^= 1u << slot;
                            if (lane == 0) mbar_arrive_expect_tx(bar, (uint32_t)(boxes * rows) * 128 * S::halves);
                            __syncwarp();
                            if (row >= 0)
                                tma_load_3d(sKV + slot * S::tile_bytes + half * kHalfBytes + box * rows * 128, kv ? &vmap : &kmap,
                                            bar, 64 * half, g.h, row);
                        }
                        row = row_next;
                    }
                }
                if (!ok || after.s < 0) break;
                g = after;
            }
            if (!ok && lane == 0) raise_error(p.err, kErrTimeout);
            // no copy may still be in flight when the CTA leaves
            for (unsigned y = x > (unsigned)S::slots ? x - S::slots : 0; y < x; ++y) {
                const int slot = y % S::slots;
                const bool raw = on_raw >> slot & 1;
                if (!mbar_wait(raw ? &sh.raw[slot] : &sh.full[slot], raw ? ~raw_phase >> slot & 1 : (y / S::slots) & 1, kDrainBudget) && lane == 0)
                    raise_error(p.err, kErrTimeout);
            }
            if (nq > 0 && !mbar_wait(&sh.q_full, (nq - 1) & 1, kDrainBudget) && lane == 0) raise_error(p.err, kErrTimeout);
        } else if (warp != kTailWarp) {
            // ================= MMA issuer of stream i.  The streams take turns, a P V and a Q K^T at a time, each from a
            // warp of its own: one waits for its operands and commits while the other's MMAs are issued
            const int i = warp - kMmaWarp;
            const uint32_t id_s = idesc_bf16_f32(kTileM, kKeys, false, false);
            const uint32_t id_o = idesc_bf16_f32(kTileM, D, false, true);
            // descriptors of this stream's Q tile, of the ring's first slot as K and as V: their upper halves are constant,
            // an offset adds its 16-byte units to the lower ones
            const uint64_t upper = smem_desc(0, 0, 1024, kSwizzle128B);
            const uint32_t q_lo = (uint32_t)smem_desc(smem_addr(sQ) + i * S::tile_bytes, 16, 0, 0);
            const uint32_t k_lo = (uint32_t)smem_desc(smem_addr(sKV), 16, 0, 0);
            const uint32_t v_lo = (uint32_t)smem_desc(smem_addr(sKV), kHalfBytes, 0, 0);
            const uint32_t t_s = tmem + i * 128, t_o = tmem + S::col_o + i * D;
            // this stream's arrival on `bar`: when its MMAs so far are done, or at once if it had none there
            auto release = [&](uint64_t* bar, bool used) {
                if (used) umma_commit(bar); else mbar_arrive(bar);
            };
            unsigned x = 0;  // ring position
            unsigned nj = 0, np = 0, turn = 0;
            int nq = 0;
            bool ok, fine = true, any = false;
            while (const Job* g = next_job(nj, ok)) {
                const int a = g->a[i], b = g->b[i], j0 = g->j0, j1 = g->j1, n = g->n;
                had_job(nj);
                if (j1 <= j0) continue;
                if (elect_one()) {  // one thread throughout: its waits need no votes
                    fine = mbar_wait(&sh.q_full, nq & 1, kWaitBudget);
                    unsigned xk = x, my_turn = turn, my_p = np;
                    for (int j = j0; j <= j1 && fine; ++j, ++my_turn, xk += 2) {  // xk: K of tile j
                        const int kslot = xk % S::slots, vslot = (xk - 1) % S::slots;
                        const bool pv = j > a && j <= b, qk = j >= a && j < b;
                        if (j < j1) fine = mbar_wait(&sh.full[kslot], (xk / S::slots) & 1, kWaitBudget);
                        if (fine && j > j0) fine = mbar_wait(&sh.full[vslot], ((xk - 1) / S::slots) & 1, kWaitBudget);
                        if (fine && pv) fine = mbar_wait(&sh.p[i], my_p++ & 1, kWaitBudget);
                        if (fine) fine = mbar_wait(&sh.turn[i], (my_turn & 1) ^ (i ^ 1), kWaitBudget);
                        if (!fine) break;
                        tc_fence_after();
                        // keys past the sequence's last in steps of 16: the tail warp has cleared the rest of a step
                        const int steps = pv ? min(kKeys / 16, (n - (j - 1) * kKeys + 15) / 16) : 0;
                        const uint32_t vl = v_lo + vslot * (S::tile_bytes >> 4), kl = k_lo + kslot * (S::tile_bytes >> 4);
                        uint32_t on = j - 1 > a ? 1u : 0u;
                        // O += P V of tile j - 1 (P's 64-key halves lie 64 columns apart)
                        if (steps == kKeys / 16) {
#pragma unroll
                            for (int kk = 0; kk < kKeys / 16; ++kk) {
                                umma_ts(t_o, t_s + (kk >> 2) * 64 + (kk & 3) * 8, upper | (vl + kk * (2048 >> 4)), id_o, on);
                                on = 1;
                            }
                        } else {
#pragma unroll 1
                            for (int kk = 0; kk < steps; ++kk) {
                                umma_ts(t_o, t_s + (kk >> 2) * 64 + (kk & 3) * 8, upper | (vl + kk * (2048 >> 4)), id_o, on);
                                on = 1;
                            }
                        }
                        if (qk) {  // S = Q K^T of tile j
                            on = 0;
#pragma unroll
                            for (int kk = 0; kk < D / 16; ++kk) {
                                const uint32_t off = ((kk >> 2) * kHalfBytes + (kk & 3) * 32) >> 4;
                                umma_ss(t_s, upper | (q_lo + off), upper | (kl + off), id_s, on);
                                on = 1;
                            }
                        }
                        mbar_arrive(&sh.turn[i ^ 1]);
                        if (qk) umma_commit(&sh.s[i]);
                        if (pv && j == b) umma_commit(&sh.o[i]);
                        if (j > j0) release(&sh.empty[vslot], pv);
                        if (j < j1) release(&sh.empty[kslot], qk);
                        if (j == j1 - 1) release(&sh.q_empty, any || b > a);
                    }
                }
                x += 2 * (j1 - j0);
                turn += j1 - j0 + 1;
                np += max(0, b - a);
                any = any || b > a;
                ++nq;
                fine = __all_sync(0xffffffffu, fine);
                if (!fine) break;
            }
            if ((!fine || !ok) && lane == 0) raise_error(p.err, kErrTimeout);
            if (any && elect_one()) {
                umma_commit(&sh.drain[i]);
                if (!mbar_wait(&sh.drain[i], 0, kDrainBudget)) raise_error(p.err, kErrTimeout);
            }
            __syncwarp();
        } else {
            // ================= V rows past a sequence's last key; what this CTA leaves to the merge
            unsigned x0 = 0, phase = 0, nj = 0;
            int4 left = make_int4(0, 0, 0, 0);
            bool ok, fine = true;
            while (const Job* job = next_job(nj, ok)) {
                const Job g = *job;
                had_job(nj);
                if (!g.first) left.x |= kHasHead | (g.last ? kHeadEnds : 0);
                if (g.first && !g.last)
                    left = make_int4(left.x | kHasTail, g.q0 + g.t * 2 * p.tokens, min(2 * p.tokens, g.B - g.t * 2 * p.tokens), g.h);
                if (g.j1 <= g.j0) continue;
                if (g.j1 * kKeys > g.n) {
                    const unsigned x = x0 + 2 * (g.j1 - 1 - g.j0) + 1;
                    const int slot = x % S::slots;
                    fine = __all_sync(0xffffffffu, mbar_wait(&sh.raw[slot], (phase >> slot) & 1, kWaitBudget));
                    if (!fine) break;
                    phase ^= 1u << slot;
                    const int from = g.n - (g.j1 - 1) * kKeys, to = (from + 15) & ~15;  // the rest of a step of 16 keys
                    for (int c = lane; c < (to - from) * 8 * S::halves; c += 32) {
                        const int r = c % (8 * S::halves);
                        *reinterpret_cast<uint4*>(sKV + slot * S::tile_bytes + (r >> 3) * kHalfBytes +
                                                  (from + c / (8 * S::halves)) * 128 + (r & 7) * 16) = make_uint4(0, 0, 0, 0);
                    }
                    fence_proxy_async_smem();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&sh.full[slot]);
                }
                x0 += 2 * (g.j1 - g.j0);
            }
            if ((!fine || !ok) && lane == 0) raise_error(p.err, kErrTimeout);
            if (lane == 0) p.info[blockIdx.x] = left;
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == kMmaWarp) {
        tc_fence_after();
        tmem_dealloc(tmem, kChunkTmem);
    }
}

// Merges the parts of every work tile that was cut: block (c, y) rows [32 y, 32 y + 32) of the tile that CTA c began and
// did not end.  Its parts are c's last and the first ones of the CTAs behind it, up to the one that ends it.  A warp has a row:
// its lanes take the parts' (m, l), 32 at a time, and weigh them; then 4 columns each, all parts' loads in flight.
// BATCH parts' loads are in flight at once: 4 where tiles have many rows (they are cut once or twice, and the registers are
// better spent on more blocks, 12 bytes spilled among them: 12 loads took 14 us more for a prompt of 8192), 16 where every sequence has one tile (its context
// may be cut for all CTAs: one token over 2048 keys took 18.7 us with 8 of them).
constexpr int kMergeThreads = 512, kMergeRows = 32;
template <int D, int BATCH>
__global__ void __launch_bounds__(kMergeThreads, BATCH <= 4 ? 3 : 1) chunk_merge_kernel(const __grid_constant__ ChunkParams p, int grid) {
    griddep_launch_dependents();
    griddep_wait();
    const int c = blockIdx.x, i = blockIdx.y * kMergeRows / kTileM, r0 = blockIdx.y * kMergeRows % kTileM, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    // this CTA's entry and the 31 behind it, in one round trip
    const int4 near = c + lane < grid ? p.info[c + lane] : make_int4(0, 0, 0, 0);
    if (!(__shfl_sync(0xffffffffu, near.x, 0) & kHasTail)) return;
    const int row0 = __shfl_sync(0xffffffffu, near.y, 0), tokens = __shfl_sync(0xffffffffu, near.z, 0);
    const int head = __shfl_sync(0xffffffffu, near.w, 0);
    const int rows = min(p.tokens, tokens - i * p.tokens) * p.group;  // of this stream
    constexpr int kCols = D / 32;
    for (int r = r0 + warp; r < min(rows, r0 + kMergeRows); r += kMergeThreads / 32) {
        const int row = i * kTileM + r;
        float acc[kCols] = {}, m = -INFINITY, l = 0.f;
        bool more = true;
        for (int base = c; more; base += 32) {  // 32 CTAs at a time
            const int e = base + lane;
            const int flags = base == c ? near.x : e < grid ? p.info[e].x : 0;
            const unsigned ends = __ballot_sync(0xffffffffu, e > c && (flags & kHeadEnds));
            const int n = ends ? __ffs(ends) : min(32, grid - base);  // of them, up to the one that ends the tile
            more = !ends && base + 32 < grid;
            const size_t slot = (size_t)e * 2 + (e == c ? 1 : 0);
            float2 ml = make_float2(-INFINITY, 0.f);
            if (lane < n && (e == c || (flags & kHasHead))) ml = p.part_ml[slot * (2 * kTileM) + row];
            // those in which the row saw a key; a part whose sum is a NaN is one (its maximum may be -inf)
            const unsigned seen = __ballot_sync(0xffffffffu, !saw_no_key(ml.x, ml.y));
            if (!seen) continue;
            float top = ml.x;
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
            const float m_new = fmaxf(m, top);
            const float w_old = m == m_new ? 1.f : chunk_exp2(m - m_new), w = ml.x == m_new ? 1.f : chunk_exp2(ml.x - m_new);
            float sum = ml.y * w;
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
            l = l * w_old + sum;
            m = m_new;
#pragma unroll
            for (int d = 0; d < kCols; ++d) acc[d] *= w_old;
#pragma unroll 1
            for (int k0 = 0; k0 < n; k0 += BATCH) {
                float v[BATCH][kCols];
#pragma unroll
                for (int k = 0; k < BATCH; ++k) {
                    const size_t s = (size_t)(base + k0 + k) * 2 + (base + k0 + k == c ? 1 : 0);
                    const float* o = p.part_o + part_at<D>(s, row, lane * kCols / 8 * 8) + lane * kCols % 8;
                    if (k0 + k >= n) break;
                    if constexpr (kCols == 4) {
                        const float4 t = *reinterpret_cast<const float4*>(o);
                        v[k][0] = t.x; v[k][1] = t.y; v[k][2] = t.z; v[k][3] = t.w;
                    } else {
                        const float2 t = *reinterpret_cast<const float2*>(o);
                        v[k][0] = t.x; v[k][1] = t.y;
                    }
                }
#pragma unroll
                for (int k = 0; k < BATCH; ++k) {
                    if (k0 + k >= n) break;
                    const float wk = __shfl_sync(0xffffffffu, w, k0 + k);
#pragma unroll
                    for (int d = 0; d < kCols; ++d) acc[d] += seen >> (k0 + k) & 1 ? wk * v[k][d] : 0.f;  // (a slot without a part holds anything)
                }
            }
        }
        const float inv = row_inverse(m, l);
        const size_t orow = (size_t)(row0 + i * p.tokens + r / p.group) * p.num_q_heads + head * p.group + r % p.group;
        __nv_bfloat16* out = p.o + orow * D + lane * kCols;
        if constexpr (kCols == 4)
            *reinterpret_cast<uint2*>(out) = make_uint2(pack_bf16x2(acc[0] * inv, acc[1] * inv), pack_bf16x2(acc[2] * inv, acc[3] * inv));
        else
            *reinterpret_cast<uint32_t*>(out) = pack_bf16x2(acc[0] * inv, acc[1] * inv);
        if (p.lse && lane == 0) p.lse[orow] = row_lse(m, l);
    }
}

template <int D>
int run(const ChunkAttentionArgs& a, const DeviceInfo& dev, cudaStream_t stream) {
    using S = Shape<D>;
    ChunkParams p;
    p.o = static_cast<__nv_bfloat16*>(a.o);
    p.lse = a.lse;
    p.cu_q = a.cu_q;
    p.cu_kv = a.cu_kv;
    p.block_table = a.block_table;
    p.num_seqs = a.num_seqs;
    p.total_q = a.total_q;
    p.num_q_heads = a.num_q_heads;
    p.num_kv_heads = a.num_kv_heads;
    p.group = a.num_q_heads / a.num_kv_heads;
    p.tokens = kTileM / p.group;
    p.pages_per_seq = a.pages_per_seq;
    p.page_shift = 0;
    while ((1 << p.page_shift) < a.page_size) ++p.page_shift;
    p.num_pages = a.num_pages;
    p.max_q = a.max_q_len;
    p.max_kv = a.max_kv_len;
    p.causal = a.mask == BP_MASK_CAUSAL_BLOCK;
    p.window = a.window;
    p.scale_log2 = a.scale * 1.4426950408889634f;
    p.err = a.err_word;
    const int grid = std::min(dev.sm_count, kChunkMaxGrid);
    p.grid_inverse = ~0ull / (unsigned)grid;
    uint8_t* at = static_cast<uint8_t*>(a.scratch);
    p.part_o = reinterpret_cast<float*>(at);
    at += (size_t)kChunkMaxGrid * 2 * 2 * kTileM * D * sizeof(float);
    p.part_ml = reinterpret_cast<float2*>(at);
    at += (size_t)kChunkMaxGrid * 2 * 2 * kTileM * sizeof(float2);
    p.info = reinterpret_cast<int4*>(at);

    CUtensorMap qmap, kmap, vmap;
    const cuuint64_t qdims[3] = {(cuuint64_t)D, (cuuint64_t)a.num_q_heads, (cuuint64_t)a.total_q};
    const cuuint64_t qstrides[2] = {(cuuint64_t)D * 2, (cuuint64_t)a.q_stride * 2};
    const cuuint32_t qbox[3] = {64, (cuuint32_t)p.group, (cuuint32_t)p.tokens};
    int rc = encode_tensor_map(&qmap, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(a.q), qdims, qstrides, qbox,
                               CU_TENSOR_MAP_SWIZZLE_128B);
    if (rc != BP_OK) return rc;
    const cuuint64_t dims[3] = {(cuuint64_t)D, (cuuint64_t)a.num_kv_heads, (cuuint64_t)a.num_pages * a.page_size};
    const cuuint64_t strides[2] = {(cuuint64_t)D * 2, (cuuint64_t)a.num_kv_heads * D * 2};
    const cuuint32_t box[3] = {64, 1, (cuuint32_t)std::min(a.page_size, kKeys)};
    rc = encode_tensor_map(&kmap, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(a.k_cache), dims, strides, box,
                           CU_TENSOR_MAP_SWIZZLE_128B);
    if (rc != BP_OK) return rc;
    rc = encode_tensor_map(&vmap, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(a.v_cache), dims, strides, box,
                           CU_TENSOR_MAP_SWIZZLE_128B);
    if (rc != BP_OK) return rc;

    static std::mutex mu;
    static bool configured[64] = {};
    if (dev.device < 0 || dev.device >= 64) return BP_ERR_UNSUPPORTED;
    {
        std::lock_guard<std::mutex> lock(mu);
        if (!configured[dev.device]) {
            if (cudaFuncSetAttribute(chunk_attention_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, chunk_smem<D>()) != cudaSuccess)
                return BP_ERR_CUDA;
            configured[dev.device] = true;
        }
    }
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.gridDim = dim3((unsigned)grid, 1, 1);
    cfg.blockDim = dim3(kChunkThreads, 1, 1);
    cfg.dynamicSmemBytes = chunk_smem<D>();
    cfg.stream = stream;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, chunk_attention_kernel<D>, p, qmap, kmap, vmap) != cudaSuccess) return BP_ERR_CUDA;
    if (a.max_kv_len <= (2 * kLeastCut - 1) * kKeys) return BP_OK;  // too short to be cut: nothing to merge
    // (rows behind the first stream's only where some sequence may have them)
    const bool few = a.max_q_len <= p.tokens;
    const int merge_rows = few ? a.max_q_len * p.group : 2 * kTileM;
    cfg.gridDim = dim3((unsigned)grid, (unsigned)((merge_rows + kMergeRows - 1) / kMergeRows), 1);
    cfg.blockDim = dim3(kMergeThreads, 1, 1);
    cfg.dynamicSmemBytes = 0;
    const cudaError_t e = few ? cudaLaunchKernelEx(&cfg, chunk_merge_kernel<D, 16>, p, grid)
                              : cudaLaunchKernelEx(&cfg, chunk_merge_kernel<D, 4>, p, grid);
    return e == cudaSuccess ? BP_OK : BP_ERR_CUDA;
}

}  // namespace

size_t chunk_attention_scratch_bytes(int head_dim) {
    return (size_t)kChunkMaxGrid * (2 * 2 * kTileM * ((size_t)head_dim * sizeof(float) + sizeof(float2)) + sizeof(int4));
}

int launch_chunk_attention(const ChunkAttentionArgs& a, const DeviceInfo& dev, cudaStream_t stream) {
    return a.head_dim == 128 ? run<128>(a, dev, stream) : run<64>(a, dev, stream);
}

}  // namespace bp
