// Attention of chunks of new tokens over a paged KV cache in 8 bits: chunk_attention.cu's operation over keys and values held
// as e4m3 codes with a power of two for each page and KV head,
//
//   O_i = sum_j softmax_j(scale <q_i, 2^a k_j>) 2^b v_j      a, b: of key j's page
//
// Nothing is rounded that a bf16 cache would not round:
//   * S = Q K^T on the codes as they lie in memory, kind::f8f6f4.  A query row, scaled by a power of two to at most 256, is the
//     sum of two e4m3 numbers, its nearest and what is left: bf16's 8 bits are twice 4.  (Elements below 2^-10 of the row's
//     largest lose bits under 2^-18 of it.)  The row's and the page's powers multiply the scores in the softmax.
//   * P V in bf16: e4m3 times a power of two is a bf16 number.  Four warps turn a tile's codes into them, in shared memory.
// The rest is as there: the line of work, two streams of a query tile each, the softmax's two threads a row, the merge.  Where
// a work tile has the rows of one stream only (blocks, decoding), both streams take its queries and every other key tile,
// and add what they have at the end: a stream alone is a chain of latencies.
//
// Roles: warps 0-7 and 8-15 softmax of stream 0 and 1 (they read and split the queries too), warp 16 lays out the jobs and
// issues the TMA copies, 17 and 18 issue the streams' MMAs, 19 notes what the merge has to do, 20-23 convert V.
#include <cuda_bf16.h>

#include <algorithm>
#include <mutex>

#include "chunk_plan.cuh"

namespace bp {
namespace {

constexpr int kHalfBytes = kKeys * 128;          // 128 rows of 64 bf16 columns (or of 128 codes), 128-byte swizzle
constexpr int kSoftmaxWarps = 16;                // two threads a row, 64 keys each
constexpr int kProducerWarp = 16, kMmaWarp = 17, kConvertWarp = 20;  // (a stream's MMA warp: kMmaWarp + stream)
constexpr int kConvertWarps = 4;                 // 32 keys of a tile each
constexpr int kFp8Threads = 32 * 24;
// Registers: 80 a thread at launch (768 x 80); 512 x 88 + 256 x 64 are as many.
constexpr int kSoftmaxRegs = 88, kOtherRegs = 64;
constexpr uint32_t kChunkTmem = 512;
constexpr int kJobs = 4;                         // jobs laid out ahead

template <int D>
struct Shape {
    static constexpr int code_bytes = kKeys * D;                // one K or V tile of codes
    static constexpr int v_bytes = 2 * code_bytes;              // one V tile in bf16
    static constexpr int q_bytes = 2 * code_bytes;              // one query tile, both parts
    static constexpr int k_slots = D == 128 ? 3 : 8;
    static constexpr int raw_slots = D == 128 ? 3 : 7;          // V's codes
    static constexpr int v_slots = D == 128 ? 2 : 4;
    static constexpr int notes = D == 128 ? 8 : 16;             // of key tiles: more than can be under way at once
    static constexpr int at_k = 2 * q_bytes;
    static constexpr int at_raw = at_k + k_slots * code_bytes;
    static constexpr int at_v = at_raw + raw_slots * code_bytes;
    static constexpr int tiles = at_v + v_slots * v_bytes;
    static constexpr uint32_t col_o = 256;                      // O of stream i: columns col_o + i * D
};
static_assert(Shape<128>::tiles >= tmem_smem_share((int)kChunkTmem, 228 * 1024) &&
                  Shape<64>::tiles >= tmem_smem_share((int)kChunkTmem, 228 * 1024),
              "leaves no other CTA's tensor memory room");

struct Fp8Params {
    ChunkParams c;
    const __nv_bfloat16* q;
    int64_t q_stride;
    const uint8_t* k_scale;
    const uint8_t* v_scale;
};

// Shared memory behind the tiles.
template <int D>
struct Shared {
    using S = Shape<D>;
    uint64_t k_full[S::k_slots], k_empty[S::k_slots], raw_full[S::raw_slots], raw_empty[S::raw_slots];
    uint64_t v_full[S::v_slots], v_empty[S::v_slots];
    uint64_t q_ready[2], drain[2], turn[2];
    uint64_t s[2], p[2], o[2];                       // of a stream: scores, weights, the accumulator
    uint64_t job_full[kJobs], job_empty[kJobs];
    uint2 nan_keys[S::notes][2];                     // of a key tile's halves: keys of which a value is none
    uint8_t k_exp[S::notes][8], v_exp[S::raw_slots][8];  // the scales of a tile's boxes
    Job job[kJobs];
    uint32_t tmem;
    int pair_failed[8];
    float row[2][2][kTileM];                         // [stream][half]: row maxima, at the end row sums
};
template <int D>
constexpr int fp8_smem() { return Shape<D>::tiles + (int)sizeof(Shared<D>); }
static_assert(fp8_smem<128>() <= 227 * 1024 && fp8_smem<64>() <= 227 * 1024, "a block's shared memory");

// 2^(e - 127) of a biased exponent below 255.
__device__ __forceinline__ float power_of(uint32_t e) { return __uint_as_float(e ? e << 23 : 0x400000u); }

template <int D>
__global__ void __launch_bounds__(kFp8Threads, 1)
chunk_attention_fp8_kernel(const __grid_constant__ Fp8Params fp, const __grid_constant__ CUtensorMap kmap,
                           const __grid_constant__ CUtensorMap vmap) {
    using S = Shape<D>;
    const ChunkParams& p = fp.c;
    extern __shared__ __align__(1024) uint8_t smem[];
    Shared<D>& sh = *reinterpret_cast<Shared<D>*>(smem + S::tiles);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int G = p.group;
    if (smem_addr(smem) & 1023) {  // (the swizzled tiles' alignment: dynamic shared memory starts on such a boundary)
        if (tid == 0) raise_error(p.err, kErrDeviceArg);
        return;
    }

    if (tid < 8) sh.pair_failed[tid] = 0;
    if (tid == 0) {
        for (int i = 0; i < S::k_slots; ++i) {
            mbar_init(&sh.k_full[i], 1);
            mbar_init(&sh.k_empty[i], 2);
        }
        for (int i = 0; i < S::raw_slots; ++i) {
            mbar_init(&sh.raw_full[i], 1);
            mbar_init(&sh.raw_empty[i], kConvertWarps);
        }
        for (int i = 0; i < S::v_slots; ++i) {
            mbar_init(&sh.v_full[i], kConvertWarps);
            mbar_init(&sh.v_empty[i], 2);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&sh.q_ready[i], 256);
            mbar_init(&sh.s[i], 1);
            mbar_init(&sh.p[i], 256);
            mbar_init(&sh.o[i], 1);
            mbar_init(&sh.drain[i], 1);
            mbar_init(&sh.turn[i], 1);
        }
        for (int i = 0; i < kJobs; ++i) {
            mbar_init(&sh.job_full[i], 1);
            mbar_init(&sh.job_empty[i], kSoftmaxWarps + 3 + kConvertWarps);
        }
        fence_mbar_init();
    }
    if (warp == kMmaWarp) {
        tmem_alloc(&sh.tmem, kChunkTmem);
        tmem_relinquish();
    }
    if (warp == kProducerWarp && lane < 2) prefetch_tensormap(lane == 0 ? &kmap : &vmap);
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
    // whether a job's rows are one stream's: then both take them, and every other key tile
    auto is_split = [&](const Job& g) { return g.t * 2 * p.tokens + p.tokens >= g.B; };

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
        const int box_shift = min(7, p.page_shift);
        unsigned ns = 0, no = 0, x0 = 0;  // scores and accumulators waited for; key tiles of the jobs before
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
            bool ok = false;
            const Job* g = failed ? nullptr : next_job(nj, ok);
            // (a warp that gave up a wait takes the three others of its rows along, here and at a split job's end)
            if (named_barrier_or(9 + quad, 128, !ok)) {
                failed = true;
                break;
            }
            if (!g) break;
            const bool split = is_split(*g);
            const int mine = split ? 0 : i;  // the query tile
            const int a = g->a[mine], b = g->b[mine], j0 = g->j0, j1 = g->j1;
            const int tok = g->t * 2 * p.tokens + mine * p.tokens + my_tok;
            const bool active = my_tok < p.tokens && tok < g->B;
            const int pos = g->n - g->B + tok;
            // (rows of none count as seeing all: their warps' tiles are not masked for their sake)
            const int hi = !active ? 0x7fffffff : p.causal ? max(0, pos + 1) : g->n;
            const int lo = active && p.window > 0 ? max(0, pos + 1 - p.window) : 0;
            const bool first = g->first, whole = first && g->last;
            // the query row's number among all, in the output (-1: none)
            const long long orow = active ? (long long)(g->q0 + tok) * p.num_q_heads + g->h * G + my_head : -1;
            const __nv_bfloat16* q = fp.q + (int64_t)(g->q0 + tok) * fp.q_stride + (g->h * G + my_head) * D + half * (D / 2);
            had_job(nj);
            const bool idle = !__any_sync(0xffffffffu, active);  // the same in all four warps of these rows
            float row_scale = 1.f;
            if (j1 > j0 && b > a && !idle) {
                // ---- this row's half of the queries: its scale, and its two parts to shared memory
                uint32_t w[D / 4];
#pragma unroll
                for (int k = 0; k < D / 16; ++k) {
                    const uint4 v = active ? __ldg(reinterpret_cast<const uint4*>(q) + k) : make_uint4(0, 0, 0, 0);
                    w[4 * k] = v.x; w[4 * k + 1] = v.y; w[4 * k + 2] = v.z; w[4 * k + 3] = v.w;
                }
                uint32_t top = 0;
#pragma unroll
                for (int k = 0; k < D / 4; ++k) top = max(top, max(w[k] & 0x7fffu, w[k] >> 16 & 0x7fffu));
                float theirs;
                meet(__uint_as_float(top), theirs);
                named_barrier(1 + pair, 64);
                top = max(top, __float_as_uint(theirs));
                // the row times 2^(7 - e) is below 256; 2^(e - 7) of it is put back with the softmax's scale
                const int e = max((int)(top >> 7), 8) - 127;
                row_scale = p.scale_log2 * __uint_as_float((uint32_t)(e - 7 + 127) << 23);
                if (top >= 0x7f80u && hi > lo) row_scale = __uint_as_float(0x7fc00000u);  // a NaN or an infinity: the row is none
                if (mine == i) {
                    const float up = __uint_as_float((uint32_t)(7 - e + 127) << 23);
                    uint8_t* const tile = smem + i * S::q_bytes + r * 128;
#pragma unroll
                    for (int k = 0; k < D / 32; ++k) {
                        uint32_t near[4], rest[4];
#pragma unroll
                        for (int c = 0; c < 4; ++c) {
                            uint32_t n2[2], r2[2];
#pragma unroll
                            for (int d = 0; d < 2; ++d) {
                                const uint32_t v = w[8 * k + 2 * c + d];
                                const float x = __uint_as_float(v << 16) * up, y = __uint_as_float(v & 0xffff0000u) * up;
                                float xn, yn;
                                n2[d] = pack_e4m3x2(x, y);
                                unpack_e4m3x2(n2[d], xn, yn);
                                r2[d] = pack_e4m3x2(x - xn, y - yn);
                            }
                            near[c] = n2[0] | n2[1] << 16;
                            rest[c] = r2[0] | r2[1] << 16;
                        }
                        // 16 bytes of either part; with 64 columns both lie in one row of 128 bytes
                        const int piece = half * (D / 32) + k, other = D == 128 ? piece : piece + 4;
                        *reinterpret_cast<uint4*>(tile + ((piece ^ (r & 7)) << 4)) = make_uint4(near[0], near[1], near[2], near[3]);
                        *reinterpret_cast<uint4*>(tile + (D == 128 ? kHalfBytes : 0) + ((other ^ (r & 7)) << 4)) =
                            make_uint4(rest[0], rest[1], rest[2], rest[3]);
                    }
                }
            }
            if (j1 > j0 && mine == i) {
                fence_proxy_async_smem();
                mbar_arrive(&sh.q_ready[i]);
            }
            float m = -INFINITY, l = 0.f;
            const int step = split ? 2 : 1, from_j = split ? a + i : a;  // (a split job's a is its j0)
            int last = -1;  // the key tile before
            // a value that is none, in a key that the row sees, makes the row none (the tiles' weights of it are 0, and
            // its values too); what a tile has of them is there when the scores of the stream's next one are
            auto see_nans = [&]() {
                const uint2 bad = sh.nan_keys[(x0 + last - j0) % S::notes][half];
                if (bad.x | bad.y) {
                    const int from = max(0, lo - last * kKeys - half * 64), to = min(64, hi - last * kKeys - half * 64);
                    if (to > from && ((uint64_t)bad.y << 32 | bad.x) & (~0ull >> (64 - (to - from)) << from))
                        l = __uint_as_float(0x7fc00000u);
                }
            };
            for (int j = from_j; j < b; j += step, ++ns) {
                failed = !__all_sync(0xffffffffu, mbar_wait(&sh.s[i], ns & 1, kWaitBudget));
                tc_fence_after();
                if (idle) {
                    if (failed) break;
                    tc_fence_before();
                    mbar_arrive(&sh.p[i]);
                    continue;
                }
                if (last >= 0) see_nans();
                last = j;
                const int from = lo - j * kKeys - half * 64, to = hi - j * kKeys - half * 64;  // visible columns
                const bool full = __all_sync(0xffffffffu, from <= 0 && to >= 64);
                // the factors of the scores, of 16 keys each (pages of 16 are the smallest); finite and above 0, so that a
                // hidden column's -inf stays one
                float f[4];
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    f[c] = row_scale * power_of(sh.k_exp[(x0 + j - j0) % S::notes][(half * 64 + c * 16) >> box_shift]);
                    if (f[c] < 1.2e-38f) f[c] = 1.2e-38f;
                    if (f[c] > 3.4e38f) f[c] = 3.4e38f;
                }
                uint32_t x[4][16];
                float mine_top;
                {
                    float mx[4];
                    if (full) {
#pragma unroll
                        for (int c = 0; c < 4; ++c) tmem_ld16_max(s_addr + c * 16, x[c], mx[c]);
                        tmem_ld_wait();
                    } else {
#pragma unroll
                        for (int c = 0; c < 4; ++c) tmem_ld16(s_addr + c * 16, x[c]);
                        tmem_ld_wait();
#pragma unroll
                        for (int c = 0; c < 4; ++c) {
                            mx[c] = -INFINITY;
#pragma unroll
                            for (int e = 0; e < 16; ++e) {
                                if (c * 16 + e < from || c * 16 + e >= to) x[c][e] = 0xff800000u;  // -inf
                                mx[c] = fmaxf(mx[c], __uint_as_float(x[c][e]));
                            }
                        }
                    }
                    mine_top = fmaxf(fmaxf(mx[0] * f[0], mx[1] * f[1]), fmaxf(mx[2] * f[2], mx[3] * f[3]));
                }
                // weights 2^(f * score - m) of columns [32 c, 32 c + 32), as packed pairs; their sum
                uint32_t pk[16];
                auto weigh = [&](int c) {
                    const float negm = m == -INFINITY ? 0.f : -m;
                    const uint64_t negm2 = pack_f32x2(negm, negm);
                    uint64_t sum2[2] = {0ull, 0ull};
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const int g16 = 2 * c + (e >> 3);
                        const uint64_t f2 = pack_f32x2(f[g16], f[g16]);
                        float u, w;
                        unpack_f32x2(fma_f32x2(pack_f32x2(__uint_as_float(x[g16][2 * (e & 7)]), __uint_as_float(x[g16][2 * (e & 7) + 1])), f2, negm2), u, w);
                        u = chunk_exp2(u);
                        w = chunk_exp2(w);
                        sum2[e & 1] = add_f32x2(sum2[e & 1], pack_f32x2(u, w));
                        pk[e] = pack_bf16x2(u, w);  // bf16, as the converted values are
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
                    if (!named_barrier_or(1 + pair, 64, failed || mine_top > m + 8.f)) break;
                    float theirs;
                    if (!meet(mine_top, theirs)) {
                        failed = true;
                        break;
                    }
                    const float top = fmaxf(mine_top, theirs);
                    const bool grew = top > m + 8.f;
                    const float alpha = grew ? chunk_exp2(m - top) : 1.f;
                    // (this tile's scores are complete, so the stream's MMAs before them, the last P V among them, are too)
                    if (__any_sync(0xffffffffu, grew && m != -INFINITY)) {
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
            const bool some = from_j < b;  // this stream had a tile
            if (!failed && some) {
                failed = !__all_sync(0xffffffffu, mbar_wait(&sh.o[i], no & 1, kWaitBudget));
                ++no;
                tc_fence_after();
                if (last >= 0) see_nans();
            }
            x0 += j1 - j0;
            float others;
            if (!meet(l, others)) failed = true;
            named_barrier(1 + pair, 64);  // both have read it before it is written again
            l = half ? others + l : l + others;
            if (!split && failed) continue;
            float w_mine = 1.f, w_other = 0.f;  // the weights of the streams' accumulators
            bool others_some = false;
            if (split) {
                // ---- the other stream's part of these rows, merged as the second kernel merges CTAs' parts
                sh.row[i][half][r] = half ? l : m;
                if (named_barrier_or(9 + quad, 128, failed)) {
                    failed = true;
                    continue;
                }
                others_some = a + (i ^ 1) < b;
                const float m2 = sh.row[i ^ 1][0][r], l2 = sh.row[i ^ 1][1][r], top = fmaxf(m, m2);
                const float u = m == top ? 1.f : chunk_exp2(m - top), v = m2 == top ? 1.f : chunk_exp2(m2 - top);
                l = i == 0 ? l * u + l2 * v : l2 * v + l * u;
                m = top;
                w_mine = u;
                w_other = v;
            }
            const float inv = whole ? row_inverse(m, l) : 1.f;
            w_mine *= inv;
            w_other *= inv;
            const size_t slot = (size_t)blockIdx.x * 2 + (first ? 1 : 0);
            // the rows of this lane's pair, both of which the two store together
            const long long rows[2] = {__shfl_sync(0xffffffffu, orow, lane & ~1), __shfl_sync(0xffffffffu, orow, lane | 1)};
            // a split job's four warps have D / 4 columns of the rows each, else a stream's D / 2
            const int col0 = split ? (2 * i + half) * (D / 4) : half * (D / 2), cols = split ? D / 4 : D / 2;
            if (!idle) {
#pragma unroll 1
                for (int col = col0; col < col0 + cols; col += 16) {
                    uint32_t v[16];
                    if (some) {
                        tmem_ld16(lanes + S::col_o + i * D + col, v);
                        tmem_ld_wait();
                    }
#pragma unroll
                    for (int e = 0; e < 16; ++e) v[e] = some ? __float_as_uint(__uint_as_float(v[e]) * w_mine) : 0u;
                    if (others_some) {
                        uint32_t t[16];
                        tmem_ld16(lanes + S::col_o + (i ^ 1) * D + col, t);
                        tmem_ld_wait();
#pragma unroll
                        for (int e = 0; e < 16; ++e) v[e] = __float_as_uint(fmaf(__uint_as_float(t[e]), w_other, __uint_as_float(v[e])));
                    }
                    if (whole) {
                        // two lanes' pieces of 8 columns (16 bytes) exchanged, so that they write 32 consecutive bytes of a row
                        uint32_t w[2][4];
#pragma unroll
                        for (int k = 0; k < 8; ++k) w[k >> 2][k & 3] = pack_bf16x2(__uint_as_float(v[2 * k]), __uint_as_float(v[2 * k + 1]));
                        const bool up = lane & 1;
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const uint32_t got = __shfl_xor_sync(0xffffffffu, up ? w[0][e] : w[1][e], 1);
                            if (up) w[0][e] = got; else w[1][e] = got;
                        }
#pragma unroll
                        for (int k = 0; k < 2; ++k)  // piece lane & 1 of the row of lane (lane & ~1) + k
                            if (rows[k] >= 0)
                                *reinterpret_cast<uint4*>(p.o + rows[k] * D + col + (lane & 1) * 8) = make_uint4(w[k][0], w[k][1], w[k][2], w[k][3]);
                    } else if (active) {
#pragma unroll
                        for (int e = 0; e < 16; e += 8)
                            st_global_f32x8(p.part_o + part_at<D>(slot, mine * kTileM + r, col + e), reinterpret_cast<const float*>(&v[e]));
                    }
                    __syncwarp();
                }
            }
            if (active && half == 0 && (!split || i == 0)) {
                if (!whole) p.part_ml[slot * (2 * kTileM) + mine * kTileM + r] = make_float2(m, l);
                else if (p.lse) p.lse[orow] = row_lse(m, l);
            }
            tc_fence_before();
        }
        if (failed && lane == 0) raise_error(p.err, kErrTimeout);
    } else {
        regs_dec<kOtherRegs>();
        if (warp == kProducerWarp) {
            // ================= this CTA's part of the line, laid out in jobs; K and V tiles of codes through their rings
            Place place[2];
            find_places(p, lane, place);
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
            const int nbox = kKeys / rows;                   // (at most 8, one a lane)
            unsigned x = 0, xv = 0;  // K and V tiles asked for
            Job g, after;
            for (bool have = false; ; have = true) {
                lay_out(after);  // one ahead of the copies
                if (!ok) break;
                if (have && g.j1 > g.j0) {
                    const int32_t* table = p.block_table + (size_t)g.s * p.pages_per_seq;
                    const int last_page = (g.n - 1) >> p.page_shift;
                    // the page of this lane's box of key tile j (-1: past the sequence's last page)
                    auto page_of = [&](int j) {
                        const int pg = (j * kKeys + lane * rows) >> p.page_shift;
                        if (lane >= nbox || pg > last_page) return -1;
                        int id = pg < p.pages_per_seq ? __ldg(table + pg) : -1;
                        if ((unsigned)id >= (unsigned)p.num_pages) {
                            raise_error(p.err, kErrDeviceArg);
                            id = 0;
                        }
                        return id;
                    };
                    auto scale_of = [&](const uint8_t* scale, int id) {
                        return id < 0 ? 127u : (uint32_t)__ldg(scale + (size_t)id * p.num_kv_heads + g.h);
                    };
                    int id = page_of(g.j0);
                    uint32_t ke = scale_of(fp.k_scale, id), ve = scale_of(fp.v_scale, id);
                    for (int j = g.j0; j < g.j1; ++j) {
                        const int id_next = j + 1 < g.j1 ? page_of(j + 1) : -1;
                        if (ke == 255 || ve == 255) {
                            raise_error(p.err, kErrDeviceArg);
                            ke = min(ke, 254u), ve = min(ve, 254u);
                        }
                        const int row = (id << p.page_shift) + ((j * kKeys + lane * rows) & ((1 << p.page_shift) - 1));
                        const int boxes = min(nbox, ((g.n - j * kKeys) + rows - 1) / rows);
                        const uint32_t bytes = (uint32_t)(boxes * rows) * D;
                        const int ks = x % S::k_slots, vs = xv % S::raw_slots;
                        const unsigned ku = x / S::k_slots, vu = xv / S::raw_slots;
                        if (ku > 0 && !__all_sync(0xffffffffu, mbar_wait(&sh.k_empty[ks], (ku - 1) & 1, kWaitBudget))) {
                            ok = false;
                            break;
                        }
                        if (lane < nbox) sh.k_exp[x % S::notes][lane] = (uint8_t)ke;
                        __syncwarp();
                        if (lane == 0) mbar_arrive_expect_tx(&sh.k_full[ks], bytes);
                        __syncwarp();
                        if (id >= 0) tma_load_3d(smem + S::at_k + ks * S::code_bytes + lane * rows * D, &kmap, &sh.k_full[ks], 0, g.h, row);
                        ++x;
                        if (vu > 0 && !__all_sync(0xffffffffu, mbar_wait(&sh.raw_empty[vs], (vu - 1) & 1, kWaitBudget))) {
                            ok = false;
                            break;
                        }
                        if (lane < nbox) sh.v_exp[vs][lane] = (uint8_t)ve;
                        __syncwarp();
                        if (lane == 0) mbar_arrive_expect_tx(&sh.raw_full[vs], bytes);
                        __syncwarp();
                        if (id >= 0) tma_load_3d(smem + S::at_raw + vs * S::code_bytes + lane * rows * D, &vmap, &sh.raw_full[vs], 0, g.h, row);
                        ++xv;
                        id = id_next;
                        ke = scale_of(fp.k_scale, id);
                        ve = scale_of(fp.v_scale, id);
                    }
                }
                if (!ok || after.s < 0) break;
                g = after;
            }
            if (!ok && lane == 0) raise_error(p.err, kErrTimeout);
            // no copy may still be in flight when the CTA leaves
            for (unsigned y = x > (unsigned)S::k_slots ? x - S::k_slots : 0; y < x; ++y)
                if (!mbar_wait(&sh.k_full[y % S::k_slots], (y / S::k_slots) & 1, kDrainBudget) && lane == 0) raise_error(p.err, kErrTimeout);
            for (unsigned y = xv > (unsigned)S::raw_slots ? xv - S::raw_slots : 0; y < xv; ++y)
                if (!mbar_wait(&sh.raw_full[y % S::raw_slots], (y / S::raw_slots) & 1, kDrainBudget) && lane == 0) raise_error(p.err, kErrTimeout);
        } else if (warp == kMmaWarp || warp == kMmaWarp + 1) {
            // ================= MMA issuer of stream i.  The streams take turns, a P V and a Q K^T at a time, each from a
            // warp of its own: one waits for its operands and commits while the other's MMAs are issued
            const int i = warp - kMmaWarp;
            const uint32_t id_s = idesc_e4m3_f32(kTileM, kKeys);
            const uint32_t id_o = idesc_bf16_f32(kTileM, D, false, true);
            // descriptors of the query tiles, of the rings' first slots as K and as V: their upper halves are constant,
            // an offset adds its 16-byte units to the lower ones
            const uint64_t upper = smem_desc(0, 0, 1024, kSwizzle128B);
            const uint64_t k_upper = D == 128 ? upper : smem_desc(0, 0, 512, kSwizzle64B);
            const uint32_t q_lo = (uint32_t)smem_desc(smem_addr(smem), 16, 0, 0);
            const uint32_t k_lo = (uint32_t)smem_desc(smem_addr(smem + S::at_k), 16, 0, 0);
            const uint32_t v_lo = (uint32_t)smem_desc(smem_addr(smem + S::at_v), kHalfBytes, 0, 0);
            const uint32_t t_s = tmem + i * 128, t_o = tmem + S::col_o + i * D;
            // this stream's arrivals on `bar`: when its MMAs so far are done, or at once if it had none there; a split job's
            // tiles are one stream's, which arrives for the other one too
            auto release = [&](uint64_t* bar, bool used, bool both) {
                if (both) mbar_arrive(bar);
                if (used) umma_commit(bar); else mbar_arrive(bar);
            };
            unsigned x = 0;  // key tiles of the jobs before
            unsigned nj = 0, np = 0, turn = 0, nq0 = 0, nq1 = 0;
            bool ok, fine = true, any = false;
            while (const Job* g = next_job(nj, ok)) {
                const bool split = is_split(*g);
                const int mine = split ? 0 : i;
                const int a = g->a[mine], b = g->b[mine], j0 = g->j0, j1 = g->j1;
                had_job(nj);
                if (j1 <= j0) continue;
                const int step = split ? 2 : 1, f = split ? j0 + i : j0;
                const int turns = (split ? (j1 - j0 + 1) / 2 : j1 - j0) + 1;
                // this stream's own tiles: first, first + step, ... below b (a split job's a is its j0)
                const int first = split ? f : a;
                const int own = b > first ? (b - first + step - 1) / step : 0, last = first + (own - 1) * step;
                if (elect_one()) {  // one thread throughout: its waits need no votes
                    fine = mbar_wait(&sh.q_ready[0], nq0 & 1, kWaitBudget);
                    if (fine && mine == 1) fine = mbar_wait(&sh.q_ready[1], nq1 & 1, kWaitBudget);
                    unsigned my_p = np;
                    const uint32_t ql = q_lo + mine * (S::q_bytes >> 4);
                    for (int k = 0; k < turns && fine; ++k) {
                        const int j = f + k * step, jp = j - step;
                        const unsigned xk = x + (j - j0), xv = x + (jp - j0);
                        const int kslot = xk % S::k_slots, vslot = xv % S::v_slots;
                        const bool pv = own && jp >= first && jp <= last, qk = own && j >= first && j <= last;
                        const bool has_k = j < j1, has_v = k > 0 && jp < j1;
                        if (has_k) fine = mbar_wait(&sh.k_full[kslot], (xk / S::k_slots) & 1, kWaitBudget);
                        if (fine && has_v) fine = mbar_wait(&sh.v_full[vslot], (xv / S::v_slots) & 1, kWaitBudget);
                        if (fine && pv) fine = mbar_wait(&sh.p[i], my_p++ & 1, kWaitBudget);
                        if (fine) fine = mbar_wait(&sh.turn[i], ((turn + k) & 1) ^ (i ^ 1), kWaitBudget);
                        if (!fine) break;
                        tc_fence_after();
                        if (pv) {  // O += P V of tile jp (P's 64-key halves lie 64 columns apart)
                            const uint32_t vl = v_lo + vslot * (S::v_bytes >> 4);
                            uint32_t on = jp > first ? 1u : 0u;
#pragma unroll
                            for (int kk = 0; kk < kKeys / 16; ++kk) {
                                umma_ts(t_o, t_s + (kk >> 2) * 64 + (kk & 3) * 8, upper | (vl + kk * (2048 >> 4)), id_o, on);
                                on = 1;
                            }
                        }
                        if (qk) {  // S = Q K^T of tile j: both parts of Q, 32 columns at a time
                            const uint32_t kl = k_lo + kslot * (S::code_bytes >> 4);
                            uint32_t on = 0;
#pragma unroll
                            for (int kk = 0; kk < D / 16; ++kk) {
                                const int part = kk / (D / 32), c = kk % (D / 32);
                                const uint32_t off = ((D == 128 ? part * kHalfBytes : part * 64) + c * 32) >> 4;
                                umma_ss_f8(t_s, upper | (ql + off), k_upper | (kl + c * 2), id_s, on);
                                on = 1;
                            }
                        }
                        mbar_arrive(&sh.turn[i ^ 1]);
                        if (qk) umma_commit(&sh.s[i]);
                        if (pv && jp == last) umma_commit(&sh.o[i]);
                        if (has_v) release(&sh.v_empty[vslot], pv, split);
                        if (has_k) release(&sh.k_empty[kslot], qk, split);
                    }
                }
                x += j1 - j0;
                turn += turns;
                np += own;
                any = any || own > 0;
                ++nq0;
                if (!split) ++nq1;
                fine = __all_sync(0xffffffffu, fine);
                if (!fine) break;
            }
            if ((!fine || !ok) && lane == 0) raise_error(p.err, kErrTimeout);
            if (any && elect_one()) {
                umma_commit(&sh.drain[i]);
                if (!mbar_wait(&sh.drain[i], 0, kDrainBudget)) raise_error(p.err, kErrTimeout);
            }
            __syncwarp();
        } else if (warp >= kConvertWarp) {
            // ================= V from codes to bf16: keys [32 w, 32 w + 32) of every tile
            const int w = warp - kConvertWarp, quarter = lane >> 3, e = lane & 7;
            const int box_shift = min(7, p.page_shift);
            unsigned x = 0, nj = 0;
            bool ok, fine = true;
            while (const Job* g = next_job(nj, ok)) {
                const int j0 = g->j0, j1 = g->j1, n = g->n;
                had_job(nj);
                for (int j = j0; j < j1; ++j, ++x) {
                    const int rs = x % S::raw_slots, vs = x % S::v_slots;
                    fine = mbar_wait(&sh.raw_full[rs], (x / S::raw_slots) & 1, kWaitBudget);
                    if (fine && x >= (unsigned)S::v_slots) fine = mbar_wait(&sh.v_empty[vs], (x / S::v_slots - 1) & 1, kWaitBudget);
                    fine = __all_sync(0xffffffffu, fine);
                    if (!fine) break;
                    const uint8_t* raw = smem + S::at_raw + rs * S::code_bytes;
                    uint8_t* out = smem + S::at_v + vs * S::v_bytes;
                    const int left = n - j * kKeys;  // keys from this one on are none: zeros
                    uint32_t bad = 0;                // keys of this warp's with a code that is none
                    // Eight lanes read all banks, and write them: a key's lower pieces of 16 codes with the next key's upper
                    // ones (of 64 columns: the two keys' pieces all together), then the other way round.
#pragma unroll
                    for (int it = 0; it < D / 16; ++it) {
                        const int key = w * 32 + (D == 128 ? it >> 1 : it) * 8 + quarter * 2 + (e >> 2);
                        const int piece = (e & 3) + (D == 128 ? 4 * (((e >> 2) ^ it) & 1) : 0);
                        uint4 c = *reinterpret_cast<const uint4*>(raw + key * D + piece * 16);
                        if (key >= left) c = make_uint4(0, 0, 0, 0);
                        uint32_t v[4] = {c.x, c.y, c.z, c.w};
                        uint32_t found = 0;  // bit 7 of a byte: its code is 0x7f or 0xff
#pragma unroll
                        for (int k = 0; k < 4; ++k) found |= (v[k] & 0x7f7f7f7fu) + 0x01010101u;
                        if (found & 0x80808080u) {
                            bad |= 1u << (key & 31);
#pragma unroll
                            for (int k = 0; k < 4; ++k) {
                                const uint32_t at = ((v[k] & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;
                                v[k] &= ~((at >> 7) * 255u);
                            }
                        }
                        // code s eeee mmm as the bf16 number s 0000eeee mmm0000 is 2^-120 of its value
                        const uint32_t ex = sh.v_exp[rs][key >> box_shift];
                        const uint32_t big = ex > 134 ? 247u : ex + 120;  // 2^120 times the scale, in two steps where that is too large
                        const uint32_t mul = (big << 7) * 0x10001u;
                        uint32_t y[8];
#pragma unroll
                        for (int k = 0; k < 8; ++k) {
                            const uint32_t z = __byte_perm(v[k >> 1], 0, k & 1 ? 0x3424 : 0x1404);  // a code in the upper byte of each half
                            y[k] = mul_bf16x2(((z >> 4) & 0x07f007f0u) | (z & 0x80008000u), mul);
                        }
                        if (ex > 134) {
#pragma unroll
                            for (int k = 0; k < 8; ++k) y[k] = mul_bf16x2(y[k], (ex << 7) * 0x10001u);
                        }
                        uint8_t* const to = out + (piece >> 2) * kHalfBytes + key * 128;
                        const int at = 2 * (piece & 3);
                        *reinterpret_cast<uint4*>(to + ((at ^ (key & 7)) << 4)) = make_uint4(y[0], y[1], y[2], y[3]);
                        *reinterpret_cast<uint4*>(to + (((at + 1) ^ (key & 7)) << 4)) = make_uint4(y[4], y[5], y[6], y[7]);
                    }
                    bad = __reduce_or_sync(0xffffffffu, bad);
                    if (lane == 0) (&sh.nan_keys[x % S::notes][0].x)[w] = bad;
                    fence_proxy_async_smem();
                    __syncwarp();
                    if (lane == 0) {
                        mbar_arrive(&sh.v_full[vs]);
                        mbar_arrive(&sh.raw_empty[rs]);
                    }
                }
                if (!fine) break;
            }
            if ((!fine || !ok) && lane == 0) raise_error(p.err, kErrTimeout);
        } else {
            // ================= what this CTA leaves to the merge
            unsigned nj = 0;
            int4 left = make_int4(0, 0, 0, 0);
            bool ok;
            while (const Job* job = next_job(nj, ok)) {
                const Job g = *job;
                had_job(nj);
                if (!g.first) left.x |= kHasHead | (g.last ? kHeadEnds : 0);
                if (g.first && !g.last)
                    left = make_int4(left.x | kHasTail, g.q0 + g.t * 2 * p.tokens, min(2 * p.tokens, g.B - g.t * 2 * p.tokens), g.h);
            }
            if (!ok && lane == 0) raise_error(p.err, kErrTimeout);
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

template <int D>
int run(const ChunkAttentionFp8Args& a, const DeviceInfo& dev, cudaStream_t stream) {
    const int grid = std::min(dev.sm_count, kChunkMaxGrid);
    Fp8Params p;
    p.c = chunk_params(a, grid);
    p.q = static_cast<const __nv_bfloat16*>(a.q);
    p.q_stride = a.q_stride;
    p.k_scale = a.k_scale;
    p.v_scale = a.v_scale;

    CUtensorMap kmap, vmap;
    const cuuint64_t dims[3] = {(cuuint64_t)D, (cuuint64_t)a.num_kv_heads, (cuuint64_t)a.num_pages * a.page_size};
    const cuuint64_t strides[2] = {(cuuint64_t)D, (cuuint64_t)a.num_kv_heads * D};
    const cuuint32_t box[3] = {D, 1, (cuuint32_t)std::min(a.page_size, kKeys)};
    int rc = encode_tensor_map(&kmap, CU_TENSOR_MAP_DATA_TYPE_UINT8, 3, const_cast<void*>(a.k_cache), dims, strides, box,
                               D == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B);
    if (rc != BP_OK) return rc;
    rc = encode_tensor_map(&vmap, CU_TENSOR_MAP_DATA_TYPE_UINT8, 3, const_cast<void*>(a.v_cache), dims, strides, box,
                           CU_TENSOR_MAP_SWIZZLE_NONE);
    if (rc != BP_OK) return rc;

    static std::mutex mu;
    static bool configured[64] = {};
    if (dev.device < 0 || dev.device >= 64) return BP_ERR_UNSUPPORTED;
    {
        std::lock_guard<std::mutex> lock(mu);
        if (!configured[dev.device]) {
            if (cudaFuncSetAttribute(chunk_attention_fp8_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, fp8_smem<D>()) != cudaSuccess)
                return BP_ERR_CUDA;
            configured[dev.device] = true;
        }
    }
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.gridDim = dim3((unsigned)grid, 1, 1);
    cfg.blockDim = dim3(kFp8Threads, 1, 1);
    cfg.dynamicSmemBytes = fp8_smem<D>();
    cfg.stream = stream;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, chunk_attention_fp8_kernel<D>, p, kmap, vmap) != cudaSuccess) return BP_ERR_CUDA;
    if (a.max_kv_len <= (2 * kLeastCut - 1) * kKeys) return BP_OK;  // too short to be cut: nothing to merge
    return launch_chunk_merge(p.c, D, grid, a.max_q_len, stream);
}

}  // namespace

int launch_chunk_attention_fp8(const ChunkAttentionFp8Args& a, const DeviceInfo& dev, cudaStream_t stream) {
    return a.head_dim == 128 ? run<128>(a, dev, stream) : run<64>(a, dev, stream);
}

}  // namespace bp
