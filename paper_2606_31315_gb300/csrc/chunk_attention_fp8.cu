// Attention of chunks of new tokens over a paged KV cache in 8 bits: chunk_attention.cu's operation over keys and values held
// as e4m3 codes with a power of two for each page and KV head,
//
//   O_i = sum_j softmax_j(scale <q_i, 2^a k_j>) 2^b v_j      a, b: of key j's page
//
// Nothing is rounded that a bf16 cache would not round:
//   * S = Q K^T on the codes as they lie in memory, kind::f8f6f4.  A query row, scaled by a power of two to at most 256, is the
//     sum of two e4m3 numbers, its nearest and what is left: bf16's 8 bits are twice 4.  (Elements below 2^-10 of the row's
//     largest lose bits under 2^-18 of it.)  The row's and the page's powers multiply the scores in the softmax.
//   * P V in fp16, which holds every e4m3 number; four warps turn a tile's codes into them, in shared memory.  The weights take
//     the values' powers of two.
// The rest is as there: the line of work, two streams of a query tile each, the merge.  Where
// a work tile has the rows of one stream only (blocks, decoding), both streams take its queries and every other key tile,
// and add what they have at the end: a stream alone is a chain of latencies.
//
// Roles: warps 0-3 and 4-7 softmax of stream 0 and 1 (a thread a row; they read and split the queries too), warp 8 lays out
// the jobs and issues K's TMA copies, 9 and 10 issue the streams' MMAs, 11 V's copies and what the merge has to know, 12-15
// convert V.
#include <cuda_bf16.h>

#include <algorithm>
#include <mutex>

#include "chunk_plan.cuh"

namespace bp {
namespace {

constexpr int kHalfBytes = kKeys * 128;          // 128 rows of 64 fp16 columns (or of 128 codes), 128-byte swizzle
constexpr int kSoftmaxWarps = 8;                 // a thread a row
constexpr int kProducerWarp = 8, kMmaWarp = 9, kConvertWarp = 12;  // (a stream's MMA warp: kMmaWarp + stream)
constexpr int kConvertWarps = 4;                 // 32 keys of a tile each
constexpr int kFp8Threads = 32 * 16;
// Registers: 128 a thread at launch (512 x 128); 256 x 192 + 256 x 64 are as many.
constexpr int kSoftmaxRegs = 192, kOtherRegs = 64;
constexpr uint32_t kChunkTmem = 512;
constexpr int kJobs = 4;                         // jobs laid out ahead

template <int D>
struct Shape {
    static constexpr int code_bytes = kKeys * D;                // one K or V tile of codes
    static constexpr int v_bytes = 2 * code_bytes;              // one V tile in fp16
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
    const uint8_t* v;  // the cache's codes
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
    float k_power[S::notes][8];                      // the scales of a tile's boxes, of keys
    uint8_t v_below[S::raw_slots][8];                // of values: how far below the tile's largest one, as powers of two
    int v_ref[S::notes];                             // that one, biased
    Job job[kJobs];
    int job_nan[kJobs];                              // a code among its values is not a number
    uint32_t tmem;
    float2 row[2][kTileM];                           // of a split job's streams: row maxima and sums
    int row_ref[2][4];                               // and what their accumulators are in units of
};
template <int D>
constexpr int fp8_smem() { return Shape<D>::tiles + (int)sizeof(Shared<D>); }
static_assert(fp8_smem<128>() <= 227 * 1024 && fp8_smem<64>() <= 227 * 1024, "a block's shared memory");

// The values' powers of two: a tile's are held against its largest one (below 2^-24 of it they are 0; fp16 has e4m3's 18
// powers and 22 more), and that one against the largest so far, `ref`: the weights take the difference, times 2^7.  So they
// are at most 2^15 in fp16, and a tile's whose values are 2^-14 of others' still have all their bits at a weight of 2^-7.
constexpr uint32_t kLeastRef = 15;  // of a tile, so that the accumulator's power is a number too

// 2^(e - 127) of a biased exponent below 255.
__device__ __forceinline__ float power_of(uint32_t e) { return __uint_as_float(e ? e << 23 : 0x400000u); }

// The 32 rows of queries that a warp's lanes have at q + at (none where at < 0: zeros) as two e4m3 parts each, in the warp's
// rows of a tile with 128-byte swizzle.  A row is scaled by 2^(134 - E), E the biased exponent of its largest element (8 at
// least): that is below 256 then, its first part the number rounded to 4 bits, its second the exact rest of bf16's 8.  The
// rows come by asynchronous copies to where the parts go, 8 elements where the first parts of 16 will be and the next 8 where
// their rests will, so that a thread turns its row in place, in short loops (unrolled over registers this was 10 us a work
// tile: instructions that run once come from L2).  Returns the bits of the largest element of the lane's row.
template <int D>
__device__ __forceinline__ uint32_t split_queries(const __nv_bfloat16* q, int64_t at, uint8_t* tile) {
    constexpr int kPieces = D / 8, kRows = 32 / kPieces;  // of a row, 8 elements each; rows of a load
    const int lane = threadIdx.x & 31;
    // 16 bytes of the first parts, and of the rests (64 columns: both in one row of 128 bytes)
    auto place = [&](int row, int part, int i) {
        return tile + row * 128 + (D == 128 ? part * kHalfBytes : 0) + (((i + (D == 128 ? 0 : part * 4)) ^ (row & 7)) << 4);
    };
    const int piece = lane % kPieces;
#pragma unroll 2
    for (int k = 0; k < kPieces; ++k) {
        const int row = k * kRows + lane / kPieces;
        const int64_t from = __shfl_sync(0xffffffffu, at, row);
        cp_async16(place(row, piece & 1, piece >> 1), q + max((long long)from, 0ll) + piece * 8, from >= 0);
    }
    cp_async_wait_all();
    __syncwarp();
    uint32_t top = 0;
#pragma unroll 2
    for (int i = 0; i < D / 8; ++i) {
        const uint4 v = *reinterpret_cast<const uint4*>(place(lane, i & 1, i >> 1));
        const uint32_t x = max(max(v.x & 0x7fffu, v.y & 0x7fffu), max(v.z & 0x7fffu, v.w & 0x7fffu));
        const uint32_t y = max(max(v.x >> 16 & 0x7fffu, v.y >> 16 & 0x7fffu), max(v.z >> 16 & 0x7fffu, v.w >> 16 & 0x7fffu));
        top = max(top, max(x, y));
    }
    const float up = __uint_as_float((261u - max(top >> 7, 8u)) << 23);
#pragma unroll 1
    for (int i = 0; i < D / 16; ++i) {
        uint4* const to[2] = {reinterpret_cast<uint4*>(place(lane, 0, i)), reinterpret_cast<uint4*>(place(lane, 1, i))};
        const uint4 v[2] = {*to[0], *to[1]};
        uint32_t part[2][4];
#pragma unroll
        for (int c = 0; c < 8; ++c) {
            const uint4& u = v[c >> 2];
            const uint32_t w = (c & 3) == 0 ? u.x : (c & 3) == 1 ? u.y : (c & 3) == 2 ? u.z : u.w;
            const float x = __uint_as_float(w << 16) * up, y = __uint_as_float(w & 0xffff0000u) * up;
            // (halves away from 0: the rest is at most 8 units of bf16's last place either way)
            const float xn = __uint_as_float((__float_as_uint(x) + 0x80000u) & 0xfff00000u);
            const float yn = __uint_as_float((__float_as_uint(y) + 0x80000u) & 0xfff00000u);
            const uint32_t near = pack_e4m3x2(xn, yn), rest = pack_e4m3x2(x - xn, y - yn);
            part[0][c >> 1] = c & 1 ? part[0][c >> 1] | near << 16 : near;
            part[1][c >> 1] = c & 1 ? part[1][c >> 1] | rest << 16 : rest;
        }
        *to[0] = make_uint4(part[0][0], part[0][1], part[0][2], part[0][3]);
        *to[1] = make_uint4(part[1][0], part[1][1], part[1][2], part[1][3]);
    }
    return top;
}

// The columns [col, end) of a warp's rows, from the accumulators at `mine` and `others` (tensor memory; 0: none) times their
// weights, to row orow of the output (-1: none) or, fp32, to row `row` of part `slot`.
template <int D>
__device__ __forceinline__ void write_rows(const ChunkParams& p, uint32_t mine, uint32_t others, float w_mine, float w_others, int col,
                                        int end, bool whole, long long orow, size_t slot, int row) {
    const int lane = threadIdx.x & 31;
    // the rows of this lane's pair, both of which the two store together
    const long long rows[2] = {__shfl_sync(0xffffffffu, orow, lane & ~1), __shfl_sync(0xffffffffu, orow, lane | 1)};
#pragma unroll 1
    for (; col < end; col += 16) {
        uint32_t v[16];
        if (mine) {
            tmem_ld16(mine + col, v);
            tmem_ld_wait();
        }
#pragma unroll
        for (int e = 0; e < 16; ++e) v[e] = mine ? __float_as_uint(__uint_as_float(v[e]) * w_mine) : 0u;
        if (others) {
            uint32_t t[16];
            tmem_ld16(others + col, t);
            tmem_ld_wait();
#pragma unroll
            for (int e = 0; e < 16; ++e) v[e] = __float_as_uint(fmaf(__uint_as_float(t[e]), w_others, __uint_as_float(v[e])));
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
        } else if (orow >= 0) {
#pragma unroll
            for (int e = 0; e < 16; e += 8)
                st_global_f32x8(p.part_o + part_at<D>(slot, row, col + e), reinterpret_cast<const float*>(&v[e]));
        }
        __syncwarp();
    }
}

// Whether one of the values of keys [key, key + 64) that lie in [lo, hi) has a code that is not a number; lo and hi are of
// the lane's row, and the whole warp calls this.
template <int D>
__device__ __forceinline__ bool sees_nan(const Fp8Params& fp, const Job& g, int key, int lo, int hi) {
    const ChunkParams& p = fp.c;
    const int lane = threadIdx.x & 31;
    bool sees = false;
    for (const int end = min(g.n, key + 64); key < end; ++key) {
        const int pg = key >> p.page_shift;
        int id = pg < p.pages_per_seq ? __ldg(p.block_table + (size_t)g.s * p.pages_per_seq + pg) : 0;
        if ((unsigned)id >= (unsigned)p.num_pages) id = 0;  // (reported where the tile was asked for)
        const int64_t row = ((int64_t)id << p.page_shift) + (key & ((1 << p.page_shift) - 1));
        uint32_t codes = 0;
        if (lane < D / 4) codes = __ldg(reinterpret_cast<const uint32_t*>(fp.v + (row * p.num_kv_heads + g.h) * D) + lane);
        const bool none = __any_sync(0xffffffffu, ((codes & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u);
        sees |= none && key >= lo && key < hi;
    }
    return sees;
}

// The boxes that a job's key tiles come in, one a page or, of larger pages, one a tile: their pages and scales, looked up by
// a whole warp, 32 boxes at a time, the next ones in flight meanwhile (tile by tile, table and then scale, they alone took
// 1.5 us a tile).
struct Boxes {
    const ChunkParams& p;
    const uint8_t* scale;
    const Job& g;
    int rows, of_tile, last_page;  // keys of a box; boxes of a tile; the sequence's last page
    int near, far, used = 0;       // this lane's page of the 32 boxes at hand and of the next 32 (-1: none); boxes done with
    uint32_t near_e, far_e;        // their scales
    uint32_t exponent;             // the scale of this lane's box of the tile that next() was for

    __device__ __forceinline__ Boxes(const ChunkParams& params, const uint8_t* scales, const Job& job)
        : p(params), scale(scales), g(job), rows(min(kKeys, 1 << params.page_shift)), of_tile(kKeys / rows),
          last_page((job.n - 1) >> params.page_shift) {
        look_up(g.j0, near, near_e);
        look_up(g.j0 + 32 / of_tile, far, far_e);
    }
    __device__ __forceinline__ void look_up(int j, int& id, uint32_t& e) const {
        const int lane = threadIdx.x & 31;
        j += lane / of_tile;
        const int pg = (j * kKeys + lane % of_tile * rows) >> p.page_shift;
        id = -1;
        e = 127;
        if (j < g.j1 && pg <= last_page) {
            id = pg < p.pages_per_seq ? __ldg(p.block_table + (size_t)g.s * p.pages_per_seq + pg) : -1;
            if ((unsigned)id >= (unsigned)p.num_pages) {
                raise_error(p.err, kErrDeviceArg);
                id = 0;
            }
            e = __ldg(scale + (size_t)id * p.num_kv_heads + g.h);
        }
    }
    // The pool row of this lane's box of tile j, -1 where it has none.
    __device__ __forceinline__ int next(int j) {
        const int lane = threadIdx.x & 31, at = (used + lane) & 31;
        const int id = __shfl_sync(0xffffffffu, near, at);
        exponent = __shfl_sync(0xffffffffu, near_e, at);
        if ((used += of_tile) == 32) {
            used = 0;
            near = far;
            near_e = far_e;
            look_up(j + 1 + 32 / of_tile, far, far_e);
        }
        if (lane >= of_tile || id < 0) return -1;
        if (exponent == 255) {
            raise_error(p.err, kErrDeviceArg);
            exponent = 254;
        }
        return (id << p.page_shift) + ((j * kKeys + lane * rows) & ((1 << p.page_shift) - 1));
    }
    // The keys of tile j's boxes.
    __device__ __forceinline__ uint32_t keys(int j) const { return min(of_tile, (g.n - j * kKeys + rows - 1) / rows) * rows; }
};

// FACTORS: scales that a tile of 128 keys may have: 8 with pages of 16, 2 from pages of 64 on.
template <int D, int FACTORS>
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
            mbar_init(&sh.q_ready[i], 4);
            mbar_init(&sh.s[i], 1);
            mbar_init(&sh.p[i], 4);
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
        // ================= softmax of stream i: a thread a row
        const int i = warp >> 2, quad = warp & 3, r = quad * 32 + lane;
        const uint32_t lanes = tmem + (static_cast<uint32_t>(quad * 32) << 16);
        const uint32_t s_addr = lanes + i * 128;  // P comes over the scores
        const int my_tok = r / G;
        const int box_shift = min(7, p.page_shift);
        unsigned ns = 0, no = 0, x0 = 0;  // scores and accumulators waited for; key tiles of the jobs before
        bool failed = false;
        unsigned nj = 0;
        for (;;) {
            bool ok = false;
            const Job* g = failed ? nullptr : next_job(nj, ok);
            // (a warp that gave up a wait takes the other stream's of its rows along, here and at a split job's end)
            if (named_barrier_or(1 + quad, 64, !ok)) {
                failed = true;
                break;
            }
            if (!g) break;
            const bool split = is_split(*g);
            const int mine = split ? 0 : i;  // the query tile
            const int a = g->a[mine], b = g->b[mine], j0 = g->j0, j1 = g->j1;
            const int tok = g->t * 2 * p.tokens + mine * p.tokens + my_tok;
            const bool active = my_tok < p.tokens && tok < g->B;
            const int pos = g->n - g->B + tok;  // (what the end needs of the job is read again there)
            // (rows of none count as seeing all: their warps' tiles are not masked for their sake)
            const int hi = !active ? 0x7fffffff : p.causal ? max(0, pos + 1) : g->n;
            const int lo = active && p.window > 0 ? max(0, pos + 1 - p.window) : 0;
            const bool idle = !__any_sync(0xffffffffu, active);  // the same in both warps of these rows
            float m = -INFINITY, l = 0.f, row_scale = 1.f;
            if (j1 > j0 && b > a && !idle) {
                // ---- the queries of this warp's rows, two parts each, to shared memory
                const int64_t at = active ? (int64_t)(g->q0 + tok) * fp.q_stride + (g->h * G + r - my_tok * G) * D : -1;
                uint32_t top = 0;
                if (mine == i) top = split_queries<D>(fp.q, at, smem + i * S::q_bytes + quad * 32 * 128);
                if (split) {  // (the other stream's threads learn of it)
                    if (i == 0) sh.row[0][r].x = __uint_as_float(top);
                    named_barrier(1 + quad, 64);
                    if (i == 1) top = __float_as_uint(sh.row[0][r].x);
                }
                // the row times 2^(7 - e) is below 256; 2^(e - 7) of it is put back with the softmax's scale
                row_scale = p.scale_log2 * __uint_as_float((max(top >> 7, 8u) - 7) << 23);
                if (top >= 0x7f80u && hi > lo) l = __uint_as_float(0x7fc00000u);  // a NaN or an infinity: the row is none
            }
            if (j1 > j0 && mine == i) {
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) mbar_arrive(&sh.q_ready[i]);
            }
            const int step = split ? 2 : 1, from_j = split ? a + i : a;  // (a split job's a is its j0)
            int from = lo - from_j * kKeys, to = hi - from_j * kKeys;    // columns that the row sees
            unsigned xt = x0 + from_j - j0;
            int ref = 0;  // the largest power of two of the stream's values so far, biased (0: none yet)
#pragma unroll 1
            for (int j = from_j; j < b; j += step, ++ns, xt += step, from -= step * kKeys, to -= step * kKeys) {
                failed = !__all_sync(0xffffffffu, mbar_wait(&sh.s[i], ns & 1, kWaitBudget));
                if (failed) break;
                tc_fence_after();
                if (!idle) {
                    const bool full = __all_sync(0xffffffffu, from <= 0 && to >= kKeys);
                    // the factors of the scores, of kKeys / FACTORS keys each; finite and above 0, so that a hidden column's
                    // -inf stays one
                    float f[FACTORS];
#pragma unroll
                    for (int c = 0; c < FACTORS; ++c)
                        f[c] = fmaxf(fminf(row_scale * sh.k_power[xt % S::notes][c * (kKeys / FACTORS) >> box_shift], 3.4e38f), 1.2e-38f);
                    uint32_t x[8][16];
                    float mx[8];
                    if (full) {
#pragma unroll
                        for (int c = 0; c < 8; ++c) tmem_ld16_max(s_addr + c * 16, x[c], mx[c]);
                        tmem_ld_wait();
                    } else {
#pragma unroll
                        for (int c = 0; c < 8; ++c) tmem_ld16(s_addr + c * 16, x[c]);
                        tmem_ld_wait();
#pragma unroll
                        for (int c = 0; c < 8; ++c) {
                            mx[c] = -INFINITY;
#pragma unroll
                            for (int e = 0; e < 16; ++e) {
                                if (c * 16 + e < from || c * 16 + e >= to) x[c][e] = 0xff800000u;  // -inf
                                mx[c] = fmaxf(mx[c], __uint_as_float(x[c][e]));
                            }
                        }
                    }
                    float top = -INFINITY;
#pragma unroll
                    for (int c = 0; c < FACTORS; ++c) {
                        float y = mx[c * (8 / FACTORS)];
#pragma unroll
                        for (int e = 1; e < 8 / FACTORS; ++e) y = fmaxf(y, mx[c * (8 / FACTORS) + e]);
                        top = fmaxf(top, y * f[c]);
                    }
                    // (with this m, 2^(score - m) stays below 2^8)
                    const bool grew = top > m + 8.f;
                    const int tile_ref = sh.v_ref[xt % S::notes];
                    if (__any_sync(0xffffffffu, grew) || tile_ref > ref) {
                        float alpha = grew ? chunk_exp2(m - top) : 1.f;
                        if (grew) l *= alpha;
                        // (this tile's scores are complete, so the stream's MMAs before them, the last P V among them, are too)
                        if (j > from_j) {
                            if (tile_ref > ref) alpha *= power_of((uint32_t)max(127 + ref - tile_ref, 0));
#pragma unroll 1
                            for (int c = 0; c < D / 16; ++c) {
                                uint32_t v[16];
                                tmem_ld16(lanes + S::col_o + i * D + c * 16, v);
                                tmem_ld_wait();
#pragma unroll
                                for (int e = 0; e < 16; ++e) v[e] = __float_as_uint(__uint_as_float(v[e]) * alpha);
                                tmem_st16(lanes + S::col_o + i * D + c * 16, v);
                            }
                        }
                        if (grew) m = top;
                        ref = max(ref, tile_ref);
                    }
                    // weights 2^(f * score - m) times the values' power and 2^7, packed in pairs over the scores; their sum
                    const int power = max(tile_ref - ref + 7, -60);
                    const float negm = (m == -INFINITY ? 0.f : -m) + (float)power;
                    const uint64_t negm2 = pack_f32x2(negm, negm);
                    uint64_t sum2[2] = {0ull, 0ull};
#pragma unroll
                    for (int c = 0; c < 8; c += 2) {
                        uint32_t pk[16];
#pragma unroll
                        for (int e = 0; e < 16; ++e) {
                            const int h = c + (e >> 3);
                            const float factor = f[h * FACTORS / 8];
                            float u, w;
                            unpack_f32x2(fma_f32x2(pack_f32x2(__uint_as_float(x[h][2 * (e & 7)]), __uint_as_float(x[h][2 * (e & 7) + 1])),
                                                   pack_f32x2(factor, factor), negm2), u, w);
                            u = chunk_exp2(u);
                            w = chunk_exp2(w);
                            sum2[e & 1] = add_f32x2(sum2[e & 1], pack_f32x2(u, w));
                            pk[e] = pack_f16x2(u, w);  // fp16, as the converted values are: 11 bits
                        }
                        tmem_st16(s_addr + c * 8, pk);
                    }
                    float u, w;
                    unpack_f32x2(add_f32x2(sum2[0], sum2[1]), u, w);
                    l = fmaf(u + w, __uint_as_float((uint32_t)(127 - power) << 23), l);
                    tmem_st_wait();
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&sh.p[i]);
            }
            const bool some = from_j < b;  // this stream had a tile
            if (!failed && some) {
                failed = !__all_sync(0xffffffffu, mbar_wait(&sh.o[i], no & 1, kWaitBudget));
                ++no;
                tc_fence_after();
                // A value that is none, in a key that the row sees, makes the row none (the tiles' weights of it are 0, and its
                // values too).  Rare: the codes are read again to find which keys have one.
                if (*const_cast<volatile int*>(&sh.job_nan[nj % kJobs]) && !idle)
                    for (int j = from_j; j < b; j += step)
                        if (sees_nan<D>(fp, *g, j * kKeys, lo, hi)) l = __uint_as_float(0x7fc00000u);
            }
            x0 += j1 - j0;
            if (!split && failed) continue;
            // the weights of the streams' accumulators, which are in units of 2^(ref - 134)
            float w_mine = some ? power_of((uint32_t)(ref - 7)) : 0.f, w_other = 0.f;
            bool others_some = false;
            if (split) {
                // ---- the other stream's part of these rows, merged as the second kernel merges CTAs' parts
                sh.row[i][r] = make_float2(m, l);
                if (lane == 0) sh.row_ref[i][quad] = some ? ref : 0;
                if (named_barrier_or(1 + quad, 64, failed)) {
                    failed = true;
                    continue;
                }
                others_some = a + (i ^ 1) < b;
                const float2 o = sh.row[i ^ 1][r];
                const float top = fmaxf(m, o.x);
                const float u = m == top ? 1.f : chunk_exp2(m - top), v = o.x == top ? 1.f : chunk_exp2(o.x - top);
                l = i == 0 ? l * u + o.y * v : o.y * v + l * u;
                m = top;
                w_mine *= u;
                if (others_some) w_other = v * power_of((uint32_t)(sh.row_ref[i ^ 1][quad] - 7));
            }
            const bool first = g->first, whole = first && g->last;
            // the query row's number among all, in the output (-1: none)
            const long long orow = active ? (long long)(g->q0 + tok) * p.num_q_heads + g->h * G + r - my_tok * G : -1;
            had_job(nj);
            const float inv = whole ? row_inverse(m, l) : 1.f;
            w_mine *= inv;
            w_other *= inv;
            const size_t slot = (size_t)blockIdx.x * 2 + (first ? 1 : 0);
            if (!idle) {
                // (a split job's two warps have half of the columns each)
                const uint32_t o_addr = lanes + S::col_o;
                write_rows<D>(p, some ? o_addr + i * D : 0, others_some ? o_addr + (i ^ 1) * D : 0, w_mine, w_other,
                              split ? i * (D / 2) : 0, split ? (i + 1) * (D / 2) : D, whole, orow, slot, mine * kTileM + r);
            }
            if (active && (!split || i == 0)) {
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
                    sh.job_nan[e] = 0;
                    mbar_arrive(&sh.job_full[e]);
                }
                ++nj;
            };
            unsigned x = 0;  // tiles asked for
            Job g, after;
            for (bool have = false; ; have = true) {
                lay_out(after);  // one ahead of the copies
                if (!ok) break;
                if (have && g.j1 > g.j0) {
                    Boxes box(p, fp.k_scale, g);
                    for (int j = g.j0; j < g.j1; ++j, ++x) {
                        const int slot = x % S::k_slots;
                        ok = x < (unsigned)S::k_slots || __all_sync(0xffffffffu, mbar_wait(&sh.k_empty[slot], (x / S::k_slots - 1) & 1, kWaitBudget));
                        if (!ok) break;
                        const int row = box.next(j);
                        // (a slot is full when lane 0 has said how many bytes it takes)
                        if (row >= 0) tma_load_3d(smem + S::at_k + slot * S::code_bytes + lane * box.rows * D, &kmap, &sh.k_full[slot], 0, g.h, row);
                        if (lane < box.of_tile) sh.k_power[x % S::notes][lane] = power_of(box.exponent);
                        __syncwarp();
                        if (lane == 0) mbar_arrive_expect_tx(&sh.k_full[slot], box.keys(j) * D);
                    }
                }
                if (!ok || after.s < 0) break;
                g = after;
            }
            if (!ok && lane == 0) raise_error(p.err, kErrTimeout);
            // no copy may still be in flight when the CTA leaves
            for (unsigned y = x > (unsigned)S::k_slots ? x - S::k_slots : 0; y < x; ++y)
                if (!mbar_wait(&sh.k_full[y % S::k_slots], (y / S::k_slots) & 1, kDrainBudget) && lane == 0) raise_error(p.err, kErrTimeout);
        } else if (warp == kMmaWarp || warp == kMmaWarp + 1) {
            // ================= MMA issuer of stream i.  The streams take turns, a P V and a Q K^T at a time, each from a
            // warp of its own: one waits for its operands and commits while the other's MMAs are issued
            const int i = warp - kMmaWarp;
            const uint32_t id_s = idesc_e4m3_f32(kTileM, kKeys);
            const uint32_t id_o = idesc_f16_f32(kTileM, D, false, true);
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
                        if (pv) {  // O += P V of tile jp
                            const uint32_t vl = v_lo + vslot * (S::v_bytes >> 4);
                            uint32_t on = jp > first ? 1u : 0u;
#pragma unroll
                            for (int kk = 0; kk < kKeys / 16; ++kk) {
                                umma_ts(t_o, t_s + kk * 8, upper | (vl + kk * (2048 >> 4)), id_o, on);
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
            // ================= V from codes to fp16: keys [32 w, 32 w + 32) of every tile
            // Eight lanes read all banks, and write them: a key's lower pieces of 16 codes with the next key's upper ones (form
            // 0; 1: the other way round; of 64 columns: the two keys' pieces all together).  From one piece of a lane to the
            // next of its form it is 8 keys, which the swizzle does not tell apart.
            constexpr int kForms = D == 128 ? 2 : 1, kPieces = 2 * kForms;  // pieces of 16 keys
            const int w = warp - kConvertWarp, e = lane & 7;
            const int key0 = w * 32 + (lane >> 3) * 2 + (e >> 2);
            int from[kForms], to[kForms];
#pragma unroll
            for (int form = 0; form < kForms; ++form) {
                const int piece = (e & 3) + (D == 128 ? 4 * ((e >> 2) ^ form) : 0);
                from[form] = key0 * D + piece * 16;
                to[form] = (piece >> 2) * kHalfBytes + key0 * 128 + (((2 * (piece & 3)) ^ (key0 & 7)) << 4);
            }
            const int box_shift = min(7, p.page_shift);
            unsigned x = 0, nj = 0;
            bool ok, fine = true;
            while (const Job* g = next_job(nj, ok)) {
                const int j0 = g->j0, j1 = g->j1, n = g->n;
                int* const nan = &sh.job_nan[nj % kJobs];
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
#pragma unroll
                    for (int h = 0; h < 2; ++h) {  // 16 keys at a time: boxes are no smaller
                        uint32_t v[kPieces][4];
#pragma unroll
                        for (int k = 0; k < kPieces; ++k) {
                            const uint4 c = *reinterpret_cast<const uint4*>(raw + from[k % kForms] + (h * kPieces + k) / kForms * 8 * D);
                            v[k][0] = c.x; v[k][1] = c.y; v[k][2] = c.z; v[k][3] = c.w;
                        }
                        if (left < kKeys) {
#pragma unroll
                            for (int k = 0; k < kPieces; ++k)
                                if (key0 + (h * kPieces + k) / kForms * 8 >= left) v[k][0] = v[k][1] = v[k][2] = v[k][3] = 0;
                        }
                        uint32_t found = 0;  // bit 7 of a byte: a code is 0x7f or 0xff
#pragma unroll
                        for (int k = 0; k < kPieces; ++k)
#pragma unroll
                            for (int c = 0; c < 4; ++c) found |= (v[k][c] & 0x7f7f7f7fu) + 0x01010101u;
                        if (__any_sync(0xffffffffu, found & 0x80808080u)) {
                            *nan = 1;  // (the softmax warps look once all of the job's values have been used)
#pragma unroll
                            for (int k = 0; k < kPieces; ++k)
#pragma unroll
                                for (int c = 0; c < 4; ++c) {
                                    const uint32_t at = ((v[k][c] & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;
                                    v[k][c] &= ~((at >> 7) * 255u);
                                }
                        }
                        const int below = sh.v_below[rs][(w * 32 + h * 16) >> box_shift];
                        const uint32_t mul = (below < 15 ? (15 - below) << 10 : below < 25 ? 1 << (24 - below) : 0) * 0x10001u;
#pragma unroll
                        for (int k = 0; k < kPieces; ++k) {
                            uint32_t y[8];
#pragma unroll
                            for (int c = 0; c < 8; ++c) y[c] = mul_f16x2(e4m3x2_to_f16x2(c & 1 ? v[k][c >> 1] >> 16 : v[k][c >> 1]), mul);
                            uint8_t* const at = out + (h * kPieces + k) / kForms * 1024;
                            *reinterpret_cast<uint4*>(at + to[k % kForms]) = make_uint4(y[0], y[1], y[2], y[3]);
                            *reinterpret_cast<uint4*>(at + (to[k % kForms] ^ 16)) = make_uint4(y[4], y[5], y[6], y[7]);
                        }
                    }
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
            // ================= V tiles of codes through their ring; what this CTA leaves to the merge
            unsigned x = 0, nj = 0;
            int4 left = make_int4(0, 0, 0, 0);
            bool ok, fine = true;
            while (const Job* job = next_job(nj, ok)) {
                const Job g = *job;
                had_job(nj);
                if (!g.first) left.x |= kHasHead | (g.last ? kHeadEnds : 0);
                if (g.first && !g.last)
                    left = make_int4(left.x | kHasTail, g.q0 + g.t * 2 * p.tokens, min(2 * p.tokens, g.B - g.t * 2 * p.tokens), g.h);
                if (g.j1 <= g.j0) continue;
                Boxes box(p, fp.v_scale, g);
                for (int j = g.j0; j < g.j1; ++j, ++x) {
                    const int slot = x % S::raw_slots;
                    fine = x < (unsigned)S::raw_slots || __all_sync(0xffffffffu, mbar_wait(&sh.raw_empty[slot], (x / S::raw_slots - 1) & 1, kWaitBudget));
                    if (!fine) break;
                    const int row = box.next(j);
                    if (row >= 0) tma_load_3d(smem + S::at_raw + slot * S::code_bytes + lane * box.rows * D, &vmap, &sh.raw_full[slot], 0, g.h, row);
                    const uint32_t ref = max(__reduce_max_sync(0xffffffffu, row >= 0 ? box.exponent : 0u), kLeastRef);
                    if (lane < box.of_tile) sh.v_below[slot][lane] = (uint8_t)(row >= 0 ? ref - box.exponent : 0u);
                    if (lane == 0) sh.v_ref[x % S::notes] = (int)ref;
                    __syncwarp();
                    if (lane == 0) mbar_arrive_expect_tx(&sh.raw_full[slot], box.keys(j) * D);
                }
                if (!fine) break;
            }
            if ((!ok || !fine) && lane == 0) raise_error(p.err, kErrTimeout);
            for (unsigned y = x > (unsigned)S::raw_slots ? x - S::raw_slots : 0; y < x; ++y)
                if (!mbar_wait(&sh.raw_full[y % S::raw_slots], (y / S::raw_slots) & 1, kDrainBudget) && lane == 0) raise_error(p.err, kErrTimeout);
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

template <int D, int FACTORS>
int run(const ChunkAttentionFp8Args& a, const DeviceInfo& dev, cudaStream_t stream) {
    const int grid = std::min(dev.sm_count, kChunkMaxGrid);
    Fp8Params p;
    p.c = chunk_params(a, grid);
    p.q = static_cast<const __nv_bfloat16*>(a.q);
    p.q_stride = a.q_stride;
    p.k_scale = a.k_scale;
    p.v_scale = a.v_scale;
    p.v = static_cast<const uint8_t*>(a.v_cache);

    CUtensorMap kmap, vmap;
    const cuuint64_t dims[3] = {(cuuint64_t)D, (cuuint64_t)a.num_kv_heads, (cuuint64_t)a.num_pages * a.page_size};
    const cuuint64_t strides[2] = {(cuuint64_t)D, (cuuint64_t)a.num_kv_heads * D};
    // (a head's row is all that is asked for: 256 bytes would be the next head's too, which another CTA reads at another time)
    const CUtensorMapL2promotion promotion = D == 128 ? CU_TENSOR_MAP_L2_PROMOTION_L2_128B : CU_TENSOR_MAP_L2_PROMOTION_L2_64B;
    const cuuint32_t box[3] = {D, 1, (cuuint32_t)std::min(a.page_size, kKeys)};
    int rc = encode_tensor_map(&kmap, CU_TENSOR_MAP_DATA_TYPE_UINT8, 3, const_cast<void*>(a.k_cache), dims, strides, box,
                               D == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, promotion);
    if (rc != BP_OK) return rc;
    rc = encode_tensor_map(&vmap, CU_TENSOR_MAP_DATA_TYPE_UINT8, 3, const_cast<void*>(a.v_cache), dims, strides, box,
                           CU_TENSOR_MAP_SWIZZLE_NONE, promotion);
    if (rc != BP_OK) return rc;

    static std::mutex mu;
    static bool configured[64] = {};
    if (dev.device < 0 || dev.device >= 64) return BP_ERR_UNSUPPORTED;
    {
        std::lock_guard<std::mutex> lock(mu);
        if (!configured[dev.device]) {
            if (cudaFuncSetAttribute(chunk_attention_fp8_kernel<D, FACTORS>, cudaFuncAttributeMaxDynamicSharedMemorySize, fp8_smem<D>()) != cudaSuccess)
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
    if (cudaLaunchKernelEx(&cfg, chunk_attention_fp8_kernel<D, FACTORS>, p, kmap, vmap) != cudaSuccess) return BP_ERR_CUDA;
    if (a.max_kv_len <= (2 * kLeastCut - 1) * kKeys) return BP_OK;  // too short to be cut: nothing to merge
    return launch_chunk_merge(p.c, D, grid, a.max_q_len, stream);
}

}  // namespace

int launch_chunk_attention_fp8(const ChunkAttentionFp8Args& a, const DeviceInfo& dev, cudaStream_t stream) {
    if (a.page_size >= 64) return a.head_dim == 128 ? run<128, 2>(a, dev, stream) : run<64, 2>(a, dev, stream);
    return a.head_dim == 128 ? run<128, 8>(a, dev, stream) : run<64, 8>(a, dev, stream);
}

}  // namespace bp
