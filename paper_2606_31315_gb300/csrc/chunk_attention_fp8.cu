// Attention of chunks of new tokens over a paged KV cache in 8 bits: chunk_attention.cu's operation over keys and values held
// as e4m3 codes with a power of two for each page and KV head,
//
//   O_i = sum_j softmax_j(scale <q_i, 2^a k_j>) 2^b v_j      a, b: of key j's page
//
//   * S = Q K^T on the codes as they lie in memory, kind::f8f6f4.  A query row, scaled by a power of two to at most 256, is the
//     sum of two e4m3 numbers: bf16's 8 bits are twice 4.  Elements below 2^-9 of the row's largest are off by up to 2^-16 of it:
//     fewer bits than the caller's, and a choice.  A third part would be half as many MMAs again, on accumulators of its own
//     that tensor memory has no room for (the parts' scales differ); K in fp16 would be V's conversion a second time.  The scores
//     of Gaussian queries lose less than their own sum in fp32 does; those of a row with one element 256 times as large, where
//     the keys are 0, as much as the queries' own rounding to bf16.  The row's and the page's powers multiply the scores in the
//     softmax.
//   * P V in fp16, which holds every e4m3 number; four warps turn a tile's codes into them, in shared memory.  The weights take
//     the values' powers of two, and are rounded to 11 bits, or at 2^-29 of the row's largest.
// The line of work and the merge are chunk_attention.cu's.  Two kernels: chunk_attention_fp8_kernel for any call, its two streams a
// query tile each (where a work tile has the rows of one only, both take them, and every other key tile, and add what they
// have at the end), and block_attention_fp8_kernel for calls whose work tiles all are such: blocks and single tokens.
//
// What bounds them (32 query and 8 KV heads of 128, pages of 64; floors at 6.75 TB/s and 1.93 PFLOP/s).  Times in this file are of single
// calls, events around each, L2 flushed before: some 8 us more than the kernels alone.
//   * a prompt of 8192, 446 us of 285: a stream's chain from tile to tile (scores out of tensor memory, maximum, weights, the turn's
//     16 MMAs and the hand-overs); two streams in turn take 2,840 cycles a pair of key tiles, 2,048 of them MMAs (which read shared
//     memory at its full rate: 128 bytes a cycle).  A job change is 18,000 cycles, half of it the queries' way in, and heads whose
//     maxima keep growing take up to 3,300 a pair, which the plan does not know.  (A bf16 cache: 369 us.)
//   * 8 blocks of 31 over 32768 keys, 139 to 144 us of 80 (3.9 TB/s): the conversion's steps one after the other, and the job
//     changes; a plain read of the same rows of 128 bytes takes 94 to 106.  (A bf16 cache: 236 us, 217 with
//     bp_block_attention_paged.)
//   * one token over 2048 keys, 21 us: the plan, two copies, a tile, the merge, one after the other.
//
// Roles: warps 0-3 and 4-7 softmax of stream 0 and 1 (a thread a row; they read and split the queries too), warp 8 lays out
// the jobs and issues K's TMA copies, 9 and 10 issue the streams' MMAs, 11 V's copies and what the merge has to know, 12-15
// convert V.
#include <cuda_bf16.h>

#include <algorithm>
#include <mutex>

namespace bp {
namespace {
// A work tile's fixed cost (queries in, output out), in keys.  One number for all calls; us with a cold L2 at 400, 700, 1000, 1400:
//   a prompt of 8192                       535  466  446  455    the same, heads of 64                   408  368  376  384
//   16 and 32 chunks among single tokens   139  130  125  133    (pages of 64)                           171  148  142  142
//   16 x 100 tokens over 1000 keys          76   73   72   71    8 x 300 to 1000 tokens, heads of 64      98  100   99  101
//   4 x 2001 in a window, heads of 64       56   58   56   58    8 x 64 over 4096                         62   61   60   65
// Blocks and single tokens, 8 x 31 over 32768 to 64 x 1 over 4096: within 3 % with all four.
constexpr int kTileCost = 1000;
}  // namespace
}  // namespace bp

#include "chunk_plan.cuh"

namespace bp {
namespace {

constexpr int kHalfBytes = kKeys * 128;          // 128 rows of 64 fp16 columns (or of 128 codes), 128-byte swizzle
constexpr uint32_t kChunkTmem = 512;
constexpr int kSoftmaxWarps = 8;                 // a thread a row, four warps a stream
constexpr int kKeyWarp = 8, kMmaWarp = 9, kValueWarp = 11, kConvertWarp = 12;  // (a stream's MMA warp: kMmaWarp + stream)
constexpr int kConvertWarps = 4;                 // 32 keys of a tile each
constexpr int kThreads = 32 * (kConvertWarp + kConvertWarps);
// Registers of the roles: 128 a thread at launch (512 x 128), as many as 256 x softmax + 128 x (convert + other).  Each role sets
// its own in its own branch (before they part: 32 x 1 tokens over 8192 keys 148 us instead of 140, and of two values there the
// compiler keeps to the lesser for both).  A prompt of 8192 takes 457 us with 192, 64 and 64, 447 with 200, 56 and 56, 454 with
// 208, 48 and 48; decoding batches 140 with the first and 144 with the second.
struct Registers {
    int softmax, convert, other;
};
constexpr Registers kRegs = {200, 56, 56}, kBlockRegs = {192, 64, 64};
static_assert(256 * kRegs.softmax + 128 * (kRegs.convert + kRegs.other) <= kThreads * 128, "the launch's registers");
static_assert(256 * kBlockRegs.softmax + 128 * (kBlockRegs.convert + kBlockRegs.other) <= kThreads * 128, "the launch's registers");
constexpr int kJobs = 4;                         // jobs laid out ahead
constexpr int kBatches = 8;                      // of 32 boxes' scales: jobs and tiles that may be under way at once, and more

// FEW: work tiles of one stream only.  Their kernel has no second query tile.
template <int D, bool FEW>
struct Shape {
    static constexpr int code_bytes = kKeys * D;                // one K or V tile of codes
    static constexpr int v_bytes = 2 * code_bytes;              // one V tile in fp16
    static constexpr int q_bytes = 2 * code_bytes;              // one query tile, both parts
    static constexpr int k_slots = D == 128 ? 3 : 8;
    static constexpr int raw_slots = (D == 128 ? 3 : 7) + 2 * FEW;  // V's codes
    static constexpr int v_slots = D == 128 ? 2 : 4;
    static constexpr int at_k = (FEW ? 1 : 2) * q_bytes;
    static constexpr int at_raw = at_k + k_slots * code_bytes;
    static constexpr int at_v = at_raw + raw_slots * code_bytes;
    static constexpr int tiles = at_v + v_slots * v_bytes;
};
struct Fp8Params {
    ChunkParams c;
    const __nv_bfloat16* q;
    int64_t q_stride;
    const uint8_t* k_scale;
    const uint8_t* v_scale;
    const uint8_t* v;  // the cache's codes
};

// Shared memory of a block that needs so much: it leaves no other CTA's tensor memory room.
constexpr int whole_sm(int bytes) {
    const int share = tmem_smem_share((int)kChunkTmem, 228 * 1024);
    return bytes > share ? bytes : share;
}

// Shared memory behind the tiles: what both kernels have.
template <int D, bool FEW>
struct Common {
    using S = Shape<D, FEW>;
    uint64_t k_full[S::k_slots], k_empty[S::k_slots], raw_full[S::raw_slots], raw_empty[S::raw_slots];
    uint64_t v_full[S::v_slots], v_empty[S::v_slots];
    uint64_t job_full[kJobs], job_empty[kJobs];
    // The scales of the boxes (Boxes), 32 at a time: of keys, bf16 numbers; of values, biased exponents, what the weights take of
    // them, the least of that in the box's tile, and what is left for the values themselves.
    alignas(16) uint16_t k_power[kBatches][32];
    alignas(8) uint8_t v_exp[kBatches][32], v_low[kBatches][32], v_below[kBatches][32];
    Job job[kJobs];
    int job_nan[kJobs];                              // a code among its values is not a number
    uint32_t tmem;
};

// The values' powers of two, 2^(e - 127): the weights take them, so that P V has the values as their codes say.  With a row's
// scores x (in powers of two) and e of their keys, M near the largest x + e that the row has seen, and m near its largest x,
//
//   P = 2^(x + e - M + 5)    O = 2^(M - m - 132) sum P code    l = sum 2^(x - m), of the same exponentials
//
// What a row cannot see has no part in its M: hidden keys cost it no bits.  M and m are whole numbers.  M is moved where x + e
// has outgrown it by 2^10 (and a half, for top_score's rounding), so that P is below 2^16 in fp16; m where x + e less the tile's least
// e has, which may put it 2^kReach above the largest x.  P has all its 11 bits from 2^-18 of the row's largest on (that is
// 2^4 at least), and below is off by 2^-29 of it (2^-25 in fp16): 2^-11 of a row after 2^18 keys.  (Moves at 2^8 and P times 2^7: a
// prompt of 8192 490 us instead of 480, at 2^12 and times 2^3 470.)
//
// l has to be exact where P is not.  In fp32 an exponential is there down to 2^-126, so e is held within 2^-kReach of the
// largest of the job's scales so far, which leaves what is 2^-60 of a row's largest weight.  What a scale lies below that is
// multiplied into its values, which fp16 holds to 2^-24 (a code whole down to 2^-15; from 2^-25 on they are 0).  It happens in
// pages of zeros.
//
// With one power a tile for all of its values, and the weights against the largest so far, pages of 16 were 5 % faster (32 x 1 token
// over 8192 keys 142 us instead of 151, chunks among decoding sequences 117 instead of 123, others the same), but a page of
// large values that a row could not see took its bits.
constexpr uint32_t kReach = 60;
constexpr uint32_t kLeastExp = 15;  // and no lower, so that O's power is a number in fp32 (the codes have 2^-15, as said)

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
#pragma unroll 8
    for (int k = 0; k < kPieces; ++k) {
        const int row = k * kRows + lane / kPieces;
        const int64_t from = __shfl_sync(0xffffffffu, at, row);
        cp_async16(place(row, piece & 1, piece >> 1), q + max((long long)from, 0ll) + piece * 8, from >= 0);
    }
    cp_async_wait_all();
    __syncwarp();
    uint32_t top = 0;
#pragma unroll 8
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

// Whether one of the values of key tile [key, key + kKeys) that lie in [lo, hi) has a code that is not a number; lo and hi are of
// the lane's row, and the whole warp calls this.
template <int D>
__device__ __forceinline__ bool sees_nan(const Fp8Params& fp, const Job& g, int key, int lo, int hi) {
    const ChunkParams& p = fp.c;
    const int lane = threadIdx.x & 31;
    bool sees = false;
    for (const int end = min(g.n, key + kKeys); key < end; ++key) {
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

// The boxes that a job's key tiles come in, one a page or, of larger pages, one a tile: looked up by a whole warp, 32 boxes (a
// batch) at a time and a lane each, the next ones in flight meanwhile.  (Tile by tile, table and then scale, they alone took 1.5 us
// a tile.)  A job begins a new batch.  SCALES: one, or the keys' and the values'.
template <int SCALES>
struct Boxes {
    const ChunkParams& p;
    const uint8_t* scale[SCALES];
    const Job& g;
    int rows, of_tile, ahead;  // keys of a box; boxes of a tile; tiles of a batch
    int row;                   // this lane's box of the batch at hand: its first key's row in the pool (-1: none)
    uint32_t exponent[SCALES]; // and its scales
    uint32_t most = 0;         // the largest of the values' ones so far (the last that are looked up)
    int far_id;                // of the next batch
    uint32_t far_exponent[SCALES];

    __device__ __forceinline__ Boxes(const ChunkParams& params, const Job& job, const uint8_t* first, const uint8_t* second = nullptr)
        : p(params), g(job), rows(min(kKeys, 1 << params.page_shift)), of_tile(kKeys / rows), ahead(32 / of_tile) {
        scale[0] = first;
        if constexpr (SCALES > 1) scale[1] = second;
        look_up(g.j0);
    }
    __device__ __forceinline__ int key_of(int j) const {
        const int lane = threadIdx.x & 31;
        return (j + lane / of_tile) * kKeys + lane % of_tile * rows;
    }
    __device__ __forceinline__ void look_up(int j) {
        const int key = key_of(j), pg = key >> p.page_shift;
        far_id = -1;
#pragma unroll
        for (int i = 0; i < SCALES; ++i) far_exponent[i] = 127;
        if (key / kKeys < g.j1 && key < g.n) {
            far_id = pg < p.pages_per_seq ? __ldg(p.block_table + (size_t)g.s * p.pages_per_seq + pg) : -1;
            if ((unsigned)far_id >= (unsigned)p.num_pages) {
                raise_error(p.err, kErrDeviceArg);
                far_id = 0;
            }
#pragma unroll
            for (int i = 0; i < SCALES; ++i) far_exponent[i] = __ldg(scale[i] + (size_t)far_id * p.num_kv_heads + g.h);
        }
    }
    // The batch that begins with tile j.
    __device__ __forceinline__ void next(int j) {
        row = far_id < 0 ? -1 : (far_id << p.page_shift) + (key_of(j) & ((1 << p.page_shift) - 1));
#pragma unroll
        for (int i = 0; i < SCALES; ++i) {
            exponent[i] = far_exponent[i];
            if (exponent[i] == 255) {
                raise_error(p.err, kErrDeviceArg);
                exponent[i] = 254;
            }
        }
        most = max(most, __reduce_max_sync(0xffffffffu, row >= 0 ? exponent[SCALES - 1] : 0u));
        look_up(j + ahead);
    }
    // What the weights take of this lane's scale of values.
    __device__ __forceinline__ uint32_t of_weights() const {
        return max(max(exponent[SCALES - 1], kLeastExp), most > kReach ? most - kReach : 0u);
    }
    // The least of it in the box's tile.
    __device__ __forceinline__ uint32_t least_of_weights() const {
        uint32_t least = row >= 0 ? of_weights() : 255u;
        for (int o = 1; o < of_tile; o <<= 1) least = min(least, __shfl_xor_sync(0xffffffffu, least, o));
        return least;
    }
    // The keys of tile j's boxes.
    __device__ __forceinline__ uint32_t keys(int j) const { return min(of_tile, (g.n - j * kKeys + rows - 1) / rows) * rows; }
};
// A job's batches before the one of its tile t, and the place of that tile's box `b` in it (of boxes of 2^shift keys).
__device__ __forceinline__ unsigned batch_of(int t, int shift) { return (unsigned)t >> (shift - 2); }
__device__ __forceinline__ int in_batch(int t, int b, int shift) { return ((t << (7 - shift)) + b) & 31; }
__device__ __forceinline__ unsigned batches_of(int tiles, int shift) { return (unsigned)(tiles + (1 << (shift - 2)) - 1) >> (shift - 2); }

// The next job, for a warp that has had `nj` of them; none if there are no more (or a wait was given up: ok is false).  The
// warp reads what it needs and calls had_job.
template <class Sh>
__device__ __forceinline__ const Job* next_job(Sh& sh, unsigned nj, bool& ok) {
    ok = __all_sync(0xffffffffu, mbar_wait(&sh.job_full[nj % kJobs], (nj / kJobs) & 1, kWaitBudget));
    if (!ok) return nullptr;
    const Job* g = &sh.job[nj % kJobs];
    return g->s >= 0 ? g : nullptr;
}
template <class Sh>
__device__ __forceinline__ void had_job(Sh& sh, unsigned& nj) {
    __syncwarp();
    if ((threadIdx.x & 31) == 0) mbar_arrive(&sh.job_empty[nj % kJobs]);
    ++nj;
}

// A warp's role: this CTA's part of the line, laid out in jobs; K tiles of codes through their ring.  It brings all that the
// softmax reads of the scales, the values' too: a tile's arrival on k_full is what its scores wait for, while V's copies (and what
// their warp writes) may come later than those.
template <int D, bool FEW, class Sh>
__device__ __forceinline__ void bring_keys(const Fp8Params& fp, const CUtensorMap* kmap, Sh& sh, uint8_t* smem) {
    using S = Shape<D, FEW>;
    const ChunkParams& p = fp.c;
    const int lane = threadIdx.x & 31;
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
    unsigned x = 0, batch = 0;  // tiles asked for, batches
    Job g, after;
    for (bool have = false; ; have = true) {
        lay_out(after);  // one ahead of the copies
        if (!ok) break;
        if (have && g.j1 > g.j0) {
            Boxes<2> box(p, g, fp.k_scale, fp.v_scale);
            for (int j = g.j0; j < g.j1 && ok; ++batch) {
                box.next(j);
                sh.k_power[batch % kBatches][lane] = (uint16_t)(__float_as_uint(power_of(box.exponent[0])) >> 16);
                const uint32_t least = box.least_of_weights();
                sh.v_exp[batch % kBatches][lane] = (uint8_t)(box.row >= 0 ? box.of_weights() : least);
                sh.v_low[batch % kBatches][lane] = (uint8_t)least;
                __syncwarp();
                for (int k = 0; k < box.ahead && j < g.j1; ++k, ++j, ++x) {
                    const int slot = x % S::k_slots;
                    ok = x < (unsigned)S::k_slots || __all_sync(0xffffffffu, mbar_wait(&sh.k_empty[slot], (x / S::k_slots - 1) & 1, kWaitBudget));
                    if (!ok) break;
                    const int mine = lane - k * box.of_tile;  // this lane's box of the tile
                    if (mine == 0) mbar_arrive_expect_tx(&sh.k_full[slot], box.keys(j) * D);
                    if (mine >= 0 && mine < box.of_tile && box.row >= 0)
                        tma_load_3d(smem + S::at_k + slot * S::code_bytes + mine * box.rows * D, kmap, &sh.k_full[slot], 0, g.h, box.row);
                    __syncwarp();
                }
            }
        }
        if (!ok || after.s < 0) break;
        g = after;
    }
    if (!ok && lane == 0) raise_error(p.err, kErrTimeout);
    // no copy may still be in flight when the CTA leaves
    for (unsigned y = x > (unsigned)S::k_slots ? x - S::k_slots : 0; y < x; ++y)
        if (!mbar_wait(&sh.k_full[y % S::k_slots], (y / S::k_slots) & 1, kDrainBudget) && lane == 0) raise_error(p.err, kErrTimeout);
}

// A warp's role: V tiles of codes through their ring; what this CTA leaves to the merge.
template <int D, bool FEW, class Sh>
__device__ __forceinline__ void bring_values(const Fp8Params& fp, const CUtensorMap* vmap, Sh& sh, uint8_t* smem) {
    using S = Shape<D, FEW>;
    const ChunkParams& p = fp.c;
    const int lane = threadIdx.x & 31;
    unsigned x = 0, batch = 0, nj = 0;
    int4 left = make_int4(0, 0, 0, 0);
    bool ok, fine = true;
    while (const Job* job = next_job(sh, nj, ok)) {
        const Job g = *job;
        had_job(sh, nj);
        if (!g.first) left.x |= kHasHead | (g.last ? kHeadEnds : 0);
        if (g.first && !g.last)
            left = make_int4(left.x | kHasTail, g.q0 + g.t * 2 * p.tokens, min(2 * p.tokens, g.B - g.t * 2 * p.tokens), g.h);
        if (g.j1 <= g.j0) continue;
        Boxes<1> box(p, g, fp.v_scale);
        for (int j = g.j0; j < g.j1 && fine; ++batch) {
            box.next(j);
            sh.v_below[batch % kBatches][lane] = (uint8_t)(box.of_weights() - box.exponent[0]);
            __syncwarp();
            for (int k = 0; k < box.ahead && j < g.j1; ++k, ++j, ++x) {
                const int slot = x % S::raw_slots;
                fine = x < (unsigned)S::raw_slots || __all_sync(0xffffffffu, mbar_wait(&sh.raw_empty[slot], (x / S::raw_slots - 1) & 1, kWaitBudget));
                if (!fine) break;
                const int mine = lane - k * box.of_tile;
                if (mine == 0) mbar_arrive_expect_tx(&sh.raw_full[slot], box.keys(j) * D);
                if (mine >= 0 && mine < box.of_tile && box.row >= 0)
                    tma_load_3d(smem + S::at_raw + slot * S::code_bytes + mine * box.rows * D, vmap, &sh.raw_full[slot], 0, g.h, box.row);
                __syncwarp();
            }
        }
        if (!fine) break;
    }
    if ((!ok || !fine) && lane == 0) raise_error(p.err, kErrTimeout);
    for (unsigned y = x > (unsigned)S::raw_slots ? x - S::raw_slots : 0; y < x; ++y)
        if (!mbar_wait(&sh.raw_full[y % S::raw_slots], (y / S::raw_slots) & 1, kDrainBudget) && lane == 0) raise_error(p.err, kErrTimeout);
    if (lane == 0) p.info[blockIdx.x] = left;
}

// The role of warp w of those that turn V from codes to fp16, in shared memory: keys [32 w, 32 w + 32) of every tile.
template <int D, bool FEW, class Sh>
__device__ __forceinline__ void convert_values(const ChunkParams& p, Sh& sh, uint8_t* smem, int w) {
    using S = Shape<D, FEW>;
    // Eight lanes read all banks, and write them: a key's lower pieces of 16 codes with the next key's upper ones (form 0; 1:
    // the other way round; of 64 columns: the two keys' pieces all together).  From one piece of a lane to the next of its
    // form it is 8 keys, which the swizzle does not tell apart.
    constexpr int kForms = D == 128 ? 2 : 1, kPieces = 2 * kForms;  // pieces of 16 keys
    const int lane = threadIdx.x & 31, e = lane & 7;
    const int key0 = w * 32 + (lane >> 3) * 2 + (e >> 2);
    int from[kForms], to[kForms];
#pragma unroll
    for (int form = 0; form < kForms; ++form) {
        const int piece = (e & 3) + (D == 128 ? 4 * ((e >> 2) ^ form) : 0);
        from[form] = key0 * D + piece * 16;
        to[form] = (piece >> 2) * kHalfBytes + key0 * 128 + (((2 * (piece & 3)) ^ (key0 & 7)) << 4);
    }
    const int box_shift = min(7, p.page_shift);
    unsigned x = 0, batch0 = 0, nj = 0;
    bool ok, fine = true;
    while (const Job* g = next_job(sh, nj, ok)) {
        const int j0 = g->j0, j1 = g->j1, n = g->n;
        int* const nan = &sh.job_nan[nj % kJobs];
        had_job(sh, nj);
        for (int j = j0; j < j1; ++j, ++x) {
            const int rs = x % S::raw_slots, vs = x % S::v_slots;
            fine = __all_sync(0xffffffffu, mbar_wait(&sh.raw_full[rs], (x / S::raw_slots) & 1, kWaitBudget));
            const uint8_t* raw = smem + S::at_raw + rs * S::code_bytes;
            uint8_t* out = smem + S::at_v + vs * S::v_bytes;
            const int left = n - j * kKeys;  // keys from this one on are none: zeros
            uint32_t look[4] = {0, 0, 0, 0};
            auto power = [&](int h) {  // what half h's values are multiplied by, as fp16
                const int below = sh.v_below[(batch0 + batch_of(j - j0, box_shift)) % kBatches][in_batch(j - j0, (w * 32 + h * 16) >> box_shift, box_shift)];
                return (below < 15 ? (15 - below) << 10 : below < 25 ? 1 << (24 - below) : 0) * 0x10001u;
            };
            // (the second half of the codes set out before the wait for a place: 64 x 1 tokens over 4096 keys 140 us instead of
            // 144, a prompt of 8192 460 instead of 478)
            uint4 in[2][kPieces];
            auto bring = [&](int h) {
#pragma unroll
                for (int k = 0; k < kPieces; ++k)
                    in[h][k] = ld_shared16(raw + from[k % kForms] + (h * kPieces + k) / kForms * 8 * D);
            };
            bring(0);
#pragma unroll
            for (int h = 0; h < 2; ++h) {  // 16 keys at a time: boxes are no smaller
                uint32_t v[kPieces][4];
#pragma unroll
                for (int k = 0; k < kPieces; ++k) {
                    const uint4 c = in[h][k];
                    v[k][0] = c.x; v[k][1] = c.y; v[k][2] = c.z; v[k][3] = c.w;
                }
                if (left < kKeys) {
#pragma unroll
                    for (int k = 0; k < kPieces; ++k)
                        if (key0 + (h * kPieces + k) / kForms * 8 >= left) v[k][0] = v[k][1] = v[k][2] = v[k][3] = 0;
                }
                uint32_t y[kPieces][8];
#pragma unroll
                for (int k = 0; k < kPieces; ++k)
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        e4m3x4_to_f16x4(v[k][c], y[k][2 * c], y[k][2 * c + 1]);
                        look[c] |= (v[k][c] & 0x7f7f7f7fu) + 0x01010101u;  // bit 7 of a byte: its code is 0x7f or 0xff
                    }
                const uint32_t mul = power(h);
                if (mul != 0x3c003c00u) {
#pragma unroll
                    for (int k = 0; k < kPieces; ++k)
#pragma unroll
                        for (int c = 0; c < 8; ++c) y[k][c] = mul_f16x2(y[k][c], mul);
                }
                if (h == 0) {
                    bring(1);
                    if (fine && x >= (unsigned)S::v_slots) fine = mbar_wait(&sh.v_empty[vs], (x / S::v_slots - 1) & 1, kWaitBudget);
                    fine = __all_sync(0xffffffffu, fine);
                    if (!fine) break;
                }
#pragma unroll
                for (int k = 0; k < kPieces; ++k) {
                    uint8_t* const at = out + (h * kPieces + k) / kForms * 1024;
                    *reinterpret_cast<uint4*>(at + to[k % kForms]) = make_uint4(y[k][0], y[k][1], y[k][2], y[k][3]);
                    *reinterpret_cast<uint4*>(at + (to[k % kForms] ^ 16)) = make_uint4(y[k][4], y[k][5], y[k][6], y[k][7]);
                }
            }
            if (!fine) break;
            // 0 in the place of what is not a number: rare, and after all is stored (with a vote before it 64 x 1 tokens over
            // 4096 keys took 187 us instead of 147).
            if ((look[0] | look[1] | look[2] | look[3]) & 0x80808080u) {
#pragma unroll 1
                for (int k = 0; k < 2 * kPieces; ++k) {
                    const int form = k % kForms, at = k / kForms * 1024;
                    const uint4 c = *reinterpret_cast<const uint4*>(raw + from[0] + (form ? from[kForms - 1] - from[0] : 0) + k / kForms * 8 * D);
                    uint8_t* const piece = out + (form ? to[kForms - 1] : to[0]) + at;
                    if (key0 + k / kForms * 8 >= left) continue;
                    const uint32_t v[4] = {c.x, c.y, c.z, c.w}, mul = power(k / kPieces);
                    uint32_t y[8], none = 0;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        e4m3x4_to_f16x4(v[i], y[2 * i], y[2 * i + 1]);
                        none |= ((v[i] & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;
                    }
                    if (!none) continue;
                    *nan = 1;  // (the softmax warps look once all of the job's values have been used)
#pragma unroll
                    for (int i = 0; i < 8; ++i) y[i] = mul_f16x2(drop_nan_f16x2(y[i]), mul);
                    *reinterpret_cast<uint4*>(piece) = make_uint4(y[0], y[1], y[2], y[3]);
                    *reinterpret_cast<uint4*>(out + ((form ? to[kForms - 1] : to[0]) ^ 16) + at) = make_uint4(y[4], y[5], y[6], y[7]);
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
        batch0 += batches_of(max(0, j1 - j0), box_shift);
    }
    if ((!fine || !ok) && lane == 0) raise_error(p.err, kErrTimeout);
}

// What both kernels begin with: barriers, tensor memory; false where the shared memory is not as they need it.
template <int D, bool FEW, class Sh>
__device__ __forceinline__ bool begin(const ChunkParams& p, const CUtensorMap* kmap, const CUtensorMap* vmap, Sh& sh, uint8_t* smem,
                                      int arrivals_empty) {
    using S = Shape<D, FEW>;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    if (smem_addr(smem) & 1023) {  // (the swizzled tiles' alignment: dynamic shared memory starts on such a boundary)
        if (tid == 0) raise_error(p.err, kErrDeviceArg);
        return false;
    }
    if (tid == 0) {
        for (int i = 0; i < S::k_slots; ++i) {
            mbar_init(&sh.k_full[i], 1);
            mbar_init(&sh.k_empty[i], arrivals_empty);
        }
        for (int i = 0; i < S::raw_slots; ++i) {
            mbar_init(&sh.raw_full[i], 1);
            mbar_init(&sh.raw_empty[i], kConvertWarps);
        }
        for (int i = 0; i < S::v_slots; ++i) {
            mbar_init(&sh.v_full[i], kConvertWarps);
            mbar_init(&sh.v_empty[i], arrivals_empty);
        }
        for (int i = 0; i < kJobs; ++i) {
            mbar_init(&sh.job_full[i], 1);
            mbar_init(&sh.job_empty[i], kSoftmaxWarps + arrivals_empty + 1 + kConvertWarps);  // (the MMA warps, V's)
        }
        sh.init();
        fence_mbar_init();
    }
    if (warp == kMmaWarp) {
        tmem_alloc(&sh.tmem, kChunkTmem);
        tmem_relinquish();
    }
    if (warp == kKeyWarp && lane < 2) prefetch_tensormap(lane == 0 ? kmap : vmap);
    griddep_wait();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    griddep_launch_dependents();
    return true;
}

// M and m of a row that has seen nothing: below every score, and a number, so that no weight needs a test.
constexpr float kNothing = -3.0e38f;
// A whole number below 2^8 as 2^23 more, from its bits alone (a conversion would take the exponentials' pipe).
__device__ __forceinline__ float plus_2_23(uint32_t e) { return __uint_as_float(0x4b000000u | e); }

// What both softmaxes do with a tile's scores.  P = 2^(f * x + e + base) of a row's columns [64 h, 64 h + 64), in pairs, fp16 as the
// converted values are, to tensor memory at `to`; their sums times 2^(low - e) to sum2.  The e as plus_2_23, at least low; base
// is 2^23 lower.  APART: the 64 columns have one e, which their sum takes at the end (the block kernel with large pages, 64 x 1 tokens over
// 4096 keys, 142 us and 146 with each pair's own; the other kernel the other way round, a prompt of 8192 459 and 443).
template <int FACTORS, bool APART>
__device__ __forceinline__ void weigh(const uint32_t (&x)[4][16], const float (&f)[FACTORS], const float (&e)[FACTORS], int h, float base,
                                      uint32_t low, uint64_t (&sum2)[2], uint32_t to) {
    static_assert(!APART || FACTORS == 2, "one e");
    uint64_t apart[2] = {0ull, 0ull};
    // 2^(low - e): of e's bits the lowest 8 are left, at the exponent's place
    auto below = [&](int i) { return __uint_as_float(((127 + low) << 23) + __float_as_uint(e[i]) * 0xff800000u); };
#pragma unroll
    for (int c = 0; c < 4; c += 2) {
        uint32_t pk[16];
#pragma unroll
        for (int k = 0; k < 16; ++k) {
            const int block = c + (k >> 3), i = (h * 4 + block) * FACTORS / 8;
            const float factor = f[i], add = base + e[i], part = below(i);
            const uint32_t* y = &x[block][2 * (k & 7)];
            float u, w;
            unpack_f32x2(fma_f32x2(pack_f32x2(__uint_as_float(y[0]), __uint_as_float(y[1])), pack_f32x2(factor, factor), pack_f32x2(add, add)), u, w);
            u = chunk_exp2(u);
            w = chunk_exp2(w);
            if constexpr (APART) apart[k & 1] = add_f32x2(apart[k & 1], pack_f32x2(u, w));
            else sum2[k & 1] = fma_f32x2(pack_f32x2(u, w), pack_f32x2(part, part), sum2[k & 1]);
            pk[k] = pack_f16x2(u, w);  // 11 bits
        }
        tmem_st16(to + h * 32 + c * 8, pk);
    }
    if constexpr (APART) sum2[0] = fma_f32x2(add_f32x2(apart[0], apart[1]), pack_f32x2(below(h), below(h)), sum2[0]);
}
// Scores of columns [64 h, 64 h + 64) at `at`, those outside [from, to) struck out unless the whole tile is seen; the maxima
// of 16 columns each.
__device__ __forceinline__ void take_scores(uint32_t at, int h, bool full, int from, int to, uint32_t (&x)[4][16], float (&mx)[4]) {
    if (full) {
#pragma unroll
        for (int c = 0; c < 4; ++c) tmem_ld16_max(at + h * 64 + c * 16, x[c], mx[c]);
        tmem_ld_wait();
    } else {
#pragma unroll
        for (int c = 0; c < 4; ++c) tmem_ld16(at + h * 64 + c * 16, x[c]);
        tmem_ld_wait();
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            mx[c] = -INFINITY;
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                if (h * 64 + c * 16 + e < from || h * 64 + c * 16 + e >= to) x[c][e] = 0xff800000u;  // -inf
                mx[c] = fmaxf(mx[c], __uint_as_float(x[c][e]));
            }
        }
    }
}
// The factors of a tile's scores and the values' powers, of kKeys / FACTORS keys each; the tile's boxes begin at place `at` of the
// batch.  Factors are finite and above 0, so that a hidden column's -inf stays one.
template <int FACTORS, class Sh>
__device__ __forceinline__ void take_scales(const Sh& sh, unsigned batch, int at, int box_shift, float row_scale, float (&f)[FACTORS],
                                            float (&e)[FACTORS]) {
    auto factor = [&](uint32_t power) { return fmaxf(fminf(row_scale * __uint_as_float(power), 3.4e38f), 1.2e-38f); };
    if constexpr (FACTORS == 8) {  // pages of 16 or 32: of their 8 or 4 boxes at once
        uint32_t k[4], v[2];
        if (box_shift == 4) {
            const uint4 a = *reinterpret_cast<const uint4*>(&sh.k_power[batch][at]);
            const uint2 b = *reinterpret_cast<const uint2*>(&sh.v_exp[batch][at]);
            k[0] = a.x, k[1] = a.y, k[2] = a.z, k[3] = a.w, v[0] = b.x, v[1] = b.y;
        } else {
            const uint2 a = *reinterpret_cast<const uint2*>(&sh.k_power[batch][at]);
            const uint32_t b = *reinterpret_cast<const uint32_t*>(&sh.v_exp[batch][at]);
            k[0] = __byte_perm(a.x, 0, 0x1010), k[1] = __byte_perm(a.x, 0, 0x3232);
            k[2] = __byte_perm(a.y, 0, 0x1010), k[3] = __byte_perm(a.y, 0, 0x3232);
            v[0] = __byte_perm(b, 0, 0x1100), v[1] = __byte_perm(b, 0, 0x3322);
        }
#pragma unroll
        for (int c = 0; c < 8; ++c) {
            f[c] = factor(c & 1 ? k[c >> 1] & 0xffff0000u : k[c >> 1] << 16);
            e[c] = __uint_as_float(__byte_perm(v[c >> 2], 0x4b000000u, 0x7540 | (c & 3)));  // plus_2_23
        }
    } else {
#pragma unroll
        for (int c = 0; c < FACTORS; ++c) {
            const int box = at + (c * (kKeys / FACTORS) >> box_shift);
            f[c] = factor((uint32_t)sh.k_power[batch][box] << 16);
            e[c] = plus_2_23(sh.v_exp[batch][box]);
        }
    }
}
// The largest of a row's scores times their factors, of the 16 columns' maxima, with the values' powers: 2^23 more, and so rounded to
// whole numbers (below 0: halves).
template <int FACTORS>
__device__ __forceinline__ float top_score(const float (&lower)[4], const float (&upper)[4], const float (&f)[FACTORS],
                                           const float (&e)[FACTORS]) {
    float top = -INFINITY;
#pragma unroll
    for (int i = 0; i < FACTORS; ++i) {
        float most;
        if constexpr (FACTORS == 2) {
            const float (&m)[4] = i ? upper : lower;
            most = fmaxf(fmaxf(m[0], m[1]), fmaxf(m[2], m[3]));
        } else {
            most = i < 4 ? lower[i & 3] : upper[i & 3];
        }
        top = fmaxf(top, fmaf(most, f[i], e[i]));
    }
    return top;
}
// A row's sum, moved where `top`, which no score of a tile is above, has outgrown m.
__device__ __forceinline__ void move_sum(float top, float& m, float& l) {
    if (top > m + 10.f) {
        const float m_new = ceilf(top);
        l *= chunk_exp2(m - m_new);
        m = m_new;
    }
}
// M - m of a row, 0 where its scores overflow.
__device__ __forceinline__ int power_between(float M, float m) { return M < INFINITY ? (int)fmaxf(M - m, -1e6f) : 0; }
// A row's (m, l) with l in [1/2, 1): what it weighs is then no larger than the values, and log2 l is small.  Returns what m grew by.
__device__ __forceinline__ int level(float& m, float& l) {
    if (m == kNothing) m = -INFINITY;
    const uint32_t e = __float_as_uint(l) >> 23;
    if (e - 1u >= 254u) return 0;  // 0, or not a number
    const int k = (int)e - 126;
    m += (float)k;
    l = __uint_as_float(__float_as_uint(l) - ((uint32_t)k << 23));
    return k;
}
// The accumulator's columns of a warp's rows times alpha.
template <int D>
__device__ __forceinline__ void rescale(uint32_t o_addr, float alpha) {
#pragma unroll 1
    for (int c = 0; c < D / 16; ++c) {
        uint32_t v[16];
        tmem_ld16(o_addr + c * 16, v);
        tmem_ld_wait();
#pragma unroll
        for (int e = 0; e < 16; ++e) v[e] = __float_as_uint(__uint_as_float(v[e]) * alpha);
        tmem_st16(o_addr + c * 16, v);
    }
}

// Shared memory of chunk_attention_fp8_kernel behind the tiles.
template <int D>
struct Shared : Common<D, false> {
    uint64_t q_ready[2], drain[2], turn[2];
    uint64_t s[2], half[2], p[2], o[2];              // of a stream: scores, a half of the weights, all of them, the accumulator
    __device__ void init() {
        for (int i = 0; i < 2; ++i) {
            mbar_init(&q_ready[i], 4);
            mbar_init(&half[i], 4);
            mbar_init(&s[i], 1);
            mbar_init(&p[i], 4);
            mbar_init(&o[i], 1);
            mbar_init(&drain[i], 1);
            mbar_init(&turn[i], 1);
        }
    }
};
template <int D>
constexpr int chunk_smem() { return whole_sm(Shape<D, false>::tiles + (int)sizeof(Shared<D>)); }
static_assert(chunk_smem<128>() <= 227 * 1024 && chunk_smem<64>() <= 227 * 1024, "a block's shared memory");

// FACTORS: scales that a tile of 128 keys may have: 8 with pages of 16, 2 from pages of 64 on.
template <int D, int FACTORS>
__global__ void __launch_bounds__(kThreads, 1)
chunk_attention_fp8_kernel(const __grid_constant__ Fp8Params fp, const __grid_constant__ CUtensorMap kmap,
                           const __grid_constant__ CUtensorMap vmap) {
    using S = Shape<D, false>;
    constexpr uint32_t kColO = 256;  // O of stream i: columns kColO + i * D
    const ChunkParams& p = fp.c;
    extern __shared__ __align__(1024) uint8_t smem[];
    Shared<D>& sh = *reinterpret_cast<Shared<D>*>(smem + S::tiles);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int G = p.group;
    if (!begin<D, false>(p, &kmap, &vmap, sh, smem, 2)) return;
    const uint32_t tmem = sh.tmem;
    // Of a split job's streams, a row's m, l and its accumulator's power: where the second query tile is otherwise, those of 32 rows
    // where these rows' queries are.  The two warps that have the rows write and read both, and their barriers are the only ones in
    // between.
    constexpr int kRowsBytes = 32 * 128;  // of 32 rows of a query tile (its first part)
    static_assert(2 * 32 * sizeof(float4) <= kRowsBytes && 4 * kRowsBytes <= S::q_bytes, "a warp's rows hold them");
    auto row = [&](int stream, int r) -> float4& {
        return reinterpret_cast<float4*>(smem + S::q_bytes + (r >> 5) * kRowsBytes)[stream * 32 + (r & 31)];
    };
    // whether a job's rows are one stream's: then both take them, and every other key tile
    auto is_split = [&](const Job& g) { return g.t * 2 * p.tokens + p.tokens >= g.B; };

    if (warp < kSoftmaxWarps) {
        regs_inc<kRegs.softmax>();
        // ================= softmax of stream i: a thread a row
        const int i = warp >> 2, quad = warp & 3, r = quad * 32 + lane;
        const uint32_t lanes = tmem + (static_cast<uint32_t>(quad * 32) << 16);
        const uint32_t s_addr = lanes + i * 128;  // P comes over the scores
        const int my_tok = r / G;
        const int box_shift = min(7, p.page_shift);
        unsigned ns = 0, no = 0, batch0 = 0;  // scores and accumulators waited for; batches of the jobs before
        bool failed = false;
        unsigned nj = 0;
        for (;;) {
            bool ok = false;
            const Job* g = failed ? nullptr : next_job(sh, nj, ok);
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
            float M = kNothing, m = kNothing, l = 0.f, row_scale = 1.f;
            if (j1 > j0 && b > a && !idle) {
                // ---- the queries of this warp's rows, two parts each, to shared memory
                const int64_t at = active ? (int64_t)(g->q0 + tok) * fp.q_stride + (g->h * G + r - my_tok * G) * D : -1;
                uint32_t top = 0;
                if (mine == i) top = split_queries<D>(fp.q, at, smem + i * S::q_bytes + quad * 32 * 128);
                if (split) {  // (the other stream's threads learn of it, where they themselves write their sums later)
                    if (i == 0) row(1, r).x = __uint_as_float(top);
                    named_barrier(1 + quad, 64);
                    if (i == 1) top = __float_as_uint(row(1, r).x);
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
#pragma unroll 1
            for (int j = from_j; j < b; j += step, ++ns, from -= step * kKeys, to -= step * kKeys) {
                failed = !__all_sync(0xffffffffu, mbar_wait(&sh.s[i], ns & 1, kWaitBudget));
                if (failed) break;
                tc_fence_after();
                if (!idle) {
                    const bool full = __all_sync(0xffffffffu, from <= 0 && to >= kKeys);
                    const unsigned batch = (batch0 + batch_of(j - j0, box_shift)) % kBatches;
                    const int boxes = in_batch(j - j0, 0, box_shift);
                    float f[FACTORS], e[FACTORS];
                    take_scales<FACTORS>(sh, batch, boxes, box_shift, row_scale, f, e);
                    uint32_t lower[4][16], upper[4][16];
                    float mx[2][4];
                    take_scores(s_addr, 0, full, from, to, lower, mx[0]);
                    take_scores(s_addr, 1, full, from, to, upper, mx[1]);
                    float top = top_score<FACTORS>(mx[0], mx[1], f, e);
                    const uint32_t low = sh.v_low[batch][boxes];
                    move_sum(top - plus_2_23(low), m, l);
                    top -= 8388608.f;
                    // (with this M, P stays below 2^16)
                    if (__any_sync(0xffffffffu, top > M + 10.f)) {
                        // (all of the warp's rows, those that need not too: their next move is later for it; a prompt of 8192
                        // with 2^8 490 us, 521 with each row moved for itself)
                        const float M_old = M;
                        M = fmaxf(M, ceilf(top));
                        // (this tile's scores are complete, so the stream's MMAs before them, the last P V among them, are too)
                        if (j > from_j) rescale<D>(lanes + kColO + i * D, M > M_old ? chunk_exp2(M_old - M) : 1.f);
                    }
                    // P in pairs over the scores, and its sum
                    const float base = 5.f - 8388608.f - M;
                    uint64_t sum2[2] = {0ull, 0ull};
                    weigh<FACTORS, false>(lower, f, e, 0, base, low, sum2, s_addr);
                    // (their P V begins; a prompt of 8192, when this was built, 538 us without, 520 with)
                    tmem_st_wait();
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&sh.half[i]);
                    weigh<FACTORS, false>(upper, f, e, 1, base, low, sum2, s_addr);
                    float u, w;
                    unpack_f32x2(add_f32x2(sum2[0], sum2[1]), u, w);
                    l = fmaf(u + w, chunk_exp2(M - m - 5.f - (float)low), l);
                    tmem_st_wait();
                } else if (lane == 0) {
                    mbar_arrive(&sh.half[i]);
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
            batch0 += batches_of(max(0, j1 - j0), box_shift);
            if (!split && failed) continue;
            // the weights of the streams' accumulators, and their powers of two
            float w_mine = some ? 1.f : 0.f, w_other = 0.f;
            int unit_mine = power_between(M, m) - 132, unit_other = 0;
            unit_mine -= level(m, l);
            bool others_some = false;
            if (split) {
                // ---- the other stream's part of these rows, merged as the second kernel merges CTAs' parts
                row(i, r) = make_float4(m, l, __int_as_float(unit_mine), 0.f);
                if (named_barrier_or(1 + quad, 64, failed)) {
                    failed = true;
                    continue;
                }
                others_some = a + (i ^ 1) < b;
                const float4 o = row(i ^ 1, r);
                const float top = fmaxf(m, o.x);
                const float u = m == top ? 1.f : chunk_exp2(m - top), v = o.x == top ? 1.f : chunk_exp2(o.x - top);
                l = i == 0 ? l * u + o.y * v : o.y * v + l * u;
                m = top;
                w_mine *= u;
                if (others_some) w_other = v, unit_other = __float_as_int(o.z);
            }
            const bool first = g->first, whole = first && g->last;
            // the query row's number among all, in the output (-1: none)
            const long long orow = active ? (long long)(g->q0 + tok) * p.num_q_heads + g->h * G + r - my_tok * G : -1;
            had_job(sh, nj);
            const float inv = whole ? row_inverse(m, l) : 1.f;
            w_mine = ldexpf(w_mine * inv, unit_mine);
            w_other = ldexpf(w_other * inv, unit_other);
            const size_t slot = (size_t)blockIdx.x * 2 + (first ? 1 : 0);
            if (!idle) {
                // (a split job's two warps have half of the columns each)
                const uint32_t o_addr = lanes + kColO;
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
    } else if (warp >= kConvertWarp) {
        regs_dec<kRegs.convert>();
        convert_values<D, false>(p, sh, smem, warp - kConvertWarp);
    } else {
        regs_dec<kRegs.other>();
        if (warp == kKeyWarp) {
            bring_keys<D, false>(fp, &kmap, sh, smem);
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
            const uint32_t t_s = tmem + i * 128, t_o = tmem + kColO + i * D;
            // this stream's arrivals on `bar`: when its MMAs so far are done, or at once if it had none there; a split job's
            // tiles are one stream's, which arrives for the other one too
            auto release = [&](uint64_t* bar, bool used, bool both) {
                if (both) mbar_arrive(bar);
                if (used) umma_commit(bar); else mbar_arrive(bar);
            };
            unsigned x = 0;  // key tiles of the jobs before
            unsigned nj = 0, np = 0, turn = 0, nq0 = 0, nq1 = 0;
            bool ok, fine = true, any = false;
            while (const Job* g = next_job(sh, nj, ok)) {
                const bool split = is_split(*g);
                const int mine = split ? 0 : i;
                const int a = g->a[mine], b = g->b[mine], j0 = g->j0, j1 = g->j1;
                had_job(sh, nj);
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
                        // (the turn before the weights: a wait takes 100 to 200 cycles even where there is nothing to wait
                        // for, and after the weights they are on the chain: 556 us, then, instead of 538)
                        if (fine) fine = mbar_wait(&sh.turn[i], ((turn + k) & 1) ^ (i ^ 1), kWaitBudget);
                        if (fine && pv) fine = mbar_wait(&sh.half[i], my_p & 1, kWaitBudget);
                        if (!fine) break;
                        tc_fence_after();
                        if (pv) {  // O += P V of tile jp
                            const uint32_t vl = v_lo + vslot * (S::v_bytes >> 4);
                            uint32_t on = jp > first ? 1u : 0u;
#pragma unroll
                            for (int kk = 0; kk < kKeys / 16; ++kk) {
                                if (kk == kKeys / 32) {
                                    fine = mbar_wait(&sh.p[i], my_p++ & 1, kWaitBudget);
                                    if (!fine) break;
                                    tc_fence_after();
                                }
                                umma_ts(t_o, t_s + kk * 8, upper | (vl + kk * (2048 >> 4)), id_o, on);
                                on = 1;
                            }
                        }
                        if (!fine) break;
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
        } else {
            bring_values<D, false>(fp, &vmap, sh, smem);
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == kMmaWarp) {
        tc_fence_after();
        tmem_dealloc(tmem, kChunkTmem);
    }
}

// Shared memory of block_attention_fp8_kernel behind the tiles.
template <int D>
struct BlockShared : Common<D, true> {
    uint64_t q_ready, drain, o;
    uint64_t s[3], p[3];                             // of a score buffer: scores, weights
    uint64_t decided[4][2];                          // of 32 rows, by the tile's parity: what follows is as after it
    float top[kTileM];                               // of a row: M so far
    uint32_t size[kTileM];                           // the bits of a row's largest query element
    __device__ void init() {
        mbar_init(&q_ready, 4);
        mbar_init(&drain, 1);
        mbar_init(&o, 1);
        for (int i = 0; i < 3; ++i) {
            mbar_init(&s[i], 1);
            mbar_init(&p[i], 4);
        }
        for (int i = 0; i < 8; ++i) mbar_init(&decided[i >> 1][i & 1], 1);
    }
};
template <int D>
constexpr int block_smem() { return whole_sm(Shape<D, true>::tiles + (int)sizeof(BlockShared<D>)); }
static_assert(block_smem<128>() <= 227 * 1024 && block_smem<64>() <= 227 * 1024, "a block's shared memory");

// The same where every work tile has the rows of one stream: blocks and single tokens, whose keys' bytes are what counts.
// Against the kernel above, us with a cold L2: 32 x 1 token over 8192 keys in pages of 16 151 (173), 64 x 1 over 4096 140 (164),
// 32 x 16 over 2048 81 (85), 8 x 16 over 32768 129 (131); 8 x 31 over 32768 139 (138), 1 x 31 52 (50).  One
// accumulator; scores in three buffers, so that a tile's are there before the softmax has done with the two before it.  The
// softmax's two groups of warps take the tiles in turn, each row's maximum handed from one tile's thread to the next one's
// (rarely another: it is moved only where a score has outgrown it by 2^10, and the accumulator with it).
template <int D, int FACTORS>
__global__ void __launch_bounds__(kThreads, 1)
block_attention_fp8_kernel(const __grid_constant__ Fp8Params fp, const __grid_constant__ CUtensorMap kmap,
                           const __grid_constant__ CUtensorMap vmap) {
    using S = Shape<D, true>;
    constexpr uint32_t kColO = 384;  // behind the score buffers
    const ChunkParams& p = fp.c;
    extern __shared__ __align__(1024) uint8_t smem[];
    BlockShared<D>& sh = *reinterpret_cast<BlockShared<D>*>(smem + S::tiles);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int G = p.group;
    if (!begin<D, true>(p, &kmap, &vmap, sh, smem, 1)) return;
    const uint32_t tmem = sh.tmem;
    // At a job's end a row's m and l, of the two groups of warps: where its queries were (the job's MMAs are done; the two warps
    // that have 32 rows read both before one of them brings the next queries there).
    constexpr int kRowsBytes = 32 * 128;
    static_assert(2 * 32 * sizeof(float2) <= kRowsBytes && 4 * kRowsBytes <= S::q_bytes, "a warp's rows hold them");
    auto row = [&](int group, int r) -> float2& { return reinterpret_cast<float2*>(smem + (r >> 5) * kRowsBytes)[group * 32 + (r & 31)]; };

    if (warp < kSoftmaxWarps) {
        regs_inc<kBlockRegs.softmax>();
        // ================= softmax of the tiles of parity i: a thread a row
        const int i = warp >> 2, quad = warp & 3, r = quad * 32 + lane;
        const uint32_t lanes = tmem + (static_cast<uint32_t>(quad * 32) << 16);
        const int my_tok = r / G;
        const int box_shift = min(7, p.page_shift);
        unsigned x0 = 0, no = 0, batch0 = 0;  // key tiles of the jobs before; accumulators waited for; batches before
        unsigned nd[2] = {0, 0};              // decisions of either group before
        bool failed = false;
        unsigned nj = 0;
        for (;;) {
            bool ok = false;
            const Job* g = failed ? nullptr : next_job(sh, nj, ok);
            // (a warp that gave up a wait takes the other group's of its rows along, here and at a job's end)
            if (named_barrier_or(1 + quad, 64, !ok)) {
                failed = true;
                break;
            }
            if (!g) break;
            const int j0 = g->j0, tiles = max(0, g->j1 - j0);
            const int tok = g->t * 2 * p.tokens + my_tok;
            const bool active = my_tok < p.tokens && tok < g->B;
            const int pos = g->n - g->B + tok;  // (what the end needs of the job is read again there)
            // (rows of none count as seeing all: their warps' tiles are not masked for their sake)
            const int hi = !active ? 0x7fffffff : p.causal ? max(0, pos + 1) : g->n;
            const int lo = active && p.window > 0 ? max(0, pos + 1 - p.window) : 0;
            const bool idle = !__any_sync(0xffffffffu, active);  // the same in both warps of these rows
            float M = kNothing, m = kNothing, l = 0.f, row_scale = 1.f;  // (m and l of this group's tiles)
            if (tiles > 0) {
                if (!idle) {
                    // ---- the queries of these rows, two parts each, to shared memory; the other group learns of their size
                    uint32_t top = 0;
                    if (i == 0) {
                        const int64_t at = active ? (int64_t)(g->q0 + tok) * fp.q_stride + (g->h * G + r - my_tok * G) * D : -1;
                        top = split_queries<D>(fp.q, at, smem + quad * 32 * 128);
                        sh.size[r] = top;
                    }
                    named_barrier(1 + quad, 64);
                    if (i == 1) top = sh.size[r];
                    // the row times 2^(7 - e) is below 256; 2^(e - 7) of it is put back with the softmax's scale
                    row_scale = p.scale_log2 * __uint_as_float((max(top >> 7, 8u) - 7) << 23);
                    if (top >= 0x7f80u && hi > lo) l = __uint_as_float(0x7fc00000u);  // a NaN or an infinity: the row is none
                }
                if (i == 0) {
                    fence_proxy_async_smem();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&sh.q_ready);
                }
            }
            int from = lo - (j0 + i) * kKeys, to = hi - (j0 + i) * kKeys;  // columns that the row sees
#pragma unroll 1
            for (int t = i; t < tiles; t += 2, from -= 2 * kKeys, to -= 2 * kKeys) {
                const unsigned x = x0 + t;
                const uint32_t s_addr = lanes + x % 3 * 128;  // P comes over the scores
                failed = !__all_sync(0xffffffffu, mbar_wait(&sh.s[x % 3], (x / 3) & 1, kWaitBudget));
                if (failed) break;
                tc_fence_after();
                if (!idle) {
                    const bool full = __all_sync(0xffffffffu, from <= 0 && to >= kKeys);
                    const unsigned batch = (batch0 + batch_of(t, box_shift)) % kBatches;
                    const int boxes = in_batch(t, 0, box_shift);
                    float f[FACTORS], e[FACTORS];
                    take_scales<FACTORS>(sh, batch, boxes, box_shift, row_scale, f, e);
                    uint32_t lower[4][16], upper[4][16];
                    float mx[2][4];
                    take_scores(s_addr, 0, full, from, to, lower, mx[0]);
                    take_scores(s_addr, 1, full, from, to, upper, mx[1]);
                    const float top_low = top_score<FACTORS>(mx[0], mx[1], f, e), top = top_low - 8388608.f;
                    // ---- M as the tile before left it
                    float M_old = kNothing;
                    if (t > 0) {
                        failed = !__all_sync(0xffffffffu, mbar_wait(&sh.decided[quad][i ^ 1], (nd[i ^ 1] + ((t - 1) >> 1)) & 1, kWaitBudget));
                        if (failed) break;
                        M_old = sh.top[r];
                        __syncwarp();
                    }
                    // (with this M, P stays below 2^16)
                    M = __any_sync(0xffffffffu, top > M_old + 10.f) ? fmaxf(M_old, ceilf(top)) : M_old;
                    const bool grew = M > M_old;
                    const bool moves = t > 0 && __any_sync(0xffffffffu, grew && M_old != kNothing);
                    if (t == 0 || grew) sh.top[r] = M;
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&sh.decided[quad][i]);
                    if (moves) {  // the accumulator with them, once the tile before is in it
                        failed = !__all_sync(0xffffffffu, mbar_wait(&sh.v_empty[(x - 1) % S::v_slots], ((x - 1) / S::v_slots) & 1, kWaitBudget));
                        if (failed) break;
                        tc_fence_after();
                        rescale<D>(lanes + kColO, grew ? chunk_exp2(M_old - M) : 1.f);
                    }
                    const uint32_t low = sh.v_low[batch][boxes];
                    move_sum(top_low - plus_2_23(low), m, l);
                    // P over the scores, and its sum
                    const float base = 5.f - 8388608.f - M;
                    uint64_t sum2[2] = {0ull, 0ull};
                    weigh<FACTORS, FACTORS == 2>(lower, f, e, 0, base, low, sum2, s_addr);
                    weigh<FACTORS, FACTORS == 2>(upper, f, e, 1, base, low, sum2, s_addr);
                    float u, w;
                    unpack_f32x2(add_f32x2(sum2[0], sum2[1]), u, w);
                    // (M is of both groups' tiles and m of this one's: where they are that far apart, these weights are nothing)
                    l = fmaf(u + w, chunk_exp2(fminf(M - m - 5.f - (float)low, 127.f)), l);
                    tmem_st_wait();
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&sh.p[x % 3]);
            }
            if (!failed && tiles > 0) {
                failed = !__all_sync(0xffffffffu, mbar_wait(&sh.o, no & 1, kWaitBudget));
                ++no;
                tc_fence_after();
                // A value that is none, in a key that the row sees, makes the row none (the tiles' weights of it are 0, and its
                // values too).  Rare: the codes are read again to find which keys have one.
                if (*const_cast<volatile int*>(&sh.job_nan[nj % kJobs]) && !idle)
                    for (int t = i; t < tiles; t += 2)
                        if (sees_nan<D>(fp, *g, (j0 + t) * kKeys, lo, hi)) l = __uint_as_float(0x7fc00000u);
            }
            x0 += tiles;
            batch0 += batches_of(tiles, box_shift);
            if (!idle) {  // (idle warps decide nothing)
                nd[0] += (tiles + 1) >> 1;
                nd[1] += tiles >> 1;
            }
            // ---- the sums of both groups' tiles
            if (tiles > 0 && !idle) M = sh.top[r];
            row(i, r) = make_float2(m, l);
            if (named_barrier_or(1 + quad, 64, failed)) {
                failed = true;
                continue;
            }
            {
                const float2 x = row(0, r), y = row(1, r);
                m = fmaxf(x.x, y.x);
                l = x.y * (x.x == m ? 1.f : chunk_exp2(x.x - m)) + y.y * (y.x == m ? 1.f : chunk_exp2(y.x - m));
            }
            int unit = power_between(M, m) - 132;
            unit -= level(m, l);
            const bool first = g->first, whole = first && g->last;
            // the query row's number among all, in the output (-1: none)
            const long long orow = active ? (long long)(g->q0 + tok) * p.num_q_heads + g->h * G + r - my_tok * G : -1;
            had_job(sh, nj);
            const float weight = tiles > 0 ? ldexpf(whole ? row_inverse(m, l) : 1.f, unit) : 0.f;
            const size_t slot = (size_t)blockIdx.x * 2 + (first ? 1 : 0);
            if (!idle)  // (each group has half of the columns)
                write_rows<D>(p, tiles > 0 ? lanes + kColO : 0, 0, weight, 0.f, i * (D / 2), (i + 1) * (D / 2), whole, orow, slot, r);
            if (active && i == 0) {
                if (!whole) p.part_ml[slot * (2 * kTileM) + r] = make_float2(m, l);
                else if (p.lse) p.lse[orow] = row_lse(m, l);
            }
            tc_fence_before();
        }
        if (failed && lane == 0) raise_error(p.err, kErrTimeout);
    } else if (warp >= kConvertWarp) {
        regs_dec<kBlockRegs.convert>();
        convert_values<D, true>(p, sh, smem, warp - kConvertWarp);
    } else {
        regs_dec<kBlockRegs.other>();
        if (warp == kKeyWarp) {
            bring_keys<D, true>(fp, &kmap, sh, smem);
        } else if (warp == kMmaWarp) {
            // ================= MMA issuer: a tile's P V, then Q K^T of the tile that has its score buffer next
            const uint32_t id_s = idesc_e4m3_f32(kTileM, kKeys);
            const uint32_t id_o = idesc_f16_f32(kTileM, D, false, true);
            // descriptors of the query tile, of the rings' first slots as K and as V: their upper halves are constant, an
            // offset adds its 16-byte units to the lower ones
            const uint64_t upper = smem_desc(0, 0, 1024, kSwizzle128B);
            const uint64_t k_upper = D == 128 ? upper : smem_desc(0, 0, 512, kSwizzle64B);
            const uint32_t q_lo = (uint32_t)smem_desc(smem_addr(smem), 16, 0, 0);
            const uint32_t k_lo = (uint32_t)smem_desc(smem_addr(smem + S::at_k), 16, 0, 0);
            const uint32_t v_lo = (uint32_t)smem_desc(smem_addr(smem + S::at_v), kHalfBytes, 0, 0);
            unsigned x0 = 0, nj = 0, nq = 0;  // key tiles of the jobs before; jobs; those with queries
            bool ok, fine = true;
            while (const Job* g = next_job(sh, nj, ok)) {
                const int tiles = max(0, g->j1 - g->j0);
                had_job(sh, nj);
                if (tiles == 0) continue;
                if (elect_one()) {  // one thread throughout: its waits need no votes
                    fine = mbar_wait(&sh.q_ready, nq & 1, kWaitBudget);
                    for (int t = -3; t < tiles && fine; ++t) {  // P V of tile t, Q K^T of tile t + 3
                        if (t >= 0) {
                            const unsigned x = x0 + t;
                            const int slot = x % S::v_slots;
                            fine = mbar_wait(&sh.v_full[slot], (x / S::v_slots) & 1, kWaitBudget) &&
                                   mbar_wait(&sh.p[x % 3], (x / 3) & 1, kWaitBudget);
                            if (!fine) break;
                            tc_fence_after();
                            const uint32_t vl = v_lo + slot * (S::v_bytes >> 4), t_p = tmem + x % 3 * 128;
                            uint32_t on = t > 0 ? 1u : 0u;
#pragma unroll
                            for (int kk = 0; kk < kKeys / 16; ++kk) {
                                umma_ts(tmem + kColO, t_p + kk * 8, upper | (vl + kk * (2048 >> 4)), id_o, on);
                                on = 1;
                            }
                            umma_commit(&sh.v_empty[slot]);
                            if (t == tiles - 1) umma_commit(&sh.o);
                        }
                        if (t + 3 < tiles) {
                            const unsigned x = x0 + t + 3;
                            const int slot = x % S::k_slots;
                            fine = mbar_wait(&sh.k_full[slot], (x / S::k_slots) & 1, kWaitBudget);
                            if (!fine) break;
                            tc_fence_after();
                            // both parts of Q, 32 columns at a time
                            const uint32_t kl = k_lo + slot * (S::code_bytes >> 4), t_s = tmem + x % 3 * 128;
                            uint32_t on = 0;
#pragma unroll
                            for (int kk = 0; kk < D / 16; ++kk) {
                                const int part = kk / (D / 32), c = kk % (D / 32);
                                const uint32_t off = ((D == 128 ? part * kHalfBytes : part * 64) + c * 32) >> 4;
                                umma_ss_f8(t_s, upper | (q_lo + off), k_upper | (kl + c * 2), id_s, on);
                                on = 1;
                            }
                            umma_commit(&sh.s[x % 3]);
                            umma_commit(&sh.k_empty[slot]);
                        }
                    }
                }
                x0 += tiles;
                ++nq;
                fine = __all_sync(0xffffffffu, fine);
                if (!fine) break;
            }
            if ((!fine || !ok) && lane == 0) raise_error(p.err, kErrTimeout);
            if (nq > 0 && elect_one()) {
                umma_commit(&sh.drain);
                if (!mbar_wait(&sh.drain, 0, kDrainBudget)) raise_error(p.err, kErrTimeout);
            }
            __syncwarp();
        } else if (warp == kValueWarp) {
            bring_values<D, true>(fp, &vmap, sh, smem);
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == kMmaWarp) {
        tc_fence_after();
        tmem_dealloc(tmem, kChunkTmem);
    }
}

template <typename Kernel>
int launch(Kernel kernel, bool (&configured)[64], int threads, int smem, const Fp8Params& p, const CUtensorMap& kmap,
           const CUtensorMap& vmap, int grid, int device, cudaStream_t stream) {
    static std::mutex mu;
    if (device < 0 || device >= 64) return BP_ERR_UNSUPPORTED;
    {
        std::lock_guard<std::mutex> lock(mu);
        if (!configured[device]) {
            if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) != cudaSuccess) return BP_ERR_CUDA;
            configured[device] = true;
        }
    }
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.gridDim = dim3((unsigned)grid, 1, 1);
    cfg.blockDim = dim3((unsigned)threads, 1, 1);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, p, kmap, vmap) == cudaSuccess ? BP_OK : BP_ERR_CUDA;
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

    static bool chunk_configured[64] = {}, block_configured[64] = {};
    if (a.max_q_len <= p.c.tokens)  // one stream's rows have any sequence's new tokens
        rc = launch(block_attention_fp8_kernel<D, FACTORS>, block_configured, kThreads, block_smem<D>(), p, kmap, vmap, grid, dev.device, stream);
    else
        rc = launch(chunk_attention_fp8_kernel<D, FACTORS>, chunk_configured, kThreads, chunk_smem<D>(), p, kmap, vmap, grid, dev.device, stream);
    if (rc != BP_OK) return rc;
    if (a.max_kv_len <= (2 * kLeastCut - 1) * kKeys) return BP_OK;  // too short to be cut: nothing to merge
    return launch_chunk_merge(p.c, D, grid, a.max_q_len, stream);
}

}  // namespace

int launch_chunk_attention_fp8(const ChunkAttentionFp8Args& a, const DeviceInfo& dev, cudaStream_t stream) {
    if (a.page_size >= 64) return a.head_dim == 128 ? run<128, 2>(a, dev, stream) : run<64, 2>(a, dev, stream);
    return a.head_dim == 128 ? run<128, 8>(a, dev, stream) : run<64, 8>(a, dev, stream);
}

}  // namespace bp
