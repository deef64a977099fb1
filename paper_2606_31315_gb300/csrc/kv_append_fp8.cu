// New keys and values to the pages of a cache in 8 bits: e4m3 codes, and a power of two for each page and head as their scale,
// held as its biased exponent b.  For the new rows X of a page and head:
//
//   b = the least in [1, 254] with max |x| <= 448 2^(b - 127)   (over finite x; 1 where all are 0)
//   of a page that held rows before: the larger of that and of its b; where it grows, its old codes q become
//   the e4m3 numbers nearest to q 2^(b_old - b)
//   code = the e4m3 number nearest to x 2^(127 - b) (ties to the even one); NaN for what is not finite
//
// A power of two, because then nothing but e4m3's own rounding is lost: a code's value is a bf16 number, and a rescaled code
// is exact unless it falls under 2^-6.  (448 / max as the scale would use up to one binade more of a type that has 18, and
// round every rescaled code and every product of a code and its scale.)
//
// A page's new rows are a unit, which has one owner: nothing is summed or ordered by atomics.  A block has a few tokens of
// one head of K or V; its threads look which of them begin a unit (a sequence's first new token, or a page's first row), then
// units of many rows are the whole block's, others a warp's.  A thread keeps its rows' pieces in registers between the
// maximum and the rounding, four of 16 elements (two of fp32); what is more (units above 64 rows of 128, 32 of fp32) is read
// again, from L2.
//
// Bound by memory: bf16 in, a byte an element out.  In graphs, 8 KV heads of 128: 8192 tokens 15.9 us over inputs in turn that L2
// does not hold (50 MB, 3.2 TB/s), 11.7 over the same ones: the units' chain, look-up, loads, maximum, stores, once a block.  32 x 16
// tokens 4.4, one token 2.3, a launch and three round trips.  Where the scale of a page that was begun before grows, its rows are
// read, rounded and written too: 3.7 us more for 59 rows in each of 32 sequences, 3.9 for 63 in one.
#include <cuda_bf16.h>

#include <algorithm>

#include "common.cuh"
#include "ptx_sm103.cuh"

namespace bp {
namespace {

constexpr int kAppendThreads = 128;
constexpr int kAppendTokens = 64;  // of a block, at most
constexpr int kWarpRows = 8;       // a unit of up to so many rows is a warp's
template <typename T>
constexpr int kKept = sizeof(T) == 2 ? 4 : 2;  // pieces that a thread keeps

struct AppendParams {
    KvAppendFp8Args a;
    int page_shift, tokens;  // tokens of a block
    unsigned piece_inverse;  // 2^32 / (pieces of a row), rounded up
};
struct Unit {
    int token, rows, seq, key;  // first new token, its rows; its sequence, and its key's number
};

// 16 elements of a row.
template <typename T>
struct Piece {
    static constexpr int W = 16 * (int)sizeof(T) / 16;
    uint4 v[W];
    __device__ __forceinline__ void load(const T* p) {
#pragma unroll
        for (int i = 0; i < W; ++i) v[i] = __ldg(reinterpret_cast<const uint4*>(p) + i);
    }
    __device__ __forceinline__ float at(int e) const {
        const uint32_t* w = reinterpret_cast<const uint32_t*>(v);
        if constexpr (sizeof(T) == 2) return __uint_as_float(e & 1 ? w[e >> 1] & 0xffff0000u : w[e >> 1] << 16);
        else return __uint_as_float(w[e]);
    }
    __device__ __forceinline__ float top(float m) const {
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const float x = fabsf(at(e));
            if (x < INFINITY) m = fmaxf(m, x);
        }
        return m;
    }
    __device__ __forceinline__ uint4 codes(float up) const {
        uint32_t c[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            float x[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float y = at(4 * k + e);
                x[e] = fabsf(y) < INFINITY ? y * up : __uint_as_float(0x7fc00000u);
            }
            c[k] = pack_e4m3x2(x[0], x[1]) | pack_e4m3x2(x[2], x[3]) << 16;
        }
        return make_uint4(c[0], c[1], c[2], c[3]);
    }
};

// 2^(e - 127)
__device__ __forceinline__ float power_of(int e) { return __uint_as_float(e > 0 ? (uint32_t)e << 23 : 0x400000u); }

// One unit by THREADS threads, of which this is the one numbered t: its maximum is formed by `reduce`, which also lets
// every thread read the page's old exponent before the new one is written.
template <typename T, int THREADS, typename Reduce>
__device__ __forceinline__ void append_unit(const AppendParams& p, const Unit& u, int head, int kv, int t, Reduce reduce) {
    const int D = p.a.head_dim, pieces = D / 16, n = u.rows * pieces, H = p.a.num_kv_heads;
    // i / pieces: right for i * pieces below 2^32
    auto row_of = [&](int i) { return pieces == 1 ? i : (int)__umulhi((unsigned)i, p.piece_inverse); };
    auto source = [&](int i) {
        const int row = row_of(i);
        return static_cast<const T*>(p.a.fresh[kv]) + (int64_t)(u.token + row) * p.a.stride[kv] + (int64_t)head * D + (i - row * pieces) * 16;
    };
    Piece<T> kept[kKept<T>];
    float top = 0.f;
#pragma unroll
    for (int k = 0; k < kKept<T>; ++k)
        if (t + k * THREADS < n) kept[k].load(source(t + k * THREADS));
    // the page is looked up while the rows are on their way
    const int index = u.key >> p.page_shift, off = u.key & ((1 << p.page_shift) - 1);
    const int page = u.key >= 0 && index < p.a.pages_per_seq ? __ldg(p.a.block_table + (size_t)u.seq * p.a.pages_per_seq + index) : -1;
    if ((unsigned)page >= (unsigned)p.a.num_pages) {
        if (t == 0) raise_error(p.a.err_word, kErrDeviceArg);
        return;  // (all of the unit's threads)
    }
    uint8_t* const to = p.a.cache[kv] + ((((int64_t)page << p.page_shift) * H) + head) * D;  // the page's first row
    uint8_t* const scale = p.a.scale[kv] + (int64_t)page * H + head;
    const int was = off > 0 ? *scale : 0;
    if (was == 255) {  // (no power of two: the rows before are none that a scale could be found for)
        if (t == 0) raise_error(p.a.err_word, kErrDeviceArg);
        return;
    }
#pragma unroll
    for (int k = 0; k < kKept<T>; ++k)
        if (t + k * THREADS < n) top = kept[k].top(top);
    for (int i = t + kKept<T> * THREADS; i < n; i += THREADS) {
        Piece<T> x;
        x.load(source(i));
        top = x.top(top);
    }
    const uint32_t bits = __float_as_uint(reduce(top));
    // 448 is 1.75 times 2^8
    const int least = bits == 0 ? 1 : max(1, (int)(bits >> 23) - 8 + ((bits & 0x7fffffu) > 0x600000u ? 1 : 0));
    const int b = max(least, was);
    if (t == 0 && b != was) *scale = (uint8_t)b;
    if (off > 0 && b > was) {
        const float down = power_of(127 + was - b);  // (0 from 2^-127 on: every code becomes 0)
        for (int i = t; i < off * pieces; i += THREADS) {
            const int row = row_of(i);
            uint4* at = reinterpret_cast<uint4*>(to + (int64_t)row * H * D + (i - row * pieces) * 16);
            uint4 c = *at;
            uint32_t* w = reinterpret_cast<uint32_t*>(&c);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                float x[4];
                unpack_e4m3x2(w[k] & 0xffffu, x[0], x[1]);
                unpack_e4m3x2(w[k] >> 16, x[2], x[3]);
                w[k] = pack_e4m3x2(x[0] * down, x[1] * down) | pack_e4m3x2(x[2] * down, x[3] * down) << 16;
            }
            *at = c;
        }
    }
    const float up = power_of(254 - b);
    auto store = [&](const Piece<T>& x, int i) {
        const int row = row_of(i);
        *reinterpret_cast<uint4*>(to + (int64_t)(off + row) * H * D + (i - row * pieces) * 16) = x.codes(up);
    };
#pragma unroll
    for (int k = 0; k < kKept<T>; ++k)
        if (t + k * THREADS < n) store(kept[k], t + k * THREADS);
    for (int i = t + kKept<T> * THREADS; i < n; i += THREADS) {
        Piece<T> x;
        x.load(source(i));
        store(x, i);
    }
}

template <typename T>
__global__ void __launch_bounds__(kAppendThreads) kv_append_fp8_kernel(const __grid_constant__ AppendParams p) {
    __shared__ Unit units[kAppendTokens];
    __shared__ int count;
    __shared__ float tops[kAppendThreads / 32];
    griddep_launch_dependents();
    griddep_wait();
    const KvAppendFp8Args& a = p.a;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, head = blockIdx.y, kv = blockIdx.z;
    if (tid == 0) count = 0;
    __syncthreads();
    if (tid < p.tokens) {
        const int t = blockIdx.x * p.tokens + tid, all = min(a.total_new, __ldg(a.cu_new + a.num_seqs));
        int s = 0;
        for (int hi = a.num_seqs; hi - s > 1;) {  // the last sequence that begins at or before t
            const int mid = (s + hi) >> 1;
            if (__ldg(a.cu_new + mid) <= t) s = mid; else hi = mid;
        }
        const int first = __ldg(a.cu_new + s), end = __ldg(a.cu_new + s + 1);
        const int len = __ldg(a.cu_kv + s + 1) - __ldg(a.cu_kv + s), pos = len - (end - first) + t - first;
        const int off = pos & ((1 << p.page_shift) - 1);
        if (t >= first && t < min(end, all) && (t == first || off == 0))
            units[atomicAdd(&count, 1)] = Unit{t, min((1 << p.page_shift) - off, min(end, all) - t), s, pos};  // (below 0: before key 0)
    }
    __syncthreads();
    const int n = count;  // (their order is that of arrival: each is by itself)
    int mine = 0;         // units for single warps, dealt out
    for (int i = 0; i < n; ++i) {
        const Unit u = units[i];
        if (u.rows > kWarpRows) {
            append_unit<T, kAppendThreads>(p, u, head, kv, tid, [&](float top) {
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
                __syncthreads();  // (the unit before is done with tops)
                if (lane == 0) tops[warp] = top;
                __syncthreads();
                float all = tops[0];
#pragma unroll
                for (int w = 1; w < kAppendThreads / 32; ++w) all = fmaxf(all, tops[w]);
                return all;
            });
        } else if (mine++ % (kAppendThreads / 32) == warp) {
            append_unit<T, 32>(p, u, head, kv, lane, [&](float top) {
                __syncwarp();  // (the page's old exponent is read before lane 0 writes the new one)
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
                return top;
            });
        }
    }
}

}  // namespace

int launch_kv_append_fp8(const KvAppendFp8Args& a, cudaStream_t stream) {
    AppendParams p;
    p.a = a;
    p.page_shift = 0;
    while ((1 << p.page_shift) < a.page_size) ++p.page_shift;
    p.piece_inverse = (unsigned)(((1ull << 32) + a.head_dim / 16 - 1) / (a.head_dim / 16));
    // as many tokens a block as a sequence brings, so that neither units wait for one another nor blocks find none (us in graphs,
    // over the same inputs, against always 4 and always 64: 32 sequences of 16 tokens 4.5, 6.7, 10.4; 256 of 1 6.7, 6.6, 20.8; 1 of
    // 8192 11.6, 35.7, 11.6)
    p.tokens = 4;
    while (p.tokens < std::min(kAppendTokens, a.page_size) && p.tokens * 2 * (long long)a.num_seqs <= a.total_new) p.tokens *= 2;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.gridDim = dim3((unsigned)((a.total_new + p.tokens - 1) / p.tokens), (unsigned)a.num_kv_heads, 2);
    cfg.blockDim = dim3(kAppendThreads, 1, 1);
    cfg.stream = stream;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    const cudaError_t e = a.dtype == BP_BF16 ? cudaLaunchKernelEx(&cfg, kv_append_fp8_kernel<__nv_bfloat16>, p)
                                             : cudaLaunchKernelEx(&cfg, kv_append_fp8_kernel<float>, p);
    return e == cudaSuccess ? BP_OK : BP_ERR_CUDA;
}

}  // namespace bp
