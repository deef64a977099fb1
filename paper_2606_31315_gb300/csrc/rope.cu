// Queries and keys on their way from a layer's projections to its attention: every head normed and rotated to its
// token's position in one pass, and, with a paged cache, the keys and values written to their pages.
//
//   y = w * x / sqrt(mean(x^2) + eps)                       (no weights: y = x)
//   pairs (a, b) of y's first R elements, the i-th one turned by the angle of the token's position:
//   a' = a c - b s,  b' = b c + a s,   c, s = cos_sin[pos][i], cos_sin[pos][R / 2 + i]
//   pair i: elements i and R / 2 + i, or (interleaved) 2 i and 2 i + 1
//
// All in fp32, rounded once to the output's type.  A head is a row of 8-element pieces, one a lane (two 16-byte loads
// in fp32); the lanes of a head sum the squares by shuffles, and in the halves' form a lane gets its pair's other
// elements from the lane R / 16 further.  A warp takes some heads of one token, so that its table row is read once.
#include <cuda_bf16.h>

#include <algorithm>

#include "common.cuh"
#include "ptx_sm103.cuh"

namespace bp {
namespace {

constexpr int kRopeThreads = 256;
constexpr int kPiece = 8;  // elements a lane holds

struct RopeParams {
    RopeArgs a;
    int page_shift;
    int heads;      // of a token: queries, keys, values
    int per_token;  // warps
    long long warps;
};

template <typename T>
struct Piece;
template <>
struct Piece<__nv_bfloat16> {
    uint4 v;
    __device__ __forceinline__ void load(const __nv_bfloat16* p) { v = *reinterpret_cast<const uint4*>(p); }
    __device__ __forceinline__ void store(__nv_bfloat16* p) const { *reinterpret_cast<uint4*>(p) = v; }
    __device__ __forceinline__ void get(float (&x)[kPiece]) const {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = __uint_as_float(w[i] << 16);
            x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
    }
    __device__ __forceinline__ void set(const float (&x)[kPiece]) {
        v = make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7]));
    }
};
template <>
struct Piece<float> {
    float4 v, w;
    __device__ __forceinline__ void load(const float* p) {
        v = *reinterpret_cast<const float4*>(p);
        w = *reinterpret_cast<const float4*>(p + 4);
    }
    __device__ __forceinline__ void store(float* p) const {
        *reinterpret_cast<float4*>(p) = v;
        *reinterpret_cast<float4*>(p + 4) = w;
    }
    __device__ __forceinline__ void get(float (&x)[kPiece]) const {
        x[0] = v.x; x[1] = v.y; x[2] = v.z; x[3] = v.w; x[4] = w.x; x[5] = w.y; x[6] = w.z; x[7] = w.w;
    }
    __device__ __forceinline__ void set(const float (&x)[kPiece]) {
        v = make_float4(x[0], x[1], x[2], x[3]);
        w = make_float4(x[4], x[5], x[6], x[7]);
    }
};

// LANES: of a head, head_dim / 8 rounded up to a power of two.  A warp takes ROUNDS x 32 / LANES heads of a token, all
// of them loaded before the first is used.
template <typename T, int LANES, int ROUNDS, bool CACHE>
__global__ void __launch_bounds__(kRopeThreads) rope_kernel(const RopeParams p) {
    griddep_launch_dependents();
    griddep_wait();
    const RopeArgs& a = p.a;
    const long long warp = (long long)blockIdx.x * (kRopeThreads / 32) + (threadIdx.x >> 5);
    if (warp >= p.warps) return;
    const int lane = threadIdx.x & 31, piece = lane % LANES, sub = lane / LANES;
    const int t = (int)(warp / p.per_token), h0 = (int)(warp % p.per_token) * (ROUNDS * (32 / LANES)) + sub;
    const int D = a.head_dim, e0 = piece * kPiece;
    const bool in = e0 < D;

    const int hq = a.num_q_heads, hk = hq + a.num_kv_heads;
    Piece<T> x[ROUNDS];
#pragma unroll
    for (int k = 0; k < ROUNDS; ++k) {
        const int h = h0 + k * (32 / LANES);
        if (h < p.heads && in) {
            const T* src = h < hq   ? static_cast<const T*>(a.q) + (size_t)t * a.q_stride + (size_t)h * D
                           : h < hk ? static_cast<const T*>(a.k) + (size_t)t * a.k_stride + (size_t)(h - hq) * D
                                    : static_cast<const T*>(a.v) + (size_t)t * a.v_stride + (size_t)(h - hk) * D;
            x[k].load(src + e0);
        }
    }

    int pos, row = 0;  // the token's position; the pool row of its key
    if (CACHE) {
        // the sequence of token t: the last one that starts at or before it
        int s = -1;
        for (int base = 0; base < a.num_seqs; base += 32) {
            const bool before = base + lane < a.num_seqs && __ldg(a.cu_new + base + lane) <= t;
            const int n = __popc(__ballot_sync(0xffffffffu, before));
            s += n;
            if (n < 32) break;
        }
        const int end = s >= 0 ? __ldg(a.cu_new + s + 1) : 0;
        if (t >= end) return;  // a row of padding behind the last sequence
        const int key = __ldg(a.cu_kv + s + 1) - __ldg(a.cu_kv + s) - (end - t);
        const int page = key >> p.page_shift;
        int id = -1;
        if (key >= 0 && page < a.pages_per_seq) id = __ldg(a.block_table + (size_t)s * a.pages_per_seq + page);
        pos = a.positions ? __ldg(a.positions + t) : key;
        if ((unsigned)id >= (unsigned)a.num_pages) {  // no place for the token's key
            if (lane == 0) raise_error(a.err_word, kErrDeviceArg);
            return;
        }
        row = (id << p.page_shift) + (key & ((1 << p.page_shift) - 1));
    } else {
        pos = __ldg(a.positions + t);
    }
    const int R = a.rotary_dim;
    if (R > 0 && (unsigned)pos >= (unsigned)a.max_pos) {
        if (lane == 0) raise_error(a.err_word, kErrDeviceArg);
        return;
    }

    // this lane's cosines and sines: x' = x c + (the pair's other) s
    const int half = R / 2;
    const bool turns = e0 < R;
    float c[kPiece], s[kPiece];
    int other = lane;
    if (turns) {
        const float* tab = a.cos_sin + (size_t)pos * R;
        if (a.interleaved) {
            const float4 cc = *reinterpret_cast<const float4*>(tab + e0 / 2), ss = *reinterpret_cast<const float4*>(tab + half + e0 / 2);
            const float cv[4] = {cc.x, cc.y, cc.z, cc.w}, sv[4] = {ss.x, ss.y, ss.z, ss.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                c[2 * i] = c[2 * i + 1] = cv[i];
                s[2 * i] = -sv[i];
                s[2 * i + 1] = sv[i];
            }
        } else {
            const bool front = e0 < half;
            const int f = front ? e0 : e0 - half;
            other = front ? lane + half / kPiece : lane - half / kPiece;
            Piece<float> cc, ss;
            cc.load(tab + f);
            ss.load(tab + half + f);
            cc.get(c);
            ss.get(s);
#pragma unroll
            for (int i = 0; i < kPiece; ++i) s[i] = front ? -s[i] : s[i];
        }
    }

#pragma unroll
    for (int k = 0; k < ROUNDS; ++k) {
        const int h = h0 + k * (32 / LANES);
        const bool there = h < p.heads && in;
        const bool query = h < hq, value = CACHE && h >= hk;
        const T* weight = static_cast<const T*>(query ? a.q_weight : a.k_weight);
        float y[kPiece] = {};
        if (there) x[k].get(y);
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < kPiece; ++i) sum += y[i] * y[i];
#pragma unroll
        for (int o = LANES / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        if (there && weight && !value) {
            const float inv = rsqrtf(sum / (float)D + a.eps);
            Piece<T> w;
            w.load(weight + e0);
            float wf[kPiece];
            w.get(wf);
#pragma unroll
            for (int i = 0; i < kPiece; ++i) y[i] = y[i] * inv * wf[i];
        }
        if (R > 0) {
            float z[kPiece];
#pragma unroll
            for (int i = 0; i < kPiece; ++i) z[i] = a.interleaved ? y[i ^ 1] : __shfl_sync(0xffffffffu, y[i], other);
            if (turns && !value) {
#pragma unroll
                for (int i = 0; i < kPiece; ++i) y[i] = y[i] * c[i] + z[i] * s[i];
            }
        }
        if (there) {
            if (!value) x[k].set(y);
            T* dst;
            if (query) dst = static_cast<T*>(a.q_out) + (size_t)t * a.q_out_stride + (size_t)h * D;
            else if (!CACHE) dst = static_cast<T*>(a.k_out) + (size_t)t * a.k_out_stride + (size_t)(h - hq) * D;
            else dst = static_cast<T*>(value ? a.v_cache : a.k_cache) + ((size_t)row * a.num_kv_heads + (value ? h - hk : h - hq)) * D;
            x[k].store(dst + e0);
        }
    }
}

template <typename T, int LANES, bool CACHE>
int run_rope(const RopeArgs& a, const DeviceInfo& dev, cudaStream_t stream) {
    constexpr int kHeads = 32 / LANES;  // of a warp in one round
    RopeParams p;
    p.a = a;
    p.page_shift = 0;
    while (CACHE && (1 << p.page_shift) < a.page_size) ++p.page_shift;
    p.heads = a.num_q_heads + (CACHE ? 2 : 1) * a.num_kv_heads;
    const int rounds = (p.heads + kHeads - 1) / kHeads;
    // one round a warp while that leaves the SMs room for all of them at once (64 warps each), else four
    const bool many = (long long)a.num_tokens * rounds > 64LL * dev.sm_count;
    p.per_token = many ? (rounds + 3) / 4 : rounds;
    p.warps = (long long)a.num_tokens * p.per_token;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[1];
    const long long blocks = (p.warps + kRopeThreads / 32 - 1) / (kRopeThreads / 32);
    if (blocks > INT32_MAX) return BP_ERR_UNSUPPORTED;
    cfg.gridDim = dim3((unsigned)blocks, 1, 1);
    cfg.blockDim = dim3(kRopeThreads, 1, 1);
    cfg.stream = stream;
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    const cudaError_t e = many ? cudaLaunchKernelEx(&cfg, rope_kernel<T, LANES, 4, CACHE>, p)
                               : cudaLaunchKernelEx(&cfg, rope_kernel<T, LANES, 1, CACHE>, p);
    return e == cudaSuccess ? BP_OK : BP_ERR_CUDA;
}

template <typename T, bool CACHE>
int run_rope(const RopeArgs& a, const DeviceInfo& dev, cudaStream_t stream) {
    if (a.head_dim <= 64) return run_rope<T, 8, CACHE>(a, dev, stream);
    if (a.head_dim <= 128) return run_rope<T, 16, CACHE>(a, dev, stream);
    return run_rope<T, 32, CACHE>(a, dev, stream);
}

}  // namespace

int launch_rope(const RopeArgs& a, const DeviceInfo& dev, cudaStream_t stream) {
    const bool cache = a.k_cache != nullptr;
    if (a.dtype == BP_BF16)
        return cache ? run_rope<__nv_bfloat16, true>(a, dev, stream) : run_rope<__nv_bfloat16, false>(a, dev, stream);
    return cache ? run_rope<float, true>(a, dev, stream) : run_rope<float, false>(a, dev, stream);
}

}  // namespace bp
