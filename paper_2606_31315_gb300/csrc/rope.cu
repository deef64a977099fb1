// Queries and keys on their way from a layer's projections to its attention: every head normed and rotated to its
// token's position in one pass, and, with a paged cache, the keys and values written to their pages.
//
//   y = w * x / sqrt(mean(x^2) + eps)                       (no weights: y = x)
//   pairs (a, b) of y's first R elements, the i-th one turned by the angle of the token's position:
//   a' = a c - b s,  b' = b c + a s,   c, s = cos_sin[pos][i], cos_sin[pos][R / 2 + i]
//   pair i: elements i and R / 2 + i, or (interleaved) 2 i and 2 i + 1
//
// All in fp32, rounded once to the output's type.  A head is a row of pieces, one a lane; the lanes of a head sum the
// squares by shuffles.  In the usual form (halves, the whole head turned) a lane has a piece of either half, so that its
// pairs are its own; in the others it gets their other elements from the lane that has them.  A round is the 32 / LANES
// heads that a warp has at once: queries, keys or values, the same in all its lanes.  A warp has all of a token's rounds
// (fewer in small calls), the next one in flight, and forms the token's cosines and sines times the norm's weights once
// for all of a kind.
//
// Memory bounds it: nothing is read or written twice.  What it takes to get near is few instructions (executed ones
// by ncu's counter: 215 a KB with eight elements a lane and their pairs in another one, 90 now) and warps enough to
// hide a token's chain of loads, position, table row, weights: more rounds in flight cost registers, and with them warps
// (80 registers and 16 bytes spilled for 24 warps an SM in bf16's usual form without a cache, 94 and none with one).
// 16381 tokens of 32 + 8 heads of 128, bf16: 59 to 61 us, 5.7 TB/s; 8192 tokens to their pages with 8 heads of values: 39
// to 41 us, 5.1 TB/s.  The forms of part of a head, of neighbours and of fp32 were not timed at such sizes.
#include <cuda_bf16.h>

#include <limits.h>

#include <algorithm>

#include "common.cuh"
#include "ptx_sm103.cuh"

namespace bp {
namespace {

constexpr int kRopeWarps = 4;  // of a block: as many tokens

struct RopeParams {
    RopeArgs a;
    int page_shift;
    int q_rounds, k_rounds, rounds;  // of a token: its queries', its keys', all
    int per;                         // of a warp
    float dim_inverse;
};

// V elements of a head, as V / 2 pairs of fp32 numbers.
template <int V>
using Pairs = uint64_t[V / 2];
template <typename T, int V>
struct Piece;
template <int V>
struct Piece<__nv_bfloat16, V> {
    static constexpr int W = V / 2;
    uint32_t v[W];
    __device__ __forceinline__ void get(Pairs<V>& x) const {
#pragma unroll
        for (int i = 0; i < W; ++i) x[i] = pack_f32x2(__uint_as_float(v[i] << 16), __uint_as_float(v[i] & 0xffff0000u));
    }
    __device__ __forceinline__ void set(const Pairs<V>& x) {
#pragma unroll
        for (int i = 0; i < W; ++i) {
            float lo, hi;
            unpack_f32x2(x[i], lo, hi);
            v[i] = pack_bf16x2(lo, hi);
        }
    }
    __device__ __forceinline__ void swap_neighbours() {
#pragma unroll
        for (int i = 0; i < W; ++i) v[i] = __funnelshift_l(v[i], v[i], 16);
    }
};
template <int V>
struct Piece<float, V> {
    static constexpr int W = V;
    uint32_t v[W];
    __device__ __forceinline__ void get(Pairs<V>& x) const {
#pragma unroll
        for (int i = 0; i < V / 2; ++i) x[i] = pack_f32x2(__uint_as_float(v[2 * i]), __uint_as_float(v[2 * i + 1]));
    }
    __device__ __forceinline__ void set(const Pairs<V>& x) {
#pragma unroll
        for (int i = 0; i < V / 2; ++i) {
            float lo, hi;
            unpack_f32x2(x[i], lo, hi);
            v[2 * i] = __float_as_uint(lo);
            v[2 * i + 1] = __float_as_uint(hi);
        }
    }
    __device__ __forceinline__ void swap_neighbours() {
#pragma unroll
        for (int i = 0; i < V; i += 2) {
            const uint32_t t = v[i];
            v[i] = v[i + 1];
            v[i + 1] = t;
        }
    }
};
// Loads and stores by 16 bytes; with `apart` the piece is two runs of V / 2 elements, that many elements apart.
template <typename T, int V>
__device__ __forceinline__ void load_piece(Piece<T, V>& x, const T* p, int apart = V / 2) {
    constexpr int W = Piece<T, V>::W;
#pragma unroll
    for (int i = 0; i < W; i += 4) {
        const uint4 t = *reinterpret_cast<const uint4*>(2 * i < W ? p + i * (V / W) : p + apart + (i - W / 2) * (V / W));
        x.v[i] = t.x; x.v[i + 1] = t.y; x.v[i + 2] = t.z; x.v[i + 3] = t.w;
    }
}
template <typename T, int V>
__device__ __forceinline__ void store_piece(const Piece<T, V>& x, T* p, int apart = V / 2) {
    constexpr int W = Piece<T, V>::W;
#pragma unroll
    for (int i = 0; i < W; i += 4)
        *reinterpret_cast<uint4*>(2 * i < W ? p + i * (V / W) : p + apart + (i - W / 2) * (V / W)) =
            make_uint4(x.v[i], x.v[i + 1], x.v[i + 2], x.v[i + 3]);
}
// 1 / the root of the mean of a head's squares (every lane of the warp calls this).
template <int V, int LANES>
__device__ __forceinline__ float head_norm(const Pairs<V>& y, bool in, float dim_inverse, float eps) {
    uint64_t sq = mul_f32x2(y[0], y[0]);
#pragma unroll
    for (int i = 1; i < V / 2; ++i) sq = fma_f32x2(y[i], y[i], sq);
    float u, v;
    unpack_f32x2(sq, u, v);
    float sum = in ? u + v : 0.f;
#pragma unroll
    for (int o = LANES / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    return rsqrtf(sum * dim_inverse + eps);
}

// What a lane knows of its piece: y = x wc + (the paired elements) ws, wc and ws the cosines and signed sines of a position
// times the weights of a norm (one more rounding in fp32: 6.1e-8 off 64 bits instead of 5.7e-8).
template <typename T, int V, int LANES, bool PLAIN>
struct Lane;

// The usual form: head_dim is LANES x V, all of it turned in halves.  A piece is V / 2 elements of either half.
template <typename T, int V, int LANES>
struct Lane<T, V, LANES, true> {
    static constexpr int kApart = LANES * V / 2, H = V / 4;  // elements between a piece's runs; pairs of one run
    const RopeArgs& a;
    int e0;
    static constexpr bool in = true;
    __device__ __forceinline__ Lane(const RopeArgs& args, int lane) : a(args), e0(lane % LANES * (V / 2)) {}
    __device__ __forceinline__ void factors(int pos, const T* weight, Pairs<V>& wc, Pairs<V>& ws) const {
        const float* tab = a.cos_sin + (size_t)pos * (2 * kApart) + e0;
        Piece<float, V> t;  // V / 2 cosines, V / 2 sines
        Pairs<V> cs;
        load_piece(t, tab, kApart);
        t.get(cs);
        const uint64_t minus = pack_f32x2(-1.f, -1.f);
#pragma unroll
        for (int i = 0; i < H; ++i) {
            wc[i] = wc[i + H] = cs[i];
            ws[i] = mul_f32x2(cs[i + H], minus);
            ws[i + H] = cs[i + H];
        }
        if (weight) {
            Piece<T, V> w;
            Pairs<V> x;
            load_piece(w, weight + e0, kApart);
            w.get(x);
#pragma unroll
            for (int i = 0; i < H; ++i) {
                wc[i] = mul_f32x2(wc[i], x[i]);
                wc[i + H] = mul_f32x2(wc[i + H], x[i + H]);
                ws[i] = mul_f32x2(ws[i], x[i + H]);
                ws[i + H] = mul_f32x2(ws[i + H], x[i]);
            }
        }
    }
    __device__ __forceinline__ void turn(Piece<T, V>& x, bool norm, float dim_inverse, const Pairs<V>& wc, const Pairs<V>& ws) const {
        Pairs<V> y;
        x.get(y);
        if (norm) {
            const float inv = head_norm<V, LANES>(y, true, dim_inverse, a.eps);
            const uint64_t inv2 = pack_f32x2(inv, inv);
#pragma unroll
            for (int i = 0; i < V / 2; ++i) y[i] = mul_f32x2(y[i], inv2);
        }
#pragma unroll
        for (int i = 0; i < H; ++i) {
            const uint64_t u = y[i], v = y[i + H];
            y[i] = fma_f32x2(v, ws[i], mul_f32x2(u, wc[i]));
            y[i + H] = fma_f32x2(u, ws[i + H], mul_f32x2(v, wc[i + H]));
        }
        x.set(y);
    }
};

// Every other: part of the head turned, or none, or neighbours paired.  A piece is V elements in a row.
template <typename T, int V, int LANES>
struct Lane<T, V, LANES, false> {
    static constexpr int kApart = V / 2;
    const RopeArgs& a;
    int e0;       // the piece's first element
    bool in;      // it is part of a head
    bool turns;   // it is rotated
    int other;    // the lane of the elements it is paired with
    int partner;  // their first element
    __device__ __forceinline__ Lane(const RopeArgs& args, int lane) : a(args) {
        e0 = lane % LANES * V;
        in = e0 < a.head_dim;
        turns = e0 < a.rotary_dim;
        const int half = a.rotary_dim / 2;
        const bool front = e0 < half;
        other = turns && !a.interleaved ? (front ? lane + half / V : lane - half / V) : lane;
        partner = turns && !a.interleaved ? (front ? e0 + half : e0 - half) : e0;
    }
    __device__ __forceinline__ void factors(int pos, const T* weight, Pairs<V>& wc, Pairs<V>& ws) const {
        const uint64_t one = pack_f32x2(1.f, 1.f), minus = pack_f32x2(-1.f, -1.f);
#pragma unroll
        for (int i = 0; i < V / 2; ++i) wc[i] = one, ws[i] = 0ull;
        if (turns) {
            const int R = a.rotary_dim;
            const float* tab = a.cos_sin + (size_t)pos * R;
            if (a.interleaved) {
#pragma unroll
                for (int i = 0; i < V / 2; ++i) {
                    const float c = tab[e0 / 2 + i], s = tab[R / 2 + e0 / 2 + i];
                    wc[i] = pack_f32x2(c, c);
                    ws[i] = pack_f32x2(-s, s);
                }
            } else {
                Piece<float, V> c, s;
                load_piece(c, tab + min(e0, partner));
                load_piece(s, tab + R / 2 + min(e0, partner));
                c.get(wc);
                s.get(ws);
                if (e0 < partner)
#pragma unroll
                    for (int i = 0; i < V / 2; ++i) ws[i] = mul_f32x2(ws[i], minus);
            }
        }
        if (weight && in) {
            Piece<T, V> w;
            Pairs<V> x;
            load_piece(w, weight + e0);
            w.get(x);
#pragma unroll
            for (int i = 0; i < V / 2; ++i) wc[i] = mul_f32x2(wc[i], x[i]);
            load_piece(w, weight + partner);
            if (a.interleaved) w.swap_neighbours();
            w.get(x);
#pragma unroll
            for (int i = 0; i < V / 2; ++i) ws[i] = mul_f32x2(ws[i], x[i]);
        }
    }
    // (every lane of the warp calls this)
    __device__ __forceinline__ void turn(Piece<T, V>& x, bool norm, float dim_inverse, const Pairs<V>& wc, const Pairs<V>& ws) const {
        Pairs<V> y, z;
        x.get(y);
        Piece<T, V> paired = x;
        if (a.interleaved) {
            paired.swap_neighbours();
        } else {
#pragma unroll
            for (int i = 0; i < Piece<T, V>::W; ++i) paired.v[i] = __shfl_sync(0xffffffffu, x.v[i], other);
        }
        paired.get(z);
        if (norm) {
            const float inv = head_norm<V, LANES>(y, in, dim_inverse, a.eps);
            const uint64_t inv2 = pack_f32x2(inv, inv);
#pragma unroll
            for (int i = 0; i < V / 2; ++i) y[i] = mul_f32x2(y[i], inv2), z[i] = mul_f32x2(z[i], inv2);
        }
#pragma unroll
        for (int i = 0; i < V / 2; ++i) {
            y[i] = mul_f32x2(y[i], wc[i]);
            if (turns) y[i] = fma_f32x2(z[i], ws[i], y[i]);
        }
        x.set(y);
    }
};

template <typename T, int V, int LANES, bool PLAIN, bool CACHE>
__global__ void __launch_bounds__(kRopeWarps * 32, CACHE ? 5 : 6) rope_kernel(const __grid_constant__ RopeParams p) {
    griddep_launch_dependents();
    griddep_wait();
    constexpr int kHeads = 32 / LANES;
    const RopeArgs& a = p.a;
    const int lane = threadIdx.x & 31, sub = lane / LANES, D = PLAIN ? LANES * V : a.head_dim;
    const Lane<T, V, LANES, PLAIN> me(a, lane);
    const int hq = a.num_q_heads, hk = a.num_kv_heads;
    const int r0 = blockIdx.x * p.per, r1 = min(p.rounds, r0 + p.per);  // (the rounds and their kinds are the block's: uniform)
    for (long long tt = (long long)blockIdx.y * kRopeWarps + (threadIdx.x >> 5); tt < a.num_tokens; tt += (long long)gridDim.y * kRopeWarps) {
        const int t = (int)tt;
        // where round r's piece of this lane is read, and written: a place that moves on by kHeads heads a round, and jumps
        // where the keys or the values begin
        const int off = sub * D + me.e0, step = kHeads * D;
        const T* from = nullptr;
        int from_r = r0, from_h = 0, from_n = 0;
        auto fetch = [&](Piece<T, V>& x) {
            if (from_r == r0 || from_r == p.q_rounds || from_r == p.q_rounds + p.k_rounds) {
                const bool q = from_r < p.q_rounds, k = !q && from_r < p.q_rounds + p.k_rounds;
                const int first = from_r - (q ? 0 : k ? p.q_rounds : p.q_rounds + p.k_rounds);
                from = static_cast<const T*>(q ? a.q : k ? a.k : a.v) + t * (q ? a.q_stride : k ? a.k_stride : a.v_stride) + first * step + off;
                from_h = first * kHeads + sub;
                from_n = q ? hq : hk;
            }
            if (from_h < from_n && me.in) load_piece(x, from, me.kApart);
            from += step;
            from_h += kHeads;
            ++from_r;
        };
        Piece<T, V> x = {};
        fetch(x);

        int pos, row = 0;  // the token's position; the pool row of its key
        if (CACHE) {
            // the sequence of token t: the last one that starts at or before it
            int s = -1;
            for (int base = 0; base < a.num_seqs; base += 32) {
                const int n = __popc(__ballot_sync(0xffffffffu, base + lane < a.num_seqs && __ldg(a.cu_new + base + lane) <= t));
                s += n;
                if (n < 32) break;
            }
            const int end = s >= 0 ? __ldg(a.cu_new + s + 1) : 0;
            if (t >= end) continue;  // a row of padding behind the last sequence
            const int key = __ldg(a.cu_kv + s + 1) - __ldg(a.cu_kv + s) - (end - t);
            const int page = key >> p.page_shift;
            int id = -1;
            if (key >= 0 && page < a.pages_per_seq) id = __ldg(a.block_table + (size_t)s * a.pages_per_seq + page);
            pos = a.positions ? __ldg(a.positions + t) : key;
            if ((unsigned)id >= (unsigned)a.num_pages) {  // no place for the token's key
                if (lane == 0) raise_error(a.err_word, kErrDeviceArg);
                continue;
            }
            row = (id << p.page_shift) + (key & ((1 << p.page_shift) - 1));
        } else {
            pos = __ldg(a.positions + t);
        }
        if (a.rotary_dim > 0 && (unsigned)pos >= (unsigned)a.max_pos) {
            if (lane == 0) raise_error(a.err_word, kErrDeviceArg);
            continue;
        }

        Pairs<V> wc, ws;
        T* to = nullptr;
        int to_h = 0, to_n = 0;
        bool norm = false;
        for (int r = r0; r < r1; ++r) {
            Piece<T, V> y = x;
            if (r + 1 < r1) fetch(x);  // the next round's, while this one is worked on
            if (r == r0 || r == p.q_rounds || r == p.q_rounds + p.k_rounds) {
                const bool q = r < p.q_rounds, k = !q && r < p.q_rounds + p.k_rounds;
                const int first = r - (q ? 0 : k ? p.q_rounds : p.q_rounds + p.k_rounds);
                to = q ? static_cast<T*>(a.q_out) + t * a.q_out_stride
                       : CACHE ? static_cast<T*>(k ? a.k_cache : a.v_cache) + (size_t)row * hk * D
                               : static_cast<T*>(a.k_out) + t * a.k_out_stride;
                to += first * step + off;
                to_h = first * kHeads + sub;
                to_n = q ? hq : hk;
                if (q || k) {
                    const T* weight = static_cast<const T*>(q ? a.q_weight : a.k_weight);
                    norm = weight != nullptr;
                    me.factors(pos, weight, wc, ws);
                }
            }
            if (!CACHE || r < p.q_rounds + p.k_rounds) me.turn(y, norm, p.dim_inverse, wc, ws);
            if (to_h < to_n && me.in) store_piece(y, to, me.kApart);
            to += step;
            to_h += kHeads;
        }
    }
}

template <typename T, int V, int LANES, bool PLAIN, bool CACHE>
int run_rope(const RopeArgs& a, const DeviceInfo& dev, cudaStream_t stream) {
    constexpr int kHeads = 32 / LANES;  // of a warp in one round
    RopeParams p;
    p.a = a;
    p.page_shift = 0;
    while (CACHE && (1 << p.page_shift) < a.page_size) ++p.page_shift;
    p.q_rounds = (a.num_q_heads + kHeads - 1) / kHeads;
    p.k_rounds = (a.num_kv_heads + kHeads - 1) / kHeads;
    p.rounds = p.q_rounds + (CACHE ? 2 : 1) * p.k_rounds;
    p.dim_inverse = 1.f / (float)a.head_dim;
    // Rounds a warp: the fewest rounds one after another, by the waves of resident warps (24 an SM, or 20) times a warp's
    // rounds and what it costs beside them (1.5 rounds).  Against one round a warp up to 32 warps an SM and all of a
    // token's beyond: 512 tokens 3.3 instead of 5.6 us, 1000 5.1 instead of 8.6, 4000 18.4 instead of 20.5.
    const long long resident = (CACHE ? 20LL : 24LL) * dev.sm_count;
    long long best = LLONG_MAX;
    p.per = p.rounds;
    for (int k = 1; k <= p.rounds; ++k) {
        const int per = (p.rounds + k - 1) / k;
        const long long cost = ((long long)a.num_tokens * ((p.rounds + per - 1) / per) + resident - 1) / resident * (2 * per + 3);
        if (cost < best) best = cost, p.per = per;
    }
    const int warps = std::min(kRopeWarps, a.num_tokens);
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[1];
    cfg.gridDim = dim3((unsigned)((p.rounds + p.per - 1) / p.per), (unsigned)std::min((a.num_tokens + kRopeWarps - 1) / kRopeWarps, 65535), 1);
    cfg.blockDim = dim3(warps * 32, 1, 1);
    cfg.stream = stream;
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, rope_kernel<T, V, LANES, PLAIN, CACHE>, p);
    return e == cudaSuccess ? BP_OK : BP_ERR_CUDA;
}

// 32 bytes a lane in the usual form, else 8 elements.
template <typename T, bool CACHE>
int run_rope(const RopeArgs& a, const DeviceInfo& dev, cudaStream_t stream) {
    constexpr int V = 32 / sizeof(T);
    if (a.rotary_dim == a.head_dim && !a.interleaved) {
        if (a.head_dim == 64) return run_rope<T, V, 64 / V, true, CACHE>(a, dev, stream);
        if (a.head_dim == 128) return run_rope<T, V, 128 / V, true, CACHE>(a, dev, stream);
    }
    if (a.head_dim <= 64) return run_rope<T, 8, 8, false, CACHE>(a, dev, stream);
    if (a.head_dim <= 128) return run_rope<T, 8, 16, false, CACHE>(a, dev, stream);
    return run_rope<T, 8, 32, false, CACHE>(a, dev, stream);
}

}  // namespace

int launch_rope(const RopeArgs& a, const DeviceInfo& dev, cudaStream_t stream) {
    const bool cache = a.k_cache != nullptr;
    if (a.dtype == BP_BF16)
        return cache ? run_rope<__nv_bfloat16, true>(a, dev, stream) : run_rope<__nv_bfloat16, false>(a, dev, stream);
    return cache ? run_rope<float, true>(a, dev, stream) : run_rope<float, false>(a, dev, stream);
}

}  // namespace bp
