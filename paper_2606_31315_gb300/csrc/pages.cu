// A step's pages: sequences grow and shrink, the pages of a pool's free list go to the block table and back, and every new
// token gets its position and its slot in the pool; all from the sequences' lengths, on the device.
//
//   sequence s holds ceil(old_s / P) pages and is to hold ceil(new_s / P)
//   R: the pages that shrinking sequences give back, sequence by sequence, each one's in the table's order
//   L = R, then the free list from its end: the pages that growing sequences take, in the same order
//   what is left of R is pushed on the free list from its end, so that it is taken in R's order again: giving back what was
//   just taken restores the free list
//
// Every block forms the prefix sums of the sequences' new tokens, taken and given pages itself (num_seqs is small beside what
// a step moves, and the lengths lie in L2), so that one launch is enough and the place of a page or token follows from its
// number alone, by a search in shared memory.  Tables and list are written in places that no block reads (a page that is taken
// stands behind its sequence's old ones, one that is given back behind the list's old end, and only where none of the old list
// is taken); the list's length is written by the last block to finish.
#include <limits.h>

#include <algorithm>
#include <mutex>

#include "common.cuh"
#include "ptx_sm103.cuh"

namespace bp {
namespace {

constexpr int kPagesThreads = 512;
constexpr int kPerThread = 4;  // tokens in a row

struct PagesParams {
    PagesUpdateArgs a;
    int page_shift;
};

// The last i of [0, n) with sums[i] <= x (sums[0] <= x).
__device__ __forceinline__ int place_of(const int* sums, int n, int x) {
    int i = 0;
    for (int hi = n; hi - i > 1;) {
        const int mid = (i + hi) >> 1;
        if (sums[mid] <= x) i = mid; else hi = mid;
    }
    return i;
}

__global__ void __launch_bounds__(kPagesThreads) pages_update_kernel(const __grid_constant__ PagesParams p) {
    extern __shared__ int sums[];  // [3][num_seqs + 1]: new tokens, taken pages, given pages of the sequences before
    __shared__ int warp_sums[4][kPagesThreads / 32];
    griddep_launch_dependents();
    griddep_wait();
    const PagesUpdateArgs& a = p.a;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, n = a.num_seqs, P = 1 << p.page_shift;
    int* const tokens = sums;
    int* const taken = sums + n + 1;
    int* const given = sums + 2 * (n + 1);
    auto pages_of = [&](int len) { return (int)(((unsigned)len + P - 1) >> p.page_shift); };

    // ---- prefix sums over the sequences, kPagesThreads at a time
    const int num_free = *a.num_free;
    int carry[4] = {0, 0, 0, 0};  // tokens, taken, given; keys after the step
    bool bad = num_free < 0 || num_free > a.num_pages;
    long long all_tokens = 0, all_keys = 0, all_given = 0;
    const bool writes = blockIdx.x == 0;
    for (int base = 0; base < n; base += kPagesThreads) {
        const int s = base + tid;
        int v[4] = {0, 0, 0, 0};
        if (s < n) {
            const int o = __ldg(a.old_lens + s), w = __ldg(a.new_lens + s);
            if (o < 0 || w < 0 || pages_of(o) > a.pages_per_seq || pages_of(w) > a.pages_per_seq) {
                bad = true;
            } else {
                v[0] = max(0, w - o);
                v[1] = max(0, pages_of(w) - pages_of(o));
                v[2] = max(0, pages_of(o) - pages_of(w));
                v[3] = w;
                all_tokens += v[0];
                all_keys += w;
                all_given += v[2];
            }
        }
        int sum[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            sum[k] = v[k];
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int y = __shfl_up_sync(0xffffffffu, sum[k], o);
                if (lane >= o) sum[k] += y;
            }
        }
        __syncthreads();  // the sequences before are done with warp_sums
        if (lane == 31)
#pragma unroll
            for (int k = 0; k < 4; ++k) warp_sums[k][warp] = sum[k];
        __syncthreads();
        int total[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int w = lane < kPagesThreads / 32 ? warp_sums[k][lane] : 0;
            int before = lane < warp ? w : 0;
            total[k] = w;
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) {
                before += __shfl_xor_sync(0xffffffffu, before, o);
                total[k] += __shfl_xor_sync(0xffffffffu, total[k], o);
            }
            sum[k] += carry[k] + before;
            carry[k] += total[k];
        }
        if (s < n) {
            tokens[s + 1] = sum[0];
            taken[s + 1] = sum[1];
            given[s + 1] = sum[2];
            if (writes && a.cu_kv) a.cu_kv[s + 1] = sum[3];  // (rewritten below where the step does not take place)
        }
    }
    if (tid == 0) tokens[0] = taken[0] = given[0] = 0;
    // (the sums above may pass 31 bits; these tell)
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        all_tokens += __shfl_xor_sync(0xffffffffu, all_tokens, o);
        all_keys += __shfl_xor_sync(0xffffffffu, all_keys, o);
        all_given += __shfl_xor_sync(0xffffffffu, all_given, o);
    }
    __shared__ long long long_sums[3][kPagesThreads / 32];
    if (lane == 0) {
        long_sums[0][warp] = all_tokens;
        long_sums[1][warp] = all_keys;
        long_sums[2][warp] = all_given;
    }
    __syncthreads();
    all_tokens = all_keys = all_given = 0;
    for (int w = 0; w < kPagesThreads / 32; ++w) {
        all_tokens += long_sums[0][w];
        all_keys += long_sums[1][w];
        all_given += long_sums[2][w];
    }
    const int A = carry[1], R = carry[2];
    bad = __syncthreads_or(bad) || all_keys > INT_MAX || all_given > a.num_pages || ((a.positions || a.slots) && all_tokens > a.total_new) ||
          (long long)num_free + R - A > a.num_pages;
    const int missing = bad ? 0 : max(0, A - R - num_free);
    const bool done = !bad && missing == 0;
    if (bad && writes && tid == 0) raise_error(a.err_word, kErrDeviceArg);

    // the page that is taken as number i, and the one that is given back as number i
    auto given_page = [&](int i) {
        const int s = place_of(given, n, i);
        return a.block_table[(size_t)s * a.pages_per_seq + pages_of(__ldg(a.new_lens + s)) + i - given[s]];
    };
    auto taken_page = [&](int i) { return i < R ? given_page(i) : a.free_pages[num_free - 1 - (i - R)]; };
    const int t0 = blockIdx.x * kPagesThreads + tid, stride = gridDim.x * kPagesThreads;
    if (done) {
        for (int i = t0; i < A; i += stride) {
            const int s = place_of(taken, n, i);
            const int page = taken_page(i);
            if ((unsigned)page >= (unsigned)a.num_pages) raise_error(a.err_word, kErrDeviceArg);
            a.block_table[(size_t)s * a.pages_per_seq + pages_of(__ldg(a.old_lens + s)) + i - taken[s]] = page;
        }
        for (int i = A + t0; i < R; i += stride) {
            const int page = given_page(i);
            if ((unsigned)page >= (unsigned)a.num_pages) raise_error(a.err_word, kErrDeviceArg);
            a.free_pages[num_free + R - 1 - i] = page;
        }
    }
    if (a.positions || a.slots) {
        const int real = done ? carry[0] : 0;
        for (int t = t0 * kPerThread; t < a.total_new; t += stride * kPerThread) {
            int s = t < real ? place_of(tokens, n, t) : 0, old = 0, held = 0, at = -1, page = 0;
            bool fresh = true;
#pragma unroll
            for (int k = 0; k < kPerThread; ++k) {
                const int x = t + k;
                if (x >= a.total_new) break;
                int pos = -1;
                int64_t slot = -1;
                if (x < real) {
                    while (x >= tokens[s + 1]) ++s, fresh = true;
                    if (fresh) old = __ldg(a.old_lens + s), held = pages_of(old), at = -1, fresh = false;
                    pos = old + x - tokens[s];
                    const int j = pos >> p.page_shift;
                    if (j != at) {
                        at = j;
                        page = j < held ? a.block_table[(size_t)s * a.pages_per_seq + j] : taken_page(taken[s] + j - held);
                    }
                    slot = ((int64_t)page << p.page_shift) + (pos & (P - 1));
                }
                if (a.positions) a.positions[x] = pos;
                if (a.slots) a.slots[x] = slot;
            }
        }
    }
    if (writes) {
        if (a.cu_new)
            for (int s = tid; s <= n; s += kPagesThreads) a.cu_new[s] = done ? tokens[s] : 0;
        if (a.cu_kv && tid == 0) {
            a.cu_kv[0] = 0;
            if (!done)  // the lengths stay (rare: by one thread)
                for (int s = 0, sum = 0; s < n; ++s) a.cu_kv[s + 1] = sum += max(0, __ldg(a.old_lens + s));
        }
        if (a.missing && tid == 0) *a.missing = missing;
    }
    // every block has read the list's length: the last one writes the new one
    __syncthreads();
    if (tid == 0) {
        __threadfence();
        if (atomicAdd(a.ticket, 1u) == gridDim.x - 1) {
            *a.ticket = 0;
            if (done) *a.num_free = num_free + R - A;
        }
    }
}

}  // namespace

int launch_pages_update(const PagesUpdateArgs& a, const DeviceInfo& dev, cudaStream_t stream) {
    PagesParams p;
    p.a = a;
    p.page_shift = 0;
    while ((1 << p.page_shift) < a.page_size) ++p.page_shift;
    const int smem = 3 * (a.num_seqs + 1) * (int)sizeof(int);
    static std::mutex mu;
    static bool configured[64] = {};
    if (dev.device < 0 || dev.device >= 64) return BP_ERR_UNSUPPORTED;
    {
        std::lock_guard<std::mutex> lock(mu);
        if (!configured[dev.device]) {
            if (cudaFuncSetAttribute(pages_update_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                     3 * (kPagesMaxSeqs + 1) * (int)sizeof(int)) != cudaSuccess)
                return BP_ERR_CUDA;
            configured[dev.device] = true;
        }
    }
    const long long tokens = a.positions || a.slots ? a.total_new : 0;
    const long long blocks = (tokens + 8ll * a.num_seqs) / (kPagesThreads * kPerThread) + 1;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.gridDim = dim3((unsigned)std::min<long long>(blocks, dev.sm_count), 1, 1);
    cfg.blockDim = dim3(kPagesThreads, 1, 1);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, pages_update_kernel, p) == cudaSuccess ? BP_OK : BP_ERR_CUDA;
}

}  // namespace bp
