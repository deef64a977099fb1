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
//
// What it has to move is small (1024 sequences with 370,000 new tokens: 4.5 MB, 0.7 us); what it takes are round trips: the
// lengths, the scan, the searches, the list's pages, the table.  2.3 us a call for one sequence, of which a launch in a graph
// is 1.5 and more; 8.4 for that large one.
#include <limits.h>

#include <algorithm>
#include <mutex>

#include "common.cuh"
#include "ptx_sm103.cuh"

namespace bp {
namespace {

constexpr int kPerThread = 4;  // tokens in a row
constexpr int kCopied = 12288; // of up to so many sequences the old lengths are in shared memory too
constexpr int pages_smem(int seqs) { return ((seqs <= kCopied ? 4 : 3) * seqs + 3) * (int)sizeof(int); }
constexpr int kMostSmem = pages_smem(kCopied) > pages_smem(kPagesMaxSeqs) ? pages_smem(kCopied) : pages_smem(kPagesMaxSeqs);
static_assert(kMostSmem <= 226 * 1024, "a block's shared memory");

struct PagesParams {
    PagesUpdateArgs a;
    int page_shift;
    int may_overflow;  // the lengths' sum may pass 31 bits
    int wide;  // positions and slots may be written by 16 bytes
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

// THREADS: 128 for up to 128 sequences whose tokens are one pass of the grid: the time is that of the steps below one after
// the other, barriers among them (us a call in graphs, against 512: 1 sequence of 1 token 2.3 and 2.7, of 8192 tokens 2.9 and
// 3.4, 8 of 16 2.7 and 3.0, 64 of 16 3.4 and 3.2, 128 of 16 3.5 and 3.8).  512 beyond: 256 of 16 5.7 against 6.4, 1024
// sequences of up to 2000 tokens 8.4 against 12.6.
template <int THREADS>
__global__ void __launch_bounds__(THREADS) pages_update_kernel(const __grid_constant__ PagesParams p) {
    constexpr int kWarps = THREADS / 32;
    // [3][num_seqs + 1]: new tokens, taken pages, given pages of the sequences before; where there is room, old_lens
    extern __shared__ int sums[];
    __shared__ int warp_sums[4][kWarps], warps_before[4][kWarps + 1];
    griddep_launch_dependents();
    griddep_wait();
    const PagesUpdateArgs& a = p.a;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, n = a.num_seqs, P = 1 << p.page_shift;
    int* const tokens = sums;
    int* const taken = sums + n + 1;
    int* const given = sums + 2 * (n + 1);
    int* const copy = n <= kCopied ? sums + 3 * (n + 1) : nullptr;
    const int* const olds = copy ? copy : a.old_lens;
    auto pages_of = [&](int len) { return (int)(((unsigned)len + P - 1) >> p.page_shift); };

    // ---- prefix sums over the sequences, THREADS at a time
    const int num_free = *a.num_free;
    int carry[4] = {0, 0, 0, 0};  // tokens, taken, given; keys after the step
    bool bad = num_free < 0 || num_free > a.num_pages;
    long long all_keys = 0, all_given = 0;
    const bool writes = blockIdx.x == 0;
    for (int base = 0; base < n; base += THREADS) {
        const int s = base + tid;
        int v[4] = {0, 0, 0, 0};
        if (s < n) {
            const int o = __ldg(a.old_lens + s), w = __ldg(a.new_lens + s);
            if (copy) copy[s] = o;
            if (o < 0 || w < 0 || pages_of(o) > a.pages_per_seq || pages_of(w) > a.pages_per_seq) {
                bad = true;
            } else {
                v[0] = max(0, w - o);
                v[1] = max(0, pages_of(w) - pages_of(o));
                v[2] = max(0, pages_of(o) - pages_of(w));
                v[3] = w;
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
        if (lane == 31)
#pragma unroll
            for (int k = 0; k < 4; ++k) warp_sums[k][warp] = sum[k];
        __syncthreads();
        if (tid < 4) {  // (a few numbers: one after the other)
            int before = 0;
            for (int w = 0; w < kWarps; ++w) {
                warps_before[tid][w] = before;
                before += warp_sums[tid][w];
            }
            warps_before[tid][kWarps] = before;
        }
        __syncthreads();  // (and the sums before are written again only behind the next one)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            sum[k] += carry[k] + warps_before[k][warp];
            carry[k] += warps_before[k][kWarps];
        }
        if (s < n) {
            tokens[s + 1] = sum[0];
            taken[s + 1] = sum[1];
            given[s + 1] = sum[2];
            if (writes && a.cu_kv) a.cu_kv[s + 1] = sum[3];  // (rewritten below where the step does not take place)
        }
        if (base + THREADS < n) __syncthreads();
    }
    if (tid == 0) tokens[0] = taken[0] = given[0] = 0;
    if (p.may_overflow) {  // the sums above may pass 31 bits: these tell
        __shared__ long long long_sums[2][kWarps];
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            all_keys += __shfl_xor_sync(0xffffffffu, all_keys, o);
            all_given += __shfl_xor_sync(0xffffffffu, all_given, o);
        }
        if (lane == 0) long_sums[0][warp] = all_keys, long_sums[1][warp] = all_given;
        __syncthreads();
        all_keys = all_given = 0;
        for (int w = 0; w < kWarps; ++w) all_keys += long_sums[0][w], all_given += long_sums[1][w];
        bad = bad || all_keys > INT_MAX || all_given > a.num_pages;
    }
    const int A = carry[1], R = carry[2];
    bad = __syncthreads_or(bad) || R > a.num_pages || ((a.positions || a.slots) && carry[0] > a.total_new) ||
          (long long)num_free + R - A > a.num_pages;
    const int missing = bad ? 0 : max(0, A - R - num_free);
    const bool done = !bad && missing == 0;
    if (bad && writes && tid == 0) raise_error(a.err_word, kErrDeviceArg);

    // the page that is taken as number i, and the one that is given back as number i
    auto given_page = [&](int i) {
        const int s = place_of(given, n, i);
        return a.block_table[(size_t)s * a.pages_per_seq + pages_of(olds[s]) + i - given[s + 1]];  // (the last of its pages)
    };
    auto taken_page = [&](int i) { return i < R ? given_page(i) : a.free_pages[num_free - 1 - (i - R)]; };
    // (pages by the last threads first, tokens by the first: few of both are moved at the same time)
    const int t0 = blockIdx.x * THREADS + tid, stride = gridDim.x * THREADS, back = stride - 1 - t0;
    if (done) {
        for (int i = back; i < A; i += stride) {
            const int s = place_of(taken, n, i);
            const int page = taken_page(i);
            if ((unsigned)page >= (unsigned)a.num_pages) raise_error(a.err_word, kErrDeviceArg);
            a.block_table[(size_t)s * a.pages_per_seq + pages_of(olds[s]) + i - taken[s]] = page;
        }
        for (int i = A + back; i < R; i += stride) {
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
            int pos[kPerThread];
            int64_t slot[kPerThread];
#pragma unroll
            for (int k = 0; k < kPerThread; ++k) {
                const int x = t + k;
                pos[k] = -1;
                slot[k] = -1;
                if (x < real) {
                    while (x >= tokens[s + 1]) ++s, fresh = true;
                    if (fresh) old = olds[s], held = pages_of(old), at = -1, fresh = false;
                    pos[k] = old + x - tokens[s];
                    const int j = pos[k] >> p.page_shift;
                    if (j != at) {
                        at = j;
                        page = j < held ? a.block_table[(size_t)s * a.pages_per_seq + j] : taken_page(taken[s] + j - held);
                    }
                    slot[k] = ((int64_t)page << p.page_shift) + (pos[k] & (P - 1));
                }
            }
            if (p.wide && t + kPerThread <= a.total_new) {
                if (a.positions) *reinterpret_cast<int4*>(a.positions + t) = make_int4(pos[0], pos[1], pos[2], pos[3]);
                if (a.slots) {
                    *reinterpret_cast<longlong2*>(a.slots + t) = make_longlong2(slot[0], slot[1]);
                    *reinterpret_cast<longlong2*>(a.slots + t + 2) = make_longlong2(slot[2], slot[3]);
                }
            } else {
#pragma unroll
                for (int k = 0; k < kPerThread; ++k) {
                    if (t + k >= a.total_new) break;
                    if (a.positions) a.positions[t + k] = pos[k];
                    if (a.slots) a.slots[t + k] = slot[k];
                }
            }
        }
    }
    if (writes) {
        if (a.cu_new)
            for (int s = tid; s <= n; s += THREADS) a.cu_new[s] = done ? tokens[s] : 0;
        if (a.cu_kv && tid == 0) a.cu_kv[0] = 0;
        if (a.cu_kv && !done) {  // the lengths stay: their prefix sums (1024 sequences 4.7 us a call, 12.2 by one thread)
            for (int base = 0, before = 0; base < n; base += THREADS) {
                const int s = base + tid;
                int sum = s < n ? max(0, __ldg(a.old_lens + s)) : 0;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const int y = __shfl_up_sync(0xffffffffu, sum, o);
                    if (lane >= o) sum += y;
                }
                if (lane == 31) warp_sums[0][warp] = sum;
                __syncthreads();
                sum += before;
                for (int w = 0; w < kWarps; ++w) {
                    if (w < warp) sum += warp_sums[0][w];
                    before += warp_sums[0][w];
                }
                if (s < n) a.cu_kv[s + 1] = sum;
                __syncthreads();
            }
        }
        if (a.missing && tid == 0) *a.missing = missing;
    }
    // the list's new length, by the last block to finish: every one has read it then
    __syncthreads();
    if (tid == 0) {
        bool last = gridDim.x == 1;
        if (!last) {
            __threadfence();
            last = atomicAdd(a.ticket, 1u) == gridDim.x - 1;
            if (last) *a.ticket = 0;
        }
        if (last && done) *a.num_free = num_free + R - A;
    }
}

}  // namespace

int launch_pages_update(const PagesUpdateArgs& a, const DeviceInfo& dev, cudaStream_t stream) {
    PagesParams p;
    p.a = a;
    p.page_shift = 0;
    while ((1 << p.page_shift) < a.page_size) ++p.page_shift;
    p.wide = reinterpret_cast<uintptr_t>(a.positions) % 16 == 0 && reinterpret_cast<uintptr_t>(a.slots) % 16 == 0;
    p.may_overflow = (long long)a.num_seqs * a.pages_per_seq * a.page_size > INT_MAX;
    const long long tokens = a.positions || a.slots ? a.total_new : 0, work = (tokens + 8ll * a.num_seqs) / kPerThread;
    const bool small = a.num_seqs <= 128 && work <= 128ll * dev.sm_count;
    const auto kernel = small ? pages_update_kernel<128> : pages_update_kernel<512>;
    const int threads = small ? 128 : 512;
    static std::mutex mu;
    static bool configured[64] = {};
    if (dev.device < 0 || dev.device >= 64) return BP_ERR_UNSUPPORTED;
    {
        std::lock_guard<std::mutex> lock(mu);
        if (!configured[dev.device]) {
            if (cudaFuncSetAttribute(pages_update_kernel<512>, cudaFuncAttributeMaxDynamicSharedMemorySize, kMostSmem) != cudaSuccess)
                return BP_ERR_CUDA;
            configured[dev.device] = true;
        }
    }
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.gridDim = dim3((unsigned)std::min<long long>(work / threads + 1, dev.sm_count), 1, 1);
    cfg.blockDim = dim3((unsigned)threads, 1, 1);
    cfg.dynamicSmemBytes = pages_smem(a.num_seqs);
    cfg.stream = stream;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, p) == cudaSuccess ? BP_OK : BP_ERR_CUDA;
}

}  // namespace bp
