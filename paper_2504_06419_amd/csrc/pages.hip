// pages.hip -- pages and slots of a paged cache from request lengths (gfx950).
//
//   page_extend   admits the new tokens of B sequences in order, hands pages of a
//                 free list to them, enters those in the block table and writes
//                 the slot and position of every token;
//   page_release  pushes the pages behind the kept lengths on the free list.
//
// Both are a prefix sum over the sequences (one workgroup: B <= 8192) followed by
// a flat pass over tokens and pages, each of which finds its sequence by bisection
// in the prefix sums.  All of it is integer arithmetic in a fixed order.  Lengths may
// be updated in place, so no second workgroup can form the sums for itself: the flat
// pass is a launch of its own, or the same workgroup's where the tokens are few.
// Bound by latency (a chain of dependent loads, and the launches), not by bytes.
#include "spire_internal.h"

namespace spire {

constexpr int kPageThreads = 1024;
constexpr int kPagePer = 8;        // sequences a thread: B <= 8192
constexpr int kOneLaunchB = 1024;  // sequences whose sums stand in LDS
// Tokens up to which the flat pass is the scanning workgroup's own.  256 sequences in one
// launch and in two, on the device: 1024 tokens 5.8 and 6.5 us, 2048 7.6 and 6.6, 4096 9.5
// and 6.5 (1024 sequences, 1024 tokens: 7.1 and 9.5); a launch costs the host 2.5 us.
constexpr int kOneLaunchTokens = 2048;
constexpr int kFillThreads = 256;

// What the prefix sums leave for the flat pass (workspace, B entries each).
struct PageState {
    int32_t *head;    // [0]: free pages before, [1]: pages pushed (release)
    int32_t *first;   // pages of the sequences before b
    int32_t *len;     // lengths before (extend), first column pushed (release)
    int32_t *given;   // pages of b; -1: refused (extend)
};

__host__ __device__ __forceinline__ PageState page_state(void *ws, int B) {
    int32_t *w = static_cast<int32_t *>(ws);
    const int n = (B + 63) & ~63;
    return PageState{w, w + 64, w + 64 + n, w + 64 + 2 * n};
}

// Exclusive prefix sums of two counts over the workgroup's threads, x and y left as
// the sums before the thread, the whole sums in all_x and all_y.
struct ScanSums {
    int64_t x[kPageThreads / 64], y[kPageThreads / 64];
};

__device__ __forceinline__ void scan_block(int64_t &x, int64_t &y, ScanSums &sums, int64_t &all_x, int64_t &all_y) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
    int64_t ix = x, iy = y;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const int64_t u = __shfl_up(ix, off), v = __shfl_up(iy, off);
        if (lane >= off) {
            ix += u;
            iy += v;
        }
    }
    if (lane == 63) {
        sums.x[wave] = ix;
        sums.y[wave] = iy;
    }
    __syncthreads();
    x = ix - x;
    y = iy - y;
    all_x = all_y = 0;
    for (int w = 0; w < waves; ++w) {
        if (w == wave) {
            x += all_x;
            y += all_y;
        }
        all_x += sums.x[w];
        all_y += sums.y[w];
    }
}

// Sum over the workgroup's threads, in every thread.
__device__ __forceinline__ int sum_block(int x, int *sums) {
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) x += __shfl_xor(x, off);
    if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = x;
    __syncthreads();
    int all = 0;
    for (int w = 0; w < (int)(blockDim.x >> 6); ++w) all += sums[w];
    return all;
}

// tokens <= INT32_MAX, page_size >= 1
__device__ __forceinline__ int pages_of(int tokens, int page_size) {
    return (int)(((uint32_t)tokens + (uint32_t)page_size - 1u) / (uint32_t)page_size);
}

struct ExtendArgs {
    int32_t *table;
    const int32_t *lens, *new_tokens, *free_pages, *n_free;
    int64_t *slots;
    int32_t *positions, *cu, *lens_out, *n_free_out;
    int32_t B, page_size, max_blocks, pool, max_tokens;
    PageState st;
};

__device__ __forceinline__ int clamp_count(int n, int pool) { return n < 0 ? 0 : (n > pool ? pool : n); }

// last b with v[b] <= x (v[0] <= x, v not decreasing)
__device__ __forceinline__ int last_at_most(const int32_t *v, int B, int x) {
    int lo = 0, hi = B - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (v[mid] <= x) lo = mid; else hi = mid - 1;
    }
    return lo;
}

// The flat pass over tokens, by `threads` threads of which this is `id`.  n: free pages
// before; first, len, given_of and cu as the sums left them.
__device__ __forceinline__ void extend_fill(const ExtendArgs &a, int64_t id, int64_t threads, int n,
                                            const int32_t *first, const int32_t *len, const int32_t *given_of,
                                            const int32_t *cu) {
    const int total = cu[a.B];
    for (int64_t i = id; i < a.max_tokens; i += threads) {
        int64_t slot = -1;
        int pos = 0;
        const int b = i < total ? last_at_most(cu, a.B, (int)i) : -1;
        if (b >= 0 && given_of[b] >= 0) {
            pos = len[b] + (int)(i - cu[b]);
            const int col = (int)((uint32_t)pos / (uint32_t)a.page_size), held = pages_of(len[b], a.page_size);
            int32_t *const entry = a.table + (int64_t)b * a.max_blocks + col;
            const int page = col < held ? *entry : a.free_pages[n - 1 - (first[b] + (col - held))];
            if (col >= held && pos == col * a.page_size) *entry = page;  // the first token of a page handed out
            if (page >= 0) slot = (int64_t)page * a.page_size + (pos - col * a.page_size);
        }
        a.slots[i] = slot;
        a.positions[i] = pos;
    }
}

// ONE: the flat pass too, from sums in LDS (B <= kOneLaunchB).  PER: most sequences a
// thread; they are held in registers, so that their loads overlap.
template <bool ONE, int PER>
__global__ __launch_bounds__(kPageThreads) void extend_scan_kernel(ExtendArgs a) {
    __shared__ ScanSums sums;
    __shared__ int given_sums[kPageThreads / 64];
    __shared__ int32_t local[ONE ? 4 * kOneLaunchB + 1 : 1];
    int32_t *const first = ONE ? local : a.st.first, *const lens = ONE ? local + kOneLaunchB : a.st.len;
    int32_t *const given_of = ONE ? local + 2 * kOneLaunchB : a.st.given, *const cu = ONE ? local + 3 * kOneLaunchB : a.cu;
    const int tid = threadIdx.x;
    const int per = (a.B + (int)blockDim.x - 1) / (int)blockDim.x;
    const int b0 = tid * per < a.B ? tid * per : a.B;
    const int b1 = b0 + per < a.B ? b0 + per : a.B;
    const int64_t room = (int64_t)a.max_blocks * a.page_size;
    auto want = [&](int b, int &len, int &fresh) -> int {  // pages of b, -1: beyond its table row
        len = a.lens[b] < 0 ? 0 : a.lens[b];
        fresh = a.new_tokens[b] < 0 ? 0 : a.new_tokens[b];
        if (fresh == 0) return 0;
        const int64_t end = (int64_t)len + fresh;
        return end > room || end > INT32_MAX ? -1 : pages_of((int)end, a.page_size) - pages_of(len, a.page_size);
    };
    const int n = clamp_count(*a.n_free, a.pool);
    int64_t page = 0, tok = 0, all_need, all_tokens;
    int len[PER], fresh[PER], want_of[PER];
#pragma unroll
    for (int j = 0; j < PER; ++j) {
        if (b0 + j >= b1) continue;
        want_of[j] = want(b0 + j, len[j], fresh[j]);
        page += want_of[j] > 0 ? want_of[j] : 0;
        tok += fresh[j];
    }
    scan_block(page, tok, sums, all_need, all_tokens);
    int mine = 0;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
        const int b = b0 + j, w = want_of[j];
        if (b >= b1) continue;
        const bool ok = w >= 0 && page + w <= n && tok + fresh[j] <= a.max_tokens;
        const int at = tok > INT32_MAX ? INT32_MAX : (int)tok;
        cu[b] = at;
        if (ONE) a.cu[b] = at;
        first[b] = page > n ? n : (int)page;
        lens[b] = len[j];
        given_of[b] = ok ? w : -1;
        if (ok && fresh[j] > 0) a.lens_out[b] = len[j] + fresh[j];
        else if (a.lens_out != a.lens) a.lens_out[b] = a.lens[b];
        mine += ok ? w : 0;
        page += w > 0 ? w : 0;
        tok += fresh[j];
    }
    const int given = sum_block(mine, given_sums);  // and every thread's sums are written
    if (tid == 0) {
        const int at = all_tokens > INT32_MAX ? INT32_MAX : (int)all_tokens;
        a.cu[a.B] = at;
        if (ONE) cu[a.B] = at;
        if (!ONE) a.st.head[0] = n;
        *a.n_free_out = n - given;
    }
    if (ONE) {
        __syncthreads();
        extend_fill(a, tid, blockDim.x, n, first, lens, given_of, cu);
    }
}

// LOCAL: the sums are brought to LDS at once (B <= kOneLaunchB); a bisection through L2 is
// a chain of log2 B loads (64 prompts of 16 to 16384 tokens: 5.8 and 7.1 us at 4 tokens a
// thread, 4.3 at one).
template <bool LOCAL>
__global__ __launch_bounds__(kFillThreads) void extend_fill_kernel(ExtendArgs a) {
    const int64_t id = (int64_t)blockIdx.x * kFillThreads + threadIdx.x, threads = (int64_t)gridDim.x * kFillThreads;
    const int n = a.st.head[0];
    if constexpr (LOCAL) {
        __shared__ int32_t local[4 * kOneLaunchB + 1];
        for (int b = threadIdx.x; b < a.B; b += kFillThreads) {
            local[b] = a.st.first[b];
            local[kOneLaunchB + b] = a.st.len[b];
            local[2 * kOneLaunchB + b] = a.st.given[b];
            local[3 * kOneLaunchB + b] = a.cu[b];
        }
        if (threadIdx.x == 0) local[3 * kOneLaunchB + a.B] = a.cu[a.B];
        __syncthreads();
        extend_fill(a, id, threads, n, local, local + kOneLaunchB, local + 2 * kOneLaunchB,
                    local + 3 * kOneLaunchB);
    } else {
        extend_fill(a, id, threads, n, a.st.first, a.st.len, a.st.given, a.cu);
    }
}

struct ReleaseArgs {
    const int32_t *table, *lens, *keep;
    int32_t *free_pages;
    const int32_t *n_free;
    int32_t *lens_out, *n_free_out;
    int32_t B, page_size, max_blocks, pool;
    PageState st;
};

template <int PER>
__global__ __launch_bounds__(kPageThreads) void release_scan_kernel(ReleaseArgs a) {
    __shared__ ScanSums sums;
    const int tid = threadIdx.x;
    const int per = (a.B + (int)blockDim.x - 1) / (int)blockDim.x;
    const int b0 = tid * per < a.B ? tid * per : a.B;
    const int b1 = b0 + per < a.B ? b0 + per : a.B;
    auto cut = [&](int b, int &kept, int &c0) -> int {  // pages of b that go back, from column c0
        const int len = a.lens[b], keep = a.keep[b] < 0 ? 0 : a.keep[b];
        kept = keep < len ? keep : len;
        c0 = pages_of(kept > 0 ? kept : 0, a.page_size);
        int c1 = pages_of(len > 0 ? len : 0, a.page_size);
        if (c1 > a.max_blocks) c1 = a.max_blocks;
        return c1 > c0 ? c1 - c0 : 0;
    };
    const int n = clamp_count(*a.n_free, a.pool);
    int64_t at = 0, unused = 0, all, all_unused;
    int kept[PER], c0[PER], c[PER];
#pragma unroll
    for (int j = 0; j < PER; ++j) {
        if (b0 + j >= b1) continue;
        c[j] = cut(b0 + j, kept[j], c0[j]);
        at += c[j];
    }
    scan_block(at, unused, sums, all, all_unused);
    const int64_t room = a.pool - n;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
        const int b = b0 + j;
        if (b >= b1) continue;
        a.st.first[b] = at > room ? (int)room : (int)at;
        a.st.len[b] = c0[j] > a.max_blocks ? a.max_blocks : c0[j];
        a.lens_out[b] = kept[j];
        at += c[j];
    }
    __syncthreads();
    if (tid == 0) {
        const int pushed = (int)(all < room ? all : room);
        a.st.head[0] = n;
        a.st.head[1] = pushed;
        *a.n_free_out = n + pushed;
    }
}

__global__ __launch_bounds__(kFillThreads) void release_fill_kernel(ReleaseArgs a) {
    const int n = a.st.head[0], pushed = a.st.head[1];
    for (int64_t q = (int64_t)blockIdx.x * kFillThreads + threadIdx.x; q < pushed; q += (int64_t)gridDim.x * kFillThreads) {
        const int b = last_at_most(a.st.first, a.B, (int)q);
        a.free_pages[n + q] = a.table[(int64_t)b * a.max_blocks + a.st.len[b] + (q - a.st.first[b])];
    }
}

size_t page_workspace_bytes(int B) { return 4 * (64 + 3 * (((size_t)B + 63) & ~(size_t)63)); }

// whole waves for B sequences
static unsigned scan_threads(int B) { return (unsigned)(B < 1 ? 64 : (B + 63) / 64 * 64); }

static unsigned fill_grid(int64_t items) {
    const int64_t g = (items + kFillThreads - 1) / kFillThreads;
    return (unsigned)(g < 1 ? 1 : (g > 4096 ? 4096 : g));
}

hipError_t launch_page_extend(const PageExtend &x, hipStream_t st) {
    ExtendArgs a{x.table, x.lens, x.new_tokens, x.free_pages, x.n_free, x.slots, x.positions, x.cu,
                 x.lens_out, x.n_free_out, x.B, x.page_size, x.max_blocks, x.pool, x.max_tokens,
                 page_state(x.ws, x.B)};
    if (x.B > kPageThreads * kPagePer) return hipErrorInvalidValue;
    if (x.B <= kOneLaunchB && x.max_tokens <= kOneLaunchTokens) {
        // 512 threads start and scan sooner than 1024 (64 sequences, 320 tokens: 4.4 us against 5.9;
        // 256 and 1024: 5.8 and 6.3), which have fewer tokens each (256 and 2048: 7.8 and 7.6)
        const int threads = x.B <= 512 && x.max_tokens <= 1536 ? 512 : kPageThreads;
        hipLaunchKernelGGL((extend_scan_kernel<true, 1>), dim3(1), dim3(threads), 0, st, a);
        return hipGetLastError();
    }
    if (x.B <= kPageThreads) hipLaunchKernelGGL((extend_scan_kernel<false, 1>), dim3(1), dim3(scan_threads(x.B)), 0, st, a);
    else hipLaunchKernelGGL((extend_scan_kernel<false, kPagePer>), dim3(1), dim3(kPageThreads), 0, st, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const dim3 grid(fill_grid(x.max_tokens)), block(kFillThreads);
    if (x.B <= kOneLaunchB) hipLaunchKernelGGL(extend_fill_kernel<true>, grid, block, 0, st, a);
    else hipLaunchKernelGGL(extend_fill_kernel<false>, grid, block, 0, st, a);
    return hipGetLastError();
}

hipError_t launch_page_release(const PageRelease &x, hipStream_t st) {
    ReleaseArgs a{x.table, x.lens, x.keep, x.free_pages, x.n_free, x.lens_out, x.n_free_out, x.B,
                  x.page_size, x.max_blocks, x.pool, page_state(x.ws, x.B)};
    if (x.B > kPageThreads * kPagePer) return hipErrorInvalidValue;
    if (x.B <= kPageThreads) hipLaunchKernelGGL(release_scan_kernel<1>, dim3(1), dim3(scan_threads(x.B)), 0, st, a);
    else hipLaunchKernelGGL(release_scan_kernel<kPagePer>, dim3(1), dim3(kPageThreads), 0, st, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(release_fill_kernel, dim3(fill_grid((int64_t)x.B * 4)), dim3(kFillThreads), 0, st, a);
    return hipGetLastError();
}

}  // namespace spire
