// pages.hip -- pages and slots of a paged cache from request lengths (gfx950).
//
//   page_extend   admits the new tokens of B sequences in order, hands pages of a
//                 free list to them, enters those in the block table and writes
//                 the slot and position of every token;
//   page_release  pushes the pages behind the kept lengths on the free list.
//
// Both are a prefix sum over the sequences (one workgroup: B <= 8192) followed by
// a flat pass over tokens and pages, each of which finds its sequence by bisection
// in the prefix sums.  All of it is integer arithmetic in a fixed order.
#include "spire_internal.h"

namespace spire {

constexpr int kPageThreads = 1024;
constexpr int kFillThreads = 256;
constexpr int kFillTokens = 4;  // consecutive tokens per thread

// What the prefix sums leave for the flat pass (workspace, B entries each).
struct PageState {
    int32_t *head;    // [0]: free pages before, [1]: pages handed out or pushed
    int32_t *first;   // pages of the sequences before b
    int32_t *len;     // lengths before (extend), first column pushed (release)
    int32_t *given;   // pages of b; -1: refused
};

__host__ __device__ __forceinline__ PageState page_state(void *ws, int B) {
    int32_t *w = static_cast<int32_t *>(ws);
    const int n = (B + 63) & ~63;
    return PageState{w, w + 64, w + 64 + n, w + 64 + 2 * n};
}

// Exclusive prefix sum over the workgroup's threads; `total` is the whole sum.
__device__ __forceinline__ int64_t scan_block(int64_t x, int64_t *sums, int64_t &total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int64_t incl = x;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const int64_t v = __shfl_up(incl, off);
        if (lane >= off) incl += v;
    }
    __syncthreads();  // the previous scan's sums have been read
    if (lane == 63) sums[wave] = incl;
    __syncthreads();
    int64_t before = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < kPageThreads / 64; ++w) {
        before += w < wave ? sums[w] : 0;
        total += sums[w];
    }
    return before + incl - x;
}

__device__ __forceinline__ int64_t pages_of(int64_t tokens, int page_size) {
    return (tokens + page_size - 1) / page_size;
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

__global__ __launch_bounds__(kPageThreads) void extend_scan_kernel(ExtendArgs a) {
    __shared__ int64_t sums[kPageThreads / 64];
    const int tid = threadIdx.x;
    const int per = (a.B + kPageThreads - 1) / kPageThreads;
    const int b0 = tid * per < a.B ? tid * per : a.B;
    const int b1 = b0 + per < a.B ? b0 + per : a.B;
    const int64_t room = (int64_t)a.max_blocks * a.page_size;
    auto want = [&](int b, int64_t &len, int64_t &fresh) -> int64_t {  // pages of b, -1: beyond its table row
        len = a.lens[b] < 0 ? 0 : a.lens[b];
        fresh = a.new_tokens[b] < 0 ? 0 : a.new_tokens[b];
        if (fresh == 0) return 0;
        const int64_t end = len + fresh;
        return end > room || end > INT32_MAX ? -1 : pages_of(end, a.page_size) - pages_of(len, a.page_size);
    };
    int64_t need = 0, tokens = 0, len, fresh;
    for (int b = b0; b < b1; ++b) {
        const int64_t w = want(b, len, fresh);
        need += w > 0 ? w : 0;
        tokens += fresh;
    }
    int64_t all_need, all_tokens;
    int64_t page = scan_block(need, sums, all_need), tok = scan_block(tokens, sums, all_tokens);
    const int n = clamp_count(*a.n_free, a.pool);
    int64_t mine = 0;
    for (int b = b0; b < b1; ++b) {
        const int64_t w = want(b, len, fresh);
        const bool ok = w >= 0 && page + w <= n && tok + fresh <= a.max_tokens;
        a.cu[b] = tok > INT32_MAX ? INT32_MAX : (int)tok;
        a.st.first[b] = page > n ? n : (int)page;
        a.st.len[b] = (int)len;
        a.st.given[b] = ok ? (int)w : -1;
        a.lens_out[b] = ok && fresh > 0 ? (int)(len + fresh) : a.lens[b];
        mine += ok ? w : 0;
        page += w > 0 ? w : 0;
        tok += fresh;
    }
    int64_t given;
    scan_block(mine, sums, given);
    if (tid == 0) {
        a.cu[a.B] = all_tokens > INT32_MAX ? INT32_MAX : (int)all_tokens;
        a.st.head[0] = n;
        a.st.head[1] = (int)given;
        *a.n_free_out = n - (int)given;
    }
}

// last b with v[b] <= x (v[0] <= x, v not decreasing)
__device__ __forceinline__ int last_at_most(const int32_t *v, int B, int x) {
    int lo = 0, hi = B - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (v[mid] <= x) lo = mid; else hi = mid - 1;
    }
    return lo;
}

__global__ __launch_bounds__(kFillThreads) void extend_fill_kernel(ExtendArgs a) {
    const int64_t id = (int64_t)blockIdx.x * kFillThreads + threadIdx.x;
    const int64_t threads = (int64_t)gridDim.x * kFillThreads;
    const int n = a.st.head[0], given = a.st.head[1], total = a.cu[a.B];
    for (int64_t q = id; q < given; q += threads) {  // pages handed out
        const int b = last_at_most(a.st.first, a.B, (int)q);
        const int64_t col = pages_of(a.st.len[b], a.page_size) + (q - a.st.first[b]);
        a.table[(int64_t)b * a.max_blocks + col] = a.free_pages[n - 1 - q];
    }
    for (int64_t i0 = id * kFillTokens; i0 < a.max_tokens; i0 += threads * kFillTokens) {
        int b = i0 < total ? last_at_most(a.cu, a.B, (int)i0) : 0;
        for (int64_t i = i0; i < i0 + kFillTokens && i < a.max_tokens; ++i) {
            int64_t slot = -1;
            int pos = 0;
            if (i < total) {
                while (a.cu[b + 1] <= i) ++b;
                if (a.st.given[b] >= 0) {
                    pos = a.st.len[b] + (int)(i - a.cu[b]);
                    const int64_t col = pos / a.page_size, held = pages_of(a.st.len[b], a.page_size);
                    const int page = col < held ? a.table[(int64_t)b * a.max_blocks + col]
                                                : a.free_pages[n - 1 - (a.st.first[b] + (col - held))];
                    if (page >= 0) slot = (int64_t)page * a.page_size + (pos - col * a.page_size);
                }
            }
            a.slots[i] = slot;
            a.positions[i] = pos;
        }
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

__global__ __launch_bounds__(kPageThreads) void release_scan_kernel(ReleaseArgs a) {
    __shared__ int64_t sums[kPageThreads / 64];
    const int tid = threadIdx.x;
    const int per = (a.B + kPageThreads - 1) / kPageThreads;
    const int b0 = tid * per < a.B ? tid * per : a.B;
    const int b1 = b0 + per < a.B ? b0 + per : a.B;
    auto cut = [&](int b, int &kept, int64_t &c0) -> int64_t {  // pages of b that go back, from column c0
        const int len = a.lens[b], keep = a.keep[b] < 0 ? 0 : a.keep[b];
        kept = keep < len ? keep : len;
        c0 = pages_of(kept > 0 ? kept : 0, a.page_size);
        int64_t c1 = pages_of(len > 0 ? len : 0, a.page_size);
        if (c1 > a.max_blocks) c1 = a.max_blocks;
        return c1 > c0 ? c1 - c0 : 0;
    };
    int64_t mine = 0, c0, all;
    int kept;
    for (int b = b0; b < b1; ++b) mine += cut(b, kept, c0);
    int64_t at = scan_block(mine, sums, all);
    const int n = clamp_count(*a.n_free, a.pool);
    const int64_t room = a.pool - n;
    for (int b = b0; b < b1; ++b) {
        const int64_t c = cut(b, kept, c0);
        a.st.first[b] = at > room ? (int)room : (int)at;
        a.st.len[b] = (int)(c0 > a.max_blocks ? a.max_blocks : c0);
        a.st.given[b] = (int)c;
        a.lens_out[b] = kept;
        at += c;
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

static unsigned fill_grid(int64_t items) {
    const int64_t g = (items + kFillThreads - 1) / kFillThreads;
    return (unsigned)(g < 1 ? 1 : (g > 4096 ? 4096 : g));
}

hipError_t launch_page_extend(const PageExtend &x, hipStream_t st) {
    ExtendArgs a{x.table, x.lens, x.new_tokens, x.free_pages, x.n_free, x.slots, x.positions, x.cu,
                 x.lens_out, x.n_free_out, x.B, x.page_size, x.max_blocks, x.pool, x.max_tokens,
                 page_state(x.ws, x.B)};
    hipLaunchKernelGGL(extend_scan_kernel, dim3(1), dim3(kPageThreads), 0, st, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(extend_fill_kernel, dim3(fill_grid(x.max_tokens / kFillTokens + x.B)), dim3(kFillThreads), 0, st, a);
    return hipGetLastError();
}

hipError_t launch_page_release(const PageRelease &x, hipStream_t st) {
    ReleaseArgs a{x.table, x.lens, x.keep, x.free_pages, x.n_free, x.lens_out, x.n_free_out, x.B,
                  x.page_size, x.max_blocks, x.pool, page_state(x.ws, x.B)};
    hipLaunchKernelGGL(release_scan_kernel, dim3(1), dim3(kPageThreads), 0, st, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(release_fill_kernel, dim3(fill_grid((int64_t)x.B * 4)), dim3(kFillThreads), 0, st, a);
    return hipGetLastError();
}

}  // namespace spire
