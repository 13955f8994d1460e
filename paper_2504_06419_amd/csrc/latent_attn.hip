// latent_attn.hip -- attention over a latent cache in fp32, and the merge of split
// sequences (gfx950).
//
// Any storage type (converted to fp32 on the way into LDS), alignment, page size
// and stride.  One workgroup of 4 waves per (group, 16-row block).  Per tile of 32
// keys: the rows are staged as fp32; wave w forms the scores' partial sums over
// its quarter of the Dc + 64 dimensions (v_mfma_f32_16x16x4_f32, S^T = K Q^T); the
// quarters meet in LDS and every wave takes the online softmax of all 32 keys;
// then wave w accumulates its quarter of the latent, O^T += C^T P^T.  The path of
// full precision checks.  Nothing is in flight while a tile is scored, and each 16-row
// block is a workgroup of its own that reads and converts every row again, so a small
// call is a chain of dependent steps (4 sequences of 512 rows of 320, 8 heads, k = 4:
// 16.7 us and 5.2 for the merge) and a large one waits at every tile (64 sequences of
// 512 to 16384 rows, 16 heads, k = 4: 2.8 ms bf16, 3.0 ms fp32; its products are about
// 0.33 ms at the peak of the fp32 matrix instructions).
#include "convert.h"
#include "combine.h"
#include "latent_common.h"

namespace spire {

typedef float f32x4_t __attribute__((ext_vector_type(4)));

constexpr int kLatF32Tile = kLatentTile;

__device__ __forceinline__ float e4m3fn_f32(uint32_t x) {
    return __builtin_amdgcn_cvt_f32_fp8((int)x, 0);
}

template <int DC>
__global__ __launch_bounds__(256) void latent_f32_kernel(Latent a) {
    constexpr int DK = DC + kLatentDr, LD = DK + 4;  // row stride: 16 rows on distinct banks
    constexpr int QS = DK / 64;      // 16-dimension steps of a wave's quarter
    constexpr int NB = DC / 64;      // 16-dimension output blocks of a wave's quarter
    __shared__ float ks[kLatF32Tile][LD];
    __shared__ float sp[4][kLatF32Tile][17];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int n16 = lane & 15, j = lane >> 4;
    const Problem &p = a.p;
    const Plan &pl = a.pl;
    int g, u;
    latent_place(a, g, u);
    int64_t pos = 0, end = 0;
    int seg = 0, tile = 0;
    if (!latent_start<256>(a, g, u, reinterpret_cast<int32_t *>(&ks[0][0]), seg, tile, pos, end)) return;
    const int64_t begin = pos;
    const int i = u / a.hb, h = 16 * (u - i * a.hb) + n16;  // units are single blocks here
    const bool row_ok = h < p.Hq;
    const float kscale = p.kv.elem == 1 ? p.kv.k_scale[0] : 1.f;

    while (pos < end) {
        const int b = seg;
        const int n = effective_keys(p, b), tiles = latent_tiles<kLatF32Tile>(n), span = tiles + pl.seg_cost;
        const int64_t left = end - pos;
        const int te = left < (int64_t)(span - tile) ? tile + (int)left : span;
        if (tile < tiles) {
            const int t1 = te < tiles ? te : tiles;
            const int lim = n - p.k + i;  // visible keys of the block
            const int64_t qrow = (((int64_t)b * (p.k + 1) + i) * p.Hq + h);
            f32x4_t q[QS];
#pragma unroll
            for (int s = 0; s < QS; ++s) {
                const int d = wave * (DK / 4) + 16 * s + 4 * j;
                q[s] = f32x4_t{0.f, 0.f, 0.f, 0.f};
                if (row_ok) {
                    if (p.q_dtype == SPIRE_F32) {
                        q[s] = *reinterpret_cast<const f32x4_t *>(reinterpret_cast<const float *>(p.q) + qrow * DK + d);
                    } else {
                        const uint2 v = *reinterpret_cast<const uint2 *>(reinterpret_cast<const uint16_t *>(p.q) + qrow * DK + d);
                        q[s] = f32x4_t{__uint_as_float(v.x << 16), __uint_as_float(v.x & 0xFFFF0000u),
                                       __uint_as_float(v.y << 16), __uint_as_float(v.y & 0xFFFF0000u)};
                    }
                }
            }
            f32x4_t acc[NB];
#pragma unroll
            for (int x = 0; x < NB; ++x) acc[x] = f32x4_t{0.f, 0.f, 0.f, 0.f};
            float m = -INFINITY, l = 0.f;
            for (int tt = tile; tt < t1; ++tt) {
                const int key0 = tt * kLatF32Tile;
                if (key0 >= lim) break;  // the same for the whole workgroup
                __syncthreads();  // the previous tile's reads
                for (int x = tid; x < kLatF32Tile * (DK / 4); x += 256) {
                    const int r = x / (DK / 4), d = 4 * (x - r * (DK / 4));
                    const int key = key0 + r;
                    f32x4_t v = f32x4_t{0.f, 0.f, 0.f, 0.f};
                    if (key < lim) {  // hidden keys are zero
                        int64_t blk = b, tok = key;
                        if (p.kv.page_size > 0) {
                            const int idx = key / p.kv.page_size;
                            int page = p.kv.block_table[(int64_t)b * p.kv.max_blocks + idx];
                            page = page < 0 ? 0 : (page >= p.kv.num_blocks ? p.kv.num_blocks - 1 : page);
                            blk = page;
                            tok = key - idx * p.kv.page_size;
                        }
                        const int64_t off = blk * p.kv.s_blk + tok * p.kv.s_tok + d;
                        if (p.kv.elem == 4) {
                            const float *src = reinterpret_cast<const float *>(p.kv.k) + off;
                            if (a.quads) v = *reinterpret_cast<const f32x4_t *>(src);
                            else v = f32x4_t{src[0], src[1], src[2], src[3]};
                        } else if (p.kv.elem == 2) {
                            const uint16_t *src = reinterpret_cast<const uint16_t *>(p.kv.k) + off;
                            uint16_t e[4];
                            if (a.quads) *reinterpret_cast<uint2 *>(e) = *reinterpret_cast<const uint2 *>(src);
                            else for (int y = 0; y < 4; ++y) e[y] = src[y];
                            for (int y = 0; y < 4; ++y) v[y] = bf16_to_f32(e[y]);
                        } else {
                            const uint8_t *src = p.kv.k + off;
                            uint8_t e[4];
                            if (a.quads) *reinterpret_cast<uint32_t *>(e) = *reinterpret_cast<const uint32_t *>(src);
                            else for (int y = 0; y < 4; ++y) e[y] = src[y];
                            for (int y = 0; y < 4; ++y) v[y] = e4m3fn_f32(e[y]) * kscale;
                        }
                    }
                    *reinterpret_cast<f32x4_t *>(&ks[r][d]) = v;
                }
                __syncthreads();
                // partial scores of this wave's dimensions: S^T[key][row]
#pragma unroll
                for (int kb = 0; kb < 2; ++kb) {
                    f32x4_t s = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int x = 0; x < QS; ++x) {
                        const f32x4_t kf = *reinterpret_cast<const f32x4_t *>(&ks[16 * kb + n16][wave * (DK / 4) + 16 * x + 4 * j]);
#pragma unroll
                        for (int e = 0; e < 4; ++e) s = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[e], q[x][e], s, 0, 0, 0);
                    }
#pragma unroll
                    for (int e = 0; e < 4; ++e) sp[wave][16 * kb + 4 * j + e][n16] = s[e];
                }
                __syncthreads();
                float pv[8], mx = m;
#pragma unroll
                for (int x = 0; x < 8; ++x) {
                    const int r = 4 * x + j;
                    const float s = (sp[0][r][n16] + sp[1][r][n16]) + (sp[2][r][n16] + sp[3][r][n16]);
                    pv[x] = key0 + r < lim ? s : -INFINITY;
                    mx = fmaxf(mx, pv[x]);
                }
                mx = fmaxf(mx, __shfl_xor(mx, 16));
                mx = fmaxf(mx, __shfl_xor(mx, 32));
                const float ref = mx == -INFINITY ? 0.f : mx;
                const float alpha = m == -INFINITY ? 0.f : exp2f((m - ref) * p.sm_scale_log2);
                m = mx;
                float sum = 0.f;
#pragma unroll
                for (int x = 0; x < 8; ++x) {
                    pv[x] = exp2f((pv[x] - ref) * p.sm_scale_log2);
                    sum += pv[x];
                }
                sum += __shfl_xor(sum, 16);
                sum += __shfl_xor(sum, 32);
                l = l * alpha + sum;
#pragma unroll
                for (int x = 0; x < NB; ++x) {
                    acc[x] *= alpha;
#pragma unroll
                    for (int s = 0; s < 8; ++s)
                        acc[x] = __builtin_amdgcn_mfma_f32_16x16x4f32(ks[4 * s + j][wave * (DC / 4) + 16 * x + n16], pv[s], acc[x], 0, 0, 0);
                }
            }
            const bool whole = tile == 0 && t1 == tiles;
            const float inv = l == 0.f ? 0.f : 1.f / l;
            const float lse2 = l == 0.f ? -INFINITY : m * p.sm_scale_log2 + log2f(l);
            if (whole) {
                if (row_ok) {
#pragma unroll
                    for (int x = 0; x < NB; ++x) {
                        const int64_t at = qrow * DC + wave * (DC / 4) + 16 * x + 4 * j;
                        uint8_t *o = static_cast<uint8_t *>(p.out) + at * (p.out_dtype == SPIRE_F32 ? 4 : 2);
                        float v[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e) v[e] = l == 0.f ? 0.f : acc[x][e] * inv;  // infinite values behind no weight
                        if (p.out_dtype == SPIRE_F32) store_quad<4>(o, v, 1.f);
                        else store_quad<2>(o, v, 1.f);
                    }
                    if (wave == 0 && j == 0 && p.lse != nullptr) p.lse[qrow] = lse2 * 0.69314718055994531f;
                }
            } else {
                const int64_t slot = 2 * (int64_t)g + (pos == begin ? 0 : 1);
                const int64_t row = slot * pl.rows + 16 * u + n16;
#pragma unroll
                for (int x = 0; x < NB; ++x)
                    *reinterpret_cast<f32x4_t *>(pl.part_o + row * DC + wave * (DC / 4) + 16 * x + 4 * j) = acc[x] * inv;
                if (wave == 0 && j == 0) pl.part_lse[row] = lse2;
            }
        }
        pos += te - tile;
        ++seg;
        tile = 0;
    }
}

// ---- merge of the partials of the sequences that several groups share --------------
// out = sum_i w_i o_i / sum_i w_i with w_i = 2^(lse_i - max).  A workgroup takes one
// sequence (or, with more sequences than groups, the one that group g is the first
// to start inside of).  What bounds it is the partials, written and read once: 100
// MB for 128 sequences of 128 rows of 512 on 256 groups (26 us, 3.8 TB/s).
struct Split {
    int b, m;            // sequence, partials; m = 0: nothing to merge
    int64_t start, wlo, T, workers;
    bool sparse, tail0;  // a position per worker, some workers without; wlo's last segment, not its first
    __device__ __forceinline__ int64_t slot(int x) const {
        return sparse ? 2 * worker_of(start + x, T, workers) : 2 * (wlo + x) + (x == 0 && tail0 ? 1 : 0);
    }
};

__device__ __forceinline__ Split split_of(const Latent &a, int block, bool per_group) {
    const Plan &pl = a.pl;
    Split s;
    s.m = 0;
    int tile0 = 1;
    s.b = block;
    if (per_group) {
        s.b = pl.wstart[2 * block];
        tile0 = pl.wstart[2 * block + 1];
        if (s.b < 0) return s;
    }
    const int span = pl.prefix[s.b + 1] - pl.prefix[s.b], tiles = span - pl.seg_cost;
    if (per_group && (tile0 == 0 || tile0 >= tiles)) return s;
    s.T = pl.prefix[a.p.B];
    s.start = pl.prefix[s.b];
    s.workers = pl.workers;
    s.wlo = worker_of(s.start, s.T, s.workers);
    const int64_t whi = worker_of(s.start + tiles - 1, s.T, s.workers);
    if (s.wlo == whi) return s;
    if (per_group && worker_begin(block, s.T, s.workers) != worker_begin(s.wlo + 1, s.T, s.workers)) return s;
    s.sparse = s.T < s.workers;
    s.m = s.sparse ? tiles : (int)(whi - s.wlo + 1);
    s.tail0 = !s.sparse && worker_begin(s.wlo, s.T, s.workers) < s.start;
    return s;
}

// The query row of partial row `row`, or -1.
__device__ __forceinline__ int64_t query_row(const Latent &a, int b, int row) {
    const int rb = row >> 4, i = rb / a.hb, h = 16 * (rb - i * a.hb) + (row & 15);
    return i > a.p.k || h >= a.p.Hq ? -1 : ((int64_t)b * (a.p.k + 1) + i) * a.p.Hq + h;
}

// M: maximum of the log-sum-exps; L: sum of the weights (0: no visible key, NaN: a NaN partial).
template <int DC>
__device__ __forceinline__ void write_row(const Latent &a, int64_t qrow, int d, f32x4_t acc, float M, float L) {
    const Problem &p = a.p;
    const float inv = L == 0.f ? 0.f : 1.f / L;
    float v[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = L == 0.f ? 0.f : acc[e] * inv;
    if (p.out_dtype == SPIRE_F32) store_quad<4>(static_cast<uint8_t *>(p.out) + (qrow * DC + d) * 4, v, 1.f);
    else store_quad<2>(static_cast<uint8_t *>(p.out) + (qrow * DC + d) * 2, v, 1.f);
    if (d == 0 && p.lse != nullptr) p.lse[qrow] = L == 0.f ? -INFINITY : (M + log2f(L)) * 0.69314718055994531f;
}

// Few partials a sequence: DC / 4 threads a row walk them, `rows` rows a workgroup.
template <int DC>
__global__ __launch_bounds__(256) void latent_combine_kernel(Latent a, int per_group, int rows) {
    constexpr int TPR = DC / 4, AT = 256 / TPR;  // threads a row, rows at a time
    const Plan &pl = a.pl;
    const Split s = split_of(a, blockIdx.x, per_group != 0);
    if (s.m == 0) return;
    const int d = 4 * (threadIdx.x % TPR);
    for (int row = blockIdx.y * rows + threadIdx.x / TPR; row < (int)(blockIdx.y + 1) * rows; row += AT) {
        const int64_t qrow = query_row(a, s.b, row);
        if (qrow < 0) continue;
        // M: the largest log-sum-exp so far (-inf: none); sums are kept relative to it
        float M = -INFINITY, L = 0.f;
        f32x4_t acc = f32x4_t{0.f, 0.f, 0.f, 0.f};
        for (int x0 = 0; x0 < s.m; x0 += 4) {
            float lp[4];
            f32x4_t o[4];
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                lp[x] = -INFINITY;
                if (x0 + x < s.m) {
                    const int64_t at = s.slot(x0 + x) * pl.rows + row;
                    lp[x] = pl.part_lse[at];
                    o[x] = *reinterpret_cast<const f32x4_t *>(pl.part_o + at * DC + d);
                }
            }
            float top = M;
#pragma unroll
            for (int x = 0; x < 4; ++x) top = fmaxf(top, lp[x]);
            const float ref = top == -INFINITY ? 0.f : top, keep = M == -INFINITY ? 0.f : exp2f(M - ref);
            M = top;
            L *= keep;
            acc *= keep;
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const float w = lp[x] == -INFINITY ? 0.f : exp2f(lp[x] - ref);  // NaN: a NaN row
                L += w;
                if (x0 + x < s.m) acc += w * o[x];  // 0 * NaN too: an infinite latent behind no weight
            }
        }
        write_row<DC>(a, qrow, d, acc, M, L);
    }
}

// Many partials a sequence (few sequences on all groups): a workgroup takes 64
// dimensions of a row, 16 threads of 4 dimensions times 16 that share the partials.
template <int DC>
__global__ __launch_bounds__(256) void latent_combine_wide_kernel(Latent a) {
    __shared__ float w[kCombineMaxWorkers];
    __shared__ f32x4_t red[256];
    __shared__ float stat[8];
    const Plan &pl = a.pl;
    const Split s = split_of(a, blockIdx.x, false);
    const int row = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    if (s.m == 0) return;
    const int64_t qrow = query_row(a, s.b, row);
    if (qrow < 0) return;
    const int col = tid & 15, pg = tid >> 4, d = 64 * blockIdx.z + 4 * col;
    auto part = [&](int x) {
        return *reinterpret_cast<const f32x4_t *>(pl.part_o + (s.slot(x) * pl.rows + row) * DC + d);
    };
    constexpr int U = 4;
    f32x4_t o[U];
#pragma unroll
    for (int x = 0; x < U; ++x) o[x] = part(pg + 16 * x < s.m ? pg + 16 * x : 0);
    float M = -INFINITY;
    bool nan = false;
    for (int x = tid; x < s.m; x += 256) {
        const float v = pl.part_lse[s.slot(x) * pl.rows + row];
        w[x] = v;
        nan |= v != v;
        M = fmaxf(M, v);
    }
#pragma unroll
    for (int o2 = 32; o2 >= 1; o2 >>= 1) M = fmaxf(M, __shfl_xor(M, o2));
    nan = __any(nan);
    if (lane == 0) stat[wave] = nan ? __builtin_nanf("") : M;
    __syncthreads();
    M = -INFINITY;
    nan = false;
#pragma unroll
    for (int x = 0; x < 4; ++x) {
        nan |= stat[x] != stat[x];
        M = fmaxf(M, stat[x]);
    }
    const float ref = M == -INFINITY ? 0.f : M;
    f32x4_t acc = f32x4_t{0.f, 0.f, 0.f, 0.f};
    float L = 0.f;
    for (int x0 = pg; x0 < s.m; x0 += 16 * U) {
#pragma unroll
        for (int x = 0; x < U; ++x)
            if (x0 + 16 * x < s.m) {
                const float v = w[x0 + 16 * x], wx = v == -INFINITY ? 0.f : exp2f(v - ref);
                L += wx;
                acc += wx * o[x];  // 0 * NaN too: an infinite latent behind no weight
            }
#pragma unroll
        for (int x = 0; x < U; ++x)
            if (x0 + 16 * (U + x) < s.m) o[x] = part(x0 + 16 * (U + x));
    }
    red[tid] = acc;
    __syncthreads();
    // the first 16 threads: sums over the partials' threads, in a fixed order
    if (pg == 0) {
#pragma unroll
        for (int x = 1; x < 16; ++x) acc += red[16 * x + col];
    }
    __syncthreads();
    red[tid][0] = L;
    __syncthreads();
    if (pg != 0) return;
    L = 0.f;
#pragma unroll
    for (int x = 0; x < 16; ++x) L += red[16 * x + col][0];
    if (nan) L = __builtin_nanf("");
    write_row<DC>(a, qrow, d, acc, M, L);
}

hipError_t launch_latent_f32(const Latent &a, hipStream_t st) {
    const dim3 grid((unsigned)(a.pl.workers * a.units)), block(256);
    if (a.p.D == 512) hipLaunchKernelGGL(latent_f32_kernel<512>, grid, block, 0, st, a);
    else hipLaunchKernelGGL(latent_f32_kernel<256>, grid, block, 0, st, a);
    return hipGetLastError();
}

// From 8 groups a sequence on, the partials are shared by threads (1 sequence of 65536
// keys, 16 rows, 256 partials: 10 us; one thread after the other 71).
hipError_t launch_latent_combine(const Latent &a, hipStream_t st) {
    if (a.pl.workers > kCombineMaxWorkers) return hipErrorInvalidValue;
    const bool big = a.p.D == 512;
    if ((int64_t)a.p.B * 8 <= a.pl.workers) {
        const dim3 grid((unsigned)a.p.B, (unsigned)a.pl.rows, (unsigned)(a.p.D / 64)), block(256);
        if (big) hipLaunchKernelGGL(latent_combine_wide_kernel<512>, grid, block, 0, st, a);
        else hipLaunchKernelGGL(latent_combine_wide_kernel<256>, grid, block, 0, st, a);
        return hipGetLastError();
    }
    // Rows a workgroup: as few as fill the device (64 sequences of 16 rows: 8 rows 17.5 us, 2
    // rows 9.0; of 80 rows: 22.2 and 17.7), 8 where there are many (128 sequences of 128
    // rows: 29.6 us, 36.4 with 2), since each finds its sequence's partials first.
    const int per_group = a.p.B > a.pl.workers, seqs = per_group ? a.pl.workers : a.p.B;
    const int64_t total = (int64_t)seqs * a.pl.rows;
    const int rows = total >= 16384 ? 8 : (total >= 8192 || !big ? 4 : 2);
    const dim3 grid((unsigned)seqs, (unsigned)((a.pl.rows + rows - 1) / rows)), block(256);
    if (big) hipLaunchKernelGGL(latent_combine_kernel<512>, grid, block, 0, st, a, per_group, rows);
    else hipLaunchKernelGGL(latent_combine_kernel<256>, grid, block, 0, st, a, per_group, rows);
    return hipGetLastError();
}

}  // namespace spire
