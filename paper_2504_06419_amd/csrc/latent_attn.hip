// latent_attn.hip -- attention over a latent cache in fp32, and the merge of split
// sequences (gfx950).
//
// Any storage type (converted to fp32 on the way into LDS), alignment, page size
// and stride.  One workgroup of 4 waves per (group, 16-row block).  Per tile of 32
// keys: the rows are staged as fp32; wave w forms the scores' partial sums over
// its quarter of the Dc + 64 dimensions (v_mfma_f32_16x16x4_f32, S^T = K Q^T); the
// quarters meet in LDS and every wave takes the online softmax of all 32 keys;
// then wave w accumulates its quarter of the latent, O^T += C^T P^T.
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
    if (g >= pl.workers) return;
    const int64_t T = (int64_t)uload(pl.prefix, p.B);
    int64_t pos = worker_begin(g, T, pl.workers);
    const int64_t end = worker_begin(g + 1, T, pl.workers);
    if (pos >= end) return;
    int seg = uload(pl.wstart, 2 * g), tile = uload(pl.wstart, 2 * g + 1);
    const int64_t begin = pos;
    const int i = u / a.hb, h = 16 * (u - i * a.hb) + n16;  // units are single blocks here
    const bool row_ok = h < p.Hq;
    const float kscale = p.kv.elem == 1 ? p.kv.k_scale[0] : 1.f;

    while (pos < end) {
        const int b = seg;
        const int span = uload(pl.prefix, b + 1) - uload(pl.prefix, b);
        const int tiles = span - pl.seg_cost;
        const int64_t left = end - pos;
        const int te = left < (int64_t)(span - tile) ? tile + (int)left : span;
        if (tile < tiles) {
            const int t1 = te < tiles ? te : tiles;
            const int n = uload(pl.nkeys, b);
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
                        const float v[4] = {acc[x][0] * inv, acc[x][1] * inv, acc[x][2] * inv, acc[x][3] * inv};
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

// Merge of the partials of the sequences that several groups share.  One
// workgroup per (group, row): the first group to start inside a sequence's tiles
// merges it.  out = sum_i w_i o_i / sum_i w_i with w_i = 2^(lse_i - max).
template <int DC>
__global__ __launch_bounds__(256) void latent_combine_kernel(Latent a) {
    constexpr int TPR = DC / 4, PG = 256 / TPR;  // threads a row, partials side by side
    __shared__ float w[kCombineMaxWorkers];
    __shared__ f32x4_t red[256];
    const Problem &p = a.p;
    const Plan &pl = a.pl;
    const int g = blockIdx.x, row = blockIdx.y, tid = threadIdx.x;
    const int rb = row >> 4, i = rb / a.hb, h = 16 * (rb - i * a.hb) + (row & 15);
    if (i > p.k || h >= p.Hq) return;
    const int b = pl.wstart[2 * g], tile0 = pl.wstart[2 * g + 1];
    if (b < 0) return;
    const int span = pl.prefix[b + 1] - pl.prefix[b], tiles = span - pl.seg_cost;
    if (tile0 == 0 || tile0 >= tiles) return;
    const int64_t T = pl.prefix[p.B], start = pl.prefix[b];
    const int64_t wlo = worker_of(start, T, pl.workers), whi = worker_of(start + tiles - 1, T, pl.workers);
    if (wlo == whi || worker_begin(g, T, pl.workers) != worker_begin(wlo + 1, T, pl.workers)) return;
    const bool sparse = T < pl.workers;  // a position per worker, some workers without
    const int m = sparse ? tiles : (int)(whi - wlo + 1);
    const bool tail0 = !sparse && worker_begin(wlo, T, pl.workers) < start;
    auto slot = [&](int x) -> int64_t {
        return sparse ? 2 * worker_of(start + x, T, pl.workers) : 2 * (wlo + x) + (x == 0 && tail0 ? 1 : 0);
    };
    float M = -INFINITY;
    bool nan = false;
    for (int x = tid; x < m; x += 256) w[x] = pl.part_lse[slot(x) * pl.rows + row];
    __syncthreads();
    for (int x = 0; x < m; ++x) {
        const float v = w[x];
        nan |= v != v;
        M = fmaxf(M, v);
    }
    const float ref = M == -INFINITY ? 0.f : M;
    __syncthreads();
    for (int x = tid; x < m; x += 256) w[x] = exp2f(w[x] - ref);
    __syncthreads();
    float L = 0.f;
    for (int x = 0; x < m; ++x) L += w[x];
    if (nan) L = __builtin_nanf("");
    const int pg = tid / TPR, d = 4 * (tid - pg * TPR);
    f32x4_t acc = f32x4_t{0.f, 0.f, 0.f, 0.f};
    for (int x = pg; x < m; x += PG) {
        const f32x4_t v = *reinterpret_cast<const f32x4_t *>(pl.part_o + (slot(x) * pl.rows + row) * DC + d);
        const float wx = w[x];
        if (wx != 0.f) acc += wx * v;
    }
    red[tid] = acc;
    __syncthreads();
    if (pg != 0) return;
#pragma unroll
    for (int x = 1; x < PG; ++x) acc += red[x * TPR + tid];
    const float inv = L == 0.f ? 0.f : 1.f / L;
    const int64_t qrow = ((int64_t)b * (p.k + 1) + i) * p.Hq + h;
    const float v[4] = {acc[0] * inv, acc[1] * inv, acc[2] * inv, acc[3] * inv};
    if (p.out_dtype == SPIRE_F32) store_quad<4>(static_cast<uint8_t *>(p.out) + (qrow * DC + d) * 4, v, 1.f);
    else store_quad<2>(static_cast<uint8_t *>(p.out) + (qrow * DC + d) * 2, v, 1.f);
    if (tid == 0 && p.lse != nullptr) p.lse[qrow] = L == 0.f ? -INFINITY : (M + log2f(L)) * 0.69314718055994531f;
}

hipError_t launch_latent_f32(const Latent &a, hipStream_t st) {
    const dim3 grid((unsigned)(a.pl.workers * a.units)), block(256);
    if (a.p.D == 512) hipLaunchKernelGGL(latent_f32_kernel<512>, grid, block, 0, st, a);
    else hipLaunchKernelGGL(latent_f32_kernel<256>, grid, block, 0, st, a);
    return hipGetLastError();
}

hipError_t launch_latent_combine(const Latent &a, hipStream_t st) {
    if (a.pl.workers > kCombineMaxWorkers) return hipErrorInvalidValue;
    const dim3 grid((unsigned)a.pl.workers, (unsigned)a.pl.rows), block(256);
    if (a.p.D == 512) hipLaunchKernelGGL(latent_combine_kernel<512>, grid, block, 0, st, a);
    else hipLaunchKernelGGL(latent_combine_kernel<256>, grid, block, 0, st, a);
    return hipGetLastError();
}

}  // namespace spire
