// rope_append.hip -- a layer's projections on their way into the cache (gfx950).
//
//   qkv_append     per-head norm and position rotation of queries and keys,
//                  queries to their buffer, keys and values to their slots;
//   latent_append  norm of the latent, rotation of the shared key part and of the
//                  queries' position parts, [latent, key part] to its slot.
//
// y = x / sqrt(mean(x^2) + eps) * w, then pair i turns by positions[axis_i] * f_i.
// The angle is a product in fp64, reduced to a fraction of a turn there (a far
// position times a frequency has more bits than fp32 holds: at position 10^6 an
// fp32 angle is off by 0.03), its sine and cosine are fp32.
#include "convert.h"

namespace spire {

// cos and sin of p * f
__device__ __forceinline__ void turn(int p, float f, float &c, float &s) {
    const double t = (double)p * (double)f * 0.15915494309189533577;  // in turns
    sincospif(2.f * (float)(t - rint(t)), &s, &c);
}

struct RopeDev {
    const int32_t *positions;
    const float *inv_freq;
    const int32_t *axis;
    int32_t axes, rot, interleaved, N;
};

__device__ __forceinline__ void angle(const RopeDev &r, int t, int i, float &c, float &s) {
    int ax = r.axis != nullptr ? r.axis[i] : 0;
    ax = ax < 0 ? 0 : (ax >= r.axes ? r.axes - 1 : ax);
    turn(r.positions[(int64_t)ax * r.N + t], r.inv_freq[i], c, s);
}

// One row of D elements: norm (weight not null), rotation of the first `rot`
// elements, stored as ES-byte elements.  One wave, any D and alignment.
__device__ __forceinline__ void row_any(const void *src, int dtype, int64_t at, int D, const float *w, float eps,
                                        const RopeDev &rope, int rot, int t, uint8_t *dst, int es, float scale,
                                        int lane) {
    float r = 1.f;
    if (w != nullptr) {
        float ss = 0.f;
        for (int d = lane; d < D; d += 64) {
            const float x = load_new(src, dtype, at + d);
            ss = fmaf(x, x, ss);
        }
#pragma unroll
        for (int o = 32; o >= 1; o >>= 1) ss += __shfl_xor(ss, o);
        r = 1.f / sqrtf(ss / (float)D + eps);
    }
    auto value = [&](int d) {
        const float x = load_new(src, dtype, at + d);
        return w != nullptr ? x * r * w[d] : x;
    };
    const int half = rot >> 1;
    for (int i = lane; i < half; i += 64) {
        const int da = rope.interleaved ? 2 * i : i, db = rope.interleaved ? 2 * i + 1 : i + half;
        float c, s;
        angle(rope, t, i, c, s);
        const float a = value(da), b = value(db);
        store_elem(dst, es, da, a * c - b * s, scale);
        store_elem(dst, es, db, b * c + a * s, scale);
    }
    for (int d = rot + lane; d < D; d += 64) store_elem(dst, es, d, value(d), scale);
}

struct QkvArgs {
    const void *q, *k, *v;
    int64_t q_stride, k_stride, v_stride;
    const float *qw, *kw;
    RopeDev rope;
    KvDev kv;
    const int64_t *slots;
    void *q_out;
    float eps;
    int32_t in_dtype, out_es, N, Hq, Hkv, D;
    int64_t rpb;  // rows per block of the view
};

// Element offset of slot s's row (head 0) in a view of rpb rows per block; -1: no storage.
__device__ __forceinline__ int64_t slot_row(int64_t s, int64_t rpb, int64_t blocks, int64_t s_blk, int64_t s_tok) {
    if (s < 0 || s >= blocks * rpb) return -1;
    int64_t blk, row;
    if (s <= UINT32_MAX) {  // 64-bit division is a long software sequence
        const uint32_t q = (uint32_t)s / (uint32_t)rpb;
        blk = q;
        row = (uint32_t)s - q * (uint32_t)rpb;
    } else {
        blk = s / rpb;
        row = s - blk * rpb;
    }
    return blk * s_blk + row * s_tok;
}

__global__ __launch_bounds__(256) void qkv_append_kernel(QkvArgs a) {
    const int lane = threadIdx.x & 63;
    const int heads = a.Hq + 2 * a.Hkv;
    const int64_t rows = (int64_t)a.N * heads;
    for (int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); row < rows; row += (int64_t)gridDim.x * 4) {
        const int t = (int)(row / heads), h = (int)(row - (int64_t)t * heads);
        if (h < a.Hq) {
            row_any(a.q, a.in_dtype, t * a.q_stride + (int64_t)h * a.D, a.D, a.qw, a.eps, a.rope, a.rope.rot, t,
                    static_cast<uint8_t *>(a.q_out) + ((int64_t)t * a.Hq + h) * a.D * a.out_es, a.out_es, 1.f, lane);
            continue;
        }
        const bool val = h >= a.Hq + a.Hkv;
        const int g = h - a.Hq - (val ? a.Hkv : 0);
        const int64_t at = slot_row(a.slots[t], a.rpb, a.kv.num_blocks, a.kv.s_blk, a.kv.s_tok);
        if (at < 0) continue;
        const int es = a.kv.elem;
        uint8_t *dst = const_cast<uint8_t *>(val ? a.kv.v : a.kv.k) + (at + g * a.kv.s_head) * es;
        const float scale = es == 1 ? (val ? a.kv.v_scale : a.kv.k_scale)[g] : 1.f;
        row_any(val ? a.v : a.k, a.in_dtype, t * (val ? a.v_stride : a.k_stride) + (int64_t)g * a.D, a.D,
                val ? nullptr : a.kw, a.eps, a.rope, val ? 0 : a.rope.rot, t, dst, es, scale, lane);
    }
}

struct LatentAppendArgs {
    const void *c, *k, *q;
    int64_t c_stride, k_stride, q_stride, q_head_stride;
    const float *w;
    RopeDev rope;
    KvDev kv;  // k, k_scale, s_blk, s_tok, elem, num_blocks
    const int64_t *slots;
    void *q_out;
    float eps;
    int32_t in_dtype, out_es, N, Hq, Dc, Dr;
    int64_t rpb;
};

__global__ __launch_bounds__(256) void latent_append_kernel(LatentAppendArgs a) {
    const int lane = threadIdx.x & 63;
    const int heads = a.Hq + 2;  // the latent, the key part, the queries' parts
    const int64_t rows = (int64_t)a.N * heads;
    for (int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); row < rows; row += (int64_t)gridDim.x * 4) {
        const int t = (int)(row / heads), h = (int)(row - (int64_t)t * heads) - 2;
        if (h >= 0) {
            uint8_t *dst = static_cast<uint8_t *>(a.q_out) +
                           (((int64_t)t * a.Hq + h) * (a.Dc + a.Dr) + a.Dc) * a.out_es;
            row_any(a.q, a.in_dtype, t * a.q_stride + h * a.q_head_stride, a.Dr, nullptr, 0.f, a.rope, a.rope.rot, t,
                    dst, a.out_es, 1.f, lane);
            continue;
        }
        const int64_t at = slot_row(a.slots[t], a.rpb, a.kv.num_blocks, a.kv.s_blk, a.kv.s_tok);
        if (at < 0) continue;
        const int es = a.kv.elem;
        uint8_t *dst = const_cast<uint8_t *>(a.kv.k) + at * es;
        const float scale = es == 1 ? a.kv.k_scale[0] : 1.f;
        if (h == -2)
            row_any(a.c, a.in_dtype, t * a.c_stride, a.Dc, a.w, a.eps, a.rope, 0, t, dst, es, scale, lane);
        else
            row_any(a.k, a.in_dtype, t * a.k_stride, a.Dr, nullptr, 0.f, a.rope, a.rope.rot, t,
                    dst + (int64_t)a.Dc * es, es, scale, lane);
    }
}

static RopeDev rope_dev(const spire_rope *r, int N) {
    if (r == nullptr || r->rot_dim == 0) return RopeDev{nullptr, nullptr, nullptr, 1, 0, 0, N};
    return RopeDev{r->positions, r->inv_freq, r->axis, r->axes, r->rot_dim, r->interleaved, N};
}

static unsigned rows_grid(int64_t rows) {
    const int64_t g = (rows + 3) / 4;
    return (unsigned)(g > 65536 ? 65536 : g);
}

hipError_t launch_qkv_append(const QkvAppend &x, hipStream_t st) {
    QkvArgs a{x.q, x.k, x.v, x.q_stride, x.k_stride, x.v_stride, x.q_weight, x.k_weight, rope_dev(x.rope, x.N),
              x.kv, x.slots, x.q_out, x.eps, x.in_dtype, x.out_dtype == SPIRE_F32 ? 4 : 2, x.N, x.Hq, x.Hkv, x.D,
              x.kv.page_size > 0 ? x.kv.page_size : x.kv.capacity};
    const int64_t rows = (int64_t)x.N * (x.Hq + 2 * x.Hkv);
    hipLaunchKernelGGL(qkv_append_kernel, dim3(rows_grid(rows)), dim3(256), 0, st, a);
    return hipGetLastError();
}

hipError_t launch_latent_append(const LatentAppend &x, hipStream_t st) {
    LatentAppendArgs a{x.c, x.k, x.q, x.c_stride, x.k_stride, x.q_stride, x.q_head_stride, x.weight,
                       rope_dev(x.rope, x.N), x.kv, x.slots, x.q_out, x.eps, x.in_dtype,
                       x.out_dtype == SPIRE_F32 ? 4 : 2, x.N, x.Hq, x.Dc, x.Dr,
                       x.kv.page_size > 0 ? x.kv.page_size : x.kv.capacity};
    const int64_t rows = (int64_t)x.N * (x.Hq + 2);
    hipLaunchKernelGGL(latent_append_kernel, dim3(rows_grid(rows)), dim3(256), 0, st, a);
    return hipGetLastError();
}

}  // namespace spire
