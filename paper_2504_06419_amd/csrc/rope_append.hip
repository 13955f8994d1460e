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

// ---- rows of 8-element items (vector paths) ---------------------------------------
//
// One workgroup takes a few tokens, every row of them.  The sines and cosines of a
// token are formed once, by the first threads, and stand in LDS for all its heads
// (fp64 products per head would cost more than the memory traffic).  A row is D / 8
// items, one per lane; item i holds two quads of elements: its 4 pairs' first and
// second halves (4 i and 4 i + rot / 2) or 4 neighbouring pairs, so a rotation stays
// in its lane.  D / 8 is a power of two up to 64: a norm's sum is a few shuffles.
// Bound by memory for prompts, by the chain position -> angle -> row for few tokens.
struct Quads {
    float a[4], b[4];
};

__device__ __forceinline__ void quad_places(int i, int rot, bool interleaved, int &oa, int &ob) {
    const bool halves = 8 * i < rot && !interleaved;
    oa = halves ? 4 * i : 8 * i;
    ob = halves ? 4 * i + (rot >> 1) : 8 * i + 4;
}

// `tab`: (cos, sin) of the token's pairs.
__device__ __forceinline__ void rotate_item(Quads &x, int i, const RopeDev &r, int rot, const float2 *tab) {
    if (8 * i >= rot) return;
    float2 t[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) t[e] = tab[4 * i + e];
    auto turn2 = [](float &u, float &v, float2 cs) {
        const float p = u * cs.x - v * cs.y, q = v * cs.x + u * cs.y;
        u = p;
        v = q;
    };
    if (r.interleaved) {
        turn2(x.a[0], x.a[1], t[0]);
        turn2(x.a[2], x.a[3], t[1]);
        turn2(x.b[0], x.b[1], t[2]);
        turn2(x.b[2], x.b[3], t[3]);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) turn2(x.a[e], x.b[e], t[e]);
    }
}

// x / sqrt(mean(x^2) + eps) * w over the `lanes` lanes (a power of two) that hold the row.
__device__ __forceinline__ void norm_item(Quads &x, const float *w, int oa, int ob, int D, int lanes, float eps) {
    float ss = 0.f;
#pragma unroll
    for (int e = 0; e < 4; ++e) ss = fmaf(x.a[e], x.a[e], fmaf(x.b[e], x.b[e], ss));
    for (int o = lanes >> 1; o >= 1; o >>= 1) ss += __shfl_xor(ss, o);
    const float r = 1.f / sqrtf(ss / (float)D + eps);
    const float4 wa = *reinterpret_cast<const float4 *>(w + oa), wb = *reinterpret_cast<const float4 *>(w + ob);
    x.a[0] *= r * wa.x; x.a[1] *= r * wa.y; x.a[2] *= r * wa.z; x.a[3] *= r * wa.w;
    x.b[0] *= r * wb.x; x.b[1] *= r * wb.y; x.b[2] *= r * wb.z; x.b[3] *= r * wb.w;
}

__device__ __forceinline__ void store_item(uint8_t *row, int es, const Quads &x, int oa, int ob, float scale) {
    if (es == 4) {
        store_quad<4>(row + 4 * oa, x.a, 1.f);
        store_quad<4>(row + 4 * ob, x.b, 1.f);
    } else if (es == 2) {
        store_quad<2>(row + 2 * oa, x.a, 1.f);
        store_quad<2>(row + 2 * ob, x.b, 1.f);
    } else {
        store_quad<1>(row + oa, x.a, scale);
        store_quad<1>(row + ob, x.b, scale);
    }
}

constexpr int kVecThreads = 256;
constexpr int kVecPairs = 512;  // (cos, sin) pairs a workgroup holds

__device__ __forceinline__ void angles_to_lds(const RopeDev &rope, int t0, int tokens, float2 *tab) {
    const int half = rope.rot >> 1;
    for (int x = threadIdx.x; x < tokens * half; x += kVecThreads) {
        const int t = x / half;
        float c, s;
        angle(rope, t0 + t, x - t * half, c, s);
        tab[x] = make_float2(c, s);
    }
}

__global__ __launch_bounds__(kVecThreads) void qkv_append_vec_kernel(QkvArgs a, int per, int shift) {
    __shared__ float2 tab[kVecPairs];
    const int t0 = blockIdx.x * per, tokens = a.N - t0 < per ? a.N - t0 : per;
    const int heads = a.Hq + 2 * a.Hkv, items = tokens * heads << shift;  // D / 8 = 1 << shift items a row
    const int i = threadIdx.x & ((1 << shift) - 1);
    struct Where {
        const void *src;
        int64_t at;
        int t, h, rot, oa, ob;
    };
    auto where = [&](int x) {
        Where w;
        const int row = x >> shift;
        w.t = tokens == 1 ? 0 : row / heads;
        w.h = row - w.t * heads;
        const int64_t tok = t0 + w.t;
        const bool q = w.h < a.Hq, val = w.h >= a.Hq + a.Hkv;
        w.src = q ? a.q : (val ? a.v : a.k);
        w.at = tok * (q ? a.q_stride : (val ? a.v_stride : a.k_stride)) +
               (int64_t)(w.h - (q ? 0 : (val ? a.Hq + a.Hkv : a.Hq))) * a.D;
        w.rot = val ? 0 : a.rope.rot;
        quad_places(i, w.rot, a.rope.interleaved != 0, w.oa, w.ob);
        return w;
    };
    auto load = [&](const Where &w) {
        Quads x;
        load_quad(w.src, a.in_dtype, w.at + w.oa, x.a);
        load_quad(w.src, a.in_dtype, w.at + w.ob, x.b);
        return x;
    };
    Where w;
    Quads x;
    if ((int)threadIdx.x < items) {  // on its way while the angles are formed
        w = where(threadIdx.x);
        x = load(w);
    }
    angles_to_lds(a.rope, t0, tokens, tab);
    __syncthreads();
    for (int y = threadIdx.x; y < items; y += kVecThreads) {
        Where wn;
        Quads xn;
        if (y + kVecThreads < items) {
            wn = where(y + kVecThreads);
            xn = load(wn);
        }
        const bool q = w.h < a.Hq, val = w.h >= a.Hq + a.Hkv;
        const float *weight = q ? a.qw : (val ? nullptr : a.kw);
        if (weight != nullptr) norm_item(x, weight, w.oa, w.ob, a.D, 1 << shift, a.eps);
        rotate_item(x, i, a.rope, w.rot, tab + w.t * (a.rope.rot >> 1));
        if (q) {
            store_item(static_cast<uint8_t *>(a.q_out) + ((int64_t)(t0 + w.t) * a.Hq + w.h) * a.D * a.out_es, a.out_es, x,
                       w.oa, w.ob, 1.f);
        } else {
            const int g = w.h - a.Hq - (val ? a.Hkv : 0), es = a.kv.elem;
            const int64_t at = slot_row(a.slots[t0 + w.t], a.rpb, a.kv.num_blocks, a.kv.s_blk, a.kv.s_tok);
            if (at >= 0)
                store_item(const_cast<uint8_t *>(val ? a.kv.v : a.kv.k) + (at + g * a.kv.s_head) * es, es, x, w.oa, w.ob,
                           es == 1 ? (val ? a.kv.v_scale : a.kv.k_scale)[g] : 1.f);
        }
        w = wn;
        x = xn;
    }
}

// The tokens' latents come first, 1 << shift items each, so that none crosses a
// wave; then rows of 1 << rshift items: a token's key part and its queries' parts.
__global__ __launch_bounds__(kVecThreads) void latent_append_vec_kernel(LatentAppendArgs a, int per, int shift, int rshift) {
    __shared__ float2 tab[kVecPairs];
    const int t0 = blockIdx.x * per, tokens = a.N - t0 < per ? a.N - t0 : per;
    const int lat = tokens << shift, items = lat + (tokens * (1 + a.Hq) << rshift);
    struct Where {
        const void *src;
        int64_t at;
        int t, h, i, rot, oa, ob;  // h: -2 the latent, -1 the key part
    };
    auto where = [&](int x) {
        Where w;
        const bool c = x < lat;
        const int row = (x - lat) >> rshift;
        w.t = c ? x >> shift : (tokens == 1 ? 0 : row / (1 + a.Hq));
        w.h = c ? -2 : row - w.t * (1 + a.Hq) - 1;
        w.i = c ? x & ((1 << shift) - 1) : (x - lat) & ((1 << rshift) - 1);
        const int64_t tok = t0 + w.t;
        w.src = c ? a.c : (w.h < 0 ? a.k : a.q);
        w.at = c ? tok * a.c_stride : (w.h < 0 ? tok * a.k_stride : tok * a.q_stride + w.h * a.q_head_stride);
        w.rot = c ? 0 : a.rope.rot;
        quad_places(w.i, w.rot, a.rope.interleaved != 0, w.oa, w.ob);
        return w;
    };
    auto load = [&](const Where &w) {
        Quads x;
        load_quad(w.src, a.in_dtype, w.at + w.oa, x.a);
        load_quad(w.src, a.in_dtype, w.at + w.ob, x.b);
        return x;
    };
    Where w;
    Quads x;
    if ((int)threadIdx.x < items) {
        w = where(threadIdx.x);
        x = load(w);
    }
    angles_to_lds(a.rope, t0, tokens, tab);
    __syncthreads();
    for (int y = threadIdx.x; y < items; y += kVecThreads) {
        Where wn;
        Quads xn;
        if (y + kVecThreads < items) {
            wn = where(y + kVecThreads);
            xn = load(wn);
        }
        if (a.w != nullptr && w.h == -2) norm_item(x, a.w, w.oa, w.ob, a.Dc, 1 << shift, a.eps);
        rotate_item(x, w.i, a.rope, w.rot, tab + w.t * (a.rope.rot >> 1));
        if (w.h >= 0) {
            store_item(static_cast<uint8_t *>(a.q_out) +
                           (((int64_t)(t0 + w.t) * a.Hq + w.h) * (a.Dc + a.Dr) + a.Dc) * a.out_es,
                       a.out_es, x, w.oa, w.ob, 1.f);
        } else {
            const int es = a.kv.elem;
            const int64_t at = slot_row(a.slots[t0 + w.t], a.rpb, a.kv.num_blocks, a.kv.s_blk, a.kv.s_tok);
            if (at >= 0)
                store_item(const_cast<uint8_t *>(a.kv.k) + (at + (w.h == -1 ? a.Dc : 0)) * es, es, x, w.oa, w.ob,
                           es == 1 ? a.kv.k_scale[0] : 1.f);
        }
        w = wn;
        x = xn;
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

// rows of `n` elements that are D / 8 items of a wave: log2 of the items, or -1
static int item_shift(int D) {
    if (D % 8 != 0 || D > 512) return -1;
    const int n = D / 8;
    return (n & (n - 1)) == 0 ? __builtin_ctz((unsigned)n) : -1;
}

// pointer and strides readable and writable 4 elements of `es` bytes at a time
static bool on_quads(const void *p, int es, int64_t s0 = 0, int64_t s1 = 0, int64_t s2 = 0) {
    return (uintptr_t)p % (4 * es) == 0 && s0 % 4 == 0 && s1 % 4 == 0 && s2 % 4 == 0;
}

static bool rope_on_items(const RopeDev &r, int D) { return r.rot % 8 == 0 && r.rot <= D && r.rot / 2 <= kVecPairs; }

// Tokens a workgroup: enough items for its threads, where that leaves workgroups
// for every CU twice over; and the angles' place.
static int tokens_per_group(int N, int items, int rot) {
    int per = items >= kVecThreads ? 1 : kVecThreads / items;
    if (rot > 0 && per > kVecPairs / (rot / 2)) per = kVecPairs / (rot / 2);
    if (per > (N + 511) / 512) per = (N + 511) / 512;
    return per < 1 ? 1 : per;
}

hipError_t launch_qkv_append(const QkvAppend &x, hipStream_t st) {
    QkvArgs a{x.q, x.k, x.v, x.q_stride, x.k_stride, x.v_stride, x.q_weight, x.k_weight, rope_dev(x.rope, x.N),
              x.kv, x.slots, x.q_out, x.eps, x.in_dtype, x.out_dtype == SPIRE_F32 ? 4 : 2, x.N, x.Hq, x.Hkv, x.D,
              x.kv.page_size > 0 ? x.kv.page_size : x.kv.capacity};
    const int shift = item_shift(x.D), ies = x.in_dtype == SPIRE_F32 ? 4 : 2, es = x.kv.elem;
    if (shift >= 0 && rope_on_items(a.rope, x.D) && on_quads(x.q, ies, x.q_stride) && on_quads(x.k, ies, x.k_stride) &&
        on_quads(x.v, ies, x.v_stride) && on_quads(x.q_out, a.out_es) && on_quads(x.q_weight, 4) && on_quads(x.k_weight, 4) &&
        on_quads(x.kv.k, es, x.kv.s_blk, x.kv.s_head, x.kv.s_tok) && on_quads(x.kv.v, es)) {
        const int per = tokens_per_group(x.N, (x.Hq + 2 * x.Hkv) << shift, a.rope.rot);
        hipLaunchKernelGGL(qkv_append_vec_kernel, dim3((unsigned)((x.N + (int64_t)per - 1) / per)), dim3(kVecThreads), 0, st, a, per, shift);
        return hipGetLastError();
    }
    const int64_t rows = (int64_t)x.N * (x.Hq + 2 * x.Hkv);
    hipLaunchKernelGGL(qkv_append_kernel, dim3(rows_grid(rows)), dim3(256), 0, st, a);
    return hipGetLastError();
}

hipError_t launch_latent_append(const LatentAppend &x, hipStream_t st) {
    LatentAppendArgs a{x.c, x.k, x.q, x.c_stride, x.k_stride, x.q_stride, x.q_head_stride, x.weight,
                       rope_dev(x.rope, x.N), x.kv, x.slots, x.q_out, x.eps, x.in_dtype,
                       x.out_dtype == SPIRE_F32 ? 4 : 2, x.N, x.Hq, x.Dc, x.Dr,
                       x.kv.page_size > 0 ? x.kv.page_size : x.kv.capacity};
    const int shift = item_shift(x.Dc), rshift = item_shift(x.Dr), ies = x.in_dtype == SPIRE_F32 ? 4 : 2, es = x.kv.elem;
    if (shift >= 0 && rshift >= 0 && rope_on_items(a.rope, x.Dr) && on_quads(x.c, ies, x.c_stride) &&
        on_quads(x.k, ies, x.k_stride) && on_quads(x.q, ies, x.q_stride, x.q_head_stride) && on_quads(x.q_out, a.out_es) &&
        on_quads(x.weight, 4) && on_quads(x.kv.k, es, x.kv.s_blk, x.kv.s_tok)) {
        const int per = tokens_per_group(x.N, (1 << shift) + ((1 + x.Hq) << rshift), a.rope.rot);
        hipLaunchKernelGGL(latent_append_vec_kernel, dim3((unsigned)((x.N + (int64_t)per - 1) / per)), dim3(kVecThreads), 0, st, a, per, shift, rshift);
        return hipGetLastError();
    }
    const int64_t rows = (int64_t)x.N * (x.Hq + 2);
    hipLaunchKernelGGL(latent_append_kernel, dim3(rows_grid(rows)), dim3(256), 0, st, a);
    return hipGetLastError();
}

}  // namespace spire
