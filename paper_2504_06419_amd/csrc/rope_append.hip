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
#include <type_traits>

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
// A row is D / 8 items, one per lane; item i holds two quads of elements: its 4 pairs'
// first and second halves (4 i and 4 i + rot / 2) or 4 neighbouring pairs, so that a
// rotation stays in its lane.  D / 8 is a power of two up to 64: a norm's sum is a few
// shuffles.  A wave takes some heads of one token, 512 / D of them a round.  A lane
// keeps its place i over the rounds, and with it its 4 sines and cosines (formed once
// a wave, one pair per lane, and passed through LDS) and its norm weights: with the
// angles formed per head the instructions, not the memory, set the time.  The next
// round's loads are on their way while a round is computed.
constexpr int kWaves = 4;         // of a workgroup
constexpr int kMaxPairs = 256;    // of a rotation: D <= 512

template <int ES>
struct Quads {  // as loaded: bf16 or fp32
    using V = typename std::conditional<ES == 4, uint4, uint2>::type;
    V a, b;
    __device__ __forceinline__ void load(const void *row, int oa, int ob) {
        a = *reinterpret_cast<const V *>(static_cast<const uint8_t *>(row) + oa * ES);
        b = *reinterpret_cast<const V *>(static_cast<const uint8_t *>(row) + ob * ES);
    }
    static __device__ __forceinline__ void floats(const V &v, float *x) {
        if constexpr (ES == 4) {
            x[0] = __uint_as_float(v.x); x[1] = __uint_as_float(v.y);
            x[2] = __uint_as_float(v.z); x[3] = __uint_as_float(v.w);
        } else {
            x[0] = __uint_as_float(v.x << 16); x[1] = __uint_as_float(v.x & 0xFFFF0000u);
            x[2] = __uint_as_float(v.y << 16); x[3] = __uint_as_float(v.y & 0xFFFF0000u);
        }
    }
    __device__ __forceinline__ void floats(float x[8]) const {
        floats(a, x);
        floats(b, x + 4);
    }
};

__device__ __forceinline__ void item_places(int i, int rot, bool interleaved, int &oa, int &ob) {
    const bool halves = 8 * i < rot && !interleaved;
    oa = halves ? 4 * i : 8 * i;
    ob = halves ? 4 * i + (rot >> 1) : 8 * i + 4;
}

__device__ __forceinline__ void rotate_pair(float &u, float &v, float2 cs) {
    const float p = u * cs.x - v * cs.y, q = v * cs.x + u * cs.y;
    u = p;
    v = q;
}

// `cs`: (cos, sin) of the item's 4 pairs; x: quad a, then quad b
__device__ __forceinline__ void rotate_item(float x[8], bool interleaved, const float2 cs[4]) {
    if (interleaved) {
#pragma unroll
        for (int e = 0; e < 4; ++e) rotate_pair(x[2 * e], x[2 * e + 1], cs[e]);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) rotate_pair(x[e], x[4 + e], cs[e]);
    }
}

// x / sqrt(mean(x^2) + eps) * w over the 1 << shift lanes that hold the row
__device__ __forceinline__ void norm_item(float x[8], const float w[8], int shift, float eps) {
    float ss = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) ss = fmaf(x[e], x[e], ss);
#pragma unroll
    for (int b = 5; b >= 0; --b)
        if (b < shift) ss += __shfl_xor(ss, 1 << b);
    const float r = 1.f / sqrtf(ss / (float)(8 << shift) + eps);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] *= r * w[e];
}

__device__ __forceinline__ void load_weights(const float *w, int oa, int ob, float x[8]) {
    if (w == nullptr) return;
    const float4 a = *reinterpret_cast<const float4 *>(w + oa), b = *reinterpret_cast<const float4 *>(w + ob);
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
    x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
}

// two fp32 -> bf16, nearest even (the conversion instruction)
__device__ __forceinline__ uint32_t bf16_pair(float a, float b) {
    typedef __bf16 pair __attribute__((ext_vector_type(2)));
    const pair p = {(__bf16)a, (__bf16)b};
    return __builtin_bit_cast(uint32_t, p);
}

__device__ __forceinline__ void store_item(uint8_t *row, int es, const float x[8], int oa, int ob, float scale) {
    if (es == 2) {
        *reinterpret_cast<uint2 *>(row + 2 * oa) = make_uint2(bf16_pair(x[0], x[1]), bf16_pair(x[2], x[3]));
        *reinterpret_cast<uint2 *>(row + 2 * ob) = make_uint2(bf16_pair(x[4], x[5]), bf16_pair(x[6], x[7]));
    } else if (es == 4) {
        store_quad<4>(row + 4 * oa, x, 1.f);
        store_quad<4>(row + 4 * ob, x + 4, 1.f);
    } else {
        store_quad<1>(row + oa, x, scale);
        store_quad<1>(row + ob, x + 4, scale);
    }
}

// The token's (cos, sin) of item i's pairs, through this wave's part of LDS.
__device__ __forceinline__ void item_angles(const RopeDev &rope, int t, int i, int lane, float2 *tab, float2 cs[4]) {
    const int half = rope.rot >> 1;
    for (int x = lane; x < half; x += 64) {
        float c, s;
        angle(rope, t, x, c, s);
        tab[x] = make_float2(c, s);
    }
    // one wave's LDS accesses keep their order; the compiler has to keep it too
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    if (8 * i < rope.rot)
#pragma unroll
        for (int e = 0; e < 4; ++e) cs[e] = tab[4 * i + e];
}

// By value: a choice between variables becomes one between their addresses, and those then live in scratch memory.
template <class T>
__device__ __forceinline__ T pick(bool first, T a, T b) {
    return first ? a : b;
}

// slices: waves a token; rounds: rounds a wave.
template <int ES>
__global__ __launch_bounds__(64 * kWaves) void qkv_append_vec_kernel(QkvArgs a, int slices, int rounds, int shift) {
    __shared__ float2 tab[kWaves][kMaxPairs];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int job = blockIdx.x * kWaves + wave, t = job / slices;
    if (t >= a.N) return;  // no barrier of the workgroup follows
    const int R = 64 >> shift, i = lane & ((1 << shift) - 1), es = a.kv.elem;
    const int heads = a.Hq + 2 * a.Hkv, h0 = (job - t * slices) * rounds * R;
    const int end = heads - h0 < rounds * R ? heads : h0 + rounds * R;
    const bool inter = a.rope.interleaved != 0;
    const uint8_t *qb = static_cast<const uint8_t *>(a.q) + t * a.q_stride * ES;
    const uint8_t *kb = static_cast<const uint8_t *>(a.k) + (t * a.k_stride - (int64_t)a.Hq * a.D) * ES;
    const uint8_t *vb = static_cast<const uint8_t *>(a.v) + (t * a.v_stride - (int64_t)(a.Hq + a.Hkv) * a.D) * ES;
    int oa, ob;
    item_places(i, a.rope.rot, inter, oa, ob);
    auto load = [&](int h, Quads<ES> &x) {
        if (h >= end) h = end - 1;  // loaded, not used
        const bool val = h >= a.Hq + a.Hkv;
        const uint8_t *b = pick(h < a.Hq, qb, pick(val, vb, kb));
        x.load(b + (int64_t)h * a.D * ES, val ? 8 * i : oa, val ? 8 * i + 4 : ob);
    };
    int h = h0 + (lane >> shift);
    Quads<ES> now, next;
    load(h, now);
    const int64_t slot = a.slots[t];
    float qw[8], kw[8];
    load_weights(a.qw, oa, ob, qw);
    load_weights(a.kw, oa, ob, kw);
    float2 cs[4];
    if (h0 < a.Hq + a.Hkv) item_angles(a.rope, t, i, lane, tab[wave], cs);
    const int64_t at = slot_row(slot, a.rpb, a.kv.num_blocks, a.kv.s_blk, a.kv.s_tok);
    uint8_t *const qo = static_cast<uint8_t *>(a.q_out) + (int64_t)t * a.Hq * a.D * a.out_es;
    uint8_t *const ko = const_cast<uint8_t *>(a.kv.k) + at * es, *const vo = const_cast<uint8_t *>(a.kv.v) + at * es;
    const float *const k_scale = a.kv.k_scale, *const v_scale = a.kv.v_scale;
    for (int n = 0; n < rounds; ++n, h += R) {
        if (n + 1 < rounds) load(h + R, next);
        if (h < end) {
            float x[8];
            now.floats(x);
            const bool q = h < a.Hq, val = h >= a.Hq + a.Hkv;
            if (q ? a.qw != nullptr : (!val && a.kw != nullptr)) {
                float w[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) w[e] = pick(q, qw[e], kw[e]);
                norm_item(x, w, shift, a.eps);
            }
            if (!val && 8 * i < a.rope.rot) rotate_item(x, inter, cs);
            const int g = h - a.Hq - (val ? a.Hkv : 0);
            uint8_t *to = q ? qo + (int64_t)h * a.D * a.out_es : pick(val, vo, ko) + g * a.kv.s_head * es;
            if (q || at >= 0)
                store_item(to, pick(q, a.out_es, es), x, val ? 8 * i : oa, val ? 8 * i + 4 : ob,
                           q || es != 1 ? 1.f : pick(val, v_scale, k_scale)[g]);
        }
        now = next;
    }
}

// The first `groups` workgroups take the latents, 512 / Dc tokens a wave, the others the
// key parts and the queries' parts.
template <int ES>
__global__ __launch_bounds__(64 * kWaves) void latent_append_vec_kernel(LatentAppendArgs a, int groups, int shift,
                                                                        int slices, int rounds, int rshift) {
    __shared__ float2 tab[kWaves][kMaxPairs];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int es = a.kv.elem;
    auto cache = [&](int64_t slot, int d) {
        const int64_t at = slot_row(slot, a.rpb, a.kv.num_blocks, a.kv.s_blk, a.kv.s_tok);
        return at < 0 ? nullptr : const_cast<uint8_t *>(a.kv.k) + (at + d) * es;
    };
    const float scale = es == 1 ? a.kv.k_scale[0] : 1.f;
    Quads<ES> now, next;
    float x[8];
    if ((int)blockIdx.x < groups) {
        const int i = lane & ((1 << shift) - 1);
        const int t = (blockIdx.x * kWaves + wave) * (64 >> shift) + (lane >> shift);
        if (t >= a.N) return;  // whole rows: the norm's lanes stay together
        now.load(static_cast<const uint8_t *>(a.c) + t * a.c_stride * ES, 8 * i, 8 * i + 4);
        const int64_t slot = a.slots[t];
        float w[8];
        load_weights(a.w, 8 * i, 8 * i + 4, w);
        uint8_t *to = cache(slot, 0);
        now.floats(x);
        if (a.w != nullptr) norm_item(x, w, shift, a.eps);
        if (to != nullptr) store_item(to, es, x, 8 * i, 8 * i + 4, scale);
        return;
    }
    const int job = (blockIdx.x - groups) * kWaves + wave, t = job / slices;
    if (t >= a.N) return;
    const int R = 64 >> rshift, i = lane & ((1 << rshift) - 1);
    const int h0 = (job - t * slices) * rounds * R, end = a.Hq + 1 - h0 < rounds * R ? a.Hq + 1 : h0 + rounds * R;
    const bool inter = a.rope.interleaved != 0;
    const uint8_t *kb = static_cast<const uint8_t *>(a.k) + t * a.k_stride * ES;
    const uint8_t *qb = static_cast<const uint8_t *>(a.q) + (t * a.q_stride - a.q_head_stride) * ES;
    int oa, ob;
    item_places(i, a.rope.rot, inter, oa, ob);
    auto load = [&](int h, Quads<ES> &y) {  // row 0: the key part
        if (h >= end) h = end - 1;
        y.load(h == 0 ? kb : qb + h * a.q_head_stride * ES, oa, ob);
    };
    int h = h0 + (lane >> rshift);
    load(h, now);
    const int64_t slot = a.slots[t];
    float2 cs[4];
    item_angles(a.rope, t, i, lane, tab[wave], cs);
    uint8_t *const to = cache(slot, a.Dc);
    const int64_t q_row = (int64_t)(a.Dc + a.Dr) * a.out_es;
    uint8_t *const qo = static_cast<uint8_t *>(a.q_out) + ((int64_t)t * a.Hq - 1) * q_row + (int64_t)a.Dc * a.out_es;
    for (int n = 0; n < rounds; ++n, h += R) {
        if (n + 1 < rounds) load(h + R, next);
        if (h < end) {
            now.floats(x);
            if (8 * i < a.rope.rot) rotate_item(x, inter, cs);
            if (h > 0 || to != nullptr) store_item(h > 0 ? qo + h * q_row : to, h > 0 ? a.out_es : es, x, oa, ob, scale);
        }
        now = next;
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

// at most 256 pairs: D <= 512
static bool rope_on_items(const RopeDev &r) { return r.rot % 8 == 0; }

// a wave's number is 32-bit
static bool in_int(int64_t N, int64_t heads) { return N * heads <= INT32_MAX - 65536; }

// Rounds a wave, of the `all` rounds of a token.  Several once every SIMD has 4 waves (at
// 1024 tokens, 32 + 2 x 8 heads of 128, bf16: 1 round a wave 14.0 us, 3 rounds 12.7); at
// most 6, where the angles no longer cost and shorter waves balance better (at 8192
// tokens: 12 rounds 51.7 us, 6 rounds 47.3).
static int rounds_per_wave(int64_t N, int all) {
    const int64_t n = N * all / 4096, most = n < 1 ? 1 : (n > 6 ? 6 : n), slices = (all + most - 1) / most;
    return (int)((all + slices - 1) / slices);
}

hipError_t launch_qkv_append(const QkvAppend &x, hipStream_t st) {
    QkvArgs a{x.q, x.k, x.v, x.q_stride, x.k_stride, x.v_stride, x.q_weight, x.k_weight, rope_dev(x.rope, x.N),
              x.kv, x.slots, x.q_out, x.eps, x.in_dtype, x.out_dtype == SPIRE_F32 ? 4 : 2, x.N, x.Hq, x.Hkv, x.D,
              x.kv.page_size > 0 ? x.kv.page_size : x.kv.capacity};
    const int shift = item_shift(x.D), ies = x.in_dtype == SPIRE_F32 ? 4 : 2, es = x.kv.elem;
    if (shift >= 0 && in_int(x.N, x.Hq + 2 * x.Hkv) && rope_on_items(a.rope) && on_quads(x.q, ies, x.q_stride) && on_quads(x.k, ies, x.k_stride) &&
        on_quads(x.v, ies, x.v_stride) && on_quads(x.q_out, a.out_es) && on_quads(x.q_weight, 4) && on_quads(x.k_weight, 4) &&
        on_quads(x.kv.k, es, x.kv.s_blk, x.kv.s_head, x.kv.s_tok) && on_quads(x.kv.v, es)) {
        const int R = 64 >> shift, all = (x.Hq + 2 * x.Hkv + R - 1) / R, rounds = rounds_per_wave(x.N, all);
        const int slices = (all + rounds - 1) / rounds;
        const dim3 grid((unsigned)(((int64_t)x.N * slices + kWaves - 1) / kWaves)), block(64 * kWaves);
        if (ies == 4) hipLaunchKernelGGL(qkv_append_vec_kernel<4>, grid, block, 0, st, a, slices, rounds, shift);
        else hipLaunchKernelGGL(qkv_append_vec_kernel<2>, grid, block, 0, st, a, slices, rounds, shift);
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
    if (shift >= 0 && rshift >= 0 && in_int(x.N, 1 + x.Hq) && rope_on_items(a.rope) && on_quads(x.c, ies, x.c_stride) &&
        on_quads(x.k, ies, x.k_stride) && on_quads(x.q, ies, x.q_stride, x.q_head_stride) && on_quads(x.q_out, a.out_es) &&
        on_quads(x.weight, 4) && on_quads(x.kv.k, es, x.kv.s_blk, x.kv.s_tok)) {
        const int R = 64 >> rshift, all = (1 + x.Hq + R - 1) / R, rounds = rounds_per_wave(x.N, all);
        const int slices = (all + rounds - 1) / rounds, per = kWaves * (64 >> shift);
        const int groups = (int)(((int64_t)x.N + per - 1) / per);
        const dim3 grid((unsigned)(groups + ((int64_t)x.N * slices + kWaves - 1) / kWaves)), block(64 * kWaves);
        if (ies == 4) hipLaunchKernelGGL(latent_append_vec_kernel<4>, grid, block, 0, st, a, groups, shift, slices, rounds, rshift);
        else hipLaunchKernelGGL(latent_append_vec_kernel<2>, grid, block, 0, st, a, groups, shift, slices, rounds, rshift);
        return hipGetLastError();
    }
    const int64_t rows = (int64_t)x.N * (x.Hq + 2);
    hipLaunchKernelGGL(latent_append_kernel, dim3(rows_grid(rows)), dim3(256), 0, st, a);
    return hipGetLastError();
}

}  // namespace spire
