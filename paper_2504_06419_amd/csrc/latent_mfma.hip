// latent_mfma.hip -- attention over a latent cache on the 16-bit matrix
// instructions (gfx950).
//
// bf16 queries, bf16 or fp8 rows.  One workgroup of 8 waves per CU holds a unit of
// NB <= 8 blocks of 16 query rows and walks tiles of 16 KT keys, copied HBM -> LDS by
// the load-to-LDS instructions into a ring of stages.  A row is key and value at
// once, so one copy of it in LDS feeds both products:
//   S^T = K Q^T     wave w scores all keys of the tile for row block w, whose
//                   queries stay in its registers, and owns the block's softmax;
//   O^T += C^T P^T  every wave takes an eighth of the latent's dimensions of all
//                   rows, C^T by transposing LDS reads, P through LDS.
// The products of a tile are a tile apart: between two barriers a wave scores tile
// t + 1 and accumulates tile t, so that while one wave of a SIMD forms
// probabilities the other feeds the matrix pipe, and one barrier a tile orders
// the ring, P and the rescaling factors.
//
// Why this split.  A CU takes some 30 GB/s from L2, whether the lines are there or
// not (8 units of 64 rows that share their keys in L2: 2.4 us a tile of 64 keys
// without any arithmetic), so rows that share keys belong into one workgroup: 128
// rows are what its registers hold (128 accumulators and 72 queries of 256).
// LDS then delivers (NB 36 + 8 (4 + NB)) 16-byte reads for (NB 36 + 8 NB 4) matrix
// instructions of a 32-key tile of 512 dimensions, at 8 rows 3072 cycles beside
// 2176 of the matrix pipes.
#include <type_traits>

#include "latent_common.h"
#include "mfma_common.h"

namespace spire {

typedef __attribute__((address_space(3))) u32x4 lds_u32x4;
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef int s32x2 __attribute__((ext_vector_type(2)));

// Load-to-LDS of 16 bytes per lane: lane L's bytes land at lds + 16 L.  Written as
// assembly because the compiler orders its transposing LDS reads behind every
// load-to-LDS that it knows of (vmcnt(0)), which would drain the ring each tile; the
// waits are the kernel's own.  No register is written; m0 names the LDS address.
template <bool NT>
__device__ __forceinline__ void copy16_s(uint64_t base, uint32_t off, uint32_t lds) {
    if constexpr (NT)
        asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1 nt" ::"v"(off), "s"(base), "s"(lds) : "memory", "m0");
    else
        asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(off), "s"(base), "s"(lds) : "memory", "m0");
}
template <bool NT>
__device__ __forceinline__ void copy16_v(uint64_t addr, uint32_t lds) {
    if constexpr (NT)
        asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off nt" ::"v"(addr), "s"(lds) : "memory", "m0");
    else
        asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(addr), "s"(lds) : "memory", "m0");
}

// Workgroup barrier for LDS contents: this wave's LDS accesses are complete; copies
// in flight stay in flight.
__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// whether one of 8 bf16 (16 e4m3fn) values is not finite
template <bool FP8> __device__ __forceinline__ bool any_nonfinite(u32x4 v) {
    bool bad = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (FP8) {
#pragma unroll
            for (int s = 0; s < 32; s += 8) bad |= ((v[i] >> s) & 0x7Fu) == 0x7Fu;
        } else {
            bad |= (v[i] & 0x7F80u) == 0x7F80u || (v[i] & 0x7F800000u) == 0x7F800000u;
        }
    }
    return bad;
}

// Keeps a lane's address a value of the current tile: what is derived from it (an
// exclusive-or per read) is formed where it is used.  Hoisted out of the tile loop
// the derived addresses would take some 50 registers.
__device__ __forceinline__ uint32_t here(uint32_t x) {
    asm volatile("" : "+v"(x));
    return x;
}
// LDS by address.
template <class V> __device__ __forceinline__ V lds_read(uint32_t at) {
    return *reinterpret_cast<const __attribute__((address_space(3))) V *>((const lds_u8 *)(uintptr_t)at);
}
template <bool FP8> __device__ __forceinline__ bool not_finite(uint32_t at) {
    return FP8 ? (lds_read<uint8_t>(at) & 0x7F) == 0x7F : (lds_read<uint16_t>(at) & 0x7F80) == 0x7F80;
}
// The kernel's arguments, read again from where it is called: what is used once per
// segment does not occupy scalar registers through the tile loop.
typedef const Latent __attribute__((address_space(4))) cLatent;
__device__ __forceinline__ cLatent *arguments() {
    uint64_t x = (uint64_t)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(x));
    return (cLatent *)x;
}

// 16-key blocks a tile: as many bytes in every form, about 36 KB.
constexpr int latent_kt(int Dc, bool fp8) { return Dc == 512 && !fp8 ? 2 : 4; }

// Stage of one tile: [TILE][DC] rows, then [TILE][64] rotated parts.  16-byte chunk q of
// row r lies at q ^ fm(r) (main part, low 4 bits) and q ^ fr(r): operand reads (16
// rows, one chunk) and transposing reads (4 rows, 2 chunks) hit distinct banks.
template <int DC, bool FP8> struct LatStage {
    static constexpr int KT = latent_kt(DC, FP8), TILE = 16 * KT;
    static constexpr int ES = FP8 ? 1 : 2;
    static constexpr int RB = DC * ES, RR = kLatentDr * ES;  // bytes of a row's parts
    static constexpr int MAIN = TILE * RB;
    static constexpr int BYTES = TILE * (RB + RR);
    static constexpr int CH = RB / 16, RCH = RR / 16;        // chunks of a row's parts
    static constexpr int ROWS = TILE / 8;                    // rows a wave copies
    static constexpr int ML = ROWS * CH / 64, RL = (ROWS * RCH + 63) / 64;  // its copies
    static constexpr int LOADS = ML + RL;
    static constexpr int PR = 2 * TILE;                      // bytes of a row of P
};
__device__ __forceinline__ int fm(int r) { return ((r & 7) << 1) | ((r >> 3) & 1); }
template <bool FP8> __device__ __forceinline__ int fr(int r) { return FP8 ? (r >> 2) & 3 : (r >> 1) & 7; }
// rows of P: 64 bytes (2 rows a 128-byte line of banks) or 128
template <int PR> __device__ __forceinline__ int fp(int r) { return PR == 64 ? (r >> 1) & 3 : r & 7; }

template <int DC, bool FP8, int NB>
__global__ __launch_bounds__(512, 2) void latent_mfma_kernel(Latent a) {
    using G = LatStage<DC, FP8>;
    constexpr int DK = DC + kLatentDr, TILE = G::TILE, KT = G::KT;
    constexpr int STEPS = DK / 32;      // QK steps of 32 dimensions
    constexpr int XB = DC / 128;        // 16-dimension output blocks of a wave
    constexpr int PB = NB * 16 * G::PR;
    constexpr int REST = 2 * PB + 2 * NB * 64 + 64;
    constexpr int NS0 = (160 * 1024 - REST) / G::BYTES, NS = NS0 > 6 ? 6 : NS0;
    static_assert(NS >= 3, "stage ring too small");
    __shared__ __attribute__((aligned(1024))) uint8_t smem[NS * G::BYTES + REST];
    lds_u8 *ring = (lds_u8 *)smem;
    float *alphas = reinterpret_cast<float *>(smem + NS * G::BYTES + 2 * PB);  // [2][16 NB]; at the end sums, references
    int *flags = reinterpret_cast<int *>(smem + NS * G::BYTES + 2 * PB + 2 * NB * 64);  // [2][8]

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const bool scorer = wave < NB;
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
    float sc = p.sm_scale_log2, vscale = 1.f;
    if (FP8) {
        vscale = uload(p.kv.k_scale, 0);
        sc *= vscale;
    }
    const float margin = kRescaleLog2 / sc;  // of raw scores

    // lane constants of the LDS accesses
    // (chunk 4 c + j of a row at 16 ((4 c + j) ^ f): only bits 4-7 of the address change with c & 3)
    const uint32_t ring0 = (uint32_t)(uintptr_t)ring;
    const uint32_t kmain0 = ring0 + n16 * G::RB + 16 * (j ^ fm(n16));
    const uint32_t krope0 = ring0 + G::MAIN + n16 * G::RR + 16 * (j ^ fr<FP8>(n16));
    // transposing reads: bf16: lane s of group j addresses key 8 j + 4 h + s / 4, 4 dimensions, and receives
    // dimension s of the group's 4 keys; fp8: key 8 j + s / 2, 8 dimensions, and receives dimension s of 8 keys
    const int vr = FP8 ? 8 * j + (n16 >> 1) : 8 * j + (n16 >> 2);
    const uint32_t v0 = ring0 + vr * G::RB + 16 * ((FP8 ? XB * wave : 2 * XB * wave + ((n16 >> 1) & 1)) ^ fm(vr & 15)) + 8 * (n16 & 1);
    const uint32_t p0 = ring0 + NS * G::BYTES + n16 * G::PR;
    const uint32_t pread0 = p0 + 16 * (j ^ fp<G::PR>(n16));
    const uint32_t pwrite0 = p0 + 16 * G::PR * wave + 16 * ((j >> 1) ^ fp<G::PR>(n16)) + 8 * (j & 1);
    const uint32_t tok_bytes = (uint32_t)(p.kv.s_tok * G::ES);

    while (pos < end) {
        const int b = seg;
        const int span = uload(pl.prefix, b + 1) - uload(pl.prefix, b);
        const int tiles = span - pl.seg_cost;
        const int64_t left = end - pos;
        const int te = left < (int64_t)(span - tile) ? tile + (int)left : span;
        if (tile >= tiles) {  // phantom positions only
            pos += te - tile;
            ++seg;
            tile = 0;
            continue;
        }
        const int t1 = te < tiles ? te : tiles;
        const int n = uload(pl.nkeys, b);
        // keys that block x of the unit sees; the first block sees the fewest
        auto limit = [&](int x) {
            cLatent *A = arguments();
            const int i = (u * NB + x) / A->hb, k = A->p.k;
            return n - k + (i <= k ? i : k);
        };
        const int least = limit(0), lim = limit(wave);
        // query of this lane in block x, or a neighbour's where the block has fewer rows
        auto row_of = [&](int x, int n16, bool &ok) {
            cLatent *A = arguments();
            const int rb = u * NB + x, i = rb / A->hb, h = 16 * (rb - i * A->hb) + n16, k = A->p.k, Hq = A->p.Hq;
            ok = i <= k && h < Hq;
            return ((int64_t)b * (k + 1) + (i <= k ? i : k)) * Hq + (h < Hq ? h : Hq - 1);
        };
        f32x4 acc[XB][NB];
        float l = 0.f, msub = 0.f, thr = -INFINITY;  // of the rows this wave scores
#pragma unroll
        for (int x = 0; x < NB; ++x)
#pragma unroll
            for (int y = 0; y < XB; ++y) acc[y][x] = f32x4{0.f, 0.f, 0.f, 0.f};
        lds_barrier();  // every wave is done with the previous segment's LDS
        if (n > 0) {
            // Copies of this wave's rows of a tile.  Where the rows lie in one run of storage
            // its address is looked up a tile ahead.
            const int last = t1 - 1;
            uint64_t from = 0, ahead = 0;
            int rmax = G::ROWS - 1, rmax_ahead = G::ROWS - 1;
            auto look_up = [&](int t) {  // into `ahead`; what was there becomes `from`
                from = ahead;
                rmax = rmax_ahead;
                int key = t * TILE + G::ROWS * wave;
                key = key < n ? key : ((n - 1) & ~(G::ROWS - 1));
                int64_t off;
                if (p.kv.page_size > 0) {
                    const uint32_t idx = a.ps_shift >= 0 ? (uint32_t)key >> a.ps_shift : (uint32_t)key / (uint32_t)p.kv.page_size;
                    int page = uload(p.kv.block_table, (int64_t)b * p.kv.max_blocks + idx);
                    page = page < 0 ? 0 : (page >= p.kv.num_blocks ? p.kv.num_blocks - 1 : page);
                    off = (int64_t)page * p.kv.s_blk + (int64_t)(key - (int)idx * p.kv.page_size) * p.kv.s_tok;
                } else {
                    off = (int64_t)b * p.kv.s_blk + (int64_t)key * p.kv.s_tok;
                    rmax_ahead = p.kv.capacity - 1 - key;  // >= 0: key < n <= capacity
                }
                ahead = (uint64_t)(uintptr_t)p.kv.k + (uint64_t)(off * G::ES);
            };
            const int r0 = (G::ROWS * wave) & 15;
            auto copy = [&](int st, int x) {  // copy x of ML + RL into stage st
                const int lane = here(tid & 63);
                const bool main = x < G::ML;
                const int y = main ? x : x - G::ML, ch = main ? G::CH : G::RCH;
                const int r = y * (64 / ch) + (ch < 64 ? lane / ch : 0);
                const uint32_t chunk = (uint32_t)(lane % ch) ^ (main ? fm(r0 + r) : fr<FP8>(r0 + r));
                const uint32_t off = (uint32_t)(r < rmax ? r : rmax) * tok_bytes + (main ? 0 : G::RB) + 16 * chunk;
                const uint32_t at = ring0 + st * G::BYTES + 1024 * y +
                                    (main ? wave * G::ROWS * G::RB : G::MAIN + wave * G::ROWS * G::RR);
                if (main || G::ROWS * G::RCH >= 64 || r < G::ROWS) {
                    if (a.units == 1) copy16_s<true>(from, off, at);
                    else copy16_s<false>(from, off, at);
                }
            };
            // any page size: lane r holds the address of row r
            auto copy_scattered = [&](int st, int t) {
                const int lane = here(tid & 63);
                int key = t * TILE + G::ROWS * wave + (lane & (G::ROWS - 1));
                key = key < n ? key : n - 1;
                const uint32_t idx = (uint32_t)key / (uint32_t)p.kv.page_size;
                int page = p.kv.block_table[(int64_t)b * p.kv.max_blocks + idx];
                page = page < 0 ? 0 : (page >= p.kv.num_blocks ? p.kv.num_blocks - 1 : page);
                const uint64_t addr = (uint64_t)(uintptr_t)p.kv.k +
                    (uint64_t)(((int64_t)page * p.kv.s_blk + (int64_t)(key - (int)idx * p.kv.page_size) * p.kv.s_tok) * G::ES);
                const uint32_t at = ring0 + st * G::BYTES;
#pragma unroll 1
                for (int x = 0; x < G::ML; ++x) {
                    const int r = x * (64 / G::CH) + lane / G::CH, q16 = (lane % G::CH) ^ fm(r0 + r);
                    copy16_v<false>(__shfl(addr, r) + 16u * q16, at + wave * G::ROWS * G::RB + x * 1024);
                }
#pragma unroll 1
                for (int x = 0; x < G::RL; ++x) {
                    const int r = x * (64 / G::RCH) + lane / G::RCH, q16 = (lane % G::RCH) ^ fr<FP8>(r0 + r);
                    const uint64_t src = __shfl(addr, r) + G::RB + 16u * q16;
                    if (r < G::ROWS) copy16_v<false>(src, at + G::MAIN + wave * G::ROWS * G::RR + x * 1024);
                }
            };
            auto issue = [&](int st, int t) {
                if (!a.uniform) return copy_scattered(st, t);
#pragma unroll
                for (int x = 0; x < G::LOADS; ++x) copy(st, x);
            };

            if (a.uniform) look_up(tile);
#pragma unroll
            for (int s = 0; s < NS - 1; ++s) {
                if (a.uniform) look_up(tile + s + 1);
                if (tile + s <= last) issue(s, tile + s);
            }
            // queries: step s of bf16 rows is dimensions 32 s + 8 j .. + 7; of fp8 rows, whose
            // 16-byte chunk feeds two steps, 64 (s / 2) + 16 j + 8 (s % 2) .. + 7
            u32x4 q[STEPS];
            {
                const int ln = here(lane);
                bool ok;
                const uint8_t *row = arguments()->p.q + row_of(scorer ? wave : 0, ln & 15, ok) * (DK * 2) + (FP8 ? 32 : 16) * (ln >> 4);
#pragma unroll
                for (int s = 0; s < STEPS; ++s)
                    q[s] = *reinterpret_cast<const u32x4 *>(row + (FP8 ? 128 * (s >> 1) + 16 * (s & 1) : 64 * s));
            }

            // ---- probabilities of tile t (stage st) into buffer `buf` ----------------
            auto score = [&](int t, int st, int buf) {
                const int key0 = t * TILE;
                const bool tail = key0 + TILE > least;
                // A hidden key's probability is 0, which clears any finite value; what is not
                // finite in this wave's rows from the first hidden key on is looked for.
                bool bad = false;
                if (tail) {
                    const int lane = here(tid & 63);
                    for (int i = lane; i < G::ROWS * G::CH; i += 64)
                        if (key0 + G::ROWS * wave + i / G::CH >= least)
                            bad |= any_nonfinite<FP8>(lds_read<u32x4>(ring0 + st * G::BYTES + wave * G::ROWS * G::RB + 16 * i));
                }
                int word = __any(bad) ? 2 : 0;
                if (scorer) {
                    const uint32_t kmain = here(kmain0 + st * G::BYTES), krope = here(krope0 + st * G::BYTES);
                    f32x4 s[KT];
#pragma unroll
                    for (int y = 0; y < KT; ++y) s[y] = f32x4{0.f, 0.f, 0.f, 0.f};
                    // K operands a group of reads ahead of the products
                    constexpr int RAWS = FP8 ? STEPS / 2 : STEPS, KG = 4 / KT;  // steps a group
                    auto read_k = [&](int c, int y) {
                        if constexpr (FP8)
                            return lds_read<u32x4>((c < DC / 64 ? (kmain ^ (64 * (c & 3))) + 256 * (c >> 2) + 16 * y * G::RB : krope + 16 * y * G::RR));
                        else
                            return lds_read<u32x4>((c < DC / 32 ? (kmain ^ (64 * (c & 3))) + 256 * (c >> 2) + 16 * y * G::RB
                                                                : (krope ^ (64 * (c - DC / 32))) + 16 * y * G::RR));
                    };
                    u32x4 kb[2][KG][KT];
                    auto fetch = [&](int into, int c0) {
#pragma unroll
                        for (int c = 0; c < KG; ++c)
#pragma unroll
                            for (int y = 0; y < KT; ++y)
                                if (c0 + c < RAWS) kb[into][c][y] = read_k(c0 + c, y);
                    };
                    fetch(0, 0);
#pragma unroll
                    for (int c0 = 0; c0 < RAWS; c0 += KG) {
                        const int cur = (c0 / KG) & 1;
                        fetch(cur ^ 1, c0 + KG);
#pragma unroll
                        for (int c = 0; c < KG; ++c)
                            if (c0 + c < RAWS) {
#pragma unroll
                                for (int y = 0; y < KT; ++y) {
                                    const u32x4 r = kb[cur][c][y];
                                    if constexpr (FP8) {
                                        s[y] = mfma_bf16(fp8x8_to_bf16x8(r.x, r.y), q[2 * (c0 + c)], s[y]);
                                        s[y] = mfma_bf16(fp8x8_to_bf16x8(r.z, r.w), q[2 * (c0 + c) + 1], s[y]);
                                    } else {
                                        s[y] = mfma_bf16(r, q[c0 + c], s[y]);
                                    }
                                }
                            }
                        __builtin_amdgcn_sched_barrier(0);
                    }
                    if (tail) {
                        const int key = key0 + 4 * (here(lane) >> 4);
#pragma unroll
                        for (int y = 0; y < KT; ++y)
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                if (key + 16 * y + e >= lim) s[y][e] = -INFINITY;
                    }
                    // lazy references: a row's moves when a score passes it by more than 2^8
                    // (NaN-propagating maximum: a NaN score never passes)
                    float top = s[0][0];
#pragma unroll
                    for (int y = 0; y < KT; ++y) top = max3n(max3n(top, s[y][0], s[y][1]), s[y][2], s[y][3]);
                    if (__any(top > thr)) {
                        float m = top != top ? -INFINITY : top;
                        m = fmaxf(m, __shfl_xor(m, 16));
                        m = fmaxf(m, __shfl_xor(m, 32));
                        float alpha = 1.f;
                        if (m > thr) {
                            alpha = thr == -INFINITY ? 0.f : fast_exp2((msub - m) * sc);
                            msub = m;
                            thr = fmaxf(m + margin, -FLT_MAX);
                            l *= alpha;
                        }
                        const int ln = here(lane);
                        if (ln < 16) alphas[buf * 16 * NB + 16 * wave + ln] = alpha;
                        word |= 1;
                    }
#pragma unroll
                    for (int y = 0; y < KT; ++y) {
                        float e[4];
#pragma unroll
                        for (int z = 0; z < 4; ++z) e[z] = fast_exp2((s[y][z] - msub) * sc);
                        l += (e[0] + e[1]) + (e[2] + e[3]);
                        const u32x2 v = {pack_p<FP8>(e[0], e[1]), pack_p<FP8>(e[2], e[3])};
                        *reinterpret_cast<__attribute__((address_space(3))) u32x2 *>((lds_u8 *)(uintptr_t)((pwrite0 ^ (32 * y)) + buf * PB)) = v;
                    }
                }
                if (here(lane) == 0) flags[8 * buf + wave] = word;
            };

            // wait for this wave's rows of tile t; behind them the copies of `behind` tiles are in flight
            auto landed = [&](int t) {
                const int behind = last - t < NS - 3 ? last - t : NS - 3;
                if (NS >= 6 && behind == 3) wait_vmcnt<3 * G::LOADS>();
                else if (NS >= 5 && behind == 2) wait_vmcnt<2 * G::LOADS>();
                else if (NS >= 4 && behind == 1) wait_vmcnt<G::LOADS>();
                else wait_vmcnt<0>();
            };
            wait_vmcnt<0>();  // the queries and the first tiles
            lds_barrier();
            score(tile, 0, 0);
            int rd = 0, buf = 0, wr = NS - 1;
            for (int tt = tile; tt <= last; ++tt) {
                landed(tt + 1);
                lds_barrier();  // tile tt + 1 and the probabilities of tt are there, tile tt - 1 is read
                if (a.uniform) look_up(tt + NS);
                if (tt + NS - 1 <= last) issue(wr, tt + NS - 1);
                wr = wr + 1 == NS ? 0 : wr + 1;
                const int st = rd, key0 = tt * TILE;
                rd = rd + 1 == NS ? 0 : rd + 1;
                const int4 f0 = *reinterpret_cast<const int4 *>(flags + 8 * buf), f1 = *reinterpret_cast<const int4 *>(flags + 8 * buf + 4);
                if (tt < last) score(tt + 1, rd, buf ^ 1);
                const int events = __builtin_amdgcn_readfirstlane(f0.x | f0.y | f0.z | f0.w | f1.x | f1.y | f1.z | f1.w);

                // Accumulators change outside the products in this one place only (each place
                // more costs the register allocator a copy of them).
                if (events != 0) {
                    const int lane = here(tid & 63), j = lane >> 4;
                    uint32_t nans[NB];  // per block: bit 4 y + e
#pragma unroll
                    for (int x = 0; x < NB; ++x) nans[x] = 0;
                    if (events & 2) {
                        // A value that is not finite makes its dimension NaN in the rows that see its
                        // key (the key's score is not finite either); then it is cleared.
                        const uint32_t sb = ring0 + st * G::BYTES;
                        const int stop = n < key0 + TILE ? n : key0 + TILE;
                        for (int key = least > key0 ? least : key0; key < stop; ++key) {
                            const int r = key - key0;
                            uint32_t bits = 0;
#pragma unroll
                            for (int y = 0; y < XB; ++y) {
                                const int byte = (wave * (DC / 8) + 16 * y + 4 * j) * G::ES;
                                const uint32_t at = sb + r * G::RB + 16 * ((byte >> 4) ^ fm(r & 15)) + (byte & 15);
#pragma unroll
                                for (int e = 0; e < 4; ++e)
                                    if (not_finite<FP8>(at + e * G::ES)) bits |= 1u << (4 * y + e);
                            }
#pragma unroll
                            for (int x = 0; x < NB; ++x) nans[x] |= key < limit(x) ? bits : 0u;
                        }
                        lds_barrier();
                        for (int i = lane; i < G::ROWS * G::CH; i += 64)
                            if (key0 + G::ROWS * wave + i / G::CH >= least) {
                                const uint32_t at = sb + wave * G::ROWS * G::RB + 16 * i;
                                for (int e = 0; e < 16; e += G::ES)
                                    if (not_finite<FP8>(at + e)) {
                                        if constexpr (FP8) *reinterpret_cast<__attribute__((address_space(3))) uint8_t *>((lds_u8 *)(uintptr_t)(at + e)) = 0;
                                        else *reinterpret_cast<__attribute__((address_space(3))) uint16_t *>((lds_u8 *)(uintptr_t)(at + e)) = 0;
                                    }
                            }
                        lds_barrier();
                    }
#pragma unroll
                    for (int x = 0; x < NB; ++x) {
                        const int f = x == 0 ? f0.x : x == 1 ? f0.y : x == 2 ? f0.z : x == 3 ? f0.w
                                    : x == 4 ? f1.x : x == 5 ? f1.y : x == 6 ? f1.z : f1.w;
                        const float alpha = f & 1 ? alphas[buf * 16 * NB + 16 * x + (lane & 15)] : 1.f;  // the reference moved
#pragma unroll
                        for (int y = 0; y < XB; ++y)
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                acc[y][x][e] = nans[x] & (1u << (4 * y + e)) ? __builtin_nanf("") : acc[y][x][e] * alpha;
                        __builtin_amdgcn_sched_barrier(0);
                    }
                }

                // ---- O^T += C^T P^T ----------------------------------------------
                const uint32_t vat = here(v0 + st * G::BYTES), pat = here(pread0 + buf * PB);
                auto read_v = [&](int ks, int y) {
                    if constexpr (FP8) {
                        const s32x2 t = __builtin_amdgcn_ds_read_tr8_b64_v2i32(
                            (__attribute__((address_space(3))) s32x2 *)(lds_u8 *)(uintptr_t)((vat ^ (16 * y)) + 32 * ks * G::RB));
                        return fp8x8_to_f16x8((uint32_t)t.x, (uint32_t)t.y);
                    } else {
                        s16x4 t[2];
#pragma unroll
                        for (int h = 0; h < 2; ++h)  // row + 4: its swizzle differs in bit 3
                            t[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                                (__attribute__((address_space(3))) s16x4 *)(lds_u8 *)(uintptr_t)((vat ^ (32 * y) ^ (128 * h)) + (32 * ks + 4 * h) * G::RB));
                        const u32x2 lo = __builtin_bit_cast(u32x2, t[0]), hi = __builtin_bit_cast(u32x2, t[1]);
                        return u32x4{lo.x, lo.y, hi.x, hi.y};
                    }
                };
#pragma unroll
                for (int ks = 0; ks < KT / 2; ++ks) {
                    u32x4 v[XB], pf[2];
#pragma unroll
                    for (int y = 0; y < XB; ++y) v[y] = read_v(ks, y);
                    auto read_p = [&](int x) { return lds_read<u32x4>((pat ^ (64 * ks)) + 16 * G::PR * x); };
                    pf[0] = read_p(0);
#pragma unroll
                    for (int x = 0; x < NB; ++x) {
                        if (x + 1 < NB) pf[(x + 1) & 1] = read_p(x + 1);
#pragma unroll
                        for (int y = 0; y < XB; ++y) acc[y][x] = mfma_pv<FP8>(v[y], pf[x & 1], acc[y][x]);
                        __builtin_amdgcn_sched_barrier(0);
                    }
                }
                buf ^= 1;
            }
        }

        // ---- row sums and references to all waves, rows out -----------------------
        const int ln = here(lane), n16 = ln & 15, j = ln >> 4;
        lds_barrier();
        l += __shfl_xor(l, 16);
        l += __shfl_xor(l, 32);
        if (scorer && j == 0) {
            alphas[16 * wave + n16] = l;
            alphas[16 * NB + 16 * wave + n16] = msub;
        }
        lds_barrier();
        cLatent *A = arguments();
        const bool whole = tile == 0 && t1 == tiles;
        const int64_t slot = 2 * (int64_t)g + (pos == begin ? 0 : 1);
#pragma unroll
        for (int x = 0; x < NB; ++x) {
            const float sum = alphas[16 * x + n16];
            const float inv = sum == 0.f ? 0.f : vscale / sum;
            const float lse2 = sum == 0.f ? -INFINITY : alphas[16 * NB + 16 * x + n16] * sc + log2f(sum);
            bool ok;
            const int64_t qrow = row_of(x, n16, ok);
            if (whole && !ok) continue;
            const int64_t row = whole ? qrow : slot * A->pl.rows + 16 * (u * NB + x) + n16;
            const int64_t at = row * DC + wave * (DC / 8) + 4 * j;
            if (whole && A->p.out_dtype == SPIRE_BF16) {
                uint16_t *o = static_cast<uint16_t *>(A->p.out) + at;
#pragma unroll
                for (int y = 0; y < XB; ++y) {
                    const f32x4 v = acc[y][x] * inv;
                    *reinterpret_cast<u32x2 *>(o + 16 * y) = u32x2{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
                }
            } else {
                float *o = (whole ? static_cast<float *>(A->p.out) : A->pl.part_o) + at;
#pragma unroll
                for (int y = 0; y < XB; ++y) *reinterpret_cast<f32x4 *>(o + 16 * y) = acc[y][x] * inv;
            }
            if (wave == 0 && j == 0) {
                if (!whole) A->pl.part_lse[row] = lse2;
                else if (A->p.lse != nullptr) A->p.lse[row] = lse2 * 0.69314718055994531f;
            }
        }
        pos += te - tile;
        ++seg;
        tile = 0;
    }
}

int latent_tile(int Dc, bool fp8) { return 16 * latent_kt(Dc, fp8); }

template <int DC, bool FP8>
static hipError_t launch_nb(const Latent &a, hipStream_t st) {
    const dim3 grid((unsigned)(a.pl.workers * a.units)), block(512);
    switch (a.nb) {
    case 1: hipLaunchKernelGGL((latent_mfma_kernel<DC, FP8, 1>), grid, block, 0, st, a); break;
    case 2: hipLaunchKernelGGL((latent_mfma_kernel<DC, FP8, 2>), grid, block, 0, st, a); break;
    case 3: hipLaunchKernelGGL((latent_mfma_kernel<DC, FP8, 3>), grid, block, 0, st, a); break;
    case 4: hipLaunchKernelGGL((latent_mfma_kernel<DC, FP8, 4>), grid, block, 0, st, a); break;
    case 5: hipLaunchKernelGGL((latent_mfma_kernel<DC, FP8, 5>), grid, block, 0, st, a); break;
    case 6: hipLaunchKernelGGL((latent_mfma_kernel<DC, FP8, 6>), grid, block, 0, st, a); break;
    case 7: hipLaunchKernelGGL((latent_mfma_kernel<DC, FP8, 7>), grid, block, 0, st, a); break;
    case 8: hipLaunchKernelGGL((latent_mfma_kernel<DC, FP8, 8>), grid, block, 0, st, a); break;
    default: return hipErrorInvalidValue;
    }
    return hipGetLastError();
}

hipError_t launch_latent_mfma(const Latent &a, hipStream_t st) {
    const bool fp8 = a.p.kv_dtype == SPIRE_FP8_E4M3FN;
    if (a.p.D == 512) return fp8 ? launch_nb<512, true>(a, st) : launch_nb<512, false>(a, st);
    return fp8 ? launch_nb<256, true>(a, st) : launch_nb<256, false>(a, st);
}

}  // namespace spire
