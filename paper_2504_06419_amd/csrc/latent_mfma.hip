// latent_mfma.hip -- attention over a latent cache on the 16-bit matrix
// instructions (gfx950).
//
// bf16 queries, bf16 or fp8 rows.  One workgroup of 4 waves (one per SIMD, one
// workgroup per CU) holds a unit of NB blocks of 16 query rows and walks tiles of
// 64 keys, copied HBM -> LDS by the load-to-LDS instructions into a ring of
// stages.  A row is key and value at once, so it is read from memory and from the
// stage's one copy for both products:
//   S^T = K Q^T   wave w takes keys 16 w .. 16 w + 15 against all rows: the K
//                 operand leaves LDS once, the queries stay in registers;
//   O^T += C^T P^T  wave w takes a quarter of the latent's dimensions of all rows
//                 and keys: C^T by transposing LDS reads, P through LDS.
// Split this way LDS delivers a row once per product instead of once per wave.  With
// 4 blocks of a 512-wide latent the queries of all blocks would take 288 registers
// beside 128 accumulators: there 2 waves share the keys and 2 the rows (60 reads
// of 16 bytes for 136 matrix instructions instead of 42).
// The softmax keeps a lazy reference per row: a wave whose scores pass it by more
// than 2^8 raises its flag along with its probabilities, and after the barrier
// all waves move the references together (rare); otherwise one barrier orders
// P and one the stage ring, per tile.
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

constexpr int kLatTile = 64;

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
__device__ __forceinline__ uint32_t here_s(uint32_t x) {
    asm volatile("" : "+s"(x));
    return x;
}
// The kernel's arguments, read again from where it is called: what is used once per
// segment does not occupy scalar registers through the tile loop.
typedef const Latent __attribute__((address_space(4))) cLatent;
__device__ __forceinline__ cLatent *arguments() {
    uint64_t x = (uint64_t)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(x));
    return (cLatent *)x;
}
template <class V> __device__ __forceinline__ V lds_read(uint32_t at) {
    return *reinterpret_cast<const __attribute__((address_space(3))) V *>((const lds_u8 *)(uintptr_t)at);
}

// Stage of one tile: [64][DC] rows, then [64][64] rotated parts.  16-byte chunk q of
// row r lies at q ^ fm(r) (main part, low 4 bits) and q ^ fr(r): operand reads (16
// rows, one chunk) and transposing reads (4 rows, 2 chunks) hit distinct banks.
template <int DC, bool FP8, int WAVES> struct LatStage {
    static constexpr int ES = FP8 ? 1 : 2;
    static constexpr int RB = DC * ES, RR = kLatentDr * ES;  // bytes of a row's parts
    static constexpr int MAIN = kLatTile * RB;
    static constexpr int BYTES = kLatTile * (RB + RR);
    static constexpr int CH = RB / 16, RCH = RR / 16;        // chunks of a row's parts
    static constexpr int ROWS = kLatTile / WAVES;            // rows a wave copies
    static constexpr int ML = ROWS * CH / 64, RL = (ROWS * RCH + 63) / 64;  // its copies
    static constexpr int LOADS = ML + RL;
};
__device__ __forceinline__ int fm(int r) { return ((r & 7) << 1) | ((r >> 3) & 1); }
template <bool FP8> __device__ __forceinline__ int fr(int r) { return FP8 ? (r >> 2) & 3 : (r >> 1) & 7; }

template <int DC, bool FP8, int NB, int WAVES>
__global__ __launch_bounds__(64 * WAVES, WAVES / 4) void latent_mfma_kernel(Latent a) {
    using G = LatStage<DC, FP8, WAVES>;
    constexpr int DK = DC + kLatentDr;
    constexpr int STEPS = DK / 32;      // QK steps of 32 dimensions
    constexpr int XB = DC / (16 * WAVES);                // 16-dimension output blocks of a wave
    constexpr int KW = 4, RW = WAVES / KW, NW = NB / RW;  // scores: waves along keys, along rows; a wave's row blocks
    static_assert(NB % RW == 0, "row blocks split evenly");
    constexpr int PB = NB * 16 * 128;   // P: [rows][64 keys] 16-bit
    // Two waves per SIMD have 256 registers each: with 4 blocks of a 512-wide latent the
    // last QL steps of the queries stay in LDS (fp8 stages are half as large: one less).
    constexpr int QL = DC == 512 && NB == 4 ? (FP8 ? 4 : 1) : 0, QR = STEPS - QL;
    constexpr int QBYTES = QL * NB * 1024;
    constexpr int NS0 = (160 * 1024 - PB - QBYTES - 2048) / G::BYTES, NS = NS0 > 4 ? 4 : NS0;
    static_assert(NS >= 2, "stage ring too small");
    __shared__ __attribute__((aligned(1024))) uint8_t smem[NS * G::BYTES + QBYTES + PB + (KW + 1) * NB * 64 + 4 * WAVES];
    lds_u8 *ring = (lds_u8 *)smem;
    lds_u8 *pbuf = ring + NS * G::BYTES + QBYTES;
    float *red = reinterpret_cast<float *>(smem + NS * G::BYTES + QBYTES + PB);  // [KW][16 NB]
    float *refs = red + KW * 16 * NB;                                  // [16 NB] references, -inf: none yet
    int *flags = reinterpret_cast<int *>(refs + 16 * NB);              // [WAVES]

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int kw = wave & (KW - 1), rw = wave / KW;
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

    // lane constants of the LDS reads
    // (chunk 4 c + j of a row at 16 ((4 c + j) ^ f): only bits 4-7 of the address change with c & 3)
    const uint32_t ring0 = (uint32_t)(uintptr_t)ring;
    const uint32_t kmain0 = (uint32_t)(16 * kw + n16) * G::RB + 16 * (j ^ fm(n16));
    const uint32_t krope0 = (uint32_t)G::MAIN + (uint32_t)(16 * kw + n16) * G::RR + 16 * (j ^ fr<FP8>(n16));
    // transposing reads: bf16: lane s of group j addresses key 8 j + 4 h + s / 4, 4 dimensions, and receives
    // dimension s of the group's 4 keys; fp8: key 8 j + s / 2, 8 dimensions, and receives dimension s of 8 keys
    const int vr = FP8 ? 8 * j + (n16 >> 1) : 8 * j + (n16 >> 2);
    const uint32_t v0 = (uint32_t)vr * G::RB + 16 * ((FP8 ? XB * wave : 2 * XB * wave + ((n16 >> 1) & 1)) ^ fm(vr & 15)) + 8 * (n16 & 1);
    const uint32_t q0 = ring0 + NS * G::BYTES + 1024 * NW * rw + 16 * lane;  // queries in LDS: [QL][NB][64 lanes]
    const uint32_t p0 = (uint32_t)(uintptr_t)pbuf + n16 * 128;
    const uint32_t pread0 = p0 + 16 * (j ^ (n16 & 7));
    const uint32_t pwrite0 = p0 + 2048 * NW * rw + 16 * ((2 * kw + (j >> 1)) ^ (n16 & 7)) + 8 * (j & 1);
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
        const int least = limit(0);
        int lim[NW];
#pragma unroll
        for (int x = 0; x < NW; ++x) lim[x] = limit(NW * rw + x);
        // query of this lane in block x, or a neighbour's where the block has fewer rows
        auto row_of = [&](int x, int n16, bool &ok) {
            cLatent *A = arguments();
            const int rb = u * NB + x, i = rb / A->hb, h = 16 * (rb - i * A->hb) + n16, k = A->p.k, Hq = A->p.Hq;
            ok = i <= k && h < Hq;
            return ((int64_t)b * (k + 1) + (i <= k ? i : k)) * Hq + (h < Hq ? h : Hq - 1);
        };
        f32x4 acc[XB][NB];
        float l[NW], msub[NW], thr[NW];  // of the rows this wave scores
#pragma unroll
        for (int x = 0; x < NW; ++x) {
            l[x] = 0.f;
            msub[x] = 0.f;
            thr[x] = -INFINITY;
        }
#pragma unroll
        for (int x = 0; x < NB; ++x)
#pragma unroll
            for (int y = 0; y < XB; ++y) acc[y][x] = f32x4{0.f, 0.f, 0.f, 0.f};
        lds_barrier();  // every wave is done with the previous segment's LDS
        if (tid < 16 * NB) refs[tid] = -INFINITY;
        if (n > 0) {
            // queries: step s of bf16 rows is dimensions 32 s + 8 j .. + 7; of fp8 rows, whose
            // 16-byte chunk feeds two steps, 64 (s / 2) + 16 j + 8 (s % 2) .. + 7
            u32x4 q[NW][QR];
            const int ln0 = here(lane);
#pragma unroll
            for (int x = 0; x < NW; ++x) {
                bool ok;
                const uint8_t *row = arguments()->p.q + row_of(NW * rw + x, ln0 & 15, ok) * (DK * 2) + (FP8 ? 32 : 16) * (ln0 >> 4);
#pragma unroll
                for (int s = 0; s < STEPS; ++s) {
                    const u32x4 v = *reinterpret_cast<const u32x4 *>(row + (FP8 ? 128 * (s >> 1) + 16 * (s & 1) : 64 * s));
                    if (s < QR) q[x][s] = v;
                    else if (kw == 0)  // shared by the waves of these rows; the first tile's barrier publishes it
                        *reinterpret_cast<lds_u32x4 *>((lds_u8 *)(uintptr_t)(q0 + 1024 * (NB * (s - QR) + x))) = v;
                }
            }

            // copies of this wave's 16 rows of tile t into stage `st`
            const int last = t1 - 1;
            auto issue = [&](int st, int t) {
                const uint32_t at = (uint32_t)(uintptr_t)(ring + st * G::BYTES) + (uint32_t)wave * G::ROWS * G::RB;
                const uint32_t rat = (uint32_t)(uintptr_t)(ring + st * G::BYTES) + G::MAIN + (uint32_t)wave * G::ROWS * G::RR;
                int key = t * kLatTile + G::ROWS * wave;
                const int r0 = (G::ROWS * wave) & 15;
                const int lane = here(tid & 63);
                if (a.uniform) {  // 16 keys in one run of storage
                    key = key < n ? key : ((n - 1) & ~(G::ROWS - 1));
                    int64_t off;
                    int rmax = 15;
                    if (p.kv.page_size > 0) {
                        const uint32_t idx = (uint32_t)key / (uint32_t)p.kv.page_size;
                        int page = uload(p.kv.block_table, (int64_t)b * p.kv.max_blocks + idx);
                        page = page < 0 ? 0 : (page >= p.kv.num_blocks ? p.kv.num_blocks - 1 : page);
                        off = (int64_t)page * p.kv.s_blk + (int64_t)(key - (int)idx * p.kv.page_size) * p.kv.s_tok;
                    } else {
                        off = (int64_t)b * p.kv.s_blk + (int64_t)key * p.kv.s_tok;
                        rmax = p.kv.capacity - 1 - key;  // >= 0: key < n <= capacity
                    }
                    const uint64_t base = (uint64_t)(uintptr_t)p.kv.k + (uint64_t)(off * G::ES);
                    auto go = [&](auto nt) {
                        constexpr bool NT = decltype(nt)::value;
const uint32_t q16 = 16u * (lane % G::CH), rq16 = 16u * (lane % G::RCH), tb = here_s(tok_bytes);
#pragma unroll
                        for (int x = 0; x < G::ML; ++x) {
                            const int r = x * (64 / G::CH) + (G::CH < 64 ? lane / G::CH : 0);
                            copy16_s<NT>(base, (uint32_t)(r < rmax ? r : rmax) * tb + (q16 ^ (16u * fm(r0 + r))), at + x * 1024);
                        }
#pragma unroll
                        for (int x = 0; x < G::RL; ++x) {
                            const int r = x * (64 / G::RCH) + lane / G::RCH;
                            if (r < G::ROWS)
                                copy16_s<NT>(base, (uint32_t)(r < rmax ? r : rmax) * tb + G::RB + (rq16 ^ (16u * fr<FP8>(r0 + r))), rat + x * 1024);
                        }
                    };
                    if (a.units == 1) go(std::true_type{});
                    else go(std::false_type{});
                    return;
                }
                // any page size: lane r holds the address of row r
                key += lane & (G::ROWS - 1);
                key = key < n ? key : n - 1;
                const uint32_t idx = (uint32_t)key / (uint32_t)p.kv.page_size;
                int page = p.kv.block_table[(int64_t)b * p.kv.max_blocks + idx];
                page = page < 0 ? 0 : (page >= p.kv.num_blocks ? p.kv.num_blocks - 1 : page);
                const uint64_t addr = (uint64_t)(uintptr_t)p.kv.k +
                    (uint64_t)(((int64_t)page * p.kv.s_blk + (int64_t)(key - (int)idx * p.kv.page_size) * p.kv.s_tok) * G::ES);
const uint32_t ln = here(lane);
#pragma unroll 1
                for (int x = 0; x < G::ML; ++x) {
                    const int r = x * (64 / G::CH) + lane / G::CH, q16 = (lane % G::CH) ^ fm(r0 + r);
                    copy16_v<false>(__shfl(addr, r) + 16u * q16, at + x * 1024);
                }
#pragma unroll 1
                for (int x = 0; x < G::RL; ++x) {
                    const int r = x * (64 / G::RCH) + lane / G::RCH, q16 = (lane % G::RCH) ^ fr<FP8>(r0 + r);
                    const uint64_t from = __shfl(addr, r) + G::RB + 16u * q16;
                    if (r < G::ROWS) copy16_v<false>(from, rat + x * 1024);
                }
            };

            wait_vmcnt<0>();  // the queries: from here on only the ring's copies are counted
#pragma unroll
            for (int s = 0; s < NS - 1; ++s) issue(s, tile + s < last ? tile + s : last);
            int rd = 0, wr = NS - 1;
            for (int tt = tile; tt <= last; ++tt) {
                wait_vmcnt<(NS - 2) * G::LOADS>();  // this wave's rows of tile tt have landed
                lds_barrier();                      // everyone's have; tile tt - 1 is fully read
                issue(wr, tt + NS - 1 < last ? tt + NS - 1 : last);
                wr = wr + 1 == NS ? 0 : wr + 1;
                const uint32_t st = ring0 + rd * G::BYTES;
                const uint32_t kmain = here(st + kmain0), krope = here(st + krope0);
                rd = rd + 1 == NS ? 0 : rd + 1;
                const int key0 = tt * kLatTile;

                // ---- S^T of this wave's keys and rows ------------------------------
                f32x4 s[NW], s2 = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int x = 0; x < NW; ++x) s[x] = f32x4{0.f, 0.f, 0.f, 0.f};
                constexpr bool TWO = NW == 1;  // one chain of dependent products: make it two
                // K operands a group of reads ahead of the products
                constexpr int READS = FP8 ? STEPS / 2 : STEPS;  // 16-byte reads
                constexpr int KG = WAVES == 4 ? (NW >= 3 ? 3 : 4) : (FP8 ? 2 : 1);
                auto read_k = [&](int c) {
                    if constexpr (FP8) return lds_read<u32x4>(c < DC / 64 ? (kmain ^ (64 * (c & 3))) + 256 * (c >> 2) : krope);
                    else return lds_read<u32x4>(c < DC / 32 ? (kmain ^ (64 * (c & 3))) + 256 * (c >> 2) : krope ^ (64 * (c - DC / 32)));
                };
                auto step = [&](int c, u32x4 k4) {
#pragma unroll
                    for (int x = 0; x < NW; ++x) {
                        const u32x4 qx = c < QR ? q[x][c] : lds_read<u32x4>(q0 + 1024 * (NB * (c - QR) + x));
                        if (TWO && (c & 1)) s2 = mfma_bf16(k4, qx, s2);
                        else s[x] = mfma_bf16(k4, qx, s[x]);
                    }
                };
                u32x4 kb[2][KG];
#pragma unroll
                for (int y = 0; y < KG; ++y) kb[0][y] = read_k(y);
#pragma unroll
                for (int i0 = 0; i0 < READS; i0 += KG) {
                    const int cur = (i0 / KG) & 1;
#pragma unroll
                    for (int y = 0; y < KG; ++y)
                        if (i0 + KG + y < READS) kb[cur ^ 1][y] = read_k(i0 + KG + y);
#pragma unroll
                    for (int y = 0; y < KG; ++y)
                        if (i0 + y < READS) {
                            const u32x4 r = kb[cur][y];
                            if constexpr (FP8) {
                                step(2 * (i0 + y), fp8x8_to_bf16x8(r.x, r.y));
                                step(2 * (i0 + y) + 1, fp8x8_to_bf16x8(r.z, r.w));
                            } else {
                                step(i0 + y, r);
                            }
                        }
                    __builtin_amdgcn_sched_barrier(0);
                }
                if (TWO) s[0] += s2;

                // ---- mask, probabilities against the current references -----------
                const bool tail = key0 + kLatTile > least;
                if (tail) {
                    const int key = key0 + 16 * kw + 4 * (here(lane) >> 4);
#pragma unroll
                    for (int x = 0; x < NW; ++x)
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (key + e >= lim[x]) s[x][e] = -INFINITY;
                }
                auto top = [&](int x) {  // NaN-propagating: a NaN score never passes a threshold
                    return __builtin_elementwise_maximum(max3n(s[x][0], s[x][1], s[x][2]), s[x][3]);
                };
                float add[NW];
                auto weigh = [&]() {
#pragma unroll
                    for (int x = 0; x < NW; ++x) {
                        float e[4];
#pragma unroll
                        for (int z = 0; z < 4; ++z) e[z] = fast_exp2((s[x][z] - msub[x]) * sc);
                        add[x] = (e[0] + e[1]) + (e[2] + e[3]);
                        const u32x2 v = {pack_p<FP8>(e[0], e[1]), pack_p<FP8>(e[2], e[3])};
                        *reinterpret_cast<__attribute__((address_space(3))) u32x2 *>((lds_u8 *)(uintptr_t)(pwrite0 + 2048 * x)) = v;
                    }
                };
                // A hidden key's probability is 0, which clears any finite value; what is not
                // finite in this wave's rows from the first hidden key on is looked for.
                bool bad = false;
                if (tail) {
                    for (int i = lane; i < G::ROWS * G::CH; i += 64)
                        if (key0 + G::ROWS * wave + i / G::CH >= least)
                            bad |= any_nonfinite<FP8>(lds_read<u32x4>(st + wave * G::ROWS * G::RB + 16 * i));
                }
                bool over = false;
#pragma unroll
                for (int x = 0; x < NW; ++x) over |= top(x) > thr[x];
                const int word = (__any(over) ? 1 : 0) | (__any(bad) ? 2 : 0);
                weigh();
                if (lane == 0) flags[wave] = word;
                lds_barrier();
                int all = 0;
#pragma unroll
                for (int w = 0; w < WAVES; w += 4) {
                    const int4 fl = *reinterpret_cast<const int4 *>(flags + w);
                    all |= fl.x | fl.y | fl.z | fl.w;
                }
                const int events = __builtin_amdgcn_readfirstlane(all);
                if (events & 1) {
                    const int ln = here(lane), n16 = ln & 15, j = ln >> 4;
                    // some row's scores pass its reference: move the references of all waves
#pragma unroll
                    for (int x = 0; x < NW; ++x) {
                        float m = top(x);
                        m = m != m ? -INFINITY : m;
                        m = fmaxf(m, __shfl_xor(m, 16));
                        m = fmaxf(m, __shfl_xor(m, 32));
                        if (j == 0) red[kw * 16 * NB + 16 * (NW * rw + x) + n16] = m;
                    }
                    lds_barrier();
                    // the reference of row r before and after, and the factor between them
                    auto moved = [&](int r, float &ref) {
                        float m = red[r];
#pragma unroll
                        for (int w = 1; w < KW; ++w) m = fmaxf(m, red[w * 16 * NB + r]);
                        const float old = refs[r];
                        ref = m > old + margin || old == -INFINITY ? m : old;
                        return ref == old ? 1.f : (old == -INFINITY ? 0.f : fast_exp2((old - ref) * sc));
                    };
                    float ref;
#pragma unroll
                    for (int x = 0; x < NB; ++x) {
                        const float alpha = moved(16 * x + n16, ref);
#pragma unroll
                        for (int y = 0; y < XB; ++y) acc[y][x] *= alpha;
                        __builtin_amdgcn_sched_barrier(0);
                    }
                    float mine[NW];
#pragma unroll
                    for (int x = 0; x < NW; ++x) {
                        l[x] *= moved(16 * (NW * rw + x) + n16, ref);
                        mine[x] = ref;
                        msub[x] = ref == -INFINITY ? 0.f : ref;
                        thr[x] = ref == -INFINITY ? -INFINITY : fmaxf(ref + margin, -FLT_MAX);
                    }
                    lds_barrier();  // the old references have been read
                    if (kw == 0 && j == 0) {
#pragma unroll
                        for (int x = 0; x < NW; ++x) refs[16 * (NW * rw + x) + n16] = mine[x];
                    }
                    weigh();
                    lds_barrier();
                }
#pragma unroll
                for (int x = 0; x < NW; ++x) l[x] += add[x];

                if (events & 2) {
                    const int j = here(lane) >> 4;
                    // A value that is not finite makes its dimension NaN in the rows that see its
                    // key (the key's score is not finite either); then it is cleared.
                    const int stop = n < key0 + kLatTile ? n : key0 + kLatTile;
                    for (int key = least > key0 ? least : key0; key < stop; ++key) {
                        const int r = key - key0;
#pragma unroll
                        for (int y = 0; y < XB; ++y) {
                            const int d = wave * (DC / WAVES) + 16 * y + 4 * j, byte = d * G::ES;
                            const uint32_t at = st + r * G::RB + 16 * ((byte >> 4) ^ fm(r & 15)) + (byte & 15);
                            f32x4 nan;
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                const bool not_finite = FP8 ? (lds_read<uint8_t>(at + e) & 0x7F) == 0x7F
                                                            : (lds_read<uint16_t>(at + 2 * e) & 0x7F80) == 0x7F80;
                                nan[e] = not_finite ? __builtin_nanf("") : 0.f;
                            }
#pragma unroll
                            for (int x = 0; x < NB; ++x)
                                if (key < limit(x)) acc[y][x] += nan;
                        }
                    }
                    lds_barrier();
                    for (int i = lane; i < G::ROWS * G::CH; i += 64)
                        if (key0 + G::ROWS * wave + i / G::CH >= least) {
                            const uint32_t at = st + wave * G::ROWS * G::RB + 16 * i;
                            if (any_nonfinite<FP8>(lds_read<u32x4>(at)))
                                for (int e = 0; e < 16; e += G::ES)
                                    if (FP8 ? (lds_read<uint8_t>(at + e) & 0x7F) == 0x7F : (lds_read<uint16_t>(at + e) & 0x7F80) == 0x7F80) {
                                        if constexpr (FP8) *reinterpret_cast<__attribute__((address_space(3))) uint8_t *>((lds_u8 *)(uintptr_t)(at + e)) = 0;
                                        else *reinterpret_cast<__attribute__((address_space(3))) uint16_t *>((lds_u8 *)(uintptr_t)(at + e)) = 0;
                                    }
                        }
                    lds_barrier();
                }

                // ---- O^T += C^T P^T ----------------------------------------------
                // C^T operand of output block y and keys 32 ks .. + 31
                const uint32_t vat = here(st + v0);
                auto read_v = [&](int i) {
                    const int ks = i / XB, y = i % XB;
                    if constexpr (FP8) {
                        const s32x2 t = __builtin_amdgcn_ds_read_tr8_b64_v2i32(
                            (__attribute__((address_space(3))) s32x2 *)(lds_u8 *)(uintptr_t)((vat ^ (16 * y)) + 32 * ks * G::RB));
                        return u32x2{(uint32_t)t.x, (uint32_t)t.y};
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
                auto value = [&](auto r) -> u32x4 {
                    if constexpr (FP8) return fp8x8_to_f16x8(r.x, r.y);
                    else return r;
                };
                constexpr int VG = WAVES == 4 ? 4 : 1;  // operands a group ahead
                decltype(read_v(0)) vb[2][VG];
                u32x4 pf[NB];
#pragma unroll
                for (int x = 0; x < NB; ++x) pf[x] = lds_read<u32x4>(pread0 + 2048 * x);
#pragma unroll
                for (int y = 0; y < VG; ++y) vb[0][y] = read_v(y);
#pragma unroll
                for (int i0 = 0; i0 < 2 * XB; i0 += VG) {
                    const int cur = (i0 / VG) & 1;
                    if (i0 == XB) {
#pragma unroll
                        for (int x = 0; x < NB; ++x) pf[x] = lds_read<u32x4>((pread0 ^ 64) + 2048 * x);
                    }
#pragma unroll
                    for (int y = 0; y < VG; ++y)
                        if (i0 + VG + y < 2 * XB) vb[cur ^ 1][y] = read_v(i0 + VG + y);
#pragma unroll
                    for (int y = 0; y < VG; ++y) {
                        const u32x4 v = value(vb[cur][y]);
#pragma unroll
                        for (int x = 0; x < NB; ++x) acc[(i0 + y) % XB][x] = mfma_pv<FP8>(v, pf[x], acc[(i0 + y) % XB][x]);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
            wait_vmcnt<0>();  // no copy is still landing when the ring is used again
        }

        // ---- row sums over the waves, rows out -------------------------------------
        const int ln = here(lane), n16 = ln & 15, j = ln >> 4;
        lds_barrier();
#pragma unroll
        for (int x = 0; x < NW; ++x) {
            l[x] += __shfl_xor(l[x], 16);
            l[x] += __shfl_xor(l[x], 32);
            if (j == 0) red[kw * 16 * NB + 16 * (NW * rw + x) + n16] = l[x];
        }
        lds_barrier();
        cLatent *A = arguments();
        const bool whole = tile == 0 && t1 == tiles;
        const int64_t slot = 2 * (int64_t)g + (pos == begin ? 0 : 1);
#pragma unroll
        for (int x = 0; x < NB; ++x) {
            float sum = 0.f;
#pragma unroll
            for (int w = 0; w < KW; ++w) sum += red[w * 16 * NB + 16 * x + n16];
            const float inv = sum == 0.f ? 0.f : vscale / sum;
            const float lse2 = sum == 0.f ? -INFINITY : refs[16 * x + n16] * sc + log2f(sum);
            bool ok;
            const int64_t qrow = row_of(x, n16, ok);
            if (whole && !ok) continue;
            const int64_t row = whole ? qrow : slot * A->pl.rows + 16 * (u * NB + x) + n16;
            const int64_t at = row * DC + wave * (DC / WAVES) + 4 * j;
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

template <int DC, bool FP8>
static hipError_t launch_nb(const Latent &a, hipStream_t st) {
    const dim3 grid((unsigned)(a.pl.workers * a.units));
    switch (a.nb) {
    case 1: hipLaunchKernelGGL((latent_mfma_kernel<DC, FP8, 1, 4>), grid, dim3(256), 0, st, a); break;
    case 2: hipLaunchKernelGGL((latent_mfma_kernel<DC, FP8, 2, 8>), grid, dim3(512), 0, st, a); break;
    case 3: hipLaunchKernelGGL((latent_mfma_kernel<DC, FP8, 3, 4>), grid, dim3(256), 0, st, a); break;
    case 4: hipLaunchKernelGGL((latent_mfma_kernel<DC, FP8, 4, 8>), grid, dim3(512), 0, st, a); break;
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
