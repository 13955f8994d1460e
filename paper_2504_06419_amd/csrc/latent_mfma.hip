// latent_mfma.hip -- attention over a latent cache on the 16-bit matrix
// instructions (gfx950).
//
// bf16 queries, bf16 or fp8 rows.  One workgroup of 8 waves per CU holds a unit of
// NB <= 8 blocks of 16 query rows and walks tiles of 16 KT keys, copied HBM -> LDS by
// the load-to-LDS instructions into a ring of stages.  A row is key and value at
// once, so one copy of it in LDS feeds both products:
//   S^T = K Q^T     waves 2 i and 2 i + 1 score all keys of the tile for row blocks
//                   2 i and 2 i + 1, each over half of the dimensions (every other 16-byte
//                   chunk group), queries in registers; they swap the halves that
//                   the other needs through LDS, and each owns one block's softmax;
//   O^T += C^T P^T  every wave takes an eighth of the latent's dimensions of all
//                   rows, C^T by transposing LDS reads, P through LDS.
// The products of a tile are a tile apart: after tile t + 1 is scored and the halves
// are swapped, a wave forms its probabilities and accumulates tile t, so that one
// wave of a SIMD feeds the matrix pipe while the other takes exponentials.
//
// Why this split.  A CU takes some 30 GB/s from L2, whether the lines are there or
// not (8 units of 64 rows that share their keys in L2: 2.4 us a tile of 64 keys
// without any arithmetic), so rows that share keys belong into one workgroup: 128
// rows are what its registers hold (128 accumulators and 72 queries of 256).
// A K operand read from LDS serves two row blocks: on a 32-key tile of 512 dimensions
// and 128 rows the workgroup makes 272 LDS accesses of 16 bytes a lane (144 of K, 32 of
// C, 64 of P, 32 of swapped halves; 8 cycles each, 2176) while a SIMD's two waves issue
// 136 matrix instructions (36 and 32 a wave; 16 cycles each, 2176).  With a wave per
// block and all dimensions it is 384 accesses (measured without copies: 2.4 us a tile).
//
// What bounds it: HBM up to 64 bf16 rows (64 sequences of 16384: 16 rows 6.5 TB/s, 64
// rows 5.5); at 128 rows the products and what stands between them, barriers,
// exponentials and exchanges, which two waves a SIMD overlap in part (128 heads, k =
// 3: 915 TFLOP/s of the 1135 of a large library product); with 16 fp8 rows the
// barriers of a tile (5.0 TB/s: without copies 154 of 176 us, without scores 136,
// without probabilities 157 on tiles of 32 keys); with few tiles a workgroup the start
// of a segment, which waits for the whole ring before its first scores.  An odd number
// of blocks leaves the last pair of waves one that is not there, scored all the same.
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
// waits are the kernel's own.  No register is written but m0, the LDS address.
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
// Probabilities are rounded to the values' operand type, as one matrix instruction takes
// both (bf16 rows: bf16, 8 bits; fp8 rows: fp16, 11 bits), their sum is not: the row sum
// and the log-sum-exp keep fp32. A second product for the rest of a probability would cost
// another matrix pass. fp16 holds a narrow range, so fp8 rows' probabilities are lifted to
// its upper end: 2^8 above the reference, the most that a lazy reference leaves, is 2^15,
// and what is lost begins at 2^-32 of the reference instead of 2^-25 (4096 keys of 2^-26
// behind a first key of 1 came out as 0).
template <bool FP8> constexpr float kLift = FP8 ? 7.f : 0.f;

// Registers that loads fill: has the compiler wait for them here.  Without it the
// wait stands at their first use in the tile loop and, taken every time round,
// also waits for the copies in flight.
template <int N> __device__ __forceinline__ void settle(u32x4 (&r)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) asm volatile("" : "+v"(r[i]));
}

// The kernel's arguments, read again from where it is called: what is used once per
// segment does not occupy scalar registers through the tile loop.
typedef const Latent __attribute__((address_space(4))) cLatent;
__device__ __forceinline__ cLatent *arguments() {
    uint64_t x = (uint64_t)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(x));
    return (cLatent *)x;
}

// Stage of one tile: [TILE][DC] rows, then [TILE][64] rotated parts.  16-byte chunk q of
// row r lies at q ^ fm(r) (main part, low 4 bits) and q ^ fr(r): operand reads (16
// rows, one chunk) and transposing reads (4 rows, 2 chunks) hit distinct banks.
template <int DC, bool FP8, int CW, int TILE_> struct LatStage {  // CW: waves that copy
    static constexpr int TILE = TILE_, KT = TILE / 16;  // 16-key blocks
    static constexpr int ES = FP8 ? 1 : 2;
    static constexpr int RB = DC * ES, RR = kLatentDr * ES;  // bytes of a row's parts
    static constexpr int MAIN = TILE * RB;
    static constexpr int BYTES = TILE * (RB + RR);
    static constexpr int CH = RB / 16, RCH = RR / 16;        // chunks of a row's parts
    static constexpr int ROWS = TILE / CW;                   // rows a copying wave takes
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
    // Waves without rows to score copy the tiles; with 7 and 8 blocks every wave does its share.
    constexpr int CW = NB <= 4 ? 4 : (NB <= 6 ? 2 : 8), TILE = latent_tile(true, DC * (FP8 ? 1 : 2), NB), SCAN = TILE / 8;  // copying waves; rows a wave looks through
    using G = LatStage<DC, FP8, CW, TILE>;
    // Streaming copies for up to 4 blocks: those are always a sequence's only unit, so its rows
    // are read once.  5 to 8 blocks can be one unit of several that share them through L2.
    constexpr bool NT = NB <= 4;
    constexpr int DK = DC + kLatentDr, KT = G::KT;
    constexpr int STEPS = DK / 32;      // QK steps of 32 dimensions
    constexpr int XB = DC / 128;        // 16-dimension output blocks of a wave
    constexpr int PB = NB * 16 * G::PR;
    constexpr int REST = 3 * PB + 2 * NB * 64 + 64;  // P twice, what the halves take beyond one of them
    // Queries (see below).  With 7 and 8 blocks of a 512-wide latent the registers run out: the
    // last group's queries lie in LDS, each lane's in a place of its own.
    constexpr int GROUPS = FP8 ? STEPS / 2 : STEPS, HG = (GROUPS + 1) / 2;  // 16-byte groups of a row, of a wave
    constexpr int QB = NB == 1 ? 1 : 2, QS = FP8 ? 2 : 1;                   // blocks, steps a group
    constexpr bool QL = DC == 512 && NB >= 7;
    constexpr int QR = QL ? HG - 1 : HG, QBYTES = QL ? 8 * QB * QS * 1024 : 0;
    constexpr int NS0 = (160 * 1024 - REST - QBYTES) / G::BYTES, NS = NS0 > 6 ? 6 : NS0;
    static_assert(NS >= 3, "stage ring too small");
    __shared__ __attribute__((aligned(1024))) uint8_t smem[NS * G::BYTES + REST + QBYTES];
    lds_u8 *ring = (lds_u8 *)smem;
    float *alphas = reinterpret_cast<float *>(smem + NS * G::BYTES + 3 * PB);  // [2][16 NB]; at the end sums, references
    int *flags = reinterpret_cast<int *>(smem + NS * G::BYTES + 3 * PB + 2 * NB * 64);  // [2][8]

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int half = wave & 1, cw = wave - (8 - CW);
    const bool copier = cw >= 0;
    const bool pair = wave < ((NB + 1) & ~1), owner = wave < NB;  // scores, owns row block `wave`
    const int n16 = lane & 15, j = lane >> 4;
    const Problem &p = a.p;
    const Plan &pl = a.pl;
    int g, u;
    latent_place(a, g, u);
    int64_t pos = 0, end = 0;
    int seg = 0, tile = 0;
    if (!latent_start<512>(a, g, u, reinterpret_cast<int32_t *>(smem), seg, tile, pos, end)) return;
    const int64_t begin = pos;
    float sc = p.sm_scale_log2, vscale = 1.f;
    if (FP8) {
        vscale = uload(p.kv.k_scale, 0);
        sc *= vscale;
    }
    const float margin = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(kRescaleLog2 / sc)));  // of raw scores

    // lane constants of the LDS accesses
    // (chunk 4 c + j of a row at 16 ((4 c + j) ^ f): only bits 4-7 of the address change with c & 3)
    const uint32_t ring0 = (uint32_t)(uintptr_t)ring;
    // a wave of a pair takes chunk groups c = 2 i + half
    const uint32_t kmain0 = ring0 + n16 * G::RB + ((16 * (j ^ fm(n16))) ^ (64 * half));
    const uint32_t krope0 = ring0 + G::MAIN + n16 * G::RR + ((16 * (j ^ fr<FP8>(n16))) ^ (FP8 ? 0 : 64 * half));
    // transposing reads: bf16: lane s of group j addresses key 8 j + 4 h + s / 4, 4 dimensions, and receives
    // dimension s of the group's 4 keys; fp8: key 8 j + s / 2, 8 dimensions, and receives dimension s of 8 keys
    const int vr = FP8 ? 8 * j + (n16 >> 1) : 8 * j + (n16 >> 2);
    const uint32_t v0 = ring0 + vr * G::RB + 16 * ((FP8 ? XB * wave : 2 * XB * wave + ((n16 >> 1) & 1)) ^ fm(vr & 15)) + 8 * (n16 & 1);
    const uint32_t p0 = ring0 + NS * G::BYTES + n16 * G::PR;
    const uint32_t pread0 = p0 + 16 * (j ^ fp<G::PR>(n16));
    const uint32_t pwrite0 = p0 + 16 * G::PR * wave + 16 * ((j >> 1) ^ fp<G::PR>(n16)) + 8 * (j & 1);
    // halves of a block's scores, 16 bytes a lane and 16 keys: in the block's P of the same tile, then behind both P
    const uint32_t x0 = ring0 + NS * G::BYTES + 16 * G::PR * wave;  // + 16 lane
    const uint32_t q0 = ring0 + NS * G::BYTES + REST + QB * QS * 1024 * wave;  // + 16 lane
    const uint32_t tok_bytes = (uint32_t)(p.kv.s_tok * G::ES);

    while (pos < end) {
        const int b = seg;
        const int n = effective_keys(p, b), tiles = latent_tiles<TILE>(n), span = tiles + pl.seg_cost;
        const int64_t left = end - pos;
        const int te = left < (int64_t)(span - tile) ? tile + (int)left : span;
        if (tile >= tiles) {  // phantom positions only
            pos += te - tile;
            ++seg;
            tile = 0;
            continue;
        }
        const int t1 = te < tiles ? te : tiles;
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
            // Copies of this wave's rows of a tile.  Where the rows lie in one run of storage,
            // the lanes hold the runs' addresses for 64 tiles, formed at once (a scalar load
            // per tile would hold up the LDS reads behind it).
            const int last = t1 - 1;
            uint64_t from = 0;
            uint32_t runs_lo = 0, runs_hi = 0;  // lane i: of tile held + i
            int rmax = G::ROWS - 1, held = -64;
            auto look_up = [&](int t) {
                if (t >= held + 64) {
                    held = t;
                    int key = (t + (int)here(lane)) * TILE + G::ROWS * cw;
                    key = key < n ? key : ((n - 1) & ~(G::ROWS - 1));
                    int64_t blk = b;
                    if (p.kv.page_size > 0) {
                        const uint32_t idx = (uint32_t)key / (uint32_t)p.kv.page_size;
                        const int page = p.kv.block_table[(int64_t)b * p.kv.max_blocks + idx];
                        blk = page < 0 ? 0 : (page >= p.kv.num_blocks ? p.kv.num_blocks - 1 : page);
                        key -= (int)idx * p.kv.page_size;
                    }
                    const uint64_t run = (uint64_t)(uintptr_t)p.kv.k + (uint64_t)((blk * p.kv.s_blk + (int64_t)key * p.kv.s_tok) * G::ES);
                    runs_lo = (uint32_t)run;
                    runs_hi = (uint32_t)(run >> 32);
                    asm volatile("" : "+v"(runs_lo), "+v"(runs_hi));  // the wait for the page ids stands here
                }
                from = (uint64_t)(uint32_t)__builtin_amdgcn_readlane(runs_lo, t - held) |
                       (uint64_t)(uint32_t)__builtin_amdgcn_readlane(runs_hi, t - held) << 32;
                if (p.kv.page_size == 0) {
                    int key = t * TILE + G::ROWS * cw;
                    key = key < n ? key : ((n - 1) & ~(G::ROWS - 1));
                    rmax = p.kv.capacity - 1 - key;  // >= 0: key < n <= capacity
                }
            };
            const int r0 = (G::ROWS * cw) & 15;
            auto copy = [&](int st, int x) {  // copy x of ML + RL into stage st
                const uint32_t lane = here(tid & 63);
                const bool main = x < G::ML;
                const int y = main ? x : x - G::ML, ch = main ? G::CH : G::RCH;
                const int r = y * (64 / ch) + (ch < 64 ? (int)(lane / ch) : 0);
                const uint32_t chunk = lane % ch ^ (main ? fm(r0 + r) : fr<FP8>(r0 + r));
                const uint32_t off = (uint32_t)(r < rmax ? r : rmax) * tok_bytes + (main ? 0 : G::RB) + 16 * chunk;
                const uint32_t at = ring0 + st * G::BYTES + 1024 * y +
                                    (main ? cw * G::ROWS * G::RB : G::MAIN + cw * G::ROWS * G::RR);
                if (main || G::ROWS * G::RCH >= 64 || r < G::ROWS) copy16_s<NT>(from, off, at);
            };
            auto copy_all = [&](int st) {
#pragma unroll
                for (int x = 0; x < G::LOADS; ++x) copy(st, x);
            };
            // any page size: lane r holds the address of row r
            auto copy_scattered = [&](int st, int t) {
                const int lane = here(tid & 63);
                int key = t * TILE + G::ROWS * cw + (lane & (G::ROWS - 1));
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
                    copy16_v<false>(__shfl(addr, r) + 16u * q16, at + cw * G::ROWS * G::RB + x * 1024);
                }
#pragma unroll 1
                for (int x = 0; x < G::RL; ++x) {
                    const int r = x * (64 / G::RCH) + lane / G::RCH, q16 = (lane % G::RCH) ^ fr<FP8>(r0 + r);
                    const uint64_t src = __shfl(addr, r) + G::RB + 16u * q16;
                    if (r < G::ROWS) copy16_v<false>(src, at + G::MAIN + cw * G::ROWS * G::RR + x * 1024);
                }
            };
            auto issue = [&](int st, int t) {
                if (a.uniform) copy_all(st);
                else copy_scattered(st, t);
            };

            if (copier) {
                for (int s = 0; s < NS - 1 && tile + s <= last; ++s) {
                    if (a.uniform) look_up(tile + s);
                    issue(s, tile + s);
                }
            }
            // queries of the wave's own block and of its partner's: group c of bf16 rows is dimensions
            // 32 c + 8 j .. + 7; of fp8 rows, whose 16-byte chunk feeds two steps, 64 c + 16 j .. + 15
            u32x4 q[QB][QR * QS];
            if (pair) {
                const int ln = here(lane);
#pragma unroll
                for (int x = 0; x < QB; ++x) {
                    bool ok;
                    const int block = NB == 1 ? 0 : wave ^ x;
                    const uint8_t *row = arguments()->p.q + row_of(block < NB ? block : 0, ln & 15, ok) * (DK * 2) + (FP8 ? 32 : 16) * (ln >> 4);
#pragma unroll
                    for (int i = 0; i < HG; ++i)
#pragma unroll
                        for (int z = 0; z < QS; ++z) {
                            const int c = 2 * i + half;
                            u32x4 v = u32x4{0, 0, 0, 0};
                            if (2 * i + 1 < GROUPS || half == 0)
                                v = *reinterpret_cast<const u32x4 *>(row + (FP8 ? 128 : 64) * c + 16 * z);
                            if (i < QR) q[x][i * QS + z] = v;
                            else *reinterpret_cast<lds_u32x4 *>((lds_u8 *)(uintptr_t)(q0 + 1024 * (x * QS + z) + 16 * ln)) = v;
                        }
                }
            }

#pragma unroll
            for (int x = 0; x < QB; ++x) settle(q[x]);

            // ---- half scores of tile t (stage st), the partner's sent to it -----------
            // `more`: the copies of tile `next` go out between the products (from the waves
            // that score: issued in a row they would stand in the way).
            f32x4 s[QB][KT];
            auto score = [&](int st, int buf, bool more, int into) {
                if (CW < 8 && copier) {
                    if (more) copy_all(into);
                    return;
                }
                if (!pair) return;
                const uint32_t kmain = here(kmain0 + st * G::BYTES), krope = here(krope0 + st * G::BYTES);
#pragma unroll
                for (int x = 0; x < QB; ++x)
#pragma unroll
                    for (int y = 0; y < KT; ++y) s[x][y] = f32x4{0.f, 0.f, 0.f, 0.f};
                // K operands a group of reads ahead of the products
                constexpr int MG = FP8 ? DC / 64 : DC / 32;  // groups of the main part
                auto read_k = [&](int i, int y) {
                    return lds_read<u32x4>(2 * i < MG ? (kmain ^ (128 * (i & 1))) + 256 * (i >> 1) + 16 * y * G::RB : krope + 16 * y * G::RR);
                };
                u32x4 kb[2][KT];
#pragma unroll
                for (int y = 0; y < KT; ++y) kb[0][y] = read_k(0, y);
#pragma unroll
                for (int i = 0; i < HG; ++i) {
                    if (i + 1 < HG) {
#pragma unroll
                        for (int y = 0; y < KT; ++y) kb[(i + 1) & 1][y] = read_k(i + 1, y);
                    }
#pragma unroll
                    for (int y = 0; y < KT; ++y) {
                        const u32x4 r = kb[i & 1][y];
                        auto query = [&](int x, int z) {
                            return i < QR ? q[x][i * QS + z] : lds_read<u32x4>(q0 + 1024 * (x * QS + z) + 16 * here(lane));
                        };
                        if constexpr (FP8) {
                            const u32x4 lo = fp8x8_to_bf16x8(r.x, r.y), hi = fp8x8_to_bf16x8(r.z, r.w);
#pragma unroll
                            for (int x = 0; x < QB; ++x) {
                                s[x][y] = mfma_bf16(lo, query(x, 0), s[x][y]);
                                s[x][y] = mfma_bf16(hi, query(x, 1), s[x][y]);
                            }
                        } else {
#pragma unroll
                            for (int x = 0; x < QB; ++x) s[x][y] = mfma_bf16(r, query(x, 0), s[x][y]);
                        }
                    }
                    if (CW == 8 && more) {
#pragma unroll
                        for (int x = 0; x < G::LOADS; ++x)
                            if (x * HG / G::LOADS == i) copy(into, x);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
                if (NB % 2 == 0 || (wave ^ 1) < NB) {
                    const uint32_t at = x0 + (half ? -16 * G::PR : 16 * G::PR) + 16 * here(lane);  // the partner's block
#pragma unroll
                    for (int y = 0; y < KT; ++y)
                        *reinterpret_cast<__attribute__((address_space(3))) f32x4 *>(
                            (lds_u8 *)(uintptr_t)(at + (y < KT / 2 ? buf * PB + 1024 * y : 2 * PB + 1024 * (y - KT / 2)))) = s[QB - 1][y];
                } else if (NB > 1) {
                    // The partner's scores are not used: nothing reads them, and the compiler does not
                    // count the wait states (8) before their registers are written again on this way.
                    asm volatile("s_nop 7" ::: "memory");
                }
            };

            // ---- probabilities of tile t (stage st) into buffer `buf` ----------------
            auto weigh = [&](int t, int st, int buf) {
                const int key0 = t * TILE;
                const bool tail = key0 + TILE > least;
                // A hidden key's probability is 0, which clears any finite value; what is not
                // finite in this wave's rows from the first hidden key on is looked for.
                bool bad = false;
                if (tail) {
                    const int lane = here(tid & 63);
                    for (int i = lane; i < SCAN * G::CH; i += 64)
                        if (key0 + SCAN * wave + i / G::CH >= least)
                            bad |= any_nonfinite<FP8>(lds_read<u32x4>(ring0 + st * G::BYTES + wave * SCAN * G::RB + 16 * i));
                }
                int word = __any(bad) ? 2 : 0;
                if (owner) {
                    const uint32_t at = x0 + 16 * here(lane);
#pragma unroll
                    for (int y = 0; y < KT; ++y)
                        s[0][y] += lds_read<f32x4>(at + (y < KT / 2 ? buf * PB + 1024 * y : 2 * PB + 1024 * (y - KT / 2)));
                    if (tail) {
                        const int key = key0 + 4 * (here(lane) >> 4);
#pragma unroll
                        for (int y = 0; y < KT; ++y)
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                if (key + 16 * y + e >= lim) s[0][y][e] = -INFINITY;
                    }
                    // lazy references: a row's moves when a score passes it by more than 2^8
                    // (NaN-propagating maximum: a NaN score never passes)
                    float top = s[0][0][0];
#pragma unroll
                    for (int y = 0; y < KT; ++y) top = max3n(max3n(top, s[0][y][0], s[0][y][1]), s[0][y][2], s[0][y][3]);
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
                        for (int z = 0; z < 4; ++z) e[z] = fast_exp2(fmaf(s[0][y][z] - msub, sc, kLift<FP8>));
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
            score(0, 0, false, 0);
            lds_barrier();
            weigh(tile, 0, 0);
            int rd = 0, buf = 0, wr = NS - 1;
            for (int tt = tile; tt <= last; ++tt) {
                landed(tt + 1);
                lds_barrier();  // tile tt + 1 and the probabilities of tt are there, tile tt - 1 is read
                const bool more = tt + NS - 1 <= last;
                if (copier && more) {
                    if (a.uniform) look_up(tt + NS - 1);
                    else copy_scattered(wr, tt + NS - 1);
                }
                const int into = wr;
                wr = wr + 1 == NS ? 0 : wr + 1;
                const int st = rd, key0 = tt * TILE;
                rd = rd + 1 == NS ? 0 : rd + 1;
                if (tt < last) {
                    score(rd, buf ^ 1, more && a.uniform, into);
                    lds_barrier();  // the halves are there
                }
                int word = 0;
                {
                    const int4 f0 = *reinterpret_cast<const int4 *>(flags + 8 * buf), f1 = *reinterpret_cast<const int4 *>(flags + 8 * buf + 4);
                    word = f0.x | f0.y | f0.z | f0.w | f1.x | f1.y | f1.z | f1.w;
                }
                if (tt < last) weigh(tt + 1, rd, buf ^ 1);
                const int events = __builtin_amdgcn_readfirstlane(word);

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
                        for (int i = lane; i < SCAN * G::CH; i += 64)
                            if (key0 + SCAN * wave + i / G::CH >= least) {
                                const uint32_t at = sb + wave * SCAN * G::RB + 16 * i;
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
                        const float alpha = flags[8 * buf + x] & 1 ? alphas[buf * 16 * NB + 16 * x + (lane & 15)] : 1.f;  // the reference moved
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
        if (owner && j == 0) {
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
            const float lse2 = sum == 0.f ? -INFINITY : alphas[16 * NB + 16 * x + n16] * sc + (log2f(sum) - kLift<FP8>);
            // an empty row is zero, also where infinite values behind no weight have made its sums NaN
            const bool empty = whole && sum == 0.f;
            auto value = [&](int y, int x) {
                f32x4 v = acc[y][x] * inv;
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = empty ? 0.f : v[e];
                return v;
            };
            bool ok;
            const int64_t qrow = row_of(x, n16, ok);
            if (whole && !ok) continue;
            const int64_t row = whole ? qrow : slot * A->pl.rows + 16 * (u * NB + x) + n16;
            const int64_t at = row * DC + wave * (DC / 8) + 4 * j;
            if (whole && A->p.out_dtype == SPIRE_BF16) {
                uint16_t *o = static_cast<uint16_t *>(A->p.out) + at;
#pragma unroll
                for (int y = 0; y < XB; ++y) {
                    const f32x4 v = value(y, x);
                    *reinterpret_cast<u32x2 *>(o + 16 * y) = u32x2{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
                }
            } else {
                float *o = (whole ? static_cast<float *>(A->p.out) : A->pl.part_o) + at;
#pragma unroll
                for (int y = 0; y < XB; ++y) *reinterpret_cast<f32x4 *>(o + 16 * y) = value(y, x);
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
