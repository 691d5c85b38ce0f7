// Products of matrices on the matrix unit, C = A B^T and its transposed forms, with something at the end
// of each tile: the core that the loss at the head and the orthogonal update share.
//
// Two blocks on neighbouring SMs form a 256 x 256 tile: each copies and keeps 128 of its rows of A, 128 of its rows of
// B, and the sums of its 128 rows. (Where C has no more than 128 rows, blocks form 128 x 256 tiles alone, each with
// all rows of B.) One warp copies stages of 64 contraction indices by TMA, one issues the matrix instructions, eight
// bring the sums out of the tensor memory, whose other half the matrix unit fills meanwhile. An operand may lie in
// memory with its contraction index fast or slow (XMN); the tiles are swizzled by the copies either way, and nothing is
// transposed.
//
// Operands have 16 bits (bf16 or fp16), sums 32. An fp32 operand goes as three bf16 terms whose sum it is exactly
// ("planes" of a 3-D tensor map), and a product of two such as six passes, over some stages at a time, from the
// smallest terms to the largest, which alone the matrix unit's truncation reaches; the three that are left out are
// below 2^-24 of the largest.
//
// What bounds it. A stage of a pair takes 512 cycles of the matrix unit, which long products keep busy 90 % of the
// time: 4100 x 2048 over 65536 bf16 (2460 rows that count) in 440 us, 1500 TFLOP/s. Below some 50 tiles it is start and
// end: 3 us until the first sums, 1 to 4 to bring a tile out.
#pragma once

#include <cuda.h>

#include "tcgen05.cuh"
#include "train.cuh"

namespace ss {

constexpr int kProdTile = 256, kProdHalf = kProdTile / 2;  // of C, in both directions; a block's share
constexpr int kProdK = 64, kProdStages = 6;                // contraction indices of a stage; stages that shared memory has room for
constexpr uint32_t kProdOperand = kProdHalf * kProdK * 2, kProdStageBytes = 2 * kProdOperand;
constexpr uint32_t kProdPanel = kProdK * 128;              // 64 elements of an operand whose contraction index is slow
constexpr int kProdOut = 256, kProdThreads = kProdOut + 64;  // warps 0-7 bring out, 8 copies, 9 issues
constexpr uint32_t kProdSquare = 32 * 32 * 4;              // an outgoing warp's own shared memory
// Of a pair's block, and of a block alone, which has all 256 rows of B: stages and their bytes.
template <bool PAIR>
struct Stage {
    static constexpr int kCount = PAIR ? kProdStages : 4;
    static constexpr uint32_t kBytes = PAIR ? 2 * kProdOperand : 3 * kProdOperand;
    static constexpr size_t kSmem = 1024 + kCount * kBytes + kProdOut / 32 * kProdSquare;
};

constexpr int kTerms = 3, kMostPasses = 6;

struct Product {
    int m, n, k;      // C is m x n, summed over k
    int batches;      // matrices one after another (the maps' third coordinate), where passes is 1
    int passes;       // pairs of planes: (plane_a[i], plane_b[i])
    int8_t plane_a[kMostPasses], plane_b[kMostPasses];
    int block;        // with passes: stages that go through all of them before the next do
    int chunk;        // stages that are summed in tensor memory before they are brought out
    int tile_m;       // rows of a tile: 256 for pairs, 128 for blocks alone
    int pairs;        // of blocks, or blocks alone
    int split;        // whether the contraction of tiles that do not fill a round of pairs may be cut into parts
    int m_fast;       // the order of tiles: neighbours share columns of C, or rows
    int upper;        // m == n: only tiles on the diagonal and above
    int small;        // blocks that share a 128 x 128 tile (1, 2, 4), or 0: pairs on 256 x 256 tiles
    int ring;         // with small: stages under way, kSmallStages or kMostSmallStages
    int bf16;         // operands: bf16 or fp16
    int follows;      // another kernel of the call goes before
    const int* live;  // rows that there are (all of the call's), or NULL
    int live_from;    // the first of them that is meant here
    int live_side;    // 1: they are m; 2: they are k
    int always;       // C is formed where no row is live, too, from a stage of zeros, as it is for the call's first rows
};

inline Product product_of(int64_t m, int64_t n, int64_t k, bool terms, int sms) {
    Product p{};
    p.tile_m = kProdTile, p.pairs = sms / 2;
    p.m = static_cast<int>(m), p.n = static_cast<int>(n), p.k = static_cast<int>(k);
    p.batches = 1, p.passes = 1, p.block = 1 << 30, p.chunk = 1 << 30, p.bf16 = 1;
    if (terms) {
        const int8_t a[kMostPasses] = {0, 2, 1, 0, 1, 0}, b[kMostPasses] = {2, 0, 1, 1, 0, 0};
        p.passes = kMostPasses;
        for (int i = 0; i < kMostPasses; ++i) p.plane_a[i] = a[i], p.plane_b[i] = b[i];
    }
    return p;
}

// The pairs of blocks take whole tiles as long as every pair gets one; the contraction of the tiles that are left over (all, if
// there are fewer than pairs) is cut into parts, so that they too keep most pairs busy. Parts are joined afterwards, in their order.
// C of at most 128 rows: blocks alone.
inline void alone(Product& p, int sms) {
    if (p.m <= kProdHalf) p.tile_m = kProdHalf, p.pairs = sms;
}

struct Schedule {
    int m, tiles_m, tiles_n, per_batch;
    int pass_stages, stages;          // of one pass; of all
    int whole, parts, part_stages, units;
    int part_block;                   // a part has whole blocks of so many stages of each pass
};
constexpr int kLeastPart = 8;         // stages: fewer do not pay for their start and for joining them

__device__ __forceinline__ Schedule schedule_of(const Product& p) {
    Schedule s;
    int m = p.m, k = p.k;
    bool any = true;
    if (p.live != nullptr) {
        const int live = max(*p.live - p.live_from, 0);
        any = live > 0 || p.live_from == 0 || p.always;
        if (p.live_side == 1) m = min(m, live);
        else k = max(min(k, live), 1);
    }
    s.m = m;
    s.tiles_m = (m + p.tile_m - 1) / p.tile_m;
    s.tiles_n = (p.n + kProdTile - 1) / kProdTile;
    s.per_batch = p.upper ? s.tiles_m * (s.tiles_m + 1) / 2 : s.tiles_m * s.tiles_n;
    s.pass_stages = (k + kProdK - 1) / kProdK;
    s.stages = s.pass_stages * p.passes;
    const int tiles = any ? s.per_batch * p.batches : 0, others = tiles % p.pairs;
    s.whole = tiles, s.parts = 1, s.part_stages = s.stages, s.part_block = p.block;
    if (p.split && others > 0) {
        const int parts = min(p.pairs / others, s.stages / kLeastPart);
        if (parts > 1) {
            s.whole = tiles - others;
            s.part_stages = (s.stages + parts - 1) / parts;
            if (p.passes > 1) {
                // A part is made of whole blocks, so that it too begins with the smallest terms and ends with the largest: one that began in the
                // middle of a block added small terms to large sums, each a truncation (dx of 3000 x 64 over 3494 fp32 2.4e-6 off, now 0.9e-6).
                s.part_block = min(p.block, (s.part_stages + p.passes - 1) / p.passes);
                const int all = p.passes * s.part_block;
                s.part_stages = (s.part_stages + all - 1) / all * all;
            }
            s.parts = (s.stages + s.part_stages - 1) / s.part_stages;
        }
    }
    s.units = s.whole + (tiles - s.whole) * s.parts;
    return s;
}

struct ProdUnit {
    int batch, m0, n0;
    int part;           // of all parts, or -1: a whole tile
    int first, stages;
};

__device__ __forceinline__ ProdUnit prod_unit(const Product& p, const Schedule& s, int u) {
    ProdUnit r;
    r.part = -1, r.first = 0, r.stages = s.stages;
    if (u >= s.whole) {
        r.part = u - s.whole;
        const int other = r.part / s.parts;
        r.first = (r.part - other * s.parts) * s.part_stages;
        r.stages = min(s.part_stages, s.stages - r.first);
        u = s.whole + other;
    }
    r.batch = u / s.per_batch;
    int t = u - r.batch * s.per_batch, i, j;
    if (p.upper) {
        for (i = 0; t >= s.tiles_m - i; ++i) t -= s.tiles_m - i;
        j = i + t;
    } else if (p.m_fast) {
        j = t / s.tiles_m, i = t - j * s.tiles_m;
    } else {
        // tiles with fewer columns come last, spread over all pairs; in their places they could all fall to some
        const int full = p.n % kProdTile == 0 || s.tiles_n == 1 ? s.tiles_n : s.tiles_n - 1;
        if (t < s.tiles_m * full) i = t / full, j = t - i * full;
        else i = t - s.tiles_m * full, j = full;
    }
    r.m0 = i * p.tile_m, r.n0 = j * kProdTile;
    return r;
}

// Columns that are formed of a tile: those that C has, up to a multiple of 32 (of 16 for each block of a pair).
__device__ __forceinline__ int tile_cols(const Product& p, const ProdUnit& u) { return min(kProdTile, (p.n - u.n0 + 31) / 32 * 32); }

struct ProdShared {
    uint64_t full[kProdStages], added[2];  // of the first block: by both blocks
    uint64_t empty[kProdStages], summed[2], last;
    uint32_t tmem;
    int abort;
};

// 32 x 32 words, a row a lane, to the warp's own shared memory: 16-byte chunk c of row r at chunk c ^ (r & 7).
__device__ __forceinline__ void square_put(uint32_t buf, int lane, const uint32_t* v) {
    const uint32_t at = buf + lane * 128 + ((lane & 7) << 4);
#pragma unroll
    for (int i = 0; i < 8; ++i)
        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at ^ (i << 4)), "r"(v[4 * i]), "r"(v[4 * i + 1]),
                     "r"(v[4 * i + 2]), "r"(v[4 * i + 3]) : "memory");
}
// Words 4 chunk .. 4 chunk + 3 of row `row`.
__device__ __forceinline__ uint32_t square_at(uint32_t buf, int row, int chunk) { return buf + row * 128 + ((chunk ^ (row & 7)) << 4); }
__device__ __forceinline__ uint4 square_get(uint32_t buf, int row, int chunk) {
    uint4 v;
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(square_at(buf, row, chunk)) : "memory");
    return v;
}
__device__ __forceinline__ void square_set(uint32_t buf, int row, int chunk, uint4 v) {
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(square_at(buf, row, chunk)), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
__device__ __forceinline__ float square_word(uint32_t buf, int row, int col) {
    float v;
    asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v) : "r"(square_at(buf, row, col >> 2) + (col & 3) * 4) : "memory");
    return v;
}

// A lane takes four neighbouring columns of every fourth row of a square: row lane / 8 + 4 i, columns 4 (lane % 8) on.
__device__ __forceinline__ void square_sums(uint32_t buf, int lane, float4 (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint4 w = square_get(buf, (lane >> 3) + 4 * i, lane & 7);
        v[i] = make_float4(__uint_as_float(w.x), __uint_as_float(w.y), __uint_as_float(w.z), __uint_as_float(w.w));
    }
}

constexpr uint32_t kNanBits = 0x7FC00000u;

// EPI brings the sums out. With EPI::kWhole a thread holds 128 columns of a row, summed over all chunks in
// registers, and gets them at once: whole(unit, m, row, col, lane, buf, sums, what ahead(m, row, lane) loaded before they had come). Otherwise a warp has an EPI::Tile for its 32 rows and 128
// columns of a unit and gets each chunk in squares of 32 x 32 in its shared memory: fetch(column) before they have come,
// square(column, ..., its sums, first chunk?). With EPI::kPacks a tile may take 64 columns at a time, rounded to 16 bits:
// packed(column, ...). EPI::kBefore: before(...) is work for the outgoing warps while the first sums form. EPI::kAhead: registers allow two squares' fetches. EPI::kSmall: it also ends the small products below; EPI::kAlone: those of blocks alone.
// A wait that ran out (each is bounded) shows as NaN in place of all sums from there on. The copying warp then copies nothing more, an outgoing one
// says no more that it has brought sums out, and the issuing one, which goes on with what there is, does not say that sums have been formed: so none that are half done
// are taken for whole ones, in this block or the pair's other one. (The answer of each wait, asked before each stage's products, cost 2 to 10 %; and what is asked stands in an `if`
// of its own before that of the elected lane, which the compiler has to recognise to keep operands in uniform registers.)
template <class EPI, bool A_MN, bool B_MN, bool PAIR>
__global__ void __launch_bounds__(kProdThreads, 1)
product_kernel(const __grid_constant__ CUtensorMap a_map, const __grid_constant__ CUtensorMap b_map, const __grid_constant__ Product p,
               const __grid_constant__ EPI epi) {
    extern __shared__ uint8_t dynamic[];
    __shared__ ProdShared sh;
    const uint32_t stages = (smem_addr(dynamic) + 1023u) & ~1023u;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    constexpr int kStages = Stage<PAIR>::kCount;
    constexpr uint32_t kStageBytes = Stage<PAIR>::kBytes;
    const int pair = PAIR ? blockIdx.x >> 1 : blockIdx.x, pairs = p.pairs;
    volatile int* abort = &sh.abort;
    uint32_t rank = 0;  // in the pair; the first block issues the matrix instructions and waits for both blocks' operands
    if constexpr (PAIR) asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));

    next_may_begin();
    if (tid == 0) {
        for (int s = 0; s < kStages; ++s) {
            mbar_init(smem_addr(&sh.full[s]), 1);
            mbar_init(smem_addr(&sh.empty[s]), 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(smem_addr(&sh.summed[b]), 1);
            mbar_init(smem_addr(&sh.added[b]), (PAIR ? 2 : 1) * kProdOut / 32);
        }
        mbar_init(smem_addr(&sh.last), 1);
        sh.abort = 0;
        mbar_init_visible();
    }
    if (warp == 0) {
        if constexpr (PAIR) tmem_alloc_pair(smem_addr(&sh.tmem), 512);
        else tmem_alloc(smem_addr(&sh.tmem), 512);
    }
    tc_fence_before();
    __syncthreads();
    if constexpr (PAIR) cluster_sync();
    tc_fence_after();
    if (p.follows) after_previous();
    const uint32_t tmem = sh.tmem;
    const Schedule sc = schedule_of(p);

    if (warp < kProdOut / 32) {
        // ---- sums out: 32 rows and half of the columns to a warp
        const int row_local = rank * kProdHalf + (warp & 3) * 32, col_local = (warp >> 2) * kProdHalf;
        const uint32_t buf = stages + kStages * kStageBytes + warp * kProdSquare;
        const uint32_t tmem_at = tmem + (static_cast<uint32_t>((warp & 3) * 32) << 16) + col_local;
        const uint32_t added = PAIR ? cluster_addr(smem_addr(&sh.added[0]), 0) : smem_addr(&sh.added[0]);
        auto arrive = [](uint32_t bar) {
            if constexpr (PAIR) mbar_arrive_pair(bar);
            else mbar_arrive(bar);
        };
        uint32_t chunk = 0;
        bool ok = true;
        if constexpr (EPI::kBefore) epi.before(warp, lane);
        for (int unit = pair; unit < sc.units; unit += pairs) {
            const ProdUnit u = prod_unit(p, sc, unit);
            const int row = u.m0 + row_local, col = u.n0 + col_local;
            if constexpr (EPI::kWhole) {
                const auto ahead = epi.ahead(sc.m, row, lane);
                float sums[kProdHalf];
#pragma unroll
                for (int i = 0; i < kProdHalf; ++i) sums[i] = 0.0f;
                for (int left = u.stages; left > 0; left -= p.chunk, ++chunk) {
                    if (ok) ok = __all_sync(0xFFFFFFFFu, mbar_wait(smem_addr(&sh.summed[chunk & 1]), (chunk >> 1) & 1, abort));
                    tc_fence_after();
                    const uint32_t src = tmem_at + (chunk & 1) * kProdTile;
#pragma unroll
                    for (int j = 0; j < kProdHalf; j += 16) {
                        uint32_t r[16];
                        tmem_load16(src + j, r);
                        tmem_load_wait();
#pragma unroll
                        for (int i = 0; i < 16; ++i) sums[j + i] += __uint_as_float(r[i]);
                    }
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0 && ok) arrive(added + (chunk & 1) * 8);
                }
                if (!ok) {
#pragma unroll
                    for (int i = 0; i < kProdHalf; ++i) sums[i] = __uint_as_float(kNanBits);
                }
                epi.whole(u, sc.m, row, col, lane, buf, sums, ahead);
            } else {
                bool first = true;
                const bool any = row < sc.m && col < p.n;
                typename EPI::Tile tile(epi, u, sc.m, row, col, lane);
                typename EPI::Fetched f;
                [[maybe_unused]] typename EPI::Fetched g;
                for (int left = u.stages; left > 0; left -= p.chunk, ++chunk) {
                    if (any) tile.fetch(epi, 0, f);
                    if (ok) ok = __all_sync(0xFFFFFFFFu, mbar_wait(smem_addr(&sh.summed[chunk & 1]), (chunk >> 1) & 1, abort));
                    tc_fence_after();
                    const uint32_t src = tmem_at + (chunk & 1) * kProdTile;
                    bool done = !any;
                    if constexpr (EPI::kPacks) {
                        if (!done && tile.packs && ok) {
                            done = true;
#pragma unroll 1
                            for (int j = 0; j < kProdHalf; j += 64) {
#pragma unroll
                                for (int h = 0; h < 2; ++h) {
                                    uint32_t r[32];
                                    tmem_load32(src + j + 32 * h, r);
                                    tmem_load_wait();
#pragma unroll
                                    for (int i = 0; i < 4; ++i)
                                        square_set(buf, lane, 4 * h + i, make_uint4(tile.pack(r[8 * i], r[8 * i + 1]), tile.pack(r[8 * i + 2], r[8 * i + 3]),
                                                                                    tile.pack(r[8 * i + 4], r[8 * i + 5]), tile.pack(r[8 * i + 6], r[8 * i + 7])));
                                }
                                __syncwarp();
                                tile.packed(j, lane, buf);
                                __syncwarp();
                            }
                        }
                    }
                    auto square = [&](int j, typename EPI::Fetched& of) {
                        uint32_t r[32];
                        tmem_load32(src + j, r);
                        tmem_load_wait();
                        if (!ok) {
#pragma unroll
                            for (int i = 0; i < 32; ++i) r[i] = kNanBits;
                        }
                        square_put(buf, lane, r);
                        __syncwarp();
                        float4 v[8];
                        square_sums(buf, lane, v);
                        tile.square(epi, j, lane, buf, v, of, first);
                        __syncwarp();
                    };
                    if constexpr (EPI::kAhead) {
#pragma unroll 1
                        for (int j = 0; !done && j < kProdHalf && col + j < p.n; j += 64) {  // what the next square needs is on its way while one is worked on
                            const bool second = col + j + 32 < p.n, third = j + 64 < kProdHalf && col + j + 64 < p.n;
                            if (second) tile.fetch(epi, j + 32, g);
                            square(j, f);
                            if (!second) break;
                            if (third) tile.fetch(epi, j + 64, f);
                            square(j + 32, g);
                        }
                    } else {  // less code, all of which the first tile has to wait for
#pragma unroll 1
                        for (int j = 0; !done && j < kProdHalf && col + j < p.n; j += 32) {
                            if (j > 0) tile.fetch(epi, j, f);
                            square(j, f);
                        }
                    }
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0 && ok) arrive(added + (chunk & 1) * 8);
                    first = false;
                }
            }
        }
    } else if (warp == kProdOut / 32) {
        // Roles of one lane each, but the whole warp walks through them, so that addresses and descriptors are formed
        // in uniform registers.
        // ---- copies: this block's halves, counted by the first block's barrier
        const uint32_t full = PAIR ? cluster_addr(smem_addr(&sh.full[0]), 0) : smem_addr(&sh.full[0]), empty = smem_addr(&sh.empty[0]);
        auto load = [](uint32_t dst, const void* map, uint32_t bar, int x, int y, int z) {
            if constexpr (PAIR) tma_load_3d_pair(dst, map, bar, x, y, z);
            else tma_load_3d(dst, map, bar, x, y, z);
        };
        const bool leader = elect_one();
        bool go = true;
        int it = 0, slot = 0, issued = 0;
        uint32_t parity = 1;
        for (int unit = pair; unit < sc.units; unit += pairs) {
            const ProdUnit u = prod_unit(p, sc, unit);
            const int m0 = u.m0 + rank * kProdHalf, n0 = u.n0 + (PAIR ? rank * (tile_cols(p, u) / 2) : 0);  // PAIR: this block's half of both
            const bool wide = tile_cols(p, u) > kProdHalf;                                                  // more than one panel of a half, or more than a half
            const int block = u.part < 0 ? p.block : sc.part_block;
            int pass = 0, k0 = u.first * kProdK, begin = 0, end = 0x7FFFFFFF;  // of the block
            if (p.passes > 1) {
                k0 = begin = u.first / p.passes * kProdK;
                end = min(begin + block * kProdK, sc.pass_stages * kProdK);
            }
#pragma unroll 1
            for (int s = 0; s < u.stages; ++s) {
                go = __all_sync(0xFFFFFFFFu, mbar_wait_uniform(empty + slot * 8, parity, &sh.abort)) && go;
                const uint32_t bar = full + slot * 8, dst = stages + slot * kStageBytes;
                const int za = p.passes > 1 ? p.plane_a[pass] : u.batch, zb = p.passes > 1 ? p.plane_b[pass] : u.batch;
                if (go) if (leader) {
                    issued = it + 1;
                    const uint32_t less = wide ? 0 : (PAIR ? (B_MN ? kProdPanel : 0) : kProdOperand);  // not copied
                    if (rank == 0) mbar_expect(smem_addr(&sh.full[0]) + slot * 8, (PAIR ? 2 : 1) * (kStageBytes - less));
                    if constexpr (A_MN) {
                        load(dst, &a_map, bar, m0, k0, za);
                        load(dst + kProdPanel, &a_map, bar, m0 + 64, k0, za);
                    } else {
                        load(dst, &a_map, bar, k0, m0, za);
                    }
#pragma unroll
                    for (int h = 0; h < (PAIR ? 1 : 2); ++h) {
                        const uint32_t to = dst + (1 + h) * kProdOperand;
                        if (h == 1 && !wide) break;
                        if constexpr (B_MN) {
                            load(to, &b_map, bar, n0 + h * kProdHalf, k0, zb);
                            if (!PAIR || wide) load(to + kProdPanel, &b_map, bar, n0 + h * kProdHalf + 64, k0, zb);
                        } else {
                            load(to, &b_map, bar, k0, n0 + h * kProdHalf, zb);
                        }
                    }
                }
                ++it;
                k0 += kProdK;
                if (k0 == end) {
                    k0 = begin;
                    if (++pass == p.passes) pass = 0, k0 = begin = end, end = min(begin + block * kProdK, sc.pass_stages * kProdK);
                }
                if (++slot == kStages) slot = 0, parity ^= 1;
            }
        }
        // the last signals, and copies, arrive in this block's memory: not before that
        const int from = it > kStages ? it - kStages : 0;
        for (int i = from; i < it; ++i) mbar_wait_uniform(empty + i % kStages * 8, (i / kStages) & 1, &sh.abort);
        if (leader && *abort != 0 && rank == 0) {
            int own = 0;
            for (int i = issued > kStages ? issued - kStages : 0; i < issued; ++i) mbar_wait(smem_addr(&sh.full[i % kStages]), (i / kStages) & 1, &own);
        }
    } else if (rank == 0) {
        // ---- matrix unit
        constexpr uint32_t kStep = kStageBytes >> 4, kStepA = (A_MN ? 2048 : 32) >> 4, kStepB = (B_MN ? 2048 : 32) >> 4;
        const uint64_t desc_a = A_MN ? tc_desc_rows(stages, kProdPanel) : tc_desc_cols(stages);
        const uint64_t desc_b = B_MN ? tc_desc_rows(stages + kProdOperand, kProdPanel) : tc_desc_cols(stages + kProdOperand);
        const uint32_t full = smem_addr(&sh.full[0]), empty = smem_addr(&sh.empty[0]);
        const bool leader = elect_one();
        bool go = true;
        auto commit = [](uint32_t bar) {
            if constexpr (PAIR) tc_commit_pair(bar);
            else tc_commit(bar);
        };
        uint32_t slot = 0, parity = 0, chunk = 0;
        for (int unit = pair; unit < sc.units; unit += pairs) {
            const ProdUnit u = prod_unit(p, sc, unit);
            const uint32_t idesc = tc_idesc(PAIR ? kProdTile : kProdHalf, tile_cols(p, u), p.bf16 != 0, A_MN, B_MN);
            for (int left = u.stages; left > 0; left -= p.chunk, ++chunk) {
                const int n = min(left, p.chunk);
                const uint32_t d = tmem + (chunk & 1) * kProdTile;
                // the half of the tensor memory is free once the chunk before the last has been brought out
                if (chunk >= 2) go = __all_sync(0xFFFFFFFFu, mbar_wait_uniform(smem_addr(&sh.added[chunk & 1]), ((chunk >> 1) & 1) ^ 1, &sh.abort)) && go;
                if (!go) break;
                tc_fence_after();
#pragma unroll 1
                for (int s = 0; s < n; ++s) {
                    mbar_wait_uniform(full + slot * 8, parity, &sh.abort);
                    tc_fence_after();
                    const uint64_t da = desc_a + slot * kStep, db = desc_b + slot * kStep;
                    if (leader) {
#pragma unroll
                        for (int k = 0; k < kProdK / 16; ++k) {
                            if constexpr (PAIR) tc_mma_f16_pair(d, da + k * kStepA, db + k * kStepB, idesc, s != 0 || k != 0);
                            else tc_mma_f16(d, da + k * kStepA, db + k * kStepB, idesc, s != 0 || k != 0);
                        }
                        commit(empty + slot * 8);
                    }
                    __syncwarp();
                    if (++slot == kStages) slot = 0, parity ^= 1;
                }
                go = __all_sync(0xFFFFFFFFu, *abort == 0);
                if (go) if (leader) commit(smem_addr(&sh.summed[chunk & 1]));
                __syncwarp();
            }
        }
        // nothing may still be running when the tensor memory is given back
        int own = 0;
        if (leader) commit(smem_addr(&sh.last));
        mbar_wait(smem_addr(&sh.last), 0, &own);
    }
    // neither block leaves while the other may still signal to it or use its operands
    tc_fence_before();
    __syncthreads();
    if constexpr (PAIR) cluster_sync();
    tc_fence_after();
    if (warp == 0) {
        if constexpr (PAIR) tmem_free_pair(tmem, 512);
        else tmem_free(tmem, 512);
    }
}

// ---- small products --------------------------------------------------------------------------------
// Products that are too small to fill the machine with pairs: one 128 x 128 tile to a cluster of 1, 2 or 4 blocks that
// share the contraction. Each forms its part of the sums, keeps it in shared memory, and adds up its share of
// the tile's squares from all of them, in the order of their ranks, before it brings it out. With three stages under way
// two blocks fit on an SM. What bounds them is latency: of the 9.5 us of S of 1000 x 2048 (36 tiles, two blocks each) 2 are the
// wait for the kernel before, 0.6 the first copies, 3.5 the products, 1.2 the sums' way to the other block, 1.2 the end of the
// tile, 0.9 the wait for the other block.
constexpr int kSmallTile = 128, kSmallStages = 3, kMostSmallStages = 6, kSmallOut = 256, kSmallThreads = kSmallOut + 64;  // warps 0-7 bring out, 8 copies, 9 issues
static_assert(kSmallTile * kSmallTile * 4 <= kSmallStages * kProdStageBytes, "the sums take the place of the operands");

struct SmallShared {
    uint64_t full[kMostSmallStages], empty[kMostSmallStages], summed, last;
    uint32_t tmem;
    int abort;
};

template <class EPI, bool A_MN, bool B_MN>
__global__ void __launch_bounds__(kSmallThreads, EPI::kSmallBlocks)
small_product_kernel(const __grid_constant__ CUtensorMap a_map, const __grid_constant__ CUtensorMap b_map, const __grid_constant__ Product p,
                     const __grid_constant__ EPI epi) {
    extern __shared__ uint8_t dynamic[];
    __shared__ SmallShared sh;
    const uint32_t stages = (smem_addr(dynamic) + 1023u) & ~1023u;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int ring = p.ring, blocks = p.small, rank = blockIdx.x % blocks;
    volatile int* abort = &sh.abort;

    next_may_begin();
    ProdUnit u;
    {
        const int tiles_m = (p.m + kSmallTile - 1) / kSmallTile, tiles_n = (p.n + kSmallTile - 1) / kSmallTile;
        const int per_batch = p.upper ? tiles_m * (tiles_m + 1) / 2 : tiles_m * tiles_n, unit = blockIdx.x / blocks;
        u.part = -1, u.batch = unit / per_batch;
        int t = unit - u.batch * per_batch, i, j;
        if (p.upper) {
            for (i = 0; t >= tiles_m - i; ++i) t -= tiles_m - i;
            j = i + t;
        } else {
            j = t / tiles_m, i = t - j * tiles_m;
        }
        u.m0 = i * kSmallTile, u.n0 = j * kSmallTile;
        const int all = (p.k + kProdK - 1) / kProdK;
        u.first = all * rank / blocks, u.stages = all * (rank + 1) / blocks - u.first;
    }
    if (tid == 0) {
        for (int s = 0; s < ring; ++s) {
            mbar_init(smem_addr(&sh.full[s]), 1);
            mbar_init(smem_addr(&sh.empty[s]), 1);
        }
        mbar_init(smem_addr(&sh.summed), 1);
        mbar_init(smem_addr(&sh.last), 1);
        sh.abort = 0;
        mbar_init_visible();
    }
    if (warp == 0) tmem_alloc(smem_addr(&sh.tmem), kSmallTile);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (p.follows) after_previous();
    const uint32_t tmem = sh.tmem;

    if (warp < kSmallOut / 32) {
        // a warp has 32 rows and two squares of them; with two blocks each takes one of the two, with four each takes its own of all four
        const int quarter = warp & 3, j0 = (warp >> 2) * 2, row = u.m0 + quarter * 32;
        typename EPI::Tile tile(epi, u, p.m, row, u.n0, lane);
        typename EPI::Fetched f;
        auto mine = [&](int j) { return (blocks == 1 || (j & (blocks - 1)) == rank) && row < p.m && u.n0 + 32 * j < p.n; };
        auto square = [&](int j) { return stages + (4 * quarter + j) * kProdSquare; };
        const int fetched = mine(j0) ? j0 : (mine(j0 + 1) ? j0 + 1 : -1);
        if (fetched >= 0) tile.fetch(epi, 32 * fetched, f);
        const bool ok = __all_sync(0xFFFFFFFFu, mbar_wait(smem_addr(&sh.summed), 0, abort));
        tc_fence_after();
#pragma unroll 1
        for (int j = j0; j < j0 + 2; ++j) {
            if (blocks == 1 && !mine(j)) continue;
            uint32_t r[32];
            tmem_load32(tmem + (static_cast<uint32_t>(quarter * 32) << 16) + 32 * j, r);
            tmem_load_wait();
            if (!ok) {
#pragma unroll
                for (int i = 0; i < 32; ++i) r[i] = kNanBits;
            }
            square_put(square(j), lane, r);
        }
        tc_fence_before();
        __syncwarp();
        if (blocks > 1) cluster_sync();
#pragma unroll 1
        for (int j = j0; j < j0 + 2; ++j) {
            if (!mine(j)) continue;
            if (j != fetched) tile.fetch(epi, 32 * j, f);
            float4 v[8];
            if (blocks == 1) {
                square_sums(square(j), lane, v);
            } else {  // eight loads of a block under way at a time
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 1
                for (int q = 0; q < blocks; ++q) {
                    float4 x[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) x[i] = cluster_load4(cluster_addr(square_at(square(j), (lane >> 3) + 4 * i, lane & 7), q));
#pragma unroll
                    for (int i = 0; i < 8; ++i) v[i].x += x[i].x, v[i].y += x[i].y, v[i].z += x[i].z, v[i].w += x[i].w;
                }
                __syncwarp();
            }
            tile.square(epi, 32 * j, lane, square(j), v, f, true);
            __syncwarp();
        }
    } else {
        if (warp == kSmallOut / 32) {
            // ---- copies
            const bool leader = elect_one();
            bool go = true;
            int slot = 0, k0 = u.first * kProdK, issued = 0;
            uint32_t parity = 1;
#pragma unroll 1
            for (int s = 0; s < u.stages; ++s, k0 += kProdK) {
                go = __all_sync(0xFFFFFFFFu, mbar_wait_uniform(smem_addr(&sh.empty[0]) + slot * 8, parity, &sh.abort)) && go;
                const uint32_t bar = smem_addr(&sh.full[0]) + slot * 8, dst = stages + slot * kProdStageBytes;
                if (go) if (leader) {
                    issued = s + 1;
                    mbar_expect(bar, kProdStageBytes);
                    if constexpr (A_MN) {
                        tma_load_3d(dst, &a_map, bar, u.m0, k0, u.batch);
                        tma_load_3d(dst + kProdPanel, &a_map, bar, u.m0 + 64, k0, u.batch);
                    } else {
                        tma_load_3d(dst, &a_map, bar, k0, u.m0, u.batch);
                    }
                    if constexpr (B_MN) {
                        tma_load_3d(dst + kProdOperand, &b_map, bar, u.n0, k0, u.batch);
                        tma_load_3d(dst + kProdOperand + kProdPanel, &b_map, bar, u.n0 + 64, k0, u.batch);
                    } else {
                        tma_load_3d(dst + kProdOperand, &b_map, bar, k0, u.n0, u.batch);
                    }
                }
                __syncwarp();
                if (++slot == ring) slot = 0, parity ^= 1;
            }
            // A copy may still be under way only if a wait ran out: it has to arrive before the block ends.
            if (leader && *abort != 0) {
                int own = 0;
                for (int i = issued > ring ? issued - ring : 0; i < issued; ++i)
                    mbar_wait(smem_addr(&sh.full[i % ring]), (i / ring) & 1, &own);
            }
        } else {
            // ---- matrix unit
            const uint32_t idesc = tc_idesc(kSmallTile, kSmallTile, p.bf16 != 0, A_MN, B_MN);
            constexpr uint32_t kStep = kProdStageBytes >> 4, kStepA = (A_MN ? 2048 : 32) >> 4, kStepB = (B_MN ? 2048 : 32) >> 4;
            const uint64_t desc_a = A_MN ? tc_desc_rows(stages, kProdPanel) : tc_desc_cols(stages);
            const uint64_t desc_b = B_MN ? tc_desc_rows(stages + kProdOperand, kProdPanel) : tc_desc_cols(stages + kProdOperand);
            const bool leader = elect_one();
            uint32_t slot = 0, parity = 0;
#pragma unroll 1
            for (int s = 0; s < u.stages; ++s) {
                mbar_wait_uniform(smem_addr(&sh.full[0]) + slot * 8, parity, &sh.abort);
                tc_fence_after();
                const uint64_t da = desc_a + slot * kStep, db = desc_b + slot * kStep;
                if (leader) {
#pragma unroll
                    for (int k = 0; k < kProdK / 16; ++k) tc_mma_f16(tmem, da + k * kStepA, db + k * kStepB, idesc, s != 0 || k != 0);
                    tc_commit(smem_addr(&sh.empty[0]) + slot * 8);
                }
                __syncwarp();
                if (++slot == ring) slot = 0, parity ^= 1;
            }
            // nothing may still be running when its results are read, the operands' place is taken and the tensor memory given back
            const uint32_t end = smem_addr(__all_sync(0xFFFFFFFFu, *abort == 0) ? &sh.summed : &sh.last);
            if (leader) tc_commit(end);
            int own = 0;
            mbar_wait(end, 0, &own);
        }
        __syncwarp();
        if (blocks > 1) cluster_sync();
    }
    tc_fence_before();
    __syncthreads();
    if (blocks > 1) cluster_sync();  // the others may still be reading this block's sums
    tc_fence_after();
    if (warp == 0) tmem_free(tmem, kSmallTile);
}

// ---- host side -------------------------------------------------------------------------------------

// An operand's map: `fast` elements of unit stride, `slow` rows `row_bytes` apart, `planes` of them. mn: the contraction index is the slow one.
inline int map_operand(CUtensorMap* map, const void* p, bool bf16, int64_t fast, int64_t slow, int64_t row_bytes, int64_t planes, int64_t plane_bytes, bool mn) {
    cudaError_t e;
    const EncodeTiled encode = encode_tiled(&e);
    if (encode == nullptr) return cuda_status_public(e);
    const cuuint64_t dims[3] = {static_cast<cuuint64_t>(fast), static_cast<cuuint64_t>(slow), static_cast<cuuint64_t>(planes)};
    const cuuint64_t strides[2] = {static_cast<cuuint64_t>(row_bytes), static_cast<cuuint64_t>(planes > 1 ? plane_bytes : row_bytes)};
    const cuuint32_t box[3] = {64, static_cast<cuuint32_t>(mn ? kProdK : kProdHalf), 1}, ones[3] = {1, 1, 1};
    return encode(map, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, const_cast<void*>(p), dims, strides, box, ones,
                  CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                  CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS ? SS_OK : SS_ERR_UNSUPPORTED;
}

inline int64_t small_tiles(const Product& p) {
    const int64_t tm = (p.m + kSmallTile - 1) / kSmallTile, tn = (p.n + kSmallTile - 1) / kSmallTile;
    return (p.upper ? tm * (tm + 1) / 2 : tm * tn) * p.batches;
}

// How many blocks share a 128 x 128 tile, and how many stages each has under way; or pairs on 256 x 256 tiles: the least of an
// estimate in ns, fitted to products of 128 to 4096 rows and contractions of 128 to 4608. With six stages a block has an SM to itself
// and takes 200 ns for one; with three, two share an SM and wait for the L2 cache, the longer the more there are. (36 tiles over 32 stages: 19.1 us in pairs;
// 13.2, 12.6 and 12.9 with 1, 2 and 4 blocks of three stages, 11.9, 9.8 and 17.7 of six, as clusters of four do not find place on all
// SMs. 144 tiles over 16: 15.4, 13.7 with three stages, 9.3 with six. 136 tiles of 256 over 64: 52 in pairs, 90 with one block a tile.)
inline void choose_small(Product* p, int sms) {
    const int64_t tm = (p->m + kProdTile - 1) / kProdTile, tn = (p->n + kProdTile - 1) / kProdTile, stages = (p->k + kProdK - 1) / kProdK;
    const int64_t tiles = (p->upper ? tm * (tm + 1) / 2 : tm * tn) * p->batches, small = small_tiles(*p);
    const int64_t pair_rounds = (tiles + p->pairs - 1) / p->pairs, hidden = stages * 370 < 6000 ? 6000 - stages * 370 : 0;
    int64_t best = pair_rounds * stages * 370 + 8500 + (pair_rounds - 1) * hidden;
    p->small = 0, p->ring = 0;
    for (int c = 1; c <= 4 && c <= stages; c *= 2) {
        const int64_t all = small * c, share = (stages + c - 1) / c;
        const int64_t joined = 5500 + (c == 2 ? 800 : (c == 4 ? 2000 + 8 * all : 0));
        int64_t t;
        int ring = kMostSmallStages;
        if (all <= (c == 4 ? sms * 6 / 7 : sms)) {
            t = share * (200 + all / 4) + joined;
        } else {
            const int64_t at_once = all < 2 * sms ? all : 2 * sms, rounds = (all + 2 * sms - 1) / (2 * sms), wait = at_once * 9 / 4;
            ring = kSmallStages;
            t = rounds * share * (170 + (wait < 350 ? wait : 350)) + (rounds - 1) * 4000 + joined;
        }
        if (t < best) best = t, p->small = c, p->ring = ring;
    }
}

template <class EPI, bool A_MN, bool B_MN>
int launch_product(const CUtensorMap& a, const CUtensorMap& b, const Product& p, const EPI& epi, cudaStream_t st) {
    cudaLaunchConfig_t cfg{};
    cudaLaunchAttribute at[2] = {};
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = 2, at[0].val.clusterDim.y = 1, at[0].val.clusterDim.z = 1;
    at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = p.follows ? 2 : 1;
    cfg.stream = st;
    cudaError_t e = cudaSuccess;
    if constexpr (EPI::kSmall) {
        if (p.small > 0) {
            const auto kernel = small_product_kernel<EPI, A_MN, B_MN>;
            struct Key {};
            e = allow_shared<Key>(reinterpret_cast<const void*>(kernel), 1024 + kMostSmallStages * static_cast<int>(kProdStageBytes));
            if (e != cudaSuccess) return cuda_status_public(e);
            cfg.gridDim = dim3(static_cast<unsigned>(small_tiles(p) * p.small));
            cfg.blockDim = dim3(kSmallThreads);
            cfg.dynamicSmemBytes = 1024 + p.ring * kProdStageBytes;
            at[0].val.clusterDim.x = p.small;
            return cuda_status_public(cudaLaunchKernelEx(&cfg, kernel, a, b, p, epi));
        }
    }
    if constexpr (EPI::kAlone && !A_MN) {
        if (p.tile_m == kProdHalf) {
            const auto kernel = product_kernel<EPI, A_MN, B_MN, false>;
            struct Key {};
            e = allow_shared<Key>(reinterpret_cast<const void*>(kernel), static_cast<int>(Stage<false>::kSmem));
            if (e != cudaSuccess) return cuda_status_public(e);
            const int64_t units = static_cast<int64_t>((p.m + kProdHalf - 1) / kProdHalf) * ((p.n + kProdTile - 1) / kProdTile);
            cfg.gridDim = dim3(static_cast<unsigned>(units > p.pairs || p.split ? p.pairs : units));
            cfg.blockDim = dim3(kProdThreads);
            cfg.dynamicSmemBytes = Stage<false>::kSmem;
            at[0].val.clusterDim.x = 1;
            return cuda_status_public(cudaLaunchKernelEx(&cfg, kernel, a, b, p, epi));
        }
    }
    const auto kernel = product_kernel<EPI, A_MN, B_MN, true>;
    struct Key {};
    e = allow_shared<Key>(reinterpret_cast<const void*>(kernel), static_cast<int>(Stage<true>::kSmem));
    if (e != cudaSuccess) return cuda_status_public(e);
    const int64_t tm = (p.m + kProdTile - 1) / kProdTile, tn = (p.n + kProdTile - 1) / kProdTile;
    int64_t units = (p.upper ? tm * (tm + 1) / 2 : tm * tn) * p.batches;
    if (units > p.pairs || p.split) units = p.pairs;
    cfg.gridDim = dim3(static_cast<unsigned>(2 * units));
    cfg.blockDim = dim3(kProdThreads);
    cfg.dynamicSmemBytes = Stage<true>::kSmem;
    return cuda_status_public(cudaLaunchKernelEx(&cfg, kernel, a, b, p, epi));
}

}  // namespace ss
