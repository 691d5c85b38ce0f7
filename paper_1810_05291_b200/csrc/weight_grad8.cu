// Weight gradient of a linear layer from its input kept in 8 bits: dW[n, k] (+)= sum_t dY[t, n] x^[t, k].
//
// The contraction runs over the rows t, so both operands lie in memory with the contraction index
// slow, and go to the matrix unit that way, without a transpose: tiles of dY by TMA, tiles of x^
// decoded by sixteen warps from the 8-bit codes straight into the swizzled operand layout. A decoded
// value has 7 significant bits and is exact in bf16; no operand is rounded. An fp32 dY goes as three
// bf16 terms whose sum it is exactly, one after another over all rows.
//
// Sums. The matrix unit adds into fp32 with truncation: of a product with inputs of mean 0 over 16384
// rows that it sums alone, 1.9e-5 is lost. So a tile is summed there over 2048 rows
// at a time, in one half of the tensor memory, and added to dW, rounded to nearest, while the matrix unit fills the
// other half: 4.5e-7 (512 rows: 1.3e-7, 1024: 2.1e-7; an fp32 product of the same: 5.1e-7).
//
// What bounds it. A launch of 16384 x 4096 x 4096 bf16 alone takes 407 to 423 us (1300 to 1350 TFLOP/s; a library product of the same
// sizes whose operands are both bf16 in memory 330 to 353), of 16384 x 2048 x 9472 444 to 463 us (1370 to 1430). In a row of calls the
// power limit lowers the clock: 465 us after 160 of them and 510 after 800 (1080 TFLOP/s; the library product 363 and 402). Shared
// memory is busy 87 % of the time and the matrix unit 76 %: for 64 rows a block copies in 24 KB, reads 8 KB of codes, writes 16 KB of operand and
// feeds 32 to 48 KB to the matrix unit, 640 to 750 cycles at 128 bytes, where the products take 512 and a stage 725.
// 4099 x 1000 x 2050 fp32 takes 73 us, of them 7 to split dY and 5 to join the parts. The three terms of 32 rows in
// one stage, decoded once, took 66 us, but the small terms, added to the large one's sums, each cost a truncation:
// 2.0e-6 instead of 5e-7, and at 352 rows a chunk, where it is 1.1e-6 like the plain form's, 73 us again.
#include "act8.cuh"
#include "tcgen05.cuh"

namespace ss {
namespace {

// Two blocks on neighbouring SMs share a 256 x 256 tile: each copies and keeps 128 of its columns
// of dY and its sums, and decodes 128 of its columns of x^ for both. Against one block for a 128 x
// 256 tile that halves the decoding and takes a third off the shared memory's traffic.
constexpr int kTileN = 256, kTileK = 256;  // of dW: n from dY, k from x^
constexpr int kBlockN = kTileN / 2, kBlockK = kTileK / 2;
constexpr int kRows = 64;                  // rows of a stage
constexpr int kStages = 5;                 // what shared memory has room for
constexpr int kCodeSlots = 6;              // stages of codes, ahead of the decoding
static_assert(kCodeSlots > kStages, "see the waits of the decoding warps");
constexpr int kChunk = 32;                 // stages summed in the matrix unit
// Stages of a part, at least: fewer do not pay for their start and for joining them. (1200 x 256 x 256 and 2048 x 512 x 512
// bf16: 14.4 us with 8; with 16 of them 16.4 and 16.5; with 4 the same.)
constexpr int kLeastPart = 8;
// Warps 0-3 bring the sums out, 4-19 decode, 20 and 22 copy, 21 issues the matrix instructions (23 is idle).
constexpr int kAdders = 128, kDecoders = 512, kThreads = kAdders + kDecoders + 128;
constexpr int kGroups = kDecoders / 128;   // a stage is decoded by four warps
constexpr uint32_t kPanel = kRows * 128;   // bytes of 64 columns of a stage
constexpr uint32_t kBytesA = kBlockN / 64 * kPanel, kBytesB = kBlockK / 64 * kPanel, kStageBytes = kBytesA + kBytesB;
constexpr uint32_t kCodeBytes = kRows * kBlockK;
constexpr uint32_t kSquareBytes = 32 * 32 * 4;  // an adding warp's way out
constexpr size_t kSmem = 1024 + kStages * kStageBytes + kCodeSlots * kCodeBytes + kAdders / 32 * kSquareBytes;

struct Plan {
    int tiles_n, tiles_k;   // tiles of dW; tile i: n index i % tiles_n
    int planes;             // bf16 terms of dY: 1, or 3 for fp32
    int stages_per_plane;   // stages of one plane
    int whole;              // tiles formed by one pair of blocks from all rows
    int parts;              // parts that each of the other tiles' rows are split in
    int part_stages;
    int units;              // whole + others * parts
};

struct WeightGrad {
    Ckpt x;
    float* dw;
    float* partial;  // one tile for each part
    int64_t dw_stride, rows, n_out, n_in;
    int accumulate, follows;  // follows: stage_dy_kernel goes before
    Plan plan;
};

struct Unit {
    int tile, first, stages;
    bool whole;
};

__device__ __forceinline__ Unit unit_of(const Plan& p, int u) {
    if (u < p.whole) return Unit{u, 0, p.planes * p.stages_per_plane, true};
    const int v = u - p.whole, part = v % p.parts, all = p.planes * p.stages_per_plane;
    const int first = part * p.part_stages;
    return Unit{p.whole + v / p.parts, first, min(p.part_stages, all - first), p.parts == 1};
}

struct Shared {
    uint64_t full[kStages], added[2];  // of the first block: by both blocks
    uint64_t empty[kStages], summed[2], last;
    uint64_t codes[kCodeSlots], taken[kCodeSlots];
    uint32_t tmem;
    int abort;
};

// A stage is decoded by one group of four warps, the next stage by the next of four groups, so that a group has four
// stages' time (it takes 1600 cycles; with eight decoding warps beside eight adding ones the product took 446 us instead of 411). Its codes come by a
// copy into a ring of their own, in rows of 128 bytes whose 16-byte chunks are swizzled like the
// operand's. (Loads to registers a stage ahead, which is all that fits, came too late: a stage took
// 1300 cycles to decode, twice what its products take.) A thread takes 16 columns of rows
// 16 apart (four, or two). Four lanes take 64 columns of a row t, the next four those of row t ^ 5: so eight lanes
// of a load (four neighbouring chunks c at c ^ (t & 7)) and of a store (every second chunk) cover all banks.
__device__ __forceinline__ int share_row(int tid) {
    const int t = 2 * ((tid >> 4) & 7);
    return (tid & 4) ? t ^ 5 : t;
}
__device__ __forceinline__ int share_panel(int tid) { return (tid >> 3) & 1; }
__device__ __forceinline__ int share_piece(int tid) { return tid & 3; }

// The exponents of a group's stages, of all units of this pair, in order. For rows and columns that
// do not exist others stand in: dY has zeros for such rows, and such columns of dW are not stored.
// (A marked group may stand in for a row: its column is NaN anyhow.)
struct Exponents {
    uint32_t e[4];
};

struct Walk {
    int unit, s, n;  // the next stage is the s-th of the unit's n
    int at;          // stage of its plane
    uint32_t group;  // of columns

    __device__ __forceinline__ void enter(const WeightGrad& a, uint32_t rank, int tid) {
        if (unit >= a.plan.units) return;
        const Unit u = unit_of(a.plan, unit);
        n = u.stages;
        at = (u.first + s) % a.plan.stages_per_plane;
        group = (u.tile / a.plan.tiles_n * kTileK + rank * kBlockK + 64 * share_panel(tid) + 16 * share_piece(tid)) >> 5;
        if (group >= a.x.groups) group = 0;
    }
    __device__ __forceinline__ void skip_units(const WeightGrad& a, int step, uint32_t rank, int tid) {
        while (unit < a.plan.units && s >= n) {
            s -= n;
            unit += step;
            enter(a, rank, tid);
        }
    }
    __device__ __forceinline__ void start(const WeightGrad& a, int first_unit, int first, int step, uint32_t rank, int tid) {
        unit = first_unit, s = first, n = 0;
        enter(a, rank, tid);
        skip_units(a, step, rank, tid);
    }
    __device__ __forceinline__ void load(const WeightGrad& a, int step, uint32_t rank, int tid, Exponents* x) {
        if (unit >= a.plan.units) return;
        const int last = static_cast<int>(a.rows) - 1, t = at * kRows + share_row(tid);
#pragma unroll
        for (int i = 0; i < 4; ++i) x->e[i] = a.x.exps[min(t + 16 * i, last) * a.x.groups + group];
        s += kGroups;
        for (at += kGroups; at >= a.plan.stages_per_plane;) at -= a.plan.stages_per_plane;  // the next plane goes over the same codes again
        skip_units(a, step, rank, tid);
    }
};

__device__ __forceinline__ void load_codes(uint32_t codes, int tid, uint4 (&q)[4]) {
    const int t = share_row(tid);
    const uint32_t at = codes + t * 128 + (((4 * share_panel(tid) + share_piece(tid)) ^ (t & 7)) << 4);
#pragma unroll
    for (int i = 0; i < 4; ++i)
        asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(q[i].x), "=r"(q[i].y), "=r"(q[i].z), "=r"(q[i].w) : "r"(at + i * 16 * 128) : "memory");
}

// To the stage's operand: column chunk c (8 columns, 16 bytes) of row t of a panel sits at chunk c ^ (t & 7).
__device__ __forceinline__ void store_codes(uint32_t stage_b, int tid, const uint4 (&q)[4], const Exponents& x) {
    const int t = share_row(tid);
    const uint32_t at = stage_b + share_panel(tid) * kPanel + t * 128, chunk = 2 * share_piece(tid);
    const uint32_t to[2] = {at + ((chunk ^ (t & 7)) << 4), at + (((chunk + 1) ^ (t & 7)) << 4)};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t e2 = act8_exponent_pair(x.e[i]);
        const uint32_t w[4] = {q[i].x, q[i].y, q[i].z, q[i].w};
#pragma unroll
        for (int h = 0; h < 2; ++h)
            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(to[h] + i * 16 * 128),
                         "r"(act8_value_pair<0>(w[2 * h], e2)), "r"(act8_value_pair<1>(w[2 * h], e2)),
                         "r"(act8_value_pair<0>(w[2 * h + 1], e2)), "r"(act8_value_pair<1>(w[2 * h + 1], e2)) : "memory");
    }
}

// Where 32 rows of a tile go: dW, or the part's own tile.
struct Dest {
    float* p;
    int64_t stride;
    int rows, cols;  // that exist, from p on
    bool add;
};

__device__ __forceinline__ Dest dest_of(const WeightGrad& a, int unit, int n_local, int k_local) {
    const Unit u = unit_of(a.plan, unit);
    if (!u.whole) {
        float* t = a.partial + static_cast<int64_t>(unit - a.plan.whole) * kTileN * kTileK;
        return Dest{t + n_local * kTileK + k_local, kTileK, kTileN - n_local, kTileK - k_local, false};
    }
    const int64_t n = static_cast<int64_t>(u.tile % a.plan.tiles_n) * kTileN + n_local;
    const int64_t k = static_cast<int64_t>(u.tile / a.plan.tiles_n) * kTileK + k_local;
    return Dest{a.dw + n * a.dw_stride + k, a.dw_stride, static_cast<int>(min(a.n_out - n, static_cast<int64_t>(kTileN))),
                static_cast<int>(min(a.n_in - k, static_cast<int64_t>(kTileK))), a.accumulate != 0};
}

// 32 x 32 sums, a row a lane, through the warp's own shared memory so that each row is written by
// neighbouring lanes. 16-byte chunk c of row r is kept at chunk c ^ (r & 7).
__device__ __forceinline__ void stage_square(uint32_t buf, int lane, const uint32_t* v) {
    const uint32_t at = buf + lane * 128 + ((lane & 7) << 4);
#pragma unroll
    for (int i = 0; i < 8; ++i)
        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at ^ (i << 4)), "r"(v[4 * i]), "r"(v[4 * i + 1]),
                     "r"(v[4 * i + 2]), "r"(v[4 * i + 3]) : "memory");
}

// Written, or (`add`) added by the memory itself: nothing is read back, and as the same lane writes
// an element of the tile each time, its sums come in their order. `row`: the lane's first row of the
// fast form, at its chunk; `step`: bytes of four rows.
__device__ __forceinline__ void store_square(uint32_t buf, int lane, const Dest& d, int col, bool add, bool vectors, char* row, int64_t step) {
    if (vectors && col + 32 <= d.cols) {
        const int first = lane >> 3;
        const uint32_t at = buf + first * 128 + (((lane & 7) ^ first) << 4);
        char* p = row + col * 4;
#pragma unroll
        for (int i = 0; i < 8; ++i, p += step) {
            float4 v;
            asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w)
                         : "r"((at ^ ((i & 1) << 6)) + i * 512) : "memory");
            if (first + 4 * i >= d.rows) continue;
            if (add) asm volatile("red.relaxed.gpu.global.add.v4.f32 [%0], {%1, %2, %3, %4};" ::"l"(__cvta_generic_to_global(p)), "f"(v.x), "f"(v.y), "f"(v.z), "f"(v.w) : "memory");
            else *reinterpret_cast<float4*>(p) = v;
        }
    } else if (col + lane < d.cols) {
#pragma unroll 2
        for (int r = 0; r < min(32, d.rows); ++r) {
            float v;
            asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v) : "r"(buf + r * 128 + (((lane >> 2) ^ (r & 7)) << 4) + (lane & 3) * 4) : "memory");
            float* p = d.p + r * d.stride + col + lane;
            if (add) asm volatile("red.relaxed.gpu.global.add.f32 [%0], %1;" ::"l"(__cvta_generic_to_global(p)), "f"(v) : "memory");
            else *p = v;
        }
    }
}

// A wait ran out: nothing of this pair's tiles can be trusted, and that shows.
__device__ __noinline__ void spoil(const WeightGrad& a, int pair, int pairs, int tid) {
    for (int unit = pair; unit < a.plan.units; unit += pairs) {
        const int tile = unit_of(a.plan, unit).tile;
        const int64_t n0 = static_cast<int64_t>(tile % a.plan.tiles_n) * kTileN, k0 = static_cast<int64_t>(tile / a.plan.tiles_n) * kTileK;
        for (int i = tid; i < kTileN * kTileK; i += kAdders) {
            const int64_t n = n0 + i / kTileK, k = k0 + i % kTileK;
            if (n < a.n_out && k < a.n_in) a.dw[n * a.dw_stride + k] = __uint_as_float(0x7FC00000u);
            if (unit >= a.plan.whole && a.plan.parts > 1)
                a.partial[static_cast<int64_t>(unit - a.plan.whole) * kTileN * kTileK + i] = __uint_as_float(0x7FC00000u);
        }
    }
}

__global__ void __launch_bounds__(kThreads, 1)
weight_grad8_kernel(const __grid_constant__ CUtensorMap dy_map, const __grid_constant__ CUtensorMap x_map, const __grid_constant__ WeightGrad a) {
    extern __shared__ uint8_t dynamic[];
    __shared__ Shared sh;
    const uint32_t stages = (smem_addr(dynamic) + 1023u) & ~1023u;
    const int tid = threadIdx.x, warp = tid >> 5;
    const int pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
    const Plan& p = a.plan;
    volatile int* abort = &sh.abort;
    uint32_t rank;  // in the pair; the first block issues the matrix instructions and waits for both blocks' operands
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));

    if (tid == 0) {
        for (int s = 0; s < kStages; ++s) {
            mbar_init(smem_addr(&sh.full[s]), 1 + 2 * 4);
            mbar_init(smem_addr(&sh.empty[s]), 1);
        }
        for (int c = 0; c < kCodeSlots; ++c) {
            mbar_init(smem_addr(&sh.codes[c]), 1);
            mbar_init(smem_addr(&sh.taken[c]), 4);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(smem_addr(&sh.summed[b]), 1);
            mbar_init(smem_addr(&sh.added[b]), 2 * kAdders / 32);
        }
        mbar_init(smem_addr(&sh.last), 1);
        sh.abort = 0;
        mbar_init_visible();
    }
    if (warp == 0) tmem_alloc_pair(smem_addr(&sh.tmem), 512);
    tc_fence_before();
    __syncthreads();
    if (a.follows) after_previous();
    asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory");
    tc_fence_after();
    const uint32_t tmem = sh.tmem;

    if (warp < kAdders / 32) {
        // ---- sums of the chunks, to dW: 32 rows of the tile to a warp
        const int lane = tid & 31, n_local = rank * kBlockN + warp * 32;
        const uint32_t out = stages + kStages * kStageBytes + kCodeSlots * kCodeBytes + warp * kSquareBytes;
        const uint32_t tmem_at = tmem + (static_cast<uint32_t>(warp * 32) << 16);
        const uint32_t added = cluster_addr(smem_addr(&sh.added[0]), 0);
        uint32_t chunk = 0;
        bool ok = true;
        for (int unit = pair; ok && unit < p.units; unit += pairs) {
            const Dest d = dest_of(a, unit, n_local, 0);
            const bool vectors = (reinterpret_cast<uintptr_t>(d.p) & 15) == 0 && (d.stride & 3) == 0;
            char* const row = reinterpret_cast<char*>(d.p + (lane >> 3) * d.stride + 4 * (lane & 7));
            bool add = d.add;
            for (int left = unit_of(p, unit).stages; left > 0; left -= kChunk, ++chunk) {
                ok = __all_sync(0xFFFFFFFFu, mbar_wait(smem_addr(&sh.summed[chunk & 1]), (chunk >> 1) & 1, abort));
                if (!ok) break;
                tc_fence_after();
                const uint32_t src = tmem_at + (chunk & 1) * kTileK;
#pragma unroll 1
                for (int j = 0; j < kTileK; j += 32) {
                    uint32_t r[32];
                    tmem_load32(src + j, r);
                    tmem_load_wait();
                    stage_square(out, lane, r);
                    __syncwarp();
                    store_square(out, lane, d, j, add, vectors, row, d.stride * 16);
                    __syncwarp();
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive_pair(added + (chunk & 1) * 8);
                add = true;
            }
        }
        if (!ok) spoil(a, pair, pairs, tid);
    } else if (warp < (kAdders + kDecoders) / 32) {
        // ---- decoding: a group's stages, the exponents of the next two on their way
        const int lane = tid & 31, group = (tid - kAdders) >> 7;
        const uint32_t full = cluster_addr(smem_addr(&sh.full[0]), 0), empty = smem_addr(&sh.empty[0]);
        const uint32_t arrived = smem_addr(&sh.codes[0]), taken = smem_addr(&sh.taken[0]);
        int total = 0, slot = group, code_slot = group;
        uint32_t parity = 1, code_parity = 0;
        for (int unit = pair; unit < p.units; unit += pairs) total += unit_of(p, unit).stages;
        Walk walk;
        Exponents exps[2];
        walk.start(a, pair, group, pairs, rank, tid);
        walk.load(a, pairs, rank, tid, &exps[0]);
        walk.load(a, pairs, rank, tid, &exps[1]);
        bool ok = true;
        auto decode = [&](Exponents* x) {
            uint4 q[4];
            // In this order: the slot is free once the stage five before has been used, so the codes of the stage six before have
            // come, and the wait for this stage's cannot take their arrival for one it has not seen yet.
            ok = __all_sync(0xFFFFFFFFu, mbar_wait(empty + slot * 8, parity, abort));
            if (!ok) return;
            ok = __all_sync(0xFFFFFFFFu, mbar_wait(arrived + code_slot * 8, code_parity, abort));
            if (!ok) return;
            load_codes(stages + kStages * kStageBytes + code_slot * kCodeBytes, tid, q);
            store_codes(stages + slot * kStageBytes + kBytesA, tid, q, *x);
            smem_to_async();
            __syncwarp();
            if (lane == 0) {
                mbar_arrive_pair(full + slot * 8);
                mbar_arrive(taken + code_slot * 8);
            }
            walk.load(a, pairs, rank, tid, x);
            slot += kGroups;
            if (slot >= kStages) slot -= kStages, parity ^= 1;
            code_slot += kGroups;
            if (code_slot >= kCodeSlots) code_slot -= kCodeSlots, code_parity ^= 1;
        };
#pragma unroll 1
        for (int i = group; ok && i < total; i += 2 * kGroups) {
            decode(&exps[0]);
            if (ok && i + kGroups < total) decode(&exps[1]);
        }
    } else {
        // Roles of one lane each, but the whole warp walks through them: so addresses and descriptors are formed in
        // uniform registers, from which the copies and the matrix instructions take them. (A lane that walked alone
        // took 700 cycles for a stage whose products take 512.)
        if (warp == (kAdders + kDecoders) / 32) {
            // ---- copies of dY: this block's half, counted by the first block's barrier
            const uint32_t full = cluster_addr(smem_addr(&sh.full[0]), 0), empty = smem_addr(&sh.empty[0]);
            const bool leader = elect_one();
            int it = 0, slot = 0;
            uint32_t parity = 1;
            for (int unit = pair; unit < p.units; unit += pairs) {
                const Unit u = unit_of(p, unit);
                const int n0 = (u.tile % p.tiles_n) * kTileN + rank * kBlockN;
                int plane = u.first / p.stages_per_plane, t0 = (u.first - plane * p.stages_per_plane) * kRows;
                const int end = p.stages_per_plane * kRows;
#pragma unroll 1
                for (int s = 0; s < u.stages; ++s) {
                    mbar_wait_uniform(empty + slot * 8, parity, &sh.abort);
                    const uint32_t bar = full + slot * 8, dst = stages + slot * kStageBytes;
                    if (leader) {
                        if (rank == 0) mbar_expect(smem_addr(&sh.full[0]) + slot * 8, 2 * kBytesA);
                        tma_load_3d_pair(dst, &dy_map, bar, n0, t0, plane);
                        tma_load_3d_pair(dst + kPanel, &dy_map, bar, n0 + 64, t0, plane);
                    }
                    ++it;
                    t0 += kRows;
                    if (t0 == end) t0 = 0, ++plane;
                    if (++slot == kStages) slot = 0, parity ^= 1;
                }
            }
            // the last signals, and copies, arrive in this block's memory: not before that
            const int from = it > kStages ? it - kStages : 0;
            for (int i = from; i < it; ++i) mbar_wait_uniform(empty + i % kStages * 8, (i / kStages) & 1, &sh.abort);
            if (*abort != 0 && rank == 0) {
                int own = 0;
                for (int i = from; i < it; ++i) mbar_wait(smem_addr(&sh.full[i % kStages]), (i / kStages) & 1, &own);
            }
        } else if (warp == (kAdders + kDecoders) / 32 + 2) {
            // ---- copies of the codes: this block's half
            const uint32_t arrived = smem_addr(&sh.codes[0]), taken = smem_addr(&sh.taken[0]);
            const bool leader = elect_one();
            int it = 0, slot = 0;
            uint32_t parity = 1;
            for (int unit = pair; unit < p.units; unit += pairs) {
                const Unit u = unit_of(p, unit);
                const int k0 = u.tile / p.tiles_n * kTileK + rank * kBlockK, end = p.stages_per_plane * kRows;
                int t0 = u.first % p.stages_per_plane * kRows;
#pragma unroll 1
                for (int s = 0; s < u.stages; ++s) {
                    mbar_wait_uniform(taken + slot * 8, parity, &sh.abort);
                    if (leader) {
                        mbar_expect(arrived + slot * 8, kCodeBytes);
                        tma_load_2d(stages + kStages * kStageBytes + slot * kCodeBytes, &x_map, arrived + slot * 8, k0, t0);
                    }
                    ++it;
                    t0 += kRows;
                    if (t0 == end) t0 = 0;
                    if (++slot == kCodeSlots) slot = 0, parity ^= 1;
                }
            }
            if (*abort != 0) {
                int own = 0;
                for (int i = it > kCodeSlots ? it - kCodeSlots : 0; i < it; ++i)
                    mbar_wait(smem_addr(&sh.codes[i % kCodeSlots]), (i / kCodeSlots) & 1, &own);
            }
        } else if (warp == (kAdders + kDecoders) / 32 + 1 && rank == 0) {
            // ---- matrix unit
            constexpr uint32_t idesc = tc_idesc_bf16_rows(kTileN, kTileK), kStep = kStageBytes >> 4;
            const uint64_t desc_a = tc_desc_rows(stages, kPanel), desc_b = tc_desc_rows(stages + kBytesA, kPanel);
            const uint32_t full = smem_addr(&sh.full[0]), empty = smem_addr(&sh.empty[0]);
            const bool leader = elect_one();
            uint32_t slot = 0, parity = 0, chunk = 0;
            for (int unit = pair; unit < p.units; unit += pairs) {
                for (int left = unit_of(p, unit).stages; left > 0; left -= kChunk, ++chunk) {
                    const int n = min(left, kChunk);
                    const uint32_t d = tmem + (chunk & 1) * kTileK;
                    // the half of the tensor memory is free once the chunk before the last has been added
                    if (chunk >= 2) mbar_wait_uniform(smem_addr(&sh.added[chunk & 1]), ((chunk >> 1) & 1) ^ 1, &sh.abort);
#pragma unroll 1
                    for (int s = 0; s < n; ++s) {
                        mbar_wait_uniform(full + slot * 8, parity, &sh.abort);
                        tc_fence_after();
                        const uint64_t da = desc_a + slot * kStep, db = desc_b + slot * kStep;
                        if (leader) {
#pragma unroll
                            for (int k = 0; k < kRows / 16; ++k) tc_mma_f16_pair(d, da + k * (2048 >> 4), db + k * (2048 >> 4), idesc, s != 0 || k != 0);
                            tc_commit_pair(empty + slot * 8);
                        }
                        __syncwarp();
                        if (++slot == kStages) slot = 0, parity ^= 1;
                    }
                    if (leader) tc_commit_pair(smem_addr(&sh.summed[chunk & 1]));
                    __syncwarp();
                }
            }
            // nothing may still be running when the tensor memory is given back
            int own = 0;
            if (leader) tc_commit_pair(smem_addr(&sh.last));
            mbar_wait(smem_addr(&sh.last), 0, &own);
        }
    }
    // neither block leaves while the other may still signal to it or use its operands
    tc_fence_before();
    __syncthreads();
    asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory");
    tc_fence_after();
    if (warp == 0) tmem_free_pair(tmem, 512);
}

// dW of the tiles whose rows were split: the parts added in their order, four columns to a thread and
// four parts under way at a time (1024 x 1024 in four parts: 5.5 us; one column and one part at a time 22 us). It reads what
// the L2 cache still holds. weight_grad8_kernel does not say early that it may begin: its few blocks
// would all sit on the SMs that are free first (65536 x 256 x 256: 52 us instead of 33.5).
__global__ void __launch_bounds__(256) join_parts_kernel(const __grid_constant__ WeightGrad a) {
    after_previous();
    const Plan& p = a.plan;
    const int other = blockIdx.x, tile = p.whole + other, i = (blockIdx.y * 256 + threadIdx.x) * 4;
    const int64_t n = static_cast<int64_t>(tile % p.tiles_n) * kTileN + i / kTileK, k = static_cast<int64_t>(tile / p.tiles_n) * kTileK + i % kTileK;
    if (n >= a.n_out || k >= a.n_in) return;
    const float4* src = reinterpret_cast<const float4*>(a.partial + static_cast<int64_t>(other) * p.parts * kTileN * kTileK + i);
    constexpr int kPart = kTileN * kTileK / 4;
    float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    for (int s = 0; s < p.parts; s += 4) {
        float4 x[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) x[u] = s + u < p.parts ? __ldcs(src + static_cast<int64_t>(s + u) * kPart) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
        for (int u = 0; u < 4; ++u) v.x += x[u].x, v.y += x[u].y, v.z += x[u].z, v.w += x[u].w;
    }
    float* d = a.dw + n * a.dw_stride + k;
    const float f[4] = {v.x, v.y, v.z, v.w};
    if (k + 4 <= a.n_in && (reinterpret_cast<uintptr_t>(d) & 15) == 0) {
        if (a.accumulate) {
            const float4 o = *reinterpret_cast<const float4*>(d);
            v.x += o.x, v.y += o.y, v.z += o.z, v.w += o.w;
        }
        *reinterpret_cast<float4*>(d) = v;
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (k + j < a.n_in) d[j] = a.accumulate ? d[j] + f[j] : f[j];
    }
}

__global__ void __launch_bounds__(256) zero_kernel(float* dw, int64_t stride, int64_t n_out, int64_t n_in) {
    const int64_t total = n_out * n_in;
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; i < total; i += static_cast<int64_t>(gridDim.x) * 256)
        dw[i / n_in * stride + i % n_in] = 0.0f;
}

// dY as the copies want it: bf16, rows at multiples of 16 bytes. An fp32 value is the sum of three
// bf16: its leading 8 bits, the next 8 and the last 8, cut off, so that the sum is exact and
// nothing overflows; an infinity or NaN is carried by the first alone.
// A thread takes four columns (4099 x 1000 fp32: 8 us; one column a thread 18). The copy is written and read once; it is small next to
// the product that follows, whose copies want rows at multiples of 16 bytes.
template <typename T>
__global__ void __launch_bounds__(256) stage_dy_kernel(const T* dy, int64_t stride, int64_t rows, int64_t n_out, uint16_t* out, int64_t out_stride) {
    next_may_begin();
    const int64_t fours = out_stride / 4, total = rows * fours, plane = rows * out_stride;
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; i < total; i += static_cast<int64_t>(gridDim.x) * 256) {
        const int64_t t = total <= 0xFFFFFFFFll ? static_cast<int64_t>(static_cast<uint32_t>(i) / static_cast<uint32_t>(fours)) : i / fours;
        const int64_t n = (i - t * fours) * 4;
        const T* const src = dy + t * stride + n;
        T v[4];
        if (sizeof(T) == 4 && n + 4 <= n_out && (reinterpret_cast<uintptr_t>(src) & 15) == 0) {
            const uint4 x = *reinterpret_cast<const uint4*>(src);
            v[0] = x.x, v[1] = x.y, v[2] = x.z, v[3] = x.w;
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = n + j < n_out ? src[j] : T(0);
        }
        uint16_t* const dst = out + t * out_stride + n;
        if constexpr (sizeof(T) == 2) {
            *reinterpret_cast<uint2*>(dst) = make_uint2(v[0] | (static_cast<uint32_t>(v[1]) << 16), v[2] | (static_cast<uint32_t>(v[3]) << 16));
        } else {
            uint32_t part[3][4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float f = __uint_as_float(v[j]);
                uint32_t hi = v[j] & 0xFFFF0000u, mid = 0, lo = 0;
                if ((hi & 0x7F800000u) == 0x7F800000u) {
                    if (f != f) hi = 0x7FC00000u;
                } else {
                    const float rest = f - __uint_as_float(hi);
                    mid = __float_as_uint(rest) & 0xFFFF0000u;
                    lo = __float_as_uint(rest - __uint_as_float(mid));
                }
                part[0][j] = hi, part[1][j] = mid, part[2][j] = lo;
            }
#pragma unroll
            for (int k = 0; k < 3; ++k)
                *reinterpret_cast<uint2*>(dst + k * plane) = make_uint2(__byte_perm(part[k][0], part[k][1], 0x7632), __byte_perm(part[k][2], part[k][3], 0x7632));
        }
    }
}

constexpr int64_t kMaxUnits = 1 << 24;  // tiles, and stages: rows and their products with kRows stay in 32 bits

// How dY reaches the matrix unit, and how the work is cut. The pairs of blocks take whole tiles as
// long as every pair gets one; the tiles that are left over (all, if there are fewer than pairs)
// have their rows split so that they too keep most SMs busy.
struct Layout {
    bool staged;
    int64_t stride, planes;  // of the staged copy
    int64_t staged_bytes, partial_bytes;
    Plan plan;
};

int layout_of(const void* dy, int64_t dy_stride, ss_dtype dt, int64_t rows, int64_t n_out, int64_t n_in, int sms, Layout* out) {
    const Mat m = mat(dy, rows, n_out, dy_stride, dtype_bytes(dt));
    out->staged = dt == SS_F32 || !m.row_aligned(16) || m.stride * 2 % 16 != 0 || m.stride * 2 >= (int64_t(1) << 40);
    out->planes = dt == SS_F32 ? 3 : 1;
    out->stride = out->staged ? (n_out + 7) / 8 * 8 : m.stride;
    out->staged_bytes = out->staged ? (out->planes * rows * out->stride * 2 + 255) / 256 * 256 : 0;
    const int64_t tn = (n_out + kTileN - 1) / kTileN, tk = (n_in + kTileK - 1) / kTileK, per = (rows + kRows - 1) / kRows;
    if (tn * tk > kMaxUnits || per * out->planes > kMaxUnits) return SS_ERR_UNSUPPORTED;
    Plan& p = out->plan;
    p.tiles_n = static_cast<int>(tn), p.tiles_k = static_cast<int>(tk);
    p.planes = static_cast<int>(out->planes), p.stages_per_plane = static_cast<int>(per);
    const int pairs = sms / 2, tiles = static_cast<int>(tn * tk), all = p.planes * p.stages_per_plane, others = tiles % pairs;
    p.whole = tiles - others;
    p.parts = 1;
    p.part_stages = all;
    if (others > 0) {
        int parts = pairs / others;
        if (parts > all / kLeastPart) parts = all / kLeastPart;
        if (parts > 1) {
            p.part_stages = (all + parts - 1) / parts;
            p.parts = (all + p.part_stages - 1) / p.part_stages;
        }
    }
    p.units = p.whole + others * p.parts;
    out->partial_bytes = p.parts > 1 ? static_cast<int64_t>(others) * p.parts * kTileN * kTileK * 4 : 0;
    return SS_OK;
}

// SMs that the plan is made for. Without a device (sizes asked for on a host without one) the B200's.
int plan_sms() {
    cudaError_t err = cudaSuccess;
    const int sms = device_sm_count(&err);
    return err == cudaSuccess && sms > 0 ? sms : 148;
}

}  // namespace
}  // namespace ss

using namespace ss;

extern "C" {
#pragma GCC visibility push(default)

int64_t ss_weight_grad8_workspace(const void* dy, int64_t dy_stride, ss_dtype dt, int64_t rows, int64_t n_out, int64_t n_in) {
    if (!dtype_known(dt) || !sides_ok(rows, n_out) || !sides_ok(rows, n_in) || !stride_ok(rows, n_out, dy_stride)) return -1;
    if (rows == 0 || n_out == 0 || n_in == 0) return 0;
    Layout l;
    if (layout_of(dy, dy_stride, dt, rows, n_out, n_in, plan_sms(), &l) != SS_OK) return -1;
    return l.staged_bytes + l.partial_bytes;
}

int ss_weight_grad8(const void* dy, int64_t dy_stride, ss_dtype dt, const uint8_t* ckpt_x, int64_t rows,
                    int64_t n_out, int64_t n_in, float* dw, int64_t dw_stride, int accumulate, void* workspace,
                    int64_t workspace_bytes, void* cuda_stream) {
    if (!dtype_known(dt) || !sides_ok(rows, n_out) || !sides_ok(rows, n_in)) return SS_ERR_INVALID_ARG;
    if (!stride_ok(rows, n_out, dy_stride) || !stride_ok(n_out, n_in, dw_stride)) return SS_ERR_INVALID_ARG;
    if (n_out == 0 || n_in == 0) return SS_OK;
    const size_t eb = dtype_bytes(dt);
    const Mat mw = mat(dw, n_out, n_in, dw_stride, 4), my = mat(dy, rows, n_out, dy_stride, eb);
    if (dw == nullptr || (rows > 0 && (dy == nullptr || ckpt_x == nullptr))) return SS_ERR_INVALID_ARG;
    if (!addr_aligned(dw, 4)) return SS_ERR_MISALIGNED;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    if (rows == 0) {
        if (accumulate) return SS_OK;
        const int64_t blocks = (n_out * n_in + 255) / 256;
        zero_kernel<<<static_cast<unsigned>(blocks < 4096 ? blocks : 4096), 256, 0, st>>>(dw, mw.stride, n_out, n_in);
        return cuda_status_public(cudaGetLastError());
    }
    if (!addr_aligned(dy, eb) || !addr_aligned(ckpt_x, 16)) return SS_ERR_MISALIGNED;
    const size_t kept = ss_act8_bytes(rows, n_in);
    if (mats_overlap(mw, my) || mat_overlaps(mw, ckpt_x, kept)) return SS_ERR_INVALID_ARG;
    Layout l;
    const int status = layout_of(dy, dy_stride, dt, rows, n_out, n_in, plan_sms(), &l);
    if (status != SS_OK) return status;
    const int64_t need = l.staged_bytes + l.partial_bytes;
    if (workspace_bytes < need || (need > 0 && workspace == nullptr)) return SS_ERR_INVALID_ARG;
    if (need > 0) {
        if (!addr_aligned(workspace, 256)) return SS_ERR_MISALIGNED;
        if (mat_overlaps(mw, workspace, need) || mat_overlaps(my, workspace, need) || bytes_overlap(ckpt_x, kept, workspace, need))
            return SS_ERR_INVALID_ARG;
    }
    cudaError_t e;
    const EncodeTiled encode = encode_tiled(&e);
    if (encode == nullptr) return cuda_status_public(e);
    const int sms = device_sm_count(&e);
    if (e != cudaSuccess) return cuda_status_public(e);

    CUtensorMap map;
    const cuuint64_t row_bytes = static_cast<cuuint64_t>(l.stride) * 2;
    const cuuint64_t dims[3] = {static_cast<cuuint64_t>(n_out), static_cast<cuuint64_t>(rows), static_cast<cuuint64_t>(l.planes)};
    const cuuint64_t strides[2] = {row_bytes, l.planes > 1 ? row_bytes * rows : row_bytes};
    const cuuint32_t box[3] = {64, kRows, 1}, ones[3] = {1, 1, 1};
    void* src = l.staged ? workspace : const_cast<void*>(dy);
    if (encode(&map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, src, dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
               CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
        return SS_ERR_UNSUPPORTED;
    CUtensorMap x_map;
    const cuuint64_t pitch = static_cast<cuuint64_t>(act8_groups(n_in)) * SS_ACT8_GROUP;
    const cuuint64_t x_dims[2] = {pitch, static_cast<cuuint64_t>(rows)};
    const cuuint32_t x_box[2] = {kBlockK, kRows};
    if (encode(&x_map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<uint8_t*>(ckpt_x), x_dims, &pitch, x_box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
               CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
        return SS_ERR_UNSUPPORTED;
    e = allow_shared<WeightGrad>(reinterpret_cast<const void*>(weight_grad8_kernel), static_cast<int>(kSmem));
    if (e != cudaSuccess) return cuda_status_public(e);

    if (l.staged) {
        const int64_t want = (rows * l.stride / 4 + 255) / 256, most = static_cast<int64_t>(sms) * 16;
        const unsigned grid = static_cast<unsigned>(want < most ? want : most);
        if (dt == SS_F32) stage_dy_kernel<uint32_t><<<grid, 256, 0, st>>>(static_cast<const uint32_t*>(dy), my.stride, rows, n_out, static_cast<uint16_t*>(workspace), l.stride);
        else stage_dy_kernel<uint16_t><<<grid, 256, 0, st>>>(static_cast<const uint16_t*>(dy), my.stride, rows, n_out, static_cast<uint16_t*>(workspace), l.stride);
        e = cudaGetLastError();
        if (e != cudaSuccess) return cuda_status_public(e);
    }
    float* partial = reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + l.staged_bytes);
    const WeightGrad a{ckpt_of(const_cast<uint8_t*>(ckpt_x), rows, n_in), dw, partial, mw.stride, rows, n_out, n_in, accumulate, l.staged, l.plan};
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(static_cast<unsigned>(2 * (l.plan.units < sms / 2 ? l.plan.units : sms / 2)));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = kSmem;
    cfg.stream = st;
    cudaLaunchAttribute at[2] = {};
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = 2, at[0].val.clusterDim.y = 1, at[0].val.clusterDim.z = 1;
    at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = l.staged ? 2 : 1;
    e = cudaLaunchKernelEx(&cfg, weight_grad8_kernel, map, x_map, a);
    if (e != cudaSuccess) return cuda_status_public(e);
    if (l.plan.parts > 1) {
        const unsigned others = static_cast<unsigned>(l.plan.tiles_n * l.plan.tiles_k - l.plan.whole);
        e = launch_next(true, join_parts_kernel, dim3(others, kTileN * kTileK / 1024), 256, st, a);
    }
    return cuda_status_public(e);
}

#pragma GCC visibility pop
}  // extern "C"
