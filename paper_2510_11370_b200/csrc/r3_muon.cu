// Newton-Schulz orthogonalisation of matrices, and the momentum step of an optimiser built on it.  With
// u the matrix, X = u / (|u|_F + eps) and per step (a, b, c):
//   A = X X^T  (X^T X where the matrix is tall: the smaller side)     B = b A + c A^2     X = a X + B X
//
// Three products a step on the tensor cores, each a batch over all matrices of a round (up to four shapes in one
// launch).  Numbers.  The iterates' singular values stay near one, so fp16 (11 bits, against bf16's 8) holds
// every operand, times 2^14 with the usual coefficients to keep small elements in its normal range.  X itself is
// carried in two fp16 planes, hi + lo (22 bits): the term a X, by which a weak direction grows a^steps-fold, then has
// no rounding to speak of, and what the products' operands lose stays about as small as the output's own rounding to
// bf16 whatever the matrix's spectrum is (simulated for full-rank, decaying and low-rank spectra and sides from 16 on:
// 1.3e-3 to 3e-3 of the result's rms, mostly below 2e-3, against 1.7e-3 for the rounding; bf16 operands with a rounded
// X lose a third of a rank-8 update).  For float32 results A and B get a second plane as well and every product is
// hi lo + lo hi + hi hi.  Lo planes hold 2^11 of their values, or they would lose what small rows have: the sum of the
// first two products is taken times 2^-11 by the multiplication that adds the third.
//
// One GEMM kernel does all three, with two CTAs per MMA (256 x 256 tiles, or 256 x 128 where they are few; 128
// rows of the left operand per CTA and k block of 64, accumulators double buffered in tensor memory).
// B = a I + b A + c A^2, the identity within, so that the last product is the whole of the new X (one product: but
// for a times the lo plane, which is no operand then and comes while the product is formed).  A and B are
// symmetric: only tiles on and below the diagonal are computed, the others are stored from the same accumulators,
// transposed.  Eight epilogue warps, each with its own 8 KB (three products: 4 KB) of shared memory, through
// which results go out by TMA in boxes of 32 rows x 64 columns and addends come in whole lines.
// 24 matrices of 768 x 2048, one product, launches by themselves: X X^T 33 to 36 us, B 21 to 23, B X 52 to 56 (with one
// plane out), of which the products of their tiles are 23, 9 and 35 at the tensor pipe's rate.  B X moves 228 MB to and
// from HBM and 796 between L2 and the SMs, 14.2 TB/s; X X^T and B wait for the first loads and the last stores of their
// few tiles.  Three products, 4096 x 4096: 3100 us for five steps at first (3450 to 3550 under load), the tensor pipe
// busy for three quarters: each 64 of k leave tensor memory for registers.  (With 128 columns the epilogue of B then
// leaves 104 bytes a thread in local memory: both planes of A stand beside the sums.)
#include <algorithm>
#include <cmath>
#include <vector>

#include "r3_muon.cuh"

namespace r3 {
namespace ns {

constexpr int BM = 128;                   // rows of the left operand per CTA and stage
constexpr int TILE = 2 * BM;              // rows of a CTA pair's output tile; its columns, TN, are 256 or 128
constexpr int BK = 64;                    // k per stage: 64 fp16 = one 128-byte swizzle row
constexpr int UK = 16;                    // k per tcgen05.mma
constexpr int OPERAND_BYTES = BM * BK * 2;
constexpr int EPI_WARPS = 8;              // two per TMEM lane quadrant, half of the columns each
constexpr int EPI_PLANE = 32 * 128;       // 32 rows x 64 columns of fp16
constexpr int BAR_BYTES = 256;
// By the products per product.  Three: a stage holds both planes of both operands, so that four tiles serve
// three products (copied for each by itself they came out of L2 no faster than 60% of the tensor pipe could
// take them), and the sum of a stage leaves tensor memory for registers, since an addition there drops what
// lies below the running sum's last place.
template <int TERMS, int TN> struct Ring {
    static constexpr int PLANES = TERMS > 1 ? 2 : 1;
    static constexpr int STAGES = TERMS > 1 ? (TN == 256 ? 3 : 4) : (TN == 256 ? 5 : 6);
    static constexpr int B_BYTES = TN / 2 * BK * 2;                      // of a plane of the right operand
    static constexpr int SIDE_BYTES = PLANES * OPERAND_BYTES;            // the left operand
    static constexpr int STAGE_BYTES = SIDE_BYTES + PLANES * B_BYTES;
    static constexpr bool SPLIT = TERMS > 1 && TN == 256;                // of the register file, see below
    static constexpr int BUFFERS = TERMS > 1 ? 1 : 2;                    // of an epilogue warp
    static constexpr int EPI_BYTES = EPI_WARPS * BUFFERS * EPI_PLANE;
    static constexpr int SMEM_BYTES = 1024 + STAGES * STAGE_BYTES + EPI_BYTES + BAR_BYTES;
};
constexpr int THREADS = 32 * (4 + EPI_WARPS);        // warp 0 copies, warp 1 multiplies, 2 and 3 fill their group
// Three products, 256 columns: the epilogue keeps 128 sums a thread, so the register file is split anew between the
// first four warps and the others; both shares together are what the launch had (checked before it).
constexpr int CONTROL_REGS = 40, EPI_REGS = 232, LAUNCH_REGS = 168;
static_assert(128 * CONTROL_REGS + 32 * EPI_WARPS * EPI_REGS <= THREADS * LAUNCH_REGS, "register split");
constexpr int MAX_CLASSES = 4;            // shapes of a launch

enum Phase { GRAM, POLY, APPLY };
// The matrices of one shape in a launch.
struct alignas(64) ClassArgs {
    CUtensorMap a[2], b[2];               // operands, planes hi and lo
    CUtensorMap out[2], mirror[2];
    const __half* in[2];                  // POLY: A; APPLY with one product: X's lo plane in [0], or null
    long long in_plane;                   // elements of a matrix there
    int in_ld;
    int rows, cols;                       // of D
    int tiles_n, tiles, first_item, kblocks;         // tiles: of one matrix
    int a_mn, b_mn;                       // the operand's rows in memory run along k
    int splits, per_split;                // GRAM: a tile's k blocks in so many parts of per_split each
    float4* partial;                      // and where their sums go (fold_kernel adds them up)
};
struct alignas(64) GemmArgs {
    ClassArgs c[MAX_CLASSES];
    int classes, items;
    int keep_lo;                          // APPLY with one product: X's lo plane is written
    float alpha, beta, diag;
    int32_t* dev_status;
};

__device__ __forceinline__ void tma_store_3d(const CUtensorMap* map, uint32_t src, int c0, int c1, int c2) {
    asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.bulk_group [%0, {%2, %3, %4}], [%1];"
                 ::"l"(map), "r"(src), "r"(c0), "r"(c1), "r"(c2) : "memory");
}
__device__ __forceinline__ void bulk_commit() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }
// All stores but the last ones have been read out of shared memory.
template <int LAST> __device__ __forceinline__ void bulk_wait_read() {
    asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(LAST) : "memory");
}
__device__ __forceinline__ void prefetch_map(const CUtensorMap* map) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory");
}

template <int TN> constexpr int SLOT = TILE * TN / 4;        // float4 of a part's sums: [rank][warp][4 columns][row]
struct Tile {
    int k, z, m, n;                       // class, matrix, tile row and column
    int k0, k1, slot;                     // k blocks; number of the part
};
// Symmetric results: the tiles on the diagonal and below it, row by row.  Those of 128 columns: 2 m + 2 of them
// in row m, the last two on the diagonal.
template <int TN> __device__ __forceinline__ void lower_tile(int r, int* m_out, int* n_out) {
    constexpr int F = TILE / TN;                         // F m (m + 1) / 2 tiles stand before row m
    int m = (int)((sqrtf(8.f / F * (float)r + 1.f) - 1.f) * 0.5f);
    while (F * m * (m + 1) / 2 > r) --m;
    while (F * (m + 1) * (m + 2) / 2 <= r) ++m;
    *m_out = m;
    *n_out = r - F * m * (m + 1) / 2;
}
template <int PHASE, int TN> __device__ __forceinline__ Tile decode(const GemmArgs& g, int item) {
    Tile t;
    t.k = 0;
#pragma unroll
    for (int i = 1; i < MAX_CLASSES; ++i)
        if (i < g.classes && item >= g.c[i].first_item) t.k = i;
    const ClassArgs& c = g.c[t.k];
    item -= c.first_item;
    t.k0 = 0;
    t.k1 = c.kblocks;
    t.slot = item;
    if (PHASE == GRAM && c.splits > 1) {
        const int split = item % c.splits;
        item /= c.splits;
        t.k0 = split * c.per_split;
        t.k1 = min(c.kblocks, t.k0 + c.per_split);
    }
    t.z = item / c.tiles;
    const int r = item - t.z * c.tiles;
    if (PHASE != APPLY) {
        lower_tile<TN>(r, &t.m, &t.n);
    } else {
        t.m = r / c.tiles_n;
        t.n = r - t.m * c.tiles_n;
    }
    return t;
}
__device__ __forceinline__ void half8(const uint4& v, float (&f)[8]) {
    const __half2* h = reinterpret_cast<const __half2*>(&v);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 t = __half22float2(h[i]);
        f[2 * i] = t.x;
        f[2 * i + 1] = t.y;
    }
}

// GRAM: A = X X^T.  POLY: B = a I + b A + c A^2.  APPLY: X = B X (one product: + a times X's lo plane, which
// is no operand then).  TERMS: products per product.
template <int PHASE, int TERMS, int TN>
__global__ void __launch_bounds__(THREADS, 1) gemm_kernel(const __grid_constant__ GemmArgs g) {
    constexpr bool SYM = PHASE != APPLY;
    constexpr int OUT = SYM && TERMS == 1 ? 1 : 2;     // planes of D
    using R = Ring<TERMS, TN>;
    constexpr int BN = TN / 2;                         // rows of the right operand per CTA and stage
    constexpr int CW = TN / 2;                         // columns of an epilogue warp
    constexpr int STAGES = R::STAGES, STAGE_BYTES = R::STAGE_BYTES, SIDE_BYTES = R::SIDE_BYTES;
    constexpr int EPI_BYTES = R::EPI_BYTES, BUFFERS = R::BUFFERS;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t* base_ptr = smem_raw + (base - smem_u32(smem_raw));
    const uint32_t epi0 = base + STAGES * STAGE_BYTES;
    const uint32_t bar0 = epi0 + EPI_BYTES;
    auto full_bar = [&](int s) { return bar0 + 8u * s; };
    auto empty_bar = [&](int s) { return bar0 + 8u * (STAGES + s); };
    auto tfull_bar = [&](int a) { return bar0 + 8u * (2 * STAGES + a); };
    auto tempty_bar = [&](int a) { return bar0 + 8u * (2 * STAGES + 2 + a); };
    uint8_t* misc = base_ptr + STAGES * STAGE_BYTES + EPI_BYTES + 192;
    volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(misc);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(misc + 4);
    static_assert(8 * (2 * STAGES + 4) <= 192, "barriers");

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_ctarank();
    const int pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;

    if (threadIdx.x == 0) {
        for (int s = 0; s < STAGES; ++s) { mbar_init(full_bar(s), 1); mbar_init(empty_bar(s), 1); }
        for (int a = 0; a < 2; ++a) {
            mbar_init(tfull_bar(a), 1);
            mbar_init(tempty_bar(a), 2 * EPI_WARPS);
        }
        *abort_flag = 0;
        fence_barrier_init();
    }
    if (warp == 1) tmem_alloc_pair(smem_u32(const_cast<uint32_t*>(tmem_slot)), 2 * TN);
    if (warp == 2 && lane < 2 * g.classes) {
        const ClassArgs& c = g.c[lane >> 1];
        if (lane & 1) {
            prefetch_map(&c.a[0]);
            prefetch_map(&c.out[0]);
        } else {
            prefetch_map(&c.b[0]);
            prefetch_map(&c.mirror[0]);
        }
    }
    tc_fence_before();
    __syncthreads();
    cluster_sync_all();
    tc_fence_after();
    const uint32_t tmem_base = *tmem_slot;
    grid_launch_dependents();
    // (who reads or writes global memory waits for the launch before this one, with the first tile already found:
    // 2048 x 2048 331 -> 263 us, 384 x 768 x 2048 under load 14.5 -> 13.6 ms)
    Tile first_tile = {};
    if (pair < g.items) first_tile = decode<PHASE, TN>(g, pair);

    // a tile on the diagonal of A or of A^2 has the same rows on both sides: copied once
    auto diagonal = [&](const Tile& t) { return SYM && t.m == t.n * TN / TILE; };
    auto alike = [&](const Tile& t) { return TN == TILE && diagonal(t); };

    if (warp < 4) {
        if constexpr (R::SPLIT) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(CONTROL_REGS));
        if (warp == 0) {
            // ------------------------------ TMA producer: this CTA's half of both operands ---------
            if (lane == 0) {
                int stage = 0;
                uint32_t phase = 0;
                bool ok = true;
                grid_dependency_wait();
                for (int item = pair; ok && item < g.items; item += pairs) {
                    const Tile t = item == pair ? first_tile : decode<PHASE, TN>(g, item);
                    const ClassArgs& c = g.c[t.k];
                    const int m0 = t.m * TILE + (int)rank * BM, n0 = t.n * TN + (int)rank * BN;
                    const bool once = alike(t);
                    // (held in registers: read again for each k block they cost more than its copies take)
                    uint64_t maps_a = reinterpret_cast<uint64_t>(&c.a[0]), maps_b = reinterpret_cast<uint64_t>(&c.b[0]);
                    int a_mn = c.a_mn, b_mn = c.b_mn, z = t.z, k1 = t.k1;
                    asm volatile("" : "+l"(maps_a), "+l"(maps_b), "+r"(a_mn), "+r"(b_mn), "+r"(z), "+r"(k1));
                    const CUtensorMap* map_a = reinterpret_cast<const CUtensorMap*>(maps_a);
                    const CUtensorMap* map_b = reinterpret_cast<const CUtensorMap*>(maps_b);
                    for (int kb = t.k0; kb < k1; ++kb) {
                        if (!mbar_wait(empty_bar(stage), phase ^ 1u, abort_flag, g.dev_status)) {
                            ok = false;
                            break;
                        }
                        const uint32_t sa = base + stage * STAGE_BYTES, sb = sa + SIDE_BYTES;
                        const uint32_t lead = mapa_shared(full_bar(stage), 0);
                        if (rank == 0) mbar_expect_tx(full_bar(stage), 2u * (uint32_t)(once ? SIDE_BYTES : STAGE_BYTES));
#pragma unroll
                        for (int pl = 0; pl < R::PLANES; ++pl) {
                            const uint32_t ta = sa + pl * OPERAND_BYTES, tb = sb + pl * R::B_BYTES;
                            if (a_mn) {
                                tma_load_3d_pair(ta, map_a + pl, m0, kb * BK, z, lead);
                                tma_load_3d_pair(ta + OPERAND_BYTES / 2, map_a + pl, m0 + 64, kb * BK, z, lead);
                            } else {
                                tma_load_3d_pair(ta, map_a + pl, kb * BK, m0, z, lead);
                            }
                            if (once) continue;
                            if (b_mn) {
                                tma_load_3d_pair(tb, map_b + pl, n0, kb * BK, z, lead);
                                if (BN > 64) tma_load_3d_pair(tb + OPERAND_BYTES / 2, map_b + pl, n0 + 64, kb * BK, z, lead);
                            } else {
                                tma_load_3d_pair(tb, map_b + pl, kb * BK, n0, z, lead);
                            }
                        }
                        if (++stage == STAGES) { stage = 0; phase ^= 1u; }
                    }
                }
                // every stage's release has landed before this CTA may leave
                for (int s = 0; ok && s < STAGES; ++s) {
                    ok = mbar_wait(empty_bar(stage), phase ^ 1u, abort_flag, g.dev_status);
                    if (++stage == STAGES) { stage = 0; phase ^= 1u; }
                }
            }
        } else if (warp == 1) {
            // ------------------------------ MMA issuer (leader CTA) ---------------------------------
            if (rank == 0) {
                int stage = 0, acc = 0;
                uint32_t phase = 0, acc_phase = 0;
                bool ok = true;
                grid_dependency_wait();                  // (or its waits' limits would run while others do)
                for (int item = pair; ok && item < g.items; item += pairs) {
                    const Tile t = item == pair ? first_tile : decode<PHASE, TN>(g, item);
                    const ClassArgs& c = g.c[t.k];
                    uint32_t idesc = (1u << 4) | ((uint32_t)(TN >> 3) << 17) | ((uint32_t)(TILE >> 4) << 24) |
                                     (c.a_mn ? 1u << 15 : 0u) | (c.b_mn ? 1u << 16 : 0u);
                    // 16 along k: 32 bytes inside the swizzled row, or two groups of 8 k rows
                    uint64_t a_step = c.a_mn ? (2048 >> 4) : 2, b_step = c.b_mn ? (2048 >> 4) : 2;
                    const uint32_t first_b = base + (alike(t) ? 0u : (uint32_t)SIDE_BYTES);
                    uint64_t first_da = c.a_mn ? smem_desc_mn_sw128(base, OPERAND_BYTES / 2) : smem_desc_sw128(base);
                    uint64_t first_db = c.b_mn ? smem_desc_mn_sw128(first_b, OPERAND_BYTES / 2) : smem_desc_sw128(first_b);
                    int k1 = t.k1;
                    asm volatile("" : "+r"(idesc), "+l"(a_step), "+l"(b_step), "+l"(first_da), "+l"(first_db), "+r"(k1));
                    for (int kb = t.k0; kb < k1; ++kb) {
                        // three products: every k block has an accumulator of its own
                        const bool fresh = TERMS > 1 || kb == t.k0, last = TERMS > 1 || kb + 1 == k1;
                        if (fresh && !__all_sync(0xffffffffu, mbar_wait(tempty_bar(acc), acc_phase ^ 1u, abort_flag,
                                                                        g.dev_status))) {
                            ok = false;
                            break;
                        }
                        if (!__all_sync(0xffffffffu,
                                        mbar_wait(full_bar(stage), phase, abort_flag, g.dev_status))) {
                            ok = false;
                            break;
                        }
                        tc_fence_after();
                        if (elect_one()) {
                            const uint32_t d_tmem = tmem_base + (uint32_t)(acc * TN);
                            // (a descriptor holds the address in units of 16 bytes)
                            const uint64_t da = first_da + (uint64_t)(stage * (STAGE_BYTES >> 4));
                            const uint64_t db = first_db + (uint64_t)(stage * (STAGE_BYTES >> 4));
#pragma unroll
                            for (int term = 0; term < TERMS; ++term) {
                                // (hi, lo), (lo, hi), (hi, hi): the small products first, 2^11 of them
                                const uint64_t ta = da + (TERMS > 1 && term == 1 ? OPERAND_BYTES >> 4 : 0);
                                const uint64_t tb = db + (TERMS > 1 && term == 0 ? R::B_BYTES >> 4 : 0);
#pragma unroll
                                for (int kk = 0; kk < BK / UK; ++kk) {
                                    if (term == 2 && kk == 0)
                                        tc_mma_bf16_pair_onto_scaled<LO_SHIFT>(d_tmem, ta, tb, idesc);
                                    else
                                        tc_mma_bf16_pair(d_tmem, ta + a_step * kk, tb + b_step * kk, idesc,
                                                         (fresh && (term | kk) == 0) ? 0u : 1u);
                                }
                            }
                            tc_commit_pair(empty_bar(stage), 3);
                            if (last) tc_commit_pair(tfull_bar(acc), 3);
                        }
                        __syncwarp();
                        if (++stage == STAGES) { stage = 0; phase ^= 1u; }
                        if (last && ++acc == 2) { acc = 0; acc_phase ^= 1u; }
                    }
                }
            }
        }
    } else {
        // ------------------------------ epilogue ------------------------------------------------
        if constexpr (R::SPLIT) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(EPI_REGS));
        const int w = warp - 4, q = warp & 3, half = w >> 2;
        const uint32_t buf = epi0 + (uint32_t)w * (BUFFERS * EPI_PLANE);
        uint8_t* buf_ptr = base_ptr + STAGES * STAGE_BYTES + w * (BUFFERS * EPI_PLANE);
        int acc = 0, turn = 0;
        uint32_t acc_phase = 0;
        bool alive = true;
        // 32 rows x 64 columns (a row's columns in pairs) to a buffer and out
        auto emit = [&](const uint32_t (&v)[32], const CUtensorMap* map, int col0, int row0, int z) {
            if (lane == 0) bulk_wait_read<BUFFERS - 1>();
            __syncwarp();
            uint8_t* to = buf_ptr + turn * EPI_PLANE + lane * 128;
#pragma unroll
            for (int j = 0; j < 8; ++j)                // at the places that the copy's swizzle gives them
                *reinterpret_cast<uint4*>(to + ((j ^ (lane & 7)) * 16)) =
                    make_uint4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
            fence_async();
            __syncwarp();
            if (lane == 0) {
                tma_store_3d(map, buf + turn * EPI_PLANE, col0, row0, z);
                bulk_commit();
            }
            if (BUFFERS > 1) turn ^= 1;
        };
        // the same values as 64 rows x 32 columns of the other triangle
        auto emit_mirror = [&](const uint32_t (&v)[32], const CUtensorMap* map, int col0, int row0, int z) {
            if (lane == 0) bulk_wait_read<BUFFERS - 1>();
            __syncwarp();
            __half* to = reinterpret_cast<__half*>(buf_ptr + turn * EPI_PLANE) + lane;
#pragma unroll
            for (int j = 0; j < 32; ++j) {
                const __half2 h = *reinterpret_cast<const __half2*>(&v[j]);
                to[2 * j * 32] = __low2half(h);
                to[2 * j * 32 + 32] = __high2half(h);
            }
            fence_async();
            __syncwarp();
            if (lane == 0) {
                tma_store_3d(map, buf + turn * EPI_PLANE, row0, col0, z);
                bulk_commit();
            }
            if (BUFFERS > 1) turn ^= 1;
        };
        grid_dependency_wait();
        for (int item = pair; item < g.items; item += pairs) {
            const Tile t = item == pair ? first_tile : decode<PHASE, TN>(g, item);
            const ClassArgs& c = g.c[t.k];
            const int row0 = t.m * TILE + (int)rank * BM + q * 32, row = row0 + lane;
            const int first = t.n * TN + half * CW;              // this warp's columns
            const bool inside = row0 < c.rows && first < c.cols;
            // what is added to the product: one plane of the warp's columns, which come while it is formed, or
            // (three products, whose sums take the registers) both planes of 64 of them at a time
            constexpr bool ADDS = PHASE == POLY || (PHASE == APPLY && TERMS == 1);
            uint4 early[ADDS ? (TERMS == 1 ? CW / 8 : 16) : 1];
            // (four rows x 128 bytes per load: row by row, 32 lines a load, the eight warps' loads took 8500 clocks)
            const int mine = row0 + (lane >> 3), left = c.rows - mine, hop = 4 * c.in_ld;
            const long long in_at = (long long)t.z * c.in_plane + (long long)mine * c.in_ld;
            auto fetch = [&](uint4* v, int plane, int p) {
                const int col = first + 64 * p + 8 * (lane & 7);
                const __half* from = c.in[plane] + in_at + col;
                const int some = col < c.in_ld ? left : 0;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    v[j] = make_uint4(0u, 0u, 0u, 0u);
                    if (4 * j < some) v[j] = *reinterpret_cast<const uint4*>(from + j * hop);
                }
            };
            // eight of them, 32 rows x 64 columns, to the lanes of their rows, by way of the next buffer
            auto to_rows = [&](uint4* v) {
                if (lane == 0) bulk_wait_read<BUFFERS - 1>();
                __syncwarp();
                uint8_t* box = buf_ptr + turn * EPI_PLANE;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int r = 4 * j + (lane >> 3);
                    *reinterpret_cast<uint4*>(box + r * 128 + (((lane & 7) ^ (r & 7)) * 16)) = v[j];
                }
                __syncwarp();
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    v[j] = *reinterpret_cast<const uint4*>(box + lane * 128 + ((j ^ (lane & 7)) * 16));
                __syncwarp();
            };
            const bool adds = ADDS && (PHASE == POLY || c.in[0] != nullptr);
            if constexpr (ADDS && TERMS == 1) {
                if (adds) {
#pragma unroll
                    for (int p = 0; p < CW / 64; ++p) fetch(early + 8 * p, 0, p);
                } else {
#pragma unroll
                    for (int j = 0; j < CW / 8; ++j) early[j] = make_uint4(0u, 0u, 0u, 0u);
                }
            }
            constexpr bool KEEP = TERMS > 1 || PHASE == GRAM;    // the sums go through registers as a whole
            float sum[KEEP ? CW : 1];
            if constexpr (KEEP) {
#pragma unroll
                for (int i = 0; i < CW; ++i) sum[i] = 0.f;
            }
            uint32_t tacc = 0;
#pragma unroll 1
            for (int kb = TERMS > 1 ? t.k0 : t.k1 - 1; kb < t.k1; ++kb) {
                if (alive) {
                    const bool ok = mbar_wait(tfull_bar(acc), acc_phase, abort_flag, g.dev_status);
                    alive = __all_sync(0xffffffffu, ok);
                }
                tc_fence_after();
                tacc = tmem_base + ((uint32_t)(q * 32) << 16) + (uint32_t)(acc * TN + half * CW);
                if constexpr (KEEP) {
                    if (alive && inside) {
#pragma unroll
                        for (int p = 0; p < CW / 32; ++p) {
                            float v[32];
                            tc_ld32(tacc + 32 * p, v);
                            tc_wait_ld();
#pragma unroll
                            for (int i = 0; i < 32; ++i) sum[32 * p + i] += v[i];
                        }
                    }
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0 && alive) mbar_arrive_cluster(mapa_shared(tempty_bar(acc), 0));
                    if (++acc == 2) { acc = 0; acc_phase ^= 1u; }
                }
            }
            if constexpr (PHASE == GRAM) {
                if (c.splits > 1) {
                    if (alive && inside) {
                        float4* to = c.partial + (size_t)t.slot * SLOT<TN> + ((int)rank * EPI_WARPS + w) * (CW / 4) * 32 + lane;
#pragma unroll
                        for (int j = 0; j < CW / 4; ++j)
                            to[j * 32] = make_float4(sum[4 * j], sum[4 * j + 1], sum[4 * j + 2], sum[4 * j + 3]);
                    }
                    continue;
                }
            }
            if (alive && inside) {
#pragma unroll
                for (int p = 0; p < CW / 64; ++p) {
                    const int col0 = first + 64 * p;
                    if (col0 >= c.cols) continue;
                    if constexpr (ADDS) {
                        if (TERMS == 1) {
                            if (adds) to_rows(early + 8 * p);
                        } else {
                            fetch(early, 0, p);
                            fetch(early + 8, 1, p);
                            to_rows(early);
                            to_rows(early + 8);
                        }
                    }
                    uint32_t packed[OUT][32];          // pairs of columns
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        float v[32];
                        if constexpr (KEEP) {
#pragma unroll
                            for (int i = 0; i < 32; ++i) v[i] = sum[64 * p + 32 * h + i];
                        } else {
                            tc_ld32(tacc + 64 * p + 32 * h, v);
                            tc_wait_ld();
                        }
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const int o = 8 * p + 4 * h + j;           // octet of the warp's columns
                            float x[8], l[8];
#pragma unroll
                            for (int i = 0; i < 8; ++i) x[i] = g.alpha * v[8 * j + i];
                            if constexpr (ADDS) {
                                half8(early[TERMS == 1 ? o : 4 * h + j], l);
                                if (TERMS > 1) {
                                    float e[8];
                                    half8(early[8 + 4 * h + j], e);
#pragma unroll
                                    for (int i = 0; i < 8; ++i) l[i] = fmaf(e[i], 1.f / LO, l[i]);
                                }
#pragma unroll
                                for (int i = 0; i < 8; ++i) x[i] = fmaf(g.beta, l[i], x[i]);
                            }
                            if (PHASE == POLY && diagonal(t)) {
#pragma unroll
                                for (int i = 0; i < 8; ++i)
                                    if (first + 8 * o + i == row) x[i] += g.diag;
                            }
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                const __half2 hi = __floats2half2_rn(x[2 * i], x[2 * i + 1]);
                                packed[0][16 * h + 4 * j + i] = *reinterpret_cast<const uint32_t*>(&hi);
                                if constexpr (OUT > 1) {
                                    const float2 f = __half22float2(hi);
                                    const __half2 lo = __floats2half2_rn((x[2 * i] - f.x) * LO, (x[2 * i + 1] - f.y) * LO);
                                    packed[1][16 * h + 4 * j + i] = *reinterpret_cast<const uint32_t*>(&lo);
                                }
                            }
                        }
                    }
#pragma unroll
                    for (int pl = 0; pl < OUT; ++pl)
                        if (TERMS > 1 || PHASE != APPLY || pl == 0 || g.keep_lo) emit(packed[pl], &c.out[pl], col0, row0, t.z);
                    if (SYM && !diagonal(t)) {
#pragma unroll
                        for (int pl = 0; pl < OUT; ++pl) emit_mirror(packed[pl], &c.mirror[pl], col0, row0, t.z);
                    }
                }
            }
            if constexpr (!KEEP) {
                tc_fence_before();
                __syncwarp();
                if (lane == 0 && alive) mbar_arrive_cluster(mapa_shared(tempty_bar(acc), 0));
                if (++acc == 2) { acc = 0; acc_phase ^= 1u; }
            }
        }
        if (lane == 0) bulk_wait_read<0>();            // (the grid's end makes what was stored visible)
    }

    // ------------------------------ teardown ---------------------------------------------------
    tc_fence_before();
    __syncthreads();
    if (*abort_flag) {
        // copies may still be in flight into this CTA's shared memory: give them time to land
        for (int i = 0; i < 1000; ++i) __nanosleep(1000);
        __syncthreads();
    }
    cluster_sync_all();
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc_pair(tmem_base, 2 * TN);
    }
}

// The parts of A's tiles added up: A = alpha sum, into both triangles.  A CTA takes what an epilogue
// warp left, 32 rows x 128 or 64 columns.
constexpr int FOLD_THREADS = 256;
struct FoldClass {
    const float4* partial;
    __half* out[2];
    int m, ld, tiles, splits, first;      // tiles of one matrix; first CTA
};
struct FoldArgs {
    FoldClass c[MAX_CLASSES];
    int classes;
    float alpha;
};
template <int PLANES, int TN>
__global__ void __launch_bounds__(FOLD_THREADS) fold_kernel(const __grid_constant__ FoldArgs a) {
    constexpr int CW = TN / 2, EACH = CW / 32;           // float4 of a thread
    __shared__ __align__(16) __half s_tile[PLANES][32][CW + 8];
    grid_launch_dependents();
    int k = 0;
#pragma unroll
    for (int i = 1; i < MAX_CLASSES; ++i)
        if (i < a.classes && (int)blockIdx.x >= a.c[i].first) k = i;
    const FoldClass& c = a.c[k];
    const int b = (int)blockIdx.x - c.first, region = b & 15, tile = b >> 4;
    const int z = tile / c.tiles, r = tile - z * c.tiles;
    int m, n;
    lower_tile<TN>(r, &m, &n);
    const int rank = region >> 3, w = region & 7;
    // (warp 4 + w of the epilogue: lane quadrant w & 3, column half w >> 2)
    const int row0 = m * TILE + rank * BM + (w & 3) * 32, col0 = n * TN + (w >> 2) * CW;
    grid_dependency_wait();
    if (row0 >= c.m || col0 >= c.m) return;
    const float4* from = c.partial + (size_t)tile * c.splits * SLOT<TN> + region * (CW / 4) * 32;
    float4 v[EACH];
#pragma unroll
    for (int e = 0; e < EACH; ++e) v[e] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
    for (int s = 0; s < c.splits; ++s) {
#pragma unroll
        for (int e = 0; e < EACH; ++e) {
            const float4 p = from[(size_t)s * SLOT<TN> + threadIdx.x + FOLD_THREADS * e];
            v[e].x += p.x;
            v[e].y += p.y;
            v[e].z += p.z;
            v[e].w += p.w;
        }
    }
#pragma unroll
    for (int e = 0; e < EACH; ++e) {
        const int i = threadIdx.x + FOLD_THREADS * e, row = i & 31, col = 4 * (i >> 5);
        const float x[4] = {a.alpha * v[e].x, a.alpha * v[e].y, a.alpha * v[e].z, a.alpha * v[e].w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const __half h = __float2half_rn(x[j]);
            s_tile[0][row][col + j] = h;
            if (PLANES > 1) s_tile[PLANES - 1][row][col + j] = __float2half_rn((x[j] - __half2float(h)) * LO);
        }
    }
    __syncthreads();
#pragma unroll
    for (int pl = 0; pl < PLANES; ++pl) {
        __half* out = c.out[pl] + (size_t)z * c.m * c.ld;
#pragma unroll
        for (int e = 0; e < CW / 64; ++e) {
            const int i = threadIdx.x + FOLD_THREADS * e;
            const int row = i / (CW / 8), col = 8 * (i % (CW / 8));
            if (row0 + row < c.m && col0 + col < c.ld)
                *reinterpret_cast<uint4*>(out + (size_t)(row0 + row) * c.ld + col0 + col) =
                    *reinterpret_cast<const uint4*>(&s_tile[pl][row][col]);
            if (m == n * TN / TILE) continue;
            const int mc = i >> 2, mr = 8 * (i & 3);   // column of the tile, eight of its rows
            if (col0 + mc >= c.m || row0 + mr >= c.ld) continue;
            __half h[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) h[j] = s_tile[pl][mr + j][mc];
            *reinterpret_cast<uint4*>(out + (size_t)(col0 + mc) * c.ld + row0 + mr) = *reinterpret_cast<const uint4*>(h);
        }
    }
}

// ---- around the iteration: elementwise, a matrix in pieces of PIECE octets -------------------------
// An octet is eight columns of a row (from a multiple of eight on; the row's last one may be short): 16 bytes
// of a plane, and of the matrix itself where its rows have a multiple of eight columns.
constexpr int EL_THREADS = 256;
constexpr int PER_THREAD = 1;             // octets under way at once (more of them cost the occupancy that hides
constexpr int TURNS = 4;                  // loads better: 43 x 768 x 2048 without the products 169 us with 1, 244 with 2, 316 with 4)
constexpr int PIECE = EL_THREADS * PER_THREAD * TURNS;

// Matrices of one stack in a launch.
struct Part {
    void* param;                          // or the result of an orthogonalisation
    float* master;
    const void* grad;                     // or its input
    float* momentum;                      // null: none
    __half *hi, *lo;                      // their planes (a result that is rounded to bf16 has no lo)
    double* norms;                        // [matrices, pieces]
    long long first;                      // number of the first of their pieces in the launch
    int rows, cols, ld, pieces;           // pieces: of one matrix
    float decay, scale;
};
struct ElemArgs {
    int parts, nesterov;
    float momentum, eps, lr;
    float up, unscale;                    // of X: times LEAST_SCALE to the operands' scale, and back to X
    const float *grad_scale, *lr_now;
    Part part[MAX_STACKS];
};
// The piece of a CTA: its stack and matrix.
struct Piece {
    const Part* part;
    int matrix, piece, octets;            // octets of a row
    long long base;                       // elements of the matrices before this one
};
__device__ __forceinline__ Piece find_piece(const ElemArgs& a) {
    int i = 0;
    for (int step = MAX_STACKS / 2; step > 0; step >>= 1)
        if (i + step < a.parts && a.part[i + step].first <= (long long)blockIdx.x) i += step;
    Piece p;
    p.part = &a.part[i];
    const uint32_t within = (uint32_t)(blockIdx.x - p.part->first), pieces = (uint32_t)p.part->pieces;
    p.matrix = (int)(within / pieces);
    p.piece = (int)(within - (uint32_t)p.matrix * pieces);
    p.octets = p.part->ld >> 3;
    p.base = (long long)p.matrix * p.part->rows * p.part->cols;
    return p;
}
// A thread's octet e of a piece: where it lies in the matrix and in the planes, and its elements.
struct Place {
    long long at, in_plane;
    int valid;
};
template <bool VEC> __device__ __forceinline__ Place octet_of(const Piece& p, int turn, int e) {
    // (below 2^25)
    const uint32_t i = (uint32_t)p.piece * PIECE + (uint32_t)((turn * PER_THREAD + e) * EL_THREADS) + threadIdx.x;
    Place t;
    t.in_plane = (long long)i * 8;
    if (VEC) {
        t.at = t.in_plane;
        t.valid = i < (uint32_t)(p.part->rows * p.octets) ? 8 : 0;
    } else {
        const uint32_t r = i / (uint32_t)p.octets, o = i - r * (uint32_t)p.octets;
        t.at = (long long)r * p.part->cols + 8 * o;
        t.valid = r < (uint32_t)p.part->rows ? min(8, p.part->cols - 8 * (int)o) : 0;
    }
    return t;
}
template <bool VEC, typename T> __device__ __forceinline__ void get_octet(const T* p, int valid, float (&f)[8]) {
    if (VEC) {
        load8(p, f);
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) f[k] = k < valid ? to_f32(p[k]) : 0.f;
    }
}
template <bool VEC, typename T> __device__ __forceinline__ void put_octet(T* p, int valid, const float (&f)[8]) {
    if (VEC) {
        store8(p, f);
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (k < valid) p[k] = from_f32<T>(f[k]);
    }
}
// Gradient and momentum of a thread's octets, all of them under way at once.
template <bool VEC, typename G>
__device__ __forceinline__ void get_pair(const Piece& p, int turn, const G* grad, const float* mom, Place (&t)[PER_THREAD],
                                         float (&g)[PER_THREAD][8], float (&m)[PER_THREAD][8]) {
#pragma unroll
    for (int e = 0; e < PER_THREAD; ++e) {
        t[e] = octet_of<VEC>(p, turn, e);
#pragma unroll
        for (int k = 0; k < 8; ++k) g[e][k] = m[e][k] = 0.f;
        if (t[e].valid > 0) {
            get_octet<VEC>(grad + t[e].at, t[e].valid, g[e]);
            if (mom) get_octet<VEC>(mom + t[e].at, t[e].valid, m[e]);
        }
    }
}

// First pass: the momentum's update and the sum of u^2 of every piece.
template <bool VEC, typename G>
__device__ __forceinline__ double norm_piece(const ElemArgs& a, const Piece& p, float gs) {
    const G* grad = static_cast<const G*>(p.part->grad) + p.base;
    float* mom = p.part->momentum ? p.part->momentum + p.base : nullptr;
    double sum = 0.0;
#pragma unroll 1
    for (int turn = 0; turn < TURNS; ++turn) {
        Place t[PER_THREAD];
        float g[PER_THREAD][8], m[PER_THREAD][8];
        get_pair<VEC>(p, turn, grad, mom, t, g, m);
#pragma unroll
        for (int e = 0; e < PER_THREAD; ++e) {
            if (mom) {
#pragma unroll
                for (int k = 0; k < 8; ++k) m[e][k] = __fadd_rn(__fmul_rn(a.momentum, m[e][k]), __fmul_rn(g[e][k], gs));
                if (t[e].valid > 0) put_octet<VEC>(mom + t[e].at, t[e].valid, m[e]);
            }
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const double u = (double)direction(a.nesterov, a.momentum, mom != nullptr, __fmul_rn(g[e][k], gs), m[e][k]);
                sum += u * u;
            }
        }
    }
    return sum;
}
template <typename G>
__global__ void __launch_bounds__(EL_THREADS, 6) norm_kernel(const __grid_constant__ ElemArgs a) {
    __shared__ double s_sum[EL_THREADS / 32];
    grid_launch_dependents();
    const Piece p = find_piece(a);
    grid_dependency_wait();
    float gs;
    double sum = 0.0;
    if (scale_of(a.grad_scale, &gs))
        sum = p.part->cols % 8 == 0 ? norm_piece<true, G>(a, p, gs) : norm_piece<false, G>(a, p, gs);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if ((threadIdx.x & 31) == 0) s_sum[threadIdx.x >> 5] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        sum = 0.0;
        for (int i = 0; i < EL_THREADS / 32; ++i) sum += s_sum[i];
        p.part->norms[(size_t)p.matrix * p.part->pieces + p.piece] = sum;
    }
}

// Second pass: X = u / (|u| + eps) into the planes.
template <bool VEC, typename G>
__device__ __forceinline__ void start_piece(const ElemArgs& a, const Piece& p, float gs, float inv) {
    const G* grad = static_cast<const G*>(p.part->grad) + p.base;
    const float* mom = p.part->momentum ? p.part->momentum + p.base : nullptr;
    const long long plane = (long long)p.matrix * p.part->rows * p.part->ld;
#pragma unroll 1
    for (int turn = 0; turn < TURNS; ++turn) {
        Place t[PER_THREAD];
        float g[PER_THREAD][8], m[PER_THREAD][8];
        get_pair<VEC>(p, turn, grad, mom, t, g, m);
#pragma unroll
        for (int e = 0; e < PER_THREAD; ++e) {
            if (t[e].valid <= 0) continue;
            uint4 h, l;
            __half2* hp = reinterpret_cast<__half2*>(&h);
            __half2* lp = reinterpret_cast<__half2*>(&l);
#pragma unroll
            for (int k = 0; k < 8; k += 2) {
                const float x0 = direction(a.nesterov, a.momentum, mom != nullptr, __fmul_rn(g[e][k], gs), m[e][k]) * inv * a.up;
                const float x1 =
                    direction(a.nesterov, a.momentum, mom != nullptr, __fmul_rn(g[e][k + 1], gs), m[e][k + 1]) * inv * a.up;
                hp[k / 2] = __floats2half2_rn(x0, x1);
                const float2 f = __half22float2(hp[k / 2]);
                lp[k / 2] = __floats2half2_rn((x0 - f.x) * LO, (x1 - f.y) * LO);
            }
            *reinterpret_cast<uint4*>(p.part->hi + plane + t[e].in_plane) = h;
            *reinterpret_cast<uint4*>(p.part->lo + plane + t[e].in_plane) = l;
        }
    }
}
template <typename G>
__global__ void __launch_bounds__(EL_THREADS, 6) start_kernel(const __grid_constant__ ElemArgs a) {
    __shared__ double s_sum[EL_THREADS / 32];
    grid_launch_dependents();
    const Piece p = find_piece(a);
    grid_dependency_wait();
    float gs;
    if (!scale_of(a.grad_scale, &gs)) return;          // the step is skipped: the planes are not looked at
    const int pieces = p.part->pieces;
    double sum = 0.0;
    for (int i = threadIdx.x; i < pieces; i += EL_THREADS) sum += p.part->norms[(size_t)p.matrix * pieces + i];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if ((threadIdx.x & 31) == 0) s_sum[threadIdx.x >> 5] = sum;
    __syncthreads();
    sum = 0.0;
#pragma unroll
    for (int i = 0; i < EL_THREADS / 32; ++i) sum += s_sum[i];
    const float inv = start_scale(sum, a.eps);
    if (p.part->cols % 8 == 0) start_piece<true, G>(a, p, gs, inv);
    else start_piece<false, G>(a, p, gs, inv);
}

// Behind the iteration: the result, or the weights' update.
template <bool VEC, typename P, bool MASTER, bool STEP>
__device__ __forceinline__ void finish_piece(const ElemArgs& a, const Piece& p) {
    P* out = static_cast<P*>(p.part->param) + p.base;
    float* master = MASTER ? p.part->master + p.base : nullptr;
    const long long plane = (long long)p.matrix * p.part->rows * p.part->ld;
    const float lr = a.lr_now ? *a.lr_now : a.lr;
    const float keep = 1.f - lr * p.part->decay, rate = lr * p.part->scale * a.unscale;
#pragma unroll 1
    for (int turn = 0; turn < TURNS; ++turn) {
        Place t[PER_THREAD];
        uint4 hi[PER_THREAD], lo[PER_THREAD];
        float w[PER_THREAD][8];
#pragma unroll
        for (int e = 0; e < PER_THREAD; ++e) {
            t[e] = octet_of<VEC>(p, turn, e);
            if (t[e].valid <= 0) continue;
            hi[e] = *reinterpret_cast<const uint4*>(p.part->hi + plane + t[e].in_plane);
            lo[e] = make_uint4(0u, 0u, 0u, 0u);
            if (p.part->lo) lo[e] = *reinterpret_cast<const uint4*>(p.part->lo + plane + t[e].in_plane);
            if (MASTER) get_octet<VEC>(master + t[e].at, t[e].valid, w[e]);
            else if (STEP) get_octet<VEC>(out + t[e].at, t[e].valid, w[e]);
        }
#pragma unroll
        for (int e = 0; e < PER_THREAD; ++e) {
            if (t[e].valid <= 0) continue;
            float o[8], l[8];
            half8(hi[e], o);
            half8(lo[e], l);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                o[k] = fmaf(l[k], 1.f / LO, o[k]);
                w[e][k] = STEP ? w[e][k] * keep - rate * o[k] : o[k] * a.unscale;
            }
            if (MASTER) put_octet<VEC>(master + t[e].at, t[e].valid, w[e]);
            put_octet<VEC>(out + t[e].at, t[e].valid, w[e]);
        }
    }
}
template <typename P, bool MASTER, bool STEP>
__global__ void __launch_bounds__(EL_THREADS, 6) finish_kernel(const __grid_constant__ ElemArgs a) {
    grid_launch_dependents();
    const Piece p = find_piece(a);
    grid_dependency_wait();
    float gs;
    if (!scale_of(a.grad_scale, &gs)) return;
    if (p.part->cols % 8 == 0) finish_piece<true, P, MASTER, STEP>(a, p);
    else finish_piece<false, P, MASTER, STEP>(a, p);
}

// ---- host side ------------------------------------------------------------------------------------
constexpr int MAX_SIDE = 16384;
constexpr float LEAST_EPS = 4e-36f;       // below it LEAST_SCALE / (norm + eps) could pass float32's range
constexpr int MAX_BATCH = 1 << 24, MAX_MATRICES = 1 << 27;   // (the latter times the CTAs of a cluster: a grid's limit)
constexpr size_t ROUND_BYTES = 512u << 20;          // workspace of a round, unless one matrix needs more

struct Coefs {
    int steps;
    float scale;                                     // of the operands
    float c[MAX_STEPS][3];
};
// The iteration's coefficients, if fp16 can hold its iterates: from singular values in [0, 1] on, X stays
// within 16, A, b A + c A^2 and a + b A + c A^2 within 60 (a bound on the norm bounds every element).
static bool read_coefs(int32_t steps, const double* given, Coefs* out) {
    if (steps < 1 || steps > MAX_STEPS) return false;
    out->steps = steps;
    double top = 1.0, most = 1.0;
    for (int k = 0; k < steps; ++k) {
        const double a = given ? given[3 * k] : 3.4445, b = given ? given[3 * k + 1] : -4.7750,
                     c = given ? given[3 * k + 2] : 2.0315;
        out->c[k][0] = (float)a;
        out->c[k][1] = (float)b;
        out->c[k][2] = (float)c;
        if (!given) continue;                        // (X within 1.3, the others within 3.4445 = a)
        if (!std::isfinite(a) || !std::isfinite(b) || !std::isfinite(c)) return false;
        double next = 0.0, poly = 0.0;
        for (int i = 0; i <= 256; ++i) {
            const double s = top * i / 256, t = s * s, p = b * t + c * t * t;
            next = std::fmax(next, std::fabs(s * (a + p)));
            poly = std::fmax(poly, std::fmax(std::fabs(p), std::fabs(a + p)));
        }
        if (!(next <= 16.0) || !(poly <= 60.0) || !(top * top <= 60.0)) return false;
        most = std::fmax(std::fmax(most, next), std::fmax(poly, top * top));
        top = next;
    }
    out->scale = MOST_SCALE;
    while (out->scale > LEAST_SCALE && out->scale * most > MAX_HALF) out->scale *= 0.5f;
    return true;
}

struct Problem {                                     // matrices of one shape
    int rows, cols, m, ld, ldm, terms;
    bool tall;
    int pieces;
};
static Problem problem_of(int rows, int cols, int terms) {
    Problem p;
    p.rows = rows;
    p.cols = cols;
    p.tall = rows > cols;
    p.m = rows < cols ? rows : cols;
    p.ld = (int)round_up((size_t)cols, 8);
    p.ldm = (int)round_up((size_t)p.m, 8);
    p.terms = terms;
    p.pieces = (int)(((long long)rows * (p.ld / 8) + PIECE - 1) / PIECE);
    return p;
}
// Places of `count` matrices in the workspace: X twice, A and B, sums.
struct Layout {
    size_t hi[2], lo[2], a[2], b[2], norms, total;
};
static Layout layout(const Problem& p, long long count) {
    Layout w;
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t here = at;
        at += round_up(bytes, 256);
        return here;
    };
    const size_t x = (size_t)count * p.rows * p.ld * 2, s = (size_t)count * p.m * p.ldm * 2;
    w.hi[0] = take(x);
    w.hi[1] = take(x);
    w.lo[0] = take(x);
    w.lo[1] = p.terms > 1 ? take(x) : w.lo[0];       // not an operand: a tile replaces its own
    w.a[0] = take(s);
    w.a[1] = p.terms > 1 ? take(s) : w.a[0];
    w.b[0] = take(s);
    w.b[1] = p.terms > 1 ? take(s) : w.b[0];
    w.norms = take((size_t)count * p.pieces * sizeof(double));
    w.total = at;
    return w;
}

// fp16 tensor [count, rows, cols] with row stride ld.
static bool make_map(CUtensorMap* m, const void* ptr, int count, int rows, int cols, int ld, int box_cols,
                     int box_rows, bool swizzle) {
    EncodeTiledFn fn = encode_fn();
    if (!fn) return false;
    cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)rows, (cuuint64_t)count};
    cuuint64_t strides[2] = {(cuuint64_t)ld * 2, (cuuint64_t)ld * rows * 2};
    cuuint32_t box[3] = {(cuuint32_t)box_cols, (cuuint32_t)box_rows, 1};
    cuuint32_t es[3] = {1, 1, 1};
    return fn(m, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, const_cast<void*>(ptr), dims, strides, box, es,
              CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_NONE,
              CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// CTA pairs of a kernel that can be resident at once (one CTA per SM), asked once per kernel and device; -1: a
// kernel that splits the register file, of which a launch has too few registers for its split.
static int resident_pairs(void (*kern)(GemmArgs), bool split, int smem, int (&cached)[64]) {
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return 0;
    if (cached[dev] == 0) {
        cudaFuncAttributes attrs;
        if (cudaFuncGetAttributes(&attrs, kern) != cudaSuccess) return 0;
        if (split && attrs.numRegs < LAUNCH_REGS) return cached[dev] = -1;
        if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) != cudaSuccess) return 0;
        cudaLaunchConfig_t cfg = {};
        cudaLaunchAttribute attr[1];
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim.x = 2;
        attr[0].val.clusterDim.y = 1;
        attr[0].val.clusterDim.z = 1;
        cfg.gridDim = dim3(2 * (sm_count() / 2));
        cfg.blockDim = dim3(THREADS);
        cfg.dynamicSmemBytes = smem;
        cfg.attrs = attr;
        cfg.numAttrs = 1;
        int n = 0;
        if (cudaOccupancyMaxActiveClusters(&n, kern, &cfg) != cudaSuccess || n <= 0) return 0;
        cached[dev] = n < sm_count() / 2 ? n : sm_count() / 2;
    }
    return cached[dev];
}
template <int PHASE, int TERMS, int TN> static int pairs_of() {
    using R = Ring<TERMS, TN>;
    static int cached[64] = {0};
    return resident_pairs(gemm_kernel<PHASE, TERMS, TN>, R::SPLIT, R::SMEM_BYTES, cached);
}
template <int TERMS, int TN> static int least_pairs() {
    return std::min({pairs_of<GRAM, TERMS, TN>(), pairs_of<POLY, TERMS, TN>(), pairs_of<APPLY, TERMS, TN>()});
}
// Tiles of 256 columns with three products need the registers of their split; how many a kernel gets is the
// compiler's choice (168 now).  Without them everything runs in tiles of 128.
static bool wide_runs(int terms) {
    if (terms == 1) return true;
    const int pairs = least_pairs<3, 256>();
    if (pairs == 0) cudaGetLastError();              // (a machine without a GPU asks for workspaces too)
    return pairs >= 0;
}
// Whether every product that a call may come to can be launched: asked before its first launch, so that what is
// refused leaves everything as it was.
static bool products_run() {
    static PerDevice ready;
    if (ready.done()) return true;
    if (least_pairs<1, 128>() <= 0 || least_pairs<1, 256>() <= 0 || least_pairs<3, 128>() <= 0 || least_pairs<3, 256>() == 0)
        return false;
    ready.mark();
    return true;
}

template <int PHASE, int TERMS, int TN> static r3_status launch_gemm(const GemmArgs& g, cudaStream_t cs) {
    auto kern = gemm_kernel<PHASE, TERMS, TN>;
    using R = Ring<TERMS, TN>;
    const int pairs = pairs_of<PHASE, TERMS, TN>();
    if (pairs <= 0) return R3_ERR_CUDA;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = 2;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.gridDim = dim3(2 * (g.items < pairs ? g.items : pairs));
    cfg.blockDim = dim3(THREADS);
    cfg.dynamicSmemBytes = R::SMEM_BYTES;
    cfg.stream = cs;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, kern, g) == cudaSuccess ? R3_OK : R3_ERR_CUDA;
}

// The matrices of one shape in a round.
struct Class {
    Problem p;
    int count;
    uint8_t* ws;
};

static int square_tiles(const Problem& p, int tn) {
    const int t = (p.m + TILE - 1) / TILE;
    return tn == TILE ? t * (t + 1) / 2 : t * (t - 1) + (p.m + tn - 1) / tn;
}
static int all_tiles(const Problem& p, int tn) { return (p.rows + TILE - 1) / TILE * ((p.cols + tn - 1) / tn); }
static int gram_blocks(const Problem& p) { return ((p.tall ? p.rows : p.cols) + BK - 1) / BK; }
// A round's tiles and the parts of its long sums, by estimates of the time in 20ths of a k block's with 256
// columns (0.27 us; three products 0.8): a CTA pair's item costs its k blocks and what stands around them.
// Tiles of 128 columns take 13 (11) of a block and half of the rest, and are twice as many: few tiles spread over
// more of the GPU (us, 256 -> 128 columns: 1024 x 1024 f32 354 -> 236, 768 x 2048 bf16 214 -> 147, 16 x 300 x 600 bf16
// 206 -> 161, 2048 x 4096 f32 890 -> 810, 4 x 1024 x 1024 bf16 199 -> 210, 8 x 768 x 2048 bf16 281 -> 323, 4096 x 4096
// bf16 1128 -> 1472).
constexpr int MAX_SPLITS = 8;
struct Cut {
    int tn, part;                         // columns of the tiles; k blocks of A = X X^T that a CTA pair takes at a time
};
static long long waves(long long items) {
    const int pairs = sm_count() / 2;
    return (items + pairs - 1) / pairs;
}
static Cut cut_of(const Class* classes, int n, int terms) {
    Cut best = {256, 1};
    long long least = -1;
    int longest = 0, side = 0;
    for (int i = 0; i < n; ++i) {
        longest = std::max(longest, gram_blocks(classes[i].p));
        side = std::max(side, (classes[i].p.m + BK - 1) / BK);
    }
    for (int tn : {256, 128}) {
        if (tn == 256 && !wide_runs(terms)) continue;
        const int block = tn == 256 ? 20 : terms > 1 ? 11 : 13;
        const int around = (terms > 1 ? 80 : 220) * tn / 256;
        long long square = 0, all = 0;
        for (int i = 0; i < n; ++i) {
            square += (long long)square_tiles(classes[i].p, tn) * classes[i].count;
            all += (long long)all_tiles(classes[i].p, tn) * classes[i].count;
        }
        const long long others = (waves(square) + waves(all)) * (side * block + around);
        // parts cost a launch that adds them up, 3 to 4 us (150 x 4000 f32, 256 columns: 444 us whole, 248 in parts when it was taken)
        const int fold = terms > 1 ? 70 : 300;
        for (int splits = 1; splits <= MAX_SPLITS; ++splits) {
            const int part = (longest + splits - 1) / splits;
            long long items = 0, slots = 0;
            for (int i = 0; i < n; ++i) {
                const int parts = (gram_blocks(classes[i].p) + part - 1) / part;
                const long long here = (long long)square_tiles(classes[i].p, tn) * classes[i].count * parts;
                items += here;
                if (parts > 1) slots += here;
            }
            if (slots > 4LL * (sm_count() / 2)) break;
            const long long cost = others + waves(items) * (part * block + around) + (slots ? fold : 0);
            if (least < 0 || cost < least) {
                least = cost;
                best = {tn, part};
            }
        }
    }
    return best;
}
static size_t partial_bytes(const Class* classes, int n, int terms, const Cut& cut) {
    size_t slots = 0;
    for (int i = 0; i < n; ++i) {
        const int parts = (gram_blocks(classes[i].p) + cut.part - 1) / cut.part;
        if (parts > 1) slots += (size_t)square_tiles(classes[i].p, cut.tn) * classes[i].count * parts;
    }
    return slots * (TILE * cut.tn / 4) * sizeof(float4);
}

// The iteration on classes whose X stand in the planes 0; on return *at says which planes hold the results.
// part: k blocks of a part of X X^T; partial: partial_bytes of memory.
template <int TERMS, int TN>
static r3_status iterate(const Class* classes, int n, int part, bool coarse, uint8_t* partial, const Coefs& coefs,
                         int32_t* dev_status, int* at, cudaStream_t cs) {
    FoldArgs fold = {};
    int fold_ctas = 0;
    float4* next_partial = reinterpret_cast<float4*>(partial);
    GemmArgs gram[2], poly, apply[2];                // by the planes that hold X
    gram[0].items = gram[1].items = poly.items = apply[0].items = apply[1].items = 0;
    bool ok = true;
    for (int i = 0; i < n; ++i) {
        const Problem& p = classes[i].p;
        const int count = classes[i].count;
        const Layout w = layout(p, count);
        uint8_t* ws = classes[i].ws;
        const int tc = (p.cols + TN - 1) / TN;
        ClassArgs& q = poly.c[i];
        // an operand with consecutive k: 64 x 128 boxes; with k along the rows: 64 x 64, two per stage
        for (int pl = 0; pl < 2; ++pl) {
            const uint8_t* A = ws + w.a[pl];
            const uint8_t* B = ws + w.b[pl];
            CUtensorMap bk;                  // (a right operand takes TN / 2 rows at a time)
            ok = ok && make_map(&q.a[pl], A, count, p.m, p.m, p.ldm, 64, BM, true) &&
                 make_map(&bk, B, count, p.m, p.m, p.ldm, 64, BM, true) &&
                 make_map(&q.out[pl], B, count, p.m, p.m, p.ldm, 64, 32, true) &&
                 make_map(&q.mirror[pl], B, count, p.m, p.m, p.ldm, 32, 64, false);
            ok = ok && make_map(&q.b[pl], A, count, p.m, p.m, p.ldm, 64, TN / 2, true);
            CUtensorMap b_right;
            ok = ok && make_map(&b_right, B, count, p.m, p.m, p.ldm, 64, TN / 2, true);
            q.in[pl] = reinterpret_cast<const __half*>(A);
            for (int k = 0; k < 2; ++k) {
                const uint8_t* x = ws + (pl ? w.lo[k] : w.hi[k]);
                const uint8_t* y = ws + (pl ? w.lo[k ^ 1] : w.hi[k ^ 1]);
                CUtensorMap xk, xmn;
                ok = ok && make_map(&xk, x, count, p.rows, p.cols, p.ld, 64, BM, true) &&
                     make_map(&xmn, x, count, p.rows, p.cols, p.ld, 64, BK, true);
                ClassArgs& gr = gram[k].c[i];
                gr.a[pl] = p.tall ? xmn : xk;
                gr.b[pl] = p.tall || TN == 128 ? xmn : xk;     // (64 x 64 either way)
                if (k == 0)
                    ok = ok && make_map(&gr.out[pl], A, count, p.m, p.m, p.ldm, 64, 32, true) &&
                         make_map(&gr.mirror[pl], A, count, p.m, p.m, p.ldm, 32, 64, false);
                else
                    gr.out[pl] = gram[0].c[i].out[pl], gr.mirror[pl] = gram[0].c[i].mirror[pl];
                gr.in[pl] = nullptr;
                ClassArgs& ap = apply[k].c[i];
                ap.a[pl] = p.tall ? xk : bk;
                ap.b[pl] = p.tall ? b_right : xmn;
                ok = ok && make_map(&ap.out[pl], y, count, p.rows, p.cols, p.ld, 64, 32, true);
                ap.mirror[pl] = ap.out[pl];
                ap.in[pl] = reinterpret_cast<const __half*>(ws + w.lo[k]);
            }
        }
        auto square = [&](GemmArgs& g, int kblocks, bool mn) {
            ClassArgs& c = g.c[i];
            c.in_plane = (long long)p.m * p.ldm;
            c.in_ld = p.ldm;
            c.rows = c.cols = p.m;
            c.tiles_n = 0;
            c.tiles = square_tiles(p, TN);
            c.first_item = g.items;
            c.kblocks = kblocks;
            c.a_mn = c.b_mn = mn;
            c.splits = 1;
            g.items += c.tiles * count;
        };
        const int km = (p.m + BK - 1) / BK;
        square(poly, km, false);
        for (int k = 0; k < 2; ++k) {
            square(gram[k], gram_blocks(p), p.tall);
            ClassArgs& gr = gram[k].c[i];
            gr.per_split = part;
            gr.splits = (gr.kblocks + part - 1) / part;
            gr.partial = next_partial;
            gram[k].items += gr.tiles * count * (gr.splits - 1);
            ClassArgs& c = apply[k].c[i];
            c.in_plane = (long long)p.rows * p.ld;
            c.in_ld = p.ld;
            c.rows = p.rows;
            c.cols = p.cols;
            c.tiles_n = tc;
            c.tiles = all_tiles(p, TN);
            c.first_item = apply[k].items;
            c.kblocks = km;
            c.a_mn = 0;
            c.b_mn = !p.tall;
            c.splits = 1;
            apply[k].items += c.tiles * count;
        }
        const ClassArgs& gr = gram[0].c[i];
        if (gr.splits > 1) {
            FoldClass& f = fold.c[fold.classes++];
            f.partial = next_partial;
            f.out[0] = reinterpret_cast<__half*>(ws + w.a[0]);
            f.out[1] = reinterpret_cast<__half*>(ws + w.a[1]);
            f.m = p.m;
            f.ld = p.ldm;
            f.tiles = gr.tiles;
            f.splits = gr.splits;
            f.first = fold_ctas;
            fold_ctas += gr.tiles * count * 2 * EPI_WARPS;
            next_partial += (size_t)gr.tiles * count * gr.splits * SLOT<TN>;
        }
    }
    fold.alpha = 1.f / coefs.scale;
    if (!ok) return R3_ERR_CUDA;
    for (GemmArgs* g : {&gram[0], &gram[1], &poly, &apply[0], &apply[1]}) {
        g->classes = n;
        g->alpha = 1.f / coefs.scale;
        g->beta = g->diag = 0.f;
        g->keep_lo = 1;
        g->dev_status = dev_status;
    }
    // `coarse`, a result that is rounded to bf16: what X's rounding to fp16 does is multiplied by a in the last step,
    // 3.4 2^-13 = 4e-4 of its rms against the 1.7e-3 of that (by a^2 in the one before it).  So the last step's X
    // needs no lo plane where a is of that size, and the result has none (384 x 768 x 2048 under load 15.07 -> 14.53 ms).
    const bool last_without = coarse && std::fabs(coefs.c[coefs.steps - 1][0]) <= 4.f;
    int k = 0;
    for (int step = 0; step < coefs.steps; ++step, k ^= 1) {
        const float *c = coefs.c[step];
        poly.alpha = c[2] / coefs.scale;
        poly.beta = c[1];
        poly.diag = c[0] * coefs.scale;
        apply[k].beta = c[0] / LO;                   // (of the lo plane)
        if (TERMS == 1) {
            const int left = coefs.steps - step;
            apply[k].keep_lo = left > 2 || (left == 2 ? !last_without : !coarse);
            if (last_without && step > 0 && step + 1 == coefs.steps)
                for (int i = 0; i < n; ++i) apply[k].c[i].in[0] = nullptr;
        }
        r3_status st = launch_gemm<GRAM, TERMS, TN>(gram[k], cs);
        if (st == R3_OK && fold_ctas &&
            launch_dependent(fold_kernel<TERMS == 1 ? 1 : 2, TN>, dim3(fold_ctas), dim3(FOLD_THREADS), 0, cs, fold) != cudaSuccess)
            st = R3_ERR_CUDA;
        if (st == R3_OK) st = launch_gemm<POLY, TERMS, TN>(poly, cs);
        if (st == R3_OK) st = launch_gemm<APPLY, TERMS, TN>(apply[k], cs);
        if (st != R3_OK) return st;
    }
    *at = k;
    return R3_OK;
}

struct Job {
    int param_dtype, grad_dtype, nesterov, terms;    // terms: as the caller has them (terms_of)
    bool master, step;
    float momentum, eps, lr;
    const float *grad_scale, *lr_now;
};
static r3_status run_small_stacks(const Job& job, const Coefs& coefs, const r3_muon_stack* const* ss, int n,
                                  int terms, int cluster, int matrices, int32_t* dev_status, cudaStream_t cs) {
    SmallArgs a = {};
    a.stacks = n;
    a.cluster = cluster;
    a.steps = coefs.steps;
    for (int k = 0; k < coefs.steps; ++k)
        for (int j = 0; j < 3; ++j) a.coefs[k][j] = coefs.c[k][j];
    a.grad_dtype = job.grad_dtype;
    a.param_dtype = job.param_dtype;
    a.step = job.step;
    a.nesterov = job.nesterov;
    a.momentum = job.momentum;
    a.eps = job.eps;
    a.lr = job.lr;
    a.scale = coefs.scale;
    a.grad_scale = job.grad_scale;
    a.lr_now = job.lr_now;
    a.dev_status = dev_status;
    int first = 0;
    for (int i = 0; i < n; ++i) {
        const r3_muon_stack& s = *ss[i];
        a.stack[i] = {s.param, s.master, s.grad, s.momentum, first, s.rows, s.cols, s.weight_decay, s.scale};
        first += s.batch;
    }
    return run_small(a, terms, matrices, cs);
}

// Matrices [begin, begin + count) of a stack, in class `cls` of the round as numbers `at` and on.
struct Slice {
    const r3_muon_stack* stack;
    int begin, count, cls, at;
};
struct Round {
    Class cls[MAX_CLASSES];
    Slice slice[MAX_STACKS];
    int classes = 0, slices = 0, terms = 0;
    size_t bytes = 0;
};
static r3_status run_round(const Job& job, const Coefs& coefs, Round& r, uint8_t* ws, int32_t* dev_status,
                           cudaStream_t cs) {
    for (int i = 0; i < r.classes; ++i) {
        r.cls[i].ws = ws;
        ws += layout(r.cls[i].p, r.cls[i].count).total;
    }
    ElemArgs a = {};
    a.parts = r.slices;
    a.nesterov = job.nesterov;
    a.momentum = job.momentum;
    a.eps = job.eps;
    a.lr = job.lr;
    a.up = coefs.scale / LEAST_SCALE;
    a.unscale = 1.f / coefs.scale;
    a.grad_scale = job.grad_scale;
    a.lr_now = job.lr_now;
    const size_t psize = job.param_dtype == R3_BF16 ? 2 : 4, gsize = job.grad_dtype == R3_BF16 ? 2 : 4;
    long long pieces = 0;
    for (int i = 0; i < r.slices; ++i) {
        const Slice& s = r.slice[i];
        const Problem& p = r.cls[s.cls].p;
        const size_t off = (size_t)s.begin * p.rows * p.cols;
        Part& t = a.part[i];
        t.param = static_cast<uint8_t*>(s.stack->param) + off * psize;
        t.master = s.stack->master ? s.stack->master + off : nullptr;
        t.grad = static_cast<const uint8_t*>(s.stack->grad) + off * gsize;
        t.momentum = s.stack->momentum ? s.stack->momentum + off : nullptr;
        t.norms = reinterpret_cast<double*>(r.cls[s.cls].ws + layout(p, r.cls[s.cls].count).norms) +
                  (size_t)s.at * p.pieces;
        t.first = pieces;
        t.rows = p.rows;
        t.cols = p.cols;
        t.ld = p.ld;
        t.pieces = p.pieces;
        t.decay = s.stack->weight_decay;
        t.scale = s.stack->scale;
        pieces += (long long)s.count * p.pieces;
    }
    auto planes = [&](int at, bool with_lo) {
        for (int i = 0; i < r.slices; ++i) {
            const Slice& s = r.slice[i];
            const Class& c = r.cls[s.cls];
            const Layout w = layout(c.p, c.count);
            const size_t off = (size_t)s.at * c.p.rows * c.p.ld;
            a.part[i].hi = reinterpret_cast<__half*>(c.ws + w.hi[at]) + off;
            a.part[i].lo = with_lo ? reinterpret_cast<__half*>(c.ws + w.lo[at]) + off : nullptr;
        }
    };
    planes(0, true);
    const dim3 grid((unsigned)pieces), block(EL_THREADS);
    cudaError_t e;
    if (job.grad_dtype == R3_BF16) {
        e = launch_dependent(norm_kernel<__nv_bfloat16>, grid, block, 0, cs, a);
        if (e == cudaSuccess) e = launch_dependent(start_kernel<__nv_bfloat16>, grid, block, 0, cs, a);
    } else {
        e = launch_dependent(norm_kernel<float>, grid, block, 0, cs, a);
        if (e == cudaSuccess) e = launch_dependent(start_kernel<float>, grid, block, 0, cs, a);
    }
    if (e != cudaSuccess) return R3_ERR_CUDA;
    int at = 0;
    const Cut cut = cut_of(r.cls, r.classes, r.terms);
    const bool coarse = r.terms == 1 && job.param_dtype == R3_BF16 && !job.master;
    const bool narrow = cut.tn == 128;
    const auto steps = r.terms > 1 ? (narrow ? iterate<3, 128> : iterate<3, 256>)
                                     : (narrow ? iterate<1, 128> : iterate<1, 256>);
    const r3_status st = steps(r.cls, r.classes, cut.part, coarse, ws, coefs, dev_status, &at, cs);
    if (st != R3_OK) return st;
    planes(at, !coarse);
    if (!job.step)
        e = job.param_dtype == R3_BF16
                ? launch_dependent(finish_kernel<__nv_bfloat16, false, false>, grid, block, 0, cs, a)
                : launch_dependent(finish_kernel<float, false, false>, grid, block, 0, cs, a);
    else if (job.param_dtype == R3_F32)
        e = launch_dependent(finish_kernel<float, false, true>, grid, block, 0, cs, a);
    else
        e = job.master ? launch_dependent(finish_kernel<__nv_bfloat16, true, true>, grid, block, 0, cs, a)
                       : launch_dependent(finish_kernel<__nv_bfloat16, false, true>, grid, block, 0, cs, a);
    return e == cudaSuccess ? R3_OK : R3_ERR_CUDA;
}

// Products per product.  One that holds for a bf16 result does so by the errors of many operands evening out: on
// matrices of a short side they come to more than the rounding (simulated for Gaussian ones: 1 x 3 up to 4e-3, 2 x 3
// 7e-3, 4 x 64 5e-3, 8 x 8 4e-3, 16 x 16 2.5e-3, 16 x 300 1.7e-3 of the result's rms, the rounding being 1.7e-3),
// so these take three (8 x 2048 41 -> 53 us, 24 x 8 x 256 29 -> 39, 12 x 4000 84 -> 111).
constexpr int LEAST_SIDE = 16;
static int terms_of(const r3_muon_stack& s, int terms) { return std::min(s.rows, s.cols) < LEAST_SIDE ? 3 : terms; }

// Cuts stacks into launches: small(members, n, terms, cluster, matrices) for each group of the on-chip form, with as
// many products and CTAs per matrix, round(r) for each round of the others: up to MAX_CLASSES shapes of as many
// products, MAX_STACKS stacks and ROUND_BYTES of workspace (one matrix at least), shapes with long products first.
template <typename Small, typename Big>
static r3_status each_launch(const r3_muon_stack* ss, int32_t count, int terms, Small small, Big big) {
    std::vector<const r3_muon_stack*> little, large;
    for (int32_t i = 0; i < count; ++i)
        if (ss[i].batch > 0) (small_cluster(ss[i].rows, ss[i].cols) ? little : large).push_back(ss + i);
    auto kind = [&](const r3_muon_stack* s) { return 4 * small_cluster(s->rows, s->cols) + terms_of(*s, terms); };
    std::stable_sort(little.begin(), little.end(),
                     [&](const r3_muon_stack* x, const r3_muon_stack* y) { return kind(x) < kind(y); });
    for (size_t i = 0; i < little.size();) {
        size_t end = i;
        long long matrices = 0;
        for (; end < little.size() && end < i + MAX_STACKS && kind(little[end]) == kind(little[i]) &&
               matrices + little[end]->batch <= MAX_MATRICES; ++end)
            matrices += little[end]->batch;
        const r3_status st = small(little.data() + i, (int)(end - i), terms_of(*little[i], terms),
                                   small_cluster(little[i]->rows, little[i]->cols), (int)matrices);
        if (st != R3_OK) return st;
        i = end;
    }
    std::stable_sort(large.begin(), large.end(), [&](const r3_muon_stack* x, const r3_muon_stack* y) {
        const int tx = terms_of(*x, terms), ty = terms_of(*y, terms);
        const int nx = std::max(x->rows, x->cols), ny = std::max(y->rows, y->cols);
        return tx != ty ? tx < ty : nx != ny ? nx > ny : x->rows != y->rows ? x->rows > y->rows : x->cols > y->cols;
    });
    Round r;
    auto flush = [&]() {
        const r3_status st = r.slices ? big(r) : R3_OK;
        r = Round();
        return st;
    };
    for (const r3_muon_stack* s : large) {
        for (int begin = 0; begin < s->batch;) {
            const Problem p = problem_of(s->rows, s->cols, terms_of(*s, terms));
            const bool same = r.classes && r.cls[r.classes - 1].p.rows == s->rows && r.cls[r.classes - 1].p.cols == s->cols;
            const long long here = same ? r.cls[r.classes - 1].count : 0;
            const size_t before = r.bytes - (same ? layout(p, here).total : 0);
            // as many of the stack's matrices as fit
            long long n = 0;
            if (r.slices < MAX_STACKS && (same || r.classes < MAX_CLASSES) && (r.slices == 0 || r.terms == p.terms)) {
                const size_t one = layout(p, 1).total;
                const size_t room = ROUND_BYTES > r.bytes ? ROUND_BYTES - r.bytes : 0;
                n = std::min<long long>((long long)(room / one), s->batch - begin);
                if (n == 0 && r.slices == 0) n = 1;
            }
            if (n == 0) {
                const r3_status st = flush();
                if (st != R3_OK) return st;
                continue;
            }
            r.terms = p.terms;
            if (!same) r.cls[r.classes++] = {p, 0, nullptr};
            Class& c = r.cls[r.classes - 1];
            r.slice[r.slices++] = {s, begin, (int)n, r.classes - 1, c.count};
            c.count += (int)n;
            r.bytes = before + layout(p, c.count).total;
            begin += (int)n;
        }
    }
    return flush();
}
// Workspace of the largest launch (0 without a matrix).
static size_t workspace_bytes(const r3_muon_stack* ss, int32_t count, int terms) {
    size_t most = 0;
    each_launch(ss, count, terms,
                [&](const r3_muon_stack* const*, int, int, int, int) {
                    most = std::max(most, (size_t)256);
                    return R3_OK;
                },
                [&](Round& r) {
                    most = std::max(most, r.bytes + partial_bytes(r.cls, r.classes, r.terms, cut_of(r.cls, r.classes, r.terms)));
                    return R3_OK;
                });
    return most;
}
static r3_status run(const Job& job, const Coefs& coefs, const r3_muon_stack* ss, int32_t count, uint8_t* ws,
                     int32_t* dev_status, cudaStream_t cs) {
    const auto large = [](const r3_muon_stack& s) { return s.batch > 0 && small_cluster(s.rows, s.cols) == 0; };
    if (std::any_of(ss, ss + count, large) && !products_run()) return R3_ERR_CUDA;
    return each_launch(ss, count, job.terms,
                       [&](const r3_muon_stack* const* group, int n, int terms, int cluster, int matrices) {
                           return run_small_stacks(job, coefs, group, n, terms, cluster, matrices, dev_status, cs);
                       },
                       [&](Round& r) { return run_round(job, coefs, r, ws, dev_status, cs); });
}

static bool good_shape(int64_t batch, int64_t rows, int64_t cols) {
    return batch >= 0 && batch <= MAX_BATCH && rows >= 1 && rows <= MAX_SIDE && cols >= 1 && cols <= MAX_SIDE;
}
static bool good_type(int t) { return t == R3_F32 || t == R3_BF16; }

static r3_status check_ortho(const r3_orthogonal* c, Coefs* coefs) {
    if (!c || !good_shape(c->batch, c->rows, c->cols) || !good_type(c->in_dtype) || !good_type(c->out_dtype))
        return R3_ERR_INVALID_ARG;
    if ((c->products != 1 && c->products != 3) || !(c->eps >= 0.0 && c->eps < 1e30)) return R3_ERR_INVALID_ARG;
    return read_coefs(c->steps, c->coefs, coefs) ? R3_OK : R3_ERR_INVALID_ARG;
}
static r3_status check_muon(const r3_muon* c, const r3_muon_stack* ss, int32_t count, Coefs* coefs) {
    if (!c || count < 0 || (count > 0 && !ss)) return R3_ERR_INVALID_ARG;
    if (!good_type(c->param_dtype) || !good_type(c->grad_dtype) || (c->products != 1 && c->products != 3))
        return R3_ERR_INVALID_ARG;
    if (c->master && c->param_dtype != R3_BF16) return R3_ERR_INVALID_ARG;
    if (!(c->lr >= 0.0 && c->lr < 1e30) || !(c->momentum >= 0.0 && c->momentum < 1.0) ||
        !(c->eps >= 0.0 && c->eps < 1e30))
        return R3_ERR_INVALID_ARG;
    for (int32_t i = 0; i < count; ++i) {
        const r3_muon_stack& s = ss[i];
        if (!good_shape(s.batch, s.rows, s.cols) || !(s.weight_decay >= 0.f && s.weight_decay < 1e30f) ||
            !(s.scale >= 0.f && s.scale < 1e30f))
            return R3_ERR_INVALID_ARG;
    }
    return read_coefs(c->steps, c->coefs, coefs) ? R3_OK : R3_ERR_INVALID_ARG;
}
static r3_status check_buffers(const r3_muon* c, const r3_muon_stack* ss, int32_t count) {
    for (int32_t i = 0; i < count; ++i) {
        const r3_muon_stack& s = ss[i];
        if (s.batch == 0) continue;
        if (!s.param || !s.grad || !s.momentum || (c->master != 0) != (s.master != nullptr))
            return R3_ERR_INVALID_ARG;
        const void* ps[] = {s.param, s.master, s.grad, s.momentum};
        for (const void* p : ps)
            if (!aligned(p, 16)) return R3_ERR_INVALID_ARG;
    }
    return R3_OK;
}

// Two buffers on the same memory would be updated at once, in no order, and what is read there would change
// under the step.
static bool distinct(const r3_muon* c, const r3_muon_stack* ss, int32_t count, const float* grad_scale,
                     const float* lr) {
    struct Range {
        uintptr_t begin, end;
        bool written;
    };
    std::vector<Range> all;
    all.reserve((size_t)count * 4 + 2);
    auto add = [&](const void* p, size_t bytes, bool written) {
        const uintptr_t at = reinterpret_cast<uintptr_t>(p);
        if (p) all.push_back({at, at + bytes, written});
    };
    for (int32_t i = 0; i < count; ++i) {
        const r3_muon_stack& s = ss[i];
        const size_t n = (size_t)s.batch * s.rows * s.cols;
        if (n == 0) continue;
        add(s.param, n * (c->param_dtype == R3_BF16 ? 2 : 4), true);
        add(s.master, n * 4, true);
        add(s.momentum, n * 4, true);
        add(s.grad, n * (c->grad_dtype == R3_BF16 ? 2 : 4), false);
    }
    add(grad_scale, 4, false);
    add(lr, 4, false);
    std::sort(all.begin(), all.end(), [](const Range& x, const Range& y) { return x.begin < y.begin; });
    uintptr_t past = 0, past_written = 0;
    for (const Range& r : all) {
        if (r.begin < (r.written ? past : past_written)) return false;
        past = std::max(past, r.end);
        if (r.written) past_written = std::max(past_written, r.end);
    }
    return true;
}

}  // namespace ns
}  // namespace r3

// (host memory may run out: nothing of that leaves a C entry)
extern "C" size_t r3_orthogonalize_workspace_bytes(const r3_orthogonal* c) {
    using namespace r3::ns;
    Coefs coefs;
    if (check_ortho(c, &coefs) != R3_OK) return 0;
    const r3_muon_stack one = {nullptr, nullptr, nullptr, nullptr, c->batch, c->rows, c->cols, 0.f, 0.f};
    try {
        return workspace_bytes(&one, 1, c->products);
    } catch (...) {
        return 0;
    }
}

extern "C" r3_status r3_orthogonalize(const r3_orthogonal* c, const void* x, void* out, void* workspace,
                                      size_t ws_bytes, int32_t* dev_status, void* stream) {
    using namespace r3;
    using namespace r3::ns;
    Coefs coefs;
    const r3_status st = check_ortho(c, &coefs);
    if (st != R3_OK) return st;
    if (c->batch == 0) return R3_OK;
    if (!x || !out || !aligned(x, 16) || !aligned(out, 16) || !aligned(dev_status, 4)) return R3_ERR_INVALID_ARG;
    // the same buffer of one type, or no memory in common: later matrices are read after earlier results
    const size_t n = (size_t)c->batch * c->rows * c->cols;
    const uintptr_t from = reinterpret_cast<uintptr_t>(x), to = reinterpret_cast<uintptr_t>(out);
    const bool same = from == to && c->in_dtype == c->out_dtype;
    if (!same && from < to + n * (c->out_dtype == R3_BF16 ? 2 : 4) && to < from + n * (c->in_dtype == R3_BF16 ? 2 : 4))
        return R3_ERR_INVALID_ARG;
    if (!workspace || !aligned(workspace, 256) || ws_bytes < r3_orthogonalize_workspace_bytes(c))
        return R3_ERR_WORKSPACE;
    const r3_muon_stack one = {out, nullptr, x, nullptr, c->batch, c->rows, c->cols, 0.f, 0.f};
    const Job job = {c->out_dtype, c->in_dtype, 0, c->products, false, false, 0.f, std::max((float)c->eps, LEAST_EPS), 0.f, nullptr,
                     nullptr};
    try {
        return run(job, coefs, &one, 1, static_cast<uint8_t*>(workspace), dev_status,
                   static_cast<cudaStream_t>(stream));
    } catch (...) {
        return R3_ERR_INVALID_ARG;
    }
}

extern "C" size_t r3_muon_workspace_bytes(const r3_muon* c, const r3_muon_stack* stacks, int32_t n_stacks) {
    using namespace r3::ns;
    Coefs coefs;
    if (check_muon(c, stacks, n_stacks, &coefs) != R3_OK) return 0;
    try {
        return workspace_bytes(stacks, n_stacks, c->products);
    } catch (...) {
        return 0;
    }
}

extern "C" r3_status r3_muon_step(const r3_muon* c, const r3_muon_stack* stacks, int32_t n_stacks,
                                  const float* grad_scale, const float* lr, void* workspace, size_t ws_bytes,
                                  int32_t* dev_status, void* stream) {
    using namespace r3;
    using namespace r3::ns;
    Coefs coefs;
    r3_status st = check_muon(c, stacks, n_stacks, &coefs);
    if (st == R3_OK) st = check_buffers(c, stacks, n_stacks);
    if (st != R3_OK) return st;
    if (!aligned(grad_scale, 4) || !aligned(lr, 4) || !aligned(dev_status, 4)) return R3_ERR_INVALID_ARG;
    try {
        if (!distinct(c, stacks, n_stacks, grad_scale, lr)) return R3_ERR_INVALID_ARG;
        const size_t need = workspace_bytes(stacks, n_stacks, c->products);
        if (need == 0) return R3_OK;                   // no matrices
        if (!workspace || !aligned(workspace, 256) || ws_bytes < need) return R3_ERR_WORKSPACE;
        const Job job = {c->param_dtype, c->grad_dtype, c->nesterov != 0, c->products, c->master != 0, true,
                         (float)c->momentum, std::max((float)c->eps, LEAST_EPS), (float)c->lr, grad_scale, lr};
        return run(job, coefs, stacks, n_stacks, static_cast<uint8_t*>(workspace), dev_status,
                   static_cast<cudaStream_t>(stream));
    } catch (...) {
        return R3_ERR_INVALID_ARG;
    }
}
