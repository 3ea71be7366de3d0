// Matrix products of 16-bit operands on the fifth-generation tensor cores, shared by the loss and the orthogonalisation:
// D[m, n] = sum_k A[m, k] B[n, k], accumulated in fp32, each accumulator tile handed to an epilogue.
//
// One persistent kernel.  A CTA (CG = 1) or a pair of CTAs on neighbouring SMs (CG = 2) owns a tile of 128 CG x BN; tiles are
// dealt out round robin.  Per CTA:
//   warp 0    moves operand blocks of 64 k (128 bytes, the swizzle width) with TMA into a ring of stages
//   warp 1    of the pair's first CTA issues tcgen05.mma over each stage and commits it back to the ring
//   warp 2    allocates and frees tensor memory: two accumulators, so the next tile's products run under an epilogue
//   warps 4-  epilogue: 32 accumulator rows each (a lane is a row), all columns with four of these warps, half of them with
//             eight; through shared memory to TMA stores where the result is a matrix; arrays that it combines with the
//             accumulators come by TMA as well (AuxRing)
// In a pair every CTA stages its own 128 rows of A and its own half of B; the tensor cores read both halves of B, which
// halves the shared-memory traffic per product.  No load is multicast.
//
// An operand is "K-major" (k contiguous in memory) or "MN-major" (its m or n index contiguous).  Both are staged with the
// 128-byte swizzle.  K-major: rows of 64 k, groups of 8 rows 1024 bytes apart.  MN-major: rows of 64 m (or n), one row per k,
// groups of 8 k 1024 bytes apart, and the next 64 m follow after the 64 k of the block (8192 bytes).
//
// Tiles: a pair's 256 x 256 loads 32 KB per CTA for 512 cycles of products, all that a CTA's path from L2 gives (64 bytes per
// cycle); smaller tiles are bound by that path and only pay where they fill SMs that large ones leave idle.  On long products
// (4096 x 32000 x 4096) it runs at 1250-1300 TFLOP/s under the power limit, where library products of these sizes run at 1340-1400
// alone.
//
// Long sums: the tensor cores truncate where they add 16 further k to an accumulator, always towards zero, which shrinks a sum of
// typical operands by 1.0e-9 of itself per k (measured at k = 768, 5120 and 16384; exact sums lose nothing).  Where that matters
// (Epi::kRunStages) a tile's k is cut into runs of that many stages, each accumulated from zero, and the epilogue warps add the runs in
// fp32 registers, rounded to nearest, and put the sum back before the epilogue proper: the two accumulators take turns run by run.
//
// Every wait is bounded (kWaitCycles, kStageCycles); a role that gives up raises the CTA's stop flag, which ends the other roles, and
// counts the failure in a word of host memory that the next call of the library reads.
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <atomic>

#include "chained.cuh"

namespace cast {
namespace product {

constexpr int kBK = 64;                          // k per block: 64 x 2 bytes = one 128-byte swizzle row
constexpr int kStageBytesA = 128 * kBK * 2;      // one block of 128 rows of A
constexpr int kSlotBytes = 4096;                 // epilogue staging: 32 rows of 128 bytes
constexpr int kRing = 3;                         // slots of an epilogue's ring (see AuxRing)
constexpr long long kWaitCycles = 4000000000ll;  // ~2 s; a copy or a stage's products take microseconds
constexpr long long kStageCycles = 4096;         // allowed on top per stage of a tile, to who waits for the whole of it (a stage takes ~512)

// Shape of one launch.  k_blocks = ceil(k / (64 blocks per stage)) stages are cut into `splits` runs of at most split_blocks, each of which
// is a tile of its own (its epilogue sees Tile::split).
struct Shape {
    int m, n;                      // result rows and columns
    int k_blocks, splits, split_blocks;
    int m_tiles, n_tiles, batch;
    int group;                     // tile rows that are walked together, so that their operands stay in L2 (symmetric: see tile_of)
    int total;                     // tiles of all batches and splits
    uint32_t idesc;                // instruction descriptor
    unsigned long long* fail_word; // host memory
};

struct Tile { int batch, split, tm, tn, kb0, kb1; };

template <bool SYM>
__device__ __forceinline__ Tile tile_of(const Shape& s, int t)
{
    Tile r;
    if constexpr (SYM) {           // tiles that touch the lower triangle, tile rows first to last; `group` tile columns per tile row
        const int per = s.group * (s.m_tiles * (s.m_tiles + 1) / 2), o = t / per;
        r.batch = o / s.splits;
        r.split = o - r.batch * s.splits;
        const int i = t - o * per, j = i / s.group;
        int row = (int)((sqrtf(8.0f * (float)j + 1.0f) - 1.0f) * 0.5f);
        while (row * (row + 1) / 2 > j) --row;
        while ((row + 1) * (row + 2) / 2 <= j) ++row;
        r.tm = row;
        r.tn = i - s.group * (row * (row + 1) / 2);
    } else {
        const int per = s.m_tiles * s.n_tiles;
        const int o = t / per;
        int i = t - o * per;
        r.batch = o / s.splits;
        r.split = o - r.batch * s.splits;
        const int band = s.group * s.n_tiles;
        const int g = i / band;
        i -= g * band;
        const int rows = min(s.group, s.m_tiles - g * s.group);
        r.tn = i / rows;
        r.tm = g * s.group + (i - r.tn * rows);
    }
    r.kb0 = r.split * s.split_blocks;
    r.kb1 = min(s.k_blocks, r.kb0 + s.split_blocks);
    return r;
}

// ------------------------------------------------------------------------------------------------ instructions

__device__ __forceinline__ uint32_t smem_u32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }

__device__ __forceinline__ void mbar_init(uint32_t bar, uint32_t count)
{
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void mbar_expect(uint32_t bar, uint32_t bytes)
{
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void mbar_arrive_cluster(uint32_t bar)      // bar: shared::cluster address
{
    asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ bool mbar_try(uint32_t bar, uint32_t parity)
{
    uint32_t done;
    asm volatile("{ .reg .pred p;\n\t"
                 "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
                 "selp.u32 %0, 1, 0, p; }" : "=r"(done) : "r"(bar), "r"(parity) : "memory");
    return done != 0;
}

// One lane of a converged warp, always the same one.
__device__ __forceinline__ bool elect_one()
{
    uint32_t p;
    asm volatile("{ .reg .pred p;\n\telect.sync _|p, 0xFFFFFFFF;\n\tselp.u32 %0, 1, 0, p; }" : "=r"(p));
    return p != 0;
}

struct Stop { volatile int* flag; unsigned long long* fail_word; };

// Waits for a phase; false once the CTA has stopped or the limit (and `more` cycles) has passed.
__device__ __forceinline__ bool mbar_wait(uint32_t bar, uint32_t parity, const Stop& stop, long long more = 0)
{
    if (mbar_try(bar, parity)) return true;
    const long long t0 = clock64();
    for (uint32_t i = 1;; ++i) {
        if (mbar_try(bar, parity)) return true;
        if ((i & 31u) == 0u) {
            if (*stop.flag) return false;
            if (clock64() - t0 > kWaitCycles + more) break;
        }
    }
    *stop.flag = 1;
    atomicAdd_system(stop.fail_word, 1ull);
    return false;
}

// The same for a converged warp, with one answer for all of its lanes (which the compiler then knows to be uniform).
__device__ __forceinline__ bool mbar_wait_warp(uint32_t bar, uint32_t parity, const Stop& stop)
{
    return __all_sync(0xFFFFFFFFu, mbar_wait(bar, parity, stop));
}

__device__ __forceinline__ uint32_t map_to_rank(uint32_t addr, uint32_t rank)
{
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
    return r;
}
__device__ __forceinline__ uint32_t cluster_rank()
{
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_barrier()
{
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

template <int CG>
__device__ __forceinline__ void tma_load(uint32_t dst, const CUtensorMap* map, uint32_t bar, int x, int y, int z)
{
    if constexpr (CG == 2)
        asm volatile("cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
                     ::"r"(dst), "l"(map), "r"(bar), "r"(x), "r"(y), "r"(z) : "memory");
    else
        asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
                     ::"r"(dst), "l"(map), "r"(bar), "r"(x), "r"(y), "r"(z) : "memory");
}
__device__ __forceinline__ void tma_store(const CUtensorMap* map, uint32_t src, int x, int y, int z)
{
    asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.tile.bulk_group [%0, {%2, %3, %4}], [%1];"
                 ::"l"(map), "r"(src), "r"(x), "r"(y), "r"(z) : "memory");
}
__device__ __forceinline__ void store_commit() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void store_wait_read() { asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ void prefetch_map(const CUtensorMap* map) { asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory"); }
__device__ __forceinline__ void store_wait_all() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }
__device__ __forceinline__ void fence_async_smem() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// Descriptors by halves: the upper ones are constants, only the addresses in the lower ones change.
template <int CG>
__device__ __forceinline__ void tc_mma(uint32_t d, uint32_t a_lo, uint32_t a_hi, uint32_t b_lo, uint32_t b_hi, uint32_t idesc, uint32_t accumulate)
{
    if constexpr (CG == 2)
        asm volatile("{ .reg .pred p;\n\t.reg .b64 a, b;\n\tsetp.ne.b32 p, %6, 0;\n\tmov.b64 a, {%1, %2};\n\tmov.b64 b, {%3, %4};\n\t"
                     "tcgen05.mma.cta_group::2.kind::f16 [%0], a, b, %5, p; }"
                     ::"r"(d), "r"(a_lo), "r"(a_hi), "r"(b_lo), "r"(b_hi), "r"(idesc), "r"(accumulate) : "memory");
    else
        asm volatile("{ .reg .pred p;\n\t.reg .b64 a, b;\n\tsetp.ne.b32 p, %6, 0;\n\tmov.b64 a, {%1, %2};\n\tmov.b64 b, {%3, %4};\n\t"
                     "tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %5, p; }"
                     ::"r"(d), "r"(a_lo), "r"(a_hi), "r"(b_lo), "r"(b_hi), "r"(idesc), "r"(accumulate) : "memory");
}
// Arrives on `bar` (at the same offset in both CTAs of a pair) once every product issued so far has been done.
template <int CG>
__device__ __forceinline__ void tc_commit(uint32_t bar)
{
    if constexpr (CG == 2)
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                     ::"r"(bar), "h"((uint16_t)3) : "memory");
    else
        asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
template <int CG>
__device__ __forceinline__ void tmem_alloc(uint32_t dst_smem, uint32_t cols)
{
    if constexpr (CG == 2) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(dst_smem), "r"(cols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    } else {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(dst_smem), "r"(cols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
}
template <int CG>
__device__ __forceinline__ void tmem_free(uint32_t tmem, uint32_t cols)
{
    if constexpr (CG == 2) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(cols));
    else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(cols));
}
// 32 consecutive accumulator columns of this lane's row.  The values may be used after tmem_wait().
__device__ __forceinline__ void tmem_load32(uint32_t addr, float (&v)[32])
{
    uint32_t r[32];
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 "
                 "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
                   "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]),
                   "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]),
                   "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
                 : "r"(addr));
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
    for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(r[i]);
}

// 16 columns, whose values may be used at once, and the reverse, complete when it returns.
__device__ __forceinline__ void tmem_load16(uint32_t addr, float (&v)[16])
{
    uint32_t r[16];
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];\n\t"
                 "tcgen05.wait::ld.sync.aligned;"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
                   "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
                 : "r"(addr) : "memory");
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = __uint_as_float(r[i]);
}
__device__ __forceinline__ void tmem_store16(uint32_t addr, const float (&v)[16])
{
    uint32_t r[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) r[i] = __float_as_uint(v[i]);
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15};\n\t"
                 "tcgen05.wait::st.sync.aligned;"
                 ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
                 "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(addr) : "memory");
}

// Shared-memory matrix descriptor, 128-byte swizzle (bits 61-63 = 2, version 1 at bit 46): start address, leading and
// stride byte offsets in units of 16 bytes.
constexpr uint32_t kDescHi = (1024u >> 4) | (1u << 14) | (2u << 29);
template <bool MN_MAJOR>
__device__ __forceinline__ uint32_t desc_lo(uint32_t addr)
{
    constexpr uint32_t lead = MN_MAJOR ? (kBK * 128) >> 4 : 1;     // next 64 m (n) of an MN-major block; unused in K-major form
    return (lead << 16) | ((addr & 0x3FFFFu) >> 4);
}
template <bool MN_MAJOR>
constexpr uint32_t kDescStep = MN_MAJOR ? (16 * 128) >> 4 : (16 * 2) >> 4;      // 16 k further

// ------------------------------------------------------------------------------------------------ the kernel

// Of Epi: kWarps epilogue warps (four where a tile is only one chunk wide), each with kStaging bytes of shared memory.  A stage is
// one 64-deep block (issued in about 250 cycles, computed in 512 by a pair and 256 by a single CTA with 128 columns), and two of
// them where they are computed in 128.
template <int CG, int BN, class Epi>
struct Config {
    static constexpr int BM = 128 * CG;
    static constexpr int warps = BN >= 128 ? Epi::kWarps : 4;
    static constexpr int threads = 128 + 32 * warps;
    static constexpr int cols = BN / (warps / 4);                  // of one epilogue warp
    static constexpr int blocks = CG == 1 && BN == 64 ? 2 : 1;
    static constexpr int b_rows = BN / CG;                         // rows of B staged by one CTA
    static constexpr int b_bytes = b_rows * kBK * 2;               // of one block
    static constexpr int stage_bytes = blocks * (kStageBytesA + b_bytes);
    static constexpr int room = (232448 - 1024 /* alignment */ - 768 /* barriers */ - warps * Epi::kStaging) / stage_bytes;
    static constexpr int stages = room < 8 ? room : 8;
    static constexpr int smem_bytes = stages * stage_bytes + warps * Epi::kStaging + 1024;
    static constexpr uint32_t tmem_cols = 2 * BN;
    static_assert(BN == 256 || BN == 128 || BN == 64, "two accumulators of BN columns: a power of two of at least 32");
    static_assert(b_rows % 64 == 0, "MN-major blocks are 64 wide");
    static_assert(stages >= 3, "a ring of stages");
};

// What an epilogue warp is given for one tile.
struct EpiTile {
    Tile tile;
    int row0;            // first result row of this warp's 32
    int col0;            // first result column of the tile
    int c0, c1;          // this warp's columns of the tile
    uint32_t acc;        // tensor-memory address of this warp's rows, column 0
    uint32_t slots;      // this warp's staging memory (slots of 4 KB, 1024-byte aligned)
    uint32_t bars;       // this warp's kRing mbarriers
    int lane;
    int first_row;       // of this warp in a tile
    int index, step;     // of the tile among all tiles, and to this CTA's next one
    const Stop* stop;
};

// 16 bytes of this lane's row in a swizzled 32 x 128-byte slot.
__device__ __forceinline__ void slot_write(uint32_t slot_addr, int lane, int chunk, uint32_t a, uint32_t b, uint32_t c, uint32_t d)
{
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(slot_addr + (uint32_t)lane * 128u + (uint32_t)((chunk ^ (lane & 7)) << 4)),
                 "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}
__device__ __forceinline__ uint4 slot_read(uint32_t slot_addr, int row, int chunk)
{
    uint4 w;
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w.x), "=r"(w.y), "=r"(w.z), "=r"(w.w)
                 : "r"(slot_addr + (uint32_t)row * 128u + (uint32_t)((chunk ^ (row & 7)) << 4)) : "memory");
    return w;
}

// One 2-byte entry of it.
__device__ __forceinline__ uint32_t slot_read_16(uint32_t slot_addr, int row, int col)
{
    unsigned short w;
    asm volatile("ld.shared.u16 %0, [%1];" : "=h"(w)
                 : "r"(slot_addr + (uint32_t)row * 128u + (uint32_t)(((col >> 3) ^ (row & 7)) << 4) + (uint32_t)(col & 7) * 2u) : "memory");
    return w;
}

// The slot of an epilogue that only stores, once the store that last used it has read it.  (One is enough: two such warps share a
// scheduler, and the other one computes meanwhile.)
__device__ __forceinline__ uint32_t slot_acquire(const EpiTile& e)
{
    if (e.lane == 0) store_wait_read<0>();
    __syncwarp();
    return e.slots;
}
// Hands a written slot to a TMA store (commits an empty group where nothing is to be stored, so that the groups count slots).
__device__ __forceinline__ void slot_store(const EpiTile& e, uint32_t slot_addr, const CUtensorMap* map, int x, int y, int z, bool any)
{
    fence_async_smem();
    __syncwarp();
    if (e.lane == 0) {
        if (any) tma_store(map, slot_addr, x, y, z);
        store_commit();
    }
}

// An epilogue provides: kSym (only tiles of the lower triangle), kInputsOnly (both operands are the caller's, whole before the
// call's first kernel began), kRunStages (of k per accumulation, see above; 0: a tile's whole k), kWarps, kStaging (bytes per warp),
// State (kept from tile to tile),
// prefetch() (its tensor maps), start() (before the first tile), tile() (false: give up).
struct StoringEpi {
    static constexpr bool kSym = false;
    static constexpr bool kInputsOnly = false;
    static constexpr int kRunStages = 0;
    static constexpr int kWarps = 8;
    static constexpr int kStaging = kSlotBytes;
    struct State {};
    template <int BM, int BN>
    __device__ __forceinline__ void start(const Shape&, const EpiTile&, State&) const {}
};

// The ring of an epilogue that combines its tile with an array of the same layout: chunks of 32 rows x 64 columns come by TMA
// into kRing slots, two chunks ahead of their use (over tile borders too), and may be replaced in place by results that leave
// by TMA from there.  A slot is loaded again once the stores of the chunk that used it have read it.
struct AuxRing {
    int index, c;        // tile and column of the chunk to load next
    Tile tile;
    int load_step, step;
    uint32_t phase;      // parity of the current use of `step`

    template <int BN, bool SYM>
    __device__ __forceinline__ void start(const Shape& s, const EpiTile& e)
    {
        index = e.index;
        c = e.c0;
        load_step = step = 0;
        phase = 0;
        find<BN, SYM>(s, e);
    }
    // The tile at `index`, or the first one after it in which this warp has columns.
    template <int BN, bool SYM>
    __device__ __forceinline__ void find(const Shape& s, const EpiTile& e)
    {
        for (; index < s.total; index += e.step) {
            tile = tile_of<SYM>(s, index);
            if (tile.tn * BN + c < s.n) break;
        }
    }
    __device__ __forceinline__ uint32_t slot(const EpiTile& e) const { return e.slots + (uint32_t)(step * kSlotBytes); }

    template <int BM, int BN, bool SYM>
    __device__ __forceinline__ void load(const Shape& s, const EpiTile& e, const CUtensorMap* map)
    {
        if (index >= s.total) return;
        if (e.lane == 0) {
            const uint32_t bar = e.bars + 8u * (uint32_t)load_step;
            mbar_expect(bar, kSlotBytes);
            tma_load<1>(e.slots + (uint32_t)(load_step * kSlotBytes), map, bar, tile.tn * BN + c, tile.tm * BM + e.first_row, tile.batch);
        }
        load_step = load_step + 1 == kRing ? 0 : load_step + 1;
        c += 64;
        if (c >= e.c1 || tile.tn * BN + c >= s.n) {
            c = e.c0;
            index += e.step;
            find<BN, SYM>(s, e);
        }
    }
    // Waits for the current chunk.
    __device__ __forceinline__ bool wait(const EpiTile& e) const
    {
        return __all_sync(0xFFFFFFFFu, mbar_wait(e.bars + 8u * (uint32_t)step, phase, *e.stop));
    }
    __device__ __forceinline__ void next()
    {
        step = step + 1 == kRing ? 0 : step + 1;
        if (step == 0) phase ^= 1u;
    }
};
// All stores of this warp have read their slots.
__device__ __forceinline__ void slots_free(const EpiTile& e)
{
    if (e.lane == 0) store_wait_read<0>();
    __syncwarp();
}

template <int CG, int BN, bool A_MN, bool B_MN, class Epi>
__global__ void __launch_bounds__((Config<CG, BN, Epi>::threads), 1)
product_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
               const __grid_constant__ Shape shape, const __grid_constant__ Epi epi)
{
    using C = Config<CG, BN, Epi>;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const uint32_t ring = base;
    const uint32_t staging = base + C::stages * C::stage_bytes;
    __shared__ __align__(8) unsigned long long bars[2 * C::stages + 4 + C::warps * kRing];
    __shared__ uint32_t tmem_base_smem;
    __shared__ int stop_flag;
    const uint32_t full0 = smem_u32(bars), empty0 = full0 + 8 * C::stages, accf0 = empty0 + 8 * C::stages, acce0 = accf0 + 16, ring0 = acce0 + 16;
    const int warp = __shfl_sync(0xFFFFFFFFu, (int)threadIdx.x >> 5, 0), lane = (int)threadIdx.x & 31;
    const uint32_t rank = CG == 2 ? __shfl_sync(0xFFFFFFFFu, cluster_rank(), 0) : 0u;

    chain_next();
    if (threadIdx.x == 0) {
        stop_flag = 0;
        for (int i = 0; i < C::stages; ++i) { mbar_init(full0 + 8 * i, 1); mbar_init(empty0 + 8 * i, 1); }
        for (int i = 0; i < 2; ++i) { mbar_init(accf0 + 8 * i, 1); mbar_init(acce0 + 8 * i, CG * C::warps); }
        for (int i = 0; i < C::warps * kRing; ++i) mbar_init(ring0 + 8 * i, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (threadIdx.x == 32) {      // descriptors are fetched while the predecessor drains
        prefetch_map(&map_a);
        prefetch_map(&map_b);
        epi.prefetch();
    }
    if (warp == 2) tmem_alloc<CG>(smem_u32(&tmem_base_smem), C::tmem_cols);
    tc_fence_before();
    __syncthreads();
    if constexpr (CG == 2) cluster_barrier();
    tc_fence_after();
    const uint32_t tmem = __shfl_sync(0xFFFFFFFFu, tmem_base_smem, 0);
    const Stop stop = {&stop_flag, shape.fail_word};
    const int first = (int)blockIdx.x / CG, step = (int)gridDim.x / CG;
    // Both operands of a symmetric product are the same array: a square tile on the diagonal stages its rows once, for A and B.
    constexpr bool kSquare = Epi::kSym && A_MN == B_MN && C::BM == BN;

    // The two issuing roles run as whole warps on uniform values, with one lane elected for the instructions themselves: in a
    // single lane's branch the compiler has to move every descriptor word from vector to uniform registers, and issuing the
    // four products of a stage took ~590 cycles, more than the 512 that they take to compute; so it is about half of that.
    if (warp == 0) {
        int s = 0;
        uint32_t phase = 0;
        bool ok = true;
        Tile tile = tile_of<Epi::kSym>(shape, first);
        const uint32_t full_base = CG == 2 ? map_to_rank(full0, 0) : full0;
        // The loop runs once without effect before the wait for the predecessor, so that its code is there when that ends.
        bool live = Epi::kInputsOnly;
        for (int t = first; ok && t < shape.total;) {
            const bool once = kSquare && tile.tm == tile.tn;
            const int m0 = tile.tm * C::BM + (int)rank * 128, n0 = tile.tn * BN + (int)rank * C::b_rows;
            for (int kb = live ? tile.kb0 : tile.kb1 - 1; kb < tile.kb1; ++kb) {
                if (!(ok = mbar_wait_warp(empty0 + 8 * s, phase ^ 1u, stop))) break;
                if (live && elect_one()) {
                    const uint32_t a = ring + s * C::stage_bytes, b = a + C::blocks * kStageBytesA, full = full_base + 8 * s;
                    if (rank == 0) mbar_expect(full0 + 8 * s, CG * (once ? C::blocks * kStageBytesA : C::stage_bytes));
#pragma unroll
                    for (int j = 0; j < C::blocks; ++j) {
                        const int k = (kb * C::blocks + j) * kBK;      // past the end of k: zeros
                        const uint32_t aj = a + j * kStageBytesA, bj = b + j * C::b_bytes;
                        if constexpr (A_MN) {
#pragma unroll
                            for (int i = 0; i < 2; ++i) tma_load<CG>(aj + i * 8192, &map_a, full, m0 + 64 * i, k, tile.batch);
                        } else {
                            tma_load<CG>(aj, &map_a, full, k, m0, tile.batch);
                        }
                        if (once) continue;
                        if constexpr (B_MN) {
#pragma unroll
                            for (int i = 0; i < C::b_rows / 64; ++i) tma_load<CG>(bj + i * 8192, &map_b, full, n0 + 64 * i, k, tile.batch);
                        } else {
                            tma_load<CG>(bj, &map_b, full, k, n0, tile.batch);
                        }
                    }
                }
                __syncwarp();
                if (live && ++s == C::stages) { s = 0; phase ^= 1u; }
            }
            if (!live) {
                live = true;
                chain_wait();
                continue;
            }
            t += step;
            if (t < shape.total) tile = tile_of<Epi::kSym>(shape, t);
        }
        // every stage handed back: nothing of this CTA is in flight when it leaves
        for (int i = 0; ok && i < C::stages; ++i) {
            ok = mbar_wait(empty0 + 8 * s, phase ^ 1u, stop);
            if (++s == C::stages) { s = 0; phase ^= 1u; }
        }
        if (!ok) {      // given up: leave copies that are under way the time to land
            const long long t0 = clock64();
            while (clock64() - t0 < 10000000ll) __nanosleep(1000);
        }
    } else if (warp == 1) {
        if (rank == 0) {
            int s = 0, n_done = 0;
            uint32_t phase = 0;
            bool ok = true;
            const uint32_t a0 = desc_lo<A_MN>(ring), b0 = desc_lo<B_MN>(ring + C::blocks * kStageBytesA);
            uint32_t at = 0;          // of the stage, in units of 16 bytes
            if constexpr (!Epi::kInputsOnly) chain_wait();      // the limits below are not for waiting for a predecessor
            Tile tile = tile_of<Epi::kSym>(shape, first);
            int run0 = tile.kb0;      // the run of stages that is accumulated next
            for (int t = first; ok && t < shape.total; ++n_done) {
                const int run1 = Epi::kRunStages ? min(tile.kb1, run0 + Epi::kRunStages) : tile.kb1;
                const int buf = n_done & 1;
                if (!(ok = mbar_wait_warp(acce0 + 8 * buf, (uint32_t)((n_done >> 1) & 1) ^ 1u, stop))) break;
                tc_fence_after();
                const uint32_t d = tmem + (uint32_t)(buf * BN);
                const uint32_t b_at = kSquare && tile.tm == tile.tn ? a0 : b0;
                uint32_t accumulate = 0;
                for (int kb = run0; kb < run1; ++kb) {
                    if (!(ok = mbar_wait_warp(full0 + 8 * s, phase, stop))) break;
                    tc_fence_after();
                    if (elect_one()) {
                        const uint32_t a = a0 + at, b = b_at + at;
#pragma unroll
                        for (int i = 0; i < C::blocks * (kBK / 16); ++i) {
                            const int j = i / (kBK / 16), k = i % (kBK / 16);
                            tc_mma<CG>(d, a + j * (kStageBytesA >> 4) + k * kDescStep<A_MN>, kDescHi, b + j * (C::b_bytes >> 4) + k * kDescStep<B_MN>,
                                       kDescHi, shape.idesc, i ? 1u : accumulate);
                        }
                        tc_commit<CG>(empty0 + 8 * s);
                        if (kb + 1 == run1) tc_commit<CG>(accf0 + 8 * buf);
                    }
                    __syncwarp();
                    accumulate = 1;
                    at += C::stage_bytes >> 4;
                    if (++s == C::stages) { s = 0; at = 0; phase ^= 1u; }
                }
                run0 = run1;
                if (run0 == tile.kb1) {
                    t += step;
                    if (t < shape.total) {
                        tile = tile_of<Epi::kSym>(shape, t);
                        run0 = tile.kb0;
                    }
                }
            }
        }
    } else if (warp >= 4) {
        EpiTile e;
        e.lane = lane;
        e.slots = staging + (uint32_t)((warp - 4) * Epi::kStaging);
        e.bars = ring0 + (uint32_t)((warp - 4) * kRing * 8);
        e.first_row = (int)rank * 128 + (warp & 3) * 32;      // a warp reads the quarter of tensor memory that its index gives
        e.c0 = (warp - 4) / 4 * C::cols;
        e.c1 = e.c0 + C::cols;
        e.index = first;
        e.step = step;
        e.stop = &stop;
        typename Epi::State state;
        chain_wait();
        epi.template start<C::BM, BN>(shape, e, state);
        int n_done = 0;
        for (int t = first; t < shape.total; t += step, ++n_done) {
            e.index = t;
            e.tile = tile_of<Epi::kSym>(shape, t);
            bool ok;
            float sum[Epi::kRunStages ? C::cols / 16 : 1][16];       // of the runs before the last
            int run0 = e.tile.kb0;
            if constexpr (Epi::kRunStages != 0) {
#pragma unroll
                for (int j = 0; j < C::cols / 16; ++j)
#pragma unroll
                    for (int i = 0; i < 16; ++i) sum[j][i] = 0.0f;
#pragma unroll 1
                for (; run0 + Epi::kRunStages < e.tile.kb1; run0 += Epi::kRunStages, ++n_done) {
                    const int buf = n_done & 1;
                    ok = mbar_wait(accf0 + 8 * buf, (uint32_t)(n_done >> 1) & 1u, stop, Epi::kRunStages * kStageCycles);
                    if (!__all_sync(0xFFFFFFFFu, ok)) break;
                    tc_fence_after();
                    const uint32_t acc = tmem + (uint32_t)(buf * BN) + ((uint32_t)((warp & 3) * 32) << 16);
#pragma unroll
                    for (int j = 0; j < C::cols / 16; ++j) {
                        float v[16];
                        tmem_load16(acc + (uint32_t)(e.c0 + 16 * j), v);
#pragma unroll
                        for (int i = 0; i < 16; ++i) sum[j][i] += v[i];
                    }
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive_cluster(map_to_rank(acce0 + 8 * buf, 0));
                }
                if (run0 + Epi::kRunStages < e.tile.kb1) break;      // given up
            }
            const int buf = n_done & 1;
            ok = mbar_wait(accf0 + 8 * buf, (uint32_t)(n_done >> 1) & 1u, stop, (e.tile.kb1 - run0) * kStageCycles);
            if (!__all_sync(0xFFFFFFFFu, ok)) break;
            tc_fence_after();
            e.row0 = e.tile.tm * C::BM + e.first_row;
            e.col0 = e.tile.tn * BN;
            e.acc = tmem + (uint32_t)(buf * BN) + ((uint32_t)((warp & 3) * 32) << 16);
            if constexpr (Epi::kRunStages != 0) {
                if (run0 != e.tile.kb0) {
#pragma unroll
                    for (int j = 0; j < C::cols / 16; ++j) {
                        float v[16];
                        tmem_load16(e.acc + (uint32_t)(e.c0 + 16 * j), v);
#pragma unroll
                        for (int i = 0; i < 16; ++i) v[i] += sum[j][i];
                        tmem_store16(e.acc + (uint32_t)(e.c0 + 16 * j), v);
                    }
                }
            }
            ok = epi.template tile<C::BM, BN>(shape, e, state);
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_cluster(map_to_rank(acce0 + 8 * buf, 0));
            if (!ok) break;
        }
        if (lane == 0) store_wait_read<0>();      // the results are on their way; the shared memory may go
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if constexpr (CG == 2) cluster_barrier();
    tc_fence_after();
    if (warp == 2) tmem_free<CG>(tmem, C::tmem_cols);
}

// ------------------------------------------------------------------------------------------------ host side

// A [batch][rows][inner] array of 2- or 4-byte elements, moved in boxes of box_rows x box_inner.  `ld` and `batch_stride`
// in elements; ld x element size and the base must be multiples of 16 bytes.
int make_map(CUtensorMap* map, const void* base, int elem_bytes, uint64_t inner, uint64_t rows, uint64_t batch, uint64_t ld,
             uint64_t batch_stride, uint32_t box_inner, uint32_t box_rows, bool swizzle);

// The operand maps: rows of A (128 per CTA) or B (b_rows per CTA).  K-major: inner = k, rows = m; MN-major: inner = m, rows = k.
template <bool MN_MAJOR>
int operand_map(CUtensorMap* map, const void* base, uint64_t mn, uint64_t k, uint64_t batch, uint64_t ld, uint64_t batch_stride, uint32_t rows_per_cta)
{
    if (MN_MAJOR) return make_map(map, base, 2, mn, k, batch, ld, batch_stride, 64, kBK, true);
    return make_map(map, base, 2, k, mn, batch, ld, batch_stride, kBK, rows_per_cta, true);
}

// Page-locked word the kernels report an abandoned wait in; CAST_ERR_STAGING once it is not zero.
int fail_word(unsigned long long** word);
int sm_count(int* n);

inline uint32_t instruction_desc(bool bf16, bool a_mn, bool b_mn, int m, int n)
{
    // D fp32 (bit 4), A and B type (bits 7, 10: 1 = bf16, 0 = f16), transposes (15, 16), n / 8 (17), m / 16 (24)
    return (1u << 4) | ((bf16 ? 1u : 0u) << 7) | ((bf16 ? 1u : 0u) << 10) | ((a_mn ? 1u : 0u) << 15) | ((b_mn ? 1u : 0u) << 16) |
           ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}

template <int CG, int BN, bool A_MN, bool B_MN, class Epi>
int make_shape(Shape* s, bool bf16, int64_t m, int64_t n, int64_t k, int64_t batch, int splits, int group)
{
    using C = Config<CG, BN, Epi>;
    constexpr bool SYM = Epi::kSym;
    const int64_t mt = (m + C::BM - 1) / C::BM, nt = (n + BN - 1) / BN;
    static_assert(!SYM || C::BM % BN == 0, "the triangle's blocks are whole tiles");
    s->m = (int)m;
    s->n = (int)n;
    s->k_blocks = (int)((k + C::blocks * kBK - 1) / (C::blocks * kBK));
    if (splits > s->k_blocks) splits = s->k_blocks;
    s->split_blocks = (s->k_blocks + splits - 1) / splits;
    s->splits = (s->k_blocks + s->split_blocks - 1) / s->split_blocks;
    s->m_tiles = (int)mt;
    s->n_tiles = (int)nt;
    s->batch = (int)batch;
    s->group = SYM ? C::BM / BN : group;
    const int64_t per = (SYM ? mt * (mt + 1) / 2 * s->group : mt * nt) * s->splits;
    if (per * batch > 0x3FFFFFFF) return CAST_ERR_SHAPE;
    s->total = (int)(per * batch);
    s->idesc = instruction_desc(bf16, A_MN, B_MN, C::BM, BN);
    return fail_word(&s->fail_word);
}

template <int CG, int BN, bool A_MN, bool B_MN, class Epi>
int launch(const CUtensorMap& a, const CUtensorMap& b, const Shape& s, const Epi& epi, cudaStream_t stream)
{
    using C = Config<CG, BN, Epi>;
    auto kernel = product_kernel<CG, BN, A_MN, B_MN, Epi>;
    int sms, rc;
    if ((rc = sm_count(&sms)) != CAST_OK) return rc;
    // once per kernel and device (setting it again, by another thread, does no harm)
    static std::atomic<uint64_t> allowed{0};
    int dev;
    CAST_CUDA_TRY(cudaGetDevice(&dev));
    if (dev >= 64 || !(allowed.load(std::memory_order_relaxed) >> dev & 1u)) {
        CAST_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, C::smem_bytes));
        if (dev < 64) allowed.fetch_or(1ull << dev, std::memory_order_relaxed);
    }
    const int units = s.total < sms / CG ? s.total : sms / CG;
    return launch_chained(false, kernel, dim3((unsigned)(units * CG)), C::threads, C::smem_bytes, stream, CG, a, b, s, epi);
}

}  // namespace product
}  // namespace cast
