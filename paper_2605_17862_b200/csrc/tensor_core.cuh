// Tensor-core products on sm_100a: PTX wrappers and the one kernel that every matrix product of the library runs in.
//
// A job (a struct with tile() and epilogue()) says what is multiplied and what becomes of the result.  The kernel stays on
// the SM and takes tiles of kCtas * 128 x kN results in turn.  Warp 0 brings operand blocks in by TMA (64 of the contraction
// at a time, 128-byte swizzle) through a ring of stages; one thread of warp 1 issues tcgen05.mma from there into one of two
// (four) accumulators in TMEM; warps 4 to 11 take a finished accumulator into registers, hand it back and work on from
// there, beside the next products.  With kCtas = 2 a pair of CTAs works on one tile: each holds half of both operands and half the
// accumulator's rows, and shared memory is read once for twice the products (cta_group::2; 64 instead of 96 bytes per SM and
// cycle at 256 columns, which with the copies coming in is what 1-CTA tiles are short of: 14 matrices of width 2,048 take 3.3 ms in
// tiles of 256 x 256 on pairs, 4.0 ms in tiles of 128 x 128).  Bound by the tensor pipe: 93 to 96 % busy at 4,096 x 151,936 x 2,048, at the
// 1.38 to 1.46 GHz that the power cap leaves.
//
// Operands are 16-bit (both bf16 or both fp16), products and sums fp32.  Either operand may lie with the contraction along
// its rows ("K-major") or across them; both come in boxes of 64 elements to a row, so that nothing is ever transposed.
//
// A matrix instruction does not round what it adds to the accumulator, it cuts it off: over K terms sums come out smaller by up to
// K / 16 units of 2^-24.  A tile has its accumulator taken out every `chunk` blocks (accumulators.cuh) and added up in registers,
// rounded to nearest: every eight blocks takes 1.5 % more time (the same case) and an error of 2.6e-7 instead of 1.2e-6.
//
// Every wait is bounded.  One that runs out raises a flag, the role leaves its loop, the others run out in turn, copies and
// products in flight are waited for (again with a limit), TMEM is given back, FOPD_DEV_TIMEOUT goes to the status word.
#pragma once

#include <cuda.h>
#include <cuda_fp16.h>

#include "accumulators.cuh"
#include "async.cuh"
#include "common.cuh"

namespace fopd {

__device__ __forceinline__ bool elect_one() {  // the same lane each time
  uint32_t yes;
  asm volatile("{\n.reg .pred p;\nelect.sync _|p, 0xffffffff;\nselp.u32 %0, 1, 0, p;\n}" : "=r"(yes));
  return yes != 0;
}

// Kernels that follow one another in a call are launched early: each lets the next one's CTAs come up as soon as its own have started
// and SMs come free, and waits here, before it reads or writes anything, until everything before it is done.
__device__ __forceinline__ void grid_wait() {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
}

// ------------------------------------------------------------------ TMA
template <int kCtas>
__device__ __forceinline__ void tma_load(uint32_t dst, const CUtensorMap *map, int x, int y, uint32_t bar) {
  if constexpr (kCtas == 2)  // (the barrier may be the other CTA's)
    asm volatile(
        "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
        "l"(map), "r"(x), "r"(y), "r"(bar)
        : "memory");
  else
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
        "l"(map), "r"(x), "r"(y), "r"(bar)
        : "memory");
}
__device__ __forceinline__ void tma_store(const CUtensorMap *map, int x, int y, uint32_t src) {
  asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.tile.bulk_group [%0, {%1, %2}], [%3];" ::"l"(map), "r"(x), "r"(y),
               "r"(src)
               : "memory");
}
__device__ __forceinline__ void tma_store_commit() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }
template <int kPending>
__device__ __forceinline__ void tma_store_wait_read() {
  asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(kPending) : "memory");
}
__device__ __forceinline__ void tma_store_wait_all() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }
__device__ __forceinline__ void fence_async_shared() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// ------------------------------------------------------------------ TMEM and tcgen05
template <int kCtas>
__device__ __forceinline__ void tmem_alloc(uint32_t dst, uint32_t cols) {
  if constexpr (kCtas == 2) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(dst), "r"(cols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
  } else {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(dst), "r"(cols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
  }
}
template <int kCtas>
__device__ __forceinline__ void tmem_free(uint32_t addr, uint32_t cols) {
  if constexpr (kCtas == 2)
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(addr), "r"(cols));
  else
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(addr), "r"(cols));
}
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

template <int kCtas>
__device__ __forceinline__ void tc_mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool accumulate) {
  if constexpr (kCtas == 2)
    asm volatile(
        "{\n.reg .pred p;\nsetp.ne.b32 p, %4, 0;\n"
        "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n}\n" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"((uint32_t)accumulate)
        : "memory");
  else
    asm volatile(
        "{\n.reg .pred p;\nsetp.ne.b32 p, %4, 0;\n"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}\n" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"((uint32_t)accumulate)
        : "memory");
}
// One arrival on the barrier at this offset, in both CTAs of a pair, once all products issued so far are done.
template <int kCtas>
__device__ __forceinline__ void tc_commit(uint32_t bar) {
  if constexpr (kCtas == 2)
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar),
                 "h"((uint16_t)3)
                 : "memory");
  else
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
// 32 columns of this warp's 32 rows: lane = row.  The values are there after tmem_wait on the same array.
__device__ __forceinline__ void tmem_load(uint32_t (&r)[32], uint32_t addr) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
      "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, "
      "[%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
        "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]),
        "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]),
        "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(addr));
}
__device__ __forceinline__ void tmem_wait(uint32_t (&r)[32]) {  // (the operands keep uses of the values behind the wait)
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]),
                 "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]), "+r"(r[16]),
                 "+r"(r[17]), "+r"(r[18]), "+r"(r[19]), "+r"(r[20]), "+r"(r[21]), "+r"(r[22]), "+r"(r[23]), "+r"(r[24]),
                 "+r"(r[25]), "+r"(r[26]), "+r"(r[27]), "+r"(r[28]), "+r"(r[29]), "+r"(r[30]), "+r"(r[31])
               :
               : "memory");
}

__device__ __forceinline__ void mbar_arrive_cluster(uint32_t cluster_bar) {
  asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_bar) : "memory");
}

__device__ __forceinline__ void mbar_expect_tx_cluster(uint32_t cluster_bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.release.cluster.shared::cluster.b64 _, [%0], %1;" ::"r"(cluster_bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void st_async_v4(uint32_t cluster_addr, int4 v, uint32_t cluster_bar) {
  asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.v4.s32 [%0], {%1, %2, %3, %4}, [%5];" ::"r"(cluster_addr),
               "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w), "r"(cluster_bar)
               : "memory");
}
__device__ __forceinline__ int load_acquire(const int *p) {
  int v;
  asm volatile("ld.acquire.gpu.global.s32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
  return v;
}
__device__ __forceinline__ void add_release(int *p, int v) {
  asm volatile("red.release.gpu.global.add.s32 [%0], %1;" ::"l"(p), "r"(v) : "memory");
}
__device__ __forceinline__ void fence_async_global() { asm volatile("fence.proxy.async.global;" ::: "memory"); }

// ------------------------------------------------------------------ tiles
constexpr int kBoxRows = 64;                    // rows of one TMA box of 64 16-bit elements, across; along twice as many
constexpr int kBoxBytes = kBoxRows * 128;
constexpr int kProductThreads = 384;
constexpr int kEpilogueWarp0 = 4, kEpilogueWarps = 8;  // two to each quarter of the rows, half of the columns each
constexpr int kStageBufBytes = 32 * 128;        // an epilogue warp's staging buffer: its 32 rows x 128 bytes
constexpr int kStageBufs = 2;
constexpr uint32_t kTmemCols = 512;
// Registers: 384 threads x 168 at launch; 128 x 64 + 256 x 216 = 63,488 of those 64,512 afterwards.
constexpr int kRoleRegs = 64, kEpilogueRegs = 216;

// One operand of a tile: where its boxes are.  Where the contraction runs along the rows a box is 128 rows of 64 elements, where it
// runs across them 64 rows: 64 of the contraction and 64 of the tile.
struct Operand {
  const CUtensorMap *map;
  int x, y;    // the first box of this CTA's part
  int kx, ky;  // from one block of 64 of the contraction to the next
  int cx, cy;  // from one box to the next
  int lo;      // rows from a plane of the values to the plane of what their rounding left (two-plane operands)
  bool across; // the contraction runs across the rows of the boxes
};
// A symmetric operand of which only the tiles on and below the diagonal are stored: from block `turn` of the contraction on it is
// read across, out of the tiles below.
struct Turn {
  int at;      // past the last block: never
  const CUtensorMap *map;
  int y, cy;   // as in Operand, with x = kx = cx = 0 and ky = 64; y for block 0
};

// The contraction may run over several pairs of planes: pass i takes a's second plane where bit i of a_lo is set, etc.
struct Tile {
  Operand a, b;
  Turn a_turn, b_turn;  // where the job has symmetric operands
  int k_blocks;  // 0: the product is zero
  int chunk;     // blocks of the last pass to an accumulator, at most kLongChunk
  int passes;    // all but the last are small terms, kLongChunk blocks to an accumulator
  uint32_t a_lo, b_lo;
};

__device__ __forceinline__ int small_blocks(const Tile &t) { return (t.passes - 1) * t.k_blocks; }
__device__ __forceinline__ uint64_t smem_descriptor(uint32_t addr) {
  // 128-byte swizzle: groups of 8 rows of 128 bytes, 1,024 bytes apart; across: 64 rows further is the next box (along, this is not
  // looked at)
  const uint64_t lbo = kBoxBytes >> 4, sbo = 1024 >> 4;
  return (uint64_t)((addr & 0x3ffff) >> 4) | (lbo << 16) | (sbo << 32) | (1ull << 46) | (2ull << 61);
}

template <int kCtas, int kN>
struct ProductShape {
  static constexpr int kBCols = kN / kCtas;  // of the tile's columns, this CTA's operand share
  static constexpr int kABoxes = 128 / kBoxRows, kBBoxes = kBCols / kBoxRows;
  static constexpr int kStageBytes = (kABoxes + kBBoxes) * kBoxBytes;
  static constexpr int kStages = 160 * 1024 / kStageBytes;
  static constexpr int kAccs = (int)kTmemCols / kN;
  static constexpr int kSmem = kStages * kStageBytes + kEpilogueWarps * kStageBufs * kStageBufBytes + 1024;
};

constexpr long long kLongWaitCycles = 2000000000;  // (~1 s: behind a claimed tile's wait for others)
constexpr int kFeed = 4;  // tiles a CTA (pair) has claimed and some role has not yet taken note of
struct ProductShared {
  unsigned long long full[8], empty[8], acc_full[4], acc_empty[4], drain, feed_full[kFeed], feed_empty[kFeed], staged[kEpilogueWarps];
  unsigned long long order_full[kEpilogueWarps], order_empty[kEpilogueWarps];
  int4 order[kEpilogueWarps];
  int4 feed[kFeed];
  uint32_t tmem;
  int failed;
};

// What an epilogue warp is given beside its values: columns half * kN / 2 and following of rows warp * 32 + lane of this CTA's 128.
struct Accumulator {
  int warp, lane, half;
  uint32_t staging;  // two staging buffers
  uint32_t staged;   // a barrier for copies into them
  uint32_t order, order_full, order_empty;  // what the storing thread is to do with them (below)
};
// Takes a part of an accumulator: v += its columns, or v = them (or zero).
template <bool kAdd, int kCols>
__device__ __forceinline__ void take_columns(float (&v)[kCols], uint32_t addr, bool zero) {
#pragma unroll
  for (int c = 0; c < kCols; c += 64) {
    uint32_t r[32], q[32];
    tmem_load(r, addr + c);
    tmem_load(q, addr + c + 32);
    tmem_wait(r);
    tmem_wait(q);
#pragma unroll
    for (int j = 0; j < 32; ++j) {
      v[c + j] = kAdd ? v[c + j] + __uint_as_float(r[j]) : zero ? 0.f : __uint_as_float(r[j]);
      v[c + 32 + j] = kAdd ? v[c + 32 + j] + __uint_as_float(q[j]) : zero ? 0.f : __uint_as_float(q[j]);
    }
  }
}

template <int kCtas, int kBoxes>
__device__ __forceinline__ void load_operand(const Operand &o, uint32_t at, uint32_t bar) {
  if (o.across) {
#pragma unroll
    for (int c = 0; c < kBoxes; ++c) tma_load<kCtas>(at + c * kBoxBytes, o.map, o.x + c * o.cx, o.y + c * o.cy, bar);
  } else {
#pragma unroll
    for (int c = 0; c < kBoxes / 2; ++c) tma_load<kCtas>(at + 2 * c * kBoxBytes, o.map, o.x + c * o.cx, o.y + c * o.cy, bar);
  }
}

// Where tiles wait for others, results are stored by a thread of their own, which waits until they are written and counts them, while
// the epilogue warps go on.  Each of the eight puts one order to a round: the boxes in its two staging buffers go to rows y and z of the map
// (negative: nothing), w counts are added to entry x of the counts; x negative: no more rounds.  The buffers are the warp's again
// after order_empty.
__device__ __forceinline__ bool store_orders(ProductShared &sh, uint32_t staging, const CUtensorMap *map, int *counts) {
  for (uint32_t turn = 0;; turn ^= 1) {
    int which = -1, units = 0;
    for (int w = 0; w < kEpilogueWarps; ++w) {
      if (!mbar_wait_bounded(smem_u32(&sh.order_full[w]), turn, kLongWaitCycles)) return false;
      int4 o;
      asm volatile("ld.shared.v4.s32 {%0, %1, %2, %3}, [%4];" : "=r"(o.x), "=r"(o.y), "=r"(o.z), "=r"(o.w) : "r"(smem_u32(&sh.order[w])) : "memory");
      if (o.x < 0) return true;  // (all of them say so)
      which = o.x;
      units += o.w;
      const uint32_t from = staging + w * kStageBufs * kStageBufBytes;
      if (o.y >= 0) tma_store(map, 0, o.y, from);
      if (o.z >= 0) tma_store(map, 0, o.z, from + kStageBufBytes);
    }
    tma_store_commit();
    tma_store_wait_read<0>();
    for (int w = 0; w < kEpilogueWarps; ++w) mbar_arrive(smem_u32(&sh.order_empty[w]));
    tma_store_wait_all();
    if (units > 0) add_release(counts + which, units);
  }
}

// Which tiles a CTA (pair) works on, as each role sees them.  Either every step-th one, or, where tiles wait for others (kClaimed),
// the next that no one has: the thread that brings the first CTA's operands in takes it from a counter when it has nothing
// left to ask for, and passes it on through shared memory.  Tiles are claimed in an order in which each comes behind those it waits for,
// and a claimed tile is worked on: whatever part of the grid is resident, the lowest unfinished tile can always go on.
// What the roles get is a ticket (16 bytes, `i` first: the tile, negative where there is no more).
template <int kCtas, class Job>
struct TileFeed {
  static constexpr long long kLimit = Job::kClaimed ? kLongWaitCycles : kWaitCycles;
  ProductShared &sh;
  const int cta;
  const int64_t n_tiles, step;
  int64_t i;
  uint32_t n = 0;
  bool ok = true;
  using Ticket = typename Job::Ticket;
  __device__ TileFeed(ProductShared &s, int c, int64_t tiles)
      : sh(s), cta(c), n_tiles(tiles), step(gridDim.x / kCtas), i((int64_t)(blockIdx.x / kCtas) - step) {}
  // (by all lanes of a warp) the next claimed tile; `asked` is what the elected lane got from the counter, -1 if it has yet to ask
  __device__ __forceinline__ Ticket next_claimed(const Job &job, bool elected, int asked) {
    const uint32_t slot = n % kFeed;
    ok = __all_sync(0xffffffffu, mbar_wait_cluster_bounded(smem_u32(&sh.feed_empty[slot]), ((n / kFeed) & 1) ^ 1, kLimit));
    Ticket ticket = {};
    ticket.i = -1;
    if (!ok) return ticket;
    ++n;
    if (elected && asked < 0) asked = atomicAdd(job.counter(), 1);
    const int v = __reduce_add_sync(0xffffffffu, elected ? asked : 0);
    if (v < n_tiles) ticket = job.ticket(v);
    static_assert(sizeof(Ticket) == 16, "goes through shared memory as one vector");
    if (elected) {
      const int4 bits = *reinterpret_cast<const int4 *>(&ticket);
      if constexpr (kCtas == 1) {
        asm volatile("st.shared.v4.s32 [%0], {%1, %2, %3, %4};" ::"r"(smem_u32(&sh.feed[slot])), "r"(bits.x), "r"(bits.y), "r"(bits.z), "r"(bits.w)
                     : "memory");
        mbar_arrive(smem_u32(&sh.feed_full[slot]));
      } else {
        for (int r = 0; r < kCtas; ++r) {
          const uint32_t bar = map_to_cta(smem_u32(&sh.feed_full[slot]), r);
          mbar_expect_tx_cluster(bar, 16);
          st_async_v4(map_to_cta(smem_u32(&sh.feed[slot]), r), bits, bar);
        }
      }
    }
    return ticket;
  }
  __device__ __forceinline__ Ticket next() {
    Ticket ticket = {};
    if constexpr (!Job::kClaimed) {
      i += step;
      ticket.i = i < n_tiles ? i : -1;
      return ticket;
    } else {
      ticket.i = -1;
      const uint32_t slot = n % kFeed;
      ok = __all_sync(0xffffffffu, mbar_wait_cluster_bounded(smem_u32(&sh.feed_full[slot]), (n / kFeed) & 1, kLimit));
      if (!ok) return ticket;
      ++n;
      int4 bits;
      asm volatile("ld.shared.v4.s32 {%0, %1, %2, %3}, [%4];"
                   : "=r"(bits.x), "=r"(bits.y), "=r"(bits.z), "=r"(bits.w)
                   : "r"(smem_u32(&sh.feed[slot]))
                   : "memory");
      bits.x = __shfl_sync(0xffffffffu, bits.x, 0);  // (the same in all lanes, and known to be)
      bits.y = __shfl_sync(0xffffffffu, bits.y, 0);
      bits.z = __shfl_sync(0xffffffffu, bits.z, 0);
      bits.w = __shfl_sync(0xffffffffu, bits.w, 0);
      ticket = *reinterpret_cast<const Ticket *>(&bits);
      if ((threadIdx.x & 31) == 0) {
        const uint32_t bar = smem_u32(&sh.feed_empty[slot]);
        if constexpr (kCtas == 2) mbar_arrive_cluster(map_to_cta(bar, 0));
        else mbar_arrive(bar);
      }
      return ticket;
    }
  }
};

// Job: Params (a kernel parameter); Job(params); Ticket; int64_t tiles(); void tile(ticket, int cta, Tile &);
// void prefetch(ticket, int cta, const Accumulator &), what an epilogue warp asks for while the products run;
// void epilogue(ticket, int cta, const Accumulator &, float (&v)[kN / 2]); int32_t *status(); static constexpr bool kFp16, kTurns (it has
// symmetric operands), kClaimed; and where that is true int *counter(), Ticket ticket(i), bool ready(ticket, limit), which returns
// when what the tile reads is there, bool finish(acc), what an epilogue warp does at the end
// (prefetch, which gets the limit too, and epilogue are bool then; false: a wait ran out), and store_map() and done_counts() for the storing thread.
struct TileNumber {
  int64_t i;
};
template <int kCtas, int kN, class Job>
__global__ void __launch_bounds__(kProductThreads, 1) product_kernel(const __grid_constant__ typename Job::Params params) {
  using Shape = ProductShape<kCtas, kN>;
  extern __shared__ uint8_t product_smem[];
  __shared__ ProductShared sh;
  const int warp = __shfl_sync(0xffffffffu, (int)threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  const uint32_t base = (smem_u32(product_smem) + 1023u) & ~1023u;
  const uint32_t staging = base + Shape::kStages * Shape::kStageBytes;
  const int cta = kCtas == 2 ? (int)cluster_ctarank() : 0;

  if (threadIdx.x == 0) {
    for (int i = 0; i < Shape::kStages; ++i) {
      mbar_init(smem_u32(&sh.full[i]), 1);
      mbar_init(smem_u32(&sh.empty[i]), 1);
    }
    for (int i = 0; i < Shape::kAccs; ++i) {
      mbar_init(smem_u32(&sh.acc_full[i]), 1);
      mbar_init(smem_u32(&sh.acc_empty[i]), kCtas * kEpilogueWarps);
    }
    for (int i = 0; i < kFeed; ++i) {  // (read by the products' thread and the epilogues; the second CTA's copies in)
      mbar_init(smem_u32(&sh.feed_full[i]), 1);
      mbar_init(smem_u32(&sh.feed_empty[i]), kCtas * (1 + kEpilogueWarps));
    }
    for (int i = 0; i < kEpilogueWarps; ++i) {
      mbar_init(smem_u32(&sh.staged[i]), 1);
      mbar_init(smem_u32(&sh.order_full[i]), 1);
      mbar_init(smem_u32(&sh.order_empty[i]), 1);
    }
    mbar_init(smem_u32(&sh.drain), 1);
    sh.failed = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 2) tmem_alloc<kCtas>(smem_u32(&sh.tmem), kTmemCols);
  tc_fence_before();
  __syncthreads();
  if constexpr (kCtas == 2) {
    cluster_arrive();
    cluster_wait();
  }
  tc_fence_after();
  grid_wait();
  const uint32_t tmem = __shfl_sync(0xffffffffu, sh.tmem, 0);

  Job job(params);
  TileFeed<kCtas, Job> feed(sh, cta, job.tiles());
  constexpr long long kLimit = TileFeed<kCtas, Job>::kLimit;

  if (warp < kEpilogueWarp0) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRoleRegs));
    // (whole warps go through these loops and one thread of each issues: what is the same in all lanes stays in uniform registers)
    const bool elected = elect_one();
    const uint32_t full = smem_u32(&sh.full[0]), empty = smem_u32(&sh.empty[0]);
    if (warp == 0) {
      // ---- copies in
      uint32_t stage = 0, used = 0, parity = 1;
      int asked = -1;
      bool ok = true;
      const uint32_t signal = kCtas == 2 ? map_to_cta(full, 0) : full;
      while (true) {
        typename Job::Ticket ticket;
        if constexpr (Job::kClaimed) ticket = cta == 0 ? feed.next_claimed(job, elected, asked) : feed.next();
        else ticket = feed.next();
        if (ticket.i < 0) break;
        Tile t;
        job.tile(ticket, cta, t);
        if constexpr (Job::kClaimed) ok = job.ready(ticket, kLimit);
        ok = __all_sync(0xffffffffu, ok);
        asked = -1;
        int left = t.passes * t.k_blocks;
        for (int pass = 0; ok && pass < t.passes; ++pass) {
          Operand a = t.a, b = t.b;
          if (t.a_lo >> pass & 1) a.y += a.lo;
          if (t.b_lo >> pass & 1) b.y += b.lo;
          for (int k = 0; k < t.k_blocks; ++k) {
            if constexpr (Job::kTurns) {
              if (k == t.a_turn.at) a = {t.a_turn.map, 0, t.a_turn.y + k * 64 + ((t.a_lo >> pass & 1) ? a.lo : 0), 0, 64, 0, t.a_turn.cy, a.lo, true};
              if (k == t.b_turn.at) b = {t.b_turn.map, 0, t.b_turn.y + k * 64 + ((t.b_lo >> pass & 1) ? b.lo : 0), 0, 64, 0, t.b_turn.cy, b.lo, true};
            }
            if (!mbar_wait_bounded(empty + stage * 8, parity, kLimit)) {
              ok = false;
              break;
            }
            if (elected) {
              // (the next tile, a little before there is nothing left to ask for: the answer takes a while)
              if constexpr (Job::kClaimed)
                if (cta == 0 && asked < 0 && left <= 3) asked = atomicAdd(job.counter(), 1);
              if (cta == 0) mbar_expect_tx(full + stage * 8, kCtas * Shape::kStageBytes);
              const uint32_t at = base + stage * Shape::kStageBytes, bar = signal + stage * 8;
              load_operand<kCtas, Shape::kABoxes>(a, at, bar);
              load_operand<kCtas, Shape::kBBoxes>(b, at + Shape::kABoxes * kBoxBytes, bar);
            }
            --left;
            a.x += a.kx, a.y += a.ky, b.x += b.kx, b.y += b.ky;
            if (used < Shape::kStages) ++used;
            if (++stage == Shape::kStages) {
              stage = 0;
              parity ^= 1;
            }
          }
        }
        ok = __all_sync(0xffffffffu, ok);
      }
      // Before this CTA may end, the stages it filled have been read (their last arrivals are in): behind the copies.
      for (uint32_t j = 0; j < used; ++j) {
        if (stage == 0) parity ^= 1;
        stage = stage == 0 ? Shape::kStages - 1 : stage - 1;
        if (!mbar_wait_bounded(empty + stage * 8, parity ^ 1, kLimit)) ok = false;
      }
      if (!ok || !feed.ok) sh.failed = 1;
    }
    if constexpr (Job::kClaimed) {
      if (warp == 2) {
        // ---- stores, and the count of what is stored
        if (elected && !store_orders(sh, staging, job.store_map(), job.done_counts())) sh.failed = 1;
        __syncwarp();
      }
    }
    if (warp == 1 && cta == 0) {
      // ---- products
      const uint32_t acc_full = smem_u32(&sh.acc_full[0]), acc_empty = smem_u32(&sh.acc_empty[0]);
      uint32_t stage = 0, parity = 0, buf = 0, turn = 1;  // turn: parity of acc_empty
      bool ok = true;
      for (typename Job::Ticket ticket; ok && (ticket = feed.next()).i >= 0;) {
        Tile t;
        job.tile(ticket, cta, t);
        constexpr uint32_t kAlong = 32 >> 4, kAcross = 16 * 128 >> 4;  // descriptors: 16 of the contraction further
        const uint32_t idesc0 = (1u << 4) | (Job::kFp16 ? 0u : (1u << 7) | (1u << 10)) | ((uint32_t)(kN >> 3) << 17) |
                                ((uint32_t)(kCtas * 128 >> 4) << 24);
        uint32_t idesc = idesc0 | ((uint32_t)t.a.across << 15) | ((uint32_t)t.b.across << 16);
        uint32_t a_step = t.a.across ? kAcross : kAlong, b_step = t.b.across ? kAcross : kAlong;
        const uint64_t a0 = smem_descriptor(base), b0 = smem_descriptor(base + Shape::kABoxes * kBoxBytes);
        const int blocks = t.passes * t.k_blocks, small = small_blocks(t), chunk = t.chunk;
        int end = accumulator_end(0, small, blocks, chunk);
        int in_pass = 0;
        int done = 0;
        do {
          if (!mbar_wait_bounded(acc_empty + buf * 8, turn, kLimit)) {
            ok = false;
            break;
          }
          tc_fence_after();
          const uint32_t d = tmem + buf * kN;
          for (int k = done; k < end; ++k) {
            if (!mbar_wait_bounded(full + stage * 8, parity, kLimit)) {
              ok = false;
              break;
            }
            tc_fence_after();
            if constexpr (Job::kTurns) {
              if (in_pass == t.k_blocks) in_pass = 0;
              const bool across_a = t.a.across || in_pass >= t.a_turn.at, across_b = t.b.across || in_pass >= t.b_turn.at;
              ++in_pass;
              idesc = idesc0 | ((uint32_t)across_a << 15) | ((uint32_t)across_b << 16);
              a_step = across_a ? kAcross : kAlong;
              b_step = across_b ? kAcross : kAlong;
            }
            const uint64_t a = a0 + stage * (Shape::kStageBytes >> 4), b = b0 + stage * (Shape::kStageBytes >> 4);
            if (elected) {
#pragma unroll
              for (int j = 0; j < 4; ++j) tc_mma<kCtas>(d, a + j * a_step, b + j * b_step, idesc, k > done || j > 0);
              tc_commit<kCtas>(empty + stage * 8);
            }
            if (++stage == Shape::kStages) {
              stage = 0;
              parity ^= 1;
            }
          }
          if (!ok) break;
          if (elected) tc_commit<kCtas>(acc_full + buf * 8);
          if (++buf == Shape::kAccs) {
            buf = 0;
            turn ^= 1;
          }
          done = end;
          end = accumulator_end(done, small, blocks, chunk);
        } while (done < blocks);
        ok = __all_sync(0xffffffffu, ok);
      }
      if (!feed.ok) sh.failed = 1;
      if (!ok) {  // let what has been issued end
        sh.failed = 1;
        if (elected) tc_commit<kCtas>(smem_u32(&sh.drain));
        mbar_wait_bounded(smem_u32(&sh.drain), 0, kWaitCycles);
      }
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kEpilogueRegs));
    // ---- results out
    Accumulator acc;
    acc.warp = (warp - kEpilogueWarp0) & 3;
    acc.half = (warp - kEpilogueWarp0) >> 2;
    acc.lane = lane;
    acc.staging = staging + (warp - kEpilogueWarp0) * kStageBufs * kStageBufBytes;
    acc.staged = smem_u32(&sh.staged[warp - kEpilogueWarp0]);
    acc.order = smem_u32(&sh.order[warp - kEpilogueWarp0]);
    acc.order_full = smem_u32(&sh.order_full[warp - kEpilogueWarp0]);
    acc.order_empty = smem_u32(&sh.order_empty[warp - kEpilogueWarp0]);
    const uint32_t mine = tmem + ((uint32_t)(acc.warp * 32) << 16) + acc.half * (kN / 2);
    uint32_t buf = 0, turn = 0;
    bool ok = true;
    const auto wait = [&] {
      ok = __all_sync(0xffffffffu, mbar_wait_bounded(smem_u32(&sh.acc_full[buf]), turn, kLimit));
      tc_fence_after();
      return ok;
    };
    const auto give_back = [&] {
      tc_fence_before();
      __syncwarp();
      if (lane == 0) {
        const uint32_t bar = smem_u32(&sh.acc_empty[buf]);
        if constexpr (kCtas == 2) mbar_arrive_cluster(map_to_cta(bar, 0));
        else mbar_arrive(bar);
      }
      if (++buf == Shape::kAccs) {
        buf = 0;
        turn ^= 1;
      }
    };
    for (typename Job::Ticket ticket; (ticket = feed.next()).i >= 0;) {
      int blocks, small, chunk;
      {
        Tile t;
        job.tile(ticket, cta, t);
        blocks = t.passes * t.k_blocks;
        small = small_blocks(t);
        chunk = t.chunk;
      }
      if constexpr (Job::kClaimed) {
        if (!(ok = job.prefetch(ticket, cta, acc, kLimit))) break;
      } else {
        job.prefetch(ticket, cta, acc);
      }
      if (!wait()) break;
      float v[kN / 2];
      take_columns<false>(v, mine + buf * kN, blocks == 0);
      give_back();
      for (int done = accumulator_end(0, small, blocks, chunk); done < blocks; done = accumulator_end(done, small, blocks, chunk)) {
        if (!wait()) break;
        take_columns<true>(v, mine + buf * kN, false);
        give_back();
      }
      if (!ok) break;
      if constexpr (Job::kClaimed) ok = job.epilogue(ticket, cta, acc, v);
      else job.epilogue(ticket, cta, acc, v);
      if (!ok) break;
      __syncwarp();
    }
    if (!ok || !feed.ok) sh.failed = 1;
    if constexpr (Job::kClaimed) {
      if (!job.finish(acc)) sh.failed = 1;
    }
    if (lane == 0) tma_store_wait_all();
  }

  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if constexpr (kCtas == 2) {
    cluster_arrive();
    cluster_wait();
  }
  tc_fence_after();
  if (warp == 2) tmem_free<kCtas>(tmem, kTmemCols);
  if (threadIdx.x == 0 && sh.failed && job.status()) atomicOr(job.status(), FOPD_DEV_TIMEOUT);
}

// ------------------------------------------------------------------ results out
// 64 columns of a warp's rows as a 128-byte-swizzled box of 16-bit values: pack(j) gives columns 2 j and 2 j + 1.
template <class Pack>
__device__ __forceinline__ void stage_box(uint32_t at, int lane, Pack pack) {
#pragma unroll
  for (int j = 0; j < 8; ++j)
    asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(at + lane * 128 + ((j ^ (lane & 7)) * 16)), "r"(pack(4 * j)),
                 "r"(pack(4 * j + 1)), "r"(pack(4 * j + 2)), "r"(pack(4 * j + 3))
                 : "memory");
}
__device__ __forceinline__ uint4 lds_vector(uint32_t addr) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
  return v;
}
// A warp's staging buffers in turn: the one whose store was read from before the last.
struct Staging {
  uint32_t turn = 0;
  __device__ __forceinline__ uint32_t next(const Accumulator &acc) {
    const uint32_t at = acc.staging + turn * kStageBufBytes;
    turn ^= 1;
    if (acc.lane == 0) tma_store_wait_read<1>();
    __syncwarp();
    return at;
  }
  // One that no store by TMA is going to read, for other uses.
  __device__ __forceinline__ uint32_t idle(const Accumulator &acc) {
    if (acc.lane == 0) tma_store_wait_read<0>();
    __syncwarp();
    return acc.staging;
  }
  __device__ __forceinline__ void send(const Accumulator &acc, const CUtensorMap *map, int x, int y, uint32_t at) {
    fence_async_shared();
    __syncwarp();
    if (acc.lane == 0) {
      tma_store(map, x, y, at);
      tma_store_commit();
    }
  }
};
// 128 bytes of each of a warp's rows to (or added to) rows at any pitch and alignment, by way of a staging buffer so that lanes lie along
// the rows: v are the lane's 32 fp32 or 64 bf16 results; `rows` and `cols` of them exist.
template <int DT>
__device__ __forceinline__ void put_rows_out(uint32_t at, int lane, const float *v, void *to, int64_t pitch, int rows, int cols, bool add) {
  constexpr int kBytes = Elem<DT>::kBytes, kPer = Elem<DT>::kPerVec, kCols = 128 / kBytes;
  if (rows <= 0 || cols <= 0) return;
  char *out = static_cast<char *>(to);
  pitch *= kBytes;
  const bool aligned = (((uintptr_t)out | (uintptr_t)pitch) & 15) == 0;
  const int piece = lane & 7;
  if (DT == FOPD_BF16 && add) {  // (sums are rounded once: the results stay fp32 up to the addition, half of the columns at a time)
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      stage_box(at, lane, [&](int j) { return __float_as_uint(v[(half * 32 + j) % kCols]); });
      __syncwarp();
      for (int r = 0; r < rows; ++r) {
        float x;
        asm volatile("ld.shared.f32 %0, [%1];" : "=f"(x) : "r"(at + r * 128 + (((lane >> 2) ^ (r & 7)) * 16) + (lane & 3) * 4) : "memory");
        if (half * 32 + lane < cols) {
          char *q = out + r * pitch + (half * 32 + lane) * kBytes;
          Elem<DT>::store1(q, 0, x + Elem<DT>::load1(q, 0));
        }
      }
      __syncwarp();
    }
    return;
  }
  stage_box(at, lane, [&](int j) {
    if constexpr (DT == FOPD_F32) return __float_as_uint(v[j]);
    const __nv_bfloat162 h = __floats2bfloat162_rn(v[(2 * j) % kCols], v[(2 * j + 1) % kCols]);
    return *reinterpret_cast<const uint32_t *>(&h);
  });
  __syncwarp();
  if (aligned) {
    for (int r = lane >> 3; r < rows; r += 4) {
      uint4 w = lds_vector(at + r * 128 + ((piece ^ (r & 7)) * 16));
      char *q = out + r * pitch + piece * 16;
      if ((piece + 1) * kPer <= cols) {
        if (DT == FOPD_F32 && add) {
          const float4 o = *reinterpret_cast<const float4 *>(q);
          w.x = __float_as_uint(__uint_as_float(w.x) + o.x), w.y = __float_as_uint(__uint_as_float(w.y) + o.y);
          w.z = __float_as_uint(__uint_as_float(w.z) + o.z), w.w = __float_as_uint(__uint_as_float(w.w) + o.w);
        }
        *reinterpret_cast<uint4 *>(q) = w;
      } else if (piece * kPer < cols) {  // the end of a row
        float x[kPer];
        Elem<DT>::unpack(w, x);
#pragma unroll
        for (int e = 0; e < kPer; ++e)
          if (piece * kPer + e < cols) Elem<DT>::store1(q, e, add ? x[e] + Elem<DT>::load1(q, e) : x[e]);
      }
    }
  } else {
    for (int r = 0; r < rows; ++r) {
      uint32_t w;
      asm volatile("ld.shared.u32 %0, [%1];" : "=r"(w) : "r"(at + r * 128 + (((lane >> 2) ^ (r & 7)) * 16) + (lane & 3) * 4) : "memory");
      char *q = out + r * pitch + lane * 4;
      if constexpr (DT == FOPD_F32) {
        if (lane < cols) *reinterpret_cast<float *>(q) = add ? *reinterpret_cast<float *>(q) + __uint_as_float(w) : __uint_as_float(w);
      } else {
        if (2 * lane < cols) *reinterpret_cast<uint16_t *>(q) = (uint16_t)w;
        if (2 * lane + 1 < cols) *reinterpret_cast<uint16_t *>(q + 2) = (uint16_t)(w >> 16);
      }
    }
  }
  __syncwarp();  // (before the buffer is written again)
}

}  // namespace fopd
