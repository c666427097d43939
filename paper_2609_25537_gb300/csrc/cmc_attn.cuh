// What the decode attention kernels over a bf16 cache (cmc_attn.cu) and over a
// cache in 8 bits (cmc_attn_q8.cu) share: PTX wrappers with bounded waits, the
// sequence state, the clusters' exchange, the workspace's layout and the rotary
// frequencies; and what the first has to itself of the walk over a launch's (unit, tile)
// list, the merge of split units and the plan.  Everything here is
// internal to the translation unit that includes it.
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include <cstring>
#include <mutex>

#include "cmc_internal.cuh"

namespace cmc {

constexpr int kWarps = 4;  // consumer warps of an attention CTA
constexpr int kThreads = 32 * kWarps;
constexpr size_t kWsHeader = 256;
// Largest cluster of CTAs that share one unit (the portable cluster size).
constexpr int kMaxClusterCtas = 8;

// fp32 partial record of one CTA's share of a unit: max[G], sum[G], then, from
// a 16-byte aligned offset, the unnormalised output [G][d].
__host__ __device__ constexpr int rec_out_offset(int G) { return (2 * G + 3) & ~3; }
__host__ __device__ constexpr int rec_floats(int G, int D) { return rec_out_offset(G) + G * D; }

struct AttnParams {
  const uint16_t* q;      // [B, L, Hq, d]
  const uint16_t* t1k;    // [B, L, Hkv, N, d]
  const uint16_t* t1v;    // [B, L, Hkv, N, d]
  const int32_t* idx;     // [B, k], or NULL: Tier-1 is rows 0 .. k-1 of t1k / t1v
  uint16_t* ring_k;       // [B, L, Hkv, W, d]
  uint16_t* ring_v;       // [B, L, Hkv, W, d]
  int64_t* pos;           // [B]
  const uint16_t* k_new;  // [B, L, Hkv, d]   (fused step only)
  const uint16_t* v_new;  // [B, L, Hkv, d]
  uint16_t* out;          // [B, L, Hq, d]
  uint32_t* status;       // workspace status word
  unsigned long long* tickets;  // [B] tiles whose pos read is done (fused step)
  float* partials;        // [units, tpu, G * (d + 2)]
  int B, L, Hq, Hkv, N, k, W;
  int tpu;                // tiles per unit: t1_tiles Tier-1 tiles, then the ring tiles
  int t1_tiles;           // of them Tier-1 tiles
  int rot;                // in-unit processing order: tile (j + rot) % tpu at position j
  int LH;                 // units per sequence: L * Hkv
  int base;               // granules per CTA (CTAs below `rem` take one more); cluster plan:
  int rem;                // tiles of the unit per CTA of the cluster, likewise
  int cm;                 // > 0: clusters of cm CTAs share each unit (CTA j of the cluster
                          // takes positions j, j + cm, ...); 0: flat split
  int slice;              // cluster plan: 4-column output groups each CTA finishes
  int gran;               // flat split: tiles per granule (1, or tpu: whole units per CTA)
  float scale_log2;       // softmax scale * log2(e)
  long long rope_offset;  // rotary embedding (GQA-layer step): position of ring token 0
  int l2_prefetch;        // box tiles per CTA prefetched into L2 before the grid dependency wait
  unsigned long long rope_turns[64];  // theta^(-2i/d) / (2 pi) of the d/2 pairs as 0.64 fixed
                                      // point (turns per position), computed on the host
  int rope_slot;          // >= 0: the same table in g_rope_tables[rope_slot] (read from there)
  uint32_t stall_tx;      // 0; the failure-path test hook: bytes every stage expects beyond
                          // what its loads deliver, so that no stage ever completes
};

// Rotary frequency tables in device memory, one per (theta, d) a device has
// seen, written once by the host before the first launch that uses it and
// never changed afterwards.  The producer reads its lanes' two entries with
// plain global loads before the grid dependency wait; reading them from the
// kernel parameters instead (lane-indexed parameter space) measured 0.2-0.3 us
// more per launch.  When no slot is available the parameters are used.
constexpr int kRopeSlots = 16;
static __device__ unsigned long long g_rope_tables[kRopeSlots][64];

// ---------------------------------------------------------------------------
// PTX wrappers
// ---------------------------------------------------------------------------

__device__ __forceinline__ uint32_t smem_addr(const void* p) {
  return static_cast<uint32_t>(__cvta_generic_to_shared(p));
}

__device__ __forceinline__ void ldsm_x4(uint32_t addr, uint32_t& r0, uint32_t& r1, uint32_t& r2,
                                        uint32_t& r3) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];\n"
               : "=r"(r0), "=r"(r1), "=r"(r2), "=r"(r3)
               : "r"(addr));
}
__device__ __forceinline__ void ldsm_x4_t(uint32_t addr, uint32_t& r0, uint32_t& r1, uint32_t& r2,
                                          uint32_t& r3) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];\n"
               : "=r"(r0), "=r"(r1), "=r"(r2), "=r"(r3)
               : "r"(addr));
}

// C[16x8] += A[16x16] B[16x8], bf16 inputs, fp32 accumulators (all 16 rows of A).
__device__ __forceinline__ void mma_16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2,
                                          uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, "
      "{%8,%9}, {%0,%1,%2,%3};\n"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// C[16x8] = A[16x16] B[16x8]: the first step of an accumulator chain (its zeros
// need no registers).
__device__ __forceinline__ void mma_16816_zero(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2,
                                               uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, "
      "{%8,%9}, {%10,%10,%10,%10};\n"
      : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}

// Transpose of an 8x8 matrix of 16-bit elements held one pair per thread
// (thread l: row l/4, columns 2(l%4) and 2(l%4)+1).
__device__ __forceinline__ uint32_t movmatrix_trans(uint32_t a) {
  uint32_t d;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;\n" : "=r"(d) : "r"(a));
  return d;
}

// 2^x with the ex2.approx instruction (ex2(-inf) = +0).
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;\n" : "=f"(y) : "f"(x));
  return y;
}

// --- mbarrier (shared::cta).  Every wait is bounded in wall time: a waiter
// that has not seen its phase complete kWaitNs after it started polling
// (%globaltimer, nanoseconds) raises the CTA's abort flag, reports
// CMC_DEVFLAG_TIMEOUT and gives up; once the flag is up every other wait of
// the CTA whose phase is not complete gives up at its next poll.  A poll-count
// cap backs the deadline up in case the timer ever stood still.  Named-barrier
// and cluster-barrier participation never depends on whether a wait succeeded
// (see the kernel), so a CTA whose waits gave up still reaches its end.
constexpr uint32_t kWaitNs = 1000000000u;  // 1 s: the kernel runs for microseconds
constexpr uint32_t kPeerWaitNs = 3000000000u;  // for a cluster's other CTAs: see mbar_wait_peers
constexpr uint32_t kDrainNs = 2000000u;    // after a timeout: wait for issued loads
constexpr uint32_t kMaxWaitPolls = 1u << 28;

// Low 32 bits of %globaltimer (nanoseconds).  Differences of readings less
// than 2^32 ns (4.29 s) apart are exact in unsigned 32-bit arithmetic.
__device__ __forceinline__ uint32_t global_ns32() {
  uint32_t t;
  asm volatile("mov.u32 %0, %%globaltimer_lo;\n" : "=r"(t));
  return t;
}

__device__ __forceinline__ void mbar_init(uint64_t* bar, uint32_t count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;\n" ::"r"(smem_addr(bar)), "r"(count));
}
__device__ __forceinline__ void mbar_arrive(uint64_t* bar) {
  asm volatile("{\n .reg .b64 st;\n mbarrier.arrive.shared::cta.b64 st, [%0];\n}\n" ::"r"(
                   smem_addr(bar))
               : "memory");
}
__device__ __forceinline__ void mbar_arrive_expect_tx(uint64_t* bar, uint32_t bytes) {
  asm volatile(
      "{\n .reg .b64 st;\n mbarrier.arrive.expect_tx.shared::cta.b64 st, [%0], %1;\n}\n" ::"r"(
          smem_addr(bar)),
      "r"(bytes)
      : "memory");
}
__device__ __forceinline__ bool mbar_try_wait(uint64_t* bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n .reg .pred p;\n mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n"
      " selp.u32 %0, 1, 0, p;\n}\n"
      : "=r"(ok)
      : "r"(smem_addr(bar)), "r"(parity)
      : "memory");
  return ok != 0;
}
// The CTA's abort flag: raised by the first wait that times out.
static __shared__ int attn_abort;

__device__ __forceinline__ bool attn_aborted() { return *static_cast<volatile int*>(&attn_abort) != 0; }

// Waits for the phase of `bar` with the given parity to complete.  False when
// the CTA's abort flag is (or goes) up, or on timeout, which raises it.
__device__ __forceinline__ bool mbar_wait_slow(uint64_t* bar, uint32_t parity) {
  const uint32_t t0 = global_ns32();
  for (uint32_t it = 0; it < kMaxWaitPolls; ++it) {
    if (mbar_try_wait(bar, parity)) return true;
    if (attn_aborted()) return false;
    if (global_ns32() - t0 > kWaitNs) break;
  }
  *static_cast<volatile int*>(&attn_abort) = 1;
  return false;
}
__device__ __forceinline__ bool mbar_wait(uint64_t* bar, uint32_t parity) {
  return mbar_try_wait(bar, parity) || mbar_wait_slow(bar, parity);
}

// --- TMA loads into shared memory, completing on an mbarrier.
// A 2-D TMA box load into shared memory, completing on an mbarrier, with an
// L2 cache policy (createpolicy) attached.
__device__ __forceinline__ void tma_box_hint(uint32_t dst, const CUtensorMap* map, int col, int row,
                                             uint64_t* bar, uint64_t policy) {
  asm volatile(
      "cp.async.bulk.tensor.2d.shared::cta.global.tile.mbarrier::complete_tx::bytes.L2::cache_hint"
      " [%0], [%1, {%2, %3}], [%4], %5;\n" ::"r"(dst),
      "l"(map), "r"(col), "r"(row), "r"(smem_addr(bar)), "l"(policy)
      : "memory");
}
__device__ __forceinline__ uint64_t policy_evict_first() {
  uint64_t pol;
  asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;\n" : "=l"(pol));
  return pol;
}
__device__ __forceinline__ void bulk_copy(uint32_t dst, const void* src, uint32_t bytes,
                                          uint64_t* bar) {
  asm volatile(
      "cp.async.bulk.shared::cta.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];\n" ::"r"(
          dst),
      "l"(src), "r"(bytes), "r"(smem_addr(bar))
      : "memory");
}

// L2 prefetch of one TMA box and of a contiguous byte range.  These are hints:
// no data reaches the issuing thread and the L2 stays coherent with the
// previous kernel's writes, so they may be issued before the grid dependency
// wait.
__device__ __forceinline__ void tma_prefetch_l2(const CUtensorMap* map, int col, int row) {
  asm volatile("cp.async.bulk.prefetch.tensor.2d.L2.global.tile [%0, {%1, %2}];\n" ::"l"(map),
               "r"(col), "r"(row)
               : "memory");
}
__device__ __forceinline__ void prefetch_map(const CUtensorMap* m) {
  asm volatile("prefetch.tensormap [%0];\n" ::"l"(m) : "memory");
}
__device__ __forceinline__ void bulk_prefetch_l2(const void* src, uint32_t bytes) {
  asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;\n" ::"l"(src), "r"(bytes) : "memory");
}

// Named barrier over the consumer warps only (the producer warp never joins).
__device__ __forceinline__ void consumer_sync() {
  asm volatile("bar.sync 1, %0;\n" ::"n"(kWarps * 32) : "memory");
}

// --- thread-block cluster: barrier (every thread of every CTA of the
// cluster arrives, then waits) and stores into a peer CTA's shared memory.
__device__ __forceinline__ void cluster_arrive() {
  asm volatile("barrier.cluster.arrive.release;\n" ::: "memory");
}
__device__ __forceinline__ void cluster_wait() {
  asm volatile("barrier.cluster.wait.acquire;\n" ::: "memory");
}
__device__ __forceinline__ void cluster_sync_all() {
  cluster_arrive();
  cluster_wait();
}
__device__ __forceinline__ uint32_t cluster_ctarank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;\n" : "=r"(r));
  return r;
}
__device__ __forceinline__ uint32_t cluster_id() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%clusterid.x;\n" : "=r"(r));
  return r;
}
__device__ __forceinline__ uint32_t peer_smem(uint32_t local_addr, uint32_t rank) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;\n" : "=r"(r) : "r"(local_addr), "r"(rank));
  return r;
}
// Asynchronous stores into a peer CTA's shared memory, counted in bytes by a
// barrier there.
__device__ __forceinline__ void st_peer_f4(uint32_t addr, const float4& v, uint32_t bar) {
  asm volatile(
      "st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.v4.f32 [%0], {%1, %2, %3, %4}, [%5];\n" ::"r"(
          addr),
      "f"(v.x), "f"(v.y), "f"(v.z), "f"(v.w), "r"(bar)
      : "memory");
}
__device__ __forceinline__ void st_peer_f2(uint32_t addr, float x, float y, uint32_t bar) {
  asm volatile(
      "st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.v2.f32 [%0], {%1, %2}, [%3];\n" ::"r"(
          addr),
      "f"(x), "f"(y), "r"(bar)
      : "memory");
}
// Out of line: the wait it belongs to is on every cluster's way to its output
// (inlined, clusters of 8 took 1 % more).
static __device__ __noinline__ void peers_gave_up() {
  *static_cast<volatile int*>(&attn_abort) = 1;
  cluster_sync_all();  // over the threads of the cluster that have not ended
  const uint32_t t0 = global_ns32();
  for (uint32_t it = 0; it < (1u << 16) && global_ns32() - t0 < kDrainNs; ++it) __nanosleep(1000);
}

// Waits for the peers' stores counted by `bar` (phase 0).  Unlike the pipeline's
// waits it does not end with the CTA's abort flag: a CTA must not leave while
// its peers still store into its shared memory.  Peers that gave up have done
// so within kWaitNs of the cluster's start and store all the same, so the
// limit (kPeerWaitNs) lies well behind theirs.  Should it pass even so, the CTA
// stays until every peer has come to the same point or has ended (each does:
// its own waits are bounded), and kDrainNs longer for stores on the way.
__device__ __forceinline__ void mbar_wait_peers(uint64_t* bar) {
  const uint32_t t0 = global_ns32();
  for (uint32_t it = 0; it < kMaxWaitPolls; ++it) {
    uint32_t ok;
    asm volatile(
        "{\n .reg .pred p;\n mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], 0;\n"
        " selp.u32 %0, 1, 0, p;\n}\n"
        : "=r"(ok)
        : "r"(smem_addr(bar))
        : "memory");
    if (ok) return;
    if (global_ns32() - t0 > kPeerWaitNs) break;
  }
  peers_gave_up();
}

// Per-stage header words: rows of the tile that may hold a key, the new
// token's ring slot and tile row (fused step; -1 if not in this tile),
// whether any of the tile's rows holds no key (its V row must be zeroed), and
// the bit masks of rows 0-31 / 32-63 whose Tier-1 index is out of range.
// Stage 0's also holds, in its last two words, pos of the CTA's first sequence
// on its way to the producer.
enum { H_NROWS = 0, H_NEWSLOT = 1, H_NEWROW = 2, H_MASKED = 3, H_BADLO = 4, H_BADHI = 5, H_POS = 6 };

// A consumer's wait for a stage.  One that gives up
//  - marks the stage's header as that of a tile without keys: the barrier, stuck
//    in its phase, reports the phase before as complete, which has the parity
//    of the stage's next tile, so the warp's wait for that one passes;
//  - ends the warp's hand-backs (`release` is 0 in lane 0 before): the producer,
//    which then finds the abort flag up, refills no stage whose loads may not
//    have landed.
// That leaves the tile loop as it was.  A flag of the warp's own tested a tile
// instead cost 0.3 % of a Llama-shaped step and 0.7 % of 8 x (30 + 130) keys, the
// abort flag read by the producer a tile up to 1.7 %.
__device__ __forceinline__ bool mbar_wait_stage(uint64_t* bar, uint32_t parity, int* header,
                                                int& release) {
  if (mbar_wait(bar, parity)) return true;
  header[H_NROWS] = 0;
  header[H_NEWROW] = -1;
  header[H_MASKED] = 1;
  release = 1;
  return false;
}

__device__ __forceinline__ long long cta_first_tile(long long c, long long base, long long rem) {
  return c * base + (c < rem ? c : rem);
}
__device__ __forceinline__ long long cta_of_tile(long long t, long long base, long long rem) {
  const long long big = rem * (base + 1);
  return t < big ? t / (base + 1) : rem + (t - big) / base;
}
// Partial-record slot (tile position within the unit) of CTA c's share of
// the unit whose first tile is ut0: the position of c's first tile in it.
__device__ __forceinline__ long long rec_slot(const AttnParams& p, long long c, long long ut0) {
  const long long t = cta_first_tile(c, p.base, p.rem);
  return t > ut0 ? t - ut0 : 0;
}

// The tile at a position of the flattened (unit, j) order, advanced one tile
// at a time so that the main loop does no integer division.  Within a unit,
// position j holds key tile lt = (j + rot) % tpu: ring tiles come first, so a
// CTA's first loads need no idx entries.  A CTA of a cluster takes every
// cm-th position of its one unit.  Units are numbered ((b L) + l) Hkv + g, so
// a unit's query and output rows start at row u G of [B, L, Hq, d].
struct TileCursor {
  int u, j, lt, b;  // unit, position and key tile within it, the unit's sequence
  int left;         // units of sequence b from u on
  __device__ __forceinline__ void init(int unit, int pos, const AttnParams& p) {
    u = unit;
    j = pos;
    lt = j + p.rot;
    if (lt >= p.tpu) lt -= p.tpu;
    b = static_cast<int>(static_cast<unsigned>(u) / static_cast<unsigned>(p.LH));
    left = (b + 1) * p.LH - u;
  }
  __device__ __forceinline__ void next(const AttnParams& p) {
    if (p.cm > 0) {
      j += p.cm;
    } else if (++j == p.tpu) {
      j = 0;
      ++u;
      if (--left == 0) {
        left = p.LH;
        ++b;
      }
    }
    lt = j + p.rot;
    if (lt >= p.tpu) lt -= p.tpu;
  }
};

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, uint32_t src_bytes) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;\n" ::"r"(dst), "l"(src), "r"(src_bytes));
}
__device__ __forceinline__ void cp_async16_hint(uint32_t dst, const void* src, uint32_t src_bytes,
                                                uint64_t policy) {
  asm volatile("cp.async.cg.shared.global.L2::cache_hint [%0], [%1], 16, %2, %3;\n" ::"r"(dst), "l"(src),
               "r"(src_bytes), "l"(policy));
}
__device__ __forceinline__ void cp_async16_all(uint32_t dst, const void* src, uint64_t policy) {
  asm volatile("cp.async.cg.shared.global.L2::cache_hint [%0], [%1], 16, %2;\n" ::"r"(dst), "l"(src),
               "l"(policy));
}
// Adds one pending arrival to `bar` now and completes it once every cp.async
// this thread issued so far has landed.
__device__ __forceinline__ void mbar_arrive_cp_async(uint64_t* bar) {
  asm volatile("cp.async.mbarrier.arrive.shared::cta.b64 [%0];\n" ::"r"(smem_addr(bar)) : "memory");
}
__device__ __forceinline__ void cp_async_4(uint32_t dst, const void* src, uint32_t src_bytes) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;\n" ::"r"(dst), "l"(src), "r"(src_bytes));
}
__device__ __forceinline__ void cp_async_8(uint32_t dst, const void* src) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 8;\n" ::"r"(dst), "l"(src));
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;\n" ::); }
template <int N>
__device__ __forceinline__ void cp_async_wait() {
  asm volatile("cp.async.wait_group %0;\n" ::"n"(N) : "memory");
}


// What a sequence's pos gives every tile of that sequence: the ring slots
// that hold keys and the new token's slot (fused step).  Computed once per
// run of tiles of one sequence.
struct SeqState {
  long long pos;
  int count;     // occupied ring slots (after the append in the fused step)
  int new_slot;  // ring slot of the new token, -1 if none
  bool bad;      // pos < 0: the sequence is skipped
};

template <bool FUSED>
__device__ __forceinline__ SeqState seq_state(const AttnParams& p, long long pos) {
  SeqState q;
  q.pos = pos;
  q.bad = pos < 0;
  q.count = 0;
  q.new_slot = -1;
  if (!q.bad) {
    if (FUSED) {
      q.count = static_cast<int>(pos + 1 < p.W ? pos + 1 : p.W);
      // a 32-bit remainder where it will do (the 64-bit one is a long call on
      // the way to every launch's first tile)
      q.new_slot = (pos >> 32) == 0
                       ? static_cast<int>(static_cast<unsigned>(pos) % static_cast<unsigned>(p.W))
                       : static_cast<int>(pos % p.W);
    } else {
      q.count = static_cast<int>(pos < p.W ? pos : p.W);
    }
  }
  return q;
}

// pos[b] through L2 (another CTA of this launch advances it once every reader
// has counted itself; the kernel before may have advanced it).
__device__ __forceinline__ long long ld_pos(const AttnParams& p, int b) {
  long long v;
  asm volatile("ld.global.cg.s64 %0, [%1];\n" : "=l"(v) : "l"(p.pos + b) : "memory");
  return v;
}

// Rotary embedding of a GQA-layer step: (cos, sin) of the angle
// p * theta^(-2i/d) of pairs i = lane and lane + 32 (i < d/2) at the new
// token's position p = rope_offset + pos.  Angles reach 10^5 rad and more, so
// they are reduced in turns with integer arithmetic: with F_i =
// theta^(-2i/d) / (2 pi) held as a 64-bit binary fraction (rounded on the
// host), p * F_i mod 2^64 is the fractional turn of the angle, off by at most
// p * 2^-65 turns; its top 32 bits, read as a signed fraction of a half turn,
// give the angle in [-pi, pi) for sincospif.  Below p = 2^32 the (cos, sin)
// pairs are within 1e-7 of exact (checked against 200-bit arithmetic); a
// double-precision product p * theta^(-2i/d) would be off by p * 2^-53 rad.
// `turns` holds F_lane and F_(lane+32) (0 past d/2), loaded from the kernel
// parameters before the grid dependency wait.
template <int D>
__device__ __forceinline__ void rope_pairs(const AttnParams& p, long long pos,
                                           const unsigned long long (&turns)[2], int lane,
                                           float2 (&cs)[2]) {
  const unsigned long long pp = static_cast<unsigned long long>(p.rope_offset + pos);
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    const int i = lane + 32 * e;
    cs[e] = make_float2(1.f, 0.f);
    if (i < D / 2) {
      const unsigned long long frac = pp * turns[e];  // mod 2^64: the fractional turn
      const int hi = static_cast<int>(static_cast<long long>(frac) >> 32);  // [-2^31, 2^31)
      // angle / pi = 2 * turn in [-1, 1)
      const float x = static_cast<float>(hi) * 4.656612873077393e-10f;  // 2^-31
      float sn, cn;
      sincospif(x, &sn, &cn);
      cs[e] = make_float2(cn, sn);
    }
  }
}

// Fused step: a CTA has read pos[b] for its run of `tiles` tiles of sequence
// b.  The run that brings the sequence's count to all of its tiles is the last
// reader of pos[b]; it advances pos[b] and clears the count for the next call.
__device__ __forceinline__ void seq_run_done(const AttnParams& p, int b, int tiles,
                                             const SeqState& sq) {
  const unsigned long long total = static_cast<unsigned long long>(p.LH) * p.tpu;
  const unsigned long long old = atomicAdd(p.tickets + b, static_cast<unsigned long long>(tiles));
  if (old + static_cast<unsigned long long>(tiles) == total) {
    if (!sq.bad) p.pos[b] = sq.pos + 1;
    p.tickets[b] = 0ull;
  }
}

// Finishes the units that two_tier_attn_kernel split between CTAs: merges
// their fp32 partial records (max, sum, output per head) with a log-sum-exp
// rescale and writes the bf16 output.  Runs after two_tier_attn_kernel on the
// same stream, only when some unit was split; one CTA per unit.
template <int D, int G>
static __global__ void __launch_bounds__(kThreads)
two_tier_combine_kernel(const AttnParams p) {
  asm volatile("griddepcontrol.wait;\n" ::: "memory");  // the attention kernel's records
  asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");
  const int u = blockIdx.x;
  const long long ut0 = static_cast<long long>(u) * p.tpu;
  const long long c0 = cta_of_tile(ut0, p.base, p.rem);
  const long long c1 = cta_of_tile(ut0 + p.tpu - 1, p.base, p.rem);
  if (c0 == c1) return;  // written by the attention kernel
  // one record per CTA that holds part of the unit, at the slot of that
  // CTA's first tile in the unit (slot 0 for c0)
  const int nrec = static_cast<int>(c1 - c0 + 1);
  constexpr int PW = rec_floats(G, D);
  const float* recs = p.partials + ut0 * PW;
  const long long out_base = static_cast<long long>(u) * (G * D);
  for (int x = threadIdx.x; x < G * D / 2; x += blockDim.x) {
    const int hh = (2 * x) / D;
    const int c = (2 * x) % D;
    float M = -INFINITY;
    for (int r = 0; r < nrec; ++r) M = fmaxf(M, recs[rec_slot(p, c0 + r, ut0) * PW + hh]);
    float Ls = 0.f, O0 = 0.f, O1 = 0.f;
    if (M != -INFINITY) {
      for (int r = 0; r < nrec; ++r) {
        const float* pr = recs + rec_slot(p, c0 + r, ut0) * PW;
        const float f = ex2(pr[hh] - M);
        const float2 o2 = *reinterpret_cast<const float2*>(pr + rec_out_offset(G) + hh * D + c);
        Ls = fmaf(f, pr[G + hh], Ls);
        O0 = fmaf(f, o2.x, O0);
        O1 = fmaf(f, o2.y, O1);
      }
    }
    const float inv = Ls > 0.f ? 1.f / Ls : 0.f;
    *reinterpret_cast<uint32_t*>(p.out + out_base + hh * D + c) = pack_bf16x2(O0 * inv, O1 * inv);
  }
}

// ---------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------

// A workspace: [0, 256) status word; then one 8-byte pos-read count per sequence
// (padded to 256 bytes); then the partial records.
static inline size_t ws_partials_off(int B) {
  return kWsHeader + ((static_cast<size_t>(B) * 8 + 255) / 256) * 256;
}

// cuTensorMapEncodeTiled, reached through the runtime's driver entry point.
typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*,
                                  const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                  const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                  CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

static EncodeTiledFn encode_fn() {
  static EncodeTiledFn fn = nullptr;
  static std::once_flag once;
  std::call_once(once, [] {
    void* f = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &q) ==
            cudaSuccess &&
        q == cudaDriverEntryPointSuccess)
      fn = reinterpret_cast<EncodeTiledFn>(f);
  });
  return fn;
}

// A [rows, d] bf16 tensor viewed by boxes of 64 columns x box_rows rows,
// Launch plan of one attention call on the current device.
struct AttnPlan {
  long long ctas, base, rem;  // grid size; flat split: granules per CTA (the first `rem` take one more)
  int gran;                   // flat split: tiles per granule
  int cm;                     // > 0: clusters of cm CTAs per unit (DSMEM merge, no combine)
  bool split;                 // flat split cuts some unit: the combine kernel runs
};

// The plan of units of `tpu` tiles each on the current device, `per_sm` CTAs of the
// attention kernel resident on an SM.
static inline void plan_grid(long long total_tiles, int tpu, int per_sm, AttnPlan* pl) {
  // Grid.  With no more units than resident CTAs: m = resident CTAs per unit,
  // at most one per tile and at most 8 (the portable cluster size).  m = 1:
  // one CTA per unit, nothing is split.  m >= 2: clusters of m CTAs per unit,
  // merged in distributed shared memory.  More units than resident CTAs: one
  // wave of CTAs, each taking a run of whole units or, when that would leave
  // too few CTAs for the last round, an equal share of the flattened tiles
  // (stream-K; the combine kernel merges the units cut between CTAs).  (A flat split
  // for few, long units -- m up to 38 at one sequence of one layer -- left
  // about one tile per CTA and a combine over 38 records: 33.4 us against
  // 9.4 us for clusters of 8 at k = 1024, W = 2048.)
  const long long slots = static_cast<long long>(per_sm) * sm_count();
  const long long units = total_tiles / tpu;
  pl->cm = 0;
  long long ctas;
  if (units <= slots) {
    long long m = slots / units;
    if (m > tpu) m = tpu;
    if (m > kMaxClusterCtas) m = kMaxClusterCtas;
    if (m >= 2) pl->cm = static_cast<int>(m);
    ctas = units * m;
  } else {
    ctas = slots;
  }
  if (ctas > total_tiles) ctas = total_tiles;
  if (ctas < 1) ctas = 1;
  pl->ctas = ctas;
  pl->gran = 1;
  pl->base = total_tiles / ctas;
  pl->rem = total_tiles % ctas;
  // More units than resident CTAs: whole units per CTA (contiguous runs, no
  // combine launch) when they divide evenly or when at least half of the CTAs
  // take one unit more -- enough CTAs then stream the last round to keep HBM
  // busy; with fewer, those few CTAs would stream their extra unit alone and
  // the balanced stream-K split with its combine is faster.  Measured at
  // 128 + 512-key units: 312 units 21.1 us stream-K / 23.7 us whole units,
  // 384 units 24.5 / 25.5, 448 units 26.0 / 26.2, 512 units 30.1 / 27.1.
  const long long ru = units % ctas;
  if (units > slots && (ru == 0 || 2 * ru >= ctas)) {
    pl->gran = tpu;
    pl->base = units / ctas;
    pl->rem = ru;
  }
  // Flat split: is any unit cut between CTAs (a CTA boundary inside a unit)?
  if (units <= slots && pl->cm == 0) {  // one CTA per unit: whole units, one each
    pl->gran = tpu;
    pl->base = 1;
    pl->rem = 0;
  }
  if (pl->cm > 0) {
    pl->base = tpu / pl->cm;
    pl->rem = tpu % pl->cm;
  }
  pl->split = false;
  for (long long c = 1; pl->cm == 0 && pl->gran == 1 && c < ctas && !pl->split; ++c) {
    const long long t = c * pl->base + (c < pl->rem ? c : pl->rem);
    pl->split = (t % tpu) != 0;
  }
}

// theta^(-2i/d) / (2 pi) -- the pair's turns per position, below 1/6 -- as a
// 64-bit binary fraction, rounded to nearest, computed in long double.
static unsigned long long rope_turns_fixed(double theta, int i, int d) {
  const long double two_pi = 6.283185307179586476925286766559L;
  const long double t = powl(static_cast<long double>(theta), -2.0L * i / d) / two_pi;
  return static_cast<unsigned long long>(t * 18446744073709551616.0L + 0.5L);  // t * 2^64
}

// The turns of all pairs of (theta, d), zero past d / 2.  The first kRopeSlots
// pairs of values seen are kept: a call otherwise computes d / 2 long-double
// powers, which where long double is a software format (Arm) is most of the
// call.  Bounded, and guarded for calls from several threads.
static void rope_turns_table(double theta, int d, unsigned long long (&out)[64]) {
  static std::mutex mu;
  static int n = 0;
  static double thetas[kRopeSlots];
  static int ds[kRopeSlots];
  static unsigned long long tables[kRopeSlots][64];
  std::lock_guard<std::mutex> lock(mu);
  for (int i = 0; i < n; ++i)
    if (thetas[i] == theta && ds[i] == d) {
      memcpy(out, tables[i], sizeof(out));
      return;
    }
  for (int i = 0; i < 64; ++i) out[i] = i < d / 2 ? rope_turns_fixed(theta, i, d) : 0ull;
  if (n < kRopeSlots) {
    memcpy(tables[n], out, sizeof(out));
    thetas[n] = theta;
    ds[n] = d;
    ++n;
  }
}

// The slot of g_rope_tables holding the table of (theta, d) on the current
// device, writing it on first use; -1 (use the kernel parameters) when the
// slots are full, the stream is being captured into a graph, or the copy
// fails.  A copy from pageable memory may return before it has reached the
// device, and is ordered with the legacy default stream only, while the kernel
// reads the table on any stream, before its grid dependency wait: so the slot
// is used once that stream has been waited for, and every later launch sees
// the table.
struct RopeSlots {
  std::mutex mu;
  int n = 0;
  double theta[kRopeSlots];
  int d[kRopeSlots];
};
static RopeSlots g_rope_slots[64];

static int rope_slot(double theta, int d, const unsigned long long* table, cudaStream_t s) {
  int dev = -1;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) {
    cudaGetLastError();
    return -1;
  }
  RopeSlots& c = g_rope_slots[dev];
  std::lock_guard<std::mutex> lock(c.mu);
  for (int i = 0; i < c.n; ++i)
    if (c.theta[i] == theta && c.d[i] == d) return i;
  if (c.n >= kRopeSlots) return -1;
  cudaStreamCaptureStatus cs = cudaStreamCaptureStatusNone;
  if (cudaStreamIsCapturing(s, &cs) != cudaSuccess || cs != cudaStreamCaptureStatusNone) {
    cudaGetLastError();
    return -1;
  }
  if (cudaMemcpyToSymbol(g_rope_tables, table, 64 * sizeof(unsigned long long),
                         static_cast<size_t>(c.n) * 64 * sizeof(unsigned long long),
                         cudaMemcpyHostToDevice) != cudaSuccess ||
      cudaStreamSynchronize(cudaStreamLegacy) != cudaSuccess) {
    cudaGetLastError();
    return -1;
  }
  c.theta[c.n] = theta;
  c.d[c.n] = d;
  return c.n++;
}
}  // namespace cmc
