// What the decode attention kernels over a bf16 cache (cmc_attn.cu) and over a
// cache in 8 bits (cmc_attn_q8.cu) share: a launch's parameters, PTX wrappers with bounded
// waits, the sequence state, the clusters' exchange, the workspace's layout and the rotary
// embedding.  (cmc_cache_q8.cu uses the waits.)  Everything here is
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

// --- Bulk copies into shared memory, completing on an mbarrier.
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
__device__ __forceinline__ void prefetch_map(const CUtensorMap* m) {
  asm volatile("prefetch.tensormap [%0];\n" ::"l"(m) : "memory");
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

// Adds one pending arrival to `bar` now and completes it once every cp.async
// this thread issued so far has landed.
__device__ __forceinline__ void mbar_arrive_cp_async(uint64_t* bar) {
  asm volatile("cp.async.mbarrier.arrive.shared::cta.b64 [%0];\n" ::"r"(smem_addr(bar)) : "memory");
}
__device__ __forceinline__ void cp_async_4(uint32_t dst, const void* src, uint32_t src_bytes) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;\n" ::"r"(dst), "l"(src), "r"(src_bytes));
}
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
// p * theta^(-2i/d) of a pair i at position p.  Angles reach 10^5 rad and more, so
// they are reduced in turns with integer arithmetic: with F =
// theta^(-2i/d) / (2 pi) held as a 64-bit binary fraction (`turns`, rounded on the
// host), p * F mod 2^64 is the fractional turn of the angle, off by at most
// p * 2^-65 turns; its top 32 bits, read as a signed fraction of a half turn,
// give the angle in [-pi, pi) for sincospif.  Below p = 2^32 the (cos, sin)
// pairs are within 1e-7 of exact (checked against 200-bit arithmetic); a
// double-precision product p * theta^(-2i/d) would be off by p * 2^-53 rad.
__device__ __forceinline__ float2 rope_cos_sin(unsigned long long p, unsigned long long turns) {
  const unsigned long long frac = p * turns;  // mod 2^64: the fractional turn
  const int hi = static_cast<int>(static_cast<long long>(frac) >> 32);  // [-2^31, 2^31)
  // angle / pi = 2 * turn in [-1, 1)
  const float x = static_cast<float>(hi) * 4.656612873077393e-10f;  // 2^-31
  float sn, cn;
  sincospif(x, &sn, &cn);
  return make_float2(cn, sn);
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
