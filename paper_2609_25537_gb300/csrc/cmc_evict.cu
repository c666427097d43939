// Eviction from a cache by accumulated attention weight (cmc_evict_cache): per (sequence, layer, KV
// head) unit the heaviest and the youngest tokens are kept and moved together, in order of age.
//
// Bound: HBM, the kept rows read and written (8 d bytes each) beside 4 bytes a token to choose by.  Two parts.  The
// choice of a unit is a CTA's: the order-preserving 32-bit keys of its tokens' weights go to shared memory, a radix
// select of up to three passes (11, 11 and 10 bits) finds the threshold, and every kept token gets its number from
// what the warps and lanes before it keep.  The copy moves blocks of rows.  Enough units for the SMs: a CTA of 256
// threads does both, its copy beside others' choices and the youngest rows, which need none, on their way to L2
// meanwhile (256 units of 512 tokens, 256 kept, 64 of them for their age: 14.4 us, without that prefetch 15.1; the
// choice is 3.5, in all CTAs at once; 10.2 at the copy rate).  Few long ones: a kernel of CTAs of 1,024 threads
// chooses, and a second one copies with all SMs: 64 units of 16,384 tokens, 2,048 kept, 35 us, 11 and 20 of them the
// two kernels', 20.9 at the copy rate.  (Both in clusters of four: 38.8 where the CTAs summed their histograms in
// distributed shared memory, which alone took 2.7 a pass, and 42 where each chose by itself; 38.7 with the rows above
// the first pass's bin prefetched one by one.)
//
// The i-th token kept is never older than the i-th of all, so in place (output and input the same tensors, the oldest
// token in row 0) a row is written only where rows of the same or of earlier blocks were read, and a barrier over the
// unit's CTAs between a block's loads and its stores is all that it takes.
#include <algorithm>
#include <atomic>

#include "cmc_attn.cuh"
#include "cmc_ranges.cuh"

namespace cmc {

constexpr int kEvictThreads = 256;   // of a CTA that copies
constexpr int kChooseThreads = 1024;  // of one that only chooses
constexpr int kEvictBatch = 4;       // rows of K and of V that a thread has in flight
constexpr int kEvictBins = 2048;     // 11 bits a pass
constexpr int kEvictAhead = 65536;   // bytes of K, of V and of the weights of a unit that are prefetched into L2
constexpr int kEvictKeys = 49152;    // keys held in shared memory; of longer units the weights are read again

struct EvictParams {
  const uint16_t* k;     // [units, T, d]
  const uint16_t* v;
  const float* weight;   // [units, T]
  const int64_t* pos;    // [B] or NULL
  uint16_t* out_k;       // [units, R, d]
  uint16_t* out_v;
  float* out_weight;     // [units, R]
  int32_t* idx;          // [units, keep]
  int64_t* out_pos;      // [B] or NULL
  int64_t* evicted;      // [B] or NULL
  uint32_t* status;
  unsigned long long* tickets;
  int T, R, keep, recent, LH, in_place;
  int cm;                // CTAs that copy a unit
};

// Larger weight, larger key; -0 is 0, a NaN is below everything.
__device__ __forceinline__ uint32_t weight_key(float w) { return w != w ? 0u : orderable(w + 0.f); }

// Ages that are numbered together: a bit each, and counts that fit in 16 bits.
constexpr int kSegment = 16384;
constexpr int kWords = kSegment / 32;

template <int NT>
struct __align__(16) ChooseSmem {
  uint32_t bins[kEvictBins];
  uint32_t gt[kWords], eq[kWords];  // above the threshold, and at it; then those that stay, and the number of the first
  uint32_t part[NT / 32];
  uint32_t found_bin, found_left, found_all;
};

// Exclusive prefix sum over the CTA, and the sum.
template <int NT>
__device__ __forceinline__ uint32_t cta_prefix(uint32_t x, uint32_t* part, uint32_t* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  uint32_t s = x;
#pragma unroll
  for (int off = 1; off < 32; off <<= 1) {
    const uint32_t y = __shfl_up_sync(0xffffffffu, s, off);
    if (lane >= off) s += y;
  }
  __syncthreads();  // the words' last readers are done
  if (lane == 31) part[warp] = s;
  __syncthreads();
  uint32_t y = lane < NT / 32 ? part[lane] : 0u;
  const uint32_t before = __reduce_add_sync(0xffffffffu, lane < warp ? y : 0u);
  *total = __reduce_add_sync(0xffffffffu, y);
  return before + s - x;
}

// A sequence's tokens, from its pos.
struct Held {
  long long pos;
  int f;     // row of the oldest
  int m;     // kept
  int young, old, need;  // the youngest, kept; the others, and how many of them are
  bool bad;
};
__device__ __forceinline__ Held held_of(const EvictParams& p, int b) {
  Held h;
  h.pos = p.pos ? *static_cast<const volatile int64_t*>(p.pos + b) : p.T;
  const int n = h.pos < p.T ? static_cast<int>(h.pos < 0 ? 0 : h.pos) : p.T;
  h.f = h.pos <= p.T            ? 0
        : (h.pos >> 32) == 0 ? static_cast<int>(static_cast<unsigned>(h.pos) % static_cast<unsigned>(p.T))
                             : static_cast<int>(h.pos % p.T);
  h.bad = h.pos < 0 || (p.in_place && h.f != 0);
  h.m = h.bad ? 0 : min(n, p.keep);
  h.young = min(p.recent, h.m);
  h.old = n - h.young;
  h.need = h.m - h.young;
  return h;
}

// The rows that unit u keeps, into its part of idx.  bins: zero (after the caller's next barrier; this function begins
// with one).
template <int NT, bool CACHED>
__device__ __forceinline__ void choose(const EvictParams& p, long long u, const Held& h, ChooseSmem<NT>& sm,
                                       uint32_t* keys) {
  constexpr int kWarps = NT / 32;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  int32_t* idx = p.idx + u * p.keep;
  const float* weight = p.weight + u * p.T;
  const int old = h.old, need = h.need;
  auto row_of = [&](int age) {
    const int r = age + h.f;
    return r >= p.T ? r - p.T : r;
  };
  auto key_at = [&](int i) { return CACHED ? keys[i] : weight_key(weight[row_of(i)]); };
  // What needs no choice: the young ones, the places that stay empty, and all where all stay.
  for (int i = need + tid; i < p.keep; i += NT) idx[i] = i < h.m ? row_of(old + i - need) : -1;
  if (need == old)
    for (int i = tid; i < old; i += NT) idx[i] = row_of(i);
  if (need == 0 || need == old) return;

  // The threshold: of the `old` tokens those are kept whose key >> shift is above `prefix`, and the
  // first `ties` of those where it is equal.
  uint32_t prefix = 0, ties = static_cast<uint32_t>(need);
  int shift = 32;
  __syncthreads();
  // The weights once from memory, eight or 16 a thread on the way; the first pass's bins with them.
  constexpr int kLoads = NT == kChooseThreads ? 16 : 8;
#pragma unroll 1
  for (int i0 = tid; i0 < old; i0 += NT * kLoads) {
    float w[kLoads];
#pragma unroll
    for (int e = 0; e < kLoads; ++e) {
      const int i = i0 + e * NT;
      w[e] = i < old ? weight[row_of(i)] : 0.f;
    }
#pragma unroll
    for (int e = 0; e < kLoads; ++e) {
      const int i = i0 + e * NT;
      if (i < old) {
        const uint32_t key = weight_key(w[e]);
        if (CACHED) keys[i] = key;
        atomicAdd(&sm.bins[key >> 21], 1u);
      }
    }
  }
#pragma unroll 1
  for (int pass = 0; pass < 3; ++pass) {
    const int bits = pass == 2 ? 10 : 11, next = shift - bits;
    if (pass > 0) {
#pragma unroll 4
      for (int i = tid; i < old; i += NT) {
        const uint32_t key = key_at(i);
        if ((key >> shift) == prefix) atomicAdd(&sm.bins[(key >> next) & ((1u << bits) - 1)], 1u);
      }
    }
    __syncthreads();
    // thread t has the kPer bins down from 2047 - kPer t, and leaves them zero
    constexpr int kPer = kEvictBins / NT;
    static_assert(kPer == 8 || kPer == 2, "read in one piece or two");
    uint32_t c[kPer], sum = 0, all;
    uint32_t* mine = sm.bins + kEvictBins - kPer - tid * kPer;
    if (kPer == 8) {
      const uint4 lo = *reinterpret_cast<const uint4*>(mine), hi = *reinterpret_cast<const uint4*>(mine + 4);
      const uint32_t x[8] = {hi.w, hi.z, hi.y, hi.x, lo.w, lo.z, lo.y, lo.x};
#pragma unroll
      for (int e = 0; e < kPer; ++e) c[e] = x[e % 8];
      *reinterpret_cast<uint4*>(mine) = *reinterpret_cast<uint4*>(mine + 4) = make_uint4(0u, 0u, 0u, 0u);
    } else {
      const uint2 x = *reinterpret_cast<const uint2*>(mine);
      c[0] = x.y;
      c[1] = x.x;
      *reinterpret_cast<uint2*>(mine) = make_uint2(0u, 0u);
    }
#pragma unroll
    for (int e = 0; e < kPer; ++e) sum += c[e];
    uint32_t above = cta_prefix<NT>(sum, sm.part, &all);
    if (above < ties && ties <= above + sum) {
      int e = 0;
      uint32_t in_bin = c[0];
#pragma unroll
      for (int x = 0; x < kPer - 1; ++x)
        if (e == x && above + c[x] < ties) {
          above += c[x];
          in_bin = c[x + 1];
          ++e;
        }
      sm.found_bin = kEvictBins - 1 - tid * kPer - e;
      sm.found_left = ties - above;
      sm.found_all = in_bin;
    }
    __syncthreads();
    prefix = (pass == 0 ? 0u : prefix << bits) | sm.found_bin;
    ties = sm.found_left;
    shift = next;
    if (sm.found_all == ties) break;  // all of the bin stay
  }

  // The numbers, a segment of the ages at a time.  A word has the bits of 32 ages; a thread a word or two: it drops the
  // ties that are too many, and learns from a prefix sum how many are kept of the ages before; then a lane an age again.
  const uint32_t below = (1u << lane) - 1;
  uint32_t kept = 0;  // of the segments before, and the ties that are left
#pragma unroll 1
  for (int a0 = 0; a0 < old; a0 += kSegment) {
    const int words = (min(old - a0, kSegment) + 31) / 32;
#pragma unroll 4
    for (int g = warp; g < words; g += kWarps) {
      const int i = a0 + 32 * g + lane;
      const uint32_t x = i < old ? key_at(i) >> shift : 0u;
      const uint32_t m_gt = __ballot_sync(0xffffffffu, i < old && x > prefix);
      const uint32_t m_eq = __ballot_sync(0xffffffffu, i < old && x == prefix);
      if (lane == 0) {
        sm.gt[g] = m_gt;
        sm.eq[g] = m_eq;
      }
    }
    __syncthreads();
    constexpr int kEach = (kWords + NT - 1) / NT;  // neighbouring words of a thread
    uint32_t count = 0, all;
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      const int g = tid * kEach + e;
      if (g < words) count += __popc(sm.gt[g]) | __popc(sm.eq[g]) << 16;
    }
    const uint32_t before = cta_prefix<NT>(count, sm.part, &all);
    uint32_t gt = before & 0xFFFFu, eq = before >> 16;
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      const int g = tid * kEach + e;
      if (g >= words) break;
      const uint32_t w_gt = sm.gt[g];
      uint32_t w_eq = sm.eq[g];
      const uint32_t n_eq = __popc(w_eq), room = ties > eq ? ties - eq : 0u;
      sm.eq[g] = kept + gt + min(eq, ties);
      for (uint32_t x = n_eq; x > room; --x) w_eq &= ~(0x80000000u >> __clz(w_eq));  // the youngest go
      sm.gt[g] = w_gt | w_eq;
      gt += __popc(w_gt);
      eq += n_eq;
    }
    __syncthreads();
#pragma unroll 4
    for (int g = warp; g < words; g += kWarps) {
      const uint32_t stay = sm.gt[g];
      if ((stay >> lane) & 1u) idx[sm.eq[g] + __popc(stay & below)] = row_of(a0 + 32 * g + lane);
    }
    kept += (all & 0xFFFFu) + min(all >> 16, ties);
    ties -= min(all >> 16, ties);
    __syncthreads();  // the words are read
  }
}

// One thread of each of a sequence's CTAs counts itself when all threads of the CTA have read pos (and used it), and in the end, the
// answer having taken a trip to L2, the last of them writes what depends on it.
__device__ __forceinline__ unsigned long long held_read(const EvictParams& p, int b) {
  return atomicAdd(p.tickets + b, 1ull);
}
__device__ __forceinline__ void held_done(const EvictParams& p, int b, const Held& h, unsigned long long ticket) {
  if (ticket + 1 != static_cast<unsigned long long>(p.LH)) return;
  if (h.bad) atomicOr(p.status, CMC_DEVFLAG_BAD_POS);
  if (p.out_pos) p.out_pos[b] = h.bad ? h.pos : h.m;
  if (p.evicted && !h.bad) p.evicted[b] += h.pos - h.m;
  p.tickets[b] = 0ull;
}

// Copies the rows of unit u that CTA `rank` of p.cm has, m in all.  A thread has chunk tid % CPR of four rows of K and of V, and, in the first kBlock
// threads, a row's weight; the next block's rows are requested before this one's are stored, their indices a block
// earlier.
template <int D>
__device__ __forceinline__ void copy_rows(const EvictParams& p, long long u, int rank, int m) {
  constexpr int CPR = D / 8;                          // 16-byte chunks per row
  constexpr int kRowsPerPass = kEvictThreads / CPR;
  constexpr int kBlock = kRowsPerPass * kEvictBatch;  // rows of a block
  const int tid = threadIdx.x;
  const int32_t* idx = p.idx + u * p.keep;
  const float* weight = p.weight + u * p.T;
  const int chunk = tid % CPR, sub = tid / CPR;
  const uint4* gk = reinterpret_cast<const uint4*>(p.k) + u * p.T * CPR + chunk;
  const uint4* gv = reinterpret_cast<const uint4*>(p.v) + u * p.T * CPR + chunk;
  uint4* ok = reinterpret_cast<uint4*>(p.out_k) + u * p.R * CPR + chunk;
  uint4* ov = reinterpret_cast<uint4*>(p.out_v) + u * p.R * CPR + chunk;
  float* ow = p.out_weight + u * p.R;
  const int hop = kBlock * p.cm;  // from a CTA's block to its next
  const int rounds = (m + hop - 1) / hop;
  struct Rows {
    uint4 k[kEvictBatch], v[kEvictBatch];
    float w;
    bool has[kEvictBatch + 1];
  };
  int src[kEvictBatch + 1];  // rows of the block to request next (-1: none), and that of this thread's weight
  auto rows_of = [&](int i0) {
#pragma unroll
    for (int e = 0; e < kEvictBatch; ++e) {
      const int i = i0 + e * kRowsPerPass + sub;
      src[e] = i < m ? idx[i] : -1;
    }
    src[kEvictBatch] = tid < kBlock && i0 + tid < m ? idx[i0 + tid] : -1;
  };
  auto request = [&](Rows& x) {
#pragma unroll
    for (int e = 0; e < kEvictBatch; ++e) {
      x.has[e] = src[e] >= 0;
      if (x.has[e]) {
        x.k[e] = gk[static_cast<long long>(src[e]) * CPR];
        x.v[e] = gv[static_cast<long long>(src[e]) * CPR];
      }
    }
    x.has[kEvictBatch] = src[kEvictBatch] >= 0;
    if (x.has[kEvictBatch]) x.w = weight[src[kEvictBatch]];
  };
  auto store = [&](const Rows& x, int i0) {
#pragma unroll
    for (int e = 0; e < kEvictBatch; ++e)
      if (x.has[e]) {
        const long long to = static_cast<long long>(i0 + e * kRowsPerPass + sub) * CPR;
        ok[to] = x.k[e];
        ov[to] = x.v[e];
      }
    if (x.has[kEvictBatch]) ow[i0 + tid] = x.w;
  };
  // In place a block is stored when all of the unit's CTAs (a cluster) have read theirs of the same round.
  auto all_read = [&]() {
    if (!p.in_place) return;
    if (p.cm > 1) cluster_sync_all();
    else __syncthreads();
  };
  Rows x, y;
  int i0 = rank * kBlock;
  rows_of(i0);
  request(x);
  rows_of(i0 + hop);
  for (int r = 0; r < rounds; r += 2) {
    request(y);
    rows_of(i0 + 2 * hop);
    all_read();
    store(x, i0);
    if (r + 1 == rounds) break;
    request(x);
    rows_of(i0 + 3 * hop);
    all_read();
    store(y, i0 + hop);
    i0 += 2 * hop;
  }
}

// The rows that stay whatever the weights are, the youngest, into L2 while the others are chosen: one of four threads takes K or
// V, and the rows before the ring's end or those behind it.
template <int D>
__device__ __forceinline__ void prefetch_young(const EvictParams& p, long long u, const Held& h, int part) {
  const int rows = min(h.young, kEvictAhead / (2 * D));
  const int r0 = h.old + h.f >= p.T ? h.old + h.f - p.T : h.old + h.f;
  const int to_end = min(rows, p.T - r0);
  const int n = part & 2 ? rows - to_end : to_end;
  const uint16_t* base = (part & 1 ? p.v : p.k) + (u * p.T + (part & 2 ? 0 : r0)) * D;
  if (n > 0) asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;\n" ::"l"(base), "r"(n * D * 2) : "memory");
}

// A unit's weights, into L2: a hint, which may come before the wait (256 units of 512 tokens 15.0 us without, 14.4 with; where a
// kernel of its own chooses it changes nothing).
__device__ __forceinline__ void prefetch_weights(const EvictParams& p, long long u) {
  const uintptr_t at = reinterpret_cast<uintptr_t>(p.weight + u * p.T);
  const uintptr_t from = (at + 15) & ~static_cast<uintptr_t>(15), to = (at + min(4ll * p.T, static_cast<long long>(kEvictAhead))) & ~static_cast<uintptr_t>(15);
  if (to > from) asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;\n" ::"l"(from), "r"(static_cast<uint32_t>(to - from)) : "memory");
}

// A unit's choice and copy.
template <int D, bool CACHED>
__global__ void __launch_bounds__(kEvictThreads, 2)
evict_kernel(const __grid_constant__ EvictParams p) {
  extern __shared__ __align__(16) uint32_t keys_s[];
  __shared__ ChooseSmem<kEvictThreads> sm;
  const long long u = blockIdx.x;
  const int b = static_cast<int>(static_cast<unsigned>(u) / static_cast<unsigned>(p.LH));
  if (threadIdx.x == 0) prefetch_weights(p, u);
  for (int i = threadIdx.x; i < kEvictBins; i += kEvictThreads) sm.bins[i] = 0u;
  pdl_wait();
  pdl_trigger();
  const Held h = held_of(p, b);
  if (threadIdx.x >= kEvictThreads - 4 && h.need != 0 && h.need != h.old) prefetch_young<D>(p, u, h, threadIdx.x & 3);
  choose<kEvictThreads, CACHED>(p, u, h, sm, keys_s);
  __syncthreads();  // the rows are known
  unsigned long long ticket = 0;
  if (threadIdx.x == 0) ticket = held_read(p, b);
  copy_rows<D>(p, u, 0, h.m);
  if (threadIdx.x == 0) held_done(p, b, h, ticket);
}

template <bool CACHED>
__global__ void __launch_bounds__(kChooseThreads)
evict_choose_kernel(const __grid_constant__ EvictParams p) {
  extern __shared__ __align__(16) uint32_t keys_s[];
  __shared__ ChooseSmem<kChooseThreads> sm;
  const long long u = blockIdx.x;
  const int b = static_cast<int>(static_cast<unsigned>(u) / static_cast<unsigned>(p.LH));
  for (int i = threadIdx.x; i < kEvictBins; i += kChooseThreads) sm.bins[i] = 0u;
  pdl_wait();
  pdl_trigger();
  const Held h = held_of(p, b);
  choose<kChooseThreads, CACHED>(p, u, h, sm, keys_s);
  __syncthreads();
  if (threadIdx.x == 0) held_done(p, b, h, held_read(p, b));
}

// The copy after evict_choose_kernel, which has written pos already: rows that stay empty are known by their -1.
template <int D>
__global__ void __launch_bounds__(kEvictThreads, 2)
evict_copy_kernel(const __grid_constant__ EvictParams p) {
  const unsigned u = blockIdx.x / static_cast<unsigned>(p.cm);
  pdl_wait();
  pdl_trigger();
  copy_rows<D>(p, u, static_cast<int>(blockIdx.x - u * p.cm), p.keep);
}

// ---------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------

// Launches with programmatic stream serialization and, with cluster > 1, a cluster dimension.
template <typename K>
static int launch_evict_kernel(K kern, long long grid, int threads, size_t smem, int cluster, cudaStream_t s,
                               const EvictParams& p) {
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = static_cast<unsigned>(cluster);
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(grid));
  cfg.blockDim = dim3(static_cast<unsigned>(threads));
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cfg.attrs = attr;
  cfg.numAttrs = cluster > 1 ? 2 : 1;
  return record_cuda_error(cudaLaunchKernelEx(&cfg, kern, p));
}

template <int D>
static int launch_evict(const EvictParams& p0, long long units, cudaStream_t s) {
  EvictParams p = p0;
  constexpr int kBlock = kEvictThreads / (D / 8) * kEvictBatch;
  static std::atomic<int> configured[64];
  int dev = 0;
  int st = record_cuda_error(cudaGetDevice(&dev));
  if (st != CMC_OK) return st;
  if (dev < 0 || dev >= 64 || !configured[dev].load(std::memory_order_acquire)) {
    const auto most = cudaFuncAttributeMaxDynamicSharedMemorySize;
    st = record_cuda_error(cudaFuncSetAttribute(evict_kernel<D, true>, most, kEvictKeys * 4));
    if (st == CMC_OK) st = record_cuda_error(cudaFuncSetAttribute(evict_choose_kernel<true>, most, kEvictKeys * 4));
    // The same part of an SM's memory for the choice and the copy: an SM has to be empty to change it (64 units of 16,384
    // tokens, 2,048 kept, 35.9 us, 41.2 where they differ, 47.7 with all of it, which leaves too little L1 for loads on their way).
    const auto carve = cudaFuncAttributePreferredSharedMemoryCarveout;
    if (st == CMC_OK) st = record_cuda_error(cudaFuncSetAttribute(evict_copy_kernel<D>, carve, 50));
    if (st == CMC_OK) st = record_cuda_error(cudaFuncSetAttribute(evict_choose_kernel<true>, carve, 50));
    if (st != CMC_OK) return st;
    if (dev >= 0 && dev < 64) configured[dev].store(1, std::memory_order_release);
  }
  // CTAs that copy a unit: as many as it takes to have about three on each SM, at most one a block, in place no
  // more than a cluster has.  One, which then chooses as well, where there are units enough or the rows that are kept are one block:
  // what it costs goes by the length of the unit too, which the rule does not look at.  (us with one kernel, 64 rows of d = 128 kept /
  // with two, 65 kept: 1, 8 and 64 units of 4,096 tokens 7.0 / 8.1, 7.5 / 8.6, 7.6 / 10.7, of 16,384 16.8 / 10.9, 17.4 / 11.2,
  // 17.8 / 11.6.)  In place against apart: 256 units of 512 tokens, 256 kept, 14.3 / 13.6, 64 of 2,048, 1,024 kept, 30.2 / 23.1, 64 of
  // 16,384, 2,048 kept, 43.0 / 35.2: a barrier over the unit's CTAs a round.
  const long long blocks = (p.keep + kBlock - 1) / kBlock;
  long long cm = std::max(1LL, std::min<long long>(blocks, 3 * sm_count() / units));
  if (p.in_place && cm > kMaxClusterCtas) cm = kMaxClusterCtas;
  p.cm = static_cast<int>(cm);
  const bool cached = p.T <= kEvictKeys;
  const size_t smem = cached ? static_cast<size_t>(p.T) * 4 : 0;
  if (cm == 1)
    return launch_evict_kernel(cached ? evict_kernel<D, true> : evict_kernel<D, false>, units, kEvictThreads, smem, 1, s, p);
  st = launch_evict_kernel(cached ? evict_choose_kernel<true> : evict_choose_kernel<false>, units, kChooseThreads, smem, 1, s, p);
  if (st != CMC_OK) return st;
  return launch_evict_kernel(evict_copy_kernel<D>, units * cm, kEvictThreads, 0, p.in_place ? p.cm : 1, s, p);
}

}  // namespace cmc

extern "C" {

int cmc_evict_cache(const void* k, const void* v, const float* weight, const int64_t* pos,
                    const cmc_dims* dims, int recent, void* out_k, void* out_v, float* out_weight,
                    int32_t* idx_out, int64_t* out_pos, int64_t* evicted, void* workspace,
                    size_t workspace_bytes, void* stream) {
  using namespace cmc;
  if (!dims) return CMC_ERR_NULL;
  cmc_dims m = *dims;
  m.Hq = m.Hkv;  // query heads play no part here
  int st = validate_dims(&m, true);
  if (st != CMC_OK) return st;
  if (m.k < 1 || m.W < m.k || recent < 0 || recent > m.k) return CMC_ERR_RANGE;
  if (!k || !v || !weight || !out_k || !out_v || !out_weight || !idx_out) return CMC_ERR_NULL;
  if (!aligned16(k) || !aligned16(v) || !aligned16(out_k) || !aligned16(out_v) ||
      ((reinterpret_cast<uintptr_t>(weight) | reinterpret_cast<uintptr_t>(out_weight) |
        reinterpret_cast<uintptr_t>(idx_out)) & 3) ||
      ((reinterpret_cast<uintptr_t>(pos) | reinterpret_cast<uintptr_t>(out_pos) |
        reinterpret_cast<uintptr_t>(evicted)) & 7))
    return CMC_ERR_ALIGN;
  if (!workspace || workspace_bytes < ws_partials_off(m.B)) return CMC_ERR_WORKSPACE;
  if (!aligned16(workspace)) return CMC_ERR_ALIGN;
  const long long units = static_cast<long long>(m.B) * m.L * m.Hkv;
  EvictParams p;
  p.in_place = k == out_k || v == out_v || weight == out_weight;
  if (p.in_place && !(k == out_k && v == out_v && weight == out_weight && m.W == m.N)) return CMC_ERR_RANGE;
  // Rows are read while others are written, and idx is read back as the rows to copy: what is written meets nothing else, but
  // for the cache in place and out_pos in pos.
  const size_t in = static_cast<size_t>(units) * m.N, out = static_cast<size_t>(units) * m.W, row = m.d * 2, each = static_cast<size_t>(m.B) * 8;
  const Range reads[] = {{k, in * row}, {v, in * row}, {weight, in * 4}, {pos, each}};
  const Range writes[] = {{out_k, out * row}, {out_v, out * row}, {out_weight, out * 4}, {idx_out, static_cast<size_t>(units) * m.k * 4},
                          {out_pos, each}, {evicted, each}, {workspace, ws_partials_off(m.B)}};
  for (int o = 0; o < 7; ++o) {
    for (int i = 0; i < 4; ++i) {
      const bool there = same(writes[o], reads[i]) && ((p.in_place && o < 3 && i < 3) || (o == 4 && i == 3));
      if (!there && meet(writes[o], reads[i])) return CMC_ERR_RANGE;
    }
    for (int i = 0; i < o; ++i)  // (a cache whose K is its V too is moved as one in place)
      if (meet(writes[o], writes[i]) && !(p.in_place && o == 1 && i == 0 && same(writes[0], writes[1]))) return CMC_ERR_RANGE;
  }
  p.k = static_cast<const uint16_t*>(k);
  p.v = static_cast<const uint16_t*>(v);
  p.weight = weight;
  p.pos = pos;
  p.out_k = static_cast<uint16_t*>(out_k);
  p.out_v = static_cast<uint16_t*>(out_v);
  p.out_weight = out_weight;
  p.idx = idx_out;
  p.out_pos = out_pos;
  p.evicted = evicted;
  char* ws = static_cast<char*>(workspace);
  p.status = reinterpret_cast<uint32_t*>(ws);
  p.tickets = reinterpret_cast<unsigned long long*>(ws + kWsHeader);
  p.T = m.N; p.R = m.W; p.keep = m.k; p.recent = recent; p.LH = m.L * m.Hkv;
  p.cm = 1;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  return m.d == 128 ? launch_evict<128>(p, units, s) : launch_evict<64>(p, units, s);
}

}  // extern "C"
