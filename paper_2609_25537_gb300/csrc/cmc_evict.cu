// Eviction from a cache by accumulated attention weight (cmc_evict_cache): per (sequence, layer, KV
// head) unit the heaviest and the youngest tokens are kept and moved together, in order of age.
//
// A unit is taken by a CTA or a cluster of up to eight.  Each CTA of the cluster finds the unit's
// threshold by itself (a radix select over the weights' order-preserving 32-bit keys, which cost a
// hundredth of the rows' bytes), numbers the tokens that stay, and copies its blocks of rows: block i of the
// output is CTA i mod cm's.  The i-th token kept is never older than the i-th of all, so in place
// (output and input the same tensors, not wrapped) a row is written only where rows of the same or of earlier blocks
// were read, and a barrier over the cluster between a block's loads and its stores is all that it takes.
#include <algorithm>
#include <atomic>

#include "cmc_attn.cuh"

namespace cmc {

constexpr int kEvictThreads = 256;
constexpr int kEvictWarps = kEvictThreads / 32;
constexpr int kEvictBatch = 4;      // rows of K and of V that a thread has in flight
constexpr int kEvictBins = 2048;    // 11 bits a pass
constexpr int kEvictKeys = 16384;   // keys held in shared memory; of longer units they are read again

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
  int T, R, keep, recent, LH, cm, in_place, cached;
};

// Larger weight, larger key; -0 is 0 and a NaN is below everything.
__device__ __forceinline__ uint32_t weight_key(float w) {
  if (w != w) return 0u;
  return orderable(w + 0.f);
}

// Exclusive prefix sum over the CTA, and the total; `part` holds kEvictWarps words.
__device__ __forceinline__ uint32_t block_prefix(uint32_t x, uint32_t* part, uint32_t* total) {
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
  uint32_t before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < kEvictWarps; ++w) {
    if (w < warp) before += part[w];
    all += part[w];
  }
  *total = all;
  return before + s - x;
}

template <int D>
__global__ void __launch_bounds__(kEvictThreads)
evict_kernel(const EvictParams p) {
  constexpr int CPR = D / 8;                          // 16-byte chunks per row
  constexpr int kRowsPerPass = kEvictThreads / CPR;
  constexpr int kBlock = kRowsPerPass * kEvictBatch;  // rows of a block
  extern __shared__ __align__(16) uint32_t keys_s[];
  __shared__ uint32_t hist[kEvictBins];
  __shared__ uint32_t part[kEvictWarps];
  __shared__ uint32_t found_bin, found_left, found_all;
  __shared__ long long pos_s;
  const int tid = threadIdx.x;
  const long long u = blockIdx.x / static_cast<unsigned>(p.cm);
  const int rank = static_cast<int>(blockIdx.x - u * p.cm);
  const int b = static_cast<int>(u / p.LH);
  pdl_wait();
  pdl_trigger();
  if (tid == 0) pos_s = p.pos ? *static_cast<const volatile int64_t*>(p.pos + b) : p.T;
  __syncthreads();
  const long long pos = pos_s;
  const int n = pos < p.T ? static_cast<int>(pos < 0 ? 0 : pos) : p.T;  // tokens held
  const int f = pos > p.T ? static_cast<int>(pos % p.T) : 0;            // row of the oldest
  const bool bad = pos < 0 || (p.in_place && f != 0);
  const int m = bad ? 0 : min(n, p.keep);
  if (tid == 0) {
    // the last of the sequence's CTAs to have read pos writes what depends on it
    __threadfence();
    if (atomicAdd(p.tickets + b, 1ull) + 1 == static_cast<unsigned long long>(p.LH) * p.cm) {
      if (bad) atomicOr(p.status, CMC_DEVFLAG_BAD_POS);
      if (p.out_pos) p.out_pos[b] = bad ? pos : m;
      if (p.evicted && !bad) p.evicted[b] += pos - m;
      p.tickets[b] = 0ull;
    }
  }
  int32_t* idx = p.idx + u * p.keep;
  if (rank == 0)
    for (int i = m + tid; i < p.keep; i += kEvictThreads) idx[i] = -1;
  if (bad) return;  // the whole cluster's CTAs
  const int young = min(p.recent, m), old = n - young, need = m - young;
  const float* weight = p.weight + u * p.T;
  auto row_of = [&](int age) {
    const int r = age + f;
    return r >= p.T ? r - p.T : r;
  };
  auto key_of = [&](int age) { return p.cached ? keys_s[age] : weight_key(weight[row_of(age)]); };

  // The threshold: of the `old` tokens those are kept whose key >> shift is above `prefix`, and the
  // first `ties` of those where it is equal.
  uint32_t prefix = 0, ties = static_cast<uint32_t>(need);
  int shift = 32;
  if (need > 0 && need < old) {
    if (p.cached)
      for (int i = tid; i < old; i += kEvictThreads) keys_s[i] = weight_key(weight[row_of(i)]);
    while (shift > 0) {
      const int bits = shift == 32 ? 11 : shift == 21 ? 11 : 10;
      const int next = shift - bits;
      for (int i = tid; i < kEvictBins; i += kEvictThreads) hist[i] = 0;
      __syncthreads();
      for (int i = tid; i < old; i += kEvictThreads) {
        const uint32_t key = key_of(i);
        if (shift == 32 || (key >> shift) == prefix) atomicAdd(&hist[(key >> next) & ((1u << bits) - 1)], 1u);
      }
      __syncthreads();
      // thread t has the eight bins down from 2047 - 8 t
      constexpr int kPer = kEvictBins / kEvictThreads;
      uint32_t c[kPer], sum = 0, all;
#pragma unroll
      for (int e = 0; e < kPer; ++e) sum += c[e] = hist[kEvictBins - 1 - tid * kPer - e];
      uint32_t above = block_prefix(sum, part, &all);
      if (above < ties && ties <= above + sum) {
        int e = 0;
#pragma unroll
        for (int x = 0; x < kPer - 1; ++x)
          if (e == x && above + c[x] < ties) {
            above += c[x];
            ++e;
          }
        found_bin = kEvictBins - 1 - tid * kPer - e;
        found_left = ties - above;
        found_all = hist[kEvictBins - 1 - tid * kPer - e];
      }
      __syncthreads();
      prefix = shift == 32 ? found_bin : (prefix << bits) | found_bin;
      ties = found_left;
      shift = next;
      if (found_all == ties) break;  // all of the bin stay
    }
  }

  // Number the tokens that stay; each CTA writes the rows of its own blocks.
  auto put = [&](int i, int age) {
    if ((i / kBlock) % p.cm == rank) idx[i] = row_of(age);
  };
  if (need > 0) {
    constexpr int kItems = 4;
    uint32_t gt0 = 0, eq0 = 0;
    for (int base = 0; base < old; base += kEvictThreads * kItems) {
      uint32_t above = 0, equal = 0;  // bits of the thread's items
      if (need == old) {
        above = (1u << kItems) - 1;
      } else {
#pragma unroll
        for (int e = 0; e < kItems; ++e) {
          const int i = base + tid * kItems + e;
          if (i < old) {
            const uint32_t key = key_of(i) >> shift;
            above |= (key > prefix ? 1u : 0u) << e;
            equal |= (key == prefix ? 1u : 0u) << e;
          }
        }
      }
      if (need == old) {
#pragma unroll
        for (int e = 0; e < kItems; ++e) {
          const int i = base + tid * kItems + e;
          if (i < old) put(i, i);
        }
        continue;
      }
      uint32_t all;
      const uint32_t pre = block_prefix(__popc(above) | (__popc(equal) << 16), part, &all);
      uint32_t gt = gt0 + (pre & 0xFFFFu), eq = eq0 + (pre >> 16);
#pragma unroll
      for (int e = 0; e < kItems; ++e) {
        if ((above >> e) & 1u) {
          put(static_cast<int>(gt + min(eq, ties)), base + tid * kItems + e);
          ++gt;
        } else if ((equal >> e) & 1u) {
          if (eq < ties) put(static_cast<int>(gt + eq), base + tid * kItems + e);
          ++eq;
        }
      }
      gt0 += all & 0xFFFFu;
      eq0 += all >> 16;
    }
  }
  for (int i = need + tid; i < m; i += kEvictThreads) put(i, old + i - need);
  __syncthreads();

  // Copy.  A thread has chunk tid % CPR of four rows of K and of V in flight.
  const int chunk = tid % CPR, sub = tid / CPR;
  const uint4* gk = reinterpret_cast<const uint4*>(p.k) + u * p.T * CPR + chunk;
  const uint4* gv = reinterpret_cast<const uint4*>(p.v) + u * p.T * CPR + chunk;
  uint4* ok = reinterpret_cast<uint4*>(p.out_k) + u * p.R * CPR + chunk;
  uint4* ov = reinterpret_cast<uint4*>(p.out_v) + u * p.R * CPR + chunk;
  float* ow = p.out_weight + u * p.R;
  const int rounds = (m + kBlock * p.cm - 1) / (kBlock * p.cm);
  for (int r = 0; r < rounds; ++r) {
    const int i0 = (r * p.cm + rank) * kBlock;
    uint4 kr[kEvictBatch], vr[kEvictBatch];
    float wr = 0.f;
    int src[kEvictBatch];
#pragma unroll
    for (int e = 0; e < kEvictBatch; ++e) {
      const int i = i0 + e * kRowsPerPass + sub;
      src[e] = i < m ? idx[i] : -1;
    }
    const bool mine = tid < kBlock && i0 + tid < m;
    if (mine) wr = weight[idx[i0 + tid]];
#pragma unroll
    for (int e = 0; e < kEvictBatch; ++e)
      if (src[e] >= 0) {
        kr[e] = gk[static_cast<long long>(src[e]) * CPR];
        vr[e] = gv[static_cast<long long>(src[e]) * CPR];
      }
    if (p.in_place) {
      if (p.cm > 1) cluster_sync_all();
      else __syncthreads();
    }
#pragma unroll
    for (int e = 0; e < kEvictBatch; ++e)
      if (src[e] >= 0) {
        const long long to = static_cast<long long>(i0 + e * kRowsPerPass + sub) * CPR;
        ok[to] = kr[e];
        ov[to] = vr[e];
      }
    if (mine) ow[i0 + tid] = wr;
  }
}

// ---------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------

template <int D>
static int launch_evict(const EvictParams& p0, long long units, cudaStream_t s) {
  EvictParams p = p0;
  constexpr int kBlock = kEvictThreads / (D / 8) * kEvictBatch;
  static std::atomic<int> configured[64];
  int dev = 0;
  int st = record_cuda_error(cudaGetDevice(&dev));
  if (st != CMC_OK) return st;
  if (dev < 0 || dev >= 64 || !configured[dev].load(std::memory_order_acquire)) {
    st = record_cuda_error(cudaFuncSetAttribute(evict_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                                kEvictKeys * 4));
    if (st != CMC_OK) return st;
    if (dev >= 0 && dev < 64) configured[dev].store(1, std::memory_order_release);
  }
  // CTAs of a unit: as many as it takes to have about three on each SM, at most one a block.
  int cm = 1;
  while (cm < kMaxClusterCtas && 2 * cm * kBlock < p.keep + kBlock && 2 * cm * units <= 3LL * sm_count()) cm *= 2;
  p.cm = cm;
  p.cached = p.T <= kEvictKeys;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = static_cast<unsigned>(cm);
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(units * cm));
  cfg.blockDim = dim3(kEvictThreads);
  cfg.dynamicSmemBytes = p.cached ? static_cast<size_t>(p.T) * 4 : 0;
  cfg.stream = s;
  cfg.attrs = attr;
  cfg.numAttrs = cm > 1 ? 2 : 1;
  return record_cuda_error(cudaLaunchKernelEx(&cfg, evict_kernel<D>, p));
}

static bool overlap(const void* a, size_t na, const void* b, size_t nb) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return x < y + nb && y < x + na;
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
  const size_t in = static_cast<size_t>(units) * m.N, out = static_cast<size_t>(units) * m.W;
  if (!p.in_place && (overlap(k, in * m.d * 2, out_k, out * m.d * 2) || overlap(k, in * m.d * 2, out_v, out * m.d * 2) ||
                      overlap(v, in * m.d * 2, out_k, out * m.d * 2) || overlap(v, in * m.d * 2, out_v, out * m.d * 2) ||
                      overlap(weight, in * 4, out_weight, out * 4)))
    return CMC_ERR_RANGE;
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
  p.cached = 0;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  return m.d == 128 ? launch_evict<128>(p, units, s) : launch_evict<64>(p, units, s);
}

}  // extern "C"
