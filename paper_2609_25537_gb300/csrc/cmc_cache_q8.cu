// Writing and reading the 8-bit two-tier cache (format: cmc_q8.cuh): rows of a
// bf16 bank quantised into a cache, a cache read back, one token appended to an
// 8-bit ring.
#include <cuda_runtime.h>
#include <stdint.h>

#include "cmc_q8.cuh"

namespace cmc {

constexpr int kRowThreads = 128;  // four warps, each with blocks of rows of its own
constexpr int kRowWarps = kRowThreads / 32;

// One warp quantises a block of 32 rows of one unit's K or V at a time: it holds
// the whole block in registers (8 KB at d = 128, 16 loads of 16 bytes a lane, all
// in flight together), so that the bf16 rows are read once for their maximum
// and their codes.
template <int D>
__global__ void __launch_bounds__(kRowThreads)
quantize_kernel(const uint4* __restrict__ bank_k, const uint4* __restrict__ bank_v,
                const int32_t* __restrict__ idx, const int64_t* __restrict__ count,
                uint8_t* __restrict__ kv, uint8_t* __restrict__ scales, uint32_t* status,
                long long jobs, int nb, int LH, int N, int k, int S) {
  constexpr int CPR = D / 8;           // 16-byte chunks of a bf16 row
  constexpr int RPP = 32 / CPR;        // rows of a pass of the warp
  constexpr int NP = kQ8Block / RPP;   // passes
  pdl_wait();
  pdl_trigger();
  const int lane = threadIdx.x & 31;
  const int chunk = lane % CPR, rsub = lane / CPR;
  for (long long job = static_cast<long long>(blockIdx.x) * kRowWarps + (threadIdx.x >> 5); job < jobs;
       job += static_cast<long long>(gridDim.x) * kRowWarps) {
    const long long uw = job / nb;  // (unit, K or V)
    const int j = static_cast<int>(job - uw * nb);
    const long long u = uw >> 1;
    const long long b = u / LH;
    const int r0 = j * kQ8Block;
    // lane r: the bank row behind row r of the block, -1 if it holds no token
    int src = -1;
    {
      const int i = r0 + lane;
      const long long n = count ? count[b] : k;
      if (i < k && i < n) {
        src = idx ? idx[b * k + i] : i;
        if (static_cast<unsigned>(src) >= static_cast<unsigned>(N)) {
          src = -1;
          if (status) atomicOr(status, CMC_DEVFLAG_BAD_INDEX);
        }
      }
    }
    const uint4* bank = ((uw & 1) ? bank_v : bank_k) + u * N * CPR + chunk;
    uint4 x[NP];
    uint32_t m = 0u;  // largest magnitude, bf16 bits in two halves
#pragma unroll
    for (int e = 0; e < NP; ++e) {
      const int row = __shfl_sync(0xffffffffu, src, e * RPP + rsub);
      x[e] = make_uint4(0u, 0u, 0u, 0u);
      if (row >= 0) x[e] = ld_stream_u4(bank + static_cast<long long>(row) * CPR);
    }
#pragma unroll
    for (int e = 0; e < NP; ++e) {
      m = __vmaxu2(m, x[e].x & 0x7FFF7FFFu);
      m = __vmaxu2(m, x[e].y & 0x7FFF7FFFu);
      m = __vmaxu2(m, x[e].z & 0x7FFF7FFFu);
      m = __vmaxu2(m, x[e].w & 0x7FFF7FFFu);
    }
    uint32_t top = __reduce_max_sync(0xffffffffu, max(m & 0xFFFFu, m >> 16));
    if (top >= 0x7F80u) {  // an infinity or NaN among them: the largest finite one
      top = 0u;
#pragma unroll
      for (int e = 0; e < NP; ++e) {
        float f[8];
        unpack8(x[e], f);
#pragma unroll
        for (int q = 0; q < 8; ++q) top = max(top, finite_bits(f[q]) >> 16);
      }
      top = __reduce_max_sync(0xffffffffu, top);
    }
    const int c = block_code(top << 16);
    const float f = code_factor(c);
    uint8_t* dst = kv + (uw * k + r0) * D + chunk * 8;
#pragma unroll
    for (int e = 0; e < NP; ++e) {
      const int row = e * RPP + rsub;
      if (r0 + row < k) {
        float v[8];
        unpack8(x[e], v);
        *reinterpret_cast<uint2*>(dst + static_cast<long long>(row) * D) =
            make_uint2(encode4(v[0], v[1], v[2], v[3], f), encode4(v[4], v[5], v[6], v[7], f));
      }
    }
    uint8_t* sc = scales + uw * S;
    if (lane == 0) sc[j] = static_cast<uint8_t>(c);
    if (j == nb - 1 && nb + lane < S) sc[nb + lane] = 0;  // the padding, at most three bytes
  }
}

// A warp reads back 32 rows of one unit's K or V at a time.
template <int D>
__global__ void __launch_bounds__(kRowThreads)
dequantize_kernel(const uint8_t* __restrict__ kv, const uint8_t* __restrict__ scales,
                  const int32_t* __restrict__ idx, uint4* __restrict__ out_k,
                  uint4* __restrict__ out_v, uint32_t* status, long long jobs, int nb, int LH, int N,
                  int k, int S) {
  constexpr int CPR = D / 8;  // 8-code chunks of a row (16 bytes of the output)
  constexpr int RPP = 32 / CPR;
  constexpr int NP = kQ8Block / RPP;
  pdl_wait();
  pdl_trigger();
  const int lane = threadIdx.x & 31;
  const int chunk = lane % CPR, rsub = lane / CPR;
  for (long long job = static_cast<long long>(blockIdx.x) * kRowWarps + (threadIdx.x >> 5); job < jobs;
       job += static_cast<long long>(gridDim.x) * kRowWarps) {
    const long long uw = job / nb;
    const int r0 = static_cast<int>(job - uw * nb) * kQ8Block;
    const long long u = uw >> 1;
    int src = -1;
    float scale = 0.f;
    if (r0 + lane < k) {
      src = idx ? idx[u / LH * k + r0 + lane] : r0 + lane;
      if (static_cast<unsigned>(src) >= static_cast<unsigned>(N)) {
        src = -1;
        if (status) atomicOr(status, CMC_DEVFLAG_BAD_INDEX);
      } else {
        scale = e8m0_to_f32(scales[uw * S + src / kQ8Block]);
      }
    }
    const uint8_t* from = kv + uw * N * D + chunk * 8;
    uint4* to = ((uw & 1) ? out_v : out_k) + (u * k + r0) * CPR + chunk;
    uint2 x[NP];
#pragma unroll
    for (int e = 0; e < NP; ++e) {
      const int row = __shfl_sync(0xffffffffu, src, e * RPP + rsub);
      x[e] = make_uint2(0u, 0u);
      if (row >= 0) x[e] = *reinterpret_cast<const uint2*>(from + static_cast<long long>(row) * D);
    }
#pragma unroll
    for (int e = 0; e < NP; ++e) {
      const float s = __shfl_sync(0xffffffffu, scale, e * RPP + rsub);
      float a[4], c[4];
      decode4(x[e].x, a);
      decode4(x[e].y, c);
      if (r0 + e * RPP + rsub < k)
        to[static_cast<long long>(e * RPP + rsub) * CPR] =
            make_uint4(pack_bf16_rn(a[0] * s, a[1] * s), pack_bf16_rn(a[2] * s, a[3] * s),
                       pack_bf16_rn(c[0] * s, c[1] * s), pack_bf16_rn(c[2] * s, c[3] * s));
    }
  }
}

// The unfused append.  A warp appends to a unit at a time, half of it K's row and half V's,
// d / 16 neighbouring elements a lane; the rows and powers of two of up to kAppendUnits units
// are requested together.  Where a block's power of two changes (or is set anew, at the
// block's first slot), the warp takes the whole block into registers, 16 bytes a lane
// and load, all in flight together.  One CTA per sequence, or a cluster of up to 8: pos is advanced
// after a barrier over every thread that reads it.
constexpr int kAppendThreads = 512;
constexpr int kAppendWarps = kAppendThreads / 32;
constexpr int kAppendUnits = 2;
constexpr int kMaxAppendCtas = 8;

// A block's other tokens: their largest value (fp32 bits) where the byte is set anew, and their codes
// for the byte that `top` (the new row's largest, fp32 bits) then gives.  `others`: the rows
// that hold another token.  Returns the byte.
template <int D>
__device__ __forceinline__ int recode_block(uint8_t* block, uint32_t others, uint32_t top, int c_old, bool anew,
                                            int lane) {
  constexpr int CPR = D / 16;  // 16-byte chunks of a row
  uint4 x[CPR];                // chunks lane, lane + 32, ... of the block
#pragma unroll
  for (int e = 0; e < CPR; ++e) {
    x[e] = make_uint4(0u, 0u, 0u, 0u);
    if ((others >> ((lane + 32 * e) / CPR)) & 1u) x[e] = reinterpret_cast<const uint4*>(block)[lane + 32 * e];
  }
  int c = max(block_code(top), c_old);
  if (anew) {
    uint32_t m = 0u;
#pragma unroll
    for (int e = 0; e < CPR; ++e) m = max_codes16(m, x[e]);
    c = block_code(max(top, __reduce_max_sync(0xffffffffu, held_bits(m, c_old))));
  }
  if (c != c_old) {
    const float f = recode_factor(c_old, c);
#pragma unroll
    for (int e = 0; e < CPR; ++e)
      if ((others >> ((lane + 32 * e) / CPR)) & 1u) reinterpret_cast<uint4*>(block)[lane + 32 * e] = recode16(x[e], f);
  }
  return c;
}

template <int D>
__global__ void __launch_bounds__(kAppendThreads, 2)
window_append_q8_kernel(uint8_t* ring, uint8_t* scales, int64_t* pos, const uint16_t* __restrict__ k_new,
                        const uint16_t* __restrict__ v_new, int LH, int W, int S, int ctas) {
  constexpr int E = D / 16;  // elements a lane has of its row
  pdl_wait();
  pdl_trigger();
  const int b = static_cast<int>(blockIdx.x) / ctas;
  const int rank = static_cast<int>(blockIdx.x) - b * ctas;
  const int lane = threadIdx.x & 31;
  const int half = lane >> 4;
  const long long pb = *static_cast<volatile const int64_t*>(pos + b);
  const int slot = pb < 0           ? 0
                   : (pb >> 32) == 0 ? static_cast<int>(static_cast<unsigned>(pb) % static_cast<unsigned>(W))
                                     : static_cast<int>(pb % W);
  const int r = slot & (kQ8Block - 1);
  const int live = static_cast<int>(pb < W ? pb : W) - (slot - r);  // tokens from the block's first slot on
  const uint32_t others = (live >= 32 ? 0xFFFFFFFFu : live <= 0 ? 0u : (1u << live) - 1u) & ~(1u << r);
  for (int x0 = rank * kAppendWarps + static_cast<int>(threadIdx.x >> 5); pb >= 0 && x0 < LH;
       x0 += ctas * kAppendWarps * kAppendUnits) {
    uint4 row[kAppendUnits];
    int old[kAppendUnits];
#pragma unroll
    for (int q = 0; q < kAppendUnits; ++q) {
      const int x = x0 + q * ctas * kAppendWarps;
      row[q] = make_uint4(0u, 0u, 0u, 0u);
      old[q] = 0;
      if (x < LH) {
        const long long u = static_cast<long long>(b) * LH + x;
        const uint16_t* from = (half ? v_new : k_new) + u * D + (lane & 15) * E;
        if (D == 128) {
          row[q] = *reinterpret_cast<const uint4*>(from);
        } else {
          const uint2 w = *reinterpret_cast<const uint2*>(from);
          row[q] = make_uint4(w.x, w.y, 0u, 0u);
        }
        old[q] = scales[(2 * u + half) * S + slot / kQ8Block];
      }
    }
#pragma unroll
    for (int q = 0; q < kAppendUnits; ++q) {
      const int x = x0 + q * ctas * kAppendWarps;
      if (x >= LH) break;
      const long long u = static_cast<long long>(b) * LH + x;
      uint8_t* block = ring + (2 * u * W + slot - r) * D;  // K's; V's is W rows on
      float v[8];
      unpack8(row[q], v);
      uint32_t top = 0u;
#pragma unroll
      for (int e = 0; e < E; ++e) top = max(top, finite_bits(v[e]));
#pragma unroll
      for (int off = 1; off < 16; off <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, off));
      const int c_old = old[q];
      int c = max(block_code(top), c_old);
      if (r == 0 || __any_sync(0xffffffffu, c != c_old)) {
        const uint32_t tk = __shfl_sync(0xffffffffu, top, 0), tv = __shfl_sync(0xffffffffu, top, 16);
        const int ok = __shfl_sync(0xffffffffu, c_old, 0), ov = __shfl_sync(0xffffffffu, c_old, 16);
        const int ck = recode_block<D>(block, others, tk, ok, r == 0, lane);
        const int cv = recode_block<D>(block + static_cast<long long>(W) * D, others, tv, ov, r == 0, lane);
        c = half ? cv : ck;
      }
      const float f = code_factor(c);
      uint8_t* to = block + (static_cast<long long>(half) * W + r) * D + (lane & 15) * E;
      const uint32_t w0 = encode4(v[0], v[1], v[2], v[3], f);
      if (D == 128) *reinterpret_cast<uint2*>(to) = make_uint2(w0, encode4(v[4], v[5], v[6], v[7], f));
      else *reinterpret_cast<uint32_t*>(to) = w0;
      if ((lane & 15) == 0 && c != c_old) scales[(2 * u + half) * S + slot / kQ8Block] = static_cast<uint8_t>(c);
    }
  }
  // every thread that reads pos[b] has read it
  if (ctas > 1) {
    asm volatile("barrier.cluster.arrive.release;\n" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire;\n" ::: "memory");
  } else {
    __syncthreads();
  }
  if (rank == 0 && threadIdx.x == 0 && pb >= 0) pos[b] = pb + 1;
}

// The sizes of a call that takes k rows out of N; an index may name rows more than
// once, so k may be larger.
static int check_rows(const cmc_dims* dims, bool by_index) {
  if (!dims) return CMC_ERR_NULL;
  cmc_dims m = *dims;
  if (m.N < 1 || m.N > (1 << 24) || m.k > (1 << 24)) return CMC_ERR_SHAPE;
  m.Hq = m.Hkv;  // query heads and the window play no part here
  m.W = 1;
  if (by_index && m.k > m.N) m.N = m.k;
  return validate_dims(&m, true);
}

static unsigned row_grid(long long jobs) {
  const long long ctas = (jobs + kRowWarps - 1) / kRowWarps;
  return static_cast<unsigned>(ctas < (1LL << 30) ? ctas : (1LL << 30));
}

}  // namespace cmc

extern "C" {

int cmc_q8_scale_bytes(int rows) { return rows < 0 || rows > (1 << 24) ? 0 : cmc::q8_scale_bytes(rows); }

int cmc_quantize_cache(const void* bank_k, const void* bank_v, const int32_t* idx, const int64_t* count,
                       const cmc_dims* dims, void* kv, void* scales, uint32_t* status, void* stream) {
  using namespace cmc;
  int st = check_rows(dims, idx != nullptr);
  if (st != CMC_OK) return st;
  const cmc_dims& m = *dims;
  if (m.k == 0) return CMC_OK;
  if (!bank_k || !bank_v || !kv || !scales) return CMC_ERR_NULL;
  if (!aligned16(bank_k) || !aligned16(bank_v) || !aligned16(kv) || !aligned16(scales) ||
      (reinterpret_cast<uintptr_t>(idx) & 3) || (reinterpret_cast<uintptr_t>(count) & 7) ||
      (reinterpret_cast<uintptr_t>(status) & 3))
    return CMC_ERR_ALIGN;
  const int nb = (m.k + kQ8Block - 1) / kQ8Block;
  const long long jobs = 2LL * m.B * m.L * m.Hkv * nb;
  auto kern = m.d == 128 ? quantize_kernel<128> : quantize_kernel<64>;
  return launch_pdl(kern, dim3(row_grid(jobs)), dim3(kRowThreads), 0, static_cast<cudaStream_t>(stream),
                    static_cast<const uint4*>(bank_k), static_cast<const uint4*>(bank_v), idx, count,
                    static_cast<uint8_t*>(kv), static_cast<uint8_t*>(scales), status, jobs, nb,
                    m.L * m.Hkv, m.N, m.k, q8_scale_bytes(m.k));
}

int cmc_dequantize_cache(const void* kv, const void* scales, const int32_t* idx, const cmc_dims* dims,
                         void* out_k, void* out_v, uint32_t* status, void* stream) {
  using namespace cmc;
  int st = check_rows(dims, idx != nullptr);
  if (st != CMC_OK) return st;
  const cmc_dims& m = *dims;
  if (m.k == 0) return CMC_OK;
  if (!kv || !scales || !out_k || !out_v) return CMC_ERR_NULL;
  if (!aligned16(kv) || !aligned16(scales) || !aligned16(out_k) || !aligned16(out_v) ||
      (reinterpret_cast<uintptr_t>(idx) & 3) || (reinterpret_cast<uintptr_t>(status) & 3))
    return CMC_ERR_ALIGN;
  const int nb = (m.k + kQ8Block - 1) / kQ8Block;
  const long long jobs = 2LL * m.B * m.L * m.Hkv * nb;
  auto kern = m.d == 128 ? dequantize_kernel<128> : dequantize_kernel<64>;
  return launch_pdl(kern, dim3(row_grid(jobs)), dim3(kRowThreads), 0, static_cast<cudaStream_t>(stream),
                    static_cast<const uint8_t*>(kv), static_cast<const uint8_t*>(scales), idx,
                    static_cast<uint4*>(out_k), static_cast<uint4*>(out_v), status, jobs, nb,
                    m.L * m.Hkv, m.N, m.k, q8_scale_bytes(m.N));
}

int cmc_window_append_q8(void* ring_kv, void* ring_scales, int64_t* pos, const void* k_new,
                         const void* v_new, const cmc_dims* dims, void* stream) {
  using namespace cmc;
  int st = validate_dims(dims, false);
  if (st != CMC_OK) return st;
  if (!ring_kv || !ring_scales || !pos || !k_new || !v_new) return CMC_ERR_NULL;
  if (!aligned16(ring_kv) || !aligned16(ring_scales) || !aligned16(k_new) || !aligned16(v_new) ||
      (reinterpret_cast<uintptr_t>(pos) & 7))
    return CMC_ERR_ALIGN;
  const cmc_dims& m = *dims;
  const int LH = m.L * m.Hkv;
  int ctas = 1;
  while (ctas < kMaxAppendCtas && LH > static_cast<long long>(ctas) * kAppendWarps) ctas *= 2;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = static_cast<unsigned>(ctas);
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(m.B) * static_cast<unsigned>(ctas));
  cfg.blockDim = dim3(kAppendThreads);
  cfg.stream = static_cast<cudaStream_t>(stream);
  cfg.attrs = attr;
  cfg.numAttrs = ctas > 1 ? 2 : 1;
  auto kern = m.d == 128 ? window_append_q8_kernel<128> : window_append_q8_kernel<64>;
  return record_cuda_error(cudaLaunchKernelEx(
      &cfg, kern, static_cast<uint8_t*>(ring_kv), static_cast<uint8_t*>(ring_scales), pos,
      static_cast<const uint16_t*>(k_new), static_cast<const uint16_t*>(v_new), LH, m.W,
      q8_scale_bytes(m.W), ctas));
}

}  // extern "C"
