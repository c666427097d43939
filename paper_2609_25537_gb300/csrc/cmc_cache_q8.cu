// Writing and reading the 8-bit two-tier cache (format: cmc_q8.cuh): rows of a
// bf16 bank quantised into a cache, a cache read back, one token appended to an
// 8-bit ring.
#include <cuda_runtime.h>
#include <stdint.h>

#include "cmc_attn.cuh"
#include "cmc_q8.cuh"

namespace cmc {

// (No __restrict__: it lets inputs be read on the read-only path, and the launch before may still have been
// writing them when this one began.)
constexpr int kRowThreads = 128;  // four warps, each with blocks of rows of its own
constexpr int kRowWarps = kRowThreads / 32;

// Four bf16 values times a power of two (bf16, in both halves of f2) to codes.  The products are exact
// but for those below bf16's smallest, which give 0 either way.
__device__ __forceinline__ uint32_t encode4_bf16(uint32_t a, uint32_t b, uint32_t f2) {
  asm("mul.rn.bf16x2 %0, %0, %1;\n" : "+r"(a) : "r"(f2));
  asm("mul.rn.bf16x2 %0, %0, %1;\n" : "+r"(b) : "r"(f2));
  return e4m3_pair(bf16lo_to_f32(a), bf16hi_to_f32(a)) | (e4m3_pair(bf16lo_to_f32(b), bf16hi_to_f32(b)) << 16);
}

// A warp quantises blocks of 32 rows of one unit's K or V, one after another, from a ring of
// NST stages in shared memory that bulk copies fill ahead of it: one copy a block, or one a
// row where an index gathers them; rows that hold no token are not read.  A block goes
// through registers once, for its maximum and for its codes.
//
// HBM bounds it where there is enough to do: 1,024 rows of 256 units 33.0 us (90 % of the copy
// rate), 16,384 rows of 64 units 127 us (94 %).  At d = 128 an SM holds 20 warps with one stage
// each and 12 with two: one stage where every block then has a warp of its own (2,048 blocks
// 4.9 us, 6.2 with two), else two (20,480 blocks, a third of their rows with a token, 24.4 us,
// 28.7 with one; 22.1 since blocks without a token are only written).
template <int D, int NST>
__global__ void __launch_bounds__(kRowThreads)
quantize_kernel(const uint16_t* bank_k, const uint16_t* bank_v,
                const int32_t* idx, const int64_t* count,
                uint8_t* kv, uint8_t* scales, uint32_t* status,
                long long jobs, int nb, int LH, int N, int k, int S, uint32_t stall_tx) {
  constexpr int kStage = kQ8Block * D * 2;
  constexpr int NP = kStage / 512;  // passes of the warp over a block, 16 bytes a lane
  constexpr int RPP = 512 / (D * 2);  // rows of a pass
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ __align__(8) uint64_t bars[kRowWarps][NST];
  struct Job {  // of a stage: (unit, K or V), first row, the rows that hold a token
    long long uw;
    int r0;
    uint32_t rows;
  };
  __shared__ Job stage_jobs[kRowWarps][NST];
  const int lane = threadIdx.x & 31;
  const int warp = threadIdx.x >> 5;
  uint8_t* stages = smem + warp * (NST * kStage);
  uint64_t* full = bars[warp];
  Job* held = stage_jobs[warp];
  if (lane == 0) {
    for (int s = 0; s < NST; ++s) mbar_init(&full[s], 1);
    if (warp == 0) attn_abort = 0;
    asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
  }
  __syncthreads();
  pdl_wait();
  pdl_trigger();
  const long long first = static_cast<long long>(blockIdx.x) * kRowWarps + warp;
  const long long stride = static_cast<long long>(gridDim.x) * kRowWarps;

  // What a block's copies need: lane r has the bank row behind row r of the block, -1 if it holds none.
  struct Plan {
    long long uw;
    int r0, src;
  };
  auto plan = [&](long long job) {
    Plan m = {0, 0, -1};
    if (job >= jobs) return m;
    m.uw = job / nb;
    m.r0 = static_cast<int>(job - m.uw * nb) * kQ8Block;
    const long long b = (m.uw >> 1) / LH;
    const int i = m.r0 + lane;
    const long long n = count ? count[b] : k;
    if (i < k) {
      const int row = idx ? idx[b * k + i] : i;
      if (i < n) {
        m.src = row;
        if (static_cast<unsigned>(row) >= static_cast<unsigned>(N)) {
          m.src = -1;
          if (status) atomicOr(status, CMC_DEVFLAG_BAD_INDEX);
        }
      }
    }
    return m;
  };
  auto request = [&](int s, const Plan& m) {
    const uint32_t rows = __ballot_sync(0xffffffffu, m.src >= 0);
    const uint16_t* bank = ((m.uw & 1) ? bank_v : bank_k) + (m.uw >> 1) * N * D;
    if (lane == 0) {
      held[s] = {m.uw, m.r0, rows};
      mbar_arrive_expect_tx(&full[s], __popc(rows) * (D * 2) + stall_tx);
    }
    __syncwarp();
    const uint32_t to = smem_addr(stages + s * kStage);
    if (idx) {
      if (m.src >= 0) bulk_copy(to + lane * (D * 2), bank + static_cast<long long>(m.src) * D, D * 2, &full[s]);
    } else if (lane == 0 && rows) {  // rows r0, r0 + 1, ...
      bulk_copy(to, bank + static_cast<long long>(m.r0) * D, __popc(rows) * (D * 2), &full[s]);
    }
  };
#pragma unroll 1
  for (int s = 0; s < NST; ++s)
    if (first + s * stride < jobs) request(s, plan(first + s * stride));
  Plan next = plan(first + NST * stride);  // its loads are on their way while a block is worked on
  __syncwarp();
  int s = 0;
  uint32_t phase = 0;
#pragma unroll 1
  for (long long job = first; job < jobs; job += stride) {
    if (__any_sync(0xffffffffu, !mbar_wait(&full[s], phase))) {  // never expected: see mbar_wait
      const uint32_t t0 = global_ns32();
      for (uint32_t it = 0; it < (1u << 16) && global_ns32() - t0 < kDrainNs; ++it) __nanosleep(1000);
      if (lane == 0 && status) atomicOr(status, CMC_DEVFLAG_TIMEOUT);
      return;
    }
    const Job h = held[s];
    const uint8_t* from = stages + s * kStage + lane * 16;
    uint8_t* dst = kv + (h.uw * k + h.r0) * D + lane * 8;
    const int jb = h.r0 / kQ8Block;
    uint8_t* sc = scales + h.uw * S;
    if (jb == nb - 1 && nb + lane < S) sc[nb + lane] = 0;  // the padding, at most three bytes
    uint4 x[NP];
    uint32_t m = 0u;  // largest magnitude, bf16 bits in two halves
    if (h.rows != 0u) {
#pragma unroll
      for (int e = 0; e < NP; ++e) {
        x[e] = make_uint4(0u, 0u, 0u, 0u);
        if ((h.rows >> (e * RPP + lane / (32 / RPP))) & 1u) x[e] = *reinterpret_cast<const uint4*>(from + e * 512);
        m = __vmaxu2(m, x[e].x & 0x7FFF7FFFu);
        m = __vmaxu2(m, x[e].y & 0x7FFF7FFFu);
        m = __vmaxu2(m, x[e].z & 0x7FFF7FFFu);
        m = __vmaxu2(m, x[e].w & 0x7FFF7FFFu);
      }
    }
    __syncwarp();  // the stage is free
    if (job + NST * stride < jobs) {
      request(s, next);
      next = plan(job + (NST + 1) * stride);
    }
    int c = 0;
    if (h.rows != 0u) {
      uint32_t top = __reduce_max_sync(0xffffffffu, max(m & 0xFFFFu, m >> 16));
      if (top >= 0x7F80u) {  // an infinity or NaN among them: both become NaN, and do not count
        top = 0u;
#pragma unroll
        for (int e = 0; e < NP; ++e) {
          uint32_t* w = reinterpret_cast<uint32_t*>(&x[e]);
#pragma unroll
          for (int q = 0; q < 4; ++q) {
#pragma unroll
            for (int sh = 0; sh < 32; sh += 16) {
              const uint32_t a = (w[q] >> sh) & 0x7FFFu;
              if (a >= 0x7F80u) w[q] |= 0x7FFFu << sh;
              else top = max(top, a);
            }
          }
        }
        top = __reduce_max_sync(0xffffffffu, top);
      }
      c = block_code(top << 16);
      const uint32_t f2 = __byte_perm(__float_as_uint(code_factor(c)), 0u, 0x3232);  // in bf16, twice
#pragma unroll
      for (int e = 0; e < NP; ++e) {
        if (h.r0 + e * RPP + lane / (32 / RPP) < k)
          *reinterpret_cast<uint2*>(dst + e * 256) =
              make_uint2(encode4_bf16(x[e].x, x[e].y, f2), encode4_bf16(x[e].z, x[e].w, f2));
      }
    } else {  // no token: codes and power of two are zero
#pragma unroll
      for (int e = 0; e < NP; ++e)
        if (h.r0 + e * RPP + lane / (32 / RPP) < k) *reinterpret_cast<uint2*>(dst + e * 256) = make_uint2(0u, 0u);
    }
    if (lane == 0) sc[jb] = static_cast<uint8_t>(c);
    if (++s == NST) {
      s = 0;
      phase ^= 1u;
    }
  }
}

// A warp reads back 32 rows of one unit's K or V at a time, all its loads in flight together; the writes
// are two thirds of the bytes.  HBM bounds it where there is enough to do: 16,384 rows of 64 units (0.8 GB
// in all) 117.5 us, the copy rate; 2,048 blocks 5.2 us, of which 3.7 are HBM's.
template <int D>
__global__ void __launch_bounds__(kRowThreads)
dequantize_kernel(const uint8_t* kv, const uint8_t* scales,
                  const int32_t* idx, uint4* out_k,
                  uint4* out_v, uint32_t* status, long long jobs, int nb, int LH, int N,
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
//
// Latency bounds it: the position, then a row and its byte, then the block where it is taken, each a trip to
// memory.  A single unit takes 1.7 to 2.1 us, 32 sequences of 256 units 6.9 us (HBM's part of that is 0.9),
// and 11.1 where more of their blocks change (with one row at a time a warp, and a changed
// block read by a lane a row, 29).  At d = 128 two blocks' chunks a lane do not fit 64 registers, which two CTAs
// an SM leave: 64 bytes are spilled.
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
    const Recode f = recode_by(c_old, c);
#pragma unroll
    for (int e = 0; e < CPR; ++e)
      if ((others >> ((lane + 32 * e) / CPR)) & 1u) reinterpret_cast<uint4*>(block)[lane + 32 * e] = recode16(x[e], f);
  }
  return c;
}

template <int D>
__global__ void __launch_bounds__(kAppendThreads, 2)
window_append_q8_kernel(uint8_t* ring, uint8_t* scales, int64_t* pos, const uint16_t* k_new,
                        const uint16_t* v_new, int LH, int W, int S, int ctas) {
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
// once, so k may be larger.  No rows can be taken out of none.
static int check_rows(const cmc_dims* dims, bool by_index) {
  if (!dims) return CMC_ERR_NULL;
  cmc_dims m = *dims;
  if (m.N < (m.k == 0 ? 0 : 1) || m.N > (1 << 24) || m.k > (1 << 24)) return CMC_ERR_SHAPE;
  m.Hq = m.Hkv;  // query heads and the window play no part here
  m.W = 1;
  if (m.N == 0 || (by_index && m.k > m.N)) m.N = m.k > 0 ? m.k : 1;
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
  const long long ctas = (jobs + kRowWarps - 1) / kRowWarps;
  const long long one = 5LL * sm_count() * (m.d == 128 ? 1 : 2);  // CTAs of one wave with one stage a warp
  const int nst = ctas <= one ? 1 : 2;
  const long long wave = nst == 1 ? one : 3LL * sm_count() * (m.d == 128 ? 1 : 2);
  auto kern = m.d == 128 ? (nst == 1 ? quantize_kernel<128, 1> : quantize_kernel<128, 2>)
                         : (nst == 1 ? quantize_kernel<64, 1> : quantize_kernel<64, 2>);
  const int smem = kRowWarps * nst * kQ8Block * m.d * 2;
  if (smem > 48 * 1024) {
    st = record_cuda_error(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
    if (st != CMC_OK) return st;
  }
  return launch_pdl(kern, dim3(static_cast<unsigned>(ctas < wave ? ctas : wave)), dim3(kRowThreads), smem,
                    static_cast<cudaStream_t>(stream), static_cast<const uint16_t*>(bank_k),
                    static_cast<const uint16_t*>(bank_v), idx, count,
                    static_cast<uint8_t*>(kv), static_cast<uint8_t*>(scales), status, jobs, nb,
                    m.L * m.Hkv, m.N, m.k, q8_scale_bytes(m.k), stall_tx_setting());
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
