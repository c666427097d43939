// Decode attention over [Tier-1 | Tier-2] that adds to each key's weight the probabilities it gets
// (cmc_two_tier_decode_attn_weighted), and the decode step around it (cmc_decode_step_weighted):
//   out[h]    = sum_j p_hj v_j,   p_hj = 2^(c (s_hj - M_h)) / l_h,   s = q_h . k_j, c = scale log2(e)
//   weight[j] += sum of p_hj over the G query heads of the KV head
// The probabilities need the final maximum M and sum l, which one pass over the keys knows only at its
// end.  So each CTA keeps the products q . k of its keys, and their weights, in shared memory (4 G + 4 bytes a key,
// beside the key's 4 d bytes in HBM), and when its unit's M and l are known goes over them once more.
//
// Bound: HBM, 4 d + 8 bytes a key against 4 G d flops.  A unit (sequence, layer, KV head) is taken by a CTA of
// four warps, a cluster of up to eight such CTAs, or, where there are many short ones, by one warp or two.  Its keys are cut
// into blocks of 32, ceil(k / 32) of Tier-1, then those of the ring's occupied slots, and warp w of the unit's n takes
// blocks w, w + n, ...  The warps have nothing to do with each other until the end: each copies its own blocks' rows (cp.async,
// 16 bytes a lane) into a stage of its own, K and V of one block, and requests the next block's K as soon as the products
// have read this one's, its V likewise.  Rows that hold no token are not read, their places are filled with zeros.  Twelve
// warps of 16 KB an SM keep enough on the way.  The two products are those of cmc_attn.cu,
//   S^T = K Q^T     16 keys as the M rows, the G query heads (padded to 8) as the columns
//   O^T += V^T P^T  16 rows of the head dimension, the heads, 16 keys as the k-step
// (mma.sync m16n8k16, ldmatrix; 4 flops a byte: the tensor pipe is all but idle).
//
// What a warp does with a block is a chain of latencies, so that its length and the warps an SM holds set the rate, not the
// bytes on the way: 32 layers of 128 + 512 keys, fused step with norm and rotation, 13.1 us (12.9 at the copy rate), with blocks of 16
// keys fed from registers 17.7 (six warps a CTA) to 22.6, through private stages with two or three blocks on the way 21.6 to 30.
//
// The new token (fused step) is read from k_new and v_new where its slot's row would be, by the warp that has
// the block, which stores it to the ring as well.  With norm or rotary embedding the warps first
// prepare q and the new key, a row a warp, while their blocks are on the way; q is then held as the sum of two bf16 (products off
// by 2^-16 of a term: the weights are sums in fp32 that outlive the call), the key rounded to bf16 as it is stored.
#include <algorithm>
#include <atomic>

#include "cmc_prep.cuh"
#include "cmc_ranges.cuh"

namespace cmc {

constexpr int kBlkKeys = 32;
constexpr int kWarpsMost = 4;  // of a CTA
// Products and weights that a CTA keeps in shared memory, in bytes: as many as leave two CTAs of four warps on an SM.
// Units too long for a cluster of eight at that keep them in the workspace (us a launch at 40 KB / 64 KB / 10 KB: 64 units of
// 16,384 keys 79 / 98 / 103, of 20,480 keys 125 / 152 / 126), but where there is no more than a CTA an SM.
constexpr int score_cap(int G) { return G == 8 ? 41472 : 46080; }
constexpr int kScoreMost = 131072;
// Blocks a warp prefetches, at most.  What it holds of the ring is not known then, so that more of them fetch rows without a token:
// us a launch with none / one / two / three, 256 units of 128 + 512 keys, rings full 15.5 / 13.7 / 13.1 / 13.5, of different fill
// 10.1 / 9.0 / 9.1 / 10.5.  A warp with a unit of its own takes one block of the ring alone: 2,048 units of 30 + 8..130 keys, step with
// rotation, 17.4 / 17.2 / 18.2 / 21.4, with one of the ring among two 17.4, and 16.5 where the second is prefetched as soon as it is
// known to hold tokens; of 128 + 256 keys, full, 62.5 / 59.3 / 57.3 / 58.2, 57.2.
constexpr int kPrefetchMost = 2;
// Blocks of a unit that is given to one warp or two, at most (see launch_weighted).
constexpr int kSoloBlocks = 16;

struct WeightedParams {
  const uint16_t* q;      // [B, L, Hq, d]
  const uint16_t* t1k;    // [B, L, Hkv, N, d]
  const uint16_t* t1v;
  float* t1w;             // [B, L, Hkv, N]
  uint16_t* ring_k;       // [B, L, Hkv, W, d]
  uint16_t* ring_v;
  float* ring_w;          // [B, L, Hkv, W]
  int64_t* pos;           // [B]
  const uint16_t* k_new;  // [B, L, Hkv, d]
  const uint16_t* v_new;
  uint16_t* out;          // [B, L, Hq, d]
  uint32_t* status;
  unsigned long long* tickets;
  float* scratch;         // products of a unit too long for shared memory, or NULL
  int B, L, Hkv, N, k, W, LH;
  int cm;                 // CTAs per unit
  int nb1;                // blocks of Tier-1
  int iters;              // blocks a warp takes at most
  int prefetch;           // blocks per warp prefetched into L2 before the grid dependency wait
  float scale_log2;
  PrepParams prep;
};

__host__ __device__ constexpr int wrow_floats(int D) { return D + 4; }

// Shared memory: the warps' stages (a block's K and V each), Q as bf16 sums and the prepared key (with PREP), the warps' maxima and
// sums, a cluster's record, then the products.  At the end a warp's stage holds its output.
template <int D, int G, bool PREP, int NW>
struct WSmem {
  static constexpr int kBlk = kBlkKeys * D * 4;                    // K and V of a block
  static constexpr int kQ = NW * kBlk;                             // [2][G][D] bf16: high and low parts
  static constexpr int kNew = kQ + (PREP ? 2 * G * D * 2 : 0);     // [D] bf16
  static constexpr int kM = kNew + (PREP ? D * 2 : 0);             // [warp][8] maxima, [warp][8] sums
  static constexpr int kRecMl = kM + NW * 16 * 4;                  // a cluster's record: [8][2] maxima and sums,
  static constexpr int kRec = kBlk / 2;                            // and, in a stage when all are done, [G][D] output
  static constexpr int kFin = kRecMl + 16 * 4;                     // [8] final maxima, [8] 1 / sums
  static constexpr int kScores = kFin + 16 * 4;
  static_assert(kScores % 16 == 0, "read by 16 bytes");
  static_assert(G * wrow_floats(D) * 4 <= kBlk / 2 && G * D * 4 <= kBlk / 2, "a stage holds an output and a record");
};

__device__ __forceinline__ void wmma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                     uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, "
      "{%8,%9}, {%0,%1,%2,%3};\n"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// 16 bytes of what a launch reads once, or as many zeros, into shared memory.
__device__ __forceinline__ void copy_once(uint32_t dst, const uint16_t* src, bool valid, uint64_t policy) {
  asm volatile("cp.async.cg.shared.global.L2::cache_hint [%0], [%1], 16, %2, %3;\n" ::"r"(dst), "l"(src),
               "r"(valid ? 16 : 0), "l"(policy)
               : "memory");
}
__device__ __forceinline__ void copy_once(uint32_t dst, const uint16_t* src, uint64_t policy) {
  asm volatile("cp.async.cg.shared.global.L2::cache_hint [%0], [%1], 16, %2;\n" ::"r"(dst), "l"(src),
               "l"(policy)
               : "memory");
}
__device__ __forceinline__ void ldsm_x4_trans(uint32_t addr, uint32_t& r0, uint32_t& r1, uint32_t& r2, uint32_t& r3) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];\n"
               : "=r"(r0), "=r"(r1), "=r"(r2), "=r"(r3)
               : "r"(addr)
               : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;\n" ::: "memory"); }

// Maxima are those of the products; a difference from one is scaled, not the products first, since what rounding leaves of two equal scores
// of 2^31 and more is a power of two that fp32 does not hold.  A maximum that differences are taken from: 0 where there is none (no key, or
// NaN alone: 2^x of those is then 0 and NaN).
__device__ __forceinline__ float finite_max(float m) { return m == -INFINITY ? 0.f : m; }

__device__ __forceinline__ float2 ld_peer_f2(uint32_t addr) {
  float2 v;
  asm volatile("ld.shared::cluster.v2.f32 {%0,%1}, [%2];\n" : "=f"(v.x), "=f"(v.y) : "r"(addr) : "memory");
  return v;
}
__device__ __forceinline__ float4 ld_peer_f4(uint32_t addr) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0,%1,%2,%3}, [%4];\n"
               : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w)
               : "r"(addr)
               : "memory");
  return v;
}

// A block of a unit: its rows in memory and how many hold keys.
struct Blk {
  const uint16_t* k;
  const uint16_t* v;
  float* w;
  int rows;     // 1 .. 32
  int new_row;  // the new token's, or -1
};

template <int D>
__device__ __forceinline__ Blk blk_of(const WeightedParams& p, long long u, int blk, int count, int new_slot) {
  Blk r;
  r.new_row = -1;
  if (blk < p.nb1) {
    const long long e = (u * p.N + blk * kBlkKeys) * D;
    r.k = p.t1k + e;
    r.v = p.t1v + e;
    r.w = p.t1w + (u * p.N + blk * kBlkKeys);
    r.rows = min(p.k - blk * kBlkKeys, kBlkKeys);
  } else {
    const int s0 = (blk - p.nb1) * kBlkKeys;
    const long long e = (u * p.W + s0) * D;
    r.k = p.ring_k + e;
    r.v = p.ring_v + e;
    r.w = p.ring_w + (u * p.W + s0);
    r.rows = min(count - s0, kBlkKeys);
    if (new_slot >= s0 && new_slot < s0 + kBlkKeys) r.new_row = new_slot - s0;
  }
  return r;
}

// Offset of 16-byte chunk c of row r within K or V of a stage: columns of 128 bytes, the chunks of a row in the
// order c ^ (r & 7), so that eight rows of a chunk lie in different banks.
template <int D>
__device__ __forceinline__ uint32_t swz(int r, int c) {
  return static_cast<uint32_t>((c >> 3) * (kBlkKeys * 128) + r * 128 + (((c & 7) ^ (r & 7)) << 4));
}

// Requests the rows of K or of V of a block into a stage: eight lanes to 128 bytes of a row, four rows at a time.
// Rows that hold no token are filled with zeros.  `fresh`: the new token's row, or NULL where it is put in later.
template <int D>
__device__ __forceinline__ void request_rows(const uint16_t* base, int rows, int new_row, const uint16_t* fresh, int lane,
                                             uint64_t pol, uint32_t to) {
  const int sub = lane >> 3, c = lane & 7;
  const uint16_t* src = base + sub * D + c * 8;
  const uint32_t even = to + sub * 128 + ((c ^ sub) << 4), odd = to + sub * 128 + ((c ^ (sub + 4)) << 4);
  if (rows == kBlkKeys && new_row < 0) {
#pragma unroll
    for (int j = 0; j < kBlkKeys / 4; ++j)
#pragma unroll
      for (int h = 0; h < D / 64; ++h)
        copy_once((j & 1 ? odd : even) + j * 512 + h * (kBlkKeys * 128), src + j * 4 * D + h * 64, pol);
    return;
  }
#pragma unroll
  for (int j = 0; j < kBlkKeys / 4; ++j) {
    const int row = 4 * j + sub;
    const bool is_new = row == new_row;
    const bool valid = row < rows && !(is_new && fresh == nullptr);
    const uint16_t* from = valid ? (is_new ? fresh + c * 8 : src + j * 4 * D) : base;
#pragma unroll
    for (int h = 0; h < D / 64; ++h)
      copy_once((j & 1 ? odd : even) + j * 512 + h * (kBlkKeys * 128), from + (valid ? h * 64 : 0), valid, pol);
  }
}

// The sum of squares of a row, four elements a lane.
__device__ __forceinline__ float row_squares(const float (&x)[4], float by) {
  float s = quad_squares(by * x[0], by * x[1], by * x[2], by * x[3]);
#pragma unroll
  for (int off = 1; off < 32; off <<= 1) s += __shfl_xor_sync(0xffffffffu, s, off);
  return s;
}

// Norm and rotation of the unit's G query heads and of the new key, a row a warp, into shared memory.  Lane i
// < d / 4 has elements 2 i, 2 i + 1 and their partners d / 2 further on.  Everything that it reads is requested at once
// (`turns` before the grid dependency wait), and the norm does not wait for pos: what is left on the way to the first
// products is one trip for pos, two sines and cosines a lane and a barrier.  (With d / 16 lanes to a row and two warps for all
// of them, as prefill_kernel has it, that took 2 us.)
template <int D, int G, int NW>
struct Preparer {
  static constexpr int kRows = (G + NW) / NW;  // rows of a warp
  unsigned long long turns[2];
  uint32_t row[kRows][2];
  float2 gain[2][2];  // of the queries, of the key
  long long moved;

  __device__ __forceinline__ void tables(const WeightedParams& p, int lane) {
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int i = (2 * lane + e) % (D / 2);
      turns[e] = p.prep.rope_slot >= 0 ? g_rope_tables[p.prep.rope_slot][i] : p.prep.rope_turns[i];
    }
  }
  __device__ __forceinline__ void request(const WeightedParams& p, long long u, int b, int warp, int lane) {
    moved = p.prep.evicted ? p.prep.evicted[b] : 0;
    const int e = 2 * lane % (D / 2);
    const size_t l = static_cast<unsigned>(u) % static_cast<unsigned>(p.LH) / static_cast<unsigned>(p.Hkv);
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const float* w = x == 0 ? p.prep.q_weight : p.prep.k_weight;
      if (w != nullptr) {
        gain[x][0] = *reinterpret_cast<const float2*>(w + l * D + e);
        gain[x][1] = *reinterpret_cast<const float2*>(w + l * D + D / 2 + e);
      }
    }
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
      const int r = warp + i * NW;
      row[i][0] = row[i][1] = 0u;
      if (r <= G && lane < D / 4) {
        const uint16_t* src = r < G ? p.q + (u * G + r) * D : p.k_new + u * D;
        row[i][0] = *reinterpret_cast<const uint32_t*>(src + e);
        row[i][1] = *reinterpret_cast<const uint32_t*>(src + D / 2 + e);
      }
    }
  }
  __device__ __forceinline__ void finish(const WeightedParams& p, long long u, long long pos, int warp, int lane,
                                         uint8_t* smem) {
    using S = WSmem<D, G, true, NW>;
    const unsigned long long at = static_cast<unsigned long long>(p.prep.rope_offset + pos) +
                                  static_cast<unsigned long long>(moved);
    float2 cs[2];
#pragma unroll
    for (int e = 0; e < 2; ++e) cs[e] = p.prep.rope ? rope_cos_sin(at, turns[e]) : make_float2(1.f, 0.f);
    float4 pair[2][2];  // of the queries, of the key
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const bool norm = (x == 0 ? p.prep.q_weight : p.prep.k_weight) != nullptr;
      pair[x][0] = pair_factors(norm ? gain[x][0].x : 1.f, norm ? gain[x][1].x : 1.f, cs[0]);
      pair[x][1] = pair_factors(norm ? gain[x][0].y : 1.f, norm ? gain[x][1].y : 1.f, cs[1]);
    }
    auto turn_and_put = [&](int r, float (&x)[4], float f) {
      prep_pair(x[0], x[2], f, p.prep.rope, r < G ? pair[0][0] : pair[1][0]);
      prep_pair(x[1], x[3], f, p.prep.rope, r < G ? pair[0][1] : pair[1][1]);
      if (lane >= D / 4) return;
      uint16_t* to = reinterpret_cast<uint16_t*>(smem + (r < G ? S::kQ + r * D * 2 : S::kNew)) + 2 * lane;
      const uint32_t a = pack_bf16_rn(x[0], x[1]), z = pack_bf16_rn(x[2], x[3]);
      *reinterpret_cast<uint32_t*>(to) = a;
      *reinterpret_cast<uint32_t*>(to + D / 2) = z;
      if (r < G) {  // what is left (nothing that can be held where the high part is infinite)
        const float h[4] = {bf16lo_to_f32(a), bf16hi_to_f32(a), bf16lo_to_f32(z), bf16hi_to_f32(z)};
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = fabsf(h[e]) < INFINITY ? x[e] - h[e] : 0.f;
        to += G * D;
        *reinterpret_cast<uint32_t*>(to) = pack_bf16_rn(x[0], x[1]);
        *reinterpret_cast<uint32_t*>(to + D / 2) = pack_bf16_rn(x[2], x[3]);
      }
    };
    auto has_norm = [&](int r) { return (r < G ? p.prep.q_weight : p.prep.k_weight) != nullptr; };
    bool odd = false;
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
      const int r = warp + i * NW;
      if (r > G) break;
      float x[4] = {bf16lo_to_f32(row[i][0]), bf16hi_to_f32(row[i][0]), bf16lo_to_f32(row[i][1]), bf16hi_to_f32(row[i][1])};
      float f = 1.f;
      if (has_norm(r)) {
        const float mean = row_mean<D>(row_squares(x, 1.f), p.prep.eps);
        f = rsqrtf(mean);
        odd |= odd_mean(mean);
      }
      turn_and_put(r, x, f);
    }
    if (odd) {  // a row whose mean is odd (the same in all lanes): the warp's rows again, from memory
#pragma unroll 1
      for (int r = warp; r <= G; r += NW) {
        if (!has_norm(r)) continue;
        const uint16_t* src = (r < G ? p.q + (u * G + r) * D : p.k_new + u * D) + 2 * lane % (D / 2);
        const uint32_t lo = lane < D / 4 ? *reinterpret_cast<const uint32_t*>(src) : 0u;
        const uint32_t hi = lane < D / 4 ? *reinterpret_cast<const uint32_t*>(src + D / 2) : 0u;
        __syncwarp();
        float x[4] = {bf16lo_to_f32(lo), bf16hi_to_f32(lo), bf16lo_to_f32(hi), bf16hi_to_f32(hi)};
        const float mean = row_mean<D>(row_squares(x, 1.f), p.prep.eps);
        if (!odd_mean(mean)) continue;
        const float by = odd_scale(mean);
        float f = rsqrtf(row_mean<D>(row_squares(x, by), p.prep.eps, by));
        if (by < 1.f) f *= by;
        else
#pragma unroll
          for (int e = 0; e < 4; ++e) x[e] *= by;
        turn_and_put(r, x, f);
      }
    }
  }
};

// NW warps a CTA, whose registers allow twelve on an SM.
template <int D, int G, bool FUSED, bool PREP, int NW, bool ORDER>
__global__ void __launch_bounds__(32 * NW, 12 / NW)
weighted_attn_kernel(const __grid_constant__ WeightedParams p) {
  using S = WSmem<D, G, PREP, NW>;
  constexpr int kThreadsOfCta = 32 * NW;
  constexpr int DP = wrow_floats(D);
  constexpr int KS = D / 16;  // k-steps of S^T, m-tiles of O^T
  extern __shared__ __align__(16) uint8_t smem[];
  float* merge_m = reinterpret_cast<float*>(smem + S::kM);
  float* merge_l = merge_m + NW * 8;
  float* rec_o = reinterpret_cast<float*>(smem + S::kRec);
  float* rec_ml = reinterpret_cast<float*>(smem + S::kRecMl);
  float* fin_m = reinterpret_cast<float*>(smem + S::kFin);
  float* fin_r = fin_m + 8;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int g = lane >> 2, t = lane & 3;
  long long u = blockIdx.x / static_cast<unsigned>(p.cm);
  const int rank = static_cast<int>(blockIdx.x - u * p.cm);
  int b = static_cast<int>(static_cast<unsigned>(u) / static_cast<unsigned>(p.LH));
  const int stride = p.cm * NW;
  const int first = rank * NW + warp;

  // The warp's first blocks, into L2: hints, which may come before the wait (where the unit is known).
  if (!ORDER && lane < 2 * p.prefetch) {
    const int blk = first + (lane >> 1) * stride;
    const uint16_t* base = nullptr;
    int rows = 0;
    if (blk < p.nb1) {
      base = ((lane & 1) ? p.t1v : p.t1k) + (u * p.N + blk * kBlkKeys) * D;
      rows = min(p.k - blk * kBlkKeys, kBlkKeys);
    } else if ((NW > 1 || lane < 2) && (blk - p.nb1) * kBlkKeys < p.W) {
      base = ((lane & 1) ? p.ring_v : p.ring_k) + (u * p.W + (blk - p.nb1) * kBlkKeys) * D;
      rows = min(p.W - (blk - p.nb1) * kBlkKeys, kBlkKeys);
    }
    if (rows > 0)
      asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;\n" ::"l"(base), "r"(rows * D * 2) : "memory");
  }
  Preparer<D, G, NW> prep;
  if (PREP) prep.tables(p, lane);  // written long before this launch
  pdl_wait();
  pdl_trigger();
  if (ORDER) {
    // The unit of place u / LH in the sequences' order by length, the longest first: a long unit that starts last sets the
    // time of the launch.  All CTAs see the same positions, which the last of them advances in the end.
    int* live = reinterpret_cast<int*>(smem);  // of the stages, which hold nothing yet
    int* seq = live + kThreadsOfCta;
    int mine = -2;
    if (tid < p.B) {
      long long x;
      asm volatile("ld.global.cg.s64 %0, [%1];\n" : "=l"(x) : "l"(p.pos + tid) : "memory");
      mine = static_cast<int>(x < 0 ? -1 : x < p.W ? x : p.W);
    }
    live[tid] = mine;
    __syncthreads();
    if (tid < p.B) {
      int place = 0;
#pragma unroll 4
      for (int i = 0; i < p.B; i += 4) {
        const int4 x = *reinterpret_cast<const int4*>(live + i);
        place += (x.x > mine || (x.x == mine && i < tid)) + (x.y > mine || (x.y == mine && i + 1 < tid)) +
                 (x.z > mine || (x.z == mine && i + 2 < tid)) + (x.w > mine || (x.w == mine && i + 3 < tid));
      }
      if (place == b) *seq = tid;
    }
    __syncthreads();
    // (A reduction, so that the compiler knows the sequence for the same in all lanes.)
    const int s0 = static_cast<int>(__reduce_max_sync(0xffffffffu, static_cast<unsigned>(*seq)));
    __syncthreads();
    u += static_cast<long long>(s0 - b) * p.LH;
    b = s0;
  }

  long long pos;
  asm volatile("ld.global.cg.s64 %0, [%1];\n" : "=l"(pos) : "l"(p.pos + b) : "memory");
  const uint16_t* newk = FUSED ? p.k_new + u * D : nullptr;
  const uint16_t* newv = FUSED ? p.v_new + u * D : nullptr;
  uint32_t qa[KS][2], ql[PREP ? KS : 1][2];  // Q^T fragments: column g, rows 16 i + 2 t and + 8; what high parts leave
#pragma unroll
  for (int i = 0; i < KS; ++i)
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      qa[i][h] = 0u;
      if (PREP) ql[PREP ? i : 0][h] = 0u;
      if (!PREP && g < G) qa[i][h] = *reinterpret_cast<const uint32_t*>(p.q + (u * G + g) * D + 16 * i + 8 * h + 2 * t);
    }
  if (PREP) prep.request(p, u, b, warp, lane);
  // Blocks of Tier-1 do not wait for pos.
  const uint64_t pol = policy_evict_first();
  // The products of this CTA's keys, [iteration][warp][32 keys][G], then their weights, [iteration][warp][32 keys].
  const int slots = p.iters * NW * kBlkKeys;
  float* scores = p.scratch ? p.scratch + static_cast<long long>(blockIdx.x) * slots * (G + 1)
                            : reinterpret_cast<float*>(smem + S::kScores);
  float* weights = scores + static_cast<long long>(slots) * G;
  const uint32_t stage = smem_addr(smem) + warp * S::kBlk;
  // Requests K, or V and the weights, of the block of iteration n, if the warp has one, into the warp's stage.
  auto request_k = [&](int blk, int last, int count, int new_slot, const uint16_t* fresh) {
    if (blk < last) {
      const Blk x = blk_of<D>(p, u, blk, count, new_slot);
      request_rows<D>(x.k, x.rows, x.new_row, fresh, lane, pol, stage);
    }
    copy_commit();
  };
  auto request_v = [&](int n, int blk, int last, int count, int new_slot, const uint16_t* fresh) {
    if (blk < last) {
      const Blk x = blk_of<D>(p, u, blk, count, new_slot);
      request_rows<D>(x.v, x.rows, x.new_row, fresh, lane, pol,
                      stage + S::kBlk / 2);
      const bool valid = lane < x.rows && lane != x.new_row;
      float* w = weights + (n * NW + warp) * kBlkKeys + lane;
      if (p.scratch) *w = valid ? x.w[lane] : 0.f;
      else cp_async_4(smem_addr(w), valid ? x.w + lane : x.w, valid ? 4u : 0u);
    }
    copy_commit();
  };
  if (first < p.nb1) {
    request_k(first, p.nb1, 0, -1, nullptr);
    request_v(0, first, p.nb1, 0, -1, nullptr);
  }
  int count = -1, new_slot = -1;
  if (pos >= 0) {
    if (FUSED) {
      count = static_cast<int>(pos + 1 < p.W ? pos + 1 : p.W);
      new_slot = (pos >> 32) == 0
                     ? static_cast<int>(static_cast<unsigned>(pos) % static_cast<unsigned>(p.W))
                     : static_cast<int>(pos % p.W);
    } else {
      count = static_cast<int>(pos < p.W ? pos : p.W);
    }
  }
  // The same in all lanes, as pos is; a reduction, so that the compiler knows it too: the loop below has instructions that a
  // warp executes as one (ldmatrix, mma, movmatrix), and what decides how often it runs, and which of its branches, comes from here.
  count = __reduce_max_sync(0xffffffffu, count);
  new_slot = __reduce_max_sync(0xffffffffu, new_slot);
  const bool bad = count < 0;
  const int nblk = bad ? 0 : p.nb1 + (count + kBlkKeys - 1) / kBlkKeys;
  if (NW == 1 && lane < 2 && p.prefetch > 1 && first + stride >= p.nb1 && first + stride < nblk) {  // the second, now known
    const Blk x = blk_of<D>(p, u, first + stride, count, new_slot);
    asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;\n" ::"l"(lane ? x.v : x.k), "r"(x.rows * D * 2) : "memory");
  }
  uint16_t* put_k = p.ring_k + (u * p.W + new_slot) * D;  // (not used without a new token)
  uint16_t* put_v = p.ring_v + (u * p.W + new_slot) * D;
  if (PREP) newk = nullptr;  // put in when it is prepared
  if (first >= p.nb1) {
    request_k(first, nblk, count, new_slot, newk);
    request_v(0, first, nblk, count, new_slot, newv);
  }
  const uint16_t* prepared = nullptr;
  if (PREP) {
    prepared = reinterpret_cast<const uint16_t*>(smem + S::kNew);
    prep.finish(p, u, pos, warp, lane, smem);
    __syncthreads();
    if (g < G) {
#pragma unroll
      for (int i = 0; i < KS; ++i)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const uint8_t* at = smem + S::kQ + (g * D + 16 * i + 8 * h + 2 * t) * 2;
          qa[i][h] = *reinterpret_cast<const uint32_t*>(at);
          if (PREP) ql[PREP ? i : 0][h] = *reinterpret_cast<const uint32_t*>(at + G * D * 2);
        }
    }
  }
  float m_run[2] = {-INFINITY, -INFINITY}, l_run[2] = {0.f, 0.f};
  float o[KS][4];
#pragma unroll
  for (int j = 0; j < KS; ++j) o[j][0] = o[j][1] = o[j][2] = o[j][3] = 0.f;
  float* sc = scores + (warp * kBlkKeys + g) * G + 2 * t;
  // ldmatrix: lanes 0-7 / 8-15 / 16-23 / 24-31 give the rows of keys 0-7 / 8-15 / 0-7 / 8-15 at chunks 2 i / same / 2 i + 1 /
  // same of K; of V (transposed) keys 0-7 / 0-7 / 8-15 / 8-15 at chunks 2 j / 2 j + 1 / same / same
  const uint32_t k_at = ((lane & 7) + ((lane >> 3) & 1) * 8) * 128, k_x = ((lane >> 4) ^ (lane & 7)) << 4;
  const uint32_t v_at = ((lane & 7) + (lane >> 4) * 8) * 128, v_x = (((lane >> 3) & 1) ^ (lane & 7)) << 4;
  int n = 0;
#pragma unroll 1
  for (int blk = first; blk < nblk; blk += stride, ++n) {
    const Blk cur = blk_of<D>(p, u, blk, count, new_slot);
    const uint32_t sK = stage, sV = stage + S::kBlk / 2;
    cp_async_wait<1>();  // K has landed, V may not
    __syncwarp();
    if (FUSED && cur.new_row >= 0) {  // this warp has the new token: its key goes to the ring
      if (lane < D / 8) {
        uint4* at = reinterpret_cast<uint4*>(smem + (sK - smem_addr(smem)) + swz<D>(cur.new_row, lane));
        if (PREP) *at = *reinterpret_cast<const uint4*>(prepared + 8 * lane);
        *reinterpret_cast<uint4*>(put_k + 8 * lane) = *at;
      }
      __syncwarp();
    }
    // ---- S^T = K Q^T, two products of 16 keys, each in two accumulator chains: the even and the odd steps, or (PREP) the
    // queries' high and low parts ----
    float sa[2][2][4];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int e = 0; e < 4; ++e) sa[h][0][e] = sa[h][1][e] = 0.f;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
      for (int i = 0; i < KS; ++i) {
        uint32_t a0, a1, a2, a3;
        ldsm_x4(sK + k_at + h * 2048 + (i >> 2) * (kBlkKeys * 128) + (((i & 3) * 32) ^ k_x), a0, a1, a2, a3);
        wmma(sa[h][PREP ? 0 : i & 1], a0, a1, a2, a3, qa[i][0], qa[i][1]);
        if (PREP) wmma(sa[h][1], a0, a1, a2, a3, ql[PREP ? i : 0][0], ql[PREP ? i : 0][1]);
      }
    }
    __syncwarp();  // the stage's K is read
    request_k(blk + stride, nblk, count, new_slot, newk);
    float v[2][4];  // keys 16 h + g (0, 1) and + 8 (2, 3), heads 2 t and 2 t + 1
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        v[h][e] = sa[h][0][e] + sa[h][1][e];
        // An infinite key has its score from the high part: the low one has any sign, or is 0, and their sum would be NaN.
        if (PREP && !(fabsf(sa[h][0][e]) < INFINITY)) v[h][e] = sa[h][0][e];
      }
    if (cur.rows < kBlkKeys) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        if (16 * h + g >= cur.rows) v[h][0] = v[h][1] = -INFINITY;
        if (16 * h + 8 + g >= cur.rows) v[h][2] = v[h][3] = -INFINITY;
      }
    }
    if (2 * t < G) {
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          if (G == 1) sc[16 * h + 8 * r] = v[h][2 * r];
          else *reinterpret_cast<float2*>(sc + (16 * h + 8 * r) * G) = make_float2(v[h][2 * r], v[h][2 * r + 1]);
        }
    }
    sc += NW * kBlkKeys * G;
    __syncwarp();
    // ---- online softmax.  The maximum over the keys is only taken where some key is above the one
    // so far. ----
    float mx[2];
#pragma unroll
    for (int e = 0; e < 2; ++e)
      mx[e] = fmaxf(fmaxf(v[0][e], v[0][2 + e]), fmaxf(v[1][e], v[1][2 + e]));
    const bool up0 = mx[0] > m_run[0], up1 = mx[1] > m_run[1];
    if (__any_sync(0xffffffffu, up0 || up1)) {
#pragma unroll
      for (int off = 4; off < 32; off <<= 1) {
        mx[0] = fmaxf(mx[0], __shfl_xor_sync(0xffffffffu, mx[0], off));
        mx[1] = fmaxf(mx[1], __shfl_xor_sync(0xffffffffu, mx[1], off));
      }
      float alpha[2];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const bool up = mx[e] > m_run[e];
        alpha[e] = up ? ex2((m_run[e] - mx[e]) * p.scale_log2) : 1.f;
        if (up) m_run[e] = mx[e];
        l_run[e] *= alpha[e];
      }
#pragma unroll
      for (int j = 0; j < KS; ++j) {
        o[j][0] *= alpha[0];
        o[j][1] *= alpha[1];
        o[j][2] *= alpha[0];
        o[j][3] *= alpha[1];
      }
    }
    uint32_t pb[2][2];
    {
      float pr[2][4];
      const float m0 = finite_max(m_run[0]), m1 = finite_max(m_run[1]);
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int e = 0; e < 4; ++e) pr[h][e] = ex2((v[h][e] - (e & 1 ? m1 : m0)) * p.scale_log2);
      l_run[0] += (pr[0][0] + pr[0][2]) + (pr[1][0] + pr[1][2]);
      l_run[1] += (pr[0][1] + pr[0][3]) + (pr[1][1] + pr[1][3]);
      // P^T as the B operand: packed to bf16 (outputs are bf16; the sums are not rounded) and transposed
      __syncwarp();  // converged for movmatrix
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        pb[h][0] = movmatrix_trans(pack_bf16_rn(pr[h][0], pr[h][1]));
        pb[h][1] = movmatrix_trans(pack_bf16_rn(pr[h][2], pr[h][3]));
      }
    }
    cp_async_wait<1>();  // V has
    __syncwarp();
    if (FUSED && cur.new_row >= 0) {  // its value too
      if (lane < D / 8)
        *reinterpret_cast<uint4*>(put_v + 8 * lane) =
            *reinterpret_cast<const uint4*>(smem + (sV - smem_addr(smem)) + swz<D>(cur.new_row, lane));
      __syncwarp();  // converged for ldmatrix
    }
    // ---- O^T += V^T P^T ----
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
      for (int j = 0; j < KS; ++j) {
        uint32_t a0, a1, a2, a3;
        ldsm_x4_trans(sV + v_at + h * 2048 + (j >> 2) * (kBlkKeys * 128) + (((j & 3) * 32) ^ v_x), a0, a1, a2, a3);
        wmma(o[j], a0, a1, a2, a3, pb[h][0], pb[h][1]);
      }
    }
    __syncwarp();  // the stage's V is read
    request_v(n + 1, blk + stride, nblk, count, new_slot, newv);
  }
  cp_async_wait<0>();  // (a bad sequence's blocks of Tier-1 were requested too)
  __syncwarp();

  // ---- the warps' states ----
#pragma unroll
  for (int off = 4; off < 32; off <<= 1) {
    l_run[0] += __shfl_xor_sync(0xffffffffu, l_run[0], off);
    l_run[1] += __shfl_xor_sync(0xffffffffu, l_run[1], off);
  }
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    const int hh = 2 * t + e;
    if (hh < G) {
      float* ow = reinterpret_cast<float*>(smem + warp * S::kBlk) + hh * DP + g;
#pragma unroll
      for (int j = 0; j < KS; ++j) {
        ow[16 * j] = o[j][e];
        ow[16 * j + 8] = o[j][2 + e];
      }
      if (g == 0) {
        merge_m[warp * 8 + hh] = m_run[e];
        merge_l[warp * 8 + hh] = l_run[e];
      }
    }
  }

  __syncthreads();
  // Every thread of the CTA has read pos (and used it); the last of the sequence's CTAs to say so advances it, in the end: the
  // answer takes a trip to L2.
  unsigned long long ticket = 0;
  if (FUSED && tid == 0) ticket = atomicAdd(p.tickets + (ORDER ? 0 : b), 1ull);

  // ---- merge: four columns of one head a thread, the warps in order ----
  constexpr int NGR = G * D / 4;
  const long long out_base = u * (G * D);
  for (int x = tid; x < NGR; x += kThreadsOfCta) {
    const int hh = (4 * x) / D, c = (4 * x) % D;
    float M = merge_m[hh];
#pragma unroll
    for (int w = 1; w < NW; ++w) M = fmaxf(M, merge_m[w * 8 + hh]);
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    float Ls = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      const float f = ex2((merge_m[w * 8 + hh] - finite_max(M)) * p.scale_log2);
      const float4 y = *reinterpret_cast<const float4*>(smem + w * S::kBlk + (hh * DP + c) * 4);
      acc.x = fmaf(f, y.x, acc.x);
      acc.y = fmaf(f, y.y, acc.y);
      acc.z = fmaf(f, y.z, acc.z);
      acc.w = fmaf(f, y.w, acc.w);
      Ls = fmaf(f, merge_l[w * 8 + hh], Ls);
    }
    if (p.cm == 1) {
      const float inv = Ls == 0.f ? 0.f : 1.f / Ls;
      *reinterpret_cast<uint2*>(p.out + out_base + hh * D + c) =
          make_uint2(pack_bf16_rn(acc.x * inv, acc.y * inv), pack_bf16_rn(acc.z * inv, acc.w * inv));
      if (c == 0) {
        fin_m[hh] = finite_max(M);
        fin_r[hh] = inv;
      }
    } else {
      *reinterpret_cast<float4*>(rec_o + hh * D + c) = acc;
      if (c == 0) {
        rec_ml[2 * hh] = M;
        rec_ml[2 * hh + 1] = Ls;
      }
    }
  }
  if (p.cm > 1) {
    // Each CTA of the cluster merges its share of the columns from its peers' records.
    cluster_sync_all();
    const uint32_t o_a = smem_addr(rec_o), ml_a = smem_addr(rec_ml);
    const int SL = (NGR + p.cm - 1) / p.cm;
    const int x1 = min((rank + 1) * SL, NGR);
    // A head's maximum and sum, and what each rank's share of it counts; all ranks' are requested at once (one after the other
    // they were 2 us of a cluster of eight).
    float f[kMaxClusterCtas];
    auto merged = [&](int hh, float& M, float& Ls) {
      float2 ml[kMaxClusterCtas];
#pragma unroll
      for (int r = 0; r < kMaxClusterCtas; ++r)
        ml[r] = r < p.cm ? ld_peer_f2(peer_smem(ml_a + 8 * hh, r)) : make_float2(-INFINITY, 0.f);
      M = ml[0].x;
#pragma unroll
      for (int r = 1; r < kMaxClusterCtas; ++r) M = fmaxf(M, ml[r].x);
      M = finite_max(M);
      Ls = 0.f;
#pragma unroll
      for (int r = 0; r < kMaxClusterCtas; ++r) {
        f[r] = ex2((ml[r].x - M) * p.scale_log2);
        Ls = fmaf(f[r], ml[r].y, Ls);
      }
    };
    for (int x = rank * SL + tid; x < x1; x += kThreadsOfCta) {
      const int hh = (4 * x) / D, c = (4 * x) % D;
      float4 y[kMaxClusterCtas];
#pragma unroll
      for (int r = 0; r < kMaxClusterCtas; ++r)
        y[r] = r < p.cm ? ld_peer_f4(peer_smem(o_a + (hh * D + c) * 4, r)) : make_float4(0.f, 0.f, 0.f, 0.f);
      float M, Ls;
      merged(hh, M, Ls);
      float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int r = 0; r < kMaxClusterCtas; ++r) {
        acc.x = fmaf(f[r], y[r].x, acc.x);
        acc.y = fmaf(f[r], y[r].y, acc.y);
        acc.z = fmaf(f[r], y[r].z, acc.z);
        acc.w = fmaf(f[r], y[r].w, acc.w);
      }
      const float inv = Ls == 0.f ? 0.f : 1.f / Ls;
      *reinterpret_cast<uint2*>(p.out + out_base + hh * D + c) =
          make_uint2(pack_bf16_rn(acc.x * inv, acc.y * inv), pack_bf16_rn(acc.z * inv, acc.w * inv));
    }
    if (tid >= kThreadsOfCta - G) {  // the heads' final maxima and sums, for the weights
      const int hh = tid - (kThreadsOfCta - G);
      float M, Ls;
      merged(hh, M, Ls);
      fin_m[hh] = M;
      fin_r[hh] = Ls == 0.f ? 0.f : 1.f / Ls;
    }
    cluster_arrive();  // this thread reads its peers' memory no more
  }
  __syncthreads();

  // ---- the weights ----
  float M[G], R[G];
#pragma unroll
  for (int h = 0; h < G; ++h) {
    M[h] = fin_m[h];
    R[h] = fin_r[h];
  }
  // Key x is row x % 32 of the block that warp x / 32 % NW took in iteration x / (32 NW).
  const int iters = nblk > rank * NW ? (nblk - rank * NW + stride - 1) / stride : 0;
  for (int x = tid; x < iters * NW * kBlkKeys; x += kThreadsOfCta) {
    const int blk = rank * NW + x / kBlkKeys % NW + x / (kBlkKeys * NW) * stride;
    const int r = x % kBlkKeys;
    const int key = (blk < p.nb1 ? blk : blk - p.nb1) * kBlkKeys + r;
    if (blk >= nblk || key >= (blk < p.nb1 ? p.k : count)) continue;
    const float* s = scores + static_cast<long long>(x) * G;
    float sum = 0.f;
#pragma unroll
    for (int h = 0; h < G; ++h) sum = fmaf(ex2((s[h] - M[h]) * p.scale_log2), R[h], sum);
    (blk < p.nb1 ? p.t1w + u * p.N : p.ring_w + u * p.W)[key] = weights[x] + sum;
  }
  if (FUSED && ORDER) {
    if (warp == 0) {
      ticket = __shfl_sync(0xffffffffu, ticket, 0);
      if (ticket + 1 == gridDim.x) {
        for (int i = lane; i < p.B; i += 32) {
          const long long x = *static_cast<volatile int64_t*>(p.pos + i);
          if (x >= 0) p.pos[i] = x + 1;
        }
        if (lane == 0) p.tickets[0] = 0ull;
      }
    }
  } else if (FUSED && tid == 0 && ticket + 1 == static_cast<unsigned long long>(p.LH) * p.cm) {
    if (!bad) p.pos[b] = pos + 1;
    p.tickets[b] = 0ull;
  }
  if (bad && tid == 0 && rank == 0) atomicOr(p.status, CMC_DEVFLAG_BAD_POS);
  if (p.cm > 1) cluster_wait();  // no peer reads this CTA's memory any more
}

// ---------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------

static long long blocks_of(const cmc_dims& m) {
  return (static_cast<long long>(m.k) + kBlkKeys - 1) / kBlkKeys + (static_cast<long long>(m.W) + kBlkKeys - 1) / kBlkKeys;
}
// Blocks that each of a unit's `warps` takes at most, and the bytes of a CTA's products and weights.
static long long iters_of(const cmc_dims& m, int warps) { return (blocks_of(m) + warps - 1) / warps; }
static size_t score_bytes(const cmc_dims& m, int cm, int nw) {
  return static_cast<size_t>(iters_of(m, cm * nw)) * nw * kBlkKeys * (m.Hq / m.Hkv + 1) * 4;
}
static bool needs_scratch(const cmc_dims& m) { return score_bytes(m, kMaxClusterCtas, kWarpsMost) > static_cast<size_t>(score_cap(m.Hq / m.Hkv)); }
static size_t weighted_ws(const cmc_dims& m) {
  const size_t units = static_cast<size_t>(m.B) * m.L * m.Hkv;
  return ws_partials_off(m.B) +
         (needs_scratch(m) ? units * kMaxClusterCtas * score_bytes(m, kMaxClusterCtas, kWarpsMost) : 0);
}

// What an SM holds of a kernel by its registers and threads, and by its shared memory.
constexpr int kSmemPerSm = 233472, kSmemReserved = 1024;

// CTAs of four warps per unit: the most that are resident together, with two blocks a warp at least (a cluster's merge
// costs more than a block: 2 units of 5 blocks 3.9 us with two CTAs, 2.5 with one); more where the unit's products would not
// go into shared memory.
static int plan_cm(const cmc_dims& m, int per_sm, int fixed_smem) {
  const long long units = static_cast<long long>(m.B) * m.L * m.Hkv;
  const size_t cap = score_cap(m.Hq / m.Hkv);
  int cm = static_cast<int>(std::max(1LL, std::min<long long>(blocks_of(m) / (2 * kWarpsMost), kMaxClusterCtas)));
  for (; cm > 1; --cm) {
    const long long smem = fixed_smem + static_cast<long long>(std::min(score_bytes(m, cm, kWarpsMost), cap)) + kSmemReserved;
    if (units * cm <= std::min<long long>(per_sm, kSmemPerSm / smem) * sm_count()) break;
  }
  while (cm < kMaxClusterCtas && score_bytes(m, cm, kWarpsMost) > cap) ++cm;
  return cm;
}

template <int D, int G, bool FUSED, bool PREP, int NW, bool ORDER>
static int per_sm_of(int* out) {
  constexpr int smem = WSmem<D, G, PREP, NW>::kScores + kScoreMost;
  auto kern = weighted_attn_kernel<D, G, FUSED, PREP, NW, ORDER>;
  static std::atomic<int> known[64];
  int dev = 0;
  int st = record_cuda_error(cudaGetDevice(&dev));
  if (st != CMC_OK) return st;
  int per_sm = (dev >= 0 && dev < 64) ? known[dev].load(std::memory_order_acquire) : 0;
  if (per_sm <= 0) {
    st = record_cuda_error(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
    if (st != CMC_OK) return st;
    st = record_cuda_error(cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, kern, 32 * NW, 0));
    if (st != CMC_OK) return st;
    if (per_sm < 1) per_sm = 1;
    if (dev >= 0 && dev < 64) known[dev].store(per_sm, std::memory_order_release);
  }
  *out = per_sm;
  return CMC_OK;
}

template <int D, int G, bool FUSED, bool PREP, int NW, bool ORDER>
static int launch_weighted_cm(WeightedParams& p, const cmc_dims& m, int cm, cudaStream_t s) {
  p.cm = cm;
  p.iters = static_cast<int>(iters_of(m, cm * NW));
  size_t bytes = score_bytes(m, cm, NW);
  const long long ctas = static_cast<long long>(m.B) * m.L * m.Hkv * cm;
  if (bytes > static_cast<size_t>(ctas <= sm_count() ? kScoreMost : score_cap(G))) bytes = 0;  // in the workspace
  else p.scratch = nullptr;
  p.prefetch = std::min({l2_prefetch_setting(), kPrefetchMost, p.iters});
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = static_cast<unsigned>(cm);
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(ctas));
  cfg.blockDim = dim3(32 * NW);
  cfg.dynamicSmemBytes = WSmem<D, G, PREP, NW>::kScores + bytes;
  cfg.stream = s;
  cfg.attrs = attr;
  cfg.numAttrs = cm > 1 ? 2 : 1;
  return record_cuda_error(cudaLaunchKernelEx(&cfg, weighted_attn_kernel<D, G, FUSED, PREP, NW, ORDER>, p));
}

// A CTA of four warps a unit, or a cluster of them; a warp a unit, or two if all of those are resident together, where there are
// more units than CTAs of four and none has more than kSoloBlocks blocks.  (us a step with rotation, four warps / one, d = 128,
// G = 4, blocks 4, 8, 12, 20:
//    512 units  10.6 / 10.7   16.9 / 15.3   22.9 / 20.1   31.4 / 29.2
//  1,024        18.2 / 13.5   28.8 / 22.2   42.8 / 29.4   58.6 / 64.8
//  2,048        31.6 / 27.7   50.4 / 44.3   77.6 / 57.5  106.1 / 107.1
//    256         6.5 /  8.7    8.3 / 18.2    9.8 / 21.9   14.7 / 27.9
// One / two, blocks 2, 6, 12, 16:
//    512         6.0 /  6.0   12.3 / 10.2   20.7 / 18.4   26.2 / 23.7
//    720         6.6 /  6.4   15.1 / 12.2   24.4 / 21.1   30.7 / 28.1
// and of 20 blocks, rings full / of different fill, four / two: 31.0 / 26.3, 12.9 / 15.7: the longest unit counts.)
// Several waves of CTAs of four warps start with the longest sequences (ORDER): ordering them, a thread a sequence, costs a CTA
// a microsecond and the prefetch before the wait, so that calls of equal lengths lose by it where clusters are used.  (us a
// launch without / with it, G = 4: 64 sequences x 8 heads of 256 + 128..2,048 keys 50.3 / 43.7, 32 + 60..1,000 25.0 / 19.5,
// 8 x 8 of 256 + 1,024..16,384 37.8 / 33.4; 64 units of 16,384 77.9 / 85.4, 512 of 6,144 246 / 250.)
template <int D, int G, bool FUSED, bool PREP>
static int launch_weighted(WeightedParams& p, const cmc_dims& m, cudaStream_t s, int* ctas) {
  int per_sm = 1;
  int st = per_sm_of<D, G, FUSED, PREP, kWarpsMost, false>(&per_sm);
  if (st != CMC_OK) return st;
  const long long units = static_cast<long long>(m.B) * m.L * m.Hkv;
  const bool brief = units > static_cast<long long>(per_sm) * sm_count() && blocks_of(m) <= kSoloBlocks;
  bool two = false;
  if (brief) {
    int per_sm2 = 1;
    st = per_sm_of<D, G, FUSED, PREP, 2, false>(&per_sm2);
    if (st != CMC_OK) return st;
    const long long smem = WSmem<D, G, PREP, 2>::kScores + static_cast<long long>(score_bytes(m, 1, 2)) + kSmemReserved;
    two = units <= std::min<long long>(per_sm2, kSmemPerSm / smem) * sm_count();
  }
  const int cm = brief ? 1 : plan_cm(m, per_sm, WSmem<D, G, PREP, kWarpsMost>::kScores);
  if (ctas) {
    *ctas = static_cast<int>(units * cm);
    return CMC_OK;
  }
  if (brief && two) return launch_weighted_cm<D, G, FUSED, PREP, 2, false>(p, m, cm, s);
  if (brief) {
    st = per_sm_of<D, G, FUSED, PREP, 1, false>(&per_sm);
    return st != CMC_OK ? st : launch_weighted_cm<D, G, FUSED, PREP, 1, false>(p, m, cm, s);
  }
  if (units * cm > static_cast<long long>(per_sm) * sm_count() && m.B > 1 && m.B <= 32 * kWarpsMost) {
    st = per_sm_of<D, G, FUSED, PREP, kWarpsMost, true>(&per_sm);
    return st != CMC_OK ? st : launch_weighted_cm<D, G, FUSED, PREP, kWarpsMost, true>(p, m, cm, s);
  }
  return launch_weighted_cm<D, G, FUSED, PREP, kWarpsMost, false>(p, m, cm, s);
}

template <bool FUSED, bool PREP>
static int dispatch_weighted(WeightedParams& p, const cmc_dims& m, cudaStream_t s, int* ctas) {
  const int G = m.Hq / m.Hkv;
  if (m.d == 128) {
    switch (G) {
      case 1: return launch_weighted<128, 1, FUSED, PREP>(p, m, s, ctas);
      case 2: return launch_weighted<128, 2, FUSED, PREP>(p, m, s, ctas);
      case 4: return launch_weighted<128, 4, FUSED, PREP>(p, m, s, ctas);
      default: return launch_weighted<128, 8, FUSED, PREP>(p, m, s, ctas);
    }
  }
  switch (G) {
    case 1: return launch_weighted<64, 1, FUSED, PREP>(p, m, s, ctas);
    case 2: return launch_weighted<64, 2, FUSED, PREP>(p, m, s, ctas);
    case 4: return launch_weighted<64, 4, FUSED, PREP>(p, m, s, ctas);
    default: return launch_weighted<64, 8, FUSED, PREP>(p, m, s, ctas);
  }
}

static int check_weighted_dims(const cmc_dims* dims) {
  int st = validate_dims(dims, true);
  if (st != CMC_OK) return st;
  const cmc_dims& m = *dims;
  const long long units = static_cast<long long>(m.B) * m.L * m.Hkv;
  if (units * m.N >= (1LL << 40) || units * m.W >= (1LL << 40)) return CMC_ERR_SHAPE;
  return CMC_OK;
}

static int run_weighted(const void* q, const void* t1k, const void* t1v, float* t1w, void* ring_k,
                        void* ring_v, float* ring_w, int64_t* pos, const void* k_new, const void* v_new,
                        const cmc_dims* dims, float scale, const cmc_qk_prep* prep, void* out,
                        void* workspace, size_t workspace_bytes, void* stream, bool fused) {
  int st = check_weighted_dims(dims);
  if (st != CMC_OK) return st;
  const cmc_dims& m = *dims;
  if (!q || !ring_k || !ring_v || !ring_w || !pos || !out) return CMC_ERR_NULL;
  if (m.k > 0 && (!t1k || !t1v || !t1w)) return CMC_ERR_NULL;
  if (fused && (!k_new || !v_new)) return CMC_ERR_NULL;
  if (!aligned16(q) || !aligned16(t1k) || !aligned16(t1v) || !aligned16(ring_k) || !aligned16(ring_v) ||
      !aligned16(out) || !aligned16(k_new) || !aligned16(v_new) ||
      ((reinterpret_cast<uintptr_t>(t1w) | reinterpret_cast<uintptr_t>(ring_w)) & 3) ||
      (reinterpret_cast<uintptr_t>(pos) & 7))
    return CMC_ERR_ALIGN;
  if (!workspace || workspace_bytes < weighted_ws(m)) return CMC_ERR_WORKSPACE;
  if (!aligned16(workspace)) return CMC_ERR_ALIGN;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  WeightedParams p;
  st = prep_params(fused ? prep : nullptr, m.d, s, &p.prep);
  if (st != CMC_OK) return st;
  // CTAs read and write in any order: what is written meets nothing else, but that a unit's output may take its queries' place (they
  // have all been read when it is stored).
  const size_t units = static_cast<size_t>(m.B) * m.L * m.Hkv, row = m.d * 2, each = static_cast<size_t>(m.B) * 8;
  const size_t bank = m.k > 0 ? units * m.N : 0, ring = units * m.W, gains = static_cast<size_t>(m.L) * m.d * 4;
  const Range heads = {q, units * (m.Hq / m.Hkv) * row}, outputs = {out, heads.bytes};
  const Range reads[] = {{t1k, bank * row}, {t1v, bank * row}, {k_new, units * row}, {v_new, units * row}, {p.prep.q_weight, gains},
                         {p.prep.k_weight, gains}, {p.prep.evicted, each}, {fused ? nullptr : ring_k, ring * row},
                         {fused ? nullptr : ring_v, ring * row}, {fused ? nullptr : pos, each}};
  const Range writes[] = {outputs, {t1w, bank * 4}, {ring_w, ring * 4}, {workspace, weighted_ws(m)}, {fused ? ring_k : nullptr, ring * row},
                          {fused ? ring_v : nullptr, ring * row}, {fused ? pos : nullptr, each}};
  if (any_meet(writes, reads) || any_meet(writes)) return CMC_ERR_RANGE;
  for (const Range& w : writes)
    if (meet(w, heads) && !same(w, heads)) return CMC_ERR_RANGE;
  p.q = static_cast<const uint16_t*>(q);
  p.t1k = static_cast<const uint16_t*>(t1k);
  p.t1v = static_cast<const uint16_t*>(t1v);
  p.t1w = t1w;
  p.ring_k = static_cast<uint16_t*>(ring_k);
  p.ring_v = static_cast<uint16_t*>(ring_v);
  p.ring_w = ring_w;
  p.pos = pos;
  p.k_new = static_cast<const uint16_t*>(k_new);
  p.v_new = static_cast<const uint16_t*>(v_new);
  p.out = static_cast<uint16_t*>(out);
  char* ws = static_cast<char*>(workspace);
  p.status = reinterpret_cast<uint32_t*>(ws);
  p.tickets = reinterpret_cast<unsigned long long*>(ws + kWsHeader);
  p.scratch = reinterpret_cast<float*>(ws + ws_partials_off(m.B));
  p.B = m.B; p.L = m.L; p.Hkv = m.Hkv; p.N = m.N; p.k = m.k; p.W = m.W; p.LH = m.L * m.Hkv;
  p.cm = 1;
  p.nb1 = (m.k + kBlkKeys - 1) / kBlkKeys;
  const float sc = scale > 0.f ? scale : 1.0f / sqrtf(static_cast<float>(m.d));
  p.scale_log2 = sc * 1.4426950408889634f;
  if (!fused) return dispatch_weighted<false, false>(p, m, s, nullptr);
  if (p.prep.rope || p.prep.q_weight || p.prep.k_weight) return dispatch_weighted<true, true>(p, m, s, nullptr);
  return dispatch_weighted<true, false>(p, m, s, nullptr);
}

}  // namespace cmc

extern "C" {

size_t cmc_decode_attn_weighted_workspace_size(const cmc_dims* dims) {
  if (cmc::check_weighted_dims(dims) != CMC_OK) return 0;
  return cmc::weighted_ws(*dims);
}

int cmc_decode_attn_weighted_plan(const cmc_dims* dims, int fused, int* ctas) {
  int st = cmc::check_weighted_dims(dims);
  if (st != CMC_OK) return st;
  if (!ctas) return CMC_ERR_NULL;
  cmc::WeightedParams p;
  return fused ? cmc::dispatch_weighted<true, false>(p, *dims, nullptr, ctas)
               : cmc::dispatch_weighted<false, false>(p, *dims, nullptr, ctas);
}

int cmc_two_tier_decode_attn_weighted(const void* q, const void* tier1_k, const void* tier1_v,
                                      float* tier1_weight, const void* ring_k, const void* ring_v,
                                      float* ring_weight, const int64_t* pos, const cmc_dims* dims,
                                      float scale, void* out, void* workspace, size_t workspace_bytes,
                                      void* stream) {
  return cmc::run_weighted(q, tier1_k, tier1_v, tier1_weight, const_cast<void*>(ring_k),
                           const_cast<void*>(ring_v), ring_weight, const_cast<int64_t*>(pos), nullptr,
                           nullptr, dims, scale, nullptr, out, workspace, workspace_bytes, stream, false);
}

int cmc_decode_step_weighted(const void* q, const void* tier1_k, const void* tier1_v, float* tier1_weight,
                             void* ring_k, void* ring_v, float* ring_weight, int64_t* pos,
                             const void* k_new, const void* v_new, const cmc_dims* dims, float scale,
                             const cmc_qk_prep* prep, void* out, void* workspace, size_t workspace_bytes,
                             void* stream) {
  return cmc::run_weighted(q, tier1_k, tier1_v, tier1_weight, ring_k, ring_v, ring_weight, pos, k_new,
                           v_new, dims, scale, prep, out, workspace, workspace_bytes, stream, true);
}

}  // extern "C"
