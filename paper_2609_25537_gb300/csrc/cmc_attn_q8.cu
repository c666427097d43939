// Decode attention over the two-tier cache held in 8 bits (format: cmc_q8.cuh),
// alone and fused with the append of the step's token.
//
// One CTA per unit (sequence, layer, KV head), or a cluster of cm CTAs; a unit's blocks of
// 32 keys, which are the format's blocks with one power of two for K and one for V, are
// ceil(k / 32) of Tier-1, then those of the ring's live slots, and warp w of the unit's 4 cm
// takes blocks w, w + 4 cm, ...  The four warps of a CTA have little to do with each
// other: each loads its own blocks into its own ring of stages, a TMA box of 32 rows of
// K and of V each (8 KB at d = 128), and refills a stage as soon as it is done with it, so
// there is no producer and no barrier between loading and computing but the stage's
// "full" one.  The first blocks do not depend on pos and are requested before it is
// known.  In the end the warps' states are merged in shared memory, the CTAs' of a
// cluster in distributed shared memory (as in cmc_attn.cu).
//
// Many short units take a warp each instead, which needs no merge (SOLO).
//
// A grid may have many more CTAs than are resident: the hardware gives a free place to the
// next unit, and what one CTA waits for (its first bytes, its merge) the others on the SM
// cover.  The depth of the rings of stages sets how many those are: see plan_q8.  Rings of
// different fill are evened out by taking the longest sequences first (p.order): a long
// unit that starts last sets the time of the launch.  512 units of 312 to 2,304 keys 24.8 us (in the order of
// the batch 30.9), 1,024 48.8; full ones 48.9 and 97.8, which in batch order and the best variant take
// 47.7 and 90.0: each CTA reads all positions, and sorts, before it knows its unit.  (Sharing out
// the live blocks of all units evenly over the warps of one wave, with a kernel to merge the
// cut units, cost 10 us a launch: 312 units of 256 + 2,048 keys 37 us, 304 of them here 28.)
//
// Both products run on fp16 operands with fp32 accumulation (mma.sync m16n8k16): the
// codes are converted to fp16 in registers, exactly, one instruction for two.  (mma.sync
// takes e4m3 operands too; the kernel then executed 672 instructions a block by the counters,
// 420 so, and was bound by them: 512 units of 312 to 2,304 keys 49.7 us, 30.8 so.)
//   S^T = K Q^T     16 keys as the rows, the G query heads as the columns, d in k-steps of 16
//   O^T += V^T P^T  16 rows of the head dimension, the heads, the block's 32 keys in two k-steps
//   q    is multiplied by a power of two so that its head's largest element is in (224, 448].  fp16
//        holds a bf16 element exactly down to 2^-22 of that, and is off by 2^-33 of it below.
//   p    is multiplied by V's power of two and divided by O's unit, times 2^15.
// K's power of two joins the softmax scale; with it, a score s is that of 2^s.  V's, 2^(c - 127), changes from
// block to block: each head's O is kept in units of 2^(U - 127), U a whole number, and p is 2^(s + c - U).  U is
// raised, and O rescaled, where a block has an s + c above it, so that p never exceeds 1; and lowered where
// all of a block's lie more than ten below, so that p has eleven significant bits down to 2^-19 of the block's
// largest and is off by 2^-30 of that below (2^-28 and 2^-39 where U is the block's own).  U stays within 64 of the
// largest that it has been, for O's sake: of tokens 2^-64 and less of the head's largest p 2^c
// the smaller values are lost.
// The sum l that divides has nothing to do with V: it takes the same p, times 2^(U - c), in units of 2^m, m the
// maximum, and so that these stay within fp32, p is taken relative to no more than 2^44 times its maximum (it
// is 0 in fp16 either way).  Scores s may be up to 2^23: beyond, fp32 holds no whole numbers next to them.
//
// The order of d in a k-step is free: lane t of a quad has the bytes 4 t .. 4 t + 3 of a
// 16-byte chunk of a key's codes, and they are its four k.  So is the order of the keys, which
// P^T's way from the accumulators of S^T to the B operand (movmatrix) fixes for the row
// addresses of V; rows 8 .. 15 of a product are keys 8 + (r ^ 4), so that eight
// consecutive rows of V lie in eight different bank groups.
#include <algorithm>
#include <atomic>

#include "cmc_attn.cuh"
#include "cmc_q8.cuh"

namespace cmc {

struct Q8Maps {
  CUtensorMap t1, ring;  // [2 units, T, d] bytes, box 2 x 32 rows
};

struct AttnQ8Params : AttnParams {  // t1k, t1v, ring_k, ring_v, idx and the tiles of cmc_attn.cu are not used
  uint8_t* ring_kv;           // [B, L, Hkv, 2, W, d]
  uint8_t* ring_scales;       // [B, L, Hkv, 2, ringS]
  const uint8_t* t1_scales;   // [B, L, Hkv, 2, t1S]
  int ringS, t1S;
  int units;
  int nb1, nb2;               // blocks of Tier-1, and of the whole ring
  int rope;                   // rotate q and the new key (fused step)
  int order;                  // units of the longest sequences first
};                            // cm: CTAs per unit

// Shared memory of a CTA: the query in fp16, its heads' factors, the rotated new key, the stages'
// powers of two, the warps' maxima and sums, what a cluster's peers send; then,
// 1,024-byte aligned, the stages.
template <int D, int G, int NST, bool SOLO>
struct Q8Smem {
  static constexpr int kV = kQ8Block * D;
  static constexpr int kStage = 2 * kQ8Block * D;
  static constexpr int kUnits = SOLO ? kWarps : 1;          // units of the CTA
  static constexpr int kQ = 0;                              // [unit][G][D] fp16
  static constexpr int kQs = kQ + kUnits * G * D * 2;       // [unit][8] fp32
  static constexpr int kKnew = kQs + kUnits * 32;           // [unit][D] fp32
  static constexpr int kScale = kKnew + kUnits * D * 4;     // [warp][NST][2] words
  static constexpr int kMl = kScale + kWarps * NST * 8;     // [warp][8 maxima, 8 sums, 8 units]
  static constexpr int kRecv = kMl + kWarps * 96;           // groups of 16 bytes, rank by rank
  static constexpr int kRecvMl = kRecv + (G * D / 4 + kMaxClusterCtas - 2) * 16;
  static constexpr int kSmall = SOLO ? kMl : kRecvMl + kMaxClusterCtas * G * 8;
  static constexpr int kBytes = kSmall + 1008 + kWarps * NST * kStage;
  static_assert(kRecv % 16 == 0, "written by 16 bytes");
};

// Offset of 16-byte chunk c of row r of a stage's K or V: TMA's 128-byte swizzle, or the
// 64-byte one for rows of 64 codes.
template <int D>
__device__ __forceinline__ uint32_t swz8(int r, int c) {
  return static_cast<uint32_t>(r * D + (D == 128 ? (c ^ (r & 7)) << 4 : (c ^ ((r >> 1) & 3)) << 4));
}

__device__ __forceinline__ void tma_box3_hint(uint32_t dst, const CUtensorMap* map, int row, int unit2,
                                              uint64_t* bar, uint64_t policy) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cta.global.tile.mbarrier::complete_tx::bytes.L2::cache_hint"
      " [%0], [%1, {%2, %3, %4}], [%5], %6;\n" ::"r"(dst),
      "l"(map), "r"(0), "r"(row), "r"(unit2), "r"(smem_addr(bar)), "l"(policy)
      : "memory");
}
__device__ __forceinline__ void tma_box3_prefetch(const CUtensorMap* map, int row, int unit2) {
  asm volatile("cp.async.bulk.prefetch.tensor.3d.L2.global.tile [%0, {%1, %2, %3}];\n" ::"l"(map), "r"(0),
               "r"(row), "r"(unit2)
               : "memory");
}

// 32 x 16 bytes, transposed: lane i gives the address of row i; r0 / r1 hold column
// i/4 / i/4 + 8 of rows 4 (i%4) .. + 3, r2 and r3 of rows 16 + those.
__device__ __forceinline__ void ldsm_b8_t(uint32_t addr, uint32_t& r0, uint32_t& r1, uint32_t& r2,
                                          uint32_t& r3) {
  asm volatile("ldmatrix.sync.aligned.m16n16.x2.trans.shared.b8 {%0,%1,%2,%3}, [%4];\n"
               : "=r"(r0), "=r"(r1), "=r"(r2), "=r"(r3)
               : "r"(addr));
}

// C[16x8] += A[16x16] B[16x8], fp16 inputs, fp32 accumulators.
__device__ __forceinline__ void mma_f16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                        uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, "
      "{%8,%9}, {%0,%1,%2,%3};\n"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_f16_zero(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                             uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, "
      "{%8,%9}, {%10,%10,%10,%10};\n"
      : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;\n" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

// Stands for minus infinity where differences of two of them are taken.
constexpr float kNone = -3e38f;

// Live blocks of a unit whose sequence's state is sq.
__device__ __forceinline__ int live_blocks(const AttnQ8Params& p, const SeqState& sq) {
  return sq.bad ? 0 : p.nb1 + (sq.count + kQ8Block - 1) / kQ8Block;
}

// Half a row of the new token each for lanes 0-15 (K) and 16-31 (V): d / 16 neighbouring elements.
// (Plain loads, here and below: the launch before may still have been writing the rows when this one began,
// which the read-only path does not allow for.)
template <int D>
__device__ __forceinline__ uint4 load_new(const AttnQ8Params& p, int u, int lane) {
  const uint16_t* row = (lane < 16 ? p.k_new : p.v_new) + static_cast<long long>(u) * D + (lane & 15) * (D / 16);
  if (D == 128) return *reinterpret_cast<const uint4*>(row);
  const uint2 w = *reinterpret_cast<const uint2*>(row);
  return make_uint4(w.x, w.y, 0u, 0u);
}

// A lane's E = d / 32 neighbouring elements of a row, and their values.
template <int E>
__device__ __forceinline__ uint2 load_part(const uint16_t* row, int lane) {
  if (E == 4) return reinterpret_cast<const uint2*>(row)[lane];
  return make_uint2(reinterpret_cast<const uint32_t*>(row)[lane], 0u);
}
template <int E>
__device__ __forceinline__ void unpack_part(const uint2& w, float (&x)[E]) {
  x[0] = bf16lo_to_f32(w.x);
  x[1] = bf16hi_to_f32(w.x);
  if (E == 4) {
    x[E - 2] = bf16lo_to_f32(w.y);
    x[E - 1] = bf16hi_to_f32(w.y);
  }
}
// Rotates a row held by a warp in parts: element c pairs with c +- d/2, the same of lane ^ 16.
template <int E>
__device__ __forceinline__ void rotate_part(float (&x)[E], const float2 (&cs)[E], int lane) {
  const float sg = lane < 16 ? -1.f : 1.f;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const float y = __shfl_xor_sync(0xffffffffu, x[e], 16);
    x[e] = fmaf(x[e], cs[e].x, sg * y * cs[e].y);
  }
}

// The rare parts of an append, out of line: the code that a launch runs through once is what it waits for
// most (its instructions come from L2), so what is not run should not lie in between either.  Rare
// for a unit, they set the time of most launches, which have some units that take them (1,216 units
// of 6 blocks 14.5 us, 13.5 where none does, and 11.9 without an append).
// A lane has 16-byte chunk lane % (d / 16) of every (512 / d)th row of a block.
// The largest values that the block's other tokens hold in K and in V (fp32 bits).
template <int D>
static __device__ __noinline__ uint2 block_held(const uint8_t* stage, uint32_t others, int lane, int kc, int vc) {
  constexpr int CPR = D / 16;
  uint32_t mk = 0u, mv = 0u;
#pragma unroll 2
  for (int row = lane / CPR; row < kQ8Block; row += 32 / CPR) {
    const uint8_t* at = stage + swz8<D>(row, lane % CPR);
    if ((others >> row) & 1u) {
      mk = max_codes16(mk, *reinterpret_cast<const uint4*>(at));
      mv = max_codes16(mv, *reinterpret_cast<const uint4*>(at + kQ8Block * D));
    }
  }
  return make_uint2(__reduce_max_sync(0xffffffffu, held_bits(mk, kc)),
                    __reduce_max_sync(0xffffffffu, held_bits(mv, vc)));
}
// The block's other tokens' codes of K or V for another power of two, in the stage and in the ring.
template <int D>
static __device__ __noinline__ void block_recode(uint8_t* rows, uint8_t* ring_row0, uint32_t others, int lane,
                                                 int c_old, int c) {
  constexpr int CPR = D / 16;
  const Recode f = recode_by(c_old, c);
#pragma unroll 2
  for (int row = lane / CPR; row < kQ8Block; row += 32 / CPR) {
    if ((others >> row) & 1u) {
      uint4* at = reinterpret_cast<uint4*>(rows + swz8<D>(row, lane % CPR));
      const uint4 y = recode16(*at, f);
      *at = y;
      *reinterpret_cast<uint4*>(ring_row0 + row * D + lane % CPR * 16) = y;
    }
  }
}

// The new token in its block: the token's codes over the stale ones, in the stage and in
// the ring; the block's other codes too where its power of two changes.  Half a warp
// each for K and V (`fresh`: load_new's; knew: the rotated key).  r: the token's row; `others`: the block's rows
// that hold another token; slot: its ring slot; kc, vc: the block's bytes.  (The rules
// are window_append_q8_kernel's.)
template <int D>
__device__ __forceinline__ void patch_block(const AttnQ8Params& p, uint8_t* stage, int u, int r, int slot,
                                            uint32_t others, const uint4& fresh, const float* knew, int& kc,
                                            int& vc, int lane) {
  constexpr int E = D / 16;  // elements a lane has of its row
  const int half = lane >> 4;
  float x[8];
  unpack8(fresh, x);
  if (p.rope && half == 0) {
#pragma unroll
    for (int e = 0; e < E; e += 4) {
      const float4 y = *reinterpret_cast<const float4*>(knew + (lane & 15) * E + e);
      x[e] = y.x; x[e + 1] = y.y; x[e + 2] = y.z; x[e + 3] = y.w;
    }
  }
  uint32_t top = 0u;
#pragma unroll
  for (int e = 0; e < E; ++e) top = max(top, finite_bits(x[e]));
#pragma unroll
  for (int off = 1; off < 16; off <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, off));
  const long long uv = 2LL * u;
  uint8_t* ring_k = p.ring_kv + (uv * p.W + slot - r) * D;  // the block's first row
  uint8_t* ring_v = ring_k + static_cast<long long>(p.W) * D;
  const int c_old = half ? vc : kc;
  int c = max(block_code(top), c_old);
  if ((slot & (kQ8Block - 1)) == 0) {
    const uint2 held = block_held<D>(stage, others, lane, kc, vc);
    c = block_code(max(top, half ? held.y : held.x));
  }
  const int kc_old = kc, vc_old = vc;
  kc = __shfl_sync(0xffffffffu, c, 0);
  vc = __shfl_sync(0xffffffffu, c, 16);
  if (kc != kc_old) block_recode<D>(stage, ring_k, others, lane, kc_old, kc);
  if (vc != vc_old) block_recode<D>(stage + kQ8Block * D, ring_v, others, lane, vc_old, vc);
  const float f = code_factor(c);
  uint8_t* at = stage + half * (kQ8Block * D);
  uint8_t* to = (half ? ring_v : ring_k) + static_cast<long long>(r) * D + (lane & 15) * E;
  const uint32_t w0 = encode4(x[0], x[1], x[2], x[3], f);
  if (D == 128) {
    const uint2 w = make_uint2(w0, encode4(x[4], x[5], x[6], x[7], f));
    *reinterpret_cast<uint2*>(at + swz8<D>(r, (lane & 15) >> 1) + (lane & 1) * 8) = w;
    *reinterpret_cast<uint2*>(to) = w;
  } else {
    *reinterpret_cast<uint32_t*>(at + swz8<D>(r, (lane & 15) >> 2) + (lane & 3) * 4) = w0;
    *reinterpret_cast<uint32_t*>(to) = w0;
  }
  if ((lane & 15) == 0 && c != c_old) p.ring_scales[(uv + half) * p.ringS + slot / kQ8Block] = static_cast<uint8_t>(c);
  __syncwarp();
}

// The units that a warp which gave up leaves alone are counted all the same, so that the counters come back
// to zero: u, u + hop, ...
static __device__ __noinline__ void count_left_units(unsigned long long* tickets, int64_t* pos, int u, int hop, int units,
                                                     int LH) {
  for (; u < units; u += hop) {
    const int b = u / LH;
    if (atomicAdd(tickets + b, 1ull) + 1 != static_cast<unsigned long long>(LH)) continue;
    const long long last = *static_cast<volatile int64_t*>(pos + b);  // all others have read it
    if (last >= 0) pos[b] = last + 1;
    tickets[b] = 0ull;
  }
}

// SOLO: a unit per warp, four a CTA, and no barrier but the warp's; the warp goes on with the unit
// gridDim x 4 after its own, whose query, position and first blocks are then already on
// their way.
// Registers: three CTAs an SM take 168 a thread (two of them with 168 instead of 200 spill: 2,048 units of 640
// keys 56 us and 54), and the fused ones spill 32 to 44 bytes; with d = 64 four SOLO CTAs fit with 128, of which
// the fused ones spill 40 to 64.
template <int D, int G, bool FUSED, int NST, bool SOLO>
__global__ void __maxnreg__(SOLO ? (D == 64 ? 128 : 240) : NST == 2 ? 168 : 200)
attn_q8_kernel(const __grid_constant__ Q8Maps maps, const AttnQ8Params p) {
  using S = Q8Smem<D, G, NST, SOLO>;
  constexpr int KS = D / 16;      // k-steps of the Q K^T product, m-tiles of O^T
  constexpr int E = D / 32;       // elements of a row a lane has
  constexpr int NGR = G * D / 4;  // groups of four rows of the head dimension of a unit's output
  extern __shared__ __align__(16) uint8_t smem[];
  __shared__ __align__(8) uint64_t full_bar[kWarps][NST];
  __shared__ __align__(8) uint64_t recv_bar;  // clusters: the peers' stores
  __shared__ int s_left[kWarps];              // where the warps left their outputs
  __shared__ long long s_pos[kWarps];
  __shared__ __align__(16) int s_live[kThreads];  // p.order: the sequences' lengths
  __shared__ int s_seq;                           // and the CTA's sequence
  __shared__ bool s_last;                         // fused: the last of the CTAs that tickets count

  const int tid = threadIdx.x;
  const int lane = tid & 31;
  const int warp = tid >> 5;
  const uintptr_t small_end = reinterpret_cast<uintptr_t>(smem + S::kSmall);
  uint8_t* stages = reinterpret_cast<uint8_t*>((small_end + 1023) & ~uintptr_t(1023)) + warp * (NST * S::kStage);
  uint8_t* scale_words = smem + S::kScale + warp * (NST * 8);
  constexpr int HPW = SOLO ? G : (G + kWarps - 1) / kWarps;  // heads whose query a warp converts:
  constexpr int HSTEP = SOLO ? 1 : kWarps;                   // h0, h0 + HSTEP, ...
  const int h0 = SOLO ? 0 : warp;
  uint8_t* q_rows = smem + S::kQ + (SOLO ? warp * (G * D * 2) : 0);
  float* knew = reinterpret_cast<float*>(smem + S::kKnew) + (SOLO ? warp * D : 0);
  float* q_factor = reinterpret_cast<float*>(smem + S::kQs) + (SOLO ? warp * 8 : 0);
  uint64_t* full = full_bar[warp];

  const int cm = SOLO ? 1 : p.cm;
  int u = SOLO     ? static_cast<int>(blockIdx.x) * kWarps + warp
          : cm > 1 ? static_cast<int>(cluster_id())
                   : static_cast<int>(blockIdx.x);
  const int hop = static_cast<int>(gridDim.x) * kWarps;  // SOLO: to the warp's next unit
  const int rank = cm > 1 ? static_cast<int>(cluster_ctarank()) : 0;
  // the warp's first block, and their distance; which thread speaks for the unit
  const int g0 = SOLO ? 0 : rank * kWarps + warp, step = SOLO ? 1 : cm * kWarps;
  const bool first_thread = SOLO ? lane == 0 : tid == 0;
  const int nb_all = p.nb1 + p.nb2;
  int b = static_cast<int>(static_cast<unsigned>(u) / static_cast<unsigned>(p.LH));  // sequence

  if (lane == 0) {
    for (int s = 0; s < NST; ++s) mbar_init(&full[s], 1);  // lane 0's arrive (plus tracked cp.async arrivals)
    if (SOLO || warp == 0) attn_abort = 0;
    if (warp == 1 && cm > 1) {  // the groups this CTA finishes and the heads' (max, sum), from each rank
      const int mine = min(max(NGR - rank * p.slice, 0), p.slice);
      mbar_init(&recv_bar, 1);
      mbar_arrive_expect_tx(&recv_bar, static_cast<uint32_t>(cm * (mine * 16 + G * 8)) + p.stall_tx);
    }
    asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
    prefetch_map((warp & 1) && p.k > 0 ? &maps.t1 : &maps.ring);
  }
  if (SOLO) {
    __syncwarp();
    if (u >= p.units) return;
  } else {
    __syncthreads();
  }
  if (cm > 1) cluster_arrive();  // waited for before the first store into a peer
  // Before the grid dependency wait: the first blocks into L2.
  if (lane == 0 && !p.order) {
#pragma unroll 1
    for (int i = 0, j = g0; i < p.l2_prefetch && j < nb_all; ++i, j += step)
      tma_box3_prefetch(j < p.nb1 ? &maps.t1 : &maps.ring, (j < p.nb1 ? j : j - p.nb1) * kQ8Block, 2 * u);
  }
  unsigned long long turns[E] = {};  // rotary frequencies of the lane's elements
  if (FUSED && p.rope) {
    const unsigned long long* f = p.rope_slot >= 0 ? g_rope_tables[p.rope_slot] : p.rope_turns;
#pragma unroll
    for (int e = 0; e < E; ++e) turns[e] = f[(lane & 15) * E + e];
  }
  asm volatile("griddepcontrol.wait;\n" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");
  if (!SOLO && p.order) {
    // The unit of place u / LH in the sequences' order by length, the longest first.  All CTAs see the
    // same positions, which the last of them advances in the end.
    int mine = -2;
    if (tid < p.B) {
      const long long x = ld_pos(p, tid);
      mine = static_cast<int>(x < 0 ? -1 : x < p.W ? x : p.W);
    }
    s_live[tid] = mine;
    __syncthreads();
    if (tid < p.B) {
      int place = 0;
#pragma unroll 4
      for (int i = 0; i < p.B; i += 4) {
        const int4 x = *reinterpret_cast<const int4*>(s_live + i);
        place += (x.x > mine || (x.x == mine && i < tid)) + (x.y > mine || (x.y == mine && i + 1 < tid)) +
                 (x.z > mine || (x.z == mine && i + 2 < tid)) + (x.w > mine || (x.w == mine && i + 3 < tid));
      }
      if (place == b) s_seq = tid;
    }
    __syncthreads();
    u += (s_seq - b) * p.LH;
    b = s_seq;
  }

  // blocks of the warp, as far as known before pos
  int n_run = SOLO ? nb_all : g0 < nb_all ? (nb_all - g0 + step - 1) / step : 0;
  int jn = g0, un = u;  // the next to request, and its unit
  const uint8_t* t1_s;  // that unit's powers of two: the rows of lane 0 (K) and lane 1 (V)
  const uint8_t* ring_s;
  auto cursor_unit = [&](int x) {
    un = x;
    t1_s = p.t1_scales + (2LL * x + (lane & 1)) * p.t1S;
    ring_s = p.ring_scales + (2LL * x + (lane & 1)) * p.ringS;
  };
  cursor_unit(u);
  // Requests the warp's next block into stage s: the codes by TMA, the two words that hold its
  // powers of two by lanes 0 and 1.  Called by the whole warp, converged.
  auto request = [&](int s) {
    const bool t1 = jn < p.nb1;
    const int jj = t1 ? jn : jn - p.nb1;
    if (lane < 2) {
      cp_async_4(smem_addr(scale_words + s * 8 + 4 * lane), (t1 ? t1_s : ring_s) + (jj & ~3), 4u);
      mbar_arrive_cp_async(&full[s]);
    }
    __syncwarp();
    if (lane == 0) {
      mbar_arrive_expect_tx(&full[s], S::kStage + p.stall_tx);
      tma_box3_hint(smem_addr(stages + s * S::kStage), t1 ? &maps.t1 : &maps.ring, jj * kQ8Block, 2 * un, &full[s],
                    policy_evict_first());
    }
    jn += step;
  };
  int issued = 0;
#pragma unroll 1
  for (; issued < NST && issued < n_run; ++issued) request(issued);
  // SOLO: stages on their way or unread, the next to fill, the blocks of unit `un` to request
  int fly = issued, fill = issued == NST ? 0 : issued, rn = n_run;
  int s = 0;           // stage
  uint32_t phase = 0;  // its parity

  // A unit's position, query (warp w takes heads w and w + 4, a lane E neighbouring elements) and new rows.
  long long pos = ld_pos(p, b);
  uint2 qw[HPW], kw = make_uint2(0u, 0u);
  uint4 fresh = make_uint4(0u, 0u, 0u, 0u), fresh_next = fresh;
  auto load_unit = [&](int x, uint4& rows) {
#pragma unroll
    for (int h = 0; h < HPW; ++h)
      if (h0 + HSTEP * h < G) qw[h] = load_part<E>(p.q + (static_cast<long long>(x) * G + h0 + HSTEP * h) * D, lane);
    if (FUSED) rows = load_new<D>(p, x, lane);
    if (FUSED && p.rope && (SOLO || warp == kWarps - 1))
      kw = load_part<E>(p.k_new + static_cast<long long>(x) * D, lane);
  };
  load_unit(u, fresh);
#pragma unroll 1
  do {  // SOLO: the warp's units
    // ---- the query, while the first blocks are on their way, and the new key ----
    float x[HPW][E], kx[E];
#pragma unroll
    for (int h = 0; h < HPW; ++h)
      if (h0 + HSTEP * h < G) unpack_part<E>(qw[h], x[h]);
    if (FUSED && p.rope) unpack_part<E>(kw, kx);
    const SeqState sq = seq_state<FUSED>(p, pos);
    unsigned long long ticket = 0;
    long long pos_next = 0;  // SOLO: what the next unit starts with
    if (SOLO && u + hop < p.units) {
      pos_next = ld_pos(p, static_cast<int>(static_cast<unsigned>(u + hop) / static_cast<unsigned>(p.LH)));
      load_unit(u + hop, fresh_next);
    }
    if (first_thread && sq.bad && rank == 0 && u % p.LH == 0) atomicOr(p.status, CMC_DEVFLAG_BAD_POS);
    if (FUSED && p.rope) {
      float2 cs[E];
      const unsigned long long pp = static_cast<unsigned long long>(p.rope_offset + (sq.bad ? 0 : pos));
#pragma unroll
      for (int e = 0; e < E; ++e) cs[e] = rope_cos_sin(pp, turns[e]);
#pragma unroll
      for (int h = 0; h < HPW; ++h)
        if (h0 + HSTEP * h < G) rotate_part<E>(x[h], cs, lane);
      if (SOLO || warp == kWarps - 1) {
        rotate_part<E>(kx, cs, lane);
#pragma unroll
        for (int e = 0; e < E; ++e) knew[lane * E + e] = kx[e];
      }
    }
#pragma unroll
    for (int h = 0; h < HPW; ++h) {
      const int hh = h0 + HSTEP * h;
      if (hh >= G) break;
      float top = 0.f;  // (a NaN does not count)
#pragma unroll
      for (int e = 0; e < E; ++e) top = fmaxf(top, fabsf(x[h][e]));
      if (__any_sync(0xffffffffu, top == INFINITY)) {  // an infinity becomes NaN and does not count either
        top = 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) {
          x[h][e] = fmaf(x[h][e], 0.f, x[h][e]);
          top = fmaxf(top, fabsf(x[h][e]));
        }
      }
#pragma unroll
      for (int off = 1; off < 32; off <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, off));
      const int qc = block_code(__float_as_uint(top));
      const float f = code_factor(qc);
      uint32_t* to = reinterpret_cast<uint32_t*>(q_rows + hh * (D * 2)) + lane * (E / 2);
#pragma unroll
      for (int e = 0; e < E; e += 2) to[e / 2] = pack_f16(x[h][e] * f, x[h][e + 1] * f);
      if (lane == 0) q_factor[hh] = e8m0_to_f32(qc) * p.scale_log2;
    }
    // Every warp has pos before the count below says so, and has not only asked for it: the store waits for
    // the load.  (Nothing reads it, so it has to be volatile to be there.)
    if (FUSED && lane == 0) *static_cast<volatile long long*>(s_pos + warp) = pos;
    if (SOLO) __syncwarp();
    else __syncthreads();
    // The last to have read pos[b] advances it (in the end: the count takes a trip to L2).
    if (FUSED && first_thread) ticket = atomicAdd(p.tickets + (p.order ? 0 : b), 1ull);

    // Live blocks; those that were requested in vain hold no key.
    const int nb = live_blocks(p, sq);
    n_run = SOLO ? nb : nb > g0 ? (nb - g0 + step - 1) / step : 0;
    if (n_run < issued) n_run = issued;
    // SOLO: as many blocks of this unit and the next are requested as there are stages
    int n_next = 0;
    if (SOLO && u + hop < p.units) n_next = live_blocks(p, seq_state<FUSED>(p, pos_next));
    if (SOLO) {
      if (un != u) {
        cursor_unit(u);
        jn = 0;
      }
      rn = n_run;
    }
    auto top_up = [&]() {
#pragma unroll 1
      while (fly < NST) {
        if (jn >= rn) {
          if (un != u || n_next == 0) break;  // (no further ahead than the next unit)
          cursor_unit(u + hop);
          jn = 0;
          rn = n_next;
        }
        request(fill);
        ++fly;
        fill = fill + 1 == NST ? 0 : fill + 1;
      }
    };
    // gq = lane / 4, tq = lane % 4: a thread has columns (heads) 2 tq and 2 tq + 1 of the products
    // (heads >= G are padding: zero queries, never written out).
    const int gq = lane >> 2;
    const int tq = lane & 3;
    uint32_t qa[KS][2];  // Q^T fragments: column gq, elements 16 ks + 4 tq .. + 3
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      uint2 f = make_uint2(0u, 0u);
      if (gq < G) f = *reinterpret_cast<const uint2*>(q_rows + (gq * D + 16 * ks + 4 * tq) * 2);
      qa[ks][0] = f.x;
      qa[ks][1] = f.y;
    }
    float unit[2], unit_top[2];       // U; the largest so far
    float qs[2], m_run[2], l_run[2];  // softmax scale * log2(e) * the heads' powers of two; maxima, sums
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      qs[e] = 2 * tq + e < G ? q_factor[2 * tq + e] : 0.f;
      m_run[e] = unit[e] = unit_top[e] = kNone;
      l_run[e] = 0.f;
    }
    float o[KS][4];
#pragma unroll
    for (int j = 0; j < KS; ++j) o[j][0] = o[j][1] = o[j][2] = o[j][3] = 0.f;

    bool gave_up = false;
    int j = g0;  // block
#pragma unroll 1
    for (int i = 0;; ++i) {
      if (SOLO) top_up();
      if (i >= n_run) break;
      uint8_t* stage = stages + s * S::kStage;
      if (__any_sync(0xffffffffu, !mbar_wait(&full[s], phase))) {
        gave_up = true;
        break;
      }
      // the block: its rows that hold a key (bit r of mk), its bytes
      const bool t1 = j < p.nb1;
      const int jj = t1 ? j : j - p.nb1;
      const int live = t1 ? (sq.bad ? 0 : p.k) : sq.count;
      const int nk = min(max(live - jj * kQ8Block, 0), kQ8Block);
      const uint32_t mk = nk == 32 ? 0xFFFFFFFFu : (1u << nk) - 1u;
      int kc = scale_words[s * 8 + (jj & 3)], vc = scale_words[s * 8 + 4 + (jj & 3)];
      bool wrote_stage = false;  // generic-proxy writes into the stage

      if (FUSED && !t1 && sq.new_slot >= 0 && sq.new_slot / kQ8Block == jj) {
        const int r = sq.new_slot & (kQ8Block - 1);
        patch_block<D>(p, stage, u, r, sq.new_slot, mk & ~(1u << r), fresh, knew, kc, vc, lane);
        wrote_stage = true;
      }

      if (mk != 0u) {
        if (mk != 0xFFFFFFFFu) {
          // Zero the V rows that hold no key: their probabilities are 0, but 0 times NaN is not.
          if (!((mk >> lane) & 1u)) {
#pragma unroll
            for (int q = 0; q < D / 16; ++q)
              *reinterpret_cast<uint4*>(stage + S::kV + swz8<D>(lane, q)) = make_uint4(0u, 0u, 0u, 0u);
          }
          __syncwarp();
          wrote_stage = true;
        }
        const uint32_t sK = smem_addr(stage);
        const uint32_t sV = smem_addr(stage + S::kV);
        // ---- S^T = K Q^T, two products of 16 keys ----
        // (two accumulator chains a product)
        float sc[2][4], sd[2][4];  // product t: keys 16 t + gq (0, 1), 16 t + 8 + (gq ^ 4) (2, 3); heads 2 tq, 2 tq + 1
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          // lanes 0-7 / 8-15 / 16-23 / 24-31: rows 0-7 / 8-15 / 0-7 / 8-15 of the product, at
          // bytes 32 kk .. + 15 / same / 32 kk + 16 .. + 31 / same
          const int key = 16 * t + ((lane & 8) ? 8 + ((lane & 7) ^ 4) : lane & 7);
#pragma unroll
          for (int kk = 0; kk < KS / 2; ++kk) {
            uint32_t r0, r1, r2, r3, a0, a1, a2, a3;
            ldsm_x4(sK + swz8<D>(key, 2 * kk + (lane >> 4)), r0, r1, r2, r3);
            codes_f16(r0, a0, a2);
            codes_f16(r1, a1, a3);
            if (kk == 0) mma_f16_zero(sc[t], a0, a1, a2, a3, qa[0][0], qa[0][1]);
            else mma_f16(sc[t], a0, a1, a2, a3, qa[2 * kk][0], qa[2 * kk][1]);
            codes_f16(r2, a0, a2);
            codes_f16(r3, a1, a3);
            if (kk == 0) mma_f16_zero(sd[t], a0, a1, a2, a3, qa[1][0], qa[1][1]);
            else mma_f16(sd[t], a0, a1, a2, a3, qa[2 * kk + 1][0], qa[2 * kk + 1][1]);
          }
#pragma unroll
          for (int e = 0; e < 4; ++e) sc[t][e] += sd[t][e];
        }
        if (mk != 0xFFFFFFFFu) {
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            if (!((mk >> (16 * t + gq)) & 1u)) sc[t][0] = sc[t][1] = -INFINITY;
            if (!((mk >> (16 * t + 8 + (gq ^ 4))) & 1u)) sc[t][2] = sc[t][3] = -INFINITY;
          }
        }
        // ---- online softmax, log2 domain: f sc (f > 0) ----
        const float ks2 = e8m0_to_f32(kc);
        // (not below fp32's normal numbers: 0 times a masked score is no score)
        constexpr float kLeast = 1.17549435e-38f;
        float f0 = qs[0] * ks2, f1 = qs[1] * ks2;
        if (f0 < kLeast) f0 = kLeast;
        if (f1 < kLeast) f1 = kLeast;
        float mx0 = fmaxf(fmaxf(sc[0][0], sc[0][2]), fmaxf(sc[1][0], sc[1][2]));
        float mx1 = fmaxf(fmaxf(sc[0][1], sc[0][3]), fmaxf(sc[1][1], sc[1][3]));
#pragma unroll
        for (int off = 4; off < 32; off <<= 1) {
          mx0 = fmaxf(mx0, __shfl_xor_sync(0xffffffffu, mx0, off));
          mx1 = fmaxf(mx1, __shfl_xor_sync(0xffffffffu, mx1, off));
        }
        mx0 *= f0;
        mx1 *= f1;
        // (a NaN for K or V, of the byte or among a block's scores, makes no maximum and no unit, but p NaN)
        const float c = vc == 255 ? e8m0_to_f32(255) : static_cast<float>(vc);
        const float a0 = mx0 + c, a1 = mx1 + c;
        const bool up0 = mx0 > m_run[0], up1 = mx1 > m_run[1];
        const bool move0 = a0 > unit[0] || a0 + 10.f < unit[0], move1 = a1 > unit[1] || a1 + 10.f < unit[1];
        if (__any_sync(0xffffffffu, up0 || up1 || move0 || move1)) {
          if (up0) {
            l_run[0] *= ex2(m_run[0] - mx0);
            m_run[0] = mx0;
          }
          if (up1) {
            l_run[1] *= ex2(m_run[1] - mx1);
            m_run[1] = mx1;
          }
          const float u0 = move0 ? ceilf(fmaxf(a0, unit_top[0] - 64.f)) : unit[0];
          const float u1 = move1 ? ceilf(fmaxf(a1, unit_top[1] - 64.f)) : unit[1];
          const float g0 = ex2(unit[0] - u0), g1 = ex2(unit[1] - u1);
          unit[0] = u0;
          unit[1] = u1;
          unit_top[0] = fmaxf(unit_top[0], u0);
          unit_top[1] = fmaxf(unit_top[1], u1);
#pragma unroll
          for (int j = 0; j < KS; ++j) {
            o[j][0] *= g0;
            o[j][1] *= g1;
            o[j][2] *= g0;
            o[j][3] *= g1;
          }
        }
        float ref0 = unit[0] - (c + 15.f), ref1 = unit[1] - (c + 15.f);  // 2^15 p = 2^(s - ref)
        if (ref0 > m_run[0] + 29.f) ref0 = m_run[0] + 29.f;
        if (ref1 > m_run[1] + 29.f) ref1 = m_run[1] + 29.f;
        uint32_t pb[2][2];  // P^T as the B operand of k-step t: heads down, keys across
        float sum0 = 0.f, sum1 = 0.f;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int r = 0; r < 2; ++r) {
            const float p0 = ex2(fmaf(sc[t][2 * r], f0, -ref0));
            const float p1 = ex2(fmaf(sc[t][2 * r + 1], f1, -ref1));
            sum0 += p0;
            sum1 += p1;
            pb[t][r] = movmatrix_trans(pack_f16(p0, p1));
          }
        l_run[0] = fmaf(sum0, ex2(ref0 - m_run[0]), l_run[0]);
        l_run[1] = fmaf(sum1, ex2(ref1 - m_run[1]), l_run[1]);
        // ---- O^T += V^T P^T: lane's V row is k = lane of the two k-steps ----
        {
          const int a = lane & 15;
          const int r = 2 * (a >> 2) + (a & 1);
          const int key = (lane & 16) + ((a & 2) ? 8 + (r ^ 4) : r);
#pragma unroll
          for (int mt = 0; mt < KS; ++mt) {
            uint32_t r0, r1, r2, r3, a0, a1, a2, a3;
            ldsm_b8_t(sV + swz8<D>(key, mt), r0, r1, r2, r3);
            codes_f16(r0, a0, a2);
            codes_f16(r1, a1, a3);
            mma_f16(o[mt], a0, a1, a2, a3, pb[0][0], pb[0][1]);
            codes_f16(r2, a0, a2);
            codes_f16(r3, a1, a3);
            mma_f16(o[mt], a0, a1, a2, a3, pb[1][0], pb[1][1]);
          }
        }
      }

      // generic-proxy writes to this stage are ordered before the next box into it
      if (SOLO ? jn < rn || u + hop < p.units : issued < n_run) {
        if (wrote_stage) asm volatile("fence.proxy.async.shared::cta;\n" ::: "memory");
        __syncwarp();
      }
      if (SOLO) {
        --fly;
      } else if (issued < n_run) {
        request(s);
        ++issued;
      }
      j += step;
      if (++s == NST) {
        s = 0;
        phase ^= 1u;
      }
    }
    if (gave_up) {
      // Loads of this warp may still be on their way into its shared memory, and its barriers are no
      // evidence: kDrainNs covers them (no load was requested since the flag went up).
      cp_async_wait<0>();
      const uint32_t t0 = global_ns32();
      for (uint32_t it = 0; it < (1u << 16) && global_ns32() - t0 < kDrainNs; ++it) __nanosleep(1000);
      if (lane == 0) atomicOr(p.status, CMC_DEVFLAG_TIMEOUT);
      l_run[0] = l_run[1] = 0.f;
    }

    // ---- the four warps' states, then the cluster's CTAs' ----
    // Every warp sums its l over the lanes and leaves O in its first stage: 8 columns of
    // D floats, just the size of K's part, columns of odd pairs shifted so that the stores hit
    // distinct banks.  After a barrier each thread takes four rows of the head dimension of one
    // head, rescales and adds what the warps left, in warp order.
    // A head's (O, U, l, m) stand for the output O 2^(U - 127 - 15) / (l 2^m), O having p's 2^15.
    // O and l grow with the number of keys, so O 2^(U - 127 - m) alone may be beyond fp32 where the output is not
    // (values from 2^88 on), and 2^(U - 127 - m) / l below it (values around 2^-120): O is divided by l first, or
    // both are kept inside its range.
    {
#pragma unroll
      for (int e = 0; e < 2; ++e)
#pragma unroll
        for (int off = 4; off < 32; off <<= 1) l_run[e] += __shfl_xor_sync(0xffffffffu, l_run[e], off);
      if constexpr (SOLO) {
        // That is all of the unit: normalised and rounded, transposed back (head gq, two neighbours of
        // the head dimension a lane) and left in the query's place, whose fragments are in registers;
        // a head's 16-byte chunks are shifted by its number so that the stores hit distinct banks.
        float f[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          float y = unit[e] - m_run[e] - 142.f;
          const float z = y < -80.f ? -64.f : y > 100.f ? 24.f : 0.f;
          if (__any_sync(0xffffffffu, z != 0.f)) {
            const float g = ex2(z);
            y -= z;
#pragma unroll
            for (int j = 0; j < KS; ++j) {
              o[j][e] *= g;
              o[j][2 + e] *= g;
            }
          }
          f[e] = l_run[e] > 0.f ? __fdividef(ex2(y), l_run[e]) : 0.f;
        }
        uint32_t* row = reinterpret_cast<uint32_t*>(q_rows + gq * (D * 2));
#pragma unroll
        for (int j = 0; j < KS; ++j) {
          const uint32_t y0 = movmatrix_trans(pack_bf16_rn(o[j][0] * f[0], o[j][1] * f[1]));
          const uint32_t y1 = movmatrix_trans(pack_bf16_rn(o[j][2] * f[0], o[j][3] * f[1]));
          if (gq < G) {
            row[((2 * j) ^ gq) * 4 + tq] = y0;
            row[((2 * j + 1) ^ gq) * 4 + tq] = y1;
          }
        }
        __syncwarp();
#pragma unroll
        for (int x0 = 0; x0 < G * D / 8; x0 += 32) {
          const int x = x0 + lane, hh = x / (D / 8), c = x % (D / 8);
          if (x < G * D / 8)
            *reinterpret_cast<uint4*>(p.out + static_cast<long long>(u) * (G * D) + 8 * x) =
                *reinterpret_cast<const uint4*>(q_rows + hh * (D * 2) + (c ^ hh) * 16);
        }
        if (FUSED && lane == 0 && ticket + 1 == static_cast<unsigned long long>(p.LH)) {
          if (!sq.bad) p.pos[b] = pos + 1;
          p.tickets[b] = 0ull;
        }
        if (gave_up) {
          if (FUSED && lane == 0) count_left_units(p.tickets, p.pos, u + hop, hop, p.units, p.LH);
          return;
        }
        __syncwarp();
        u += hop;
        if (u >= p.units) return;
        b = static_cast<int>(static_cast<unsigned>(u) / static_cast<unsigned>(p.LH));
        pos = pos_next;
        fresh = fresh_next;
        issued = 0;
        continue;
      }
      __syncwarp();  // the warp is done with the stage
      float* ow = reinterpret_cast<float*>(stages);
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        float* col = ow + (2 * tq + e) * D;
        if (2 * tq + e < G) {
#pragma unroll
          for (int j = 0; j < KS; ++j) {
            col[(16 * j + gq) ^ (8 * tq)] = o[j][e];
            col[(16 * j + 8 + gq) ^ (8 * tq)] = o[j][2 + e];
          }
        }
      }
      if (gq == 0) {
        float* ml = reinterpret_cast<float*>(smem + S::kMl) + warp * 24 + 2 * tq;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          ml[e] = m_run[e];
          ml[8 + e] = l_run[e];
          ml[16 + e] = unit[e];
        }
      }
      if (lane == 0) s_left[warp] = static_cast<int>(stages - smem);
      if (FUSED && tid == 0) s_last = ticket + 1 == static_cast<unsigned long long>(p.order ? p.units : p.LH) * cm;
    }
    __syncthreads();
    if (FUSED && s_last && tid < (p.order ? p.B : 1)) {
      const long long x = p.order ? ld_pos(p, tid) : pos;
      if (x >= 0) p.pos[p.order ? tid : b] = x + 1;
      if (tid == 0) p.tickets[p.order ? 0 : b] = 0ull;
    }
    const long long out_base = static_cast<long long>(u) * (G * D);
    const float* ml = reinterpret_cast<const float*>(smem + S::kMl);
    constexpr int XPT = (NGR + kThreads - 1) / kThreads;  // groups per thread
    float4 cacc[XPT];
    float cls[XPT], cmx[XPT];
#pragma unroll
    for (int xi = 0; xi < XPT; ++xi) {
      const int x = tid + xi * kThreads;
      if (x >= NGR) break;
      const int hh = (4 * x) / D;
      const int c = (4 * x) % D;
      float M = ml[hh], U = ml[16 + hh];
#pragma unroll
      for (int v = 1; v < kWarps; ++v) {
        M = fmaxf(M, ml[v * 24 + hh]);
        U = fmaxf(U, ml[v * 24 + 16 + hh]);
      }
      float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
      float Ls = 0.f;
#pragma unroll
      for (int v = 0; v < kWarps; ++v) {
        const float f = ex2(ml[v * 24 + 16 + hh] - U);
        const float* left = reinterpret_cast<const float*>(smem + s_left[v]);
        const float4 y = *reinterpret_cast<const float4*>(left + hh * D + (c ^ (8 * (hh >> 1))));
        acc.x = fmaf(f, y.x, acc.x); acc.y = fmaf(f, y.y, acc.y);
        acc.z = fmaf(f, y.z, acc.z); acc.w = fmaf(f, y.w, acc.w);
        Ls = fmaf(ex2(ml[v * 24 + hh] - M), ml[v * 24 + 8 + hh], Ls);
      }
      // times 2^y, in two factors where it is far from 1
      const float y = U - M - 142.f, y0 = fminf(fmaxf(y, -80.f), 100.f);
      const float f0 = Ls > 0.f ? __fdividef(ex2(y0), Ls) : 0.f, f1 = ex2(y - y0);
      acc = make_float4(acc.x * f0 * f1, acc.y * f0 * f1, acc.z * f0 * f1, acc.w * f0 * f1);
      if (cm == 1) {
        *reinterpret_cast<uint2*>(p.out + out_base + hh * D + c) =
            make_uint2(pack_bf16_rn(acc.x, acc.y), pack_bf16_rn(acc.z, acc.w));
      } else {
        cacc[xi] = acc;
        cls[xi] = Ls;
        cmx[xi] = M;
      }
    }
    if (cm == 1) return;
    // One share of the unit per CTA: its output, and the maxima and sums that weigh it, stored into the
    // peers' receive areas, to each the groups that peer finishes; then merged in rank order.
    const int SL = p.slice;
    const uint32_t recv_a = smem_addr(smem + S::kRecv), ml_a = smem_addr(smem + S::kRecvMl);
    const uint32_t bar_a = smem_addr(&recv_bar);
    cluster_wait();
#pragma unroll
    for (int xi = 0; xi < XPT; ++xi) {
      const int x = tid + xi * kThreads;
      if (x >= NGR) break;
      const int hh = (4 * x) / D;
      const int to = x / SL;
      st_peer_f4(peer_smem(recv_a + (rank * SL + x - to * SL) * 16, to), cacc[xi], peer_smem(bar_a, to));
      if ((4 * x) % D == 0) {
        for (int r = 0; r < cm; ++r)
          st_peer_f2(peer_smem(ml_a + (rank * G + hh) * 8, r), cmx[xi], cls[xi], peer_smem(bar_a, r));
      }
    }
    mbar_wait_peers(&recv_bar);
    const int x0 = rank * SL, x1 = min(x0 + SL, NGR);
    for (int x = x0 + tid; x < x1; x += kThreads) {
      const int hh = (4 * x) / D;
      const int c = (4 * x) % D;
      const float2* pl = reinterpret_cast<const float2*>(smem + S::kRecvMl) + hh;
      float M = kNone;
#pragma unroll
      for (int r = 0; r < kMaxClusterCtas; ++r)
        if (r < cm) M = fmaxf(M, pl[r * G].x);
      float w[kMaxClusterCtas], Ls = 0.f;
#pragma unroll
      for (int r = 0; r < kMaxClusterCtas; ++r) {
        if (r < cm) {
          w[r] = ex2(pl[r * G].x - M) * pl[r * G].y;
          Ls += w[r];
        }
      }
      const float inv = Ls > 0.f ? __frcp_rn(Ls) : 0.f;
      float4 O = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int r = 0; r < kMaxClusterCtas; ++r) {
        if (r < cm) {
          const float4 o4 = *reinterpret_cast<const float4*>(smem + S::kRecv + (r * SL + x - x0) * 16);
          const float f = w[r] * inv;
          O.x = fmaf(f, o4.x, O.x);
          O.y = fmaf(f, o4.y, O.y);
          O.z = fmaf(f, o4.z, O.z);
          O.w = fmaf(f, o4.w, O.w);
        }
      }
      *reinterpret_cast<uint2*>(p.out + out_base + hh * D + c) =
          make_uint2(pack_bf16_rn(O.x, O.y), pack_bf16_rn(O.z, O.w));
    }
    if (tid == 0 && attn_aborted()) atomicOr(p.status, CMC_DEVFLAG_TIMEOUT);
  } while (SOLO);
}

// ---------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------

// T rows of codes of every (unit, K or V), `stride` rows apart.
static bool encode_q8(CUtensorMap* map, const void* base, long long units2, int T, int stride, int d) {
  EncodeTiledFn enc = encode_fn();
  if (!enc) return false;
  cuuint64_t dims[3] = {static_cast<cuuint64_t>(d), static_cast<cuuint64_t>(T), static_cast<cuuint64_t>(units2)};
  cuuint64_t strides[2] = {static_cast<cuuint64_t>(d), static_cast<cuuint64_t>(stride) * d};
  cuuint32_t box[3] = {static_cast<cuuint32_t>(d), kQ8Block, 2};
  cuuint32_t es[3] = {1, 1, 1};
  return enc(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 3, const_cast<void*>(base), dims, strides, box, es,
             CU_TENSOR_MAP_INTERLEAVE_NONE, d == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B,
             CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

static int q8_blocks(int rows) { return (rows + kQ8Block - 1) / kQ8Block; }

// How a call's units are put on the GPU.  Three variants of the kernel:
//   wide   a CTA (or cluster) per unit, three stages a warp, two CTAs an SM: few or long units
//   spread the same with two stages a warp and three CTAs an SM: when the units, or their
//          clusters, just miss one wave of the first (176 x 61 blocks: two CTAs a unit in one
//          wave 15.9 us, one a unit of the first 20.1)
//   solo   a warp per unit, three stages a warp, two CTAs (eight units) an SM: many short units.  Of
//          units of up to twelve blocks a warp takes one after another, from a grid of one wave (8,192 of 6
//          blocks 61.4 us, 75.7 with a CTA for every four; ragged 42.5 and 56.4; 2,048 19.9 and 22.0); longer
//          ones are evened out better by the hardware (8,192 of 20 blocks 207.8 and 196.7)
struct Q8Plan {
  enum { kWide, kSpread, kSolo } variant;
  int cm;      // CTAs per unit
  int ctas;    // grid size
  bool order;  // the units of the longest sequences first
};

// CTAs of a variant that fit an SM of the current device.
template <int D, int G, bool FUSED, int NST, bool SOLO>
static int per_sm_q8(int* per_sm) {
  constexpr int smem = Q8Smem<D, G, NST, SOLO>::kBytes;
  auto kern = attn_q8_kernel<D, G, FUSED, NST, SOLO>;
  int st = record_cuda_error(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
  if (st != CMC_OK) return st;
  st = record_cuda_error(cudaOccupancyMaxActiveBlocksPerMultiprocessor(per_sm, kern, kThreads, smem));
  if (st == CMC_OK && *per_sm < 1) *per_sm = 1;
  return st;
}

// CTAs of the three variants that the current device holds at a time; looked up once per device
// (idempotent), and kept as 20 bits each.
template <int D, int G, bool FUSED>
static int resident_q8(int* wide, int* spread, int* solo) {
  static std::atomic<uint64_t> known[64];
  int dev = 0;
  int st = record_cuda_error(cudaGetDevice(&dev));
  if (st != CMC_OK) return st;
  uint64_t v = dev >= 0 && dev < 64 ? known[dev].load(std::memory_order_acquire) : 0;
  if (v == 0) {
    int a = 0, b = 0, c = 0;
    st = per_sm_q8<D, G, FUSED, 3, false>(&a);
    if (st == CMC_OK) st = per_sm_q8<D, G, FUSED, 2, false>(&b);
    if (st == CMC_OK) st = per_sm_q8<D, G, FUSED, 3, true>(&c);
    if (st != CMC_OK) return st;
    const uint64_t sms = static_cast<uint64_t>(sm_count());
    v = (a * sms) | (b * sms) << 20 | (c * sms) << 40;
    if (dev >= 0 && dev < 64) known[dev].store(v, std::memory_order_release);
  }
  *wide = static_cast<int>(v & 0xFFFFF);
  *spread = static_cast<int>((v >> 20) & 0xFFFFF);
  *solo = static_cast<int>((v >> 40) & 0xFFFFF);
  return CMC_OK;
}

// The variant and cluster size whose time comes out least by
//   waves * (3 us + blocks of a warp * P),  P = 1.1 us with eight warps an SM and 1.5 with twelve,
// a rough fit to the following (us a launch in a graph, G = 4, d = 128; wide with the largest
// cluster that fits one wave / spread / solo):
//   16 x  2 blocks 3.4 / 3.4 / 5.8       300 x  3   4.0 /  4.6 /  5.3    512 x  3   7.2 /  7.0 /  5.5
//   256 x 20       9.3 / 10.4 / 18.7     512 x 10  12.9 / 12.3 / 11.5    768 x 20  29.1 / 25.6 / 23.6
//   256 x 40      14.8 / 17.0 / 33.9    1024 x 10  24.3 / 20.7 / 14.8   1216 x 20  41.3 / 38.7 / 31.1
//   312 x 72      40.4 / 30.6 / -       2048 x  6  33.5 / 26.6 / 19.9   2048 x 10  45.5 / 36.5 / 29.2
//   512 x 72      47.9 / 56.6 / -       2048 x  1  21.3 / 16.4 /  7.2   2048 x 20  65.6 / 60.1 / 53.8
// (The blocks are those of a full ring: pos is on the device.)  Several waves of long units, ordered by
// length, count for 85 % of their time: where rings differ they are evened out, which a warp with a long unit of its own
// is not (1,024 x 72 blocks, wide / solo: full 97.8 / 90.0 us, ragged 48.8 / 72.5).
template <int D, int G, bool FUSED>
static int plan_q8(long long units, int B, int nb, Q8Plan* pl) {
  int wide = 0, spread = 0, solo = 0;  // CTAs resident at a time
  const int st = resident_q8<D, G, FUSED>(&wide, &spread, &solo);
  if (st != CMC_OK) return st;
  // in tenths of a microsecond
  auto cost = [&](long long ctas, int slots, int blocks, int per_block) {
    return (ctas + slots - 1) / slots * (30 + static_cast<long long>(blocks) * per_block);
  };
  const long long quads = (units + kWarps - 1) / kWarps;
  const bool order = B > 1 && B <= kThreads;
  long long best = -1;
  for (int cm = 1; cm <= kMaxClusterCtas && (cm == 1 || kWarps * cm / 2 < nb); cm *= 2) {
    const int blocks = (nb + kWarps * cm - 1) / (kWarps * cm), merge = cm > 1 ? 3 : 0;  // a cluster's: 0.3 us
    // A cluster lies in one group of SMs, and eight CTAs do not fill every group: 56 clusters of eight in
    // 456 places took two waves (56 x 128 blocks 17.5 us, with clusters of four 12.8).
    const int w = cm == 8 ? wide * 7 / 8 : wide, p3 = cm == 8 ? spread * 7 / 8 : spread;
    // several waves of whole units only
    if (cm == 1 || units * cm <= w) {
      const bool ordered = order && units * cm > w;
      long long t = cost(units * cm, w, blocks, 11) + merge;
      if (ordered && nb >= 32) t = t * 17 / 20;
      if (best < 0 || t < best) {
        best = t;
        *pl = {Q8Plan::kWide, cm, static_cast<int>(units * cm), ordered};
      }
    }
    if (cm == 1 || units * cm <= p3) {
      const long long t = cost(units * cm, p3, blocks, 15) + merge;
      if (t < best) {
        best = t;
        *pl = {Q8Plan::kSpread, cm, static_cast<int>(units * cm), order && units * cm > p3};
      }
    }
  }
  if (cost(quads, solo, nb, 11) < best)
    *pl = {Q8Plan::kSolo, 1, static_cast<int>(nb <= 12 ? std::min<long long>(quads, solo) : quads), false};
  return CMC_OK;
}

template <int D, int G, bool FUSED, int NST, bool SOLO>
static int launch_q8(const Q8Maps& maps, AttnQ8Params& p, const Q8Plan& pl, cudaStream_t s) {
  p.cm = pl.cm;
  p.slice = pl.cm > 1 ? (G * D / 4 + pl.cm - 1) / pl.cm : 0;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = static_cast<unsigned>(pl.cm);
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(pl.ctas));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = Q8Smem<D, G, NST, SOLO>::kBytes;
  cfg.stream = s;
  cfg.attrs = attr;
  cfg.numAttrs = pl.cm > 1 ? 2 : 1;
  return record_cuda_error(cudaLaunchKernelEx(&cfg, attn_q8_kernel<D, G, FUSED, NST, SOLO>, maps, p));
}

// Calls F<D, G>::run(args...) for the call's head dimension and group size.
template <template <int, int> class F, typename... Args>
static int by_shape(int d, int G, Args&&... args) {
  if (d == 128) {
    switch (G) {
      case 1: return F<128, 1>::run(args...);
      case 2: return F<128, 2>::run(args...);
      case 4: return F<128, 4>::run(args...);
      default: return F<128, 8>::run(args...);
    }
  }
  switch (G) {
    case 1: return F<64, 1>::run(args...);
    case 2: return F<64, 2>::run(args...);
    case 4: return F<64, 4>::run(args...);
    default: return F<64, 8>::run(args...);
  }
}
template <int D, int G>
struct PlanQ8 {
  static int run(bool fused, long long units, int B, int nb, Q8Plan* pl) {
    return fused ? plan_q8<D, G, true>(units, B, nb, pl) : plan_q8<D, G, false>(units, B, nb, pl);
  }
};
template <int D, int G>
struct LaunchQ8 {
  template <bool FUSED>
  static int go(const Q8Maps& maps, AttnQ8Params& p, long long units, cudaStream_t s) {
    Q8Plan pl;
    int st = plan_q8<D, G, FUSED>(units, p.B, p.nb1 + p.nb2, &pl);
    if (st != CMC_OK) return st;
    p.order = pl.order;
    switch (pl.variant) {
      case Q8Plan::kSolo: return launch_q8<D, G, FUSED, 3, true>(maps, p, pl, s);
      case Q8Plan::kSpread: return launch_q8<D, G, FUSED, 2, false>(maps, p, pl, s);
      default: return launch_q8<D, G, FUSED, 3, false>(maps, p, pl, s);
    }
  }
  static int run(bool fused, const Q8Maps& maps, AttnQ8Params& p, long long units, cudaStream_t s) {
    return fused ? go<true>(maps, p, units, s) : go<false>(maps, p, units, s);
  }
};

static int run_attention_q8(const void* q, const void* t1_kv, const void* t1_scales, void* ring_kv,
                            void* ring_scales, int64_t* pos, const void* k_new, const void* v_new,
                            const cmc_dims* dims, float scale, double rope_theta, long long rope_offset,
                            void* out, void* workspace, size_t workspace_bytes, void* stream, bool fused) {
  int st = validate_dims(dims, true);
  if (st != CMC_OK) return st;
  const cmc_dims& m = *dims;
  if (!q || !ring_kv || !ring_scales || !pos || !out) return CMC_ERR_NULL;
  if (m.k > 0 && (!t1_kv || !t1_scales)) return CMC_ERR_NULL;
  if (fused && (!k_new || !v_new)) return CMC_ERR_NULL;
  const bool rope = rope_theta != 0.0;
  if (rope && !(rope_theta > 0.0 && rope_theta < 1e300)) return CMC_ERR_RANGE;
  if (rope && (rope_offset < 0 || rope_offset > (1LL << 32))) return CMC_ERR_RANGE;
  if (!aligned16(q) || !aligned16(ring_kv) || !aligned16(ring_scales) || !aligned16(out) ||
      (reinterpret_cast<uintptr_t>(pos) & 7))
    return CMC_ERR_ALIGN;
  if (m.k > 0 && (!aligned16(t1_kv) || !aligned16(t1_scales))) return CMC_ERR_ALIGN;
  if (fused && (!aligned16(k_new) || !aligned16(v_new))) return CMC_ERR_ALIGN;
  if (!workspace || workspace_bytes < ws_partials_off(m.B)) return CMC_ERR_WORKSPACE;
  if (!aligned16(workspace)) return CMC_ERR_ALIGN;

  const long long units = static_cast<long long>(m.B) * m.L * m.Hkv;
  const int nb1 = q8_blocks(m.k), nb2 = q8_blocks(m.W);

  Q8Maps maps;
  memset(&maps, 0, sizeof(maps));
  if (!encode_q8(&maps.ring, ring_kv, 2 * units, m.W, m.W, m.d)) return CMC_ERR_CUDA;
  if (m.k > 0 && !encode_q8(&maps.t1, t1_kv, 2 * units, m.k, m.N, m.d)) return CMC_ERR_CUDA;

  AttnQ8Params p = {};
  p.q = static_cast<const uint16_t*>(q);
  p.pos = pos;
  p.k_new = static_cast<const uint16_t*>(k_new);
  p.v_new = static_cast<const uint16_t*>(v_new);
  p.out = static_cast<uint16_t*>(out);
  char* ws = static_cast<char*>(workspace);
  p.status = reinterpret_cast<uint32_t*>(ws);
  p.tickets = reinterpret_cast<unsigned long long*>(ws + kWsHeader);
  p.B = m.B; p.L = m.L; p.Hq = m.Hq; p.Hkv = m.Hkv; p.N = m.N; p.k = m.k; p.W = m.W;
  p.LH = m.L * m.Hkv;
  p.units = static_cast<int>(units);
  p.nb1 = nb1;
  p.nb2 = nb2;
  const float sc = scale > 0.f ? scale : 1.0f / sqrtf(static_cast<float>(m.d));
  p.scale_log2 = sc * 1.4426950408889634f;
  // At most as many blocks a warp as it has stages: with five, blocks are fetched that hold no key, or that
  // the warp's own requests would have reached in time (1,216 units of 6 blocks 11.8 us, 11.3 with three and
  // 12.6 with none; 400 of 72 36.8, 35.8 and 37.8).
  p.l2_prefetch = std::min(l2_prefetch_setting(), 3);
  p.stall_tx = stall_tx_setting();
  p.ring_kv = static_cast<uint8_t*>(ring_kv);
  p.ring_scales = static_cast<uint8_t*>(ring_scales);
  p.t1_scales = static_cast<const uint8_t*>(t1_scales);
  p.ringS = q8_scale_bytes(m.W);
  p.t1S = q8_scale_bytes(m.N);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  p.rope_slot = -1;
  if (rope) {
    p.rope = 1;
    p.rope_offset = rope_offset;
    rope_turns_table(rope_theta, m.d, p.rope_turns);
    p.rope_slot = rope_slot(rope_theta, m.d, p.rope_turns, s);
  }
  return by_shape<LaunchQ8>(m.d, m.Hq / m.Hkv, fused, maps, p, units, s);
}

}  // namespace cmc

extern "C" {

size_t cmc_decode_attn_q8_workspace_size(const cmc_dims* dims) {
  return cmc::validate_dims(dims, true) == CMC_OK ? cmc::ws_partials_off(dims->B) : 0;
}

int cmc_two_tier_decode_attn_q8(const void* q, const void* tier1_kv, const void* tier1_scales,
                                const void* ring_kv, const void* ring_scales, const int64_t* pos,
                                const cmc_dims* dims, float scale, void* out, void* workspace,
                                size_t workspace_bytes, void* stream) {
  return cmc::run_attention_q8(q, tier1_kv, tier1_scales, const_cast<void*>(ring_kv),
                               const_cast<void*>(ring_scales), const_cast<int64_t*>(pos), nullptr, nullptr,
                               dims, scale, 0.0, 0, out, workspace, workspace_bytes, stream, false);
}

int cmc_decode_step_q8(const void* q, const void* tier1_kv, const void* tier1_scales, void* ring_kv,
                       void* ring_scales, int64_t* pos, const void* k_new, const void* v_new,
                       const cmc_dims* dims, float scale, double rope_theta, int64_t rope_offset, void* out,
                       void* workspace, size_t workspace_bytes, void* stream) {
  return cmc::run_attention_q8(q, tier1_kv, tier1_scales, ring_kv, ring_scales, pos, k_new, v_new, dims,
                               scale, rope_theta, rope_offset, out, workspace, workspace_bytes, stream, true);
}

int cmc_decode_attn_q8_plan(const cmc_dims* dims, int fused, int* ctas) {
  using namespace cmc;
  int st = validate_dims(dims, true);
  if (st != CMC_OK) return st;
  if (!ctas) return CMC_ERR_NULL;
  const cmc_dims& m = *dims;
  const long long units = static_cast<long long>(m.B) * m.L * m.Hkv;
  Q8Plan pl;
  st = by_shape<PlanQ8>(m.d, m.Hq / m.Hkv, fused != 0, units, m.B, q8_blocks(m.k) + q8_blocks(m.W), &pl);
  if (st != CMC_OK) return st;
  *ctas = pl.ctas;
  return CMC_OK;
}

}  // extern "C"
