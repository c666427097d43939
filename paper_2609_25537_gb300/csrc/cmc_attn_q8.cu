// Decode attention over the two-tier cache held in 8 bits (format: cmc_q8.cuh),
// alone and fused with the append of the step's token.
//
// Work decomposition, pipeline and merges are those of the attention over a bf16
// cache (cmc_attn.cu): units (sequence, layer, KV head), a producer warp and four
// consumer warps a CTA, clusters for few long units, runs of whole units or
// stream-K for many.  What differs follows from the 8 bits.
//
// Tiles of 128 keys: 128 codes rows of K and of V, 32 KB at d = 128, come as one TMA
// box of a [2 units, T, d] tensor (rows past T are not read), as many bytes as
// the 64-key tiles of the bf16 kernel.  A warp owns 32 keys, which are one block
// with one power of two for K and one for V; the tile's four of each are one
// aligned word, copied by cp.async next to the tile.
//
// Both products run on e4m3 operands (mma.sync m16n8k32, fp32 accumulation,
// exact products), so no code is ever converted: K by ldmatrix, V by the byte
// transposing ldmatrix of sm_100.  The other operands are written as two e4m3
// pieces, x = hi + lo / 16, each with four significant bits:
//   q    times a power of two so that its largest element is in (224, 448].  A bf16
//        element has eight significant bits, so hi + lo / 16 is exact down to 2^-14 of
//        the largest, and off by 2^-22 of the largest below.
//   p    256 times the probability relative to the largest so far: rounded to eight
//        significant bits (2^-8, as a bf16 probability) down to 2^-14, and off by 2^-22
//        below.
// A product has eight columns and a KV head G query heads.  For G <= 4 the lo
// pieces are the columns 4 .. 7 of the same products, so they cost nothing; for
// G = 8 they take products of their own.
//   S^T = K Q^T   16 keys as the rows, d in k-steps of 32
//   O^T += V^T P^T  16 rows of the head dimension, the warp's 32 keys as the k-step
// K's power of two joins the softmax scale.  V's cannot (it changes from block to
// block): O is kept in units of 2^(E - 127) with E the byte of a recent block, and
// rescaled, as for a new maximum, when a block's byte is above E or more than four
// below it; in between p is multiplied by the difference.
//
// P^T has to go from the accumulators of S^T (keys down the rows) to the B operand
// (four neighbouring k a register).  A pair of codes is one 16-bit element of an
// 8 x 8 transpose (movmatrix) if its two keys are those of the two 16-key products'
// same row; the k order that this gives is met by the order of V's row addresses.
// The second product's rows are exchanged by halves (row r is key 16 + (r ^ 4)) so
// that eight consecutive k lie in eight different bank groups.
#include <atomic>

#include "cmc_attn.cuh"
#include "cmc_q8.cuh"

namespace cmc {

constexpr int kQ8Tile = 128;  // keys per pipeline tile; each consumer warp owns 32 of them
constexpr int kQ8Stages = 3;
static_assert(kQ8Tile == kWarps * kQ8Block, "a warp's keys are one block");
enum { H_KSCALES = H_BADLO, H_VSCALES = H_BADHI };  // the tile's four bytes of K and of V

struct Q8Maps {
  CUtensorMap t1, ring;  // [2 units, T, d] bytes, box 2 x 128 rows
};

struct AttnQ8Params : AttnParams {  // t1k, t1v, ring_k, ring_v, idx are not used
  uint8_t* ring_kv;           // [B, L, Hkv, 2, W, d]
  uint8_t* ring_scales;       // [B, L, Hkv, 2, ringS]
  const uint8_t* t1_scales;   // [B, L, Hkv, 2, t1S]
  int ringS, t1S;
  int rope;                   // rotate q and the new key (fused step)
};

// Shared memory: the stages (codes of K, then of V), one slot per stage with what a
// unit needs besides (its query rows, the new token's rows, the rotary table),
// the headers, the warps' (max, sum) for the merge.
//
// Slots go by unit, in turn: a unit's slot is taken again three units later, when
// at least three tiles were handed back since.  Under a cluster plan a CTA has
// one unit, so slots 1 and 2 are free for what its peers send (see recv_group).
template <int D, int G>
struct Q8Smem {
  static constexpr int kV = kQ8Tile * D;
  static constexpr int kStage = 2 * kQ8Tile * D;
  static constexpr int kQ = 0;                   // query rows [G][D] bf16
  static constexpr int kNew = G * D * 2;         // new token K row, V row (bf16)
  static constexpr int kRope = kNew + 2 * D * 2; // d/2 (cos, sin) pairs
  static constexpr int kSlot = kRope + D * 4;
  static constexpr int kSlots = kQ8Stages * kStage;  // offsets from the aligned base
  static constexpr int kHdrs = kSlots + kQ8Stages * kSlot;
  static constexpr int kMergeM = kHdrs + kQ8Stages * 32;
  static constexpr int kMergeL = kMergeM + kWarps * 8 * 4;
  static constexpr int kBytes = kMergeL + kWarps * 8 * 4 + 1008;  // the base is 16-byte aligned
  // received: cm * ceil(G D / 4 / cm) groups of 16 bytes, then (max, sum) of G heads from each rank
  static constexpr int kRecv = kSlots + kSlot;
  static constexpr int kRecvMl = kRecv + (G * D / 4 + kMaxClusterCtas - 2) * 16;
  static_assert(kRecvMl + kMaxClusterCtas * G * 8 <= kHdrs, "slots 1 and 2 hold what the peers send");
};

// Offset of 16-byte chunk c of row r in a K or V region: TMA's 128-byte swizzle, or the
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

// C[16x8] += A[16x32] B[32x8], e4m3 inputs, fp32 accumulators.
__device__ __forceinline__ void mma_e4m3(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2,
                                         uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k32.row.col.f32.e4m3.e4m3.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, "
      "{%8,%9}, {%0,%1,%2,%3};\n"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_e4m3_zero(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2,
                                              uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k32.row.col.f32.e4m3.e4m3.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, "
      "{%8,%9}, {%10,%10,%10,%10};\n"
      : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}

// Two probabilities as two e4m3 pieces each (a in the low byte): hi, and lo = 16 (x - hi).
// Through fp16, whose 11 bits and steps of 2^-24 lose nothing that the pieces keep.
__device__ __forceinline__ void two_pieces(float a, float b, uint32_t& hi, uint32_t& lo) {
  uint16_t h, l;
  asm("{\n .reg .b32 x, y, s;\n"
      " cvt.rn.f16x2.f32 x, %3, %2;\n"
      " cvt.rn.satfinite.e4m3x2.f16x2 %0, x;\n"
      " cvt.rn.f16x2.e4m3x2 y, %0;\n"
      " sub.rn.f16x2 y, x, y;\n"
      " mov.b32 s, 0x4C004C00;\n"  // 16, 16
      " mul.rn.f16x2 y, y, s;\n"
      " cvt.rn.satfinite.e4m3x2.f16x2 %1, y;\n}\n"
      : "=&h"(h), "=&h"(l)
      : "f"(a), "f"(b));
  hi = h;
  lo = l;
}

__device__ __forceinline__ int tile_row(const AttnQ8Params& p, const TileCursor& c) {
  return (c.lt < p.t1_tiles ? c.lt : c.lt - p.t1_tiles) * kQ8Tile;
}
__device__ __forceinline__ const CUtensorMap* tile_map(const AttnQ8Params& p, const Q8Maps& maps,
                                                       const TileCursor& c) {
  return c.lt < p.t1_tiles ? &maps.t1 : &maps.ring;
}
// The producer's lanes 0 and 1: the tile's powers of two of K and of V into the header.
__device__ __forceinline__ void load_scales(const AttnQ8Params& p, const TileCursor& c, uint8_t* hdr,
                                            int lane) {
  const bool t1 = c.lt < p.t1_tiles;
  const int S = t1 ? p.t1S : p.ringS;
  const uint8_t* from = (t1 ? p.t1_scales : p.ring_scales) + (2LL * c.u + lane) * S +
                        (t1 ? c.lt : c.lt - p.t1_tiles) * 4;
  cp_async_4(smem_addr(hdr + 4 * (lane ? H_VSCALES : H_KSCALES)), from, 4u);
}

// The new token in its block, by the consumer warp that owns it: the token's codes over
// the stale ones, in the tile and in the ring; the block's other codes too where
// its power of two changes.  `others`: the block's rows that hold another token.
// Returns the block's byte.  (The rules are window_append_q8_kernel's.)
template <int D>
__device__ __forceinline__ int patch_block(uint8_t* rows /* the tile's K or V */, uint8_t* ring_row0,
                                           uint8_t* ring_scale, const float (&x)[4], int r, int c_old,
                                           bool first, uint32_t others, int lane, int warp) {
  uint32_t top = 0u;
#pragma unroll
  for (int e = 0; e < D / 32; ++e) top = max(top, finite_bits(x[e]));
  top = __reduce_max_sync(0xffffffffu, top);
  const bool mine = (others >> lane) & 1u;  // the lane's row of the block
  const int row = 32 * warp + lane;
  int c;
  if (first) {
    uint32_t m = 0u;
    if (mine)
      for (int q = 0; q < D / 16; ++q) m = max_codes16(m, *reinterpret_cast<const uint4*>(rows + swz8<D>(row, q)));
    c = block_code(max(top, __reduce_max_sync(0xffffffffu, held_bits(m, c_old))));
  } else {
    c = max(block_code(top), c_old);
  }
  if (c != c_old && mine) {
    const float f = recode_factor(c_old, c);
    for (int q = 0; q < D / 16; ++q) {
      uint4* at = reinterpret_cast<uint4*>(rows + swz8<D>(row, q));
      const uint4 y = recode16(*at, f);
      *at = y;
      reinterpret_cast<uint4*>(ring_row0 + static_cast<long long>(lane) * D)[q] = y;
    }
  }
  const float f = code_factor(c);
  uint8_t* to = ring_row0 + static_cast<long long>(r) * D;
  if (D == 128) {
    const uint32_t w = encode4(x[0], x[1], x[2], x[3], f);
    *reinterpret_cast<uint32_t*>(rows + swz8<D>(32 * warp + r, lane >> 2) + (lane & 3) * 4) = w;
    reinterpret_cast<uint32_t*>(to)[lane] = w;
  } else {
    const uint16_t w = static_cast<uint16_t>(e4m3_pair(scaled(x[0], f), scaled(x[1], f)));
    *reinterpret_cast<uint16_t*>(rows + swz8<D>(32 * warp + r, lane >> 3) + (lane & 7) * 2) = w;
    reinterpret_cast<uint16_t*>(to)[lane] = w;
  }
  if (lane == 0) *ring_scale = static_cast<uint8_t>(c);
  return c;
}

template <int D, int G, bool FUSED>
__global__ void __maxnreg__(D == 64 ? 96 : 128)
attn_q8_kernel(const __grid_constant__ Q8Maps maps, const AttnQ8Params p) {
  using S = Q8Smem<D, G>;
  constexpr int NST = kQ8Stages;
  constexpr int KS = D / 32;         // k-steps of the Q K^T product
  constexpr int MT = D / 16;         // m-tiles of O^T
  constexpr bool PAIRED = G <= 4;    // hi and lo pieces in one product
  constexpr int NV = PAIRED ? 2 : 4; // scores a thread has of each of its two heads
  extern __shared__ __align__(16) uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* slot0 = smem + S::kSlots;
  uint8_t* hdr0 = smem + S::kHdrs;
  float* merge_m = reinterpret_cast<float*>(smem + S::kMergeM);  // [kWarps][8]
  float* merge_l = reinterpret_cast<float*>(smem + S::kMergeL);
  __shared__ __align__(8) uint64_t full_bar[NST];
  __shared__ __align__(8) uint64_t empty_bar[NST];
  __shared__ __align__(8) uint64_t recv_bar;  // cluster plan: the peers' stores

  const int tid = threadIdx.x;
  const int lane = tid & 31;
  const int warp = tid >> 5;

  // This CTA's first tile and its tiles, in order.
  int u_begin, j_begin = 0, n_tiles;
  {
    const int cta = static_cast<int>(blockIdx.x);
    if (p.cm > 0) {
      u_begin = static_cast<int>(cluster_id());
      j_begin = static_cast<int>(cluster_ctarank());
      n_tiles = p.base + (j_begin < p.rem ? 1 : 0);
    } else {
      const int first = cta * p.base + min(cta, p.rem);
      const int n = p.base + (cta < p.rem ? 1 : 0);
      if (p.gran > 1) {  // whole units
        u_begin = first;
        n_tiles = n * p.gran;
      } else {
        u_begin = static_cast<int>(static_cast<unsigned>(first) / static_cast<unsigned>(p.tpu));
        j_begin = first - u_begin * p.tpu;
        n_tiles = n;
      }
    }
  }
  TileCursor c0;
  c0.init(u_begin, j_begin, p);

  if (tid == 0) {
    for (int s = 0; s < NST; ++s) {
      mbar_init(&full_bar[s], 1);        // the producer's arrive (plus tracked cp.async arrivals)
      mbar_init(&empty_bar[s], kWarps);  // one arrive per consumer warp
    }
    attn_abort = 0;
    asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
  }
  if (tid == 32 && p.cm > 0) {  // the groups this CTA finishes and the heads' (max, sum), from each rank
    const int mine = min(max(G * D / 4 - j_begin * p.slice, 0), p.slice);
    mbar_init(&recv_bar, 1);
    asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
    mbar_arrive_expect_tx(&recv_bar, static_cast<uint32_t>(p.cm * (mine * 16 + G * 8)) + p.stall_tx);
  }
  __syncthreads();
  if (p.cm > 0) cluster_arrive();  // waited for before the first store into a peer
  // Before the grid dependency wait: the first tiles into L2.
  if (lane == 0 && warp < kWarps) {
    prefetch_map((warp & 1) && p.k > 0 ? &maps.t1 : &maps.ring);
    TileCursor cp = c0;
    const int npf = n_tiles < p.l2_prefetch ? n_tiles : p.l2_prefetch;
    for (int i = 0; i < npf; ++i) {
      if (i % kWarps == warp) tma_box3_prefetch(tile_map(p, maps, cp), tile_row(p, cp), 2 * cp.u);
      cp.next(p);
    }
  }
  int last_b = c0.b;  // the sequence of the CTA's last tile (how far pos is read ahead)
  if (warp == kWarps) {
    if (lane == 0 && p.l2_prefetch > 0)
      bulk_prefetch_l2(p.q + static_cast<long long>(c0.u) * (G * D), G * D * 2);
    if (p.cm == 0 && n_tiles > p.tpu)
      last_b = static_cast<int>(static_cast<unsigned>(c0.u + (c0.j + n_tiles - 1) / p.tpu) /
                                static_cast<unsigned>(p.LH));
    else if (p.cm == 0 && c0.j + n_tiles > p.tpu && c0.left == 1)
      last_b = c0.b + 1;
  }
  unsigned long long turns[2] = {0ull, 0ull};  // this producer lane's rotary frequencies
  if (FUSED && warp == kWarps && p.rope) {
    if (p.rope_slot >= 0) {
      turns[0] = g_rope_tables[p.rope_slot][lane];
      if (lane + 32 < D / 2) turns[1] = g_rope_tables[p.rope_slot][lane + 32];
    } else {
      turns[0] = p.rope_turns[lane];
      if (lane + 32 < D / 2) turns[1] = p.rope_turns[lane + 32];
    }
  }
  asm volatile("griddepcontrol.wait;\n" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");

  if (warp == kWarps) {
    // ======================= producer warp =======================
    long long* pos_s = reinterpret_cast<long long*>(hdr0 + 4 * H_POS);
    if (lane == 0) {
      cp_async_8(smem_addr(pos_s), p.pos + c0.b);
      bulk_copy(smem_addr(slot0 + S::kQ), p.q + static_cast<long long>(c0.u) * (G * D), G * D * 2,
                &full_bar[0]);
    }
    cp_async_commit();
    // the first stages' powers of two: they do not depend on pos
    TileCursor ci = c0;
#pragma unroll
    for (int i = 0; i < NST; ++i) {
      if (i < n_tiles && lane < 2) {
        load_scales(p, ci, hdr0 + i * 32, lane);
        mbar_arrive_cp_async(&full_bar[i]);
      }
      ci.next(p);
    }
    cp_async_commit();
    ci = c0;
    int run_b = ci.b;        // sequence of the current run of tiles
    long long pos_next = 0;  // pos of the sequence after it, ahead of its use
    if (run_b < last_b) pos_next = ld_pos(p, run_b + 1);
    int issued = 0;
    int run_tiles = 0;       // tiles in that run so far
    int slot = 0;            // the unit's slot
    float2 rope[2] = {make_float2(1.f, 0.f), make_float2(1.f, 0.f)};
    cp_async_wait<1>();
    __syncwarp();  // pos has landed
    SeqState sq = seq_state<FUSED>(p, *pos_s);
    if (FUSED && p.rope && !sq.bad) rope_pairs<D>(p, sq.pos, turns, lane, rope);
    for (int i = 0; i < n_tiles; ++i) {
      const int s = i % NST;
      uint8_t* hdr = hdr0 + s * 32;
      if (i >= NST) {
        int ok = 0;
        if (lane == 0) ok = mbar_wait(&empty_bar[s], static_cast<uint32_t>((i / NST - 1) & 1)) ? 1 : 0;
        __syncwarp();
        ok = __shfl_sync(0xffffffffu, ok, 0);
        if (!ok) break;
      }
      const bool with_q = i == 0 || (p.cm == 0 && ci.j == 0);  // a unit's first tile in this CTA
      if (with_q && i > 0) slot = slot == NST - 1 ? 0 : slot + 1;
      uint8_t* aux = slot0 + slot * S::kSlot;
      if (ci.b != run_b) {  // a new sequence: pos-derived state, once per run
        if (FUSED && lane == 0) seq_run_done(p, run_b, run_tiles, sq);
        run_b = ci.b;
        run_tiles = 0;
        sq = seq_state<FUSED>(p, pos_next);
        if (FUSED && p.rope && !sq.bad) rope_pairs<D>(p, sq.pos, turns, lane, rope);
        if (run_b < last_b) pos_next = ld_pos(p, run_b + 1);
      }
      ++run_tiles;
      const bool t1 = ci.lt < p.t1_tiles;
      const int r0 = tile_row(p, ci);
      int n_rows, new_row = -1;
      if (t1) {
        n_rows = sq.bad ? 0 : min(p.k - r0, kQ8Tile);
      } else {
        n_rows = min(max(sq.count - r0, 0), kQ8Tile);
        if (FUSED && sq.new_slot >= r0 && sq.new_slot - r0 < n_rows) new_row = sq.new_slot - r0;
      }
      // (a tile without keys is loaded only among the first stages, before pos is known)
      const bool loaded = i < NST || n_rows > 0;
      if (i >= NST && loaded) {
        if (lane < 2) {
          load_scales(p, ci, hdr, lane);
          mbar_arrive_cp_async(&full_bar[s]);
        }
        if (lane == 0)
          tma_box3_hint(smem_addr(smem + s * S::kStage), tile_map(p, maps, ci), r0, 2 * ci.u, &full_bar[s],
                        policy_evict_first());
      }
      if (FUSED && p.rope && with_q) {
        float2* tab = reinterpret_cast<float2*>(aux + S::kRope);
        tab[lane] = rope[0];
        if (lane + 32 < D / 2) tab[lane + 32] = rope[1];
      }
      __syncwarp();
      if (lane == 0) {
        if (sq.bad && ci.lt == 0) atomicOr(p.status, CMC_DEVFLAG_BAD_POS);
        int* hw = reinterpret_cast<int*>(hdr);
        hw[H_NROWS] = n_rows;
        hw[H_NEWSLOT] = sq.new_slot;
        hw[H_NEWROW] = new_row;
        uint32_t tx = p.stall_tx;
        if (loaded) tx += S::kStage;
        if (with_q) tx += G * D * 2;
        if (new_row >= 0) tx += 2 * D * 2;
        mbar_arrive_expect_tx(&full_bar[s], tx);  // releases the header
        if (with_q && i > 0)
          bulk_copy(smem_addr(aux + S::kQ), p.q + static_cast<long long>(ci.u) * (G * D), G * D * 2,
                    &full_bar[s]);
        if (new_row >= 0) {
          bulk_copy(smem_addr(aux + S::kNew), p.k_new + static_cast<long long>(ci.u) * D, D * 2, &full_bar[s]);
          bulk_copy(smem_addr(aux + S::kNew + D * 2), p.v_new + static_cast<long long>(ci.u) * D, D * 2,
                    &full_bar[s]);
        }
      }
      ci.next(p);
      issued = i + 1;
    }
    if (FUSED && issued == n_tiles && lane == 0) seq_run_done(p, run_b, run_tiles, sq);
    cp_async_wait<0>();
    // No CTA exits while loads it issued may still be writing into its shared
    // memory: the last stage's barrier covers them, and after a timeout, when
    // barriers are no evidence, kDrainNs does (every load was issued before it).
    if (lane == 0 && issued > 0 &&
        (!mbar_wait(&full_bar[(issued - 1) % NST], static_cast<uint32_t>(((issued - 1) / NST) & 1)) ||
         attn_aborted())) {
      const uint32_t t0 = global_ns32();
      for (uint32_t it = 0; it < (1u << 16) && global_ns32() - t0 < kDrainNs; ++it) __nanosleep(1000);
    }
    if (lane == 0 && attn_aborted()) atomicOr(p.status, CMC_DEVFLAG_TIMEOUT);
    __syncwarp();
    if (p.cm > 0) cluster_wait();  // every thread that arrived waits
    return;
  }

  // ======================= consumer warps =======================
  // The boxes of the first stages, one warp each: they do not depend on pos.
  if (lane == 0) {
    TileCursor cl = c0;
#pragma unroll
    for (int i = 0; i < NST; ++i) {
      if (i == warp && i < n_tiles)
        tma_box3_hint(smem_addr(smem + i * S::kStage), tile_map(p, maps, cl), tile_row(p, cl), 2 * cl.u,
                      &full_bar[i], policy_evict_first());
      cl.next(p);
    }
  }
  __syncwarp();
  // gq = lane / 4, tq = lane % 4.  A thread's two heads (columns 2 tq, 2 tq + 1 of the
  // products): h0 + e, e = 0, 1; for G <= 4 threads with tq >= 2 have the lo pieces.
  const int gq = lane >> 2;
  const int tq = lane & 3;
  const int h0 = PAIRED ? 2 * (tq & 1) : 2 * tq;
  TileCursor cc = c0;
  int cur_u = -1, first_j = 0, slot = -1;
  uint32_t qa[KS][2], qb[PAIRED ? 1 : KS][2];  // Q^T fragments: hi (or both pieces); G = 8: lo
  float qs[2] = {0.f, 0.f};                    // softmax scale * log2(e) * the heads' powers of two
  float m_run[2] = {-INFINITY, -INFINITY}, l_run[2] = {0.f, 0.f};
  int e_cur = 0, e_top = 0;                    // the byte O is in units of; the largest so far
  float o[MT][4];
#pragma unroll
  for (int j = 0; j < MT; ++j) o[j][0] = o[j][1] = o[j][2] = o[j][3] = 0.f;
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) {
    qa[ks][0] = qa[ks][1] = 0u;
    if (!PAIRED) qb[ks][0] = qb[ks][1] = 0u;
  }
  int release = lane;  // 0: this lane hands the warp's stages back

  for (int i = 0; i < n_tiles; ++i) {
    const int s = i % NST;
    uint8_t* stage = smem + s * S::kStage;
    uint8_t* hdr = hdr0 + s * 32;
    // A stage whose wait gave up is skipped by every lane alike: no key, no patch.
    const bool dead = __any_sync(0xffffffffu, !mbar_wait_stage(&full_bar[s], static_cast<uint32_t>((i / NST) & 1),
                                                               reinterpret_cast<int*>(hdr), release));
    const int4 hw = reinterpret_cast<const int4*>(hdr)[0];  // rows, slot, row
    const int u = cc.u;
    if (u != cur_u) slot = slot == NST - 1 ? 0 : slot + 1;
    const uint8_t* aux = slot0 + slot * S::kSlot;
    int kc = hdr[4 * H_KSCALES + warp], vc = hdr[4 * H_VSCALES + warp];
    // bit r: row r of this warp's 32 holds a key
    const int nk = dead ? 0 : min(max(hw.x - 32 * warp, 0), 32);
    const uint32_t mk = nk == 32 ? 0xFFFFFFFFu : (1u << nk) - 1u;
    const int new_row = dead ? -1 : hw.z;
    bool wrote_stage = false;  // generic-proxy writes into the stage by this warp

    if (FUSED && new_row >= 0 && (new_row >> 5) == warp) {
      const int r = new_row & 31;
      const uint32_t others = mk & ~(1u << r);
      const bool first = (hw.y & 31) == 0;
      // ring rows of the block: slot hw.y is row r
#pragma unroll
      for (int w = 0; w < 2; ++w) {
        const uint16_t* row = reinterpret_cast<const uint16_t*>(aux + S::kNew + w * D * 2);
        float x[4] = {0.f, 0.f, 0.f, 0.f};
        constexpr int E = D / 32;
#pragma unroll
        for (int e = 0; e < E; ++e) x[e] = bf16lo_to_f32(row[E * lane + e]);
        if (w == 0 && p.rope) {  // elements c pair with c + d/2
          const float2* tab = reinterpret_cast<const float2*>(aux + S::kRope);
          const float sg = lane < 16 ? -1.f : 1.f;
#pragma unroll
          for (int e = 0; e < E; ++e) {
            const float2 cs = tab[(E * lane + e) & (D / 2 - 1)];
            x[e] = fmaf(x[e], cs.x, sg * bf16lo_to_f32(row[(E * lane + e) ^ (D / 2)]) * cs.y);
          }
        }
        const long long uw = 2LL * u + w;
        uint8_t* ring0 = p.ring_kv + (uw * p.W + hw.y - r) * D;
        const int c = patch_block<D>(stage + w * S::kV, ring0, p.ring_scales + uw * p.ringS + (hw.y >> 5), x, r,
                                     w ? vc : kc, first, others, lane, warp);
        if (w) vc = c;
        else kc = c;
      }
      __syncwarp();
      wrote_stage = true;
    }

    if (u != cur_u) {  // first tile of a unit in this CTA
      cur_u = u;
      first_j = cc.j;
      // The query as two e4m3 pieces.  Thread: head (column) gq, of the elements
      // 32 ks + 16 hf + 4 tq .. + 3; those and the other three tq's are the head.
      const int head = PAIRED ? (gq & 3) : gq;
      const uint8_t* qrow = aux + S::kQ + head * D * 2;
      float x[KS][2][4];
#pragma unroll
      for (int ks = 0; ks < KS; ++ks)
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
          uint2 w = make_uint2(0u, 0u);
          if (head < G && !dead) w = *reinterpret_cast<const uint2*>(qrow + (32 * ks + 16 * hf + 4 * tq) * 2);
          x[ks][hf][0] = bf16lo_to_f32(w.x); x[ks][hf][1] = bf16hi_to_f32(w.x);
          x[ks][hf][2] = bf16lo_to_f32(w.y); x[ks][hf][3] = bf16hi_to_f32(w.y);
        }
      if (FUSED && p.rope && !dead) {  // k-steps ks and ks + KS/2 hold the partners
        const float2* tab = reinterpret_cast<const float2*>(aux + S::kRope);
#pragma unroll
        for (int ks = 0; ks < KS / 2; ++ks)
#pragma unroll
          for (int hf = 0; hf < 2; ++hf)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float2 cs = tab[32 * ks + 16 * hf + 4 * tq + e];
              const float a = x[ks][hf][e], b = x[ks + KS / 2][hf][e];
              x[ks][hf][e] = fmaf(a, cs.x, -b * cs.y);
              x[ks + KS / 2][hf][e] = fmaf(b, cs.x, a * cs.y);
            }
      }
      uint32_t top = 0u;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks)
#pragma unroll
        for (int hf = 0; hf < 2; ++hf)
#pragma unroll
          for (int e = 0; e < 4; ++e) top = max(top, finite_bits(x[ks][hf][e]));
      top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
      top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
      const int qc = block_code(top);
      const float f = code_factor(qc);
#pragma unroll
      for (int ks = 0; ks < KS; ++ks)
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
          float y[4], h[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) y[e] = scaled(x[ks][hf][e], f);
          const uint32_t hi = e4m3_pair(y[0], y[1]) | (e4m3_pair(y[2], y[3]) << 16);
          decode4(hi, h);
#pragma unroll
          for (int e = 0; e < 4; ++e) y[e] = 16.f * (y[e] - h[e]);
          const uint32_t lo = e4m3_pair(y[0], y[1]) | (e4m3_pair(y[2], y[3]) << 16);
          if (PAIRED) {
            qa[ks][hf] = gq < 4 ? hi : lo;
          } else {
            qa[ks][hf] = hi;
            qb[ks][hf] = lo;
          }
        }
      const float qscale = e8m0_to_f32(qc) * p.scale_log2;
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        qs[e] = __shfl_sync(0xffffffffu, qscale, 4 * (h0 + e));
        m_run[e] = -INFINITY;
        l_run[e] = 0.f;
      }
      e_cur = e_top = -1;
#pragma unroll
      for (int j = 0; j < MT; ++j) o[j][0] = o[j][1] = o[j][2] = o[j][3] = 0.f;
    }

    if (mk != 0u) {
      if (mk != 0xFFFFFFFFu) {
        // Zero the V rows that hold no key: their probabilities are 0, but 0 times NaN is not.
        if (!((mk >> lane) & 1u)) {
#pragma unroll
          for (int q = 0; q < D / 16; ++q)
            *reinterpret_cast<uint4*>(stage + S::kV + swz8<D>(32 * warp + lane, q)) = make_uint4(0u, 0u, 0u, 0u);
        }
        __syncwarp();
        wrote_stage = true;
      }
      const uint32_t sK = smem_addr(stage);
      const uint32_t sV = smem_addr(stage + S::kV);
      // ---- S^T = K Q^T, two products of 16 keys ----
      float sa[2][4], sb[2][4];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        // lanes 0-7 / 8-15 / 16-23 / 24-31: rows 0-7 / 8-15 / 0-7 / 8-15 of the product, at
        // bytes 32 ks .. + 15 / same / 32 ks + 16 .. + 31 / same
        const int key = 32 * warp + 16 * t + ((lane & 7) ^ (4 * t)) + ((lane >> 3) & 1) * 8;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          uint32_t a0, a1, a2, a3;
          ldsm_x4(sK + swz8<D>(key, 2 * ks + (lane >> 4)), a0, a1, a2, a3);
          if (ks == 0) mma_e4m3_zero(sa[t], a0, a1, a2, a3, qa[ks][0], qa[ks][1]);
          else mma_e4m3(sa[t], a0, a1, a2, a3, qa[ks][0], qa[ks][1]);
          if (!PAIRED) {
            if (ks == 0) mma_e4m3_zero(sb[t], a0, a1, a2, a3, qb[ks][0], qb[ks][1]);
            else mma_e4m3(sb[t], a0, a1, a2, a3, qb[ks][0], qb[ks][1]);
          }
        }
      }
      // ---- the thread's scores, log2 domain: v[e][t], head h0 + e of row gq (tq < 2) or
      // gq + 8 of product t; for G = 8, v[e][2 t + r] of row gq + 8 r ----
      const float ks2 = e8m0_to_f32(kc);
      float v[2][NV];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const float f = qs[e] * ks2;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          if (PAIRED) {
            // threads tq < 2 have the hi column of rows gq and gq + 8, threads tq + 2 the lo
            // column: they exchange what the other needs and keep one row each
            const float give = tq < 2 ? sa[t][2 + e] : sa[t][e];
            const float keep = tq < 2 ? sa[t][e] : sa[t][2 + e];
            const float got = __shfl_xor_sync(0xffffffffu, give, 2);
            v[e][t] = (tq < 2 ? fmaf(got, 0.0625f, keep) : fmaf(keep, 0.0625f, got)) * f;
          } else {
            v[e][2 * t] = fmaf(sb[t][e], 0.0625f, sa[t][e]) * f;
            v[e][2 * t + 1] = fmaf(sb[t][2 + e], 0.0625f, sa[t][2 + e]) * f;
          }
        }
      }
      if (mk != 0xFFFFFFFFu) {
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int r = 0; r < NV / 2; ++r) {
            const int row = gq + 8 * (PAIRED ? tq >> 1 : r);
            if (!((mk >> (16 * t + (row ^ (4 * t)))) & 1u))
              v[0][t * (NV / 2) + r] = v[1][t * (NV / 2) + r] = -INFINITY;
          }
      }
      // ---- online softmax ----
      float mx[2];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        mx[e] = v[e][0];
#pragma unroll
        for (int n = 1; n < NV; ++n) mx[e] = fmaxf(mx[e], v[e][n]);
#pragma unroll
        for (int off = PAIRED ? 2 : 4; off < 32; off <<= 1)
          mx[e] = fmaxf(mx[e], __shfl_xor_sync(0xffffffffu, mx[e], off));
      }
      // The unit of O: at least 2^-64 of the largest block's, so that O stays far inside fp32.
      int e_new = e_cur;
      if (vc != 255) {
        e_top = max(e_top, vc);
        const int want = max(vc, e_top - 64);
        if (want > e_cur || want + 4 < e_cur) e_new = want;
      }
      const bool up0 = mx[0] > m_run[0], up1 = mx[1] > m_run[1];
      if (__any_sync(0xffffffffu, up0 || up1 || e_new != e_cur)) {
        // (with e_cur = -1, before the first block, O is zero)
        const float fe = e_cur < 0 ? 1.f : recode_factor(e_cur, max(e_new, 0));
        e_cur = e_new;
        const float alpha0 = up0 ? ex2(m_run[0] - mx[0]) : 1.f;
        const float alpha1 = up1 ? ex2(m_run[1] - mx[1]) : 1.f;
        if (up0) m_run[0] = mx[0];
        if (up1) m_run[1] = mx[1];
        l_run[0] *= alpha0;
        l_run[1] *= alpha1;
        const float f0 = alpha0 * fe, f1 = alpha1 * fe;
#pragma unroll
        for (int j = 0; j < MT; ++j) {
          o[j][0] *= f0;
          o[j][1] *= f1;
          o[j][2] *= f0;
          o[j][3] *= f1;
        }
      }
      // 256 times the probabilities; times V's power of two in O's unit
      const float pv = vc == 255 ? e8m0_to_f32(255) : recode_factor(vc, e_cur);
      float pr[2][NV];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const float ref = m_run[e] == -INFINITY ? 0.f : m_run[e] - 8.f;
#pragma unroll
        for (int n = 0; n < NV; ++n) {
          pr[e][n] = ex2(v[e][n] - ref);
          l_run[e] += pr[e][n];
          pr[e][n] *= pv;
        }
      }
      // ---- P^T as the B operand: 16-bit elements (key of product 0, key of product 1) ----
      uint32_t b0, b1, b2, b3;
      if (PAIRED) {
        uint32_t hi0, lo0, hi1, lo1;
        two_pieces(pr[0][0], pr[0][1], hi0, lo0);
        two_pieces(pr[1][0], pr[1][1], hi1, lo1);
        const uint32_t hi = hi0 | (hi1 << 16), lo = lo0 | (lo1 << 16);
        // columns 0-3 hi, 4-7 lo; first the rows gq, then the rows gq + 8
        const uint32_t got = __shfl_xor_sync(0xffffffffu, tq < 2 ? lo : hi, 2);
        b0 = movmatrix_trans(tq < 2 ? hi : got);
        b1 = movmatrix_trans(tq < 2 ? got : lo);
        b2 = b3 = 0u;
      } else {
        uint32_t hi[2][2], lo[2][2];  // [head][row]
#pragma unroll
        for (int e = 0; e < 2; ++e)
#pragma unroll
          for (int r = 0; r < 2; ++r) two_pieces(pr[e][r], pr[e][2 % NV + r], hi[e][r], lo[e][r]);
        b0 = movmatrix_trans(hi[0][0] | (hi[1][0] << 16));
        b1 = movmatrix_trans(hi[0][1] | (hi[1][1] << 16));
        b2 = movmatrix_trans(lo[0][0] | (lo[1][0] << 16));
        b3 = movmatrix_trans(lo[0][1] | (lo[1][1] << 16));
      }
      // ---- O^T += V^T P^T: lane's V row is k = lane of the product ----
      {
        const int row = 2 * ((lane & 15) >> 2) + ((lane >> 1) & 1) + 8 * (lane >> 4);
        const int key = 32 * warp + ((lane & 1) ? 16 + (row ^ 4) : row);
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
          uint32_t a0, a1, a2, a3;
          ldsm_b8_t(sV + swz8<D>(key, mt), a0, a1, a2, a3);
          mma_e4m3(o[mt], a0, a1, a2, a3, b0, b1);
          if (!PAIRED) {
            float x[4];
            mma_e4m3_zero(x, a0, a1, a2, a3, b2, b3);
#pragma unroll
            for (int e = 0; e < 4; ++e) o[mt][e] = fmaf(x[e], 0.0625f, o[mt][e]);
          }
        }
      }
    }

    // ---- end of a unit within this CTA: merge warps, write out or a partial ----
    const bool unit_end = (i + 1 == n_tiles) || (p.cm == 0 && cc.j == p.tpu - 1);
    if (unit_end) {
      // Every warp leaves its maximum and sum, and its unnormalised output in its own 32
      // rows of the stage's K (8 columns of d floats: just their size), columns of odd
      // pairs shifted so that the stores hit distinct banks.  After a barrier each
      // thread takes four rows of the head dimension of one head, rescales and adds
      // the warps' in warp order.
#pragma unroll
      for (int e = 0; e < 2; ++e)
#pragma unroll
        for (int off = PAIRED ? 2 : 4; off < 32; off <<= 1)
          l_run[e] += __shfl_xor_sync(0xffffffffu, l_run[e], off);
      __syncwarp();  // the warp is done with its K rows
      {
        float* ow = reinterpret_cast<float*>(stage) + warp * 8 * D;
        const float fo = e_cur < 0 ? 0.f : e8m0_to_f32(e_cur);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          float* col = ow + (2 * tq + e) * D;
#pragma unroll
          for (int j = 0; j < MT; ++j) {
            col[(16 * j + gq) ^ (8 * tq)] = o[j][e] * fo;
            col[(16 * j + 8 + gq) ^ (8 * tq)] = o[j][2 + e] * fo;
          }
          if (gq == 0 && (!PAIRED || tq < 2)) {
            merge_m[warp * 8 + h0 + e] = m_run[e];
            merge_l[warp * 8 + h0 + e] = l_run[e];
          }
        }
      }
      wrote_stage = true;
      consumer_sync();

      const bool whole = p.cm == 0 && first_j == 0 && cc.j == p.tpu - 1;
      const long long out_base = static_cast<long long>(u) * (G * D);
      constexpr int NGR = G * D / 4;                        // 4-row groups of the unit's output
      constexpr int XPT = (NGR + kThreads - 1) / kThreads;  // groups per thread
      const bool clus = !whole && p.cm > 0;
      float4 cacc[XPT];
      float cls[XPT], cmx[XPT];
#pragma unroll
      for (int xi = 0; xi < XPT; ++xi) {
        const int x = tid + xi * kThreads;
        if (x >= NGR) break;
        const int hh = (4 * x) / D;
        const int c = (4 * x) % D;
        float M = merge_m[hh];
#pragma unroll
        for (int w = 1; w < kWarps; ++w) M = fmaxf(M, merge_m[w * 8 + hh]);
        const float Mr = M == -INFINITY ? 0.f : M;  // (a NaN among the warps' outputs stays one)
        float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
        float Ls = 0.f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
          const float f = ex2(merge_m[w * 8 + hh] - Mr);
          const float* ow = reinterpret_cast<const float*>(stage) + w * 8 * D;
          float4 y = *reinterpret_cast<const float4*>(ow + hh * D + (c ^ (8 * (hh >> 1))));
          if (PAIRED) {
            const int hl = hh + 4;
            const float4 z = *reinterpret_cast<const float4*>(ow + hl * D + (c ^ (8 * (hl >> 1))));
            y.x = fmaf(z.x, 0.0625f, y.x); y.y = fmaf(z.y, 0.0625f, y.y);
            y.z = fmaf(z.z, 0.0625f, y.z); y.w = fmaf(z.w, 0.0625f, y.w);
          }
          acc.x = fmaf(f, y.x, acc.x); acc.y = fmaf(f, y.y, acc.y);
          acc.z = fmaf(f, y.z, acc.z); acc.w = fmaf(f, y.w, acc.w);
          Ls = fmaf(f, merge_l[w * 8 + hh], Ls);
        }
        if (whole) {
          const float inv = Ls > 0.f ? __fdividef(1.f, Ls) : 0.f;
          *reinterpret_cast<uint2*>(p.out + out_base + hh * D + c) =
              make_uint2(pack_bf16_rn(acc.x * inv, acc.y * inv), pack_bf16_rn(acc.z * inv, acc.w * inv));
        } else if (clus) {  // merged across the cluster below
          cacc[xi] = acc;
          cls[xi] = Ls;
          cmx[xi] = M;
        } else {  // merged by two_tier_combine_kernel
          constexpr int PW = rec_floats(G, D);
          float* rec = p.partials + (static_cast<long long>(u) * p.tpu + first_j) * PW;
          if (c == 0) {
            rec[hh] = M;
            rec[G + hh] = Ls;
          }
          *reinterpret_cast<float4*>(rec + rec_out_offset(G) + hh * D + c) = acc;
        }
      }
      if (clus) {
        // One share of the unit per CTA: stored into the peers' receive areas, to each the
        // groups that peer finishes; then merged in rank order (see cmc_attn.cu).
        const int cm = p.cm;
        const int rank = static_cast<int>(cluster_ctarank());
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
          const float2* ml = reinterpret_cast<const float2*>(smem + S::kRecvMl) + hh;
          float M = -INFINITY;
#pragma unroll
          for (int r = 0; r < kMaxClusterCtas; ++r)
            if (r < cm) M = fmaxf(M, ml[r * G].x);
          if (M == -INFINITY) M = 0.f;
          float Ls = 0.f;
          float4 O = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
          for (int r = 0; r < kMaxClusterCtas; ++r) {
            if (r < cm) {
              const float2 mr = ml[r * G];
              const float4 o4 = *reinterpret_cast<const float4*>(smem + S::kRecv + (r * SL + x - x0) * 16);
              const float f = ex2(mr.x - M);
              Ls = fmaf(f, mr.y, Ls);
              O.x = fmaf(f, o4.x, O.x);
              O.y = fmaf(f, o4.y, O.y);
              O.z = fmaf(f, o4.z, O.z);
              O.w = fmaf(f, o4.w, O.w);
            }
          }
          const float inv = Ls > 0.f ? __frcp_rn(Ls) : 0.f;
          *reinterpret_cast<uint2*>(p.out + out_base + hh * D + c) =
              make_uint2(pack_bf16_rn(O.x * inv, O.y * inv), pack_bf16_rn(O.z * inv, O.w * inv));
        }
      }
      if (i + 1 < n_tiles) consumer_sync();  // merge_m and merge_l are written again by the next unit
    }
    if (wrote_stage) {
      // generic-proxy writes to this stage are ordered before the producer's next box
      asm volatile("fence.proxy.async.shared::cta;\n" ::: "memory");
    }
    __syncwarp();
    if (release == 0) mbar_arrive(&empty_bar[s]);  // this warp is done with stage s
    cc.next(p);
  }
  if (tid == 0 && attn_aborted()) atomicOr(p.status, CMC_DEVFLAG_TIMEOUT);
}

// ---------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------

// rows of T codes rows of every (unit, K or V), `stride` rows apart.
static bool encode_q8(CUtensorMap* map, const void* base, long long units2, int T, int stride, int d) {
  EncodeTiledFn enc = encode_fn();
  if (!enc) return false;
  cuuint64_t dims[3] = {static_cast<cuuint64_t>(d), static_cast<cuuint64_t>(T), static_cast<cuuint64_t>(units2)};
  cuuint64_t strides[2] = {static_cast<cuuint64_t>(d), static_cast<cuuint64_t>(stride) * d};
  cuuint32_t box[3] = {static_cast<cuuint32_t>(d), kQ8Tile, 2};
  cuuint32_t es[3] = {1, 1, 1};
  return enc(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 3, const_cast<void*>(base), dims, strides, box, es,
             CU_TENSOR_MAP_INTERLEAVE_NONE, d == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B,
             CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

static int q8_tiles(int rows) { return (rows + kQ8Tile - 1) / kQ8Tile; }

template <int D, int G, bool FUSED>
static int plan_q8(long long tiles, int tpu, AttnPlan* pl) {
  constexpr int smem = Q8Smem<D, G>::kBytes;
  auto kern = attn_q8_kernel<D, G, FUSED>;
  static std::atomic<int> configured[64];  // per device: attribute set and occupancy known (idempotent)
  int dev = 0;
  int st = record_cuda_error(cudaGetDevice(&dev));
  if (st != CMC_OK) return st;
  int per_sm = (dev >= 0 && dev < 64) ? configured[dev].load(std::memory_order_acquire) : 0;
  if (per_sm <= 0) {
    st = record_cuda_error(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
    if (st != CMC_OK) return st;
    st = record_cuda_error(cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, kern, kThreads + 32, smem));
    if (st != CMC_OK) return st;
    if (per_sm < 1) per_sm = 1;
    if (dev >= 0 && dev < 64) configured[dev].store(per_sm, std::memory_order_release);
  }
  plan_grid(tiles, tpu, per_sm, pl);
  return CMC_OK;
}

template <int D, int G, bool FUSED>
static int launch_q8(const Q8Maps& maps, AttnQ8Params p, long long tiles, cudaStream_t s) {
  AttnPlan pl;
  int st = plan_q8<D, G, FUSED>(tiles, p.tpu, &pl);
  if (st != CMC_OK) return st;
  p.base = static_cast<int>(pl.base);
  p.rem = static_cast<int>(pl.rem);
  p.cm = pl.cm;
  p.gran = pl.gran;
  p.slice = pl.cm > 0 ? (G * D / 4 + pl.cm - 1) / pl.cm : 0;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = static_cast<unsigned>(pl.cm > 0 ? pl.cm : 1);
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(pl.ctas));
  cfg.blockDim = dim3(kThreads + 32);
  cfg.dynamicSmemBytes = Q8Smem<D, G>::kBytes;
  cfg.stream = s;
  cfg.attrs = attr;
  cfg.numAttrs = pl.cm > 0 ? 2 : 1;
  st = record_cuda_error(cudaLaunchKernelEx(&cfg, attn_q8_kernel<D, G, FUSED>, maps, p));
  if (st != CMC_OK || !pl.split) return st;
  return launch_pdl(two_tier_combine_kernel<D, G>, dim3(static_cast<unsigned>(tiles / p.tpu)), dim3(kThreads),
                    0, s, static_cast<const AttnParams&>(p));
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
  static int run(bool fused, long long tiles, int tpu, AttnPlan* pl) {
    return fused ? plan_q8<D, G, true>(tiles, tpu, pl) : plan_q8<D, G, false>(tiles, tpu, pl);
  }
};
template <int D, int G>
struct LaunchQ8 {
  static int run(bool fused, const Q8Maps& maps, const AttnQ8Params& p, long long tiles, cudaStream_t s) {
    return fused ? launch_q8<D, G, true>(maps, p, tiles, s) : launch_q8<D, G, false>(maps, p, tiles, s);
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
  if (!workspace || workspace_bytes < cmc_decode_attn_workspace_size(dims)) return CMC_ERR_WORKSPACE;
  if (!aligned16(workspace)) return CMC_ERR_ALIGN;

  const long long units = static_cast<long long>(m.B) * m.L * m.Hkv;
  const int t1_tiles = q8_tiles(m.k);
  const int tpu = t1_tiles + q8_tiles(m.W);
  const long long tiles = units * tpu;
  if (tiles >= (1LL << 31)) return CMC_ERR_SHAPE;

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
  p.partials = reinterpret_cast<float*>(ws + ws_partials_off(m.B));
  p.B = m.B; p.L = m.L; p.Hq = m.Hq; p.Hkv = m.Hkv; p.N = m.N; p.k = m.k; p.W = m.W;
  p.tpu = tpu;
  p.LH = m.L * m.Hkv;
  p.t1_tiles = t1_tiles;
  const float sc = scale > 0.f ? scale : 1.0f / sqrtf(static_cast<float>(m.d));
  p.scale_log2 = sc * 1.4426950408889634f;
  p.l2_prefetch = l2_prefetch_setting();
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
  return by_shape<LaunchQ8>(m.d, m.Hq / m.Hkv, fused, maps, p, tiles, s);
}

}  // namespace cmc

extern "C" {

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

int cmc_decode_attn_q8_plan(const cmc_dims* dims, int fused, int* ctas, int* launches) {
  using namespace cmc;
  int st = validate_dims(dims, true);
  if (st != CMC_OK) return st;
  if (!ctas || !launches) return CMC_ERR_NULL;
  const cmc_dims& m = *dims;
  const int tpu = q8_tiles(m.k) + q8_tiles(m.W);
  const long long tiles = static_cast<long long>(m.B) * m.L * m.Hkv * tpu;
  if (tiles >= (1LL << 31)) return CMC_ERR_SHAPE;
  AttnPlan pl;
  st = by_shape<PlanQ8>(m.d, m.Hq / m.Hkv, fused != 0, tiles, tpu, &pl);
  if (st != CMC_OK) return st;
  *ctas = static_cast<int>(pl.ctas);
  *launches = pl.split ? 2 : 1;
  return CMC_OK;
}

}  // extern "C"
