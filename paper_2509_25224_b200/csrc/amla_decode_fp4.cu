// Tensor-core MLA decode kernel for a cache held in 4 bits (format: amla_fp4.cuh), sm_100a.
//
// A key is 324 bytes.  Widened to 16 bits it is 1152 for K and 1024 for V, and a kernel that keeps widened operands in shared
// memory writes and reads all of that there.  Here they never are in shared memory: the raw page is, and the widening warps put what
// they make of it straight into tensor memory, as the A operand of transposed products.  With that the rows are N:
//
//   S^T = K Q^T       A = K: 128 keys (two pages) are the lanes, 64 of the 576 columns at a time; B = Q (shared memory, K-major)
//   O^T += V^T P~^T   A = V^T: V's columns are the lanes, 2 x 128 of them and 32 keys at a time; B = P~ (shared memory, MN-major)
//
// One CTA works on up to 16, 32 or 64 rows of a sequence and a range of its pages; O^T is four blocks of kN columns of tensor
// memory (256 for 64 rows), S^T two of kN, and the rest a ring of operand chunks of 32 columns.  A 128-key tile is 17 chunks: nine of K
// (128 keys x 64 columns), eight of V (256 columns x 32 keys), four MMAs each.
//
// Everything is f16, not bf16: an E2M1 times an E4M3 number is exact in either, P~ has three more bits, and the conversion from
// E2M1 gives f16.  Q is bf16: a row is multiplied by the power of two that brings its largest magnitude into [2^14, 2^15), which
// leaves every element within 2^-32 of the row's largest exact, and smaller ones off by at most 2^-25 in units of which the largest has 2^14.
//
// The reference of the online softmax is an integer number of octaves n, so that a rescale of O and l is an add to the exponent
// bits and exact (nothing is left over to compensate).  P~ = 2^(a_j - n + 9): a move puts the largest P~ of a row into (2^8, 2^9], the
// next one comes when a key would exceed 2^15, and what f16 rounds to nothing is below 2^-33 of the reference.
//
// Warps 0-3: Q into f16, softmax (a thread is a key and has all rows; its share of the row sums stays in registers until the unit's
// end), rescale, epilogue.  Warps 4-11 widen K and 12-19 V, four at a time by turns; warp 20 issues the products of K, 21
// those of V; warp 22 loads pages (bulk copies).
//
// All waits are bounded; on expiry the kernel records kStatusTimeout and unwinds.
#define AMLA_SELDOM __forceinline__
#include "amla_common.cuh"
#include "amla_fp4.cuh"
#include "amla_host.cuh"
#include "amla_sm100.cuh"
#include "amla_units.cuh"

namespace amla {

using namespace sm100;

namespace {

constexpr int kSoftmaxWarps = 4, kWidenWarps = 16;      // K: two groups of four, V: two groups of four
constexpr int kQkWarp = 20, kPvWarp = 21, kLoadWarp = 22;
constexpr int kThreads = 32 * 24;                       // (registers are given out by groups of four warps: 23 has no role)
constexpr int kLaunchRegs = 80;                         // a thread's at launch: 65536 / 768, rounded down to a multiple of 8
constexpr int kColBlocks = kDqk / 64;                   // K chunks of a tile
constexpr int kVChunks = 8;                             // V chunks of a tile: (2 halves of the columns) x (4 quarters of the keys)
constexpr uint32_t kPBytes = 128 * 128;                 // P~: [128 keys][64 rows of f16], 128-byte swizzle
constexpr int kSmemPlanItems = 512;
constexpr float kPBias = 9.f, kPLimit = 15.f;           // P~ = 2^(a - n + 9), at most 2^15
constexpr float kFar = 1e30f;                           // n of a row that has seen no key is -kFar

template <int kN>
struct Shape {
  // Registers a thread, by warpgroup (softmax; four of widening; issue): together what the block is launched with
  static constexpr int kSoftmaxRegs = kN == 64 ? 224 : 168, kWidenRegs = kN == 64 ? 48 : 64, kIssueRegs = kN == 64 ? 64 : 56;
  static_assert(kSoftmaxRegs + 4 * kWidenRegs + kIssueRegs <= 6 * kLaunchRegs, "the block has no more to give out");
  static constexpr int kCols = kN < 32 ? kN : 32;       // rows that the softmax has in registers at a time
  static constexpr int kParts = kN / kCols;
  static constexpr int kSlots = kN == 64 ? 6 : kN == 32 ? 8 : 9;      // pages in shared memory
  // Operand chunks in tensor memory, of K and of V: numbers that divide a tile's, so that a tile's chunks always have the same places.
  static constexpr int kKBufs = 3, kVBufs = kN == 64 ? 2 : 4;
  static constexpr int kSBufs = kN == 64 ? 1 : 2;       // score tiles in tensor memory
  static constexpr uint32_t kQBlock = kN * 128;         // [rows][64 columns of f16], 128-byte swizzle
  static constexpr uint32_t kOffP = kColBlocks * kQBlock;
  static constexpr uint32_t kOffRaw = kOffP + kPBytes;
  static constexpr uint32_t kOffMult = kOffRaw + kSlots * kPageBytes4;      // float [2 units][rows]: logit per product, in octaves
  static constexpr uint32_t kOffNeg = kOffMult + 2 * kN * 4;                // float [4 warps][rows]: 9 - n
  static constexpr uint32_t kOffInv = kOffNeg + 4 * kN * 4;                 // float [4 warps][rows]
  static constexpr uint32_t kOffVis = kOffInv + 4 * kN * 4;                 // int [2 units][rows]: keys that the row sees
  static constexpr uint32_t kOffSums = kOffVis + 2 * kN * 4;                // float [2 units][4 warps][rows]
  static constexpr uint32_t kOffMax = kOffSums + 8 * kN * 4;                // float [2][4 warps][32]
  static constexpr uint32_t kOffMoves = kOffMax + 2 * 4 * 32 * 4;               // uint32 [2][4 warps]
  static constexpr uint32_t kOffInfo = kOffMoves + 32;                      // int [slots]: keys of the page that count
  static constexpr uint32_t kOffBars = kOffInfo + 48;
  static constexpr uint32_t kBarBytes = 384;
  static constexpr uint32_t kOffPlan = kOffBars + kBarBytes;
  static constexpr uint32_t kOffLens = kOffPlan + ((kSmemPlanItems + 1) * 4 + 15) / 16 * 16;
  static constexpr uint32_t kOffFirst = kOffLens + kSmemPlanItems * 4;
  static constexpr uint32_t kBytes = kOffFirst + sizeof(FirstUnit);
  // tensor-memory columns
  static constexpr uint32_t kOCol = 0, kSCol = 4 * kN, kKCol = 512 - 32 * (kKBufs + kVBufs), kVCol = 512 - 32 * kVBufs;
  enum { X_FULL = 0, X_EMPTY = X_FULL + kSlots, X_KFULL = X_EMPTY + kSlots, X_KEMPTY = X_KFULL + kKBufs, X_VFULL = X_KEMPTY + kKBufs, X_VEMPTY = X_VFULL + kVBufs, X_QREADY = X_VEMPTY + kVBufs,
         X_SFULL, X_SEMPTY = X_SFULL + kSBufs, X_PREADY = X_SEMPTY + kSBufs, X_PVDONE, X_MOVES, X_MAX, X_SUMS, X_NUM };
  static_assert(X_NUM * 8 + 8 <= kBarBytes, "barrier area too small");
  static_assert(kBytes <= 232448, "exceeds the shared memory a block can opt in to");
  static_assert(kOffP % 1024 == 0 && kOffRaw % 1024 == 0 && kPageBytes4 % 16 == 0 && kOffBars % 8 == 0 && kOffMoves % 16 == 0 && kOffMult % 16 == 0, "alignment");
  static_assert(kSCol + kSBufs * kN <= kKCol && kSlots <= 12, "tensor memory");
  static_assert(kColBlocks % kKBufs == 0 && kVChunks % kVBufs == 0 && (kVBufs == 2 || kVBufs == 4), "places of chunks");
};

__device__ __forceinline__ void report_timeout(int* status) { atomicExch(status, kStatusTimeout); }
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity) { return __all_sync(0xffffffffu, mbar_wait_inline(bar, parity)); }

using Tiles = TileIter<2>;

__device__ __forceinline__ float ld_shared_f32(uint32_t addr) { return __uint_as_float(ld_shared_b32(addr)); }
__device__ __forceinline__ float warp_max(float v) {
  float r;
  asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
  return r;
}
// 16 lanes x 8 columns: thread (g = lane / 4, q = lane % 4) gives columns 2q, 2q + 1 of lanes g (r0, r1) and g + 8 (r2, r3)
__device__ __forceinline__ void tmem_st_16x256b_x1(uint32_t taddr, const uint32_t (&r)[4]) {
  asm volatile("tcgen05.st.sync.aligned.16x256b.x1.b32 [%0], {%1, %2, %3, %4};" ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]) : "memory");
}
template <int kCount>
__device__ __forceinline__ void tmem_ld_cols(uint32_t taddr, uint32_t (&r)[kCount]) {
  if constexpr (kCount == 32) tmem_ld_32x32b_x32(taddr, r);
  else tmem_ld_32x32b_x16(taddr, r);
}
template <int kCount>
__device__ __forceinline__ void tmem_st_cols(uint32_t taddr, const uint32_t (&r)[kCount]) {
  if constexpr (kCount == 32) tmem_st_32x32b_x32(taddr, r);
  else tmem_st_32x32b_x16(taddr, r);
}
// E4M3 scales as f16: a NaN becomes 448, the largest.
__device__ __forceinline__ uint32_t number_f16x2(uint32_t s) {
  uint32_t r;
  asm("min.f16x2 %0, %1, %2;" : "=r"(r) : "r"(s), "r"(0x5f005f00u));
  return r;
}
// kind::f16 with f16 operands and FP32 accumulation (make_idesc_bf16's other type: 0)
__host__ __device__ constexpr uint32_t make_idesc_f16(int m, int n, bool a_mn_major, bool b_mn_major) {
  return make_idesc_bf16(m, n, a_mn_major, b_mn_major) & ~((1u << 7) | (1u << 10));
}
// f * 2^d on the exponent bits, d <= 0; zeros stay zero, what would leave the normal range becomes zero or denormal, and what is not a
// finite number stays what it is.
__device__ __forceinline__ float lower_octaves(float f, int d_bits) {
  return (__float_as_uint(f) & 0x7f800000u) == 0x7f800000u ? f : exponent_add_guarded(f, d_bits);
}
// v[r] of 32 lanes added up: lane i gets row i % kCount
template <int kCount>
__device__ __forceinline__ float sum_rows(float (&v)[kCount], int lane) {
  if constexpr (kCount == 16) {
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], 16);
  }
#pragma unroll
  for (int o = kCount / 2; o; o >>= 1) {
#pragma unroll
    for (int i = 0; i < o; ++i) {
      const float send = (lane & o) ? v[i] : v[i + o], keep = (lane & o) ? v[i + o] : v[i];
      v[i] = keep + __shfl_xor_sync(0xffffffffu, send, o);
    }
  }
  return v[0];
}

}  // namespace

template <int kN>
__global__ void __launch_bounds__(kThreads, 1) decode_fp4_kernel(const DecodeParams prm) {
  using C = Shape<kN>;
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  const uint32_t smem_base = smem_u32(smem_raw);
  const int tid = threadIdx.x, wid = tid >> 5, lane = tid & 31;
  const int part = blockIdx.x;
  if (tid == 0) AMLA_STAMP(prm, part, 20, 0);
  if (smem_base & 1023u) {   // the swizzled tiles assume a 1024-byte aligned window
    if (tid == 0) report_timeout(prm.status);
    return;
  }
  const uint32_t bars = smem_base + C::kOffBars;
  auto bar = [&](int i) { return bars + 8u * i; };
  const uint32_t tmem_slot = bars + C::kBarBytes - 8;

  // Set-up: as in the kernel for few rows.
  const bool plan_here = prm.fused_plan && prm.n_items <= kSmemPlanItems;
  int* plan_smem = reinterpret_cast<int*>(smem_raw + C::kOffPlan);
  int* lens_smem = reinterpret_cast<int*>(smem_raw + C::kOffLens);
  FirstUnit* first_smem = reinterpret_cast<FirstUnit*>(smem_raw + C::kOffFirst);
  const bool by_warp = prm.n_items <= kWarpPlanItems;
  if (plan_here && (!by_warp || wid == kLoadWarp)) plan_lengths(prm, plan_smem, lens_smem, by_warp ? lane : tid, by_warp ? 32 : kThreads);
  if (tid == 0) {
    for (int i = 0; i < C::kSlots; ++i) { mbar_init(bar(C::X_FULL + i), 1); mbar_init(bar(C::X_EMPTY + i), kWidenWarps); }
    for (int i = 0; i < C::kKBufs; ++i) { mbar_init(bar(C::X_KFULL + i), 4); mbar_init(bar(C::X_KEMPTY + i), 1); }
    for (int i = 0; i < C::kVBufs; ++i) { mbar_init(bar(C::X_VFULL + i), 4); mbar_init(bar(C::X_VEMPTY + i), 1); }
    mbar_init(bar(C::X_QREADY), kSoftmaxWarps);
    for (int i = 0; i < C::kSBufs; ++i) { mbar_init(bar(C::X_SFULL + i), 1); mbar_init(bar(C::X_SEMPTY + i), kSoftmaxWarps); }
    mbar_init(bar(C::X_PREADY), kSoftmaxWarps);
    mbar_init(bar(C::X_PVDONE), 1);
    mbar_init(bar(C::X_MOVES), kSoftmaxWarps);
    mbar_init(bar(C::X_MAX), kSoftmaxWarps);
    mbar_init(bar(C::X_SUMS), kSoftmaxWarps);
    fence_mbar_init();
  }
  if (wid == kQkWarp) { tmem_alloc(tmem_slot, 512); tmem_relinquish(); }
  if (plan_here) {
    if (by_warp) __syncwarp(); else __syncthreads();
    if (wid == kLoadWarp) plan_units(prm, plan_smem, lens_smem, first_smem, part, lane);
  }
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  // All 512 columns: they begin at 0.  (An address that is a constant keeps the issue of an MMA short.)
  constexpr uint32_t tbase = 0;
  if (ld_shared_b32(tmem_slot) != 0) {
    if (tid == 0) report_timeout(prm.status);
    return;
  }

  const int* prefix = plan_here ? plan_smem : prm.prefix;
  const int* seqlens = plan_here ? lens_smem : prm.seqlens;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;");
  if (plan_here) {
    if (plan_is_stale(prm, plan_smem, lens_smem, first_smem, tid, kThreads)) {
      plan_lengths(prm, plan_smem, lens_smem, tid, kThreads);
      __syncthreads();
      if (wid == kLoadWarp) plan_units(prm, plan_smem, lens_smem, first_smem, part, lane);
      __syncthreads();
    }
    if (blockIdx.x == 0 && tid == 0) *prm.status = kStatusOk;
  } else if (prm.fused_plan) {  // (kSmemPlanItems, kFusedPlanMaxItems] items: every CTA writes the same prefix to the workspace
    if (wid == 0) {
      plan_in_workspace(prm, lane);
      if (tid == 0 && blockIdx.x == 0) *prm.status = kStatusOk;
      __threadfence_block();
    }
    __syncthreads();
  }
  bool ok = true;
  Tiles tile(UnitIter(prm, prefix, seqlens, part), plan_here ? first_smem : nullptr);

  if (wid < kSoftmaxWarps) {
    // ======================================================== Q, softmax, rescale, epilogue
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(C::kSoftmaxRegs));
    const uint32_t lane_base = static_cast<uint32_t>(wid * 32) << 16;
    const uint32_t o_addr = tbase + lane_base + C::kOCol;
    const uint32_t neg = smem_base + C::kOffNeg + wid * kN * 4, invs = smem_base + C::kOffInv + wid * kN * 4;
    // Key 32 wid + lane of the tile is row k of P~: the order in which the widening warps put V's keys (see there).
    const int q4 = (lane >> 2) & 3, k = 32 * wid + (lane & 16) + 4 * q4 + (((lane & 3) - q4) & 3);
    const uint32_t p_dst = smem_base + C::kOffP + k * 128, p_sw = k & 7;
    uint32_t gs = 0, un = 0, moves = 0, maxes = 0;

    // The next unit's Q rows into f16, and what its rows need: the factor from a product to a logit and the keys that they see.
    auto load_q = [&](const Unit& u, uint32_t unit) {
      const uint32_t mult = smem_base + C::kOffMult + (unit & 1) * kN * 4, vis = smem_base + C::kOffVis + (unit & 1) * kN * 4;
      constexpr int kEach = kN / kSoftmaxWarps, kAtOnce = 4;
#pragma unroll 1
      for (int r0 = wid * kEach; r0 < (wid + 1) * kEach; r0 += kAtOnce) {
        uint4 x[kAtOnce][3];
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) {
          const int row = u.r0 + r0 + i;
          const uint4* src = reinterpret_cast<const uint4*>(prm.q + (static_cast<size_t>(u.b) * prm.R + row) * kDqk) + lane;
          const bool live = row < prm.R;
          x[i][0] = live ? __ldg(src) : make_uint4(0, 0, 0, 0);
          x[i][1] = live ? __ldg(src + 32) : make_uint4(0, 0, 0, 0);
          x[i][2] = live && lane < 8 ? __ldg(src + 64) : make_uint4(0, 0, 0, 0);
        }
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) {
          const int r = r0 + i;
          uint32_t top = 0;
#pragma unroll
          for (int j = 0; j < 3; ++j) {
            const uint32_t w[4] = {x[i][j].x, x[i][j].y, x[i][j].z, x[i][j].w};
#pragma unroll
            for (int c = 0; c < 4; ++c) top = max(top, max((w[c] << 16) & 0x7fffffffu, w[c] & 0x7fff0000u));
          }
          const uint32_t e = __reduce_max_sync(0xffffffffu, top) >> 23;
          // 2^(14 - (e - 127)) and its inverse; the largest powers that FP32 has for rows below 2^-113, 1 for rows that are not finite
          const float up = e == 255 ? 1.f : __uint_as_float(e <= 14 ? 254u << 23 : (268u - e) << 23);
          const float down = e == 255 ? 1.f : __uint_as_float(e <= 14 ? 0x00400000u : (e - 14u) << 23);
#pragma unroll
          for (int j = 0; j < 3; ++j) {
            const uint32_t w[4] = {x[i][j].x, x[i][j].y, x[i][j].z, x[i][j].w};
            uint32_t h[4];
#pragma unroll
            for (int c = 0; c < 4; ++c) h[c] = pack_f16x2(__uint_as_float(w[c] << 16) * up, __uint_as_float(w[c] & 0xffff0000u) * up);
            const int chunk = lane + 32 * j;
            if (j < 2 || lane < 8)
              st_shared_v4(smem_base + (chunk >> 3) * C::kQBlock + r * 128 + (((chunk & 7) ^ (r & 7)) << 4), h[0], h[1], h[2], h[3]);
          }
          if (lane == 0) {
            st_shared_b32(mult + 4 * r, __float_as_uint(prm.scale_log2 * down));
            st_shared_b32(vis + 4 * r, static_cast<uint32_t>(min(u.n_b, u.n_b - prm.Sq + (u.r0 + r) / prm.H + 1)));
          }
        }
      }
#pragma unroll
      for (int r = lane; r < kN; r += 32) st_shared_b32(neg + 4 * r, __float_as_uint(kFar));
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(C::X_QREADY));
    };

    if (tid == 0) AMLA_STAMP(prm, part, 20, 1);
    if (tile.valid) load_q(tile.u, 0);
    if (tid == 0) AMLA_STAMP(prm, part, 20, 2);
    if (tid == 0) merge_begin(prm, part);
    write_empty_items(prm, prefix, part, prm.P, 0, kN, tid, 32 * kSoftmaxWarps);
    while (ok && tile.valid) {
      const Unit u = tile.u;
      const int all_see = max(u.n_b - prm.Sq + 1, 0);                  // keys in front of this one are seen by every row
      const uint32_t mult = smem_base + C::kOffMult + (un & 1) * kN * 4, vis = smem_base + C::kOffVis + (un & 1) * kN * 4;
      float l[kN];
#pragma unroll
      for (int i = 0; i < kN; ++i) l[i] = 0.f;
      ok = warp_wait(bar(C::X_QREADY), un & 1);                        // the other warps' rows
      if (!ok) break;
      bool more = true;
      while (more) {
        const uint32_t sb = gs % C::kSBufs, s_addr = tbase + lane_base + C::kSCol + sb * kN;
        ok = warp_wait(bar(C::X_SFULL) + 8 * sb, (gs / C::kSBufs) & 1);
        if (!ok) break;
        tc_fence_after_sync();
        if (tid == 0) AMLA_STAMP(prm, part, 7, gs);
        const bool plain = tile.np == 2 && (tile.t + 2) * kPage <= all_see;
        const int in_tile = 32 * wid + lane;
        const int key = in_tile < tile.np * kPage ? tile.t * kPage + in_tile : 0x7fffffff;
        float y[kN];                                                   // a - n + 9, in octaves
        // The second pass is for a tile that moved the reference (a unit's first always does).
#pragma unroll 1
        for (bool moved = false;;) {
          bool move = tile.first;
          if (moved || !move) {
            float top = -INFINITY;
#pragma unroll
            for (int h = 0; h < C::kParts; ++h) {
              uint32_t s[C::kCols];
              tmem_ld_cols<C::kCols>(s_addr + C::kCols * h, s);
              tmem_wait_ld();
#pragma unroll
              for (int r = 0; r < C::kCols; r += 4) {
                uint32_t m[4], n[4];
                ld_shared_v4(mult + 4 * (C::kCols * h + r), m[0], m[1], m[2], m[3]);
                ld_shared_v4(neg + 4 * (C::kCols * h + r), n[0], n[1], n[2], n[3]);
#pragma unroll
                for (int i = 0; i < 4; ++i) y[C::kCols * h + r + i] = fmaf(__uint_as_float(s[r + i]), __uint_as_float(m[i]), __uint_as_float(n[i]));
              }
            }
            if (!plain) {
#pragma unroll
              for (int r = 0; r < kN; ++r) y[r] = key < static_cast<int>(ld_shared_b32(vis + 4 * r)) ? y[r] : -INFINITY;
            }
            if (moved) break;
#pragma unroll
            for (int r = 0; r < kN; r += 2) top = fmax3(top, y[r], y[r + 1]);
            // Does any key of the tile exceed what P~ may reach?  The four warps decide together.
            const bool mine = __any_sync(0xffffffffu, top > kPLimit);
            const uint32_t at = smem_base + C::kOffMoves + (moves & 1) * 16;
            if (lane == 0) { st_shared_b32(at + 4 * wid, mine); mbar_arrive(bar(C::X_MOVES)); }
            ok = warp_wait(bar(C::X_MOVES), moves & 1);
            if (!ok) break;
            ++moves;
            uint32_t f[4];
            ld_shared_v4(at, f[0], f[1], f[2], f[3]);
            move = (f[0] | f[1] | f[2] | f[3]) != 0;
          }
          if (!move) break;
          moved = true;
#pragma unroll
          for (int h = 0; h < C::kParts; ++h) {
            // The largest logit of every row: over the warp, then over the four warps; lane r keeps row r.
            float mine = -INFINITY;
            uint32_t s[C::kCols];
            tmem_ld_cols<C::kCols>(s_addr + C::kCols * h, s);
            tmem_wait_ld();
#pragma unroll
            for (int r = 0; r < C::kCols; ++r) {
              float a = __uint_as_float(s[r]) * ld_shared_f32(mult + 4 * (C::kCols * h + r));
              if (!plain) a = key < static_cast<int>(ld_shared_b32(vis + 4 * (C::kCols * h + r))) ? a : -INFINITY;
              a = warp_max(a);
              if (lane == r) mine = a;
            }
            const uint32_t at_max = smem_base + C::kOffMax + (maxes & 1) * 512;
            st_shared_b32(at_max + 4 * (32 * wid + lane), __float_as_uint(mine));
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(C::X_MAX));
            ok = warp_wait(bar(C::X_MAX), maxes & 1);
            if (!ok) break;
            ++maxes;
#pragma unroll
            for (int w = 0; w < kSoftmaxWarps; ++w) mine = fmaxf(mine, ld_shared_f32(at_max + 4 * (32 * w + lane)));
            // Every row of the part whose maximum rose moves (moving early is always allowed).
            int d_bits = 0;
            if (lane < C::kCols) {
              const uint32_t at = neg + 4 * (C::kCols * h + lane);
              const float old = ld_shared_f32(at);                     // 9 - n
              if (mine + old > kPBias) {
                const float now = kPBias - ceilf(mine);
                st_shared_b32(at, __float_as_uint(now));
                d_bits = static_cast<int>(fmaxf(now - old, -255.f)) * (1 << 23);
              }
            }
            __syncwarp();
            if (!tile.first && __any_sync(0xffffffffu, d_bits != 0)) {
              // O <- AS_FP32(AS_INT32(O) + d * 2^23): O^T has a row per column, a thread the same d for all of a row
              ok = warp_wait(bar(C::X_PVDONE), (gs - 1) & 1);
              if (!ok) break;
              tc_fence_after_sync();
#pragma unroll 1
              for (int m = 0; m < 4; ++m) {
                uint32_t o[C::kCols];
                tmem_ld_cols<C::kCols>(o_addr + kN * m + C::kCols * h, o);
                tmem_wait_ld();
#pragma unroll
                for (int r = 0; r < C::kCols; ++r) o[r] = __float_as_uint(lower_octaves(__uint_as_float(o[r]), __shfl_sync(0xffffffffu, d_bits, r)));
                tmem_st_cols<C::kCols>(o_addr + kN * m + C::kCols * h, o);
              }
              tmem_wait_st();
#pragma unroll
              for (int r = 0; r < C::kCols; ++r) l[C::kCols * h + r] = lower_octaves(l[C::kCols * h + r], __shfl_sync(0xffffffffu, d_bits, r));
            }
          }
          if (!ok) break;
        }
        if (!ok) break;
        tc_fence_before_sync();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(C::X_SEMPTY) + 8 * sb);         // the scores have been read
        uint32_t pk[kN / 2];
#pragma unroll
        for (int r = 0; r < kN; r += 2) {
          const float p0 = ex2_approx(y[r]), p1 = ex2_approx(y[r + 1]);
          l[r] += p0;
          l[r + 1] += p1;
          pk[r / 2] = pack_f16x2(p0, p1);
        }
        if (tid == 0) AMLA_STAMP(prm, part, 9, gs);
        if (gs > 0) {
          ok = warp_wait(bar(C::X_PVDONE), (gs - 1) & 1);              // the P~V of the tile before has read the P buffer
          if (!ok) break;
        }
#pragma unroll
        for (int c = 0; c < kN / 8; ++c) st_shared_v4(p_dst + ((c ^ p_sw) << 4), pk[4 * c], pk[4 * c + 1], pk[4 * c + 2], pk[4 * c + 3]);
        tc_fence_before_sync();                                        // O (perhaps) rewritten
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(C::X_PREADY));
        if (tid == 0) AMLA_STAMP(prm, part, 8, gs);
        ++gs;
        more = !tile.last();
        if (more) tile.next();
      }
      if (!ok) break;
      float n_of[C::kParts];                                           // 9 - n of rows kCols h + lane
#pragma unroll
      for (int h = 0; h < C::kParts; ++h) n_of[h] = ld_shared_f32(neg + 4 * (C::kCols * h + lane % C::kCols));
      __syncwarp();
      // the next unit's Q: all Q K^T of this one have been waited for
      tile.next();
      if (tid == 0) AMLA_STAMP(prm, part, 10, un);
      if (tile.valid) load_q(tile.u, un + 1);
      if (tid == 0) AMLA_STAMP(prm, part, 11, un);
      // ---- epilogue: out = O / l, lse = n + log2 l
      int2 info;
      const int pslot = tile.units.slot_of(u, &info);                  // partial slot, or -1
      if (tid == 0) merge_note(prm, part, u.it, info);
      const uint32_t sums = smem_base + C::kOffSums + (un & 1) * 4 * kN * 4;
#pragma unroll
      for (int h = 0; h < C::kParts; ++h) {
        float v[C::kCols];
#pragma unroll
        for (int r = 0; r < C::kCols; ++r) v[r] = l[C::kCols * h + r];
        const float x = sum_rows<C::kCols>(v, lane);
        if (lane < C::kCols) st_shared_b32(sums + 4 * (kN * wid + C::kCols * h + lane), __float_as_uint(x));
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(C::X_SUMS));
      ok = warp_wait(bar(C::X_SUMS), un & 1);
      if (!ok) break;
      const size_t row0 = static_cast<size_t>(u.b) * prm.R + u.r0, prow0 = static_cast<size_t>(pslot < 0 ? 0 : pslot) * kN;
      const int rows = prm.R - u.r0;                                   // live ones among the kN
      // A partial is an average of values of at most 2688, in half precision as it is; the power of two of out_scale is its chunks' scale
      // byte, the rest of out_scale (in [1, 2)) is multiplied in.
      const uint32_t scale_bits = __float_as_uint(prm.out_scale);
      const float factor = pslot < 0 ? prm.out_scale : __uint_as_float((scale_bits & 0x7fffffu) | (127u << 23));
      const uint32_t byte4 = (scale_bits >> 23) * 0x01010101u;
#pragma unroll
      for (int h = 0; h < C::kParts; ++h) {
        const int r = C::kCols * h + lane;
        if (lane < C::kCols) {
          float total = 0.f;
#pragma unroll
          for (int w = 0; w < kSoftmaxWarps; ++w) total += ld_shared_f32(sums + 4 * (kN * w + r));
          const float lse = total == 0.f ? -INFINITY : (log2f(total) - n_of[h]) * kLn2;
          st_shared_b32(invs + 4 * r, __float_as_uint(total == 0.f ? 0.f : factor / total));
          if (wid == 0 && r < rows) {
            if (pslot < 0) prm.lse[row0 + r] = lse;
            else prm.part_lse[prow0 + r] = lse;
          }
          if (wid == 1 && pslot >= 0) reinterpret_cast<uint4*>(partial_scales(prm))[prow0 + r] = make_uint4(byte4, byte4, byte4, byte4);
        }
      }
      __syncwarp();
      ok = warp_wait(bar(C::X_PVDONE), (gs - 1) & 1);
      if (!ok) break;
      tc_fence_after_sync();
      // Lane L of block 2p (2p + 1) of O^T is column 64 (4p + wid) + 8 (L % 8) + L / 8 (+ 4): the four lanes with one L % 8 hold eight
      // neighbouring columns of every row.  They exchange four rows, a lane is left with eight columns of one: 16 bytes.
      uint16_t* dst = pslot < 0 ? reinterpret_cast<uint16_t*>(prm.out) + row0 * kDv : partial_halves(prm) + prow0 * kDv;
      const int last = pslot < 0 ? rows : kN;
      const bool b0 = lane & 8, b1 = lane & 16;
      dst += 64 * wid + 8 * (lane & 7) + static_cast<size_t>(lane >> 3) * kDv;
#pragma unroll 1
      for (int i = 0; i < kN / 16 * 2; ++i) {
        const int p = i & 1, rb = (i >> 1) * 16;
        uint32_t lo[16], hi[16];
        tmem_ld_32x32b_x16(o_addr + kN * (2 * p) + rb, lo);
        tmem_ld_32x32b_x16(o_addr + kN * (2 * p + 1) + rb, hi);
        tmem_wait_ld();
#pragma unroll
        for (int j = 0; j < 16; j += 4) {
          uint32_t a[4], f[4];
          ld_shared_v4(invs + 4 * (rb + j), f[0], f[1], f[2], f[3]);
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            const float x = __uint_as_float(lo[j + c]) * __uint_as_float(f[c]), z = __uint_as_float(hi[j + c]) * __uint_as_float(f[c]);
            a[c] = pslot < 0 ? pack_bf16x2(x, z) : pack_f16x2(x, z);
          }
          const uint32_t g0 = __shfl_xor_sync(0xffffffffu, b1 ? a[0] : a[2], 16), g1 = __shfl_xor_sync(0xffffffffu, b1 ? a[1] : a[3], 16);
          const uint32_t k0 = b1 ? a[2] : a[0], k1 = b1 ? a[3] : a[1];               // rows 2 b1 + 0, 1: own, and (g) of the lane 16 away
          const uint32_t t0 = __shfl_xor_sync(0xffffffffu, b0 ? k0 : k1, 8), t1 = __shfl_xor_sync(0xffffffffu, b0 ? g0 : g1, 8);
          const uint32_t kk = b0 ? k1 : k0, kg = b0 ? g1 : g0;                        // row 2 b1 + b0 from lanes L, L ^ 16, L ^ 8 (t0), L ^ 24 (t1)
          const uint32_t m0 = b0 ? t0 : kk, m1 = b0 ? kk : t0, n0 = b0 ? t1 : kg, n1 = b0 ? kg : t1;
          const uint32_t c0 = b1 ? n0 : m0, c1 = b1 ? n1 : m1, c2 = b1 ? m0 : n0, c3 = b1 ? m1 : n1;   // columns (i, i + 4)
          const int row = rb + j + (lane >> 3);
          if (row < last)
            stg_128(dst + static_cast<size_t>(rb + j) * kDv + 256 * p, __byte_perm(c0, c1, 0x5410), __byte_perm(c2, c3, 0x5410), __byte_perm(c0, c1, 0x7632), __byte_perm(c2, c3, 0x7632));
        }
      }
      if (tid == 0) AMLA_STAMP(prm, part, 12, un);
      tc_fence_before_sync();      // O has been read: this warp's next PREADY arrival lets the next unit overwrite it
      ++un;
    }
    if (!ok && lane == 0) report_timeout(prm.status);
  } else if (wid < kSoftmaxWarps + kWidenWarps) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(C::kWidenRegs));
    // ======================================================== widening: raw pages -> operand chunks in tensor memory
    const int quad = wid & 3;
    const uint32_t raw = smem_base + C::kOffRaw, infos = smem_base + C::kOffInfo, lanes = tbase + (static_cast<uint32_t>(quad * 32) << 16);
    const uint32_t group = (wid >> 2) & 1 ^ 1;               // of the two that take turns by chunk: warps 4-7 and 12-15, 8-11 and 16-19
    uint32_t slot = 0, par = 0, tiles = 0;
    [[maybe_unused]] int kc = 0;                            // (trace builds)
    auto next_slot = [&](uint32_t x) { return x + 1 == C::kSlots ? 0u : x + 1; };
    auto pages_here = [&](uint32_t slot1) {
      ok = mbar_wait_inline(bar(C::X_FULL) + 8 * slot, par);
      if (slot1 != slot) ok &= mbar_wait_inline(bar(C::X_FULL) + 8 * slot1, slot1 == 0 ? par ^ 1 : par);
    };
    auto pages_done = [&](uint32_t slot1) {                  // (what was read of them is in registers)
      __syncwarp();
      mbar_arrive_if(lane == 0, bar(C::X_EMPTY) + 8 * slot);
      mbar_arrive_if(lane == 0 && slot1 != slot, bar(C::X_EMPTY) + 8 * slot1);
      if (slot1 < slot) par ^= 1;
      slot = next_slot(slot1);
      if (slot == 0) par ^= 1;
      ++tiles;
      tile.next();
    };
    auto place = [&](uint32_t empty, uint32_t use) {
      ok &= mbar_wait_inline(empty, (use & 1) ^ 1);
      __syncwarp();
      tc_fence_after_sync();
    };
    auto hand_over = [&](uint32_t full) {
      tmem_wait_st();
      tc_fence_before_sync();
      __syncwarp();
      mbar_arrive_if(lane == 0, full);
    };
    if (wid < kSoftmaxWarps + kWidenWarps / 2) {
      // ---- K: lane = key of the tile, 64 columns a chunk, 32 at a time
      while (tile.valid) {
        const uint32_t slot1 = tile.np == 2 ? next_slot(slot) : slot;
        pages_here(slot1);
        const uint32_t mine = quad < 2 ? slot : slot1, key = 32 * (quad & 1) + lane;
        const uint32_t codes = raw + mine * kPageBytes4 + key * kCodeRow, scales = raw + mine * kPageBytes4 + kCodeBytes + key * kScaleRow;
        const uint32_t there = ld_shared_b32(infos + 4 * mine) != 0 ? 0xffffffffu : 0u;      // a page outside the cache: zeros
#pragma unroll 1
        for (uint32_t c = (group + tiles) & 1; c < kColBlocks; c += 2) {      // (nine a tile: the groups change places)
          if (quad == 0 && lane == 0) AMLA_STAMP(prm, part, 0, tiles * 9 + c);
          uint32_t w[8];
          ld_shared_v4(codes + 32 * c, w[0], w[1], w[2], w[3]);
          ld_shared_v4(codes + 32 * c + 16, w[4], w[5], w[6], w[7]);
          const uint32_t sw = ld_shared_b32(scales + 4 * c) & there;
          const uint32_t buf = c % C::kKBufs;
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            uint32_t r[16];
            const uint32_t s2 = e4m3x2_to_f16x2(h == 0 ? sw & 0xffffu : sw >> 16);
            const uint32_t sc[2] = {__byte_perm(s2, 0, 0x1010), __byte_perm(s2, 0, 0x3232)};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              uint32_t x[4];
              e2m1x8_to_f16x2(w[4 * h + j], x);
#pragma unroll
              for (int i = 0; i < 4; ++i) r[4 * j + i] = mul_f16x2(x[i], sc[j / 2]);
            }
            if (h == 0) place(bar(C::X_KEMPTY) + 8 * buf, tiles + c / C::kKBufs);
            tmem_st_32x32b_x16(lanes + C::kKCol + 32 * buf + 16 * h, r);
          }
          hand_over(bar(C::X_KFULL) + 8 * buf);
        }
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        pages_done(slot1);
      }
    } else {
      // ---- V: lanes = its columns, 32 keys a chunk, 16 at a time.  A thread (g = lane / 4, q = lane % 4) takes the 32-bit words g, eight
      // neighbouring columns, of warp `quad`'s 64 columns, for four keys: words of two keys are interleaved by nibbles and converted, which
      // gives pairs of keys.  Column i of a word goes to block 2p + i / 4, lane 32 quad + g + 8 (i % 4).  Key k = 4 q + e of the product's 16 is
      // key 4 q + (q + e) % 4, so that the four q read four different residues (a row is 72 words: else all from the same banks).
      // A scale that is a NaN becomes a number here: through K the rows that see the key have a NaN for its P~, and those that do
      // not have a zero, which a NaN in V would turn into one.
      const int g = lane >> 2, q = lane & 3;
      const uint32_t pick = (g >> 1) | ((4 + (g >> 1)) << 4);   // this thread's group, of the four that a scale word holds, of either key
      while (tile.valid) {
        const uint32_t slot1 = tile.np == 2 ? next_slot(slot) : slot;
        pages_here(slot1);
#pragma unroll 1
        for (uint32_t c = group; c < kVChunks; c += 2) {
          if (quad == 0 && lane == 0) AMLA_STAMP(prm, part, 13, tiles * 8 + c);
          const uint32_t mine = (c & 2) ? slot1 : slot, buf = c & (C::kVBufs - 1);
          const uint32_t page = raw + mine * kPageBytes4, codes = page + (c & 1) * (32 * kCodeRow) + (c >> 2) * 128 + 32 * quad + 4 * g;
          const uint32_t scales = page + kCodeBytes + (c & 1) * (32 * kScaleRow) + (c >> 2) * 16 + 4 * quad;
          const int count = ((c & 2) && tile.np == 1 ? 0 : static_cast<int>(ld_shared_b32(infos + 4 * mine))) - 32 * static_cast<int>(c & 1);   // keys of the chunk that count
#pragma unroll
          for (int b = 0; b < 2; ++b) {
            uint32_t w[4], sw[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const uint32_t key = 4 * q + ((q + e) & 3);
              w[e] = ld_shared_b32(codes + key * kCodeRow + 16 * b * kCodeRow);
              sw[e] = ld_shared_b32(scales + key * kScaleRow + 16 * b * kScaleRow);
            }
            if (count < 32) {                                 // what is beyond the sequence's end may be anything: scales of zero
#pragma unroll
              for (int e = 0; e < 4; ++e) sw[e] = 16 * b + 4 * q + ((q + e) & 3) < count ? sw[e] : 0u;
            }
            uint32_t r[2][2][4];
#pragma unroll
            for (int j = 0; j < 2; ++j) {                     // keys e = 2j, 2j + 1
              const uint32_t w0 = w[2 * j], w1 = w[2 * j + 1];
              const uint32_t even = (w0 & 0x0f0f0f0fu) | ((w1 << 4) & 0xf0f0f0f0u), odd = ((w0 >> 4) & 0x0f0f0f0fu) | (w1 & 0xf0f0f0f0u);
              const uint32_t sc = number_f16x2(e4m3x2_to_f16x2(__byte_perm(sw[2 * j], sw[2 * j + 1], pick)));
              uint32_t x[4], z[4];
              e2m1x8_to_f16x2(even, x);
              e2m1x8_to_f16x2(odd, z);
#pragma unroll
              for (int i = 0; i < 4; ++i) {                   // columns 2i (lanes .. + g) and 2i + 1 (.. + 8 + g)
                r[i >> 1][i & 1][j] = mul_f16x2(x[i], sc);
                r[i >> 1][i & 1][2 + j] = mul_f16x2(z[i], sc);
              }
            }
            if (b == 0) place(bar(C::X_VEMPTY) + 8 * buf, C::kVBufs == 4 ? c >> 2 : c >> 1);
#pragma unroll
            for (int m = 0; m < 2; ++m)
#pragma unroll
              for (int hh = 0; hh < 2; ++hh) tmem_st_16x256b_x1(lanes + (static_cast<uint32_t>(16 * hh) << 16) + C::kVCol + 32 * buf + 16 * m + 8 * b, r[m][hh]);
          }
          hand_over(bar(C::X_VFULL) + 8 * buf);
        }
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        pages_done(slot1);
      }
    }
    if (!ok && lane == 0) report_timeout(prm.status);
  } else {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(C::kIssueRegs));
    constexpr uint32_t dhi = smem_desc_hi_sw128(1024);
    if (wid == kQkWarp) {
      // ======================================================== S^T = K Q^T
      // (Constants wherever they can be: an accumulate flag out of a register alone costs as much issue as an MMA.)
      if (elect_one()) {
        constexpr uint32_t idesc = make_idesc_f16(128, kN, false, false);
        uint32_t gs = 0, un = 0, par = 0;
        while (tile.valid) {
          if (tile.first) ok = mbar_wait_inline(bar(C::X_QREADY), un++ & 1);
          const uint32_t sb = gs % C::kSBufs, d = C::kSCol + sb * kN;
          ok &= mbar_wait_inline(bar(C::X_SEMPTY) + 8 * sb, ((gs / C::kSBufs) & 1) ^ 1);
          tc_fence_after_sync();
          constexpr uint32_t kQStep = C::kQBlock >> 4;
          const uint32_t ql = smem_desc_lo(smem_base, 16);
#pragma unroll
          for (int c = 0; c < kColBlocks; ++c) {
            constexpr int kB = C::kKBufs;
            ok &= mbar_wait_inline(bar(C::X_KFULL + c % kB), par ^ ((c / kB) & 1));
            tc_fence_after_sync();
            AMLA_STAMP(prm, part, 5, gs * 9 + c);
#pragma unroll
            for (int kk = 0; kk < 4; ++kk)
              mma_ts(d, C::kKCol + 32 * (c % kB) + 8 * kk, smem_desc_join(ql + c * kQStep + 2 * kk, dhi), idesc, c == 0 && kk == 0 ? 0 : 1);
            mma_commit(bar(C::X_KEMPTY + c % kB));
          }
          mma_commit(bar(C::X_SFULL) + 8 * sb);
          if (!ok) break;
          par ^= 1;                                          // (nine chunks in three places)
          ++gs;
          tile.next();
        }
        if (!ok) report_timeout(prm.status);
      }
      __syncwarp();
    } else if (wid == kPvWarp) {
      // ======================================================== O^T (+)= V^T P~^T
      if (elect_one()) {
        constexpr uint32_t idesc = make_idesc_f16(128, kN, false, true);
        uint32_t gp = 0;
        while (tile.valid) {
          ok = mbar_wait_inline(bar(C::X_PREADY), gp & 1);
          tc_fence_after_sync();                              // (O may have been rescaled)
          const uint32_t pl = smem_desc_lo(smem_base + C::kOffP, 16);
          const bool fresh = tile.first;
#pragma unroll
          for (int c = 0; c < kVChunks; ++c) {
            constexpr int kB = C::kVBufs;
            const int p = c >> 2, kq = c & 3;
            ok &= mbar_wait_inline(bar(C::X_VFULL + c % kB), (c / kB) & 1);
            tc_fence_after_sync();
            AMLA_STAMP(prm, part, 17, gp * 8 + c);
            const uint32_t a = C::kVCol + 32 * (c % kB), pc = pl + kq * (32 * 128 >> 4);
#pragma unroll
            for (int m = 0; m < 2; ++m) {
              const uint32_t d = C::kOCol + kN * (2 * p + m);
              if (kq == 0 && fresh) mma_ts(d, a + 16 * m, smem_desc_join(pc, dhi), idesc, 0);
              else mma_ts(d, a + 16 * m, smem_desc_join(pc, dhi), idesc, 1);
              mma_ts(d, a + 16 * m + 8, smem_desc_join(pc + (16 * 128 >> 4), dhi), idesc, 1);
            }
            mma_commit(bar(C::X_VEMPTY + c % kB));
          }
          mma_commit(bar(C::X_PVDONE));
          if (!ok) break;
          ++gp;
          tile.next();
        }
        if (!ok) report_timeout(prm.status);
      }
      __syncwarp();
    } else if (wid == kLoadWarp) {
    // ======================================================== pages in order
    if (elect_one()) {
      uint32_t slot = 0, par = 1, n_issued = 0;
      int i = 0;                                            // page of the tile
      auto entry = [&]() { return __ldg(prm.block_table + static_cast<size_t>(tile.u.b) * prm.max_blocks_per_seq + tile.t + i); };
      int page = tile.valid ? entry() : 0;
      while (tile.valid) {
        const int here = page, keys = min(kPage, tile.u.n_b - (tile.t + i) * kPage);
        if (++i == tile.np) { i = 0; tile.next(); }
        if (tile.valid) page = entry();                     // on its way while this page waits for its slot
        ok = mbar_wait_inline(bar(C::X_EMPTY) + 8 * slot, par);
        if (!ok) break;
        const bool there = here >= 0 && here < prm.num_blocks;
        const uint32_t full = bar(C::X_FULL) + 8 * slot;
        st_shared_b32(smem_base + C::kOffInfo + 4 * slot, there ? static_cast<uint32_t>(keys) : 0u);
        if (there) {
          mbar_arrive_expect_tx(full, kPageBytes4);
          bulk_load(smem_base + C::kOffRaw + slot * kPageBytes4, prm.kv4 + static_cast<size_t>(here) * kPageBytes4, kPageBytes4, full);
        } else {
          mbar_arrive(full);
        }
        ++n_issued;
        if (++slot == C::kSlots) { slot = 0; par ^= 1; }
      }
      if (!ok) {
        report_timeout(prm.status);
        // let the copies that may still be in flight land before the CTA exits
        for (uint32_t k = 0; k < C::kSlots && k < n_issued; ++k) {
          const uint32_t j = n_issued - 1 - k;
          mbar_wait_inline(bar(C::X_FULL) + 8 * (j % C::kSlots), (j / C::kSlots) & 1);
        }
      }
    }
    __syncwarp();
    }
  }

  tc_fence_before_sync();
  __syncthreads();
  if (tid == 0) AMLA_STAMP(prm, part, 21, 0);
  if (wid == kQkWarp) tmem_dealloc(tbase, 512);
}

// ---------------------------------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------------------------------
int fp4_item_rows(int rows) { return rows <= 16 ? 16 : rows <= 32 ? 32 : 64; }

cudaError_t launch_decode_fp4(const DecodeParams& prm, cudaStream_t stream) {
  static std::atomic<uint64_t> done16{0}, done32{0}, done64{0};
  if (prm.item_rows == 16) return launch_serialized(decode_fp4_kernel<16>, done16, prm.P, kThreads, Shape<16>::kBytes, stream, prm);
  if (prm.item_rows == 32) return launch_serialized(decode_fp4_kernel<32>, done32, prm.P, kThreads, Shape<32>::kBytes, stream, prm);
  return launch_serialized(decode_fp4_kernel<64>, done64, prm.P, kThreads, Shape<64>::kBytes, stream, prm);
}

}  // namespace amla
