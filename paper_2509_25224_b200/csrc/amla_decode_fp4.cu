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
// end), rescale, epilogue.  Warps 4-11: widening, two groups of four that take turns by chunk.  Warp 12 issues MMAs: Q K^T of the
// next tile in front of P~V of this one, but for a unit's last tile, whose P~V comes first (the next unit's Q is on its way
// meanwhile).  Warp 13 loads pages (bulk copies).
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

constexpr int kSoftmaxWarps = 4, kWidenWarps = 8;
constexpr int kMmaWarp = 12, kLoadWarp = 13;
constexpr int kThreads = 32 * 16;                        // (registers are given out by groups of four warps: 14, 15 have no role)
// Registers a thread, by warpgroup: what the block is launched with is 512 threads x 128
constexpr int kSoftmaxRegs = 232, kWidenRegs = 96, kIssueRegs = 80;
static_assert(kSoftmaxRegs + 2 * kWidenRegs + kIssueRegs <= 4 * 128, "the block has no more to give out");
constexpr int kColBlocks = kDqk / 64;                   // K chunks of a tile
constexpr int kVChunks = 8;                             // V chunks of a tile: (2 halves of the columns) x (4 quarters of the keys)
constexpr uint32_t kPBytes = 128 * 128;                 // P~: [128 keys][64 rows of f16], 128-byte swizzle
constexpr int kSmemPlanItems = 512;
constexpr float kPBias = 9.f, kPLimit = 15.f;           // P~ = 2^(a - n + 9), at most 2^15
constexpr float kFar = 1e30f;                           // n of a row that has seen no key is -kFar

template <int kN>
struct Shape {
  static constexpr int kCols = kN < 32 ? kN : 32;       // rows that the softmax has in registers at a time
  static constexpr int kParts = kN / kCols;
  static constexpr int kSlots = kN == 64 ? 6 : kN == 32 ? 8 : 9;      // pages in shared memory
  static constexpr int kBufs = kN == 64 ? 4 : 8;        // operand chunks in tensor memory
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
  static constexpr uint32_t kOCol = 0, kSCol = 4 * kN, kRing = 512 - 32 * kBufs;
  enum { X_FULL = 0, X_EMPTY = X_FULL + kSlots, X_AFULL = X_EMPTY + kSlots, X_AEMPTY = X_AFULL + kBufs, X_QREADY = X_AEMPTY + kBufs, X_SFULL, X_SEMPTY = X_SFULL + 2, X_PREADY = X_SEMPTY + 2,
         X_PVDONE, X_MOVES, X_MAX, X_SUMS, X_NUM };
  static_assert(X_NUM * 8 + 8 <= kBarBytes, "barrier area too small");
  static_assert(kBytes <= 232448, "exceeds the shared memory a block can opt in to");
  static_assert(kOffP % 1024 == 0 && kOffRaw % 1024 == 0 && kPageBytes4 % 16 == 0 && kOffBars % 8 == 0 && kOffMoves % 16 == 0 && kOffMult % 16 == 0, "alignment");
  static_assert(kSCol + 2 * kN <= kRing && kSlots <= 12, "tensor memory");
};

__device__ __forceinline__ void report_timeout(int* status) { atomicExch(status, kStatusTimeout); }
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity) { return __all_sync(0xffffffffu, mbar_wait(bar, parity)); }

using Tiles = TileIter<2>;

__device__ __forceinline__ float ld_shared_f32(uint32_t addr) { return __uint_as_float(ld_shared_b32(addr)); }
__device__ __forceinline__ uint32_t ld_shared_u8(uint32_t addr) {
  uint32_t v;
  asm volatile("ld.shared.u8 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
  return v;
}
__device__ __forceinline__ float warp_max(float v) {
  float r;
  asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
  return r;
}
// 16 lanes x 16 columns: thread (g = lane / 4, q = lane % 4) gives columns 2q, 2q + 1 of lanes g (r0, r1) and g + 8 (r2, r3), then
// the same of columns 8 ..
__device__ __forceinline__ void tmem_st_16x256b_x2(uint32_t taddr, const uint32_t (&r)[8]) {
  asm volatile("tcgen05.st.sync.aligned.16x256b.x2.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
               : "memory");
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
    for (int i = 0; i < C::kBufs; ++i) { mbar_init(bar(C::X_AFULL + i), 4); mbar_init(bar(C::X_AEMPTY + i), 1); }
    mbar_init(bar(C::X_QREADY), kSoftmaxWarps);
    for (int i = 0; i < 2; ++i) { mbar_init(bar(C::X_SFULL + i), 1); mbar_init(bar(C::X_SEMPTY + i), kSoftmaxWarps); }
    mbar_init(bar(C::X_PREADY), kSoftmaxWarps);
    mbar_init(bar(C::X_PVDONE), 1);
    mbar_init(bar(C::X_MOVES), kSoftmaxWarps);
    mbar_init(bar(C::X_MAX), kSoftmaxWarps);
    mbar_init(bar(C::X_SUMS), kSoftmaxWarps);
    fence_mbar_init();
  }
  if (wid == kMmaWarp) { tmem_alloc(tmem_slot, 512); tmem_relinquish(); }
  if (plan_here) {
    if (by_warp) __syncwarp(); else __syncthreads();
    if (wid == kLoadWarp) plan_units(prm, plan_smem, lens_smem, first_smem, part, lane);
  }
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tbase = ld_shared_b32(tmem_slot);

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
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kSoftmaxRegs));
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

    if (tile.valid) load_q(tile.u, 0);
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
        const uint32_t sb = gs & 1, s_addr = tbase + lane_base + C::kSCol + sb * kN;
        ok = warp_wait(bar(C::X_SFULL + sb), (gs >> 1) & 1);
        if (!ok) break;
        tc_fence_after_sync();
        const bool plain = tile.np == 2 && (tile.t + 2) * kPage <= all_see;
        const int in_tile = 32 * wid + lane;
        const int key = in_tile < tile.np * kPage ? tile.t * kPage + in_tile : 0x7fffffff;
        uint32_t pk[kN / 2];
#pragma unroll
        for (int h = 0; h < C::kParts; ++h) {
          float y[C::kCols];
          auto scores = [&](uint32_t (&s)[C::kCols]) {
            tmem_ld_cols<C::kCols>(s_addr + 32 * h, s);
            tmem_wait_ld();
          };
          auto logits = [&]() {                                        // a - n + 9, in octaves; the largest of the thread's
            uint32_t s[C::kCols];
            scores(s);
            float top = -INFINITY;
#pragma unroll
            for (int r = 0; r < C::kCols; r += 4) {
              uint32_t m[4], n[4];
              ld_shared_v4(mult + 4 * (C::kCols * h + r), m[0], m[1], m[2], m[3]);
              ld_shared_v4(neg + 4 * (C::kCols * h + r), n[0], n[1], n[2], n[3]);
#pragma unroll
              for (int i = 0; i < 4; ++i) y[r + i] = fmaf(__uint_as_float(s[r + i]), __uint_as_float(m[i]), __uint_as_float(n[i]));
            }
            if (!plain) {
#pragma unroll
              for (int r = 0; r < C::kCols; ++r) y[r] = key < static_cast<int>(ld_shared_b32(vis + 4 * (C::kCols * h + r))) ? y[r] : -INFINITY;
            }
#pragma unroll
            for (int r = 0; r < C::kCols; r += 2) top = fmax3(top, y[r], y[r + 1]);
            return top;
          };
          bool move = tile.first;
          float top = 0.f;
          if (!move) top = logits();
          // Does any key of the tile exceed what P~ may reach?  The four warps decide together (a unit's first tile always moves).
          if (!move) {
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
          if (move) {
            // The largest logit of every row: over the warp, then over the four warps; lane r keeps row r.
            float mine = -INFINITY;
            uint32_t s[C::kCols];
            scores(s);
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
            logits();
          }
          if (h == C::kParts - 1) {
            tc_fence_before_sync();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(C::X_SEMPTY + sb));         // the scores have been read
          }
#pragma unroll
          for (int r = 0; r < C::kCols; r += 2) {
            const float p0 = ex2_approx(y[r]), p1 = ex2_approx(y[r + 1]);
            l[C::kCols * h + r] += p0;
            l[C::kCols * h + r + 1] += p1;
            pk[(C::kCols * h + r) / 2] = pack_f16x2(p0, p1);
          }
        }
        if (!ok) break;
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
      if (tile.valid) load_q(tile.u, un + 1);
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
      tc_fence_before_sync();      // O has been read: this warp's next PREADY arrival lets the next unit overwrite it
      ++un;
    }
    if (!ok && lane == 0) report_timeout(prm.status);
  } else if (wid < kSoftmaxWarps + kWidenWarps) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kWidenRegs));
    // ======================================================== widening: raw pages -> operand chunks in tensor memory
    const int quad = wid & 3, group = (wid >> 2) - 1;
    const uint32_t ring = tbase + (static_cast<uint32_t>(quad * 32) << 16) + C::kRing;
    const uint32_t raw = smem_base + C::kOffRaw, infos = smem_base + C::kOffInfo;
    uint32_t cc = 0;                                        // chunks so far: chunk cc is for group cc % 2
    uint32_t kslot = 0, kpar = 0, vslot = 0;
    auto next_slot = [&](uint32_t s) { return s + 1 == C::kSlots ? 0u : s + 1; };
    // waits for chunk cc's place, and hands it over
    auto place = [&]() {
      const bool free = warp_wait(bar(C::X_AEMPTY) + 8 * (cc % C::kBufs), ((cc / C::kBufs) & 1) ^ 1);
      tc_fence_after_sync();
      return free;
    };
    auto hand_over = [&]() {
      tmem_wait_st();
      tc_fence_before_sync();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(C::X_AFULL) + 8 * (cc % C::kBufs));
    };
    Tiles vt = tile;
    auto widen_k = [&](int np) {                            // lane = key of the tile, 64 columns a chunk
      const uint32_t slot1 = np == 2 ? next_slot(kslot) : kslot;
      ok = warp_wait(bar(C::X_FULL) + 8 * kslot, kpar);
      if (ok && np == 2) ok = warp_wait(bar(C::X_FULL) + 8 * slot1, slot1 == 0 ? kpar ^ 1 : kpar);
      if (!ok) return;
      const uint32_t slot = quad < 2 ? kslot : slot1, key = 32 * (quad & 1) + lane;
      const uint32_t codes = raw + slot * kPageBytes4 + key * kCodeRow, scales = raw + slot * kPageBytes4 + kCodeBytes + key * kScaleRow;
      const uint32_t there = ld_shared_b32(infos + 4 * slot) != 0 ? 0xffffffffu : 0u;      // a page outside the cache: zeros
#pragma unroll 1
      for (int c = 0; c < kColBlocks; ++c, ++cc) {
        if ((cc & 1) != static_cast<uint32_t>(group)) continue;
        uint32_t w[8], r[32];
        ld_shared_v4(codes + 32 * c, w[0], w[1], w[2], w[3]);
        ld_shared_v4(codes + 32 * c + 16, w[4], w[5], w[6], w[7]);
        const uint32_t s = ld_shared_b32(scales + 4 * c) & there;
        const uint32_t s01 = e4m3x2_to_f16x2(s & 0xffffu), s23 = e4m3x2_to_f16x2(s >> 16);
        const uint32_t sc[4] = {__byte_perm(s01, 0, 0x1010), __byte_perm(s01, 0, 0x3232), __byte_perm(s23, 0, 0x1010), __byte_perm(s23, 0, 0x3232)};
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          uint32_t x[4];
          e2m1x8_to_f16x2(w[j], x);
#pragma unroll
          for (int i = 0; i < 4; ++i) r[4 * j + i] = mul_f16x2(x[i], sc[j / 2]);
        }
        ok = place();
        if (!ok) return;
        tmem_st_32x32b_x32(ring + 32 * (cc % C::kBufs), r);
        hand_over();
      }
      kslot = next_slot(kslot);
      if (kslot == 0) kpar ^= 1;
      if (np == 2) { kslot = next_slot(kslot); if (kslot == 0) kpar ^= 1; }
    };
    // Lanes = V's columns, 32 keys a chunk.  A thread (g = lane / 4, q = lane % 4) takes the 32-bit words g, eight neighbouring
    // columns, of warp `quad`'s 64 columns, for eight keys: words of two keys are interleaved by nibbles and converted, which
    // gives pairs of keys.  Column i of a word goes to block 2p + i / 4, lane 32 quad + g + 8 (i % 4).  A step of the product is 16 keys, k = 4 q + e:
    // key 4 q + (q + e) % 4, so that the four q read four different residues (a row is 72 words: else all from the same banks).
    // A scale that is a NaN becomes a number here: through K the rows that see the key have a NaN for its P~, and those that do
    // not have a zero, which a NaN in V would turn into one.
    auto widen_v = [&](int np, int t, int n_b) {
      const uint32_t slot1 = np == 2 ? next_slot(vslot) : vslot;
      const int g = lane >> 2, q = lane & 3;
#pragma unroll 1
      for (int c = 0; c < kVChunks; ++c, ++cc) {
        if ((cc & 1) != static_cast<uint32_t>(group)) continue;
        const int p = c >> 2, kq = c & 3;
        const uint32_t slot = kq < 2 ? vslot : slot1;
        const uint32_t page = raw + slot * kPageBytes4, first = 32 * (kq & 1);
        const int count = (kq < 2 || np == 2 ? static_cast<int>(ld_shared_b32(infos + 4 * slot)) : 0) - static_cast<int>(first);   // keys of this quarter that count
        uint32_t r[2][2][8];
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          uint32_t w[4], s[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int in_quarter = 16 * b + 4 * q + ((q + e) & 3);
            const uint32_t key = first + in_quarter;
            w[e] = ld_shared_b32(page + key * kCodeRow + 32 * (4 * p + quad) + 4 * g);
            s[e] = ld_shared_u8(page + kCodeBytes + key * kScaleRow + 4 * (4 * p + quad) + (g >> 1));
          }
          if (count < 32) {                                 // what is beyond the sequence's end may be anything: a scale of zero
#pragma unroll
            for (int e = 0; e < 4; ++e) s[e] = 16 * b + 4 * q + ((q + e) & 3) < count ? s[e] : 0u;
          }
#pragma unroll
          for (int j = 0; j < 2; ++j) {                     // keys e = 2j, 2j + 1
            const uint32_t w0 = w[2 * j], w1 = w[2 * j + 1];
            const uint32_t even = (w0 & 0x0f0f0f0fu) | ((w1 << 4) & 0xf0f0f0f0u), odd = ((w0 >> 4) & 0x0f0f0f0fu) | (w1 & 0xf0f0f0f0u);
            const uint32_t sc = number_f16x2(e4m3x2_to_f16x2(s[2 * j] | (s[2 * j + 1] << 8)));
            uint32_t x[4], z[4];
            e2m1x8_to_f16x2(even, x);
            e2m1x8_to_f16x2(odd, z);
#pragma unroll
            for (int i = 0; i < 4; ++i) {                   // columns 2i (lanes .. + g) and 2i + 1 (.. + 8 + g)
              r[i >> 1][i & 1][4 * b + j] = mul_f16x2(x[i], sc);
              r[i >> 1][i & 1][4 * b + 2 + j] = mul_f16x2(z[i], sc);
            }
          }
        }
        ok = place();
        if (!ok) return;
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
          for (int hh = 0; hh < 2; ++hh) tmem_st_16x256b_x2(ring + (static_cast<uint32_t>(16 * hh) << 16) + 32 * (cc % C::kBufs) + 16 * m, r[m][hh]);
        hand_over();
      }
      if (lane == 0) {                                      // (the words are in registers, and in tensor memory)
        mbar_arrive(bar(C::X_EMPTY) + 8 * vslot);
        if (np == 2) mbar_arrive(bar(C::X_EMPTY) + 8 * slot1);
      }
      vslot = next_slot(slot1);
    };
    // The order of the MMA warp.  K is always one tile ahead of V, but at the end of a unit (tile is the one behind vt, or vt's own while
    // a unit begins).
    auto k_next = [&]() { widen_k(tile.np); tile.next(); };
    if (tile.valid) k_next();
    while (ok && vt.valid) {
      if (tile.valid && !tile.first) k_next();
      if (!ok) break;
      widen_v(vt.np, vt.t, vt.u.n_b);
      if (!ok) break;
      vt.next();
      if (vt.valid && vt.first) k_next();
    }
    if (!ok && lane == 0) report_timeout(prm.status);
  } else {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kIssueRegs));
    if (wid == kMmaWarp) {
    // ======================================================== MMAs
    if (elect_one()) {
      constexpr uint32_t idesc_s = make_idesc_f16(128, kN, false, false), idesc_o = make_idesc_f16(128, kN, false, true);
      constexpr uint32_t dhi = smem_desc_hi_sw128(1024);
      const uint32_t qlo = smem_desc_lo(smem_base, 16), plo = smem_desc_lo(smem_base + C::kOffP, 16);
      const uint32_t ring = tbase + C::kRing;
      uint32_t cc = 0, gs = 0, gp = 0, un = 0;
      Tiles vt = tile;
      auto chunk = [&]() {
        ok = mbar_wait(bar(C::X_AFULL) + 8 * (cc % C::kBufs), (cc / C::kBufs) & 1);
        if (ok) tc_fence_after_sync();
        return ok;
      };
      auto qk = [&]() {
        if (tile.first) {
          ok = mbar_wait(bar(C::X_QREADY), un & 1);
          if (!ok) return;
          ++un;
        }
        const uint32_t sb = gs & 1, d = tbase + C::kSCol + sb * kN;
        ok = mbar_wait(bar(C::X_SEMPTY) + 8 * sb, ((gs >> 1) & 1) ^ 1);
        if (!ok) return;
        tc_fence_after_sync();
        uint32_t ql = qlo;
#pragma unroll 1
        for (int c = 0; c < kColBlocks; ++c) {
          if (!chunk()) return;
          const uint32_t a = ring + 32 * (cc % C::kBufs);
#pragma unroll
          for (int kk = 0; kk < 4; ++kk) mma_ts(d, a + 8 * kk, smem_desc_join(ql + 2 * kk, dhi), idesc_s, (c | kk) != 0);
          mma_commit(bar(C::X_AEMPTY) + 8 * (cc % C::kBufs));
          ++cc;
          ql += C::kQBlock >> 4;
        }
        mma_commit(bar(C::X_SFULL) + 8 * sb);
        ++gs;
        tile.next();
      };
      auto pv = [&]() {
        ok = mbar_wait(bar(C::X_PREADY), gp & 1);
        if (!ok) return;
        tc_fence_after_sync();
        const uint32_t acc = vt.first ? 0u : 1u;
#pragma unroll 1
        for (int c = 0; c < kVChunks; ++c) {
          if (!chunk()) return;
          const uint32_t a = ring + 32 * (cc % C::kBufs), kq = c & 3;
          const uint32_t d = tbase + C::kOCol + 2 * kN * (c >> 2), pl = plo + kq * (32 * 128 >> 4);
#pragma unroll
          for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int kk = 0; kk < 2; ++kk) mma_ts(d + kN * m, a + 16 * m + 8 * kk, smem_desc_join(pl + kk * (16 * 128 >> 4), dhi), idesc_o, (kq | kk) != 0 ? 1u : acc);
          mma_commit(bar(C::X_AEMPTY) + 8 * (cc % C::kBufs));
          ++cc;
        }
        mma_commit(bar(C::X_PVDONE));
        ++gp;
        vt.next();
      };
      if (tile.valid) qk();
      while (ok && vt.valid) {
        if (tile.valid && !tile.first) qk();
        if (ok) pv();
        if (ok && vt.valid && vt.first) qk();
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
        ok = mbar_wait(bar(C::X_EMPTY) + 8 * slot, par);
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
          mbar_wait(bar(C::X_FULL) + 8 * (j % C::kSlots), (j / C::kSlots) & 1);
        }
      }
    }
    __syncwarp();
    }
  }

  tc_fence_before_sync();
  __syncthreads();
  if (wid == kMmaWarp) tmem_dealloc(tbase, 512);
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
