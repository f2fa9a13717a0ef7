// Tensor-core MLA decode kernel for a cache held in 4 bits (format: amla_fp4.cuh), sm_100a.
//
// A key is 324 bytes.  Widened to 16 bits it is 1152 for K and 1024 for V, and a kernel that keeps widened operands in shared
// memory writes and reads all of that there.  Here they never are in shared memory: the raw page is, and the widening warps put what
// they make of it straight into tensor memory, as the A operand of transposed products.  With that the rows are N:
//
//   S^T = K Q^T       A = K: 128 keys (two pages) are the lanes, 64 of the 576 columns at a time; B = Q (shared memory, K-major)
//   O^T += V^T P~^T   A = V^T: V's columns are the lanes, 4 x 128 of them and 16 keys at a time; B = P~ (shared memory, MN-major)
//
// One CTA works on up to 16, 32 or 64 rows of a sequence and a range of its pages; O^T is four blocks of kN columns of tensor
// memory (256 for 64 rows), S^T one or more of kN, and the rest operand chunks of 32 columns, four places for K and two (64 rows) or four
// for V.  A 128-key tile is 17 chunks: nine of K (128 keys x 64 columns), eight of V (512 columns x 16 keys), four MMAs each.
//
// Everything is f16, not bf16: an E2M1 times an E4M3 number is exact in either, P~ has three more bits, and the conversion from
// E2M1 gives f16.  Q is bf16: a row is multiplied by the power of two that brings its largest magnitude into [2^14, 2^15), which
// leaves every element within 2^-31 of the row's largest exact, and smaller ones off by at most 2^-25 in units of which the largest has 2^14.
//
// The reference of the online softmax is an integer number of octaves n, so that a rescale of O and l is an add to the exponent
// bits and exact (nothing is left over to compensate).  P~ = 2^(a_j - n + 9): a move puts the largest P~ of a row into (2^8, 2^9], the
// next one comes when a key would exceed 2^15, and what f16 rounds to nothing is below 2^-33 of the reference.
//
// Warps: 4 (64 rows: 8, of 32 rows each group of four) for softmax, rescale and epilogue: a thread is a key and has all its rows, its share of the
// row sums stays in registers until the unit's end.  Then 8 that widen K and 8 that widen V, in two groups of four that take chunks by
// turns, and bring Q (all 16 of a part's first unit, K's of the others); then one each that issues K's products, V's, and the loads, which are
// whole tiles of raw pages (bulk copies), with a note on each tile that the other warps go by.
//
// What bounds it: the widening.  A tile at 64 rows takes ~4650 clk, of which the tensor pipe is busy 1750 and HBM's share is ~1850; ~3300
// instructions a scheduler are issued in them (16 rows: 3700, 2750), most of which convert (a pair of E2M1 numbers is one operation of 2 clk), multiply by the
// scales (another 2) and, for V, pair keys.  What changes the waits between the roles and not that work changed nothing or cost 2-3 %: more operand
// places, one ring for K and V, a chunk handed over later or two at a time, P~ in two halves, the next raw tile fetched as far as L2.
// About 26 K clk a CTA (16 rows: 20) are no tile's: set-up and first load 8, Q 2-6, the first tile's way through all roles, the last product
// and the epilogue 3-6; a further unit costs ~10, since there is one buffer of Q and one O^T, and the warps that widen K bring Q.  With 16 rows that is 20 of 50
// K clk, as much as the widening in the others.
// 32 x 4096 keys, 128 heads: 57.0 us a call, 641 TFLOP/s (the bf16 cache: 50.1); 64 x 1024-8192, two tokens: 205 (bf16: 168); 32 x 1024-8192, 16 heads: 30.3,
// 1.6 TB/s of 4-bit pages (bf16: 36.3), 32 heads: 33.1 (41.4), 64: 43.8 (54.0).  (In turn on one GPU, a second each.)  Widening the pages into a bf16 copy in
// front of the bf16 kernels took 90 for the first.
//
// Why 64 rows at most: O^T of 128 would be all of a CTA's tensor memory.  So 128 heads widen every page twice, two tokens of them four times, and are slower than
// from a bf16 cache; calls of few rows gain, and those of more pages than memory would hold at 16 bits.  (A pair MMA, M = 256, takes each half of A from
// its own CTA's tensor memory, so that a pair could widen half a page each for 128 rows: not built.)
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

constexpr int kWidenWarps = 16;                         // K: two groups of four, V: two groups of four
constexpr int kColBlocks = kDqk / 64;                   // K chunks of a tile
constexpr int kVChunks = 8;                             // V chunks of a tile: 16 keys, all 512 columns
constexpr uint32_t kPBytes = 128 * 128;                 // P~: [128 keys][64 rows of f16], 128-byte swizzle
constexpr uint32_t kTileBytes = 2 * kPageBytes4;
constexpr int kSmemPlanItems = 512;
constexpr float kPBias = 9.f, kPLimit = 15.f;           // P~ = 2^(a - n + 9), at most 2^15
constexpr int kUnitsAhead = 4;                          // units that may be between Q's loading and the softmax, and one

// What the loader says of a tile: how many keys of its two pages count (none: no such page, or one outside the cache, which is zeros),
// whether it has two, whether it opens or ends a unit, and whether it is the part's last.
constexpr int kNotes = 16;                              // tiles (and units) between the loader and the products of V at most, and more
constexpr uint32_t kKeysMask = 127, kSecondPage = 8, kTwoPages = 1 << 15, kFirstTile = 1 << 16, kEndsUnit = 1 << 17, kLastTile = 1 << 18;

template <int kN>
struct Shape {
  static constexpr int kGroups = kN == 64 ? 2 : 1;      // softmax warpgroups, each of them with its own rows
  static constexpr int kCols = kN / kGroups;
  static constexpr int kSoftmaxWarps = 4 * kGroups, kKWarp = kSoftmaxWarps, kVWarp = kKWarp + kWidenWarps / 2;
  static constexpr int kQkWarp = kVWarp + kWidenWarps / 2, kPvWarp = kQkWarp + 1, kLoadWarp = kQkWarp + 2;   // (the one behind them has no role)
  static constexpr int kThreads = 32 * (kQkWarp + 4);
  // Registers a thread, by warpgroup: together what the block is launched with
  static constexpr int kLaunchRegs = 65536 / kThreads / 8 * 8;
  static constexpr int kSoftmaxRegs = kN == 64 ? 104 : 136, kWidenRegs = kN == 64 ? 64 : 72, kIssueRegs = kN == 64 ? 40 : 56;
  static_assert(kGroups * kSoftmaxRegs + 4 * kWidenRegs + kIssueRegs <= kThreads / 128 * kLaunchRegs, "the block has no more to give out");
  static constexpr int kSlots = kN == 64 ? 3 : 4;       // tiles (two pages) in shared memory
  // Operand chunks in tensor memory, of K and of V: a tile's always have the same places, and a place is always the same group's.
  static constexpr int kKBufs = 4, kVBufs = kN == 64 ? 2 : 4;
  static constexpr int kSBufs = kN == 64 ? 1 : 2;       // score tiles in tensor memory
  static constexpr uint32_t kQBlock = kN * 128;         // [rows][64 columns of f16], 128-byte swizzle
  static constexpr uint32_t kOffP = kColBlocks * kQBlock;
  static constexpr uint32_t kOffRaw = kOffP + kPBytes;
  static constexpr uint32_t kOffMult = kOffRaw + kSlots * kTileBytes;      // float [units ahead][rows]: logit per product, in octaves
  static constexpr uint32_t kOffVis = kOffMult + kUnitsAhead * kN * 4;      // int [units ahead][rows]: keys that the row sees
  static constexpr uint32_t kOffNeg = kOffVis + kUnitsAhead * kN * 4;       // float [softmax warps][columns]: 9 - n
  static constexpr uint32_t kOffAdd = kOffNeg + kSoftmaxWarps * kCols * 4;  // float [softmax warps][columns]: the octaves of a move; 1 / l at the end
  static constexpr uint32_t kOffSums = kOffAdd + kSoftmaxWarps * kCols * 4; // float [2 units][softmax warps][columns]
  static constexpr uint32_t kOffMax = kOffSums + 2 * kSoftmaxWarps * kCols * 4;   // float [2][softmax warps][32]
  static constexpr uint32_t kOffMoves = kOffMax + 2 * kSoftmaxWarps * 32 * 4;     // uint32 [2][softmax warps]
  static_assert(kOffMoves % 16 == 0 && kOffNeg % 16 == 0, "read four at a time");
  static constexpr uint32_t kOffNotes = kOffMoves + 2 * kSoftmaxWarps * 4;  // uint2 [notes]: what the loader says of a tile, its first key
  static constexpr uint32_t kOffUnits = kOffNotes + kNotes * 8;             // int4 [notes][2] of a unit: sequence, first row, keys, -; slot of its partial (-1:
                                                                            // none), item, slot of the item's first partial, partials
  static constexpr uint32_t kOffBars = kOffUnits + kNotes * 32;
  static constexpr uint32_t kBarBytes = 384;
  static constexpr uint32_t kOffPlan = kOffBars + kBarBytes;
  static constexpr uint32_t kOffLens = kOffPlan + ((kSmemPlanItems + 1) * 4 + 15) / 16 * 16;
  static constexpr uint32_t kOffFirst = kOffLens + kSmemPlanItems * 4;
  static constexpr uint32_t kBytes = kOffFirst + sizeof(FirstUnit);
  // tensor-memory columns
  static constexpr uint32_t kOCol = 0, kSCol = 4 * kN, kKCol = 512 - 32 * (kKBufs + kVBufs), kVCol = 512 - 32 * kVBufs;
  enum { X_FULL = 0, X_EMPTY = X_FULL + kSlots, X_KFULL = X_EMPTY + kSlots, X_KEMPTY = X_KFULL + kKBufs, X_VFULL = X_KEMPTY + kKBufs, X_VEMPTY = X_VFULL + kVBufs, X_QREADY = X_VEMPTY + kVBufs,
         X_SFULL = X_QREADY + kUnitsAhead, X_SEMPTY = X_SFULL + kSBufs, X_PREADY = X_SEMPTY + kSBufs, X_PVDONE, X_MOVES, X_MAX = X_MOVES + kGroups, X_SUMS = X_MAX + kGroups,
         X_START = X_SUMS + kGroups, X_QKDRAIN, X_PVDRAIN, X_NUM };
  static_assert(X_NUM * 8 + 8 <= kBarBytes, "barrier area too small");
  static_assert(kBytes <= 232448, "exceeds the shared memory a block can opt in to");
  static_assert(kOffP % 1024 == 0 && kOffRaw % 1024 == 0 && kTileBytes % 16 == 0 && kOffBars % 8 == 0, "alignment");
  static_assert(kSCol + kSBufs * kN <= kKCol && kSlots + 4 < kNotes, "tensor memory");
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
// 16 lanes x 16 columns in two blocks of eight: thread (g = lane / 4, q = lane % 4) gives columns 2q, 2q + 1 of lanes g (r0, r1) and g + 8 (r2, r3) of
// either block
__device__ __forceinline__ void tmem_st_16x256b_x2(uint32_t taddr, const uint32_t (&r)[8]) {
  asm volatile("tcgen05.st.sync.aligned.16x256b.x2.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]),
               "r"(r[6]), "r"(r[7])
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
__global__ void __launch_bounds__(Shape<kN>::kThreads, 1) decode_fp4_kernel(const DecodeParams prm) {
  using C = Shape<kN>;
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  const uint32_t smem_base = smem_u32(smem_raw);
  constexpr int kThreads = C::kThreads, kSoftmaxWarps = C::kSoftmaxWarps, kLoadWarp = C::kLoadWarp;
  const int tid = threadIdx.x, lane = tid & 31;
  const int wid = __shfl_sync(0xffffffffu, tid >> 5, 0);     // (the compiler then knows that it is the same in the whole warp)
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
    for (int i = 0; i < kUnitsAhead; ++i) mbar_init(bar(C::X_QREADY + i), kWidenWarps);
    for (int i = 0; i < C::kSBufs; ++i) { mbar_init(bar(C::X_SFULL + i), 1); mbar_init(bar(C::X_SEMPTY + i), kSoftmaxWarps); }
    mbar_init(bar(C::X_PREADY), kSoftmaxWarps);
    mbar_init(bar(C::X_PVDONE), 1);
    mbar_init(bar(C::X_START), 1);
    mbar_init(bar(C::X_QKDRAIN), 1);
    mbar_init(bar(C::X_PVDRAIN), 1);
    for (int i = 0; i < C::kGroups; ++i) { mbar_init(bar(C::X_MOVES + i), 4); mbar_init(bar(C::X_MAX + i), 4); mbar_init(bar(C::X_SUMS + i), 4); }
    fence_mbar_init();
  }
  if (wid == C::kQkWarp) { tmem_alloc(tmem_slot, 512); tmem_relinquish(); }
  if (plan_here) {
    if (by_warp) __syncwarp(); else __syncthreads();
    if (wid == kLoadWarp) {
      plan_units(prm, plan_smem, lens_smem, first_smem, part, lane);
      __syncwarp();
      // the first unit's Q on its way (into L2, where it is coherent: the guess may be wrong, and Q may still be written)
      const Unit& u = first_smem->u;
      if (lane == 0 && u.t1 > u.t0)
        bulk_prefetch_l2(prm.q + (static_cast<size_t>(u.b) * prm.R + u.r0) * kDqk, static_cast<uint32_t>(min(kN, prm.R - u.r0)) * (kDqk * 2));
    }
  }
  if (tid == 0) AMLA_STAMP(prm, part, 20, 1);
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  if (tid == 0) AMLA_STAMP(prm, part, 20, 2);
  // All 512 columns: they begin at 0.  (An address that is a constant keeps the issue of an MMA short.)
  constexpr uint32_t tbase = 0;
  if (ld_shared_b32(tmem_slot) != 0) {
    if (tid == 0) report_timeout(prm.status);
    if (wid == C::kQkWarp) tmem_dealloc(ld_shared_b32(tmem_slot), 512);
    return;
  }

  const int* prefix = plan_here ? plan_smem : prm.prefix;
  const int* seqlens = plan_here ? lens_smem : prm.seqlens;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;");
  if (tid == 0) AMLA_STAMP(prm, part, 20, 3);
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
  if (tid == 0) AMLA_STAMP(prm, part, 20, 4);
  bool ok = true;
  const FirstUnit* first = plan_here ? first_smem : nullptr;

  if (wid < kSoftmaxWarps) {
    // ======================================================== softmax, rescale, epilogue
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(C::kSoftmaxRegs));
    constexpr int kCols = C::kCols;
    const int quad = wid & 3, group = wid >> 2, col0 = group * kCols;  // this group's rows are col0 ..
    const uint32_t lane_base = static_cast<uint32_t>(quad * 32) << 16;
    const uint32_t o_addr = tbase + lane_base + C::kOCol + col0;
    const uint32_t neg = smem_base + C::kOffNeg + wid * kCols * 4, add = smem_base + C::kOffAdd + wid * kCols * 4;
    // Key 32 quad + lane of the tile is row k of P~: the order in which the widening warps put V's keys (see there).
    const int q4 = (lane >> 2) & 3, k = 32 * quad + (lane & 16) + 4 * q4 + (((lane & 3) - q4) & 3);
    const uint32_t p_dst = smem_base + C::kOffP + k * 128, p_sw = k & 7;
    uint32_t gs = 0, un = 0, moves = 0, maxes = 0;
    if (tid == 0) merge_begin(prm, part);
    write_empty_items(prm, prefix, part, prm.P, 0, kN, tid, 32 * kSoftmaxWarps);
    ok = warp_wait(bar(C::X_START), 0);
    bool units_left = ok && static_cast<int>(ld_shared_b32(smem_base + C::kOffUnits + 8)) > 0;
    while (units_left) {
      const uint32_t unit = smem_base + C::kOffUnits + (un % kNotes) * 32;
      const uint32_t mult = smem_base + C::kOffMult + ((un % kUnitsAhead) * kN + col0) * 4, vis = smem_base + C::kOffVis + ((un % kUnitsAhead) * kN + col0) * 4;
      float l[kCols];
#pragma unroll
      for (int i = 0; i < kCols; ++i) l[i] = 0.f;
      if (lane < kCols) st_shared_b32(neg + 4 * lane, 0u);
      __syncwarp();
      ok = warp_wait(bar(C::X_QREADY + un % kUnitsAhead), (un / kUnitsAhead) & 1);   // mult, vis
      if (!ok) break;
      uint32_t note = 0;
      do {
        const uint32_t sb = gs % C::kSBufs;
        ok = warp_wait(bar(C::X_SFULL) + 8 * sb, (gs / C::kSBufs) & 1);
        if (!ok) break;
        tc_fence_after_sync();
        if (tid == 0) AMLA_STAMP(prm, part, 7, gs);
        float y[kCols];                                                // a - n + 9, in octaves (a unit's first tile: a, as long as n is not known)
        {
          uint32_t s[kCols];
          tmem_ld_cols<kCols>(tbase + lane_base + C::kSCol + sb * kN + col0, s);
          tmem_wait_ld();
          tc_fence_before_sync();
          __syncwarp();
          mbar_arrive_if(lane == 0, bar(C::X_SEMPTY) + 8 * sb);        // the scores are in registers
#pragma unroll
          for (int r = 0; r < kCols; r += 4) {
            uint32_t m[4], n[4];
            ld_shared_v4(mult + 4 * r, m[0], m[1], m[2], m[3]);
            ld_shared_v4(neg + 4 * r, n[0], n[1], n[2], n[3]);
#pragma unroll
            for (int i = 0; i < 4; i += 2)
              unpack_f32x2(fma_f32x2(pack_f32x2(__uint_as_float(s[r + i]), __uint_as_float(s[r + i + 1])), pack_f32x2(__uint_as_float(m[i]), __uint_as_float(m[i + 1])),
                                     pack_f32x2(__uint_as_float(n[i]), __uint_as_float(n[i + 1]))),
                           y[r + i], y[r + i + 1]);
          }
        }
        uint32_t key0;
        ld_shared_v2(smem_base + C::kOffNotes + 8 * (gs % kNotes), note, key0);
        const bool first = note & kFirstTile, two = note & kTwoPages;
        // all rows see what is in front of their sequence's last Sq - 1 keys
        const bool plain = two && static_cast<int>(key0) + 2 * kPage <= static_cast<int>(ld_shared_b32(unit + 8)) - prm.Sq + 1;
        if (!plain) {
          const int in_tile = 32 * quad + lane;
          const int key = two || in_tile < kPage ? static_cast<int>(key0) + in_tile : 0x7fffffff;
#pragma unroll
          for (int r = 0; r < kCols; ++r) y[r] = key < static_cast<int>(ld_shared_b32(vis + 4 * r)) ? y[r] : -INFINITY;
        }
        bool move = first;
        if (!move) {
          // Does any key of the tile exceed what P~ may reach?  The group's four warps decide together.
          float top = -INFINITY;
#pragma unroll
          for (int r = 0; r < kCols; r += 2) top = fmax3(top, y[r], y[r + 1]);
          const uint32_t mine = __any_sync(0xffffffffu, top > kPLimit) ? 1u : 0u;
          const uint32_t at = smem_base + C::kOffMoves + (moves & 1) * (kSoftmaxWarps * 4) + group * 16;
          if (lane == 0) st_shared_b32(at + 4 * quad, mine);
          mbar_arrive_if(lane == 0, bar(C::X_MOVES + group));
          ok = warp_wait(bar(C::X_MOVES + group), moves & 1);
          if (!ok) break;
          ++moves;
          uint32_t f[4];
          ld_shared_v4(at, f[0], f[1], f[2], f[3]);
          move = (f[0] | f[1] | f[2] | f[3]) != 0;
        }
        if (move) {
          // The largest of every row: over the warp, then over the four warps; lane r keeps row r.
          float mine = -INFINITY;
#pragma unroll
          for (int r = 0; r < kCols; ++r) {
            const float a = warp_max(y[r]);
            if (lane == r) mine = a;
          }
          const uint32_t at_max = smem_base + C::kOffMax + ((maxes & 1) * kSoftmaxWarps + 4 * group) * 128 + 4 * lane;
          st_shared_b32(at_max + 128 * quad, __float_as_uint(mine));
          __syncwarp();
          mbar_arrive_if(lane == 0, bar(C::X_MAX + group));
          ok = warp_wait(bar(C::X_MAX + group), maxes & 1);
          if (!ok) break;
          ++maxes;
#pragma unroll
          for (int w = 0; w < 4; ++w) mine = fmaxf(mine, ld_shared_f32(at_max + 128 * w));
          // Every row whose maximum rose above the reference moves to it (moving early is always allowed), in a unit's first tile all do.
          float d = 0.f;
          if (lane < kCols) {
            if (first ? mine > -INFINITY : mine > kPBias) d = kPBias - ceilf(mine);
            st_shared_b32(neg + 4 * lane, __float_as_uint(ld_shared_f32(neg + 4 * lane) + d));
            st_shared_b32(add + 4 * lane, __float_as_uint(d));
          }
          __syncwarp();
#pragma unroll
          for (int r = 0; r < kCols; r += 4) {
            uint32_t x[4];
            ld_shared_v4(add + 4 * r, x[0], x[1], x[2], x[3]);
#pragma unroll
            for (int i = 0; i < 4; ++i) y[r + i] += __uint_as_float(x[i]);
          }
          if (!first) {
            // O <- AS_FP32(AS_INT32(O) + d * 2^23): O^T has a row per column, a thread the same d for all of a row
            const int d_bits = static_cast<int>(fmaxf(d, -255.f)) * (1 << 23);
            ok = warp_wait(bar(C::X_PVDONE), (gs - 1) & 1);
            if (!ok) break;
            tc_fence_after_sync();
#pragma unroll 1
            for (int m = 0; m < 4; ++m) {
              uint32_t o[kCols];
              tmem_ld_cols<kCols>(o_addr + kN * m, o);
              tmem_wait_ld();
#pragma unroll
              for (int r = 0; r < kCols; ++r) o[r] = __float_as_uint(lower_octaves(__uint_as_float(o[r]), __shfl_sync(0xffffffffu, d_bits, r)));
              tmem_st_cols<kCols>(o_addr + kN * m, o);
            }
            tmem_wait_st();
#pragma unroll
            for (int r = 0; r < kCols; ++r) l[r] = lower_octaves(l[r], __shfl_sync(0xffffffffu, d_bits, r));
          }
        }
        uint32_t pk[kCols / 2];
#pragma unroll
        for (int r = 0; r < kCols; r += 2) {
          const float p0 = ex2_approx(y[r]), p1 = ex2_approx(y[r + 1]);
          unpack_f32x2(add_f32x2(pack_f32x2(l[r], l[r + 1]), pack_f32x2(p0, p1)), l[r], l[r + 1]);
          pk[r / 2] = pack_f16x2(p0, p1);
        }
        if (tid == 0) AMLA_STAMP(prm, part, 9, gs);
        if (gs > 0) {
          ok = warp_wait(bar(C::X_PVDONE), (gs - 1) & 1);              // the P~V of the tile before has read the P buffer
          if (!ok) break;
        }
#pragma unroll
        for (int c = 0; c < kCols / 8; ++c) st_shared_v4(p_dst + (((c + col0 / 8) ^ p_sw) << 4), pk[4 * c], pk[4 * c + 1], pk[4 * c + 2], pk[4 * c + 3]);
        tc_fence_before_sync();                                        // O (perhaps) rewritten
        fence_proxy_async_smem();
        __syncwarp();
        mbar_arrive_if(lane == 0, bar(C::X_PREADY));
        if (tid == 0) AMLA_STAMP(prm, part, 8, gs);
        ++gs;
      } while (!(note & kEndsUnit));
      if (!ok) break;
      // ---- epilogue: out = O / l, lse = n + log2 l
      if (tid == 0) AMLA_STAMP(prm, part, 10, un);
      uint32_t u_b, u_r0, u_n, unused, u_slot, u_item, info_x, info_y;
      ld_shared_v4(unit, u_b, u_r0, u_n, unused);
      ld_shared_v4(unit + 16, u_slot, u_item, info_x, info_y);
      const int pslot = static_cast<int>(u_slot);                      // partial slot, or -1
      if (tid == 0) merge_note(prm, part, u_item, make_int2(info_x, info_y));
      const uint32_t sums = smem_base + C::kOffSums + ((un & 1) * kSoftmaxWarps + 4 * group) * (kCols * 4) + 4 * (lane % kCols);
      const float mine = sum_rows<kCols>(l, lane);
      if (lane < kCols) st_shared_b32(sums + quad * (kCols * 4), __float_as_uint(mine));
      __syncwarp();
      mbar_arrive_if(lane == 0, bar(C::X_SUMS + group));
      ok = warp_wait(bar(C::X_SUMS + group), un & 1);
      if (!ok) break;
      const size_t row0 = static_cast<size_t>(u_b) * prm.R + u_r0 + col0, prow0 = static_cast<size_t>(pslot < 0 ? 0 : pslot) * kN + col0;
      const int rows = prm.R - static_cast<int>(u_r0) - col0;                            // live ones among the group's
      // A partial travels in half precision.  It is an average of values of at most 2688, so that 8 times it, and the part of out_scale in [1, 2),
      // is below a half's 65504; the power of two that is left of out_scale is its chunks' scale byte.
      const uint32_t scale_bits = __float_as_uint(prm.out_scale);
      const int scale_exp = static_cast<int>(scale_bits >> 23) - 3;
      const float factor = pslot < 0 ? prm.out_scale : __uint_as_float((scale_bits & 0x7fffffu) | (130u << 23));
      auto scale_word = [&](int r) -> uint32_t& { return reinterpret_cast<uint32_t*>(partial_scales(prm))[(prow0 + r) * 4 + quad]; };   // of this warp's 128 columns
      if (lane < kCols) {
        float total = 0.f;
#pragma unroll
        for (int w = 0; w < 4; ++w) total += ld_shared_f32(sums + w * (kCols * 4));
        st_shared_b32(add + 4 * lane, __float_as_uint(total == 0.f ? 0.f : factor / total));
        if (quad == 0 && lane < rows) {
          const float lse = total == 0.f ? -INFINITY : (log2f(total) - ld_shared_f32(neg + 4 * lane)) * kLn2;
          if (pslot < 0) prm.lse[row0 + lane] = lse;
          else prm.part_lse[prow0 + lane] = lse;
        }
        if (pslot >= 0) scale_word(lane) = static_cast<uint32_t>(scale_exp) * 0x01010101u;
      }
      __syncwarp();
      ok = warp_wait(bar(C::X_PVDONE), (gs - 1) & 1);
      if (!ok) break;
      tc_fence_after_sync();
      // Lane L of block m of O^T is column 128 quad + 16 (L % 8) + 4 m + (L / 8) % 4: the four lanes with one L % 8 hold eight neighbouring
      // columns of every row in two blocks.  They exchange four rows, a lane is left with eight columns of one: 16 bytes.
      uint16_t* dst = pslot < 0 ? reinterpret_cast<uint16_t*>(prm.out) + row0 * kDv : partial_halves(prm) + prow0 * kDv;
      const int last = pslot < 0 ? rows : kCols;
      const bool b0 = lane & 8, b1 = lane & 16;
      dst += 128 * quad + 16 * (lane & 7) + static_cast<size_t>(lane >> 3) * kDv;
      // (Four rows at a time in a loop that stays rolled: it is run through once, and what costs is to fetch its code.)
      uint32_t again = 0;
#pragma unroll 1
      while (true) {
        uint16_t* to = dst;
        bool small = false;
#pragma unroll 1
        for (int j = 0; j < kCols; j += 4) {
          uint32_t o[4][4], f[4], any = 0;
#pragma unroll
          for (int m = 0; m < 4; ++m) tmem_ld_32x32b_x4(o_addr + kN * m + j, o[m]);
          ld_shared_v4(add + 4 * j, f[0], f[1], f[2], f[3]);
          tmem_wait_ld();
          const int row = j + (lane >> 3);
#pragma unroll
          for (int p = 0; p < 2; ++p) {                                // blocks 2p, 2p + 1
            uint32_t a[4];
#pragma unroll
            for (int c = 0; c < 4; ++c) {
              const float x = __uint_as_float(o[2 * p][c]) * __uint_as_float(f[c]), z = __uint_as_float(o[2 * p + 1][c]) * __uint_as_float(f[c]);
              a[c] = pslot < 0 ? pack_bf16x2(x, z) : pack_f16x2(x, z);
            }
            const uint32_t g0 = __shfl_xor_sync(0xffffffffu, b1 ? a[0] : a[2], 16), g1 = __shfl_xor_sync(0xffffffffu, b1 ? a[1] : a[3], 16);
            const uint32_t k0 = b1 ? a[2] : a[0], k1 = b1 ? a[3] : a[1];             // rows 2 b1 + 0, 1: own, and (g) of the lane 16 away
            const uint32_t t0 = __shfl_xor_sync(0xffffffffu, b0 ? k0 : k1, 8), t1 = __shfl_xor_sync(0xffffffffu, b0 ? g0 : g1, 8);
            const uint32_t kk = b0 ? k1 : k0, kg = b0 ? g1 : g0;                      // row 2 b1 + b0 from lanes L, L ^ 16, L ^ 8 (t0), L ^ 24 (t1)
            const uint32_t m0 = b0 ? t0 : kk, m1 = b0 ? kk : t0, n0 = b0 ? t1 : kg, n1 = b0 ? kg : t1;
            const uint32_t c0 = b1 ? n0 : m0, c1 = b1 ? n1 : m1, c2 = b1 ? m0 : n0, c3 = b1 ? m1 : n1;   // columns (i, i + 4)
            any |= c0 | c1 | c2 | c3;
            if (row < last)
              stg_128(to + 8 * p, __byte_perm(c0, c1, 0x5410), __byte_perm(c2, c3, 0x5410), __byte_perm(c0, c1, 0x7632), __byte_perm(c2, c3, 0x7632));
          }
          small |= (any & 0x60006000u) == 0;
          to += 4 * kDv;
        }
        // Where 16 columns of a row have a half of 2^-7 or more, its smallest step is 2^-17 of that, and what is above 2^-8 of it has the bits of bf16
        // and more.  An average of many small values may be smaller, and then the partial's rows get powers of two of their own (the largest of a row's
        // 128 columns into [1, 2)), and are written once more.  (With those always, 32 x 4096 keys took 58.5 us against 56.5.)
        asm volatile("" : "+r"(again));
        if (pslot < 0 || again != 0 || !__any_sync(0xffffffffu, small)) break;
        again = 1;
#pragma unroll 1
        for (int r = 0; r < kCols; ++r) {
          uint32_t o[4];
#pragma unroll
          for (int m = 0; m < 4; ++m) tmem_ld_32x32b_x1(o_addr + kN * m + r, o[m]);
          const float f = ld_shared_f32(add + 4 * r);
          tmem_wait_ld();
          float top = 0.f, unused_factor;
#pragma unroll
          for (int m = 0; m < 4; ++m) top = fmaxf(top, fabsf(__uint_as_float(o[m]) * f));
          // (not below FP32's least with out_scale in it)
          const int e = max(static_cast<int>(partial_scale_byte(warp_max(top), &unused_factor)), 128 - scale_exp);
          if (lane == r) {
            st_shared_b32(add + 4 * r, __float_as_uint(f * __uint_as_float(static_cast<uint32_t>(254 - e) << 23)));
            scale_word(r) = static_cast<uint32_t>(e + scale_exp - 127) * 0x01010101u;
          }
        }
        __syncwarp();
      }
      if (tid == 0) AMLA_STAMP(prm, part, 12, un);
      tc_fence_before_sync();      // O has been read: this warp's next PREADY arrival lets the next unit overwrite it
      ++un;
      units_left = !(note & kLastTile);
    }
    if (!ok && lane == 0) report_timeout(prm.status);
  } else if (wid < kSoftmaxWarps + kWidenWarps) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(C::kWidenRegs));
    // ======================================================== widening: raw pages -> operand chunks in tensor memory
    const int quad = wid & 3;
    const uint32_t raw = smem_base + C::kOffRaw, lanes = tbase + (static_cast<uint32_t>(quad * 32) << 16);
    const uint32_t group = ((wid - C::kKWarp) >> 2) & 1;     // of the two that take turns by chunk
    uint32_t slot = 0, par = 0, tiles = 0, note = 0;
    int left = kWaitTries;
    auto tile_here = [&]() {                                 // false: the wait ran out
      mbar_wait_spend(bar(C::X_FULL) + 8 * slot, par, left);
      note = ld_shared_b32(smem_base + C::kOffNotes + 8 * (tiles % kNotes));
      ok = __all_sync(0xffffffffu, left > 0);
      left = kWaitTries;
      return ok;
    };
    auto tile_done = [&]() {                                 // (what was read of it is in registers)
      __syncwarp();
      mbar_arrive_if(lane == 0, bar(C::X_EMPTY) + 8 * slot);
      if (++slot == C::kSlots) { slot = 0; par ^= 1; }
      ++tiles;
      return !(note & kLastTile);
    };
    auto place = [&](uint32_t empty, uint32_t use) {
      mbar_wait_spend(empty, (use & 1) ^ 1, left);
      __syncwarp();
      tc_fence_after_sync();
    };
    auto hand_over = [&](uint32_t full) {
      tmem_wait_st();
      tc_fence_before_sync();
      __syncwarp();
      mbar_arrive_if(lane == 0, full);
    };
    // ---- Q: a unit's rows into f16, by the warps that widen K and, for a part's first unit, those that widen V too; and what the softmax needs of them: the factor from a product to a
    // logit and the keys that a row sees.  The bytes land where the operand is to be and are converted in place.
    auto load_q = [&](uint32_t un, int each, bool alone) {
      uint32_t b, unit_r0, n_b, unused;
      ld_shared_v4(smem_base + C::kOffUnits + (un % kNotes) * 32, b, unit_r0, n_b, unused);
      const int left = prm.R - static_cast<int>(unit_r0);      // rows of the sequence from here on
      const __nv_bfloat16* rows = prm.q + (static_cast<size_t>(b) * prm.R + unit_r0) * kDqk;
      const uint32_t mult = smem_base + C::kOffMult + (un % kUnitsAhead) * kN * 4, vis = smem_base + C::kOffVis + (un % kUnitsAhead) * kN * 4;
      const int r0 = (wid - C::kKWarp) * each;
      auto piece = [&](int r, int j) { return smem_base + ((lane + 32 * j) >> 3) * C::kQBlock + r * 128 + ((((lane + 32 * j) & 7) ^ (r & 7)) << 4); };
#pragma unroll 1
      for (int i = 0; i < each; ++i) {
        const bool live = r0 + i < left;
        const __nv_bfloat16* src = rows + static_cast<size_t>(live ? r0 + i : 0) * kDqk + 8 * lane;
        cp_async_16(piece(r0 + i, 0), src, live);
        cp_async_16(piece(r0 + i, 1), src + 256, live);
        if (lane < 8) cp_async_16(piece(r0 + i, 2), src + 512, live);
      }
      cp_async_wait_all();
#pragma unroll 1
      for (int r = r0; r < r0 + each; ++r) {              // (a thread converts what it has brought itself)
        uint32_t x[3][4], top = 0;                           // the largest magnitude, of either half of the words, as integers
#pragma unroll
        for (int j = 0; j < 3; ++j) {
          x[j][0] = x[j][1] = x[j][2] = x[j][3] = 0;
          if (j < 2 || lane < 8) ld_shared_v4(piece(r, j), x[j][0], x[j][1], x[j][2], x[j][3]);
          top = __vimax3_u16x2(top, x[j][0] & 0x7fff7fffu, x[j][1] & 0x7fff7fffu);
          top = __vimax3_u16x2(top, x[j][2] & 0x7fff7fffu, x[j][3] & 0x7fff7fffu);
        }
        const uint32_t e = __reduce_max_sync(0xffffffffu, max(top >> 16, top & 0xffffu)) >> 7;
        // 2^(14 - (e - 127)) and its inverse; the largest powers that FP32 has for rows below 2^-113, 1 for rows that are not finite
        const float up = e == 255 ? 1.f : __uint_as_float(e <= 14 ? 254u << 23 : (268u - e) << 23);
        const float down = e == 255 ? 1.f : __uint_as_float(e <= 14 ? 0x00400000u : (e - 14u) << 23);
        const uint64_t up2 = pack_f32x2(up, up);
#pragma unroll
        for (int j = 0; j < 3; ++j) {
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            float lo, hi;
            unpack_f32x2(mul_f32x2(pack_f32x2(__uint_as_float(x[j][c] << 16), __uint_as_float(x[j][c] & 0xffff0000u)), up2), lo, hi);
            x[j][c] = pack_f16x2(lo, hi);
          }
          if (j < 2 || lane < 8) st_shared_v4(piece(r, j), x[j][0], x[j][1], x[j][2], x[j][3]);
        }
        if (lane == 0) {
          st_shared_b32(mult + 4 * r, __float_as_uint(prm.scale_log2 * down));
          st_shared_b32(vis + 4 * r, static_cast<uint32_t>(min(static_cast<int>(n_b), static_cast<int>(n_b) - prm.Sq + (static_cast<int>(unit_r0) + r) / prm.H + 1)));
        }
      }
      fence_proxy_async_smem();
      __syncwarp();
      if (alone) mbar_arrive_2_if(lane == 0, bar(C::X_QREADY + un % kUnitsAhead));
      else mbar_arrive_if(lane == 0, bar(C::X_QREADY + un % kUnitsAhead));
    };
    // the part's first unit, as soon as it is known
    auto any_unit = [&]() {
      ok = warp_wait(bar(C::X_START), 0);
      return ok && static_cast<int>(ld_shared_b32(smem_base + C::kOffUnits + 8)) > 0;
    };
    const bool any = any_unit();
    if (tid == 32 * C::kKWarp) AMLA_STAMP(prm, part, 20, 5);
    if (any) load_q(0, kN / kWidenWarps, false);
    if (tid == 32 * C::kKWarp) AMLA_STAMP(prm, part, 20, 6);
    if (!any) {
    } else if (wid < C::kVWarp) {
      uint32_t un = 1;
      const uint32_t key = 32 * (quad & 1) + lane, page = raw + (quad >> 1) * kPageBytes4;
      const uint32_t code_of = page + key * kCodeRow + 32 * group, scale_of = page + kCodeBytes + key * kScaleRow + 4 * group;
      // ---- K: lane = key of the tile, 64 columns a chunk
      do {
        if (!tile_here()) break;
        if (quad == 0 && lane == 0) AMLA_STAMP(prm, part, 19, tiles);
        if ((note & kFirstTile) && tiles > 0) {
          // the products of the unit before have read its Q
          ok = warp_wait(bar(C::X_SFULL) + 8 * ((tiles - 1) % C::kSBufs), ((tiles - 1) / C::kSBufs) & 1);
          if (!ok) break;
          load_q(un, kN / (kWidenWarps / 2), true);
          ++un;
        }
        uint32_t codes = code_of + slot * kTileBytes, scales = scale_of + slot * kTileBytes;
        const uint32_t there = (note >> (quad < 2 ? 0 : kSecondPage)) & kKeysMask ? 0xffffffffu : 0u;
#pragma unroll 1
        for (uint32_t c = group; c < kColBlocks; c += 2) {
          if (quad == 0 && lane == 0) AMLA_STAMP(prm, part, 0, tiles * 9 + c);
          uint32_t w[8];
          ld_shared_v4(codes, w[0], w[1], w[2], w[3]);
          ld_shared_v4(codes + 16, w[4], w[5], w[6], w[7]);
          const uint32_t sw = ld_shared_b32(scales) & there;
          codes += 64;
          scales += 8;
          const uint32_t buf = c & 3;
#pragma unroll
          for (int h = 0; h < 2; ++h) {                      // (half at a time: registers)
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
            if (h == 0) place(bar(C::X_KEMPTY) + 8 * buf, (buf == 0 ? tiles : 0) + (c >> 2));      // three chunks a tile in place 0, two in the others
            tmem_st_32x32b_x16(lanes + C::kKCol + 32 * buf + 16 * h, r);
          }
          hand_over(bar(C::X_KFULL) + 8 * buf);
        }
      } while (tile_done());
    } else {
      // ---- V: lanes = its columns, 16 keys a chunk.  A thread (g = lane / 4, q = lane % 4) takes columns 128 quad + 16 g .., one group with one scale, of
      // four keys: words of two keys are interleaved by nibbles and converted, which gives pairs of keys.  Column i of the sixteen goes to
      // block i / 4, lane 32 quad + g + 8 (i % 4).  Key k = 4 q + e of the product's 16 is key 4 q + (q + e) % 4, so that the four q read four
      // different residues (a row is 72 words: else all from the same banks).
      // A scale that is a NaN becomes a number here: through K the rows that see the key have a NaN for its P~, and those that do
      // not have a zero, which a NaN in V would turn into one.
      const int g = lane >> 2, q = lane & 3;
      uint32_t code_of[4], scale_of[4];                      // of this group's chunks: keys 16 group .., 16 group + 32 .. of a page
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t key = 16 * group + 4 * q + ((q + e) & 3);
        code_of[e] = raw + key * kCodeRow + 64 * quad + 8 * g;
        scale_of[e] = raw + kCodeBytes + key * kScaleRow + 8 * quad + 4 * (g >> 2);
      }
      const uint32_t pick = (g & 3) | ((4 + (g & 3)) << 4);     // this thread's group, of the four that a scale word holds, of either key
      do {
        if (!tile_here()) break;
        if (quad == 0 && lane == 0) AMLA_STAMP(prm, part, 19, tiles);
        uint32_t codes[4], scales[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) { codes[e] = code_of[e] + slot * kTileBytes; scales[e] = scale_of[e] + slot * kTileBytes; }
#pragma unroll 1
        for (uint32_t h = 0; h < 2; ++h) {                    // page
          const int count = static_cast<int>((note >> (h * kSecondPage)) & kKeysMask) - 16 * static_cast<int>(group);   // keys that count
#pragma unroll
          for (int i = 0; i < 2; ++i) {                       // chunk 4 h + 2 i + group
            if (quad == 0 && lane == 0) AMLA_STAMP(prm, part, 13, tiles * 8 + 4 * h + 2 * i + group);
            uint32_t w[4][2], sw[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              ld_shared_v2(codes[e] + 32 * i * kCodeRow, w[e][0], w[e][1]);
              sw[e] = ld_shared_b32(scales[e] + 32 * i * kScaleRow);
            }
            if (count < 32 * i + 16) {                        // what is beyond the sequence's end may be anything: scales of zero
#pragma unroll
              for (int e = 0; e < 4; ++e) sw[e] = 32 * i + 4 * q + ((q + e) & 3) < count ? sw[e] : 0u;
            }
            uint32_t sc[2];
#pragma unroll
            for (int j = 0; j < 2; ++j) sc[j] = number_f16x2(e4m3x2_to_f16x2(__byte_perm(sw[2 * j], sw[2 * j + 1], pick)));
            const uint32_t buf = C::kVBufs == 4 ? 2 * i + group : group;
#pragma unroll
            for (int x8 = 0; x8 < 2; ++x8) {                  // columns 8 x8 .. (half at a time: registers)
              uint32_t r[2][8];                               // [lanes .. + 16 hh][block, (row g, row g + 8), key pair]
#pragma unroll
              for (int j = 0; j < 2; ++j) {                   // keys e = 2j, 2j + 1
                const uint32_t w0 = w[2 * j][x8], w1 = w[2 * j + 1][x8];
                const uint32_t even = (w0 & 0x0f0f0f0fu) | ((w1 << 4) & 0xf0f0f0f0u), odd = ((w0 >> 4) & 0x0f0f0f0fu) | (w1 & 0xf0f0f0f0u);
                uint32_t x[4], z[4];
                e2m1x8_to_f16x2(even, x);
                e2m1x8_to_f16x2(odd, z);
#pragma unroll
                for (int m = 0; m < 4; ++m) {                 // columns 8 x8 + 2 m (lanes 16 hh + g) and + 1 (.. + 8): block 2 x8 + m / 2, hh = m % 2
                  r[m & 1][4 * (m >> 1) + j] = mul_f16x2(x[m], sc[j]);
                  r[m & 1][4 * (m >> 1) + 2 + j] = mul_f16x2(z[m], sc[j]);
                }
              }
              if (x8 == 0) place(bar(C::X_VEMPTY) + 8 * buf, C::kVBufs == 4 ? h : i);
              tmem_st_16x256b_x2(lanes + C::kVCol + 32 * buf + 16 * x8, r[0]);
              tmem_st_16x256b_x2(lanes + (16u << 16) + C::kVCol + 32 * buf + 16 * x8, r[1]);
            }
            hand_over(bar(C::X_VFULL) + 8 * buf);
          }
#pragma unroll
          for (int e = 0; e < 4; ++e) { codes[e] += kPageBytes4; scales[e] += kPageBytes4; }
        }
      } while (tile_done());
    }
    ok = __all_sync(0xffffffffu, ok && left > 0);
    if (!ok && lane == 0) report_timeout(prm.status);
  } else {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(C::kIssueRegs));
    constexpr uint32_t dhi = smem_desc_hi_sw128(1024);
    // A wait that runs out is noticed at the end of its tile, so that products have been issued behind it: they are waited for, before the tensor memory
    // that they read and write is given back.
    auto give_up = [&](uint32_t drained) {
      report_timeout(prm.status);
      mma_commit(drained);
      mbar_wait_inline(drained, 0);
    };
    if (wid == C::kQkWarp) {
      // ======================================================== S^T = K Q^T
      // (Constants wherever they can be: an accumulate flag out of a register alone costs as much issue as an MMA.)
      if (elect_one()) {
        constexpr uint32_t idesc = make_idesc_f16(128, kN, false, false);
        uint32_t gs = 0, un = 0;
        int left = kWaitTries;
        ok = mbar_wait_inline(bar(C::X_START), 0);
        bool more = ok && static_cast<int>(ld_shared_b32(smem_base + C::kOffUnits + 8)) > 0;
        while (more) {
          const uint32_t sb = gs % C::kSBufs, d = C::kSCol + sb * kN, par = gs & 1;
          mbar_wait_spend(bar(C::X_SEMPTY) + 8 * sb, ((gs / C::kSBufs) & 1) ^ 1, left);
          constexpr uint32_t kQStep = C::kQBlock >> 4;
          const uint32_t ql = smem_desc_lo(smem_base, 16);
          uint32_t note = 0;
#pragma unroll
          for (int c = 0; c < kColBlocks; ++c) {
            constexpr int kB = C::kKBufs;
            mbar_wait_spend(bar(C::X_KFULL + c % kB), (c % kB == 0 ? par : 0) ^ ((c / kB) & 1), left);      // (three chunks a tile in place 0, two in the others)
            if (c == 0) {
              note = ld_shared_b32(smem_base + C::kOffNotes + 8 * (gs % kNotes));
              if (note & kFirstTile) { mbar_wait_spend(bar(C::X_QREADY + un % kUnitsAhead), (un / kUnitsAhead) & 1, left); ++un; }
            }
            tc_fence_after_sync();
            AMLA_STAMP(prm, part, 5, gs * 9 + c);
#pragma unroll
            for (int kk = 0; kk < 4; ++kk)
              mma_ts(d, C::kKCol + 32 * (c % kB) + 8 * kk, smem_desc_join(ql + c * kQStep + 2 * kk, dhi), idesc, c == 0 && kk == 0 ? 0 : 1);
            mma_commit(bar(C::X_KEMPTY + c % kB));
          }
          mma_commit(bar(C::X_SFULL) + 8 * sb);
          ++gs;
          ok = left > 0;
          left = kWaitTries;
          more = ok && !(note & kLastTile);
        }
        if (!ok) give_up(bar(C::X_QKDRAIN));
      }
      __syncwarp();
    } else if (wid == C::kPvWarp) {
      // ======================================================== O^T (+)= V^T P~^T
      if (elect_one()) {
        constexpr uint32_t idesc = make_idesc_f16(128, kN, false, true);
        uint32_t gp = 0;
        int left = kWaitTries;
        ok = mbar_wait_inline(bar(C::X_START), 0);
        bool more = ok && static_cast<int>(ld_shared_b32(smem_base + C::kOffUnits + 8)) > 0;
        while (more) {
          mbar_wait_spend(bar(C::X_PREADY), gp & 1, left);
          const uint32_t pl = smem_desc_lo(smem_base + C::kOffP, 16);
          uint32_t note = 0;
#pragma unroll
          for (int c = 0; c < kVChunks; ++c) {
            constexpr int kB = C::kVBufs;
            mbar_wait_spend(bar(C::X_VFULL + c % kB), (c / kB) & 1, left);
            if (c == 0) note = ld_shared_b32(smem_base + C::kOffNotes + 8 * (gp % kNotes));
            tc_fence_after_sync();                            // (V, and at first P~; O may have been rescaled)
            AMLA_STAMP(prm, part, 17, gp * 8 + c);
            const uint32_t a = C::kVCol + 32 * (c % kB), pc = pl + c * (16 * 128 >> 4);
            if (c == 0 && (note & kFirstTile)) {
#pragma unroll
              for (int m = 0; m < 4; ++m) mma_ts(C::kOCol + kN * m, a + 8 * m, smem_desc_join(pc, dhi), idesc, 0);
            } else {
#pragma unroll
              for (int m = 0; m < 4; ++m) mma_ts(C::kOCol + kN * m, a + 8 * m, smem_desc_join(pc, dhi), idesc, 1);
            }
            mma_commit(bar(C::X_VEMPTY + c % kB));
          }
          mma_commit(bar(C::X_PVDONE));
          ++gp;
          ok = left > 0;
          left = kWaitTries;
          more = ok && !(note & kLastTile);
        }
        if (!ok) give_up(bar(C::X_PVDRAIN));
      }
      __syncwarp();
    } else if (wid == kLoadWarp) {
    // ======================================================== pages in order
    if (elect_one()) {
      Tiles tile(UnitIter(prm, prefix, seqlens, part), first);
      uint32_t slot = 0, par = 1, n_issued = 0, un = 0;
      auto note_unit = [&]() {
        const uint32_t at = smem_base + C::kOffUnits + (un++ % kNotes) * 32;
        st_shared_v4(at, tile.u.b, tile.u.r0, tile.valid ? tile.u.n_b : 0, 0);
        if (!tile.valid) return;
        int2 info;
        const int pslot = tile.units.slot_of(tile.u, &info);
        st_shared_v4(at + 16, pslot, tile.u.it, info.x, info.y);
      };
      note_unit();
      mbar_arrive(bar(C::X_START));
      int page[2] = {0, 0};                                 // the next tile's
      auto look_up = [&]() {
        const int32_t* entry = prm.block_table + static_cast<size_t>(tile.u.b) * prm.max_blocks_per_seq + tile.t;
        page[0] = ldg_here(entry);
        if (tile.np == 2) page[1] = ldg_here(entry + 1);
      };
      if (tile.valid) look_up();
      while (tile.valid) {
        const bool opens = tile.first;
        const int np = tile.np, here[2] = {page[0], page[1]};
        const uint32_t key0 = tile.t * kPage;
        uint32_t note = (opens ? kFirstTile : 0) | (np == 2 ? kTwoPages : 0), bytes = 0;
#pragma unroll
        for (int i = 0; i < 2; ++i)
          if (i < np && here[i] >= 0 && here[i] < prm.num_blocks) {
            note |= static_cast<uint32_t>(min(kPage, tile.u.n_b - (tile.t + i) * kPage)) << (i * kSecondPage);
            bytes += kPageBytes4;
          }
        if (opens && n_issued > 0) {
          note_unit();
          // a unit's Q is asked for by the warps that widen K, when that of the unit before is done with: bring it near
          const size_t row = static_cast<size_t>(tile.u.b) * prm.R + tile.u.r0;
          bulk_prefetch_l2(prm.q + row * kDqk, static_cast<uint32_t>(min(kN, prm.R - tile.u.r0)) * (kDqk * 2));
        }
        tile.next();
        if (tile.valid) look_up();                          // on its way while this tile waits for its slot
        if (!tile.valid) note |= kLastTile;
        if (!tile.valid || tile.first) note |= kEndsUnit;
        ok = mbar_wait_inline(bar(C::X_EMPTY) + 8 * slot, par);
        if (!ok) break;
        const uint32_t full = bar(C::X_FULL) + 8 * slot;
        st_shared_v2(smem_base + C::kOffNotes + 8 * (n_issued % kNotes), note, key0);
        if (bytes != 0) mbar_arrive_expect_tx(full, bytes); else mbar_arrive(full);
#pragma unroll
        for (int i = 0; i < 2; ++i)
          if ((note >> (i * kSecondPage)) & kKeysMask)
            bulk_load(smem_base + C::kOffRaw + slot * kTileBytes + i * kPageBytes4, prm.kv4 + static_cast<size_t>(here[i]) * kPageBytes4, kPageBytes4, full);
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
  if (wid == C::kQkWarp) tmem_dealloc(tbase, 512);
}

// ---------------------------------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------------------------------
int fp4_item_rows(int rows) { return rows <= 16 ? 16 : rows <= 32 ? 32 : 64; }

cudaError_t launch_decode_fp4(const DecodeParams& prm, cudaStream_t stream) {
  static std::atomic<uint64_t> done16{0}, done32{0}, done64{0};
  if (prm.item_rows == 16) return launch_serialized(decode_fp4_kernel<16>, done16, prm.P, Shape<16>::kThreads, Shape<16>::kBytes, stream, prm);
  if (prm.item_rows == 32) return launch_serialized(decode_fp4_kernel<32>, done32, prm.P, Shape<32>::kThreads, Shape<32>::kBytes, stream, prm);
  return launch_serialized(decode_fp4_kernel<64>, done64, prm.P, Shape<64>::kThreads, Shape<64>::kBytes, stream, prm);
}

}  // namespace amla
