// Which pages of a long context a query token attends to: scores from the pages' means, and the choice.
#include "../../include/amla.h"
#include "amla_fp4.cuh"
#include "amla_host.cuh"
#include "amla_select.cuh"
#include "amla_sm100.cuh"
#include "amla_tokens.cuh"

namespace amla {

using namespace sm100;

namespace {

__host__ __device__ __forceinline__ int logit_stride(int width) { return (width + 31) / 32 * 32; }

__device__ __forceinline__ int seen_by(const int32_t* seqlens, int b, int Sq, int t, int width) {
  const long long n = seqlens[b] < static_cast<long long>(width) * kPage ? seqlens[b] : width * kPage;
  return n - Sq + t + 1 > 0 ? static_cast<int>(n - Sq + t + 1) : 0;
}
// pages in front of the one that holds the token's own position
__device__ __forceinline__ int candidates(int seen) { return seen > 0 ? (seen - 1) / kPage : 0; }

// A block of the products: 128 rows (query tokens' heads) times up to 256 pages.  The operands come through a ring of places for 64 of the 576 columns
// of either, by the same warps that then make numbers of the products; one more warp issues those.
constexpr int kTileRows = 128, kTilePages = 256, kLoadWarps = 8, kLoadThreads = 32 * kLoadWarps, kThreads = kLoadThreads + 32;
constexpr int kStages = 4, kChunks = kDqk / 64;
constexpr uint32_t kQBytes = kTileRows * 128, kPlaceBytes = kQBytes + kTilePages * 128;       // rows of 128 B, 128-byte swizzle
constexpr uint32_t kOffPages = kStages * kPlaceBytes, kOffBars = kOffPages + kTilePages * 4, kScoreSmem = kOffBars + 128;
enum { X_FULL = 0, X_EMPTY = kStages, X_DONE = 2 * kStages, X_NUM };
static_assert(8 * X_NUM + 8 <= 128, "barrier area too small");

// What is known of a row's logits over kStatPages pages: their maximum, and the sum of 2^(logit - maximum).
constexpr int kStatPages = 128;
__host__ __device__ __forceinline__ int stats_of(int pages) { return (pages + kStatPages - 1) / kStatPages; }
__device__ __forceinline__ float2* stats_at(const ScoreParams& p, int b, int stat) {
  const size_t rows = static_cast<size_t>(p.Sq) * p.H;
  return reinterpret_cast<float2*>(p.logits + p.B * rows * logit_stride(p.width)) + (static_cast<size_t>(b) * stats_of(p.width) + stat) * rows;
}

}  // namespace

// Logits (base 2) of a block's rows and pages, and their statistics.
__global__ void __launch_bounds__(kThreads, 1) page_logits_kernel(const ScoreParams p) {
  extern __shared__ __align__(1024) uint8_t smem[];
  const int tid = threadIdx.x, wid = tid >> 5, lane = tid & 31, R = p.Sq * p.H;
  const int tiles = (p.width + kTilePages - 1) / kTilePages, row_tiles = (R + kTileRows - 1) / kTileRows;
  const int page0 = blockIdx.x % tiles * kTilePages, row0 = blockIdx.x / tiles % row_tiles * kTileRows, b = blockIdx.x / tiles / row_tiles;
  const uint32_t base = smem_u32(smem), bars = base + kOffBars, tmem_slot = bars + 128 - 8;
  auto bar = [&](int i) { return bars + 8u * i; };
  int* pages = reinterpret_cast<int*>(smem + kOffPages);
  if (tid == 0) {
    for (int i = 0; i < kStages; ++i) { mbar_init(bar(X_FULL + i), kLoadThreads); mbar_init(bar(X_EMPTY + i), 1); }
    mbar_init(bar(X_DONE), 1);
    fence_mbar_init();
  }
  behind_the_kernel_in_front();
  if (blockIdx.x == 0 && tid == 0) *p.status = kStatusOk;
  const int most = candidates(seen_by(p.seqlens, b, p.Sq, p.Sq - 1, p.width));
  if (page0 >= most) return;
  if (base & 1023u) {                                          // the swizzled tiles assume a 1024-byte aligned window
    if (tid == 0) atomicExch(p.status, kStatusTimeout);
    return;
  }
  const int here = min(most - page0, kTilePages), n = (here + 15) / 16 * 16;      // pages, as products take them
  if (wid == kLoadWarps) { tmem_alloc(tmem_slot, kTilePages); tmem_relinquish(); }
  if (tid < kTilePages) {
    const int page = tid < here ? p.block_table[static_cast<size_t>(b) * p.width + page0 + tid] : -1;
    pages[tid] = page < p.num_blocks ? page : -1;
  }
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tmem = ld_shared_b32(tmem_slot);
  bool ok = true;

  if (wid == kLoadWarps) {
    if (elect_one()) {
      const uint32_t idesc = make_idesc_bf16(kTileRows, 16, false, false) + (static_cast<uint32_t>(n / 8 - 2) << 17);
      constexpr uint32_t hi = smem_desc_hi_sw128(1024);
#pragma unroll 1
      for (int c = 0; c < kChunks && ok; ++c) {
        const uint32_t place = c % kStages;
        ok = mbar_wait(bar(X_FULL + place), (c / kStages) & 1);
        if (!ok) break;
        fence_proxy_async_smem();                              // the copies are ordinary writes
        const uint32_t a = smem_desc_lo(base + place * kPlaceBytes, 16), k = smem_desc_lo(base + place * kPlaceBytes + kQBytes, 16);
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) mma_ss(tmem, smem_desc_join(a + 2 * kk, hi), smem_desc_join(k + 2 * kk, hi), idesc, (c | kk) != 0 ? 1u : 0u);
        mma_commit(bar(X_EMPTY + place));
      }
      mma_commit(bar(X_DONE));
      if (!ok) { atomicExch(p.status, kStatusTimeout); mbar_wait(bar(X_DONE), 0); }
    }
    __syncwarp();
  } else {
    // a thread brings 16 bytes of every 32nd row of either operand (rows that there are not: whatever is there, in rows of the result that nobody reads)
    const int j = tid & 7, r0 = tid >> 3;
    const __nv_bfloat16* q = p.q + (static_cast<size_t>(b) * R + row0 + r0) * kDqk + 8 * j;
    const int q_rows = min(R - row0, kTileRows) - r0;
    int mine[kTilePages / 32];                                 // -1: outside the cache
#pragma unroll
    for (int i = 0; i < kTilePages / 32; ++i) mine[i] = pages[r0 + 32 * i];
    const uint32_t dst = base + sw128_offset(r0, j);           // (32 rows further on the swizzle is the same)
#pragma unroll 1
    for (int c = 0; c < kChunks; ++c) {
      const uint32_t place = c % kStages, to = dst + place * kPlaceBytes;
      if (c >= kStages) {
        ok = mbar_wait(bar(X_EMPTY + place), (c / kStages - 1) & 1);
        if (!ok) break;
      }
#pragma unroll
      for (int i = 0; i < kTileRows / 32; ++i)
        if (32 * i < q_rows) cp_async_16(to + 4096 * i, q + 32 * i * kDqk + 64 * c, true);
#pragma unroll
      for (int i = 0; i < kTilePages / 32; ++i)
        if (r0 + 32 * i < n) cp_async_16(to + kQBytes + 4096 * i, p.means + static_cast<size_t>(max(mine[i], 0)) * kDqk + 8 * j + 64 * c, mine[i] >= 0);
      cp_async_arrive(bar(X_FULL + place));
    }
    ok = ok && mbar_wait(bar(X_DONE), 0);
    ok = __all_sync(0xffffffffu, ok);
    tc_fence_after_sync();
    // a thread has a row and 128 of the pages, 64 at a time
    const int quarter = wid & 3, half = wid >> 2, row = row0 + 32 * quarter + lane, first = kStatPages * half;
    if (ok && first < here) {
      const int token = min(row, R - 1) / p.H, count = row < R ? candidates(seen_by(p.seqlens, b, p.Sq, token, p.width)) - page0 - first : 0;
      float* out = p.logits + (static_cast<size_t>(b) * R + row) * logit_stride(p.width) + page0 + first;
      float top = -INFINITY, sum = 0.f;
#pragma unroll 1
      for (int part = 0; part < kStatPages; part += 64) {
        if (first + part >= here) break;
        uint32_t v[2][32];
        const uint32_t at = tmem + (static_cast<uint32_t>(32 * quarter) << 16) + first + part;
        tmem_ld_32x32b_x32(at, v[0]);
        tmem_ld_32x32b_x32(at + 32, v[1]);
        tmem_wait_ld();
        const int left = count - part;
        float most_here = top;
#pragma unroll
        for (int i = 0; i < 64; ++i) {
          const float l = __uint_as_float(v[i >> 5][i & 31]) * p.scale_log2;
          v[i >> 5][i & 31] = __float_as_uint(l);
          most_here = max_nan(most_here, i < left ? l : -INFINITY);
        }
        const float off = most_here == -INFINITY ? 0.f : most_here;
        sum *= ex2_approx(top - off);
        top = most_here;
#pragma unroll
        for (int i = 0; i < 64; ++i) sum += i < left ? ex2_approx(__uint_as_float(v[i >> 5][i & 31]) - off) : 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (4 * i < left) stg_128(out + part + 4 * i, v[i >> 3][4 * i & 31], v[i >> 3][(4 * i & 31) + 1], v[i >> 3][(4 * i & 31) + 2], v[i >> 3][(4 * i & 31) + 3]);
      }
      if (row < R) stats_at(p, b, (page0 + first) / kStatPages)[row] = make_float2(top, sum);
    }
    if (!ok && lane == 0) atomicExch(p.status, kStatusTimeout);
    cp_async_wait_all();
  }
  tc_fence_before_sync();
  __syncthreads();
  if (wid == kLoadWarps) tmem_dealloc(tmem, kTilePages);
}

namespace {

constexpr int kMassPages = 128, kMassWarps = 16, kMassThreads = 32 * kMassWarps, kMostHeads = 128;
constexpr int kMassHeads = kMostHeads / kMassWarps;           // of a warp

// (top, sum) of two sets of logits together
__device__ __forceinline__ float2 join(float2 a, float2 b) {
  const float top = max_nan(a.x, b.x), off = top == -INFINITY ? 0.f : top;
  return make_float2(top, a.y * ex2_approx(a.x - off) + b.y * ex2_approx(b.x - off));
}

}  // namespace

// A block: 128 pages of a query token.  A warp brings all of them for every 16th head, four neighbouring pages a lane.
__global__ void __launch_bounds__(kMassThreads) page_mass_kernel(const ScoreParams p) {
  __shared__ float2 known[kMassThreads / kMostHeads][kMostHeads];
  __shared__ float lse[kMostHeads];
  __shared__ float4 sums[kMassWarps][32];
  behind_the_kernel_in_front();
  const int tid = threadIdx.x, wid = tid / 32, lane = tid % 32, chunks = (p.width + kMassPages - 1) / kMassPages;
  const int token = blockIdx.x / chunks, first = blockIdx.x % chunks * kMassPages, b = token / p.Sq, t = token % p.Sq;
  const int count = candidates(seen_by(p.seqlens, b, p.Sq, t, p.width)), stride = logit_stride(p.width), stats = stats_of(count);
  float* out = p.scores + static_cast<size_t>(token) * p.width;
  if (first >= count) {
    if (tid < kMassPages && first + tid < p.width) out[first + tid] = 0.f;
    return;
  }
  float4 l[kMassHeads];
  const int page = first + 4 * lane;
#pragma unroll
  for (int i = 0; i < kMassHeads; ++i) {
    const int h = wid + kMassWarps * i;
    if (h < p.H && page < count) l[i] = *reinterpret_cast<const float4*>(p.logits + (static_cast<size_t>(token) * p.H + h) * stride + page);
  }
  {
    const int h = tid % kMostHeads, side = tid / kMostHeads;
    float2 all = make_float2(-INFINITY, 0.f);
    if (h < p.H) {
#pragma unroll 4
      for (int i = side; i < stats; i += kMassThreads / kMostHeads) all = join(all, stats_at(p, b, i)[t * p.H + h]);
    }
    known[side][h] = all;
  }
  __syncthreads();
  if (tid < p.H) {
    const float2 all = join(join(known[0][tid], known[1][tid]), join(known[2][tid], known[3][tid]));
    lse[tid] = all.x + log2f(all.y);
  }
  __syncthreads();
  float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
  for (int i = 0; i < kMassHeads; ++i) {
    const int h = wid + kMassWarps * i;
    if (h < p.H && page < count) {
      const float z = lse[h];
      s.x += ex2_approx(l[i].x - z); s.y += ex2_approx(l[i].y - z); s.z += ex2_approx(l[i].z - z); s.w += ex2_approx(l[i].w - z);
    }
  }
  sums[wid][lane] = s;
  __syncthreads();
  if (tid < kMassPages && first + tid < p.width) {
    float all = 0.f;
#pragma unroll
    for (int w = 0; w < kMassWarps; ++w) all += reinterpret_cast<const float*>(sums[w])[tid];
    out[first + tid] = first + tid < count ? all : 0.f;
  }
}

namespace {

constexpr int kSelectThreads = 1024, kSelectWarps = kSelectThreads / 32;
constexpr int kHeldKeys = 32768;                               // scores whose order is kept in shared memory; of longer rows it is worked out again each time

// A number's place in the order of scores: larger for larger ones, the same for both zeros, that of -infinity for a NaN.
__device__ __forceinline__ uint32_t order_of(float f) {
  if (f != f) return 0x007fffffu;
  const uint32_t u = __float_as_uint(f + 0.f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

}  // namespace

// A block, a query token.  The scores' order is looked at eight bits at a time, from the top: how many of those that agree with the bits found
// so far have which next eight; the one that is looked for lies in one of these 256, and if all of those are wanted the bits suffice.
template <bool kHeld>
__global__ void __launch_bounds__(kSelectThreads) pages_select_kernel(const SelectParams p) {
  extern __shared__ uint32_t held_keys[];
  __shared__ int hist[256];
  __shared__ int found[3];                                     // next eight bits, wanted among those, how many there are
  __shared__ int2 totals[kSelectWarps];
  behind_the_kernel_in_front();
  const int tid = threadIdx.x, wid = tid >> 5, lane = tid & 31, row = blockIdx.x, b = row / p.Sq, t = row % p.Sq;
  const int seen = seen_by(p.seqlens, b, p.Sq, t, p.width), count = (seen + kPage - 1) / kPage;
  const int32_t* entries = p.block_table + static_cast<size_t>(b) * p.width;
  int32_t* table = p.table + static_cast<size_t>(row) * p.keep;
  int32_t* chosen = p.chosen ? p.chosen + static_cast<size_t>(row) * p.keep : nullptr;
  const int kept = min(count, p.keep);
  for (int i = kept + tid; i < p.keep; i += kSelectThreads) {
    table[i] = -1;
    if (chosen) chosen[i] = -1;
  }
  if (p.clear && row == 0 && tid == 0) *p.clear = kStatusOk;
  if (tid == 0) p.lens[row] = seen - (count - kept) * kPage;
  if (count <= p.keep) {
    for (int i = tid; i < count; i += kSelectThreads) {
      table[i] = entries[i];
      if (chosen) chosen[i] = i;
    }
    return;
  }
  const float* scores = p.scores + static_cast<size_t>(row) * p.width;
  const int first = p.sink, end = count - p.recent;            // the others; more than are wanted
  auto key = [&](int i) { return kHeld ? held_keys[i - first] : order_of(scores[i]); };
  if (kHeld) {
    for (int i = first + tid; i < end; i += kSelectThreads) held_keys[i - first] = order_of(scores[i]);
  }
  int left = p.keep - p.sink - p.recent, shift = 32;           // wanted of those that agree in the bits from `shift` on
  uint32_t prefix = 0;
  if (left > 0) {
    do {
      shift -= 8;
      if (tid < 256) hist[tid] = 0;
      __syncthreads();
      for (int i = first + tid; i < end; i += kSelectThreads) {
        const uint32_t k = key(i);
        if (shift == 24 || (k ^ prefix) >> (shift + 8) == 0) atomicAdd(&hist[(k >> shift) & 255], 1);
      }
      __syncthreads();
      if (wid == 0) {                                          // lane 0 has the largest eight
        int mine[8], sum = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) { mine[i] = hist[255 - 8 * lane - i]; sum += mine[i]; }
        int above = sum;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) { const int x = __shfl_up_sync(0xffffffffu, above, o); if (lane >= o) above += x; }
        above -= sum;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          if (above < left && left <= above + mine[i]) { found[0] = 255 - 8 * lane - i; found[1] = left - above; found[2] = mine[i]; }
          above += mine[i];
        }
      }
      __syncthreads();
      prefix |= static_cast<uint32_t>(found[0]) << shift;
      left = found[1];
    } while (shift > 0 && left < found[2]);
  } else {
    __syncthreads();
    shift = 0;
    prefix = 0xffffffffu;                                      // (no score is)
  }
  prefix >>= shift;
  // those above, and the first `left` of those that agree: a warp goes through neighbouring pages, 32 at a time
  const int each = (count + kSelectThreads - 1) / kSelectThreads * 32, lo = min(wid * each, count), hi = min(lo + each, count);
  auto kinds = [&](int i, uint32_t* equal) {                   // which of a warp's 32 are taken anyway, and which agree
    bool take = false, same = false;
    if (i < hi) {
      if (i < first || i >= end) {
        take = true;
      } else {
        const uint32_t k = key(i) >> shift;
        take = k > prefix;
        same = k == prefix;
      }
    }
    *equal = __ballot_sync(0xffffffffu, same);
    return __ballot_sync(0xffffffffu, take);
  };
  int2 n = make_int2(0, 0);
  for (int i = lo; i < hi; i += 32) {
    uint32_t equal;
    n.x += __popc(kinds(i + lane, &equal));
    n.y += __popc(equal);
  }
  if (lane == 0) totals[wid] = n;
  __syncthreads();
  n = lane < wid ? totals[lane] : make_int2(0, 0);             // in front of this warp's
#pragma unroll
  for (int o = 16; o; o >>= 1) { n.x += __shfl_xor_sync(0xffffffffu, n.x, o); n.y += __shfl_xor_sync(0xffffffffu, n.y, o); }
  for (int i = lo; i < hi; i += 32) {
    uint32_t equal;
    const uint32_t take = kinds(i + lane, &equal), below = (1u << lane) - 1;
    const int same = n.y + __popc(equal & below), to = n.x + __popc(take & below) + min(same, left);
    if ((take >> lane & 1) || ((equal >> lane & 1) && same < left)) {
      table[to] = entries[i + lane];
      if (chosen) chosen[to] = i + lane;
    }
    n.x += __popc(take);
    n.y += __popc(equal);
  }
}

size_t score_scratch_bytes(int B, int Sq, int H, int width) {
  return static_cast<size_t>(B) * Sq * H * (sizeof(float) * logit_stride(width) + sizeof(float2) * stats_of(width));
}

cudaError_t launch_page_scores(const ScoreParams& p, cudaStream_t stream) {
  static std::atomic<uint64_t> done{0};
  const int R = p.Sq * p.H;
  const cudaError_t err = launch_serialized(page_logits_kernel, done, p.B * ((p.width + kTilePages - 1) / kTilePages) * ((R + kTileRows - 1) / kTileRows), kThreads, kScoreSmem, stream, p);
  if (err != cudaSuccess) return err;
  return launch_in_order(page_mass_kernel, dim3(p.B * p.Sq * ((p.width + kMassPages - 1) / kMassPages)), kMassThreads, 0, stream, p);
}

cudaError_t launch_pages_select(const SelectParams& p, cudaStream_t stream) {
  static std::atomic<uint64_t> done{0};
  const dim3 grid(p.B * p.Sq);
  if (p.width > kHeldKeys) return launch_in_order(pages_select_kernel<false>, grid, kSelectThreads, 0, stream, p);
  const cudaError_t err = allow_shared(pages_select_kernel<true>, done, kHeldKeys * sizeof(uint32_t));
  if (err != cudaSuccess) return err;
  return launch_in_order(pages_select_kernel<true>, grid, kSelectThreads, p.width <= p.keep ? 0 : p.width * static_cast<uint32_t>(sizeof(uint32_t)), stream, p);
}

}  // namespace amla
