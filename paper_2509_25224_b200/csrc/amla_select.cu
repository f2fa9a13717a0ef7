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

// A block: 128 rows (query tokens' heads) times 128 pages.  The operands come through a ring of kStages places for 64 of the 576 columns of either.
constexpr int kTileRows = 128, kTilePages = 128, kStatPages = 64, kThreads = 256;
constexpr int kStages = 3, kChunks = kDqk / 64;
constexpr uint32_t kOperandBytes = 128 * 128;                  // [128 rows][128 B], 128-byte swizzle
constexpr uint32_t kOffPages = kStages * 2 * kOperandBytes, kOffBars = kOffPages + kTilePages * 4, kScoreSmem = kOffBars + 64;

// The maximum of a row's logits over 64 pages, and the sum of 2^(logit - maximum)
__host__ __device__ __forceinline__ int stats_of(int width) { return (width + kStatPages - 1) / kStatPages; }
__device__ __forceinline__ float2* stats_at(const ScoreParams& p) { return reinterpret_cast<float2*>(p.logits + static_cast<size_t>(p.B) * p.Sq * p.H * logit_stride(p.width)); }

}  // namespace

// Logits (base 2) of a block's rows and pages, and their statistics by 64 pages.
__global__ void __launch_bounds__(kThreads, 2) page_logits_kernel(const ScoreParams p) {
  extern __shared__ __align__(1024) uint8_t smem[];
  const int tid = threadIdx.x, wid = tid >> 5, lane = tid & 31, R = p.Sq * p.H;
  const int tiles = (p.width + kTilePages - 1) / kTilePages, row_tiles = (R + kTileRows - 1) / kTileRows;
  const int page0 = blockIdx.x % tiles * kTilePages, row0 = blockIdx.x / tiles % row_tiles * kTileRows, b = blockIdx.x / tiles / row_tiles;
  const uint32_t base = smem_u32(smem), bars = base + kOffBars, tmem_slot = bars + 48;
  int* pages = reinterpret_cast<int*>(smem + kOffPages);
  if (tid == 0) {
    for (int i = 0; i < kStages; ++i) mbar_init(bars + 8 * i, 1);
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
  if (wid == 0) { tmem_alloc(tmem_slot, kTilePages); tmem_relinquish(); }
  if (tid < kTilePages) {
    const int page = page0 + tid < most ? p.block_table[static_cast<size_t>(b) * p.width + page0 + tid] : -1;
    pages[tid] = page < p.num_blocks ? page : -1;
  }
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tmem = ld_shared_b32(tmem_slot);

  // a thread brings 16 bytes of every 32nd row of either operand
  const int j = tid & 7, r0 = tid >> 3;
  const __nv_bfloat16* q = p.q + (static_cast<size_t>(b) * R + row0) * kDqk + 8 * j;
  const __nv_bfloat16* rows[4];
  uint32_t live = 0, dst[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = r0 + 32 * i, page = pages[r];
    rows[i] = p.means + static_cast<size_t>(max(page, 0)) * kDqk + 8 * j;
    live |= (page >= 0 ? 1u : 0u) << i;
    live |= (row0 + r < R ? 16u : 0u) << i;
    dst[i] = base + sw128_offset(r, j);
  }
  auto load = [&](int c) {
    const uint32_t at = c % kStages * 2 * kOperandBytes;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const bool mine = live >> (4 + i) & 1;
      cp_async_16(dst[i] + at, mine ? q + (r0 + 32 * i) * kDqk + 64 * c : p.q, mine);
      cp_async_16(dst[i] + at + kOperandBytes, rows[i] + 64 * c, live >> i & 1);
    }
  };
  bool ok = true;
  for (int c = 0; c < kStages - 1; ++c) { load(c); cp_async_commit(); }
#pragma unroll 1
  for (int c = 0; c < kChunks; ++c) {
    cp_async_wait_group<kStages - 2>();
    fence_proxy_async_smem();
    __syncthreads();
    if (wid == 0 && elect_one()) {
      constexpr uint32_t idesc = make_idesc_bf16(kTileRows, kTilePages, false, false), hi = smem_desc_hi_sw128(1024);
      const uint32_t a = smem_desc_lo(base + c % kStages * 2 * kOperandBytes, 16), k = smem_desc_lo(base + c % kStages * 2 * kOperandBytes + kOperandBytes, 16);
#pragma unroll
      for (int kk = 0; kk < 4; ++kk) mma_ss(tmem, smem_desc_join(a + 2 * kk, hi), smem_desc_join(k + 2 * kk, hi), idesc, (c | kk) != 0 ? 1u : 0u);
      mma_commit(bars + 8 * (c % kStages));
    }
    const int next = c + kStages - 1;
    if (next < kChunks) {
      if (c > 0 && ok) ok = mbar_wait(bars + 8 * (next % kStages), ((c - 1) / kStages) & 1);      // the products that read this place
      if (ok) load(next);
    }
    cp_async_commit();                                         // (perhaps an empty group)
  }
  if (ok) ok = mbar_wait(bars + 8 * ((kChunks - 1) % kStages), ((kChunks - 1) / kStages) & 1);
  __syncwarp();
  tc_fence_after_sync();
  if (__all_sync(0xffffffffu, ok)) {
    // a thread has a row and 64 of the pages
    const int quarter = wid & 3, half = wid >> 2, row = row0 + 32 * quarter + lane, first = page0 + kStatPages * half;
    uint32_t v[2][32];
    const uint32_t at = tmem + (static_cast<uint32_t>(32 * quarter) << 16) + kStatPages * half;
    tmem_ld_32x32b_x32(at, v[0]);
    tmem_ld_32x32b_x32(at + 32, v[1]);
    tmem_wait_ld();
    if (row < R && first < most) {
      const int count = candidates(seen_by(p.seqlens, b, p.Sq, row / p.H, p.width)) - first;
      float* out = p.logits + (static_cast<size_t>(b) * R + row) * logit_stride(p.width) + first;
      float top = -INFINITY;
#pragma unroll
      for (int i = 0; i < 64; ++i) {
        const float l = __uint_as_float(v[i >> 5][i & 31]) * p.scale_log2;
        v[i >> 5][i & 31] = __float_as_uint(l);
        top = max_nan(top, i < count ? l : -INFINITY);
      }
      float sum = 0.f;
      const float off = top == -INFINITY ? 0.f : top;
#pragma unroll
      for (int i = 0; i < 64; ++i) sum += i < count ? ex2_approx(__uint_as_float(v[i >> 5][i & 31]) - off) : 0.f;
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (4 * i < count) stg_128(out + 4 * i, v[i >> 3][4 * i & 31], v[i >> 3][(4 * i & 31) + 1], v[i >> 3][(4 * i & 31) + 2], v[i >> 3][(4 * i & 31) + 3]);
      stats_at(p)[(static_cast<size_t>(b) * R + row) * stats_of(p.width) + first / kStatPages] = make_float2(top, sum);
    }
  } else if (lane == 0) {
    atomicExch(p.status, kStatusTimeout);
  }
  cp_async_wait_all();
  tc_fence_before_sync();
  __syncthreads();
  if (wid == 0) tmem_dealloc(tmem, kTilePages);
}

namespace {
constexpr int kMassPages = 128, kMassThreads = 256;
}  // namespace

// A block: 128 pages of a query token, half of the heads by either half of the threads.
__global__ void __launch_bounds__(kMassThreads) page_mass_kernel(const ScoreParams p) {
  __shared__ float lse[128], part[kMassPages];
  behind_the_kernel_in_front();
  const int tid = threadIdx.x, wid = tid / 32, lane = tid % 32, chunks = (p.width + kMassPages - 1) / kMassPages;
  const int token = blockIdx.x / chunks, first = blockIdx.x % chunks * kMassPages, b = token / p.Sq, t = token % p.Sq;
  const int count = candidates(seen_by(p.seqlens, b, p.Sq, t, p.width)), stride = logit_stride(p.width), stats = stats_of(count);
  float* out = p.scores + static_cast<size_t>(token) * p.width;
  if (first >= count) {
    if (tid < kMassPages && first + tid < p.width) out[first + tid] = 0.f;
    return;
  }
  for (int h = wid; h < p.H; h += kMassThreads / 32) {
    const float2* row = stats_at(p) + (static_cast<size_t>(token) * p.H + h) * stats_of(p.width);
    float top = -INFINITY, sum = 0.f;
    for (int i = lane; i < stats; i += 32) {
      const float2 s = row[i];
      const float m = max_nan(top, s.x);
      sum = m == -INFINITY ? 0.f : sum * ex2_approx(top - m) + s.y * ex2_approx(s.x - m);
      top = m;
    }
    float all = top;
#pragma unroll
    for (int o = 16; o; o >>= 1) all = max_nan(all, __shfl_xor_sync(0xffffffffu, all, o));
    sum = top == -INFINITY ? 0.f : sum * ex2_approx(top - all);
#pragma unroll
    for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (lane == 0) lse[h] = all + log2f(sum);
  }
  __syncthreads();
  const int at = tid % kMassPages, side = tid / kMassPages, page = first + at;
  float s = 0.f;
  if (page < count) {
    const float* l = p.logits + static_cast<size_t>(token) * p.H * stride + page;
#pragma unroll 8
    for (int h = side; h < p.H; h += 2) s += ex2_approx(l[static_cast<size_t>(h) * stride] - lse[h]);
  }
  if (side == 1) part[at] = s;
  __syncthreads();
  if (side == 0 && page < p.width) out[page] = s + part[at];
}

namespace {

constexpr int kSelectThreads = 512;

// A number's place in the order of scores: larger for larger ones, the same for both zeros, that of -infinity for a NaN.
__device__ __forceinline__ uint32_t order_of(float f) {
  if (f != f) return 0x007fffffu;
  const uint32_t u = __float_as_uint(f + 0.f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// Sum over the block in front of this thread; *all = over all of it.
__device__ __forceinline__ int2 scan2(int2 v, int2* all) {
  __shared__ int2 warps[kSelectThreads / 32];
  const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
  int2 upto = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int x = __shfl_up_sync(0xffffffffu, upto.x, o), y = __shfl_up_sync(0xffffffffu, upto.y, o);
    if (lane >= o) { upto.x += x; upto.y += y; }
  }
  if (lane == 31) warps[wid] = upto;
  __syncthreads();
  int2 front = make_int2(0, 0), sum = make_int2(0, 0);
  for (int i = 0; i < kSelectThreads / 32; ++i) {
    const int2 w = warps[i];
    if (i < wid) { front.x += w.x; front.y += w.y; }
    sum.x += w.x; sum.y += w.y;
  }
  *all = sum;
  return make_int2(front.x + upto.x - v.x, front.y + upto.y - v.y);
}

}  // namespace

// A block, a query token.  The scores' order is looked at eight bits at a time, from the top: how many of those that agree with the bits found
// so far have which next eight; the place that is looked for lies in one of these 256.
__global__ void __launch_bounds__(kSelectThreads) pages_select_kernel(const SelectParams p) {
  __shared__ int hist[256];
  __shared__ uint32_t found_digit;
  __shared__ int found_left;
  behind_the_kernel_in_front();
  const int tid = threadIdx.x, row = blockIdx.x, b = row / p.Sq, t = row % p.Sq;
  const int seen = seen_by(p.seqlens, b, p.Sq, t, p.width), count = (seen + kPage - 1) / kPage;
  const int32_t* entries = p.block_table + static_cast<size_t>(b) * p.width;
  int32_t* table = p.table + static_cast<size_t>(row) * p.keep;
  int32_t* chosen = p.chosen ? p.chosen + static_cast<size_t>(row) * p.keep : nullptr;
  const int held = min(count, p.keep);
  for (int i = held + tid; i < p.keep; i += kSelectThreads) {
    table[i] = -1;
    if (chosen) chosen[i] = -1;
  }
  if (p.clear && row == 0 && tid == 0) *p.clear = kStatusOk;
  if (tid == 0) p.lens[row] = seen - (count - held) * kPage;
  if (count <= p.keep) {
    for (int i = tid; i < count; i += kSelectThreads) {
      table[i] = entries[i];
      if (chosen) chosen[i] = i;
    }
    return;
  }
  const float* scores = p.scores + static_cast<size_t>(row) * p.width;
  const int first = p.sink, end = count - p.recent;           // the others; more than are wanted
  int left = p.keep - p.sink - p.recent;                      // wanted of them
  uint32_t prefix = 0;
  if (left > 0) {
    for (int shift = 24; shift >= 0; shift -= 8) {
      for (int i = tid; i < 256; i += kSelectThreads) hist[i] = 0;
      __syncthreads();
      for (int i = first + tid; i < end; i += kSelectThreads) {
        const uint32_t k = order_of(scores[i]);
        if (shift == 24 || (k >> (shift + 8)) == (prefix >> (shift + 8))) atomicAdd(&hist[(k >> shift) & 255], 1);
      }
      __syncthreads();
      if (tid < 32) {
        int mine[8], sum = 0;                                 // lane 0 has the largest eight
        for (int i = 0; i < 8; ++i) { mine[i] = hist[255 - 8 * tid - i]; sum += mine[i]; }
        int upto = sum;
        for (int o = 1; o < 32; o <<= 1) { const int x = __shfl_up_sync(0xffffffffu, upto, o); if (tid >= o) upto += x; }
        int above = upto - sum;
        for (int i = 0; i < 8; ++i) {
          if (above < left && left <= above + mine[i]) { found_digit = 255 - 8 * tid - i; found_left = left - above; }
          above += mine[i];
        }
      }
      __syncthreads();
      prefix |= found_digit << shift;
      left = found_left;                                      // of those that are equal in all bits so far
    }
  } else {
    prefix = 0xffffffffu;                                     // (no score is)
  }
  // larger ones, and the first `left` that are equal: a thread has neighbouring pages
  const int each = (count + kSelectThreads - 1) / kSelectThreads, lo = min(tid * each, count), hi = min(lo + each, count);
  auto kind = [&](int i) {                                    // 2: taken, 1: equal, 0: not
    if (i < first || i >= end) return 2;
    const uint32_t k = order_of(scores[i]);
    return k > prefix ? 2 : k == prefix ? 1 : 0;
  };
  int2 n = make_int2(0, 0), all;
  for (int i = lo; i < hi; ++i) { const int k = kind(i); n.x += k == 2; n.y += k == 1; }
  const int2 front = scan2(n, &all);
  int taken = front.x, equal = front.y;
  for (int i = lo; i < hi; ++i) {
    const int k = kind(i);
    if (k == 2 || (k == 1 && equal < left)) {
      const int to = taken + min(equal, left);
      table[to] = entries[i];
      if (chosen) chosen[to] = i;
    }
    taken += k == 2;
    equal += k == 1;
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
  return launch_in_order(page_mass_kernel, dim3(p.B * p.Sq * ((p.width + kMassPages - 1) / kMassPages)), kMassThreads, stream, p);
}

cudaError_t launch_pages_select(const SelectParams& p, cudaStream_t stream) {
  return launch_in_order(pages_select_kernel, dim3(p.B * p.Sq), kSelectThreads, stream, p);
}

}  // namespace amla
