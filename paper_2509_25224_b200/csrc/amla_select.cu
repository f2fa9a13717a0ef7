// Which pages of a long context a query token attends to: scores from the pages' means, and the choice.
#include "../../include/amla.h"
#include "amla_host.cuh"
#include "amla_select.cuh"
#include "amla_tokens.cuh"

namespace amla {

namespace {

__host__ __device__ __forceinline__ int logit_stride(int width) { return (width + 31) / 32 * 32; }

__device__ __forceinline__ int seen_by(const int32_t* seqlens, int b, int Sq, int t, int width) {
  const long long n = seqlens[b] < static_cast<long long>(width) * kPage ? seqlens[b] : width * kPage;
  return n - Sq + t + 1 > 0 ? static_cast<int>(n - Sq + t + 1) : 0;
}
// pages in front of the one that holds the token's own position
__device__ __forceinline__ int candidates(int seen) { return seen > 0 ? (seen - 1) / kPage : 0; }

constexpr int kTile = 64, kThreads = 256;

}  // namespace

// logits (base 2) of 64 rows and 64 pages
__global__ void __launch_bounds__(kThreads) page_logits_kernel(const ScoreParams p) {
  __shared__ float qs[16][kTile + 1], ms[16][kTile + 1];
  __shared__ int pages[kTile];
  behind_the_kernel_in_front();
  const int tid = threadIdx.x, R = p.Sq * p.H, tiles = (p.width + kTile - 1) / kTile, row_tiles = (R + kTile - 1) / kTile;
  const int page0 = blockIdx.x % tiles * kTile, row0 = blockIdx.x / tiles % row_tiles * kTile, b = blockIdx.x / tiles / row_tiles;
  if (blockIdx.x == 0 && tid == 0) *p.status = kStatusOk;
  const int most = candidates(seen_by(p.seqlens, b, p.Sq, p.Sq - 1, p.width));
  if (page0 >= most) return;
  if (tid < kTile) pages[tid] = page0 + tid < most ? p.block_table[static_cast<size_t>(b) * p.width + page0 + tid] : -1;
  float acc[4][4] = {};
  const int tx = tid % 16, ty = tid / 16;
  for (int k0 = 0; k0 < kDqk; k0 += 16) {
    __syncthreads();
    for (int i = tid; i < 16 * kTile; i += kThreads) {
      const int k = i % 16, r = i / 16, page = pages[r];
      qs[k][r] = row0 + r < R ? __bfloat162float(p.q[(static_cast<size_t>(b) * R + row0 + r) * kDqk + k0 + k]) : 0.f;
      ms[k][r] = page >= 0 && page < p.num_blocks ? __bfloat162float(p.means[static_cast<size_t>(page) * kDqk + k0 + k]) : 0.f;
    }
    __syncthreads();
    for (int k = 0; k < 16; ++k)
      for (int i = 0; i < 4; ++i)
        for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(qs[k][ty * 4 + i], ms[k][tx + 16 * j], acc[i][j]);
  }
  for (int i = 0; i < 4; ++i)
    for (int j = 0; j < 4; ++j) {
      const int r = row0 + ty * 4 + i, page = page0 + tx + 16 * j;
      if (r < R && page < most) p.logits[(static_cast<size_t>(b) * R + r) * logit_stride(p.width) + page] = acc[i][j] * p.scale_log2;
    }
}

// a block, a query token
__global__ void __launch_bounds__(kThreads) page_mass_kernel(const ScoreParams p) {
  __shared__ float lse[128];
  behind_the_kernel_in_front();
  const int tid = threadIdx.x, wid = tid / 32, lane = tid % 32, b = blockIdx.x / p.Sq, t = blockIdx.x % p.Sq;
  const int count = candidates(seen_by(p.seqlens, b, p.Sq, t, p.width)), stride = logit_stride(p.width);
  const float* logits = p.logits + (static_cast<size_t>(b) * p.Sq + t) * p.H * stride;
  for (int h = wid; h < p.H; h += kThreads / 32) {
    const float* row = logits + static_cast<size_t>(h) * stride;
    float top = -INFINITY, sum = 0.f;
    for (int i = lane; i < count; i += 32) top = fmaxf(top, row[i]);
    for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    for (int i = lane; i < count; i += 32) sum += exp2f(row[i] - top);
    for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (lane == 0) lse[h] = top + log2f(sum);
  }
  __syncthreads();
  float* out = p.scores + static_cast<size_t>(blockIdx.x) * p.width;
  for (int i = tid; i < p.width; i += kThreads) {
    float s = 0.f;
    if (i < count)
      for (int h = 0; h < p.H; ++h) s += exp2f(logits[static_cast<size_t>(h) * stride + i] - lse[h]);
    out[i] = s;
  }
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

size_t score_scratch_bytes(int B, int Sq, int H, int width) { return sizeof(float) * static_cast<size_t>(B) * Sq * H * logit_stride(width); }

cudaError_t launch_page_scores(const ScoreParams& p, cudaStream_t stream) {
  const int R = p.Sq * p.H;
  cudaError_t err = launch_in_order(page_logits_kernel, dim3(p.B * ((p.width + kTile - 1) / kTile) * ((R + kTile - 1) / kTile)), kThreads, stream, p);
  if (err != cudaSuccess) return err;
  return launch_in_order(page_mass_kernel, dim3(p.B * p.Sq), kThreads, stream, p);
}

cudaError_t launch_pages_select(const SelectParams& p, cudaStream_t stream) {
  return launch_in_order(pages_select_kernel, dim3(p.B * p.Sq), kSelectThreads, stream, p);
}

}  // namespace amla
