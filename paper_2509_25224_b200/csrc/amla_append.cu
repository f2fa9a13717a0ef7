// New tokens into a paged cache of any format, with what a model does to them directly in front of it, and the summaries of the pages
// that they fill.
//
// append: of a token's 576 columns the first 512 (the latent) are normed, c' = c * rsqrt(mean(c^2) + eps) * w, the other 64 rotated by
// the angles of its position, (x, y) -> (x cos - y sin, y cos + x sin) for 32 pairs; the result is rounded once, to what the cache holds:
// bf16, E4M3 times one factor, or E2M1 numbers against an E4M3 scale for 16 columns (amla_fp4.cuh).  The queries' 64 columns are rotated
// by the same angles into their places behind the 512 that the absorbed projection writes.
// The squares (exact: a bf16 squared has 16 bits) are added up in FP64, in a fixed order, the factor and the products are FP32; products and sums of the
// rotation are rounded one by one.
//
// A launch and a chain of reads (which sequence, its page, the angles) are what a step's tokens cost: 96 tokens of 128 heads 3.2 us, in which 3.4 MB move; with one
// block for a token, which looked for its place first, 5.7.  4 x 2048 tokens of 16 heads take 14.4 us (47 MB, 3.3 TB/s; without queries 5.9): queries are pieces of 128 bytes that lie 384
// and 1152 bytes apart, and 56 to 68 registers a thread leave room for a good half of the 8192 warps at a time.  Heads a warp, 4 / 8 / 16 / 32: 17.3 / 14.4 / 14.3 / 15.9, and for 1024
// tokens of 128 heads 13.6 / 11.0 / 9.6 / 11.4.
//
// means: the mean of a page's 64 keys, as attention sees them, summed in FP32 in a fixed order and rounded to bf16, which is what the
// products with the queries take.  3.6 us for a step (one page in 64 is filled), 5.5 for 148 pages: the tokens' places, then a page's bytes.
#include <cuda_bf16.h>

#include "../../include/amla.h"
#include "amla_fp4.cuh"
#include "amla_host.cuh"
#include "amla_sm100.cuh"
#include "amla_tokens.cuh"

namespace amla {

namespace {

constexpr int kRope = kDqk - kDv;                    // 64
constexpr int kPairs = kRope / 2;
constexpr int kWarps = 4;
constexpr int kThreads = 32 * kWarps;

struct AppendParams {
  const __nv_bfloat16* kv;       // [n, 576], rows row_stride apart
  long long row_stride;
  Tokens tokens;
  void* cache;
  float kv_scale, inv_scale;
  const float* cos_sin;          // [n_positions, 64]: cosines, then sines, of the 32 angles
  int n_positions;
  const int32_t* positions;      // [n], or null: a token's place in its sequence
  const void* weight;            // [512] or null
  int weight_f32;
  float eps;
  const __nv_bfloat16* q_pe;     // [n, H, 64]
  long long q_pe_token, q_pe_head;
  __nv_bfloat16* q;              // [n, H, 576]
  long long q_token, q_head;
  int H;                         // 0: no queries
};

template <bool kWide>
__device__ __forceinline__ uint4 load8(const __nv_bfloat16* p) {
  if (kWide) return *reinterpret_cast<const uint4*>(p);
  uint32_t w[4];
  const unsigned short* h = reinterpret_cast<const unsigned short*>(p);
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = h[2 * i] | (static_cast<uint32_t>(h[2 * i + 1]) << 16);
  return make_uint4(w[0], w[1], w[2], w[3]);
}
template <bool kWide>
__device__ __forceinline__ void store8(__nv_bfloat16* p, uint4 v) {
  if (kWide) {
    *reinterpret_cast<uint4*>(p) = v;
  } else {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    unsigned short* h = reinterpret_cast<unsigned short*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) { h[2 * i] = static_cast<unsigned short>(w[i]); h[2 * i + 1] = static_cast<unsigned short>(w[i] >> 16); }
  }
}
__device__ __forceinline__ float low(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float high(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
__device__ __forceinline__ void unpack8(uint4 v, float (&x)[8]) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) { x[2 * i] = low(w[i]); x[2 * i + 1] = high(w[i]); }
}

// (rounded one by one: a contraction into one operation would depend on the compiler)
__device__ __forceinline__ float turn_first(float a, float b, float c, float s) { return __fsub_rn(__fmul_rn(a, c), __fmul_rn(b, s)); }
__device__ __forceinline__ float turn_second(float a, float b, float c, float s) { return __fadd_rn(__fmul_rn(b, c), __fmul_rn(a, s)); }

// x / kv_scale as E4M3, saturating.  (One correction by the remainder, as for the 4-bit format; numbers that saturate anyway and infinities go without.)
__device__ __forceinline__ uint32_t e4m3_byte_pair(float a, float b, float scale, float inv) {
  auto over = [&](float x) {
    const float y = x * inv;
    return copysignf(fabsf(y) < 1024.f ? fmaf(fmaf(-y, scale, x), inv, y) : y, x);
  };
  uint32_t r;
  asm("{\n\t.reg .b16 t;\n\tcvt.rn.satfinite.e4m3x2.f32 t, %1, %2;\n\tcvt.u32.u16 %0, t;\n\t}" : "=r"(r) : "f"(over(b)), "f"(over(a)));
  return r;
}

// N neighbouring columns of a key from `first` on, a group of 16 columns being 16 / N neighbouring lanes.
template <int kFormat, int N>
__device__ __forceinline__ void put(const AppendParams& p, Place at, int first, const float (&x)[N]) {
  if constexpr (kFormat == AMLA_CACHE_BF16) {
    __nv_bfloat16* dst = static_cast<__nv_bfloat16*>(p.cache) + (at.page * kPage + at.row) * kDqk + first;
    uint32_t w[N / 2];
#pragma unroll
    for (int i = 0; i < N / 2; ++i) w[i] = sm100::pack_bf16x2(x[2 * i], x[2 * i + 1]);
    if constexpr (N == 8) *reinterpret_cast<uint4*>(dst) = make_uint4(w[0], w[1], w[2], w[3]);
    else *reinterpret_cast<uint32_t*>(dst) = w[0];
  } else if constexpr (kFormat == AMLA_CACHE_E4M3) {
    uint8_t* dst = static_cast<uint8_t*>(p.cache) + (at.page * kPage + at.row) * kDqk + first;
    uint32_t b[N / 2];
#pragma unroll
    for (int i = 0; i < N / 2; ++i) b[i] = e4m3_byte_pair(x[2 * i], x[2 * i + 1], p.kv_scale, p.inv_scale);
    if constexpr (N == 8) *reinterpret_cast<uint2*>(dst) = make_uint2(b[0] | (b[1] << 16), b[2] | (b[3] << 16));
    else *reinterpret_cast<uint16_t*>(dst) = static_cast<uint16_t>(b[0]);
  } else {
    float top = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) top = max_nan(top, fabsf(x[i]));
#pragma unroll
    for (int o = 1; o < kGroup / N; o <<= 1) top = max_nan(top, __shfl_xor_sync(0xffffffffu, top, o));
    const float want = __fdiv_rn(top, 6.f * p.kv_scale);
    uint32_t byte;
    asm("{\n\t.reg .b16 t;\n\tcvt.rn.satfinite.e4m3x2.f32 t, %1, %2;\n\tcvt.u32.u16 %0, t;\n\t}" : "=r"(byte) : "f"(0.f), "f"(want));
    const float step = unpack_f16x2(e4m3x2_to_f16x2(byte)).x * p.kv_scale;
    const float inv = step > 0.f ? __frcp_rn(step) : 0.f;
    uint32_t codes = 0;
#pragma unroll
    for (int i = 0; i < N / 2; ++i) codes |= e2m1_byte(quotient(x[2 * i], step, inv), quotient(x[2 * i + 1], step, inv)) << (8 * i);
    uint8_t* page = static_cast<uint8_t*>(p.cache) + at.page * kPageBytes4;
    uint8_t* dst = page + at.row * kCodeRow + first / 2;
    if constexpr (N == 8) *reinterpret_cast<uint32_t*>(dst) = codes;
    else *dst = static_cast<uint8_t>(codes);
    if (first % kGroup == 0) page[kCodeBytes + at.row * kScaleRow + first / kGroup] = static_cast<uint8_t>(byte);
  }
}

// A token's key as a lane has it: columns 8 lane .. and 256 + 8 lane .. of the latent, and columns 2 lane, 2 lane + 1 of the position part,
// whose partners are its own (interleaved) or those of lane ^ 16.
struct Key { uint4 latent[2]; float pe[2]; };

template <bool kWide>
__device__ __forceinline__ Key load_key(const AppendParams& p, int token, int lane) {
  const __nv_bfloat16* row = p.kv + token * p.row_stride;
  const unsigned short* tail = reinterpret_cast<const unsigned short*>(row + kDv + 2 * lane);
  Key k;
  k.latent[0] = load8<kWide>(row + 8 * lane);
  k.latent[1] = load8<kWide>(row + kDv / 2 + 8 * lane);
  if (kWide) {
    const uint32_t w = *reinterpret_cast<const uint32_t*>(tail);
    k.pe[0] = low(w);
    k.pe[1] = high(w);
  } else {
    k.pe[0] = __uint_as_float(static_cast<uint32_t>(tail[0]) << 16);
    k.pe[1] = __uint_as_float(static_cast<uint32_t>(tail[1]) << 16);
  }
  return k;
}

template <int kFormat, bool kWide, bool kInterleaved>
__device__ __forceinline__ void store_key(const AppendParams& p, const Key& key, Place at, int position, int lane) {
  const float* angles = p.cos_sin + static_cast<size_t>(position) * kRope;
  float2 c, s;
  if (kInterleaved) {
    c.x = c.y = angles[lane];
    s.x = s.y = angles[kPairs + lane];
  } else {
    c = *reinterpret_cast<const float2*>(angles + 2 * (lane & 15));
    s = *reinterpret_cast<const float2*>(angles + kPairs + 2 * (lane & 15));
  }
  float x[2][8];
  unpack8(key.latent[0], x[0]);
  unpack8(key.latent[1], x[1]);
  if (p.weight) {
    float w[2][8];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int first = h * (kDv / 2) + 8 * lane;
      if (p.weight_f32) {
        const float* f = static_cast<const float*>(p.weight) + first;
#pragma unroll
        for (int i = 0; i < 8; ++i) w[h][i] = f[i];
      } else {
        unpack8(load8<kWide>(static_cast<const __nv_bfloat16*>(p.weight) + first), w[h]);
      }
    }
    double sum = 0.;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const double y = x[i >> 3][i & 7];
      sum = fma(y, y, sum);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    const double mean = sum * (1. / kDv) + static_cast<double>(p.eps);
    const float m = static_cast<float>(mean);
    float r;
    if (m >= 0x1p-126f && m <= 0x1.fffffep127f) {
      r = rsqrtf(m);
    } else {                                         // squares may leave FP32's range where their root does not; below 2^-128 so does the root's inverse,
      const bool small = mean < 1.;                  // and the numbers themselves (which are below 2^-58) take its power of two
      r = rsqrtf(static_cast<float>(mean * (small ? 0x1p160 : 0x1p-160)));
      if (!small) r *= 0x1p-80f;
      else
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i >> 3][i & 7] *= 0x1p80f;
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i >> 3][i & 7] = __fmul_rn(__fmul_rn(x[i >> 3][i & 7], r), w[i >> 3][i & 7]);
  }
  float y[2];
  if (kInterleaved) {
    y[0] = turn_first(key.pe[0], key.pe[1], c.x, s.x);
    y[1] = turn_second(key.pe[0], key.pe[1], c.x, s.x);
  } else {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const float other = __shfl_xor_sync(0xffffffffu, key.pe[i], 16), cc = i ? c.y : c.x, ss = i ? s.y : s.x;
      y[i] = lane < 16 ? turn_first(key.pe[i], other, cc, ss) : turn_second(other, key.pe[i], cc, ss);
    }
  }
  put<kFormat, 8>(p, at, 8 * lane, x[0]);
  put<kFormat, 8>(p, at, kDv / 2 + 8 * lane, x[1]);
  put<kFormat, 2>(p, at, kDv + 2 * lane, y);
}

// The angles of a query's eight columns 8 i .., whose partners are their own neighbours (interleaved) or those of lane i ^ 4.
template <bool kInterleaved>
struct Angles {
  static constexpr int kCount = kInterleaved ? 4 : 8;
  float c[kCount], s[kCount];
  __device__ __forceinline__ Angles(const float* row, int i) {
    const float* a = row + (kInterleaved ? 4 * i : 8 * (i & 3));
#pragma unroll
    for (int k = 0; k < kCount; k += 4) {
      const float4 x = *reinterpret_cast<const float4*>(a + k), y = *reinterpret_cast<const float4*>(a + kPairs + k);
      c[k] = x.x; c[k + 1] = x.y; c[k + 2] = x.z; c[k + 3] = x.w;
      s[k] = y.x; s[k + 1] = y.y; s[k + 2] = y.z; s[k + 3] = y.w;
    }
  }
};
template <bool kInterleaved>
__device__ __forceinline__ uint4 rotate8(uint4 v, const Angles<kInterleaved>& a, int i) {
  float x[8], y[8];
  unpack8(v, x);
  if constexpr (kInterleaved) {
#pragma unroll
    for (int k = 0; k < 4; ++k) { y[2 * k] = turn_first(x[2 * k], x[2 * k + 1], a.c[k], a.s[k]); y[2 * k + 1] = turn_second(x[2 * k], x[2 * k + 1], a.c[k], a.s[k]); }
  } else {
    uint4 other;
    other.x = __shfl_xor_sync(0xffffffffu, v.x, 4);
    other.y = __shfl_xor_sync(0xffffffffu, v.y, 4);
    other.z = __shfl_xor_sync(0xffffffffu, v.z, 4);
    other.w = __shfl_xor_sync(0xffffffffu, v.w, 4);
    float z[8];
    unpack8(other, z);
#pragma unroll
    for (int k = 0; k < 8; ++k) y[k] = i < 4 ? turn_first(x[k], z[k], a.c[k], a.s[k]) : turn_second(z[k], x[k], a.c[k], a.s[k]);
  }
  return make_uint4(sm100::pack_bf16x2(y[0], y[1]), sm100::pack_bf16x2(y[2], y[3]), sm100::pack_bf16x2(y[4], y[5]), sm100::pack_bf16x2(y[6], y[7]));
}

constexpr int kWarpHeads = 16, kRounds = kWarpHeads / 4;      // queries of a warp: four at a time, eight lanes each

}  // namespace

// A warp: up to sixteen of a token's queries and, the token's first warp, its key.  What it reads of the token is on its way before it looks for the
// token's place; it finds that by itself, so that no warp waits for another.
template <int kFormat, bool kWide, bool kInterleaved>
__global__ void __launch_bounds__(kThreads) append_kernel(const AppendParams p, uint32_t warps_of_token) {
  behind_the_kernel_in_front();
  const int lane = threadIdx.x & 31;
  const uint32_t unit = blockIdx.x * kWarps + (threadIdx.x >> 5);
  if (unit / warps_of_token >= static_cast<uint32_t>(p.tokens.n)) return;
  const int token = unit / warps_of_token, mine = unit % warps_of_token;
  const int i = lane & 7, head = mine * kWarpHeads + (lane >> 3);
  uint4 v[kRounds];
#pragma unroll
  for (int k = 0; k < kRounds; ++k)
    v[k] = head + 4 * k < p.H ? load8<kWide>(p.q_pe + token * p.q_pe_token + (head + 4 * k) * p.q_pe_head + 8 * i) : make_uint4(0, 0, 0, 0);
  Key key;
  if (mine == 0) key = load_key<kWide>(p, token, lane);
  const Place at = place_of_token(p.tokens, token, lane);
  const int position = p.positions ? p.positions[token] : at.position;
  if (position < 0 || position >= p.n_positions) return;
  if (mine * kWarpHeads < p.H) {
    const Angles<kInterleaved> angles(p.cos_sin + static_cast<size_t>(position) * kRope, i);
#pragma unroll
    for (int k = 0; k < kRounds; ++k) {
      const uint4 y = rotate8<kInterleaved>(v[k], angles, i);
      if (head + 4 * k < p.H) store8<kWide>(p.q + token * p.q_token + (head + 4 * k) * p.q_head + kDv + 8 * i, y);
    }
  }
  if (mine == 0 && at.page >= 0) store_key<kFormat, kWide, kInterleaved>(p, key, at, position, lane);
}

namespace {

constexpr int kColumns8 = kDqk / 8;                  // 72
constexpr int kRowGroups = 4;
constexpr int kMeanThreads = kColumns8 * kRowGroups; // 288
constexpr int kMostWindow = 64;

// Eight columns of key `row`, without the cache's factor.
template <int kFormat>
__device__ __forceinline__ void key8(const void* cache, long long page, int row, int col8, float (&x)[8]) {
  if constexpr (kFormat == AMLA_CACHE_BF16) {
    unpack8(*reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(cache) + (page * kPage + row) * kDqk + 8 * col8), x);
  } else if constexpr (kFormat == AMLA_CACHE_E4M3) {
    const uint2 w = *reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(cache) + (page * kPage + row) * kDqk + 8 * col8);
    const uint32_t pair[4] = {w.x & 0xffffu, w.x >> 16, w.y & 0xffffu, w.y >> 16};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 f = unpack_f16x2(e4m3x2_to_f16x2(pair[i]));
      x[2 * i] = f.x; x[2 * i + 1] = f.y;
    }
  } else {
    const uint8_t* base = static_cast<const uint8_t*>(cache) + page * kPageBytes4;
    const uint32_t codes = *reinterpret_cast<const uint32_t*>(base + row * kCodeRow + 4 * col8), byte = base[kCodeBytes + row * kScaleRow + col8 / 2];
    const uint32_t s2 = e4m3x2_to_f16x2(byte | (byte << 8));
    uint32_t h[4];
    e2m1x8_to_f16x2(codes, h);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 f = unpack_f16x2(mul_f16x2(h[i], s2));
      x[2 * i] = f.x; x[2 * i + 1] = f.y;
    }
  }
}

}  // namespace

// A block looks at `window` tokens and does the pages that are filled by one of them, one after the other: a thread has eight columns of
// sixteen of the 64 keys.
template <int kFormat>
__global__ void __launch_bounds__(kMeanThreads) page_means_kernel(const void* cache, float kv_scale, const Tokens tokens, int window, __nv_bfloat16* means) {
  __shared__ int pages[kMostWindow];
  __shared__ int count;
  __shared__ float sums[kRowGroups - 1][kDqk];
  behind_the_kernel_in_front();
  const int tid = threadIdx.x, wid = tid >> 5, lane = tid & 31;
  if (tid == 0) count = 0;
  __syncthreads();
  for (int i = wid; i < window; i += kMeanThreads / 32) {
    const uint32_t token = blockIdx.x * window + i;
    if (token >= static_cast<uint32_t>(tokens.n)) break;
    const Place at = place_of_token(tokens, token, lane);
    if (lane == 0 && at.page >= 0 && at.row == kPage - 1) pages[atomicAdd(&count, 1)] = static_cast<int>(at.page);
  }
  __syncthreads();
  const int col8 = tid % kColumns8, group = tid / kColumns8;
  for (int k = 0; k < count; ++k) {
    float sum[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) sum[i] = 0.f;
#pragma unroll 8
    for (int r = 0; r < kPage / kRowGroups; ++r) {
      float x[8];
      key8<kFormat>(cache, pages[k], r * kRowGroups + group, col8, x);
#pragma unroll
      for (int i = 0; i < 8; ++i) sum[i] += x[i];
    }
    if (group > 0) {
#pragma unroll
      for (int i = 0; i < 8; ++i) sums[group - 1][8 * col8 + i] = sum[i];
    }
    __syncthreads();
    if (group == 0) {
      const float f = kFormat == AMLA_CACHE_BF16 ? 1.f / kPage : kv_scale * (1.f / kPage);
#pragma unroll
      for (int i = 0; i < 8; ++i) sum[i] = ((sum[i] + sums[0][8 * col8 + i]) + (sums[1][8 * col8 + i] + sums[2][8 * col8 + i])) * f;
      *reinterpret_cast<uint4*>(means + static_cast<size_t>(pages[k]) * kDqk + 8 * col8) =
          make_uint4(sm100::pack_bf16x2(sum[0], sum[1]), sm100::pack_bf16x2(sum[2], sum[3]), sm100::pack_bf16x2(sum[4], sum[5]), sm100::pack_bf16x2(sum[6], sum[7]));
    }
    __syncthreads();
  }
}

namespace {

bool aligned(const void* p, int bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }

int check_books(const int32_t* starts, const void* cache, const int32_t* block_table, const int32_t* seqlens, int format, float kv_scale, int n_tokens, int B, int num_blocks,
                int max_blocks_per_seq) {
  if (format != AMLA_CACHE_BF16 && format != AMLA_CACHE_E4M3 && format != AMLA_CACHE_FP4) return AMLA_ERR_INVALID_ARG;
  if (!starts || !cache || !block_table || !seqlens) return AMLA_ERR_INVALID_ARG;
  if (n_tokens < 0 || B <= 0 || num_blocks <= 0 || max_blocks_per_seq <= 0) return AMLA_ERR_INVALID_ARG;
  if (format != AMLA_CACHE_BF16 && !fp4_scale_ok(kv_scale)) return AMLA_ERR_INVALID_ARG;
  if (!aligned(cache, 16) || !aligned(starts, 4) || !aligned(block_table, 4) || !aligned(seqlens, 4)) return AMLA_ERR_INVALID_ARG;
  return AMLA_OK;
}

template <int kFormat, bool kWide, bool kInterleaved>
cudaError_t launch_append(const AppendParams& p, cudaStream_t stream) {
  const uint32_t warps = p.H > kWarpHeads ? (p.H + kWarpHeads - 1) / kWarpHeads : 1;
  return launch_in_order(append_kernel<kFormat, kWide, kInterleaved>, dim3((p.tokens.n * warps + kWarps - 1) / kWarps), kThreads, 0, stream, p, warps);
}
template <int kFormat>
cudaError_t launch_append(const AppendParams& p, bool wide, bool interleaved, cudaStream_t stream) {
  if (wide) return interleaved ? launch_append<kFormat, true, true>(p, stream) : launch_append<kFormat, true, false>(p, stream);
  return interleaved ? launch_append<kFormat, false, true>(p, stream) : launch_append<kFormat, false, false>(p, stream);
}

}  // namespace

}  // namespace amla

using namespace amla;

extern "C" int amla_cache_append(int format, const void* kv, long long row_stride, int n_tokens, const int32_t* starts, void* kv_cache, float kv_scale, const int32_t* block_table,
                                 const int32_t* seqlens, int B, int num_blocks, int max_blocks_per_seq, const float* cos_sin, int n_positions, const int32_t* positions,
                                 const void* norm_weight, int weight_is_f32, float eps, int interleaved, const void* q_pe, long long q_pe_token_stride, long long q_pe_head_stride, void* q,
                                 long long q_token_stride, long long q_head_stride, int H, void* cuda_stream) {
  const int rc = check_books(starts, kv_cache, block_table, seqlens, format, kv_scale, n_tokens, B, num_blocks, max_blocks_per_seq);
  if (rc != AMLA_OK) return rc;
  if (!cos_sin || n_positions <= 0 || !aligned(cos_sin, 16) || !aligned(positions, 4) || H < 0 || !(eps >= 0.f)) return AMLA_ERR_INVALID_ARG;
  if (!aligned(norm_weight, weight_is_f32 ? 4 : 2)) return AMLA_ERR_INVALID_ARG;
  if (n_tokens == 0) return AMLA_OK;
  if (!kv || !aligned(kv, 2) || (n_tokens > 1 && row_stride < kDqk)) return AMLA_ERR_INVALID_ARG;
  if (H > 0) {
    if (!q_pe || !q || !aligned(q_pe, 2) || !aligned(q, 2) || q_pe_token_stride < 0 || q_pe_head_stride < 0) return AMLA_ERR_INVALID_ARG;
    if ((n_tokens > 1 && q_token_stride < kDqk) || (H > 1 && q_head_stride < kDqk)) return AMLA_ERR_INVALID_ARG;
    if (H > 1024 || static_cast<long long>(n_tokens) * H > (1ll << 34)) return AMLA_ERR_UNSUPPORTED;      // (warps are counted in 32 bits)
  }
  AppendParams p = {};
  p.kv = static_cast<const __nv_bfloat16*>(kv);
  p.row_stride = row_stride;
  p.tokens = Tokens{starts, block_table, seqlens, B, num_blocks, max_blocks_per_seq, n_tokens};
  p.cache = kv_cache;
  p.kv_scale = kv_scale;
  p.inv_scale = format == AMLA_CACHE_BF16 ? 1.f : 1.f / kv_scale;
  p.cos_sin = cos_sin;
  p.n_positions = n_positions;
  p.positions = positions;
  p.weight = norm_weight;
  p.weight_f32 = weight_is_f32;
  p.eps = eps;
  p.q_pe = static_cast<const __nv_bfloat16*>(q_pe);
  p.q_pe_token = q_pe_token_stride;
  p.q_pe_head = q_pe_head_stride;
  p.q = static_cast<__nv_bfloat16*>(q);
  p.q_token = q_token_stride;
  p.q_head = q_head_stride;
  p.H = H;
  bool wide = aligned(kv, 16) && (n_tokens <= 1 || row_stride % 8 == 0) && aligned(norm_weight, 16);
  if (H > 0)
    wide = wide && aligned(q_pe, 16) && aligned(q, 16) && (n_tokens <= 1 || (q_pe_token_stride % 8 == 0 && q_token_stride % 8 == 0)) &&
           (H <= 1 || (q_pe_head_stride % 8 == 0 && q_head_stride % 8 == 0));
  cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  const cudaError_t err = format == AMLA_CACHE_BF16   ? launch_append<AMLA_CACHE_BF16>(p, wide, interleaved != 0, stream)
                          : format == AMLA_CACHE_E4M3 ? launch_append<AMLA_CACHE_E4M3>(p, wide, interleaved != 0, stream)
                                                      : launch_append<AMLA_CACHE_FP4>(p, wide, interleaved != 0, stream);
  if (err != cudaSuccess) { cudaGetLastError(); return AMLA_ERR_CUDA; }
  return AMLA_OK;
}

extern "C" int amla_page_means(int format, const void* kv_cache, float kv_scale, const int32_t* block_table, const int32_t* seqlens, const int32_t* starts, int n_tokens, int B, int num_blocks,
                               int max_blocks_per_seq, void* means, void* cuda_stream) {
  const int rc = check_books(starts, kv_cache, block_table, seqlens, format, kv_scale, n_tokens, B, num_blocks, max_blocks_per_seq);
  if (rc != AMLA_OK) return rc;
  if (!means || !aligned(means, 16)) return AMLA_ERR_INVALID_ARG;
  if (n_tokens == 0) return AMLA_OK;
  // A block's pages come one after the other: a token a block where there are few, at most 64 (a page of one sequence) where there are many, eight blocks for each of a B200's 148 SMs
  // in between.  (Tokens a block, 1 / 8 / 32 / 64, us: 96 tokens 3.8 / 3.8 / 5.3 / 9.1; 2048 of one sequence 4.9 / 4.1 / 4.5 / 5.3; 5 x 1900 12.4 / 5.4 / 4.7 / 5.2; 20 x 2048 48.7 / 15.8 / 14.0 / 15.3;
  // 80 x 2048 176 / 45 / 39 / 37; 1600 x 5 13.4 / 7.4 / 10.0 / 14.0.)
  const int window = n_tokens / (148 * 8) < 1 ? 1 : n_tokens / (148 * 8) > kMostWindow ? kMostWindow : n_tokens / (148 * 8);
  const Tokens tokens{starts, block_table, seqlens, B, num_blocks, max_blocks_per_seq, n_tokens};
  const int grid = (n_tokens - 1) / window + 1;
  cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  __nv_bfloat16* out = static_cast<__nv_bfloat16*>(means);
  const cudaError_t err = format == AMLA_CACHE_BF16   ? launch_in_order(page_means_kernel<AMLA_CACHE_BF16>, dim3(grid), kMeanThreads, 0, stream, kv_cache, kv_scale, tokens, window, out)
                          : format == AMLA_CACHE_E4M3 ? launch_in_order(page_means_kernel<AMLA_CACHE_E4M3>, dim3(grid), kMeanThreads, 0, stream, kv_cache, kv_scale, tokens, window, out)
                                                      : launch_in_order(page_means_kernel<AMLA_CACHE_FP4>, dim3(grid), kMeanThreads, 0, stream, kv_cache, kv_scale, tokens, window, out);
  if (err != cudaSuccess) { cudaGetLastError(); return AMLA_ERR_CUDA; }
  return AMLA_OK;
}
