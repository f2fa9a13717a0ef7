// Tokens into a 4-bit cache and back (the format is in amla_fp4.cuh).
//
// store: a group's scale is the E4M3 number nearest to max|x| / (6 kv_scale), 6 being E2M1's largest; its elements are the
// E2M1 numbers nearest to x / (scale * kv_scale), ties to even for both.  With bf16 inputs ties are common (x has eight bits, a
// midpoint times a scale at most seven), so the quotient has to be the true one there: x * fl(1 / step) alone is off at eleven of
// the 56 pairs of mantissas, with one correction by the remainder it is exact wherever the quotient is representable.
// A group that holds a NaN gets the scale NaN and reads back as NaN; an infinity saturates (2688 kv_scale).
//
// Both are streams: 1152 bytes of bf16 and 324 of cache a token.  A thread does eight columns (16 bytes of bf16, one 32-bit
// word of codes), 72 threads a token, so that every access of a warp is to whole neighbouring sectors.  A step's 96 tokens take 3.0 us, to load them 2.8
// (a launch, and a search for the sequence, its length and its page, each read after the other), and 7 of the host.  4 x 2048 tokens are stored in 5.7 us and
// 23 k loaded in 10.0, from memory (2.1 and 3.4 TB/s; 4.4 and 7.3 from L2), which is as long as the host takes for the two calls.
#include <cuda_bf16.h>

#include "../../include/amla.h"
#include "amla_fp4.cuh"
#include "amla_sm100.cuh"

namespace amla {

namespace {

constexpr int kTokenThreads = kDqk / 8;              // 72
constexpr int kTokens = 4;                           // tokens a block has in hand at a time
constexpr int kThreads = kTokens * kTokenThreads;    // 288
constexpr int kRounds = 2;                           // and how often, per block

// Where token `token` of the batch lies: byte offset of its page, and its row in the page; -1 if it has no place.  The tokens
// starts[b] .. starts[b+1] - 1 are the last ones of sequence b, in order.
struct Place { long long page_off; int row; };
__device__ __forceinline__ Place place_of(const int32_t* starts, const int32_t* block_table, const int32_t* seqlens, int B, int num_blocks, int max_blocks_per_seq, int token) {
  Place p{-1, 0};
  int lo = 0, hi = B - 1;                            // the sequence: the last one that begins at or before the token (one without tokens holds none)
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (starts[mid] <= token) lo = mid; else hi = mid - 1;
  }
  if (token < starts[lo] || token >= starts[lo + 1]) return p;
  const long long at = static_cast<long long>(seqlens[lo]) - (starts[lo + 1] - token);
  if (at < 0 || at >= static_cast<long long>(max_blocks_per_seq) * kPage) return p;
  const int page = block_table[static_cast<size_t>(lo) * max_blocks_per_seq + at / kPage];
  if (page < 0 || page >= num_blocks) return p;
  p.page_off = static_cast<long long>(page) * kPageBytes4;
  p.row = static_cast<int>(at % kPage);
  return p;
}

__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
// x / step, inv = fl(1 / step) (0 for a group of zeros).  What is beyond E2M1's 6 by far saturates whatever its last bits are (and the
// remainder of an infinity is a NaN).  The sign is x's, of a zero too (the remainder of -0 is +0).
__device__ __forceinline__ float quotient(float x, float step, float inv) {
  const float y = x * inv;
  return copysignf(fabsf(y) < 16.f ? fmaf(fmaf(-y, step, x), inv, y) : y, x);
}
// low half: a, high half: b
__device__ __forceinline__ uint32_t e2m1_byte(float a, float b) {
  uint32_t r;
  asm("{\n\t.reg .b8 t;\n\tcvt.rn.satfinite.e2m1x2.f32 t, %1, %2;\n\tcvt.u32.u8 %0, t;\n\t}" : "=r"(r) : "f"(b), "f"(a));
  return r;
}

// (Ordinary loads, here and of all pointers below: the kernel in front may still be writing the tokens when this one is placed.)
// kWide: rows begin at 16 bytes, so that eight columns are one access
template <bool kWide>
__device__ __forceinline__ uint4 load_columns(const __nv_bfloat16* p) {
  if (kWide) return *reinterpret_cast<const uint4*>(p);
  uint32_t w[4];
  const unsigned short* h = reinterpret_cast<const unsigned short*>(p);
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = h[2 * i] | (static_cast<uint32_t>(h[2 * i + 1]) << 16);
  return make_uint4(w[0], w[1], w[2], w[3]);
}
template <bool kWide>
__device__ __forceinline__ void store_columns(__nv_bfloat16* p, const uint32_t (&w)[4]) {
  if (kWide) {
    *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
  } else {
    unsigned short* h = reinterpret_cast<unsigned short*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) { h[2 * i] = static_cast<unsigned short>(w[i]); h[2 * i + 1] = static_cast<unsigned short>(w[i] >> 16); }
  }
}

}  // namespace

template <bool kWide>
__global__ void __launch_bounds__(kThreads) store_fp4_kernel(const __nv_bfloat16* kv, long long row_stride, int n_tokens, const int32_t* starts,
                                                             uint8_t* cache, float kv_scale, const int32_t* block_table,
                                                             const int32_t* seqlens, int B, int num_blocks, int max_blocks_per_seq) {
  __shared__ Place places[kTokens * kRounds];
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;");
  const int token0 = blockIdx.x * (kTokens * kRounds), mine = threadIdx.x / kTokenThreads, col = threadIdx.x % kTokenThreads;
  uint4 x[kRounds];
#pragma unroll
  for (int k = 0; k < kRounds; ++k) {
    const int token = token0 + k * kTokens + mine;
    x[k] = token < n_tokens ? load_columns<kWide>(kv + token * row_stride + 8 * col) : make_uint4(0, 0, 0, 0);
  }
  if (threadIdx.x < kTokens * kRounds) {
    const int token = token0 + threadIdx.x;
    places[threadIdx.x] = token < n_tokens ? place_of(starts, block_table, seqlens, B, num_blocks, max_blocks_per_seq, token) : Place{-1, 0};
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < kRounds; ++k) {
    const uint32_t w[4] = {x[k].x, x[k].y, x[k].z, x[k].w};
    float v[8], top = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __uint_as_float(w[i] << 16);
      v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
      top = max_nan(top, max_nan(fabsf(v[2 * i]), fabsf(v[2 * i + 1])));
    }
    top = max_nan(top, __shfl_xor_sync(0xffffffffu, top, 1));        // the other half of the group
    const float want = __fdiv_rn(top, 6.f * kv_scale);
    uint32_t byte;
    asm("{\n\t.reg .b16 t;\n\tcvt.rn.satfinite.e4m3x2.f32 t, %1, %2;\n\tcvt.u32.u16 %0, t;\n\t}" : "=r"(byte) : "f"(0.f), "f"(want));
    const float step = unpack_f16x2(e4m3x2_to_f16x2(byte)).x * kv_scale;
    const float inv = step > 0.f ? __frcp_rn(step) : 0.f;
    uint32_t codes = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) codes |= e2m1_byte(quotient(v[2 * i], step, inv), quotient(v[2 * i + 1], step, inv)) << (8 * i);
    const Place p = places[k * kTokens + mine];
    if (p.page_off >= 0) {
      uint8_t* page = cache + p.page_off;
      *reinterpret_cast<uint32_t*>(page + p.row * kCodeRow + 4 * col) = codes;
      if ((col & 1) == 0) page[kCodeBytes + p.row * kScaleRow + col / 2] = static_cast<uint8_t>(byte);
    }
  }
}

template <bool kWide>
__global__ void __launch_bounds__(kThreads) load_fp4_kernel(const uint8_t* cache, float kv_scale, const int32_t* block_table,
                                                            const int32_t* seqlens, const int32_t* starts, int B, int num_blocks,
                                                            int max_blocks_per_seq, __nv_bfloat16* out, long long row_stride, int n_tokens) {
  __shared__ Place places[kTokens * kRounds];
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;");
  const int token0 = blockIdx.x * (kTokens * kRounds), mine = threadIdx.x / kTokenThreads, col = threadIdx.x % kTokenThreads;
  if (threadIdx.x < kTokens * kRounds) {
    const int token = token0 + threadIdx.x;
    places[threadIdx.x] = token < n_tokens ? place_of(starts, block_table, seqlens, B, num_blocks, max_blocks_per_seq, token) : Place{-1, 0};
  }
  __syncthreads();
  uint32_t codes[kRounds], byte[kRounds];
#pragma unroll
  for (int k = 0; k < kRounds; ++k) {
    const Place p = places[k * kTokens + mine];
    codes[k] = byte[k] = 0;
    if (p.page_off >= 0) {
      codes[k] = *reinterpret_cast<const uint32_t*>(cache + p.page_off + p.row * kCodeRow + 4 * col);
      byte[k] = cache[p.page_off + kCodeBytes + p.row * kScaleRow + col / 2];
    }
  }
#pragma unroll
  for (int k = 0; k < kRounds; ++k) {
    const int token = token0 + k * kTokens + mine;
    const uint32_t s2 = e4m3x2_to_f16x2(byte[k] | (byte[k] << 8));
    uint32_t h[4], w[4];
    e2m1x8_to_f16x2(codes[k], h);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 f = unpack_f16x2(mul_f16x2(h[i], s2));
      w[i] = sm100::pack_bf16x2(f.x * kv_scale, f.y * kv_scale);
    }
    if (token < n_tokens) store_columns<kWide>(out + token * row_stride + 8 * col, w);
  }
}

namespace {

template <typename... Args>
cudaError_t launch_tokens(void (*kern)(Args...), int n_tokens, cudaStream_t stream, Args... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((n_tokens + kTokens * kRounds - 1) / (kTokens * kRounds));
  cfg.blockDim = dim3(kThreads);
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kern, args...);
}

int check_tokens(const void* rows, long long row_stride, int n_tokens, const int32_t* starts, const void* cache, float kv_scale, const int32_t* block_table, const int32_t* seqlens,
                 int B, int num_blocks, int max_blocks_per_seq) {
  if (!starts || !cache || !block_table || !seqlens || (!rows && n_tokens > 0)) return AMLA_ERR_INVALID_ARG;
  if (n_tokens < 0 || B <= 0 || num_blocks <= 0 || max_blocks_per_seq <= 0 || (n_tokens > 1 && row_stride < kDqk)) return AMLA_ERR_INVALID_ARG;
  if (!fp4_scale_ok(kv_scale)) return AMLA_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(cache) & 15) || (reinterpret_cast<uintptr_t>(rows) & 1)) return AMLA_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(starts) | reinterpret_cast<uintptr_t>(block_table) | reinterpret_cast<uintptr_t>(seqlens)) & 3) return AMLA_ERR_INVALID_ARG;
  return AMLA_OK;
}

bool wide_rows(const void* rows, long long row_stride) { return ((reinterpret_cast<uintptr_t>(rows) & 15) == 0) && (row_stride % 8 == 0); }

}  // namespace

}  // namespace amla

using namespace amla;

extern "C" int amla_cache_store_fp4(const void* kv, long long row_stride, int n_tokens, const int32_t* starts, void* cache, float kv_scale, const int32_t* block_table,
                                    const int32_t* seqlens, int B, int num_blocks, int max_blocks_per_seq, void* cuda_stream) {
  const int rc = check_tokens(kv, row_stride, n_tokens, starts, cache, kv_scale, block_table, seqlens, B, num_blocks, max_blocks_per_seq);
  if (rc != AMLA_OK || n_tokens == 0) return rc;
  const cudaError_t err = launch_tokens(wide_rows(kv, row_stride) ? store_fp4_kernel<true> : store_fp4_kernel<false>, n_tokens, static_cast<cudaStream_t>(cuda_stream),
                                        static_cast<const __nv_bfloat16*>(kv), row_stride, n_tokens, starts, static_cast<uint8_t*>(cache), kv_scale, block_table, seqlens, B,
                                        num_blocks, max_blocks_per_seq);
  if (err != cudaSuccess) { cudaGetLastError(); return AMLA_ERR_CUDA; }
  return AMLA_OK;
}

extern "C" int amla_cache_load_fp4(const void* cache, float kv_scale, const int32_t* block_table, const int32_t* seqlens, const int32_t* starts, int B, int num_blocks,
                                   int max_blocks_per_seq, void* out, long long row_stride, int n_tokens, void* cuda_stream) {
  const int rc = check_tokens(out, row_stride, n_tokens, starts, cache, kv_scale, block_table, seqlens, B, num_blocks, max_blocks_per_seq);
  if (rc != AMLA_OK || n_tokens == 0) return rc;
  const cudaError_t err = launch_tokens(wide_rows(out, row_stride) ? load_fp4_kernel<true> : load_fp4_kernel<false>, n_tokens, static_cast<cudaStream_t>(cuda_stream),
                                        static_cast<const uint8_t*>(cache), kv_scale, block_table, seqlens, starts, B, num_blocks, max_blocks_per_seq,
                                        static_cast<__nv_bfloat16*>(out), row_stride, n_tokens);
  if (err != cudaSuccess) { cudaGetLastError(); return AMLA_ERR_CUDA; }
  return AMLA_OK;
}
