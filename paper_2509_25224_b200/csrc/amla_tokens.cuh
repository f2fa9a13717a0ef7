// Where the tokens of a call lie in a paged cache: rows starts[b] .. starts[b + 1] - 1 of a call's tokens are the last ones of sequence b.
#pragma once

#include <stdint.h>

#include "amla_common.cuh"

namespace amla {

struct Tokens {
  const int32_t* starts;         // [B + 1]
  const int32_t* block_table;    // [B, width]
  const int32_t* seqlens;        // [B]
  int B, num_blocks, width, n;
};

struct Place {
  long long page;                // -1: none
  int row;                       // in the page
  int position;                  // in the sequence; -1: none
};

// Behind this, what the kernel in front on the stream wrote may be read.  (By ordinary loads: kernels that call this are placed while it is still
// writing, so that none of their pointers may promise that nobody else writes.)
__device__ __forceinline__ void behind_the_kernel_in_front() {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;");
}

// By a whole warp, which gets the same answer in every lane.  The sequence is the last one that begins at or before the token (one without
// tokens holds none): 32 candidates at a time, the last 32 with their ends and lengths, so that up to 32 sequences take two dependent reads
// (the other is the page number), up to 1024 three.
__device__ __forceinline__ Place place_of_token(const Tokens& t, int token, int lane) {
  Place p{-1, 0, -1};
  int lo = 0, n = t.B;
  while (n > 32) {
    const int step = (n + 31) / 32, at = lane * step;
    const uint32_t yes = __ballot_sync(0xffffffffu, at < n && t.starts[lo + at] <= token);
    const int last = yes ? 31 - __clz(yes) : 0;
    lo += last * step;
    n = min(step, n - last * step);
  }
  const int start = t.starts[lo + min(lane, n)], len = t.seqlens[lo + min(lane, n - 1)];
  const uint32_t yes = __ballot_sync(0xffffffffu, lane < n && start <= token);
  const int last = yes ? 31 - __clz(yes) : 0;
  const int begin = __shfl_sync(0xffffffffu, start, last), next = __shfl_sync(0xffffffffu, start, min(last + 1, 31)), keys = __shfl_sync(0xffffffffu, len, last);
  const int end = last < 31 ? next : t.starts[lo + 32];
  lo += last;
  if (token < begin || token >= end) return p;
  const long long at = static_cast<long long>(keys) - (end - token);
  if (at < 0) return p;
  p.position = static_cast<int>(at);
  p.row = static_cast<int>(at % kPage);
  if (at >= static_cast<long long>(t.width) * kPage) return p;
  const int page = t.block_table[static_cast<size_t>(lo) * t.width + at / kPage];
  if (page >= 0 && page < t.num_blocks) p.page = page;
  return p;
}

}  // namespace amla
