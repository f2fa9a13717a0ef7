// Care of a cache's pages on the device: copying them, and the books of which sequence holds which (block table, lengths, and a
// count of references for every page; a page without references is free).  No entry reads a device value on the host, so a
// serving loop can enqueue its steps, or replay them from a graph, without waiting.
//
// free, fork, reserve and compact follow one rule: pages are handed out lowest first, in the order of the requests.  That is a rank
// among the free pages (or, to compact, among those in use), which blocks of a grid find from one another's totals: a launch
// counts by chunks of kChunk pages, the next adds the totals up in front of its chunk.  Up to kChunk pages the first launch is left out.
//
// What bounds them: the books are some kilobytes, so that free, fork, reserve and a compaction that finds nothing to move cost their launches
// and a few dependent reads (1.3, 3.6, 2.8 and 8.2 us in a graph, 64 rows of 128 entries and 8192 pages); copies are bound by the
// memory, which takes 16 bytes a thread four deep at full occupancy: a list of 5000 pages of 36 864 bytes moves at 98 % of the rate of a plain copy, a
// compaction of 2900 of 73 728 at 85 % with its launches.
#include <algorithm>

#include "../../include/amla.h"
#include "amla_common.cuh"

namespace amla {

namespace {

constexpr int kScanThreads = 1024;
constexpr int kPerThread = 8;
constexpr int kChunk = kScanThreads * kPerThread;    // pages a block looks at
constexpr int kRowThreads = 256;
constexpr int kCopyThreads = 256;
constexpr int kCopyUnroll = 4;
constexpr int kSegment = kCopyThreads * kCopyUnroll; // 16-byte pieces that a block copies at a time
// Blocks that move pages.  How many there are to move is only known on the device, so that a block takes every kMoveBlocks-th piece
// of the work.  9 948 moves of 20 736 bytes (412 MB), with the launches in front and the events' own 5 us: 87 us with the eight
// blocks that an SM holds (the second segment of a page is short, and a block has always the one kind or the other), 79 with four
// times as many, which are dealt out as others end, 97 with one for every piece that there might be.  (2900 moves of 73 728, 428 MB, with the call and a copy of
// the books and without events: 82.6, 78.4.  A compaction of 8192 pages that finds nothing to move: 4.2, 8.2.)
constexpr int kMoveBlocks = 148 * 32;
constexpr size_t kAlign = 256;

size_t align_up(size_t x) { return (x + kAlign - 1) / kAlign * kAlign; }
int chunks_of(int num_blocks) { return (num_blocks + kChunk - 1) / kChunk; }
__host__ __device__ __forceinline__ int pages_of(int n) { return n > 0 ? (n - 1) / kPage + 1 : 0; }
__device__ __forceinline__ int length_of(const int32_t* seqlens, int row, int width) { return min(max(seqlens[row], 0), width * kPage); }

// scratch: [0] pages counted in all (free, or in use), [1] pages to move | totals by chunk | three lists of pages | a rank for every row
struct Scratch { int* head; int* totals; int* list; int* list2; int* rank; int* row_rank; };
size_t scratch_bytes(int num_blocks, int rows) {
  return kAlign + align_up(sizeof(int) * static_cast<size_t>(chunks_of(num_blocks))) + 3 * align_up(sizeof(int) * static_cast<size_t>(num_blocks)) +
         align_up(sizeof(int) * static_cast<size_t>(rows));
}
Scratch carve(void* workspace, int num_blocks) {
  char* p = static_cast<char*>(workspace);
  Scratch s;
  s.head = reinterpret_cast<int*>(p); p += kAlign;
  s.totals = reinterpret_cast<int*>(p); p += align_up(sizeof(int) * static_cast<size_t>(chunks_of(num_blocks)));
  const size_t list = align_up(sizeof(int) * static_cast<size_t>(num_blocks));
  s.list = reinterpret_cast<int*>(p); p += list;
  s.list2 = reinterpret_cast<int*>(p); p += list;
  s.rank = reinterpret_cast<int*>(p); p += list;
  s.row_rank = reinterpret_cast<int*>(p);
  return s;
}

// Sum over the block in front of this thread; *all = over all of it.
template <int kThreads, typename T>
__device__ __forceinline__ T block_scan(T v, T* all) {
  __shared__ T warps[kThreads / 32];
  const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
  auto scan = [&](T x) {
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const T y = __shfl_up_sync(0xffffffffu, x, o);
      if (lane >= o) x += y;
    }
    return x;
  };
  const T upto = scan(v);
  __syncthreads();                                   // (an earlier scan has been read)
  if (lane == 31) warps[wid] = upto;
  __syncthreads();
  const T w = lane < kThreads / 32 ? warps[lane] : T(0);
  const T sums = scan(w);
  *all = __shfl_sync(0xffffffffu, sums, kThreads / 32 - 1);
  return __shfl_sync(0xffffffffu, sums - w, wid) + upto - v;
}

// Which of a thread's kPerThread neighbouring pages are in use, as bits; beyond the cache: neither in use nor free.
__device__ __forceinline__ uint32_t used_bits(const int32_t* refs, int num_blocks, int first, uint32_t* exist) {
  uint32_t used = 0, there = 0;
  if (first + kPerThread <= num_blocks && (reinterpret_cast<uintptr_t>(refs) & 15) == 0) {
    int v[kPerThread];
#pragma unroll
    for (int i = 0; i < kPerThread / 4; ++i) {
      const int4 x = reinterpret_cast<const int4*>(refs + first)[i];
      v[4 * i] = x.x; v[4 * i + 1] = x.y; v[4 * i + 2] = x.z; v[4 * i + 3] = x.w;
    }
#pragma unroll
    for (int i = 0; i < kPerThread; ++i) used |= (v[i] > 0 ? 1u : 0u) << i;
    there = (1u << kPerThread) - 1;
  } else {
#pragma unroll
    for (int i = 0; i < kPerThread; ++i)
      if (first + i < num_blocks) { there |= 1u << i; used |= (refs[first + i] > 0 ? 1u : 0u) << i; }
  }
  *exist = there;
  return used;
}

// Behind this, what the kernel in front wrote may be read.  (By ordinary loads: the kernels here are placed while it is still writing,
// so that none of their pointers may be __restrict__ or go through __ldg, which promise that nobody else writes.)
__device__ __forceinline__ void begin() {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;");
}

// Pages of a chunk that are in use (kUsed) or free.
template <bool kUsed>
__global__ void __launch_bounds__(kScanThreads) count_pages_kernel(const int32_t* refs, int num_blocks, int* totals) {
  begin();
  uint32_t there;
  const uint32_t used = used_bits(refs, num_blocks, blockIdx.x * kChunk + threadIdx.x * kPerThread, &there);
  int all;
  block_scan<kScanThreads>(__popc(kUsed ? used : there & ~used), &all);
  if (threadIdx.x == 0) totals[blockIdx.x] = all;
}
// The totals in front of this block's chunk, and of all `chunks`.
__device__ __forceinline__ int chunks_before(const int* totals, int chunks, int* all) {
  int front = 0, sum = 0;
  for (int c = threadIdx.x; c < chunks; c += kScanThreads) {
    const int v = totals[c];
    sum += v;
    if (c < static_cast<int>(blockIdx.x)) front += v;
  }
  int total_front;
  block_scan<kScanThreads>(front, &total_front);
  block_scan<kScanThreads>(sum, all);
  return total_front;
}

// What a call asks pages for.  fork: one for each parent that ends inside a page; reserve: those between the old and the new length.
struct Requests {
  const int32_t* seqlens;
  const int32_t* parents;       // fork (else null)
  const int32_t* children;
  const int32_t* new_lens;      // reserve
  int n, B, width;
};
__device__ __forceinline__ bool fork_asked(const Requests& q, int k) {
  const int p = q.parents[k], c = q.children[k];
  return p >= 0 && p < q.B && c >= 0 && c < q.B && p != c;
}
// (a length that the table has no room for asks for none)
__device__ __forceinline__ int reserve_asks(const Requests& q, int row) {
  const int now = length_of(q.seqlens, row, q.width), then = q.new_lens[row];
  return then > now && then <= q.width * kPage ? pages_of(then) - pages_of(now) : 0;
}
__device__ __forceinline__ int asks(const Requests& q, int k) {
  if (q.parents == nullptr) return reserve_asks(q, k);
  return fork_asked(q, k) && length_of(q.seqlens, q.parents[k], q.width) % kPage != 0 ? 1 : 0;
}

// The block's requests in order, one a thread, for `more` pages each: where a request's pages begin among the free ones, of which `given`
// are given out and `pages` are there; -1 if they do not suffice.  Such a request takes none, so that a smaller one behind it may find its own.
// Returns it, and leaves in *given what is given out behind the block's requests.
// Where all find theirs, which is always but when a cache runs full, the sum of the requests in front says it.  Else a warp goes through
// them one by one (whether one is served depends on all in front of it): 2.1 us more with 64 rows, 11.6 with 1024.
__device__ __forceinline__ int place_requests(int more, int pages, int* given) {
  __shared__ int places[kScanThreads];
  __shared__ int behind;
  long long all;
  const long long before = block_scan<kScanThreads, long long>(more, &all);
  const int at0 = *given;
  if (at0 + all <= pages) {
    *given = static_cast<int>(at0 + all);
    return static_cast<int>(at0 + before);
  }
  places[threadIdx.x] = more;
  __syncthreads();
  if (threadIdx.x < 32) {
    int at = at0;
#pragma unroll 1
    for (int w = threadIdx.x; w < kScanThreads; w += 32) {
      const int mine = places[w];
      int place = at;
      if (__any_sync(0xffffffffu, mine > 0)) {
#pragma unroll
        for (int i = 0; i < 32; ++i) {
          const int n = __shfl_sync(0xffffffffu, mine, i);
          const bool fits = n <= pages - at;
          if (static_cast<int>(threadIdx.x) == i) place = fits ? at : -1;
          at += fits ? n : 0;
        }
      }
      places[w] = place;
    }
    if (threadIdx.x == 0) behind = at;
  }
  __syncthreads();
  *given = behind;
  return places[threadIdx.x];
}
constexpr int kNoLimit = 1 << 30;                    // more pages than any cache has

// The free pages in order: list[rank], for the first `most` of them; head[0] = how many there are.  A block more than there are chunks
// works out where every request's pages begin among them (here, since the launch that serves the requests changes the lengths): a reserve's with
// the free pages as their limit, a fork's, which are for one page at most, without: the launch that serves them holds them against head[0].
__global__ void __launch_bounds__(kScanThreads) list_free_kernel(const int32_t* refs, int num_blocks, const int* totals, int most, int* head,
                                                                 int* list, const Requests q, int* row_rank) {
  begin();
  const int chunks = gridDim.x - 1;
  if (static_cast<int>(blockIdx.x) == chunks) {
    int pages = kNoLimit, given = 0;
    if (q.parents == nullptr) chunks_before(totals, chunks, &pages);
    for (int k0 = 0; k0 < q.n; k0 += kScanThreads) {
      const int k = k0 + threadIdx.x, place = place_requests(k < q.n ? asks(q, k) : 0, pages, &given);
      if (k < q.n) row_rank[k] = place;
    }
    return;
  }
  uint32_t there;
  const int first = blockIdx.x * kChunk + threadIdx.x * kPerThread;
  const uint32_t used = used_bits(refs, num_blocks, first, &there);
  uint32_t open = there & ~used;
  int all = 0, before = 0, here;
  if (chunks > 1) before = chunks_before(totals, chunks, &all);
  int rank = before + block_scan<kScanThreads>(__popc(open), &here);
  if (threadIdx.x == 0 && blockIdx.x == 0) head[0] = chunks > 1 ? all : here;
  for (; open != 0 && rank < most; open &= open - 1) list[rank++] = first + __ffs(open) - 1;
}

// One block per listed row.  A row's length says whether it still holds its pages: who sets it to zero gives them up, so that a row
// that is listed twice is freed once.
__global__ void __launch_bounds__(kRowThreads) free_rows_kernel(int32_t* block_table, int32_t* seqlens, int32_t* refs, const int32_t* rows,
                                                                int B, int num_blocks, int width) {
  __shared__ int length;
  begin();
  const int row = rows[blockIdx.x];
  if (row < 0 || row >= B) return;
  if (threadIdx.x == 0) length = min(max(atomicExch(seqlens + row, 0), 0), width * kPage);
  __syncthreads();
  const int n = pages_of(length);
  int32_t* mine = block_table + static_cast<size_t>(row) * width;
  for (int i = threadIdx.x; i < n; i += kRowThreads) {
    const int page = mine[i];
    if (page >= 0 && page < num_blocks) atomicSub(refs + page, 1);
    mine[i] = -1;
  }
}

// One row of blocks per fork, blockIdx.y of which share the copy of its last page; the first also does the books.  (Parents and
// children are different rows, so that what is read here of a parent is not written here.)
__global__ void __launch_bounds__(kCopyThreads) fork_rows_kernel(uint4* cache, int page_pieces, int32_t* block_table, int32_t* seqlens,
                                                                 int32_t* refs, const Requests q, int num_blocks, const int* head,
                                                                 const int* list, const int* row_rank, int32_t* served) {
  begin();
  const int k = blockIdx.x, width = q.width;
  const bool asked = fork_asked(q, k);
  const int parent = q.parents[k], child = q.children[k];
  const int n = asked ? length_of(seqlens, parent, width) : 0, full = n / kPage;
  const bool ragged = n % kPage != 0;
  const int rank = row_rank[k];
  const bool ok = asked && (!ragged || rank < min(head[0], q.n));
  const int fresh = ok && ragged ? list[rank] : -1;
  const int32_t* from = block_table + static_cast<size_t>(asked ? parent : 0) * width;
  const int last = ragged ? from[full] : -1;
  if (blockIdx.y == 0) {
    int32_t* to = block_table + static_cast<size_t>(asked ? child : 0) * width;
    if (asked)
      for (int i = threadIdx.x; i < width; i += kCopyThreads) {
        int page = -1;
        if (ok && i < full) {
          page = from[i];
          if (page >= 0 && page < num_blocks) atomicAdd(refs + page, 1);
        } else if (ok && i == full && ragged) {
          page = fresh;
        }
        to[i] = page;
      }
    if (threadIdx.x == 0) {
      if (fresh >= 0) refs[fresh] = 1;
      if (asked) seqlens[child] = ok ? n : 0;
      if (served) served[k] = ok ? 1 : 0;
    }
  }
  if (fresh < 0) return;
  const bool there = last >= 0 && last < num_blocks;  // (a page outside the cache reads as zeros)
  const uint4* src = cache + static_cast<size_t>(there ? last : 0) * page_pieces;
  uint4* dst = cache + static_cast<size_t>(fresh) * page_pieces;
  for (int i = blockIdx.y * kSegment + threadIdx.x; i < page_pieces; i += gridDim.y * kSegment) {
    uint4 x[kCopyUnroll];
#pragma unroll
    for (int u = 0; u < kCopyUnroll; ++u) x[u] = there && i + u * kCopyThreads < page_pieces ? src[i + u * kCopyThreads] : make_uint4(0, 0, 0, 0);
#pragma unroll
    for (int u = 0; u < kCopyUnroll; ++u)
      if (i + u * kCopyThreads < page_pieces) dst[i + u * kCopyThreads] = x[u];
  }
}

// The whole of it by one block, for a cache of at most kChunk pages: the free pages are listed in shared memory, a thread serves a
// row's first page and its books, the warp the others.  (64 rows, 8192 pages: 2.7 us, and 7 us of the host; as the two launches that
// larger caches take 3.1 us, and 13.)
__global__ void __launch_bounds__(kScanThreads) reserve_small_kernel(int32_t* block_table, int32_t* seqlens, int32_t* refs, int num_blocks, const Requests q,
                                                                     int32_t* granted) {
  __shared__ int list[kChunk];
  begin();
  const int tid = threadIdx.x, lane = tid & 31;
  uint32_t there;
  const uint32_t used = used_bits(refs, num_blocks, tid * kPerThread, &there);
  uint32_t open = there & ~used;
  int pages;
  int at = block_scan<kScanThreads>(__popc(open), &pages);
  for (; open != 0; open &= open - 1) list[at++] = tid * kPerThread + __ffs(open) - 1;
  __syncthreads();
  int given = 0;
  for (int row0 = 0; row0 < q.B; row0 += kScanThreads) {
    const int row = row0 + tid;
    const bool mine = row < q.B;
    const int now = mine ? length_of(q.seqlens, row, q.width) : 0, then = mine ? q.new_lens[row] : 0, more = mine ? reserve_asks(q, row) : 0;
    const int rank = place_requests(more, pages, &given);
    const bool ok = then <= q.width * kPage && rank >= 0;
    const size_t entry = static_cast<size_t>(mine ? row : 0) * q.width + pages_of(now);
    if (ok && more > 0) {
      const int page = list[rank];
      block_table[entry] = page;
      refs[page] = 1;
    }
    if (mine && ok && then > now) seqlens[row] = then;
    if (mine && granted) granted[row] = ok ? 1 : 0;
    for (uint32_t todo = __ballot_sync(0xffffffffu, ok && more > 1); todo != 0; todo &= todo - 1) {
      const int who = __ffs(todo) - 1, count = __shfl_sync(0xffffffffu, more, who), first = __shfl_sync(0xffffffffu, rank, who);
      const size_t to = __shfl_sync(0xffffffffu, static_cast<unsigned long long>(entry), who);
      for (int i = 1 + lane; i < count; i += 32) {
        const int page = list[first + i];
        block_table[to + i] = page;
        refs[page] = 1;
      }
    }
  }
}

// One block per row.
__global__ void __launch_bounds__(kRowThreads) reserve_rows_kernel(int32_t* block_table, int32_t* seqlens, int32_t* refs, const Requests q,
                                                                   const int* list, const int* row_rank, int32_t* granted) {
  begin();
  const int row = blockIdx.x;
  const int now = length_of(q.seqlens, row, q.width), then = q.new_lens[row], more = reserve_asks(q, row), rank = row_rank[row];
  const bool ok = then <= q.width * kPage && rank >= 0;
  if (ok)
    for (int i = threadIdx.x; i < more; i += kRowThreads) {
      const int page = list[rank + i];
      block_table[static_cast<size_t>(row) * q.width + pages_of(now) + i] = page;
      refs[page] = 1;
    }
  __syncthreads();                                   // the length has been read by all
  if (threadIdx.x == 0) {
    if (ok && then > now) seqlens[row] = then;
    if (granted) granted[row] = ok ? 1 : 0;
  }
}

// Compaction, with `live` pages in use: the holes in front of page `live` in order (holes[i]), the pages in use behind it from the
// last to the first (high[i]; rank[page] = i), and how many those are (head[1]).
__global__ void __launch_bounds__(kScanThreads) list_moves_kernel(const int32_t* refs, int num_blocks, const int* totals, int* head, int* holes,
                                                                  int* high, int* rank, int32_t* live_out) {
  begin();
  uint32_t there;
  const int first = blockIdx.x * kChunk + threadIdx.x * kPerThread;
  const uint32_t used = used_bits(refs, num_blocks, first, &there);
  int live = 0, before = 0, here;
  if (gridDim.x > 1) before = chunks_before(totals, gridDim.x, &live);
  int u = before + block_scan<kScanThreads>(__popc(used), &here);
  if (gridDim.x == 1) live = here;
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    head[0] = live;
    if (live_out) *live_out = live;
    if (live == num_blocks) head[1] = 0;
  }
#pragma unroll
  for (int i = 0; i < kPerThread; ++i) {
    const int page = first + i;
    if (page < num_blocks) {
      const bool in_use = (used >> i) & 1;
      if (page == live) head[1] = live - u;           // u pages in use in front of the line
      if (page < live && !in_use) holes[page - u] = page;
      if (page >= live && in_use) { high[live - 1 - u] = page; rank[page] = live - 1 - u; }
      u += in_use;
    }
  }
}
__global__ void __launch_bounds__(kCopyThreads) move_pages_kernel(uint4* cache, int page_pieces, int32_t* block_table, const int32_t* seqlens,
                                                                  int32_t* refs, int B, int num_blocks, int width, const int* head, const int* holes,
                                                                  const int* high, const int* rank) {
  begin();
  const int live = head[0], moves = head[1], segments = (page_pieces + kSegment - 1) / kSegment;
  // (the i-th hole takes the i-th page behind the line, which is the last but i of `high`)
  const long long work = static_cast<long long>(moves) * segments;
  for (long long w = blockIdx.x; w < work; w += gridDim.x) {
    const int m = static_cast<int>(w / segments), seg = static_cast<int>(w - static_cast<long long>(m) * segments);
    const int src_page = high[moves - 1 - m], dst_page = holes[m];
    const uint4* src = cache + static_cast<size_t>(src_page) * page_pieces + seg * kSegment + threadIdx.x;
    uint4* dst = cache + static_cast<size_t>(dst_page) * page_pieces + seg * kSegment + threadIdx.x;
    const int left = page_pieces - seg * kSegment - threadIdx.x;
    uint4 x[kCopyUnroll];
#pragma unroll
    for (int u = 0; u < kCopyUnroll; ++u) if (u * kCopyThreads < left) x[u] = src[u * kCopyThreads];
#pragma unroll
    for (int u = 0; u < kCopyUnroll; ++u) if (u * kCopyThreads < left) dst[u * kCopyThreads] = x[u];
    if (seg == 0 && threadIdx.x == 0) { refs[dst_page] = refs[src_page]; refs[src_page] = 0; }
  }
  if (moves == 0) return;
  const long long entries = static_cast<long long>(B) * width;
  for (long long e = static_cast<long long>(blockIdx.x) * kCopyThreads + threadIdx.x; e < entries; e += static_cast<long long>(gridDim.x) * kCopyThreads) {
    const int row = static_cast<int>(e / width), i = static_cast<int>(e - static_cast<long long>(row) * width);
    if (i >= pages_of(length_of(seqlens, row, width))) continue;
    const int page = block_table[e];
    if (page < live || page >= num_blocks) continue;
    const int r = rank[page];                         // (a page without references has no rank: the table and the counts disagree)
    if (r >= 0 && r < moves && high[r] == page) block_table[e] = holes[moves - 1 - r];
  }
}

// Pages src[i] -> dst[i]; a pair with a page outside the cache is skipped.
__global__ void __launch_bounds__(kCopyThreads) copy_pages_kernel(uint4* cache, int page_pieces, int num_blocks, const int32_t* src, const int32_t* dst,
                                                                  int segments) {
  begin();
  const int m = blockIdx.x / segments, seg = blockIdx.x - m * segments;
  const int s = src[m], d = dst[m];
  if (s < 0 || s >= num_blocks || d < 0 || d >= num_blocks || s == d) return;
  const uint4* from = cache + static_cast<size_t>(s) * page_pieces + seg * kSegment + threadIdx.x;
  uint4* to = cache + static_cast<size_t>(d) * page_pieces + seg * kSegment + threadIdx.x;
  const int left = page_pieces - seg * kSegment - threadIdx.x;
  uint4 x[kCopyUnroll];
#pragma unroll
  for (int u = 0; u < kCopyUnroll; ++u) if (u * kCopyThreads < left) x[u] = from[u * kCopyThreads];
#pragma unroll
  for (int u = 0; u < kCopyUnroll; ++u) if (u * kCopyThreads < left) to[u * kCopyThreads] = x[u];
}

template <typename... Params, typename... Args>
cudaError_t launch(void (*kern)(Params...), dim3 grid, int threads, cudaStream_t stream, Args... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kern, static_cast<Params>(args)...);
}
int done(cudaError_t err) {
  if (err == cudaSuccess) return AMLA_OK;
  cudaGetLastError();
  return AMLA_ERR_CUDA;
}

constexpr int kMaxPages = 1 << 28;                    // every list index and chunk fits 32 bits

int check_cache(const void* cache, long long page_bytes, int num_blocks) {
  if (!cache || num_blocks <= 0 || page_bytes <= 0 || page_bytes % 16 != 0 || (reinterpret_cast<uintptr_t>(cache) & 15)) return AMLA_ERR_INVALID_ARG;
  return num_blocks > kMaxPages || page_bytes > (1ll << 30) ? AMLA_ERR_UNSUPPORTED : AMLA_OK;
}
int check_books(const int32_t* block_table, const int32_t* seqlens, const int32_t* refs, int B, int num_blocks, int width) {
  if (!block_table || !seqlens || !refs || B <= 0 || num_blocks <= 0 || width <= 0) return AMLA_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(block_table) | reinterpret_cast<uintptr_t>(seqlens) | reinterpret_cast<uintptr_t>(refs)) & 3) return AMLA_ERR_INVALID_ARG;
  if (num_blocks > kMaxPages || static_cast<long long>(width) * kPage > (1ll << 30) || B > (1 << 24)) return AMLA_ERR_UNSUPPORTED;
  return AMLA_OK;
}
int check_workspace(const void* workspace, size_t bytes, int num_blocks, int rows) {
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & (kAlign - 1))) return AMLA_ERR_INVALID_ARG;
  return bytes < scratch_bytes(num_blocks, rows) ? AMLA_ERR_WORKSPACE : AMLA_OK;
}
bool overlap(const int32_t* a, const int32_t* b, int n) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b), bytes = sizeof(int32_t) * static_cast<uintptr_t>(n);
  return a != nullptr && x < y + bytes && y < x + bytes;
}
bool odd_int(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3) != 0; }

cudaError_t list_free(const int32_t* refs, int num_blocks, long long most, const Requests& q, const Scratch& s, cudaStream_t stream) {
  const int chunks = chunks_of(num_blocks);
  if (chunks > 1) {
    const cudaError_t err = launch(count_pages_kernel<false>, dim3(chunks), kScanThreads, stream, refs, num_blocks, s.totals);
    if (err != cudaSuccess) return err;
  }
  return launch(list_free_kernel, dim3(chunks + 1), kScanThreads, stream, refs, num_blocks, s.totals, static_cast<int>(std::min<long long>(most, num_blocks)), s.head, s.list, q,
                s.row_rank);
}

}  // namespace

}  // namespace amla

using namespace amla;

extern "C" int amla_pages_workspace_size(int num_blocks, int B, size_t* bytes_out) {
  if (!bytes_out || num_blocks <= 0 || B <= 0) return AMLA_ERR_INVALID_ARG;
  if (num_blocks > kMaxPages || B > (1 << 24)) return AMLA_ERR_UNSUPPORTED;
  *bytes_out = scratch_bytes(num_blocks, B);
  return AMLA_OK;
}

extern "C" int amla_pages_copy(void* cache, long long page_bytes, int num_blocks, const int32_t* src, const int32_t* dst, int n, void* cuda_stream) {
  const int rc = check_cache(cache, page_bytes, num_blocks);
  if (rc != AMLA_OK) return rc;
  if (n < 0 || (n > 0 && (!src || !dst)) || odd_int(src) || odd_int(dst)) return AMLA_ERR_INVALID_ARG;
  if (n == 0) return AMLA_OK;
  const int pieces = static_cast<int>(page_bytes / 16), segments = (pieces + kSegment - 1) / kSegment;
  if (static_cast<long long>(n) * segments > 0x7fffffffll) return AMLA_ERR_UNSUPPORTED;
  return done(launch(copy_pages_kernel, dim3(n * segments), kCopyThreads, static_cast<cudaStream_t>(cuda_stream), static_cast<uint4*>(cache), pieces, num_blocks, src, dst, segments));
}

extern "C" int amla_pages_free(int32_t* block_table, int32_t* seqlens, int32_t* refs, const int32_t* rows, int n, int B, int num_blocks, int max_blocks_per_seq, void* cuda_stream) {
  const int rc = check_books(block_table, seqlens, refs, B, num_blocks, max_blocks_per_seq);
  if (rc != AMLA_OK) return rc;
  if (n < 0 || (n > 0 && !rows) || odd_int(rows)) return AMLA_ERR_INVALID_ARG;
  if (n == 0) return AMLA_OK;
  return done(launch(free_rows_kernel, dim3(n), kRowThreads, static_cast<cudaStream_t>(cuda_stream), block_table, seqlens, refs, rows, B, num_blocks, max_blocks_per_seq));
}

extern "C" int amla_pages_fork(void* cache, long long page_bytes, int32_t* block_table, int32_t* seqlens, int32_t* refs, const int32_t* parents, const int32_t* children, int n, int B,
                               int num_blocks, int max_blocks_per_seq, int32_t* served, void* workspace, size_t workspace_bytes, void* cuda_stream) {
  int rc = check_cache(cache, page_bytes, num_blocks);
  if (rc == AMLA_OK) rc = check_books(block_table, seqlens, refs, B, num_blocks, max_blocks_per_seq);
  if (rc != AMLA_OK) return rc;
  if (n < 0 || n > B || (n > 0 && (!parents || !children)) || odd_int(parents) || odd_int(children) || odd_int(served)) return AMLA_ERR_INVALID_ARG;
  if (n == 0) return AMLA_OK;
  rc = check_workspace(workspace, workspace_bytes, num_blocks, B);
  if (rc != AMLA_OK) return rc;
  const Scratch s = carve(workspace, num_blocks);
  cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  const Requests q{seqlens, parents, children, nullptr, n, B, max_blocks_per_seq};
  const cudaError_t err = list_free(refs, num_blocks, n, q, s, stream);
  if (err != cudaSuccess) return done(err);
  const int pieces = static_cast<int>(page_bytes / 16), segments = std::min((pieces + kSegment - 1) / kSegment, 65535);
  return done(launch(fork_rows_kernel, dim3(n, segments), kCopyThreads, stream, static_cast<uint4*>(cache), pieces, block_table, seqlens, refs, q, num_blocks, s.head,
                     s.list, s.row_rank, served));
}

extern "C" int amla_pages_reserve(int32_t* block_table, int32_t* seqlens, int32_t* refs, const int32_t* new_lens, int B, int num_blocks, int max_blocks_per_seq, int32_t* granted,
                                  void* workspace, size_t workspace_bytes, void* cuda_stream) {
  int rc = check_books(block_table, seqlens, refs, B, num_blocks, max_blocks_per_seq);
  if (rc != AMLA_OK) return rc;
  if (!new_lens || odd_int(new_lens) || odd_int(granted)) return AMLA_ERR_INVALID_ARG;
  // (a row is served by one thread, or block: what it writes must not be what another one still reads)
  if (overlap(new_lens, seqlens, B)) return AMLA_ERR_INVALID_ARG;
  rc = check_workspace(workspace, workspace_bytes, num_blocks, B);
  if (rc != AMLA_OK) return rc;
  if (overlap(granted, seqlens, B) || (granted != new_lens && overlap(granted, new_lens, B))) return AMLA_ERR_INVALID_ARG;
  cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  const Requests q{seqlens, nullptr, nullptr, new_lens, B, B, max_blocks_per_seq};
  if (chunks_of(num_blocks) == 1) return done(launch(reserve_small_kernel, dim3(1), kScanThreads, stream, block_table, seqlens, refs, num_blocks, q, granted));
  const Scratch s = carve(workspace, num_blocks);
  const cudaError_t err = list_free(refs, num_blocks, static_cast<long long>(B) * max_blocks_per_seq, q, s, stream);
  if (err != cudaSuccess) return done(err);
  return done(launch(reserve_rows_kernel, dim3(B), kRowThreads, stream, block_table, seqlens, refs, q, s.list, s.row_rank, granted));
}

extern "C" int amla_pages_compact(void* cache, long long page_bytes, int32_t* block_table, const int32_t* seqlens, int32_t* refs, int B, int num_blocks, int max_blocks_per_seq, int32_t* live,
                                  void* workspace, size_t workspace_bytes, void* cuda_stream) {
  int rc = check_cache(cache, page_bytes, num_blocks);
  if (rc == AMLA_OK) rc = check_books(block_table, seqlens, refs, B, num_blocks, max_blocks_per_seq);
  if (rc != AMLA_OK) return rc;
  if (odd_int(live)) return AMLA_ERR_INVALID_ARG;
  rc = check_workspace(workspace, workspace_bytes, num_blocks, B);
  if (rc != AMLA_OK) return rc;
  const Scratch s = carve(workspace, num_blocks);
  cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  const int chunks = chunks_of(num_blocks);
  cudaError_t err = cudaSuccess;
  if (chunks > 1) err = launch(count_pages_kernel<true>, dim3(chunks), kScanThreads, stream, refs, num_blocks, s.totals);
  if (err != cudaSuccess) return done(err);
  err = launch(list_moves_kernel, dim3(chunks), kScanThreads, stream, refs, num_blocks, s.totals, s.head, s.list, s.list2, s.rank, live);
  if (err != cudaSuccess) return done(err);
  const int pieces = static_cast<int>(page_bytes / 16), segments = (pieces + kSegment - 1) / kSegment;
  const long long most = std::max<long long>(static_cast<long long>(num_blocks / 2 + 1) * segments, (static_cast<long long>(B) * max_blocks_per_seq + kCopyThreads - 1) / kCopyThreads);
  return done(launch(move_pages_kernel, dim3(static_cast<int>(std::min<long long>(most, kMoveBlocks))), kCopyThreads, stream, static_cast<uint4*>(cache), pieces, block_table, seqlens, refs, B,
                     num_blocks, max_blocks_per_seq, s.head, s.list, s.list2, s.rank));
}
