// Which pages of a long context a query token attends to: scores from the pages' means, and the choice.
//
// scores: l[h,p] = scale q_h . mean_p (products of bf16 on the tensor cores, FP32 sums), score[p] = sum_h 2^(l[h,p] - lse_h), lse_h over all pages p in front of the
// token's own.  A head's lse needs all of its pages before any share of it is known: blocks of a cluster keep their logits in tensor memory until they have
// exchanged a maximum and a sum for each row, so that every mean is read once and no logit is written.  (Logits by way of memory, two launches:
// 32 x 65536 keys 23 us, 15.5 this way.  A sum of heads, not a maximum, because all heads attend to what is selected.)
// What bounds it, 32 x 65536 keys of 128 heads, 15.4 us, 26 K clk a block: 2.5 K until the length is there; the first means 4.5 K later; then 37.7 MB of means at
// 6.4 TB/s until 16.5 K; statistics 2.8 K and shares 2.9 K (2 K each are exponentials, sixteen a clock), exchange 1.4 K, sums 1.9 K.  Short contexts (8 x 1.5-4 K, 16 heads) take 6.9 us, a
// launch and that chain; long ragged ones (12 x 9-262 K, two tokens, 25.4 us) wait for the longest sequences, which come first where not all clusters have room (26.9 in order, by clusters
// of four; 24 x 9-262 K 40.3 -> 34.1; with smaller clusters it is of no use: 120 x 1-65 K 36.2 in order, 39.4 the longest first).
// One lane a scheduler is all that a loading warp gets, so that every address is at hand before the loop (1200 -> 350 clk for an operand place of a short context).
// Tried: Q kept in shared memory beside a ring of 64 KB (a third of the bytes under way: 16.4 us, 45.7 for the long ragged ones); 16 summing warps (16.1); shares of the last
// tile kept from the first pass over its logits (0.5 less, 1.5 more for the long ragged ones).
//
// select: a block for a query token; in a sparse call one of the scoring's cluster (32 x 8-65 K keys 48.8 -> 48.2 us, and 2 us of host time), where there are no scores if all pages are kept anyway
// (32 x 0.2-3 K keys of 128 heads, 64 pages kept: 35.7 -> 28.5 us; 2 x 300 of 16 heads 19.4 -> 12.3).  By itself 4.5 us for 512 pages, 10.8 for 16 K: a launch, the length, the scores, and two or three times eight bits of their order; code that
// runs once, which rolled loops of 256 threads do in less time than unrolled ones of 1024 (up to 2048 pages).
#include <climits>
#include <type_traits>

#include "../../include/amla.h"
#include "amla_fp4.cuh"
#include "amla_host.cuh"
#include "amla_select.cuh"
#include "amla_sm100.cuh"
#include "amla_tokens.cuh"

namespace amla {

using namespace sm100;

namespace {

__device__ __forceinline__ int seen_by(const int32_t* seqlens, int b, int Sq, int t, int width) {
  const long long n = seqlens[b] < static_cast<long long>(width) * kPage ? seqlens[b] : width * kPage;
  return n - Sq + t + 1 > 0 ? static_cast<int>(n - Sq + t + 1) : 0;
}
// pages in front of the one that holds the token's own position
__device__ __forceinline__ int candidates(int seen) { return seen > 0 ? (seen - 1) / kPage : 0; }

// Selection, by a block.
constexpr int kHeldPages = 24576;                              // up to so many pages a row's scores, as their order, and what is chosen of them are kept in shared memory

// A number's place in the order of scores: larger for larger ones, the same for both zeros, that of -infinity for a NaN.
__device__ __forceinline__ uint32_t order_of(float f) {
  if (f != f) return 0x007fffffu;
  const uint32_t u = __float_as_uint(f + 0.f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

template <int kSelectThreads>
struct __align__(16) SelectScratch {
  int counts[4][256];                                          // a table for each of the four times, the largest eight bits first
  int4 found;                                                  // the next eight bits, how many are wanted of those that have them, how many there are
  int2 totals[kSelectThreads / 32];
  uint2 kinds[kSelectThreads];                                 // of 32 pages each: which are taken anyway, and which agree
  __device__ __forceinline__ void clear() {
    for (int i = threadIdx.x; i < 1024; i += kSelectThreads) (&counts[0][0])[i] = 0;
  }
};

// The choice for query token `row` = b * Sq + t, which sees `seen` keys.  The scores' order is looked at eight bits at a time, from the top: how many of those that
// agree with the bits found so far have which next eight; the one that is looked for lies in one of these 256, and if all of those are wanted the bits suffice.
// kHeld: held_keys [width] has the order of the row's scores (written by these threads), and room for [keep] positions behind it.  sm is clear.
template <int kSelectThreads, bool kHeld>
__device__ __forceinline__ void select_row(const SelectParams& p, int row, int seen, uint32_t* held_keys, SelectScratch<kSelectThreads>& sm) {
  const int tid = threadIdx.x, wid = tid >> 5, lane = tid & 31, count = (seen + kPage - 1) / kPage;
  const float* scores = p.scores + static_cast<size_t>(row) * p.width;
  const int32_t* entries = p.block_table + static_cast<size_t>(row / p.Sq) * p.width;
  int32_t* table = p.table + static_cast<size_t>(row) * p.keep;
  int32_t* chosen = p.chosen ? p.chosen + static_cast<size_t>(row) * p.keep : nullptr;
  const int kept = min(count, p.keep);
  for (int i = kept + tid; i < p.keep; i += kSelectThreads) {
    table[i] = -1;
    if (chosen) chosen[i] = -1;
  }
  if (tid == 0) p.lens[row] = seen - (count - kept) * kPage;
  if (count <= p.keep) {
    for (int i = tid; i < count; i += kSelectThreads) {
      table[i] = entries[i];
      if (chosen) chosen[i] = i;
    }
    return;
  }
  const int first = p.sink, end = count - p.recent;            // the others; more than are wanted
  auto key = [&](int i) { return kHeld ? held_keys[i] : order_of(scores[i]); };
  int left = p.keep - p.sink - p.recent, shift = 32;           // wanted of those that agree in the bits from `shift` on
  uint32_t prefix = 0;
  __syncthreads();
  if (left > 0) {
    int there;
    do {
      shift -= 8;
      int* const table_of = sm.counts[shift >> 3];
#pragma unroll 1
      for (int i = first + tid; i < end; i += kSelectThreads) {
        const uint32_t k = key(i);
        if (shift == 24 || (k ^ prefix) >> (shift + 8) == 0) atomicAdd(&table_of[~(k >> shift) & 255], 1);
      }
      __syncthreads();
      if (wid == 0) {                                          // lane 0 has the largest eight
        const int4 a = *reinterpret_cast<const int4*>(table_of + 8 * lane), c = *reinterpret_cast<const int4*>(table_of + 8 * lane + 4);
        const int mine[8] = {a.x, a.y, a.z, a.w, c.x, c.y, c.z, c.w}, sum = ((a.x + a.y) + (a.z + a.w)) + ((c.x + c.y) + (c.z + c.w));
        int above = sum;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) { const int x = __shfl_up_sync(0xffffffffu, above, o); if (lane >= o) above += x; }
        above -= sum;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          if (above < left && left <= above + mine[i]) sm.found = make_int4(255 - 8 * lane - i, left - above, mine[i], 0);
          above += mine[i];
        }
      }
      __syncthreads();
      prefix |= static_cast<uint32_t>(sm.found.x) << shift;
      left = sm.found.y;
      there = sm.found.z;
    } while (shift > 0 && left < there);
  } else {
    shift = 0;
    prefix = 0xfffffffeu;                                      // above every score, below the pages that are taken anyway
  }
  prefix >>= shift;
  // Those above, and the first `left` of those that agree.  A warp notes for 32 neighbouring pages which are what, as bits; then a thread has 32 pages.
  int* const list = kHeld ? reinterpret_cast<int*>(held_keys + p.width) : nullptr;
  int2 front = make_int2(0, 0);                                // of the pages before these
  for (int page0 = 0; page0 < count; page0 += 32 * kSelectThreads) {
    const int pieces = min((count - page0 + 31) / 32, kSelectThreads);
#pragma unroll 1
    for (int c = wid; c < pieces; c += kSelectThreads / 32) {
      const int i = page0 + 32 * c + lane;
      const uint32_t k = i >= count ? 0u : i < first || i >= end ? 0xffffffffu : key(i) >> shift;      // (what is behind the last page may agree, and is not among the first)
      const uint32_t take = __ballot_sync(0xffffffffu, k > prefix), same = __ballot_sync(0xffffffffu, k == prefix);
      if (lane == 0) sm.kinds[c] = make_uint2(take, same);
    }
    __syncthreads();
    const uint2 mine = tid < pieces ? sm.kinds[tid] : make_uint2(0, 0);
    int2 n = make_int2(__popc(mine.x), __popc(mine.y));
    const int2 own = n;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int x = __shfl_up_sync(0xffffffffu, n.x, o), y = __shfl_up_sync(0xffffffffu, n.y, o);
      if (lane >= o) { n.x += x; n.y += y; }
    }
    if (lane == 31) sm.totals[wid] = n;
    __syncthreads();
    const int2 all = lane < kSelectThreads / 32 ? sm.totals[lane] : make_int2(0, 0);
    int2 others = lane < wid ? all : make_int2(0, 0);          // of the warps in front
#pragma unroll
    for (int o = 16; o; o >>= 1) { others.x += __shfl_xor_sync(0xffffffffu, others.x, o); others.y += __shfl_xor_sync(0xffffffffu, others.y, o); }
    n.x += front.x + others.x - own.x;
    n.y += front.y + others.y - own.y;
#pragma unroll 1
    for (uint32_t bits = mine.x | (n.y < left ? mine.y : 0u); bits; bits &= bits - 1) {
      const int at = __ffs(bits) - 1, same = n.y + __popc(mine.y & ((1u << at) - 1)), to = n.x + __popc(mine.x & ((1u << at) - 1)) + min(same, left);
      const int page = page0 + 32 * tid + at;
      if ((!(mine.x >> at & 1) && same >= left) || static_cast<uint32_t>(to) >= static_cast<uint32_t>(p.keep)) continue;      // (no more than `keep`, should the scores change meanwhile)
      if (kHeld) {
        list[to] = page;
      } else {
        table[to] = entries[page];
        if (chosen) chosen[to] = page;
      }
    }
    if (page0 + 32 * kSelectThreads < count) {
      front.x += __reduce_add_sync(0xffffffffu, all.x);
      front.y += __reduce_add_sync(0xffffffffu, all.y);
    }
    __syncthreads();
  }
  if (kHeld) {
    for (int i = tid; i < p.keep; i += kSelectThreads) {
      const int page = min(static_cast<uint32_t>(list[i]), static_cast<uint32_t>(p.width - 1));         // (of a page, whatever a scoring that gave up has left)
      table[i] = entries[page];
      if (chosen) chosen[i] = page;
    }
  }
}

// Scores.  An item is some query tokens of a sequence, as many as have 128 rows (a row: a head) between them; a cluster of up to sixteen blocks has an item,
// a block a share of its pages.  It multiplies the rows by its pages' means, up to 256 pages at a time (a tile), keeps the logits of the
// last two tiles in tensor memory, sends what it knows of every row (maximum and sum) to the others of the cluster and, with what they know,
// makes shares of attention of its logits and adds them up over the heads.  Of more than two tiles the earlier ones are multiplied again.
constexpr int kTileRows = 128, kTilePages = 256, kMostBlocks = 16;
constexpr int kLoadWarps = 4, kLoadThreads = 32 * kLoadWarps, kSumWarps = 8, kSumThreads = 32 * kSumWarps, kMmaWarp = kLoadWarps + kSumWarps;
constexpr int kThreads = 32 * (kMmaWarp + 1);
constexpr int kPart = 64;                                     // pages that a thread has in hand at a time
constexpr int kMostStages = 9, kChunks = kDqk / 64;           // places of the ring, each for 64 of the 576 columns of either operand
constexpr uint32_t kQBytes = kTileRows * 128;                 // rows of 128 B, 128-byte swizzle
// Shared memory: the ring, in which a block of up to two tiles adds up its shares when all products are done ([128 rows][256 pages]); with more tiles the ring
// is shorter and has [128 rows][128 pages] behind it.  Rows are 16 bytes longer than a multiple of 128: no two lanes of a store meet in a bank.  The others'
// statistics come in at the end, which is no place of the ring, and have been read when shares are added up.
constexpr uint32_t kWorkBytes = 227328, kStatsBytes = kMostBlocks * kTileRows * 8, kFewBytes = kTileRows * (kTilePages / 2 + 4) * 4;
constexpr uint32_t kOffStats = kWorkBytes - kStatsBytes, kOffKnown = kWorkBytes, kOffLse = kOffKnown + kTileRows * 8;
constexpr uint32_t kOffHalves = kOffLse + kTileRows * 4, kOffBars = kOffHalves + kTilePages / 2 * 4, kScoreSmem = kOffBars + 256;
// Behind the barriers: which sequence a block has, where the longest come first (a word of its own: a warp may read it late, when others are far ahead), whether a peer's statistics were
// late, and the address of tensor memory.
constexpr uint32_t kOffFound = kOffBars + 256 - 16, kOffLate = kOffFound + 4;
enum { X_FULL = 0, X_EMPTY = kMostStages, X_DONE = 2 * kMostStages, X_FREE = X_DONE + 2, X_STATS = X_FREE + 2, X_GIVE_UP, X_NUM };
constexpr uint32_t kOffScratch = kWorkBytes - sizeof(SelectScratch<kThreads>);
static_assert(2 * kHeldPages * 4 <= kOffScratch && kOffScratch % 16 == 0, "selection");
static_assert(8 * X_NUM + 16 <= 256 && kScoreSmem <= 232448 && kWorkBytes % 1024 == 0, "shared memory");
static_assert(kTileRows * (kTilePages + 4) * 4 <= kOffStats && kStatsBytes <= kFewBytes && (kWorkBytes - kFewBytes) / (kQBytes + kTilePages * 128) >= 3, "ring");

__host__ __device__ __forceinline__ int tokens_of_item(int Sq, int H) { return Sq < kTileRows / H ? Sq : kTileRows / H; }

// (maximum, sum of 2^(logit - maximum)) of two sets of logits together
__device__ __forceinline__ float2 join(float2 a, float2 b) {
  const float top = max_nan(a.x, b.x), off = top == -INFINITY ? 0.f : top;
  return make_float2(top, a.y * ex2_approx(a.x - off) + b.y * ex2_approx(b.x - off));
}
template <int kBar, int kCount>
__device__ __forceinline__ void meet() { asm volatile("bar.sync %0, %1;" ::"n"(kBar), "n"(kCount) : "memory"); }

__device__ const uint4 zero_row[kDqk / 8] = {};

}  // namespace

__global__ void __launch_bounds__(kThreads, 1) page_scores_kernel(const ScoreParams p, int blocks, int longest_first, const SelectParams select) {
  extern __shared__ __align__(1024) uint8_t smem[];
  const int tid = threadIdx.x, wid = tid >> 5, lane = tid & 31;
  const int tokens_most = tokens_of_item(p.Sq, p.H), items = (p.Sq + tokens_most - 1) / tokens_most;
  const int rank = blockIdx.x % blocks, item = blockIdx.x / blocks % items;
  int b = blockIdx.x / blocks / items;
  const int t0 = item * tokens_most, tokens = min(p.Sq - t0, tokens_most), rows = tokens * p.H;
  const uint32_t base = smem_u32(smem), bars = base + kOffBars, tmem_slot = bars + 256 - 8;
  auto bar = [&](int i) { return bars + 8u * i; };
  int* const late = reinterpret_cast<int*>(smem + kOffLate);   // (the same for all threads behind the barrier at the end)
  if (tid == 0) {
    *late = 0;
    for (int i = 0; i < kMostStages; ++i) { mbar_init(bar(X_FULL + i), kLoadThreads); mbar_init(bar(X_EMPTY + i), 1); }
    for (int i = 0; i < 2; ++i) { mbar_init(bar(X_DONE + i), 1); mbar_init(bar(X_FREE + i), kSumWarps); }
    mbar_init(bar(X_STATS), 1);
    mbar_init(bar(X_GIVE_UP), 1);
    fence_mbar_init();
    mbar_arrive_expect_tx(bar(X_STATS), blocks * kTileRows * 8);
  }
  if (wid == kMmaWarp) { tmem_alloc(tmem_slot, 2 * kTilePages); tmem_relinquish(); }
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  cluster_arrive_relaxed();
  const uint32_t tmem = ld_shared_b32(tmem_slot);
  behind_the_kernel_in_front();
  if (blockIdx.x == 0 && tid == 0) *p.status = kStatusOk;
  if (longest_first) {                                         // the b-th longest sequence, of up to as many as there are threads
    int4* lens = reinterpret_cast<int4*>(smem);
    int* found = reinterpret_cast<int*>(smem + kOffFound);
    const int mine = tid < p.B ? ldg_here(p.seqlens + tid) : INT_MIN;
    reinterpret_cast<int*>(lens)[tid] = mine;
    __syncthreads();
    int before = 0;
    for (int i = 0; i < (p.B + 3) / 4; ++i) {
      const int4 l = lens[i];
      before += (l.x > mine || (l.x == mine && 4 * i < tid)) + (l.y > mine || (l.y == mine && 4 * i + 1 < tid)) + (l.z > mine || (l.z == mine && 4 * i + 2 < tid)) +
                (l.w > mine || (l.w == mine && 4 * i + 3 < tid));
    }
    if (tid < p.B && before == b) *found = tid;
    __syncthreads();
    b = *found;
  }

  // (in a sparse call that leaves none of the sequence's pages out there is nothing to score)
  const int seen = seen_by(p.seqlens, b, p.Sq, t0 + tokens - 1, p.width);
  const int most = select.table != nullptr && seen <= select.keep * static_cast<long long>(kPage) ? 0 : candidates(seen);
  const bool work = most > 0 || select.table == nullptr;
  const int share = ((most + blocks - 1) / blocks + 15) / 16 * 16, page0 = min(rank * share, most), here = min(share, most - page0);
  const int tiles = (here + kTilePages - 1) / kTilePages, again = max(tiles - 2, 0);
  // the k-th tile to be multiplied: all of them, then those that have left tensor memory, backwards
  auto tile_of = [&](int k) { return k < tiles ? k : tiles - 3 - (k - tiles); };
  const uint32_t place_bytes = kQBytes + (min(here, kTilePages) + 15) / 16 * 2048;
  const uint32_t stages = min((kWorkBytes - (again ? kFewBytes : kStatsBytes)) / place_bytes, static_cast<uint32_t>(kMostStages));
  cluster_wait();
  bool ok = (base & 1023u) == 0;                               // (the swizzled tiles assume a 1024-byte aligned window)

  if (!work) {
  } else if (wid < kLoadWarps) {
    // a thread brings 16 bytes of every 16th row of either operand (rows that there are not: whatever is there, in rows of the result that nobody reads)
    const int j = tid & 7, r0 = tid >> 3;
    const uint32_t dst = base + sw128_offset(r0, j);           // (16 rows further on the swizzle is the same)
    const __nv_bfloat16* q = p.q + ((static_cast<size_t>(b) * p.Sq + t0) * p.H + r0) * kDqk + 8 * j;
    const int rows_here = rows - r0;
    uint32_t place = 0, par = 1;
#pragma unroll 1
    for (int k = 0; k < tiles + again && ok; ++k) {
      const int first = tile_of(k) * kTilePages, n = (min(here - first, kTilePages) + 15) / 16 * 16;
      const uint4* from[kTilePages / 16];                      // (a page outside the cache: zeros)
#pragma unroll
      for (int i = 0; i < kTilePages / 16; ++i) {
        const int at = first + r0 + 16 * i, page = at < here ? p.block_table[static_cast<size_t>(b) * p.width + page0 + at] : -1;
        from[i] = (page >= 0 && page < p.num_blocks ? reinterpret_cast<const uint4*>(p.means) + static_cast<size_t>(page) * (kDqk / 8) : zero_row) + j;
      }
#pragma unroll
      for (int c = 0; c < kChunks; ++c) {                      // (unrolled, so that an address is one that is at hand and a constant: a scheduler has one of these warps)
        ok = ok && mbar_wait(bar(X_EMPTY + place), par);
        if (!ok) break;
        const uint32_t to = dst + place * place_bytes;
#pragma unroll
        for (int i = 0; i < kTileRows / 16; ++i)
          if (16 * i < rows_here) cp_async_16(to + 2048 * i, q + 16 * i * kDqk + 64 * c);
#pragma unroll
        for (int i = 0; i < kTilePages / 16; ++i)
          if (16 * i < n) cp_async_16(to + kQBytes + 2048 * i, from[i] + 8 * c);
        cp_async_arrive(bar(X_FULL + place));
        if (++place == stages) { place = 0; par ^= 1; }
      }
    }
    cp_async_wait_all();
  } else if (wid == kMmaWarp) {
    if (elect_one()) {
      constexpr uint32_t hi = smem_desc_hi_sw128(1024);
      uint32_t place = 0, par = 0, used[2] = {0, 0};
#pragma unroll 1
      for (int k = 0; k < tiles + again && ok; ++k) {
        const int tile = tile_of(k), n = (min(here - tile * kTilePages, kTilePages) + 15) / 16 * 16;
        const uint32_t idesc = make_idesc_bf16(kTileRows, 16, false, false) + (static_cast<uint32_t>(n / 8 - 2) << 17), buf = tile & 1, d = tmem + kTilePages * buf;
        if (used[buf] > 0) ok = mbar_wait(bar(X_FREE + buf), (used[buf] - 1) & 1);
        if (!ok) break;
        ++used[buf];
        tc_fence_after_sync();
#pragma unroll 1
        for (int c = 0; c < kChunks; ++c) {
          ok = mbar_wait(bar(X_FULL + place), par);
          if (!ok) break;
          fence_proxy_async_smem();                            // the copies are ordinary writes
          const uint32_t a = smem_desc_lo(base + place * place_bytes, 16), m = smem_desc_lo(base + place * place_bytes + kQBytes, 16);
#pragma unroll
          for (int kk = 0; kk < 4; ++kk) mma_ss(d, smem_desc_join(a + 2 * kk, hi), smem_desc_join(m + 2 * kk, hi), idesc, (c | kk) != 0 ? 1u : 0u);
          mma_commit(bar(X_EMPTY + place));
          if (++place == stages) { place = 0; par ^= 1; }
        }
        if (ok) mma_commit(bar(X_DONE + buf));
      }
      // What has been issued ends before tensor memory is given back, also where those who add it up have given up on it.
      if (!ok) {
        mma_commit(bar(X_GIVE_UP));
        mbar_wait(bar(X_GIVE_UP), 0);
      }
#pragma unroll
      for (int i = 0; i < 2; ++i)
        if (ok && used[i] > 0) ok = mbar_wait(bar(X_DONE + i), (used[i] - 1) & 1);
    }
    __syncwarp();
  } else {
    // a thread has a row and 128 of a tile's pages, 64 at a time; when shares are added up, a page and half of the rows
    const int quarter = wid & 3, half = (wid - kLoadWarps) >> 2, mine = (wid - kLoadWarps) * 32 + lane, row = 32 * quarter + lane;
    const int token = min(row / p.H, tokens - 1), count = row < rows ? min(candidates(seen_by(p.seqlens, b, p.Sq, t0 + token, p.width)) - page0, here) : 0;
    float* const out = p.scores + (static_cast<size_t>(b) * p.Sq + t0) * p.width;
    for (int k = 0; k < tokens && select.table == nullptr; ++k)                    // pages that are not scored (the selection reads none of them)
      for (int i = candidates(seen_by(p.seqlens, b, p.Sq, t0 + k, p.width)) + rank * kSumThreads + mine; i < p.width; i += blocks * kSumThreads) out[static_cast<size_t>(k) * p.width + i] = 0.f;
    const uint32_t lanes = tmem + (static_cast<uint32_t>(32 * quarter) << 16) + kTilePages / 2 * half;
    auto logits = [&](int tile, int part, uint32_t (&v)[2][32]) {
      const uint32_t at = lanes + kTilePages * (tile & 1) + part;
      tmem_ld_32x32b_x32(at, v[0]);
      tmem_ld_32x32b_x32(at + 32, v[1]);
      tmem_wait_ld();
    };
    // (a comparison and a choice for every logit take as long as half of its exponential: only where a row of the warp does not have all 64 pages)
    auto for_all_or_some = [&](int left, auto body) {
      if (__all_sync(0xffffffffu, left >= kPart || row >= rows)) body(std::false_type{}); else body(std::true_type{});
    };
    const uint64_t scale2 = pack_f32x2(p.scale_log2, p.scale_log2);
    uint32_t done[2] = {0, 0};
    auto wait_for = [&](int tile) {
      const uint32_t buf = tile & 1;
      ok = ok && mbar_wait(bar(X_DONE + buf), done[buf] & 1);
      ok = __all_sync(0xffffffffu, ok);
      ++done[buf];
      tc_fence_after_sync();
    };
    auto give_back = [&](int tile) {
      tc_fence_before_sync();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(X_FREE + (tile & 1)));
    };
    float2 known = make_float2(-INFINITY, 0.f);
#pragma unroll 1
    for (int tile = 0; tile < tiles && ok; ++tile) {
      wait_for(tile);
      if (!ok) break;
#pragma unroll 1
      for (int part = 0; part < kTilePages / 2; part += kPart) {
        const int first = tile * kTilePages + kTilePages / 2 * half + part;
        if (first >= here) break;
        uint32_t v[2][32];
        logits(tile, part, v);
        const int left = count - first;
        for_all_or_some(left, [&](auto some) {
          constexpr bool kSome = decltype(some)::value;
          // (the maximum of those that are numbers: one that is not makes the sum one)
          float2 more = make_float2(-INFINITY, 0.f);
          float tops[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
          for (int i = 0; i < kPart; i += 2) {
            float x, y;
            unpack_f32x2(mul_f32x2(pack_f32x2(__uint_as_float(v[i >> 5][i & 31]), __uint_as_float(v[i >> 5][(i & 31) + 1])), scale2), x, y);
            if (kSome) {
              if (i >= left) x = -INFINITY;
              if (i + 1 >= left) y = -INFINITY;
            }
            v[i >> 5][i & 31] = __float_as_uint(x);
            v[i >> 5][(i & 31) + 1] = __float_as_uint(y);
            tops[i / 2 & 3] = fmax3(tops[i / 2 & 3], x, y);
          }
          more.x = fmaxf(fmax3(tops[0], tops[1], tops[2]), tops[3]);
          const float off = more.x == -INFINITY ? 0.f : more.x;
          const uint64_t off2 = pack_f32x2(-off, -off);
          uint64_t sums[2] = {0, 0};
#pragma unroll
          for (int i = 0; i < kPart; i += 2) {
            float x, y;
            unpack_f32x2(add_f32x2(pack_f32x2(__uint_as_float(v[i >> 5][i & 31]), __uint_as_float(v[i >> 5][(i & 31) + 1])), off2), x, y);
            sums[i / 2 & 1] = add_f32x2(sums[i / 2 & 1], pack_f32x2(ex2_approx(x), ex2_approx(y)));
          }
          float x, y;
          unpack_f32x2(add_f32x2(sums[0], sums[1]), x, y);
          more.y = x + y;
          known = join(known, more);
        });
      }
      if (tile < again) give_back(tile);
    }
    float2* both = reinterpret_cast<float2*>(smem + kOffKnown);
    float2* stats = reinterpret_cast<float2*>(smem + kOffStats);
    float* lse = reinterpret_cast<float*>(smem + kOffLse);
    if (half == 1) both[row] = known;
    meet<1, kSumThreads>();
    if (half == 0) {
      known = join(known, both[row]);
      const uint32_t at = base + kOffStats + (rank * kTileRows + row) * 8;
      for (int i = 0; i < blocks; ++i) st_async_v2(map_to_cta(at, i), __float_as_uint(known.x), __float_as_uint(known.y), map_to_cta(bar(X_STATS), i));
      const bool told = mbar_wait<true>(bar(X_STATS), 0);
      ok = __all_sync(0xffffffffu, told && ok);
      if (!told) *late = 1;
      float2 all = stats[row];
      for (int i = 1; i < blocks; ++i) all = join(all, stats[i * kTileRows + row]);
      lse[row] = all.x + log2f(all.y);
    }
    meet<1, kSumThreads>();
    const uint64_t off2 = pack_f32x2(-lse[row], -lse[row]);
    // a round: all of a tile's pages where there is room, else 64 of either half
    const int rounds = again ? 2 : 1, wide = kTilePages / rounds, stride = wide + 4;
    float* const shares = reinterpret_cast<float*>(smem + (again ? kWorkBytes - kFewBytes : 0));
    float* const halves = reinterpret_cast<float*>(smem + kOffHalves);
    const int column = mine % wide, side = mine / wide;
#pragma unroll 1
    for (int tile = tiles - 1; tile >= 0; --tile) {
      if (tile < again) wait_for(tile);
#pragma unroll 1
      for (int round = 0; round < rounds; ++round) {
#pragma unroll 1
        for (int part = round * kPart; part < (rounds == 1 ? kTilePages / 2 : (round + 1) * kPart); part += kPart) {
          const int first = tile * kTilePages + kTilePages / 2 * half + part, left = count - first;
          if (first >= here || !ok) break;
          float* to = shares + row * stride + wide / 2 * half + (rounds == 1 ? part : 0);
          uint32_t v[2][32];
          logits(tile, part, v);
          for_all_or_some(left, [&](auto some) {
            constexpr bool kSome = decltype(some)::value;
#pragma unroll
            for (int i = 0; i < kPart; i += 4) {
              float e[4];
#pragma unroll
              for (int k = 0; k < 4; k += 2) {
                unpack_f32x2(fma_f32x2(pack_f32x2(__uint_as_float(v[i >> 5][(i & 31) + k]), __uint_as_float(v[i >> 5][(i & 31) + k + 1])), scale2, off2), e[k], e[k + 1]);
                e[k] = !kSome || i + k < left ? ex2_approx(e[k]) : 0.f;
                e[k + 1] = !kSome || i + k + 1 < left ? ex2_approx(e[k + 1]) : 0.f;
              }
              *reinterpret_cast<float4*>(to + i) = make_float4(e[0], e[1], e[2], e[3]);
            }
          });
        }
        meet<1, kSumThreads>();
        // (of a round of two halves of 64 pages, the second is 128 pages further on)
        const int at = tile * kTilePages + (rounds == 1 ? column : round * kPart + column + (column >= kPart ? kPart : 0));
        const float* const from = shares + column;
        auto sum = [&](int r, int end) {
          float s[4] = {0.f, 0.f, 0.f, 0.f};
          for (; r + 16 <= end; r += 16) {
#pragma unroll
            for (int i = 0; i < 16; ++i) s[i & 3] += from[(r + i) * stride];
          }
          for (; r < end; ++r) s[0] += from[r * stride];
          return (s[0] + s[1]) + (s[2] + s[3]);
        };
        if (rounds == 1) {
          if (at < here)
            for (int k = 0; k < tokens; ++k) out[static_cast<size_t>(k) * p.width + page0 + at] = sum(k * p.H, (k + 1) * p.H);
        } else if (tokens == 1) {
          const int middle = (p.H + 1) / 2;
          const float s = side == 0 ? sum(0, middle) : sum(middle, p.H);
          if (side == 1) halves[column] = s;
          meet<1, kSumThreads>();
          if (side == 0 && at < here) out[page0 + at] = s + halves[column];
        } else {
          for (int k = side; k < tokens; k += 2) {
            const float s = sum(k * p.H, (k + 1) * p.H);
            if (at < here) out[static_cast<size_t>(k) * p.width + page0 + at] = s;
          }
        }
        if (tile > 0 || round + 1 < rounds) meet<1, kSumThreads>();
      }
      if (tile >= 2) give_back(tile);
    }
  }
  if (!ok) atomicExch(p.status, kStatusTimeout);
  tc_fence_before_sync();
  __syncthreads();
  if (wid == kMmaWarp) tmem_dealloc(tmem, 2 * kTilePages);
  // The choice, by a block of the cluster for each of the tokens: behind the cluster's barrier all of its scores are there, and nobody writes to another's shared memory any more.
  auto& scratch = *reinterpret_cast<SelectScratch<kThreads>*>(smem + kOffScratch);
  uint32_t* held_keys = reinterpret_cast<uint32_t*>(smem);
  if (*late) {                                                 // (this block has given up on what a peer sends before it comes to the barrier: it must not be gone, nor use the place, before that is in)
    cluster_arrive();
    cluster_wait();
    mbar_wait<true>(bar(X_STATS), 0);
    if (select.table == nullptr) return;
    scratch.clear();
  } else if (select.table == nullptr) {
    cluster_arrive_relaxed();                                  // (who gave up must not be gone when another's statistics arrive)
    cluster_wait();
    return;
  } else {
    scratch.clear();
    cluster_arrive();
    cluster_wait();
  }
#pragma unroll 1
  for (int k = rank; k < tokens; k += blocks) {
    const int row = b * p.Sq + t0 + k, sees = seen_by(p.seqlens, b, p.Sq, t0 + k, p.width), scored = work ? candidates(sees) : 0;
    for (int i = tid; i < scored; i += kThreads) held_keys[i] = order_of(p.scores[static_cast<size_t>(row) * p.width + i]);
    select_row<kThreads, true>(select, row, sees, held_keys, scratch);
    if (k + blocks < tokens) {
      __syncthreads();
      scratch.clear();
    }
  }
}

// A block, a query token.
template <int kSelectThreads, bool kHeld>
__global__ void __launch_bounds__(kSelectThreads) pages_select_kernel(const SelectParams p) {
  extern __shared__ uint32_t held_keys[];
  __shared__ SelectScratch<kSelectThreads> scratch;
  const int row = blockIdx.x;
  scratch.clear();
  behind_the_kernel_in_front();
  const int seen = seen_by(p.seqlens, row / p.Sq, p.Sq, row % p.Sq, p.width);
  if (kHeld && p.width > p.keep) {                             // (all of the row, since the length is on its way)
    const float* scores = p.scores + static_cast<size_t>(row) * p.width;
#pragma unroll 4
    for (int i = threadIdx.x; i < p.width; i += kSelectThreads) held_keys[i] = order_of(scores[i]);
  }
  if (p.clear && row == 0 && threadIdx.x == 0) *p.clear = kStatusOk;
  select_row<kSelectThreads, kHeld>(p, row, seen, held_keys, scratch);
}

namespace {

cudaLaunchConfig_t score_config(int clusters, int blocks, cudaStream_t stream, cudaLaunchAttribute (&attr)[2]) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(clusters * blocks);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = kScoreSmem;
  cfg.stream = stream;
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = blocks;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cfg;
}

// How many clusters of sixteen blocks the current device has room for (a property of it, looked up once).
int clusters_of_16() {
  static std::atomic<int> known[64];                           // one more than the number
  int device = 0;
  if (cudaGetDevice(&device) != cudaSuccess) { cudaGetLastError(); return 0; }
  std::atomic<int>& k = known[device & 63];
  if (k.load(std::memory_order_acquire) == 0) {
    int n = 0;
    cudaLaunchAttribute attr[2];
    const cudaLaunchConfig_t cfg = score_config(1, 16, nullptr, attr);
    if (cudaFuncSetAttribute(page_scores_kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess || cudaOccupancyMaxActiveClusters(&n, page_scores_kernel, &cfg) != cudaSuccess) {
      cudaGetLastError();
      n = 0;
    }
    k.store(n + 1, std::memory_order_release);
  }
  return k.load(std::memory_order_acquire) - 1;
}

// Blocks in a cluster: as many as there are SMs for, as long as a block has more than 32 pages of the table's width; more than that where a block would else have more than
// two tiles (which are multiplied twice), the longest sequences first then; and sixteen only where blocks of eight would have more than a tile and all clusters have room at once.
// By the table's width, since lengths are not known on the host: in one far wider than its sequences each of them gets a cluster for sequences as long as the table (at 1024 and from 2049 pages, us:
// 128 x 16384 keys 23.7 and 107, against 17.4 in a table of 256; 64 x 1-65 K 21 and 54; 32 x 65536 15.4 and 33.5; 8 x 1.5-4 K of 16 heads 7.0 and 7.0).
// Measured (blocks 1 / 2 / 4 / 8 / 16, us): 32 x 65536 keys 38.3 / 20.7 / 15.7 / 31.2; 128 x 16384 17.9 / 23.8 / 36.6 / 77.3; 64 x 1-65 K 38.5 / 21.2 / 25.6 / 45.5; 16 x 65536 of two
// tokens 35.4 / 18.4 / 12.9 / 28.1; 1 x 262144 100 / 52 / 28 / 14.4 / 10.8; 8 x 262144, of whose clusters of sixteen seven have room, - / - / - / 20.6 / 27.8; 24 x 262144 - / 79.0 /
// 46.4 / 44.7; 60 x 131072 - / 50.5 / 48.5 / 61.9; 120 x 65536 - / 49.5 / 61.1 / 85.8.
int score_blocks(int items, int width, int sms) {
  int blocks = 1;
  while (blocks < 8 && width > 64 * blocks && (static_cast<long long>(items) * 2 * blocks <= sms || width > 2 * kTilePages * blocks)) blocks *= 2;
  if (blocks == 8 && width > 8 * kTilePages && items <= sms / 16 && items <= clusters_of_16()) blocks = 16;
  return blocks;
}

}  // namespace

cudaError_t launch_page_scores(const ScoreParams& p, const SelectParams* select, int sms, cudaStream_t stream) {
  static std::atomic<uint64_t> done{0};
  const int items = p.B * ((p.Sq + tokens_of_item(p.Sq, p.H) - 1) / tokens_of_item(p.Sq, p.H));
  const cudaError_t err = allow_shared(page_scores_kernel, done, kScoreSmem);
  if (err != cudaSuccess) return err;
  const int blocks = score_blocks(items, p.width, sms);
  cudaLaunchAttribute attr[2];
  const cudaLaunchConfig_t cfg = score_config(items, blocks, stream, attr);
  const int longest_first = blocks == 8 && items * 8 > sms && p.B <= kThreads;
  return cudaLaunchKernelEx(&cfg, page_scores_kernel, p, blocks, longest_first, select ? *select : SelectParams{});
}

namespace {

template <int kSelectThreads>
cudaError_t launch_select(const SelectParams& p, cudaStream_t stream) {
  static std::atomic<uint64_t> done{0};
  const cudaError_t err = allow_shared(pages_select_kernel<kSelectThreads, true>, done, 2 * kHeldPages * sizeof(uint32_t));
  if (err != cudaSuccess) return err;
  return launch_in_order(pages_select_kernel<kSelectThreads, true>, dim3(p.B * p.Sq), kSelectThreads, p.width <= p.keep ? 0 : (p.width + p.keep) * static_cast<uint32_t>(sizeof(uint32_t)),
                         stream, p);
}

}  // namespace

bool scores_select(int width) { return width <= kHeldPages; }

cudaError_t launch_pages_select(const SelectParams& p, cudaStream_t stream) {
  if (p.width > kHeldPages) return launch_in_order(pages_select_kernel<1024, false>, dim3(p.B * p.Sq), 1024, 0, stream, p);
  return p.width <= 2048 ? launch_select<256>(p, stream) : launch_select<1024>(p, stream);
}

}  // namespace amla
