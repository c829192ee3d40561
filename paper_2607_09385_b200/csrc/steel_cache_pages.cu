// Page management of the 4-bit cache, on the device: extend, fork, free, compact (include/steel_cache.h).
//
// Who owns what is decided by one cluster of eight CTAs, which can wait for one another: each checks the whole batch for itself and nothing
// is changed unless all of it is as it should be, so that a call either is done or changes nothing.  What another CTA of the cluster reads
// for its answer is changed behind a cluster barrier only: extend takes free pages, writes table entries and counts behind one and lengths
// behind another; fork takes down all rows (and counts them, by atomics that nobody reads) before it overwrites any, so that rows may be read and
// written by the same call; free checks all lengths before it changes any.  A page is free where refs is 0, and the lowest free pages are given out
// in the order of the batch, a lane a page: every result is fixed by the call's inputs, whatever the timing.  Bound by the latency of its dependent
// reads (slot -> length -> last page -> refs) and the barriers.  One CTA, without the barriers between CTAs, is no variant of its own: a fork of up to
// 512 table entries takes 3.7 us by one and 3.9 by eight, of 16384 24 to 32 and 6 to 7; extend for 8 sequences 5.5 and 5.6, for 256 10.1 and 7.0;
// free for 8 1.65 and 1.67, for 256 5.9 and 2.4; compaction's plan over 2048 pages 4.9 and 5.0, over 16384 8.3 and 5.4.
// Contents move in a kernel of their own on all SMs, bound by memory; it finds its list in scratch memory, and where nothing is to be
// moved (the usual extend) it returns at once.  (Movers in the same launch as extend's cluster, waiting for its list, saved a launch's 2.3 us
// of host time and cost 2 us on the device, which is what the steps wait for.)
#include <cooperative_groups.h>

#include "sm100_ptx.cuh"
#include "steel_cache.cuh"

namespace cg = cooperative_groups;

namespace steel {

namespace {

constexpr int kCtas = 8, kThreads = 512, kWarps = kThreads / 32;
constexpr int kMoveThreads = 256;

struct Move {
  int32_t src, dst, units, unused;  // the first `units` units of every head
};
// Scratch memory: a head of 128 bytes, then the moves and, for compact, the rank of each page that moves; for fork the rows.
struct ScratchHead {
  int32_t moves, live;
};
constexpr int64_t kScratchHead = 128;
__device__ Move *moves_of(void *scratch) { return reinterpret_cast<Move *>(static_cast<char *>(scratch) + kScratchHead); }

// Exclusive prefix sums over a CTA of one value a thread; `total` for everybody.
template <class T>
__device__ T block_exclusive(T value, T *warp_sums, T *total) {
  const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
  T inclusive = value;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const T below = __shfl_up_sync(0xffffffffu, inclusive, d);
    if (lane >= d) inclusive += below;
  }
  __syncthreads();  // warp_sums may still be read from the scan before
  if (lane == 31) warp_sums[warp] = inclusive;
  __syncthreads();
  T before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) {
    const T s = warp_sums[w];
    if (w < warp) before += s;
    all += s;
  }
  *total = all;
  return before + inclusive - value;
}

// A bit for each slot that a batch has named.  Cleared before the kernel waits for the one before it.
__device__ __forceinline__ void clear_seen(const CacheView &c, uint32_t *seen) {
  for (int i = threadIdx.x; i < (c.slots + 31) / 32; i += kThreads) seen[i] = 0;
  __syncthreads();
}
__device__ __forceinline__ bool named_before(uint32_t *seen, int slot) {
  return atomicOr(&seen[slot / 32], 1u << (slot % 32)) >> (slot % 32) & 1u;
}

// The words of this CTA's share of the pages: bit = page is free.  -> how many of its pages are.
struct Share {
  int begin, words;  // first page, words of 32 pages
};
__host__ __device__ int share_words(int pages) {
  return ((pages + 31) / 32 + kCtas - 1) / kCtas;
}
__device__ Share share_of(int pages, int rank) {
  const int words = (pages + 31) / 32, each = share_words(pages);
  const int first = min(words, rank * each);
  return {first * 32, min(words, first + each) - first};
}
__device__ void free_pages(const CacheView &c, Share s, uint32_t *free_bits, int warp, int warps) {
  const int lane = threadIdx.x % 32;
  constexpr int kUnroll = 8;
  for (int w0 = warp * kUnroll; w0 < s.words; w0 += warps * kUnroll) {
    int ref[kUnroll];
#pragma unroll
    for (int j = 0; j < kUnroll; ++j) {
      const int page = s.begin + (w0 + j) * 32 + lane;
      ref[j] = w0 + j < s.words && page < c.pages ? c.refs[page] : 1;
    }
#pragma unroll
    for (int j = 0; j < kUnroll; ++j) {
      const uint32_t bits = __ballot_sync(0xffffffffu, ref[j] == 0);
      if (lane == 0 && w0 + j < s.words) free_bits[w0 + j] = bits;
    }
  }
}

// Free pages before each word of the share, counted from its beginning; `total` in the share.
__device__ void rank_words(Share s, const uint32_t *bits, int *ranks, int *sums, int *total) {
  const int each = (s.words + kThreads - 1) / kThreads, w0 = min(s.words, int(threadIdx.x) * each), w1 = min(s.words, w0 + each);
  int mine = 0;
  for (int w = w0; w < w1; ++w) mine += __popc(bits[w]);
  int rank = block_exclusive(mine, sums, total);
  for (int w = w0; w < w1; ++w) {
    ranks[w] = rank;
    rank += __popc(bits[w]);
  }
}

// Values that the CTAs of the cluster tell one another.  -> those of the lower ranks added up; `total` of all.
__device__ int cluster_exclusive(cg::cluster_group &cluster, int *mine, int value, int *total) {
  if (threadIdx.x == 0) *mine = value;
  cluster.sync();
  int before = 0, all = 0;
  const int rank = cluster.block_rank();
#pragma unroll
  for (int r = 0; r < kCtas; ++r) {
    const int v = *cluster.map_shared_rank(mine, r);
    if (r < rank) before += v;
    all += v;
  }
  *total = all;
  return before;
}

__device__ __forceinline__ int pages_for(const CacheView &c, int tokens) {
  return (tokens + (1 << c.page_shift) - 1) >> c.page_shift;
}

// Each move takes `units` units of every head of every layer from one page to another; they are contiguous in a head.  A warp takes (move, layer,
// head) after (move, layer, head), with nine 16-byte reads a lane in flight: a page of 64 tokens at head_dim 128 is twice that.
__device__ __forceinline__ void move_units(const CacheView &c, const Move *moves, int n, int unit, int warp, int warps) {
  const int64_t head_bytes = int64_t(unit) << c.page_shift >> 4, jobs = int64_t(n) * c.layers * c.heads_kv;
  const int of_move = c.layers * c.heads_kv, lane = threadIdx.x % 32;
  for (int64_t job = warp; job < jobs; job += warps) {
    const int m = int(job / of_move), rest = int(job % of_move);
    const Move move = moves[m];
    unsigned char *at = c.pool + rest / c.heads_kv * c.layer_bytes + rest % c.heads_kv * head_bytes;
    const uint4 *from = reinterpret_cast<const uint4 *>(at + move.src * c.page_bytes);
    uint4 *to = reinterpret_cast<uint4 *>(at + move.dst * c.page_bytes);
    const int words = move.units * (unit / 16);
    constexpr int kUnroll = 9;
    for (int i = lane; i < words; i += 32 * kUnroll) {
      uint4 x[kUnroll];
#pragma unroll
      for (int j = 0; j < kUnroll; ++j)
        if (i + j * 32 < words) x[j] = from[i + j * 32];
#pragma unroll
      for (int j = 0; j < kUnroll; ++j)
        if (i + j * 32 < words) to[i + j * 32] = x[j];
    }
  }
}

// ------------------------------------------------------------------------------------------------------------- extend
// Shared memory: `before` [n + 1] pages wanted before sequence i, `first` [n] the first table column that gets a page (bit 31: the
// page that is there now is shared and copied), `copies` [n] copies before i, the bits of seen slots, the free bits and how many free pages
// of this CTA's share stand before each word of them.
__global__ void __cluster_dims__(kCtas, 1, 1) __launch_bounds__(kThreads)
    extend_kernel(CacheView c, CacheBatch b, void *scratch) {
  extern __shared__ uint32_t smem[];
  __shared__ int told, int_sums[kWarps];
  __shared__ long long sums[kWarps];
  cg::cluster_group cluster = cg::this_cluster();
  const int n = b.batch, tid = threadIdx.x;
  int *before = reinterpret_cast<int *>(smem), *copies = before + n + 1;
  uint32_t *first = reinterpret_cast<uint32_t *>(copies + n), *seen = first + n, *bits = seen + (c.slots + 31) / 32;
  int *ranks = reinterpret_cast<int *>(bits + share_words(c.pages));
  clear_seen(c, seen);
  grid_dependency_wait();
  grid_launch_dependents();

  // half of the warps look at the batch, the others at the pages: both are chains of reads
  constexpr int kBatchThreads = kThreads / 2;
  const Share share = share_of(c.pages, cluster.block_rank());
  const int each = (n + kBatchThreads - 1) / kBatchThreads, i0 = tid < kBatchThreads ? min(n, tid * each) : n, i1 = min(n, i0 + each);
  bool good = true;
  long long want = 0;  // pages in the low 40 bits, copies above
  if (tid < kBatchThreads) {
    const int most = max_tokens(c);
    for (int i = i0; i < i1; ++i) {
      const int s = slot_of(c, b.slots, i), count = b.counts[i];
      const int len = s < 0 ? -1 : c.lens[s];
      int pages = 0, copy = 0;
      if (len < 0 || count < 0 || len > most || count > most - len || named_before(seen, s)) {
        good = false;
      } else {
        const int held = pages_for(c, len);
        if (count > 0 && (len & ((1 << c.page_shift) - 1))) {
          const int last = c.table[int64_t(s) * c.max_pages + held - 1];
          if (last < 0 || last >= c.pages) good = false;
          else copy = c.refs[last] > 1;
        }
        pages = pages_for(c, len + count) - held + copy;
        first[i] = uint32_t(held - copy) | uint32_t(copy) << 31;
      }
      before[i] = pages;
      copies[i] = copy;
      want += pages + (static_cast<long long>(copy) << 40);
    }
  } else {
    free_pages(c, share, bits, tid / 32 - kBatchThreads / 32, kWarps - kBatchThreads / 32);
  }
  good = __syncthreads_and(good);
  long long all;
  long long run = block_exclusive(want, sums, &all);
  const long long wanted = all & ((1ll << 40) - 1);
  for (int i = i0; i < i1; ++i) {  // at most 2^20 pages where the call is done
    const int pages = before[i], copy = copies[i];
    before[i] = int(min(run & ((1ll << 40) - 1), 1ll << 30));
    copies[i] = int(run >> 40);
    run += pages + (static_cast<long long>(copy) << 40);
  }
  if (tid == 0) before[n] = int(min(wanted, 1ll << 30));

  int here;
  rank_words(share, bits, ranks, int_sums, &here);
  int free_total;
  const int below = cluster_exclusive(cluster, &told, here, &free_total);  // and the barrier between reads and writes
  // every CTA has read what it reads, and comes to the same answer
  const bool room = wanted <= free_total;
  if (good && room) {
    // a lane a page
    for (int w = tid / 32; w < share.words && below + ranks[w] < wanted; w += kWarps) {
      const uint32_t free_here = bits[w];
      const int rank = below + ranks[w] + __popc(free_here & ((1u << (tid % 32)) - 1u));
      if (!(free_here >> (tid % 32) & 1u) || rank >= wanted) continue;
      const int page = share.begin + w * 32 + tid % 32;
      int lo = 0, hi = n;  // the sequence: before[lo] <= rank < before[lo + 1]
      while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        (before[mid] <= rank ? lo : hi) = mid;
      }
      const int slot = b.slots ? b.slots[lo] : lo;
      const uint32_t f = first[lo];
      const int nth = rank - before[lo];
      int32_t *entry = c.table + int64_t(slot) * c.max_pages + int(f & 0x7fffffffu) + nth;
      if (nth == 0 && f >> 31) {
        const int old = *entry, tokens = c.lens[slot] & ((1 << c.page_shift) - 1);
        atomicSub(&c.refs[old], 1);
        moves_of(scratch)[copies[lo]] = Move{old, page, (tokens + kUnitTokens - 1) / kUnitTokens, 0};
      }
      *entry = page;
      c.refs[page] = 1;
    }
  }
  cluster.sync();  // lens are read above; and no CTA leaves while its `told` may be read
  if (cluster.block_rank() == 0) {
    if (good && room)
      for (int i = tid; i < n; i += kThreads) c.lens[b.slots ? b.slots[i] : i] += b.counts[i];
    if (tid == 0) {
      static_cast<ScratchHead *>(scratch)->moves = good && room ? int(all >> 40) : 0;
      if (!good) report(c.status, STEEL_ERR_INVALID_ARG);
      else if (!room) report(c.status, STEEL_ERR_NO_PAGES);
    }
  }
}

// ---------------------------------------------------------------------------------------------------------------- fork
__global__ void __cluster_dims__(kCtas, 1, 1) __launch_bounds__(kThreads)
    fork_kernel(CacheView c, void *scratch, int n, const int32_t *src, const int32_t *dst) {
  extern __shared__ uint32_t smem[];
  cg::cluster_group cluster = cg::this_cluster();
  clear_seen(c, smem);
  grid_dependency_wait();
  grid_launch_dependents();
  bool good = true;
  const int most = max_tokens(c);
  for (int i = threadIdx.x; i < n; i += kThreads) {
    const int s = slot_of(c, src, i), d = slot_of(c, dst, i);
    if (s < 0 || d < 0 || named_before(smem, d) || c.lens[s] < 0 || c.lens[s] > most || c.lens[d] < 0 || c.lens[d] > most) good = false;
  }
  good = __syncthreads_and(good);
  // rows are taken down, and counted, before any is overwritten; lengths beside them.  The warps share the sequences: `per` warps each.
  int32_t *rows = reinterpret_cast<int32_t *>(static_cast<char *>(scratch) + kScratchHead), *lens = rows + int64_t(n) * c.max_pages,
          *given_up = lens + n;
  constexpr int kAllWarps = kCtas * kWarps;
  const int warp = cluster.block_rank() * kWarps + threadIdx.x / 32, lane = threadIdx.x % 32, per = max(kAllWarps / n, 1),
            from = warp % per * 32 + lane, step = per * 32;
  bool bad_page = false;
  if (good) {
    for (int i = warp / per; i < n; i += kAllWarps / per) {
      const int len = c.lens[src[i]], held = pages_for(c, len), left = pages_for(c, c.lens[dst[i]]);
      const int32_t *taken = c.table + int64_t(src[i]) * c.max_pages, *old = c.table + int64_t(dst[i]) * c.max_pages;
      for (int j = from; j < held; j += step) {
        const int page = taken[j];
        rows[int64_t(i) * c.max_pages + j] = page;
        if (page >= 0 && page < c.pages) atomicAdd(&c.refs[page], 1);
        else bad_page = true;
      }
      for (int j = from; j < left; j += step) {
        const int page = old[j];
        if (page >= 0 && page < c.pages) atomicSub(&c.refs[page], 1);
        else bad_page = true;
      }
      if (from == 0) lens[i] = len, given_up[i] = left;
    }
  }
  if (bad_page) report(c.status, STEEL_ERR_INVALID_ARG);
  __threadfence();
  cluster.sync();
  if (good) {
    for (int i = warp / per; i < n; i += kAllWarps / per) {
      const int len = lens[i], held = pages_for(c, len), entries = max(held, given_up[i]);
      int32_t *to = c.table + int64_t(dst[i]) * c.max_pages;
      for (int j = from; j < entries; j += step) to[j] = j < held ? rows[int64_t(i) * c.max_pages + j] : -1;
      if (from == 0) c.lens[dst[i]] = len;  // no other sequence of the batch has this slot
    }
  } else if (cluster.block_rank() == 0 && threadIdx.x == 0) {
    report(c.status, STEEL_ERR_INVALID_ARG);
  }
}

// ---------------------------------------------------------------------------------------------------------------- free
__global__ void __cluster_dims__(kCtas, 1, 1) __launch_bounds__(kThreads) free_kernel(CacheView c, CacheBatch b) {
  extern __shared__ uint32_t smem[];
  cg::cluster_group cluster = cg::this_cluster();
  clear_seen(c, smem);
  grid_dependency_wait();
  grid_launch_dependents();
  const int n = b.batch, most = max_tokens(c);
  bool good = true;
  for (int i = threadIdx.x; i < n; i += kThreads) {
    const int s = slot_of(c, b.slots, i), keep = b.counts ? b.counts[i] : 0;
    if (s < 0 || keep < 0 || named_before(smem, s) || keep > c.lens[s] || c.lens[s] > most) good = false;
  }
  good = __syncthreads_and(good);
  cluster.sync();
  if (good) {
    bool bad_page = false;
    // a warp a sequence
    for (int i = cluster.block_rank() * kWarps + threadIdx.x / 32; i < n; i += kCtas * kWarps) {
      const int s = b.slots ? b.slots[i] : i, keep = b.counts ? b.counts[i] : 0, end = pages_for(c, c.lens[s]);
      int32_t *row = c.table + int64_t(s) * c.max_pages;
      for (int j = pages_for(c, keep) + threadIdx.x % 32; j < end; j += 32) {
        const int page = row[j];
        if (page >= 0 && page < c.pages) atomicSub(&c.refs[page], 1);
        else bad_page = true;
        row[j] = -1;
      }
      __syncwarp();
      if (threadIdx.x % 32 == 0) c.lens[s] = keep;
    }
    if (bad_page) report(c.status, STEEL_ERR_INVALID_ARG);
  } else if (cluster.block_rank() == 0 && threadIdx.x == 0) {
    report(c.status, STEEL_ERR_INVALID_ARG);
  }
}

// ------------------------------------------------------------------------------------------------------------- compact
// With `live` pages in use, the k-th free page below `live` is the k-th hole, the k-th page in use from `live` up the k-th
// mover; there are as many of the ones as of the others.  A hole's rank is the free pages before it; a mover's the pages in use before
// it less those below `live`.
__global__ void __cluster_dims__(kCtas, 1, 1) __launch_bounds__(kThreads)
    compact_kernel(CacheView c, void *scratch, int32_t *live_out) {
  extern __shared__ uint32_t bits[];
  int *ranks = reinterpret_cast<int *>(bits + share_words(c.pages));
  __shared__ int told, told_holes;
  __shared__ int sums[kWarps];
  cg::cluster_group cluster = cg::this_cluster();
  grid_dependency_wait();
  grid_launch_dependents();
  const int tid = threadIdx.x;
  const Share share = share_of(c.pages, cluster.block_rank());
  free_pages(c, share, bits, tid / 32, kWarps);
  __syncthreads();
  int here, free_total;
  rank_words(share, bits, ranks, sums, &here);
  const int below = cluster_exclusive(cluster, &told, here, &free_total);  // free pages before this CTA's; a barrier too
  const int live = c.pages - free_total;
  // holes: free pages below `live`.  One CTA has that page, or all of its pages are on one side.
  int holes_here = live <= share.begin ? 0 : here;
  const int in_share = live - share.begin;
  if (in_share > 0 && in_share < share.words * 32)
    holes_here = ranks[in_share / 32] + __popc(bits[in_share / 32] & ((1u << (in_share % 32)) - 1u));
  int holes;
  cluster_exclusive(cluster, &told_holes, holes_here, &holes);

  Move *moves = moves_of(scratch);
  int32_t *rank_of = reinterpret_cast<int32_t *>(moves + (c.pages + 1) / 2);
  for (int w = tid / 32; w < share.words; w += kWarps) {
    const uint32_t free_here = bits[w];
    const int page = share.begin + w * 32 + tid % 32, rank = below + ranks[w] + __popc(free_here & ((1u << (tid % 32)) - 1u));
    if (page >= c.pages) continue;
    if (free_here >> (tid % 32) & 1u) {
      if (page < live) moves[rank].dst = page;
    } else if (page >= live) {
      const int k = page - rank - (live - holes);  // pages in use before it, less those below `live`
      moves[k].src = page;
      moves[k].units = (1 << c.page_shift) / kUnitTokens;
      rank_of[page] = k;
    }
  }
  cluster.sync();  // no CTA leaves while another may read what it has told
  if (cluster.block_rank() == 0 && tid == 0) {
    static_cast<ScratchHead *>(scratch)->moves = holes;
    static_cast<ScratchHead *>(scratch)->live = live;
    if (live_out) *live_out = live;
  }
}

// Contents; for compact also counts and tables.
template <bool kCompact>
__global__ void __launch_bounds__(kMoveThreads) move_kernel(CacheView c, void *scratch, int unit) {
  grid_dependency_wait();
  grid_launch_dependents();
  const int listed = static_cast<const ScratchHead *>(scratch)->moves, live = static_cast<const ScratchHead *>(scratch)->live;
  if (listed == 0) return;
  const Move *moves = moves_of(scratch);
  move_units(c, moves, listed, unit, blockIdx.x * (kMoveThreads / 32) + threadIdx.x / 32, gridDim.x * (kMoveThreads / 32));
  if (!kCompact) return;
  const int32_t *rank_of = reinterpret_cast<const int32_t *>(moves + (c.pages + 1) / 2);
  const int stride = gridDim.x * kMoveThreads, id = blockIdx.x * kMoveThreads + threadIdx.x;
  for (int m = id; m < listed; m += stride) {
    const Move move = moves[m];
    c.refs[move.dst] = c.refs[move.src];
    c.refs[move.src] = 0;
  }
  for (int s = id / 32; s < c.slots; s += stride / 32) {  // a warp a slot
    const int held = min(pages_for(c, min(max(c.lens[s], 0), max_tokens(c))), c.max_pages);
    int32_t *row = c.table + int64_t(s) * c.max_pages;
    for (int j = threadIdx.x % 32; j < held; j += 32) {
      const int page = row[j];
      if (page >= 0 && page < live) continue;
      // a page that the table names and refs calls free has no place in the list: nothing has written its rank
      const int k = page >= 0 && page < c.pages ? rank_of[page] : -1;
      const Move move = k >= 0 && k < listed ? moves[k] : Move{-1, -1, 0, 0};
      if (page >= 0 && move.src == page) row[j] = move.dst;
      else report(c.status, STEEL_ERR_INVALID_ARG);
    }
  }
}

constexpr int kMaxSeenBytes = kMaxSlots / 8, kMaxBitsBytes = 2 * (kMaxCachePages / 8 / kCtas + 4);
int bits_bytes(int pages) { return 2 * 4 * share_words(pages); }  // and ranks
int seen_bytes(int slots) { return (slots + 31) / 32 * 4; }

}  // namespace

int64_t pages_scratch_bytes(int slots, int max_pages, int pages) {
  const int64_t fork = int64_t(slots) * (max_pages + 2) * 4, extend = int64_t(slots) * int64_t(sizeof(Move)),
                compact = (int64_t(pages) + 1) / 2 * int64_t(sizeof(Move)) + int64_t(pages) * 4;
  const int64_t most = fork > extend ? (fork > compact ? fork : compact) : (extend > compact ? extend : compact);
  return kScratchHead + (most + 127) / 128 * 128;
}

cudaError_t configure_pages() {
  return cudaFuncSetAttribute(extend_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                              (3 * kMaxSlots + 1) * 4 + kMaxSeenBytes + kMaxBitsBytes);
}

cudaError_t launch_extend(const CacheView &c, int head_dim, void *scratch, const CacheBatch &b, int sms, cudaStream_t stream) {
  const int smem = (3 * b.batch + 1) * 4 + seen_bytes(c.slots) + bits_bytes(c.pages);
  const cudaError_t e = launch_overlapping(extend_kernel, dim3(kCtas), dim3(kThreads), smem, stream, c, b, scratch);
  if (e != cudaSuccess) return e;
  return launch_overlapping(move_kernel<false>, dim3(sms * 2), dim3(kMoveThreads), 0, stream, c, scratch, unit_bytes(head_dim));
}

cudaError_t launch_fork(const CacheView &c, void *scratch, int n, const int32_t *src, const int32_t *dst, cudaStream_t stream) {
  return launch_overlapping(fork_kernel, dim3(kCtas), dim3(kThreads), seen_bytes(c.slots), stream, c, scratch, n, src, dst);
}

cudaError_t launch_free(const CacheView &c, const CacheBatch &b, cudaStream_t stream) {
  return launch_overlapping(free_kernel, dim3(kCtas), dim3(kThreads), seen_bytes(c.slots), stream, c, b);
}

cudaError_t launch_compact(const CacheView &c, int head_dim, void *scratch, int32_t *live, int sms, cudaStream_t stream) {
  const cudaError_t e = launch_overlapping(compact_kernel, dim3(kCtas), dim3(kThreads), bits_bytes(c.pages), stream, c, scratch, live);
  if (e != cudaSuccess) return e;
  return launch_overlapping(move_kernel<true>, dim3(sms * 8), dim3(kMoveThreads), 0, stream, c, scratch, unit_bytes(head_dim));
}

}  // namespace steel
