// Pages of a cache, kept on the device (sp_pages_*): reserve, fork, release, compact, and the copies that forks and compactions ask for.
//
// The state is one array, ref_counts, the number of block-table entries that hold a page; a page is free if it is 0.  There is no
// list of free pages whose order would depend on history: a call that takes pages reads the counts once, into a bit set
// (64 pages a word) and a sum per segment of kSegment pages, and the k-th page that it takes is the k-th free one.  That costs 4 bytes
// per page of the pool, but nothing orders one workgroup of the scan behind another, every workgroup of the
// second launch finds its pages by itself, and the result does not depend on timing.
//
// Launches: reserve and fork two (scan and plan; apply), compact three (scan; ranks; apply), each one on small pools; release and
// copy one.  All but the copy are bound by their chains of memory round trips, the copy by HBM.
#include "attn_tile.h"

namespace sp {

constexpr int kPageThreads = 256, kPageWaves = kPageThreads / 64;
constexpr int kSegment = 4096;              // pages per workgroup of the scan
constexpr int kSegWords = kSegment / 64;    // 64: one per lane

static __device__ __forceinline__ int lane_prefix(int x) { return wave_scan_incl(x); }
static __device__ __forceinline__ long lane_prefix(long x) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const long y = __shfl_up(x, d);
    if ((int)(threadIdx.x & 63) >= d) x += y;
  }
  return x;
}
// Inclusive sum over the workgroup's threads, and the sum of all; wave_sums: kPageWaves values in LDS.
template <typename T>
static __device__ __forceinline__ T block_prefix(T x, T *wave_sums, T *total) {
  const int w = threadIdx.x >> 6;
  const T incl = lane_prefix(x);
  __syncthreads();  // wave_sums may still be read
  if ((threadIdx.x & 63) == 63) wave_sums[w] = incl;
  __syncthreads();
  T before = 0, all = 0;
#pragma unroll
  for (int u = 0; u < kPageWaves; ++u) {
    before += u < w ? wave_sums[u] : 0;
    all += wave_sums[u];
  }
  *total = all;
  return before + incl;
}

__host__ __device__ __forceinline__ int pages_of(int tokens) { return tokens <= 0 ? 0 : (int)(((unsigned)tokens + kPage - 1) / kPage); }

struct PagesArgs {
  int32_t *refs, *table, *lens;
  const int32_t *written;  // or null: rows are written up to their length
  int num_pages, num_rows, max_pages, nseg;
  uint64_t *free_bits;  // [nseg * kSegWords]
  int32_t *seg_free;    // [nseg] free pages of a segment
  // reserve, fork
  const int32_t *a, *b;  // rows and new lengths; parents and children
  int n;
  int32_t *plan;   // [n + 1] pages that the entries before take
  int32_t *sizes;  // [n] fork: the parent's written tokens, -1 for a skipped entry; reserve: the row's pages to be, 0 for a skipped entry
  int32_t *shortfall, *copy_src, *copy_dst, *copy_rows;
  // compact
  int32_t *new_table, *new_refs, *move_src, *move_dst, *moved;
  int32_t *rank, *moved_refs;  // [num_pages] of holes and of pages that move; [num_pages / 2] counts of the latter
};

// Tokens of a row, none beyond what its table row holds.
static __device__ __forceinline__ int row_tokens(const PagesArgs &p, int row) {
  const long most = (long)p.max_pages * kPage;
  const int len = p.lens[row];
  return len < 0 ? 0 : len > most ? (int)most : len;
}

// Those of them that a fork takes over.  Pages behind them are the row's own: it is still to append there.
static __device__ __forceinline__ int forked_tokens(const PagesArgs &p, int row) {
  const int room = row_tokens(p, row);
  return p.written ? min(max(p.written[row], 0), room) : room;
}

enum { kCompact, kReserve, kFork };

// Workgroup s < nseg: the free pages of segment s.  Workgroup nseg: what every entry takes, and the sums of that before it.
template <int OP>
__global__ __launch_bounds__(kPageThreads) void pages_scan_kernel(PagesArgs p) {
  __shared__ int wave_sums[kPageWaves];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  if ((int)blockIdx.x < p.nseg) {
    constexpr int PER = kSegWords / kPageWaves;  // words of a wave
    const long base = (long)blockIdx.x * kSegment + w * (PER * 64) + lane;
    int refs[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) refs[i] = p.refs[min(base + 64 * i, p.num_pages - 1L)];  // no branch: each load would wait for the one before
    uint64_t mine = 0;
    int free_pages = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const uint64_t bits = __builtin_amdgcn_ballot_w64(refs[i] <= 0 && base + 64 * i < p.num_pages);
      free_pages += __builtin_popcountll(bits);
      if (lane == i) mine = bits;
    }
    if (lane < PER) p.free_bits[(long)blockIdx.x * kSegWords + w * PER + lane] = mine;
    if (lane == 0) wave_sums[w] = free_pages;
    __syncthreads();
    if (threadIdx.x == 0) {
      int sum = 0;
#pragma unroll
      for (int u = 0; u < kPageWaves; ++u) sum += wave_sums[u];
      p.seg_free[blockIdx.x] = sum;
    }
    return;
  }
  if constexpr (OP != kCompact) {
    __shared__ long long_sums[kPageWaves];
    long before = 0;  // what the entries take together may pass 32 bits: then it is more than any pool has, and is stored as the most
    for (long i0 = 0; i0 < p.n; i0 += kPageThreads) {
      const long i = i0 + threadIdx.x;
      long need = 0;
      if (i < p.n) {
        const int a = p.a[i], b = p.b[i];
        int size = OP == kFork ? -1 : 0;
        if (a >= 0 && a < p.num_rows) {
          if (OP == kFork) {
            if (b >= 0 && b < p.num_rows && p.lens[b] == 0) {
              size = forked_tokens(p, a);
              need = size % kPage != 0;
            }
          } else if (pages_of(b) <= p.max_pages) {
            size = pages_of(b);
            need = max(size - pages_of(row_tokens(p, a)), 0);
          }
        }
        p.sizes[i] = size;
      }
      long total;
      const long incl = block_prefix(need, long_sums, &total);
      if (i < p.n) p.plan[i + 1] = (int)min(before + incl, 0x7fffffffL);
      before += total;
    }
    if (threadIdx.x == 0) p.plan[0] = 0;
  }
}

// The free pages of 64 words, one per lane, that are number 0 .. m - 1 from some page on: take(k, page).  rank: number of the word's
// first one; page0: first page of lane 0's word.  A word at a time, a lane per page: a lane that went through its own word would
// skip the pages before number 0 one by one (64 entries of a few pages each: 55 us a pass of fork and reserve, 24 so).
template <typename Take>
static __device__ __forceinline__ void take_words(uint64_t bits, int rank, int page0, int m, Take take) {
  const int lane = threadIdx.x & 63, n = __builtin_popcountll(bits);
  for (uint64_t words = __builtin_amdgcn_ballot_w64(n > 0 && rank < m && rank + n > 0); words != 0; words &= words - 1) {
    const int l = __builtin_ctzll(words);
    const uint32_t lo = __builtin_amdgcn_readlane((uint32_t)bits, l), hi = __builtin_amdgcn_readlane((uint32_t)(bits >> 32), l);
    const int k = __builtin_amdgcn_readlane(rank, l) + __builtin_amdgcn_mbcnt_hi(hi, __builtin_amdgcn_mbcnt_lo(lo, 0));
    if (((lane < 32 ? lo >> lane : hi >> (lane - 32)) & 1) != 0 && k >= 0 && k < m) take(k, page0 + 64 * l + lane);
  }
}

// Which segments hold the pool's free pages number `first` and on.  seg_before[q]: free pages before segment s0 + q, for the
// kPageThreads segments from s0 on.
struct FreePages {
  int *wave_sums, *seg_before;  // LDS: kPageWaves and kPageThreads + 1 ints
  int s0, upto;                 // upto: free pages before segment s0 + kPageThreads

  // Segments from s on, of which `before` free pages lie before; by the whole workgroup.  c: seg_free of segment s + threadIdx.x, 0 behind the last.
  __device__ __forceinline__ void look(int s, int before, int c) {
    int total;
    const int incl = block_prefix(c, wave_sums, &total);  // nobody reads seg_before any more when its barriers are passed
    seg_before[threadIdx.x + 1] = before + incl;
    if (threadIdx.x == 0) seg_before[0] = before;
    __syncthreads();
    s0 = s;
    upto = before + total;
  }
  // take(k, page) for k = 0 .. m - 1: the page that is number first + k of the free ones; by the whole workgroup, any thread takes any.
  template <typename Take>
  __device__ __forceinline__ void take_pages(const PagesArgs &p, int first, int m, Take take) {
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    for (;;) {
      if (upto > first) {
        int lo = 0, hi = kPageThreads;  // the first of these segments that ends behind `first`
        while (lo < hi) {
          const int mid = (lo + hi) >> 1;
          if (seg_before[mid + 1] > first) hi = mid;
          else lo = mid + 1;
        }
        for (int q = lo + w; q < kPageThreads && s0 + q < p.nseg && seg_before[q] < first + m; q += kPageWaves) {
          const uint64_t bits = p.free_bits[(long)(s0 + q) * kSegWords + lane];
          const int mine = __builtin_popcountll(bits);
          take_words(bits, seg_before[q] + lane_prefix(mine) - mine - first, (s0 + q) * kSegment, m, take);
        }
      }
      const int next = s0 + kPageThreads;
      if (upto >= first + m || next >= p.nseg) return;  // uniform
      const int s = next + threadIdx.x;
      look(next, upto, s < p.nseg ? p.seg_free[s] : 0);
    }
  }
};

// One workgroup per entry.
template <int OP>
__global__ __launch_bounds__(kPageThreads) void pages_take_kernel(PagesArgs p) {
  __shared__ int wave_sums[kPageWaves], seg_before[kPageThreads + 1], s_old, s_page;
  const int i = blockIdx.x, a = p.a[i], b = p.b[i];
  const int first = p.plan[i], need = p.plan[i + 1] - first, wanted = p.plan[p.n], size = p.sizes[i];
  FreePages pool = {wave_sums, seg_before, 0, 0};
  pool.look(0, 0, (int)threadIdx.x < p.nseg ? p.seg_free[threadIdx.x] : 0);
  int all_free = pool.upto;
  if (p.nseg > kPageThreads) {
    int c = 0, more;
    for (int s = threadIdx.x + kPageThreads; s < p.nseg; s += kPageThreads) c += p.seg_free[s];
    block_prefix(c, wave_sums, &more);
    all_free += more;
  }
  const int missing = max(wanted - all_free, 0);
  if (i == 0 && threadIdx.x == 0) *p.shortfall = missing;
  if constexpr (OP == kReserve) {
    if (missing > 0 || size == 0) return;  // size > 0: a is a row of the table, and holds no more pages than b takes
    // The entry that raises the length takes the pages: of several for one row each takes different ones.
    if (threadIdx.x == 0) s_old = atomicMax(p.lens + a, b);
    __syncthreads();
    const int has = pages_of(s_old), m = min(size - has, need);
    if (m <= 0) return;
    int32_t *row = p.table + (long)a * p.max_pages + has;
    pool.take_pages(p, first, m, [&](int k, int page) __attribute__((always_inline)) {
      row[k] = page;
      p.refs[page] = 1;
    });
  } else {
    bool taken = missing == 0 && size >= 0;
    const int full = taken ? size / kPage : 0;
    const int32_t *from = p.table + (long)a * p.max_pages;
    int32_t *to = p.table + (long)b * p.max_pages;
    // the parent's first pages, the new page and the claim of the child in one round trip
    const int page0 = (int)threadIdx.x < full ? from[threadIdx.x] : -1;
    int old = 0;
    if (threadIdx.x == 0 && taken && size > 0) old = atomicCAS(p.lens + b, 0, size);
    const int last = threadIdx.x == 0 && taken && need > 0 ? from[full] : -1;
    if (taken && need > 0) pool.take_pages(p, first, 1, [&](int, int page) __attribute__((always_inline)) { s_page = page; });
    if (threadIdx.x == 0) s_old = old;
    __syncthreads();
    taken = taken && s_old == 0;
    if (threadIdx.x == 0) {
      const bool copy = taken && need > 0;
      if (copy) {
        to[full] = s_page;
        p.refs[s_page] = 1;
      }
      p.copy_src[i] = copy ? last : -1;
      p.copy_dst[i] = copy ? s_page : -1;
      p.copy_rows[i] = copy ? size % kPage : 0;
    }
    if (!taken) return;
    for (int c = threadIdx.x; c < full; c += kPageThreads) {
      const int page = c < kPageThreads ? page0 : from[c];
      to[c] = page;
      if (page >= 0 && page < p.num_pages) atomicAdd(p.refs + page, 1);
    }
  }
}

// Few entries on a small pool: scan, plan and entries in one workgroup, up to four entries a wave, so one launch instead of two.  Of several
// entries for one child the first is taken, and entries for one row get their room one after the other.
constexpr int kSmallWaves = 16, kSmallEntries = 64, kSmallPages = kSmallWaves * 1024, kSmallWidth = 1024;
constexpr int kSmallPer = kSmallPages / (64 * kSmallWaves);  // words of a wave, every kSmallWaves-th: small pools occupy all waves alike

// The counts of this wave's words, and their free pages to s_bits.
static __device__ __forceinline__ void small_scan(const PagesArgs &p, int lane, int w, int (&refs)[kSmallPer]) {
#pragma unroll
  for (int i = 0; i < kSmallPer; ++i) {
    refs[i] = 0;
    if (64 * kSmallWaves * i >= p.num_pages) continue;  // uniform
    refs[i] = p.refs[min(64 * (kSmallWaves * i + w) + lane, p.num_pages - 1)];
  }
}
static __device__ __forceinline__ void small_bits(const PagesArgs &p, int lane, int w, const int (&refs)[kSmallPer], uint64_t *s_bits) {
  uint64_t mine = 0;
#pragma unroll
  for (int i = 0; i < kSmallPer; ++i) {
    const uint64_t bits = __builtin_amdgcn_ballot_w64(refs[i] <= 0 && 64 * (kSmallWaves * i + w) + lane < p.num_pages);
    if (lane == i) mine = bits;
  }
  if (lane < kSmallPer) s_bits[kSmallWaves * lane + w] = mine;
}

template <int OP>
__global__ __launch_bounds__(64 * kSmallWaves) void pages_small_kernel(PagesArgs p) {
  constexpr int WORDS = kSmallWaves * kSmallPer, LANE = WORDS / 64;
  __shared__ uint64_t s_bits[WORDS];
  __shared__ int s_a[kSmallEntries], s_b[kSmallEntries], s_size[kSmallEntries], s_first[kSmallEntries + 1];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int refs[kSmallPer];
  small_scan(p, lane, w, refs);
  if (w == 0) {
    const bool mine = lane < p.n;
    const int a = mine ? p.a[lane] : -1, b = mine ? p.b[lane] : -1;
    const bool row = a >= 0 && a < p.num_rows, child = OP == kFork && row && b >= 0 && b < p.num_rows;
    const int tokens = !row ? 0 : OP == kFork ? forked_tokens(p, a) : row_tokens(p, a), child_len = child ? p.lens[b] : 1;
    int size = OP == kFork ? (child && child_len == 0 ? tokens : -1) : (row && pages_of(b) <= p.max_pages ? pages_of(b) : 0);
    int has = pages_of(tokens);
    for (int j = 0; j < p.n - 1; ++j) {  // entries before this one
      const int aj = __builtin_amdgcn_readlane(a, j), bj = __builtin_amdgcn_readlane(b, j), sj = __builtin_amdgcn_readlane(size, j);
      if (j >= lane) continue;
      if (OP == kFork && bj == b && sj > 0) size = -1;
      if (OP == kReserve && aj == a) has = max(has, sj);
    }
    const int need = OP == kFork ? (size > 0 && size % kPage != 0) : max(size - has, 0);
    const int incl = wave_scan_incl(need);  // entries of at most kSmallWidth pages: no overflow
    if (mine) {
      s_a[lane] = a;
      s_b[lane] = b;
      s_size[lane] = size;
      s_first[lane] = incl - need;
      if (lane == p.n - 1) s_first[p.n] = incl;
    }
  }
  small_bits(p, lane, w, refs, s_bits);
  __syncthreads();
  if (w >= p.n) return;
  // every wave by itself: its entries, and the free pages before each of the lane's words
  uint64_t bits[LANE];
  int before[LANE], all_free = 0;
#pragma unroll
  for (int i = 0; i < LANE; ++i) {
    bits[i] = s_bits[64 * i + lane];
    const int count = __builtin_popcountll(bits[i]), incl = wave_scan_incl(count);
    before[i] = all_free + incl - count;
    all_free += __builtin_amdgcn_readlane(incl, 63);
  }
  const int missing = max(s_first[p.n] - all_free, 0);
  if (w == 0 && lane == 0) *p.shortfall = missing;
  for (int e = w; e < p.n; e += kSmallWaves) {
    const int a = s_a[e], b = s_b[e], size = s_size[e], first = s_first[e], need = s_first[e + 1] - first;
    auto take_pages = [&](auto take) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < LANE; ++i) take_words(bits[i], before[i] - first, 64 * 64 * i, need, take);
    };
    if constexpr (OP == kReserve) {
      if (missing > 0 || size == 0) continue;
      if (lane == 0) atomicMax(p.lens + a, b);
      int32_t *row = p.table + (long)a * p.max_pages + size - need;
      take_pages([&](int k, int page) __attribute__((always_inline)) {
        row[k] = page;
        p.refs[page] = 1;
      });
    } else {
      const bool taken = missing == 0 && size >= 0;
      if (!(taken && need > 0) && lane == 0) {
        p.copy_src[e] = p.copy_dst[e] = -1;
        p.copy_rows[e] = 0;
      }
      if (!taken || size == 0) continue;
      const int32_t *from = p.table + (long)a * p.max_pages;
      int32_t *to = p.table + (long)b * p.max_pages;
      const int full = size / kPage;
      if (lane == 0) p.lens[b] = size;
      take_pages([&](int, int page) __attribute__((always_inline)) {
        p.copy_src[e] = from[full];
        p.copy_dst[e] = page;
        p.copy_rows[e] = size % kPage;
        to[full] = page;
        p.refs[page] = 1;
      });
      for (int c = lane; c < full; c += 64) {
        const int page = from[c];
        to[c] = page;
        if (page >= 0 && page < p.num_pages) atomicAdd(p.refs + page, 1);
      }
    }
  }
}

// One workgroup per entry.  Lowering the length claims the pages behind it, so of several entries for one row each gives back
// different ones.
__global__ __launch_bounds__(kPageThreads) void pages_release_kernel(PagesArgs p, const int32_t *keep_lens) {
  __shared__ int s_old;
  const int row = p.a[blockIdx.x], keep = keep_lens ? max(keep_lens[blockIdx.x], 0) : 0;
  if (row < 0 || row >= p.num_rows) return;
  int32_t *entries = p.table + (long)row * p.max_pages;
  const int c0 = (int)min((long)pages_of(keep) + threadIdx.x, (long)p.max_pages);
  const int page0 = c0 < p.max_pages ? entries[c0] : -1;  // in the same round trip as the claim
  if (threadIdx.x == 0) s_old = atomicMin(p.lens + row, keep);
  __syncthreads();
  const int end = min(pages_of(s_old), p.max_pages);
  for (int c = c0; c < end; c += kPageThreads) {
    const int page = c == c0 ? page0 : entries[c];
    entries[c] = -1;
    if (page >= 0 && page < p.num_pages) atomicSub(p.refs + page, 1);
  }
}

// Compaction, second launch: where the pages in use from U on go.  With M free pages below U, a free page below U has as many free
// ones before it as its rank says, and a page in use from U on has its rank plus U - M pages in use before it.
__global__ __launch_bounds__(kPageThreads) void pages_rank_kernel(PagesArgs p) {
  __shared__ int wave_sums[kPageWaves], s_before[kSegWords], s_seg[2];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, seg = blockIdx.x;
  const uint64_t my_bits = p.free_bits[(long)seg * kSegWords + lane];
  constexpr int PER = kSegWords / kPageWaves;
  int refs[PER];  // requested first: inside the loop below every count would be waited for by itself (a pool of 4138 pages 7.9 us)
#pragma unroll
  for (int i = 0; i < PER; ++i) refs[i] = p.refs[min((long)seg * kSegment + 64 * (w + i * kPageWaves) + lane, p.num_pages - 1L)];
  int sum = 0, below = 0, total_free, before_seg;
  for (int s = threadIdx.x; s < p.nseg; s += kPageThreads) {
    const int c = p.seg_free[s];
    sum += c;
    below += s < seg ? c : 0;
  }
  block_prefix(sum, wave_sums, &total_free);
  block_prefix(below, wave_sums, &before_seg);
  const int used = p.num_pages - total_free, useg = used / kSegment;
  // M: free pages below U
  below = 0;
  for (int s = threadIdx.x; s < useg; s += kPageThreads) below += p.seg_free[s];
  if (useg < p.nseg && (int)threadIdx.x < kSegWords) {
    const uint64_t bits = p.free_bits[(long)useg * kSegWords + threadIdx.x];
    const int n = min(max(used - useg * kSegment - 64 * (int)threadIdx.x, 0), 64);  // its pages below U
    below += __builtin_popcountll(n == 64 ? bits : bits & ((1ull << n) - 1));
  }
  int holes;
  block_prefix(below, wave_sums, &holes);
  if (seg == 0 && threadIdx.x == 0) {
    p.moved[0] = holes;
    p.moved[1] = used;
  }
  if (holes == 0) return;
  if (w == 0) {
    const int c = __builtin_popcountll(my_bits);
    s_before[lane] = before_seg + lane_prefix(c) - c;
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int k = w + i * kPageWaves;
    const long page = (long)seg * kSegment + 64 * k + lane;
    const uint64_t bits = __shfl(my_bits, k);  // by all lanes
    if (page >= p.num_pages) continue;
    const int free_before = s_before[k] + __builtin_popcountll(bits & ((1ull << lane) - 1));
    const bool is_free = (bits >> lane) & 1;
    if (is_free && page < used) {
      p.move_dst[free_before] = (int)page;
      p.rank[page] = free_before;
    } else if (!is_free && page >= used) {
      const int r = (int)page - free_before - (used - holes);
      p.move_src[r] = (int)page;
      p.rank[page] = r;
      p.moved_refs[r] = refs[i];
    }
  }
}

// Compaction of a small pool with a small table in one launch: what the three do, in one workgroup.  New counts and entries are written
// when all old ones have been read, as both may be the table's own arrays.
constexpr int kSmallTable = 16 * 1024;  // entries

__global__ __launch_bounds__(64 * kSmallWaves) void pages_compact_small_kernel(PagesArgs p) {
  constexpr int PER = kSmallPer, WORDS = kSmallWaves * PER, LANE = WORDS / 64;
  __shared__ uint64_t s_bits[WORDS];
  __shared__ int s_before[WORDS];                      // free pages before a word
  __shared__ int s_refs[kSmallPages / 2];              // of the i-th page that moves: its count,
  __shared__ uint16_t s_dst[kSmallPages / 2];          // and where it goes
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int entries = p.num_rows * p.max_pages;  // at most kSmallTable
  int refs[PER], entry[kSmallTable / (64 * kSmallWaves)], len[kSmallTable / (64 * kSmallWaves)];
  small_scan(p, lane, w, refs);
#pragma unroll
  for (int i = 0; i < kSmallTable / (64 * kSmallWaves); ++i) {
    const int at = 1024 * i + threadIdx.x;
    entry[i] = len[i] = 0;
    if (1024 * i >= entries) continue;  // uniform
    entry[i] = p.table[min(at, entries - 1)];
    len[i] = p.lens[min(at, entries - 1) / p.max_pages];
  }
  small_bits(p, lane, w, refs, s_bits);
  __syncthreads();
  if (w == 0) {
    int c[LANE], count = 0;
#pragma unroll
    for (int i = 0; i < LANE; ++i) {
      c[i] = count;
      count += __builtin_popcountll(s_bits[LANE * lane + i]);
    }
    const int before = wave_scan_incl(count) - count;
#pragma unroll
    for (int i = 0; i < LANE; ++i) s_before[LANE * lane + i] = before + c[i];
  }
  __syncthreads();
  auto free_before = [&](int page) __attribute__((always_inline)) {  // page < kSmallPages
    return s_before[page >> 6] + __builtin_popcountll(s_bits[page >> 6] & ((1ull << (page & 63)) - 1));
  };
  auto is_free = [&](int page) __attribute__((always_inline)) { return ((s_bits[page >> 6] >> (page & 63)) & 1) != 0; };
  const int used = p.num_pages - s_before[WORDS - 1] - __builtin_popcountll(s_bits[WORDS - 1]);
  const int holes = used < kSmallPages ? free_before(used) : 0;
  auto mover = [&](int page) __attribute__((always_inline)) { return page - free_before(page) - (used - holes); };
  if (threadIdx.x == 0) {
    p.moved[0] = holes;
    p.moved[1] = used;
  }
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int page = 64 * (kSmallWaves * i + w) + lane;
    if (page >= p.num_pages || holes == 0) continue;
    if (page < used && is_free(page)) {
      const int r = free_before(page);
      s_dst[r] = (uint16_t)page;
      p.move_dst[r] = page;
    } else if (page >= used && !is_free(page)) {
      const int r = mover(page);
      s_refs[r] = refs[i];
      p.move_src[r] = page;
    }
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int page = 64 * (kSmallWaves * i + w) + lane;
    if (page < p.num_pages) p.new_refs[page] = page >= used ? 0 : is_free(page) ? s_refs[free_before(page)] : refs[i];
  }
#pragma unroll
  for (int i = 0; i < kSmallTable / (64 * kSmallWaves); ++i) {
    const int at = 1024 * i + threadIdx.x;
    if (at >= entries || at % p.max_pages >= pages_of(len[i])) continue;
    const int page = entry[i];
    p.new_table[at] = page >= used && page < p.num_pages && !is_free(page) ? s_dst[mover(page)] : page;
  }
}

// Third launch: the counts (the first workgroups) and the rows.
__global__ __launch_bounds__(kPageThreads) void pages_move_kernel(PagesArgs p, int count_groups) {
  const int used = p.moved[1];
  auto is_free = [&](long page) __attribute__((always_inline)) { return ((p.free_bits[page >> 6] >> (page & 63)) & 1) != 0; };
  if ((int)blockIdx.x < count_groups) {
    for (long page = (long)blockIdx.x * kPageThreads + threadIdx.x; page < p.num_pages; page += (long)count_groups * kPageThreads)
      p.new_refs[page] = page >= used ? 0 : is_free(page) ? p.moved_refs[p.rank[page]] : p.refs[page];
    return;
  }
  const int row = blockIdx.x - count_groups, n = pages_of(row_tokens(p, row));
  for (int c = threadIdx.x; c < n; c += kPageThreads) {
    const int page = p.table[(long)row * p.max_pages + c];
    const bool moves = page >= used && page < p.num_pages && !is_free(page);
    p.new_table[(long)row * p.max_pages + c] = moves ? p.move_dst[p.rank[page]] : page;
  }
}

// ---- copies.  A wave copies 2 or 4 KiB of one pool's page at a time: everything that it looks up is wave-uniform.  Bound: HBM
// (3.8 GB read and written: 4.96 TB/s, a plain copy of that size 4.94; 419 MB, in the last-level cache: 6.8).  Stores that leave no
// line behind in L2: 419 MB 85 -> 70 us; loads of that kind as well: 84.
constexpr int kCopyCaches = 64;  // caches of one launch: their pools are kernel arguments
struct CopyArgs {
  char *pools[2 * kCopyCaches];
  const int32_t *src, *dst, *rows, *count;
  int n, num_pools, num_pages, parts;  // parts: of a pool's page
  int row_shift;                       // log2 of the 16-byte chunks of a row
};

template <int PER>  // chunks of a lane
__global__ __launch_bounds__(kPageThreads) void pages_copy_kernel(CopyArgs a) {
  const int lane = threadIdx.x & 63;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n = a.count ? min(a.n, *a.count) : a.n;
  const unsigned per_pair = (unsigned)(a.num_pools * a.parts);
  const long units = (long)n * per_pair;
  for (long u = (long)blockIdx.x * kPageWaves + w; u < units; u += (long)gridDim.x * kPageWaves) {
    const int i = units >> 32 == 0 ? (int)((unsigned)u / per_pair) : (int)(u / per_pair);  // 32 bits where they do: 7.1 -> 6.0 us on 39 MB
    const int rem = (int)(u - (long)i * per_pair), pool = rem / a.parts, part = rem - pool * a.parts;
    const int src = a.src[i], dst = a.dst[i], rows = a.rows ? a.rows[i] : kPage;
    if (src < 0 || src >= a.num_pages || dst < 0 || dst >= a.num_pages || src == dst) continue;
    const size_t bytes = (size_t)a.parts * PER * 1024;
    const u32x4 *from = (const u32x4 *)(a.pools[pool] + src * bytes);
    u32x4 *to = (u32x4 *)(a.pools[pool] + dst * bytes);
    u32x4 x[PER];
    bool there[PER];
#pragma unroll
    for (int k = 0; k < PER; ++k) {
      const int c = (part * PER + k) * 64 + lane;
      there[k] = ((c >> a.row_shift) & (kPage - 1)) < rows;
      if (there[k]) x[k] = from[c];
    }
#pragma unroll
    for (int k = 0; k < PER; ++k)
      if (there[k]) __builtin_nontemporal_store(x[k], to + (part * PER + k) * 64 + lane);
  }
}

// ---- host

static size_t align16(size_t n) { return (n + 15) / 16 * 16; }
static int segments(int num_pages) { return (int)(((long)num_pages + kSegment - 1) / kSegment); }

size_t pages_workspace_bytes(int num_pages, int n) {
  const size_t nseg = segments(num_pages), scan = nseg * kSegWords * 8 + align16(nseg * 4);
  return scan + (n > 0 ? (size_t)align16(((size_t)n + 1) * 4) + (size_t)n * 4 : align16((size_t)num_pages * 4) + (size_t)(num_pages / 2) * 4);
}

static PagesArgs pages_args(const sp_page_table &t, void *workspace, int n) {
  PagesArgs p = {};
  p.refs = t.ref_counts;
  p.table = t.block_table;
  p.lens = t.seq_lens;
  p.written = t.written_lens;
  p.num_pages = t.num_pages;
  p.num_rows = t.num_rows;
  p.max_pages = t.max_pages_per_seq;
  p.nseg = segments(t.num_pages);
  p.n = n;
  char *ws = (char *)workspace;
  p.free_bits = (uint64_t *)ws;
  ws += (size_t)p.nseg * kSegWords * 8;
  p.seg_free = (int32_t *)ws;
  ws += align16((size_t)p.nseg * 4);
  if (n > 0) {
    p.plan = (int32_t *)ws;
    p.sizes = (int32_t *)(ws + align16(((size_t)n + 1) * 4));
  } else {
    p.rank = (int32_t *)ws;
    p.moved_refs = (int32_t *)(ws + align16((size_t)t.num_pages * 4));
  }
  return p;
}

static int launched(const char *what) {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? SP_OK : fail(SP_ERR_HIP, "%s launch: %s", what, hipGetErrorString(e));
}

// Scan and take, or both in one launch where one workgroup is quick enough: up to an entry a wave, or rows that are short together.  A
// pass of release, fork, copy and reserve: 4 forks of a row of 19 pages 24.8 us with two launches each, 16.6 with one; 41 of up to 17
// 26 and 21; but 52 of 212 pages 27 and 40.
template <int OP>
static void launch_take(const PagesArgs &p, hipStream_t stream) {
  if (p.num_pages <= kSmallPages && p.max_pages <= kSmallWidth && (p.n <= kSmallWaves || (p.n <= kSmallEntries && (long)p.n * p.max_pages <= 4096))) {
    hipLaunchKernelGGL(pages_small_kernel<OP>, dim3(1), dim3(64 * kSmallWaves), 0, stream, p);
    return;
  }
  hipLaunchKernelGGL(pages_scan_kernel<OP>, dim3(p.nseg + 1), dim3(kPageThreads), 0, stream, p);
  hipLaunchKernelGGL(pages_take_kernel<OP>, dim3(p.n), dim3(kPageThreads), 0, stream, p);
}

int launch_pages_reserve(const sp_page_table &t, const int32_t *rows, const int32_t *new_lens, int n, int32_t *shortfall, void *workspace,
                         hipStream_t stream) {
  PagesArgs p = pages_args(t, workspace, n);
  p.a = rows;
  p.b = new_lens;
  p.shortfall = shortfall;
  launch_take<kReserve>(p, stream);
  return launched("sp_pages_reserve");
}

int launch_pages_fork(const sp_page_table &t, const int32_t *parents, const int32_t *children, int n, int32_t *copy_src, int32_t *copy_dst,
                      int32_t *copy_rows, int32_t *shortfall, void *workspace, hipStream_t stream) {
  PagesArgs p = pages_args(t, workspace, n);
  p.a = parents;
  p.b = children;
  p.copy_src = copy_src;
  p.copy_dst = copy_dst;
  p.copy_rows = copy_rows;
  p.shortfall = shortfall;
  launch_take<kFork>(p, stream);
  return launched("sp_pages_fork");
}

int launch_pages_release(const sp_page_table &t, const int32_t *rows, const int32_t *keep_lens, int n, hipStream_t stream) {
  PagesArgs p = pages_args(t, nullptr, n);
  p.a = rows;
  hipLaunchKernelGGL(pages_release_kernel, dim3(n), dim3(kPageThreads), 0, stream, p, keep_lens);
  return launched("sp_pages_release");
}

int launch_pages_compact(const sp_page_table &t, int32_t *new_block_table, int32_t *new_ref_counts, int32_t *move_src, int32_t *move_dst,
                         int32_t *moved, void *workspace, hipStream_t stream) {
  PagesArgs p = pages_args(t, workspace, 0);
  p.new_table = new_block_table;
  p.new_refs = new_ref_counts;
  p.move_src = move_src;
  p.move_dst = move_dst;
  p.moved = moved;
  if (t.num_pages <= kSmallPages && (long)t.num_rows * t.max_pages_per_seq <= kSmallTable) {
    hipLaunchKernelGGL(pages_compact_small_kernel, dim3(1), dim3(64 * kSmallWaves), 0, stream, p);
    return launched("sp_pages_compact");
  }
  const int count_groups = (int)min((long)1024, ((long)t.num_pages + kPageThreads - 1) / kPageThreads);
  hipLaunchKernelGGL(pages_scan_kernel<kCompact>, dim3(p.nseg), dim3(kPageThreads), 0, stream, p);
  hipLaunchKernelGGL(pages_rank_kernel, dim3(p.nseg), dim3(kPageThreads), 0, stream, p);
  hipLaunchKernelGGL(pages_move_kernel, dim3((unsigned)count_groups + (unsigned)t.num_rows), dim3(kPageThreads), 0, stream, p, count_groups);
  return launched("sp_pages_compact");
}

int launch_pages_copy(const sp_cache_desc *caches, int num_caches, const int32_t *src, const int32_t *dst, const int32_t *rows,
                      const int32_t *count, int n, hipStream_t stream) {
  const int row_chunks = caches[0].head_dim / 8, chunks = caches[0].num_kv_heads * kPage * row_chunks;  // a multiple of 128
  const bool four = chunks % 256 == 0;
  for (int c0 = 0; c0 < num_caches; c0 += kCopyCaches) {
    CopyArgs a;
    const int m = min(num_caches - c0, kCopyCaches);
    for (int i = 0; i < kCopyCaches; ++i) {
      a.pools[2 * i] = i < m ? (char *)caches[c0 + i].k_pages : nullptr;
      a.pools[2 * i + 1] = i < m ? (char *)caches[c0 + i].v_pages : nullptr;
    }
    a.src = src;
    a.dst = dst;
    a.rows = rows;
    a.count = count;
    a.n = n;
    a.num_pools = 2 * m;
    a.num_pages = caches[0].num_pages;
    a.parts = chunks / (four ? 256 : 128);
    a.row_shift = row_chunks == 16 ? 4 : 3;
    const long units = (long)n * a.num_pools * a.parts;
    // A workgroup per four units: 419 MB in 62 us, 3.8 GB in 766; with eight workgroups a CU that go on to the next 70 and 780.  Where
    // the number of pairs is only known on the device most of them may find nothing, so no more than 32 a CU (63 and 777).
    const unsigned groups = (unsigned)min((units + kPageWaves - 1) / kPageWaves, count ? 256L * 32 : 256L * 4096);
    if (four) hipLaunchKernelGGL(pages_copy_kernel<4>, dim3(groups), dim3(kPageThreads), 0, stream, a);
    else hipLaunchKernelGGL(pages_copy_kernel<2>, dim3(groups), dim3(kPageThreads), 0, stream, a);
  }
  return launched("sp_pages_copy");
}

}  // namespace sp
