// Changes of a paged K/V cache: room for more tokens, new tokens into the pages, branches, pages given back, compaction.
//
// What a call decides (which page goes where) is a few thousand integers: one kernel, a cluster of CTAs on one GPC, whose steps are
// separated by cluster barriers instead of launches (about 0.5 us each against 2-3).  What it moves (page contents) is
// a second kernel over the whole GPU behind it, bound by HBM: every byte read once and written once (compaction of 1.5 GB: 499 us, 5.9 TB/s; 8 parents with four
// branches each, 1.3 GB read and written: 228 us, 5.5 TB/s).
//
// Free pages are those with ref == 0; they are taken in ascending order, so that a result is determined by the state alone and what
// is in use stays low in the pool.
#include <climits>

#include "avsa_common.cuh"
#include "sm100_ptx.cuh"

namespace avsa {

constexpr int kMetaThreads = 1024, kMetaWarps = kMetaThreads / 32;
// CTAs of the cluster: one as long as it has no more than this many integers to look at or copy, else the portable maximum.
constexpr int kMetaCluster = 8;
constexpr long long kMetaSingle = 16384;

enum CacheWhere { kCacheSeq = 201, kCacheTwice, kCacheLength, kCachePage, kCacheRef, kCacheFull, kCacheChild };

// One entry of a call's list, decided by the first CTA: sequences, what they hold, and where their free pages begin.
struct ListEntry {
  int seq, other;       // other: fork's parent; seq < 0: left out
  int tokens, new_tokens;
  int first, need;      // free pages [first, first + need) of the list of free pages
  int pad[2];
};
static_assert(sizeof(ListEntry) == 32, "two 16-byte accesses");

// A workspace: status record | counts of the CTAs | claims [seqs] | list entries [n] | free pages [pages] | moves [max(n, pages)] int4
struct CacheWs {
  StatusRecord* status;
  int* counts;       // [3][kMetaCluster], then [62] moves in all, [63] needed pages in all
  int* claims;
  ListEntry* list;
  int* free_pages;
  int4* moves;       // from, to, ref
  static size_t bytes(int seqs, int pages, int n) {
    const size_t m = static_cast<size_t>(n > pages ? n : pages);
    return kStatusBytes + 256 + align_up(static_cast<size_t>(seqs) * 4, 256) + align_up(static_cast<size_t>(n) * sizeof(ListEntry), 256) +
           align_up(static_cast<size_t>(pages) * 4, 256) + align_up(m * sizeof(int4), 256);
  }
  CacheWs(void* ws, int seqs, int pages, int n) {
    uint8_t* p = static_cast<uint8_t*>(ws);
    status = reinterpret_cast<StatusRecord*>(p);
    counts = reinterpret_cast<int*>(p + kStatusBytes);
    p += kStatusBytes + 256;
    claims = reinterpret_cast<int*>(p);
    p += align_up(static_cast<size_t>(seqs) * 4, 256);
    list = reinterpret_cast<ListEntry*>(p);
    p += align_up(static_cast<size_t>(n) * sizeof(ListEntry), 256);
    free_pages = reinterpret_cast<int*>(p);
    p += align_up(static_cast<size_t>(pages) * 4, 256);
    moves = reinterpret_cast<int4*>(p);
  }
};
constexpr int kNumMoves = 62, kNumNeeded = 63;

struct MetaArgs {
  avsa_cache c;
  CacheWs w;
  const int32_t* seq;       // extend, free; fork: child
  const int32_t* other;     // extend: count; fork: parent
  int n;
  int32_t* n_live;
  int32_t* granted;         // extend: [n], or NULL
  int32_t* log;
};

__device__ __forceinline__ int cluster_rank() {
  int r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ int cluster_size() {
  int r;
  asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ unsigned lanes_below() {
  unsigned m;
  asm volatile("mov.u32 %0, %%lanemask_lt;" : "=r"(m));
  return m;
}

// Sum over the CTA, for every thread.  `sm`: kMetaWarps ints; a barrier has to lie between two uses.
__device__ __forceinline__ int block_sum(int v, int* sm) {
  v = __reduce_add_sync(0xffffffffu, v);
  if ((threadIdx.x & 31) == 0) sm[threadIdx.x >> 5] = v;
  __syncthreads();
  return __reduce_add_sync(0xffffffffu, sm[threadIdx.x & 31]);
}
// Sum of the threads before this one, and of all; the same conditions.
__device__ __forceinline__ int block_scan(int v, int& all, int* sm) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int inc = v;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int o = __shfl_up_sync(0xffffffffu, inc, d);
    if (lane >= d) inc += o;
  }
  if (lane == 31) sm[warp] = inc;
  __syncthreads();
  const int mine = sm[lane];
  all = __reduce_add_sync(0xffffffffu, mine);
  return __reduce_add_sync(0xffffffffu, lane < warp ? mine : 0) + inc - v;
}

constexpr int kVals = 8;      // values a thread has in flight in the passes over `ref`
constexpr size_t kScanBytes = kVals * 32 * sizeof(int);      // of the kernels' own shared memory, for their counts

// Calls emit(index, value, rank) for the indices of [lo, hi) whose value is taken, in ascending order from rank `base` on; the rank behind the last one.
template <class Take, class Emit>
__device__ __forceinline__ int for_taken(const int32_t* v, int lo, int hi, int base, Take take, Emit emit, int* sm) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  for (int t0 = lo; t0 < hi; t0 += kMetaThreads * kVals) {
    int x[kVals];
    unsigned m[kVals];
#pragma unroll
    for (int i = 0; i < kVals; i++) {
      const int at = t0 + i * kMetaThreads + threadIdx.x;
      x[i] = at < hi ? v[at] : 0;
    }
#pragma unroll
    for (int i = 0; i < kVals; i++) {
      const int at = t0 + i * kMetaThreads + threadIdx.x;
      m[i] = __ballot_sync(0xffffffffu, at < hi && take(at, x[i]));
      if (lane == 0) sm[i * 32 + warp] = __popc(m[i]);
    }
    __syncthreads();
    // every warp sums what lies before it itself: the counts of 32 warps are one load
    int before = base;
#pragma unroll
    for (int i = 0; i < kVals; i++) {
      const int c = sm[i * 32 + lane];
      const int mine = before + __reduce_add_sync(0xffffffffu, lane < warp ? c : 0);
      const int at = t0 + i * kMetaThreads + threadIdx.x;
      if ((m[i] >> lane) & 1u) emit(at, x[i], mine + __popc(m[i] & lanes_below()));
      before += __reduce_add_sync(0xffffffffu, c);
    }
    base = before;
    __syncthreads();
  }
  return base;
}
template <class Take>
__device__ __forceinline__ int count_taken(const int32_t* v, int lo, int hi, Take take, int* sm) {
  int n = 0;
  for (int t0 = lo + threadIdx.x; t0 < hi; t0 += kMetaThreads * kVals) {
    int x[kVals];
#pragma unroll
    for (int i = 0; i < kVals; i++) x[i] = t0 + i * kMetaThreads < hi ? v[t0 + i * kMetaThreads] : 0;
#pragma unroll
    for (int i = 0; i < kVals; i++) n += t0 + i * kMetaThreads < hi && take(t0 + i * kMetaThreads, x[i]);
  }
  const int all = block_sum(n, sm);
  __syncthreads();
  return all;
}

// The cluster's share of an array copied to another, if it is another.
__device__ __forceinline__ void copy_ints(const int32_t* from, int32_t* to, long long n, int rank, int ctas) {
  if (from == to) return;
  const long long step = static_cast<long long>(ctas) * kMetaThreads;
  for (long long i = static_cast<long long>(rank) * kMetaThreads + threadIdx.x; i < n; i += step * 4) {
    int x[4];
#pragma unroll
    for (int u = 0; u < 4; u++)
      if (i + u * step < n) x[u] = from[i + u * step];
#pragma unroll
    for (int u = 0; u < 4; u++)
      if (i + u * step < n) to[i + u * step] = x[u];
  }
}
__device__ __forceinline__ void copy_state(const avsa_cache& c, int rank, int ctas) {
  copy_ints(c.table, c.table_out, static_cast<long long>(c.seqs) * c.width, rank, ctas);
  copy_ints(c.length, c.length_out, c.seqs, rank, ctas);
  copy_ints(c.ref, c.ref_out, c.pages, rank, ctas);
}
__device__ __forceinline__ void clear_status(StatusRecord* st) {
  st->code = st->where = st->item = st->aux = st->redo_count = st->next_item = 0;
}
__device__ __forceinline__ void page_share(const avsa_cache& c, int rank, int ctas, int& lo, int& hi) {
  const int part = (c.pages + ctas - 1) / ctas;
  lo = min(c.pages, rank * part);
  hi = min(c.pages, lo + part);
}

// Pages of so many tokens.
__device__ __forceinline__ int pages_of(int tokens, int page) { return tokens / page + (tokens % page != 0); }

enum { kExtend = 0, kFork = 1 };

// What a call hands from one step to the next.  A single CTA keeps it in shared memory as far as it fits (a step of an ordinary call is then two trips to L2 deep
// instead of eight: 16 sequences and 150 pages 8.3 -> 7.4 us); the CTAs of a cluster, and longer lists, in the workspace.  Its free pages it lists in one pass,
// all of them, while the list is on its way (in a loop of calls 6.1 -> 5.3 us).
// (As large as the call needs it: up to 48 KB, the kernels' own arrays among them, need no kernel attribute, which costs the host as much as an argument check.)
constexpr int kOwnClaims = 4096, kOwnList = 1024;
struct AssignSmem {
  size_t claims, free_pages, bytes;      // offsets behind the list entries
  __host__ __device__ AssignSmem(const avsa_cache& c, int n)
      : claims(n <= kOwnList ? static_cast<size_t>(n) * sizeof(ListEntry) : 0), free_pages(claims + (c.seqs <= kOwnClaims ? static_cast<size_t>(c.seqs) * 4 : 0)),
        bytes(free_pages + static_cast<size_t>(c.pages) * 4) {}
};
constexpr size_t kAssignMost = kOwnList * sizeof(ListEntry) + kOwnClaims * 4 + kMetaSingle * 4;      // (a single CTA has kMetaSingle pages at most)

// extend and fork: which free pages go to which sequence.
template <int OP>
__global__ void __launch_bounds__(kMetaThreads, 1) assign_pages_kernel(const MetaArgs a) {
  extern __shared__ __align__(16) uint8_t smem[];
  __shared__ int sm[kVals * 32];
  pdl_wait();
  pdl_launch();
  const avsa_cache& c = a.c;
  const CacheWs& w = a.w;
  const int rank = cluster_rank(), ctas = cluster_size(), tid = threadIdx.x, lane = tid & 31;
  const bool alone = ctas == 1;
  const AssignSmem own(c, a.n);
  int* const claims = alone && c.seqs <= kOwnClaims ? reinterpret_cast<int*>(smem + own.claims) : w.claims;
  ListEntry* const list = alone && a.n <= kOwnList ? reinterpret_cast<ListEntry*>(smem) : w.list;
  int* const free_pages = alone ? reinterpret_cast<int*>(smem + own.free_pages) : w.free_pages;
  // the thread's first entry: sequence, count or parent, tokens
  int s0 = -1, o0 = -1, n0 = 0;
  if (rank == 0 && tid < a.n) {
    s0 = a.seq[tid];
    o0 = a.other[tid];
  }
  if (rank == 0 && tid == 0) clear_status(w.status);
  copy_state(c, rank, ctas);
  {
    const int of = OP == kFork ? o0 : s0;
    if (of >= 0 && of < c.seqs) n0 = c.length[of];
  }
  // the list: entries that name a sequence again lose to the first one (of those that are not left out)
  auto seq_of = [&](int k) { return k == tid ? s0 : a.seq[k]; };
  auto claims_of = [&](int k) {
    const int s = seq_of(k), o = k == tid ? o0 : a.other[k];
    return s < c.seqs && (OP == kExtend || o >= 0) ? s : -1;
  };
  if (rank == 0) {
    for (int k = tid; k < a.n; k += kMetaThreads) {
      const int s = claims_of(k);
      if (s >= 0) claims[s] = INT_MAX;
    }
  }
  int lo, hi;
  page_share(c, rank, ctas, lo, hi);
  auto is_free = [](int, int r) { return r <= 0; };
  int n_free = 0;
  if (alone) {
    n_free = for_taken(c.ref, lo, hi, 0, is_free, [&](int page, int, int at) { free_pages[at] = page; }, sm);
    // (its last step is a barrier)
  } else {
    const int mine = count_taken(c.ref, lo, hi, is_free, sm);
    if (tid == 0) w.counts[rank] = mine;
  }
  if (rank == 0) {
    for (int k = tid; k < a.n; k += kMetaThreads) {
      const int s = claims_of(k);
      if (s >= 0) atomicMin(&claims[s], k);
    }
    __syncthreads();
    int taken = 0;
    for (int k0 = 0; k0 < a.n; k0 += kMetaThreads) {
      const int k = k0 + tid;
      ListEntry e = {};
      e.seq = -1;
      if (k < a.n) {
        const int s = seq_of(k), o = k0 == 0 ? o0 : a.other[k];
        int bad = 0, code = AVSA_ERR_BAD_TABLE;
        if (s >= 0 && (OP == kExtend || o >= 0)) {
          if (s >= c.seqs || (OP == kFork && o >= c.seqs)) bad = kCacheSeq;
          else if (*static_cast<volatile int*>(&claims[s]) != k) bad = kCacheTwice;
          else {
            const int n = k0 == 0 ? n0 : c.length[OP == kFork ? o : s];
            const long long room = min(static_cast<long long>(c.width) * c.page, static_cast<long long>(INT_MAX));      // (a length has 31 bits)
            if (n < 0 || n > room || (OP == kExtend && o < 0)) bad = kCacheLength;
            else if (OP == kFork && c.length[s] != 0) bad = kCacheChild;
            else if (OP == kExtend && n + static_cast<long long>(o) > room) bad = kCacheFull, code = AVSA_ERR_NO_PAGES;
            else {
              e.seq = s;
              e.other = o;
              e.tokens = n;
              if (OP == kExtend) {
                e.new_tokens = o;
                e.need = pages_of(n + o, c.page) - pages_of(n, c.page);
              } else {
                e.need = n % c.page != 0;
              }
            }
          }
        }
        if (bad) report_logged(w.status, a.log, code, bad, k, s);
      }
      int all;
      e.first = taken + block_scan(e.need, all, sm);
      taken += all;
      if (k < a.n) list[k] = e;
      __syncthreads();
    }
    if (tid == 0 && !alone) w.counts[kNumNeeded] = taken;
  }
  if (!alone) {
    cluster_sync_all();
    const int needed = __ldcg(&w.counts[kNumNeeded]);
    int base = 0;
    for (int r = 0; r < ctas; r++) {
      const int m = __ldcg(&w.counts[r]);
      if (r < rank) base += m;
      n_free += m;
    }
    if (base < needed) {      // (uniform over the CTA)
      // (ref has not been written yet: in place it is still the state before the call)
      for_taken(c.ref, lo, hi, base, is_free, [&](int page, int, int at) { if (at < needed) free_pages[at] = page; }, sm);
    }
    cluster_sync_all();
  }
  const int warps = ctas * kMetaWarps;
  for (int k = rank * kMetaWarps + (tid >> 5); k < a.n; k += warps) {      // a warp to an entry
    int4 e0, e1;
    if (alone) {
      e0 = *reinterpret_cast<const int4*>(&list[k]), e1 = *(reinterpret_cast<const int4*>(&list[k]) + 1);
    } else {
      e0 = __ldcg(reinterpret_cast<const int4*>(&list[k])), e1 = __ldcg(reinterpret_cast<const int4*>(&list[k]) + 1);
    }
    const int s = e0.x, other = e0.y, tokens = e0.z, new_tokens = e0.w, first = e1.x, need = e1.y;
    auto free_page = [&](int at) { return alone ? free_pages[at] : __ldcg(&free_pages[at]); };
    const bool refused = s >= 0 && need > 0 && first + need > n_free;
    if (refused && lane == 0) report_logged(w.status, a.log, AVSA_ERR_NO_PAGES, kCacheFull, k, s);
    if (OP == kExtend && lane == 0 && a.granted != nullptr) a.granted[k] = s < 0 || refused ? 0 : new_tokens;
    if (OP == kFork && lane == 0 && (s < 0 || refused || need == 0)) w.moves[k] = make_int4(-1, -1, 0, 0);
    if (s < 0 || refused) continue;
    int32_t* row = c.table_out + static_cast<long long>(s) * c.width;
    if (OP == kExtend) {
      const int have = pages_of(tokens, c.page);
      for (int j = lane; j < need; j += 32) {
        const int page = free_page(first + j);
        row[have + j] = page;
        c.ref_out[page] = 1;
      }
      if (lane == 0) c.length_out[s] = tokens + new_tokens;
    } else {
      const int whole = tokens / c.page;
      const int32_t* from = c.table + static_cast<long long>(other) * c.width;
      for (int j = lane; j < c.width; j += 32) {
        int page = -1;
        if (j < whole) {
          page = from[j];
          if (page >= 0 && page < c.pages) {
            atomicAdd(&c.ref_out[page], 1);
          } else {
            report_logged(w.status, a.log, AVSA_ERR_BAD_TABLE, kCachePage, other, j);
          }
        } else if (j == whole && need) {
          page = free_page(first);
          c.ref_out[page] = 1;
          const int src = from[j];
          const bool good = src >= 0 && src < c.pages;
          w.moves[k] = good ? make_int4(src, page, 1, 0) : make_int4(-1, -1, 0, 0);
          if (!good) report_logged(w.status, a.log, AVSA_ERR_BAD_TABLE, kCachePage, other, j);
        }
        row[j] = page;
      }
      if (lane == 0) c.length_out[s] = tokens;
    }
  }
}

__global__ void __launch_bounds__(kMetaThreads, 1) free_pages_kernel(const MetaArgs a) {
  pdl_wait();
  pdl_launch();
  const avsa_cache& c = a.c;
  const int rank = cluster_rank(), ctas = cluster_size(), tid = threadIdx.x, lane = tid & 31;
  if (rank == 0 && tid == 0) clear_status(a.w.status);
  const int k0 = rank * kMetaWarps + (tid >> 5), s0 = k0 < a.n ? a.seq[k0] : -1;
  copy_state(c, rank, ctas);
  cluster_sync_all();
  for (int k = k0; k < a.n; k += ctas * kMetaWarps) {
    const int s = k == k0 ? s0 : a.seq[k];
    if (s < 0) continue;
    if (s >= c.seqs) {
      if (lane == 0) report_logged(a.w.status, a.log, AVSA_ERR_BAD_TABLE, kCacheSeq, k, s);
      continue;
    }
    // whoever takes an entry of the row gives its page back: a sequence that is listed again has none left by then
    int32_t* row = c.table_out + static_cast<long long>(s) * c.width;
    for (int j = lane; j < c.width; j += 32) {
      const int page = atomicExch(&row[j], -1);
      if (page == -1) continue;
      if (page < -1 || page >= c.pages) report_logged(a.w.status, a.log, AVSA_ERR_BAD_TABLE, kCachePage, s, j);
      else if (atomicSub(&c.ref_out[page], 1) <= 0) report_logged(a.w.status, a.log, AVSA_ERR_BAD_TABLE, kCacheRef, s, page);
    }
    if (lane == 0) c.length_out[s] = 0;
  }
}

// Which pages move, and the references behind the moves.  Both lists are ascending, so the k-th move is known from the k-th
// free place below n_live and the k-th page in use from n_live on.  A single CTA keeps them in shared memory (freed and compacted, 3 kernels, 4.9 MB moved: 14.5 -> 12.6 us).
__host__ __device__ inline int most_moves(const avsa_cache& c) { return c.pages / 2; }      // (as many places below n_live as pages behind)
constexpr size_t kMoveBytes = 12, kPlanMost = kMetaSingle / 2 * kMoveBytes;

__global__ void __launch_bounds__(kMetaThreads, 1) plan_compaction_kernel(const MetaArgs a) {
  extern __shared__ __align__(16) uint8_t smem[];
  __shared__ int sm[kVals * 32];
  pdl_wait();
  pdl_launch();
  const avsa_cache& c = a.c;
  const CacheWs& w = a.w;
  const int rank = cluster_rank(), ctas = cluster_size(), tid = threadIdx.x;
  const bool alone = ctas == 1;
  if (rank == 0 && tid == 0) clear_status(w.status);
  copy_ints(c.length, c.length_out, c.seqs, rank, ctas);
  int lo, hi;
  page_share(c, rank, ctas, lo, hi);
  auto is_free = [](int, int r) { return r <= 0; };
  auto in_use = [](int, int r) { return r > 0; };
  int* const own_from = reinterpret_cast<int*>(smem);
  int* const own_to = own_from + most_moves(c);
  int* const own_ref = own_to + most_moves(c);
  const int mine = count_taken(c.ref, lo, hi, in_use, sm);
  int n_live = mine, hole0 = 0, move0 = 0, n_moves = 0;
  if (!alone) {
    if (tid == 0) w.counts[rank] = mine;
    cluster_sync_all();
    n_live = 0;
    for (int r = 0; r < ctas; r++) n_live += __ldcg(&w.counts[r]);
    const int holes = count_taken(c.ref, lo, min(hi, n_live), is_free, sm);
    // (pages in use from n_live on: all in use but those below n_live)
    const int below = max(0, min(hi, n_live) - lo) - holes;
    if (tid == 0) {
      w.counts[kMetaCluster + rank] = holes;
      w.counts[2 * kMetaCluster + rank] = mine - below;
    }
    cluster_sync_all();
    for (int r = 0; r < ctas; r++) {
      const int h = __ldcg(&w.counts[kMetaCluster + r]), m = __ldcg(&w.counts[2 * kMetaCluster + r]);
      if (r < rank) hole0 += h, move0 += m;
      n_moves += h;
    }
  }
  int* const move_words = reinterpret_cast<int*>(w.moves);
  const int holes_end = for_taken(c.ref, lo, min(hi, n_live), hole0, is_free, [&](int page, int, int at) {
    if (alone) own_to[at] = page;
    else move_words[4 * at + 1] = page;
  }, sm);
  if (alone) n_moves = holes_end;
  for_taken(c.ref, max(lo, min(hi, n_live)), hi, move0, in_use, [&](int page, int r, int at) {
    if (alone) {
      own_from[at] = page;
      own_ref[at] = r;
    } else {
      move_words[4 * at] = page;
      move_words[4 * at + 2] = r;
    }
  }, sm);
  if (rank == 0 && tid == 0) {
    a.n_live[0] = n_live;
    w.counts[kNumMoves] = n_moves;
  }
  __syncthreads();
  for (int p = lo + tid; p < hi; p += kMetaThreads) {
    const int r = c.ref[p];
    if (p >= n_live) {
      c.ref_out[p] = 0;
      w.free_pages[p] = -1;
    } else if (r > 0) {
      c.ref_out[p] = r;
    }
  }
  if (alone) __syncthreads();
  else cluster_sync_all();
  // free_pages[p] is where page p >= n_live has gone, -1 for one that was not in use
  for (int k = rank * kMetaThreads + tid; k < n_moves; k += ctas * kMetaThreads) {
    const int4 m = alone ? make_int4(own_from[k], own_to[k], own_ref[k], 0) : __ldcg(&w.moves[k]);
    if (alone) w.moves[k] = m;
    c.ref_out[m.y] = m.z;
    w.free_pages[m.x] = m.y;
  }
}

// ------------------------------------------------------------------------------------------------ page contents
constexpr int kCopyThreads = 256, kCopyVecs = 4;
constexpr int kCopyChunk = kCopyThreads * kCopyVecs * 16;      // bytes a CTA moves at a time

struct CopyArgs {
  avsa_pages pool;
  const int4* moves;
  const int* n_moves;       // or NULL: n
  int n;
  // compaction: the table's pages by their new numbers
  const int32_t* table;
  int32_t* table_out;
  const int32_t* place;
  const int32_t* n_live;
  int seqs, width, pages, page;
  StatusRecord* status;
  int32_t* log;
};

__global__ void __launch_bounds__(kCopyThreads) move_pages_kernel(const CopyArgs a) {
  pdl_wait();
  pdl_launch();
  const int tid = threadIdx.x;
  if (a.table != nullptr) {
    const int n_live = a.n_live[0];
    const long long entries = static_cast<long long>(a.seqs) * a.width;
    for (long long i = static_cast<long long>(blockIdx.x) * kCopyThreads + tid; i < entries; i += static_cast<long long>(gridDim.x) * kCopyThreads) {
      const int page = a.table[i];
      int to = page;
      bool bad = page >= a.pages || page < -1;
      if (!bad && page >= n_live) {
        to = a.place[page];
        bad = to < 0;
      }
      if (bad) report_logged(a.status, a.log, AVSA_ERR_BAD_TABLE, kCachePage, static_cast<int>(i / a.width), static_cast<int>(i % a.width));
      if (a.table != a.table_out || to != page) a.table_out[i] = to;
    }
  }
  const int n = a.n_moves != nullptr ? a.n_moves[0] : a.n;
  const long long chunks = (a.pool.page_bytes + kCopyChunk - 1) / kCopyChunk;
  const long long total = static_cast<long long>(n) * a.pool.planes * chunks;
  for (long long u = blockIdx.x; u < total; u += gridDim.x) {
    // the moves side by side: branches of one parent read its page together, once from HBM (fork of 8 x 4 branches, 1.3 GB read and written: 293 -> 228 us)
    const long long r = u / n;
    const int k = static_cast<int>(u - r * n), plane = static_cast<int>(r / chunks), chunk = static_cast<int>(r - plane * chunks);
    const int4 m = a.moves[k];
    if (m.x < 0) continue;
    uint8_t* const base = static_cast<uint8_t*>(a.pool.ptr) + plane * a.pool.stride_plane;
    const long long at = static_cast<long long>(chunk) * kCopyChunk + tid * 16;
    const uint4* const from = reinterpret_cast<const uint4*>(base + m.x * a.pool.stride_page + at);
    uint4* const to = reinterpret_cast<uint4*>(base + m.y * a.pool.stride_page + at);
    uint4 x[kCopyVecs];
#pragma unroll
    for (int i = 0; i < kCopyVecs; i++)
      if (at + i * kCopyThreads * 16 < a.pool.page_bytes) x[i] = from[i * kCopyThreads];
#pragma unroll
    for (int i = 0; i < kCopyVecs; i++)
      if (at + i * kCopyThreads * 16 < a.pool.page_bytes) __stcs(to + i * kCopyThreads, x[i]);
  }
}

struct WriteArgs {
  avsa_bf16_4d k_new, v_new, k_pool, v_pool;
  const int32_t *table, *length, *seq, *count;
  int Hkv, L;
  int vec_shift, head_shift, tokens;      // a CTA's tile: 2^vec_shift vectors of 16 bytes of 2^head_shift heads of `tokens` tokens
  int page_shift, pages, seqs, width;
};
constexpr int kWriteVecs = 4;      // of each tensor a thread

// A CTA takes a tile of tokens by heads of one list entry: what it reads is contiguous over the heads of a token, what it writes over the tokens of a head in a page
// (4 x 1560 tokens of 24 heads, 77 MB in and as much out: 23.9 us, 6.4 TB/s).
__global__ void __launch_bounds__(kCopyThreads) write_tokens_kernel(const WriteArgs a) {
  pdl_wait();
  pdl_launch();
  const int k = blockIdx.z;
  const int s = a.seq != nullptr ? a.seq[k] : k;
  if (s < 0 || s >= a.seqs) return;
  const int count = a.count != nullptr ? min(a.count[k], a.L) : a.L;
  const int t0 = blockIdx.x * a.tokens, h0 = blockIdx.y << a.head_shift;
  if (t0 >= count) return;
  const long long start = static_cast<long long>(a.length[s]) - count;
  const int32_t* const row = a.table + static_cast<long long>(s) * a.width;
  uint4 x[kWriteVecs], y[kWriteVecs];
  long long to_k[kWriteVecs], to_v[kWriteVecs];
#pragma unroll
  for (int u = 0; u < kWriteVecs; u++) {
    const int i = threadIdx.x + u * kCopyThreads;
    const int c = (i & ((1 << a.vec_shift) - 1)) * 8, h = h0 + ((i >> a.vec_shift) & ((1 << a.head_shift) - 1));
    const int in_tile = i >> (a.vec_shift + a.head_shift), t = t0 + in_tile;
    const long long pos = start + t;
    to_k[u] = -1;
    if (in_tile >= a.tokens || t >= count || h >= a.Hkv || pos < 0 || (pos >> a.page_shift) >= a.width) continue;
    const int page = row[pos >> a.page_shift];
    if (page < 0 || page >= a.pages) continue;
    const long long in = pos & ((1 << a.page_shift) - 1);
    to_k[u] = page * a.k_pool.stride_b + h * a.k_pool.stride_h + in * a.k_pool.stride_n + c;
    to_v[u] = page * a.v_pool.stride_b + h * a.v_pool.stride_h + in * a.v_pool.stride_n + c;
    x[u] = __ldcs(reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(a.k_new.ptr) + k * a.k_new.stride_b + h * a.k_new.stride_h + t * a.k_new.stride_n + c));
    y[u] = __ldcs(reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(a.v_new.ptr) + k * a.v_new.stride_b + h * a.v_new.stride_h + t * a.v_new.stride_n + c));
  }
#pragma unroll
  for (int u = 0; u < kWriteVecs; u++) {
    if (to_k[u] < 0) continue;
    *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(const_cast<void*>(a.k_pool.ptr)) + to_k[u]) = x[u];
    *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(const_cast<void*>(a.v_pool.ptr)) + to_v[u]) = y[u];
  }
}

// ------------------------------------------------------------------------------------------------ host side
static bool page_size_ok(int page) { return page == 16 || page == 32 || page == 64 || page == 128; }

// As tensor_ok, but an axis of one element has no stride to speak of.
static bool tokens_ok(avsa_bf16_4d t, int B, int H, int N) {
  if (N == 1) t.stride_n = 8;
  return tensor_ok(t, B, H);
}

// [p, p + n) and [q, q + m) in ints share nothing
static bool apart(const int32_t* p, long long n, const int32_t* q, long long m) {
  const uintptr_t a = reinterpret_cast<uintptr_t>(p), b = reinterpret_cast<uintptr_t>(q);
  return a + 4 * static_cast<uintptr_t>(n) <= b || b + 4 * static_cast<uintptr_t>(m) <= a;
}

static int check_cache(const avsa_cache& c, bool by_page) {
  if (c.seqs <= 0 || c.width <= 0 || c.pages <= 0) return AVSA_ERR_INVALID_ARG;
  if ((by_page && !page_size_ok(c.page)) || static_cast<long long>(c.seqs) * c.width > INT_MAX || c.pages > (1 << 30)) return AVSA_ERR_UNSUPPORTED;
  const int32_t* in[] = {c.table, c.length, c.ref};
  const int32_t* out[] = {c.table_out, c.length_out, c.ref_out};
  const long long size[] = {static_cast<long long>(c.seqs) * c.width, c.seqs, c.pages};
  for (int i = 0; i < 3; i++) {
    if (in[i] == nullptr || out[i] == nullptr || !aligned4(in[i]) || !aligned4(out[i]))
      return AVSA_ERR_INVALID_ARG;
    for (int j = 0; j < 3; j++) {
      if (i == j && in[i] == out[i]) continue;
      if (!apart(out[i], size[i], in[j], size[j]) || (i < j && !apart(out[i], size[i], out[j], size[j]))) return AVSA_ERR_INVALID_ARG;
    }
  }
  return AVSA_OK;
}
// An output of n ints shares nothing with the state that the call reads or writes.
static bool apart_from_state(const avsa_cache& c, const int32_t* p, long long n) {
  const long long entries = static_cast<long long>(c.seqs) * c.width;
  return apart(p, n, c.table, entries) && apart(p, n, c.table_out, entries) && apart(p, n, c.length, c.seqs) && apart(p, n, c.length_out, c.seqs) &&
         apart(p, n, c.ref, c.pages) && apart(p, n, c.ref_out, c.pages);
}
static int check_list(const avsa_cache& c, const int32_t* a, const int32_t* b, int n, const void* ws, size_t ws_bytes,
                      bool by_page = true) {
  const int st = check_cache(c, by_page);
  if (st != AVSA_OK) return st;
  if (n < 0 || (n > 0 && (a == nullptr || b == nullptr)) || !aligned4(a) || !aligned4(b)) return AVSA_ERR_INVALID_ARG;
  if (ws == nullptr || ws_bytes < CacheWs::bytes(c.seqs, c.pages, n)) return AVSA_ERR_WORKSPACE;
  if (!ws_aligned(ws, kWsVectors)) return AVSA_ERR_INVALID_ARG;
  return AVSA_OK;
}
static int check_log(const avsa_cache& c, const int32_t* log) {
  return log == nullptr || (aligned4(log) && apart_from_state(c, log, 4)) ? AVSA_OK : AVSA_ERR_INVALID_ARG;
}
static int check_pool(const avsa_pages& p, int pages) {
  if (p.ptr == nullptr || !aligned16(p.ptr) || p.planes <= 0 || p.page_bytes <= 0 || p.page_bytes % 16 != 0) return AVSA_ERR_INVALID_ARG;
  if (pages > 1 && (p.stride_page < p.page_bytes || p.stride_page % 16 != 0)) return AVSA_ERR_INVALID_ARG;
  if (p.planes > 1 && (p.stride_plane <= 0 || p.stride_plane % 16 != 0)) return AVSA_ERR_INVALID_ARG;
  return AVSA_OK;
}

static unsigned meta_cluster(const avsa_cache& c) {
  long long ints = c.pages;
  if (c.table != c.table_out) ints += static_cast<long long>(c.seqs) * c.width;
  return ints <= kMetaSingle ? 1u : static_cast<unsigned>(kMetaCluster);
}
// `most`: the largest `smem` of any call of the kernel.  The limit belongs to the kernel, not to the call: host threads with pools of different sizes would lower it
// for one another between setting it and the launch, so all of them set the same.
static cudaError_t launch_meta(void (*kernel)(MetaArgs), const MetaArgs& a, cudaStream_t st, size_t smem = 0, size_t most = 0) {
  const unsigned ctas = meta_cluster(a.c);
  if (ctas > 1) smem = 0;
  if (smem + kScanBytes > 48 * 1024) {
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(most));
    if (e != cudaSuccess) return e;
  }
  return launch_pdl_clusters(kernel, ctas, ctas, kMetaThreads, smem, st, a);
}
static int launch_moves(const CopyArgs& a, long long most, cudaStream_t st) {
  const long long chunks = (a.pool.page_bytes + kCopyChunk - 1) / kCopyChunk;
  long long want = most * a.pool.planes * chunks;
  if (a.table != nullptr) {
    const long long rows = (static_cast<long long>(a.seqs) * a.width + kCopyThreads - 1) / kCopyThreads;
    want = want > rows ? want : rows;
  }
  const int grid = persistent_grid(1 << 30) * 8;
  return launch_pdl(move_pages_kernel, static_cast<unsigned>(want < grid ? want : grid), kCopyThreads, 0, st, a) == cudaSuccess ? AVSA_OK
                                                                                                                     : AVSA_ERR_CUDA;
}
static int done() { return cudaGetLastError() == cudaSuccess ? AVSA_OK : AVSA_ERR_CUDA; }

}  // namespace avsa

using namespace avsa;

extern "C" size_t avsa_cache_workspace_bytes(int seqs, int pages, int n) {
  if (seqs <= 0 || pages <= 0 || n < 0) return 0;
  return CacheWs::bytes(seqs, pages, n);
}

extern "C" int avsa_cache_extend_step(avsa_cache c, const int32_t* seq, const int32_t* count, int n, int32_t* granted, int32_t* log, void* ws,
                                      size_t ws_bytes, void* stream) {
  int st = check_list(c, seq, count, n, ws, ws_bytes);
  if (st == AVSA_OK) st = check_log(c, log);
  if (st != AVSA_OK) return st;
  if (granted != nullptr) {
    if (!aligned4(granted) || !apart_from_state(c, granted, n) || !apart(granted, n, seq, n) || !apart(granted, n, count, n)) return AVSA_ERR_INVALID_ARG;
  }
  if (!device_is_sm100()) return AVSA_ERR_UNSUPPORTED;
  const MetaArgs a = {c, CacheWs(ws, c.seqs, c.pages, n), seq, count, n, nullptr, granted, log};
  if (launch_meta(assign_pages_kernel<kExtend>, a, as_stream(stream), AssignSmem(c, n).bytes, kAssignMost) != cudaSuccess) return AVSA_ERR_CUDA;
  return done();
}

extern "C" int avsa_cache_extend(avsa_cache c, const int32_t* seq, const int32_t* count, int n, void* ws, size_t ws_bytes, void* stream) {
  return avsa_cache_extend_step(c, seq, count, n, nullptr, nullptr, ws, ws_bytes, stream);
}

extern "C" int avsa_cache_fork_step(avsa_cache c, avsa_pages pool, const int32_t* parent, const int32_t* child, int n, int32_t* log, void* ws,
                                    size_t ws_bytes, void* stream) {
  int st = check_list(c, parent, child, n, ws, ws_bytes);
  if (st == AVSA_OK) st = check_pool(pool, c.pages);
  if (st == AVSA_OK) st = check_log(c, log);
  if (st != AVSA_OK) return st;
  if (!device_is_sm100()) return AVSA_ERR_UNSUPPORTED;
  const MetaArgs a = {c, CacheWs(ws, c.seqs, c.pages, n), child, parent, n, nullptr, nullptr, log};
  if (launch_meta(assign_pages_kernel<kFork>, a, as_stream(stream), AssignSmem(c, n).bytes, kAssignMost) != cudaSuccess) return AVSA_ERR_CUDA;
  if (n > 0) {
    CopyArgs m = {};
    m.pool = pool;
    m.moves = a.w.moves;
    m.n = n;
    m.status = a.w.status;
    m.log = log;
    if (launch_moves(m, n, as_stream(stream)) != AVSA_OK) return AVSA_ERR_CUDA;
  }
  return done();
}

extern "C" int avsa_cache_fork(avsa_cache c, avsa_pages pool, const int32_t* parent, const int32_t* child, int n, void* ws, size_t ws_bytes,
                               void* stream) {
  return avsa_cache_fork_step(c, pool, parent, child, n, nullptr, ws, ws_bytes, stream);
}

extern "C" int avsa_cache_free_step(avsa_cache c, const int32_t* seq, int n, int32_t* log, void* ws, size_t ws_bytes, void* stream) {
  int st = check_list(c, seq, seq, n, ws, ws_bytes, false);
  if (st == AVSA_OK) st = check_log(c, log);
  if (st != AVSA_OK) return st;
  if (!device_is_sm100()) return AVSA_ERR_UNSUPPORTED;
  const MetaArgs a = {c, CacheWs(ws, c.seqs, c.pages, n), seq, nullptr, n, nullptr, nullptr, log};
  if (launch_meta(free_pages_kernel, a, as_stream(stream)) != cudaSuccess) return AVSA_ERR_CUDA;
  return done();
}

extern "C" int avsa_cache_free(avsa_cache c, const int32_t* seq, int n, void* ws, size_t ws_bytes, void* stream) {
  return avsa_cache_free_step(c, seq, n, nullptr, ws, ws_bytes, stream);
}

extern "C" int avsa_cache_compact_step(avsa_cache c, avsa_pages pool, int32_t* n_live, int32_t* log, void* ws, size_t ws_bytes, void* stream) {
  int st = check_list(c, nullptr, nullptr, 0, ws, ws_bytes);
  if (st == AVSA_OK) st = check_pool(pool, c.pages);
  if (st == AVSA_OK) st = check_log(c, log);
  if (st != AVSA_OK) return st;
  if (n_live == nullptr || !aligned4(n_live)) return AVSA_ERR_INVALID_ARG;
  if (!device_is_sm100()) return AVSA_ERR_UNSUPPORTED;
  const MetaArgs a = {c, CacheWs(ws, c.seqs, c.pages, 0), nullptr, nullptr, 0, n_live, nullptr, log};
  if (launch_meta(plan_compaction_kernel, a, as_stream(stream), most_moves(c) * kMoveBytes, kPlanMost) != cudaSuccess) return AVSA_ERR_CUDA;
  CopyArgs m = {};
  m.pool = pool;
  m.moves = a.w.moves;
  m.n_moves = a.w.counts + kNumMoves;
  m.table = c.table;
  m.table_out = c.table_out;
  m.place = a.w.free_pages;
  m.n_live = n_live;
  m.seqs = c.seqs;
  m.width = c.width;
  m.pages = c.pages;
  m.status = a.w.status;
  m.log = log;
  if (launch_moves(m, c.pages, as_stream(stream)) != AVSA_OK) return AVSA_ERR_CUDA;
  return done();
}

extern "C" int avsa_cache_compact(avsa_cache c, avsa_pages pool, int32_t* n_live, void* ws, size_t ws_bytes, void* stream) {
  return avsa_cache_compact_step(c, pool, n_live, nullptr, ws, ws_bytes, stream);
}

extern "C" int avsa_cache_write(int n, int Hkv, int L, int d, int page, int pages, int seqs, int width, avsa_bf16_4d k_new,
                                avsa_bf16_4d v_new, avsa_bf16_4d k_pool, avsa_bf16_4d v_pool, const int32_t* table,
                                const int32_t* length, const int32_t* seq, const int32_t* count, void* stream) {
  if (n < 0 || Hkv <= 0 || L < 0 || pages <= 0 || seqs <= 0 || width <= 0) return AVSA_ERR_INVALID_ARG;
  if ((d != 64 && d != 128) || !page_size_ok(page) || n > 65535 || Hkv > 65535 || static_cast<long long>(seqs) * width > INT_MAX) return AVSA_ERR_UNSUPPORTED;
  if (seq == nullptr && n > seqs) return AVSA_ERR_INVALID_ARG;
  if (table == nullptr || length == nullptr || !tensor_ok(k_pool, pages, Hkv) || !tensor_ok(v_pool, pages, Hkv)) return AVSA_ERR_INVALID_ARG;
  if (!aligned4(table) || !aligned4(length) || !aligned4(seq) || !aligned4(count)) return AVSA_ERR_INVALID_ARG;
  if (n == 0 || L == 0) return AVSA_OK;
  if (!tokens_ok(k_new, n, Hkv, L) || !tokens_ok(v_new, n, Hkv, L)) return AVSA_ERR_INVALID_ARG;
  if (!device_is_sm100()) return AVSA_ERR_UNSUPPORTED;
  WriteArgs a = {k_new, v_new, k_pool, v_pool, table, length, seq, count, Hkv, L, d == 128 ? 4 : 3, 0, 0, 0, pages, seqs, width};
  while ((1 << a.page_shift) < page) a.page_shift++;
  // eight tokens (as many as there are), and as many heads as make four vectors a thread
  const int vecs = kCopyThreads * kWriteVecs >> a.vec_shift;
  a.tokens = L < 8 ? L : 8;
  while (a.tokens << (a.head_shift + 1) <= vecs && (1 << a.head_shift) < Hkv) a.head_shift++;
  a.tokens = vecs >> a.head_shift;
  const dim3 grid(static_cast<unsigned>((L + a.tokens - 1) / a.tokens), static_cast<unsigned>((Hkv + (1 << a.head_shift) - 1) >> a.head_shift),
                  static_cast<unsigned>(n));
  if (launch_pdl(write_tokens_kernel, grid, kCopyThreads, 0, as_stream(stream), a) != cudaSuccess) return AVSA_ERR_CUDA;
  return done();
}
