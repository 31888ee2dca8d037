// Attention over a paged cache: the tile kernel, and the kernel that joins what it has cut.
//
// A tile is 128 query rows against 128 keys of one key/value head.  Query rows are all that share keys: the L queries times the G query heads of
// that key head (row i*G + g of a batch entry), and, over the beginning that the whole batch shares, those of all batch
// entries one after the other ("stacked").  One token of 64 sequences with 4 query heads to a key head makes 4 rows a sequence, which leave 124 rows of a
// tile empty, but 256 rows stacked: the beginning is read twice instead of 64 times, and the tensor cores work on full tiles.
//
// Work.  An item is a row tile with all its keys; its key tiles, and a few more for what an item costs by itself, are units.  Which units a CTA takes:
//   - prefix pieces: the key tiles of the beginning, head after head, are one stream of columns; `chunk` row tiles go through it side by side (a CTA each, so that
//     the second reader of a key tile finds it in L2), and each group of `chunk` CTAs gets the same number of columns;
//   - B pieces: the own items of all sequences, one after the other, are a stream that is cut into equal pieces: lengths as ragged as they may be,
//     every CTA gets the same number of units, and all of them stream pages from HBM side by side;
//   - A pieces: with several row tiles to a sequence (long blocks of queries) and more keys than L2 keeps, whole items come off a queue, so that CTAs that run at the
//     same time work on the same keys (as equal shares of the stream they would be heads apart: each tile from HBM), and only last ones that are few are cut.
// What a cut or a stacked item leaves are fp32 rows, normalised by their own sum, and their log2 sums; prefix_merge_kernel joins them in a fixed order.
// Lengths are on the device: every CTA's scheduler warp counts the units itself (a scan over the batch), nothing comes back to the host.
//
// Pipeline (one persistent CTA per SM): as in attn_persist_kernel.cuh, whose softmax against one fixed reference per row this is:
// K and V tiles through two rings of TMA loads, here page by page (a page id beyond the pool reads as zeros: what lies behind the
// last page), S = Q K^T and O += P V by tcgen05 from two issuing warps, two softmax groups of four warps on alternate key tiles.  The query rows of an item are a
// box of (heads, tokens, batch entries) where the sizes allow it, else two warps gather them with cp.async (1500 cycles more).  An item with a row that outgrew its reference runs again
// in the same CTA: once for the row maxima alone, once with these as the references.
//
// Bound by the exponentials (1024 cycles of a tile) and the products (1024 with 128 channels) in turn, 1450 cycles a tile, and by 4000 cycles an item for its query rows, first
// maxima and epilogue: 4 x 1560 queries of 24 heads against 13976 keys each, 128 channels, 880 us (1218 TFLOP/s, in a longer loop under the power limit 1060); 148 x 8 items of
// three tiles 64 us.
#pragma once
#include <math.h>

#include "attn_persist_kernel.cuh"

namespace avsa {

constexpr int kPxThreads = 512;
// 512 x 128 registers at launch; then 8 service warps of 64 and 8 softmax warps of 192: 65536 both ways.
constexpr int kPxServiceRegs = 64, kPxSoftmaxRegs = 192;
static_assert(8 * 32 * kPxServiceRegs + 8 * 32 * kPxSoftmaxRegs <= kPxThreads * 128, "setmaxnreg budget exceeded");
constexpr int kPxRing = 4, kPxRedo = 14;
constexpr int kPxQWarps = 2;             // warps 13 and 14 gather query rows
constexpr int kPxConsumers = 4 + kPxQWarps + 8;      // warps that read the item ring

enum PrefixWhere {
  kPrefixPage = 221, kPrefixLength, kPrefixSeq, kPxItem, kPxItemEmpty, kPxQEmpty, kPxQFull, kPxKEmpty, kPxVEmpty, kPxKFull, kPxVFull, kPxSFull, kPxSFree,
  kPxPFull, kPxPFree, kPxOFull, kPxOFree, kPxMref, kPxLsum, kPxAlign, kPrefixCount
};

// A divisor known on the host: n / d for 0 <= n < 2^31 without a division (which is 30 dependent instructions).
struct Divisor {
  uint32_t d, mul, shift;
  __host__ __device__ Divisor() {}
  __host__ explicit Divisor(int n) : d(static_cast<uint32_t>(n)), mul(0), shift(31) {
    while ((1ull << (shift - 31)) < d) shift++;
    mul = static_cast<uint32_t>(((1ull << shift) + d - 1) / d);
  }
  __device__ __forceinline__ int div(int n) const { return static_cast<int>((static_cast<uint64_t>(static_cast<uint32_t>(n)) * mul) >> shift); }
};
// One that is not: the quotient of floats, put right.
__device__ __forceinline__ int float_div(int a, int b) {
  int q = __float2int_rz(__fdividef(static_cast<float>(a), static_cast<float>(b)));
  int r = a - q * b;
  while (r < 0) q--, r += b;
  while (r >= b) q++, r -= b;
  return q;
}

// What of the work depends on sizes alone.
struct PrefixShape {
  int B, Hkv, G, L;
  int R;               // query rows of a batch entry and key head: L*G
  int TO, F;           // row tiles of these, and of the whole batch (F = B*TO)
  int stack;           // the beginning's pages are read for the stacked rows
  int k0;              // first key of the own items: 0, or behind the beginning
  int TP, chunk, nrc;  // row tiles of the stacked rows, taken `chunk` at a time (nrc times)
  int rows;            // rows of an own item's partial result: min(128, R)
  int queue;           // whole items off a queue
  int own_off;         // the beginning alone: the own items are another kernel's
  int cg;              // columns of a group then (as if all sequences had the whole beginning)
  int pre_box, own_box;        // rows of the TMA box that holds the query rows of an item; 0: they are gathered
  int nb_max;          // B pieces at most
  int page, page_shift, pages, seqs, width;
  int causal;
  Divisor by_R, by_G, by_TO, by_F, by_chunk, by_nrc, by_cg;
};

struct PrefixParams {
  PrefixShape s;
  avsa_bf16_4d q;
  __nv_bfloat16* o;
  float* lse;
  const int32_t *table, *length, *seq;
  const int32_t* count;        // queries of a batch entry, or NULL: L
  float scale_log2;
  // workspace
  StatusRecord* status;
  int32_t* log;        // the caller's record of the first error, or NULL
  int* counter;        // head of the queue
  int* plan;           // for the merge: PT, columns a group, B pieces
  int4* cta_err;       // [2 * CTAs]: code, where, item, aux; recomputed items
  int2* own_rec;       // stack: [Hkv*F] first B piece and number of parts of an own item
  int2* cut_rec;       // else: [nb_max] the item that a B piece begins and does not end, and its number of parts
  float* part_o;       // [rows][D]: prefix slots of 128 rows, own items (stack), two cut ends a B piece
  float* part_lse2;
  int own_row0, cut_row0;      // first rows of the latter two
  int tile_ctas;       // CTAs of the tile kernel
  struct PrefixItem* redo;     // [CTAs][kPxRedo] items to run again
};

struct PrefixItem {
  int type;            // -1: no more; bit 0: stacked rows, bits 1-2: 0, or 1 maxima only, 2 with given maxima
  int b, hk, row0, nrows;
  int pos0, cnt, kv_end;       // first key, key tiles, end of the keys
  int slot;            // row of the page table
  int len;             // own items: tokens of the sequence
  int out;             // first partial row, -1: final rows
  int pad;
};
static_assert(sizeof(PrefixItem) == 48, "three 16-byte accesses");

// Words of the CTA's `misc`.
enum { kPxTmem = 0, kPxStop, kPxWhere, kPxProgress, kPxFlag /* + item parity */, kPxListed = kPxFlag + 2, kPxRecomputed, kPxErr, kPxWords = kPxErr + 4 };

template <int D>
struct PrefixSmem {
  static constexpr int kTile = 128 * D * 2;
  static constexpr int kKS = D == 128 ? 3 : 6, kVS = D == 128 ? 3 : 6;
  // (64 channels: two buffers of query rows)
  static constexpr int kQ = 0, kQSlot = D == 64 ? 16384 : 0;
  static constexpr int kK = 32768;
  static constexpr int kV = kK + kKS * kTile;
  static constexpr int kBars = kV + kVS * kTile;
  static constexpr int kNumBars = 4 + 2 * kKS + 2 * kVS + 13 + 2 * kPxRing + 6;
  static constexpr int kStats = (kBars + kNumBars * 8 + 15) / 16 * 16;       // float mref[128], lsum[2][128]
  static constexpr int kItems = kStats + 3 * 128 * 4;
  static constexpr int kPages = kItems + 48 * kPxRing;                        // int[kPxRing][32]: an item's first pages
  static constexpr int kMisc = kPages + 128 * kPxRing;
  static constexpr int kTotal = kMisc + 48;
  static_assert(kPxWords * 4 <= 48, "words of the CTA");
  static_assert(kTotal <= 232448, "shared memory of a CTA exceeded");
};

// ------------------------------------------------------------------------------------------------ sizes on the device
// Table row of a batch entry (-1: none) and its tokens.  `bad`: what is out of range.
__device__ __forceinline__ int prefix_sequence(const PrefixParams& p, int b, int& slot, int& bad) {
  const int s = p.seq != nullptr ? p.seq[b] : b;
  slot = s < 0 || s >= p.s.seqs ? -1 : s;
  bad = s >= p.s.seqs ? kPrefixSeq : 0;
  if (slot < 0) return 0;
  const int n = p.length[slot], most = p.s.width << p.s.page_shift;
  if (n < 0 || n > most) bad = kPrefixLength;
  if (p.count != nullptr && (p.count[b] < 0 || p.count[b] > p.s.L)) bad = kPrefixCount;
  return n < 0 ? 0 : n > most ? most : n;
}
// Queries of a batch entry that are tokens of its sequence, its last ones.
__device__ __forceinline__ int prefix_queries(const PrefixParams& p, int b) {
  return p.count != nullptr ? min(max(p.count[b], 0), p.s.L) : p.s.L;
}
// How many of the n tokens of its sequence query i of batch entry b sees (less than one: none).
__device__ __forceinline__ int prefix_limit(const PrefixParams& p, int b, int n, int i) {
  if (!p.s.causal) return n;
  const int q = prefix_queries(p, b);
  return i < q ? n - q + i + 1 : 0;
}
// Key tiles of an own item: row tile rt of batch entry b, whose sequence has n tokens.
__device__ __forceinline__ int prefix_own_tiles(const PrefixParams& p, int b, int n, int rt) {
  const PrefixShape& s = p.s;
  if (s.own_off) return 0;
  int end = n;
  if (s.causal) {
    const int q = prefix_queries(p, b);
    end = s.by_G.div(rt * 128) < q ? n - q + min(q, s.by_G.div(rt * 128 + 127) + 1) : 0;
  }
  const int x = end - s.k0;
  const int t = x > 0 ? (x + 127) >> 7 : 0;
  return s.stack ? t : max(t, 1);      // (without a beginning of its own every row tile is written by somebody)
}

__device__ __forceinline__ void cp_async_16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(reinterpret_cast<uint64_t>(src)) : "memory");
}

constexpr int kPxMinPiece = 4;       // units: a CTA with fewer ends later than one that takes another's as well
// Units that an own item counts for beyond its key tiles, in front of them: what it costs apart from these (3 sequences of 500 to 9000 tokens under 300
// queries each, us: 102 without, 82 with them; two or four instead of three are within 3 %).
constexpr int kPxItemUnits = 3;

// How the units are cut: the same in every CTA.
struct PrefixPlan {
  int PT, PE, donor;           // key tiles and tokens of the beginning, the table row that names its pages
  int cg, groups;              // columns of a group
  int W, MA, uA;               // units of a key head; items of the queue, their units
  int TB, sB, NB;              // units of the B pieces, of one, pieces
};

// The CTA's first error, for the merge kernel to report.  (Not inlined: a call's first items run through cold code, and what stands between the lines that
// they need is fetched with them.)
__device__ __noinline__ void px_report(int* err, int code, int where, int item, int aux) {
  if (atomicCAS(err, 0, code) == 0) {
    err[1] = where;
    err[2] = item;
    err[3] = aux;
  }
}

template <int D>
__global__ void __launch_bounds__(kPxThreads, 1)
prefix_attn_kernel(const __grid_constant__ CUtensorMap tmk, const __grid_constant__ CUtensorMap tmv, const __grid_constant__ CUtensorMap tmq_own,
                   const __grid_constant__ CUtensorMap tmq_pre, const __grid_constant__ CUtensorMap tmo, const __grid_constant__ PrefixParams p) {
  using L_ = PrefixSmem<D>;
  constexpr int NPANEL = D / 64, PANEL = 128 * 128, KS = L_::kKS, VS = L_::kVS;
  constexpr unsigned FULLM = 0xffffffffu;
  extern __shared__ __align__(1024) uint8_t smem[];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const PrefixShape& S = p.s;

  const uint32_t bar0 = smem_u32(smem + L_::kBars);
  auto BAR = [&](int i) { return bar0 + static_cast<uint32_t>(i) * 8u; };
  constexpr int Q_FULL = 0, Q_EMPTY = 2, K_FULL = 4, K_EMPTY = K_FULL + KS, V_FULL = K_EMPTY + KS, V_EMPTY = V_FULL + VS,
                S_FULL = V_EMPTY + VS, S_FREE = S_FULL + 2, P_FULL = S_FREE + 2 /* + 2*group + half */, P_FREE = P_FULL + 4, O_FULL = P_FREE + 2,
                O_FREE = O_FULL + 1, MREF = O_FREE + 1, ITEM_FULL = MREF + 1, ITEM_EMPTY = ITEM_FULL + kPxRing, QK_DRAIN = ITEM_EMPTY + kPxRing,
                PV_DRAIN = QK_DRAIN + 1, LSUM_A = PV_DRAIN + 1, LSUM_B = LSUM_A + 1, STAGED = LSUM_B + 1,
                DONE = STAGED + 1;
  static_assert(DONE + 1 <= L_::kNumBars, "barrier table too small");
  constexpr uint32_t TM_O = 256, TM_P = 256 + D;      // tensor memory: S of group 0 | S of group 1 | O | P of group 0 | P of group 1
  float* mref_s = reinterpret_cast<float*>(smem + L_::kStats);
  float* lsum_s = mref_s + 128;
  PrefixItem* ring = reinterpret_cast<PrefixItem*>(smem + L_::kItems);
  int* ring_pages = reinterpret_cast<int*>(smem + L_::kPages);
  PrefixItem* redo = p.redo + blockIdx.x * kPxRedo;
  volatile int* misc = reinterpret_cast<volatile int*>(smem + L_::kMisc);

  const bool aligned = (smem_u32(smem) & 1023u) == 0u;
  if (tid == 0) {
    for (int s = 0; s < 2; s++) {
      mbar_init(BAR(Q_FULL + s), 32 * kPxQWarps);
      mbar_init(BAR(Q_EMPTY + s), 1);
    }
    for (int s = 0; s < KS; s++) {
      mbar_init(BAR(K_FULL + s), 1);
      mbar_init(BAR(K_EMPTY + s), 1);
    }
    for (int s = 0; s < VS; s++) {
      mbar_init(BAR(V_FULL + s), 1);
      mbar_init(BAR(V_EMPTY + s), 1);
    }
    for (int g = 0; g < 2; g++) {
      mbar_init(BAR(S_FULL + g), 1);
      mbar_init(BAR(S_FREE + g), 128);
      mbar_init(BAR(P_FULL + 2 * g), 128);
      mbar_init(BAR(P_FULL + 2 * g + 1), 128);
      mbar_init(BAR(P_FREE + g), 1);
    }
    for (int r = 0; r < kPxRing; r++) {
      mbar_init(BAR(ITEM_FULL + r), 1);
      mbar_init(BAR(ITEM_EMPTY + r), kPxConsumers);
    }
    mbar_init(BAR(O_FULL), 1);
    mbar_init(BAR(O_FREE), 256);
    mbar_init(BAR(MREF), 128);
    mbar_init(BAR(QK_DRAIN), 1);
    mbar_init(BAR(PV_DRAIN), 1);
    mbar_init(BAR(LSUM_A), 256);
    mbar_init(BAR(LSUM_B), 256);
    mbar_init(BAR(STAGED), 256);
    mbar_init(BAR(DONE), 1);
    for (int i = kPxStop; i < kPxWords; i++) misc[i] = 0;
    fence_mbar_init();
    prefetch_tmap(&tmk);
    prefetch_tmap(&tmv);
    prefetch_tmap(&tmq_own);
    if (S.stack) prefetch_tmap(&tmq_pre);
  }
  if (warp == 2) {
    tmem_alloc(smem_u32(smem + L_::kMisc), 512);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = misc[kPxTmem];
  pdl_wait();
  pdl_launch();

  // Final rows go out through shared memory, 128-byte swizzled, and a TMA store where they are a box (16-byte stores by row took 2000 cycles an item; 128 channels,
  // 1024 items, us: of one key tile 69 by row, 46 by box, of eight 98 and 94); its place is the last V stage, which such a call does without.
  const bool staging = S.own_box > 0 && !S.own_off && !S.stack;
  const int n_vs = staging ? VS - 1 : VS;
  uint8_t* const stage_out = smem + L_::kV + (VS - 1) * L_::kTile;
  auto report = [&](int code, int where, int item, int aux) { px_report(const_cast<int*>(misc) + kPxErr, code, where, item, aux); };
  // A wait is as few instructions as it can be: an item runs through a dozen of them, and items of few tiles are short of instructions (the SM's cache holds less than the
  // roles' code: a third of its lookups missed with 3 tiles to an item).  So no wait looks at the clock; the watch of warp 15 sets the word that ends them all.
  auto wait_or_stop = [&](int bar, uint32_t parity, int where) -> bool {
    while (!mbar_try_wait(BAR(bar), parity))
      if (misc[kPxStop] != 0) {
        misc[kPxWhere] = where;
        return false;
      }
    return true;
  };
  // The warps that load ahead wait most of the time, for a place: with sleeps between their looks the others have the issue slots (frames of 4 candidates, us: 952, with
  // sleeps 880).
  auto wait_idly = [&](int bar, uint32_t parity, int where) -> bool {
    while (!mbar_try_wait(BAR(bar), parity)) {
      if (misc[kPxStop] != 0) {
        misc[kPxWhere] = where;
        return false;
      }
      __nanosleep(64);
    }
    return true;
  };
  auto wait_all = [&](int bar, uint32_t parity, int where) -> bool { return __all_sync(FULLM, wait_or_stop(bar, parity, where)); };
  auto get_item = [&](int n, PrefixItem& it) -> bool {     // false: stopped, or no more items
    const int slot = n % kPxRing;
    if (!wait_all(ITEM_FULL + slot, (n / kPxRing) & 1, kPxItem)) return false;
    it = ring[slot];
    return it.type >= 0;
  };
  auto item_done = [&](int n) {
    __syncwarp();
    if (lane == 0) mbar_arrive(BAR(ITEM_EMPTY + n % kPxRing));
  };

  // (every role changes its registers by itself, as its first step: the compiler goes by that)
  if (!aligned) {
    if (tid == 0) report(AVSA_ERR_CUDA, kPxAlign, blockIdx.x, 0);
    if (tid == 0 && blockIdx.x == 0) p.plan[0] = p.plan[2] = 0;
  } else if (warp == 0 || warp == 12) {
    // ------------------------------------------------------------------ TMA producers: warp 0 K, warp 12 V
    asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
    const bool is_k = warp == 0;
    const CUtensorMap* tm = is_k ? &tmk : &tmv;
    const int FULL = is_k ? K_FULL : V_FULL, EMPTY = is_k ? K_EMPTY : V_EMPTY, STAGES = is_k ? KS : n_vs;
    const uint32_t base = smem_u32(smem + (is_k ? L_::kK : L_::kV));
    const int ppt_shift = 7 - S.page_shift, ppt = 1 << ppt_shift;      // pages of a tile
    int stage = 0, round = 0, loads = 0;
    bool ok = true;
#pragma unroll 1
    for (int n = 0; ok; n++) {
      PrefixItem it;
      if (!get_item(n, it)) break;
      if (is_k || (it.type >> 1) != 1) {
        const int32_t* row = p.table + static_cast<int64_t>(max(it.slot, 0)) * S.width;
        const int e0 = it.pos0 >> S.page_shift;      // its pages
        const int e1 = min(e0 + (it.cnt << ppt_shift), (it.kv_end + S.page - 1) >> S.page_shift);
        const int per = 32 >> ppt_shift;       // tiles whose pages a warp holds at once; the first come with the item
        int mine = ring_pages[(n % kPxRing) * 32 + lane];
#pragma unroll 1
        for (int t0 = 0; t0 < it.cnt && ok; t0 += per) {
          int next = S.pages;                  // behind the last page: beyond the pool, where the copy reads zeros
          const int e = e0 + ((t0 + per) << ppt_shift) + lane;
          if (e < e1) next = row[e];
          const int nn = min(per, it.cnt - t0);
#pragma unroll 1
          for (int j = 0; j < nn; j++) {
            const int id = __shfl_sync(FULLM, mine, (j << ppt_shift) + (lane & (ppt - 1)));
            int good = 1;
            if (lane == 0) {
              if (round > 0) good = wait_idly(EMPTY + stage, (round - 1) & 1, is_k ? kPxKEmpty : kPxVEmpty) ? 1 : 0;
              if (good) mbar_expect_tx(BAR(FULL + stage), L_::kTile);
            }
            good = __shfl_sync(FULLM, good, 0);
            if (!good) {
              ok = false;
              break;
            }
            if (lane < ppt * NPANEL) {
              const int panel = lane >> ppt_shift, in = lane & (ppt - 1);
              tma_load_4d(base + stage * L_::kTile + panel * PANEL + ((in << S.page_shift) << 7), tm, BAR(FULL + stage), panel * 64, 0, it.hk, id);
            }
            __syncwarp();
            loads++;
            if (is_k && lane == 0) misc[kPxProgress] = loads;
            if (++stage == STAGES) {
              stage = 0;
              round++;
            }
          }
          if (next < 0 || next > S.pages) {
            report(AVSA_ERR_BAD_TABLE, kPrefixPage, it.slot, e);
            next = S.pages;
          }
          mine = next;
        }
      }
      if (ok) item_done(n);
    }
    if (lane == 0 && misc[kPxStop] != 0)      // loads still in flight must land before this CTA's shared memory is given away
      for (int c = max(0, loads - STAGES); c < loads; c++) mbar_wait(BAR(FULL + c % STAGES), (c / STAGES) & 1);
  } else if (warp == 13 || warp == 14) {
    // ------------------------------------------------------------------ query rows into shared memory, 128-byte swizzled like a TMA tile
    asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
    constexpr int VPR = D / 8, RPI = 32 / VPR;      // 16-byte vectors of a row; rows of an instruction
    const uint32_t base = smem_u32(smem + L_::kQ);
    int q_loads = 0;          // items up to the last one whose rows came by TMA
    bool ok = true;
#pragma unroll 1
    for (int n = 0; ok; n++) {
      PrefixItem it;
      if (!get_item(n, it)) break;
      if (n >= 2) ok = __all_sync(FULLM, wait_idly(Q_EMPTY + (n & 1), ((n >> 1) - 1) & 1, kPxQEmpty));
      if (ok && n >= 1 && L_::kQSlot == 0) ok = __all_sync(FULLM, wait_idly(Q_EMPTY + ((n - 1) & 1), ((n - 1) >> 1) & 1, kPxQEmpty));      // one buffer
      if (!ok) break;
      const uint32_t dst = base + (n & 1) * L_::kQSlot;
      const bool stacked = (it.type & 1) != 0;
      const int box = stacked ? S.pre_box : S.own_box;
      if (box > 0) {
        if (warp == 13 && lane == 0) {
          mbar_expect_tx(BAR(Q_FULL + (n & 1)), box * 128 * NPANEL);
          const int token = stacked ? 0 : S.by_G.div(it.row0), entry = stacked ? S.by_R.div(it.row0) : it.b;
          for (int pn = 0; pn < NPANEL; pn++)
            tma_load_4d(dst + pn * PANEL, stacked ? &tmq_pre : &tmq_own, BAR(Q_FULL + (n & 1)), pn * 64, it.hk * S.G, token, entry);
        } else {
          mbar_arrive(BAR(Q_FULL + (n & 1)));
        }
        q_loads = n + 1;
        item_done(n);
        continue;
      }
#pragma unroll 1
      for (int r0 = (warp - 13) * 32; r0 < it.nrows; r0 += 32 * kPxQWarps) {
        int64_t off = 0;
        if (r0 + lane < it.nrows) {
          int rr = it.row0 + r0 + lane, b = it.b;
          if (it.type & 1) {
            b = S.by_R.div(rr);
            rr -= b * S.R;
          }
          const int i = S.by_G.div(rr), g = rr - i * S.G;
          off = b * p.q.stride_b + (it.hk * S.G + g) * p.q.stride_h + i * p.q.stride_n;
        }
        const int rows = min(32, it.nrows - r0);
#pragma unroll 1
        for (int k = 0; k < rows; k += RPI) {
          const int rl = k + lane / VPR, c = lane % VPR;
          const int64_t o = __shfl_sync(FULLM, off, rl & 31);
          const int r = r0 + rl;
          if (rl < rows)
            cp_async_16(dst + (c >> 3) * PANEL + r * 128 + (((c & 7) ^ (r & 7)) << 4), static_cast<const __nv_bfloat16*>(p.q.ptr) + o + c * 8);
        }
      }
      asm volatile("cp.async.wait_all;" ::: "memory");
      fence_proxy_async();
      mbar_arrive(BAR(Q_FULL + (n & 1)));
      item_done(n);
    }
    if (misc[kPxStop] != 0)
      for (int c = max(0, q_loads - 2); c < q_loads; c++) mbar_wait(BAR(Q_FULL + (c & 1)), (c >> 1) & 1);
  } else if (warp == 3) {
    // ------------------------------------------------------------------ scheduler
    asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
    const int n_cta = gridDim.x;
    int published = 0;
    // The last published item, and all before it, are done.
    auto all_done = [&]() -> bool {
      const int m = published - 1;
      return m < 0 || wait_all(ITEM_EMPTY + m % kPxRing, (m / kPxRing) & 1, kPxItemEmpty);
    };
    auto publish = [&](const PrefixItem& it) -> bool {
      const int m = published, slot = m % kPxRing;
      int page = S.pages;
      const int e0 = it.pos0 >> S.page_shift, e = e0 + lane;
      if (e < min(e0 + (it.cnt << (7 - S.page_shift)), (it.kv_end + S.page - 1) >> S.page_shift)) {
        page = p.table[static_cast<int64_t>(it.slot) * S.width + e];
        if (page < 0 || page >= S.pages) {
          report(AVSA_ERR_BAD_TABLE, kPrefixPage, it.slot, e);
          page = S.pages;
        }
      }
      if (m >= kPxRing && !wait_all(ITEM_EMPTY + slot, ((m / kPxRing) - 1) & 1, kPxItemEmpty)) return false;
      ring_pages[slot * 32 + lane] = page;
      if (lane == 0) ring[slot] = it;
      __syncwarp();
      if (lane == 0) mbar_arrive(BAR(ITEM_FULL + slot));
      published++;
      return true;
    };
    // Publishes `it` (`last`: nothing), and in front of it, when the list is nearly full or this is the end, the items with a row that outgrew its reference again.
    auto emit = [&](const PrefixItem& it, bool last) -> bool {
      int again = 0;
      if (last || __shfl_sync(FULLM, misc[kPxListed], 0) >= kPxRedo - kPxRing - 1) {
        if (!all_done()) return false;
        again = __shfl_sync(FULLM, misc[kPxListed], 0);
        if (lane == 0) misc[kPxListed] = 0;
      }
      const int n = 2 * again + (last ? 0 : 1);
#pragma unroll 1
      for (int i = 0; i < n; i++) {
        PrefixItem x = it;
        if (i < 2 * again) {
          x = redo[i >> 1];
          x.type |= i & 1 ? 4 : 2;
        }
        if (!publish(x)) return false;
      }
      return again == 0 || !last || all_done();
    };
    // Lane l: the own item f0 + l of a key head.
    auto own_items = [&](int f0, int& nt, int& len, int& slot) {
      nt = len = 0;
      slot = -1;
      const int f = f0 + lane;
      if (f < S.F) {
        const int b = S.by_TO.div(f);
        int bad;
        len = prefix_sequence(p, b, slot, bad);
        if (bad && blockIdx.x == 0) report(AVSA_ERR_BAD_TABLE, bad, b, slot);
        nt = prefix_own_tiles(p, b, len, f - b * S.TO);
      }
    };
    auto scan = [&](int v) {      // of the lanes up to this one
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const int o = __shfl_up_sync(FULLM, v, d);
        if (lane >= d) v += o;
      }
      return v;
    };
    auto units = [](int nt) { return nt > 0 ? nt + kPxItemUnits : 0; };
    int nt0 = 0, len0 = 0, slot0 = -1;      // own_items(0)
    // ---- the plan
    PrefixPlan P = {};
    int n_pre = 0;
    bool queue = S.queue != 0;
    {
      int most = 0, at = 0, W = 0, tiles = 0;
#pragma unroll 1
      for (int f0 = 0; f0 < S.F; f0 += 32) {
        int nt, len, slot;
        own_items(f0, nt, len, slot);
        if (f0 == 0) nt0 = nt, len0 = len, slot0 = slot;
        W += units(nt);
        tiles += nt;
        if (len > most) most = len, at = slot;
      }
      P.W = __reduce_add_sync(FULLM, W);
      // keys and values that stay in L2 need no CTAs that work on the same ones (us, with them and without: the sequences of kPxItemUnits, 64 MB at most, 126 and 82;
      // 30000 tokens under 4096 queries, 123 MB, 1420 and 1566)
      const float bytes = static_cast<float>(__reduce_add_sync(FULLM, tiles)) * S.Hkv * (128.f * D * 4.f);
      queue = queue && bytes > static_cast<float>(kL2KeepBytes) * S.TO;
      if (S.stack) {
        const int top = __reduce_max_sync(FULLM, most);
        P.donor = __shfl_sync(FULLM, at, __ffs(__ballot_sync(FULLM, most == top)) - 1);
        P.PE = min(S.k0, top);
        P.PT = (P.PE + 127) >> 7;
        if (S.own_off) P.PT = (S.k0 + 127) >> 7;      // (a shorter one's last tiles read as zeros, and nobody sees them)
      }
      const int T = P.W * S.Hkv, columns = S.Hkv * S.nrc * P.PT;
      if (S.own_off) {
        P.cg = S.cg;
        P.groups = float_div(columns + P.cg - 1, P.cg);
        n_pre = P.groups * S.chunk;
      } else if (columns > 0) {
        const float share = static_cast<float>(S.Hkv) * S.TP * P.PT;
        // (with a queue rather one more than one less: who is done early takes more off it; 400 queries of
        // 16 sequences behind 30000 tokens, us: the nearest number 2555, the next one 2411; elsewhere within 2 %)
        int groups = max(1, __float2int_rz(__fdividef(n_cta * share, (share + T) * S.chunk) + (queue ? 0.999f : 0.5f)));
        groups = min(groups, max(1, S.by_chunk.div(T > 0 ? n_cta - 1 : n_cta)));
        groups = min(groups, (columns + kPxMinPiece - 1) / kPxMinPiece);
        P.cg = float_div(columns + groups - 1, groups);
        P.groups = float_div(columns + P.cg - 1, P.cg);
        n_pre = P.groups * S.chunk;
      }
      P.TB = T;
      int want = min(max(1, n_cta - n_pre), (T + kPxMinPiece - 1) / kPxMinPiece);
      if (queue && T > 0) {
        // Whole items, but those that would leave half of the CTAs or more without one at the end: they are cut into as many parts as there are CTAs for each
        // (a part costs four tiles' time and its rows' merge: 1024 items of 16 tiles, 6.9 a CTA, us: the last one of every CTA in quarters 152, none cut 123).
        const int items = S.Hkv * S.F, over = items - float_div(items, n_cta) * n_cta, parts = over > 0 ? min(8, float_div(n_cta, over)) : 1;
        P.MA = items;
        P.uA = T;
        if (parts > 1) {
          P.MA = items - over;
          const int hk = S.by_F.div(P.MA), f = P.MA - hk * S.F;
          int before = 0;
#pragma unroll 1
          for (int f0 = 0; f0 < f; f0 += 32) {
            int nt, len, slot;
            own_items(f0, nt, len, slot);
            before += __reduce_add_sync(FULLM, f0 + lane < f ? units(nt) : 0);
          }
          P.uA = hk * P.W + before;
        }
        P.TB = T - P.uA;
        want = min(over * parts, (P.TB + kPxMinPiece - 1) / kPxMinPiece);
      }
      want = max(1, min(want, S.nb_max));
      P.sB = max(1, float_div(P.TB + want - 1, want));
      P.NB = float_div(P.TB + P.sB - 1, P.sB);
      if (blockIdx.x == 0 && lane == 0) {
        p.plan[0] = P.PT;
        p.plan[1] = P.cg;
        p.plan[2] = P.NB;
      }
    }
    // ---- the pieces: `n_pre` of the beginning, P.MA whole own items, P.NB of the others' stream
    bool ok = true;
    const int pieces = n_pre + P.MA + P.NB;
#pragma unroll 1
    for (int id = blockIdx.x; ok && id < pieces;) {
      // its units [u, u1) of a stream that goes head after head (or chunk of row tiles after chunk), `per` units each; whole items: item `only`
      int head = 0, only = -1, u, u1, per, j = 0;
      const int piece = id - n_pre - P.MA;
      if (id < n_pre) {
        const int g = S.by_chunk.div(id);
        j = id - g * S.chunk;
        per = P.PT;
        u = g * P.cg;
        u1 = min(u + P.cg, S.Hkv * S.nrc * P.PT);
      } else if (piece < 0) {
        const int m = id - n_pre;
        head = S.by_F.div(m);
        only = m - head * S.F;
        per = P.W;
        u = 0;
        u1 = P.W;
      } else {
        per = P.W;
        u = P.uA + piece * P.sB;
        u1 = min(u + P.sB, P.uA + P.TB);
        if (!S.stack && lane == 0) p.cut_rec[piece] = make_int2(-1, 0);
      }
      if (only < 0) {
        head = float_div(u, per);
        u -= head * per;
        u1 -= head * per;
      }
#pragma unroll 1
      while (ok && u < u1) {       // one head's
        int before = 0;
        const int f_end = id < n_pre ? 1 : S.F;
#pragma unroll 1
        for (int f0 = only < 0 ? 0 : only & ~31; ok && f0 < f_end && before < u1; f0 += 32) {
          int nt = 0, len = 0, slot = -1;
          if (id < n_pre) {
            if (lane == 0) nt = per;
          } else if (f0 == 0) {
            nt = nt0, len = len0, slot = slot0;
          } else {
            own_items(f0, nt, len, slot);
          }
          const int inc = scan(id < n_pre ? nt : units(nt)), first = before + inc - nt;
          const int lo = only < 0 ? max(u, first) : first, hi = only < 0 ? min(u1, before + inc) : only == f0 + lane ? first + nt : first;
          before += __shfl_sync(FULLM, inc, 31);
#pragma unroll 1
          for (unsigned todo = __ballot_sync(FULLM, hi > lo); todo != 0u && ok; todo &= todo - 1) {
            const int l = __ffs(todo) - 1, f = f0 + l;
            const int kt = __shfl_sync(FULLM, lo - first, l), take = __shfl_sync(FULLM, hi - lo, l);
            PrefixItem it = {};
            it.cnt = take;
            if (id < n_pre) {
              const int hk = S.by_nrc.div(head), rt = (head - hk * S.nrc) * S.chunk + j;
              if (rt >= S.TP) continue;
              it.type = 1;
              it.hk = hk;
              it.row0 = rt * 128;
              it.nrows = min(128, S.B * S.R - it.row0);
              it.pos0 = kt * 128;
              it.kv_end = P.PE;
              it.slot = P.donor;
              it.out = ((S.by_chunk.div(id) + head) * S.chunk + j) * 128;
            } else {
              const int all = __shfl_sync(FULLM, nt, l), b = S.by_TO.div(f), m = head * S.F + f;
              it.b = b;
              it.hk = head;
              it.row0 = (f - b * S.TO) * 128;
              it.nrows = min(128, S.R - it.row0);
              it.pos0 = S.k0 + kt * 128;
              it.len = it.kv_end = __shfl_sync(FULLM, len, l);
              it.slot = __shfl_sync(FULLM, slot, l);
              const bool whole = take == all;
              it.out = whole ? (S.stack ? p.own_row0 + m * S.rows : -1) : p.cut_row0 + (2 * piece + (kt == 0 ? 1 : 0)) * S.rows;
              if (kt == 0) {
                // the item's parts: this piece's and those of the pieces up to its last unit
                const int last = head * P.W + __shfl_sync(FULLM, first, l) + all - 1 - P.uA;
                const int parts = whole ? 1 : float_div(last, P.sB) - piece + 1;
                if (lane == 0) {
                  if (S.stack) p.own_rec[m] = make_int2(whole ? 0 : piece, parts);
                  else if (!whole) p.cut_rec[piece] = make_int2(m, parts);
                }
              }
            }
            ok = emit(it, false);
          }
        }
        // the next head's
        if (only >= 0) break;
        head++;
        u = 0;
        u1 -= per;
      }
      if (queue) {
        // (one item beyond the one being worked on: whatever else this CTA held, others could not take at the end)
        const int m = published - 2;
        if (ok && m >= 0) ok = wait_all(ITEM_EMPTY + m % kPxRing, (m / kPxRing) & 1, kPxItemEmpty);
        int next = 0;
        if (lane == 0) next = n_cta + atomicAdd(p.counter, 1);
        id = __shfl_sync(FULLM, next, 0);
      } else {
        id += n_cta;
      }
    }
    // (a row can outgrow its reference only in the first run, so once is enough)
    if (ok) ok = emit(PrefixItem{}, true);
    if (ok && lane == 0) {      // (all items are done: the slot is free)
      ring[published % kPxRing].type = -1;
      mbar_arrive(BAR(ITEM_FULL + published % kPxRing));
    }
  } else if (warp == 1) {
    // ------------------------------------------------------------------ Q K^T issuer
    asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
    const bool leader = elect_one_sync();
    constexpr uint32_t desc_hi = (1024u >> 4) | (1u << 14) | (2u << 29);
    constexpr uint32_t idesc_qk = make_idesc_bf16(128, 128, 0, 0);
    const uint32_t tmem_u = __shfl_sync(FULLM, tmem, 0);
    auto desc64 = [](uint32_t lo) { return (static_cast<uint64_t>(desc_hi) << 32) | lo; };
    const uint32_t q_lo = ((smem_u32(smem + L_::kQ) & 0x3FFFFu) >> 4) | (1u << 16);
    const uint32_t k_lo0 = ((smem_u32(smem + L_::kK) & 0x3FFFFu) >> 4) | (1u << 16);
    int stage = 0, round = 0;
    int used[2] = {0, 0};
    bool ok = true;
#pragma unroll 1
    for (int n = 0; ok; n++) {
      PrefixItem it;
      if (!get_item(n, it)) break;
      const int cnt = it.cnt;
      ok = wait_all(Q_FULL + (n & 1), (n >> 1) & 1, kPxQFull);
      const uint32_t qw_lo = q_lo + (n & 1) * (L_::kQSlot >> 4);
#pragma unroll 1
      for (int t = 0; t < cnt && ok; t++) {
        const int j = t & 1;
        ok = wait_all(K_FULL + stage, round & 1, kPxKFull);
        if (!ok) break;
        if (used[j] > 0) {
          ok = wait_all(S_FREE + j, (used[j] - 1) & 1, kPxSFree);
          if (!ok) break;
        }
        tc_fence_after();
        const uint32_t k_lo = k_lo0 + stage * (L_::kTile >> 4);
        const uint32_t tm_s = tmem_u + j * 128;
        if (leader) {
#pragma unroll
          for (int ks = 0; ks < D / 16; ks++) {
            const uint32_t off = ((ks >> 2) * PANEL + (ks & 3) * 32) >> 4;
            umma_ss(tm_s, desc64(qw_lo + off), desc64(k_lo + off), idesc_qk, ks > 0 ? 1u : 0u);
          }
          umma_commit(BAR(S_FULL + j));
          umma_commit(BAR(K_EMPTY + stage));
          if (t == cnt - 1) umma_commit(BAR(Q_EMPTY + (n & 1)));
        }
        __syncwarp();
        used[j]++;
        if (++stage == KS) {
          stage = 0;
          round++;
        }
      }
      if (ok) item_done(n);
    }
    // tensor memory must not be freed under a running product (of items that have been read out none is)
    if (misc[kPxStop] != 0) {
      if (leader) umma_commit(BAR(QK_DRAIN));
      __syncwarp();
      mbar_wait(BAR(QK_DRAIN), 0);
    }
  } else if (warp == 2) {
    // ------------------------------------------------------------------ P V issuer
    asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
    const bool leader = elect_one_sync();
    constexpr uint32_t desc_hi = (1024u >> 4) | (1u << 14) | (2u << 29);
    constexpr uint32_t idesc_pv = make_idesc_bf16(128, D, 0, 1);
    const uint32_t tmem_u = __shfl_sync(FULLM, tmem, 0);
    auto desc64 = [](uint32_t lo) { return (static_cast<uint64_t>(desc_hi) << 32) | lo; };
    const uint32_t v_lo0 = ((smem_u32(smem + L_::kV) & 0x3FFFFu) >> 4) | (static_cast<uint32_t>(PANEL >> 4) << 16);
    auto issue_half = [&](uint32_t tm_buf, uint32_t v_lo, int half, uint32_t acc_first) {
#pragma unroll
      for (int kk = 0; kk < 4; kk++) {
        const int ks = half * 4 + kk;
        umma_ts(tmem_u + TM_O, tm_buf + ks * 8, desc64(v_lo + ks * (2048 >> 4)), idesc_pv, kk > 0 ? 1u : acc_first);
      }
    };
    int stage = 0, round = 0, outputs = 0;
    int used[2] = {0, 0};
    bool ok = true;
#pragma unroll 1
    for (int n = 0; ok; n++) {
      PrefixItem it;
      if (!get_item(n, it)) break;
      if ((it.type >> 1) != 1) {
        const int cnt = it.cnt;
#pragma unroll 1
        for (int t = 0; t < cnt && ok; t++) {
          const int j = t & 1;
          ok = wait_all(V_FULL + stage, round & 1, kPxVFull);
          if (!ok) break;
          const int valid = it.kv_end - it.pos0 - t * 128;
          if (valid > 0 && valid < 128 && (valid & (S.page - 1)) != 0) {
            // behind the last token its page may hold anything; P is zero there, and 0 * NaN is not
            const int end = (valid + S.page - 1) & ~(S.page - 1);
            uint8_t* tile = smem + L_::kV + stage * L_::kTile;
#pragma unroll 1
            for (int c = valid * 8 + lane; c < end * 8; c += 32) {
#pragma unroll
              for (int pn = 0; pn < NPANEL; pn++) *reinterpret_cast<uint4*>(tile + pn * PANEL + c * 16) = make_uint4(0u, 0u, 0u, 0u);
            }
            fence_proxy_async();
            __syncwarp();
          }
          ok = wait_all(P_FULL + 2 * j, used[j] & 1, kPxPFull);
          if (!ok) break;
          if (t == 0 && outputs > 0) {
            ok = wait_all(O_FREE, (outputs - 1) & 1, kPxOFree);
            if (!ok) break;
          }
          tc_fence_after();
          const uint32_t v_lo = v_lo0 + stage * (L_::kTile >> 4);
          const uint32_t tm_buf = tmem_u + TM_P + j * 64;
          if (leader) issue_half(tm_buf, v_lo, 0, t > 0 ? 1u : 0u);
          __syncwarp();
          ok = wait_all(P_FULL + 2 * j + 1, used[j] & 1, kPxPFull);
          if (!ok) break;
          tc_fence_after();
          if (leader) {
            issue_half(tm_buf, v_lo, 1, 1u);
            umma_commit(BAR(P_FREE + j));
            umma_commit(BAR(V_EMPTY + stage));
            if (t == cnt - 1) umma_commit(BAR(O_FULL));
          }
          __syncwarp();
          used[j]++;
          if (++stage == n_vs) {
            stage = 0;
            round++;
          }
        }
        outputs++;
      }
      if (ok) item_done(n);
    }
    if (misc[kPxStop] != 0) {
      if (leader) umma_commit(BAR(PV_DRAIN));
      __syncwarp();
      mbar_wait(BAR(PV_DRAIN), 0);
    }
  } else if (warp == 15) {
    // ------------------------------------------------------------------ the watch: no key tile for a second, and every wait ends
    asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
    if (lane == 0) {
      long long since = clock64();
      int seen = 0;
      while (!mbar_try_wait(BAR(DONE), 0) && misc[kPxStop] == 0) {
        const int now = misc[kPxProgress];
        if (now != seen) {
          seen = now;
          since = clock64();
        } else if (clock64() - since > AVSA_WAIT_LIMIT_CYCLES) {
          misc[kPxStop] = 1;
        }
      }
    }
  } else {
    // ------------------------------------------------------------------ softmax groups + epilogue
    asm volatile("setmaxnreg.inc.sync.aligned.u32 192;");
    const int w = (warp - 4) >> 2;
    const int row = ((warp & 3) << 5) + lane;
    const uint32_t lane_off = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const uint32_t tm_s = tmem + w * 128 + lane_off;
    const uint32_t tm_p = tmem + TM_P + w * 64 + lane_off;
    int tiles = 0;              // S tiles this group has taken, over all items
    int used = 0;               // P tiles it has written
    int mrefs = 0, outputs = 0; // items with a first-tile reference, with an output
    int n_staged = 0;           // with final rows by TMA
    float m_given = 0.f;
    bool ok = true;
#pragma unroll 1
    for (int n = 0; ok; n++) {
      PrefixItem it;
      if (!get_item(n, it)) break;
      const int cnt = it.cnt, run = it.type >> 1;
      if ((warp & 3) * 32 >= it.nrows) {
        // no rows in this warp: its arrivals alone
#pragma unroll 1
        for (int t = w; t < cnt && ok; t += 2) {
          ok = wait_all(S_FULL + w, tiles & 1, kPxSFull);
          if (!ok) break;
          mbar_arrive(BAR(S_FREE + w));
          tiles++;
          if (run == 1) continue;
          if (run == 0 && t == 0) mbar_arrive(BAR(MREF));
          if (used > 0) ok = wait_all(P_FREE + w, (used - 1) & 1, kPxPFree);
          if (!ok) break;
          mbar_arrive(BAR(P_FULL + 2 * w));
          mbar_arrive(BAR(P_FULL + 2 * w + 1));
          used++;
        }
        if (!ok) break;
        if (run == 0) mrefs++;
        mbar_arrive(BAR(LSUM_A));
        ok = wait_all(LSUM_A, n & 1, kPxLsum);
        if (!ok) break;
        mbar_arrive(BAR(LSUM_B));
        ok = wait_all(LSUM_B, n & 1, kPxLsum);
        if (!ok) break;
        if (run != 1) {
          ok = wait_all(O_FULL, outputs & 1, kPxOFull);
          if (!ok) break;
          outputs++;
          mbar_arrive(BAR(O_FREE));
          if (staging && it.out < 0) {
            mbar_arrive(BAR(STAGED));
            n_staged++;
          }
        }
        item_done(n);
        continue;
      }
      // the thread's row: where it goes, how far it sees
      int b = it.b, i = 0, g = 0, rel = 0x7fffffff;
      if (row < it.nrows) {
        int rr = it.row0 + row, len = it.len;
        if (it.type & 1) {
          b = S.by_R.div(rr);
          rr -= b * S.R;
          int slot, bad;
          len = prefix_sequence(p, b, slot, bad);
        }
        i = S.by_G.div(rr);
        g = rr - i * S.G;
        rel = min(it.kv_end, prefix_limit(p, b, len, i)) - it.pos0;
      }
      float m_ref = run == 2 ? m_given : 0.f, m_max = -INFINITY;
      uint64_t sum2[4] = {0ull, 0ull, 0ull, 0ull};
#pragma unroll 1
      for (int t = w; t < cnt && ok; t += 2) {
        ok = __all_sync(FULLM, wait_or_stop(S_FULL + w, tiles & 1, kPxSFull));
        if (!ok) break;
        tc_fence_after();
        uint32_t s[128];
#pragma unroll
        for (int c = 0; c < 4; c++) tmem_ld32(tm_s + c * 32, *reinterpret_cast<uint32_t(*)[32]>(&s[c * 32]));
        tmem_wait_ld();
        tc_fence_before();
        mbar_arrive(BAR(S_FREE + w));
        tiles++;
        const int see = rel - t * 128;
        if (__any_sync(FULLM, see < 128)) {
#pragma unroll
          for (int c = 0; c < 4; c++) {      // (bits of a register: eight of them become predicates at once)
            const uint32_t seen = see >= 32 * c + 32 ? 0xffffffffu : see <= 32 * c ? 0u : (1u << (see - 32 * c)) - 1u;
#pragma unroll
            for (int j = 0; j < 32; j++) s[c * 32 + j] = seen & (1u << j) ? s[c * 32 + j] : 0xff800000u;
          }
        }
        if (run == 1 || (run == 0 && t == 0)) {
          float mx8[8];
#pragma unroll
          for (int u = 0; u < 8; u++) mx8[u] = fmaxf(__uint_as_float(s[2 * u]), __uint_as_float(s[2 * u + 1]));
#pragma unroll
          for (int j = 16; j < 128; j += 16) {
#pragma unroll
            for (int u = 0; u < 8; u++) mx8[u] = max3f(mx8[u], __uint_as_float(s[j + 2 * u]), __uint_as_float(s[j + 2 * u + 1]));
          }
          const float mx = p.scale_log2 * fmaxf(max3f(mx8[0], mx8[1], mx8[2]), fmaxf(max3f(mx8[3], mx8[4], mx8[5]), fmaxf(mx8[6], mx8[7])));
          if (run == 1) {
            m_max = fmaxf(m_max, mx);
            continue;
          }
          // a row that sees nothing here sees nothing in later tiles either; one that does, but nothing with a weight, has no reference for them
          m_ref = mx == -INFINITY ? 0.f : mx;
          if (mx == -INFINITY && rel > 0 && row < it.nrows) misc[kPxFlag + (n & 1)] = 1;
          mref_s[row] = m_ref;
          mbar_arrive(BAR(MREF));
        } else if (run == 0 && t == 1) {
          ok = __all_sync(FULLM, wait_or_stop(MREF, mrefs & 1, kPxMref));
          if (!ok) break;
          m_ref = mref_s[row];
        }
        const uint64_t c2 = pack_f32x2(p.scale_log2, p.scale_log2);
        const uint64_t nm2 = pack_f32x2(-m_ref, -m_ref);
#pragma unroll
        for (int c = 0; c < 4; c++) {
          uint32_t pk[16];
#pragma unroll
          for (int j = 0; j < 16; j++) {
            float x0, x1;
            unpack_f32x2(fma_f32x2(pack_f32x2(__uint_as_float(s[c * 32 + 2 * j]), __uint_as_float(s[c * 32 + 2 * j + 1])), c2, nm2), x0, x1);
            const float p0 = fast_exp2(x0), p1 = fast_exp2(x1);
            sum2[j & 3] = add_f32x2(sum2[j & 3], pack_f32x2(p0, p1));
            pk[j] = pack_bf16x2(p0, p1);
          }
          if (c == 0 && used > 0) {
            ok = __all_sync(FULLM, wait_or_stop(P_FREE + w, (used - 1) & 1, kPxPFree));
            if (!ok) break;
          }
          tmem_st16(tm_p + c * 16, pk);
          if (c == 1 || c == 3) {
            tmem_wait_st();
            tc_fence_before();
            mbar_arrive(BAR(P_FULL + 2 * w + (c >> 1)));
          }
        }
        if (ok) used++;
      }
      if (!ok) break;
      if (run == 0) mrefs++;
      float l_run;
      {
        float sa, sb;
        unpack_f32x2(add_f32x2(add_f32x2(sum2[0], sum2[1]), add_f32x2(sum2[2], sum2[3])), sa, sb);
        l_run = sa + sb;
      }
      // (a group without a tile of its own has no sum; the reference is the other one's)
      if (run == 0 && row < it.nrows && !(l_run <= kFastRowSumLimit)) misc[kPxFlag + (n & 1)] = 1;
      lsum_s[w * 128 + row] = run == 1 ? m_max : l_run;
      if (tid == 128) tma_store_wait_read();      // the rows staged before have been read when the groups have met
      mbar_arrive(BAR(LSUM_A));
      ok = __all_sync(FULLM, wait_or_stop(LSUM_A, n & 1, kPxLsum));
      if (!ok) break;
      const float other = lsum_s[(1 - w) * 128 + row];
      const bool again = misc[kPxFlag + (n & 1)] != 0;
      if (run == 0 && cnt == 1 && w == 1) m_ref = mref_s[row];
      mbar_arrive(BAR(LSUM_B));
      ok = __all_sync(FULLM, wait_or_stop(LSUM_B, n & 1, kPxLsum));
      if (!ok) break;
      if (run == 1) {
        m_given = fmaxf(m_max, other);
        if (m_given == -INFINITY) m_given = 0.f;
        item_done(n);
        continue;
      }
      if (tid == 128) {
        misc[kPxFlag + (n & 1)] = 0;
        if (again) {
          redo[misc[kPxListed]] = it;
          misc[kPxListed] = misc[kPxListed] + 1;
          misc[kPxRecomputed] = misc[kPxRecomputed] + 1;
        }
      }
      ok = __all_sync(FULLM, wait_or_stop(O_FULL, outputs & 1, kPxOFull));
      if (!ok) break;
      outputs++;
      tc_fence_after();
      constexpr int HALF = D / 2;
      uint32_t o0[HALF];
#pragma unroll
      for (int c = 0; c < HALF / 32; c++)
        tmem_ld32(tmem + TM_O + lane_off + w * HALF + c * 32, *reinterpret_cast<uint32_t(*)[32]>(&o0[c * 32]));
      tmem_wait_ld();
      tc_fence_before();
      mbar_arrive(BAR(O_FREE));
      // (the short forms of quotient and logarithm: 1 to 2^64 as sums go, two units in the last place of fp32 and 1e-7; the long ones are 60 instructions)
      const float sum = l_run + other;
      const float inv = sum > 0.f || sum != sum ? __fdividef(1.0f, sum) : 0.f;
      const float lse2 = sum != 0.f ? m_ref + __log2f(sum) : -INFINITY;
      if (it.out < 0 && !again && w == 0 && row < it.nrows && p.lse != nullptr)
        p.lse[(static_cast<int64_t>(b) * S.Hkv * S.G + it.hk * S.G + g) * S.L + i] = lse2 * 0.6931471805599453f;
      if (staging && it.out < 0) {
#pragma unroll
        for (int c = 0; c < HALF / 8; c++) {
          const int col = w * HALF + c * 8;
          uint4 v;
          v.x = pack_bf16x2(__uint_as_float(o0[c * 8 + 0]) * inv, __uint_as_float(o0[c * 8 + 1]) * inv);
          v.y = pack_bf16x2(__uint_as_float(o0[c * 8 + 2]) * inv, __uint_as_float(o0[c * 8 + 3]) * inv);
          v.z = pack_bf16x2(__uint_as_float(o0[c * 8 + 4]) * inv, __uint_as_float(o0[c * 8 + 5]) * inv);
          v.w = pack_bf16x2(__uint_as_float(o0[c * 8 + 6]) * inv, __uint_as_float(o0[c * 8 + 7]) * inv);
          *reinterpret_cast<uint4*>(stage_out + (col >> 6) * PANEL + row * 128 + ((((col & 63) >> 3) ^ (row & 7)) << 4)) = v;
        }
        fence_proxy_async();
        mbar_arrive(BAR(STAGED));
        if (tid == 128 && wait_or_stop(STAGED, n_staged & 1, kPxLsum) && !again) {
          for (int pn = 0; pn < NPANEL; pn++) tma_store_4d(&tmo, smem_u32(stage_out) + pn * PANEL, pn * 64, it.hk * S.G, S.by_G.div(it.row0), it.b);
          tma_store_commit();
        }
        n_staged++;
      } else if (!again && row < it.nrows) {
        if (it.out >= 0) {
          const int64_t at = it.out + row;
          if (w == 0) p.part_lse2[at] = lse2;
          float* dst = p.part_o + at * D + w * HALF;
#pragma unroll
          for (int c = 0; c < HALF / 8; c++) {
            uint32_t r[8];
#pragma unroll
            for (int x = 0; x < 8; x++) r[x] = __float_as_uint(__uint_as_float(o0[c * 8 + x]) * inv);
            st_global_v8(dst + c * 8, r);
          }
        } else {
          uint4* dst = reinterpret_cast<uint4*>(p.o + b * p.q.stride_b + (it.hk * S.G + g) * p.q.stride_h + i * p.q.stride_n + w * HALF);
#pragma unroll
          for (int c = 0; c < HALF / 8; c++) {
            uint4 v;
            v.x = pack_bf16x2(__uint_as_float(o0[c * 8 + 0]) * inv, __uint_as_float(o0[c * 8 + 1]) * inv);
            v.y = pack_bf16x2(__uint_as_float(o0[c * 8 + 2]) * inv, __uint_as_float(o0[c * 8 + 3]) * inv);
            v.z = pack_bf16x2(__uint_as_float(o0[c * 8 + 4]) * inv, __uint_as_float(o0[c * 8 + 5]) * inv);
            v.w = pack_bf16x2(__uint_as_float(o0[c * 8 + 6]) * inv, __uint_as_float(o0[c * 8 + 7]) * inv);
            dst[c] = v;
          }
        }
      }
      item_done(n);
    }
    if (tid == 128) {
      tma_store_wait_read();      // (the last rows)
      mbar_arrive(BAR(DONE));
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 2) tmem_dealloc(tmem, 512);
  if (tid == 0) {
    p.cta_err[2 * blockIdx.x] = misc[kPxStop] != 0 ? make_int4(AVSA_ERR_TIMEOUT, misc[kPxWhere], blockIdx.x, misc[kPxProgress])
                                          : make_int4(misc[kPxErr], misc[kPxErr + 1], misc[kPxErr + 2], misc[kPxErr + 3]);
    p.cta_err[2 * blockIdx.x + 1] = make_int4(misc[kPxRecomputed], 0, 0, 0);
  }
}

// ------------------------------------------------------------------------------------------------ joining the parts
// Four channels of a row to a thread.  Parts are joined in the order of the key axis.  Stacked rows: the groups of the beginning, whose numbers
// follow from the plan, and the parts of the row's own item.  Else: the rows of the items that a B piece begins and another ends.
constexpr int kPxMergeThreads = 256;
constexpr __host__ __device__ int prefix_merge_rows(int D) { return kPxMergeThreads / (D / 4); }      // rows of a CTA

// Adds parts 0 .. n-1, which are rows at(k), to the four channels of a row that stand at `col`: acc is the sum of weights times values and L that of the weights, against
// the reference M (L == 0: nothing yet).  Eight parts' sums and values are on their way together: one trip to L2.
template <int D, class At>
__device__ __forceinline__ void join_parts(const PrefixParams& p, At at, int n, int col, float4& acc, float& M, float& L, bool& nan) {
  constexpr int U = 8;
  for (int k0 = 0; k0 < n; k0 += U) {
    float y[U];
    float4 v[U];
#pragma unroll
    for (int u = 0; u < U; u++) {
      const int64_t row = at(min(k0 + u, n - 1));
      y[u] = p.part_lse2[row];
      v[u] = *reinterpret_cast<const float4*>(p.part_o + row * D + col);
    }
    float top = L != 0.f ? M : -INFINITY;
#pragma unroll
    for (int u = 0; u < U; u++) {
      if (k0 + u >= n) y[u] = -INFINITY;
      nan = nan || y[u] != y[u];
      top = fmaxf(top, y[u]);
    }
    const float ref = top == -INFINITY ? 0.f : top, f = L != 0.f ? fast_exp2(M - ref) : 0.f;
    M = ref;
    L *= f;
    acc = make_float4(acc.x * f, acc.y * f, acc.z * f, acc.w * f);
#pragma unroll
    for (int u = 0; u < U; u++) {
      const float w = fast_exp2(y[u] - ref);
      L += w;
      if (w != 0.f) acc = make_float4(acc.x + w * v[u].x, acc.y + w * v[u].y, acc.z + w * v[u].z, acc.w + w * v[u].w);
    }
  }
}

// The parts of a row and their order: n_first of the beginning, `step` apart, one at `second`, and the others of the n_second from `next` on, second_step apart.
struct PrefixRow {
  int first, step, n_first, second, n_second, next, second_step;
  __device__ __forceinline__ int64_t operator()(int k) const {
    if (k < n_first) return first + static_cast<int64_t>(k) * step;
    k -= n_first;
    return k == 0 ? second : next + static_cast<int64_t>(k - 1) * second_step;
  }
};
// Thread x of the row's D/4: the final row.
template <int D>
__device__ __forceinline__ void prefix_final_row(const PrefixParams& p, float4 o, float M, float L, bool nan, int b, int head, int i, int x) {
  const float inv = nan ? NAN : L > 0.f ? 1.0f / L : 0.f;
  __nv_bfloat16* dst = p.o + b * p.q.stride_b + head * p.q.stride_h + i * p.q.stride_n + 4 * x;
  *reinterpret_cast<uint2*>(dst) = make_uint2(pack_bf16x2(o.x * inv, o.y * inv), pack_bf16x2(o.z * inv, o.w * inv));
  if (x == 0 && p.lse != nullptr)
    p.lse[(static_cast<int64_t>(b) * p.s.Hkv * p.s.G + head) * p.s.L + i] = nan ? NAN : L > 0.f ? (M + log2f(L)) * 0.6931471805599453f : -INFINITY;
}
template <int D>
__device__ __forceinline__ void prefix_merge_row(const PrefixParams& p, const PrefixRow& row, int b, int head, int i, int x) {
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  float M = 0.f, L = 0.f;
  bool nan = false;
  join_parts<D>(p, row, row.n_first + row.n_second, 4 * x, o, M, L, nan);
  prefix_final_row<D>(p, o, M, L, nan, b, head, i, x);
}

template <int D>
__global__ void __launch_bounds__(kPxMergeThreads) prefix_merge_kernel(const __grid_constant__ PrefixParams p, int n_cta) {
  pdl_wait();
  pdl_launch();
  const PrefixShape& S = p.s;
  constexpr int ROWS = prefix_merge_rows(D);
  const int x = threadIdx.x % (D / 4);
  if (blockIdx.x == 0 && threadIdx.x < 32) {
    // the status record: the first CTA's error, and how many items were recomputed
    const int lane = threadIdx.x;
    int4 err = make_int4(0, 0, 0, 0);
    int again = 0;
    for (int c = lane; c < n_cta; c += 32) {
      const int4 e = p.cta_err[2 * c];
      if (err.x == 0) err = e;
      again += p.cta_err[2 * c + 1].x;
    }
    again = __reduce_add_sync(0xffffffffu, again);
    const unsigned who = __ballot_sync(0xffffffffu, err.x != 0);
    const int from = who ? __ffs(who) - 1 : 0;
    if (lane == from) {
      p.status->code = p.status->where = p.status->item = p.status->aux = p.status->next_item = 0;
      p.status->redo_count = again;
      if (err.x != 0) report_logged(p.status, p.log, err.x, err.y, err.z, err.w);
    }
  }
  if (S.stack) {
    const int PT = p.plan[0], cg = p.plan[1];
    const int rows = S.B * S.R;                // of a key head, stacked
    const int64_t r = static_cast<int64_t>(blockIdx.x) * ROWS + threadIdx.x / (D / 4);
    if (r >= static_cast<int64_t>(rows) * S.Hkv) return;
    const int hk = static_cast<int>(r / rows), rho = static_cast<int>(r - static_cast<int64_t>(hk) * rows);
    const int b = S.by_R.div(rho), rr = rho - b * S.R, i = S.by_G.div(rr), g = rr - i * S.G, own = rr >> 7, in = rr & 127;
    const int m = hk * S.F + b * S.TO + own;
    int2 rec = p.own_rec[m];      // (where there is an own item; read beside the length that says so)
    int slot, bad;
    const int len = prefix_sequence(p, b, slot, bad);
    PrefixRow row = {};
    if (PT > 0) {
      const int rt = rho >> 7, rc = S.by_chunk.div(rt), j = rt - rc * S.chunk, U = hk * S.nrc + rc;
      const int g0 = U * PT / cg, g1 = ((U + 1) * PT - 1) / cg;
      row.first = ((g0 + U) * S.chunk + j) * 128 + (rho & 127);
      row.step = S.chunk * 128;
      row.n_first = g1 - g0 + 1;
    }
    if (prefix_own_tiles(p, b, len, own) > 0) {
      // (a kernel that gave up, for a wait that ran out, may have left records unwritten)
      if (rec.x < 0 || rec.y < 1 || (rec.y > 1 && rec.x > p.plan[2] - rec.y)) rec = make_int2(0, 0);
      row.n_second = rec.y;
      row.second = rec.y == 1 ? p.own_row0 + m * S.rows + in : p.cut_row0 + (2 * rec.x + 1) * S.rows + in;
      row.next = p.cut_row0 + (2 * rec.x + 2) * S.rows + in;
      row.second_step = 2 * S.rows;
    }
    prefix_merge_row<D>(p, row, b, hk * S.G + g, i, x);
  } else {
    const int NB = p.plan[2];
    for (int at = blockIdx.x * ROWS + threadIdx.x / (D / 4); at < S.nb_max * 128; at += gridDim.x * ROWS) {
      const int piece = at >> 7, in = at & 127;
      const int2 rec = p.cut_rec[piece];
      if (piece >= NB) break;
      // (one that a kernel that gave up did not write either)
      if (rec.x < 0 || rec.x >= S.Hkv * S.F || rec.y < 1 || rec.y > NB - piece) continue;
      const int hk = S.by_F.div(rec.x), f = rec.x - hk * S.F, b = S.by_TO.div(f), rr = (f - b * S.TO) * 128 + in;
      if (in >= S.rows || rr >= S.R) continue;
      const int i = S.by_G.div(rr), g = rr - i * S.G, end = p.cut_row0 + (2 * piece + 1) * S.rows + in;
      const PrefixRow row = {0, 0, 0, end, rec.y, end + S.rows, 2 * S.rows};
      prefix_merge_row<D>(p, row, b, hk * S.G + g, i, x);
    }
  }
}

}  // namespace avsa
