// Attention of few query rows over a paged cache: keys and values go from HBM into warp-level products, once.
//
// One token of a sequence has G query rows against thousands of keys: 2 FLOPs a byte and row, so nothing counts but how many bytes are on their way from HBM
// and how soon the first of them are.  The tile kernel's machinery (tensor memory, tile rings, a plan, roles that wait for one another) takes 5 us before its
// first product; here a warp reads a length, a page id, and 16 keys at a time: 4 KB of K and 4 KB of V (128 channels) by TMA into a ring of its own, whose
// 16-byte vectors are exactly the operands of mma.m16n8k16.  No warp waits for another before the end.
//   S^T = K Q^T    16 keys by 8 query rows.  The contraction runs over the channels in any order: lane (n, c) = (lane/4, lane%4) reads channels 32j + 8c .. +7 of
//                  keys n and n + 8, and takes words 0-1 and 2-3 of each vector as the operands of steps 2j and 2j + 1; Q is laid out to match, in registers;
//   P^T            keys come out of S^T in rows and go into the next product in pairs: one movmatrix for 8 x 8 of them;
//   O^T += V^T P^T 16 channels by 8 query rows, and the rows of a product are any channels: lane (n, c) reads channels 64j + 8n .. +7 of keys 2c, 2c+1, 8+2c, 9+2c,
//                  word y of which are rows n and n + 8 of product (j, y); two keys of a channel meet in a register by byte permutes.
// With the query rows as columns a product is half as wide as with them as rows (8 against 16 that one token hardly ever has); more than 8 rows are two columns' products
// on the same operands.  What counts then is how much is in flight (64 sequences x 8 key heads x 2048 keys, 537 MB, us: vectors to registers, 60 KB of an SM ahead, 117; by
// cp.async to shared memory, 96 KB ahead, 132, and the loop without its products 125: 16-byte copies reach no more; by TMA, 128 KB ahead, 93).
// Each warp has its own running maximum and sum (rescaled when a maximum grew by more than 2^8) and takes every (warps of the item)-th 16 keys; warps are joined
// through shared memory, the CTAs of an item (a cluster) through each other's.  Then a row is final, or meets the parts of the beginning, or is a part itself.
#pragma once
#include <math.h>

#include "prefix_attn_kernel.cuh"
#include "q4.cuh"

namespace avsa {

constexpr int kStWarps = 4, kStThreads = 32 * kStWarps;
// Query rows of an item, at most, by its products of 8 columns; where there are more than two, all rows are one item.
constexpr int stream_item_rows(int NT) { return NT > 2 ? 8 * NT : 16; }

// What a launch of the kernel below works on.
struct StreamParams {
  int stacked;         // items are row tiles of the beginning (row tile, key head), else of the sequences (row tile, key head, batch entry)
  int tiles, rows;     // row tiles of an item's key head, and their rows
  int items;
  int splits;          // parts that an item's keys are cut into, each of them a cluster; with more than one, or stacked, the rows are parts
  int first;           // no kernel of this call in front of it
  int begin;           // the first CTA clears the status record
  int check;           // the first cluster looks for what is out of range
  int join;            // 0, or the beginning's parts are in kStJoinStream's or kStJoinTile's places
  int join_tiles, join_rows, join_splits;
  int out0;            // first partial row
};
enum { kStJoinStream = 1, kStJoinTile = 2 };

__device__ __forceinline__ void mma_16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// The first of a chain: no accumulator.
__device__ __forceinline__ void mma_16816_first(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
      : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}
// Transposes 8 x 8 16-bit elements: the lane's two of row lane/4 become its two of column lane/4.
__device__ __forceinline__ uint32_t transpose_8x8(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
__device__ __forceinline__ void cluster_store_f32x4(uint32_t addr, float4 v) {
  asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "f"(v.x), "f"(v.y), "f"(v.z), "f"(v.w) : "memory");
}
// A CTA's shared memory is there once the CTA has begun: each says so at once, and waits for the others only before it writes to them.
__device__ __forceinline__ void cluster_begun() { asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_all_begun() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ uint32_t stream_cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ uint32_t stream_cluster_size() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
  return r;
}

// The longest sequence of the batch.  A warp.
__device__ __forceinline__ void longest_sequence(const PrefixParams& p, int& slot, int& tokens, int& entry) {
  int top = 0;
  slot = entry = 0;
  for (int b = threadIdx.x & 31; b < p.s.B; b += 32) {
    int s, bad;
    const int len = prefix_sequence(p, b, s, bad);
    if (len > top) top = len, slot = s, entry = b;
  }
  tokens = first_longest(top, entry, slot);
}

// The call's status: what is out of range in the sequences of the batch, else the first error of a CTA of the tile kernel in front (`wait`: nothing has waited for it
// yet).  One CTA, the call's first one to write the record (a wait of the stream kernel that runs out does so a second later).
static __device__ __noinline__ void prefix_check(const PrefixParams& p, int n_cta, int wait) {
  __shared__ int worst, tile_error, again;
  const PrefixShape& S = p.s;
  if (threadIdx.x == 0) worst = 0x7fffffff, tile_error = 0x7fffffff, again = 0;
  __syncthreads();
  constexpr int U = 8;      // loads in flight
  // the pages that are read: of every sequence those behind the shared ones, and these of the longest
  for (int b = threadIdx.x >> 5; b < S.B; b += blockDim.x >> 5) {
    int slot, bad;
    const int len = prefix_sequence(p, b, slot, bad);
    const int used = (len + S.page - 1) >> S.page_shift;
    for (int e0 = (S.k0 >> S.page_shift) + (threadIdx.x & 31); e0 < used; e0 += 32 * U) {
      int page[U];
#pragma unroll
      for (int u = 0; u < U; u++) page[u] = e0 + 32 * u < used ? p.table[static_cast<int64_t>(slot) * S.width + e0 + 32 * u] : 0;
#pragma unroll
      for (int u = 0; u < U; u++)
        if (page[u] < 0 || page[u] >= S.pages) bad = kPrefixPage;
    }
    if (bad) atomicMin(&worst, (b << 9) | bad);
  }
  if (S.stack) {
    int slot, top, who;
    longest_sequence(p, slot, top, who);
    const int used = (min(top, S.k0) + S.page - 1) >> S.page_shift;
    for (int e = threadIdx.x; e < used; e += blockDim.x) {
      const int page = p.table[static_cast<int64_t>(slot) * S.width + e];
      if (page < 0 || page >= S.pages) atomicMin(&worst, (who << 9) | kPrefixPage);
    }
  }
  if (wait) {
    pdl_wait();
    pdl_launch();
  }
  for (int c = threadIdx.x; c < n_cta; c += blockDim.x) {
    const int code = p.cta_err[2 * c].x, more = p.cta_err[2 * c + 1].x;
    if (code != 0 && code != AVSA_ERR_BAD_TABLE) atomicMin(&tile_error, c);
    if (more != 0) atomicAdd(&again, more);
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    p.status->redo_count = again;
    if (tile_error != 0x7fffffff) {
      const int4 e = p.cta_err[2 * tile_error];
      report_logged(p.status, p.log, e.x, e.y, e.z, e.w);
    } else if (worst != 0x7fffffff) {
      report_logged(p.status, p.log, AVSA_ERR_BAD_TABLE, worst & 511, worst >> 9, 0);
    }
  }
}
__device__ __forceinline__ void prefix_check_begin(const PrefixParams& p) {
  if (threadIdx.x == 0) {
    StatusRecord* st = p.status;
    st->code = st->where = st->item = st->aux = st->redo_count = st->next_item = 0;
  }
}

// CTAs that an SM holds, by shared memory: with one product's columns three of two stages (of 8 KB; 64 sequences of 100 to 2048 keys, us: 55.4, two of three stages 58.7),
// with two products' the warps take longer and want more ahead (32 sequences x 8 x 2048 keys, 16 rows: 71.5 and 58.0).  Codes: by registers, 128 a thread, 234, 250 and 254 (32 x 8 items of
// 2048 keys, 16 rows, us, with two, three and four CTAs of them: 33, 46, 39); two stages (of 4.6 KB) are as good as three.
constexpr int stream_ctas(int NT, bool q4) { return q4 ? (NT == 1 ? 4 : 2) : NT == 1 ? 3 : 2; }

template <int D, int NT, bool Q4>
struct StreamSmem {
  static constexpr int kRows = stream_item_rows(NT);
  static constexpr int kPanel = 16 * 128, kBlock = q4_block_bytes(D);
  static constexpr int kStages = (NT == 1 ? 2 : 3) * (128 / D);
  static constexpr int kStage = Q4 ? 4 * kBlock : 2 * (D / 64) * kPanel;      // a stage: panels of K, panels of V, or two blocks of each
  union {
    uint8_t ring[kStWarps][kStages][kStage];      // 128-byte swizzled
    float4 o[kStWarps][kRows][D / 4];           // behind the keys
  };
  uint64_t full[kStWarps][kStages];
  float m[kStWarps][kRows], l[kStWarps][kRows];
  // what the CTAs of a cluster send this one: its share of the rows' vectors, and what they are relative to (reference, sum of weights)
  float4 in_o[8 * NT * (D / 4) + 8];
  float2 in_ml[8 * NT * (D / 4) + 8];
  int per, by_per;      // vectors of each CTA, at most; at / per is at * by_per >> 20 for all of them (at * (by_per * per - 2^20) is at most 2^18)
};

// The key of a block of codes that is row r (of 8) of S^T.  Keys' codes are 64 bytes apart (128 channels), so that a product's operands come from shared memory without
// two lanes of a phase at one bank where neighbouring rows, and rows two apart, alternate between even and odd keys.
__device__ __forceinline__ int stream_key(int r) { return r ^ ((r >> 1) & 1); }

// The pages of a warp's first 8 blocks of 16 keys, `step` apart (PAIRS: and of the one behind each), by one load, a lane each, which asks for them before the sequence's
// length is known where it can.  (One at a time, each asked for when the one before had come, the six stages of a ring took 2 us to fill.)
template <bool PAIRS>
struct FirstPages {
  const int32_t* row;
  int step, id0 = 0, id1 = 0;
  __device__ __forceinline__ FirstPages(const PrefixParams& p, int slot, int step_) : row(p.table + static_cast<int64_t>(max(slot, 0)) * p.s.width), step(step_) {}
  __device__ __forceinline__ void look_up(const PrefixShape& S, int blk) {
    const int mine = blk + static_cast<int>(threadIdx.x & 7) * step, last = S.width - 1;
    id0 = row[min(mine >> (S.page_shift - 4), last)];
    if (PAIRS && S.page_shift == 4) id1 = row[min(mine + 1, last)];
  }
  __device__ __forceinline__ int page(int k) const { return __shfl_sync(0xffffffffu, id0, k); }
  __device__ __forceinline__ int page_behind(const PrefixShape& S, int k) const { return __shfl_sync(0xffffffffu, PAIRS && S.page_shift == 4 ? id1 : id0, k); }
};

// The ring of a warp whose keys are codes: a stage has a pair of blocks of 16 keys (one piece of memory of 4.6 KB each of K and V, with pages of 32 and more).
template <int D, class Smem>
struct CodePairs {
  static constexpr int BLOCK = Smem::kBlock;
  const PrefixCodes& src;
  Smem& sm;
  const PrefixShape& S;
  const int32_t* row;
  int b1, step, at, next0, next1, warp, lane;
  uint32_t ring, full;
  const uint8_t *k_head, *v_head;
  __device__ __forceinline__ CodePairs(const PrefixCodes& src_, const PrefixShape& S_, Smem& sm_, const FirstPages<true>& ids, int hk, int blk, int b1_)
      : src(src_), sm(sm_), S(S_), row(ids.row), b1(b1_), step(ids.step), at(blk), warp(threadIdx.x >> 5), lane(threadIdx.x & 31),
        ring(smem_u32(&sm_.ring[threadIdx.x >> 5][0][0])), full(smem_u32(&sm_.full[threadIdx.x >> 5][0])), k_head(src_.k.ptr + hk * src_.k.stride_head),
        v_head(src_.v.ptr + hk * src_.v.stride_head) {
    static_assert(Smem::kStages < 8, "the pages of a ring and the next one");
#pragma unroll 1
    for (int k = 0; k < Smem::kStages; k++) {
      load(at, ids.page(k), ids.page_behind(S, k), k);
      at += step;
    }
    next0 = ids.page(Smem::kStages);
    next1 = ids.page_behind(S, Smem::kStages);
  }
  __device__ __forceinline__ bool single() const { return S.page_shift == 4; }      // a page is one block: pairs are two pages
  __device__ __forceinline__ bool exists(int page) const { return static_cast<unsigned>(page) < static_cast<unsigned>(S.pages); }
  __device__ __forceinline__ int page_of(int blk) const { return blk < b1 ? row[blk >> (S.page_shift - 4)] : -1; }
  __device__ __forceinline__ void load_next(int stage) {
    const int blk = at, page0 = next0, page1 = next1;
    at += step;
    next0 = page_of(at);
    next1 = single() ? page_of(at + 1) : next0;
    load(blk, page0, page1, stage);
  }
  __device__ __forceinline__ void load(int blk, int page0, int page1, int stage) {
    if (blk >= b1) return;
    const uint32_t bar = full + stage * 8, dst = ring + stage * Smem::kStage;
    const bool has0 = exists(page0), has1 = exists(page1);
    if (!(has0 && (has1 || blk + 1 >= b1))) {
      // a page that does not exist reads as zeros: scales of zero, the codes may be anything
      for (int h = 0; h < 2; h++)
        if (!(h == 0 ? has0 : has1))
          for (int w = lane; w < D / 4; w += 32) {
            *reinterpret_cast<uint32_t*>(&sm.ring[warp][stage][h * BLOCK + q4_scales_at(D) + 4 * w]) = 0u;
            *reinterpret_cast<uint32_t*>(&sm.ring[warp][stage][(2 + h) * BLOCK + q4_scales_at(D) + 4 * w]) = 0u;
          }
      fence_proxy_async();      // (a copy lands there later)
      __syncwarp();
    }
    if (lane == 0) {
      if (!single() && has0) {
        const int64_t in = page0 * src.k.stride_page + static_cast<int64_t>(blk & ((1 << (S.page_shift - 4)) - 1)) * BLOCK;
        const int64_t in_v = page0 * src.v.stride_page + static_cast<int64_t>(blk & ((1 << (S.page_shift - 4)) - 1)) * BLOCK;
        mbar_expect_tx(bar, 4 * BLOCK);
        bulk_load_1d(dst, k_head + in, 2 * BLOCK, bar);
        bulk_load_1d(dst + 2 * BLOCK, v_head + in_v, 2 * BLOCK, bar);
      } else if (single() && (has0 || has1)) {
        mbar_expect_tx(bar, ((has0 ? 2 : 0) + (has1 ? 2 : 0)) * BLOCK);
        if (has0) {
          bulk_load_1d(dst, k_head + page0 * src.k.stride_page, BLOCK, bar);
          bulk_load_1d(dst + 2 * BLOCK, v_head + page0 * src.v.stride_page, BLOCK, bar);
        }
        if (has1) {
          bulk_load_1d(dst + BLOCK, k_head + page1 * src.k.stride_page, BLOCK, bar);
          bulk_load_1d(dst + 3 * BLOCK, v_head + page1 * src.v.stride_page, BLOCK, bar);
        }
      } else {
        mbar_arrive(bar);
      }
    }
  }
  __device__ __forceinline__ bool wait(int stage, int round) const { return __all_sync(0xffffffffu, mbar_wait(full + stage * 8, round & 1)); }
  // a load never came: the status says so, the rows lack this warp's keys from there on, and what is under way lands before this memory is given away
  __device__ __forceinline__ void give_up(const PrefixParams& p, int item, int blk, int stage, int round) const {
    report_logged(p.status, p.log, AVSA_ERR_TIMEOUT, kPxKFull, item, blk);
    for (int k = 0; k < Smem::kStages; k++) mbar_wait(full + k * 8, (round + (k < stage ? 1 : 0)) & 1);
  }
};

// The keys of a warp, where they are codes: pairs of blocks of 16 (one piece of memory of 4.6 KB each of K and V, with pages of 32 and more), from block `blk` on, every
// `step`-th.  Rows as in the kernel below.  A block takes some 310 instructions, 3 for each pair of values, of which half are the ALU's (two cycles each), where its bytes take
// 100 cycles of the SM's share of HBM: what counts is how many are issued.  Hence two blocks side by side, for each of which the other's latencies are filled; the rows'
// maxima looked at by every lane for itself, and brought together only where one has outgrown its reference; sums and exponents two at a time.  (64 x 8 x 2048 keys,
// 151 MB, us: one block at a time 73, two 60, with the masks' constant in a register 51, and one CTA an item 44; 32 x 8 x 16 rows x 2048 keys, 75 MB, 31.)
// Three products, 17 to 24 rows, on the same operands instead of two items (us): 64 x 8 x 700 keys 45 and 33, 8 x 8 x 2000 17.4 and 14.5, of 64 channels 12.9 and 10.3; of 128
// channels one block after the other then.  Four, up to 32 rows of 64 channels: 64 x 8 x 700 32.4 and 25.3, 8 x 8 x 2000 13.0 and 11.6.
template <int D, int NT, class Smem>
__device__ __forceinline__ void stream_codes(const PrefixCodes& src, const PrefixParams& p, Smem& sm, const FirstPages<true>& ids, int hk, int blk, int b1, int k1,
                                             int rel_min, const int (&see)[NT][2], const uint4 (&q)[NT][D / 32], float (&o)[NT][D / 16][4], float (&m)[NT][2],
                                             float (&l)[NT][2], int item) {
  constexpr unsigned FULLM = 0xffffffffu;
  constexpr int STAGES = Smem::kStages, BLOCK = Smem::kBlock, G = D / kQ4Group;
  constexpr int H = NT * D > 256 ? 1 : 2;      // blocks side by side (registers)
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, n = lane >> 2, c = lane & 3;
  const uint32_t sixteen = src.k.sixteen;
  const int step = ids.step;
  CodePairs<D, Smem> pairs(src, p.s, sm, ids, hk, blk, b1);
  const int key = stream_key(n), key0 = stream_key(2 * c), key1 = stream_key(2 * c + 1);      // as an operand's rows; as its columns
  const float inv_scale = 1.0f / p.scale_log2;
  const uint64_t scale2 = pack_f32x2(p.scale_log2, p.scale_log2);
  float limit[NT][2], ref[NT][2];      // logits above it outgrow the reference; the reference, 0 where there is none
#pragma unroll
  for (int x = 0; x < NT; x++) limit[x][0] = limit[x][1] = -INFINITY, ref[x][0] = ref[x][1] = 0.f;
  int stage = 0, round = 0;
  bool ok = true;
#pragma unroll 1
  for (; blk < b1; blk += step) {
    if (!pairs.wait(stage, round)) {
      ok = false;
      break;
    }
#pragma unroll 1
    for (int h0 = 0; h0 < 2; h0 += H) {
      const uint8_t* const tile = &sm.ring[warp][stage][h0 * BLOCK];
      const int first = (blk + h0) * 16;
      // ---- S^T: lane (n, c) has a quarter of the channels of keys `key` and `key` + 8, in whole words
      float s[H][NT][4];
#pragma unroll
      for (int h = 0; h < H; h++) {
        constexpr int W = D / 32;
        const uint8_t* const k = tile + h * BLOCK;
        uint32_t ka[W], kb[W];
        if constexpr (W == 4) {
          *reinterpret_cast<uint4*>(ka) = *reinterpret_cast<const uint4*>(k + key * (D / 2) + 16 * c);
          *reinterpret_cast<uint4*>(kb) = *reinterpret_cast<const uint4*>(k + (key + 8) * (D / 2) + 16 * c);
        } else {
          *reinterpret_cast<uint2*>(ka) = *reinterpret_cast<const uint2*>(k + key * (D / 2) + 8 * c);
          *reinterpret_cast<uint2*>(kb) = *reinterpret_cast<const uint2*>(k + (key + 8) * (D / 2) + 8 * c);
        }
        const uint16_t* const scales = reinterpret_cast<const uint16_t*>(k + q4_scales_at(D)) + c * (D / 4) / kQ4Group;
        uint32_t sa = scales[key * G], sb = scales[(key + 8) * G];
        sa |= sa << 16;
        sb |= sb << 16;
        const uint32_t oa = q4_offset(sa), ob = q4_offset(sb);
#pragma unroll
        for (int j = 0; j < W; j++) {
          uint32_t a[4], b[4];
#pragma unroll
          for (int i = 0; i < 4; i++) a[i] = q4_pair(ka[j], i, sa, oa, sixteen), b[i] = q4_pair(kb[j], i, sb, ob, sixteen);
#pragma unroll
          for (int x = 0; x < NT; x++) {
            if (j == 0)
              mma_16816_first(s[h][x], a[0], b[0], a[1], b[1], q[x][j].x, q[x][j].y);
            else
              mma_16816(s[h][x], a[0], b[0], a[1], b[1], q[x][j].x, q[x][j].y);
            mma_16816(s[h][x], a[2], b[2], a[3], b[3], q[x][j].z, q[x][j].w);
          }
        }
      }
      if (first + 16 * H > rel_min || first + 16 * H > k1) {
#pragma unroll
        for (int h = 0; h < H; h++)
#pragma unroll
          for (int x = 0; x < NT; x++)
#pragma unroll
            for (int e = 0; e < 4; e++)
              if (first + 16 * h + key + 8 * (e >> 1) >= min(see[x][e & 1], k1)) s[h][x][e] = -INFINITY;
      }
      // ---- maxima
      float top[NT][2];
      bool grown = false;
#pragma unroll
      for (int x = 0; x < NT; x++)
#pragma unroll
        for (int e = 0; e < 2; e++) {
          top[x][e] = H == 2 ? fmaxf(max3f(s[0][x][e], s[0][x][2 + e], s[H - 1][x][e]), s[H - 1][x][2 + e]) : fmaxf(s[0][x][e], s[0][x][2 + e]);
          grown = grown || top[x][e] > limit[x][e];
        }
      if (__any_sync(FULLM, grown)) {
#pragma unroll
        for (int x = 0; x < NT; x++)
#pragma unroll
          for (int e = 0; e < 2; e++) {
            float up = top[x][e];
#pragma unroll
            for (int d = 4; d < 32; d <<= 1) up = fmaxf(up, __shfl_xor_sync(FULLM, up, d));
            up = fmaxf(m[x][e], up * p.scale_log2);
            const float f = m[x][e] == -INFINITY ? 0.f : fast_exp2(m[x][e] - up);
            m[x][e] = up;
            limit[x][e] = (up + 8.f) * inv_scale;
            ref[x][e] = up == -INFINITY ? 0.f : up;
            l[x][e] *= f;
#pragma unroll
            for (int y = 0; y < D / 16; y++) {
              o[x][y][e] *= f;
              o[x][y][2 + e] *= f;
            }
          }
      }
      // ---- P^T
      uint32_t pt[H][NT][2];
#pragma unroll
      for (int h = 0; h < H; h++)
#pragma unroll
        for (int x = 0; x < NT; x++) {
          float w[4];
          const uint64_t no_ref = pack_f32x2(-ref[x][0], -ref[x][1]);
          uint64_t sum = pack_f32x2(l[x][0], l[x][1]);
#pragma unroll
          for (int e = 0; e < 4; e += 2) {
            unpack_f32x2(fma_f32x2(pack_f32x2(s[h][x][e], s[h][x][e + 1]), scale2, no_ref), w[e], w[e + 1]);
            w[e] = fast_exp2(w[e]);
            w[e + 1] = fast_exp2(w[e + 1]);
            sum = add_f32x2(sum, pack_f32x2(w[e], w[e + 1]));
          }
          unpack_f32x2(sum, l[x][0], l[x][1]);
          pt[h][x][0] = transpose_8x8(pack_bf16x2(w[0], w[1]));
          pt[h][x][1] = transpose_8x8(pack_bf16x2(w[2], w[3]));
        }
      // ---- O^T: lane (n, c) has an eighth of the channels of the keys that are rows 2c, 2c + 1, 2c + 8 and 2c + 9 of S^T
#pragma unroll
      for (int h = 0; h < H; h++) {
        constexpr int W = D / 64;
        const uint8_t* const v = tile + (2 + h) * BLOCK;
        uint32_t w0[W], w1[W], w2[W], w3[W];
        auto codes = [&](int at, uint32_t (&w)[W]) {
          if constexpr (W == 2) {
            *reinterpret_cast<uint2*>(w) = *reinterpret_cast<const uint2*>(v + at * (D / 2) + 8 * n);
          } else {
            w[0] = *reinterpret_cast<const uint32_t*>(v + at * (D / 2) + 4 * n);
          }
        };
        codes(key0, w0);
        codes(key1, w1);
        codes(key0 + 8, w2);
        codes(key1 + 8, w3);
        const uint16_t* const scales = reinterpret_cast<const uint16_t*>(v + q4_scales_at(D)) + n * (D / 8) / kQ4Group;
        uint32_t s0 = scales[key0 * G], s1 = scales[key1 * G], s2 = scales[(key0 + 8) * G], s3 = scales[(key1 + 8) * G];
        if (first + 16 * H > k1) {
          // behind the last token its page may hold anything; P is zero there, and 0 * NaN is not
          const int left = k1 - first - 16 * h;
          if (key0 >= left) s0 = 0u;
          if (key1 >= left) s1 = 0u;
          if (key0 + 8 >= left) s2 = 0u;
          if (key1 + 8 >= left) s3 = 0u;
        }
        s0 |= s1 << 16;
        s2 |= s3 << 16;
        const uint32_t o0 = q4_offset(s0), o2 = q4_offset(s2);
#pragma unroll
        for (int j = 0; j < W; j++) {
          const uint32_t e0 = __byte_perm(w0[j], w1[j], 0x5410), d0 = __byte_perm(w0[j], w1[j], 0x7632);      // even channels of both keys, odd ones
          const uint32_t e2 = __byte_perm(w2[j], w3[j], 0x5410), d2 = __byte_perm(w2[j], w3[j], 0x7632);
#pragma unroll
          for (int i = 0; i < 4; i++) {
            const uint32_t a0 = q4_pair(e0, i, s0, o0, sixteen), a1 = q4_pair(d0, i, s0, o0, sixteen), a2 = q4_pair(e2, i, s2, o2, sixteen), a3 = q4_pair(d2, i, s2, o2, sixteen);
#pragma unroll
            for (int x = 0; x < NT; x++) mma_16816(o[x][4 * j + i], a0, a1, a2, a3, pt[h][x][0], pt[h][x][1]);
          }
        }
      }
    }
    __syncwarp();      // all lanes have read the stage
    pairs.load_next(stage);
    if (++stage == STAGES) {
      stage = 0;
      round++;
    }
  }
  if (!ok) pairs.give_up(p, item, blk, stage, round);
}

// Where the parts of the beginning of stacked row rho are: `n` of them, `step` rows apart.
__device__ __forceinline__ void prefix_parts(const PrefixParams& p, const StreamParams& t, int hk, int rho, int& first, int& step, int& n) {
  const PrefixShape& S = p.s;
  if (t.join == kStJoinStream) {
    const int tile = t.join_tiles > 1 ? rho >> 4 : 0;
    step = t.join_rows;
    n = t.join_splits;
    first = (hk * t.join_tiles + tile) * n * step + rho - 16 * tile;
    return;
  }
  const int PT = (S.k0 + 127) >> 7;
  const int rt = rho >> 7, rc = S.by_chunk.div(rt), j = rt - rc * S.chunk, U = hk * S.nrc + rc;
  const int g0 = S.by_cg.div(U * PT), g1 = S.by_cg.div((U + 1) * PT - 1);
  step = S.chunk * 128;
  first = ((g0 + U) * S.chunk + j) * 128 + (rho & 127);
  n = g1 - g0 + 1;
}

// Four channels of a row: acc is the sum of its weights times values against the reference M, L the sum of its weights.
template <int D>
__device__ __forceinline__ void stream_finish(const PrefixParams& p, const StreamParams& t, int item, int split, int hk, int entry, int row0, int r, int x, float4 acc,
                                              float M, float L) {
  const PrefixShape& S = p.s;
  float lse2 = L != 0.f ? M + log2f(L) : -INFINITY, inv = L > 0.f || L != L ? 1.0f / L : 0.f;
  if (t.stacked || t.splits > 1) {
    const int64_t at = t.out0 + (static_cast<int64_t>(item) * t.splits + split) * t.rows + r;
    *reinterpret_cast<float4*>(p.part_o + at * D + 4 * x) = make_float4(acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv);
    if (x == 0) p.part_lse2[at] = lse2;
    return;
  }
  const int rr = row0 + r, i = S.by_G.div(rr), g = rr - i * S.G, head = hk * S.G + g;
  if (t.join != 0) {
    int first, step, n;
    prefix_parts(p, t, hk, entry * S.R + rr, first, step, n);
    bool nan = lse2 != lse2;
    join_parts<D>(p, [=](int k) { return first + static_cast<int64_t>(k) * step; }, n, 4 * x, acc, M, L, nan);
    lse2 = nan ? NAN : L > 0.f ? M + log2f(L) : -INFINITY;
    inv = nan ? NAN : L > 0.f ? 1.0f / L : 0.f;
  }
  __nv_bfloat16* dst = p.o + entry * p.q.stride_b + head * p.q.stride_h + i * p.q.stride_n + 4 * x;
  *reinterpret_cast<uint2*>(dst) = make_uint2(pack_bf16x2(acc.x * inv, acc.y * inv), pack_bf16x2(acc.z * inv, acc.w * inv));
  if (x == 0 && p.lse != nullptr) p.lse[(static_cast<int64_t>(entry) * S.Hkv * S.G + head) * S.L + i] = lse2 * 0.6931471805599453f;
}

// NT: products of 8 query rows, 1 or 2 (of codes up to 3, or, with 64 channels, 4).
template <int D, int NT, class Source>
__global__ void __launch_bounds__(kStThreads, stream_ctas(NT, Source::kQ4))
prefix_stream_kernel(const __grid_constant__ Source src, const __grid_constant__ PrefixParams p, const StreamParams t) {
  extern __shared__ __align__(1024) uint8_t smem[];
  constexpr bool Q4 = Source::kQ4;
  using L_ = StreamSmem<D, NT, Q4>;
  L_& sm = *reinterpret_cast<L_*>(smem);
  constexpr unsigned FULLM = 0xffffffffu;
  const PrefixShape& S = p.s;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, n = lane >> 2, c = lane & 3;
  const int rank = static_cast<int>(stream_cluster_rank()), ctas = static_cast<int>(stream_cluster_size());
  if (lane == 0) {
    for (int k = 0; k < L_::kStages; k++) mbar_init(smem_u32(&sm.full[warp][k]), 1);
    fence_mbar_init();
    if constexpr (!Q4) {
      prefetch_tmap(&src.k);
      prefetch_tmap(&src.v);
    }
  }
  __syncwarp();
  if (t.first) {
    pdl_wait();
    pdl_launch();
  }
  if (t.begin && blockIdx.x == 0) prefix_check_begin(p);
  int id = static_cast<int>(blockIdx.x) / ctas;
  if (t.check) {
    if (id == 0) {
      if (rank == 0) {
        prefix_check(p, t.join == kStJoinTile ? p.tile_ctas : 0, !t.first);
      } else if (!t.first) {
        pdl_wait();
        pdl_launch();
      }
      return;
    }
    id--;
  }
  if (ctas > 1) cluster_begun();
  // ---- the item: rows, keys
  const int split = t.splits > 1 ? id % t.splits : 0;
  if (t.splits > 1) id /= t.splits;
  const int item = id, tile = t.tiles > 1 ? id % t.tiles : 0;
  if (t.tiles > 1) id /= t.tiles;
  const int hk = id % S.Hkv, entry = id / S.Hkv;
  const int row0 = tile * L_::kRows, n_rows = t.stacked ? S.B * S.R : S.R, rows = min(L_::kRows, n_rows - row0);
  int slot, bad, k0, k1;
  if (t.stacked) {
    int most, who;
    longest_sequence(p, slot, most, who);
    k0 = 0;
    k1 = min(S.k0, most);
  } else {
    k0 = S.k0;
    k1 = prefix_sequence(p, entry, slot, bad);
  }
  if (ctas > 1 && threadIdx.x == 0) {
    sm.per = (rows * (D / 4) + ctas - 1) / ctas;
    sm.by_per = (1 << 20) / sm.per + 1;
  }
  constexpr int PER = Q4 ? 2 : 1;      // blocks that a warp takes at a time
  FirstPages<Q4> ids(p, slot, PER * ctas * kStWarps);
  const int ahead = PER * (rank * kStWarps + warp);
  if (t.splits <= 1) ids.look_up(S, (k0 >> 4) + ahead);
  // Lane r: how far row r sees.  The thread's columns are rows 8x + 2c and 8x + 2c + 1 of S^T and O^T; as an operand, Q is row 8x + n.
  auto row_of = [&](int r, int& b, int& i, int& head, int& len) {
    int rr = row0 + r;
    b = entry;
    len = k1;
    if (t.stacked) {
      b = S.by_R.div(rr);
      rr -= b * S.R;
      int s;
      len = prefix_sequence(p, b, s, bad);
    }
    i = S.by_G.div(rr);
    head = hk * S.G + rr - i * S.G;
  };
  int rel = 0x7fffffff;
  if (lane < rows) {
    int b, i, head, len;
    row_of(lane, b, i, head, len);
    rel = prefix_limit(p, b, len, i);
  }
  const int rel_min = __reduce_min_sync(FULLM, rel);
  k1 = min(k1, __reduce_max_sync(FULLM, lane < rows ? rel : 0));
  int see[NT][2];
#pragma unroll
  for (int x = 0; x < NT; x++)
#pragma unroll
    for (int e = 0; e < 2; e++) see[x][e] = __shfl_sync(FULLM, rel, 8 * x + 2 * c + e);
  uint4 q[NT][D / 32];
#pragma unroll
  for (int x = 0; x < NT; x++) {
    const bool have = 8 * x + n < rows;
    int b = 0, i = 0, head = 0, len;
    if (have) row_of(8 * x + n, b, i, head, len);
    const __nv_bfloat16* at = static_cast<const __nv_bfloat16*>(p.q.ptr) + b * p.q.stride_b + head * p.q.stride_h + i * p.q.stride_n + (Q4 ? D / 4 : 8) * c;
#pragma unroll
    for (int j = 0; j < D / 32; j++) q[x][j] = have ? *reinterpret_cast<const uint4*>(at + (Q4 ? 8 : 32) * j) : make_uint4(0u, 0u, 0u, 0u);
  }
  // 16-key blocks [b0, b1) of the part, every `step`-th from the warp's own on
  int b0 = k0 >> 4, b1 = (k1 + 15) >> 4;
  if (t.splits > 1) {
    int per = (b1 - b0 + t.splits - 1) / t.splits;
    if (Q4) per = (per + 1) & ~1;      // (pairs of blocks)
    b0 = min(b1, b0 + split * per);
    b1 = min(b1, b0 + per);
    ids.look_up(S, b0 + ahead);
  }
  float o[NT][D / 16][4];       // product 4j + y: {channel 64j + 8n + 2y (of codes (D/8)n + 8j + 2y), the next} x {row 2c, the next}, as [2 * channel + row]
#pragma unroll
  for (int x = 0; x < NT; x++)
#pragma unroll
    for (int y = 0; y < D / 16; y++) o[x][y][0] = o[x][y][1] = o[x][y][2] = o[x][y][3] = 0.f;
  float m[NT][2], l[NT][2];
#pragma unroll
  for (int x = 0; x < NT; x++) m[x][0] = m[x][1] = -INFINITY, l[x][0] = l[x][1] = 0.f;
  if constexpr (Q4) {
    stream_codes<D, NT>(src, p, sm, ids, hk, b0 + ahead, b1, k1, rel_min, see, q, o, m, l, item);
  } else {
    const int step = ctas * kStWarps;
    const int block_shift = S.page_shift - 4;
    constexpr int STAGES = L_::kStages, PANEL = L_::kPanel, NPANEL = D / 64;
    const uint32_t ring = smem_u32(&sm.ring[warp][0][0]), full = smem_u32(&sm.full[warp][0]);
    // (a page that does not exist reads as zeros)
    auto load = [&](int blk, int page, int stage) {
      if (lane == 0 && blk < b1) {
        const uint32_t bar = full + stage * 8, dst = ring + stage * L_::kStage;
        const int in = (blk & ((1 << block_shift) - 1)) * 16, pg = page < 0 ? S.pages : page;
        mbar_expect_tx(bar, L_::kStage);
        for (int pn = 0; pn < NPANEL; pn++) tma_load_4d(dst + pn * PANEL, &src.k, bar, pn * 64, in, hk, pg);
        for (int pn = 0; pn < NPANEL; pn++) tma_load_4d(dst + (NPANEL + pn) * PANEL, &src.v, bar, pn * 64, in, hk, pg);
      }
    };
    // vectors of a stage: `chunk` of 16 bytes of row `key` in a panel
    auto vec = [&](int stage, int panel, int key, int chunk) {
      return *reinterpret_cast<const uint4*>(&sm.ring[warp][stage][panel * PANEL + key * 128 + ((chunk ^ (key & 7)) << 4)]);
    };
    auto page_of = [&](int blk) { return blk < b1 ? ids.row[blk >> block_shift] : -1; };

    int blk = b0 + ahead, at = blk;
#pragma unroll
    for (int k = 0; k < STAGES; k++) {
      load(at, ids.page(k), k);
      at += step;
    }
    int next = ids.page(STAGES);
    int stage = 0, round = 0;
    bool ok = true;
#pragma unroll 1
    for (; blk < b1; blk += step) {
      if (!__all_sync(FULLM, mbar_wait(full + stage * 8, round & 1))) {
        ok = false;
        break;
      }
      float s[NT][2][4] = {};      // two chains of products each
#pragma unroll
      for (int j = 0; j < D / 32; j++) {
        const uint4 ka = vec(stage, j >> 1, n, (j & 1) * 4 + c), kb = vec(stage, j >> 1, n + 8, (j & 1) * 4 + c);
#pragma unroll
        for (int x = 0; x < NT; x++) {
          mma_16816(s[x][0], ka.x, kb.x, ka.y, kb.y, q[x][j].x, q[x][j].y);
          mma_16816(s[x][1], ka.z, kb.z, ka.w, kb.w, q[x][j].z, q[x][j].w);
        }
      }
      uint32_t pt[NT][2];
#pragma unroll
      for (int x = 0; x < NT; x++) {
        float v[4];      // key n: rows 2c, 2c + 1; key n + 8: the same
#pragma unroll
        for (int e = 0; e < 4; e++) v[e] = s[x][0][e] + s[x][1][e];
        if (blk * 16 + 16 > rel_min || blk * 16 + 16 > k1) {
#pragma unroll
          for (int e = 0; e < 4; e++)
            if (blk * 16 + n + 8 * (e >> 1) >= min(see[x][e & 1], k1)) v[e] = -INFINITY;
        }
        float top[2];
#pragma unroll
        for (int e = 0; e < 2; e++) top[e] = fmaxf(v[e], v[2 + e]) * p.scale_log2;
#pragma unroll
        for (int d = 4; d < 32; d <<= 1) {
          top[0] = fmaxf(top[0], __shfl_xor_sync(FULLM, top[0], d));
          top[1] = fmaxf(top[1], __shfl_xor_sync(FULLM, top[1], d));
        }
        if (__any_sync(FULLM, top[0] > m[x][0] + 8.f || top[1] > m[x][1] + 8.f)) {
#pragma unroll
          for (int e = 0; e < 2; e++) {
            const float up = fmaxf(m[x][e], top[e]);
            const float f = m[x][e] == -INFINITY ? 0.f : fast_exp2(m[x][e] - up);
            m[x][e] = up;
            l[x][e] *= f;
#pragma unroll
            for (int y = 0; y < D / 16; y++) {
              o[x][y][e] *= f;
              o[x][y][2 + e] *= f;
            }
          }
        }
        float e4[4];
#pragma unroll
        for (int e = 0; e < 4; e++) {
          const float ref = m[x][e & 1] == -INFINITY ? 0.f : m[x][e & 1];
          e4[e] = fast_exp2(fmaf(v[e], p.scale_log2, -ref));
          l[x][e & 1] += e4[e];
        }
        pt[x][0] = transpose_8x8(pack_bf16x2(e4[0], e4[1]));
        pt[x][1] = transpose_8x8(pack_bf16x2(e4[2], e4[3]));
      }
#pragma unroll
      for (int j = 0; j < D / 64; j++) {
        uint32_t v0[4], v1[4], v2[4], v3[4];
        *reinterpret_cast<uint4*>(v0) = vec(stage, NPANEL + j, 2 * c, n);
        *reinterpret_cast<uint4*>(v1) = vec(stage, NPANEL + j, 2 * c + 1, n);
        *reinterpret_cast<uint4*>(v2) = vec(stage, NPANEL + j, 2 * c + 8, n);
        *reinterpret_cast<uint4*>(v3) = vec(stage, NPANEL + j, 2 * c + 9, n);
        if (blk * 16 + 16 > k1) {
          // behind the last token its page may hold anything; P is zero there, and 0 * NaN is not
          const int left = k1 - blk * 16 - 2 * c;
#pragma unroll
          for (int y = 0; y < 4; y++) {
            if (left < 1) v0[y] = 0u;
            if (left < 2) v1[y] = 0u;
            if (left < 9) v2[y] = 0u;
            if (left < 10) v3[y] = 0u;
          }
        }
#pragma unroll
        for (int y = 0; y < 4; y++) {
          const uint32_t a0 = __byte_perm(v0[y], v1[y], 0x5410), a1 = __byte_perm(v0[y], v1[y], 0x7632);
          const uint32_t a2 = __byte_perm(v2[y], v3[y], 0x5410), a3 = __byte_perm(v2[y], v3[y], 0x7632);
#pragma unroll
          for (int x = 0; x < NT; x++) mma_16816(o[x][4 * j + y], a0, a1, a2, a3, pt[x][0], pt[x][1]);
        }
      }
      __syncwarp();      // all lanes have read the stage
      {
        const int page = next;
        next = page_of(at + step);
        load(at, page, stage);
        at += step;
      }
      if (++stage == STAGES) {
        stage = 0;
        round++;
      }
    }
    if (!ok) {
      // a load never came: the status says so, the rows lack this warp's keys from there on, and what is under way lands before this memory is given away
      report_logged(p.status, p.log, AVSA_ERR_TIMEOUT, kPxKFull, item, blk);
      for (int k = 0; k < STAGES; k++) mbar_wait(full + k * 8, (round + (k < stage ? 1 : 0)) & 1);
    }
  }
  __syncthreads();      // the ring is the warps' rows from here on

  // ---- the warps of the CTA
  // (the vectors of a row change places by its number: lanes of four rows write at a time, whose distance is a multiple of all banks; 16 rows took 1.5 us here)
  auto turned = [](int r) { return Q4 && D == 128 ? (r >> 1) & 3 : ((r >> 1) & 1) | (r & 4); };
#pragma unroll
  for (int x = 0; x < NT; x++)
#pragma unroll
    for (int e = 0; e < 2; e++) {
#pragma unroll
      for (int d = 4; d < 32; d <<= 1) l[x][e] += __shfl_xor_sync(FULLM, l[x][e], d);
      const int r = 8 * x + 2 * c + e;
      if (r < rows) {
        if (n == 0) {
          sm.m[warp][r] = m[x][e];
          sm.l[warp][r] = l[x][e];
        }
#pragma unroll
        for (int y = 0; y < D / 16; y += 2)
          sm.o[warp][r][(((y >> 2) * (Q4 ? 8 : 64) + (Q4 ? D / 8 : 8) * n + 2 * (y & 3)) / 4) ^ turned(r)] = make_float4(o[x][y][e], o[x][y][2 + e], o[x][y + 1][e], o[x][y + 1][2 + e]);
      }
    }
  __syncthreads();
  if (!t.first) {      // (until here nothing was read that the kernel in front of this one writes)
    pdl_wait();
    pdl_launch();
  }
  constexpr int V = D / 4;       // vectors of a row
  const int total = rows * V;
  float4 acc;
  float M, L;
  auto of_warps = [&](int r, int x) {
    M = -INFINITY;
#pragma unroll
    for (int w = 0; w < kStWarps; w++) M = fmaxf(M, sm.m[w][r]);
    L = 0.f;
    acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int w = 0; w < kStWarps; w++) {
      const float f = sm.m[w][r] == -INFINITY ? 0.f : fast_exp2(sm.m[w][r] - M);
      const float4 v = sm.o[w][r][x ^ turned(r)];
      L += f * sm.l[w][r];
      acc.x += f * v.x;
      acc.y += f * v.y;
      acc.z += f * v.z;
      acc.w += f * v.w;
    }
  };
  if (ctas == 1) {
    for (int at = threadIdx.x; at < total; at += kStThreads) {
      of_warps(at / V, at % V);
      stream_finish<D>(p, t, item, split, hk, entry, row0, at / V, at % V, acc, M, L);
    }
  } else {
    const int per = sm.per, by_per = sm.by_per;
    cluster_all_begun();
    // each vector to the CTA that has it among its own: it then reads its own memory, and nobody waits until it has (each reading the others' instead, behind one barrier and
    // before another: 24 heads of 300 keys, codes, us in a row, 5.8, now 5.2; 21 rows x 5 x 8 x 1300 keys of 64 channels 10.7 and 9.3)
    for (int at = threadIdx.x; at < total; at += kStThreads) {
      of_warps(at / V, at % V);
      const int to = at * by_per >> 20;
      const uint32_t place = rank * per + at - to * per;
      cluster_store_f32x4(cluster_addr(smem_u32(&sm.in_o[place]), to), acc);
      cluster_store_f32x2(cluster_addr(smem_u32(&sm.in_ml[place]), to), M, L);
    }
    cluster_sync_all();
    for (int i = threadIdx.x; i < per && rank * per + i < total; i += kStThreads) {
      const int at = rank * per + i;
      float2 ml[8];
      M = -INFINITY;
#pragma unroll
      for (int k = 0; k < 8; k++) {
        ml[k] = k < ctas ? sm.in_ml[k * per + i] : make_float2(-INFINITY, 0.f);
        M = fmaxf(M, ml[k].x);
      }
      L = 0.f;
      acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int k = 0; k < 8; k++) {
        if (k >= ctas) break;
        const float f = ml[k].x == -INFINITY ? 0.f : fast_exp2(ml[k].x - M);
        const float4 v = sm.in_o[k * per + i];
        L += f * ml[k].y;
        acc.x += f * v.x;
        acc.y += f * v.y;
        acc.z += f * v.z;
        acc.w += f * v.w;
      }
      stream_finish<D>(p, t, item, split, hk, entry, row0, at / V, at % V, acc, M, L);
    }
  }
}

// The rows of own items whose keys were cut into parts, a CTA each: there are few of them and up to hundreds of parts, which groups of D/4 threads join side by side
// (one key head, 30000 keys in 443 parts: the call 54 us with a group a row, 15 with a CTA).
template <int D>
__global__ void __launch_bounds__(kPxMergeThreads) prefix_join_kernel(const __grid_constant__ PrefixParams p, const StreamParams t) {
  constexpr int GROUPS = prefix_merge_rows(D);
  __shared__ float4 part[GROUPS][D / 4];
  __shared__ float part_m[GROUPS], part_l[GROUPS];      // (a sum that is no number: the row is none)
  pdl_wait();
  pdl_launch();
  const PrefixShape& S = p.s;
  const int at = static_cast<int>(blockIdx.x), group = threadIdx.x / (D / 4), x = threadIdx.x % (D / 4);      // ((entry, key head), row)
  const int pair = S.by_R.div(at), rr = at - pair * S.R, entry = pair / S.Hkv, hk = pair - entry * S.Hkv;
  const int i = S.by_G.div(rr), g = rr - i * S.G;
  PrefixRow row = {};
  if (t.join != 0) prefix_parts(p, t, hk, entry * S.R + rr, row.first, row.step, row.n_first);
  const int tile = t.tiles > 1 ? rr >> 4 : 0;
  row.second = t.out0 + (pair * t.tiles + tile) * t.splits * t.rows + rr - 16 * tile;
  row.n_second = t.splits;
  row.next = row.second + t.rows;
  row.second_step = t.rows;
  const int n = row.n_first + row.n_second, per = (n + GROUPS - 1) / GROUPS, k0 = min(n, group * per);
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  float M = 0.f, L = 0.f;
  bool nan = false;
  join_parts<D>(p, [&](int k) { return row(k0 + k); }, min(per, n - k0), 4 * x, o, M, L, nan);
  part[group][x] = o;
  if (x == 0) {
    part_m[group] = M;
    part_l[group] = nan ? NAN : L;
  }
  __syncthreads();
  if (group != 0) return;
  float top = -INFINITY;
#pragma unroll
  for (int k = 0; k < GROUPS; k++) top = fmaxf(top, part_l[k] != 0.f ? part_m[k] : -INFINITY);
  o = make_float4(0.f, 0.f, 0.f, 0.f);
  L = 0.f;
#pragma unroll
  for (int k = 0; k < GROUPS; k++) {
    const float l = part_l[k], f = l != 0.f ? fast_exp2(part_m[k] - top) : 0.f;
    nan = nan || l != l;
    L += f * l;
    if (f != 0.f) o = make_float4(o.x + f * part[k][x].x, o.y + f * part[k][x].y, o.z + f * part[k][x].z, o.w + f * part[k][x].w);
  }
  prefix_final_row<D>(p, o, top, L, nan, entry, hk * S.G + g, i, x);
}

}  // namespace avsa
