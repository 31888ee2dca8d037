// Attention of a batch that shares a long beginning, over a paged cache.
#include <math.h>

#include "prefix_stream.cuh"

namespace avsa {

static __global__ void clear_counter_kernel(int* counter) {
  pdl_wait();
  pdl_launch();
  *counter = 0;
}

constexpr int kChunk = 8;        // row tiles that go through the beginning side by side, at most

constexpr int kStreamRows = 32;      // query rows of a batch entry and key head that the stream kernel takes, at most; of the stacked rows as well

// The same of codes, by the keys of all heads and sequences that the table has room for: the stream kernel makes each of them bf16 for every item, the tile kernel once for 128
// rows, but starts later, and does not mind room that no sequence uses.  us, stream and tile kernel, sequences x heads x keys:
//                              8 x 8 x 2000   64 x 8 x 800   12 x 8 x 6000   16 x 8 x 6000   64 x 24 x 600
//   128 channels, 20 rows         15, 26         37, 58          63, 58          84, 74         87, 114      one item
//                 30 rows         18, 27         57, 59          96, 59          91, 74        129, 114      two
//    64 channels, 20 rows         10, 21         25, 47          44, 45          57, 55         59, 93       one
//                 30 rows         12, 21         29, 48          48, 45          61, 56         68, 93       one
// and with room for 16384 keys, 64 x 8 x 700, 128 channels: 20 rows 127, 53; 30 rows 214, 54.  A sum of keys tells few long sequences from many short ones no better than
// this: 64 x 24 x 600 go to the slower one, and of two items 4 x 8 x 8000 (48, 33).
static int stream_rows(bool codes, long long keys) { return !codes || keys <= 512 * 1024 ? kStreamRows : keys <= 704 * 1024 ? 24 : 16; }

constexpr int kWidenTiles = 6;       // row tiles that read a tile of codes, beyond which it is made bf16 once for all of them

// Products of 8 columns for so many query rows: with 8 or less the second one's would be empty; three or four of codes, which then become bf16 once instead of twice
// (as many as there are registers for).
static int stream_products(bool codes, int d, long long rows) {
  if (rows <= 16 || !codes || rows > (d == 64 ? 32 : 24)) return rows <= 8 ? 1 : 2;
  return rows <= 24 ? 3 : 4;
}

struct PrefixLayout {
  PrefixShape s;
  int n_cta;                    // of the tile kernel
  int tile;                     // there is one
  int pre_stream, own_stream;   // the stream kernel takes the beginning, the own items
  StreamParams pre, own;
  int own_cluster;
  size_t rows;                  // partial rows
  int own_row0, cut_row0;
  size_t plan, cta_err, own_rec, cut_rec, redo, lse, o, wide, total;       // offsets in the workspace
  size_t wide_pool;             // bytes of the keys as bf16, and of the values, where pages of codes become that before the tile kernel; else 0
  size_t room;                  // what the query says: of a call that names as many pages as the pool has
};

// False: more units, or key positions rounded up to a tile, than 32 bits count.  `codes`: pages of a pool held in 4 bits, or 0.
static bool prefix_layout(int B, int H, int Hkv, int L, int d, int page, int width, int prefix_pages, int causal, int codes, PrefixLayout& y) {
  PrefixShape& s = y.s;
  s = {};
  s.B = B;
  s.Hkv = Hkv;
  s.G = H / Hkv;
  s.L = L;
  const long long R = static_cast<long long>(L) * s.G, TO = (R + 127) / 128, F = TO * B, RS = R * B, TP = (RS + 127) / 128;
  const long long most = (static_cast<long long>(width) * page + 127) / 128, PT = static_cast<long long>(prefix_pages) * page / 128;
  if (static_cast<long long>(width) * page > 0x7fffff80ll || RS > 0x3fffffffll || F * Hkv > 0x3fffffffll || RS * Hkv > 0x3fffffffll || F * Hkv * (most + kPxItemUnits) > 0x7fffffffll) return false;
  s.R = static_cast<int>(R);
  s.TO = static_cast<int>(TO);
  s.F = static_cast<int>(F);
  s.rows = R < 128 ? s.R : 128;
  s.causal = causal;
  s.page = page;
  s.width = width;
  s.shared = prefix_pages;
  s.page_shift = page == 16 ? 4 : page == 32 ? 5 : page == 64 ? 6 : 7;
  const int sms = persistent_grid(1 << 30);
  // Stacked, the beginning's key tiles are walked TP times a head instead of F times, but every row goes through the merge, which costs a key
  // tile's time for about six rows (149760 rows: 108 us, a tile of every SM 0.8), and the call has a kernel more (about eight tiles' time of every SM).
  s.stack = TP * PT + RS / 6 < F * PT && (F * PT - TP * PT - RS / 6) * Hkv > 8 * sms;
  if (s.stack) s.k0 = prefix_pages * page;
  y.own_stream = R <= stream_rows(codes > 0, (static_cast<long long>(width) * page - s.k0) * B * Hkv);
  y.pre_stream = s.stack && RS <= stream_rows(codes > 0, static_cast<long long>(s.k0) * Hkv);
  y.tile = !y.own_stream || (s.stack && !y.pre_stream);
  s.own_off = y.own_stream;
  const long long units = (y.own_stream ? 0 : F * Hkv * most) + (s.stack ? TP * Hkv * PT : 0);
  y.n_cta = static_cast<int>(units < sms ? units : sms);
  if (y.n_cta < 1) y.n_cta = 1;
  if (s.stack) {
    s.TP = static_cast<int>(TP);
    const int side = kChunk < y.n_cta ? kChunk : y.n_cta;
    s.nrc = (s.TP + side - 1) / side;
    s.chunk = (s.TP + s.nrc - 1) / s.nrc;
    const int columns = Hkv * s.nrc * ((s.k0 + 127) / 128), most_groups = y.n_cta / s.chunk, by_piece = (columns + kPxMinPiece - 1) / kPxMinPiece;
    const int groups = most_groups < by_piece ? most_groups : by_piece;
    s.cg = (columns + groups - 1) / groups;
    s.groups = (columns + s.cg - 1) / s.cg;
  }
  // Query rows as a box of a tensor map: (G heads, tokens, batch entries) that are the item's rows in their order.
  if (128 % s.G == 0) s.own_box = 128;
  if (s.stack && 128 % s.R == 0) s.pre_box = 128;
  s.queue = !y.own_stream && TO > 1 && F * Hkv > y.n_cta;
  s.nb_max = s.queue ? 8 * y.n_cta : y.n_cta;
  size_t rows = 0;
  y.pre = {};
  y.own = {};
  if (y.pre_stream) {
    y.pre.stacked = 1;
    y.pre.first = 1;
    y.pre.begin = 1;
    y.pre.rows = stream_item_rows(stream_products(codes > 0, d, RS));
    y.pre.tiles = static_cast<int>((RS + y.pre.rows - 1) / y.pre.rows);
    y.pre.items = y.pre.tiles * Hkv;
    const int slots = sms * stream_ctas(stream_products(codes > 0, d, RS), codes > 0);      // CTAs of the stream kernel that the SMs hold
    const long long by_keys = PT / 2;      // 256 keys a CTA at least: four blocks a warp
    y.pre.splits = static_cast<int>(slots / y.pre.items < by_keys ? slots / y.pre.items : by_keys);
    // The kernel behind joins a row's parts eight at a time, 0.7 us each, so with few heads fewer and longer parts end earlier (4 heads x 60000 keys, us: 111 parts 35.8, 70 31.7).
    while (y.pre.splits > 8 && 12ll * y.pre.splits * y.pre.splits > s.k0) y.pre.splits--;
    if (y.pre.splits < 1) y.pre.splits = 1;
    rows += static_cast<size_t>(y.pre.items) * y.pre.splits * y.pre.rows;
  } else if (s.stack) {
    rows += (static_cast<size_t>(y.n_cta) + static_cast<size_t>(Hkv) * s.nrc * s.chunk) * 128;
  }
  const size_t own0 = rows;
  if (y.own_stream) {
    y.own.first = !s.stack;
    y.own.join = !s.stack ? 0 : y.pre_stream ? kStJoinStream : kStJoinTile;
    y.own.join_tiles = y.pre.tiles;
    y.own.join_splits = y.pre.splits;
    y.own.join_rows = y.pre.rows;
    y.own.rows = stream_item_rows(stream_products(codes > 0, d, R));
    y.own.tiles = static_cast<int>((R + y.own.rows - 1) / y.own.rows);
    y.own.items = y.own.tiles * Hkv * B;
    y.own.out0 = static_cast<int>(own0);
    const long long keys = static_cast<long long>(width) * page - s.k0;      // at most
    const int slots = sms * stream_ctas(stream_products(codes > 0, d, R), codes > 0);
    // An item's keys over a cluster, 64 keys a CTA at least (a block a warp), as many CTAs as the SMs hold side by side: nine tenths of the slots, since a cluster takes its
    // own from one GPC and what does not fit waits for a whole item (us, filled to the last slot and like this: 96 items of 500 keys of 64 channels 14.4 and 9.7, 72
    // of 900 keys of 128 channels 16.4 and 10.3, 144 of 800 17.5 and 13.0).  No CTA has more than 1024 keys while others may have none (30 x 8 items of 1 to 1500
    // keys 15.7, of up to 1500 keys a CTA 17.0, but all of 1500 keys 24.5 and 19.7).  What eight CTAs an item do not fill is cut into parts that a kernel behind joins.
    const long long fit = slots * 9ll / 10 / (y.own.items + 1ll), by_keys = keys / 64;
    long long ctas = fit < by_keys ? fit : by_keys;
    ctas = ctas < 1 ? 1 : ctas > 8 ? 8 : ctas;
    // (Codes: no second CTA up to 2048 keys for items that fill three quarters of the slots by themselves and whose start and end weigh more, being half as long or, with
    // 16 rows, twice as many.  us, 1024 and 2048 keys a CTA, sequences x heads of so many keys:
    //                            64 x 8 of 2048   1000 to 2048   100 to 2048   20 x 24 of 1 to 2000
    //   64 channels, one row        27, 26           26, 25         23, 23           22, 22
    //                16 rows        49, 40           43, 36         36, 32           34, 31
    //   128 channels, 16 rows       69, 58           61, 52         49, 45           47, 44
    //                 one row       44, 42           39, 39         32, 36           30, 34      (not taken)
    // )
    const bool short_items = codes > 0 && (d == 64 || R > 8) && 4ll * y.own.items >= 3ll * slots;
    const long long most_keys = short_items ? 2048 : 1024;
    while (ctas < 8 && y.own.items < (1 << 27) && keys > most_keys * ctas) ctas = 2 * ctas < 8 ? 2 * ctas : 8;
    y.own_cluster = static_cast<int>(ctas);
    y.own.splits = 1;
    // (codes: where eight CTAs an item leave half of the slots empty, and at least 256 keys a part; 24 items of 40000 keys, us, as clusters 59, in 24 parts 40)
    if (static_cast<long long>(y.own.items) * 8 < (codes > 0 ? slots / 2 : sms) && keys >= (codes > 0 ? 8192 : 4096)) {
      y.own_cluster = 1;
      y.own.splits = (slots - 1) / y.own.items;      // (one slot for the check of the tables)
      if (codes > 0 && keys / 256 < y.own.splits) y.own.splits = static_cast<int>(keys / 256);
      rows += static_cast<size_t>(y.own.items) * y.own.splits * y.own.rows;
    }
    y.own.check = 1;
    y.own.begin = !y.pre_stream;
  } else {
    const size_t own = s.stack ? static_cast<size_t>(F) * Hkv * s.rows : 0;
    y.cut_row0 = static_cast<int>(own0 + own);
    rows = own0 + own + 2 * static_cast<size_t>(s.nb_max) * s.rows;
  }
  y.own_row0 = static_cast<int>(own0);
  y.rows = rows;
  if (y.rows > 0x7fffffffu) return false;
  s.by_R = Divisor(s.R);
  s.by_G = Divisor(s.G);
  s.by_TO = Divisor(s.TO);
  s.by_F = Divisor(s.F);
  s.by_chunk = Divisor(s.chunk > 0 ? s.chunk : 1);
  s.by_nrc = Divisor(s.nrc > 0 ? s.nrc : 1);
  s.by_cg = Divisor(s.cg > 0 ? s.cg : 1);
  size_t at = kStatusBytes;
  y.plan = at;
  at += 256;
  y.cta_err = at;
  at += align_up(static_cast<size_t>(y.n_cta) * 32, 256);
  y.own_rec = at;
  at += align_up(s.stack && !y.own_stream ? static_cast<size_t>(F) * Hkv * 8 : 0, 256);
  y.cut_rec = at;
  at += align_up(static_cast<size_t>(s.nb_max) * 8, 256);
  y.redo = at;
  at += align_up(static_cast<size_t>(y.n_cta) * kPxRedo * sizeof(PrefixItem), 256);
  y.lse = at;
  at += align_up(y.rows * 4, 256);
  y.o = at;
  y.total = at + y.rows * d * 4;
  y.wide = y.wide_pool = 0;
  y.room = y.total;
  // Pages of codes become tiles in the tile kernel, or, where a key tile meets many row tiles (each of which would do it again), bf16 pages in the workspace first.
  // us, in the kernel and before it, by row tiles:
  //                                             two        four        six         seven       eight       twelve
  //   2 x 16 heads x 12000 keys, 128 channels   74, 125    134, 197    185, 206    255, 235    252, 238    393, 351
  //                               64 channels   56, 73     98, 111     141, 147    194, 191    194, 191    285, 272
  //   8 heads x 12800 shared keys, 128          31, 49     47, 64      70, 88                  86, 79      121, 106
  //                                 64          26, 30     37, 40      55, 57                  66, 66      91, 88
  const long long own = y.own_stream ? 0 : s.stack ? most - PT : most, shared = s.stack ? PT : 0;
  if (codes > 0 && y.tile && TP * shared + F * own > kWidenTiles * (shared + B * own)) {
    // Room for the pages that the rows can name, which is what the copy is laid out by where the pool has more.
    const long long named = prefix_pages + (y.own_stream ? 0ll : (static_cast<long long>(width) - prefix_pages) * B);
    const size_t bytes = static_cast<size_t>(Hkv) * page * d * 2;
    if (named < codes) s.places = static_cast<int>(named);
    y.wide = align_up(y.total, 256);
    y.wide_pool = (s.places > 0 ? s.places : codes) * bytes;      // (below 2^62)
    y.total = y.wide + 2 * y.wide_pool;
    y.room = y.own_stream ? y.total : y.wide + 2 * (codes * bytes);
  }
  return true;
}

constexpr size_t kSmOnly = 116 * 1024;      // two CTAs with so much shared memory do not fit an SM (228 KB)

template <int D, int NT, class Source>
static int launch_stream_of(const Source& src, const PrefixParams& p, const StreamParams& t, int cluster, cudaStream_t st) {
  auto kernel = prefix_stream_kernel<D, NT, Source>;
  constexpr size_t kSmem = sizeof(StreamSmem<D, NT, Source::kQ4>);
  // Codes: no more CTAs to an SM than the call needs, by asking for more shared memory than there is for another one; else some SMs get four of 385 CTAs and others two (16 x 24
  // items of 1 to 1000 keys, us: 18.6, 17.1).  The limit belongs to the kernel, so every call sets the same.
  constexpr size_t kMost = Source::kQ4 ? kSmOnly : kSmem;
  static_assert(kSmem <= kMost, "shared memory of a CTA");
  const unsigned grid = static_cast<unsigned>((static_cast<long long>(t.items) * t.splits + t.check) * cluster);
  size_t smem = kSmem;
  if (Source::kQ4) {
    const unsigned sms = static_cast<unsigned>(persistent_grid(1 << 30)), ctas = (grid + sms - 1) / sms;
    if (ctas < static_cast<unsigned>(stream_ctas(NT, true)) && kSmOnly * 2 / (ctas + 1) > smem) smem = kSmOnly * 2 / (ctas + 1);
  }
  if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMost) != cudaSuccess) return AVSA_ERR_CUDA;
  return launch_pdl_clusters(kernel, cluster, grid, kStThreads, smem, st, src, p, t) == cudaSuccess ? AVSA_OK : AVSA_ERR_CUDA;
}
template <int D, class Source>
static int launch_stream(const Source& src, const PrefixParams& p, const StreamParams& t, int cluster, cudaStream_t st) {
  const int products = stream_products(Source::kQ4, D, t.stacked ? static_cast<long long>(p.s.B) * p.s.R : p.s.R);
  if constexpr (Source::kQ4)
    if (products == 3) return launch_stream_of<D, 3>(src, p, t, cluster, st);
  if constexpr (Source::kQ4 && D == 64)
    if (products == 4) return launch_stream_of<D, 4>(src, p, t, cluster, st);
  return products == 1 ? launch_stream_of<D, 1>(src, p, t, cluster, st) : launch_stream_of<D, 2>(src, p, t, cluster, st);
}

// `src`: of pages, where it is bf16.
template <int D, class Source>
static int launch_tile(const PrefixLayout& y, const Source& src, const PrefixParams& p, cudaStream_t st) {
  const PrefixShape& s = y.s;
  CUtensorMap tq_own = {}, tq_pre = {}, to = {};      // (not looked at where there is no box)
  // (an axis of one element has no stride to speak of: any multiple of 16 bytes)
  const int H = s.Hkv * s.G;
  const int64_t sh = H > 1 ? p.q.stride_h : D, sn = s.L > 1 ? p.q.stride_n : D, sb = s.B > 1 ? p.q.stride_b : D;
  auto box = [&](CUtensorMap* map, const void* ptr, int tokens, int entries) {
    return encode_bf16_map(map, ptr, {D, H, s.L, s.B}, {sh, sn, sb}, {64, s.G, tokens, entries});
  };
  if (!s.own_off && s.own_box > 0 && !(box(&tq_own, p.q.ptr, s.own_box / s.G, 1) && box(&to, p.o, s.own_box / s.G, 1))) return AVSA_ERR_CUDA;
  if (s.pre_box > 0 && !box(&tq_pre, p.q.ptr, s.L, s.pre_box / s.R)) return AVSA_ERR_CUDA;
  if (s.queue && launch_pdl(clear_counter_kernel, 1, 1, 0, st, p.counter) != cudaSuccess) return AVSA_ERR_CUDA;
  auto kernel = prefix_attn_kernel<D, Source>;
  if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, PrefixSmem<D, Source::kQ4>::kTotal) != cudaSuccess) return AVSA_ERR_CUDA;
  return launch_pdl(kernel, y.n_cta, px_threads(Source::kQ4), PrefixSmem<D, Source::kQ4>::kTotal, st, src, tq_own, tq_pre, to, p) == cudaSuccess ? AVSA_OK : AVSA_ERR_CUDA;
}

// The pools of a call: bf16, or codes, whose pages that the tile kernel reads are made bf16 in the workspace first.
struct PrefixPools {
  bool codes;
  avsa_bf16_4d k, v;
  avsa_q4_pool k4, v4;
};

// `src` is what the stream kernel reads, `tiles` what the tile kernel does.
template <int D, class Source, class TileSource>
static int launch_kernels(const PrefixLayout& y, const Source& src, const TileSource& tiles, const PrefixParams& p, cudaStream_t st) {
  const PrefixShape& s = y.s;
  constexpr int kRows = prefix_merge_rows(D);
  int r = AVSA_OK;
  if (y.pre_stream) r = launch_stream<D>(src, p, y.pre, 1, st);
  if (y.tile) r = launch_tile<D>(y, tiles, p, st);
  if (r != AVSA_OK) return r;
  if (y.own_stream) {
    r = launch_stream<D>(src, p, y.own, y.own_cluster, st);
    if (r != AVSA_OK) return r;
    if (y.own.splits > 1) {
      const long long rows = static_cast<long long>(s.B) * s.Hkv * s.R;
      if (launch_pdl(prefix_join_kernel<D>, static_cast<unsigned>(rows), kPxMergeThreads, 0, st, p, y.own) != cudaSuccess)
        return AVSA_ERR_CUDA;
    }
  } else {
    // (cut rows: at most nb_max times 128)
    const long long most = static_cast<long long>(s.nb_max) * 128 / kRows, ctas = 8ll * y.n_cta;
    dim3 grid(static_cast<unsigned>(most < ctas ? most : ctas));
    if (s.stack) grid = dim3(static_cast<unsigned>((static_cast<long long>(s.B) * s.R * s.Hkv + kRows - 1) / kRows));
    if (launch_pdl(prefix_merge_kernel<D>, grid, kPxMergeThreads, 0, st, p, y.n_cta) != cudaSuccess) return AVSA_ERR_CUDA;
  }
  return cudaGetLastError() == cudaSuccess ? AVSA_OK : AVSA_ERR_CUDA;
}

// Tensor maps of a bf16 pool, `rows` keys each.
template <int D>
static bool encode_tiles(PrefixTiles& t, const PrefixShape& s, int pages, const avsa_bf16_4d& k, const avsa_bf16_4d& v, int rows) {
  return encode_bf16_tile_map(&t.k, k.ptr, pages, s.Hkv, s.page, D, k.stride_b, k.stride_h, k.stride_n, rows) &&
         encode_bf16_tile_map(&t.v, v.ptr, pages, s.Hkv, s.page, D, v.stride_b, v.stride_h, v.stride_n, rows);
}

template <int D>
static int launch_prefix(const PrefixLayout& y, const PrefixPools& pools, const PrefixParams& p, uint8_t* ws, cudaStream_t st) {
  const PrefixShape& s = y.s;
  if (pools.codes) {
    const PrefixCodes src = {q4_pool(pools.k4), q4_pool(pools.v4)};
    if (y.wide_pool == 0) return launch_kernels<D>(y, src, src, p, st);
    avsa_bf16_4d k = {ws + y.wide, static_cast<int64_t>(s.Hkv) * s.page * D, static_cast<int64_t>(s.page) * D, D}, v = k;
    v.ptr = ws + y.wide + y.wide_pool;
    PrefixTiles wide;
    if (!encode_tiles<D>(wide, s, s.places > 0 ? s.places : s.pages, k, v, s.page)) return AVSA_ERR_CUDA;
    const int r = launch_widen(p, src.k, src.v, ws + y.wide, ws + y.wide + y.wide_pool, !y.own_stream, D, st);
    return r != AVSA_OK ? r : launch_kernels<D>(y, src, wide, p, st);
  }
  PrefixTiles few = {}, tiles = {};
  if ((y.own_stream && !encode_tiles<D>(few, s, s.pages, pools.k, pools.v, 16)) || (y.tile && !encode_tiles<D>(tiles, s, s.pages, pools.k, pools.v, s.page))) return AVSA_ERR_CUDA;
  return launch_kernels<D>(y, few, tiles, p, st);
}

static bool rows_ok(avsa_bf16_4d t, int B, int H, int N) {
  if (N == 1) t.stride_n = 8;      // (an axis of one element has no stride to speak of)
  return tensor_ok(t, B, H);
}

}  // namespace avsa

using namespace avsa;

static bool prefix_sizes_ok(int B, int H, int Hkv, int L, int d, int page, int width, int prefix_pages) {
  return B > 0 && H > 0 && Hkv > 0 && L > 0 && width > 0 && prefix_pages >= 0 && prefix_pages <= width && H % Hkv == 0 && H / Hkv <= 128 &&
         (d == 64 || d == 128) && (page == 16 || page == 32 || page == 64 || page == 128) && H <= 65535 && B <= 65535;
}

extern "C" size_t avsa_prefix_attn_workspace_bytes(int B, int H, int Hkv, int L, int d, int page, int width, int prefix_pages) {
  PrefixLayout y;
  if (!prefix_sizes_ok(B, H, Hkv, L, d, page, width, prefix_pages) || !prefix_layout(B, H, Hkv, L, d, page, width, prefix_pages, 0, 0, y)) return 0;
  return y.total;
}

extern "C" size_t avsa_prefix_attn_q4_workspace_bytes(int B, int H, int Hkv, int L, int d, int page, int pages, int width, int prefix_pages) {
  PrefixLayout y;
  if (pages <= 0 || !prefix_sizes_ok(B, H, Hkv, L, d, page, width, prefix_pages) || !prefix_layout(B, H, Hkv, L, d, page, width, prefix_pages, 0, pages, y)) return 0;
  return y.room;
}

static int prefix_attn(int B, int H, int Hkv, int L, int d, int page, int pages, int seqs, int width, avsa_bf16_4d q, const PrefixPools& pools, const int32_t* table,
                       const int32_t* length, const int32_t* seq, const int32_t* count, int prefix_pages, unsigned flags, float softmax_scale, void* o_bf16,
                       float* lse, int32_t* log, void* ws, size_t ws_bytes, void* stream) {
  if (B < 0 || H <= 0 || Hkv <= 0 || L < 0 || pages <= 0 || seqs <= 0 || width <= 0 || prefix_pages < 0 || prefix_pages > width) return AVSA_ERR_INVALID_ARG;
  if (H % Hkv != 0 || (flags & ~AVSA_CAUSAL) != 0 || (seq == nullptr && B > seqs)) return AVSA_ERR_INVALID_ARG;
  if ((d != 64 && d != 128) || (page != 16 && page != 32 && page != 64 && page != 128)) return AVSA_ERR_UNSUPPORTED;
  if (H > 65535 || B > 65535 || H / Hkv > 128) return AVSA_ERR_UNSUPPORTED;
  if (static_cast<long long>(seqs) * width > 0x7fffffffll || static_cast<long long>(width) * page > 0x7fffffffll ||
      static_cast<long long>(B) * H * L > 0x3fffffffll)
    return AVSA_ERR_UNSUPPORTED;
  if (!(softmax_scale >= 0.f) || isinf(softmax_scale)) return AVSA_ERR_INVALID_ARG;
  if (B == 0 || L == 0) return AVSA_OK;
  if (!rows_ok(q, B, H, L)) return AVSA_ERR_INVALID_ARG;
  if (pools.codes ? !q4_pool_ok(pools.k4, pages, Hkv, page, d) || !q4_pool_ok(pools.v4, pages, Hkv, page, d)
                  : !tensor_ok(pools.k, pages, Hkv) || !tensor_ok(pools.v, pages, Hkv))
    return AVSA_ERR_INVALID_ARG;
  if (table == nullptr || length == nullptr || o_bf16 == nullptr || !aligned16(o_bf16)) return AVSA_ERR_INVALID_ARG;
  if (!aligned4(table) || !aligned4(length) || !aligned4(seq) || !aligned4(count) || !aligned4(lse) || !aligned4(log)) return AVSA_ERR_INVALID_ARG;
  PrefixLayout y;
  if (!prefix_layout(B, H, Hkv, L, d, page, width, prefix_pages, flags & AVSA_CAUSAL ? 1 : 0, pools.codes ? pages : 0, y)) return AVSA_ERR_UNSUPPORTED;
  if (ws == nullptr || ws_bytes < y.total) return AVSA_ERR_WORKSPACE;
  if (!ws_aligned(ws, kWsParts)) return AVSA_ERR_INVALID_ARG;
  if (!device_is_sm100()) return AVSA_ERR_UNSUPPORTED;
  const float scale = softmax_scale != 0.f ? softmax_scale : 1.0f / sqrtf(static_cast<float>(d));
  uint8_t* w = static_cast<uint8_t*>(ws);
  y.s.pages = pages;
  y.s.seqs = seqs;
  PrefixParams p = {};
  p.s = y.s;
  p.q = q;
  p.o = static_cast<__nv_bfloat16*>(o_bf16);
  p.lse = lse;
  p.table = table;
  p.length = length;
  p.seq = seq;
  p.count = count;
  p.scale_log2 = scale * 1.4426950408889634f;
  p.status = static_cast<StatusRecord*>(ws);
  p.log = log;
  p.plan = reinterpret_cast<int*>(w + y.plan);
  p.counter = p.plan + 32;
  p.cta_err = reinterpret_cast<int4*>(w + y.cta_err);
  p.own_rec = reinterpret_cast<int2*>(w + y.own_rec);
  p.cut_rec = reinterpret_cast<int2*>(w + y.cut_rec);
  p.redo = reinterpret_cast<PrefixItem*>(w + y.redo);
  p.part_lse2 = reinterpret_cast<float*>(w + y.lse);
  p.part_o = reinterpret_cast<float*>(w + y.o);
  p.tile_ctas = y.tile ? y.n_cta : 0;
  p.own_row0 = y.own_row0;
  p.cut_row0 = y.cut_row0;
  return d == 128 ? launch_prefix<128>(y, pools, p, w, as_stream(stream)) : launch_prefix<64>(y, pools, p, w, as_stream(stream));
}

extern "C" int avsa_prefix_attn_step(int B, int H, int Hkv, int L, int d, int page, int pages, int seqs, int width, avsa_bf16_4d q,
                                     avsa_bf16_4d k_pool, avsa_bf16_4d v_pool, const int32_t* table, const int32_t* length,
                                     const int32_t* seq, const int32_t* count, int prefix_pages, unsigned flags, float softmax_scale,
                                     void* o_bf16, float* lse, int32_t* log, void* ws, size_t ws_bytes, void* stream) {
  const PrefixPools pools = {false, k_pool, v_pool, {}, {}};
  return prefix_attn(B, H, Hkv, L, d, page, pages, seqs, width, q, pools, table, length, seq, count, prefix_pages, flags, softmax_scale, o_bf16, lse, log, ws,
                     ws_bytes, stream);
}

extern "C" int avsa_prefix_attn_q4(int B, int H, int Hkv, int L, int d, int page, int pages, int seqs, int width, avsa_bf16_4d q, avsa_q4_pool k_pool,
                                   avsa_q4_pool v_pool, const int32_t* table, const int32_t* length, const int32_t* seq, const int32_t* count, int prefix_pages,
                                   unsigned flags, float softmax_scale, void* o_bf16, float* lse, int32_t* log, void* ws, size_t ws_bytes, void* stream) {
  const PrefixPools pools = {true, {}, {}, k_pool, v_pool};
  return prefix_attn(B, H, Hkv, L, d, page, pages, seqs, width, q, pools, table, length, seq, count, prefix_pages, flags, softmax_scale, o_bf16, lse, log, ws,
                     ws_bytes, stream);
}

extern "C" int avsa_prefix_attn(int B, int H, int Hkv, int L, int d, int page, int pages, int seqs, int width, avsa_bf16_4d q,
                                avsa_bf16_4d k_pool, avsa_bf16_4d v_pool, const int32_t* table, const int32_t* length,
                                const int32_t* seq, int prefix_pages, unsigned flags, float softmax_scale, void* o_bf16, float* lse,
                                void* ws, size_t ws_bytes, void* stream) {
  return avsa_prefix_attn_step(B, H, Hkv, L, d, page, pages, seqs, width, q, k_pool, v_pool, table, length, seq, nullptr, prefix_pages, flags,
                               softmax_scale, o_bf16, lse, nullptr, ws, ws_bytes, stream);
}
