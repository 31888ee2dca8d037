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

// Products of 8 columns for so many query rows: with 8 or less the second one's would be empty.
static int stream_products(long long rows) { return rows <= 8 ? 1 : 2; }

struct PrefixLayout {
  PrefixShape s;
  int n_cta;                    // of the tile kernel
  int tile;                     // there is one
  int pre_stream, own_stream;   // the stream kernel takes the beginning, the own items
  StreamParams pre, own;
  int own_cluster;
  size_t rows;                  // partial rows
  int own_row0, cut_row0;
  size_t plan, cta_err, own_rec, cut_rec, redo, lse, o, total;       // offsets in the workspace
};

// False: more units, or key positions rounded up to a tile, than 32 bits count.
static bool prefix_layout(int B, int H, int Hkv, int L, int d, int page, int width, int prefix_pages, int causal, PrefixLayout& y) {
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
  s.page_shift = page == 16 ? 4 : page == 32 ? 5 : page == 64 ? 6 : 7;
  const int sms = persistent_grid(1 << 30);
  // Stacked, the beginning's key tiles are walked TP times a head instead of F times, but every row goes through the merge, which costs a key
  // tile's time for about six rows (149760 rows: 108 us, a tile of every SM 0.8), and the call has a kernel more (about eight tiles' time of every SM).
  s.stack = TP * PT + RS / 6 < F * PT && (F * PT - TP * PT - RS / 6) * Hkv > 8 * sms;
  if (s.stack) s.k0 = prefix_pages * page;
  y.own_stream = R <= kStreamRows;
  y.pre_stream = s.stack && RS <= kStreamRows;
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
    y.pre.tiles = static_cast<int>((RS + kStRows - 1) / kStRows);
    y.pre.items = y.pre.tiles * Hkv;
    const int slots = sms * stream_ctas(stream_products(RS));      // CTAs of the stream kernel that the SMs hold
    const long long by_keys = PT / 2;      // 256 keys a CTA at least: four blocks a warp
    y.pre.splits = static_cast<int>(slots / y.pre.items < by_keys ? slots / y.pre.items : by_keys);
    // The kernel behind joins a row's parts eight at a time, 0.7 us each, so with few heads fewer and longer parts end earlier (4 heads x 60000 keys, us: 111 parts 35.8, 70 31.7).
    while (y.pre.splits > 8 && 12ll * y.pre.splits * y.pre.splits > s.k0) y.pre.splits--;
    if (y.pre.splits < 1) y.pre.splits = 1;
    rows += static_cast<size_t>(y.pre.items) * y.pre.splits * kStRows;
  } else if (s.stack) {
    rows += (static_cast<size_t>(y.n_cta) + static_cast<size_t>(Hkv) * s.nrc * s.chunk) * 128;
  }
  const size_t own0 = rows;
  if (y.own_stream) {
    y.own.first = !s.stack;
    y.own.join = !s.stack ? 0 : y.pre_stream ? kStJoinStream : kStJoinTile;
    y.own.join_tiles = y.pre.tiles;
    y.own.join_splits = y.pre.splits;
    y.own.tiles = static_cast<int>((R + kStRows - 1) / kStRows);
    y.own.items = y.own.tiles * Hkv * B;
    y.own.out0 = static_cast<int>(own0);
    const long long keys = static_cast<long long>(width) * page - s.k0;      // at most
    const int slots = sms * stream_ctas(stream_products(R));
    // An item's keys over a cluster, 64 keys a CTA at least (a block a warp), as many CTAs as the SMs hold side by side: nine tenths of the slots, since a cluster takes its
    // own from one GPC and what does not fit waits for a whole item (us, filled to the last slot and like this: 96 items of 500 keys of 64 channels 14.4 and 9.7, 72
    // of 900 keys of 128 channels 16.4 and 10.3, 144 of 800 17.5 and 13.0).  No CTA has more than 1024 keys while others may have none (30 x 8 items of 1 to 1500
    // keys 15.7, of up to 1500 keys a CTA 17.0, but all of 1500 keys 24.5 and 19.7).  What eight CTAs an item do not fill is cut into parts that a kernel behind joins.
    const long long fit = slots * 9ll / 10 / (y.own.items + 1ll), by_keys = keys / 64;
    long long ctas = fit < by_keys ? fit : by_keys;
    ctas = ctas < 1 ? 1 : ctas > 8 ? 8 : ctas;
    while (ctas < 8 && y.own.items < (1 << 27) && keys > 1024 * ctas) ctas = 2 * ctas < 8 ? 2 * ctas : 8;
    y.own_cluster = static_cast<int>(ctas);
    y.own.splits = 1;
    if (static_cast<long long>(y.own.items) * 8 < sms && keys >= 4096) {
      y.own_cluster = 1;
      y.own.splits = (slots - 1) / y.own.items;      // (one slot for the check of the tables)
      rows += static_cast<size_t>(y.own.items) * y.own.splits * kStRows;
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
  return true;
}

template <int D, int NT>
static int launch_stream_of(const CUtensorMap& tk, const CUtensorMap& tv, const PrefixParams& p, const StreamParams& t, int cluster, cudaStream_t st) {
  auto kernel = prefix_stream_kernel<D, NT>;
  constexpr size_t kSmem = sizeof(StreamSmem<D, NT>);
  if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem) != cudaSuccess) return AVSA_ERR_CUDA;
  const unsigned grid = static_cast<unsigned>((static_cast<long long>(t.items) * t.splits + t.check) * cluster);
  return launch_pdl_clusters(kernel, cluster, grid, kStThreads, kSmem, st, tk, tv, p, t) == cudaSuccess ? AVSA_OK : AVSA_ERR_CUDA;
}
template <int D>
static int launch_stream(const CUtensorMap& tk, const CUtensorMap& tv, const PrefixParams& p, const StreamParams& t, int cluster, cudaStream_t st) {
  return stream_products(t.stacked ? static_cast<long long>(p.s.B) * p.s.R : p.s.R) == 1 ? launch_stream_of<D, 1>(tk, tv, p, t, cluster, st)
                                                                                          : launch_stream_of<D, 2>(tk, tv, p, t, cluster, st);
}

template <int D>
static int launch_tile(const PrefixLayout& y, const avsa_bf16_4d& k, const avsa_bf16_4d& v, const PrefixParams& p, cudaStream_t st) {
  const PrefixShape& s = y.s;
  CUtensorMap tk, tv, tq_own, tq_pre, to;
  if (!encode_bf16_tile_map(&tk, k.ptr, s.pages, s.Hkv, s.page, D, k.stride_b, k.stride_h, k.stride_n, s.page) ||
      !encode_bf16_tile_map(&tv, v.ptr, s.pages, s.Hkv, s.page, D, v.stride_b, v.stride_h, v.stride_n, s.page))
    return AVSA_ERR_CUDA;
  // (an axis of one element has no stride to speak of: any multiple of 16 bytes)
  const int H = s.Hkv * s.G;
  const int64_t sh = H > 1 ? p.q.stride_h : D, sn = s.L > 1 ? p.q.stride_n : D, sb = s.B > 1 ? p.q.stride_b : D;
  auto box = [&](CUtensorMap* map, const void* ptr, int tokens, int entries) {
    return encode_bf16_map(map, ptr, {D, H, s.L, s.B}, {sh, sn, sb}, {64, s.G, tokens, entries});
  };
  tq_own = tq_pre = to = tk;      // (where there is no box)
  if (!s.own_off && s.own_box > 0 && !(box(&tq_own, p.q.ptr, s.own_box / s.G, 1) && box(&to, p.o, s.own_box / s.G, 1))) return AVSA_ERR_CUDA;
  if (s.pre_box > 0 && !box(&tq_pre, p.q.ptr, s.L, s.pre_box / s.R)) return AVSA_ERR_CUDA;
  if (s.queue && launch_pdl(clear_counter_kernel, 1, 1, 0, st, p.counter) != cudaSuccess) return AVSA_ERR_CUDA;
  if (cudaFuncSetAttribute(prefix_attn_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, PrefixSmem<D>::kTotal) != cudaSuccess) return AVSA_ERR_CUDA;
  return launch_pdl(prefix_attn_kernel<D>, y.n_cta, kPxThreads, PrefixSmem<D>::kTotal, st, tk, tv, tq_own, tq_pre, to, p) == cudaSuccess ? AVSA_OK : AVSA_ERR_CUDA;
}

template <int D>
static int launch_prefix(const PrefixLayout& y, const avsa_bf16_4d& k, const avsa_bf16_4d& v, const PrefixParams& p, cudaStream_t st) {
  const PrefixShape& s = y.s;
  constexpr int kRows = prefix_merge_rows(D);
  int r = AVSA_OK;
  CUtensorMap tk, tv;      // of 16 keys
  if (y.own_stream && (!encode_bf16_tile_map(&tk, k.ptr, s.pages, s.Hkv, s.page, D, k.stride_b, k.stride_h, k.stride_n, 16) ||
                       !encode_bf16_tile_map(&tv, v.ptr, s.pages, s.Hkv, s.page, D, v.stride_b, v.stride_h, v.stride_n, 16)))
    return AVSA_ERR_CUDA;
  if (y.pre_stream) r = launch_stream<D>(tk, tv, p, y.pre, 1, st);
  if (y.tile) r = launch_tile<D>(y, k, v, p, st);
  if (r != AVSA_OK) return r;
  if (y.own_stream) {
    r = launch_stream<D>(tk, tv, p, y.own, y.own_cluster, st);
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
  if (!prefix_sizes_ok(B, H, Hkv, L, d, page, width, prefix_pages) || !prefix_layout(B, H, Hkv, L, d, page, width, prefix_pages, 0, y)) return 0;
  return y.total;
}

extern "C" int avsa_prefix_attn_step(int B, int H, int Hkv, int L, int d, int page, int pages, int seqs, int width, avsa_bf16_4d q,
                                     avsa_bf16_4d k_pool, avsa_bf16_4d v_pool, const int32_t* table, const int32_t* length,
                                     const int32_t* seq, const int32_t* count, int prefix_pages, unsigned flags, float softmax_scale,
                                     void* o_bf16, float* lse, int32_t* log, void* ws, size_t ws_bytes, void* stream) {
  if (B < 0 || H <= 0 || Hkv <= 0 || L < 0 || pages <= 0 || seqs <= 0 || width <= 0 || prefix_pages < 0 || prefix_pages > width) return AVSA_ERR_INVALID_ARG;
  if (H % Hkv != 0 || (flags & ~AVSA_CAUSAL) != 0 || (seq == nullptr && B > seqs)) return AVSA_ERR_INVALID_ARG;
  if ((d != 64 && d != 128) || (page != 16 && page != 32 && page != 64 && page != 128)) return AVSA_ERR_UNSUPPORTED;
  if (H > 65535 || B > 65535 || H / Hkv > 128) return AVSA_ERR_UNSUPPORTED;
  if (static_cast<long long>(seqs) * width > 0x7fffffffll || static_cast<long long>(width) * page > 0x7fffffffll ||
      static_cast<long long>(B) * H * L > 0x3fffffffll)
    return AVSA_ERR_UNSUPPORTED;
  if (!(softmax_scale >= 0.f) || isinf(softmax_scale)) return AVSA_ERR_INVALID_ARG;
  if (B == 0 || L == 0) return AVSA_OK;
  if (!rows_ok(q, B, H, L) || !tensor_ok(k_pool, pages, Hkv) || !tensor_ok(v_pool, pages, Hkv)) return AVSA_ERR_INVALID_ARG;
  if (table == nullptr || length == nullptr || o_bf16 == nullptr || !aligned16(o_bf16)) return AVSA_ERR_INVALID_ARG;
  if (!aligned4(table) || !aligned4(length) || !aligned4(seq) || !aligned4(count) || !aligned4(lse) || !aligned4(log)) return AVSA_ERR_INVALID_ARG;
  PrefixLayout y;
  if (!prefix_layout(B, H, Hkv, L, d, page, width, prefix_pages, flags & AVSA_CAUSAL ? 1 : 0, y)) return AVSA_ERR_UNSUPPORTED;
  if (ws == nullptr || ws_bytes < y.total) return AVSA_ERR_WORKSPACE;
  if (!ws_aligned(ws, kWsParts)) return AVSA_ERR_INVALID_ARG;
  if (!device_is_sm100()) return AVSA_ERR_UNSUPPORTED;
  const float scale = softmax_scale != 0.f ? softmax_scale : 1.0f / sqrtf(static_cast<float>(d));
  uint8_t* w = static_cast<uint8_t*>(ws);
  y.s.pages = pages;
  y.s.seqs = seqs;
  y.s.width = width;
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
  return d == 128 ? launch_prefix<128>(y, k_pool, v_pool, p, as_stream(stream)) : launch_prefix<64>(y, k_pool, v_pool, p, as_stream(stream));
}

extern "C" int avsa_prefix_attn(int B, int H, int Hkv, int L, int d, int page, int pages, int seqs, int width, avsa_bf16_4d q,
                                avsa_bf16_4d k_pool, avsa_bf16_4d v_pool, const int32_t* table, const int32_t* length,
                                const int32_t* seq, int prefix_pages, unsigned flags, float softmax_scale, void* o_bf16, float* lse,
                                void* ws, size_t ws_bytes, void* stream) {
  return avsa_prefix_attn_step(B, H, Hkv, L, d, page, pages, seqs, width, q, k_pool, v_pool, table, length, seq, nullptr, prefix_pages, flags,
                               softmax_scale, o_bf16, lse, nullptr, ws, ws_bytes, stream);
}
