// A paged cache held in 4 bits: new tokens into the pages, tokens out of them again, and the pages of an attention call as bf16.
//
// All three are bound by HBM (2.56 bytes a value, 2 outside and 4.5 bits inside; 49152 tokens of 8 heads of 128 channels read, 258 MB, 41.7 us, 6.2 TB/s; 6018 tokens of 24 heads
// written, 95 MB, 17.9 us, of which three are the length, the page and the launch before the first token is asked for).  A thread has the 32 channels of a scale, so a group's maximum needs no other thread, and
// its codes are one 16-byte access.  Neighbouring threads have a token's groups, then the tokens of a head: the codes of a warp's eight tokens (128 channels) are
// 512 contiguous bytes.
#include "prefix_stream.cuh"

namespace avsa {

constexpr int kQ4Threads = 128;      // eight CTAs of 64 registers (us, the write and the read above: 19.0 and 41.8; CTAs of 256 threads 21.6 and 46.1, four of them forced 19.7 and 42.3)

// 64 bytes of a thread's own, in vectors of 32 bytes where they are aligned to these.
template <bool WIDE>
__device__ __forceinline__ void load_group(const __nv_bfloat16* at, uint32_t (&x)[16]) {
  if constexpr (WIDE) {
#pragma unroll
    for (int i = 0; i < 16; i += 8)
      asm volatile("ld.global.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                   : "=r"(x[i]), "=r"(x[i + 1]), "=r"(x[i + 2]), "=r"(x[i + 3]), "=r"(x[i + 4]), "=r"(x[i + 5]), "=r"(x[i + 6]), "=r"(x[i + 7])
                   : "l"(at + 2 * i));
  } else {
#pragma unroll
    for (int i = 0; i < 16; i += 4) *reinterpret_cast<uint4*>(&x[i]) = *reinterpret_cast<const uint4*>(at + 2 * i);
  }
}
template <bool WIDE>
__device__ __forceinline__ void store_group(__nv_bfloat16* at, const uint32_t (&x)[16]) {
  if constexpr (WIDE) {
    st_global_v8(at, *reinterpret_cast<const uint32_t(*)[8]>(&x[0]));
    st_global_v8(at + 16, *reinterpret_cast<const uint32_t(*)[8]>(&x[8]));
  } else {
#pragma unroll
    for (int i = 0; i < 16; i += 4) *reinterpret_cast<uint4*>(at + 2 * i) = *reinterpret_cast<const uint4*>(&x[i]);
  }
}

// Codes and scale (bf16 bits) of 32 channels.
__device__ __forceinline__ uint4 quantise(const uint32_t (&x)[16], uint32_t& scale) {
  uint32_t top2 = 0;      // largest magnitudes, NaN where there is one: as numbers of 16 bits above infinity, which is above what is finite
#pragma unroll
  for (int i = 0; i < 16; i++)
    asm("{.reg .b32 y; abs.bf16x2 y, %1; max.NaN.bf16x2 %0, %0, y;}" : "+r"(top2) : "r"(x[i]));
  const uint32_t top = max(top2 >> 16, top2 & 0xffffu);
  const uint32_t third = __float_as_uint(__fdiv_rn(__uint_as_float(top << 16), 7.0f));
  const uint32_t s32 = (third + 0x40000u) & ~0x7ffffu;      // five significant bits
  const bool some = top >= kQ4Least && top < kQ4Most;
  scale = some ? s32 >> 16 : top >= kQ4Most ? 0x7fffu : 0u;
  const float inv = some ? __frcp_rn(__uint_as_float(s32)) : 0.f;
  const uint64_t inv2 = pack_f32x2(inv, inv), grid = pack_f32x2(1536.f, 1536.f), no_grid = pack_f32x2(-1536.f, -1536.f), whole = pack_f32x2(12582920.f, 12582920.f);
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 16; i++) {
    // x / s is a half of an odd number or at least 2^-10 away from one (x has 8 significant bits and s 5), and x * inv is within 2^-21 of it: to a grid of 2^-13
    // first, ties are ties again, and the last addition rounds as the quotient would (to even), and leaves the code, + 8, in the low bits.  Both values of a
    // register in one instruction each (the write was 62 % of the issue slots, a frame's 19 us).
    const uint64_t y = add_f32x2(add_f32x2(fma_f32x2(pack_f32x2(__uint_as_float(x[i] << 16), __uint_as_float(x[i] & 0xffff0000u)), inv2, grid), no_grid), whole);
    float a, b;
    unpack_f32x2(y, a, b);
    const uint32_t pair = __byte_perm(__float_as_uint(a), __float_as_uint(b), 0x5410);
    w[i >> 2] = (i & 3) == 0 ? pair : w[i >> 2] | pair << (4 * (i & 3));
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// The other way: pairs of neighbours.
__device__ __forceinline__ void widen(uint4 codes, uint32_t scale, uint32_t sixteen, uint32_t (&x)[16]) {
  const uint32_t s2 = scale | scale << 16, c2 = q4_offset(s2), w[4] = {codes.x, codes.y, codes.z, codes.w};
#pragma unroll
  for (int i = 0; i < 16; i++) x[i] = q4_pair(w[i >> 2], i & 3, s2, c2, sixteen);
}

// Where token `in` of a page has the codes and the scale of a group.
template <int D>
__device__ __forceinline__ void q4_places(const Q4Pool& p, int page, int head, int in, int group, uint8_t*& codes, uint16_t*& scale) {
  uint8_t* const block = p.ptr + page * p.stride_page + head * p.stride_head + static_cast<int64_t>(in / kQ4Tokens) * q4_block_bytes(D);
  codes = block + (in % kQ4Tokens) * (D / 2) + group * (kQ4Group / 2);
  scale = reinterpret_cast<uint16_t*>(block + q4_scales_at(D)) + (in % kQ4Tokens) * (D / kQ4Group) + group;
}

struct TokensQ4Args {
  avsa_bf16_4d k, v;       // [n,Hkv,T,d]
  Q4Pool k_pool, v_pool;
  const int32_t *table, *length, *seq, *count;
  int Hkv, T;
  int head_shift, token_shift;      // a CTA's tile: 2^head_shift heads of 2^token_shift tokens
  int page_shift, pages, seqs, width;
};

// The last count[k] of the length[s] tokens of sequence s = seq[k].  READ: out of the pages, and zeros where there is none; else into them.
template <int D, bool READ, bool WIDE>
__global__ void __launch_bounds__(kQ4Threads, 8) tokens_q4_kernel(const __grid_constant__ TokensQ4Args a) {
  pdl_wait();
  pdl_launch();
  constexpr int G = D / kQ4Group;
  const int e = blockIdx.z, s = a.seq != nullptr ? a.seq[e] : e;
  const bool known = s >= 0 && s < a.seqs;
  const int count = !known ? 0 : a.count != nullptr ? min(a.count[e], a.T) : a.T;
  const int t0 = blockIdx.x << a.token_shift, h0 = blockIdx.y << a.head_shift;
  if (!READ && t0 >= count) return;
  const long long start = known ? static_cast<long long>(a.length[s]) - count : 0;
  const int32_t* const row = a.table + static_cast<long long>(known ? s : 0) * a.width;
  for (int i = threadIdx.x; i < G << (a.token_shift + a.head_shift); i += kQ4Threads) {
    const int group = i % G, r = i / G, t = t0 + (r & ((1 << a.token_shift) - 1)), h = h0 + (r >> a.token_shift);
    if (h >= a.Hkv || t >= a.T) continue;
    __nv_bfloat16* const k = static_cast<__nv_bfloat16*>(const_cast<void*>(a.k.ptr)) + e * a.k.stride_b + h * a.k.stride_h + t * a.k.stride_n + group * kQ4Group;
    __nv_bfloat16* const v = static_cast<__nv_bfloat16*>(const_cast<void*>(a.v.ptr)) + e * a.v.stride_b + h * a.v.stride_h + t * a.v.stride_n + group * kQ4Group;
    uint32_t x[16], y[16];
    if (!READ && t < count) {      // (asked for beside the page, which hardly a token lacks: 18.4 us behind it)
      load_group<WIDE>(k, x);
      load_group<WIDE>(v, y);
    }
    const long long pos = start + t;
    int page = -1;
    if (t < count && pos >= 0 && (pos >> a.page_shift) < a.width) page = row[pos >> a.page_shift];
    const bool there = page >= 0 && page < a.pages;
    const int in = static_cast<int>(pos & ((1 << a.page_shift) - 1));
    uint8_t *k_codes, *v_codes;
    uint16_t *k_scale, *v_scale;
    q4_places<D>(a.k_pool, there ? page : 0, h, in, group, k_codes, k_scale);
    q4_places<D>(a.v_pool, there ? page : 0, h, in, group, v_codes, v_scale);
    if constexpr (READ) {
      uint4 kc = make_uint4(0u, 0u, 0u, 0u), vc = kc;
      uint32_t ks = 0, vs = 0;
      if (there) {
        kc = *reinterpret_cast<const uint4*>(k_codes);
        vc = *reinterpret_cast<const uint4*>(v_codes);
        ks = *k_scale;
        vs = *v_scale;
      }
      widen(kc, ks, a.k_pool.sixteen, x);      // (a scale of zero: 16 * 0 - 24 * 0 = 0)
      widen(vc, vs, a.k_pool.sixteen, y);
      store_group<WIDE>(k, x);
      store_group<WIDE>(v, y);
    } else if (there) {
      uint32_t ks, vs;
      const uint4 kc = quantise(x, ks), vc = quantise(y, vs);
      *reinterpret_cast<uint4*>(k_codes) = kc;
      *reinterpret_cast<uint4*>(v_codes) = vc;
      *k_scale = static_cast<uint16_t>(ks);
      *v_scale = static_cast<uint16_t>(vs);
    }
  }
}

// The pages that the batch of an attention call reads, as bf16: those of batch entry `entry` behind the shared ones, or, of the entry behind the last one, the beginning, as
// the longest sequence's row of the table has it.  Laid out by page numbers, entries whose neighbour in front has the same page at the same place leave it to that one (branches of
// one parent; of others that share a page several write the same values); by places, each entry has its own, and what the beginning lacks is zeros (the tile kernel goes by
// the rows of its items).  2.56 bytes a value, and the copy is read from L2 or HBM once more by the tile kernel.
template <int D>
__global__ void __launch_bounds__(kQ4Threads) widen_pages_kernel(const __grid_constant__ PrefixParams p, Q4Pool k4, Q4Pool v4, __nv_bfloat16* k, __nv_bfloat16* v,
                                                                 int chunks, int first) {
  pdl_wait();
  pdl_launch();
  constexpr int G = D / kQ4Group, GS = G == 4 ? 2 : 1;
  const PrefixShape& S = p.s;
  const int entry = blockIdx.x / chunks, chunk = blockIdx.x - entry * chunks, b = first + entry, h = blockIdx.y;
  const bool by_place = S.places > 0;
  const int shared = by_place || S.stack ? S.shared : 0;
  int slot, bad, e0 = shared, e1 = 0, before = -1, before_e1 = 0;
  if (b < S.B) {
    e1 = (prefix_sequence(p, b, slot, bad) + S.page - 1) >> S.page_shift;
    if (b > 0 && !by_place) before_e1 = (prefix_sequence(p, b - 1, before, bad) + S.page - 1) >> S.page_shift;
  } else {
    int tokens, who;
    longest_sequence(p, slot, tokens, who);
    e0 = 0;
    e1 = min(shared, (tokens + S.page - 1) >> S.page_shift);
  }
  const int shift = S.page_shift + GS;      // threads of a page
  const long long n = static_cast<long long>(e1 - e0) << shift;
  for (long long u = static_cast<long long>(chunk) * kQ4Threads + threadIdx.x; u < n; u += static_cast<long long>(chunks) * kQ4Threads) {
    const int e = e0 + static_cast<int>(u >> shift), i = static_cast<int>(u & ((1 << shift) - 1)), in = i / G, group = i % G;
    const int page = p.table[static_cast<int64_t>(slot) * S.width + e];
    const bool there = page >= 0 && page < S.pages;
    if (!there && !by_place) continue;
    if (e < before_e1 && p.table[static_cast<int64_t>(before) * S.width + e] == page) continue;
    uint8_t *k_codes, *v_codes;
    uint16_t *k_scale, *v_scale;
    q4_places<D>(k4, there ? page : 0, h, in, group, k_codes, k_scale);
    q4_places<D>(v4, there ? page : 0, h, in, group, v_codes, v_scale);
    const uint4 kc = *reinterpret_cast<const uint4*>(k_codes), vc = *reinterpret_cast<const uint4*>(v_codes);
    const uint32_t ks = there ? *k_scale : 0u, vs = there ? *v_scale : 0u;
    const int64_t at = by_place ? prefix_place(S, e, b < S.B ? b : 0) : page;
    const int64_t to = ((at * S.Hkv + h) * S.page + in) * D + group * kQ4Group;
    uint32_t x[16];
    widen(kc, ks, k4.sixteen, x);
    store_group<true>(k + to, x);
    widen(vc, vs, k4.sixteen, x);
    store_group<true>(v + to, x);
  }
}

int launch_widen(const PrefixParams& p, Q4Pool k4, Q4Pool v4, void* k, void* v, bool own, int d, cudaStream_t st) {
  const PrefixShape& s = p.s;
  const int first = own ? 0 : s.B;
  const long long entries = static_cast<long long>(s.B) - first + (s.stack || (s.places > 0 && s.shared > 0) ? 1 : 0);
  const long long most = static_cast<long long>(s.width) * s.page * (d / kQ4Group) / kQ4Threads + 1;      // CTAs that the longest row could use
  // As many CTAs to an entry whatever it has: a beginning is most of all pages, so four times what the SMs hold (a frame of 4 candidates by places, us: 16 CTAs an SM 1067, 32 1054, 64 1049).
  long long chunks = persistent_grid(1 << 30) * 64ll / (entries * s.Hkv) + 1;
  if (chunks > most) chunks = most;
  const dim3 grid(static_cast<unsigned>(chunks * entries), static_cast<unsigned>(s.Hkv));
  auto kernel = d == 128 ? widen_pages_kernel<128> : widen_pages_kernel<64>;
  return launch_pdl(kernel, grid, kQ4Threads, 0, st, p, k4, v4, static_cast<__nv_bfloat16*>(k), static_cast<__nv_bfloat16*>(v), static_cast<int>(chunks), first) ==
                 cudaSuccess
             ? AVSA_OK
             : AVSA_ERR_CUDA;
}

static bool rows_fit(avsa_bf16_4d t, int B, int H, int N) {
  if (N == 1) t.stride_n = 8;      // (an axis of one element has no stride to speak of)
  return tensor_ok(t, B, H);
}
static bool wide_rows(const avsa_bf16_4d& t, int B, int H, int N) {
  return (reinterpret_cast<uintptr_t>(t.ptr) & 31u) == 0 && (B == 1 || t.stride_b % 16 == 0) && (H == 1 || t.stride_h % 16 == 0) && (N == 1 || t.stride_n % 16 == 0);
}

template <bool READ>
static int tokens_q4(int n, int Hkv, int T, int d, int page, int pages, int seqs, int width, const avsa_bf16_4d& k, const avsa_bf16_4d& v, const avsa_q4_pool& k_pool,
                     const avsa_q4_pool& v_pool, const int32_t* table, const int32_t* length, const int32_t* seq, const int32_t* count, void* stream) {
  if (n < 0 || Hkv <= 0 || T < 0 || pages <= 0 || seqs <= 0 || width <= 0) return AVSA_ERR_INVALID_ARG;
  if ((d != 64 && d != 128) || (page != 16 && page != 32 && page != 64 && page != 128) || n > 65535 || Hkv > 65535 || T > (1 << 30) || static_cast<long long>(seqs) * width > 0x7fffffffll)
    return AVSA_ERR_UNSUPPORTED;
  if (seq == nullptr && n > seqs) return AVSA_ERR_INVALID_ARG;
  if (table == nullptr || length == nullptr || !q4_pool_ok(k_pool, pages, Hkv, page, d) || !q4_pool_ok(v_pool, pages, Hkv, page, d)) return AVSA_ERR_INVALID_ARG;
  if (!aligned4(table) || !aligned4(length) || !aligned4(seq) || !aligned4(count)) return AVSA_ERR_INVALID_ARG;
  if (n == 0 || T == 0) return AVSA_OK;
  if (!rows_fit(k, n, Hkv, T) || !rows_fit(v, n, Hkv, T)) return AVSA_ERR_INVALID_ARG;
  if (!device_is_sm100()) return AVSA_ERR_UNSUPPORTED;
  TokensQ4Args a = {k, v, q4_pool(k_pool), q4_pool(v_pool), table, length, seq, count, Hkv, T, 0, 0, 0, pages, seqs, width};
  while ((1 << a.page_shift) < page) a.page_shift++;
  // sixteen tokens (as many as there are), and as many heads as give every thread a group
  const int units = kQ4Threads / (d / kQ4Group);
  while ((1 << a.token_shift) < T && a.token_shift < 4) a.token_shift++;
  while (1 << (a.token_shift + a.head_shift + 1) <= units && (1 << a.head_shift) < Hkv) a.head_shift++;
  while (1 << (a.token_shift + a.head_shift + 1) <= units && (1 << a.token_shift) < T) a.token_shift++;
  const dim3 grid(static_cast<unsigned>((T + (1 << a.token_shift) - 1) >> a.token_shift), static_cast<unsigned>((Hkv + (1 << a.head_shift) - 1) >> a.head_shift), static_cast<unsigned>(n));
  const bool wide = wide_rows(k, n, Hkv, T) && wide_rows(v, n, Hkv, T);
  auto kernel = d == 128 ? (wide ? tokens_q4_kernel<128, READ, true> : tokens_q4_kernel<128, READ, false>)
                         : (wide ? tokens_q4_kernel<64, READ, true> : tokens_q4_kernel<64, READ, false>);
  if (launch_pdl(kernel, grid, kQ4Threads, 0, as_stream(stream), a) != cudaSuccess) return AVSA_ERR_CUDA;
  return cudaGetLastError() == cudaSuccess ? AVSA_OK : AVSA_ERR_CUDA;
}

}  // namespace avsa

using namespace avsa;

extern "C" int avsa_cache_write_q4(int n, int Hkv, int L, int d, int page, int pages, int seqs, int width, avsa_bf16_4d k_new, avsa_bf16_4d v_new,
                                   avsa_q4_pool k_pool, avsa_q4_pool v_pool, const int32_t* table, const int32_t* length, const int32_t* seq, const int32_t* count,
                                   void* stream) {
  return tokens_q4<false>(n, Hkv, L, d, page, pages, seqs, width, k_new, v_new, k_pool, v_pool, table, length, seq, count, stream);
}

extern "C" int avsa_cache_read_q4(int n, int Hkv, int T, int d, int page, int pages, int seqs, int width, avsa_q4_pool k_pool, avsa_q4_pool v_pool,
                                  const int32_t* table, const int32_t* length, const int32_t* seq, const int32_t* count, avsa_bf16_4d k, avsa_bf16_4d v, void* stream) {
  return tokens_q4<true>(n, Hkv, T, d, page, pages, seqs, width, k, v, k_pool, v_pool, table, length, seq, count, stream);
}
