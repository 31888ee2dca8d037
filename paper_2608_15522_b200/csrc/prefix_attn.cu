// Attention of a batch that shares a long beginning, over a paged cache.
#include <math.h>

#include "avsa_common.cuh"
#include "sm100_ptx.cuh"

namespace avsa {

enum PrefixWhere { kPrefixPage = 221, kPrefixLength, kPrefixSeq };

struct PrefixParams {
  avsa_bf16_4d q, k, v;
  __nv_bfloat16* o;
  float* lse;
  const int32_t *table, *length, *seq;
  StatusRecord* status;
  int B, H, G, L;           // G: query heads of a key head
  int page, pages, seqs, width;
  int causal;
  float scale_log2;
};

// A warp per row, key after key: the running maximum and sum, the row of O in registers.
template <int D>
__global__ void __launch_bounds__(256) prefix_rows_kernel(const PrefixParams p) {
  pdl_wait();
  pdl_launch();
  const long long r = static_cast<long long>(blockIdx.x) * 8 + (threadIdx.x >> 5);
  const int lane = threadIdx.x & 31;
  if (r >= static_cast<long long>(p.B) * p.H * p.L) return;
  const int i = static_cast<int>(r % p.L), h = static_cast<int>(r / p.L % p.H), b = static_cast<int>(r / p.L / p.H);
  constexpr int C = D / 32;
  float q[C], o[C] = {};
  const __nv_bfloat16* qr = static_cast<const __nv_bfloat16*>(p.q.ptr) + b * p.q.stride_b + h * p.q.stride_h + i * p.q.stride_n;
#pragma unroll
  for (int c = 0; c < C; c++) q[c] = __bfloat162float(qr[lane * C + c]) * p.scale_log2;
  const int s = p.seq != nullptr ? p.seq[b] : b;
  long long lim = 0;
  if (s >= p.seqs) {
    if (lane == 0) report_status(p.status, AVSA_ERR_BAD_TABLE, kPrefixSeq, b, s);
  } else if (s >= 0) {
    long long n = p.length[s];
    if (n < 0 || n > static_cast<long long>(p.width) * p.page) {
      if (lane == 0) report_status(p.status, AVSA_ERR_BAD_TABLE, kPrefixLength, s, static_cast<int>(n));
      n = n < 0 ? 0 : static_cast<long long>(p.width) * p.page;
    }
    lim = p.causal ? n - p.L + i + 1 : n;
  }
  float m = -INFINITY, l = 0.f;
  for (int t = 0; t < lim; t++) {
    const int page = p.table[static_cast<long long>(s) * p.width + t / p.page];
    if (page < 0 || page >= p.pages) {
      if (lane == 0) report_status(p.status, AVSA_ERR_BAD_TABLE, kPrefixPage, s, t / p.page);
      continue;
    }
    const __nv_bfloat16* kr = static_cast<const __nv_bfloat16*>(p.k.ptr) + page * p.k.stride_b + h / p.G * p.k.stride_h + t % p.page * p.k.stride_n;
    const __nv_bfloat16* vr = static_cast<const __nv_bfloat16*>(p.v.ptr) + page * p.v.stride_b + h / p.G * p.v.stride_h + t % p.page * p.v.stride_n;
    float x = 0.f;
#pragma unroll
    for (int c = 0; c < C; c++) x += q[c] * __bfloat162float(kr[lane * C + c]);
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) x += __shfl_xor_sync(0xffffffffu, x, d);
    const float m2 = fmaxf(m, x);
    const float a = m2 == -INFINITY ? 1.f : exp2f(m - m2), e = m2 == -INFINITY ? 0.f : exp2f(x - m2);
    m = m2;
    l = l * a + e;
#pragma unroll
    for (int c = 0; c < C; c++) o[c] = o[c] * a + e * __bfloat162float(vr[lane * C + c]);
  }
  __nv_bfloat16* orow = p.o + b * p.q.stride_b + h * p.q.stride_h + i * p.q.stride_n;
#pragma unroll
  for (int c = 0; c < C; c++) orow[lane * C + c] = __float2bfloat16(l != 0.f ? o[c] / l : 0.f);
  if (lane == 0 && p.lse != nullptr) p.lse[r] = l != 0.f ? (m + log2f(l)) * 0.6931471805599453f : -INFINITY;
}

static bool rows_ok(avsa_bf16_4d t, int B, int H, int N) {
  if (N == 1) t.stride_n = 8;      // (an axis of one element has no stride to speak of)
  return tensor_ok(t, B, H);
}

}  // namespace avsa

using namespace avsa;

extern "C" size_t avsa_prefix_attn_workspace_bytes(int B, int H, int Hkv, int L, int d, int page, int width, int prefix_pages) {
  if (B <= 0 || H <= 0 || Hkv <= 0 || L <= 0 || d <= 0 || page <= 0 || width <= 0 || prefix_pages < 0) return 0;
  return kStatusBytes;
}

extern "C" int avsa_prefix_attn(int B, int H, int Hkv, int L, int d, int page, int pages, int seqs, int width, avsa_bf16_4d q,
                                avsa_bf16_4d k_pool, avsa_bf16_4d v_pool, const int32_t* table, const int32_t* length,
                                const int32_t* seq, int prefix_pages, unsigned flags, float softmax_scale, void* o_bf16, float* lse,
                                void* ws, size_t ws_bytes, void* stream) {
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
  if (ws == nullptr || ws_bytes < avsa_prefix_attn_workspace_bytes(B, H, Hkv, L, d, page, width, prefix_pages)) return AVSA_ERR_WORKSPACE;
  if (!ws_aligned(ws, kWsParts)) return AVSA_ERR_INVALID_ARG;
  if (!device_is_sm100()) return AVSA_ERR_UNSUPPORTED;
  const cudaStream_t st = as_stream(stream);
  const float scale = softmax_scale != 0.f ? softmax_scale : 1.0f / sqrtf(static_cast<float>(d));
  const PrefixParams p = {q, k_pool, v_pool, static_cast<__nv_bfloat16*>(o_bf16), lse, table, length, seq, static_cast<StatusRecord*>(ws), B, H, H / Hkv, L,
                          page, pages, seqs, width, flags & AVSA_CAUSAL ? 1 : 0, scale * 1.4426950408889634f};
  if (launch_pdl(clear_status_kernel, 1, 1, 0, st, p.status) != cudaSuccess) return AVSA_ERR_CUDA;
  const unsigned grid = static_cast<unsigned>((static_cast<long long>(B) * H * L + 7) / 8);
  if (launch_pdl(d == 128 ? prefix_rows_kernel<128> : prefix_rows_kernel<64>, grid, 256, 0, st, p) != cudaSuccess) return AVSA_ERR_CUDA;
  return cudaGetLastError() == cudaSuccess ? AVSA_OK : AVSA_ERR_CUDA;
}
