// Rotary positions with several axes.
//
//   (y_a, y_b) = (x_a cos t - x_b sin t, x_a sin t + x_b cos t),  t = 2 pi pos[axis of the pair] freq[pair],  for channel pairs (2i, 2i+1) or (i, i + d/2)
//
// Bound by HBM: 4 bytes a value (32760 tokens of 24 + 24 heads of 128 channels, 805 MB: 120 us, 6.7 TB/s).  A thread has 16 bytes of a head (of both halves, where they are the pairs), works out
// their sines and cosines once, and turns those channels of kRopeHeads heads, all of whose loads are under way together; queries and keys are one list of heads, so a
// layer's two tensors are one launch.  Neighbouring threads have neighbouring channels, then the next heads of the same token, so what a CTA touches is
// contiguous however the caller keeps heads and tokens.  A thread's heads are of one tensor and a step apart: with an address worked out for each of them, in the tensor that
// it belonged to, three quarters of the issue slots were taken and the call took 148 us.  CTAs of 128 threads and 64 registers (131 us then; of 256 threads 134 to 143) and
// accesses that do not stay in the caches (161 without).
// An angle is a number of turns: in fp64, because a position of 2^20 times a frequency in fp32 is off by 2^-4 of a radian; its fraction then goes to fp32 (2^-25 of a turn).
#include "avsa_common.cuh"
#include "sm100_ptx.cuh"

namespace avsa {

constexpr int kRopeThreads = 128;
constexpr int kRopeHeads = 8;       // heads of a thread, at most
constexpr int kRopePlaces = 8;      // CTAs of an SM

struct RopeArgs {
  avsa_bf16_4d q, k, q_out, k_out;
  const int32_t* pos;
  int64_t pos_stride;      // of batch entries
  const double* freq;
  int H, Hk, N, axes;
  int end[AVSA_ROPE_AXES];      // first pair behind each axis
  int per, q_slices, slices;    // heads of a thread, of q or of k; threads that share a token's heads of q, of both
  long long items;              // (batch entry, token, slice)
  float sign;
};

__device__ __forceinline__ void turn(uint32_t& x, float c, float s) {
  const float a = __uint_as_float(x << 16), b = __uint_as_float(x & 0xffff0000u);
  x = pack_bf16x2(a * c - b * s, a * s + b * c);
}
__device__ __forceinline__ void turn_halves(uint32_t& x, uint32_t& y, const float* c, const float* s) {
  const float a0 = __uint_as_float(x << 16), a1 = __uint_as_float(x & 0xffff0000u), b0 = __uint_as_float(y << 16), b1 = __uint_as_float(y & 0xffff0000u);
  x = pack_bf16x2(a0 * c[0] - b0 * s[0], a1 * c[1] - b1 * s[1]);
  y = pack_bf16x2(a0 * s[0] + b0 * c[0], a1 * s[1] + b1 * c[1]);
}

template <int D, bool HALVES>
__global__ void __launch_bounds__(kRopeThreads, kRopePlaces) rope_kernel(const __grid_constant__ RopeArgs a) {
  pdl_wait();
  pdl_launch();
  constexpr int V = HALVES ? D / 16 : D / 8, P = HALVES ? 8 : 4, U = HALVES ? kRopeHeads / 2 : kRopeHeads;      // threads of a head, their pairs; loads under way
  const long long at = static_cast<long long>(blockIdx.x) * (kRopeThreads / V) + threadIdx.x / V;
  const int v = threadIdx.x % V;
  if (at >= a.items) return;
  const int bn = static_cast<int>(at / a.slices), slice = static_cast<int>(at - static_cast<long long>(bn) * a.slices);
  const int b = bn / a.N, n = bn - b * a.N;
  const int32_t* const pos = a.pos + b * a.pos_stride + static_cast<int64_t>(n) * a.axes;
  float c[P], s[P];
#pragma unroll
  for (int i = 0; i < P; i++) {
    const int pair = v * P + i;
    int axis = 0;
#pragma unroll
    for (int x = 0; x + 1 < AVSA_ROPE_AXES; x++) axis += pair >= a.end[x];
    double turns = pos[axis] * a.freq[pair];
    turns -= rint(turns);
    sincospif(2.f * static_cast<float>(turns), &s[i], &c[i]);
    s[i] *= a.sign;
  }
  const bool of_q = slice < a.q_slices;
  const avsa_bf16_4d &in = of_q ? a.q : a.k, &out = of_q ? a.q_out : a.k_out;
  const int h0 = (of_q ? slice : slice - a.q_slices) * a.per, h1 = min(of_q ? a.H : a.Hk, h0 + a.per);
  const __nv_bfloat16* from = static_cast<const __nv_bfloat16*>(in.ptr) + b * in.stride_b + h0 * in.stride_h + n * in.stride_n + 8 * v;
  __nv_bfloat16* to = static_cast<__nv_bfloat16*>(const_cast<void*>(out.ptr)) + b * out.stride_b + h0 * out.stride_h + n * out.stride_n + 8 * v;
  const int64_t in_step = in.stride_h, out_step = out.stride_h;
  for (int h = h0; h < h1; h += U) {
    uint4 x[U], y[U];
#pragma unroll
    for (int u = 0; u < U; u++) {
      if (h + u < h1) {
        x[u] = __ldcs(reinterpret_cast<const uint4*>(from));
        if (HALVES) y[u] = __ldcs(reinterpret_cast<const uint4*>(from + D / 2));
      }
      from += in_step;
    }
#pragma unroll
    for (int u = 0; u < U; u++) {
      if (h + u < h1) {
        if constexpr (HALVES) {
          turn_halves(x[u].x, y[u].x, c, s);
          turn_halves(x[u].y, y[u].y, c + 2, s + 2);
          turn_halves(x[u].z, y[u].z, c + 4, s + 4);
          turn_halves(x[u].w, y[u].w, c + 6, s + 6);
          __stcs(reinterpret_cast<uint4*>(to + D / 2), y[u]);
        } else {
          turn(x[u].x, c[0], s[0]);
          turn(x[u].y, c[1], s[1]);
          turn(x[u].z, c[2], s[2]);
          turn(x[u].w, c[3], s[3]);
        }
        __stcs(reinterpret_cast<uint4*>(to), x[u]);
      }
      to += out_step;
    }
  }
}

static bool rope_view_ok(avsa_bf16_4d t, int B, int H, int N) {
  if (N == 1) t.stride_n = 8;      // (an axis of one element has no stride to speak of)
  return tensor_ok(t, B, H);
}
// An output may be its input, and then has to have its strides.
static bool rope_pair_ok(const avsa_bf16_4d& x, const avsa_bf16_4d& y, int B, int H, int N) {
  if (!rope_view_ok(x, B, H, N) || !rope_view_ok(y, B, H, N)) return false;
  return x.ptr != y.ptr || ((B == 1 || x.stride_b == y.stride_b) && (H == 1 || x.stride_h == y.stride_h) && (N == 1 || x.stride_n == y.stride_n));
}

}  // namespace avsa

using namespace avsa;

extern "C" int avsa_rope(int B, int H, int Hk, int N, int d, avsa_bf16_4d q, avsa_bf16_4d k, avsa_bf16_4d q_out, avsa_bf16_4d k_out, const int32_t* pos,
                         int64_t pos_stride_b, int axes, const int* sections, const double* freq, unsigned flags, void* stream) {
  if (B < 0 || H < 0 || Hk < 0 || N < 0 || axes < 1 || sections == nullptr || (flags & ~(AVSA_ROPE_HALVES | AVSA_ROPE_INVERSE)) != 0) return AVSA_ERR_INVALID_ARG;
  if ((d != 64 && d != 128) || axes > AVSA_ROPE_AXES || B > 65535 || H > 65535 || Hk > 65535) return AVSA_ERR_UNSUPPORTED;
  RopeArgs a = {};
  long long pairs = 0;
  for (int i = 0; i < axes; i++) {
    if (sections[i] < 0) return AVSA_ERR_INVALID_ARG;
    pairs += sections[i];
    if (pairs > d / 2) return AVSA_ERR_INVALID_ARG;
    a.end[i] = static_cast<int>(pairs);
  }
  if (pairs != d / 2) return AVSA_ERR_INVALID_ARG;
  for (int i = axes; i < AVSA_ROPE_AXES; i++) a.end[i] = d / 2;
  if (pos_stride_b < 0) return AVSA_ERR_INVALID_ARG;
  if (static_cast<long long>(B) * N > 0x7fffffffll) return AVSA_ERR_UNSUPPORTED;
  if (B == 0 || N == 0 || H + Hk == 0) return AVSA_OK;
  if (pos == nullptr || !aligned4(pos) || freq == nullptr || (reinterpret_cast<uintptr_t>(freq) & 7u) != 0) return AVSA_ERR_INVALID_ARG;
  if (H > 0 && !rope_pair_ok(q, q_out, B, H, N)) return AVSA_ERR_INVALID_ARG;
  if (Hk > 0 && !rope_pair_ok(k, k_out, B, Hk, N)) return AVSA_ERR_INVALID_ARG;
  if (!device_is_sm100()) return AVSA_ERR_UNSUPPORTED;
  a.q = q;
  a.k = k;
  a.q_out = q_out;
  a.k_out = k_out;
  a.pos = pos;
  a.pos_stride = pos_stride_b;
  a.freq = freq;
  a.H = H;
  a.Hk = Hk;
  a.N = N;
  a.axes = axes;
  a.sign = flags & AVSA_ROPE_INVERSE ? -1.f : 1.f;
  const bool halves = (flags & AVSA_ROPE_HALVES) != 0;
  const int V = halves ? d / 16 : d / 8, per_cta = kRopeThreads / V;
  // Few tokens: fewer heads to a thread, until every SM has a CTA.
  const long long tokens = static_cast<long long>(B) * N;
  const int sms = persistent_grid(1 << 30);
  auto slices = [&](int heads) { return (heads + a.per - 1) / a.per; };
  a.per = kRopeHeads;
  while (a.per > 1 && tokens * (slices(H) + slices(Hk)) < static_cast<long long>(sms) * per_cta) a.per /= 2;
  a.q_slices = slices(H);
  a.slices = a.q_slices + slices(Hk);
  a.items = tokens * a.slices;
  const long long ctas = (a.items + per_cta - 1) / per_cta;
  if (ctas > 0x7fffffffll) return AVSA_ERR_UNSUPPORTED;
  auto kernel = d == 128 ? (halves ? rope_kernel<128, true> : rope_kernel<128, false>) : (halves ? rope_kernel<64, true> : rope_kernel<64, false>);
  if (launch_pdl(kernel, static_cast<unsigned>(ctas), kRopeThreads, 0, as_stream(stream), a) != cudaSuccess) return AVSA_ERR_CUDA;
  return cudaGetLastError() == cudaSuccess ? AVSA_OK : AVSA_ERR_CUDA;
}
