// The head in 8 bits: logits[t, v] = (sum over k of codes[t, k] * w_codes[v, k]) * scales[t] * w_scales[v], sums in 32-bit integers (exact), the
// scales in float32, one rounding to the output's type.
// Bound: for few tokens the weights, read once (one token, 128,256 x 4096: 93 us, 5.7 TB/s); for many the matrix rate (2048 tokens against the same: 910 to 1010 us on different boards, 2.1 to 2.4 POP/s, the
// 525 MB of logits written among it).
#include "simple_tiles.hpp"

namespace simple {
namespace head {

using namespace tiles;

constexpr int64_t MAX_K = 131071;  // 128 * 128 * K stays below 2^31

struct Args {
  Operand tokens, weights;
  int k_bytes, out_type;
  Plan plan;
  const float *scales, *w_scales;
  void* out;
  int64_t out_stride;
};

template <typename T> __device__ __forceinline__ void put4(T* to, int64_t n, const float (&v)[4]) {
  T x[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i] = down<T>(v[i]);
  if (n >= 4) __builtin_memcpy(to, x, sizeof(x));  // (any alignment)
  else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i < n) to[i] = x[i];
  }
}

template <class S, bool DIRECT> constexpr bool many = DIRECT && Cut<S>::CAN;  // (staged through registers as well, the products' own would spill)

template <class S, bool DIRECT, typename T>
__global__ __launch_bounds__(S::THREADS) void linear_int8_kernel(Args a) {
  __shared__ __align__(1024) unsigned char lds[S::LDS];
  planned<S, DIRECT, many<S, DIRECT>>(a.tokens, a.weights, a.k_bytes, a.plan, lds, [&](auto shape, auto& acc, int64_t p0, int64_t q0) {
    using R = decltype(shape);
    const int lane = opaque_lane(), wave = threadIdx.x >> 6;
    const int64_t p1 = p0 + wave % R::NWP * R::FP * 16 + (lane & 15), q1 = q0 + wave / R::NWP * R::FQ * 16 + (lane >> 4) * 4;
    const int64_t V = a.weights.rows;
    float ws[R::FQ][4];
#pragma unroll
    for (int i = 0; i < R::FQ; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) ws[i][e] = a.w_scales[min(q1 + i * 16 + e, V - 1)];
    float ts[R::FP];
#pragma unroll
    for (int j = 0; j < R::FP; ++j) ts[j] = a.scales[min(p1 + j * 16, a.tokens.rows - 1)];
#pragma unroll
    for (int i = 0; i < R::FQ; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) arrived_value(ws[i][e]);
#pragma unroll
    for (int j = 0; j < R::FP; ++j) arrived_value(ts[j]);
#pragma unroll
    for (int j = 0; j < R::FP; ++j) {
      const int64_t p = p1 + j * 16;
      const float s = ts[j];
      T* row = (T*)a.out + p * a.out_stride;
      if constexpr (sizeof(T) == 2 && R::FQ % 2 == 0) {
        const int g = lane >> 4;
        const int64_t q2 = q1 - g * 4 + 16 * (g / 2) + 8 * (g % 2);
#pragma unroll
        for (int i = 0; i < R::FQ; i += 2) {
          uint2 x[2];
#pragma unroll
          for (int h = 0; h < 2; ++h)
            x[h] = uint2{two_bf16((float)acc[i + h][j][0] * s * ws[i + h][0], (float)acc[i + h][j][1] * s * ws[i + h][1]),
                         two_bf16((float)acc[i + h][j][2] * s * ws[i + h][2], (float)acc[i + h][j][3] * s * ws[i + h][3])};
          eight_of(x[0], x[1]);
          if (p < a.tokens.rows) put8((uint16_t*)row + q2 + i * 16, V - (q2 + i * 16), uint4{x[0].x, x[0].y, x[1].x, x[1].y});
        }
      } else {
#pragma unroll
        for (int i = 0; i < R::FQ; ++i) {
          float v[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = (float)acc[i][j][e] * s * ws[i][e];
          if (p < a.tokens.rows) put4<T>(row + q1 + i * 16, V - (q1 + i * 16), v);
        }
      }
    }
  });
}

template <class S, bool DIRECT> void launch(Args a, hipStream_t st) {
  a.plan = plan<S, many<S, DIRECT>>(a.tokens.rows, a.weights.rows);
  const dim3 grid((unsigned)a.plan.grid), block(S::THREADS);
  if (a.out_type == SIMPLE_F32) hipLaunchKernelGGL((linear_int8_kernel<S, DIRECT, float>), grid, block, 0, st, a);
  else hipLaunchKernelGGL((linear_int8_kernel<S, DIRECT, uint16_t>), grid, block, 0, st, a);
}
template <bool DIRECT> void launch_for(const Args& a, hipStream_t st) {
  shaped<Int8>(tiles_for(a.tokens.rows, a.weights.rows), [&](auto shape) { launch<decltype(shape), DIRECT>(a, st); });
}

}  // namespace head
}  // namespace simple

using namespace simple::head;

extern "C" int64_t simple_linear_int8_workspace(int64_t T, int64_t V, int64_t K) {
  if (T < 0 || V <= 0 || K <= 0) return SIMPLE_EINVAL;
  return T <= FEW_TOKENS ? 0 : (T + (V < ALIGN_ROWS ? V : ALIGN_ROWS)) * aligned_stride(K);
}

extern "C" int simple_linear_int8(const int8_t* codes_dev, int64_t code_stride, const float* scales_dev, const int8_t* w_codes_dev,
                                  int64_t w_code_stride, const float* w_scales_dev, int64_t T, int64_t V, int64_t K, void* out_dev,
                                  int64_t out_stride, int out_dtype, void* workspace_dev, int64_t workspace_bytes, void* hip_stream) {
  if (T < 0 || V <= 0 || K <= 0 || code_stride < K || w_code_stride < K || out_stride < V || !good_type(out_dtype)) return SIMPLE_EINVAL;
  if (K > MAX_K || T > ((int64_t)1 << 24) || V > ((int64_t)1 << 28)) return SIMPLE_ECAPACITY;
  if (T == 0) return SIMPLE_OK;
  if (!codes_dev || !scales_dev || !w_codes_dev || !w_scales_dev || !out_dev) return SIMPLE_EINVAL;
  if (workspace_dev && ((uintptr_t)workspace_dev & 15u) != 0) return SIMPLE_EINVAL;
  if (workspace_dev && workspace_bytes < simple_linear_int8_workspace(T, V, K)) return SIMPLE_ECAPACITY;
  if (ceil_div(T, 16) * ceil_div(V, 64) > (int64_t)0x7FFFFFFF) return SIMPLE_ECAPACITY;
  const int64_t e = type_bytes(out_dtype);
  Args a{{(const unsigned char*)codes_dev, code_stride, T}, {(const unsigned char*)w_codes_dev, w_code_stride, V}, (int)K, out_dtype, Plan{}, scales_dev,
         w_scales_dev, out_dev, out_stride};
  hipStream_t st = (hipStream_t)hip_stream;
  const Operand weights = a.weights;
  const bool tokens_fit = direct(a.tokens, K), weights_fit = direct(weights, K);
  if (tokens_fit && weights_fit) {
    launch_for<true>(a, st);
  } else if (T <= FEW_TOKENS || !workspace_dev) {
    launch_for<false>(a, st);
  } else {  // copies with aligned rows, of the weights ALIGN_ROWS at a time
    unsigned char* ws = (unsigned char*)workspace_dev;
    const int64_t stride = aligned_stride(K);
    a.k_bytes = (int)stride;
    a.tokens = aligned_copy<1>(a.tokens, K, ws, st);
    for (int64_t v0 = 0; v0 < V; v0 += ALIGN_ROWS) {
      a.weights = aligned_copy<1>(Operand{weights.p + v0 * weights.stride, weights.stride, V - v0 < ALIGN_ROWS ? V - v0 : ALIGN_ROWS}, K, ws + T * stride, st);
      a.w_scales = w_scales_dev + v0;
      a.out = (unsigned char*)out_dev + v0 * e;
      launch_for<true>(a, st);
    }
  }
  return launched();
}
