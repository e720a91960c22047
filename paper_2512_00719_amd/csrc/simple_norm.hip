// Root-mean-square norm of rows: with the residual's addition ahead of it, its output in the rows' own type or in 8-bit codes with a scale
// a row; its gradient; and the codes alone (for a head's weights).
//
// All of them are bound by memory: a row is read once into registers, its sum (or largest magnitude) formed by the row's
// threads, and everything written from the registers.
#include <type_traits>

#include "simple_vocabdev.hpp"

namespace simple {
namespace norm {

using namespace vocab;

constexpr int WG = 256;             // threads of a workgroup, unless a row takes 1024
constexpr int64_t MAX_D = 32768;    // 1024 threads of 32 values
constexpr int64_t MAX_GRAD_WGS = 1024;  // workgroups of the gradient, each with one row of partial sums of the weight's gradient

enum { NORM = 0, NORM8 = 1, QUANT = 2 };

struct Args {
  const void *x, *residual, *weight;
  int64_t x_stride, residual_stride, h_stride, out_stride, T;
  int D;
  float eps;
  void *h, *out;
  float *rstd, *scales;
};

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}
__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = max(v, (uint32_t)__shfl_xor((int)v, o, 64));
  return v;
}

// Sum and maximum over the NT threads of a row.  With more than one wave through LDS: the caller has a barrier between two uses of `part`.
template <int NT> __device__ __forceinline__ void row_reduce(float& sum, uint32_t& top, float* part) {
  sum = wave_sum(sum);
  top = wave_max(top);
  if constexpr (NT > 64) {
    constexpr int NW = NT / 64;
    const int wave = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0) { part[wave] = sum; part[NW + wave] = __uint_as_float(top); }
    __syncthreads();
    sum = 0.f;
    top = 0u;
#pragma unroll
    for (int w = 0; w < NW; ++w) { sum += part[w]; top = max(top, __float_as_uint(part[NW + w])); }
  }
}

// NT threads a row, NV groups of VEC values a thread: a row is in registers between its one read and its writes, whatever is computed of it.  Bound:
// memory; 8192 bfloat16 rows of 4096 with a residual, 268 MB, 44 us (6.1 TB/s, part of it from the caches), 8 rows in 8 bits 5 us (latency).
template <typename T, int VEC, bool WHOLE, int NT, int NV, int OUT>
__global__ __launch_bounds__(NT > WG ? NT : WG) void rows_kernel(Args a) {
  constexpr int ROWS = NT > WG ? 1 : WG / NT;
  __shared__ float part[2 * (NT > 64 ? NT / 64 : 1)];
  const int t = threadIdx.x % NT;
  const int64_t row = (int64_t)blockIdx.x * ROWS + threadIdx.x / NT;
  if (row >= a.T) return;  // (a whole wave: rows of several waves have a workgroup of their own)
  const T* x = (const T*)a.x + row * a.x_stride;
  float h[NV][VEC], w[NV][VEC];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = (i * NT + t) * VEC;
    if (c < a.D) {
      load_some<T, VEC, WHOLE>(x, c, a.D, h[i]);
      if constexpr (OUT != QUANT) load_some<T, VEC, WHOLE>((const T*)a.weight, c, a.D, w[i]);
    }
  }
  if (OUT != QUANT && a.residual) {
    const T* r = (const T*)a.residual + row * a.residual_stride;
    float e[NV][VEC];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (i * NT + t) * VEC;
      if (c < a.D) load_some<T, VEC, WHOLE>(r, c, a.D, e[i]);
    }
#pragma unroll
    for (int i = 0; i < NV; ++i)  // the norm is of the stream as it is kept, so that its gradient finds the same values
#pragma unroll
      for (int j = 0; j < VEC; ++j) h[i][j] = up(down<T>(h[i][j] + e[i][j]));
  }
  float sum = 0.f;
  uint32_t top = 0u;  // magnitudes as their bits: in that order a NaN is above infinity, and infinity above every number
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = (i * NT + t) * VEC;
    if (c < a.D) {
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        if constexpr (OUT != QUANT) sum = fmaf(h[i][j], h[i][j], sum);
        if constexpr (OUT == NORM8) w[i][j] = h[i][j] * w[i][j];
        if constexpr (OUT == QUANT) w[i][j] = h[i][j];
        if constexpr (OUT != NORM) top = max(top, __float_as_uint(w[i][j]) & 0x7FFFFFFFu);
      }
    }
  }
  row_reduce<NT>(sum, top, part);
  const float s = OUT == QUANT ? 1.f : 1.f / sqrtf(sum / (float)a.D + a.eps);
  // (behind the reduction, whose barrier every thread of the row reaches after its loads: the stream may be written in place)
  if (OUT != QUANT && a.h) {
    T* ho = (T*)a.h + row * a.h_stride;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (i * NT + t) * VEC;
      if (c < a.D) store_some<T, VEC, WHOLE>(ho + c, a.D - c, h[i]);
    }
  }
  if (OUT != QUANT && a.rstd && t == 0) a.rstd[row] = s;
  if constexpr (OUT == NORM) {
    T* o = (T*)a.out + row * a.out_stride;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (i * NT + t) * VEC;
      if (c < a.D) {
        float y[VEC];
#pragma unroll
        for (int j = 0; j < VEC; ++j) y[j] = h[i][j] * s * w[i][j];
        store_some<T, VEC, WHOLE>(o + c, a.D - c, y);
      }
    }
  } else {
    const bool bad = top >= 0x7F800000u, none = top < 0x03800000u;  // 2^-120: 127 over it is a number
    const float m = __uint_as_float(top), r = (bad || none) ? 0.f : 127.f / m;
    if (t == 0) a.scales[row] = bad ? __uint_as_float(0x7FC00000u) : none ? 0.f : m * s / 127.f;
    int8_t* o = (int8_t*)a.out + row * a.out_stride;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (i * NT + t) * VEC;
      if (c < a.D) {
        int8_t q[VEC];
#pragma unroll
        for (int j = 0; j < VEC; ++j) q[j] = (bad || none) ? (int8_t)0 : (int8_t)(int)rintf(w[i][j] * r);
        put_some<int8_t, VEC, WHOLE>(o + c, a.D - c, q);
      }
    }
  }
}

struct GradArgs {
  const void *dy, *h, *weight, *dh;
  const float* rstd;
  int64_t dy_stride, h_stride, dh_stride, dx_stride, T;
  int D;
  void* dx;
  float* partial;  // [workgroups][D]
};

// A workgroup takes rows a grid apart, so that each of its threads adds up the same columns' weight gradient in registers over all of
// them; the workgroups' sums are joined by column_sums_kernel in their order.  Bound: memory; 8192 bfloat16 rows of 4096 with dh, 268 MB, 46 us, and 5 for
// joining 1024 workgroups' rows.  Rows of more than 8192 values hold more than a thread's 128 registers do and spill (1024 x 16,384 162 us, 0.8 TB/s in bfloat16 and 1.65 in float32; 1024 x 8192 32
// and 36).
template <typename T, int VEC, bool WHOLE, int NT, int NV>
__global__ __launch_bounds__(NT > WG ? NT : WG) void grad_kernel(GradArgs a) {
  constexpr int ROWS = NT > WG ? 1 : WG / NT;
  __shared__ float part[2][2 * (NT > 64 ? NT / 64 : 1)];
  __shared__ float joined[ROWS > 1 ? ROWS * NT * NV * VEC : 1];
  const int t = threadIdx.x % NT, sub = threadIdx.x / NT;
  float w[NV][VEC], dw[NV][VEC];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = (i * NT + t) * VEC;
    if (c < a.D) load_some<T, VEC, WHOLE>((const T*)a.weight, c, a.D, w[i]);
#pragma unroll
    for (int j = 0; j < VEC; ++j) dw[i][j] = 0.f;
  }
  int turn = 0;
  for (int64_t row = (int64_t)blockIdx.x * ROWS + sub; row < a.T; row += (int64_t)gridDim.x * ROWS) {
    const T *dy = (const T*)a.dy + row * a.dy_stride, *h = (const T*)a.h + row * a.h_stride;
    const float s = a.rstd[row];
    float g[NV][VEC], n[NV][VEC], e[NV][VEC];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (i * NT + t) * VEC;
      if (c < a.D) {
        load_some<T, VEC, WHOLE>(dy, c, a.D, g[i]);
        load_some<T, VEC, WHOLE>(h, c, a.D, n[i]);
        if (a.dh) load_some<T, VEC, WHOLE>((const T*)a.dh + row * a.dh_stride, c, a.D, e[i]);
      }
    }
    float sum = 0.f;
    uint32_t none = 0u;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (i * NT + t) * VEC;
      if (c < a.D) {
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
          n[i][j] *= s;
          dw[i][j] = fmaf(g[i][j], n[i][j], dw[i][j]);
          g[i][j] *= w[i][j];
          sum = fmaf(g[i][j], n[i][j], sum);
        }
      }
    }
    if constexpr (!WHOLE) {  // a row's last group overlaps its neighbour's: dh, where dx goes in its place, is here before anything is written
      if (a.dh) {
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
          for (int j = 0; j < VEC; ++j) asm volatile("" : "+v"(e[i][j]));
      }
    }
    row_reduce<NT>(sum, none, part[turn & 1]);  // (two areas in turn: one barrier a row)
    ++turn;
    const float m = sum / (float)a.D;
    T* dx = (T*)a.dx + row * a.dx_stride;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (i * NT + t) * VEC;
      if (c < a.D) {
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
          g[i][j] = s * (g[i][j] - n[i][j] * m);
          if (a.dh) g[i][j] += e[i][j];
        }
        store_some<T, VEC, WHOLE>(dx + c, a.D - c, g[i]);
      }
    }
  }
  float* out = a.partial + (int64_t)blockIdx.x * a.D;
  if constexpr (ROWS > 1) {  // the workgroup's rows at once: one row of sums for all of them
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int j = 0; j < VEC; ++j) joined[sub * (NT * NV * VEC) + (i * NT + t) * VEC + j] = dw[i][j];
    __syncthreads();
    for (int c = threadIdx.x; c < a.D; c += WG) {
      float v = joined[c];
#pragma unroll
      for (int r = 1; r < ROWS; ++r) v += joined[r * (NT * NV * VEC) + c];
      out[c] = v;
    }
  } else {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (i * NT + t) * VEC;
      if (c < a.D) store_some<float, VEC, WHOLE>(out + c, a.D - c, dw[i]);
    }
  }
}

// out[c] = sum over the P rows of `rows`, in an order that depends on P alone.  P = 0 gives zeros.
constexpr int CS_COLS = 32, CS_GROUPS = 32;
__global__ __launch_bounds__(CS_COLS * CS_GROUPS) void column_sums_kernel(const float* rows, int P, int D, float* out) {
  __shared__ float part[CS_GROUPS][CS_COLS + 1];
  const int lane = threadIdx.x % CS_COLS, grp = threadIdx.x / CS_COLS;
  const int64_t c = (int64_t)blockIdx.x * CS_COLS + lane;
  float v = 0.f;
  if (c < D) {
#pragma unroll 8
    for (int p = grp; p < P; p += CS_GROUPS) v += rows[(int64_t)p * D + c];
  }
  part[grp][lane] = v;
  __syncthreads();
  if (grp == 0 && c < D) {
    v = part[0][lane];
#pragma unroll
    for (int g = 1; g < CS_GROUPS; ++g) v += part[g][lane];
    out[c] = v;
  }
}

// A row's threads: a wave up to 1024 values, then 256 threads up to 8192, then 1024; values a thread: 8, 16 or 32.
template <typename F> void shaped(int64_t D, F&& f) {
  using std::integral_constant;
  if (D <= 512) f(integral_constant<int, 64>{}, integral_constant<int, 8>{});
  else if (D <= 1024) f(integral_constant<int, 64>{}, integral_constant<int, 16>{});
  else if (D <= 2048) f(integral_constant<int, 256>{}, integral_constant<int, 8>{});
  else if (D <= 4096) f(integral_constant<int, 256>{}, integral_constant<int, 16>{});
  else if (D <= 8192) f(integral_constant<int, 256>{}, integral_constant<int, 32>{});
  else f(integral_constant<int, 1024>{}, integral_constant<int, 32>{});
}
// 16 bytes a load.  Rows that are not aligned, or end inside one: bfloat16 takes unaligned loads (8192 rows of 2047 values: norm 32 us and its gradient 38, 40 and 58
// by single elements; aligned rows of 2048 24 and 28), float32 single elements (46 and 56 us, 57 and 64 by unaligned loads; aligned 42 and 52).
template <typename F> void typed(int dtype, bool whole, F&& f) {
  using std::bool_constant;
  using std::integral_constant;
  if (dtype == SIMPLE_F32) {
    if (whole) f((float*)nullptr, integral_constant<int, 4>{}, bool_constant<true>{});
    else f((float*)nullptr, integral_constant<int, 1>{}, bool_constant<true>{});
  } else {
    if (whole) f((uint16_t*)nullptr, integral_constant<int, 8>{}, bool_constant<true>{});
    else f((uint16_t*)nullptr, integral_constant<int, 8>{}, bool_constant<false>{});
  }
}

bool bad_rows(const void* p, int64_t stride, int64_t D) { return p == nullptr || stride < D; }

template <int OUT> int launch_rows(Args a, int dtype, hipStream_t st) {
  const int64_t e = type_bytes(dtype);
  const int64_t vec = 16 / e;
  const bool whole = a.D % vec == 0 && rows_aligned(a.x, a.x_stride, e, 16) && rows_aligned(a.residual, a.residual_stride, e, 16) &&
                     rows_aligned(a.weight, 0, e, 16) && rows_aligned(a.h, a.h_stride, e, 16) &&
                     (OUT == NORM ? rows_aligned(a.out, a.out_stride, e, 16) : rows_aligned(a.out, a.out_stride, 1, vec));
  typed(dtype, whole, [&](auto* type, auto vec, auto aligned) {
    shaped(a.D, [&](auto nt, auto ept) {
      using T = std::remove_pointer_t<decltype(type)>;
      constexpr int NT = decltype(nt)::value, VEC = decltype(vec)::value, NV = decltype(ept)::value / VEC;
      constexpr int ROWS = NT > WG ? 1 : WG / NT;
      constexpr int64_t E = sizeof(T), OE = OUT == NORM ? E : 1;
      auto on = [](auto* p, int64_t bytes) { return p ? (decltype(p))((uintptr_t)p + (uintptr_t)bytes) : p; };
      for (int64_t left = a.T; left > 0; left -= a.T) {
        a.T = left < ROWS * LAUNCH_WGS ? left : ROWS * LAUNCH_WGS;
        hipLaunchKernelGGL((rows_kernel<T, VEC, decltype(aligned)::value, NT, NV, OUT>), dim3((unsigned)ceil_div(a.T, ROWS)), dim3(NT > WG ? NT : WG), 0, st, a);
        a.x = on(a.x, a.T * a.x_stride * E);
        a.residual = on(a.residual, a.T * a.residual_stride * E);
        a.h = on(a.h, a.T * a.h_stride * E);
        a.out = on(a.out, a.T * a.out_stride * OE);
        a.rstd = on(a.rstd, a.T * (int64_t)sizeof(float));
        a.scales = on(a.scales, a.T * (int64_t)sizeof(float));
      }
    });
  });
  return launched();
}

int64_t grad_workgroups(int64_t T, int64_t D) {
  const int64_t rows = D <= 1024 ? WG / 64 : 1, n = ceil_div(T, rows);
  return n < MAX_GRAD_WGS ? n : MAX_GRAD_WGS;
}

}  // namespace norm
}  // namespace simple

using namespace simple::norm;

namespace {
int check_rows(int64_t T, int64_t D, int dtype) {
  if (T < 0 || D <= 0 || !good_type(dtype)) return SIMPLE_EINVAL;
  if (D > MAX_D || T > (int64_t)0x7FFFFFFF) return SIMPLE_ECAPACITY;
  return SIMPLE_OK;
}
int check_norm(const void* x, int64_t x_stride, const void* residual, int64_t residual_stride, const void* weight, int64_t D, float eps,
               const void* h, int64_t h_stride) {
  if (bad_rows(x, x_stride, D) || !weight || !(eps >= 0.f)) return SIMPLE_EINVAL;
  if (residual && (residual_stride < D || !h)) return SIMPLE_EINVAL;
  if (h && h_stride < D) return SIMPLE_EINVAL;
  return SIMPLE_OK;
}
}  // namespace

extern "C" int simple_rms_norm(const void* x_dev, int64_t x_stride, const void* residual_dev, int64_t residual_stride, const void* weight_dev,
                               int64_t T, int64_t D, int dtype, float eps, void* h_out_dev, int64_t h_stride, void* out_dev,
                               int64_t out_stride, float* rstd_dev, void* hip_stream) {
  int rc = check_rows(T, D, dtype);
  if (rc != SIMPLE_OK || T == 0) return rc;
  rc = check_norm(x_dev, x_stride, residual_dev, residual_stride, weight_dev, D, eps, h_out_dev, h_stride);
  if (rc != SIMPLE_OK || bad_rows(out_dev, out_stride, D)) return SIMPLE_EINVAL;
  const Args a{x_dev, residual_dev, weight_dev, x_stride, residual_stride, h_stride, out_stride, T, (int)D, eps, h_out_dev, out_dev, rstd_dev, nullptr};
  return launch_rows<NORM>(a, dtype, (hipStream_t)hip_stream);
}

extern "C" int simple_rms_norm_int8(const void* x_dev, int64_t x_stride, const void* residual_dev, int64_t residual_stride,
                                    const void* weight_dev, int64_t T, int64_t D, int dtype, float eps, void* h_out_dev, int64_t h_stride,
                                    int8_t* codes_dev, int64_t code_stride, float* scales_dev, void* hip_stream) {
  int rc = check_rows(T, D, dtype);
  if (rc != SIMPLE_OK || T == 0) return rc;
  rc = check_norm(x_dev, x_stride, residual_dev, residual_stride, weight_dev, D, eps, h_out_dev, h_stride);
  if (rc != SIMPLE_OK || bad_rows(codes_dev, code_stride, D) || !scales_dev) return SIMPLE_EINVAL;
  const Args a{x_dev, residual_dev, weight_dev, x_stride, residual_stride, h_stride, code_stride, T, (int)D, eps, h_out_dev, codes_dev, nullptr, scales_dev};
  return launch_rows<NORM8>(a, dtype, (hipStream_t)hip_stream);
}

extern "C" int simple_quantize_rows(const void* x_dev, int64_t x_stride, int64_t T, int64_t D, int dtype, int8_t* codes_dev,
                                    int64_t code_stride, float* scales_dev, void* hip_stream) {
  const int rc = check_rows(T, D, dtype);
  if (rc != SIMPLE_OK || T == 0) return rc;
  if (bad_rows(x_dev, x_stride, D) || bad_rows(codes_dev, code_stride, D) || !scales_dev) return SIMPLE_EINVAL;
  const Args a{x_dev, nullptr, nullptr, x_stride, 0, 0, code_stride, T, (int)D, 0.f, nullptr, codes_dev, nullptr, scales_dev};
  return launch_rows<QUANT>(a, dtype, (hipStream_t)hip_stream);
}

extern "C" int64_t simple_rms_norm_grad_workspace(int64_t T, int64_t D) {
  if (T < 0 || D <= 0) return SIMPLE_EINVAL;
  return grad_workgroups(T, D) * D * (int64_t)sizeof(float);
}

extern "C" int simple_rms_norm_grad(const void* dy_dev, int64_t dy_stride, const void* h_dev, int64_t h_stride, const void* weight_dev,
                                    const float* rstd_dev, const void* dh_dev, int64_t dh_stride, int64_t T, int64_t D, int dtype,
                                    void* dx_dev, int64_t dx_stride, float* dweight_dev, void* workspace_dev, int64_t workspace_bytes,
                                    void* hip_stream) {
  const int rc = check_rows(T, D, dtype);
  if (rc != SIMPLE_OK) return rc;
  if (!dweight_dev) return SIMPLE_EINVAL;
  hipStream_t st = (hipStream_t)hip_stream;
  if (T > 0) {
    if (bad_rows(dy_dev, dy_stride, D) || bad_rows(h_dev, h_stride, D) || bad_rows(dx_dev, dx_stride, D) || !weight_dev || !rstd_dev) return SIMPLE_EINVAL;
    if (dh_dev && dh_stride < D) return SIMPLE_EINVAL;
    if (!workspace_dev || ((uintptr_t)workspace_dev & 15u) != 0) return SIMPLE_EINVAL;
    if (workspace_bytes < simple_rms_norm_grad_workspace(T, D)) return SIMPLE_ECAPACITY;
    const GradArgs a{dy_dev, h_dev, weight_dev, dh_dev, rstd_dev, dy_stride, h_stride, dh_stride, dx_stride, T, (int)D, dx_dev, (float*)workspace_dev};
    const int64_t e = type_bytes(dtype);
    const bool whole = D % (16 / e) == 0 && rows_aligned(dy_dev, dy_stride, e, 16) && rows_aligned(h_dev, h_stride, e, 16) &&
                       rows_aligned(weight_dev, 0, e, 16) && rows_aligned(dh_dev, dh_stride, e, 16) && rows_aligned(dx_dev, dx_stride, e, 16);
    typed(dtype, whole, [&](auto* type, auto vec, auto aligned) {
      shaped(D, [&](auto nt, auto ept) {
        using E = std::remove_pointer_t<decltype(type)>;
        constexpr int NT = decltype(nt)::value, VEC = decltype(vec)::value, NV = decltype(ept)::value / VEC;
        hipLaunchKernelGGL((grad_kernel<E, VEC, decltype(aligned)::value, NT, NV>), dim3((unsigned)grad_workgroups(T, D)), dim3(NT > WG ? NT : WG), 0, st, a);
      });
    });
  }
  hipLaunchKernelGGL(column_sums_kernel, dim3((unsigned)ceil_div(D, CS_COLS)), dim3(CS_COLS * CS_GROUPS), 0, st, (const float*)workspace_dev,
                     T > 0 ? (int)grad_workgroups(T, D) : 0, (int)D, dweight_dev);
  return launched();
}
