// Softmax cross entropy of a head's logits z = c H W^T over a large vocabulary, without the [T, V] matrix, and its gradient.
//
// Forward: a workgroup forms a tile of logits in registers (simple_tiles.hpp), reduces it to a maximum and a sum of
// exponentials a token, and passes these on; a second kernel joins the tiles' pairs:  M = max m, S = sum s exp(m - M), lse = M + log S.
// The tile that holds a token's target also stores that logit.  Bound: the matrix rate, or for few tokens one read of the weights.
//
// Gradient: G = c dl (exp(z - lse) - [v = y]), dH = G W, dW = G^T H.  The vocabulary is taken in pieces; of a piece the logits are formed again (2 T V D more
// operations; keeping them would take T V floats), turned into G in the registers, and G is kept for the two products, in both orders because the products want
// k along the rows.  G is kept in 16 bits, and 16-bit floats of 11 bits it is: bfloat16's 8 cost the gradients twice the error of
// their own rounding.  What their range lacks is made up for by powers of two, which round nothing: a token's row
// (exp(z - lse) - [v = y]) has its largest magnitude, 1 - p_y, brought to 2^13 .. 2^14, so that a probability 2^-28 of it still has
// its 11 bits (at 1 those of rare tokens, 1e-6 and below, would have had fewer than bfloat16's); the factor c dl goes with the token's states into the
// product for dW, and behind the sum in dH; states and weights are brought below 2^14 by their largest magnitude.  Weights are then
// exact (8 bits within 28 binades of the largest), G and the states (the factor is no power of two) rounded once, to 11 bits; what is smaller than 2^-28 of its
// row's largest, or of all tokens' states', loses bits, and below 2^-39 is zero.  dH is summed over the pieces in float32.
// Tokens whose target is outside the vocabulary or whose dl is 0 take no part: their states are read as zeros where sums over tokens are
// formed, so that a NaN in them stays with them.
#include <algorithm>
#include <type_traits>

#include "simple_tiles.hpp"

namespace simple {
namespace xent {

using namespace tiles;

constexpr float LOG2E = 1.44269504088896340736f;
__device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(x * LOG2E); }

struct Pair { float m, s; };
__device__ __forceinline__ Pair join(Pair a, Pair b) {
  const float m = fmaxf(a.m, b.m), base = m == -INFINITY ? 0.f : m;  // (nothing in either: exp(-inf) twice)
  return Pair{m, a.s * exp_of(a.m - base) + b.s * exp_of(b.m - base)};
}

struct Args {
  Operand hidden, weight;  // of the weights: the piece's rows
  int k_bytes;
  Plan plan;
  float scale;
  const int32_t* targets;
  int64_t V, v0;           // whole vocabulary, the piece's first row
  // forward
  Pair* pairs;             // [tiles of the piece][T]
  float* at_target;        // [T]
  // gradient
  const struct Token* tokens;
  uint16_t *g, *gt;        // [T][g_stride], [rows of the piece][gt_stride]; either may be null
  int64_t g_stride, gt_stride;
  const float *lse, *dloss;  // of few tokens, who have no Token
  int64_t g_plane, gt_plane;
};

template <class S> constexpr int stats_room = S::BP * S::NWQ * (int)sizeof(Pair);  // (a cut tile's parts need a half of it)
template <class S>
__device__ __forceinline__ void stats_of(const Args& a, typename S::Acc (&acc)[S::FQ][S::FP], int64_t p0, int64_t q0, unsigned char* room) {
  const int64_t T = a.hidden.rows;
  const int lane = opaque_lane(), wave = threadIdx.x >> 6, wp = wave % S::NWP, wq = wave / S::NWP;
  const int64_t q1 = q0 + wq * S::FQ * 16 + (lane >> 4) * 4;
  const int left = (int)min((int64_t)S::BQ, a.weight.rows - q1);  // the lane's columns that exist
  if (q0 + S::BQ > a.weight.rows) {
#pragma unroll
    for (int i = 0; i < S::FQ; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (i * 16 + e >= left) {
#pragma unroll
          for (int j = 0; j < S::FP; ++j) acc[i][j][e] = -INFINITY;  // (the scale is positive)
        }
  }
  Pair(*part)[S::BP] = reinterpret_cast<Pair(*)[S::BP]>(room);  // (a tile has a barrier at least ahead of the next one's use)
  const float scale2 = a.scale * LOG2E;
#pragma unroll
  for (int j = 0; j < S::FP; ++j) {
    const int pl = (wp * S::FP + j) * 16 + (lane & 15);
    const int64_t p = p0 + pl;
    const int64_t target = p < T ? (int64_t)a.targets[p] - a.v0 - q1 : -1;
    if (target >= 0 && target < S::FQ * 16 && target < left) {  // (few tiles hold a token's target)
#pragma unroll
      for (int i = 0; i < S::FQ; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (target == i * 16 + e) a.at_target[p] = acc[i][j][e] * a.scale;
    }
    float m = -INFINITY;
#pragma unroll
    for (int i = 0; i < S::FQ; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) m = fmaxf(m, acc[i][j][e]);
    m = fmaxf(m, __shfl_xor(m, 16, 64));
    m = fmaxf(m, __shfl_xor(m, 32, 64));
    const float base = m == -INFINITY ? 0.f : m * scale2;
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < S::FQ; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) s += __builtin_amdgcn_exp2f(fmaf(acc[i][j][e], scale2, -base));
    s += __shfl_xor(s, 16, 64);
    s += __shfl_xor(s, 32, 64);
    if (lane < 16) part[wq][pl] = Pair{m * a.scale, s};
  }
  __syncthreads();
  for (int t = threadIdx.x; t < S::BP; t += S::THREADS) {
    if (p0 + t >= T) break;
    Pair v = part[0][t];
#pragma unroll
    for (int w = 1; w < S::NWQ; ++w) v = join(v, part[w][t]);
    a.pairs[q0 / S::BQ * T + p0 + t] = v;
  }
}
// 8192 tokens against 128,256 x 4096 6.05 to 6.4 ms (1.34 to 1.42 PFLOP/s, by the board); 16 tokens 169 us (1.05 GB of weights, 6.2 TB/s).
template <class S, bool DIRECT>
__global__ __launch_bounds__(S::THREADS) void stats_kernel(Args a) {
  __shared__ __align__(1024) unsigned char lds[S::LDS + stats_room<S>];
  planned<S, DIRECT, false>(a.hidden, a.weight, a.k_bytes, a.plan, lds,
                     [&](auto shape, auto& acc, int64_t p0, int64_t q0) { stats_of<decltype(shape)>(a, acc, p0, q0, lds + S::LDS); });
}

// The tiles' pairs of FIN_T tokens a workgroup, by groups of tiles, FIN_AHEAD pairs in flight a thread: latency.  Up to FEW_FIN tokens by twos, or one
// workgroup reads them all (a call of 1 token against 154,187 x 68 18 us, 24 by 16; of 40 against 260,000 x 256 36 and 38; of 128 against 128,256 x 64 20 and 19).
constexpr int FIN_THREADS = 1024, FIN_AHEAD = 8;
constexpr int64_t FEW_FIN = 64;
template <int FIN_T>
__global__ __launch_bounds__(FIN_THREADS) void finish_kernel(const Pair* pairs, int nq, int64_t T, int64_t V, const int32_t* targets,
                                                                    const float* at_target, float* loss, float* lse) {
  constexpr int FIN_GROUPS = FIN_THREADS / FIN_T;
  __shared__ Pair part[FIN_GROUPS][FIN_T];
  const int lane = threadIdx.x % FIN_T, grp = threadIdx.x / FIN_T;
  const int64_t t = (int64_t)blockIdx.x * FIN_T + lane;
  Pair v{-INFINITY, 0.f};
  if (t < T) {
    for (int q0 = grp; q0 < nq; q0 += FIN_GROUPS * FIN_AHEAD) {
      Pair x[FIN_AHEAD];
#pragma unroll
      for (int u = 0; u < FIN_AHEAD; ++u) {
        const int q = q0 + u * FIN_GROUPS;
        x[u] = q < nq ? pairs[(int64_t)q * T + t] : Pair{-INFINITY, 0.f};
      }
#pragma unroll
      for (int n = FIN_AHEAD / 2; n > 0; n /= 2)
#pragma unroll
        for (int u = 0; u < n; ++u) x[u] = join(x[u], x[u + n]);
      v = join(v, x[0]);
    }
  }
  part[grp][lane] = v;
  for (int n = FIN_GROUPS / 2; n > 0; n /= 2) {
    __syncthreads();
    if (grp < n) part[grp][lane] = v = join(v, part[grp + n][lane]);
  }
  if (grp == 0 && t < T) {
    const float l = v.m + logf(v.s);  // (a NaN logit is in s)
    const int32_t y = targets[t];
    lse[t] = l;
    loss[t] = y >= 0 && y < V ? l - at_target[t] : 0.f;
  }
}

__device__ __forceinline__ bool takes_part(int32_t target, float dloss, int64_t V) { return target >= 0 && target < V && dloss != 0.f; }

// What the gradient knows of a token: its target (-1: it takes no part), lse, the power of two on its row of G, and what the row still lacks of
// the gradient, c dl over that power.
struct Token { int32_t y; float lse, up, rest; };

// Powers of two that bring values whose largest magnitude has the bits `top` below 2^14, and back.
__device__ __forceinline__ float to_range(uint32_t top) {
  const int e = (int)(top >> 23);  // (sign 0)
  if (e == 0 || e == 255) return 1.f;
  return __uint_as_float((uint32_t)min(max(267 - e, 14), 240) << 23);
}
__device__ __forceinline__ float from_range(uint32_t top) { return 1.f / to_range(top); }
enum { TOP_STATES = 0, TOP_WEIGHTS = 1, TOPS = 2 };

// The larger magnitude, a NaN above all.
__device__ __forceinline__ float larger(float a, float b) { return __uint_as_float(max(__float_as_uint(a) & 0x7FFFFFFFu, __float_as_uint(b) & 0x7FFFFFFFu)); }

struct PrepareArgs {
  const uint16_t *hidden, *weight;
  int64_t hidden_stride, weight_stride, T, V, D;
  const int32_t* targets;
  const float *lse, *dloss;
  float scale;
  Token* tokens;
  float* partial;  // a workgroup's largest magnitude each
  int token_wgs;
};
// The largest magnitude of a workgroup of NW waves.
template <int NW> __device__ __forceinline__ float top_of(float v, float* part) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = larger(v, __shfl_xor(v, o, 64));
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
  __syncthreads();
  v = part[0];
#pragma unroll
  for (int w = 1; w < NW; ++w) v = larger(v, part[w]);
  return v;
}
// The first workgroups: a wave a token, its logit at the target once more (for the power of two alone, so its order of summation does not matter)
// and its largest state.  The rest: the weights' largest magnitude, rows in turn.
template <int VEC>
__global__ __launch_bounds__(256) void prepare_kernel(PrepareArgs a) {
  __shared__ float part[4];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  float most = 0.f;
  if ((int)blockIdx.x < a.token_wgs) {
    const int64_t t = (int64_t)blockIdx.x * 4 + wave;
    const int32_t y = t < a.T ? a.targets[t] : -1;
    const float dl = t < a.T ? a.dloss[t] : 0.f;
    const bool on = takes_part(y, dl, a.V);
    Token k{-1, 0.f, 1.f, 0.f};
    if (on) {
      const uint16_t *h = a.hidden + t * a.hidden_stride, *w = a.weight + y * a.weight_stride;
      float dot = 0.f, sizes = 0.f, top = 0.f;
      for (int64_t c = lane * VEC; c < a.D; c += 64 * VEC) {
        float x[VEC], v[VEC];
        load<uint16_t, VEC>(h + c, x);
        load<uint16_t, VEC>(w + c, v);
#pragma unroll
        for (int e = 0; e < VEC; ++e) { dot = fmaf(x[e], v[e], dot); sizes = fmaf(fabsf(x[e]), fabsf(v[e]), sizes); top = larger(top, x[e]); }
      }
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) { dot += __shfl_xor(dot, o, 64); sizes += __shfl_xor(sizes, o, 64); }
      // 1 - p_y, and no less than what the logit may be off by here and in the tile (a random walk of D roundings): what is
      // below that is noise, and must not be scaled beyond the type's range, 4 times the row's aim
      const float lse = a.lse[t], left = -expm1f(dot * a.scale - lse);
      const float noise = 5.9604645e-8f * (sqrtf((float)a.D) * sizes * fabsf(a.scale) + fabsf(lse) + 1.f);
      const float aim = left < noise ? noise : left;
      const int e = (aim < 1.f ? ilogbf(aim) + 1 : 0) - 14;
      k = Token{y, lse, ldexpf(1.f, -e), dl * a.scale * ldexpf(1.f, e)};
      most = top * k.rest;
    }
    if (t < a.T && lane == 0) a.tokens[t] = k;
    most = top_of<4>(most, part);
    if (threadIdx.x == 0) a.partial[blockIdx.x] = most;
    return;
  }
  constexpr int AHEAD = 8;  // loads in flight
  float top = 0.f;
  const int64_t waves = ((int64_t)gridDim.x - a.token_wgs) * 4;
  const int64_t first = ((int64_t)blockIdx.x - a.token_wgs) * 4 + wave;
  // `n` rows of `len` values in groups of W, a wave's loads of a row in flight together
  auto look = [&](auto width, const uint16_t* w, int64_t stride, int64_t n, int64_t len) {
    constexpr int W = decltype(width)::value;
    for (int64_t v = first; v < n; v += waves)
      for (int64_t c = lane * W; c < len; c += 64 * W * AHEAD) {
        float x[AHEAD][W];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
#pragma unroll
          for (int e = 0; e < W; ++e) x[u][e] = 0.f;
          if (c + u * 64 * W < len) load<uint16_t, W>(w + v * stride + c + u * 64 * W, x[u]);
        }
#pragma unroll
        for (int u = 0; u < AHEAD; ++u)
#pragma unroll
          for (int e = 0; e < W; ++e) top = larger(top, x[u][e]);
      }
  };
  const int64_t all = a.V * a.D;
  if (a.weight_stride == a.D && ((uintptr_t)a.weight & 15u) == 0) {  // one long row, whatever D is: rows of a wave's loads, then what is left
    constexpr int64_t LONG = 64 * 8 * AHEAD;
    look(std::integral_constant<int, 8>{}, a.weight, LONG, all / LONG, LONG);
    if (first == 0) {
      for (int64_t c = all / LONG * LONG + lane; c < all; c += 64) top = larger(top, up(a.weight[c]));
    }
  } else {
    look(std::integral_constant<int, VEC>{}, a.weight, a.weight_stride, a.V, a.D);
  }
  top = top_of<4>(top, part);
  if (threadIdx.x == 0) a.partial[blockIdx.x] = top;
}
// (By atomics on two words instead, thousands of workgroups waited for each other: 102 MB of weights took 120 us, 30 so.)
__global__ __launch_bounds__(1024) void tops_kernel(const float* partial, int token_wgs, int wgs, uint32_t* tops) {
  __shared__ float part[2][16];
  float v[2] = {0.f, 0.f};
  for (int i = threadIdx.x; i < wgs; i += 1024) v[i >= token_wgs] = larger(v[i >= token_wgs], partial[i]);
  const float states = top_of<16>(v[0], part[0]), weights = top_of<16>(v[1], part[1]);
  if (threadIdx.x == 0) { tops[TOP_STATES] = __float_as_uint(states); tops[TOP_WEIGHTS] = __float_as_uint(weights); }
}

__device__ __forceinline__ uint32_t f16_bits(float f) { return (uint32_t)__builtin_bit_cast(uint16_t, (_Float16)f); }

// 8192 tokens against a piece of 16,128 rows of 4096: 0.86 ms, 0.77 of it the product.
// G of a tile, in both orders.  Columns behind the piece's last and tokens behind the last are zeros: sums run over them.
// FEW: the gradient itself, as the sum of two bfloat16 values in planes of their own.
template <class S, bool FEW>
__device__ __forceinline__ void g_of(const Args& a, typename S::Acc (&acc)[S::FQ][S::FP], int64_t p0, int64_t q0, unsigned char* lds) {
  const int64_t T = a.hidden.rows;
  const int lane = opaque_lane(), wave = threadIdx.x >> 6, wp = wave % S::NWP, wq = wave / S::NWP;
  const int ql = wq * S::FQ * 16 + (lane >> 4) * 4;  // the lane's first column in the tile
  const int64_t q1 = q0 + ql;
  const int left = (int)min((int64_t)S::BQ, a.weight.rows - q1);
  // The second order of a tile that LDS holds whole is made there: two tokens of a column in a word, rows of all the tile's tokens whose 16-byte
  // chunks are stored in an order that spreads a store's eight rows over the banks.  (Stored by single values, it took 25 of a 256 x 256 tile's
  // 130 us; a quarter of the tile at a time, beside the next tile's loads, 6 more than so.)
  constexpr bool TURN = !FEW;
  static_assert(!TURN || S::BP * S::BQ * 2 <= S::LDS, "room");
  constexpr int CHUNKS = S::BP / 8;  // of a row
  auto place = [](int q, int chunk) { return q * (S::BP * 2) + ((chunk ^ ((((q >> 2) & 3) * 2 + (q & 1) * 8) & (CHUNKS - 1))) << 4); };
  if constexpr (TURN) __syncthreads();  // (the last step is read)
#pragma unroll
  for (int j = 0; j < S::FP; ++j) {
    const int pl = (wp * S::FP + j) * 16 + (lane & 15);
    const int64_t p = p0 + pl;
    Token k{-1, 0.f, 1.f, 0.f};
    if constexpr (FEW) {
      if (p < T && takes_part(a.targets[p], a.dloss[p], a.V)) k = Token{a.targets[p], a.lse[p], a.dloss[p] * a.scale, 0.f};
    } else {
      if (p < T) k = a.tokens[p];
    }
    const int64_t target = (int64_t)k.y - a.v0 - q1;
    const bool here = k.y >= 0 && target >= 0 && target < S::FQ * 16;
    constexpr int PAIR = S::FQ % 2 == 0 ? 2 : 1;
#pragma unroll
    for (int i0 = 0; i0 < S::FQ; i0 += PAIR) {
      uint2 word[PAIR];
#pragma unroll
      for (int n = 0; n < PAIR; ++n) {
        const int i = i0 + n;
        float f[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) f[e] = exp_of(acc[i][j][e] * a.scale - k.lse);
        if (here) {  // (few tiles hold a token's target)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (target == i * 16 + e) f[e] -= 1.f;
        }
        uint32_t v[4];
        if constexpr (FEW) {
          uint32_t low[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float x = k.y >= 0 && i * 16 + e < left ? f[e] * k.up : 0.f;
            v[e] = to_bf16(x);
            low[e] = to_bf16(x - up((uint16_t)v[e]));
          }
          if (a.g && p < T) *reinterpret_cast<uint2*>(a.g + a.g_plane + p * a.g_stride + q1 + i * 16) = uint2{low[0] | low[1] << 16, low[2] | low[3] << 16};
          if (a.gt && p < a.gt_stride) {
#pragma unroll
            for (int e = 0; e < 4; ++e) a.gt[a.gt_plane + (q1 + i * 16 + e) * a.gt_stride + p] = (uint16_t)low[e];
          }
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = k.y >= 0 && i * 16 + e < left ? f16_bits(f[e] * k.up) : 0u;
        }
        word[n] = uint2{v[0] | v[1] << 16, v[2] | v[3] << 16};
        if constexpr (TURN) {
          if (a.gt) {
            // of each pair of columns the even lane takes the first for both tokens, the odd one the second
            const bool odd = lane & 1;
#pragma unroll
            for (int e = 0; e < 4; e += 2) {
              const uint32_t other = (uint32_t)__builtin_amdgcn_mov_dpp((int)(odd ? v[e] : v[e + 1]), 0xB1, 0xF, 0xF, true);  // quad_perm 1 0 3 2
              *reinterpret_cast<uint32_t*>(lds + place(ql + i * 16 + e + odd, pl >> 3) + (pl & 6) * 2) = odd ? other | v[e + 1] << 16 : v[e] | other << 16;
            }
          }
        } else if (a.gt && p < a.gt_stride) {
#pragma unroll
          for (int e = 0; e < 4; ++e) a.gt[(q1 + i * 16 + e) * a.gt_stride + p] = (uint16_t)v[e];
        }
      }
      if (a.g) {
        if constexpr (PAIR == 2) {
          eight_of(word[0], word[1]);
          const int g = lane >> 4;
          if (p < T) *reinterpret_cast<uint4*>(a.g + p * a.g_stride + q1 - g * 4 + 16 * (g / 2) + 8 * (g % 2) + i0 * 16) = uint4{word[0].x, word[0].y, word[1].x, word[1].y};
        } else if (p < T) {
          *reinterpret_cast<uint2*>(a.g + p * a.g_stride + q1 + i0 * 16) = word[0];
        }
      }
    }
  }
  if constexpr (TURN) {
    if (!a.gt) return;
    __syncthreads();
    for (int n = threadIdx.x; n < S::BQ * CHUNKS; n += S::THREADS) {
      const int q = n / CHUNKS, c = n % CHUNKS;
      if (p0 + c * 8 < a.gt_stride)  // (a multiple of 16)
        *reinterpret_cast<i32x4*>(a.gt + (q0 + q) * a.gt_stride + p0 + c * 8) = *reinterpret_cast<const i32x4*>(lds + place(q, c));
    }
  }
}
template <class S, bool DIRECT, bool FEW>
__global__ __launch_bounds__(S::THREADS) void g_kernel(Args a) {
  __shared__ __align__(1024) unsigned char lds[S::LDS];
  planned<S, DIRECT, false>(a.hidden, a.weight, a.k_bytes, a.plan, lds,
                            [&](auto shape, auto& acc, int64_t p0, int64_t q0) { g_of<decltype(shape), FEW>(a, acc, p0, q0, lds); });
}

// out[c][r] = in[r][c], from bfloat16 to 16-bit floats of 11 bits in range: rows behind the last and rows of tokens that take no part are zeros,
// up to `r_out` rows.  Bound: memory, 264 MB in 56 us.
constexpr int TT = 64;
template <bool VEC>
__global__ __launch_bounds__(256) void transpose_kernel(const uint16_t* in, int64_t stride, int64_t rows, int64_t cols, uint16_t* out, int64_t out_stride,
                                                        int64_t r_out, const Token* tokens, const uint32_t* top) {
  __shared__ uint16_t tile[TT][TT + 2];
  const int64_t r0 = (int64_t)blockIdx.x * TT, c0 = (int64_t)blockIdx.y * TT;
  const float range = to_range(*top);
#pragma unroll
  for (int u = 0; u < TT * TT / 8 / 256; ++u) {
    const int i = u * 256 + threadIdx.x, r = i / (TT / 8), c = i % (TT / 8) * 8;
    const int64_t rr = r0 + r, cc = c0 + c;
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = 0.f;
    float m = range;
    bool on = rr < rows;
    if (on && tokens) {
      const Token k = tokens[rr];
      on = k.y >= 0;
      m *= k.rest;
    }
    if (on) {
      const uint16_t* p = in + rr * stride + cc;
      if (VEC && cc + 8 <= cols) load<uint16_t, 8>(p, v);
      else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (cc + e < cols) v[e] = up(p[e]);
      }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) tile[r][c + e] = (uint16_t)f16_bits(v[e] * m);
  }
  __syncthreads();
#pragma unroll
  for (int u = 0; u < TT * TT / 8 / 256; ++u) {
    const int i = u * 256 + threadIdx.x, c = i / (TT / 8), r = i % (TT / 8) * 8;
    if (c0 + c >= cols || r0 + r >= r_out) continue;  // (r_out is a multiple of 8)
    Group<uint16_t, 8> v;
#pragma unroll
    for (int e = 0; e < 8; ++e) v.v[e] = tile[r + e][c];
    *reinterpret_cast<Group<uint16_t, 8>*>(out + (c0 + c) * out_stride + r0 + r) = v;
  }
}

struct MulArgs {
  Operand p, q;
  int k_bytes, k_split;  // each of gridDim.y workgroups of a tile takes k_split bytes of k
  Plan plan;
  void* out;
  int64_t stride, split_stride;
  bool vec;                      // rows are 16-byte aligned
  const uint32_t* top;           // not null: the sums are brought back by from_range
};
// out[p][q] (+)= sum over k, in float32 or rounded once.  8192 x 4096 x 16,128 either way 0.78 ms (1.38 PFLOP/s).
template <class S, typename T, bool ADD>
__global__ __launch_bounds__(S::THREADS) void mul_kernel(MulArgs a) {
  __shared__ __align__(1024) unsigned char lds[S::LDS];
  const int k0 = blockIdx.y * a.k_split;
  a.p.p += k0;
  a.q.p += k0;
  const float back = a.top ? from_range(*a.top) : 1.f;
  planned<S, true, Cut<S>::CAN>(a.p, a.q, max(0, min(a.k_split, a.k_bytes - k0)), a.plan, lds, [&](auto shape, auto& acc, int64_t p0, int64_t q0) {
    using R = decltype(shape);
    const int lane = opaque_lane(), wave = threadIdx.x >> 6, g = lane >> 4;
    const int64_t p1 = p0 + wave % R::NWP * R::FP * 16 + (lane & 15), q1 = q0 + wave / R::NWP * R::FQ * 16;
    constexpr int PAIR = sizeof(T) == 2 && !ADD && R::FQ % 2 == 0 ? 2 : 1;
#pragma unroll
    for (int j = 0; j < R::FP; ++j) {
      const bool in = p1 + j * 16 < a.p.rows;
      T* row = (T*)a.out + blockIdx.y * a.split_stride + (p1 + j * 16) * a.stride;
#pragma unroll
      for (int i = 0; i < R::FQ; i += PAIR) {
        if constexpr (PAIR == 2) {
          uint2 x[2];
#pragma unroll
          for (int h = 0; h < 2; ++h)
            x[h] = uint2{two_bf16(acc[i + h][j][0] * back, acc[i + h][j][1] * back), two_bf16(acc[i + h][j][2] * back, acc[i + h][j][3] * back)};
          eight_of(x[0], x[1]);
          const int64_t q = q1 + i * 16 + 16 * (g / 2) + 8 * (g % 2);
          if (in) put8((uint16_t*)row + q, a.q.rows - q, uint4{x[0].x, x[0].y, x[1].x, x[1].y});
        } else {
          const int64_t q = q1 + i * 16 + g * 4;
          float v[4] = {acc[i][j][0] * back, acc[i][j][1] * back, acc[i][j][2] * back, acc[i][j][3] * back};
          if (in && a.vec && q + 4 <= a.q.rows) {
            if constexpr (ADD) {
              float o[4];
              load<T, 4>(row + q, o);
#pragma unroll
              for (int e = 0; e < 4; ++e) v[e] += o[e];
            }
            store<T, 4>(row + q, v);
          } else if (in) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (q + e < a.q.rows) row[q + e] = down<T>(ADD ? v[e] + up(row[q + e]) : v[e]);
          }
        }
      }
      __builtin_amdgcn_sched_barrier(0);  // (a row's values at a time: they are many beside the sums)
    }
  });
}

// dH: the splits' sums, in an order that depends on their number alone, times what G's rows and the weights' range lack; zeros for tokens that
// take no part.  HID_GROUPS threads share a column group's splits where there are several.
constexpr int HID_GROUPS = 4;
template <int VEC>
__global__ __launch_bounds__(64 * HID_GROUPS) void hidden_kernel(const float* sums, int64_t sums_stride, int splits, int64_t T, int64_t D, const Token* tokens, const uint32_t* top,
                                                                 const int32_t* targets, const float* dloss, int64_t V, uint16_t* out, int64_t stride) {
  __shared__ float part[HID_GROUPS][64 * VEC];
  const int64_t t = blockIdx.x;
  const bool on = takes_part(targets[t], dloss[t], V);
  const float m = tokens ? tokens[t].rest * from_range(*top) : 1.f;
  const bool shared_out = splits > 1;
  const int lane = threadIdx.x & 63, grp = threadIdx.x >> 6;
  const int64_t c = shared_out ? ((int64_t)blockIdx.y * 64 + lane) * VEC : ((int64_t)blockIdx.y * (64 * HID_GROUPS) + threadIdx.x) * VEC;
  float v[VEC];
#pragma unroll
  for (int e = 0; e < VEC; ++e) v[e] = 0.f;
  if (c < D && on) {
    const float* p = sums + t * sums_stride + c;
#pragma unroll 8
    for (int s = shared_out ? grp : 0; s < splits; s += HID_GROUPS) {
      float x[VEC];
      load<float, VEC>(p + (int64_t)s * T * sums_stride, x);
#pragma unroll
      for (int e = 0; e < VEC; ++e) v[e] += x[e];
    }
  }
  if (shared_out) {
#pragma unroll
    for (int e = 0; e < VEC; ++e) part[grp][lane * VEC + e] = v[e];
    __syncthreads();
    if (grp > 0) return;
#pragma unroll
    for (int g = 1; g < HID_GROUPS; ++g)
#pragma unroll
      for (int e = 0; e < VEC; ++e) v[e] += part[g][lane * VEC + e];
  }
  if (c < D) {
#pragma unroll
    for (int e = 0; e < VEC; ++e) v[e] = on ? v[e] * m : 0.f;
    store<uint16_t, VEC>(out + t * stride + c, v);
  }
}

// ---- few tokens: the weights are what is read, and each product takes them as they lie ----
// G is the sum of two bfloat16 values, 16 bits that need no range, so that neither weights nor states are copied into another type; twice the matrix
// instructions are free where the memory is the bound.
// Both outputs of 64 tokens against 128,256 x 4096, 50,001 x 1024 and 33,858 x 1408: 1017, 111 and 106 us so, 1407, 153 and 154 the other way (of 16 tokens 753, 85 and 77; 1378, 143
// and 147); 65 tokens, the other way, 1454, 162 and 160.  The bound is where this way's fragments in registers end, not where it stops paying.
constexpr int64_t FEW_GRAD = 64;
constexpr int FEW_STAGES = 3, FEW_K = 64;  // rows of the weights a step

// Fragments with k across an LDS tile's rows: each 16 lanes are given 4 rows of 16 values, and a lane gets its column's four.
typedef short s16x4 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ i32x4 turned(const unsigned char* rows0, const unsigned char* rows4) {
  typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
  const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(s16x4*)rows0), b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(s16x4*)rows4);
  const int2 x = __builtin_bit_cast(int2, a), y = __builtin_bit_cast(int2, b);
  return i32x4{x.x, x.y, y.x, y.y};
}

struct FewArgs {
  Operand weight;          // the piece's rows
  const uint16_t* g;       // two planes [T][g_stride]
  int64_t g_stride, g_plane, T, D;  // D: a multiple of 8, the weights' rows have as many values
  int split_rows;          // of the weights, a multiple of FEW_K
  float* sums;             // [splits][T][D]
  int add;
};
// sums[split][t][d] (+)= sum over the split's rows v of G[t][v] W[v][d]: a workgroup has 64 columns d, 16 a wave.  Bound: one read of the weights.
template <int BP>
__global__ __launch_bounds__(256) void dh_few_kernel(FewArgs a) {
  constexpr int FP = BP / 16, W_BYTES = FEW_K * KB, STAGE = W_BYTES + 2 * BP * KB;
  constexpr int GROUPS = 2 * BP / 8, LG = GROUPS / 4, NL = 2 + LG;  // loads a wave: its quarter of 8 + GROUPS groups of 8 rows
  __shared__ __align__(1024) unsigned char lds[FEW_STAGES * STAGE];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), row8 = lane >> 3, chunk = (lane & 7) ^ row8;
  const int64_t d0 = (int64_t)blockIdx.x * 64, v0 = (int64_t)blockIdx.y * a.split_rows;
  const int rows = (int)max((int64_t)0, min((int64_t)a.split_rows, a.weight.rows - v0)), steps = (rows + FEW_K - 1) / FEW_K;
  f32x4 acc[FP];
#pragma unroll
  for (int j = 0; j < FP; ++j) acc[j] = f32x4{0.f, 0.f, 0.f, 0.f};
  const Operand g{(const unsigned char*)a.g, a.g_stride * 2, a.T};
  const int g_bytes = (int)(a.g_stride * 2);
  const i32x4 res_hi = resource_of(g, 0, BP, g_bytes), res_lo = resource_of(Operand{g.p + a.g_plane * 2, g.stride, g.rows}, 0, BP, g_bytes);
  uint32_t off_w[2], off_g[LG];
  const uint32_t base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)lds;
#pragma unroll
  for (int i = 0; i < 2; ++i) off_w[i] = (uint32_t)((wave * 2 + i) * 8 + row8) * (uint32_t)a.weight.stride + (uint32_t)d0 * 2 + chunk * 16;
#pragma unroll
  for (int i = 0; i < LG; ++i) off_g[i] = (uint32_t)min(((wave * LG + i) * 8 + row8) % BP, (int)a.T - 1) * (uint32_t)g.stride + (uint32_t)v0 * 2 + chunk * 16;
  auto issue = [&](int s, int stage) {
    const uint32_t to = base + stage * STAGE;
    // (rows behind the last read as zeros)
    const i32x4 res_w = resource_of(a.weight, v0 + s * FEW_K, FEW_K, (int)(a.D * 2));
#pragma unroll
    for (int i = 0; i < 2; ++i) to_lds(to + (wave * 2 + i) * 1024, off_w[i], res_w, 0u);
#pragma unroll
    for (int i = 0; i < LG; ++i) to_lds(to + W_BYTES + (wave * LG + i) * 1024, off_g[i], (wave * LG + i) * 8 < BP ? res_hi : res_lo, (uint32_t)s * KB);
  };
  const int i16 = lane & 15, grp = lane >> 4, w_chunk = wave * 2 + ((i16 & 3) >> 1);
  const uint32_t at_w0 = (grp * 8 + i16 / 4) * KB + ((w_chunk ^ (i16 / 4)) << 4) + (i16 & 1) * 8;
  const uint32_t at_w4 = (grp * 8 + 4 + i16 / 4) * KB + ((w_chunk ^ (4 + i16 / 4)) << 4) + (i16 & 1) * 8;
  int in_flight = 0;
  for (; in_flight < FEW_STAGES - 1 && in_flight < steps; ++in_flight) issue(in_flight, in_flight);
  int stage = 0, next = in_flight;
  for (int s = 0; s < steps; ++s) {
    if (in_flight == FEW_STAGES - 1) arrived<(FEW_STAGES - 2) * NL>();
    else arrived<0>();
    if (next < steps) { issue(next, stage == 0 ? FEW_STAGES - 1 : stage - 1); ++next; }
    else --in_flight;
    const unsigned char* b = lds + stage * STAGE;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const i32x4 w = turned(b + at_w0 + h * 32 * KB, b + at_w4 + h * 32 * KB);
      const uint32_t c = (uint32_t)((h * 4 + grp) ^ (lane & 7)) * 16;
#pragma unroll
      for (int j = 0; j < FP; ++j) {
        const unsigned char* r = b + W_BYTES + (j * 16 + i16) * KB + c;
        acc[j] = Bf16::mma(w, *reinterpret_cast<const i32x4*>(r), acc[j]);
        acc[j] = Bf16::mma(w, *reinterpret_cast<const i32x4*>(r + BP * KB), acc[j]);
      }
    }
    stage = stage + 1 == FEW_STAGES ? 0 : stage + 1;
  }
#pragma unroll
  for (int j = 0; j < FP; ++j) {
    const int64_t t = j * 16 + i16, d = d0 + wave * 16 + grp * 4;
    if (t >= a.T || d >= a.D) continue;
    float* to = a.sums + ((int64_t)blockIdx.y * a.T + t) * a.D + d;
    float v[4] = {acc[j][0], acc[j][1], acc[j][2], acc[j][3]};
    if (a.add) {
      float o[4];
      load<float, 4>(to, o);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] += o[e];
    }
    store<float, 4>(to, v);
  }
}

// States with tokens along the rows, [D][t_pad] bfloat16: zeros for tokens that take no part, and behind the last.
__global__ __launch_bounds__(256) void states_few_kernel(const uint16_t* h, int64_t stride, int64_t T, int64_t D, int t_pad, const int32_t* targets, const float* dloss,
                                                         int64_t V, uint16_t* out) {
  const int64_t d = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int t0 = blockIdx.y * 8;
  if (d >= D) return;
  Group<uint16_t, 8> v;
#pragma unroll
  for (int e = 0; e < 8; ++e) v.v[e] = t0 + e < T && takes_part(targets[t0 + e], dloss[t0 + e], V) ? h[(t0 + e) * stride + d] : (uint16_t)0;
  *reinterpret_cast<Group<uint16_t, 8>*>(out + d * t_pad + t0) = v;
}

// dW[v][d] (+)= sum over the tokens of G[t][v] H[t][d]: a wave has 16 FEW_V rows v, whose fragments stay in registers, against the columns d in turn, 32 at a time.  Nothing goes
// through LDS: the states, [D][t_pad], come from the caches.  Bound: one write of the gradient.  `past`: a wave's stores are whole 64-byte pieces, which then go past
// the caches (a call of 12 tokens, 109,627 x 960: 191 us for 213; with pieces in two lines, 128,256 x 1016, 556 for 426).
constexpr int FEW_COLUMNS = 256, FEW_V = 4;
template <int KS, typename T, bool ADD>
__global__ __launch_bounds__(256) void dw_few_kernel(const uint16_t* gt, int64_t plane, const uint16_t* ht, int t_pad, int64_t n, int64_t D, T* out, int64_t stride, bool past) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i16 = lane & 15, grp = lane >> 4;
  const int64_t v0 = ((int64_t)blockIdx.x * 4 + wave) * (16 * FEW_V);
  if (v0 >= n) return;
  i32x4 hi[FEW_V][KS], lo[FEW_V][KS];
#pragma unroll
  for (int p = 0; p < FEW_V; ++p)
#pragma unroll
    for (int k = 0; k < KS; ++k) {
      const int t = k * 32 + grp * 8;
      const uint16_t* row = gt + min(v0 + p * 16 + i16, n - 1) * t_pad + t;
      hi[p][k] = lo[p][k] = i32x4{0, 0, 0, 0};
      if (t < t_pad) {
        hi[p][k] = *reinterpret_cast<const i32x4*>(row);
        lo[p][k] = *reinterpret_cast<const i32x4*>(row + plane);
      }
    }
  const int64_t d_end = min(D, ((int64_t)blockIdx.y + 1) * FEW_COLUMNS);
  for (int64_t d0 = (int64_t)blockIdx.y * FEW_COLUMNS; d0 < d_end; d0 += 32) {
    i32x4 h[2][KS];
#pragma unroll
    for (int q = 0; q < 2; ++q)
#pragma unroll
      for (int k = 0; k < KS; ++k) {
        const int t = k * 32 + grp * 8;
        h[q][k] = i32x4{0, 0, 0, 0};
        if (t < t_pad) h[q][k] = *reinterpret_cast<const i32x4*>(ht + min(d0 + q * 16 + i16, D - 1) * t_pad + t);
      }
#pragma unroll
    for (int p = 0; p < FEW_V; ++p) {
      f32x4 acc[2] = {f32x4{0.f, 0.f, 0.f, 0.f}, f32x4{0.f, 0.f, 0.f, 0.f}};
#pragma unroll
      for (int q = 0; q < 2; ++q)
#pragma unroll
        for (int k = 0; k < KS; ++k) {
          acc[q] = Bf16::mma(h[q][k], hi[p][k], acc[q]);
          acc[q] = Bf16::mma(h[q][k], lo[p][k], acc[q]);
        }
      const int64_t v = v0 + p * 16 + i16;
      const bool in = v < n;
      T* row = out + v * stride;
      if constexpr (sizeof(T) == 2 && !ADD) {
        uint2 x[2] = {uint2{two_bf16(acc[0][0], acc[0][1]), two_bf16(acc[0][2], acc[0][3])}, uint2{two_bf16(acc[1][0], acc[1][1]), two_bf16(acc[1][2], acc[1][3])}};
        eight_of(x[0], x[1]);
        const int64_t d = d0 + 16 * (grp / 2) + 8 * (grp % 2);
        const uint4 eight{x[0].x, x[0].y, x[1].x, x[1].y};
        if (in && past) put8<true>((uint16_t*)row + d, D - d, eight);
        else if (in) put8((uint16_t*)row + d, D - d, eight);
      } else {
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          const int64_t d = d0 + q * 16 + grp * 4;
          if (!in || d >= D) continue;
          T four[4];
          const bool all = d + 4 <= D;
          if constexpr (ADD) {
            if (all) __builtin_memcpy(four, row + d, sizeof(four));
            else
#pragma unroll
              for (int e = 0; e < 4; ++e) four[e] = d + e < D ? row[d + e] : (T)0;
          }
#pragma unroll
          for (int e = 0; e < 4; ++e) four[e] = down<T>(ADD ? acc[q][e] + up(four[e]) : acc[q][e]);
          if (all) __builtin_memcpy(row + d, four, sizeof(four));
          else
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (d + e < D) row[d + e] = four[e];
        }
      }
    }
  }
}

constexpr int SHORT_K = 4 * KB;
constexpr int64_t PIECE = (int64_t)1 << 27;   // values of G kept at a time (256 MB in each order)
constexpr int64_t ROUND = 256;                // a piece's rows: a multiple of every tile
constexpr int64_t MOST_ROWS = (int64_t)1 << 20;  // rows of G stay within what a buffer resource spans
int64_t piece_rows(int64_t T, int64_t V) {
  const int64_t most = std::min(MOST_ROWS, std::max<int64_t>(4096, PIECE / std::max<int64_t>(T, 1))), n = ceil_div(V, most);
  return ceil_div(ceil_div(V, n), ROUND) * ROUND;
}
// Workgroups a tile of dH: enough to fill the chip, each with at least 16 steps of k.
int hidden_splits(int64_t T, int64_t V, int64_t D) {
  const int64_t side = T <= 128 ? 128 : 256, tiles = std::max<int64_t>(1, ceil_div(T, side) * ceil_div(D, side)), want = T <= 128 ? 512 : 256;
  const int64_t most = std::max<int64_t>(1, piece_rows(T, V) * 2 / (16 * KB));
  return (int)std::max<int64_t>(1, std::min(most, want / tiles));
}

constexpr int64_t WEIGHT_WGS = 2048;  // workgroups that look for the weights' largest magnitude
struct Layout { int64_t copy_h, copy_w, tops, partial, tokens, g, gt, wt, ht, sums, total, rows, t16; int splits; };
// Totals are in whole pieces of 64 KB: a small call's is the same whether rows are aligned or not.
int64_t in_pieces(int64_t bytes) { return ceil_div(bytes, 65536) * 65536; }
Layout layout(int64_t T, int64_t V, int64_t D, bool hidden, bool weight, bool copies) {
  Layout L{};
  auto take = [&](int64_t bytes) { const int64_t at = L.total; L.total += (bytes + 255) & ~(int64_t)255; return at; };
  L.rows = piece_rows(T, V);
  L.t16 = ceil_div(T, 16) * 16;
  if (copies) {
    L.copy_h = take(T * aligned_stride(D * 2));
    L.copy_w = take(L.rows * aligned_stride(D * 2));
  }
  L.tops = take(TOPS * 4);
  L.partial = take((ceil_div(T, 4) + WEIGHT_WGS) * 4);
  L.tokens = take(T * (int64_t)sizeof(Token));
  if (hidden) {
    L.splits = hidden_splits(T, V, D);
    L.g = take(T * L.rows * 2);
    L.wt = take(D * L.rows * 2);
    L.sums = take((int64_t)L.splits * T * D * 4);
  }
  if (weight) {
    L.gt = take(L.rows * L.t16 * 2);
    L.ht = take(D * L.t16 * 2);
  }
  L.total = in_pieces(L.total);
  return L;
}

struct FewLayout { int64_t copy_h, copy_w, g, gt, ht, sums, total, rows, d_pad; int t_pad, splits, split_rows; };
FewLayout few_layout(int64_t T, int64_t V, int64_t D, bool hidden, bool weight, bool copies) {
  FewLayout L{};
  auto take = [&](int64_t bytes) { const int64_t at = L.total; L.total += (bytes + 255) & ~(int64_t)255; return at; };
  L.rows = copies ? std::min(ALIGN_ROWS, ceil_div(V, ROUND) * ROUND) : piece_rows(T, V);
  L.t_pad = (int)(ceil_div(T, 16) * 16);
  L.d_pad = ceil_div(D, 8) * 8;
  if (copies) {
    L.copy_h = take(T * L.d_pad * 2);
    L.copy_w = take(L.rows * L.d_pad * 2);
  }
  if (hidden) {
    // enough workgroups to fill the chip, each with at least eight steps
    const int64_t want = std::min(std::max<int64_t>(1, 1024 / ceil_div(D, 64)), std::max<int64_t>(1, L.rows / (8 * FEW_K)));
    L.split_rows = (int)(ceil_div(ceil_div(L.rows, want), FEW_K) * FEW_K);
    L.splits = (int)ceil_div(L.rows, L.split_rows);
    L.g = take(2 * T * L.rows * 2);
    L.sums = take((int64_t)L.splits * T * L.d_pad * 4);
  }
  if (weight) {
    L.gt = take(2 * L.rows * L.t_pad * 2);
    L.ht = take(D * L.t_pad * 2);
  }
  L.total = in_pieces(L.total);
  return L;
}

void transpose(const uint16_t* in, int64_t stride, int64_t rows, int64_t cols, uint16_t* out, int64_t out_stride, int64_t r_out, const Token* tokens,
               const uint32_t* top, hipStream_t st) {
  const dim3 grid((unsigned)ceil_div(r_out, TT), (unsigned)ceil_div(cols, TT));
  if (rows_aligned(in, stride, 2, 16))
    hipLaunchKernelGGL(transpose_kernel<true>, grid, dim3(256), 0, st, in, stride, rows, cols, out, out_stride, r_out, tokens, top);
  else
    hipLaunchKernelGGL(transpose_kernel<false>, grid, dim3(256), 0, st, in, stride, rows, cols, out, out_stride, r_out, tokens, top);
}

// Few steps of k, as dW of few tokens has: a tile is mostly stored, and two smaller ones on a compute unit do so in turn.  So too where a tile of 256
// columns would be half empty.
int multiply_tiles(int64_t p, int64_t q, int64_t k_bytes, int splits) {
  const int tiles = tiles_for(p, q);
  return k_bytes <= SHORT_K || q <= 128 ? std::min<int>(tiles, TILE_128) : splits > 1 && p > 128 ? TILE_256 : tiles;
}
void multiply(MulArgs a, int type, bool add, int splits, hipStream_t st) {
  a.k_split = (int)(ceil_div(ceil_div(a.k_bytes, splits), KB) * KB);
  a.vec = rows_aligned(a.out, a.stride, type_bytes(type), 16);
  shaped<F16>(multiply_tiles(a.p.rows, a.q.rows, a.k_bytes, splits), [&](auto shape) {
    using S = decltype(shape);
    a.plan = plan<S, Cut<S>::CAN>(a.p.rows, a.q.rows, splits == 1);
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3((unsigned)a.plan.grid, (unsigned)splits), dim3(S::THREADS), 0, st, a); };
    if (type == SIMPLE_F32) { if (add) go(mul_kernel<S, float, true>); else go(mul_kernel<S, float, false>); }
    else { if (add) go(mul_kernel<S, uint16_t, true>); else go(mul_kernel<S, uint16_t, false>); }
  });
}

}  // namespace xent
}  // namespace simple

using namespace simple::xent;

namespace {
constexpr int64_t MAX_T = (int64_t)1 << 20, MAX_V = (int64_t)1 << 28, MAX_D = 65536;

int check_sizes(int64_t T, int64_t V, int64_t D) {
  if (T < 0 || V <= 0 || D <= 0) return SIMPLE_EINVAL;
  return T > MAX_T || V > MAX_V || D > MAX_D ? SIMPLE_ECAPACITY : SIMPLE_OK;
}
bool good_scale(float s) { return s > 0.f && s <= 3.4e38f; }
// (Tiles are numbered in 32 bits.)
bool too_many_tiles(int64_t T, int64_t V) { return ceil_div(T, 16) * ceil_div(V, 64) > (int64_t)0x7FFFFFFF; }
int64_t pairs_bytes(int64_t T, int64_t V) { return ((ceil_div(V, tile_columns(tiles_for(T, V))) * T * (int64_t)sizeof(Pair) + 255) & ~(int64_t)255); }
// What a call needs beyond the sizes' least: copies of operands whose rows are not aligned (`fits`: both are).
int64_t xent_bytes(int64_t T, int64_t V, int64_t D, bool fits) {
  const int64_t copies = !fits && T > FEW_TOKENS ? (T + std::min(V, ALIGN_ROWS)) * aligned_stride(D * 2) : 0;
  return in_pieces(pairs_bytes(T, V) + ((T * 4 + 255) & ~(int64_t)255) + copies);
}
int64_t grad_bytes(int64_t T, int64_t V, int64_t D, bool hidden, bool weight, bool fits) {
  if (T > FEW_GRAD || T == 0) return layout(T, V, D, hidden, weight, !fits && T > FEW_TOKENS).total;
  const int64_t least = few_layout(T, V, D, hidden, weight, false).total;
  return fits ? least : std::max(least, few_layout(T, V, D, hidden, weight, true).total);
}
}  // namespace

extern "C" int64_t simple_xent_workspace(int64_t T, int64_t V, int64_t D) {
  const int rc = check_sizes(T, V, D);
  return rc != SIMPLE_OK ? rc : xent_bytes(T, V, D, false);
}
extern "C" int64_t simple_xent_workspace_aligned(int64_t T, int64_t V, int64_t D) {
  const int rc = check_sizes(T, V, D);
  return rc != SIMPLE_OK ? rc : xent_bytes(T, V, D, true);
}

extern "C" int simple_xent(const void* hidden_dev, int64_t hidden_stride, const void* weight_dev, int64_t weight_stride, const int32_t* targets_dev,
                           int64_t T, int64_t V, int64_t D, float logit_scale, float* loss_dev, float* lse_dev, void* workspace_dev,
                           int64_t workspace_bytes, void* hip_stream) {
  const int rc = check_sizes(T, V, D);
  if (rc != SIMPLE_OK) return rc;
  if (hidden_stride < D || weight_stride < D || !good_scale(logit_scale)) return SIMPLE_EINVAL;
  if (T == 0) return SIMPLE_OK;
  if (!hidden_dev || !weight_dev || !targets_dev || !loss_dev || !lse_dev) return SIMPLE_EINVAL;
  if (!workspace_dev || ((uintptr_t)workspace_dev & 15u) != 0) return SIMPLE_EINVAL;
  Args a{};
  a.hidden = {(const unsigned char*)hidden_dev, hidden_stride * 2, T};
  const Operand weight{(const unsigned char*)weight_dev, weight_stride * 2, V};
  const bool fits = direct(a.hidden, D * 2) && direct(weight, D * 2);
  if (too_many_tiles(T, V) || workspace_bytes < xent_bytes(T, V, D, fits)) return SIMPLE_ECAPACITY;
  hipStream_t st = (hipStream_t)hip_stream;
  unsigned char* ws = (unsigned char*)workspace_dev;
  a.k_bytes = (int)(D * 2);
  a.scale = logit_scale;
  a.targets = targets_dev;
  a.V = V;
  a.at_target = (float*)(ws + pairs_bytes(T, V));
  const int tiles = tiles_for(T, V);
  const int64_t columns = tile_columns(tiles), tiles_q = ceil_div(V, columns);
  auto stats = [&](const Operand& w, int64_t v0, bool dir) {
    a.weight = w;
    a.v0 = v0;
    a.pairs = (Pair*)ws + v0 / columns * T;
    shaped<Bf16>(tiles, [&](auto shape) {
      using S = decltype(shape);
      a.plan = plan<S, false>(T, w.rows);
      const dim3 grid((unsigned)a.plan.grid), block(S::THREADS);
      if (dir) hipLaunchKernelGGL((stats_kernel<S, true>), grid, block, 0, st, a);
      else hipLaunchKernelGGL((stats_kernel<S, false>), grid, block, 0, st, a);
    });
  };
  auto pieces = [&](bool dir) {  // one, but for tens of thousands of tokens against millions of weights
    const int64_t most = LAUNCH_WGS / ceil_div(T, tile_rows(tiles)) * columns;
    for (int64_t v0 = 0; v0 < V; v0 += most) stats(Operand{weight.p + v0 * weight.stride, weight.stride, std::min(most, V - v0)}, v0, dir);
  };
  if (fits) {
    pieces(true);
  } else if (T <= FEW_TOKENS) {
    pieces(false);
  } else {  // copies with aligned rows, of the weights ALIGN_ROWS (a multiple of every tile) at a time
    unsigned char* room = ws + pairs_bytes(T, V) + ((T * 4 + 255) & ~(int64_t)255);
    a.hidden = aligned_copy<2>(a.hidden, D * 2, room, st);
    a.k_bytes = (int)a.hidden.stride;
    for (int64_t v0 = 0; v0 < V; v0 += ALIGN_ROWS)
      stats(aligned_copy<2>(Operand{weight.p + v0 * weight.stride, weight.stride, std::min(ALIGN_ROWS, V - v0)}, D * 2, room + T * a.hidden.stride, st), v0, true);
  }
  auto finish = [&](auto tokens) {
    constexpr int N = decltype(tokens)::value;
    hipLaunchKernelGGL((finish_kernel<N>), dim3((unsigned)ceil_div(T, N)), dim3(FIN_THREADS), 0, st, (const Pair*)ws, (int)tiles_q, T, V, targets_dev,
                       (const float*)a.at_target, loss_dev, lse_dev);
  };
  if (T <= FEW_FIN) finish(std::integral_constant<int, 2>{});
  else finish(std::integral_constant<int, 16>{});
  return launched();
}

extern "C" int64_t simple_xent_grad_workspace(int64_t T, int64_t V, int64_t D, int want_dhidden, int want_dweight) {
  const int rc = check_sizes(T, V, D);
  if (rc != SIMPLE_OK) return rc;
  return grad_bytes(T, V, D, want_dhidden != 0, want_dweight != 0, false);
}
extern "C" int64_t simple_xent_grad_workspace_aligned(int64_t T, int64_t V, int64_t D, int want_dhidden, int want_dweight) {
  const int rc = check_sizes(T, V, D);
  if (rc != SIMPLE_OK) return rc;
  return grad_bytes(T, V, D, want_dhidden != 0, want_dweight != 0, true);
}

extern "C" int simple_xent_grad(const float* dloss_dev, const void* hidden_dev, int64_t hidden_stride, const void* weight_dev, int64_t weight_stride,
                                const int32_t* targets_dev, const float* lse_dev, int64_t T, int64_t V, int64_t D, float logit_scale,
                                void* dhidden_dev, int64_t dhidden_stride, void* dweight_dev, int64_t dweight_stride, int dweight_dtype,
                                int accumulate, void* workspace_dev, int64_t workspace_bytes, void* hip_stream) {
  const int rc = check_sizes(T, V, D);
  if (rc != SIMPLE_OK) return rc;
  if (hidden_stride < D || weight_stride < D || (dhidden_dev && dhidden_stride < D) || (dweight_dev && dweight_stride < D)) return SIMPLE_EINVAL;
  if (!good_type(dweight_dtype) || !good_scale(logit_scale)) return SIMPLE_EINVAL;
  if (T == 0) dhidden_dev = nullptr;
  if (!dhidden_dev && (!dweight_dev || (T == 0 && accumulate))) return SIMPLE_OK;
  hipStream_t st = (hipStream_t)hip_stream;
  const Operand all_rows{(const unsigned char*)weight_dev, weight_stride * 2, V};
  const bool fits = direct(Operand{(const unsigned char*)hidden_dev, hidden_stride * 2, T}, D * 2) && direct(all_rows, D * 2);
  const bool copies = !fits && T > FEW_TOKENS;
  const Layout L = layout(T, V, D, dhidden_dev != nullptr, dweight_dev != nullptr, copies);
  if (T > 0) {
    if (!dloss_dev || !hidden_dev || !weight_dev || !targets_dev || !lse_dev || !workspace_dev || ((uintptr_t)workspace_dev & 15u) != 0) return SIMPLE_EINVAL;
    if (too_many_tiles(T, V) || workspace_bytes < grad_bytes(T, V, D, dhidden_dev != nullptr, dweight_dev != nullptr, fits)) return SIMPLE_ECAPACITY;
  }
  unsigned char* ws = (unsigned char*)workspace_dev;
  Args a{};
  a.hidden = {(const unsigned char*)hidden_dev, hidden_stride * 2, T};
  a.k_bytes = (int)(D * 2);
  a.scale = logit_scale;
  a.targets = targets_dev;
  a.V = V;
  a.lse = lse_dev;
  a.dloss = dloss_dev;
  auto hidden = [&](const float* sums, int64_t sums_stride, int splits, const Token* tokens, const uint32_t* top) {
    auto go = [&](auto kernel, int vec) {
      const int64_t columns = (int64_t)64 * vec * (splits > 1 ? 1 : HID_GROUPS);
      hipLaunchKernelGGL(kernel, dim3((unsigned)T, (unsigned)ceil_div(D, columns)), dim3(64 * HID_GROUPS), 0, st, sums, sums_stride, splits, T, D, tokens, top, targets_dev, dloss_dev, V,
                         (uint16_t*)dhidden_dev, dhidden_stride);
    };
    if (D % 4 == 0 && sums_stride % 4 == 0 && rows_aligned(dhidden_dev, dhidden_stride, 2, 8)) go(hidden_kernel<4>, 4);
    else go(hidden_kernel<1>, 1);
  };
  if (T > 0 && T <= FEW_GRAD) {
    // (rows that are not aligned: copies, of the weights a piece at a time)
    const FewLayout F = few_layout(T, V, D, dhidden_dev != nullptr, dweight_dev != nullptr, !fits);
    a.k_bytes = (int)(F.d_pad * 2);
    if (!fits) a.hidden = aligned_copy<2>(a.hidden, D * 2, ws + F.copy_h, st);
    if (dhidden_dev) { a.g = (uint16_t*)(ws + F.g); a.g_stride = F.rows; a.g_plane = T * F.rows; }
    if (dweight_dev) { a.gt = (uint16_t*)(ws + F.gt); a.gt_stride = F.t_pad; a.gt_plane = F.rows * F.t_pad; }
    if (dweight_dev)
      hipLaunchKernelGGL(states_few_kernel, dim3((unsigned)ceil_div(D, 256), (unsigned)(F.t_pad / 8)), dim3(256), 0, st, (const uint16_t*)hidden_dev, hidden_stride, T, D,
                         F.t_pad, targets_dev, dloss_dev, V, (uint16_t*)(ws + F.ht));
    for (int64_t v0 = 0; v0 < V; v0 += F.rows) {
      const int64_t n = std::min(F.rows, V - v0);
      a.weight = {all_rows.p + v0 * all_rows.stride, all_rows.stride, n};
      a.v0 = v0;
      if (!fits) a.weight = aligned_copy<2>(a.weight, D * 2, ws + F.copy_w, st);
      auto form = [&](auto shape) {
        using S = decltype(shape);
        a.plan = plan<S, false>(T, n);
        hipLaunchKernelGGL((g_kernel<S, true, true>), dim3((unsigned)a.plan.grid), dim3(S::THREADS), 0, st, a);
      };
      if (T <= 16) form(Shape<Bf16, 16, 64, 1, 4, 4>{});
      else if (T <= 32) form(Shape<Bf16, 32, 64, 1, 4, 4>{});
      else form(Shape<Bf16, 64, 128, 1, 4, 3>{});
      if (dhidden_dev) {
        const FewArgs f{a.weight, a.g, a.g_stride, a.g_plane, T, F.d_pad, F.split_rows, (float*)(ws + F.sums), v0 > 0};
        const dim3 grid((unsigned)ceil_div(D, 64), (unsigned)F.splits);
        if (T <= 16) hipLaunchKernelGGL(dh_few_kernel<16>, grid, dim3(256), 0, st, f);
        else if (T <= 32) hipLaunchKernelGGL(dh_few_kernel<32>, grid, dim3(256), 0, st, f);
        else hipLaunchKernelGGL(dh_few_kernel<64>, grid, dim3(256), 0, st, f);
      }
      if (dweight_dev) {
        auto go = [&](auto kernel, auto* type) {
          hipLaunchKernelGGL(kernel, dim3((unsigned)ceil_div(n, 64 * FEW_V), (unsigned)ceil_div(D, FEW_COLUMNS)), dim3(256), 0, st, (const uint16_t*)a.gt, a.gt_plane,
                             (const uint16_t*)(ws + F.ht), F.t_pad, n, D, (decltype(type))dweight_dev + v0 * dweight_stride, dweight_stride,
                             rows_aligned(dweight_dev, dweight_stride, type_bytes(dweight_dtype), 64));
        };
        auto typed = [&](auto ks) {
          constexpr int KS = decltype(ks)::value;
          if (dweight_dtype == SIMPLE_F32) { if (accumulate) go(dw_few_kernel<KS, float, true>, (float*)0); else go(dw_few_kernel<KS, float, false>, (float*)0); }
          else { if (accumulate) go(dw_few_kernel<KS, uint16_t, true>, (uint16_t*)0); else go(dw_few_kernel<KS, uint16_t, false>, (uint16_t*)0); }
        };
        if (T <= 32) typed(std::integral_constant<int, 1>{});
        else typed(std::integral_constant<int, 2>{});
      }
    }
    if (dhidden_dev) hidden((const float*)(ws + F.sums), F.d_pad, F.splits, nullptr, nullptr);
    return launched();
  }
  uint32_t* tops = (uint32_t*)(ws + L.tops);
  Token* tokens = (Token*)(ws + L.tokens);
  a.tokens = tokens;
  if (dhidden_dev) { a.g = (uint16_t*)(ws + L.g); a.g_stride = L.rows; }
  if (dweight_dev) { a.gt = (uint16_t*)(ws + L.gt); a.gt_stride = L.t16; }
  const unsigned char* weight = (const unsigned char*)weight_dev;
  if (T > 0) {
    PrepareArgs r{(const uint16_t*)hidden_dev, (const uint16_t*)weight_dev, hidden_stride, weight_stride, T, V, D, targets_dev, lse_dev, dloss_dev,
                  logit_scale, tokens, (float*)(ws + L.partial), (int)ceil_div(T, 4)};
    // (the weights' range is dH's: its product alone reads them in 16-bit floats)
    const dim3 grid((unsigned)(r.token_wgs + (dhidden_dev ? std::min<int64_t>(WEIGHT_WGS, ceil_div(V, 4)) : 0)));
    if (D % 8 == 0 && rows_aligned(hidden_dev, hidden_stride, 2, 16) && rows_aligned(weight_dev, weight_stride, 2, 16))
      hipLaunchKernelGGL(prepare_kernel<8>, grid, dim3(256), 0, st, r);
    else
      hipLaunchKernelGGL(prepare_kernel<1>, grid, dim3(256), 0, st, r);
    hipLaunchKernelGGL(tops_kernel, dim3(1), dim3(1024), 0, st, (const float*)r.partial, r.token_wgs, (int)grid.x, tops);
    if (dweight_dev)
      transpose((const uint16_t*)hidden_dev, hidden_stride, T, D, (uint16_t*)(ws + L.ht), L.t16, L.t16, tokens, tops + TOP_STATES, st);
  }
  if (copies) {
    a.hidden = aligned_copy<2>(a.hidden, D * 2, ws + L.copy_h, st);
    a.k_bytes = (int)a.hidden.stride;
  }
  for (int64_t v0 = 0; v0 < V; v0 += L.rows) {
    const int64_t n = std::min(L.rows, V - v0), n8 = ceil_div(n, 8) * 8;
    a.weight = {weight + v0 * weight_stride * 2, weight_stride * 2, n};
    a.v0 = v0;
    if (copies) a.weight = aligned_copy<2>(a.weight, D * 2, ws + L.copy_w, st);
    if (T > 0) {
      const bool dir = direct(a.hidden, a.k_bytes) && direct(a.weight, a.k_bytes);
      auto form = [&](auto shape) {
        using S = decltype(shape);
        a.plan = plan<S, false>(T, n);
        const dim3 grid((unsigned)a.plan.grid), block(S::THREADS);
        if (dir) hipLaunchKernelGGL((g_kernel<S, true, false>), grid, block, 0, st, a);
        else hipLaunchKernelGGL((g_kernel<S, false, false>), grid, block, 0, st, a);
      };
      if (tiles_for(T, n) == TILE_256) form(Shape<Bf16, 256, 256, 2, 4, 2>{});
      else form(Shape<Bf16, 128, 128, 2, 2, 2>{});
    }
    if (dhidden_dev) {
      transpose((const uint16_t*)a.weight.p, a.weight.stride / 2, n, D, (uint16_t*)(ws + L.wt), L.rows, n8, nullptr, tops + TOP_WEIGHTS, st);
      MulArgs m{};
      m.p = {(const unsigned char*)a.g, a.g_stride * 2, T};
      m.q = {ws + L.wt, L.rows * 2, D};
      m.k_bytes = (int)(n8 * 2);
      m.out = ws + L.sums;
      m.stride = D;
      m.split_stride = T * D;
      multiply(m, SIMPLE_F32, v0 > 0, L.splits, st);
    }
    if (dweight_dev) {
      MulArgs m{};
      m.p = {(const unsigned char*)a.gt, a.gt_stride * 2, n};
      m.q = {ws + L.ht, L.t16 * 2, D};
      m.k_bytes = (int)(L.t16 * 2);
      m.out = (unsigned char*)dweight_dev + v0 * dweight_stride * type_bytes(dweight_dtype);
      m.stride = dweight_stride;
      m.top = T > 0 ? tops + TOP_STATES : nullptr;
      multiply(m, dweight_dtype, accumulate != 0, 1, st);
    }
  }
  if (dhidden_dev) hidden((const float*)(ws + L.sums), D, L.splits, tokens, tops + TOP_WEIGHTS);
  return launched();
}
