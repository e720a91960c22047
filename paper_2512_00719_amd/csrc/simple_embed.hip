// Embedding lookup with scaling, and its gradient.
//
// Lookup: bound by memory, one read and one write of a row's bytes; nothing is computed but the scale.
//
// Gradient: the tokens are sorted by id (stable, so that a row's tokens keep their order; few tokens are found where a sort would put them), then summed in chunks of CHUNK sorted
// places (FEW_CHUNK up to FEW tokens).  A row whose tokens lie within a chunk is finished there; one that runs on leaves a partial sum in each chunk, and the
// chunk that it began in joins them in order.  No atomics on sums: a row's order of additions depends on the ids and their number alone, not
// on the order of workgroups, on the width or on the types.  A
// frequent token (8 % of a text's tokens are one word) is so spread over many workgroups.
// Bound: the zeros of the rows without a token, V * D values, are most of what is written.
#include <algorithm>

#include "simple_vocabdev.hpp"

namespace simple {
namespace embed {

using namespace vocab;

constexpr int WG = 256;
constexpr int RD = 4;              // rows in flight per thread of the lookup
constexpr int TILE = 1024;         // tokens a workgroup of the sort
constexpr int BITS = 9, BINS = 1 << BITS;
constexpr int CHUNK = 32;          // sorted places a workgroup of the sums
constexpr int FEW_CHUNK = 16;      // the same of up to FEW tokens, whose sums wait for one workgroup's rows (600 tokens of 1024 values: 9.6 us, 16.7 with 32)
constexpr int ROUNDS = TILE / WG;  // a wave's tokens, 64 at a time

// ---- lookup ----
// A thread has RD rows' loads in flight; 8192 rows of 4096 bfloat16 values of 128,256, 134 MB, 19 us (frequent rows come from the caches).
template <typename T, int VEC, bool WHOLE>
__global__ __launch_bounds__(WG) void lookup_kernel(const int32_t* ids, const T* table, int64_t table_stride, int64_t n, int64_t V, int64_t D,
                                                    float scale, T* out, int64_t out_stride) {
  const int64_t c = ((int64_t)blockIdx.y * blockDim.x + threadIdx.x) * VEC;
  if (c >= D) return;
  const int64_t r0 = (int64_t)blockIdx.x * (blockDim.y * RD) + threadIdx.y;
  float v[RD][VEC];
#pragma unroll
  for (int k = 0; k < RD; ++k) {
    const int64_t r = r0 + k * blockDim.y;
    const int id = r < n ? ids[r] : -1;
#pragma unroll
    for (int j = 0; j < VEC; ++j) v[k][j] = 0.f;
    if (id >= 0 && id < V) load_some<T, VEC, WHOLE>(table + id * table_stride, c, D, v[k]);
  }
#pragma unroll
  for (int k = 0; k < RD; ++k) {
    const int64_t r = r0 + k * blockDim.y;
    if (r >= n) return;
#pragma unroll
    for (int j = 0; j < VEC; ++j) v[k][j] *= scale;
    store_some<T, VEC, WHOLE>(out + r * out_stride + c, D - c, v[k]);
  }
}

// ---- zeros ----
struct Fill {
  unsigned char* p;
  int64_t rows, row_bytes, stride_bytes, first;  // first: the share's number in the table
};
// Zeros are written beside the sort's kernels, a share of the table by each: the sort leaves most of the chip idle.  Workgroup `at` of a
// kernel takes one store of 16 bytes a thread: 525 MB at 6.7 TB/s so, 5.9 with pieces of 16 KB, 5.0 to 5.5 with 64 KB, 4.4 with workgroups
// that go on to other pieces.  The stores are non-temporal, which leaves what the sums read next in the caches (16,384 tokens of 2048 bfloat16 values: sums
// 23 us, 36 behind ordinary stores).
typedef uint32_t v4u __attribute__((ext_vector_type(4)));
__device__ __forceinline__ void fill_piece(unsigned char* p, int64_t bytes) {  // 2-byte aligned
  const int64_t head = min(bytes, (int64_t)((16u - (uint32_t)(uintptr_t)p) & 15u)), body = (bytes - head) / 16;
  v4u* q = reinterpret_cast<v4u*>(p + head);
  const v4u zero = {0u, 0u, 0u, 0u};
  for (int64_t i = threadIdx.x; i < body; i += blockDim.x) __builtin_nontemporal_store(zero, q + i);
  for (int64_t k = 2 * threadIdx.x; k < head; k += 2 * blockDim.x) *reinterpret_cast<uint16_t*>(p + k) = 0;
  for (int64_t k = head + 16 * body + 2 * threadIdx.x; k < bytes; k += 2 * blockDim.x) *reinterpret_cast<uint16_t*>(p + k) = 0;
}
__device__ __forceinline__ void fill_share(const Fill& f, int64_t at) {
  const int64_t piece = 16 * (int64_t)blockDim.x;
  at += f.first;
  if (f.row_bytes == f.stride_bytes) {  // one long row
    const int64_t all = f.rows * f.row_bytes, b = at * piece;
    if (b < all) fill_piece(f.p + b, min(piece, all - b));
  } else {
    const int64_t each = max((int64_t)1, piece / f.row_bytes), r1 = min(f.rows, (at + 1) * each);
    for (int64_t r = at * each; r < r1; ++r) fill_piece(f.p + r * f.stride_bytes, f.row_bytes);
  }
}
inline int64_t fill_workgroups(const Fill& f, int threads) {
  const int64_t piece = 16 * (int64_t)threads;
  return f.row_bytes == f.stride_bytes ? ceil_div(f.rows * f.row_bytes, piece) : ceil_div(f.rows, std::max<int64_t>(1, piece / f.row_bytes));
}

// ---- sort: stable, BITS bits of the id a pass, from the lowest ----
struct Sort {
  const int32_t *key_in, *pos_in;  // pos_in null: first pass, the tokens in their own order
  int32_t *key_out, *pos_out;
  int32_t* counts;                 // [tiles][BINS]
  int64_t n, V;
  int tiles, shift;
};
// An id outside the vocabulary sorts behind all others, as V.
__device__ __forceinline__ int32_t key_of(const Sort& s, int64_t i) {
  const int32_t k = s.key_in[i];
  return (k < 0 || k >= s.V) ? (int32_t)s.V : k;
}

__global__ __launch_bounds__(WG) void count_kernel(Sort s, Fill f) {
  if ((int)blockIdx.x >= s.tiles) { fill_share(f, (int)blockIdx.x - s.tiles); return; }
  __shared__ int32_t cnt[BINS];
  for (int i = threadIdx.x; i < BINS; i += WG) cnt[i] = 0;
  __syncthreads();
  const int64_t t0 = (int64_t)blockIdx.x * TILE;
  for (int k = 0; k < ROUNDS; ++k) {
    const int64_t i = t0 + k * WG + threadIdx.x;
    if (i < s.n) atomicAdd(&cnt[((uint32_t)key_of(s, i) >> s.shift) & (BINS - 1)], 1);
  }
  __syncthreads();
  for (int i = threadIdx.x; i < BINS; i += WG) s.counts[(int64_t)blockIdx.x * BINS + i] = cnt[i];
}

// Places of a tile's tokens by one digit: behind all tokens of lower digits, those of the same digit in earlier tiles (`ahead`, of `all`), in earlier
// waves of the tile, in earlier rounds of the wave and in lower lanes.  Thread t's digits are 2t and 2t + 1 below BINS.  Each wave holds R rounds of 64
// consecutive tokens, `n` of the tile's exist; place[k] is round k's.
template <int NW, int R>
__device__ __forceinline__ void places(const int32_t (&key)[R], int n, int shift, bool alone, const int32_t (&ahead)[2], int32_t (&all)[2], int32_t (*cnt)[BINS],
                                       int32_t* scan, int32_t (&place)[R]) {
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  for (int i = tid; i < NW * BINS; i += 64 * NW) (&cnt[0][0])[i] = 0;
  __syncthreads();
#pragma unroll
  for (int k = 0; k < R; ++k) {
    const bool in = wave * (R * 64) + k * 64 + lane < n;
    const uint32_t d = ((uint32_t)key[k] >> shift) & (BINS - 1);
    uint64_t same = __ballot(in);
#pragma unroll
    for (int b = 0; b < BITS; ++b) {
      const uint64_t set = __ballot((d >> b) & 1u);
      same &= ((d >> b) & 1u) ? set : ~set;
    }
    const int first = in ? __ffsll((unsigned long long)same) - 1 : lane;
    int32_t old = 0;
    if (in && lane == first) old = atomicAdd(&cnt[wave][d], (int32_t)__popcll(same));
    place[k] = __shfl(old, first, 64) + (int32_t)__popcll(same & ((1ull << lane) - 1ull));
  }
  __syncthreads();
  int32_t own[2] = {0, 0};
  const bool digits = 2 * tid < BINS;
  if (digits) {
#pragma unroll
    for (int w = 0; w < NW; ++w) { own[0] += cnt[w][2 * tid]; own[1] += cnt[w][2 * tid + 1]; }
  }
  if (alone) { all[0] = own[0]; all[1] = own[1]; }
  int32_t pre = all[0] + all[1];
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int32_t up = __shfl_up(pre, o, 64);
    if (lane >= o) pre += up;
  }
  if (lane == 63) scan[wave] = pre;
  __syncthreads();
  for (int w = 0; w < wave; ++w) pre += scan[w];
  if (digits) {
    int32_t base[2] = {pre - all[0] - all[1] + ahead[0], pre - all[1] + ahead[1]};
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      const int32_t c0 = cnt[w][2 * tid], c1 = cnt[w][2 * tid + 1];
      cnt[w][2 * tid] = base[0]; cnt[w][2 * tid + 1] = base[1];
      base[0] += c0; base[1] += c1;
    }
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < R; ++k) place[k] += cnt[wave][((uint32_t)key[k] >> shift) & (BINS - 1)];
}

// (A pass over 16,384 tokens, count_kernel and this, takes 8 us; with a quarter of 525 MB of zeros beside each of the four kernels 20 us each.)
__global__ __launch_bounds__(WG) void place_kernel(Sort s, Fill f) {
  if ((int)blockIdx.x >= s.tiles) { fill_share(f, (int)blockIdx.x - s.tiles); return; }
  __shared__ int32_t cnt[WG / 64][BINS];
  __shared__ int32_t scan[WG / 64];
  static_assert(2 * WG >= BINS, "two digits a thread");
  const int tid = threadIdx.x;
  int32_t ahead[2] = {0, 0}, all[2] = {0, 0};  // counts of the tiles ahead, and of all
  // (Each tile counting all of them itself would spare a kernel a pass: 16,384 tokens 125 us so, 117 with the counts of the kernel before.)
#pragma unroll 4
  for (int t = 0; t < s.tiles; ++t) {
    const int2 c = *reinterpret_cast<const int2*>(s.counts + (int64_t)t * BINS + 2 * tid);
    all[0] += c.x; all[1] += c.y;
    if (t < (int)blockIdx.x) { ahead[0] += c.x; ahead[1] += c.y; }
  }
  const int64_t w0 = (int64_t)blockIdx.x * TILE + (tid >> 6) * (ROUNDS * 64) + (tid & 63);
  int32_t key[ROUNDS], pos[ROUNDS], place[ROUNDS];
#pragma unroll
  for (int k = 0; k < ROUNDS; ++k) {
    const int64_t i = w0 + k * 64;
    key[k] = i < s.n ? key_of(s, i) : 0;
    pos[k] = i < s.n ? (s.pos_in ? s.pos_in[i] : (int32_t)i) : 0;
  }
  places<WG / 64, ROUNDS>(key, (int)min((int64_t)TILE, s.n - (int64_t)blockIdx.x * TILE), s.shift, false, ahead, all, cnt, scan, place);
#pragma unroll
  for (int k = 0; k < ROUNDS; ++k) {
    if (w0 + k * 64 < s.n) {
      s.key_out[place[k]] = key[k];
      s.pos_out[place[k]] = pos[k];
    }
  }
}

// The whole sort of up to FEW tokens by one workgroup, which passes them through LDS from digit to digit (5 us for 1605 tokens; as kernels of their own
// the four steps took 16).
constexpr int FEW_WG = 1024, FEW = 4096, FEW_ROUNDS = FEW / FEW_WG;
__global__ __launch_bounds__(FEW_WG) void sort_few_kernel(Sort s, int passes, Fill f) {
  if (blockIdx.x > 0 || s.n == 0) { fill_share(f, (int)blockIdx.x - (s.n > 0)); return; }
  __shared__ int32_t cnt[FEW_WG / 64][BINS];
  __shared__ int32_t scan[FEW_WG / 64];
  __shared__ int2 held[FEW];
  const int w0 = (threadIdx.x >> 6) * (FEW_ROUNDS * 64) + (threadIdx.x & 63), n = (int)s.n;
  int32_t key[FEW_ROUNDS], pos[FEW_ROUNDS], place[FEW_ROUNDS];
#pragma unroll
  for (int k = 0; k < FEW_ROUNDS; ++k) {
    key[k] = w0 + k * 64 < n ? key_of(s, w0 + k * 64) : 0;
    pos[k] = w0 + k * 64;
  }
  for (int p = 0; p < passes; ++p) {
    const int32_t ahead[2] = {0, 0};
    int32_t all[2] = {0, 0};
    places<FEW_WG / 64, FEW_ROUNDS>(key, n, p * BITS, true, ahead, all, cnt, scan, place);
    __syncthreads();  // (what was held is read)
#pragma unroll
    for (int k = 0; k < FEW_ROUNDS; ++k)
      if (w0 + k * 64 < n) held[place[k]] = int2{key[k], pos[k]};
    __syncthreads();
#pragma unroll
    for (int k = 0; k < FEW_ROUNDS; ++k)
      if (w0 + k * 64 < n) { key[k] = held[w0 + k * 64].x; pos[k] = held[w0 + k * 64].y; }
  }
#pragma unroll
  for (int k = 0; k < FEW_ROUNDS; ++k)
    if (w0 + k * 64 < n) { s.key_out[w0 + k * 64] = key[k]; s.pos_out[w0 + k * 64] = pos[k]; }
}

// ---- sums ----
// 16,384 tokens of 2048 bfloat16 values: 23 us with eight rows in flight a thread, 44 with a branch ahead of each load.
struct Sums {
  const int32_t *key, *pos;  // sorted
  const void* dout;
  int64_t dout_stride, n, V, D;
  float scale;
  void* dtable;
  int64_t dtable_stride;
  int chunk;       // sorted places a workgroup of the sums
  int64_t first;   // the launch's first chunk
  float* partial;  // [chunks][2][D]: of the row that the chunk begins inside, and of the one that it ends inside
};

template <typename TO, int VEC, bool WHOLE, bool ADD> __device__ __forceinline__ void finish(const Sums& s, int32_t id, int64_t c, float (&acc)[VEC]) {
  TO* row = (TO*)s.dtable + id * s.dtable_stride;
  float v[VEC];
#pragma unroll
  for (int j = 0; j < VEC; ++j) v[j] = 0.f;
  if constexpr (ADD) load_some<TO, VEC, WHOLE>(row, c, s.D, v);
#pragma unroll
  for (int j = 0; j < VEC; ++j) v[j] = fmaf(acc[j], s.scale, v[j]);
  store_some<TO, VEC, WHOLE>(row + c, s.D - c, v);
}

template <typename T, typename TO, int VEC, bool ADD>
__global__ __launch_bounds__(WG) void sums_kernel(Sums s) {
  __shared__ int32_t key[CHUNK + 2], pos[CHUNK];
  const int64_t chunk = s.first + blockIdx.x, s0 = chunk * s.chunk;
  int m = (int)min((int64_t)s.chunk, s.n - s0);
  for (int i = threadIdx.x; i < s.chunk + 2; i += blockDim.x) {
    const int64_t at = s0 + i - 1;
    key[i] = at >= 0 && at < s.n ? s.key[at] : -1;
    if (i < s.chunk) pos[i] = s.pos[s0 + (i < m ? i : 0)];
  }
  __syncthreads();
  const int64_t c = ((int64_t)blockIdx.y * blockDim.x + threadIdx.x) * VEC;
  while (m > 0 && key[m] >= s.V) --m;  // (tokens outside the vocabulary are sorted behind the others)
  if (c >= s.D || m == 0) return;
  const T* d = (const T*)s.dout + c;
  float acc[VEC];
#pragma unroll
  for (int j = 0; j < VEC; ++j) acc[j] = 0.f;
  bool inside = key[0] == key[1];  // the row began in an earlier chunk
  constexpr int AHEAD = 8;
  static_assert(CHUNK % AHEAD == 0 && FEW_CHUNK % AHEAD == 0, "loads in flight");
  for (int i0 = 0; i0 < m; i0 += AHEAD) {
    float v[AHEAD][VEC];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) load<T, VEC>(d + pos[i0 + u] * s.dout_stride, v[u]);  // (places behind the last hold the first one's token)
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      const int i = i0 + u;
      if (i >= m) break;
#pragma unroll
      for (int j = 0; j < VEC; ++j) acc[j] += v[u][j];
      const bool last = key[1 + i] != key[2 + i];  // the row's last token
      if (!last && i < m - 1) continue;
      if (last && !inside) finish<TO, VEC, true, ADD>(s, key[1 + i], c, acc);
      else store<float, VEC>(s.partial + (2 * chunk + (inside ? 0 : 1)) * s.D + c, acc);
#pragma unroll
      for (int j = 0; j < VEC; ++j) acc[j] = 0.f;
      inside = false;
    }
  }
}

// Chunks' sums of a row behind its first chunk's are added JOIN at a time, in pairs; zeros where there are no more.
constexpr int JOIN = 8;
__device__ __forceinline__ float joined(const float (&v)[JOIN]) { return ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7])); }

// The row that chunk blockIdx.x ends inside, if it began there: its partial sums, in order.  12 us where the most frequent of 16,384 tokens has 1300 of them, 41
// chunks; eight partial rows in flight, added in pairs.
template <typename TO, int VEC, bool ADD>
__global__ __launch_bounds__(WG) void join_kernel(Sums s) {
  const int64_t chunk = s.first + blockIdx.x, e = (chunk + 1) * s.chunk;  // (the grid leaves the last chunk out)
  const int32_t id = s.key[e - 1];
  if (id >= s.V || s.key[e] != id) return;
  if (s.key[chunk * s.chunk] == id && chunk > 0 && s.key[chunk * s.chunk - 1] == id) return;
  // the first chunk that the row does not run out of
  __shared__ int32_t found;
  int64_t end = chunk + 1;
  for (bool more = true; more; ) {
    if (threadIdx.x == 0) found = (int32_t)blockDim.x;
    __syncthreads();
    const int64_t after = (end + threadIdx.x + 1) * s.chunk;  // the place behind chunk end + threadIdx.x
    if (after >= s.n || s.key[after] != id) atomicMin(&found, (int32_t)threadIdx.x);
    __syncthreads();
    end += found;
    more = found == (int32_t)blockDim.x;
    __syncthreads();
  }
  const int64_t c = ((int64_t)blockIdx.y * blockDim.x + threadIdx.x) * VEC;
  if (c >= s.D) return;
  float acc[VEC];
  load<float, VEC>(s.partial + (2 * chunk + 1) * s.D + c, acc);
  const float* p = s.partial + 2 * (chunk + 1) * s.D + c;
  const int64_t m = end - chunk;
  for (int64_t k = 0; k < m; k += JOIN) {
    float v[JOIN][VEC];
#pragma unroll
    for (int u = 0; u < JOIN; ++u) {
#pragma unroll
      for (int j = 0; j < VEC; ++j) v[u][j] = 0.f;
      if (k + u < m) load<float, VEC>(p + 2 * (k + u) * s.D, v[u]);
    }
#pragma unroll
    for (int j = 0; j < VEC; ++j) {
      float w[JOIN];
#pragma unroll
      for (int u = 0; u < JOIN; ++u) w[u] = v[u][j];
      acc[j] += joined(w);
    }
  }
  finish<TO, VEC, true, ADD>(s, id, c, acc);
}

// Up to DIRECT tokens need no sort: the workgroup of an id's first token finds the others, and from how many tokens have lower ids where a sort would put them, and sums
// them in the same chunks and joins those in the same order as the two kernels above, so that no bit depends on which way is taken.  Chunks go to the groups of
// `blockDim.x` threads in turn (512 tokens of one id, 1024 values: 24.2 us of kernels, 20.7 with chunks counted from the row's first token and joined by groups, in an order that
// changed with the width; of 512 ids 6.7 and 6.6).  One kernel where five steps of 3 to 5 us each would wait for each other (a call with 219 tokens of
// 89 values float32 26 us sorted, 14 so; 300 and 512 of 1024 bfloat16 33 and 15).  Every token has its workgroups: no more than DIRECT_WGS, two rounds of the chip
// (512 tokens of 7172 values, 4096 workgroups: 28 us sorted, 36 so).  600 tokens of 1024 values took 18 us this way, but 46 with one id in most of them, 28 sorted.
constexpr int DIRECT = 512, DIRECT_WG = 512, DIRECT_X = 128;  // DIRECT_X: threads along a row at most
static_assert(DIRECT <= FEW, "chunks of FEW_CHUNK");
constexpr int64_t DIRECT_WGS = 2048;
template <typename T, typename TO, int VEC, bool WHOLE, bool ADD>
__global__ __launch_bounds__(DIRECT_WG) void direct_kernel(Sums s, const int32_t* ids) {
  __shared__ int32_t id[DIRECT], same[DIRECT];
  __shared__ int found, ahead;
  __shared__ float others[JOIN * VEC * DIRECT_X];
  const int t = blockIdx.x, n = (int)s.n, thread = threadIdx.y * blockDim.x + threadIdx.x;
  for (int i = thread; i < n; i += blockDim.x * blockDim.y) id[i] = ids[i];
  __syncthreads();
  const int32_t own = id[t];
  if (own < 0 || own >= s.V) return;
  if (thread < 64) {  // places of the id's tokens, in order; none if this is not its first
    int m = 0;
    for (int i0 = 0; i0 < n; i0 += 64) {
      const int i = i0 + thread;
      const bool is = i < n && id[i] == own;
      const uint64_t all = __ballot(is);
      if (m == 0 && all != 0 && i0 + __ffsll((unsigned long long)all) - 1 != t) break;
      if (is) same[m + (int)__popcll(all & ((1ull << thread) - 1ull))] = i;
      m += (int)__popcll(all);
    }
    if (thread == 0) found = m;
  } else if (thread < 128) {  // how many tokens a sort would have ahead of them
    int low = 0;
    for (int i = thread - 64; i < n; i += 64) low += (uint32_t)id[i] < (uint32_t)own;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) low += __shfl_xor(low, o, 64);
    if (thread == 64) ahead = low;
  }
  __syncthreads();
  const int m = found;
  const int64_t c = ((int64_t)blockIdx.y * blockDim.x + threadIdx.x) * VEC;
  if (m == 0) return;
  const T* d = (const T*)s.dout;
  const int64_t from = min(c, s.D - (WHOLE ? VEC : 1));
  auto sum = [&](int begin, int end, float (&acc)[VEC]) {
    constexpr int AHEAD = 8;
#pragma unroll
    for (int j = 0; j < VEC; ++j) acc[j] = 0.f;
    for (int i0 = begin; i0 < end; i0 += AHEAD) {
      float v[AHEAD][VEC];
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) load_some<T, VEC, WHOLE>(d + same[min(i0 + u, end - 1)] * s.dout_stride, from, s.D, v[u]);
#pragma unroll
      for (int u = 0; u < AHEAD; ++u)
        if (i0 + u < end) {
#pragma unroll
          for (int j = 0; j < VEC; ++j) acc[j] += v[u][j];
        }
    }
  };
  // The row's first chunk ends where a sort's would.  JOIN of those behind it at a time, by groups in turn, the first group last.
  const int first = min(m, s.chunk - (ahead & (s.chunk - 1))), groups = blockDim.y, group = (threadIdx.y - 1) & (groups - 1);
  float acc[VEC];
  if (threadIdx.y == 0) sum(0, first, acc);
  for (int k0 = first; k0 < m; k0 += JOIN * s.chunk) {
    for (int u = group; u < JOIN; u += groups) {
      float v[VEC];
      const int begin = k0 + u * s.chunk;
      sum(begin, min(begin + s.chunk, m), v);
#pragma unroll
      for (int j = 0; j < VEC; ++j) others[(u * VEC + j) * DIRECT_X + threadIdx.x] = v[j];
    }
    __syncthreads();
    if (threadIdx.y == 0) {
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        float v[JOIN];
#pragma unroll
        for (int u = 0; u < JOIN; ++u) v[u] = others[(u * VEC + j) * DIRECT_X + threadIdx.x];
        acc[j] += joined(v);
      }
    }
    __syncthreads();
  }
  if (threadIdx.y == 0 && c < s.D) finish<TO, VEC, WHOLE, ADD>(s, own, c, acc);
}

struct Layout { int64_t key[2], pos[2], counts, partial, total; int tiles, passes, chunk; };
Layout layout(int64_t T, int64_t V, int64_t D) {
  Layout L{};
  auto take = [&](int64_t bytes) { const int64_t at = L.total; L.total += (bytes + 255) & ~(int64_t)255; return at; };
  L.tiles = (int)ceil_div(T, TILE);
  L.passes = 1;
  while ((V >> (L.passes * BITS)) != 0) ++L.passes;
  for (int i = 0; i < 2; ++i) { L.key[i] = take(T * 4); L.pos[i] = take(T * 4); }
  L.counts = take((int64_t)L.tiles * BINS * 4);
  L.chunk = T <= FEW ? FEW_CHUNK : CHUNK;
  L.partial = take(ceil_div(T, L.chunk) * 2 * D * 4);
  return L;
}

}  // namespace embed
}  // namespace simple

using namespace simple::embed;

namespace {
int check_sizes(int64_t T, int64_t V, int64_t D, int dtype) {
  if (T < 0 || V <= 0 || D <= 0 || !good_type(dtype)) return SIMPLE_EINVAL;
  if (T > (int64_t)0x7FFFFFFF || V >= (int64_t)0x7FFFFFFF || D > ((int64_t)1 << 22)) return SIMPLE_ECAPACITY;
  return SIMPLE_OK;
}
int shape_of(int64_t units) {  // threads along a row
  int x = 8;
  while (x < WG && x < units) x *= 2;
  return x;
}
}  // namespace

extern "C" int simple_embed(const int32_t* ids_dev, const void* table_dev, int64_t table_stride, int64_t T, int64_t V, int64_t D, int dtype,
                            float scale, void* out_dev, int64_t out_stride, void* hip_stream) {
  const int rc = check_sizes(T, V, D, dtype);
  if (rc != SIMPLE_OK) return rc;
  if (table_stride < D || out_stride < D) return SIMPLE_EINVAL;
  if (T == 0) return SIMPLE_OK;
  if (!ids_dev || !table_dev || !out_dev) return SIMPLE_EINVAL;
  const int64_t e = type_bytes(dtype);
  const bool wide = D % (16 / e) == 0 && rows_aligned(table_dev, table_stride, e, 16) && rows_aligned(out_dev, out_stride, e, 16);
  // (rows that are not aligned: bfloat16 by unaligned loads, 19 us for 8192 rows of 2047 values against 26 by single elements)
  const int64_t units = wide || dtype == SIMPLE_BF16 ? ceil_div(D, 16 / e) : D;
  const int x = shape_of(units), y = WG / x;
  if (ceil_div(units, x) > 65535) return SIMPLE_ECAPACITY;
  auto go = [&](auto kernel, auto* type) {
    using T_ = std::remove_pointer_t<decltype(type)>;
    const int64_t most = LAUNCH_WGS * y * RD;
    for (int64_t t0 = 0; t0 < T; t0 += most) {
      const int64_t n = std::min(most, T - t0);
      hipLaunchKernelGGL(kernel, dim3((unsigned)ceil_div(n, (int64_t)y * RD), (unsigned)ceil_div(units, x)), dim3(x, y), 0, (hipStream_t)hip_stream, ids_dev + t0,
                         (const T_*)table_dev, table_stride, n, V, D, scale, (T_*)out_dev + t0 * out_stride, out_stride);
    }
  };
  if (dtype == SIMPLE_F32) { if (wide) go(lookup_kernel<float, 4, true>, (float*)0); else go(lookup_kernel<float, 1, true>, (float*)0); }
  else { if (wide) go(lookup_kernel<uint16_t, 8, true>, (uint16_t*)0); else go(lookup_kernel<uint16_t, 8, false>, (uint16_t*)0); }
  return launched();
}

extern "C" int64_t simple_embed_grad_workspace(int64_t T, int64_t V, int64_t D) {
  const int rc = check_sizes(T, V, D, SIMPLE_F32);
  return rc != SIMPLE_OK ? rc : layout(T, V, D).total;
}

extern "C" int simple_embed_grad(const int32_t* ids_dev, const void* dout_dev, int64_t dout_stride, int64_t T, int64_t V, int64_t D, int dtype,
                                 float scale, void* dtable_dev, int64_t dtable_stride, int table_dtype, int accumulate,
                                 void* workspace_dev, int64_t workspace_bytes, void* hip_stream) {
  const int rc = check_sizes(T, V, D, dtype);
  if (rc != SIMPLE_OK) return rc;
  if (!good_type(table_dtype) || !dtable_dev || dtable_stride < D || dout_stride < D) return SIMPLE_EINVAL;
  if (T == 0 && accumulate) return SIMPLE_OK;
  const Layout L = layout(T, V, D);
  if (T > 0) {
    if (!ids_dev || !dout_dev || !workspace_dev || ((uintptr_t)workspace_dev & 15u) != 0) return SIMPLE_EINVAL;
    if (workspace_bytes < L.total) return SIMPLE_ECAPACITY;
  }
  hipStream_t st = (hipStream_t)hip_stream;
  unsigned char* ws = (unsigned char*)workspace_dev;
  const int64_t eo = type_bytes(table_dtype), ei = type_bytes(dtype);
  // groups of 8 bfloat16 or 4 float32, by the wider of the two types
  const int64_t vec = dtype == SIMPLE_BF16 && table_dtype == SIMPLE_BF16 ? 8 : 4;
  const bool wide = D % vec == 0 && rows_aligned(dout_dev, dout_stride, ei, std::min<int64_t>(16, vec * ei)) &&
                    rows_aligned(dtable_dev, dtable_stride, eo, std::min<int64_t>(16, vec * eo));
  const int few_x = std::max(64, std::min(DIRECT_X, shape_of(ceil_div(D, vec))));
  const dim3 few((unsigned)T, (unsigned)ceil_div(ceil_div(D, vec), few_x));
  const bool no_sort = T <= DIRECT && T * few.y <= DIRECT_WGS;
  Sort s{ids_dev, nullptr, (int32_t*)(ws + L.key[0]), (int32_t*)(ws + L.pos[0]), (int32_t*)(ws + L.counts), T, V, L.tiles, 0};
  Fill zeros{(unsigned char*)dtable_dev, V, D * eo, dtable_stride * eo, 0};
  auto zeros_alone = [&](int64_t shares, int threads) {  // from share zeros.first on
    Sort none = s;
    none.n = 0;
    for (; shares > 0; shares -= LAUNCH_WGS, zeros.first += LAUNCH_WGS)
      hipLaunchKernelGGL(sort_few_kernel, dim3((unsigned)std::min(shares, LAUNCH_WGS)), dim3(threads), 0, st, none, 0, zeros);
  };
  if (no_sort) {
    if (!accumulate) zeros_alone(fill_workgroups(zeros, FEW_WG), FEW_WG);
  } else if (T <= FEW) {
    const int64_t all = accumulate ? 0 : fill_workgroups(zeros, FEW_WG), shares = std::min(all, LAUNCH_WGS);
    hipLaunchKernelGGL(sort_few_kernel, dim3((unsigned)(shares + 1)), dim3(FEW_WG), 0, st, s, L.passes, zeros);
    zeros.first = shares;
    zeros_alone(all - shares, FEW_WG);
    s.key_in = s.key_out; s.pos_in = s.pos_out;
  } else {
    const int kernels = 2 * L.passes;
    const int64_t all = accumulate ? 0 : fill_workgroups(zeros, WG), shares = std::min(all, kernels * LAUNCH_WGS);
    int kernel = 0;
    auto beside = [&](auto* f) {  // the kernel's share of the zeros, behind its own workgroups
      zeros.first = shares * kernel / kernels;
      const int64_t n = shares * (kernel + 1) / kernels - zeros.first;
      ++kernel;
      hipLaunchKernelGGL(f, dim3((unsigned)(L.tiles + n)), dim3(WG), 0, st, s, zeros);
    };
    for (int p = 0; p < L.passes; ++p) {
      beside(count_kernel);
      beside(place_kernel);
      s.key_in = s.key_out; s.pos_in = s.pos_out;
      s.key_out = (int32_t*)(ws + L.key[(p + 1) & 1]); s.pos_out = (int32_t*)(ws + L.pos[(p + 1) & 1]);
      s.shift += BITS;
    }
    zeros.first = shares;
    zeros_alone(all - shares, WG);
  }
  if (T == 0) return launched();
  Sums m{s.key_in, s.pos_in, dout_dev, dout_stride, T, V, D, scale, dtable_dev, dtable_stride, L.chunk, 0, (float*)(ws + L.partial)};
  const int64_t units = wide ? D / vec : D, chunks = ceil_div(T, L.chunk);
  const int x = std::max(64, shape_of(units));
  const unsigned across = (unsigned)ceil_div(units, x);
  auto go = [&](auto in, auto out, auto group, auto whole, auto add) {
    using I = decltype(in);
    using O = decltype(out);
    constexpr int N = decltype(group)::value;
    constexpr bool W = decltype(whole)::value, A = decltype(add)::value;
    if (no_sort) {
      hipLaunchKernelGGL((direct_kernel<I, O, N, W, A>), few, dim3(few_x, DIRECT_WG / few_x), 0, st, m, ids_dev);
      return;
    }
    constexpr int S = W ? N : 1;
    for (m.first = 0; m.first < chunks; m.first += LAUNCH_WGS)
      hipLaunchKernelGGL((sums_kernel<I, O, S, A>), dim3((unsigned)std::min(LAUNCH_WGS, chunks - m.first), across), dim3(x), 0, st, m);
    for (m.first = 0; m.first < chunks - 1; m.first += LAUNCH_WGS)
      hipLaunchKernelGGL((join_kernel<O, S, A>), dim3((unsigned)std::min(LAUNCH_WGS, chunks - 1 - m.first), across), dim3(x), 0, st, m);
  };
  auto typed = [&](auto in, auto out, auto group) {
    auto added = [&](auto whole) {
      if (accumulate) go(in, out, group, whole, std::true_type{});
      else go(in, out, group, whole, std::false_type{});
    };
    if (wide) added(std::true_type{});
    else added(std::false_type{});
  };
  const std::integral_constant<int, 8> eight;
  const std::integral_constant<int, 4> four;
  if (dtype == SIMPLE_BF16 && table_dtype == SIMPLE_BF16) typed((uint16_t)0, (uint16_t)0, eight);
  else if (dtype == SIMPLE_BF16) typed((uint16_t)0, 0.f, four);
  else if (table_dtype == SIMPLE_BF16) typed(0.f, (uint16_t)0, four);
  else typed(0.f, 0.f, four);
  return launched();
}
