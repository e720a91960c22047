// Matrix products out[p, q] = sum_k P[p, k] * Q[q, k] on the matrix cores: both operands row-major with k along the rows, of 16-bit
// floating or 8-bit integer elements.  The kernels of the 8-bit head and of the cross entropy are made of this with
// what they do to a finished tile.
//
// A workgroup forms a BP x BQ tile.  Rows are staged through LDS 128 bytes of k at a time; a fragment of 16 rows and 64 bytes
// of k is one 16-byte read a lane whatever the element is, and feeds one 16x16 instruction (32 k of bfloat16, 64 of int8).
// A row's 16-byte chunks are stored in the order chunk ^ (row & 7), so that the 16 rows of a fragment spread over all banks.
#pragma once
#include "simple_vocabdev.hpp"

namespace simple {
namespace tiles {

using namespace vocab;

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int i32x4 __attribute__((ext_vector_type(4)));

struct Bf16 {
  using Acc = f32x4;
  static constexpr int BYTES = 2;
  static __device__ __forceinline__ Acc mma(i32x4 a, i32x4 b, Acc c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  }
};
struct F16 {
  using Acc = f32x4;
  static constexpr int BYTES = 2;
  static __device__ __forceinline__ Acc mma(i32x4 a, i32x4 b, Acc c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  }
};
struct Int8 {
  using Acc = i32x4;
  static constexpr int BYTES = 1;
  static __device__ __forceinline__ Acc mma(i32x4 a, i32x4 b, Acc c) { return __builtin_amdgcn_mfma_i32_16x16x64_i8(a, b, c, 0, 0, 0); }
};

constexpr int KB = 128;  // bytes of k a step

// One operand: `rows` rows of `k_bytes` bytes, `stride` bytes apart.
struct Operand {
  const unsigned char* p;
  int64_t stride, rows;
};

// ---- staging by the memory system itself: 16 bytes a lane go from memory to LDS without a register ----
// The wave's 64 lanes write 1 KB from `lds` on in lane order: 8 rows of a step.  Nothing here is seen by the compiler's own count of loads
// in flight; arrived() below waits for them, and no register is written but m0, which the compiler keeps out of all allocation (named among the asm's it is
// refused) and which nothing else in these kernels uses.
__device__ __forceinline__ void to_lds(uint32_t lds, uint32_t offset, i32x4 resource, uint32_t k) {
  // (scalar operands, whatever register the optimiser has kept them in)
  lds = (uint32_t)__builtin_amdgcn_readfirstlane((int)lds);
  k = (uint32_t)__builtin_amdgcn_readfirstlane((int)k);
  resource = i32x4{__builtin_amdgcn_readfirstlane(resource.x), __builtin_amdgcn_readfirstlane(resource.y), __builtin_amdgcn_readfirstlane(resource.z),
                   __builtin_amdgcn_readfirstlane(resource.w)};
  asm volatile("s_mov_b32 m0, %0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" ::"s"(lds), "v"(offset), "s"(resource), "s"(k) : "memory");
}
// All but the `N` newest of this wave's loads have arrived, and those of the workgroup's other waves; what the waves read of LDS before is in
// their registers.
template <int N> __device__ __forceinline__ void arrived() {
  static_assert(N < 64, "six bits");
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}
// A buffer resource over the operand's rows from `row0` on, at most `n` of them.  Addresses behind its end read as zeros.
__device__ __forceinline__ i32x4 resource_of(const Operand& o, int64_t row0, int n, int k_bytes) {
  const int64_t left = o.rows - row0;
  const uint32_t m = (uint32_t)(left < n ? left : n);
  const uint64_t a = (uint64_t)(uintptr_t)(o.p + row0 * o.stride);
  i32x4 r;
  r.x = __builtin_amdgcn_readfirstlane((int)(uint32_t)a);
  r.y = __builtin_amdgcn_readfirstlane((int)(uint32_t)(a >> 32) & 0xFFFF);
  r.z = __builtin_amdgcn_readfirstlane((int)((m - 1) * (uint32_t)o.stride + (uint32_t)k_bytes));
  r.w = 0x00020000;
  return r;
}


// The lane, hidden from the optimiser, which would otherwise keep what follows from it in registers through the products.
__device__ __forceinline__ int opaque_lane() {
  int lane = threadIdx.x & 63;
  asm volatile("" : "+v"(lane));
  return lane;
}

// A workgroup's tile, its waves (NWP along P times NWQ along Q), and how many steps are staged at once.
template <class E_, int BP_, int BQ_, int NWP_, int NWQ_, int STAGES_> struct Shape {
  using E = E_;
  using Acc = typename E::Acc;
  static constexpr int BP = BP_, BQ = BQ_, NWP = NWP_, NWQ = NWQ_, NW = NWP * NWQ, THREADS = 64 * NW, STAGES = STAGES_;
  static constexpr int FP = BP / NWP / 16, FQ = BQ / NWQ / 16;                     // fragments a wave
  static constexpr int GP = BP / 8, GQ = BQ / 8;                                   // groups of 8 rows, one load instruction each
  static constexpr int LP = (GP + NW - 1) / NW, LQ = (GQ + NW - 1) / NW;           // loads a wave and step (more waves than groups: twice the same)
  static constexpr int STAGE = (BP + BQ) * KB, LDS = STAGE * STAGES;
  static_assert(FP * NWP * 16 == BP && FQ * NWQ * 16 == BQ && LDS <= 160 * 1024, "shape");
};

// The order of `np * nq` tiles.  Workgroups go to the eight XCDs in turn, each with an L2 of its own: an XCD gets consecutive places of an order in
// which GROUP tiles along P share their Q rows, so that what its 32 compute units read at a time is few rows of both.
constexpr int XCDS = 8, GROUP = 8, CUS = 256;
__device__ __forceinline__ void tile_at(int at, int np, int nq, int& p, int& q) {
  const int g = at / (GROUP * nq), first = g * GROUP, size = min(GROUP, np - first), r = at - first * nq;
  p = first + r % size;
  q = r / size;
}
__device__ __forceinline__ int place_of(int id, int n) {
  const int per = n / XCDS, more = n % XCDS, x = id % XCDS;
  return x * per + min(x, more) + id / XCDS;
}

// Tiles of 256 x 256 have a compute unit each: with MANY, as many workgroups as there are take them in rounds, one after the other, so that a workgroup's loads run
// on from a tile to the next while the finished one is stored.  (Smaller tiles, several of them on a compute unit, are left to the dispatcher, one a
// workgroup: taken in rounds, one token against 128,256 x 4096 int8 weights took 117 us, 92 so.)  Tiles of a last round that is at most a quarter full are cut in
// four along P instead, eight waves to each part, a workgroup to each: the round then takes about 0.35 of a whole one.
template <typename T> __device__ __forceinline__ void arrived_value(T& v) { asm volatile("" : "+v"(v)); }
template <class S> struct Cut {
  static constexpr bool CAN = S::BP == 256 && S::BQ == 256;
  using Part = Shape<typename S::E, CAN ? 64 : S::BP, S::BQ, CAN ? 1 : S::NWP, CAN ? 8 : S::NWQ, S::STAGES>;
};
struct Plan { int np, nq, whole, wgs, grid; };  // whole tiles, workgroups that take them, and workgroups in all
template <class S, bool MANY> inline Plan plan(int64_t p_rows, int64_t q_rows, bool may_cut = true) {
  Plan r{(int)ceil_div(p_rows, S::BP), (int)ceil_div(q_rows, S::BQ), 0, 0, 0};
  const int n = r.np * r.nq, last = n % CUS, slots = MANY ? CUS : n;
  const bool cut = may_cut && Cut<S>::CAN && last > 0 && last * 4 <= CUS;
  r.whole = cut ? n - last : n;
  r.wgs = r.whole < slots ? r.whole : slots;
  r.grid = r.wgs + (n - r.whole) * 4;
  return r;
}

// 16 bytes of a row from byte `k` on, zeros behind its end; any alignment.  A row's last bytes come from the 16 that end with it.  In two parts, so
// that what is loaded is not looked at before it is wanted: taken_from() makes of the loaded what it stands for.
typedef unsigned __int128 u128;
template <int BYTES> __device__ __forceinline__ u128 chunk_at(const unsigned char* row, int k, int k_bytes) {
  u128 v = 0;
  if (k_bytes >= 16) {
    __builtin_memcpy(&v, row + min(k, k_bytes - 16), 16);
  } else if (k == 0) {
#pragma unroll
    for (int i = 0; i < 16; i += BYTES)
      if (i < k_bytes) v |= (u128)(BYTES == 1 ? (uint32_t)row[i] : (uint32_t)*reinterpret_cast<const uint16_t*>(row + i)) << (8 * i);
  }
  return v;
}
__device__ __forceinline__ i32x4 taken_from(u128 v, int k, int k_bytes) {
  const int over = k + 16 - max(k_bytes, 16);  // bytes of the chunk behind the row's end
  if (over > 0) v = over < 16 ? v >> (8 * over) : 0;
  return __builtin_bit_cast(i32x4, v);
}

// Rows of a tile on their way to LDS by to_lds().  Rows behind an operand's last repeat it (what they give is not stored).
template <class S> struct Loader {
  i32x4 res_p, res_q;
  uint32_t off_p[S::LP], off_q[S::LQ];
  int wave;
  __device__ __forceinline__ void to(const Operand& P, const Operand& Q, int64_t p0, int64_t q0, int k_bytes) {
    const int lane = opaque_lane(), row8 = lane >> 3, chunk = (lane & 7) ^ row8;  // what a lane stages of its group of 8 rows
    res_p = resource_of(P, p0, S::BP, k_bytes);
    res_q = resource_of(Q, q0, S::BQ, k_bytes);
    const int p_rows = (int)min((int64_t)S::BP, P.rows - p0), q_rows = (int)min((int64_t)S::BQ, Q.rows - q0);
#pragma unroll
    for (int i = 0; i < S::LP; ++i) off_p[i] = (uint32_t)min((wave + i * S::NW) % S::GP * 8 + row8, p_rows - 1) * (uint32_t)P.stride + chunk * 16;
#pragma unroll
    for (int i = 0; i < S::LQ; ++i) off_q[i] = (uint32_t)min((wave + i * S::NW) % S::GQ * 8 + row8, q_rows - 1) * (uint32_t)Q.stride + chunk * 16;
  }
  // Ahead of the last step's loads: chunks behind the rows' end go behind the resources' end, which reads as zeros.
  __device__ __forceinline__ void end_at(int left) {
    const int lane = opaque_lane(), chunk = (lane & 7) ^ (lane >> 3);
    if (chunk * 16 >= left) {
#pragma unroll
      for (int i = 0; i < S::LP; ++i) off_p[i] = 0x80000000u;
#pragma unroll
      for (int i = 0; i < S::LQ; ++i) off_q[i] = 0x80000000u;
    }
  }
  // load n of step s: the LP of P, then the LQ of Q
  __device__ __forceinline__ void load(int s, uint32_t stage, int n) const {
    const uint32_t k = (uint32_t)s * KB;
    if (n < S::LP) to_lds(stage + (wave + n * S::NW) % S::GP * 1024, off_p[n], res_p, k);
    else to_lds(stage + S::BP * KB + (wave + (n - S::LP) * S::NW) % S::GQ * 1024, off_q[n - S::LP], res_q, k);
  }
};

// Forms tiles `tile(0)`, `tile(1)`, ... (which says whether there is one, and where; the first alone without MANY) and calls done(acc, p0, q0) for each.
// With MANY the products come after done()'s code in a loop: a value that done() loads is to be used on each of its paths (arrived_value), or the
// compiler waits for every load in flight when it gives the register to the products.
// acc[i][j] of a lane: rows q0 + (wave along Q * FQ + i) * 16 + (lane >> 4) * 4 + 0..3 of Q against row p0 + (wave along P * FP + j) * 16 + (lane & 15) of P.
// DIRECT: rows are staged by to_lds(), which wants them 16-byte aligned with k_bytes a multiple of 16; else through registers,
// any alignment.  `lds` are S::LDS bytes; done() must not write them with MANY, and without only behind a barrier of its own.
template <class S, bool DIRECT, bool MANY, typename Tile, typename Done>
__device__ __forceinline__ void products(const Operand& P, const Operand& Q, int k_bytes, unsigned char* lds, Tile&& tile, Done&& done) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wp = wave % S::NWP, wq = wave / S::NWP;
  const int steps = (k_bytes + KB - 1) / KB;
  typename S::Acc acc[S::FQ][S::FP];
  auto clear = [&] {
#pragma unroll
    for (int i = 0; i < S::FQ; ++i)
#pragma unroll
      for (int j = 0; j < S::FP; ++j) acc[i][j] = typename S::Acc{0, 0, 0, 0};
  };
  uint32_t at_p[2], at_q[2];  // the lane's place in the first fragment, for both halves of a step
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const uint32_t c = (uint32_t)((h * 4 + (lane >> 4)) ^ (lane & 7)) * 16;
    at_p[h] = (wp * S::FP * 16 + (lane & 15)) * KB + c;
    at_q[h] = S::BP * KB + (wq * S::FQ * 16 + (lane & 15)) * KB + c;
  }
  // fragment n of half h of a stage: the FP of P, then the FQ of Q
  auto read = [&](int stage, int h, int n, i32x4 (&fp)[S::FP], i32x4 (&fq)[S::FQ]) {
    const unsigned char* b = lds + stage * S::STAGE;
    if (n < S::FP) fp[n] = *reinterpret_cast<const i32x4*>(b + at_p[h] + n * 16 * KB);
    else fq[n - S::FP] = *reinterpret_cast<const i32x4*>(b + at_q[h] + (n - S::FP) * 16 * KB);
  };
  auto step = [&](int stage) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      i32x4 fp[S::FP], fq[S::FQ];
#pragma unroll
      for (int n = 0; n < S::FP + S::FQ; ++n) read(stage, h, n, fp, fq);
#pragma unroll
      for (int i = 0; i < S::FQ; ++i)
#pragma unroll
        for (int j = 0; j < S::FP; ++j) acc[i][j] = S::E::mma(fq[i], fp[j], acc[i][j]);
    }
  };
  int64_t p0, q0;
  if (steps == 0) {
    for (int n = 0; tile(n, p0, q0); ++n) {
      clear();
      done(acc, p0, q0);
      if constexpr (!MANY) break;
    }
    return;
  }
  if constexpr (DIRECT) {
    const uint32_t base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)lds;
    constexpr int NL = S::LP + S::LQ;
    // the step that is loaded next: step ls of tile lt, if there is one
    Loader<S> from;
    from.wave = wave;
    int lt = 0, ls = 0;
    bool more;
    const int left = k_bytes - (steps - 1) * KB;  // bytes of the last step
    {
      int64_t lp, lq;
      more = tile(0, lp, lq);
      if (!more) return;
      from.to(P, Q, lp, lq, k_bytes);
      if (steps == 1 && left < KB) from.end_at(left);
    }
    auto onward = [&] {
      if (++ls == steps) {
        more = false;
        if constexpr (MANY) {
          ls = 0;
          int64_t lp, lq;
          more = tile(++lt, lp, lq);
          if (more) from.to(P, Q, lp, lq, k_bytes);
        }
      }
      if (ls == steps - 1 && left < KB && more) from.end_at(left);
    };
    auto issue = [&](int stage) {
#pragma unroll
      for (int n = 0; n < NL; ++n) from.load(ls, base + stage * S::STAGE, n);
      onward();
    };
    if constexpr (S::STAGES == 2) {
      // Bound by the matrix instructions.  A half's fragments are read while the half before is multiplied, and the barrier stands in the middle of a
      // step: there all of its fragments are in registers, the stage is free, and the step after has arrived.  Loads go out
      // one at a time between groups of products: eight in a row fill the memory pipeline's queue, and the wave waits there with its products (bfloat16
      // 8192 x 128,256 x 4096: 1.34 PFLOP/s so, 1.26 with the loads in front, 1.24 with neither).
      constexpr int NF = S::FP + S::FQ, NM = S::FP * S::FQ, GROUPS = 8, MG = NM / GROUPS, RG = GROUPS - 2;
      static_assert(NM % GROUPS == 0, "groups");
      i32x4 fp0[S::FP], fq0[S::FQ], fp1[S::FP], fq1[S::FQ];
      auto half = [&](i32x4 (&fp)[S::FP], i32x4 (&fq)[S::FQ], bool next, int stage, int h, i32x4 (&np)[S::FP], i32x4 (&nq)[S::FQ], bool ahead, uint32_t to) {
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) {
          if (next) {
#pragma unroll
            for (int n = g * NF / RG; n < min(NF, (g + 1) * NF / RG); ++n) read(stage, h, n, np, nq);
          }
          if (ahead) {
#pragma unroll
            for (int n = g * NL / GROUPS; n < (g + 1) * NL / GROUPS; ++n) from.load(ls, to, n);
          }
#pragma unroll
          for (int m = g * MG; m < (g + 1) * MG; ++m) acc[m / S::FP][m % S::FP] = S::E::mma(fq[m / S::FP], fp[m % S::FP], acc[m / S::FP][m % S::FP]);
          __builtin_amdgcn_sched_barrier(0);
        }
      };
      issue(0);
      const bool two = more;
      if (two) { issue(1); arrived<NL>(); }
      else arrived<0>();
      int stage = 0;
      for (int n = 0; tile(n, p0, q0); ++n) {
        clear();
#pragma unroll
        for (int f = 0; f < NF; ++f) read(stage, 0, f, fp0, fq0);
        for (int s = 0; s < steps; ++s) {
          half(fp0, fq0, true, stage, 1, fp1, fq1, false, 0);
          arrived<0>();
          __builtin_amdgcn_sched_barrier(0);
          const bool ahead = more;
          half(fp1, fq1, s + 1 < steps, stage ^ 1, 0, fp0, fq0, ahead, base + stage * S::STAGE);
          if (ahead) onward();
          stage ^= 1;
        }
        done(acc, p0, q0);
        if constexpr (!MANY) break;
      }
    } else {
      // Bound by memory: more stages, all of a step's loads at once.
      int in_flight = 0;  // steps loaded and not yet multiplied
      for (; in_flight < S::STAGES - 1 && more; ++in_flight) issue(in_flight);
      int stage = 0;
      for (int n = 0; tile(n, p0, q0); ++n) {
        clear();
        for (int s = 0; s < steps; ++s) {
          // the newest loads in flight are those of the steps behind this one
          if (in_flight == S::STAGES - 1) arrived<(S::STAGES - 2) * NL>();
          else arrived<0>();
          if (more) issue(stage == 0 ? S::STAGES - 1 : stage - 1);  // the stage of the step before: read by all
          else --in_flight;
          step(stage);
          stage = stage + 1 == S::STAGES ? 0 : stage + 1;
        }
        done(acc, p0, q0);
        if constexpr (!MANY) break;
      }
    }
  } else {
    const int row8 = lane >> 3, chunk = (lane & 7) ^ row8;  // what a lane stages of its group of 8 rows
    for (int n = 0; tile(n, p0, q0); ++n) {
      const int p_rows = (int)min((int64_t)S::BP, P.rows - p0), q_rows = (int)min((int64_t)S::BQ, Q.rows - q0);
      const unsigned char *row_p[S::LP], *row_q[S::LQ];
#pragma unroll
      for (int i = 0; i < S::LP; ++i) row_p[i] = P.p + (p0 + min((wave + i * S::NW) % S::GP * 8 + row8, p_rows - 1)) * P.stride;
#pragma unroll
      for (int i = 0; i < S::LQ; ++i) row_q[i] = Q.p + (q0 + min((wave + i * S::NW) % S::GQ * 8 + row8, q_rows - 1)) * Q.stride;
      // AHEAD steps in registers: as many in flight as the direct stages have where the memory is what bounds
      constexpr int AHEAD = S::STAGES > 2 ? S::STAGES - 1 : S::BP * S::BQ <= 128 * 128 ? 2 : 1, NL = S::LP + S::LQ;
      u128 v[AHEAD][NL];
      auto fetch = [&](int s, u128 (&x)[NL]) {
        const int k = s * KB + chunk * 16;
#pragma unroll
        for (int i = 0; i < S::LP; ++i) x[i] = chunk_at<S::E::BYTES>(row_p[i], k, k_bytes);
#pragma unroll
        for (int i = 0; i < S::LQ; ++i) x[S::LP + i] = chunk_at<S::E::BYTES>(row_q[i], k, k_bytes);
      };
      auto put = [&](int s, const u128 (&x)[NL]) {
        const int k = s * KB + chunk * 16;
        unsigned char* b = lds + (s & 1) * S::STAGE + lane * 16;
#pragma unroll
        for (int i = 0; i < S::LP; ++i) *reinterpret_cast<i32x4*>(b + (wave + i * S::NW) % S::GP * 1024) = taken_from(x[i], k, k_bytes);
#pragma unroll
        for (int i = 0; i < S::LQ; ++i) *reinterpret_cast<i32x4*>(b + S::BP * KB + (wave + i * S::NW) % S::GQ * 1024) = taken_from(x[S::LP + i], k, k_bytes);
      };
      clear();
#pragma unroll
      for (int u = 0; u < AHEAD; ++u)
        if (u < steps) fetch(u, v[u]);
      for (int s0 = 0; s0 < steps; s0 += AHEAD) {
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
          const int s = s0 + u;
          if (s < steps) {
            put(s, v[u]);  // read last two steps ago, ahead of the barrier of the step before
            if (s + AHEAD < steps) fetch(s + AHEAD, v[u]);
            __syncthreads();
            step(s & 1);
          }
        }
      }
      __syncthreads();  // (the next tile's first step, or done())
      done(acc, p0, q0);
      if constexpr (!MANY) break;
    }
  }
}

// A workgroup's share of the plan: its tiles in rounds, or one part of a cut tile.  done(shape, acc, p0, q0).
template <class S, bool DIRECT, bool MANY, typename Done>
__device__ __forceinline__ void planned(const Operand& P, const Operand& Q, int k_bytes, const Plan& r, unsigned char* lds, Done&& done) {
  if constexpr (Cut<S>::CAN) {
    using Part = typename Cut<S>::Part;
    if ((int)blockIdx.x >= r.wgs) {
      const int i = place_of((int)blockIdx.x - r.wgs, r.grid - r.wgs);
      products<Part, DIRECT, false>(P, Q, k_bytes, lds, [&](int n, int64_t& p0, int64_t& q0) {
        int p, q;
        tile_at(r.whole + i / 4, r.np, r.nq, p, q);
        p0 = (int64_t)p * S::BP + i % 4 * Part::BP;
        q0 = (int64_t)q * S::BQ;
        return n == 0 && p0 < P.rows;
      }, [&](auto& acc, int64_t p0, int64_t q0) { done(Part{}, acc, p0, q0); });
      return;
    }
  }
  products<S, DIRECT, MANY>(P, Q, k_bytes, lds, [&](int n, int64_t& p0, int64_t& q0) {
    const int first = n * r.wgs, count = min(r.wgs, r.whole - first);
    if ((int)blockIdx.x >= count) return false;
    int p, q;
    tile_at(first + place_of((int)blockIdx.x, count), r.np, r.nq, p, q);
    p0 = (int64_t)p * S::BP;
    q0 = (int64_t)q * S::BQ;
    return true;
  }, [&](auto& acc, int64_t p0, int64_t q0) { done(S{}, acc, p0, q0); });
}

// Shapes by the number of P's rows.  Few read every row of Q once, in three or four stages that keep the memory busy (64 rows against 128,256 x 4096 bfloat16:
// 180 us in tiles of 64 x 128, 208 in those of 64 x 64).  Many run at the matrix rate, in the tiles that
// take fewer rounds: one of 256 x 256 a compute unit, or two of 128 x 128, at 0.8 of the rate (256 tokens x 32,000 x 4096 int8: 125 of the one kind
// leave half of the chip idle).
enum { TILE_16, TILE_32, TILE_64, TILE_128, TILE_256 };
inline int tiles_for(int64_t p, int64_t q) {
  if (p <= 16) return TILE_16;
  if (p <= 32) return TILE_32;
  if (p <= 64) return TILE_64;
  if (p <= 128) return TILE_128;
  const int64_t large = ceil_div(p, 256) * ceil_div(q, 256), small = ceil_div(p, 128) * ceil_div(q, 128), last = large % CUS;
  const double rounds = (double)(large / CUS) + (last == 0 ? 0.0 : last * 4 <= CUS ? 0.35 : 1.0);
  return rounds <= 0.625 * (double)ceil_div(small, 2 * CUS) ? TILE_256 : TILE_128;
}
inline int64_t tile_rows(int tiles) { return (int64_t)16 << (tiles - TILE_16); }
inline int64_t tile_columns(int tiles) { return tiles <= TILE_32 ? 64 : tiles <= TILE_128 ? 128 : 256; }
template <class E, typename F> void shaped(int tiles, F&& f) {
  if (tiles == TILE_16) f(Shape<E, 16, 64, 1, 4, 4>{});
  else if (tiles == TILE_32) f(Shape<E, 32, 64, 1, 4, 4>{});
  else if (tiles == TILE_64) f(Shape<E, 64, 128, 1, 4, 3>{});
  else if (tiles == TILE_128) f(Shape<E, 128, 128, 2, 2, 2>{});
  else f(Shape<E, 256, 256, 2, 4, 2>{});
}

// Rows of any alignment, copied to rows of `out_stride` bytes (a multiple of 16), zeros behind their end.  Many tokens read a weight
// row often, few do not repay the copy: scored against 50,001 x 1023 bfloat16 2000 tokens take 234 us with copies and 286 without, 1000 147 and 160; against
// 100,000 x 1023 512 take 188 and 178, 256 150 and 112; of the 8-bit head's 100,000 x 2047 1000 take 299 and 353, 500 197 and 195, 200 149 and 118.
constexpr int64_t FEW_TOKENS = 512;
constexpr int64_t ALIGN_ROWS = 65536;  // weights at a time
template <int BYTES> __global__ __launch_bounds__(256) void align_kernel(const unsigned char* in, int64_t stride, int64_t rows, int64_t bytes, unsigned char* out,
                                                                         int64_t out_stride) {
  const int64_t chunks = out_stride / 16, c = (int64_t)blockIdx.y * blockDim.x + threadIdx.x;
  if (c >= chunks) return;
  const int64_t r0 = (int64_t)blockIdx.x * (blockDim.y * 4) + threadIdx.y;
  u128 v[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) v[k] = chunk_at<BYTES>(in + min(r0 + k * blockDim.y, rows - 1) * stride, (int)c * 16, (int)bytes);
#pragma unroll
  for (int k = 0; k < 4; ++k)
    if (r0 + k * blockDim.y < rows) *reinterpret_cast<i32x4*>(out + (r0 + k * blockDim.y) * out_stride + c * 16) = taken_from(v[k], (int)c * 16, (int)bytes);
}
inline int64_t aligned_stride(int64_t k_bytes) { return ceil_div(k_bytes, 16) * 16; }
template <int BYTES> inline Operand aligned_copy(const Operand& o, int64_t k_bytes, unsigned char* to, hipStream_t st) {
  const int64_t stride = aligned_stride(k_bytes), chunks = stride / 16;
  int x = 8;
  while (x < 256 && x < chunks) x *= 2;
  hipLaunchKernelGGL((align_kernel<BYTES>), dim3((unsigned)ceil_div(o.rows, 256 / x * 4), (unsigned)ceil_div(chunks, x)), dim3(x, 256 / x), 0, st, o.p, o.stride,
                     o.rows, k_bytes, to, stride);
  return Operand{to, stride, o.rows};
}

// Whether products<S, true> takes the operand: its resource's offsets stay below 2^31.
inline bool direct(const Operand& o, int64_t k_bytes) {
  return ((uintptr_t)o.p & 15u) == 0 && (o.stride & 15) == 0 && (k_bytes & 15) == 0 && o.stride <= ((int64_t)1 << 22) && k_bytes <= ((int64_t)1 << 30);
}

}  // namespace tiles
}  // namespace simple
