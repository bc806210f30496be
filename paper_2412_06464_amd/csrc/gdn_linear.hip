// Linear attention with a decay for each head:
//     S_t = alpha_t S_{t-1} + k_t v_t^T,   o_t = S_t^T q_t.
// A chunk of 64 tokens with entry state S and G_t = log2 alpha_1 + .. + log2 alpha_t:
//     o_t    = 2^G_t S^T q_t + sum_{s <= t} 2^(G_t - G_s) (k_s . q_t) v_s
//     S_next = 2^G_64 S + sum_s k_s (2^(G_64 - G_s) v_s)^T
// k_linear walks the chunks of a sequence (or of a segment of it) for one head and a
// slice of dv, with the state slice in fp32 accumulators from the first chunk to
// the last: HBM sees q, k, v and o once and no chunk's state.  Every wave owns
// 16 columns of the slice, and the waves share out the tiles of P.  All products use the permuted
// contraction order of gdn_device.h, in which accumulator tiles are operands as
// they stand:
//     P   = K Q^T        (rows s, columns t)  A = K rows, B = Q rows, from LDS
//     O^T = S^T Q^T + V^T P^T (rows n, columns t)  A = S tiles and V^T, B = Q rows and P
//     S   = K^T V'       (rows dk, columns n) A = K^T, B = V' (v weighted)
// K^T and V^T come by transposing LDS reads (bf16).
//
// Where the sequences and heads do not fill the GPU, a sequence is cut into
// segments: k_linear<OUT = false> finds what each adds to the state,
// k_linear_scan turns that into entry states, and the segments are walked side by
// side.
//
// In bf16 the entry state and P are operands as two values each (PARTS), so that o is off by its
// own rounding alone; as one they left 1.4 times that, at 433 us of 487 for the packed prompts
// below, 412 of 485 for the wide heads (P's second value 6%, the state's the rest).
//
// Bound by a wave's chain of products, exponentials and barriers for each chunk, two waves
// to a SIMD (registers: 128 x 16 NC of the state, v and the outputs; the walks of 128 columns keep
// 64, at dk = 256 20 bytes a lane in scratch memory): 16 packed prompts of up to
// 8192 tokens, 16 heads of 128 x 128, bf16, 487 us (972 MB, a copy takes 187).  8 prompts of 4096, 6
// heads of 256 x 512: 192 workgroups, one to a CU, 7.6 us a chunk, 485 us (a copy takes 126).
#include <hip/hip_runtime.h>
#include <math.h>

#include "gdn_device.h"
#include "gdn_linear.h"

namespace gdn {

typedef bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));

#define LDS_AS __attribute__((address_space(3)))

constexpr float LOG2E = 1.4426950408889634f;

// One piece of a sequence: its tokens [t0, t1) of the call's rows.
struct Segment {
  int n, j;        // sequence, place in it
  int t0, t1;
  bool real, last;
};
__device__ inline Segment segment(const LinearArgs& a, int slot) {
  Segment s;
  int begin, end;
  if (a.len == 0) {
    s.n = slot;
    s.j = 0;
  } else if (a.cu) {
    int lo = 0, hi = a.N;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (a.cu[mid] / a.len + mid <= slot) lo = mid; else hi = mid;
    }
    s.n = lo;
    s.j = slot - (a.cu[lo] / a.len + lo);
  } else {
    const int per = (a.T - 1) / a.len + 1;
    s.n = slot / per;
    s.j = slot - s.n * per;
  }
  begin = a.cu ? a.cu[s.n] : s.n * a.T;
  end = a.cu ? a.cu[s.n + 1] : begin + a.T;
  const int64_t from = (int64_t)begin + (int64_t)s.j * a.len;
  s.real = s.j == 0 || from < end;
  s.t0 = (int)(from < end ? from : end);
  s.t1 = a.len && from + a.len < end ? (int)(from + a.len) : end;
  s.last = s.t1 == end;
  return s;
}

// log_alpha with -infinity as a finite value whose exponential is 0 too: differences of the
// sums stay defined.
__device__ inline float finite_log(float x) { return x < -1e4f ? -1e4f : x; }

// Two values as bf16 in a word, and what they left over.  (The word is opaque: the compiler would
// convert each again for the difference.  Wide heads, below, 508 us -> 485; the weighted v's three
// values, put this way, take registers that the walk does not have: 524.)
__device__ inline unsigned rounded(float a, float b, float& left_a, float& left_b) {
  const bf16x2 x = {(bf16)a, (bf16)b};
  unsigned w = *reinterpret_cast<const unsigned*>(&x);
  asm("" : "+v"(w));
  left_a = a - __uint_as_float(w << 16);
  left_b = b - __uint_as_float(w & 0xffff0000u);
  return w;
}
__device__ inline unsigned rounded(float a, float b) {
  const bf16x2 x = {(bf16)a, (bf16)b};
  return *reinterpret_cast<const unsigned*>(&x);
}
__device__ inline float finite(float x) { return fabsf(x) < INFINITY ? x : 0.f; }

// Four rows of two accumulator tiles (bf16), or one element (fp32), as an operand.  In bf16 as
// two: the values rounded, and what that left over (2^-16 of the value is lost).  FINITE: of an
// infinity or NaN nothing is left.
template <bool FINITE>
__device__ inline void operands(const f32x4* t, int stride, int kt, bf16x8 (&to)[2]) {
  u32x4 hi, lo;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const f32x4 x = t[(2 * kt + (j >> 1)) * stride];
    float a, b;
    hi[j] = rounded(x[2 * j & 3], x[2 * j + 1 & 3], a, b);
    lo[j] = FINITE ? rounded(finite(a), finite(b)) : rounded(a, b);
  }
  to[0] = *reinterpret_cast<const bf16x8*>(&hi);
  to[1] = *reinterpret_cast<const bf16x8*>(&lo);
}
template <bool FINITE>
__device__ inline void operands(const f32x4* t, int stride, int kt, float (&to)[1]) {
  to[0] = t[(kt >> 2) * stride][kt & 3];
}

// Matrices in LDS.  In bf16 an operand read takes 8 bytes of each of 16 rows, a transposing one
// 32 bytes of each of 4: with rows 8 banks apart (of 32) and the four 8-byte units of a 32-byte
// block exchanged by unit XOR (row / 4) % 4, both meet every bank once, and so do the
// accumulators' stores.  In fp32 they take 16 bytes of 8 rows, or 64 bytes of 2 rows 4 apart:
// rows 4 banks apart.
template <class E> struct Lds {
  static constexpr int PAD = sizeof(E) == 2 ? 16 : 4;  // DK, NV and 64 are multiples of 32 banks
};
__device__ inline int units(int row) { return (row >> 2) & 3; }

// 16-byte piece p of row r (its first element; row stride LD).
template <class E, int LD> __device__ inline u32x4* piece(E* m, int r, int p) {
  const int x = sizeof(E) == 2 ? p ^ (units(r) >> 1) : p;
  return reinterpret_cast<u32x4*>(m + r * LD + x * (16 / (int)sizeof(E)));
}
// A piece as it stands there, or back.
template <class E> __device__ inline u32x4 turned(u32x4 x, int r) {
  if constexpr (sizeof(E) == 4) return x;
  return units(r) & 1 ? u32x4{x[2], x[3], x[0], x[1]} : x;
}

// This lane's part (columns 4 g .. of every 16) of row 16 x + c16: its first element.
template <class E, int LD> __device__ inline E* row_part(E* m, int x) {
  const int c16 = lane_id() & 15, g = lane_id() >> 4;
  return m + (16 * x + c16) * LD + 4 * (sizeof(E) == 2 ? g ^ units(c16) : g);
}
// Operand of k-step kt of the row with this part.
template <class E> __device__ inline typename Mfma<E>::frag row_operand(const E* p, int kt) {
  if constexpr (sizeof(E) == 2) {
    const bf16x4 x = *reinterpret_cast<const bf16x4*>(p + 32 * kt);
    const bf16x4 y = *reinterpret_cast<const bf16x4*>(p + 32 * kt + 16);
    return __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
  } else {
    return p[16 * (kt >> 2) + (kt & 3)];
  }
}

// Operand of column c0 + (lane & 15) of an LDS matrix (row stride LD), rows of k-step kt.
template <class E, int LD>
__device__ inline typename Mfma<E>::frag col_operand(const E* m, int c0, int kt) {
  const int c16 = lane_id() & 15, g = lane_id() >> 4;
  if constexpr (sizeof(E) == 2) {
    // lane i of 16 points at 4 columns of row i / 4 and receives column i of the 4 rows
    // (units(row) is g)
    const E* p = m + (32 * kt + 4 * g + (c16 >> 2)) * LD + c0 + 4 * ((c16 & 3) ^ g);
    const s16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_AS s16x4*)p);
    const s16x4 y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_AS s16x4*)(p + 16 * LD));
    const s16x8 z = __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
    return *reinterpret_cast<const bf16x8*>(&z);
  } else {
    return m[(16 * (kt >> 2) + 4 * g + (kt & 3)) * LD + c0 + c16];
  }
}

// Infinities and NaN: the largest of the pieces' values without their signs (bf16: of each half
// of the words), and whether it is one.
template <class E> __device__ inline void see_odd(unsigned& most, u32x4 w) {
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if constexpr (sizeof(E) == 2) {
      const unsigned x = w[i] & 0x7fff7fffu;
      const u16x2 y = __builtin_elementwise_max(*reinterpret_cast<const u16x2*>(&most),
                                                *reinterpret_cast<const u16x2*>(&x));
      most = *reinterpret_cast<const unsigned*>(&y);
    } else {
      most = max(most, w[i] & 0x7fffffffu);
    }
}
template <class E> __device__ inline bool is_odd(unsigned most) {
  return most >= 0x7f800000u || (sizeof(E) == 2 && (most & 0xffffu) >= 0x7f80u);
}

// An operand with zeros in their place.
__device__ inline bf16x8 without_odd(bf16x8 x) {
  u32x4 w = *reinterpret_cast<const u32x4*>(&x);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if ((w[i] & 0x7f800000u) == 0x7f800000u) w[i] &= 0xffffu;
    if ((w[i] & 0x7f80u) == 0x7f80u) w[i] &= 0xffff0000u;
  }
  return *reinterpret_cast<const bf16x8*>(&w);
}

// Inclusive prefix sums over the 64 lanes: within rows of 16 lanes by shifts of 1, 2, 4 and
// 8, then each row's last to the row behind it, then the lower half's to the upper.  By DPP: six
// exchanges of 64 bits through LDS took 4,000 clocks of a chunk's 17,000.
template <int CTRL, int ROWS> __device__ inline double dpp_or_zero(double x) {
  const long long b = __double_as_longlong(x);
  const int lo = __builtin_amdgcn_update_dpp(0, (int)b, CTRL, ROWS, 0xf, false);
  const int hi = __builtin_amdgcn_update_dpp(0, (int)(b >> 32), CTRL, ROWS, 0xf, false);
  return __longlong_as_double(((long long)hi << 32) | (unsigned)lo);
}
__device__ inline double wave_sums(double x) {
  x += dpp_or_zero<0x111, 0xf>(x);  // row_shr 1
  x += dpp_or_zero<0x112, 0xf>(x);
  x += dpp_or_zero<0x114, 0xf>(x);
  x += dpp_or_zero<0x118, 0xf>(x);
  x += dpp_or_zero<0x142, 0xa>(x);  // row_bcast 15, to rows 1 and 3
  x += dpp_or_zero<0x143, 0xc>(x);  // row_bcast 31, to rows 2 and 3
  return x;
}

// One token's sum G of log2 alphas in a chunk (its value in fp32, and what that leaves
// over), 2^(G_64 - G) and 2^G.
struct Gates {
  float2 G[64];
  float left[64], grown[64];
};

// How a workgroup's DK x NV of the state lie over its waves: DK / KS rows and 16 NC
// columns each.
template <class E, int DK, int NV, bool OUT> struct LinearCfg {
  static constexpr int KS = DK == 256 ? 2 : 1;
  static constexpr int NC = sizeof(E) == 2 && NV == 128 && (OUT || DK == 256) ? 2 : 1;
};

// Waves a SIMD that the registers are to leave room for.
template <class E, int DK, int NV, int KS, int NC, bool OUT> constexpr int linear_waves() {
  constexpr int own = KS * NV / (16 * NC) / 4;
  if (sizeof(E) == 2 && KS == 1) return OUT ? (NC == 2 ? 2 : own) : 4;
  return own;
}

// Grid: groups of 8 units (slot, head) x slices of dv, a unit's slices 8 apart, so that
// they share the q and k of an XCD's L2.
template <class E, int DK, int NV, int KS, int NC, bool OUT>
__global__ __launch_bounds__(64 * KS * NV / (16 * NC), (linear_waves<E, DK, NV, KS, NC, OUT>()))
void k_linear(LinearArgs a) {
  using M = Mfma<E>;
  using frag = typename M::frag;
  constexpr int CW = NV / (16 * NC), W = CW * KS, NTH = 64 * W;
  constexpr int LK = DK + Lds<E>::PAD, LV = NV + Lds<E>::PAD, LP = 64 + Lds<E>::PAD;  // row strides
  constexpr int EPP = 16 / (int)sizeof(E);     // elements of a piece
  constexpr int PK = DK / EPP, PV = NV / EPP;  // pieces of a row
  constexpr int RK = 64 * PK / NTH, RV = 64 * PV / NTH;
  constexpr int KQ = DK / M::K / KS, KT = 64 / M::K, IT = DK / 16 / KS;
  constexpr int PARTS = sizeof(E) == 2 ? 2 : 1;  // operands that stand for the state, or for P
  constexpr int BP = PARTS * 64 * LP * (int)sizeof(E), BX = KS > 1 ? W * 2 * NC * 1024 : 0;
  // where LDS is short, P and the sums that waves exchange take the place of q, at the price
  // of a barrier
  constexpr bool OVER = OUT && 64 * (2 * LK + LV) * (int)sizeof(E) + BP + BX > 156 * 1024;
  __shared__ __align__(16) E sq[OUT ? 64 * LK : 16];
  __shared__ __align__(16) E sk[64 * LK];
  __shared__ __align__(16) E sv[64 * LV];
  __shared__ __align__(16) unsigned char more[OUT && !OVER ? BP + BX : 16];
  __shared__ Gates gates[2];
  __shared__ int sodd[2];
  E* const sp = OVER ? sq : (E*)more;                                       // P [part][t][s]
  f32x4* const sx = (f32x4*)((OVER ? (unsigned char*)sq : more) + BP);      // sums to add
  static_assert(!OVER || 64 * LK * (int)sizeof(E) >= BP + BX, "q's place is too small");

  const int tid = threadIdx.x, lane = lane_id(), g = lane >> 4, c16 = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(wave_id());
  const int kh = KS == 1 ? 0 : wave / CW, cw = KS == 1 ? wave : wave % CW;
  constexpr int GATES = W >= 8 ? W - 1 : 0;  // the wave that finds the gates
  const int slices = a.dv / NV;
  const int grp = blockIdx.x / (8 * slices), rest = blockIdx.x - grp * 8 * slices;
  const int slice = rest >> 3, unit = grp * 8 + (rest & 7);
  if (unit >= a.slots * a.H) return;
  const int slot = unit / a.H, h = unit - slot * a.H;
  const Segment seg = segment(a, slot);
  if (!seg.real || (!OUT && seg.last)) return;
  const int n0 = slice * NV + cw * 16 * NC;  // this wave's columns
  const int k0 = kh * (DK / KS);             // and rows
  const E* const Q = (const E*)a.q + (size_t)h * DK;
  const E* const K = (const E*)a.k + (size_t)h * DK;
  const E* const V = (const E*)a.v + (size_t)h * a.dv + slice * NV;
  const size_t rk = (size_t)a.H * DK, rv = (size_t)a.H * a.dv;  // elements between tokens

  // the state: rows k0 + 16 i + 4 g + e, column n0 + 16 c + c16
  f32x4 S[IT][NC];
  const size_t matrix = (size_t)DK * a.dv;
  {
    const float* from = nullptr;
    if (OUT && a.len) from = a.states + ((size_t)slot * a.H + h) * matrix;
    else if (seg.j == 0 && a.h0) from = a.h0 + ((size_t)seg.n * a.H + h) * matrix;
#pragma unroll
    for (int i = 0; i < IT; ++i)
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          S[i][c][e] =
              from ? from[(size_t)(k0 + 16 * i + 4 * g + e) * a.dv + n0 + 16 * c + c16] : 0.f;
  }

  // the next chunk's rows, on their way
  // (rows past the segment's last: that one again, cleared where they are stored)
  u32x4 nq[OUT ? RK : 1], nk[RK], nv[RV];
  const int pk = tid % PK * EPP, pv = tid % PV * EPP;  // NTH is a multiple of PK and PV
  auto fetch = [&](int t) {
#pragma unroll
    for (int i = 0; i < RK; ++i) {
      const size_t at = (size_t)min(t + tid / PK + NTH / PK * i, seg.t1 - 1) * rk + pk;
      if (OUT) nq[i] = *reinterpret_cast<const u32x4*>(Q + at);
      nk[i] = *reinterpret_cast<const u32x4*>(K + at);
    }
#pragma unroll
    for (int i = 0; i < RV; ++i)
      nv[i] = *reinterpret_cast<const u32x4*>(
          V + (size_t)min(t + tid / PV + NTH / PV * i, seg.t1 - 1) * rv + pv);
  };
  float la = 0.f;  // of the chunk whose gates are found next
  auto fetch_la = [&](int t) {
    la = 0.f;
    if (a.log_alpha && t + lane < seg.t1)
      la = a.log_alpha[a.per_head ? h : (size_t)(t + lane) * a.H + h];
  };
  double total = 0;  // log2 of the segment's product of alphas
  auto find_gates = [&](Gates& to) {
    // summed in 64 bits: the differences of two sums are what weighs
    const double x = wave_sums((double)finite_log(la) * 1.4426950408889634074);
    const double end = __shfl(x, 63);
    const float hi = (float)x;
    to.G[lane] = make_float2(hi, (float)(x - (double)hi));
    to.left[lane] = __builtin_amdgcn_exp2f((float)(end - x));
    to.grown[lane] = __builtin_amdgcn_exp2f((float)x);
    total += end;
  };
  if (seg.t0 < seg.t1) {
    fetch(seg.t0);
    if (wave == GATES) {
      fetch_la(seg.t0);
      find_gates(gates[0]);
      fetch_la(seg.t0 + 64);
    }
  }
  if (tid < 2) sodd[tid] = 0;
  auto put_out = [&](int t, int r, u32x4 x) {
    if (t + r < seg.t1)
      *reinterpret_cast<u32x4*>((E*)a.o + (size_t)(t + r) * rv + (size_t)h * a.dv + slice * NV + pv) =
          turned<E>(x, r);
  };

  int buf = 0, t = seg.t0;
  for (; t < seg.t1; t += 64, buf ^= 1) {
    lds_barrier();  // what stood there is no longer read; the outputs are in v's place
    if (t + 64 > seg.t1) {
#pragma unroll
      for (int i = 0; i < RK; ++i)
        if (t + tid / PK + NTH / PK * i >= seg.t1) {
          if (OUT) nq[i] = u32x4{0, 0, 0, 0};
          nk[i] = u32x4{0, 0, 0, 0};
        }
#pragma unroll
      for (int i = 0; i < RV; ++i)
        if (t + tid / PV + NTH / PV * i >= seg.t1) nv[i] = u32x4{0, 0, 0, 0};
    }
#pragma unroll
    for (int i = 0; i < RK; ++i) {
      const int r = tid / PK + NTH / PK * i;
      if (OUT) *piece<E, LK>(sq, r, tid % PK) = turned<E>(nq[i], r);
      *piece<E, LK>(sk, r, tid % PK) = turned<E>(nk[i], r);
    }
    unsigned most = 0;
#pragma unroll
    for (int i = 0; i < RK; ++i)
      if (sizeof(E) == 2) see_odd<E>(most, nk[i]);
#pragma unroll
    for (int i = 0; i < RV; ++i) {
      const int r = tid / PV + NTH / PV * i;
      u32x4* const at = piece<E, LV>(sv, r, tid % PV);
      // stored here, the outputs are long gone when the next rows are waited for (one
      // counter holds both)
      if (OUT && t > seg.t0) put_out(t - 64, r, *at);
      *at = turned<E>(nv[i], r);
      see_odd<E>(most, nv[i]);
    }
    if (is_odd<E>(most)) sodd[buf] = 1;
    if (t + 64 < seg.t1) fetch(t + 64);
    lds_barrier();
    const Gates& gt = gates[buf];
    const bool careful = __builtin_amdgcn_readfirstlane(sodd[buf]) != 0;
    if (tid == 0) sodd[buf ^ 1] = 0;
    if (wave == GATES) {
      find_gates(gates[buf ^ 1]);
      fetch_la(t + 128);
    }

    frag vf[KT][NC];
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
      for (int c = 0; c < NC; ++c) vf[kt][c] = col_operand<E, LV>(sv, cw * 16 * NC + 16 * c, kt);

    constexpr int MINE = KS == 1 ? 4 : 2;  // token tiles whose outputs this wave finishes
    f32x4 mine[MINE][NC];
    if constexpr (OUT) {
      // P: rows s, columns t.  Tasks of two tiles side by side, of one
      auto task = [&](auto count, int tt, int s) {
        constexpr int CNT = decltype(count)::value;
        f32x4 p[CNT], r[CNT];  // sums of even and odd steps
#pragma unroll
        for (int j = 0; j < CNT; ++j) p[j] = r[j] = f32x4{0.f, 0.f, 0.f, 0.f};
        constexpr int PART = DK / M::K > 8 ? DK / M::K / 8 : 1;  // (fp32: a part of a row at a time)
#pragma unroll
        for (int x = 0; x < PART; ++x) {
          constexpr int D = DK / PART;
          frag q[D / M::K], k[CNT][D / M::K];
          const E* const pq = row_part<E, LK>(sq, tt) + x * D;
#pragma unroll
          for (int kt = 0; kt < D / M::K; ++kt) q[kt] = row_operand<E>(pq, kt);
#pragma unroll
          for (int j = 0; j < CNT; ++j) {
            const E* const p = row_part<E, LK>(sk, s + j) + x * D;
#pragma unroll
            for (int kt = 0; kt < D / M::K; ++kt) k[j][kt] = row_operand<E>(p, kt);
          }
#pragma unroll
          for (int kt = 0; kt < D / M::K; ++kt)
#pragma unroll
            for (int j = 0; j < CNT; ++j) {
              f32x4& to = kt & 1 ? r[j] : p[j];
              to = M::mma(k[j][kt], q[kt], to);
            }
        }
#pragma unroll
        for (int j = 0; j < CNT; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) p[j][e] += r[j][e];
        const float2 Gt = gt.G[16 * tt + c16];
#pragma unroll
        for (int j = 0; j < CNT; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float2 Gs = gt.G[16 * (s + j) + 4 * g + e];
            float w = __builtin_amdgcn_exp2f((Gt.x - Gs.x) + (Gt.y - Gs.y));
            asm("" : "+v"(w));  // (or each stands behind a branch of its own)
            p[j][e] = s + j < tt || 4 * g + e <= c16 ? p[j][e] * w : 0.f;
          }
        if constexpr (OVER) lds_barrier();
#pragma unroll
        for (int j = 0; j < CNT; ++j) {
          E* const to = row_part<E, LP>(sp, tt) + 16 * (s + j);
          if constexpr (PARTS == 1) {
            *reinterpret_cast<f32x4*>(to) = p[j];
          } else {  // (of an infinity nothing is left over)
            float r[4];
            u32x2 y, z;
            y[0] = rounded(p[j][0], p[j][1], r[0], r[1]);
            y[1] = rounded(p[j][2], p[j][3], r[2], r[3]);
            z[0] = rounded(finite(r[0]), finite(r[1]));
            z[1] = rounded(finite(r[2]), finite(r[3]));
            *reinterpret_cast<u32x2*>(to) = y;
            *reinterpret_cast<u32x2*>(to + 64 * LP) = z;
          }
        }
      };
      // the entry state's part
      f32x4 o[4][NC];
      auto state_part = [&](auto finite) {
        constexpr bool FINITE = decltype(finite)::value;
#pragma unroll
        for (int tt = 0; tt < 4; ++tt)
#pragma unroll
          for (int c = 0; c < NC; ++c) o[tt][c] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int kt = 0; kt < KQ; ++kt) {
          frag sf[NC][PARTS];
#pragma unroll
          for (int c = 0; c < NC; ++c) operands<FINITE>(&S[0][c], NC, kt, sf[c]);
#pragma unroll
          for (int tt = 0; tt < 4; ++tt) {
            frag q = row_operand<E>(row_part<E, LK>(sq, tt) + k0, kt);
#pragma unroll
            for (int c = 0; c < NC; ++c) o[tt][c] = M::mma(sf[c][0], q, o[tt][c]);
            if constexpr (PARTS == 2) {
              if constexpr (FINITE) q = without_odd(q);
#pragma unroll
              for (int c = 0; c < NC; ++c) o[tt][c] = M::mma(sf[c][1], q, o[tt][c]);
            }
          }
        }
      };
      auto from_state = [&]() {
        state_part(std::false_type{});
        if constexpr (PARTS == 2) {
          // An infinity of the state or of q meets the first parts alone: the second ones
          // may be NaN, 0, or of the other sign.
          float most = 0.f;  // (a NaN stays one)
#pragma unroll
          for (int tt = 0; tt < 4; ++tt)
#pragma unroll
            for (int c = 0; c < NC; ++c)
#pragma unroll
              for (int e = 0; e < 4; ++e)
                most = __builtin_elementwise_maximum(most, fabsf(o[tt][c][e]));
          if (__any(!(most < INFINITY))) {
            // (opaque, or the first pass' operands are kept in registers for this one)
#pragma unroll
            for (int i = 0; i < IT; ++i)
#pragma unroll
              for (int c = 0; c < NC; ++c) asm volatile("" : "+v"(S[i][c])::"memory");
            state_part(std::true_type{});
          }
        }
      };
      constexpr std::integral_constant<int, 1> one{};
      constexpr std::integral_constant<int, 2> two{};
      if constexpr (OVER) {
        static_assert(!OVER || W == 8, "each wave has one task");
        from_state();
        // (a wave without a task meets the others' barrier alone)
        if (wave < 4) task(two, wave < 2 ? 3 : 4 - wave, wave == 1 ? 2 : 0);
        else if (wave < 6) task(one, wave == 4 ? 2 : 0, wave == 4 ? 2 : 0);
        else lds_barrier();
      } else {
        if (wave < 4) task(two, wave < 2 ? 3 : 4 - wave, wave == 1 ? 2 : 0);
        const int x = W >= 8 ? wave : wave + 2;
        if (x == 4 || x == 5) task(one, x == 4 ? 2 : 0, x == 4 ? 2 : 0);
        from_state();
      }
      // two waves of the same columns: each adds up two of the four token tiles
      if constexpr (KS == 1) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int c = 0; c < NC; ++c) mine[j][c] = o[j][c];
      } else {
#pragma unroll
        for (int c = 0; c < NC; ++c) {
          mine[0][c] = kh ? o[1][c] : o[0][c];
          mine[1][c] = kh ? o[2][c] : o[3][c];
          sx[((wave * 2 + 0) * NC + c) * 64 + lane] = kh ? o[0][c] : o[1][c];
          sx[((wave * 2 + 1) * NC + c) * 64 + lane] = kh ? o[3][c] : o[2][c];
        }
      }
    }

    // the state: v weighted, in bf16 as three values, which is all of its 24 bits.  (One value
    // would leave the state with eight; two, with the state 1.4e-6 off, 10% faster)
    const float fe = gt.grown[63];
#pragma unroll
    for (int i = 0; i < IT; ++i)
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int e = 0; e < 4; ++e) S[i][c][e] *= fe;
#pragma unroll
    for (int kt = 0; kt < KT; ++kt) {
      frag hi[NC], lo[NC], rest[NC];
      if constexpr (sizeof(E) == 2) {
        const f32x4 w0 = *reinterpret_cast<const f32x4*>(gt.left + 32 * kt + 4 * g);
        const f32x4 w1 = *reinterpret_cast<const f32x4*>(gt.left + 32 * kt + 16 + 4 * g);
#pragma unroll
        for (int c = 0; c < NC; ++c) {
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const float x = (float)vf[kt][c][j] * (j < 4 ? w0[j & 3] : w1[j & 3]);
            hi[c][j] = (bf16)x;
            const float y = x - (float)hi[c][j];
            lo[c][j] = (bf16)y;
            rest[c][j] = (bf16)(y - (float)lo[c][j]);
          }
          if (careful)  // (an infinity less itself)
#pragma unroll
            for (int j = 0; j < 8; ++j)
              if ((float)lo[c][j] != (float)lo[c][j]) lo[c][j] = rest[c][j] = (bf16)0.f;
        }
      } else {
        const float w = gt.left[16 * (kt >> 2) + 4 * g + (kt & 3)];
#pragma unroll
        for (int c = 0; c < NC; ++c) hi[c] = vf[kt][c] * w;
      }
      // (four row tiles at a time: products that follow each other do not wait for one another)
#pragma unroll
      for (int i0 = 0; i0 < IT; i0 += 4) {
        frag x[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = col_operand<E, LK>(sk, k0 + 16 * (i0 + i), kt);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int c = 0; c < NC; ++c) S[i0 + i][c] = M::mma(x[i], hi[c], S[i0 + i][c]);
        if constexpr (sizeof(E) == 2) {
          // (an infinity meets the first value: the others may be 0, or of the other sign)
          if (careful)
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = without_odd(x[i]);
#pragma unroll
          for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int c = 0; c < NC; ++c) S[i0 + i][c] = M::mma(x[i], lo[c], S[i0 + i][c]);
#pragma unroll
          for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int c = 0; c < NC; ++c) S[i0 + i][c] = M::mma(x[i], rest[c], S[i0 + i][c]);
        }
      }
    }

    if constexpr (OUT) {
      lds_barrier();
      auto tile = [&](int j) { return KS == 1 ? j : kh ? 1 + j : 3 * j; };
#pragma unroll
      for (int j = 0; j < MINE; ++j) {
        const float et = gt.grown[16 * tile(j) + c16];
#pragma unroll
        for (int c = 0; c < NC; ++c) {
          if constexpr (KS > 1) {
            const f32x4 y = sx[(((wave ^ CW) * 2 + j) * NC + c) * 64 + lane];
#pragma unroll
            for (int e = 0; e < 4; ++e) mine[j][c][e] += y[e];
          }
#pragma unroll
          for (int e = 0; e < 4; ++e) mine[j][c][e] *= et;
        }
      }
      if (!careful) {
#pragma unroll
        for (int j = 0; j < MINE; ++j) {
          const int tt = tile(j), most = KS == 1 ? j : 1 + 2 * j;  // (most: at compile time)
#pragma unroll
          for (int part = 0; part < PARTS; ++part) {
            frag x[KT];
            const E* const p = row_part<E, LP>(sp, tt) + part * 64 * LP;
#pragma unroll
            for (int kt = 0; kt < KT; ++kt) x[kt] = row_operand<E>(p, kt);
#pragma unroll
            for (int kt = 0; kt < KT; ++kt) {
              // what is past the diagonal tile was not written
              if constexpr (sizeof(E) == 2) {
                if (2 * kt > most) continue;
                const bf16x8 half = __builtin_shufflevector(x[kt], bf16x8{}, 0, 1, 2, 3, 8, 9, 10, 11);
                x[kt] = 2 * kt < tt ? x[kt] : half;
              } else {
                if (kt / 4 > most) continue;
                x[kt] = kt / 4 <= tt ? x[kt] : 0.f;
              }
#pragma unroll
              for (int c = 0; c < NC; ++c) mine[j][c] = M::mma(vf[kt][c], x[kt], mine[j][c]);
            }
          }
        }
      } else {
        // an infinity or NaN in v must not meet the zeros of earlier tokens
#pragma unroll
        for (int j = 0; j < MINE; ++j) {
          const int tt = tile(j);
#pragma unroll 1
          for (int s = 0; s <= 16 * tt + c16; ++s) {
            const bool b = sizeof(E) == 2;
            const E* const p = sp + (16 * tt + c16) * LP + (b ? s ^ 4 * units(c16) : s);
            const float w = to_f(p[0]) + (PARTS == 2 ? to_f(p[(PARTS - 1) * 64 * LP]) : 0.f);
            const E* from = sv + s * LV + cw * 16 * NC + 4 * (b ? g ^ units(s) : g);
#pragma unroll
            for (int c = 0; c < NC; ++c)
#pragma unroll
              for (int e = 0; e < 4; ++e) mine[j][c][e] += w * to_f(from[16 * c + e]);
          }
        }
        lds_barrier();
      }
      // v is in registers, or read: o takes its place
#pragma unroll
      for (int j = 0; j < MINE; ++j)
#pragma unroll
        for (int c = 0; c < NC; ++c)
          *reinterpret_cast<typename Raw4<E>::type*>(row_part<E, LV>(sv, tile(j)) + cw * 16 * NC +
                                                     16 * c) =
              typename Raw4<E>::type{to_e<E>(mine[j][c][0]), to_e<E>(mine[j][c][1]),
                                     to_e<E>(mine[j][c][2]), to_e<E>(mine[j][c][3])};
    }
  }
  if (OUT && t > seg.t0) {
    lds_barrier();
#pragma unroll
    for (int i = 0; i < RV; ++i) {
      const int r = tid / PV + NTH / PV * i;
      put_out(t - 64, r, *piece<E, LV>(sv, r, tid % PV));
    }
  }

  float* to = nullptr;
  if (!OUT) {
    to = a.states + ((size_t)slot * a.H + h) * matrix;
    // (the gates of one more chunk are in the total: those past the segment are 0)
    if (slice == 0 && wave == GATES && lane == 0)
      a.fade[(size_t)slot * a.H + h] = (float)exp2(total);
  } else if (seg.last && a.ht) {
    to = a.ht + ((size_t)seg.n * a.H + h) * matrix;
  }
  if (to) {
#pragma unroll
    for (int i = 0; i < IT; ++i)
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          to[(size_t)(k0 + 16 * i + 4 * g + e) * a.dv + n0 + 16 * c + c16] = S[i][c][e];
  }
}

// Entry states of a sequence's segments from what each adds: E_0 = h0,
// E_{j+1} = fade_j E_j + Z_j, in place (the first segment's Z holds h0 already, and
// its E takes h0's copy, so that ht may be h0).  HBM: each state once in, once out (126 MB:
// 22 us).
// Grid: ((n * H + h) * pieces + piece), a thread 4 values.
__global__ __launch_bounds__(256) void k_linear_scan(LinearArgs a) {
  const int matrix = a.dk * a.dv, pieces = matrix / 1024;
  const int nh = blockIdx.x / pieces, at = (blockIdx.x - nh * pieces) * 1024 + threadIdx.x * 4;
  const int n = nh / a.H, h = nh - n * a.H;
  const int begin = a.cu ? a.cu[n] : 0, end = a.cu ? a.cu[n + 1] : a.T;
  const int per = (a.T - 1) / a.len + 1;
  const int slot = a.cu ? begin / a.len + n : n * per;
  const int J = end > begin ? (end - begin - 1) / a.len + 1 : 1;
  f32x4 E = {0.f, 0.f, 0.f, 0.f};
  if (a.h0) E = *reinterpret_cast<const f32x4*>(a.h0 + (size_t)nh * matrix + at);
  auto place = [&](int j) {
    return reinterpret_cast<f32x4*>(a.states + ((size_t)(slot + j) * a.H + h) * matrix + at);
  };
  f32x4 z = E;
  if (J > 1) z = *place(0);
  *place(0) = E;
  // (eight loads on their way at a time)
  constexpr int AHEAD = 8;
  for (int j0 = 1; j0 < J; j0 += AHEAD) {
    f32x4 y[AHEAD];
    float f[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      if (j0 + i + 1 >= J) break;  // (the last's is not needed)
      y[i] = *place(j0 + i);
      f[i] = a.fade[(size_t)(slot + j0 + i) * a.H + h];
    }
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      if (j0 + i >= J) break;
      E = z;
      if (j0 + i + 1 < J)
#pragma unroll
        for (int e = 0; e < 4; ++e) z[e] = fmaf(f[i], E[e], y[i][e]);
      *place(j0 + i) = E;
    }
  }
}

// Token by token.  A workgroup owns DK x 64 of the state, in registers from the first token
// to the last: thread (rg, cg) holds rows rg + 16 i, columns 4 cg.. of it.  Bound by
// the state's way from and to HBM: 256 single tokens, 6 heads of 256 x 512, 314 us, 5.1 TB/s;
// 4 of 16 heads of 128 x 128, 4.3 us.
template <class E, int DK>
__global__ __launch_bounds__(256) void k_linear_recurrent(LinearArgs a) {
  constexpr int NR = DK / 16;
  __shared__ float skq[2][2][DK];   // k, q of the token, two buffers
  __shared__ f32x4 sred[2][4][16];  // the waves' sums, two buffers
  const int tid = threadIdx.x, lane = lane_id(), w = wave_id();
  const int cg = tid & 15, rg = tid >> 4;
  const int tiles = a.dv / 64, nh = blockIdx.x / tiles;
  const int n = nh / a.H, h = nh - n * a.H, v0 = (blockIdx.x - nh * tiles) * 64 + 4 * cg;
  const int begin = a.cu ? a.cu[n] : n * a.T, end = a.cu ? a.cu[n + 1] : begin + a.T;
  const size_t at = (size_t)nh * DK * a.dv + (size_t)rg * a.dv + v0, step = (size_t)16 * a.dv;
  f32x4 S[NR];
#pragma unroll
  for (int i = 0; i < NR; ++i)
    S[i] = a.h0 ? *reinterpret_cast<const f32x4*>(a.h0 + at + i * step) : f32x4{0.f, 0.f, 0.f, 0.f};
  for (int t = begin; t < end; ++t) {
    const size_t row = (size_t)t * a.H + h;
    const int buf = (t - begin) & 1;
    for (int x = tid; x < DK; x += 256) {
      skq[buf][0][x] = to_f(((const E*)a.k)[row * DK + x]);
      skq[buf][1][x] = to_f(((const E*)a.q)[row * DK + x]);
    }
    const f32x4 v = load4<E>((const E*)a.v + row * a.dv + v0);
    const float al =
        a.log_alpha ? __builtin_amdgcn_exp2f(a.log_alpha[a.per_head ? h : row] * LOG2E) : 1.f;
    lds_barrier();
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < NR; ++i) {
      const float k = skq[buf][0][rg + 16 * i], q = skq[buf][1][rg + 16 * i];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        S[i][e] = fmaf(k, v[e], al * S[i][e]);
        o[e] = fmaf(q, S[i][e], o[e]);
      }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      o[e] += __shfl_xor(o[e], 16, 64);
      o[e] += __shfl_xor(o[e], 32, 64);
    }
    if (lane < 16) sred[buf][w][lane] = o;
    lds_barrier();
    if (tid < 16) {
      f32x4 y = sred[buf][0][tid];
#pragma unroll
      for (int x = 1; x < 4; ++x)
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] += sred[buf][x][tid][e];
      store4<E>((E*)a.o + row * a.dv + v0, y);
    }
  }
  if (a.ht) {
#pragma unroll
    for (int i = 0; i < NR; ++i) *reinterpret_cast<f32x4*>(a.ht + at + i * step) = S[i];
  }
}

// ---- launchers

namespace {

template <class F> hipError_t by_dk(Dt dt, int dk, F&& f) {
  auto go = [&](auto e) {
    using E = decltype(e);
    if (dk == 64) return f(E{}, std::integral_constant<int, 64>{});
    if (dk == 128) return f(E{}, std::integral_constant<int, 128>{});
    return f(E{}, std::integral_constant<int, 256>{});
  };
  if (dk != 64 && dk != 128 && dk != 256) return hipErrorInvalidValue;
  return dt == Dt::F32 ? go(float{}) : go(bf16{});
}

template <bool OUT> hipError_t launch(Dt dt, const LinearArgs& a, hipStream_t s) {
  const int nv = linear_slice(dt, a.dk, a.dv);
  const int64_t units = (int64_t)a.slots * a.H;
  const unsigned grid = (unsigned)((units + 7) / 8 * 8 * (a.dv / nv));
  return by_dk(dt, a.dk, [&](auto e, auto dim) {
    using E = decltype(e);
    constexpr int DK = decltype(dim)::value;
    auto go = [&](auto columns) {
      constexpr int NV = decltype(columns)::value;
      using C = LinearCfg<E, DK, NV, OUT>;
      hipLaunchKernelGGL((k_linear<E, DK, NV, C::KS, C::NC, OUT>), dim3(grid),
                         dim3(64 * C::KS * NV / (16 * C::NC)), 0, s, a);
      return hipGetLastError();
    };
    if constexpr (sizeof(E) == 2 || DK < 256)
      if (nv == 128) return go(std::integral_constant<int, 128>{});
    return go(std::integral_constant<int, 64>{});
  });
}

}  // namespace

int linear_slice(Dt dt, int dk, int dv) {
  // (fp32 rows of 256: q, k and 128 columns of v would pass a CU's LDS)
  return dv % 128 || (dt == Dt::F32 && dk == 256) ? 64 : 128;
}

hipError_t launch_linear_states(Dt dt, const LinearArgs& a, hipStream_t s) {
  const hipError_t e = launch<false>(dt, a, s);
  if (e != hipSuccess) return e;
  const unsigned grid = (unsigned)((int64_t)a.N * a.H * (a.dk * a.dv / 1024));
  hipLaunchKernelGGL(k_linear_scan, dim3(grid), dim3(256), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_linear_walk(Dt dt, const LinearArgs& a, hipStream_t s) {
  return launch<true>(dt, a, s);
}

hipError_t launch_linear_recurrent(Dt dt, const LinearArgs& a, hipStream_t s) {
  const unsigned grid = (unsigned)((int64_t)a.N * a.H * (a.dv / 64));
  return by_dk(dt, a.dk, [&](auto e, auto dim) {
    using E = decltype(e);
    hipLaunchKernelGGL((k_linear_recurrent<E, decltype(dim)::value>), dim3(grid), dim3(256), 0, s, a);
    return hipGetLastError();
  });
}

}  // namespace gdn
