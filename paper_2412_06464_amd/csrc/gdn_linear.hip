// Linear attention with a decay for each head:
//     S_t = alpha_t S_{t-1} + k_t v_t^T,   o_t = S_t^T q_t.
// A chunk of 64 tokens with entry state S and G_t = log2 alpha_1 + .. + log2 alpha_t:
//     o_t    = 2^G_t S^T q_t + sum_{s <= t} 2^(G_t - G_s) (k_s . q_t) v_s
//     S_next = 2^G_64 S + sum_s k_s (2^(G_64 - G_s) v_s)^T
// k_linear walks the chunks of a sequence (or of a segment of it) for one head and a
// slice of dv, with the state slice in fp32 accumulators from the first chunk to
// the last: HBM sees q, k, v and o once and no chunk's state.  Every wave owns
// 16 or 32 columns of the slice and needs nothing of the others but the rows of
// q, k and v in LDS, so a chunk takes two barriers.  All products use the permuted
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
#include <hip/hip_runtime.h>
#include <math.h>

#include "gdn_device.h"
#include "gdn_linear.h"

namespace gdn {

typedef bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

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

// Four rows of two accumulator tiles (bf16), or one element (fp32), as an operand.
template <class E> __device__ inline typename Mfma<E>::frag operand(const f32x4* tiles, int stride, int kt);
template <> __device__ inline bf16x8 operand<bf16>(const f32x4* t, int stride, int kt) {
  const f32x4 x = t[2 * kt * stride], y = t[(2 * kt + 1) * stride];
  return bf16x8{(bf16)x[0], (bf16)x[1], (bf16)x[2], (bf16)x[3],
                (bf16)y[0], (bf16)y[1], (bf16)y[2], (bf16)y[3]};
}
template <> __device__ inline float operand<float>(const f32x4* t, int stride, int kt) {
  return t[(kt >> 2) * stride][kt & 3];
}

// Operands of a row in LDS (p: the row's element 4 (lane >> 4)), all k-steps of KD.
template <class E, int KD>
__device__ inline void row_operands(typename Mfma<E>::frag (&f)[KD / Mfma<E>::K], const E* p) {
  if constexpr (sizeof(E) == 2) {
#pragma unroll
    for (int kt = 0; kt < KD / 32; ++kt) {
      const bf16x4 x = *reinterpret_cast<const bf16x4*>(p + 32 * kt);
      const bf16x4 y = *reinterpret_cast<const bf16x4*>(p + 32 * kt + 16);
      f[kt] = __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
    }
  } else {
#pragma unroll
    for (int i = 0; i < KD / 16; ++i) {
      const f32x4 x = *reinterpret_cast<const f32x4*>(p + 16 * i);
#pragma unroll
      for (int e = 0; e < 4; ++e) f[4 * i + e] = x[e];
    }
  }
}

// Operand of column c0 + (lane & 15) of an LDS matrix (row stride LD), rows of k-step kt.
template <class E, int LD>
__device__ inline typename Mfma<E>::frag col_operand(const E* m, int c0, int kt) {
  const int c16 = lane_id() & 15, g = lane_id() >> 4;
  if constexpr (sizeof(E) == 2) {
    // lane i of 16 points at 4 columns of row i / 4 and receives column i of the 4 rows
    const E* p = m + (32 * kt + 4 * g + (c16 >> 2)) * LD + c0 + 4 * (c16 & 3);
    const s16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_AS s16x4*)p);
    const s16x4 y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_AS s16x4*)(p + 16 * LD));
    const s16x8 z = __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
    return *reinterpret_cast<const bf16x8*>(&z);
  } else {
    return m[(16 * (kt >> 2) + 4 * g + (kt & 3)) * LD + c0 + c16];
  }
}

template <class E> __device__ inline bool has_odd(u32x4 w) {
  bool odd = false;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    odd = odd || (w[i] & 0x7f800000u) == 0x7f800000u ||
          (sizeof(E) == 2 && (w[i] & 0x7f80u) == 0x7f80u);
  return odd;
}

// DK x (64 NC) of the state a workgroup, 16 NC columns of it a wave.
// Grid: groups of 8 units (slot, head) x slices of dv, a unit's slices 8 apart, so that
// they share the q and k of an XCD's L2.
template <class E, int DK, int NC, bool OUT>
__global__ __launch_bounds__(256) void k_linear(LinearArgs a) {
  using M = Mfma<E>;
  constexpr int NV = 64 * NC, PAD = sizeof(E) == 2 ? 16 : 4;
  constexpr int LK = DK + PAD, LV = NV + PAD;  // row strides: operand reads spread over the banks
  constexpr int EPP = 16 / (int)sizeof(E);     // elements of a piece
  constexpr int PK = DK / EPP, PV = NV / EPP;  // pieces of a row
  constexpr int RK = 64 * PK / 256, RV = 64 * PV / 256;
  constexpr int KQ = DK / M::K, KT = 64 / M::K, IT = DK / 16;
  __shared__ __align__(16) E sq[OUT ? 64 * LK : 16];
  __shared__ __align__(16) E sk[64 * LK];
  __shared__ __align__(16) E sv[64 * LV];
  __shared__ float2 sg[64];  // G: its value in fp32, and what that leaves over
  __shared__ int sodd;

  const int tid = threadIdx.x, lane = lane_id(), g = lane >> 4, c16 = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(wave_id());
  const int slices = a.dv / NV;
  const int grp = blockIdx.x / (8 * slices), rest = blockIdx.x - grp * 8 * slices;
  const int slice = rest >> 3, unit = grp * 8 + (rest & 7);
  if (unit >= a.slots * a.H) return;
  const int slot = unit / a.H, h = unit - slot * a.H;
  const Segment seg = segment(a, slot);
  if (!seg.real || (!OUT && seg.last)) return;
  const int n0 = slice * NV + wave * 16 * NC;  // this wave's columns
  const E* const Q = (const E*)a.q + (size_t)h * DK;
  const E* const K = (const E*)a.k + (size_t)h * DK;
  const E* const V = (const E*)a.v + (size_t)h * a.dv + slice * NV;
  const size_t rk = (size_t)a.H * DK, rv = (size_t)a.H * a.dv;  // elements between tokens

  // the state: rows 16 i + 4 g + e, column n0 + 16 c + c16
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
          S[i][c][e] = from ? from[(size_t)(16 * i + 4 * g + e) * a.dv + n0 + 16 * c + c16] : 0.f;
  }

  // the next chunk's rows, on their way
  u32x4 nq[OUT ? RK : 1], nk[RK], nv[RV];
  float nla = 0.f;
  auto fetch = [&](int t) {
    const u32x4 none = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < RK; ++i) {
      const int x = tid + 256 * i, r = x / PK, p = x - r * PK;
      const bool in = t + r < seg.t1;
      const size_t at = (size_t)(t + r) * rk + p * EPP;
      if (OUT) nq[i] = in ? *reinterpret_cast<const u32x4*>(Q + at) : none;
      nk[i] = in ? *reinterpret_cast<const u32x4*>(K + at) : none;
    }
#pragma unroll
    for (int i = 0; i < RV; ++i) {
      const int x = tid + 256 * i, r = x / PV, p = x - r * PV;
      nv[i] = t + r < seg.t1 ? *reinterpret_cast<const u32x4*>(V + (size_t)(t + r) * rv + p * EPP)
                             : none;
    }
    nla = 0.f;
    if (wave == 0 && a.log_alpha && t + lane < seg.t1)
      nla = a.log_alpha[a.per_head ? h : (size_t)(t + lane) * a.H + h];
  };
  if (seg.t0 < seg.t1) fetch(seg.t0);
  double total = 0;  // log2 of the segment's product of alphas

  for (int t = seg.t0; t < seg.t1; t += 64) {
    if (tid == 0) sodd = 0;
    lds_barrier();  // the rows before are no longer read
    bool odd = false;
#pragma unroll
    for (int i = 0; i < RK; ++i) {
      const int x = tid + 256 * i, r = x / PK, p = x - r * PK;
      if (OUT) *reinterpret_cast<u32x4*>(sq + r * LK + p * EPP) = nq[i];
      *reinterpret_cast<u32x4*>(sk + r * LK + p * EPP) = nk[i];
    }
#pragma unroll
    for (int i = 0; i < RV; ++i) {
      const int x = tid + 256 * i, r = x / PV, p = x - r * PV;
      *reinterpret_cast<u32x4*>(sv + r * LV + p * EPP) = nv[i];
      if (OUT) odd = odd || has_odd<E>(nv[i]);
    }
    if (OUT && odd) sodd = 1;
    if (wave == 0) {
      // summed in 64 bits: the differences of two sums are what weighs
      double x = (double)finite_log(nla) * 1.4426950408889634074;
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) {
        const double y = __shfl_up(x, d, 64);
        if (lane >= d) x += y;
      }
      const float hi = (float)x;
      sg[lane] = make_float2(hi, (float)(x - (double)hi));
    }
    if (t + 64 < seg.t1) fetch(t + 64);
    lds_barrier();

    float2 G[4][4];  // of tokens 16 s + 4 g + e
#pragma unroll
    for (int s = 0; s < 4; ++s)
#pragma unroll
      for (int e = 0; e < 4; ++e) G[s][e] = sg[16 * s + 4 * g + e];
    const float2 end = sg[63];
    total += (double)end.x + (double)end.y;

    typename M::frag vf[KT][NC];
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
      for (int c = 0; c < NC; ++c)
        vf[kt][c] = col_operand<E, LV>(sv, wave * 16 * NC + 16 * c, kt);

    if constexpr (OUT) {
      typename M::frag sf[KQ][NC];  // the state as an operand
#pragma unroll
      for (int kt = 0; kt < KQ; ++kt)
#pragma unroll
        for (int c = 0; c < NC; ++c) sf[kt][c] = operand<E>(&S[0][c], NC, kt);
      const bool careful = sodd != 0;
#pragma unroll
      for (int tt = 0; tt < 4; ++tt) {
        typename M::frag q[KQ];
        row_operands<E, DK>(q, sq + (16 * tt + c16) * LK + 4 * g);
        const float2 Gt = sg[16 * tt + c16];
        f32x4 o[NC];
#pragma unroll
        for (int c = 0; c < NC; ++c) o[c] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int kt = 0; kt < KQ; ++kt)
#pragma unroll
          for (int c = 0; c < NC; ++c) o[c] = M::mma(sf[kt][c], q[kt], o[c]);
        const float et = __builtin_amdgcn_exp2f(Gt.x + Gt.y);
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
          for (int e = 0; e < 4; ++e) o[c][e] *= et;
        f32x4 p[4];
#pragma unroll
        for (int s = 0; s < 4; ++s) p[s] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s = 0; s <= tt; ++s) {
          typename M::frag k[KQ];
          row_operands<E, DK>(k, sk + (16 * s + c16) * LK + 4 * g);
#pragma unroll
          for (int kt = 0; kt < KQ; ++kt) p[s] = M::mma(k[kt], q[kt], p[s]);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float w = __builtin_amdgcn_exp2f((Gt.x - G[s][e].x) + (Gt.y - G[s][e].y));
            p[s][e] = s < tt || 4 * g + e <= c16 ? p[s][e] * w : 0.f;
          }
        }
        if (!careful) {
#pragma unroll
          for (int kt = 0; kt < KT; ++kt) {
            if (kt * M::K >= 16 * (tt + 1)) break;
            const typename M::frag x = operand<E>(p, 1, kt);
#pragma unroll
            for (int c = 0; c < NC; ++c) o[c] = M::mma(vf[kt][c], x, o[c]);
          }
        } else {
          // an infinity or NaN in v must not meet the zeros of earlier tokens
#pragma unroll
          for (int s = 0; s <= tt; ++s)
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll 1
              for (int x = j; x < 16; x += 4) {
                const float w = __shfl(p[s][j], (x >> 2) * 16 + c16);
                if (s == tt && x > c16) continue;
                const E* from = sv + (16 * s + x) * LV + wave * 16 * NC + 4 * g;
#pragma unroll
                for (int c = 0; c < NC; ++c)
#pragma unroll
                  for (int e = 0; e < 4; ++e) o[c][e] += w * to_f(from[16 * c + e]);
              }
        }
        const int row = t + 16 * tt + c16;
        if (row < seg.t1) {
          E* to = (E*)a.o + (size_t)row * rv + (size_t)h * a.dv + n0 + 4 * g;
#pragma unroll
          for (int c = 0; c < NC; ++c) {
            typename Raw4<E>::type y = {to_e<E>(o[c][0]), to_e<E>(o[c][1]), to_e<E>(o[c][2]),
                                        to_e<E>(o[c][3])};
            *reinterpret_cast<typename Raw4<E>::type*>(to + 16 * c) = y;
          }
        }
      }
    }

    // the state: v weighted, in bf16 as two values (2^-17 of it is lost, where one
    // value would leave the state with eight bits)
    const float fe = __builtin_amdgcn_exp2f(end.x + end.y);
#pragma unroll
    for (int i = 0; i < IT; ++i)
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int e = 0; e < 4; ++e) S[i][c][e] *= fe;
    float w[4][4];
#pragma unroll
    for (int s = 0; s < 4; ++s)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        w[s][e] = __builtin_amdgcn_exp2f((end.x - G[s][e].x) + (end.y - G[s][e].y));
#pragma unroll
    for (int kt = 0; kt < KT; ++kt) {
      typename M::frag hi[NC], lo[NC];
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        if constexpr (sizeof(E) == 2) {
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const float x = (float)vf[kt][c][j] * w[2 * kt + (j >> 2)][j & 3];
            const bf16 y = (bf16)x;
            const float z = x - (float)y;
            hi[c][j] = y;
            lo[c][j] = (bf16)(z - z == 0.f ? z : 0.f);
          }
        } else {
          hi[c] = vf[kt][c] * w[kt >> 2][kt & 3];
        }
      }
#pragma unroll
      for (int i = 0; i < IT; ++i) {
        const typename M::frag x = col_operand<E, LK>(sk, 16 * i, kt);
#pragma unroll
        for (int c = 0; c < NC; ++c) {
          S[i][c] = M::mma(x, hi[c], S[i][c]);
          if constexpr (sizeof(E) == 2) S[i][c] = M::mma(x, lo[c], S[i][c]);
        }
      }
    }
  }

  float* to = nullptr;
  if (!OUT) {
    to = a.states + ((size_t)slot * a.H + h) * matrix;
    if (slice == 0 && tid == 0) a.fade[(size_t)slot * a.H + h] = (float)exp2(total);
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
          to[(size_t)(16 * i + 4 * g + e) * a.dv + n0 + 16 * c + c16] = S[i][c][e];
  }
}

// Entry states of a sequence's segments from what each adds: E_0 = h0,
// E_{j+1} = fade_j E_j + Z_j, in place (the first segment's Z holds h0 already, and
// its E takes h0's copy, so that ht may be h0).  HBM: each state once in, once out.
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
#pragma unroll 4
  for (int j = 1; j < J; ++j) {
    E = z;
    if (j + 1 < J) {
      const float f = a.fade[(size_t)(slot + j) * a.H + h];
      const f32x4 y = *place(j);
#pragma unroll
      for (int e = 0; e < 4; ++e) z[e] = fmaf(f, E[e], y[e]);
    }
    *place(j) = E;
  }
}

// Token by token.  A workgroup owns DK x 64 of the state, in registers from the first token
// to the last: thread (rg, cg) holds rows rg + 16 i, columns 4 cg.. of it.  Bound by
// the state's way from and to HBM.
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
    if constexpr (sizeof(E) == 2 || DK < 256) {
      if (nv == 128) {
        hipLaunchKernelGGL((k_linear<E, DK, 2, OUT>), dim3(grid), dim3(256), 0, s, a);
        return hipGetLastError();
      }
    }
    hipLaunchKernelGGL((k_linear<E, DK, 1, OUT>), dim3(grid), dim3(256), 0, s, a);
    return hipGetLastError();
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
