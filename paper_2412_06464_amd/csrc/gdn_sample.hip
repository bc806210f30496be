// The choice of the next token: temperature, top-k, top-p, min-p and a given random
// number.
//
// One workgroup a row.  All that a draw needs are places in the order of falling
// logits: the k-th token, the one where the sum of weights reaches top_p of it, the
// one where it passes u times the sum of what is kept (min_p needs none: what it
// keeps is a prefix too, and the shortest prefix has the smallest sum).  A histogram over
// the logarithm of the weight, with counts and sums, says in which bin a place lies;
// the bin's tokens are gathered, sorted and summed.  No row is sorted.
//
// Weights are whole multiples of 2^-42 of the largest (found with an exponential in 64
// bits), so that sums are exact, whatever their order, atomics included, and two
// places that differ are told apart: with weights in 32 bits one draw in 10^5 from a flat
// distribution would be off by a token.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "../../include/gdn_sample.h"
#include "gdn_device.h"

namespace {

using gdn::lane_id;
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned long long u64;

constexpr int NTH = 1024, NW = NTH / 64;
constexpr int BINS = 2048, CAP = 2048;  // of a histogram; tokens gathered at a time
constexpr double LOWEST = -43;          // log2 of the least weight that counts
constexpr int SCALE = 42;               // weights are multiples of 2^-SCALE
constexpr unsigned INDEX = (1u << 20) - 1;

struct SampleArgs {
  const unsigned char* logits;
  int64_t stride;  // bytes
  int vocab;
  const float *temperature, *top_p, *min_p, *u;
  const int* top_k;
  int* tokens;
  float* logprob;
};

// Tokens in the order of draws: a larger place comes first.  (A zero has no sign here.)
__device__ inline unsigned rank_of(float x) {
  const unsigned b = __float_as_uint(x + 0.f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ inline float value_of(unsigned r) {
  return __uint_as_float(r & 0x80000000u ? r & 0x7fffffffu : ~r);
}
__device__ inline u64 place_of(float x, int i) {
  return (u64)rank_of(x) << 20 | (INDEX - (unsigned)i);
}

struct Scale {
  float top;       // the largest logit
  double per;      // log2(e) / T
  // log2 of the weight of x; below LOWEST (or NaN): none
  __device__ double log2w(float x) const {
    if (isinf(top)) return x == top ? 0.0 : -1e9;
    return ((double)x - (double)top) * per;
  }
};

// 2^y in units of 2^-SCALE, LOWEST <= y <= 0: e^(f ln 2) for |f| <= 1/2 by its Taylor
// series, whose first term left out is 2e-13, under a unit of the largest weight.
__device__ inline u64 weight(double y) {
  const double n = __builtin_rint(y), f = (y - n) * 0.6931471805599453;
  double p = 1.0 / 3628800;
  p = __builtin_fma(p, f, 1.0 / 362880);
  p = __builtin_fma(p, f, 1.0 / 40320);
  p = __builtin_fma(p, f, 1.0 / 5040);
  p = __builtin_fma(p, f, 1.0 / 720);
  p = __builtin_fma(p, f, 1.0 / 120);
  p = __builtin_fma(p, f, 1.0 / 24);
  p = __builtin_fma(p, f, 1.0 / 6);
  p = __builtin_fma(p, f, 0.5);
  p = __builtin_fma(p, f, 1.0);
  p = __builtin_fma(p, f, 1.0);
  // rounded to a whole number by the addition
  const double v = __builtin_ldexp(p, (int)n + SCALE) + 4503599627370496.0;
  return (u64)__double_as_longlong(v) & 0xfffffffffffffull;
}

struct Found {
  int j;         // bin
  u64 before;    // sum of what comes before it
  unsigned n;    // and how many
};

struct Shared {
  unsigned count[2][BINS];
  u64 sum[2][BINS];
  u64 list[CAP];
  u64 part[2][NW];
  unsigned partc[NW];
  unsigned listed;
  int at;
  u64 before;
  unsigned nbefore;
  u64 lo, hi;
};

__device__ inline u64 wave_scan(u64 x) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const u64 y = __shfl_up(x, d, 64);
    if (lane_id() >= d) x += y;
  }
  return x;
}

// Inclusive sums over the workgroup's threads of two values at a time.
__device__ inline void block_scan(Shared& s, u64& x, u64& c) {
  const int w = threadIdx.x >> 6;
  x = wave_scan(x);
  c = wave_scan(c);
  __syncthreads();
  if (lane_id() == 63) {
    s.part[0][w] = x;
    s.part[1][w] = c;
  }
  __syncthreads();
  for (int i = 0; i < w; ++i) {
    x += s.part[0][i];
    c += s.part[1][i];
  }
}

// A row's logits, 16 bytes a thread at a time; what is past its ends is NaN.
template <class E> struct Row {
  static constexpr int N = 16 / (int)sizeof(E);
  const unsigned char* at;  // down to a multiple of 16 bytes
  int off, vocab, pieces;   // elements before the first; pieces in all
  __device__ Row(const unsigned char* p, int v) {
    off = (int)((uintptr_t)p & 15) / (int)sizeof(E);
    at = p - off * (int)sizeof(E);
    vocab = v;
    pieces = (off + v + N - 1) / N;
  }
  __device__ u32x4 load(int j) const {
    if (j > 0 && j < pieces - 1) return *reinterpret_cast<const u32x4*>(at + (int64_t)j * 16);
    u32x4 x = {~0u, ~0u, ~0u, ~0u};
    if (j >= pieces) return x;
#pragma unroll
    for (int e = 0; e < N; ++e) {
      const int i = j * N + e - off;
      if (i < 0 || i >= vocab) continue;
      if constexpr (sizeof(E) == 4) {
        x[e] = reinterpret_cast<const unsigned*>(at)[j * N + e];
      } else {
        const unsigned b = reinterpret_cast<const unsigned short*>(at)[j * N + e];
        x[e >> 1] = e & 1 ? (x[e >> 1] & 0xffffu) | b << 16 : (x[e >> 1] & 0xffff0000u) | b;
      }
    }
    return x;
  }
  __device__ static float get(const u32x4& x, int e) {
    if constexpr (sizeof(E) == 4) return __uint_as_float(x[e]);
    return __uint_as_float(e & 1 ? x[e >> 1] & 0xffff0000u : x[e >> 1] << 16);
  }
};

template <class E> __global__ __launch_bounds__(NTH) void k_sample(SampleArgs a) {
  constexpr int N = Row<E>::N;
  __shared__ Shared s;
  const int tid = threadIdx.x, wave = tid >> 6, r = blockIdx.x;
  const Row<E> row(a.logits + r * a.stride, a.vocab);
  // f(x, index) for this thread's tokens; two loads ahead.  Whole waves take part.
  auto each = [&](auto&& f) {
    u32x4 x = row.load(tid), y = row.load(tid + NTH);
#pragma unroll 1
    for (int j = tid; j - tid < row.pieces; j += NTH) {
      const u32x4 z = row.load(j + 2 * NTH);
#pragma unroll
      for (int e = 0; e < N; ++e) f(Row<E>::get(x, e), j * N + e - row.off);
      x = y;
      y = z;
    }
  };

  // the largest, the lowest index first
  u64 best = 0;
  {
    float top = -INFINITY;
    int at = -1;
    each([&](float x, int i) {
      if (x > top) top = x, at = i;
    });
    if (at >= 0) best = place_of(top, at);
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) best = max(best, (u64)__shfl_xor(best, d, 64));
    if (lane_id() == 0) s.part[0][wave] = best;
    __syncthreads();
    for (int i = 0; i < NW; ++i) best = max(best, s.part[0][i]);
    __syncthreads();
  }
  const float T = a.temperature ? a.temperature[r] : 1.f;
  if (best == 0 || !(T > 0.f)) {  // nothing to draw, or no draw
    if (tid == 0) {
      a.tokens[r] = best ? (int)(INDEX - (unsigned)(best & INDEX)) : -1;
      if (a.logprob) a.logprob[r] = best ? 0.f : -INFINITY;
    }
    return;
  }
  const Scale sc{value_of((unsigned)(best >> 20)), 1.4426950408889634074 / (double)T};
  const int k = a.top_k ? a.top_k[r] : 0;
  const double p = a.top_p ? (double)a.top_p[r] : 1.0, mp = a.min_p ? (double)a.min_p[r] : 0.0;
  const float un = a.u ? a.u[r] : 0.f;
  const double u = un > 0.f ? fmin((double)un, 1 - 0x1p-24) : 0.0;
  const bool by_k = k > 0 && k < a.vocab, by_p = p < 1.0, by_m = mp > 0.0;

  const double per_bin = -BINS / (1 - LOWEST);
  auto bin_of = [&](double y) { return (int)(y * per_bin); };  // y in [LOWEST, 0]

  auto clear = [&](int h) {
    for (int i = tid; i < BINS; i += NTH) {
      s.count[h][i] = 0;
      s.sum[h][i] = 0;
    }
    __syncthreads();
  };
  // one token into histogram h; what a whole wave has in one bin goes there at once
  auto add = [&](int h, bool in, int b, bool sums, u64 w) {
    const u64 who = __ballot(in);
    if (!who) return;
    const int first = __builtin_amdgcn_readlane(b, __ffsll(who) - 1);
    if (__popcll(who) > 8 && __ballot(in && b == first) == who) {
      u64 x = in ? w : 0;
      if (sums)
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) x += __shfl_xor(x, d, 64);
      if (lane_id() == 0) {
        atomicAdd(&s.count[h][first], (unsigned)__popcll(who));
        if (sums) atomicAdd(&s.sum[h][first], x);
      }
    } else if (in) {
      atomicAdd(&s.count[h][b], 1u);
      if (sums) atomicAdd(&s.sum[h][b], w);
    }
  };
  u64 kept_m = 0;  // sum of the weights that min_p keeps
  auto histogram = [&](bool sums) {
    clear(0);
    u64 mine = 0;
    each([&](float x, int) {
      const double y = sc.log2w(x);
      const bool in = y >= LOWEST;
      u64 w = 0;
      if (sums && in) {
        w = weight(y);
        if (by_m && (double)w >= mp * 0x1p42) mine += w;
      }
      add(0, in, in ? bin_of(y) : 0, sums, w);
    });
    __syncthreads();
    if (sums && by_m) {
      u64 none = 0;
      block_scan(s, mine, none);
      __syncthreads();
      if (tid == NTH - 1) s.before = mine;
      __syncthreads();
      kept_m = s.before;
    }
  };

  // The first bin of histogram h up to which, `base` and `nbase` before it, test(sum, count)
  // holds; the last that holds anything if none does.
  auto find_bin = [&](int h, u64 base, u64 nbase, auto&& test) {
    u64 x[2], c[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) x[i] = s.sum[h][2 * tid + i], c[i] = s.count[h][2 * tid + i];
    u64 sx = x[0] + x[1], scn = c[0] + c[1];
    block_scan(s, sx, scn);
    if (tid == 0) s.at = BINS;
    __syncthreads();
    u64 before = base + sx - x[0] - x[1], n = nbase + scn - c[0] - c[1];
    int mine = BINS;
    u64 mb = 0, mn = 0;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      if (mine == BINS && c[i] && test(before + x[i], n + c[i])) mine = 2 * tid + i, mb = before, mn = n;
      before += x[i];
      n += c[i];
    }
    if (mine < BINS) atomicMin(&s.at, mine);
    __syncthreads();
    if (s.at == BINS) {  // (never for a sum that the caller has from the same histogram)
      __syncthreads();
      if (tid == 0) s.at = -1;
      __syncthreads();
      const int last = c[1] ? 2 * tid + 1 : c[0] ? 2 * tid : -1;
      if (last >= 0) atomicMax(&s.at, last);
      __syncthreads();
      if (last >= 0 && last == s.at) mine = last, mb = before - x[last & 1], mn = n - c[last & 1];
    }
    if (mine == s.at) {
      s.before = mb;
      s.nbefore = (unsigned)mn;
    }
    __syncthreads();
    const Found f{s.at, s.before, s.nbefore};
    __syncthreads();
    return f;
  };

  // Gathers the tokens for which in(y, place) holds, at most CAP, and sorts them.
  auto gather = [&](auto&& in) {
    if (tid == 0) s.listed = 0;
    __syncthreads();
    each([&](float x, int i) {
      const double y = sc.log2w(x);
      if (!(y >= LOWEST)) return;
      const u64 c = place_of(x, i);
      if (in(y, c)) {
        const unsigned at = atomicAdd(&s.listed, 1u);
        if (at < CAP) s.list[at] = c;
      }
    });
    __syncthreads();
    const int n = min((int)s.listed, CAP);
    if (n <= 512) {  // each finds its place by comparing with all others
      const u64 mine = tid < n ? s.list[tid] : 0;
      int at = 0;
      if (tid < n)
        for (int i = 0; i < n; ++i) at += s.list[i] > mine;
      __syncthreads();
      if (tid < n) s.list[at] = mine;
      __syncthreads();
      return n;
    }
    const int m = n <= 1024 ? 1024 : 2048;
    for (int i = n + tid; i < m; i += NTH) s.list[i] = 0;
    __syncthreads();
    for (int size = 2; size <= m; size <<= 1)
      for (int step = size >> 1; step > 0; step >>= 1) {
        if (tid < m / 2) {
          const int i = 2 * tid - (tid & (step - 1)), j = i + step;
          const u64 x = s.list[i], y = s.list[j];
          if ((x < y) == ((i & size) == 0)) s.list[i] = y, s.list[j] = x;
        }
        __syncthreads();
      }
    return n;
  };
  // The first token of the sorted list up to which test(sum, count) holds (the last if none
  // does): its place, and the sum with it.
  u64 got_place = 0, got_sum = 0;
  auto find_listed = [&](int n, u64 base, u64 nbase, auto&& test) {
    u64 w[2], c[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      c[i] = 2 * tid + i < n;
      w[i] = c[i] ? weight(sc.log2w(value_of((unsigned)(s.list[2 * tid + i] >> 20)))) : 0;
    }
    u64 x = w[0] + w[1], cn = c[0] + c[1];
    block_scan(s, x, cn);
    if (tid == 0) s.at = n - 1;
    __syncthreads();
    u64 sum = base + x - w[0] - w[1], cnt = nbase + cn - c[0] - c[1];
    u64 sums[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      sum += w[i];
      cnt += c[i];
      sums[i] = sum;
      if (c[i] && test(sum, cnt)) atomicMin(&s.at, 2 * tid + i);
    }
    __syncthreads();
    if (s.at >> 1 == tid) s.before = sums[s.at & 1];
    __syncthreads();
    got_place = s.list[s.at];
    got_sum = s.before;
    __syncthreads();
  };
  // The same among the tokens of bin f.j, which may be more than the list holds: their places,
  // which are all different, are cut ever finer.
  auto find_in_bin = [&](const Found& f, auto&& test) {
    unsigned n = s.count[0][f.j];
    u64 lo = 0, hi = ~0ull, base = f.before, nbase = f.n;
    if (n > CAP) {
      u64 mlo = ~0ull, mhi = 0;
      each([&](float x, int i) {
        const double y = sc.log2w(x);
        if (!(y >= LOWEST) || bin_of(y) != f.j) return;
        const u64 c = place_of(x, i);
        mlo = min(mlo, c);
        mhi = max(mhi, c);
      });
      if (tid == 0) s.lo = ~0ull, s.hi = 0;
      __syncthreads();
      atomicMin(&s.lo, mlo);
      atomicMax(&s.hi, mhi);
      __syncthreads();
      lo = s.lo;
      hi = s.hi;
    }
    while (n > CAP) {
      int shift = 0;
      while ((hi - lo) >> shift >= BINS) ++shift;
      clear(1);
      each([&](float x, int i) {
        const double y = sc.log2w(x);
        const u64 c = place_of(x, i);
        const bool in = y >= LOWEST && bin_of(y) == f.j && c >= lo && c <= hi;
        add(1, in, in ? (int)((hi - c) >> shift) : 0, true, in ? weight(y) : 0);
      });
      __syncthreads();
      const Found g = find_bin(1, base, nbase, test);
      n = s.count[1][g.j];
      base = g.before;
      nbase = g.n;
      hi -= (u64)g.j << shift;
      const u64 width = ((u64)1 << shift) - 1;
      if (hi - lo > width) lo = hi - width;
      __syncthreads();
    }
    const int m = gather([&](double y, u64 c) { return bin_of(y) == f.j && c >= lo && c <= hi; });
    find_listed(m, base, nbase, test);
  };

  // Where top_k leaves few tokens, counts alone say in which bin the last of them lies, and
  // the list of all tokens up to there is all that is looked at from then on.
  const bool counts = by_k && k <= CAP / 2;
  histogram(!counts);
  int listed = 0;  // tokens of the list, if it holds all that can be kept
  auto reaches_k = [&](u64, u64 n) { return n >= (u64)k; };
  if (counts) {
    const Found f = find_bin(0, 0, 0, reaches_k);
    if (f.n + s.count[0][f.j] <= CAP)
      listed = gather([&](double y, u64) { return bin_of(y) <= f.j; });
    else
      histogram(true);
  }
  u64 total;
  if (listed) {
    find_listed(listed, 0, 0, reaches_k);
    total = got_sum;
  } else if (by_k) {
    const Found f = find_bin(0, 0, 0, reaches_k);
    find_in_bin(f, reaches_k);
    total = got_sum;
  } else {
    // (all: the bin past the last)
    const Found f = find_bin(0, 0, 0, [&](u64, u64) { return false; });
    total = f.before + s.sum[0][f.j];
  }
  if (by_p) {
    const double want = p * (double)total;
    auto reaches = [&](u64 x, u64) { return (double)x >= want; };
    if (!listed) {
      const Found f = find_bin(0, 0, 0, reaches);
      if (f.n + s.count[0][f.j] <= CAP)
        listed = gather([&](double y, u64) { return bin_of(y) <= f.j; });
      else
        find_in_bin(f, reaches);
    }
    if (listed) find_listed(listed, 0, 0, reaches);
    total = min(total, got_sum);
  }
  if (by_m) {
    if (counts && kept_m == 0) {
      // (no sums over all: the list's)
      u64 x = 0, none = 0;
      for (int i = tid; i < listed; i += NTH) {
        const u64 w = weight(sc.log2w(value_of((unsigned)(s.list[i] >> 20))));
        if ((double)w >= mp * 0x1p42) x += w;
      }
      block_scan(s, x, none);
      __syncthreads();
      if (tid == NTH - 1) s.before = x;
      __syncthreads();
      kept_m = s.before;
      __syncthreads();
    }
    total = min(total, max(kept_m, (u64)1 << SCALE));  // (at least the first)
  }
  const double want = u * (double)total;
  auto passes = [&](u64 x, u64) { return (double)x > want; };
  if (listed)
    find_listed(listed, 0, 0, passes);
  else
    find_in_bin(find_bin(0, 0, 0, passes), passes);
  if (tid == 0) {
    a.tokens[r] = (int)(INDEX - (unsigned)(got_place & INDEX));
    if (a.logprob) {
      const double y = sc.log2w(value_of((unsigned)(got_place >> 20)));
      a.logprob[r] = (float)((y + SCALE - log2((double)total)) * 0.6931471805599453);
    }
  }
}

}  // namespace

extern "C" gdn_status gdn_sample(const gdn_sampling* s, int32_t* tokens, float* logprob,
                                 void* stream) {
  if (!s) return GDN_ERR_NULL;
  if (s->dtype != GDN_F32 && s->dtype != GDN_BF16) return GDN_ERR_UNSUPPORTED;
  // a launch holds less than 2^32 threads
  if (s->rows < 1 || s->rows >= 1 << 22 || s->vocab < 1 || s->vocab > 1 << 20) return GDN_ERR_SHAPE;
  const int64_t e = s->dtype == GDN_F32 ? 4 : 2;
  if (s->row_stride > (int64_t)1 << 40 || s->row_stride < -((int64_t)1 << 40)) return GDN_ERR_SHAPE;
  if (!s->logits || !tokens || (!s->u && !s->temperature)) return GDN_ERR_NULL;
  const void* words[] = {s->temperature, s->top_k, s->top_p, s->min_p, s->u, tokens, logprob};
  for (const void* p : words)
    if ((uintptr_t)p & 3) return GDN_ERR_ALIGN;
  if ((uintptr_t)s->logits % e) return GDN_ERR_ALIGN;
  const SampleArgs a{(const unsigned char*)s->logits, s->row_stride * e, s->vocab, s->temperature,
                     s->top_p, s->min_p, s->u, s->top_k, tokens, logprob};
  const hipStream_t st = (hipStream_t)stream;
  const dim3 grid(s->rows), block(NTH);
  if (s->dtype == GDN_F32)
    hipLaunchKernelGGL(k_sample<float>, grid, block, 0, st, a);
  else
    hipLaunchKernelGGL(k_sample<gdn::bf16>, grid, block, 0, st, a);
  return hipGetLastError() == hipSuccess ? GDN_OK : GDN_ERR_HIP;
}
