// The choice of the next token: temperature, top-k, top-p, min-p and a given random
// number.
//
// One workgroup a row.  All that a draw needs are places in the order of falling
// logits: the k-th token, the one where the sum of weights reaches top_p of it, the
// one where it passes u times the sum of what is kept (min_p needs none: what it
// keeps is a prefix too, and the shortest prefix has the smallest sum).  No row is sorted:
//   - with a top_k of few tokens, the k-th largest of the threads' largest logits is a
//     bound that the k largest reach; what reaches it is gathered and sorted;
//   - otherwise, in bf16, the tokens of each of the 2^16 values are counted, weights are found
//     once for a value, and the place among its equals by a second pass over the row;
//   - otherwise a histogram of weights over their logarithm says in which bin a place lies,
//     and the bin's tokens (or all up to there, where they are few) are gathered.
//
// Weights are whole multiples of 2^-42 of the largest (found with an exponential in 64
// bits), so that sums are exact, whatever their order, atomics included, and two
// places that differ are told apart: with weights in 32 bits one draw in 10^5 from a flat
// distribution would be off by a token.
#include <float.h>
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "../../include/gdn_sample.h"
#include "gdn_device.h"

namespace {

using gdn::lane_id;
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned long long u64;
// (a lambda that is called keeps what it refers to in memory)
#define INLINE __attribute__((always_inline))

constexpr int NTH = 1024, NW = NTH / 64;
constexpr int BINS = 2048, CAP = 2048;  // of a histogram; tokens of the list
constexpr int FEW = 512;                // top_k up to which the list is tried first
constexpr int ROUNDS = 6;               // of the search for a bound of the k largest
constexpr double LOWEST = -43;          // log2 of the least weight that counts
constexpr int SCALE = 42;               // weights are multiples of 2^-SCALE
// log2 of the weights that have bins of their own: with 16 one draw in 200 from a normal
// distribution (of 2.5 at T = 1, 128,000 tokens) was from the last bin, and took another histogram
constexpr double RANGE = 22;
constexpr unsigned INDEX = (1u << 20) - 1;
// bf16 logits as keys, in their order: that of the least finite one, of infinity; words of two counts
constexpr unsigned LOW_KEY = 0x80, INF_KEY = 0xff80;
constexpr int WORDS = 1 << 15;

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
__device__ inline float value_at(u64 place) { return value_of((unsigned)(place >> 20)); }
// The upper half of rank_of(x) where x is a bf16 value.
__device__ inline unsigned key_of(float x) {
  const unsigned b = __float_as_uint(x) >> 16, key = b & 0x8000u ? 0xffffu - b : b | 0x8000u;
  return key + (key == 0x7fff);
}
__device__ inline float value_of_key(unsigned key) {
  return __uint_as_float((key & 0x8000u ? key & 0x7fffu : 0xffffu - key) << 16);
}

struct Common {
  double power[128];  // 2^(SCALE + j / 128)
  u64 part[2][NW];
  u64 votes[ROUNDS];
  unsigned listed;
  int at;
  u64 before, nbefore, lo, hi;
};
template <class E> struct Shared : Common {
  union {
    struct {
      unsigned count[BINS];
      // (the last bin's, of the many small weights, in a place for each lane)
      u64 sum[BINS - 1 + 64];
      u64 list[CAP];  // places
      u64 run[CAP];   // sums of weights up to each
    };
    u32x4 words[sizeof(E) == 2 ? WORDS / 4 : 1];  // counts of bf16 keys, two to a word
  };
};

struct Scale {
  double top;  // the largest logit
  double per;  // log2(e) / T
  // (an infinity: so far above all that is finite that nothing of that has weight)
  __device__ Scale(float x, float T)
      : top(x == INFINITY ? 1e39 : (double)x),
        per(x == INFINITY ? 1e300 : 1.4426950408889634074 / (double)T) {}
  // log2 of the weight; NONE where there is none (NaN, or below LOWEST)
  __device__ double log2w(float x) const {
    return __builtin_fmin(__builtin_fmax(((double)x - top) * per, NONE), 0.0);
  }
  static constexpr double NONE = -64;
};

// 2^y in units of 2^-SCALE, y <= 0 (0 at NONE), from a table of 2^(j / 128) and the Taylor series
// of the rest, whose first term left out is 2.2e-12 at most.
__device__ inline u64 weight(const Common& s, double y) {
  // the sum's last bits are round(128 y)
  const double shift = 0x1.8p45, z = y + shift, f = y - (z - shift);
  const int i = (int)__double_as_longlong(z);
  double p = __builtin_fma(f, 0.05550410866482158, 0.2402265069591007);
  p = __builtin_fma(p, f, 0.6931471805599453);
  p = __builtin_fma(p, f, 1.0);
  const long long t = __double_as_longlong(s.power[i & 127]) + ((long long)((i << 13) & 0xfff00000) << 32);
  // rounded to a whole number by the addition
  return (u64)__double_as_longlong(__builtin_fma(p, __longlong_as_double(t), 0x1p52)) &
         0xfffffffffffffull;
}

// Inclusive prefix sums over the 64 lanes (as in rows of 16 lanes, then across them).
template <int CTRL, int ROWS> __device__ inline u64 dpp_or_zero(u64 x) {
  const int lo = __builtin_amdgcn_update_dpp(0, (int)x, CTRL, ROWS, 0xf, false);
  const int hi = __builtin_amdgcn_update_dpp(0, (int)(x >> 32), CTRL, ROWS, 0xf, false);
  return (u64)(unsigned)hi << 32 | (unsigned)lo;
}
__device__ inline u64 wave_scan(u64 x) {
  x += dpp_or_zero<0x111, 0xf>(x);  // row_shr 1, 2, 4, 8
  x += dpp_or_zero<0x112, 0xf>(x);
  x += dpp_or_zero<0x114, 0xf>(x);
  x += dpp_or_zero<0x118, 0xf>(x);
  x += dpp_or_zero<0x142, 0xa>(x);  // row_bcast 15, to rows 1 and 3
  x += dpp_or_zero<0x143, 0xc>(x);  // row_bcast 31, to rows 2 and 3
  return x;
}

// Inclusive sums over the workgroup's threads of two values at a time.
__device__ inline void block_scan(Common& s, u64& x, u64& c) {
  const int w = threadIdx.x >> 6;
  x = wave_scan(x);
  c = wave_scan(c);
  __syncthreads();
  if (lane_id() == 63) {
    s.part[0][w] = x;
    s.part[1][w] = c;
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < NW - 1; ++i) {
    x += i < w ? s.part[0][i] : 0;
    c += i < w ? s.part[1][i] : 0;
  }
}
// The sum over the workgroup's threads, for all of them.
__device__ inline u64 block_sum(Common& s, u64 x) {
  x = wave_scan(x);
  __syncthreads();
  if (lane_id() == 63) s.part[0][threadIdx.x >> 6] = x;
  __syncthreads();
  u64 all = 0;
#pragma unroll
  for (int i = 0; i < NW; ++i) all += s.part[0][i];
  return all;
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

// Bound by instructions for each token, not by HBM.  64 rows of 100,003 in fp32 (25.6 MB; a copy
// takes 4.9 us): top_p 72 us, the histogram's 64-bit exponentials and sums; top_k of 50 24, the
// likeliest alone 11.  256 rows of 128,000 in bf16 (65.5 MB, 12.6): top_p 58 us (102 by
// the histogram; twice the row 87, so half of it is passes over the tokens, half the
// values' weights and the searches), top_k of 50 34, the likeliest 16.  Equal logits meet in one LDS
// word: 64 flat rows of 100,003 in fp32 265 us, 256 of 128,000 in bf16 400 (their counts
// pass 16 bits, and the histogram follows).  All paths are one kernel at 128 registers: 80 (fp32) and 112
// (bf16) bytes a lane are in scratch memory.
template <class E> __global__ __launch_bounds__(NTH) void k_sample(SampleArgs a) {
  constexpr int N = Row<E>::N;
  __shared__ Shared<E> s;
  const int tid = threadIdx.x, wave = tid >> 6, r = blockIdx.x;
  const Row<E> row(a.logits + r * a.stride, a.vocab);
  const float T = a.temperature ? a.temperature[r] : 1.f;
  const int k = a.top_k ? a.top_k[r] : 0;
  const double p = a.top_p ? (double)a.top_p[r] : 1.0, mp = a.min_p ? (double)a.min_p[r] : 0.0;
  const float un = a.u ? a.u[r] : 0.f;
  // f(x, index) for this thread's tokens; two loads ahead.  Whole waves take part.
  auto each = [&](auto&& f) INLINE {
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

  const double u = un > 0.f ? fmin((double)un, 1 - 0x1p-24) : 0.0;
  const bool by_k = k > 0 && k < a.vocab, by_p = p < 1.0, by_m = mp > 0.0;
  // What is looked for: the token with which the count reaches n, the sum `want`, or passes it.
  enum Kind { COUNT, REACHES, PASSES };
  struct Target {
    Kind kind;
    u64 n;
    double want;
    __device__ bool operator()(u64 sum, u64 count) const {
      if (kind == COUNT) return count >= n;
      return kind == REACHES ? (double)sum >= want && sum > 0 : (double)sum > want;
    }
  };
      if (tid < 128) {
        // 2^(1/2), 2^(1/4), .. 2^(1/128)
        constexpr double root[7] = {1.4142135623730951, 1.189207115002721,  1.0905077326652577,
                                    1.0442737824274138, 1.0218971486541166, 1.0108892860517005,
                                    1.0054299011128027};
        double p = 0x1p42;
  #pragma unroll
        for (int b = 0; b < 7; ++b) p *= tid >> (6 - b) & 1 ? root[b] : 1.0;
        s.power[tid] = p;
      }

  // ---- bf16: a row has few different logits, and counts of each are all that a draw needs
  if constexpr (sizeof(E) == 2)
    if (T > 0.f && !(by_k && k <= FEW)) {
      unsigned* const words = reinterpret_cast<unsigned*>(s.words);
      for (int i = tid; i < WORDS / 4; i += NTH) s.words[i] = u32x4{0, 0, 0, 0};
      __syncthreads();
      unsigned top = 0, low = 0, counted = 0;
      each([&](float x, int) INLINE {
        const unsigned key = key_of(x);
        const bool in = key - (LOW_KEY + 1) < INF_KEY - LOW_KEY;
        // (the least finite value stands for all that is masked: counted apart)
        low += (unsigned)__popcll(__ballot(key == LOW_KEY));
        counted += (unsigned)__popcll(__ballot(in));
        if (in) {
          top = max(top, key);
          atomicAdd(&words[key >> 1], key & 1 ? 0x10000u : 1u);
        }
      });
      if (low) top = max(top, LOW_KEY);
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) top = max(top, (unsigned)__shfl_xor((int)top, d, 64));
      if (lane_id() == 0) {
        s.part[0][wave] = top;
        s.part[1][wave] = (u64)low << 32 | counted;
      }
      __syncthreads();
      low = counted = 0;
#pragma unroll
      for (int i = 0; i < NW; ++i) {
        top = max(top, (unsigned)s.part[0][i]);
        low += (unsigned)(s.part[1][i] >> 32);
        counted += (unsigned)s.part[1][i];
      }
      if (top == 0) {
        if (tid == 0) {
          a.tokens[r] = -1;
          if (a.logprob) a.logprob[r] = -INFINITY;
        }
        return;
      }
      const Scale sc(value_of_key(top), T);
      // A thread has OWN words, the first thread those of the largest keys: the upper half of a
      // word is the larger key.  (Each lane begins at another of its words: another bank.)
      constexpr int OWN = WORDS / NTH;
      auto count = [&](unsigned key) INLINE {
        return key == LOW_KEY ? low : words[key >> 1] >> (key & 1 ? 16 : 0) & 0xffffu;
      };
      u64 sum = 0, kept = 0;
      unsigned n = 0, stored = 0;
#pragma unroll 2
      for (int step = 0; step < OWN; ++step) {
        const int at = WORDS - 1 - tid * OWN - ((step + lane_id()) & (OWN - 1));
        const unsigned c = words[at];
        stored += (c >> 16) + (c & 0xffffu);
        if (!__ballot(c != 0 || (low && at == LOW_KEY / 2))) continue;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const unsigned key = 2 * at + 1 - i;
          const unsigned m = i == 0 ? c >> 16 : key == LOW_KEY ? low : c & 0xffffu;
          const double y = sc.log2w(value_of_key(key));
          const u64 w = weight(s, y), all = w * m;
          sum += all;
          n += y >= LOWEST ? m : 0;
          if ((double)w >= mp * 0x1p42) kept += all;
        }
      }
      u64 upto = sum, both = (u64)stored << 32 | n;
      block_scan(s, upto, both);
      const u64 nupto = (unsigned)both;
      if (tid == NTH - 1) {
        s.before = upto;
        s.nbefore = both >> 32;
      }
      if (by_m) kept = block_sum(s, kept);
      __syncthreads();
      u64 total = s.before;
      const bool fits = s.nbefore == counted;  // no count has passed 16 bits
      __syncthreads();
      if (fits) {
        // The key of the token that the test first holds with (the last with any weight if none
        // does), which of the key's tokens it is, and the sum with it.
        u64 got = 0;
        auto find = [&](const Target& test) INLINE {
          if (tid == 0) s.at = -1;
          __syncthreads();
          const bool is = test(upto, nupto), was = tid > 0 && test(upto - sum, nupto - n);
          if (is && !was) s.at = tid;
          __syncthreads();
          int at = s.at;
          const bool none = at < 0;
          __syncthreads();
          if (none) {
            if (sum) atomicMax(&s.at, tid);
            __syncthreads();
            at = s.at;
          }
          if (tid == at) {
            s.before = upto - sum;
            s.nbefore = nupto - n;
          }
          __syncthreads();
          if (wave == 0) {  // a lane for each of the thread's keys
            const unsigned key = 2 * (WORDS - at * OWN) - 1 - lane_id();
            const double y = sc.log2w(value_of_key(key));
            const u64 one = weight(s, y), most = y >= LOWEST ? count(key) : 0;
            const u64 b = s.before + wave_scan(one * most) - one * most;
            const u64 nb = s.nbefore + wave_scan(most) - most;
            const u64 hits = none ? 0 : __ballot(test(b + one * most, nb + most));
            const u64 some = __ballot(one * most != 0);
            if (lane_id() == (hits ? __ffsll(hits) - 1 : 63 - __clzll(some))) {
              u64 lo = hits ? 1 : most, hi = most;  // the least with which the test holds
              while (lo < hi) {
                const u64 mid = (lo + hi) >> 1;
                if (test(b + one * mid, nb + mid)) hi = mid; else lo = mid + 1;
              }
              s.at = (int)key;
              s.lo = hi;
              s.hi = most;
              s.before = b + one * hi;
            }
          }
          __syncthreads();
          got = s.before;
        };
#pragma unroll 1
        for (int step = 0; step < 3; ++step) {  // the k-th, the one that reaches top_p, the drawn one
          if (step == 0 ? !by_k : step == 1 ? !by_p : false) continue;
          Target t{COUNT, (u64)max(k, 0), 0};
          if (step == 1) t = {REACHES, 0, p * (double)total};
          if (step == 2) {
            if (by_m) total = min(total, max(kept, (u64)1 << SCALE));  // (at least the first)
            t = {PASSES, 0, u * (double)total};
          }
          find(t);
          if (step < 2) total = min(total, got);
          __syncthreads();
        }
        const float x = value_of_key((unsigned)s.at);
        const unsigned nth = (unsigned)s.lo, most = (unsigned)s.hi;
        if (tid == 0 && a.logprob)
          a.logprob[r] = (float)((sc.log2w(x) + SCALE - log2((double)total)) * 0.6931471805599453);
        // the nth token of this value
        if (most <= 512) {
          if (tid == 0) s.listed = 0;
          __syncthreads();
          each([&](float y, int i) INLINE {
            if (y != x) return;
            const unsigned at = atomicAdd(&s.listed, 1u);
            if (at < CAP) s.list[at] = (u64)i;
          });
          __syncthreads();
          if (tid < (int)most) {
            const u64 mine = s.list[tid];
            unsigned before = 0;
#pragma unroll 8
            for (unsigned i = 0; i < most; ++i) before += s.list[i] < mine;
            if (before + 1 == nth) a.tokens[r] = (int)mine;
          }
          return;
        }
        // by counts: a wave has a sixteenth of the row
        const int per = (row.pieces + NW - 1) / NW, from = wave * per, to = min(from + per, row.pieces);
        auto equal = [&](const u32x4& y) INLINE {
          unsigned c = 0;
#pragma unroll
          for (int e = 0; e < N; ++e) c += Row<E>::get(y, e) == x;
          return c;
        };
        unsigned mine = 0;
#pragma unroll 2
        for (int j = from + lane_id(); j < to; j += 64) mine += equal(row.load(j));
        const u64 sums = wave_scan(mine);
        if (lane_id() == 63) s.part[0][wave] = sums;
        __syncthreads();
        unsigned before = 0;
        int w = 0;
        while (w < NW - 1 && before + (unsigned)s.part[0][w] < nth) before += (unsigned)s.part[0][w++];
        if (wave == w)
          for (int j = from; j < to; j += 64) {
            const u32x4 y = j + lane_id() < to ? row.load(j + lane_id()) : u32x4{~0u, ~0u, ~0u, ~0u};
            const unsigned c = equal(y), upto = before + (unsigned)wave_scan(c);
            if (upto >= nth && upto - c < nth) {
              unsigned left = nth - (upto - c);
#pragma unroll
              for (int e = 0; e < N; ++e)
                if (Row<E>::get(y, e) == x && --left == 0)
                  a.tokens[r] = (j + lane_id()) * N + e - row.off;
            }
            before = (unsigned)__shfl((int)upto, 63);
            if (before >= nth) break;
          }
        return;
      }
      __syncthreads();  // many equal logits: as below
    }

  // the largest, the lowest index first; the smallest
  float mine = -INFINITY, low = INFINITY;
  u64 best = 0;
  {
    int at = -1;
    each([&](float x, int i) INLINE {
      low = fminf(low, x);
      if (x > mine) mine = x, at = i;
    });
    if (at >= 0) best = place_of(mine, at);
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      best = max(best, (u64)__shfl_xor(best, d, 64));
      low = fminf(low, __shfl_xor(low, d, 64));
    }
    if (lane_id() == 0) {
      s.part[0][wave] = best;
      s.part[1][wave] = __float_as_uint(low);
    }
    if (tid < ROUNDS) s.votes[tid] = 0;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < NW; ++i) {
      best = max(best, s.part[0][i]);
      low = fminf(low, __uint_as_float((unsigned)s.part[1][i]));
    }
  }
  if (best == 0 || !(T > 0.f)) {  // nothing to draw, or no draw
    if (tid == 0) {
      a.tokens[r] = best ? (int)(INDEX - (unsigned)(best & INDEX)) : -1;
      if (a.logprob) a.logprob[r] = best ? 0.f : -INFINITY;
    }
    return;
  }
  const Scale sc(value_at(best), T);
  // Gathers the tokens for which in(x, index) holds; how many they are (they are all in the list
  // if that is at most CAP).
  auto gather = [&](auto&& in) INLINE {
    if (tid == 0) s.listed = 0;
    __syncthreads();
    each([&](float x, int i) INLINE {
      if (in(x, i)) {
        const unsigned at = atomicAdd(&s.listed, 1u);
        if (at < CAP) s.list[at] = place_of(x, i);
      }
    });
    __syncthreads();
    const int n = (int)s.listed;
    __syncthreads();
    return n;
  };
  // Sorts the list's n tokens, and sums their weights up to each from `base` on.
  auto sort = [&](int n, u64 base) INLINE {
    if (n <= 512) {  // each finds its place by comparing with all others
      const u64 x = tid < n ? s.list[tid] : 0;
      int at = 0;
      if (tid < n)
#pragma unroll 8
        for (int i = 0; i < n; ++i) at += s.list[i] > x;
      __syncthreads();
      if (tid < n) s.list[at] = x;
      __syncthreads();
    } else {
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
    }
    u64 w[2], none = 0;
#pragma unroll
    for (int i = 0; i < 2; ++i)
      w[i] = 2 * tid + i < n ? weight(s, sc.log2w(value_at(s.list[2 * tid + i]))) : 0;
    u64 x = w[0] + w[1];
    block_scan(s, x, none);
    x += base;
    s.run[2 * tid] = x - w[1];
    s.run[2 * tid + 1] = x;
    __syncthreads();
  };
  // The first token of the sorted list up to which the test holds (the last if none does): its
  // place, and the sum with it.
  u64 got_place = 0, got_sum = 0;
  auto find_listed = [&](int n, u64 nbase, const Target& test) INLINE {
    if (tid == 0) s.at = max(n - 1, 0);
    __syncthreads();
    bool was = tid > 0 && 2 * tid <= n && test(s.run[2 * tid - 1], nbase + 2 * tid);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int j = 2 * tid + i;
      const bool is = j < n && test(s.run[j], nbase + j + 1);
      if (is && !was) s.at = j;
      was = is;
    }
    __syncthreads();
    got_place = s.list[s.at];
    got_sum = s.run[s.at];
    __syncthreads();
  };

  u64 total = 0;  // of the weights that are kept
  auto put = [&]() INLINE {
    if (tid) return;
    a.tokens[r] = (int)(INDEX - (unsigned)(got_place & INDEX));
    if (a.logprob) {
      const double y = sc.log2w(value_at(got_place));
      a.logprob[r] = (float)((y + SCALE - log2((double)total)) * 0.6931471805599453);
    }
  };

  // ---- few tokens, by a bound that the k largest reach
  if (by_k && k <= FEW && value_at(best) < INFINITY) {
    // A bound that the largest of at least k threads reach, and of not many more: five values
    // at a time between the ends, 11 bits of a word for the count of each.  The first bound is one
    // that all tokens with a weight reach: the row's lowest logit as it is, or (half a power below
    // LOWEST) where the temperature ends the weights.  A difference rounded and taken from
    // the top again may lie above the lowest logit, and lose it.  Both ends are finite, and
    // their difference, which may not be, is not formed: of -infinity and the largest float
    // beside an enormous temperature, too, the bounds are numbers.
    float least = fmaxf(fmaxf(low, -FLT_MAX), (float)(sc.top + (LOWEST - 0.5) / sc.per));
    float end = (float)sc.top;
#pragma unroll 1
    for (int i = 0; i < ROUNDS; ++i) {
      float bound[5];  // (what is counted and what is kept are the same floats)
      const float step = end * (1 / 6.f) - least * (1 / 6.f);
      u64 n = 0;
#pragma unroll
      for (int c = 0; c < 5; ++c) {
        bound[c] = least + step * (c + 1);
        n |= (u64)__popcll(__ballot(mine >= bound[c])) << (11 * c);
      }
      if (lane_id() == 0) atomicAdd(&s.votes[i], n);
      __syncthreads();
      n = s.votes[i];
      unsigned most = 1 << 30;
      bool over = false;
#pragma unroll
      for (int x = 0; x < 5; ++x) {
        const unsigned m = (unsigned)(n >> (11 * x)) & 2047;
        if (m >= (unsigned)k) {  // the last that k reach
          least = bound[x], most = m;
        } else if (!over) {
          end = bound[x], over = true;
        }
      }
      if (most <= 2 * (unsigned)k + 64) break;
    }
    const int n = gather([&](float x, int) INLINE { return x >= least; });
    if (n <= CAP) {
      sort(n, 0);
      // the k-th, the one that reaches top_p, the drawn one
#pragma unroll 1
      for (int step = 0; step < 3; ++step) {
        if (step == 1 && !by_p) continue;
        Target t{COUNT, (u64)k, 0};
        if (step == 1) t = {REACHES, 0, p * (double)total};
        if (step == 2 && by_m) {
          u64 x = 0;
          for (int i = tid; i < n; i += NTH) {
            const u64 w = s.run[i] - (i ? s.run[i - 1] : 0);
            if ((double)w >= mp * 0x1p42) x += w;
          }
          total = min(total, max(block_sum(s, x), (u64)1 << SCALE));  // (at least the first)
        }
        if (step == 2) t = {PASSES, 0, u * (double)total};
        find_listed(n, 0, t);
        if (step < 2) total = got_sum;
      }
      return put();
    }
  }

  int listed = 0;  // tokens of the list, if it holds all that can be kept
  u64 kept_m = 0;
  // ---- otherwise by a histogram: bins of equal width in log2 of the weight, from `first` on, as
  // fine as the row's range has it; the last takes all that is below
  double first = 0, fine = 0;
  auto binned = [](double y, double first, double fine) INLINE {
    return (int)fmax(0.0, fmin((first - y) * fine, BINS - 1.0));
  };
  auto bin_of = [&](double y) INLINE { return binned(y, first, fine); };
  // Sums of the weights for which bin_if(x, index, y) is not negative, and their counts if by_k.
  auto histogram = [&](auto&& bin_if) INLINE {
    for (int i = tid; i < BINS - 1 + 64; i += NTH) s.sum[i] = 0;
    for (int i = tid; i < BINS; i += NTH) s.count[i] = 0;
    __syncthreads();
    auto fill = [&](auto counts, auto keeps) INLINE {
      each([&](float x, int i) INLINE {
        const double y = sc.log2w(x);
        const int b = bin_if(x, i, y);
        const u64 w = weight(s, y);
        if (b >= 0) atomicAdd(&s.sum[b < BINS - 1 ? b : BINS - 1 + lane_id()], w);
        if constexpr (decltype(keeps)::value)
          if ((double)w >= mp * 0x1p42) kept_m += w;
        if constexpr (decltype(counts)::value)
          if (b >= 0 && y >= LOWEST) atomicAdd(&s.count[b], 1u);
      });
    };
    constexpr std::true_type yes{};
    constexpr std::false_type no{};
    if (by_k)
      by_m ? fill(yes, yes) : fill(yes, no);
    else
      by_m ? fill(no, yes) : fill(no, no);
    __syncthreads();
    if (wave == 0) {
      const u64 x = wave_scan(s.sum[BINS - 1 + tid]);
      if (tid == 63) s.sum[BINS - 1] = x;
    }
    __syncthreads();
  };
  // The first bin up to which, with base and nbase before the first, the test holds (the
  // last with any weight if none does); s.before and s.nbefore then are before it.
  auto find_bin = [&](u64 base, u64 nbase, const Target& test) INLINE {
    u64 x[2], c[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) x[i] = s.sum[2 * tid + i], c[i] = s.count[2 * tid + i];
    u64 sx = x[0] + x[1], sn = c[0] + c[1];
    block_scan(s, sx, sn);
    if (tid == 0) s.at = -1;
    __syncthreads();
    const u64 before = base + sx - x[0] - x[1], n = nbase + sn - c[0] - c[1];
    const bool was = test(before, n);
    const bool mid = test(before + x[0], n + c[0]), end = test(before + x[0] + x[1], n + c[0] + c[1]);
    if (end && !was) s.at = mid ? 2 * tid : 2 * tid + 1;
    __syncthreads();
    int at = s.at;
    __syncthreads();
    if (at < 0) {
      if (x[0] + x[1]) atomicMax(&s.at, x[1] ? 2 * tid + 1 : 2 * tid);
      __syncthreads();
      at = max(s.at, 0);
      __syncthreads();
    }
    if (at >> 1 == tid) {
      s.before = before + (at & 1 ? x[0] : 0);
      s.nbefore = n + (at & 1 ? c[0] : 0);
    }
    __syncthreads();
    return at;
  };
  bool fresh = false;  // the histogram of all tokens stands
  auto whole = [&]() INLINE {
    first = 0;
    const double range = fmin(RANGE, fmax(0x1p-20, -sc.log2w(low)));
    fine = (BINS - 1) / range;
    kept_m = 0;
    histogram([&](float, int, double y) INLINE { return bin_of(y); });
    if (by_m) kept_m = block_sum(s, kept_m);
    fresh = true;
  };
  // The token of bin j that the search is for.
  auto find_in_bin = [&](int j, const Target& test) INLINE {
    u64 base = s.before, nbase = s.nbefore, lo = 0, hi = ~0ull;
    // logits that can be in the bin: a hair beyond its ends
    float above, below;
    auto ends = [&]() INLINE {
      const double top = sc.top, hi = top + (first - j / fine) / sc.per,
                   lo = top + (first - (j + 1) / fine) / sc.per;
      above = j == 0 ? INFINITY : (float)(hi + 1e-6 * (1 + fabs(top) + fabs(hi)));
      below = j == BINS - 1 ? -INFINITY : (float)(lo - 1e-6 * (1 + fabs(top) + fabs(lo)));
      if (value_at(best) == INFINITY) above = INFINITY, below = -INFINITY;
    };
    ends();
    auto in = [&](float x, int i) INLINE {
      if (!(x >= below && x <= above)) return false;
      const double y = sc.log2w(x);
      if (y < LOWEST || bin_of(y) != j) return false;
      const u64 c = place_of(x, i);
      return c >= lo && c <= hi;
    };
    int n = gather(in);
    if (n > CAP) {
      const u64 keep = kept_m;
      fresh = false;
      // the last bin: its range in finer bins
      if (j == BINS - 1) {
        const double from = first - j / fine;
        histogram([&](float, int, double y) INLINE {
          if (y < LOWEST || bin_of(y) != j) return -1;
          return binned(y, from, (BINS - 1) / (0.5 - LOWEST - RANGE));
        });
        j = find_bin(base, nbase, test);
        base = s.before;
        nbase = s.nbefore;
        const double old_first = first, old_fine = fine;
        first = from;
        fine = (BINS - 1) / (0.5 - LOWEST - RANGE);
        ends();
        if (j == 0) above = INFINITY;
        n = gather([&](float x, int i) INLINE {
          if (!(x >= below && x <= above)) return false;
          const double y = sc.log2w(x);
          return y >= LOWEST && binned(y, old_first, old_fine) == BINS - 1 && bin_of(y) == j;
        });
        if (n > CAP) {
          // (what follows tells the tokens by their places alone)
          if (tid == 0) s.lo = ~0ull, s.hi = 0;
          __syncthreads();
          u64 mlo = ~0ull, mhi = 0;
          each([&](float x, int i) INLINE {
            const double y = sc.log2w(x);
            if (y < LOWEST || binned(y, old_first, old_fine) != BINS - 1 || bin_of(y) != j) return;
            const u64 c = place_of(x, i);
            mlo = min(mlo, c);
            mhi = max(mhi, c);
          });
          atomicMin(&s.lo, mlo);
          atomicMax(&s.hi, mhi);
          __syncthreads();
          lo = s.lo;
          hi = s.hi;
        }
      } else {
        if (tid == 0) s.lo = ~0ull, s.hi = 0;
        __syncthreads();
        u64 mlo = ~0ull, mhi = 0;
        each([&](float x, int i) INLINE {
          if (!in(x, i)) return;
          const u64 c = place_of(x, i);
          mlo = min(mlo, c);
          mhi = max(mhi, c);
        });
        atomicMin(&s.lo, mlo);
        atomicMax(&s.hi, mhi);
        __syncthreads();
        lo = s.lo;
        hi = s.hi;
      }
      // many equal, or nearly so: their places, which are all different, are cut ever finer
      while (n > CAP) {
        int shift = 0;
        while ((hi - lo) >> shift >= BINS) ++shift;
        histogram([&](float x, int i, double) INLINE {
          const u64 c = place_of(x, i);
          return x == x && c >= lo && c <= hi ? (int)((hi - c) >> shift) : -1;
        });
        const int g = find_bin(base, nbase, test);
        base = s.before;
        nbase = s.nbefore;
        hi -= (u64)g << shift;
        const u64 width = ((u64)1 << shift) - 1;
        if (hi - lo > width) lo = hi - width;
        __syncthreads();
        n = gather([&](float x, int i) INLINE {
          const u64 c = place_of(x, i);
          return x == x && c >= lo && c <= hi;
        });
      }
      kept_m = keep;
    }
    sort(n, base);
    find_listed(n, nbase, test);
  };
  // the same for all tokens, as a list where those up to there are few
  auto find = [&](auto&& test, bool list) INLINE {
    if (!fresh) whole();
    const int j = find_bin(0, 0, test);
    if (list && j < BINS - 1) {
      // how many that are: a bin's tokens weigh alike
      float n = 0;
#pragma unroll
      for (int i = 0; i < 2; ++i)
        if (2 * tid + i <= j) n += (float)s.sum[2 * tid + i] * __builtin_amdgcn_exp2f((2 * tid + i + 0.5f) / (float)fine - SCALE);
      if (block_sum(s, (u64)(n * 1024)) < (u64)500 * 1024) {  // (quickly sorted)
        const int n = gather([&](float x, int) INLINE { return bin_of(sc.log2w(x)) <= j; });
        if (n <= CAP) {
          listed = n;
          sort(n, 0);
          find_listed(n, 0, test);
          return;
        }
      }
    }
    find_in_bin(j, test);
  };

  whole();
  if (!by_k) total = block_sum(s, s.sum[2 * tid] + s.sum[2 * tid + 1]);
#pragma unroll 1
  for (int step = 0; step < 3; ++step) {  // as above
    if (step == 0 ? !by_k : step == 1 ? !by_p : false) continue;
    Target t{COUNT, (u64)max(k, 0), 0};
    if (step == 1) t = {REACHES, 0, p * (double)total};
    if (step == 2) {
      if (by_m) total = min(total, max(kept_m, (u64)1 << SCALE));  // (at least the first)
      t = {PASSES, 0, u * (double)total};
    }
    if (listed)
      find_listed(listed, 0, t);
    else
      find(t, step == 1);
    if (step < 2) total = step == 0 ? got_sum : min(total, got_sum);
  }
  put();
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
