// Rotary positions, storing new tokens in a paged cache, and the management of
// its pages.  All of it moves data once and computes little: bound by HBM, and
// by launches where there is little to move.
#include <hip/hip_runtime.h>
#include <math.h>

#include <algorithm>

#include "gdn_device.h"
#include "gdn_paged_kernels.h"

namespace gdn {

// ------------------------------------------------------------------ rotation

namespace {

// cos and sin of a fraction of a turn, |f| <= 1/2.  bf16: the hardware's
// v_sin and v_cos (absolute error about 2e-7 at this range... far below a
// bf16 rounding); fp32: the library functions, correct to an ulp or two.
template <class E> __device__ inline float2 cos_sin(float f) {
  if constexpr (sizeof(E) == 2)
    return make_float2(__builtin_amdgcn_cosf(f), __builtin_amdgcn_sinf(f));
  float s, c;
  sincospif(2.f * f, &s, &c);
  return make_float2(c, s);
}

template <class E> struct Pc {  // 16 bytes of channels
  static constexpr int N = 16 / sizeof(E);
  E e[N];
};
template <class E> __device__ inline Pc<E> load_piece(const unsigned char* p) {
  const uint4 x = *reinterpret_cast<const uint4*>(p);
  return *reinterpret_cast<const Pc<E>*>(&x);
}
template <class E> __device__ inline void store_piece(unsigned char* p, const Pc<E>& x) {
  *reinterpret_cast<uint4*>(p) = *reinterpret_cast<const uint4*>(&x);
}

}  // namespace

constexpr int ROT_TOKENS = 4;                  // most tokens of a workgroup
constexpr unsigned ROT_GRID = 1 << 22;         // workgroups in a grid's first direction
constexpr int ROT_TABLE = ROT_TOKENS * 256 / 2;  // angles it holds (d <= 256)

// Rotation of pairs: y1 = s (x1 cos a - x2 sin a), y2 = s (x2 cos a + x1 sin a), a the
// token's position times the pair's frequency, reduced to a turn in 64 bits; the
// gradient is the rotation by -a.  Bound by HBM: each row is read once and
// written once.  A workgroup takes a.per tokens: the cos and sin of their angles
// go into LDS, once for all heads, with each token's place, while the first rows of
// q, k (and v) are on their way.  Four tokens and two rows of a thread at a time:
// 55,700 tokens of 16 + 4 heads, d = 128, bf16, 103 us a direction, 5.5 TB/s (16 tokens,
// four rows 117; 2 tokens 108; the loads after the angles 119 with 16 and four); prompts
// into the cache, 137 MB, 25 us (27.5), after a cache-evicting write 46 (54; a copy
// of as many bytes 39).  A token each for 256 sequences 7 us a call, 4.6 in a replayed
// graph.
//   WIDE: a unit is one 16-byte piece (interleaved pairs lie inside one) or, in
//   the layout of halves, the two pieces that hold the two sides of its pairs,
//   where those start at multiples of 16 bytes; else a unit is one piece, and the
//   other side of its pairs is read element by element.
//   LIST: there is a list of sequences to leave alone.  The look at it, one more load of
//   every thread, takes 0.2 of the 4.6 us above and 0.8 of the prompts' 25, which calls
//   without one do not pay.
template <class E, bool WIDE, bool LIST>
__global__ __launch_bounds__(256) void k_rotate(RotateArgs a) {
  constexpr int N = Pc<E>::N;
  __shared__ float2 cs[ROT_TABLE];
  __shared__ int64_t kat[ROT_TOKENS];  // where the token's k and v go; -1: nowhere
  const int half = a.rot / 2;
  // (in a grid of several rows the last may end past the tokens, within 2^31 + 2^24; a
  // branch there would hold up the loads of the other arguments)
  const unsigned group = blockIdx.y * ROT_GRID + blockIdx.x, total = a.tok.total;
  const int t0 = (int)min(group * a.per, total), nt = min(a.per, (int)total - t0);
  const bool halves = a.layout == 0;
  // units of a row, the first `turn` of them the two sides of pairs
  const int turn = WIDE && halves ? half / N : 0, units = a.d / N - turn;

  // A thread keeps its unit p and steps through the rows (of q and k, or of v) of
  // the workgroup's tokens, BATCH at a time (a token nt or past it: none).
  constexpr int BATCH = 2;
  struct Walk {
    int H, p, t, h, dt, dh;
    __device__ Walk(int tid, int heads, int per_row, int nt) {
      H = heads;
      const int step = 256 / per_row;  // rows a pass; the threads left over idle
      p = tid % per_row;
      const int row = tid / per_row;
      dt = step / H;
      dh = step - dt * H;
      t = row < step ? row / H : nt;
      h = row % H;
    }
    __device__ void next(int (&ts)[BATCH], int (&hs)[BATCH]) {
#pragma unroll
      for (int j = 0; j < BATCH; ++j) {
        ts[j] = t;
        hs[j] = h;
        t += dt;
        h += dh;
        if (h >= H) {
          h -= H;
          ++t;
        }
      }
    }
  };
  const int nq = a.q.data ? a.Hq : 0, nk = a.k.data ? a.Hk : 0;
  // (plain values: a choice between two structures would put them in memory)
  unsigned char *const qd = a.q.data, *const kd = a.k.data - nq * a.k.hs;
  const int64_t qts = a.q.ts, qhs = a.q.hs, kts = a.k.ts, khs = a.k.hs;
  auto from = [&](int tt, int h) {
    const bool is_q = h < nq;
    return (is_q ? qd : kd) + (int64_t)(t0 + tt) * (is_q ? qts : kts) + h * (is_q ? qhs : khs);
  };
  unsigned char* const qod = a.q_out.data;
  const int64_t qots = a.q_out.ts, qohs = a.q_out.hs;
  const int64_t kots = a.append ? 0 : a.k_out.ts, kohs = a.append ? a.cache.head : a.k_out.hs;
  unsigned char* const kod = (a.append ? a.cache.k : a.k_out.data) - nq * kohs;
  auto to = [&](int tt, int h) {
    const bool is_q = h < nq;
    unsigned char* r =
        (is_q ? qod : kod) + (int64_t)(t0 + tt) * (is_q ? qots : kots) + h * (is_q ? qohs : kohs);
    return a.append && !is_q ? r + kat[tt] : r;
  };
  Walk wq(threadIdx.x, nq + nk, units, nt);
  const int p = wq.p;
  // WIDE: the unit's pieces, its own, or those of both sides of its pairs
  const bool both = WIDE && halves && p < turn;
  const int at1 = (WIDE && halves && p >= turn ? turn + p : p) * 16, at2 = (p + turn) * 16;
  uint4 x1[BATCH], x2[WIDE ? BATCH : 1];
  E other[WIDE ? 1 : BATCH][N];
  int ts[BATCH], hs[BATCH];
  auto load = [&]() {
    wq.next(ts, hs);
#pragma unroll
    for (int j = 0; j < BATCH; ++j) {
      x1[j] = make_uint4(0, 0, 0, 0);
      if constexpr (WIDE) x2[j] = make_uint4(0, 0, 0, 0);
      if (ts[j] < nt) {
        const unsigned char* r = from(ts[j], hs[j]);
        x1[j] = *reinterpret_cast<const uint4*>(r + at1);
        if constexpr (WIDE) {
          if (both) x2[j] = *reinterpret_cast<const uint4*>(r + at2);
        } else {
#pragma unroll
          for (int e = 0; e < N; ++e) {
            const int c = p * N + e;
            other[j][e] =
                c < a.rot ? reinterpret_cast<const E*>(r)[c < half ? c + half : c - half] : to_e<E>(0.f);
          }
        }
      }
    }
  };
  // v from the other end: where there are few tokens, by the waves that have no q
  Walk wv(255 - threadIdx.x, max(a.Hk, 1), a.d / N, nt);
  if (!a.v.data) wv.t = nt;
  uint4 y[BATCH];
  int vt[BATCH], vh[BATCH];
  auto load_v = [&]() {
    wv.next(vt, vh);
#pragma unroll
    for (int j = 0; j < BATCH; ++j) {
      y[j] = make_uint4(0, 0, 0, 0);
      if (vt[j] < nt)
        y[j] = *reinterpret_cast<const uint4*>(a.v.data + (int64_t)(t0 + vt[j]) * a.v.ts +
                                               vh[j] * a.v.hs + wv.p * 16);
    }
  };
  // the first rows are on their way while the angles are found
  load();
  load_v();

  for (int i = threadIdx.x; i < nt * max(half, 1); i += 256) {
    const int tt = half ? i / half : i, j = half ? i - tt * half : 0, t = t0 + tt;
    int pos;
    if (a.positions) {
      pos = a.positions[t];
    } else {
      const int n = seq_of(a.tok, t), q0 = seq_start(a.tok, n);
      pos = t - q0;
      if (a.append) {
        pos += cached<LIST>(a.cache, n) - (seq_start(a.tok, n + 1) - q0);
        if (j == 0) {
          int64_t at = -1;
          if (pos >= 0) {
            const int p = a.cache.table[(int64_t)n * a.cache.max_blocks + (pos >> a.cache.shift)];
            if ((unsigned)p < (unsigned)a.cache.num_pages)
              at = p * a.cache.page + (pos & ((1 << a.cache.shift) - 1)) * a.cache.slot;
          }
          kat[tt] = at;
        }
      }
    }
    if (half) {
      const double f = (double)pos * a.turns[j];
      float2 x = cos_sin<E>((float)(f - rint(f)));
      x.x *= a.scale;
      x.y *= a.scale * a.sign;
      cs[i] = x;
    }
  }
  __syncthreads();

  for (;;) {
#pragma unroll
    for (int j = 0; j < BATCH; ++j) {
      if (ts[j] >= nt || (a.append && hs[j] >= nq && kat[ts[j]] < 0)) continue;
      unsigned char* r = to(ts[j], hs[j]);
      const float2* w = cs + ts[j] * half;
      Pc<E> u = *reinterpret_cast<const Pc<E>*>(&x1[j]);
      if constexpr (WIDE) {
        if (both) {
          Pc<E> z = *reinterpret_cast<const Pc<E>*>(&x2[j]);
#pragma unroll
          for (int e = 0; e < N; ++e) {
            const float2 c = w[p * N + e];
            const float u1 = to_f(u.e[e]), u2 = to_f(z.e[e]);
            u.e[e] = to_e<E>(u1 * c.x - u2 * c.y);
            z.e[e] = to_e<E>(u2 * c.x + u1 * c.y);
          }
          store_piece(r + at2, z);
        } else if (!halves) {
#pragma unroll
          for (int e = 0; e < N / 2; ++e) {
            const int pair = p * (N / 2) + e;
            if (pair < half) {
              const float2 c = w[pair];
              const float u1 = to_f(u.e[2 * e]), u2 = to_f(u.e[2 * e + 1]);
              u.e[2 * e] = to_e<E>(u1 * c.x - u2 * c.y);
              u.e[2 * e + 1] = to_e<E>(u2 * c.x + u1 * c.y);
            }
          }
        }
      } else {
        // halves that do not start at multiples of 16 bytes: a piece of the result, its
        // partners one by one.  In place this holds because the units of a row lie in
        // one wave (d / N divides 64), which reads all of it before it writes any.
#pragma unroll
        for (int e = 0; e < N; ++e) {
          const int c = p * N + e;
          if (c < a.rot) {
            const float2 cw = w[c < half ? c : c - half];
            const float sin = c < half ? -cw.y : cw.y;
            u.e[e] = to_e<E>(to_f(u.e[e]) * cw.x + to_f(other[j][e]) * sin);
          }
        }
      }
      store_piece(r + at1, u);
    }
    if (wq.t >= nt) break;
    load();
  }
  if (!a.v.data) return;
  for (;;) {
#pragma unroll
    for (int j = 0; j < BATCH; ++j)
      if (vt[j] < nt && kat[vt[j]] >= 0)
        *reinterpret_cast<uint4*>(a.cache.v + kat[vt[j]] + vh[j] * a.cache.head + wv.p * 16) = y[j];
    if (wv.t >= nt) break;
    load_v();
  }
}

hipError_t launch_rotate(Dt dt, RotateArgs a, hipStream_t s) {
  // Tokens of a workgroup: enough to fill it a few times over where there are
  // many, one where there are few.
  int per = (a.tok.total + 2047) / 2048;
  per = per < 1 ? 1 : per > ROT_TOKENS ? ROT_TOKENS : per;
  const int half = a.rot / 2;
  a.per = per;
  // (a launch holds less than 2^32 threads in one direction)
  const unsigned groups = ((unsigned)a.tok.total + per - 1) / per;
  const dim3 grid(std::min(groups, ROT_GRID), (groups + ROT_GRID - 1) / ROT_GRID);
  const int n = dt == Dt::F32 ? 4 : 8;
  const bool wide = a.layout == 1 || half % n == 0;
  using T = std::true_type;
  using F = std::false_type;
  auto go = [&](auto e) {
    using E = decltype(e);
    auto run = [&](auto w, auto l) {
      hipLaunchKernelGGL((k_rotate<E, decltype(w)::value, decltype(l)::value>), grid, dim3(256), 0,
                         s, a);
      return hipGetLastError();
    };
    if (a.cache.skip) return wide ? run(T{}, T{}) : run(F{}, T{});
    return wide ? run(T{}, F{}) : run(F{}, F{});
  };
  return dt == Dt::F32 ? go(float{}) : go(bf16{});
}

// ------------------------------------------------------------------ pages
//
// What a page call decides is a few prefix sums over the sequences and over
// refs: one workgroup of 16 waves does it (k_*_plan), in index order, so the
// result is the same on every run; the rows of the table and the data follow
// in kernels over the whole GPU.  The plans are latency (256 sequences of up to 1200
// tokens in pages of 64: 7.5 us); the data is HBM: a step of a beam search over them,
// 104 MB, 19.5 us a call; 347 MB compacted 57, and 108 after a cache-evicting write (a
// copy of as many bytes 86).

namespace {

constexpr int PLAN = 1024;

__device__ inline int blocks_of(int len, const Book& b) {
  const int64_t n = ((int64_t)max(len, 0) + b.page_size - 1) / b.page_size;
  return (int)min(n, (int64_t)b.max_blocks);
}
__device__ inline bool held(const Book& b, int p) { return (unsigned)p < (unsigned)b.num_pages; }

// Exclusive prefix sum over the workgroup's threads; *total: the sum.
__device__ inline int scan(int x, int* total) {
  __shared__ int wsum[PLAN / 64];
  const int lane = lane_id(), wave = wave_id();
  int v = x;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int y = __shfl_up(v, d);
    if (lane >= d) v += y;
  }
  __syncthreads();  // wsum of an earlier call is read
  if (lane == 63) wsum[wave] = v;
  __syncthreads();
  int before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < PLAN / 64; ++w) {
    if (w < wave) before += wsum[w];
    all += wsum[w];
  }
  *total = all;
  return before + v - x;
}

constexpr int SCAN_PER = 8;  // pages of a thread in one step

// Calls f(page, place) for every page in [0, num) with pick(page) in index
// order of place = its rank among them; returns how many there are.
template <class Pick, class F> __device__ inline int ranked(int num, Pick&& pick, F&& f) {
  int base = 0;
  for (int p0 = 0; p0 < num; p0 += PLAN * SCAN_PER) {
    const int mine = p0 + threadIdx.x * SCAN_PER;
    unsigned bits = 0;
#pragma unroll
    for (int j = 0; j < SCAN_PER; ++j)
      if (mine + j < num && pick(mine + j)) bits |= 1u << j;
    int total, at = base + scan(__popc(bits), &total);
#pragma unroll
    for (int j = 0; j < SCAN_PER; ++j)
      if (bits >> j & 1) f(mine + j, at++);
    base += total;
  }
  return base;
}

}  // namespace

// Page copies in units of 16 KiB: (pair, part, unit), strided over `groups`
// workgroups of which this is number `me`.  Streaming stores: with plain ones the calls
// above take 30.5 and 69.5 us; 2048 or 16384 workgroups are within 2%.
constexpr int MOVE_UNIT = 16384;
constexpr int MOVE_GROUPS = 4096;
__device__ inline void move_pages(const Pool& p, const int32_t* src, const int32_t* dst, int n,
                                  int64_t me, int64_t groups) {
  const int64_t per = (p.bytes + MOVE_UNIT - 1) / MOVE_UNIT;
  const int64_t units = (int64_t)n * p.parts * per;
  for (int64_t u = me; u < units; u += groups) {
    const int64_t i = u / (p.parts * per), r = u - i * (p.parts * per);
    const int part = (int)(r / per);
    const int64_t at = (r - part * per) * MOVE_UNIT;
    const int from = src[i], to = dst[i];
    if ((unsigned)from >= (unsigned)p.num_pages || (unsigned)to >= (unsigned)p.num_pages) continue;
    const unsigned char* x = p.data + part * p.part + from * p.page + at;
    unsigned char* y = p.data + part * p.part + to * p.page + at;
    const int64_t left = p.bytes - at;
    if (left >= MOVE_UNIT) {
      uint4 v[4];
#pragma unroll
      for (int j = 0; j < 4; ++j)
        v[j] = *reinterpret_cast<const uint4*>(x + j * 4096 + threadIdx.x * 16);
#pragma unroll
      for (int j = 0; j < 4; ++j) store_stream(y + j * 4096 + threadIdx.x * 16, v[j]);
    } else {
      for (int64_t o = threadIdx.x * 16; o < left; o += 4096)
        store_stream(y + o, *reinterpret_cast<const uint4*>(x + o));
    }
  }
}
// Workgroups that move the pages of at most n pairs.
inline unsigned move_groups(const Pool* p, int64_t n) {
  if (!p) return 0;
  const int64_t per = (p->bytes + MOVE_UNIT - 1) / MOVE_UNIT;
  return (unsigned)std::min<int64_t>(n * p->parts * per, MOVE_GROUPS);
}

// Block i of row s of the extended table; a new block's page is marked held.
__device__ inline void extend_block(const Book& b, const PageWork& w, int s, int i) {
  const int first = w.rank[s], old = blocks_of(w.lens[s], b);
  const int64_t at = (int64_t)s * b.max_blocks + i;
  if (first >= 0 && i >= old && i < blocks_of(b.lens_out[s], b)) {
    const int p = w.dst[first + i - old];
    b.table_out[at] = p;
    b.refs_out[p] = 1;
  } else if (b.table_out != b.table) {
    b.table_out[at] = b.table[at];
  }
}

// rank[s] = the place, among the pages given out, of sequence s's first (-1:
// it gets none); dst[i] = the i-th free page; refs_out, lens_out, short_of.
// ROWS: the table too, where it is small.
template <bool ROWS>
__global__ __launch_bounds__(PLAN) void k_extend_plan(Book b, const int32_t* add,
                                                      int32_t* short_of, PageWork w) {
  const int found = ranked(
      b.num_pages,
      [&](int p) {
        const int r = b.refs[p];
        if (b.refs_out != b.refs) b.refs_out[p] = r;
        return r <= 0;
      },
      [&](int p, int i) { w.dst[i] = p; });
  int base = 0;
  for (int s0 = 0; s0 < b.S; s0 += PLAN) {
    const int s = s0 + threadIdx.x;
    int need = 0, len = 0, more = 0;
    bool fits = false;
    if (s < b.S) {
      len = max(b.lens[s], 0);
      more = max(add[s], 0);
      const int64_t blocks = ((int64_t)len + more + b.page_size - 1) / b.page_size;
      const int64_t old = ((int64_t)len + b.page_size - 1) / b.page_size;
      need = (int)min(blocks - old, (int64_t)1 << 30);
      fits = blocks <= b.max_blocks;
    }
    // what a sequence wants is cut at found + 1, which keeps the sums in range
    // and refuses the same sequences
    const int want = fits ? min(need, found + 1) : 0;
    int total;
    const int before = min(base, found + 1) + scan(want, &total);
    const bool served = fits && (need == 0 || before + want <= found);
    if (s < b.S) {
      w.rank[s] = served && need > 0 ? before : -1;
      short_of[s] = served ? 0 : need;
      w.lens[s] = len;  // the old length, for the rows
      b.lens_out[s] = served ? len + more : len;
    }
    base = min(base, found + 1) + total;
  }
  if constexpr (ROWS) {
    __syncthreads();
    for (int i = threadIdx.x; i < b.S * b.max_blocks; i += PLAN)
      extend_block(b, w, i / b.max_blocks, i % b.max_blocks);
  }
}

// Rows of the table, one workgroup each.
__global__ __launch_bounds__(256) void k_extend_rows(Book b, PageWork w) {
  for (int i = threadIdx.x; i < b.max_blocks; i += 256) extend_block(b, w, blockIdx.x, i);
}

hipError_t launch_extend(const Book& b, const int32_t* add, int32_t* short_of, const PageWork& w,
                         hipStream_t s) {
  // A small table goes along in the one workgroup, which saves a launch (55 rows of up
  // to 6 blocks: 13.4 us a call with two, 10.6 with one).
  if ((int64_t)b.S * b.max_blocks <= 8192) {
    hipLaunchKernelGGL(k_extend_plan<true>, dim3(1), dim3(PLAN), 0, s, b, add, short_of, w);
    return hipGetLastError();
  }
  hipLaunchKernelGGL(k_extend_plan<false>, dim3(1), dim3(PLAN), 0, s, b, add, short_of, w);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(k_extend_rows, dim3(b.S), dim3(256), 0, s, b, w);
  return hipGetLastError();
}

// count[0] = copies; src, dst: their pages; rank[i]: row i's copy or -1, -2: no
// page was left.  w.lens, w.table hold the old lengths and, in place, rows.
__global__ __launch_bounds__(PLAN) void k_select_plan(Book b, const int32_t* parents,
                                                      int32_t* short_of, PageWork w) {
  const int tid = threadIdx.x;
  for (int s = tid; s < b.S; s += PLAN) {
    __hip_atomic_store(&w.heir[s], b.S, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    w.lens[s] = b.lens[s];
  }
  __syncthreads();
  for (int i = tid; i < b.S; i += PLAN) {
    const int p = parents[i];
    if ((unsigned)p < (unsigned)b.S) atomicMin(&w.heir[p], i);
  }
  const int found = ranked(
      b.num_pages,
      [&](int p) {
        const int r = b.refs[p];
        if (b.refs_out != b.refs) b.refs_out[p] = r;
        return r <= 0;
      },
      [&](int p, int i) { w.dst[i] = p; });
  __syncthreads();
  int base = 0;
  for (int i0 = 0; i0 < b.S; i0 += PLAN) {
    const int i = i0 + tid;
    int src = -1;
    if (i < b.S) {
      const int p = parents[i];
      if ((unsigned)p < (unsigned)b.S) {
        const int len = b.lens[p], last = len / b.page_size;
        if (len > 0 && len % b.page_size != 0 && last < b.max_blocks &&
            __hip_atomic_load(&w.heir[p], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) != i) {
          src = b.table[(int64_t)p * b.max_blocks + last];
          if (!held(b, src)) src = -1;
        }
      }
    }
    int total;
    const int at = base + scan(src >= 0, &total);
    if (i < b.S) {
      const bool none = src >= 0 && at >= found;
      if (src >= 0 && !none) w.src[at] = src;
      w.rank[i] = src < 0 ? -1 : none ? -2 : at;
      short_of[i] = none;
    }
    base += total;
  }
  if (tid == 0) w.count[0] = min(base, found);
}

__global__ __launch_bounds__(256) void k_copy_ints(const int32_t* x, int32_t* y, int64_t n) {
  for (int64_t i = blockIdx.x * 256ll + threadIdx.x; i < n; i += gridDim.x * 256ll) y[i] = x[i];
}

// New rows, one workgroup each, and the references of old and new ones; the
// workgroups past the rows copy the pages.
__global__ __launch_bounds__(256) void k_select_rows(Book b, const int32_t* parents, PageWork w,
                                                     const int32_t* table, Pool pool) {
  if ((int)blockIdx.x >= b.S) {
    move_pages(pool, w.src, w.dst, w.count[0], blockIdx.x - b.S, gridDim.x - b.S);
    return;
  }
  const int i = blockIdx.x, p = parents[i], rank = w.rank[i];
  const bool real = (unsigned)p < (unsigned)b.S && rank != -2;
  const int len = real ? max(w.lens[p], 0) : 0, now = blocks_of(len, b);
  const int was = blocks_of(w.lens[i], b);
  if (threadIdx.x == 0) b.lens_out[i] = len;
  for (int j = threadIdx.x; j < b.max_blocks; j += 256) {
    if (j < was) {
      const int o = table[(int64_t)i * b.max_blocks + j];
      if (held(b, o)) atomicAdd(&b.refs_out[o], -1);
    }
    int x = -1;
    if (j < now) {
      x = rank >= 0 && j == now - 1 ? w.dst[rank] : table[(int64_t)p * b.max_blocks + j];
      if (held(b, x)) atomicAdd(&b.refs_out[x], 1);
    }
    b.table_out[(int64_t)i * b.max_blocks + j] = x;
  }
}

hipError_t launch_select(const Book& b, const int32_t* parents, const Pool* pool,
                         int32_t* short_of, const PageWork& w, hipStream_t s) {
  const int32_t* table = b.table;
  if (b.table_out == b.table) {
    const int64_t n = (int64_t)b.S * b.max_blocks;
    hipLaunchKernelGGL(k_copy_ints, dim3((unsigned)std::min<int64_t>((n + 255) / 256, 2048)),
                       dim3(256), 0, s, b.table, w.table, n);
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    table = w.table;
  }
  hipLaunchKernelGGL(k_select_plan, dim3(1), dim3(PLAN), 0, s, b, parents, short_of, w);
  if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  hipLaunchKernelGGL(k_select_rows, dim3(b.S + move_groups(pool, b.S)), dim3(256), 0, s, b, parents,
                     w, table, pool ? *pool : Pool{});
  return hipGetLastError();
}

// count[0] = moves, count[1] = pages in use; src, dst: the moves; map.
__global__ __launch_bounds__(PLAN) void k_compact_plan(Book b, int32_t* map, PageWork w) {
  int mine = 0;
  for (int p = threadIdx.x; p < b.num_pages; p += PLAN) mine += b.refs[p] > 0;
  int n;
  scan(mine, &n);
  // below n the free ones (holes), from n on those in use: as many
  const int moves = ranked(n, [&](int p) { return b.refs[p] <= 0; },
                           [&](int p, int i) { w.dst[i] = p; });
  ranked(b.num_pages - n, [&](int p) { return b.refs[n + p] > 0; },
         [&](int p, int i) { w.src[i] = n + p; });
  for (int p = threadIdx.x; p < b.num_pages; p += PLAN)
    map[p] = p < n && b.refs[p] > 0 ? p : -1;
  __syncthreads();
  for (int i = threadIdx.x; i < moves; i += PLAN) map[w.src[i]] = w.dst[i];
  if (threadIdx.x == 0) {
    w.count[0] = moves;
    w.count[1] = n;
  }
}

// Rows of the table, renumbered (what a sequence does not hold becomes -1) by the
// first `rows` workgroups, refs by the next `refs`, the data by the others.
// refs: the moves take theirs along; a page that is moved from lies at n or past
// it, one that is moved to below, so no thread reads what another writes.
__global__ __launch_bounds__(256) void k_compact_rest(Book b, const int32_t* map, PageWork w,
                                                      Pool pool, int rows, int refs) {
  const int me = blockIdx.x;
  if (me < rows) {
    const int64_t n = (int64_t)b.S * b.max_blocks;
    for (int64_t i = me * 256ll + threadIdx.x; i < n; i += rows * 256ll) {
      const int s = (int)(i / b.max_blocks), j = (int)(i - (int64_t)s * b.max_blocks);
      int x = -1;
      if (j < blocks_of(b.lens[s], b)) {
        x = b.table[i];
        x = held(b, x) ? map[x] : -1;
      }
      b.table_out[i] = x;
    }
  } else if (me < rows + refs) {
    const int n = w.count[1];
    for (int p = (me - rows) * 256 + threadIdx.x; p < b.num_pages; p += refs * 256) {
      if (p < n) {
        if (map[p] >= 0 && b.refs_out != b.refs) b.refs_out[p] = b.refs[p];
      } else {
        if (map[p] >= 0) b.refs_out[map[p]] = b.refs[p];
        b.refs_out[p] = 0;
      }
    }
  } else {
    move_pages(pool, w.src, w.dst, w.count[0], me - rows - refs, gridDim.x - rows - refs);
  }
}

hipError_t launch_compact(const Book& b, const Pool* pool, int32_t* map, const PageWork& w,
                          hipStream_t s) {
  hipLaunchKernelGGL(k_compact_plan, dim3(1), dim3(PLAN), 0, s, b, map, w);
  if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  const int64_t n = (int64_t)b.S * b.max_blocks;
  const int rows = (int)std::min<int64_t>((n + 255) / 256, 2048);
  const int refs = std::min((b.num_pages + 255) / 256, 1024);
  hipLaunchKernelGGL(k_compact_rest, dim3(rows + refs + move_groups(pool, b.num_pages)), dim3(256),
                     0, s, b, map, w, pool ? *pool : Pool{}, rows, refs);
  return hipGetLastError();
}

__global__ __launch_bounds__(256) void k_move(Pool p, const int32_t* src, const int32_t* dst, int n) {
  move_pages(p, src, dst, n, blockIdx.x, gridDim.x);
}

hipError_t launch_move(const Pool& p, const int32_t* src, const int32_t* dst, int n,
                       hipStream_t s) {
  hipLaunchKernelGGL(k_move, dim3(move_groups(&p, n)), dim3(256), 0, s, p, src, dst, n);
  return hipGetLastError();
}

}  // namespace gdn
