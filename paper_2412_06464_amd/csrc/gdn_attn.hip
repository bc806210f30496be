// Attention of new tokens over a cache in pages.
//
// The rows of one cache head are the new tokens' query heads that read it:
// row r of a sequence is (token r / G, head r % G of the group), so a group of
// heads shares every key that is loaded.  A workgroup takes a block of rows and
// a range of keys, walks the range in tiles with the running maximum m and sum
// l of the softmax, and keeps everything transposed:
//     S^T = K Q^T   (A = K rows from LDS, B = Q in registers)
//     O^T += V^T P^T (A = V^T from LDS by transposing reads, B = P)
// so that a row is a column (lane & 15) of every accumulator: its maximum and
// sum take two lane exchanges a tile, its rescaling none, and the accumulator
// tiles of S^T are, as they stand, the B operand of the second product (the
// permuted contraction order of gdn_device.h).
//
// Two kernels from one body:
//   k_attn_tile  many rows: 4 waves with 32 (or 16) rows each share a tile of keys;
//   k_attn_few   few rows (at most 32): 4 waves share the rows, each walks its
//                own keys of a tile and the results are joined in LDS.
// Where the row blocks do not fill the GPU, a block's keys are split over
// several workgroups, whose unnormalised sums k_attn_join adds.
//
// Times in the comments are of the present kernels, both sides of a choice in turn in
// one process; the same call differs by up to 4% between two runs on one GPU.
#include <hip/hip_runtime.h>
#include <math.h>

#include "gdn_device.h"
#include "gdn_paged_kernels.h"

namespace gdn {

typedef bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));

#define LDS_AS __attribute__((address_space(3)))
#define CONST_AS __attribute__((address_space(4)))

// 64 lanes x 16 bytes from base + off (bytes, one per lane) straight into LDS
// at lds + lane * 16; base and lds are the same for the whole wave.  As
// dma_frag: the caller waits.
__device__ inline void dma_rows(const unsigned char* base, unsigned off, unsigned lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds),
               "v"(off), "s"(base)
               : "memory");
}

// One row block's place in the problem.
struct Block {
  int n, hk;          // sequence, cache head
  int q0, m;          // first token row of the sequence, its new tokens
  int kv;             // its cached tokens
  int r0, r1;         // rows [r0, r1) of the m * G
  int seen, hi;       // keys that some row sees lie in [seen, hi)
  int lo;             // seen, down to a multiple of 16
  // first and one past the last key that token i sees
  __device__ int first(const AttnArgs& a, int i) const {
    // (a token before the cache's first sees nothing; its place may not pass 32 bits)
    return a.window > 0 ? max(0, max(0, kv - m + i + 1) - a.window) : 0;
  }
  __device__ int last(const AttnArgs& a, int i) const {
    return a.causal ? max(0, kv - m + i + 1) : kv;
  }
  __device__ void range(const AttnArgs& a) {
    seen = first(a, r0 / a.G);
    lo = seen & ~15;
    hi = min(kv, last(a, (r1 - 1) / a.G));
  }
};

template <class E, int D, int QT, int RW, int KW, int KT> struct AttnCfg {
  static constexpr int NK = KT / KW;                // keys of a wave
  static constexpr int NTH = 64 * RW * KW;
  static constexpr int RB = D * (int)sizeof(E);     // bytes of a key
  static constexpr int NP = RB / 16;                // 16-byte pieces of it
  static constexpr int ROWS = RW * QT * 16;
  static constexpr int TILE = KT * RB;              // bytes of a tile of k (or v)
  // rows of the waves' sums, 4 banks apart: 16 of them are written at a time
  static constexpr int JR = D + 4;
  static constexpr int JOIN = KW > 1 ? KW * ROWS * (JR + 2) * 4 : 0;
  static constexpr int LDS = 4 * TILE > JOIN ? 4 * TILE : JOIN;
  static constexpr int RPI = 64 / NP;               // keys of one wave-wide copy
  static_assert(NK % 16 == 0 && KT % 16 == 0, "a wave works on whole groups of 16 keys");
};

// Place of 16-byte piece p of key row r in a tile: the pieces of a row are
// exchanged by an XOR that spreads the rows a read touches over the banks.
// K is read 16 rows at a time, the same piece of each: 16 different pieces.
template <int NP> __device__ inline int k_swz(int r) { return NP >= 16 ? r & 15 : (r >> 1) & 7; }
// bf16 V is read two neighbouring pieces of 4 rows by 16 lanes (8 rows by 32),
// fp32 V four neighbouring pieces of rows 4 apart.
template <class E, int NP> __device__ inline int v_swz(int r) {
  if constexpr (sizeof(E) == 4) return ((r >> 2) & 3) << 2;
  return NP >= 16 ? (r & 7) << 1 : ((r >> 1) & 3) << 1;
}

template <class E> struct Piece;  // 16 bytes of channels and their products
template <> struct Piece<bf16> {
  using type = bf16x8;
  __device__ static inline f32x4 mma(type a, type b, f32x4 c) { return Mfma<bf16>::mma(a, b, c); }
};
template <> struct Piece<float> {
  using type = f32x4;
  __device__ static inline f32x4 mma(type a, type b, f32x4 c) {
#pragma unroll
    for (int j = 0; j < 4; ++j) c = Mfma<float>::mma(a[j], b[j], c);
    return c;
  }
};

// x without its infinities and NaN; true if there were any.
template <class E> __device__ inline bool clear_odd(uint4& x) {
  unsigned* w = reinterpret_cast<unsigned*>(&x);
  bool odd = false;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const unsigned u = w[i];
    if ((u & 0x7f800000u) == 0x7f800000u) w[i] &= sizeof(E) == 4 ? 0u : 0xffffu, odd = true;
    if (sizeof(E) == 2 && (u & 0x7f80u) == 0x7f80u) w[i] &= 0xffff0000u, odd = true;
  }
  return odd;
}

// Over the four lanes (16 apart) of a column: the largest value, the sum.
// v_permlane swaps move the other halves next to each other without LDS.
__device__ inline float col_max(float x) {
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ inline float col_sum(float x) {
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// The running maximum follows only when a score passes it by this much (in
// base 2): p stays below 2^8, which costs no accuracy (p, l and o keep their
// relative precision), and o is rescaled a few times instead of in most tiles
// (a prompt of 8192 tokens, d = 128: 279 us, with 0 306).
constexpr float SLACK = 8.f;

template <class E, int D, int QT, int RW, int KW, int KT>
__device__ inline void attn_block(const AttnArgs& a, const Block& b, int split,
                                  unsigned char* smem) {
  using C = AttnCfg<E, D, QT, RW, KW, KT>;
  using P = Piece<E>;
  constexpr int NK = C::NK, NT = NK / 16, RB = C::RB, NP = C::NP, KB = RB / 64, DT = D / 16;
  constexpr int GROUPS = KT / 16;
  // Where two waves share a SIMD, the one in its products goes first: the other
  // fills in with its softmax (a prompt of 8192 tokens, d = 128: 275 us, without 285;
  // with three waves, bf16 at d = 64, 174 and 166, so not there).
  constexpr bool PRIO = KW == 1 && RB >= 256 && RB <= 512;
  // The bf16 values that stand for a weight p in its product with v.  Two (p's rounding, and
  // what that left over: 2^-16 of p is lost) make o exact but for its own rounding; one
  // leaves its error, against 64 bits, at 1.3 to 1.4 times that.  With few rows the keys'
  // way from HBM hides the second product (256 single tokens in a 2K window 147.2 us, with
  // one 147.4; two with 131072 keys 96.7 and 96.6; 8 tokens a sequence, up to 4000 keys,
  // 55.3 and 55.8).  With many it is matrix cores' time that binds (a prompt of 8192 tokens
  // 345 us, with one 269; d = 64 245 and 165; prompts in a 2K window, d = 256, 201 and 164).
  constexpr int PARTS = KW == 1 ? 1 : 2;
  constexpr int MINE = KW == 1 ? (GROUPS + RW - 1) / RW : NT;  // groups this wave copies
  const int lane = lane_id(), g = lane >> 4, c16 = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int rw = KW == 1 ? wave : 0, kw = KW == 1 ? 0 : wave;

  // the last range goes to the end, however long the cache has become
  const int begin = b.lo + split * a.len;
  const int end = split == a.splits - 1 ? b.hi : min(b.hi, begin + a.len);
  const int tiles = (end - begin + KT - 1) / KT;

  const CONST_AS int* pages = (const CONST_AS int*)(a.cache.table + (int64_t)b.n * a.cache.max_blocks);
  const int shift = a.cache.shift, mask = (1 << shift) - 1, num_pages = a.cache.num_pages;
  const unsigned char* const kbase = a.cache.k + (int64_t)b.hk * a.cache.head;
  const unsigned char* const vbase = a.cache.v + (int64_t)b.hk * a.cache.head;
  const unsigned lds0 = (unsigned)(uintptr_t)smem;

  // Pages of the groups of 16 keys of the tile from k0 on that this wave works
  // on (KW == 1: all of the tile's); they are looked up a tile ahead of their
  // use, by scalar loads, which the copies in flight do not delay.
  auto look_up = [&](int k0, int (&pg)[NT]) {
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const int key = k0 + kw * NK + 16 * t;
      pg[t] = key < end ? pages[__builtin_amdgcn_readfirstlane(key) >> shift] : -1;
    }
  };
  auto there = [&](int page) { return (unsigned)page < (unsigned)num_pages; };
  // This wave's copies of a tile: groups of 16 keys, of k and of v (a group
  // that is not there is read from page 0 and not used).
  unsigned koff[16 / C::RPI], voff[16 / C::RPI];
#pragma unroll
  for (int j = 0; j < 16 / C::RPI; ++j) {
    const int r = j * C::RPI + lane / NP, p = lane % NP;
    koff[j] = r * (unsigned)a.cache.slot + ((p ^ k_swz<NP>(r)) << 4);
    voff[j] = r * (unsigned)a.cache.slot + ((p ^ v_swz<E, NP>(r)) << 4);
  }
  auto copy_tile = [&](int k0, const int (&pg)[NT], int buf) {
#pragma unroll
    for (int i = 0; i < MINE; ++i) {
      const int grp = KW == 1 ? wave + i * RW : wave * NT + i;
      if (KW == 1 && GROUPS % RW && grp >= GROUPS) break;
      int page = pg[0];
#pragma unroll
      for (int t = 0; t < NT; ++t)
        if (KW == 1 ? grp == t : i == t) page = pg[t];
      if (!there(page)) page = 0;
      const int64_t off = (int64_t)page * a.cache.page + (int64_t)((k0 + 16 * grp) & mask) * a.cache.slot;
      const unsigned dst = lds0 + buf * 2 * C::TILE + grp * 16 * RB;
#pragma unroll
      for (int j = 0; j < 16 / C::RPI; ++j) dma_rows(kbase + off, koff[j], dst + j * 1024);
#pragma unroll
      for (int j = 0; j < 16 / C::RPI; ++j)
        dma_rows(vbase + off, voff[j], dst + C::TILE + j * 1024);
    }
  };

  int pg[NT];   // pages of the tile to copy next
  unsigned gone = 0;  // groups of the tile in hand that are not there
  look_up(begin, pg);

  // this lane's rows: Q in registers, the keys each sees
  typename P::type q[QT][KB];
  int first[QT], last[QT];
  const int wr0 = b.r0 + rw * QT * 16;
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    const int r = wr0 + t * 16 + c16;
    const bool real = r < b.r1;
    const int i = real ? r / a.G : 0, h = b.hk * a.G + (real ? r - i * a.G : 0);
    const unsigned char* p = a.q.data + (int64_t)(b.q0 + i) * a.q.ts + h * a.q.hs;
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
      uint4 x = make_uint4(0, 0, 0, 0);
      if (real) x = *reinterpret_cast<const uint4*>(p + (4 * kb + g) * 16);
      q[t][kb] = *reinterpret_cast<typename P::type*>(&x);
    }
    first[t] = b.first(a, i);
    last[t] = real ? min(end, b.last(a, i)) : 0;
  }
  // the keys that all rows of the block see, and that some row of the wave sees
  const int all_lo = b.first(a, (b.r1 - 1) / a.G), all_hi = min(end, b.last(a, b.r0 / a.G));
  const int we = min(b.r1, wr0 + QT * 16) - 1;
  const bool idle = wr0 >= b.r1;
  const int w_begin = idle ? 0 : b.first(a, wr0 / a.G), w_end = idle ? 0 : min(end, b.last(a, we / a.G));

  f32x4 o[DT][QT];
  float m[QT], l[QT];
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    m[t] = -INFINITY;
    l[t] = 0.f;
#pragma unroll
    for (int d = 0; d < DT; ++d) o[d][t] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  if (tiles > 0) {
    copy_tile(begin, pg, 0);
#pragma unroll
    for (int t = 0; t < NT; ++t) gone |= (unsigned)!there(pg[t]) << t;
    look_up(begin + KT, pg);
  }
  // Q is waited for here, so that no wait for it stands in the loop, where it
  // would wait for the copies too
#pragma unroll
  for (int t = 0; t < QT; ++t)
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) asm volatile("" : "+v"(q[t][kb]));

  // One tile.  EDGE: some row does not see some key of it.
  // This lane's LDS addresses in the first buffer: K row c16, and V row (bf16)
  // 4 g + c16 / 4, 4 of its channels, or (fp32) 4 g, one channel.  A row starts
  // at a multiple of its pieces' span, so piece p ^ swizzle lies at the address
  // of the lane's piece 0 XOR 16 p.
  const int vr = sizeof(E) == 4 ? 4 * g : 4 * g + (c16 >> 2);
  const unsigned kaddr0 = lds0 + (kw * NK + c16) * RB + ((g ^ k_swz<NP>(c16)) << 4);
  const unsigned vaddr0 =
      lds0 + C::TILE + (kw * NK + vr) * RB +
      (sizeof(E) == 4 ? (((c16 >> 2) ^ v_swz<E, NP>(vr)) << 4) + (c16 & 3) * 4
                      : ((((c16 >> 1) & 1) ^ v_swz<E, NP>(vr)) << 4) + (c16 & 1) * 8);
  auto step = [&](auto edge, int kw0, unsigned buf, unsigned gone) {
    constexpr bool EDGE = decltype(edge)::value;
    unsigned kaddr = kaddr0 + buf, vaddr = vaddr0 + buf;
    // opaque, or all the addresses below are kept in registers across the loop
    asm volatile("" : "+v"(kaddr), "+v"(vaddr));
    // S^T
    f32x4 s[NT][QT];
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int u = 0; u < QT; ++u) s[t][u] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (PRIO) __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        const auto x = *(LDS_AS const typename P::type*)((kaddr ^ (kb << 6)) + t * 16 * RB);
#pragma unroll
        for (int u = 0; u < QT; ++u) s[t][u] = P::mma(x, q[u][kb], s[t][u]);
      }
    }
    if (PRIO) __builtin_amdgcn_s_setprio(0);
    if constexpr (EDGE) {  // what a row does not see
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int key = kw0 + 16 * t + 4 * g + e;
#pragma unroll
          for (int u = 0; u < QT; ++u)
            if (key >= last[u] || key < first[u] || (gone >> t & 1)) s[t][u][e] = -INFINITY;
        }
    }
    // running softmax in base 2
    float mx[QT], ref[QT];
    bool grow = false;
#pragma unroll
    for (int u = 0; u < QT; ++u) {
      mx[u] = -INFINITY;
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) mx[u] = fmaxf(mx[u], s[t][u][e]);
      mx[u] = col_max(mx[u]) * a.c;
      grow = grow || mx[u] > m[u] + SLACK;
    }
    if (__any(grow)) {
#pragma unroll
      for (int u = 0; u < QT; ++u) {
        const float mn = fmaxf(m[u], mx[u]);
        // nothing seen so far: m is -inf and everything summed is 0
        const float al = __builtin_amdgcn_exp2f(m[u] - (mn == -INFINITY ? 0.f : mn));
        l[u] *= al;
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
          for (int e = 0; e < 4; ++e) o[d][u][e] *= al;
        m[u] = mn;
      }
    }
#pragma unroll
    for (int u = 0; u < QT; ++u) {
      ref[u] = m[u] == -INFINITY ? 0.f : m[u];
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float p = __builtin_amdgcn_exp2f(fmaf(s[t][u][e], a.c, -ref[u]));
          s[t][u][e] = p;
          l[u] += p;
        }
    }
    // O^T
    if (PRIO) __builtin_amdgcn_s_setprio(1);
    if constexpr (sizeof(E) == 4) {
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int d = 0; d < DT; ++d) {
            const float x = *(LDS_AS const float*)((vaddr ^ (d << 6)) + (16 * t + e) * RB);
#pragma unroll
            for (int u = 0; u < QT; ++u) o[d][u] = Mfma<float>::mma(x, s[t][u][e], o[d][u]);
          }
    } else {
      // l sums p in fp32; here it is an operand in bf16 (see PARTS)
      // Lane i of 16 points at 4 channels of key row i / 4 and receives one
      // channel (its own, i) of the 4 rows.
      auto turned = [&](int t, int d) {
        return __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (LDS_AS s16x4*)((vaddr ^ (d << 5)) + t * 16 * RB));
      };
      auto part = [&](int i, float p) {
        const bf16 hi = (bf16)p;
        return i == 0 ? hi : (bf16)(p - (float)hi);
      };
      if constexpr (NT == 1) {
        s16x4 p[QT][PARTS];
#pragma unroll
        for (int u = 0; u < QT; ++u)
#pragma unroll
          for (int i = 0; i < PARTS; ++i) {
            const bf16x4 x = {part(i, s[0][u][0]), part(i, s[0][u][1]), part(i, s[0][u][2]),
                              part(i, s[0][u][3])};
            p[u][i] = *reinterpret_cast<const s16x4*>(&x);
          }
#pragma unroll
        for (int d = 0; d < DT; ++d) {
          const s16x4 x = turned(0, d);
#pragma unroll
          for (int i = 0; i < PARTS; ++i)
#pragma unroll
            for (int u = 0; u < QT; ++u)
              o[d][u] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(x, p[u][i], o[d][u], 0, 0, 0);
        }
      } else {
#pragma unroll
        for (int t = 0; t < NT; t += 2) {
          bf16x8 p[QT][PARTS];
#pragma unroll
          for (int u = 0; u < QT; ++u)
#pragma unroll
            for (int i = 0; i < PARTS; ++i)
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                p[u][i][e] = part(i, s[t][u][e]);
                p[u][i][4 + e] = part(i, s[t + 1][u][e]);
              }
#pragma unroll
          for (int d = 0; d < DT; ++d) {
            const s16x4 x0 = turned(t, d), x1 = turned(t + 1, d);
            const s16x8 x = __builtin_shufflevector(x0, x1, 0, 1, 2, 3, 4, 5, 6, 7);
#pragma unroll
            for (int i = 0; i < PARTS; ++i)
#pragma unroll
              for (int u = 0; u < QT; ++u)
                o[d][u] = Mfma<bf16>::mma(*reinterpret_cast<const bf16x8*>(&x), p[u][i], o[d][u]);
          }
        }
      }
    }
    if (PRIO) __builtin_amdgcn_s_setprio(0);
  };

  // The copies of tile `it` are there and the other buffer is no longer read;
  // the next tile's copies start.  Returns the groups of the tile that are gone.
  auto next_tile = [&](int it) {
    wait_vmcnt<0>();
    if (KW == 1)
      lds_barrier();
    else
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    const unsigned now = gone;
    if (it + 1 < tiles) {
      const int k0 = begin + it * KT;
      copy_tile(k0 + KT, pg, (it + 1) & 1);
      gone = 0;
#pragma unroll
      for (int t = 0; t < NT; ++t) gone |= (unsigned)!there(pg[t]) << t;
      look_up(k0 + 2 * KT, pg);
    }
    return now;
  };
  bool odd = false;
  int it = 0;
  while (it < tiles) {
    unsigned now;
    // tiles all of whose keys all rows see: a loop of its own, so that what it
    // carries stays in place
#pragma unroll 1
    for (;;) {
      now = next_tile(it);
      const int f0 = begin + it * KT + kw * NK;
      if (f0 + NK > all_hi || f0 < all_lo || now) break;
      step(std::false_type{}, f0, (it & 1) * 2 * C::TILE, 0u);
      if (++it == tiles) break;
    }
    if (it == tiles) break;
    // Keys that no row sees may hold anything: their v is cleared.  Where some
    // rows see a key and others do not, an infinity or NaN in its v must not
    // meet a p of zero: it is taken out too, and added to the rows that do see it
    // after the end.
    const unsigned buf = (it & 1) * 2 * C::TILE;
    const int kw0 = begin + it * KT + kw * NK;  // this wave's keys
#pragma unroll 1
    for (int i = KW == 1 ? (int)threadIdx.x : lane; i < NK * NP; i += KW == 1 ? C::NTH : 64) {
      const int r = i / NP, key = kw0 + r;
      uint4* p = reinterpret_cast<uint4*>(smem + buf + C::TILE + kw * NK * RB + i * 16);
      if (key >= end || key < b.seen || (now >> (r >> 4) & 1)) {
        *p = make_uint4(0, 0, 0, 0);
      } else {
        uint4 x = *p;
        if (clear_odd<E>(x)) {
          *p = x;
          odd = true;
        }
      }
    }
    if (KW == 1)
      lds_barrier();
    else
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    if (!idle && kw0 < w_end && kw0 + NK > w_begin) step(std::true_type{}, kw0, buf, now);
    ++it;
  }

#pragma unroll
  for (int u = 0; u < QT; ++u) l[u] = col_sum(l[u]);

  const int64_t rows = (int64_t)a.tok.total * a.Hq;
  // channels ch.. of row r, unnormalised sums x, maximum and sum mm, ll
  auto put = [&](int r, int ch, f32x4 x, float mm, float ll) {
    const int i = r / a.G, h = b.hk * a.G + r - i * a.G;
    const int64_t at = (int64_t)(b.q0 + i) * a.Hq + h;
    if (a.splits > 1) {
      const int64_t w = split * rows + at;
      *reinterpret_cast<f32x4*>(a.part + w * D + ch) = x;
      if (ch == 0) {
        a.part_ml[2 * w] = mm;
        a.part_ml[2 * w + 1] = ll;
      }
      return;
    }
    const float inv = ll == 0.f ? 0.f : 1.f / ll;
    E* p = reinterpret_cast<E*>(a.o.data + (int64_t)(b.q0 + i) * a.o.ts + h * a.o.hs) + ch;
    if constexpr (sizeof(E) == 4) {
      *reinterpret_cast<f32x4*>(p) = f32x4{x[0] * inv, x[1] * inv, x[2] * inv, x[3] * inv};
    } else {
      const bf16x4 y = {(bf16)(x[0] * inv), (bf16)(x[1] * inv), (bf16)(x[2] * inv),
                        (bf16)(x[3] * inv)};
      *reinterpret_cast<bf16x4*>(p) = y;
    }
    if (ch == 0 && a.lse)
      a.lse[at] = ll == 0.f ? -INFINITY : (mm + log2f(ll)) * 0.6931471805599453f;
  };

  if constexpr (KW == 1) {
#pragma unroll
    for (int u = 0; u < QT; ++u) {
      const int r = wr0 + u * 16 + c16;
      if (r < b.r1)
#pragma unroll
        for (int d = 0; d < DT; ++d) put(r, 16 * d + 4 * g, o[d][u], m[u], l[u]);
    }
  } else {
    // join the waves' sums in LDS
    constexpr int R = C::ROWS, JR = C::JR;
    float* sum = reinterpret_cast<float*>(smem);
    float* ml = sum + KW * R * JR;
    __syncthreads();
#pragma unroll
    for (int u = 0; u < QT; ++u) {
      const int r = u * 16 + c16;
#pragma unroll
      for (int d = 0; d < DT; ++d)
        *reinterpret_cast<f32x4*>(sum + ((kw * R + r) * JR + 16 * d + 4 * g)) = o[d][u];
      if (g == 0) {
        ml[(kw * R + r) * 2] = m[u];
        ml[(kw * R + r) * 2 + 1] = l[u];
      }
    }
    __syncthreads();
    const int nr = b.r1 - b.r0;
    for (int i = threadIdx.x; i < nr * (D / 4); i += C::NTH) {
      const int r = i / (D / 4), ch = (i - r * (D / 4)) * 4;
      float mx = -INFINITY, ll = 0.f;
#pragma unroll
      for (int w = 0; w < KW; ++w) mx = fmaxf(mx, ml[(w * R + r) * 2]);
      const float ref = mx == -INFINITY ? 0.f : mx;
      f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < KW; ++w) {
        const float al = __builtin_amdgcn_exp2f(ml[(w * R + r) * 2] - ref);
        const f32x4 y = *reinterpret_cast<const f32x4*>(sum + ((w * R + r) * JR + ch));
        ll += al * ml[(w * R + r) * 2 + 1];
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] += al * y[e];
      }
      put(b.r0 + r, ch, x, mx, ll);
    }
  }

  // The infinities and NaN that were taken out: a thread owns 16 bytes of channels
  // of all rows, reads them again of every key of those tiles, and adds what it
  // finds to the rows that see the key (whatever their weight and scale, it makes
  // them infinite or NaN).
  if (!__syncthreads_or(odd)) return;
  if (threadIdx.x >= NP) return;
  constexpr int N = 16 / (int)sizeof(E);
#pragma unroll 1
  for (int f0 = begin; f0 < end; f0 += NK) {
    bool gap = false;
#pragma unroll 1
    for (int k = f0; k < min(f0 + NK, end); k += 16) gap = gap || !there(pages[k >> shift]);
    if (f0 + NK <= all_hi && f0 >= all_lo && f0 + NK <= end && !gap) continue;
#pragma unroll 1
    for (int key = max(f0, b.seen); key < min(f0 + NK, end); ++key) {
      const int page = pages[key >> shift];
      if (!there(page)) continue;
      uint4 x = *reinterpret_cast<const uint4*>(vbase + (int64_t)page * a.cache.page +
                                                (int64_t)(key & mask) * a.cache.slot +
                                                threadIdx.x * 16);
      const uint4 was = x;
      if (!clear_odd<E>(x)) continue;
      const E* v = reinterpret_cast<const E*>(&was);
#pragma unroll 1
      for (int r = b.r0; r < b.r1; ++r) {
        const int i = r / a.G, h = b.hk * a.G + r - i * a.G;
        if (key < b.first(a, i) || key >= b.last(a, i)) continue;
        const int64_t at = (int64_t)(b.q0 + i) * a.Hq + h;
        float* w = a.part + (split * rows + at) * D + threadIdx.x * N;
        E* y = reinterpret_cast<E*>(a.o.data + (int64_t)(b.q0 + i) * a.o.ts + h * a.o.hs) +
               threadIdx.x * N;
#pragma unroll 1
        for (int e = 0; e < N; ++e) {
          const float z = to_f(v[e]);
          if (z - z == 0.f) continue;
          if (a.splits > 1)
            w[e] += z;
          else
            y[e] = to_e<E>(to_f(y[e]) + z);
        }
      }
    }
  }
}

// Few rows: one row block per sequence and cache head, its keys split.  Bound by HBM,
// each key read once for all heads that share it, with two buffers of a CU's whole LDS
// in flight: a token each for 256 sequences in a 2K window (797 MB) 147 us, 5.4 TB/s; two
// with 131072 keys (537 MB) 97 us with the join, 5.5 TB/s; four with 1000 keys 10.4 us with
// the join, latency.
// Grid: ((n * splits + split) * Hk + hk).
template <class E, int D, int QT, int KW, int KT>
__global__ __launch_bounds__(64 * KW, 1) void k_attn_few(AttnArgs a) {
  using C = AttnCfg<E, D, QT, 1, KW, KT>;
  __shared__ __align__(1024) unsigned char smem[C::LDS];
  Block b;
  b.hk = blockIdx.x % a.Hk;
  const int rest = blockIdx.x / a.Hk, split = rest % a.splits;
  b.n = rest / a.splits;
  b.q0 = seq_start(a.tok, b.n);
  b.m = seq_start(a.tok, b.n + 1) - b.q0;
  b.r0 = 0;
  // (more rows than the plan had: boundaries that have changed on the device since)
  if (b.m == 0 || (int64_t)b.m * a.G > C::ROWS) return;
  b.r1 = b.m * a.G;
  b.kv = cached(a.cache, b.n);
  b.range(a);
  // a range past the keys: no partial result is read there
  if (split > 0 && b.lo + split * a.len >= b.hi) return;
  attn_block<E, D, QT, 1, KW, KT>(a, b, split, smem);
}

// The row block that comes at `rank` when all sequences' blocks are ordered by the
// keys they see, longest first, for at most 64 sequences: a lane holds one.  Block
// t of a sequence whose first new token has `base` row blocks' worth of keys before
// it sees depth = min(base + t, cap) of them, so count(K), the blocks with
// depth >= K, is a sum over the sequences, and the block at `rank` has the largest K
// with count(K) > rank: 64 values of K are tried at a time, one a lane.  False past
// the last block.
__device__ inline bool longest_first(const AttnArgs& a, int R, int rank, int* seq, int* tile) {
  const int lane = lane_id(), N = a.tok.N;
  int base = 0, blocks = 0;
  if (lane < N) {
    const int m = seq_start(a.tok, lane + 1) - seq_start(a.tok, lane);
    base = (int)min((int64_t)1 << 29, (int64_t)max(0, cached(a.cache, lane) - m) * a.G / R);
    blocks = (int)(((int64_t)m * a.G + R - 1) / R);
  }
  const int cap = a.window > 0 ? (int)min((int64_t)1 << 30, (int64_t)a.window * a.G / R + 1) : 1 << 30;
  int top = 0, total = 0;
#pragma unroll 1
  for (int n = 0; n < N; ++n) {
    const int bn = __builtin_amdgcn_readlane(base, n), tn = __builtin_amdgcn_readlane(blocks, n);
    top = max(top, bn + tn);
    total += tn;
  }
  if (rank >= total) return false;
  int k = 0, next = 0;  // count(k) > rank; next: count(k + 1)
  int step = min(top, cap + 1) / 63 + 1;
  for (;;) {
    const int K = k + lane * step;
    int count = 0;
#pragma unroll 1
    for (int n = 0; n < N; ++n) {
      const int bn = __builtin_amdgcn_readlane(base, n), tn = __builtin_amdgcn_readlane(blocks, n);
      count += max(0, tn - max(0, K - bn));
    }
    if (K > cap) count = 0;
    const int at = 63 - __clzll(__ballot(count > rank));
    k += at * step;
    next = __builtin_amdgcn_readlane(count, at + 1);
    if (step == 1) break;
    step = (step + 62) / 63;
  }
  // of the blocks with depth k, the one at rank - next
  int j = rank - next;
  const int mine = max(0, blocks - max(0, k - base)) - (k < cap ? max(0, blocks - max(0, k + 1 - base)) : 0);
#pragma unroll 1
  for (int n = 0; n < N; ++n) {
    const int x = __builtin_amdgcn_readlane(mine, n);
    if (j < x) {
      *seq = n;
      *tile = k < cap ? k - __builtin_amdgcn_readlane(base, n) : __builtin_amdgcn_readlane(blocks, n) - 1 - j;
      return true;
    }
    j -= x;
  }
  return false;
}

// Many rows: 4 d flop for a row and a key it sees.  Bound by the matrix cores and the
// exponentials of the softmax in turn, one workgroup's beside the other's.  A prompt
// of 8192 tokens of 16 heads, 4 cache heads, bf16: 165 us at d = 64 (832 TFLOP/s), 269 at
// 128 (1,021), 530 at 256 (1,038); two of 2048 in fp32, 8 heads, 164 at d = 128 (105).
// Grid: ((slot * splits + split) * Hk + hk); the sequence and row
// block of a slot follow from the boundaries: sequence n's slots begin at
// floor(cu[n] G / R) + n, which leaves at least ceil(m G / R) of them before
// the next one's.
template <class E, int D, int QT, int KT>
__global__ __launch_bounds__(256, sizeof(E) * D <= 512 ? 2 : 1) void k_attn_tile(AttnArgs a,
                                                                                int slots) {
  using C = AttnCfg<E, D, QT, 4, 1, KT>;
  constexpr int R = C::ROWS;
  __shared__ __align__(1024) unsigned char smem[C::LDS];
  Block b;
  // A second workgroup for some CUs, but no third for any: they come in reverse, the
  // shortest beside the longest (a prompt of 4096 tokens, 16 heads, d = 128: 111 us, in
  // order 113; of 2048 in fp32, 8 heads, d = 64: 57 and 79, two at d = 128 166 and 259).
  const int id =
      gridDim.x > 512 || blockIdx.x < 256 ? blockIdx.x : 255 + gridDim.x - blockIdx.x;
  b.hk = id % a.Hk;
  const int rest = id / a.Hk, split = rest % a.splits;
  int tile;
  if (a.longest) {
    if (!longest_first(a, R, rest / a.splits, &b.n, &tile)) return;
  } else {
    // the last row blocks of a sequence see the most keys: they go first
    const int slot = slots - 1 - rest / a.splits;
    if (a.tok.cu) {
      const int64_t G = a.G;
      int lo = 0, hi = a.tok.N;
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if ((int)(a.tok.cu[mid] * G / R) + mid <= slot) lo = mid; else hi = mid;
      }
      b.n = lo;
      tile = slot - ((int)(a.tok.cu[lo] * G / R) + lo);
    } else {
      const int per = (int)(((int64_t)a.tok.T * a.G + R - 1) / R);
      b.n = slot / per;
      tile = slot - b.n * per;
    }
  }
  b.q0 = seq_start(a.tok, b.n);
  b.m = seq_start(a.tok, b.n + 1) - b.q0;
  const int64_t rows = (int64_t)b.m * a.G;
  if ((int64_t)tile * R >= rows) return;
  b.r0 = tile * R;
  b.r1 = (int)min(rows, (int64_t)b.r0 + R);
  b.kv = cached(a.cache, b.n);
  b.range(a);
  if (split > 0 && b.lo + split * a.len >= b.hi) return;
  attn_block<E, D, QT, 4, 1, KT>(a, b, split, smem);
}

// Joins the splits' sums of a row by T threads: they turn the splits' maxima m_s into
// weights 2^(m_s - max m), then T / (D / 4) groups of them add up the weighted sums of
// every so many-th split, four loads in flight each.  Latency, or HBM where there are
// many rows.  T = 256 where a row has many splits (32 rows of 32: 5.0 us); T = D / 4, so
// several rows to a workgroup and no exchange between threads, where it has few (64
// rows of 8: 3.0 us; 16000 rows of 3 splits: 25 us with 256 threads a row).
template <class E, int D, int T> __global__ __launch_bounds__(256) void k_attn_join(AttnArgs a) {
  constexpr int TPR = D / 4, NG = T / TPR, PER = 256 / T;
  const int64_t rows = (int64_t)a.tok.total * a.Hq;
  const int64_t at = (int64_t)blockIdx.x * PER + (PER > 1 ? threadIdx.x / T : 0);
  if (at >= rows) return;
  const int tid = PER > 1 ? threadIdx.x % T : threadIdx.x;
  const int t = (int)(at / a.Hq), h = (int)(at - (int64_t)t * a.Hq);
  Block b;
  b.n = seq_of(a.tok, t);
  b.q0 = seq_start(a.tok, b.n);
  b.m = seq_start(a.tok, b.n + 1) - b.q0;
  const int64_t all = (int64_t)b.m * a.G;
  const int r = (t - b.q0) * a.G + h % a.G;
  b.r0 = r / a.block * a.block;
  b.r1 = (int)min(all, (int64_t)b.r0 + a.block);
  b.kv = cached(a.cache, b.n);
  b.range(a);
  // (as a quotient that stays within 32 bits at the longest caches)
  const int live = b.hi > b.lo ? min(a.splits, (b.hi - b.lo - 1) / a.len + 1) : 1;

  const float2* const ml = reinterpret_cast<const float2*>(a.part_ml);
  float mx = -INFINITY, ll = 0.f;
  f32x4 x = {0.f, 0.f, 0.f, 0.f};
  const int grp = tid / TPR, ch = (tid % TPR) * 4;
  if constexpr (PER > 1) {
    static_assert(NG == 1, "one group of threads a row");
#pragma unroll 4
    for (int s = 0; s < live; ++s) mx = fmaxf(mx, ml[s * rows + at].x);
    const float ref = mx == -INFINITY ? 0.f : mx;
#pragma unroll 4
    for (int s = 0; s < live; ++s) {
      const float2 z = ml[s * rows + at];
      const f32x4 y = *reinterpret_cast<const f32x4*>(a.part + (s * rows + at) * D + ch);
      const float w = __builtin_amdgcn_exp2f(z.x - ref);
      ll += w * z.y;
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = fmaf(w, y[e], x[e]);
    }
  } else {
    __shared__ float weight[MAX_SPLITS];
    __shared__ float red[8];
    __shared__ f32x4 sums[256];
    constexpr int J = (MAX_SPLITS + 255) / 256;
    float m[J], l[J];
#pragma unroll
    for (int j = 0; j < J; ++j) {
      const int s = tid + 256 * j;
      const float2 z = s < live ? ml[s * rows + at] : make_float2(-INFINITY, 0.f);
      m[j] = z.x;
      l[j] = z.y;
      mx = fmaxf(mx, z.x);
    }
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) mx = fmaxf(mx, __shfl_xor(mx, d));
    if (lane_id() == 0) red[wave_id()] = mx;
    __syncthreads();
    mx = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
    const float ref = mx == -INFINITY ? 0.f : mx;
#pragma unroll
    for (int j = 0; j < J; ++j) {
      const float w = __builtin_amdgcn_exp2f(m[j] - ref);
      if (tid + 256 * j < live) weight[tid + 256 * j] = w;
      ll += w * l[j];
    }
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) ll += __shfl_xor(ll, d);
    if (lane_id() == 0) red[4 + wave_id()] = ll;
    __syncthreads();
    ll = (red[4] + red[5]) + (red[6] + red[7]);
#pragma unroll 4
    for (int s = grp; s < live; s += NG) {
      const f32x4 y = *reinterpret_cast<const f32x4*>(a.part + (s * rows + at) * D + ch);
      const float w = weight[s];
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = fmaf(w, y[e], x[e]);
    }
    sums[tid] = x;
    __syncthreads();
    if (tid >= TPR) return;
#pragma unroll
    for (int j = 1; j < NG; ++j) {
      const f32x4 y = sums[tid + j * TPR];
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] += y[e];
    }
  }
  const float inv = ll == 0.f ? 0.f : 1.f / ll;
  E* p = reinterpret_cast<E*>(a.o.data + (int64_t)t * a.o.ts + h * a.o.hs) + ch;
  store4<E>(p, f32x4{x[0] * inv, x[1] * inv, x[2] * inv, x[3] * inv});
  if (ch == 0 && a.lse)
    a.lse[at] = ll == 0.f ? -INFINITY : (mx + log2f(ll)) * 0.6931471805599453f;
}

// ---- launchers

namespace {

// Tiles.  The few-rows kernel: as many keys as fill a CU's LDS with two buffers
// of k and v (most bytes in flight), four waves where that leaves each a group
// of 16.  The other: as many as let two workgroups share a CU (64 KB of buffers),
// so that one's products run beside the other's softmax: at d = 256 in bf16 32
// keys, prompts in a 2K window 174 us, with 64 and one workgroup 247; at d = 64 in bf16
// 64 keys leave room for three or four (a prompt of 8192 tokens 173 us, with 128 200).
template <class E, int D> struct Few {
  static constexpr int RB = D * (int)sizeof(E);
  static constexpr int KW = RB >= 1024 ? 2 : 4;
  static constexpr int KT = RB <= 256 ? 128 : RB == 512 ? 64 : 32;
};
template <class E, int D> struct Tile {
  static constexpr int KT = D * (int)sizeof(E) >= 512 ? 32 : 64;
};

template <class F> hipError_t by_dim(Dt dt, int d, F&& f) {
  auto go = [&](auto e) {
    using E = decltype(e);
    if (d == 64) return f(E{}, std::integral_constant<int, 64>{});
    if (d == 128) return f(E{}, std::integral_constant<int, 128>{});
    return f(E{}, std::integral_constant<int, 256>{});
  };
  if (d != 64 && d != 128 && d != 256) return hipErrorInvalidValue;
  return dt == Dt::F32 ? go(float{}) : go(bf16{});
}

}  // namespace

int attn_few_keys(Dt dt, int d) {
  const int rb = d * (dt == Dt::F32 ? 4 : 2);
  return rb <= 256 ? 128 : rb == 512 ? 64 : 32;
}
int attn_tile_keys(Dt dt, int d) { return d * (dt == Dt::F32 ? 4 : 2) >= 512 ? 32 : 64; }

hipError_t launch_attn_few(Dt dt, int d, const AttnArgs& a, hipStream_t s) {
  const unsigned grid = (unsigned)((int64_t)a.tok.N * a.splits * a.Hk);
  return by_dim(dt, d, [&](auto e, auto dim) {
    using E = decltype(e);
    constexpr int D = decltype(dim)::value;
    using F = Few<E, D>;
    if (a.block == 16)
      hipLaunchKernelGGL((k_attn_few<E, D, 1, F::KW, F::KT>), dim3(grid), dim3(64 * F::KW), 0, s, a);
    else
      hipLaunchKernelGGL((k_attn_few<E, D, 2, F::KW, F::KT>), dim3(grid), dim3(64 * F::KW), 0, s, a);
    return hipGetLastError();
  });
}

hipError_t launch_attn_tile(Dt dt, int d, int slots, const AttnArgs& a, hipStream_t s) {
  const unsigned grid = (unsigned)((int64_t)slots * a.splits * a.Hk);
  return by_dim(dt, d, [&](auto e, auto dim) {
    using E = decltype(e);
    constexpr int D = decltype(dim)::value;
    if (a.block == 64)
      hipLaunchKernelGGL((k_attn_tile<E, D, 1, Tile<E, D>::KT>), dim3(grid), dim3(256), 0, s, a, slots);
    else
      hipLaunchKernelGGL((k_attn_tile<E, D, 2, Tile<E, D>::KT>), dim3(grid), dim3(256), 0, s, a, slots);
    return hipGetLastError();
  });
}

hipError_t launch_attn_join(Dt dt, int d, const AttnArgs& a, hipStream_t s) {
  const int64_t rows = (int64_t)a.tok.total * a.Hq;
  return by_dim(dt, d, [&](auto e, auto dim) {
    using E = decltype(e);
    constexpr int D = decltype(dim)::value, T = D / 4, PER = 256 / T;
    if (a.splits <= 16)
      hipLaunchKernelGGL((k_attn_join<E, D, T>), dim3((unsigned)((rows + PER - 1) / PER)), dim3(256),
                         0, s, a);
    else
      hipLaunchKernelGGL((k_attn_join<E, D, 256>), dim3((unsigned)rows), dim3(256), 0, s, a);
    return hipGetLastError();
  });
}

}  // namespace gdn
