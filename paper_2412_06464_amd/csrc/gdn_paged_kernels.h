// Kernel argument blocks and launcher declarations of the attention layer
// (rotary positions, paged cache, attention over it, management of pages).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "gdn_kernels.h"

namespace gdn {

// The tokens of a call: dense rows of T tokens (cu == nullptr) or packed.
struct Tokens {
  const int32_t* cu;  // device boundaries [N + 1] or nullptr
  int N;              // sequences
  int T;              // dense: tokens of each
  int total;          // tokens in all
};

struct Rows {  // row (token, head) at data + token * ts + head * hs (bytes)
  unsigned char* data;
  int64_t ts, hs;
};

struct Cache {
  unsigned char *k, *v;
  int64_t page, head, slot;  // strides in bytes
  const int32_t* table;      // [N, max_blocks]
  const int32_t* lens;       // [N]
  const int32_t* skip;       // [N] or nullptr: non-zero: taken as holding no tokens
  int num_pages, shift, max_blocks;  // page_size = 1 << shift
};

struct RotateArgs {
  Tokens tok;
  Rows q, k, v, q_out, k_out;  // data null: absent
  Cache cache;                 // append: where k and v go (k_out unused)
  const int32_t* positions;    // or nullptr: place in the sequence
  const double* turns;         // [rot / 2]
  int Hq, Hk, d, rot, layout, append;
  float scale, sign;           // sign: 1 forward, -1 backward
  int per;                     // tokens of a workgroup
};
hipError_t launch_rotate(Dt dt, RotateArgs a, hipStream_t s);

struct AttnArgs {
  Tokens tok;
  Rows q, o;
  Cache cache;
  float* lse;       // [tokens, Hq] or nullptr
  float* part;      // [splits][tokens * Hq][d] unnormalised sums, then
  float* part_ml;   // [splits][tokens * Hq][2] {maximum (log2), sum}
  int Hq, Hk, G;    // G = Hq / Hk
  int causal, window;
  float c;          // scale * log2(e)
  int block;        // rows of a block
  int splits, len;  // key ranges of `len` keys (the last: all that follow)
  int longest;      // row blocks of all sequences in the order of their keys
};
// Calls whose sequences have at most this many rows (new tokens x query heads of a
// cache head) take the kernel whose waves share the rows and split the keys.
constexpr int FEW_ROWS = 32;
constexpr int MAX_SPLITS = 512;

// keys of a tile: the unit of `len`
int attn_few_keys(Dt dt, int d);
int attn_tile_keys(Dt dt, int d);
// a.block: 16 or 32 rows, no sequence more
hipError_t launch_attn_few(Dt dt, int d, const AttnArgs& a, hipStream_t s);
// a.block: 64 or 128 rows; slots: row blocks
hipError_t launch_attn_tile(Dt dt, int d, int slots, const AttnArgs& a, hipStream_t s);
hipError_t launch_attn_join(Dt dt, int d, const AttnArgs& a, hipStream_t s);

struct Book {
  int S, max_blocks, num_pages, page_size;
  const int32_t *table, *lens, *refs;
  int32_t *table_out, *lens_out, *refs_out;
};
struct Pool {
  unsigned char* data;
  int parts, num_pages;
  int64_t part, page, bytes;
};
// Workspace of the page calls.
struct PageWork {
  int32_t* count;   // [4] counters
  int32_t* src;     // [max(S, num_pages)] pages to copy from
  int32_t* dst;     // [max(S, num_pages)] and to; pages given out
  int32_t* heir;    // [S]
  int32_t* rank;    // [S]
  int32_t* lens;    // [S] old lengths (a call in place)
  int32_t* table;   // [S, max_blocks] old rows (a call in place)
};
hipError_t launch_extend(const Book& b, const int32_t* add, int32_t* short_of, const PageWork& w,
                         hipStream_t s);
// (pool: nullptr where no data moves)
hipError_t launch_select(const Book& b, const int32_t* parents, const Pool* pool,
                         int32_t* short_of, const PageWork& w, hipStream_t s);
hipError_t launch_compact(const Book& b, const Pool* pool, int32_t* map, const PageWork& w,
                          hipStream_t s);
// Copies page src[i] to dst[i], i < n (n >= 1).
hipError_t launch_move(const Pool& p, const int32_t* src, const int32_t* dst, int n,
                       hipStream_t s);

// ---- device helpers

// Sequence of token t: the last n with cu[n] <= t < cu[n + 1].
__device__ inline int seq_of(const Tokens& k, int t) {
  if (!k.cu) return t / k.T;
  int lo = 0, hi = k.N;  // cu[lo] <= t < cu[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (k.cu[mid] <= t) lo = mid; else hi = mid;
  }
  return lo;
}
__device__ inline int seq_start(const Tokens& k, int n) { return k.cu ? k.cu[n] : n * k.T; }
// Tokens a sequence holds in the cache, within what its row of the table can; none if it
// is to be left alone (LIST false: there is no list of those).
template <bool LIST = true> __device__ inline int cached(const Cache& c, int n) {
  const int64_t most = (int64_t)c.max_blocks << c.shift;
  const int x = c.lens[n];
  int skip = 0;
  // (without a list the length once more, a load beside the other: a branch around it
  // would stand between the loads before and behind it)
  if (LIST) skip = (c.skip ? c.skip : c.lens)[n];
  return x < 0 || (LIST && c.skip && skip != 0) ? 0 : (x > most ? (int)most : x);
}

}  // namespace gdn
