// C ABI of the attention layer: argument validation, workspace and launch
// sizes.  Every check runs before the first launch; nothing here allocates,
// frees or synchronises.
#include <math.h>
#include <stdint.h>
#include <string.h>

#include <algorithm>

#include "../../include/gdn_paged.h"
#include "gdn_paged_kernels.h"

namespace {

using gdn::AttnArgs;
using gdn::Dt;

constexpr int64_t MAX_STRIDE = (int64_t)1 << 27;  // bytes between slots of a page
constexpr int64_t MAX_PAGES = (int64_t)1 << 20;   // of a book

bool aligned(const void* p, size_t n) { return ((uintptr_t)p & (n - 1)) == 0; }
size_t up(size_t x) { return (x + 255) / 256 * 256; }
Dt type_of(gdn_dtype d) { return d == GDN_F32 ? Dt::F32 : Dt::BF16; }
int size_of(gdn_dtype d) { return d == GDN_F32 ? 4 : 2; }
gdn_status done(hipError_t e) { return e == hipSuccess ? GDN_OK : GDN_ERR_HIP; }

gdn_status check_tokens(const gdn_tokens* t, gdn::Tokens* out) {
  if (!t) return GDN_ERR_NULL;
  if (t->dtype != GDN_F32 && t->dtype != GDN_BF16) return GDN_ERR_UNSUPPORTED;
  if (t->d != 64 && t->d != 128 && t->d != 256) return GDN_ERR_UNSUPPORTED;
  if (t->B < 1 || t->T < 1 || t->Hq < 1 || t->Hk < 1) return GDN_ERR_SHAPE;
  const int64_t total = (int64_t)t->B * t->T;
  // rows (tokens x heads) are counted in 31 bits
  if (total * std::max(t->Hq, t->Hk) >= (int64_t)1 << 31) return GDN_ERR_SHAPE;
  out->total = (int)total;
  out->cu = t->cu_seqlens;
  out->N = t->B;
  out->T = t->T;
  if (t->cu_seqlens) {
    if (t->B != 1) return GDN_ERR_SHAPE;
    const int32_t* cu = t->cu_seqlens_host;
    if (!cu || t->num_seqs < 1 || cu[0] != 0 || cu[t->num_seqs] != t->T) return GDN_ERR_CU_SEQLENS;
    for (int n = 0; n < t->num_seqs; ++n)
      if (cu[n + 1] < cu[n]) return GDN_ERR_CU_SEQLENS;
    if (!aligned(t->cu_seqlens, 4)) return GDN_ERR_ALIGN;
    out->N = t->num_seqs;
    out->T = 0;
  } else if (t->cu_seqlens_host) {
    return GDN_ERR_CU_SEQLENS;
  }
  return GDN_OK;
}

// A row tensor (nullptr or no data: absent) in bytes.
gdn_status check_rows(const gdn_rows* r, int esz, gdn::Rows* out) {
  if (!r || !r->data) return GDN_ERR_NULL;
  if (!aligned(r->data, 16) || r->token_stride * esz % 16 || r->head_stride * esz % 16)
    return GDN_ERR_ALIGN;
  out->data = (unsigned char*)r->data;
  out->ts = r->token_stride * esz;
  out->hs = r->head_stride * esz;
  return GDN_OK;
}

gdn_status check_cache(const gdn_cache* c, int esz, bool pointers, gdn::Cache* out) {
  if (!c) return GDN_ERR_NULL;
  if (c->num_pages < 1 || c->max_blocks < 1 || c->page_size < 16 || c->page_size > 1024 ||
      (c->page_size & (c->page_size - 1)))
    return GDN_ERR_SHAPE;
  // the kernels look a few tiles past a range of keys, and ranges are whole tiles
  if ((int64_t)c->max_blocks * c->page_size > ((int64_t)1 << 31) - (1 << 18)) return GDN_ERR_SHAPE;
  if (pointers) {
    if (!c->k || !c->v || !c->table || !c->kv_lens) return GDN_ERR_NULL;
    if (!aligned(c->k, 16) || !aligned(c->v, 16) || !aligned(c->table, 4) ||
        !aligned(c->kv_lens, 4) || !aligned(c->skip, 4) || c->page_stride * esz % 16 || c->head_stride * esz % 16 ||
        c->token_stride * esz % 16)
      return GDN_ERR_ALIGN;
    if (c->token_stride < 0 || c->token_stride * esz >= MAX_STRIDE) return GDN_ERR_SHAPE;
  }
  out->k = (unsigned char*)c->k;
  out->v = (unsigned char*)c->v;
  out->page = c->page_stride * esz;
  out->head = c->head_stride * esz;
  out->slot = c->token_stride * esz;
  out->table = c->table;
  out->lens = c->kv_lens;
  out->skip = c->skip;
  out->num_pages = c->num_pages;
  out->shift = 0;
  while ((1 << out->shift) < c->page_size) ++out->shift;
  out->max_blocks = c->max_blocks;
  return GDN_OK;
}

gdn_status check_rotary(const gdn_rotary* r, int d) {
  if (r->rot < 2 || r->rot > d || r->rot % 2 || (r->layout != 0 && r->layout != 1) ||
      !isfinite(r->scale))
    return GDN_ERR_VALUE;
  if (!r->turns) return GDN_ERR_NULL;
  return aligned(r->turns, 8) ? GDN_OK : GDN_ERR_ALIGN;
}

gdn_status rotate(const gdn_tokens* t, const gdn_rotary* r, const gdn_rows* q, const gdn_rows* k,
                  const int32_t* positions, const gdn_rows* q_out, const gdn_rows* k_out,
                  float sign, void* stream) {
  gdn::RotateArgs a;
  memset(&a, 0, sizeof a);
  gdn_status st = check_tokens(t, &a.tok);
  if (st != GDN_OK) return st;
  if (!r) return GDN_ERR_NULL;
  if ((st = check_rotary(r, t->d)) != GDN_OK) return st;
  const int esz = size_of(t->dtype);
  if ((st = check_rows(q, esz, &a.q)) != GDN_OK) return st;
  if ((st = check_rows(q_out, esz, &a.q_out)) != GDN_OK) return st;
  const bool has_k = k && k->data;
  if (has_k != (k_out && k_out->data)) return GDN_ERR_NULL;
  if (has_k) {
    if ((st = check_rows(k, esz, &a.k)) != GDN_OK) return st;
    if ((st = check_rows(k_out, esz, &a.k_out)) != GDN_OK) return st;
  }
  if (!aligned(positions, 4)) return GDN_ERR_ALIGN;
  a.positions = positions;
  a.turns = r->turns;
  a.Hq = t->Hq;
  a.Hk = t->Hk;
  a.d = t->d;
  a.rot = r->rot;
  a.layout = r->layout;
  a.scale = r->scale;
  a.sign = sign;
  return done(gdn::launch_rotate(type_of(t->dtype), a, (hipStream_t)stream));
}

// How a call's work is cut: which kernel, its row blocks, splits of their keys.
struct Plan {
  bool few = false;
  int block = 0;               // rows of a block
  int64_t slots = 0;           // blocks of the tile kernel's grid
  int splits = 1, len = 0;     // key ranges
  bool longest = false;        // longest row blocks of all sequences first
  size_t part = 0, bytes = 0;  // workspace: offset of {maximum, sum}; size
};

gdn_status plan_attn(const gdn_tokens* t, const gdn::Tokens& tok, const gdn_cache* c,
                     const gdn_attn* a, Plan* out) {
  if (!a) return GDN_ERR_NULL;
  if (!(a->scale > 0.f) || !isfinite(a->scale) || a->window < 0 || a->max_kv < 0 ||
      (a->window > 0 && !a->causal))
    return GDN_ERR_VALUE;
  if (t->Hq % t->Hk) return GDN_ERR_SHAPE;
  Plan p;
  const int64_t G = t->Hq / t->Hk;
  const Dt dt = type_of(t->dtype);
  int64_t seqs = 0, most = 0;           // sequences with new tokens; the most of one
  int64_t blocks64 = 0, blocks128 = 0;  // row blocks
  auto see = [&](int64_t m) {
    if (m == 0) return;
    ++seqs;
    most = std::max(most, m);
    blocks64 += (m * G + 63) / 64;
    blocks128 += (m * G + 127) / 128;
  };
  if (tok.cu) {
    for (int n = 0; n < tok.N; ++n) see(t->cu_seqlens_host[n + 1] - t->cu_seqlens_host[n]);
  } else {
    see(tok.T);
    seqs *= tok.N;
    blocks64 *= tok.N;
    blocks128 *= tok.N;
  }
  const int64_t room = (int64_t)c->max_blocks * c->page_size;
  const int64_t kv = std::max<int64_t>(1, a->max_kv > 0 ? std::min<int64_t>(a->max_kv, room) : room);
  // A block of m tokens sees at most window + m - 1 keys, and its range begins
  // at a multiple of 16.
  auto keys = [&](int64_t m) { return a->window > 0 ? std::min(kv, a->window + m + 14) : kv; };
  auto cut = [&](int64_t range, int64_t splits, int step) {
    p.len = (int)(((range + splits - 1) / splits + step - 1) / step * step);
    p.splits = (int)((range + p.len - 1) / p.len);
  };

  // Where every sequence has few rows, their kernel, whose waves take different
  // keys: 8 tokens of 4 heads over up to 4000 keys, 64 sequences, 57 us, in the
  // other 76; 12 sequences of up to 5 in fp32, 8 cache heads, up to 3000 keys 22 and
  // 44; fp32 single tokens over 2000 keys 93 and 149.  Bf16 single tokens that
  // fill the GPU take the same in both (a batch of 256 in a 2K window 149 and 147
  // us), and where their keys are so few that a workgroup's start counts, two of the
  // other to a CU are the faster (212 sequences, 8 cache heads: 70 keys 39 and 27
  // us, 500 94 and 87, 1000 156 and 160; 836 units of 3 keys 19 and 11; but 176 in
  // fp32, 2 cache heads, 317 keys 30 and 45).  With larger sequences beside them, all
  // in one launch of the other: 127 single tokens and 512 of one sequence over up to
  // 4000 keys 123 us, in a launch each (as before that) 150.
  const int64_t few_units = std::max<int64_t>(1, seqs * t->Hk), few_keys = keys(most);
  p.few = most * G <= gdn::FEW_ROWS &&
          (few_units <= 256 || few_keys * (dt == Dt::F32 ? 8 : 1) > 1024);
  if (p.few) {
    p.block = most * G <= 16 ? 16 : 32;
    // A workgroup of this kernel has a CU to itself (128 KB of LDS at most head
    // dims): 256 of them are wanted; more cost more partial sums than they
    // balance (two sequences of 131072 keys, 4 cache heads: 97 us, with 512 100,
    // with 2048 113; 12 of up to 3000 keys in fp32, 8 heads: 22.4 and 26.4).
    const int step = gdn::attn_few_keys(dt, t->d);
    const int64_t s = few_units >= 128 ? 1 : std::min((255 + few_units) / few_units, few_keys / step);
    cut(few_keys, std::max<int64_t>(1, s), step);
  } else {
    // Rows of a block and splits of its keys, by what each choice would take: a
    // start of 5 us; for 64 keys of 128 rows 0.8, 1.3 and 2.9 us at d = 64, 128 and
    // 256 in bf16 where a workgroup is alone on its CU, 4.7, 8.2 and 18 in fp32, 0.62 of
    // that with 64 rows (0.9 at d = 64, where it is the copies' latency); 1.5 (fp32 1.9)
    // times as long where two share it, 1.25 with three at d = 64; no less than half
    // of what the cache would take from HBM at its longest; with splits, the partial
    // sums' way through memory and the join's launch.  (1000 tokens of 16 heads, 4 cache
    // heads: 1 split 23 us, 3 46.  32 sequences of 100 tokens, 500 keys: blocks of 128
    // 32 us, of 64 38; 156 sequences, 175 tokens in one and one in the others, d = 256:
    // 29 and 20.)
    const int step = gdn::attn_tile_keys(dt, t->d);
    const bool f32 = dt == Dt::F32, thin = !f32 && t->d == 64;
    const double alone = t->d == 64 ? (f32 ? 4.7 : 0.8) : t->d == 128 ? (f32 ? 8.2 : 1.3)
                                                                     : (f32 ? 18. : 2.9);
    const double hbm = 1.0 * seqs * t->Hk * keys(most) * t->d * size_of(t->dtype) / 5.3e6;
    const double fit = thin ? 768 : 512, together = thin ? 1.25 : f32 ? 1.9 : 1.5;
    // In fp32 the matrix cores alone bind, so a block is slow beside a second one only as
    // long as that lasts.  Where the new tokens are much of the keys and sequences are
    // alike, the longest block has the shortest beside it, of `least` of its keys (two
    // prompts of 2048 tokens, 8 heads, 4 cache heads, d = 128: 168 us, without this term,
    // in 128 rows, 276; 5 of up to 900 88 and 139; one of 2000, 16 heads 163 and 270).  In
    // bf16 it would choose 64 rows where 128 are better (d = 256, 4096 tokens: 162 and 141).
    const bool pairs = f32 && a->causal && a->window == 0 && 2 * (int64_t)tok.total >= seqs * most;
    const double least = std::max(0., 1 - (double)most / kv);
    double best = 0;
    int64_t at = 0;
    for (int block : {128, 64}) {
      const int64_t units = (block == 64 ? blocks64 : blocks128) * t->Hk;
      const int64_t range = keys(std::min<int64_t>(most, block / G + 2));
      const double tile = alone * (block == 128 ? 1 : thin ? 0.9 : 0.62);
      for (int64_t s = 1; s <= gdn::MAX_SPLITS; s += s < 4 ? 1 : s / 4) {
        cut(range, s, step);
        const double n = (double)units * p.splits;
        if (at && p.splits > 1 && n > 1.5 * fit) break;  // far more than run at once: no gain
        double share = n <= 256 ? 1 : together * (n <= fit ? 1 : n / fit + 0.5);
        if (pairs && n > 256 && n <= 512 && p.splits == 1)
          share = std::max(1 + (together - 1) * least, together * (1 + least) / 2);
        const double us =
            std::max(p.len / 64.0 * tile * share, hbm) + 5 +
            (p.splits > 1 ? 5 + 8.0 * p.splits * tok.total * t->Hq * t->d / 8e6 : 0);
        if (!at || us < best) {
          best = us;
          at = s;
          p.block = block;
        }
        if (p.len == step) break;
      }
    }
    cut(keys(std::min<int64_t>(most, p.block / G + 2)), at, step);
    // Several sequences' blocks that do not all run at once start in the order of their
    // keys, or a long one begins when most of the GPU is done: 8 prompts in a 2K
    // window, d = 256, 171 us, in the sequences' order 209; 60 sequences of up to 300
    // tokens over up to 3000 keys 112 and 141; 8 of 2048 tokens 159 and 173 (2 of 4000
    // 142 and 137).  A lane holds a sequence: more than 64 come in their own order.  The bf16 blocks of d = 64 are too short for the search that finds
    // each its place (40 sequences in a window of 512: 66 and 59).
    p.longest = a->causal && !thin && tok.N > 1 && tok.N <= 64 &&
                (p.block == 64 ? blocks64 : blocks128) * t->Hk * p.splits > fit;
    p.slots = tok.cu ? (int64_t)tok.total * G / p.block + tok.N
                     : tok.N * (((int64_t)tok.T * G + p.block - 1) / p.block);
  }
  // a launch holds less than 2^32 threads, 256 to a workgroup
  if ((p.few ? tok.N : p.slots) * p.splits * t->Hk >= (int64_t)1 << 24)
    return GDN_ERR_SHAPE;
  if (p.splits > 1) {
    const int64_t rows = (int64_t)tok.total * t->Hq;
    p.part = up((size_t)(p.splits * rows * t->d * 4));
    p.bytes = p.part + up((size_t)(p.splits * rows * 8));
  }
  *out = p;
  return GDN_OK;
}

gdn_status check_book(const gdn_book* b, bool lens_out, gdn::Book* out) {
  if (!b) return GDN_ERR_NULL;
  if (b->S < 1 || b->max_blocks < 1 || b->num_pages < 1 || b->page_size < 1 ||
      b->num_pages > MAX_PAGES || b->S > MAX_PAGES || (int64_t)b->max_blocks * b->page_size >= (int64_t)1 << 31)
    return GDN_ERR_SHAPE;
  if (!b->table || !b->lens || !b->refs || !b->table_out || !b->refs_out ||
      (lens_out && !b->lens_out))
    return GDN_ERR_NULL;
  const void* ptrs[] = {b->table, b->lens, b->refs, b->table_out, b->lens_out, b->refs_out};
  for (const void* p : ptrs)
    if (!aligned(p, 4)) return GDN_ERR_ALIGN;
  *out = gdn::Book{b->S,    b->max_blocks, b->num_pages, b->page_size, b->table,
                   b->lens, b->refs,       b->table_out, b->lens_out,  b->refs_out};
  return GDN_OK;
}

gdn_status check_pool(const gdn_pool* p, gdn::Pool* out) {
  if (!p->data) return GDN_ERR_NULL;
  if (p->parts < 1 || p->num_pages < 1 || p->page_bytes < 16) return GDN_ERR_SHAPE;
  if (!aligned(p->data, 16) || p->part_stride % 16 || p->page_stride % 16 || p->page_bytes % 16)
    return GDN_ERR_ALIGN;
  *out = gdn::Pool{(unsigned char*)p->data, p->parts,       p->num_pages,
                   p->part_stride,          p->page_stride, p->page_bytes};
  return GDN_OK;
}

size_t carve_pages(int64_t S, int64_t blocks, int64_t pages, unsigned char* base,
                   gdn::PageWork* w) {
  size_t off = 0;
  auto take = [&](int64_t n) {
    int32_t* p = base ? (int32_t*)(base + off) : nullptr;
    off += up((size_t)n * 4);
    return p;
  };
  const int64_t list = std::max(S, pages);
  gdn::PageWork x;
  x.count = take(4);
  x.src = take(list);
  x.dst = take(list);
  x.heir = take(S);
  x.rank = take(S);
  x.lens = take(S);
  x.table = take(S * blocks);
  if (w) *w = x;
  return off;
}

gdn_status pages_call(const gdn_book* b, bool lens_out, const gdn_pool* pool, void* workspace,
                      size_t bytes, gdn::Book* book, gdn::Pool* pl, gdn::PageWork* w) {
  gdn_status st = check_book(b, lens_out, book);
  if (st != GDN_OK) return st;
  if (pool) {
    if ((st = check_pool(pool, pl)) != GDN_OK) return st;
    if (pool->num_pages != b->num_pages) return GDN_ERR_SHAPE;
  }
  if (workspace && !aligned(workspace, 16)) return GDN_ERR_ALIGN;
  const size_t need = carve_pages(b->S, b->max_blocks, b->num_pages, nullptr, nullptr);
  if (!workspace || bytes < need) return GDN_ERR_WORKSPACE;
  carve_pages(b->S, b->max_blocks, b->num_pages, (unsigned char*)workspace, w);
  return GDN_OK;
}

}  // namespace

extern "C" {

gdn_status gdn_rotary_turns(int32_t rot, double base, int32_t scaling, double factor,
                            double original, double slow, double fast, double* turns,
                            float* scale) {
  if (!turns || !scale) return GDN_ERR_NULL;
  if (rot < 2 || rot % 2 || !(base > 1) || !isfinite(base) || scaling < 0 || scaling > 3)
    return GDN_ERR_VALUE;
  if (scaling != GDN_ROTARY_PLAIN && (!(factor >= 1) || !isfinite(factor))) return GDN_ERR_VALUE;
  if (scaling == GDN_ROTARY_PARTS &&
      (!(original >= 1) || !isfinite(original) || !isfinite(slow) || !isfinite(fast) ||
       !(fast > slow)))
    return GDN_ERR_VALUE;
  const double turn = 6.283185307179586476925286766559;
  if (scaling == GDN_ROTARY_BASE && rot > 2) base *= pow(factor, (double)rot / (rot - 2));
  *scale = scaling == GDN_ROTARY_PARTS ? (float)(0.1 * log(factor) + 1.0) : 1.f;
  for (int i = 0; i < rot / 2; ++i) {
    double f = pow(base, -2.0 * i / rot) / turn;
    if (scaling == GDN_ROTARY_LINEAR) f /= factor;
    if (scaling == GDN_ROTARY_PARTS) {
      const double g = std::min(1.0, std::max(0.0, (original * f - slow) / (fast - slow)));
      f = f / factor * (1 - g) + f * g;
    }
    turns[i] = f;
  }
  return GDN_OK;
}

gdn_status gdn_rotary_fwd(const gdn_tokens* t, const gdn_rotary* r, const gdn_rows* q,
                          const gdn_rows* k, const int32_t* positions, const gdn_rows* q_out,
                          const gdn_rows* k_out, void* stream) {
  return rotate(t, r, q, k, positions, q_out, k_out, 1.f, stream);
}

gdn_status gdn_rotary_bwd(const gdn_tokens* t, const gdn_rotary* r, const gdn_rows* dq_out,
                          const gdn_rows* dk_out, const int32_t* positions, const gdn_rows* dq,
                          const gdn_rows* dk, void* stream) {
  return rotate(t, r, dq_out, dk_out, positions, dq, dk, -1.f, stream);
}

gdn_status gdn_cache_append(const gdn_tokens* t, const gdn_rotary* r, const gdn_rows* q,
                            const gdn_rows* k, const gdn_rows* v, const gdn_cache* cache,
                            const gdn_rows* q_out, void* stream) {
  gdn::RotateArgs a;
  memset(&a, 0, sizeof a);
  gdn_status st = check_tokens(t, &a.tok);
  if (st != GDN_OK) return st;
  const int esz = size_of(t->dtype);
  if (r && (st = check_rotary(r, t->d)) != GDN_OK) return st;
  if ((st = check_cache(cache, esz, true, &a.cache)) != GDN_OK) return st;
  if ((st = check_rows(k, esz, &a.k)) != GDN_OK) return st;
  if ((st = check_rows(v, esz, &a.v)) != GDN_OK) return st;
  const bool has_q = q && q->data;
  if (has_q != (q_out && q_out->data)) return GDN_ERR_NULL;
  if (has_q) {
    if ((st = check_rows(q, esz, &a.q)) != GDN_OK) return st;
    if ((st = check_rows(q_out, esz, &a.q_out)) != GDN_OK) return st;
  }
  a.Hq = t->Hq;
  a.Hk = t->Hk;
  a.d = t->d;
  a.append = 1;
  a.sign = 1.f;
  if (r) {
    a.turns = r->turns;
    a.rot = r->rot;
    a.layout = r->layout;
    a.scale = r->scale;
  }
  return done(gdn::launch_rotate(type_of(t->dtype), a, (hipStream_t)stream));
}

size_t gdn_cache_attn_workspace_size(const gdn_tokens* t, const gdn_cache* cache,
                                     const gdn_attn* a) {
  gdn::Tokens tok;
  gdn::Cache c;
  Plan p;
  if (check_tokens(t, &tok) != GDN_OK || check_cache(cache, 1, false, &c) != GDN_OK ||
      plan_attn(t, tok, cache, a, &p) != GDN_OK)
    return 0;
  return p.bytes;
}

gdn_status gdn_cache_attn(const gdn_tokens* t, const gdn_attn* at, const gdn_rows* q,
                          const gdn_cache* cache, const gdn_rows* o, float* lse, void* workspace,
                          size_t workspace_bytes, void* stream) {
  AttnArgs a;
  memset(&a, 0, sizeof a);
  gdn_status st = check_tokens(t, &a.tok);
  if (st != GDN_OK) return st;
  const int esz = size_of(t->dtype);
  if ((st = check_cache(cache, esz, true, &a.cache)) != GDN_OK) return st;
  if ((st = check_rows(q, esz, &a.q)) != GDN_OK) return st;
  if ((st = check_rows(o, esz, &a.o)) != GDN_OK) return st;
  if (!aligned(lse, 4)) return GDN_ERR_ALIGN;
  Plan p;
  if ((st = plan_attn(t, a.tok, cache, at, &p)) != GDN_OK) return st;
  if (p.bytes) {
    if (!workspace || workspace_bytes < p.bytes) return GDN_ERR_WORKSPACE;
    if (!aligned(workspace, 16)) return GDN_ERR_ALIGN;
    a.part = (float*)workspace;
    a.part_ml = (float*)((unsigned char*)workspace + p.part);
  }
  a.lse = lse;
  a.Hq = t->Hq;
  a.Hk = t->Hk;
  a.G = t->Hq / t->Hk;
  a.causal = at->causal != 0;
  a.window = at->window;
  a.c = at->scale * 1.4426950408889634f;
  const Dt dt = type_of(t->dtype);
  hipStream_t s = (hipStream_t)stream;
  a.block = p.block;
  a.splits = p.splits;
  a.len = p.len;
  a.longest = p.longest;
  hipError_t e = p.few ? gdn::launch_attn_few(dt, t->d, a, s)
                       : gdn::launch_attn_tile(dt, t->d, (int)p.slots, a, s);
  if (e == hipSuccess && p.splits > 1) e = gdn::launch_attn_join(dt, t->d, a, s);
  return done(e);
}

size_t gdn_pages_workspace_size(const gdn_book* b) {
  if (!b || b->S < 1 || b->max_blocks < 1 || b->num_pages < 1 ||
      b->num_pages > MAX_PAGES || b->S > MAX_PAGES)
    return 0;
  return carve_pages(b->S, b->max_blocks, b->num_pages, nullptr, nullptr);
}

gdn_status gdn_pages_extend(const gdn_book* b, const int32_t* add, int32_t* short_of,
                            void* workspace, size_t workspace_bytes, void* stream) {
  gdn::Book book;
  gdn::PageWork w;
  gdn_status st = pages_call(b, true, nullptr, workspace, workspace_bytes, &book, nullptr, &w);
  if (st != GDN_OK) return st;
  if (!add || !short_of) return GDN_ERR_NULL;
  if (!aligned(add, 4) || !aligned(short_of, 4)) return GDN_ERR_ALIGN;
  return done(gdn::launch_extend(book, add, short_of, w, (hipStream_t)stream));
}

gdn_status gdn_pages_select(const gdn_book* b, const int32_t* parents, const gdn_pool* pool,
                            int32_t* short_of, void* workspace, size_t workspace_bytes,
                            void* stream) {
  gdn::Book book;
  gdn::Pool pl;
  gdn::PageWork w;
  gdn_status st = pages_call(b, true, pool, workspace, workspace_bytes, &book, &pl, &w);
  if (st != GDN_OK) return st;
  if (!parents || !short_of) return GDN_ERR_NULL;
  if (!aligned(parents, 4) || !aligned(short_of, 4)) return GDN_ERR_ALIGN;
  return done(gdn::launch_select(book, parents, pool ? &pl : nullptr, short_of, w,
                                 (hipStream_t)stream));
}

gdn_status gdn_pages_compact(const gdn_book* b, const gdn_pool* pool, int32_t* map,
                             void* workspace, size_t workspace_bytes, void* stream) {
  gdn::Book book;
  gdn::Pool pl;
  gdn::PageWork w;
  gdn_status st = pages_call(b, false, pool, workspace, workspace_bytes, &book, &pl, &w);
  if (st != GDN_OK) return st;
  if (!map) return GDN_ERR_NULL;
  if (!aligned(map, 4)) return GDN_ERR_ALIGN;
  return done(gdn::launch_compact(book, pool ? &pl : nullptr, map, w, (hipStream_t)stream));
}

gdn_status gdn_pages_copy(const gdn_pool* pool, const int32_t* src, const int32_t* dst, int32_t n,
                          void* stream) {
  if (!pool) return GDN_ERR_NULL;
  gdn::Pool pl;
  gdn_status st = check_pool(pool, &pl);
  if (st != GDN_OK) return st;
  if (n < 0) return GDN_ERR_SHAPE;
  if (n == 0) return GDN_OK;
  if (!src || !dst) return GDN_ERR_NULL;
  if (!aligned(src, 4) || !aligned(dst, 4)) return GDN_ERR_ALIGN;
  return done(gdn::launch_move(pl, src, dst, n, (hipStream_t)stream));
}

}  // extern "C"
