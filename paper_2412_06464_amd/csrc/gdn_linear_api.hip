// C ABI of linear attention with a decay: argument validation, workspace and launch
// sizes.  Every check runs before the first launch; nothing here allocates,
// frees or synchronises.
#include <stdint.h>
#include <string.h>

#include <algorithm>

#include "../../include/gdn_linear.h"
#include "gdn_linear.h"

namespace {

using gdn::Dt;
using gdn::LinearArgs;

constexpr int64_t MAX_GRID = (int64_t)1 << 24;  // workgroups of 256: a launch holds under 2^32 threads

bool aligned16(const void* p) { return ((uintptr_t)p & 15u) == 0; }
size_t up(size_t x) { return (x + 255) / 256 * 256; }
Dt type_of(gdn_dtype d) { return d == GDN_F32 ? Dt::F32 : Dt::BF16; }
gdn_status done(hipError_t e) { return e == hipSuccess ? GDN_OK : GDN_ERR_HIP; }

// Checks a problem and fills in its description; *longest: tokens of the longest sequence.
gdn_status check_problem(const gdn_problem* p, LinearArgs* a, int64_t* longest) {
  if (!p) return GDN_ERR_NULL;
  if (p->dtype != GDN_F32 && p->dtype != GDN_BF16) return GDN_ERR_UNSUPPORTED;
  if (p->B < 1 || p->T < 1 || p->H < 1) return GDN_ERR_SHAPE;
  if (p->dk != 64 && p->dk != 128 && p->dk != 256) return GDN_ERR_UNSUPPORTED;
  if (p->dv != 64 && p->dv != 128 && p->dv != 256 && p->dv != 512) return GDN_ERR_UNSUPPORTED;
  const int64_t total = (int64_t)p->B * p->T;
  if (total >= ((int64_t)1 << 31) - 64) return GDN_ERR_SHAPE;  // (a chunk past the end is looked at)
  memset(a, 0, sizeof *a);
  a->N = p->B;
  a->T = p->T;
  a->H = p->H;
  a->dk = p->dk;
  a->dv = p->dv;
  *longest = p->T;
  if (p->cu_seqlens) {
    if (p->B != 1) return GDN_ERR_SHAPE;
    const int32_t* cu = p->cu_seqlens_host;
    if (!cu || p->num_seqs < 1 || cu[0] != 0 || cu[p->num_seqs] != p->T) return GDN_ERR_CU_SEQLENS;
    *longest = 0;
    for (int n = 0; n < p->num_seqs; ++n) {
      if (cu[n + 1] < cu[n]) return GDN_ERR_CU_SEQLENS;
      *longest = std::max<int64_t>(*longest, cu[n + 1] - cu[n]);
    }
    a->cu = p->cu_seqlens;
    a->N = p->num_seqs;
  } else if (p->cu_seqlens_host) {
    return GDN_ERR_CU_SEQLENS;
  }
  if ((int64_t)a->N * a->H * (a->dk * a->dv / 1024) >= MAX_GRID) return GDN_ERR_SHAPE;
  return GDN_OK;
}

// How the sequences are cut; bytes of the segments' states.
size_t plan(const gdn_problem* p, int64_t longest, LinearArgs* a) {
  const int64_t slices = a->dv / gdn::linear_slice(type_of(p->dtype), a->dk, a->dv);
  const int64_t total = (int64_t)p->B * p->T;
  const int64_t whole = a->N * a->H * slices;
  a->slots = a->N;
  a->len = 0;
  if (whole >= 256 || longest <= 512) return 0;
  const int64_t want = 512 / (a->H * slices);  // segments
  const int64_t len = std::max<int64_t>(256, (total + want * 64 - 1) / std::max<int64_t>(1, want * 64) * 64);
  if (len >= longest) return 0;
  a->len = (int)len;
  a->slots = a->cu ? (int)(total / len + a->N) : (int)(a->N * ((p->T - 1) / len + 1));
  return up((size_t)a->slots * a->H * a->dk * a->dv * 4) + up((size_t)a->slots * a->H * 4);
}

gdn_status fill(const gdn_problem* p, const void* q, const void* k, const void* v,
                const float* log_alpha, int32_t per_head, const float* h0, void* o, float* ht,
                LinearArgs* a) {
  if (!q || !k || !v || !o) return GDN_ERR_NULL;
  const void* ptrs[] = {q, k, v, log_alpha, h0, o, ht};
  for (const void* x : ptrs)
    if (!aligned16(x)) return GDN_ERR_ALIGN;
  a->q = q;
  a->k = k;
  a->v = v;
  a->o = o;
  a->log_alpha = log_alpha;
  a->per_head = per_head != 0;
  a->h0 = h0;
  a->ht = ht;
  return GDN_OK;
}

}  // namespace

extern "C" {

size_t gdn_linear_chunk_fwd_workspace_size(const gdn_problem* p) {
  LinearArgs a;
  int64_t longest;
  return check_problem(p, &a, &longest) == GDN_OK ? plan(p, longest, &a) : 0;
}

gdn_status gdn_linear_chunk_fwd(const gdn_problem* p, const void* q, const void* k, const void* v,
                                const float* log_alpha, int32_t per_head, const float* h0, void* o,
                                float* ht, void* workspace, size_t workspace_bytes, void* stream) {
  LinearArgs a;
  int64_t longest;
  gdn_status st = check_problem(p, &a, &longest);
  if (st != GDN_OK) return st;
  if ((st = fill(p, q, k, v, log_alpha, per_head, h0, o, ht, &a)) != GDN_OK) return st;
  const size_t need = plan(p, longest, &a);
  const Dt dt = type_of(p->dtype);
  const hipStream_t s = (hipStream_t)stream;
  if (need) {
    if (!workspace || workspace_bytes < need) return GDN_ERR_WORKSPACE;
    if (!aligned16(workspace)) return GDN_ERR_ALIGN;
    a.states = (float*)workspace;
    a.fade = (float*)((unsigned char*)workspace + up((size_t)a.slots * a.H * a.dk * a.dv * 4));
    const hipError_t e = gdn::launch_linear_states(dt, a, s);
    if (e != hipSuccess) return GDN_ERR_HIP;
  }
  return done(gdn::launch_linear_walk(dt, a, s));
}

gdn_status gdn_linear_recurrent_fwd(const gdn_problem* p, const void* q, const void* k,
                                    const void* v, const float* log_alpha, int32_t per_head,
                                    const float* h0, void* o, float* ht, void* stream) {
  LinearArgs a;
  int64_t longest;
  gdn_status st = check_problem(p, &a, &longest);
  if (st != GDN_OK) return st;
  if ((st = fill(p, q, k, v, log_alpha, per_head, h0, o, ht, &a)) != GDN_OK) return st;
  return done(gdn::launch_linear_recurrent(type_of(p->dtype), a, (hipStream_t)stream));
}

}  // extern "C"
