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

// Checks a problem and fills in its description.
gdn_status check_problem(const gdn_problem* p, LinearArgs* a) {
  if (!p) return GDN_ERR_NULL;
  if (p->dtype != GDN_F32 && p->dtype != GDN_BF16) return GDN_ERR_UNSUPPORTED;
  if (p->B < 1 || p->T < 1 || p->H < 1) return GDN_ERR_SHAPE;
  if (p->dk != 64 && p->dk != 128 && p->dk != 256) return GDN_ERR_UNSUPPORTED;
  if (p->dv != 64 && p->dv != 128 && p->dv != 256 && p->dv != 512) return GDN_ERR_UNSUPPORTED;
  const int64_t total = (int64_t)p->B * p->T;
  if (total >= ((int64_t)1 << 31) - 256) return GDN_ERR_SHAPE;  // (chunks past the end are asked for)
  memset(a, 0, sizeof *a);
  a->N = p->B;
  a->T = p->T;
  a->H = p->H;
  a->dk = p->dk;
  a->dv = p->dv;
  if (p->cu_seqlens) {
    if (p->B != 1) return GDN_ERR_SHAPE;
    const int32_t* cu = p->cu_seqlens_host;
    if (!cu || p->num_seqs < 1 || cu[0] != 0 || cu[p->num_seqs] != p->T) return GDN_ERR_CU_SEQLENS;
    for (int n = 0; n < p->num_seqs; ++n)
      if (cu[n + 1] < cu[n]) return GDN_ERR_CU_SEQLENS;
    a->cu = p->cu_seqlens;
    a->N = p->num_seqs;
  } else if (p->cu_seqlens_host) {
    return GDN_ERR_CU_SEQLENS;
  }
  if ((int64_t)a->N * a->H * (a->dk * a->dv / 1024) >= MAX_GRID) return GDN_ERR_SHAPE;
  return GDN_OK;
}

// What a chunk takes, in us: of a workgroup that has its CU to itself, of one of as many as
// a CU holds, and how many those are.  (The weights of a choice: in bf16 a chunk takes 3 to 15%
// more, which added to these picks worse lengths for packed prompts, 512 for 1024.)
struct Pace {
  double alone, full;
  int held;
};
Pace pace(Dt dt, int dk, int slice) {
  if (dt == Dt::F32) {
    if (dk == 64) return slice == 64 ? Pace{6.1, 9, 2} : Pace{7, 7, 1};
    return dk == 256 ? Pace{15, 15, 1} : slice == 64 ? Pace{10, 10, 1} : Pace{13, 13, 1};
  }
  if (dk == 64) return slice == 64 ? Pace{2.5, 5, 3} : Pace{3.4, 5.8, 2};
  if (dk == 128) return slice == 64 ? Pace{3.5, 5.2, 2} : Pace{5.5, 10.3, 2};
  return slice == 64 ? Pace{5.9, 5.9, 1} : Pace{7, 7, 1};
}

// How the sequences are cut, by what each length of the segments would take; bytes of the
// segments' states.  Cut: the walk is shorter where it does not fill the GPU, or where long
// sequences outlast the others, but what the segments add has to be found first (0.35 of
// the walk's time a chunk, for all but each sequence's last) and their states pass through
// memory four times.  (us, whole | segments of 64, 128, 256, 512, 1024, 2048 tokens, * the rule's; bf16:
// 16 packed prompts of up to 8192 tokens, 16 heads of 128 x 128, 899 | -, 795, 587, 515, 482*, 577; one
// of 8192 820 | 158, 115, 88, 97*, 153, 284, of 512 54 | 28*, 32, 45, four of 300 37* | 37, 37, 51; 8 of
// 4096, 6 heads of 256 x 512, 485* | -, -, 856, 673, 599, 634, one of 1000 119 | 66, 48*, 65, 101; fp32,
// two of 1001, 4 heads of 64 x 64, 89 | 20*, 26, 41, 71.)
size_t plan(const gdn_problem* p, LinearArgs* a) {
  const int slice = gdn::linear_slice(type_of(p->dtype), a->dk, a->dv);
  const Pace pc = pace(type_of(p->dtype), a->dk, slice);
  const double units = a->H * (a->dv / slice), state = 4.0 * a->H * a->dk * a->dv;
  const int64_t total = (int64_t)p->B * p->T;
  auto run = [&](double segments, double longest, double chunks) {
    const double w = segments * units;
    if (w <= 256) return longest * pc.alone;
    if (w <= 256.0 * pc.held)
      return longest * (pc.alone + (pc.full - pc.alone) * (w / 256 - 1) / std::max(1, pc.held - 1));
    // (more than a CU holds at once: the last to start outlast the others)
    return std::max(longest * pc.full, chunks * units * pc.full / (256.0 * pc.held) + longest * pc.full / 2);
  };
  int64_t most = 0;  // tokens of the longest
  auto cost = [&](int64_t len) {
    double segments = 0, chunks = 0, before = 0, longest = 0;
    auto see = [&](int64_t m, int64_t times) {
      const int64_t n = m > 0 ? (m - 1) / len + 1 : 1;
      segments += (double)n * times;
      chunks += (double)((m + 63) / 64) * times;
      before += (double)((n - 1) * (len / 64)) * times;
      longest = std::max(longest, (double)((std::min(m, len) + 63) / 64));
      most = std::max(most, m);
    };
    if (a->cu)
      for (int n = 0; n < a->N; ++n) see(p->cu_seqlens_host[n + 1] - p->cu_seqlens_host[n], 1);
    else
      see(p->T, a->N);
    double us = run(segments, longest, chunks);
    if (before > 0)
      us += 0.35 * run(segments - a->N, len / 64, before) + 4 * segments * state / 5e6 + 8;
    return us;
  };
  a->len = 0;
  a->slots = a->N;
  double best = cost((int64_t)1 << 40);
  for (int64_t len = 64; len < most; len *= 2) {
    const int64_t slots = a->cu ? total / len + a->N : a->N * ((p->T - 1) / len + 1);
    if (slots * a->H * (a->dv / 64) >= MAX_GRID) continue;
    const double us = cost(len);
    if (us < best) {
      best = us;
      a->len = (int)len;
      a->slots = (int)slots;
    }
  }
  if (a->len == 0) return 0;
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
  return check_problem(p, &a) == GDN_OK ? plan(p, &a) : 0;
}

gdn_status gdn_linear_chunk_fwd(const gdn_problem* p, const void* q, const void* k, const void* v,
                                const float* log_alpha, int32_t per_head, const float* h0, void* o,
                                float* ht, void* workspace, size_t workspace_bytes, void* stream) {
  LinearArgs a;
  gdn_status st = check_problem(p, &a);
  if (st != GDN_OK) return st;
  if ((st = fill(p, q, k, v, log_alpha, per_head, h0, o, ht, &a)) != GDN_OK) return st;
  const size_t need = plan(p, &a);
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
  gdn_status st = check_problem(p, &a);
  if (st != GDN_OK) return st;
  if ((st = fill(p, q, k, v, log_alpha, per_head, h0, o, ht, &a)) != GDN_OK) return st;
  return done(gdn::launch_linear_recurrent(type_of(p->dtype), a, (hipStream_t)stream));
}

}  // extern "C"
