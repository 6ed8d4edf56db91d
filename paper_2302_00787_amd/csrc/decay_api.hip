// C ABI of linear attention with a decay for each head: argument validation, segments and workspaces, launches.
#include "../../include/favorsharp.h"

#include <algorithm>
#include <cmath>

#include "api_common.h"
#include "decay_common.h"

using namespace fs;

namespace {

constexpr long long kMaxRows = 1 << 29;          // rows of one state in a call: they are counted in 32 bits

// Segments of a sequence, as many as give the chip workgroups enough (`full`: two eight-wave ones a CU for wide rows, three of four
// waves for others), of four chunks at least, of two where that leaves CUs without one; the query heads of a key head in workgroups of
// their own where that does, too.
struct Plan {
  int nseg, seg_rows, parts;
  size_t states, ends, total;                    // bytes of one set of segment states; of the states that end a walk; of a workspace
};
Plan plan(int B, int H, int heads, int L, int d, int dv, int sets, bool ends) {
  Plan p;
  const int chunks = ceil_div(std::max(L, 1), dec::kChunk), G = H / heads;
  const bool wide = std::max(d, dv) > 64;
  const long long full = wide ? 512 : 768, states = (long long)B * heads;
  long long nseg = 1;
  if (states < 512) {
    nseg = std::min<long long>((full + states - 1) / states, chunks / 4);
    if (states * nseg < 256) nseg = std::min<long long>((256 + states - 1) / states, chunks / 2);
    nseg = std::max<long long>(nseg, 1);
  }
  const int each = ceil_div(chunks, (int)nseg);
  p.nseg = ceil_div(chunks, each);
  p.seg_rows = each * dec::kChunk;
  p.parts = states * p.nseg < 512 ? G : 1;
  p.states = p.nseg > 1 ? align_up((size_t)B * heads * p.nseg * d * dv * sizeof(float)) : 0;
  p.ends = ends ? align_up((size_t)B * heads * d * dv * sizeof(float)) : 0;
  p.total = sets * p.states + p.ends;
  return p;
}
// Workgroups that share the heads of a state read the pool that one of them would write where a call is in place: the states after it stay in
// the workspace until all have ended.  (Segments read copies of the states before them.)  That is a launch more: 32 heads, 8 key heads of 64, a prompt
// of 64 in bf16 11 us into another pool, 14 in place; 63 such sequences 16 and 24.
Plan plan_forward(int B, int H, int heads, int L, int d, int dv) {
  Plan p = plan(B, H, heads, L, d, dv, 1, false);
  if (p.nseg == 1 && p.parts > 1) p.total = p.ends = align_up((size_t)B * heads * d * dv * sizeof(float));
  return p;
}
Plan plan_backward(int B, int H, int heads, int L, int d, int dv, bool dbefore) { return plan(B, H, heads, L, d, dv, 2, dbefore); }

int sizes(int B, int H, int heads, int L, int d, int dv) {
  if (B < 1 || L < 0 || d < 1 || dv < 1 || H < 1 || heads < 1 || H % heads) return FS_ERR_INVALID_ARG;
  if (d > 128 || dv > 128 || !sequences_ok(B, H) || (long long)L * (H / heads) > kMaxRows) return FS_ERR_UNSUPPORTED;
  return FS_OK;
}
// offsets within a chunk of rows have 32 bits
constexpr int64_t kMaxStride = 1 << 22;
bool strides_ok(std::initializer_list<const fs_tensor*> list, int L) {
  for (const fs_tensor* t : list)
    if (L > 1 && t->stride_l > kMaxStride) return false;
  return true;
}
// (a sequence of one row may have any stride from row to row: a pitch that fits, as none is used)
TensorDev rows_of(const fs_tensor* t, int L) {
  TensorDev x = dev(t);
  if (L <= 1) x.sl = 128;
  return x;
}
int pools(std::initializer_list<const fs_decay_state*> list, int heads, int* slots) {
  *slots = 0;
  for (const fs_decay_state* s : list) {
    if (s == nullptr) continue;
    if (s->S == nullptr || (uintptr_t)s->S % 16 || s->slots < 1 || (*slots && *slots != s->slots)) return FS_ERR_INVALID_ARG;
    if (!sequences_ok(s->slots, heads)) return FS_ERR_UNSUPPORTED;
    *slots = s->slots;
  }
  return FS_OK;
}
bool numbers_ok(const float* log_decay, float scale, const int32_t* slots, const int32_t* lengths) {
  return log_decay != nullptr && (uintptr_t)log_decay % 4 == 0 && std::isfinite(scale) && (uintptr_t)slots % 4 == 0 && (uintptr_t)lengths % 4 == 0;
}
dec::Call call_of(int B, int heads, int L, int d, int dv, const float* log_decay, const int32_t* lengths, const int32_t* slots, int nslots, int unique,
                  const Plan& p, int32_t* left_out) {
  return dec::Call{B, heads, L, lengths, nslots ? slots : nullptr, nslots, unique, log_decay, p.nseg, p.seg_rows, d * dv, left_out};
}

}  // namespace

extern "C" {

size_t favorsharp_decay_attention_workspace_bytes(int B, int H, int heads, int L, int d, int dv) {
  return sizes(B, H, heads, L, d, dv) == FS_OK ? plan_forward(B, H, heads, L, d, dv).total : 0;
}

int favorsharp_decay_attention(const fs_tensor* Q, const fs_tensor* K, const fs_tensor* V, int B, int H, int heads, int L, int d, int dv,
                               const float* log_decay, float scale, const fs_decay_state* before, const fs_decay_state* after,
                               const int32_t* slots, const int32_t* lengths, const fs_tensor* Y, int32_t* left_out, void* workspace,
                               size_t workspace_bytes, void* stream) {
  int nslots;
  if (int rc = sizes(B, H, heads, L, d, dv)) return rc;
  if (int rc = pools({before, after}, heads, &nslots)) return rc;
  if (!numbers_ok(log_decay, scale, slots, lengths) || (uintptr_t)left_out % 4 || (uintptr_t)workspace % 16) return FS_ERR_INVALID_ARG;
  if (!tensor_ok(Q, d, L > 0) || !tensor_ok(K, d, L > 0) || !tensor_ok(V, dv, L > 0) || !tensor_ok(Y, dv, L > 0)) return FS_ERR_INVALID_ARG;
  if (Q->dtype != K->dtype || Q->dtype != V->dtype) return FS_ERR_INVALID_ARG;
  if (!strides_ok({Q, K, V, Y}, L)) return FS_ERR_UNSUPPORTED;
  const Plan p = plan_forward(B, H, heads, L, d, dv);
  const bool apart = p.ends > 0 && before != nullptr && after != nullptr && before->S == after->S;
  const size_t need = p.states + (apart ? p.ends : 0);
  if (need > 0 && workspace == nullptr) return FS_ERR_INVALID_ARG;
  if (workspace_bytes < need) return FS_ERR_WORKSPACE_TOO_SMALL;
  if (L == 0 && after == nullptr) return FS_OK;
  hipStream_t s = (hipStream_t)stream;
  float *states = (float*)workspace, *ends = (float*)((char*)workspace + p.states);
  dec::WalkSet a{};
  a.c = call_of(B, heads, L, d, dv, log_decay, lengths, slots, nslots, after != nullptr, p, left_out);
  a.w[0] = dec::Walk{rows_of(Q, L), rows_of(K, L), rows_of(V, L), rows_of(Y, L), H / heads / p.parts, 1, p.parts, d, dv, scale, scale, 1.f, 1, 0, before ? before->S : nullptr,
                     apart ? ends : (after ? after->S : nullptr), dv, 1, apart ? 0 : 1};
  a.prefix[0] = states;
  if (p.nseg > 1) {
    dec::SumSet m{};
    m.c = a.c;
    m.w[0] = a.w[0];
    m.part[0] = states;
    m.last = after != nullptr;
    if (int rc = dec::launch_sums(m, 1, Q->dtype, s)) return rc;
    dec::JoinSet j{};
    j.c = a.c;
    j.part[0] = states;
    j.init[0] = a.w[0].init;
    j.end[0] = a.w[0].end;
    j.end_pool[0] = 1;
    j.count = 1;
    if (int rc = dec::launch_join(j, s)) return rc;
  }
  if (int rc = dec::launch_walks(a, 0, 1, Q->dtype, s)) return rc;
  return apart ? dec::launch_put(a.c, ends, after->S, s) : FS_OK;
}

size_t favorsharp_decay_attention_backward_workspace_bytes(int B, int H, int heads, int L, int d, int dv, int with_dbefore) {
  return sizes(B, H, heads, L, d, dv) == FS_OK ? plan_backward(B, H, heads, L, d, dv, with_dbefore != 0).total : 0;
}

int favorsharp_decay_attention_backward(const fs_tensor* Q, const fs_tensor* K, const fs_tensor* V, const fs_tensor* dY, int B, int H, int heads,
                                        int L, int d, int dv, const float* log_decay, float scale, const fs_decay_state* before,
                                        const fs_decay_state* dafter, const int32_t* slots, const int32_t* lengths, int exclusive,
                                        const fs_tensor* dQ, const fs_tensor* dK, const fs_tensor* dV, const fs_decay_state* dbefore,
                                        void* workspace, size_t workspace_bytes, void* stream) {
  int nslots;
  if (int rc = sizes(B, H, heads, L, d, dv)) return rc;
  if (int rc = pools({before, dafter, dbefore}, heads, &nslots)) return rc;
  if (!numbers_ok(log_decay, scale, slots, lengths) || (uintptr_t)workspace % 16) return FS_ERR_INVALID_ARG;
  if ((exclusive != 0 && exclusive != 1) || (dafter != nullptr && !exclusive) || (exclusive && nslots == 0)) return FS_ERR_INVALID_ARG;
  if (!tensor_ok(Q, d, L > 0) || !tensor_ok(K, d, L > 0) || !tensor_ok(V, dv, L > 0) || !tensor_ok(dY, dv, L > 0)) return FS_ERR_INVALID_ARG;
  if (!tensor_ok(dQ, d, L > 0) || !tensor_ok(dK, d, L > 0) || !tensor_ok(dV, dv, L > 0)) return FS_ERR_INVALID_ARG;
  if (Q->dtype != K->dtype || Q->dtype != V->dtype || Q->dtype != dY->dtype) return FS_ERR_INVALID_ARG;
  if (!strides_ok({Q, K, V, dY, dQ, dK, dV}, L)) return FS_ERR_UNSUPPORTED;
  const Plan p = plan_backward(B, H, heads, L, d, dv, dbefore != nullptr);
  if (p.total > 0 && workspace == nullptr) return FS_ERR_INVALID_ARG;
  if (workspace_bytes < p.total) return FS_ERR_WORKSPACE_TOO_SMALL;
  if (L == 0 && dbefore == nullptr) return FS_OK;
  hipStream_t s = (hipStream_t)stream;
  float *prefix = (float*)workspace, *suffix = (float*)((char*)workspace + p.states), *ends = (float*)((char*)workspace + 2 * p.states);
  // a pool whose slots are the sequences takes their gradients as they are; others their sums
  const bool direct = slots == nullptr && nslots == B;
  const int G = H / heads;
  dec::WalkSet a{};
  a.c = call_of(B, heads, L, d, dv, log_decay, lengths, slots, nslots, exclusive, p, nullptr);
  const float* last = dafter ? dafter->S : nullptr;
  float* end = dbefore == nullptr ? nullptr : (direct ? dbefore->S : ends);
  a.w[0] = dec::Walk{rows_of(dY, L), rows_of(V, L), rows_of(K, L), rows_of(dQ, L), G / p.parts, 1, p.parts, dv, d, scale, scale, 1.f, 1, 0, before ? before->S : nullptr, nullptr, 1, dv, 0};
  a.w[1] = dec::Walk{rows_of(V, L), rows_of(dY, L), rows_of(Q, L), rows_of(dK, L), 1, G, 1, dv, d, scale, 1.f, scale, 0, 1, last, nullptr, 1, dv, 0};
  a.w[2] = dec::Walk{rows_of(K, L), rows_of(Q, L), rows_of(dY, L), rows_of(dV, L), 1, G, 1, d, dv, scale, 1.f, scale, 0, 1, last, end, dv, 1, direct ? 1 : 0};
  a.prefix[0] = prefix;
  a.prefix[1] = a.prefix[2] = suffix;
  if (p.nseg > 1) {
    dec::SumSet m{};
    m.c = a.c;
    m.w[0] = dec::Walk{rows_of(Q, L), rows_of(K, L), rows_of(V, L), rows_of(dY, L), G, 1, 1, d, dv, 1.f, 1.f, 1.f, 1, 0, nullptr, nullptr, dv, 1, 0};
    m.w[1] = a.w[2];
    m.part[0] = prefix;
    m.part[1] = suffix;
    m.last = dbefore != nullptr;
    if (int rc = dec::launch_sums(m, 2, Q->dtype, s)) return rc;
    dec::JoinSet j{};
    j.c = a.c;
    j.part[0] = prefix;
    j.part[1] = suffix;
    j.init[0] = a.w[0].init;
    j.init[1] = last;
    j.end[1] = end;
    j.end_pool[1] = direct ? 1 : 0;
    j.count = 2;
    if (int rc = dec::launch_join(j, s)) return rc;
  }
  // dK and dV in one walk, but fp32 rows of more than 32, whose registers leave a wave to a SIMD, where heads do not share states (B64 H8 L512
  // d64: 192 us in one walk, 163; B2 H8/2 L4096: 89, 115)
  const bool one = std::max(d, dv) <= 64 && (Q->dtype == FS_BF16 || std::max(d, dv) <= 32 || G > 1);
  // dQ by itself where heads share states: the other two have a form of their own then
  const bool alone = one || G > 1;
  if (int rc = dec::launch_walks(a, 0, alone ? 1 : 3, Q->dtype, s)) return rc;
  if (alone)
    if (int rc = one ? dec::launch_back(a, 1, Q->dtype, s) : dec::launch_walks(a, 1, 2, Q->dtype, s)) return rc;
  return dbefore != nullptr && !direct ? dec::launch_slot_sums(a.c, ends, dbefore->S, s) : FS_OK;
}

int favorsharp_decay_step(const fs_decay_state* state, const int32_t* slots, const fs_tensor* Q, const fs_tensor* K, const fs_tensor* V, int B, int H,
                          int heads, int d, int dv, const float* log_decay, float scale, const fs_tensor* Y, int32_t* left_out, void* stream) {
  int nslots;
  if (state == nullptr) return FS_ERR_INVALID_ARG;
  if (int rc = sizes(B, H, heads, 1, d, dv)) return rc;
  if (int rc = pools({state}, heads, &nslots)) return rc;
  if (!numbers_ok(log_decay, scale, slots, nullptr) || (uintptr_t)left_out % 4) return FS_ERR_INVALID_ARG;
  if (!tensor_ok(Q, d) || !tensor_ok(K, d) || !tensor_ok(V, dv) || !tensor_ok(Y, dv)) return FS_ERR_INVALID_ARG;
  if (Q->dtype != K->dtype || Q->dtype != V->dtype) return FS_ERR_INVALID_ARG;
  return dec::launch_step(dec::StepArgs{dev(Q), dev(K), dev(V), dev(Y), state->S, slots, log_decay, nslots, B, H, heads, d, dv, scale, left_out},
                          (hipStream_t)stream);
}

}  // extern "C"
