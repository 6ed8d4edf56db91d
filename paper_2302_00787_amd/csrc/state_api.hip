// C ABI of rotary positions and of attention through kept states: argument validation, workspace plans, launches.
#include "../../include/favorsharp.h"

#include <algorithm>
#include <cmath>

#include "api_common.h"
#include "state_common.h"

using namespace fs;
using fs::st::FeaturePlan;

namespace {

constexpr int kMaxFeatures = 2048;               // references of a state's partial sums in LDS; features of a token in LDS
constexpr int kMaxRows = 1 << 29;                // rows of one state in a call: they are counted in 32 bits

bool rotary_ok(const fs_rotary* r, int d) {
  return r->freqs != nullptr && r->rot_dim >= 2 && r->rot_dim % 2 == 0 && r->rot_dim <= d && (r->interleaved == 0 || r->interleaved == 1) &&
         r->stride_b >= 0 && r->stride_l >= 0 && std::isfinite(r->amplitude) && (uintptr_t)r->freqs % 8 == 0 && (uintptr_t)r->positions % 4 == 0;
}
st::RotaryDev dev(const fs_rotary* r) {
  if (r == nullptr) return st::RotaryDev{nullptr, nullptr, 0, 0, 0, 0, 1.f};
  return st::RotaryDev{r->freqs, r->positions, r->stride_b, r->stride_l, r->rot_dim, r->interleaved, r->amplitude};
}

// What the entry points on states ask of the constants, the pool and the sizes.
int check(const fs_features* f, const fs_state* s, bool shift, int B, int H, int L, int dv, const fs_rotary* rot) {
  if (f == nullptr || s == nullptr || f->ptr == nullptr) return FS_ERR_INVALID_ARG;
  if (f->heads < 1 || f->d < 1 || f->M < 1 || (f->sets != 1 && f->sets != f->heads) || (f->dense_c2 != 0 && f->dense_c2 != 1)) return FS_ERR_INVALID_ARG;
  if (B < 1 || L < 0 || dv < 1 || H < 1 || H % f->heads) return FS_ERR_INVALID_ARG;
  if (f->d > 128 || dv > 128 || f->M > kMaxFeatures || !sequences_ok(B, H) || (long long)L * (H / f->heads) > kMaxRows) return FS_ERR_UNSUPPORTED;
  if (s->T == nullptr || s->z == nullptr || (shift && s->shift == nullptr) || s->slots < 1) return FS_ERR_INVALID_ARG;
  if ((uintptr_t)s->T % 16 || (uintptr_t)s->z % 4 || (uintptr_t)s->shift % 4) return FS_ERR_INVALID_ARG;
  if (!sequences_ok(s->slots, f->heads)) return FS_ERR_UNSUPPORTED;
  if (f->bytes < st::feature_plan(f->d, f->M, f->sets).total) return FS_ERR_WORKSPACE_TOO_SMALL;
  if (rot != nullptr && !rotary_ok(rot, f->d)) return FS_ERR_INVALID_ARG;
  return FS_OK;
}
st::Features features_of(const fs_features* f) {
  st::Features r;
  r.base = (const char*)f->ptr + 256;
  r.p = st::feature_plan(f->d, f->M, f->sets);
  r.sets = f->sets; r.d = f->d; r.M = f->M;
  r.scale2 = f->qk_scale * f->qk_scale;
  r.dense = f->dense_c2;
  return r;
}
st::State state_of(const fs_state* s) { return st::State{s->T, s->z, s->shift, s->slots}; }

// Sums over `rows` rows of every state (append; gradient of a state): the workgroups that share them, and what a call keeps between its launches.
struct SumPlan {
  int nwg;
  size_t off_table, off_terms, off_weights, off_old, off_parts, off_refs, off_part, off_zpart, total;
};
SumPlan plan_sum(int B, int heads, long long tokens, long long rows, int d, int dv, int M, int rot, bool terms, bool weights, bool sums) {
  SumPlan p;
  const int Mp = (M + 31) / 32 * 32, BH = B * heads;
  const st::BuildShape shape = st::build_shape(d, dv, Mp);
  const int nblock = ceil_div(Mp, shape.features);
  // as many as the chip holds at a time, but a few chunks of 32 rows each at least (a part is a state written and read again, what a chunk or
  // two take; 8 states of 10 chunks, 64 x 256: 21 us in pieces of four, 14 of two, of 20 chunks 18 and 15) and 64 to a state; a workgroup
  // for each state where it has no more chunks than that (15 states of 3 chunks, 32 x 512: 10.7 us, 12.5 in pieces of one), where there
  // are eight states a CU, or more sequences than a wave should count
  const long long each = (rows + 31) / 32, chunks = each * BH, few = st::width_class(d, dv) <= 64 ? 4 : 2,
                  piece = (long long)BH * nblock <= 64 ? 2 : few;
  p.nwg = B > 256 || each <= few || (long long)BH * nblock >= 2048
              ? 0
              : (int)std::max<long long>(1, std::min<long long>({256 * shape.per_cu / nblock, (chunks + piece - 1) / piece, 64ll * BH}));
  size_t off = 0;
  p.off_table = off; off = align_up(off + (size_t)tokens * (rot / 2) * sizeof(float2));
  p.off_terms = off; off = align_up(off + (terms ? (size_t)BH * rows * sizeof(float) : 0));
  p.off_weights = off; off = align_up(off + (weights ? (size_t)BH * rows * sizeof(float) : 0));
  const size_t parts = sums ? (size_t)BH + p.nwg : 0;
  p.off_old = off; off = align_up(off + (sums ? (size_t)BH * sizeof(float) : 0));
  p.off_parts = off; off = align_up(off + (sums ? (size_t)BH * sizeof(int2) : 0));
  p.off_refs = off; off = align_up(off + parts * (Mp / 16) * sizeof(float2));
  p.off_part = off; off = align_up(off + parts * M * dv * sizeof(float));
  p.off_zpart = off; off = align_up(off + parts * M * sizeof(float));
  p.total = off;
  return p;
}
SumPlan plan_append(const fs_features* f, int B, int L, int dv, int rot) {
  return plan_sum(B, f->heads, (long long)B * L, L, f->d, dv, f->M, rot, f->dense_c2 != 0, false, true);
}
SumPlan plan_rows(int B, int L, int rot) { return plan_sum(1, 1, (long long)B * L, 0, 1, 1, 1, rot, false, false, false); }
SumPlan plan_attention_backward(const fs_features* f, int B, int H, int L, int dv, int rot) {
  return plan_sum(B, f->heads, (long long)B * L, (long long)L * (H / f->heads), f->d, dv, f->M, rot, true, true, true);
}
bool sizes_ok(const fs_features* f, int B, int H, int L, int dv, int rot) {
  return f != nullptr && f->heads >= 1 && f->d >= 1 && f->d <= 128 && f->M >= 1 && f->M <= kMaxFeatures && B >= 1 && H >= 1 && H % f->heads == 0 &&
         L >= 0 && dv >= 1 && dv <= 128 && rot >= 0 && rot <= f->d && sequences_ok(B, H) && (long long)L * (H / f->heads) <= kMaxRows;
}

// The table of the angles, where there are any.
int turn_of(const fs_rotary* rot, int B, int L, char* ws, size_t off, st::Turn* turn, hipStream_t stream) {
  if (rot == nullptr) return FS_OK;
  turn->table = (const float2*)(ws + off);
  turn->rot = rot->rot_dim;
  turn->interleaved = rot->interleaved;
  return st::launch_rotary_table(dev(rot), B, L, (float2*)(ws + off), stream);
}

// Rows turned by their positions, of either kind.
int turn_rows(const st::RotaryDev& r, const st::AxesDev& axes, const fs_tensor* X, int H, const fs_tensor* X2, int H2, int B, int L, int d, int transposed,
              const fs_tensor* Y, const fs_tensor* Y2, hipStream_t stream) {
  if (B < 1 || L < 0 || d < 1 || H < 1 || H2 < 0 || (transposed != 0 && transposed != 1)) return FS_ERR_INVALID_ARG;
  if (!tensor_ok(X, d, L > 0) || !tensor_ok(Y, d, L > 0)) return FS_ERR_INVALID_ARG;
  if (H2 > 0 && (!tensor_ok(X2, d, L > 0) || !tensor_ok(Y2, d, L > 0))) return FS_ERR_INVALID_ARG;
  if (d > 1024 || (long long)H + H2 > 65535 || (long long)B * L > (1ll << 31)) return FS_ERR_UNSUPPORTED;
  // in place: the same rows, or none of them
  auto same = [](const fs_tensor* a, const fs_tensor* b) {
    return a->ptr != b->ptr || (a->dtype == b->dtype && a->stride_b == b->stride_b && a->stride_h == b->stride_h && a->stride_l == b->stride_l);
  };
  if (!same(X, Y) || (H2 > 0 && !same(X2, Y2))) return FS_ERR_INVALID_ARG;
  if (L == 0) return FS_OK;
  const TensorDev none{nullptr, 0, 0, 0, 0};
  return st::launch_rotary(r, axes, fs::dev(X), H, H2 ? fs::dev(X2) : none, H2, B, L, d, transposed, fs::dev(Y), H2 ? fs::dev(Y2) : none, stream);
}

}  // namespace

extern "C" {

// ------------------------------------------------------------------------------------------ rotary positions
int favorsharp_rotary_frequencies(int rot_dim, double base, int scaling, double factor, int original_length, double low_turns, double high_turns,
                                  double* host_freqs) {
  if (host_freqs == nullptr || rot_dim < 2 || rot_dim % 2 || !(base > 1.0) || !std::isfinite(base)) return FS_ERR_INVALID_ARG;
  if (scaling < FS_ROTARY_PLAIN || scaling > FS_ROTARY_BLEND) return FS_ERR_INVALID_ARG;
  if (scaling != FS_ROTARY_PLAIN && (!(factor > 0.0) || !std::isfinite(factor))) return FS_ERR_INVALID_ARG;
  if (scaling == FS_ROTARY_BLEND && (original_length < 1 || !(low_turns > 0.0) || !(high_turns > low_turns) || !std::isfinite(high_turns)))
    return FS_ERR_INVALID_ARG;
  if (scaling == FS_ROTARY_BASE && rot_dim > 2) base *= std::pow(factor, rot_dim / (rot_dim - 2.0));
  for (int i = 0; i < rot_dim / 2; ++i) {
    double f = std::pow(base, -2.0 * i / rot_dim);
    if (scaling == FS_ROTARY_LINEAR) f /= factor;
    if (scaling == FS_ROTARY_BLEND) {
      const double turns = original_length * f / 6.283185307179586477;
      const double keep = std::min(1.0, std::max(0.0, (turns - low_turns) / (high_turns - low_turns)));
      f = f * keep + f / factor * (1.0 - keep);
    }
    host_freqs[i] = f;
  }
  return FS_OK;
}

int favorsharp_rotary(const fs_rotary* rot, const fs_tensor* X, int H, const fs_tensor* X2, int H2, int B, int L, int d, int transposed,
                      const fs_tensor* Y, const fs_tensor* Y2, void* stream) {
  if (rot == nullptr || d < 1 || !rotary_ok(rot, d)) return FS_ERR_INVALID_ARG;
  return turn_rows(dev(rot), st::AxesDev{}, X, H, X2, H2, B, L, d, transposed, Y, Y2, (hipStream_t)stream);
}

int favorsharp_rotary_sections(int axes, const int32_t* host_pairs, double base, int order, int whole, double* host_freqs, int32_t* host_axis_of) {
  if (axes < 1 || axes > FS_ROTARY_MAX_AXES || host_pairs == nullptr || host_freqs == nullptr || host_axis_of == nullptr || !(base > 1.0) ||
      !std::isfinite(base) || (order != FS_AXES_BLOCKS && order != FS_AXES_CYCLIC) || (whole != 0 && whole != 1))
    return FS_ERR_INVALID_ARG;
  int pairs = 0, used[FS_ROTARY_MAX_AXES] = {};
  for (int a = 0; a < axes; ++a) {
    if (host_pairs[a] < 0 || host_pairs[a] > 512) return FS_ERR_INVALID_ARG;       // rows of up to 1024 numbers
    pairs += host_pairs[a];
  }
  if (pairs < 1 || pairs > 512) return FS_ERR_INVALID_ARG;
  for (int p = 0, a = order == FS_AXES_BLOCKS ? 0 : axes - 1; p < pairs; ++p) {
    if (order == FS_AXES_CYCLIC) a = (a + 1) % axes;
    while (used[a] == host_pairs[a]) a = (a + 1) % axes;
    host_axis_of[p] = a;
    host_freqs[p] = std::pow(base, whole ? -(double)p / pairs : -(double)used[a] / host_pairs[a]);
    ++used[a];
  }
  return FS_OK;
}

int favorsharp_rotary_axes(const fs_rotary_axes* rot, const fs_tensor* X, int H, const fs_tensor* X2, int H2, int B, int L, int d, int transposed,
                           const fs_tensor* Y, const fs_tensor* Y2, void* stream) {
  if (rot == nullptr || d < 1) return FS_ERR_INVALID_ARG;
  const fs_rotary r{rot->freqs, rot->positions, rot->stride_b, rot->stride_l, rot->rot_dim, rot->interleaved, rot->amplitude};
  if (!rotary_ok(&r, d) || rot->positions == nullptr || rot->stride_a < 0 || rot->axis_of == nullptr || (uintptr_t)rot->axis_of % 4 || rot->axes < 1 ||
      rot->axes > FS_ROTARY_MAX_AXES)
    return FS_ERR_INVALID_ARG;
  const st::AxesDev axes{rot->axis_of, rot->positions, rot->stride_a, rot->stride_b, rot->stride_l, rot->axes};
  return turn_rows(dev(&r), axes, X, H, X2, H2, B, L, d, transposed, Y, Y2, (hipStream_t)stream);
}

// ------------------------------------------------------------------------------------------ states
size_t favorsharp_state_features_bytes(int heads, int d, int M, int groups, int omega_groups) {
  if (heads < 1 || d < 1 || d > 128 || M < 1 || M > kMaxFeatures) return 0;
  if ((groups != 1 && groups != heads) || (omega_groups != 1 && omega_groups != heads)) return 0;
  return st::feature_plan(d, M, std::max(groups, omega_groups)).total;
}

int favorsharp_state_prepare(const float* theta, int groups, const float* Omega, int omega_groups, int heads, int d, int M, float qk_scale,
                             fs_features* host_features, void* stream) {
  if (host_features == nullptr || host_features->ptr == nullptr || theta == nullptr || Omega == nullptr || !(qk_scale > 0.f)) return FS_ERR_INVALID_ARG;
  if (heads < 1 || d < 1 || M < 1 || (groups != 1 && groups != heads) || (omega_groups != 1 && omega_groups != heads)) return FS_ERR_INVALID_ARG;
  if ((uintptr_t)host_features->ptr % 16) return FS_ERR_INVALID_ARG;
  const size_t need = favorsharp_state_features_bytes(heads, d, M, groups, omega_groups);
  if (need == 0 || !sequences_ok(1, heads)) return FS_ERR_UNSUPPORTED;
  if (host_features->bytes < need) return FS_ERR_WORKSPACE_TOO_SMALL;
  hipStream_t s = (hipStream_t)stream;
  const int sets = std::max(groups, omega_groups);
  if (int rc = st::launch_prepare(theta, groups, Omega, omega_groups, sets, d, M, qk_scale, (char*)host_features->ptr,
                                  st::feature_plan(d, M, sets), s))
    return rc;
  unsigned dense = 0;
  if (hipMemcpyAsync(&dense, host_features->ptr, sizeof(dense), hipMemcpyDeviceToHost, s) != hipSuccess) return FS_ERR_DEVICE;
  if (hipStreamSynchronize(s) != hipSuccess) return FS_ERR_DEVICE;
  host_features->heads = heads;
  host_features->d = d;
  host_features->M = M;
  host_features->sets = sets;
  host_features->dense_c2 = (int32_t)(dense & 1);
  host_features->qk_scale = qk_scale;
  return FS_OK;
}

size_t favorsharp_state_append_workspace_bytes(const fs_features* f, int B, int L, int dv, int rot_dim) {
  if (!sizes_ok(f, B, f ? f->heads : 0, L, dv, rot_dim)) return 0;
  return plan_append(f, B, L, dv, rot_dim).total;
}

int favorsharp_state_append(const fs_features* f, const fs_state* state, const int32_t* slots, const fs_tensor* K, const fs_tensor* V, int B, int L,
                            int dv, const int32_t* lengths, const fs_rotary* rot, int fresh, int32_t* left_out, void* workspace,
                            size_t workspace_bytes, void* stream) {
  if (int rc = check(f, state, true, B, f ? f->heads : 0, L, dv, rot)) return rc;
  if (fresh != 0 && fresh != 1) return FS_ERR_INVALID_ARG;
  if (!tensor_ok(K, f->d, L > 0) || !tensor_ok(V, dv, L > 0) || K->dtype != V->dtype || workspace == nullptr || (uintptr_t)workspace % 16) return FS_ERR_INVALID_ARG;
  const SumPlan p = plan_append(f, B, L, dv, rot ? rot->rot_dim : 0);
  if (workspace_bytes < p.total) return FS_ERR_WORKSPACE_TOO_SMALL;
  hipStream_t s = (hipStream_t)stream;
  char* ws = (char*)workspace;
  st::BuildArgs a{};
  a.f = features_of(f);
  a.side = 1;
  a.x = st::Rows{dev(K), L, 1, lengths, f->d, st::Turn{}};
  a.v = st::Rows{dev(V), L, 1, lengths, dv, st::Turn{}};
  a.slots = slots; a.nslots = state->slots;
  a.B = B; a.Hk = f->heads; a.dv = dv;
  a.nwg = p.nwg; a.parts = (int2*)(ws + p.off_parts);
  a.part = (float*)(ws + p.off_part); a.zpart = (float*)(ws + p.off_zpart); a.refs = (float2*)(ws + p.off_refs);
  if (!fresh) { a.shift = state->shift; a.old_shift = (float*)(ws + p.off_old); }
  if (L > 0) {
    if (int rc = turn_of(rot, B, L, ws, p.off_table, &a.x.turn, s)) return rc;
    if (f->dense_c2) {
      a.terms = (float*)(ws + p.off_terms);
      if (int rc = st::launch_row_terms(a.f, a.x, B, f->heads, (float*)(ws + p.off_terms), s)) return rc;
    }
  }
  if (int rc = st::launch_build(a, s)) return rc;
  st::JoinArgs j{a.part, a.zpart, a.refs, a.old_shift, slots, state_of(state), a.parts, B, f->heads, f->M, a.f.p.Mp, dv, left_out};
  return st::launch_join(j, s);
}

size_t favorsharp_state_attention_workspace_bytes(const fs_features* f, int B, int H, int L, int dv, int rot_dim) {
  if (!sizes_ok(f, B, H, L, dv, rot_dim)) return 0;
  return plan_rows(B, L, rot_dim).total;
}

int favorsharp_state_attention(const fs_features* f, const fs_state* state, const int32_t* slots, const fs_tensor* Q, int B, int H, int L, int dv,
                               const int32_t* lengths, const fs_rotary* rot, const fs_tensor* Y, int32_t* unread, void* workspace,
                               size_t workspace_bytes, void* stream) {
  if (int rc = check(f, state, true, B, H, L, dv, rot)) return rc;
  if (!tensor_ok(Q, f->d, L > 0) || !tensor_ok(Y, dv, L > 0) || (uintptr_t)workspace % 16) return FS_ERR_INVALID_ARG;
  const SumPlan p = plan_rows(B, L, rot ? rot->rot_dim : 0);
  if (p.total > 0 && workspace == nullptr) return FS_ERR_INVALID_ARG;
  if (workspace_bytes < p.total) return FS_ERR_WORKSPACE_TOO_SMALL;
  if (L == 0) return FS_OK;
  hipStream_t s = (hipStream_t)stream;
  st::ValueArgs a{};
  a.f = features_of(f);
  a.x = st::Rows{dev(Q), L, H / f->heads, lengths, f->d, st::Turn{}};
  if (int rc = turn_of(rot, B, L, (char*)workspace, p.off_table, &a.x.turn, s)) return rc;
  a.slots = slots;
  a.state = state_of(state);
  a.B = B; a.Hk = f->heads; a.dv = dv;
  a.Y = dev(Y);
  a.unread = unread;
  return st::launch_values(a, s);
}

size_t favorsharp_state_step_workspace_bytes(const fs_features* f, int B, int H) {
  if (!sizes_ok(f, B, H, 1, 1, 0)) return 0;
  return align_up(st::step_floats(B, H, f->heads, f->d, st::feature_plan(f->d, f->M, 1).Mp) * sizeof(float));
}

int favorsharp_state_step(const fs_features* f, const fs_state* state, const int32_t* slots, const fs_tensor* Q, const fs_tensor* K,
                          const fs_tensor* V, int B, int H, int dv, const fs_rotary* rot, const fs_tensor* Y, int32_t* unread,
                          void* workspace, size_t workspace_bytes, void* stream) {
  if (int rc = check(f, state, true, B, H, 1, dv, rot)) return rc;
  if (!tensor_ok(Q, f->d) || !tensor_ok(K, f->d) || !tensor_ok(V, dv) || !tensor_ok(Y, dv)) return FS_ERR_INVALID_ARG;
  if (Q->dtype != K->dtype || Q->dtype != V->dtype || (uintptr_t)workspace % 16) return FS_ERR_INVALID_ARG;
  const size_t need = favorsharp_state_step_workspace_bytes(f, B, H);
  if (need > 0 && workspace == nullptr) return FS_ERR_INVALID_ARG;
  if (workspace_bytes < need) return FS_ERR_WORKSPACE_TOO_SMALL;
  st::StepArgs a{};
  a.f = features_of(f);
  a.state = state_of(state);
  a.slots = slots;
  a.Q = dev(Q); a.K = dev(K); a.V = dev(V); a.Y = dev(Y);
  a.B = B; a.H = H; a.Hk = f->heads; a.dv = dv;
  a.rot = dev(rot);
  a.unread = unread;
  return st::launch_step(a, (float*)workspace, (hipStream_t)stream);
}

size_t favorsharp_state_attention_backward_workspace_bytes(const fs_features* f, int B, int H, int L, int dv, int rot_dim) {
  if (!sizes_ok(f, B, H, L, dv, rot_dim)) return 0;
  return plan_attention_backward(f, B, H, L, dv, rot_dim).total;
}

int favorsharp_state_attention_backward(const fs_features* f, const fs_state* state, const int32_t* slots, const fs_tensor* Q, const fs_tensor* dY,
                                        int B, int H, int L, int dv, const int32_t* lengths, const fs_rotary* rot, const fs_tensor* dQ,
                                        const fs_state* dstate, void* workspace, size_t workspace_bytes, void* stream) {
  if (int rc = check(f, state, true, B, H, L, dv, rot)) return rc;
  if (int rc = check(f, dstate, false, B, H, L, dv, rot)) return rc;
  if (dstate->slots != state->slots) return FS_ERR_INVALID_ARG;
  if (!tensor_ok(Q, f->d, L > 0) || !tensor_ok(dY, dv, L > 0) || !tensor_ok(dQ, f->d, L > 0) || workspace == nullptr || (uintptr_t)workspace % 16)
    return FS_ERR_INVALID_ARG;
  const SumPlan p = plan_attention_backward(f, B, H, L, dv, rot ? rot->rot_dim : 0);
  if (workspace_bytes < p.total) return FS_ERR_WORKSPACE_TOO_SMALL;
  hipStream_t s = (hipStream_t)stream;
  char* ws = (char*)workspace;
  const int G = H / f->heads;
  // the rows' gradients with their normalisers and dY . Y, then the states'
  st::GradArgs g{};
  g.f = features_of(f);
  g.x = st::Rows{dev(Q), L, G, lengths, f->d, st::Turn{}};
  g.r = st::Rows{dev(dY), L, G, lengths, dv, st::Turn{}};
  g.lse = (float*)(ws + p.off_terms);
  g.weights = (float*)(ws + p.off_weights);
  g.slots = slots;
  g.state = state_of(state);
  g.B = B; g.Hk = f->heads; g.dv = dv;
  g.dx = dev(dQ);
  if (L > 0) {
    if (int rc = turn_of(rot, B, L, ws, p.off_table, &g.x.turn, s)) return rc;
    if (int rc = st::launch_query_grads(g, s)) return rc;
  }
  st::BuildArgs a{};
  a.f = g.f;
  a.side = 0;
  a.x = g.x;
  a.v = g.r;
  a.terms = g.lse; a.weights = g.weights;
  a.slots = slots; a.nslots = state->slots;
  a.B = B; a.Hk = f->heads; a.dv = dv;
  a.nwg = p.nwg; a.parts = (int2*)(ws + p.off_parts);
  a.part = (float*)(ws + p.off_part); a.zpart = (float*)(ws + p.off_zpart); a.refs = (float2*)(ws + p.off_refs);
  if (int rc = st::launch_build(a, s)) return rc;
  st::JoinArgs j{a.part, a.zpart, a.refs, nullptr, slots, state_of(dstate), a.parts, B, f->heads, f->M, a.f.p.Mp, dv, nullptr};
  return st::launch_join_sum(j, s);
}

size_t favorsharp_state_append_backward_workspace_bytes(const fs_features* f, int B, int L, int dv, int rot_dim) {
  if (!sizes_ok(f, B, f ? f->heads : 0, L, dv, rot_dim)) return 0;
  return plan_rows(B, L, rot_dim).total;
}

int favorsharp_state_append_backward(const fs_features* f, const fs_state* state, const int32_t* slots, const fs_state* dstate, const fs_tensor* K,
                                     const fs_tensor* V, int B, int L, int dv, const int32_t* lengths, const fs_rotary* rot, const fs_tensor* dK,
                                     const fs_tensor* dV, void* workspace, size_t workspace_bytes, void* stream) {
  if (int rc = check(f, state, true, B, f ? f->heads : 0, L, dv, rot)) return rc;
  if (int rc = check(f, dstate, false, B, f->heads, L, dv, rot)) return rc;
  if (dstate->slots != state->slots) return FS_ERR_INVALID_ARG;
  if (!tensor_ok(K, f->d, L > 0) || !tensor_ok(V, dv, L > 0) || !tensor_ok(dK, f->d, L > 0) || !tensor_ok(dV, dv, L > 0) || K->dtype != V->dtype ||
      (uintptr_t)workspace % 16)
    return FS_ERR_INVALID_ARG;
  const SumPlan p = plan_rows(B, L, rot ? rot->rot_dim : 0);
  if (p.total > 0 && workspace == nullptr) return FS_ERR_INVALID_ARG;
  if (workspace_bytes < p.total) return FS_ERR_WORKSPACE_TOO_SMALL;
  if (L == 0) return FS_OK;
  hipStream_t s = (hipStream_t)stream;
  char* ws = (char*)workspace;
  st::GradArgs g{};
  g.f = features_of(f);
  g.x = st::Rows{dev(K), L, 1, lengths, f->d, st::Turn{}};
  g.r = st::Rows{dev(V), L, 1, lengths, dv, st::Turn{}};
  if (int rc = turn_of(rot, B, L, ws, p.off_table, &g.x.turn, s)) return rc;
  g.shift = state->shift;
  g.slots = slots;
  g.state = state_of(dstate);
  g.B = B; g.Hk = f->heads; g.dv = dv;
  g.dx = dev(dK);
  g.dr = dev(dV);
  return st::launch_key_grads(g, s);
}

}  // extern "C"
