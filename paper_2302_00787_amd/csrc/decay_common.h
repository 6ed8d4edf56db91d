// Linear attention with a decay for each head: what its kernels and entry points share.
//
// A state S [d][dv] of a sequence and a key head forgets: S_i = lambda S_(i-1) + k_i v_i', y_i = scale q_i S_i, lambda = exp(log decay).
// Over the rows of a call, r = 0 .. n - 1, that is the walk
//   y_r = s_score sum_(r' <= r) lambda^(r - r') (x_r . a_r') b_r' + s_inter lambda^(r + first) x_r S_init,
//   S_end = lambda^n S_init + s_update sum_r' lambda^(n - r' - first) a_r' b_r',
// with x, a, b = q, k, v, first = 1.  The gradients are walks, too: dq with x, a, b = dy, v, k and the transposed state; dk and dv from
// the last row to the first (r counts back) with v, dy, q and k, q, dy, first = 0 and the states D, of which S_end is the gradient of the
// state before the call.
#pragma once
#include "fs_common.h"
#include "state_common.h"

namespace fs {
namespace dec {

constexpr int kChunk = 64;

// A walk over the rows of every state.  G heads of X and Y, or of A and B, share a state (the other side has one).
struct Walk {
  TensorDev X, A, B, Y;
  int GX, GA, parts;             // parts: workgroups that share the G heads of X
  int wa, wb;                    // numbers of a row of X and A, of B and Y
  float s_score, s_inter, s_update;
  int first, back;               // back: row r is the sequence's row n - 1 - r
  // states before the rows: those of the pool `init` (nullptr: empty), or of the workspace where there are segments; element (a, b) at
  // a sa + b sb of one
  const float* init;
  float* end;                    // S_end: of a pool, or [state] (end_pool = 0); nullptr: not wanted
  int sa, sb, end_pool;
};
// What the walks of a call have in common.
struct Call {
  int B, Hk, L;
  const int32_t* lengths;
  const int32_t* slots;
  int nslots, unique;            // unique: a sequence whose slot is an earlier one's is left out
  const float* log_decay;        // [Hk]
  int nseg, seg_rows;            // segments of a sequence, rows of one (a multiple of kChunk)
  int state;                     // numbers of a state
  int* left_out;
};
struct WalkSet {
  Call c;
  Walk w[3];
  float* prefix[3];              // [state][nseg][numbers of a state] states before the segments (nseg > 1)
};
// Sums of the segments into `part` [state][nseg][state numbers], for the walks that they are needed for.
struct SumSet {
  Call c;
  Walk w[2];                     // A, B, GA, wa, wb, s_update, first, back
  float* part[2];
  int last;                      // the last segment is wanted, too
};
// Sums become states before the segments.
struct JoinSet {
  Call c;
  float* part[2];
  const float* init[2];          // pools or nullptr
  float* end[2];                 // of a pool, or [state]; nullptr: not wanted
  int end_pool[2];
  int count;
};
int launch_walks(const WalkSet& a, int from, int count, int dtype, hipStream_t st);
int launch_back(const WalkSet& a, int from, int dtype, hipStream_t st);
int launch_sums(const SumSet& a, int count, int dtype, hipStream_t st);
int launch_join(const JoinSet& a, hipStream_t st);
// States [state] of the sequences that have a slot of their own, into the pool.
int launch_put(const Call& c, const float* each, float* pool, hipStream_t st);
// Pool of gradients: the sums over the sequences that read a slot, in their order (zeros where none does).
int launch_slot_sums(const Call& c, const float* each, float* pool, hipStream_t st);

struct StepArgs {
  TensorDev Q, K, V, Y;
  float* state;
  const int32_t* slots;
  const float* log_decay;
  int nslots, B, H, Hk, d, dv;
  float scale;
  int* left_out;
};
int launch_step(const StepArgs& a, hipStream_t st);

// exp(n log_decay) for a whole number n >= 0; log decays above zero count as zero, those below -10^30 as that (0 times -infinity would be
// none).  The product's rounding error goes into the result (|x| 2^-24 of it otherwise).
struct Exponent { float x, rest; };
__device__ __forceinline__ Exponent exponent(float log_decay, float n) {
  const float g = log_decay > 0.f ? 0.f : fmaxf(log_decay, -1e30f), x = n * g;
  return {log_decay != log_decay ? log_decay : x, fmaf(n, g, -x)};
}
__device__ __forceinline__ float power(float log_decay, int n) {
  const Exponent e = exponent(log_decay, (float)n);
  const float p = expf(e.x);
  return e.x < -104.f ? p : fmaf(p, e.rest, p);
}
// A state's factor lambda^n: as S + S (lambda^n - 1) where it is near one, as that rounds the product alone, and not the factor in the same
// way at every chunk of a long sequence.
struct Keep { float part; bool near; };
__device__ __forceinline__ Keep keep_of(float log_decay, int n) {
  const Exponent e = exponent(log_decay, (float)n);
  if (e.x > -0.69f) {
    const float p = expm1f(e.x);
    return {fmaf(1.f + p, e.rest, p), true};
  }
  return {power(log_decay, n), false};
}
__device__ __forceinline__ float kept(Keep k, float s) { return k.near ? fmaf(s, k.part, s) : s * k.part; }

}  // namespace dec
}  // namespace fs
