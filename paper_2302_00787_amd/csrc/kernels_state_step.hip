// The next token of every sequence: its key and value onto the state, then its queries against it.
//
// The states are read once and written once (2 M (dv + 1) numbers of 4 bytes a key head), which bounds the call.  A launch of its own makes the
// exponents first, sixteen rows of a head at a time on the matrix instructions as in the other kernels, so that W is read once for sixteen
// rows and not once for each state, whose size it has; it also keeps the states' z and shift as they were, so that the second launch can
// cut a state into columns for as many workgroups as fill the chip.  Few small states (at most 256, as many as CUs, one query head to a
// key head, W of 256 features of 64 numbers, 32 features a wave): one launch (ONE), a state a workgroup, W from L2.  (Kernels' us, one launch /
// two: 8 states of 256 x 64 10.5 / 14.3, 248 of them 13.1 / 18.6; where the rule ends: 8 of 512 x 128 19.4 / 18.0, 8 of 1024 x 64 19.5 / 19.6,
// 128 of those 30.1 / 28.0, 180 of 512 x 128 with four query heads 49.8 / 38.5.  Two launches: 2048 of 256 x 64 55.)
#include <algorithm>

#include "state_common.h"

namespace fs {
namespace st {
namespace {

// W of 32 features and a row of LDS (zeros behind its end) as operands.
template <int S> struct StepWeights {
  f16x8 p[S][2][2];              // [step][piece][tile]
  __device__ __forceinline__ void load(const char* img, int fb, int steps, int lane) {
    const uint16_t* at = (const uint16_t*)img + (size_t)fb * steps * 2048 + lane * 8;
#pragma unroll
    for (int s = 0; s < S; ++s)
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int ft = 0; ft < 2; ++ft) p[s][i][ft] = *(const f16x8*)(at + (min(s, steps - 1) * 2 + i) * 1024 + ft * 512);
  }
};
template <int S> struct StepRow {
  Op16<2> x[S];
  float undo, norm;              // norm: |x|^2
  __device__ __forceinline__ void load(const float* row, int lane) {
    f32x8 n[S];
    float most = 0.f;
    norm = 0.f;
#pragma unroll
    for (int s = 0; s < S; ++s) {
      const f32x4 a = *(const f32x4*)(row + 32 * s + 8 * (lane >> 4)), b = *(const f32x4*)(row + 32 * s + 8 * (lane >> 4) + 4);
      n[s] = f32x8{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
      most = fmaxf(most, largest_of(n[s]));
#pragma unroll
      for (int i = 0; i < 8; ++i) norm += n[s][i] * n[s][i];
    }
    most = fmaxf(most, __shfl_xor(most, 16));
    most = fmaxf(most, __shfl_xor(most, 32));
    norm += __shfl_xor(norm, 16);
    norm += __shfl_xor(norm, 32);
    const float scale = up_to_2_14(most);
    undo = power_inverse(scale);
#pragma unroll
    for (int s = 0; s < S; ++s) x[s] = as_op16<2>(n[s] * scale);
  }
  // of 32 features to `to`, of which this lane writes its column's where `mine`
  __device__ __forceinline__ void exponents(const StepWeights<S>& w, float scale, const float* bias, float* to, bool mine, int lane) const {
    f32x4 E[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
    for (int s = 0; s < S; ++s)
      each_product<2, 2>([&](int i, int j) {
#pragma unroll
        for (int ft = 0; ft < 2; ++ft) E[ft] = mfma(w.p[s][i][ft], x[s].p[j], E[ft]);
      });
    if (mine)
#pragma unroll
      for (int ft = 0; ft < 2; ++ft) {
        const int m = 16 * ft + 4 * (lane >> 4);
        *(f32x4*)(to + m) = E[ft] * (undo * scale) + *(const f32x4*)(bias + m);
      }
  }
};

// x' (C2 + C2') x / 2 of the rows' keys, coordinates of sixteen w, w + of, ... (y: the row that this lane has in the operands).
template <int S>
__device__ __forceinline__ float form_of(const StepRow<S>& row, const Features& f, const char* set, const float* y, int w, int of, int lane) {
  float sum = 0.f;
  const int steps = f.p.steps;
#pragma unroll 1
  for (int ct = w; ct < 2 * steps; ct += of) {
    f32x4 q = {0.f, 0.f, 0.f, 0.f};
    const uint16_t* img = (const uint16_t*)(set + f.p.off_csym) + (size_t)ct * steps * 1024 + lane * 8;
#pragma unroll
    for (int s = 0; s < S; ++s) {                // (behind d the row is zeros)
      const uint16_t* from = img + min(s, steps - 1) * 1024;
      const f16x8 p[2] = {*(const f16x8*)from, *(const f16x8*)(from + 512)};
      each_product<2, 2>([&](int i, int j) { q = mfma(p[i], row.x[s].p[j], q); });
    }
    const f32x4 k = *(const f32x4*)(y + 16 * ct + 4 * (lane >> 4));
#pragma unroll
    for (int r = 0; r < 4; ++r) sum += q[r] * k[r];
  }
  sum += __shfl_xor(sum, 16);
  sum += __shfl_xor(sum, 32);
  return sum * (0.5f * kLog2e * f.scale2 * row.undo * *(const float*)(set + f.p.off_cscale));
}

// ---------------------------------------------------------------------------------------------- exponents
// Tiles of sixteen rows: keys of sequences (first a.key_tiles of them), then queries, row v = query head v % G of sequence v / G.  Workgroups x have
// 128 features each; where quadratic forms are dense, one more makes the keys' row terms meanwhile, its waves sixteen coordinates at a time.
template <int S>
__global__ void __launch_bounds__(256) k_step_exponents(StepArgs a) {
  __shared__ __align__(16) float x[16][132];
  __shared__ int position[16];
  __shared__ float parts[4][16];
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), g = lane >> 4, c = lane & 15;
  const int h = blockIdx.y, G = a.H / a.Hk, fb = blockIdx.x * 4 + w, Mp = a.f.p.Mp, nfb = Mp / 32, steps = a.f.p.steps, M = a.f.M;
  const bool keys = (int)blockIdx.z < a.key_tiles, form = a.f.dense && blockIdx.x == gridDim.x - 1;
  if (form && !keys) return;
  const int per = keys ? 1 : G, rows = a.B * per, v0 = 16 * (keys ? blockIdx.z : blockIdx.z - a.key_tiles);
  const char* set = a.f.set(h);
  StepWeights<S> weights;
  if (fb < nfb) weights.load(set + a.f.p.off_row[keys], fb, steps, lane);
  // the rows' numbers: a thread has a column of every other row, all on their way together
  const TensorDev& X = keys ? a.K : a.Q;
  const int col = tid & 127, at_col = min(col, a.f.d - 1);
  long long at[8];
  uint32_t bits[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int r = min(v0 + 2 * i + (tid >> 7), rows - 1);
    at[i] = row_base(X, r / per, keys ? h : h * G + r % per, 0) + at_col;
  }
  if (X.dtype == 0) {
#pragma unroll
    for (int i = 0; i < 8; ++i) bits[i] = ((const uint32_t*)X.ptr)[at[i]];
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) bits[i] = (uint32_t)((const uint16_t*)X.ptr)[at[i]] << 16;
  }
  const int v = v0 + c, vc = min(v, rows - 1), b = vc / per;
  if (tid < 16 && a.rot.rot > 0) position[tid] = position_of(a.rot, b, 0);
#pragma unroll
  for (int i = 0; i < 8; ++i) x[2 * i + (tid >> 7)][col] = col < a.f.d ? __uint_as_float(bits[i]) : 0.f;
  __syncthreads();
  const int pairs = a.rot.rot >> 1;
#pragma unroll 1
  for (int e = tid; e < 16 * pairs; e += 256) {
    const int r = e / pairs, i = e - r * pairs, i0 = a.rot.interleaved ? 2 * i : i, i1 = a.rot.interleaved ? 2 * i + 1 : i + pairs;
    const float2 cs = cos_sin(position[r], a.rot.freqs[i], a.rot.amplitude);
    const float p = x[r][i0], q = x[r][i1];
    x[r][i0] = p * cs.x - q * cs.y;
    x[r][i1] = q * cs.x + p * cs.y;
  }
  __syncthreads();
  StepRow<S> row;
  row.load(&x[c][0], lane);
  const int slot = slot_of(a.slots, a.state.slots, b);
  const float shift = keys && v < rows && slot >= 0 ? a.state.shift[(size_t)slot * a.Hk + h] : kNone;
  if (form) {
    parts[w][c] = form_of(row, a.f, set, &x[c][0], w, 4, lane);
    __syncthreads();
    if (w > 0 || g > 0 || v >= rows) return;
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) sum += parts[i][c];
    a.old_shift[b * a.Hk + h] = make_float2(shift, sum);
    return;
  }
  if (fb >= nfb) return;
  row.exponents(weights, ((const float*)(set + a.f.p.off_scale[keys]))[fb], (const float*)(set + a.f.p.off_bias) + 32 * fb,
                a.exps + ((size_t)(b * a.Hk + h) * (1 + G) + (keys ? 0 : 1 + vc % per)) * Mp + 32 * fb, v < rows, lane);
  if (!keys) return;
  // the sequences' z of these features as they are, and once their shift and the keys' row terms
  if (v < rows && slot >= 0) {
    const float* z = a.state.z + ((size_t)slot * a.Hk + h) * M;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int m = 32 * fb + 8 * g + i;
      if (m < M) a.old_z[(size_t)(b * a.Hk + h) * Mp + m] = z[m];
    }
  }
  if (fb == 0 && !a.f.dense && v < rows && g == 0) a.old_shift[b * a.Hk + h] = make_float2(shift, -0.5f * kLog2e * a.f.scale2 * row.norm);
}

// ---------------------------------------------------------------------------------------------- states
// Floats in LDS: features (key, GC queries), z, the threads' partial outputs, maxima and normalisers by wave.
template <int GC, int NTH> __host__ __device__ constexpr int step_lds_floats(int Mp) {
  return (GC + 2) * Mp + 4 * GC * NTH + (1 + GC) * 2 * (NTH / 64) + (GC + 1) * 128 + NTH / 64;
}

// GC: query heads that a pass over the state serves.  Workgroup z has the columns z cols .. (z + 1) cols - 1.
template <int S, int VEC, int GC, int NTH, bool ONE>
__global__ void __launch_bounds__(NTH, ONE ? 2 : 4) k_step(StepArgs a) {
  typedef __attribute__((ext_vector_type(VEC))) float vec;
  constexpr int NW = NTH / 64, AHEAD = GC == 1 ? 8 : 4;   // fours of the state on their way for each thread
  extern __shared__ __align__(16) float lds[];
  const int Mp = a.f.p.Mp, M = a.f.M, dv = a.dv, tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  float* feat = lds;                           // [GC + 1][Mp]
  float* zs = feat + (GC + 1) * Mp;            // [Mp]
  float* part = zs + Mp;                       // [GC][rows of a pass][columns]
  float* tops = part + 4 * GC * NTH;           // [GC + 1][NW]
  float* dens = tops + (1 + GC) * NW;          // [GC][NW]
  float* x = dens + (1 + GC) * NW;             // (ONE) [2][128] the key, the query
  float* word = x + (GC + 1) * 128;            // (ONE) the key's row term by wave
  const int b = blockIdx.x, h = blockIdx.y, G = GC == 1 ? 1 : a.H / a.Hk, col0 = blockIdx.z * a.cols, cols = min(a.cols, dv - col0);
  const int slot = unique_slot_of(a.slots, a.state.slots, b);
  if (slot < 0) {
    for (int e = tid; e < G * cols; e += NTH) store_elem(a.Y, row_base(a.Y, b, h * G + e / cols, 0) + col0 + e % cols, 0.f);
    if (tid == 0 && blockIdx.z == 0 && a.unread != nullptr) atomicAdd(a.unread, G);
    return;
  }
  const size_t at = (size_t)slot * a.Hk + h, bh = (size_t)b * a.Hk + h;
  const int quads = (cols + VEC - 1) / VEC, pass = NTH / quads, q0 = tid % quads, r0 = tid / quads;       // rows of a pass over the state
  const bool worker = r0 < pass;
  const int mine = worker ? (M - r0 + pass - 1) / pass : 0, step = pass * (dv / VEC);                      // rows r0, r0 + pass, ...: `mine` of them
  vec* T = (vec*)(a.state.T + at * M * dv + col0) + (worker ? r0 * (dv / VEC) + q0 : 0);
  vec t[AHEAD];
#pragma unroll
  for (int i = 0; i < AHEAD; ++i)
    if (i < mine) t[i] = T[(size_t)i * step];
  float2 before;                               // shift, the key's row term
  const char* set = a.f.set(h);
  const int steps = a.f.p.steps, nfb = Mp / 32, pairs = a.rot.rot >> 1;
  StepWeights<S> weights[2];     // (ONE) the queries', the key's
  if constexpr (ONE) {
    before = make_float2(a.state.shift[at], 0.f);
    if (w < nfb)
#pragma unroll
      for (int i = 0; i < 2; ++i) weights[i].load(set + a.f.p.off_row[i], w, steps, lane);
  } else {
    before = a.old_shift[bh];
  }
  vec v;
#pragma unroll
  for (int i = 0; i < VEC; ++i) v[i] = worker ? load_elem(a.V, row_base(a.V, b, h, 0) + col0 + VEC * q0 + i) : 0.f;
  const float* exps = ONE ? nullptr : a.exps + bh * (1 + G) * Mp;
  const float* old_z = ONE ? a.state.z + at * M : a.old_z + bh * Mp;
  float keep = 0.f;
  int unread = 0;
  for (int g0 = 0; g0 < G; g0 += GC) {
    const int n = GC == 1 ? 1 : min(GC, G - g0);
    if (g0 > 0) __syncthreads();
    if constexpr (ONE) {
      // rows: a thread a number, of a turned pair both
      for (int e = tid; e < 256; e += NTH) {
        const int r = e >> 7, c = e & 127;
        const TensorDev& src = r == 0 ? a.K : a.Q;
        const long long base = row_base(src, b, h, 0);
        float* to = x + r * 128;
        if (c < pairs) {
          const int i0 = a.rot.interleaved ? 2 * c : c, i1 = a.rot.interleaved ? 2 * c + 1 : c + pairs;
          const float u = load_elem(src, base + i0), q = load_elem(src, base + i1);
          const float2 cs = cos_sin(position_of(a.rot, b, 0), a.rot.freqs[c], a.rot.amplitude);
          to[i0] = u * cs.x - q * cs.y;
          to[i1] = q * cs.x + u * cs.y;
        }
        if (c >= 2 * pairs) to[c] = c < a.f.d ? load_elem(src, base + c) : 0.f;
      }
      __syncthreads();
      // exponents: the same row in every column of the operands
      const float* bias = (const float*)(set + a.f.p.off_bias) + 32 * w;
      StepRow<S> row;
      row.load(x, lane);
      if (w < nfb) row.exponents(weights[1], ((const float*)(set + a.f.p.off_scale[1]))[w], bias, feat + 32 * w, (lane & 15) == 0, lane);
      const float term = a.f.dense ? form_of(row, a.f, set, x, w, NW, lane) : w == 0 ? -0.5f * kLog2e * a.f.scale2 * row.norm : 0.f;
      if (lane == 0) word[w] = term;
      row.load(x + 128, lane);
      if (w < nfb) row.exponents(weights[0], ((const float*)(set + a.f.p.off_scale[0]))[w], bias, feat + Mp + 32 * w, (lane & 15) == 0, lane);
      __syncthreads();
      before.y = 0.f;
#pragma unroll
      for (int i = 0; i < NW; ++i) before.y += word[i];
    }
    // features: a thread has the same ones of all rows; the key's again with every pass
    float top = kNone;
    bool no_number = before.x != before.x;       // (maxima pass over what is not a number)
    for (int m = tid; m < Mp; m += NTH) {
      const float e = (ONE ? feat[m] : exps[m]) + before.y;
      feat[m] = e;
      top = fmaxf(top, e);
      no_number |= e != e;
      if constexpr (!ONE)
#pragma unroll
        for (int j = 1; j <= GC; ++j)
          if (j <= n) feat[j * Mp + m] = exps[(size_t)(g0 + j) * Mp + m];
    }
    auto largest = [](float v) {
      v = over_lanes<32>(v, [](float p, float q) { return fmaxf(p, q); });
      return fmaxf(v, __shfl_xor(v, 32));
    };
    top = largest(top);
    if (lane == 0) tops[w] = top;
    const bool lost = __syncthreads_or(no_number);
#pragma unroll
    for (int i = 0; i < NW; ++i) top = fmaxf(top, tops[i]);
    top = lost ? kNoNumber : fmaxf(top, before.x);               // (and with it all of the state)
    keep = before.x == kNone ? 0.f : fast_exp2(before.x - top);
    // z, and the queries' references: their largest contribution p z, to its power of two
    float most[GC];
#pragma unroll
    for (int j = 0; j < GC; ++j) most[j] = kNone;
    for (int m = tid; m < Mp; m += NTH) {
      const float s = top == kNone ? 0.f : fast_exp2(feat[m] - top);
      float z = s;
      if (keep != 0.f && m < M) z += keep * old_z[m];
      feat[m] = s;
      zs[m] = z;
      if (m < M && g0 == 0 && blockIdx.z == 0) a.state.z[at * M + m] = z;
      const float power = z == 0.f ? kNone : (float)__builtin_amdgcn_frexp_expf(z);
#pragma unroll
      for (int j = 0; j < GC; ++j)
        if (j < n) most[j] = fmaxf(most[j], feat[(1 + j) * Mp + m] + power);
    }
    if (tid == 0 && g0 == 0 && blockIdx.z == 0) a.state.shift[at] = top;
#pragma unroll
    for (int j = 0; j < GC; ++j) {
      most[j] = largest(most[j]);
      if (lane == 0) tops[(1 + j) * NW + w] = most[j];
    }
    __syncthreads();
    // p, 2^24 below: up to 2^124 where z is the smallest number
    float den[GC];
#pragma unroll
    for (int j = 0; j < GC; ++j) {
      den[j] = 0.f;
#pragma unroll
      for (int i = 0; i < NW; ++i) most[j] = fmaxf(most[j], tops[(1 + j) * NW + i]);
    }
    for (int m = tid; m < Mp; m += NTH) {
      const float z = zs[m];
#pragma unroll
      for (int j = 0; j < GC; ++j)
        if (j < n) {
          const float p = z == 0.f ? 0.f : fast_exp2(feat[(1 + j) * Mp + m] - most[j] - 24.f);
          feat[(1 + j) * Mp + m] = p;
          den[j] += p * z;
        }
    }
#pragma unroll
    for (int j = 0; j < GC; ++j) {
      den[j] = over_lanes<32>(den[j], [](float p, float q) { return p + q; });
      den[j] += __shfl_xor(den[j], 32);
      if (lane == 0) dens[j * NW + w] = den[j];
    }
    __syncthreads();
    // the state
    vec acc[GC] = {};
    for (int k0 = 0; k0 < mine; k0 += AHEAD) {
      if (g0 > 0 || k0 > 0)
#pragma unroll
        for (int i = 0; i < AHEAD; ++i)
          if (k0 + i < mine) t[i] = T[(size_t)(k0 + i) * step];
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) {
        if (k0 + i >= mine) continue;
        const int m = r0 + (k0 + i) * pass;
        if (g0 == 0) {
          t[i] = keep != 0.f ? keep * t[i] + feat[m] * v : feat[m] * v;
          T[(size_t)(k0 + i) * step] = t[i];
        }
#pragma unroll
        for (int j = 0; j < GC; ++j)
          if (j < n) acc[j] += feat[(1 + j) * Mp + m] * t[i];
      }
    }
    if (worker)
#pragma unroll
      for (int j = 0; j < GC; ++j)
        if (j < n)
#pragma unroll
          for (int i = 0; i < VEC; ++i) part[(j * pass + r0) * cols + VEC * q0 + i] = acc[j][i];
    __syncthreads();
    for (int e = tid; e < n * cols; e += NTH) {
      const int j = e / cols, c = e - j * cols;
      float sum = 0.f, d = 0.f;
#pragma unroll 4
      for (int r = 0; r < pass; ++r) sum += part[(j * pass + r) * cols + c];
#pragma unroll
      for (int i = 0; i < NW; ++i) d += dens[j * NW + i];
      store_elem(a.Y, row_base(a.Y, b, h * G + g0 + j, 0) + col0 + c, d == 0.f ? 0.f : sum / d);
      unread += col0 + c == 0 && d == 0.f;
    }
  }
  if (unread > 0 && a.unread != nullptr) atomicAdd(a.unread, unread);
}

template <int S, int VEC, int GC, int NTH, bool ONE> int step(const StepArgs& a, hipStream_t st) {
  const size_t lds = step_lds_floats<GC, NTH>(a.f.p.Mp) * sizeof(float);
  auto kernel = k_step<S, VEC, GC, NTH, ONE>;
  if (lds > 64 * 1024 && hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds) != hipSuccess) {
    (void)hipGetLastError();
    return 5;
  }
  hipLaunchKernelGGL(kernel, dim3(a.B, a.Hk, (a.dv + a.cols - 1) / a.cols), dim3(NTH), lds, st, a);
  return hipGetLastError() == hipSuccess ? 0 : 5;
}
template <int S> int step_one(const StepArgs& a, hipStream_t st) {
  return a.dv % 4 == 0 ? step<S, 4, 1, 512, true>(a, st) : step<S, 1, 1, 512, true>(a, st);
}
bool step_in_one(int B, int H, int Hk, int d, int Mp) { return H == Hk && (long long)B * Hk <= 256 && d <= 64 && Mp <= 256; }

}  // namespace

size_t step_floats(int B, int H, int Hk, int d, int Mp) {
  return step_in_one(B, H, Hk, d, Mp) ? 0 : (size_t)B * ((size_t)(H + Hk) * Mp + (size_t)Hk * Mp + 2 * Hk) + 4;
}

int launch_step(StepArgs a, float* room, hipStream_t st) {
  const int Mp = a.f.p.Mp, steps = a.f.p.steps, G = a.H / a.Hk;
  a.cols = a.dv;
  if (step_in_one(a.B, a.H, a.Hk, a.f.d, Mp)) return steps == 1 ? step_one<1>(a, st) : step_one<2>(a, st);
  a.old_shift = (float2*)room;
  a.exps = room + 2 * (size_t)a.B * a.Hk;
  a.exps += (4 - ((a.exps - room) & 3)) & 3;
  a.old_z = a.exps + (size_t)a.B * (a.H + a.Hk) * Mp;
  a.key_tiles = (a.B + 15) / 16;
  const long long tiles = a.key_tiles + ((long long)a.B * G + 15) / 16;
  const dim3 grid((Mp / 32 + 3) / 4 + (a.f.dense ? 1 : 0), a.Hk, (unsigned)tiles);
  if (steps == 1) hipLaunchKernelGGL(k_step_exponents<1>, grid, dim3(256), 0, st, a);
  else if (steps == 2) hipLaunchKernelGGL(k_step_exponents<2>, grid, dim3(256), 0, st, a);
  else hipLaunchKernelGGL(k_step_exponents<4>, grid, dim3(256), 0, st, a);
  if (hipGetLastError() != hipSuccess) return 5;
  // a state in halves or quarters of its columns, 16 at least, until four workgroups a CU are there
  while ((long long)a.B * a.Hk * ((a.dv + a.cols - 1) / a.cols) < 1024 && a.cols % 32 == 0 && 4 * a.cols > a.dv) a.cols /= 2;
  if (G == 1) return a.dv % 4 == 0 ? step<1, 4, 1, 256, false>(a, st) : step<1, 1, 1, 256, false>(a, st);
  return a.dv % 4 == 0 ? step<1, 4, 4, 256, false>(a, st) : step<1, 1, 4, 256, false>(a, st);
}

}  // namespace st
}  // namespace fs
