// States of sequences: the projection constants they are built and read with, sums over rows (keys and values onto a state; the gradient of
// a state), and the join of partial sums.
//
// k_build: a workgroup takes a part of the rows 32 at a time; its waves have 32 features each, whose rows of W and of the sum stay in
// registers.  Rows are read, turned and split into bf16 pieces once for all waves (split3.h: fp32 products on the bf16 matrix
// instructions).  The exponents come out feature by lane and row by register: two stacked tiles are, without a move, the operand of
// the sum over rows.  A wave has a reference of its own, raised when an exponent passes it by 2^16 (never after the first rows, as a
// rule): features lie up to 2^8 above one at first, so that those far below the largest still split into whole pieces.
#include <algorithm>

#include "state_common.h"

namespace fs {
namespace st {
namespace {

// ---------------------------------------------------------------------------------------------- projection constants
// Sums in 64 bits: the constants are made once and used for every row.
__global__ void __launch_bounds__(256) k_prepare(const float* theta, int groups, const float* Omega, int omega_groups, int d, int M, float scale,
                                                 char* buf, FeaturePlan p) {
  __shared__ float om[32][128];
  const int blk = blockIdx.x, side = blockIdx.y, set = blockIdx.z, tid = threadIdx.x;
  const size_t dd = (size_t)d * d;
  const float* th = theta + (size_t)(groups == 1 ? 0 : set) * (FS_THETA_HEADER_ + d + 4 * dd);
  const float* omega = Omega + (size_t)(omega_groups == 1 ? 0 : set) * M * d;
  const float *A = th + FS_THETA_HEADER_, *Bm = A + d + side * dd, *C2 = A + d + 3 * dd;
  char* base = buf + 256 + (size_t)set * p.set;
  for (int i = tid; i < 32 * 128; i += 256) {
    const int m = 32 * blk + (i >> 7), c = i & 127;
    om[i >> 7][c] = m < M && c < d ? omega[(size_t)m * d + c] : 0.f;
  }
  __syncthreads();
  uint16_t *row = (uint16_t*)(base + p.off_row[side]), *col = (uint16_t*)(base + p.off_col[side]);
  float* w = (float*)(base + p.off_w[side]);
  for (int i = tid; i < 32 * 32 * p.steps; i += 256) {
    const int f = i / (32 * p.steps), c = i - f * 32 * p.steps, m = 32 * blk + f, tile = f >> 4, r = f & 15;
    double sum = 0.0;
    if (c < d)
      for (int l = 0; l < d; ++l) sum += (double)om[f][l] * (double)Bm[(size_t)l * d + c];
    const float v = (float)(sum * (double)scale * 1.4426950408889634074);
    split3_store(row + ((size_t)blk * p.steps + (c >> 5)) * 3 * 1024 + tile * 512 + ((c & 31) / 8 * 16 + r) * 8 + (c & 7), 1024, v);
    split3_store(col + ((size_t)blk * p.tiles + (c >> 4)) * 3 * 512 + (r / 4 * 16 + (c & 15)) * 8 + 4 * tile + (r & 3), 512, v);
    if (c < 4 * p.d4) w[((size_t)(c >> 2) * p.Mp + m) * 4 + (c & 3)] = v;
  }
  if (side == 0) {
    if (tid < 32) {
      const int m = 32 * blk + tid;
      double q = 0.0;
      for (int l = 0; l < d; ++l) q += (double)A[l] * (double)om[tid][l] * (double)om[tid][l];
      ((float*)(base + p.off_bias))[m] = m < M ? (float)((q + (double)th[0] - 0.5 * log((double)M)) * 1.4426950408889634074) : kNone;
    }
    return;
  }
  if (blk == 0) {
    uint16_t* csym = (uint16_t*)(base + p.off_csym);
    const int n = 32 * p.steps;
    for (int i = tid; i < n * n; i += 256) {
      const int a = i / n, c = i - a * n;
      const float v = a < d && c < d ? C2[(size_t)a * d + c] + C2[(size_t)c * d + a] : 0.f;
      split3_store(csym + ((size_t)(c >> 4) * p.steps + (a >> 5)) * 3 * 512 + ((a & 31) / 8 * 16 + (c & 15)) * 8 + (a & 7), 512, v);
    }
    for (int i = tid; i < (int)dd; i += 256) ((float*)(base + p.off_c2))[i] = C2[i];
    if (tid == 0 && ((int)th[2] & 1) == 0) atomicOr((unsigned*)buf, 1u);
  }
}

// ---------------------------------------------------------------------------------------------- row terms of dense quadratic forms
__global__ void __launch_bounds__(256) k_row_terms(Features f, Rows x, int Hk, const float* shift, const int32_t* slots, int nslots, float* terms) {
  __shared__ float y[16][132];
  const int bh = blockIdx.y, b = bh / Hk, h = bh - b * Hk, r0 = 16 * blockIdx.x;
  const int row = threadIdx.x >> 4, u = threadIdx.x & 15, len = length_of(x, b);
  const int slot = shift ? unique_slot_of(slots, nslots, b) : 0;
  const bool live = r0 + row < len && slot >= 0;
  f32x8 v = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  if (live) v = row8(x, b, h, RowAt{0, r0 + row}, 8 * u);
#pragma unroll
  for (int i = 0; i < 8; ++i) y[row][8 * u + i] = v[i];
  __syncthreads();
  float sum = 0.f;
  if (f.dense) {
    const float* C2 = (const float*)(f.set(h) + f.p.off_c2);
    for (int c = u; c < f.d; c += 16) {
      float z = 0.f;
      for (int a = 0; a < f.d; ++a) z += y[row][a] * C2[a * f.d + c];
      sum += z * y[row][c];
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) sum += v[i] * v[i];
    sum *= -0.5f;
  }
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
  if (u == 0 && r0 + row < x.L)
    terms[(size_t)bh * x.L + r0 + row] = live ? kLog2e * f.scale2 * sum - (shift ? shift[(size_t)slot * Hk + h] : 0.f) : kNone;
}

// ---------------------------------------------------------------------------------------------- sums over rows
template <int W, int XP, int VP> struct BuildLds {
  uint16_t x[2][XP][32][W + 8];
  uint16_t v[2][VP][32][W + 8];
  float term[2][32], weight[2][32];
};

template <int W, int XP, int VP, int NW>
__global__ void __launch_bounds__(64 * NW) k_build(BuildArgs a) {
  constexpr int S = STEPS<W>, VT = TILES<W>, UPR = W / 8, NTH = 64 * NW, U = (64 * UPR + NTH - 1) / NTH, LD = W + 8;
  extern __shared__ __align__(16) char lds_raw[];
  BuildLds<W, XP, VP>& lds = *(BuildLds<W, XP, VP>*)lds_raw;
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), g = lane >> 4, c = lane & 15;
  const int split = blockIdx.x, bh = blockIdx.z, b = bh / a.Hk, h = bh - b * a.Hk;
  const int fb = blockIdx.y * NW + w, nfb = a.f.p.Mp / 32, steps = a.f.p.steps, dv = a.dv;
  const int slot = slot_of(a.slots, a.nslots, b);
  if (a.old_shift != nullptr && split == 0 && blockIdx.y == 0 && tid == 0) a.old_shift[bh] = slot >= 0 ? a.shift[(size_t)slot * a.Hk + h] : kNone;
  const int len = length_of(a.x, b), rows = a.x.L * a.x.G;
  const int v0 = split * a.rows_per_split, v1 = slot < 0 ? 0 : min(a.x.G == 1 ? len : rows, v0 + a.rows_per_split);
  const bool active = fb < nfb;
  if (v0 >= v1) {
    if (active && lane == 0) a.refs[((size_t)bh * a.nsplit + split) * nfb + fb] = make_float2(0.f, kNone);
    return;
  }
  const char* set = a.f.set(h);
  Op<3> wop[2][S];
  float bias[2] = {kNone, kNone};
  if (active) {
    const uint16_t* img = (const uint16_t*)(set + a.f.p.off_row[a.side]) + (size_t)fb * steps * 3 * 1024;
#pragma unroll
    for (int s = 0; s < S; ++s)
      if (s < steps)
#pragma unroll
        for (int ft = 0; ft < 2; ++ft)
#pragma unroll
          for (int p = 0; p < 3; ++p) wop[ft][s].p[p] = *(const bf16x8*)(img + (s * 3 + p) * 1024 + ft * 512 + lane * 8);
#pragma unroll
    for (int ft = 0; ft < 2; ++ft) bias[ft] = ((const float*)(set + a.f.p.off_bias))[32 * fb + 16 * ft + c];
  }
  f32x4 T[2][VT];
  float z[2] = {0.f, 0.f}, ref = kNone, top = kNone;
#pragma unroll
  for (int ft = 0; ft < 2; ++ft)
#pragma unroll
    for (int vt = 0; vt < VT; ++vt) T[ft][vt] = f32x4{0.f, 0.f, 0.f, 0.f};

  // units of eight numbers of a row: those of x, then those of v
  f32x8 next[U];
  float next_term[U], next_weight[U];
  auto fetch = [&](int v) {
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int e = tid + NTH * i;
      const bool is_x = e < 32 * UPR;
      const int q = is_x ? e : e - 32 * UPR, row = q / UPR, c0 = 8 * (q % UPR);
      next[i] = f32x8{0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
      next_term[i] = kNone;
      next_weight[i] = 0.f;
      if (q >= 32 * UPR || v + row >= v1) continue;
      const RowAt at = row_at(a.x, v + row);
      if (at.row >= len) continue;
      if (is_x) {
        next[i] = row8(a.x, b, h, at, c0);
        next_term[i] = a.terms ? a.terms[(size_t)bh * rows + v + row] : 0.f;
        next_weight[i] = a.weights ? a.weights[(size_t)bh * rows + v + row] : 1.f;
      } else {
        next[i] = row8(a.v, b, h, at, c0);
      }
    }
  };
  auto put = [&](int buf) {
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int e = tid + NTH * i;
      const bool is_x = e < 32 * UPR;
      const int q = is_x ? e : e - 32 * UPR, row = q / UPR, u = q % UPR;
      if (q >= 32 * UPR) continue;
      if (is_x) {
        const Op<XP> o = as_op<XP>(next[i]);
#pragma unroll
        for (int p = 0; p < XP; ++p) *(bf16x8*)&lds.x[buf][p][row][8 * u] = o.p[p];
        float t = next_term[i];
        if (a.terms == nullptr) {                       // C2 = -I / 2
          float n = 0.f;
#pragma unroll
          for (int j = 0; j < 8; ++j) n += next[i][j] * next[i][j];
#pragma unroll
          for (int o2 = UPR / 2; o2 > 0; o2 >>= 1) n += __shfl_xor(n, o2);
          t += -0.5f * kLog2e * a.f.scale2 * n;
        }
        if (u == 0) {
          lds.term[buf][row] = t;
          lds.weight[buf][row] = next_weight[i];
        }
      } else {
        const Op<VP> o = as_op<VP>(next[i]);
#pragma unroll
        for (int p = 0; p < VP; ++p) *(bf16x8*)&lds.v[buf][p][row][8 * u] = o.p[p];
      }
    }
  };

  fetch(v0);
  put(0);
  __syncthreads();
  int buf = 0;
  for (int v = v0; v < v1; v += 32, buf ^= 1) {
    const bool more = v + 32 < v1;
    if (more) fetch(v + 32);
    if (active) {
      f32x4 E[2][2];             // [tile of rows][tile of features]
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
        E[t][0] = E[t][1] = zero;
#pragma unroll
        for (int s = 0; s < S; ++s)
          if (s < steps) {
            const Op<XP> x = row_op<XP>(&lds.x[buf][0][16 * t + c][32 * s + 8 * g], 32 * LD);
            E[t][0] = times(x, wop[0][s], E[t][0]);
            E[t][1] = times(x, wop[1][s], E[t][1]);
          }
      }
      f32x4 weight[2];
      float most = kNone;
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const f32x4 term = *(const f32x4*)&lds.term[buf][16 * t + 4 * g];
        weight[t] = *(const f32x4*)&lds.weight[buf][16 * t + 4 * g];
#pragma unroll
        for (int ft = 0; ft < 2; ++ft)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            E[t][ft][r] = (E[t][ft][r] + bias[ft]) + term[r];
            most = fmaxf(most, E[t][ft][r]);
          }
      }
      top = fmaxf(top, most);
      if (__any(most > ref + 16.f)) {
        float m = most;
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
        const float keep = fast_exp2(ref - (m - 8.f));
        ref = m - 8.f;
#pragma unroll
        for (int ft = 0; ft < 2; ++ft) {
          z[ft] *= keep;
#pragma unroll
          for (int vt = 0; vt < VT; ++vt) T[ft][vt] *= keep;
        }
      }
      const float at = ref == kNone ? 0.f : ref;
      Op<3> so[2];
#pragma unroll
      for (int ft = 0; ft < 2; ++ft) {
        f32x8 sv;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const float x = fast_exp2(E[t][ft][r] - at);
            sv[4 * t + r] = x;
            z[ft] += x * weight[t][r];
          }
        so[ft] = as_op<3>(sv);
      }
#pragma unroll
      for (int vt = 0; vt < VT; ++vt)
        if (16 * vt < dv) {
          const Op<VP> vo = column_op<VP>(&lds.v[buf][0][0][16 * vt] + lane_tr(lane, LD), LD, 32 * LD);
          T[0][vt] = times(so[0], vo, T[0][vt]);
          T[1][vt] = times(so[1], vo, T[1][vt]);
        }
    }
    if (more) put(buf ^ 1);
    __syncthreads();
  }
  if (!active) return;
  const size_t at = (size_t)bh * a.nsplit + split;
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
  if (lane == 0) a.refs[at * nfb + fb] = make_float2(ref, top);
#pragma unroll
  for (int ft = 0; ft < 2; ++ft) {
    const int m0 = 32 * fb + 16 * ft;
    float zs = z[ft];
    zs += __shfl_xor(zs, 16);
    zs += __shfl_xor(zs, 32);
    if (g == 0 && m0 + c < a.f.M) a.zpart[at * a.f.M + m0 + c] = zs;
#pragma unroll
    for (int vt = 0; vt < VT; ++vt)
      if (16 * vt + c < dv)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (m0 + 4 * g + r < a.f.M) a.part[(at * a.f.M + m0 + 4 * g + r) * dv + 16 * vt + c] = T[ft][vt][r];
  }
}

// ---------------------------------------------------------------------------------------------- join
constexpr int kJoinWeights = 4096;       // references of a state's partial sums: at most 64 splits of 2048 features

__device__ __forceinline__ float block_max(float v, float* tmp) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o));
  if ((threadIdx.x & 63) == 0) tmp[threadIdx.x >> 6] = v;
  __syncthreads();
  return fmaxf(fmaxf(tmp[0], tmp[1]), fmaxf(tmp[2], tmp[3]));
}

template <int VEC>
__global__ void __launch_bounds__(256) k_join(JoinArgs a) {
  __shared__ float weight[kJoinWeights], tmp[4];
  typedef __attribute__((ext_vector_type(VEC))) float vec;
  const int bh = blockIdx.y, b = bh / a.Hk, h = bh - b * a.Hk, tid = threadIdx.x, nfb = a.Mp / 32;
  const int slot = unique_slot_of(a.slots, a.state.slots, b);
  if (slot < 0) {
    if (blockIdx.x == 0 && h == 0 && tid == 0 && a.left_out != nullptr) atomicAdd(a.left_out, 1);
    return;
  }
  const int n = a.nsplit * nfb;
  const float2* refs = a.refs + (size_t)bh * n;
  const float old = a.old_shift ? a.old_shift[bh] : kNone;
  float top = old;
  for (int i = tid; i < n; i += 256) top = fmaxf(top, refs[i].y);
  top = block_max(top, tmp);
  for (int i = tid; i < n; i += 256) weight[i] = refs[i].y == kNone ? 0.f : fast_exp2(refs[i].x - top);
  __syncthreads();
  const float keep = old == kNone ? 0.f : fast_exp2(old - top);
  const size_t at = (size_t)slot * a.Hk + h;
  const int nt = a.M * a.dv / VEC;
  for (int e = blockIdx.x * 256 + tid; e < nt + a.M; e += gridDim.x * 256) {
    if (e < nt) {
      const int m = e * VEC / a.dv, fb = m >> 5;
      vec* to = (vec*)(a.state.T + at * a.M * a.dv) + e;
      vec x = {};
      if (keep != 0.f) x = keep * *to;
      for (int s = 0; s < a.nsplit; ++s) {
        const float k = weight[s * nfb + fb];
        if (k != 0.f) x += k * ((const vec*)(a.part + ((size_t)bh * a.nsplit + s) * a.M * a.dv))[e];
      }
      *to = x;
    } else {
      const int m = e - nt, fb = m >> 5;
      float* to = a.state.z + at * a.M + m;
      float x = keep != 0.f ? keep * *to : 0.f;
      for (int s = 0; s < a.nsplit; ++s) {
        const float k = weight[s * nfb + fb];
        if (k != 0.f) x += k * a.zpart[((size_t)bh * a.nsplit + s) * a.M + m];
      }
      *to = x;
    }
  }
  if (blockIdx.x == 0 && tid == 0) a.state.shift[at] = top;
}

template <int VEC>
__global__ void __launch_bounds__(256) k_join_sum(JoinArgs a) {
  typedef __attribute__((ext_vector_type(VEC))) float vec;
  const int sh = blockIdx.y, slot = sh / a.Hk, h = sh - slot * a.Hk, nfb = a.Mp / 32, nt = a.M * a.dv / VEC;
  const int b0 = a.slots ? 0 : slot, b1 = a.slots ? a.B : min(slot + 1, a.B);
  for (int e = blockIdx.x * 256 + threadIdx.x; e < nt + a.M; e += gridDim.x * 256) {
    const int m = e < nt ? e * VEC / a.dv : e - nt, fb = m >> 5;
    vec x = {};
    for (int b = b0; b < b1; ++b) {
      if (slot_of(a.slots, a.state.slots, b) != slot) continue;
      const size_t at = ((size_t)b * a.Hk + h) * a.nsplit;
      for (int s = 0; s < a.nsplit; ++s) {
        const float2 ref = a.refs[(at + s) * nfb + fb];
        if (ref.y == kNone) continue;
        const float k = fast_exp2(ref.x);
        if (e < nt) x += k * ((const vec*)(a.part + (at + s) * a.M * a.dv))[e];
        else x[0] += k * a.zpart[(at + s) * a.M + m];
      }
    }
    if (e < nt) ((vec*)(a.state.T + (size_t)sh * a.M * a.dv))[e] = x;
    else a.state.z[(size_t)sh * a.M + m] = x[0];
  }
}

template <int W, int XP, int VP, int NW> int build(const BuildArgs& a, hipStream_t st) {
  constexpr size_t lds = sizeof(BuildLds<W, XP, VP>);
  auto kernel = k_build<W, XP, VP, NW>;
  if (lds > 64 * 1024 && hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds) != hipSuccess) {
    (void)hipGetLastError();
    return 5;
  }
  hipLaunchKernelGGL(kernel, dim3(a.nsplit, a.nblock, a.B * a.Hk), dim3(64 * NW), lds, st, a);
  return hipGetLastError() == hipSuccess ? 0 : 5;
}
template <int W, int XP, int VP> int build_nw(const BuildArgs& a, hipStream_t st) {
  return a.f.p.Mp > 128 ? build<W, XP, VP, 8>(a, st) : build<W, XP, VP, 4>(a, st);
}
template <int W> int build_pieces(const BuildArgs& a, hipStream_t st) {
  if (a.v.X.dtype == 1) return a.x.X.dtype == 1 && a.x.turn.rot == 0 ? build_nw<W, 1, 1>(a, st) : build_nw<W, 3, 1>(a, st);
  return build_nw<W, 3, 3>(a, st);
}
int join_grid(const JoinArgs& a, int vec) { return std::max(1, std::min((a.M * a.dv / vec + a.M + 255) / 256, 64)); }

}  // namespace

int launch_build(const BuildArgs& a, hipStream_t st) {
  switch (width_class(a.f.d, a.dv)) {
    case 32: return build_pieces<32>(a, st);
    case 64: return build_pieces<64>(a, st);
    default: return build_pieces<128>(a, st);
  }
}
int launch_join(const JoinArgs& a, hipStream_t st) {
  if (a.dv % 4 == 0) hipLaunchKernelGGL(k_join<4>, dim3(join_grid(a, 4), a.B * a.Hk), dim3(256), 0, st, a);
  else hipLaunchKernelGGL(k_join<1>, dim3(join_grid(a, 1), a.B * a.Hk), dim3(256), 0, st, a);
  return hipGetLastError() == hipSuccess ? 0 : 5;
}
int launch_join_sum(const JoinArgs& a, hipStream_t st) {
  if (a.dv % 4 == 0) hipLaunchKernelGGL(k_join_sum<4>, dim3(join_grid(a, 4), a.state.slots * a.Hk), dim3(256), 0, st, a);
  else hipLaunchKernelGGL(k_join_sum<1>, dim3(join_grid(a, 1), a.state.slots * a.Hk), dim3(256), 0, st, a);
  return hipGetLastError() == hipSuccess ? 0 : 5;
}
int launch_prepare(const float* theta, int groups, const float* Omega, int omega_groups, int sets, int d, int M, float scale, char* buf,
                   const FeaturePlan& p, hipStream_t st) {
  if (int rc = launch_fill_u32((uint32_t*)buf, 0u, 1, st)) return rc;
  hipLaunchKernelGGL(k_prepare, dim3(p.Mp / 32, 2, sets), dim3(256), 0, st, theta, groups, Omega, omega_groups, d, M, scale, buf, p);
  return hipGetLastError() == hipSuccess ? 0 : 5;
}
int launch_row_terms(const Features& f, const Rows& k, int B, int Hk, const float* shift, const int32_t* slots, int nslots, float* terms,
                     hipStream_t st) {
  hipLaunchKernelGGL(k_row_terms, dim3((k.L + 15) / 16, B * Hk), dim3(256), 0, st, f, k, Hk, shift, slots, nslots, terms);
  return hipGetLastError() == hipSuccess ? 0 : 5;
}

}  // namespace st
}  // namespace fs
