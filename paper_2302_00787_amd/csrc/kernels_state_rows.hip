// Rows against a finished state: the features of queries (or keys) times the state's rows, and the gradient of rows through their features.
//
// A wave takes whole rows (16 RT of them) through all features, 32 at a time; the workgroup brings the operand images of W and the
// state's 32 rows, split into bf16 pieces, to LDS for all its waves, the next ones on their way meanwhile.  The exponents come out
// row by lane and feature by register: two stacked tiles are, without a move, the operand of the product with the state (whose
// columns come from the transposing LDS read) and of that with W.  A row's reference is raised when an exponent passes it by 2^16,
// which its first 32 features as a rule prevent; the quotient loses it.
#include <algorithm>

#include "state_common.h"

namespace fs {
namespace st {
namespace {

// What a step of 32 features needs in LDS.
template <int W, bool COL> struct StepLds {
  uint16_t row[STEPS<W>][3][1024];
  uint16_t col[COL ? TILES<W> : 1][3][COL ? 512 : 8];
  uint16_t t[3][32][W + 8];
  float z[32], bias[32];
};
template <int W, bool COL, int NW> struct Stage {
  static constexpr int NTH = 64 * NW, NI = (STEPS<W> * 384 + NTH - 1) / NTH, NT = (8 * W + NTH - 1) / NTH;
  u32x4 row[NI], col[COL ? NI : 1];
  f32x4 t[NT];
  float z, bias;
  const char *row_img, *col_img;
  const float *T, *zs, *biases;
  int units, M, dv;                 // units of 16 bytes of an image of 32 features

  __device__ __forceinline__ void start(const Features& f, int side, const char* set, const float* T_, const float* z_, int dv_) {
    row_img = set + f.p.off_row[side];
    col_img = set + f.p.off_col[side];
    biases = (const float*)(set + f.p.off_bias);
    T = T_; zs = z_; dv = dv_; M = f.M;
    units = f.p.steps * 384;
  }
  __device__ __forceinline__ void fetch(int fb, int tid) {
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const int e = tid + NTH * i;
      if (e < units) {
        row[i] = *(const u32x4*)(row_img + ((size_t)fb * units + e) * 16);
        if constexpr (COL) col[i] = *(const u32x4*)(col_img + ((size_t)fb * units + e) * 16);
      }
    }
#pragma unroll
    for (int i = 0; i < NT; ++i) {
      const int e = tid + NTH * i, m = 32 * fb + e / (W / 4), c = 4 * (e % (W / 4));
      t[i] = f32x4{0.f, 0.f, 0.f, 0.f};
      if (e < 8 * W && m < M && c < dv) {
        const float* p = T + (size_t)m * dv + c;
        if ((dv & 3) == 0) t[i] = *(const f32x4*)p;
        else
#pragma unroll
          for (int j = 0; j < 4; ++j) t[i][j] = c + j < dv ? p[j] : 0.f;
      }
    }
    if (tid < 32) {
      z = zs != nullptr && 32 * fb + tid < M ? zs[32 * fb + tid] : 0.f;
      bias = biases[32 * fb + tid];
    }
  }
  __device__ __forceinline__ void put(StepLds<W, COL>& lds, int tid) {
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const int e = tid + NTH * i;
      if (e < units) {
        *(u32x4*)((char*)lds.row + e * 16) = row[i];
        if constexpr (COL) *(u32x4*)((char*)lds.col + e * 16) = col[i];
      }
    }
#pragma unroll
    for (int i = 0; i < NT; ++i) {
      const int e = tid + NTH * i, m = e / (W / 4), c = 4 * (e % (W / 4));
      if (e < 8 * W) {
        const Split3 s = split3(t[i], t[i]);
        *(u32x2*)&lds.t[0][m][c] = u32x2{__builtin_bit_cast(u32x4, s.h)[0], __builtin_bit_cast(u32x4, s.h)[1]};
        *(u32x2*)&lds.t[1][m][c] = u32x2{__builtin_bit_cast(u32x4, s.m)[0], __builtin_bit_cast(u32x4, s.m)[1]};
        *(u32x2*)&lds.t[2][m][c] = u32x2{__builtin_bit_cast(u32x4, s.l)[0], __builtin_bit_cast(u32x4, s.l)[1]};
      }
    }
    if (tid < 32) {
      lds.z[tid] = z;
      lds.bias[tid] = bias;
    }
  }
};

// A tile of 16 rows from the accumulators (register r of lane (g, c): row 4 g + r, column 16 ct + c) to a wave's own part of LDS.
template <int W> __device__ __forceinline__ void tile_to_lds(float* dst, const f32x4 (&acc)[TILES<W>], int lane) {
  const int g = lane >> 4, c = lane & 15;
#pragma unroll
  for (int ct = 0; ct < TILES<W>; ++ct)
#pragma unroll
    for (int r = 0; r < 4; ++r) dst[(4 * g + r) * (W + 4) + 16 * ct + c] = acc[ct][r];
  __builtin_amdgcn_wave_barrier();
  asm volatile("" ::: "memory");
}

template <int W, int XP, int NW>
__global__ void __launch_bounds__(64 * NW) k_values(ValueArgs a) {
  constexpr int S = STEPS<W>, VT = TILES<W>, RT = 2, LD = W + 8;
  extern __shared__ __align__(16) char lds_raw[];
  StepLds<W, false>* lds = (StepLds<W, false>*)lds_raw;
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), g = lane >> 4, c = lane & 15;
  const int bh = blockIdx.y, b = bh / a.Hk, h = bh - b * a.Hk, steps = a.f.p.steps, dv = a.dv, nfb = a.f.p.Mp / 32;
  const int slot = slot_of(a.slots, a.state.slots, b), len = length_of(a.x, b), rows = a.x.L * a.x.G;
  const int v0 = (blockIdx.x * NW + w) * 16 * RT;
  const char* set = a.f.set(h);
  const size_t st = (size_t)max(slot, 0) * a.Hk + h;

  // this lane's row of each tile: row v0 + 16 rt + c
  Op<XP> x[RT][S];
  float term[RT], ref[RT], den[RT];
  f32x4 acc[RT][VT];
  bool live[RT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const int v = v0 + 16 * rt + c;
    const RowAt at = row_at(a.x, min(v, rows - 1));
    live[rt] = v < rows && at.row < len;
    term[rt] = a.terms && live[rt] ? a.terms[(size_t)bh * rows + v] : 0.f;
    ref[rt] = kNone;
    den[rt] = 0.f;
#pragma unroll
    for (int s = 0; s < S; ++s)
      if (s < steps) {
        f32x8 n = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (live[rt]) n = row8(a.x, b, h, at, 32 * s + 8 * g);
        x[rt][s] = as_op<XP>(n);
      }
#pragma unroll
    for (int vt = 0; vt < VT; ++vt) acc[rt][vt] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  if (slot >= 0) {
    Stage<W, false, NW> stage;
    stage.start(a.f, a.side, set, a.state.T + st * a.f.M * dv, a.state.z ? a.state.z + st * a.f.M : nullptr, dv);
    stage.fetch(0, tid);
    stage.put(lds[0], tid);
    __syncthreads();
    for (int fb = 0; fb < nfb; ++fb) {
      const StepLds<W, false>& l = lds[fb & 1];
      const bool more = fb + 1 < nfb;
      if (more) stage.fetch(fb + 1, tid);
      f32x4 E[RT][2];
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) E[rt][0] = E[rt][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int s = 0; s < S; ++s)
        if (s < steps)
#pragma unroll
          for (int ft = 0; ft < 2; ++ft) {
            Op<3> wo;
#pragma unroll
            for (int p = 0; p < 3; ++p) wo.p[p] = *(const bf16x8*)&l.row[0][0][(s * 3 + p) * 1024 + ft * 512 + lane * 8];
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) E[rt][ft] = times(wo, x[rt][s], E[rt][ft]);
          }
      f32x4 zf[2];
      Op<3> po[RT];
#pragma unroll
      for (int ft = 0; ft < 2; ++ft) {
        const f32x4 bias = *(const f32x4*)&l.bias[16 * ft + 4 * g];
        zf[ft] = *(const f32x4*)&l.z[16 * ft + 4 * g];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
#pragma unroll
          for (int r = 0; r < 4; ++r) E[rt][ft][r] = (E[rt][ft][r] + bias[r]) + term[rt];
      }
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        float most = kNone;
#pragma unroll
        for (int ft = 0; ft < 2; ++ft)
#pragma unroll
          for (int r = 0; r < 4; ++r) most = fmaxf(most, E[rt][ft][r]);
        if (__any(most > ref[rt] + 16.f)) {
          most = fmaxf(most, __shfl_xor(most, 16));
          most = fmaxf(most, __shfl_xor(most, 32));
          const float now = most > ref[rt] + 16.f ? most - 8.f : ref[rt];
          const float keep = now == ref[rt] ? 1.f : fast_exp2(ref[rt] - now);
          ref[rt] = now;
          den[rt] *= keep;
          f32x4 k;
#pragma unroll
          for (int r = 0; r < 4; ++r) k[r] = __shfl(keep, 4 * g + r);
#pragma unroll
          for (int vt = 0; vt < VT; ++vt)
#pragma unroll
            for (int r = 0; r < 4; ++r) acc[rt][vt][r] *= k[r];
        }
        const float at = ref[rt] == kNone ? 0.f : ref[rt];
        f32x8 p;
#pragma unroll
        for (int ft = 0; ft < 2; ++ft)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            p[4 * ft + r] = fast_exp2(E[rt][ft][r] - at);
            den[rt] += p[4 * ft + r] * zf[ft][r];
          }
        po[rt] = as_op<3>(p);
      }
#pragma unroll
      for (int vt = 0; vt < VT; ++vt)
        if (16 * vt < dv) {
          const Op<3> t = column_op<3>(&l.t[0][0][16 * vt] + lane_tr(lane, LD), LD, 32 * LD);
#pragma unroll
          for (int rt = 0; rt < RT; ++rt) acc[rt][vt] = times(po[rt], t, acc[rt][vt]);
        }
      if (more) stage.put(lds[(fb + 1) & 1], tid);
      __syncthreads();
    }
  }
  float* tile = (float*)lds_raw + w * 16 * (W + 4);
  int unread = 0;
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    den[rt] += __shfl_xor(den[rt], 16);
    den[rt] += __shfl_xor(den[rt], 32);
    const int v = v0 + 16 * rt + c;
    float factor;
    if (a.mode == OUT_SUM) factor = ref[rt] == kNone ? 0.f : fast_exp2(ref[rt]);
    else factor = den[rt] == 0.f ? 0.f : 1.f / den[rt];
    unread += g == 0 && live[rt] && den[rt] == 0.f;
    if (a.mode == OUT_STATS) {
      const float inv = factor;
      float delta[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int vr = v0 + 16 * rt + 4 * g + r;
        const RowAt at = row_at(a.x, min(vr, rows - 1));
        if (vr < rows && at.row < len) {
          const long long base = row_base(a.dY, b, h * a.x.G + at.head, at.row);
#pragma unroll
          for (int vt = 0; vt < VT; ++vt)
            if (16 * vt + c < dv) delta[r] += acc[rt][vt][r] * load_elem(a.dY, base + 16 * vt + c);
        }
#pragma unroll
        for (int o = 8; o > 0; o >>= 1) delta[r] += __shfl_xor(delta[r], o);
        delta[r] *= __shfl(inv, 4 * g + r);
        if (c == 0 && vr < rows) a.weights[(size_t)bh * rows + vr] = -delta[r];
      }
      if (g == 0 && v < rows) a.lse[(size_t)bh * rows + v] = live[rt] && den[rt] != 0.f ? -(ref[rt] + __log2f(den[rt])) : kNone;
      continue;
    }
    f32x4 k;
#pragma unroll
    for (int r = 0; r < 4; ++r) k[r] = __shfl(factor, 4 * g + r);
#pragma unroll
    for (int vt = 0; vt < VT; ++vt)
#pragma unroll
      for (int r = 0; r < 4; ++r) acc[rt][vt][r] *= k[r];
    tile_to_lds<W>(tile, acc[rt], lane);
    for (int u = lane; u < 16 * (W / 8); u += 64) {
      const int r = u / (W / 8), c0 = 8 * (u % (W / 8)), vr = v0 + 16 * rt + r;
      if (vr >= rows || c0 >= dv) continue;
      const RowAt at = row_at(a.x, vr);
      f32x8 y;
#pragma unroll
      for (int i = 0; i < 8; ++i) y[i] = tile[r * (W + 4) + c0 + i];
      if (at.row >= len) y = f32x8{0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
      store8(a.out, row_base(a.out, b, h * a.x.G + at.head, at.row), c0, dv, y);
    }
    __builtin_amdgcn_wave_barrier();
    asm volatile("" ::: "memory");
  }
  if (a.unread != nullptr) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) unread += __shfl_xor(unread, o);
    if (lane == 0 && unread > 0) atomicAdd(a.unread, unread);
  }
}

template <int W, int XP, int RP, int NW, int RT>
__global__ void __launch_bounds__(64 * NW) k_grads(GradArgs a) {
  constexpr int S = STEPS<W>, CT = TILES<W>;
  extern __shared__ __align__(16) char lds_raw[];
  StepLds<W, true>* lds = (StepLds<W, true>*)lds_raw;
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), g = lane >> 4, c = lane & 15;
  const int bh = blockIdx.y, b = bh / a.Hk, h = bh - b * a.Hk, steps = a.f.p.steps, dv = a.dv, nfb = a.f.p.Mp / 32, d = a.f.d;
  const int slot = slot_of(a.slots, a.state.slots, b);
  const int len = length_of(a.x, b), rows = a.x.L * a.x.G;
  const int v0 = (blockIdx.x * NW + w) * 16 * RT;
  const char* set = a.f.set(h);
  const size_t st = (size_t)max(slot, 0) * a.Hk + h;

  Op<XP> x[RT][S];
  Op<RP> rr[RT][S];
  float term[RT], weight[RT], rho[RT];
  f32x4 acc[RT][CT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const int v = v0 + 16 * rt + c;
    const RowAt at = row_at(a.x, min(v, rows - 1));
    const bool live = slot >= 0 && v < rows && at.row < len;
    term[rt] = kNone;
    weight[rt] = rho[rt] = 0.f;
#pragma unroll
    for (int s = 0; s < S; ++s) {
      if (s < steps) {
        f32x8 n = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (live) n = row8(a.x, b, h, at, 32 * s + 8 * g);
        x[rt][s] = as_op<XP>(n);
      }
      if (32 * s < dv) {
        f32x8 n = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (live) n = row8(a.r, b, h, at, 32 * s + 8 * g);
        rr[rt][s] = as_op<RP>(n);
      }
    }
    if (live) {
      term[rt] = a.terms[(size_t)bh * rows + v];
      weight[rt] = a.weights ? a.weights[(size_t)bh * rows + v] : 1.f;
    }
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) acc[rt][ct] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  if (slot >= 0) {
    Stage<W, true, NW> stage;
    stage.start(a.f, a.side, set, a.state.T + st * a.f.M * dv, a.state.z + st * a.f.M, dv);
    stage.fetch(0, tid);
    stage.put(lds[0], tid);
    __syncthreads();
    for (int fb = 0; fb < nfb; ++fb) {
      const StepLds<W, true>& l = lds[fb & 1];
      const bool more = fb + 1 < nfb;
      if (more) stage.fetch(fb + 1, tid);
      f32x4 E[RT][2], P[RT][2];
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) E[rt][0] = E[rt][1] = P[rt][0] = P[rt][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int s = 0; s < S; ++s)
        if (s < steps)
#pragma unroll
          for (int ft = 0; ft < 2; ++ft) {
            Op<3> wo;
#pragma unroll
            for (int p = 0; p < 3; ++p) wo.p[p] = *(const bf16x8*)&l.row[0][0][(s * 3 + p) * 1024 + ft * 512 + lane * 8];
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) E[rt][ft] = times(wo, x[rt][s], E[rt][ft]);
          }
#pragma unroll
      for (int s = 0; s < S; ++s)
        if (32 * s < dv)
#pragma unroll
          for (int ft = 0; ft < 2; ++ft) {
            const Op<3> t = row_op<3>(&l.t[0][16 * ft + c][32 * s + 8 * g], 32 * (W + 8));
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) P[rt][ft] = times(t, rr[rt][s], P[rt][ft]);
          }
      Op<3> uo[RT];
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        f32x8 u;
#pragma unroll
        for (int ft = 0; ft < 2; ++ft) {
          const f32x4 bias = *(const f32x4*)&l.bias[16 * ft + 4 * g], zf = *(const f32x4*)&l.z[16 * ft + 4 * g];
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const float p = fast_exp2((E[rt][ft][r] + bias[r]) + term[rt]);
            u[4 * ft + r] = p * (P[rt][ft][r] + weight[rt] * zf[r]);
            rho[rt] += u[4 * ft + r];
          }
        }
        uo[rt] = as_op<3>(u);
      }
#pragma unroll
      for (int ct = 0; ct < CT; ++ct)
        if (16 * ct < d) {
          const Op<3> wo = image_op<3>(&l.col[ct][0][0], lane);
#pragma unroll
          for (int rt = 0; rt < RT; ++rt) acc[rt][ct] = times(uo[rt], wo, acc[rt][ct]);
        }
      if (more) stage.put(lds[(fb + 1) & 1], tid);
      __syncthreads();
    }
  }
  float* tile = (float*)lds_raw + w * 16 * (W + 4);
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    rho[rt] += __shfl_xor(rho[rt], 16);
    rho[rt] += __shfl_xor(rho[rt], 32);
    f32x4 rho_row;                   // of row 4 g + r, with the factor of the row term's gradient
#pragma unroll
    for (int r = 0; r < 4; ++r) rho_row[r] = __shfl(rho[rt], 4 * g + r) * a.f.scale2;
#pragma unroll
    for (int ct = 0; ct < CT; ++ct)
      if (16 * ct < d) {
        acc[rt][ct] *= kLn2;
        if (a.side == 1 && a.f.dense) {
          f32x4 q = {0.f, 0.f, 0.f, 0.f};
          const uint16_t* img = (const uint16_t*)(set + a.f.p.off_csym) + (size_t)ct * steps * 3 * 512;
#pragma unroll
          for (int s = 0; s < S; ++s)
            if (s < steps) q = times(x[rt][s], image_op<3>(img + s * 3 * 512, lane), q);
#pragma unroll
          for (int r = 0; r < 4; ++r) acc[rt][ct][r] += rho_row[r] * q[r];
        }
      }
    tile_to_lds<W>(tile, acc[rt], lane);
    for (int u = lane; u < 16 * (W / 8); u += 64) {
      const int r = u / (W / 8), c0 = 8 * (u % (W / 8)), vr = v0 + 16 * rt + r;
      const float rho_r = __shfl(rho[rt], r & 15) * a.f.scale2;      // (every lane takes part: 16 W / 8 units are whole waves or W = 32's one)
      if (vr >= rows || c0 >= d) continue;
      const RowAt at = row_at(a.x, vr);
      const long long base = row_base(a.dx, b, h * a.x.G + at.head, at.row);
      f32x8 y = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
      if (slot >= 0 && at.row < len) {
        if (a.side == 1 && !a.f.dense) {       // C2 + C2' = -I, onto the tile itself: the numbers of a pair meet when they are turned back
          const f32x8 xs = row8(a.x, b, h, at, c0);
#pragma unroll
          for (int i = 0; i < 8; ++i) tile[r * (W + 4) + c0 + i] -= rho_r * xs[i];
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = tile[r * (W + 4) + c0 + i];
      }
      if (a.x.turn.rot == 0) store8(a.dx, base, c0, d, y);
    }
    __builtin_amdgcn_wave_barrier();
    asm volatile("" ::: "memory");
    if (a.x.turn.rot > 0)
      for (int u = lane; u < 16 * (W / 8); u += 64) {
        const int r = u / (W / 8), c0 = 8 * (u % (W / 8)), vr = v0 + 16 * rt + r;
        if (vr >= rows || c0 >= d) continue;
        const RowAt at = row_at(a.x, vr);
        f32x8 y = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (slot >= 0 && at.row < len) {
          const float* q = tile + r * (W + 4);
          auto eight = [&](int col) {
            f32x8 e;
#pragma unroll
            for (int i = 0; i < 8; ++i) e[i] = q[col + i];
            return e;
          };
          const float2* cs = a.x.turn.table + ((long long)b * a.x.L + at.row) * (a.x.turn.rot >> 1);
          y = turned8(eight(c0), c0, a.x.turn, cs, -1.f, [&](int col) { return q[col]; }, eight);
        }
        store8(a.dx, row_base(a.dx, b, h * a.x.G + at.head, at.row), c0, d, y);
      }
    __builtin_amdgcn_wave_barrier();
    asm volatile("" ::: "memory");
  }
}

int lds_room(const void* kernel, size_t lds) {
  if (lds > 64 * 1024 && hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds) != hipSuccess) {
    (void)hipGetLastError();
    return 5;
  }
  return 0;
}
template <int W, int XP, int NW> int values(const ValueArgs& a, hipStream_t st) {
  constexpr size_t lds = 2 * sizeof(StepLds<W, false>);
  static_assert(lds >= sizeof(float) * NW * 16 * (W + 4), "the waves' tiles of output rows");
  auto kernel = k_values<W, XP, NW>;
  if (int rc = lds_room((const void*)kernel, lds)) return rc;
  hipLaunchKernelGGL(kernel, dim3((a.x.L * a.x.G + 32 * NW - 1) / (32 * NW), a.B * a.Hk), dim3(64 * NW), lds, st, a);
  return hipGetLastError() == hipSuccess ? 0 : 5;
}
template <int W, int XP> int values_nw(const ValueArgs& a, hipStream_t st) {
  return a.x.L * a.x.G > 128 ? values<W, XP, 8>(a, st) : values<W, XP, 4>(a, st);
}
template <int W> int values_pieces(const ValueArgs& a, hipStream_t st) {
  return a.x.X.dtype == 1 && a.x.turn.rot == 0 ? values_nw<W, 1>(a, st) : values_nw<W, 3>(a, st);
}
template <int W, int XP, int RP, int NW> int grads(const GradArgs& a, hipStream_t st) {
  constexpr size_t lds = 2 * sizeof(StepLds<W, true>);
  constexpr int RT = W == 128 ? 1 : 2;
  static_assert(lds >= sizeof(float) * NW * 16 * (W + 4) && lds <= 160 * 1024, "the waves' tiles of output rows; LDS of a CU");
  auto kernel = k_grads<W, XP, RP, NW, RT>;
  if (int rc = lds_room((const void*)kernel, lds)) return rc;
  hipLaunchKernelGGL(kernel, dim3((a.x.L * a.x.G + 16 * RT * NW - 1) / (16 * RT * NW), a.B * a.Hk), dim3(64 * NW), lds, st, a);
  return hipGetLastError() == hipSuccess ? 0 : 5;
}
template <int W, int XP, int RP> int grads_nw(const GradArgs& a, hipStream_t st) {
  return a.x.L * a.x.G > 128 ? grads<W, XP, RP, 8>(a, st) : grads<W, XP, RP, 4>(a, st);
}
template <int W> int grads_pieces(const GradArgs& a, hipStream_t st) {
  if (a.r.X.dtype == 1) return a.x.X.dtype == 1 && a.x.turn.rot == 0 ? grads_nw<W, 1, 1>(a, st) : grads_nw<W, 3, 1>(a, st);
  return grads_nw<W, 3, 3>(a, st);
}

}  // namespace

int launch_values(const ValueArgs& a, hipStream_t st) {
  switch (width_class(a.f.d, a.dv)) {
    case 32: return values_pieces<32>(a, st);
    case 64: return values_pieces<64>(a, st);
    default: return values_pieces<128>(a, st);
  }
}
int launch_grads(const GradArgs& a, hipStream_t st) {
  switch (width_class(a.f.d, a.dv)) {
    case 32: return grads_pieces<32>(a, st);
    case 64: return grads_pieces<64>(a, st);
    default: return grads_pieces<128>(a, st);
  }
}

}  // namespace st
}  // namespace fs
