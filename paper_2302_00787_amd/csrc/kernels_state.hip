// States of sequences: the projection constants they are built and read with, sums over rows (keys and values onto a state; the gradient of
// a state), and the join of partial sums.
//
// k_build: a workgroup takes a part of the rows 32 at a time; its waves have 16 or 32 features each, whose rows of W and of the sum stay in
// registers.  Rows are read, turned and split into pieces once for all waves.  The exponents come out feature by lane and row by
// register: two stacked tiles are, without a move, the operand of the sum over rows.  A wave has a reference of its own,
// raised when an exponent passes it by 2^16 (never after the first rows, as a rule): features lie up to 2^8 above one at first, so that
// those far below the largest still split into whole pieces.  Vector instructions (exponentials, pieces) and matrix instructions share the
// SIMDs' issue and bound it: 64 states of up to 4096 rows, 64 x 256, bf16: 35 us, turned on the way 57, of which the bytes need 10.
#include <algorithm>
#include <type_traits>

#include "state_common.h"

namespace fs {
namespace st {
namespace {

// ---------------------------------------------------------------------------------------------- projection constants
// Sums in 64 bits: the constants are made once and used for every row.
__device__ __forceinline__ void split2_store(uint16_t* at, size_t piece_stride, float v) {
  const _Float16 h = (_Float16)v, m = (_Float16)(v - (float)h);
  at[0] = __builtin_bit_cast(uint16_t, h);
  at[piece_stride] = __builtin_bit_cast(uint16_t, m);
}
__device__ __forceinline__ float block_max(float v, float* tmp) {         // of 256 threads
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) tmp[threadIdx.x >> 6] = v;
  __syncthreads();
  return fmaxf(fmaxf(tmp[0], tmp[1]), fmaxf(tmp[2], tmp[3]));
}
__global__ void __launch_bounds__(256) k_prepare(const float* theta, int groups, const float* Omega, int omega_groups, int d, int M, float scale,
                                                 char* buf, FeaturePlan p) {
  __shared__ float om[32][128], wv[32][128], tmp[4];
  const int blk = blockIdx.x, side = blockIdx.y, set = blockIdx.z, tid = threadIdx.x, n = 32 * p.steps;
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
  float most = 0.f;
  for (int i = tid; i < 32 * n; i += 256) {
    const int f = i / n, c = i - f * n, tile = f >> 4, r = f & 15;
    double sum = 0.0;
    if (c < d)
      for (int l = 0; l < d; ++l) sum += (double)om[f][l] * (double)Bm[(size_t)l * d + c];
    const float v = (float)(sum * (double)scale * 1.4426950408889634074);
    wv[f][c] = v;
    most = fmaxf(most, fabsf(v));
    split3_store(col + ((size_t)blk * p.tiles + (c >> 4)) * 3 * 512 + (r / 4 * 16 + (c & 15)) * 8 + 4 * tile + (r & 3), 512, v);
  }
  const float up = up_to_2_14(block_max(most, tmp));
  for (int i = tid; i < 32 * n; i += 256) {
    const int f = i / n, c = i - f * n, tile = f >> 4, r = f & 15;
    split2_store(row + ((size_t)blk * p.steps + (c >> 5)) * 2 * 1024 + tile * 512 + ((c & 31) / 8 * 16 + r) * 8 + (c & 7), 1024, wv[f][c] * up);
  }
  if (tid == 0) ((float*)(base + p.off_scale[side]))[blk] = power_inverse(up);
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
    most = 0.f;
    for (int i = tid; i < (int)dd; i += 256) {
      const int a = i / d, c = i - a * d;
      most = fmaxf(most, fabsf(C2[i] + C2[(size_t)c * d + a]));
    }
    const float cup = up_to_2_14(block_max(most, tmp));
    for (int i = tid; i < n * n; i += 256) {
      const int a = i / n, c = i - a * n;
      const float v = a < d && c < d ? C2[(size_t)a * d + c] + C2[(size_t)c * d + a] : 0.f;
      split2_store(csym + ((size_t)(c >> 4) * p.steps + (a >> 5)) * 2 * 512 + ((a & 31) / 8 * 16 + (c & 15)) * 8 + (a & 7), 512, v * cup);
    }
    if (tid == 0) {
      *(float*)(base + p.off_cscale) = power_inverse(cup);
      if (((int)th[2] & 1) == 0) atomicOr((unsigned*)buf, 1u);
    }
  }
}

// ---------------------------------------------------------------------------------------------- row terms
// x' C2 x = x' (C2 + C2') x / 2 of sixteen rows a workgroup on matrix instructions, for dense quadratic forms.  A wave has sixteen coordinates of the
// product, or twice that, and brings their part of the form while the rows are on their way: the call is the latency of both.  (6000
// rows of 128: 14 us where a wave took all coordinates, one after the other, 7.1 so.)
template <int W>
__global__ void __launch_bounds__(W == 32 ? 128 : 256) k_row_terms(Features f, Rows x, int Hk, float* terms) {
  constexpr int S = STEPS<W>, NW = W == 32 ? 2 : 4, CT = 2 * S / NW;
  __shared__ __align__(16) float rows[NW][16][W + 4];
  __shared__ float parts[NW][16];
  const int bh = blockIdx.y, b = bh / Hk, h = bh - b * Hk, lane = threadIdx.x & 63, w = threadIdx.x >> 6, g = lane >> 4, c = lane & 15;
  const int v0 = 16 * (blockIdx.x + (blockIdx.z << 20)), row = v0 + c, len = length_of(x, b), at = min(row, x.L - 1);
  if (v0 >= x.L) return;
  const char* set = f.set(h);
  const long long base = row_base(x.X, b, h, at);
  RowUnits<S, false, true> units;
  units.fetch(x.X, base, x.cols, x.turn, g);
  Op16<2> form[CT][S];
#pragma unroll
  for (int i = 0; i < CT; ++i)
#pragma unroll
    for (int s = 0; s < S; ++s)                  // (behind d the row is zeros)
#pragma unroll
      for (int p = 0; p < 2; ++p)
        form[i][s].p[p] = *(const f16x8*)((const uint16_t*)(set + f.p.off_csym) + (size_t)min(w + NW * i, f.p.tiles - 1) * f.p.steps * 1024 +
                                          (min(s, f.p.steps - 1) * 2 + p) * 512 + lane * 8);
  const float undo = *(const float*)(set + f.p.off_cscale);
  f32x8 n[S];
  units.finish(x.X, base, x.cols, x.turn, x.turn.table + ((long long)b * x.L + at) * (x.turn.rot >> 1), row < len, g, n);
  float most = 0.f, sum = 0.f;
#pragma unroll
  for (int s = 0; s < S; ++s) most = fmaxf(most, largest_of(n[s]));
  most = fmaxf(most, __shfl_xor(most, 16));
  most = fmaxf(most, __shfl_xor(most, 32));
  const float scale = up_to_2_14(most);
  Op16<2> xo[S];
#pragma unroll
  for (int s = 0; s < S; ++s) {
    xo[s] = as_op16<2>(n[s] * scale);
    *(f32x4*)&rows[w][c][32 * s + 8 * g] = f32x4{n[s][0], n[s][1], n[s][2], n[s][3]};
    *(f32x4*)&rows[w][c][32 * s + 8 * g + 4] = f32x4{n[s][4], n[s][5], n[s][6], n[s][7]};
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < CT; ++i) {
    f32x4 q = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int s = 0; s < S; ++s) each_product<2, 2>([&](int j, int k) { q = mfma(form[i][s].p[j], xo[s].p[k], q); });
    const f32x4 y = *(const f32x4*)&rows[w][c][16 * (w + NW * i) + 4 * g];
#pragma unroll
    for (int r = 0; r < 4; ++r) sum += q[r] * y[r];
  }
  sum += __shfl_xor(sum, 16);
  sum += __shfl_xor(sum, 32);
  parts[w][c] = sum;
  __syncthreads();
  if (w > 0 || g > 0 || row >= x.L) return;
  sum = 0.f;
#pragma unroll
  for (int i = 0; i < NW; ++i) sum += parts[i][c];
  terms[(size_t)bh * x.L + row] = row < len ? 0.5f * kLog2e * f.scale2 * power_inverse(scale) * undo * sum : kNone;
}

// ---------------------------------------------------------------------------------------------- sums over rows
template <int W, int XP, int VP> struct BuildLds {
  uint16_t x[2][XP][32][W + 8];
  uint16_t v[2][VP][32][W + 8];
  float term[2][32], weight[2][32], undo[2][32];
};

// Four numbers of a row (columns c0 ..), their partners and angles, on their way to LDS: as they lie, so that nothing waits for them before they are
// put there.  TURN = false: numbers alone.
template <bool FULL, bool TURN> struct Four {
  u32x4 x, p;
  f32x4 cs[TURN ? 2 : 1];
  __device__ __forceinline__ static u32x4 bits(const TensorDev& t, long long base, int c, int cols) {
    u32x4 v = {0u, 0u, 0u, 0u};
    if (FULL || c + 4 <= cols) {
      if (t.dtype == 0) {
        v = *(const u32x4*)((const float*)t.ptr + base + c);
      } else {
        const u32x2 u = *(const u32x2*)((const uint16_t*)t.ptr + base + c);
        v[0] = u[0];
        v[1] = u[1];
      }
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (c + i < cols) v[i] = t.dtype == 0 ? ((const uint32_t*)t.ptr)[base + c + i] : (uint32_t)((const uint16_t*)t.ptr)[base + c + i];
    }
    return v;
  }
  __device__ __forceinline__ static f32x4 numbers(u32x4 v, int dtype, int c, int cols) {
    if (dtype == 0) return __builtin_bit_cast(f32x4, v);
    if (!FULL && c + 4 > cols) return f32x4{__uint_as_float(v[0] << 16), __uint_as_float(v[1] << 16), __uint_as_float(v[2] << 16), 0.f};
    return f32x4{__uint_as_float(v[0] << 16), __uint_as_float(v[0] & 0xffff0000u), __uint_as_float(v[1] << 16), __uint_as_float(v[1] & 0xffff0000u)};
  }
  __device__ __forceinline__ void none() { x = u32x4{0u, 0u, 0u, 0u}; }
  // base: the row's first number; a: its angles
  __device__ __forceinline__ void get(const Rows& r, long long base, const float2* a, int c0) {
    none();
    if (!FULL && c0 >= r.cols) return;
    x = bits(r.X, base, c0, r.cols);
    if (!TURN || c0 >= r.turn.rot) return;
    const int half = r.turn.rot >> 1;
    if (r.turn.interleaved) {
      const float2 u = a[c0 >> 1], v = a[min((c0 >> 1) + 1, half - 1)];
      cs[0] = f32x4{u.x, u.y, v.x, v.y};
    } else if ((half & 3) == 0) {
      const int i = c0 >= half ? c0 - half : c0;
      p = bits(r.X, base, c0 >= half ? i : c0 + half, r.cols);
      cs[0] = *(const f32x4*)(a + i);
      cs[1] = *(const f32x4*)(a + i + 2);
    } else {                     // (partners one by one)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int c = c0 + i;
        if (c < r.turn.rot) {
          const int k = c >= half ? c - half : c, o = c >= half ? k : c + half;
          p[i] = r.X.dtype == 0 ? ((const uint32_t*)r.X.ptr)[base + o] : (uint32_t)((const uint16_t*)r.X.ptr)[base + o] << 16;
          const float2 u = a[k];
          cs[i >> 1][2 * (i & 1)] = u.x;
          cs[i >> 1][2 * (i & 1) + 1] = u.y;
        }
      }
    }
  }
  __device__ __forceinline__ f32x4 put(const Rows& r, int c0, bool live) const {
    const f32x4 v = numbers(x, r.X.dtype, c0, r.cols);
    if (!TURN || !live || c0 >= r.turn.rot) return v;
    const int half = r.turn.rot >> 1;
    f32x4 y = v;
    if (r.turn.interleaved) {
      y[0] = v[0] * cs[0][0] - v[1] * cs[0][1];
      y[1] = v[1] * cs[0][0] + v[0] * cs[0][1];
      if (c0 + 2 < r.turn.rot) {
        y[2] = v[2] * cs[0][2] - v[3] * cs[0][3];
        y[3] = v[3] * cs[0][2] + v[2] * cs[0][3];
      }
    } else {
      const bool quad = (half & 3) == 0;
      const f32x4 q = quad ? numbers(p, r.X.dtype, c0, r.turn.rot) : __builtin_bit_cast(f32x4, p);
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (quad || c0 + i < r.turn.rot)
          y[i] = v[i] * cs[i >> 1][2 * (i & 1)] + q[i] * (c0 + i >= half ? cs[i >> 1][2 * (i & 1) + 1] : -cs[i >> 1][2 * (i & 1) + 1]);
    }
    return y;
  }
};

// How the rows of a call are shared out.  Chunks of 32 rows, head by head and sequence by sequence, are one line that `nwg` workgroups cut into
// equal pieces, so that a padded batch keeps all of them busy alike; what a workgroup sums of one state is a part, number (workgroup +
// states before).  nwg = 0: a workgroup and a part for every state.
struct Shares {
  const Rows& x;
  const int32_t* slots;
  int nslots, B, Hk, nwg;
  __device__ __forceinline__ int rows_of(int b) const {
    const int len = slot_of(slots, nslots, b) < 0 ? 0 : length_of(x, b);
    return x.G == 1 || len == 0 ? len : x.L * x.G;
  }
  __device__ __forceinline__ int chunks_of(int b) const { return (rows_of(b) + 31) / 32; }
  __device__ __forceinline__ static int scan(int v, int lane) {
#pragma unroll
    for (int o = 1; o < 64; o *= 2) {
      const int t = __shfl_up(v, o);
      if (lane >= o) v += t;
    }
    return v;
  }
  // chunks of the sequences before b of one head (b = B: of all); each wave for itself
  __device__ __forceinline__ long long before(int b, int lane) const {
    long long sum = 0;
    for (int b0 = 0; b0 < b; b0 += 64) sum += __builtin_amdgcn_readlane(scan(b0 + lane < b ? chunks_of(b0 + lane) : 0, lane), 63);
    return sum;
  }
  // the sequence of chunk q of a head, and the chunks before it
  __device__ __forceinline__ int find(long long q, int lane, long long* first) const {
    long long sum = 0;
    for (int b0 = 0;; b0 += 64) {
      const int n = b0 + lane < B ? chunks_of(b0 + lane) : 0, upto = scan(n, lane);
      const unsigned long long behind = __ballot(sum + upto > q);
      if (behind != 0ull || b0 + 64 >= B) {
        const int l = behind != 0ull ? __builtin_ctzll(behind) : 63;
        *first = sum + __builtin_amdgcn_readlane(upto - n, l);
        return b0 + l;
      }
      sum += __builtin_amdgcn_readlane(upto, 63);
    }
  }
  __device__ __forceinline__ static long long start(long long i, long long total, long long n) { return i * total / n; }
};

// ONE: rows of fours of known type, turned in halves, fours whole, or (TURN = false) not at all: their way to LDS is without a branch (a chunk's loads
// take 1100 cycles of a wave where their addresses and conditions are found one by one).
template <int W, int XP, int VP, int NW, int FT, bool FULL, bool ONE, bool TURN>
__device__ __forceinline__ void build_part(const BuildArgs& a, BuildLds<W, XP, VP>& lds, int b, int h, int v0, int v1, size_t part) {
  // a row's numbers in fours: N of x and N of v for a thread, or of one of them where there are threads for both (APART)
  constexpr int S = STEPS<W>, VT = TILES<W>, UPR = W / 4, NTH = 64 * NW, ROWS = (NTH < 32 * UPR ? NTH : 32 * UPR) / UPR, N = 32 / ROWS, LD = W + 8;
  constexpr bool APART = NTH >= 64 * UPR;
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), g = lane >> 4, c = lane & 15;
  const int bh = b * a.Hk + h, tile = (blockIdx.y * NW + w) * FT, ntiles = a.f.p.Mp / 16, steps = FULL ? S : a.f.p.steps, dv = FULL ? W : a.dv;
  const int len = length_of(a.x, b), rows = a.x.L * a.x.G;
  const bool active = tile < ntiles;
  const char* set = a.f.set(h);
  Four<FULL, XP == 2> next_x[N];
  Four<FULL, false> next_v[N];
  bool next_live[N];
  float next_term[N], next_weight[N];
  const float *terms = a.terms ? a.terms + (size_t)bh * rows : nullptr, *weights = a.weights ? a.weights + (size_t)bh * rows : nullptr;
  const int row0 = (APART ? tid % (32 * UPR) : tid) / UPR, c0 = 4 * (tid % UPR);
  const bool do_x = !APART || w < UPR / 2, do_v = !APART || (w >= UPR / 2 && w < UPR);       // (32 UPR threads are UPR / 2 waves)
  auto fetch = [&](int v) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int row = row0 + ROWS * i;
      next_x[i].none();
      next_v[i].none();
      next_live[i] = false;
      next_term[i] = kNone;
      next_weight[i] = 0.f;
      if (v + row >= v1) continue;
      const RowAt at = row_at(a.x, v + row);
      if (at.row >= len) continue;
      next_live[i] = true;
      if (do_x) next_x[i].get(a.x, row_base(a.x.X, b, h * a.x.G + at.head, at.row), a.x.turn.table + ((long long)b * a.x.L + at.row) * (a.x.turn.rot >> 1), c0);
      if (do_v) next_v[i].get(a.v, row_base(a.v.X, b, h * a.v.G + at.head, at.row), nullptr, c0);
      next_term[i] = terms ? terms[v + row] : 0.f;
      next_weight[i] = weights ? weights[v + row] : 1.f;
    }
  };
  // (ONE)
  constexpr int DT = VP == 1 ? 1 : 0;
  typedef typename std::conditional<DT == 1, u32x2, u32x4>::type quad;
  quad one_x[N], one_p[N], one_v[N];
  f32x4 one_cs[N][2];
  const int half = a.x.turn.rot >> 1;            // (a multiple of 4: fours are turned whole)
  const bool turned = c0 < 2 * half;
  // (fours behind the end of a row are its last one, and put as zeros)
  const int xc = FULL ? c0 : min(c0, a.f.d - 4), vc = FULL ? c0 : min(c0, dv - 4);
  const bool in_x = FULL || c0 < a.f.d, in_v = FULL || c0 < dv;
  const int other0 = c0 < half ? c0 + half : turned ? c0 - half : xc, pair0 = c0 < half ? c0 : turned ? c0 - half : 0;
  const float sgn = c0 < half ? -1.f : turned ? 1.f : 0.f;
  const float *one_t = terms ? terms : (const float*)a.f.base, *one_w = weights ? weights : (const float*)a.f.base;
  const int t_step = terms ? 1 : 0, w_step = weights ? 1 : 0;
  const char *xp = (const char*)a.x.X.ptr, *vp = (const char*)a.v.X.ptr;
  const long long x0 = row_base(a.x.X, b, h * a.x.G, 0), y0 = row_base(a.v.X, b, h * a.v.G, 0);
  const float2* cs0 = half > 0 ? a.x.turn.table + (long long)b * a.x.L * half : (const float2*)a.f.base;
  auto fetch_one = [&](int v) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int mine = v + row0 + ROWS * i, at = min(mine, v1 - 1);          // (rows behind the last one are it, and put as zeros)
      constexpr int E = DT == 1 ? 2 : 4;
      long long xo = x0 + xc, vo = y0 + vc;
      int row = at;
      if (a.x.G > 1) {
        const int head = at / a.x.L;
        row -= head * a.x.L;
        xo += head * a.x.X.sh;
        vo += head * a.v.X.sh;
      }
      next_live[i] = mine < v1 && row < len;
      xo += row * a.x.X.sl;
      vo += row * a.v.X.sl;
      if (do_v) one_v[i] = *(const quad*)(vp + vo * E);
      if (do_x) {
        one_x[i] = *(const quad*)(xp + xo * E);
        if constexpr (TURN) {
          one_p[i] = *(const quad*)(xp + (xo - xc + other0) * E);
          const f32x4* cs = (const f32x4*)(cs0 + (long long)row * half + pair0);
          one_cs[i][0] = cs[0];
          one_cs[i][1] = cs[1];
        }
        next_term[i] = one_t[at * t_step];
        next_weight[i] = one_w[at * w_step];
      }
    }
  };
  auto numbers = [](quad q) {
    if constexpr (DT == 1)
      return f32x4{__uint_as_float(q[0] << 16), __uint_as_float(q[0] & 0xffff0000u), __uint_as_float(q[1] << 16), __uint_as_float(q[1] & 0xffff0000u)};
    else return __builtin_bit_cast(f32x4, q);
  };
  auto put = [&](int buf) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int row = row0 + ROWS * i, u = tid % UPR;
      const bool live = next_live[i];
      if (do_x) {
        f32x4 x;
        if constexpr (ONE) {
          x = numbers(one_x[i]);
          if constexpr (TURN) {
            const f32x4 p = numbers(one_p[i]) * sgn;
            f32x4(&cs)[2] = one_cs[i];
#pragma unroll
            for (int j = 0; j < 2; ++j) cs[j][0] = turned ? cs[j][0] : 1.f, cs[j][2] = turned ? cs[j][2] : 1.f;
            x = f32x4{x[0] * one_cs[i][0][0] + p[0] * one_cs[i][0][1], x[1] * one_cs[i][0][2] + p[1] * one_cs[i][0][3],
                      x[2] * one_cs[i][1][0] + p[2] * one_cs[i][1][1], x[3] * one_cs[i][1][2] + p[3] * one_cs[i][1][3]};
          }
#pragma unroll
          for (int j = 0; j < 4; ++j) x[j] = live && in_x ? x[j] : 0.f;
        } else {
          x = next_x[i].put(a.x, 4 * u, live);
        }
        const float most = over_lanes<UPR>(fmaxf(fmaxf(fabsf(x[0]), fabsf(x[1])), fmaxf(fabsf(x[2]), fabsf(x[3]))), [](float p, float q) { return fmaxf(p, q); });
        const float n = over_lanes<UPR>(x[0] * x[0] + x[1] * x[1] + (x[2] * x[2] + x[3] * x[3]), [](float p, float q) { return p + q; });
        const float scale = up_to_2_14(most);
        const Op16<XP> o = as_op16<XP>(f32x8{x[0], x[1], x[2], x[3], 0.f, 0.f, 0.f, 0.f} * scale);
#pragma unroll
        for (int p = 0; p < XP; ++p) {
          const u32x4 bits = __builtin_bit_cast(u32x4, o.p[p]);
          *(u32x2*)&lds.x[buf][p][row][4 * u] = u32x2{bits[0], bits[1]};
        }
        if (u == 0) {
          const float t = a.terms ? next_term[i] : -0.5f * kLog2e * a.f.scale2 * n;        // (C2 = -I / 2)
          lds.term[buf][row] = live ? t : kNone;
          lds.weight[buf][row] = a.weights ? next_weight[i] : 1.f;
          lds.undo[buf][row] = power_inverse(scale);
        }
      }
      if (!do_v) continue;
      if constexpr (ONE) {
        quad q = one_v[i];
#pragma unroll
        for (int j = 0; j < (DT == 1 ? 2 : 4); ++j) q[j] = live && in_v ? q[j] : 0u;
        if constexpr (DT == 1) {
          *(u32x2*)&lds.v[buf][0][row][4 * u] = q;
        } else {
          const f32x4 y = numbers(q);
          const Op<VP> o3 = as_op<VP>(f32x8{y[0], y[1], y[2], y[3], 0.f, 0.f, 0.f, 0.f});
#pragma unroll
          for (int p = 0; p < VP; ++p) {
            const u32x4 bits = __builtin_bit_cast(u32x4, o3.p[p]);
            *(u32x2*)&lds.v[buf][p][row][4 * u] = u32x2{bits[0], bits[1]};
          }
        }
      } else if (VP == 1 && (FULL || 4 * u + 4 <= dv)) {
        *(u32x2*)&lds.v[buf][0][row][4 * u] = u32x2{next_v[i].x[0], next_v[i].x[1]};
      } else {
        const f32x4 y = next_v[i].put(a.v, 4 * u, false);
        const Op<VP> q = as_op<VP>(f32x8{y[0], y[1], y[2], y[3], 0.f, 0.f, 0.f, 0.f});
#pragma unroll
        for (int p = 0; p < VP; ++p) {
          const u32x4 bits = __builtin_bit_cast(u32x4, q.p[p]);
          *(u32x2*)&lds.v[buf][p][row][4 * u] = u32x2{bits[0], bits[1]};
        }
      }
    }
  };

  auto bring = [&](int v) {
    if constexpr (ONE) fetch_one(v);
    else fetch(v);
  };
  bring(v0);
  Op16<2> wop[S][FT];
  float bias[FT], wscale = 0.f;
  if (active) {
    const uint16_t* img = (const uint16_t*)(set + a.f.p.off_row[a.side]) + (size_t)(tile >> 1) * steps * 2 * 1024 + (tile & 1) * 512;
#pragma unroll
    for (int s = 0; s < S; ++s)
      if (FULL || s < steps)
#pragma unroll
        for (int ft = 0; ft < FT; ++ft)
#pragma unroll
          for (int p = 0; p < 2; ++p) wop[s][ft].p[p] = *(const f16x8*)(img + (s * 2 + p) * 1024 + ft * 512 + lane * 8);
#pragma unroll
    for (int ft = 0; ft < FT; ++ft) bias[ft] = ((const float*)(set + a.f.p.off_bias))[16 * (tile + ft) + c];
    wscale = ((const float*)(set + a.f.p.off_scale[a.side]))[tile >> 1];
  }
  f32x4 T[FT][VT];
  float z[FT], ref = 0.f, top = kNone;
  bool referred = false;
#pragma unroll
  for (int ft = 0; ft < FT; ++ft)
#pragma unroll
    for (int vt = 0; vt < VT; ++vt) T[ft][vt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int ft = 0; ft < FT; ++ft) z[ft] = 0.f;
  put(0);
  __syncthreads();
  int buf = 0;
  for (int v = v0; v < v1; v += 32, buf ^= 1) {
    const bool more = v + 32 < v1;
    if (more) bring(v + 32);
    if (active) {
      f32x4 E[2][FT];            // [tile of rows][tile of features]
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int ft = 0; ft < FT; ++ft) E[t][ft] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int s = 0; s < S; ++s)
        if (FULL || s < steps) {
          Op16<XP> x[2];
#pragma unroll
          for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int p = 0; p < XP; ++p) x[t].p[p] = *(const f16x8*)&lds.x[buf][p][16 * t + c][32 * s + 8 * g];
          outer(x, wop[s], E);
        }
      f32x4 weight[2];
      float most = kNone;
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const f32x4 term = *(const f32x4*)&lds.term[buf][16 * t + 4 * g], undo = *(const f32x4*)&lds.undo[buf][16 * t + 4 * g] * wscale;
        weight[t] = *(const f32x4*)&lds.weight[buf][16 * t + 4 * g];
#pragma unroll
        for (int ft = 0; ft < FT; ++ft)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            E[t][ft][r] = E[t][ft][r] * undo[r] + (bias[ft] + (term[r] - ref));
            most = fmaxf(most, E[t][ft][r]);
          }
      }
      top = fmaxf(top, ref + most);
      if (__any(most > 16.f || (!referred && most > kNone))) {
        float m = most;
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
        const float up = m - 8.f, keep = referred ? fast_exp2(-up) : 0.f;
        ref += up;
        referred = true;
#pragma unroll
        for (int ft = 0; ft < FT; ++ft) {
          z[ft] *= keep;
#pragma unroll
          for (int vt = 0; vt < VT; ++vt) T[ft][vt] *= keep;
#pragma unroll
          for (int t = 0; t < 2; ++t) E[t][ft] -= up;
        }
      }
      Op<3> so[FT];
#pragma unroll
      for (int ft = 0; ft < FT; ++ft) {
        f32x8 sv;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const float x = fast_exp2(E[t][ft][r]);
            sv[4 * t + r] = x;
            z[ft] += x * weight[t][r];
          }
        so[ft] = as_op<3>(sv);
      }
#pragma unroll
      for (int vt = 0; vt < VT; vt += 2)
        if (FULL || 16 * vt < dv) {
          const uint16_t* at_v = &lds.v[buf][0][0][16 * vt] + lane_tr(lane, LD);
          const Op<VP> vo[2] = {column_op<VP>(at_v, LD, 32 * LD), column_op<VP>(at_v + 16, LD, 32 * LD)};
          outer_at(so, vo, T, vt);
        }
    }
    if (more) put(buf ^ 1);
    __syncthreads();
  }
  if (!active) return;
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
  // (maxima pass over what is not a number: a row that is none must not pass for one that is not there)
  bool no_number = false;
#pragma unroll
  for (int ft = 0; ft < FT; ++ft) no_number |= z[ft] != z[ft];
  if (__any(no_number)) ref = top = kNoNumber;
  if (lane < FT) a.refs[part * ntiles + tile + lane] = make_float2(ref, top);
#pragma unroll
  for (int ft = 0; ft < FT; ++ft) {
    const int m0 = 16 * (tile + ft);
    float zs = z[ft];
    zs += __shfl_xor(zs, 16);
    zs += __shfl_xor(zs, 32);
    if (g == 0 && m0 + c < a.f.M) a.zpart[part * a.f.M + m0 + c] = zs;
#pragma unroll
    for (int vt = 0; vt < VT; ++vt)
      if (FULL || 16 * vt + c < dv)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (m0 + 4 * g + r < a.f.M) a.part[(part * a.f.M + m0 + 4 * g + r) * dv + 16 * vt + c] = T[ft][vt][r];
  }
}

template <int W, int XP, int VP, int NW, int FT, bool FULL, bool ONE, bool TURN>
__global__ void __launch_bounds__(64 * NW) k_build(BuildArgs a) {
  extern __shared__ __align__(16) char lds_raw[];
  BuildLds<W, XP, VP>& lds = *(BuildLds<W, XP, VP>*)lds_raw;
  const int lane = threadIdx.x & 63;
  const Shares shares{a.x, a.slots, a.nslots, a.B, a.Hk, a.nwg};
  // the state's shift as it is before the call, for the join, by whoever has its first rows
  auto keep_shift = [&](int b, int h) {
    if (a.old_shift != nullptr && blockIdx.y == 0 && threadIdx.x == 0) {
      const int slot = slot_of(a.slots, a.nslots, b);
      a.old_shift[b * a.Hk + h] = slot >= 0 ? a.shift[(size_t)slot * a.Hk + h] : kNone;
    }
  };
  if (a.nwg == 0) {
    const int b = blockIdx.x / a.Hk, h = blockIdx.x - b * a.Hk, rows = shares.rows_of(b);
    keep_shift(b, h);
    if (blockIdx.y == 0 && threadIdx.x == 0) a.parts[blockIdx.x] = make_int2(blockIdx.x, rows > 0 ? 1 : 0);
    if (rows > 0) build_part<W, XP, VP, NW, FT, FULL, ONE, TURN>(a, lds, b, h, 0, rows, blockIdx.x);
    return;
  }
  const long long C = shares.before(a.B, lane), total = C * a.Hk, n = min((long long)a.nwg, total);
  // the parts of the states, for the join
  if (blockIdx.y == 0 && threadIdx.x >= 64 * (NW - 1))
    for (int bh = blockIdx.x; bh < a.B * a.Hk; bh += gridDim.x) {
      const int b = bh / a.Hk, h = bh - b * a.Hk;
      const long long S = h * C + shares.before(b, lane), mine = shares.chunks_of(b);
      const long long i0 = mine > 0 ? ((S + 1) * n - 1) / total : 0, i1 = mine > 0 ? ((S + mine) * n - 1) / total : -1;
      if (lane == 0) a.parts[bh] = make_int2((int)(i0 + (long long)h * a.B + b), (int)(i1 - i0 + 1));
    }
  if ((long long)blockIdx.x >= n) return;
  long long q = Shares::start(blockIdx.x, total, n);
  const long long end = Shares::start((long long)blockIdx.x + 1, total, n);
  while (q < end) {
    const int h = (int)(q / C);
    long long first;
    const int b = shares.find(q - h * C, lane, &first);
    const long long at = q - h * C - first, here = min(end - q, shares.chunks_of(b) - at);
    if (at == 0) keep_shift(b, h);
    build_part<W, XP, VP, NW, FT, FULL, ONE, TURN>(a, lds, b, h, (int)(32 * at), min((int)(32 * (at + here)), shares.rows_of(b)),
                                                  (size_t)blockIdx.x + (size_t)h * a.B + b);
    q += here;
  }
}

// ---------------------------------------------------------------------------------------------- join
// x += the parts' numbers, from their references to `top`: eight loads on their way at a time.  HIGH: references can be more than 2^127 above `top` and
// the products still be numbers, or zeros.
template <bool HIGH, class V>
__device__ __forceinline__ void sum_parts(V& x, const V* from, size_t stride, int n, const float2* refs, int ref_stride, float top) {
  for (int s0 = 0; s0 < n; s0 += 8) {
    V v[8];
    float2 ref[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      v[i] = from[(size_t)min(s0 + i, n - 1) * stride];
      ref[i] = refs[min(s0 + i, n - 1) * ref_stride];
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float up = ref[i].x - top;
      const bool high = HIGH && up > 64.f;
      const float k = s0 + i < n && ref[i].y != kNone ? fast_exp2(high ? 64.f : up) : 0.f;
      if (k != 0.f) x += HIGH ? (high ? fast_exp2(up - 64.f) : 1.f) * (k * v[i]) : k * v[i];
    }
  }
}

template <int VEC>
__global__ void __launch_bounds__(256) k_join(JoinArgs a) {
  __shared__ float tmp[4];
  typedef __attribute__((ext_vector_type(VEC))) float vec;
  const int bh = blockIdx.y, b = bh / a.Hk, h = bh - b * a.Hk, tid = threadIdx.x, nfb = a.Mp / 16;
  const int slot = unique_slot_of(a.slots, a.state.slots, b);
  if (slot < 0) {
    if (blockIdx.x == 0 && h == 0 && tid == 0 && a.left_out != nullptr) atomicAdd(a.left_out, 1);
    return;
  }
  const size_t part = a.parts[bh].x;
  const int parts = a.parts[bh].y;
  if (parts == 0 && a.old_shift != nullptr) return;              // nothing was appended: the state is what it was
  const float2* refs = a.refs + part * nfb;
  const float old = a.old_shift ? a.old_shift[bh] : kNone;
  float top = old;
  bool no_number = old != old;
  for (int i = tid; i < parts * nfb; i += 256) {
    const float part_top = refs[i].y;
    top = fmaxf(top, part_top);
    no_number |= part_top != part_top;
  }
  top = block_max(top, tmp);
  if (__syncthreads_or(no_number)) top = kNoNumber;              // (and with it all of the state)
  const float keep = old == kNone ? 0.f : fast_exp2(old - top);
  const size_t at = (size_t)slot * a.Hk + h;
  const int nt = a.M * a.dv / VEC;
  for (int e = blockIdx.x * 256 + tid; e < nt + a.M; e += gridDim.x * 256) {
    if (e < nt) {
      const int m = e * VEC / a.dv, fb = m >> 4;
      vec* to = (vec*)(a.state.T + at * a.M * a.dv) + e;
      vec x = {};
      if (keep != 0.f) x = keep * *to;
      sum_parts<false>(x, (const vec*)(a.part + part * a.M * a.dv) + e, nt, parts, refs + fb, nfb, top);
      *to = x;
    } else {
      const int m = e - nt, fb = m >> 4;
      float* to = a.state.z + at * a.M + m;
      float x = keep != 0.f ? keep * *to : 0.f;
      sum_parts<false>(x, a.zpart + part * a.M + m, a.M, parts, refs + fb, nfb, top);
      *to = x;
    }
  }
  if (blockIdx.x == 0 && tid == 0) a.state.shift[at] = top;
}

// A workgroup lists a slot's readers, in the sequences' order, once for all of its numbers (each thread looking through the sequences for each number: 8192
// slots of 64 x 256 and as many sequences 98 ms, of which the sums are 1.1).  A slot with more readers than the list holds has them listed a part
// at a time, for every round of numbers again.
template <int VEC>
__global__ void __launch_bounds__(256) k_join_sum(JoinArgs a) {
  typedef __attribute__((ext_vector_type(VEC))) float vec;
  constexpr int LIST = 1024;
  __shared__ int2 readers[LIST];                 // first part, how many
  __shared__ int found[4];
  const int sh = blockIdx.y, slot = sh / a.Hk, h = sh - slot * a.Hk, nfb = a.Mp / 16, nt = a.M * a.dv / VEC, tid = threadIdx.x, w = tid >> 6;
  const int b0 = a.slots ? 0 : slot, b1 = a.slots ? a.B : min(slot + 1, a.B);
  int n = 0;                                     // readers in the list
  // lists those of the sequences from `from` on; the sequence after the last one looked at
  auto list = [&](int from) {
    __syncthreads();                             // (the list before has been read)
    for (n = 0; from < b1 && n + 256 <= LIST; from += 256) {
      const int b = from + tid;
      const bool mine = b < b1 && slot_of(a.slots, a.state.slots, b) == slot;
      const unsigned long long votes = __ballot(mine);
      if ((tid & 63) == 0) found[w] = __popcll(votes);
      __syncthreads();
      int at = n + __popcll(votes & ((1ull << (tid & 63)) - 1ull));
      for (int i = 0; i < 4; ++i) {
        if (i < w) at += found[i];
        n += found[i];
      }
      if (mine) readers[at] = a.parts[b * a.Hk + h];
      __syncthreads();
    }
    return from;
  };
  const int after = list(b0);
  for (int e0 = blockIdx.x * 256; e0 < nt + a.M; e0 += gridDim.x * 256) {
    const int e = e0 + tid, m = e < nt ? e * VEC / a.dv : e - nt, fb = m >> 4;
    vec x = {};
    for (int from = after;; from = list(from)) {
      if (e < nt + a.M)
        for (int i = 0; i < n; ++i) {
          const size_t part = readers[i].x;
          const int parts = readers[i].y;
          if (e < nt) sum_parts<true>(x, (const vec*)(a.part + part * a.M * a.dv) + e, nt, parts, a.refs + part * nfb + fb, nfb, 0.f);
          else {
            float y = x[0];
            sum_parts<true>(y, a.zpart + part * a.M + m, a.M, parts, a.refs + part * nfb + fb, nfb, 0.f);
            x[0] = y;
          }
        }
      if (from >= b1) break;
    }
    if (after < b1) list(b0);
    if (e < nt) ((vec*)(a.state.T + (size_t)sh * a.M * a.dv))[e] = x;
    else if (e < nt + a.M) a.state.z[(size_t)sh * a.M + m] = x[0];
  }
}

template <int W, int XP, int VP, int NW, int FT, bool FULL, bool ONE, bool TURN> int build(const BuildArgs& a, hipStream_t st) {
  constexpr size_t lds = sizeof(BuildLds<W, XP, VP>);
  auto kernel = k_build<W, XP, VP, NW, FT, FULL, ONE, TURN>;
  if (lds > 64 * 1024 && hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds) != hipSuccess) {
    (void)hipGetLastError();
    return 5;
  }
  hipLaunchKernelGGL(kernel, dim3(a.nwg > 0 ? a.nwg : a.B * a.Hk, (a.f.p.Mp / 16 + NW * FT - 1) / (NW * FT)), dim3(64 * NW), lds, st, a);
  return hipGetLastError() == hipSuccess ? 0 : 5;
}
template <int W, int XP, int VP, bool FULL, bool ONE, bool TURN> int build_waves(const BuildArgs& a, hipStream_t st) {
  // sixteen features a wave and sixteen waves, four to a SIMD, where the rows of W and of the sum leave a wave 128 registers; else 32
  if constexpr (W <= 64 && ONE && FULL) return a.f.p.Mp > 64 ? build<W, XP, VP, 16, 1, FULL, ONE, TURN>(a, st) : build<W, XP, VP, 4, 1, FULL, ONE, TURN>(a, st);
  else if constexpr (W <= 64) return a.f.p.Mp > 64 ? build<W, XP, VP, 8, 2, FULL, ONE, TURN>(a, st) : build<W, XP, VP, 4, 1, FULL, ONE, TURN>(a, st);
  else if constexpr (ONE && FULL) return a.f.p.Mp > 128 ? build<W, XP, VP, 8, 2, FULL, ONE, TURN>(a, st) : build<W, XP, VP, 4, 2, FULL, ONE, TURN>(a, st);
  else return build<W, XP, VP, 4, 2, FULL, ONE, TURN>(a, st);
}
template <int W> int build_width(const BuildArgs& a, hipStream_t st) {
  const Turn& t = a.x.turn;
  const bool bf16 = a.x.X.dtype == 1 && a.v.X.dtype == 1, fours = t.rot % 8 == 0 && !t.interleaved;
  if (a.f.d == W && a.dv == W && a.x.X.dtype == a.v.X.dtype && fours) {
    if (bf16) return t.rot == 0 ? build_waves<W, 1, 1, true, true, false>(a, st) : build_waves<W, 2, 1, true, true, true>(a, st);
    return t.rot == 0 ? build_waves<W, 2, 3, true, true, false>(a, st) : build_waves<W, 2, 3, true, true, true>(a, st);
  }
  if (a.f.d % 4 == 0 && a.dv % 4 == 0 && a.x.X.dtype == a.v.X.dtype && fours)
    return bf16 ? build_waves<W, 2, 1, false, true, true>(a, st) : build_waves<W, 2, 3, false, true, true>(a, st);
  return a.v.X.dtype == 1 ? build_waves<W, 2, 1, false, false, true>(a, st) : build_waves<W, 2, 3, false, false, true>(a, st);
}
// Workgroups for a state: one for 256 numbers, up to 64, and 4096 for all states (what a workgroup does first, its state's parts and their
// largest reference, is three loads in a chain: 660 states of 48 x 512, 64 each 65 us, 46 so).
int join_grid(const JoinArgs& a, int vec, int states) {
  return std::max(1, std::min({(a.M * a.dv / vec + a.M + 255) / 256, 64, (4096 + states - 1) / states}));
}

}  // namespace

int launch_build(const BuildArgs& a, hipStream_t st) {
  switch (width_class(a.f.d, a.dv)) {
    case 32: return build_width<32>(a, st);
    case 64: return build_width<64>(a, st);
    default: return build_width<128>(a, st);
  }
}
int launch_join(const JoinArgs& a, hipStream_t st) {
  if (a.dv % 4 == 0) hipLaunchKernelGGL(k_join<4>, dim3(join_grid(a, 4, a.B * a.Hk), a.B * a.Hk), dim3(256), 0, st, a);
  else hipLaunchKernelGGL(k_join<1>, dim3(join_grid(a, 1, a.B * a.Hk), a.B * a.Hk), dim3(256), 0, st, a);
  return hipGetLastError() == hipSuccess ? 0 : 5;
}
int launch_join_sum(const JoinArgs& a, hipStream_t st) {
  if (a.dv % 4 == 0) hipLaunchKernelGGL(k_join_sum<4>, dim3(join_grid(a, 4, a.state.slots * a.Hk), a.state.slots * a.Hk), dim3(256), 0, st, a);
  else hipLaunchKernelGGL(k_join_sum<1>, dim3(join_grid(a, 1, a.state.slots * a.Hk), a.state.slots * a.Hk), dim3(256), 0, st, a);
  return hipGetLastError() == hipSuccess ? 0 : 5;
}
int launch_prepare(const float* theta, int groups, const float* Omega, int omega_groups, int sets, int d, int M, float scale, char* buf,
                   const FeaturePlan& p, hipStream_t st) {
  if (int rc = launch_fill_u32((uint32_t*)buf, 0u, 1, st)) return rc;
  hipLaunchKernelGGL(k_prepare, dim3(p.Mp / 32, 2, sets), dim3(256), 0, st, theta, groups, Omega, omega_groups, d, M, scale, buf, p);
  return hipGetLastError() == hipSuccess ? 0 : 5;
}
int launch_row_terms(const Features& f, const Rows& k, int B, int Hk, float* terms, hipStream_t st) {
  const int n = (k.L + 15) / 16;         // (workgroups times threads of a dimension have 32 bits)
  const dim3 grid(std::min(n, 1 << 20), B * Hk, (n + (1 << 20) - 1) >> 20);
  if (f.d <= 32) hipLaunchKernelGGL(k_row_terms<32>, grid, dim3(128), 0, st, f, k, Hk, terms);
  else if (f.d <= 64) hipLaunchKernelGGL(k_row_terms<64>, grid, dim3(256), 0, st, f, k, Hk, terms);
  else hipLaunchKernelGGL(k_row_terms<128>, grid, dim3(256), 0, st, f, k, Hk, terms);
  return hipGetLastError() == hipSuccess ? 0 : 5;
}

}  // namespace st
}  // namespace fs
