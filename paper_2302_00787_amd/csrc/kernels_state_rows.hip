// Rows against finished states: queries times a state's rows, and the gradients of queries, keys and values.
//
// All of them walk the features 32 at a time.  The exponents come out row by lane and feature by register: two stacked tiles are,
// without a move, the operand of the products with the state (whose columns come from the transposing LDS read) and with W.  The
// state's rows are split into three bf16 pieces, 24 bits, on their way to LDS, for results of either type: the two sums of a gradient of queries, and
// the two terms of V . dT + dz, cancel where values share a mean, and what pieces had lost would stay.
//
// Queries: a feature's T and z are divided by the power of two of its z on their way to LDS, which its exponent gets instead, p_m T_m = (p_m 2^e) (T_m 2^-e):
// so exponents say what a feature contributes, and a row's reference is the largest of those.  A row that reads only what its state holds very
// little of (keys far below the largest) then has a normaliser of 2^7 or more and all bits of T in the pieces, which end at 2^-133.  The reference is
// raised when an exponent passes it by 2^16, which a row's first 32 features as a rule prevent; the quotient loses it.
//
// Many rows (DIRECT = false): a wave takes 16 RT rows of its own through all features, the workgroup brings images of W and the
// state to LDS for all its waves, the next ones on their way meanwhile.  Few rows: the waves of a workgroup take the same rows and a part of the
// features each, with the state in LDS of their own and W in registers, no barrier until their sums meet at the end.
// Vector and matrix instructions on the same SIMDs bound many rows (64 x 256, bf16; vector issue and busy matrix pipes, of a SIMD's cycles: values of
// 262144 queries 84 us, 55 % and 34 %; gradients of 23000 keys of each of 8 heads 97 us, 43 and 39; of 8192 queries of each 41, 42 and 39); loads and
// barriers few rows (1499 keys of 4 heads, 128 x 512, fp32: 57 us).
#include <algorithm>

#include "state_common.h"

namespace fs {
namespace st {
namespace {

constexpr int P = 3;                    // bf16 pieces of features, of the state and of W's columns

// 32 features' rows of the state.
template <int W> struct StateLds {
  uint16_t t[P][32][W + 8];
  float z[32], bias[32], scale[4];      // scale (its first): of W's 32 features
};
template <int W, bool COLS> struct ImageLds {
  uint16_t row[STEPS<W>][2][1024];
  uint16_t col[COLS ? TILES<W> : 1][COLS ? P : 1][COLS ? 512 : 8];
};
// Where they come from; NTH threads carry them.
// (SCALED: T and z by the powers of two of z)
template <int W, bool COLS, bool SCALED, int NTH, bool FULL, bool IMAGES> struct Stage {
  static constexpr int NR = IMAGES ? (STEPS<W> * 256 + NTH - 1) / NTH : 1, NC = IMAGES && COLS ? (TILES<W> * P * 64 + NTH - 1) / NTH : 1,
                       NT = (8 * W + NTH - 1) / NTH;
  u32x4 row[NR], col[NC];
  f32x4 t[NT];
  float z, bias, scale;
  const char *row_img, *col_img;
  const float *T, *zs, *biases, *scales;
  int steps, M, dv;

  __device__ __forceinline__ void start(const Features& f, int side, const char* set, const float* T_, const float* z_, int dv_) {
    row_img = set + f.p.off_row[side];
    col_img = set + f.p.off_col[side];
    biases = (const float*)(set + f.p.off_bias);
    scales = (const float*)(set + f.p.off_scale[side]);
    T = T_; zs = z_; dv = FULL ? W : dv_; M = f.M;
    steps = FULL ? STEPS<W> : f.p.steps;
  }
  __device__ __forceinline__ void fetch(int fb, int tid) {
    if constexpr (IMAGES) {
#pragma unroll
      for (int i = 0; i < NR; ++i) {
        const int e = tid + NTH * i;
        if (e < steps * 256) row[i] = *(const u32x4*)(row_img + ((size_t)fb * steps * 256 + e) * 16);
      }
      if constexpr (COLS)
#pragma unroll
        for (int i = 0; i < NC; ++i) {
          const int e = tid + NTH * i;
          if (e < 2 * steps * P * 64) col[i] = *(const u32x4*)(col_img + ((size_t)fb * 2 * steps * P * 64 + e) * 16);
        }
    }
#pragma unroll
    for (int i = 0; i < NT; ++i) {
      const int e = tid + NTH * i, m = 32 * fb + e / (W / 4), c = 4 * (e % (W / 4));
      t[i] = f32x4{0.f, 0.f, 0.f, 0.f};
      if (e < 8 * W && m < M && (FULL || c < dv)) {
        const float* p = T + (size_t)m * dv + c;
        if (FULL || (dv & 3) == 0) t[i] = *(const f32x4*)p;
        else
#pragma unroll
          for (int j = 0; j < 4; ++j) t[i][j] = c + j < dv ? p[j] : 0.f;
      }
    }
    z = 32 * fb + (tid & 31) < M ? zs[32 * fb + (tid & 31)] : 0.f;
    if (tid < 32) {
      bias = biases[32 * fb + tid];
      scale = scales[fb];
    }
  }
  __device__ __forceinline__ void put(StateLds<W>& s, ImageLds<W, COLS>* img, int tid) {
    if constexpr (IMAGES) {
#pragma unroll
      for (int i = 0; i < NR; ++i) {
        const int e = tid + NTH * i;
        if (e < steps * 256) *(u32x4*)((char*)img->row + e * 16) = row[i];
      }
      if constexpr (COLS)
#pragma unroll
        for (int i = 0; i < NC; ++i) {
          const int e = tid + NTH * i;
          if (e < 2 * steps * P * 64) *(u32x4*)((char*)img->col + e * 16) = col[i];
        }
    }
    const int power = SCALED ? __builtin_amdgcn_frexp_expf(z) : 0;       // of feature tid % 32 (0 where z is 0 or not finite)
#pragma unroll
    for (int i = 0; i < NT; ++i) {
      const int e = tid + NTH * i, m = e / (W / 4), c = 4 * (e % (W / 4));
      if (e < 8 * W) {
        f32x8 v = {t[i][0], t[i][1], t[i][2], t[i][3], 0.f, 0.f, 0.f, 0.f};
        if constexpr (SCALED) {
          const int down = __builtin_amdgcn_ds_bpermute(4 * m, -power);
          v[0] = __builtin_amdgcn_ldexpf(v[0], down);
          v[1] = __builtin_amdgcn_ldexpf(v[1], down);
          v[2] = __builtin_amdgcn_ldexpf(v[2], down);
          v[3] = __builtin_amdgcn_ldexpf(v[3], down);
        }
        const Op<P> o = as_op<P>(v);
#pragma unroll
        for (int p = 0; p < P; ++p) {
          const u32x4 u = __builtin_bit_cast(u32x4, o.p[p]);
          *(u32x2*)&s.t[p][m][c] = u32x2{u[0], u[1]};
        }
      }
    }
    if (tid < 32) {
      s.z[tid] = __builtin_amdgcn_ldexpf(z, -power);
      s.bias[tid] = SCALED && z == 0.f ? kNone : bias + (float)power;
      if (tid < 4) s.scale[tid] = scale;
    }
  }
};
// W of 32 features as operands: from LDS where the workgroup has the images there, or (DIRECT) in registers, on their way long before their use
// (the rows of the next 32 features once this wave's exponents are done, the columns ahead of the exponents).
template <int W, bool COLS, bool DIRECT> struct Weights {
  const ImageLds<W, COLS>* img;
  int fb;
  __device__ __forceinline__ Op16<2> row(int s, int ft, int lane) const {
    Op16<2> o;
#pragma unroll
    for (int p = 0; p < 2; ++p) o.p[p] = *(const f16x8*)&img->row[s][p][ft * 512 + lane * 8];
    return o;
  }
  __device__ __forceinline__ Op<P> col(int ct, int lane) const { return image_op<P>(&img->col[ct][0][0], lane); }
  __device__ __forceinline__ void rows_used(int) {}
};
template <int W, bool COLS> struct Weights<W, COLS, true> {
  static constexpr int S = STEPS<W>, CT = COLS ? TILES<W> : 1;
  const char *row_img, *col_img;
  int fb, next, steps;
  Op16<2> rows[S][2];
  Op<P> cols[CT];
  __device__ __forceinline__ void load_rows(int f, int lane) {
    const uint16_t* at = (const uint16_t*)row_img + (size_t)f * steps * 2048 + lane * 8;
#pragma unroll
    for (int s = 0; s < S; ++s)
#pragma unroll
      for (int ft = 0; ft < 2; ++ft)
#pragma unroll
        for (int p = 0; p < 2; ++p) rows[s][ft].p[p] = *(const f16x8*)(at + (min(s, steps - 1) * 2 + p) * 1024 + ft * 512);
  }
  __device__ __forceinline__ void load_cols(int lane) {
    if constexpr (COLS)
#pragma unroll
      for (int ct = 0; ct < CT; ++ct) cols[ct] = image_op<P>((const uint16_t*)col_img + (size_t)(fb * 2 * steps + min(ct, 2 * steps - 1)) * 1536, lane);
  }
  __device__ __forceinline__ Op16<2> row(int s, int ft, int) const { return rows[s][ft]; }
  __device__ __forceinline__ Op<P> col(int ct, int) const { return cols[ct]; }
  __device__ __forceinline__ void rows_used(int lane) {
    if (next >= 0) load_rows(next, lane);
  }
};

__device__ __forceinline__ void wave_fence() {
  __builtin_amdgcn_wave_barrier();
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_wave_barrier();
}

// The rows of a wave: their number as operands of the exponents and what undoes their scale.
template <int W, int XP, int RT, bool FULL> struct RowOps {
  static constexpr int S = STEPS<W>;
  Op16<XP> x[RT][S];
  float undo[RT], square[RT];    // square: this lane's part of |x|^2
  RowAt at[RT];
  bool live[RT];
  __device__ __forceinline__ void load(const Rows& r, int b, int h, int v0, int rows, int len, int steps, int lane) {
    const int g = lane >> 4, c = lane & 15;
    RowUnits<S, FULL, XP == 2, XP == 1 ? 1 : -1> units[RT];
    long long base[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      const int v = v0 + 16 * rt + c;
      at[rt] = row_at(r, min(v, rows - 1));
      live[rt] = v < rows && at[rt].row < len;
      base[rt] = row_base(r.X, b, h * r.G + at[rt].head, at[rt].row);
      units[rt].fetch(r.X, base[rt], r.cols, r.turn, g);
    }
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      f32x8 n[S];
      units[rt].finish(r.X, base[rt], r.cols, r.turn, r.turn.table + ((long long)b * r.L + at[rt].row) * (r.turn.rot >> 1), live[rt], g, n);
      float most = 0.f;
      square[rt] = 0.f;
#pragma unroll
      for (int s = 0; s < S; ++s) {
        most = fmaxf(most, largest_of(n[s]));
#pragma unroll
        for (int i = 0; i < 8; ++i) square[rt] += n[s][i] * n[s][i];
      }
      most = fmaxf(most, __shfl_xor(most, 16));
      most = fmaxf(most, __shfl_xor(most, 32));
      const float scale = up_to_2_14(most);
      undo[rt] = power_inverse(scale);
#pragma unroll
      for (int s = 0; s < S; ++s) x[rt][s] = as_op16<XP>(n[s] * scale);
    }
  }
};
template <int W, int XP, bool COLS, int RT, bool FULL, bool DIRECT>
__device__ __forceinline__ void exponents(const RowOps<W, XP, RT, FULL>& x, Weights<W, COLS, DIRECT>& weights, int steps, int lane, f32x4 (&E)[RT][2]) {
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) E[rt][0] = E[rt][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int s = 0; s < STEPS<W>; ++s)
    if (FULL || s < steps) {
      const Op16<2> w[2] = {weights.row(s, 0, lane), weights.row(s, 1, lane)};
      each_product<2, XP>([&](int i, int j) {
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
#pragma unroll
          for (int ft = 0; ft < 2; ++ft) E[rt][ft] = mfma(w[ft].p[i], x.x[rt][s].p[j], E[rt][ft]);
      });
    }
  weights.rows_used(lane);
}
__device__ __forceinline__ float over_groups_max(float v) {
  v = fmaxf(v, __shfl_xor(v, 16));
  return fmaxf(v, __shfl_xor(v, 32));
}
__device__ __forceinline__ float over_groups_sum(float v) {
  v += __shfl_xor(v, 16);
  return v + __shfl_xor(v, 32);
}
// Numbers of rows 4 g .. 4 g + 3 of a tile from the lanes of the rows.
__device__ __forceinline__ f32x4 by_row(float v, int lane) {
  f32x4 k;
#pragma unroll
  for (int r = 0; r < 4; ++r) k[r] = __shfl(v, 4 * (lane >> 4) + r);
  return k;
}
// E: exponents of a tile of rows less their references.  Raises those that an exponent passes by `limit` (2^16; -inf: there is no reference yet, 0, and
// nothing summed), and what was summed to them.
template <int N, int K, int TA, int TB>
__device__ __forceinline__ void raise(f32x4 (&E)[2], float& ref, float& limit, float (&sums)[N], f32x4 (&acc)[K][TA], f32x4 (&more)[K][TB], int rt,
                                      int lane) {
  float most = kNone;
#pragma unroll
  for (int ft = 0; ft < 2; ++ft)
#pragma unroll
    for (int r = 0; r < 4; ++r) most = fmaxf(most, E[ft][r]);
  if (__any(most > limit)) {
    most = over_groups_max(most);
    const bool raised = most > limit;
    const float up = raised ? most - 8.f : 0.f, keep = limit == kNone ? 1.f : fast_exp2(-up);
    ref += up;
    limit = raised ? 16.f : limit;
#pragma unroll
    for (int n = 0; n < N; ++n) sums[n] *= keep;
    const f32x4 k = by_row(keep, lane);
#pragma unroll
    for (int t = 0; t < TA; ++t) acc[rt][t] *= k;
#pragma unroll
    for (int t = 0; t < TB; ++t) more[rt][t] *= k;
#pragma unroll
    for (int ft = 0; ft < 2; ++ft) E[ft] -= up;
  }
}

// A tile of 16 rows from the accumulators (register r of lane (g, c): row 4 g + r, column 16 ct + c), times a number of the row, to LDS.
template <int W> __device__ __forceinline__ void tile_to_lds(float* dst, const f32x4 (&acc)[TILES<W>], f32x4 factor, int lane) {
  const int g = lane >> 4, c = lane & 15;
#pragma unroll
  for (int ct = 0; ct < TILES<W>; ++ct)
#pragma unroll
    for (int r = 0; r < 4; ++r) dst[(4 * g + r) * (W + 4) + 16 * ct + c] = acc[ct][r] * factor[r];
}
template <int W> __device__ __forceinline__ f32x8 from_tile(const float* row, int c0) {
  const f32x4 a = *(const f32x4*)(row + c0), b = *(const f32x4*)(row + c0 + 4);
  return f32x8{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
}

// A workgroup's state and piece of rows.  Workgroups go to the eight XCDs in turn, so that with eight states or a multiple the pieces of a state
// meet in one L2; where sequences have lengths of their own and an XCD would have some of them only, the states turn with the piece.  (Cross
// attention of 8 padded sequences with 8 heads, gradients of the keys: pieces in turn, so that two XCDs had the sequences' ends, 109 us.)
struct Piece { int bh, rows; };
__device__ __forceinline__ Piece piece_of(int BH, int Hk, bool padded) {
  const int y = blockIdx.y + (blockIdx.z << 15);
  return Piece{(int)(padded && Hk % 8 != 0 ? (blockIdx.x + (unsigned)y) % (unsigned)BH : blockIdx.x), y};
}
dim3 pieces(int BH, long long n) { return dim3(BH, (unsigned)std::min(n, 1ll << 15), (unsigned)((n + (1 << 15) - 1) >> 15)); }

constexpr size_t most_of(size_t a, size_t b) { return a > b ? a : b; }
template <int W, bool COLS, int NW, int RT, bool DIRECT> constexpr size_t rows_lds() {
  return DIRECT ? most_of(NW * sizeof(StateLds<W>), (size_t)NW * 16 * RT * (W + 4) * 4)
                : most_of(2 * (sizeof(StateLds<W>) + sizeof(ImageLds<W, COLS>)), (size_t)NW * 16 * (W + 4) * 4);
}

// Whether a workgroup's rows v0 .. v0 + n - 1 are all padding; they are then zeros of `out`.
template <int W, int NTH>
__device__ __forceinline__ bool all_padding(const Rows& r, int b, int h, int v0, int n, int len, const TensorDev& out, int cols, int tid) {
  const int rows = r.L * r.G, v1 = min(v0 + n, rows), first = v0 % r.L;
  // (a row below `len` is among them unless they end before the next head's first one)
  if (first < len || (first + (v1 - v0) > r.L && len > 0)) return false;
  const f32x8 zero = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  for (int u = tid; u < (v1 - v0) * (W / 8); u += NTH) {
    const int c0 = 8 * (u % (W / 8));
    const RowAt at = row_at(r, v0 + u / (W / 8));
    if (c0 < cols) store8(out, row_base(out, b, h * r.G + at.head, at.row), c0, cols, zero);
  }
  return true;
}

// Calls body(state in LDS, W) for the features of this wave.
template <int W, bool COLS, bool SCALED, int NW, bool FULL, bool DIRECT, class Body>
__device__ __forceinline__ void walk_features(const Features& f, int side, const char* set, const float* T, const float* z, int dv, char* lds, int w,
                                              int tid, int lane, Body body) {
  const int nfb = f.p.Mp / 32;
  if constexpr (DIRECT) {
    Stage<W, false, SCALED, 64, FULL, false> stage;
    stage.start(f, side, set, T, z, dv);
    StateLds<W>& mine = ((StateLds<W>*)lds)[w];
    Weights<W, COLS, true> weights;
    weights.row_img = stage.row_img;
    weights.col_img = stage.col_img;
    weights.steps = stage.steps;
    if (w < nfb) {
      stage.fetch(w, lane);
      weights.load_rows(w, lane);
    }
    for (int fb = w; fb < nfb; fb += NW) {
      weights.fb = fb;
      weights.next = fb + NW < nfb ? fb + NW : -1;
      stage.put(mine, nullptr, lane);
      weights.load_cols(lane);
      if (fb + NW < nfb) stage.fetch(fb + NW, lane);
      wave_fence();
      body(mine, weights);
      wave_fence();
    }
  } else {
    Stage<W, COLS, SCALED, 64 * NW, FULL, true> stage;
    stage.start(f, side, set, T, z, dv);
    struct Both { StateLds<W> s; ImageLds<W, COLS> img; };
    Both* both = (Both*)lds;
    stage.fetch(0, tid);
    stage.put(both[0].s, &both[0].img, tid);
    __syncthreads();
    for (int fb = 0; fb < nfb; ++fb) {
      Both &now = both[fb & 1], &next = both[~fb & 1];
      const bool more = fb + 1 < nfb;
      if (more) stage.fetch(fb + 1, tid);
      Weights<W, COLS, false> weights{&now.img, fb};
      body(now.s, weights);
      if (more) stage.put(next.s, &next.img, tid);
      __syncthreads();
    }
  }
}
// Common reference and sums of a row over the waves of a DIRECT workgroup: what this wave's are multiplied by.  A wave without a reference (-inf) has
// sums of zeros, or of what is not a number.  red: [RT][NW][16] refs, then N times the same of sums.
template <int NW, int RT, int N>
__device__ __forceinline__ void meet(float (&ref)[RT], float (&sums)[RT][N], float (&factor)[RT], float* red, int w, int lane) {
  const int c = lane & 15;
  if (lane < 16)
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      red[(rt * NW + w) * 16 + c] = ref[rt];
#pragma unroll
      for (int n = 0; n < N; ++n) red[((n + 1) * RT * NW + rt * NW + w) * 16 + c] = sums[rt][n];
    }
  __syncthreads();
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    float top = kNone;
    for (int i = 0; i < NW; ++i) top = fmaxf(top, red[(rt * NW + i) * 16 + c]);
    auto to_top = [&](float from) { return from == kNone ? 1.f : fast_exp2(from - top); };
    factor[rt] = to_top(ref[rt]);
#pragma unroll
    for (int n = 0; n < N; ++n) {
      float sum = 0.f;
      for (int i = 0; i < NW; ++i) sum += to_top(red[(rt * NW + i) * 16 + c]) * red[((n + 1) * RT * NW + rt * NW + i) * 16 + c];
      sums[rt][n] = sum;
    }
    ref[rt] = top;
  }
}

template <int W, int XP, int NW, int RT, bool FULL, bool DIRECT>
__global__ void __launch_bounds__(64 * NW, W == 64 && !DIRECT ? 4 : 1) k_values(ValueArgs a) {
  constexpr int VT = TILES<W>, LD = W + 8;
  extern __shared__ __align__(16) char lds[];
  __shared__ float red[DIRECT ? 2 * RT * NW * 16 : 1];
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), g = lane >> 4;
  const Piece piece = piece_of(a.B * a.Hk, a.Hk, a.x.lengths != nullptr);
  const int bh = piece.bh, b = bh / a.Hk, h = bh - b * a.Hk, steps = a.f.p.steps, dv = FULL ? W : a.dv;
  const int slot = slot_of(a.slots, a.state.slots, b), len = length_of(a.x, b), rows = a.x.L * a.x.G;
  const int v0 = (DIRECT ? piece.rows : piece.rows * NW + w) * 16 * RT;
  const char* set = a.f.set(h);
  const size_t st = (size_t)max(slot, 0) * a.Hk + h;
  constexpr int WG_ROWS = 16 * RT * (DIRECT ? 1 : NW);
  if (piece.rows * WG_ROWS >= rows) return;
  if (all_padding<W, 64 * NW>(a.x, b, h, piece.rows * WG_ROWS, WG_ROWS, len, a.Y, dv, tid)) return;

  RowOps<W, XP, RT, FULL> x;
  x.load(a.x, b, h, v0, rows, len, steps, lane);
  float ref[RT], limit[RT], den[RT][1];
  f32x4 acc[RT][VT], none[RT][1];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    ref[rt] = 0.f;
    limit[rt] = kNone;
    den[rt][0] = 0.f;
#pragma unroll
    for (int vt = 0; vt < VT; ++vt) acc[rt][vt] = f32x4{0.f, 0.f, 0.f, 0.f};
    none[rt][0] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  if (slot >= 0)
    walk_features<W, false, true, NW, FULL, DIRECT>(
        a.f, 0, set, a.state.T + st * a.f.M * dv, a.state.z + st * a.f.M, dv, lds, w, tid, lane,
        [&](const StateLds<W>& l, Weights<W, false, DIRECT>& weights) {
          f32x4 E[RT][2];
          exponents(x, weights, steps, lane, E);
          const float scale = l.scale[0];
          f32x4 bias[2], zf[2];
#pragma unroll
          for (int ft = 0; ft < 2; ++ft) {
            bias[ft] = *(const f32x4*)&l.bias[16 * ft + 4 * g];
            zf[ft] = *(const f32x4*)&l.z[16 * ft + 4 * g];
          }
          Op<P> po[RT];
#pragma unroll
          for (int rt = 0; rt < RT; ++rt) {
            const float undo = x.undo[rt] * scale;
#pragma unroll
            for (int ft = 0; ft < 2; ++ft) E[rt][ft] = E[rt][ft] * undo + (bias[ft] - ref[rt]);
            raise(E[rt], ref[rt], limit[rt], den[rt], acc, none, rt, lane);
            f32x8 p;
#pragma unroll
            for (int ft = 0; ft < 2; ++ft)
#pragma unroll
              for (int r = 0; r < 4; ++r) {
                p[4 * ft + r] = fast_exp2(E[rt][ft][r]);
                den[rt][0] += p[4 * ft + r] * zf[ft][r];
              }
            po[rt] = as_op<P>(p);
          }
#pragma unroll
          for (int vt = 0; vt < VT; vt += 2)
            if (FULL || 16 * vt < dv) {
              const uint16_t* at_t = &l.t[0][0][16 * vt] + lane_tr(lane, LD);
              const Op<P> t[2] = {column_op<P>(at_t, LD, 32 * LD), column_op<P>(at_t + 16, LD, 32 * LD)};
              outer_at(po, t, acc, vt);
            }
        });
  float factor[RT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    den[rt][0] = over_groups_sum(den[rt][0]);
    factor[rt] = 1.f;
    if (limit[rt] == kNone) ref[rt] = kNone;
  }
  if constexpr (DIRECT) {
    __syncthreads();       // (the waves' states in LDS make room for their sums)
    meet<NW, RT, 1>(ref, den, factor, red, w, lane);
  }
  int unread = 0;
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const bool zero = den[rt][0] == 0.f;
    unread += (lane < 16) && (!DIRECT || w == 0) && x.live[rt] && zero;
    const f32x4 k = by_row(zero ? 0.f : factor[rt] / den[rt][0], lane);
    float* tile = (float*)lds + (DIRECT ? (size_t)w * RT + rt : (size_t)w) * 16 * (W + 4);
    tile_to_lds<W>(tile, acc[rt], k, lane);
    if constexpr (!DIRECT) {
      wave_fence();
      for (int u = lane; u < 16 * (W / 8); u += 64) {
        const int r = u / (W / 8), c0 = 8 * (u % (W / 8)), vr = v0 + 16 * rt + r;
        if (vr >= rows || (!FULL && c0 >= dv)) continue;
        const RowAt at = row_at(a.x, vr);
        f32x8 y = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (at.row < len) y = from_tile<W>(tile + r * (W + 4), c0);
        store8(a.Y, row_base(a.Y, b, h * a.x.G + at.head, at.row), c0, dv, y);
      }
      wave_fence();
    }
  }
  if constexpr (DIRECT) {
    __syncthreads();
    for (int u = tid; u < 16 * RT * (W / 8); u += 64 * NW) {
      const int r = u / (W / 8), c0 = 8 * (u % (W / 8)), vr = v0 + r;
      if (vr >= rows || (!FULL && c0 >= dv)) continue;
      const RowAt at = row_at(a.x, vr);
      f32x8 y = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
      if (at.row < len)
        for (int i = 0; i < NW; ++i) y += from_tile<W>((const float*)lds + (size_t)(i * 16 * RT + r) * (W + 4), c0);
      store8(a.Y, row_base(a.Y, b, h * a.x.G + at.head, at.row), c0, dv, y);
    }
  }
  if (a.unread != nullptr) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) unread += __shfl_xor(unread, o);
    if (lane == 0 && unread > 0) atomicAdd(a.unread, unread);
  }
}

// Gradients.  KEYS = false: with p relative to a row's reference, u = p (dY . T + 0) and p z against W in two sums, of which, with the row's
// normaliser and delta = sum u / sum p z, dx = (first - delta second) / normaliser.  KEYS = true: the features are those the state has
// (terms hold its shift): u = s (r . T + z) against W, s against T.
template <int W, int XP, int RP, int NW, int RT, bool FULL, bool DIRECT, bool KEYS>
__global__ void __launch_bounds__(64 * NW, W == 64 && RP == 1 ? 2 : 1) k_grads(GradArgs a) {
  constexpr int S = STEPS<W>, CT = TILES<W>, LD = W + 8;
  extern __shared__ __align__(16) char lds[];
  __shared__ __align__(16) float red[DIRECT ? 3 * RT * NW * 16 : KEYS ? RT * NW * 16 : 1];
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), g = lane >> 4, c = lane & 15;
  const Piece piece = piece_of(a.B * a.Hk, a.Hk, a.x.lengths != nullptr);
  const int bh = piece.bh, b = bh / a.Hk, h = bh - b * a.Hk, steps = FULL ? S : a.f.p.steps, dv = FULL ? W : a.dv, d = FULL ? W : a.f.d;
  const int slot = KEYS ? unique_slot_of(a.slots, a.state.slots, b) : slot_of(a.slots, a.state.slots, b), len = length_of(a.x, b),
            rows = a.x.L * a.x.G;
  const int v0 = (DIRECT ? piece.rows : piece.rows * NW + w) * 16 * RT;
  const char* set = a.f.set(h);
  const size_t st = (size_t)max(slot, 0) * a.Hk + h;
  constexpr int WG_ROWS = 16 * RT * (DIRECT ? 1 : NW);
  if (piece.rows * WG_ROWS >= rows) return;
  if (all_padding<W, 64 * NW>(a.x, b, h, piece.rows * WG_ROWS, WG_ROWS, len, a.dx, d, tid)) {
    if constexpr (KEYS) all_padding<W, 64 * NW>(a.x, b, h, piece.rows * WG_ROWS, WG_ROWS, len, a.dr, dv, tid);
    else
      for (int v = piece.rows * WG_ROWS + tid; v < min((piece.rows + 1) * WG_ROWS, rows); v += 64 * NW) {
        a.lse[(size_t)bh * rows + v] = kNone;
        a.weights[(size_t)bh * rows + v] = 0.f;
      }
    return;
  }

  RowOps<W, XP, RT, FULL> x;
  x.load(a.x, b, h, v0, rows, len, steps, lane);
  Op<RP> rr[RT][S];
  float ref[RT], limit[RT], term[RT], sums[RT][2];            // queries: normaliser, sum u; keys: -, sum u
  f32x4 acc[RT][CT], more[RT][CT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
#pragma unroll
    for (int s = 0; s < S; ++s) {
      if constexpr (RP == 1) {
        u32x4 n = row8_bits<FULL>(a.r, b, h, x.at[rt], 32 * s + 8 * g);
#pragma unroll
        for (int i = 0; i < 4; ++i) n[i] = x.live[rt] ? n[i] : 0u;
        rr[rt][s].p[0] = __builtin_bit_cast(bf16x8, n);
      } else {
        f32x8 n = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        const int c0 = 32 * s + 8 * g;
        if (x.live[rt] && (FULL || c0 < dv))
          n = load8<FULL>(a.r.X, row_base(a.r.X, b, h * a.r.G + x.at[rt].head, x.at[rt].row), c0, dv);
        rr[rt][s] = as_op<RP>(n);
      }
    }
    term[rt] = over_groups_sum(x.square[rt]) * -0.5f * kLog2e * a.f.scale2;     // (keys)
    ref[rt] = sums[rt][0] = sums[rt][1] = 0.f;
    limit[rt] = kNone;
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) acc[rt][ct] = more[rt][ct] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  // (C2 + C2') x of a tile's rows, sixteen coordinates; waves that have the same rows take them in turn
  auto form_of = [&](int rt, int ct) {
    f32x4 q = {0.f, 0.f, 0.f, 0.f};
    const uint16_t* img = (const uint16_t*)(set + a.f.p.off_csym) + (size_t)ct * steps * 2 * 512;
#pragma unroll
    for (int s = 0; s < S; ++s)
      if (FULL || s < steps) {
        Op16<2> co;
#pragma unroll
        for (int p = 0; p < 2; ++p) co.p[p] = *(const f16x8*)(img + (s * 2 + p) * 512 + lane * 8);
        each_product<XP, 2>([&](int i, int j) { q = mfma(x.x[rt][s].p[i], co.p[j], q); });
      }
    return q;
  };
  if constexpr (KEYS) {
    if (a.f.dense) {
      const float undo = 0.5f * kLog2e * a.f.scale2 * *(const float*)(set + a.f.p.off_cscale);
      float* tile = (float*)lds + (size_t)w * 16 * (W + 4);
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
#pragma unroll
        for (int s = 0; s < S; ++s)
#pragma unroll
          for (int i = 0; i < 8; i += 4) {
            f32x4 y;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              y[j] = (float)x.x[rt][s].p[0][i + j];
              if constexpr (XP == 2) y[j] += (float)x.x[rt][s].p[1][i + j];
            }
            *(f32x4*)(tile + c * (W + 4) + 32 * s + 8 * g + i) = y;
          }
        wave_fence();
        f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int ct = 0; ct < CT; ++ct)
          if ((FULL || 16 * ct < d) && (!DIRECT || ct % NW == w)) {
            const f32x4 q = form_of(rt, ct);
#pragma unroll
            for (int r = 0; r < 4; ++r) sum[r] += q[r] * tile[(4 * g + r) * (W + 4) + 16 * ct + c];
          }
#pragma unroll
        for (int r = 0; r < 4; ++r) sum[r] = over_lanes<16>(sum[r], [](float p, float q) { return p + q; });
        if (c == 0) *(f32x4*)&red[(rt * NW + w) * 16 + 4 * g] = sum;
        wave_fence();
      }
      __syncthreads();         // (and the tiles make room for the state)
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        term[rt] = 0.f;
#pragma unroll
        for (int i = 0; i < NW; ++i)
          if (DIRECT || i == w) term[rt] += red[(rt * NW + i) * 16 + c];
        term[rt] = term[rt] * x.undo[rt] * (x.undo[rt] * undo);
      }
      if constexpr (DIRECT) __syncthreads();      // (red is used again)
    }
    const float shift = slot >= 0 ? a.shift[st] : 0.f;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) term[rt] = x.live[rt] && slot >= 0 ? term[rt] - shift : kNone;
  }
  if (slot >= 0)
    walk_features<W, true, !KEYS, NW, FULL, DIRECT>(
        a.f, KEYS, set, a.state.T + st * a.f.M * dv, a.state.z + st * a.f.M, dv, lds, w, tid, lane,
        [&](const StateLds<W>& l, Weights<W, true, DIRECT>& weights) {
          f32x4 E[RT][2], D[RT][2], bias[2], zf[2];
#pragma unroll
          for (int ft = 0; ft < 2; ++ft) {
            bias[ft] = *(const f32x4*)&l.bias[16 * ft + 4 * g];
            zf[ft] = *(const f32x4*)&l.z[16 * ft + 4 * g];
          }
          exponents(x, weights, steps, lane, E);
#pragma unroll
          for (int rt = 0; rt < RT; ++rt)
#pragma unroll
            for (int ft = 0; ft < 2; ++ft) D[rt][ft] = KEYS ? zf[ft] : f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int s = 0; s < S; ++s)
            if (FULL || 32 * s < dv) {
              const Op<P> t[2] = {row_op<P>(&l.t[0][c][32 * s + 8 * g], 32 * LD), row_op<P>(&l.t[0][16 + c][32 * s + 8 * g], 32 * LD)};
              each_product<P, RP>([&](int i, int j) {
#pragma unroll
                for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                  for (int ft = 0; ft < 2; ++ft) D[rt][ft] = mfma(t[ft].p[i], rr[rt][s].p[j], D[rt][ft]);
              });
            }
          const float scale = l.scale[0];
          Op<P> uo[RT], so[RT];
#pragma unroll
          for (int rt = 0; rt < RT; ++rt) {
            const float undo = x.undo[rt] * scale;
#pragma unroll
            for (int ft = 0; ft < 2; ++ft) E[rt][ft] = E[rt][ft] * undo + (KEYS ? bias[ft] + term[rt] : bias[ft] - ref[rt]);
            if constexpr (!KEYS) raise(E[rt], ref[rt], limit[rt], sums[rt], acc, more, rt, lane);
            f32x8 u, s;
#pragma unroll
            for (int ft = 0; ft < 2; ++ft)
#pragma unroll
              for (int r = 0; r < 4; ++r) {
                const float p = fast_exp2(E[rt][ft][r]);
                u[4 * ft + r] = p * D[rt][ft][r];
                s[4 * ft + r] = KEYS ? p : p * zf[ft][r];
                sums[rt][1] += u[4 * ft + r];
                if constexpr (!KEYS) sums[rt][0] += s[4 * ft + r];
              }
            uo[rt] = as_op<P>(u);
            so[rt] = as_op<P>(s);
          }
#pragma unroll
          for (int ct = 0; ct < CT; ct += 2) {
            if (FULL || 16 * ct < d) {
              const Op<P> wo[2] = {weights.col(ct, lane), weights.col(ct + 1, lane)};
              outer_at(uo, wo, acc, ct);
              if constexpr (!KEYS) outer_at(so, wo, more, ct);
            }
            if constexpr (KEYS)
              if (FULL || 16 * ct < dv) {
                const uint16_t* at_t = &l.t[0][0][16 * ct] + lane_tr(lane, LD);
                const Op<P> t[2] = {column_op<P>(at_t, LD, 32 * LD), column_op<P>(at_t + 16, LD, 32 * LD)};
                outer_at(so, t, more, ct);
              }
          }
        });
  float factor[RT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    sums[rt][0] = over_groups_sum(sums[rt][0]);
    sums[rt][1] = over_groups_sum(sums[rt][1]);
    factor[rt] = 1.f;
    if (!KEYS && limit[rt] == kNone) ref[rt] = kNone;
  }
  if constexpr (DIRECT) {
    __syncthreads();
    meet<NW, RT, 2>(ref, sums, factor, red, w, lane);
  }
  float* tiles = (float*)lds;
  // out (of n numbers a row) from the tiles: row r of the workgroup's, or of the wave's, rows
  auto store = [&](const TensorDev& out, int n, int rt, const Turn* turn, auto&& finish) {
    const float* tile = tiles + (DIRECT ? 0 : (size_t)w * 16 * (W + 4));
    for (int u = DIRECT ? tid : lane; u < 16 * (DIRECT ? RT : 1) * (W / 8); u += DIRECT ? 64 * NW : 64) {
      const int r = u / (W / 8), c0 = 8 * (u % (W / 8)), vr = v0 + (DIRECT ? 0 : 16 * rt) + r;
      if (vr >= rows || (!FULL && c0 >= n)) continue;
      const RowAt at = row_at(a.x, vr);
      f32x8 y = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
      if (slot >= 0 && at.row < len) y = finish(tile, r, at, c0, turn);
      store8(out, row_base(out, b, h * a.x.G + at.head, at.row), c0, n, y);
    }
  };
  auto sum_of = [&](const float* tile, int r, int c0) {
    f32x8 y = from_tile<W>(tile + r * (W + 4), c0);
    if constexpr (DIRECT)
      for (int i = 1; i < NW; ++i) y += from_tile<W>(tile + (size_t)(i * 16 * RT + r) * (W + 4), c0);
    return y;
  };
  auto turned_back = [&](const float* tile, int r, RowAt at, int c0, const Turn* turn) {
    const f32x8 y = sum_of(tile, r, c0);
    if (XP == 1 || turn == nullptr || turn->rot == 0) return y;
    const float2* cs = turn->table + ((long long)b * a.x.L + at.row) * (turn->rot >> 1);
    return turned8(y, c0, *turn, cs, -1.f,
                   [&](int col) {
                     float q = tile[r * (W + 4) + col];
                     if constexpr (DIRECT)
                       for (int i = 1; i < NW; ++i) q += tile[(size_t)(i * 16 * RT + r) * (W + 4) + col];
                     return q;
                   },
                   [&](int col) { return sum_of(tile, r, col); });
  };
#pragma unroll
  for (int part = 0; part < (KEYS ? 2 : 1); ++part) {
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      float* tile = tiles + (DIRECT ? (size_t)w * RT + rt : (size_t)w) * 16 * (W + 4);
      if (part == 1) {
        tile_to_lds<W>(tile, more[rt], f32x4{1.f, 1.f, 1.f, 1.f}, lane);
      } else if constexpr (KEYS) {
        // the row term: (sum u) s^2 (C2 + C2') x; waves that have the same rows take sixteen columns each in turn
        const f32x4 rho4 = by_row(sums[rt][1] * a.f.scale2 * x.undo[rt], lane) * *(const float*)(set + a.f.p.off_cscale);
#pragma unroll
        for (int ct = 0; ct < CT; ++ct)
          if (FULL || 16 * ct < d) {
            acc[rt][ct] *= kLn2;
            if (!DIRECT || ct % NW == w) acc[rt][ct] += rho4 * form_of(rt, ct);
          }
        tile_to_lds<W>(tile, acc[rt], f32x4{1.f, 1.f, 1.f, 1.f}, lane);
      } else {
        const bool zero = sums[rt][0] == 0.f;
        const float inv = zero ? 0.f : 1.f / sums[rt][0], delta = zero ? 0.f : sums[rt][1] / sums[rt][0];
        const int v = v0 + 16 * rt + c;
        if (lane < 16 && v < rows && (!DIRECT || w == 0)) {
          a.lse[(size_t)bh * rows + v] = x.live[rt] && slot >= 0 && !zero ? -(ref[rt] + __log2f(sums[rt][0])) : kNone;
          a.weights[(size_t)bh * rows + v] = -delta;
        }
        const f32x4 d4 = by_row(delta, lane);
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) acc[rt][ct] -= d4 * more[rt][ct];
        tile_to_lds<W>(tile, acc[rt], by_row(kLn2 * inv * factor[rt], lane), lane);
      }
      if constexpr (!DIRECT) {
        wave_fence();
        if (part == 0) store(a.dx, d, rt, &a.x.turn, turned_back);
        else store(a.dr, dv, rt, nullptr, turned_back);
        wave_fence();
      }
    }
    if constexpr (DIRECT) {
      __syncthreads();
      if (part == 0) store(a.dx, d, 0, &a.x.turn, turned_back);
      else store(a.dr, dv, 0, nullptr, turned_back);
      __syncthreads();
    }
  }
}

int lds_room(const void* kernel, size_t lds) {
  if (lds > 64 * 1024 && hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds) != hipSuccess) {
    (void)hipGetLastError();
    return 5;
  }
  return 0;
}
// Few rows: fewer than `most` pieces of 256, a quarter of the CUs, for gradients of up to 64 numbers 40, but those of 64-wide queries.  (us, few rows' form / the
// other.  8 states of 64 x 256, bf16: values of 512 rows each 9.3 / 15.4, 1536 17.3 / 15.8, 4096 34 / 18; gradients of keys 9.7 / 27, 25 / 28, 64 / 30;
// of queries, with the state's, 25 / 54, 47 / 62, 88 / 68, in fp32 29 / 48, 56 / 57, 106 / 66.  8 of 32 x 128: keys 512 rows 7.0 / 10.5, 1280 12.9 / 11.0.  4 of
// 128 x 512, fp32: values of 2048 rows 26 / 64, 4096 50 / 66, 8192 97 / 72; gradients of keys 51 / 91, 102 / 96, 192 / 112.)
bool few_rows(int BH, long long rows, int most) { return BH * ((rows + 255) / 256) < most; }

// Waves of a workgroup and tiles of sixteen rows of a wave.  Values of 64 numbers: eight waves of one tile, which have 128 registers (262144 queries of
// 64 x 256, bf16: 94 us traced, four waves of two tiles 100).  Their gradients, bf16: two tiles and 256 registers, queries in eight waves (46; 61 in four),
// keys in four (112; 125 in eight, 135 of one tile); in fp32, which would not fit in 256, four waves to a CU (keys 179; 221 with spills).
template <int W, int XP, bool FULL, bool DIRECT> int values(const ValueArgs& a, hipStream_t st) {
  constexpr int NW = DIRECT == (W == 128) && W != 64 ? 4 : 8, RT = W == 64 && !DIRECT ? 1 : 2, ROWS = 16 * RT * (DIRECT ? 1 : NW);
  constexpr size_t lds = rows_lds<W, false, NW, RT, DIRECT>();
  static_assert(lds <= 156 * 1024, "LDS of a CU");
  auto kernel = k_values<W, XP, NW, RT, FULL, DIRECT>;
  if (int rc = lds_room((const void*)kernel, lds)) return rc;
  hipLaunchKernelGGL(kernel, pieces(a.B * a.Hk, ((long long)a.x.L * a.x.G + ROWS - 1) / ROWS), dim3(64 * NW), lds, st, a);
  return hipGetLastError() == hipSuccess ? 0 : 5;
}
template <int W, int XP, bool FULL> int values_rows(const ValueArgs& a, hipStream_t st) {
  return few_rows(a.B * a.Hk, (long long)a.x.L * a.x.G, 64) ? values<W, XP, FULL, true>(a, st) : values<W, XP, FULL, false>(a, st);
}
template <int W, bool FULL> int values_pieces(const ValueArgs& a, hipStream_t st) {
  return a.x.X.dtype == 1 && a.x.turn.rot == 0 ? values_rows<W, 1, FULL>(a, st) : values_rows<W, 2, FULL>(a, st);
}
template <int W> int values_width(const ValueArgs& a, hipStream_t st) {
  return a.f.d == W && a.dv == W ? values_pieces<W, true>(a, st) : values_pieces<W, false>(a, st);
}

template <int W, int XP, int RP, bool FULL, bool DIRECT, bool KEYS> int grads(const GradArgs& a, hipStream_t st) {
  constexpr int NW = DIRECT == (W == 128) && !(W == 64 && RP == 1 && !KEYS) ? 4 : 8, RT = W == 128 || (DIRECT && W == 64) ? 1 : 2,
                ROWS = 16 * RT * (DIRECT ? 1 : NW);
  constexpr size_t lds = rows_lds<W, true, NW, RT, DIRECT>();
  static_assert(lds <= 156 * 1024, "LDS of a CU");
  auto kernel = k_grads<W, XP, RP, NW, RT, FULL, DIRECT, KEYS>;
  if (int rc = lds_room((const void*)kernel, lds)) return rc;
  hipLaunchKernelGGL(kernel, pieces(a.B * a.Hk, ((long long)a.x.L * a.x.G + ROWS - 1) / ROWS), dim3(64 * NW), lds, st, a);
  return hipGetLastError() == hipSuccess ? 0 : 5;
}
template <int W, int XP, int RP, bool FULL, bool KEYS> int grads_rows(const GradArgs& a, hipStream_t st) {
  return few_rows(a.B * a.Hk, (long long)a.x.L * a.x.G, W == 128 || (W == 64 && !KEYS) ? 64 : 40) ? grads<W, XP, RP, FULL, true, KEYS>(a, st)
                                                                                                     : grads<W, XP, RP, FULL, false, KEYS>(a, st);
}
template <int W, bool FULL, bool KEYS> int grads_pieces(const GradArgs& a, hipStream_t st) {
  if (a.r.X.dtype == 1 && a.x.X.dtype == 1)
    return a.x.turn.rot == 0 ? grads_rows<W, 1, 1, FULL, KEYS>(a, st) : grads_rows<W, 2, 1, FULL, KEYS>(a, st);
  return grads_rows<W, 2, 3, FULL, KEYS>(a, st);
}
template <int W, bool KEYS> int grads_width(const GradArgs& a, hipStream_t st) {
  return a.f.d == W && a.dv == W ? grads_pieces<W, true, KEYS>(a, st) : grads_pieces<W, false, KEYS>(a, st);
}
template <bool KEYS> int grads_any(const GradArgs& a, hipStream_t st) {
  switch (width_class(a.f.d, a.dv)) {
    case 32: return grads_width<32, KEYS>(a, st);
    case 64: return grads_width<64, KEYS>(a, st);
    default: return grads_width<128, KEYS>(a, st);
  }
}

}  // namespace

int launch_values(const ValueArgs& a, hipStream_t st) {
  switch (width_class(a.f.d, a.dv)) {
    case 32: return values_width<32>(a, st);
    case 64: return values_width<64>(a, st);
    default: return values_width<128>(a, st);
  }
}
int launch_query_grads(const GradArgs& a, hipStream_t st) { return grads_any<false>(a, st); }
int launch_key_grads(const GradArgs& a, hipStream_t st) { return grads_any<true>(a, st); }

}  // namespace st
}  // namespace fs
