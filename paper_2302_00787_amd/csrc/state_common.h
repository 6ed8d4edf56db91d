// What the kernels on kept states share: rows turned by their positions, operands as bf16 pieces, the buffer of projection constants.
//
// A state of a sequence and a key head is shift = max e, z_m = sum_j 2^(e_jm - shift), T_m = sum_j 2^(e_jm - shift) V_j over the keys
// appended so far, with e_jm = (W2 k_j)_m + bias_m + r(k_j) (base 2, scale of the keys and log2 e inside W2, bias and r); a query reads it
// with the features 2^((W1 q)_m + bias_m).
#pragma once
#include "fs_common.h"
#include "kernels.h"
#include "split3.h"

namespace fs {
namespace st {

typedef __attribute__((ext_vector_type(8))) float f32x8;
typedef __attribute__((ext_vector_type(4))) short s16x4;

constexpr float kNone = -__builtin_huge_valf(), kNoNumber = __builtin_nanf("");

// Widths: rows of up to 32, 64 and 128 numbers, in steps of 32 (an operand's contraction) and tiles of 16 (its columns).
template <int W> constexpr int STEPS = W / 32;
template <int W> constexpr int TILES = W / 16;
inline int width_class(int d, int dv) { const int n = d > dv ? d : dv; return n <= 32 ? 32 : (n <= 64 ? 64 : 128); }

// ---------------------------------------------------------------------------------------------- projection constants
// One block per parameter set.  Row images of W1 and W2 (the coordinates are the contraction index: [32 features][steps][2 pieces][2 tiles x
// 512 numbers]) and C2 + C2' ([coordinate tiles][steps][2][512]) are two fp16 pieces of a number: exponents and row terms need absolute
// accuracy only, so 22 bits of the largest number of a row or of 32 features do, and three products of pieces (two against bf16 rows) take half of
// what bf16 pieces need.  `scale` is what a block of 32 features (or C2 + C2') was divided by, to lie below 2^14.  Column images (the features
// are the contraction index: [32 features][coordinate tiles][3][512]) in bf16 pieces, biases (-inf behind the last feature).
struct FeaturePlan {
  int Mp, steps, tiles;          // features in 32s, steps of 32 coordinates, tiles of 16 coordinates
  size_t off_row[2], off_scale[2], off_col[2], off_csym, off_cscale, off_bias, set, total;
};
inline FeaturePlan feature_plan(int d, int M, int sets) {
  FeaturePlan p;
  p.Mp = (M + 31) / 32 * 32;
  p.steps = (d + 31) / 32;
  p.tiles = 2 * p.steps;
  auto up = [](size_t x) { return (x + 255) / 256 * 256; };
  size_t off = 0;
  for (int s = 0; s < 2; ++s) { p.off_row[s] = off; off = up(off + (size_t)p.Mp * p.steps * 2 * 32 * 2); }
  for (int s = 0; s < 2; ++s) { p.off_scale[s] = off; off = up(off + (size_t)p.Mp / 32 * 4); }
  for (int s = 0; s < 2; ++s) { p.off_col[s] = off; off = up(off + (size_t)p.Mp * p.steps * 3 * 32 * 2); }
  p.off_csym = off; off = up(off + (size_t)p.tiles * p.steps * 2 * 512 * 2);
  p.off_cscale = off; off = up(off + 4);
  p.off_bias = off; off = up(off + (size_t)p.Mp * 4);
  p.set = off;
  p.total = 256 + (size_t)sets * p.set;       // a word that says whether some C2 is dense, then the sets
  return p;
}
struct Features {
  const char* base;              // the first set
  FeaturePlan p;
  int sets, d, M;
  float scale2;                  // qk_scale^2
  int dense;
  __device__ const char* set(int h) const { return base + (sets == 1 ? 0 : (size_t)h * p.set); }
};

// ---------------------------------------------------------------------------------------------- rows
struct RotaryDev {
  const double* freqs;           // [rot / 2] radians a position
  const int32_t* positions;      // [B][L] or nullptr: row l is at position l
  long long sb, sl;
  int rot, interleaved;
  float amplitude;
};
// The angle is taken in turns and in 64 bits (position f / 2 pi, less its nearest whole number): in 32 a position of 2^20 would leave
// four bits of it.  What is left, within half a turn, goes to cosine and sine in 32 bits, and the bits that it loses there to their first-order
// correction (without it the angle alone costs 1.6 steps of 2^-24).
__device__ __forceinline__ float2 cos_sin(int position, double freq, float amplitude) {
  const double turns = (double)position * (freq * 0.15915494309189533577);        // 1 / (2 pi)
  const double halves = 2.0 * (turns - rint(turns));
  const float near = (float)halves, rest = (float)(halves - (double)near) * 3.14159265f;
  float s, c;
  sincospif(near, &s, &c);
  return make_float2(amplitude * (c - s * rest), amplitude * (s + c * rest));
}
__device__ __forceinline__ int position_of(const RotaryDev& r, int b, int l) { return r.positions ? r.positions[b * r.sb + l * r.sl] : l; }
// Positions with several axes: pair p of a row is at positions[axis_of[p]] of it (at zero where that is no axis).  axes = 0: there are none.
struct AxesDev {
  const int32_t* axis_of;        // [rot / 2]
  const int32_t* positions;
  long long sa, sb, sl;
  int axes;
};
__device__ __forceinline__ int position_of(const AxesDev& x, int axis, int b, int l) {
  return axis >= 0 && axis < x.axes ? x.positions[axis * x.sa + b * x.sb + l * x.sl] : 0;
}

// Rotary positions as the kernels on states see them: rot = 0: rows as they are.  `table` [B][L][rot / 2] holds amplitude (cos, sin).
struct Turn {
  const float2* table = nullptr;
  int rot = 0, interleaved = 0;
};
struct Rows {
  TensorDev X;
  int L, G;                      // rows of a sequence and heads (G to a state): row v is row v % L of head v / L
  const int32_t* lengths;        // [B] or nullptr
  int cols;
  Turn turn;
};
__device__ __forceinline__ int length_of(const Rows& r, int b) { return r.lengths ? max(0, min(r.lengths[b], r.L)) : r.L; }
struct RowAt { int head, row; };
__device__ __forceinline__ RowAt row_at(const Rows& r, int v) {
  const int g = r.G == 1 ? 0 : v / r.L;
  return {g, v - g * r.L};
}
__device__ __forceinline__ long long row_base(const TensorDev& t, int b, int h, int row) { return b * t.sb + h * t.sh + row * t.sl; }

// Eight numbers of a row from column c0 (a multiple of eight) on, zero from `cols` on: as they lie, so that nothing waits for them until they are
// expanded.  FULL: rows have no ragged end.
// DT: the tensor's dtype where the kernel is made for one (-1: whichever it is).
struct Raw8 { u32x4 a, b; };
template <bool FULL = false, int DT = -1> __device__ __forceinline__ Raw8 fetch8(const TensorDev& t, long long base, int c0, int cols) {
  Raw8 r{{0u, 0u, 0u, 0u}, {0u, 0u, 0u, 0u}};
  if (FULL || c0 + 8 <= cols) {
    if (DT == 0 || (DT < 0 && t.dtype == 0)) {
      r.a = *(const u32x4*)((const float*)t.ptr + base + c0);
      r.b = *(const u32x4*)((const float*)t.ptr + base + c0 + 4);
    } else {
      r.a = *(const u32x4*)((const uint16_t*)t.ptr + base + c0);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (c0 + i < cols) {
        const uint32_t v = t.dtype == 0 ? ((const uint32_t*)t.ptr)[base + c0 + i] : (uint32_t)((const uint16_t*)t.ptr)[base + c0 + i];
        if (i < 4) r.a[i] = v;
        else r.b[i - 4] = v;
      }
  }
  return r;
}
template <bool FULL = false, int DT = -1> __device__ __forceinline__ f32x8 expand8(const Raw8& r, int any_dtype, int c0, int cols) {
  f32x8 x;
  const int dtype = DT < 0 ? any_dtype : DT;
  if (dtype == 0 || (!FULL && c0 + 8 > cols)) {
    const int up = dtype == 0 ? 0 : 16;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[i] = __uint_as_float(r.a[i] << up);
      x[4 + i] = __uint_as_float(r.b[i] << up);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(r.a[i] << 16);
      x[2 * i + 1] = __uint_as_float(r.a[i] & 0xffff0000u);
    }
  }
  return x;
}
template <bool FULL = false> __device__ __forceinline__ f32x8 load8(const TensorDev& t, long long base, int c0, int cols) {
  return expand8<FULL>(fetch8<FULL>(t, base, c0, cols), t.dtype, c0, cols);
}
__device__ __forceinline__ void store8(const TensorDev& t, long long base, int c0, int cols, f32x8 x) {
  if (c0 + 8 <= cols) {
    if (t.dtype == 0) {
      float* p = (float*)t.ptr + base + c0;
      *(f32x4*)p = f32x4{x[0], x[1], x[2], x[3]};
      *(f32x4*)(p + 4) = f32x4{x[4], x[5], x[6], x[7]};
    } else {
      *(bf16x8*)((uint16_t*)t.ptr + base + c0) = __builtin_convertvector(x, bf16x8);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (c0 + i < cols) store_elem(t, base + c0 + i, x[i]);
  }
}
// x turned by the angles cs of its row: y = x cos - partner sin for the first of a pair, x cos + partner sin for the second (sgn -1: turned
// back).  other(c) gives number c of the row, other8(c0) eight of them.
template <class Other, class Other8>
__device__ __forceinline__ f32x8 turned8(f32x8 x, int c0, const Turn& t, const float2* cs, float sgn, Other other, Other8 other8) {
  if (c0 >= t.rot) return x;
  const int r = t.rot >> 1;
  f32x8 y = x;
  if (t.interleaved) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (c0 + 2 * i < t.rot) {
        const float2 a = cs[(c0 >> 1) + i];
        const float s = sgn * a.y;
        y[2 * i] = x[2 * i] * a.x - x[2 * i + 1] * s;
        y[2 * i + 1] = x[2 * i + 1] * a.x + x[2 * i] * s;
      }
  } else if ((r & 7) == 0) {
    const bool second = c0 >= r;
    const f32x8 p = other8(second ? c0 - r : c0 + r);
    const float2* a = cs + (second ? c0 - r : c0);
    const float s = second ? sgn : -sgn;
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = x[i] * a[i].x + p[i] * (s * a[i].y);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int c = c0 + i;
      if (c < t.rot) {
        const bool second = c >= r;
        const float2 a = cs[second ? c - r : c];
        y[i] = x[i] * a.x + other(second ? c - r : c + r) * ((second ? sgn : -sgn) * a.y);
      }
    }
  }
  return y;
}
// Units of eight numbers 32 s + 8 g .. of a row (s < S), turned: what a lane of group g has of an operand.  All of them are on their way before
// the first is waited for.
// live: the row is there (others are zeros; what is read for them is some row of the tensor).
template <int S, bool FULL, bool TURN, int DT = -1> struct RowUnits {
  Raw8 raw[S], other[TURN ? S : 1];
  __device__ __forceinline__ void fetch(const TensorDev& X, long long base, int cols, const Turn& turn, int g) {
    const int r = turn.rot >> 1;
    const bool whole = TURN && !turn.interleaved && (r & 7) == 0;        // (a unit's partners are a unit)
#pragma unroll
    for (int s = 0; s < S; ++s) {
      const int c0 = 32 * s + 8 * g;
      if (FULL) {
        raw[s] = fetch8<FULL, DT>(X, base, c0, cols);
      } else {
        raw[s] = Raw8{{0u, 0u, 0u, 0u}, {0u, 0u, 0u, 0u}};
        if (c0 < cols) raw[s] = fetch8<FULL, DT>(X, base, c0, cols);
      }
      if constexpr (TURN)
        if (whole && c0 < turn.rot) other[s] = fetch8<FULL, DT>(X, base, c0 >= r ? c0 - r : c0 + r, cols);
    }
  }
  __device__ __forceinline__ void finish(const TensorDev& X, long long base, int cols, const Turn& turn, const float2* cs, bool live, int g,
                                         f32x8 (&n)[S]) const {
#pragma unroll
    for (int s = 0; s < S; ++s) {
      const int c0 = 32 * s + 8 * g;
      n[s] = expand8<FULL, DT>(raw[s], X.dtype, c0, cols);
      if constexpr (TURN)
        if (c0 < turn.rot)
          n[s] = turned8(n[s], c0, turn, cs, 1.f, [&](int c) { return load_elem(X, base + c); },
                         [&](int c) { return expand8<FULL, DT>(other[s], X.dtype, c, cols); });
#pragma unroll
      for (int i = 0; i < 8; ++i) n[s][i] = live ? n[s][i] : 0.f;
    }
  }
};

// The same of a bf16 tensor that is not turned, bits as they are.
template <bool FULL>
__device__ __forceinline__ u32x4 row8_bits(const Rows& r, int b, int state_head, RowAt at, int c0) {
  if (!FULL && c0 >= r.cols) return u32x4{0u, 0u, 0u, 0u};
  const uint16_t* p = (const uint16_t*)r.X.ptr + row_base(r.X, b, state_head * r.G + at.head, at.row) + c0;
  if (FULL || c0 + 8 <= r.cols) return *(const u32x4*)p;
  u32x4 u;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    u[i] = (c0 + 2 * i < r.cols ? (uint32_t)p[2 * i] : 0u) | (c0 + 2 * i + 1 < r.cols ? (uint32_t)p[2 * i + 1] << 16 : 0u);
  return u;
}

// ---------------------------------------------------------------------------------------------- slots
// Slot of sequence b, -1 where there is none.  unique: also where an earlier sequence has the same one (for all threads of a workgroup).
__device__ __forceinline__ int slot_of(const int32_t* slots, int nslots, int b) {
  const int s = slots ? slots[b] : b;
  return s >= 0 && s < nslots ? s : -1;
}
__device__ __forceinline__ int unique_slot_of(const int32_t* slots, int nslots, int b) {
  const int s = slot_of(slots, nslots, b);
  if (slots == nullptr || s < 0) return s;
  int twice = 0;
  for (int i = threadIdx.x; i < b; i += blockDim.x) twice |= slots[i] == s;
  return __syncthreads_or(twice) ? -1 : s;
}

// ---------------------------------------------------------------------------------------------- operands
// P bf16 pieces of an operand: 1 (a bf16 number is its own piece) or 3 (24 bits).
template <int P> struct Op { bf16x8 p[P]; };
template <int P> __device__ __forceinline__ Op<P> as_op(f32x8 x) {
  Op<P> o;
  if constexpr (P == 1) {
    o.p[0] = __builtin_convertvector(x, bf16x8);
  } else {
    const Split3 s = split3(f32x4{x[0], x[1], x[2], x[3]}, f32x4{x[4], x[5], x[6], x[7]});
    o.p[0] = s.h; o.p[1] = s.m; o.p[2] = s.l;
  }
  return o;
}
template <int P> __device__ __forceinline__ Op<P> image_op(const uint16_t* img, int lane) {      // images of 512 numbers, one per piece
  Op<P> o;
#pragma unroll
  for (int i = 0; i < P; ++i) o.p[i] = *(const bf16x8*)(img + i * 512 + lane * 8);
  return o;
}

// Sum and largest over N = 4, 8, 16 or 32 neighbouring lanes: within sixteen by the lane permutations of a vector instruction.
template <int CTRL> __device__ __forceinline__ float dpp(float v) {
  return __uint_as_float(__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), CTRL, 0xf, 0xf, true));
}
template <int N, class Op2> __device__ __forceinline__ float over_lanes(float v, Op2 op) {
  v = op(v, dpp<0xb1>(v));                          // lanes 1 0 3 2 of a quad
  v = op(v, dpp<0x4e>(v));                          // 2 3 0 1
  if constexpr (N >= 8) v = op(v, dpp<0x141>(v));   // eight lanes backwards
  if constexpr (N >= 16) v = op(v, dpp<0x140>(v));  // sixteen
  if constexpr (N >= 32) v = op(v, __shfl_xor(v, 16));
  return v;
}

// fp16 pieces of the factors of an exponent (see FeaturePlan): 2, or 1 of a bf16 number.  The numbers of a row are multiplied by a power of
// two first, that of up_to_2_14, so that the largest is below 2^14; what is below 2^-39 of it is lost.
typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;
template <int P> struct Op16 { f16x8 p[P]; };
template <int P> __device__ __forceinline__ Op16<P> as_op16(f32x8 x) {
  Op16<P> o;
  o.p[0] = __builtin_convertvector(x, f16x8);
  if constexpr (P == 2) o.p[1] = __builtin_convertvector(x - __builtin_convertvector(o.p[0], f32x8), f16x8);
  return o;
}
// (2^13 <= factor * largest < 2^14; 1 where largest is zero, subnormal or not finite; the factor's inverse is a power of two, too)
__device__ __forceinline__ float up_to_2_14(float largest) {
  const int e = (int)(__float_as_uint(largest) >> 23 & 255u);
  return e == 0 || e == 255 ? 1.f : __uint_as_float((uint32_t)min(max(127 + 127 + 13 - e, 1), 253) << 23);
}
__device__ __forceinline__ float power_inverse(float p) { return __uint_as_float((254u << 23) - __float_as_uint(p)); }
__device__ __forceinline__ float largest_of(f32x8 x) {
  float m = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = fmaxf(m, fabsf(x[i]));
  return m;
}
template <int P> __device__ __forceinline__ Op<P> row_op(const uint16_t* s, int plane) {         // eight numbers of a row
  Op<P> o;
#pragma unroll
  for (int i = 0; i < P; ++i) o.p[i] = *(const bf16x8*)(s + i * plane);
  return o;
}
__device__ __forceinline__ u32x2 read_tr(const uint16_t* p) {
  return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(p)));
}
// A column of the rows 4 g .. 4 g + 3 and 16 + 4 g .. of a tile of 32 (lane l = (g, c) = (l / 16, l % 16)): the order in which two stacked
// accumulators hold their rows.  s: this lane's piece of row 4 g (see lane_tr).
template <int P> __device__ __forceinline__ Op<P> column_op(const uint16_t* s, int ld, int plane) {
  Op<P> o;
#pragma unroll
  for (int i = 0; i < P; ++i) {
    const u32x2 a = read_tr(s + i * plane), b = read_tr(s + i * plane + 16 * ld);
    o.p[i] = __builtin_bit_cast(bf16x8, u32x4{a[0], a[1], b[0], b[1]});
  }
  return o;
}
// Lanes 4 i + a of a group of sixteen name the four 8-byte pieces a of row 4 g + i; lane (a, b) = (c / 4, c % 4) gets column c of the rows.
__device__ __forceinline__ int lane_tr(int lane, int ld) { return (4 * (lane >> 4) + ((lane & 15) >> 2)) * ld + 4 * (lane & 3); }

// f(i, j) for the products of piece i of an operand of PA and piece j of one of PB that are above 2^-24 (fp16 pieces 2^-22) of it, small ones first.
// One product for all accumulators before the next: those of one accumulator wait for each other.
template <int PA, int PB, class F> __device__ __forceinline__ void each_product(F f) {
#pragma unroll
  for (int sum = (PA > PB ? PA : PB) - 1; sum >= 0; --sum)
#pragma unroll
    for (int i = PA - 1; i >= 0; --i)
      if (sum - i >= 0 && sum - i < PB) f(i, sum - i);
}
__device__ __forceinline__ f32x4 mfma(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x4 mfma(f16x8 a, f16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
// c[i][j] += a[i] b[j]
template <template <int> class O, int PA, int PB, int NA, int NB>
__device__ __forceinline__ void outer(const O<PA> (&a)[NA], const O<PB> (&b)[NB], f32x4 (&c)[NA][NB]) {
  each_product<PA, PB>([&](int pa, int pb) {
#pragma unroll
    for (int i = 0; i < NA; ++i)
#pragma unroll
      for (int j = 0; j < NB; ++j) c[i][j] = mfma(a[i].p[pa], b[j].p[pb], c[i][j]);
  });
}
// c[i][at + j] += a[i] b[j]
template <int PA, int PB, int NA, int NB, int NC>
__device__ __forceinline__ void outer_at(const Op<PA> (&a)[NA], const Op<PB> (&b)[NB], f32x4 (&c)[NA][NC], int at) {
  each_product<PA, PB>([&](int pa, int pb) {
#pragma unroll
    for (int i = 0; i < NA; ++i)
#pragma unroll
      for (int j = 0; j < NB; ++j) c[i][at + j] = mfma(a[i].p[pa], b[j].p[pb], c[i][at + j]);
  });
}

// ---------------------------------------------------------------------------------------------- arguments of the kernels
struct State {
  float *T, *z, *shift;
  int slots;
};
// Sums over rows: T[m][c] += 2^(e_vm - ref) V_v[c], z[m] += 2^(e_vm - ref) w_v.
struct BuildArgs {
  Features f;
  int side;                      // 0: features of queries, 1: of keys
  Rows x, v;
  const float* terms;            // [B*Hk][rows] row terms (nullptr: those of C2 = -I / 2); -inf: the row is left out
  const float* weights;          // [B*Hk][rows] w (nullptr: ones)
  const int32_t* slots;
  int nslots;
  int B, Hk, dv;
  int nwg;                       // (struct Shares in kernels_state.hip; the parts are nwg + B*Hk or, nwg = 0, B*Hk)
  float *part, *zpart;           // [parts][M][dv], [parts][M]
  float2* refs;                  // [parts][Mp / 16]: reference and largest exponent (-inf: nothing summed)
  int2* parts;                   // [B*Hk] number of a state's first part, and how many
  const float* shift;            // of the pool, copied to old_shift (nullptr: not)
  float* old_shift;              // [B*Hk]
};
// Workgroups of k_build that a CU holds, by the registers of its waves, and the features of one, for whole rows of 32, 64 or 128 numbers in bf16.  A
// workspace's size does not depend on the tensors, so others are counted alike: rows of 65 to 127 numbers, interleaved pairs and tensors of two
// dtypes have 128 features a workgroup at W = 128, fp32 rows LDS for one workgroup (of two) or three (of four), and these calls up to twice the
// workgroups that the chip holds at a time.
struct BuildShape { int per_cu, features; };
inline BuildShape build_shape(int d, int dv, int Mp) {
  if (width_class(d, dv) <= 64) return Mp > 64 ? BuildShape{1, 256} : BuildShape{4, 64};
  return Mp > 128 ? BuildShape{1, 256} : BuildShape{2, 128};
}
int launch_build(const BuildArgs& a, hipStream_t st);
// Partial sums onto the states (append), or their sum alone (gradients: slots that no sequence names get zeros).
struct JoinArgs {
  const float *part, *zpart;
  const float2* refs;
  const float* old_shift;        // nullptr: new states
  const int32_t* slots;
  State state;
  const int2* parts;
  int B, Hk, M, Mp, dv;
  int* left_out;
};
int launch_join(const JoinArgs& a, hipStream_t st);
int launch_join_sum(const JoinArgs& a, hipStream_t st);

// Rows against states: Y = P T / P z.
struct ValueArgs {
  Features f;
  Rows x;
  const int32_t* slots;
  State state;
  int B, Hk, dv;
  TensorDev Y;
  int* unread;                   // rows without a normaliser are added to it
};
int launch_values(const ValueArgs& a, hipStream_t st);
// Gradients of rows.  Queries: dx of Y = P T / P z for dY = r, and what the state's gradient needs of each row: -log2 of its normaliser,
// -dY . Y.  Keys: dx and dr of T = S' r, z = S' 1 for the gradients T, z of those in `state`.
struct GradArgs {
  Features f;
  Rows x, r;
  const float* shift;            // keys: [slots][Hk] of the states
  float *lse, *weights;          // queries: [B*Hk][rows]
  const int32_t* slots;
  State state;
  int B, Hk, dv;
  TensorDev dx, dr;
};
int launch_query_grads(const GradArgs& a, hipStream_t st);
int launch_key_grads(const GradArgs& a, hipStream_t st);

int launch_prepare(const float* theta, int groups, const float* Omega, int omega_groups, int sets, int d, int M, float scale, char* buf,
                   const FeaturePlan& p, hipStream_t st);
// Row terms r(k) of turned keys with a dense quadratic form, rows behind the lengths -inf.
int launch_row_terms(const Features& f, const Rows& k, int B, int Hk, float* terms, hipStream_t st);

int launch_rotary(const RotaryDev& r, const AxesDev& axes, const TensorDev& X, int H, const TensorDev& X2, int H2, int B, int L, int d, int transposed,
                  const TensorDev& Y, const TensorDev& Y2, hipStream_t st);
int launch_rotary_table(const RotaryDev& r, int B, int L, float2* table, hipStream_t st);

struct StepArgs {
  Features f;
  State state;
  const int32_t* slots;
  TensorDev Q, K, V, Y;
  int B, H, Hk, dv;
  RotaryDev rot;                 // rot = 0: rows as they are
  int* unread;
  // (launch_step's own)
  float *exps, *old_z;           // [B][Hk][1 + H / Hk][Mp] exponents of the key (less its row term) and the queries; [B][Hk][Mp]
  float2* old_shift;             // [B][Hk] shift before, the key's row term
  int key_tiles, cols;
};
size_t step_floats(int B, int H, int Hk, int d, int Mp);
int launch_step(StepArgs a, float* room, hipStream_t st);

}  // namespace st
}  // namespace fs
