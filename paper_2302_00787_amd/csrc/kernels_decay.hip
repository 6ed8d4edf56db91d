// Linear attention with a decay for each head, rows of prompts and of training: chunks of 64 rows, within a chunk by the scores of its rows,
// between chunks by the state.  See decay_common.h for the formulas.
//
// A workgroup of four waves walks the chunks of a segment of one state, 64 columns of it, whose numbers stay in the accumulators of
// the waves.  A wave has sixteen rows of x as operands (read once, from memory); it takes their scores with the chunk's rows a (LDS), weighs
// them by powers of lambda from registers, and multiplies them with the rows b, and x with the state's image (LDS).  Scores and state are fp32
// and go into the next product as PM bf16 pieces: two (16 bits) where the results are rounded to bf16 (8), three (24) otherwise.  Rows
// of a in the sums of the state are weighed in 32 bits and have three pieces, as the states themselves are results in fp32.
#include "decay_common.h"

namespace fs {
namespace dec {
namespace {

using st::Op;
using st::Raw8;
using st::f32x8;
using st::each_product;
using st::read_tr;

template <int P> __device__ __forceinline__ Op<P> pieces(f32x8 x) {
  if constexpr (P == 2) {
    Op<2> o;
    o.p[0] = __builtin_convertvector(x, bf16x8);
    o.p[1] = __builtin_convertvector(x - __builtin_convertvector(o.p[0], f32x8), bf16x8);
    return o;
  } else {
    return st::as_op<P>(x);
  }
}
template <int P> __device__ __forceinline__ f32x8 number(const Op<P>& o) {
  f32x8 x = __builtin_convertvector(o.p[P - 1], f32x8);
#pragma unroll
  for (int i = P - 2; i >= 0; --i) x += __builtin_convertvector(o.p[i], f32x8);
  return x;
}

struct Place { int b, h, seg, cb, slot, len; };
// Units of a grid: (sequence, key head, segment), their column blocks eight workgroups apart, on one XCD.  slot -2: left out.
__device__ __forceinline__ bool place(const Call& c, int nseg, int ncb, Place* p) {
  const int x = blockIdx.x, q = x / (8 * ncb), rest = x - q * 8 * ncb;
  p->cb = rest / 8;
  const long long u = (long long)q * 8 + (rest & 7);
  if (u >= (long long)c.B * c.Hk * nseg) return false;
  p->seg = (int)(u % nseg);
  const int s = (int)(u / nseg);
  p->b = s / c.Hk;
  p->h = s - p->b * c.Hk;
  p->len = c.lengths ? max(0, min(c.lengths[p->b], c.L)) : c.L;
  if (c.unique) {
    p->slot = st::unique_slot_of(c.slots, c.nslots, p->b);
    if (p->slot < 0) { p->slot = -2; p->len = 0; }
  } else {
    p->slot = st::slot_of(c.slots, c.nslots, p->b);
  }
  return true;
}

// Rows of a chunk, from memory to LDS as P bf16 pieces: 256 threads, units of eight numbers.
template <int P, int W, bool FULL, int DT> struct Stage {
  static constexpr int UNITS = W / 8, N = kChunk * UNITS / 256, LD = W + 8, PLANE = kChunk * LD;
  Raw8 raw[N];
  // rows r0 .. of the walk (n of them are there), numbers c0 .. c0 + W - 1
  __device__ __forceinline__ void fetch(const TensorDev& t, int b, int h, int r0, int n, int len, int back, int c0, int cols) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int id = threadIdx.x + 256 * i, row = id / UNITS, c = c0 + 8 * (id % UNITS);
      raw[i] = Raw8{{0u, 0u, 0u, 0u}, {0u, 0u, 0u, 0u}};
      if (row < n && c < cols) raw[i] = st::fetch8<FULL, DT>(t, st::row_base(t, b, h, back ? len - 1 - r0 - row : r0 + row), c, cols);
    }
  }
  __device__ __forceinline__ void store(uint16_t* s, int c0, int cols) const {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int id = threadIdx.x + 256 * i, row = id / UNITS, c = 8 * (id % UNITS);
      uint16_t* to = s + row * LD + c;
      if constexpr (P == 1 && FULL) {
        *(u32x4*)to = raw[i].a;
      } else {
        // (number by number: they are numbers of different rows or columns of a state)
        const f32x8 x = st::expand8<FULL, DT>(raw[i], DT, c0 + c, cols);
        if constexpr (P == 1) {
          *(bf16x8*)to = __builtin_convertvector(x, bf16x8);
        } else {
          const Split3 o = split3_each(f32x4{x[0], x[1], x[2], x[3]}, f32x4{x[4], x[5], x[6], x[7]});
          *(bf16x8*)to = o.h;
          *(bf16x8*)(to + PLANE) = o.m;
          *(bf16x8*)(to + 2 * PLANE) = o.l;
        }
      }
    }
  }
};

// Sixteen columns of rows 4 g .. 4 g + 3 of two tiles of sixteen rows (at s0 and s1).
template <int P> __device__ __forceinline__ Op<P> columns(const uint16_t* s0, const uint16_t* s1, int plane) {
  Op<P> o;
#pragma unroll
  for (int i = 0; i < P; ++i) {
    const u32x2 a = read_tr(s0 + i * plane), b = read_tr(s1 + i * plane);
    o.p[i] = __builtin_bit_cast(bf16x8, u32x4{a[0], a[1], b[0], b[1]});
  }
  return o;
}

// The part of a state that a wave holds: AT x BT tiles of 16 x 16, tile (i, j) at rows 16 (at + i), columns 16 (bt + j); lane (g, c) has
// rows 4 g .. 4 g + 3 of column c.
template <int W, int TB> struct Tiles {
  static constexpr int TA = W / 16, AT = TA >= 4 ? TA / 4 : 1, BT = TA >= 4 ? TB : TB / 2;
  int at, bt;
  __device__ __forceinline__ Tiles(int wave) : at(TA >= 4 ? wave * AT : (wave & 1)), bt(TA >= 4 ? 0 : (wave >> 1) * BT) {}
};

template <int W, int TB> using StateTiles = f32x4[Tiles<W, TB>::AT][Tiles<W, TB>::BT];

template <int W, int TB>
__device__ __forceinline__ void load_state(StateTiles<W, TB>& S, const Tiles<W, TB>& t, const float* from, int sa, int sb, int wa, int wb, int b0) {
  const int lane = threadIdx.x & 63, g = lane >> 4, c = lane & 15;
#pragma unroll
  for (int i = 0; i < Tiles<W, TB>::AT; ++i)
#pragma unroll
    for (int j = 0; j < Tiles<W, TB>::BT; ++j)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int a = 16 * (t.at + i) + 4 * g + r, b = b0 + 16 * (t.bt + j) + c;
        S[i][j][r] = from != nullptr && a < wa && b < wb ? from[(size_t)a * sa + (size_t)b * sb] : 0.f;
      }
}
template <int W, int TB>
__device__ __forceinline__ void store_state(const StateTiles<W, TB>& S, const Tiles<W, TB>& t, float* to, int sa, int sb, int wa, int wb, int b0) {
  const int lane = threadIdx.x & 63, g = lane >> 4, c = lane & 15;
#pragma unroll
  for (int i = 0; i < Tiles<W, TB>::AT; ++i)
#pragma unroll
    for (int j = 0; j < Tiles<W, TB>::BT; ++j)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int a = 16 * (t.at + i) + 4 * g + r, b = b0 + 16 * (t.bt + j) + c;
        if (a < wa && b < wb) to[(size_t)a * sa + (size_t)b * sb] = S[i][j][r];
      }
}

// Weights of a chunk's n rows in the sums of a state: lambda^(n - j - first) of rows j = 32 q + 4 g + r and 32 q + 16 + 4 g + r.
__device__ __forceinline__ void update_weights(f32x8 (&w)[2], const float* pw, int n, int first, float scale) {
  const int g = (threadIdx.x & 63) >> 4;
#pragma unroll
  for (int q = 0; q < 2; ++q)
#pragma unroll
    for (int r = 0; r < 8; ++r) w[q][r] = scale * pw[max(0, n - first - (32 * q + 16 * (r >> 2) + 4 * g + (r & 3)))];
}
// S += sum over the chunk's rows of w a b'
template <int P, int W, int TB>
__device__ __forceinline__ void add_chunk(StateTiles<W, TB>& S, const Tiles<W, TB>& t, const uint16_t* sa, const uint16_t* sb, const f32x8 (&w)[2]) {
  constexpr int LDA = W + 8, LDB = 16 * TB + 8, PA = kChunk * LDA, PB = kChunk * LDB, AT = Tiles<W, TB>::AT, BT = Tiles<W, TB>::BT;
  const int lane = threadIdx.x & 63;
  const uint16_t *la = sa + st::lane_tr(lane, LDA), *lb = sb + st::lane_tr(lane, LDB);
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    Op<3> a[AT];
#pragma unroll
    for (int i = 0; i < AT; ++i) {
      const uint16_t* p = la + 32 * q * LDA + 16 * (t.at + i);
      a[i] = st::as_op<3>(number<P>(columns<P>(p, p + 16 * LDA, PA)) * w[q]);
    }
#pragma unroll
    for (int j = 0; j < BT; ++j) {
      const uint16_t* p = lb + 32 * q * LDB + 16 * (t.bt + j);
      const Op<P> b = columns<P>(p, p + 16 * LDB, PB);
      each_product<3, P>([&](int x, int y) {
#pragma unroll
        for (int i = 0; i < AT; ++i) S[i][j] = st::mfma(a[i].p[x], b.p[y], S[i][j]);
      });
    }
  }
}

// ------------------------------------------------------------------------------------------------ rows
template <int P, int PM, int W, int TB, bool FULL, int DT>
__global__ void __launch_bounds__(256) k_decay_walk(WalkSet set, int ncb) {
  constexpr int NB = 16 * TB, STEPS = W / 32, LDA = W + 8, LDB = NB + 8, PA = kChunk * LDA, PB = kChunk * LDB;
  constexpr int IMG = STEPS * PM * 512;                       // numbers of one column tile of the state's image
  extern __shared__ char lds[];
  uint16_t *sa = (uint16_t*)lds, *sb = sa + P * PA, *img = sb + P * PB;
  float* pw = (float*)(img + TB * IMG);                       // lambda^0 .. lambda^64
  const Call& c = set.c;
  const Walk& w = set.w[blockIdx.y];
  Place p;
  if (!place(c, c.nseg, ncb, &p)) return;
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, g = lane >> 4, col = lane & 15, b0 = 64 * p.cb;
  if (b0 >= w.wb) return;
  if (c.left_out && p.slot == -2 && p.h == 0 && p.cb == 0 && p.seg == 0 && tid == 0 && blockIdx.y == 0) atomicAdd(c.left_out, 1);
  const int lo = p.seg * c.seg_rows, hi = min(p.len, lo + c.seg_rows);
  // rows behind the sequence
  const int pad0 = max(lo, p.len), pad1 = p.seg == c.nseg - 1 ? c.L : min(c.L, lo + c.seg_rows);
  if (pad0 < pad1) {
    const int nb = min(64, w.wb - b0), per = (pad1 - pad0) * nb;
    for (int gx = 0; gx < w.GX; ++gx)
      for (int id = tid; id < per; id += 256) {
        const int row = id / nb;
        store_elem(w.Y, st::row_base(w.Y, p.b, p.h * w.GX + gx, pad0 + row) + b0 + id - row * nb, 0.f);
      }
  }
  const int s = p.b * c.Hk + p.h;
  const bool ends = w.end != nullptr && c.nseg == 1 && (p.slot >= 0 || !w.end_pool);
  if (hi <= lo && !ends) return;
  const float ld = c.log_decay[p.h];
  for (int i = tid; i <= kChunk; i += 256) pw[i] = power(ld, i);
  const Keep whole = keep_of(ld, kChunk);
  const Tiles<W, TB> t(wave);
  StateTiles<W, TB> S;
  // (with segments the pool may hold the states after the call already)
  const float* from = w.init == nullptr && p.seg == 0 ? nullptr
                      : c.nseg > 1                    ? set.prefix[blockIdx.y] + ((size_t)s * c.nseg + p.seg) * c.state
                                                      : (p.slot >= 0 ? w.init + ((size_t)p.slot * c.Hk + p.h) * c.state : nullptr);
  load_state<W, TB>(S, t, from, w.sa, w.sb, w.wa, w.wb, b0);
  bool filled = from != nullptr;
  __syncthreads();
  f32x4 near[4];
#pragma unroll
  for (int q = 0; q < 4; ++q)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int n = 16 * q + col - 4 * g - r;
      near[q][r] = n >= 0 ? w.s_score * pw[max(n, 0)] : 0.f;
    }
  const float inter = w.s_inter * pw[16 * wave + col + w.first];
  f32x8 uw[2];
  update_weights(uw, pw, kChunk, w.first, w.s_update);

  auto put_image = [&]() {
#pragma unroll
    for (int i = 0; i < Tiles<W, TB>::AT; ++i)
#pragma unroll
      for (int j = 0; j < Tiles<W, TB>::BT; ++j) {
        const int a = 16 * (t.at + i) + 4 * g;
        uint16_t* to = img + (t.bt + j) * IMG + (a >> 5) * PM * 512 + ((((a & 31) >> 3) * 16 + col) * 8 + (a & 7));
        f32x4 x = S[i][j];
#pragma unroll
        for (int k = 0; k < PM; ++k) {
          typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4;
          const bf16x4 h = __builtin_convertvector(x, bf16x4);
          *(bf16x4*)(to + k * 512) = h;
          x -= __builtin_convertvector(h, f32x4);
        }
      }
  };

  Stage<P, W, FULL, DT> ra;
  Stage<P, NB, FULL, DT> rb;
  Raw8 rx[STEPS];
  auto fetch_x = [&](int r0, int gx) {
    const int row = r0 + 16 * wave + col;
#pragma unroll
    for (int k = 0; k < STEPS; ++k) {
      const int c0 = 32 * k + 8 * g;
      rx[k] = Raw8{{0u, 0u, 0u, 0u}, {0u, 0u, 0u, 0u}};
      if (row < hi && c0 < w.wa)
        rx[k] = st::fetch8<FULL, DT>(w.X, st::row_base(w.X, p.b, p.h * w.GX + gx, w.back ? p.len - 1 - row : row), c0, w.wa);
    }
  };
  auto fetch_rows = [&](int r0, int ga) {
    const int n = min(kChunk, hi - r0);
    ra.fetch(w.A, p.b, p.h * w.GA + ga, r0, n, p.len, w.back, 0, w.wa);
    rb.fetch(w.B, p.b, p.h * w.GA + ga, r0, n, p.len, w.back, b0, w.wb);
  };
  if (lo < hi) { fetch_rows(lo, 0); fetch_x(lo, 0); }
  if (filled) put_image();
  Op<P> x[STEPS];
  f32x4 acc[TB];
  for (int r0 = lo; r0 < hi; r0 += kChunk) {
    const int n = min(kChunk, hi - r0);
    const bool more = r0 + kChunk < hi, update = more || ends;
    for (int ga = 0; ga < w.GA; ++ga) {
      ra.store(sa, 0, w.wa);
      rb.store(sb, b0, w.wb);
      __syncthreads();
      if (ga + 1 < w.GA) fetch_rows(r0, ga + 1);
      else if (more) fetch_rows(r0 + kChunk, 0);
      for (int gx = 0; gx < w.GX; ++gx) {
        if (ga == 0) {
#pragma unroll
          for (int k = 0; k < STEPS; ++k) {
            if constexpr (P == 1 && FULL) x[k].p[0] = __builtin_bit_cast(bf16x8, rx[k].a);
            else x[k] = st::as_op<P>(st::expand8<FULL, DT>(rx[k], DT, 32 * k + 8 * g, w.wa));
          }
          if (gx + 1 < w.GX) fetch_x(r0, gx + 1);
          else if (more) fetch_x(r0 + kChunk, 0);
#pragma unroll
          for (int j = 0; j < TB; ++j) acc[j] = f32x4{0.f, 0.f, 0.f, 0.f};
          if (filled) {
#pragma unroll
            for (int k = 0; k < STEPS; ++k)
#pragma unroll
              for (int j = 0; j < TB; ++j) {
                const Op<PM> o = st::image_op<PM>(img + j * IMG + k * PM * 512, lane);
                each_product<PM, P>([&](int m, int y) { acc[j] = st::mfma(o.p[m], x[k].p[y], acc[j]); });
              }
#pragma unroll
            for (int j = 0; j < TB; ++j) acc[j] *= inter;
          }
        }
        // scores with the tiles of rows wave, wave - 1, ... two at a time
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          const int j0 = wave - 2 * q, j1 = max(j0 - 1, 0);
          if (j0 < 0 || 16 * j0 >= n) continue;
          f32x4 sc[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
          for (int k = 0; k < STEPS; ++k) {
            const Op<P> o0 = st::row_op<P>(sa + (16 * j0 + col) * LDA + 32 * k + 8 * g, PA);
            const Op<P> o1 = st::row_op<P>(sa + (16 * j1 + col) * LDA + 32 * k + 8 * g, PA);
            each_product<P, P>([&](int m, int y) {
              sc[0] = st::mfma(o0.p[m], x[k].p[y], sc[0]);
              sc[1] = st::mfma(o1.p[m], x[k].p[y], sc[1]);
            });
          }
          f32x8 v;
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            v[r] = q > 0 || col >= 4 * g + r ? sc[0][r] * near[2 * q][r] : 0.f;
            v[4 + r] = j0 > 0 ? sc[1][r] * near[2 * q + 1][r] : 0.f;
          }
          const Op<PM> o = pieces<PM>(v);
          const uint16_t* lb = sb + st::lane_tr(lane, LDB);
#pragma unroll
          for (int j = 0; j < TB; ++j) {
            const Op<P> bt = columns<P>(lb + 16 * j0 * LDB + 16 * j, lb + 16 * j1 * LDB + 16 * j, PB);
            each_product<P, PM>([&](int m, int y) { acc[j] = st::mfma(bt.p[m], o.p[y], acc[j]); });
          }
        }
        const int row = r0 + 16 * wave + col;
        if (ga == w.GA - 1 && row < hi) {
          const long long to = st::row_base(w.Y, p.b, p.h * w.GX + gx, w.back ? p.len - 1 - row : row);
#pragma unroll
          for (int j = 0; j < TB; ++j) {
            const int b = b0 + 16 * j + 4 * g;
            if (FULL ? b < w.wb : b + 4 <= w.wb) {
              if (w.Y.dtype == 0) {
                *(f32x4*)((float*)w.Y.ptr + to + b) = acc[j];
              } else {
                typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4;
                *(bf16x4*)((uint16_t*)w.Y.ptr + to + b) = __builtin_convertvector(acc[j], bf16x4);
              }
            } else if (!FULL) {
#pragma unroll
              for (int r = 0; r < 4; ++r)
                if (b + r < w.wb) store_elem(w.Y, to + b + r, acc[j][r]);
            }
          }
        }
      }
      if (update) {
        if (n < kChunk) update_weights(uw, pw, n, w.first, w.s_update);
        if (ga == 0) {
          const Keep keep = n < kChunk ? keep_of(ld, n) : whole;
#pragma unroll
          for (int i = 0; i < Tiles<W, TB>::AT; ++i)
#pragma unroll
            for (int j = 0; j < Tiles<W, TB>::BT; ++j)
#pragma unroll
              for (int r = 0; r < 4; ++r) S[i][j][r] = kept(keep, S[i][j][r]);
        }
        add_chunk<P, W, TB>(S, t, sa, sb, uw);
      }
      __syncthreads();
    }
    if (more) { put_image(); filled = true; }
  }
  if (ends)
    store_state<W, TB>(S, t, w.end + (w.end_pool ? (size_t)p.slot * c.Hk + p.h : (size_t)s) * c.state, w.sa, w.sb, w.wa, w.wb, b0);
}

// ------------------------------------------------------------------------------------------------ sums of segments
template <int P, int W, int TB, bool FULL, int DT>
__global__ void __launch_bounds__(256) k_decay_sum(SumSet set, int ncb) {
  constexpr int NB = 16 * TB, PA = kChunk * (W + 8), PB = kChunk * (NB + 8);
  extern __shared__ char lds[];
  uint16_t *sa = (uint16_t*)lds, *sb = sa + P * PA;
  float* pw = (float*)(sb + P * PB);
  const Call& c = set.c;
  const Walk& w = set.w[blockIdx.y];
  Place p;
  const int wanted = set.last ? c.nseg : c.nseg - 1;
  if (!place(c, wanted, ncb, &p)) return;
  const int tid = threadIdx.x, b0 = 64 * p.cb;
  const int lo = p.seg * c.seg_rows, hi = min(p.len, lo + c.seg_rows);
  if (hi <= lo || b0 >= w.wb) return;
  const float ld = c.log_decay[p.h];
  for (int i = tid; i <= kChunk; i += 256) pw[i] = power(ld, i);
  const Keep whole = keep_of(ld, kChunk);
  const Tiles<W, TB> t(tid >> 6);
  StateTiles<W, TB> S;
  load_state<W, TB>(S, t, nullptr, 0, 0, 0, 0, 0);
  __syncthreads();
  f32x8 uw[2];
  update_weights(uw, pw, kChunk, w.first, w.s_update);
  Stage<P, W, FULL, DT> ra;
  Stage<P, NB, FULL, DT> rb;
  auto fetch_rows = [&](int r0, int ga) {
    const int n = min(kChunk, hi - r0);
    ra.fetch(w.A, p.b, p.h * w.GA + ga, r0, n, p.len, w.back, 0, w.wa);
    rb.fetch(w.B, p.b, p.h * w.GA + ga, r0, n, p.len, w.back, b0, w.wb);
  };
  fetch_rows(lo, 0);
  for (int r0 = lo; r0 < hi; r0 += kChunk) {
    const int n = min(kChunk, hi - r0);
    if (n < kChunk) update_weights(uw, pw, n, w.first, w.s_update);
    for (int ga = 0; ga < w.GA; ++ga) {
      ra.store(sa, 0, w.wa);
      rb.store(sb, b0, w.wb);
      __syncthreads();
      if (ga + 1 < w.GA) fetch_rows(r0, ga + 1);
      else if (r0 + kChunk < hi) fetch_rows(r0 + kChunk, 0);
      if (ga == 0 && r0 > lo) {
        const Keep keep = n < kChunk ? keep_of(ld, n) : whole;
#pragma unroll
        for (int i = 0; i < Tiles<W, TB>::AT; ++i)
#pragma unroll
          for (int j = 0; j < Tiles<W, TB>::BT; ++j)
#pragma unroll
            for (int r = 0; r < 4; ++r) S[i][j][r] = kept(keep, S[i][j][r]);
      }
      add_chunk<P, W, TB>(S, t, sa, sb, uw);
      __syncthreads();
    }
  }
  const size_t s = (size_t)p.b * c.Hk + p.h;
  store_state<W, TB>(S, t, set.part[blockIdx.y] + (s * c.nseg + p.seg) * c.state, w.sa, w.sb, w.wa, w.wb, b0);
}

// Sums of the segments -> states before them, in place; eight segments on their way at a time.
__global__ void __launch_bounds__(256) k_decay_join(JoinSet set) {
  const Call& c = set.c;
  const int which = blockIdx.z, s = blockIdx.y, b = s / c.Hk, h = s - b * c.Hk;
  int len = c.lengths ? max(0, min(c.lengths[b], c.L)) : c.L, slot;
  if (c.unique) {
    slot = st::unique_slot_of(c.slots, c.nslots, b);
    if (slot < 0) { slot = -2; len = 0; }
  } else {
    slot = st::slot_of(c.slots, c.nslots, b);
  }
  const int id = blockIdx.x * 256 + threadIdx.x;
  if (id >= c.state) return;
  const float ld = c.log_decay[h];
  const float* init = set.init[which];
  float S = init != nullptr && slot >= 0 ? init[((size_t)slot * c.Hk + h) * c.state + id] : 0.f;
  float* part = set.part[which] + (size_t)s * c.nseg * c.state + id;
  const Keep whole = keep_of(ld, c.seg_rows);
  for (int s0 = 0; s0 < c.nseg; s0 += 8) {
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const bool there = s0 + i < c.nseg && (long long)(s0 + i) * c.seg_rows < len && (s0 + i < c.nseg - 1 || set.end[which] != nullptr);
      v[i] = there ? part[(size_t)(s0 + i) * c.state] : 0.f;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (s0 + i >= c.nseg) continue;
      const long long at = (long long)(s0 + i) * c.seg_rows;
      if (at >= len) continue;
      part[(size_t)(s0 + i) * c.state] = S;
      const int n = (int)min((long long)c.seg_rows, len - at);
      S = kept(n < c.seg_rows ? keep_of(ld, n) : whole, S) + v[i];
    }
  }
  if (set.end[which] != nullptr && (slot >= 0 || !set.end_pool[which]))
    set.end[which][(set.end_pool[which] ? (size_t)slot * c.Hk + h : (size_t)s) * c.state + id] = S;
}

// The readers of a slot are found once for 1024 numbers of its states, in the order of the sequences.
__global__ void __launch_bounds__(256) k_decay_slot_sums(Call c, const float* each, float* pool) {
  __shared__ int list[256], count[4];
  const int slot = blockIdx.y / c.Hk, h = blockIdx.y - slot * c.Hk, tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  float sum[4] = {0.f, 0.f, 0.f, 0.f};
  const int id = blockIdx.x * 1024 + tid;
  bool found = false;
  for (int b0 = 0; b0 < c.B; b0 += 256) {
    const int b = b0 + tid;
    const bool reads = b < c.B && st::slot_of(c.slots, c.nslots, b) == slot;
    const unsigned long long m = __ballot(reads);
    if (lane == 0) count[wave] = __popcll(m);
    __syncthreads();
    int before = __popcll(m & ((1ull << lane) - 1)), total = 0;
    for (int i = 0; i < 4; ++i) {
      before += i < wave ? count[i] : 0;
      total += count[i];
    }
    if (reads) list[before] = b;
    __syncthreads();
    if (c.unique) total = found ? 0 : min(total, 1);          // the first sequence of a slot alone had it
    for (int i = 0; i < total; ++i) {
      const float* from = each + ((size_t)list[i] * c.Hk + h) * c.state;
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (id + 256 * k < c.state) sum[k] += from[id + 256 * k];
    }
    found = found || total > 0;
    __syncthreads();
  }
  float* to = pool + ((size_t)slot * c.Hk + h) * c.state;
#pragma unroll
  for (int k = 0; k < 4; ++k)
    if (id + 256 * k < c.state) to[id + 256 * k] = sum[k];
}

int status() { return hipGetLastError() == hipSuccess ? 0 : 5; }

// More LDS than a launch has by itself is asked for once for a kernel and device.
template <class K> int room(K kernel, size_t bytes) {
  if (bytes <= 65536) return 0;
  return hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes) == hipSuccess ? 0 : 5;
}

template <int P, int PM, int W, int TB, bool FULL, int DT>
int walk_launch(const WalkSet& a, int count, hipStream_t st) {
  int ncb = 1;
  for (int i = 0; i < count; ++i) ncb = max(ncb, (a.w[i].wb + 16 * TB - 1) / (16 * TB));
  const size_t lds = (size_t)P * kChunk * (W + 8 + 16 * TB + 8) * 2 + (size_t)TB * (W / 32) * PM * 1024 + 68 * 4;
  if (int rc = room(k_decay_walk<P, PM, W, TB, FULL, DT>, lds)) return rc;
  const long long units = ((long long)a.c.B * a.c.Hk * a.c.nseg + 7) / 8 * 8;
  if (units * ncb > 0x7fffffffLL) return 2;
  hipLaunchKernelGGL((k_decay_walk<P, PM, W, TB, FULL, DT>), dim3((unsigned)(units * ncb), count), dim3(256), lds, st, a, ncb);
  return status();
}
template <int P, int W, int TB, bool FULL, int DT>
int sum_launch(const SumSet& a, int count, hipStream_t st) {
  int ncb = 1;
  for (int i = 0; i < count; ++i) ncb = max(ncb, (a.w[i].wb + 16 * TB - 1) / (16 * TB));
  const size_t lds = (size_t)P * kChunk * (W + 8 + 16 * TB + 8) * 2 + 68 * 4;
  if (int rc = room(k_decay_sum<P, W, TB, FULL, DT>, lds)) return rc;
  const long long units = ((long long)a.c.B * a.c.Hk * (a.last ? a.c.nseg : a.c.nseg - 1) + 7) / 8 * 8;
  if (units == 0) return 0;
  if (units * ncb > 0x7fffffffLL) return 2;
  hipLaunchKernelGGL((k_decay_sum<P, W, TB, FULL, DT>), dim3((unsigned)(units * ncb), count), dim3(256), lds, st, a, ncb);
  return status();
}

int class_of(int n) { return n <= 32 ? 32 : (n <= 64 ? 64 : 128); }

template <int P, int PM, bool FULL, int DT> int walk_width(const WalkSet& a, int count, int wa, int wb, hipStream_t st) {
  if (class_of(wa) == 128) return walk_launch<P, PM, 128, 4, FULL, DT>(a, count, st);
  if (class_of(wa) == 64) return walk_launch<P, PM, 64, 4, FULL, DT>(a, count, st);
  return wb <= 32 ? walk_launch<P, PM, 32, 2, FULL, DT>(a, count, st) : walk_launch<P, PM, 32, 4, FULL, DT>(a, count, st);
}
template <int P, bool FULL, int DT> int sum_width(const SumSet& a, int count, int wa, int wb, hipStream_t st) {
  if (class_of(wa) == 128) return sum_launch<P, 128, 4, FULL, DT>(a, count, st);
  if (class_of(wa) == 64) return sum_launch<P, 64, 4, FULL, DT>(a, count, st);
  return wb <= 32 ? sum_launch<P, 32, 2, FULL, DT>(a, count, st) : sum_launch<P, 32, 4, FULL, DT>(a, count, st);
}

}  // namespace

// Walks from .. from + count - 1 in one launch.  fine: results in fp32.
int launch_walks(const WalkSet& all, int from, int count, int dtype, bool fine, hipStream_t st) {
  WalkSet a = all;
  int wa = 0, wb = 0;
  bool full = true;
  for (int i = 0; i < count; ++i) {
    a.w[i] = all.w[from + i];
    a.prefix[i] = all.prefix[from + i];
    wa = max(wa, a.w[i].wa);
    wb = max(wb, a.w[i].wb);
    full = full && a.w[i].wa % 8 == 0 && a.w[i].wb % 8 == 0;
  }
  if (dtype == 0) return full ? walk_width<3, 3, true, 0>(a, count, wa, wb, st) : walk_width<3, 3, false, 0>(a, count, wa, wb, st);
  if (fine) return full ? walk_width<1, 3, true, 1>(a, count, wa, wb, st) : walk_width<1, 3, false, 1>(a, count, wa, wb, st);
  return full ? walk_width<1, 2, true, 1>(a, count, wa, wb, st) : walk_width<1, 2, false, 1>(a, count, wa, wb, st);
}

int launch_sums(const SumSet& a, int count, int dtype, hipStream_t st) {
  int wa = 0, wb = 0;
  bool full = true;
  for (int i = 0; i < count; ++i) {
    wa = max(wa, a.w[i].wa);
    wb = max(wb, a.w[i].wb);
    full = full && a.w[i].wa % 8 == 0 && a.w[i].wb % 8 == 0;
  }
  if (dtype == 0) return full ? sum_width<3, true, 0>(a, count, wa, wb, st) : sum_width<3, false, 0>(a, count, wa, wb, st);
  return full ? sum_width<1, true, 1>(a, count, wa, wb, st) : sum_width<1, false, 1>(a, count, wa, wb, st);
}

int launch_join(const JoinSet& a, hipStream_t st) {
  hipLaunchKernelGGL(k_decay_join, dim3((a.c.state + 255) / 256, a.c.B * a.c.Hk, a.count), dim3(256), 0, st, a);
  return status();
}

int launch_slot_sums(const Call& c, const float* each, float* pool, hipStream_t st) {
  hipLaunchKernelGGL(k_decay_slot_sums, dim3((c.state + 1023) / 1024, c.nslots * c.Hk), dim3(256), 0, st, c, each, pool);
  return status();
}

}  // namespace dec
}  // namespace fs
