// Linear attention with a decay for each head, rows of prompts and of training: chunks of 64 rows, within a chunk by the scores of its rows,
// between chunks by the state.  See decay_common.h for the formulas.
//
// A workgroup of four waves walks the chunks of a segment of one state, 64 columns of it, whose numbers stay in the accumulators of
// the waves.  A wave has sixteen rows of x as operands (read once, from memory); it takes their scores with the chunk's rows a (LDS), weighs
// them by powers of lambda from registers, and multiplies them with the rows b, and x with the state's image (LDS).  Scores and state are fp32
// and go into the next product as PM bf16 pieces: two (16 bits) where the results are rounded to bf16 (8), three (24) otherwise.  Rows
// of a in the sums of the state are weighed in 32 bits and have three pieces, as the states themselves are results in fp32.
#include "decay_common.h"

#include <type_traits>

namespace fs {
namespace dec {
namespace {

using st::Op;
using st::Raw8;
using st::f32x8;
using st::each_product;
using st::read_tr;

__device__ __forceinline__ int wave_id() { return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); }      // (a scalar: branches on it, too)
__device__ __forceinline__ float scalar(float x) { return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(x))); }
__device__ __forceinline__ Keep scalar(Keep k) { return {scalar(k.part), __builtin_amdgcn_readfirstlane((int)k.near) != 0}; }

__device__ __forceinline__ void scale_by(f32x4& v, float f) {       // (one register for the factor, where v *= f takes four)
#pragma unroll
  for (int r = 0; r < 4; ++r) v[r] *= f;
}

// Operands of a part of a chunk are not fetched before the part: that would take registers that hold more waves otherwise.
__device__ __forceinline__ void phase() { __builtin_amdgcn_sched_barrier(0); }

template <int P> __device__ __forceinline__ Op<P> pieces(f32x8 x) {
  if constexpr (P == 2) {          // (numbers that are summed: one that is not finite makes its neighbour NaN)
    u32x4 h, m;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const f32x2_t v = {x[2 * i], x[2 * i + 1]};
      const bf16x2_t top = __builtin_convertvector(v, bf16x2_t);
      h[i] = __builtin_bit_cast(uint32_t, top);
      m[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(less_piece(v, top), bf16x2_t));
    }
    Op<2> o;
    o.p[0] = __builtin_bit_cast(bf16x8, h);
    o.p[1] = __builtin_bit_cast(bf16x8, m);
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
  int len = c.lengths ? max(0, min(c.lengths[p->b], c.L)) : c.L, slot;
  if (c.unique) {
    slot = st::unique_slot_of(c.slots, c.nslots, p->b);
    if (slot < 0) { slot = -2; len = 0; }
  } else {
    slot = st::slot_of(c.slots, c.nslots, p->b);
  }
  p->len = __builtin_amdgcn_readfirstlane(len);          // (the same in all lanes; addresses are to be scalar)
  p->slot = __builtin_amdgcn_readfirstlane(slot);
  return true;
}

// A chunk's n rows of one head: `at` is their lowest in memory, row i at i pitch (back: (n - 1 - i) pitch) bytes.
struct Chunk {
  const char* at;
  int n, pitch, back;
  // offset of row i where there are kChunk rows -> the present one; rows from n on get offsets that are out of the buffer
  __device__ __forceinline__ int shift() const { return back ? (kChunk - n) * pitch : 0; }
  __device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer() const {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(at), 0, n * pitch, 0x00027000);
  }
};
// Offsets from here on, and those less a shift, are out of every buffer: reads give zeros, writes nothing.  (kChunk pitches are at most 2^30.)
constexpr int kNowhere = (int)0x80000000u;
// A head's rows (of `heads` consecutive ones), and a chunk's of them.
struct Head {
  const char* at;
  long long next;                // bytes from head to head
  int pitch;
  __device__ __forceinline__ Head(const TensorDev& t, int b, int h) {
    const int size = t.dtype == 0 ? 4 : 2;
    at = (const char*)t.ptr + st::row_base(t, b, h, 0) * size;
    next = t.sh * size;
    pitch = (int)t.sl * size;
  }
  __device__ __forceinline__ Chunk chunk(int i, int r0, int n, int len, int back) const {
    return {at + i * next + (long long)(back ? len - r0 - n : r0) * pitch, n, pitch, back};
  }
};
typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4;

// From memory to LDS as P bf16 pieces: 256 threads, units of eight numbers.  FULL: rows have no ragged end, and units are loads whose
// offsets from the chunk's first row stay; else number by number at the ends.
template <int P, int W, bool FULL, int DT> struct Stage {
  static constexpr int UNITS = W / 8, N = kChunk * UNITS / 256, LD = W + 8, PLANE = kChunk * LD, SIZE = DT == 0 ? 4 : 2;
  Raw8 raw[N];
  int off[N], c, cols;
  // numbers c0 .. c0 + W - 1 of the rows
  __device__ __forceinline__ Stage(const Head& h, int c0, int ncols, int back) : cols(ncols) {
    c = c0 + 8 * (threadIdx.x % UNITS);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int row = (threadIdx.x + 256 * i) / UNITS;
      off[i] = c < cols ? (back ? kChunk - 1 - row : row) * h.pitch + c * SIZE : kNowhere;
    }
  }
  __device__ __forceinline__ void fetch(const Chunk& k) {
    const int shift = k.shift();
    if constexpr (FULL) {
      const __amdgpu_buffer_rsrc_t r = k.buffer();
#pragma unroll
      for (int i = 0; i < N; ++i) {
        raw[i].a = __builtin_amdgcn_raw_buffer_load_b128(r, off[i] - shift, 0, 0);
        if constexpr (DT == 0) raw[i].b = __builtin_amdgcn_raw_buffer_load_b128(r, off[i] - shift, 16, 0);
      }
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        raw[i] = Raw8{{0u, 0u, 0u, 0u}, {0u, 0u, 0u, 0u}};
        if (c < cols && (unsigned)(off[i] - shift) < (unsigned)(k.n * k.pitch))
          raw[i] = st::fetch8<FULL, DT>(TensorDev{k.at + (off[i] - shift - c * SIZE), DT, 0, 0, 0}, 0, c, cols);
      }
    }
  }
  __device__ __forceinline__ void store(uint16_t* s, int c0) const {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      uint16_t* to = s + (threadIdx.x + 256 * i) / UNITS * LD + (c - c0);
      if constexpr (P == 1 && FULL) {
        *(u32x4*)to = raw[i].a;
      } else {
        // (number by number: they are numbers of different rows or columns of a state)
        const f32x8 x = st::expand8<FULL, DT>(raw[i], DT, c, cols);
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

// A wave's sixteen rows as operands: a lane has eight numbers 32 k + 8 g .. of row 16 wave + (lane % 16) for each step k, or (PERM) numbers
// 32 k + 4 g .. and 32 k + 16 + 4 g .., the order in which two stacked accumulators hold theirs.
template <int P, int STEPS, bool FULL, int DT, bool PERM = false> struct RowOps {
  static constexpr int SIZE = DT == 0 ? 4 : 2, PARTS = PERM ? 2 : 1;
  Raw8 raw[STEPS];
  int row, off[STEPS][PARTS], cols;
  __device__ __forceinline__ RowOps(const Head& h, int ncols, int back) : cols(ncols) {
    const int g = (threadIdx.x & 63) >> 4, i = 16 * wave_id() + (threadIdx.x & 15);
    row = (back ? kChunk - 1 - i : i) * h.pitch;
#pragma unroll
    for (int k = 0; k < STEPS; ++k)
#pragma unroll
      for (int j = 0; j < PARTS; ++j) {
        const int c = 32 * k + (PERM ? 16 * j + 4 * g : 8 * g);
        off[k][j] = c < cols ? row + c * SIZE : kNowhere;
      }
  }
  __device__ __forceinline__ void fetch(const Chunk& k) {
    const int g = (threadIdx.x & 63) >> 4, shift = k.shift();
    if constexpr (FULL) {
      const __amdgpu_buffer_rsrc_t r = k.buffer();
#pragma unroll
      for (int i = 0; i < STEPS; ++i) {
        if constexpr (!PERM) {
          raw[i].a = __builtin_amdgcn_raw_buffer_load_b128(r, off[i][0] - shift, 0, 0);
          if constexpr (DT == 0) raw[i].b = __builtin_amdgcn_raw_buffer_load_b128(r, off[i][0] - shift, 16, 0);
        } else if constexpr (DT == 0) {
          raw[i].a = __builtin_amdgcn_raw_buffer_load_b128(r, off[i][0] - shift, 0, 0);
          raw[i].b = __builtin_amdgcn_raw_buffer_load_b128(r, off[i][PARTS - 1] - shift, 0, 0);
        } else {
          const u32x2 x = __builtin_amdgcn_raw_buffer_load_b64(r, off[i][0] - shift, 0, 0), y = __builtin_amdgcn_raw_buffer_load_b64(r, off[i][PARTS - 1] - shift, 0, 0);
          raw[i].a = u32x4{x[0], x[1], y[0], y[1]};
        }
      }
    } else {
      const bool there = (unsigned)(row - shift) < (unsigned)(k.n * k.pitch);
      const TensorDev t{k.at + (there ? row - shift : 0), DT, 0, 0, 0};
#pragma unroll
      for (int i = 0; i < STEPS; ++i) {
        raw[i] = Raw8{{0u, 0u, 0u, 0u}, {0u, 0u, 0u, 0u}};
        if constexpr (!PERM) {
          if (there && 32 * i + 8 * g < cols) raw[i] = st::fetch8<FULL, DT>(t, 0, 32 * i + 8 * g, cols);
        } else {
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const int n = 32 * i + 16 * (j >> 2) + 4 * g + (j & 3);
            if (there && n < cols) {
              const uint32_t v = __float_as_uint(load_elem(t, n));
              if (j < 4) raw[i].a[j] = v;
              else raw[i].b[j - 4] = v;
            }
          }
        }
      }
    }
  }
  __device__ __forceinline__ void ops(Op<P> (&x)[STEPS]) const {
    const int g = (threadIdx.x & 63) >> 4;
#pragma unroll
    for (int i = 0; i < STEPS; ++i) {
      if constexpr (P == 1 && FULL) x[i].p[0] = __builtin_bit_cast(bf16x8, raw[i].a);
      else if constexpr (PERM && !FULL) x[i] = st::as_op<P>(st::expand8<false, 0>(raw[i], 0, 0, 8));
      else x[i] = st::as_op<P>(st::expand8<FULL, DT>(raw[i], DT, 32 * i + 8 * g, cols));
    }
  }
};

// Numbers b0 + 16 j + 4 g .. of a wave's rows to a result; OUT: its dtype where the kernel knows it (-1: it does not).
template <int TB, bool FULL, int OUT> struct RowStore {
  int row, b, wb, size;
  __device__ __forceinline__ RowStore(const Head& h, int dtype, int b0, int width, int back) : wb(width), size((OUT < 0 ? dtype : OUT) == 0 ? 4 : 2) {
    const int i = 16 * wave_id() + (threadIdx.x & 15);
    b = b0 + 4 * ((threadIdx.x & 63) >> 4);
    row = (back ? kChunk - 1 - i : i) * h.pitch;
  }
  __device__ __forceinline__ void put(const Chunk& k, const f32x4 (&acc)[TB]) const {
    const int first = row - k.shift();
    if constexpr (FULL) {
      const __amdgpu_buffer_rsrc_t r = k.buffer();
      const int at = first + b * size;
#pragma unroll
      for (int j = 0; j < TB; ++j) {
        const int o = b + 16 * j < wb ? at : kNowhere;
        if (OUT == 0 || (OUT < 0 && size == 4)) __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, acc[j]), r, o + 64 * j, 0, 0);
        else __builtin_amdgcn_raw_buffer_store_b64(__builtin_bit_cast(u32x2, __builtin_convertvector(acc[j], bf16x4)), r, o + 32 * j, 0, 0);
      }
    } else if ((unsigned)first < (unsigned)(k.n * k.pitch)) {
      const TensorDev t{k.at + first, size == 4 ? 0 : 1, 0, 0, 0};
#pragma unroll
      for (int j = 0; j < TB; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (b + 16 * j + i < wb) store_elem(t, b + 16 * j + i, acc[j][i]);
    }
  }
};

// Zeros for the rows of a segment that lie behind the sequence.
__device__ __forceinline__ void zero_rows(const TensorDev& Y, int b, int h, int heads, int from, int to, int b0, int cols) {
  if (from >= to) return;
  const int per = (to - from) * cols;
  for (int i = 0; i < heads; ++i)
    for (int id = threadIdx.x; id < per; id += 256) {
      const int row = id / cols;
      store_elem(Y, st::row_base(Y, b, h * heads + i, from + row) + b0 + id - row * cols, 0.f);
    }
}

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

// Weights of a chunk's n rows in the sums of a state, lambda^(n - j - first) scale for row j, in LDS from the powers there.
__device__ __forceinline__ void put_weights(float* uw, const float* pw, int n, int first, float scale) {
  if (threadIdx.x < kChunk) uw[threadIdx.x] = scale * pw[max(0, n - first - (int)threadIdx.x)];
}
// S += sum over the chunk's rows of w a b', w a as PU pieces
template <int P, int PU, int W, int TB>
__device__ __forceinline__ void add_chunk(StateTiles<W, TB>& S, const Tiles<W, TB>& t, const uint16_t* sa, const uint16_t* sb, const float* uw) {
  constexpr int LDA = W + 8, LDB = 16 * TB + 8, PA = kChunk * LDA, PB = kChunk * LDB, AT = Tiles<W, TB>::AT, BT = Tiles<W, TB>::BT;
  const int lane = threadIdx.x & 63;
  const uint16_t *la = sa + st::lane_tr(lane, LDA), *lb = sb + st::lane_tr(lane, LDB);
  const float* u = uw + 4 * (lane >> 4);
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    phase();
    const f32x4 w0 = *(const f32x4*)(u + 32 * q), w1 = *(const f32x4*)(u + 32 * q + 16);
    const f32x8 w = {w0[0], w0[1], w0[2], w0[3], w1[0], w1[1], w1[2], w1[3]};
    Op<PU> a[AT];
#pragma unroll
    for (int i = 0; i < AT; ++i) {
      const uint16_t* p = la + 32 * q * LDA + 16 * (t.at + i);
      a[i] = pieces<PU>(number<P>(columns<P>(p, p + 16 * LDA, PA)) * w);
    }
    Op<P> b[BT];
#pragma unroll
    for (int j = 0; j < BT; ++j) {
      const uint16_t* p = lb + 32 * q * LDB + 16 * (t.bt + j);
      b[j] = columns<P>(p, p + 16 * LDB, PB);
    }
    each_product<PU, P>([&](int x, int y) {
#pragma unroll
      for (int j = 0; j < BT; ++j)
#pragma unroll
        for (int i = 0; i < AT; ++i) S[i][j] = st::mfma(a[i].p[x], b[j].p[y], S[i][j]);
    });
  }
}

constexpr size_t kTables = (kChunk + 68) * 4;             // bytes of the weights and the powers
template <int W, int TB> __device__ __forceinline__ void decay_state(StateTiles<W, TB>& S, Keep k) {
#pragma unroll
  for (int i = 0; i < Tiles<W, TB>::AT; ++i)
#pragma unroll
    for (int j = 0; j < Tiles<W, TB>::BT; ++j) {
      if (k.near) {
#pragma unroll
        for (int r = 0; r < 4; ++r) S[i][j][r] = fmaf(S[i][j][r], k.part, S[i][j][r]);
      } else {
        scale_by(S[i][j], k.part);
      }
    }
}
// Weights s lambda^(16 q + col - 4 g - r) of the scores of rows 4 g + r with the row col, q tiles of sixteen apart.
__device__ __forceinline__ void score_weights(f32x4 (&near)[4], const float* pw, float s) {
  const int g = (threadIdx.x & 63) >> 4, col = threadIdx.x & 15;
#pragma unroll
  for (int q = 0; q < 4; ++q)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int n = 16 * q + col - 4 * g - r;
      near[q][r] = n >= 0 ? s * pw[max(n, 0)] : 0.f;
    }
}
// acc[j] += B' (weighed scores of the rows x with the rows A), both of a chunk of n rows in LDS; PERM: the order of x's numbers (RowOps).
template <int P, int PM, int STEPS, int TB, bool PERM>
__device__ __forceinline__ void add_scores(f32x4 (&acc)[TB], const Op<P> (&x)[STEPS], const uint16_t* sa, int LDA, const uint16_t* sb, int LDB,
                                           const f32x4 (&near)[4]) {
  const int wave = wave_id(), lane = threadIdx.x & 63, g = lane >> 4, col = lane & 15, PA = kChunk * LDA, PB = kChunk * LDB;
  // tiles of rows wave, wave - 1, ... two at a time
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    const int j0 = wave - 2 * q, j1 = max(j0 - 1, 0);
    phase();
    if (j0 < 0) continue;
    f32x4 sc[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
    for (int k = 0; k < STEPS; ++k) {
      auto row = [&](int j) {
        if constexpr (!PERM) {
          return st::row_op<P>(sa + (16 * j + col) * LDA + 32 * k + 8 * g, PA);
        } else {
          Op<P> o;
          const uint16_t* p = sa + (16 * j + col) * LDA + 32 * k + 4 * g;
#pragma unroll
          for (int i = 0; i < P; ++i) {
            const u32x2 a = *(const u32x2*)(p + i * PA), b = *(const u32x2*)(p + i * PA + 16);
            o.p[i] = __builtin_bit_cast(bf16x8, u32x4{a[0], a[1], b[0], b[1]});
          }
          return o;
        }
      };
      const Op<P> o0 = row(j0), o1 = row(j1);
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
    const uint16_t* lb = sb + st::lane_tr(lane, LDB);
    Op<P> bt[TB];
#pragma unroll
    for (int j = 0; j < TB; ++j) bt[j] = columns<P>(lb + 16 * j0 * LDB + 16 * j, lb + 16 * j1 * LDB + 16 * j, PB);
    const Op<PM> o = pieces<PM>(v);
    each_product<P, PM>([&](int m, int y) {
#pragma unroll
      for (int j = 0; j < TB; ++j) acc[j] = st::mfma(bt[j].p[m], o.p[y], acc[j]);
    });
  }
}

// ------------------------------------------------------------------------------------------------ rows
// Waves to a SIMD: what LDS allows, or registers without spills.
constexpr int walk_waves(int P, int W) { return P == 1 ? (W <= 64 ? 3 : 2) : (W <= 64 ? 2 : 1); }
template <int P, int PM, int PU, int W, int TB, bool FULL, int DT>
__global__ void __launch_bounds__(256, walk_waves(P, W)) k_decay_walk(WalkSet set, int ncb) {
  constexpr int NB = 16 * TB, STEPS = W / 32, LDA = W + 8, LDB = NB + 8, PA = kChunk * LDA, PB = kChunk * LDB;
  constexpr int OUT = P == 1 && PM == 2 ? 1 : -1;             // (two pieces are for results in bf16)
  constexpr int IMG = STEPS * PM * 512;                       // numbers of one column tile of the state's image
  extern __shared__ char lds[];
  uint16_t *sa = (uint16_t*)lds, *sb = sa + P * PA, *img = sb + P * PB;
  float *uw = (float*)(img + TB * IMG), *pw = uw + kChunk;    // weights of the chunk's rows; lambda^0 .. lambda^64
  const Call& c = set.c;
  const Walk& w = set.w[blockIdx.y];
  Place p;
  if (!place(c, c.nseg, ncb, &p)) return;
  const int tid = threadIdx.x, wave = wave_id(), lane = tid & 63, g = lane >> 4, col = lane & 15, b0 = 64 * p.cb;
  if (b0 >= w.wb) return;
  if (c.left_out && p.slot == -2 && p.h == 0 && p.cb == 0 && p.seg == 0 && tid == 0 && blockIdx.y == 0) atomicAdd(c.left_out, 1);
  const int lo = p.seg * c.seg_rows, hi = min(p.len, lo + c.seg_rows);
  zero_rows(w.Y, p.b, p.h, w.GX, max(lo, p.len), p.seg == c.nseg - 1 ? c.L : min(c.L, lo + c.seg_rows), b0, min(64, w.wb - b0));
  const int s = p.b * c.Hk + p.h;
  const bool ends = w.end != nullptr && c.nseg == 1 && (p.slot >= 0 || !w.end_pool);
  if (hi <= lo && !ends) return;
  const float ld = c.log_decay[p.h];
  for (int i = tid; i <= kChunk; i += 256) pw[i] = power(ld, i);
  Keep keep = scalar(keep_of(ld, kChunk));
  const Tiles<W, TB> t(wave);
  StateTiles<W, TB> S;
  // (with segments the pool may hold the states after the call already)
  const float* from = w.init == nullptr && p.seg == 0 ? nullptr
                      : c.nseg > 1                    ? set.prefix[blockIdx.y] + ((size_t)s * c.nseg + p.seg) * c.state
                                                      : (p.slot >= 0 ? w.init + ((size_t)p.slot * c.Hk + p.h) * c.state : nullptr);
  load_state<W, TB>(S, t, from, w.sa, w.sb, w.wa, w.wb, b0);
  const int back = w.back, GX = w.GX, GA = w.GA, first = w.first;
  const float s_update = w.s_update;
  const Head hx(w.X, p.b, p.h * GX), ha(w.A, p.b, p.h * GA), hb(w.B, p.b, p.h * GA), hy(w.Y, p.b, p.h * GX);
  Stage<P, W, FULL, DT> ra(ha, 0, w.wa, back);
  Stage<P, NB, FULL, DT> rb(hb, b0, w.wb, back);
  RowOps<P, STEPS, FULL, DT> rx(hx, w.wa, back);
  const RowStore<TB, FULL, OUT> ry(hy, w.Y.dtype, b0, w.wb, back);
  auto fetch_x = [&](int r0, int gx) { rx.fetch(hx.chunk(gx, r0, min(kChunk, hi - r0), p.len, back)); };
  auto fetch_rows = [&](int r0, int ga) {
    const int n = min(kChunk, hi - r0);
    ra.fetch(ha.chunk(ga, r0, n, p.len, back));
    rb.fetch(hb.chunk(ga, r0, n, p.len, back));
  };
  if (lo < hi) { fetch_rows(lo, 0); fetch_x(lo, 0); }
  __syncthreads();
  f32x4 near[4];
  score_weights(near, pw, w.s_score);
  const float inter = w.s_inter * pw[16 * wave + col + first];
  put_weights(uw, pw, kChunk, first, s_update);

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
          const bf16x4 h = __builtin_convertvector(x, bf16x4);
          *(bf16x4*)(to + k * 512) = h;
          x -= __builtin_convertvector(h, f32x4);
        }
      }
  };
  put_image();
  Op<P> x[STEPS];
  f32x4 acc[TB];
  for (int r0 = lo; r0 < hi; r0 += kChunk) {
    int n = min(kChunk, hi - r0);
    const bool more = r0 + kChunk < hi;
    if (n < kChunk && ends) {
      asm("" : "+s"(n));                                      // (or powers for it would be found for every chunk)
      put_weights(uw, pw, n, first, s_update);
      keep = scalar(keep_of(ld, n));
    }
    for (int ga = 0; ga < GA; ++ga) {
      ra.store(sa, 0);
      rb.store(sb, b0);
      __syncthreads();
      if (ga + 1 < GA) fetch_rows(r0, ga + 1);
      else if (more) fetch_rows(r0 + kChunk, 0);
      for (int gx = 0; gx < GX; ++gx) {
        if (ga == 0) {
          rx.ops(x);
          if (gx + 1 < GX) fetch_x(r0, gx + 1);
          else if (more) fetch_x(r0 + kChunk, 0);
#pragma unroll
          for (int j = 0; j < TB; ++j) acc[j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int k = 0; k < STEPS; ++k) {
            Op<PM> o[TB];
#pragma unroll
            for (int j = 0; j < TB; ++j) o[j] = st::image_op<PM>(img + j * IMG + k * PM * 512, lane);
            each_product<PM, P>([&](int m, int y) {
#pragma unroll
              for (int j = 0; j < TB; ++j) acc[j] = st::mfma(o[j].p[m], x[k].p[y], acc[j]);
            });
          }
#pragma unroll
          for (int j = 0; j < TB; ++j) scale_by(acc[j], inter);
        }
        add_scores<P, PM, STEPS, TB, false>(acc, x, sa, LDA, sb, LDB, near);
        if (ga == GA - 1) ry.put(hy.chunk(gx, r0, n, p.len, back), acc);
      }
      if (more || ends) {
        if (ga == 0) decay_state<W, TB>(S, keep);
        add_chunk<P, PU, W, TB>(S, t, sa, sb, uw);
      }
      __syncthreads();
    }
    if (more) put_image();
  }
  if (ends)
    store_state<W, TB>(S, t, w.end + (w.end_pool ? (size_t)p.slot * c.Hk + p.h : (size_t)s) * c.state, w.sa, w.sb, w.wa, w.wb, b0);
}

// Gradients of keys and values in one walk from the last row to the first: dk_j = D_j v_j, dv_j = D_j' k_j with the state D of the rows q and
// dy behind, in LDS as rows of D', of which the one takes columns and the other rows.  set.w[0]: the values (X = V, A = dY, B = Q, Y = dK),
// set.w[1]: the keys (X = K, A = Q, B = dY, Y = dV).
template <int P, int PM, int PU, int W, bool FULL, int DT>
__global__ void __launch_bounds__(256, P == 1 ? 3 : 1) k_decay_back(WalkSet set) {
  constexpr int TB = W / 16, STEPS = W / 32, LD = W + 8, PL = kChunk * LD, PI = W * LD, OUT = P == 1 && PM == 2 ? 1 : -1;
  extern __shared__ char lds[];
  uint16_t *sq = (uint16_t*)lds, *sd = sq + P * PL, *img = sd + P * PL;
  float *uw = (float*)(img + PM * PI), *pw = uw + kChunk;
  const Call& c = set.c;
  const Walk &wk = set.w[0], &wv = set.w[1];
  Place p;
  if (!place(c, c.nseg, 1, &p)) return;
  const int tid = threadIdx.x, wave = wave_id(), lane = tid & 63, g = lane >> 4, col = lane & 15;
  const int lo = p.seg * c.seg_rows, hi = min(p.len, lo + c.seg_rows), pad = p.seg == c.nseg - 1 ? c.L : min(c.L, lo + c.seg_rows);
  zero_rows(wk.Y, p.b, p.h, 1, max(lo, p.len), pad, 0, wk.wb);
  zero_rows(wv.Y, p.b, p.h, 1, max(lo, p.len), pad, 0, wv.wb);
  const int s = p.b * c.Hk + p.h, G = wv.GA;
  const bool ends = wv.end != nullptr && c.nseg == 1 && (p.slot >= 0 || !wv.end_pool);
  if (hi <= lo && !ends) return;
  const float ld = c.log_decay[p.h];
  for (int i = tid; i <= kChunk; i += 256) pw[i] = power(ld, i);
  Keep keep = scalar(keep_of(ld, kChunk));
  const Tiles<W, TB> t(wave);
  StateTiles<W, TB> S;
  const float* from = wv.init == nullptr && p.seg == 0 ? nullptr
                      : c.nseg > 1                     ? set.prefix[1] + ((size_t)s * c.nseg + p.seg) * c.state
                                                       : (p.slot >= 0 ? wv.init + ((size_t)p.slot * c.Hk + p.h) * c.state : nullptr);
  load_state<W, TB>(S, t, from, wv.sa, wv.sb, wv.wa, wv.wb, 0);
  const Head hq(wv.A, p.b, p.h * G), hd(wv.B, p.b, p.h * G), hk(wv.X, p.b, p.h), hv(wk.X, p.b, p.h), hdk(wk.Y, p.b, p.h), hdv(wv.Y, p.b, p.h);
  Stage<P, W, FULL, DT> rq(hq, 0, wv.wa, 1), rd(hd, 0, wv.wb, 1);
  RowOps<P, STEPS, FULL, DT> rk(hk, wv.wa, 1);
  RowOps<P, STEPS, FULL, DT, true> rv(hv, wk.wa, 1);
  const RowStore<TB, FULL, OUT> to_k(hdk, wk.Y.dtype, 0, wk.wb, 1), to_v(hdv, wv.Y.dtype, 0, wv.wb, 1);
  const float s_update = wv.s_update;
  auto fetch_x = [&](int r0) {
    const int n = min(kChunk, hi - r0);
    rk.fetch(hk.chunk(0, r0, n, p.len, 1));
    rv.fetch(hv.chunk(0, r0, n, p.len, 1));
  };
  auto fetch_rows = [&](int r0, int ga) {
    const int n = min(kChunk, hi - r0);
    rq.fetch(hq.chunk(ga, r0, n, p.len, 1));
    rd.fetch(hd.chunk(ga, r0, n, p.len, 1));
  };
  if (lo < hi) { fetch_rows(lo, 0); fetch_x(lo); }
  __syncthreads();
  f32x4 near[4];
  score_weights(near, pw, wv.s_score);
  const float inter = pw[16 * wave + col];
  put_weights(uw, pw, kChunk, 0, s_update);
  auto put_image = [&]() {
#pragma unroll
    for (int i = 0; i < Tiles<W, TB>::AT; ++i)
#pragma unroll
      for (int j = 0; j < Tiles<W, TB>::BT; ++j) {
        uint16_t* to = img + (16 * (t.bt + j) + col) * LD + 16 * (t.at + i) + 4 * g;
        f32x4 x = S[i][j];
#pragma unroll
        for (int k = 0; k < PM; ++k) {
          const bf16x4 h = __builtin_convertvector(x, bf16x4);
          *(bf16x4*)(to + k * PI) = h;
          x -= __builtin_convertvector(h, f32x4);
        }
      }
  };
  put_image();
  Op<P> xk[STEPS], xv[STEPS];
  f32x4 dk[TB], dv[TB];
  const uint16_t *rows = img + col * LD + 8 * g, *cols = img + st::lane_tr(lane, LD);
  for (int r0 = lo; r0 < hi; r0 += kChunk) {
    int n = min(kChunk, hi - r0);
    const bool more = r0 + kChunk < hi;
    if (n < kChunk && ends) {
      asm("" : "+s"(n));
      put_weights(uw, pw, n, 0, s_update);
      keep = scalar(keep_of(ld, n));
    }
    for (int ga = 0; ga < G; ++ga) {
      rq.store(sq, 0);
      rd.store(sd, 0);
      __syncthreads();
      if (ga + 1 < G) fetch_rows(r0, ga + 1);
      else if (more) fetch_rows(r0 + kChunk, 0);
      if (ga == 0) {
        rk.ops(xk);
        rv.ops(xv);
        if (more) fetch_x(r0 + kChunk);
#pragma unroll
        for (int j = 0; j < TB; ++j) dk[j] = dv[j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < STEPS; ++k) {
          phase();
          Op<PM> o[TB];
#pragma unroll
          for (int j = 0; j < TB; ++j) o[j] = st::row_op<PM>(rows + 16 * j * LD + 32 * k, PI);
          each_product<PM, P>([&](int m, int y) {
#pragma unroll
            for (int j = 0; j < TB; ++j) dv[j] = st::mfma(o[j].p[m], xk[k].p[y], dv[j]);
          });
          phase();
#pragma unroll
          for (int j = 0; j < TB; ++j) o[j] = columns<PM>(cols + 32 * k * LD + 16 * j, cols + (32 * k + 16) * LD + 16 * j, PI);
          each_product<PM, P>([&](int m, int y) {
#pragma unroll
            for (int j = 0; j < TB; ++j) dk[j] = st::mfma(o[j].p[m], xv[k].p[y], dk[j]);
          });
        }
#pragma unroll
        for (int j = 0; j < TB; ++j) {
          scale_by(dk[j], inter);
          scale_by(dv[j], inter);
        }
      }
      add_scores<P, PM, STEPS, TB, true>(dk, xv, sd, LD, sq, LD, near);
      add_scores<P, PM, STEPS, TB, false>(dv, xk, sq, LD, sd, LD, near);
      if (ga == G - 1) {
        to_k.put(hdk.chunk(0, r0, n, p.len, 1), dk);
        to_v.put(hdv.chunk(0, r0, n, p.len, 1), dv);
      }
      if (more || ends) {
        if (ga == 0) decay_state<W, TB>(S, keep);
        add_chunk<P, PU, W, TB>(S, t, sq, sd, uw);
      }
      __syncthreads();
    }
    if (more) put_image();
  }
  if (ends)
    store_state<W, TB>(S, t, wv.end + (wv.end_pool ? (size_t)p.slot * c.Hk + p.h : (size_t)s) * c.state, wv.sa, wv.sb, wv.wa, wv.wb, 0);
}

// ------------------------------------------------------------------------------------------------ sums of segments
template <int P, int W, int TB, bool FULL, int DT>
__global__ void __launch_bounds__(256) k_decay_sum(SumSet set, int ncb) {
  constexpr int NB = 16 * TB, PA = kChunk * (W + 8), PB = kChunk * (NB + 8);
  extern __shared__ char lds[];
  uint16_t *sa = (uint16_t*)lds, *sb = sa + P * PA;
  float *uw = (float*)(sb + P * PB), *pw = uw + kChunk;
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
  Keep keep = scalar(keep_of(ld, kChunk));
  const Tiles<W, TB> t(wave_id());
  StateTiles<W, TB> S;
  load_state<W, TB>(S, t, nullptr, 0, 0, 0, 0, 0);
  const Head ha(w.A, p.b, p.h * w.GA), hb(w.B, p.b, p.h * w.GA);
  Stage<P, W, FULL, DT> ra(ha, 0, w.wa, w.back);
  Stage<P, NB, FULL, DT> rb(hb, b0, w.wb, w.back);
  auto fetch_rows = [&](int r0, int ga) {
    const int n = min(kChunk, hi - r0);
    ra.fetch(ha.chunk(ga, r0, n, p.len, w.back));
    rb.fetch(hb.chunk(ga, r0, n, p.len, w.back));
  };
  fetch_rows(lo, 0);
  __syncthreads();
  put_weights(uw, pw, kChunk, w.first, w.s_update);
  for (int r0 = lo; r0 < hi; r0 += kChunk) {
    int n = min(kChunk, hi - r0);
    if (n < kChunk) {
      asm("" : "+s"(n));
      put_weights(uw, pw, n, w.first, w.s_update);
      keep = scalar(keep_of(ld, n));
    }
    for (int ga = 0; ga < w.GA; ++ga) {
      ra.store(sa, 0);
      rb.store(sb, b0);
      __syncthreads();
      if (ga + 1 < w.GA) fetch_rows(r0, ga + 1);
      else if (r0 + kChunk < hi) fetch_rows(r0 + kChunk, 0);
      if (ga == 0 && r0 > lo) decay_state<W, TB>(S, keep);
      add_chunk<P, 3, W, TB>(S, t, sa, sb, uw);
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

// Sums of the readers of a slot, for 64 numbers of its states a workgroup: its sixteen groups of sixteen lanes take every sixteenth
// reader each, in their order, and are then added in theirs.
__global__ void __launch_bounds__(256) k_decay_slot_sums(Call c, const float* each, float* pool) {
  __shared__ int list[256], count[4];
  __shared__ float part[16][64];
  const int slot = blockIdx.y / c.Hk, h = blockIdx.y - slot * c.Hk, tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, group = tid >> 4;
  float sum[4] = {0.f, 0.f, 0.f, 0.f};
  const int id = blockIdx.x * 64 + 4 * (tid & 15);
  bool found = false;
  int before_all = 0;
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
    for (int i = (group - before_all) & 15; i < total; i += 16) {
      const float* from = each + ((size_t)list[i] * c.Hk + h) * c.state + id;
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (id + k < c.state) sum[k] += from[k];
    }
    before_all += total;
    found = found || total > 0;
    __syncthreads();
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) part[group][4 * (tid & 15) + k] = sum[k];
  __syncthreads();
  if (tid < 64 && blockIdx.x * 64 + tid < c.state) {
    float t = 0.f;
    for (int i = 0; i < 16; ++i) t += part[i][tid];
    pool[((size_t)slot * c.Hk + h) * c.state + blockIdx.x * 64 + tid] = t;
  }
}

int status() { return hipGetLastError() == hipSuccess ? 0 : 5; }

// More LDS than a launch has by itself is asked for once for a kernel and device.
template <class K> int room(K kernel, size_t bytes) {
  if (bytes <= 65536) return 0;
  return hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes) == hipSuccess ? 0 : 5;
}

template <int P, int PM, int PU, int W, int TB, bool FULL, int DT>
int walk_launch(const WalkSet& a, int count, hipStream_t st) {
  int ncb = 1;
  for (int i = 0; i < count; ++i) ncb = max(ncb, (a.w[i].wb + 16 * TB - 1) / (16 * TB));
  const size_t lds = (size_t)P * kChunk * (W + 8 + 16 * TB + 8) * 2 + (size_t)TB * (W / 32) * PM * 1024 + kTables;
  if (int rc = room(k_decay_walk<P, PM, PU, W, TB, FULL, DT>, lds)) return rc;
  const long long units = ((long long)a.c.B * a.c.Hk * a.c.nseg + 7) / 8 * 8;
  if (units * ncb > 0x7fffffffLL) return 2;
  hipLaunchKernelGGL((k_decay_walk<P, PM, PU, W, TB, FULL, DT>), dim3((unsigned)(units * ncb), count), dim3(256), lds, st, a, ncb);
  return status();
}
template <int P, int PM, int PU, int W, bool FULL, int DT>
int back_launch(const WalkSet& a, hipStream_t st) {
  const size_t lds = (size_t)P * kChunk * (W + 8) * 4 + (size_t)PM * W * (W + 8) * 2 + kTables;
  if (int rc = room(k_decay_back<P, PM, PU, W, FULL, DT>, lds)) return rc;
  const long long units = ((long long)a.c.B * a.c.Hk * a.c.nseg + 7) / 8 * 8;
  if (units > 0x7fffffffLL) return 2;
  hipLaunchKernelGGL((k_decay_back<P, PM, PU, W, FULL, DT>), dim3((unsigned)units), dim3(256), lds, st, a);
  return status();
}
template <int P, int W, int TB, bool FULL, int DT>
int sum_launch(const SumSet& a, int count, hipStream_t st) {
  int ncb = 1;
  for (int i = 0; i < count; ++i) ncb = max(ncb, (a.w[i].wb + 16 * TB - 1) / (16 * TB));
  const size_t lds = (size_t)P * kChunk * (W + 8 + 16 * TB + 8) * 2 + kTables;
  if (int rc = room(k_decay_sum<P, W, TB, FULL, DT>, lds)) return rc;
  const long long units = ((long long)a.c.B * a.c.Hk * (a.last ? a.c.nseg : a.c.nseg - 1) + 7) / 8 * 8;
  if (units == 0) return 0;
  if (units * ncb > 0x7fffffffLL) return 2;
  hipLaunchKernelGGL((k_decay_sum<P, W, TB, FULL, DT>), dim3((unsigned)(units * ncb), count), dim3(256), lds, st, a, ncb);
  return status();
}

int class_of(int n) { return n <= 32 ? 32 : (n <= 64 ? 64 : 128); }

template <int P, int PM, int PU, bool FULL, int DT> int walk_width(const WalkSet& a, int count, int wa, int wb, hipStream_t st) {
  if (class_of(wa) == 128) return walk_launch<P, PM, PU, 128, 4, FULL, DT>(a, count, st);
  if (class_of(wa) == 64) return walk_launch<P, PM, PU, 64, 4, FULL, DT>(a, count, st);
  return wb <= 32 ? walk_launch<P, PM, PU, 32, 2, FULL, DT>(a, count, st) : walk_launch<P, PM, PU, 32, 4, FULL, DT>(a, count, st);
}
template <int P, int PM, int PU, bool FULL, int DT> int back_width(const WalkSet& a, int w, hipStream_t st) {
  return w <= 32 ? back_launch<P, PM, PU, 32, FULL, DT>(a, st) : back_launch<P, PM, PU, 64, FULL, DT>(a, st);
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
  bool full = true, ends = false;
  for (int i = 0; i < count; ++i) {
    a.w[i] = all.w[from + i];
    ends = ends || (a.w[i].end != nullptr && a.c.nseg == 1);
    a.prefix[i] = all.prefix[from + i];
    wa = max(wa, a.w[i].wa);
    wb = max(wb, a.w[i].wb);
    full = full && a.w[i].wa % 8 == 0 && a.w[i].wb % 8 == 0;
  }
  auto go = [&](auto full_rows) {
    constexpr bool F = decltype(full_rows)::value;
    if (dtype == 0) return walk_width<3, 3, 3, F, 0>(a, count, wa, wb, st);
    if (fine) return walk_width<1, 3, 3, F, 1>(a, count, wa, wb, st);
    return ends ? walk_width<1, 2, 3, F, 1>(a, count, wa, wb, st) : walk_width<1, 2, 2, F, 1>(a, count, wa, wb, st);
  };
  return full ? go(std::true_type{}) : go(std::false_type{});
}

// The walks of dK and dV (from, from + 1) as one.
int launch_back(const WalkSet& all, int from, int dtype, bool fine, hipStream_t st) {
  WalkSet a = all;
  for (int i = 0; i < 2; ++i) {
    a.w[i] = all.w[from + i];
    a.prefix[i] = all.prefix[from + i];
  }
  const Walk& w = a.w[1];
  const int n = max(w.wa, w.wb);
  const bool ends = w.end != nullptr && a.c.nseg == 1;
  auto go = [&](auto full_rows) {
    constexpr bool F = decltype(full_rows)::value;
    if (dtype == 0) return back_width<3, 3, 3, F, 0>(a, n, st);
    if (fine) return back_width<1, 3, 3, F, 1>(a, n, st);
    return ends ? back_width<1, 2, 3, F, 1>(a, n, st) : back_width<1, 2, 2, F, 1>(a, n, st);
  };
  return w.wa % 8 == 0 && w.wb % 8 == 0 ? go(std::true_type{}) : go(std::false_type{});
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
  hipLaunchKernelGGL(k_decay_slot_sums, dim3((c.state + 63) / 64, c.nslots * c.Hk), dim3(256), 0, st, c, each, pool);
  return status();
}

}  // namespace dec
}  // namespace fs
