// Linear attention with a decay for each head, rows of prompts and of training: chunks of 64 rows (32 in the walk by columns and in the sums of fp32
// rows), within a chunk by the scores of its rows, between chunks by the state.  See decay_common.h for the formulas.
//
// Segments of a sequence are walked side by side: sums of the segments (k_decay_sum), states before them (k_decay_join), then the walks.
//   k_decay_walk  rows x and a of bf16 up to 64 numbers, rows b in blocks of 64.  A wave has sixteen rows of x as operands, read once from memory,
//                 and results in whole rows; the state's numbers are shared out to the waves' accumulators and reach the others as an image in LDS.
//   k_decay_cols  wider rows x and a, and all of fp32.  A wave has sixteen columns of the state and of the results, the rows x go through LDS:
//                 the state never does (an image of 128 x 128 in three pieces would take 96 KB).
//   k_decay_back  dK and dV of rows up to 64 in one walk: q, dy and the state are read once for both.
// Scores, states and the weighed rows in the sums of a state are fp32 and go into the next product as three bf16 pieces (24 bits), for results of
// either dtype: what a query reads of a state can be far smaller than the state (rows with a mean), and two pieces, 16 bits, would keep too
// little of it (states of mean 22962: 0.0056 - 0.0073 off instead of the rounding to bf16, 0.0017; a tenth to a fifth faster).
//
// What bounds them, rows of 64 in bf16 (4 x 8 states, 16384 rows: sums 30 us, 134 MB, a walk 68, 268 MB, dK and dV 108, 403 MB: 3.7 - 4.5 TB/s,
// where a large copy reaches 5.2): the CU.  Rows that are in the L2 already take nearly as long, 83 instead of 92 us with the sums.  Of the
// cycles of a SIMD 35 % issue vector and 29 % run matrix instructions (dK and dV 33 and 32).  Rows of 128 in bf16 (16 states, 65536 rows: sums 130 us,
// the walk 344, 3.1 TB/s) the CU, too: rows in the L2 take 397 of 460 us; vector instructions 33 %, matrix 40 %, three barriers a chunk between them.
// Rows of fp32 six matrix products for one (three pieces of each side).
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
typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4;

__device__ __forceinline__ int wave_id() { return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); }      // (a scalar: branches on it, too)
__device__ __forceinline__ float scalar(float x) { return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(x))); }
__device__ __forceinline__ Keep scalar(Keep k) { return {scalar(k.part), __builtin_amdgcn_readfirstlane((int)k.near) != 0}; }

__device__ __forceinline__ void scale_by(f32x4& v, float f) {       // (one register for the factor, where v *= f takes four)
#pragma unroll
  for (int r = 0; r < 4; ++r) v[r] *= f;
}

// A value that the compiler has to take as it finds it in every turn: what follows from it is worked out there and not kept in registers, or
// in memory, for all turns.
__device__ __forceinline__ int afresh(int x) {
  asm volatile("" : "+s"(x));
  return x;
}
__device__ __forceinline__ int afresh_lane(int x) {
  asm volatile("" : "+v"(x));
  return x;
}

// Operands of a part of a chunk are not fetched before the part: that would take registers that hold more waves otherwise.
__device__ __forceinline__ void phase() { __builtin_amdgcn_sched_barrier(0); }

// What a piece leaves of four numbers that are summed, exact.
__device__ __forceinline__ f32x4 rest_of(f32x4 x, bf16x4 h) {
  const f32x2_t a = less_piece(f32x2_t{x[0], x[1]}, bf16x2_t{h[0], h[1]}), b = less_piece(f32x2_t{x[2], x[3]}, bf16x2_t{h[2], h[3]});
  return f32x4{a[0], a[1], b[0], b[1]};
}
constexpr int kPieces = 3;                                  // of a number of 32 bits
__device__ __forceinline__ Op<kPieces> pieces(f32x8 x) { return st::as_op<kPieces>(x); }
template <int P> __device__ __forceinline__ f32x8 number(const Op<P>& o) {
  f32x8 x = __builtin_convertvector(o.p[P - 1], f32x8);
#pragma unroll
  for (int i = P - 2; i >= 0; --i) x += __builtin_convertvector(o.p[i], f32x8);
  return x;
}

struct Place { int b, h, seg, cb, part, slot, len; };
// Units of a grid: (sequence, key head, segment), their column blocks and parts of the heads eight workgroups apart, on one XCD.  slot -2:
// left out.
__device__ __forceinline__ bool place(const Call& c, int nseg, int ncb, int parts, Place* p) {
  // (quotients come from vector instructions: in scalars again, so that addresses are)
  auto uniform = [](int x) { return __builtin_amdgcn_readfirstlane(x); };
  const int x = blockIdx.x, each = 8 * ncb * parts, q = uniform(x / each), rest = x - q * each;
  p->part = uniform((rest >> 3) / ncb);
  p->cb = (rest >> 3) - p->part * ncb;
  const long long u = (long long)q * 8 + (rest & 7);
  if (u >= (long long)c.B * c.Hk * nseg) return false;
  const int s = uniform((int)u / nseg);                       // (the grid has fewer than 2^31 workgroups)
  p->seg = (int)u - s * nseg;
  p->b = uniform(s / c.Hk);
  p->h = s - p->b * c.Hk;
  int len = c.lengths ? max(0, min(c.lengths[p->b], c.L)) : c.L, slot;
  if (c.unique) {
    slot = st::unique_slot_of(c.slots, c.nslots, p->b);
    if (slot < 0) { slot = -2; len = 0; }
  } else {
    slot = st::slot_of(c.slots, c.nslots, p->b);
  }
  p->len = uniform(len);
  p->slot = uniform(slot);
  return true;
}

// A buffer of `bytes` from p on.  (In scalars whatever way they came: a buffer in vector registers is a loop over the lanes at each load.)
__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer_of(const void* p, int bytes) {
  const uint64_t u = (uint64_t)p;
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)u), hi = __builtin_amdgcn_readfirstlane((uint32_t)(u >> 32));
  return __builtin_amdgcn_make_buffer_rsrc((void*)((uint64_t)hi << 32 | lo), 0, __builtin_amdgcn_readfirstlane(bytes), 0x00027000);
}
// A chunk's n rows of one head: `at` is their lowest in memory, row i at i pitch (back: (n - 1 - i) pitch) bytes.
struct Chunk {
  const char* at;
  int n, pitch, back;
  // offset of row i where there are `rows` of them -> the present one; rows from n on get offsets that are out of the buffer
  __device__ __forceinline__ int shift(int rows = kChunk) const { return back ? (rows - n) * pitch : 0; }
  __device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer() const { return buffer_of(at, n * pitch); }
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

// Numbers from row to row in LDS: neither rows that sixteen lanes read nor columns that they read transposed meet in a bank so (8 more than the
// width: twice the cycles for both).
constexpr int stride(int width) { return width + 16; }
// Columns of two neighbouring tiles of sixteen in pairs: tile 2 k + h, place 4 i + r is column 32 k + 8 i + 4 h + r, so that a lane's fours of
// accumulators of the two follow each other.  tile_pair: the first column of a tile; lane_tr8: lane_tr for them.
__device__ __forceinline__ int tile_pair(int j) { return 32 * (j >> 1) + 4 * (j & 1); }
__device__ __forceinline__ int lane_tr8(int lane, int ld) { return (4 * (lane >> 4) + ((lane & 15) >> 2)) * ld + 8 * (lane & 3); }

// From memory to LDS as P bf16 pieces: T threads, units of eight numbers.  FULL: rows have no ragged end, and units are loads whose
// offsets from the chunk's first row stay; else number by number at the ends.
template <int P, int W, bool FULL, int DT, int ROWS = kChunk, int T = 256> struct Stage {
  static constexpr int UNITS = W / 8, N = (ROWS * UNITS + T - 1) / T, LD = stride(W), PLANE = ROWS * LD, SIZE = DT == 0 ? 4 : 2;
  static constexpr bool EVEN = ROWS * UNITS % T == 0;        // (else the last threads have no unit)
  Raw8 raw[N];
  int cols, pitch, back;
  int c, off;                    // a thread's first unit: its number in the row, its offset from the chunk's first row
  // numbers c0 .. c0 + W - 1 of the rows
  __device__ __forceinline__ Stage(const Head& h, int c0, int ncols, int backwards) : cols(ncols), pitch(h.pitch), back(backwards) {
    const int row = (int)threadIdx.x / UNITS;
    c = c0 + 8 * ((int)threadIdx.x % UNITS);
    off = c < cols && (EVEN || row < ROWS) ? (back ? ROWS - 1 - row : row) * pitch + c * SIZE : kNowhere;
  }
  __device__ __forceinline__ void fetch(const Chunk& k) {
    const int shift = k.shift(ROWS);
    if constexpr (FULL) {
      const __amdgpu_buffer_rsrc_t r = k.buffer();
      const uint32_t first = afresh_lane((int)((uint32_t)off - shift));      // (modulo 2^32, as kNowhere may pass its end)
      const int step = (back ? -T / UNITS : T / UNITS) * pitch;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int o = (int)(first + i * step);
        raw[i].a = __builtin_amdgcn_raw_buffer_load_b128(r, o, 0, 0);
        if constexpr (DT == 0) raw[i].b = __builtin_amdgcn_raw_buffer_load_b128(r, o, 16, 0);
      }
    } else {
      const int step = (back ? -T / UNITS : T / UNITS) * pitch;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int o = (int)((uint32_t)off + (i * step - shift));
        raw[i] = Raw8{{0u, 0u, 0u, 0u}, {0u, 0u, 0u, 0u}};
        if (c < cols && (unsigned)o < (unsigned)(k.n * k.pitch))
          raw[i] = st::fetch8<FULL, DT>(TensorDev{k.at + (o - c * SIZE), DT, 0, 0, 0}, 0, c, cols);
      }
    }
  }
  __device__ __forceinline__ void store(uint16_t* s) const {
    const int tid = threadIdx.x;
    uint16_t* at = s + tid / UNITS * LD + 8 * (tid % UNITS);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if (!EVEN && threadIdx.x + T * i >= ROWS * UNITS) break;
      uint16_t* to = at + T / UNITS * i * LD;
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

// A wave's sixteen rows as operands: a lane has eight numbers 32 k + 8 g .. of row 16 wave + (lane % 16) for each step k.
template <int P, int STEPS, bool FULL, int DT> struct RowOps {
  static constexpr int SIZE = DT == 0 ? 4 : 2;
  Raw8 raw[STEPS];
  int row, cols;
  __device__ __forceinline__ RowOps(const Head& h, int ncols, int back) : cols(ncols) {
    const int i = 16 * wave_id() + (threadIdx.x & 15);
    row = (back ? kChunk - 1 - i : i) * h.pitch;
  }
  __device__ __forceinline__ void fetch(const Chunk& k) {
    const int g = (threadIdx.x & 63) >> 4, shift = k.shift();
    if constexpr (FULL) {
      const __amdgpu_buffer_rsrc_t r = k.buffer();
      const int first = afresh_lane(row - shift + 8 * g * SIZE);
#pragma unroll
      for (int i = 0; i < STEPS; ++i) {
        const int o = 32 * i + 8 * g < cols ? first + 32 * i * SIZE : kNowhere;
        raw[i].a = __builtin_amdgcn_raw_buffer_load_b128(r, o, 0, 0);
        if constexpr (DT == 0) raw[i].b = __builtin_amdgcn_raw_buffer_load_b128(r, o, 16, 0);
      }
    } else {
      const bool there = (unsigned)(row - shift) < (unsigned)(k.n * k.pitch);
      const TensorDev t{k.at + (there ? row - shift : 0), DT, 0, 0, 0};
#pragma unroll
      for (int i = 0; i < STEPS; ++i) {
        raw[i] = Raw8{{0u, 0u, 0u, 0u}, {0u, 0u, 0u, 0u}};
        if (there && 32 * i + 8 * g < cols) raw[i] = st::fetch8<FULL, DT>(t, 0, 32 * i + 8 * g, cols);
      }
    }
  }
  __device__ __forceinline__ void ops(Op<P> (&x)[STEPS]) const {
    const int g = (threadIdx.x & 63) >> 4;
#pragma unroll
    for (int i = 0; i < STEPS; ++i) {
      if constexpr (P == 1 && FULL) x[i].p[0] = __builtin_bit_cast(bf16x8, raw[i].a);
      else x[i] = st::as_op<P>(st::expand8<FULL, DT>(raw[i], DT, 32 * i + 8 * g, cols));
    }
  }
};

// Results are not read again by these calls: they go past the caches, which keep rows for the next launch (64 sequences of 1024 rows of 8
// heads of 64 in bf16, forward and backward: 234 -> 224 us; others within 1 %).  Not those of the walk by columns: pieces of 32 bytes, which the
// caches join (H16 L65536 d128 465 us, past them 553).
constexpr int kStream = 2;
// Numbers b0 + 32 k + 8 g .. of a wave's rows, which two accumulators have, to a result.
template <int TB, bool FULL> struct RowStore {
  int row, b, wb, size;
  __device__ __forceinline__ RowStore(const Head& h, int dtype, int b0, int width, int back) : wb(width), size(dtype == 0 ? 4 : 2) {
    const int i = 16 * wave_id() + (threadIdx.x & 15);
    b = b0 + 8 * ((threadIdx.x & 63) >> 4);
    row = (back ? kChunk - 1 - i : i) * h.pitch;
  }
  __device__ __forceinline__ void put(const Chunk& k, const f32x4 (&acc)[TB]) const {
    const int first = afresh_lane(row - k.shift());
    if constexpr (FULL) {
      const __amdgpu_buffer_rsrc_t r = k.buffer();
      const int at = first + b * size;
#pragma unroll
      for (int j = 0; j < TB; j += 2) {
        const int o = b + 16 * j < wb ? at : kNowhere;
        if (size == 4) {
          __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, acc[j]), r, o + 64 * j, 0, kStream);
          __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, acc[j + 1]), r, o + 64 * j + 16, 0, kStream);
        } else {
          const f32x8 v = {acc[j][0], acc[j][1], acc[j][2], acc[j][3], acc[j + 1][0], acc[j + 1][1], acc[j + 1][2], acc[j + 1][3]};
          __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, __builtin_convertvector(v, bf16x8)), r, o + 32 * j, 0, kStream);
        }
      }
    } else if ((unsigned)first < (unsigned)(k.n * k.pitch)) {
      const TensorDev t{k.at + first, size == 4 ? 0 : 1, 0, 0, 0};
#pragma unroll
      for (int j = 0; j < TB; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int n = b + tile_pair(j) + i;
          if (n < wb) store_elem(t, n, acc[j][i]);
        }
    }
  }
};

// Zeros for the rows of a segment that lie behind the sequence, numbers b0 .. b0 + cols - 1 of each.
__device__ __forceinline__ void zero_rows(const TensorDev& Y, int b, int h, int heads, int from, int to, int b0, int cols) {
  if (from >= to) return;
  const int units = (cols + 7) / 8;
  const long long count = (long long)(to - from) * units;
  for (int i = 0; i < heads; ++i)
    for (long long id = threadIdx.x; id < count; id += blockDim.x) {
      const long long row = id / units;
      const int c = 8 * (int)(id - row * units);
      st::store8(Y, st::row_base(Y, b, h * heads + i, from + (int)row) + b0, c, cols, f32x8{0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f});
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

// Tiles (ti + i, tj + j) of a state in memory, its rows (RP) or columns (CP) in pairs of tiles, columns from b0 on: element (a, b) at a sa + b sb;
// zeros outside it.
template <bool RP, bool CP, int NI, int NJ, class F>
__device__ __forceinline__ void each_number(const float* state, int sa, int sb, int wa, int wb, int ti, int tj, int b0, F f) {
  const int lane = threadIdx.x & 63, g = lane >> 4, c = lane & 15, row = RP ? 8 * g : 4 * g, column = b0 + (CP ? 8 * (c >> 2) + (c & 3) : c);
  const __amdgpu_buffer_rsrc_t m = buffer_of(state, wa * wb * 4);
#pragma unroll
  for (int i = 0; i < NI; ++i)
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      const int a = row + (RP ? tile_pair(ti + i) : 16 * (ti + i)), b = column + (CP ? tile_pair(tj + j) : 16 * (tj + j)), at = (a * sa + b * sb) * 4;
#pragma unroll
      for (int r = 0; r < 4; ++r) f(m, i, j, r, a + r < wa && b < wb ? at + r * sa * 4 : kNowhere);
    }
}
template <bool RP, bool CP, int NI, int NJ>
__device__ __forceinline__ void load_state(f32x4 (&S)[NI][NJ], const float* from, int sa, int sb, int wa, int wb, int ti, int tj, int b0) {
  if (from == nullptr) {
#pragma unroll
    for (int i = 0; i < NI; ++i)
#pragma unroll
      for (int j = 0; j < NJ; ++j) S[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    return;
  }
  each_number<RP, CP, NI, NJ>(from, sa, sb, wa, wb, ti, tj, b0, [&](__amdgpu_buffer_rsrc_t m, int i, int j, int r, int o) {
    S[i][j][r] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(m, o, 0, 0));
  });
}
template <bool RP, bool CP, int NI, int NJ>
__device__ __forceinline__ void store_state(const f32x4 (&S)[NI][NJ], float* to, int sa, int sb, int wa, int wb, int ti, int tj, int b0) {
  each_number<RP, CP, NI, NJ>(to, sa, sb, wa, wb, ti, tj, b0, [&](__amdgpu_buffer_rsrc_t m, int i, int j, int r, int o) {
    __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(S[i][j][r]), m, o, 0, 0);
  });
}
template <int NI, int NJ> __device__ __forceinline__ void decay_state(f32x4 (&S)[NI][NJ], Keep k) {
  const float part = scalar(k.part);
  if (__builtin_amdgcn_readfirstlane((int)k.near)) {
#pragma unroll
    for (int i = 0; i < NI; ++i)
#pragma unroll
      for (int j = 0; j < NJ; ++j)
#pragma unroll
        for (int r = 0; r < 4; ++r) S[i][j][r] = fmaf(S[i][j][r], part, S[i][j][r]);
  } else {
#pragma unroll
    for (int i = 0; i < NI; ++i)
#pragma unroll
      for (int j = 0; j < NJ; ++j) scale_by(S[i][j], part);
  }
}

// Weights of a chunk's n rows in the sums of a state, lambda^(n - j - first) scale for row j, in LDS from the powers there.
__device__ __forceinline__ void put_weights(float* uw, const float* pw, int n, int first, float scale) {
  if (threadIdx.x < kChunk) uw[threadIdx.x] = scale * pw[max(0, n - first - (int)threadIdx.x)];
}
// S += sum over the chunk's rows of w a b'
template <int P, int W, int TB>
__device__ __forceinline__ void add_chunk(StateTiles<W, TB>& S, const Tiles<W, TB>& t, const uint16_t* sa, const uint16_t* sb, const float* uw) {
  constexpr int LDA = stride(W), LDB = stride(16 * TB), PA = kChunk * LDA, PB = kChunk * LDB, AT = Tiles<W, TB>::AT, BT = Tiles<W, TB>::BT;
  const int lane = threadIdx.x & 63;
  const uint16_t *la = sa + st::lane_tr(lane, LDA), *lb = sb + lane_tr8(lane, LDB);
  const float* u = uw + 4 * (lane >> 4);
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    phase();
    const f32x4 w0 = *(const f32x4*)(u + 32 * q), w1 = *(const f32x4*)(u + 32 * q + 16);
    const f32x8 w = {w0[0], w0[1], w0[2], w0[3], w1[0], w1[1], w1[2], w1[3]};
    Op<kPieces> a[AT];
#pragma unroll
    for (int i = 0; i < AT; ++i) {
      const uint16_t* p = la + 32 * q * LDA + 16 * (t.at + i);
      a[i] = pieces(number<P>(columns<P>(p, p + 16 * LDA, PA)) * w);
    }
    Op<P> b[BT];
#pragma unroll
    for (int j = 0; j < BT; ++j) {
      const uint16_t* p = lb + 32 * q * LDB + tile_pair(t.bt + j);
      b[j] = columns<P>(p, p + 16 * LDB, PB);
    }
    each_product<kPieces, P>([&](int x, int y) {
#pragma unroll
      for (int j = 0; j < BT; ++j)
#pragma unroll
        for (int i = 0; i < AT; ++i) S[i][j] = st::mfma(a[i].p[x], b[j].p[y], S[i][j]);
    });
  }
}

constexpr size_t kTables = (kChunk + 80 + 68) * 4;        // bytes of the weights and the powers
// Weights of scores in LDS, s lambda^n at place 63 - n, zeros for n = -1 .. -15: a lane's four rows follow each other.
constexpr int kNear = 80;
__device__ __forceinline__ void put_near(float* near, const float* pw, float s) {
  const int i = (int)threadIdx.x - 128;                        // (the third wave; the first has the other weights)
  if (i >= 0 && i < kNear) near[i] = i < kChunk ? s * pw[kChunk - 1 - i] : 0.f;
}
// acc[j] += B' (weighed scores of the rows x with the rows A), both of a chunk in LDS; columns of B in pairs of
// tiles.
template <int P, int STEPS, int TB>
__device__ __forceinline__ void add_scores(f32x4 (&acc)[TB], const Op<P> (&x)[STEPS], const uint16_t* sa, int LDA, const uint16_t* sb, int LDB,
                                           const float* near) {
  const int wave = wave_id(), lane = threadIdx.x & 63, g = lane >> 4, col = lane & 15, PA = kChunk * LDA, PB = kChunk * LDB;
  // tiles of rows wave, wave - 1, ... two at a time
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    const int j0 = afresh(wave) - 2 * q, j1 = max(j0 - 1, 0);
    phase();
    if (j0 < 0) continue;
    f32x4 sc[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
    for (int k = 0; k < STEPS; ++k) {
      auto row = [&](int j) { return st::row_op<P>(sa + (16 * j + col) * LDA + 32 * k + 8 * g, PA); };
      const Op<P> o0 = row(j0), o1 = row(j1);
      each_product<P, P>([&](int m, int y) {
        sc[0] = st::mfma(o0.p[m], x[k].p[y], sc[0]);
        sc[1] = st::mfma(o1.p[m], x[k].p[y], sc[1]);
      });
    }
    f32x8 v;
    const float* w = near + (kChunk - 1 - 32 * q - col + 4 * g);
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      v[r] = (q > 0 || col >= 4 * g + r ? sc[0][r] : 0.f) * w[r];
      v[4 + r] = (j0 > 0 ? sc[1][r] : 0.f) * w[r - 16];
    }
    const uint16_t* lb = sb + lane_tr8(lane, LDB);
    Op<P> bt[TB];
#pragma unroll
    for (int j = 0; j < TB; ++j) bt[j] = columns<P>(lb + 16 * j0 * LDB + tile_pair(j), lb + 16 * j1 * LDB + tile_pair(j), PB);
    const Op<kPieces> o = pieces(v);
    each_product<P, kPieces>([&](int m, int y) {
#pragma unroll
      for (int j = 0; j < TB; ++j) acc[j] = st::mfma(bt[j].p[m], o.p[y], acc[j]);
    });
  }
}

// ------------------------------------------------------------------------------------------------ rows
// Waves to a SIMD: what LDS allows, or registers without spills.
constexpr int cols_waves(int P, int WAVES, bool full, int shared) { return full && P == 1 && WAVES == 8 && !(shared & 1) ? 4 : (P == 1 ? 2 : 3); }
constexpr int walk_waves(bool full, bool shared) { return full && !shared ? 4 : (full ? 3 : 2); }
// SHARED: heads of X share states.  (Those of A and B do in k_decay_back and k_decay_cols.)
template <int P, int W, int TB, bool FULL, int DT, bool SHARED>
__global__ void __launch_bounds__(256, walk_waves(FULL, SHARED)) k_decay_walk(WalkSet set, int ncb, int parts) {
  constexpr int NB = 16 * TB, STEPS = W / 32, LDA = stride(W), LDB = stride(NB), PA = kChunk * LDA, PB = kChunk * LDB;
  constexpr int IMG = STEPS * kPieces * 512;                       // numbers of one column tile of the state's image
  extern __shared__ char lds[];
  uint16_t *sa = (uint16_t*)lds, *sb = sa + P * PA, *img = sb + P * PB;
  float *uw = (float*)(img + TB * IMG), *near = uw + kChunk, *pw = near + kNear;      // weights; lambda^0 .. lambda^64
  const Call& c = set.c;
  const Walk& w = set.w[blockIdx.y];
  Place p;
  if (!place(c, c.nseg, ncb, parts, &p) || p.part >= w.parts) return;
  const int tid = threadIdx.x, wave = wave_id(), lane = tid & 63, g = lane >> 4, col = lane & 15, b0 = 64 * p.cb;
  if (b0 >= w.wb) return;
  if (c.left_out && p.slot == -2 && p.h == 0 && p.cb == 0 && p.part == 0 && p.seg == 0 && tid == 0 && blockIdx.y == 0) atomicAdd(c.left_out, 1);
  const int lo = p.seg * c.seg_rows, hi = min(p.len, lo + c.seg_rows);
  zero_rows(w.Y, p.b, p.h * w.parts + p.part, w.GX, max(lo, p.len), p.seg == c.nseg - 1 ? c.L : min(c.L, lo + c.seg_rows), b0, min(64, w.wb - b0));
  const int s = p.b * c.Hk + p.h;
  const bool ends = w.end != nullptr && c.nseg == 1 && p.part == 0 && (p.slot >= 0 || !w.end_pool);
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
  load_state<false, true>(S, from, w.sa, w.sb, w.wa, w.wb, t.at, t.bt, b0);
  const int back = w.back, GX = SHARED ? w.GX : 1, first = w.first;
  const float s_update = w.s_update;
  const int hq = (p.h * w.parts + p.part) * GX;
  const Head hx(w.X, p.b, hq), ha(w.A, p.b, p.h), hb(w.B, p.b, p.h), hy(w.Y, p.b, hq);
  Stage<P, W, FULL, DT> ra(ha, 0, w.wa, back);
  Stage<P, NB, FULL, DT> rb(hb, b0, w.wb, back);
  RowOps<P, STEPS, FULL, DT> rx(hx, w.wa, back);
  const RowStore<TB, FULL> ry(hy, w.Y.dtype, b0, w.wb, back);
  auto fetch_x = [&](int r0, int gx) { rx.fetch(hx.chunk(gx, r0, min(kChunk, hi - r0), p.len, back)); };
  auto fetch_rows = [&](int r0) {
    const int n = min(kChunk, hi - r0);
    ra.fetch(ha.chunk(0, r0, n, p.len, back));
    rb.fetch(hb.chunk(0, r0, n, p.len, back));
  };
  if (lo < hi) { fetch_rows(lo); fetch_x(lo, 0); }
  __syncthreads();
  put_near(near, pw, w.s_score);
  const float inter = w.s_inter * pw[16 * wave + col + first];
  put_weights(uw, pw, kChunk, first, s_update);

  auto put_image = [&]() {
#pragma unroll
    for (int i = 0; i < Tiles<W, TB>::AT; ++i)
#pragma unroll
      for (int j = 0; j < Tiles<W, TB>::BT; ++j) {
        const int a = 16 * (t.at + i) + 4 * g;
        uint16_t* to = img + (t.bt + j) * IMG + (a >> 5) * kPieces * 512 + ((((a & 31) >> 3) * 16 + col) * 8 + (a & 7));
        f32x4 x = S[i][j];
#pragma unroll
        for (int k = 0; k < kPieces; ++k) {
          const bf16x4 h = __builtin_convertvector(x, bf16x4);
          *(bf16x4*)(to + k * 512) = h;
          if (k + 1 < kPieces) x = rest_of(x, h);
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
    ra.store(sa);
    rb.store(sb);
    __syncthreads();
    if (more) fetch_rows(r0 + kChunk);
    for (int gx = 0; gx < GX; ++gx) {
      rx.ops(x);
      if (gx + 1 < GX) fetch_x(r0, gx + 1);
#pragma unroll
      for (int j = 0; j < TB; ++j) acc[j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int k = 0; k < STEPS; ++k) {
        Op<kPieces> o[TB];
#pragma unroll
        for (int j = 0; j < TB; ++j) o[j] = st::image_op<kPieces>(img + j * IMG + k * kPieces * 512, lane);
        each_product<kPieces, P>([&](int m, int y) {
#pragma unroll
          for (int j = 0; j < TB; ++j) acc[j] = st::mfma(o[j].p[m], x[k].p[y], acc[j]);
        });
      }
#pragma unroll
      for (int j = 0; j < TB; ++j) scale_by(acc[j], inter);
      add_scores<P, STEPS, TB>(acc, x, sa, LDA, sb, LDB, near);
      ry.put(hy.chunk(gx, r0, n, p.len, back), acc);
    }
    if (more) fetch_x(r0 + kChunk, 0);                          // (here x's registers are free)
    if (more || ends) {
      decay_state(S, keep);
      add_chunk<P, W, TB>(S, t, sa, sb, uw);
    }
    __syncthreads();
    if (more) put_image();
  }
  if (ends)
    store_state<false, true>(S, w.end + (w.end_pool ? (size_t)p.slot * c.Hk + p.h : (size_t)s) * c.state, w.sa, w.sb, w.wa, w.wb, t.at, t.bt, b0);
}

// The same by columns: a wave has sixteen columns of the state, all of its rows, in accumulators whose order of rows is that of an operand, so
// that the state never goes through LDS; the rows x do (every wave needs all of them), and so do the chunk's scores, whose tiles the waves share
// out.  Chunks of 16 NT rows.
template <int P, int W, int WAVES, int NT, bool FULL, int DT, int SHARED>
__global__ void __launch_bounds__(64 * WAVES, P == 3 && W == 128 ? 2 : cols_waves(P, WAVES, FULL, SHARED)) k_decay_cols(WalkSet set, int ncb, int parts) {
  constexpr int C = 16 * NT, T = 64 * WAVES, NB = 16 * WAVES, TA = W / 16, STEPS = W / 32, LDA = stride(W), LDB = stride(NB), PA = C * LDA, PB = C * LDB, NQ = NT / 2;
  constexpr int TILES = NT * (NT + 1) / 2;
  extern __shared__ char lds[];
  uint16_t *sx = (uint16_t*)lds, *sa = sx + P * PA, *sb = sa + P * PA, *ps = sb + P * PB;
  float *uw = (float*)(ps + NT * NQ * kPieces * 512), *near = uw + kChunk, *pw = near + kNear;
  const Call& c = set.c;
  const Walk& w = set.w[blockIdx.y];
  Place p;
  if (!place(c, c.nseg, ncb, parts, &p) || p.part >= w.parts) return;
  const int tid = threadIdx.x, wave = wave_id(), lane = tid & 63, g = lane >> 4, col = lane & 15, b0 = NB * p.cb, bw = b0 + 16 * wave;
  if (b0 >= w.wb) return;
  if (c.left_out && p.slot == -2 && p.h == 0 && p.cb == 0 && p.part == 0 && p.seg == 0 && tid == 0 && blockIdx.y == 0) atomicAdd(c.left_out, 1);
  const int lo = p.seg * c.seg_rows, hi = min(p.len, lo + c.seg_rows);
  zero_rows(w.Y, p.b, p.h * w.parts + p.part, w.GX, max(lo, p.len), p.seg == c.nseg - 1 ? c.L : min(c.L, lo + c.seg_rows), b0, min(NB, w.wb - b0));
  const int s = p.b * c.Hk + p.h;
  const bool ends = w.end != nullptr && c.nseg == 1 && p.part == 0 && (p.slot >= 0 || !w.end_pool);
  if (hi <= lo && !ends) return;
  const float ld = c.log_decay[p.h];
  for (int i = tid; i <= kChunk; i += T) pw[i] = power(ld, i);
  for (int i = tid; i < NT * NQ * kPieces * 64; i += T) *(u32x4*)(ps + 8 * i) = u32x4{0u, 0u, 0u, 0u};      // (tiles above the diagonal stay so)
  Keep keep = scalar(keep_of(ld, C));
  f32x4 S[TA][1];
  // (with segments the pool may hold the states after the call already)
  const float* from = w.init == nullptr && p.seg == 0 ? nullptr
                      : c.nseg > 1                    ? set.prefix[blockIdx.y] + ((size_t)s * c.nseg + p.seg) * c.state
                                                      : (p.slot >= 0 ? w.init + ((size_t)p.slot * c.Hk + p.h) * c.state : nullptr);
  load_state<true, false>(S, from, w.sa, w.sb, w.wa, w.wb, 0, 0, bw);
  const int back = w.back, GX = SHARED & 2 ? w.GX : 1, GA = SHARED & 1 ? w.GA : 1, first = w.first, wb = w.wb;
  const float s_update = w.s_update;
  const int hq = (p.h * w.parts + p.part) * GX;
  const Head hx(w.X, p.b, hq), ha(w.A, p.b, p.h * GA), hb(w.B, p.b, p.h * GA), hy(w.Y, p.b, hq);
  Stage<P, W, FULL, DT, C, T> rx(hx, 0, w.wa, back), ra(ha, 0, w.wa, back);
  Stage<P, NB, FULL, DT, C, T> rb(hb, b0, wb, back);
  const int size = w.Y.dtype == 0 ? 4 : 2, yrow = (back ? C - 1 - col : col) * hy.pitch + (bw + 4 * g) * size;
  const int ystep = back ? -16 * hy.pitch : 16 * hy.pitch;
  auto fetch_x = [&](int r0, int gx) { rx.fetch(hx.chunk(gx, r0, min(C, hi - r0), p.len, back)); };
  auto fetch_rows = [&](int r0, int ga) {
    const int n = min(C, hi - r0);
    ra.fetch(ha.chunk(ga, r0, n, p.len, back));
    rb.fetch(hb.chunk(ga, r0, n, p.len, back));
  };
  if (lo < hi) { fetch_rows(lo, 0); fetch_x(lo, 0); }
  __syncthreads();
  put_near(near, pw, w.s_score);
  put_weights(uw, pw, C, first, s_update);
  float inter[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) inter[t] = w.s_inter * pw[16 * t + col + first];
  f32x4 acc[NT];
  for (int r0 = lo; r0 < hi; r0 += C) {
    int n = min(C, hi - r0);
    const bool more = r0 + C < hi;
    if (n < C && ends) {
      asm("" : "+s"(n));                                      // (or powers for it would be found for every chunk)
      put_weights(uw, pw, n, first, s_update);
      keep = scalar(keep_of(ld, n));
    }
    for (int ga = 0; ga < GA; ++ga)
      for (int gx = 0; gx < GX; ++gx) {
        if (ga == 0) rx.store(sx);
        if (gx == 0) {
          ra.store(sa);
          rb.store(sb);
        }
        __syncthreads();
        // scores: tiles (t, j <= t) of rows x and rows a in turn to the waves
#pragma unroll
        for (int k0 = 0; k0 < TILES; k0 += WAVES) {
          const int k = afresh(k0 + wave);
          if (k >= TILES) break;
          phase();
          const int t = (k >= 1) + (k >= 3) + (k >= 6), j = k - t * (t + 1) / 2;
          f32x4 sc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int i = 0; i < STEPS; ++i) {
            const Op<P> a = st::row_op<P>(sa + (16 * j + col) * LDA + 32 * i + 8 * g, PA), x = st::row_op<P>(sx + (16 * t + col) * LDA + 32 * i + 8 * g, PA);
            each_product<P, P>([&](int m, int y) { sc = st::mfma(a.p[m], x.p[y], sc); });
          }
          const float* wn = near + (kChunk - 1 - 16 * (t - j) - col + 4 * g);
          f32x4 v;
#pragma unroll
          for (int r = 0; r < 4; ++r) v[r] = (t > j || col >= 4 * g + r ? sc[r] : 0.f) * wn[r];
          uint16_t* to = ps + (t * NQ + (j >> 1)) * kPieces * 512 + lane * 8 + 4 * (j & 1);
#pragma unroll
          for (int m = 0; m < kPieces; ++m) {
            const bf16x4 h = __builtin_convertvector(v, bf16x4);
            *(bf16x4*)(to + m * 512) = h;
            if (m + 1 < kPieces) v = rest_of(v, h);
          }
        }
        if (ga == 0) {
#pragma unroll
          for (int t = 0; t < NT; ++t) acc[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int i = 0; i < STEPS; ++i) {
            Op<P> x[NT];
#pragma unroll
            for (int t = 0; t < NT; ++t) x[t] = st::row_op<P>(sx + (16 * t + col) * LDA + 32 * i + 8 * g, PA);
            const f32x4 u = S[2 * i][0], v = S[2 * i + 1][0];
            const Op<kPieces> o = pieces(f32x8{u[0], u[1], u[2], u[3], v[0], v[1], v[2], v[3]});
            each_product<kPieces, P>([&](int m, int y) {
#pragma unroll
              for (int t = 0; t < NT; ++t) acc[t] = st::mfma(o.p[m], x[t].p[y], acc[t]);
            });
          }
#pragma unroll
          for (int t = 0; t < NT; ++t) scale_by(acc[t], inter[t]);
        }
        __syncthreads();
        // what the next turn stages: rows a and b from here on, rows x when the results' registers are free
        const bool last_x = gx == GX - 1, update = last_x && (more || ends);
        if (last_x && ga + 1 < GA) fetch_rows(r0, ga + 1);
        else if (last_x && more) fetch_rows(r0 + C, 0);
        // scores times rows b
        const uint16_t *la = sa + lane_tr8(lane, LDA), *lb = sb + st::lane_tr(lane, LDB) + 16 * wave;
        Op<P> b[NQ];
#pragma unroll
        for (int q = 0; q < NQ; ++q) {
          phase();
          b[q] = columns<P>(lb + 32 * q * LDB, lb + (32 * q + 16) * LDB, PB);
#pragma unroll
          for (int t = 2 * q; t < NT; ++t) {
            const Op<kPieces> o = st::image_op<kPieces>(ps + (t * NQ + q) * kPieces * 512, lane);
            each_product<P, kPieces>([&](int m, int y) { acc[t] = st::mfma(b[q].p[m], o.p[y], acc[t]); });
          }
        }
        if (ga == GA - 1) {
          phase();
          const Chunk k = hy.chunk(gx, r0, n, p.len, back);
          const int at = afresh_lane(yrow - k.shift(C));
#pragma unroll
          for (int t = 0; t < NT; ++t) {
            const int b = bw + 4 * g, o = at + t * ystep;
            if constexpr (FULL) {
              const __amdgpu_buffer_rsrc_t r = k.buffer();
              if (size == 4) __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, acc[t]), r, b < wb ? o : kNowhere, 0, 0);
              else __builtin_amdgcn_raw_buffer_store_b64(__builtin_bit_cast(u32x2, __builtin_convertvector(acc[t], bf16x4)), r, b < wb ? o : kNowhere, 0, 0);
            } else if (16 * t + col < n) {
              const TensorDev y{k.at + o, size == 4 ? 0 : 1, 0, 0, 0};
#pragma unroll
              for (int i = 0; i < 4; ++i)
                if (b + i < wb) store_elem(y, i, acc[t][i]);
            }
          }
          phase();
        }
        if (gx + 1 < GX) fetch_x(r0, gx + 1);
        else if (ga == GA - 1 && more) fetch_x(r0 + C, 0);
        // the sums of the state
        if (update) {
          if (ga == 0) decay_state(S, keep);
#pragma unroll
          for (int q = 0; q < NQ; ++q) {
            phase();
            const f32x4 w0 = *(const f32x4*)(uw + 4 * g + 32 * q), w1 = *(const f32x4*)(uw + 4 * g + 32 * q + 16);
            const f32x8 wt = {w0[0], w0[1], w0[2], w0[3], w1[0], w1[1], w1[2], w1[3]};
            const Op<kPieces> u = pieces(number<P>(b[q]) * wt);
#pragma unroll
            for (int i = 0; i < TA; i += 2) {
              Op<P> a[2];
#pragma unroll
              for (int k = 0; k < 2; ++k) a[k] = columns<P>(la + 32 * q * LDA + tile_pair(i + k), la + (32 * q + 16) * LDA + tile_pair(i + k), PA);
              each_product<P, kPieces>([&](int m, int y) {
#pragma unroll
                for (int k = 0; k < 2; ++k) S[i + k][0] = st::mfma(a[k].p[m], u.p[y], S[i + k][0]);
              });
            }
          }
        }
        __syncthreads();
      }
  }
  if (ends) store_state<true, false>(S, w.end + (w.end_pool ? (size_t)p.slot * c.Hk + p.h : (size_t)s) * c.state, w.sa, w.sb, w.wa, w.wb, 0, 0, bw);
}

// Gradients of keys and values in one walk (two walks of rows of 64 in bf16 read 403 MB where this one reads 268) from the last row to the first: dk_j = D_j v_j, dv_j = D_j' k_j with the state D of the rows q and
// dy behind, in LDS as rows of D', of which the one takes columns and the other rows.  set.w[0]: the values (X = V, A = dY, B = Q, Y = dK),
// set.w[1]: the keys (X = K, A = Q, B = dY, Y = dV).
template <int P, int W, bool FULL, int DT, bool SHARED>
__global__ void __launch_bounds__(256, P == 1 ? (FULL ? 3 : 2) : 1) k_decay_back(WalkSet set) {
  constexpr int TB = W / 16, STEPS = W / 32, LD = stride(W), PL = kChunk * LD, PI = W * LD;
  extern __shared__ char lds[];
  uint16_t *sq = (uint16_t*)lds, *sd = sq + P * PL, *img = sd + P * PL;
  float *uw = (float*)(img + kPieces * PI), *near = uw + kChunk, *pw = near + kNear;
  const Call& c = set.c;
  const Walk &wk = set.w[0], &wv = set.w[1];
  Place p;
  if (!place(c, c.nseg, 1, 1, &p)) return;
  const int tid = threadIdx.x, wave = wave_id(), lane = tid & 63, g = lane >> 4, col = lane & 15;
  const int lo = p.seg * c.seg_rows, hi = min(p.len, lo + c.seg_rows), pad = p.seg == c.nseg - 1 ? c.L : min(c.L, lo + c.seg_rows);
  zero_rows(wk.Y, p.b, p.h, 1, max(lo, p.len), pad, 0, wk.wb);
  zero_rows(wv.Y, p.b, p.h, 1, max(lo, p.len), pad, 0, wv.wb);
  const int s = p.b * c.Hk + p.h, G = SHARED ? wv.GA : 1;
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
  load_state<false, true>(S, from, wv.sa, wv.sb, wv.wa, wv.wb, t.at, t.bt, 0);
  const Head hq(wv.A, p.b, p.h * G), hd(wv.B, p.b, p.h * G), hk(wv.X, p.b, p.h), hv(wk.X, p.b, p.h), hdk(wk.Y, p.b, p.h), hdv(wv.Y, p.b, p.h);
  Stage<P, W, FULL, DT> rq(hq, 0, wv.wa, 1), rd(hd, 0, wv.wb, 1);
  RowOps<P, STEPS, FULL, DT> rk(hk, wv.wa, 1), rv(hv, wk.wa, 1);
  const RowStore<TB, FULL> to_k(hdk, wk.Y.dtype, 0, wk.wb, 1), to_v(hdv, wv.Y.dtype, 0, wv.wb, 1);
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
  put_near(near, pw, wv.s_score);
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
        for (int k = 0; k < kPieces; ++k) {
          const bf16x4 h = __builtin_convertvector(x, bf16x4);
          *(bf16x4*)(to + k * PI) = h;
          x -= __builtin_convertvector(h, f32x4);
        }
      }
  };
  put_image();
  Op<P> xk[STEPS], xv[STEPS];
  f32x4 dk[TB], dv[TB];
  const uint16_t *rows = img + col * LD + 8 * g, *cols = img + lane_tr8(lane, LD);
  for (int r0 = lo; r0 < hi; r0 += kChunk) {
    int n = min(kChunk, hi - r0);
    const bool more = r0 + kChunk < hi;
    if (n < kChunk && ends) {
      asm("" : "+s"(n));
      put_weights(uw, pw, n, 0, s_update);
      keep = scalar(keep_of(ld, n));
    }
    for (int ga = 0; ga < G; ++ga) {
      rq.store(sq);
      rd.store(sd);
      __syncthreads();
      if (ga + 1 < G) fetch_rows(r0, ga + 1);
      else if (more) fetch_rows(r0 + kChunk, 0);
      if (ga == 0) {
        rk.ops(xk);
        rv.ops(xv);
#pragma unroll
        for (int j = 0; j < TB; ++j) dk[j] = dv[j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < STEPS; ++k) {
          phase();
          Op<kPieces> o[TB];
#pragma unroll
          for (int j = 0; j < TB; ++j) o[j] = st::row_op<kPieces>(rows + 16 * j * LD + 32 * k, PI);
          each_product<kPieces, P>([&](int m, int y) {
#pragma unroll
            for (int j = 0; j < TB; ++j) dv[j] = st::mfma(o[j].p[m], xk[k].p[y], dv[j]);
          });
          phase();
#pragma unroll
          for (int j = 0; j < TB; ++j) o[j] = columns<kPieces>(cols + 32 * k * LD + tile_pair(j), cols + (32 * k + 16) * LD + tile_pair(j), PI);
          each_product<kPieces, P>([&](int m, int y) {
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
      add_scores<P, STEPS, TB>(dk, xv, sd, LD, sq, LD, near);
      add_scores<P, STEPS, TB>(dv, xk, sq, LD, sd, LD, near);
      if (ga == G - 1) {
        to_k.put(hdk.chunk(0, r0, n, p.len, 1), dk);
        to_v.put(hdv.chunk(0, r0, n, p.len, 1), dv);
        if (more) fetch_x(r0 + kChunk);                          // (here the operands' registers are free)
      }
      if (more || ends) {
        if (ga == 0) decay_state(S, keep);
        add_chunk<P, W, TB>(S, t, sq, sd, uw);
      }
      __syncthreads();
    }
    if (more) put_image();
  }
  if (ends)
    store_state<false, true>(S, wv.end + (wv.end_pool ? (size_t)p.slot * c.Hk + p.h : (size_t)s) * c.state, wv.sa, wv.sb, wv.wa, wv.wb, t.at, t.bt, 0);
}

// ------------------------------------------------------------------------------------------------ sums of segments
// A wave has sixteen columns of the sums, all of their rows; the rows b are weighed.  Two chunks are on their way at a time where heads do not share states.
template <int P, int W, int WAVES, int C, bool FULL, int DT, bool SHARED>
__global__ void __launch_bounds__(64 * WAVES) k_decay_sum(SumSet set, int ncb) {
  constexpr int T = 64 * WAVES, NB = 16 * WAVES, TA = W / 16, LDA = stride(W), LDB = stride(NB), PA = C * LDA, PB = C * LDB;
  extern __shared__ char lds[];
  uint16_t *sa = (uint16_t*)lds, *sb = sa + P * PA;
  float *uw = (float*)(sb + P * PB), *pw = uw + kChunk;
  const Call& c = set.c;
  const Walk& w = set.w[blockIdx.y];
  Place p;
  if (!place(c, set.last ? c.nseg : c.nseg - 1, ncb, 1, &p)) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = wave_id(), b0 = NB * p.cb, first = w.first;
  const int lo = p.seg * c.seg_rows, hi = min(p.len, lo + c.seg_rows), back = w.back, GA = SHARED ? w.GA : 1;
  const float s_update = w.s_update;
  if (hi <= lo || b0 >= w.wb) return;
  const float ld = c.log_decay[p.h];
  for (int i = tid; i <= kChunk; i += T) pw[i] = power(ld, i);
  Keep keep = scalar(keep_of(ld, C));
  f32x4 S[TA][1];
  load_state<false, false>(S, nullptr, 0, 0, 0, 0, 0, 0, 0);
  const Head ha(w.A, p.b, p.h * GA), hb(w.B, p.b, p.h * GA);
  constexpr int AHEAD = SHARED || !FULL ? 1 : 2;
  Stage<P, W, FULL, DT, C, T> ra[2]{{ha, 0, w.wa, back}, {ha, 0, w.wa, back}};
  Stage<P, NB, FULL, DT, C, T> rb[2]{{hb, b0, w.wb, back}, {hb, b0, w.wb, back}};
  auto fetch_rows = [&](int i, int r0, int ga) {
    const int n = min(C, hi - r0);
    ra[i].fetch(ha.chunk(ga, r0, n, p.len, back));
    rb[i].fetch(hb.chunk(ga, r0, n, p.len, back));
  };
  fetch_rows(0, lo, 0);
  if (AHEAD == 2 && lo + C < hi) fetch_rows(1, lo + C, 0);
  __syncthreads();
  put_weights(uw, pw, C, first, s_update);
  const uint16_t *la = sa + st::lane_tr(lane, LDA), *lb = sb + st::lane_tr(lane, LDB) + 16 * wave;
  auto chunk = [&](int i, int r0) {
    int n = min(C, hi - r0);
    if (n < C) {
      asm("" : "+s"(n));
      put_weights(uw, pw, n, first, s_update);
      keep = scalar(keep_of(ld, n));
    }
    for (int ga = 0; ga < GA; ++ga) {
      ra[i].store(sa);
      rb[i].store(sb);
      __syncthreads();
      if (ga + 1 < GA) fetch_rows(i, r0, ga + 1);
      else if (r0 + AHEAD * C < hi) fetch_rows(i, r0 + AHEAD * C, 0);
      if (ga == 0 && r0 > lo) decay_state(S, keep);
#pragma unroll
      for (int q = 0; q < C / 32; ++q) {
        phase();
        const f32x4 w0 = *(const f32x4*)(uw + 4 * (lane >> 4) + 32 * q), w1 = *(const f32x4*)(uw + 4 * (lane >> 4) + 32 * q + 16);
        const f32x8 wt = {w0[0], w0[1], w0[2], w0[3], w1[0], w1[1], w1[2], w1[3]};
        const Op<kPieces> u = pieces(number<P>(columns<P>(lb + 32 * q * LDB, lb + (32 * q + 16) * LDB, PB)) * wt);
#pragma unroll
        for (int t = 0; t < TA; t += 2) {
          Op<P> a[2];
#pragma unroll
          for (int k = 0; k < 2; ++k) a[k] = columns<P>(la + 32 * q * LDA + 16 * (t + k), la + (32 * q + 16) * LDA + 16 * (t + k), PA);
          each_product<P, kPieces>([&](int m, int y) {
#pragma unroll
            for (int k = 0; k < 2; ++k) S[t + k][0] = st::mfma(a[k].p[m], u.p[y], S[t + k][0]);
          });
        }
      }
      __syncthreads();
    }
  };
  for (int r0 = lo; r0 < hi; r0 += AHEAD * C) {
    chunk(0, r0);
    if (AHEAD == 2 && r0 + C < hi) chunk(1, r0 + C);
  }
  const size_t s = (size_t)p.b * c.Hk + p.h;
  store_state<false, false>(S, set.part[blockIdx.y] + (s * c.nseg + p.seg) * c.state, w.sa, w.sb, w.wa, w.wb, 0, 0, b0 + 16 * wave);
}

// Sums of the segments -> states before them, in place; up to MANY segments on their way at a time.  What is read behind the segments that have
// sums is zeros, what is written behind those that have rows is nowhere: no branches (24 segments of 32 states of 64 x 64: 12.4 us with them, 9.6
// so, of which a launch with a load and a store is about 5).
template <int MANY> __global__ void __launch_bounds__(256) k_decay_join(JoinSet set) {
  const Call& c = set.c;
  const int which = blockIdx.z, s = blockIdx.y, b = s / c.Hk, h = s - b * c.Hk;
  int len = c.lengths ? max(0, min(c.lengths[b], c.L)) : c.L, slot;
  if (c.unique) {
    slot = st::unique_slot_of(c.slots, c.nslots, b);
    if (slot < 0) { slot = -2; len = 0; }
  } else {
    slot = st::slot_of(c.slots, c.nslots, b);
  }
  const int id = blockIdx.x * 256 + threadIdx.x, size = c.state * 4;
  if (id >= c.state) return;
  const int held = __builtin_amdgcn_readfirstlane((len + c.seg_rows - 1) / c.seg_rows);       // segments with rows
  // the last segment's sum is there (and wanted) where the states after it are
  const int sums = set.end[which] != nullptr ? held : min(held, c.nseg - 1);
  const float* part = set.part[which] + (size_t)s * c.nseg * c.state;
  const __amdgpu_buffer_rsrc_t from = buffer_of(part, sums * size), to = buffer_of(part, held * size);
  const float* init = set.init[which];
  float v[MANY];
#pragma unroll
  for (int i = 0; i < MANY; ++i) v[i] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(from, 4 * id + i * size, 0, 0));
  float S = init != nullptr && slot >= 0 ? init[((size_t)slot * c.Hk + h) * c.state + id] : 0.f;
  const float ld = c.log_decay[h];
  const Keep whole = scalar(keep_of(ld, c.seg_rows)), last = scalar(keep_of(ld, len - (held - 1) * c.seg_rows));
  for (int s0 = 0; s0 < held; s0 += MANY) {
    if (s0 > 0) {
#pragma unroll
      for (int i = 0; i < MANY; ++i) v[i] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(from, 4 * id + (s0 + i) * size, 0, 0));
    }
#pragma unroll
    for (int i = 0; i < MANY; ++i) {
      __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(S), to, 4 * id + (s0 + i) * size, 0, 0);
      const float next = kept(s0 + i == held - 1 ? last : whole, S) + v[i];
      S = s0 + i < held ? next : S;
    }
  }
  if (set.end[which] != nullptr && (slot >= 0 || !set.end_pool[which]))
    set.end[which][(set.end_pool[which] ? (size_t)slot * c.Hk + h : (size_t)s) * c.state + id] = S;
}

// States that a call in place has kept apart, into their slots (a launch of its own: what reads the pool has ended).
__global__ void __launch_bounds__(256) k_decay_put(Call c, const float* each, float* pool) {
  const int s = blockIdx.y, b = s / c.Hk, h = s - b * c.Hk, id = blockIdx.x * 256 + threadIdx.x;
  const int slot = st::unique_slot_of(c.slots, c.nslots, b);
  if (slot >= 0 && id < c.state) pool[((size_t)slot * c.Hk + h) * c.state + id] = each[(size_t)s * c.state + id];
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

// More LDS than a launch has by itself is asked for before it, on its device.
template <class K> int room(K kernel, size_t bytes) {
  if (bytes <= 65536) return 0;
  return hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes) == hipSuccess ? 0 : 5;
}

int most_parts(const WalkSet& a, int count) {
  int n = 1;
  for (int i = 0; i < count; ++i) n = max(n, a.w[i].parts);
  return n;
}

template <int P, int W, int TB, bool FULL, int DT, bool SHARED>
int walk_launch(const WalkSet& a, int count, hipStream_t st) {
  int ncb = 1;
  for (int i = 0; i < count; ++i) ncb = max(ncb, (a.w[i].wb + 16 * TB - 1) / (16 * TB));
  const size_t lds = (size_t)P * kChunk * (stride(W) + stride(16 * TB)) * 2 + (size_t)TB * (W / 32) * kPieces * 1024 + kTables;
  if (int rc = room(k_decay_walk<P, W, TB, FULL, DT, SHARED>, lds)) return rc;
  const long long units = ((long long)a.c.B * a.c.Hk * a.c.nseg + 7) / 8 * 8;
  const int parts = most_parts(a, count);
  if (units * ncb * parts > 0x7fffffffLL) return 2;
  hipLaunchKernelGGL((k_decay_walk<P, W, TB, FULL, DT, SHARED>), dim3((unsigned)(units * ncb * parts), count), dim3(256), lds, st, a, ncb, parts);
  return status();
}
template <int P, int W, int WAVES, bool FULL, int DT, int SHARED>
int cols_launch(const WalkSet& a, int count, hipStream_t st) {
  constexpr int NT = P == 1 ? 4 : 2, C = 16 * NT, NB = 16 * WAVES;
  int ncb = 1;
  for (int i = 0; i < count; ++i) ncb = max(ncb, (a.w[i].wb + NB - 1) / NB);
  const size_t lds = (size_t)P * C * (2 * stride(W) + stride(NB)) * 2 + (size_t)NT * (NT / 2) * kPieces * 1024 + kTables;
  if (int rc = room(k_decay_cols<P, W, WAVES, NT, FULL, DT, SHARED>, lds)) return rc;
  const long long units = ((long long)a.c.B * a.c.Hk * a.c.nseg + 7) / 8 * 8;
  const int parts = most_parts(a, count);
  if (units * ncb * parts > 0x7fffffffLL) return 2;
  hipLaunchKernelGGL((k_decay_cols<P, W, WAVES, NT, FULL, DT, SHARED>), dim3((unsigned)(units * ncb * parts), count), dim3(64 * WAVES), lds, st, a, ncb, parts);
  return status();
}
template <int P, int W, bool FULL, int DT, bool SHARED>
int back_launch(const WalkSet& a, hipStream_t st) {
  const size_t lds = (size_t)P * kChunk * stride(W) * 4 + (size_t)kPieces * W * stride(W) * 2 + kTables;
  if (int rc = room(k_decay_back<P, W, FULL, DT, SHARED>, lds)) return rc;
  const long long units = ((long long)a.c.B * a.c.Hk * a.c.nseg + 7) / 8 * 8;
  if (units > 0x7fffffffLL) return 2;
  hipLaunchKernelGGL((k_decay_back<P, W, FULL, DT, SHARED>), dim3((unsigned)units), dim3(256), lds, st, a);
  return status();
}
template <int P, int W, int WAVES, bool FULL, int DT, bool SHARED>
int sum_launch(const SumSet& a, int count, hipStream_t st) {
  constexpr int C = P == 1 ? 64 : 32, NB = 16 * WAVES;
  int ncb = 1;
  for (int i = 0; i < count; ++i) ncb = max(ncb, (a.w[i].wb + NB - 1) / NB);
  const size_t lds = (size_t)P * C * (stride(W) + stride(NB)) * 2 + kTables;
  if (int rc = room(k_decay_sum<P, W, WAVES, C, FULL, DT, SHARED>, lds)) return rc;
  const long long units = ((long long)a.c.B * a.c.Hk * (a.last ? a.c.nseg : a.c.nseg - 1) + 7) / 8 * 8;
  if (units == 0) return 0;
  if (units * ncb > 0x7fffffffLL) return 2;
  hipLaunchKernelGGL((k_decay_sum<P, W, WAVES, C, FULL, DT, SHARED>), dim3((unsigned)(units * ncb), count), dim3(64 * WAVES), lds, st, a, ncb);
  return status();
}

int class_of(int n) { return n <= 32 ? 32 : (n <= 64 ? 64 : 128); }

// (Heads of A and B share states, SHARED = 1, where dK and dV are two walks, whose sides are both as wide as the wider one of the rows: more than 64.)
template <int P, bool FULL, int DT, int SHARED> int walk_width(const WalkSet& a, int count, int wa, int wb, hipStream_t st) {
  if constexpr (SHARED == 1) {
    return class_of(wa) == 128 && wb > 64 ? cols_launch<P, 128, 8, FULL, DT, SHARED>(a, count, st) : 2;
  } else {
    if (class_of(wa) == 128)
      return wb > 64 ? cols_launch<P, 128, 8, FULL, DT, SHARED>(a, count, st) : cols_launch<P, 128, 4, FULL, DT, SHARED>(a, count, st);
    if constexpr (P == 3) {
      return class_of(wa) == 64 ? cols_launch<P, 64, 4, FULL, DT, SHARED>(a, count, st) : cols_launch<P, 32, 4, FULL, DT, SHARED>(a, count, st);
    } else {
      if (class_of(wa) == 64) return walk_launch<P, 64, 4, FULL, DT, (SHARED > 0)>(a, count, st);
      return wb <= 32 ? walk_launch<P, 32, 2, FULL, DT, (SHARED > 0)>(a, count, st) : walk_launch<P, 32, 4, FULL, DT, (SHARED > 0)>(a, count, st);
    }
  }
}
// (fp32 rows of more than 32 only where heads share states)
template <int P, bool FULL, int DT, bool SHARED> int back_width(const WalkSet& a, int w, hipStream_t st) {
  if (w <= 32) return back_launch<P, 32, FULL, DT, SHARED>(a, st);
  if constexpr (P == 1 || SHARED) return back_launch<P, 64, FULL, DT, SHARED>(a, st);
  else return 2;
}
template <int P, bool FULL, int DT, bool G> int sum_width(const SumSet& a, int count, int wa, int wb, hipStream_t st) {
  if (class_of(wa) == 128) return wb > 64 ? sum_launch<P, 128, 8, FULL, DT, G>(a, count, st) : sum_launch<P, 128, 4, FULL, DT, G>(a, count, st);
  if (class_of(wa) == 64) return wb > 32 ? sum_launch<P, 64, 4, FULL, DT, G>(a, count, st) : sum_launch<P, 64, 2, FULL, DT, G>(a, count, st);
  return wb > 32 ? sum_launch<P, 32, 4, FULL, DT, G>(a, count, st) : sum_launch<P, 32, 2, FULL, DT, G>(a, count, st);
}

// A kernel's form for rows without a ragged end, for heads that share states.  (Where none do, loops of one turn are left out: fewer registers.)
template <class F> int each_form(bool full, bool shared, F go) {
  if (full) return shared ? go(std::true_type{}, std::true_type{}) : go(std::true_type{}, std::false_type{});
  return go(std::false_type{}, std::true_type{});
}

}  // namespace

// Walks from .. from + count - 1 in one launch.
int launch_walks(const WalkSet& all, int from, int count, int dtype, hipStream_t st) {
  WalkSet a = all;
  int wa = 0, wb = 0;
  int shared = 0;                // 1: heads of A and B share states, 2: of X
  bool full = true;
  for (int i = 0; i < count; ++i) {
    shared |= (all.w[from + i].GA > 1 ? 1 : 0) | (all.w[from + i].GX > 1 ? 2 : 0);
    a.w[i] = all.w[from + i];
    a.prefix[i] = all.prefix[from + i];
    wa = max(wa, a.w[i].wa);
    wb = max(wb, a.w[i].wb);
    full = full && a.w[i].wa % 8 == 0 && a.w[i].wb % 8 == 0;
  }
  auto go = [&](auto full_rows, auto shared_heads) {
    constexpr bool F = decltype(full_rows)::value;
    constexpr int G = decltype(shared_heads)::value;
    return dtype == 0 ? walk_width<3, F, 0, G>(a, count, wa, wb, st) : walk_width<1, F, 1, G>(a, count, wa, wb, st);
  };
  using std::integral_constant;
  if (!full) return go(std::false_type{}, integral_constant<int, 3>{});
  if (shared == 0) return go(std::true_type{}, integral_constant<int, 0>{});
  // (heads of X share states in the walks of rows and of dQ, those of A and B in the walks of dK and dV: not in one launch)
  return shared == 1 ? go(std::true_type{}, integral_constant<int, 1>{}) : go(std::true_type{}, integral_constant<int, 2>{});
}

// The walks of dK and dV (from, from + 1) as one.
int launch_back(const WalkSet& all, int from, int dtype, hipStream_t st) {
  WalkSet a = all;
  for (int i = 0; i < 2; ++i) {
    a.w[i] = all.w[from + i];
    a.prefix[i] = all.prefix[from + i];
  }
  const Walk& w = a.w[1];
  const int n = max(w.wa, w.wb);
  auto go = [&](auto full_rows, auto shared_heads) {
    constexpr bool F = decltype(full_rows)::value, G = decltype(shared_heads)::value;
    return dtype == 0 ? back_width<3, F, 0, G>(a, n, st) : back_width<1, F, 1, G>(a, n, st);
  };
  return each_form(w.wa % 8 == 0 && w.wb % 8 == 0, w.GA > 1, go);
}

int launch_sums(const SumSet& a, int count, int dtype, hipStream_t st) {
  int wa = 0, wb = 0;
  bool full = true, shared = false;
  for (int i = 0; i < count; ++i) {
    shared = shared || a.w[i].GA > 1;
    wa = max(wa, a.w[i].wa);
    wb = max(wb, a.w[i].wb);
    full = full && a.w[i].wa % 8 == 0 && a.w[i].wb % 8 == 0;
  }
  auto go = [&](auto full_rows, auto shared_heads) {
    constexpr bool F = decltype(full_rows)::value, G = decltype(shared_heads)::value;
    return dtype == 0 ? sum_width<3, F, 0, G>(a, count, wa, wb, st) : sum_width<1, F, 1, G>(a, count, wa, wb, st);
  };
  return each_form(full, shared, go);
}

int launch_join(const JoinSet& a, hipStream_t st) {
  const dim3 grid((a.c.state + 255) / 256, a.c.B * a.c.Hk, a.count);
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(256), 0, st, a); };
  a.c.nseg <= 8 ? go(k_decay_join<8>) : a.c.nseg <= 16 ? go(k_decay_join<16>) : a.c.nseg <= 24 ? go(k_decay_join<24>) : go(k_decay_join<32>);
  return status();
}

int launch_put(const Call& c, const float* each, float* pool, hipStream_t st) {
  hipLaunchKernelGGL(k_decay_put, dim3((c.state + 255) / 256, c.B * c.Hk), dim3(256), 0, st, c, each, pool);
  return status();
}

int launch_slot_sums(const Call& c, const float* each, float* pool, hipStream_t st) {
  hipLaunchKernelGGL(k_decay_slot_sums, dim3((c.state + 63) / 64, c.nslots * c.Hk), dim3(256), 0, st, c, each, pool);
  return status();
}

}  // namespace dec
}  // namespace fs
