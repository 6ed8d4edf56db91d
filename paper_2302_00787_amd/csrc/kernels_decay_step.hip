// Linear attention with a decay for each head, one token of every sequence: S = lambda S + k v', y = scale q S, the state in place.
//
// The state is read and written once, which bounds it.  A workgroup has all rows of a state and 4 C4 of its columns: the columns of y are its
// own, so that nothing is joined.  A thread has four columns of every (256 / C4)th row, all of them on their way before anything is waited for,
// and keeps them for the query heads that share the state; y is summed over lanes, then over waves, for four heads at a time.
// 256 x 8 states of 64 x 64, 69 MB: 12.2 us, 5.6 TB/s (in the last cache in part); 8 states: 4.8 us, a launch and a chain of two loads; 45 x 4
// states of 128 x 128 with four heads each: 9.0.
#include "decay_common.h"

#include <type_traits>

namespace fs {
namespace dec {
namespace {

constexpr int kHeads = 4;
constexpr int R_of(int D, int C4) { return D * C4 >= 256 ? D * C4 / 256 : 1; }                  // rows of a thread

// D: rows of a state at most, 64 or 128; VEC: they are at multiples of 16 bytes.  Eight waves to a SIMD, so that the loads of all that a chip
// holds are on their way together.
template <int D, int C4, bool VEC>
__global__ void __launch_bounds__(256, R_of(D, C4) > 6 ? 6 : 8) k_decay_step(StepArgs a, int ncb) {
  constexpr int ROWS = 256 / C4, R = R_of(D, C4);
  __shared__ float ks[128], qs[kHeads][128];
  __shared__ f32x4 sums[kHeads][4][C4];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int s = blockIdx.x / ncb, cb = blockIdx.x - s * ncb, b = s / a.Hk, h = s - b * a.Hk, G = a.H / a.Hk;
  const int slot = st::unique_slot_of(a.slots, a.nslots, b);
  const int c0 = 4 * (cb * C4 + tid % C4), row0 = tid / C4;
  if (slot < 0) {
    if (a.left_out && h == 0 && cb == 0 && tid == 0) atomicAdd(a.left_out, 1);
    for (int id = tid; id < G * 4 * C4; id += 256) {
      const int col = 4 * cb * C4 + id % (4 * C4);
      if (col < a.dv) store_elem(a.Y, st::row_base(a.Y, b, h * G + id / (4 * C4), 0) + col, 0.f);
    }
    return;
  }
  float* S = a.state + ((size_t)__builtin_amdgcn_readfirstlane(slot) * a.Hk + h) * a.d * a.dv;       // (a scalar, offsets 32 bits)
  const bool mine = c0 < a.dv;
  f32x4 x[R];
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const int row = row0 + i * ROWS;
    x[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (mine && row < a.d) {
      const float* p = S + (uint32_t)(row * a.dv + c0);
      if (VEC) {
        x[i] = *(const f32x4*)p;
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (c0 + j < a.dv) x[i][j] = p[j];
      }
    }
  }
  const long long kb = st::row_base(a.K, b, h, 0), vb = st::row_base(a.V, b, h, 0);
  f32x4 v;
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = c0 + i < a.dv ? load_elem(a.V, vb + c0 + i) : 0.f;
  const float lambda = power(a.log_decay[h], 1);
  if (tid < 128) ks[tid] = tid < a.d ? load_elem(a.K, kb + tid) : 0.f;
  for (int g0 = 0; g0 < G; g0 += kHeads) {
    for (int id = tid; id < kHeads * 128; id += 256) {
      const int g = g0 + id / 128, i = id % 128;
      qs[id / 128][i] = g < G && i < a.d ? load_elem(a.Q, st::row_base(a.Q, b, h * G + g, 0) + i) : 0.f;
    }
    __syncthreads();
    if (g0 == 0) {
#pragma unroll
      for (int i = 0; i < R; ++i) {
        const int row = row0 + i * ROWS;
        if (!mine || row >= a.d) continue;
#pragma unroll
        for (int j = 0; j < 4; ++j) x[i][j] = fmaf(lambda, x[i][j], ks[row] * v[j]);
        float* p = S + (uint32_t)(row * a.dv + c0);
        if (VEC) {
          *(f32x4*)p = x[i];
        } else {
#pragma unroll
          for (int j = 0; j < 4; ++j)
            if (c0 + j < a.dv) p[j] = x[i][j];
        }
      }
    }
#pragma unroll
    for (int g = 0; g < kHeads; ++g) {
      if (g0 + g >= G) break;
      f32x4 y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < R; ++i) {
        const float q = qs[g][row0 + i * ROWS];
#pragma unroll
        for (int j = 0; j < 4; ++j) y[j] = fmaf(q, x[i][j], y[j]);
      }
#pragma unroll
      for (int m = C4; m < 64; m *= 2)
#pragma unroll
        for (int j = 0; j < 4; ++j) y[j] += __shfl_xor(y[j], m);
      if (lane < C4) sums[g][wave][lane] = y;
    }
    __syncthreads();
    for (int id = tid; id < kHeads * 4 * C4; id += 256) {
      const int g = id / (4 * C4), i = id % (4 * C4), col = 4 * cb * C4 + i;
      if (g0 + g >= G || col >= a.dv) continue;
      float t = 0.f;
#pragma unroll
      for (int w = 0; w < 4; ++w) t += ((const float*)&sums[g][w][0])[i];
      store_elem(a.Y, st::row_base(a.Y, b, h * G + g0 + g, 0) + col, a.scale * t);
    }
  }
}

}  // namespace

int launch_step(const StepArgs& a, hipStream_t st) {
  auto go = [&](auto kernel, int cols) {
    const int ncb = (a.dv + cols - 1) / cols;
    hipLaunchKernelGGL(kernel, dim3((unsigned)(a.B * a.Hk * ncb)), dim3(256), 0, st, a, ncb);
  };
  const bool vec = a.dv % 4 == 0;
  // narrower workgroups where there are few states
  const int states = a.B * a.Hk, wide = states * ((a.dv + 63) / 64), half = states * ((a.dv + 31) / 32);
  auto rows = [&](auto most) {
    constexpr int D = decltype(most)::value;
    if (wide >= 512) vec ? go(k_decay_step<D, 16, true>, 64) : go(k_decay_step<D, 16, false>, 64);
    else if (half >= 256) vec ? go(k_decay_step<D, 8, true>, 32) : go(k_decay_step<D, 8, false>, 32);
    else vec ? go(k_decay_step<D, 4, true>, 16) : go(k_decay_step<D, 4, false>, 16);
  };
  if (a.d <= 64) rows(std::integral_constant<int, 64>{});
  else rows(std::integral_constant<int, 128>{});
  return hipGetLastError() == hipSuccess ? 0 : 5;
}

}  // namespace dec
}  // namespace fs
