// Linear attention with a decay for each head, one token of every sequence: S = lambda S + k v', y = scale q S, the state in place.
//
// The state is read and written once, which bounds it.  A workgroup has all rows of a state and `cols` of its columns: the columns of y are
// its own, so that nothing is joined.  A thread has four columns of every 256 / (cols / 4)th row; y is summed over lanes and waves.
#include "decay_common.h"

namespace fs {
namespace dec {
namespace {

// C4: groups of four columns in a workgroup; R: rows of a thread on their way at a time; VEC: rows of the state at multiples of 16 bytes.
template <int C4, int R, bool VEC>
__global__ void __launch_bounds__(256) k_decay_step(StepArgs a, int ncb) {
  constexpr int ROWS = 256 / C4;
  __shared__ float qk[128 * 2];
  __shared__ float4 sums[4][C4];
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
  float* S = a.state + ((size_t)slot * a.Hk + h) * a.d * a.dv;
  const float lambda = power(a.log_decay[h], 1);
  const long long kb = st::row_base(a.K, b, h, 0), vb = st::row_base(a.V, b, h, 0);
  float v[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = c0 + i < a.dv ? load_elem(a.V, vb + c0 + i) : 0.f;
  for (int i = tid; i < a.d; i += 256) qk[i] = load_elem(a.K, kb + i);
  auto at = [&](int row, float4* x) {
    const float* p = S + (size_t)row * a.dv + c0;
    if (VEC) *x = *(const float4*)p;
    else *x = make_float4(p[0], c0 + 1 < a.dv ? p[1] : 0.f, c0 + 2 < a.dv ? p[2] : 0.f, c0 + 3 < a.dv ? p[3] : 0.f);
  };
  const bool mine = c0 < a.dv;
  for (int g = 0; g < G; ++g) {
    const long long qb = st::row_base(a.Q, b, h * G + g, 0);
    for (int i = tid; i < a.d; i += 256) qk[128 + i] = load_elem(a.Q, qb + i);
    __syncthreads();
    float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
    if (mine)
      for (int r0 = row0; r0 < a.d; r0 += R * ROWS) {
        float4 x[R];
#pragma unroll
        for (int i = 0; i < R; ++i)
          if (r0 + i * ROWS < a.d) at(r0 + i * ROWS, &x[i]);
#pragma unroll
        for (int i = 0; i < R; ++i) {
          const int row = r0 + i * ROWS;
          if (row >= a.d) continue;
          if (g == 0) {
            const float k = qk[row];
            x[i] = make_float4(fmaf(lambda, x[i].x, k * v[0]), fmaf(lambda, x[i].y, k * v[1]), fmaf(lambda, x[i].z, k * v[2]), fmaf(lambda, x[i].w, k * v[3]));
            float* p = S + (size_t)row * a.dv + c0;
            if (VEC) {
              *(float4*)p = x[i];
            } else {
              p[0] = x[i].x;
              if (c0 + 1 < a.dv) p[1] = x[i].y;
              if (c0 + 2 < a.dv) p[2] = x[i].z;
              if (c0 + 3 < a.dv) p[3] = x[i].w;
            }
          }
          const float q = qk[128 + row];
          y = make_float4(fmaf(q, x[i].x, y.x), fmaf(q, x[i].y, y.y), fmaf(q, x[i].z, y.z), fmaf(q, x[i].w, y.w));
        }
      }
#pragma unroll
    for (int m = C4; m < 64; m *= 2) {
      y.x += __shfl_xor(y.x, m);
      y.y += __shfl_xor(y.y, m);
      y.z += __shfl_xor(y.z, m);
      y.w += __shfl_xor(y.w, m);
    }
    if (lane < C4) sums[wave][lane] = y;
    __syncthreads();
    if (tid < 4 * C4 && 4 * cb * C4 + tid < a.dv) {
      float t = 0.f;
#pragma unroll
      for (int i = 0; i < 4; ++i) t += ((const float*)&sums[i][0])[tid];
      store_elem(a.Y, st::row_base(a.Y, b, h * G + g, 0) + 4 * cb * C4 + tid, a.scale * t);
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
  // narrow workgroups where there are few states
  if (a.B * a.Hk >= 512) vec ? go(k_decay_step<16, 4, true>, 64) : go(k_decay_step<16, 4, false>, 64);
  else vec ? go(k_decay_step<4, 2, true>, 16) : go(k_decay_step<4, 2, false>, 16);
  return hipGetLastError() == hipSuccess ? 0 : 5;
}

}  // namespace dec
}  // namespace fs
