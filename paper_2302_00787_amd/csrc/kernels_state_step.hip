// The next token of every sequence: its key and value onto the state, then its queries against it, in one launch.
//
// A workgroup has a state of one key head: it reads it once and writes it once, which bounds the call (2 M (dv + 1) numbers of 4 bytes).  Its
// first rows are on their way from the start, while the exponents are made (a thread a feature, W in fp32 from L2, the row from LDS); the
// shift is the largest exponent ever met, exactly as in kernels_state.hip.
#include <algorithm>

#include "state_common.h"

namespace fs {
namespace st {
namespace {

constexpr int NTH = 512, NW = NTH / 64, GC = 4, AHEAD = 8;     // GC: query heads served by a pass over the state

__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o));
  return v;
}
__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
  return v;
}

// Floats in LDS: rows (key, queries), value, angles, exponents and features (key, queries), z, the partial outputs.
__host__ __device__ inline int step_lds_floats(int Mp) { return (GC + 1) * 128 + 128 + 128 + (GC + 2) * Mp + 4 * GC * NTH + 16; }

template <int VEC>
__global__ void __launch_bounds__(NTH) k_step(StepArgs a) {
  typedef __attribute__((ext_vector_type(VEC))) float vec;
  extern __shared__ __align__(16) float lds[];
  const int Mp = a.f.p.Mp, M = a.f.M, d = a.f.d, dv = a.dv, tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  float* x = lds;                              // [GC + 1][128]: the key, then queries
  float* value = x + (GC + 1) * 128;
  float2* cs = (float2*)(value + 128);         // [64]
  float* feat = (float*)cs + 128;              // [GC + 1][Mp]
  float* zn = feat + (GC + 1) * Mp;            // [Mp]
  float* part = zn + Mp;                       // [GC][rows of the pass][dv]
  float* word = part + 4 * GC * NTH;           // keep; row term by wave; normalisers
  const int b = blockIdx.x, h = blockIdx.y, G = a.H / a.Hk;
  const int slot = unique_slot_of(a.slots, a.state.slots, b);
  if (slot < 0) {
    for (int e = tid; e < G * dv; e += NTH) store_elem(a.Y, row_base(a.Y, b, h * G + e / dv, 0) + e % dv, 0.f);
    if (tid == 0 && a.unread != nullptr) atomicAdd(a.unread, G);
    return;
  }
  const size_t at = (size_t)slot * a.Hk + h;
  const int quads = (dv + VEC - 1) / VEC, pass = NTH / quads, q0 = tid % quads, r0 = tid / quads;       // rows of a pass over the state
  const bool worker = r0 < pass;
  vec* T = (vec*)(a.state.T + at * M * dv);
  vec first[AHEAD];
#pragma unroll
  for (int i = 0; i < AHEAD; ++i) {
    const int m = r0 + i * pass;
    if (worker && m < M) first[i] = T[(size_t)m * quads + q0];
  }
  const char* set = a.f.set(h);
  const float *W1 = (const float*)(set + a.f.p.off_w[0]), *W2 = (const float*)(set + a.f.p.off_w[1]), *bias = (const float*)(set + a.f.p.off_bias);
  const float old = a.state.shift[at];
  const int pairs = a.rot.rot >> 1;
  if (tid < pairs) cs[tid] = cos_sin(position_of(a.rot, b, 0), a.rot.freqs[tid], a.rot.amplitude);
  if (tid >= 128 && tid < 128 + dv) value[tid - 128] = load_elem(a.V, row_base(a.V, b, h, 0) + tid - 128);
  float keep = 0.f;
  int unread = 0;
  for (int g0 = 0; g0 < G; g0 += GC) {
    const int n = min(GC, G - g0), from = g0 == 0 ? 0 : 1;        // rows of x: the key in the first pass only
    __syncthreads();
    for (int e = tid + from * 128; e < (n + 1) * 128; e += NTH) {
      const int r = e >> 7, c = e & 127;
      const TensorDev& t = r == 0 ? a.K : a.Q;
      const long long base = row_base(t, b, r == 0 ? h : h * G + g0 + r - 1, 0);
      float y = 0.f;
      if (c < d) {
        y = load_elem(t, base + c);
        if (c < a.rot.rot) {
          const bool second = a.rot.interleaved ? c & 1 : c >= pairs;
          const int i = a.rot.interleaved ? c >> 1 : (second ? c - pairs : c);
          const float other = load_elem(t, base + (a.rot.interleaved ? c ^ 1 : (second ? c - pairs : c + pairs)));
          y = y * cs[i].x + (second ? other : -other) * cs[i].y;
        }
      }
      x[e] = y;
    }
    __syncthreads();
    // row term of the key: wave w sums over the columns c = w, w + NW, ...
    if (g0 == 0) {
      float sum = 0.f;
      if (a.f.dense) {
        const float* C2 = (const float*)(set + a.f.p.off_c2);
        for (int c = w; c < d; c += NW) {
          float z = 0.f;
          for (int l = lane; l < d; l += 64) z += x[l] * C2[c * d + l];
          sum += x[c] * z;
        }
      } else if (w == 0) {
        sum = -0.5f * (x[lane] * x[lane] + x[64 + lane] * x[64 + lane]);
      }
      sum = wave_sum(sum);
      if (lane == 0) word[w] = sum;
    }
    // exponents: features of the key, then those of the queries
    for (int e = tid + from * Mp; e < 2 * Mp; e += NTH) {
      const bool key = e < Mp;
      const int m = key ? e : e - Mp;
      const float* Wm = (key ? W2 : W1) + (size_t)m * 4;
      float s[GC] = {0.f, 0.f, 0.f, 0.f};
      if (key || n == 1) {
        const float* row = x + (key ? 0 : 128);
#pragma unroll 8
        for (int c = 0; c < a.f.p.d4; ++c) {
          const f32x4 u = *(const f32x4*)(Wm + (size_t)c * Mp * 4), v = *(const f32x4*)(row + 4 * c);
#pragma unroll
          for (int i = 0; i < 4; ++i) s[0] += u[i] * v[i];
        }
      } else {
#pragma unroll 4
        for (int c = 0; c < a.f.p.d4; ++c) {
          const f32x4 u = *(const f32x4*)(Wm + (size_t)c * Mp * 4);
#pragma unroll
          for (int j = 0; j < GC; ++j) {
            const f32x4 v = *(const f32x4*)(x + (1 + min(j, n - 1)) * 128 + 4 * c);
#pragma unroll
            for (int i = 0; i < 4; ++i) s[j] += u[i] * v[i];
          }
        }
      }
      if (key) feat[m] = s[0] + bias[m];
      else
#pragma unroll
        for (int j = 0; j < GC; ++j)
          if (j < n) feat[(1 + j) * Mp + m] = s[j] + bias[m];
    }
    __syncthreads();
    // features: wave 0 the key's and z, the others the queries'
    if (w == 0 && g0 == 0) {
      float term = 0.f;
#pragma unroll
      for (int i = 0; i < NW; ++i) term += word[i];
      term *= kLog2e * a.f.scale2;
      float top = kNone;
      for (int m = lane; m < Mp; m += 64) top = fmaxf(top, feat[m] + term);
      top = fmaxf(wave_max(top), old);
      const float k = old == kNone ? 0.f : fast_exp2(old - top);
      for (int m = lane; m < Mp; m += 64) {
        const float s = top == kNone ? 0.f : fast_exp2((feat[m] + term) - top);
        feat[m] = s;
        float z = s;
        if (m < M) {
          float* to = a.state.z + at * M + m;
          if (k != 0.f) z += k * *to;
          *to = z;
        }
        zn[m] = z;
      }
      if (lane == 0) {
        word[8] = k;
        a.state.shift[at] = top;
      }
    } else {
      const int j = w - (g0 == 0 ? 1 : 0);
      if (j < n) {
        float* p = feat + (1 + j) * Mp;
        float top = kNone;
        for (int m = lane; m < Mp; m += 64) top = fmaxf(top, p[m]);
        top = wave_max(top);
        for (int m = lane; m < Mp; m += 64) p[m] = fast_exp2(p[m] - top);
      }
    }
    __syncthreads();
    keep = word[8];
    if (w < n) {
      float den = 0.f;
      for (int m = lane; m < Mp; m += 64) den += feat[(1 + w) * Mp + m] * zn[m];
      den = wave_sum(den);
      if (lane == 0) word[12 + w] = den;
    }
    // the state
    vec acc[GC] = {};
    vec v;
#pragma unroll
    for (int i = 0; i < VEC; ++i) v[i] = worker ? value[VEC * q0 + i] : 0.f;
    if (worker)
      for (int m0 = r0; m0 < M; m0 += AHEAD * pass) {
        vec t[AHEAD];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
          const int m = m0 + i * pass;
          if (g0 == 0 && m0 == r0) t[i] = first[i];
          else if (m < M) t[i] = T[(size_t)m * quads + q0];
        }
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
          const int m = m0 + i * pass;
          if (m >= M) continue;
          if (g0 == 0) {
            vec n2 = feat[m] * v;
            if (keep != 0.f) n2 += keep * t[i];
            t[i] = n2;
            T[(size_t)m * quads + q0] = n2;
          }
#pragma unroll
          for (int j = 0; j < GC; ++j)
            if (j < n) acc[j] += feat[(1 + j) * Mp + m] * t[i];
        }
      }
    if (worker)
#pragma unroll
      for (int j = 0; j < GC; ++j)
        if (j < n)
#pragma unroll
          for (int i = 0; i < VEC; ++i) part[(j * pass + r0) * dv + VEC * q0 + i] = acc[j][i];
    __syncthreads();
    for (int e = tid; e < n * dv; e += NTH) {
      const int j = e / dv, c = e - j * dv;
      float sum = 0.f;
      for (int r = 0; r < pass; ++r) sum += part[(j * pass + r) * dv + c];
      const float den = word[12 + j];
      store_elem(a.Y, row_base(a.Y, b, h * G + g0 + j, 0) + c, den == 0.f ? 0.f : sum / den);
      unread += c == 0 && den == 0.f;
    }
  }
  if (unread > 0 && a.unread != nullptr) atomicAdd(a.unread, unread);
}

}  // namespace

int launch_step(const StepArgs& a, hipStream_t st) {
  const size_t lds = step_lds_floats(a.f.p.Mp) * sizeof(float);
  auto kernel = a.dv % 4 == 0 ? k_step<4> : k_step<1>;
  if (lds > 64 * 1024 && hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds) != hipSuccess) {
    (void)hipGetLastError();
    return 5;
  }
  hipLaunchKernelGGL(kernel, dim3(a.B, a.Hk), dim3(NTH), lds, st, a);
  return hipGetLastError() == hipSuccess ? 0 : 5;
}

}  // namespace st
}  // namespace fs
