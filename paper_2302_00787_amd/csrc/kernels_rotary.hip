// Rotary positions: pairs of a row's first `rot` numbers turned by position times frequency, Y = amplitude R(position f) X.
//
// A thread has eight numbers of a row and their eight partners in registers, its angles once for all heads of its token (a part of
// the heads where there are few tokens): one read and one write of the rows bounds it.  The rows of the next head come while one is
// turned: 65536 tokens of 16 heads of 64 in bf16, 268 MB, 73.7 us without, 56.1 so, 4.8 TB/s, where a large copy reaches 5.1 (fp32
// rows of 128, 87 MB: 20.4 without, 21.2 so).
#include "state_common.h"

namespace fs {
namespace st {
namespace {

struct RotaryArgs {
  RotaryDev r;
  TensorDev X, X2, Y, Y2;
  int H, H2, B, L, d, units, heads_per_part;
  float sgn;
};

// Threads: units of sixteen turned numbers (pairs 8 u .. 8 u + 7 with their partners), then units of eight that stay; FAST: rot a multiple of
// 16, so that both halves of a unit are whole.
template <bool FAST>
__global__ void __launch_bounds__(256) k_rotary(RotaryArgs a) {
  const long long id = (long long)blockIdx.x * 256 + threadIdx.x;
  const int u = (int)(id % a.units);
  const long long token = id / a.units;
  if (token >= (long long)a.B * a.L) return;
  const int b = (int)(token / a.L), l = (int)(token - (long long)b * a.L);
  const int h0 = blockIdx.y * a.heads_per_part, h1 = min(h0 + a.heads_per_part, a.H + a.H2);
  const int r = a.r.rot >> 1, nturn = (r + 7) / 8;
  if (u < nturn) {
    // a head's numbers are on their way while the angles are found, or the head before is turned and stored
    const int f0 = a.r.interleaved ? 16 * u : 8 * u, f1 = a.r.interleaved ? 16 * u + 8 : r + 8 * u;
    Raw8 next[2];
    auto bring = [&](int h) {
      const TensorDev& X = h >= a.H ? a.X2 : a.X;
      const long long from = row_base(X, b, h >= a.H ? h - a.H : h, l);
      next[0] = fetch8<true>(X, from, f0, a.d);
      next[1] = fetch8<true>(X, from, f1, a.d);
    };
    if constexpr (FAST) bring(h0);
    const int pos = position_of(a.r, b, l);
    float cs[8], sn[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int p = 8 * u + i;
      const float2 x = cos_sin(pos, a.r.freqs[min(p, r - 1)], a.r.amplitude);
      cs[i] = x.x;
      sn[i] = a.sgn * x.y;
    }
    for (int h = h0; h < h1; ++h) {
      const bool two = h >= a.H;
      const TensorDev &X = two ? a.X2 : a.X, &Y = two ? a.Y2 : a.Y;
      const int hh = two ? h - a.H : h;
      const long long from = row_base(X, b, hh, l), to = row_base(Y, b, hh, l);
      if constexpr (FAST) {
        const f32x8 x = expand8<true>(next[0], X.dtype, f0, a.d), y = expand8<true>(next[1], X.dtype, f1, a.d);
        if (h + 1 < h1) bring(h + 1);
        f32x8 v, w;
        if (a.r.interleaved) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            v[2 * i] = x[2 * i] * cs[i] - x[2 * i + 1] * sn[i];
            v[2 * i + 1] = x[2 * i + 1] * cs[i] + x[2 * i] * sn[i];
            w[2 * i] = y[2 * i] * cs[4 + i] - y[2 * i + 1] * sn[4 + i];
            w[2 * i + 1] = y[2 * i + 1] * cs[4 + i] + y[2 * i] * sn[4 + i];
          }
        } else {
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            v[i] = x[i] * cs[i] - y[i] * sn[i];
            w[i] = y[i] * cs[i] + x[i] * sn[i];
          }
        }
        store8(Y, to, f0, a.d, v);
        store8(Y, to, f1, a.d, w);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int p = 8 * u + i;
          if (p < r) {
            const int c0 = a.r.interleaved ? 2 * p : p, c1 = a.r.interleaved ? 2 * p + 1 : r + p;
            const float x = load_elem(X, from + c0), y = load_elem(X, from + c1);
            store_elem(Y, to + c0, x * cs[i] - y * sn[i]);
            store_elem(Y, to + c1, y * cs[i] + x * sn[i]);
          }
        }
      }
    }
  } else {
    const int c0 = a.r.rot + 8 * (u - nturn);
    for (int h = h0; h < h1; ++h) {
      const bool two = h >= a.H;
      const TensorDev &X = two ? a.X2 : a.X, &Y = two ? a.Y2 : a.Y;
      if (X.ptr == Y.ptr) continue;                        // in place
      const int hh = two ? h - a.H : h;
      const long long from = row_base(X, b, hh, l), to = row_base(Y, b, hh, l);
      if constexpr (FAST) {
        store8(Y, to, c0, a.d, load8(X, from, c0, a.d));
      } else {
        for (int c = c0; c < min(c0 + 8, a.d); ++c) store_elem(Y, to + c, load_elem(X, from + c));
      }
    }
  }
}

__global__ void __launch_bounds__(256) k_rotary_table(RotaryDev r, int B, int L, float2* table) {
  const int pairs = r.rot >> 1;
  const long long id = (long long)blockIdx.x * 256 + threadIdx.x;
  const long long token = id / pairs;
  if (token >= (long long)B * L) return;
  const int p = (int)(id - token * pairs), b = (int)(token / L), l = (int)(token - (long long)b * L);
  table[id] = cos_sin(position_of(r, b, l), r.freqs[p], r.amplitude);
}

}  // namespace

int launch_rotary(const RotaryDev& r, const TensorDev& X, int H, const TensorDev& X2, int H2, int B, int L, int d, int transposed,
                  const TensorDev& Y, const TensorDev& Y2, hipStream_t st) {
  RotaryArgs a{r, X, X2, Y, Y2, H, H2, B, L, d, 0, 0, transposed ? -1.f : 1.f};
  a.units = (r.rot / 2 + 7) / 8 + (d - r.rot + 7) / 8;
  const long long threads = (long long)B * L * a.units, blocks = (threads + 255) / 256;
  if (blocks > 0xffffffLL) return 2;             // (threads of a launch have 32 bits)
  // a token's heads in one thread only where that leaves a workgroup for every place of a CU (32 tokens of 16 heads: 4.2 us a head a
  // thread)
  int parts = 1;
  while (parts < H + H2 && blocks * parts < 2048) parts *= 2;
  a.heads_per_part = (H + H2 + parts - 1) / parts;
  const dim3 grid((unsigned)blocks, (H + H2 + a.heads_per_part - 1) / a.heads_per_part);
  if (r.rot % 16 == 0) hipLaunchKernelGGL(k_rotary<true>, grid, dim3(256), 0, st, a);
  else hipLaunchKernelGGL(k_rotary<false>, grid, dim3(256), 0, st, a);
  return hipGetLastError() == hipSuccess ? 0 : 5;
}

int launch_rotary_table(const RotaryDev& r, int B, int L, float2* table, hipStream_t st) {
  const long long n = (long long)B * L * (r.rot / 2);
  if ((n + 255) / 256 > 0xffffffLL) return 2;
  hipLaunchKernelGGL(k_rotary_table, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, st, r, B, L, table);
  return hipGetLastError() == hipSuccess ? 0 : 5;
}

}  // namespace st
}  // namespace fs
