// msa_attend_mass: the attention weight that every row of the local cache receives from the tokens of a call,
//     out[b][g][t] = decay mass[b][g][t] + sum over tokens m and heads h of group g that see row t of
//                    exp(q[b][m][h] . Kloc[b][g][t] / sqrt(d) - lse[b][m][h])
// with the log-sums that the attention left.  A wave owns 32 rows, which stay in registers; the (token, head) pairs go by sixteen at
// a time, scores by 16x16x32 bf16 MFMA (rows of K against columns of pairs), and every lane adds up its rows' weights, joined over
// the sixteen columns at the end.  Nothing depends on an order of arrival.
#include "msa_encoded.h"

namespace msa {

template <int D>
__global__ __launch_bounds__(256) void mass_rows_kernel(MassArgs a, int n_blocks) {
  constexpr int NS = D / 32;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int qd = lane >> 4, n = lane & 15, r = a.r;
  const long long pair = blockIdx.x / n_blocks;
  const int t0 = ((int)(blockIdx.x % n_blocks) * 4 + wave) * 32;
  if (t0 >= a.Lloc) return;  // no barrier below
  const int g = (int)(pair % a.Hkv);
  const long long b = pair / a.Hkv;
  float sum[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) sum[i] = 0.f;
  bool loaded = false;
  bf16x8_t k[2][NS];
  const int cols = a.M * r;
  for (int c0 = 0; c0 < cols; c0 += 16) {
    const int c = c0 + n < cols ? c0 + n : cols - 1;
    const long long tok = b * a.M + c / r;
    const long long qh = tok * a.Hq + g * r + c % r;
    const long long pl = (long long)a.q_pos[tok] - a.pos0;
    // rows t <= p with t >= lo or t < sinks
    int p = c0 + n < cols ? (pl < -1 ? -1 : (pl < a.Lloc ? (int)pl : a.Lloc - 1)) : -1;
    const float ls = a.lse[qh] * 1.4426950408889634f;
    if (ls == -INFINITY) p = -1;  // a token that saw nothing
    const long long lol = pl - a.window + 1;
    const int lo = lol < 0 ? 0 : (lol < a.Lloc ? (int)lol : a.Lloc);
    if (__ballot(t0 <= p && (t0 + 31 >= lo || t0 < a.sinks)) == 0) continue;
    if (!loaded) {
      loaded = true;
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const int row = t0 + 16 * t + n < a.Lloc ? t0 + 16 * t + n : a.Lloc - 1;
#pragma unroll
        for (int s = 0; s < NS; ++s)
          k[t][s] = as_bf16x8(*reinterpret_cast<const uint4*>(a.Kloc + (pair * a.Lloc + row) * D + 32 * s + 8 * qd));
      }
    }
    f32x4_t sc[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      const bf16x8_t q = as_bf16x8(*reinterpret_cast<const uint4*>(a.q + qh * D + 32 * s + 8 * qd));
      sc[0] = mfma16(k[0][s], q, sc[0]);
      sc[1] = mfma16(k[1][s], q, sc[1]);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int t = t0 + 16 * (i >> 2) + 4 * qd + (i & 3);
      const float w = __builtin_amdgcn_exp2f(fmaf(sc[i >> 2][i & 3], a.qscale, -ls));
      sum[i] += t <= p && (t >= lo || t < a.sinks) ? w : 0.f;
    }
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) sum[i] = add_over_16(sum[i]);
  if (n < 8) {
    float v = sum[0];
#pragma unroll
    for (int i = 1; i < 8; ++i) v = n == i ? sum[i] : v;
    const int t = t0 + 16 * (n >> 2) + 4 * qd + (n & 3);
    if (t < a.Lloc) {
      const long long at = pair * a.Lloc + t;
      if (a.mass != nullptr && a.decay != 0.f) v = fmaf(a.mass[at], a.decay, v);
      a.out[at] = v;
    }
  }
}

MassPlan plan_mass(const Dims& dm, int B, int M, int Lloc, int window, int sinks) {
  MassPlan p = {};
  const long long blocks = (long long)B * dm.Hkv * ((Lloc + 127) / 128);
  if (blocks >= 1 << 24) return p;
  p.ws_bytes = 256;
  return p;
}

int launch_mass(const Dims& dm, const MassPlan& pl, MassArgs a, int B, void* ws, hipStream_t st) {
  a.Hq = dm.Hq;
  a.Hkv = dm.Hkv;
  a.r = dm.r;
  a.qscale = (float)(1.4426950408889634 / sqrt((double)dm.d));
  const int n_blocks = (a.Lloc + 127) / 128;
  const dim3 grid((unsigned)((long long)B * dm.Hkv * n_blocks));
  if (dm.d == 128)
    hipLaunchKernelGGL(mass_rows_kernel<128>, grid, dim3(256), 0, st, a, n_blocks);
  else
    hipLaunchKernelGGL(mass_rows_kernel<64>, grid, dim3(256), 0, st, a, n_blocks);
  return hipGetLastError() == hipSuccess ? MSA_OK : MSA_ERR_HIP;
}

}  // namespace msa
