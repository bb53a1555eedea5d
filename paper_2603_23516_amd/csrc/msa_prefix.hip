// msa_prefix_attend: one softmax over the rows of a prefix that all sequences share and over the rows of a sequence's own cache.
//
// A workgroup of four waves has sixteen columns, (token, query head) pairs of one (sequence, KV head), and deals the rows they see,
// 32 at a time, to its waves: S^T[key][col] = K q^T by 16x16x32 bf16 MFMA with the keys straight from memory, an online softmax per
// column, O^T[dd][col] += V^T P^T with the value rows through LDS and transposing reads.
#include "msa_prefix.h"

namespace msa {

__device__ __forceinline__ float max_over_quads(float x) {  // over the lanes that share lane % 16
  uint32_t u = __float_as_uint(x);
  auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  x = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
  u = __float_as_uint(x);
  r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// What a wave holds of sixteen columns: lane (qd, n) rows 16 c + 4 qd .. + 3 of column n's output.
template <int D>
struct Columns {
  float m_run, l_run;
  f32x4_t o[D / 16];
};

// Rows [0, end) of K, V, [end][D], in steps of 32: steps s, s + stride, ... below s_end.  Column n sees the rows below lim; least is
// the smallest lim of the wave's columns.  vt: 32 rows of LDS of the wave's own.
template <int D>
__device__ __forceinline__ void attend_rows(const uint16_t* K, const uint16_t* V, int end, int s, int s_end, int stride,
                                            const bf16x8_t (&bq)[D / 32], int lim, int least, float qscale, unsigned char* vt,
                                            Columns<D>& x) {
  constexpr int NS = D / 32, NC = D / 16, ROW = D * 2;
  const int lane = threadIdx.x & 63, qd = lane >> 4, n = lane & 15;
  // Value rows in LDS: 16-byte piece p of row i lies at place p ^ swz(i), so that neither the writes (16 rows, one piece) nor
  // the transposing reads (four rows, two pieces) meet in a bank.
  auto swz = [](int i) { return D == 128 ? 2 * (i & 7) : 2 * ((i >> 1) & 3); };
  uint4 kx[2][NS], vx[2][NS];
  auto load = [&](int t0) __attribute__((always_inline)) {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      int row = t0 + 16 * t + n;
      row = row < end ? row : end - 1;
      const long long at = (long long)row * D + 8 * qd;
#pragma unroll
      for (int j = 0; j < NS; ++j) {
        kx[t][j] = *reinterpret_cast<const uint4*>(K + at + 32 * j);
        vx[t][j] = *reinterpret_cast<const uint4*>(V + at + 32 * j);
      }
    }
  };
  if (s >= s_end) return;
  load(32 * s);
  for (; s < s_end; s += stride) {
    f32x4_t sc[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int j = 0; j < NS; ++j) {
        sc[t] = mfma16(as_bf16x8(kx[t][j]), bq[j], sc[t]);
        *reinterpret_cast<uint4*>(vt + (16 * t + n) * ROW + (((4 * j + qd) ^ swz(16 * t + n)) * 16)) = vx[t][j];
      }
    if (s + stride < s_end) load(32 * (s + stride));  // under way while this step's weights are worked out
    const int t0 = 32 * s;
    float w[8], mx = -INFINITY;
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = sc[i >> 2][i & 3] * qscale;
    if (t0 + 32 > least) {
#pragma unroll
      for (int i = 0; i < 8; ++i) w[i] = t0 + (i >> 2) * 16 + 4 * qd + (i & 3) < lim ? w[i] : -INFINITY;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) mx = fmaxf(mx, w[i]);
    mx = max_over_quads(mx);
    // m_run is what the weights are taken relative to, not the maximum itself: it follows once that is 2^8 ahead
    if (__ballot(mx > x.m_run + 8.f) != 0) {
      const float m_new = fmaxf(x.m_run, mx);
      const float alpha = x.m_run == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(x.m_run - m_new);
      x.m_run = m_new;
      x.l_run *= alpha;
#pragma unroll
      for (int c = 0; c < NC; ++c) x.o[c] *= alpha;
    }
    const float m_use = x.m_run == -INFINITY ? 0.f : x.m_run;
    uint32_t pw[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float p0 = __builtin_amdgcn_exp2f(w[2 * j] - m_use), p1 = __builtin_amdgcn_exp2f(w[2 * j + 1] - m_use);
      x.l_run += p0 + p1;
      pw[j] = pack_bf16(p0, p1);
    }
    const bf16x8_t pb = as_bf16x8(make_uint4(pw[0], pw[1], pw[2], pw[3]));
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    const int row = 4 * qd + (n >> 2);
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const unsigned char* vp = vt + row * ROW + (((2 * c + ((n & 3) >> 1)) ^ swz(row)) * 16) + 8 * (n & 1);
      const s16x4_t v0 = lds_read_tr16(vp), v1 = lds_read_tr16(vp + 16 * ROW);  // rows 16 apart: the same swizzle
      const bf16x8_t av = __builtin_bit_cast(bf16x8_t, __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7));
      x.o[c] = mfma16(av, pb, x.o[c]);
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }
}

template <int D>
__global__ __launch_bounds__(256) void prefix_rows_kernel(PrefixArgs a, int groups) {
  constexpr int NS = D / 32, NC = D / 16;
  constexpr int ROW = D * 2, OROW = D + 4;  // bytes of a value row, floats of a row of a wave's output in the merge
  constexpr int STAGE = 32 * ROW > 16 * OROW * 4 ? 32 * ROW : 16 * OROW * 4;
  __shared__ __attribute__((aligned(16))) unsigned char stage[4][STAGE];
  __shared__ float wm[4][16], wl[4][16];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int qd = lane >> 4, n = lane & 15, r = a.r, tpl = 16 / r;
  const int g = (int)(blockIdx.x % a.Hkv), x = (int)(blockIdx.x / a.Hkv), m0 = x % groups * tpl;
  const long long b = x / groups;
  const int tl = n / r, tok = m0 + tl;
  const bool ok = tl < tpl && tok < a.M;
  const long long qh = (b * a.M + (ok ? tok : m0)) * a.Hq + g * r + (ok ? n - tl * r : 0);
  bf16x8_t bq[NS];
#pragma unroll
  for (int s = 0; s < NS; ++s) {
    uint4 v = *reinterpret_cast<const uint4*>(a.q + qh * D + 32 * s + 8 * qd);
    if (!ok) v = make_uint4(0, 0, 0, 0);
    bq[s] = as_bf16x8(v);
  }
  int pre = a.Lpre;
  if (a.pre_lens != nullptr) {
    pre = a.pre_lens[b];
    pre = pre < 0 ? 0 : (pre > a.Lpre ? a.Lpre : pre);
  }
  pre = __builtin_amdgcn_readfirstlane(pre);
  const long long p1 = (long long)a.q_pos[b * a.M + (ok ? tok : m0)] - a.pos0 + 1;
  const int lim = ok ? (p1 < 0 ? 0 : (p1 < a.Lloc ? (int)p1 : a.Lloc)) : 0;
  int least = ok ? lim : INT32_MAX, most = lim;
#pragma unroll
  for (int off = 8; off > 0; off >>= 1) {
    const int u = __shfl_xor(least, off, 64), v = __shfl_xor(most, off, 64);
    least = u < least ? u : least;
    most = v > most ? v : most;
  }
  least = __builtin_amdgcn_readfirstlane(least);
  most = __builtin_amdgcn_readfirstlane(most);
  Columns<D> y;
  y.m_run = -INFINITY;
  y.l_run = 0.f;
#pragma unroll
  for (int c = 0; c < NC; ++c) y.o[c] = (f32x4_t){0.f, 0.f, 0.f, 0.f};
  attend_rows<D>(a.Kpre + (long long)g * a.Lpre * D, a.Vpre + (long long)g * a.Lpre * D, pre, wave, (pre + 31) / 32, 4, bq,
                 ok ? pre : 0, pre, a.qscale, stage[wave], y);
  const long long loc = (b * a.Hkv + g) * a.Lloc * D;
  attend_rows<D>(a.Kloc + loc, a.Vloc + loc, most, wave, (most + 31) / 32, 4, bq, lim, least, a.qscale, stage[wave], y);

  // the four waves' results
  y.l_run = add_xor32(add_xor16(y.l_run));
  float* const mine = reinterpret_cast<float*>(stage[wave]);
#pragma unroll
  for (int c = 0; c < NC; ++c) *reinterpret_cast<f32x4_t*>(mine + n * OROW + 16 * c + 4 * qd) = y.o[c];
  if (qd == 0) {
    wm[wave][n] = y.m_run;
    wl[wave][n] = y.l_run;
  }
  __syncthreads();
  for (int e = tid; e < 16 * D; e += 256) {
    const int c = e / D, dd = e % D, t = c / r;
    if (t >= tpl || m0 + t >= a.M) continue;
    const long long at = (b * a.M + m0 + t) * a.Hq + g * r + (c - t * r);
    float m = wm[0][c];
#pragma unroll
    for (int w = 1; w < 4; ++w) m = fmaxf(m, wm[w][c]);
    float l = 0.f, v = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float f = wm[w][c] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(wm[w][c] - m);
      l += f * wl[w][c];
      v += f * reinterpret_cast<const float*>(stage[w])[c * OROW + dd];
    }
    a.out[at * D + dd] = (uint16_t)pack_bf16(l > 0.f ? v / l : 0.f, 0.f);
    if (dd == 0 && a.lse != nullptr) a.lse[at] = l > 0.f ? (m + log2f(l)) * 0.6931471805599453f : -INFINITY;
  }
}

PrefixPlan plan_prefix(const Dims& dm, int B, int M, int Lpre, int Lloc) {
  PrefixPlan p = {};
  const int tpl = 16 / dm.r;
  if ((long long)B * ((M + tpl - 1) / tpl) * dm.Hkv >= 1 << 24) return p;
  p.ws_bytes = 256;
  return p;
}

int launch_prefix(const Dims& dm, const PrefixPlan& pl, PrefixArgs a, void* ws, hipStream_t st) {
  a.Hq = dm.Hq;
  a.Hkv = dm.Hkv;
  a.r = dm.r;
  a.qscale = (float)(1.4426950408889634 / sqrt((double)dm.d));
  const int tpl = 16 / dm.r, groups = (a.M + tpl - 1) / tpl;
  const dim3 grid((unsigned)((long long)a.B * groups * dm.Hkv));
  if (dm.d == 128)
    hipLaunchKernelGGL(prefix_rows_kernel<128>, grid, dim3(256), 0, st, a, groups);
  else
    hipLaunchKernelGGL(prefix_rows_kernel<64>, grid, dim3(256), 0, st, a, groups);
  return hipGetLastError() == hipSuccess ? MSA_OK : MSA_ERR_HIP;
}

}  // namespace msa
