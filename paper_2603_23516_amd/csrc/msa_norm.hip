// msa_norm_rotate: what stands between the projections of a layer and its attention, in one pass over them:
//     y = x * rsqrt(mean_u x_u^2 + eps) * w          per head, in fp32
//     (y_u, y_{u + d/2}) turned by p * base^(-2u/d)    p the token's position
// rounded to bf16 once, queries to a dense tensor, keys and values into the rows of the local cache that msa_sparse_attend,
// msa_window_attend and msa_sparse_attend4 read.  Every element is read once and written once: bound by HBM for a prompt
// (16384 tokens of 48 heads of 128, 403 MB in and out: 75 us, 5.4 TB/s), by the latency of a load, the angles and a store
// for a few tokens (8: 4.2 us).  Stores carry the streaming hint at every size: kept in the L2 they displace what is still to
// be read (16384 tokens 85.5 us for 74.7, 4096 25.5 for 17.8).
//
// A row of d elements is held by d/16 lanes, eight elements at u0 = 8 l and their partners at u0 + d/2, so that a rotation
// needs no other lane and both loads are 16 bytes; a wave takes 64 / (d/16) heads of one token at a time.  A lane's eight
// angles are the same for all heads: the wave works out the d/2 angles of its token once, one per lane in double, and
// passes them around through LDS.
//
// msa_norm_rotate_axes is the same pass with several positions per token: the lane that works out angle u takes the position of
// axis axes[u], and the row of the cache comes with the token (AXES; a variant of its own, so that the other keeps its
// registers; the same times: 16384 tokens 74 us, 8 tokens 4.2).
#include "msa_attend.h"

namespace msa {

// The sum of a head's squares, in every lane that holds a part of it.
template <int LPH>
__device__ __forceinline__ float head_sum_of_squares(const float (&f1)[8], const float (&f2)[8]) {
  float ss = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) ss += f1[e] * f1[e] + f2[e] * f2[e];
  ss += dpp_f<kDppXor1>(ss);
  ss += dpp_f<kDppXor2>(ss);
  if (LPH == 8) ss += dpp_f<kDppHalfMirror>(ss);
  return ss;
}

// (Eight waves to a SIMD: the path of large squares would make it seven.)
template <int D, bool STREAM, bool AXES>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(8))) void norm_rotate_kernel(NormArgs a, NormTheta th) {
  constexpr int HALF = D / 2;
  constexpr int LPH = D / 16;    // lanes per head
  constexpr int HPW = 64 / LPH;  // heads per wave and turn
  __shared__ __attribute__((aligned(16))) float2 angles[4][HALF];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const long long job = (long long)blockIdx.x * 4 + wave;  // (token, share of its heads)
  const long long bm = job / a.shares;
  const int share = (int)(job - bm * a.shares);
  if (bm >= a.BM) return;  // wave-uniform; no barrier below
  const int32_t* const at = a.pos + (AXES ? bm * a.n_axes : bm);
  const int p = at[0];
  if (p < 0) return;  // padding
  const int l = lane % LPH, hl = lane / LPH;
  const long long row = AXES && a.rows != nullptr ? a.rows[bm] : (long long)p - a.pos0;
  const bool stored = row >= 0 && row < a.Lloc;
  const long long b = bm / a.M;

  if (a.rotate) {
    if (lane < HALF) angles[wave][lane] = cis_pos(AXES ? at[(a.axes[lane / 32] >> (2 * (lane % 32))) & 3] : p, th.th[lane]);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }
  float2 c[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) c[e] = a.rotate ? angles[wave][8 * l + e] : make_float2(1.f, 0.f);

  // turns over the heads: queries, then keys, then values, each in groups of HPW
  for (int t = share; t < a.turns; t += a.shares) {  // wave-uniform
    const int kind = t < a.turns_q ? 0 : (t < a.turns_q + a.turns_k ? 1 : 2);
    const int h = (t - (kind == 0 ? 0 : kind == 1 ? a.turns_q : a.turns_q + a.turns_k)) * HPW + hl;
    if (kind != 0 && !stored) return;  // keys and values come last
    if (h >= (kind == 0 ? a.Hq : a.Hkv)) continue;
    const uint16_t* src = (kind == 0 ? a.q + bm * a.q_stride : kind == 1 ? a.k + bm * a.k_stride : a.v + bm * a.v_stride) +
                          h * D + 8 * l;
    uint16_t* dst = (kind == 0 ? a.q_out + (bm * a.Hq + h) * D
                               : (kind == 1 ? a.Kloc : a.Vloc) + ((b * a.Hkv + h) * a.Lloc + row) * D) +
                    8 * l;
    const uint4 x1 = STREAM ? load_stream16(src) : *reinterpret_cast<const uint4*>(src);
    const uint4 x2 = STREAM ? load_stream16(src + HALF) : *reinterpret_cast<const uint4*>(src + HALF);
    if (kind == 2) {
      store_stream16(dst, x1);
      store_stream16(dst + HALF, x2);
      continue;
    }
    const uint32_t w1[4] = {x1.x, x1.y, x1.z, x1.w}, w2[4] = {x2.x, x2.y, x2.z, x2.w};
    float f1[8], f2[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      f1[e] = e & 1 ? bf16_hi(w1[e / 2]) : bf16_lo(w1[e / 2]);
      f2[e] = e & 1 ? bf16_hi(w2[e / 2]) : bf16_lo(w2[e / 2]);
    }
    const uint16_t* wt = kind == 0 ? a.qw : a.kw;
    if (wt != nullptr) {
      float ss = head_sum_of_squares<LPH>(f1, f2), eps = a.eps;
      if (__ballot(ss == INFINITY) != 0) {  // elements of 2^60 and more, whose squares fp32 does not hold: 2^-70 of them
        const float c = ss == INFINITY ? 0x1p-70f : 1.f;  // (the lanes of a head agree)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          f1[e] *= c;
          f2[e] *= c;
        }
        ss = head_sum_of_squares<LPH>(f1, f2);
        eps *= c;
        eps *= c;
      }
      const float rs = 1.0f / sqrtf(ss * (1.0f / D) + eps);
      const uint4 g1 = *reinterpret_cast<const uint4*>(wt + 8 * l), g2 = *reinterpret_cast<const uint4*>(wt + HALF + 8 * l);
      const uint32_t v1[4] = {g1.x, g1.y, g1.z, g1.w}, v2[4] = {g2.x, g2.y, g2.z, g2.w};
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        f1[e] *= rs * (e & 1 ? bf16_hi(v1[e / 2]) : bf16_lo(v1[e / 2]));
        f2[e] *= rs * (e & 1 ? bf16_hi(v2[e / 2]) : bf16_lo(v2[e / 2]));
      }
    }
    uint32_t y1[4], y2[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float2 c0 = c[2 * j], c1 = c[2 * j + 1];
      const float p0 = f1[2 * j], p1 = f1[2 * j + 1], q0 = f2[2 * j], q1 = f2[2 * j + 1];
      y1[j] = pack_bf16(p0 * c0.x - q0 * c0.y, p1 * c1.x - q1 * c1.y);
      y2[j] = pack_bf16(q0 * c0.x + p0 * c0.y, q1 * c1.x + p1 * c1.y);
    }
    store_stream16(dst, make_uint4(y1[0], y1[1], y1[2], y1[3]));
    store_stream16(dst + HALF, make_uint4(y2[0], y2[1], y2[2], y2[3]));
  }
}

int launch_norm_rotate(const Dims& dm, NormArgs a, hipStream_t st) {
  const int hpw = dm.d == 128 ? 8 : 16;
  a.Hq = dm.Hq;
  a.Hkv = dm.Hkv;
  a.turns_q = a.q != nullptr ? (dm.Hq + hpw - 1) / hpw : 0;
  a.turns_k = a.k != nullptr ? (dm.Hkv + hpw - 1) / hpw : 0;
  a.turns = a.turns_q + a.turns_k + (a.v != nullptr ? (dm.Hkv + hpw - 1) / hpw : 0);
  a.shares = 1;
  while (a.shares < a.turns && a.BM * a.shares < 4096) ++a.shares;
  NormTheta th;
  const RopeTheta& table = rope_table(dm.base, dm.d);
  for (int u = 0; u < kMaxHalf; ++u) th.th[u] = table.th[u];
  const long long blocks = (a.BM * a.shares + 3) / 4;
  // Projections that the caches do not hold: streaming loads.  us for 48 heads of 128, with plain loads / streaming ones, inputs
  // changing from call to call and, in brackets, right behind the product that wrote the projection: 16384 tokens (201 MB)
  // 81.7 / 74.7 [85.6 / 70.0], 12288 63.4 / 57.5 [65.7 / 54.5], 8192 (101 MB) 43.9 / 39.6 [34.4 / 34.6], 4096 17.8 / 22.0
  // [19.7 / 20.0].
  const int heads = (a.q != nullptr ? dm.Hq : 0) + (a.k != nullptr ? dm.Hkv : 0) + (a.v != nullptr ? dm.Hkv : 0);
  const bool stream = a.BM * heads * dm.d * 2 >= (128ll << 20);
#define MSA_NORM(DD, SS, AA) \
  hipLaunchKernelGGL((norm_rotate_kernel<DD, SS, AA>), dim3((unsigned)blocks), dim3(256), 0, st, a, th)
#define MSA_NORM_OF(AA)                                                     \
  if (dm.d == 128) {                                                        \
    if (stream) MSA_NORM(128, true, AA); else MSA_NORM(128, false, AA);     \
  } else {                                                                  \
    if (stream) MSA_NORM(64, true, AA); else MSA_NORM(64, false, AA);       \
  }
  if (a.n_axes > 0) {
    MSA_NORM_OF(true)
  } else {
    MSA_NORM_OF(false)
  }
#undef MSA_NORM_OF
#undef MSA_NORM
  return hipGetLastError() == hipSuccess ? MSA_OK : MSA_ERR_HIP;
}

}  // namespace msa
