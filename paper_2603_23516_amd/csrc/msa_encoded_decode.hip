// Attention of single query tokens over position-encoded keys: msa_window_attend with few tokens, msa_sparse_attend4 where
// every token has documents of its own.  Each row is read once per (token, KV head) and serves the r query heads of the group.
//
// The rows that a (token, KV head) pair sees are numbered through, the bank's rows first (document by document, pads and rows
// past a document's end left out), then the local ones, in steps of 32; a workgroup has a contiguous range of steps, dealt to
// its four waves in turn.  Per step, with 16x16x32 bf16 MFMA:
//   S^T[key][col] = K q^T        A: lane (qd, n) holds dims of key row n; columns h and 8 + h both hold query head h
//   softmax over the keys, online, per column, in powers of two
//   O^T[dd][col] += V^T[dd][key] P^T[key][col]
//                                B: columns h hold the bf16 weights and columns 8 + h what they lack (weights of 16 bits at
//                                   no matrix work more: r <= 8 heads leave those columns empty)
//                                A: value rows go through LDS and come back transposed (ds_read_b64_tr_b16)
// Bank rows in four bits: lane (qd, n) takes the qd-th quarter of row n, 16 bytes at d = 128, and turns it into bf16 (exactly)
// by v_cvt_scalef32_pk_bf16_fp4, which applies the block's scale; the query's dims are laid out to match.
// The workgroup that arrives last at a pair merges its splits.
//
// Bound by HBM: 40 tokens that see 4100 rows of 8 heads of 128 (672 MB) 103 us, 6.5 TB/s; 40 tokens of 16 documents in four
// bits and 1800 rows in bf16 (474 MB) 75 us, 6.3 TB/s; 8 tokens of 32 documents (210 MB) 40 us, of which about 9 are the first
// loads and the joins.  One token of 64 dims over 32 + 256 rows 5.8: the loads that wait for one another.  Two waves to a SIMD
// (registers for two sets of loads); eight waves to a workgroup, a second set for local rows, sixteen
// parts at a time in the join and a launch of its own for it gave nothing or were slower.
#include "msa_encoded.h"

namespace msa {

__device__ __forceinline__ float max_xor16_32(float x) {
  uint32_t u = __float_as_uint(x);
  auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  x = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
  u = __float_as_uint(x);
  r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

constexpr int kLocalCost = 3;

template <int D>
struct Raw4 {  // a quarter of a row in four bits
  uint32_t w[D / 32];
};
template <int D>
__device__ __forceinline__ Raw4<D> load_raw4(const uint8_t* p) {
  Raw4<D> x;
  if constexpr (D == 128) {
    const uint4 v = *reinterpret_cast<const uint4*>(p);
    x.w[0] = v.x; x.w[1] = v.y; x.w[2] = v.z; x.w[3] = v.w;
  } else {
    const uint2 v = *reinterpret_cast<const uint2*>(p);
    x.w[0] = v.x; x.w[1] = v.y;
  }
  return x;
}

template <int D, bool BANK4>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2, 2))) void encoded_decode_kernel(EncodedArgs a) {
  constexpr int NS = D / 32;   // contraction slices of the score product, and 32-bit words of a quarter row's codes
  constexpr int NC = D / 16;   // 16-row tiles of the output product
  constexpr int ROW = D * 2;   // bytes of a value row in LDS
  constexpr int OROW = D + 4;  // floats of a row of a wave's output in the merge
  constexpr int STAGE = 32 * ROW > 8 * OROW * 4 ? 32 * ROW : 8 * OROW * 4;
  __shared__ __attribute__((aligned(16))) unsigned char stage[4][STAGE];
  __shared__ float wm[4][8], wl[4][8];
  __shared__ int pre[MSA_MAX_TOPK + 1];
  __shared__ long long base[MSA_MAX_TOPK];  // bank row of a slot's row i (numbered through) less i
  __shared__ uint32_t arrived;

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int qd = lane >> 4, n = lane & 15, h = n & 7;
  const int sp = blockIdx.x, g = blockIdx.y, bm = blockIdx.z, b = bm / a.M, r = a.r;
  const int q_pos = a.q_pos[bm];  // (asked for together with the queries and the selection: each is a microsecond away)
  // queries: column n holds head n % 8; B operand of slice s: dims 32 s + 8 qd .. + 8 (local rows), or the s-th eight dims of
  // the qd-th quarter (bank rows)
  bf16x8_t bq[NS], bq4[BANK4 ? NS : 1];
  {
    const uint16_t* qp = a.q + ((long long)bm * a.Hq + g * r + (h < r ? h : 0)) * D;
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      uint4 x = *reinterpret_cast<const uint4*>(qp + 32 * s + 8 * qd);
      if (h >= r) x = make_uint4(0, 0, 0, 0);
      bq[s] = as_bf16x8(x);
      if (BANK4) {
        x = *reinterpret_cast<const uint4*>(qp + (D / 4) * qd + 8 * s);
        if (h >= r) x = make_uint4(0, 0, 0, 0);
        bq4[s] = as_bf16x8(x);
      }
    }
  }

  const Seen see = seen_rows((long long)q_pos - a.pos0, a.Lloc, a.window, a.sinks);

  int rows_mem = 0;
  if (BANK4) {
    if (wave == 0) {
      int before;  // (from the register: pre[lane] is another lane's to write, and nothing waits for it here)
      const int doc = number_rows(a, b, bm, g, lane, pre, before);
      base[lane] = ((long long)doc * a.Hkv + g) * a.G - before;
    }
    lds_barrier();
    rows_mem = __builtin_amdgcn_readfirstlane(pre[MSA_MAX_TOPK]);
  }
  const int steps_mem = (rows_mem + 31) / 32, steps_a = (see.first + 31) / 32, steps_b = (see.to - see.from + 31) / 32;
  // A step of local rows is 16 KiB, one of bank rows 4.25 (d = 128): it counts as kLocalCost of those in the shares.
  const long long cost = steps_mem + (long long)kLocalCost * (steps_a + steps_b);
  auto share = [&](int i) {
    const int c = (int)(cost * i / a.n_splits);
    return c <= steps_mem ? c : steps_mem + (c - steps_mem) / kLocalCost;
  };
  const int s_begin = share(sp), s_end = share(sp + 1);

  unsigned long long* const ticket = a.tickets + (long long)bm * a.Hkv + g;
  if (a.n_splits > 1 && sp == 0 && tid == 192) expect_arrivals(ticket, a.nonce);  // (a wave that does not number the rows)

  // Value rows in LDS: 16-byte piece p of row i lies at place p ^ swz(i), so that neither the writes (16 rows, one piece) nor
  // the transposing reads (four rows, two pieces) meet in a bank.
  unsigned char* const vt = stage[wave];
  auto swz = [](int i) { return D == 128 ? 2 * (i & 7) : 2 * ((i >> 1) & 3); };
  auto put = [&](int i, int p, uint4 x) { *reinterpret_cast<uint4*>(vt + i * ROW + ((p ^ swz(i)) * 16)) = x; };

  float m_run = -INFINITY, l_run = 0.f;
  f32x4_t o[NC];
#pragma unroll
  for (int c = 0; c < NC; ++c) o[c] = (f32x4_t){0.f, 0.f, 0.f, 0.f};

  // scores of a step's 32 keys (of which `cnt` exist) -> weights, and the second product over the rows in LDS
  auto finish = [&](f32x4_t s0, f32x4_t s1, int cnt) __attribute__((always_inline)) {
    float x[8];
    float mx = -INFINITY;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int key = (i >> 2) * 16 + 4 * qd + (i & 3);
      x[i] = key < cnt ? (i < 4 ? s0[i & 3] : s1[i & 3]) * a.qscale : -INFINITY;
      mx = fmaxf(mx, x[i]);
    }
    mx = max_xor16_32(mx);
    // m_run is what the weights are taken relative to, not the maximum itself: it follows once that is 2^8 ahead
    if (__ballot(mx > m_run + 8.f) != 0) {
      const float m_new = fmaxf(m_run, mx);
      const float alpha = m_run == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m_run - m_new);
      m_run = m_new;
      l_run *= alpha;
#pragma unroll
      for (int c = 0; c < NC; ++c) o[c] *= alpha;
    }
    const float m_use = m_run == -INFINITY ? 0.f : m_run;
    uint32_t pw[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float p0 = __builtin_amdgcn_exp2f(x[2 * j] - m_use), p1 = __builtin_amdgcn_exp2f(x[2 * j + 1] - m_use);
      l_run += p0 + p1;
      uint32_t hi, lo;
      split_pack_bf16(p0, p1, hi, lo);
      pw[j] = n < 8 ? hi : lo;
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
      o[c] = mfma16(av, pb, o[c]);
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  };

  int s = s_begin + wave;
  if (BANK4) {
    // The wave's steps of bank rows, two in flight: a set of registers is filled again as soon as its codes have been turned
    // into operands.  Loads have no condition (the wait for the older set would have to be one for everything): behind the
    // last step they repeat it, out of the caches.
    struct Set {
      Raw4<D> k[2], v[2];
      uint32_t ks[2], vs[2];
    } sets[2];
    const int s_stop = s_end < steps_mem ? s_end : steps_mem;
    int slot[2] = {0, 0}, row[2], last[2];  // last: rows in front of the next slot
    long long at[2];                        // bank row
    int s_load = s;                         // the step that the next load brings
    auto find = [&](int t) __attribute__((always_inline)) {
      const int rc = row[t] < rows_mem ? row[t] : rows_mem - 1;
      while (rc >= pre[slot[t] + 1]) ++slot[t];  // ends: rc < pre[k]
      last[t] = pre[slot[t] + 1];
      at[t] = base[slot[t]] + rc;
    };
    auto load = [&](Set& x) __attribute__((always_inline)) {
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const long long c = at[t] * (D / 2) + (D / 8) * qd, e = at[t] * (D / 32) + (D == 128 ? qd : qd >> 1);
        x.k[t] = load_raw4<D>(a.K4 + c);
        x.v[t] = load_raw4<D>(a.V4 + c);
        x.ks[t] = a.K4s[e];
        x.vs[t] = a.V4s[e];
      }
      if (s_load + 4 < s_stop) {
        s_load += 4;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          row[t] += 128;
          at[t] += 128;
          if (row[t] >= last[t]) find(t);
        }
      }
    };
    auto turn = [&](Set& x) __attribute__((always_inline)) {
      f32x4_t sc[2];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        sc[t] = (f32x4_t){0.f, 0.f, 0.f, 0.f};
        const float ks = __uint_as_float(x.ks[t] << 23), vs = __uint_as_float(x.vs[t] << 23);
#pragma unroll
        for (int j = 0; j < NS; ++j) {
          sc[t] = mfma16(as_bf16x8(fp4x8_to_bf16(x.k[t].w[j], ks)), bq4[j], sc[t]);
          put(16 * t + n, NS * qd + j, fp4x8_to_bf16(x.v[t].w[j], vs));
        }
      }
      load(x);
      finish(sc[0], sc[1], rows_mem - 32 * s < 32 ? rows_mem - 32 * s : 32);
      s += 4;
    };
    if (s < s_stop) {
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        row[t] = 32 * s + 16 * t + n;
        find(t);
      }
      load(sets[0]);
      load(sets[1]);
      while (s + 4 < s_stop) {  // (in pairs, without a way out between them: the count of loads in flight stays known)
        turn(sets[0]);
        turn(sets[1]);
      }
      if (s < s_stop) turn(sets[0]);
    }
  }
  const long long loc = ((long long)b * a.Hkv + g) * a.Lloc;
  if (s < s_end) {
    uint4 kx[2][NS], vx[2][NS];
    int cnt = 0, t0 = 0, end = 0;
    auto place = [&](int st) __attribute__((always_inline)) {
      const int j0 = st - steps_mem;
      t0 = 32 * j0;
      end = see.first;
      if (j0 >= steps_a) {
        t0 += see.from - 32 * steps_a;
        end = see.to;
      }
    };
    auto load = [&]() __attribute__((always_inline)) {
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        int row = t0 + 16 * t + n;
        row = row < end ? row : end - 1;
        const uint16_t* kp = a.Kloc + (loc + row) * D + 8 * qd;
        const uint16_t* vp = a.Vloc + (loc + row) * D + 8 * qd;
#pragma unroll
        for (int j = 0; j < NS; ++j) {
          kx[t][j] = *reinterpret_cast<const uint4*>(kp + 32 * j);
          vx[t][j] = *reinterpret_cast<const uint4*>(vp + 32 * j);
        }
      }
    };
    place(s);
    load();
    for (; s < s_end; s += 4) {
      f32x4_t sc[2];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        sc[t] = (f32x4_t){0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < NS; ++j) {
          sc[t] = mfma16(as_bf16x8(kx[t][j]), bq[j], sc[t]);
          put(16 * t + n, 4 * j + qd, vx[t][j]);
        }
      }
      cnt = end - t0 < 32 ? end - t0 : 32;
      if (s + 4 < s_end) {
        place(s + 4);
        load();  // under way while this step's weights are worked out
      }
      finish(sc[0], sc[1], cnt);
    }
  }

  // ---- the four waves' results, then the splits' --------------------------------------------------------------
  l_run = add_xor32(add_xor16(l_run));
#pragma unroll
  for (int c = 0; c < NC; ++c)
#pragma unroll
    for (int i = 0; i < 4; ++i) o[c][i] += dpp_f<kDppRor8>(o[c][i]);  // columns h and 8 + h
  float* const mine = reinterpret_cast<float*>(stage[wave]);
  if (n < r) {
#pragma unroll
    for (int c = 0; c < NC; ++c) *reinterpret_cast<f32x4_t*>(mine + n * OROW + 16 * c + 4 * qd) = o[c];
    if (qd == 0) {
      wm[wave][n] = m_run;
      wl[wave][n] = l_run;
    }
  }
  __syncthreads();
  const long long qh0 = (long long)bm * a.Hq + g * r;
  for (int e = tid; e < r * D; e += 256) {
    const int hh = e / D, dd = e % D;
    float m = wm[0][hh];
#pragma unroll
    for (int w = 1; w < 4; ++w) m = fmaxf(m, wm[w][hh]);
    float l = 0.f, x = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float f = wm[w][hh] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(wm[w][hh] - m);
      l += f * wl[w][hh];
      x += f * reinterpret_cast<const float*>(stage[w])[hh * OROW + dd];
    }
    if (a.n_splits == 1) {
      a.out[(qh0 + hh) * D + dd] = (uint16_t)pack_bf16(l > 0.f ? x / l : 0.f, 0.f);
      if (dd == 0 && a.lse != nullptr) a.lse[qh0 + hh] = l > 0.f ? (m + log2f(l)) * 0.6931471805599453f : -INFINITY;
    } else {
      const long long ph = (qh0 + hh) * a.n_splits + sp;
      store_dev(a.part_o + ph * D + dd, x);
      if (dd == 0)
        store_dev(reinterpret_cast<unsigned long long*>(a.part_ml + ph),
                  ((unsigned long long)__float_as_uint(l) << 32) | __float_as_uint(m));
    }
  }
  if (a.n_splits == 1) return;
  wait_stores_done();
  __syncthreads();
  if (tid == 0) arrived = arrive_at(ticket, a.nonce);
  __syncthreads();
  if (arrived != (uint32_t)a.n_splits - 1) return;
  if (tid == 0) store_dev(ticket, 0ull);
  // All (max, sum) pairs at once, then the outputs eight splits at a time: loads past the L2 take over a microsecond, and one
  // after another for 16 splits they were a third of a call of 92 us.
  float2* const parts = reinterpret_cast<float2*>(stage[0]);  // [r][n_splits], 256 at most
  for (int e = tid; e < r * a.n_splits; e += 256) {
    const unsigned long long ml = load_dev(reinterpret_cast<const unsigned long long*>(a.part_ml + qh0 * a.n_splits + e));
    parts[e] = make_float2(__uint_as_float((uint32_t)ml), __uint_as_float((uint32_t)(ml >> 32)));
  }
  __syncthreads();
  for (int e = 2 * tid; e < r * D; e += 512) {
    const int hh = e / D, dd = e % D;
    const float2* const ml = parts + hh * a.n_splits;
    float m = -INFINITY, l = 0.f, x0 = 0.f, x1 = 0.f;
    for (int i = 0; i < a.n_splits; ++i) m = fmaxf(m, ml[i].x);
    const float* const po = a.part_o + (qh0 + hh) * a.n_splits * D + dd;
    for (int i0 = 0; i0 < a.n_splits; i0 += 8) {
      unsigned long long v[8];
#pragma unroll
      for (int u = 0; u < 8; ++u)
        v[u] = load_dev(reinterpret_cast<const unsigned long long*>(po + (i0 + u < a.n_splits ? i0 + u : a.n_splits - 1) * D));
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        float f = 0.f;
        if (i0 + u < a.n_splits && ml[i0 + u].x != -INFINITY) f = __builtin_amdgcn_exp2f(ml[i0 + u].x - m);
        if (i0 + u < a.n_splits) l += f * ml[i0 + u].y;
        x0 += f * __uint_as_float((uint32_t)v[u]);
        x1 += f * __uint_as_float((uint32_t)(v[u] >> 32));
      }
    }
    const float inv = l > 0.f ? 1.f / l : 0.f;
    *reinterpret_cast<uint32_t*>(a.out + (qh0 + hh) * D + dd) = pack_bf16(x0 * inv, x1 * inv);
    if (dd == 0 && a.lse != nullptr) a.lse[qh0 + hh] = l > 0.f ? (m + log2f(l)) * 0.6931471805599453f : -INFINITY;
  }
}

static EncodedPlan plan_of(const Dims& dm, int B, int M, long long mem_rows, bool shared, long long local_rows, int Lloc,
                           bool expand) {
  EncodedPlan p = {};
  const long long pairs = (long long)B * M * dm.Hkv;
  // Tokens that share their rows go through the tiled kernel where the single-token kernel would take long over them: its steps
  // of all tokens (`work`; local ones count kLocalCost) against what the tiled kernel's launches, its thin tiles and the
  // documents' expansion cost.  us in a graph, tiled / one by one, M tokens; 8 KV heads of 128, r = 4, if nothing else is said:
  //   a window of 2048                               M = 8 17 / 14, 12 18 / 19, 16 18 / 21, 24 19 / 35
  //   2 sequences, 4096                              M = 3 24 / 20, 4 24 / 22, 6 24 / 30, 8 24 / 35
  //   8 sequences, 4096                              M = 2 48 / 39, 3 49 / 66, 4 50 / 65, 6 39 / 97, 8 40 / 118
  //   32768                                          M = 2 54 / 38, 3 57 / 58, 4 57 / 68
  //   4 sequences, 512, 4 KV heads, r = 8            M = 16 16 / 12, 24 16 / 19
  //   2048, 64 dims, r = 1                           M = 12 14 / 12, 16 14 / 13, 24 14 / 20
  //   16 documents of 512, 512 local rows            M = 12 37 / 29, 16 38 / 34, 24 39 / 53
  //   8 sequences, 16 documents of 512, 2048 local   M = 6 145 / 116, 8 145 / 130, 12 148 / 210
  //   3 sequences, 8 documents of 64, 512 local      M = 8 21 / 17, 12 22 / 25, 16 22 / 25
  //   8 sequences, 32 documents of 8, 2048 local     M = 6 31 / 66, 8 31 / 66, 16 35 / 129
  // The border is off by up to an eighth on its tiled side and a fifth on the other; 3 tokens of many sequences, and 3 to 7 tokens
  // with few documents beside a long context, go one by one though tiles would take half to four fifths of the time.
  // (More rows never lead back to the single-token kernel: both sides count them in whole steps, M of them on the left and 8 on
  // the right, which applies from M = 8 on.)
  const long long steps_mem = (mem_rows + 31) / 32, cost = steps_mem + kLocalCost * ((local_rows + 31) / 32);
  const double work = (double)pairs * cost, least = 20000 + (double)(8 * pairs / M) * steps_mem;  // (past 64 bits at the largest sizes)
  p.tiled = !expand || ((mem_rows == 0 || shared) && (M >= 32 || (M >= (mem_rows > 0 ? 8 : 4) && work >= least))) ? 1 : 0;
  int n_most;  // splits that the workspace holds: grows with the rows, so that one sized for the longest call serves all
  long long most1 = (cost + 15) / 16;
  if (most1 > 2048 / pairs) most1 = 2048 / pairs;
  const int single_most = (int)(most1 < 1 ? 1 : (most1 > 32 ? 32 : most1));
  if (p.tiled) {
    // 128 columns to a workgroup.  With one, two or three on every CU a step takes 0.80, 0.95 or 1.32 us (d = 64: 0.48, 0.56,
    // 0.76), a workgroup 6 beside its steps.  Two parts are joined by the last workgroup, 7 us (d = 64: 4);
    // more by a launch, 4 us and 0.25 + 0.05 n for every 1000 of the (token, head) rows, and n rows of d floats
    // at 5 TB/s.  (1000 tokens over 8192 and 1000 rows, 8 heads: n = 1 245 us, 2 161, 3 166, 4 171, 8 183; 128 tokens over
    // 4096: 95, 54, 41, 35, n = 8 28, 16 29; 4 times 509 tokens of 64 dims over 1000 rows: 26, 24, 37, 39.)
    p.tpw = 32 / dm.r;
    p.n_tiles = (M + 4 * p.tpw - 1) / (4 * p.tpw);
    const long long tiles = (long long)B * p.n_tiles * dm.Hkv, heads = (long long)B * M * dm.Hq;
    if (tiles >= 1 << 24) return p;  // (parts: 1024 workgroups in all at most)
    const long long seen = local_rows + 4 * p.tpw;
    const long long all_steps = (mem_rows + 31) / 32 + ((seen < Lloc ? seen : Lloc) + 31) / 32;
    long long most = all_steps / 4;
    if (most > 1024 / tiles) most = 1024 / tiles;
    n_most = (int)(most < 1 ? 1 : (most > 32 ? 32 : most));
    const int ns_per_step[2][3] = {{480, 560, 760}, {800, 950, 1320}};
    long long best = -1;
    for (int n = 1; n <= n_most; ++n) {
      const long long all = tiles * n, steps = (all_steps + n - 1) / n;
      const long long per_cu = (all + 255) / 256 < 3 ? (all + 255) / 256 : 3;
      long long t = steps * ns_per_step[dm.d == 128][per_cu - 1];
      if (all > 768) t = t * all / 768;
      t += 6000;
      if (n == 2)
        t += dm.d == 128 ? 7000 : 4000;
      else if (n > 2)
        t += 4000 + heads * (250 + 50 * n) / 1000 + heads * n * dm.d * 4 / 5000;
      if (best < 0 || t < best) {
        best = t;
        p.n_splits = n;
      }
    }
  } else {
    // Two workgroups fit a CU.  A workgroup takes about 9 us beside its steps (three loads that wait for one another, then
    // the joining of four waves), its steps 0.7 us each where it has a CU to itself and 1.2 beside another, and the join of
    // n parts 3 us and 0.3 for each (8 heads, 8 streams, 512 steps of bank rows and 64 local ones: n = 2 76 us, 4 45,
    // 8 41, 12 46, 16 49; 32 streams, 8 and 32 steps: n = 2 29 us, 4 35, 8 52, 16 93; one stream, 256 local steps: n = 4 34, 8
    // 21, 12 17, 16 15.2, 24 14.4, 32 15.8).
    if ((long long)B * M > 65535) return p;
    n_most = single_most;
    long long best = -1;
    for (int n = 1; n <= n_most; ++n) {
      const long long all = pairs * n, steps = (cost + 4 * n - 1) / (4 * n);
      const long long t = (all + 511) / 512 * (90 + (all <= 256 ? 7 : 12) * steps) + (n > 1 ? 30 + 3 * n : 0);
      if (best < 0 || t < best) {
        best = t;
        p.n_splits = n;
      }
    }
  }
  const size_t rows = (size_t)B * M * dm.Hq;
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t here = at;
    at += round_up256(bytes);
    return here;
  };
  auto take_parts = [&](int n, size_t of, size_t floats, size_t sums, size_t counters) {  // n parts of `of`, and the counters
    if (n < 2) return;
    take(of * n * floats * sizeof(float));
    p.off_ml = take(of * n * sums * sizeof(float2));
    p.off_tickets = take(counters * sizeof(unsigned long long));
  };
  size_t single = 0;
  if (p.tiled && expand && M < 32) {  // what a shorter call, which takes its tokens one by one, asks for
    take_parts(single_most, rows, dm.d, 1, (size_t)pairs);
    single = at;
    at = 0;
  }
  if (p.tiled) {
    const size_t tiles = (size_t)B * p.n_tiles * dm.Hkv;
    take_parts(n_most, tiles, 128 * (size_t)dm.d, 256, tiles);  // (no fewer than by rows)
  } else {
    take_parts(n_most, rows, dm.d, 1, (size_t)pairs);
  }
  if (p.tiled && mem_rows > 0 && expand) {
    const size_t x = (size_t)B * dm.Hkv * mem_rows * dm.d * 2;
    p.off_kx = take(x);
    p.off_vx = take(x);
    p.off_mem_rows = take((size_t)B * dm.Hkv * sizeof(int));
  }
  if (at < single) at = single;
  p.ws_bytes = at > 256 ? at : 256;
  return p;
}

EncodedPlan plan_encoded(const Dims& dm, int B, int M, long long mem_rows, bool shared, long long local_rows, int Lloc) {
  return plan_of(dm, B, M, mem_rows, shared, local_rows, Lloc, true);
}
EncodedPlan plan_encoded_prefix(const Dims& dm, int B, int M, long long mem_rows, int Lloc) {
  return plan_of(dm, B, M, mem_rows, true, Lloc, Lloc, false);
}

int launch_encoded(const Dims& dm, const EncodedPlan& pl, EncodedArgs a, int B, void* ws, hipStream_t st) {
  unsigned char* const w = (unsigned char*)ws;
  a.Hq = dm.Hq;
  a.Hkv = dm.Hkv;
  a.r = dm.r;
  a.G = dm.G;
  a.N = dm.N;
  a.idx_sel = dm.scope_all ? 1 : dm.Hkv;
  a.idx_rows_per_b = dm.token_pool ? 1 : a.M;
  a.lens = dm.lens;
  a.qscale = (float)(1.4426950408889634 / sqrt((double)dm.d));
  a.n_splits = pl.n_splits;
  a.part_o = (float*)w;
  a.part_ml = (float2*)(w + pl.off_ml);
  if (!pl.tiled || pl.n_splits == 2) a.tickets = (unsigned long long*)(w + pl.off_tickets);
  a.nonce = launch_nonce48();
  if (pl.tiled) {
    TiledArgs ta = {};
    ta.tpw = pl.tpw;
    ta.n_tiles = pl.n_tiles;
    if (a.K4 != nullptr) {
      ta.Kx = (uint16_t*)(w + pl.off_kx);
      ta.Vx = (uint16_t*)(w + pl.off_vx);
      ta.mem_rows = (int*)(w + pl.off_mem_rows);
      ta.mem_cap = a.k * dm.G;
    }
    return launch_encoded_tiled(dm, a, ta, B, st);
  }
  const dim3 grid(a.n_splits, dm.Hkv, B * a.M), block(256);
  if (dm.d == 128) {
    if (a.K4 != nullptr) hipLaunchKernelGGL((encoded_decode_kernel<128, true>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((encoded_decode_kernel<128, false>), grid, block, 0, st, a);
  } else {
    if (a.K4 != nullptr) hipLaunchKernelGGL((encoded_decode_kernel<64, true>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((encoded_decode_kernel<64, false>), grid, block, 0, st, a);
  }
  return hipGetLastError() == hipSuccess ? MSA_OK : MSA_ERR_HIP;
}

}  // namespace msa
