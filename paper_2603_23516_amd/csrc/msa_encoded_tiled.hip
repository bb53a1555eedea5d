// Attention of many query tokens that share position-encoded keys: msa_window_attend over a prompt or a chunk of one,
// msa_sparse_attend4 where the tokens of a sequence share their documents (token_pool = 1).  Bound by the matrix cores.
//
// A workgroup owns a tile of tokens of one (sequence, KV head); its columns are the (token, query head) pairs, 32 to a column
// block, CB blocks to a wave.  The rows any token of the tile sees go by in steps of 32: rows of the documents (expanded to
// bf16 once per call, expand4_kernel), the first rows of the cache, the window's.  Per step:
//   copies    32 key and 32 value rows go global -> LDS asynchronously, two steps ahead of their use (four stages), their
//             16-byte pieces placed so that the reads below meet no bank twice
//   scores    S^T[32 keys][32 cols] = K q^T with v_mfma_f32_32x32x16_bf16; the queries stay in registers
//   softmax   online, per column (16 keys in a lane, the other 16 in lane ^ 32)
//   product   O^T[dd][col] += V^T[dd][key] P^T[key][col], the weights in bf16 (an element of the output is off by
//             what 2^-9 of every weight comes to; their sum is taken before the rounding), V^T by transposing LDS reads
// Masks are worked out only in steps that some column of the wave does not see whole; steps that a wave does not see at all
// are passed over.
#include "msa_encoded.h"

namespace msa {

typedef float f32x16e_t __attribute__((ext_vector_type(16)));

__device__ __forceinline__ f32x16e_t mfma32e(bf16x8_t a, bf16x8_t b, f32x16e_t c) {
  // D(32x32) += A(32x16) * B(16x32).  Lane l: A[l%32][8(l/32)..+8], B[8(l/32)..+8][l%32],
  // D register i: row (i%4) + 8(i/4) + 4(l/32), column l%32.
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ float max_xor32(float x) {
  const uint32_t u = __float_as_uint(x);
  const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// ---- the selected documents of every (sequence, KV head), in bf16, one after another ---------------------------------------
template <int D>
__global__ __launch_bounds__(256) void expand4_kernel(EncodedArgs a, uint16_t* __restrict__ Kx, uint16_t* __restrict__ Vx,
                                                      int* __restrict__ mem_rows, int mem_cap) {
  constexpr int LPR = D / 8, RPB = 256 / LPR;
  __shared__ int pre[MSA_MAX_TOPK + 1], docs[MSA_MAX_TOPK];
  const int tid = threadIdx.x, g = blockIdx.y, b = blockIdx.z;
  if (tid < 64) number_rows(a, b, b, g, tid, pre, docs);
  __syncthreads();
  const int rows = pre[MSA_MAX_TOPK];
  const long long pair = (long long)b * a.Hkv + g;
  if (blockIdx.x == 0 && tid == 0) mem_rows[pair] = rows;
  const int lr = tid % LPR;
  for (int row = blockIdx.x * RPB + tid / LPR; row < rows; row += gridDim.x * RPB) {
    int slot = 0;
#pragma unroll
    for (int s = 32; s > 0; s /= 2)
      if (row >= pre[slot + s]) slot += s;  // the last slot whose rows begin at or before this one
    const long long at = ((long long)docs[slot] * a.Hkv + g) * a.G + (row - pre[slot]);
    const long long to = (pair * mem_cap + row) * D + 8 * lr;
    const uint32_t kc = *reinterpret_cast<const uint32_t*>(a.K4 + at * (D / 2) + 4 * lr);
    const uint32_t vc = *reinterpret_cast<const uint32_t*>(a.V4 + at * (D / 2) + 4 * lr);
    const float ks = __uint_as_float((uint32_t)a.K4s[at * (D / 32) + lr / 4] << 23);
    const float vs = __uint_as_float((uint32_t)a.V4s[at * (D / 32) + lr / 4] << 23);
    *reinterpret_cast<uint4*>(Kx + to) = fp4x8_to_bf16(kc, ks);
    *reinterpret_cast<uint4*>(Vx + to) = fp4x8_to_bf16(vc, vs);
  }
}

// ---- the tiled kernel -------------------------------------------------------------------------------------------------
template <int D, int CB, int NW>
__global__ __launch_bounds__(NW * 64) __attribute__((amdgpu_waves_per_eu(CB == 2 ? 1 : 2)))
void encoded_tiled_kernel(EncodedArgs a, TiledArgs ta) {
  constexpr int NP = D / 8;      // 16-byte pieces per row
  constexpr int NS = D / 16;     // contraction slices of the score product
  constexpr int NT = D / 32;     // 32-row tiles of the output product
  constexpr int ROW = D * 2;
  constexpr int TILE = 32 * ROW;  // bytes of 32 key or value rows
  constexpr int NBUF = 4;
  constexpr int NI = 32 * NP / 64;     // wave-wide copies for 32 rows
  constexpr int NPW = 2 * NI / NW;     // copies of a wave per step, keys and values together
  static_assert(NPW >= 1 && NPW * NW == 2 * NI, "a step is a whole number of copies per wave");
  __shared__ __attribute__((aligned(16))) unsigned char smem[NBUF * 2 * TILE];
  __shared__ int pmin_s[NW], pmax_s[NW];

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int hf = lane >> 5, col = lane & 31, r = a.r;
  // (tile, split, KV head): the KV head fastest, so that an XCD (every eighth workgroup) keeps to few heads' rows; late tiles,
  // which see most, first
  int x = blockIdx.x;
  const int g = x % a.Hkv;
  x /= a.Hkv;
  const int sp = x % a.n_splits;
  x /= a.n_splits;
  const int b = x / ta.n_tiles, tile = ta.n_tiles - 1 - x % ta.n_tiles;
  const int m_wave = (tile * NW + wave) * ta.tpw;  // first token of the wave

  // this lane's columns: token and head of each, and the rows it sees: t <= p and (t >= lo or t < sinks)
  int p[CB], lo[CB], tok[CB], head[CB];
  bool ok[CB];
  int pmin = INT32_MAX, pmax = -1;
#pragma unroll
  for (int c = 0; c < CB; ++c) {
    const int cc = 32 * c + col;
    const int tl = cc / r;
    head[c] = cc - tl * r;
    tok[c] = m_wave + tl;
    ok[c] = tl < ta.tpw && tok[c] < a.M;
    long long pc = -1;
    if (ok[c]) {
      pc = (long long)a.q_pos[(long long)b * a.M + tok[c]] - a.pos0;
      pc = pc < -1 ? -1 : pc;
      pmin = (int)pc < pmin ? (int)pc : pmin;
      pmax = (int)pc > pmax ? (int)pc : pmax;
    }
    p[c] = (int)pc;
    lo[c] = (int)(pc - a.window + 1);
  }
  int plow = pmin;  // the lowest position of a token that sees anything
#pragma unroll
  for (int c = 0; c < CB; ++c) plow = c == 0 ? (ok[0] && p[0] >= 0 ? p[0] : INT32_MAX) : (ok[c] && p[c] >= 0 && p[c] < plow ? p[c] : plow);
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) {
    const int u = __shfl_xor(pmin, off, 64), v = __shfl_xor(pmax, off, 64), w = __shfl_xor(plow, off, 64);
    pmin = u < pmin ? u : pmin;
    pmax = v > pmax ? v : pmax;
    plow = w < plow ? w : plow;
  }
  const int pmin_w = __builtin_amdgcn_readfirstlane(pmin), pmax_w = __builtin_amdgcn_readfirstlane(pmax);
  const int plow_w = __builtin_amdgcn_readfirstlane(plow);
  if (lane == 0) {
    pmin_s[wave] = plow_w;
    pmax_s[wave] = pmax_w;
  }
  __syncthreads();
  int plow_t = pmin_s[0], pmax_t = pmax_s[0];
#pragma unroll
  for (int w = 1; w < NW; ++w) {
    plow_t = pmin_s[w] < plow_t ? pmin_s[w] : plow_t;
    pmax_t = pmax_s[w] > pmax_t ? pmax_s[w] : pmax_t;
  }
  plow_t = __builtin_amdgcn_readfirstlane(plow_t);
  pmax_t = __builtin_amdgcn_readfirstlane(pmax_t);
  // rows of the cache that the tile goes through: [0, first) and [from, to)
  Seen see = {0, 0, 0};
  if (pmax_t >= 0) {
    see = seen_rows(plow_t, a.Lloc, a.window, a.sinks);
    see.to = pmax_t + 1LL < a.Lloc ? pmax_t + 1 : a.Lloc;
    if (see.from > see.to) see.from = see.to;
  }
  const long long pair = (long long)b * a.Hkv + g;
  const int rows_mem = ta.Kx != nullptr ? __builtin_amdgcn_readfirstlane(ta.mem_rows[pair]) : 0;
  const int steps_mem = (rows_mem + 31) / 32, steps_a = (see.first + 31) / 32, steps_b = (see.to - see.from + 31) / 32;
  const int steps = steps_mem + steps_a + steps_b;
  const int sb = (int)((long long)steps * sp / a.n_splits), se = (int)((long long)steps * (sp + 1) / a.n_splits);
  const uint16_t* const kmem = ta.Kx != nullptr ? ta.Kx + pair * ta.mem_cap * D : nullptr;
  const uint16_t* const vmem = ta.Kx != nullptr ? ta.Vx + pair * ta.mem_cap * D : nullptr;
  const uint16_t* const kloc = a.Kloc + pair * a.Lloc * D;
  const uint16_t* const vloc = a.Vloc + pair * a.Lloc * D;

  // queries: B operand of slice s: dims 16 s + 8 hf .. + 8 of the column's head
  bf16x8_t bq[CB][NS];
#pragma unroll
  for (int c = 0; c < CB; ++c) {
    const uint16_t* qp = a.q + (((long long)b * a.M + (ok[c] ? tok[c] : 0)) * a.Hq + g * r + (ok[c] ? head[c] : 0)) * D + 8 * hf;
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      uint4 v = *reinterpret_cast<const uint4*>(qp + 16 * s);
      if (!ok[c]) v = make_uint4(0, 0, 0, 0);
      bq[c][s] = as_bf16x8(v);
    }
  }

  // places of the 16-byte pieces of a row in LDS
  auto swz_k = [](int i) { return D == 128 ? (i & 15) : ((i >> 1) & 7); };
  auto swz_v = [](int i) { return D == 128 ? 4 * (i & 3) : 4 * ((i >> 1) & 1); };

  auto step_rows = [&](int s, int& t0, int& cnt, bool& mem) __attribute__((always_inline)) {
    mem = s < steps_mem;
    const int j = s - steps_mem;
    t0 = mem ? 32 * s : (j < steps_a ? 32 * j : see.from + 32 * (j - steps_a));
    const int end = mem ? rows_mem : (j < steps_a ? see.first : see.to);
    cnt = end - t0 < 32 ? end - t0 : 32;
  };
  auto issue = [&](int s, int into) __attribute__((always_inline)) {
    int t0, cnt;
    bool mem;
    step_rows(s, t0, cnt, mem);
    const uint16_t* const kb = (mem ? kmem : kloc) + (long long)t0 * D;
    const uint16_t* const vb = (mem ? vmem : vloc) + (long long)t0 * D;
#pragma unroll
    for (int i = 0; i < NPW; ++i) {
      const int j = i * NW + wave;  // wave-uniform: copy j of keys, or j - NI of values
      const int y = (j < NI ? j : j - NI) * 64 + lane;
      const int row = y / NP, at = y % NP;
      const int piece = at ^ (j < NI ? swz_k(row) : swz_v(row));
      const int src = row < cnt ? row : cnt - 1;
      copy16_to_lds_async(j < NI ? kb : vb, src * ROW + piece * 16, smem + into * 2 * TILE + j * 1024);
    }
  };

  const int j16 = lane & 15, q16 = (lane >> 4) & 1;
  const int vrow = 4 * hf + (j16 >> 2);
  auto scores = [&](int stage, f32x16e_t (&acc)[CB]) __attribute__((always_inline)) {
#pragma unroll
    for (int c = 0; c < CB; ++c)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[c][i] = 0.f;
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      const bf16x8_t ak = as_bf16x8(*reinterpret_cast<const uint4*>(
          smem + stage * 2 * TILE + col * ROW + (((2 * s + hf) ^ swz_k(col)) * 16)));
#pragma unroll
      for (int c = 0; c < CB; ++c) acc[c] = mfma32e(ak, bq[c][s], acc[c]);
    }
  };

  float m_run[CB], l_run[CB];
  f32x16e_t o[CB][NT];
#pragma unroll
  for (int c = 0; c < CB; ++c) {
    m_run[c] = -INFINITY;
    l_run[c] = 0.f;
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[c][t][i] = 0.f;
  }

  if (sb < se) issue(sb, 0);
  if (sb + 1 < se) issue(sb + 1, 1);
  for (int s = sb; s < se; ++s) {
    const int buf = (s - sb) & 3;
    if (s + 1 < se)
      wait_copies_but<NPW>();
    else
      wait_copies_but<0>();
    __builtin_amdgcn_s_barrier();  // step s is staged for everyone; everyone is done with step s - 2's stage
    asm volatile("" ::: "memory");
    if (s + 2 < se) issue(s + 2, (buf + 2) & 3);
    int t0, cnt;
    bool mem;
    step_rows(s, t0, cnt, mem);
    // what this wave sees of the step (uniform)
    const bool any = mem || (t0 <= pmax_w && ((long long)t0 + 31 >= (long long)plow_w - a.window + 1 || t0 < a.sinks));
    if (!any) continue;
    const bool whole = cnt == 32 && (mem || (t0 + 31 <= pmin_w && (t0 >= (long long)pmax_w - a.window + 1 || t0 + 31 < a.sinks)));
    f32x16e_t sc[CB];
    scores(buf, sc);
    bf16x8_t pb[CB][2];
#pragma unroll
    for (int c = 0; c < CB; ++c) {
      float xs[16];
      float mx = -INFINITY;
#pragma unroll
      for (int i = 0; i < 16; ++i) xs[i] = sc[c][i];
      if (!whole) {  // keys most .. least of the step are seen, and those in front of `few` (no branches: one compare each)
        const int seen = mem ? 31 : p[c] - t0;
        const int most = (seen < cnt - 1 ? seen : cnt - 1) - 4 * hf;
        const int least = (mem ? 0 : lo[c] - t0) - 4 * hf, few = (mem ? 0 : a.sinks - t0) - 4 * hf;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int key = (i & 3) + 8 * (i >> 2);
          const bool live = (key <= most) & ((key >= least) | (key < few));
          xs[i] = live ? xs[i] : -INFINITY;
        }
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) mx = fmaxf(mx, xs[i]);
      mx = max_xor32(mx) * a.qscale;
      if (__ballot(mx > m_run[c]) != 0) {
        const float m_new = fmaxf(m_run[c], mx);
        const float alpha = m_run[c] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m_run[c] - m_new);
        m_run[c] = m_new;
        l_run[c] *= alpha;
#pragma unroll
        for (int t = 0; t < NT; ++t) o[c][t] *= alpha;
      }
      const float m_use = m_run[c] == -INFINITY ? 0.f : m_run[c];
      uint32_t pw[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float p0 = __builtin_amdgcn_exp2f(fmaf(xs[2 * i], a.qscale, -m_use));
        const float p1 = __builtin_amdgcn_exp2f(fmaf(xs[2 * i + 1], a.qscale, -m_use));
        l_run[c] += p0 + p1;
        pw[i] = pack_bf16(p0, p1);
      }
      pb[c][0] = as_bf16x8(make_uint4(pw[0], pw[1], pw[2], pw[3]));
      pb[c][1] = as_bf16x8(make_uint4(pw[4], pw[5], pw[6], pw[7]));
    }
    // contraction slot j of slice sg and half hf is key 16 sg + (j % 4) + 8 (j / 4) + 4 hf: the lane's own registers
#pragma unroll
    for (int sg = 0; sg < 2; ++sg)
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        const int row = 16 * sg + vrow;  // the second read's row is 8 on, with the same places
        const unsigned char* vp = smem + buf * 2 * TILE + TILE + row * ROW +
                                  (((4 * t + 2 * q16 + ((j16 & 3) >> 1)) ^ swz_v(row)) * 16) + 8 * (j16 & 1);
        const s16x4_t v0 = lds_read_tr16(vp), v1 = lds_read_tr16(vp + 8 * ROW);
        const bf16x8_t av = __builtin_bit_cast(bf16x8_t, __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
        for (int c = 0; c < CB; ++c) o[c][t] = mfma32e(av, pb[c][sg], o[c][t]);
      }
  }

#pragma unroll
  for (int c = 0; c < CB; ++c) {
    const uint32_t u = __float_as_uint(l_run[c]);
    const auto both = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    const float l = __uint_as_float(both[0]) + __uint_as_float(both[1]);
    if (!ok[c]) continue;
    const long long qh = ((long long)b * a.M + tok[c]) * a.Hq + g * r + head[c];
    if (a.n_splits == 1) {
      const float inv = l > 0.f ? 1.f / l : 0.f;
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          *reinterpret_cast<uint2*>(a.out + qh * D + 32 * t + 8 * i + 4 * hf) =
              make_uint2(pack_bf16(o[c][t][4 * i] * inv, o[c][t][4 * i + 1] * inv),
                         pack_bf16(o[c][t][4 * i + 2] * inv, o[c][t][4 * i + 3] * inv));
      if (hf == 0 && a.lse != nullptr)
        a.lse[qh] = l > 0.f ? (m_run[c] + log2f(l)) * 0.6931471805599453f : -INFINITY;
    } else {
      const long long ph = qh * a.n_splits + sp;
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          *reinterpret_cast<f32x4_t*>(a.part_o + ph * D + 32 * t + 8 * i + 4 * hf) =
              (f32x4_t){o[c][t][4 * i], o[c][t][4 * i + 1], o[c][t][4 * i + 2], o[c][t][4 * i + 3]};
      if (hf == 0) a.part_ml[ph] = make_float2(m_run[c], l);
    }
  }
}

int launch_encoded_tiled(const Dims& dm, const EncodedArgs& a, TiledArgs ta, int B, hipStream_t st) {
  if (a.K4 != nullptr) {
    const dim3 grid((ta.mem_cap + 63) / 64 < 64 ? (ta.mem_cap + 63) / 64 : 64, dm.Hkv, B);
    if (dm.d == 128)
      hipLaunchKernelGGL(expand4_kernel<128>, grid, dim3(256), 0, st, a, ta.Kx, ta.Vx, ta.mem_rows, ta.mem_cap);
    else
      hipLaunchKernelGGL(expand4_kernel<64>, grid, dim3(256), 0, st, a, ta.Kx, ta.Vx, ta.mem_rows, ta.mem_cap);
    if (hipGetLastError() != hipSuccess) return MSA_ERR_HIP;
  }
  const dim3 grid((unsigned)((long long)B * ta.n_tiles * a.n_splits * dm.Hkv));
#define MSA_TILED(DD, CC) hipLaunchKernelGGL((encoded_tiled_kernel<DD, CC, 4>), grid, dim3(256), 0, st, a, ta)
  if (dm.d == 128) {
    if (ta.cb == 2) MSA_TILED(128, 2); else MSA_TILED(128, 1);
  } else {
    if (ta.cb == 2) MSA_TILED(64, 2); else MSA_TILED(64, 1);
  }
#undef MSA_TILED
  if (hipGetLastError() != hipSuccess) return MSA_ERR_HIP;
  if (a.n_splits > 1)
    return launch_merge2(dm.d, a.part_o, a.part_ml, a.n_splits, a.part_o, a.part_ml, 0, a.out, a.lse, 0,
                         (long long)B * a.M * dm.Hq, st);
  return MSA_OK;
}

}  // namespace msa
