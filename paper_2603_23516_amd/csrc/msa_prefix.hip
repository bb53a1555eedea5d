// msa_prefix_attend: one softmax over the rows of a prefix that all sequences share and over the rows of a sequence's own cache.
//
// Where a sequence has tokens enough to fill tiles of its own, encoded_tiled_kernel takes them over the prefix and the cache in one
// go (8 questions of 128 tokens, 32 / 8 heads of 128, over 16384 + 640 rows 298 to 308 us by card, 0.92 to 0.95 PFLOP/s).  With fewer, one launch has
// workgroups of two kinds:
//   over the prefix  tiles of 128 columns, (token, query head) pairs of one KV head and of all sequences together, 32 to a wave, so
//                    that a row is read once for all of them (per tile).  As encoded_tiled_kernel, without windows and runs: 32 key
//                    and 32 value rows a step, global -> LDS asynchronously, two steps ahead, in n parts of which each takes every
//                    n-th step.  Bound by what follows on what in a wave, scores, weights and second product in turn, with one
//                    workgroup on a CU: a step takes 0.96 us (8 tokens over 65536 rows 63 us, 4.3 TB/s).
//   over the caches  sixteen columns of one (sequence, KV head); the rows go straight from memory into registers, dealt to the
//                    four waves 32 at a time.  Bound by memory (64 tokens, 1024 rows each, 268 MB: 59 us).
// Both leave (max, sum, output) parts by (token, head) row, which a launch joins.  The two kinds fill each other's gaps: 64 tokens
// over 32768 rows 70 us, over up to 1024 rows of caches 44, both 87.  256 workgroups over the prefix, one to a CU, leave the
// others of a CU to the caches: with 384, 512 and 768 the call of 87 us takes 85, 86 and 101 (without caches 70: 72, 68, 73), one of
// 16 x 4 tokens over 8000 rows and up to 1500 of caches 40 and 43 for 34.
// Softmax weights go into the second product as bf16 (hi, lo) pairs, off by 2^-16 of themselves at most, as in msa_window_attend's
// kernel for single tokens: these are single tokens, or a few of them, in both kinds.  Over the caches the second half of that
// product costs nothing beside the loads, over the prefix 8 us of 70 (weights rounded to bf16, off by 2^-8: 64 tokens over
// 32768 rows 62 us, with their caches 80 for 87, 24 x 5 tokens of 64 dims over 4999 rows 18.2 for 19.2, 16 over 8000 27.4 for 27.2;
// products and the other half's exponentials one by one in turn: the same as products first).
#include "msa_prefix.h"

#include <type_traits>
#include <utility>

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

// What sequence b sees of the prefix.
__device__ __forceinline__ int prefix_of(const PrefixArgs& a, long long b) {
  if (a.pre_lens == nullptr) return a.Lpre;
  const int n = a.pre_lens[b];
  return n < 0 ? 0 : (n < a.Lpre ? n : a.Lpre);
}

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
  u32x4_t kx[2][NS], vx[2][NS];
  auto load = [&](int t0) __attribute__((always_inline)) {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      int row = t0 + 16 * t + n;
      row = row < end ? row : end - 1;
      const long long at = (long long)row * D + 8 * qd;
#pragma unroll
      for (int j = 0; j < NS; ++j) {
        kx[t][j] = *reinterpret_cast<const u32x4_t*>(K + at + 32 * j);
        vx[t][j] = *reinterpret_cast<const u32x4_t*>(V + at + 32 * j);
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
        sc[t] = mfma16(__builtin_bit_cast(bf16x8_t, kx[t][j]), bq[j], sc[t]);
        *reinterpret_cast<u32x4_t*>(vt + (16 * t + n) * ROW + (((4 * j + qd) ^ swz(16 * t + n)) * 16)) = vx[t][j];
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
    uint32_t hi[4], lo[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float p0 = __builtin_amdgcn_exp2f(w[2 * j] - m_use), p1 = __builtin_amdgcn_exp2f(w[2 * j + 1] - m_use);
      x.l_run += p0 + p1;
      split_pack_bf16(p0, p1, hi[j], lo[j]);
    }
    const bf16x8_t ph = as_bf16x8(make_uint4(hi[0], hi[1], hi[2], hi[3])), pl = as_bf16x8(make_uint4(lo[0], lo[1], lo[2], lo[3]));
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    const int row = 4 * qd + (n >> 2);
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const unsigned char* vp = vt + row * ROW + (((2 * c + ((n & 3) >> 1)) ^ swz(row)) * 16) + 8 * (n & 1);
      const s16x4_t v0 = lds_read_tr16(vp), v1 = lds_read_tr16(vp + 16 * ROW);  // rows 16 apart: the same swizzle
      const bf16x8_t av = __builtin_bit_cast(bf16x8_t, __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7));
      x.o[c] = mfma16(av, pl, mfma16(av, ph, x.o[c]));
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }
}

constexpr int kPrefixParts = 192;  // of a row at most, 32 of them over the cache
constexpr int kPrefixStages = 3;
constexpr int kPrefixWaves = 4;

template <int D>
__device__ __forceinline__ void over_prefix(const PrefixArgs& a, int x, unsigned char* smem) {
  constexpr int NW = kPrefixWaves, STAGES = kPrefixStages, AHEAD = STAGES - 1;  // steps whose copies are under way
  constexpr int NP = D / 8;            // 16-byte pieces per row
  constexpr int NS = D / 16;           // contraction slices of the score product
  constexpr int NT = D / 32;           // 32-row tiles of the output product
  constexpr int ROW = D * 2;
  constexpr int TILE = 32 * ROW;       // bytes of 32 key or value rows
  constexpr int NI = 32 * NP / 64;     // wave-wide copies for 32 rows
  constexpr int NPW = 2 * NI / NW;     // copies of a wave per step, keys and values together
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int hf = lane >> 5, col = lane & 31, r = a.r;
  // (tile, part, KV head): the KV head fastest, so that an XCD (every eighth workgroup) keeps to few heads' rows
  const int g = x % a.Hkv;
  x /= a.Hkv;
  const int sp = x % a.n_pre, tile = x / a.n_pre;
  const int BM = a.B * a.M;  // (2^25 at most)

  // this lane's column, and the rows [0, lim) that it sees
  const int tl = col / r, head = col - tl * r;
  const int tok = (tile * NW + wave) * a.tpw + tl;
  const bool ok = tl < a.tpw && tok < BM;
  bf16x8_t bq[NS];
  const long long qh = (long long)(ok ? tok : 0) * a.Hq + g * r + (ok ? head : 0);
#pragma unroll
  for (int s = 0; s < NS; ++s)
    bq[s] = as_bf16x8(keep_if(*reinterpret_cast<const uint4*>(a.q + qh * D + 8 * hf + 16 * s), ok));
  const int lim = ok ? prefix_of(a, tok / a.M) : 0;
  int least = ok ? lim : INT32_MAX, most = lim;
  least = min_of_lanes<32>(least);
  most = max_of_lanes<32>(most);
  int* const most_s = reinterpret_cast<int*>(smem);
  if (lane == 0) most_s[wave] = most;
  __syncthreads();
  int end = most_s[0];
#pragma unroll
  for (int w = 1; w < NW; ++w) end = most_s[w] > end ? most_s[w] : end;
  end = __builtin_amdgcn_readfirstlane(end);
  __syncthreads();  // (the copies come to the same place)
  const int steps = (end + 31) / 32;
  const int se = (steps - sp + a.n_pre - 1) / a.n_pre;  // this part's steps: sp, sp + n_pre, ...

  // (waited for here: at their first use, in the loop, the wait would be one for all copies in flight as well)
#pragma unroll
  for (int s = 0; s < NS; ++s) asm volatile("" : "+v"(bq[s]));

  // Places of the 16-byte pieces of a row in LDS: piece p of row i lies at p ^ swz(i), so that the reads meet no bank twice.
  auto swz_k = [](int i) { return D == 128 ? (i & 15) : ((i >> 1) & 7); };
  auto swz_v = [](int i) { return D == 128 ? 4 * (i & 3) : 4 * ((i >> 1) & 1); };
  const int j16 = lane & 15, vrow = 4 * hf + (j16 >> 2);
  int kat[NS], vat[NT];
#pragma unroll
  for (int s = 0; s < NS; ++s) kat[s] = (col * ROW + ((hf ^ swz_k(col)) * 16)) ^ (32 * s);
#pragma unroll
  for (int t = 0; t < NT; ++t)
    vat[t] = TILE + ((vrow * ROW + (((2 * ((lane >> 4) & 1) + ((j16 & 3) >> 1)) ^ swz_v(vrow)) * 16) + 8 * (j16 & 1)) ^ (64 * t));
  int coff[NPW];
#pragma unroll
  for (int i = 0; i < NPW; ++i) {
    const int j = i * NW + wave, y = (j < NI ? j : j - NI) * 64 + lane, row = y / NP;
    coff[i] = row * ROW + ((y % NP) ^ (j < NI ? swz_k(row) : swz_v(row))) * 16;
  }
  const uint32_t lds0 = __builtin_amdgcn_readfirstlane(lds_addr_of(smem) + wave * 1024);
  const long long at0 = ((long long)g * a.Lpre + 32LL * sp) * D;
  const uint16_t *n_k = a.Kpre + at0, *n_v = a.Vpre + at0;
  int n_cnt = end - 32 * sp;  // rows from the next copy's first one on
  auto issue = [&](auto stage) __attribute__((always_inline)) {
    constexpr int INTO = decltype(stage)::value;
#pragma unroll
    for (int i = 0; i < NPW; ++i) {
      const uint16_t* src = n_v;
      if (i * NW + wave < NI) src = n_k;
      int off = coff[i];
      if (n_cnt < 32) {  // rows that nobody sees: the last one that somebody does
        const int last = (n_cnt - 1) * ROW + (off & (ROW - 1));
        off = off < last ? off : last;
      }
      copy16_to_lds_async_at(src, off, lds0 + INTO * 2 * TILE + i * NW * 1024);
    }
    n_cnt -= 32 * a.n_pre;
    n_k += (long long)a.n_pre * 32 * D;
    n_v += (long long)a.n_pre * 32 * D;
  };

  float m_run = -INFINITY, l_run = 0.f;
  f32x16e_t o[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[t][i] = 0.f;

  auto step = [&](int s, auto stage) __attribute__((always_inline)) {
    constexpr int BUF = decltype(stage)::value;
    unsigned char* const st = smem + BUF * 2 * TILE;
    if (s + AHEAD - 1 < se)
      wait_copies_but<(AHEAD - 1) * NPW>();
    else
      wait_copies_but<0>();
    // step s is staged for everyone; everyone is done with step s - 1's stage (its LDS reads have come back)
    lds_barrier();
    if (s + AHEAD < se) issue(std::integral_constant<int, (BUF + AHEAD) % STAGES>());
    const int t0 = 32 * (sp + s * a.n_pre);
    if (t0 >= most) return;  // this wave sees nothing of the step (uniform)
    f32x16e_t sc;
#pragma unroll
    for (int i = 0; i < 16; ++i) sc[i] = 0.f;
#pragma unroll
    for (int k = 0; k < NS; ++k) sc = mfma32e(as_bf16x8(*reinterpret_cast<const uint4*>(st + kat[k])), bq[k], sc);
    if (t0 + 32 > least) {
      const int left = lim - t0 - 4 * hf;
#pragma unroll
      for (int i = 0; i < 16; ++i) sc[i] = (i & 3) + 8 * (i >> 2) < left ? sc[i] : -INFINITY;
    }
    float mx = sc[0];
#pragma unroll
    for (int i = 1; i < 16; ++i) mx = fmaxf(mx, sc[i]);
    mx = max_xor32(mx) * a.qscale;
    if (__ballot(mx > m_run + 8.f) != 0) {  // m_run follows the maximum once that is 2^8 ahead
      const float m_new = fmaxf(m_run, mx);
      const float alpha = m_run == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m_run - m_new);
      m_run = m_new;
      l_run *= alpha;
#pragma unroll
      for (int t = 0; t < NT; ++t) o[t] *= alpha;
    }
    const float m_use = m_run == -INFINITY ? 0.f : m_run;
    // contraction slot j of slice sg and half hf is key 16 sg + (j % 4) + 8 (j / 4) + 4 hf: the lane's own registers
#pragma unroll
    for (int sg = 0; sg < 2; ++sg) {
      uint32_t hi[4], lo[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float p0 = __builtin_amdgcn_exp2f(fmaf(sc[8 * sg + 2 * i], a.qscale, -m_use));
        const float p1 = __builtin_amdgcn_exp2f(fmaf(sc[8 * sg + 2 * i + 1], a.qscale, -m_use));
        l_run += p0 + p1;
        split_pack_bf16(p0, p1, hi[i], lo[i]);
      }
      const bf16x8_t ph = as_bf16x8(make_uint4(hi[0], hi[1], hi[2], hi[3])), pl = as_bf16x8(make_uint4(lo[0], lo[1], lo[2], lo[3]));
      __builtin_amdgcn_sched_barrier(0);  // (the products of one half beside the exponentials of the other)
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        const s16x4_t v0 = lds_read_tr16(st + vat[t] + 16 * sg * ROW), v1 = lds_read_tr16(st + vat[t] + (16 * sg + 8) * ROW);
        const bf16x8_t av = __builtin_bit_cast(bf16x8_t, __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7));
        o[t] = mfma32e(av, pl, mfma32e(av, ph, o[t]));
      }
    }
  };
  // stages by number, so that LDS addresses are constants
  each_stage(std::make_integer_sequence<int, AHEAD>(), [&](auto stage) {
    if (decltype(stage)::value < se) issue(stage);
  });
  for (int s = 0; s < se; s += STAGES)
    each_stage(std::make_integer_sequence<int, STAGES>(), [&](auto stage) __attribute__((always_inline)) {
      if (s + decltype(stage)::value < se) step(s + decltype(stage)::value, stage);
    });
  const uint32_t u = __float_as_uint(l_run);
  const auto both = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  const float l = __uint_as_float(both[0]) + __uint_as_float(both[1]);
  if (!ok) return;
  const long long ph = qh * a.n_pre + sp;
  if (hf == 0) a.pre_ml[ph] = make_float2(m_run, l);
  if (m_run == -INFINITY) return;  // (an empty part's outputs are not read)
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      *reinterpret_cast<f32x4_t*>(a.pre_o + ph * D + 32 * t + 8 * i + 4 * hf) =
          (f32x4_t){o[t][4 * i], o[t][4 * i + 1], o[t][4 * i + 2], o[t][4 * i + 3]};
}

// A column of a workgroup over a cache: column n is head n % r of token m0 + n / r of sequence b, and sees the rows below lim.
struct CacheColumn {
  bool ok;          // there is such a token ...
  int tok, head;    // ... else another that there is
  int lim;
  int least, most;  // of the sixteen columns' lim, those that are
};
__device__ __forceinline__ CacheColumn cache_column(const PrefixArgs& a, long long b, int m0, int n) {
  CacheColumn c;
  const int tl = n / a.r;
  c.ok = tl < a.tpl && m0 + tl < a.M;
  c.tok = c.ok ? m0 + tl : m0;
  c.head = c.ok ? n - tl * a.r : 0;
  const long long p1 = (long long)a.q_pos[b * a.M + c.tok] - a.pos0 + 1;
  c.lim = c.ok ? (p1 < 0 ? 0 : (p1 < a.Lloc ? (int)p1 : a.Lloc)) : 0;
  c.least = min_of_lanes<16>(c.ok ? c.lim : INT32_MAX);
  c.most = max_of_lanes<16>(c.lim);
  return c;
}

template <int D>
__device__ __forceinline__ void over_cache(const PrefixArgs& a, int x, unsigned char* smem) {
  constexpr int NW = kPrefixWaves, NS = D / 32, NC = D / 16;
  constexpr int OROW = D + 4;  // floats of a row of a wave's output in the merge
  constexpr int STAGE = 16 * OROW * 4;
  static_assert(STAGE >= 32 * D * 2, "32 value rows");
  float* const wm = reinterpret_cast<float*>(smem + NW * STAGE);  // [NW][16] maxima, sums
  float* const wl = wm + 16 * NW;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int qd = lane >> 4, n = lane & 15, r = a.r;
  const int g = x % a.Hkv;
  x /= a.Hkv;
  const int sp = x % a.n_loc;
  x /= a.n_loc;
  const int m0 = x % a.groups * a.tpl;
  const long long b = x / a.groups;
  const CacheColumn col = cache_column(a, b, m0, n);
  const long long qh = (b * a.M + col.tok) * a.Hq + g * r + col.head;
  bf16x8_t bq[NS];
#pragma unroll
  for (int s = 0; s < NS; ++s)
    bq[s] = as_bf16x8(keep_if(*reinterpret_cast<const uint4*>(a.q + qh * D + 32 * s + 8 * qd), col.ok));
  const int steps = (col.most + 31) / 32;
  const int sb = (int)((long long)steps * sp / a.n_loc), se = (int)((long long)steps * (sp + 1) / a.n_loc);
  Columns<D> y;
  y.m_run = -INFINITY;
  y.l_run = 0.f;
#pragma unroll
  for (int c = 0; c < NC; ++c) y.o[c] = (f32x4_t){0.f, 0.f, 0.f, 0.f};
  const long long loc = (b * a.Hkv + g) * a.Lloc * D;
  attend_rows<D>(a.Kloc + loc, a.Vloc + loc, col.most, sb + wave, se, NW, bq, col.lim, col.least, a.qscale, smem + wave * STAGE, y);

  // the waves' results
  y.l_run = add_xor32(add_xor16(y.l_run));
  float* const mine = reinterpret_cast<float*>(smem + wave * STAGE);
#pragma unroll
  for (int c = 0; c < NC; ++c) *reinterpret_cast<f32x4_t*>(mine + n * OROW + 16 * c + 4 * qd) = y.o[c];
  if (qd == 0) {
    wm[16 * wave + n] = y.m_run;
    wl[16 * wave + n] = y.l_run;
  }
  __syncthreads();
  for (int e = tid; e < 16 * D / 4; e += 64 * NW) {
    const int c = e / (D / 4), dd = e % (D / 4) * 4, t = c / r;
    if (t >= a.tpl || m0 + t >= a.M) continue;
    const long long ph = ((b * a.M + m0 + t) * a.Hq + g * r + (c - t * r)) * a.n_loc + sp;
    float m = wm[c];
#pragma unroll
    for (int w = 1; w < NW; ++w) m = fmaxf(m, wm[16 * w + c]);
    float l = 0.f;
    f32x4_t v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      const float f = wm[16 * w + c] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(wm[16 * w + c] - m);
      l += f * wl[16 * w + c];
      v += f * *reinterpret_cast<const f32x4_t*>(smem + w * STAGE + (c * OROW + dd) * 4);
    }
    if (dd == 0) a.loc_ml[ph] = make_float2(m, l);
    *reinterpret_cast<f32x4_t*>(a.loc_o + ph * D + dd) = v;
  }
}

template <int D>
__global__ __launch_bounds__(64 * kPrefixWaves) __attribute__((amdgpu_waves_per_eu(3))) void prefix_kernel(PrefixArgs a) {
  constexpr int BYTES = kPrefixStages * 2 * 32 * D * 2;
  constexpr int CACHE = kPrefixWaves * (16 * (D + 4) * 4 + 128);
  __shared__ __attribute__((aligned(16))) unsigned char smem[BYTES > CACHE ? BYTES : CACHE];
  if ((int)blockIdx.x < a.pre_groups)
    over_prefix<D>(a, blockIdx.x, smem);
  else
    over_cache<D>(a, blockIdx.x - a.pre_groups, smem);
}

// The parts of every (token, head): a workgroup to a row, its waves the parts i, i + 4, ..., eight of them at a time under way
// together with all (max, sum) pairs.  2048 rows of 17 parts 6.4 us.  (A wave to a row, as the other paths join theirs, is one part
// after another where rows are few and parts many: 256 rows of 68 parts 22 us for 5, 2048 of 33 13 for 8.)
template <int D>
__global__ __launch_bounds__(256) void prefix_join_kernel(PrefixArgs a, long long rows) {
  constexpr int V = D / 64, U = 8;
  typedef float vec_t __attribute__((ext_vector_type(V)));
  __shared__ float o_s[4][D];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const long long row = (long long)blockIdx.y * gridDim.x + blockIdx.x;
  if (row >= rows) return;
  const int n1 = a.n_pre, ns = n1 + a.n_loc;
  const float2 *const m1 = a.pre_ml + row * n1, *const m2 = a.loc_ml + row * a.n_loc;
  const float *const p1 = a.pre_o + row * n1 * D + lane * V, *const p2 = a.loc_o + row * a.n_loc * D + lane * V;
  vec_t v[U];
  auto fetch = [&](int s0) {  // (past the end: the last one again)
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int s = s0 + 4 * u < ns ? s0 + 4 * u : ns - 1;
      v[u] = *reinterpret_cast<const vec_t*>(s < n1 ? p1 + (long long)s * D : p2 + (long long)(s - n1) * D);
    }
  };
  auto pair_at = [&](int s) {  // (no load under a condition of its own: they are under way together)
    const int at = s < ns ? s : ns - 1;
    float2 ml = *(at < n1 ? m1 + at : m2 + (at - n1));
    if (s >= ns) ml.x = -INFINITY;
    return ml;
  };
  fetch(wave);
  float2 ml[kPrefixParts / 64];
  ml[0] = pair_at(lane);
#pragma unroll
  for (int i = 1; i < kPrefixParts / 64; ++i) {
    ml[i] = make_float2(-INFINITY, 0.f);
    if (64 * i < ns) ml[i] = pair_at(lane + 64 * i);
  }
  float mx = -INFINITY;
#pragma unroll
  for (int i = 0; i < kPrefixParts / 64; ++i) mx = fmaxf(mx, ml[i].x);
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) mx = fmaxf(mx, __shfl_xor(mx, off, 64));
  float lsum = 0.f, w[kPrefixParts / 64];
#pragma unroll
  for (int i = 0; i < kPrefixParts / 64; ++i) {
    const bool empty = ml[i].x == -INFINITY;  // (its outputs may be anything)
    w[i] = empty ? -1.f : __builtin_amdgcn_exp2f(ml[i].x - mx);
    lsum += empty ? 0.f : w[i] * ml[i].y;
  }
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) lsum += __shfl_xor(lsum, off, 64);
  vec_t acc = 0.f;
#pragma unroll
  for (int i = 0; i < kPrefixParts / 64; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j) {  // parts 64 i + 32 j + wave, + 4, ... of this wave
      const int s0 = 64 * i + 32 * j;
      if (s0 + wave >= ns) continue;
      if (s0 > 0) fetch(s0 + wave);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const float f = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(w[i]), 32 * j + wave + 4 * u));
        if (s0 + wave + 4 * u < ns && !(f < 0.f)) acc += f * v[u];  // wave-uniform
      }
    }
#pragma unroll
  for (int c = 0; c < V; ++c) o_s[wave][lane * V + c] = acc[c];
  __syncthreads();
  if (threadIdx.x < D / 2) {
    const int d = 2 * threadIdx.x;
    float x0 = 0.f, x1 = 0.f;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      x0 += o_s[u][d];
      x1 += o_s[u][d + 1];
    }
    const float inv = lsum > 0.f ? 1.f / lsum : 0.f;
    reinterpret_cast<uint32_t*>(a.out + row * D)[threadIdx.x] = pack_bf16(x0 * inv, x1 * inv);
    if (threadIdx.x == 0 && a.lse != nullptr) a.lse[row] = lsum > 0.f ? (mx + log2f(lsum)) * 0.6931471805599453f : -INFINITY;
  }
}

PrefixPlan plan_prefix(const Dims& dm, int B, int M, int Lpre, int Lloc) {
  PrefixPlan p = {};
  // A sequence's tokens in tiles of their own, where they fill three quarters of one and the batch fills three.  us, so / with tiles of
  // all sequences' tokens, 32 / 8 heads of 128, 600 rows of a cache, a prefix of 2000 (16384):
  //   1 sequence    M = 32 21 / 17 (35 / 32), 48 21 / 20 (43 / 45)
  //   2 sequences   M = 24 21 / 20 (43 / 44), 48 26 / 28 (56 / 75)
  //   8 sequences   M = 16 26 / 29 (99 / 81), 24 29 / 46 (91 / 133), 48 41 / 66 (156 / 234)
  //   32 sequences  M = 12 57 / 72 (269 / 246), 24 61 / 119 (287 / 386), 48 95 / 207 (560 / 746)
  //   4 sequences, 8 / 8 heads of 64, 4000   M = 64 22 / 17, 128 24 / 25
  if (M * dm.r >= 96 && (long long)B * M * dm.r >= 384) {
    p.tiled = 1;
    p.tiles = plan_encoded_prefix(dm, B, M, Lpre, Lloc);
    p.ws_bytes = p.tiles.ws_bytes;
    return p;
  }
  const long long BM = (long long)B * M, rows = BM * dm.Hq;
  const int tpw = 32 / dm.r, tpl = 16 / dm.r;
  const long long tiles = (BM + kPrefixWaves * tpw - 1) / (kPrefixWaves * tpw) * dm.Hkv, groups = (long long)B * ((M + tpl - 1) / tpl) * dm.Hkv;
  if (tiles + groups >= 1 << 22) return p;
  auto parts = [](long long steps, long long units, long long wanted, long long least, int most) {
    long long n = (wanted + units - 1) / units;
    if (n > steps / least) n = steps / least;
    return (int)(n < 1 ? 1 : (n > most ? most : n));
  };
  p.n_pre = Lpre > 0 ? parts((Lpre + 31) / 32, tiles, 256, 4, kPrefixParts - 32) : 0;
  p.n_loc = Lloc > 0 ? parts((Lloc + 31) / 32, groups, 512, 8, 32) : 0;
  size_t at = round_up256((size_t)rows * p.n_pre * dm.d * sizeof(float));
  p.off_pre_ml = at;
  at += round_up256((size_t)rows * p.n_pre * sizeof(float2));
  p.off_loc_o = at;
  at += round_up256((size_t)rows * p.n_loc * dm.d * sizeof(float));
  p.off_loc_ml = at;
  at += round_up256((size_t)rows * p.n_loc * sizeof(float2));
  p.ws_bytes = at;
  return p;
}

int launch_prefix(const Dims& dm, const PrefixPlan& pl, PrefixArgs a, void* ws, hipStream_t st) {
  unsigned char* const w = (unsigned char*)ws;
  a.Hq = dm.Hq;
  a.Hkv = dm.Hkv;
  a.r = dm.r;
  a.qscale = (float)(1.4426950408889634 / sqrt((double)dm.d));
  if (pl.tiled) {
    EncodedArgs e = {};
    e.q = a.q;
    e.Kloc = a.Kloc;
    e.Vloc = a.Vloc;
    e.q_pos = a.q_pos;
    e.out = a.out;
    e.lse = a.lse;
    e.part_o = (float*)w;
    e.part_ml = (float2*)(w + pl.tiles.off_ml);
    e.M = a.M;
    e.Hq = a.Hq;
    e.Hkv = a.Hkv;
    e.r = a.r;
    e.Lloc = a.Lloc;
    e.pos0 = a.pos0;
    no_window(&e);
    e.n_splits = pl.tiles.n_splits;
    e.qscale = a.qscale;
    if (e.n_splits == 2) e.tickets = (unsigned long long*)(w + pl.tiles.off_tickets);
    e.nonce = launch_nonce48();
    TiledArgs ta = {};
    ta.tpw = pl.tiles.tpw;
    ta.n_tiles = pl.tiles.n_tiles;
    if (a.Lpre > 0) {
      ta.Kx = const_cast<uint16_t*>(a.Kpre);
      ta.Vx = const_cast<uint16_t*>(a.Vpre);
      ta.mem_cap = a.Lpre;
      ta.shared = 1;
      ta.shared_lens = a.pre_lens;
    }
    return launch_encoded_tiled(dm, e, ta, a.B, st);
  }
  const long long BM = (long long)a.B * a.M;
  a.tpw = 32 / dm.r;
  a.tpl = 16 / dm.r;
  a.groups = (a.M + a.tpl - 1) / a.tpl;
  a.n_pre = pl.n_pre;
  a.n_loc = pl.n_loc;
  a.pre_o = (float*)w;
  a.pre_ml = (float2*)(w + pl.off_pre_ml);
  a.loc_o = (float*)(w + pl.off_loc_o);
  a.loc_ml = (float2*)(w + pl.off_loc_ml);
  a.pre_groups = (int)((BM + kPrefixWaves * a.tpw - 1) / (kPrefixWaves * a.tpw) * dm.Hkv * a.n_pre);
  const dim3 grid((unsigned)(a.pre_groups + (long long)a.B * a.groups * dm.Hkv * a.n_loc));
  if (dm.d == 128)
    hipLaunchKernelGGL(prefix_kernel<128>, grid, dim3(64 * kPrefixWaves), 0, st, a);
  else
    hipLaunchKernelGGL(prefix_kernel<64>, grid, dim3(64 * kPrefixWaves), 0, st, a);
  if (hipGetLastError() != hipSuccess) return MSA_ERR_HIP;
  const long long rows = BM * dm.Hq;
  const dim3 joins((unsigned)(rows < 1 << 20 ? rows : 1 << 20), (unsigned)((rows + (1 << 20) - 1) >> 20));
  if (dm.d == 128)
    hipLaunchKernelGGL(prefix_join_kernel<128>, joins, dim3(256), 0, st, a, rows);
  else
    hipLaunchKernelGGL(prefix_join_kernel<64>, joins, dim3(256), 0, st, a, rows);
  return hipGetLastError() == hipSuccess ? MSA_OK : MSA_ERR_HIP;
}

}  // namespace msa
