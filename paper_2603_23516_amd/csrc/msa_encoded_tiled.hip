// Attention of many query tokens that share position-encoded keys: msa_window_attend over a prompt or a chunk of one,
// msa_sparse_attend4 where the tokens of a sequence share their documents (token_pool = 1).  Bound by the matrix cores.
//
// A workgroup owns a tile of tokens of one (sequence, KV head); its columns are the (token, query head) pairs, 32 to a
// wave.  The rows any token of the tile sees go by in steps of 32: rows of the documents (expanded to
// bf16 once per call, expand4_kernel), the first rows of the cache, the window's.  Per step:
//   copies    32 key and 32 value rows go global -> LDS asynchronously, two steps ahead of their use (three stages), their
//             16-byte pieces placed so that the reads below meet no bank twice
//   scores    S^T[32 keys][32 cols] = K q^T with v_mfma_f32_32x32x16_bf16; the queries stay in registers
//   softmax   online, per column (16 keys in a lane, the other 16 in lane ^ 32)
//   product   O^T[dd][col] += V^T[dd][key] P^T[key][col], the weights in bf16, V^T by transposing LDS reads
// A weight in bf16 is off by 2^-8 of itself at most, either way, and the output by what that comes to; their sum is taken before
// the rounding.  As (hi, lo) pairs, as the single-token kernel carries them at no cost, they would take the second product twice:
// relative error against 64 bits 0.0023 -> 0.0017 (what rounding the output costs by itself), window_prefill 407 -> 535 us,
// window_chunk_64 25 -> 28, attend4_question 168 -> 211.
// Masks are worked out only in steps that some column of the wave does not see whole; steps that a wave does not see at all
// are passed over.
//
// 8192 tokens of 32 / 8 heads of 128, window 4096 (413 GFLOP) 391 to 430 us by card with other work between the calls, 0.96 to
// 1.05 PFLOP/s, and up to 494 us, 0.84, back to back on a card that has warmed up; a product of 8192^3 by the library runs at 1.21.
// The matrix pipe is busy 58 % of the time and the vector ALU 61 %: maximum, exponentials and rounding of 32 x 32 weights take 7.3
// instructions per product, the two meet in one issue slot, and the chip lowers its clock to 1.7 .. 1.9 GHz under both.  1000
// tokens over 16 documents of 512 rows: 165 to 184 us behind 11 of expansion.  Three workgroups of four waves on a CU, 32 columns
// to a wave, was the best shape;
// each at its time, against what it would have replaced: 64 columns to a wave, half of the LDS reads, 859 us for 492; eight
// waves to a workgroup 565 for 492; the scores a step ahead of their weights 457 for 392; a raised wave priority around
// the products slower.
#include "msa_encoded.h"

#include <type_traits>

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
  int before;
  if (tid < 64) docs[tid] = number_rows(a, b, b, g, tid, pre, before);
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
constexpr int kTiledWaves = 4;
constexpr int kTiledStages = 3;

template <int D>
__global__ __launch_bounds__(kTiledWaves * 64) __attribute__((amdgpu_waves_per_eu(3)))
void encoded_tiled_kernel(EncodedArgs a, TiledArgs ta) {
  constexpr int NW = kTiledWaves;
  constexpr int NP = D / 8;      // 16-byte pieces per row
  constexpr int NS = D / 16;     // contraction slices of the score product
  constexpr int NT = D / 32;     // 32-row tiles of the output product
  constexpr int ROW = D * 2;
  constexpr int TILE = 32 * ROW;  // bytes of 32 key or value rows
  constexpr int NI = 32 * NP / 64;     // wave-wide copies for 32 rows
  constexpr int NPW = 2 * NI / NW;     // copies of a wave per step, keys and values together
  static_assert(NPW >= 1 && NPW * NW == 2 * NI, "a step is a whole number of copies per wave");
  __shared__ __attribute__((aligned(16))) unsigned char smem[kTiledStages * 2 * TILE];
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
  if (a.n_splits > 1 && a.tickets != nullptr && sp == 0 && tid == NW * 64 - 1)
    expect_arrivals(a.tickets + (long long)(b * ta.n_tiles + tile) * a.Hkv + g, a.nonce);

  // this lane's column: a (token, head) pair that sees the rows t <= p with t >= lo or t < sinks
  int tl = col / r, head = col - tl * r, tok = (tile * NW + wave) * ta.tpw + tl;
  bool ok = tl < ta.tpw && tok < a.M;
  int p = -1, pmin = INT32_MAX, pmax = -1, plow = INT32_MAX;  // plow: of the tokens that see anything
  if (ok) {
    const long long pl = (long long)a.q_pos[(long long)b * a.M + tok] - a.pos0;
    p = pl < -1 ? -1 : (int)pl;
    pmin = pmax = p;
    if (p >= 0) plow = p;
  }
  int lo = p - a.window + 1;
  if (lo < 0) lo = 0;  // (differences from it stay in 32 bits)
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
  // rows of the cache that the tile goes through: [0, first) and [from, to)
  int first = 0, from = 0, to = 0;
  if (pmax_t >= 0) {
    const Seen see = seen_rows(plow_t, a.Lloc, a.window, a.sinks);
    first = __builtin_amdgcn_readfirstlane(see.first);
    from = __builtin_amdgcn_readfirstlane(see.from);
    to = __builtin_amdgcn_readfirstlane(pmax_t + 1LL < a.Lloc ? pmax_t + 1 : a.Lloc);
  }
  const long long pair = (long long)b * a.Hkv + g;
  const int rows_mem = ta.Kx != nullptr ? __builtin_amdgcn_readfirstlane(ta.mem_rows[pair]) : 0;
  const int steps_mem = (rows_mem + 31) / 32, steps_a = (first + 31) / 32, steps_b = (to - from + 31) / 32;
  const int steps = steps_mem + steps_a + steps_b;
  const int sb = (int)((long long)steps * sp / a.n_splits), se = (int)((long long)steps * (sp + 1) / a.n_splits);
  const uint16_t* const kloc = a.Kloc + pair * a.Lloc * D;
  const uint16_t* const vloc = a.Vloc + pair * a.Lloc * D;

  // queries: B operand of slice s: dims 16 s + 8 hf .. + 8 of the column's head
  bf16x8_t bq[NS];
  const uint16_t* qp = a.q + (((long long)b * a.M + (ok ? tok : 0)) * a.Hq + g * r + (ok ? head : 0)) * D + 8 * hf;
#pragma unroll
  for (int s = 0; s < NS; ++s) {
    uint4 v = *reinterpret_cast<const uint4*>(qp + 16 * s);
    if (!ok) v = make_uint4(0, 0, 0, 0);
    bq[s] = as_bf16x8(v);
  }

  // Places of the 16-byte pieces of a row in LDS: piece p of row i lies at p ^ swz(i).  What a lane reads of slice s (keys) or
  // tile t (values) is then its first address with 32 s or 64 t xored in; rows further on and stages are constants.
  auto swz_k = [](int i) { return D == 128 ? (i & 15) : ((i >> 1) & 7); };
  auto swz_v = [](int i) { return D == 128 ? 4 * (i & 3) : 4 * ((i >> 1) & 1); };
  const int j16 = lane & 15, vrow = 4 * hf + (j16 >> 2);
  int kat[NS], vat[NT];
#pragma unroll
  for (int s = 0; s < NS; ++s) kat[s] = (col * ROW + ((hf ^ swz_k(col)) * 16)) ^ (32 * s);
#pragma unroll
  for (int t = 0; t < NT; ++t)
    vat[t] = TILE + ((vrow * ROW + (((2 * ((lane >> 4) & 1) + ((j16 & 3) >> 1)) ^ swz_v(vrow)) * 16) + 8 * (j16 & 1)) ^ (64 * t));

  // A wave's copies of a step: copy j (j < NI: keys, else values) brings 1 KiB to place j of the stage; its lane's 16 bytes come
  // from byte coff of the step's rows.
  int coff[NPW];
#pragma unroll
  for (int i = 0; i < NPW; ++i) {
    const int j = i * NW + wave, y = (j < NI ? j : j - NI) * 64 + lane, row = y / NP;
    coff[i] = row * ROW + ((y % NP) ^ (j < NI ? swz_k(row) : swz_v(row))) * 16;
  }
  const uint32_t lds0 = __builtin_amdgcn_readfirstlane(lds_addr_of(smem) + wave * 1024);

  // The run of rows that copies have come to: from row n_t0 to n_end, of the documents (n_run 0), the first rows (1) or the
  // window's (2).  (Written with assignments: a choice between variables, c ? x : y, is taken between their places, which then
  // are in scratch memory, and a load from there waits for every copy in flight; the kernel took 1.2 times as long.)
  int n_run = 2, n_t0 = from + 32 * (sb - steps_mem - steps_a), n_end = to;
  const uint16_t *n_k = kloc + (long long)n_t0 * D, *n_v = vloc + (long long)n_t0 * D;
  if (sb < steps_mem) {
    n_run = 0;
    n_t0 = 32 * sb;
    n_end = rows_mem;
    n_k = ta.Kx + (pair * ta.mem_cap + n_t0) * D;
    n_v = ta.Vx + (pair * ta.mem_cap + n_t0) * D;
  } else if (sb < steps_mem + steps_a) {
    n_run = 1;
    n_t0 = 32 * (sb - steps_mem);
    n_end = first;
    n_k = kloc + (long long)n_t0 * D;
    n_v = vloc + (long long)n_t0 * D;
  }
  int t0_of[kTiledStages], cnt_of[kTiledStages];  // of the step in each stage: first row (-1: of the documents) and rows
  auto issue = [&](auto stage) __attribute__((always_inline)) {
    constexpr int INTO = decltype(stage)::value;
    int cnt = n_end - n_t0;
    if (cnt > 32) cnt = 32;
    cnt_of[INTO] = cnt;
    t0_of[INTO] = n_t0;
    if (n_run == 0) t0_of[INTO] = -1;
#pragma unroll
    for (int i = 0; i < NPW; ++i) {
      const uint16_t* src = n_v;
      if (i * NW + wave < NI) src = n_k;
      int off = coff[i];
      if (cnt < 32) {  // rows that do not exist: the last one that does
        const int last = (cnt - 1) * ROW + (off & (ROW - 1));
        off = off < last ? off : last;
      }
      copy16_to_lds_async_at(src, off, lds0 + INTO * 2 * TILE + i * NW * 1024);
    }
    n_t0 += 32;
    n_k += 32 * D;
    n_v += 32 * D;
    if (n_t0 >= n_end) {  // on to the next run (behind the last: nothing asks for it)
      if (n_run == 0 && first > 0) {
        n_run = 1;
        n_t0 = 0;
        n_end = first;
      } else {
        n_run = 2;
        n_t0 = from;
        n_end = to;
      }
      n_k = kloc + (long long)n_t0 * D;
      n_v = vloc + (long long)n_t0 * D;
    }
  };

  float m_run = -INFINITY, l_run = 0.f;
  f32x16e_t o[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[t][i] = 0.f;
  const int lo_first = plow_w - a.window + 1, lo_last = pmax_w - a.window + 1;  // first rows of the wave's windows

  auto step = [&](int s, auto stage) __attribute__((always_inline)) {
    constexpr int BUF = decltype(stage)::value;
    unsigned char* const st = smem + BUF * 2 * TILE;
    if (s + 1 < se)
      wait_copies_but<NPW>();
    else
      wait_copies_but<0>();
    // step s is staged for everyone; everyone is done with step s - 1's stage (its LDS reads have come back)
    lds_barrier();
    if (s + 2 < se) issue(std::integral_constant<int, (BUF + 2) % kTiledStages>());
    const int t0 = t0_of[BUF], cnt = cnt_of[BUF];
    const bool mem = t0 < 0;
    // what this wave sees of the step (uniform)
    if (!(mem | ((t0 <= pmax_w) & ((t0 + 31 >= lo_first) | (t0 < a.sinks))))) return;
    const bool whole = (cnt == 32) & (mem | ((t0 + 31 <= pmin_w) & ((t0 >= lo_last) | (t0 + 31 < a.sinks))));
    f32x16e_t sc;
#pragma unroll
    for (int i = 0; i < 16; ++i) sc[i] = 0.f;
#pragma unroll
    for (int k = 0; k < NS; ++k) sc = mfma32e(as_bf16x8(*reinterpret_cast<const uint4*>(st + kat[k])), bq[k], sc);
    if (!whole) {  // keys most .. least of the step are seen, and those in front of `few` (no branches: one compare each)
      int most = p - t0, least = lo - t0, few = a.sinks - t0;
      if (mem) {
        most = 31;
        least = 0;
      }
      most = (most < cnt - 1 ? most : cnt - 1) - 4 * hf;
      least -= 4 * hf;
      few -= 4 * hf;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int key = (i & 3) + 8 * (i >> 2);
        const bool live = (key <= most) & ((key >= least) | (key < few));
        sc[i] = live ? sc[i] : -INFINITY;
      }
    }
    float mx = sc[0];
#pragma unroll
    for (int i = 1; i < 16; ++i) mx = fmaxf(mx, sc[i]);
    mx = max_xor32(mx) * a.qscale;
    // m_run is what the weights are taken relative to, not the maximum itself: it follows once that is 2^8 ahead (of 128
    // steps some column of 32 meets a new maximum in 76, and every correction is 64 multiplications)
    if (__ballot(mx > m_run + 8.f) != 0) {
      const float m_new = fmaxf(m_run, mx);
      const float alpha = m_run == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m_run - m_new);
      m_run = m_new;
      l_run *= alpha;
#pragma unroll
      for (int t = 0; t < NT; ++t) o[t] *= alpha;
    }
    const float m_use = m_run == -INFINITY ? 0.f : m_run;
    // contraction slot j of slice sg and half hf is key 16 sg + (j % 4) + 8 (j / 4) + 4 hf: the lane's own registers; half of
    // the weights at a time, so that the products of the first half run beside the exponentials of the second
#pragma unroll
    for (int sg = 0; sg < 2; ++sg) {
      uint32_t pw[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float p0 = __builtin_amdgcn_exp2f(fmaf(sc[8 * sg + 2 * i], a.qscale, -m_use));
        const float p1 = __builtin_amdgcn_exp2f(fmaf(sc[8 * sg + 2 * i + 1], a.qscale, -m_use));
        l_run += p0 + p1;
        pw[i] = pack_bf16(p0, p1);
      }
      const bf16x8_t pb = as_bf16x8(make_uint4(pw[0], pw[1], pw[2], pw[3]));
      // (the compiler left to itself puts all sixteen exponentials first: one workgroup on a CU 260 us for 238)
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        const s16x4_t v0 = lds_read_tr16(st + vat[t] + 16 * sg * ROW), v1 = lds_read_tr16(st + vat[t] + (16 * sg + 8) * ROW);
        const bf16x8_t av = __builtin_bit_cast(bf16x8_t, __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7));
        o[t] = mfma32e(av, pb, o[t]);
      }
    }
  };
  if (sb < se) issue(std::integral_constant<int, 0>());
  if (sb + 1 < se) issue(std::integral_constant<int, 1>());
  for (int s = sb; s < se; s += kTiledStages) {  // stages by number, so that LDS addresses are constants
    step(s, std::integral_constant<int, 0>());
    if (s + 1 < se) step(s + 1, std::integral_constant<int, 1>());
    if (s + 2 < se) step(s + 2, std::integral_constant<int, 2>());
  }

  const uint32_t u = __float_as_uint(l_run);
  const auto both = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  float l = __uint_as_float(both[0]) + __uint_as_float(both[1]);

  // ---- the splits' results ----------------------------------------------------------------------------------------
  // Two of them: a part is stored as the registers hold it, each store 512 bytes in a row, past the caches, and the workgroup
  // that arrives last adds the other's to its own.  More are stored by (token, head) row for a launch that joins them: here one
  // part after another comes past the caches at 3 us each (128 tokens over 4096 rows in 8 parts 35 us, by a launch 27; 1000
  // tokens over 9192 in 2 parts 161, by a launch 168; 4096 tokens of 64 dims in 2 parts 55, 76).
  if (a.n_splits > 1 && a.tickets != nullptr) {
    constexpr int PAIRS = NT * 8;  // pairs of floats of a thread
    const long long part0 = ((long long)(b * ta.n_tiles + tile) * a.Hkv + g) * a.n_splits;
    unsigned long long* const po = reinterpret_cast<unsigned long long*>(a.part_o) + part0 * (PAIRS * 256);
    unsigned long long* const pm = reinterpret_cast<unsigned long long*>(a.part_ml) + part0 * 256;
    {
      unsigned long long* const mine = po + (long long)sp * (PAIRS * 256);
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int i = 0; i < 8; ++i)
          store_dev(&mine[(8 * t + i) * 256 + tid],
                    ((unsigned long long)__float_as_uint(o[t][2 * i + 1]) << 32) | __float_as_uint(o[t][2 * i]));
      store_dev(&pm[sp * 256 + tid], ((unsigned long long)__float_as_uint(l) << 32) | __float_as_uint(m_run));
    }
    wait_stores_done();
    __syncthreads();
    unsigned long long* const ticket = a.tickets + (long long)(b * ta.n_tiles + tile) * a.Hkv + g;
    if (tid == 0) pmin_s[0] = (int)arrive_at(ticket, a.nonce);
    __syncthreads();
    if (pmin_s[0] != a.n_splits - 1) return;
    if (tid == 0) store_dev(ticket, 0ull);
    {
      // Products and sums rounded one by one: the result does not depend on which of the two was the last.
#pragma clang fp contract(off)
      const int other = 1 - sp;
      const unsigned long long ml = load_dev(&pm[other * 256 + tid]);
      const float mi = __uint_as_float((uint32_t)ml), m = fmaxf(m_run, mi);
      const float f = m_run == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m_run - m);
      const float fi = mi == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mi - m);
      m_run = m;
      l = l * f + __uint_as_float((uint32_t)(ml >> 32)) * fi;
      const unsigned long long* const theirs = po + (long long)other * (PAIRS * 256);
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        unsigned long long v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = load_dev(&theirs[(8 * t + i) * 256 + tid]);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          o[t][2 * i] = o[t][2 * i] * f + __uint_as_float((uint32_t)v[i]) * fi;
          o[t][2 * i + 1] = o[t][2 * i + 1] * f + __uint_as_float((uint32_t)(v[i] >> 32)) * fi;
        }
      }
    }
  }
  {  // which column this is, again: kept through the loop it would be registers that the loop does not have
    int c = col;
    asm volatile("" : "+v"(c));
    tl = c / r;
    head = c - tl * r;
    tok = (tile * NW + wave) * ta.tpw + tl;
    ok = tl < ta.tpw && tok < a.M;
  }
  if (!ok) return;
  const long long qh = ((long long)b * a.M + tok) * a.Hq + g * r + head;
  if (a.n_splits > 1 && a.tickets == nullptr) {
    const long long ph = qh * a.n_splits + sp;
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *reinterpret_cast<f32x4_t*>(a.part_o + ph * D + 32 * t + 8 * i + 4 * hf) =
            (f32x4_t){o[t][4 * i], o[t][4 * i + 1], o[t][4 * i + 2], o[t][4 * i + 3]};
    if (hf == 0) a.part_ml[ph] = make_float2(m_run, l);
    return;
  }
  const float inv = l > 0.f ? 1.f / l : 0.f;
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      *reinterpret_cast<uint2*>(a.out + qh * D + 32 * t + 8 * i + 4 * hf) =
          make_uint2(pack_bf16(o[t][4 * i] * inv, o[t][4 * i + 1] * inv),
                     pack_bf16(o[t][4 * i + 2] * inv, o[t][4 * i + 3] * inv));
  if (hf == 0 && a.lse != nullptr) a.lse[qh] = l > 0.f ? (m_run + log2f(l)) * 0.6931471805599453f : -INFINITY;
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
  if (dm.d == 128)
    hipLaunchKernelGGL(encoded_tiled_kernel<128>, grid, dim3(kTiledWaves * 64), 0, st, a, ta);
  else
    hipLaunchKernelGGL(encoded_tiled_kernel<64>, grid, dim3(kTiledWaves * 64), 0, st, a, ta);
  if (hipGetLastError() != hipSuccess) return MSA_ERR_HIP;
  if (a.n_splits > 1 && a.tickets == nullptr)
    return launch_merge2(dm.d, a.part_o, a.part_ml, a.n_splits, a.part_o, a.part_ml, 0, a.out, a.lse, 0,
                         (long long)B * a.M * dm.Hq, st);
  return MSA_OK;
}

}  // namespace msa
