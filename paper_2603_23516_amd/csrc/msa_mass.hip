// msa_attend_mass: the attention weight that every row of the local cache receives from the tokens of a call,
//     out[b][g][t] = decay mass[b][g][t] + sum over tokens m and heads h of group g that see row t of
//                    exp(q[b][m][h] . Kloc[b][g][t] / sqrt(d) - lse[b][m][h])
// with the log-sums that the attention left.  The product has rows of K against columns, (token, head) pairs of one (sequence, KV
// head); a weight is one fma and one exponential, and every lane adds up its rows' weights over the columns it meets, the lanes of a
// row at the end.  Nothing depends on an order of arrival.  Queries and keys are bf16 as given, products and sums fp32: nothing is
// rounded to fewer bits.
//
// mass_rows_kernel, up to 64 columns: a wave to 32 rows, all of them and all columns in registers.  Bound by memory: K is read once,
// and of it the blocks of 32 rows that some column sees (16 sequences of 8192 rows under a window of 1024 13.4 us,
// without that 32).
//
// mass_tiled_kernel, more columns: a wave keeps 32 rows in registers, the queries come by in steps of 32 columns through LDS, with them
// the log-sum and the position of every column.  Per 32 x 32 weights stand 8 products of 32x32x16 (d = 128) against 80 vector
// instructions, of which 48 are the weights (fma, exponential, sum) and 16 of these take twice the time: 8192 tokens of 32 / 8 heads of
// 128 (275 GFLOP) 330 to 345 us by card, 0.80 to 0.83 PFLOP/s, vector ALU 74 % and matrix pipe 46 % busy.  64 rows to a wave would halve what is not
// the weights and leave two waves to a SIMD for four: 367.  The columns that a tile of 128 rows needs are shared out to several
// workgroups, whose sums mass_join_kernel adds in order (2048 workgroups in all: with 1024 362, with 4096 333 and short calls up to
// 40 % longer; eight steps at least to a part).
#include "msa_encoded.h"

#include <type_traits>
#include <utility>

namespace msa {

constexpr float kLog2e = 1.4426950408889634f;

// Which rows a token sees: t <= p with t >= lo or t < sinks; none: p = -1.
struct SeenBy {
  int p, lo;
};
__device__ __forceinline__ SeenBy seen_by(const MassArgs& a, int32_t q_pos) {
  const int pl = __builtin_elementwise_sub_sat(q_pos, a.pos0);  // (saturated: in front of the cache all the same)
  SeenBy s;
  s.p = pl < -1 ? -1 : (pl < a.Lloc ? pl : a.Lloc - 1);
  const int lo = __builtin_elementwise_sub_sat(pl, a.window - 1);
  s.lo = lo < 0 ? 0 : lo;
  return s;
}
// Bits 0 to x; none for x < 0, all for x > 30.
__device__ __forceinline__ uint32_t up_to(int x) { return x < 0 ? 0u : ~0u >> (x < 31 ? 31 - x : 0); }
__device__ __forceinline__ float old_weight(const MassArgs& a, long long at) {
  return a.mass != nullptr && a.decay != 0.f ? a.mass[at] * a.decay : 0.f;
}

// ---- few columns ---------------------------------------------------------------------------------------------------------
// (A wave to 32 rows, a workgroup of its own, and eight of them to a SIMD: 40 sequences of 8192 rows, 8 heads of 128, 114 us, 6.0 TB/s,
// of 0 to 8192 rows, 4000 on average, 67.  Two, four, eight and sixteen waves to a workgroup 116, 114, 118, 121 and 69, 72, 77, 80; waves
// that go on through 64 to 512 rows with one or two blocks ahead 120 to 139 and 88 to 93; 64 rows at once 119 and 73; workgroups by rows
// first and sequences second 127 and 79.  What a wave does ahead of its rows counts, since half of the waves have none: workgroup
// numbers and columns taken apart by division and their ends compared through LDS 115 and 69.)
constexpr int kRowsRows = 32;  // rows of a wave
template <int D, int CG>  // CG: groups of 16 columns
__global__ __launch_bounds__(64) __attribute__((amdgpu_waves_per_eu(CG == 1 ? 8 : 1))) void mass_rows_kernel(MassArgs a, uint32_t by_r) {
  constexpr int NS = D / 32;  // by_r: 2^16 / r and one more, so that col / r = col by_r / 2^16 for all 64 columns
  const int lane = threadIdx.x;
  const int qd = lane >> 4, n = lane & 15, r = a.r;
  const int t0 = (int)blockIdx.x * kRowsRows, g = blockIdx.y;
  if (t0 >= a.Lloc) return;
  const long long b = blockIdx.z, pair = b * a.Hkv + g;
  const int cols = a.M * r;
  const bool weighed = a.mass != nullptr && a.decay != 0.f;
  float old[2];  // of row 4 qd + n % 4 of either half of the 32
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int t = t0 + 16 * k + 4 * qd + (n & 3);
    old[k] = weighed ? a.mass[pair * a.Lloc + (t < a.Lloc ? t : a.Lloc - 1)] : 0.f;
  }
  bf16x8_t q[CG][NS];
  float ls[CG];
  SeenBy see[CG];
  int most = -1, least = INT32_MAX;  // the last row that any column sees, and the first one of the windows
#pragma unroll
  for (int c = 0; c < CG; ++c) {
    const int at = 16 * c + n, col = at < cols ? at : cols - 1;
    const int m = (int)((uint32_t)col * by_r >> 16);
    const long long tok = b * a.M + m, qh = tok * a.Hq + g * r + (col - m * r);
    see[c] = seen_by(a, a.q_pos[tok]);
    ls[c] = a.lse[qh] * kLog2e;
    if (at >= cols || ls[c] == -INFINITY) see[c].p = -1;  // (a token that saw nothing)
    most = see[c].p > most ? see[c].p : most;
    least = see[c].p >= 0 && see[c].lo < least ? see[c].lo : least;
#pragma unroll
    for (int s = 0; s < NS; ++s) q[c][s] = as_bf16x8(*reinterpret_cast<const uint4*>(a.q + qh * D + 32 * s + 8 * qd));
  }
  most = max_of_lanes<16>(most);
  least = min_of_lanes<16>(least);
  const bool seen = t0 <= most && (t0 + kRowsRows > least || t0 < a.sinks);  // wave-uniform
  if (!seen && a.mass == a.out && a.decay == 1.f) return;  // rows that nobody sees, in place: as they are
  float sum[2][4];
#pragma unroll
  for (int k = 0; k < 2; ++k)
#pragma unroll
    for (int i = 0; i < 4; ++i) sum[k][i] = 0.f;
  if (seen) {
    const uint16_t* const keys = a.Kloc + pair * a.Lloc * D + 8 * qd;
    u32x4_t key[2][NS];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      int row = t0 + 16 * k + n;
      row = row <= most ? row : most;
#pragma unroll
      for (int s = 0; s < NS; ++s) key[k][s] = *reinterpret_cast<const u32x4_t*>(keys + (long long)row * D + 32 * s);
    }
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int c = 0; c < CG; ++c) {
        f32x4_t sc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s = 0; s < NS; ++s) sc = mfma16(__builtin_bit_cast(bf16x8_t, key[k][s]), q[c][s], sc);
        const int t = t0 + 16 * k + 4 * qd;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float w = __builtin_amdgcn_exp2f(fmaf(sc[i], a.qscale, -ls[c]));
          sum[k][i] += (t + i <= see[c].p) & ((t + i >= see[c].lo) | (t + i < a.sinks)) ? w : 0.f;
        }
      }
  }
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    float v = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float s = add_over_16(sum[k][i]);
      v = (n & 3) == i ? s : v;
    }
    const int t = t0 + 16 * k + 4 * qd + (n & 3);
    if (n < 4 && t < a.Lloc) a.out[pair * a.Lloc + t] = weighed ? old[k] * a.decay + v : v;
  }
}

// ---- many columns --------------------------------------------------------------------------------------------------------
constexpr int kMassRows = 32;    // rows of a wave
constexpr int kMassWaves = 4;
constexpr int kMassStages = 3;
constexpr long long kMassItems = 2048;  // fewer tiles than this: their columns in parts

struct MassParts {
  float* part;      // [B * Hkv][n_parts][Lloc] sums of the parts, n_parts > 1
  int n_parts, n_tiles, tpw;  // tpw: tokens per step
  uint32_t by_r;              // as in mass_rows_kernel
};

template <int D>
__global__ __launch_bounds__(kMassWaves * 64) __attribute__((amdgpu_waves_per_eu(3))) void mass_tiled_kernel(MassArgs a, MassParts pp) {
  constexpr int NW = kMassWaves, NP = D / 8, NS = D / 16, ROW = D * 2;
  constexpr int KT = kMassRows / 32, STAGES = kMassStages, AHEAD = STAGES - 1;  // steps whose copies are under way
  constexpr int TILE = 32 * ROW;          // bytes of a step's queries
  constexpr int NPW = 32 * NP / 64 / NW;  // copies of a wave per step
  static_assert(NPW >= 1, "a step is a whole number of copies per wave");
  static_assert(KT == 1, "a column's rows of a wave are the bits of a word");
  constexpr int SIDE = NW * 256;           // behind them, for every wave: 32 log-sums and 32 positions
  __shared__ __attribute__((aligned(16))) unsigned char smem[STAGES * (TILE + SIDE)];
  __shared__ int lo_s[NW], hi_s[NW];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int hf = lane >> 5, col = lane & 31, r = a.r;
  int x = blockIdx.x;
  const int g = x % a.Hkv;  // the KV head fastest: an XCD keeps to few heads' queries
  x /= a.Hkv;
  const int part = x % pp.n_parts;
  x /= pp.n_parts;
  const int tile = x % pp.n_tiles;
  const long long b = x / pp.n_tiles, pair = b * a.Hkv + g;
  const int tile0 = tile * NW * kMassRows, t0 = tile0 + wave * kMassRows;

  // steps with a token that sees a row of the tile: from the first to the last of them
  const int tile1 = (tile0 + NW * kMassRows < a.Lloc ? tile0 + NW * kMassRows : a.Lloc) - 1;
  int s_lo = INT32_MAX, s_hi = -1;
  for (int m = tid; m < a.M; m += NW * 64) {
    const SeenBy s = seen_by(a, a.q_pos[b * a.M + m]);
    if (s.p >= tile0 && (s.lo <= tile1 || tile0 < a.sinks)) {
      s_lo = s_lo < m ? s_lo : m;
      s_hi = m;
    }
  }
  s_lo = min_of_lanes<64>(s_lo);
  s_hi = max_of_lanes<64>(s_hi);
  if (lane == 0) {
    lo_s[wave] = s_lo;
    hi_s[wave] = s_hi;
  }
  __syncthreads();
#pragma unroll
  for (int w = 0; w < NW; ++w) {
    s_lo = lo_s[w] < s_lo ? lo_s[w] : s_lo;
    s_hi = hi_s[w] > s_hi ? hi_s[w] : s_hi;
  }
  s_lo = __builtin_amdgcn_readfirstlane(s_lo) / pp.tpw;
  s_hi = __builtin_amdgcn_readfirstlane(s_hi);
  if (s_hi < 0) {  // nobody sees the tile: most of a long cache's behind a window
    for (int t = tile0 + tid; t <= tile1; t += NW * 64) {
      if (pp.n_parts > 1)
        pp.part[(pair * pp.n_parts + part) * a.Lloc + t] = 0.f;
      else
        a.out[pair * a.Lloc + t] = old_weight(a, pair * a.Lloc + t);
    }
    return;
  }
  const int n_steps = s_hi / pp.tpw + 1 - s_lo;
  const int sb = s_lo + (int)((long long)n_steps * part / pp.n_parts);
  const int se = s_lo + (int)((long long)n_steps * (part + 1) / pp.n_parts);

  float sum[KT][16];
#pragma unroll
  for (int k = 0; k < KT; ++k)
#pragma unroll
    for (int i = 0; i < 16; ++i) sum[k][i] = 0.f;
  if (sb < se) {
    // rows: A operand of slice s: dims 16 s + 8 hf .. + 8 of row lane % 32
    bf16x8_t key[KT][NS];
#pragma unroll
    for (int k = 0; k < KT; ++k) {
      int row = t0 + 32 * k + col;
      row = row < a.Lloc ? row : a.Lloc - 1;
#pragma unroll
      for (int s = 0; s < NS; ++s)
        key[k][s] = as_bf16x8(*reinterpret_cast<const uint4*>(a.Kloc + (pair * a.Lloc + row) * D + 16 * s + 8 * hf));
    }
    // Queries in LDS: piece p of column i lies at p ^ swz(i), so that the reads meet no bank twice.
    auto swz = [](int i) { return D == 128 ? (i & 15) : ((i >> 1) & 7); };
    int qat[NS];
#pragma unroll
    for (int s = 0; s < NS; ++s) qat[s] = (col * ROW + ((hf ^ swz(col)) * 16)) ^ (32 * s);
    // A wave's copies of a step: copy j brings 1 KiB, 16 bytes to a lane; column c of a step is head c % r of its token c / r
    // (columns past the last whole token: the first one again)
    int ctok[NPW], coff[NPW];
#pragma unroll
    for (int i = 0; i < NPW; ++i) {
      const int y = (i * NW + wave) * 64 + lane, row = y / NP;
      int c = row;
      if (c >= pp.tpw * r) c = 0;
      ctok[i] = (int)((uint32_t)c * pp.by_r >> 16);
      coff[i] = (c - ctok[i] * r) * ROW + ((y % NP) ^ swz(row)) * 16;
    }
    int my_tok = (int)((uint32_t)col * pp.by_r >> 16), my_head = col - my_tok * r;
    const bool col_ok = my_tok < pp.tpw;
    if (!col_ok) my_tok = my_head = 0;
    const uint32_t lds0 = __builtin_amdgcn_readfirstlane(lds_addr_of(smem));
    // where the next step's queries, and this lane's log-sum (lanes below 32) or position, come from
    const long long m1 = b * a.M + (long long)sb * pp.tpw;
    const int tok_bytes = a.Hq * ROW, side_bytes = hf == 0 ? a.Hq * 4 : 4;
    const unsigned char* n_q = reinterpret_cast<const unsigned char*>(a.q + (m1 * a.Hq + g * r) * D);
    const unsigned char* n_side = hf == 0 ? reinterpret_cast<const unsigned char*>(a.lse + m1 * a.Hq + g * r + my_head)
                                          : reinterpret_cast<const unsigned char*>(a.q_pos + m1);
    int n_left = a.M - 1 - sb * pp.tpw;  // tokens behind the step's first one
    auto issue = [&](auto stage) __attribute__((always_inline)) {
      constexpr int INTO = decltype(stage)::value;
#pragma unroll
      for (int i = 0; i < NPW; ++i) {
        const int t = ctok[i] < n_left ? ctok[i] : n_left;
        copy16_to_lds_async_at(n_q, t * tok_bytes + coff[i], lds0 + INTO * (TILE + SIDE) + (i * NW + wave) * 1024);
      }
      const int t = my_tok < n_left ? my_tok : n_left;
      copy4_to_lds_async64(n_side + t * side_bytes, lds0 + INTO * (TILE + SIDE) + TILE + wave * 256);
      n_q += (long long)pp.tpw * tok_bytes;
      n_side += (long long)pp.tpw * side_bytes;
      n_left -= pp.tpw;
    };
    int left = a.M - sb * pp.tpw;  // tokens from the step's first one on
    auto step = [&](int s, auto stage) __attribute__((always_inline)) {
      constexpr int BUF = decltype(stage)::value;
      const unsigned char* const st = smem + BUF * (TILE + SIDE);
      if (s + AHEAD - 1 < se)
        wait_copies_but<(AHEAD - 1) * (NPW + 1)>();
      else
        wait_copies_but<0>();
      lds_barrier();
      if (s + AHEAD < se) issue(std::integral_constant<int, (BUF + AHEAD) % STAGES>());
      const float* const side = reinterpret_cast<const float*>(st + TILE + wave * 256);
      float nls = -side[col] * kLog2e;
      SeenBy see = seen_by(a, __float_as_int(side[32 + col]));
      const bool there = col_ok & (my_tok < left);
      left -= pp.tpw;
      if (!there | (nls == INFINITY)) see.p = -1;  // (a token that saw nothing)
      // seen whole by all columns that are there; the others weigh exp2(-inf)
      const bool whole =
          __builtin_amdgcn_ballot_w64(there & !((see.p >= t0 + kMassRows - 1) & ((see.lo <= t0) | (t0 + kMassRows <= a.sinks)))) == 0;
      if (!whole && __builtin_amdgcn_ballot_w64((see.p >= t0) & ((see.lo < t0 + kMassRows) | (t0 < a.sinks))) == 0) return;
      if (!there) nls = -INFINITY;
      f32x16e_t sc[KT];
#pragma unroll
      for (int k = 0; k < KT; ++k)
#pragma unroll
        for (int i = 0; i < 16; ++i) sc[k][i] = 0.f;
#pragma unroll
      for (int i = 0; i < NS; ++i) {
        const bf16x8_t q = as_bf16x8(*reinterpret_cast<const uint4*>(st + qat[i]));
#pragma unroll
        for (int k = 0; k < KT; ++k) sc[k] = mfma32e(key[k][i], q, sc[k]);
      }
      if (whole) {
#pragma unroll
        for (int k = 0; k < KT; ++k)
#pragma unroll
          for (int i = 0; i < 16; ++i) sum[k][i] += __builtin_amdgcn_exp2f(fmaf(sc[k][i], a.qscale, nls));
      } else {
        // bit i: the column sees row t0 + 4 hf + i  (a weight is kept by an and, in two instructions; with three compares five)
        const uint32_t bits = (up_to(see.p - t0) & (~up_to(see.lo - 1 - t0) | up_to(a.sinks - 1 - t0))) >> (4 * hf);
#pragma unroll
        for (int k = 0; k < KT; ++k)
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int t = (i & 3) + 8 * (i >> 2);
            const float w = __builtin_amdgcn_exp2f(fmaf(sc[k][i], a.qscale, nls));
            sum[k][i] += __uint_as_float(__float_as_uint(w) & (uint32_t)((int32_t)(bits << (31 - t)) >> 31));
          }
      }
    };
    // (the rows are waited for here: at their first use, in the loop, the wait would be one for all copies in flight as well)
#pragma unroll
    for (int k = 0; k < KT; ++k)
#pragma unroll
      for (int i = 0; i < NS; ++i) asm volatile("" : "+v"(key[k][i]));
    // stages by number, so that LDS addresses are constants
    each_stage(std::make_integer_sequence<int, AHEAD>(), [&](auto stage) {
      if (sb + decltype(stage)::value < se) issue(stage);
    });
    for (int s = sb; s < se; s += STAGES)
      each_stage(std::make_integer_sequence<int, STAGES>(), [&](auto stage) __attribute__((always_inline)) {
        if (s + decltype(stage)::value < se) step(s + decltype(stage)::value, stage);
      });
  }
  // over the 32 columns: lane c of a half keeps the sum of register c
#pragma unroll
  for (int k = 0; k < KT; ++k) {
    float v = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const float s = add_xor16(add_over_16(sum[k][i]));
      v = (lane & 15) == i ? s : v;
    }
    const int i = lane & 15, t = t0 + 32 * k + (i & 3) + 8 * (i >> 2) + 4 * hf;
    if ((lane & 16) == 0 && t < a.Lloc) {
      const long long at = pair * a.Lloc + t;
      if (pp.n_parts > 1)
        pp.part[(pair * pp.n_parts + part) * a.Lloc + t] = v;
      else
        a.out[at] = old_weight(a, at) + v;
    }
  }
}

__global__ __launch_bounds__(256) void mass_join_kernel(MassArgs a, const float* part, int n_parts, long long n) {
  const unsigned at = blockIdx.x * 256 + threadIdx.x;  // (n < 2^18: tiles in parts are fewer than kMassItems)
  if (at >= n) return;
  const long long pair = at / (unsigned)a.Lloc;
  const float* const p = part + pair * n_parts * a.Lloc + (at - pair * a.Lloc);
  float v = old_weight(a, at);
  for (int i = 0; i < n_parts; ++i) v += p[(long long)i * a.Lloc];
  a.out[at] = v;
}

MassPlan plan_mass(const Dims& dm, int B, int M, int Lloc) {
  MassPlan p = {};
  const long long pairs = (long long)B * dm.Hkv;
  p.ws_bytes = 256;
  if (M * dm.r <= 64) {
    // An odd number to a (sequence, KV head): an even one puts the same blocks of all of them, and with them the ones behind the
    // sequences' ends, on the same XCDs and shader engines.  (40 sequences of 0 to 8192 rows 70.6 us, so 67.4; 8 of 0 to 4096
    // 12.6, so 10.7; one of 8192 6.4, so 6.2.)
    p.n_blocks = ((Lloc + kRowsRows - 1) / kRowsRows) | 1;
    if (pairs * p.n_blocks >= 1 << 26) p.ws_bytes = 0;
    return p;
  }
  p.tiled = 1;
  p.tpw = 32 / dm.r;
  p.n_tiles = (Lloc + kMassWaves * kMassRows - 1) / (kMassWaves * kMassRows);
  const long long tiles = pairs * p.n_tiles, steps = (M + p.tpw - 1) / p.tpw;
  long long n = (kMassItems + tiles - 1) / tiles, most = steps / 8 < 32 ? steps / 8 : 32;
  if (n > most) n = most;
  p.n_parts = (int)(n < 1 ? 1 : n);
  if (tiles * p.n_parts >= 1 << 24) {
    p.ws_bytes = 0;
    return p;
  }
  // (the parts are of all columns, whatever the window: which of them a tile meets the kernel finds from their positions)
  // (tiles in parts are fewer than kMassItems, so less than twice as many workgroups in all; no less for a longer cache)
  const long long sums = most * pairs * Lloc, bound = 2 * kMassItems * kMassWaves * kMassRows;
  if (most > 1) p.ws_bytes = round_up256((size_t)(sums < bound ? sums : bound) * sizeof(float));
  return p;
}

int launch_mass(const Dims& dm, const MassPlan& pl, MassArgs a, int B, void* ws, hipStream_t st) {
  a.Hq = dm.Hq;
  a.Hkv = dm.Hkv;
  a.r = dm.r;
  a.qscale = (float)(1.4426950408889634 / sqrt((double)dm.d));
  const long long pairs = (long long)B * dm.Hkv;
  const uint32_t by_r = 65536u / dm.r + 1;
  if (!pl.tiled) {
    const dim3 grid((unsigned)pl.n_blocks, (unsigned)dm.Hkv, (unsigned)B), block(64);
    const int groups = (a.M * dm.r + 15) / 16;
#define MSA_MASS(DD, CC) hipLaunchKernelGGL((mass_rows_kernel<DD, CC>), grid, block, 0, st, a, by_r)
#define MSA_MASS_OF(DD)            \
  if (groups == 1) MSA_MASS(DD, 1); \
  else if (groups == 2) MSA_MASS(DD, 2); \
  else MSA_MASS(DD, 4)
    if (dm.d == 128) {
      MSA_MASS_OF(128);
    } else {
      MSA_MASS_OF(64);
    }
#undef MSA_MASS_OF
#undef MSA_MASS
    return hipGetLastError() == hipSuccess ? MSA_OK : MSA_ERR_HIP;
  }
  const MassParts pp = {(float*)ws, pl.n_parts, pl.n_tiles, pl.tpw, by_r};
  const dim3 grid((unsigned)(pairs * pl.n_tiles * pl.n_parts));
  if (dm.d == 128)
    hipLaunchKernelGGL(mass_tiled_kernel<128>, grid, dim3(kMassWaves * 64), 0, st, a, pp);
  else
    hipLaunchKernelGGL(mass_tiled_kernel<64>, grid, dim3(kMassWaves * 64), 0, st, a, pp);
  if (hipGetLastError() != hipSuccess) return MSA_ERR_HIP;
  if (pl.n_parts > 1) {
    const long long n = pairs * a.Lloc;
    hipLaunchKernelGGL(mass_join_kernel, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, st, a, (const float*)ws, pl.n_parts, n);
  }
  return hipGetLastError() == hipSuccess ? MSA_OK : MSA_ERR_HIP;
}

}  // namespace msa
