// msa_evict: of every (sequence, KV head) the rows of the cache that weigh most, the first ones and the last ones, moved together.
//
// Two launches.  evict_select_kernel, a workgroup to a (sequence, KV head), finds the weight of the lightest row that stays (as an
// integer of the same order, in digits of up to 11 bits from the top, each by counting), then lists the rows that stay in
// ascending order and moves their weights.  Counted in LDS, where the order of additions changes nothing.  evict_move_kernel copies
// the rows of K and V, 64 to a workgroup.
//
// The copy is bound by memory (32 sequences of 8 heads of 128 cut to 4096 rows, 830 MB in and out, 149 us, 5.6 TB/s), the choice by
// what follows on what in one workgroup: 16384 rows 16 us, of which the first loads 5, a digit 2.6 and the listing 5 (bit by bit with
// the weights in registers 35, with the weights read for every bit 118; digits of all 32 bits 20).
#include "msa_device.h"
#include "msa_host.h"

namespace msa {

constexpr int kSelectThreads = 1024;
constexpr int kBins = 2048;  // values of a digit, two to a thread
constexpr int kListed = 64;  // a lane to each
static_assert(kListed * 2 <= kBins, "a list in the counters' memory");
static_assert(kBins == 2 * kSelectThreads, "two bins to a thread");

// The order of weights as an integer: what is no number comes last, the zeros are equal.
__device__ __forceinline__ uint32_t weight_key(float x) {
  if (x != x) return 0u;
  return orderable(x == 0.f ? 0.f : x);
}

// REGS: rows of a thread, held in registers, of at most 1024 REGS in all; 0: any number, read again for every digit (20000 rows 35 us
// for 23, 32768 58 for 33).
template <int REGS>
__global__ __launch_bounds__(kSelectThreads) void evict_select_kernel(EvictArgs a) {
  constexpr int WAVES = kSelectThreads / 64;
  __shared__ int cnt_s[2][WAVES], found[3], listed;
  __shared__ uint32_t ends_s[2][WAVES];
  __shared__ __attribute__((aligned(8))) int bins[kBins];
  uint2* const list = reinterpret_cast<uint2*>(bins);
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const long long pair = blockIdx.x;
  int n = a.lens[blockIdx.x / (unsigned)a.Hkv];
  n = n < 0 ? 0 : (n > a.Lloc ? a.Lloc : n);
  const float* const mass = a.mass + pair * a.Lloc;
  float* const mass_out = a.mass_out + pair * a.Lout;
  int32_t* const rows = a.rows + pair * a.keep;
  if (n <= a.keep) {
    for (int i = tid; i < a.keep; i += kSelectThreads) {
      rows[i] = i < n ? i : -1;
      if (i < n && mass_out != mass) mass_out[i] = mass[i];
    }
    for (int i = n + tid; i < a.Lout; i += kSelectThreads) mass_out[i] = 0.f;
    return;
  }
  const int m0 = a.sinks, m1 = n - a.recent, need = a.keep - a.sinks - a.recent;  // of rows m0 .. m1 - 1, need < m1 - m0 stay
  int turn = 0;
  auto total = [&](int of_wave, int& before) {  // the same in a wave's lanes; the workgroup's sum, and that of the waves before
    int* const c = cnt_s[turn ^= 1];            // (the other one may still be read)
    if (lane == 0) c[wave] = of_wave;
    __syncthreads();
    int sum = 0;
    before = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
      if (w == wave) before = sum;
      sum += c[w];
    }
    return sum;
  };
  static_assert(REGS <= 32, "a bit per row");
  // a wave's rows are `blocks` times 64 in a row, from w0 on; without registers the workgroup's are taken 1024 at a time
  const int blocks = (n + kSelectThreads - 1) / kSelectThreads;
  int w0 = wave * blocks * 64 + lane;
  // Beside the weights their order and whether a row is in the middle: of up to 16 rows kept as well; of 32 worked out again where it is
  // wanted, from the weights and a bit per row (kept, they went to scratch memory: 16 x 8 heads of 32768 rows 45 us for 35).
  constexpr bool KEPT = REGS <= 16;
  float x[REGS > 0 ? REGS : 1];
  uint32_t keys[KEPT && REGS > 0 ? REGS : 1], inner = 0u;
  if constexpr (REGS > 0) {
#pragma unroll
    for (int u = 0; u < REGS; ++u) x[u] = u < blocks && w0 + 64 * u < n ? mass[w0 + 64 * u] : 0.f;
#pragma unroll
    for (int u = 0; u < REGS; ++u) {
      if constexpr (KEPT)
        keys[u] = weight_key(x[u]);
      else
        inner |= u < blocks && w0 + 64 * u >= m0 && w0 + 64 * u < m1 ? 1u << u : 0u;
    }
  }
  auto again = [&](auto& v) {  // (what follows from v is not kept from here on)
    if constexpr (!KEPT) asm volatile("" : "+v"(v));
  };
  auto key = [&](int u) {
    if constexpr (KEPT) return keys[u];
    again(x[u]);
    return weight_key(x[u]);
  };
  auto in_middle = [&](int u) -> bool {
    if constexpr (KEPT) return w0 + 64 * u >= m0 && w0 + 64 * u < m1;  // (of rows that are its own)
    return (inner >> u) & 1u;
  };
  auto each = [&](auto f) {  // the weights of this thread's rows in the middle
    if constexpr (REGS > 0) {
      again(inner);
      again(w0);
#pragma unroll
      for (int u = 0; u < REGS; ++u) {
        const int i = w0 + 64 * u;
        if constexpr (KEPT) {  // (as a condition and not a value: 22 us for 23 over 16384 rows)
          if (u < blocks && i >= m0 && i < m1) f(keys[u], i);
        } else {
          if (in_middle(u)) f(key(u), i);
        }
      }
    } else {
      for (int i = m0 + tid; i < m1; i += kSelectThreads) f(weight_key(mass[i]), i);
    }
  };
  uint32_t lo = UINT32_MAX, hi = 0u;
  each([&](uint32_t k, int) {
    lo = k < lo ? k : lo;
    hi = k > hi ? k : hi;
  });
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) {
    const uint32_t u = __shfl_xor(lo, off, 64), v = __shfl_xor(hi, off, 64);
    lo = u < lo ? u : lo;
    hi = v > hi ? v : hi;
  }
  if (lane == 0) {
    ends_s[0][wave] = lo;
    ends_s[1][wave] = hi;
  }
  __syncthreads();
#pragma unroll
  for (int w = 0; w < WAVES; ++w) {
    lo = ends_s[0][w] < lo ? ends_s[0][w] : lo;
    hi = ends_s[1][w] > hi ? ends_s[1][w] : hi;
  }
  // Digit by digit from the top of what the weights (less the least of them) span: the rows that agree with kth so far, counted by
  // their next digit; the lightest row that stays has the largest digit from which on there are as many as are wanted.  (Digits of
  // the span and not of 32 bits: weights within a few octaves are in many counters then, and lanes of a wave seldom in the same.)
  const int span = hi > lo ? 32 - __clz(hi - lo) : 1;
  uint32_t kth = 0u;  // less lo.  Rows heavier than kth stay, and of those that weigh kth the first `ties`
  int ties = need, tie_row = -1;  // ... or those up to tie_row
  for (int bits = span < 11 ? span : 11, shift = span - bits; need > 0;) {
    const uint32_t mask = (1u << bits) - 1u, above = shift + bits >= span ? 0u : ~0u << (shift + bits);
    *reinterpret_cast<int2*>(&bins[2 * tid]) = make_int2(0, 0);
    if (tid == 0) listed = 0;
    __syncthreads();
    each([&](uint32_t k, int) {
      k -= lo;
      if (((k ^ kth) & above) == 0u) atomicAdd(&bins[(k >> shift) & mask], 1);
    });
    __syncthreads();
    const int top = kBins - 1 - 2 * tid;  // this thread's two digits: top and the one below
    const int2 two = *reinterpret_cast<const int2*>(&bins[top - 1]);
    int upto = two.x + two.y;
#pragma unroll
    for (int off = 1; off < 64; off *= 2) {
      const int v = __shfl_up(upto, off, 64);
      if (lane >= off) upto += v;
    }
    int before;
    total(__builtin_amdgcn_readlane(upto, 63), before);
    upto += before;  // rows of these two digits and all larger ones
    const int over = upto - two.x - two.y;
    if (over < ties && upto >= ties) {  // one thread's, since 0 < ties <= all that were counted
      const bool lower = over + two.y < ties;
      found[0] = lower ? top - 1 : top;
      found[1] = ties - over - (lower ? two.y : 0);
      found[2] = lower ? two.x : two.y;
    }
    __syncthreads();
    kth |= (uint32_t)found[0] << shift;
    ties = found[1];
    const int agree = found[2];
    if (ties == agree) {  // all that agree so far stay: those from kth on, which is not 0, since some row goes
      --kth;
      ties = 0;
      break;
    }
    if (shift == 0) break;
    if (agree <= kListed) {  // few: each is compared with all of them (the counters' memory is free for the list)
      const uint32_t agreed = ~0u << shift;
      each([&](uint32_t k, int i) {
        k -= lo;
        if (((k ^ kth) & agreed) == 0u) list[atomicAdd(&listed, 1)] = make_uint2(k, (uint32_t)i);
      });
      __syncthreads();
      const uint2 other = list[lane < agree ? lane : 0];
      for (int c = wave; c < agree; c += WAVES) {  // a wave to each of them
        const uint2 mine = list[c];
        const bool better = lane < agree && (other.x > mine.x || (other.x == mine.x && other.y < mine.y));
        if (__popcll(__ballot(better)) == ties - 1 && lane == 0) {
          found[1] = (int)mine.x;
          found[2] = (int)mine.y;
        }
      }
      __syncthreads();
      kth = (uint32_t)found[1];
      tie_row = found[2];
      ties = 0;
      break;
    }
    bits = shift < 11 ? shift : 11;
    shift -= bits;
  }
  kth = need > 0 ? kth + lo : UINT32_MAX;
  int tied_before = 0;
  if constexpr (REGS > 0) {
    if (ties > 0) {
      int c = 0;
      again(inner);
#pragma unroll
      for (int u = 0; u < REGS; ++u)
        if (u < blocks) c += __popcll(__ballot(in_middle(u) && key(u) == kth));
      total(c, tied_before);
    }
    uint32_t kept = 0u;  // bit u: row w0 + 64 u stays
    int c = 0, at;
    again(inner);
    again(w0);
#pragma unroll
    for (int u = 0; u < REGS; ++u) {
      if (u >= blocks) continue;
      const int i = w0 + 64 * u;
      const bool middle = in_middle(u);
      const uint32_t k = key(u);
      bool stays = i < n && (!middle || k > kth || (k == kth && i <= tie_row));
      if (ties > 0) {
        const unsigned long long tie = __ballot(middle && k == kth);
        stays |= middle && k == kth && tied_before + __popcll(tie & ((1ull << lane) - 1ull)) < ties;
        tied_before += __popcll(tie);
      }
      kept |= stays ? 1u << u : 0u;
      c += __popcll(__ballot(stays));
    }
    total(c, at);  // (behind its barrier every weight is in a register)
    again(w0);
#pragma unroll
    for (int u = 0; u < REGS; ++u) {
      if (u >= blocks) continue;
      const bool stays = (kept >> u) & 1u;
      const unsigned long long all = __ballot(stays);
      if (stays) {
        const int to = at + __popcll(all & ((1ull << lane) - 1ull));
        rows[to] = w0 + 64 * u;
        mass_out[to] = x[u];
      }
      at += __popcll(all);
    }
  } else {
    int at = 0;
    for (int i0 = 0; i0 < n; i0 += kSelectThreads) {
      const int i = i0 + tid;
      const float w = mass[i < n ? i : n - 1];
      const uint32_t k = weight_key(w);
      const bool middle = i >= m0 && i < m1;
      const unsigned long long tie = __ballot(middle && k == kth);
      int t0, k0;
      const int tied = total(__popcll(tie), t0);  // (behind its barrier every weight of this turn is in a register)
      const bool stays = i < n && (!middle || k > kth || (k == kth && i <= tie_row) || (k == kth && tied_before + t0 + __popcll(tie & ((1ull << lane) - 1ull)) < ties));
      const unsigned long long kept = __ballot(stays);
      const int all = total(__popcll(kept), k0);
      if (stays) {
        const int to = at + k0 + __popcll(kept & ((1ull << lane) - 1ull));  // to <= i
        rows[to] = i;
        mass_out[to] = w;
      }
      at += all;
      tied_before += tied;
    }
  }
  for (int i = a.keep + tid; i < a.Lout; i += kSelectThreads) mass_out[i] = 0.f;
}

template <int D>
__global__ __launch_bounds__(256) void evict_move_kernel(EvictArgs a, int chunks) {
  constexpr int LPR = D / 8, RPB = 256 / LPR, TURNS = 4;
  const int chunk = (int)(blockIdx.x % (unsigned)chunks);
  const long long pair = blockIdx.x / (unsigned)chunks;
  const int lr = threadIdx.x % LPR, j0 = chunk * (RPB * TURNS) + threadIdx.x / LPR;
  const int32_t* const rows = a.rows + pair * a.keep;
  const uint16_t* const src = (blockIdx.y == 0 ? a.K : a.V) + pair * a.Lloc * D + 8 * lr;
  uint16_t* const dst = (blockIdx.y == 0 ? a.Kout : a.Vout) + pair * a.Lout * D + 8 * lr;
  int row[TURNS];
#pragma unroll
  for (int t = 0; t < TURNS; ++t) row[t] = j0 + t * RPB < a.keep ? rows[j0 + t * RPB] : -1;
  uint4 v[TURNS];
#pragma unroll
  for (int t = 0; t < TURNS; ++t)
    if (row[t] >= 0) v[t] = load_stream16(src + (long long)row[t] * D);
#pragma unroll
  for (int t = 0; t < TURNS; ++t)
    if (row[t] >= 0) store_stream16(dst + (long long)(j0 + t * RPB) * D, v[t]);
}

// In place: a workgroup has 64 bytes of every row of a (sequence, KV head), so that no other one's rows are in its way.  Row j comes
// from row rows[j] >= j: a turn's rows are all in registers before the first of them is stored, and what later turns read lies
// behind what this one stores.  (32 sequences of 8 heads of 128, 4224 rows cut to 4096, 1.07 GB in and out, 259 us, 4.1 TB/s, where
// the kernel above takes 177; of 2112 to 4224 rows 28; one sequence of 16384 cut to 4096 13.5, for 5.5.  The rows as uint4 in an array
// went to 64 KiB of LDS: 273, 39, 18.)
template <int D>
__global__ __launch_bounds__(1024) void evict_move_in_place_kernel(EvictArgs a) {
  constexpr int LPR = 4, RPB = 1024 / LPR, TURNS = 4, SLICES = D * 2 / 64;
  const int slice = blockIdx.x % SLICES;
  const long long pair = blockIdx.x / SLICES;
  const int lr = threadIdx.x % LPR, jt = threadIdx.x / LPR;
  const int32_t* const rows = a.rows + pair * a.keep;
  uint16_t* const x = (blockIdx.y == 0 ? a.Kout : a.Vout) + pair * a.Lloc * D + slice * 32 + 8 * lr;
  for (int j0 = 0; j0 < a.keep; j0 += RPB * TURNS) {
    int row[TURNS];
#pragma unroll
    for (int t = 0; t < TURNS; ++t) {
      const int j = j0 + t * RPB + jt;
      row[t] = j < a.keep ? rows[j] : -1;
      if (row[t] == j) row[t] = -1;  // stays where it is
    }
    u32x4_t v[TURNS];
#pragma unroll
    for (int t = 0; t < TURNS; ++t)
      if (row[t] >= 0) v[t] = *reinterpret_cast<const u32x4_t*>(x + (long long)row[t] * D);
    wait_stores_done();  // (the loads too)
    __syncthreads();
#pragma unroll
    for (int t = 0; t < TURNS; ++t)
      if (row[t] >= 0) *reinterpret_cast<u32x4_t*>(x + (long long)(j0 + t * RPB + jt) * D) = v[t];
  }
}

int launch_evict(const Dims& dm, const EvictArgs& a, int B, hipStream_t st) {
  const unsigned pairs = (unsigned)B * dm.Hkv;
  if (a.Lloc <= 8 * kSelectThreads)
    hipLaunchKernelGGL(evict_select_kernel<8>, dim3(pairs), dim3(kSelectThreads), 0, st, a);
  else if (a.Lloc <= 16 * kSelectThreads)
    hipLaunchKernelGGL(evict_select_kernel<16>, dim3(pairs), dim3(kSelectThreads), 0, st, a);
  else if (a.Lloc <= 32 * kSelectThreads)
    hipLaunchKernelGGL(evict_select_kernel<32>, dim3(pairs), dim3(kSelectThreads), 0, st, a);
  else
    hipLaunchKernelGGL(evict_select_kernel<0>, dim3(pairs), dim3(kSelectThreads), 0, st, a);
  if (hipGetLastError() != hipSuccess) return MSA_ERR_HIP;
  if (a.Kout == a.K) {
    if (dm.d == 128)
      hipLaunchKernelGGL(evict_move_in_place_kernel<128>, dim3(pairs * 4, 2), dim3(1024), 0, st, a);
    else
      hipLaunchKernelGGL(evict_move_in_place_kernel<64>, dim3(pairs * 2, 2), dim3(1024), 0, st, a);
  } else {
    const int chunk = 4 * 256 / (dm.d / 8), chunks = (a.keep + chunk - 1) / chunk;
    if (dm.d == 128)
      hipLaunchKernelGGL(evict_move_kernel<128>, dim3(pairs * chunks, 2), dim3(256), 0, st, a, chunks);
    else
      hipLaunchKernelGGL(evict_move_kernel<64>, dim3(pairs * chunks, 2), dim3(256), 0, st, a, chunks);
  }
  return hipGetLastError() == hipSuccess ? MSA_OK : MSA_ERR_HIP;
}

}  // namespace msa
