// msa_pack_kv4, msa_unpack_kv4: a bank's keys and values in four bits.
//
// A row of d elements is d/32 blocks of 32.  A block has one power of two s = 2^(e - 127), held as the byte e, and 32 codes of
// four bits (sign, two bits of exponent, one of mantissa: 0, 0.5, 1, 1.5, 2, 3, 4, 6), the format that gfx950's conversions
// (v_cvt_scalef32_pk_*_fp4) take apart for nothing.  s is the smallest with max|x| <= 7 s: 7 rounds to 6, so that no element
// is off by more than half the step at its place, and all of it is exact arithmetic (a shift of the exponent and one rounding
// to nearest, ties to even), the same on every machine.  e stays in 2 .. 252, where every value is a normal bf16 number;
// beyond 2^125 * 6 values saturate.
//
// Both are streams: 2 bytes read and 0.53 written per element, or the other way round; bound by HBM (2 million rows of 128
// dims, K and V, 1.36 GB: packed in 221 us, 6.2 TB/s, unpacked in 257, 5.3 TB/s).  Rows that are unpacked are stored with the
// streaming hint (262144 rows packed and unpacked 56.8 -> 52.5 us, 64064 rows 18.1 -> 16.4).  A lane takes eight elements (one
// 16-byte access in bf16, 4 bytes of codes); the block's maximum comes from the quad of lanes that share it.
#include "msa_attend.h"

namespace msa {

__device__ __forceinline__ uint32_t quad_max_u(uint32_t x) {
  uint32_t y = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, kDppXor1, 0xf, 0xf, false);
  x = x > y ? x : y;
  y = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, kDppXor2, 0xf, 0xf, false);
  return x > y ? x : y;
}

// The scale byte of a block from the bits of its largest magnitude (fp32): 1.f * 2^x <= 1.75 * 2^(k + 2) decides.
__device__ __forceinline__ int scale_byte(uint32_t amax_bits) {
  int e = (int)(amax_bits >> 23) - 2 + ((amax_bits & 0x7fffffu) > 0x600000u ? 1 : 0);
  return e < 2 ? 2 : (e > 252 ? 252 : e);
}

// Eight elements of a row of a block -> their codes; the quad's first lane writes the block's scale byte.
template <int D, bool STREAM>
__device__ __forceinline__ void pack4_eight(const float (&f)[8], uint8_t* __restrict__ codes, uint8_t* __restrict__ scales,
                                            long long row, int lr) {
  uint32_t amax = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const uint32_t m = __float_as_uint(f[j]) & 0x7fffffffu;
    amax = m > amax ? m : amax;
  }
  const int e = scale_byte(quad_max_u(amax));
  const float s = __uint_as_float((uint32_t)e << 23);
  uint32_t c4 = 0;
  c4 = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c4, f[0], f[1], s, 0);
  c4 = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c4, f[2], f[3], s, 1);
  c4 = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c4, f[4], f[5], s, 2);
  c4 = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c4, f[6], f[7], s, 3);
  uint32_t* const to = reinterpret_cast<uint32_t*>(codes + row * (D / 2) + 4 * lr);
  if (STREAM)
    __builtin_nontemporal_store(c4, to);
  else
    *to = c4;
  if ((lr & 3) == 0) scales[row * (D / 32) + lr / 4] = (uint8_t)e;
}

// ROT: keys that are not position-encoded yet are turned by their position in the document before they are rounded.  The
// angles cost more than the bytes (2 million rows of keys and values, each row with angles of its own 380 us, rows of one
// position in four documents or heads together 236 to 264, nothing turned 221).
// A thread has ROWS rows in flight.  STREAM: 1 streaming loads, 2 streaming stores of the codes as well.
template <int D, bool ROT, int ROWS, int STREAM>
__device__ __forceinline__ void pack4_rows(const uint16_t* __restrict__ X, uint8_t* __restrict__ codes,
                                           uint8_t* __restrict__ scales, const int32_t* __restrict__ lens, int doc_begin,
                                           long long n_rows, int Hkv, int G, const NormTheta& th) {
  constexpr int LPR = D / 8;          // lanes per row
  constexpr int RPB = 256 / LPR;      // rows per workgroup and turn
  const int lr = threadIdx.x % LPR;
  const long long row0 = (long long)doc_begin * Hkv * G;
  const long long turns = ROT ? (n_rows / G + ROWS - 1) / ROWS * G : (n_rows + ROWS - 1) / ROWS;
  for (long long i = (long long)blockIdx.x * RPB + threadIdx.x / LPR; i < (turns + RPB - 1) / RPB * RPB;
       i += (long long)gridDim.x * RPB) {
    // rows of this turn: RPB apart, or, to be turned, of one position in ROWS (document, head) pairs
    const long long r0 = ROT ? i / G * ROWS * G + i % G : i / RPB * (RPB * ROWS) + i % RPB;
    const long long apart = ROT ? G : RPB;
    uint4 x[ROWS];
#pragma unroll
    for (int u = 0; u < ROWS; ++u) {
      const long long r = r0 + u * apart, row = row0 + r;
      bool live = r < n_rows;
      if (live && lens != nullptr) {
        const long long slab = row / G;
        int len = lens[slab / Hkv];
        len = len < 1 ? 1 : (len > G ? G : len);
        live = row - slab * G < len;
      }
      x[u] = make_uint4(0, 0, 0, 0);
      if (live) x[u] = STREAM ? load_stream16(X + row * D + 8 * lr) : *reinterpret_cast<const uint4*>(X + row * D + 8 * lr);
    }
    float2 c[ROT ? 8 : 1];
    const bool second = lr >= LPR / 2;
    if (ROT) {  // a lane works out four of its eight angles, the one that holds the partners the others
      const int p = (int)(i % G), u0 = 8 * (lr & (LPR / 2 - 1));
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float2 m = cis_pos(p, th.th[u0 + j + (second ? 4 : 0)]);
        const float2 o = make_float2(__shfl_xor(m.x, LPR / 2, 64), __shfl_xor(m.y, LPR / 2, 64));
        c[j] = second ? o : m;
        c[j + 4] = second ? m : o;
      }
    }
#pragma unroll
    for (int u = 0; u < ROWS; ++u) {
      const long long r = r0 + u * apart;
      if (r >= n_rows) break;  // the same for the lanes of a row
      const uint32_t w[4] = {x[u].x, x[u].y, x[u].z, x[u].w};
      float f[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) f[j] = j & 1 ? bf16_hi(w[j / 2]) : bf16_lo(w[j / 2]);
      if (ROT) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float o = __shfl_xor(f[j], LPR / 2, 64);
          f[j] = fmaf(f[j], c[j].x, (second ? o : -o) * c[j].y);  // (spelt out: the same bits from every variant)
        }
      }
      pack4_eight<D, (STREAM > 1)>(f, codes, scales, row0 + r, lr);
    }
  }
}

// Keys by the first row of workgroups, values by the second; either may be absent.
template <int D, bool ROT, int ROWS, int STREAM>
__global__ __launch_bounds__(256) void pack4_kernel(Pack4Args a, NormTheta th) {
  const bool values = a.x[0] == nullptr || blockIdx.y == 1;
  if (!values)
    pack4_rows<D, ROT, ROWS, STREAM>(a.x[0], a.codes[0], a.scales[0], a.lens, a.doc_begin, a.n_rows, a.Hkv, a.G, th);
  else
    pack4_rows<D, false, ROWS, STREAM>(a.x[1], a.codes[1], a.scales[1], a.lens, a.doc_begin, a.n_rows, a.Hkv, a.G, th);
}

template <int D>
__global__ __launch_bounds__(256) void unpack4_kernel(Pack4Args a) {
  const int i = a.x[0] == nullptr || blockIdx.y == 1 ? 1 : 0;
  const uint8_t* const codes = a.codes[i];
  const uint8_t* const scales = a.scales[i];
  uint16_t* const X = a.x[i];
  const long long n_rows = a.n_rows, row0 = (long long)a.doc_begin * a.Hkv * a.G;
  constexpr int LPR = D / 8;
  constexpr int RPB = 256 / LPR;
  const int lr = threadIdx.x % LPR;
  for (long long r = (long long)blockIdx.x * RPB + threadIdx.x / LPR; r < n_rows; r += (long long)gridDim.x * RPB) {
    const long long row = row0 + r;
    const uint32_t c4 = *reinterpret_cast<const uint32_t*>(codes + row * (D / 2) + 4 * lr);
    const float s = __uint_as_float((uint32_t)scales[row * (D / 32) + lr / 4] << 23);
    store_stream16(X + row * D + 8 * lr, fp4x8_to_bf16(c4, s));
  }
}

constexpr long long kStreamBytes = 128ll << 20, kStreamCodes = 256ll << 20;

static unsigned stream_blocks(long long n_rows, int rows_per_block) {
  const long long n = (n_rows + rows_per_block - 1) / rows_per_block;
  return (unsigned)(n < 1 ? 1 : (n > 16384 ? 16384 : n));
}

static Pack4Args pack4_args(const Dims& dm, Pack4Args a, int doc_begin, int doc_count) {
  a.lens = dm.lens;
  a.doc_begin = doc_begin;
  a.n_rows = (long long)doc_count * dm.Hkv * dm.G;
  a.Hkv = dm.Hkv;
  a.G = dm.G;
  return a;
}

int launch_pack4(const Dims& dm, Pack4Args x, int doc_begin, int doc_count, bool rotate, hipStream_t st) {
  const Pack4Args a = pack4_args(dm, x, doc_begin, doc_count);
  if (a.n_rows == 0) return MSA_OK;
  NormTheta th = {};
  rotate = rotate && a.x[0] != nullptr;
  if (rotate) {
    const RopeTheta& table = rope_table(dm.base, dm.d);
    for (int u = 0; u < kMaxHalf; ++u) th.th[u] = table.th[u];
  }
  // Two rows to a thread (against one, packed and unpacked: 128000 rows of 128 dims 30.8 -> 28.4 us, 64064 17.1 -> 16.6), from
  // 131072 rows of a tensor on four, which gives fewer waves with more in flight each (against one: 262144 rows 58 -> 53;
  // 64064 rows 17.4 -> 19.0), from 128 MiB on streaming loads (2 million rows 540 -> 504 with both), and streaming stores of
  // codes that the 256 MiB behind the L2s do not hold for the next reader either.  Packed and unpacked with plain stores /
  // streaming ones, 8 heads of 128: 384 documents of 512 rows (204 MiB of codes) 345 / 348, 448 (238) 384 / 414, 480 (255)
  // 423 / 444, 496 (264) 463 / 459, 512 (272) 495 / 475, 640 (340) 635 / 611; 64 dims: 960 documents (255) 409 / 442, 1024
  // (272) 500 / 475.  (Packing alone gains from 192 documents on, 88 / 82, 512 245 / 221, but what is packed is read.)  Keys to
  // be turned have four rows to a thread at any size, which share their angles (one row to a thread, 64064 rows of keys and
  // values 15.4 us for 13.4).
  const int n_tensors = a.x[0] != nullptr && a.x[1] != nullptr ? 2 : 1;
  const bool many = rotate || a.n_rows >= 131072;
  const long long bytes = a.n_rows * dm.d * 2 * n_tensors, codes = a.n_rows * (dm.d / 2 + dm.d / 32) * n_tensors;
  const dim3 grid(stream_blocks(a.n_rows, 256 / (dm.d / 8) * (many ? 4 : 2)), n_tensors);
#define MSA_PACK4(DD, RR, ROWS, SS) hipLaunchKernelGGL((pack4_kernel<DD, RR, ROWS, SS>), grid, dim3(256), 0, st, a, th)
#define MSA_PACK4_MANY(DD, RR)                                 \
  do {                                                         \
    if (bytes < kStreamBytes) MSA_PACK4(DD, RR, 4, 0);         \
    else if (codes < kStreamCodes) MSA_PACK4(DD, RR, 4, 1);    \
    else MSA_PACK4(DD, RR, 4, 2);                              \
  } while (0)
  if (dm.d == 128) {
    if (rotate) MSA_PACK4_MANY(128, true);
    else if (many) MSA_PACK4_MANY(128, false);
    else MSA_PACK4(128, false, 2, 0);
  } else {
    if (rotate) MSA_PACK4_MANY(64, true);
    else if (many) MSA_PACK4_MANY(64, false);
    else MSA_PACK4(64, false, 2, 0);
  }
#undef MSA_PACK4_MANY
#undef MSA_PACK4
  return hipGetLastError() == hipSuccess ? MSA_OK : MSA_ERR_HIP;
}

int launch_unpack4(const Dims& dm, Pack4Args x, int doc_begin, int doc_count, hipStream_t st) {
  const Pack4Args a = pack4_args(dm, x, doc_begin, doc_count);
  if (a.n_rows == 0) return MSA_OK;
  const dim3 grid(stream_blocks(a.n_rows, 256 / (dm.d / 8)), a.x[0] != nullptr && a.x[1] != nullptr ? 2 : 1);
  if (dm.d == 128)
    hipLaunchKernelGGL(unpack4_kernel<128>, grid, dim3(256), 0, st, a);
  else
    hipLaunchKernelGGL(unpack4_kernel<64>, grid, dim3(256), 0, st, a);
  return hipGetLastError() == hipSuccess ? MSA_OK : MSA_ERR_HIP;
}

}  // namespace msa
