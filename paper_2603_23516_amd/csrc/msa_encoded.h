// Attention over position-encoded keys (as msa_norm_rotate writes them): what msa_window_attend and msa_sparse_attend4 share.
// A kernel for single tokens (msa_encoded_decode.hip) and a tiled one for many tokens that share keys
// (msa_encoded_tiled.hip).
#pragma once
#include "msa_attend.h"

namespace msa {

struct EncodedArgs {
  const uint16_t* q;       // [BM][Hq][D]
  const uint8_t *K4, *K4s, *V4, *V4s;  // bank in four bits, or null: the local cache alone
  const int32_t* idx;      // [BM or B][Hkv or 1][k]
  const int32_t* lens;     // [N] or null
  const uint16_t *Kloc, *Vloc;  // [B][Hkv][Lloc][D]
  const int32_t* q_pos;    // [BM]
  uint16_t* out;           // [BM][Hq][D]
  float* lse;              // [BM][Hq] or null
  float* part_o;           // [BM][Hq][n_splits][D] unnormalised partial outputs, where n_splits > 1
  float2* part_ml;         // [BM][Hq][n_splits]    (running max in log2 units, sum); tiled kernel with tickets: both by workgroup,
                           // as registers hold them
  unsigned long long* tickets;  // arrival counters, one per (token, KV head) or, of two parts, (tile, KV head); null: a launch
                                // joins the parts
  unsigned long long nonce;
  int M, Hq, Hkv, r, G, k, N, Lloc, pos0, window, sinks;
  int idx_sel, idx_rows_per_b, n_splits;
  float qscale;            // log2(e) / sqrt(d)
};

struct TiledArgs {
  uint16_t *Kx, *Vx;  // [B][Hkv][mem_cap][D] rows of the selected documents in bf16, or null
  int* mem_rows;      // [B][Hkv] how many there are
  int mem_cap;        // k G
  int tpw, n_tiles;   // tokens per wave, tiles per sequence
};

struct EncodedPlan {
  int tiled;           // 1: encoded_tiled_kernel, 0: encoded_decode_kernel
  int n_splits, tpw, n_tiles;
  size_t off_ml, off_tickets;           // partials first, then their (max, sum), then the arrival counters
  size_t off_kx, off_vx, off_mem_rows;  // tiled, bank in four bits
  size_t ws_bytes;
};
// mem_rows: k G, 0 without a bank; shared: the tokens of a sequence have their bank rows in common; local_rows: rows of the
// cache that a token can see.  ws_bytes is 0 where the grid does not hold the call: one workgroup per token in its third
// dimension, or tiles in its first, whose threads count to 2^32.
EncodedPlan plan_encoded(const Dims& dm, int B, int M, long long mem_rows, bool shared, long long local_rows, int Lloc);
int launch_encoded(const Dims& dm, const EncodedPlan& pl, EncodedArgs a, int B, void* ws, hipStream_t st);
int launch_encoded_tiled(const Dims& dm, const EncodedArgs& a, TiledArgs ta, int B, hipStream_t st);

// The rows of a selection numbered through, by the 64 lanes of one wave: pre[j] rows lie in front of slot j's document, which
// lane j gets back, `before` with pre[lane]; pads, ids outside the bank and rows past a document's end are left out.  pre has
// MSA_MAX_TOPK + 1 entries.
__device__ __forceinline__ int number_rows(const EncodedArgs& a, int b, long long bm, int g, int lane, int* pre, int& before) {
  int doc = -1, len = 0;
  if (lane < a.k) {
    doc = a.idx[((a.idx_rows_per_b == 1 ? b : bm) * a.idx_sel + (a.idx_sel == 1 ? 0 : g)) * a.k + lane];
    if (doc >= 0 && doc < a.N) {
      len = a.G;
      if (a.lens != nullptr) {
        len = a.lens[doc];
        len = len < 1 ? 1 : (len > a.G ? a.G : len);
      }
    }
  }
  int sum = len;
#pragma unroll
  for (int off = 1; off < 64; off *= 2) {
    const int up = __shfl_up(sum, off, 64);
    if (lane >= off) sum += up;
  }
  pre[lane + 1] = sum;
  if (lane == 0) pre[0] = 0;
  before = sum - len;
  return doc;
}

// Rows of the local cache that a token at position p (counted from the cache's first row) sees: [0, first) and [from, to).
struct Seen {
  int first, from, to;
};
__host__ __device__ __forceinline__ Seen seen_rows(long long p, int Lloc, int window, int sinks) {
  Seen s;
  s.to = p < 0 ? 0 : (p + 1 < Lloc ? (int)(p + 1) : Lloc);
  const long long lo = p - window + 1;
  s.from = lo < 0 ? 0 : (lo < s.to ? (int)lo : s.to);
  s.first = sinks < s.from ? sinks : s.from;
  if (s.first == s.from) s.first = s.from = 0;  // they meet: one run
  return s;
}

}  // namespace msa
