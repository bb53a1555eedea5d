// Attention of a batch over a prefix that its sequences share and over their own local caches (msa_prefix.hip).
#pragma once
#include "msa_encoded.h"

namespace msa {

struct PrefixArgs {
  const uint16_t* q;            // [BM][Hq][D]
  const uint16_t *Kpre, *Vpre;  // [Hkv][Lpre][D]
  const int32_t* pre_lens;      // [B] or null: all of Lpre
  const uint16_t *Kloc, *Vloc;  // [B][Hkv][Lloc][D]
  const int32_t* q_pos;         // [BM]
  uint16_t* out;                // [BM][Hq][D]
  float* lse;                   // [BM][Hq] or null
  int B, M, Hq, Hkv, r, Lpre, Lloc, pos0;
  float qscale;                 // log2(e) / sqrt(d)
  // tokens of all sequences together over the prefix: tiles of 4 tpw tokens, their rows in n_pre parts
  int tpw, n_pre, pre_groups;   // pre_groups: workgroups of this kind
  // tokens of a sequence over its cache: groups of tpl tokens, n_loc parts
  int tpl, groups, n_loc;
  float *pre_o, *loc_o;         // [BM][Hq][parts][D] unnormalised partial outputs
  float2 *pre_ml, *loc_ml;      // [BM][Hq][parts]    (running max in log2 units, sum)
};
struct PrefixPlan {
  int tiled;                    // 1: encoded_tiled_kernel, a sequence's tokens in tiles of their own
  EncodedPlan tiles;
  int n_pre, n_loc;
  size_t off_pre_ml, off_loc_o, off_loc_ml;  // partials over the prefix first
  size_t ws_bytes;
};
PrefixPlan plan_prefix(const Dims& dm, int B, int M, int Lpre, int Lloc);
int launch_prefix(const Dims& dm, const PrefixPlan& pl, PrefixArgs a, void* ws, hipStream_t st);

}  // namespace msa
