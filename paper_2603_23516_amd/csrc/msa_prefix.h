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
};
struct PrefixPlan {
  size_t ws_bytes;
};
PrefixPlan plan_prefix(const Dims& dm, int B, int M, int Lpre, int Lloc);
int launch_prefix(const Dims& dm, const PrefixPlan& pl, PrefixArgs a, void* ws, hipStream_t st);

}  // namespace msa
