// Host-side sanitizer driver of the entry points around the life of a local cache, like encoded_sanitize.cpp: CPU only, no device
// visible, so that a valid request comes back as MSA_ERR_HIP from its launch and everything before it -- validation, work plans,
// workspace sizes -- runs under the address, undefined-behaviour and integer sanitizers.
#include <cstdint>
#include <cstdio>
#include <cstdlib>

#include "msa.h"

static int fails = 0;
#define CHECK(cond)                                              \
  do {                                                           \
    if (!(cond)) {                                               \
      std::printf("FAILED %s:%d: %s\n", __FILE__, __LINE__, #cond); \
      ++fails;                                                   \
    }                                                            \
  } while (0)

static msa_config_t cfg(int32_t Hq, int32_t Hkv, int32_t d) {
  msa_config_t c{};
  c.n_docs = c.doc_len = c.chunk = 1;
  c.n_q_heads = Hq; c.n_kv_heads = Hkv; c.head_dim = d;
  c.rope_base = 1e6f; c.sim = MSA_SIM_COS; c.select_scope = MSA_SCOPE_GROUP;
  return c;
}

int main() {
  setenv("HIP_VISIBLE_DEVICES", "-1", 1);
  setenv("ROCR_VISIBLE_DEVICES", "", 1);
  void* p = reinterpret_cast<void*>(0x10000);
  void* o = reinterpret_cast<void*>(0x20000);
  int32_t* ip = reinterpret_cast<int32_t*>(p);
  float *fp = reinterpret_cast<float*>(p), *fo = reinterpret_cast<float*>(o);
  const size_t big = ~(size_t)0 >> 1;
  const int32_t heads[][2] = {{1, 1}, {8, 1}, {24, 8}, {32, 8}, {64, 64}, {8192, 1024}, {65535, 65535}};
  const int32_t BMs[][2] = {{1, 1}, {1, 4}, {8, 1}, {3, 7}, {65535, 1}, {65536, 1}, {8191, 8}, {65535, 8}, {1 << 22, 8},
                            {1, 31}, {1, 32}, {65535, 32}, {1 << 20, 32}, {1, 1 << 25}, {1, (1 << 25) + 1}, {0x7fffffff, 0x7fffffff}};
  const int32_t lengths[] = {0, 1, 33, 4096, 1 << 24, 1 << 28, (1 << 28) + 1, 0x7fffffff};
  int runs = 0, refused = 0;
  for (auto& h : heads)
    for (int d : {64, 128}) {
      const msa_config_t c = cfg(h[0], h[1], d);
      int32_t axes[64] = {};
      for (auto& bm : BMs) {
        for (int32_t P : lengths)
          for (int32_t L : lengths) {
            const size_t ws = msa_prefix_attend_workspace_bytes(&c, bm[0], bm[1], P, L);
            auto status = [&](size_t bytes) {
              return msa_prefix_attend(&c, p, bm[0], bm[1], p, p, P, ip, p, p, L, 0x7fffffff, ip, o, fo, p, bytes, nullptr);
            };
            const int rc = status(big);
            CHECK(rc == (ws != 0 ? MSA_ERR_HIP : P == 0 && L == 0 ? MSA_ERR_INVALID_ARG : MSA_ERR_UNSUPPORTED));
            if (ws != 0) CHECK(ws >= 256 && ws % 256 == 0 && status(ws) == MSA_ERR_HIP && status(ws - 1) == MSA_ERR_WORKSPACE);
            ++(ws != 0 ? runs : refused);
          }
        for (int32_t L : lengths)
          for (int32_t W : {1, 1000, 0x7fffffff})
            for (int32_t S : {0, 0x7fffffff}) {
              const size_t ws = msa_attend_mass_workspace_bytes(&c, bm[0], bm[1], L, W, S);
              auto status = [&](size_t bytes) {
                return msa_attend_mass(&c, p, bm[0], bm[1], p, L, 0x7fffffff, W, S, ip, fp, fp, 0.5f, fo, p, bytes, nullptr);
              };
              const int rc = status(big);
              CHECK(rc == (ws != 0 ? MSA_ERR_HIP : L == 0 ? MSA_ERR_INVALID_ARG : MSA_ERR_UNSUPPORTED));
              if (ws != 0) CHECK(ws >= 256 && ws % 256 == 0 && status(ws) == MSA_ERR_HIP && status(ws - 1) == MSA_ERR_WORKSPACE);
              ++(ws != 0 ? runs : refused);
            }
        const int rc = msa_norm_rotate_axes(&c, p, (int64_t)h[0] * d, p, (int64_t)h[1] * d, p, (int64_t)1 << 40, p, p, 1e-6f, 1, ip, 4,
                                            axes, ip, bm[0], bm[1], o, o, o, 1 << 20, 1 << 30, nullptr);
        CHECK(rc == ((int64_t)bm[0] * bm[1] <= 1 << 25 ? MSA_ERR_HIP : MSA_ERR_UNSUPPORTED));
      }
      for (int32_t B : {1, 7, 64, 65535, 65536, 0x7fffffff})
        for (int32_t L : {1, 8192, 16385, 32769, 1 << 28, (1 << 28) + 1, 0x7fffffff})
          for (int32_t keep : {1, 100, 1 << 20, 1 << 28}) {
            const bool fits = (int64_t)B * h[1] <= 1 << 16 && L <= 1 << 28 && (int64_t)B * h[1] * keep <= 1 << 29;
            CHECK(msa_evict(&c, p, p, fp, ip, B, L, keep, keep / 2, keep - keep / 2, o, o, fo, keep, ip, nullptr) ==
                  (fits ? MSA_ERR_HIP : MSA_ERR_UNSUPPORTED));
            if (keep <= L && L <= 1 << 28)
              CHECK(msa_evict(&c, p, p, fp, ip, B, L, keep, 0, 0, p, p, fp, L, ip, nullptr) == (fits ? MSA_ERR_HIP : MSA_ERR_UNSUPPORTED));
            CHECK(msa_evict(&c, p, p, fp, ip, B, L, keep, 0x7fffffff, 0x7fffffff, o, o, fo, keep, ip, nullptr) == MSA_ERR_INVALID_ARG);
          }
    }
  std::printf("%d run, %d refused\n", runs, refused);
  if (fails == 0 && runs > 0 && refused > 0) std::printf("cache_sanitize: ok\n");
  return fails != 0;
}
