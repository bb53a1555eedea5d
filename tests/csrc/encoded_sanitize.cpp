// Host-side sanitizer driver of the entry points around the local cache and the bank in four bits, like boundary_sanitize.cpp: CPU only,
// no device visible, so that a valid request comes back as MSA_ERR_HIP from its launch and everything before it -- validation,
// work plans, workspace sizes -- runs under the address, undefined-behaviour and integer sanitizers.
#include <cmath>
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

static msa_config_t cfg(int32_t N, int32_t G, int32_t Hq, int32_t Hkv, int32_t d) {
  msa_config_t c{};
  c.n_docs = N; c.doc_len = G; c.chunk = 1; c.n_q_heads = Hq; c.n_kv_heads = Hkv; c.head_dim = d;
  c.rope_base = 1e6f; c.sim = MSA_SIM_COS; c.select_scope = MSA_SCOPE_GROUP;
  return c;
}

int main() {
  setenv("HIP_VISIBLE_DEVICES", "-1", 1);
  setenv("ROCR_VISIBLE_DEVICES", "", 1);
  void* p = reinterpret_cast<void*>(0x10000);
  const int32_t* ip = reinterpret_cast<const int32_t*>(p);
  float* fp = reinterpret_cast<float*>(p);
  uint8_t* bp = reinterpret_cast<uint8_t*>(p);
  const size_t big = ~(size_t)0 >> 1;
  const int32_t heads[][2] = {{1, 1}, {8, 1}, {24, 8}, {32, 8}, {64, 64}, {8192, 1024}};
  const int32_t BMs[][2] = {{1, 1}, {1, 4}, {8, 1}, {3, 7}, {65535, 1}, {65536, 1}, {8191, 8}, {65535, 8}, {1 << 22, 8}, {1 << 23, 4},
                            {1 << 25, 1}, {1, 31}, {1, 32}, {65535, 32}, {65536, 32}, {1 << 20, 32}, {1, 1 << 25}, {1, (1 << 25) + 1},
                            {0x7fffffff, 0x7fffffff}};
  const int32_t lengths[] = {1, 2, 33, 4096, 1 << 24, 1 << 28, (1 << 28) + 1, 0x7fffffff};
  int runs = 0, refused = 0;
  for (auto& h : heads)
    for (int d : {64, 128})
      for (auto& bm : BMs) {
        msa_config_t c = cfg(1, 1, h[0], h[1], d);
        // ---- window attention
        for (int32_t L : lengths)
          for (int32_t W : {1, 1000, 0x7fffffff})
            for (int32_t S : {0, 5, 0x7fffffff}) {
              const size_t ws = msa_window_attend_workspace_bytes(&c, bm[0], bm[1], L, W, S);
              auto status = [&](size_t bytes) {
                return msa_window_attend(&c, p, bm[0], bm[1], p, p, L, 0x7fffffff, W, S, ip, p, fp, p, bytes, nullptr);
              };
              const int rc = status(big);
              CHECK(rc == (ws == 0 ? MSA_ERR_UNSUPPORTED : MSA_ERR_HIP));
              if (ws != 0) {
                CHECK(ws >= 256 && ws % 256 == 0 && status(ws) == MSA_ERR_HIP && status(ws - 1) == MSA_ERR_WORKSPACE);
                ++runs;
              } else {
                ++refused;
              }
            }
        // ---- attention over a bank in four bits
        for (int32_t G : {1, 8, 512, 1 << 22, 1 << 28, 0x7fffffff})
          for (int32_t k : {1, 33, 64})
            for (int32_t L : {0, 1, 3000, 1 << 28})
              for (int pool : {0, 1}) {
                msa_config_t c4 = cfg(1000, G, h[0], h[1], d);
                c4.token_pool = pool;
                const size_t ws = msa_sparse_attend4_workspace_bytes(&c4, bm[0], bm[1], k, L);
                auto status = [&](size_t bytes) {
                  return msa_sparse_attend4(&c4, p, bm[0], bm[1], bp, bp, bp, bp, ip, k, p, p, L, 0x7fffffff, ip, p, fp, p, bytes, nullptr);
                };
                const int rc = status(big);
                CHECK(rc == (ws == 0 ? MSA_ERR_UNSUPPORTED : MSA_ERR_HIP));
                if (ws != 0) {
                  CHECK(ws % 256 == 0 && status(ws) == MSA_ERR_HIP && status(ws - 1) == MSA_ERR_WORKSPACE);
                  ++runs;
                } else {
                  ++refused;
                }
              }
        // ---- norms
        const int64_t stride = (int64_t)(h[0] + 2 * h[1]) * d;
        for (int32_t L : {0, 1, 1 << 28}) {
          const int rc = msa_norm_rotate(&c, p, stride, p, stride, p, stride, p, p, 1e-6f, 1, ip, bm[0], bm[1], p, p, p, L, 7, nullptr);
          CHECK(rc == ((int64_t)bm[0] * bm[1] > (1 << 25) ? MSA_ERR_UNSUPPORTED : MSA_ERR_HIP));
        }
      }
  CHECK(runs > 0 && refused > 0);
  // ---- packing: ranges of huge banks
  for (int32_t N : {1, 1000, (1 << 28) - 1, 0x7fffffff})
    for (int32_t G : {1, 512, 1 << 20}) {
      msa_config_t c = cfg(N, G, 32, 8, 128);
      for (int rotated : {0, 1}) {
        c.bank_keys_rotated = rotated;
        CHECK(msa_pack_kv4(&c, p, p, 0, N, p, p, p, p, nullptr) == MSA_ERR_HIP);
        CHECK(msa_pack_kv4(&c, p, nullptr, N - 1, 1, p, p, nullptr, nullptr, nullptr) == MSA_ERR_HIP);
        CHECK(msa_pack_kv4(&c, p, p, N, 0, p, p, p, p, nullptr) == MSA_OK);
        CHECK(msa_pack_kv4(&c, p, p, N, 1, p, p, p, p, nullptr) == MSA_ERR_INVALID_ARG);
        CHECK(msa_pack_kv4(&c, p, p, 0x7fffffff, 0x7fffffff, p, p, p, p, nullptr) == MSA_ERR_INVALID_ARG);
        CHECK(msa_unpack_kv4(&c, p, p, p, p, 0, N, p, p, nullptr) == MSA_ERR_HIP);
        CHECK(msa_unpack_kv4(&c, p, p, p, p, 1, 0x7fffffff, p, p, nullptr) == MSA_ERR_INVALID_ARG);
      }
    }
  std::printf(fails ? "encoded_sanitize: %d check(s) failed\n" : "encoded_sanitize: ok\n", fails);
  return fails ? 1 : 0;
}
