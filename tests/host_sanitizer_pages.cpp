// Host-side sanitizer run of the argument checks and workspace plans of the calls over pages, as host_sanitizer_main.cpp is for
// the others: every call only computes a size or fails a check before the first launch (the last one is the workspace's size,
// which is passed as 0, or a pointer that is not aligned), so nothing touches a device.
#include <cstdint>
#include <cstdio>
#include <cstring>
#include <vector>

#include "chunkkv.h"

static int failures = 0;
#define EXPECT(cond)                                                    \
  do {                                                                  \
    if (!(cond)) { std::printf("FAILED line %d: %s\n", __LINE__, #cond); ++failures; } \
  } while (0)

int main() {
  void *fake = (void *)0x1000, *odd = (void *)0x1008;   // never dereferenced
  const int lengths[9] = {0, 1, 31, 500, 961, 13171, 131072, (1 << 24) - 1, 1 << 24};
  int64_t n_cases = 0;
  for (int dt = 0; dt < 3; ++dt)
    for (int d : {64, 128})
      for (int batch : {1, 3, 64, 65, 200})
        for (int hkv : {1, 8, 1023})
          for (int g : {1, 5, 8, 17, 256})
            for (int page : {16, 48, 4096})
              for (int li = 0; li < 9; ++li) {
                std::vector<int32_t> most(batch), budget(batch), news(batch);
                int top = 1;
                for (int b = 0; b < batch; ++b) {
                  most[b] = lengths[(li + b) % (li + 1)];
                  budget[b] = b % 3 == 0 ? most[b] / 2 : (b % 3 == 1 ? most[b] : INT32_MAX);
                  news[b] = b % 4;
                  top = most[b] > top ? most[b] : top;
                }
                chunkkv_pages p;
                std::memset(&p, 0, sizeof(p));
                p.batch = batch; p.n_q_heads = hkv * g; p.n_kv_heads = hkv; p.head_dim = d; p.dtype = dt;
                p.page_tokens = page; p.n_pages = INT32_MAX; p.table_pitch = (top + page - 1) / page; p.slot_pitch = top;
                p.stride_tok = d; p.stride_head = (int64_t)page * d; p.stride_page = hkv * p.stride_head;
                p.max_tokens = most.data();
                const size_t plain = chunkkv_paged_decode_workspace_bytes(&p, 0), with = chunkkv_paged_decode_workspace_bytes(&p, 1);
                EXPECT(plain > 0 && with >= 256);
                // a pair and d numbers at least for every query head of a sequence of a launch
                EXPECT(plain >= (size_t)(batch < 64 ? batch : 64) * p.n_q_heads * (2 + d) * 4);
                for (void *w : {(void *)nullptr, fake}) {
                  EXPECT(chunkkv_paged_decode_attention(&p, (int32_t *)fake, nullptr, fake, fake, fake, (float *)fake, nullptr, (float *)w, fake, 0, nullptr) == CHUNKKV_ERR_WORKSPACE);
                  EXPECT(chunkkv_paged_decode_attention(&p, (int32_t *)fake, nullptr, fake, fake, fake, (float *)fake, nullptr, (float *)w, fake, (w ? with : plain) - 1, nullptr) == CHUNKKV_ERR_WORKSPACE);
                }
                EXPECT(chunkkv_paged_append(&p, news.data(), nullptr, 0, fake, (int64_t)hkv * d, odd, (int64_t)hkv * d, (int32_t *)fake, nullptr, nullptr, 0.f, nullptr, 0, 0, nullptr,
                                            (int32_t *)fake, fake, fake, (int32_t *)fake, (int32_t *)fake, nullptr, nullptr, nullptr) == CHUNKKV_ERR_SHAPE || (batch == 1 && news[0] == 0));
                for (int layers : {1, 61}) {
                  std::vector<void *> pools(layers, fake);
                  const size_t need = chunkkv_paged_evict_workspace_bytes(&p, layers, budget.data());
                  EXPECT(need >= (size_t)layers * batch * hkv * 4);
                  EXPECT(chunkkv_paged_evict(&p, layers, budget.data(), 0, (int32_t *)fake, pools.data(), pools.data(), (int32_t *)fake, (int32_t *)fake, (float *)fake, fake, need - 1, nullptr) == CHUNKKV_ERR_WORKSPACE);
                  pools[layers - 1] = nullptr;
                  EXPECT(chunkkv_paged_evict(&p, layers, budget.data(), 0, (int32_t *)fake, pools.data(), pools.data(), (int32_t *)fake, (int32_t *)fake, (float *)fake, fake, need, nullptr) == CHUNKKV_ERR_NULL);
                }
                ++n_cases;
              }
  std::printf("%lld cases, %d failures\n", (long long)n_cases, failures);
  if (failures == 0) std::printf("HOST SANITIZER RUN OK\n");
  return failures != 0;
}
