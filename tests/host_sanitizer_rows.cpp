// Host-side sanitizer run of the argument checks and workspace plans of the calls for a cache that many queries read, as
// host_sanitizer_pages.cpp is for those over pages: every call only computes a size or fails a check before the first launch.
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
  const int lengths[9] = {0, 1, 63, 65, 961, 13171, 131072, (1 << 24) - 1, 1 << 24};
  const int queries[6] = {0, 1, 17, 4096, 100000, 1 << 21};
  int64_t n_cases = 0;
  for (int dt = 0; dt < 3; ++dt)
    for (int d : {64, 128})
      for (int batch : {1, 3, 32, 33, 200})
        for (int hkv : {1, 8, 1023})
          for (int g : {1, 5, 256})
            for (int li = 0; li < 9; ++li) {
              std::vector<int32_t> q_len(batch), seqlen(batch), budget(batch);
              std::vector<int64_t> base(batch, (int64_t)1 << 40), zero(batch, 0);
              int64_t rows = 0;
              int top = 1;
              for (int b = 0; b < batch; ++b) {
                q_len[b] = queries[(li + b) % 6];
                seqlen[b] = lengths[(li + b) % (li + 1)];
                rows += (int64_t)q_len[b] * g;
                top = seqlen[b] > top ? seqlen[b] : top;
              }
              chunkkv_cross c;
              std::memset(&c, 0, sizeof(c));
              c.batch = batch; c.n_q_heads = hkv * g; c.n_kv_heads = hkv; c.head_dim = d; c.dtype = dt;
              c.q_len = q_len.data(); c.seqlen = seqlen.data(); c.q_base = zero.data(); c.kv_base = base.data(); c.out_base = zero.data();
              c.q_stride_head = c.out_stride_head = c.kv_stride_head = d;
              c.q_stride_tok = c.out_stride_tok = (int64_t)hkv * g * d; c.kv_stride_tok = (int64_t)hkv * d;
              c.mask_pitch = top;
              const size_t need = chunkkv_cross_workspace_bytes(&c);
              const int rc = chunkkv_cross_attention(&c, nullptr, (uint8_t *)fake, odd, fake, fake, fake, (float *)fake, fake, (size_t)-1, nullptr);
              EXPECT(rc == (need ? CHUNKKV_ERR_SHAPE : CHUNKKV_ERR_UNSUPPORTED) || rc == CHUNKKV_ERR_NULL);
              if (need > 256) EXPECT(chunkkv_cross_attention(&c, nullptr, nullptr, fake, fake, fake, fake, nullptr, fake, need - 1, nullptr) == CHUNKKV_ERR_WORKSPACE);
              // the sequences are what a prefix has, their lengths those of prefixes and of own pages
              for (int prefixes : {1, 2, 17, 40}) {
                std::vector<int32_t> sharing(prefixes), most(prefixes);
                int left = batch;
                for (int i = 0; i < prefixes; ++i) {
                  sharing[i] = i + 1 == prefixes ? left : (left > i ? i % 3 : 0);
                  left -= sharing[i];
                  most[i] = lengths[(li + i) % (li + 1)];
                  top = most[i] > top ? most[i] : top;
                }
                chunkkv_pages p;
                std::memset(&p, 0, sizeof(p));
                p.batch = batch; p.n_q_heads = hkv * g; p.n_kv_heads = hkv; p.head_dim = d; p.dtype = dt;
                p.page_tokens = 48; p.n_pages = INT32_MAX; p.table_pitch = (top + 47) / 48; p.slot_pitch = top;
                p.stride_tok = d; p.stride_head = (int64_t)48 * d; p.stride_page = hkv * p.stride_head;
                p.max_tokens = seqlen.data();
                chunkkv_pages w = p;
                w.batch = prefixes; w.max_tokens = most.data();
                const size_t size = chunkkv_shared_decode_workspace_bytes(&w, &p, sharing.data());
                if (left < 0 || size == 0) continue;
                EXPECT(chunkkv_shared_decode_attention(&w, &p, sharing.data(), (int32_t *)fake, nullptr, (int32_t *)fake, nullptr, odd, fake, fake, fake, nullptr, fake, size, nullptr) == CHUNKKV_ERR_SHAPE);
                if (size > 256)
                  EXPECT(chunkkv_shared_decode_attention(&w, &p, sharing.data(), (int32_t *)fake, nullptr, (int32_t *)fake, nullptr, fake, fake, fake, fake, nullptr, fake, size - 1, nullptr) == CHUNKKV_ERR_WORKSPACE);
                sharing[0] += 1;
                EXPECT(chunkkv_shared_decode_workspace_bytes(&w, &p, sharing.data()) == 0);
              }
              ++n_cases;
            }
  for (int d : {64, 128})
    for (int64_t stride : {(int64_t)0, (int64_t)d, (int64_t)1 << 56, INT64_MAX / 8 * 8}) {
      chunkkv_rows r;
      std::memset(&r, 0, sizeof(r));
      r.in = fake; r.out = (void *)0x2000; r.n_heads = 3;
      r.in_stride_seq = r.in_stride_head = r.in_stride_tok = r.out_stride_seq = r.out_stride_head = r.out_stride_tok = stride;
      for (int dt = 0; dt < 3; ++dt) EXPECT(chunkkv_rotate(dt, d, 1, 1, &r, nullptr, nullptr, (float *)fake, d, 0, 1.f, nullptr) != CHUNKKV_OK);
      float f[64];
      EXPECT(chunkkv_rotary_frequencies(d, 1e4, 2.0, 1.0, 32.0, 4096.0, f) == CHUNKKV_OK);
      ++n_cases;
    }
  std::printf("%lld cases, %d failures\n", (long long)n_cases, failures);
  if (failures == 0) std::printf("HOST SANITIZER RUN OK\n");
  return failures != 0;
}
