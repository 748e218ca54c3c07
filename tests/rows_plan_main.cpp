// What chunkkv_cross_attention and chunkkv_shared_decode_attention launch, without a GPU: the host side of the library with launches that
// write their arguments down.  One call per line of the input, one line of JSON each:
//   cross  dtype hq hkv d B  q_len[B]  seqlen[B]          outputs packed, [tokens][hq][d]
//   shared dtype hq hkv d P B  n_sharing[P]  prefix slots[P]  own slots[B]
#include "rows_api.hip"

#include <cstdio>
#include <cstring>
#include <string>
#include <vector>

static std::string said;
static char line[512];
#define SAY(...) (std::snprintf(line, sizeof(line), __VA_ARGS__), said += line)

template <int N>
static int attention(const RowsArgs<N> &r) {
  SAY("%s{\"kind\": \"rows\", \"tile\": %d, \"seq0\": %d, \"prefixes\": %d, \"prefix0\": %d, \"blocks\": %d, \"segments\": [", said.back() == '[' ? "" : ", ", r.tile, r.seq0, r.prefixes, r.prefix0,
      r.first[r.segments]);
  for (int i = 0; i < r.segments; ++i) {
    const RowsSegment &s = r.segment[i];
    SAY("%s[%d, %d, %d, %d, %d, %d, %d, %d]", i ? ", " : "", r.first[i], s.rows, s.most, s.row0, s.splits, s.tiles, s.part, s.splits > 0 ? rows_range(s.most, s.splits) : 0);
  }
  said += "]}";
  return CHUNKKV_OK;
}

namespace ckv {
int launch_cross_bf16(int, const CrossArgs &a, hipStream_t) { return attention(a.r); }
int launch_cross_f16(int, const CrossArgs &a, hipStream_t) { return attention(a.r); }
int launch_cross_f32(int, const CrossArgs &a, hipStream_t) { return attention(a.r); }
int launch_shared_bf16(int, const SharedArgs &a, hipStream_t) { return attention(a.r); }
int launch_shared_f16(int, const SharedArgs &a, hipStream_t) { return attention(a.r); }
int launch_shared_f32(int, const SharedArgs &a, hipStream_t) { return attention(a.r); }
int launch_join(int, int, const JoinArgs &a, hipStream_t) {
  SAY("%s{\"kind\": \"join\", \"tokens\": %d, \"segments\": [", said.back() == '[' ? "" : ", ", a.tokens);
  for (int i = 0; i < a.segments; ++i) {
    const JoinSegment &s = a.segment[i];
    SAY("%s[%d, %d, %d, %d, %d, %d, %d, %d, %d, %lld]", i ? ", " : "", a.first[i], s.part, s.splits, s.rows, s.token0, s.prefix_part, s.prefix_splits, s.prefix_rows, s.prefix_row0,
        (long long)s.out_base);
  }
  said += "]}";
  return CHUNKKV_OK;
}
}  // namespace ckv

static std::vector<int32_t> numbers(int n) {
  std::vector<int32_t> x(n);
  for (int32_t &i : x)
    if (std::scanf("%d", &i) != 1) std::abort();
  return x;
}

int main() {
  void *fake = (void *)0x1000;   // never dereferenced
  char what[16];
  while (std::scanf("%15s", what) == 1) {
    const std::vector<int32_t> head = numbers(4);
    const int dtype = head[0], hq = head[1], hkv = head[2], d = head[3];
    said = "[";
    size_t bytes;
    int rc;
    if (!std::strcmp(what, "cross")) {
      const int B = numbers(1)[0];
      const std::vector<int32_t> q_len = numbers(B), seqlen = numbers(B);
      std::vector<int64_t> zero(B, 0), out(B);
      int64_t at = 0;
      for (int b = 0; b < B; ++b) {
        out[b] = at;
        at += (int64_t)q_len[b] * hq * d;
      }
      chunkkv_cross c;
      std::memset(&c, 0, sizeof(c));
      c.batch = B; c.n_q_heads = hq; c.n_kv_heads = hkv; c.head_dim = d; c.dtype = dtype;
      c.q_len = q_len.data(); c.seqlen = seqlen.data(); c.q_base = c.out_base = out.data(); c.kv_base = zero.data();
      c.q_stride_head = c.out_stride_head = c.kv_stride_head = d;
      c.q_stride_tok = c.out_stride_tok = (int64_t)hq * d; c.kv_stride_tok = (int64_t)hkv * d;
      bytes = chunkkv_cross_workspace_bytes(&c);
      rc = chunkkv_cross_attention(&c, nullptr, nullptr, fake, fake, fake, fake, nullptr, fake, bytes, nullptr);
    } else {
      const int P = numbers(1)[0], B = numbers(1)[0];
      const std::vector<int32_t> sharing = numbers(P), prefix = numbers(P), own = numbers(B);
      chunkkv_pages p;
      std::memset(&p, 0, sizeof(p));
      p.batch = B; p.n_q_heads = hq; p.n_kv_heads = hkv; p.head_dim = d; p.dtype = dtype;
      p.page_tokens = 4096; p.n_pages = 1 << 20; p.table_pitch = 1 << 12;
      p.stride_tok = d; p.stride_head = (int64_t)4096 * d; p.stride_page = hkv * p.stride_head;
      p.max_tokens = own.data();
      chunkkv_pages w = p;
      w.batch = P; w.max_tokens = prefix.data();
      bytes = chunkkv_shared_decode_workspace_bytes(&w, &p, sharing.data());
      rc = chunkkv_shared_decode_attention(&w, &p, sharing.data(), (int32_t *)fake, nullptr, (int32_t *)fake, nullptr, fake, fake, fake, fake, nullptr, fake, bytes, nullptr);
    }
    std::printf("{\"rc\": %d, \"bytes\": %zu, \"launches\": %s]}\n", rc, bytes, said.c_str());
  }
  return 0;
}
