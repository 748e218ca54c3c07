// Compaction into pages: Algorithm 1's gather with slots of a paged cache as its destination.
//
// A workgroup takes `entries` consecutive selection entries of one (layer, sequence, kv-head); the window is handled as
// extra entries of up to `chunk` rows.  The lengths of the entries before them give its first slot.  Rows are taken 128 at
// a time: one thread per row finds source token and slot, writes position and weight, and leaves both addresses in LDS;
// then all threads copy K and V rows as 16-byte segments.
// The grid covers the ceil(n_keep / c) + 1 entries that a selection has where one chunk is cut.  Where sel_cap has room for more, a
// workgroup goes on to a second group and further ones (MORE), which costs a layer of 8192 tokens 0.3 us of 4.7.
// Bound by HBM over a stack (every row read and written once), by latency over a layer.  The full cache is read with streaming
// loads: nobody needs it again.  Stores are streaming where what is written is more than half of the memory-side cache; below, the
// next decoding step finds the pages there.  32 layers of 32768 tokens at 20 %: 309 us (5.6 TB/s; at 80 rows per workgroup 316, and
// with plain stores 340).
// Grid: x = group of entries, y = (sequence, kv-head), z = layer.
#include "paged.h"

namespace ckv {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
constexpr int kPagedRows = 128, kAhead = 5;

template <int NSEG, bool STREAM, bool MORE>   // 16-byte segments per row; streaming stores
__global__ __launch_bounds__(kThreads) void paged_compact_kernel(PagedCompactArgs a) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int bl = blockIdx.y / a.n_kv_heads, h = blockIdx.y % a.n_kv_heads, b = a.batch0 + bl, layer = blockIdx.z;
  const int n_keep = CKV_ARG(PagedCompactArgs, seq.n_keep, bl), w = a.window, c = a.chunk;
  const int P = CKV_ARG(PagedCompactArgs, seq.seqlen, bl) - w, ne = a.entries, n_win = (w + c - 1) / c;
  const int64_t selrow = ((int64_t)((a.layer0 + layer) / a.reuse) * a.batch_total + b) * a.n_kv_heads + h;
  const int32_t *sel_chunk = a.sel_chunk + selrow * a.sel_cap, *sel_len = a.sel_len + selrow * a.sel_cap;
  int e0 = blockIdx.x * ne;
  int count = n_keep > 0 ? a.sel_count[selrow] : 0;
  const int most = n_keep < a.sel_cap ? n_keep : a.sel_cap;   // an entry keeps a token at least
  count = count < 0 ? 0 : (count > most ? most : count);
  if (e0 >= count + n_win) return;

  __shared__ int s_src[kCompactEntries], s_dst[kCompactEntries], s_len[kCompactEntries], s_red[kThreads / 64];
  __shared__ int64_t s_from[kPagedRows], s_to[kPagedRows];
  int summed = 0, before = 0;   // entries whose tokens are added up, and these
  for (;;) {
    // kept tokens before entry min(e0, count)
    const int lim = e0 < count ? e0 : count;
    int sum = 0;
    for (int i = summed + (int)threadIdx.x; i < lim; i += kThreads) sum += sel_len[i];
    for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
    if (lane == 0) s_red[wave] = sum;
    __syncthreads();
    before += s_red[0] + s_red[1] + s_red[2] + s_red[3];
    summed = lim;
    if (wave == 0) {
      const int e = e0 + lane;
      const bool mine = lane < ne && e < count + n_win, chosen = mine && e < count;
      int ch = 0, len = 0;
      if (chosen) { ch = sel_chunk[e]; len = sel_len[e]; }
      int inc = len;
      for (int o = 1; o < 64; o <<= 1) {
        const int y = __shfl_up(inc, o);
        if (lane >= o) inc += y;
      }
      int src = ch * c, dst = before + inc - len;
      // Exact budget: the window follows at n_keep, whatever the entries say.  Whole chunks: at their sum; a group that holds
      // window entries has seen all of them by its last lane.
      int kept = a.whole_chunks ? before + __shfl(inc, 63) : n_keep;
      kept = kept < 0 ? 0 : (kept > n_keep ? n_keep : kept);
      if (chosen) {   // a malformed entry is skipped, never followed out of bounds
        if (ch < 0 || len < 1 || len > c || (int64_t)ch * c + len > P || dst < 0 || dst > n_keep - len) len = src = 0;
      } else if (mine) {
        const int wi = e - count;
        src = P + wi * c;
        len = w - wi * c < c ? w - wi * c : c;
        dst = kept + wi * c;
        if (wi == n_win - 1 && a.kv_len != nullptr)
          a.kv_len[((int64_t)layer * a.batch_total + b) * a.n_kv_heads + h] = kept + w;
      }
      if (lane < ne) { s_src[lane] = src; s_dst[lane] = dst; s_len[lane] = mine ? len : 0; }
    }
    __syncthreads();

    const int64_t esz = a.elem_bytes, in_tok = a.kv_stride_tok * esz;
    const int64_t in_head = (CKV_ARG(PagedCompactArgs, seq.kv_base, bl) + (int64_t)h * a.kv_stride_head) * esz;
    const char *kin = (const char *)CKV_ARG(PagedCompactArgs, k, layer) + in_head, *vin = (const char *)CKV_ARG(PagedCompactArgs, v, layer) + in_head;
    char *kout = (char *)CKV_ARG(PagedCompactArgs, k_pages, layer), *vout = (char *)CKV_ARG(PagedCompactArgs, v_pages, layer);
    const int32_t *table = a.geom.table + (int64_t)b * a.geom.pitch;
    const int64_t slots = (((int64_t)layer * a.batch_total + b) * a.n_kv_heads + h) * a.slot_pitch;
    const float *imp = CKV_ARG(PagedCompactArgs, importance, layer);
    const int live_entries = count + n_win - e0 < ne ? count + n_win - e0 : ne;
    // rows of this workgroup's list: c per entry, or one entry's own length; rows past an entry's length copy nothing
    const int rows = ne > 1 ? live_entries * c : s_len[0];
    for (int r0 = 0; r0 < rows; r0 += kPagedRows) {
      const int n = rows - r0 < kPagedRows ? rows - r0 : kPagedRows;
      if ((int)threadIdx.x < n) {
        const int row = r0 + threadIdx.x, en = ne > 1 ? row / c : 0, i = row - en * c;
        int64_t from = 0, to = -1;
        if (i < s_len[en]) {
          const int token = s_src[en] + i, slot = s_dst[en] + i;
          from = (int64_t)token * in_tok;
          to = slot_offset(a.geom, table, h, slot);
          if (a.token_pos != nullptr) a.token_pos[slots + slot] = token;
          if (a.token_weight != nullptr)
            a.token_weight[slots + slot] = imp != nullptr && token < P ? imp[((int64_t)b * a.n_kv_heads + h) * a.imp_pitch + token] : 0.f;
        }
        s_from[threadIdx.x] = from;
        s_to[threadIdx.x] = to;
      }
      __syncthreads();
      const int total = 2 * n * NSEG;
      for (int u0 = threadIdx.x; u0 < total; u0 += kAhead * kThreads) {
        u32x4 x[kAhead];
        char *to[kAhead];
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
          const int u = u0 + j * kThreads < total ? u0 + j * kThreads : u0;   // lanes without a segment read one of theirs again
          const bool is_v = u >= n * NSEG;
          const int uu = is_v ? u - n * NSEG : u, row = uu / NSEG, seg = uu % NSEG;
          x[j] = __builtin_nontemporal_load((const u32x4 *)((is_v ? vin : kin) + s_from[row] + seg * 16));
          to[j] = s_to[row] >= 0 && u0 + j * kThreads < total ? (is_v ? vout : kout) + s_to[row] + seg * 16 : nullptr;
        }
#pragma unroll
        for (int j = 0; j < kAhead; ++j)
          if (to[j] != nullptr) {
            if constexpr (STREAM) __builtin_nontemporal_store(x[j], (u32x4 *)to[j]);
            else *(u32x4 *)to[j] = x[j];
          }
      }
      __syncthreads();
    }
    e0 += gridDim.x * ne;
    if (!MORE || e0 >= count + n_win) return;
  }
}

int launch_paged_compact(int row_bytes, const PagedCompactArgs &args, int n_layers, int batch, hipStream_t s) {
  PagedCompactArgs a = args;
  // About 40 rows per workgroup.  us for 20 / 40 / 80 / 160, from a graph: a layer of 8192 tokens at 10 % 4.7 / 4.6 / 5.5 / 8.3; 32 layers of it
  // 47 / 40 / 40 / 43; 32 layers of 32768 at 20 % 334 / 301 / 307 / 333.
  int n = 40 / a.chunk;
  a.entries = n < 1 ? 1 : (n > kCompactEntries ? kCompactEntries : n);
  int most = 0, longest = 0;
  for (int i = 0; i < batch; ++i) {
    const int e = a.seq.n_keep[i] > 0 ? (a.seq.n_keep[i] + a.chunk - 1) / a.chunk + 1 : 0;
    most = e > most ? e : most;
    longest = a.seq.n_keep[i] > longest ? a.seq.n_keep[i] : longest;
  }
  const bool more = (longest < a.sel_cap ? longest : a.sel_cap) > most;
  const dim3 grid((most + (a.window + a.chunk - 1) / a.chunk + a.entries - 1) / a.entries, batch * a.n_kv_heads, n_layers);
  auto go = [&](auto kern) { hipLaunchKernelGGL(kern, grid, dim3(kThreads), 0, s, a); };
  auto of_row = [&](auto nseg) {
    constexpr int N = decltype(nseg)::value;
    if (more) a.stream ? go(paged_compact_kernel<N, true, true>) : go(paged_compact_kernel<N, false, true>);
    else a.stream ? go(paged_compact_kernel<N, true, false>) : go(paged_compact_kernel<N, false, false>);
  };
  if (row_bytes == 128) of_row(std::integral_constant<int, 8>());
  else if (row_bytes == 256) of_row(std::integral_constant<int, 16>());
  else of_row(std::integral_constant<int, 32>());
  return hipGetLastError() == hipSuccess ? CHUNKKV_OK : CHUNKKV_ERR_LAUNCH;
}

}  // namespace ckv
