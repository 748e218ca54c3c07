// Eviction by accumulated attention weight, in place.
//
// A workgroup has one (layer, sequence, kv-head).  The budget_b-th slot in the order (protected, weight, slot) is found as
// chunks are selected (select.h, chunks of one token).  Kept slots below the budget stay; the others move into the slots
// that became free there.  Sources lie at or above the budget and destinations below it, so nothing that is read is
// written and the moves have no order; only slots that move cost bytes of K and V, twice the number of tokens to drop
// at most.
#include "paged.h"
#include "select.h"

namespace ckv {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

// Slot i as it is ranked: protected ones above every weight, infinite ones included.
struct EvictKey {
  const float *weight;
  const int32_t *pos;
  int64_t since;   // positions above it are protected
  __device__ __forceinline__ uint32_t operator[](int i) const {
    const uint32_t w = order_key(weight[i]);
    return (int64_t)pos[i] > since ? 0xFFFFFFFFu : w;
  }
};

template <int T, int KR, bool REG>
__global__ __launch_bounds__(T) void paged_evict_kernel(PagedEvictArgs a) {
  const int bl = blockIdx.x / a.n_kv_heads, h = blockIdx.x % a.n_kv_heads, b = a.batch0 + bl, layer = blockIdx.y;
  const int64_t head = ((int64_t)layer * a.batch_total + b) * a.n_kv_heads + h;
  const int m = CKV_ARG(PagedEvictArgs, budget, bl), most = CKV_ARG(PagedEvictArgs, max_tokens, bl), tid = threadIdx.x;
  int n = a.kv_len[head];
  n = n > most ? most : n;
  if (n <= m) return;
  int32_t *pos = a.token_pos + head * a.slot_pitch;
  float *weight = a.token_weight + head * a.slot_pitch;
  int32_t *source = a.lists + head * (2 * a.pitch + 1), *target = source + a.pitch;

  __shared__ int s_newest[T / 64], s_moves;
  int newest = INT32_MIN;
  for (int i = tid; i < n; i += T) newest = pos[i] > newest ? pos[i] : newest;
  for (int o = 32; o > 0; o >>= 1) {
    const int y = __shfl_xor(newest, o);
    newest = y > newest ? y : newest;
  }
  if ((tid & 63) == 0) s_newest[tid >> 6] = newest;
  if (tid == 0) s_moves = 0;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < T / 64; ++i) newest = s_newest[i] > newest ? s_newest[i] : newest;
  if (m > 0) {
    const EvictKey key{weight, pos, (int64_t)newest - a.recent};
    select_chunks<T, KR, REG>(key, n, 1, m, false, 0, [&](auto ranked, auto selected) __attribute__((always_inline)) {
      ranked([&](int i, uint32_t k) { return i >= m && i < n && selected(i, k); }, [&](int i, int rank) {
        source[rank] = i;
        atomicMax(&s_moves, rank + 1);
      });
      __syncthreads();
      ranked([&](int i, uint32_t k) { return i < m && !selected(i, k); }, [&](int i, int rank) { target[rank] = i; });
    });
  }
  __syncthreads();
  const int moves = s_moves;
  const int segs = a.row_bytes / 16;
  char *kp = (char *)CKV_ARG(PagedEvictArgs, k_pages, layer), *vp = (char *)CKV_ARG(PagedEvictArgs, v_pages, layer);
  const int32_t *table = a.geom.table + (int64_t)b * a.geom.pitch;
  for (int u = tid; u < moves * segs; u += T) {
    const int i = u / segs, seg = u % segs, from = source[i], to = target[i];
    const int64_t f = slot_offset(a.geom, table, h, from), t = slot_offset(a.geom, table, h, to);
    if (f >= 0 && t >= 0) {
      *(u32x4 *)(kp + t + seg * 16) = *(const u32x4 *)(kp + f + seg * 16);
      *(u32x4 *)(vp + t + seg * 16) = *(const u32x4 *)(vp + f + seg * 16);
    }
    if (seg == 0) {
      pos[to] = pos[from];
      weight[to] = weight[from];
    }
  }
  if (tid == 0) a.kv_len[head] = m;
}

int launch_paged_evict(const PagedEvictArgs &a, int n_layers, int batch, int max_tokens, hipStream_t s) {
  const dim3 grid(batch * a.n_kv_heads, n_layers);
  if (max_tokens <= 256) hipLaunchKernelGGL((paged_evict_kernel<256, 1, true>), grid, dim3(256), 0, s, a);
  else if (max_tokens <= 1024) hipLaunchKernelGGL((paged_evict_kernel<256, 4, true>), grid, dim3(256), 0, s, a);
  else if (max_tokens <= 4096) hipLaunchKernelGGL((paged_evict_kernel<1024, 4, true>), grid, dim3(1024), 0, s, a);
  else if (max_tokens <= 16384) hipLaunchKernelGGL((paged_evict_kernel<1024, 16, true>), grid, dim3(1024), 0, s, a);
  else hipLaunchKernelGGL((paged_evict_kernel<1024, 16, false>), grid, dim3(1024), 0, s, a);
  return hipGetLastError() == hipSuccess ? CHUNKKV_OK : CHUNKKV_ERR_LAUNCH;
}

}  // namespace ckv
