// Eviction by accumulated attention weight, in place.
//
// A workgroup selects for one (layer, sequence, kv-head): the budget_b-th slot in the order (protected, weight, slot) is
// found as chunks are selected (select.h, chunks of one token).  Kept slots below the budget stay; the others move into the
// slots that became free there.  Sources lie at or above the budget and destinations below it, so nothing that is read is
// written and the moves have no order; only slots that move cost bytes of K and V.
// Up to kFewMoves slots move in the selecting workgroup, more of them in a launch of their own, which has workgroups for 64
// moves each and is bound by HBM.
// The selection is bound by latency.  Weights and positions of all slots that there is room for are read together with the
// length, before it is known how many count, and ranked out of LDS, up to 16384 of them (64 KB); more are read again in every step.
#include "paged.h"
#include "select.h"

namespace ckv {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

constexpr int kFewMoves = 64;

// Slots as they are ranked: by weight, protected ones above all of them.
struct EvictKeys {
  const float *weight;
  const int32_t *pos;
  int64_t since;   // positions above it are protected
  __device__ __forceinline__ uint32_t operator[](int i) const {
    const uint32_t w = order_key(weight[i]);
    return (int64_t)pos[i] > since ? 0xFFFFFFFFu : w;
  }
};

// Moves [i0, i0 + n) of a head's lists, one after the other for the threads of a workgroup.
__device__ __forceinline__ void move_slots(const PagedEvictArgs &a, int layer, int b, int h, int64_t head, const int32_t *source, const int32_t *target, int n) {
  const int segs = a.row_bytes / 16;
  char *kp = (char *)CKV_ARG(PagedEvictArgs, k_pages, layer), *vp = (char *)CKV_ARG(PagedEvictArgs, v_pages, layer);
  const int32_t *table = a.geom.table + (int64_t)b * a.geom.pitch;
  int32_t *pos = a.token_pos + head * a.slot_pitch;
  float *weight = a.token_weight + head * a.slot_pitch;
  for (int u = threadIdx.x; u < n * segs; u += blockDim.x) {
    const int i = u / segs, seg = u % segs, from = source[i], to = target[i];
    const int64_t f = slot_offset(a.geom, table, h, from), t = slot_offset(a.geom, table, h, to);
    if (f >= 0 && t >= 0) {
      const u32x4 x = *(const u32x4 *)(kp + f + seg * 16), y = *(const u32x4 *)(vp + f + seg * 16);
      *(u32x4 *)(kp + t + seg * 16) = x;
      *(u32x4 *)(vp + t + seg * 16) = y;
    }
    if (seg == 0) {
      pos[to] = pos[from];
      weight[to] = weight[from];
    }
  }
}

// T threads, KR slots each; REG: all of them stay in registers and LDS
template <int T, int KR, bool REG>
__global__ __launch_bounds__(T) void paged_evict_kernel(PagedEvictArgs a) {
  const int bl = blockIdx.x / a.n_kv_heads, h = blockIdx.x % a.n_kv_heads, b = a.batch0 + bl, layer = blockIdx.y;
  const int64_t head = ((int64_t)layer * a.batch_total + b) * a.n_kv_heads + h;
  const int m = CKV_ARG(PagedEvictArgs, budget, bl), most = CKV_ARG(PagedEvictArgs, max_tokens, bl), tid = threadIdx.x;
  const int32_t *pos = a.token_pos + head * a.slot_pitch;
  const float *weight = a.token_weight + head * a.slot_pitch;
  int32_t *moves = a.lists + head * (2 * (int64_t)a.pitch + 1), *source = moves + 1, *target = source + a.pitch;

  __shared__ int s_newest[T / 64], s_list[2][kFewMoves];
  __shared__ uint32_t s_top[T / 64];
  __shared__ uint32_t s_key[REG ? T * KR : 1];
  float w[REG ? KR : 1];
  int32_t p[REG ? KR : 1];
  if constexpr (REG) {   // room for `most` slots there is, however many hold a token
#pragma unroll
    for (int j = 0; j < KR; ++j) {
      const bool in = j * T + tid < most;
      w[j] = in ? weight[j * T + tid] : 0.f;
      p[j] = in ? pos[j * T + tid] : 0;
    }
  }
  int n = a.kv_len[head];
  n = n > most ? most : n;
  if (n <= m) {
    if (a.apart && tid == 0) *moves = 0;
    return;
  }
  int newest = INT32_MIN;
  if constexpr (REG) {
#pragma unroll
    for (int j = 0; j < KR; ++j) newest = j * T + tid < n && p[j] > newest ? p[j] : newest;
  } else {
    for (int i = tid; i < n; i += T) newest = pos[i] > newest ? pos[i] : newest;
  }
  for (int o = 32; o > 0; o >>= 1) {
    const int y = __shfl_xor(newest, o);
    newest = y > newest ? y : newest;
  }
  if ((tid & 63) == 0) s_newest[tid >> 6] = newest;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < T / 64; ++i) newest = s_newest[i] > newest ? s_newest[i] : newest;
  const int64_t since = (int64_t)newest - a.recent;
  if constexpr (REG) {   // read again by the same thread, or behind a barrier
    // Protected slots right above the largest weight: the selection's digits are then spread over the weights alone.
    uint32_t top = 0, own[KR];
#pragma unroll
    for (int j = 0; j < KR; ++j) {
      own[j] = j * T + tid < n && (int64_t)p[j] <= since ? order_key(w[j]) : 0u;
      top = own[j] > top ? own[j] : top;
    }
    for (int o = 32; o > 0; o >>= 1) {
      const uint32_t y = __shfl_xor(top, o);
      top = y > top ? y : top;
    }
    if ((tid & 63) == 0) s_top[tid >> 6] = top;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < T / 64; ++i) top = s_top[i] > top ? s_top[i] : top;
    const uint32_t above = top + (top != 0xFFFFFFFFu ? 1u : 0u);   // there is room for one more above infinity's key
#pragma unroll
    for (int j = 0; j < KR; ++j) s_key[j * T + tid] = own[j] != 0 ? own[j] : above;
  }
  const bool few = !a.apart;
  int count = 0;   // slots that move
  if (m > 0) {
    auto lists = [&](auto ranked, auto selected) __attribute__((always_inline)) {
      count = ranked([&](int i, uint32_t k) { return i >= m && i < n && selected(i, k); }, [&](int i, int rank) {
        if (few) s_list[0][rank] = i;
        else source[rank] = i;
      });
      __syncthreads();
      ranked([&](int i, uint32_t k) { return i < m && !selected(i, k); }, [&](int i, int rank) {
        if (few) s_list[1][rank] = i;
        else target[rank] = i;
      });
    };
    if constexpr (REG) select_chunks<T, KR, REG>((const uint32_t *)s_key, n, 1, m, false, 0, lists);
    else select_chunks<T, KR, REG>(EvictKeys{weight, pos, since}, n, 1, m, false, 0, lists);
  }
  __syncthreads();
  if (few) move_slots(a, layer, b, h, head, s_list[0], s_list[1], count);
  if (tid == 0) {
    a.kv_len[head] = m;
    if (!few) *moves = count;
  }
}

// The moves of a head, kMovesPerGroup a workgroup: one thread per move looks up both places and takes position and weight
// along, then all copy rows as 16-byte segments, four of K or V in flight per thread.  Streaming loads and, where the moves may be
// more than half of the memory-side cache, streaming stores, as in the compaction: half of 53385 slots in 8 layers 79 us, plain 86.
// Grid: x = group of moves, y = (sequence, kv-head), z = layer.
constexpr int kMovesPerGroup = 64;
template <int NSEG, bool STREAM>   // 16-byte segments per row; streaming stores
__global__ __launch_bounds__(kThreads) void paged_move_kernel(PagedEvictArgs a) {
  const int bl = blockIdx.y / a.n_kv_heads, h = blockIdx.y % a.n_kv_heads, b = a.batch0 + bl, layer = blockIdx.z;
  const int64_t head = ((int64_t)layer * a.batch_total + b) * a.n_kv_heads + h;
  const int32_t *moves = a.lists + head * (2 * (int64_t)a.pitch + 1);
  const int i0 = blockIdx.x * kMovesPerGroup, all = *moves, n = all - i0 < kMovesPerGroup ? all - i0 : kMovesPerGroup;
  if (n <= 0) return;
  __shared__ int64_t s_from[kMovesPerGroup], s_to[kMovesPerGroup];
  if ((int)threadIdx.x < n) {
    const int from = moves[1 + i0 + threadIdx.x], to = moves[1 + a.pitch + i0 + threadIdx.x];
    const int32_t *table = a.geom.table + (int64_t)b * a.geom.pitch;
    const int64_t f = slot_offset(a.geom, table, h, from), t = slot_offset(a.geom, table, h, to);
    s_from[threadIdx.x] = t >= 0 ? f : -1;
    s_to[threadIdx.x] = t;
    int32_t *pos = a.token_pos + head * a.slot_pitch;
    float *weight = a.token_weight + head * a.slot_pitch;
    pos[to] = pos[from];
    weight[to] = weight[from];
  }
  __syncthreads();
  char *kp = (char *)CKV_ARG(PagedEvictArgs, k_pages, layer), *vp = (char *)CKV_ARG(PagedEvictArgs, v_pages, layer);
  const int half = n * NSEG, total = 2 * half;
  for (int u0 = threadIdx.x; u0 < total; u0 += 4 * kThreads) {
    u32x4 x[4];
    char *to[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int u = u0 + j * kThreads, uu = u >= half ? u - half : u, row = uu / NSEG, seg = uu % NSEG;
      to[j] = nullptr;
      if (u < total && s_from[row] >= 0) {
        char *pool = u >= half ? vp : kp;
        x[j] = __builtin_nontemporal_load((const u32x4 *)(pool + s_from[row] + seg * 16));   // nobody reads this slot again
        to[j] = pool + s_to[row] + seg * 16;
      }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (to[j] != nullptr) {
        if constexpr (STREAM) __builtin_nontemporal_store(x[j], (u32x4 *)to[j]);
        else *(u32x4 *)to[j] = x[j];
      }
  }
}

bool paged_moves_apart(const PagedEvictArgs &a) { return a.pitch > kFewMoves; }

int launch_paged_evict(const PagedEvictArgs &args, int n_layers, int batch, int max_tokens, hipStream_t s) {
  PagedEvictArgs a = args;
  a.apart = paged_moves_apart(a);
  const dim3 grid(batch * a.n_kv_heads, n_layers);
  if (max_tokens <= 256) hipLaunchKernelGGL((paged_evict_kernel<256, 1, true>), grid, dim3(256), 0, s, a);
  else if (max_tokens <= 1024) hipLaunchKernelGGL((paged_evict_kernel<256, 4, true>), grid, dim3(256), 0, s, a);
  else if (max_tokens <= 4096) hipLaunchKernelGGL((paged_evict_kernel<1024, 4, true>), grid, dim3(1024), 0, s, a);
  else if (max_tokens <= 8192) hipLaunchKernelGGL((paged_evict_kernel<1024, 8, true>), grid, dim3(1024), 0, s, a);
  else if (max_tokens <= 16384) hipLaunchKernelGGL((paged_evict_kernel<1024, 16, true>), grid, dim3(1024), 0, s, a);
  else hipLaunchKernelGGL((paged_evict_kernel<1024, 16, false>), grid, dim3(1024), 0, s, a);
  return hipGetLastError() == hipSuccess ? CHUNKKV_OK : CHUNKKV_ERR_LAUNCH;
}

int launch_paged_move(const PagedEvictArgs &a, int n_layers, int batch, hipStream_t s) {
  const dim3 grid((a.pitch + kMovesPerGroup - 1) / kMovesPerGroup, batch * a.n_kv_heads, n_layers);
  auto go = [&](auto kern) { hipLaunchKernelGGL(kern, grid, dim3(kThreads), 0, s, a); };
  if (a.row_bytes == 128) a.stream ? go(paged_move_kernel<8, true>) : go(paged_move_kernel<8, false>);
  else if (a.row_bytes == 256) a.stream ? go(paged_move_kernel<16, true>) : go(paged_move_kernel<16, false>);
  else a.stream ? go(paged_move_kernel<32, true>) : go(paged_move_kernel<32, false>);
  return hipGetLastError() == hipSuccess ? CHUNKKV_OK : CHUNKKV_ERR_LAUNCH;
}

}  // namespace ckv
