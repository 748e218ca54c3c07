// Eviction by accumulated attention weight, in place.
//
// A workgroup selects for one (layer, sequence, kv-head): the budget_b-th slot in the order (protected by slot, weight, slot) is
// found as chunks are selected (select.h, chunks of one token).  Kept slots below the budget stay; the others move into the
// slots that became free there.  Sources lie at or above the budget and destinations below it, so nothing that is read is
// written and the moves have no order; only slots that move cost bytes of K and V.
// Up to kFewMoves slots move in the selecting workgroup, more of them in a launch of their own, which has workgroups for 64
// moves each and is bound by HBM.  us, so and in a launch: 200 moves of 8 heads 14.3 / 16.3, of 256 heads 21.7 / 29.0; 400 moves 17.0 / 16.3 and
// 31.5 / 34.5 (these and those at the launcher from a graph, with a copy that brings positions and weights back before every call).
// The selection is bound by latency for few slots (849 of 8 heads 8.3 us with its one move) and by the instructions of one workgroup's
// passes over a head for many.  Up to 8192 slots a thread has its own in registers, read together with the length, before it is
// known how many count; up to 32768 their keys are in LDS, beyond in the workspace.
// One pass of ranks gives both lists: slots on the wrong side of the budget, in ascending order, are the free ones, then the
// ones that move, as many.
#include "paged.h"
#include "select.h"

namespace ckv {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

constexpr int kFewMoves = 256, kMovesPerGroup = 64;

// All n moves of a head by one workgroup, a segment of K and of V per thread at a time; looking both places up once per move, behind a
// barrier, is slower for so few of them (200 moves 17.3 us, 14.6 so).
__device__ __forceinline__ void move_slots(const PagedEvictArgs &a, int layer, int b, int h, int64_t head, const int32_t *source, const int32_t *target, int n) {
  char *kp = (char *)CKV_ARG(PagedEvictArgs, k_pages, layer), *vp = (char *)CKV_ARG(PagedEvictArgs, v_pages, layer);
  const int32_t *table = a.geom.table + (int64_t)b * a.geom.pitch;
  int32_t *pos = a.token_pos + head * a.slot_pitch;
  float *weight = a.token_weight + head * a.slot_pitch;
  for (int u = threadIdx.x; u < n << a.row_shift; u += blockDim.x) {
    const int i = u >> a.row_shift, seg = u & ((1 << a.row_shift) - 1), from = source[i], to = target[i];
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

// Where a workgroup's keys are while it selects: KR of every thread in registers and LDS, all in LDS, in the workspace.
enum Keys { kInRegisters, kInLds, kInMemory };

// Largest over the T threads of a workgroup; s_red has room for one value per wavefront.
template <int T, typename V>
__device__ __forceinline__ V block_max(V x, V *s_red) {
  for (int o = 32; o > 0; o >>= 1) {
    const V y = __shfl_xor(x, o);
    x = y > x ? y : x;
  }
  if ((threadIdx.x & 63) == 0) s_red[threadIdx.x >> 6] = x;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < T / 64; ++i) x = s_red[i] > x ? s_red[i] : x;
  return x;
}

// T threads, KR slots each in a round
template <int T, int KR, int KEYS>
__global__ __launch_bounds__(T) void paged_evict_kernel(PagedEvictArgs a) {
  constexpr bool REG = KEYS == kInRegisters;
  const int bl = blockIdx.x / a.n_kv_heads, h = blockIdx.x % a.n_kv_heads, b = a.batch0 + bl, layer = blockIdx.y;
  const int64_t head = ((int64_t)layer * a.batch_total + b) * a.n_kv_heads + h;
  const int m = CKV_ARG(PagedEvictArgs, budget, bl), most = CKV_ARG(PagedEvictArgs, max_tokens, bl), tid = threadIdx.x;
  const int32_t *pos = a.token_pos + head * a.slot_pitch;
  const float *weight = a.token_weight + head * a.slot_pitch;
  int32_t *moves = a.lists + head * (2 * (int64_t)a.pitch + 1), *list = moves + 1;

  __shared__ int s_newest[T / 64], s_list[2 * kFewMoves];
  __shared__ uint32_t s_top[T / 64];
  __shared__ uint32_t s_key[REG ? T * KR : (KEYS == kInLds ? kEvictLdsKeys : 1)];
  uint32_t *key = KEYS == kInMemory ? a.keys + head * a.key_pitch : s_key;
  float w[KR];
  int32_t p[KR];
  // the round of slots from i0 on; there is room for `most` of them, however many hold a token
  auto read = [&](int i0, int end) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < KR; ++j) {
      const bool in = i0 + j * T + tid < end;
      w[j] = in ? weight[i0 + j * T + tid] : 0.f;
      p[j] = in ? pos[i0 + j * T + tid] : INT32_MIN;
    }
  };
  if constexpr (REG) read(0, most);   // beside the length
  int n = a.kv_len[head];
  n = n > most ? most : n;
  if (n <= m) {
    if (a.apart && tid == 0) *moves = 0;
    return;
  }
  int newest = INT32_MIN;
  for (int i0 = 0; i0 < (REG ? 1 : n); i0 += T * KR) {
    if constexpr (!REG) read(i0, n);
#pragma unroll
    for (int j = 0; j < KR; ++j) newest = i0 + j * T + tid < n && p[j] > newest ? p[j] : newest;
  }
  newest = block_max<T>(newest, s_newest);
  // positions from `since` on are protected; with recent = 0 none
  const int64_t since64 = (int64_t)newest - a.recent + 1;
  const int32_t since = since64 < INT32_MIN ? INT32_MIN : (int32_t)since64;
  const bool protects = a.recent > 0;
  // Slots as they are ranked: by weight, protected ones right above the largest, so that the selection's digits are spread over
  // the weights alone.
  uint32_t top = 0;
  for (int i0 = 0; i0 < (REG ? 1 : n); i0 += T * KR) {
    if constexpr (!REG) read(i0, n);
#pragma unroll
    for (int j = 0; j < KR; ++j) {
      const int i = i0 + j * T + tid;
      const uint32_t own = i < n && !(protects && p[j] >= since) ? order_key(w[j]) : 0u;
      top = own > top ? own : top;
      if (REG || i < n) key[i] = own;   // read again by the same thread, or behind a barrier
    }
  }
  top = block_max<T>(top, s_top);
  top += top != 0xFFFFFFFFu ? 1u : 0u;   // there is room for one more above infinity's key
  for (int i = tid; i < n; i += T)
    if (key[i] == 0) key[i] = top;
  const bool few = !a.apart;
  int count = 0;   // slots that move
  if (m > 0) {
    // Slots on the wrong side of the budget, in ascending order: the free ones, then as many that move into them.
    auto lists = [&](auto ranked, auto selected) __attribute__((always_inline)) {
      count = ranked([&](int i, uint32_t k) { return i < n && (i < m) != selected(i, k); }, [&](int i, int rank) {
        if (few) s_list[rank] = i;
        else list[rank] = i;
      }) / 2;
    };
    __syncthreads();
    select_chunks<T, KR, REG>((const uint32_t *)key, n, 1, m, false, 0, lists);
  }
  __syncthreads();
  if (few) move_slots(a, layer, b, h, head, s_list + count, s_list, count);
  if (tid == 0) {
    a.kv_len[head] = m;
    if (!few) *moves = count;
  }
}

// The moves of a head, kMovesPerGroup a workgroup: one thread per move looks up both places and takes position and weight
// along, then all copy rows as 16-byte segments, four of K or V in flight per thread.  Streaming loads and, where the moves may be
// more than half of the memory-side cache, streaming stores, as in the compaction: half of 53385 slots in 8 layers 79 us, plain 86.
// Grid: x = group of moves, y = (sequence, kv-head), z = layer.
template <bool STREAM>
__global__ __launch_bounds__(kThreads) void paged_move_kernel(PagedEvictArgs a) {
  const int bl = blockIdx.y / a.n_kv_heads, h = blockIdx.y % a.n_kv_heads, b = a.batch0 + bl, layer = blockIdx.z;
  const int64_t head = ((int64_t)layer * a.batch_total + b) * a.n_kv_heads + h;
  const int32_t *moves = a.lists + head * (2 * (int64_t)a.pitch + 1);
  const int i0 = blockIdx.x * kMovesPerGroup, all = *moves, n = all - i0 < kMovesPerGroup ? all - i0 : kMovesPerGroup;
  if (n <= 0) return;
  __shared__ int64_t s_from[kMovesPerGroup], s_to[kMovesPerGroup];
  const int tid = threadIdx.x;
  if (tid < n) {
    const int to = moves[1 + i0 + tid], from = moves[1 + all + i0 + tid];
    const int32_t *table = a.geom.table + (int64_t)b * a.geom.pitch;
    const int64_t f = slot_offset(a.geom, table, h, from), t = slot_offset(a.geom, table, h, to);
    s_from[tid] = t >= 0 ? f : -1;
    s_to[tid] = t;
    int32_t *pos = a.token_pos + head * a.slot_pitch;
    float *weight = a.token_weight + head * a.slot_pitch;
    pos[to] = pos[from];
    weight[to] = weight[from];
  }
  __syncthreads();
  char *kp = (char *)CKV_ARG(PagedEvictArgs, k_pages, layer), *vp = (char *)CKV_ARG(PagedEvictArgs, v_pages, layer);
  const int half = n << a.row_shift, total = 2 * half;
  for (int u0 = tid; u0 < total; u0 += 4 * kThreads) {
    u32x4 x[4];
    char *to[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int u = u0 + j * kThreads, uu = u >= half ? u - half : u, row = uu >> a.row_shift, seg = uu & ((1 << a.row_shift) - 1);
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

// Threads and slots of each: the variant that a head of max_tokens just fits.  us for 8 heads / 512 heads: 500 slots, 512 x 1 7.7 / 15.1,
// 256 x 2 7.9 / 15.5; 849, 512 x 2 8.2 / 21.0, 256 x 4 8.5 / 21.8, 1024 x 1 9.0 / 22.9; 2000, 512 x 4 9.2 / 22.2, 1024 x 2 9.6 / 23.0; 4000, 1024 x 4
// 10.4 / 28.3, 1024 x 8 11.7 / 31.0; 8000, 1024 x 8 14.2 / 41.9, in LDS 16.3 / 41.7; 16000, 1024 x 16 21.5 / 73.8, in LDS 21.0 / 66.5 (where half of the
// slots leave, the registers are 3 % faster); 30000, in LDS 32.8 / 119.6, in the workspace 43.5 / 132.3.
int launch_paged_evict(const PagedEvictArgs &args, int n_layers, int batch, int max_tokens, hipStream_t s) {
  PagedEvictArgs a = args;
  a.apart = paged_moves_apart(a);
  const dim3 grid(batch * a.n_kv_heads, n_layers);
  auto go = [&](auto kern, int threads) { hipLaunchKernelGGL(kern, grid, dim3(threads), 0, s, a); };
  if (max_tokens <= 256) go(paged_evict_kernel<256, 1, kInRegisters>, 256);
  else if (max_tokens <= 512) go(paged_evict_kernel<512, 1, kInRegisters>, 512);
  else if (max_tokens <= 1024) go(paged_evict_kernel<512, 2, kInRegisters>, 512);
  else if (max_tokens <= 2048) go(paged_evict_kernel<512, 4, kInRegisters>, 512);
  else if (max_tokens <= 4096) go(paged_evict_kernel<1024, 4, kInRegisters>, 1024);
  else if (max_tokens <= 8192) go(paged_evict_kernel<1024, 8, kInRegisters>, 1024);
  else if (max_tokens <= kEvictLdsKeys) go(paged_evict_kernel<1024, 16, kInLds>, 1024);
  else go(paged_evict_kernel<1024, 16, kInMemory>, 1024);
  return hipGetLastError() == hipSuccess ? CHUNKKV_OK : CHUNKKV_ERR_LAUNCH;
}

int launch_paged_move(const PagedEvictArgs &a, int n_layers, int batch, hipStream_t s) {
  const dim3 grid((a.pitch + kMovesPerGroup - 1) / kMovesPerGroup, batch * a.n_kv_heads, n_layers);
  if (a.stream) hipLaunchKernelGGL(paged_move_kernel<true>, grid, dim3(kThreads), 0, s, a);
  else hipLaunchKernelGGL(paged_move_kernel<false>, grid, dim3(kThreads), 0, s, a);
  return hipGetLastError() == hipSuccess ? CHUNKKV_OK : CHUNKKV_ERR_LAUNCH;
}

}  // namespace ckv
