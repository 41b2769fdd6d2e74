// Eviction from the cache by the attention that slots have gathered: which slots stay, and where their rows go.
//
// What stays is a set of slots, and attention does not ask for their order: a slot below the budget that stays keeps its place, and only the
// survivors behind it move, into the freed places.  Sources (at or behind the budget) and destinations (below it) never meet, so all rows move at
// once, in place too; a step that drops one token moves one row of each head.
#include "cache_internal.h"

namespace tc {

// A slot's place in the order, larger is better: protected slots first, then weights descending (+0 and -0 alike), NaN last.  Never 0.
__device__ inline uint32_t evict_key(int pos, float w, int sink, int recent, int newest) {
  if (pos < sink || (long long)pos > (long long)newest - recent) return 0xffffffffu;
  if (w != w) w = -INFINITY;
  return (uint32_t)(order_key(w, 0) >> 32);
}

// One workgroup per sequence and head.  The slots are dealt to the wavefronts in runs, a run's 64 lanes side by side, KPT keys of a lane in
// registers (KPT = 0: any number of slots, the keys formed anew each time).  The threshold, the largest key that at least `budget` slots reach, is
// found two bits at a time from counts of three candidates; equal keys stay from the lowest slot on.  Then each freed place takes the survivor of
// its rank.
template <int NT, int KPT>
__global__ __launch_bounds__(NT) void evict_select_kernel(const int32_t* __restrict__ len, const int32_t* __restrict__ slot_pos,
                                                          const float* __restrict__ weight, int32_t* __restrict__ source,
                                                          int32_t* __restrict__ list, int32_t* __restrict__ len_out, int Hk, int cap,
                                                          int max_len, int budget, int sink, int recent) {
  constexpr int W = NT / 64, UN = KPT > 0 ? KPT : 1;
  __shared__ int count[3][3], part[4][W];
  __shared__ uint16_t moved_lds[KPT > 0 ? NT * KPT / 2 : 1];  // at most half of the slots move
  const size_t bh = blockIdx.x;
  const int b = (int)(bh / Hk), tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = clamp_len(len[b], max_len);
  if (bh % Hk == 0 && tid == 0) len_out[b] = min(n, budget);
  int32_t* src = source + bh * budget;
  if (n <= budget) {
    for (int j = tid; j < n; j += NT) src[j] = j;
    return;
  }
  const int32_t* pos = slot_pos + bh * cap;
  const float* wgt = weight + bh * cap;
  const int rounds = KPT > 0 ? KPT : (n + NT - 1) / NT, first = wave * 64 * rounds + lane;

  int newest = INT32_MIN;
  int rpos[KPT > 0 ? KPT : 1];
  float rw[KPT > 0 ? KPT : 1];
  uint32_t rkey[KPT > 0 ? KPT : 1];
  if constexpr (KPT > 0) {
#pragma unroll
    for (int k = 0; k < KPT; k++) {
      const int i = first + 64 * k;
      rpos[k] = i < n ? pos[i] : INT32_MIN;
      rw[k] = i < n ? wgt[i] : 0.f;
    }
#pragma unroll
    for (int k = 0; k < KPT; k++) newest = max(newest, rpos[k]);
  } else {
    for (int k = 0; k < rounds; k++)
      if (first + 64 * k < n) newest = max(newest, pos[first + 64 * k]);
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) newest = max(newest, __shfl_xor(newest, o, 64));
  if (lane == 0) part[0][wave] = newest;
  if (tid < 9) count[tid / 3][tid % 3] = 0;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < W; w++) newest = max(newest, part[0][w]);
  if constexpr (KPT > 0) {
#pragma unroll
    for (int k = 0; k < KPT; k++) rkey[k] = first + 64 * k < n ? evict_key(rpos[k], rw[k], sink, recent, newest) : 0;
  }
  // key of this lane's k-th slot, 0 behind the last one
  auto key = [&](int k) -> uint32_t {
    if constexpr (KPT > 0) return rkey[k];
    const int i = first + 64 * k;
    return i < n ? evict_key(pos[i], wgt[i], sink, recent, newest) : 0;
  };

  uint32_t thr = 0;
  for (int step = 0; step < 16; step++) {
    const uint32_t unit = 1u << (30 - 2 * step);
    int c1 = 0, c2 = 0, c3 = 0;
#pragma unroll UN
    for (int k = 0; k < rounds; k++) {
      const uint32_t x = key(k);
      c1 += __popcll(__ballot(x >= thr + unit));
      c2 += __popcll(__ballot(x >= thr + 2 * unit));
      c3 += __popcll(__ballot(x >= thr + 3 * unit));
    }
    int* now = count[step % 3];
    if (lane == 0) {
      atomicAdd(now, c1);
      atomicAdd(now + 1, c2);
      atomicAdd(now + 2, c3);
    }
    if (tid < 3) count[(step + 1) % 3][tid] = 0;  // (last read two barriers ago)
    __syncthreads();
    thr += now[2] >= budget ? 3 * unit : now[1] >= budget ? 2 * unit : now[0] >= budget ? unit : 0;
  }

  int above = 0, equal = 0;
#pragma unroll UN
  for (int k = 0; k < rounds; k++) {
    above += __popcll(__ballot(key(k) > thr));
    equal += __popcll(__ballot(key(k) == thr));
  }
  if (lane == 0) {
    part[1][wave] = above;
    part[2][wave] = equal;
  }
  __syncthreads();
  int room = budget, equal_at = 0;  // equal keys that stay; rank of this wavefront's first one
#pragma unroll
  for (int w = 0; w < W; w++) {
    room -= part[1][w];
    equal_at += w < wave ? part[2][w] : 0;
  }
  const unsigned long long below = (1ull << lane) - 1;
  // whether this lane's k-th slot stays; call for every k in turn, `at` the rank of the next equal key
  auto stays = [&](int k, int& at) -> bool {
    const uint32_t x = key(k);
    const unsigned long long eq = __ballot(x == thr);
    const bool yes = x > thr || (x == thr && at + __popcll(eq & below) < room);
    at += __popcll(eq);
    return yes;
  };
  uint32_t kept = 0;
  int freed = 0, moved = 0, at = equal_at;
#pragma unroll UN
  for (int k = 0; k < rounds; k++) {
    const bool yes = stays(k, at);
    if constexpr (KPT > 0) kept |= (uint32_t)yes << k;
    const int i = first + 64 * k;
    freed += __popcll(__ballot(i < budget && !yes));
    moved += __popcll(__ballot(i >= budget && yes));
  }
  if (lane == 0) {
    part[0][wave] = freed;
    part[3][wave] = moved;
  }
  __syncthreads();
  int freed_at = 0, moved_at = 0;
#pragma unroll
  for (int w = 0; w < W; w++) {
    freed_at += w < wave ? part[0][w] : 0;
    moved_at += w < wave ? part[3][w] : 0;
  }
  at = equal_at;
#pragma unroll UN
  for (int k = 0; k < rounds; k++) {
    bool yes;
    if constexpr (KPT > 0) yes = kept >> k & 1; else yes = stays(k, at);
    const int i = first + 64 * k;
    const bool go = i >= budget && yes;
    const unsigned long long who = __ballot(go);
    const int rank = moved_at + __popcll(who & below);
    if (go) {
      if constexpr (KPT > 0) moved_lds[rank] = (uint16_t)i; else list[bh * budget + rank] = i;
    }
    moved_at += __popcll(who);
  }
  __syncthreads();
  at = equal_at;
#pragma unroll UN
  for (int k = 0; k < rounds; k++) {
    bool yes;
    if constexpr (KPT > 0) yes = kept >> k & 1; else yes = stays(k, at);
    const int i = first + 64 * k;
    const bool gone = i < budget && !yes;
    const unsigned long long who = __ballot(gone);
    const int rank = freed_at + __popcll(who & below);
    if (i < budget) {
      int from = i;
      if (gone) {
        if constexpr (KPT > 0) from = moved_lds[rank]; else from = list[bh * budget + rank];
      }
      src[i] = from;
    }
    freed_at += __popcll(who);
  }
}

// Rows to their places: a row's 16-byte vectors side by side, EV_ROWS rows of keys and values of a thread in flight.
constexpr int EV_ROWS = 4;
__global__ __launch_bounds__(256) void evict_move_kernel(const int32_t* __restrict__ len, const int32_t* __restrict__ source, const uint4* K,
                                                         const uint4* V, const int32_t* pos, const float* weight, uint4* Ko, uint4* Vo,
                                                         int32_t* po, float* wo, int Hk, int cap, int out_cap, int max_len, int budget,
                                                         int vecs, int chunks, int in_place) {
  const size_t bh = blockIdx.x / chunks;
  const int per = 256 / vecs, v = threadIdx.x % vecs, first = (int)(blockIdx.x % chunks) * per * EV_ROWS + threadIdx.x / vecs;
  const int n = min(clamp_len(len[bh / Hk], max_len), budget);
  int s[EV_ROWS];
  uint4 k[EV_ROWS], w[EV_ROWS];
#pragma unroll
  for (int r = 0; r < EV_ROWS; r++) {
    const int j = first + r * per;
    s[r] = j < n ? source[bh * budget + j] : -1;
    if (in_place && s[r] == j) s[r] = -1;
  }
#pragma unroll
  for (int r = 0; r < EV_ROWS; r++)
    if (s[r] >= 0) {
      k[r] = K[(bh * cap + s[r]) * vecs + v];
      w[r] = V[(bh * cap + s[r]) * vecs + v];
    }
#pragma unroll
  for (int r = 0; r < EV_ROWS; r++)
    if (s[r] >= 0) {
      const size_t to = bh * out_cap + first + r * per;
      Ko[to * vecs + v] = k[r];
      Vo[to * vecs + v] = w[r];
      if (v == 0) {
        po[to] = pos[bh * cap + s[r]];
        wo[to] = weight[bh * cap + s[r]];
      }
    }
}

// The most slots of the variants that keep keys in registers.
constexpr int EV_SMALL = 256 * 4, EV_MIDDLE = 1024 * 4, EV_LARGE = 1024 * 32;

size_t evict_bytes(const CachePlan& pl) {  // where rows come from; beyond the registers the list of survivors
  return (size_t)pl.B * pl.Hk * pl.budget * 4 * (pl.cap > EV_LARGE ? 2 : 1);
}

}  // namespace tc

using namespace tc;

extern "C" int tc_cache_evict(const tc_cache* c, const int32_t* len, const void* K_cache, const void* V_cache, const int32_t* slot_pos,
                              const float* weight, void* K_out, void* V_out, int32_t* pos_out, float* weight_out, int32_t out_capacity,
                              int32_t* len_out, void* ws, size_t ws_bytes, void* stream) {
  CachePlan pl;
  int rc = make_cache_plan(c, &pl);
  if (rc != TC_OK) return rc;
  if (pl.budget < 1) return TC_ERR_PARAM;
  if (pl.B == 0) return TC_OK;
  if (!len || !K_cache || !V_cache || !slot_pos || !weight || !K_out || !V_out || !pos_out || !weight_out || !len_out) return TC_ERR_NULL;
  if (out_capacity < pl.budget) return TC_ERR_SHAPE;
  if (misaligned(len) || misaligned(K_cache) || misaligned(V_cache) || misaligned(slot_pos) || misaligned(weight) || misaligned(K_out) ||
      misaligned(V_out) || misaligned(pos_out) || misaligned(weight_out) || misaligned(len_out))
    return TC_ERR_ALIGN;
  const int same = (K_out == K_cache) + (V_out == V_cache) + (pos_out == slot_pos) + (weight_out == weight);
  if ((same != 0 && same != 4) || (same == 4 && out_capacity != pl.cap) || len_out == len) return TC_ERR_PARAM;
  if ((rc = check_cache_ws(pl, ws, ws_bytes)) != TC_OK) return rc;
  const hipStream_t st = (hipStream_t)stream;
  int32_t* source = at<int32_t>(ws, 0);
  int32_t* list = source + (size_t)pl.B * pl.Hk * pl.budget;
  const unsigned heads = (unsigned)(pl.B * pl.Hk);  // at most 2^26
#define TC_EVICT(NT_, KPT_)                                                                                                             \
  evict_select_kernel<NT_, KPT_><<<heads, NT_, 0, st>>>(len, slot_pos, weight, source, list, len_out, pl.Hk, pl.cap, pl.max_len, pl.budget, \
                                                        pl.sink, pl.recent)
  if (pl.max_len <= EV_SMALL)
    TC_EVICT(256, 4);
  else if (pl.max_len <= EV_MIDDLE)
    TC_EVICT(1024, 4);
  else if (pl.max_len <= EV_LARGE)
    TC_EVICT(1024, 32);
  else
    TC_EVICT(1024, 0);
#undef TC_EVICT
  if (same == 4 && pl.max_len <= pl.budget) return check_launch();  // nothing can move
  const int vecs = pl.dh * pl.esize / 16, rows = 256 / vecs * EV_ROWS, most = pl.max_len < pl.budget ? pl.max_len : pl.budget;
  const int chunks = (most + rows - 1) / rows;
  if ((long long)heads * chunks > 0x7fffffffLL) return TC_ERR_SHAPE;
  evict_move_kernel<<<heads * chunks, 256, 0, st>>>(len, source, (const uint4*)K_cache, (const uint4*)V_cache, slot_pos, weight, (uint4*)K_out,
                                                    (uint4*)V_out, pos_out, weight_out, pl.Hk, pl.cap, out_capacity, pl.max_len, pl.budget, vecs,
                                                    chunks, same == 4);
  return check_launch();
}
