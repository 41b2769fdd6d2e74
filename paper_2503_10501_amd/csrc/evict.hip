// Eviction from the cache by the attention that slots have gathered: which slots stay, and where their rows go.
//
// What stays is a set of slots, and attention does not ask for their order: a slot below the budget that stays keeps its place, and only the
// survivors behind it move, into the freed places.  Sources (at or behind the budget) and destinations (below it) never meet, so all rows move at
// once, in place too; a step that drops one token moves one row of each head.
#include "cache_internal.h"

namespace tc {

// A slot's place in the order, larger is better: protected slots (position below `sink`, or `late` and above) first, then weights descending
// (+0 and -0 alike), NaN last.  Never 0.
__device__ inline uint32_t evict_key(int pos, float w, int sink, bool any_late, int late) {
  const uint32_t key = (uint32_t)(order_key(w == w ? w : -INFINITY, 0) >> 32);
  return pos < sink || (any_late && pos >= late) ? 0xffffffffu : key;
}

// Sum (or largest) over the 16 lanes of a row, in each of them.
template <typename F>
__device__ inline int row16(int x, F f) {
  x = f(x, __builtin_amdgcn_mov_dpp(x, 0xB1, 0xF, 0xF, false));   // quad_perm [1,0,3,2]
  x = f(x, __builtin_amdgcn_mov_dpp(x, 0x4E, 0xF, 0xF, false));   // quad_perm [2,3,0,1]
  x = f(x, __builtin_amdgcn_mov_dpp(x, 0x141, 0xF, 0xF, false));  // row_half_mirror
  return f(x, __builtin_amdgcn_mov_dpp(x, 0x140, 0xF, 0xF, false));  // row_mirror
}
__device__ inline int row16_sum(int x) {
  return row16(x, [](int a, int b) { return a + b; });
}

struct EvictArgs {
  const int32_t *len, *slot_pos;
  const float* weight;
  int32_t *source, *list, *len_out;
  int Hk, cap, max_len, budget, sink, recent;
  // moves that the selection makes itself, in place
  uint4 *K, *V;
  int32_t* pos_out;
  float* weight_out;
  int vecs;
};
constexpr int EV_FUSED = 64;  // at most so many slots beyond the budget: the selection moves their rows itself (one launch in place of two)

// One workgroup per sequence and head.  The slots are dealt to the wavefronts in runs, a run's 64 lanes side by side, KPT keys of a lane in
// registers (KPT = 0: any number of slots, the keys formed anew each time).  The threshold, the largest key that at least `budget` slots reach, is
// found two bits at a time from counts of three candidates, until one is reached by `budget` slots exactly; equal keys stay from the lowest
// slot on.  Then each freed place takes the survivor of its rank.  A chain of at most 16 counts and barriers bounds it, not its bytes (8 for a slot):
// 8 x 32 heads of up to 2944 slots 12.9 us; counts by atomics on a histogram in LDS took longer than a wavefront's ballots.
template <int NT, int KPT, bool FUSED>
__global__ __launch_bounds__(NT) void evict_select_kernel(EvictArgs a) {
  constexpr int W = NT / 64, UN = KPT > 0 ? KPT : 1;
  static_assert(W <= 16, "what wavefronts say to one another is read by a row of 16 lanes");
  __shared__ int part[5][W], count[2][2][W];
  __shared__ uint16_t moved_lds[KPT > 0 && !FUSED ? NT * KPT / 2 : 1];         // at most half of the slots move
  __shared__ int from[FUSED ? EV_FUSED : 1], to[FUSED ? EV_FUSED : 1];
  const int Hk = a.Hk, cap = a.cap, budget = a.budget, sink = a.sink, recent = a.recent;
  const size_t bh = blockIdx.x;
  const int b = (int)(bh / Hk), tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = clamp_len(a.len[b], a.max_len);
  if (bh % Hk == 0 && tid == 0) a.len_out[b] = min(n, budget);
  int32_t* src = a.source + bh * budget;
  if (n <= budget) {
    if (FUSED) return;
    for (int j = tid; j < n; j += NT) src[j] = j;
    return;
  }
  const int32_t* pos = a.slot_pos + bh * cap;
  const float* wgt = a.weight + bh * cap;
  const int rounds = KPT > 0 ? KPT : (n + NT - 1) / NT, first = wave * 64 * rounds + lane;

  int newest = INT32_MIN;
  int rpos[KPT > 0 ? KPT : 1];
  float rw[KPT > 0 ? KPT : 1];
  uint32_t rkey[KPT > 0 ? KPT : 1];
  if constexpr (KPT > 0) {
#pragma unroll
    for (int k = 0; k < KPT; k++) {
      const int i = first + 64 * k;
      rpos[k] = pos[min(i, n - 1)];  // (behind the last slot that one again)
      rw[k] = wgt[min(i, n - 1)];
    }
#pragma unroll
    for (int k = 0; k < KPT; k++) newest = max(newest, rpos[k]);
  } else {
    for (int k = 0; k < rounds; k++)
      if (first + 64 * k < n) newest = max(newest, pos[first + 64 * k]);
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) newest = max(newest, __shfl_xor(newest, o, 64));
  const int other = min(lane & 15, W - 1);  // the wavefront whose word this lane reads
  const bool each = (lane & 15) < W, before = (lane & 15) < wave;
  if (lane == 0) part[0][wave] = newest;
  __syncthreads();
  newest = row16(part[0][other], [](int a, int b) { return max(a, b); });
  const long long from_late = (long long)newest - recent + 1;
  const int late = from_late < INT32_MIN ? INT32_MIN : (int)from_late;
  const bool any_late = recent > 0;
  if constexpr (KPT > 0) {
#pragma unroll
    for (int k = 0; k < KPT; k++) rkey[k] = first + 64 * k < n ? evict_key(rpos[k], rw[k], sink, any_late, late) : 0;
  }
  // key of this lane's k-th slot, 0 behind the last one
  auto key = [&](int k) -> uint32_t {
    if constexpr (KPT > 0) return rkey[k];
    const int i = first + 64 * k;
    return i < n ? evict_key(pos[i], wgt[i], sink, any_late, late) : 0;
  };

  static_assert(NT * KPT < 1 << 16, "two counts in a word");
  uint32_t thr = 0;
  int seen = n;  // slots that reach thr
  // (two bits a step; without registers a step is a sweep over the slots, and counts pass 16 bits: one bit)
  constexpr int BITS = KPT > 0 ? 2 : 1;
  for (int shift = 32 - BITS; shift >= 0 && seen != budget; shift -= BITS) {
    const uint32_t unit = 1u << shift;
    unsigned c1 = 0, c2 = 0, c3 = 0;
#pragma unroll UN
    for (int k = 0; k < rounds; k++) {
      const uint32_t x = key(k);
      c1 += __popcll(__ballot(x >= thr + unit));
      if constexpr (BITS == 2) {
        c2 += __popcll(__ballot(x >= thr + 2 * unit));
        c3 += __popcll(__ballot(x >= thr + 3 * unit));
      }
    }
    int(&now)[2][W] = count[shift / BITS % 2];  // (the other one is still being read)
    if (lane == 0) {
      now[0][wave] = (int)(c1 | c2 << 16);
      if constexpr (BITS == 2) now[1][wave] = (int)c3;
    }
    __syncthreads();
    const unsigned s12 = (unsigned)row16_sum(each ? now[0][other] : 0);
    int s1 = (int)s12, s2 = 0, s3 = 0;
    if constexpr (BITS == 2) {
      s3 = row16_sum(each ? now[1][other] : 0);
      s1 = (int)(s12 & 0xffffu);
      s2 = (int)(s12 >> 16);
    }
    const int up = s3 >= budget ? 3 : s2 >= budget ? 2 : s1 >= budget ? 1 : 0;
    thr += up * unit;
    seen = up == 3 ? s3 : up == 2 ? s2 : up == 1 ? s1 : seen;
    thr = __builtin_amdgcn_readfirstlane(thr);
    seen = __builtin_amdgcn_readfirstlane(seen);
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
  // equal keys that stay; rank of this wavefront's first one
  const int room = __builtin_amdgcn_readfirstlane(budget - row16_sum(each ? part[1][other] : 0));
  const int equal_at = __builtin_amdgcn_readfirstlane(row16_sum(before ? part[2][other] : 0));
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
    part[3][wave] = freed;
    part[4][wave] = moved;
  }
  __syncthreads();
  int freed_at = __builtin_amdgcn_readfirstlane(row16_sum(before ? part[3][other] : 0));
  int moved_at = __builtin_amdgcn_readfirstlane(row16_sum(before ? part[4][other] : 0));
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
      if constexpr (FUSED) from[rank] = i;
      else if constexpr (KPT > 0) moved_lds[rank] = (uint16_t)i;
      else a.list[bh * budget + rank] = i;
    }
    moved_at += __popcll(who);
  }
  if constexpr (!FUSED) __syncthreads();
  at = equal_at;
#pragma unroll UN
  for (int k = 0; k < rounds; k++) {
    bool yes;
    if constexpr (KPT > 0) yes = kept >> k & 1; else yes = stays(k, at);
    const int i = first + 64 * k;
    const bool gone = i < budget && !yes;
    const unsigned long long who = __ballot(gone);
    const int rank = freed_at + __popcll(who & below);
    if constexpr (FUSED) {
      if (gone) to[rank] = i;
    } else if (i < budget) {
      int come = i;
      if (gone) {
        if constexpr (KPT > 0) come = moved_lds[rank]; else come = a.list[bh * budget + rank];
      }
      src[i] = come;
    }
    freed_at += __popcll(who);
  }
  if constexpr (FUSED) {
    __syncthreads();
    const int rows = row16_sum(each ? part[4][other] : 0);  // at most n - budget <= EV_FUSED
    for (int x = tid; x < rows * a.vecs; x += NT) {
      const int r = x / a.vecs, v = x % a.vecs;
      const size_t come = (bh * cap + from[r]) * a.vecs + v, go = (bh * cap + to[r]) * a.vecs + v;
      const uint4 k = a.K[come], w = a.V[come];
      a.K[go] = k;
      a.V[go] = w;
      if (v == 0) {
        a.pos_out[bh * cap + to[r]] = pos[from[r]];
        a.weight_out[bh * cap + to[r]] = wgt[from[r]];
      }
    }
  }
}

// Rows to their places: a row's 16-byte vectors side by side, one of keys and one of values for a thread.  (8 x 32 heads, 640 rows of 256 bytes each out
// of up to 2944: 27 us, 5.8 TB/s; two rows a thread 36, four 52: the loads of rows that may not move are not issued together.)
__global__ __launch_bounds__(256) void evict_move_kernel(const int32_t* __restrict__ len, const int32_t* __restrict__ source, const uint4* K,
                                                         const uint4* V, const int32_t* pos, const float* weight, uint4* Ko, uint4* Vo,
                                                         int32_t* po, float* wo, int Hk, int cap, int out_cap, int max_len, int budget,
                                                         int vecs, int chunks, int in_place) {
  const unsigned bh = blockIdx.x / chunks;
  const int v = threadIdx.x % vecs, j = (int)(blockIdx.x % chunks) * (256 / vecs) + threadIdx.x / vecs;
  if (j >= min(clamp_len(len[bh / Hk], max_len), budget)) return;
  const int s = source[(size_t)bh * budget + j];
  if (in_place && s == j) return;
  const size_t from = (size_t)bh * cap + s, to = (size_t)bh * out_cap + j;
  const uint4 k = K[from * vecs + v], w = V[from * vecs + v];
  Ko[to * vecs + v] = k;
  Vo[to * vecs + v] = w;
  if (v == 0) {
    po[to] = pos[from];
    wo[to] = weight[from];
  }
}

// The most slots of the variants that keep keys in registers.  (1136 heads of up to 1790 slots: 36 us by 512 threads a head, 26 by 256; 256 heads of 2944
// 41 by 512 threads, 42 by 1024, 45 by 256.  8 heads of up to 8000 and 12000 slots, with 8 and 16 keys a thread 20 and 28; with 32, whose masks pass the
// scalar registers, 58 and 56.)
constexpr int EV_SMALL = 256 * 4, EV_HALF = 256 * 8, EV_MIDDLE = 512 * 8, EV_DOUBLE = 1024 * 8, EV_QUADRUPLE = 1024 * 16, EV_LARGE = 1024 * 32;

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
  const int vecs = pl.dh * pl.esize / 16;
  EvictArgs a = {len, slot_pos, weight, source, list, len_out, pl.Hk, pl.cap, pl.max_len, pl.budget, pl.sink, pl.recent, (uint4*)K_out, (uint4*)V_out,
                 pos_out, weight_out, vecs};
  const bool fused = same == 4 && pl.max_len - pl.budget <= EV_FUSED;
  const int rows = 256 / vecs, most = pl.max_len < pl.budget ? pl.max_len : pl.budget, chunks = (most + rows - 1) / rows;
  const int threads = pl.max_len <= EV_HALF ? 256 : pl.max_len <= EV_MIDDLE ? 512 : 1024;
  if (!grid_fits(heads, threads) || (!fused && !grid_fits((long long)heads * chunks, 256))) return TC_ERR_SHAPE;
#define TC_EVICT(NT_, KPT_)                                        \
  do {                                                             \
    if (fused)                                                     \
      evict_select_kernel<NT_, KPT_, true><<<heads, NT_, 0, st>>>(a);  \
    else                                                           \
      evict_select_kernel<NT_, KPT_, false><<<heads, NT_, 0, st>>>(a); \
  } while (0)
  if (pl.max_len <= EV_SMALL)
    TC_EVICT(256, 4);
  else if (pl.max_len <= EV_HALF)
    TC_EVICT(256, 8);
  else if (pl.max_len <= EV_MIDDLE)
    TC_EVICT(512, 8);
  else if (pl.max_len <= EV_DOUBLE)
    TC_EVICT(1024, 8);
  else if (pl.max_len <= EV_QUADRUPLE)
    TC_EVICT(1024, 16);
  else if (pl.max_len <= EV_LARGE)
    TC_EVICT(1024, 32);
  else
    TC_EVICT(1024, 0);
#undef TC_EVICT
  if (fused) return check_launch();
  evict_move_kernel<<<heads * chunks, 256, 0, st>>>(len, source, (const uint4*)K_cache, (const uint4*)V_cache, slot_pos, weight, (uint4*)K_out,
                                                    (uint4*)V_out, pos_out, weight_out, pl.Hk, pl.cap, out_capacity, pl.max_len, pl.budget, vecs,
                                                    chunks, same == 4);
  return check_launch();
}
