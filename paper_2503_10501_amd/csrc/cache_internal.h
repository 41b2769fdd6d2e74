// What the translation units behind the compression share: rows of 16 bytes in each storage type, and the checks of rotary parameters.
#pragma once
#include "tc_internal.h"

namespace tc {

// N elements of storage type T in 16 bytes (T = uint16_t: bf16, f16_t: half).
template <typename T> struct Vec16 {
  static constexpr int N = 8;
  __device__ static inline void unpack(const uint4& w, float* f) {
    unpack2<T>(w.x, f, f + 1);
    unpack2<T>(w.y, f + 2, f + 3);
    unpack2<T>(w.z, f + 4, f + 5);
    unpack2<T>(w.w, f + 6, f + 7);
  }
  __device__ static inline uint4 pack(const float* f) {
    return uint4{pack2<T>(f[0], f[1]), pack2<T>(f[2], f[3]), pack2<T>(f[4], f[5]), pack2<T>(f[6], f[7])};
  }
  __device__ static inline float one(T v) {
    float lo, hi;
    unpack2<T>((uint32_t)__builtin_bit_cast(uint16_t, v), &lo, &hi);
    return lo;
  }
  __device__ static inline T round(float f) { return __builtin_bit_cast(T, (uint16_t)pack2<T>(f, 0.f)); }
};
template <> struct Vec16<float> {
  static constexpr int N = 4;
  __device__ static inline void unpack(const uint4& w, float* f) {
    f[0] = __uint_as_float(w.x); f[1] = __uint_as_float(w.y); f[2] = __uint_as_float(w.z); f[3] = __uint_as_float(w.w);
  }
  __device__ static inline uint4 pack(const float* f) {
    return uint4{__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])};
  }
  __device__ static inline float one(float v) { return v; }
  __device__ static inline float round(float f) { return f; }
};

inline int elem_size(int dtype) { return dtype == TC_F32 ? 4 : 2; }
inline bool known_dtype(int dtype) { return dtype == TC_F32 || dtype == TC_BF16 || dtype == TC_F16; }

int check_rope(const tc_rope* r);  // tc_status
inline int rope_dim(const tc_rope* r) { return r->rot_dim > 0 ? r->rot_dim : r->head_dim; }

// Strides along which there is more than one entry (`output`: rows of `width` elements that are written, which must not overlap).
inline bool bad_strides(const tc_strides* s, int esize, int batch, int heads, int rows, int width, bool output) {
  const int64_t v[3] = {s->batch, s->head, s->row};
  const int n[3] = {batch, heads, rows};
  for (int i = 0; i < 3; i++)
    if (n[i] > 1 && (v[i] < 0 || v[i] > (int64_t(1) << 44) || v[i] * esize % 16 != 0 || (output && v[i] < width))) return true;
  return false;
}

// A call on the cache, checked.
struct CachePlan {
  int B, H, Hk, G, dh, T, cap, max_len, images, each, P, esize;
  int R;         // rows of queries per sequence and key/value head: the G heads that share it, T rows each, head after head
  float scale;
  int budget, sink, recent;
  size_t total;  // bytes of workspace
};
int make_cache_plan(const tc_cache* c, CachePlan* plan);
size_t evict_bytes(const CachePlan& pl);
size_t attention_bytes(const CachePlan& pl);

inline int check_cache_ws(const CachePlan& pl, const void* ws, size_t ws_bytes) {
  if (!ws) return TC_ERR_NULL;
  if (misaligned(ws)) return TC_ERR_ALIGN;
  return ws_bytes < pl.total ? TC_ERR_WORKSPACE : TC_OK;
}

// Workgroups of a launch and their threads: a grid counts its threads in 32 bits.
inline bool grid_fits(long long workgroups, int threads) { return workgroups * threads < (1LL << 32); }

__device__ inline int clamp_len(int n, int most) { return n < 0 ? 0 : (n > most ? most : n); }

}  // namespace tc
