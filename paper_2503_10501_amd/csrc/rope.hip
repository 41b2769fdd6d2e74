// Rotary positions: the tables of any positions, and their application to the rows of heads.  Pair (a, b) of a row is the complex number
// a + i b, a position turns it by its angle; the transposed turn is the gradient.
#include <cmath>

#include "cache_internal.h"

namespace tc {

int check_rope(const tc_rope* r) {
  if (!r) return TC_ERR_NULL;
  if ((r->head_dim != 64 && r->head_dim != 128) || r->rot_dim < 0 || r->rot_dim > r->head_dim || r->rot_dim % 2 != 0) return TC_ERR_SHAPE;
  if ((r->layout != TC_ROPE_HALF && r->layout != TC_ROPE_INTERLEAVED) || r->scaling < TC_ROPE_PLAIN || r->scaling > TC_ROPE_BANDS ||
      !(r->base > 1.f) || !std::isfinite(r->base) || !(r->magnitude >= 0.f) || !std::isfinite(r->magnitude))
    return TC_ERR_PARAM;
  if (r->scaling != TC_ROPE_PLAIN && (!(r->factor >= 1.f) || !std::isfinite(r->factor))) return TC_ERR_PARAM;
  if (r->scaling == TC_ROPE_BASE && rope_dim(r) <= 2) return TC_ERR_PARAM;
  if (r->scaling == TC_ROPE_BANDS &&
      (r->original_len < 1 || !(r->low >= 0.f) || !(r->high > r->low) || !std::isfinite(r->high)))
    return TC_ERR_PARAM;
  return TC_OK;
}

// Sine and cosine of an angle of at most 2^31: the nearest multiple of pi/2 is taken off in two parts (the first product is exact inside the
// multiply-add, what it rounds is below 2^-53), then the Taylor series up to 1/13! and 1/14!, whose next terms are below 2^-45 at pi/4:
// far inside the rounding to float32.  (The library's routine, which serves any angle: 13.6 us for 23552 positions of 64 pairs, this 9.)
__device__ inline void sin_cos(double x, double* sn, double* cs) {
  const double q = rint(x * 0.63661977236758134308);  // 2 / pi
  double r = fma(-q, 1.5707963267948965580, x);
  r = fma(-q, 6.1232339957367658860e-17, r);
  const double z = r * r;
  double s = 1.0 / 6227020800.0, c = -1.0 / 87178291200.0;
  s = fma(s, z, -1.0 / 39916800.0); c = fma(c, z, 1.0 / 479001600.0);
  s = fma(s, z, 1.0 / 362880.0);    c = fma(c, z, -1.0 / 3628800.0);
  s = fma(s, z, -1.0 / 5040.0);     c = fma(c, z, 1.0 / 40320.0);
  s = fma(s, z, 1.0 / 120.0);       c = fma(c, z, -1.0 / 720.0);
  s = fma(s, z, -1.0 / 6.0);        c = fma(c, z, 1.0 / 24.0);
  s = fma(s * z, r, r);             c = fma(c, z, -0.5);
  c = fma(c, z, 1.0);
  const int k = (int)q;
  const double a = k & 1 ? c : s, b = k & 1 ? s : c;
  *sn = k & 2 ? -a : a;
  *cs = (k + 1) & 2 ? -b : b;
}

// One thread has one pair's angle per position, an exponential in float64, and goes over some positions, one after another: a load and some thirty
// float64 operations that wait for each other.  Up to some thousand positions the launch and that chain bound it (16 pairs, 2103 positions 3.2 us; a single
// position 2.0), above that the chains of up to eight positions a thread (64 pairs, 23552 positions 9.0 us for 12 MB, which alone would take 2.4).
__global__ __launch_bounds__(256) void rope_tables_kernel(const int32_t* __restrict__ pos, long long n, float* __restrict__ c,
                                                          float* __restrict__ s, int half, double log_base, int scaling, double factor,
                                                          double original_len, double low, double high, double magnitude, int per) {
  const int k = threadIdx.x % half, rows = 256 / half;
  if ((int)threadIdx.x >= rows * half) return;
  double theta = exp(-(double)k / (double)half * log_base);
  if (scaling == TC_ROPE_LINEAR) theta /= factor;
  if (scaling == TC_ROPE_BANDS) {
    const double turns = original_len * theta * 0.15915494309189533577;  // 1 / 2 pi
    const double g = fmin(fmax((turns - low) / (high - low), 0.0), 1.0);
    theta *= g + (1.0 - g) / factor;
  }
  const long long first = (long long)blockIdx.x * per * rows + threadIdx.x / half;
  for (int j = 0; j < per; j++) {
    const long long i = first + (long long)j * rows;
    if (i >= n) return;
    double sn, cs;
    sin_cos((double)pos[i] * theta, &sn, &cs);
    c[i * half + k] = (float)(cs * magnitude);
    s[i * half + k] = (float)(sn * magnitude);
  }
}

// The elements of a head are dealt to threads in items: VEC: the 16-byte vectors of a pair of halves (or one, whose pairs are
// neighbours), behind them vectors that are copied; else single pairs, behind them single elements.  (64 x 128 tokens, 32 heads of 128, bf16: vectors 23 to 25
// us; single pairs 113 for r = 24 in halves, mostly single elements, 70 for r = 126.)
__host__ __device__ inline int rope_items(int dh, int r, int n16, bool inter, bool vec) {
  if (vec) return inter ? dh / n16 : dh / n16 - r / (2 * n16);
  return r / 2 + dh - r;
}
template <typename T>
inline bool rope_vec(int r, bool inter) { return r % ((inter ? 1 : 2) * Vec16<T>::N) == 0; }

// What an item needs of the tables, and the turn of a head's item.  `sign`: -1 for the transposed turn.
template <typename T, bool INTER, bool VEC>
struct RopeItem {
  static constexpr int N = Vec16<T>::N, NT = VEC ? (INTER ? N / 2 : N) : 1;
  float c[NT], s[NT];
  int item, r;
  bool turned;
  __device__ inline RopeItem(const float* cs, const float* sn, int item_, int r_, float sign) : item(item_), r(r_) {
    turned = item < (VEC ? (INTER ? r / N : r / (2 * N)) : r / 2);
    if (turned && cs) {
#pragma unroll
      for (int k = 0; k < NT; k++) {
        c[k] = cs[item * NT + k];
        s[k] = sign * sn[item * NT + k];
      }
    }
  }
  struct Data { uint4 a, b; };
  __device__ inline void load(const T* x, Data& v) const {
    if constexpr (VEC) {
      const uint4* p = reinterpret_cast<const uint4*>(x);
      v.a = p[INTER || turned ? item : item + r / (2 * N)];
      if (!INTER && turned) v.b = p[item + r / (2 * N)];
    } else {
      v.a.x = __float_as_uint(Vec16<T>::one(x[turned ? (INTER ? 2 * item : item) : item + r / 2]));
      if (turned) v.b.x = __float_as_uint(Vec16<T>::one(x[INTER ? 2 * item + 1 : item + r / 2]));
    }
  }
  __device__ inline void turn(Data& v) const {
    if (!turned) return;
    if constexpr (VEC && INTER) {
      float f[N];
      Vec16<T>::unpack(v.a, f);
#pragma unroll
      for (int k = 0; k < NT; k++) {
        const float a = f[2 * k], b = f[2 * k + 1];
        f[2 * k] = a * c[k] - b * s[k];
        f[2 * k + 1] = b * c[k] + a * s[k];
      }
      v.a = Vec16<T>::pack(f);
    } else if constexpr (VEC) {
      float a[N], b[N];
      Vec16<T>::unpack(v.a, a);
      Vec16<T>::unpack(v.b, b);
#pragma unroll
      for (int k = 0; k < NT; k++) {
        const float x = a[k], y = b[k];
        a[k] = x * c[k] - y * s[k];
        b[k] = y * c[k] + x * s[k];
      }
      v.a = Vec16<T>::pack(a);
      v.b = Vec16<T>::pack(b);
    } else {
      const float a = __uint_as_float(v.a.x), b = __uint_as_float(v.b.x);
      v.a.x = __float_as_uint(a * c[0] - b * s[0]);
      v.b.x = __float_as_uint(b * c[0] + a * s[0]);
    }
  }
  __device__ inline void store(T* y, const Data& v) const {
    if constexpr (VEC) {
      uint4* p = reinterpret_cast<uint4*>(y);
      p[INTER || turned ? item : item + r / (2 * N)] = v.a;
      if (!INTER && turned) p[item + r / (2 * N)] = v.b;
    } else {
      y[turned ? (INTER ? 2 * item : item) : item + r / 2] = Vec16<T>::round(__uint_as_float(v.a.x));
      if (turned) y[INTER ? 2 * item + 1 : item + r / 2] = Vec16<T>::round(__uint_as_float(v.b.x));
    }
  }
};

// Token, head and item of a thread: items fastest, then heads, then tokens.
struct RopeThread {
  long long token;
  int head, item;
};
__device__ inline RopeThread rope_thread(int items, int heads) {
  const unsigned per = (unsigned)(items * heads);
  const unsigned long long at = (unsigned long long)blockIdx.x * 256;
  const unsigned long long t0 = at / per;
  const unsigned off = (unsigned)(at - t0 * per) + threadIdx.x, in = off % per;
  return {(long long)(t0 + off / per), (int)(in / (unsigned)items), (int)(in % (unsigned)items)};
}

// One item a thread: the memory's rate bounds it, and what a thread reads of the tables its neighbours' heads have just read.  (64 x 128 tokens, 32 heads
// of 128, bf16: 24.7 us, 5.4 TB/s; two heads a thread, which read the tables once, 26.2, four 29.3: fewer threads with loads in flight.)
template <typename T, bool INTER, bool VEC>
__global__ __launch_bounds__(256) void rope_apply_kernel(const T* x, tc_strides xs, const float* __restrict__ c, const float* __restrict__ s,
                                                         T* y, tc_strides ys, long long tokens, int rows, int heads, int items, int r,
                                                         float sign) {
  const RopeThread me = rope_thread(items, heads);
  if (me.token >= tokens) return;
  const long long b = me.token / rows, t = me.token % rows;
  typedef RopeItem<T, INTER, VEC> Item;
  const Item it(c + me.token * (r / 2), s + me.token * (r / 2), me.item, r, sign);
  typename Item::Data v;
  it.load(x + b * xs.batch + t * xs.row + me.head * xs.head, v);
  it.turn(v);
  it.store(y + b * ys.batch + t * ys.row + me.head * ys.head, v);
}

template <typename T, bool INTER, bool VEC>
static int rope_launch(const tc_rope* p, int batch, int heads, int rows, const void* x, const tc_strides* xs, const float* c, const float* s,
                       void* y, const tc_strides* ys, int transposed, hipStream_t st) {
  const int r = rope_dim(p), items = rope_items(p->head_dim, r, Vec16<T>::N, INTER, VEC);
  const long long tokens = (long long)batch * rows, blocks = (tokens * heads * items + 255) / 256;
  if (!grid_fits(blocks, 256)) return TC_ERR_SHAPE;
  rope_apply_kernel<T, INTER, VEC><<<(unsigned)blocks, 256, 0, st>>>((const T*)x, *xs, c, s, (T*)y, *ys, tokens, rows, heads, items, r,
                                                                     transposed ? -1.f : 1.f);
  return check_launch();
}

// New tokens of a cache: the heads of a token are those of its query, key and value in turn.  Queries and keys are turned, queries go to
// the rows of the output, keys and values to their slots.  One pass, every row read and written once, so that the memory's rate bounds it (64 sequences
// of up to 28 tokens, 32 heads and 8 for keys and values, of 128, bf16: 9.6 us for 30 MB, of which the launch and the lengths' loads are three).
template <typename T, bool INTER, bool VEC>
__global__ __launch_bounds__(256) void append_kernel(const T* __restrict__ Q, tc_strides qs, const T* __restrict__ K, tc_strides ks,
                                                     const T* __restrict__ V, tc_strides vs, const float* __restrict__ c,
                                                     const float* __restrict__ s, const int32_t* __restrict__ pos,
                                                     const int32_t* __restrict__ len, const int32_t* __restrict__ q_len, T* __restrict__ Qo,
                                                     T* __restrict__ Kc, T* __restrict__ Vc, int32_t* __restrict__ slot_pos,
                                                     float* __restrict__ weight, CachePlan pl, int items, int r) {
  const int heads = pl.H + 2 * pl.Hk;
  const RopeThread me = rope_thread(items, heads);
  if (me.token >= (long long)pl.B * pl.T) return;
  const int b = (int)(me.token / pl.T), t = (int)(me.token % pl.T), h = me.head;
  typedef RopeItem<T, INTER, VEC> Item;
  // (without tables nothing is turned: the item's own part of the row is copied)
  const Item it(c ? c + me.token * (r / 2) : c, s ? s + me.token * (r / 2) : s, me.item, r, 1.f);
  const int m = q_len ? clamp_len(q_len[b], pl.T) : pl.T, slot = clamp_len(len[b], pl.max_len) - m + t;
  const bool live = t < m;
  typename Item::Data v;
  if (h < pl.H) {
    if (live) {
      it.load(Q + b * qs.batch + h * qs.head + t * qs.row, v);
      if (c) it.turn(v);
    } else {
      v.a = v.b = uint4{0, 0, 0, 0};
    }
    it.store(Qo + (((size_t)b * pl.H + h) * pl.T + t) * pl.dh, v);
    return;
  }
  if (!live || slot < 0 || slot >= pl.cap) return;
  const bool key = h < pl.H + pl.Hk;
  const int j = h - (key ? pl.H : pl.H + pl.Hk);
  const tc_strides& st = key ? ks : vs;
  const size_t at = ((size_t)b * pl.Hk + j) * pl.cap + slot;
  it.load((key ? K : V) + b * st.batch + j * st.head + t * st.row, v);
  if (key && c) it.turn(v);
  it.store((key ? Kc : Vc) + at * pl.dh, v);
  if (key && me.item == 0) {
    slot_pos[at] = pos[me.token];
    weight[at] = 0.f;
  }
}

template <typename T, bool INTER, bool VEC>
static int append_launch(const CachePlan& pl, int r, const void* Q, const tc_strides* qs, const void* K, const tc_strides* ks, const void* V,
                         const tc_strides* vs, const float* c, const float* s, const int32_t* pos, const int32_t* len, const int32_t* q_len,
                         void* Qo, void* Kc, void* Vc, int32_t* slot_pos, float* weight, hipStream_t st) {
  const int heads = pl.H + 2 * pl.Hk, items = rope_items(pl.dh, r, Vec16<T>::N, INTER, VEC);
  const long long blocks = ((long long)pl.B * pl.T * heads * items + 255) / 256;
  if (!grid_fits(blocks, 256)) return TC_ERR_SHAPE;
  append_kernel<T, INTER, VEC><<<(unsigned)blocks, 256, 0, st>>>((const T*)Q, *qs, (const T*)K, *ks, (const T*)V, *vs, c, s, pos, len, q_len,
                                                                 (T*)Qo, (T*)Kc, (T*)Vc, slot_pos, weight, pl, items, r);
  return check_launch();
}

// F<T, INTER, VEC>(args) for the storage type, the layout and whether the rotated part falls into vectors.
#define TC_ROPE_CALL(F, dtype, r, layout, ...)                                                                     \
  [&]() -> int {                                                                                                   \
    const bool inter = (layout) == TC_ROPE_INTERLEAVED;                                                            \
    auto by = [&](auto tag) -> int {                                                                               \
      typedef decltype(tag) T;                                                                                     \
      if (rope_vec<T>(r, inter)) return inter ? F<T, true, true>(__VA_ARGS__) : F<T, false, true>(__VA_ARGS__); \
      return inter ? F<T, true, false>(__VA_ARGS__) : F<T, false, false>(__VA_ARGS__);                             \
    };                                                                                                             \
    return (dtype) == TC_F32 ? by(0.f) : (dtype) == TC_BF16 ? by(uint16_t(0)) : by(f16_t{0});                      \
  }()

}  // namespace tc

using namespace tc;

extern "C" int tc_rope_tables(const tc_rope* r, const int32_t* pos_ids, int64_t n, float* cos, float* sin, void* stream) {
  const int rc = check_rope(r);
  if (rc != TC_OK) return rc;
  if (n < 0 || n > (int64_t(1) << 36)) return TC_ERR_SHAPE;
  if (n == 0) return TC_OK;
  if (!pos_ids || !cos || !sin) return TC_ERR_NULL;
  if (misaligned(pos_ids) || misaligned(cos) || misaligned(sin)) return TC_ERR_ALIGN;
  const int rd = rope_dim(r), half = rd / 2, rows = 256 / half;
  double log_base = std::log((double)r->base);
  if (r->scaling == TC_ROPE_BASE) log_base += std::log((double)r->factor) * rd / (rd - 2.0);
  const int64_t blocks1 = (n + rows - 1) / rows;
  const int per = blocks1 >= 8 * 1024 ? 8 : blocks1 >= 2 * 1024 ? (int)(blocks1 / 1024) : 1;  // positions of a thread: its angle is worth keeping once the chip is full
  const int64_t blocks = (blocks1 + per - 1) / per;
  if (!grid_fits(blocks, 256)) return TC_ERR_SHAPE;
  rope_tables_kernel<<<(unsigned)blocks, 256, 0, (hipStream_t)stream>>>(pos_ids, n, cos, sin, half, log_base, r->scaling, (double)r->factor,
                                                                        (double)r->original_len, (double)r->low, (double)r->high,
                                                                        r->magnitude > 0.f ? (double)r->magnitude : 1.0, per);
  return check_launch();
}

extern "C" int tc_rope_apply(const tc_rope* r, int32_t dtype, int32_t batch, int32_t n_heads, int32_t n_rows, const void* x,
                             const tc_strides* xs, const float* cos, const float* sin, void* y, const tc_strides* ys,
                             int32_t transposed, void* stream) {
  const int rc = check_rope(r);
  if (rc != TC_OK) return rc;
  if (!known_dtype(dtype)) return TC_ERR_DTYPE;
  if (batch < 0 || batch > (1 << 16) || n_heads < 1 || n_heads > 1024 || n_rows < 0 || n_rows > (1 << 20)) return TC_ERR_SHAPE;
  if (batch == 0 || n_rows == 0) return TC_OK;
  if (!x || !xs || !cos || !sin || !y || !ys) return TC_ERR_NULL;
  const int es = elem_size(dtype);
  if (bad_strides(xs, es, batch, n_heads, n_rows, r->head_dim, false) || bad_strides(ys, es, batch, n_heads, n_rows, r->head_dim, true)) return TC_ERR_SHAPE;
  if (misaligned(x) || misaligned(cos) || misaligned(sin) || misaligned(y)) return TC_ERR_ALIGN;
  if (x == y && ((batch > 1 && xs->batch != ys->batch) || (n_heads > 1 && xs->head != ys->head) || (n_rows > 1 && xs->row != ys->row)))
    return TC_ERR_PARAM;
  return TC_ROPE_CALL(rope_launch, dtype, rope_dim(r), r->layout, r, batch, n_heads, n_rows, x, xs, cos, sin, y, ys, transposed, (hipStream_t)stream);
}

extern "C" int tc_cache_append(const tc_cache* cache, const tc_rope* r, const void* Q, const tc_strides* qs, const void* K,
                               const tc_strides* ks, const void* V, const tc_strides* vs, const float* cos, const float* sin,
                               const int32_t* pos_ids, const int32_t* len, const int32_t* q_len, void* Q_out, void* K_cache, void* V_cache,
                               int32_t* slot_pos, float* weight, void* stream) {
  CachePlan pl;
  int rc = make_cache_plan(cache, &pl);
  if (rc != TC_OK) return rc;
  if (r && (rc = check_rope(r)) != TC_OK) return rc;
  if (r && r->head_dim != pl.dh) return TC_ERR_SHAPE;
  if (pl.B == 0) return TC_OK;
  if (!Q || !qs || !K || !ks || !V || !vs || !pos_ids || !len || !Q_out || !K_cache || !V_cache || !slot_pos || !weight) return TC_ERR_NULL;
  if ((cos == nullptr) != (r == nullptr) || (sin == nullptr) != (r == nullptr)) return TC_ERR_NULL;
  if (bad_strides(qs, pl.esize, pl.B, pl.H, pl.T, pl.dh, false) || bad_strides(ks, pl.esize, pl.B, pl.Hk, pl.T, pl.dh, false) ||
      bad_strides(vs, pl.esize, pl.B, pl.Hk, pl.T, pl.dh, false))
    return TC_ERR_SHAPE;
  if (misaligned(Q) || misaligned(K) || misaligned(V) || misaligned(cos) || misaligned(sin) || misaligned(pos_ids) || misaligned(len) ||
      misaligned(q_len) || misaligned(Q_out) || misaligned(K_cache) || misaligned(V_cache) || misaligned(slot_pos) || misaligned(weight))
    return TC_ERR_ALIGN;
  const int rd = r ? rope_dim(r) : pl.dh;
  return TC_ROPE_CALL(append_launch, cache->dtype, rd, r ? r->layout : TC_ROPE_HALF, pl, rd, Q, qs, K, ks, V, vs, cos, sin, pos_ids, len,
                      q_len, Q_out, K_cache, V_cache, slot_pos, weight, (hipStream_t)stream);
}
