// Attention of a call's tokens over a shared prefix and their own cache, and the attention that slots gather.
//
// The rows of queries of a sequence that read one key/value head, G heads of T rows, lie side by side in Q and are one matrix: row r = g T + t.
// Scores are formed transposed, S^T = K Q^T, on the matrix cores, so that a lane has one row's scores and the probabilities are the operand of
// O^T += V^T P^T as they lie; one pass over the keys with the running maximum and sum of the softmax in base 2.  Keys are split
// between workgroups where rows are few; what these find, (maximum, sum, O), is joined by a second kernel.
#include <cmath>

#include "cache_internal.h"

namespace tc {

typedef __attribute__((ext_vector_type(8))) __bf16 bfrag;
typedef __attribute__((ext_vector_type(8))) _Float16 hfrag;
typedef __attribute__((ext_vector_type(4))) short short4v;
typedef __attribute__((ext_vector_type(4))) float f4;
typedef __attribute__((ext_vector_type(4))) unsigned int u4;
typedef __attribute__((ext_vector_type(2))) unsigned int u2;
typedef __attribute__((ext_vector_type(2))) float f2;
typedef __attribute__((ext_vector_type(2))) __bf16 bf2;
typedef __attribute__((ext_vector_type(2))) _Float16 h2;
typedef __attribute__((ext_vector_type(16))) float f16v;

__device__ inline float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }  // (results below the smallest normal number: 0)

// Products of 16 x 16 tiles over 32 elements: lane i + 16 g holds elements 8 g .. 8 g + 7 of row i of A and of column i of B, and gets rows
// 4 g .. 4 g + 3 of column i of the product.  For float32 in eight steps of four elements.
template <typename T> struct Mma;
template <> struct Mma<uint16_t> {
  typedef union { u4 u; uint32_t w[4]; bfrag v; short4v h[2]; } frag;
  static constexpr bool WIDE = true;  // exponents of float32: sums of unscaled probabilities times values could pass its range
  __device__ static inline f4 mul(const frag& a, const frag& b, f4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.v, b.v, c, 0, 0, 0); }
  static __device__ inline f16v mul32(const frag& a, const frag& b, f16v c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.v, b.v, c, 0, 0, 0); }
  // two floats as packed 16-bit heads, and what this rounding leaves
  __device__ static inline uint32_t head(float x, float y) {
    union { bf2 v; uint32_t w; } h;
    h.v = __builtin_convertvector(f2{x, y}, bf2);
    return h.w;
  }
  __device__ static inline void split(float x, float y, uint32_t& h, uint32_t& r) {
    h = head(x, y);
    r = head(x - __uint_as_float(h << 16), y - __uint_as_float(h & 0xffff0000u));
  }
};
template <> struct Mma<f16_t> {
  typedef union { u4 u; uint32_t w[4]; hfrag v; short4v h[2]; } frag;
  static constexpr bool WIDE = false;
  __device__ static inline f4 mul(const frag& a, const frag& b, f4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a.v, b.v, c, 0, 0, 0); }
  static __device__ inline f16v mul32(const frag& a, const frag& b, f16v c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a.v, b.v, c, 0, 0, 0); }
  __device__ static inline uint32_t head(float x, float y) {
    union { h2 v; uint32_t w; } h;
    h.v = __builtin_convertvector(f2{x, y}, h2);
    return h.w;
  }
  __device__ static inline void split(float x, float y, uint32_t& h, uint32_t& r) {
    union { h2 v; uint32_t w; } q;
    q.w = h = head(x, y);
    r = head(x - (float)q.v[0], y - (float)q.v[1]);
  }
};
template <> struct Mma<float> {
  typedef union { u4 u[2]; float f[8]; } frag;
  static constexpr bool WIDE = true;
  __device__ static inline f4 mul(const frag& a, const frag& b, f4 c) {
#pragma unroll
    for (int j = 0; j < 8; j++) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a.f[j], b.f[j], c, 0, 0, 0);
    return c;
  }
};
// elements 8 at .. 8 at + 7 of a row of 16-byte vectors
template <typename T>
__device__ inline typename Mma<T>::frag frag_of(const u4* row, int at) {
  typename Mma<T>::frag f;
  if constexpr (sizeof(T) == 4) {
    f.u[0] = row[2 * at];
    f.u[1] = row[2 * at + 1];
  } else {
    f.u = row[at];
  }
  return f;
}

// The larger of a value and that of the lanes 16, 32 and 48 further on: the lanes that share a column of a product.
__device__ inline float col_max(float x) {
  const u2 a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const u2 b = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ inline float col_sum(float x) {
  const u2 a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  const u2 b = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// What is subtracted from scores whose largest is `top`: top + offset (AttnArgs).  Scores beyond 2^24 round this sum; where an offset below 0 would grow by it,
// probabilities could pass the range of half, and it is left out.
template <typename T>
__device__ inline float reference(float top, float offset) {
  const float r = top + offset;
  if constexpr (Mma<T>::WIDE) return r;
  else return top - r > -offset ? top : r;
}

// The value of the lane that a data-parallel permutation pairs this one with, within 16 lanes.
template <int CTRL>
__device__ inline float lane_of(float x) {
  return __uint_as_float(__builtin_amdgcn_mov_dpp(__float_as_uint(x), CTRL, 0xF, 0xF, false));
}

// LDS that only one wavefront uses: its accesses are executed in order, and the compiler keeps that order here.
__device__ inline void wave_lds_order() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// Division of 0 .. 2^31 - 1 by a number that the host knows: with l = ceil(log2 d) and mul = floor(2^32 (2^l - d) / d) + 1 the quotient is
// (mulhi(n, mul) + n) >> l (Granlund and Montgomery 1994).  What a workgroup does before its first tile is a chain of such divisions and of loads: with
// the compiler's, 40 instructions each, it took 7000 cycles in the kernel of many rows.
struct Div {
  uint32_t d, mul, shift;
  Div() = default;
  explicit Div(uint32_t by) : d(by < 1 ? 1 : by), mul(0), shift(0) {
    while ((1ull << shift) < d) shift++;
    mul = (uint32_t)(((1ull << 32) * ((1ull << shift) - d)) / d + 1);
  }
  __device__ inline int quot(int n) const { return (int)((__umulhi((uint32_t)n, mul) + (uint32_t)n) >> shift); }
  __device__ inline int rem(int n) const { return n - quot(n) * (int)d; }
};

// What the kernels are told.
struct AttnArgs {
  const void *Q, *Kp, *Vp, *Kc, *Vc;
  const int32_t *len, *q_len;
  void* O;
  float* weight;
  f2* ml;       // [part][row]: running maximum (base 2, with the offset below) and sum
  float* part;  // [part][row][d_h]
  float* lse;   // [row]: base-2 logarithm of the sum of all probabilities' numerators; +inf: the row gives nothing to anyone
  float* score; // [row][score_ld]: base-2 scores of the cache's keys, where rows are few
  int score_ld;
  int H, Hk, G, T, R, cap, max_len, each, P;
  Div by_T, by_R, by_H, by_Hk, by_each;
  int rows;     // all rows: B H T
  int parts;    // parts of the keys of a row
  float scale2; // scale log2(e)
  float offset; // probabilities are formed as 2^(s - m - offset): for exponents of float32 so that sums of them times values stay within float32; half:
                // as large as the type holds, which sets the small ones apart from 0 (65536 keys of 2^-26 of the largest are a thousandth)
};

// A share of a call: the rows of a group against the keys of a prefix, of the group's cache, or both.  A group is what has one
// key/value head in common: a sequence's R rows, or, `packed`, the rows of all sequences of an image, which then read its prefix once.
struct Job {
  int groups, rows, tiles, splits, part0;  // part0: the first of the `splits` parts that this share writes
  bool packed, prefix, cache, many;        // many: by many_kernel
  bool wide;                               // eight wavefronts
  int share;                               // tiles of a workgroup at most
  Div by_splits, by_tiles;
};

// Row r of a group: its place among all rows.
__device__ inline int row_of(const AttnArgs& a, const Job& j, int group, int r) {
  if (!j.packed) return group * a.R + r;
  const int image = a.by_Hk.quot(group), sequence = a.by_R.quot(r);
  return ((image * a.each + sequence) * a.Hk + group - image * a.Hk) * a.R + r - sequence * a.R;
}

// Tokens of a sequence in this call, and slots in use.
__device__ inline int tokens_of(const AttnArgs& a, int b) { return a.q_len ? clamp_len(a.q_len[b], a.T) : a.T; }
__device__ inline int slots_of(const AttnArgs& a, int b) { return clamp_len(a.len[b], a.max_len); }

// What token t of m sees of the n slots.  Rows behind the last token see what that one sees; nothing of them is kept.
__device__ inline int seen(int t, int n, int m) { return clamp_len(n - m + min(t, m - 1) + 1, n); }

// The least and the most that rows first .. last of a sequence see.
__device__ inline void seen_by(const AttnArgs& a, int first, int last, int n, int m, int& least, int& most) {
  const int g0 = a.by_T.quot(first), g1 = a.by_T.quot(last);
  least = seen(g0 == g1 ? first - g0 * a.T : 0, n, m);
  most = seen(g0 == g1 ? last - g0 * a.T : a.T - 1, n, m);
}

// Share `split` of `all` tiles.
__device__ inline void share_of(const Job& j, int all, int split, int& t0, int& t1) {
  const int q = j.by_splits.quot(all), more = all - q * j.splits;
  t0 = q * split + min(split, more);
  t1 = t0 + q + (split < more ? 1 : 0);
}

// Where token t of head h lies in the output.
__device__ inline size_t out_row(const AttnArgs& a, int b, int h, int t, int dh) { return (((size_t)b * a.T + t) * a.H + h) * dh; }

template <typename T>
__device__ inline bool not_finite(T v) {
  if constexpr (sizeof(T) == 4) return (__float_as_uint(v) & 0x7f800000u) == 0x7f800000u;
  else if constexpr (Mma<T>::WIDE) return (v & 0x7f80u) == 0x7f80u;
  else return (__builtin_bit_cast(uint16_t, v) & 0x7c00u) == 0x7c00u;
}
// A vector's values, those that are not finite as zero.
template <typename T>
__device__ inline u4 finite_only(u4 w) {
#pragma unroll
  for (int i = 0; i < 4; i++) {
    const uint32_t x = w[i];
    if constexpr (sizeof(T) == 4) {
      if ((x & 0x7f800000u) == 0x7f800000u) w[i] = 0;
    } else {
      constexpr uint32_t E = Mma<T>::WIDE ? 0x7f80u : 0x7c00u;
      w[i] = ((x & E) == E ? 0 : x & 0xffffu) | ((x & E << 16) == E << 16 ? 0 : x & 0xffff0000u);
    }
  }
  return w;
}
template <typename T>
__device__ inline bool any_not_finite(const u4& w) {
  bool bad = false;
#pragma unroll
  for (int i = 0; i < 4; i++) {
    const uint32_t x = w[i];
    if constexpr (sizeof(T) == 4) {
      bad |= (x & 0x7f800000u) == 0x7f800000u;
    } else {
      constexpr uint32_t E = Mma<T>::WIDE ? 0x7f80u : 0x7c00u;
      bad |= (x & E) == E || (x & E << 16) == E << 16;
    }
  }
  return bad;
}

// Values that are not finite.  In tiles of which some row does not see all, they are kept out of the product (0 times them is NaN), in others the product
// takes them as they come, and a probability that has become 0, or whose head and remainder differ in sign, makes NaN of an infinity.  So behind the
// last tile a wavefront that has met one sets what it has found right: an element of a row's output is the sum of such values among those that the row
// sees, if there are any.

// A partial output's element times a factor of the softmax, 0 .. 1: what is not finite stays so where the factor has become 0.
__device__ inline float scaled(float x, float f) {
  const float y = x * f;
  return y == y ? y : x;
}

// Whether a value of these rows is not finite, by a wavefront.
template <typename T, int DH>
__device__ inline bool any_odd(const T* V, int rows, int lane) {
  const u4* v = reinterpret_cast<const u4*>(V);
  bool odd = false;
#pragma unroll 4
  for (int at = lane; at < rows * (DH * (int)sizeof(T) / 16); at += 64) odd |= any_not_finite<T>(v[at]);
  return __ballot(odd) != 0;
}

// Adds the values that are not finite among elements `first` + STEP j .. + 3 of rows 0 .. min(rows, lim) - 1 to sum[j].
template <typename T, int DH, int STEP>
__device__ inline void add_odd(const T* V, int rows, int lim, int first, f4 (&sum)[DH / STEP]) {
#pragma unroll 1
  for (int k = 0; k < rows; k++)
#pragma unroll
    for (int j = 0; j < DH / STEP; j++)
#pragma unroll
      for (int e = 0; e < 4; e++) {
        const T v = V[(size_t)k * DH + first + STEP * j + e];
        if (k < lim && not_finite(v)) sum[j][e] += Vec16<T>::one(v);
      }
}

// Rows of keys and values from `first` on to registers, N threads side by side: they are one run of 16-byte vectors.  Behind the `there` rows
// that exist the last vector of these is read; of values zero stands in its place (zero_behind) before they are used.
template <int N, int VEC, int NV>
__device__ __forceinline__ void fetch_tile(const void* K, const void* V, size_t first, int there, int id, u4 (&kr)[NV], u4 (&vr)[NV]) {
  const char* Kb = static_cast<const char*>(K) + first * VEC * 16;
  const char* Vb = static_cast<const char*>(V) + first * VEC * 16;
  const int end = min(there, N * NV / VEC) * VEC - 1;
#pragma unroll
  for (int j = 0; j < NV; j++) {
    const unsigned off = (unsigned)min(id + N * j, end) * 16;
    kr[j] = *reinterpret_cast<const u4*>(Kb + off);
    vr[j] = *reinterpret_cast<const u4*>(Vb + off);
  }
}
template <int N, int VEC, int NV>
__device__ __forceinline__ void zero_behind(int there, int id, u4 (&vr)[NV]) {
#pragma unroll
  for (int j = 0; j < NV; j++)
    if (id + N * j >= there * VEC) vr[j] = u4{0, 0, 0, 0};
}

// A sum of probabilities of the R rows: no more than R of them, which the rounding of a logarithm beyond 2^24 could make of it (NaN stays).
__device__ inline float share(const AttnArgs& a, float sum) { return sum > (float)a.R ? (float)a.R : sum; }

// Slots k .. k + 3 of a sequence and head gather the probabilities of its few rows, from the scores that were kept.  A row's scores are there up to
// the tile that the last row sees; what lies behind what the row sees is read and left out (loads under conditions would wait for one another:
// 2 sequences of 10 rows 4.8 us of 11.5).
__device__ inline void add_weights(const AttnArgs& a, int group, int k, int n, int m, const float* lse) {
  float* w = a.weight + (size_t)group * a.cap + k;
  const float* score = a.score + (size_t)group * a.R * a.score_ld + k;
  f4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int r = 0; r < a.R; r++) {
    const int end = lse[r] == INFINITY ? 0 : seen(a.by_T.rem(r), n, m);
    const f4 s = *reinterpret_cast<const f4*>(score + (size_t)r * a.score_ld);
#pragma unroll
    for (int e = 0; e < 4; e++) {
      const float p = exp2_fast(s[e] - lse[r]);
      acc[e] += k + e < end ? p : 0.f;
    }
  }
#pragma unroll
  for (int e = 0; e < 4; e++)
    if (k + e < n) w[e] += share(a, acc[e]);
}

// ---- few rows: one workgroup has 16 rows, its one to eight wavefronts share the keys, 32 at a time, without waiting for one another ----
//
// The keys' and values' bytes bound it: each is read once, as whole lines, to registers while the tile before it is in work, and passes through LDS that
// is the wavefront's own, so that no barrier stands between loads.  bf16, heads of 128: 64 sequences of 32 heads sharing 8 prefixes of 640 keys, up to
// 200 slots: 39 us; 4 sequences of 8 heads for 32, up to 32768 slots: 84 us, 4.9 TB/s (a copy reaches 5.1).  One sequence of 32 heads and 640
// slots: 10.2 us, of which the chain launch, length, two or three tiles, joining of eight wavefronts is nearly all.

constexpr int FK = 32;  // keys of a wavefront's tile
template <typename T, int DH>
struct FewShape {
  static constexpr int ES = sizeof(T), VEC = DH * ES / 16;             // 16-byte vectors of a row
  static constexpr int KLD = DH * ES + 16, VLD = DH * ES + (ES == 2 ? 32 : 16);  // rows in LDS: lanes of a product's operand meet other banks
  static constexpr int NV = FK * VEC / 64;                             // vectors of a lane
  static constexpr int WAVE = FK * (KLD + VLD);
  static constexpr int MOST = 8 * WAVE <= 160 * 1024 - 2048 ? 8 : 4;   // wavefronts that fit
  static_assert(16 * (DH + 4) * 4 <= WAVE, "the partial output takes the place of the tiles");
};

// KEEP: scores of the cache's keys are written.  Unconditionally, so that the count of accesses in flight is known and a tile's loads need not wait
// for them: lanes behind the last row have its scores, and scores of a prefix go to FK places behind a row's own.
template <typename T, int DH, bool KEEP, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void few_kernel(AttnArgs a, Job first, Job second) {
  typedef FewShape<T, DH> S;
  typedef Mma<T> M;
  typedef typename M::frag frag;
  constexpr int ES = S::ES, VEC = S::VEC, NV = S::NV, DT = DH / 16;
  extern __shared__ __attribute__((aligned(16))) unsigned char cache_smem[];
  __shared__ float wave_m[WAVES][16], wave_l[WAVES][16], row_sum[16], row_lse[16];  // row_sum: infinite for a row whose output is zero
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), i = lane & 15, g = lane >> 4;
  const unsigned in_first = (unsigned)first.groups * first.tiles * first.splits;
  const bool other = blockIdx.x >= in_first;
  const Job job = other ? second : first;
  const unsigned item = blockIdx.x - (other ? in_first : 0);
  const int at_tile = job.by_splits.quot(item), split = item - at_tile * job.splits;
  const int group = job.by_tiles.quot(at_tile), tile = at_tile - group * job.tiles;
  const int b = a.by_Hk.quot(group), hk = group - b * a.Hk;  // (packed: b is the image)
  const int r = tile * 16 + i, row = row_of(a, job, group, min(r, job.rows - 1));  // this lane's row of queries
  const bool mine = r < job.rows;
  const size_t head = (size_t)group * a.cap, phead = job.prefix ? ((size_t)(job.packed ? b : a.by_each.quot(b)) * a.Hk + hk) * a.P : 0;
  unsigned char* Ks = cache_smem + wave * S::WAVE;
  unsigned char* Vs = Ks + FK * S::KLD;
  u4 kr[NV], vr[NV];
  // Where the keys are one part each wavefront's first tile is known before the sequence's length is (of which it may hold less, or nothing): it
  // comes at once, and the queries.
  const bool ahead = job.splits == 1;
  if (ahead) {
    const int tiles = job.prefix ? (a.P + FK - 1) / FK : 0;
    const bool pre = wave < tiles;
    const int k0 = (pre ? wave : wave - tiles) * FK, there = pre ? a.P : job.cache ? a.cap : 0;
    if (k0 < there) fetch_tile<64, VEC>(pre ? a.Kp : a.Kc, pre ? a.Vp : a.Vc, (pre ? phead : head) + k0, there - k0, lane, kr, vr);
  }
  frag q[DH / 32];
  {
    const u4* Qr = reinterpret_cast<const u4*>(static_cast<const T*>(a.Q) + (size_t)row * DH);
#pragma unroll
    for (int s = 0; s < DH / 32; s++) q[s] = frag_of<T>(Qr, 4 * s + g);
  }
  int n = 0, m = 1, end = 0, most = 0, least = 0;
  bool live = mine;
  if (job.cache) {
    n = slots_of(a, b);
    m = tokens_of(a, b);
    const int tok = a.by_T.rem(min(r, a.R - 1));
    live = mine && tok < m;
    end = seen(tok, n, m);
    seen_by(a, tile * 16, min(tile * 16 + 15, a.R - 1), n, m, least, most);
  }
  // tiles of the prefix, then of the cache; this workgroup's share of them, dealt to its wavefronts in turn
  const int np = job.prefix && m > 0 ? (a.P + FK - 1) / FK : 0, all = m > 0 ? np + (most + FK - 1) / FK : 0;
  int t0, t1;
  share_of(job, all, split, t0, t1);
  auto fetch = [&](int t) {
    const bool pre = t < np;
    const int k0 = (pre ? t : t - np) * FK;
    fetch_tile<64, VEC>(pre ? a.Kp : a.Kc, pre ? a.Vp : a.Vc, (pre ? phead : head) + k0, (pre ? a.P : most) - k0, lane, kr, vr);
  };

  f4 o[DT];
#pragma unroll
  for (int d = 0; d < DT; d++) o[d] = f4{0.f, 0.f, 0.f, 0.f};
  float mx = -INFINITY, sum = 0.f;
  bool odd = false;  // a value that is not finite was kept out of a product

  int t = t0 + wave;
  if (!ahead && t < t1) fetch(t);
  for (; t < t1; t += WAVES) {
    const bool pre = t < np;
    const int k0 = (pre ? t : t - np) * FK, last = pre ? a.P : most;
    const bool masked = k0 + FK > (pre ? a.P : least);  // some row does not see some key
    if (masked) {
      zero_behind<64, VEC>(last - k0, lane, vr);
      bool found = false;
#pragma unroll
      for (int j = 0; j < NV; j++) found |= any_not_finite<T>(vr[j]);
      if (__ballot(found)) {
        odd = true;
#pragma unroll
        for (int j = 0; j < NV; j++) vr[j] = finite_only<T>(vr[j]);
      }
    }
#pragma unroll
    for (int j = 0; j < NV; j++) {
      const int at = lane + 64 * j, key = at / VEC, c = at % VEC;
      *reinterpret_cast<u4*>(Ks + key * S::KLD + c * 16) = kr[j];
      *reinterpret_cast<u4*>(Vs + key * S::VLD + c * 16) = vr[j];
    }
    if (t + WAVES < t1) fetch(t + WAVES);
    wave_lds_order();

    f4 s[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
    for (int c = 0; c < DH / 32; c++)
#pragma unroll
      for (int u = 0; u < 2; u++)
        s[u] = M::mul(frag_of<T>(reinterpret_cast<const u4*>(Ks + (16 * u + i) * S::KLD), 4 * c + g), q[c], s[u]);
    float top = -INFINITY;
#pragma unroll
    for (int u = 0; u < 2; u++)
#pragma unroll
      for (int e = 0; e < 4; e++) {
        const int key = k0 + 16 * u + 4 * g + e;
        s[u][e] = !masked || key < (pre ? last : end) ? s[u][e] * a.scale2 : -INFINITY;
        top = fmaxf(top, s[u][e]);
      }
    if (KEEP) {
      float* to = a.score + (size_t)row * a.score_ld + (pre ? a.score_ld - FK : k0) + 4 * g;
#pragma unroll
      for (int u = 0; u < 2; u++) *reinterpret_cast<f4*>(to + 16 * u) = s[u];
    }
    top = fmaxf(mx, col_max(top));
    const float ref = top == -INFINITY ? 0.f : reference<T>(top, a.offset);
    if (__ballot(top > mx)) {
      const float f = exp2_fast(reference<T>(mx, a.offset) - ref);
      sum *= f;
#pragma unroll
      for (int d = 0; d < DT; d++) o[d] *= f;
    }
    mx = top;
    float p[8];
#pragma unroll
    for (int u = 0; u < 2; u++)
#pragma unroll
      for (int e = 0; e < 4; e++) {
        p[4 * u + e] = exp2_fast(s[u][e] - ref);
        sum += p[4 * u + e];
      }
    // element j of a lane's operands is key 4 g + j, from j = 4 on key 16 + 4 g + j - 4
    frag ph, pr;
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int j = 0; j < 8; j++) ph.f[j] = p[j];
    } else {
      // probabilities enter as a 16-bit head and the remainder: O is accurate to its own rounding
#pragma unroll
      for (int j = 0; j < 4; j++) M::split(p[2 * j], p[2 * j + 1], ph.w[j], pr.w[j]);
    }
#pragma unroll
    for (int d = 0; d < DT; d++) {
      frag v;
      if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int j = 0; j < 8; j++)
          v.f[j] = *reinterpret_cast<const float*>(Vs + (4 * g + (j & 3) + 16 * (j >> 2)) * S::VLD + (16 * d + i) * 4);
      } else {
        // the transposing read: 16 lanes name four rows of 16 elements and get a column each
#pragma unroll
        for (int u = 0; u < 2; u++) {
          unsigned char* at = Vs + (16 * u + 4 * g + i / 4) * S::VLD + (16 * d + 4 * (i % 4)) * 2;
          v.h[u] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) short4v*)at);
        }
      }
      o[d] = M::mul(v, ph, o[d]);
      if constexpr (sizeof(T) == 2) o[d] = M::mul(v, pr, o[d]);
    }
    wave_lds_order();
  }
  if (!odd) {
    f4 z = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int d = 0; d < DT; d++)
#pragma unroll
      for (int e = 0; e < 4; e++) z[e] = fmaf(o[d][e], 0.f, z[e]);
    odd = __ballot(live && z[0] + z[1] + z[2] + z[3] != 0.f) != 0;
  }
  if (__builtin_expect(odd, 0)) {
    f4 add[DT];
#pragma unroll
    for (int d = 0; d < DT; d++) add[d] = f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
    for (int u = t0 + wave; u < t1; u += WAVES) {
      const bool pre = u < np;
      const int k0 = (pre ? u : u - np) * FK, keys = min(FK, (pre ? a.P : most) - k0);
      const T* V = static_cast<const T*>(pre ? a.Vp : a.Vc) + ((pre ? phead : head) + k0) * DH;
      if (any_odd<T, DH>(V, keys, lane)) add_odd<T, DH, 16>(V, keys, (pre ? a.P : end) - k0, 4 * g, add);
    }
#pragma unroll
    for (int d = 0; d < DT; d++)
#pragma unroll
      for (int e = 0; e < 4; e++)
        if (add[d][e] != 0.f) o[d][e] = add[d][e];
  }
  sum = col_sum(sum);

  // the wavefronts' parts
  mx = reference<T>(mx, a.offset);  // (-inf of nothing)
  if (g == 0) {
    wave_m[wave][i] = mx;
    wave_l[wave][i] = sum;
  }
  __syncthreads();
  float top = -INFINITY, total = 0.f;
#pragma unroll
  for (int w = 0; w < WAVES; w++) top = fmaxf(top, wave_m[w][i]);
  const float ref = top == -INFINITY ? 0.f : top;
#pragma unroll
  for (int w = 0; w < WAVES; w++) total += wave_l[w][i] * exp2_fast(wave_m[w][i] - ref);
  const float f = exp2_fast(mx - ref);
  float* part = reinterpret_cast<float*>(cache_smem + wave * S::WAVE);
#pragma unroll
  for (int d = 0; d < DT; d++) {
    f4 v = o[d] * f;
    if (odd) {
#pragma unroll
      for (int e = 0; e < 4; e++) v[e] = scaled(o[d][e], f);
    }
    *reinterpret_cast<f4*>(part + i * (DH + 4) + 16 * d + 4 * g) = v;
  }
  if (threadIdx.x < 16 && mine) {  // (wavefront 0, lane i: row i)
    const float lse = live ? ref + log2f(total) : INFINITY;
    if (a.parts > 1) a.ml[(size_t)(job.part0 + split) * a.rows + row] = f2{top, total};
    else if (a.lse) a.lse[row] = lse;
    row_lse[i] = lse;
    row_sum[i] = live && a.P + end > 0 ? total : INFINITY;
  }
  __syncthreads();
  if (a.parts > 1 && t0 >= t1) return;
  for (int at = threadIdx.x; at < 16 * DH / 4; at += 64 * WAVES) {
    const int rr = at / (DH / 4), c = at % (DH / 4);
    if (tile * 16 + rr >= job.rows) continue;
    f4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < WAVES; w++) v += *reinterpret_cast<const f4*>(cache_smem + w * S::WAVE + (rr * (DH + 4) + 4 * c) * 4);
    if (a.parts > 1) {
      const int to = row_of(a, job, group, tile * 16 + rr);
      *reinterpret_cast<f4*>(a.part + ((size_t)(job.part0 + split) * a.rows + to) * DH + 4 * c) = v;
    } else {
      v = row_sum[rr] < INFINITY || row_sum[rr] != row_sum[rr] ? v / row_sum[rr] : f4{0.f, 0.f, 0.f, 0.f};
      const int head_of = a.by_T.quot(tile * 16 + rr);
      T* out = static_cast<T*>(a.O) + out_row(a, b, hk * a.G + head_of, tile * 16 + rr - head_of * a.T, DH) + 4 * c;
#pragma unroll
      for (int e = 0; e < 4; e++) out[e] = Vec16<T>::round(v[e]);
    }
  }
  // the only part: this workgroup has written all scores of its rows (and the barriers above stand between)
  if (KEEP && a.parts == 1)
    for (int k = 4 * threadIdx.x; k < n; k += 4 * 64 * WAVES) add_weights(a, group, k, n, m, row_lse);
}

// ---- many rows, 16-bit storage: one workgroup has 128 rows, a wavefront 32 of them, all go over the same tiles of 64 keys; or (KW = 2) 64 rows,
// and two wavefronts share the keys of a tile ----
//
// Products of 32 x 32 tiles: a lane has row lane % 32, and of each 32 keys those with (key / 4) % 2 = lane / 32, which are the ones that its
// operand of the second product wants.  A tile is in one of two stages of LDS while the next one is written into the other and the one
// after that comes to registers: one barrier a tile.
//
// 64 x 40 heads of 128, 576 rows, 640 keys, bf16: 469 us one after another, 570 TFLOP/s of what is seen (485 to 515 in single passes, at lower clocks; tiles of
// 64 keys by 128 rows compute a fifth more at the diagonal; 40 heads, 2048 rows of 16000 keys: 766 us, 820).  Two wavefronts on a SIMD have 2048 cycles of products and 2300 of vector work a pair of tiles, the LDS of a
// compute unit 2560, which overlap by half.  64 rows a wavefront (half of the LDS reads, one wavefront on a SIMD) took 850 us, the keys two tiles ahead
// in L2 617, a priority for the products changed nothing.  With 64 rows a workgroup, heads of 64 (1024 groups of 1 to 61 rows, 640 + 90 keys): 27 us, 32 with
// the weights, which a kernel of their own took 8 for.  Rows behind q_len are computed like tokens: half of all rows here, and a quarter of the wavefronts has no
// other.
constexpr int MK = 64, MROWS = 128;
template <int DH>
struct ManyShape {
  static constexpr int VEC = DH / 8, NV = MK * VEC / 256;         // 16-byte vectors of a row, of a thread
  static constexpr int KLD = DH * 2 + 16, VLD = DH * 2 + 32;      // rows in LDS: 16 lanes of a read meet other banks; heads of 64: four workgroups fit
  static constexpr int STAGE = MK * (KLD + VLD), LDS = 2 * STAGE;
  static_assert(4 * 32 * KLD <= LDS && 2 * 64 * (DH / 2 + 2) * 4 + 2 * 32 * KLD <= LDS, "outputs take the place of the tiles");
};
// The running maximum is raised when a row's passes it by more than 2^8: up to there the probabilities are larger than 1, which neither
// the sums in float32 nor the heads mind, and the partial output need not be scaled.
constexpr float LAZY = 8.f;
// The largest score is rounded, the product that the probabilities are formed of is not.  From here on they differ by what an exponent may not be off
// by: a workgroup that has met such a score goes over its keys again with scores that are rounded before.
constexpr float LARGE = 0x1p22f;

template <bool B> struct Flag { static constexpr bool value = B; };

template <typename T, int DH, int KW>
struct ManyWave {
  static constexpr int NU = 2 / KW;  // runs of 32 keys of a tile that are the wavefront's
  typedef Mma<T> M;
  typedef typename M::frag frag;
  typedef ManyShape<DH> S;
  frag q[DH / 16];
  f16v o[DH / 32];
  float mx, sum;

  // One tile.  `masked`: some row of the wavefront does not see some key; keys below `lim` are seen by this lane's row.  (One body for both: with
  // two the partial output would move between registers.)  `large` is set where a score has reached LARGE, ROUNDED: scores are rounded.
  template <bool ROUNDED>
  __device__ __forceinline__ void step(const unsigned char* Ks, const unsigned char* Vs, int k0, int lim, bool masked, float scale2, float offset,
                                       int lane, int* large) {
    const int half = lane >> 5, i = lane & 31;
    f16v s[NU];
#pragma unroll
    for (int u = 0; u < NU; u++)
#pragma unroll
      for (int e = 0; e < 16; e++) s[u][e] = 0.f;
    const unsigned char* kr = Ks + i * S::KLD + 16 * half;
#pragma unroll
    for (int c = 0; c < DH / 16; c++)
#pragma unroll
      for (int u = 0; u < NU; u++) {
        frag k;
        k.u = *reinterpret_cast<const u4*>(kr + u * 32 * S::KLD + 32 * c);
        s[u] = M::mul32(k, q[c], s[u]);
      }
    if constexpr (ROUNDED) {
#pragma unroll
      for (int u = 0; u < NU; u++)
#pragma unroll
        for (int e = 0; e < 16; e++) s[u][e] *= scale2;
      scale2 = 1.f;
    }
    if (masked) {
#pragma unroll
      for (int u = 0; u < NU; u++)
#pragma unroll
        for (int e = 0; e < 16; e++)
          if (k0 + 32 * u + 8 * (e >> 2) + 4 * half + (e & 3) >= lim) s[u][e] = -INFINITY;
    }
    float top = -INFINITY;
#pragma unroll
    for (int u = 0; u < NU; u++)
#pragma unroll
      for (int e = 0; e < 16; e++) top = fmaxf(top, s[u][e]);
    const u2 w = __builtin_amdgcn_permlane32_swap(__float_as_uint(top), __float_as_uint(top), false, false);
    top = fmaxf(__uint_as_float(w[0]), __uint_as_float(w[1])) * scale2;
    if (__ballot(top > mx + LAZY)) {
      const float now = fmaxf(mx, top), f = now == -INFINITY ? 1.f : exp2_fast(reference<T>(mx, offset) - reference<T>(now, offset));
      if (!ROUNDED && fabsf(now) >= LARGE && fabsf(now) < INFINITY) *large = 1;
      mx = now;
      sum *= f;
#pragma unroll
      for (int d = 0; d < DH / 32; d++) o[d] *= f;
    }
    const float ref = mx == -INFINITY ? 0.f : reference<T>(mx, offset);
#pragma unroll
    for (int u = 0; u < NU; u++) {
      float p[16];
#pragma unroll
      for (int e = 0; e < 16; e++) {
        p[e] = exp2_fast(fmaf(s[u][e], scale2, -ref));
        sum += p[e];
      }
#pragma unroll
      for (int v = 0; v < 2; v++) {
        // probabilities enter as they round to 16 bits: an error of the size of the output's own rounding, half of the products of
        // the exact form
        frag ph;
#pragma unroll
        for (int j = 0; j < 4; j++) ph.w[j] = M::head(p[8 * v + 2 * j], p[8 * v + 2 * j + 1]);
#pragma unroll
        for (int d = 0; d < DH / 32; d++) {
          frag x;
#pragma unroll
          for (int j = 0; j < 2; j++) {
            const unsigned char* at = Vs + (32 * u + 16 * v + 8 * j + 4 * half + (i & 15) / 4) * S::VLD + (32 * d + (i & 16) + 4 * (i & 3)) * 2;
            x.h[j] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) short4v*)const_cast<unsigned char*>(at));
          }
          o[d] = M::mul32(x, ph, o[d]);
        }
      }
    }
  }
};

// GATHER: the workgroup has all rows of its group and all of their keys, and adds what the slots gather itself, from scores formed again, with the keys
// in the lanes and the rows in registers.
template <typename T, int DH, int KW, bool GATHER>
__global__ __launch_bounds__(256, KW == 2 && DH == 64 ? 4 : 2) void many_kernel(AttnArgs a, Job job) {
  typedef ManyShape<DH> S;
  typedef ManyWave<T, DH, KW> Wave;
  constexpr int ROWS = MROWS / KW, RW = 4 / KW;  // rows of the workgroup, wavefronts that share them
  const float offset = a.offset + LAZY;          // (a probability may pass that of the running maximum so far)
  extern __shared__ __attribute__((aligned(16))) unsigned char cache_smem[];
  __shared__ int large_scores, odd_values;  // a score has reached LARGE; values that are not finite were kept out of a product
  __shared__ size_t places[4][32];  // of rows in the output
  // where it gathers: behind the outputs, in the place of the tiles
  constexpr int KEYS = 32 * Wave::NU, GBYTES = ROWS * 8 + 2 * 4 * KEYS * 4;
  static_assert((KW - 1) * 2 * 64 * (DH / 2 + 2) * 4 + RW * 32 * S::KLD <= S::LDS - GBYTES && GBYTES % 16 == 0);
  float* row_lse = reinterpret_cast<float*>(cache_smem + S::LDS - GBYTES);
  int* row_end = reinterpret_cast<int*>(row_lse + ROWS);
  float* sums = reinterpret_cast<float*>(row_end + ROWS);  // [2][wavefront][key]
  int group, item;
  if (!group_on_xcd(blockIdx.x, job.tiles * job.splits, job.groups, &group, &item)) return;
  const int back = job.by_splits.quot(item), split = item - back * job.splits, tile = job.tiles - 1 - back;  // (the rows that see the most first)
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), half = lane >> 5, i = lane & 31;
  const int b = a.by_Hk.quot(group), hk = group - b * a.Hk;  // (packed: b is the image)
  // The tiles are laid so that the last one is full: the empty rows are in the first one, which sees the fewest keys.
  const int tile0 = tile * ROWS - (job.tiles * ROWS - job.rows), r0 = tile0 + wave % RW * 32, r = r0 + i, row = row_of(a, job, group, max(r, 0));
  const int ku = KW == 2 ? wave / RW * 32 : 0;  // the wavefront's first key of a tile
  const bool mine = r >= 0, idle = r0 + 31 < 0;
  const size_t head = (size_t)group * a.cap, phead = job.prefix ? ((size_t)(job.packed ? b : a.by_each.quot(b)) * a.Hk + hk) * a.P : 0;
  u4 kr[S::NV], vr[S::NV];
  // Where the keys are one part its first tile is known before the sequence's length is (of which it may hold less): it comes at once, and the
  // queries.
  const bool ahead = job.splits == 1;
  if (ahead) fetch_tile<256, S::VEC>(job.prefix ? a.Kp : a.Kc, job.prefix ? a.Vp : a.Vc, job.prefix ? phead : head, job.prefix ? a.P : a.cap, tid, kr, vr);
  Wave w;
  {
    const u4* Qr = reinterpret_cast<const u4*>(static_cast<const T*>(a.Q) + (size_t)row * DH);
#pragma unroll
    for (int c = 0; c < DH / 16; c++) w.q[c].u = Qr[2 * c + half];
  }
  int m = 1, end = 0, most = 0, least = 0, wave_most = 0, wave_least = 0, head_of = 0, tok = 0;
  bool live = mine;
  if (job.cache) {
    const int n = slots_of(a, b);
    m = tokens_of(a, b);
    head_of = a.by_T.quot(max(r, 0));
    tok = max(r, 0) - head_of * a.T;
    live = mine && tok < m;
    end = seen(tok, n, m);
    seen_by(a, max(tile0, 0), tile0 + ROWS - 1, n, m, least, most);
    seen_by(a, max(r0, 0), max(r0 + 31, 0), n, m, wave_least, wave_most);
  }
  if (tid == 0) large_scores = odd_values = 0;
  __syncthreads();
  const int np = job.prefix && m > 0 ? (a.P + MK - 1) / MK : 0, all = m > 0 ? np + (most + MK - 1) / MK : 0;
  int t0, t1;
  share_of(job, all, split, t0, t1);

  auto fetch = [&](int t) {
    const bool pre = t < np;
    const int k0 = (pre ? t : t - np) * MK;
    fetch_tile<256, S::VEC>(pre ? a.Kp : a.Kc, pre ? a.Vp : a.Vc, (pre ? phead : head) + k0, (pre ? a.P : most) - k0, tid, kr, vr);
  };
  auto store = [&](int t) {
    unsigned char* Ks = cache_smem + (t & 1) * S::STAGE;
    unsigned char* Vs = Ks + MK * S::KLD;
    const bool pre = t < np;
    const int k0 = (pre ? t : t - np) * MK;
    if (k0 + MK > (pre ? a.P : least)) {  // rows differ in what they see: is every value finite?
      bool odd = false;
      zero_behind<256, S::VEC>((pre ? a.P : most) - k0, tid, vr);
#pragma unroll
      for (int j = 0; j < S::NV; j++) odd |= any_not_finite<T>(vr[j]);
      if (odd) {
        odd_values = 1;
#pragma unroll
        for (int j = 0; j < S::NV; j++) vr[j] = finite_only<T>(vr[j]);
      }
    }
#pragma unroll
    for (int j = 0; j < S::NV; j++) {
      const int at = tid + 256 * j, key = at / S::VEC, c = at % S::VEC;
      *reinterpret_cast<u4*>(Ks + key * S::KLD + c * 16) = kr[j];
      *reinterpret_cast<u4*>(Vs + key * S::VLD + c * 16) = vr[j];
    }
  };

  auto sweep = [&](auto rounded) __attribute__((always_inline)) {
    constexpr bool ROUNDED = decltype(rounded)::value;
#pragma unroll
    for (int d = 0; d < DH / 32; d++)
#pragma unroll
      for (int e = 0; e < 16; e++) w.o[d][e] = 0.f;
    w.mx = -INFINITY;
    w.sum = 0.f;
    if (t0 < t1) {
      if (ROUNDED || !ahead) fetch(t0);
      store(t0);
      if (t0 + 1 < t1) fetch(t0 + 1);
      __syncthreads();
    }
    for (int t = t0; t < t1; t++) {
      const bool pre = t < np;
      const int k0 = (pre ? t : t - np) * MK + ku, lim = pre ? a.P : end;
      const unsigned char* Ks = cache_smem + (t & 1) * S::STAGE;
      if (!idle && k0 < (pre ? a.P : wave_most)) {
        const bool masked = k0 + MK / KW > (pre ? a.P : wave_least);
        w.template step<ROUNDED>(Ks + ku * S::KLD, Ks + MK * S::KLD + ku * S::VLD, k0, lim, masked, a.scale2, offset, lane, &large_scores);
      }
      if (t + 1 < t1) store(t + 1);  // the other stage was last read before the last barrier
      __syncthreads();
      if (t + 2 < t1) fetch(t + 2);
    }
  };
  sweep(Flag<false>());
  if (__builtin_expect(t0 < t1 && __builtin_amdgcn_readfirstlane(large_scores), 0)) sweep(Flag<true>());
  w.mx = reference<T>(w.mx, offset);  // (-inf of nothing)
  const u2 x = __builtin_amdgcn_permlane32_swap(__float_as_uint(w.sum), __float_as_uint(w.sum), false, false);
  float total = __uint_as_float(x[0]) + __uint_as_float(x[1]);
  if constexpr (KW == 2) {  // the second wavefront of the rows hands its share to the first (behind the last barrier nobody reads the tiles)
    float* at = reinterpret_cast<float*>(cache_smem) + wave % RW * (64 * (DH / 2 + 2)) + lane;
    if (wave >= RW) {
      at[0] = w.mx;
      at[64] = total;
#pragma unroll
      for (int d = 0; d < DH / 32; d++)
#pragma unroll
        for (int e = 0; e < 16; e++) at[64 * (2 + 16 * d + e)] = w.o[d][e];
    }
    __syncthreads();
    if (!GATHER && wave >= RW) return;
    const float mx = fmaxf(w.mx, at[0]), ref = mx == -INFINITY ? 0.f : mx;
    const float f0 = exp2_fast(w.mx - ref), f1 = exp2_fast(at[0] - ref);
    total = total * f0 + at[64] * f1;
#pragma unroll
    for (int d = 0; d < DH / 32; d++)
#pragma unroll
      for (int e = 0; e < 16; e++) w.o[d][e] = w.o[d][e] * f0 + at[64 * (2 + 16 * d + e)] * f1;
    w.mx = mx;
    wave_lds_order();
  }
  bool odd = __builtin_amdgcn_readfirstlane(odd_values) != 0;
  if (!odd) {
    f4 z = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int d = 0; d < DH / 32; d++)
#pragma unroll
      for (int e = 0; e < 16; e++) z[e % 4] = fmaf(w.o[d][e], 0.f, z[e % 4]);
    odd = __ballot(live && z[0] + z[1] + z[2] + z[3] != 0.f) != 0;
  }
  if (__builtin_expect(odd && !idle && wave % RW == wave, 0)) {
    f4 add[DH / 8];
#pragma unroll
    for (int j = 0; j < DH / 8; j++) add[j] = f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
    for (int t = t0; t < t1; t++) {
      const bool pre = t < np;
      const int k0 = (pre ? t : t - np) * MK, keys = min(MK, (pre ? a.P : wave_most) - k0);
      const T* V = static_cast<const T*>(pre ? a.Vp : a.Vc) + ((pre ? phead : head) + k0) * DH;
      if (any_odd<T, DH>(V, keys, lane)) add_odd<T, DH, 8>(V, keys, (pre ? a.P : end) - k0, 4 * half, add);
    }
#pragma unroll
    for (int d = 0; d < DH / 32; d++)
#pragma unroll
      for (int e = 0; e < 16; e++)
        if (add[4 * d + e / 4][e % 4] != 0.f) w.o[d][e] = add[4 * d + e / 4][e % 4];
  }
  if (a.parts > 1) {
    if (!mine) return;
    const size_t at = (size_t)(job.part0 + split) * a.rows + row;
    if (half == 0) a.ml[at] = f2{w.mx, total};
    if (t0 >= t1) return;
#pragma unroll
    for (int d = 0; d < DH / 32; d++)
#pragma unroll
      for (int e = 0; e < 4; e++)
        *reinterpret_cast<f4*>(a.part + at * DH + 32 * d + 8 * e + 4 * half) = f4{w.o[d][4 * e], w.o[d][4 * e + 1], w.o[d][4 * e + 2], w.o[d][4 * e + 3]};
    return;
  }
  if (!GATHER && idle) return;
  const float lse = live ? (w.mx == -INFINITY ? 0.f : w.mx) + log2f(total) : INFINITY;
  // keys of the slots as operands, 32 of a wavefront's in each run: lane i has part of slot k0 + i
  typename Mma<T>::frag ks[GATHER ? Wave::NU : 1][DH / 16];
  auto load_slots = [&](int k0) {
#pragma unroll
    for (int u = 0; u < Wave::NU; u++) {
      const u4* Kr = reinterpret_cast<const u4*>(static_cast<const T*>(a.Kc) + (head + min(k0 + ku + 32 * u + i, a.cap - 1)) * DH);
#pragma unroll
      for (int c = 0; c < DH / 16; c++) ks[u][c].u = Kr[2 * c + half];
    }
  };
  if constexpr (GATHER) {
    load_slots(0);
    if (half == 0 && (KW == 1 || wave < RW)) {
      row_lse[wave % RW * 32 + i] = lse;
      row_end[wave % RW * 32 + i] = live ? end : 0;
    }
  } else if (a.lse && half == 0 && mine) {
    a.lse[row] = lse;
  }
  const bool sees = live && a.P + end > 0;
  if (!GATHER || (!idle && wave % RW == wave)) {
    const float inv = 1.f / total;
    unsigned char* Os = cache_smem + 2 * 64 * (DH / 2 + 2) * 4 * (KW - 1) + wave * 32 * S::KLD;
    if (half == 0) places[wave][i] = out_row(a, b, hk * a.G + head_of, tok, DH);
#pragma unroll
    for (int d = 0; d < DH / 32; d++)
#pragma unroll
      for (int e = 0; e < 8; e++) {
        const float y0 = sees ? w.o[d][2 * e] * inv : 0.f, y1 = sees ? w.o[d][2 * e + 1] * inv : 0.f;
        *reinterpret_cast<uint32_t*>(Os + i * S::KLD + (32 * d + 8 * (e >> 1) + 4 * half + 2 * (e & 1)) * 2) = Mma<T>::head(y0, y1);
      }
    wave_lds_order();
#pragma unroll
    for (int j = 0; j < 32 * S::VEC / 64; j++) {
      const int at = lane + 64 * j, rr = at / S::VEC, c = at % S::VEC;
      if (r0 + rr >= 0)
        *reinterpret_cast<u4*>(static_cast<T*>(a.O) + places[wave][rr] + 8 * c) = *reinterpret_cast<const u4*>(Os + rr * S::KLD + c * 16);
    }
  }
  if constexpr (GATHER) {
    __syncthreads();
    // element e of a product is that of row 8 (e / 4) + 4 half + e % 4 and the lane's key
    float rl[16];
    int re[16];
#pragma unroll
    for (int e = 0; e < 4; e++) {
      const int at = wave % RW * 32 + 8 * e + 4 * half;
      *reinterpret_cast<f4*>(rl + 4 * e) = *reinterpret_cast<const f4*>(row_lse + at);
      *reinterpret_cast<u4*>(re + 4 * e) = *reinterpret_cast<const u4*>(row_end + at);
    }
    if (m == 0) most = 0;
    for (int k0 = 0; k0 < most; k0 += MK) {
      float* now = sums + (k0 / MK & 1) * 4 * KEYS;  // (the other one is still being read)
#pragma unroll
      for (int u = 0; u < Wave::NU; u++) {
        const int key = k0 + ku + 32 * u + i;
        f16v s;
#pragma unroll
        for (int e = 0; e < 16; e++) s[e] = 0.f;
#pragma unroll
        for (int c = 0; c < DH / 16; c++) s = Mma<T>::mul32(w.q[c], ks[u][c], s);
        float acc = 0.f;
#pragma unroll
        for (int e = 0; e < 16; e++) {
          const float p = exp2_fast(fmaf(s[e], a.scale2, -rl[e]));
          acc += key < re[e] ? p : 0.f;
        }
        const u2 y = __builtin_amdgcn_permlane32_swap(__float_as_uint(acc), __float_as_uint(acc), false, false);
        if (half == 0) now[wave * KEYS + 32 * u + i] = __uint_as_float(y[0]) + __uint_as_float(y[1]);
      }
      if (k0 + MK < most) load_slots(k0 + MK);
      __syncthreads();
      if (tid < MK && k0 + tid < most) {
        float all = 0.f;
#pragma unroll
        for (int x = 0; x < RW; x++) all += now[(tid / KEYS * RW + x) * KEYS + tid % KEYS];
        a.weight[head + k0 + tid] += share(a, all);
      }
    }
  }
}

// Maximum and sum of a row over its parts, by a whole wavefront: lane s has part s, s + 64, ...
__device__ inline void row_stats(const AttnArgs& a, int row, int lane, float& ref, float& total) {
  float top = -INFINITY;
  for (int s = lane; s < a.parts; s += 64) top = fmaxf(top, a.ml[(size_t)s * a.rows + row][0]);
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o, 64));
  ref = top == -INFINITY ? 0.f : top;
  total = 0.f;
  for (int s = lane; s < a.parts; s += 64) {
    const f2 x = a.ml[(size_t)s * a.rows + row];
    total += x[1] * exp2_fast(x[0] - ref);
  }
  total = wave_sum(total);
}
__device__ inline bool row_live(const AttnArgs& a, int row, bool& sees) {
  const int head = a.by_T.quot(row), t = row - head * a.T, b = a.by_H.quot(head);
  const int n = slots_of(a, b), m = tokens_of(a, b);
  sees = t < m && a.P + seen(t, n, m) > 0;
  return t < m;
}

// The parts of a row joined by a wavefront (ROW_WAVES = 1) or, where they are many, by a workgroup: a lane has four elements of every
// ROW_WAVES 256 / d_h -th part.  (One sequence of 32768 keys, 32 rows of 128 parts: 37 us by a wavefront each, 8 by a workgroup.)
template <typename T, int DH, int ROW_WAVES>
__device__ inline void join_row(const AttnArgs& a, int row, float* lds) {
  constexpr int C = DH / 4, GR = ROW_WAVES * 64 / C;  // lanes of an output, parts at a time
  const int id = threadIdx.x % (ROW_WAVES * 64), lane = id & 63, c = id % C, p = id / C;
  float ref, total;
  bool sees;
  const bool live = row_live(a, row, sees);
  row_stats(a, row, lane, ref, total);
  f4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int s = p; s < a.parts; s += GR) {
    const f2 x = a.ml[(size_t)s * a.rows + row];
    if (x[0] == -INFINITY && x[1] == 0.f) continue;  // saw nothing: its part is not written
    const f4 y = *reinterpret_cast<const f4*>(a.part + ((size_t)s * a.rows + row) * DH + 4 * c);
    const float f = exp2_fast(x[0] - ref);
#pragma unroll
    for (int e = 0; e < 4; e++) {
      const float x = v[e];
      v[e] += f * y[e];
      if (v[e] != v[e]) v[e] = x + scaled(y[e], f);
    }
  }
#pragma unroll
  for (int e = 0; e < 4; e++)
#pragma unroll
    for (int o = C; o < 64; o <<= 1) v[e] += __shfl_xor(v[e], o, 64);
  if constexpr (ROW_WAVES > 1) {
    f4* part = reinterpret_cast<f4*>(lds);  // [wavefront][C]
    if (lane < C) part[id / 64 * C + lane] = v;
    __syncthreads();
    if (id < C) {
      v = part[id];
#pragma unroll
      for (int w = 1; w < ROW_WAVES; w++) v += part[w * C + id];
    }
  }
  if (p == 0) {
    const int head = a.by_T.quot(row), b = a.by_H.quot(head);
    T* out = static_cast<T*>(a.O) + out_row(a, b, head - b * a.H, row - head * a.T, DH) + 4 * c;
#pragma unroll
    for (int e = 0; e < 4; e++) out[e] = Vec16<T>::round(sees ? v[e] / total : 0.f);
  }
  if (a.lse && id == 0) a.lse[row] = live ? ref + log2f(total) : INFINITY;
}
constexpr int WIDE_JOIN = 9;  // parts from which on a workgroup joins a row
template <typename T, int DH>
__device__ inline void join_rows(const AttnArgs& a, float* lds) {
  if (a.parts >= WIDE_JOIN) {
    join_row<T, DH, 4>(a, blockIdx.x, lds);
  } else {
    const int row = blockIdx.x * 4 + (threadIdx.x >> 6);
    if (row < a.rows) join_row<T, DH, 1>(a, row, lds);
  }
}
inline int join_workgroups(const AttnArgs& a) { return a.parts >= WIDE_JOIN ? a.rows : a.parts > 1 ? (a.rows + 3) / 4 : 0; }

template <typename T, int DH>
__global__ __launch_bounds__(256) void join_kernel(AttnArgs a) {
  __shared__ __attribute__((aligned(16))) float lds[4 * DH];
  join_rows<T, DH>(a, lds);
}

// Few rows: the parts joined, and what slots gather from the scores that were kept.  The first workgroups join rows, each of the others adds the
// probabilities of a sequence's rows to GW slots of a head.
constexpr int GW = 1024;
template <typename T, int DH>
__global__ __launch_bounds__(256) void join_gather_kernel(AttnArgs a, int row_wgs, Div by_chunks) {
  __shared__ float lse[16];
  __shared__ __attribute__((aligned(16))) float lds[4 * DH];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  if ((int)blockIdx.x < row_wgs) {
    join_rows<T, DH>(a, lds);
    return;
  }
  const int item = blockIdx.x - row_wgs, bh = by_chunks.quot(item);
  const int b = a.by_Hk.quot(bh), first = (item - bh * (int)by_chunks.d) * GW, n = slots_of(a, b);
  if (first >= n) return;
  for (int r = wave; r < a.R; r += 4) {
    const int row = bh * a.R + r;
    float ref, total;
    bool sees;
    const bool live = row_live(a, row, sees);
    row_stats(a, row, lane, ref, total);
    if (lane == 0) lse[r] = live ? ref + log2f(total) : INFINITY;
  }
  __syncthreads();
  const int k = first + 4 * (int)threadIdx.x;
  if (k < n) add_weights(a, bh, k, n, tokens_of(a, b), lse);
}

// What slots gather where rows are many and many_kernel has not added it.  float32: 32 keys per wavefront, kept in registers; the rows of queries pass by,
// GR of 16 at a time, whose loads are issued together.  The keys and the first rows come before the length is known.  Products of four float32 elements and their
// loads bound it (128 heads of 64, 40 rows, up to 3000 slots: 39 us).
constexpr int GR = 2, GK = 128;  // (GK: keys of a workgroup)
template <int DH>
__global__ __launch_bounds__(256) void gather_kernel(AttnArgs a, Div by_chunks) {
  typedef float T;
  typedef Mma<T> M;
  typedef typename M::frag frag;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), i = lane & 15, g = lane >> 4;
  const int bh = by_chunks.quot(blockIdx.x), b = a.by_Hk.quot(bh), k0 = (int)(blockIdx.x - bh * by_chunks.d) * GK + wave * 32;
  frag k[2][DH / 32], q[GR][DH / 32];
  float lse[GR];
#pragma unroll
  for (int u = 0; u < 2; u++) {
    const u4* Kr = reinterpret_cast<const u4*>(static_cast<const T*>(a.Kc) + ((size_t)bh * a.cap + min(k0 + 16 * u + i, a.cap - 1)) * DH);
#pragma unroll
    for (int s = 0; s < DH / 32; s++) k[u][s] = frag_of<T>(Kr, 4 * s + g);
  }
  auto load = [&](int r0) {
#pragma unroll
    for (int x = 0; x < GR; x++) {
      const int r = r0 + 16 * x + i;
      const size_t row = (size_t)bh * a.R + min(r, a.R - 1);
      const u4* Qr = reinterpret_cast<const u4*>(static_cast<const T*>(a.Q) + row * DH);
#pragma unroll
      for (int c = 0; c < DH / 32; c++) q[x][c] = frag_of<T>(Qr, 4 * c + g);
      lse[x] = a.lse[row];
      if (r >= a.R) lse[x] = INFINITY;
    }
  };
  load(0);
  const int n = slots_of(a, b), m = tokens_of(a, b);
  if (k0 >= n || m == 0) return;
  f4 acc[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
  for (int r0 = 0; r0 < a.R; r0 += 16 * GR) {
    if (r0 > 0) load(r0);
#pragma unroll
    for (int x = 0; x < GR; x++) {
      const int end = lse[x] == INFINITY ? 0 : seen(a.by_T.rem(min(r0 + 16 * x + i, a.R - 1)), n, m);
#pragma unroll
      for (int u = 0; u < 2; u++) {
        f4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int c = 0; c < DH / 32; c++) s = M::mul(k[u][c], q[x][c], s);
#pragma unroll
        for (int e = 0; e < 4; e++) {
          const float p = exp2_fast(s[e] * a.scale2 - lse[x]);
          acc[u][e] += k0 + 16 * u + 4 * g + e < end ? p : 0.f;
        }
      }
    }
  }
  // the rows' sums: lane i = 0 .. 3 of each 16 takes key 4 g + i
#pragma unroll
  for (int u = 0; u < 2; u++) {
#pragma unroll
    for (int e = 0; e < 4; e++) {
      acc[u][e] += lane_of<0xB1>(acc[u][e]);   // L ^ 1
      acc[u][e] += lane_of<0x4E>(acc[u][e]);   // L ^ 2
      acc[u][e] += lane_of<0x141>(acc[u][e]);  // 7 - L of each 8
      acc[u][e] += lane_of<0x140>(acc[u][e]);  // 15 - L of each 16
    }
    const int at = k0 + 16 * u + 4 * g + i;
    if (i < 4 && at < n) a.weight[(size_t)bh * a.cap + at] += share(a, i == 0 ? acc[u][0] : i == 1 ? acc[u][1] : i == 2 ? acc[u][2] : acc[u][3]);
  }
}

// 16-bit storage: 128 keys a workgroup, 32 of them in a wavefront's registers as the operand of 32 x 32 tiles; 64 rows at a time pass through LDS for all
// four (two stages, as in many_kernel).  Rows that see none of the keys are not fetched.  The scores are formed a second time, since kept they
// would be 4 bytes for each.  (64 x 40 heads of 128, 576 rows, 640 keys: 296 us beside the 469 of the attention.  128 heads of 64, 40 rows, up to 3000
// keys in parts: 15; with the rows in registers, as for float32, 19.5.)
template <typename T, int DH>
__global__ __launch_bounds__(256, 2) void gather_many_kernel(AttnArgs a, Div by_chunks) {
  typedef Mma<T> M;
  typedef typename M::frag frag;
  constexpr int VEC = DH / 8, NV = 64 * VEC / 256, LD = DH * 2 + 16;
  __shared__ __attribute__((aligned(16))) unsigned char rows[2][64 * LD];
  __shared__ float lses[2][64], sums[4][32];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), half = lane >> 5, i = lane & 31;
  const int bh = by_chunks.quot(blockIdx.x), b = a.by_Hk.quot(bh), kmin = (int)(blockIdx.x - bh * by_chunks.d) * GK, k0 = kmin + wave * 32;
  frag k[DH / 16];
  const u4* Kr = reinterpret_cast<const u4*>(static_cast<const T*>(a.Kc) + ((size_t)bh * a.cap + min(k0 + i, a.cap - 1)) * DH);
#pragma unroll
  for (int c = 0; c < DH / 16; c++) k[c].u = Kr[2 * c + half];
  const int n = slots_of(a, b), m = tokens_of(a, b), tiles = (a.R + 63) / 64;
  if (kmin >= n || m == 0) return;
  // the next tile from t on of which some row sees the first key
  auto next = [&](int t) {
    for (; t < tiles; t++) {
      int least, most;
      seen_by(a, t * 64, min(t * 64 + 63, a.R - 1), n, m, least, most);
      if (most > kmin) break;
    }
    return t;
  };
  u4 qr[NV];
  float lse = INFINITY;
  auto fetch = [&](int t) {
    const u4* Qr = reinterpret_cast<const u4*>(static_cast<const T*>(a.Q) + ((size_t)bh * a.R + t * 64) * DH);
    const int there = min(64, a.R - t * 64) * VEC - 1;
#pragma unroll
    for (int j = 0; j < NV; j++) qr[j] = Qr[min(tid + 256 * j, there)];
    const int r = t * 64 + (tid & 63);
    lse = a.lse[(size_t)bh * a.R + min(r, a.R - 1)];
    if (r >= a.R) lse = INFINITY;
  };
  auto store = [&](int stage) {
#pragma unroll
    for (int j = 0; j < NV; j++) {
      const int at = tid + 256 * j;
      *reinterpret_cast<u4*>(rows[stage] + at / VEC * LD + at % VEC * 16) = qr[j];
    }
    if (tid < 64) lses[stage][tid] = lse;
  };
  float acc[16];
#pragma unroll
  for (int e = 0; e < 16; e++) acc[e] = 0.f;
  int t = next(0), stage = 0;
  if (t < tiles) {
    fetch(t);
    store(0);
  }
  int t2 = next(t + 1);
  if (t2 < tiles) fetch(t2);
  __syncthreads();
  while (t < tiles) {
#pragma unroll
    for (int u = 0; u < 2; u++) {
      const int r = t * 64 + 32 * u + i;
      const float l = lses[stage][32 * u + i];
      const int end = l == INFINITY ? 0 : seen(a.by_T.rem(min(r, a.R - 1)), n, m);
      if (!__ballot(end > k0)) continue;
      f16v s;
#pragma unroll
      for (int e = 0; e < 16; e++) s[e] = 0.f;
      const unsigned char* qrow = rows[stage] + (32 * u + i) * LD + 16 * half;
#pragma unroll
      for (int c = 0; c < DH / 16; c++) {
        frag q;
        q.u = *reinterpret_cast<const u4*>(qrow + 32 * c);
        s = M::mul32(k[c], q, s);
      }
      if (!__ballot(end < k0 + 32)) {
#pragma unroll
        for (int e = 0; e < 16; e++) acc[e] += exp2_fast(fmaf(s[e], a.scale2, -l));
      } else {
#pragma unroll
        for (int e = 0; e < 16; e++) {
          const float p = exp2_fast(fmaf(s[e], a.scale2, -l));
          acc[e] += k0 + 8 * (e >> 2) + 4 * half + (e & 3) < end ? p : 0.f;
        }
      }
    }
    if (t2 < tiles) store(stage ^ 1);  // (last read before the last barrier)
    __syncthreads();
    t = t2;
    stage ^= 1;
    t2 = next(t + 1);
    if (t2 < tiles) fetch(t2);
  }
#pragma unroll
  for (int e = 0; e < 16; e++) {
    float x = acc[e];
    x += lane_of<0xB1>(x);
    x += lane_of<0x4E>(x);
    x += lane_of<0x141>(x);
    x += lane_of<0x140>(x);
    const u2 w = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    if (i == 0) sums[wave][8 * (e >> 2) + 4 * half + (e & 3)] = __uint_as_float(w[0]) + __uint_as_float(w[1]);
  }
  wave_lds_order();
  if (lane < 32 && k0 + lane < n) a.weight[(size_t)bh * a.cap + k0 + lane] += share(a, sums[wave][lane]);
}

// How a call is cut.  The prefix of an image's sequences is read once for all of them where the rows of one sequence do not fill a
// tile by themselves; else a sequence's rows go over its prefix and its cache in one sweep.
constexpr int FEW_ROWS = 16;
static Job make_job(const CachePlan& pl, int groups, int rows, int keys, bool packed, bool prefix, bool cache, bool alone) {
  const bool many = rows > FEW_ROWS && pl.esize == 2;
  const int per = !many ? FEW_ROWS : rows <= MROWS / 2 ? MROWS / 2 : MROWS, tile = many ? MK : FK, least = 4;
  Job j = {groups, rows, (rows + per - 1) / per, 1, 0, packed, prefix, cache, many, false, 0, Div(1), Div(1)};
  j.by_tiles = Div((uint32_t)j.tiles);
  const long long items = (long long)groups * j.tiles, tiles = (keys + tile - 1) / tile + (prefix && cache ? 1 : 0);
  // Few rows on a part of the chip, up to 768 keys: eight wavefronts take all keys, and nothing has to be joined.  (One sequence, 32 heads,
  // us in one sweep and in parts: 640 keys 10.5 and 11.9, 1000 14.3 and 12.5, 2000 21 and 15.)
  j.wide = !many && alone && items <= 256 && tiles > 4 && tiles <= 24 && !(pl.esize == 4 && pl.dh == 128);
  j.share = (int)tiles;
  if (j.wide) return j;
  // Parts of the keys: two workgroups for each compute unit, if there are four tiles for each.  Many rows: no more than two, since a second round of
  // workgroups costs what the parts spare, and their joining more (us, with up to three and two: 96 heads of 592 rows and 540 keys 89 and 56; 64 of 552
  // rows and 532 keys 68 and 49; 120 of 108 rows and 111 keys, where parts had two tiles, 29 and 13).  Few rows
  // of long caches take four of them, which evens out sequences of different lengths, where a wavefront still has four tiles.  (us, two and
  // four: 4 sequences of up to 32768 keys 99 and 94; one 24 and 29.)
  long long s = many ? 512 / items : (512 + items - 1) / items;
  if (s > (tiles + least - 1) / least) s = (tiles + least - 1) / least;
  if (!many) {
    long long t = (1024 + items - 1) / items;
    if (t > tiles / 16) t = tiles / 16;
    if (t > s) s = t;
  }
  j.splits = s < 1 ? 1 : (int)s;
  j.share = (int)((tiles + j.splits - 1) / j.splits);
  j.by_splits = Div((uint32_t)j.splits);
  return j;
}
struct Cut {
  int jobs;
  Job job[2];
  int parts;
};
static Cut make_cut(const CachePlan& pl, int max_len) {
  Cut c = {};
  // Reading a prefix once pays for a second kind of parts and their joining (5 us) from 32 MB on that are not read again.
  const double again = (double)pl.images * (pl.each - 1) * pl.Hk * pl.P * pl.dh * 2.0 * pl.esize;
  if (pl.images > 0 && pl.R <= FEW_ROWS && again >= 32e6) {
    c.jobs = 2;
    c.job[0] = make_job(pl, pl.images * pl.Hk, pl.each * pl.R, pl.P, true, true, false, false);
    c.job[1] = make_job(pl, pl.B * pl.Hk, pl.R, max_len, false, false, true, false);
    c.job[1].part0 = c.job[0].splits;
    c.parts = c.job[0].splits + c.job[1].splits;
  } else {
    c.jobs = 1;
    c.job[0] = make_job(pl, pl.B * pl.Hk, pl.R, pl.P + max_len, false, pl.P > 0, true, true);
    c.parts = c.job[0].splits;
  }
  return c;
}

// Rows of parts (none where a row has a single one).
static size_t part_rows(const CachePlan& pl) {
  if (pl.B == 0) return 0;
  // the most parts of any max_len: longer caches are cut into no fewer
  const int parts = make_cut(pl, pl.cap).parts;
  return parts > 1 ? (size_t)pl.B * pl.H * pl.T * parts : 0;
}
// Few rows of a sequence: their scores are kept, so that the keys are read once.
static bool keeps_scores(const CachePlan& pl) { return pl.R <= FEW_ROWS; }
static int score_ld(int max_len) { return round_up(max_len, FK) + FK; }
static size_t score_elems(const CachePlan& pl) {
  return keeps_scores(pl) ? (size_t)pl.B * pl.H * pl.T * score_ld(pl.cap) : 0;
}
size_t attention_bytes(const CachePlan& pl) {
  return align256((size_t)pl.B * pl.H * pl.T * 4) + align256(part_rows(pl) * 8) + align256(score_elems(pl) * 4) + part_rows(pl) * pl.dh * 4;
}

template <typename K>
static bool allow_lds(K kernel, int bytes) {  // (and up to 2 KB that the kernels declare)
  return bytes + 2048 <= 64 * 1024 ||
         hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, bytes) == hipSuccess;
}
static long long workgroups(const Job& j) { return (long long)j.groups * j.tiles * j.splits; }

template <typename T, int DH>
static int attention_launch(const CachePlan& pl, AttnArgs a, hipStream_t st) {
  const Cut cut = make_cut(pl, pl.max_len);
  a.parts = cut.parts;
  const int row_wgs = join_workgroups(a);
  // slots of a workgroup that gathers: from the scores that were kept, where parts are joined, or by scores formed anew
  const int per = a.score ? GW : GK;
  const long long chunks = ((long long)pl.max_len + per - 1) / per, gather_wgs = a.weight ? chunks * pl.B * pl.Hk : 0;
  if (!grid_fits(workgroups(cut.job[0]) + workgroups(cut.job[1]), cut.job[0].wide ? 512 : 256) || !grid_fits(row_wgs + gather_wgs, 256)) return TC_ERR_SHAPE;
  // many_kernel gathers itself where its workgroups have all rows and all keys of a group, but for more than 64 rows of heads of 128: two wavefronts
  // on a SIMD, each with a chain of loads and products, take longer than a kernel of its own (us, here and there, 1024 heads: 100 rows of 64, 640 + 150 keys, 54 and 61;
  // 128 rows of 128, 1000 keys, 242 and 215; 40 rows of 128, 300 keys, 2048 heads, 106 and 110).
  constexpr bool WIDE_ROWS = DH == 64;
  const bool gathers = a.weight && cut.parts == 1 && cut.job[0].many && cut.job[0].tiles == 1 && (WIDE_ROWS || cut.job[0].rows <= MROWS / 2);
  Job few[2] = {};
  int nf = 0;
  for (int k = 0; k < cut.jobs; k++) {
    if (!cut.job[k].many) {
      few[nf++] = cut.job[k];
      continue;
    }
    if constexpr (sizeof(T) == 2) {
      const auto kernel = cut.job[k].rows <= MROWS / 2 ? (gathers ? many_kernel<T, DH, 2, true> : many_kernel<T, DH, 2, false>)
                                                       : (WIDE_ROWS && gathers ? many_kernel<T, DH, 1, WIDE_ROWS> : many_kernel<T, DH, 1, false>);
      if (!allow_lds(kernel, ManyShape<DH>::LDS)) return TC_ERR_HIP;
      kernel<<<(unsigned)workgroups(cut.job[k]), 256, ManyShape<DH>::LDS, st>>>(a, cut.job[k]);
    }
  }
  if (nf > 0) {
    typedef FewShape<T, DH> F;
    // Where there are more workgroups than fit on the chip at once, and each has few tiles, one or two wavefronts have them: more are resident, no
    // wavefront is idle and there is less to join.  (1960 heads of 128, bf16, us by 1, 2 and 4 wavefronts: 10 keys 12, 17 and 28; 160 keys
    // 32, 35 and 40; 300 keys 58, 60 and 64; 700 keys 157, 154 and 151.  2048 heads of 200 keys and 256 prefixes of 640: 48, 46 and 54.)
    const long long wgs = workgroups(few[0]) + workgroups(few[1]);
    const int share = few[0].share > few[1].share ? few[0].share : few[1].share;
    const bool crowded = wgs > 256 * (160 * 1024 / (4 * F::WAVE + 1024));
    const int waves = few[0].wide ? F::MOST : crowded && share <= 6 ? 1 : crowded && share <= 10 ? 2 : 4;
    auto launch = [&](auto kernel) -> int {
      if (!allow_lds(kernel, waves * F::WAVE)) return TC_ERR_HIP;
      kernel<<<(unsigned)wgs, 64 * waves, waves * F::WAVE, st>>>(a, few[0], few[1]);
      return TC_OK;
    };
    const int rc = waves == 1 ? launch(a.score ? few_kernel<T, DH, true, 1> : few_kernel<T, DH, false, 1>)
                 : waves == 2 ? launch(a.score ? few_kernel<T, DH, true, 2> : few_kernel<T, DH, false, 2>)
                 : waves == 4 ? launch(a.score ? few_kernel<T, DH, true, 4> : few_kernel<T, DH, false, 4>)
                              : launch(a.score ? few_kernel<T, DH, true, F::MOST> : few_kernel<T, DH, false, F::MOST>);
    if (rc != TC_OK) return rc;
  }
  if (a.score) {
    if (a.parts > 1) join_gather_kernel<T, DH><<<(unsigned)(row_wgs + gather_wgs), 256, 0, st>>>(a, row_wgs, Div((uint32_t)chunks));
    return check_launch();  // (a single part: few_kernel has gathered)
  }
  if (a.parts > 1) join_kernel<T, DH><<<row_wgs, 256, 0, st>>>(a);
  if (a.weight && !gathers) {
    const Div by_chunks((uint32_t)chunks);
    if constexpr (sizeof(T) == 2) gather_many_kernel<T, DH><<<(unsigned)gather_wgs, 256, 0, st>>>(a, by_chunks);
    else gather_kernel<DH><<<(unsigned)gather_wgs, 256, 0, st>>>(a, by_chunks);
  }
  return check_launch();
}

}  // namespace tc

using namespace tc;

extern "C" int tc_cache_attention(const tc_cache* c, const void* Q, const void* K_prefix, const void* V_prefix, const void* K_cache,
                                  const void* V_cache, const int32_t* len, const int32_t* q_len, void* O, float* weight, void* ws,
                                  size_t ws_bytes, void* stream) {
  CachePlan pl;
  int rc = make_cache_plan(c, &pl);
  if (rc != TC_OK) return rc;
  if (pl.B == 0) return TC_OK;
  if (!Q || !K_cache || !V_cache || !len || !O || (pl.P > 0 && (!K_prefix || !V_prefix))) return TC_ERR_NULL;
  if (misaligned(Q) || misaligned(K_prefix) || misaligned(V_prefix) || misaligned(K_cache) || misaligned(V_cache) || misaligned(len) ||
      misaligned(q_len) || misaligned(O) || misaligned(weight))
    return TC_ERR_ALIGN;
  if ((rc = check_cache_ws(pl, ws, ws_bytes)) != TC_OK) return rc;
  AttnArgs a = {};
  a.Q = Q; a.Kp = K_prefix; a.Vp = V_prefix; a.Kc = K_cache; a.Vc = V_cache; a.len = len; a.q_len = q_len; a.O = O; a.weight = weight;
  a.H = pl.H; a.Hk = pl.Hk; a.G = pl.G; a.T = pl.T; a.R = pl.R; a.cap = pl.cap; a.max_len = pl.max_len; a.each = pl.each; a.P = pl.P;
  a.by_T = Div(a.T); a.by_R = Div(a.R); a.by_H = Div(a.H); a.by_Hk = Div(a.Hk); a.by_each = Div(a.each);
  a.rows = pl.B * pl.H * pl.T;
  a.scale2 = pl.scale * 1.44269504088896340736f;
  int bits = 1;  // 2^bits is more than twice the keys of a row
  while ((1LL << bits) <= 2LL * pl.P + 2LL * pl.max_len) bits++;
  a.offset = c->dtype == TC_F16 ? -15.f : (float)bits;  // (half: its values times sums of 2^15 are far from the range of float32)
  char* w = static_cast<char*>(ws);
  a.lse = weight ? reinterpret_cast<float*>(w) : nullptr;
  w += align256((size_t)a.rows * 4);
  a.ml = reinterpret_cast<f2*>(w);
  w += align256(part_rows(pl) * 8);
  a.score = weight && keeps_scores(pl) ? reinterpret_cast<float*>(w) : nullptr;
  a.score_ld = score_ld(pl.max_len);
  w += align256(score_elems(pl) * 4);
  a.part = reinterpret_cast<float*>(w);
  const hipStream_t st = (hipStream_t)stream;
  if (pl.dh == 64)
    return c->dtype == TC_F32 ? attention_launch<float, 64>(pl, a, st) : c->dtype == TC_BF16 ? attention_launch<uint16_t, 64>(pl, a, st)
                                                                                              : attention_launch<f16_t, 64>(pl, a, st);
  return c->dtype == TC_F32 ? attention_launch<float, 128>(pl, a, st) : c->dtype == TC_BF16 ? attention_launch<uint16_t, 128>(pl, a, st)
                                                                                            : attention_launch<f16_t, 128>(pl, a, st);
}
