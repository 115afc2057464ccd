// Loss of a student that learns from a teacher's largest logits and from labels, and the
// gradient of the student's logits, on the whole vocabulary or one rank's share of it.
//
// A token has the student's logits z over the vocabulary, the teacher's entries (id_k, t_k),
// k < K, and a label c.  With the temperature T and the weight a:
//   p = softmax(t / T) over the entries that are there
//   loss = a T^2 sum_k p_k (log p_k - log softmax(z / T)[id_k]) - (1 - a) log softmax(z)[c]
//   dz_v = w (a T (P softmax(z / T)_v - sum_{k: id_k = v} p_k) + (1 - a) L (softmax(z)_v - [v = c])),
// w the gradient that reaches the loss; P = sum p_k is 1, or 0 without entries, L is 1, or 0
// without a label.  With m = max z, S_T = sum exp((z - m) / T) and S_1 = sum exp(z - m),
//   loss = a T^2 P log S_T + (1 - a) L log S_1 - lin,
//   lin = sum_k (a T p_k (z_k - m) - a T^2 p_k log p_k) + (1 - a) L (z_c - m).
// Everything in z is a difference from m, so a common offset of the logits costs nothing.  A
// rank has its columns' m and sums, the part of lin, P and L that its columns hold, and the
// teacher's own maximum and sum (which all ranks form from all entries): the token's row of
// statistics.  Ranks' rows join by moving to the largest m.
//
// Bound by memory: the logits are read once (maximum and sums in one pass, the sums rescaled
// when the maximum grows), the gradient is written once.  8192 x 50304 in bf16 with 64 entries, T =
// 2, the kernels in passes over changing inputs: loss 142 us (5.8 TB/s, reading only; a large copy has
// 5.1 both ways), loss and gradient 302 (5.5); called one after another on buffers in turn: loss with
// statistics 164, loss and gradient 294, gradient from the statistics 269 (6.1), in fp32 on half
// the rows 152, 301 and 270.  Three quarters of the loss's time the vector units are busy too: two
// exponentials a logit.  Sums are fp32, of no more than some hundred terms in a row, each value of
// the gradient is formed in fp32 and rounded once, nothing depends on timing.
#include <algorithm>

#include "common.h"
#include "kernels.h"
#include "wave.h"

namespace merak {

constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// A launch's tokens; what it needs of the call.
struct DistillArgs {
  int tokens, vocab, ld, top;
  int slots;                     // of the entries' table
  long long first, total;
  float alpha, tau;
  float rate_t, rate_1;          // log2(e) / T, log2(e); with one sum rate_t is its rate
  bool want_t, want_1;           // sums that the loss needs
  bool id64, label64, teacher_bf16;
  bool past;                     // the gradient is written past the caches
  const void* ids;               // [tokens][top], null without entries
  const void* teacher;
  const void* labels;            // null without labels
};

__device__ __forceinline__ long long id_at(const void* p, bool wide, size_t i) {
  return wide ? static_cast<const long long*>(p)[i] : static_cast<const int*>(p)[i];
}

// The token's own columns of the vocabulary, -1 for an id that is another rank's or none's.
__device__ __forceinline__ int column_of(const DistillArgs& a, long long id) {
  return id >= a.first && id < a.total && id - a.first < a.vocab ? (int)(id - a.first) : -1;
}

__device__ __forceinline__ float teacher_at(const DistillArgs& a, size_t i) {
  return a.teacher_bf16 ? bf2f(static_cast<const bf16_t*>(a.teacher)[i]) : static_cast<const float*>(a.teacher)[i];
}

// A token's entries and its label (entry `top`) in LDS.  For the gradient there is a hash table of
// the entries' columns too, as an id may be there more than once.  A column's first entry (the label,
// where there is none) forms the gradient there, and is listed for the thread that writes the 16 bytes
// around it.  It needs the sum of the column's p = exp((t - max) / T), the same in any order: of two
// entries it is their fp32 sum, of more a whole number of units of 2^-44 of the largest one's power of two.
struct Slot {
  int col, first, last;
};
struct Entry {
  int col;      // own column, or -1
  float t;      // teacher's logit; then p
  float z;      // student's logit at the column; then the bits of the gradient there
  int next;     // place in the table; then the thread's next entry, -1 at the end
};
struct Entries {
  Entry* at;
  // gradient only
  unsigned long long* sum;  // how many came behind the first one; then see sum_many
  Slot* slot;
  int* head;    // [threads] the thread's first entry
  int* flags;   // whether a column has more than two entries; whether the label's has one
  int slots;    // a power of two
};
__host__ __device__ constexpr int entry_slots(int top) {
  int n = 32;
  while (4 * n < 5 * (top + 1)) n *= 2;
  return n;
}
__host__ __device__ constexpr size_t entries_bytes(int top, int nt, bool grad) {
  return (size_t)(top + 1) * sizeof(Entry) + (grad ? nt * 4 + (size_t)entry_slots(top) * (8 + sizeof(Slot)) : 0);
}
__device__ __forceinline__ Entries entries_in(char* lds, int* flags, int top, int slots) {
  Entries en;
  en.flags = flags;
  en.at = reinterpret_cast<Entry*>(lds);
  en.sum = reinterpret_cast<unsigned long long*>(en.at + top + 1);
  en.slot = reinterpret_cast<Slot*>(en.sum + slots);
  en.head = reinterpret_cast<int*>(en.slot + slots);
  en.slots = slots;
  return en;
}

// An empty table and empty lists; a barrier follows before the first entry.
template <int NT>
__device__ __forceinline__ void clear_table(const Entries& en) {
  for (int i = threadIdx.x; i < en.slots; i += NT) {
    en.sum[i] = 0;
    en.slot[i] = Slot{-1, 0x7fffffff, -1};
  }
  en.head[threadIdx.x] = -1;
  if (threadIdx.x < 2) en.flags[threadIdx.x] = 0;
}

// Entry k into the table.  (The count stands behind the loop: in it, it cost 3% of the loss and gradient of
// 8192 x 6288 with 1024 entries where no id repeats; the label in the table as well, 3% of 333 x 50257.)
__device__ __forceinline__ void into_table(const Entries& en, int k, int c, int label) {
  int h = (int)(((unsigned)c * 2654435761u >> 8) & (unsigned)(en.slots - 1));
  int was;
  while ((was = atomicCAS(&en.slot[h].col, -1, c)) != -1 && was != c)  // there are more slots than entries
    h = (h + 1) & (en.slots - 1);
  en.at[k].next = h;
  atomicMin(&en.slot[h].first, k);
  atomicMax(&en.slot[h].last, k);
  if (__builtin_expect(was == c, 0) && atomicAdd(&en.sum[h], 1ull) > 0) en.flags[0] = 1;
  if (c == label) en.flags[1] = 1;
}

constexpr int kUnitBits = 44, kSumBits = 56;  // 1024 p below 2^45 units each

__device__ __forceinline__ unsigned long long sum_now(const unsigned long long& sum) {
  return __hip_atomic_load(&sum, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
}

// The sums of p (a normal number) of columns with more than two entries, between barriers: the
// exponent of the largest one goes into the upper 8 bits (more than any number of entries), then all
// into the others in units of 2^-44 of that (what is below one is cut off: 2^-34 of the sum at most).
// In units that are the same for all columns the small p of such a column lose their digits, which
// the gradient has where the student's probability is as small.
template <int NT>
__device__ __forceinline__ void sum_many(const Entries& en, int top) {
  if (!en.flags[0]) return;  // the same for the whole workgroup
  auto each = [&](auto f) {
    for (int k = threadIdx.x; k < top; k += NT) {
      const Entry e = en.at[k];
      if (e.col >= 0 && sum_now(en.sum[e.next]) > 1) f(en.sum[e.next], __float_as_uint(e.t));
    }
    __syncthreads();
  };
  each([](unsigned long long& sum, uint32_t p) {
    atomicMax(&sum, (unsigned long long)(p >> 23 & 255) << kSumBits);
  });
  each([](unsigned long long& sum, uint32_t p) {
    const int most = (int)(sum_now(sum) >> kSumBits);
    const int shift = kUnitBits - 23 - (most - (int)(p >> 23 & 255));
    const unsigned long long m = (p & 0x7fffffu) | 0x800000u;
    atomicAdd(&sum, shift >= 0 ? m << shift : shift > -24 ? m >> -shift : 0);
  });
}

// The sum of p of a column with the first entry's p.
__device__ __forceinline__ float column_sum(const Entries& en, int h, const Slot& at, float p) {
  if (at.first == at.last) return p;
  const unsigned long long s = en.sum[h];
  if (s == 1) return p + en.at[at.last].t;
  return ldexpf(__ull2float_rn(s & ((1ull << kSumBits) - 1)), (int)(s >> kSumBits) - 127 - kUnitBits);
}

// 16 bytes of logits as floats; NONE is -infinity in each of them.
template <typename T> struct Vec;
template <> struct Vec<bf16_t> {
  static constexpr int N = 8;
  static constexpr uint32_t NONE = 0xff80ff80u;
  static __device__ __forceinline__ void get(u32x4_t r, float (&v)[8]) { unpack8(r, v); }
  static __device__ __forceinline__ u32x4_t put(const float (&v)[8]) {
    return u32x4_t{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])};
  }
};
template <> struct Vec<float> {
  static constexpr int N = 4;
  static constexpr uint32_t NONE = 0xff800000u;
  static __device__ __forceinline__ void get(u32x4_t r, float (&v)[4]) {
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = __uint_as_float(r[e]);
  }
  static __device__ __forceinline__ u32x4_t put(const float (&v)[4]) {
    return u32x4_t{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
  }
};

// The first `n` values of r, `rest` in the places of the others.
template <typename T>
__device__ __forceinline__ u32x4_t first_values(u32x4_t r, int n, float rest) {
  float v[Vec<T>::N];
  Vec<T>::get(r, v);
#pragma unroll
  for (int e = 0; e < Vec<T>::N; ++e) v[e] = e < n ? v[e] : rest;
  return Vec<T>::put(v);
}

// What a maximum's differences are formed from: 0 where nothing was above -infinity.
__device__ __forceinline__ float base_of(float m) { return m == -INFINITY ? 0.0f : m; }

// By how much sums relative to the maximum m move to those relative to `base` (sums that are 0
// stay 0: the difference from a base far below 0 would have no finite exponential).
__device__ __forceinline__ float moved(float m, float base) { return m == -INFINITY ? 0.0f : m - base; }

// A sum or maximum over the workgroup, behind which all its threads see the entries in LDS (a
// workgroup of one wave exchanges nothing through LDS for it, so the barrier comes by itself).
template <typename Op, int NT, int N>
__device__ __forceinline__ void reduce_behind_barrier(float (&v)[N], float* red) {
  block_reduce<Op, NT>(v, red);
  if constexpr (NT == 64) __syncthreads();
}

struct Stats {
  float m, s1, st, lin, mass, label, tm, ts;
};

__device__ __forceinline__ float loss_of(const Stats& s, float alpha, float tau) {
  float l = -s.lin;
  if (s.mass != 0.0f) l += alpha * tau * tau * s.mass * logf(s.st);
  if (s.label != 0.0f) l += (1.0f - alpha) * s.label * logf(s.s1);
  return l;
}

__device__ __forceinline__ void store_stats(float* p, const Stats& s) {
  reinterpret_cast<f32x4_t*>(p)[0] = f32x4_t{s.m, s.s1, s.st, s.lin};
  reinterpret_cast<f32x4_t*>(p)[1] = f32x4_t{s.mass, s.label, s.tm, s.ts};
}
__device__ __forceinline__ Stats load_stats(const float* p) {
  const f32x4_t a = reinterpret_cast<const f32x4_t*>(p)[0], b = reinterpret_cast<const f32x4_t*>(p)[1];
  return Stats{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
}

// exp((z - base) / T) as 2^(z rate - c), c = base * rate rounded: one fused step an element.  What c
// is off by, the same for every z, is put back into the sum of them (`off`, a factor that stays
// within 2^-4 and 2^4 for bases up to 2^16, at every temperature).
struct Exponent {
  float rate, c, base;
  __device__ __forceinline__ Exponent(float base, float rate) : rate(rate), c(base * rate), base(base) {}
  __device__ __forceinline__ float of(float z) const { return exp2_fast(fmaf(z, rate, -c)); }
  __device__ __forceinline__ float off() const { return exp2_fast(fmaf(-base, rate, c)); }
};

// Where the maximum is further out (logits with a large offset; a row that is masked with the type's
// lowest value) the base is subtracted first and the exponentials' own base is 0.
constexpr float kFar = 0x1p16f;
__device__ __forceinline__ bool is_far(float base) { return fabsf(base) > kFar && fabsf(base) < INFINITY; }
__device__ __forceinline__ float near_base(float m) { return m == -INFINITY ? 0.0f : fminf(fmaxf(m, -kFar), kFar); }

// The two exponentials, exp((z - base) / T) and exp(z - base): ONE is enough where the loss needs
// one or T = 1, at T = 2 and T = 4 the second is the first's square or its square's (their c and
// off are exact multiples then; the first's relative error is doubled or taken four times), else
// there are TWO.  In passes over changing inputs the loss of 8192 x 50304 in bf16 takes 142 us at T = 2,
// 166 with both (T = 3).
enum Sums { ONE = 0, TWO = 1, SQUARE = 2, FOURTH = 4 };
template <int M>
struct Exponents {
  Exponent t, one;
  __device__ __forceinline__ Exponents(const DistillArgs& a, float base) : t(base, a.rate_t), one(base, a.rate_1) {}
  __device__ __forceinline__ void of(float z, float* et, float* e1) const {
    *et = t.of(z);
    if (M == ONE) *e1 = *et;
    else if (M == TWO) *e1 = one.of(z);
    else if (M == SQUARE) *e1 = *et * *et;
    else *e1 = (*et * *et) * (*et * *et);
  }
};

// The gradient's factors of the two exponentials (with one, `t` is that of both).
template <int M>
struct Slopes {
  Exponents<M> exps;
  float t, one;
  __device__ __forceinline__ Slopes(const DistillArgs& a, const Stats& s, float w, bool far)
      : exps(a, far ? 0.0f : base_of(s.m)) {
    t = s.mass != 0.0f ? w * a.alpha * a.tau * s.mass / s.st : 0.0f;
    one = s.label != 0.0f ? w * (1.0f - a.alpha) * s.label / s.s1 : 0.0f;
    if (M == ONE) t += one;
    t *= exps.t.off();
    one *= exps.one.off();
  }
  __device__ __forceinline__ float of(float z) const {
    float et, e1;
    exps.of(z, &et, &e1);
    if (M == ONE) return t * et;
    if (M == SQUARE) return et * fmaf(one, et, t);
    return fmaf(one, e1, t * et);
  }
};

// 16 bytes of the gradient from those of the logits, less `from`, of which `n` are columns of the
// vocabulary.
template <typename T, int M, bool FAR = false>
__device__ __forceinline__ u32x4_t slopes_of(const Slopes<M>& f, u32x4_t z, int n, float from = 0.0f) {
  constexpr int N = Vec<T>::N;
  float v[N];
  Vec<T>::get(z, v);
#pragma unroll
  for (int e = 0; e < N; ++e) v[e] = f.of(FAR ? v[e] - from : v[e]);
  if (n < N) {
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] = e < n ? v[e] : 0.0f;
  }
  return Vec<T>::put(v);
}

// Which of a thread's chunks (NT threads, from column lo on) have entries: bit i for chunk i, at most 32.
template <typename T, int NT>
__device__ __forceinline__ uint32_t chunks_with_entries(const Entries& en, int lo) {
  uint32_t m = 0;
  for (int k = en.head[threadIdx.x]; k >= 0; k = en.at[k].next) m |= 1u << ((en.at[k].col - lo) / (Vec<T>::N * NT));
  return m;
}

// x's bits in the place of value e of 16 bytes, if it is one of theirs.
__device__ __forceinline__ void put_value(u32x4_t& v, int e, uint32_t x, bf16_t) {
  const uint32_t shift = (e & 1) * 16, mask = 0xffffu << shift, bits = x << shift;
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = (e >> 1) == i ? (v[i] & ~mask) | bits : v[i];
}
__device__ __forceinline__ void put_value(u32x4_t& v, int e, uint32_t x, float) {
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = e == i ? x : v[i];
}
__device__ __forceinline__ uint32_t bits_of(float x, bf16_t) { return f2bf(x); }
__device__ __forceinline__ uint32_t bits_of(float x, float) { return __float_as_uint(x); }

// A thread's 16 bytes from column c on, with the entries' values in their places.
template <typename T>
__device__ __forceinline__ u32x4_t with_entries(const Entries& en, u32x4_t v, int c) {
  for (int k = en.head[threadIdx.x]; k >= 0;) {
    const Entry e = en.at[k];
    put_value(v, e.col - c, __float_as_uint(e.z), T());
    k = e.next;
  }
  return v;
}

// Columns [lo, hi) of a row: dz from z (the same memory, or another row's), U loads in flight.
template <typename T, int NT, int M, bool FAR>
__device__ __forceinline__ void write_slopes(const DistillArgs& a, const Slopes<M>& f, const Entries& en, const T* z,
                                             T* dz, int lo, int hi, float base) {
  constexpr int N = Vec<T>::N, U = 4;
  for (int c0 = lo + (int)threadIdx.x * N; c0 < hi; c0 += NT * N * U) {
    u32x4_t r[U] = {};
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (c0 + NT * N * u < hi) r[u] = *reinterpret_cast<const u32x4_t*>(z + c0 + NT * N * u);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int c = c0 + NT * N * u;
      if (c < hi)
        *reinterpret_cast<u32x4_t*>(dz + c) = with_entries<T>(en, slopes_of<T, M, FAR>(f, r[u], a.vocab - c, base), c);
    }
  }
}

// Zeros behind the vocabulary in the 16 bytes that hold its end (where the row's factors are NaN
// the -infinity there has become NaN too), by the thread that has written them.
template <typename T, int NT>
__device__ __forceinline__ void write_padding(const DistillArgs& a, T* dz, int lo) {
  constexpr int N = Vec<T>::N;
  if (a.vocab % N && (int)threadIdx.x == (a.vocab - lo) / N % NT)
    for (int c = a.vocab; c % N; ++c) dz[c] = T(0);
}

// A thread's maximum and sums of a part of its columns, relative to near_base(m).
struct Part {
  float m, st, s1;
};

template <int M>
__device__ __forceinline__ void join_part(const DistillArgs& a, Part& all, const Part& p) {
  if (all.m == -INFINITY || p.m == -INFINITY) {  // a sum of nothing is 0 (or NaN) and stays it, wherever the base goes
    all = Part{fmaxf(all.m, p.m), all.st + p.st, all.s1 + p.s1};
    return;
  }
  const float m = fmaxf(all.m, p.m);
  const Exponents<M> now(a, near_base(m)), x(a, near_base(all.m)), y(a, near_base(p.m));
  all.st = all.st * exp2_fast(x.t.c - now.t.c) + p.st * exp2_fast(y.t.c - now.t.c);
  if (M != ONE) all.s1 = all.s1 * exp2_fast(x.one.c - now.one.c) + p.s1 * exp2_fast(y.one.c - now.one.c);
  all.m = m;
}

// A thread's sums of exponentials where the maximum is far, kFarRun at a time.
constexpr int kFarRun = 1024;
template <typename T, int NT, int M>
__device__ __forceinline__ void far_sums(const DistillArgs& a, const T* z, float base, float* st, float* s1) {
  const Exponents<M> exps(a, 0.0f);
  *st = *s1 = 0.0f;
  for (int c = threadIdx.x; c < a.vocab;) {
    float rt = 0.0f, r1 = 0.0f;
    for (int n = 0; n < kFarRun && c < a.vocab; ++n, c += NT) {
      float et, e1;
      exps.of(Elem<T>::to_f(z[c]) - base, &et, &e1);
      rt += et;
      r1 += e1;
    }
    *st += rt;
    *s1 += r1;
  }
}

template <typename T, int NT>
__device__ __forceinline__ void write_zeros(const DistillArgs& a, T* dz, int lo, int hi) {
  for (int c = lo + (int)threadIdx.x * Vec<T>::N; c < hi; c += NT * Vec<T>::N) {
    if (a.past) store16<true>(dz + c, u32x4_t{0, 0, 0, 0});
    else store16<false>(dz + c, u32x4_t{0, 0, 0, 0});
  }
}

// The gradient at the columns that have entries: the table is filled (behind a barrier), the lists
// are whole behind the next one.  A column's place in a list is the one thing that depends on
// timing, and it changes nothing.  wt: weight of p, wl: of the label.
// (Written by a store of its own behind that of the 16 bytes, each entry cost a part of a line once
// more: loss and gradient of 32768 x 6288 with 64 entries 266 us, 201 so, in the form of that time
// (now 180).  Looking for repeated ids by comparing every pair instead of a table: 8192 x 50304 with
// 256 entries 409 us, with 1024 1697; so 307 and 500.)
template <typename T, int NT, int M>
__device__ __forceinline__ void resolve_entries(const DistillArgs& a, const Slopes<M>& f, const Entries& en, float wt,
                                                float wl, int lo, bool far, float base) {
  sum_many<NT>(en, a.top);
  const int label = en.at[a.top].col;
  for (int e = threadIdx.x; e <= a.top; e += NT) {
    const Entry own = en.at[e];
    const int c = own.col;
    if (c < 0) continue;
    float p = 0.0f;
    if (e < a.top) {
      const Slot s = en.slot[own.next];
      if (s.first != e) continue;
      p = column_sum(en, own.next, s, own.t);
    } else if (en.flags[1]) {
      continue;
    }
    const float g = f.of(far ? own.z - base : own.z) - (wt * p + (c == label ? wl : 0.0f));
    en.at[e].z = __uint_as_float(bits_of(g, T()));
    en.at[e].next = atomicExch(&en.head[(c - lo) / Vec<T>::N % NT], e);
  }
}

// Entry k of the token `row` into LDS, from its loaded id and logit; the teacher's logit for the
// maximum.
template <typename T>
__device__ __forceinline__ float keep_entry(const DistillArgs& a, const Entries& en, const T* zr, int k, long long id,
                                            float t) {
  const int c = column_of(a, id);
  if (id < 0 || id >= a.total) t = -INFINITY;
  en.at[k].col = c;
  en.at[k].t = t;
  en.at[k].z = c >= 0 ? Elem<T>::to_f(zr[c]) : 0.0f;
  return t != t ? INFINITY : t;  // NaN: no probabilities
}

// The token's label as entry `top`.
template <typename T>
__device__ __forceinline__ void keep_label(const DistillArgs& a, const Entries& en, const T* zr, long long label) {
  if (threadIdx.x == 0) {
    const int c = column_of(a, label);
    en.at[a.top].col = c;
    en.at[a.top].z = c >= 0 ? Elem<T>::to_f(zr[c]) : 0.0f;
  }
}

// The sums of a token over its workgroup, once its maxima are known: st and s1 are the thread's
// (relative to base), the rest comes from the entries, which keep p = exp((t - max) / T) and, for
// the gradient, go into the table.
template <int NT, int M, bool GRAD>
__device__ __forceinline__ Stats token_stats(const DistillArgs& a, const Entries& en, float m, float base, float tmax,
                                             float st, float s1, bool labelled, float* red, float* inv_teacher,
                                             bool* idle) {
  const float tm = base_of(tmax);
  const float zl = en.at[a.top].z;  // (its place is used again behind the next barrier)
  // S_T, S_1, teacher's sum, mass here, sum p (z - m), sum p t
  float s[6] = {st, s1, 0.0f, 0.0f, 0.0f, 0.0f};
  for (int k = threadIdx.x; k < a.top; k += NT) {
    const float d = en.at[k].t - tm, p = exp2_fast(d * a.rate_t);
    en.at[k].t = p;
    if (p == 0.0f) {
      en.at[k].col = -1;
      continue;
    }
    s[2] += p;
    if (en.at[k].col >= 0) {
      s[3] += p;
      s[4] += p * (en.at[k].z - base);
      s[5] += p * d;
    }
  }
  if (GRAD) {  // (in a loop of its own: both at once need registers that the row has)
    const int label = en.at[a.top].col;
    for (int k = threadIdx.x; k < a.top; k += NT) {
      const int c = en.at[k].col;
      if (c < 0) continue;
      into_table(en, k, c, label);
    }
  }
  reduce_behind_barrier<AddOp, NT>(s, red);
  Stats r;
  r.m = m;
  r.st = a.want_t ? s[0] : 0.0f;
  r.s1 = a.want_1 ? (M != ONE ? s[1] : s[0]) : 0.0f;
  r.tm = tm;
  r.ts = s[2];
  const float inv = s[2] != 0.0f ? 1.0f / s[2] : 0.0f;
  r.mass = s[3] * inv;
  r.label = labelled && en.at[a.top].col >= 0 ? 1.0f : 0.0f;
  r.lin = 0.0f;
  if (s[2] != 0.0f) r.lin = a.alpha * a.tau * (inv * s[4] - inv * s[5] + a.tau * r.mass * logf(s[2]));
  if (r.label != 0.0f) r.lin += (1.0f - a.alpha) * (zl - base);
  *inv_teacher = inv;
  *idle = s[2] == 0.0f && !labelled;  // nothing to learn here
  return r;
}

// One workgroup a token: statistics, loss and, with GRAD, the gradient (a second look at the
// row).
template <typename T, int NT, int M, bool GRAD>
__global__ void __launch_bounds__(NT) distill_kernel(DistillArgs a, const T* z, float* __restrict__ stats,
                                                     float* __restrict__ loss, const float* __restrict__ dloss, T* dz) {
  extern __shared__ __align__(16) char smem[];
  __shared__ float red[2][NT / 64 * 6];
  __shared__ int flags[2];
  const Entries en = entries_in(smem, flags, a.top, GRAD ? a.slots : 0);
  if (GRAD) clear_table<NT>(en);
  const size_t row = blockIdx.x;
  const T* zr = z + row * a.ld;

  float mx[2] = {-INFINITY, -INFINITY};  // of the student's logits, of the teacher's
  for (int k = threadIdx.x; k < a.top; k += NT) {
    const size_t i = row * a.top + k;
    mx[1] = fmaxf(mx[1], keep_entry(a, en, zr, k, id_at(a.ids, a.id64, i), teacher_at(a, i)));
  }
  const long long label = a.labels ? id_at(a.labels, a.label64, row) : -1;
  const bool labelled = label >= 0 && label < a.total;
  keep_label(a, en, zr, label);

  // Maximum and sums of the logits in one pass: a thread's sums are relative to the maximum of what
  // it has seen (kept within 2^16: see Exponent), of a batch of U loads at a time.  A batch is
  // summed by itself, and so are kRun of them, so that a row of 2^28 columns (2^19 a thread) has no
  // chain of more than about 800 additions and rescalings in fp32.
  constexpr int N = Vec<T>::N, U = 4, kRun = 128;
  Part all{-INFINITY, 0.0f, 0.0f}, p = all;
  int run = 0;
  for (int c0 = (int)threadIdx.x * N; c0 < a.vocab; c0 += NT * N * U) {
    u32x4_t raw[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int c = c0 + NT * N * u;
      if (c < a.vocab) raw[u] = *reinterpret_cast<const u32x4_t*>(zr + c);
      else raw[u] = u32x4_t{Vec<T>::NONE, Vec<T>::NONE, Vec<T>::NONE, Vec<T>::NONE};
    }
    float m = p.m;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int c = c0 + NT * N * u;
      if (c < a.vocab && c + N > a.vocab) raw[u] = first_values<T>(raw[u], a.vocab - c, -INFINITY);
      float v[N];
      Vec<T>::get(raw[u], v);
#pragma unroll
      for (int e = 0; e < N; ++e) m = fmaxf(m, v[e]);
    }
    const Exponents<M> exps(a, near_base(m));
    if (m > p.m && p.m != -INFINITY) {  // (a sum of nothing stays 0, wherever the base goes)
      const Exponents<M> old(a, near_base(p.m));
      p.st *= exp2_fast(old.t.c - exps.t.c);
      if (M != ONE) p.s1 *= exp2_fast(old.one.c - exps.one.c);
    }
    float bt = 0.0f, b1 = 0.0f;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float v[N];
      Vec<T>::get(raw[u], v);
#pragma unroll
      for (int e = 0; e < N; ++e) {
        float et, e1;
        exps.of(v[e], &et, &e1);
        bt += et;
        if (M != ONE) b1 += e1;
      }
    }
    p = Part{m, p.st + bt, p.s1 + b1};
    if (++run == kRun) {
      join_part<M>(a, all, p);
      p = Part{-INFINITY, 0.0f, 0.0f};
      run = 0;
    }
  }
  join_part<M>(a, all, p);
  const float own = mx[0] = all.m;
  reduce_behind_barrier<MaxOp, NT>(mx, red[0]);
  const float base = base_of(mx[0]);
  const bool far = is_far(base);
  float st = all.st, s1 = all.s1;
  if (far) {
    far_sums<T, NT, M>(a, zr, base, &st, &s1);
  } else if (own != -INFINITY) {
    st *= exp2_fast(fmaf(-base, a.rate_t, Exponent(near_base(own), a.rate_t).c));
    if (M != ONE) s1 *= exp2_fast(fmaf(-base, a.rate_1, Exponent(near_base(own), a.rate_1).c));
  }
  float inv;
  bool idle;
  const Stats r = token_stats<NT, M, GRAD>(a, en, mx[0], base, mx[1], st, s1, labelled, red[1], &inv, &idle);
  if (threadIdx.x == 0) {
    if (stats) store_stats(stats + row * kDistillStats, r);
    if (loss) loss[row] = idle ? 0.0f : loss_of(r, a.alpha, a.tau);
  }
  if constexpr (GRAD) {
    T* dr = dz + row * a.ld;
    const float w = dloss[row];
    if (idle || w == 0.0f) {
      write_zeros<T, NT>(a, dr, 0, a.ld);
      return;
    }
    const Slopes<M> f(a, r, w, far);
    resolve_entries<T, NT, M>(a, f, en, w * a.alpha * a.tau * inv, w * (1.0f - a.alpha), 0, far, base);
    __syncthreads();
    if (far) write_slopes<T, NT, M, true>(a, f, en, zr, dr, 0, a.ld, base);
    else write_slopes<T, NT, M, false>(a, f, en, zr, dr, 0, a.ld, base);
  }
}

__device__ __forceinline__ __amdgpu_buffer_rsrc_t row_buffer(const void* p, uint32_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), (short)0, (int)bytes, 0x00020000);
}

constexpr int kPast = 2;  // a buffer access past the caches

// The 16 bytes at `off` of part `i` (of `part` bytes) of a row of `bytes`; behind them nothing is
// written.  The part moves the buffer's start and does not become the store's SGPR offset: the
// compiler takes a store with an SGPR offset to have read its data when the next instruction
// writes those registers, and of such stores, one multiply behind each, some had their first 4
// bytes replaced by that product.
__device__ __forceinline__ void store_at(bool past, u32x4_t v, void* row, uint32_t bytes, uint32_t off, int i, uint32_t part) {
  const uint32_t start = i * part;
  const __amdgpu_buffer_rsrc_t to = row_buffer((char*)row + start, bytes > start ? bytes - start : 0);
  if (past) __builtin_amdgcn_raw_buffer_store_b128(v, to, off, 0, kPast);
  else __builtin_amdgcn_raw_buffer_store_b128(v, to, off, 0, 0);
  __builtin_amdgcn_sched_barrier(0);  // chunk by chunk: several at a time cost more registers than they gain
}

// Makes the compiler forget what it has derived of r, so that it unpacks the values again instead
// of keeping them unpacked (twice the registers, for bf16) from one look at the row to the next.
__device__ __forceinline__ void forget(u32x4_t& r) { asm volatile("" : "+v"(r)); }

// Loss and gradient of a token whose row stays in the registers of its workgroup, CH chunks of 16
// bytes a thread: the logits are read once.
template <typename T, int NT, int CH, int M>
__global__ void __launch_bounds__(NT) distill_row_kernel(DistillArgs a, const T* z, float* __restrict__ loss,
                                                         const float* __restrict__ dloss, T* dz) {
  extern __shared__ __align__(16) char smem[];
  __shared__ float red[2][NT / 64 * 6];
  constexpr int N = Vec<T>::N;
  __shared__ int flags[2];
  const Entries en = entries_in(smem, flags, a.top, a.slots);
  clear_table<NT>(en);
  const size_t row = blockIdx.x;
  const T* zr = z + row * a.ld;
  T* dr = dz + row * a.ld;
  // the first entries come ahead of the row
  const int k0 = threadIdx.x;
  long long id0 = -1;
  float t0 = 0.0f;
  if (k0 < a.top) {
    id0 = id_at(a.ids, a.id64, row * a.top + k0);
    t0 = teacher_at(a, row * a.top + k0);
  }
  const long long label = a.labels ? id_at(a.labels, a.label64, row) : -1;
  const bool labelled = label >= 0 && label < a.total;
  const float w = dloss[row];
  // Chunks behind the vocabulary read as zeros and are not written (the buffers end there).
  const uint32_t bytes = (uint32_t)(((unsigned)a.vocab + N - 1) / N * 16), off = threadIdx.x * 16;
  const __amdgpu_buffer_rsrc_t zb = row_buffer(zr, bytes);
  u32x4_t raw[CH];
#pragma unroll
  for (int i = 0; i < CH; ++i) raw[i] = __builtin_amdgcn_raw_buffer_load_b128(zb, off, i * NT * 16, kPast);
  float mx[2] = {-INFINITY, -INFINITY};
  if (k0 < a.top) mx[1] = keep_entry(a, en, zr, k0, id0, t0);
  for (int k = k0 + NT; k < a.top; k += NT) {
    const size_t i = row * a.top + k;
    mx[1] = fmaxf(mx[1], keep_entry(a, en, zr, k, id_at(a.ids, a.id64, i), teacher_at(a, i)));
  }
  keep_label(a, en, zr, label);
#pragma unroll
  for (int i = 0; i < CH; ++i) {
    if ((i + 1) * NT * N > a.vocab) {  // the same for the whole workgroup
      const int c = ((int)threadIdx.x + NT * i) * N;
      if (c + N > a.vocab) raw[i] = first_values<T>(raw[i], a.vocab - c, -INFINITY);
    }
    float v[N];
    Vec<T>::get(raw[i], v);
#pragma unroll
    for (int e = 0; e < N; ++e) mx[0] = fmaxf(mx[0], v[e]);
  }
  reduce_behind_barrier<MaxOp, NT>(mx, red[0]);
  const float base = base_of(mx[0]);
  const bool far = is_far(base);
#pragma unroll
  for (int i = 0; i < CH; ++i) forget(raw[i]);
  float st = 0.0f, s1 = 0.0f;
  if (far) {
    far_sums<T, NT, M>(a, zr, base, &st, &s1);
  } else {
    const Exponents<M> exps(a, base);
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      float v[N];
      Vec<T>::get(raw[i], v);
#pragma unroll
      for (int e = 0; e < N; ++e) {
        float et, e1;
        exps.of(v[e], &et, &e1);
        st += et;
        if (M != ONE) s1 += e1;
      }
    }
    st *= exps.t.off();
    s1 *= exps.one.off();
  }
  float inv;
  bool idle;
  const Stats r = token_stats<NT, M, true>(a, en, mx[0], base, mx[1], st, s1, labelled, red[1], &inv, &idle);
  if (threadIdx.x == 0) loss[row] = idle ? 0.0f : loss_of(r, a.alpha, a.tau);
  if (idle || w == 0.0f) {  // whatever the logits are
    write_zeros<T, NT>(a, dr, 0, a.ld);
    return;
  }
#pragma unroll
  for (int i = 0; i < CH; ++i) forget(raw[i]);
  const Slopes<M> f(a, r, w, far);
  resolve_entries<T, NT, M>(a, f, en, w * a.alpha * a.tau * inv, w * (1.0f - a.alpha), 0, far, base);
  __syncthreads();
  if (far) {
    write_slopes<T, NT, M, true>(a, f, en, zr, dr, 0, a.ld, base);
  } else {
    const uint32_t mine = chunks_with_entries<T, NT>(en, 0);
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      u32x4_t v = slopes_of<T, M>(f, raw[i], N);
      if (mine >> i & 1) v = with_entries<T>(en, v, ((int)threadIdx.x + NT * i) * N);
      store_at(a.past, v, dr, bytes, off, i, NT * 16);
    }
    write_padding<T, NT>(a, dr, 0);
    write_zeros<T, NT>(a, dr, (a.vocab + N - 1) / N * N, a.ld);
  }
}

// The gradient from a token's (joined) statistics: a workgroup U times NT * 16 bytes of a row,
// loaded before anything else.
template <typename T, int NT, int U, int M>
__global__ void __launch_bounds__(NT) distill_bwd_kernel(DistillArgs a, int pieces, const T* z,
                                                         const float* __restrict__ stats,
                                                         const float* __restrict__ dloss, T* dz) {
  extern __shared__ __align__(16) char smem[];
  constexpr int N = Vec<T>::N, piece = NT * N * U;
  __shared__ int flags[2];
  const Entries en = entries_in(smem, flags, a.top, a.slots);
  const size_t row = blockIdx.x / pieces;
  const int lo = (int)(blockIdx.x % pieces) * piece, hi = min(lo + piece, a.ld);
  const T* zr = z + row * a.ld;
  T* dr = dz + row * a.ld;
  const Stats s = load_stats(stats + row * kDistillStats);
  const float w = dloss[row];
  if ((s.mass == 0.0f && s.label == 0.0f) || w == 0.0f) {
    write_zeros<T, NT>(a, dr, lo, hi);
    return;
  }
  const int end = (a.vocab + N - 1) / N * N;  // behind it there are zeros
  const uint32_t bytes = (uint32_t)max(min(hi, end) - lo, 0) * sizeof(T), off = threadIdx.x * 16;
  const __amdgpu_buffer_rsrc_t zb = row_buffer(zr + lo, bytes);
  u32x4_t raw[U];
#pragma unroll
  for (int u = 0; u < U; ++u) raw[u] = __builtin_amdgcn_raw_buffer_load_b128(zb, off, u * NT * 16, kPast);
  const int label = a.labels ? column_of(a, id_at(a.labels, a.label64, row)) : -1;
  clear_table<NT>(en);
  __syncthreads();
  for (int k = threadIdx.x; k <= a.top; k += NT) {
    int c = -1;
    float p = 0.0f;
    if (k < a.top) {
      const size_t i = row * a.top + k;
      c = column_of(a, id_at(a.ids, a.id64, i));
      p = exp2_fast((teacher_at(a, i) - s.tm) * a.rate_t);
      if (p == 0.0f) c = -1;
    } else {
      c = label;
    }
    if (c < lo || c >= hi) c = -1;
    en.at[k].col = c;
    if (c < 0) continue;
    en.at[k].t = p;
    en.at[k].z = Elem<T>::to_f(zr[c]);
    if (k == a.top) continue;
    into_table(en, k, c, label);
  }
  __syncthreads();  // the entries' logits are read, too: dz may be z
  const bool far = is_far(s.m);
  const Slopes<M> f(a, s, w, far);
  resolve_entries<T, NT, M>(a, f, en, s.ts != 0.0f ? w * a.alpha * a.tau / s.ts : 0.0f, w * (1.0f - a.alpha), lo, far,
                            s.m);
  __syncthreads();
  if (far) {
    write_slopes<T, NT, M, true>(a, f, en, zr, dr, lo, hi, s.m);
  } else {
    const uint32_t mine = chunks_with_entries<T, NT>(en, lo);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      u32x4_t v = slopes_of<T, M>(f, raw[u], N);
      if (mine >> u & 1) v = with_entries<T>(en, v, lo + ((int)threadIdx.x + NT * u) * N);
      store_at(a.past, v, dr + lo, bytes, off, u, NT * 16);
    }
    if (lo <= a.vocab && a.vocab < hi) write_padding<T, NT>(a, dr, lo);
    write_zeros<T, NT>(a, dr, max(lo, end), hi);
  }
}

// Ranks' statistics [ranks][tokens] to the whole vocabulary's, in the ranks' order, summed kJoinRun at
// a time.
constexpr int kJoinRun = 256;
__global__ void __launch_bounds__(256) distill_join_kernel(int tokens, int ranks, float alpha, float tau, float rate_t,
                                                           const float* __restrict__ parts, float* __restrict__ stats,
                                                           float* __restrict__ loss) {
  const long long t = (long long)blockIdx.x * 256 + threadIdx.x;
  if (t >= tokens) return;
  float m = -INFINITY;
  for (int r = 0; r < ranks; ++r) m = fmaxf(m, parts[((size_t)r * tokens + t) * kDistillStats]);
  const float base = base_of(m);
  Stats s{m, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
  for (int r = 0; r < ranks;) {
    float s1 = 0.0f, st = 0.0f, lin = 0.0f, mass = 0.0f, label = 0.0f;
    for (int n = 0; n < kJoinRun && r < ranks; ++n, ++r) {
      const Stats p = load_stats(parts + ((size_t)r * tokens + t) * kDistillStats);
      const float d = moved(p.m, base);
      s1 += p.s1 * exp2_fast(d * kLog2e);
      st += p.st * exp2_fast(d * rate_t);
      lin += p.lin;
      if (p.mass != 0.0f) lin += alpha * tau * p.mass * d;
      if (p.label != 0.0f) lin += (1.0f - alpha) * p.label * d;
      mass += p.mass;
      label += p.label;
      s.tm = p.tm;
      s.ts = p.ts;
    }
    s.s1 += s1;
    s.st += st;
    s.lin += lin;
    s.mass += mass;
    s.label += label;
  }
  store_stats(stats + t * kDistillStats, s);
  loss[t] = loss_of(s, alpha, tau);
}

// ---------------------------------------------------------------------------
// Host launchers
// ---------------------------------------------------------------------------
static DistillArgs distill_args(const DistillShape& q) {
  DistillArgs a{};
  a.vocab = q.vocab, a.ld = q.ld;
  a.first = q.first, a.total = q.total;
  a.alpha = q.alpha, a.tau = q.tau;
  a.want_t = q.top > 0 && q.alpha > 0.0f;
  a.want_1 = q.labels && q.alpha < 1.0f;
  a.top = a.want_t ? q.top : 0;
  a.slots = entry_slots(a.top);
  a.rate_1 = kLog2e;
  a.rate_t = a.want_t ? kLog2e / q.tau : kLog2e;
  a.id64 = q.id_type == ID_I64, a.label64 = q.label_type == ID_I64, a.teacher_bf16 = q.teacher_type == DT_BF16;
  a.ids = q.ids, a.teacher = q.teacher, a.labels = a.want_1 ? q.labels : nullptr;
  return a;
}

// Moves a launch's arguments to the tokens [t, t + n).
static DistillArgs at_tokens(const DistillShape& q, DistillArgs a, long long t, int n) {
  a.tokens = n;
  if (a.top) {
    a.ids = (const char*)a.ids + (size_t)t * a.top * (a.id64 ? 8 : 4);
    a.teacher = (const char*)a.teacher + (size_t)t * a.top * (a.teacher_bf16 ? 2 : 4);
  }
  if (a.labels) a.labels = (const char*)a.labels + (size_t)t * (a.label64 ? 8 : 4);
  return a;
}

// Which exponentials a loss needs (Sums).
static int sums_of(const DistillShape& q) {
  const DistillArgs a = distill_args(q);
  if (!a.want_t || !a.want_1 || q.tau == 1.0f) return ONE;
  return q.tau == 2.0f ? SQUARE : q.tau == 4.0f ? FOURTH : TWO;
}

struct DistillCall {
  const DistillShape& q;
  const void* z;
  float *stats, *loss;        // forward
  const float *in, *dloss;    // gradient
  void* dz;
  hipStream_t s;
};

// Launches `run(arguments, first token)` over the call's tokens, as many at a time as a launch of
// `groups` workgroups of `threads` for each of them can have.
template <typename F>
static hipError_t over_tokens(const DistillShape& q, int threads, int groups, size_t out_bytes, F run) {
  DistillArgs all = distill_args(q);
  all.past = out_bytes >= kStreamBytes;
  const long long most = max_groups(threads) / groups;
  for (long long t = 0; t < q.tokens; t += most) {
    run(at_tokens(q, all, t, (int)std::min(most, q.tokens - t)), t);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

template <typename T>
static size_t out_bytes(const DistillShape& q) { return (size_t)q.tokens * q.ld * sizeof(T); }

template <typename T, int NT, int M, bool GRAD>
static hipError_t run_rows(const DistillCall& c) {
  const DistillShape& q = c.q;
  return over_tokens(q, NT, 1, GRAD ? out_bytes<T>(q) : 0, [&](const DistillArgs& a, long long t) {
    hipLaunchKernelGGL((distill_kernel<T, NT, M, GRAD>), dim3(a.tokens), dim3(NT), entries_bytes(a.top, NT, GRAD), c.s, a,
                       (const T*)c.z + t * q.ld, c.stats ? c.stats + t * kDistillStats : nullptr,
                       c.loss ? c.loss + t : nullptr, GRAD ? c.dloss + t : nullptr, GRAD ? (T*)c.dz + t * q.ld : nullptr);
  });
}

template <typename T, int NT, int CH, int M>
static hipError_t run_kept(const DistillCall& c) {
  const DistillShape& q = c.q;
  return over_tokens(q, NT, 1, out_bytes<T>(q), [&](const DistillArgs& a, long long t) {
    hipLaunchKernelGGL((distill_row_kernel<T, NT, CH, M>), dim3(a.tokens), dim3(NT), entries_bytes(a.top, NT, true), c.s, a,
                       (const T*)c.z + t * q.ld, c.loss + t, c.dloss + t, (T*)c.dz + t * q.ld);
  });
}

// Threads for a row of n chunks of 16 bytes.  A short row has few threads, so that as many bytes
// are on their way in a CU as its registers hold: 32768 x 6288 (n = 786) loss 90 us with 128
// threads (108 with 256), loss and gradient 178 with 128 (202 with 256; in fp32, where a row has half
// the columns, 191 and 168).  Few rows have more: what counts then is how long one takes (32 x 6288
// 7.7 us with 512, 8.9 with 128; 200 x 25152 11.4 with 512, 13.5 with 256; 700 x 25152 22.6 and
// 23.4).  So have rows with many entries, whose table leaves room for fewer workgroups in a CU from 204
// and from 409 entries on.  Loss and gradient of 8192 x 3496: with 203 entries 67 us on 128
// threads and on 256, with 204 66 and 57; on 256 and 512 with 408 entries 83 and 101, with 409
// 75 and 73, with 1024 228 and 157.  (On 64 threads, which these rows have up to 203 entries, 64
// entries take 39 us, 47 on 128; 128 take 54 and 50, 203 78 and 67.)  The loss alone, of 8192 x
// 1000: 256 entries 14.6 us on 64 threads and 18.3 on 128, 512 28.9 and 24.6, 768 36 on 128 and 32 on
// 256; of 8192 x 6288 512 entries 58 on 128 and 41 on 256; of 8192 x 12568 1000 entries 98 on 256 and 77
// on 512.
static bool many_entries(int top) { return entry_slots(top) >= 512; }       // 204 and more
static bool most_entries(int top) { return entry_slots(top) >= 1024; }      // 409 and more

static int loss_threads(int n, int top) {
  if (n <= 256) return top <= 256 ? 64 : top <= 512 ? 128 : 256;
  const int few = n <= 1024 ? 128 : n <= 2048 ? 256 : 512;
  return few < 512 && top > 2 * few ? 2 * few : few;
}

template <typename T, int M>
static hipError_t run_forward(const DistillCall& c) {
  const int n = (c.q.vocab + Vec<T>::N - 1) / Vec<T>::N, top = distill_args(c.q).top;
  if (!c.dz) {
    switch (loss_threads(n, top)) {
      case 64: return run_rows<T, 64, M, false>(c);
      case 128: return run_rows<T, 128, M, false>(c);
      case 256: return run_rows<T, 256, M, false>(c);
      default: return run_rows<T, 512, M, false>(c);
    }
  }
  if ((c.q.tokens <= 1024 && n > 256) || most_entries(top)) {
    if (n <= 1024) return run_kept<T, 512, 2, M>(c);
    if (n <= 3584) return run_kept<T, 512, 7, M>(c);
  }
  if (many_entries(top) && n <= 1024) return run_kept<T, 256, 4, M>(c);
  if (n <= 128) return run_kept<T, 64, 2, M>(c);
  if (n <= 256) return run_kept<T, 64, 4, M>(c);
  if (n <= 512) return run_kept<T, 64, 8, M>(c);
  if (n <= 896) return run_kept<T, 128, 7, M>(c);
  if (n <= 1792) return run_kept<T, 256, 7, M>(c);  // 4096 x 12568, 64 entries 52 us (57 with 128 x 13)
  if (n <= 3328) return run_kept<T, 256, 13, M>(c);
  if (n <= 6656) return run_kept<T, 512, 13, M>(c);
  if (n <= 9728) return run_kept<T, 512, 19, M>(c);
  if (n <= 12800) return run_kept<T, 512, 25, M>(c);
  if (n <= 16384) return run_kept<T, 512, 32, M>(c);
  return run_rows<T, 512, M, true>(c);  // more than the registers hold: a second look at the row
}

template <typename T, int NT, int U, int M>
static hipError_t run_pieces(const DistillCall& c) {
  constexpr int piece = NT * Vec<T>::N * U;
  const DistillShape& q = c.q;
  const int pieces = (q.ld + piece - 1) / piece;
  return over_tokens(q, NT, pieces, out_bytes<T>(q), [&](const DistillArgs& a, long long t) {
    hipLaunchKernelGGL((distill_bwd_kernel<T, NT, U, M>), dim3((unsigned)(a.tokens * pieces)), dim3(NT),
                       entries_bytes(a.top, NT, true), c.s, a, pieces, (const T*)c.z + t * q.ld, c.in + t * kDistillStats,
                       c.dloss + t, (T*)c.dz + t * q.ld);
  });
}

// Threads and pieces of a row of n chunks.  Many entries: as above (4096 x 6288 with 256 entries
// 46 us on 128 threads and 35 on 256, with 203 43 and 41; 8192 x 1000 with 1000 199 on 256 and 140 on
// 512; 2048 x 25152 with 512 71 on 256 and 59 on 512).  One piece a row up to 3328 chunks; longer ones are
// cut small (8192 x 50304 276 us with U = 4, 304 with 13), and so are few rows (300 x 12800 9.5 and
// 11.5, but 300 x 50304 18.0 and 16.7), but for a number of rows that fills the card once in large
// pieces (600 x 50304 28.9 and 25.6).
template <typename T, int M>
static hipError_t run_backward(const DistillCall& c) {
  const int n = c.q.ld / Vec<T>::N, tokens = c.q.tokens, top = distill_args(c.q).top;
  if (n <= 1024 && many_entries(top))
    return entry_slots(top) >= 2048 ? run_pieces<T, 512, 2, M>(c) : run_pieces<T, 256, 4, M>(c);
  if (most_entries(top)) return run_pieces<T, 512, 7, M>(c);
  if (n <= 128) return run_pieces<T, 64, 2, M>(c);
  if (n <= 896) return run_pieces<T, 128, 7, M>(c);
  if (tokens < 512 || (n > 3328 && tokens >= 1024)) return run_pieces<T, 256, 4, M>(c);
  return n <= 1792 ? run_pieces<T, 256, 7, M>(c) : run_pieces<T, 256, 13, M>(c);
}

template <typename T, int M>
static hipError_t run_mode(const DistillCall& c) {
  return c.in ? run_backward<T, M>(c) : run_forward<T, M>(c);
}

template <typename T>
static hipError_t run_type(const DistillCall& c) {
  switch (sums_of(c.q)) {
    case ONE: return run_mode<T, ONE>(c);
    case SQUARE: return run_mode<T, SQUARE>(c);
    case FOURTH: return run_mode<T, FOURTH>(c);
    default: return run_mode<T, TWO>(c);
  }
}

hipError_t launch_distill(int dtype, const DistillShape& q, const void* z, float* stats, float* loss,
                          const float* dloss, void* dz, hipStream_t s) {
  const DistillCall c{q, z, stats, loss, nullptr, dloss, dz, s};
  return dtype == DT_BF16 ? run_type<bf16_t>(c) : run_type<float>(c);
}

hipError_t launch_distill_bwd(int dtype, const DistillShape& q, const void* z, const float* stats, const float* dloss,
                              void* dz, hipStream_t s) {
  const DistillCall c{q, z, nullptr, nullptr, stats, dloss, dz, s};
  return dtype == DT_BF16 ? run_type<bf16_t>(c) : run_type<float>(c);
}

hipError_t launch_distill_join(int tokens, int ranks, float alpha, float tau, const float* parts, float* stats,
                               float* loss, hipStream_t s) {
  hipLaunchKernelGGL(distill_join_kernel, dim3((unsigned)(((long long)tokens + 255) / 256)), dim3(256), 0, s, tokens,
                     ranks, alpha, tau, kLog2e / tau, parts, stats, loss);
  return hipGetLastError();
}

}  // namespace merak
