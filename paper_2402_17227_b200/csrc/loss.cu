// Log probabilities of given tokens with entropy and top alternatives, and their gradient (vcas_loss_fwd, vcas_loss_bwd).
//
// Forward: one pass over the logits.  A thread keeps the largest value it has seen, m, with S = sum exp(x - m) and
// T = sum exp(x - m) (x - m), all in fp32; two such triples join by rescaling the one with the smaller m.  Then
//   lse = m + log S,   logp = (x_t - m) - log S,   entropy = log S - T / S.
// Differences to the maximum are taken before anything else, so that logits of any size lose nothing.
// Top alternatives: what a thread kept, its maximum and the vector that holds it, gives a bound: with 64 (32) groups of threads, the
// k-th largest of the groups' maxima is not above the k-th largest logit.  Only the threads whose maximum reaches the bound (about
// k) look at their values again, in L2, and pass on the few that reach it; those are ranked by counting.  Values compare with
// their index (larger first, then lower index), so that ties, a row of equal values among them, are as cheap as others.
//
// Long rows come near HBM's rate: 2 bytes a logit in bf16 and one exponential each, of which the SMs have 4.5e12 a second and the copy rate needs
// 3.3e12.  2048 rows of 131072 in bf16, five alternatives: DRAM 66 % in use, special function unit 62 %, issue slots 63 %.  A row's end
// (joins, alternatives) costs more where rows are short: 16384 of 4096 take 42 us without alternatives and 71 with five, for 20 at the copy rate.
#include <new>

#include "common.cuh"
#include "vcas_train.h"

namespace vcas {
namespace {

constexpr int MAX_TOP = 32;
constexpr int MAX_SLICES = 32;           // CTAs that share a row: a lane each when they are joined
constexpr int MAX_UNITS = 2048;          // (row, slice) pairs of a call whose rows are shared
// values at or above the bound that a CTA of NT threads ranks; the keys of all slices of a row fit as well
template <int NT> constexpr int CANDIDATES = NT < 64 ? 512 : MAX_SLICES * MAX_TOP;

struct Loss {
  vcas_loss_desc desc;
  int device, num_sms;
  void* base;
  float4* part;        // [MAX_UNITS] m, S, T of a slice (backward: the slice's sum of squares in x)
  uint64_t* keys;      // [MAX_UNITS][top] a slice's largest values with their indices
  int32_t* tickets;    // [MAX_UNITS] slices of a row that are done
  int32_t* status;
};

constexpr float LOWEST = -3.402823466e+38f;
constexpr float FAR = -1e30f;            // exp of it is 0, and 0 times it too
// What lower logits, -inf among them, count as: the difference to any fp32 maximum stays finite, exp of it is 0, and 0 times it too.
constexpr float FLOOR = -0x1.92p+99f;   // about -1e30, 0xf149 in bf16
constexpr float LOG2E = 1.4426950408889634f;

__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// the larger of the two, NaN if one is
__device__ __forceinline__ float max_nan(float a, float b) {
  float y;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
  return y;
}

template <typename T> struct Vec;
template <> struct Vec<__nv_bfloat16> {
  static constexpr int N = 8;
  static __device__ __forceinline__ void unpack(uint4 v, float (&f)[8]) {
    const uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { f[2 * i] = __uint_as_float(u[i] << 16); f[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u); }
  }
  // the largest value, NaN aside
  static __device__ __forceinline__ float top(uint4 v) {
    uint32_t a, b;
    asm("max.bf16x2 %0, %1, %2;" : "=r"(a) : "r"(v.x), "r"(v.y));
    asm("max.bf16x2 %0, %1, %2;" : "=r"(b) : "r"(v.z), "r"(v.w));
    asm("max.bf16x2 %0, %1, %2;" : "=r"(a) : "r"(a), "r"(b));
    return fmaxf(__uint_as_float(a << 16), __uint_as_float(a & 0xffff0000u));
  }
  // -inf and all below FLOOR become FLOOR, NaN stays
  static __device__ __forceinline__ uint4 raise(uint4 v) {
    constexpr uint32_t FLOOR2 = 0xf149f149u;         // FLOOR in bf16, twice
    uint4 o;
    asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(o.x) : "r"(v.x), "r"(FLOOR2));
    asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(o.y) : "r"(v.y), "r"(FLOOR2));
    asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(o.z) : "r"(v.z), "r"(FLOOR2));
    asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(o.w) : "r"(v.w), "r"(FLOOR2));
    return o;
  }
  static __device__ __forceinline__ uint4 pack(float (&f)[8]) {       // f becomes what is stored
    uint32_t o[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 t = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
      o[i] = *reinterpret_cast<const uint32_t*>(&t);
      f[2 * i] = __uint_as_float(o[i] << 16);
      f[2 * i + 1] = __uint_as_float(o[i] & 0xffff0000u);
    }
    return make_uint4(o[0], o[1], o[2], o[3]);
  }
  static __device__ __forceinline__ float one(__nv_bfloat16 x) { return __bfloat162float(x); }
  static __device__ __forceinline__ float put(float x, __nv_bfloat16* p) {
    const __nv_bfloat16 b = __float2bfloat16_rn(x);
    *p = b;
    return __bfloat162float(b);
  }
};
template <> struct Vec<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ void unpack(uint4 v, float (&f)[4]) {
    f[0] = __uint_as_float(v.x); f[1] = __uint_as_float(v.y); f[2] = __uint_as_float(v.z); f[3] = __uint_as_float(v.w);
  }
  static __device__ __forceinline__ float top(uint4 v) {
    return fmaxf(fmaxf(__uint_as_float(v.x), __uint_as_float(v.y)), fmaxf(__uint_as_float(v.z), __uint_as_float(v.w)));
  }
  static __device__ __forceinline__ uint4 raise(uint4 v) {
    return make_uint4(one_up(v.x), one_up(v.y), one_up(v.z), one_up(v.w));
  }
  static __device__ __forceinline__ uint32_t one_up(uint32_t v) {
    return __float_as_uint(max_nan(__uint_as_float(v), FLOOR));
  }
  static __device__ __forceinline__ uint4 pack(float (&f)[4]) {
    return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
  }
  static __device__ __forceinline__ float one(float x) { return x; }
  static __device__ __forceinline__ float put(float x, float* p) { *p = x; return x; }
};

struct Sums { float m, s, t; };
__device__ __forceinline__ void rescale(Sums& a, float m) {       // m >= a.m
  const float d = max_nan(a.m - m, FAR);
  const float c = exp2_fast(d * LOG2E);
  a.t = c * fmaf(a.s, d, a.t);
  a.s *= c;
  a.m = m;
}
__device__ __forceinline__ uint32_t ordered(float x) {
  const uint32_t b = __float_as_uint(x);
  return (b & 0x80000000u) ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float unordered(uint32_t o) { return __uint_as_float((o & 0x80000000u) ? o & 0x7fffffffu : ~o); }
__device__ __forceinline__ float warp_top(float m) { return unordered(__reduce_max_sync(0xffffffffu, ordered(m))); }
// Of all lanes, in every lane: all are made relative to the largest maximum, then added in a fixed order.  (Joined two by two, each
// time with both rescaled, 16384 rows of 32000 took 253 us, now 211.)
__device__ __forceinline__ Sums join_lanes(Sums a) {
  rescale(a, warp_top(a.m));
  a.s = warp_sum(a.s);
  a.t = warp_sum(a.t);
  return a;
}

// A value and its index as one number: larger values first, then lower indices.  -0 counts as 0.
__device__ __forceinline__ uint64_t key_of(float x, uint32_t idx) {
  return ((uint64_t)ordered(x + 0.0f) << 32) | (uint32_t)~idx;
}
__device__ __forceinline__ float key_value(uint64_t k) {
  return unordered((uint32_t)(k >> 32));
}
__device__ __forceinline__ int key_index(uint64_t k) { return (int)~(uint32_t)k; }

struct FwdParams {
  const void* x; int64_t ld; const void* tokens; int token_bytes;
  float *logp, *entropy, *lse, *top_logp; int32_t* top_ids;
  int rows, V, top, slices, per;         // per: values of a slice, a multiple of the vector length
  float4* part; uint64_t* keys; int32_t* tickets; int32_t* status;
};

__device__ __forceinline__ int64_t token_of(const void* tokens, int bytes, int64_t r) {
  return bytes == 8 ? ((const int64_t*)tokens)[r] : ((const int32_t*)tokens)[r];
}

// The NT threads that share a row or a slice of it: a CTA, or one of its eight warps.
template <int NT>
struct Team {
  static constexpr int PER_CTA = NT == 32 ? 8 : 1;
  static __device__ __forceinline__ int tid() { return NT == 32 ? threadIdx.x & 31 : threadIdx.x; }
  static __device__ __forceinline__ int place() { return NT == 32 ? threadIdx.x >> 5 : 0; }
  static __device__ __forceinline__ void sync() {
    if (NT == 32) __syncwarp(); else __syncthreads();
  }
};

// The values [c0, c1) of a row as a thread sees them: single values up to the first 16-byte boundary (thread 0 has them), whole
// vectors dealt out to the threads in turn, single values behind them (thread 0 again).
template <typename T, int NT>
struct Slice {
  static constexpr int BATCH = 4;          // vectors a thread has on their way at once
  const T* row;
  int c0, head, nv, c1;
  __device__ Slice(const T* row_, int c0_, int c1_) : row(row_), c0(c0_), c1(c1_) {
    const int off = (int)(((uintptr_t)(row + c0) & 15) / sizeof(T));
    head = min(c1 - c0, off == 0 ? 0 : Vec<T>::N - off);
    nv = (c1 - c0 - head) / Vec<T>::N;
  }
  __device__ const uint4* vectors() const { return reinterpret_cast<const uint4*>(row + c0 + head); }
  __device__ int at(int v) const { return c0 + head + v * Vec<T>::N; }       // index of a vector's first value
  // f(vector, its number) for every vector of this thread
  template <typename F>
  __device__ __forceinline__ void each_vector(F f) const {
    const uint4* xv = vectors();
    int v = Team<NT>::tid();
    for (; v + (BATCH - 1) * NT < nv; v += BATCH * NT) {
      uint4 raw[BATCH];
#pragma unroll
      for (int q = 0; q < BATCH; ++q) raw[q] = __ldg(xv + v + q * NT);
#pragma unroll
      for (int q = 0; q < BATCH; ++q) f(raw[q], v + q * NT);
    }
    uint4 raw[BATCH - 1];
#pragma unroll
    for (int q = 0; q < BATCH - 1; ++q)
      if (v + q * NT < nv) raw[q] = __ldg(xv + v + q * NT);
#pragma unroll
    for (int q = 0; q < BATCH - 1; ++q)
      if (v + q * NT < nv) f(raw[q], v + q * NT);
  }
  // f(value, index) for the values of a vector, and for the single ones
  template <typename F>
  __device__ __forceinline__ void each_of(uint4 raw, int v, F f) const {
    float x[Vec<T>::N];
    Vec<T>::unpack(raw, x);
#pragma unroll
    for (int e = 0; e < Vec<T>::N; ++e) f(x[e], at(v) + e);
  }
  template <typename F>
  __device__ __forceinline__ void each_single(F f) const {
    for (int i = c0; i < c0 + head; ++i) f(Vec<T>::one(row[i]), i);
    for (int i = at(nv); i < c1; ++i) f(Vec<T>::one(row[i]), i);
  }
};

// The k largest of n keys in shared memory, by counting how many are larger; the others' places stay as they are.
template <int NT, typename F>
__device__ __forceinline__ void rank_keys(const uint64_t* keys, int n, int k, F f) {
  for (int i = Team<NT>::tid(); i < n; i += NT) {
    const uint64_t mine = keys[i];
    int larger = 0;
#pragma unroll 8
    for (int j = 0; j < n; ++j) larger += keys[j] > mine;
    if (larger < k && mine != 0) f(larger, mine);
  }
}

template <int NT, bool TOP>
struct FwdShared {
  float m[NT / 32];
  float2 sums[NT / 32];
  int last;
};
template <int NT>
struct FwdShared<NT, true> {
  float m[NT / 32];
  float2 sums[NT / 32];
  int last, count, holders;
  uint64_t group[NT < 64 ? NT : 64];
  uint64_t bound, best, taken;
  uint64_t cand[CANDIDATES<NT>];
  uint64_t out[MAX_TOP];
  int holder[NT];
};

// big: the thread's largest value, big_at: the index of the first of the vector that holds it (or its own; -1: no values)
template <typename T, int NT>
__device__ __forceinline__ void top_of_slice(const Slice<T, NT>& s, float big, int big_at, FwdShared<NT, true>& sh, int k) {
  constexpr int GROUPS = NT < 64 ? NT : 64, PER = NT / GROUPS, VN = Vec<T>::N;
  using Te = Team<NT>;
  const int tid = Te::tid();
  // the group's largest, at the last place its value can have; 0: a group without values
  uint64_t g = big_at < 0 ? 0 : key_of(big, (uint32_t)min(big_at + VN - 1, s.c1 - 1));
#pragma unroll
  for (int o = 1; o < PER; o <<= 1) { const uint64_t v = __shfl_xor_sync(0xffffffffu, g, o); g = v > g ? v : g; }
  if (tid % PER == 0) sh.group[tid / PER] = g;
  if (tid == 0) { sh.bound = 0; sh.count = 0; sh.holders = 0; }
  if (tid < MAX_TOP) sh.out[tid] = 0;
  Te::sync();
  rank_keys<NT>(sh.group, GROUPS, k, [&](int rank, uint64_t key) { if (rank == k - 1) sh.bound = key; });
  Te::sync();
  const uint64_t bound = sh.bound;
  auto keep = [&](float x, int i) {
    const uint64_t key = key_of(x, (uint32_t)i);
    if (key >= bound) {
      const int at = atomicAdd(&sh.count, 1);
      if (at < CANDIDATES<NT>) sh.cand[at] = key;
    }
  };
  if (big_at >= 0 && key_of(big, (uint32_t)big_at) >= bound) {
    sh.holder[atomicAdd(&sh.holders, 1)] = tid;
    if (tid == 0) s.each_single(keep);
  }
  Te::sync();
  // the holders' vectors, by all threads (each holder its own, one after the other, took 25 us a row of 131072)
  const int holders = sh.holders, rounds = (s.nv + NT - 1) / NT;
  const uint4* xv = s.vectors();
  for (int i = tid; i < holders * rounds; i += NT) {
    const int v = sh.holder[i % holders] + i / holders * NT;
    if (v < s.nv) s.each_of(__ldg(xv + v), v, keep);
  }
  Te::sync();
  const int n = sh.count;
  if (n <= CANDIDATES<NT>) {
    rank_keys<NT>(sh.cand, n, k, [&](int rank, uint64_t key) { sh.out[rank] = key; });
    Te::sync();
    return;
  }
  // a few threads hold most of the large values: one alternative a pass over the slice
  if (tid == 0) sh.taken = ~0ull;
  for (int j = 0; j < k; ++j) {
    if (tid == 0) sh.best = 0;
    Te::sync();
    uint64_t b = 0;
    const uint64_t below = sh.taken;
    auto look = [&](float x, int i) {
      const uint64_t key = key_of(x, (uint32_t)i);
      if (key < below && key > b) b = key;
    };
    s.each_vector([&](uint4 raw, int v) { s.each_of(raw, v, look); });
    if (tid == 0) s.each_single(look);
    atomicMax((unsigned long long*)&sh.best, (unsigned long long)b);
    Te::sync();
    if (tid == 0) { sh.out[j] = sh.best; sh.taken = sh.best; }
    Te::sync();
  }
}

// Of the whole team: m in every thread, s and t in those of its first warp.
template <int NT, typename Sh>
__device__ __forceinline__ Sums join_team(Sums a, Sh& sh) {
  if (NT == 32) return join_lanes(a);
  const int tid = Team<NT>::tid(), warp = tid >> 5;
  float m = warp_top(a.m);
  Team<NT>::sync();                      // those of before have been read
  if ((tid & 31) == 0) sh.m[warp] = m;
  Team<NT>::sync();
#pragma unroll
  for (int w = 0; w < NT / 32; ++w) m = fmaxf(m, sh.m[w]);
  rescale(a, m);
  a.s = warp_sum(a.s);
  a.t = warp_sum(a.t);
  if ((tid & 31) == 0) sh.sums[warp] = make_float2(a.s, a.t);
  Team<NT>::sync();
  if (warp == 0) {
    a.s = a.t = 0.f;
#pragma unroll
    for (int w = 0; w < NT / 32; ++w) { a.s += sh.sums[w].x; a.t += sh.sums[w].y; }
  }
  return a;
}

// A row without a value above FLOOR (the type's lowest value as a mask, or -inf, throughout): relative to what it has, in a pass of
// its own.
template <typename T, int NT, typename Sh>
__device__ __noinline__ Sums sums_of_low_row(Slice<T, NT> s, Sh& sh) {
  Sums a = {LOWEST, 0.f, 0.f};
  auto add = [&](float x, int) {
    if (x > a.m) rescale(a, x);
    const float d = max_nan(x - a.m, FAR), e = exp2_fast(d * LOG2E);
    a.s += e;
    a.t = fmaf(e, d, a.t);
  };
  s.each_vector([&](uint4 raw, int v) { s.each_of(raw, v, add); });
  if (Team<NT>::tid() == 0) s.each_single(add);
  return join_team<NT>(a, sh);
}

template <typename T, int NT, bool TOP>
__global__ void __launch_bounds__(NT * Team<NT>::PER_CTA) loss_fwd_kernel(FwdParams P) {
  constexpr int VN = Vec<T>::N;
  using Te = Team<NT>;
  __shared__ FwdShared<NT, TOP> shared[Te::PER_CTA];
  FwdShared<NT, TOP>& sh = shared[Te::place()];
  const int tid = Te::tid();
  const int64_t unit = (int64_t)blockIdx.x * Te::PER_CTA + Te::place(), r = unit / P.slices;
  if (r >= P.rows) return;               // a whole warp, where a CTA has several rows
  const int slice = (int)(unit - r * P.slices);
  const T* row = (const T*)P.x + r * P.ld;
  const int c0 = slice * P.per, c1 = min(P.V, c0 + P.per);
  const Slice<T, NT> s(row, c0, c1);

  Sums a = {FLOOR, 0.f, 0.f};
  float big = 0.f;                       // the largest value and the index of its vector (or its own, outside the vectors)
  int big_at = -1;
  auto single = [&](float x, int i) {
    if (big_at < 0 || x > big) { big = x; big_at = i; }
    if (x > a.m) rescale(a, x);
    const float d = max_nan(x, FLOOR) - a.m, e = exp2_fast(d * LOG2E);
    a.s += e;
    a.t = fmaf(e, d, a.t);
  };
  if (tid == 0)
    for (int i = c0; i < c0 + s.head; ++i) single(Vec<T>::one(row[i]), i);
  uint64_t s2 = 0, t2 = 0;               // two sums each, of even and odd places
  auto vector = [&](uint4 raw, int v) {
    float x[VN];
    const float top = Vec<T>::top(raw);
    if (big_at < 0 || top > big) {
      big = top;
      big_at = s.at(v);
      if (top > a.m) {
        float p, q;
        unpack2(s2, p, q);
        a.s += p + q;
        unpack2(t2, p, q);
        a.t += p + q;
        s2 = t2 = 0;
        rescale(a, top);
      }
    }
    Vec<T>::unpack(Vec<T>::raise(raw), x);
    const uint64_t nm = pack2(-a.m, -a.m), log2e = pack2(LOG2E, LOG2E);
#pragma unroll
    for (int e = 0; e < VN; e += 2) {
      float y0, y1;
      const uint64_t d = add2(pack2(x[e], x[e + 1]), nm);
      unpack2(mul2(d, log2e), y0, y1);
      const uint64_t w = pack2(exp2_fast(y0), exp2_fast(y1));
      s2 = add2(s2, w);
      t2 = fma2(w, d, t2);
    }
  };
  s.each_vector(vector);
  {
    float p, q;
    unpack2(s2, p, q);
    a.s += p + q;
    unpack2(t2, p, q);
    a.t += p + q;
  }
  if (tid == 0)
    for (int i = s.at(s.nv); i < c1; ++i) single(Vec<T>::one(row[i]), i);

  a = join_team<NT>(a, sh);
  if constexpr (TOP) top_of_slice<T, NT>(s, big, big_at, sh, P.top);

  if (P.slices > 1) {
    // the row's last CTA joins the slices, in their order
    const int first = (int)r * P.slices;
    if constexpr (TOP) {
      if (tid < P.top) P.keys[(size_t)unit * P.top + tid] = sh.out[tid];
    }
    if (tid == 0) P.part[unit] = make_float4(a.m, a.s, a.t, 0.f);
    Te::sync();
    if (tid == 0) {
      __threadfence();                   // for all of the CTA, which the barrier put before it
      const int done = atomicAdd(P.tickets + r, 1);
      sh.last = done == P.slices - 1;
      if (sh.last) P.tickets[r] = 0;     // for the next call
    }
    Te::sync();
    if (!sh.last) return;
    __threadfence();
    // lane i has slice i, neighbours join first
    const int lane = tid & 31;
    a = {FLOOR, 0.f, 0.f};
    if (lane < P.slices) {
      const float4 f = __ldcg(P.part + first + lane);
      a = {f.x, f.y, f.z};
    }
    a = join_lanes(a);
    if constexpr (TOP) {
      // each slice's keys are in descending order: one warp merges them, a lane holding the first of its slice that is not taken
      const int n = P.slices * P.top;
      for (int i = tid; i < n; i += NT) sh.cand[i] = __ldcg(P.keys + (size_t)first * P.top + i);
      if (tid < MAX_TOP) sh.out[tid] = 0;
      Te::sync();
      if (tid < 32) {
        int next = 1;
        uint64_t mine = lane < P.slices ? sh.cand[lane * P.top] : 0;
        for (int j = 0; j < P.top; ++j) {
          const uint32_t hi = __reduce_max_sync(0xffffffffu, (uint32_t)(mine >> 32));
          const uint32_t lo = __reduce_max_sync(0xffffffffu, (uint32_t)(mine >> 32) == hi ? (uint32_t)mine : 0);
          const uint64_t best = ((uint64_t)hi << 32) | lo;
          if (mine == best && best != 0) {
            sh.out[j] = mine;
            mine = next < P.top ? sh.cand[lane * P.top + next] : 0;
            ++next;
          }
        }
      }
      Te::sync();
    }
  }
  if (a.m == FLOOR) a = sums_of_low_row<T, NT>(Slice<T, NT>(row, 0, P.V), sh);
  if (tid >= 32) return;
  const bool none = a.s == 0.f;          // -inf throughout
  const float log_s = logf(a.s);
  if (tid == 0) {
    if (P.lse != nullptr) P.lse[r] = none ? __int_as_float(0xff800000) : a.m + log_s;
    if (P.entropy != nullptr) P.entropy[r] = none ? 0.f : log_s - a.t / a.s;
    if (P.logp != nullptr) {
      int64_t t = P.tokens != nullptr ? token_of(P.tokens, P.token_bytes, r) : -1;
      if (t >= P.V) { t = -1; atomicExch(P.status, (int32_t)VCAS_ERR_BAD_ARG); }
      float lp = 0.f;
      if (t >= 0) lp = none ? __int_as_float(0xff800000) : (Vec<T>::one(row[t]) - a.m) - log_s;
      P.logp[r] = lp;
    }
  }
  if constexpr (TOP) {
    if (tid >= P.top) return;
    const uint64_t key = sh.out[tid];
    const float x = key_value(key);
    const float bad = __int_as_float(0x7fc00000);
    if (P.top_ids != nullptr) P.top_ids[r * P.top + tid] = key == 0 ? -1 : key_index(key);
    if (P.top_logp != nullptr)
      P.top_logp[r * P.top + tid] = key == 0 ? bad : none ? __int_as_float(0xff800000) : (x - a.m) - log_s;
  }
}

struct BwdParams {
  const void* x; int64_t ld; const void* tokens; int token_bytes;
  const float *lse, *entropy, *g_logp, *g_entropy;
  void* dx; int64_t ld_d; float* a_out;
  int V, slices, per;
  float4* part; int32_t* tickets; int32_t* status;
};

// x - lse is good to 2^-25 |lse|, and p to as much relative to itself: 2^-15 here, where bf16's own rounding is 2^-9.  Rows farther from 0
// have their log probabilities from the logits again (with lse, a row throughout at the type's lowest value would have p = 1).
constexpr float LSE_FAR = 1024.0f;

// Such a row, by a whole CTA: the largest logit, log sum exp(x - it), then the gradient.  All of it is read before any is written, for the
// two may be the same.  Returns this thread's sum of squares.
template <typename T, int NT>
__device__ __noinline__ float far_row(const T* row, T* out, int V, int64_t t, float gl, float nge, float base, float* s_sum) {
  auto joined = [&](float x, auto join) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x = join(x, __shfl_xor_sync(0xffffffffu, x, o));
    __syncthreads();                     // what was there before has been read
    if ((threadIdx.x & 31) == 0) s_sum[threadIdx.x / 32] = x;
    __syncthreads();
    x = s_sum[0];
#pragma unroll
    for (int w = 1; w < NT / 32; ++w) x = join(x, s_sum[w]);
    return x;
  };
  float m = __int_as_float(0xff800000), s = 0.f, sq = 0.f;
  for (int i = threadIdx.x; i < V; i += NT) m = fmaxf(m, Vec<T>::one(row[i]));
  m = joined(m, [](float a, float b) { return fmaxf(a, b); });
  for (int i = threadIdx.x; i < V; i += NT) s += exp2_fast(max_nan(Vec<T>::one(row[i]) - m, FAR) * LOG2E);
  const float log_s = logf(joined(s, [](float a, float b) { return a + b; }));
  for (int i = threadIdx.x; i < V; i += NT) {
    const float lp = max_nan((Vec<T>::one(row[i]) - m) - log_s, FAR);
    float d = exp2_fast(lp * LOG2E) * fmaf(nge, lp, base);
    if (i == t) d += gl;
    d = Vec<T>::put(d, out + i);
    sq = fmaf(d, d, sq);
  }
  __syncthreads();                       // s_sum is free again
  return sq;
}

// dx_j = g_logp (1[j = t] - p_j) - g_entropy p_j (log p_j + entropy): one read and one write of HBM.  The row's square-norm is
// summed over the stored values on the way.
template <typename T, int NT>
__global__ void __launch_bounds__(NT) loss_bwd_kernel(BwdParams P) {
  constexpr int VN = Vec<T>::N;
  __shared__ float s_sum[NT / 32];
  __shared__ int s_last;
  const int64_t r = blockIdx.x / P.slices;
  const int slice = blockIdx.x - (int)r * P.slices;
  const T* row = (const T*)P.x + r * P.ld;
  T* out = (T*)P.dx + r * P.ld_d;
  int c0 = slice * P.per, c1 = min(P.V, c0 + P.per);
  int64_t t = token_of(P.tokens, P.token_bytes, r);
  if (t >= P.V) {
    t = -1;
    if (threadIdx.x == 0) atomicExch(P.status, (int32_t)VCAS_ERR_BAD_ARG);
  }
  const float lse = P.lse[r];
  const float gl = t >= 0 ? P.g_logp[r] : 0.f, ge = P.g_entropy != nullptr ? P.g_entropy[r] : 0.f;
  const float H = P.g_entropy != nullptr ? P.entropy[r] : 0.f;
  const bool zero = (gl == 0.f && ge == 0.f) || lse == __int_as_float(0xff800000);
  const float base = -fmaf(ge, H, gl);                   // dx = p (base - ge log p), + gl at the token
  const float nge = -ge;
  auto value = [&](float x) {
    const float lp = max_nan(x - lse, FAR);
    return exp2_fast(lp * LOG2E) * fmaf(nge, lp, base);
  };
  float sq = 0.f;
  if (fabsf(lse) >= LSE_FAR && !zero) {
    // by the row's first CTA; the others have nothing to do with it
    if (slice == 0) sq = far_row<T, NT>(row, out, P.V, t, gl, nge, base, s_sum);
    c0 = c1 = 0;
  }
  auto single = [&](int i) {
    float d = zero ? 0.f : value(Vec<T>::one(row[i]));
    if (i == t && !zero) d += gl;
    d = Vec<T>::put(d, out + i);
    sq = fmaf(d, d, sq);
  };
  const int off = (int)(((uintptr_t)(out + c0) & 15) / sizeof(T));
  const int head = min(c1 - c0, off == 0 ? 0 : VN - off);
  const bool same = (((uintptr_t)(row + c0) ^ (uintptr_t)(out + c0)) & 15) == 0 || zero;
  if (!same) {
    for (int i = c0 + threadIdx.x; i < c1; i += NT) single(i);
  } else {
    const int nv = (c1 - c0 - head) / VN, b = c0 + head;
    for (int i = c0 + threadIdx.x; i < b; i += NT) single(i);
    for (int i = b + nv * VN + threadIdx.x; i < c1; i += NT) single(i);
    const uint4* xv = reinterpret_cast<const uint4*>(row + b);
    uint4* dv = reinterpret_cast<uint4*>(out + b);
    const int tv = t >= b ? (int)((t - b) / VN) : -1, te = t >= b ? (int)((t - b) % VN) : 0;
    if (zero) {
      for (int v = threadIdx.x; v < nv; v += NT) dv[v] = make_uint4(0, 0, 0, 0);
    } else {
      auto vector = [&](uint4 raw, int v) {
        float x[VN];
        Vec<T>::unpack(raw, x);
#pragma unroll
        for (int e = 0; e < VN; ++e) x[e] = value(x[e]);
        if (v == tv) {
#pragma unroll
          for (int e = 0; e < VN; ++e)
            if (e == te) x[e] += gl;
        }
        dv[v] = Vec<T>::pack(x);
#pragma unroll
        for (int e = 0; e < VN; ++e) sq = fmaf(x[e], x[e], sq);
      };
      int v = threadIdx.x;
      for (; v + 3 * NT < nv; v += 4 * NT) {
        uint4 raw[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) raw[q] = xv[v + q * NT];
#pragma unroll
        for (int q = 0; q < 4; ++q) vector(raw[q], v + q * NT);
      }
      for (; v < nv; v += NT) vector(xv[v], v);
    }
  }
  if (P.a_out == nullptr) return;
  sq = warp_sum(sq);
  if ((threadIdx.x & 31) == 0) s_sum[threadIdx.x / 32] = sq;
  __syncthreads();
  if (threadIdx.x == 0) {
    float all = 0.f;
#pragma unroll
    for (int w = 0; w < NT / 32; ++w) all += s_sum[w];
    if (P.slices == 1) {
      P.a_out[r] = all;
    } else {
      P.part[blockIdx.x].x = all;
      __threadfence();
      s_last = atomicAdd(P.tickets + r, 1) == P.slices - 1;
      if (s_last) {
        __threadfence();
        P.tickets[r] = 0;
        float sum = 0.f;
        for (int i = 0; i < P.slices; ++i) sum += __ldcg(&P.part[r * P.slices + i].x);
        P.a_out[r] = sum;
      }
    }
  }
}

// Threads a row: enough for four vectors each.  Slices: while there are fewer rows than CTAs the SMs hold, rows are shared, down to
// 2048 values a slice.
struct Shape { int threads, slices, per; };
Shape shape_of(const Loss* l, int rows, int vn) {
  const int V = l->desc.vocab, nv = (V + vn - 1) / vn;
  Shape s;
  int slices = 1;
  const int want = 4 * l->num_sms;
  if (rows < want) {
    slices = want / rows;
    if (slices > (V + 2047) / 2048) slices = (V + 2047) / 2048;
    if (slices > MAX_SLICES) slices = MAX_SLICES;
    if (slices > MAX_UNITS / rows) slices = MAX_UNITS / rows;
    if (slices < 1) slices = 1;
  }
  s.per = ((nv + slices - 1) / slices) * vn;
  s.slices = (V + s.per - 1) / s.per;
  const int each = s.per / vn;
  s.threads = each <= 128 ? 32 : each <= 512 ? 128 : 256;
  return s;
}

template <typename T, int NT>
void launch_fwd(const FwdParams& P, unsigned grid, cudaStream_t st) {
  constexpr unsigned PER = Team<NT>::PER_CTA;
  if (P.top > 0) loss_fwd_kernel<T, NT, true><<<(grid + PER - 1) / PER, NT * PER, 0, st>>>(P);
  else loss_fwd_kernel<T, NT, false><<<(grid + PER - 1) / PER, NT * PER, 0, st>>>(P);
}
template <typename T>
cudaError_t run_fwd(const Loss* l, FwdParams& P, int rows, cudaStream_t st) {
  Shape s = shape_of(l, rows, Vec<T>::N);
  if (s.slices > 1 && s.threads == 32) s.threads = 128;      // room for the keys of all slices; a CTA has one row's slice
  P.slices = s.slices; P.per = s.per; P.rows = rows;
  const unsigned grid = (unsigned)rows * s.slices;
  if (s.threads == 32) launch_fwd<T, 32>(P, grid, st);
  else if (s.threads == 128) launch_fwd<T, 128>(P, grid, st);
  else launch_fwd<T, 256>(P, grid, st);
  return cudaGetLastError();
}
template <typename T>
cudaError_t run_bwd(const Loss* l, BwdParams& P, int rows, cudaStream_t st) {
  const Shape s = shape_of(l, rows, Vec<T>::N);
  P.slices = s.slices; P.per = s.per;
  const unsigned grid = (unsigned)rows * s.slices;
  if (s.threads == 32) loss_bwd_kernel<T, 32><<<grid, 32, 0, st>>>(P);
  else if (s.threads == 128) loss_bwd_kernel<T, 128><<<grid, 128, 0, st>>>(P);
  else loss_bwd_kernel<T, 256><<<grid, 256, 0, st>>>(P);
  return cudaGetLastError();
}

inline Loss* L(vcas_loss l) { return reinterpret_cast<Loss*>(l); }
size_t elem(int dtype) { return dtype == VCAS_DTYPE_BF16 ? 2 : 4; }
bool off_grid(const void* p, size_t to) { return ((uintptr_t)p & (to - 1)) != 0; }

}  // namespace
}  // namespace vcas

using namespace vcas;

extern "C" int vcas_loss_create(vcas_loss* out, const vcas_loss_desc* desc) {
  if (out == nullptr || desc == nullptr) return VCAS_ERR_BAD_ARG;
  *out = nullptr;
  if (desc->dtype != VCAS_DTYPE_F32 && desc->dtype != VCAS_DTYPE_BF16) return VCAS_ERR_DTYPE;
  if (desc->max_rows <= 0 || desc->max_rows > (1 << 30) || desc->vocab <= 0 || desc->vocab > (1 << 30)) return VCAS_ERR_SHAPE;
  if (desc->top < 0 || desc->top > MAX_TOP || desc->top > desc->vocab) return VCAS_ERR_SHAPE;
  Loss* l = new (std::nothrow) Loss();
  if (l == nullptr) return VCAS_ERR_WORKSPACE;
  l->desc = *desc;
  const size_t part = MAX_UNITS * sizeof(float4), keys = (size_t)MAX_UNITS * MAX_TOP * 8, tick = MAX_UNITS * 4;
  const size_t bytes = part + keys + tick + 256;
  if (cudaGetDevice(&l->device) != cudaSuccess ||
      cudaDeviceGetAttribute(&l->num_sms, cudaDevAttrMultiProcessorCount, l->device) != cudaSuccess) {
    delete l;
    return VCAS_ERR_CUDA;
  }
  if (cudaMalloc(&l->base, bytes) != cudaSuccess) {
    cudaGetLastError();
    delete l;
    return VCAS_ERR_WORKSPACE;
  }
  uint8_t* b = (uint8_t*)l->base;
  l->part = (float4*)b;
  l->keys = (uint64_t*)(b + part);
  l->tickets = (int32_t*)(b + part + keys);
  l->status = (int32_t*)(b + part + keys + tick);
  if (cudaMemset(l->base, 0, bytes) != cudaSuccess || cudaDeviceSynchronize() != cudaSuccess) {
    cudaFree(l->base);
    delete l;
    return VCAS_ERR_CUDA;
  }
  *out = reinterpret_cast<vcas_loss>(l);
  return VCAS_OK;
}

extern "C" int vcas_loss_destroy(vcas_loss ll) {
  if (ll == nullptr) return VCAS_ERR_BAD_ARG;
  Loss* l = L(ll);
  DeviceScope on(l->device);
  const cudaError_t e = cudaFree(l->base);
  delete l;
  return e == cudaSuccess ? VCAS_OK : VCAS_ERR_CUDA;
}

extern "C" int vcas_loss_fwd(vcas_loss ll, const void* logits, int64_t ld, const void* tokens, int32_t token_bytes, int32_t rows,
                             float* logp, float* entropy, float* lse, float* top_logp, int32_t* top_ids, vcas_stream stream) {
  if (ll == nullptr) return VCAS_ERR_BAD_ARG;
  Loss* l = L(ll);
  const vcas_loss_desc& d = l->desc;
  if (rows < 0 || rows > d.max_rows || ld < d.vocab) return VCAS_ERR_SHAPE;
  if (token_bytes != 4 && token_bytes != 8) return VCAS_ERR_DTYPE;
  if (rows == 0) return VCAS_OK;
  if (logits == nullptr || (logp != nullptr && tokens == nullptr)) return VCAS_ERR_BAD_ARG;
  if (d.top == 0 && (top_logp != nullptr || top_ids != nullptr)) return VCAS_ERR_BAD_ARG;
  if (off_grid(logits, elem(d.dtype)) || off_grid(tokens, token_bytes)) return VCAS_ERR_BAD_ARG;
  DeviceScope on(l->device);
  if (!on.ok) return VCAS_ERR_CUDA;
  FwdParams P = {};
  P.x = logits; P.ld = ld; P.tokens = tokens; P.token_bytes = token_bytes;
  P.logp = logp; P.entropy = entropy; P.lse = lse; P.top_logp = top_logp; P.top_ids = top_ids;
  P.V = d.vocab; P.top = top_logp != nullptr || top_ids != nullptr ? d.top : 0;
  P.part = l->part; P.keys = l->keys; P.tickets = l->tickets; P.status = l->status;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  const cudaError_t e = d.dtype == VCAS_DTYPE_BF16 ? run_fwd<__nv_bfloat16>(l, P, rows, st) : run_fwd<float>(l, P, rows, st);
  return e == cudaSuccess ? VCAS_OK : VCAS_ERR_CUDA;
}

extern "C" int vcas_loss_bwd(vcas_loss ll, const void* logits, int64_t ld, const void* tokens, int32_t token_bytes, int32_t rows,
                             const float* lse, const float* entropy, const float* g_logp, const float* g_entropy, void* dlogits,
                             int64_t ld_d, float* a_out, vcas_stream stream) {
  if (ll == nullptr) return VCAS_ERR_BAD_ARG;
  Loss* l = L(ll);
  const vcas_loss_desc& d = l->desc;
  if (rows < 0 || rows > d.max_rows || ld < d.vocab || ld_d < d.vocab) return VCAS_ERR_SHAPE;
  if (token_bytes != 4 && token_bytes != 8) return VCAS_ERR_DTYPE;
  if (rows == 0) return VCAS_OK;
  if (logits == nullptr || tokens == nullptr || lse == nullptr || g_logp == nullptr || dlogits == nullptr ||
      (g_entropy != nullptr && entropy == nullptr))
    return VCAS_ERR_BAD_ARG;
  if (dlogits == logits && ld != ld_d) return VCAS_ERR_BAD_ARG;
  if (off_grid(logits, elem(d.dtype)) || off_grid(dlogits, elem(d.dtype)) || off_grid(tokens, token_bytes)) return VCAS_ERR_BAD_ARG;
  DeviceScope on(l->device);
  if (!on.ok) return VCAS_ERR_CUDA;
  BwdParams P = {};
  P.x = logits; P.ld = ld; P.tokens = tokens; P.token_bytes = token_bytes;
  P.lse = lse; P.entropy = entropy; P.g_logp = g_logp; P.g_entropy = g_entropy;
  P.dx = dlogits; P.ld_d = ld_d; P.a_out = a_out; P.V = d.vocab;
  P.part = l->part; P.tickets = l->tickets; P.status = l->status;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  const cudaError_t e = d.dtype == VCAS_DTYPE_BF16 ? run_bwd<__nv_bfloat16>(l, P, rows, st) : run_bwd<float>(l, P, rows, st);
  return e == cudaSuccess ? VCAS_OK : VCAS_ERR_CUDA;
}

extern "C" int vcas_loss_status(vcas_loss ll, int32_t* status) {
  if (ll == nullptr || status == nullptr) return VCAS_ERR_BAD_ARG;
  Loss* l = L(ll);
  DeviceScope on(l->device);
  if (!on.ok || cudaDeviceSynchronize() != cudaSuccess ||
      cudaMemcpy(status, l->status, sizeof(int32_t), cudaMemcpyDeviceToHost) != cudaSuccess ||
      cudaMemset(l->status, 0, sizeof(int32_t)) != cudaSuccess)
    return VCAS_ERR_CUDA;
  return VCAS_OK;
}
