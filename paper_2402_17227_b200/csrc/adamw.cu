// AdamW over many tensors in one launch (vcas_adamw_step).
//
// HBM-bound: a thread takes eight consecutive elements, every array is read and written once with the widest access there is (32
// bytes of fp32, 16 of bf16, 8 of e4m3), and the whole table of tensors travels in the kernel's parameters, so that a step
// neither copies a table to the device nor keeps one there.  A warp's 256 elements are the block of an 8-bit state's scale: its
// largest value is one warp reduction, on the bits as integers, which carry a NaN along.
// The states' multiplications and additions are rounded one by one (no contraction to fma), with 32-bit states all of the update's: it is
// then the same to the bit wherever it is computed from the formulas.
#include <cmath>

#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include "common.cuh"
#include "vcas_train.h"

namespace vcas {
namespace {

// 8-bit states need arithmetic between their loads and stores, and smaller CTAs mix these better (314 M elements: 512 threads 914 us, 256
// 880, 128 862; several chunks by one CTA, which saves finding the tensor, 916 and more).
template <int BITS> constexpr int THREADS = BITS == 8 ? 128 : 256;
template <int BITS> constexpr int CHUNK = THREADS<BITS> * 8;       // elements a CTA works on

struct Entry {
  void* p; const void* g; void* m; void* v; float* m_scale; float* v_scale; void* copy;
  int64_t n;
  float keep, decay;                     // 1 - lr wd, wd
  uint32_t first;                        // first chunk of this tensor in the launch
  uint32_t place;                        // in the caller's list, and in the top bit whether all pointers are aligned
};
// Kernel parameters hold 32 KB; most lists are short, and a small table is launched faster.
constexpr int SMALL = 48, LARGE = 384;
template <int CAP>
struct Table {
  Entry e[CAP];
  int count;
  float b1, c1, b2, c2, eps, step_size, inv;
  uint32_t seed_lo, seed_hi;
  const float* grad_scale; const float* rates; const uint64_t* seed_dev;
};
static_assert(sizeof(Table<LARGE>) <= 32764, "kernel parameters");

// ---- eight consecutive elements
__device__ __forceinline__ void ld8(const float* p, float (&f)[8]) {
  asm volatile("ld.global.v8.f32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
               : "=f"(f[0]), "=f"(f[1]), "=f"(f[2]), "=f"(f[3]), "=f"(f[4]), "=f"(f[5]), "=f"(f[6]), "=f"(f[7]) : "l"(p) : "memory");
}
__device__ __forceinline__ void st8(float* p, const float (&f)[8]) {
  asm volatile("st.global.v8.f32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};"
               ::"l"(p), "f"(f[0]), "f"(f[1]), "f"(f[2]), "f"(f[3]), "f"(f[4]), "f"(f[5]), "f"(f[6]), "f"(f[7]) : "memory");
}
__device__ __forceinline__ void ld8(const __nv_bfloat16* p, float (&f)[8]) {
  const uint4 v = *reinterpret_cast<const uint4*>(p);
  const uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) { f[2 * i] = __uint_as_float(u[i] << 16); f[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u); }
}
__device__ __forceinline__ void st8(__nv_bfloat16* p, const float (&f)[8]) {
  uint32_t u[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __nv_bfloat162 t = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
    u[i] = *reinterpret_cast<const uint32_t*>(&t);
  }
  *reinterpret_cast<uint4*>(p) = make_uint4(u[0], u[1], u[2], u[3]);
}
__device__ __forceinline__ float widen(float x) { return x; }
__device__ __forceinline__ float widen(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ void narrow(float x, float* p) { *p = x; }
__device__ __forceinline__ void narrow(float x, __nv_bfloat16* p) { *p = __float2bfloat16_rn(x); }

// the group's first `have` elements; the others count as zeros
template <typename T>
__device__ __forceinline__ void load(const T* p, int have, bool wide, float (&f)[8]) {
  if (wide) { ld8(p, f); return; }
#pragma unroll
  for (int i = 0; i < 8; ++i) f[i] = i < have ? widen(p[i]) : 0.f;
}
template <typename T>
__device__ __forceinline__ void store(T* p, int have, bool wide, const float (&f)[8]) {
  if (wide) { st8(p, f); return; }
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (i < have) narrow(f[i], p + i);
}
__device__ __forceinline__ uint2 load_codes(const uint8_t* p, int have, bool wide) {
  if (wide) return *reinterpret_cast<const uint2*>(p);
  uint32_t w[2] = {0, 0};
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (i < have) w[i / 4] |= (uint32_t)p[i] << (8 * (i % 4));
  return make_uint2(w[0], w[1]);
}
__device__ __forceinline__ void store_codes(uint8_t* p, int have, bool wide, uint2 c) {
  if (wide) { *reinterpret_cast<uint2*>(p) = c; return; }
  const uint32_t w[2] = {c.x, c.y};
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (i < have) p[i] = (uint8_t)(w[i / 4] >> (8 * (i % 4)));
}

// ---- pairs of elements
struct Eight { uint64_t p[4]; };
__device__ __forceinline__ Eight pairs(const float (&f)[8]) {
  Eight e;
#pragma unroll
  for (int i = 0; i < 4; ++i) e.p[i] = pack2(f[2 * i], f[2 * i + 1]);
  return e;
}
__device__ __forceinline__ void singles(const Eight& e, float (&f)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) unpack2(e.p[i], f[2 * i], f[2 * i + 1]);
}
__device__ __forceinline__ Eight scaled(const Eight& a, float by) {
  const uint64_t b = pack2(by, by);
  Eight e;
#pragma unroll
  for (int i = 0; i < 4; ++i) e.p[i] = mul2(a.p[i], b);
  return e;
}
__device__ __forceinline__ Eight square(const Eight& a) {
  Eight e;
#pragma unroll
  for (int i = 0; i < 4; ++i) e.p[i] = mul2(a.p[i], a.p[i]);
  return e;
}
// Sums of products are made one by one: mul.f32x2 in front of add.f32x2 became one fma, with a rounding less.
__device__ __forceinline__ Eight plus(const Eight& a, const Eight& b) {
  float x[8], y[8];
  singles(a, x);
  singles(b, y);
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = __fadd_rn(x[i], y[i]);
  return pairs(x);
}
__device__ __forceinline__ Eight times_plus(const Eight& a, float by, const Eight& b) {
  const uint64_t k = pack2(by, by);
  Eight e;
#pragma unroll
  for (int i = 0; i < 4; ++i) e.p[i] = fma2(a.p[i], k, b.p[i]);
  return e;
}

// ---- e4m3
__device__ __forceinline__ Eight decode(uint2 c, float scale) {
  float f[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t two = (i < 2 ? c.x : c.y) >> (16 * (i % 2));
    const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)two, __NV_E4M3);      // exact
    const float2 v = __half22float2(__half2(h));
    f[2 * i] = v.x;
    f[2 * i + 1] = v.y;
  }
  return scaled(pairs(f), scale);
}
// A value times 2^-120 has its e4m3 exponent and mantissa in bits 20-26, subnormals included; what is below them decides together with the
// random bits (in bits 12-19, and half of their step) whether the code goes up by one.  BYTE: of each element's halfword.
// POSITIVE: no signs, a positive value does not become 0, and an infinite one (a finite gradient whose square is not) is held as 2^63:
// as infinity it would take the scale, and with it the block's other states, along.  A value may come out up to 3 steps of fp32
// above 448, too few to reach the next code: what is added is at most 2^20 - 2048.
__device__ __forceinline__ uint32_t largest(uint32_t top, float a, float b) {
  float r;
  asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(__uint_as_float(top)), "f"(a), "f"(b));
  return __float_as_uint(r);
}
__device__ __forceinline__ float largest_of_block(const float (&f)[8]) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 8; i += 2) top = largest(top, f[i], f[i + 1]);
  return __uint_as_float(__reduce_max_sync(0xffffffffu, top));
}
template <bool POSITIVE, int BYTE>
__device__ __forceinline__ uint2 encode(float (&f)[8], const uint32_t (&rnd)[4], float* scale_at, int lane) {
  float big = largest_of_block(f);
  if (POSITIVE && big == __int_as_float(0x7f800000)) {       // the same in all lanes
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = f[i] == __int_as_float(0x7f800000) ? 0x1p63f : f[i];
    big = largest_of_block(f);
  }
  if (lane == 0) *scale_at = __fmul_rn(big, 1.0f / 448.0f);
  // under 2^-100 (sqrt(v) is never that small) 1 / big would leave fp32's range: such an m is held as 0
  const float inv = big >= 0x1p-100f ? __fmul_rn(__frcp_rn(big), 448.0f) : 0.f;
  uint32_t w[2] = {0, 0};
  float z[8];
  singles(scaled(scaled(pairs(f), inv), 0x1p-120f), z);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    // bytes 0, 0, random, 0x80: shifted left by 4 that is the random byte in bits 12-19 and 2048
    const uint32_t r = __byte_perm(rnd[i / 2], 0x80u, 0x5504 | ((2 * (i % 2) + BYTE) << 4));
    uint32_t c = __float_as_uint(z[i]) + (r << 4);
    if (POSITIVE) c = max(c, min(__float_as_uint(f[i]), 1u << 20));
    c <<= 4;                                         // the code in the top byte
    if (!POSITIVE) c = (c & 0x7fffffffu) | (__float_as_uint(f[i]) & 0x80000000u);
    w[i / 4] = __byte_perm(w[i / 4], c, 0x7321);     // and in behind those before it
  }
  return make_uint2(w[0], w[1]);
}

// sqrt(x), rounded correctly but for the rarest x: x / sqrt(x) and one step of Newton's iteration on its exact residual.  x under fp32's
// normal numbers counts as the least of them: the approximation would take it for 0.  The minimum with x 2^126, which is above
// the root of any other number, gives 0 its root, and infinity, of whose root the iteration makes a NaN; a NaN stays one.
__device__ __forceinline__ float root_of(float x) {
  float y, r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(x), "f"(0x1p-126f));
  asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(y));
  const float s = __fmul_rn(y, r);
  return fminf(fmaf(fmaf(-s, s, y), 0.5f * r, s), __fmul_rn(x, 0x1p126f));
}
// 1 / x, good to an ulp, of a normal x
__device__ __forceinline__ float reciprocal(float x) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}

__device__ __forceinline__ void philox(uint32_t c0, uint32_t c1, uint32_t c2, uint32_t k0, uint32_t k1, uint32_t (&out)[4]) {
  uint32_t c3 = 0;
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const uint32_t hi0 = __umulhi(0xD2511F53u, c0), lo0 = 0xD2511F53u * c0;
    const uint32_t hi1 = __umulhi(0xCD9E8D57u, c2), lo1 = 0xCD9E8D57u * c2;
    c0 = hi1 ^ c1 ^ k0; c1 = lo1; c2 = hi0 ^ c3 ^ k1; c3 = lo0;
    k0 += 0x9E3779B9u; k1 += 0xBB67AE85u;
  }
  out[0] = c0; out[1] = c1; out[2] = c2; out[3] = c3;
}

template <typename P, typename G, int BITS, int CAP>
__global__ void __launch_bounds__(THREADS<BITS>, BITS == 8 ? 12 : 4) adamw_kernel(const __grid_constant__ Table<CAP> t) {
  // the tensor this chunk belongs to: the last one that begins at or before it
  int lo = 0, hi = t.count - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (t.e[mid].first <= blockIdx.x) lo = mid; else hi = mid - 1;
  }
  const Entry& e = t.e[lo];
  const int lane = threadIdx.x & 31;
  float keep = e.keep, step_size = t.step_size, inv = t.inv, scale_g = 1.f;
  if (t.rates != nullptr) {
    keep = (float)(1.0 - (double)t.rates[0] * (double)e.decay);
    step_size = t.rates[1];
    inv = t.rates[2];
  }
  if (t.grad_scale != nullptr) scale_g = *t.grad_scale;
  uint32_t k0 = t.seed_lo, k1 = t.seed_hi;
  if (BITS == 8 && t.seed_dev != nullptr) { const uint64_t s = *t.seed_dev; k0 = (uint32_t)s; k1 = (uint32_t)(s >> 32); }
  const int64_t at = (int64_t)(blockIdx.x - e.first) * CHUNK<BITS> + threadIdx.x * 8;
  const int64_t left = e.n - at;
  const int have = left >= 8 ? 8 : left > 0 ? (int)left : 0;
  // a whole warp without elements has nothing to do; the others keep all lanes for the block's largest value
  if (__all_sync(0xffffffffu, have == 0)) return;
  const bool wide = have == 8 && (e.place >> 31);
  const int64_t block = at >> 8;
  float x[8], root[8];
  uint2 mc = make_uint2(0, 0), vc = make_uint2(0, 0);
  float ms = 0.f, vs = 0.f;
  Eight p, g, m, v;
  load((const G*)e.g + at, have, wide, x);
  g = pairs(x);
  if (BITS == 32) {
    load((const float*)e.m + at, have, wide, x);
    m = pairs(x);
    load((const float*)e.v + at, have, wide, x);
    v = pairs(x);
  } else {
    mc = load_codes((const uint8_t*)e.m + at, have, wide);
    vc = load_codes((const uint8_t*)e.v + at, have, wide);
    ms = e.m_scale[block];
    vs = e.v_scale[block];
  }
  load((const P*)e.p + at, have, wide, x);
  p = pairs(x);
  if (t.grad_scale != nullptr) g = scaled(g, scale_g);
  if (BITS == 8) {
    m = decode(mc, ms);
    v = decode(vc, vs);
    v = square(v);
  }
  m = plus(scaled(m, t.b1), scaled(g, t.c1));
  v = plus(scaled(v, t.b2), scaled(square(g), t.c2));
  singles(v, root);
  // 32-bit states: the correctly rounded root and quotient, which HBM leaves time for.  With 8-bit ones, half the bytes, it does
  // not (issue slots were 81 % in use at 62 % of its bandwidth): a root in fewer steps, and for p, on which no state depends, a quotient
  // good to two ulp and fused sums (314 M elements: 1266 us with the former, 862 so).
  if (BITS == 8) {
    float denom[8];
    const float least = t.eps > 0.f ? fmaxf(t.eps, 0x1p-126f) : t.eps;        // denom is normal, or 0 as the formula has it
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      root[i] = root_of(root[i]);
      denom[i] = least;
    }
    singles(times_plus(pairs(root), inv, pairs(denom)), denom);
#pragma unroll
    for (int i = 0; i < 8; ++i) denom[i] = reciprocal(denom[i]);
    const Eight step = scaled(m, -step_size), d = pairs(denom);
    Eight q;
#pragma unroll
    for (int i = 0; i < 4; ++i) q.p[i] = mul2(step.p[i], d.p[i]);
    singles(times_plus(p, keep, q), x);
  } else {
    float step[8], denom[8], kept[8];
    singles(scaled(m, step_size), step);
    singles(scaled(p, keep), kept);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      denom[i] = __fadd_rn(__fmul_rn(__fsqrt_rn(root[i]), inv), t.eps);
      x[i] = __fsub_rn(kept[i], __fdiv_rn(step[i], denom[i]));
    }
  }
  store((P*)e.p + at, have, wide, x);
  if (sizeof(P) == 4 && e.copy != nullptr) store((__nv_bfloat16*)e.copy + at, have, wide, x);
  singles(m, x);
  if (BITS == 32) {
    store((float*)e.m + at, have, wide, x);
    singles(v, x);
    store((float*)e.v + at, have, wide, x);
  } else {
    // elements behind the tensor's end count as zeros (0 / (0 + eps) leaves m and r at 0)
    uint32_t rnd[4];
    philox((uint32_t)(at >> 3), e.place & 0x7fffffffu, 3u, k0, k1, rnd);
    const uint2 mo = encode<false, 0>(x, rnd, e.m_scale + block, lane);
    const uint2 vo = encode<true, 1>(root, rnd, e.v_scale + block, lane);
    store_codes((uint8_t*)e.m + at, have, wide, mo);
    store_codes((uint8_t*)e.v + at, have, wide, vo);
  }
}

bool aligned(const void* p, size_t to) { return ((uintptr_t)p & (to - 1)) == 0; }

template <typename P, typename G, int BITS, int CAP>
cudaError_t launch(const Table<CAP>& t, uint32_t chunks, cudaStream_t st) {
  adamw_kernel<P, G, BITS, CAP><<<chunks, THREADS<BITS>, 0, st>>>(t);
  return cudaGetLastError();
}
template <int CAP>
cudaError_t launch_class(int cls, const Table<CAP>& t, uint32_t chunks, cudaStream_t st) {
  using B = __nv_bfloat16;
  switch (cls) {
    case 0: return launch<float, float, 32, CAP>(t, chunks, st);
    case 1: return launch<B, float, 32, CAP>(t, chunks, st);
    case 2: return launch<float, B, 32, CAP>(t, chunks, st);
    case 3: return launch<B, B, 32, CAP>(t, chunks, st);
    case 4: return launch<float, float, 8, CAP>(t, chunks, st);
    case 5: return launch<B, float, 8, CAP>(t, chunks, st);
    case 6: return launch<float, B, 8, CAP>(t, chunks, st);
    default: return launch<B, B, 8, CAP>(t, chunks, st);
  }
}

int class_of(const vcas_adamw_tensor& x) {
  return (x.p_dtype == VCAS_DTYPE_BF16 ? 1 : 0) + (x.g_dtype == VCAS_DTYPE_BF16 ? 2 : 0) + (x.state_bits == 8 ? 4 : 0);
}

// The next launch of one class: tensors from `from` on, at most CAP of them and 2^30 chunks.
template <int CAP>
int fill(const vcas_adamw_tensor* ts, int n, int cls, int from, double lr, Table<CAP>& t, uint32_t* chunks) {
  t.count = 0;
  *chunks = 0;
  int i = from;
  for (; i < n && t.count < CAP; ++i) {
    const vcas_adamw_tensor& x = ts[i];
    if (x.n == 0 || class_of(x) != cls) continue;
    const int64_t chunk = x.state_bits == 8 ? CHUNK<8> : CHUNK<32>, c = (x.n + chunk - 1) / chunk;
    if (*chunks + c > (1u << 30)) break;
    Entry& e = t.e[t.count++];
    e.p = x.p; e.g = x.g; e.m = x.m; e.v = x.v; e.m_scale = x.m_scale; e.v_scale = x.v_scale; e.copy = x.copy;
    e.n = x.n;
    e.keep = (float)(1.0 - lr * (double)x.weight_decay);
    e.decay = x.weight_decay;
    e.first = *chunks;
    const size_t pa = x.p_dtype == VCAS_DTYPE_BF16 ? 16 : 32, ga = x.g_dtype == VCAS_DTYPE_BF16 ? 16 : 32;
    const size_t sa = x.state_bits == 8 ? 8 : 32;
    const bool wide = aligned(x.p, pa) && aligned(x.g, ga) && aligned(x.m, sa) && aligned(x.v, sa) && aligned(x.copy, 16);
    e.place = (uint32_t)i | (wide ? 0x80000000u : 0u);
    *chunks += (uint32_t)c;
  }
  return i;
}

template <int CAP>
cudaError_t run(const vcas_adamw_tensor* ts, int n, int cls, const vcas_adamw_args& a, cudaStream_t st) {
  Table<CAP> t;
  t.b1 = (float)a.beta1; t.c1 = (float)(1.0 - a.beta1);
  t.b2 = (float)a.beta2; t.c2 = (float)(1.0 - a.beta2);
  t.eps = (float)a.eps;
  t.step_size = t.inv = 0.f;
  double lr = a.lr;
  if (a.rates == nullptr) {
    float r[3];
    vcas_adamw_rates(a.lr, a.beta1, a.beta2, a.step, r);
    t.step_size = r[1];
    t.inv = r[2];
  } else {
    lr = 0.0;
  }
  t.seed_lo = (uint32_t)a.seed; t.seed_hi = (uint32_t)(a.seed >> 32);
  t.grad_scale = a.grad_scale; t.rates = a.rates; t.seed_dev = a.seed_dev;
  for (int from = 0; from < n;) {
    uint32_t chunks = 0;
    from = fill<CAP>(ts, n, cls, from, lr, t, &chunks);
    if (t.count == 0) continue;
    const cudaError_t e = launch_class<CAP>(cls, t, chunks, st);
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

bool in_unit(double b) { return b >= 0.0 && b < 1.0; }

}  // namespace
}  // namespace vcas

using namespace vcas;

extern "C" int vcas_adamw_rates(double lr, double beta1, double beta2, int64_t step, float* rates) {
  if (rates == nullptr || !std::isfinite(lr) || lr < 0.0 || !in_unit(beta1) || !in_unit(beta2) || step < 1) return VCAS_ERR_BAD_ARG;
  rates[0] = (float)lr;
  rates[1] = (float)(lr / (1.0 - std::pow(beta1, (double)step)));
  rates[2] = (float)(1.0 / std::sqrt(1.0 - std::pow(beta2, (double)step)));
  return VCAS_OK;
}

extern "C" int vcas_adamw_step(const vcas_adamw_tensor* ts, int32_t n, const vcas_adamw_args* args, vcas_stream stream) {
  if (n < 0 || args == nullptr || (n > 0 && ts == nullptr)) return VCAS_ERR_BAD_ARG;
  float unused[3];
  const vcas_adamw_args& a = *args;
  const int rc = vcas_adamw_rates(a.rates == nullptr ? a.lr : 0.0, a.beta1, a.beta2, a.rates == nullptr ? a.step : 1, unused);
  if (rc != VCAS_OK) return rc;
  if (!std::isfinite(a.eps) || a.eps < 0.0) return VCAS_ERR_BAD_ARG;
  int in_class[8] = {};
  for (int i = 0; i < n; ++i) {
    const vcas_adamw_tensor& x = ts[i];
    if (x.n < 0 || x.n > (int64_t)1 << 34) return VCAS_ERR_SHAPE;
    if ((x.p_dtype != VCAS_DTYPE_F32 && x.p_dtype != VCAS_DTYPE_BF16) ||
        (x.g_dtype != VCAS_DTYPE_F32 && x.g_dtype != VCAS_DTYPE_BF16) || (x.state_bits != 8 && x.state_bits != 32))
      return VCAS_ERR_DTYPE;
    if (!std::isfinite(x.weight_decay) || x.weight_decay < 0.f) return VCAS_ERR_BAD_ARG;
    if (x.copy != nullptr && x.p_dtype != VCAS_DTYPE_F32) return VCAS_ERR_DTYPE;
    if (x.n == 0) continue;
    if (x.p == nullptr || x.g == nullptr || x.m == nullptr || x.v == nullptr ||
        (x.state_bits == 8 && (x.m_scale == nullptr || x.v_scale == nullptr)))
      return VCAS_ERR_BAD_ARG;
    const size_t pa = x.p_dtype == VCAS_DTYPE_BF16 ? 2 : 4, ga = x.g_dtype == VCAS_DTYPE_BF16 ? 2 : 4;
    const size_t sa = x.state_bits == 8 ? 1 : 4;
    if (!aligned(x.p, pa) || !aligned(x.g, ga) || !aligned(x.m, sa) || !aligned(x.v, sa) || !aligned(x.copy, 2) ||
        !aligned(x.m_scale, 4) || !aligned(x.v_scale, 4))
      return VCAS_ERR_BAD_ARG;
    ++in_class[class_of(x)];
  }
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  for (int c = 0; c < 8; ++c) {
    if (in_class[c] == 0) continue;
    const cudaError_t e = in_class[c] <= SMALL ? run<SMALL>(ts, n, c, a, st) : run<LARGE>(ts, n, c, a, st);
    if (e != cudaSuccess) return VCAS_ERR_CUDA;
  }
  return VCAS_OK;
}
