// Attention over packed sequences: C entry points, and the kernels that serve every type, alignment and stride (fp32 layers, and
// bf16 tensors that TMA cannot address) on the fp32 FMA pipe.  The tensor-core kernels are in attn_umma.cu.
//
// The forward keeps, per row, the running maximum m of the scores and l = sum exp(S - m); a new maximum rescales l and the
// accumulated O by exp(m_old - m_new), so that one pass over K and V is enough.  The backward recomputes P = exp(S - lse).  It runs
// as two kernels, one over query tiles (dQ) and one over key tiles (dK, dV, over all query heads that share them), so that every
// sum has one owner and a fixed order: no atomics, and two calls give the same bits; the price is a second S and dP.
#include <new>

#include "attn.cuh"

namespace vcas {
namespace {

constexpr int TILE = 64;                 // rows of a query tile and of a key tile
constexpr int THREADS = 256;             // 16 x 16, each 4 x 4 scores

__device__ __forceinline__ float widen(float x) { return x; }
__device__ __forceinline__ float widen(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ void put(float* p, float x) { *p = x; }
__device__ __forceinline__ void put(__nv_bfloat16* p, float x) { *p = __float2bfloat16_rn(x); }

// Rows t0 .. t0 + 63 of one head, zeros behind the sequence's end and the head's width: a thread's share in registers (all of its loads
// are on their way at once), then in shared memory.  fp32 rows that allow it are read 16 bytes at a time.
template <typename T, int DP>
struct TileLoad {
  static constexpr int N = TILE * DP / 4 / THREADS;
  float4 v[N];
  __device__ __forceinline__ void get(const Strided& x, int first, int len, int t0, int head, int dim) {
    const T* base = (const T*)x.p + (int64_t)head * x.head + (int64_t)(first + t0) * x.token;
    const bool wide = sizeof(T) == 4 && ((uintptr_t)base & 15) == 0 && (x.token & 3) == 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int at = (threadIdx.x + i * THREADS) * 4, r = at / DP, d = at % DP;
      v[i] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (t0 + r < len && d < dim) {       // dim is a multiple of 8
        const T* p = base + (int64_t)r * x.token + d;
        if (wide) v[i] = __ldg(reinterpret_cast<const float4*>(p));
        else v[i] = make_float4(widen(p[0]), widen(p[1]), widen(p[2]), widen(p[3]));
      }
    }
  }
  __device__ __forceinline__ void put(float* dst) const {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int at = (threadIdx.x + i * THREADS) * 4;
      *reinterpret_cast<float4*>(dst + at / DP * (DP + 4) + at % DP) = v[i];
    }
  }
};
template <typename T, int DP>
__device__ __forceinline__ void load_tile(float* dst, const Strided& x, int first, int len, int t0, int head, int dim) {
  TileLoad<T, DP> l;
  l.get(x, first, len, t0, head, dim);
  l.put(dst);
}
template <typename T, int DP>
__device__ __forceinline__ void load_two(float* da, const Strided& a, float* db, const Strided& b, int first, int len, int t0, int head,
                                         int dim) {
  TileLoad<T, DP> la, lb;
  la.get(a, first, len, t0, head, dim);
  lb.get(b, first, len, t0, head, dim);
  la.put(da);
  lb.put(db);
}
// s[i][j] = sum_d a[ty * 4 + i][d] b[tx + 16 j][d]
template <int DP>
__device__ __forceinline__ void dots(const float* a, const float* b, int tx, int ty, float (&s)[4][4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) s[i][j] = 0.f;
#pragma unroll 4
  for (int d = 0; d < DP; d += 4) {
    float4 x[4], y[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = *reinterpret_cast<const float4*>(a + (ty * 4 + i) * (DP + 4) + d);
#pragma unroll
    for (int j = 0; j < 4; ++j) y[j] = *reinterpret_cast<const float4*>(b + (tx + 16 * j) * (DP + 4) + d);
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        s[i][j] = fmaf(x[i].x, y[j].x, fmaf(x[i].y, y[j].y, fmaf(x[i].z, y[j].z, fmaf(x[i].w, y[j].w, s[i][j]))));
  }
}
// acc[i][c] += sum_r w(i, r) x[r][column c of this thread], columns tx * 4 + 64 jj + e
template <int DP, typename W>
__device__ __forceinline__ void weighted(const float* x, int tx, float (&acc)[4][DP / 16], W w) {
#pragma unroll 4
  for (int r = 0; r < TILE; ++r) {
    float f[4];
    w(r, f);
#pragma unroll
    for (int jj = 0; jj < DP / 64; ++jj) {
      const float4 y = *reinterpret_cast<const float4*>(x + r * (DP + 4) + tx * 4 + 64 * jj);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        acc[i][jj * 4 + 0] = fmaf(f[i], y.x, acc[i][jj * 4 + 0]);
        acc[i][jj * 4 + 1] = fmaf(f[i], y.y, acc[i][jj * 4 + 1]);
        acc[i][jj * 4 + 2] = fmaf(f[i], y.z, acc[i][jj * 4 + 2]);
        acc[i][jj * 4 + 3] = fmaf(f[i], y.w, acc[i][jj * 4 + 3]);
      }
    }
  }
}
template <typename T, int DP>
__device__ __forceinline__ void store_rows(const Strided& x, int first, int len, int t0, int head, int dim, int tx, int ty,
                                           const float (&acc)[4][DP / 16], const float (&factor)[4]) {
  T* base = (T*)const_cast<void*>(x.p) + (int64_t)head * x.head;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int t = t0 + ty * 4 + i;
    if (t >= len) continue;
#pragma unroll
    for (int c = 0; c < DP / 16; ++c) {
      const int d = tx * 4 + 64 * (c / 4) + c % 4;
      if (d < dim) put(base + (int64_t)(first + t) * x.token + d, acc[i][c] * factor[i]);
    }
  }
}

struct Place { int first, len, t0, head; bool any; };
// rows: of a tile; last_first: the last tile of a sequence (the longest row of a causal one) comes first
__device__ __forceinline__ Place place_of(const Seqs& q, int heads, bool last_first) {
  __shared__ Place s;
  if (threadIdx.x < 32) {
    Place p = {0, 0, 0, (int)(blockIdx.x % (unsigned)heads), false};
    int place = 0;
    p.any = find_tile(q, (int)(blockIdx.x / (unsigned)heads), TILE, threadIdx.x, p.first, p.len, place);
    p.t0 = (last_first ? (p.len + TILE - 1) / TILE - 1 - place : place) * TILE;
    if (threadIdx.x == 0) s = p;
  }
  __syncthreads();
  return s;
}

template <typename T, int DP>
__global__ void __launch_bounds__(THREADS) attn_fma_fwd_kernel(AttnCall C) {
  extern __shared__ __align__(16) float sm[];
  float *sq = sm, *sk = sq + TILE * (DP + 4), *sv = sk + TILE * (DP + 4), *sp = sv + TILE * (DP + 4);
  const Place p = place_of(C.seqs, C.heads_q, C.causal);
  if (!p.any) return;
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  load_tile<T, DP>(sq, C.q, p.first, p.len, p.t0, p.head, C.dim);
  const float c = C.scale * ATTN_LOG2E;
  const int end = C.causal ? min(p.len, p.t0 + TILE) : p.len;
  float m[4], l[4], acc[4][DP / 16];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    m[i] = __int_as_float(0xff800000);
    l[i] = 0.f;
#pragma unroll
    for (int d = 0; d < DP / 16; ++d) acc[i][d] = 0.f;
  }
  for (int j0 = 0; j0 < end; j0 += TILE) {
    __syncthreads();
    load_two<T, DP>(sk, C.k, sv, C.v, p.first, p.len, j0, p.head / C.group, C.dim);
    __syncthreads();
    float s[4][4];
    dots<DP>(sq, sk, tx, ty, s);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int row = p.t0 + ty * 4 + i;
      float top = m[i];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int col = j0 + tx + 16 * j;
        s[i][j] = col < p.len && (!C.causal || col <= row) ? s[i][j] * c : __int_as_float(0xff800000);
        top = fmaxf(top, s[i][j]);
      }
#pragma unroll
      for (int o = 1; o < 16; o <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
      const float ref = top == __int_as_float(0xff800000) ? 0.f : top;       // nothing seen yet: exp(-inf - 0) = 0
      const float f = attn_exp2(m[i] - ref);
      m[i] = top;
      l[i] *= f;
#pragma unroll
      for (int d = 0; d < DP / 16; ++d) acc[i][d] *= f;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float e = attn_exp2(s[i][j] - ref);
        l[i] += e;
        sp[(ty * 4 + i) * (TILE + 4) + tx + 16 * j] = e;
      }
    }
    __syncwarp();                        // a row's probabilities are made and read by one half-warp
    weighted<DP>(sv, tx, acc, [&](int r, float (&f)[4]) {
#pragma unroll
      for (int i = 0; i < 4; ++i) f[i] = sp[(ty * 4 + i) * (TILE + 4) + r];
    });
  }
  float inv[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
#pragma unroll
    for (int o = 1; o < 16; o <<= 1) l[i] += __shfl_xor_sync(0xffffffffu, l[i], o);
    inv[i] = 1.0f / l[i];
    const int t = p.t0 + ty * 4 + i;
    if (tx == 0 && t < p.len) C.lse[(int64_t)p.head * C.seqs.total + p.first + t] = m[i] * ATTN_LN2 + logf(l[i]);
  }
  store_rows<T, DP>(C.o, p.first, p.len, p.t0, p.head, C.dim, tx, ty, acc, inv);
}

// P and dS of one pair of tiles for this thread's 4 x 4 places, 0 where a row does not look
__device__ __forceinline__ void p_and_ds(const AttnCall& C, const Place& p, int i0, int j0, int tx, int ty, const float (&lse)[4],
                                         const float (&delta)[4], float (&s)[4][4], float (&dp)[4][4]) {
  const float c = C.scale * ATTN_LOG2E;
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int row = i0 + ty * 4 + i, col = j0 + tx + 16 * j;
      const bool see = row < p.len && col < p.len && (!C.causal || col <= row);
      const bool alone = C.causal ? row == 0 : p.len == 1;       // one key: P = 1, dS = 0
      s[i][j] = !see ? 0.f : alone ? 1.f : attn_exp2(s[i][j] * c - lse[i]);
      dp[i][j] = see && !alone ? s[i][j] * (dp[i][j] - delta[i]) : 0.f;
    }
}
// rowsum(dO O) of this thread's rows, from tiles of both; every thread of a row has it
template <int DP>
__device__ __forceinline__ void row_sums(const float* a, const float* b, int tx, int ty, float (&sum)[4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    sum[i] = 0.f;
#pragma unroll
    for (int jj = 0; jj < DP / 64; ++jj) {
      const int at = (ty * 4 + i) * (DP + 4) + tx * 4 + 64 * jj;
      const float4 x = *reinterpret_cast<const float4*>(a + at), y = *reinterpret_cast<const float4*>(b + at);
      sum[i] = fmaf(x.x, y.x, fmaf(x.y, y.y, fmaf(x.z, y.z, fmaf(x.w, y.w, sum[i]))));
    }
#pragma unroll
    for (int o = 1; o < 16; o <<= 1) sum[i] += __shfl_xor_sync(0xffffffffu, sum[i], o);
  }
}
// lse in units of log 2, and delta, of this thread's rows
__device__ __forceinline__ void row_values(const AttnCall& C, const Place& p, int i0, int head, int ty, float (&lse)[4], float (&delta)[4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int t = i0 + ty * 4 + i;
    const int64_t at = (int64_t)head * C.seqs.total + p.first + t;
    lse[i] = t < p.len ? C.lse[at] * ATTN_LOG2E : 0.f;
    delta[i] = t < p.len ? C.delta[at] : 0.f;
  }
}

template <typename T, int DP>
__global__ void __launch_bounds__(THREADS) attn_fma_dq_kernel(AttnCall C) {
  extern __shared__ __align__(16) float sm[];
  constexpr int SZ = TILE * (DP + 4);
  float *sq = sm, *sdo = sq + SZ, *sk = sdo + SZ, *sv = sk + SZ, *sds = sv + SZ;
  const Place p = place_of(C.seqs, C.heads_q, C.causal);
  if (!p.any) return;
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  load_two<T, DP>(sq, C.q, sdo, C.d_o, p.first, p.len, p.t0, p.head, C.dim);
  load_tile<T, DP>(sk, C.o, p.first, p.len, p.t0, p.head, C.dim);
  float lse[4], delta[4], acc[4][DP / 16];
  __syncthreads();
  row_sums<DP>(sdo, sk, tx, ty, delta);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int t = p.t0 + ty * 4 + i;
    const int64_t at = (int64_t)p.head * C.seqs.total + p.first + t;
    lse[i] = t < p.len ? C.lse[at] * ATTN_LOG2E : 0.f;
    if (tx == 0 && t < p.len) C.delta[at] = delta[i];        // for the dK, dV kernel
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int d = 0; d < DP / 16; ++d) acc[i][d] = 0.f;
  const int end = C.causal ? min(p.len, p.t0 + TILE) : p.len;
  for (int j0 = 0; j0 < end; j0 += TILE) {
    __syncthreads();
    load_two<T, DP>(sk, C.k, sv, C.v, p.first, p.len, j0, p.head / C.group, C.dim);
    __syncthreads();
    float s[4][4], dp[4][4];
    dots<DP>(sq, sk, tx, ty, s);
    dots<DP>(sdo, sv, tx, ty, dp);
    p_and_ds(C, p, p.t0, j0, tx, ty, lse, delta, s, dp);
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) sds[(ty * 4 + i) * (TILE + 4) + tx + 16 * j] = dp[i][j];
    __syncwarp();
    weighted<DP>(sk, tx, acc, [&](int r, float (&f)[4]) {
#pragma unroll
      for (int i = 0; i < 4; ++i) f[i] = sds[(ty * 4 + i) * (TILE + 4) + r];
    });
  }
  const float f[4] = {C.scale, C.scale, C.scale, C.scale};
  store_rows<T, DP>(C.dq, p.first, p.len, p.t0, p.head, C.dim, tx, ty, acc, f);
}

template <typename T, int DP>
__global__ void __launch_bounds__(THREADS) attn_fma_dkv_kernel(AttnCall C) {
  extern __shared__ __align__(16) float sm[];
  constexpr int SZ = TILE * (DP + 4);
  float *sk = sm, *sv = sk + SZ, *sq = sv + SZ, *sdo = sq + SZ, *sp = sdo + SZ, *sds = sp + TILE * (TILE + 4);
  const Place p = place_of(C.seqs, C.heads_kv, false);
  if (!p.any) return;
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  load_two<T, DP>(sk, C.k, sv, C.v, p.first, p.len, p.t0, p.head, C.dim);
  float dk[4][DP / 16], dv[4][DP / 16];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int d = 0; d < DP / 16; ++d) dk[i][d] = dv[i][d] = 0.f;
  for (int g = 0; g < C.group; ++g) {
    const int head = p.head * C.group + g;
    for (int i0 = C.causal ? p.t0 : 0; i0 < p.len; i0 += TILE) {
      __syncthreads();
      load_two<T, DP>(sq, C.q, sdo, C.d_o, p.first, p.len, i0, head, C.dim);
      float lse[4], delta[4];
      row_values(C, p, i0, head, ty, lse, delta);
      __syncthreads();
      float s[4][4], dp[4][4];
      dots<DP>(sq, sk, tx, ty, s);
      dots<DP>(sdo, sv, tx, ty, dp);
      p_and_ds(C, p, i0, p.t0, tx, ty, lse, delta, s, dp);
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          sp[(ty * 4 + i) * (TILE + 4) + tx + 16 * j] = s[i][j];
          sds[(ty * 4 + i) * (TILE + 4) + tx + 16 * j] = dp[i][j];
        }
      __syncthreads();
      auto columns = [&](const float* from) {
        return [=](int r, float (&f)[4]) {
          const float4 v = *reinterpret_cast<const float4*>(from + r * (TILE + 4) + ty * 4);
          f[0] = v.x; f[1] = v.y; f[2] = v.z; f[3] = v.w;
        };
      };
      weighted<DP>(sdo, tx, dv, columns(sp));
      weighted<DP>(sq, tx, dk, columns(sds));
    }
  }
  const float one[4] = {1.f, 1.f, 1.f, 1.f}, f[4] = {C.scale, C.scale, C.scale, C.scale};
  store_rows<T, DP>(C.dv, p.first, p.len, p.t0, p.head, C.dim, tx, ty, dv, one);
  store_rows<T, DP>(C.dk, p.first, p.len, p.t0, p.head, C.dim, tx, ty, dk, f);
}

// Zeros in the gradients' rows of the sequences that are not worked on.  A warp has some tokens one behind the other, and finds their
// sequences by bisection.  Whether these are kept it reads from the list, as it goes through it once; a long one that ascends is
// searched by bisection too.  wide: rows can be written 16 bytes at a time.
template <typename T>
__global__ void __launch_bounds__(128, 16) attn_zero_kernel(AttnCall C, bool wide) {
  pdl_trigger();                         // what follows works on other sequences
  const Seqs& q = C.seqs;
  const int lane = threadIdx.x & 31, in_cta = (int)(blockDim.x >> 5), warps = (int)gridDim.x * in_cta;
  const int warp = (int)blockIdx.x * in_cta + (int)(threadIdx.x >> 5);
  const int count = seq_count(q);
  bool in_order = false;
  if (count > 256) {
    int good = 1;
#pragma unroll 4
    for (int k = threadIdx.x; k < count; k += 128) {
      const int n = __ldcg(q.alive + k), before = k > 0 ? __ldcg(q.alive + k - 1) : -1;
      good &= n < q.N && n > before;
    }
    in_order = __syncthreads_and(good);
  }
  // a row of zeros in pieces of 16 bytes: this lane's piece of a head, and its heads mine, mine + at_once, ...
  constexpr int VN = 16 / sizeof(T);
  const int per = C.dim / VN, at_once = 32 / per, piece = lane % per, mine = lane / per < at_once ? lane / per : 1 << 20;
  auto zero_row = [&](int t) {
    auto zero = [&](const Strided& x, int heads) {
      T* base = (T*)const_cast<void*>(x.p) + (int64_t)t * x.token;
      if (wide) {
        base += mine * x.head + piece * VN;
        const int64_t step = at_once * x.head;
#pragma unroll 4
        for (int h = mine; h < heads; h += at_once, base += step) *reinterpret_cast<uint4*>(base) = make_uint4(0, 0, 0, 0);
      } else {
        for (int i = lane; i < heads * C.dim; i += 32) put(base + (int64_t)(i / C.dim) * x.head + i % C.dim, 0.f);
      }
    };
    zero(C.dq, C.heads_q);
    zero(C.dk, C.heads_kv);
    zero(C.dv, C.heads_kv);
  };
  // The entries that count (see seq_listed) ascend, and the first that is n or more is one of them.  at: where in the list it may be; a
  // later sequence's is not before it.
  int at = 0;
  auto is_kept = [&](int n) {
    if (in_order) {
      int a = 0, b = count;
      while (a < b) {
        const int mid = (a + b) >> 1;
        if (q.alive[mid] < n) a = mid + 1; else b = mid;
      }
      return a < count && q.alive[a] == n;
    }
    for (; at < count; at += 32) {
      const int v = at + lane < count ? __ldcg(q.alive + at + lane) : -1;
      const unsigned hit = __ballot_sync(0xffffffffu, v >= n && v < q.N);
      if (hit != 0) return __shfl_sync(0xffffffffu, v, __ffs(hit) - 1) == n;
    }
    return false;
  };
  const int each = (q.total + warps - 1) / warps;
  const int64_t from = (int64_t)warp * each;
  const int to = (int)min((int64_t)q.total, from + each);
  int first = 0, end = 0;                // the sequence that t lies in, once found
  bool kept = false;
  for (int t = (int)min((int64_t)q.total, from); t < to; ++t) {
    if (t < first || t >= end) {
      // the last sequence that begins at or before t (the empty ones before it begin there too)
      int lo = 0, hi = q.N - 1;
      while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (q.starts[mid] <= t) lo = mid; else hi = mid - 1;
      }
      const int len = seq_length(q, lo, first);
      end = first + len;
      if (t < first || t >= end) continue;
      kept = is_kept(lo);
    }
    if (kept) t = end - 1;               // nothing to do up to there
    else zero_row(t);
  }
}

template <typename K>
cudaError_t run(K kernel, size_t smem, long grid, const AttnCall& c, cudaStream_t st) {
  if (grid > 0x7fffffffl) return cudaErrorInvalidValue;
  kernel<<<(unsigned)grid, THREADS, smem, st>>>(c);
  return cudaGetLastError();
}
template <int DP> constexpr size_t smem_of(int tiles, int squares) {
  return (size_t)(tiles * TILE * (DP + 4) + squares * TILE * (TILE + 4)) * sizeof(float);
}
template <typename T, int DP>
cudaError_t fwd(const AttnCall& c, cudaStream_t st) {
  const long tiles = tile_bound(c.seqs.total, c.seqs.N, TILE);
  return run(attn_fma_fwd_kernel<T, DP>, smem_of<DP>(3, 1), tiles * c.heads_q, c, st);
}
template <typename T, int DP>
cudaError_t bwd(const AttnCall& c, cudaStream_t st) {
  const long tiles = tile_bound(c.seqs.total, c.seqs.N, TILE);
  const cudaError_t e = run(attn_fma_dq_kernel<T, DP>, smem_of<DP>(4, 1), tiles * c.heads_q, c, st);
  return e != cudaSuccess ? e : run(attn_fma_dkv_kernel<T, DP>, smem_of<DP>(4, 2), tiles * c.heads_kv, c, st);
}

inline Attn* A(vcas_attn a) { return reinterpret_cast<Attn*>(a); }

// Shared checks of a call's tensors; elements are addressed one by one, so that only the dtype's own alignment is asked for.
bool good(const vcas_attn_tensor* x, size_t elem) {
  return x != nullptr && x->ptr != nullptr && ((uintptr_t)x->ptr & (elem - 1)) == 0 && x->token >= 0 && x->head >= 0 &&
         x->token < (1ll << 40) && x->head < (1ll << 40);
}
// of one that is written, no two elements in one place
bool good_out(const vcas_attn_tensor* x, int total, int heads, int dim, size_t elem) {
  if (!good(x, elem)) return false;
  const bool inner_head = x->head <= x->token;
  const int64_t s0 = inner_head ? x->head : x->token, s1 = inner_head ? x->token : x->head;
  const int64_t n0 = inner_head ? heads : total, n1 = inner_head ? total : heads;
  return (n0 <= 1 || s0 >= dim) && (n1 <= 1 || s1 >= (n0 > 1 ? s0 * n0 : dim));
}
Strided S(const vcas_attn_tensor* x) { return Strided{x->ptr, x->token, x->head}; }

int begin(const Attn* a, const int32_t* starts, int32_t N, int32_t total, const int32_t* alive, const int32_t* cnt, AttnCall& c) {
  const vcas_attn_desc& d = a->desc;
  if (N < 0 || N > d.max_seqs || total < 0 || total > d.max_tokens) return VCAS_ERR_SHAPE;
  if (N > 0 && starts == nullptr) return VCAS_ERR_BAD_ARG;
  if ((alive == nullptr) != (cnt == nullptr)) return VCAS_ERR_BAD_ARG;
  c.seqs = Seqs{starts, alive, cnt, N, total, a->status};
  c.delta = a->delta;
  c.heads_q = d.heads_q; c.heads_kv = d.heads_kv; c.group = d.heads_q / d.heads_kv;
  c.dim = d.head_dim; c.causal = d.causal != 0; c.scale = a->scale;
  return VCAS_OK;
}

}  // namespace

template <typename T, int DP>
static cudaError_t room() {
  auto set = [](const void* k, size_t bytes) { return cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes); };
  cudaError_t e = set((const void*)attn_fma_fwd_kernel<T, DP>, smem_of<DP>(3, 1));
  if (e == cudaSuccess) e = set((const void*)attn_fma_dq_kernel<T, DP>, smem_of<DP>(4, 1));
  if (e == cudaSuccess) e = set((const void*)attn_fma_dkv_kernel<T, DP>, smem_of<DP>(4, 2));
  return e;
}
cudaError_t attn_fma_prepare() {
  cudaError_t e = room<float, 64>();
  if (e == cudaSuccess) e = room<float, 128>();
  if (e == cudaSuccess) e = room<__nv_bfloat16, 64>();
  if (e == cudaSuccess) e = room<__nv_bfloat16, 128>();
  // an SM divides its memory anew only when it is idle: as the kernel needs it that is to begin beside this one
  auto beside = [](const void* k) { return cudaFuncSetAttribute(k, cudaFuncAttributePreferredSharedMemoryCarveout, cudaSharedmemCarveoutMaxShared); };
  if (e == cudaSuccess) e = beside((const void*)attn_zero_kernel<float>);
  if (e == cudaSuccess) e = beside((const void*)attn_zero_kernel<__nv_bfloat16>);
  return e;
}
cudaError_t launch_attn_fma_fwd(const Attn* a, const AttnCall& c, cudaStream_t st) {
  if (a->desc.dtype == VCAS_DTYPE_BF16)
    return c.dim <= 64 ? fwd<__nv_bfloat16, 64>(c, st) : fwd<__nv_bfloat16, 128>(c, st);
  return c.dim <= 64 ? fwd<float, 64>(c, st) : fwd<float, 128>(c, st);
}
cudaError_t launch_attn_fma_bwd(const Attn* a, const AttnCall& c, cudaStream_t st) {
  if (c.seqs.alive != nullptr && !c.skip_dropped) {
    const cudaError_t e = launch_attn_zero(a, c, st);
    if (e != cudaSuccess) return e;
  }
  if (a->desc.dtype == VCAS_DTYPE_BF16)
    return c.dim <= 64 ? bwd<__nv_bfloat16, 64>(c, st) : bwd<__nv_bfloat16, 128>(c, st);
  return c.dim <= 64 ? bwd<float, 64>(c, st) : bwd<float, 128>(c, st);
}
cudaError_t launch_attn_zero(const Attn* a, const AttnCall& c, cudaStream_t st) {
  // Beside the kernel that follows: one small CTA an SM leaves it its registers, and as all of them begin at once, so does that kernel
  // (64 x 197 tokens of 12 heads of 64, 40 % kept: 57.7 us for the whole backward, 64.8 with a warp a token).
  const int threads = 128, most = (c.seqs.total + threads / 32 - 1) / (threads / 32);
  const unsigned grid = (unsigned)(most < a->num_sms ? most : a->num_sms);
  const int elem = a->desc.dtype == VCAS_DTYPE_BF16 ? 2 : 4, vn = 16 / elem;
  auto wide = [&](const Strided& x) { return ((uintptr_t)x.p & 15) == 0 && x.token % vn == 0 && x.head % vn == 0; };
  const bool w = wide(c.dq) && wide(c.dk) && wide(c.dv);
  if (elem == 2) attn_zero_kernel<__nv_bfloat16><<<grid, threads, 0, st>>>(c, w);
  else attn_zero_kernel<float><<<grid, threads, 0, st>>>(c, w);
  return cudaGetLastError();
}

}  // namespace vcas

using namespace vcas;

extern "C" int vcas_attn_create(vcas_attn* out, const vcas_attn_desc* desc) {
  if (out == nullptr || desc == nullptr) return VCAS_ERR_BAD_ARG;
  *out = nullptr;
  const vcas_attn_desc& d = *desc;
  if (d.dtype != VCAS_DTYPE_F32 && d.dtype != VCAS_DTYPE_BF16) return VCAS_ERR_DTYPE;
  if (d.max_tokens <= 0 || d.max_tokens > (1 << 30) || d.max_seqs <= 0 || d.max_seqs > (1 << 24)) return VCAS_ERR_SHAPE;
  if (d.heads_kv <= 0 || d.heads_q <= 0 || d.heads_q > 1024 || d.heads_q % d.heads_kv != 0) return VCAS_ERR_SHAPE;
  if (d.head_dim <= 0 || d.head_dim > 128 || d.head_dim % 8 != 0) return VCAS_ERR_SHAPE;
  if (!(d.scale >= 0.f) || d.scale > 1e30f) return VCAS_ERR_BAD_ARG;
  Attn* a = new (std::nothrow) Attn();
  if (a == nullptr) return VCAS_ERR_WORKSPACE;
  a->desc = d;
  a->scale = d.scale > 0.f ? d.scale : 1.0f / sqrtf((float)d.head_dim);
  a->wait_limit_ns = 2000000000ull;
  a->stall_once = 0;
  int major = 0;
  if (cudaGetDevice(&a->device) != cudaSuccess ||
      cudaDeviceGetAttribute(&a->num_sms, cudaDevAttrMultiProcessorCount, a->device) != cudaSuccess ||
      cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, a->device) != cudaSuccess) {
    delete a;
    return VCAS_ERR_CUDA;
  }
  a->tensor_ok = d.dtype == VCAS_DTYPE_BF16 && major == 10;
  if (attn_fma_prepare() != cudaSuccess || (a->tensor_ok && attn_umma_prepare() != cudaSuccess)) {
    cudaGetLastError();
    delete a;
    return VCAS_ERR_CUDA;
  }
  const size_t delta = ((size_t)d.heads_q * d.max_tokens * sizeof(float) + 255) & ~(size_t)255;
  a->bytes = delta + 256;
  if (cudaMalloc(&a->base, a->bytes) != cudaSuccess) {
    cudaGetLastError();
    delete a;
    return VCAS_ERR_WORKSPACE;
  }
  a->delta = (float*)a->base;
  a->status = (int32_t*)((uint8_t*)a->base + delta);
  a->next = a->status + 1;
  if (cudaMemset(a->base, 0, a->bytes) != cudaSuccess || cudaDeviceSynchronize() != cudaSuccess) {
    cudaFree(a->base);
    delete a;
    return VCAS_ERR_CUDA;
  }
  *out = reinterpret_cast<vcas_attn>(a);
  return VCAS_OK;
}

extern "C" int vcas_attn_destroy(vcas_attn aa) {
  if (aa == nullptr) return VCAS_ERR_BAD_ARG;
  Attn* a = A(aa);
  DeviceScope on(a->device);
  const cudaError_t e = cudaFree(a->base);
  delete a;
  return e == cudaSuccess ? VCAS_OK : VCAS_ERR_CUDA;
}

extern "C" int vcas_attn_workspace_bytes(vcas_attn a, size_t* bytes) {
  if (a == nullptr || bytes == nullptr) return VCAS_ERR_BAD_ARG;
  *bytes = A(a)->bytes;
  return VCAS_OK;
}

extern "C" int vcas_attn_fwd(vcas_attn aa, const vcas_attn_tensor* q, const vcas_attn_tensor* k, const vcas_attn_tensor* v,
                             const int32_t* starts, int32_t N, int32_t total, const vcas_attn_tensor* o, float* lse,
                             vcas_stream stream) {
  if (aa == nullptr) return VCAS_ERR_BAD_ARG;
  Attn* a = A(aa);
  AttnCall c = {};
  const int rc = begin(a, starts, N, total, nullptr, nullptr, c);
  if (rc != VCAS_OK) return rc;
  if (N == 0 || total == 0) return VCAS_OK;
  const size_t elem = a->desc.dtype == VCAS_DTYPE_BF16 ? 2 : 4;
  const int D = c.dim;
  if (!good(q, elem) || !good(k, elem) || !good(v, elem) || !good_out(o, total, c.heads_q, D, elem) || lse == nullptr)
    return VCAS_ERR_BAD_ARG;
  c.q = S(q); c.k = S(k); c.v = S(v); c.o = S(o); c.lse = lse;
  DeviceScope on(a->device);
  if (!on.ok) return VCAS_ERR_CUDA;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  const cudaError_t e = attn_umma_ok(a, c, false) ? launch_attn_umma_fwd(a, c, st) : launch_attn_fma_fwd(a, c, st);
  return e == cudaSuccess ? VCAS_OK : VCAS_ERR_CUDA;
}

extern "C" int vcas_attn_bwd(vcas_attn aa, const vcas_attn_tensor* d_o, const vcas_attn_tensor* q, const vcas_attn_tensor* k,
                             const vcas_attn_tensor* v, const vcas_attn_tensor* o, const float* lse, const int32_t* starts, int32_t N,
                             int32_t total, const int32_t* alive_in, const int32_t* alive_cnt_in, int32_t skip_dropped_rows,
                             const vcas_attn_tensor* dq, const vcas_attn_tensor* dk, const vcas_attn_tensor* dv, vcas_stream stream) {
  if (aa == nullptr) return VCAS_ERR_BAD_ARG;
  Attn* a = A(aa);
  AttnCall c = {};
  const int rc = begin(a, starts, N, total, alive_in, alive_cnt_in, c);
  if (rc != VCAS_OK) return rc;
  if (N == 0 || total == 0) return VCAS_OK;
  const size_t elem = a->desc.dtype == VCAS_DTYPE_BF16 ? 2 : 4;
  const int D = c.dim;
  if (!good(q, elem) || !good(k, elem) || !good(v, elem) || !good(o, elem) || !good(d_o, elem) ||
      !good_out(dq, total, c.heads_q, D, elem) || !good_out(dk, total, c.heads_kv, D, elem) ||
      !good_out(dv, total, c.heads_kv, D, elem) || lse == nullptr)
    return VCAS_ERR_BAD_ARG;
  c.q = S(q); c.k = S(k); c.v = S(v); c.o = S(o); c.d_o = S(d_o); c.dq = S(dq); c.dk = S(dk); c.dv = S(dv);
  c.lse = const_cast<float*>(lse);
  c.skip_dropped = skip_dropped_rows != 0;
  DeviceScope on(a->device);
  if (!on.ok) return VCAS_ERR_CUDA;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  const cudaError_t e = attn_umma_ok(a, c, true) ? launch_attn_umma_bwd(a, c, st) : launch_attn_fma_bwd(a, c, st);
  return e == cudaSuccess ? VCAS_OK : VCAS_ERR_CUDA;
}

extern "C" int vcas_attn_status(vcas_attn aa, int32_t* status) {
  if (aa == nullptr || status == nullptr) return VCAS_ERR_BAD_ARG;
  Attn* a = A(aa);
  DeviceScope on(a->device);
  if (!on.ok || cudaDeviceSynchronize() != cudaSuccess ||
      cudaMemcpy(status, a->status, sizeof(int32_t), cudaMemcpyDeviceToHost) != cudaSuccess ||
      cudaMemset(a->status, 0, sizeof(int32_t)) != cudaSuccess)
    return VCAS_ERR_CUDA;
  return VCAS_OK;
}

extern "C" int vcas_attn_set_wait_limit(vcas_attn aa, uint64_t limit_ns, int32_t stall_once) {
  if (aa == nullptr || limit_ns == 0) return VCAS_ERR_BAD_ARG;
  A(aa)->wait_limit_ns = limit_ns;
  A(aa)->stall_once = stall_once != 0;
  return VCAS_OK;
}
