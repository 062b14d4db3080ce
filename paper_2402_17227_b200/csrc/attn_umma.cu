// Attention over packed sequences on the tensor cores (bf16, tcgen05): one forward and two backward kernels.
//
// A CTA owns a tile of 128 rows of one head and walks over the tiles of the other side.  One warp loads tiles with TMA, one lane
// issues the products, four (forward) or eight (backward) warps turn scores into probabilities, a row of TMEM being a lane's
// own.  Scores stay in TMEM; P and dS go back there as bf16, over the scores they came from, and are the A operand of the
// product that follows.  tcgen05.mma of one thread run in order, so a tile of scores may be overwritten by the next
// product as soon as the product that reads it is issued.
//   forward    S = Q K^T,  P = exp(S - m),  O += P V; O is rescaled only where the maximum rose by more than 2^8
//   dQ         rows are queries: S, dP = dO V^T, dS = P (dP - delta), dQ += dS K
//   dK, dV     rows are keys:    S^T = K Q^T, dV += P^T dO, dP^T = V dO^T, dK += dS^T Q, over all query heads of the group
// A tile that reaches past its sequence's end holds rows of the next one (or zeros): their scores are masked, and where such rows
// would be summed over they are zeroed in shared memory, so that nothing of them, a NaN included, gets in.
#include "attn.cuh"
#include "umma.cuh"

namespace vcas {
namespace {

constexpr int CHUNK = 128 * 64 * 2;      // 128 rows of 64 bf16: one 128-byte swizzled block

// ------------------------------------------------------------------------------- TMEM and operands
// 32 lanes x 64 columns
__device__ __forceinline__ void tmem_ld64(uint32_t taddr, uint32_t (&v)[64]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x64.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17,"
      " %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32, %33, %34, %35, %36, %37, %38, %39, %40, %41,"
      " %42, %43, %44, %45, %46, %47, %48, %49, %50, %51, %52, %53, %54, %55, %56, %57, %58, %59, %60, %61, %62, %63}, [%64];\n\t"
      "tcgen05.wait::ld.sync.aligned;"
      : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]), "=r"(v[9]),
        "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15]), "=r"(v[16]), "=r"(v[17]), "=r"(v[18]),
        "=r"(v[19]), "=r"(v[20]), "=r"(v[21]), "=r"(v[22]), "=r"(v[23]), "=r"(v[24]), "=r"(v[25]), "=r"(v[26]), "=r"(v[27]),
        "=r"(v[28]), "=r"(v[29]), "=r"(v[30]), "=r"(v[31]), "=r"(v[32]), "=r"(v[33]), "=r"(v[34]), "=r"(v[35]), "=r"(v[36]),
        "=r"(v[37]), "=r"(v[38]), "=r"(v[39]), "=r"(v[40]), "=r"(v[41]), "=r"(v[42]), "=r"(v[43]), "=r"(v[44]), "=r"(v[45]),
        "=r"(v[46]), "=r"(v[47]), "=r"(v[48]), "=r"(v[49]), "=r"(v[50]), "=r"(v[51]), "=r"(v[52]), "=r"(v[53]), "=r"(v[54]),
        "=r"(v[55]), "=r"(v[56]), "=r"(v[57]), "=r"(v[58]), "=r"(v[59]), "=r"(v[60]), "=r"(v[61]), "=r"(v[62]), "=r"(v[63])
      : "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_st32(uint32_t taddr, const uint32_t (&v)[32]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17,"
      " %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};"
      ::"r"(taddr), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]),
        "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]), "r"(v[16]), "r"(v[17]), "r"(v[18]), "r"(v[19]),
        "r"(v[20]), "r"(v[21]), "r"(v[22]), "r"(v[23]), "r"(v[24]), "r"(v[25]), "r"(v[26]), "r"(v[27]), "r"(v[28]), "r"(v[29]),
        "r"(v[30]), "r"(v[31]) : "memory");
}
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// D[tmem] (+)= A[tmem] B[smem]
__device__ __forceinline__ void umma_bf16_ts(uint32_t tmem_d, uint32_t tmem_a, uint64_t desc_b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
      ::"r"(tmem_d), "r"(tmem_a), "l"(desc_b), "r"(idesc), "r"(accumulate) : "memory");
}
// A tile of 128 rows is CHUNK bytes for each 64 columns.  Its rows as the summed-over side of a product: 64-wide chunks CHUNK apart.
__device__ __forceinline__ uint64_t desc_rows(uint32_t saddr) {
  return (uint64_t)((saddr & 0x3ffffu) >> 4) | ((uint64_t)(CHUNK >> 4) << 16) | ((uint64_t)(1024 >> 4) << 32) | (1ull << 46) | (2ull << 61);
}
// D [128 x 128] = A B^T, both tiles of 128 rows, summed over their 64 * DC columns
template <int DC>
__device__ __forceinline__ void product_tiles(uint32_t d, uint32_t a, uint32_t b) {
  constexpr uint32_t idesc = make_idesc(128, false, false);
#pragma unroll
  for (int c = 0; c < DC; ++c) {
    const uint64_t da = desc_kmajor(a + c * CHUNK), db = desc_kmajor(b + c * CHUNK);
#pragma unroll
    for (int k = 0; k < 4; ++k) umma_bf16(d, da + (uint64_t)(k * 2), db + (uint64_t)(k * 2), idesc, (c | k) != 0 ? 1u : 0u);
  }
}
// D [128 x 64 DC] (+)= A B, A [128 x 128] bf16 in TMEM (its upper 64 columns `gap` TMEM columns behind the lower), B a tile
template <int DC>
__device__ __forceinline__ void product_rows(uint32_t d, uint32_t a, int gap, uint32_t b, bool add) {
  constexpr uint32_t idesc = make_idesc(64 * DC, false, true);
  const uint64_t db = desc_rows(b);
#pragma unroll
  for (int k = 0; k < 8; ++k)
    umma_bf16_ts(d, a + (uint32_t)((k & 3) * 8 + (k >> 2) * gap), db + (uint64_t)(k * (16 * 128 >> 4)), idesc, add || k != 0 ? 1u : 0u);
}
// rows have .. 127 of a tile become 0, by one warp; the products after it see them
template <int DC>
__device__ __forceinline__ void zero_rows(uint8_t* tile, int have, int lane) {
  for (int i = have * 8 + lane; i < 128 * 8; i += 32)
#pragma unroll
    for (int c = 0; c < DC; ++c) *reinterpret_cast<uint4*>(tile + c * CHUNK + i * 16) = make_uint4(0, 0, 0, 0);
}
template <int DC>
__device__ __forceinline__ void load_tile(uint8_t* dst, const CUtensorMap* map, int head, int token, uint64_t* bar) {
#pragma unroll
  for (int c = 0; c < DC; ++c) tma_load_3d(dst + c * CHUNK, map, 64 * c, head, token, bar);
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  const __nv_bfloat162 t = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&t);
}
// this lane's row of a [128 x 64 DC] accumulator, times f, to a row of a tensor
template <int DC>
__device__ __forceinline__ void store_row(uint32_t taddr, __nv_bfloat16* row, int dim, bool in, float f) {
#pragma unroll
  for (int c = 0; c < 2 * DC; ++c) {
    uint32_t v[32];
    tmem_ld32(taddr + c * 32, v);
#pragma unroll
    for (int e = 0; e < 32; e += 8) {
      const int d = c * 32 + e;
      if (in && d < dim) {
        uint32_t o[4];
#pragma unroll
        for (int h = 0; h < 4; ++h) o[h] = pack_bf16(__uint_as_float(v[e + 2 * h]) * f, __uint_as_float(v[e + 2 * h + 1]) * f);
        *reinterpret_cast<uint4*>(row + d) = make_uint4(o[0], o[1], o[2], o[3]);
      }
    }
  }
}

// ----------------------------------------------------------------------------------------- the CTA
constexpr int MAX_STAGES = 4;
struct Shared {
  uint64_t full[MAX_STAGES], empty[MAX_STAGES], own, scores[2], dscores, ready[2], done, drain;
  uint32_t tmem;
  int abort_flag;                        // mbar_wait finds the limit 20 bytes behind it
  int first, len, t0, any;
  unsigned long long limit;
};
static_assert(offsetof(Shared, limit) == offsetof(Shared, abort_flag) + 20, "see mbar_wait");

struct UmmaCall {
  AttnCall c;
  unsigned long long wait_limit_ns;
  int stall_once;
};

// A whole warp waits and goes on, or gives up, together: what follows are instructions of all its lanes.
__device__ __forceinline__ bool warp_wait(uint64_t* bar, uint32_t parity, volatile int* ab, int32_t* status) {
  return __all_sync(0xffffffffu, mbar_wait(bar, parity, ab, status));
}

// Finds the CTA's tile, sets the barriers up and takes TMEM; false where there is no tile.
__device__ __forceinline__ bool begin(Shared& s, const UmmaCall& P, int heads, bool last_first, int stages, uint32_t readers, uint32_t columns) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (warp == 0) {
    int first = 0, len = 0, place = 0;
    const bool any = find_tile(P.c.seqs, (int)(blockIdx.x / (unsigned)heads), 128, lane, first, len, place);
    if (lane == 0) {
      s.first = first; s.len = len; s.any = any;
      s.t0 = (last_first ? (len + 127) / 128 - 1 - place : place) * 128;
    }
  } else if (warp == 1 && lane == 0) {
    for (int i = 0; i < stages; ++i) { mbar_init(&s.full[i], 1); mbar_init(&s.empty[i], 1); }
    mbar_init(&s.own, 1);
    mbar_init(&s.scores[0], 1);
    mbar_init(&s.scores[1], 1);
    mbar_init(&s.dscores, 1);
    mbar_init(&s.ready[0], readers);
    mbar_init(&s.ready[1], readers);
    mbar_init(&s.done, 1);
    mbar_init(&s.drain, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    s.abort_flag = 0;
    s.limit = P.wait_limit_ns;
  }
  __syncthreads();
  if (!s.any) return false;
  if (warp == 2) tmem_alloc(&s.tmem, columns);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  return true;
}
__device__ __forceinline__ void end(Shared& s, uint32_t columns) {
  tc_fence_before();
  __syncthreads();
  if ((threadIdx.x >> 5) == 2) {
    tc_fence_after();
    tmem_dealloc(s.tmem, columns);
  }
}
// A ring position
struct Ring {
  int stage = 0;
  uint32_t phase = 0;
  __device__ __forceinline__ void next(int stages) {
    if (++stage == stages) { stage = 0; phase ^= 1u; }
  }
};

// ------------------------------------------------------------------------------------------ forward
// Two CTAs an SM, each with 128 query rows: while one turns scores into probabilities the other's products run.  K and V tiles take
// turns in the ring; a score tile takes 128 columns of TMEM and O another 64 DC.
template <int DC> constexpr int FWD_STAGES = DC == 1 ? 4 : 2;
constexpr int FWD_THREADS = 192;

template <int DC>
__global__ void __launch_bounds__(FWD_THREADS, 2)
attn_fwd_kernel(const __grid_constant__ CUtensorMap mq, const __grid_constant__ CUtensorMap mk, const __grid_constant__ CUtensorMap mv,
                const __grid_constant__ UmmaCall P) {
  constexpr int STAGES = FWD_STAGES<DC>, TILE_BYTES = DC * CHUNK;
  extern __shared__ uint8_t raw[];
  __shared__ Shared s;
  uint8_t* smem = reinterpret_cast<uint8_t*>(((uintptr_t)raw + 1023) & ~(uintptr_t)1023);
  uint8_t *sq = smem, *ring = smem + TILE_BYTES;
  const AttnCall& C = P.c;
  if (!begin(s, P, C.heads_q, C.causal, STAGES, 128, 256)) return;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int head = (int)(blockIdx.x % (unsigned)C.heads_q), first = s.first, len = s.len, t0 = s.t0;
  const int end_col = C.causal ? min(len, t0 + 128) : len, tiles = (end_col + 127) / 128;
  const uint32_t ts = s.tmem, to = s.tmem + 128;
  volatile int* ab = &s.abort_flag;
  int32_t* status = C.seqs.status;

  if (warp == 5) {
    if (elect_one()) {
      mbar_expect_tx(&s.own, TILE_BYTES);
      load_tile<DC>(sq, &mq, head, first + t0, &s.own);
      Ring r;
      uint32_t filled = 0;
      const int kv = head / C.group;
      bool ok = true;
      for (int i = 0; i < 2 * tiles && ok; ++i) {
        ok = mbar_wait(&s.empty[r.stage], r.phase ^ 1u, ab, status);
        if (!ok) break;
        if (P.stall_once && blockIdx.x == 0 && i == 0) { r.next(STAGES); continue; }
        mbar_expect_tx(&s.full[r.stage], TILE_BYTES);
        load_tile<DC>(ring + r.stage * TILE_BYTES, (i & 1) ? &mv : &mk, kv, first + (i >> 1) * 128, &s.full[r.stage]);
        r.next(STAGES);
        ++filled;
      }
      if (*ab) {
        mbar_wait(&s.own, 0, ab, status);
        drain_loads(s.full, STAGES, r.stage, r.phase, filled, ab, status);
      }
    }
  } else if (warp == 4) {
    const bool leader = elect_one();
    bool ok = warp_wait(&s.own, 0, ab, status);
    Ring r;
    for (int j = 0; j < tiles && ok; ++j) {
      ok = warp_wait(&s.full[r.stage], r.phase, ab, status);
      if (!ok) break;
      tc_fence_after();
      if (leader) {
        product_tiles<DC>(ts, smem_u32(sq), smem_u32(ring + r.stage * TILE_BYTES));
        umma_commit(&s.empty[r.stage]);
        umma_commit(&s.scores[0]);
      }
      r.next(STAGES);
      ok = warp_wait(&s.full[r.stage], r.phase, ab, status);
      if (!ok) break;
      if (len - j * 128 < 128) {
        zero_rows<DC>(ring + r.stage * TILE_BYTES, len - j * 128, lane);
        fence_async_smem();
        __syncwarp();
      }
      ok = warp_wait(&s.ready[0], j & 1, ab, status);
      if (!ok) break;
      tc_fence_after();
      if (leader) {
        product_rows<DC>(to, ts, 32, smem_u32(ring + r.stage * TILE_BYTES), j != 0);
        umma_commit(&s.empty[r.stage]);
      }
      r.next(STAGES);
    }
    if (leader) {
      if (ok) umma_commit(&s.done);
      else drain_products(&s.drain, ab, status);
    }
  } else {
    const int row = t0 + threadIdx.x;                // in the sequence
    const uint32_t lanes = (uint32_t)(warp * 32) << 16;
    const float c = C.scale * ATTN_LOG2E, none = __int_as_float(0xff800000);
    float m = none, l = 0.f;
    bool ok = true;
    for (int j = 0; j < tiles; ++j) {
      ok = warp_wait(&s.scores[0], j & 1, ab, status);
      if (!ok) break;
      tc_fence_after();
      uint32_t a[64], b[64];
      tmem_ld64(ts + lanes, a);
      tmem_ld64(ts + lanes + 64, b);
      // columns this row sees in the tile
      const int see = min(128, (C.causal ? min(len, row + 1) : len) - j * 128);
      if (__any_sync(0xffffffffu, see < 128)) {
#pragma unroll
        for (int i = 0; i < 64; ++i) {
          a[i] = i < see ? a[i] : 0xff800000u;
          b[i] = i + 64 < see ? b[i] : 0xff800000u;
        }
      }
      float t[4] = {none, none, none, none};
#pragma unroll
      for (int i = 0; i < 64; ++i) t[i & 3] = fmaxf(t[i & 3], fmaxf(__uint_as_float(a[i]), __uint_as_float(b[i])));
      const float top = fmaxf(fmaxf(t[0], t[1]), fmaxf(t[2], t[3]));
      if (j == 0) {
        m = top;
      } else {
        // the sums are relative to m; it follows the maximum once that has risen far enough for P to lose range
        const bool rise = (top - m) * c > 8.0f;
        if (__any_sync(0xffffffffu, rise)) {
          const float f = rise ? attn_exp2((m - top) * c) : 1.0f;
          m = rise ? top : m;
          l *= f;
#pragma unroll
          for (int q = 0; q < 2 * DC; ++q) {
            uint32_t o[32];
            tmem_ld32(to + lanes + q * 32, o);
#pragma unroll
            for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
            tmem_st32(to + lanes + q * 32, o);
          }
        }
      }
      const float ref = m == none ? 0.f : m;
      const uint64_t c2 = pack2(c, c), n2 = pack2(-ref * c, -ref * c);
      uint64_t l2[2] = {0, 0};
      auto half = [&](const uint32_t (&x)[64], uint32_t at) {
        uint32_t o[32];
#pragma unroll
        for (int i = 0; i < 32; ++i) {
          float e0, e1;
          unpack2(fma2(pack2(__uint_as_float(x[2 * i]), __uint_as_float(x[2 * i + 1])), c2, n2), e0, e1);
          e0 = attn_exp2(e0);
          e1 = attn_exp2(e1);
          l2[i & 1] = add2(l2[i & 1], pack2(e0, e1));
          o[i] = pack_bf16(e0, e1);
        }
        tmem_st32(at, o);
      };
      half(a, ts + lanes);
      half(b, ts + lanes + 32);
      float x0, x1;
      unpack2(add2(l2[0], l2[1]), x0, x1);
      l += x0 + x1;
      tmem_wait_st();
      tc_fence_before();
      mbar_arrive(&s.ready[0]);
    }
    ok = ok && warp_wait(&s.done, 0, ab, status);
    if (ok) {
      tc_fence_after();
      __nv_bfloat16* o = (__nv_bfloat16*)const_cast<void*>(C.o.p) + (int64_t)(first + row) * C.o.token + (int64_t)head * C.o.head;
      store_row<DC>(to + lanes, o, C.dim, row < len, 1.0f / l);
      if (row < len) C.lse[(int64_t)head * C.seqs.total + first + row] = (m * c) * ATTN_LN2 + logf(l);
    }
  }
  end(s, 256);
}

// ------------------------------------------------------------------------------------------ backward
constexpr int BWD_THREADS = 320;         // eight warps for the scores: 32 rows and 64 columns each

// Rows are queries.  TMEM: two score tiles in turn (dS replaces its own), dP, dQ.
template <int DC>
__global__ void __launch_bounds__(BWD_THREADS, 1)
attn_dq_kernel(const __grid_constant__ CUtensorMap mq, const __grid_constant__ CUtensorMap mdo, const __grid_constant__ CUtensorMap mk,
               const __grid_constant__ CUtensorMap mv, const __grid_constant__ UmmaCall P) {
  constexpr int STAGES = 2, TILE_BYTES = DC * CHUNK;
  extern __shared__ uint8_t raw[];
  __shared__ Shared s;
  uint8_t* smem = reinterpret_cast<uint8_t*>(((uintptr_t)raw + 1023) & ~(uintptr_t)1023);
  uint8_t *sq = smem, *sdo = smem + TILE_BYTES, *ring = smem + 2 * TILE_BYTES;      // a stage: K, V
  const AttnCall& C = P.c;
  if (!begin(s, P, C.heads_q, C.causal, STAGES, 256, 512)) return;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int head = (int)(blockIdx.x % (unsigned)C.heads_q), first = s.first, len = s.len, t0 = s.t0;
  const int end_col = C.causal ? min(len, t0 + 128) : len, tiles = (end_col + 127) / 128;
  const uint32_t ts = s.tmem, tdp = s.tmem + 256, tdq = s.tmem + 384;
  volatile int* ab = &s.abort_flag;
  int32_t* status = C.seqs.status;

  if (warp == 9) {
    if (elect_one()) {
      mbar_expect_tx(&s.own, 2 * TILE_BYTES);
      load_tile<DC>(sq, &mq, head, first + t0, &s.own);
      load_tile<DC>(sdo, &mdo, head, first + t0, &s.own);
      Ring r;
      uint32_t filled = 0;
      const int kv = head / C.group;
      for (int j = 0; j < tiles; ++j) {
        if (!mbar_wait(&s.empty[r.stage], r.phase ^ 1u, ab, status)) break;
        if (P.stall_once && blockIdx.x == 0 && j == 0) { r.next(STAGES); continue; }
        mbar_expect_tx(&s.full[r.stage], 2 * TILE_BYTES);
        uint8_t* to = ring + r.stage * 2 * TILE_BYTES;
        load_tile<DC>(to, &mk, kv, first + j * 128, &s.full[r.stage]);
        load_tile<DC>(to + TILE_BYTES, &mv, kv, first + j * 128, &s.full[r.stage]);
        r.next(STAGES);
        ++filled;
      }
      if (*ab) {
        mbar_wait(&s.own, 0, ab, status);
        drain_loads(s.full, STAGES, r.stage, r.phase, filled, ab, status);
      }
    }
  } else if (warp == 8) {
    const bool leader = elect_one();
    bool ok = warp_wait(&s.own, 0, ab, status);
    Ring load, use;
    auto scores = [&](int j) {           // waits for tile j and multiplies it with Q
      ok = warp_wait(&s.full[load.stage], load.phase, ab, status);
      if (!ok) return;
      uint8_t* at = ring + load.stage * 2 * TILE_BYTES;
      if (len - j * 128 < 128) {
        zero_rows<DC>(at, len - j * 128, lane);
        zero_rows<DC>(at + TILE_BYTES, len - j * 128, lane);
        fence_async_smem();
        __syncwarp();
      }
      tc_fence_after();
      if (leader) {
        product_tiles<DC>(ts + (j & 1) * 128, smem_u32(sq), smem_u32(at));
        umma_commit(&s.scores[j & 1]);
      }
    };
    auto dscores = [&]() {
      if (leader) {
        product_tiles<DC>(tdp, smem_u32(sdo), smem_u32(ring + load.stage * 2 * TILE_BYTES + TILE_BYTES));
        umma_commit(&s.dscores);
      }
    };
    if (ok) scores(0);
    if (ok) dscores();
    for (int j = 0; j < tiles && ok; ++j) {
      if (j + 1 < tiles) {
        load.next(STAGES);
        scores(j + 1);
        if (!ok) break;
      }
      ok = warp_wait(&s.ready[0], j & 1, ab, status);
      if (!ok) break;
      tc_fence_after();
      if (j + 1 < tiles) dscores();
      if (leader) {
        product_rows<DC>(tdq, ts + (j & 1) * 128, 64, smem_u32(ring + use.stage * 2 * TILE_BYTES), j != 0);
        umma_commit(&s.empty[use.stage]);
      }
      use.next(STAGES);
    }
    if (leader) {
      if (ok) umma_commit(&s.done);
      else drain_products(&s.drain, ab, status);
    }
  } else {
    const int row = t0 + (warp & 3) * 32 + lane, part = warp >> 2;       // columns part * 64 ..
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const float c = C.scale * ATTN_LOG2E;
    float lse = 0.f, delta = 0.f;
    if (row < len) {
      const int64_t at = (int64_t)head * C.seqs.total + first + row;
      lse = C.lse[at] * ATTN_LOG2E;
      delta = C.delta[at];
    }
    const uint64_t c2 = pack2(c, c), n2 = pack2(-lse, -lse), d2 = pack2(-delta, -delta);
    bool ok = true;
    for (int j = 0; j < tiles; ++j) {
      ok = warp_wait(&s.scores[j & 1], (j >> 1) & 1, ab, status);
      if (!ok) break;
      tc_fence_after();
      const uint32_t at = ts + lanes + (j & 1) * 128 + part * 64;
      uint32_t a[64];
      tmem_ld64(at, a);
#pragma unroll
      for (int i = 0; i < 32; ++i) {
        float e0, e1;
        unpack2(fma2(pack2(__uint_as_float(a[2 * i]), __uint_as_float(a[2 * i + 1])), c2, n2), e0, e1);
        a[2 * i] = __float_as_uint(attn_exp2(e0));
        a[2 * i + 1] = __float_as_uint(attn_exp2(e1));
      }
      ok = warp_wait(&s.dscores, j & 1, ab, status);
      if (!ok) break;
      tc_fence_after();
      uint32_t o[32];
      const int see = min(128, (C.causal ? min(len, row + 1) : len) - j * 128) - part * 64;
      const bool whole = !__any_sync(0xffffffffu, see < 64);
      {
        uint32_t b[64];
        tmem_ld64(tdp + lanes + part * 64, b);
#pragma unroll
        for (int i = 0; i < 32; ++i) {
          float s0, s1;
          unpack2(mul2(pack2(__uint_as_float(a[2 * i]), __uint_as_float(a[2 * i + 1])),
                       add2(pack2(__uint_as_float(b[2 * i]), __uint_as_float(b[2 * i + 1])), d2)), s0, s1);
          if (!whole) {
            s0 = 2 * i < see ? s0 : 0.f;
            s1 = 2 * i + 1 < see ? s1 : 0.f;
          }
          o[i] = pack_bf16(s0, s1);
        }
      }
      tmem_st32(at, o);
      tmem_wait_st();
      tc_fence_before();
      mbar_arrive(&s.ready[0]);
    }
    ok = ok && warp_wait(&s.done, 0, ab, status);
    if (ok && part < DC) {
      // each half of the warps stores 64 columns (all of them where there are no more)
      tc_fence_after();
      __nv_bfloat16* o = (__nv_bfloat16*)const_cast<void*>(C.dq.p) + (int64_t)(first + row) * C.dq.token + (int64_t)head * C.dq.head;
      store_row<1>(tdq + lanes + part * 64, o + part * 64, C.dim - part * 64, row < len, C.scale);
    }
  }
  end(s, 512);
}

// Rows are keys.  TMEM: S^T (P^T replaces it), dP^T (dS^T replaces it), dV, dK.  The products of tile i + 1's scores are issued
// between those of tile i: S^T(i + 1) behind dV(i), dP^T(i + 1) behind dK(i), so that the tensor pipe works while the other
// warps do exponentials.
template <int DC>
__global__ void __launch_bounds__(BWD_THREADS, 1)
attn_dkv_kernel(const __grid_constant__ CUtensorMap mq, const __grid_constant__ CUtensorMap mdo, const __grid_constant__ CUtensorMap mk,
                const __grid_constant__ CUtensorMap mv, const __grid_constant__ UmmaCall P) {
  constexpr int STAGES = 2, TILE_BYTES = DC * CHUNK;
  extern __shared__ uint8_t raw[];
  __shared__ Shared s;
  __shared__ __align__(16) float s_rows[8][2][128];      // each warp's own: lse and delta of its 64 queries, two items
  uint8_t* smem = reinterpret_cast<uint8_t*>(((uintptr_t)raw + 1023) & ~(uintptr_t)1023);
  uint8_t *sk = smem, *sv = smem + TILE_BYTES, *ring = smem + 2 * TILE_BYTES;       // a stage: Q, dO
  const AttnCall& C = P.c;
  if (!begin(s, P, C.heads_kv, false, STAGES, 256, 512)) return;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int kv = (int)(blockIdx.x % (unsigned)C.heads_kv), first = s.first, len = s.len, t0 = s.t0;
  const int q0 = C.causal ? t0 / 128 : 0, per_head = (len + 127) / 128 - q0, items = per_head * C.group;
  const uint32_t ts = s.tmem, tdp = s.tmem + 128, tdv = s.tmem + 256, tdk = s.tmem + 384;
  volatile int* ab = &s.abort_flag;
  int32_t* status = C.seqs.status;
  auto head_of = [&](int i) { return kv * C.group + i / per_head; };
  auto row_of = [&](int i) { return (q0 + i % per_head) * 128; };          // first query of item i

  if (warp == 9) {
    if (elect_one()) {
      mbar_expect_tx(&s.own, 2 * TILE_BYTES);
      load_tile<DC>(sk, &mk, kv, first + t0, &s.own);
      load_tile<DC>(sv, &mv, kv, first + t0, &s.own);
      Ring r;
      uint32_t filled = 0;
      for (int i = 0; i < items; ++i) {
        if (!mbar_wait(&s.empty[r.stage], r.phase ^ 1u, ab, status)) break;
        if (P.stall_once && blockIdx.x == 0 && i == 0) { r.next(STAGES); continue; }
        mbar_expect_tx(&s.full[r.stage], 2 * TILE_BYTES);
        uint8_t* to = ring + r.stage * 2 * TILE_BYTES;
        load_tile<DC>(to, &mq, head_of(i), first + row_of(i), &s.full[r.stage]);
        load_tile<DC>(to + TILE_BYTES, &mdo, head_of(i), first + row_of(i), &s.full[r.stage]);
        r.next(STAGES);
        ++filled;
      }
      if (*ab) {
        mbar_wait(&s.own, 0, ab, status);
        drain_loads(s.full, STAGES, r.stage, r.phase, filled, ab, status);
      }
    }
  } else if (warp == 8) {
    const bool leader = elect_one();
    bool ok = warp_wait(&s.own, 0, ab, status);
    Ring load, use;
    auto scores = [&](int i) {
      ok = warp_wait(&s.full[load.stage], load.phase, ab, status);
      if (!ok) return;
      uint8_t* at = ring + load.stage * 2 * TILE_BYTES;
      const int have = len - row_of(i);
      if (have < 128) {
        zero_rows<DC>(at, have, lane);
        zero_rows<DC>(at + TILE_BYTES, have, lane);
        fence_async_smem();
        __syncwarp();
      }
      tc_fence_after();
      if (leader) {
        product_tiles<DC>(ts, smem_u32(sk), smem_u32(at));
        umma_commit(&s.scores[0]);
      }
    };
    auto dscores = [&]() {
      if (leader) {
        product_tiles<DC>(tdp, smem_u32(sv), smem_u32(ring + load.stage * 2 * TILE_BYTES + TILE_BYTES));
        umma_commit(&s.dscores);
      }
    };
    if (ok) scores(0);
    if (ok) dscores();
    for (int i = 0; i < items && ok; ++i) {
      const uint32_t at = smem_u32(ring + use.stage * 2 * TILE_BYTES);
      ok = warp_wait(&s.ready[0], i & 1, ab, status);
      if (!ok) break;
      tc_fence_after();
      if (leader) product_rows<DC>(tdv, ts, 64, at + TILE_BYTES, i != 0);
      if (i + 1 < items) {
        load.next(STAGES);
        scores(i + 1);
        if (!ok) break;
      }
      ok = warp_wait(&s.ready[1], i & 1, ab, status);
      if (!ok) break;
      tc_fence_after();
      if (leader) {
        product_rows<DC>(tdk, tdp, 64, at, i != 0);
        umma_commit(&s.empty[use.stage]);
      }
      use.next(STAGES);
      if (i + 1 < items) dscores();
    }
    if (leader) {
      if (ok) umma_commit(&s.done);
      else drain_products(&s.drain, ab, status);
    }
  } else {
    const int row = t0 + (warp & 3) * 32 + lane, part = warp >> 2;
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const float c = C.scale * ATTN_LOG2E;
    const uint64_t c2 = pack2(c, c);
    // a lane's two queries of an item: their lse (in units of log 2) and delta, negative
    auto fetch = [&](int i) -> float4 {
      const int t = row_of(i) + part * 64 + 2 * lane;
      const int64_t at = (int64_t)head_of(i) * C.seqs.total + first + t;
      float4 f = make_float4(0.f, 0.f, 0.f, 0.f);
      if (t < len) { f.x = -C.lse[at] * ATTN_LOG2E; f.z = -C.delta[at]; }
      if (t + 1 < len) { f.y = -C.lse[at + 1] * ATTN_LOG2E; f.w = -C.delta[at + 1]; }
      return f;
    };
    auto keep = [&](int i, float4 f) {
      float* at = s_rows[warp][i & 1] + 2 * lane;
      *reinterpret_cast<float2*>(at) = make_float2(f.x, f.y);
      *reinterpret_cast<float2*>(at + 64) = make_float2(f.z, f.w);
      __syncwarp();
    };
    keep(0, fetch(0));
    bool ok = true;
    for (int i = 0; i < items; ++i) {
      const float4 ahead = i + 1 < items ? fetch(i + 1) : make_float4(0.f, 0.f, 0.f, 0.f);
      ok = warp_wait(&s.scores[0], i & 1, ab, status);
      if (!ok) break;
      tc_fence_after();
      const int base = row_of(i) + part * 64;        // first query of this warp's columns
      const bool cut = len - base < 64 || (C.causal && base < t0 + 128);
      const int lo = C.causal ? row - base : 0, hi = len - base;         // the columns that look at this key
      uint32_t a[64];
      tmem_ld64(ts + lanes + part * 64, a);
      uint32_t o[32];
#pragma unroll
      for (int e = 0; e < 32; e += 2) {
        const float4 n = *reinterpret_cast<const float4*>(&s_rows[warp][i & 1][2 * e]);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int x = 2 * (e + h);
          float e0, e1;
          unpack2(fma2(pack2(__uint_as_float(a[x]), __uint_as_float(a[x + 1])), c2, h == 0 ? pack2(n.x, n.y) : pack2(n.z, n.w)), e0, e1);
          e0 = attn_exp2(e0);
          e1 = attn_exp2(e1);
          if (cut) {
            e0 = x >= lo && x < hi ? e0 : 0.f;
            e1 = x + 1 >= lo && x + 1 < hi ? e1 : 0.f;
          }
          a[x] = __float_as_uint(e0);
          a[x + 1] = __float_as_uint(e1);
          o[e + h] = pack_bf16(e0, e1);
        }
      }
      tmem_st32(ts + lanes + part * 64, o);
      tmem_wait_st();
      tc_fence_before();
      mbar_arrive(&s.ready[0]);
      ok = warp_wait(&s.dscores, i & 1, ab, status);
      if (!ok) break;
      tc_fence_after();
      {
        uint32_t b[64];
        tmem_ld64(tdp + lanes + part * 64, b);
#pragma unroll
        for (int e = 0; e < 32; e += 2) {
          const float4 n = *reinterpret_cast<const float4*>(&s_rows[warp][i & 1][64 + 2 * e]);
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const int x = 2 * (e + h);
            float s0, s1;
            unpack2(mul2(pack2(__uint_as_float(a[x]), __uint_as_float(a[x + 1])),
                         add2(pack2(__uint_as_float(b[x]), __uint_as_float(b[x + 1])), h == 0 ? pack2(n.x, n.y) : pack2(n.z, n.w))), s0, s1);
            o[e + h] = pack_bf16(s0, s1);
          }
        }
      }
      tmem_st32(tdp + lanes + part * 64, o);
      tmem_wait_st();
      tc_fence_before();
      mbar_arrive(&s.ready[1]);
      if (i + 1 < items) keep(i + 1, ahead);
    }
    ok = ok && warp_wait(&s.done, 0, ab, status);
    if (ok) {
      // one half of the warps stores dV, the other dK
      tc_fence_after();
      const Strided& x = part == 0 ? C.dv : C.dk;
      __nv_bfloat16* o = (__nv_bfloat16*)const_cast<void*>(x.p) + (int64_t)(first + row) * x.token + (int64_t)kv * x.head;
      store_row<DC>((part == 0 ? tdv : tdk) + lanes, o, C.dim, row < len, part == 0 ? 1.0f : C.scale);
    }
  }
  end(s, 512);
}

// --------------------------------------------------------------------------------------------- host
// [total, heads, dim] with a box of 64 columns of one head of 128 tokens
bool attn_map(CUtensorMap* m, const Strided& x, int heads, int dim, int total) {
  const uint64_t dims[3] = {(uint64_t)dim, (uint64_t)heads, (uint64_t)total};
  // a stride along an extent of one is never used, but has to be a valid one
  const uint64_t strides[2] = {heads > 1 ? (uint64_t)x.head * 2 : 16, total > 1 ? (uint64_t)x.token * 2 : 16};
  const uint32_t box[3] = {64, 1, 128};
  return make_map(m, x.p, 3, dims, strides, box);
}
bool addressable(const Strided& x, int heads, int total) {
  return ((uintptr_t)x.p & 15) == 0 && (total == 1 || (x.token % 8 == 0 && x.token > 0)) && (heads == 1 || (x.head % 8 == 0 && x.head > 0)) &&
         x.token < (1ll << 36) && x.head < (1ll << 36);
}
template <typename K, typename... M>
cudaError_t run(K kernel, int tiles_of_smem, int threads, long grid, const Attn* a, const AttnCall& c, int dc, cudaStream_t st, const M&... maps) {
  if (grid > 0x7fffffffl) return cudaErrorInvalidValue;
  const int smem = tiles_of_smem * dc * CHUNK + 1024;
  const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (e != cudaSuccess) return e;
  const UmmaCall P = {c, a->wait_limit_ns, a->stall_once};
  kernel<<<(unsigned)grid, threads, smem, st>>>(maps..., P);
  return cudaGetLastError();
}

}  // namespace

bool attn_umma_ok(const Attn* a, const AttnCall& c, bool backward) {
  const int total = c.seqs.total;
  if (!a->tensor_ok || !addressable(c.q, c.heads_q, total) || !addressable(c.k, c.heads_kv, total) || !addressable(c.v, c.heads_kv, total) ||
      !addressable(c.o, c.heads_q, total))
    return false;
  return !backward || (addressable(c.d_o, c.heads_q, total) && addressable(c.dq, c.heads_q, total) && addressable(c.dk, c.heads_kv, total) &&
                       addressable(c.dv, c.heads_kv, total));
}

cudaError_t launch_attn_umma_fwd(const Attn* a, const AttnCall& c, cudaStream_t st) {
  const int total = c.seqs.total;
  CUtensorMap mq, mk, mv;
  if (!attn_map(&mq, c.q, c.heads_q, c.dim, total) || !attn_map(&mk, c.k, c.heads_kv, c.dim, total) ||
      !attn_map(&mv, c.v, c.heads_kv, c.dim, total))
    return cudaErrorInvalidValue;
  const long grid = tile_bound(total, c.seqs.N, 128) * c.heads_q;
  return c.dim <= 64 ? run(attn_fwd_kernel<1>, 1 + FWD_STAGES<1>, FWD_THREADS, grid, a, c, 1, st, mq, mk, mv)
                     : run(attn_fwd_kernel<2>, 1 + FWD_STAGES<2>, FWD_THREADS, grid, a, c, 2, st, mq, mk, mv);
}

cudaError_t launch_attn_umma_bwd(const Attn* a, const AttnCall& c, cudaStream_t st) {
  const int total = c.seqs.total;
  CUtensorMap mq, mdo, mk, mv;
  if (!attn_map(&mq, c.q, c.heads_q, c.dim, total) || !attn_map(&mdo, c.d_o, c.heads_q, c.dim, total) ||
      !attn_map(&mk, c.k, c.heads_kv, c.dim, total) || !attn_map(&mv, c.v, c.heads_kv, c.dim, total))
    return cudaErrorInvalidValue;
  const long tiles = tile_bound(total, c.seqs.N, 128);
  const int dc = c.dim <= 64 ? 1 : 2;
  const cudaError_t e = dc == 1 ? run(attn_dq_kernel<1>, 6, BWD_THREADS, tiles * c.heads_q, a, c, dc, st, mq, mdo, mk, mv)
                                : run(attn_dq_kernel<2>, 6, BWD_THREADS, tiles * c.heads_q, a, c, dc, st, mq, mdo, mk, mv);
  if (e != cudaSuccess) return e;
  return dc == 1 ? run(attn_dkv_kernel<1>, 6, BWD_THREADS, tiles * c.heads_kv, a, c, dc, st, mq, mdo, mk, mv)
                 : run(attn_dkv_kernel<2>, 6, BWD_THREADS, tiles * c.heads_kv, a, c, dc, st, mq, mdo, mk, mv);
}

}  // namespace vcas
