// Attention over packed sequences on the tensor cores (bf16, tcgen05): one forward and two backward kernels.
//
// A CTA stays for as long as there are tiles of 128 rows of one head to be had, and walks each against the tiles of the other
// side.  One warp takes tiles from a counter and loads with TMA, ahead of the others and across tiles; one lane of another (in the forward
// of two heads, of one for each) issues the products; four or eight warps turn scores into probabilities, a row of TMEM being a lane's
// own.  Scores stay in TMEM; P goes back there as bf16 over S, dS over dP, as the A operand of the product that follows.
// tcgen05.mma of one thread run in order, so a tile of scores may be overwritten by the next product as soon as the product that
// reads it is issued.
//   forward    S = Q K^T,  P = exp(S - m),  O += P V; O is rescaled only where the maximum has risen by more than 2^8
//   dQ         rows are queries: S, dP = dO V^T, dS = P (dP - delta), dQ += dS K
//   dK, dV     rows are keys:    S^T = K Q^T, dV += P^T dO, dP^T = V dO^T, dK += dS^T Q, over all query heads of the group
// P and dS are rounded to bf16, each by up to 2^-8 of itself: over many keys that makes a result's error 0.0024 of its norm, of which
// 0.0017 are its own rounding; over few keys single ones show, and more than that.  So the first tile of rows that see FEW keys or less
// is multiplied as a sum of two bf16 (`few`), with the low parts in the other half of the scores' columns, which leaves such
// results their own rounding alone; for every tile it would be one product more of two (forward) or five.  8 x 2048 tokens, 32/8
// heads of 128, causal: forward 267 -> 271 us; backward over 16 sequences of 1 to 2048: 408 -> 411 us.
// A tile that reaches past its sequence's end holds rows of the next one (or zeros): their scores are masked, and where such rows
// would be summed over they are zeroed in shared memory, so that nothing of them, a NaN included, gets in.
#include <type_traits>

#include "attn.cuh"
#include "umma.cuh"

namespace vcas {
namespace {

// A tile of ROWS rows is one block of 128-byte swizzled rows (64 bf16) for each 64 of its columns.
template <int ROWS> constexpr int CHUNK = ROWS * 64 * 2;

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
// A tile's rows as the summed-over side of a product: its 64-wide blocks lie CHUNK apart.
template <int ROWS>
__device__ __forceinline__ uint64_t desc_rows(uint32_t saddr) {
  return (uint64_t)((saddr & 0x3ffffu) >> 4) | ((uint64_t)(CHUNK<ROWS> >> 4) << 16) | ((uint64_t)(1024 >> 4) << 32) | (1ull << 46) | (2ull << 61);
}
// D [128 x TN] = A B^T, tiles of 128 and TN rows, summed over their 64 * DC columns
template <int DC, int TN>
__device__ __forceinline__ void product_tiles(uint32_t d, uint32_t a, uint32_t b) {
  constexpr uint32_t idesc = make_idesc(TN, false, false);
#pragma unroll
  for (int c = 0; c < DC; ++c) {
    const uint64_t da = desc_kmajor(a + c * CHUNK<128>), db = desc_kmajor(b + c * CHUNK<TN>);
#pragma unroll
    for (int k = 0; k < 4; ++k) umma_bf16(d, da + (uint64_t)(k * 2), db + (uint64_t)(k * 2), idesc, (c | k) != 0 ? 1u : 0u);
  }
}
// the same with A in TMEM, 32 DC columns of bf16 pairs
template <int DC, int TN>
__device__ __forceinline__ void product_tiles_ts(uint32_t d, uint32_t a, uint32_t b) {
  constexpr uint32_t idesc = make_idesc(TN, false, false);
#pragma unroll
  for (int c = 0; c < DC; ++c) {
    const uint64_t db = desc_kmajor(b + c * CHUNK<TN>);
#pragma unroll
    for (int k = 0; k < 4; ++k) umma_bf16_ts(d, a + (uint32_t)(c * 32 + k * 8), db + (uint64_t)(k * 2), idesc, (c | k) != 0 ? 1u : 0u);
  }
}
// D [128 x 64 DC] (+)= A B, A [128 x TN] bf16 in TMEM (each 64 of its columns `gap` TMEM columns behind the 64 before), B a tile of
// TN rows
template <int DC, int TN>
__device__ __forceinline__ void product_rows(uint32_t d, uint32_t a, int gap, uint32_t b, bool add) {
  constexpr uint32_t idesc = make_idesc(64 * DC, false, true);
  const uint64_t db = desc_rows<TN>(b);
#pragma unroll
  for (int k = 0; k < TN / 16; ++k)
    umma_bf16_ts(d, a + (uint32_t)((k & 3) * 8 + (k >> 2) * gap), db + (uint64_t)(k * (16 * 128 >> 4)), idesc, add || k != 0 ? 1u : 0u);
}
// the rows from `have` on of a tile become 0, by one warp; the products after it see them
template <int DC, int ROWS>
__device__ __forceinline__ void zero_rows(uint8_t* tile, int have, int lane) {
  for (int i = have * 8 + lane; i < ROWS * 8; i += 32)
#pragma unroll
    for (int c = 0; c < DC; ++c) *reinterpret_cast<uint4*>(tile + c * CHUNK<ROWS> + i * 16) = make_uint4(0, 0, 0, 0);
}
template <int DC, int ROWS>
__device__ __forceinline__ void load_tile(uint8_t* dst, const CUtensorMap* map, int head, int token, uint64_t* bar) {
#pragma unroll
  for (int c = 0; c < DC; ++c) tma_load_3d(dst + c * CHUNK<ROWS>, map, 64 * c, head, token, bar);
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  const __nv_bfloat162 t = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&t);
}
// What rounding x to the pairs `hi` left, rounded in its turn: the sum of both has 16 bits and more.
__device__ __forceinline__ void low_parts(const uint32_t (&x)[64], const uint32_t (&hi)[32], uint32_t (&lo)[32]) {
#pragma unroll
  for (int i = 0; i < 32; ++i)
    lo[i] = pack_bf16(__uint_as_float(x[2 * i]) - __uint_as_float(hi[i] << 16), __uint_as_float(x[2 * i + 1]) - __uint_as_float(hi[i] & 0xffff0000u));
}
// 64 columns of a row of a tile of 128 rows, as 32 pairs
__device__ __forceinline__ void read_row(const uint8_t* tile, int row, uint32_t (&v)[32]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint4 x = *reinterpret_cast<const uint4*>(tile + row * 128 + ((i ^ (row & 7)) << 4));        // the 128-byte swizzle
    v[4 * i] = x.x; v[4 * i + 1] = x.y; v[4 * i + 2] = x.z; v[4 * i + 3] = x.w;
  }
}
// the sum of its products with v
__device__ __forceinline__ float row_dot(const uint8_t* tile, int row, const uint32_t (&v)[32]) {
  float s0 = 0.f, s1 = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint4 x = *reinterpret_cast<const uint4*>(tile + row * 128 + ((i ^ (row & 7)) << 4));
    const uint32_t xs[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      s0 = fmaf(__uint_as_float(xs[e] << 16), __uint_as_float(v[4 * i + e] << 16), s0);
      s1 = fmaf(__uint_as_float(xs[e] & 0xffff0000u), __uint_as_float(v[4 * i + e] & 0xffff0000u), s1);
    }
  }
  return s0 + s1;
}
// A warp's 32 rows of a [128 x 64 DC] accumulator, times f (each lane its row's), to rows of a tensor; `rows` of them exist.  Four lanes
// exchange 16-byte pieces of their rows, so that a store instruction writes 64 bytes in a row (a lane writing its own row, 16 bytes of 32
// rows at a time, took 1.4 us a tile, half as long as a tile of scores).
template <int DC>
__device__ __forceinline__ void store_rows(uint32_t taddr, const Strided& x, int64_t first, int head, int dim, int rows, float f) {
  const int lane = threadIdx.x & 31, unit = lane & 3;
  __nv_bfloat16* base = (__nv_bfloat16*)const_cast<void*>(x.p) + (first + (lane & ~3)) * x.token + (int64_t)head * x.head + unit * 8;
#pragma unroll
  for (int c = 0; c < 2 * DC; ++c) {
    uint32_t v[32], u[4][4];
    tmem_ld32(taddr + c * 32, v);
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
      for (int e = 0; e < 4; ++e) u[k][e] = pack_bf16(__uint_as_float(v[8 * k + 2 * e]) * f, __uint_as_float(v[8 * k + 2 * e + 1]) * f);
    // the 4 x 4 pieces of four lanes, turned over
    auto swap = [&](uint32_t (&lo)[4], uint32_t (&hi)[4], int bit) {
      const bool up = (lane & bit) != 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t got = __shfl_xor_sync(0xffffffffu, up ? lo[e] : hi[e], bit);
        if (up) lo[e] = got; else hi[e] = got;
      }
    };
    swap(u[0], u[1], 1);
    swap(u[2], u[3], 1);
    swap(u[0], u[2], 2);
    swap(u[1], u[3], 2);
    if (c * 32 + unit * 8 < dim) {
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if ((lane & ~3) + k < rows)
          *reinterpret_cast<uint4*>(base + (int64_t)k * x.token + c * 32) = make_uint4(u[k][0], u[k][1], u[k][2], u[k][3]);
    }
  }
}

// ----------------------------------------------------------------------------------------- the CTA
constexpr int MAX_STAGES = 10;
constexpr int FEW = 64;                              // at most a tile of keys
struct Item { int first, len, t0, head, any; };      // a tile of 128 rows: its sequence, its first row in there, its head
// whether the first rows of a sequence see FEW keys or less
__device__ __forceinline__ bool few_keys(const Item& it, bool causal) { return causal || it.len <= FEW; }
struct Shared {
  uint64_t full[MAX_STAGES], empty[MAX_STAGES];      // ring of the other side's tiles
  uint64_t item_full[2], item_empty[2];
  uint64_t own_full, own_empty;                      // the item's own tiles
  uint64_t scores[4], dscores;                       // products of which the scores' warps wait
  uint64_t ready[4];                                 // P, dS written
  uint64_t done[2], acc_empty[2];                    // accumulators complete, and read
  uint64_t taken, drain[2];                          // dQ: the own tiles have been read
  uint64_t sums;                                     // dQ: parts of delta from P and dP
  uint64_t added[2];                                 // forward: P V of a tile is in O
  uint64_t rows_full[2][2];                          // dK, dV: the queries' values, by column half and buffer
  uint32_t tmem;
  int abort_flag;                                    // mbar_wait finds the limit 20 bytes behind it
  int pad[4];
  unsigned long long limit;
  Item item[2];
};
static_assert(offsetof(Shared, limit) == offsetof(Shared, abort_flag) + 20, "see mbar_wait");

struct UmmaCall {
  AttnCall c;
  int32_t* next;                                     // two counters: tiles taken, CTAs that are through
  unsigned long long wait_limit_ns;
  int stall_once;
};

// A whole warp waits and goes on, or gives up, together: what follows are instructions of all its lanes.
__device__ __forceinline__ bool warp_wait(uint64_t* bar, uint32_t parity, volatile int* ab, int32_t* status) {
  return __all_sync(0xffffffffu, mbar_wait(bar, parity, ab, status));
}
__device__ __forceinline__ void warp_arrive(uint64_t* bar) {
  __syncwarp();
  if ((threadIdx.x & 31) == 0) mbar_arrive(bar);
}

// Shared memory is all dynamic, its tiles first: they have to begin on a 1024-byte boundary, where the CTA's part begins.
__device__ __forceinline__ bool in_place(const uint8_t* smem, int32_t* status) {
  if ((smem_u32(smem) & 1023u) == 0) return true;
  if (threadIdx.x == 0) atomicExch(status, (int32_t)VCAS_ERR_INTERNAL);
  return false;
}
// Sets the barriers up and takes TMEM.  warps: those that work on scores, `team` of them on the same ones.
// issuers: warps that issue products; own_arrivals: with which the own tiles are given back.
__device__ __forceinline__ void begin(Shared& s, const UmmaCall& P, int stages, uint32_t warps, uint32_t team, uint32_t issuers,
                                      uint32_t own_arrivals, uint32_t columns) {
  if (threadIdx.x == 0) {
    for (int i = 0; i < stages; ++i) { mbar_init(&s.full[i], 1); mbar_init(&s.empty[i], issuers); }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&s.item_full[i], 1);
      mbar_init(&s.item_empty[i], warps + issuers);
      mbar_init(&s.done[i], 1);
      mbar_init(&s.acc_empty[i], team);
      mbar_init(&s.added[i], 1);
    }
    for (int i = 0; i < 4; ++i) { mbar_init(&s.scores[i], 1); mbar_init(&s.ready[i], team); }
    mbar_init(&s.own_full, 1);
    mbar_init(&s.own_empty, own_arrivals);
    mbar_init(&s.dscores, 1);
    mbar_init(&s.taken, warps);
    mbar_init(&s.sums, warps);
    for (int i = 0; i < 4; ++i) mbar_init(&s.rows_full[i >> 1][i & 1], 4);
    mbar_init(&s.drain[0], 1);
    mbar_init(&s.drain[1], 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    s.abort_flag = 0;
    s.limit = P.wait_limit_ns;
  }
  if ((threadIdx.x >> 5) == 2) tmem_alloc(&s.tmem, columns);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
}
__device__ __forceinline__ void end(Shared& s, const UmmaCall& P, uint32_t columns) {
  tc_fence_before();
  __syncthreads();
  if ((threadIdx.x >> 5) == 2) {
    tc_fence_after();
    tmem_dealloc(s.tmem, columns);
  }
  // the last CTA leaves the counters as it found them
  if (threadIdx.x == 0 && atomicAdd(P.next + 1, 1) == (int)gridDim.x - 1) {
    P.next[0] = 0;
    P.next[1] = 0;
  }
}
__device__ __forceinline__ void prefetch_map(const CUtensorMap* m) { asm volatile("prefetch.tensormap [%0];" ::"l"(m) : "memory"); }
// A ring position
struct Ring {
  int stage = 0;
  uint32_t phase = 0;
  uint32_t filled = 0;
  __device__ __forceinline__ void next(int stages) {
    if (++stage == stages) { stage = 0; phase ^= 1u; }
  }
  template <int STAGES>
  __device__ __forceinline__ void skip(int n) {
    stage += n;
    phase ^= (uint32_t)(stage / STAGES) & 1u;
    stage %= STAGES;
  }
};
// The loading warp's part: takes the next tile off the counter and tells the others.  The counter goes through the heads first, so that
// CTAs at work at the same time share the other side's tiles, then through the tiles in the order of `Order`.
// With lse, [2][128] floats of shared memory, the rows' lse comes along (a load of their own, at the start of a tile, was 1100 cycles).
__device__ __forceinline__ bool take_item(Shared& s, const UmmaCall& P, const Order& order, int n, int heads, Item& it, float* lse = nullptr) {
  const int lane = threadIdx.x & 31;
  volatile int* ab = &s.abort_flag;
  if (!warp_wait(&s.item_empty[n & 1], ((n >> 1) & 1) ^ 1, ab, P.c.seqs.status)) return false;
  int at = (int)blockIdx.x;                          // the first one needs no counter
  if (n > 0) {
    if (lane == 0) at = (int)gridDim.x + atomicAdd(P.next, 1);
    at = __shfl_sync(0xffffffffu, at, 0);
  }
  int place = 0;
  it.first = it.len = 0;
  it.head = at % heads;
  it.any = order.find(P.c.seqs, at / heads, lane, it.first, it.len, place);
  it.t0 = place * 128;
  if (lse != nullptr && it.any) {
    const float* from = P.c.lse + (int64_t)it.head * P.c.seqs.total + it.first + it.t0;
#pragma unroll
    for (int i = 0; i < 4; ++i) lse[(n & 1) * 128 + 32 * i + lane] = it.t0 + 32 * i + lane < it.len ? __ldcg(from + 32 * i + lane) : 0.f;
  }
  if (lane == 0) s.item[n & 1] = it;
  warp_arrive(&s.item_full[n & 1]);
  return it.any;
}
// The others' part.  False: no more, or given up.  lse: of one row of the tile.
__device__ __forceinline__ bool get_item(Shared& s, int n, int32_t* status, Item& it, const float* lse = nullptr, float* mine = nullptr) {
  if (!warp_wait(&s.item_full[n & 1], (n >> 1) & 1, &s.abort_flag, status)) return false;
  it = s.item[n & 1];
  if (lse != nullptr) *mine = lse[(n & 1) * 128];
  warp_arrive(&s.item_empty[n & 1]);
  return it.any;
}
// Loads a tile of the ring; `skip`: the test hook that leaves the copy out.
template <int DC, int ROWS>
__device__ __forceinline__ bool fill(Shared& s, Ring& r, int stages, uint8_t* ring, const CUtensorMap* map, int head, int token, bool skip,
                                     int32_t* status) {
  constexpr int BYTES = DC * CHUNK<ROWS>;
  if (!warp_wait(&s.empty[r.stage], r.phase ^ 1u, &s.abort_flag, status)) return false;
  if (!skip) {
    if (elect_one()) {
      mbar_expect_tx(&s.full[r.stage], BYTES);
      load_tile<DC, ROWS>(ring + r.stage * BYTES, map, head, token, &s.full[r.stage]);
    }
    ++r.filled;
  }
  r.next(stages);
  return true;
}
// After a wait that ran out: nothing may arrive in shared memory that is no longer this CTA's.
__device__ __forceinline__ void drain(Shared& s, const Ring& r, int stages, uint32_t own_filled, int32_t* status) {
  if (!*(volatile int*)&s.abort_flag) return;
  if (own_filled != 0) mbar_wait(&s.own_full, (own_filled - 1) & 1, &s.abort_flag, status);
  drain_loads(s.full, stages, r.stage, r.phase, r.filled, &s.abort_flag, status);
}

// ------------------------------------------------------------------------------------------ forward
// 128 query rows of one head (two CTAs an SM) or of two heads that share keys and values (one), against tiles of 64 keys: two tiles of
// scores of each head are in TMEM (64 columns each, beside O's 64 DC), so that a tile's scores are there when the warps come from the
// one before, and the products of two heads or CTAs fill the tensor pipe.  (Key tiles of 128, one at a time: 1506 of a tile's 3644 cycles
// went by between the last P and the next scores.)
// Q is read for each tile of keys (there is no room for it in TMEM): 64-wide products with both operands in shared memory take 427
// cycles for 256 of arithmetic.  Two heads on one copy of K and V save a sixth of the bytes that the tiles bring in: for heads wider
// than 64 in groups of an even number (8 x 2048 tokens, 32/8 heads of 128, causal: 282 us by one head, 267 by two, both before `few`);
// narrower ones are bound by their exponentials.  Over the whole kernel nothing counted is full there: tensor pipe 51 % of the cycles,
// its reads of shared memory 50 %, special function unit 51 %, issue slots 38 %; the rest goes by in the chain scores -> exponentials -> P ->
// product of each 64 keys, which two heads fill only in part.  (A part of the exponentials as polynomials on the FMA pipe: 298 us for one in eight
// of the pairs where all by the special function unit took 292; the warps' issue slots were what it cost.)
constexpr int FWD_TN = 64;
template <int DC, int HEADS> constexpr int FWD_STAGES = HEADS == 2 ? 10 : DC == 1 ? 8 : 5;
template <int HEADS> constexpr int FWD_THREADS = 160 * HEADS + 32;

template <int DC, int HEADS>
__global__ void __launch_bounds__(FWD_THREADS<HEADS>, HEADS == 2 ? 1 : 2)
attn_fwd_kernel(const __grid_constant__ CUtensorMap mq, const __grid_constant__ CUtensorMap mk, const __grid_constant__ CUtensorMap mv,
                const __grid_constant__ UmmaCall P) {
  constexpr int STAGES = FWD_STAGES<DC, HEADS>, TN = FWD_TN, OWN = DC * CHUNK<128>, TILE = DC * CHUNK<TN>, COLUMNS = 256 * HEADS;
  extern __shared__ __align__(1024) uint8_t smem[];
  uint8_t *sq = smem, *ring = smem + HEADS * OWN;
  Shared& s = *reinterpret_cast<Shared*>(ring + STAGES * TILE);
  const AttnCall& C = P.c;
  if (!in_place(smem, C.seqs.status)) return;
  begin(s, P, STAGES, 4 * HEADS, 4, HEADS, HEADS, COLUMNS);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  // TMEM of head h: two tiles of scores, O
  auto scores_of = [&](int h) { return s.tmem + (uint32_t)(h * 256); };
  auto out_of = [&](int h) { return s.tmem + (uint32_t)(h * 256 + 2 * TN); };
  volatile int* ab = &s.abort_flag;
  int32_t* status = C.seqs.status;
  auto tiles_of = [&](const Item& it) { return ((C.causal ? min(it.len, it.t0 + 128) : it.len) + TN - 1) / TN; };

  if (warp == 5 * HEADS) {
    const Order order(C.seqs, lane, C.causal, false);
    Ring r;
    Item it;
    uint32_t own = 0;
    if (lane == 0) {
      prefetch_map(&mq);
      prefetch_map(&mk);
      prefetch_map(&mv);
    }
    for (int n = 0; take_item(s, P, order, n, C.heads_q / HEADS, it); ++n) {
      bool ok = warp_wait(&s.own_empty, (n & 1) ^ 1, ab, status);
      if (!ok) break;
      if (elect_one()) {
        mbar_expect_tx(&s.own_full, HEADS * OWN);
#pragma unroll
        for (int h = 0; h < HEADS; ++h) load_tile<DC, 128>(sq + h * OWN, &mq, it.head * HEADS + h, it.first + it.t0, &s.own_full);
      }
      ++own;
      const int tiles = tiles_of(it), kv = it.head * HEADS / C.group;
      const bool stall = P.stall_once && blockIdx.x == 0 && n == 0;
      // in the order of their use: K 0, K 1, V 0, K 2, V 1, ...
      for (int j = 0; j <= tiles && ok; ++j) {
        if (j < tiles) ok = fill<DC, TN>(s, r, STAGES, ring, &mk, kv, it.first + j * TN, stall && j == 0, status);
        if (j > 0) ok = ok && fill<DC, TN>(s, r, STAGES, ring, &mv, kv, it.first + (j - 1) * TN, false, status);
      }
      if (!ok) break;
    }
    if (lane == 0) drain(s, r, STAGES, own, status);
  } else if (warp >= 4 * HEADS) {
    // one for each head: a head's products do not wait for the other's probabilities
    const int h = warp - 4 * HEADS;
    const uint32_t ts = scores_of(h), to = out_of(h), q = smem_u32(sq + h * OWN);
    const bool leader = elect_one();
    Ring r;
    Item it;
    uint32_t made = 0, score = 0;        // P tiles, score tiles so far
    bool ok = true;
    for (int n = 0; ok && get_item(s, n, status, it); ++n) {
      const int tiles = tiles_of(it);
      const bool few = it.t0 == 0 && few_keys(it, C.causal);
      ok = warp_wait(&s.own_full, n & 1, ab, status);
      if (!ok) break;
      auto scores = [&](bool last) {
        ok = warp_wait(&s.full[r.stage], r.phase, ab, status);
        if (!ok) return;
        tc_fence_after();
        if (leader) {
          product_tiles<DC, TN>(ts + (score & 1) * TN, q, smem_u32(ring + r.stage * TILE));
          umma_commit(&s.empty[r.stage]);
          umma_commit(&s.scores[2 * h + (score & 1)]);
          if (last) umma_commit(&s.own_empty);
        }
        ++score;
        r.next(STAGES);
      };
      scores(tiles == 1);
      if (ok && tiles > 1) scores(tiles == 2);
      for (int j = 0; j < tiles && ok; ++j, ++made) {
        ok = warp_wait(&s.full[r.stage], r.phase, ab, status);
        if (!ok) break;
        const int have = it.len - j * TN, place = r.stage;
        if (have < TN) {                 // zeros over zeros where the other head's warp has been
          zero_rows<DC, TN>(ring + place * TILE, have, lane);
          fence_async_smem();
          __syncwarp();
        }
        r.next(STAGES);
        if (j == 0) ok = warp_wait(&s.acc_empty[h], (n & 1) ^ 1, ab, status);
        ok = ok && warp_wait(&s.ready[2 * h + (made & 1)], (made >> 1) & 1, ab, status);
        if (!ok) break;
        tc_fence_after();
        if (leader) {
          product_rows<DC, TN>(to, ts + (made & 1) * TN, 0, smem_u32(ring + place * TILE), j != 0);
          if (j == 0 && few) product_rows<DC, TN>(to, ts + (made & 1) * TN + 32, 0, smem_u32(ring + place * TILE), true);
          umma_commit(&s.empty[place]);
          umma_commit(&s.added[h]);
          if (j == tiles - 1) umma_commit(&s.done[h]);
        }
        if (j + 2 < tiles) scores(j + 3 == tiles);
      }
    }
    if (leader && *ab) drain_products(&s.drain[h], ab, status);
  } else {
    const int h = warp >> 2, in = threadIdx.x & 127;
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16, ts = scores_of(h), to = out_of(h);
    const float c = C.scale * ATTN_LOG2E, none = __int_as_float(0xff800000);
    const uint64_t c2 = pack2(c, c);
    Item it;
    uint32_t made = 0;
    bool ok = true;
    for (int n = 0; ok && get_item(s, n, status, it); ++n) {
      const int row = it.t0 + in, tiles = tiles_of(it), head = it.head * HEADS + h;      // row: in the sequence
      // Sums are relative to 2^m, m near the largest score so far (times c).  They are floats, so it need not be the largest:
      // exponentials are taken before the tile's own maximum is known (with it first, 395 cycles per 128 keys went by without an
      // exponential on its way), m follows once the maximum is 8 above it, and at once where 2^64 is passed.
      float m = 0.f, l = 0.f, over = 0.f;            // over: the last tile's maximum above m
      auto lift = [&](float by, bool mine) {
        // O must be complete up to the tile before this one
        ok = warp_wait(&s.added[h], (made - 1) & 1, ab, status);
        if (!ok) return;
        tc_fence_after();
        const float f = mine ? attn_exp2(-by) : 1.0f;
        m += mine ? by : 0.f;
        l *= f;
#pragma unroll
        for (int q = 0; q < 2 * DC; ++q) {
          uint32_t o[32];
          tmem_ld32(to + lanes + q * 32, o);
#pragma unroll
          for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
          tmem_st32(to + lanes + q * 32, o);
        }
        tmem_wait_st();
      };
      for (int j = 0; j < tiles; ++j, ++made) {
        ok = warp_wait(&s.scores[2 * h + (made & 1)], (made >> 1) & 1, ab, status);
        if (!ok) break;
        tc_fence_after();
        const uint32_t at = ts + lanes + (made & 1) * TN;
        // columns this row sees in the tile
        const int see = min(TN, (C.causal ? min(it.len, row + 1) : it.len) - j * TN);
        const bool cut = __any_sync(0xffffffffu, see < TN);
        uint32_t x[64], o[32];
        auto read = [&]() {
          tmem_ld64(at, x);
          if (cut) {
#pragma unroll
            for (int i = 0; i < 64; ++i) x[i] = i < see ? x[i] : 0xff800000u;
          }
        };
        read();
        if (j == 0) {
          float t[4] = {none, none, none, none};
#pragma unroll
          for (int i = 0; i < 64; ++i) t[i & 3] = fmaxf(t[i & 3], __uint_as_float(x[i]));
          m = fmaxf(fmaxf(t[0], t[1]), fmaxf(t[2], t[3])) * c;
          if (m == none) m = 0.f;
        } else if (__any_sync(0xffffffffu, over > 8.0f)) {
          lift(over, over > 8.0f);
          if (!ok) break;
        }
        float sum;
        auto exps = [&](auto keep) {
          const uint64_t n2 = pack2(-m, -m);
          uint64_t l2[2] = {0, 0};
          float t[2] = {none, none};
#pragma unroll
          for (int i = 0; i < 32; ++i) {
            float e0, e1;
            unpack2(fma2(pack2(__uint_as_float(x[2 * i]), __uint_as_float(x[2 * i + 1])), c2, n2), e0, e1);
            t[i & 1] = fmaxf(t[i & 1], fmaxf(e0, e1));
            e0 = attn_exp2(e0);
            e1 = attn_exp2(e1);
            l2[i & 1] = add2(l2[i & 1], pack2(e0, e1));
            o[i] = pack_bf16(e0, e1);
            if constexpr (keep.value) {
              x[2 * i] = __float_as_uint(e0);
              x[2 * i + 1] = __float_as_uint(e1);
            }
          }
          float y0, y1;
          unpack2(add2(l2[0], l2[1]), y0, y1);
          sum = y0 + y1;
          over = fmaxf(t[0], t[1]);
        };
        if (j == 0 && it.t0 == 0 && few_keys(it, C.causal)) {
          exps(std::true_type());
          uint32_t lo[32];
          low_parts(x, o, lo);
          tmem_st32(at + 32, lo);
        } else {
          exps(std::false_type());
        }
        if (j != 0 && __any_sync(0xffffffffu, over > 64.0f)) {
          lift(over, over > 64.0f);
          if (!ok) break;
          read();
          exps(std::false_type());
        }
        l += sum;
        tmem_st32(at, o);
        tmem_wait_st();
        tc_fence_before();
        warp_arrive(&s.ready[2 * h + (made & 1)]);
      }
      ok = ok && warp_wait(&s.done[h], n & 1, ab, status);
      if (!ok) break;
      tc_fence_after();
      const int warp_row = it.t0 + (warp & 3) * 32;
      store_rows<DC>(to + lanes, C.o, (int64_t)it.first + warp_row, head, C.dim, it.len - warp_row, 1.0f / l);
      tc_fence_before();
      warp_arrive(&s.acc_empty[h]);
      if (row < it.len) C.lse[(int64_t)head * C.seqs.total + it.first + row] = m * ATTN_LN2 + logf(l);
    }
  }
  end(s, P, COLUMNS);
}

// ------------------------------------------------------------------------------------------ backward
// The other side comes in tiles of TN rows.  Heads of up to 64: 64, which leaves room for two CTAs an SM (TMEM holds 256 columns of
// each), so that one computes while the other starts, waits or stores.  Wider ones: 128, one CTA.  A warp has 32 rows and 64 columns of
// scores.  The ring's tiles are used two at a time and given back one by one: with five, the tiles of the next step are on their way
// one step ahead.
template <int DC> constexpr int TN_OF = DC == 1 ? 64 : 128;
template <int DC> constexpr int BWD_WARPS = 4 * TN_OF<DC> / 64;
template <int DC> constexpr int BWD_THREADS = 32 * (BWD_WARPS<DC> + 2);
template <int DC> constexpr int BWD_CTAS = DC == 1 ? 2 : 1;
template <int DC> constexpr int BWD_STAGES = DC == 1 ? 6 : 5;

// Rows are queries.  TMEM: S, dP (dS replaces it), dQ, and Q and dO as A operands of all products with them: read from shared memory for
// each tile, with both operands there, they took most of its bandwidth (a tile of 128 keys 2290 cycles; with them in TMEM, and one S in
// place of two, 2140).  S is free for the next tile's scores as soon as the warps have read it.  O comes once a tile of rows, for
// delta = rowsum(dO O): in the ring where its tiles are as large (DC = 2), else beside Q and dO.
template <int DC>
__global__ void __launch_bounds__(BWD_THREADS<DC>, BWD_CTAS<DC>)
attn_dq_kernel(const __grid_constant__ CUtensorMap mq, const __grid_constant__ CUtensorMap mdo, const __grid_constant__ CUtensorMap mo,
               const __grid_constant__ CUtensorMap mk, const __grid_constant__ CUtensorMap mv, const __grid_constant__ UmmaCall P) {
  constexpr int STAGES = BWD_STAGES<DC>, TN = TN_OF<DC>, WARPS = BWD_WARPS<DC>, OWN = DC * CHUNK<128>, TILE = DC * CHUNK<TN>;
  constexpr bool O_IN_RING = DC == 2;
  static_assert(!O_IN_RING || TN == 128, "as large as a tile of the ring");
  static_assert(WARPS == 4 * DC, "every 64 columns have a warp");
  extern __shared__ __align__(1024) uint8_t smem[];
  uint8_t *sq = smem, *sdo = sq + OWN, *so = sdo + OWN, *ring = O_IN_RING ? so : so + OWN;
  float* s_half = reinterpret_cast<float*>(ring + STAGES * TILE);    // [DC][128] parts of delta
  float* s_lse = s_half + DC * 128;                                  // [2][128]
  Shared& s = *reinterpret_cast<Shared*>(s_lse + 2 * 128);
  const AttnCall& C = P.c;
  if (!in_place(smem, C.seqs.status)) return;
  // The kernel before it may be the one that writes zeros to the other sequences' rows, which runs beside this one (it has begun, so
  // all before it is done); the wait at the end makes sure that this one does not end first.  The dK, dV kernel's CTAs may come as
  // soon as the last ones of this grid have begun.
  pdl_trigger();
  begin(s, P, STAGES, WARPS, WARPS, 1, WARPS, 4 * TN);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t ts = s.tmem, tdp = ts + TN, tdq = ts + 2 * TN, tq = tdq + 64 * DC, tdo = tq + 32 * DC;
  static_assert(2 * TN + 128 * DC == 4 * TN, "all columns");
  volatile int* ab = &s.abort_flag;
  int32_t* status = C.seqs.status;
  auto tiles_of = [&](const Item& it) { return ((C.causal ? min(it.len, it.t0 + 128) : it.len) + TN - 1) / TN; };

  if (warp == WARPS + 1) {
    const Order order(C.seqs, lane, C.causal, false);
    Ring r;
    Item it;
    uint32_t own = 0;
    if (lane == 0) {
      prefetch_map(&mq);
      prefetch_map(&mdo);
      prefetch_map(&mo);
      prefetch_map(&mk);
      prefetch_map(&mv);
    }
    // Q, dO (and O) of a tile of rows: their place is free as soon as those of the one before have been taken
    auto load_own = [&](int n, const Item& x) -> bool {
      if (!warp_wait(&s.own_empty, (n & 1) ^ 1, ab, status)) return false;
      if (elect_one()) {
        mbar_expect_tx(&s.own_full, (O_IN_RING ? 2 : 3) * OWN);
        load_tile<DC, 128>(sq, &mq, x.head, x.first + x.t0, &s.own_full);
        load_tile<DC, 128>(sdo, &mdo, x.head, x.first + x.t0, &s.own_full);
        if (!O_IN_RING) load_tile<DC, 128>(so, &mo, x.head, x.first + x.t0, &s.own_full);
      }
      ++own;
      return true;
    };
    bool more = take_item(s, P, order, 0, C.heads_q, it, s_lse), ok = !more || load_own(0, it);
    for (int n = 0; more && ok; ++n) {
      Item next = it;
      const int tiles = tiles_of(it), kv = it.head / C.group, from = O_IN_RING ? -1 : 0, loads = 2 * tiles - from;
      const bool stall = P.stall_once && blockIdx.x == 0 && n == 0;
      for (int i = from; i < 2 * tiles && ok; ++i) {
        if (i < 0) ok = fill<DC, TN>(s, r, STAGES, ring, &mo, it.head, it.first + it.t0, false, status);
        else ok = fill<DC, TN>(s, r, STAGES, ring, (i & 1) ? &mv : &mk, kv, it.first + (i >> 1) * TN, stall && i == 0, status);
        if (ok && i - from == min(loads, STAGES) - 1) {
          // the ring is full or this tile's loads are on their way: time to see to the next one
          more = take_item(s, P, order, n + 1, C.heads_q, next, s_lse);
          if (more) ok = load_own(n + 1, next);
        }
      }
      it = next;
    }
    if (lane == 0) drain(s, r, STAGES, own, status);
  } else if (warp == WARPS) {
    const bool leader = elect_one();
    Ring r;
    Item it;
    uint32_t made = 0;                   // tiles of scores so far
    bool ok = true;
    for (int n = 0; ok && get_item(s, n, status, it); ++n) {
      const int tiles = tiles_of(it);
      const bool few = it.t0 == 0 && few_keys(it, C.causal);
      // Q and dO are in TMEM, and O has been read
      ok = warp_wait(&s.taken, n & 1, ab, status);
      if (!ok) break;
      tc_fence_after();
      if (O_IN_RING) {
        if (leader) mbar_arrive(&s.empty[r.stage]);
        r.next(STAGES);
      }
      int k_now = 0, k_next = 0;         // ring places of this tile's K and the next one's
      // waits for the next tile of the ring; rows behind the sequence's end become 0
      auto arrived = [&](int j) {
        const int place = r.stage, have = it.len - j * TN;
        ok = warp_wait(&s.full[place], r.phase, ab, status);
        if (ok && have < TN) {
          zero_rows<DC, TN>(ring + place * TILE, have, lane);
          fence_async_smem();
          __syncwarp();
        }
        r.next(STAGES);
        tc_fence_after();
        return place;
      };
      auto scores = [&](int j) {
        k_next = arrived(j);
        if (!ok) return;
        if (leader) {
          product_tiles_ts<DC, TN>(ts, tq, smem_u32(ring + k_next * TILE));
          umma_commit(&s.scores[0]);
        }
      };
      auto dscores = [&](int j) {
        const int v = arrived(j);
        if (!ok) return;
        if (leader) {
          product_tiles_ts<DC, TN>(tdp, tdo, smem_u32(ring + v * TILE));
          umma_commit(&s.dscores);
          umma_commit(&s.empty[v]);
        }
      };
      scores(0);
      if (!ok) break;
      dscores(0);
      if (!ok) break;
      for (int j = 0; j < tiles; ++j, ++made) {
        k_now = k_next;
        ok = warp_wait(&s.ready[1], made & 1, ab, status);       // S has been read
        if (!ok) break;
        tc_fence_after();
        if (j + 1 < tiles) {
          scores(j + 1);
          if (!ok) break;
        }
        if (j == 0) ok = warp_wait(&s.acc_empty[0], (n & 1) ^ 1, ab, status);
        ok = ok && warp_wait(&s.ready[0], made & 1, ab, status);
        if (!ok) break;
        tc_fence_after();
        if (leader) {
          product_rows<DC, TN>(tdq, tdp, 64, smem_u32(ring + k_now * TILE), j != 0);
          if (j == 0 && few) product_rows<DC, TN>(tdq, tdp + 32, 64, smem_u32(ring + k_now * TILE), true);
          umma_commit(&s.empty[k_now]);
          if (j == tiles - 1) umma_commit(&s.done[0]);
        }
        if (j + 1 < tiles) dscores(j + 1);
        if (!ok) break;
      }
    }
    if (leader && *ab) drain_products(&s.drain[0], ab, status);
  } else {
    const int part = warp >> 2, in = (warp & 3) * 32 + lane;     // columns part * 64 ..; row of the tile
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const float c = C.scale * ATTN_LOG2E;
    const uint64_t c2 = pack2(c, c);
    Item it, prev;
    float lse = 0.f, delta = 0.f;
    uint32_t made = 0, summed = 0;
    Ring r;                              // the loads, to find O among them
    bool ok = true;
    // The next tile of rows: Q and dO to TMEM, delta.  s_half: every warp has read what the tile before left there.  It reads delta before
    // it arrives at a barrier that all of the tile's later steps wait for, but the sums of a single tile of keys as the last.
    auto take = [&](int n) -> bool {
      const bool single = DC == 2 && n > 0 && tiles_of(it) == 1;
      if (!get_item(s, n, status, it, s_lse + in, &lse)) return false;
      if (single) ok = warp_wait(&s.sums, summed++ & 1, ab, status);
      if (!ok) return false;
      ok = warp_wait(&s.own_full, n & 1, ab, status);
      if (!ok) return false;
      uint32_t v[32];
      read_row(sq + part * CHUNK<128>, in, v);
      tmem_st32(tq + lanes + part * 32, v);
      read_row(sdo + part * CHUNK<128>, in, v);
      tmem_st32(tdo + lanes + part * 32, v);
      const uint8_t* o_tile = so;
      if (O_IN_RING) {
        ok = warp_wait(&s.full[r.stage], r.phase, ab, status);
        if (!ok) return false;
        o_tile = ring + r.stage * TILE;
        r.skip<STAGES>(1 + 2 * tiles_of(it));
      }
      delta = row_dot(o_tile + part * CHUNK<128>, in, v);
      if (DC == 2) s_half[part * 128 + in] = delta;
      tmem_wait_st();
      tc_fence_before();
      warp_arrive(&s.taken);
      warp_arrive(&s.own_empty);
      return true;
    };
    bool more = take(0);
    for (int n = 0; more; ++n) {
      const int tiles = tiles_of(it), row = it.t0 + in;
      if (DC == 2) {
        ok = warp_wait(&s.taken, n & 1, ab, status);
        if (!ok) break;
        // with a single tile of keys delta is rowsum(P dP), whose parts another warp may already be writing there
        if (tiles > 1) delta = s_half[in] + s_half[128 + in];
      }
      const float nl = -lse * ATTN_LOG2E;
      const uint64_t n2 = pack2(nl, nl);
      uint64_t d2 = pack2(-delta, -delta);
      const bool low = it.t0 == 0 && few_keys(it, C.causal);
      for (int j = 0; j < tiles; ++j, ++made) {
        ok = warp_wait(&s.scores[0], made & 1, ab, status);
        if (!ok) break;
        tc_fence_after();
        uint32_t a[64];
        tmem_ld64(ts + lanes + part * 64, a);
        tc_fence_before();
        warp_arrive(&s.ready[1]);
#pragma unroll
        for (int i = 0; i < 32; ++i) {
          float e0, e1;
          unpack2(fma2(pack2(__uint_as_float(a[2 * i]), __uint_as_float(a[2 * i + 1])), c2, n2), e0, e1);
          a[2 * i] = __float_as_uint(attn_exp2(e0));
          a[2 * i + 1] = __float_as_uint(attn_exp2(e1));
        }
        const int see = min(TN, (C.causal ? min(it.len, row + 1) : it.len) - j * TN) - part * 64;
        if (__any_sync(0xffffffffu, see < 64)) {
#pragma unroll
          for (int i = 0; i < 64; ++i) a[i] = i < see ? a[i] : 0u;
        }
        ok = warp_wait(&s.dscores, made & 1, ab, status);
        if (!ok) break;
        tc_fence_after();
        uint32_t o[32];
        {
          uint32_t b[64];
          tmem_ld64(tdp + lanes + part * 64, b);
          if (j == 0) {
            // Rows that see no more than this tile: delta = rowsum(P dP), free of the rounding of O, which few keys average little
            // (causal sequences of a few tokens: dQ off by 0.0034 of its norm with rowsum(dO O) where 0.0025 is its rounding and that of dS).
            const int seen = C.causal ? min(it.len, row + 1) : it.len;
            const bool here = seen <= TN;
            if (part == 0 && seen == 1) a[0] = 0x3f800000u;        // P = 1, and so dS = 0
            if (DC == 2 ? tiles == 1 : __any_sync(0xffffffffu, here)) {
              uint64_t t = 0;
#pragma unroll
              for (int i = 0; i < 32; ++i)
                t = fma2(pack2(__uint_as_float(a[2 * i]), __uint_as_float(a[2 * i + 1])),
                         pack2(__uint_as_float(b[2 * i]), __uint_as_float(b[2 * i + 1])), t);
              float t0, t1;
              unpack2(t, t0, t1);
              t0 += t1;
              if (DC == 2) {
                s_half[part * 128 + in] = t0;
                warp_arrive(&s.sums);
                ok = warp_wait(&s.sums, summed++ & 1, ab, status);
                if (!ok) break;
                t0 = s_half[in] + s_half[128 + in];
                warp_arrive(&s.sums);            // read; see take
              }
              if (here) delta = t0;
            }
            d2 = pack2(-delta, -delta);
            // for the dK, dV kernel
            if (part == 0 && row < it.len) C.delta[(int64_t)it.head * C.seqs.total + it.first + row] = delta;
          }
          auto dscores = [&](auto few) {
#pragma unroll
            for (int i = 0; i < 32; ++i) {
              float s0, s1;
              unpack2(mul2(pack2(__uint_as_float(a[2 * i]), __uint_as_float(a[2 * i + 1])),
                           add2(pack2(__uint_as_float(b[2 * i]), __uint_as_float(b[2 * i + 1])), d2)), s0, s1);
              o[i] = pack_bf16(s0, s1);
              if constexpr (few.value) {
                b[2 * i] = __float_as_uint(s0);
                b[2 * i + 1] = __float_as_uint(s1);
              }
            }
            if constexpr (few.value) {
              uint32_t rest[32];
              low_parts(b, o, rest);
              tmem_st32(tdp + lanes + part * 64 + 32, rest);
            }
          };
          if (j == 0 && low)
            dscores(std::true_type());
          else
            dscores(std::false_type());
        }
        tmem_st32(tdp + lanes + part * 64, o);
        tmem_wait_st();
        tc_fence_before();
        warp_arrive(&s.ready[0]);
      }
      if (!ok) break;
      // the next tile's Q and dO go to TMEM beside the last product (S and dP, for which they were needed, are done), and its first products
      // run while this one's rows are stored, 64 columns by a warp
      prev = it;
      more = take(n + 1);
      ok = ok && warp_wait(&s.done[0], n & 1, ab, status);
      if (!ok) break;
      tc_fence_after();
      Strided x = C.dq;
      x.p = (const __nv_bfloat16*)x.p + part * 64;
      const int warp_row = prev.t0 + (warp & 3) * 32;
      store_rows<1>(tdq + lanes + part * 64, x, (int64_t)prev.first + warp_row, prev.head, C.dim - part * 64, prev.len - warp_row, C.scale);
      tc_fence_before();
      warp_arrive(&s.acc_empty[0]);
    }
  }
  pdl_wait();
  end(s, P, 4 * TN);
}

// Rows are keys.  TMEM: S^T (P^T replaces it), dP^T (dS^T replaces it), dV, dK.  The products of tile i + 1's scores are issued
// between those of tile i: S^T(i + 1) behind dV(i), dP^T(i + 1) behind dK(i), so that the tensor pipe works while the other
// warps do exponentials.
template <int DC>
__global__ void __launch_bounds__(BWD_THREADS<DC>, BWD_CTAS<DC>)
attn_dkv_kernel(const __grid_constant__ CUtensorMap mq, const __grid_constant__ CUtensorMap mdo, const __grid_constant__ CUtensorMap mk,
                const __grid_constant__ CUtensorMap mv, const __grid_constant__ UmmaCall P) {
  constexpr int STAGES = BWD_STAGES<DC>, TN = TN_OF<DC>, WARPS = BWD_WARPS<DC>, OWN = DC * CHUNK<128>, TILE = DC * CHUNK<TN>;
  extern __shared__ __align__(1024) uint8_t smem[];
  uint8_t *sk = smem, *sv = sk + OWN, *ring = sv + OWN;
  float* s_rows = reinterpret_cast<float*>(ring + STAGES * TILE);    // [2 steps][TN / 64 parts]: lse and delta of 64 queries
  Shared& s = *reinterpret_cast<Shared*>(s_rows + 2 * (TN / 64) * 128);
  const AttnCall& C = P.c;
  if (!in_place(smem, C.seqs.status)) return;
  begin(s, P, STAGES, WARPS, WARPS, 1, 1, 4 * TN);
  pdl_wait();                            // delta comes from the dQ kernel
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t ts = s.tmem, tdp = ts + TN, tdv = ts + 2 * TN, tdk = tdv + 64 * DC;
  volatile int* ab = &s.abort_flag;
  int32_t* status = C.seqs.status;
  // An item's steps: the query tiles from the first that sees a key of this tile, for one head of the group after the other.
  auto first_tile = [&](const Item& it) { return C.causal ? it.t0 / TN : 0; };
  auto per_head = [&](const Item& it) { return (it.len + TN - 1) / TN - first_tile(it); };
  struct Step { int head, row; };
  auto first_step = [&](const Item& it) { return Step{it.head * C.group, first_tile(it) * TN}; };
  auto advance = [&](const Item& it, Step& st) {
    st.row += TN;
    if (st.row >= it.len) {
      st.row = first_tile(it) * TN;
      ++st.head;
    }
  };

  if (warp == WARPS + 1) {
    const Order order(C.seqs, lane, C.causal, true);
    Ring r;
    Item it;
    uint32_t own = 0;
    if (lane == 0) {
      prefetch_map(&mq);
      prefetch_map(&mdo);
      prefetch_map(&mk);
      prefetch_map(&mv);
    }
    for (int n = 0; take_item(s, P, order, n, C.heads_kv, it); ++n) {
      bool ok = warp_wait(&s.own_empty, (n & 1) ^ 1, ab, status);
      if (!ok) break;
      if (elect_one()) {
        mbar_expect_tx(&s.own_full, 2 * OWN);
        load_tile<DC, 128>(sk, &mk, it.head, it.first + it.t0, &s.own_full);
        load_tile<DC, 128>(sv, &mv, it.head, it.first + it.t0, &s.own_full);
      }
      ++own;
      const int steps = per_head(it) * C.group;
      const bool stall = P.stall_once && blockIdx.x == 0 && n == 0;
      Step st = first_step(it);
      for (int i = 0; i < 2 * steps && ok; ++i) {
        ok = fill<DC, TN>(s, r, STAGES, ring, (i & 1) ? &mdo : &mq, st.head, it.first + st.row, stall && i == 0, status);
        if (i & 1) advance(it, st);
      }
      if (!ok) break;
    }
    if (lane == 0) drain(s, r, STAGES, own, status);
  } else if (warp == WARPS) {
    const bool leader = elect_one();
    Ring r;
    Item it;
    uint32_t made = 0;
    bool ok = true;
    for (int n = 0; ok && get_item(s, n, status, it); ++n) {
      const int steps = per_head(it) * C.group;
      ok = warp_wait(&s.own_full, n & 1, ab, status);
      if (!ok) break;
      int q_next = 0, g_next = 0;        // ring places of the next step's Q and dO
      Step st = first_step(it);          // the step whose scores were issued last
      const bool low = few_keys(it, C.causal);
      auto arrived = [&]() {
        const int place = r.stage, have = it.len - st.row;
        ok = warp_wait(&s.full[place], r.phase, ab, status);
        if (ok && have < TN) {
          zero_rows<DC, TN>(ring + place * TILE, have, lane);
          fence_async_smem();
          __syncwarp();
        }
        r.next(STAGES);
        tc_fence_after();
        return place;
      };
      auto scores = [&]() {
        q_next = arrived();
        if (!ok) return;
        if (leader) {
          product_tiles<DC, TN>(ts, smem_u32(sk), smem_u32(ring + q_next * TILE));
          umma_commit(&s.scores[0]);
        }
      };
      auto dscores = [&](int i) {
        g_next = arrived();
        if (!ok) return;
        if (leader) {
          product_tiles<DC, TN>(tdp, smem_u32(sv), smem_u32(ring + g_next * TILE));
          umma_commit(&s.dscores);
          if (i == steps - 1) umma_commit(&s.own_empty);
        }
      };
      scores();
      if (!ok) break;
      dscores(0);
      if (!ok) break;
      for (int i = 0; i < steps; ++i, ++made) {
        const bool few = low && st.row == 0;
        if (i == 0) ok = warp_wait(&s.acc_empty[0], (n & 1) ^ 1, ab, status);
        ok = ok && warp_wait(&s.ready[0], made & 1, ab, status);
        if (!ok) break;
        tc_fence_after();
        const int q = q_next, g = g_next;
        if (leader) {
          product_rows<DC, TN>(tdv, ts, 64, smem_u32(ring + g * TILE), i != 0);
          if (few) product_rows<DC, TN>(tdv, ts + 32, 64, smem_u32(ring + g * TILE), true);
          umma_commit(&s.empty[g]);
        }
        if (i + 1 < steps) {
          advance(it, st);
          scores();
          if (!ok) break;
        }
        ok = warp_wait(&s.ready[1], made & 1, ab, status);
        if (!ok) break;
        tc_fence_after();
        if (leader) {
          product_rows<DC, TN>(tdk, tdp, 64, smem_u32(ring + q * TILE), i != 0);
          if (few) product_rows<DC, TN>(tdk, tdp + 32, 64, smem_u32(ring + q * TILE), true);
          umma_commit(&s.empty[q]);
          if (i == steps - 1) umma_commit(&s.done[0]);
        }
        if (i + 1 < steps) dscores(i + 1);
        if (!ok) break;
      }
    }
    if (leader && *ab) drain_products(&s.drain[0], ab, status);
  } else {
    const int part = warp >> 2;
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const float c = C.scale * ATTN_LOG2E;
    const uint64_t c2 = pack2(c, c);
    Item it;
    uint32_t made = 0;
    bool ok = true;
    for (int n = 0; ok && get_item(s, n, status, it); ++n) {
      const int steps = per_head(it) * C.group, warp_row = it.t0 + (warp & 3) * 32, row = warp_row + lane;
      // Negative lse (in units of log 2) and delta of a step's 64 queries, for the four warps of this half: a warp brings 16 of them.
      Step st = first_step(it), ahead_st = st;
      auto fetch = [&](const Step& st) -> float {
        const int t = st.row + part * 64 + (warp & 3) * 16 + (lane & 15);
        const int64_t at = (int64_t)st.head * C.seqs.total + it.first + t;
        return t >= it.len ? 0.f : lane < 16 ? C.lse[at] : C.delta[at];
      };
      auto keep = [&](uint32_t k, float f) {
        s_rows[((k & 1) * (TN / 64) + part) * 128 + (lane >> 4) * 64 + (warp & 3) * 16 + (lane & 15)] = lane < 16 ? -f * ATTN_LOG2E : -f;
        warp_arrive(&s.rows_full[part][k & 1]);
      };
      keep(made, fetch(st));
      auto step = [&](int i, auto few) -> bool {
        advance(it, ahead_st);
        const float ahead = i + 1 < steps ? fetch(ahead_st) : 0.f;
        const float* mine = s_rows + ((made & 1) * (TN / 64) + part) * 128;
        ok = warp_wait(&s.rows_full[part][made & 1], (made >> 1) & 1, ab, status) && warp_wait(&s.scores[0], made & 1, ab, status);
        if (!ok) return false;
        tc_fence_after();
        const int base = st.row + part * 64;                       // first query of this warp's columns
        const bool cut = it.len - base < 64 || (C.causal && base < it.t0 + 128);
        const int lo = C.causal ? row - base : 0, hi = it.len - base;    // the columns that look at this key
        uint32_t a[64];
        tmem_ld64(ts + lanes + part * 64, a);
        uint32_t o[32];
#pragma unroll
        for (int e = 0; e < 32; e += 2) {
          const float4 f = *reinterpret_cast<const float4*>(mine + 2 * e);
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const int x = 2 * (e + h);
            float e0, e1;
            unpack2(fma2(pack2(__uint_as_float(a[x]), __uint_as_float(a[x + 1])), c2, h == 0 ? pack2(f.x, f.y) : pack2(f.z, f.w)), e0, e1);
            a[x] = __float_as_uint(attn_exp2(e0));
            a[x + 1] = __float_as_uint(attn_exp2(e1));
          }
        }
        if (cut) {
#pragma unroll
          for (int x = 0; x < 64; ++x) a[x] = x >= lo && x < hi ? a[x] : 0u;
        }
#pragma unroll
        for (int e = 0; e < 32; ++e) o[e] = pack_bf16(__uint_as_float(a[2 * e]), __uint_as_float(a[2 * e + 1]));
        tmem_st32(ts + lanes + part * 64, o);
        if constexpr (few.value) {
          uint32_t rest[32];
          low_parts(a, o, rest);
          tmem_st32(ts + lanes + part * 64 + 32, rest);
        }
        tmem_wait_st();
        tc_fence_before();
        warp_arrive(&s.ready[0]);
        if (base == 0 && (C.causal || it.len == 1)) a[0] = 0u;     // a query that sees one key: dS = 0
        ok = warp_wait(&s.dscores, made & 1, ab, status);
        if (!ok) return false;
        tc_fence_after();
        {
          uint32_t b[64];
          tmem_ld64(tdp + lanes + part * 64, b);
#pragma unroll
          for (int e = 0; e < 32; e += 2) {
            const float4 f = *reinterpret_cast<const float4*>(mine + 64 + 2 * e);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const int x = 2 * (e + h);
              float s0, s1;
              unpack2(mul2(pack2(__uint_as_float(a[x]), __uint_as_float(a[x + 1])),
                           add2(pack2(__uint_as_float(b[x]), __uint_as_float(b[x + 1])), h == 0 ? pack2(f.x, f.y) : pack2(f.z, f.w))), s0, s1);
              o[e + h] = pack_bf16(s0, s1);
              if constexpr (few.value) {
                b[x] = __float_as_uint(s0);
                b[x + 1] = __float_as_uint(s1);
              }
            }
          }
          if constexpr (few.value) {
            uint32_t rest[32];
            low_parts(b, o, rest);
            tmem_st32(tdp + lanes + part * 64 + 32, rest);
          }
        }
        tmem_st32(tdp + lanes + part * 64, o);
        tmem_wait_st();
        tc_fence_before();
        warp_arrive(&s.ready[1]);
        if (i + 1 < steps) keep(made + 1, ahead);
        st = ahead_st;
        return true;
      };
      const bool low = few_keys(it, C.causal);
      for (int i = 0; ok && i < steps; ++i, ++made)
        ok = low && st.row == 0 ? step(i, std::true_type()) : step(i, std::false_type());
      ok = ok && warp_wait(&s.done[0], n & 1, ab, status);
      if (!ok) break;
      // with eight warps one half stores dV, the other dK
      tc_fence_after();
#pragma unroll 1
      for (int which = WARPS == 4 ? 0 : part; which < (WARPS == 4 ? 2 : part + 1); ++which)
        store_rows<DC>((which == 0 ? tdv : tdk) + lanes, which == 0 ? C.dv : C.dk, (int64_t)it.first + warp_row, it.head, C.dim,
                       it.len - warp_row, which == 0 ? 1.0f : C.scale);
      tc_fence_before();
      warp_arrive(&s.acc_empty[0]);
    }
  }
  end(s, P, 4 * TN);
}

// --------------------------------------------------------------------------------------------- host
// [total, heads, dim] with a box of 64 columns of one head of `rows` tokens
bool attn_map(CUtensorMap* m, const Strided& x, int heads, int dim, int total, int rows) {
  const uint64_t dims[3] = {(uint64_t)dim, (uint64_t)heads, (uint64_t)total};
  // a stride along an extent of one is never used, but has to be a valid one
  const uint64_t strides[2] = {heads > 1 ? (uint64_t)x.head * 2 : 16, total > 1 ? (uint64_t)x.token * 2 : 16};
  const uint32_t box[3] = {64, 1, (uint32_t)rows};
  return make_map(m, x.p, 3, dims, strides, box);
}
bool addressable(const Strided& x, int heads, int total) {
  return ((uintptr_t)x.p & 15) == 0 && (total == 1 || (x.token % 8 == 0 && x.token > 0)) && (heads == 1 || (x.head % 8 == 0 && x.head > 0)) &&
         x.token < (1ll << 36) && x.head < (1ll << 36);
}
// shared memory beside the Shared struct
template <int DC, int HEADS> constexpr int FWD_BYTES = DC * (HEADS * CHUNK<128> + FWD_STAGES<DC, HEADS> * CHUNK<FWD_TN>);
template <int DC> constexpr int DQ_BYTES = DC * ((DC == 1 ? 3 : 2) * CHUNK<128> + BWD_STAGES<DC> * CHUNK<TN_OF<DC>> + 512) + 1024;
template <int DC> constexpr int DKV_BYTES = DC * (2 * CHUNK<128> + BWD_STAGES<DC> * CHUNK<TN_OF<DC>>) + 2 * (TN_OF<DC> / 64) * 512;
// A CTA of the dK, dV kernel holds TMEM while it waits for the dQ kernel's grid.  It must not come to an SM where that keeps a CTA of
// the latter from its columns: beside as many as fill TMEM there is no shared memory for it (nor for three of any kind here).
constexpr int SM_BYTES = 228 * 1024;
static_assert(BWD_CTAS<1> * DQ_BYTES<1> + DKV_BYTES<1> > SM_BYTES && BWD_CTAS<2> * DQ_BYTES<2> + DKV_BYTES<2> > SM_BYTES, "see above");
static_assert(3 * DKV_BYTES<1> > SM_BYTES && 3 * FWD_BYTES<1, 1> > SM_BYTES && DKV_BYTES<2> + FWD_BYTES<1, 1> > SM_BYTES, "see above");

template <typename... KArgs, typename... M>
cudaError_t run(void (*kernel)(KArgs...), bool after, int which, int bytes, int threads, int ctas, long tiles, const Attn* a,
                const AttnCall& c, cudaStream_t st, const M&... maps) {
  if (tiles + (long)ctas * a->num_sms > 0x7fffffffl) return cudaErrorInvalidValue;       // the counter's range
  const long grid = tiles < (long)ctas * a->num_sms ? tiles : (long)ctas * a->num_sms;
  const UmmaCall P = {c, a->next + 2 * which, a->wait_limit_ns, a->stall_once};
  return launch_maybe_after(after, kernel, dim3((unsigned)grid), dim3(threads), bytes + sizeof(Shared), st, maps..., P);
}
template <int DC>
cudaError_t backward(const Attn* a, const AttnCall& c, bool after, cudaStream_t st) {
  constexpr int TN = TN_OF<DC>;
  const int total = c.seqs.total, hq = c.heads_q, hk = c.heads_kv, d = c.dim;
  CUtensorMap q, g, o, k, v, qt, gt, kt, vt;         // tiles of 128 rows, and of TN
  if (!attn_map(&q, c.q, hq, d, total, 128) || !attn_map(&g, c.d_o, hq, d, total, 128) || !attn_map(&o, c.o, hq, d, total, 128) ||
      !attn_map(&kt, c.k, hk, d, total, TN) || !attn_map(&vt, c.v, hk, d, total, TN) || !attn_map(&qt, c.q, hq, d, total, TN) ||
      !attn_map(&gt, c.d_o, hq, d, total, TN) || !attn_map(&k, c.k, hk, d, total, 128) || !attn_map(&v, c.v, hk, d, total, 128))
    return cudaErrorInvalidValue;
  const long tiles = tile_bound(total, c.seqs.N, 128);
  const cudaError_t e = run(attn_dq_kernel<DC>, after, 1, DQ_BYTES<DC>, BWD_THREADS<DC>, BWD_CTAS<DC>, tiles * hq, a, c, st, q, g, o, kt, vt);
  if (e != cudaSuccess) return e;
  return run(attn_dkv_kernel<DC>, true, 2, DKV_BYTES<DC>, BWD_THREADS<DC>, BWD_CTAS<DC>, tiles * hk, a, c, st, qt, gt, k, v);
}

}  // namespace

cudaError_t attn_umma_prepare() {
  auto room = [](const void* kernel, int bytes) {
    return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes + (int)sizeof(Shared));
  };
  cudaError_t e = room((const void*)attn_fwd_kernel<1, 1>, FWD_BYTES<1, 1>);
  if (e == cudaSuccess) e = room((const void*)attn_fwd_kernel<2, 1>, FWD_BYTES<2, 1>);
  if (e == cudaSuccess) e = room((const void*)attn_fwd_kernel<2, 2>, FWD_BYTES<2, 2>);
  if (e == cudaSuccess) e = room((const void*)attn_dq_kernel<1>, DQ_BYTES<1>);
  if (e == cudaSuccess) e = room((const void*)attn_dq_kernel<2>, DQ_BYTES<2>);
  if (e == cudaSuccess) e = room((const void*)attn_dkv_kernel<1>, DKV_BYTES<1>);
  if (e == cudaSuccess) e = room((const void*)attn_dkv_kernel<2>, DKV_BYTES<2>);
  return e;
}

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
  if (!attn_map(&mq, c.q, c.heads_q, c.dim, total, 128) || !attn_map(&mk, c.k, c.heads_kv, c.dim, total, FWD_TN) ||
      !attn_map(&mv, c.v, c.heads_kv, c.dim, total, FWD_TN))
    return cudaErrorInvalidValue;
  const long tiles = tile_bound(total, c.seqs.N, 128) * c.heads_q;
  if (c.dim <= 64) return run(attn_fwd_kernel<1, 1>, false, 0, FWD_BYTES<1, 1>, FWD_THREADS<1>, 2, tiles, a, c, st, mq, mk, mv);
  if (c.group % 2 != 0) return run(attn_fwd_kernel<2, 1>, false, 0, FWD_BYTES<2, 1>, FWD_THREADS<1>, 2, tiles, a, c, st, mq, mk, mv);
  return run(attn_fwd_kernel<2, 2>, false, 0, FWD_BYTES<2, 2>, FWD_THREADS<2>, 1, tiles / 2, a, c, st, mq, mk, mv);
}

cudaError_t launch_attn_umma_bwd(const Attn* a, const AttnCall& c, cudaStream_t st) {
  const bool zeros = c.seqs.alive != nullptr && !c.skip_dropped;
  if (zeros) {
    const cudaError_t e = launch_attn_zero(a, c, st);
    if (e != cudaSuccess) return e;
  }
  return c.dim <= 64 ? backward<1>(a, c, zeros, st) : backward<2>(a, c, zeros, st);
}

}  // namespace vcas
