// What the attention kernels share: the handle, the tensors of a call, and how a CTA finds its part of a packed sequence.
#pragma once

#include "common.cuh"
#include "vcas_train.h"

namespace vcas {

struct Attn {
  vcas_attn_desc desc;
  int device, num_sms;
  float scale;
  bool tensor_ok;        // bf16 on a device with tcgen05
  void* base;
  size_t bytes;
  float* delta;          // [heads_q][max_tokens] rowsum(dO O)
  int32_t* next;         // tile counters of the tensor-core kernels, two for each
  int32_t* status;
  unsigned long long wait_limit_ns;
  int stall_once;
};

// The sequences of a call.  alive (with its length): the only ones that are worked on.
struct Seqs {
  const int32_t* starts;
  const int32_t* alive; const int32_t* alive_cnt;
  int N, total;
  int32_t* status;
};

struct Strided { const void* p; int64_t token, head; };

struct AttnCall {
  Seqs seqs;
  Strided q, k, v, o, d_o, dq, dk, dv;       // o is written by the forward, dq, dk and dv by the backward
  float* lse;                                // [heads_q][total]
  float* delta;                              // [heads_q][total]
  int heads_q, heads_kv, group, dim, causal;
  float scale;
  int skip_dropped;
};

constexpr float ATTN_LOG2E = 1.4426950408889634f, ATTN_LN2 = 0.6931471805599453f;

__device__ __forceinline__ float attn_exp2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

__device__ __forceinline__ bool seq_sane(const Seqs& q, int s, int e) { return s >= 0 && e >= s && e <= q.total; }
// Sequence n: its first token and length; 0 tokens and a note in the status word where starts make no sense there.
__device__ __forceinline__ int seq_length(const Seqs& q, int n, int& first) {
  const int s = __ldcg(q.starts + n), e = __ldcg(q.starts + n + 1);   // past L1: a kernel may begin beside the one before it
  first = s;
  if (!seq_sane(q, s, e)) {
    atomicExch(q.status, (int32_t)VCAS_ERR_BAD_ARG);
    return 0;
  }
  return e - s;
}
__device__ __forceinline__ int seq_count(const Seqs& q) {
  if (q.alive == nullptr) return q.N;
  const int c = __ldcg(q.alive_cnt);
  if (c >= 0 && c <= q.N) return c;
  atomicExch(q.status, (int32_t)VCAS_ERR_BAD_ARG);
  return 0;
}
// Entries of the list of sequences to be worked on count while they are in 0 .. N - 1 and above all entries before them.
// The part of seq_listed for lists that are not in order.  top: the largest entry so far, or -2 where all up to this block ascend.
// Returns the entry, or -1 where it does not count, and the new top.
__device__ __noinline__ inline int2 seq_listed_anyhow(int raw, int before, bool there, int N, int top, int lane, int32_t* status) {
  if (top == -2) top = __shfl_sync(0xffffffffu, before, 0);
  const bool in = there && raw >= 0 && raw < N;
  int below = __shfl_up_sync(0xffffffffu, in ? raw : -1, 1);
  below = lane == 0 ? top : max(below, top);
#pragma unroll 1
  for (int o = 1; o < 32; o <<= 1) {
    const int v = __shfl_up_sync(0xffffffffu, below, o);
    if (lane >= o) below = max(below, v);
  }
  if (there && !(in && raw > below)) atomicExch(status, (int32_t)VCAS_ERR_BAD_ARG);
  return make_int2(in && raw > below ? raw : -1, max(top, __reduce_max_sync(0xffffffffu, in ? raw : -1)));
}
// Entry k of the list, a lane's own of 32 one behind the other, by a full warp that goes through the list from its beginning (top: -2
// there); -1 behind its end and, with a note, where it does not count.
__device__ __forceinline__ int seq_listed(const Seqs& q, int k, int count, int lane, int& top) {
  const bool there = k < count;
  if (q.alive == nullptr) return there ? k : -1;
  const int n = there ? __ldcg(q.alive + k) : -1, before = there && k > 0 ? __ldcg(q.alive + k - 1) : -1;
  if (top == -2 && __all_sync(0xffffffffu, (n < q.N && n > before) || !there)) return n;
  const int2 r = seq_listed_anyhow(n, before, there, q.N, top, lane, q.status);
  top = r.y;
  return r.x;
}

// Tile number `tile` of all sequences cut into tiles of `rows` tokens, sequence by sequence: its sequence's first token and length, and
// its place in the sequence.  By one full warp, 32 sequences at a time; false where there are not that many tiles.
__device__ __forceinline__ bool find_tile(const Seqs& q, int tile, int rows, int lane, int& first, int& len, int& place) {
  const int count = seq_count(q);
  int before = 0, top = -2;
  for (int b = 0; b < count; b += 32) {
    const int n = seq_listed(q, b + lane, count, lane, top);
    int s = 0, l = 0;
    if (n >= 0) l = seq_length(q, n, s);
    const int tiles = (l + rows - 1) / rows;
    int upto = tiles;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int v = __shfl_up_sync(0xffffffffu, upto, o);
      if (lane >= o) upto += v;
    }
    const unsigned hit = __ballot_sync(0xffffffffu, tile < before + upto);
    if (hit != 0) {
      const int at = __ffs(hit) - 1;
      first = __shfl_sync(0xffffffffu, s, at);
      len = __shfl_sync(0xffffffffu, l, at);
      place = tile - before - __shfl_sync(0xffffffffu, upto - tiles, at);
      return true;
    }
    before += __shfl_sync(0xffffffffu, upto, 31);
  }
  return false;
}

// The order in which tiles of 128 rows are worked on: the most work first, so that all CTAs end at about the same time (in the order of
// the sequences the longest CTA of a packed backward had 22 % more tiles than the median).  A tile of a causal call has as much
// work as there are tiles on the other side that it sees: each sequence of L tiles has one tile of every amount from 1 to L, in the
// forward's and dQ's direction the amount-th, in the other one counted from its end.  Without a mask the tiles of a sequence have L each.
// One warp holds the lengths of up to 128 sequences; more are taken as they come.
struct Order {
  static constexpr int SLOTS = 4;
  int first[SLOTS], len[SLOTS], tiles[SLOTS];
  bool sorted, causal, keys;
  __device__ __forceinline__ Order(const Seqs& q, int lane, bool causal_, bool keys_) : causal(causal_), keys(keys_) {
    const int count = seq_count(q);
    sorted = count <= 32 * SLOTS;
    bool astray = false;                 // lists that are not in order: as find_tile goes through them
#pragma unroll
    for (int i = 0; i < SLOTS; ++i) {
      first[i] = len[i] = 0;
      const int k = 32 * i + lane;
      if (sorted && k < count) {
        const int n = q.alive == nullptr ? k : __ldcg(q.alive + k), before = q.alive == nullptr || k == 0 ? -1 : __ldcg(q.alive + k - 1);
        if (n < q.N && n > before) len[i] = seq_length(q, n, first[i]); else astray = true;
      }
      tiles[i] = (len[i] + 127) / 128;
    }
    if (__any_sync(0xffffffffu, astray)) sorted = false;
    // sequences of one length: in their order, whose tiles share more in L2 (8 x 2048 tokens forward: 283 us, sorted 291)
    int most = 0, least = 1 << 30;
#pragma unroll
    for (int i = 0; i < SLOTS; ++i) {
      most = max(most, tiles[i]);
      if (tiles[i] > 0) least = min(least, tiles[i]);
    }
    if (__reduce_max_sync(0xffffffffu, most) <= __reduce_min_sync(0xffffffffu, least)) sorted = false;
  }
  // tiles with more work than w
  __device__ __forceinline__ int above(int w) const {
    int sum = 0;
#pragma unroll
    for (int i = 0; i < SLOTS; ++i) sum += causal ? max(tiles[i] - w, 0) : tiles[i] > w ? tiles[i] : 0;
    return __reduce_add_sync(0xffffffffu, sum);
  }
  // Tile number t: its sequence's first token and length, and its place in the sequence.  By a full warp; false: there are not that many.
  __device__ __forceinline__ bool find(const Seqs& q, int t, int lane, int& first_, int& len_, int& place) const {
    if (!sorted) {
      if (!find_tile(q, t, 128, lane, first_, len_, place)) return false;
      if (causal && !keys) place = (len_ + 127) / 128 - 1 - place;         // a sequence's longest first
      return true;
    }
    if (t >= above(0)) return false;
    int lo = 1, hi = 1;                  // the work of tile t: the least w with no more than t tiles above it
#pragma unroll
    for (int i = 0; i < SLOTS; ++i) hi = max(hi, tiles[i]);
    hi = __reduce_max_sync(0xffffffffu, hi);
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (above(mid) <= t) hi = mid; else lo = mid + 1;
    }
    const int w = lo;
    int rank = t - above(w), in = 0;     // among the tiles of this work; place in the sequence where all have it
    if (!causal) { in = rank % w; rank /= w; }
#pragma unroll
    for (int i = 0; i < SLOTS; ++i) {
      const bool mine = causal ? tiles[i] >= w : tiles[i] == w;
      const unsigned has = __ballot_sync(0xffffffffu, mine);
      const int here = __popc(has);
      if (rank < here) {
        const int from = __ffs(__ballot_sync(0xffffffffu, mine && __popc(has & ((1u << lane) - 1u)) == rank)) - 1;
        first_ = __shfl_sync(0xffffffffu, first[i], from);
        len_ = __shfl_sync(0xffffffffu, len[i], from);
        place = !causal ? in : keys ? (len_ + 127) / 128 - w : w - 1;
        return true;
      }
      rank -= here;
    }
    return false;
  }
};

// No more tiles than these exist where sequences do not overlap: a sequence adds one that is not full at most.  If one is left out, or
// there are more than tokens, one tile is not found, and looking for it sees every sequence (what is wrong with any is noted).
inline long tile_bound(int total, int N, int rows) { return total / rows + (N < total ? N : total + 1); }

cudaError_t attn_fma_prepare();
cudaError_t launch_attn_fma_fwd(const Attn* a, const AttnCall& c, cudaStream_t st);
cudaError_t launch_attn_fma_bwd(const Attn* a, const AttnCall& c, cudaStream_t st);
// Zeros into dq, dk, dv on the rows of the sequences that are not worked on.
cudaError_t launch_attn_zero(const Attn* a, const AttnCall& c, cudaStream_t st);
cudaError_t attn_umma_prepare();         // on the current device, before the first launch there
bool attn_umma_ok(const Attn* a, const AttnCall& c, bool backward);
cudaError_t launch_attn_umma_fwd(const Attn* a, const AttnCall& c, cudaStream_t st);
cudaError_t launch_attn_umma_bwd(const Attn* a, const AttnCall& c, cudaStream_t st);

}  // namespace vcas
