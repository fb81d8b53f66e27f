// Append to and eviction from the paged key-value cache.
#pragma once
#include "cluster.cuh"
#include "paged_common.cuh"

namespace lsp {

// ---- append --------------------------------------------------------------------------------------------------------------
// Row i of sequence b (packed row row_off[b] + i) goes to slot lens[b] + i.  Bound by HBM for prompts and by latency for single
// tokens: a block has its rows under way to registers (16 KB, a row or as many as that is) while it finds their places (offsets -> lengths ->
// pages).  (Longer-lived blocks, a warp a half row at a time, were slower: 3063 rows of 16 KB 24.6 us where these took
// 19.8; 18.6 now, 12264 rows 56.6 = 6.4 TB/s.)
constexpr int PP_THREADS = 256;
constexpr int PP_VEC = 4;               // 16-byte pieces of a thread that are under way at once
constexpr int PP_ROWS = 32;             // rows of a block at most

struct PagedAppendArgs {
  PagedView pv;
  const char *k_new, *v_new;
  long long ld_new;                     // bytes
  const int *lens, *row_off, *seen;
  int max_rows, n_rows, esz, head_bytes;      // head_bytes = head_dim * esz
  int rows_block;                       // rows of a block
  int* lens_out;
  int* seen_out;
  float* weights;
  int* pos;
};

// All rows of a call whose offsets descend somewhere (so there are bad ones), by one block, a sequence with good offsets after another.  Such offsets
// cannot be searched: the other blocks' search for a row's sequence misses rows, and the good offsets may name a row more than once.  (What the
// others do write is right, and the same.)
__device__ __forceinline__ void pp_any_order(const PagedAppendArgs& a) {
  const int cap = pg_capacity(a.pv), head_pieces = a.head_bytes / 16, pieces = a.pv.hkv * head_pieces;
#pragma unroll 1
  for (int b = 0; b < a.pv.batch; ++b) {
    const RowSpan rs = pg_rows(a.pv, a.row_off, b, a.max_rows, a.n_rows);
    const int len = pg_len(a.pv, a.lens[b]);
#pragma unroll 1
    for (int r = 0; r < min(rs.n, cap - len); ++r) {
      const long long at = pg_slot(a.pv, b, len + r);
      if (at < 0) continue;
#pragma unroll 1
      for (int c = threadIdx.x; c < 2 * pieces; c += PP_THREADS) {
        const int v = c >= pieces ? 1 : 0, p = c - v * pieces, h = p / head_pieces;
        char* dst = (v ? a.pv.v : a.pv.k) + (at + (long long)h * a.pv.head_stride) * a.esz + (p - h * head_pieces) * 16;
        *reinterpret_cast<uint4*>(dst) = reinterpret_cast<const uint4*>((v ? a.v_new : a.k_new) + (long long)(rs.first + r) * a.ld_new)[p];
      }
#pragma unroll 1
      for (int h = threadIdx.x; h < a.pv.hkv; h += PP_THREADS) {
        const long long x = ((long long)b * a.pv.hkv + h) * cap + len + r;
        if (a.weights) a.weights[x] = 0.f;
        if (a.pos) a.pos[x] = a.seen ? a.seen[b] + r : len + r;
      }
    }
  }
}

// Blocks ahead of the last: rows_block packed rows each.  The last block: the lengths, and what the others miss where offsets descend.
// (Five blocks an SM, 48 registers: with 40 16 x 1000 rows of 512 bytes took 6.2 us, with 64 7.4, so 5.6.)
__global__ void __launch_bounds__(PP_THREADS, 5) k_paged_append(const PagedAppendArgs a) {
  extern __shared__ int offsets[];      // [batch] row_off, [batch] lens (with offsets: a row's sequence is searched for)
  __shared__ int seqs[PP_ROWS], slots[PP_ROWS], poss[PP_ROWS];
  __shared__ long long places[PP_ROWS]; // bytes, -1: nowhere
  const int B = a.pv.batch, cap = pg_capacity(a.pv);
  pdl_release();
  pg_prefetch_table(a.pv);
  pg_prefetch_grid(a.lens, B * 4);
  pdl_wait();
  if (blockIdx.x == gridDim.x - 1) {
    bool descend = false;
    for (int b = threadIdx.x; b < B; b += PP_THREADS) {
      const RowSpan rs = pg_rows(a.pv, a.row_off, b, a.max_rows, a.n_rows);
      const int n = pg_len(a.pv, a.lens[b]);
      int fit = rs.n;
      if (fit > cap - n) {
        pg_flag(a.pv, PG_BAD_LEN);
        fit = cap - n;
      }
      a.lens_out[b] = n + fit;
      if (a.seen_out) a.seen_out[b] = a.seen[b] + fit;
      descend |= a.row_off && a.row_off[b] > a.row_off[b + 1];
    }
    if (a.row_off && __syncthreads_or(descend)) pp_any_order(a);
    return;
  }
  const int r0 = blockIdx.x * a.rows_block, n = min(a.rows_block, a.n_rows - r0);
  const int pieces = a.pv.hkv * a.head_bytes / 16, total = n * 2 * pieces;      // of a row's K or V; of the block
  // piece c of the block: row, K or V, piece of that
  struct Piece { int row, v, c; };
  auto piece = [&](int c) {
    Piece p;
    p.row = a.rows_block == 1 ? 0 : c / (2 * pieces);
    p.c = c - p.row * 2 * pieces;
    p.v = p.c >= pieces ? 1 : 0;
    p.c -= p.v ? pieces : 0;
    return p;
  };
  auto load = [&](int c) {
    const Piece p = piece(c);
    return reinterpret_cast<const uint4*>((p.v ? a.v_new : a.k_new) + (long long)(r0 + p.row) * a.ld_new)[p.c];
  };
  uint4 x[PP_VEC];
#pragma unroll
  for (int i = 0; i < PP_VEC; ++i) {
    const int c = i * PP_THREADS + threadIdx.x;
    if (c < total) x[i] = load(c);
  }
  if (a.row_off) {
    for (int b = threadIdx.x; b < B; b += PP_THREADS) {
      offsets[b] = a.row_off[b];
      offsets[B + b] = a.lens[b];
    }
    __syncthreads();
  }
  if (threadIdx.x < n) {
    const int r = r0 + threadIdx.x;
    long long place = -1;
    int b, slot = 0, position = 0;
    if (!a.row_off) {
      b = r / a.max_rows;
    } else {                            // the last sequence that starts at or ahead of the row (of those that start there, the one with rows)
      int lo = -1, up = B;
      while (up - lo > 1) {
        const int mid = (lo + up) >> 1;
        if (offsets[mid] <= r) lo = mid; else up = mid;
      }
      b = lo;
    }
    if (b >= 0) {
      const RowSpan rs = pg_rows(a.pv, a.row_off, b, a.max_rows, a.n_rows);
      const int len = pg_len(a.pv, a.row_off ? offsets[B + b] : a.lens[b]), i = r - rs.first;
      if (i >= 0 && i < rs.n && len + i < cap) {
        slot = len + i;
        place = pg_slot(a.pv, b, slot);
        if (place >= 0) place *= a.esz;
        position = a.seen ? a.seen[b] + i : slot;
      }
    }
    places[threadIdx.x] = place;
    seqs[threadIdx.x] = b;
    slots[threadIdx.x] = slot;
    poss[threadIdx.x] = position;
  }
  __syncthreads();
  const int shift = 31 - __clz(a.head_bytes / 16);    // pieces of a head: 8, 16 or 32
  for (int c0 = threadIdx.x; c0 < total; c0 += PP_VEC * PP_THREADS) {
    if (c0 >= PP_VEC * PP_THREADS) {
#pragma unroll
      for (int i = 0; i < PP_VEC; ++i)
        if (c0 + i * PP_THREADS < total) x[i] = load(c0 + i * PP_THREADS);
    }
#pragma unroll
    for (int i = 0; i < PP_VEC; ++i) {
      if (c0 + i * PP_THREADS >= total) break;
      const Piece p = piece(c0 + i * PP_THREADS);
      const long long place = places[p.row];
      if (place < 0) continue;
      char* dst = (p.v ? a.pv.v : a.pv.k) + place + (long long)(p.c >> shift) * a.pv.head_stride * a.esz + (p.c & ((1 << shift) - 1)) * 16;
      *reinterpret_cast<uint4*>(dst) = x[i];
    }
  }
  if (a.weights || a.pos)
    for (int i = threadIdx.x; i < n * a.pv.hkv; i += PP_THREADS) {
      const int r = i % n, h = i / n;                // (rows of a sequence lie one behind the other in a head's array)
      if (places[r] < 0) continue;
      const long long at = ((long long)seqs[r] * a.pv.hkv + h) * cap + slots[r];
      if (a.weights) a.weights[at] = 0.f;
      if (a.pos) a.pos[at] = poss[r];
    }
}

// ---- eviction ------------------------------------------------------------------------------------------------------------
// Selection, a cluster of CTAs per (sequence, KV head): the budget smallest of the keys (falling weight, position), by radix selection; then
// the kept slots as a bitmap, whose counts give every slot that moves its partner: the i-th kept slot behind the budget goes to the i-th
// freed slot ahead of it.  Sources and targets are disjoint, so k_paged_move needs no order between its blocks.
// Each CTA of the cluster has a run of the slots, their weights, positions and keys in shared memory (read from global memory once); a digit's
// counts are added over distributed shared memory.  Bound by the chain of passes: a digit costs 1.3 us (a read of the keys from shared memory
// and four barriers; with a cluster 2.5).
constexpr int PE_MAX_CAP = 1 << 20;     // slots of a sequence: a bitmap of 128 KB
constexpr int PE_BITS = 11, PE_BINS = 1 << PE_BITS;      // a digit
constexpr int PE_CLUSTER = 8;           // CTAs of a unit at most
constexpr int PE_KEYS = 13 * 1024;      // slots of a CTA whose weights, positions and keys fit shared memory; beyond that a pass reads them again
constexpr int PM_WARPS = 8;
constexpr int PM_PAIRS = 4;             // pairs of a warp that are under way at once

struct PagedEvictArgs {
  PagedView pv;
  const float* weights;
  const int *pos, *lens, *seen;
  int budget, n_sink, n_recent, max_moves;
  float* weights_out;
  int* pos_out;
  int* lens_out;
  int* moves;                  // [batch * hkv][1 + 2 max_moves]: count, sources, targets
  int head_bytes, esz;
  int cluster, slots, in_smem; // CTAs of a unit, most slots of one (a multiple of 32), weights, positions and keys are kept in shared memory
};

// Order of the weights, heaviest first: 0 = protected, then falling weight (-0 as 0), NaN last.
__device__ __forceinline__ unsigned pe_key(float w) {
  if (w != w) return 0xffffffffu;
  unsigned u = __float_as_uint(w == 0.f ? 0.f : w);
  u = (u >> 31) ? ~u : u | 0x80000000u;       // ascending with w
  return ~u;                                  // +inf: 0x007fffff
}

// x and y of this thread added up over the threads before it; all: over all of the block's.
template <int THREADS>
__device__ __forceinline__ int2 pe_sums_before(int2 v, int2* warp_sums, int2& all) {
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  auto scan = [&](int2 x) {
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int p = __shfl_up_sync(0xffffffffu, x.x, o), q = __shfl_up_sync(0xffffffffu, x.y, o);
      if (lane >= o) {
        x.x += p;
        x.y += q;
      }
    }
    return x;
  };
  const int2 x = scan(v);
  __syncthreads();
  if (lane == 31) warp_sums[w] = x;
  __syncthreads();
  const int2 s = lane < THREADS / 32 ? warp_sums[lane] : make_int2(0, 0), t = scan(s);      // every warp adds the sums up for itself
  all = make_int2(__shfl_sync(0xffffffffu, t.x, 31), __shfl_sync(0xffffffffu, t.y, 31));
  return make_int2(x.x - v.x + __shfl_sync(0xffffffffu, t.x - s.x, w), x.y - v.y + __shfl_sync(0xffffffffu, t.y - s.y, w));
}

// x of this lane added up over the lanes before it.
__device__ __forceinline__ int pe_warp_sum_before(int x) {
  int y = x;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int p = __shfl_up_sync(0xffffffffu, y, o);
    if ((int)(threadIdx.x & 31) >= o) y += p;
  }
  return y - x;
}

// Words of shared memory of another CTA of the cluster.
__device__ __forceinline__ int ld_cluster_s32(uint32_t addr) {
  int v;
  asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
  return v;
}
__device__ __forceinline__ int2 ld_cluster_s32x2(uint32_t addr) {
  int2 v;
  asm volatile("ld.shared::cluster.v2.s32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(addr) : "memory");
  return v;
}
__device__ __forceinline__ uint4 ld_cluster_u4(uint32_t addr) {
  uint4 v;
  asm volatile("ld.shared::cluster.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
  return v;
}

// Shared memory of a selection, in words: counts, weights, positions and keys, bitmap, holes and movers ahead of each of its words.
__host__ __device__ inline int pe_words(int slots, int in_smem) { return 2 * PE_BINS + slots / 32 * 3 + 4 + (in_smem ? 3 * slots : 0); }

// What moves of a unit, the pairs (source[i], target[i]): weight, position and rows, by n_warps warps, this one the w-th.  A warp takes PM_PAIRS
// pairs at a time; the K row in the first half of the lanes, the V row in the second (rows of 512 bytes in two turns).  A turn's rows are under
// way while the next one's pages, and the slots of the one behind it, are looked up: without that the chain of the reads is what a warp waits
// for.
__device__ __forceinline__ void pe_move(const PagedEvictArgs& a, int unit, const int* source, const int* target, int n, int w, int n_warps) {
  const int b = unit / a.pv.hkv, kvh = unit % a.pv.hkv, lane = threadIdx.x & 31;
  const int* list = lane < PM_PAIRS ? source : target;      // lanes 0 .. 3: sources, lanes 4 .. 7: targets
  const int step = n_warps * PM_PAIRS;
  int i0 = w * PM_PAIRS;
  if (i0 >= n) return;
  const int cap = pg_capacity(a.pv);
  auto slot = [&](int i) {
    i += lane % PM_PAIRS;
    const int j = lane < 2 * PM_PAIRS && i < n ? list[i] : -1;
    return j < cap ? j : -1;
  };
  const long long base = (long long)unit * cap;
  auto offset = [&](int j) -> long long {
    const long long at = j >= 0 ? pg_slot(a.pv, b, j) : -1;
    return at < 0 ? -1 : (at + (long long)kvh * a.pv.head_stride) * a.esz;
  };
  int j = slot(i0), j2 = slot(i0 + step);
  long long off = offset(j);
  char* pool = lane < 16 ? a.pv.k : a.pv.v;
  for (; i0 < n; i0 += step) {
    const int to_slot = __shfl_down_sync(0xffffffffu, j, PM_PAIRS);
    long long from[PM_PAIRS], to[PM_PAIRS];
#pragma unroll
    for (int i = 0; i < PM_PAIRS; ++i) {
      from[i] = __shfl_sync(0xffffffffu, off, i);
      to[i] = __shfl_sync(0xffffffffu, off, PM_PAIRS + i);
      if (from[i] < 0) to[i] = -1;
    }
    const int c0 = (lane & 15) * 16;
    uint4 x[PM_PAIRS];
#pragma unroll
    for (int i = 0; i < PM_PAIRS; ++i)
      if (to[i] >= 0 && c0 < a.head_bytes) x[i] = *reinterpret_cast<const uint4*>(pool + from[i] + c0);
    const bool mine = lane < PM_PAIRS && j >= 0 && to_slot >= 0;
    float weight = mine ? a.weights[base + j] : 0.f;
    int p = mine && a.pos ? a.pos[base + j] : j;
    bool moved = true;
#pragma unroll
    for (int i = 0; i < PM_PAIRS; ++i) moved = lane == i ? to[i] >= 0 : moved;
    const int j3 = slot(i0 + 2 * step);
    const long long off2 = offset(j2);
#pragma unroll
    for (int i = 0; i < PM_PAIRS; ++i)
      if (to[i] >= 0 && c0 < a.head_bytes) *reinterpret_cast<uint4*>(pool + to[i] + c0) = x[i];
    if (c0 + 256 < a.head_bytes) {
#pragma unroll
      for (int i = 0; i < PM_PAIRS; ++i)
        if (to[i] >= 0) x[i] = *reinterpret_cast<const uint4*>(pool + from[i] + c0 + 256);
#pragma unroll
      for (int i = 0; i < PM_PAIRS; ++i)
        if (to[i] >= 0) *reinterpret_cast<uint4*>(pool + to[i] + c0 + 256) = x[i];
    }
    if (mine && !moved) {                            // a slot of the pair has no page: the one ahead keeps what is in it
      weight = a.weights[base + to_slot];
      p = a.pos ? a.pos[base + to_slot] : to_slot;
    }
    if (mine) {
      a.weights_out[base + to_slot] = weight;
      if (a.pos_out) a.pos_out[base + to_slot] = p;
    }
    j = j2;
    j2 = j3;
    off = off2;
  }
}

// MOVE: the CTA moves what it selected (one CTA a unit); else k_paged_move does.
template <int THREADS, bool MOVE>
__global__ void __launch_bounds__(THREADS) k_paged_select(const PagedEvictArgs a) {
  extern __shared__ __align__(16) unsigned pe_smem[];
  // behind two sets of counts: weights, positions and keys [slots], if they are kept here; kept slots of this CTA [slots / 32]
  float* own_weights = reinterpret_cast<float*>(pe_smem + 2 * PE_BINS);
  int* own_pos = reinterpret_cast<int*>(own_weights + a.slots);
  unsigned* own_keys = reinterpret_cast<unsigned*>(own_pos + a.slots);
  unsigned* bits = pe_smem + 2 * PE_BINS + (a.in_smem ? 3 * a.slots : 0);
  int* holes_at = reinterpret_cast<int*>(bits + a.slots / 32);
  int* movers_at = holes_at + a.slots / 32;
  __shared__ int2 warp_sums[32];
  __shared__ __align__(16) int found[4], shared_counts[4];
  __shared__ unsigned warp_or[32], the_value;
  __shared__ uint2 bits_of[2][32];
  __shared__ int groups_of[2][PE_BINS / 64];
  int turn = 0;
  const int CL = MOVE ? 1 : a.cluster, rank = CL > 1 ? (int)cluster_ctarank() : 0, tid = threadIdx.x, lane = tid & 31;
  auto barrier = [&]() { if (CL > 1) cluster_sync(); else __syncthreads(); };
  const int unit = blockIdx.x / CL, b = unit / a.pv.hkv, cap = pg_capacity(a.pv);
  const long long base = (long long)unit * cap;
  pdl_release();
  {
    // (a sequence to thin has more slots than the budget; of the others fewer are read)
    const long long bytes = (long long)min(cap, a.budget) * 4;
    pg_prefetch_grid(a.lens, a.pv.batch * 4);
    pg_prefetch(a.weights + base, bytes, tid + rank * THREADS, CL * THREADS);
    if (a.pos) pg_prefetch(a.pos + base, bytes, tid + rank * THREADS, CL * THREADS);
    pg_prefetch_table(a.pv);
  }
  pdl_wait();
  const int n = pg_len(a.pv, a.lens[b]);
  int* moves = a.moves + (long long)unit * (1 + 2 * (long long)a.max_moves);
  if (unit % a.pv.hkv == 0 && rank == 0 && tid == 0) a.lens_out[b] = min(n, a.budget);
  // this CTA's slots: [s0, s0 + ns)
  const int run = ((n + 31) / 32 + CL - 1) / CL * 32, s0 = min(n, rank * run), ns = min(n, s0 + run) - s0;
  const float* weights = a.weights + base + s0;
  const int* pos = a.pos ? a.pos + base + s0 : nullptr;
  float* weights_out = a.weights_out + base + s0;
  int* pos_out = a.pos_out ? a.pos_out + base + s0 : nullptr;
  if (n <= a.budget) {
    if (!MOVE && rank == 0 && tid == 0) moves[0] = 0;
    for (int j = tid; j < ns; j += THREADS) {
      weights_out[j] = weights[j];
      if (pos_out) pos_out[j] = pos ? pos[j] : s0 + j;
    }
    return;
  }
  const int seen = a.seen ? a.seen[b] : n;
  auto key_of = [&](int p, float w) { return (p < a.n_sink || p >= seen - a.n_recent) ? 0u : pe_key(w); };
  unsigned any = 0;                                // bits that some position has
  if (a.in_smem) {
    // four slots a load where a KV head's array begins on 16 bytes, the last ones one by one
    const bool by4 = (cap & 3) == 0 && (((uintptr_t)weights | (uintptr_t)pos) & 15) == 0;
    const int ahead4 = by4 ? ns / 4 : 0;
#pragma unroll 2
    for (int i = tid; i < ahead4; i += THREADS) {
      const float4 w = reinterpret_cast<const float4*>(weights)[i];
      const int j = s0 + 4 * i;
      const int4 p = pos ? reinterpret_cast<const int4*>(pos)[i] : make_int4(j, j + 1, j + 2, j + 3);
      reinterpret_cast<float4*>(own_weights)[i] = w;
      reinterpret_cast<int4*>(own_pos)[i] = p;
      reinterpret_cast<uint4*>(own_keys)[i] = make_uint4(key_of(p.x, w.x), key_of(p.y, w.y), key_of(p.z, w.z), key_of(p.w, w.w));
      any |= (unsigned)(p.x | p.y | p.z | p.w);
    }
#pragma unroll 4
    for (int j = 4 * ahead4 + tid; j < ns; j += THREADS) {
      const int p = pos ? pos[j] : s0 + j;
      const float w = weights[j];
      own_weights[j] = w;
      own_pos[j] = p;
      own_keys[j] = key_of(p, w);
      any |= (unsigned)p;
    }
  } else {
    for (int j = tid; j < ns; j += THREADS) any |= (unsigned)(pos ? pos[j] : s0 + j);
  }
  auto pos_of = [&](int j) { return a.in_smem ? own_pos[j] : pos ? pos[j] : s0 + j; };
  auto weight_of = [&](int j) { return a.in_smem ? own_weights[j] : weights[j]; };
  auto key = [&](int j) { return a.in_smem ? own_keys[j] : key_of(pos_of(j), weight_of(j)); };
  any = __reduce_or_sync(0xffffffffu, any);
  if (lane == 0) warp_or[tid >> 5] = any;
  // The need-th smallest value of at most `width` bits that `get` gives for the slots it says true of: the value, how many are below it, how many
  // equal it.  (Where all values of a prefix are wanted, the rest of the digits are: value = the largest with that prefix.)
  auto select = [&](auto get, int width, int need, unsigned& value, int& below, int& equal) {
    unsigned prefix = 0, mask = width == 32 ? 0u : ~0u << width;
    below = 0;
#pragma unroll 1
    for (int shift = max(0, width - PE_BITS);; shift = max(0, shift - PE_BITS)) {
      const unsigned digit = ~mask >> shift;         // mask of the digit's bits (the last one may be shorter)
      turn ^= 1;                                     // two sets of counts in turn: another CTA may still be reading the last pass's
      unsigned* hist = pe_smem + turn * PE_BINS;
      int* groups = groups_of[turn];
#pragma unroll
      for (int i = tid; i < PE_BINS / 4; i += THREADS) reinterpret_cast<uint4*>(hist)[i] = make_uint4(0, 0, 0, 0);
      __syncthreads();
      // Between the first and the last digit: bits that all / some of the values counted here have.  Where one value is all there is (slots that
      // nobody attends to weigh 0) no further digit is needed.
      const bool look = CL == 1 && shift > 0 && shift + PE_BITS < width;
      unsigned all_of = 0xffffffffu, some_of = 0;
#pragma unroll 4
      for (int j = tid; j < ns; j += THREADS) {
        unsigned k;
        if (get(j, k) && (k & mask) == prefix) {
          atomicAdd(&hist[(k >> shift) & digit], 1u);
          all_of &= k;
          some_of |= k;
        }
      }
      if (look) {
        all_of = __reduce_and_sync(0xffffffffu, all_of);
        some_of = __reduce_or_sync(0xffffffffu, some_of);
        if (lane == 0) bits_of[turn][tid >> 5] = make_uint2(all_of, some_of);
      }
      __syncthreads();
      // counts of 64 bins each, a warp a group; the first warp finds the group in which the need-th lies, then the bin
      for (int g = tid >> 5; g < PE_BINS / 64; g += THREADS / 32) {
        const uint2 x = reinterpret_cast<const uint2*>(hist)[g * 32 + lane];
        const unsigned s = __reduce_add_sync(0xffffffffu, x.x + x.y);
        if (lane == 0) groups[g] = s;
      }
      barrier();
      if (tid < 32) {
        const int want = need - below;               // rank, from 1, among what is left
        int x = CL == 1 ? groups[lane] : 0;
        if (CL > 1) {
          int y[PE_CLUSTER];
#pragma unroll
          for (int r = 0; r < PE_CLUSTER; ++r) y[r] = r < CL ? ld_cluster_s32(cluster_map(smem_u32(groups + lane), r)) : 0;
#pragma unroll
          for (int r = 0; r < PE_CLUSTER; ++r) x += y[r];
        }
        int up = pe_warp_sum_before(x) + x;
        const int g = __ffs(__ballot_sync(0xffffffffu, want <= up) | 0x80000000u) - 1, base_g = __shfl_sync(0xffffffffu, up - x, g);
        int2 h = make_int2(0, 0);
        const unsigned* mine = hist + g * 64 + lane * 2;
        if (CL == 1) {
          h = *reinterpret_cast<const int2*>(mine);
        } else {
          int2 y[PE_CLUSTER];
#pragma unroll
          for (int r = 0; r < PE_CLUSTER; ++r) y[r] = r < CL ? ld_cluster_s32x2(cluster_map(smem_u32(mine), r)) : make_int2(0, 0);
#pragma unroll
          for (int r = 0; r < PE_CLUSTER; ++r) {
            h.x += y[r].x;
            h.y += y[r].y;
          }
        }
        up = base_g + pe_warp_sum_before(h.x + h.y) + h.x + h.y;
        const int l = __ffs(__ballot_sync(0xffffffffu, want <= up) | 0x80000000u) - 1;
        if (lane == l) {
          const int before = up - h.x - h.y;
          const bool second = want > before + h.x;
          found[0] = g * 64 + lane * 2 + (second ? 1 : 0);
          found[1] = second ? before + h.x : before;
          found[2] = second ? h.y : h.x;
        }
        if (look) {
          const uint2 x = lane < THREADS / 32 ? bits_of[turn][lane] : make_uint2(0xffffffffu, 0u);
          all_of = __reduce_and_sync(0xffffffffu, x.x);
          some_of = __reduce_or_sync(0xffffffffu, x.y);
          if (lane == 0) {
            found[3] = all_of == some_of;
            the_value = all_of;
          }
        }
      }
      __syncthreads();
      if (look && found[3]) {
        prefix = the_value;
        mask = 0xffffffffu;
        below += found[1];
        equal = found[2];
        break;
      }
      prefix |= (unsigned)found[0] << shift;
      mask |= digit << shift;
      below += found[1];
      equal = found[2];
      if (shift == 0 || below + equal == need) break;
    }
    value = prefix | ~mask;
  };
  unsigned key_at, pos_at = 0xffffffffu, slot_at = 0xffffffffu, flip = 0;
  int below, equal;
  select([&](int j, unsigned& k) { k = key(j); return true; }, 32, a.budget, key_at, below, equal);
  const bool ties = below + equal > a.budget;
  if (ties) {                                       // ties of the weight: the lower positions
    unsigned bits_used = 0;
    for (int i = 0; i < THREADS / 32; ++i) bits_used |= warp_or[i];
    if (CL > 1) {
      if (tid == 0) shared_counts[2] = (int)bits_used;
      cluster_sync();
      for (int r = 0; r < CL; ++r) bits_used |= ld_cluster_u4(cluster_map(smem_u32(shared_counts), r)).z;
    }
    flip = bits_used & 0x80000000u;                 // (negative positions are lower than others)
    int need = a.budget - below;
    select([&](int j, unsigned& k) { const bool tie = key(j) == key_at; k = tie ? (unsigned)pos_of(j) ^ flip : 0u; return tie; }, 32 - __clz(bits_used | 1u), need,
           pos_at, below, equal);
    if (below + equal > need) {                     // the same position twice: the lower slots
      need -= below;
      select([&](int j, unsigned& k) { k = (unsigned)(s0 + j); return key(j) == key_at && ((unsigned)pos_of(j) ^ flip) == pos_at; }, 32 - __clz(n), need, slot_at, below,
             equal);
    }
  }
  auto kept = [&](int j) {
    const unsigned k = key(j);
    if (k != key_at || !ties) return k <= key_at;
    const unsigned p = (unsigned)pos_of(j) ^ flip;
    return p < pos_at || (p == pos_at && (unsigned)(s0 + j) <= slot_at);
  };
  // bitmap of this CTA's run, a word a warp and turn
  const int words = (ns + 31) / 32;
  for (int j0 = tid & ~31; j0 < words * 32; j0 += THREADS) {
    const int j = j0 + lane;
    const unsigned m = __ballot_sync(0xffffffffu, j < ns && kept(j));
    if (lane == 0) bits[j0 >> 5] = m;
  }
  __syncthreads();
  // freed slots ahead of the budget and kept ones behind it: how many lie ahead of each word; a thread takes a run of words
  auto ahead = [&](int w) { const int r = a.budget - (s0 + w * 32); return r >= 32 ? 0xffffffffu : r <= 0 ? 0u : (1u << r) - 1; };   // bits of slots < budget
  const int per = (words + THREADS - 1) / THREADS;
  const int w0 = min(words, tid * per), w1 = min(words, w0 + per);
  int2 count = make_int2(0, 0), all;
  for (int w = w0; w < w1; ++w) {
    count.x += __popc(~bits[w] & ahead(w));
    count.y += __popc(bits[w] & ~ahead(w));
  }
  int2 at = pe_sums_before<THREADS>(count, warp_sums, all);
  int holes = all.x, movers = all.y;                 // (as many, and at most max_moves, unless the inputs change underneath)
  if (CL > 1) {
    if (tid == 0) {
      shared_counts[0] = all.x;
      shared_counts[1] = all.y;
    }
    cluster_sync();
    uint4 x[PE_CLUSTER];
#pragma unroll
    for (int r = 0; r < PE_CLUSTER; ++r)
      if (r < CL) x[r] = ld_cluster_u4(cluster_map(smem_u32(shared_counts), r));
    holes = movers = 0;
#pragma unroll
    for (int r = 0; r < PE_CLUSTER; ++r)
      if (r < CL) {
        at.x += r < rank ? (int)x[r].x : 0;
        at.y += r < rank ? (int)x[r].y : 0;
        holes += (int)x[r].x;
        movers += (int)x[r].y;
      }
    // Nobody leaves while another reads its counts: arrived here, behind those reads and ahead of the stores below (an arrival behind them would
    // wait for them).
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  }
  for (int w = w0; w < w1; ++w) {
    holes_at[w] = at.x;
    movers_at[w] = at.y;
    at.x += __popc(~bits[w] & ahead(w));
    at.y += __popc(bits[w] & ~ahead(w));
  }
  __syncthreads();
  const int n_moves = min(min(holes, movers), a.max_moves);
  if (!MOVE && rank == 0 && tid == 0) moves[0] = n_moves;
  int* src = moves + 1;
  int* dst = src + a.max_moves;
  const unsigned lower = (1u << lane) - 1;
  constexpr int AT_ONCE = 4;                         // words of a warp whose weights and positions are under way
  for (int w4 = tid >> 5; w4 < words; w4 += AT_ONCE * (THREADS / 32)) {
    float weight[AT_ONCE];
    int p[AT_ONCE];
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i) {
      const int w = w4 + i * (THREADS / 32);
      const bool stays = w < words && ((bits[w] & ahead(w)) >> lane & 1);
      weight[i] = stays ? weight_of(w * 32 + lane) : 0.f;
      p[i] = stays && pos_out ? pos_of(w * 32 + lane) : 0;
    }
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i) {
      const int w = w4 + i * (THREADS / 32);
      if (w >= words) break;
      const unsigned m = bits[w], front = ahead(w);
      const int j = w * 32 + lane;
      const bool is_kept = (m >> lane) & 1, is_front = (front >> lane) & 1;
      if (is_front && is_kept) {                     // stays
        weights_out[j] = weight[i];
        if (pos_out) pos_out[j] = p[i];
      }
      if (is_front != is_kept) {                     // a freed one ahead, a kept one behind
        const int i = is_front ? holes_at[w] + __popc(~m & front & lower) : movers_at[w] + __popc(m & ~front & lower);
        if (i < a.max_moves) (is_front ? dst : src)[i] = s0 + j;
      }
    }
  }
  if (CL > 1) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
  if (MOVE) {
    __syncthreads();
    pe_move(a, unit, src, dst, n_moves, tid >> 5, THREADS / 32);
  }
}

// The moves of all units: blocks (unit, y).
__global__ void __launch_bounds__(PM_WARPS * 32) k_paged_move(const PagedEvictArgs a) {
  pdl_begin();
  const int* moves = a.moves + (long long)blockIdx.x * (1 + 2 * (long long)a.max_moves);
  pe_move(a, blockIdx.x, moves + 1, moves + 1 + a.max_moves, moves[0], blockIdx.y * PM_WARPS + (threadIdx.x >> 5), gridDim.y * PM_WARPS);
}

}  // namespace lsp
