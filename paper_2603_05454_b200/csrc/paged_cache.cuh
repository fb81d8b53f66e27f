// Append to and eviction from the paged key-value cache.
#pragma once
#include "cluster.cuh"
#include "paged_common.cuh"

namespace lsp {

// ---- append --------------------------------------------------------------------------------------------------------------
// Row i of sequence b (packed row row_off[b] + i) goes to slot lens[b] + i.  Bound by HBM for prompts and by latency for single
// tokens: a thread has its share of the row in registers before it knows where the row goes.
constexpr int PP_THREADS = 256;
constexpr int PP_VEC = 4;               // 16-byte pieces of a thread that are under way at once

struct PagedAppendArgs {
  PagedView pv;
  const char *k_new, *v_new;
  long long ld_new;                     // bytes
  const int *lens, *row_off, *seen;
  int max_rows, n_rows, esz, head_bytes;      // head_bytes = head_dim * esz
  int* lens_out;
  int* seen_out;
  float* weights;
  int* pos;
};

// Blocks [0, n_rows): a packed row each.  The last block: the lengths.
__global__ void __launch_bounds__(PP_THREADS) k_paged_append(const PagedAppendArgs a) {
  __shared__ int place[4];              // sequence, slot, page, position
  pdl_begin();
  const int B = a.pv.batch, cap = pg_capacity(a.pv);
  if ((int)blockIdx.x == a.n_rows) {
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
    }
    return;
  }
  const int r = blockIdx.x;
  const int row_bytes = a.pv.hkv * a.head_bytes, pieces = row_bytes / 16;
  const char* ksrc = a.k_new + (long long)r * a.ld_new;
  const char* vsrc = a.v_new + (long long)r * a.ld_new;
  uint4 x[PP_VEC];
#pragma unroll
  for (int i = 0; i < PP_VEC; ++i) {
    const int c = threadIdx.x + i * PP_THREADS;
    if (c < 2 * pieces) x[i] = c < pieces ? reinterpret_cast<const uint4*>(ksrc)[c] : reinterpret_cast<const uint4*>(vsrc)[c - pieces];
  }
  // the sequence: the last one that starts at or ahead of row r (of those that start there, the one with rows)
  int b = 0;
  if (!a.row_off) {
    b = r / a.max_rows;
  } else {
    int n = 0;
    for (int b0 = 0; b0 < B; b0 += PP_THREADS) {
      const int i = b0 + threadIdx.x;
      n += __syncthreads_count(i < B && a.row_off[i] <= r);
    }
    b = n - 1;
  }
  if (threadIdx.x == 0) {
    place[0] = -1;
    if (b >= 0) {
      const RowSpan rs = pg_rows(a.pv, a.row_off, b, a.max_rows, a.n_rows);
      const int n = pg_len(a.pv, a.lens[b]), i = r - rs.first;
      if (i >= 0 && i < rs.n && n + i < cap) {
        const int id = pg_page(a.pv, b, n + i);
        if (id >= 0) {
          place[0] = b;
          place[1] = n + i;
          place[2] = id;
          place[3] = a.pos ? (a.seen ? a.seen[b] : n) + i : 0;
        }
      }
    }
  }
  __syncthreads();
  if (place[0] < 0) return;
  b = place[0];
  const int slot = place[1];
  const long long at = (long long)place[2] * a.pv.page_stride + (long long)(slot % a.pv.page) * a.pv.row_stride;
  const int per_head = a.head_bytes / 16;
  for (int c0 = 0; c0 < 2 * pieces; c0 += PP_VEC * PP_THREADS) {
    if (c0 > 0) {
#pragma unroll
      for (int i = 0; i < PP_VEC; ++i) {
        const int c = c0 + threadIdx.x + i * PP_THREADS;
        if (c < 2 * pieces) x[i] = c < pieces ? reinterpret_cast<const uint4*>(ksrc)[c] : reinterpret_cast<const uint4*>(vsrc)[c - pieces];
      }
    }
#pragma unroll
    for (int i = 0; i < PP_VEC; ++i) {
      const int c = c0 + threadIdx.x + i * PP_THREADS;
      if (c >= 2 * pieces) break;
      const int d = c < pieces ? c : c - pieces;
      char* pool = c < pieces ? a.pv.k : a.pv.v;
      *reinterpret_cast<uint4*>(pool + (at + (long long)(d / per_head) * a.pv.head_stride) * a.esz + (d % per_head) * 16) = x[i];
    }
  }
  if (a.weights || a.pos)
    for (int h = threadIdx.x; h < a.pv.hkv; h += PP_THREADS) {
      const long long w = ((long long)b * a.pv.hkv + h) * cap + slot;
      if (a.weights) a.weights[w] = 0.f;
      if (a.pos) a.pos[w] = place[3];
    }
}

// ---- eviction ------------------------------------------------------------------------------------------------------------
// Selection, a cluster of CTAs per (sequence, KV head): the budget smallest of the keys (falling weight, position), by radix selection; then
// the kept slots as a bitmap, whose counts give every slot that moves its partner: the i-th kept slot behind the budget goes to the i-th
// freed slot ahead of it.  Sources and targets are disjoint, so k_paged_move needs no order between its blocks.
// Each CTA of the cluster has a run of the slots, their keys in shared memory (read from global memory once); a digit's counts
// are added over distributed shared memory.  Bound by the chain of passes: a digit costs a read of the keys from shared memory and four barriers.
constexpr int PE_MAX_CAP = 1 << 20;     // slots of a sequence: a bitmap of 128 KB
constexpr int PE_KEYS = 40 * 1024;      // slots of a CTA whose keys fit shared memory; beyond that a pass reads them again
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
  int cluster, slots, in_smem; // CTAs of a unit, most slots of one (a multiple of 32), their keys are kept in shared memory
};

// Order of the weights, heaviest first: 0 = protected, then falling weight (-0 as 0), NaN last.
__device__ __forceinline__ unsigned pe_key(float w) {
  if (w != w) return 0xffffffffu;
  unsigned u = __float_as_uint(w == 0.f ? 0.f : w);
  u = (u >> 31) ? ~u : u | 0x80000000u;       // ascending with w
  return ~u;                                  // +inf: 0x007fffff
}

// n of this thread added up over the threads before it; all: over all of the block's.
template <int THREADS>
__device__ __forceinline__ int pe_sum_before(int n, int* warp_sums, int& all) {
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  int x = n;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  __syncthreads();
  if (lane == 31) warp_sums[w] = x;
  __syncthreads();
  const int s = lane < THREADS / 32 ? warp_sums[lane] : 0;      // every warp adds the sums up for itself
  int t = s;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, t, o);
    if (lane >= o) t += y;
  }
  all = __shfl_sync(0xffffffffu, t, 31);
  return x - n + __shfl_sync(0xffffffffu, t - s, w);
}

__device__ __forceinline__ int ld_cluster_s32(uint32_t addr) {
  int v;
  asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
  return v;
}

template <int THREADS>
__global__ void __launch_bounds__(THREADS) k_paged_select(const PagedEvictArgs a) {
  constexpr int BINS = 2 * THREADS, BITS = THREADS == 1024 ? 11 : THREADS == 512 ? 10 : 9;      // two bins a thread
  static_assert(1 << BITS == BINS, "two bins a thread");
  extern __shared__ unsigned pe_smem[];
  unsigned* hist = pe_smem;                        // [BINS]
  unsigned* bits = pe_smem + BINS;                 // [slots / 32] kept slots of this CTA
  unsigned* keys = bits + a.slots / 32;            // [slots]
  __shared__ int warp_sums[32], found[3], counts[2];
  const int CL = a.cluster, rank = CL > 1 ? (int)cluster_ctarank() : 0, tid = threadIdx.x;
  auto barrier = [&]() { if (CL > 1) cluster_sync(); else __syncthreads(); };
  pdl_begin();
  const int unit = blockIdx.x / CL, b = unit / a.pv.hkv, cap = pg_capacity(a.pv);
  const int n = pg_len(a.pv, a.lens[b]);
  const long long base = (long long)unit * cap;
  int* moves = a.moves + (long long)unit * (1 + 2 * (long long)a.max_moves);
  if (unit % a.pv.hkv == 0 && rank == 0 && tid == 0) a.lens_out[b] = min(n, a.budget);
  // this CTA's slots: [s0, s0 + ns)
  const int run = ((n + 31) / 32 + CL - 1) / CL * 32, s0 = min(n, rank * run), ns = min(n, s0 + run) - s0;
  const float* weights = a.weights + base + s0;
  const int* pos = a.pos ? a.pos + base + s0 : nullptr;
  if (n <= a.budget) {
    if (rank == 0 && tid == 0) moves[0] = 0;
    for (int j = tid; j < ns; j += THREADS) {
      a.weights_out[base + s0 + j] = weights[j];
      if (a.pos_out) a.pos_out[base + s0 + j] = pos ? pos[j] : s0 + j;
    }
    return;
  }
  const int seen = a.seen ? a.seen[b] : n;
  auto pos_of = [&](int j) { return pos ? pos[j] : s0 + j; };
  auto read_key = [&](int j) {
    const int p = pos_of(j);
    const float w = weights[j];
    return (p < a.n_sink || p >= seen - a.n_recent) ? 0u : pe_key(w);
  };
  if (a.in_smem)
    for (int j = tid; j < ns; j += THREADS) keys[j] = read_key(j);
  auto key = [&](int j) { return a.in_smem ? keys[j] : read_key(j); };
  // The need-th smallest 32-bit value that `get` gives for the slots it says true of: the value, how many are below it, how many equal it.
  // (Where all values of a prefix are wanted, the rest of the digits are: value = the largest with that prefix.)
  auto select = [&](auto get, int need, unsigned& value, int& below, int& equal) {
    unsigned prefix = 0, mask = 0;
    below = 0;
#pragma unroll 1
    for (int shift = 32 - BITS;; shift = max(0, shift - BITS)) {
      const unsigned digit = ~mask >> shift;         // mask of the digit's bits (the last one may be shorter)
      hist[tid] = 0;
      hist[tid + THREADS] = 0;
      __syncthreads();
#pragma unroll 4
      for (int j = tid; j < ns; j += THREADS) {
        unsigned k;
        if (get(j, k) && (k & mask) == prefix) atomicAdd(&hist[(k >> shift) & digit], 1u);
      }
      barrier();
      int h0 = 0, h1 = 0;
      if (CL == 1) {
        const uint2 h = reinterpret_cast<const uint2*>(hist)[tid];
        h0 = h.x;
        h1 = h.y;
      } else {
        const uint32_t mine = smem_u32(hist + 2 * tid);
        for (int r = 0; r < CL; ++r) {
          const uint32_t at = cluster_map(mine, r);
          h0 += ld_cluster_s32(at);
          h1 += ld_cluster_s32(at + 4);
        }
      }
      int all;
      const int before = pe_sum_before<THREADS>(h0 + h1, warp_sums, all);
      const int want = need - below;                 // rank, from 1, among what is left
      if (before < want && want <= before + h0 + h1) {
        const bool second = want > before + h0;
        found[0] = 2 * tid + (second ? 1 : 0);
        found[1] = before + (second ? h0 : 0);
        found[2] = second ? h1 : h0;
      }
      barrier();                                     // (and the others have read this CTA's counts)
      prefix |= (unsigned)found[0] << shift;
      mask |= digit << shift;
      below += found[1];
      equal = found[2];
      if (shift == 0 || below + equal == need) break;
    }
    value = prefix | ~mask;
  };
  unsigned key_at, pos_at = 0xffffffffu, slot_at = 0xffffffffu;
  int below, equal;
  __syncthreads();
  select([&](int j, unsigned& k) { k = key(j); return true; }, a.budget, key_at, below, equal);
  if (below + equal > a.budget) {                   // ties of the weight: the lower positions
    int need = a.budget - below;
    select([&](int j, unsigned& k) { const bool tie = key(j) == key_at; k = tie ? (unsigned)pos_of(j) ^ 0x80000000u : 0u; return tie; }, need, pos_at, below, equal);
    if (below + equal > need) {                     // the same position twice: the lower slots
      need -= below;
      select([&](int j, unsigned& k) { k = (unsigned)(s0 + j); return key(j) == key_at && ((unsigned)pos_of(j) ^ 0x80000000u) == pos_at; }, need, slot_at, below, equal);
    }
  }
  const bool by_pos = pos_at != 0xffffffffu || slot_at != 0xffffffffu;
  auto kept = [&](int j) {
    const unsigned k = key(j);
    if (k != key_at || !by_pos) return k <= key_at;
    const unsigned p = (unsigned)pos_of(j) ^ 0x80000000u;
    return p < pos_at || (p == pos_at && (unsigned)(s0 + j) <= slot_at);
  };
  // bitmap of this CTA's run, a word a warp and turn
  const int words = (ns + 31) / 32;
  for (int j0 = tid & ~31; j0 < words * 32; j0 += THREADS) {
    const int j = j0 + (tid & 31);
    const unsigned m = __ballot_sync(0xffffffffu, j < ns && kept(j));
    if ((tid & 31) == 0) bits[j0 >> 5] = m;
  }
  __syncthreads();
  // freed slots ahead of the budget and kept ones behind it, in slot order; a thread takes a run of words
  const int per = (words + THREADS - 1) / THREADS;
  const int w0 = min(words, tid * per), w1 = min(words, w0 + per);
  auto ahead = [&](int w) { const int r = a.budget - (s0 + w * 32); return r >= 32 ? 0xffffffffu : r <= 0 ? 0u : (1u << r) - 1; };   // bits of slots < budget
  int holes = 0, movers = 0;
  for (int w = w0; w < w1; ++w) {
    holes += __popc(~bits[w] & ahead(w));
    movers += __popc(bits[w] & ~ahead(w));
  }
  int all_holes, all_movers;
  int ih = pe_sum_before<THREADS>(holes, warp_sums, all_holes);
  int im = pe_sum_before<THREADS>(movers, warp_sums, all_movers);
  if (CL > 1) {
    if (tid == 0) {
      counts[0] = all_holes;
      counts[1] = all_movers;
    }
    cluster_sync();
    all_movers = 0;
    for (int r = 0; r < CL; ++r) {
      const uint32_t at = cluster_map(smem_u32(counts), r);
      const int h = ld_cluster_s32(at), m = ld_cluster_s32(at + 4);
      ih += r < rank ? h : 0;
      im += r < rank ? m : 0;
      all_movers += m;
    }
  }
  if (rank == 0 && tid == 0) moves[0] = all_movers;
  int* src = moves + 1;
  int* dst = src + a.max_moves;
  for (int w = w0; w < w1; ++w) {
    for (unsigned m = ~bits[w] & ahead(w); m; m &= m - 1) dst[ih++] = s0 + w * 32 + __ffs(m) - 1;
    for (unsigned m = bits[w] & ~ahead(w); m; m &= m - 1) src[im++] = s0 + w * 32 + __ffs(m) - 1;
  }
  for (int j = tid; j < min(ns, a.budget - s0); j += THREADS)
    if ((bits[j >> 5] >> (j & 31)) & 1) {
      a.weights_out[base + s0 + j] = weights[j];
      if (a.pos_out) a.pos_out[base + s0 + j] = pos_of(j);
    }
  if (CL > 1) cluster_sync();                        // nobody leaves while another reads its counts
}

// What moves: weight, position and rows.  A warp takes PM_PAIRS pairs of slots at a time; the K row in the first half of the lanes, the V row in
// the second (rows of 512 bytes in two turns).
__global__ void __launch_bounds__(PM_WARPS * 32) k_paged_move(const PagedEvictArgs a) {
  pdl_begin();
  const int unit = blockIdx.x, b = unit / a.pv.hkv, kvh = unit % a.pv.hkv, lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  const int* moves = a.moves + (long long)unit * (1 + 2 * (long long)a.max_moves);
  const int n = moves[0];
  const int i0 = (blockIdx.y * PM_WARPS + w) * PM_PAIRS;
  if (i0 >= n) return;
  // lanes 0 .. 3: source of a pair, lanes 4 .. 7: its target
  long long off = -1;
  int j = 0;
  const bool mine = lane < 2 * PM_PAIRS && i0 + lane % PM_PAIRS < n;
  if (mine) {
    j = moves[1 + (lane < PM_PAIRS ? 0 : a.max_moves) + i0 + lane % PM_PAIRS];
    const int id = pg_page(a.pv, b, j);
    if (id >= 0) off = ((long long)id * a.pv.page_stride + (long long)(j % a.pv.page) * a.pv.row_stride + (long long)kvh * a.pv.head_stride) * a.esz;
  }
  const int target = __shfl_down_sync(0xffffffffu, j, PM_PAIRS);
  if (mine && lane < PM_PAIRS) {
    const long long base = (long long)unit * pg_capacity(a.pv);
    a.weights_out[base + target] = a.weights[base + j];
    if (a.pos_out) a.pos_out[base + target] = a.pos ? a.pos[base + j] : j;
  }
  long long from[PM_PAIRS], to[PM_PAIRS];
#pragma unroll
  for (int i = 0; i < PM_PAIRS; ++i) {
    from[i] = __shfl_sync(0xffffffffu, off, i);
    to[i] = __shfl_sync(0xffffffffu, off, PM_PAIRS + i);
    if (from[i] < 0) to[i] = -1;
  }
  char* pool = lane < 16 ? a.pv.k : a.pv.v;
  for (int c = (lane & 15) * 16; c < a.head_bytes; c += 256) {
    uint4 x[PM_PAIRS];
#pragma unroll
    for (int i = 0; i < PM_PAIRS; ++i)
      if (to[i] >= 0) x[i] = *reinterpret_cast<const uint4*>(pool + from[i] + c);
#pragma unroll
    for (int i = 0; i < PM_PAIRS; ++i)
      if (to[i] >= 0) *reinterpret_cast<uint4*>(pool + to[i] + c) = x[i];
  }
}

}  // namespace lsp
