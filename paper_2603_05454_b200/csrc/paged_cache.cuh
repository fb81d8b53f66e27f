// Append to and eviction from the paged key-value cache.
#pragma once
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
// Selection, a CTA per (sequence, KV head): the budget smallest of the keys (falling weight, position), by radix selection on 11 bits at a
// time; then the kept slots as a bitmap, whose counts give every slot that moves its partner: the i-th kept slot behind the budget goes to
// the i-th freed slot ahead of it.  Sources and targets are disjoint, so k_paged_move needs no order between its blocks.
constexpr int PE_THREADS = 1024;
constexpr int PE_BITS = 11;
constexpr int PE_BINS = 1 << PE_BITS;
constexpr int PE_MAX_CAP = 1 << 20;     // slots of a sequence: a bitmap of 128 KB
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
};

// Order of the weights, heaviest first: 0 = protected, then falling weight (-0 as 0), NaN last.
__device__ __forceinline__ unsigned pe_key(float w) {
  if (w != w) return 0xffffffffu;
  unsigned u = __float_as_uint(w == 0.f ? 0.f : w);
  u = (u >> 31) ? ~u : u | 0x80000000u;       // ascending with w
  return ~u;                                  // +inf: 0x007fffff
}

struct PeSlot { unsigned key, pos; };

template <int THREADS>
__device__ __forceinline__ int pe_block_sum_before(int n, int* warp_sums, int& all) {
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
  if (w == 0) {
    int s = lane < THREADS / 32 ? warp_sums[lane] : 0;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, s, o);
      if (lane >= o) s += y;
    }
    warp_sums[lane] = s;
  }
  __syncthreads();
  all = warp_sums[THREADS / 32 - 1];
  return x - n + (w ? warp_sums[w - 1] : 0);
}

__global__ void __launch_bounds__(PE_THREADS) k_paged_select(const PagedEvictArgs a) {
  extern __shared__ unsigned pe_smem[];
  unsigned* hist = pe_smem;                        // [PE_BINS]
  unsigned* bits = pe_smem + PE_BINS;              // [(cap + 31) / 32] kept slots
  __shared__ int warp_sums[32];
  __shared__ unsigned found[3];                    // bin, count ahead of it, count in it
  pdl_begin();
  const int unit = blockIdx.x, b = unit / a.pv.hkv, cap = pg_capacity(a.pv), tid = threadIdx.x;
  const int n = pg_len(a.pv, a.lens[b]);
  const long long base = (long long)unit * cap;
  int* moves = a.moves + (long long)unit * (1 + 2 * (long long)a.max_moves);
  if (unit % a.pv.hkv == 0 && tid == 0) a.lens_out[b] = min(n, a.budget);
  if (n <= a.budget) {
    if (tid == 0) moves[0] = 0;
    for (int j = tid; j < n; j += PE_THREADS) {
      a.weights_out[base + j] = a.weights[base + j];
      if (a.pos_out) a.pos_out[base + j] = a.pos ? a.pos[base + j] : j;
    }
    return;
  }
  const int seen = a.seen ? a.seen[b] : n;
  auto slot = [&](int j) {
    const int p = a.pos ? a.pos[base + j] : j;
    PeSlot s;
    s.key = (p < a.n_sink || p >= seen - a.n_recent) ? 0u : pe_key(a.weights[base + j]);
    s.pos = (unsigned)p ^ 0x80000000u;
    return s;
  };
  // The need-th smallest of 32-bit keys among the slots for which key_of says true: its value, how many are below it, how many equal it.
  auto select = [&](auto key_of, int need, unsigned& value, int& below, int& equal) {
    unsigned prefix = 0, mask = 0;
    below = 0;
#pragma unroll 1
    for (int shift = 32 - PE_BITS; ; shift = shift > PE_BITS ? shift - PE_BITS : 0) {
      const int width = mask == 0 || shift > 0 ? PE_BITS : 32 - 2 * PE_BITS;
      for (int i = tid; i < PE_BINS; i += PE_THREADS) hist[i] = 0;
      __syncthreads();
      for (int j = tid; j < n; j += PE_THREADS) {
        unsigned k;
        if (key_of(j, k) && (k & mask) == prefix) atomicAdd(&hist[(k >> shift) & ((1u << width) - 1)], 1u);
      }
      __syncthreads();
      // two bins a thread; the bin in which the need-th lies
      const unsigned h0 = hist[2 * tid], h1 = hist[2 * tid + 1];
      int all;
      const int before = pe_block_sum_before<PE_THREADS>((int)(h0 + h1), warp_sums, all);
      const int want = need - below;                 // 1-based rank inside what is left
      if (before < want && want <= before + (int)(h0 + h1)) {
        const bool second = want > before + (int)h0;
        found[0] = 2 * tid + (second ? 1 : 0);
        found[1] = before + (second ? h0 : 0);
        found[2] = second ? h1 : h0;
      }
      __syncthreads();
      prefix |= found[0] << shift;
      mask |= ((1u << width) - 1) << shift;
      below += (int)found[1];
      equal = (int)found[2];
      __syncthreads();
      if (shift == 0) break;
    }
    value = prefix;
  };
  unsigned key_at = 0, pos_at = 0xffffffffu, slot_at = 0xffffffffu;
  int below, equal;
  select([&](int j, unsigned& k) { k = slot(j).key; return true; }, a.budget, key_at, below, equal);
  if (below + equal > a.budget) {                   // ties of the weight: the lower positions
    int need = a.budget - below;
    select([&](int j, unsigned& k) { const PeSlot s = slot(j); k = s.pos; return s.key == key_at; }, need, pos_at, below, equal);
    if (below + equal > need) {                     // the same position twice: the lower slots
      need -= below;
      select([&](int j, unsigned& k) { const PeSlot s = slot(j); k = (unsigned)j; return s.key == key_at && s.pos == pos_at; }, need, slot_at, below, equal);
    }
  }
  auto kept = [&](int j) {
    const PeSlot s = slot(j);
    return s.key < key_at || (s.key == key_at && (s.pos < pos_at || (s.pos == pos_at && (unsigned)j <= slot_at)));
  };
  // bitmap, a word per warp turn
  const int words = (n + 31) / 32;
  for (int j0 = tid & ~31; j0 < words * 32; j0 += PE_THREADS) {
    const int j = j0 + (tid & 31);
    const unsigned m = __ballot_sync(0xffffffffu, j < n && kept(j));
    if ((tid & 31) == 0) bits[j0 >> 5] = m;
  }
  __syncthreads();
  // freed slots ahead of the budget and kept ones behind it, in slot order; a thread takes a run of words
  int* src = moves + 1;
  int* dst = src + a.max_moves;
  const int per = (words + PE_THREADS - 1) / PE_THREADS;
  const int w0 = min(words, tid * per), w1 = min(words, w0 + per);
  auto ahead = [&](int w) { const int r = a.budget - w * 32; return r >= 32 ? 0xffffffffu : r <= 0 ? 0u : (1u << r) - 1; };   // bits of slots < budget
  int nh = 0, nm = 0;
  for (int w = w0; w < w1; ++w) {
    nh += __popc(~bits[w] & ahead(w));
    nm += __popc(bits[w] & ~ahead(w));
  }
  int holes, movers;
  int ih = pe_block_sum_before<PE_THREADS>(nh, warp_sums, holes);
  int im = pe_block_sum_before<PE_THREADS>(nm, warp_sums, movers);
  for (int w = w0; w < w1; ++w) {
    for (unsigned m = ~bits[w] & ahead(w); m; m &= m - 1) dst[ih++] = w * 32 + __ffs(m) - 1;
    for (unsigned m = bits[w] & ~ahead(w); m; m &= m - 1) src[im++] = w * 32 + __ffs(m) - 1;
  }
  __syncthreads();
  if (tid == 0) moves[0] = movers;
  for (int j = tid; j < a.budget; j += PE_THREADS)
    if ((bits[j >> 5] >> (j & 31)) & 1) {
      a.weights_out[base + j] = a.weights[base + j];
      if (a.pos_out) a.pos_out[base + j] = a.pos ? a.pos[base + j] : j;
    }
  for (int i = tid; i < movers; i += PE_THREADS) {
    const int s = src[i], d = dst[i];
    a.weights_out[base + d] = a.weights[base + s];
    if (a.pos_out) a.pos_out[base + d] = a.pos ? a.pos[base + s] : s;
  }
}

// The rows of the movers: a warp per pair of slots, PM_PAIRS of them at a time; the K row in the first half of the lanes, the V row in
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
  if (lane < 2 * PM_PAIRS && i0 + lane % PM_PAIRS < n) {
    const int j = moves[1 + (lane < PM_PAIRS ? 0 : a.max_moves) + i0 + lane % PM_PAIRS];
    const int id = pg_page(a.pv, b, j);
    if (id >= 0) off = ((long long)id * a.pv.page_stride + (long long)(j % a.pv.page) * a.pv.row_stride + (long long)kvh * a.pv.head_stride) * a.esz;
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
