// Attention of a few new rows per sequence over a paged key-value cache, split over the cache's length and joined.
//
// For a sequence's rows r, query heads h of a KV head's group and cached slots j < len:
//   s = scale q[r,h] . k[j],  out[r,h] = sum_j e^{s - m} v[j] / sum_j e^{s - m},  lse = m + ln(sum),
//   weights_out[j] = weights_in[j] + sum over (r, h) of e^{s - lse}.
// Every row sees every slot (the library's attention is bidirectional).
//
// The stream of K and V from HBM bounds it: 4 dh rows * group flops per 4 dh bytes.  So:
//  * The slots of every unit, a (sequence, KV head, tile of 16 (row, head) pairs), are cut into chunks of 64; all chunks of the batch are
//    numbered through, with room for what a unit costs besides, and each CTA of a grid that fills the SMs takes an equal run of the
//    numbers, whatever the lengths are.  A unit that one CTA holds whole is written by it; the parts (m, l, o) of a unit that a run's
//    end cuts go to the workspace, and the last of its CTAs to arrive adds them in their order: the same bits every time.
//  * Where there are several tiles of rows, as many CTAs share a run, a tile ("lane") each: they go over the same slots at the same time, so
//    that all but one of them find the rows in L2.
//  * A warp takes 16 slots of a chunk and loads them itself: a ring of its own in shared memory, filled by cp.async, page ids a window
//    of chunks ahead of the rows they lead to, the queries of the next unit with its first chunk.  The warps of a CTA meet only where a
//    unit begins and ends.
//  * mma.sync m16n8k16, not tcgen05: a tile has at most 16 rows (often one), an M of 128 would be 1/8 to 1/128 full.  What a warp has to
//    issue is what competes with the bytes: 16 slots cost it some 300 instructions (655 once, when 16 x 2047 slots took 77 us).
// Measured on one B200 (copy rate 6.53 TB/s): 16 x 12000 slots of 32 KV heads of 128 350 us = 6.79 TB/s; 16 x 2047 ragged (406 MB) 67.7 us =
// 6.0 TB/s, of which 60 are the stream, 4 the chain lengths -> pages -> rows, 4 the uneven end and the adding of parts.
#pragma once
#include "attention_mma.cuh"
#include "paged_common.cuh"

namespace lsp {

constexpr int PA_CHUNK = 64;            // slots of a chunk: 16 per warp
constexpr int PA_WARPS = 4;
constexpr int PA_THREADS = PA_WARPS * 32;
constexpr int PA_ROWS = 16;             // (row, head) pairs of a unit
constexpr int PA_MAX_BATCH = 1024;
// CTAs that share a run at most.  28 / 56 pairs over 32 x 30000 slots of 4 heads: 305 / 591 us with two, 421 / 822 each for itself (the warps'
// instructions, not the bytes, are the time then); with four the same, and blocks of one to eight rows a sequence 589 where two take 453 to
// 489 and each for itself 528.
constexpr int PA_LANE_BITS = 1;
// CTAs of a launch at most (workspaces are sized by it), and on an SM: those that 64 warps' registers allow, so that 128 KB are in flight
__host__ __device__ constexpr int pa_max_ctas(int dh) { return dh == 64 ? 1024 : 512; }
__host__ __device__ constexpr int pa_ctas_sm(int dh, int esz) { return dh == 64 && esz == 2 ? 4 : dh == 128 && esz == 4 ? 1 : 2; }
constexpr int PA_UNIT_COST = 3;         // what a unit costs besides its chunks, in chunks (queries, adding the warps' parts)
constexpr int PW_THREADS = 256;
constexpr int PW_AHEAD = 8;             // scores of a thread under way at once

struct PagedAttnArgs {
  PagedView pv;
  const void* q;
  void* out;
  long long ldq, ldo;
  const int *lens, *row_off;
  int hq, group, max_rows, n_rows;
  int n_runs, lane_bits;       // CTA x has run x >> lane_bits; of each group of 1 << lane_bits tiles of rows the one of its lower bits
  __device__ __forceinline__ int lanes() const { return 1 << lane_bits; }
  __device__ __forceinline__ int lane() const { return blockIdx.x & ((1 << lane_bits) - 1); }
  float scale_log2;
  float* lse;                  // [n_rows][hq] or null
  unsigned* arrived;           // [CTA]: parts of the cut unit that begins in the CTA's run; 0 between calls
  float* part_o;               // [2 CTAs][16][dh]
  float2* part_ml;             // [2 CTAs][16]: m (in log2 units), l
  float* scores;               // [n_rows][hq][capacity] in log2 units, or null: no weights wanted
  float* row_lse;              // [n_rows][hq]: log2 of the sum of exponentials (with weights)
  const float* weights_in;
  float* weights_out;
  int q_rows, merge_rows;      // rows of a query tile in shared memory (fp32: the kernel's NR); rows that the warps' parts are added for at a time
};

// Shared memory: queries (tiles in turn, a unit each), rings, parts of the warps, their (m, l), chunks before each sequence.
template <typename T, int DH>
struct PaSmem {
  static constexpr int STAGE = 2 * 16 * DH * (int)sizeof(T);          // 16 rows of K, 16 of V
  // Two, 128 KB in flight an SM: 16 sequences of 12000 slots of 32 heads take 353 us, with three 376, with six 429 (one CTA an SM).
  static constexpr int STAGES = 2;
  // Tiles of queries: those of as many units as chunks are asked for ahead, the next one's, and where the queries are not copied to registers at
  // once the present one's (a warp may still be in it when another has reached the next).
  static constexpr int Q_TILES = sizeof(T) == 4 ? STAGES + 1 : STAGES;
  static constexpr int RINGS = PA_WARPS * STAGES * STAGE;
  __host__ __device__ static int q_tile(int q_rows) { return q_rows * DH * (int)sizeof(T); }
  __host__ __device__ static int rings(int q_rows) { return (Q_TILES * q_tile(q_rows) + 127) / 128 * 128; }
  __host__ __device__ static int merge(int q_rows) { return rings(q_rows) + RINGS; }
  __host__ __device__ static int ml(int q_rows, int merge_rows) { return merge(q_rows) + PA_WARPS * merge_rows * DH * 4; }
  __host__ __device__ static int pre(int q_rows, int merge_rows) { return ml(q_rows, merge_rows) + PA_WARPS * 4 * 8; }
  __host__ __device__ static int total(int q_rows, int merge_rows, int batch) { return pre(q_rows, merge_rows) + (batch + 1) * 4; }
};

__device__ __forceinline__ int pa_chunks(int len) { return (len + PA_CHUNK - 1) / PA_CHUNK; }

// pre[b] = numbers of all sequences before b, b <= batch.  Up to 32 sequences every warp computes and stores all of it (the same values) and waits
// for no other; with more the block reads the lengths, all under way at once, and the first warp adds them up.
__device__ __forceinline__ void pa_prefix(const PagedAttnArgs& a, int* pre) {
  const int B = a.pv.batch, lane = threadIdx.x & 31;
  if (B > 32) {
    for (int b = threadIdx.x; b < B; b += PA_THREADS) pre[b] = a.lens[b];
    __syncthreads();
  }
  if (B <= 32 || threadIdx.x < 32) {
    int carry = 0;
#pragma unroll 1
    for (int b0 = 0; b0 < B; b0 += 32) {
      const int b = b0 + lane;
      int n = 0;
      if (b < B) {
        const RowSpan rs = pg_rows(a.pv, a.row_off, b, a.max_rows, a.n_rows);
        const int chunks = pa_chunks(pg_len(a.pv, B > 32 ? pre[b] : a.lens[b]));
        n = chunks == 0 ? 0 : (chunks + PA_UNIT_COST) * a.pv.hkv * ((rs.n * a.group + PA_ROWS * a.lanes() - 1) / PA_ROWS >> a.lane_bits);
      }
      int x = n;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, x, o);
        if (lane >= o) x += y;
      }
      if (b < B) pre[b] = carry + x - n;
      carry += __shfl_sync(0xffffffffu, x, 31);
    }
    if (lane == 0) pre[B] = carry;
  }
  if (B > 32) __syncthreads();
  else __syncwarp();
}

// Ahead of the wait for the preceding kernel: lengths, offsets and page table into L2.  They are read only behind it, and the chain lengths
// -> pages -> rows is what a launch begins with: 16 x 2047 slots of 32 heads 70.6 -> 69.9 us, 4 x 512 13.8 -> 13.1.
__device__ __forceinline__ void pa_prefetch(const PagedAttnArgs& a) {
  pg_prefetch_grid(a.lens, a.pv.batch * 4);
  pg_prefetch_grid(a.row_off, a.pv.batch * 4);
  pg_prefetch_table(a.pv);
}

// How the numbers are dealt: run i of n (those that get at least one) is numbers [run(i), run(i + 1)), run(i) = floor(total i / n).
struct PaDeal {
  int total, n, q, r;
  __device__ __forceinline__ PaDeal(int total_, int n_runs) : total(total_), n(min(total_, n_runs)), q(0), r(0) {
    if (n > 0) {
      q = total / n;
      r = total - q * n;
    }
  }
  __device__ __forceinline__ int run(int i) const { return i * q + pg_div(i * r, n); }
  // the run that holds number c (the estimate is off by one at most: 2^-24 of at most 1024, and the runs' rounding)
  __device__ __forceinline__ int owner(int c) const {
    int i = min(n - 1, (int)((float)c / (float)total * (float)n));
    while (run(i) > c) --i;
    while (run(i + 1) <= c) ++i;
    return i;
  }
};

// A place in the run: sequence, KV head, row tile, chunk of the unit.
struct PaPlace {
  int b, kvh, rt, chunk, chunks, len;
  int u0, left;                 // the number of the unit's first chunk; chunks of the unit that belong to the run, from here on
  __device__ __forceinline__ int next() const { return u0 + chunks + PA_UNIT_COST; }      // the following unit
};
// The place of the first chunk at or behind number c (some numbers are no chunks, and where a sequence's last group of tiles is not full its units
// are not those of all lanes); left = 0 where the run holds none.
__device__ __forceinline__ PaPlace pa_place(const PagedAttnArgs& a, const int* pre, int c, int hi) {
  PaPlace p;
  p.left = 0;
  while (c < hi) {
    int lo = 0, up = a.pv.batch;                   // pre[lo] <= c < pre[up]
    while (up - lo > 1) {
      const int mid = (lo + up) >> 1;
      if (pre[mid] <= c) lo = mid; else up = mid;
    }
    p.b = lo;
    const int n = a.lens[lo], cap = pg_capacity(a.pv);
    p.len = n > cap ? cap : n;
    p.chunks = pa_chunks(p.len);
    // (quotients: a sequence's KV heads times groups of tiles, at most 2^20 by the call's limits)
    const int span = p.chunks + PA_UNIT_COST, groups = pg_div(pre[lo + 1] - pre[lo], span * a.pv.hkv);
    const int u = pg_div(c - pre[lo], span);
    p.u0 = pre[lo] + u * span;
    p.chunk = c - p.u0;
    p.kvh = pg_div(u, groups);
    p.rt = ((u - p.kvh * groups) << a.lane_bits) + a.lane();
    if (p.chunk < p.chunks && (a.lane_bits == 0 || p.rt * PA_ROWS < pg_rows(a.pv, a.row_off, lo, a.max_rows, a.n_rows).n * a.group)) {
      p.left = min(p.chunks - p.chunk, hi - c);
      break;
    }
    c = p.next();
  }
  return p;
}

// A part of a cut unit, noted until the run's end: the unit, and runs first .. last, whose CTAs (of this lane) have a part each; the first one's
// is its second part where the unit begins in its run.
struct PaCut {
  PaPlace p;
  int first, last, second;
};

// Where a (row, head) pair of a unit lies: packed row and query head; false behind the sequence's last row.
__device__ __forceinline__ bool pa_row(const PagedAttnArgs& a, const RowSpan& rs, const PaPlace& p, int i, int& row, int& head) {
  const int x = p.rt * PA_ROWS + i;
  if (x >= rs.n * a.group) return false;
  const int r = pg_div(x, a.group);
  row = rs.first + r;
  head = p.kvh * a.group + x - r * a.group;
  return true;
}

__device__ __forceinline__ void cp_async16_all(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}

// Byte offset of 16-byte chunk c of row r in a [16][DH] tile: chunks are exchanged within groups of eight by the row, so that eight
// rows' chunks c lie in different banks.
template <typename T, int DH>
__device__ __forceinline__ int pa_at(int r, int c) {
  return r * DH * (int)sizeof(T) + ((c ^ (r & 7)) << 4);
}
// The same in a tile of queries; fp32: not exchanged (eight lanes read eight chunks of one row).
template <typename T, int DH>
__device__ __forceinline__ int pa_q_at(int r, int c) {
  if constexpr (sizeof(T) == 2) return pa_at<T, DH>(r, c);
  else return r * DH * 4 + c * 16;
}

// One warp's loads: the rows of its 16 slots of a chunk, K then V, into one stage of its ring; and its part of the queries of a unit
// that begins with the chunk.  A16: a page holds a multiple of 16 slots, so the 16 lie in one page, one behind the other; else every slot's page is
// looked up.  (16 sequences of 2047 slots of 32 heads: 70.7 us, all looked up 72.6; 16 x 12000 of 4 heads of 64 33.1 and 35.0.)
template <typename T, int DH, bool A16>
struct PaLoader {
  static constexpr int CPR = DH * (int)sizeof(T) / 16;      // 16-byte chunks of a row
  static constexpr int RPI = 32 / CPR;                      // rows of an instruction
  static constexpr int WINDOW = A16 ? 32 : 2;               // chunks whose pages a lane's ids cover
  const PagedAttnArgs& a;
  const int* pre;
  int hi, w, lane;
  PaPlace p;
  bool first;                   // the next chunk is the run's first of its unit
  int tile;                     // of the unit that comes next
  // Pages ahead, and rows in the page: A16: lane i those of the warp's slots of chunk base + i; else lanes 0 to 15 those of the slots of
  // chunk `base`, 16 to 31 of the one behind it.  The second ones, a window on, are under way.
  int base, id, rem, id2, rem2;
  __device__ __forceinline__ PaLoader(const PagedAttnArgs& a_, const int* pre_, int hi_, const PaPlace& p_)
      : a(a_), pre(pre_), hi(hi_), w(threadIdx.x >> 5), lane(threadIdx.x & 31), p(p_), first(true), tile(0) {
    begin();
  }
  __device__ __forceinline__ void ask(int chunk, int& page, int& row) const {
    const int j = A16 ? (chunk + lane) * PA_CHUNK + w * 16 : (chunk + (lane >> 4)) * PA_CHUNK + w * 16 + (lane & 15);
    const int end = A16 ? min(p.len, (p.chunk + p.left) * PA_CHUNK) : p.len;      // (no pages of chunks that are another CTA's)
    const int n = pg_div(j, a.pv.page);
    page = j < end ? pg_page(a.pv, p.b, n) : -1;
    row = j - n * a.pv.page;
  }
  __device__ __forceinline__ void begin() {
    base = p.chunk;
    ask(base, id, rem);
    ask(base + WINDOW, id2, rem2);
  }
  // Returns a mask of the rows that are real slots.
  __device__ __forceinline__ unsigned issue(char* stage, char* q_tiles) {
    unsigned live = 0;
    if (p.left > 0) {
      if (first) {
        const RowSpan rs = pg_rows(a.pv, a.row_off, p.b, a.max_rows, a.n_rows);
        char* q_tile = q_tiles + tile * PaSmem<T, DH>::q_tile(a.q_rows);
        if (++tile == PaSmem<T, DH>::Q_TILES) tile = 0;
        const int pieces = min(PA_ROWS, rs.n * a.group - p.rt * PA_ROWS) * CPR;
#pragma unroll 1
        for (int i = threadIdx.x; i < pieces; i += PA_THREADS) {
          int row, head;
          pa_row(a, rs, p, i / CPR, row, head);
          cp_async16(smem_u32(q_tile + pa_q_at<T, DH>(i / CPR, i % CPR)), (const T*)a.q + (long long)row * a.ldq + head * DH + (i % CPR) * (16 / (int)sizeof(T)), true);
        }
      }
      // this lane's piece of row (lane / CPR) of the tile; the rows an instruction further on: exchanged chunks differ in the row's low bits
      const int r0 = lane / CPR, ch = lane % CPR;
      const uint32_t ks = smem_u32(stage), vs = ks + 16 * DH * (int)sizeof(T);
      const uint32_t at = r0 * DH * (int)sizeof(T) + ((ch ^ r0) << 4);
      auto dst = [&](int i) { return i * RPI * DH * (int)sizeof(T) + (at ^ (((i * RPI) & 7) << 4)); };
      if constexpr (A16) {
        const int from = p.chunk - base, page = __shfl_sync(0xffffffffu, id, from), row = __shfl_sync(0xffffffffu, rem, from);
        const int n = page < 0 ? 0 : min(16, p.len - (p.chunk * PA_CHUNK + w * 16));
        live = n >= 16 ? 0xffffu : n <= 0 ? 0u : (1u << n) - 1;
        const long long step = a.pv.row_stride * RPI * (int)sizeof(T);
        const long long off = n <= 0 ? 0 : ((long long)page * a.pv.page_stride + (long long)(row + r0) * a.pv.row_stride + (long long)p.kvh * a.pv.head_stride) * (int)sizeof(T) + ch * 16;
        const char *k = a.pv.k + off, *v = a.pv.v + off;
        if (n >= 16) {
#pragma unroll
          for (int i = 0; i < 16 / RPI; ++i) {
            cp_async16_all(ks + dst(i), k);
            cp_async16_all(vs + dst(i), v);
            k += step;
            v += step;
          }
        } else {
#pragma unroll 1
          for (int i = 0; i < 16 / RPI; ++i) {
            const bool there = i * RPI + r0 < n;
            cp_async16(ks + dst(i), there ? k : a.pv.k, there);
            cp_async16(vs + dst(i), there ? v : a.pv.v, there);
            k += step;
            v += step;
          }
        }
      } else {
        const int page = __shfl_sync(0xffffffffu, id, (p.chunk - base) * 16 + (lane & 15)), row = __shfl_sync(0xffffffffu, rem, (p.chunk - base) * 16 + (lane & 15));
        live = __ballot_sync(0xffffffffu, page >= 0) & 0xffffu;
        const long long off = page < 0 ? 0 : (long long)page * a.pv.page_stride + (long long)row * a.pv.row_stride + (long long)p.kvh * a.pv.head_stride;
#pragma unroll
        for (int i = 0; i < 16 / RPI; ++i) {
          const int r = i * RPI + r0;
          const long long o = __shfl_sync(0xffffffffu, off, r) * (int)sizeof(T) + ch * 16;
          const bool there = (live >> r) & 1;
          cp_async16(ks + dst(i), a.pv.k + (there ? o : 0), there);
          cp_async16(vs + dst(i), a.pv.v + (there ? o : 0), there);
        }
      }
      first = --p.left == 0;
      if (first) {
        p = pa_place(a, pre, p.next(), hi);
        if (p.left > 0) begin();
      } else if (++p.chunk == base + WINDOW) {
        base += WINDOW;
        id = id2;
        rem = rem2;
        ask(base + WINDOW, id2, rem2);
      }
    }
    cp_async_commit();
    return live;
  }
};

// The ring of a warp: which stage is next, what is in flight.
template <typename T, int DH, bool A16>
struct PaRing {
  using S = PaSmem<T, DH>;
  PaLoader<T, DH, A16> ld;
  char *q_tiles, *ring;
  int q_tile_bytes, stage = 0, tile = 0;
  unsigned live[S::STAGES];     // masks of the stages in flight, oldest first
  __device__ __forceinline__ PaRing(const PagedAttnArgs& a, const int* pre, int hi, const PaPlace& p, char* smem)
      : ld(a, pre, hi, p), q_tiles(smem), ring(smem + S::rings(a.q_rows) + (threadIdx.x >> 5) * S::STAGES * S::STAGE), q_tile_bytes(S::q_tile(a.q_rows)) {
#pragma unroll
    for (int s = 0; s < S::STAGES - 1; ++s) live[s] = ld.issue(ring + s * S::STAGE, q_tiles);
    live[S::STAGES - 1] = 0;
  }
  // Asks for one chunk more (into the stage that was read last turn) and waits for the oldest; its rows and their mask.
  __device__ __forceinline__ unsigned turn(char*& rows) {
    int s = stage + S::STAGES - 1;
    if (s >= S::STAGES) s -= S::STAGES;
    __syncwarp();
    live[S::STAGES - 1] = ld.issue(ring + s * S::STAGE, q_tiles);
    cp_async_wait<S::STAGES - 1>();
    __syncwarp();
    const unsigned mask = live[0];
#pragma unroll
    for (int i = 0; i + 1 < S::STAGES; ++i) live[i] = live[i + 1];
    rows = ring + stage * S::STAGE;
    if (++stage == S::STAGES) stage = 0;
    return mask;
  }
  // The queries of the unit that begins: there for all warps behind the barrier that follows its first turn.
  __device__ __forceinline__ const char* queries() {
    const char* q = q_tiles + tile * q_tile_bytes;
    if (++tile == S::Q_TILES) tile = 0;
    return q;
  }
};

__device__ __forceinline__ float pa_exp2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// 2^(m_old - m_new) of the online softmax; -inf - -inf (nothing seen yet) counts as nothing.
__device__ __forceinline__ float pa_scale(float m_old, float m_new) { return m_old == -INFINITY ? 0.f : pa_exp2(m_old - m_new); }

// A lane's share of a result row: VEC = DH / 32 neighbouring elements, sums o over weights that sum to l.
template <typename T, int DH>
__device__ __forceinline__ void pa_write_row(const PagedAttnArgs& a, int row, int head, const float (&o)[DH / 32], float m, float l) {
  constexpr int VEC = DH / 32;
  const int lane = threadIdx.x & 31;
  const float inv = l == 0.f ? 0.f : 1.f / l;                 // (no slot, or all scores -inf: the sums are 0)
  T* dst = (T*)a.out + (long long)row * a.ldo + head * DH + lane * VEC;
  if constexpr (sizeof(T) == 2) {
#pragma unroll
    for (int e = 0; e < VEC; e += 2) reinterpret_cast<uint32_t*>(dst)[e / 2] = pack_bf16(o[e] * inv, o[e + 1] * inv);
  } else {
#pragma unroll
    for (int e = 0; e < VEC; ++e) dst[e] = o[e] * inv;
  }
  if (lane == 0) {
    const long long at = (long long)row * a.hq + head;
    const float x = l == 0.f ? -INFINITY : m + log2f(l);
    if (a.lse) a.lse[at] = x * 0.6931471805599453f;
    if (a.scores) a.row_lse[at] = x;
  }
}

// The end of a unit, or of the run's part of it.  The warps' parts are added for merge_rows rows at a time: put(i, n, o, ml) leaves this warp's
// rows i .. i + n - 1 ([n][DH], pairs of elements exchanged by 4 (row & 3)) and their (m, l); warp w adds row i + w.  A part of a cut unit
// is noted in cut[] (at most one that begins ahead of the run and one that ends behind it).
template <typename T, int DH, typename Put>
__device__ __forceinline__ void pa_finish(const PagedAttnArgs& a, const PaDeal& deal, const PaPlace& p, const RowSpan& rs, int lo, PaCut* cut, char* smem, Put put) {
  constexpr int VEC = DH / 32;
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  float* merge = reinterpret_cast<float*>(smem + PaSmem<T, DH>::merge(a.q_rows));
  float2* ml = reinterpret_cast<float2*>(smem + PaSmem<T, DH>::ml(a.q_rows, a.merge_rows));
  const int n_real = min(PA_ROWS, rs.n * a.group - p.rt * PA_ROWS);
  const bool whole = p.left == p.chunks;
  const int second = lo >= p.u0 ? 0 : 1, part = 2 * blockIdx.x + second;
  if (!whole && threadIdx.x == PA_THREADS - 1) {      // (the last warp adds rows last, if any)
    const int first = deal.owner(p.u0);
    cut[second] = PaCut{p, first, deal.owner(p.u0 + p.chunks - 1), deal.run(first) < p.u0 ? 1 : 0};
  }
  for (int i = 0; i < n_real; i += a.merge_rows) {
    if (i > 0) __syncthreads();
    put(i, a.merge_rows, merge + w * a.merge_rows * DH, ml + w * a.merge_rows);
    __syncthreads();
    if (w < a.merge_rows && i + w < n_real) {
      float m = -INFINITY, l = 0.f, o[VEC];
#pragma unroll
      for (int e = 0; e < VEC; ++e) o[e] = 0.f;
#pragma unroll
      for (int k = 0; k < PA_WARPS; ++k) m = fmaxf(m, ml[k * a.merge_rows + w].x);
#pragma unroll
      for (int k = 0; k < PA_WARPS; ++k) {
        const float2 x = ml[k * a.merge_rows + w];
        const float f = pa_scale(x.x, m);
        l = fmaf(x.y, f, l);
        const float* src = merge + (k * a.merge_rows + w) * DH;
#pragma unroll
        for (int e = 0; e < VEC; e += 2) {
          const float2 y = *reinterpret_cast<const float2*>(src + (((lane * VEC + e) / 2) ^ (4 * w)) * 2);
          o[e] = fmaf(y.x, f, o[e]);
          o[e + 1] = fmaf(y.y, f, o[e + 1]);
        }
      }
      if (whole) {
        int row, head;
        pa_row(a, rs, p, i + w, row, head);
        pa_write_row<T, DH>(a, row, head, o, m, l);
      } else {
        float* dst = a.part_o + ((long long)part * PA_ROWS + i + w) * DH + lane * VEC;
#pragma unroll
        for (int e = 0; e < VEC; ++e) dst[e] = o[e];
        if (lane == 0) a.part_ml[part * PA_ROWS + i + w] = make_float2(m, l);
      }
    }
  }
}

// The end of the run: its parts of cut units are there; the last CTA of a unit to say so adds them all, in their order.  A warp takes a
// row at a time, 32 parts' (m, l) on its lanes and PA_AHEAD parts' o under way; the code is short because it is fetched cold.
constexpr int PA_AHEAD = 16;
template <typename T, int DH>
__device__ __forceinline__ void pa_join(const PagedAttnArgs& a, const PaCut* cut) {
  constexpr int VEC = DH / 32;
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  __shared__ int mine[2];                          // a unit is this CTA's to add
  cp_async_wait<0>();
  __syncthreads();
  if (threadIdx.x < 2) {
    const PaCut& c = cut[threadIdx.x];
    bool last = false;
    if (c.p.left > 0) {
      __threadfence();
      unsigned* arrived = a.arrived + (c.first << a.lane_bits) + a.lane();
      last = atomicAdd(arrived, 1u) == (unsigned)(c.last - c.first);
      if (last) *arrived = 0;
      __threadfence();
    }
    mine[threadIdx.x] = last;
  }
  __syncthreads();
  // the rows of both units dealt to the warps
  int skip = w;
#pragma unroll 1
  for (int which = 0; which < 2; ++which) {
    if (!mine[which]) continue;
    const PaPlace p = cut[which].p;
    const int i0 = cut[which].first, second = cut[which].second, n = cut[which].last - i0 + 1;
    const RowSpan rs = pg_rows(a.pv, a.row_off, p.b, a.max_rows, a.n_rows);
    const int n_real = min(PA_ROWS, rs.n * a.group - p.rt * PA_ROWS);
    int r = skip;
#pragma unroll 1
    for (; r < n_real; r += PA_WARPS) {
      float m = -INFINITY, l = 0.f, o[VEC];
#pragma unroll
      for (int e = 0; e < VEC; ++e) o[e] = 0.f;
#pragma unroll 1
      for (int k0 = 0; k0 < n; k0 += 32) {
        const int k = min(k0 + lane, n - 1);
        const int slot = (2 * (((i0 + k) << a.lane_bits) + a.lane()) + (k == 0 ? second : 0)) * PA_ROWS + r;
        const float2 x = __ldcg(a.part_ml + slot);
        float y[PA_AHEAD][VEC], f = 0.f;
#pragma unroll 1
        for (int q = 0; q < 32 && k0 + q < n; q += PA_AHEAD) {
#pragma unroll
          for (int i = 0; i < PA_AHEAD; ++i) {
            const float* src = a.part_o + (long long)__shfl_sync(0xffffffffu, slot, q + i) * DH + lane * VEC;
            if constexpr (VEC == 4) {
              const float4 z = __ldcg(reinterpret_cast<const float4*>(src));
              y[i][0] = z.x; y[i][1] = z.y; y[i][2] = z.z; y[i][3] = z.w;
            } else {
              const float2 z = __ldcg(reinterpret_cast<const float2*>(src));
              y[i][0] = z.x; y[i][1] = z.y;
            }
          }
          if (q == 0) {                                // (while they are under way)
            const float top = fmaxf(m, warp_max(x.x)), f0 = pa_scale(m, top);
            f = k0 + lane < n ? pa_scale(x.x, top) : 0.f;
            m = top;
            l = l * f0 + warp_sum(x.y * f);
#pragma unroll
            for (int e = 0; e < VEC; ++e) o[e] *= f0;
          }
#pragma unroll
          for (int i = 0; i < PA_AHEAD; ++i) {
            const float g = __shfl_sync(0xffffffffu, f, q + i);
#pragma unroll
            for (int e = 0; e < VEC; ++e) o[e] = fmaf(y[i][e], g, o[e]);
          }
        }
      }
      int row, head;
      pa_row(a, rs, p, r, row, head);
      pa_write_row<T, DH>(a, row, head, o, m, l);
    }
    skip = r - n_real;
  }
}

// Rows of sequences without a slot: 0.  (The grid's CTAs take the sequences in turn.)
template <typename T, int DH>
__device__ __forceinline__ void pa_empty(const PagedAttnArgs& a, const int* pre) {
  const int w = threadIdx.x >> 5;
  for (int b = blockIdx.x; b < a.pv.batch; b += gridDim.x) {
    if (pre[b + 1] > pre[b]) continue;
    const RowSpan rs = pg_rows(a.pv, a.row_off, b, a.max_rows, a.n_rows);
    const float o[DH / 32] = {};
    for (int i = w; i < rs.n * a.hq; i += PA_WARPS) pa_write_row<T, DH>(a, rs.first + i / a.hq, i % a.hq, o, -INFINITY, 0.f);
  }
}

// ---- bf16: tensor cores --------------------------------------------------------------------------------------------------
// Softmax weights are fed to the P V product as the sum of two bf16 numbers (16 bits of mantissa): the tensor pipe has the time, and
// ahead of its rounding the output is within 2e-6 of one with fp32 weights (a last bit of bf16 differs in one element of some 400).
// The maximum is raised only where a score is more than 2^PA_LAZY times the weight of the present one (the sums have room for that), so that most
// chunks need neither its exchange over the lanes nor a rescale.
constexpr float PA_LAZY = 8.f;
template <int DH, bool A16>
__global__ void __launch_bounds__(PA_THREADS, pa_ctas_sm(DH, 2)) k_paged_attn_mma(const PagedAttnArgs a) {
  extern __shared__ __align__(128) char pa_smem[];
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
  int* pre = reinterpret_cast<int*>(pa_smem + PaSmem<bf16, DH>::pre(a.q_rows, a.merge_rows));
  pdl_release();
  pa_prefetch(a);
  pdl_wait();
  pa_prefix(a, pre);
  pa_empty<bf16, DH>(a, pre);
  const PaDeal deal(pre[a.pv.batch], a.n_runs);
  const int run = (int)blockIdx.x >> a.lane_bits;
  if (run >= deal.n) return;
  const int lo = deal.run(run), hi = deal.run(run + 1);
  PaPlace p = pa_place(a, pre, lo, hi);
  if (p.left == 0) return;
  __shared__ PaCut cut[2];
  if (threadIdx.x < 2) cut[threadIdx.x].p.left = 0;

  PaRing<bf16, DH, A16> ring(a, pre, hi, p, pa_smem);
  // this lane's rows and chunks of the K and V tiles (ldmatrix); chunk c lies at c ^ (row & 7): further chunks are the same address with
  // bits 5, 6 flipped, or 128 bytes on
  const uint32_t k_at = pa_at<bf16, DH>(lane & 7, lane >> 3), v_at = pa_at<bf16, DH>((lane & 7) + ((lane >> 3) & 1) * 8, lane >> 4);
  const float lazy = PA_LAZY / a.scale_log2;
  for (; p.left > 0; p = pa_place(a, pre, p.next(), hi)) {
    // ---- a unit, or the part of it that belongs to this run
    const RowSpan rs = pg_rows(a.pv, a.row_off, p.b, a.max_rows, a.n_rows);
    const int n_real = min(PA_ROWS, rs.n * a.group - p.rt * PA_ROWS);
    float* score[2] = {nullptr, nullptr};         // where the two rows' scores go
    if (a.scores) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        int row, head;
        if (pa_row(a, rs, p, g + 8 * h, row, head)) score[h] = a.scores + ((long long)row * a.hq + head) * pg_capacity(a.pv) + 2 * t;
      }
    }
    uint32_t qf[DH / 16][4];
    float o[DH / 8][4];
#pragma unroll
    for (int i = 0; i < DH / 8; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;
    // per row: the maximum (unscaled), where it is raised, what is added to a scaled score, the sum of this lane's weights
    float m[2] = {-INFINITY, -INFINITY}, limit[2] = {-INFINITY, -INFINITY}, shift[2] = {0.f, 0.f}, l[2] = {0.f, 0.f};

#pragma unroll 1
    for (int k = 0; k < p.left; ++k) {
      char* rows;
      const unsigned mask = ring.turn(rows);
      if (k == 0) {
        __syncthreads();                        // all warps' parts of the queries are there (and the last unit's parts have been read)
        const int r = min((lane & 7) + ((lane >> 3) & 1) * 8, n_real - 1);      // rows that are none repeat the last one
        const uint32_t qs = smem_u32(ring.queries());
#pragma unroll
        for (int kk = 0; kk < DH / 16; ++kk) ldsm_x4(qs + pa_q_at<bf16, DH>(r, kk * 2 + (lane >> 4)), qf[kk][0], qf[kk][1], qf[kk][2], qf[kk][3]);
        __syncthreads();                        // before anyone asks for further queries in their place
      }
      const int j0 = (p.chunk + k) * PA_CHUNK + w * 16;
      if (mask == 0 && (!a.scores || j0 >= p.len)) continue;
      const uint32_t ks = smem_u32(rows), vs = ks + 16 * DH * 2;
      // S = Q K^T: 16 rows x 16 slots
      float s[2][4];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        float s2[4] = {0.f, 0.f, 0.f, 0.f};
        s[j][0] = s[j][1] = s[j][2] = s[j][3] = 0.f;
#pragma unroll
        for (int kk = 0; kk < DH / 16; kk += 2) {
          uint32_t b0, b1, b2, b3;
          ldsm_x4(ks + (k_at ^ ((kk * 2 & 4) << 4)) + j * 8 * DH * 2 + (kk >= 4 ? 128 : 0), b0, b1, b2, b3);
          mma_bf16(s[j], qf[kk][0], qf[kk][1], qf[kk][2], qf[kk][3], b0, b1);
          mma_bf16(s2, qf[kk + 1][0], qf[kk + 1][1], qf[kk + 1][2], qf[kk + 1][3], b2, b3);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) s[j][e] += s2[e];
      }
      if (mask != 0xffffu) {
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (!((mask >> (j * 8 + 2 * t + (e & 1))) & 1)) s[j][e] = -INFINITY;
      }
      if (a.scores) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
          if (score[h]) {
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
              for (int e = 0; e < 2; ++e)
                if (j0 + j * 8 + 2 * t + e < p.len) score[h][j0 + j * 8 + e] = s[j][2 * h + e] * a.scale_log2;
          }
      }
      float mx[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) mx[h] = fmaxf(fmaxf(s[0][2 * h], s[0][2 * h + 1]), fmaxf(s[1][2 * h], s[1][2 * h + 1]));
      if (__any_sync(0xffffffffu, mx[0] > limit[0] || mx[1] > limit[1])) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          mx[h] = fmaxf(mx[h], __shfl_xor_sync(0xffffffffu, mx[h], 1));
          mx[h] = fmaxf(mx[h], __shfl_xor_sync(0xffffffffu, mx[h], 2));
          const float top = fmaxf(m[h], mx[h]), corr = m[h] == -INFINITY ? 0.f : pa_exp2((m[h] - top) * a.scale_log2);
          m[h] = top;
          limit[h] = top + lazy;
          shift[h] = top == -INFINITY ? 0.f : -top * a.scale_log2;
          l[h] *= corr;
#pragma unroll
          for (int i = 0; i < DH / 8; ++i) {
            o[i][2 * h] *= corr;
            o[i][2 * h + 1] *= corr;
          }
        }
      }
      uint32_t hi_[4], lo_[4];
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const float p0 = pa_exp2(fmaf(s[j][2 * h], a.scale_log2, shift[h])), p1 = pa_exp2(fmaf(s[j][2 * h + 1], a.scale_log2, shift[h]));
          l[h] += p0 + p1;
          const uint32_t x = pack_bf16(p0, p1);
          hi_[j * 2 + h] = x;
          lo_[j * 2 + h] = pack_bf16(p0 - __uint_as_float(x << 16), p1 - __uint_as_float(x & 0xffff0000u));
        }
      // O += P V
#pragma unroll
      for (int nt = 0; nt < DH / 8; nt += 2) {
        uint32_t b0, b1, b2, b3;
        ldsm_x4_t(vs + (v_at ^ ((nt & 6) << 4)) + (nt >= 8 ? 128 : 0), b0, b1, b2, b3);
        mma_bf16(o[nt], hi_[0], hi_[1], hi_[2], hi_[3], b0, b1);
        mma_bf16(o[nt + 1], hi_[0], hi_[1], hi_[2], hi_[3], b2, b3);
        mma_bf16(o[nt], lo_[0], lo_[1], lo_[2], lo_[3], b0, b1);
        mma_bf16(o[nt + 1], lo_[0], lo_[1], lo_[2], lo_[3], b2, b3);
      }
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      l[h] += __shfl_xor_sync(0xffffffffu, l[h], 1);
      l[h] += __shfl_xor_sync(0xffffffffu, l[h], 2);
      m[h] *= a.scale_log2;
    }
    pa_finish<bf16, DH>(a, deal, p, rs, lo, cut, pa_smem, [&](int i0, int n, float* dst, float2* ml) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int r = g + 8 * h - i0;
        if (r < 0 || r >= n) continue;
#pragma unroll
        for (int i = 0; i < DH / 8; ++i) *reinterpret_cast<float2*>(dst + r * DH + ((i * 4 + t) ^ (4 * r)) * 2) = make_float2(o[i][2 * h], o[i][2 * h + 1]);
        if (t == 0) ml[r] = make_float2(m[h], l[h]);
      }
    });
  }
  pa_join<bf16, DH>(a, cut);
}

// ---- fp32: CUDA cores ----------------------------------------------------------------------------------------------------
// A lane's tile of the products is wide both ways, since a 16-byte load of shared memory takes a warp as long as 16 FMAs or more.  Scores: eight
// lanes of each slot, a quarter of the slots a lane, so that 4 + NR loads feed 16 NR FMAs; the eight lanes' sums are then scattered, NR / 2
// (row, slot)s each, and the softmax is done there, once.  P V: a lane takes DH / 32 dimensions of all rows; the weights reach it through
// the K rows' place, which nobody reads any more.  (One slot and half of the dimensions a lane, the weights by a shuffle each: 4 x 4000 slots of 32
// heads of 128, 1 / 4 / 8 rows 72 / 98 / 158 us, so 70 / 74 / 88; 67 are the bytes.)  Sixteen rows of 128 are bound by the latency of the four
// warps that an SM's registers and rings leave.
// A kernel for every power of two of rows: the work a slot costs goes with the rows.
template <int DH, int NR, bool A16>
__global__ void __launch_bounds__(PA_THREADS, pa_ctas_sm(DH, 4)) k_paged_attn_simt(const PagedAttnArgs a) {
  extern __shared__ __align__(128) char pa_smem[];
  constexpr int VEC = DH / 32;                  // dimensions of a lane in P V
  constexpr int OWN = NR >= 2 ? NR / 2 : 1;     // (row, slot)s of a lane in the softmax: RO rows of KO slots
  constexpr int RO = NR == 16 ? 2 : 1, KO = OWN / RO;
  // Loops as long as the instruction cache holds: sixteen rows of 128 (16 x 12000 slots of 4 heads, groups of 7) 185 us, unrolled as fewer rows are 297;
  // eight rows 111, as short as sixteen's 123.
  constexpr bool LONG = NR * DH == 16 * 128;
  constexpr int UNROLL_S = LONG ? 1 : DH / 32, UNROLL_O = LONG ? 4 : 8;
  constexpr int SHARE = NR >= 8 ? 0 : 8 / NR - 1;       // the bits of a lane in which those that share a row differ, besides 8 and 16
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  int* pre = reinterpret_cast<int*>(pa_smem + PaSmem<float, DH>::pre(a.q_rows, a.merge_rows));
  pdl_release();
  pa_prefetch(a);
  pdl_wait();
  pa_prefix(a, pre);
  pa_empty<float, DH>(a, pre);
  const PaDeal deal(pre[a.pv.batch], a.n_runs);
  const int run = (int)blockIdx.x >> a.lane_bits;
  if (run >= deal.n) return;
  const int lo = deal.run(run), hi = deal.run(run + 1);
  PaPlace p = pa_place(a, pre, lo, hi);
  if (p.left == 0) return;
  __shared__ PaCut cut[2];
  if (threadIdx.x < 2) cut[threadIdx.x].p.left = 0;

  PaRing<float, DH, A16> ring(a, pre, hi, p, pa_smem);
  // slots kq + 4 i; of their rows' 16-byte chunks those with d as their lower bits; in the softmax rows r0 .. of slots kq + 4 (i0 ..)
  const int kq = lane >> 3, d = lane & 7;
  const int r0 = NR == 16 ? 2 * d : NR == 1 ? 0 : d * NR / 8, i0 = NR >= 8 ? 0 : NR == 1 ? d >> 1 : d * OWN % 4;
  for (; p.left > 0; p = pa_place(a, pre, p.next(), hi)) {
    const RowSpan rs = pg_rows(a.pv, a.row_off, p.b, a.max_rows, a.n_rows);
    const int nr = min(PA_ROWS, rs.n * a.group - p.rt * PA_ROWS);
    float o[NR][VEC], m[RO], l[RO];             // m: the same in all lanes that share the row; l: this lane's slots
#pragma unroll
    for (int r = 0; r < NR; ++r)
#pragma unroll
      for (int e = 0; e < VEC; ++e) o[r][e] = 0.f;
#pragma unroll
    for (int r = 0; r < RO; ++r) {
      m[r] = -INFINITY;
      l[r] = 0.f;
    }
    const char* qs = nullptr;
#pragma unroll 1
    for (int k = 0; k < p.left; ++k) {
      char* rows;
      const unsigned mask = ring.turn(rows);
      if (k == 0) {
        __syncthreads();
        qs = ring.queries();
      }
      const int j0 = (p.chunk + k) * PA_CHUNK + w * 16;
      if (mask == 0 && (!a.scores || j0 >= p.len)) continue;
      const char* vs = rows + 16 * DH * 4;
      float s[4 * NR];                          // [row][i]
#pragma unroll
      for (int x = 0; x < 4 * NR; ++x) s[x] = 0.f;
#pragma unroll UNROLL_S
      for (int ch = 0; ch < DH / 32; ++ch) {
        float4 kv[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) kv[i] = *reinterpret_cast<const float4*>(rows + pa_at<float, DH>(kq + 4 * i, ch * 8 + d));
#pragma unroll
        for (int r = 0; r < NR; ++r) {
          const float4 qv = *reinterpret_cast<const float4*>(qs + pa_q_at<float, DH>(r, ch * 8 + d));    // (r >= nr: what lies there; nobody reads its sums)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            float& x = s[r * 4 + i];
            x = fmaf(qv.x, kv[i].x, fmaf(qv.y, kv[i].y, fmaf(qv.z, kv[i].z, fmaf(qv.w, kv[i].w, x))));
          }
        }
      }
      // the eight lanes' sums: halves are exchanged until each lane has its OWN ones
#pragma unroll
      for (int b = 4, n = 4 * NR; b >= 1; b >>= 1) {
        if (n > 1) {
          n >>= 1;
          const bool up = (d & b) != 0;
#pragma unroll
          for (int x = 0; x < 2 * NR; ++x)
            if (x < n) {
              const float give = up ? s[x] : s[x + n], keep = up ? s[x + n] : s[x];
              s[x] = keep + __shfl_xor_sync(0xffffffffu, give, b);
            }
        } else {
          s[0] += __shfl_xor_sync(0xffffffffu, s[0], b);
        }
      }
      __syncwarp();                             // the K rows have been read: the weights [slot][row] take their place
      float* ps = reinterpret_cast<float*>(rows);
      float corr[RO], pr[RO][KO];
      bool raised = false;
#pragma unroll
      for (int r = 0; r < RO; ++r) {
        float top = -INFINITY;
#pragma unroll
        for (int i = 0; i < KO; ++i) {
          float& x = s[r * KO + i];
          x = (mask >> (kq + 4 * (i0 + i))) & 1 ? x * a.scale_log2 : -INFINITY;
          top = fmaxf(top, x);
        }
        if (a.scores && r0 + r < nr) {
          int row, head;
          pa_row(a, rs, p, r0 + r, row, head);
          float* dst = a.scores + ((long long)row * a.hq + head) * pg_capacity(a.pv);
#pragma unroll
          for (int i = 0; i < KO; ++i) {
            const int j = j0 + kq + 4 * (i0 + i);
            if (j < p.len) dst[j] = s[r * KO + i];
          }
        }
#pragma unroll
        for (int b = 1; b < 32; b <<= 1)
          if (b >= 8 || (SHARE & b)) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, b));
        // (a maximum that rises by little is left: the weights are then at most 2^PA_LAZY)
        corr[r] = 1.f;
        if (top > m[r] + PA_LAZY) {
          corr[r] = pa_scale(m[r], top);
          m[r] = top;
          raised = true;
        }
        l[r] *= corr[r];
#pragma unroll
        for (int i = 0; i < KO; ++i) {
          const float x = s[r * KO + i];
          pr[r][i] = x == -INFINITY ? 0.f : pa_exp2(x - m[r]);
          l[r] += pr[r][i];
        }
      }
#pragma unroll
      for (int i = 0; i < KO; ++i) {
        float* dst = ps + (kq + 4 * (i0 + i)) * NR + r0;
        if constexpr (RO == 2) *reinterpret_cast<float2*>(dst) = make_float2(pr[0][i], pr[1][i]);
        else *dst = pr[0][i];
      }
      if (__any_sync(0xffffffffu, raised)) {
#pragma unroll
        for (int r = 0; r < NR; ++r) {
          const float c = __shfl_sync(0xffffffffu, corr[r % RO], NR == 16 ? r / 2 : r * 8 / NR);
#pragma unroll
          for (int e = 0; e < VEC; ++e) o[r][e] *= c;
        }
      }
      __syncwarp();
#pragma unroll UNROLL_O
      for (int i = 0; i < 16; ++i) {
        float v[VEC], x[NR];
        if constexpr (VEC == 4) {
          const float4 y = *reinterpret_cast<const float4*>(vs + pa_at<float, DH>(i, lane));
          v[0] = y.x; v[1] = y.y; v[2] = y.z; v[3] = y.w;
        } else {
          const float2 y = *reinterpret_cast<const float2*>(vs + pa_at<float, DH>(i, lane >> 1) + (lane & 1) * 8);
          v[0] = y.x; v[1] = y.y;
        }
        if constexpr (NR >= 4) {
#pragma unroll
          for (int r = 0; r < NR; r += 4) {
            const float4 y = *reinterpret_cast<const float4*>(ps + i * NR + r);
            x[r] = y.x; x[r + 1] = y.y; x[r + 2] = y.z; x[r + 3] = y.w;
          }
        } else {
#pragma unroll
          for (int r = 0; r < NR; ++r) x[r] = ps[i * NR + r];
        }
#pragma unroll
        for (int r = 0; r < NR; ++r)
#pragma unroll
          for (int e = 0; e < VEC; ++e) o[r][e] = fmaf(x[r], v[e], o[r][e]);
      }
    }
#pragma unroll
    for (int r = 0; r < RO; ++r)
#pragma unroll
      for (int b = 1; b < 32; b <<= 1)
        if (b >= 8 || (SHARE & b & (NR == 1 ? 6 : 7))) l[r] += __shfl_xor_sync(0xffffffffu, l[r], b);     // (one row: two lanes have each slot)
    pa_finish<float, DH>(a, deal, p, rs, lo, cut, pa_smem, [&](int i0, int n, float* dst, float2* ml) {
#pragma unroll
      for (int r = 0; r < NR; ++r) {
        const int i = r - i0;
        if (i < 0 || i >= n) continue;
#pragma unroll
        for (int e = 0; e < VEC; e += 2) *reinterpret_cast<float2*>(dst + i * DH + (((lane * VEC + e) / 2) ^ (4 * i)) * 2) = make_float2(o[r][e], o[r][e + 1]);
        if (lane == (NR == 16 ? r / 2 : r * 8 / NR)) ml[i] = make_float2(m[r % RO], l[r % RO]);
      }
    });
  }
  pa_join<float, DH>(a, cut);
}

// ---- gathered weights ----------------------------------------------------------------------------------------------------
// KPT slots a thread of one (sequence, KV head), from the scores that the kernel above left: e^{s - lse} of all rows and heads of the group.
// Bound by latency where there are few slots, by the scores' bytes (4 a slot and row) where there are many: PW_AHEAD scores are under way at
// once.
template <int KPT>
__global__ void __launch_bounds__(PW_THREADS) k_paged_weights(const PagedAttnArgs a, int key_blocks) {
  constexpr int ROWS = PW_AHEAD / KPT;
  extern __shared__ float lse2[];                 // [max_rows * group]
  pdl_begin();
  int u = blockIdx.x;
  const int j0 = (u % key_blocks) * (KPT * PW_THREADS);
  u /= key_blocks;
  const int kvh = u % a.pv.hkv, b = u / a.pv.hkv;
  const int len = pg_len(a.pv, a.lens[b]), cap = pg_capacity(a.pv);
  const RowSpan rs = pg_rows(a.pv, a.row_off, b, a.max_rows, a.n_rows);
  if (j0 >= len) return;
  const int n = rs.n * a.group;
  for (int x = threadIdx.x; x < n; x += PW_THREADS) {
    const float l = a.row_lse[(long long)(rs.first + x / a.group) * a.hq + kvh * a.group + x % a.group];
    lse2[x] = l == -INFINITY ? INFINITY : l;      // a row that saw nothing has no weight
  }
  const long long base = ((long long)b * a.pv.hkv + kvh) * cap;
  const int j = j0 + threadIdx.x;
  // scores of row x of the group's: `heads` of a row lie one behind the other, the next row's a.hq heads on
  const float* src = a.scores + ((long long)rs.first * a.hq + kvh * a.group) * cap + j;
  const long long wrap = (long long)(a.hq - a.group + 1) * cap;
  int h = 0;
  float s[ROWS][KPT];
  auto load = [&](int x) {
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
#pragma unroll
      for (int k = 0; k < KPT; ++k) s[i][k] = x + i < n && j + k * PW_THREADS < len ? __ldcg(src + k * PW_THREADS) : -INFINITY;
      const bool last = ++h == a.group;
      src += last ? wrap : cap;
      h = last ? 0 : h;
    }
  };
  load(0);                                        // (while the rows' sums are on their way)
  float sum[KPT];
#pragma unroll
  for (int k = 0; k < KPT; ++k) sum[k] = j + k * PW_THREADS < len && a.weights_in ? a.weights_in[base + j + k * PW_THREADS] : 0.f;
  __syncthreads();
  float add[KPT] = {};
  for (int x = 0; x < n; x += ROWS) {
#pragma unroll
    for (int i = 0; i < ROWS; ++i)
#pragma unroll
      for (int k = 0; k < KPT; ++k) add[k] += pa_exp2(s[i][k] - lse2[min(x + i, n - 1)]);
    if (x + ROWS < n) load(x + ROWS);
  }
#pragma unroll
  for (int k = 0; k < KPT; ++k)
    if (j + k * PW_THREADS < len) a.weights_out[base + j + k * PW_THREADS] = sum[k] + add[k];
}

}  // namespace lsp
