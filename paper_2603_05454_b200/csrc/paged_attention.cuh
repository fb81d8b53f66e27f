// Attention of a few new rows per sequence over a paged key-value cache, split over the cache's length and joined.
//
// For a sequence's rows r, query heads h of a KV head's group and cached slots j < len:
//   s = scale q[r,h] . k[j],  out[r,h] = sum_j e^{s - m} v[j] / sum_j e^{s - m},  lse = m + ln(sum),
//   weights_out[j] = weights_in[j] + sum over (r, h) of e^{s - lse}.
// Every row sees every slot (the library's attention is bidirectional).
//
// The stream of K and V from HBM bounds it: 4 dh rows * group flops per 4 dh bytes.  So:
//  * The slots of every (sequence, KV head, tile of 16 (row, head) pairs) are cut into chunks of 64, all chunks of the batch are
//    numbered through, and each CTA of a grid that fills the SMs takes an equal run of them, whatever the lengths are.  A unit
//    that one CTA holds whole is written by it; the parts (m, l, o) of a unit that a run's end cuts go to the workspace and
//    k_paged_join adds them in order.  No atomics, no counters, the same bits every time.
//  * A warp takes 16 slots of a chunk and loads them itself: a ring of its own in shared memory, filled by cp.async, page ids one
//    turn ahead of the rows they lead to.  The warps of a CTA meet only where a unit ends.
//  * mma.sync m16n8k16, not tcgen05: a tile has at most 16 rows (often one), an M of 128 would be 1/8 to 1/128 full, and the
//    legacy pipe needs a third of the time that the bytes take.
#pragma once
#include "attention_mma.cuh"
#include "paged_common.cuh"

namespace lsp {

constexpr int PA_CHUNK = 64;            // slots of a chunk: 16 per warp
constexpr int PA_WARPS = 4;
constexpr int PA_STAGES = 3;
constexpr int PA_ROWS = 16;             // (row, head) pairs of a unit
constexpr int PA_MAX_BATCH = 1024;
constexpr int PA_MAX_CTAS = 512;
constexpr int PJ_THREADS = 256;
constexpr int PJ_KEYS = 1024;           // slots of a weights block

struct PagedAttnArgs {
  PagedView pv;
  const void* q;
  void* out;
  long long ldq, ldo;
  const int *lens, *row_off;
  int hq, group, max_rows, n_rows, n_cta;
  float scale_log2;
  float* lse;                  // [n_rows][hq] or null
  float* part_o;               // [2 n_cta][16][dh]
  float2* part_ml;             // [2 n_cta][16]: m (in log2 units), l
  float* scores;               // [n_rows][hq][capacity] in log2 units, or null: no weights wanted
  float2* row_ml;              // [n_rows][hq]: m, l of units that one CTA held whole (with weights)
  const float* weights_in;
  float* weights_out;
};

template <typename T, int DH>
constexpr int pa_stage_bytes() { return 2 * 16 * DH * (int)sizeof(T); }
template <typename T, int DH>
constexpr int pa_merge_bytes() { return 2 * 8 * DH * 4; }
template <typename T, int DH>
constexpr int pa_smem_bytes() {
  return PA_WARPS * PA_STAGES * pa_stage_bytes<T, DH>() + pa_merge_bytes<T, DH>() + PA_WARPS * PA_ROWS * 8 + (PA_MAX_BATCH + 1) * 4 +
         (sizeof(T) == 4 ? PA_ROWS * (DH + 4) * 4 : 0);
}

// Chunks of the units of sequence b, all KV heads and row tiles together, before b in pre[]; chunks of one unit: pa_chunks.
__device__ __forceinline__ int pa_chunks(int len) { return (len + PA_CHUNK - 1) / PA_CHUNK; }

// pre[b] = chunks of all sequences before b, b <= batch (a block-wide scan; ends with a barrier).
template <int THREADS>
__device__ __forceinline__ void pa_prefix(const PagedAttnArgs& a, int* pre, int* warp_sums) {
  const int B = a.pv.batch, lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  int carry = 0;
  for (int b0 = 0; b0 < B; b0 += THREADS) {
    const int b = b0 + threadIdx.x;
    int n = 0;
    if (b < B) {
      const RowSpan rs = pg_rows(a.pv, a.row_off, b, a.max_rows, a.n_rows);
      n = pa_chunks(pg_len(a.pv, a.lens, b)) * a.pv.hkv * ((rs.n * a.group + PA_ROWS - 1) / PA_ROWS);
    }
    int x = n;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, x, o);
      if (lane >= o) x += y;
    }
    if (lane == 31) warp_sums[w] = x;
    __syncthreads();
    int before = carry, all = carry;
#pragma unroll
    for (int i = 0; i < THREADS / 32; ++i) {
      const int s = warp_sums[i];
      before += i < w ? s : 0;
      all += s;
    }
    if (b < B) pre[b] = before + x - n;
    carry = all;
    __syncthreads();
  }
  if (threadIdx.x == 0) pre[B] = carry;
  __syncthreads();
}
// CTAs that get a run (at least a chunk each); first chunk of CTA i's run.
__device__ __forceinline__ int pa_ctas(int total, int n_cta) { return min(total, n_cta); }
__device__ __forceinline__ int pa_run(int total, int i, int n_cta) { return (int)((long long)total * i / n_cta); }
// The CTA whose run holds chunk c.
__device__ __forceinline__ int pa_owner(int total, int c, int n_cta) { return (int)((((long long)c + 1) * n_cta - 1) / total); }

// A place in the run: sequence, KV head, row tile, chunk of the unit.
struct PaPlace {
  int b, kvh, rt, chunk, chunks, len, left;        // left: chunks of this unit that belong to the run, from here on
};
__device__ __forceinline__ PaPlace pa_place(const PagedAttnArgs& a, const int* pre, int c, int hi) {
  PaPlace p;
  int lo = 0, up = a.pv.batch;                     // pre[lo] <= c < pre[up]
  while (up - lo > 1) {
    const int mid = (lo + up) >> 1;
    if (pre[mid] <= c) lo = mid; else up = mid;
  }
  p.b = lo;
  const int n = a.lens[lo], cap = pg_capacity(a.pv);
  p.len = n > cap ? cap : n;
  p.chunks = pa_chunks(p.len);
  const int tiles = (pre[lo + 1] - pre[lo]) / (p.chunks * a.pv.hkv);
  const int u = (c - pre[lo]) / p.chunks;
  p.chunk = c - pre[lo] - u * p.chunks;
  p.kvh = u / tiles;
  p.rt = u - p.kvh * tiles;
  p.left = min(p.chunks - p.chunk, hi - c);
  return p;
}

// Byte offset of 16-byte chunk c of row r in a [16][DH] tile: chunks are exchanged within groups of eight by the row, so that eight
// rows' chunks c lie in different banks.
template <typename T, int DH>
__device__ __forceinline__ int pa_at(int r, int c) {
  return r * DH * (int)sizeof(T) + ((c ^ (r & 7)) << 4);
}

// One warp's loads: the rows of its 16 slots of a chunk, K then V, into one stage of its ring.
template <typename T, int DH>
struct PaLoader {
  static constexpr int CPR = DH * (int)sizeof(T) / 16;      // 16-byte chunks of a row
  const PagedAttnArgs& a;
  const int* pre;
  int c, hi, w, lane;
  PaPlace p;
  int page_id;                  // (lanes 0 to 15) page of this lane's slot of chunk c, asked for a turn ahead
  __device__ __forceinline__ PaLoader(const PagedAttnArgs& a_, const int* pre_, int lo, int hi_, int w_, int lane_)
      : a(a_), pre(pre_), c(lo), hi(hi_), w(w_), lane(lane_), page_id(-1) {
    if (c < hi) {
      p = pa_place(a, pre, c, hi);
      ask();
    }
  }
  __device__ __forceinline__ int slot() const { return p.chunk * PA_CHUNK + w * 16 + (lane & 15); }
  __device__ __forceinline__ void ask() {
    const int j = slot();
    page_id = j < p.len ? pg_page(a.pv, p.b, j) : -1;
  }
  // Returns a mask of the rows that are real slots.
  __device__ __forceinline__ unsigned issue(char* stage) {
    unsigned live = 0;
    if (c < hi) {
      const int j = slot();
      const bool ok = page_id >= 0;
      live = __ballot_sync(0xffffffffu, ok) & 0xffffu;
      const long long off = ok ? ((long long)page_id * a.pv.page_stride + (long long)(j % a.pv.page) * a.pv.row_stride + (long long)p.kvh * a.pv.head_stride) : 0;
      const uint32_t ks = smem_u32(stage), vs = ks + 16 * DH * (int)sizeof(T);
#pragma unroll
      for (int i = 0; i < 16 * CPR / 32; ++i) {
        const int r = (i * 32 + lane) / CPR, ch = (i * 32 + lane) % CPR;
        const long long o = __shfl_sync(0xffffffffu, off, r) * (int)sizeof(T) + ch * 16;
        const bool v = (live >> r) & 1;
        const int d = pa_at<T, DH>(r, ch);
        cp_async16(ks + d, a.pv.k + (v ? o : 0), v);
        cp_async16(vs + d, a.pv.v + (v ? o : 0), v);
      }
      ++c;
      if (c < hi) {
        if (--p.left > 0) ++p.chunk;
        else p = pa_place(a, pre, c, hi);
        ask();
      }
    }
    cp_async_commit();
    return live;
  }
};

// Where a (row, head) pair of a unit lies: packed row and query head; false behind the sequence's last row.
__device__ __forceinline__ bool pa_row(const PagedAttnArgs& a, const RowSpan& rs, const PaPlace& p, int i, int& row, int& head) {
  const int x = p.rt * PA_ROWS + i;
  if (x >= rs.n * a.group) return false;
  row = rs.first + x / a.group;
  head = p.kvh * a.group + x % a.group;
  return true;
}

// e^(x) of the online softmax in log2 units; -inf - -inf (nothing seen yet) counts as nothing.
__device__ __forceinline__ float pa_scale(float m_old, float m_new) { return m_old == -INFINITY ? 0.f : exp2f(m_old - m_new); }

// Natural log of the sum of exponentials from the maximum in log2 units and the sum; -inf where nothing was seen.
__device__ __forceinline__ float pa_lse(float m, float l) { return l == 0.f ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f; }

// ---- bf16: tensor cores --------------------------------------------------------------------------------------------------
// Softmax weights are fed to the P V product as the sum of two bf16 numbers (16 bits of mantissa): the tensor pipe has the time,
// and the output is then as exact as one with fp32 weights.
template <int DH>
__global__ void __launch_bounds__(PA_WARPS * 32, 2) k_paged_attn_mma(const PagedAttnArgs a) {
  extern __shared__ __align__(128) char pa_smem[];
  constexpr int SB = pa_stage_bytes<bf16, DH>();
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
  char* ring = pa_smem + w * PA_STAGES * SB;
  float* merge = reinterpret_cast<float*>(pa_smem + PA_WARPS * PA_STAGES * SB);
  float2* ml_s = reinterpret_cast<float2*>(merge + 2 * 8 * DH);       // [warp][16]
  int* pre = reinterpret_cast<int*>(ml_s + PA_WARPS * PA_ROWS);
  __shared__ int warp_sums[PA_WARPS];
  pdl_begin();
  pa_prefix<PA_WARPS * 32>(a, pre, warp_sums);
  const int total = pre[a.pv.batch];
  const int n_cta = pa_ctas(total, a.n_cta);
  if ((int)blockIdx.x >= n_cta) return;
  const int lo = pa_run(total, blockIdx.x, n_cta), hi = pa_run(total, blockIdx.x + 1, n_cta);

  PaLoader<bf16, DH> ld(a, pre, lo, hi, w, lane);
  unsigned live[PA_STAGES];                   // masks of the stages in flight, oldest first
#pragma unroll
  for (int s = 0; s < PA_STAGES - 1; ++s) live[s] = ld.issue(ring + s * SB);
  live[PA_STAGES - 1] = 0;

  int c = lo, stage = 0;
  while (c < hi) {
    // ---- a unit, or the part of it that belongs to this run
    const PaPlace p = pa_place(a, pre, c, hi);
    const RowSpan rs = pg_rows(a.pv, a.row_off, p.b, a.max_rows, a.n_rows);
    uint32_t qf[DH / 16][4];
    int row[2], head[2];
    bool real[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      real[h] = pa_row(a, rs, p, g + 8 * h, row[h], head[h]);
      const uint32_t* src = reinterpret_cast<const uint32_t*>((const bf16*)a.q + (real[h] ? (long long)row[h] * a.ldq + head[h] * DH : 0)) + t;
#pragma unroll
      for (int kk = 0; kk < DH / 16; ++kk) {
        qf[kk][h] = real[h] ? src[kk * 8] : 0u;
        qf[kk][2 + h] = real[h] ? src[kk * 8 + 4] : 0u;
      }
    }
    float o[DH / 8][4];
#pragma unroll
    for (int i = 0; i < DH / 8; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;
    float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};

    for (int k = 0; k < p.left; ++k) {
      // the next chunk's rows into the stage that was read last turn
      {
        int s = stage + PA_STAGES - 1;
        if (s >= PA_STAGES) s -= PA_STAGES;
        __syncwarp();
        live[PA_STAGES - 1] = ld.issue(ring + s * SB);
      }
      cp_async_wait<PA_STAGES - 1>();
      __syncwarp();
      const unsigned mask = live[0];
#pragma unroll
      for (int s = 0; s + 1 < PA_STAGES; ++s) live[s] = live[s + 1];
      const uint32_t ks = smem_u32(ring + stage * SB), vs = ks + 16 * DH * 2;
      if (++stage == PA_STAGES) stage = 0;
      const int j0 = (p.chunk + k) * PA_CHUNK + w * 16;
      if (mask == 0 && (!a.scores || j0 >= p.len)) continue;
      // S = Q K^T: 16 rows x 16 slots
      float s[2][4];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        float s2[4] = {0.f, 0.f, 0.f, 0.f};
        s[j][0] = s[j][1] = s[j][2] = s[j][3] = 0.f;
#pragma unroll
        for (int kk = 0; kk < DH / 16; kk += 2) {
          uint32_t b0, b1, b2, b3;
          ldsm_x4(ks + pa_at<bf16, DH>(j * 8 + (lane & 7), kk * 2 + (lane >> 3)), b0, b1, b2, b3);
          mma_bf16(s[j], qf[kk][0], qf[kk][1], qf[kk][2], qf[kk][3], b0, b1);
          mma_bf16(s2, qf[kk + 1][0], qf[kk + 1][1], qf[kk + 1][2], qf[kk + 1][3], b2, b3);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) s[j][e] += s2[e];
      }
      float mx[2] = {-INFINITY, -INFINITY};
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          s[j][e] = (mask >> (j * 8 + 2 * t + (e & 1))) & 1 ? s[j][e] * a.scale_log2 : -INFINITY;
          mx[e >> 1] = fmaxf(mx[e >> 1], s[j][e]);
        }
      if (a.scores) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
          if (real[h]) {
            float* dst = a.scores + ((long long)row[h] * a.hq + head[h]) * pg_capacity(a.pv) + j0 + 2 * t;
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
              for (int e = 0; e < 2; ++e)
                if (j0 + j * 8 + 2 * t + e < p.len) dst[j * 8 + e] = s[j][2 * h + e];
          }
      }
      float corr[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        mx[h] = fmaxf(mx[h], __shfl_xor_sync(0xffffffffu, mx[h], 1));
        mx[h] = fmaxf(mx[h], __shfl_xor_sync(0xffffffffu, mx[h], 2));
        const float m_new = fmaxf(m[h], mx[h]);
        corr[h] = pa_scale(m[h], m_new);
        m[h] = m_new;
      }
      uint32_t hi_[4], lo_[4];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        l[h] *= corr[h];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const float x = s[j][2 * h], y = s[j][2 * h + 1];
          const float p0 = x == -INFINITY ? 0.f : exp2f(x - m[h]), p1 = y == -INFINITY ? 0.f : exp2f(y - m[h]);
          l[h] += p0 + p1;
          const __nv_bfloat162 ph = __floats2bfloat162_rn(p0, p1);
          hi_[j * 2 + h] = *reinterpret_cast<const uint32_t*>(&ph);
          lo_[j * 2 + h] = pack_bf16(p0 - __bfloat162float(ph.x), p1 - __bfloat162float(ph.y));
        }
      }
      if (__any_sync(0xffffffffu, corr[0] != 1.f || corr[1] != 1.f)) {
#pragma unroll
        for (int i = 0; i < DH / 8; ++i) {
          o[i][0] *= corr[0]; o[i][1] *= corr[0];
          o[i][2] *= corr[1]; o[i][3] *= corr[1];
        }
      }
      // O += P V
#pragma unroll
      for (int nt = 0; nt < DH / 8; nt += 2) {
        uint32_t b0, b1, b2, b3;
        ldsm_x4_t(vs + pa_at<bf16, DH>((lane & 7) + ((lane >> 3) & 1) * 8, nt + (lane >> 4)), b0, b1, b2, b3);
        mma_bf16(o[nt], hi_[0], hi_[1], hi_[2], hi_[3], b0, b1);
        mma_bf16(o[nt + 1], hi_[0], hi_[1], hi_[2], hi_[3], b2, b3);
        mma_bf16(o[nt], lo_[0], lo_[1], lo_[2], lo_[3], b0, b1);
        mma_bf16(o[nt + 1], lo_[0], lo_[1], lo_[2], lo_[3], b2, b3);
      }
    }

    // ---- the four warps' parts of the unit: to one maximum, then added in pairs (half of the rows at a time)
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      l[h] += __shfl_xor_sync(0xffffffffu, l[h], 1);
      l[h] += __shfl_xor_sync(0xffffffffu, l[h], 2);
      if (t == 0) ml_s[w * PA_ROWS + g + 8 * h] = make_float2(m[h], l[h]);
    }
    __syncthreads();
    float mt[2], lt[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      mt[h] = -INFINITY;
      lt[h] = 0.f;
#pragma unroll
      for (int i = 0; i < PA_WARPS; ++i) mt[h] = fmaxf(mt[h], ml_s[i * PA_ROWS + g + 8 * h].x);
#pragma unroll
      for (int i = 0; i < PA_WARPS; ++i) {
        const float2 x = ml_s[i * PA_ROWS + g + 8 * h];
        lt[h] += x.y * pa_scale(x.x, mt[h]);
      }
      const float f = pa_scale(m[h], mt[h]);
#pragma unroll
      for (int i = 0; i < DH / 8; ++i) {
        o[i][2 * h] *= f;
        o[i][2 * h + 1] *= f;
      }
    }
    const int n_real = rs.n * a.group - p.rt * PA_ROWS;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      if (8 * h >= n_real) break;               // (the same for the whole block)
#pragma unroll
      for (int step = 0; step < 2; ++step) {
        const int half = 2 >> step;             // warps [half, 2 half) hand over to [0, half)
        if (w >= half && w < 2 * half) {
          float2* dst = reinterpret_cast<float2*>(merge + ((w - half) * 8 + g) * DH);
#pragma unroll
          for (int i = 0; i < DH / 8; ++i) dst[(i * 4 + t) ^ g] = make_float2(o[i][2 * h], o[i][2 * h + 1]);
        }
        __syncthreads();
        if (w < half) {
          const float2* src = reinterpret_cast<const float2*>(merge + (w * 8 + g) * DH);
#pragma unroll
          for (int i = 0; i < DH / 8; ++i) {
            const float2 x = src[(i * 4 + t) ^ g];
            o[i][2 * h] += x.x;
            o[i][2 * h + 1] += x.y;
          }
        }
        __syncthreads();
      }
    }
    if (w == 0) {
      if (p.left == p.chunks) {                 // the whole unit: the result
#pragma unroll
        for (int h = 0; h < 2; ++h)
          if (real[h]) {
            const float inv = 1.f / lt[h];
            uint32_t* dst = reinterpret_cast<uint32_t*>((bf16*)a.out + (long long)row[h] * a.ldo + head[h] * DH) + t;
#pragma unroll
            for (int i = 0; i < DH / 8; ++i) dst[i * 4] = lt[h] == 0.f ? 0u : pack_bf16(o[i][2 * h] * inv, o[i][2 * h + 1] * inv);
            if (t == 0) {
              const long long at = (long long)row[h] * a.hq + head[h];
              if (a.lse) a.lse[at] = pa_lse(mt[h], lt[h]);
              if (a.scores) a.row_ml[at] = make_float2(mt[h], lt[h]);
            }
          }
      } else {
        const int part = 2 * blockIdx.x + (c == lo ? 0 : 1);
#pragma unroll
        for (int h = 0; h < 2; ++h)
          if (real[h]) {
            float2* dst = reinterpret_cast<float2*>(a.part_o + ((long long)part * PA_ROWS + g + 8 * h) * DH) + t;
#pragma unroll
            for (int i = 0; i < DH / 8; ++i) dst[i * 4] = make_float2(o[i][2 * h], o[i][2 * h + 1]);
            if (t == 0) a.part_ml[part * PA_ROWS + g + 8 * h] = make_float2(mt[h], lt[h]);
          }
      }
    }
    c += p.left;
  }
  cp_async_wait<0>();
}

// ---- fp32: CUDA cores ----------------------------------------------------------------------------------------------------
// Scores: a lane takes one slot and half of the dimensions; P V: a lane takes DH / 32 dimensions.  16 rows cost 256 FMAs a lane and
// 16 slots either way, a third of the time the bytes take.
template <int DH>
__global__ void __launch_bounds__(PA_WARPS * 32) k_paged_attn_simt(const PagedAttnArgs a) {
  extern __shared__ __align__(128) char pa_smem[];
  constexpr int SB = pa_stage_bytes<float, DH>();
  constexpr int VEC = DH / 32;                  // dimensions of a lane in P V
  constexpr int HALF = DH / 2;
  constexpr int LDQ = DH + 4;                   // second half of a query 16 bytes on: the two half-warps read different banks
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  char* ring = pa_smem + w * PA_STAGES * SB;
  float* merge = reinterpret_cast<float*>(pa_smem + PA_WARPS * PA_STAGES * SB);
  float2* ml_s = reinterpret_cast<float2*>(merge + 2 * 8 * DH);
  float* qs = reinterpret_cast<float*>(ml_s + PA_WARPS * PA_ROWS);    // [16][DH + 4]
  int* pre = reinterpret_cast<int*>(qs + PA_ROWS * LDQ);
  __shared__ int warp_sums[PA_WARPS];
  pdl_begin();
  pa_prefix<PA_WARPS * 32>(a, pre, warp_sums);
  const int total = pre[a.pv.batch];
  const int n_cta = pa_ctas(total, a.n_cta);
  if ((int)blockIdx.x >= n_cta) return;
  const int lo = pa_run(total, blockIdx.x, n_cta), hi = pa_run(total, blockIdx.x + 1, n_cta);

  PaLoader<float, DH> ld(a, pre, lo, hi, w, lane);
  unsigned live[PA_STAGES];
#pragma unroll
  for (int s = 0; s < PA_STAGES - 1; ++s) live[s] = ld.issue(ring + s * SB);
  live[PA_STAGES - 1] = 0;

  int c = lo, stage = 0;
  const int key = lane & 15, half = lane >> 4;
  while (c < hi) {
    const PaPlace p = pa_place(a, pre, c, hi);
    const RowSpan rs = pg_rows(a.pv, a.row_off, p.b, a.max_rows, a.n_rows);
    const int nr = min(PA_ROWS, rs.n * a.group - p.rt * PA_ROWS);
    for (int i = threadIdx.x; i < nr * DH; i += PA_WARPS * 32) {
      const int r = i / DH, d = i % DH;
      int row, head;
      pa_row(a, rs, p, r, row, head);
      qs[r * LDQ + d + (d >= HALF ? 4 : 0)] = ((const float*)a.q)[(long long)row * a.ldq + head * DH + d];
    }
    __syncthreads();
    float o[PA_ROWS][VEC], m[PA_ROWS], l[PA_ROWS];       // m: the same in all lanes; l: this lane's slots
#pragma unroll
    for (int r = 0; r < PA_ROWS; ++r) {
      m[r] = -INFINITY;
      l[r] = 0.f;
#pragma unroll
      for (int e = 0; e < VEC; ++e) o[r][e] = 0.f;
    }
    for (int k = 0; k < p.left; ++k) {
      {
        int s = stage + PA_STAGES - 1;
        if (s >= PA_STAGES) s -= PA_STAGES;
        __syncwarp();
        live[PA_STAGES - 1] = ld.issue(ring + s * SB);
      }
      cp_async_wait<PA_STAGES - 1>();
      __syncwarp();
      const unsigned mask = live[0];
#pragma unroll
      for (int s = 0; s + 1 < PA_STAGES; ++s) live[s] = live[s + 1];
      const char* ks = ring + stage * SB;
      const char* vs = ks + 16 * DH * 4;
      if (++stage == PA_STAGES) stage = 0;
      const int j = (p.chunk + k) * PA_CHUNK + w * 16 + key;
      if (mask == 0 && (!a.scores || j - key >= p.len)) continue;
      float s[PA_ROWS];
#pragma unroll
      for (int r = 0; r < PA_ROWS; ++r) s[r] = 0.f;
#pragma unroll 4
      for (int ch = 0; ch < HALF / 4; ++ch) {
        const float4 kv = *reinterpret_cast<const float4*>(ks + pa_at<float, DH>(key, half * (HALF / 4) + ch));
#pragma unroll
        for (int r = 0; r < PA_ROWS; ++r)
          if (r < nr) {
            const float4 qv = *reinterpret_cast<const float4*>(qs + r * LDQ + half * (HALF + 4) + ch * 4);
            s[r] = fmaf(qv.x, kv.x, fmaf(qv.y, kv.y, fmaf(qv.z, kv.z, fmaf(qv.w, kv.w, s[r]))));
          }
      }
#pragma unroll
      for (int r = 0; r < PA_ROWS; ++r)
        if (r < nr) {
          s[r] += __shfl_xor_sync(0xffffffffu, s[r], 16);
          s[r] = (mask >> key) & 1 ? s[r] * a.scale_log2 : -INFINITY;
          if (a.scores && half == 0 && j < p.len) {
            int row, head;
            pa_row(a, rs, p, r, row, head);
            a.scores[((long long)row * a.hq + head) * pg_capacity(a.pv) + j] = s[r];
          }
          const float m_new = fmaxf(m[r], warp_max(s[r]));
          const float corr = pa_scale(m[r], m_new);
          m[r] = m_new;
          s[r] = s[r] == -INFINITY ? 0.f : exp2f(s[r] - m_new);
          l[r] = l[r] * corr + s[r];
#pragma unroll
          for (int e = 0; e < VEC; ++e) o[r][e] *= corr;
        }
#pragma unroll 4
      for (int i = 0; i < 16; ++i) {
        float v[VEC];
        if constexpr (VEC == 4) {
          const float4 x = *reinterpret_cast<const float4*>(vs + pa_at<float, DH>(i, lane));
          v[0] = x.x; v[1] = x.y; v[2] = x.z; v[3] = x.w;
        } else {
          const float2 x = *reinterpret_cast<const float2*>(vs + pa_at<float, DH>(i, lane >> 1) + (lane & 1) * 8);
          v[0] = x.x; v[1] = x.y;
        }
#pragma unroll
        for (int r = 0; r < PA_ROWS; ++r)
          if (r < nr) {
            const float pr = __shfl_sync(0xffffffffu, s[r], i);
#pragma unroll
            for (int e = 0; e < VEC; ++e) o[r][e] = fmaf(pr, v[e], o[r][e]);
          }
      }
    }
    // ---- join the four warps
#pragma unroll
    for (int r = 0; r < PA_ROWS; ++r)
      if (r < nr) {
        const float s = warp_sum(half == 0 ? l[r] : 0.f);
        if (lane == 0) ml_s[w * PA_ROWS + r] = make_float2(m[r], s);
      }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < PA_ROWS; ++r)
      if (r < nr) {
        float mt = -INFINITY, lt = 0.f;
#pragma unroll
        for (int i = 0; i < PA_WARPS; ++i) mt = fmaxf(mt, ml_s[i * PA_ROWS + r].x);
#pragma unroll
        for (int i = 0; i < PA_WARPS; ++i) lt += ml_s[i * PA_ROWS + r].y * pa_scale(ml_s[i * PA_ROWS + r].x, mt);
        const float f = pa_scale(m[r], mt);
#pragma unroll
        for (int e = 0; e < VEC; ++e) o[r][e] *= f;
        m[r] = mt;
        l[r] = lt;
      }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      if (8 * h >= nr) break;
#pragma unroll
      for (int step = 0; step < 2; ++step) {
        const int n = 2 >> step;
        if (w >= n && w < 2 * n)
#pragma unroll
          for (int r = 0; r < 8; ++r)
#pragma unroll
            for (int e = 0; e < VEC; ++e) merge[((w - n) * 8 + r) * DH + lane * VEC + e] = o[8 * h + r][e];
        __syncthreads();
        if (w < n)
#pragma unroll
          for (int r = 0; r < 8; ++r)
#pragma unroll
            for (int e = 0; e < VEC; ++e) o[8 * h + r][e] += merge[(w * 8 + r) * DH + lane * VEC + e];
        __syncthreads();
      }
    }
    if (w == 0) {
      const bool whole = p.left == p.chunks;
      const int part = 2 * blockIdx.x + (c == lo ? 0 : 1);
#pragma unroll
      for (int r = 0; r < PA_ROWS; ++r)
        if (r < nr) {
          int row, head;
          pa_row(a, rs, p, r, row, head);
          float* dst = whole ? (float*)a.out + (long long)row * a.ldo + head * DH : a.part_o + ((long long)part * PA_ROWS + r) * DH;
          const float inv = whole ? (l[r] == 0.f ? 0.f : 1.f / l[r]) : 1.f;
#pragma unroll
          for (int e = 0; e < VEC; ++e) dst[lane * VEC + e] = o[r][e] * inv;
          if (lane == 0) {
            if (whole) {
              const long long at = (long long)row * a.hq + head;
              if (a.lse) a.lse[at] = pa_lse(m[r], l[r]);
              if (a.scores) a.row_ml[at] = make_float2(m[r], l[r]);
            } else {
              a.part_ml[part * PA_ROWS + r] = make_float2(m[r], l[r]);
            }
          }
        }
    }
    c += p.left;
  }
  cp_async_wait<0>();
}

// ---- join ----------------------------------------------------------------------------------------------------------------
// The parts of unit (b, kvh, rt): CTAs first..last of the attention kernel's grid hold one each.
struct PaParts {
  int first, last, u0, total, n_cta;
  __device__ __forceinline__ int slot(int i) const { return 2 * i + (pa_run(total, i, n_cta) >= u0 ? 0 : 1); }
};
__device__ __forceinline__ PaParts pa_parts(const PagedAttnArgs& a, const int* pre, int b, int unit, int chunks) {
  PaParts p;
  p.total = pre[a.pv.batch];
  p.n_cta = pa_ctas(p.total, a.n_cta);
  p.u0 = pre[b] + unit * chunks;
  p.first = pa_owner(p.total, p.u0, p.n_cta);
  p.last = pa_owner(p.total, p.u0 + chunks - 1, p.n_cta);
  return p;
}

// Blocks [0, join_blocks): one (unit, row) each, the warps take its parts in turn.  The others: PJ_KEYS slots of one (sequence, KV head) each, the
// rows' weights there from the scores, which were left in log2 units.
template <typename T, int DH>
__global__ void __launch_bounds__(PJ_THREADS) k_paged_join(const PagedAttnArgs a, int tiles, int rows_tile, int join_blocks, int key_blocks) {
  __shared__ int pre[PA_MAX_BATCH + 1];
  __shared__ int warp_sums[PJ_THREADS / 32];
  __shared__ float acc[PJ_THREADS / 32][DH];
  constexpr int VEC = DH / 32, NW = PJ_THREADS / 32;
  extern __shared__ float lse2[];                 // [max_rows * group] (weights blocks)
  pdl_begin();
  pa_prefix<PJ_THREADS>(a, pre, warp_sums);
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  if ((int)blockIdx.x < join_blocks) {
    const int i = blockIdx.x % rows_tile;
    int u = blockIdx.x / rows_tile;
    PaPlace p;
    p.rt = u % tiles;
    u /= tiles;
    p.kvh = u % a.pv.hkv;
    p.b = u / a.pv.hkv;
    const RowSpan rs = pg_rows(a.pv, a.row_off, p.b, a.max_rows, a.n_rows);
    int row, head;
    if (!pa_row(a, rs, p, i, row, head)) return;
    const int chunks = pa_chunks(pg_len(a.pv, a.lens, p.b));
    T* out = (T*)a.out + (long long)row * a.ldo + head * DH;
    const long long at = (long long)row * a.hq + head;
    if (chunks == 0) {                            // no slot: nothing seen
      if (threadIdx.x < DH) out[threadIdx.x] = from_f<T>(0.f);
      if (threadIdx.x == 0 && a.lse) a.lse[at] = -INFINITY;
      return;
    }
    const int my_tiles = (rs.n * a.group + PA_ROWS - 1) / PA_ROWS;
    const PaParts pt = pa_parts(a, pre, p.b, p.kvh * my_tiles + p.rt, chunks);
    if (pt.first == pt.last) return;              // one CTA had it whole and wrote the result
    float m = -INFINITY;
    for (int k = pt.first + lane; k <= pt.last; k += 32) m = fmaxf(m, a.part_ml[pt.slot(k) * PA_ROWS + i].x);
    m = warp_max(m);
    float l = 0.f, o[VEC];
#pragma unroll
    for (int e = 0; e < VEC; ++e) o[e] = 0.f;
#pragma unroll 4
    for (int k = pt.first + w; k <= pt.last; k += NW) {
      const int s = pt.slot(k) * PA_ROWS + i;
      const float2 ml = a.part_ml[s];
      const float f = pa_scale(ml.x, m);
      const float* src = a.part_o + (long long)s * DH + lane * VEC;
      l += ml.y * f;
#pragma unroll
      for (int e = 0; e < VEC; ++e) o[e] = fmaf(src[e], f, o[e]);
    }
#pragma unroll
    for (int e = 0; e < VEC; ++e) acc[w][lane * VEC + e] = o[e];
    float* ls = reinterpret_cast<float*>(warp_sums);
    if (lane == 0) ls[w] = l;
    __syncthreads();
    float lt = 0.f;
#pragma unroll
    for (int k = 0; k < NW; ++k) lt += ls[k];
    if (threadIdx.x < DH) {
      float s = 0.f;
#pragma unroll
      for (int k = 0; k < NW; ++k) s += acc[k][threadIdx.x];
      out[threadIdx.x] = from_f<T>(lt == 0.f ? 0.f : s / lt);
    }
    if (threadIdx.x == 0 && a.lse) a.lse[at] = pa_lse(m, lt);
    return;
  }
  // ---- gathered weights
  int u = blockIdx.x - join_blocks;
  const int j0 = (u % key_blocks) * PJ_KEYS;
  u /= key_blocks;
  const int kvh = u % a.pv.hkv, b = u / a.pv.hkv;
  const int len = pg_len(a.pv, a.lens, b), chunks = pa_chunks(len), cap = pg_capacity(a.pv);
  if (j0 >= len) return;
  const RowSpan rs = pg_rows(a.pv, a.row_off, b, a.max_rows, a.n_rows);
  const int n = rs.n * a.group, my_tiles = (n + PA_ROWS - 1) / PA_ROWS;
  for (int x = w; x < n; x += NW) {
    const PaParts pt = pa_parts(a, pre, b, kvh * my_tiles + x / PA_ROWS, chunks);
    float m = -INFINITY, l = 0.f;
    if (pt.first == pt.last) {
      const float2 ml = a.row_ml[(long long)(rs.first + x / a.group) * a.hq + kvh * a.group + x % a.group];
      m = ml.x;
      l = ml.y;
    } else {
      for (int k = pt.first + lane; k <= pt.last; k += 32) m = fmaxf(m, a.part_ml[pt.slot(k) * PA_ROWS + x % PA_ROWS].x);
      m = warp_max(m);
      for (int k = pt.first + lane; k <= pt.last; k += 32) {
        const float2 ml = a.part_ml[pt.slot(k) * PA_ROWS + x % PA_ROWS];
        l += ml.y * pa_scale(ml.x, m);
      }
      l = warp_sum(l);
    }
    if (lane == 0) lse2[x] = l == 0.f ? INFINITY : m + log2f(l);
  }
  __syncthreads();
  const long long base = ((long long)b * a.pv.hkv + kvh) * cap;
  for (int j = j0 + threadIdx.x; j < min(j0 + PJ_KEYS, len); j += PJ_THREADS) {
    float s = a.weights_in ? a.weights_in[base + j] : 0.f;
    for (int x = 0; x < n; ++x)
      s += exp2f(a.scores[((long long)(rs.first + x / a.group) * a.hq + kvh * a.group + x % a.group) * cap + j] - lse2[x]);
    a.weights_out[base + j] = s;
  }
}

}  // namespace lsp
