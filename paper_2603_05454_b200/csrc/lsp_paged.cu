// C ABI of the paged key-value cache (see include/lsp.h for the contract).
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <initializer_list>

#include "../../include/lsp.h"
#include "paged_attention.cuh"
#include "paged_cache.cuh"

using namespace lsp;

namespace {

struct Err {
  char* buf;
  size_t len;
  int fail(int code, const char* fmt, ...) const {
    if (buf && len) {
      va_list ap;
      va_start(ap, fmt);
      vsnprintf(buf, len, fmt, ap);
      va_end(ap);
    }
    return code;
  }
};

size_t align256(size_t x) { return (x + 255) / 256 * 256; }

// What every call checks of the cache's description.
int check_view(const Err& e, const char* who, const lsp_paged_kv* kv, PagedView* pv) {
  if (!kv || !kv->k || !kv->v) return e.fail(LSP_ERR_ARG, "%s: NULL cache or pool", who);
  if (kv->dtype != 0 && kv->dtype != 1) return e.fail(LSP_ERR_ARG, "%s: dtype %d is neither 0 (fp32) nor 1 (bf16)", who, kv->dtype);
  if (kv->head_dim != 64 && kv->head_dim != 128) return e.fail(LSP_ERR_SHAPE, "%s: head_dim %d is neither 64 nor 128", who, kv->head_dim);
  if (kv->n_pages < 1 || kv->page_size < 1 || kv->max_pages < 1 || kv->n_kv_heads < 1 || kv->batch < 1)
    return e.fail(LSP_ERR_ARG, "%s: n_pages, page_size, max_pages, n_kv_heads and batch must be positive", who);
  if (kv->batch > PA_MAX_BATCH) return e.fail(LSP_ERR_SHAPE, "%s: batch %d exceeds %d", who, kv->batch, PA_MAX_BATCH);
  if (kv->n_kv_heads > 1024) return e.fail(LSP_ERR_SHAPE, "%s: n_kv_heads %d exceeds 1024", who, kv->n_kv_heads);
  if ((long long)kv->max_pages * kv->page_size > PE_MAX_CAP)
    return e.fail(LSP_ERR_SHAPE, "%s: max_pages x page_size = %lld slots exceed %d", who, (long long)kv->max_pages * kv->page_size, PE_MAX_CAP);
  if (!kv->page_table && (long long)kv->batch * kv->max_pages > kv->n_pages)
    return e.fail(LSP_ERR_ARG, "%s: without a page table the pool needs batch x max_pages pages", who);
  const int per16 = kv->dtype == 0 ? 4 : 8;
  if (kv->page_stride % per16 || kv->row_stride % per16 || kv->head_stride % per16 || ((uintptr_t)kv->k & 15) || ((uintptr_t)kv->v & 15))
    return e.fail(LSP_ERR_ARG, "%s: pools and their strides must be multiples of 16 bytes", who);
  if (kv->page_stride < 0 || kv->row_stride < kv->head_dim || kv->head_stride < (kv->n_kv_heads > 1 ? kv->head_dim : 0))
    return e.fail(LSP_ERR_ARG, "%s: strides smaller than a head", who);
  if (((uintptr_t)kv->page_table & 3) || ((uintptr_t)kv->status & 3)) return e.fail(LSP_ERR_ARG, "%s: page_table or status misaligned", who);
  *pv = PagedView{(char*)kv->k, (char*)kv->v, kv->page_table, kv->status, kv->page_stride, kv->row_stride, kv->head_stride,
                  kv->n_pages, kv->page_size, kv->max_pages, kv->batch, kv->n_kv_heads};
  return LSP_OK;
}

// A launch or attribute call that failed: the message, and no error left behind for the caller's next CUDA call.
int cuda_failed(const Err& e, const char* who, cudaError_t ce) {
  cudaGetLastError();
  return e.fail(LSP_ERR_CUDA, "%s: launch failed (%s)", who, cudaGetErrorString(ce));
}

int check_rows(const Err& e, const char* who, const lsp_paged_kv* kv, const int32_t* row_off, int max_rows, int n_rows) {
  if (max_rows < 1 || n_rows < 0) return e.fail(LSP_ERR_ARG, "%s: max_rows %d or n_rows %d", who, max_rows, n_rows);
  if (!row_off && (long long)kv->batch * max_rows != n_rows)
    return e.fail(LSP_ERR_ARG, "%s: without row offsets every sequence has max_rows = %d rows: n_rows must be %lld, not %d", who, max_rows,
                  (long long)kv->batch * max_rows, n_rows);
  return LSP_OK;
}

// int32 and float arrays (and the status word) lie on their own boundary
template <typename... P>
bool off_boundary(const P*... p) { return (((uintptr_t)p & 3) | ...); }

bool overlap(const void* a, const void* b, size_t bytes_a, size_t bytes_b) {
  return a && b && (const char*)a < (const char*)b + bytes_b && (const char*)b < (const char*)a + bytes_a;
}
struct Array { const void* p; size_t bytes; };
// An output that overlaps an input or another output (where NULL nothing does).
bool outputs_overlap(std::initializer_list<Array> outputs, std::initializer_list<Array> inputs) {
  for (const Array* o = outputs.begin(); o != outputs.end(); ++o) {
    for (const Array& i : inputs)
      if (overlap(o->p, i.p, o->bytes, i.bytes)) return true;
    for (const Array* q = outputs.begin(); q != o; ++q)
      if (overlap(o->p, q->p, o->bytes, q->bytes)) return true;
  }
  return false;
}

constexpr size_t kCounters = 4096;        // the first bytes of a workspace: arrival counters, 0 between calls
static_assert(pa_max_ctas(64) * 4 <= kCounters && pa_max_ctas(128) * 4 <= kCounters, "a counter per CTA");

struct AttnLayout { size_t part_o, part_ml, row_lse, scores, total; };
AttnLayout attn_layout(const lsp_paged_kv* kv, int n_heads, int n_rows, int with_weights) {
  AttnLayout L;
  size_t at = kCounters;
  auto take = [&](size_t bytes) { const size_t o = at; at += align256(bytes); return o; };
  L.part_o = take((size_t)2 * pa_max_ctas(kv->head_dim) * PA_ROWS * kv->head_dim * 4);
  L.part_ml = take((size_t)2 * pa_max_ctas(kv->head_dim) * PA_ROWS * 8);
  L.row_lse = take(with_weights ? (size_t)n_rows * n_heads * 4 : 0);
  L.scores = take(with_weights ? (size_t)n_rows * n_heads * kv->max_pages * kv->page_size * 4 : 0);
  L.total = at;
  return L;
}

long long evict_moves(const lsp_paged_kv* kv, int budget) {
  const long long cap = (long long)kv->max_pages * kv->page_size;
  return cap > budget ? std::min<long long>(budget, cap - budget) : 0;
}

template <typename T, int DH>
cudaError_t launch_attention(const PagedAttnArgs& a0, int tiles, cudaStream_t stream) {
  PagedAttnArgs a = a0;
  using S = PaSmem<T, DH>;
  void (*kern)(PagedAttnArgs) = nullptr;
  a.q_rows = std::min(PA_ROWS, a.max_rows * a.group);
  const bool a16 = a.pv.page % 16 == 0;
  if constexpr (sizeof(T) == 2) {
    kern = a16 ? k_paged_attn_mma<DH, true> : k_paged_attn_mma<DH, false>;
  } else {
    // (pages of other sizes: every slot's page is looked up, by the one kernel for any number of rows)
    int rows = 1;
    while (rows < a.q_rows || (!a16 && rows < PA_ROWS)) rows *= 2;
    a.q_rows = rows;
    kern = !a16 ? k_paged_attn_simt<DH, 16, false> : rows == 1 ? k_paged_attn_simt<DH, 1, true> : rows == 2 ? k_paged_attn_simt<DH, 2, true>
         : rows == 4 ? k_paged_attn_simt<DH, 4, true> : rows == 8 ? k_paged_attn_simt<DH, 8, true> : k_paged_attn_simt<DH, 16, true>;
  }
  // As many CTAs an SM as its registers hold, unless their shared memory forbids; as many rows added at a time as there is room for.
  constexpr int kStatic = 128, kSm = 228 * 1024, kCta = 227 * 1024 - kStatic, kOwn = 1024 + kStatic;
  int n_per_sm = 0, smem = 0;
  for (int want = pa_ctas_sm(DH, sizeof(T)); want >= 1 && !n_per_sm; --want)
    for (int rows = 4; rows >= 1 && !n_per_sm; rows /= 2) {
      smem = S::total(a.q_rows, rows, a.pv.batch);
      if (smem <= kCta && want * (smem + kOwn) <= kSm) {
        a.merge_rows = rows;
        n_per_sm = want;
      }
    }
  if (!n_per_sm) return cudaErrorInvalidConfiguration;
  int dev = 0, n_sm = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&n_sm, cudaDevAttrMultiProcessorCount, dev);
  // (the limit belongs to the CUDA context: set with every call, to the same value, since another thread may be between here and its launch)
  if (e == cudaSuccess) e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, kCta);
  if (e != cudaSuccess) return e;
  const long long cap = (long long)a.pv.max_pages * a.pv.page;
  a.lane_bits = tiles > 1 ? PA_LANE_BITS : 0;
  const long long units = (long long)a.pv.batch * a.pv.hkv * ((tiles + (1 << a.lane_bits) - 1) >> a.lane_bits);      // of a lane
  const long long most = ((cap + PA_CHUNK - 1) / PA_CHUNK + PA_UNIT_COST) * units;       // numbers to deal, if every sequence were full
  // At most 32 times as many runs as units: one CTA adds a unit's parts, 32 of them where the sequences are alike.  One sequence of 8000 / 30011 slots
  // of 4 KV heads: 16.0 / 27.4 us, without the bound (74 parts) 21.5 / 30.3, with 16 16.8 / 36.3.  (Beside short sequences a long one's units have more
  // parts: 8000 beside seven of 100 57, 16.3 us where it takes 14.0 alone; 30011 beside seven of 300 66, 22.6 and 23.8.)
  a.n_runs = (int)std::min({most, 32 * units, (long long)std::min(n_per_sm * n_sm, pa_max_ctas(DH)) >> a.lane_bits});
  e = launch_k(1, kern, dim3(a.n_runs << a.lane_bits), dim3(PA_THREADS), (size_t)smem, stream, a);
  if (e != cudaSuccess || !a.scores) return e;
  // a slot a thread, and four where that still leaves four blocks an SM
  const long long heads = (long long)a.pv.batch * a.pv.hkv;
  const int kpt = heads * ((cap + 4 * PW_THREADS - 1) / (4 * PW_THREADS)) >= 4 * n_sm ? 4 : 1;
  const int key_blocks = (int)((cap + kpt * PW_THREADS - 1) / (kpt * PW_THREADS));
  return launch_k(1, kpt == 4 ? k_paged_weights<4> : k_paged_weights<1>, dim3((unsigned)(heads * key_blocks)), dim3(PW_THREADS), (size_t)a.max_rows * a.group * 4,
                  stream, a, key_blocks);
}

// Where there are more units than SMs, of at most 4096 slots: a CTA of 256 threads each (four fit an SM up to some 3200 slots, three beyond), which
// moves what it selected.  Else CTAs of 1024 threads, a cluster of them per unit while that fills no more than the SMs and leaves each CTA 3000
// slots (or where a CTA cannot hold them), and the moves over the whole grid.  `cap`, the table's width, stands for the slots, which only the device
// knows: a table far wider than its sequences costs time (512 units of about 1030 slots to 1024: tables for 1088 / 4096 slots 9.7 / 9.0 us, 4160 /
// 8192 22.1, 32768 92).  Measured with tables as wide as the sequences, us: 512 units of about 1030 / up to 2047 slots moved by their CTAs 12.4 /
// 44.8, over the grid 14.2 / 46.8 (of 2047 each to 1024 64.4 and 64.3); 16 units of up to 4093 slots without a cluster 12.6, with two CTAs
// 13.3; 4 units of 30000 slots with eight CTAs 19.1, four 24.0, two 29.4.
cudaError_t launch_evict(PagedEvictArgs& a, int units, int cap, int n_sm, cudaStream_t stream) {
  const bool small = units > n_sm && cap <= 4096;
  a.cluster = 1;
  while (!small && a.cluster < PE_CLUSTER && (cap > PE_KEYS * a.cluster || (2 * a.cluster * units <= n_sm && cap / (2 * a.cluster) >= 3000))) a.cluster *= 2;
  a.slots = ((cap + 31) / 32 + a.cluster - 1) / a.cluster * 32;
  a.in_smem = a.slots <= PE_KEYS ? 1 : 0;
  const size_t smem = (size_t)pe_words(a.slots, a.in_smem) * 4;
  void (*kern)(PagedEvictArgs) = small ? k_paged_select<256, true> : k_paged_select<1024, false>;
  cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, 224 * 1024);      // (see launch_attention)
  if (e == cudaSuccess) e = launch_k(1, kern, dim3(units * a.cluster), dim3(small ? 256 : 1024), smem, stream, a.cluster, a);
  if (e != cudaSuccess || small || a.max_moves == 0) return e;
  // As many blocks as are resident at once (four an SM), whose warps take pairs in turn; six an SM where that leaves each four turns, since units
  // differ: 32 units of 30000 slots to 4096 43.6 us with four, 40.1 with six; 4 units of 65521 to 8192 22.4 and 23.2.
  const int most = (a.max_moves + PM_WARPS * PM_PAIRS - 1) / (PM_WARPS * PM_PAIRS);
  const int blocks = ((long long)most * units >= 4 * 6 * n_sm ? 6 : 4) * n_sm, fill = (blocks + units - 1) / units;
  return launch_k(1, k_paged_move, dim3(units, std::min(most, fill)), dim3(PM_WARPS * 32), 0, stream, a);
}

}  // namespace

extern "C" {

int lsp_paged_append(const lsp_paged_kv* kv, const void* k_new, const void* v_new, long long ld_new, const int32_t* lens, const int32_t* row_off,
                     int max_rows, int n_rows, int32_t* lens_out, float* weights, int32_t* pos, const int32_t* seen, int32_t* seen_out,
                     void* cuda_stream, char* err, size_t err_len) {
  const Err e{err, err_len};
  const char* who = "lsp_paged_append";
  PagedAppendArgs a;
  int rc = check_view(e, who, kv, &a.pv);
  if (rc) return rc;
  rc = check_rows(e, who, kv, row_off, max_rows, n_rows);
  if (rc) return rc;
  if (!lens || !lens_out || (n_rows > 0 && (!k_new || !v_new))) return e.fail(LSP_ERR_ARG, "%s: NULL pointer", who);
  if (off_boundary(lens, row_off, lens_out, weights, pos, seen, seen_out)) return e.fail(LSP_ERR_ARG, "%s: misaligned array", who);
  if ((seen_out != nullptr) != (seen != nullptr)) return e.fail(LSP_ERR_ARG, "%s: seen and seen_out come together", who);
  const size_t nb = (size_t)kv->batch * 4, nt = nb * kv->max_pages;
  if (outputs_overlap({{lens_out, nb}, {seen_out, nb}}, {{lens, nb}, {seen, nb}, {row_off, nb + 4}, {kv->page_table, nt}}))
    return e.fail(LSP_ERR_ARG, "%s: lens_out and seen_out must not overlap what the call reads, nor one another", who);
  a.esz = kv->dtype == 0 ? 4 : 2;
  if ((ld_new * a.esz) % 16 || ((uintptr_t)k_new & 15) || ((uintptr_t)v_new & 15) || ld_new < (long long)kv->n_kv_heads * kv->head_dim)
    return e.fail(LSP_ERR_ARG, "%s: new rows must be 16-byte aligned and at least n_kv_heads x head_dim elements apart", who);
  a.k_new = (const char*)k_new;
  a.v_new = (const char*)v_new;
  a.ld_new = ld_new * a.esz;
  a.lens = lens;
  a.row_off = row_off;
  a.seen = seen;
  a.max_rows = max_rows;
  a.n_rows = n_rows;
  a.head_bytes = kv->head_dim * a.esz;
  a.lens_out = lens_out;
  a.seen_out = seen_out;
  a.weights = weights;
  a.pos = pos;
  // rows of a block: what its threads hold, as long as that leaves four blocks an SM
  const int row_bytes = 2 * kv->n_kv_heads * a.head_bytes;
  int dev = 0, n_sm = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&n_sm, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
    return e.fail(LSP_ERR_CUDA, "%s: no usable current device", who);
  a.rows_block = std::max(1, std::min({PP_ROWS, PP_THREADS * PP_VEC * 16 / row_bytes, n_rows / (4 * n_sm)}));
  const cudaError_t ce = launch_k(1, k_paged_append, dim3((n_rows + a.rows_block - 1) / a.rows_block + 1), dim3(PP_THREADS), row_off ? (size_t)kv->batch * 8 : 0,
                                  (cudaStream_t)cuda_stream, a);
  if (ce != cudaSuccess) return cuda_failed(e, who, ce);
  return LSP_OK;
}

size_t lsp_paged_attention_workspace(const lsp_paged_kv* kv, int n_heads, int n_rows, int with_weights) {
  PagedView pv;
  if (check_view(Err{nullptr, 0}, "", kv, &pv) != LSP_OK || n_heads < 1 || n_rows < 0) return 0;
  return attn_layout(kv, n_heads, n_rows, with_weights).total;
}

int lsp_paged_attention(const lsp_paged_kv* kv, const void* q, long long ldq, int n_heads, const int32_t* lens, const int32_t* row_off,
                        int max_rows, int n_rows, float scale, void* out, long long ldo, float* lse, const float* weights_in,
                        float* weights_out, void* workspace, size_t workspace_bytes, void* cuda_stream, char* err, size_t err_len) {
  const Err e{err, err_len};
  const char* who = "lsp_paged_attention";
  PagedAttnArgs a;
  int rc = check_view(e, who, kv, &a.pv);
  if (rc) return rc;
  rc = check_rows(e, who, kv, row_off, max_rows, n_rows);
  if (rc) return rc;
  if (!lens || !workspace || (n_rows > 0 && (!q || !out))) return e.fail(LSP_ERR_ARG, "%s: NULL pointer", who);
  if (off_boundary(lens, row_off, lse, weights_in, weights_out)) return e.fail(LSP_ERR_ARG, "%s: misaligned array", who);
  if (n_heads < 1 || n_heads % kv->n_kv_heads) return e.fail(LSP_ERR_SHAPE, "%s: %d query heads over %d KV heads", who, n_heads, kv->n_kv_heads);
  if (!(scale > 0.f) || std::isinf(scale)) return e.fail(LSP_ERR_ARG, "%s: scale must be positive and finite", who);
  if (weights_in && !weights_out) return e.fail(LSP_ERR_ARG, "%s: weights_in without weights_out", who);
  const size_t nw = (size_t)kv->batch * kv->n_kv_heads * kv->max_pages * kv->page_size * 4;
  if (weights_in != weights_out && overlap(weights_in, weights_out, nw, nw))
    return e.fail(LSP_ERR_ARG, "%s: weights_in and weights_out must be the same array or not overlap", who);
  const int esz = kv->dtype == 0 ? 4 : 2;
  const long long qd = (long long)n_heads * kv->head_dim;
  if ((ldq * esz) % 16 || (ldo * esz) % 16 || ((uintptr_t)q & 15) || ((uintptr_t)out & 15) || ldq < qd || ldo < qd)
    return e.fail(LSP_ERR_ARG, "%s: rows of q and out must be 16-byte aligned and at least n_heads x head_dim elements apart", who);
  if ((uintptr_t)workspace & 255) return e.fail(LSP_ERR_ARG, "%s: the workspace must be 256-byte aligned", who);
  const AttnLayout L = attn_layout(kv, n_heads, n_rows, weights_out != nullptr);
  if (workspace_bytes < L.total) return e.fail(LSP_ERR_WORKSPACE, "%s: workspace of %zu bytes, %zu needed", who, workspace_bytes, L.total);
  a.group = n_heads / kv->n_kv_heads;
  const long long rows_unit = (long long)max_rows * a.group, tiles = (rows_unit + PA_ROWS - 1) / PA_ROWS;
  const long long cap = (long long)kv->max_pages * kv->page_size, units = tiles * kv->batch * kv->n_kv_heads;
  if ((long long)kv->batch * kv->n_kv_heads * (cap / PW_THREADS + 1) > 0x7fffffffll || units * (cap / PA_CHUNK + 1 + PA_UNIT_COST) > 0x7fffffffll ||
      (long long)max_rows * n_heads > 0x3fffffffll || max_rows > (1 << 20) || tiles * kv->n_kv_heads > (1 << 20))
    return e.fail(LSP_ERR_SHAPE, "%s: batch x heads x rows x slots too large for one call", who);
  if (weights_out && rows_unit > 8192) return e.fail(LSP_ERR_SHAPE, "%s: weights of more than 8192 (row, head) pairs per KV head", who);
  if (n_rows == 0 && !weights_out) return LSP_OK;
  char* ws = (char*)workspace;
  a.q = q;
  a.out = out;
  a.ldq = ldq;
  a.ldo = ldo;
  a.lens = lens;
  a.row_off = row_off;
  a.hq = n_heads;
  a.max_rows = max_rows;
  a.n_rows = n_rows;
  a.n_runs = 0;
  a.scale_log2 = scale * 1.4426950408889634f;
  a.lse = lse;
  a.part_o = (float*)(ws + L.part_o);
  a.part_ml = (float2*)(ws + L.part_ml);
  a.arrived = (unsigned*)ws;
  a.row_lse = (float*)(ws + L.row_lse);
  a.scores = weights_out ? (float*)(ws + L.scores) : nullptr;
  a.weights_in = weights_in;
  a.weights_out = weights_out;
  const cudaStream_t st = (cudaStream_t)cuda_stream;
  cudaError_t ce;
  if (kv->dtype == 1)
    ce = kv->head_dim == 128 ? launch_attention<bf16, 128>(a, (int)tiles, st) : launch_attention<bf16, 64>(a, (int)tiles, st);
  else
    ce = kv->head_dim == 128 ? launch_attention<float, 128>(a, (int)tiles, st) : launch_attention<float, 64>(a, (int)tiles, st);
  if (ce != cudaSuccess) return cuda_failed(e, who, ce);
  return LSP_OK;
}

size_t lsp_paged_evict_workspace(const lsp_paged_kv* kv, int budget) {
  PagedView pv;
  if (check_view(Err{nullptr, 0}, "", kv, &pv) != LSP_OK || budget < 1) return 0;
  return kCounters + align256((size_t)kv->batch * kv->n_kv_heads * (1 + 2 * (size_t)evict_moves(kv, budget)) * 4);
}

int lsp_paged_evict(const lsp_paged_kv* kv, const float* weights, const int32_t* pos, const int32_t* lens, const int32_t* seen, int budget,
                    int n_sink, int n_recent, float* weights_out, int32_t* pos_out, int32_t* lens_out, void* workspace,
                    size_t workspace_bytes, void* cuda_stream, char* err, size_t err_len) {
  const Err e{err, err_len};
  const char* who = "lsp_paged_evict";
  PagedEvictArgs a;
  int rc = check_view(e, who, kv, &a.pv);
  if (rc) return rc;
  if (!weights || !lens || !weights_out || !lens_out || !workspace) return e.fail(LSP_ERR_ARG, "%s: NULL pointer", who);
  if (off_boundary(weights, pos, lens, seen, weights_out, pos_out, lens_out)) return e.fail(LSP_ERR_ARG, "%s: misaligned array", who);
  if (pos && !pos_out) return e.fail(LSP_ERR_ARG, "%s: pos without pos_out", who);
  if (budget < 1 || n_sink < 0 || n_recent < 0 || (long long)n_sink + n_recent > budget)
    return e.fail(LSP_ERR_ARG, "%s: budget %d must be positive and hold n_sink %d + n_recent %d", who, budget, n_sink, n_recent);
  const long long cap = (long long)kv->max_pages * kv->page_size;
  const size_t nb = (size_t)kv->batch * 4, nw = nb * kv->n_kv_heads * cap, nt = nb * kv->max_pages;
  if (outputs_overlap({{weights_out, nw}, {pos_out, nw}, {lens_out, nb}}, {{weights, nw}, {pos, nw}, {lens, nb}, {seen, nb}, {kv->page_table, nt}}))
    return e.fail(LSP_ERR_ARG, "%s: outputs must not overlap what the call reads, nor one another", who);
  if ((uintptr_t)workspace & 255) return e.fail(LSP_ERR_ARG, "%s: the workspace must be 256-byte aligned", who);
  const size_t need = lsp_paged_evict_workspace(kv, budget);
  if (workspace_bytes < need) return e.fail(LSP_ERR_WORKSPACE, "%s: workspace of %zu bytes, %zu needed", who, workspace_bytes, need);
  a.weights = weights;
  a.pos = pos;
  a.lens = lens;
  a.seen = seen;
  a.budget = budget;
  a.n_sink = n_sink;
  a.n_recent = n_recent;
  a.max_moves = (int)evict_moves(kv, budget);
  a.weights_out = weights_out;
  a.pos_out = pos_out;
  a.lens_out = lens_out;
  a.moves = (int*)((char*)workspace + kCounters);
  a.esz = kv->dtype == 0 ? 4 : 2;
  a.head_bytes = kv->head_dim * a.esz;
  const cudaStream_t st = (cudaStream_t)cuda_stream;
  const int units = kv->batch * kv->n_kv_heads;
  int dev = 0, n_sm = 0;
  cudaError_t ce = cudaGetDevice(&dev);
  if (ce == cudaSuccess) ce = cudaDeviceGetAttribute(&n_sm, cudaDevAttrMultiProcessorCount, dev);
  if (ce == cudaSuccess) ce = launch_evict(a, units, (int)cap, n_sm, st);
  if (ce != cudaSuccess) return cuda_failed(e, who, ce);
  return LSP_OK;
}

}  // extern "C"
