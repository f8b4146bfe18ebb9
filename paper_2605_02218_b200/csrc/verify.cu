// Host part of the verification operators: argument checks and launches of the paged cache, the attention over it and the edits
// of logits (include/covspec.h).
#include "covspec.h"

#include <limits.h>

#include <algorithm>
#include <atomic>

#include "attend_call.cuh"
#include "host.cuh"
#include "logits_kernels.cuh"

using namespace covspec;

namespace {

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
int bytes_of(int dtype) { return dtype == COVSPEC_F32 ? 4 : dtype == COVSPEC_BF16 || dtype == COVSPEC_F16 ? 2 : 1; }
bool is_dtype(int dtype) { return dtype == COVSPEC_F32 || dtype == COVSPEC_BF16 || dtype == COVSPEC_F16; }

int check_cache(const covspec_cache* c) {
  if (!c || !c->k || !c->v) return COVSPEC_ERR_ARG;
  if (c->store < COVSPEC_F32 || c->store > COVSPEC_INT8) return COVSPEC_ERR_ARG;
  if (c->store >= COVSPEC_E4M3 && (!c->k_scale || !c->v_scale || !aligned16(c->k_scale) || !aligned16(c->v_scale))) return COVSPEC_ERR_ARG;
  if (c->head_dim != 64 && c->head_dim != 128) return COVSPEC_ERR_UNSUPPORTED;
  if (c->page_size < 8 || c->page_size > 4096 || (c->page_size & (c->page_size - 1))) return COVSPEC_ERR_UNSUPPORTED;
  if (c->pages < 1 || c->heads < 1 || (long long)c->heads * c->page_size * c->head_dim > INT_MAX) return COVSPEC_ERR_SHAPE;
  const long long least = (long long)c->heads * c->page_size * c->head_dim;
  if (c->k_page_stride < least || c->v_page_stride < least) return COVSPEC_ERR_SHAPE;
  const int e = bytes_of(c->store);
  // the kernels count rows of a cache in 16 bytes
  if (std::max(c->k_page_stride, c->v_page_stride) > (1ll << 36) / e / c->pages) return COVSPEC_ERR_UNSUPPORTED;
  if (c->k_page_stride * e % 16 || c->v_page_stride * e % 16 || !aligned16(c->k) || !aligned16(c->v)) return COVSPEC_ERR_ARG;
  return COVSPEC_OK;
}
int check_tokens(const covspec_tokens* t) {
  if (!t || !t->offsets || !t->lengths || !t->table) return COVSPEC_ERR_ARG;
  if (t->batch < 1 || t->table_width < 1 || t->table_stride < t->table_width) return COVSPEC_ERR_SHAPE;
  return COVSPEC_OK;
}
cache::Pages pages_of(const covspec_cache* c) {
  cache::Pages p{};
  p.k = c->k; p.v = c->v; p.k_scale = c->k_scale; p.v_scale = c->v_scale;
  p.k_page = c->k_page_stride; p.v_page = c->v_page_stride;
  p.pages = c->pages; p.heads = c->heads;
  while ((1 << p.page_shift) < c->page_size) ++p.page_shift;
  return p;
}
cache::Tokens tokens_of(const covspec_tokens* t) {
  return cache::Tokens{t->batch, t->offsets, t->lengths, t->table, t->table_stride, t->table_width};
}

// Calls f with a null pointer of the type and the constants that the arguments name.
template <typename F>
cudaError_t with_type(int dtype, F f) {
  return dtype == COVSPEC_F32 ? f((float*)nullptr) : dtype == COVSPEC_BF16 ? f((__nv_bfloat16*)nullptr) : f((__half*)nullptr);
}
template <int V> using Const = std::integral_constant<int, V>;
template <typename F>
cudaError_t with_store(int store, F f) {
  switch (store) {
    case COVSPEC_F32: return f(Const<cache::kF32>());
    case COVSPEC_BF16: return f(Const<cache::kBF16>());
    case COVSPEC_F16: return f(Const<cache::kF16>());
    case COVSPEC_E4M3: return f(Const<cache::kE4M3>());
    default: return f(Const<cache::kInt8>());
  }
}
template <typename F>
cudaError_t with_dim(int dim, F f) { return dim == 64 ? f(Const<64>()) : f(Const<128>()); }

int sm_count(int* sms) {
  int dev = 0;
  CUDA_TRY(cudaGetDevice(&dev));
  CUDA_TRY(cudaDeviceGetAttribute(sms, cudaDevAttrMultiProcessorCount, dev));
  return COVSPEC_OK;
}

// CTAs of the cache kernels for `rows` (token, head) rows of `lanes` lanes each, `passes` times a warp's.
int cache_grid(int rows, int lanes, int passes) {
  const int per = (32 / lanes) * passes * (cache::kThreads / 32);
  return (int)(((long long)rows + per - 1) / per);
}

long long part_bytes(int ctas, int rows, int dim) { return 2ll * ctas * rows * (dim + 2) * 4; }

int cache_attend(const covspec_cache* cache, const covspec_tokens* tokens, int dtype, int n, const void* q, long long q_stride,
                 int q_heads, float scale, int window, int max_new, void* out, long long out_stride, float* lse, void* workspace,
                 long long workspace_bytes, uint32_t polls, int stop_share, int stop_unit, void* stream) {
  int st = check_cache(cache);
  if (st == COVSPEC_OK) st = check_tokens(tokens);
  if (st != COVSPEC_OK) return st;
  if (dtype != COVSPEC_BF16 && dtype != COVSPEC_F16) return COVSPEC_ERR_UNSUPPORTED;
  if (cache->store != dtype && cache->store < COVSPEC_E4M3) return COVSPEC_ERR_UNSUPPORTED;
  if (n < 0 || q_heads < 1 || q_heads % cache->heads || (long long)n * q_heads > INT_MAX / 2) return COVSPEC_ERR_SHAPE;
  if (window < 0 || max_new < 0 || !(scale == scale)) return COVSPEC_ERR_ARG;
  if (n == 0) return COVSPEC_OK;
  const long long width = (long long)q_heads * cache->head_dim;
  if (!q || !out || !workspace || !aligned16(q) || !aligned16(out) || !aligned16(workspace)) return COVSPEC_ERR_ARG;
  if (q_stride < width || out_stride < width) return COVSPEC_ERR_SHAPE;
  if (q_stride % 8 || out_stride % 8) return COVSPEC_ERR_ARG;
  const long long need = covspec_cache_attend_workspace(cache, q_heads);
  if (need < 0) return (int)need;
  if (workspace_bytes < need) return COVSPEC_ERR_WORKSPACE;
  int sms = 0;
  if (const int e = sm_count(&sms)) return e;

  attend::Params prm{};
  prm.c = pages_of(cache);
  prm.t = tokens_of(tokens);
  prm.q = q; prm.out = out; prm.lse = lse;
  prm.q_ld = q_stride; prm.out_ld = out_stride;
  prm.n = n; prm.q_heads = q_heads; prm.group = q_heads / cache->heads;
  prm.window = std::min(window, 1 << 30);
  prm.scale_log2 = scale * 1.4426950408889634f;
  prm.rows_over = 0; prm.rows_upto = INT_MAX;
  prm.least_units = 1;
  prm.polls = polls; prm.stop_share = stop_share; prm.stop_unit = stop_unit;
  prm.open = static_cast<int4*>(workspace);
  prm.part = reinterpret_cast<float*>(prm.open + 2ll * (attend::kRowsCtas + 1) * sms);
  // rows of a key head in the largest request.  Where some may have many, each of the two kernels takes its requests
  const long long most = (long long)(max_new > 0 ? std::min(max_new, n) : n) * prm.group;
  const int rows = most <= 16 ? 16 : most <= 32 ? 32 : 64;
  const bool both = most > attend::kFewRows && cache->store < COVSPEC_E4M3;
  // no more CTAs than there can be units
  auto ctas_of = [&](int rows, int keys, int ctas) {
    const long long items = ((long long)n * prm.group / rows + prm.t.batch) * cache->heads;
    return (int)std::min<long long>(ctas, items * (((long long)prm.t.width * cache->page_size + keys - 1) / keys + 1));
  };
  const int ctas = ctas_of(rows, 64, attend::kRowsCtas * sms);
  attend::Params wide = prm;
  wide.rows_over = attend::kFewRows;
  wide.open = prm.open + 2ll * attend::kRowsCtas * sms;
  wide.part = prm.part + part_bytes(attend::kRowsCtas * sms, attend::kFewRows, cache->head_dim) / 4;
  const int wide_ctas = ctas_of(attend::kWideRows, attend::kWideKeys, sms);
  if (both) prm.rows_upto = attend::kFewRows;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  const attend::Call call{prm, wide, cache, rows, ctas, both ? wide_ctas : 0, s};
  return status_of("attention", [&] { return dtype == COVSPEC_BF16 ? attend::launch_bf16(call) : attend::launch_f16(call); });
}

}  // namespace

extern "C" {

int covspec_cache_write(const covspec_cache* cache, const covspec_tokens* tokens, int dtype, int n, const void* k, const void* v,
                        long long k_stride, long long v_stride, const int* rows, const int* row_offsets, int source_rows,
                        void* stream) {
  int st = check_cache(cache);
  if (st == COVSPEC_OK) st = check_tokens(tokens);
  if (st != COVSPEC_OK) return st;
  if (!is_dtype(dtype) || (rows && !row_offsets)) return COVSPEC_ERR_ARG;
  if (n < 0 || source_rows < 0 || (!rows && source_rows < n)) return COVSPEC_ERR_SHAPE;
  if (n == 0) return COVSPEC_OK;
  const long long width = (long long)cache->heads * cache->head_dim;
  if (!k || !v || !aligned16(k) || !aligned16(v)) return COVSPEC_ERR_ARG;
  if (k_stride < width || v_stride < width) return COVSPEC_ERR_SHAPE;
  if (k_stride * bytes_of(dtype) % 16 || v_stride * bytes_of(dtype) % 16) return COVSPEC_ERR_ARG;
  if ((long long)n * cache->heads > INT_MAX / 2) return COVSPEC_ERR_SHAPE;
  // few rows: one look-up and one row a lane group, for the latency (256 tokens x 8 heads 9.8 -> 4.6 us); many: the look-ups
  // of four at a time (27.8 k tokens x 8 heads 84 -> 63 us)
  int sms = 0;
  if (const int e = sm_count(&sms)) return e;
  const int one = cache_grid(n * cache->heads, cache->head_dim / 8, 1), passes = one <= 8 * sms ? 1 : cache::kPasses;
  const int grid = passes == 1 ? one : cache_grid(n * cache->heads, cache->head_dim / 8, passes);
  cache::WriteParams prm{pages_of(cache), tokens_of(tokens), k, v, k_stride, v_stride, n, rows, row_offsets, source_rows, passes};
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  CUDA_TRY(with_type(dtype, [&](auto* tag) {
    using T = std::remove_pointer_t<decltype(tag)>;
    return with_store(cache->store, [&](auto store) {
      return with_dim(cache->head_dim, [&](auto dim) {
        return launch_dependent(cache::write_kernel<T, decltype(store)::value, decltype(dim)::value>, dim3((unsigned)grid), cache::kThreads, 0, s, prm);
      });
    });
  }));
  return COVSPEC_OK;
}

int covspec_cache_read(const covspec_cache* cache, const covspec_tokens* tokens, int dtype, int n, void* k, void* v, void* stream) {
  int st = check_cache(cache);
  if (st == COVSPEC_OK) st = check_tokens(tokens);
  if (st != COVSPEC_OK) return st;
  if (!is_dtype(dtype)) return COVSPEC_ERR_ARG;
  if (n < 0) return COVSPEC_ERR_SHAPE;
  if (n == 0) return COVSPEC_OK;
  if (!k || !v || !aligned16(k) || !aligned16(v)) return COVSPEC_ERR_ARG;
  if ((long long)n * cache->heads > INT_MAX / 2) return COVSPEC_ERR_SHAPE;
  const int grid = cache_grid(n * cache->heads, cache->head_dim * bytes_of(cache->store) / 16, cache::kPasses);
  cache::ReadParams prm{pages_of(cache), tokens_of(tokens), k, v, n};
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  CUDA_TRY(with_type(dtype, [&](auto* tag) {
    using T = std::remove_pointer_t<decltype(tag)>;
    return with_store(cache->store, [&](auto store) {
      return with_dim(cache->head_dim, [&](auto dim) {
        return launch_dependent(cache::read_kernel<T, decltype(store)::value, decltype(dim)::value>, dim3((unsigned)grid), cache::kThreads, 0, s, prm);
      });
    });
  }));
  return COVSPEC_OK;
}

long long covspec_cache_attend_workspace(const covspec_cache* cache, int q_heads) {
  const int st = check_cache(cache);
  if (st != COVSPEC_OK) return st;
  if (q_heads < 1 || q_heads % cache->heads) return COVSPEC_ERR_SHAPE;
  int sms = 0;
  if (const int e = sm_count(&sms)) return e;
  return part_bytes(attend::kRowsCtas * sms, attend::kFewRows, cache->head_dim) + part_bytes(sms, attend::kWideRows, cache->head_dim) +
         32ll * (attend::kRowsCtas + 1) * sms;
}

int covspec_cache_attend(const covspec_cache* cache, const covspec_tokens* tokens, int dtype, int n, const void* q,
                         long long q_stride, int q_heads, float scale, int window, int max_new, void* out, long long out_stride,
                         float* lse, void* workspace, long long workspace_bytes, void* stream) {
  return cache_attend(cache, tokens, dtype, n, q, q_stride, q_heads, scale, window, max_new, out, out_stride, lse, workspace,
                      workspace_bytes, attend::kPolls, -1, 0, stream);
}

int covspec_selftest_attend_timeout(const covspec_cache* cache, const covspec_tokens* tokens, int dtype, int n, const void* q,
                                    long long q_stride, int q_heads, float scale, int window, int max_new, void* out,
                                    long long out_stride, float* lse, void* workspace, long long workspace_bytes, int block, int unit,
                                    void* stream) {
  return cache_attend(cache, tokens, dtype, n, q, q_stride, q_heads, scale, window, max_new, out, out_stride, lse, workspace,
                      workspace_bytes, block < 0 ? 0u : attend::kPolls / 16, std::max(block, -1), unit, stream);
}

int covspec_edit_logits(int logit_dtype, int rows, int vocab, long long ld, const void* z, void* out, const covspec_edits* edits,
                        void* stream) {
  if (!edits || !edits->row_offsets || !is_dtype(logit_dtype)) return COVSPEC_ERR_ARG;
  const covspec_edits& e = *edits;
  if ((e.history && !e.history_offsets) || (e.bias_ids && (!e.bias_values || !e.bias_offsets))) return COVSPEC_ERR_ARG;
  if (rows < 0 || vocab < 1 || ld < vocab || ld * bytes_of(logit_dtype) % 16 || e.batch < 1 || e.history_len < 0 || e.bias_len < 0 ||
      (e.mask && e.mask_stride < (vocab + 7) / 8))
    return COVSPEC_ERR_SHAPE;
  if (rows == 0) return COVSPEC_OK;
  if (!z || !out || !aligned16(z) || !aligned16(out)) return COVSPEC_ERR_ARG;
  edit::Params prm{};
  prm.z = z; prm.out = out; prm.ld = ld; prm.rows = rows; prm.vocab = vocab; prm.batch = e.batch;
  prm.row_offsets = e.row_offsets;
  prm.history = e.history; prm.history_offsets = e.history_offsets; prm.history_len = e.history_len;
  prm.prompt = e.prompt_lengths; prm.drafted = e.drafted;
  prm.repetition = e.repetition; prm.presence = e.presence; prm.frequency = e.frequency;
  prm.bias_ids = e.bias_ids; prm.bias = e.bias_values; prm.bias_offsets = e.bias_offsets; prm.bias_len = e.bias_len;
  prm.mask = static_cast<const unsigned char*>(e.mask); prm.mask_ld = e.mask_stride;
  int sms = 0;
  if (const int st = sm_count(&sms)) return st;
  // Rows of a CTA share the tables of their request, which cost a pass over the history; segments of 4096 entries and groups of
  // rows (of one block mostly) as long as four CTAs an SM are left, smaller segments where there are not two (1024 rows x 151674,
  // groups of 16 / 8 / 4: 188 / 172 / 203 us).
  prm.segment = 4096;
  prm.group = 1;
  auto segments_of = [&] { return (unsigned)((vocab + prm.segment - 1) / prm.segment); };
  while (prm.group < 8 && prm.group < rows && (long long)segments_of() * ((rows + 2 * prm.group - 1) / (2 * prm.group)) >= 4ll * sms) prm.group *= 2;
  while (prm.segment > 2048 && (long long)segments_of() * rows < 2ll * sms) prm.segment /= 2;
  while ((rows + prm.group - 1) / prm.group > 65535) prm.group *= 2;
  const unsigned segments = segments_of();
  const int groups = (rows + prm.group - 1) / prm.group;
  const int smem = prm.segment / 8 + prm.segment * (e.bias_ids ? 8 : 4);
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  CUDA_TRY(with_type(logit_dtype, [&](auto* tag) {
    using T = std::remove_pointer_t<decltype(tag)>;
    const cudaError_t err = allow_shared<edit::edit_kernel<T>>(4096 / 8 + 4096 * 8);
    if (err != cudaSuccess) return err;
    return launch_dependent(edit::edit_kernel<T>, dim3(segments, (unsigned)groups), edit::kThreads, (size_t)smem, s, prm);
  }));
  return COVSPEC_OK;
}

}  // extern "C"
