// Launches of the attention kernels for one type of queries.
#pragma once
#include <algorithm>

#include "attend_call.cuh"
#include "attend_kernels.cuh"
#include "attend_tc.cuh"
#include "host.cuh"

namespace covspec {
namespace attend {
namespace {

// The keys or the values of a cache as [pages, heads * page_size, dim]: boxes of a page's rows of one head, at most `keys`, 128 bytes
// wide (64 where a row has no more), in tiles with the swizzle of that width.
bool make_page_map(CUtensorMap* map, const covspec_cache* c, const void* base, long long page_stride, int keys) {
  EncodeTiledFn encode = encode_tiled_fn();
  if (!encode) {
    g_cuda_error = "cuTensorMapEncodeTiled is not available";
    return false;
  }
  const int e = c->store >= COVSPEC_E4M3 ? 1 : 2;
  const cuuint64_t dims[3] = {(cuuint64_t)c->head_dim, (cuuint64_t)c->heads * c->page_size, (cuuint64_t)c->pages};
  const cuuint64_t strides[2] = {(cuuint64_t)c->head_dim * e, (cuuint64_t)page_stride * e};
  const cuuint32_t width = (cuuint32_t)std::min(c->head_dim * e, 128);
  const cuuint32_t box[3] = {width / e, (cuuint32_t)std::min(c->page_size, keys), 1}, step[3] = {1, 1, 1};
  const CUresult r = encode(map, e == 1 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_UINT16, 3,
                            const_cast<void*>(base), dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
                            width == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B,
                            CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  if (r != CUDA_SUCCESS) g_cuda_error = "cuTensorMapEncodeTiled failed with code " + std::to_string((int)r);
  return r == CUDA_SUCCESS;
}

template <typename T, int STORE, int DIM, int ROWS>
cudaError_t launch_rows(const Params& prm, const covspec_cache* cache, int ctas, cudaStream_t s) {
  constexpr auto kernel = attend_kernel<T, STORE, DIM, ROWS>;
  using L = Layout<STORE, DIM, ROWS>;
  cudaError_t e = allow_shared<kernel>(L::kSmem);
  if (e != cudaSuccess) return e;
  CUtensorMap map_k, map_v;
  if (!make_page_map(&map_k, cache, cache->k, cache->k_page_stride, L::kKeys) || !make_page_map(&map_v, cache, cache->v, cache->v_page_stride, L::kKeys))
    return cudaErrorInvalidValue;
  e = launch_dependent(kernel, dim3((unsigned)ctas), kThreads, L::kSmem, s, map_k, map_v, prm);
  if (e != cudaSuccess) return e;
  return launch_dependent(attend_join_kernel<T, ROWS, L::kKeys, kOpen, DIM>, dim3((unsigned)ctas, ROWS / 4), 128, 0, s, prm);
}

template <typename T, int STORE, int DIM>
cudaError_t launch_wide(const Params& prm, const covspec_cache* cache, int ctas, cudaStream_t s) {
  constexpr auto kernel = wide::attend_wide_kernel<T, STORE, DIM>;
  constexpr int smem = wide::Layout<STORE, DIM>::kSmem;
  cudaError_t e = allow_shared<kernel>(smem);
  if (e != cudaSuccess) return e;
  CUtensorMap map_k{}, map_v{};
  if (!make_page_map(&map_k, cache, cache->k, cache->k_page_stride, kWideKeys) || !make_page_map(&map_v, cache, cache->v, cache->v_page_stride, kWideKeys))
    return cudaErrorInvalidValue;
  e = launch_dependent(kernel, dim3((unsigned)ctas), wide::kThreads, smem, s, map_k, map_v, prm);
  if (e != cudaSuccess) return e;
  return launch_dependent(attend_join_kernel<T, kWideRows, kWideKeys, wide::kOpen, DIM>, dim3((unsigned)ctas, kWideRows / 4), 128, 0, s, prm);
}

template <typename T, int STORE, int DIM>
cudaError_t launch_store(const Call& c) {
  if constexpr (STORE < cache::kE4M3) {
    if (c.many_ctas)
      if (const cudaError_t e = launch_wide<T, STORE, DIM>(c.many, c.cache, c.many_ctas, c.stream); e != cudaSuccess) return e;
  }
  return c.rows == 16 ? launch_rows<T, STORE, DIM, 16>(c.few, c.cache, c.ctas, c.stream)
         : c.rows == 32 ? launch_rows<T, STORE, DIM, 32>(c.few, c.cache, c.ctas, c.stream)
                        : launch_rows<T, STORE, DIM, 64>(c.few, c.cache, c.ctas, c.stream);
}
template <typename T, int DIM>
cudaError_t launch_dim(const Call& c) {
  constexpr int kOwn = __is_same(T, __half) ? cache::kF16 : cache::kBF16;
  return c.cache->store == COVSPEC_E4M3 ? launch_store<T, cache::kE4M3, DIM>(c)
         : c.cache->store == COVSPEC_INT8 ? launch_store<T, cache::kInt8, DIM>(c) : launch_store<T, kOwn, DIM>(c);
}
template <typename T>
cudaError_t launch(const Call& c) { return c.cache->head_dim == 64 ? launch_dim<T, 64>(c) : launch_dim<T, 128>(c); }

}  // namespace
}  // namespace attend
}  // namespace covspec
