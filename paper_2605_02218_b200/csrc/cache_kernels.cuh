// The paged cache of keys and values: written token by token, held in 32 or 16 bits as they are or in 8 bits with a scale for
// each token and head, and read back.
//
// Pages [pages, heads, page_size, dim]; position t of request b lies in page table[b][t / page_size] at place t % page_size.  A
// request's tokens of a call are the last ones of its length: token i of n has position length - n + i.
// 8-bit form of a row x: scale = max(max|x| / L, 2^-100) in float32, L = 448 (e4m3) or 127; held = x / scale, rounded once,
// half to even, from the exact quotient.  The bound on the scale keeps the quotients normal numbers; a row with a value that
// is not finite gets the scale NaN and so reads back as NaN.
#pragma once
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include "common.cuh"

namespace covspec {
namespace cache {

enum Store { kF32 = 0, kBF16 = 1, kF16 = 2, kE4M3 = 3, kInt8 = 4 };

struct Pages {
  void *k, *v;
  float *k_scale, *v_scale;
  long long k_page, v_page;      // elements from page to page
  int pages, heads, page_shift;
};
struct Tokens {
  int batch;
  const int* offsets;            // [batch + 1] first token of each request
  const int* lengths;            // [batch] positions in the cache, the call's tokens included
  const int* table;              // [batch, width] page ids
  long long table_ld;
  int width;
};

constexpr int kThreads = 256;
constexpr float kLeastScale = 7.888609052210118e-31f;   // 2^-100

// Request of token i, or -1 where it belongs to none.
__device__ __forceinline__ int request_of(const Tokens& t, int i) {
  int lo = 0, hi = t.batch - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (t.offsets[mid] <= i) lo = mid; else hi = mid - 1;
  }
  return t.offsets[lo] <= i && i < t.offsets[lo + 1] ? lo : -1;
}
// Row (page * heads + head) * page_size + place of token i of request b; page -1 where it has no place in the cache.
__device__ __forceinline__ int page_of(const Tokens& t, const Pages& c, int b, int i, int& place) {
  const long long pos = (long long)t.lengths[b] - t.offsets[b + 1] + i;
  place = (int)(pos & ((1ll << c.page_shift) - 1));
  const long long slot = pos >> c.page_shift;
  if (pos < 0 || slot >= t.width) return -1;
  const int page = t.table[b * t.table_ld + slot];
  return (unsigned)page < (unsigned)c.pages ? page : -1;
}

template <typename T> __device__ __forceinline__ void load8f(const T* p, float (&v)[8]);
template <> __device__ __forceinline__ void load8f<float>(const float* p, float (&v)[8]) { load8(p, v); }
template <> __device__ __forceinline__ void load8f<__nv_bfloat16>(const __nv_bfloat16* p, float (&v)[8]) { load8(p, v); }
template <> __device__ __forceinline__ void load8f<__half>(const __half* p, float (&v)[8]) {
  const uint4 t = *reinterpret_cast<const uint4*>(p);
  const unsigned w[4] = {t.x, t.y, t.z, t.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
    v[2 * i] = f.x;
    v[2 * i + 1] = f.y;
  }
}
template <typename T> __device__ __forceinline__ void store8f(T* p, const float (&v)[8]);
template <> __device__ __forceinline__ void store8f<float>(float* p, const float (&v)[8]) {
  reinterpret_cast<float4*>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
  reinterpret_cast<float4*>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
}
template <> __device__ __forceinline__ void store8f<__nv_bfloat16>(__nv_bfloat16* p, const float (&v)[8]) {
  __nv_bfloat162 t[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) t[i] = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
  *reinterpret_cast<uint4*>(p) = *reinterpret_cast<uint4*>(t);
}
template <> __device__ __forceinline__ void store8f<__half>(__half* p, const float (&v)[8]) {
  __half2 t[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) t[i] = __floats2half2_rn(v[2 * i], v[2 * i + 1]);
  *reinterpret_cast<uint4*>(p) = *reinterpret_cast<uint4*>(t);
}

// x / s towards zero, with its last bit set where that is not exact: rounding it again to fewer bits gives what rounding the
// exact quotient gives.  s is finite and at least 2^-100, |x / s| at most L (1 + 2^-23).
__device__ __forceinline__ float quotient_sticky(float x, float s) {
  const float t = __fdiv_rz(x, s);
  const float rest = fmaf(-t, s, x);
  return rest != 0.f ? __uint_as_float(__float_as_uint(t) | 1u) : t;
}

// The 8-bit form of eight values, as the bytes of a uint2.
template <int STORE>
__device__ __forceinline__ uint2 held8(const float (&x)[8], float s) {
  uint2 r = make_uint2(0u, 0u);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float t = quotient_sticky(x[i], s);
    unsigned byte;
    if constexpr (STORE == kE4M3) {
      byte = __nv_cvt_float_to_fp8(t, __NV_SATFINITE, __NV_E4M3);
    } else {
      byte = (unsigned)max(-127, min(127, __float2int_rn(t))) & 0xffu;
    }
    (i < 4 ? r.x : r.y) |= byte << (8 * (i & 3));
  }
  return r;
}

struct WriteParams {
  Pages c;
  Tokens t;
  const void *k, *v;
  long long k_ld, v_ld;          // elements from row to row
  int n;                         // tokens
  const int* rows;               // [n] source row of each token inside its request, or null: row i is token i
  const int* row_offsets;        // [batch + 1] first source row of each request
  int source_rows;
};

// dim / 8 lanes per (token, head): one 16-byte load of the key's and one of the value's row per lane (two each for float32).
template <typename T, int STORE, int DIM>
__global__ void __launch_bounds__(kThreads) write_kernel(WriteParams p) {
  constexpr int kLanes = DIM / 8;
  const long long unit = ((long long)blockIdx.x * kThreads + threadIdx.x) / kLanes;
  const int lane = threadIdx.x % kLanes;
  const int i = (int)min(unit / p.c.heads, (long long)p.n), head = (int)(unit % p.c.heads);
  int page = -1, place = 0;
  long long source = i;
  if (i < p.n) {
    const int b = request_of(p.t, i);
    if (b >= 0) {
      page = page_of(p.t, p.c, b, i, place);
      if (p.rows) {
        source = (long long)p.row_offsets[b] + p.rows[i];
        if (source < 0 || source >= p.source_rows) page = -1;
      }
    }
  }
  float x[2][8];
  if (page >= 0) {
    load8f(static_cast<const T*>(p.k) + source * p.k_ld + head * DIM + lane * 8, x[0]);
    load8f(static_cast<const T*>(p.v) + source * p.v_ld + head * DIM + lane * 8, x[1]);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) x[0][e] = x[1][e] = 0.f;
  }
  const int row = (head << p.c.page_shift) + place;
#pragma unroll
  for (int kv = 0; kv < 2; ++kv) {
    void* base = kv ? p.c.v : p.c.k;
    const long long at = page * (kv ? p.c.v_page : p.c.k_page) + (long long)row * DIM + lane * 8;
    if constexpr (STORE >= kE4M3) {
      float top = 0.f;
      bool bad = false;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        top = fmaxf(top, fabsf(x[kv][e]));
        bad |= !(fabsf(x[kv][e]) <= 3.402823466e38f);
      }
      if (bad) top = INFINITY;
#pragma unroll
      for (int o = kLanes / 2; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
      const bool finite = top <= 3.402823466e38f;
      const float s = finite ? fmaxf(__fdiv_rn(top, STORE == kE4M3 ? 448.f : 127.f), kLeastScale) : __int_as_float(0x7fffffff);
      if (page >= 0) {
        const uint2 held = finite ? held8<STORE>(x[kv], s) : make_uint2(0u, 0u);
        *reinterpret_cast<uint2*>(static_cast<unsigned char*>(base) + at) = held;
        if (lane == 0) (kv ? p.c.v_scale : p.c.k_scale)[(((long long)page * p.c.heads) << p.c.page_shift) + row] = s;
      }
    } else if (page >= 0) {
      if constexpr (STORE == kF32) store8f(static_cast<float*>(base) + at, x[kv]);
      else if constexpr (STORE == kBF16) store8f(static_cast<__nv_bfloat16*>(base) + at, x[kv]);
      else store8f(static_cast<__half*>(base) + at, x[kv]);
    }
  }
}

struct ReadParams {
  Pages c;
  Tokens t;
  void *k, *v;                   // dense rows [n, heads, dim]
  int n;
};

template <typename T, int STORE, int DIM>
__global__ void __launch_bounds__(kThreads) read_kernel(ReadParams p) {
  constexpr int kLanes = DIM / 8;
  const long long unit = ((long long)blockIdx.x * kThreads + threadIdx.x) / kLanes;
  const int lane = threadIdx.x % kLanes;
  const int i = (int)min(unit / p.c.heads, (long long)p.n), head = (int)(unit % p.c.heads);
  if (i >= p.n) return;
  const int b = request_of(p.t, i);
  if (b < 0) return;
  int place;
  const int page = page_of(p.t, p.c, b, i, place);
  const int row = (head << p.c.page_shift) + place;
#pragma unroll
  for (int kv = 0; kv < 2; ++kv) {
    float x[8];
    if (page >= 0) {
      const void* base = kv ? p.c.v : p.c.k;
      const long long at = page * (kv ? p.c.v_page : p.c.k_page) + (long long)row * DIM + lane * 8;
      if constexpr (STORE >= kE4M3) {
        const uint2 h = *reinterpret_cast<const uint2*>(static_cast<const unsigned char*>(base) + at);
        const float s = (kv ? p.c.v_scale : p.c.k_scale)[(((long long)page * p.c.heads) << p.c.page_shift) + row];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const unsigned byte = ((e < 4 ? h.x : h.y) >> (8 * (e & 3))) & 0xffu;
          if constexpr (STORE == kE4M3) {
            x[e] = s * __half2float(__half(__nv_cvt_fp8_to_halfraw((__nv_fp8_storage_t)byte, __NV_E4M3)));
          } else {
            x[e] = s * (float)(signed char)byte;
          }
        }
      } else if constexpr (STORE == kF32) {
        load8f(static_cast<const float*>(base) + at, x);
      } else if constexpr (STORE == kBF16) {
        load8f(static_cast<const __nv_bfloat16*>(base) + at, x);
      } else {
        load8f(static_cast<const __half*>(base) + at, x);
      }
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = 0.f;
    }
    store8f(static_cast<T*>(kv ? p.v : p.k) + ((long long)i * p.c.heads + head) * DIM + lane * 8, x);
  }
}

}  // namespace cache
}  // namespace covspec
