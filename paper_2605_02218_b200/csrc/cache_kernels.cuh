// The paged cache of keys and values: written token by token, held in 32 or 16 bits as they are or in 8 bits with a scale for
// each token and head, and read back.
//
// Pages [pages, heads, page_size, dim]; position t of request b lies in page table[b][t / page_size] at place t % page_size.  A
// request's tokens of a call are the last ones of its length: token i of n has position length - n + i.
// 8-bit form of a row x: scale = max(max|x| / L, 2^-100) in float32, L = 448 (e4m3) or 127; held = x / scale, rounded once,
// half to even, from the exact quotient.  The bound on the scale keeps the quotients normal numbers; a row with a value that
// is not finite gets the scale NaN and so reads back as NaN.
//
// Both directions are bound by HBM when they are large.  27.8 k kept tokens x 8 heads x 128 from bf16 to int8: 49 us, 3.5 TB/s (the
// quantising arithmetic, about 13 instructions a value, is not hidden entirely); e4m3 back to bf16, 146 k tokens: 155-160 us, 5.7 TB/s.
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

// Last of the `batch` segments that begins at or before i, by ascending first elements: seven of them looked at together, so that a
// few hundred segments take three dependent loads.
__device__ __forceinline__ int segment_of(const int* offsets, int batch, int i) {
  int lo = 0, n = batch;                 // it is among lo .. lo + n - 1
  while (n > 1) {
    const int step = (n + 7) / 8;
    int before = 0;
#pragma unroll
    for (int j = 1; j < 8; ++j) before += j * step < n && offsets[lo + j * step] <= i;
    lo += before * step;
    n = min(step, n - before * step);
  }
  return lo;
}
// Request of token i, or -1 where it belongs to none.
__device__ __forceinline__ int request_of(const Tokens& t, int i) {
  const int b = segment_of(t.offsets, t.batch, i);
  return t.offsets[b] <= i && i < t.offsets[b + 1] ? b : -1;
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
// The 8-bit form of eight values, as the bytes of a uint2.  t = x times the rounded 1 / s is off by less than 2^-22 of the quotient;
// what decides next to a border between two held values is the exact rest x - border * s.  Quotients of 16-bit numbers meet
// borders all the time (half of the largest value is 63.5 steps of int8), so the rest costs no division: with one for each
// value 27.8 k tokens x 8 heads x 128 features took 132 us, and with one where it is close 178.
//  int8: the rest of the nearest step k, a multiple of half a unit in the last place of s below s, is exact in float32.
//  e4m3: 20 of the 23 bits go, a border is a half of the last that stays; below the normal numbers the quotient itself is taken.
// Either is looked for in all eight values at once and mended in a branch that few warps take.
template <int STORE>
__device__ __forceinline__ uint2 held8(const float (&x)[8], float s) {
  const float inv = __frcp_rn(s);
  uint2 r = make_uint2(0u, 0u);
  if constexpr (STORE == kInt8) {
    constexpr float kMagic = 12582912.f;             // 1.5 * 2^23: the sum's last bits are the rounded number
    const float half = 0.5f * s;
    float m[8], most = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      m[i] = fmaf(x[i], inv, kMagic);
      most = fmaxf(most, fabsf(fmaf(kMagic - m[i], s, x[i])));
    }
    if (most >= half) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float rest = fmaf(kMagic - m[i], s, x[i]);
        if (fabsf(rest) > half || (fabsf(rest) == half && (__float_as_uint(m[i]) & 1u))) m[i] += rest > 0.f ? 1.f : -1.f;
      }
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const uint32_t a = __byte_perm(__float_as_uint(m[4 * i]), __float_as_uint(m[4 * i + 1]), 0x0040);
      const uint32_t b = __byte_perm(__float_as_uint(m[4 * i + 2]), __float_as_uint(m[4 * i + 3]), 0x0040);
      (i ? r.y : r.x) = __byte_perm(a, b, 0x5410);
    }
  } else {
    float t[8], least = 1.f;
    uint32_t near = 0xffffffffu;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      t[i] = x[i] * inv;
      least = fminf(least, fabsf(t[i]));
      near = min(near, (__float_as_uint(t[i]) + 0x80008u) & 0xfffffu);
    }
    if (near <= 16u || least < 0.015625f) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const uint32_t bits = __float_as_uint(t[i]);
        if (((bits + 0x80008u) & 0xfffffu) <= 16u) {
          const uint32_t border = (bits + 8u) & 0xfff00000u | 0x80000u;
          const float rest = fmaf(-__uint_as_float(border), s, x[i]);
          t[i] = __uint_as_float(rest == 0.f ? border : (rest > 0.f) == (x[i] > 0.f) ? border + 1u : border - 1u);
        }
        if (fabsf(t[i]) < 0.015625f && x[i] != 0.f) t[i] = quotient_sticky(x[i], s);
      }
    }
#pragma unroll
    for (int i = 0; i < 8; i += 2)
      (i < 4 ? r.x : r.y) |= (uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(t[i], t[i + 1]), __NV_SATFINITE, __NV_E4M3) << (8 * (i & 3));
  }
  return r;
}

// A warp takes several times as many neighbouring (token, head) rows as its lanes cover with 16 bytes each.  Every lane finds the
// place of one row, so the chain of look-ups (request, length, page) is gone through once per warp.
constexpr int kPasses = 4;
struct Spot {
  int page, row, source;       // page -1: none; row (head * page_size + place) in it; row of the dense side
};
__device__ __forceinline__ Spot spot_of(const Tokens& t, const Pages& c, int unit, int n, const int* rows, const int* row_offsets,
                                        int source_rows) {
  Spot s{-1, 0, -1};
  const int i = unit / c.heads, head = unit % c.heads;
  if (i >= n) return s;
  const int b = request_of(t, i);
  if (b < 0) return s;
  int place;
  s.page = page_of(t, c, b, i, place);
  s.row = (head << c.page_shift) + place;
  s.source = i;
  if (rows) {
    const long long source = (long long)row_offsets[b] + rows[i];
    if (source < 0 || source >= source_rows) s.page = -1;
    s.source = (int)source;
  }
  return s;
}
__device__ __forceinline__ Spot handed(const Spot& s, int lane) {
  return Spot{__shfl_sync(0xffffffffu, s.page, lane), __shfl_sync(0xffffffffu, s.row, lane), __shfl_sync(0xffffffffu, s.source, lane)};
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
  int passes;                    // 1 or kPasses
};

// Eight features a lane: one 16-byte load (two for float32).
template <typename T, int STORE, int DIM>
__global__ void __launch_bounds__(kThreads) write_kernel(WriteParams p) {
  constexpr int kLanes = DIM / 8, kRows = 32 / kLanes;
  const int lane = threadIdx.x & 31, sub = lane / kLanes, feature = lane % kLanes * 8, mine = kRows * p.passes;
  const int unit0 = (blockIdx.x * (kThreads / 32) + warp_index()) * mine;
  wait_for_previous_kernel();
  const Spot spot = lane < mine ? spot_of(p.t, p.c, unit0 + lane, p.n, p.rows, p.row_offsets, p.source_rows) : Spot{-1, 0, -1};
  struct Raw { uint4 w[2][sizeof(T) / 2]; } raw{};             // a key's and a value's eight features
  auto fetch = [&](const Spot& s) {
    if (s.page < 0) return;
    const int head = s.row >> p.c.page_shift;
    const uint4* k = reinterpret_cast<const uint4*>(static_cast<const T*>(p.k) + s.source * p.k_ld + head * DIM + feature);
    const uint4* v = reinterpret_cast<const uint4*>(static_cast<const T*>(p.v) + s.source * p.v_ld + head * DIM + feature);
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) { raw.w[0][i] = k[i]; raw.w[1][i] = v[i]; }
  };
  Spot s = handed(spot, sub);
  fetch(s);
  for (int first = 0; first < mine; first += kRows) {
    float x[2][8];
#pragma unroll
    for (int kv = 0; kv < 2; ++kv) load8f(reinterpret_cast<const T*>(raw.w[kv]), x[kv]);
    const Spot next = first + kRows < mine ? handed(spot, first + kRows + sub) : Spot{-1, 0, -1};
    fetch(next);                 // under way while this row is worked on
#pragma unroll
    for (int kv = 0; kv < 2; ++kv) {
      void* base = kv ? p.c.v : p.c.k;
      const long long at = s.page * (kv ? p.c.v_page : p.c.k_page) + (long long)s.row * DIM + feature;
      if constexpr (STORE >= kE4M3) {
        float top = 0.f;
        bool bad = false;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          top = fmaxf(top, fabsf(x[kv][e]));
          bad |= x[kv][e] != x[kv][e];
        }
        if (bad) top = INFINITY;
#pragma unroll
        for (int o = kLanes / 2; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
        const bool finite = top <= 3.402823466e38f;
        const float scale = finite ? fmaxf(__fdiv_rn(top, STORE == kE4M3 ? 448.f : 127.f), kLeastScale) : __int_as_float(0x7fffffff);
        if (s.page >= 0) {
          *reinterpret_cast<uint2*>(static_cast<unsigned char*>(base) + at) = finite ? held8<STORE>(x[kv], scale) : make_uint2(0u, 0u);
          if (feature == 0) (kv ? p.c.v_scale : p.c.k_scale)[(((long long)s.page * p.c.heads) << p.c.page_shift) + s.row] = scale;
        }
      } else if (s.page >= 0) {
        if constexpr (STORE == kF32) store8f(static_cast<float*>(base) + at, x[kv]);
        else if constexpr (STORE == kBF16) store8f(static_cast<__nv_bfloat16*>(base) + at, x[kv]);
        else store8f(static_cast<__half*>(base) + at, x[kv]);
      }
    }
    s = next;
  }
}

struct ReadParams {
  Pages c;
  Tokens t;
  void *k, *v;                   // dense rows [n, heads, dim]
  int n;
};

// 16 bytes of the cache a lane, as E floats.
template <int STORE, int E> __device__ __forceinline__ void widen_held(const uint4& h, float s, float (&x)[E]) {
  const unsigned w[4] = {h.x, h.y, h.z, h.w};
#pragma unroll
  for (int e = 0; e < E; ++e) {
    if constexpr (STORE == kE4M3) {
      x[e] = s * __half2float(__half(__nv_cvt_fp8_to_halfraw((__nv_fp8_storage_t)((w[e / 4] >> (8 * (e & 3))) & 0xffu), __NV_E4M3)));
    } else if constexpr (STORE == kInt8) {
      x[e] = s * (float)(signed char)((w[e / 4] >> (8 * (e & 3))) & 0xffu);
    } else if constexpr (STORE == kBF16) {
      x[e] = __uint_as_float(e & 1 ? w[e / 2] & 0xffff0000u : w[e / 2] << 16);
    } else if constexpr (STORE == kF16) {
      x[e] = __half2float(__ushort_as_half((unsigned short)(w[e / 2] >> (16 * (e & 1)))));
    } else {
      x[e] = __uint_as_float(w[e]);
    }
  }
}
template <typename T, int E> __device__ __forceinline__ void store_row(T* p, const float (&x)[E]) {
  if constexpr (E == 4) {
    if constexpr (sizeof(T) == 4) {
      *reinterpret_cast<float4*>(p) = make_float4(x[0], x[1], x[2], x[3]);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if constexpr (__is_same(T, __half)) p[e] = __float2half_rn(x[e]);
        else p[e] = __float2bfloat16_rn(x[e]);
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < E; i += 8) {
      float y[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = x[i + e];
      store8f(p + i, y);
    }
  }
}

template <typename T, int STORE, int DIM>
__global__ void __launch_bounds__(kThreads) read_kernel(ReadParams p) {
  constexpr int E = STORE >= kE4M3 ? 16 : STORE == kF32 ? 4 : 8, kBytes = 16 / E;
  constexpr int kLanes = DIM / E, kRows = 32 / kLanes;
  const int lane = threadIdx.x & 31, sub = lane / kLanes, feature = lane % kLanes * E;
  const int unit0 = (blockIdx.x * (kThreads / 32) + warp_index()) * (kRows * kPasses);
  wait_for_previous_kernel();
  Spot mine = lane < kRows * kPasses ? spot_of(p.t, p.c, unit0 + lane, p.n, nullptr, nullptr, 0) : Spot{-1, 0, -1};
  uint4 h[kPasses][2];
  [[maybe_unused]] float scale[kPasses][2];
#pragma unroll
  for (int a = 0; a < kPasses; ++a) {
    const Spot s = handed(mine, a * kRows + sub);
#pragma unroll
    for (int kv = 0; kv < 2; ++kv) {
      h[a][kv] = make_uint4(0u, 0u, 0u, 0u);
      scale[a][kv] = 0.f;
      if (s.page >= 0) {
        const char* base = static_cast<const char*>(kv ? p.c.v : p.c.k);
        h[a][kv] = *reinterpret_cast<const uint4*>(base + (s.page * (kv ? p.c.v_page : p.c.k_page) + (long long)s.row * DIM + feature) * kBytes);
        if constexpr (STORE >= kE4M3) scale[a][kv] = (kv ? p.c.v_scale : p.c.k_scale)[(((long long)s.page * p.c.heads) << p.c.page_shift) + s.row];
      }
    }
  }
#pragma unroll
  for (int a = 0; a < kPasses; ++a) {
    if (__shfl_sync(0xffffffffu, mine.source, a * kRows + sub) < 0) continue;
#pragma unroll
    for (int kv = 0; kv < 2; ++kv) {
      float x[E];
      widen_held<STORE, E>(h[a][kv], scale[a][kv], x);
      store_row<T, E>(static_cast<T*>(kv ? p.v : p.k) + (long long)(unit0 + a * kRows + sub) * DIM + feature, x);
    }
  }
}

}  // namespace cache
}  // namespace covspec
