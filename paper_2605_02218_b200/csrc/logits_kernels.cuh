// Edits of the logits of drafted blocks before they are corrected: penalties for repeated tokens, biases, grammar masks.
//
// For row j of request b, with h the request's history (its first `prompt` tokens the prompt) and y the tokens drafted at the
// rows before j of the same request:
//   seen_w  = w occurs in h or y,   c_w = occurrences of w in h[prompt..) and y
//   x = z_w;  if seen_w: x = x > 0 ? x / r_b : x * r_b;  x = x - f_b c_w;  if c_w > 0: x = x - a_b;  x = x + bias_w;
//   if w is not allowed: x = -inf
// in float32, rounded once to the type of z.  Entries that none of it concerns are copied bit by bit.
#pragma once
#include <cuda_fp16.h>

#include "common.cuh"

namespace covspec {
namespace edit {

constexpr int kThreads = 256;
constexpr unsigned kSeen = 0x80000000u;   // a word of the table: this bit from the prompt, below it the occurrences after it

struct Params {
  const void* z;
  void* out;
  long long ld;
  int rows, vocab, batch;
  const int* row_offsets;       // [batch + 1]
  const int* history;
  const int* history_offsets;   // [batch + 1]
  int history_len;
  const int* prompt;            // [batch] or null: no prompt
  const int* drafted;           // [rows] or null
  const float *repetition, *presence, *frequency;   // [batch] each, or null
  const int* bias_ids;
  const float* bias;
  const int* bias_offsets;      // [batch + 1]
  int bias_len;
  const unsigned char* mask;    // rows of mask_ld bytes, bit w % 8 of byte w / 8
  long long mask_ld;
  int segment;                  // entries of a row that one CTA holds the table of; a multiple of 256
  int group;                    // rows that one CTA goes through
};

__device__ __forceinline__ float as_float(float v) { return v; }
__device__ __forceinline__ float as_float(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float as_float(__half v) { return __half2float(v); }
template <typename T> __device__ __forceinline__ T rounded(float v);
template <> __device__ __forceinline__ float rounded<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 rounded<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half rounded<__half>(float v) { return __float2half_rn(v); }

// One CTA: `segment` entries of `group` rows.  Shared memory: a word per entry with what the history says of it, and (with
// biases) the place of its bias in the list + 1; a later place wins over an earlier one, whatever the order of the atomics.
template <typename T>
__global__ void __launch_bounds__(kThreads) edit_kernel(Params p) {
  extern __shared__ unsigned table[];
  constexpr int kVec = 16 / sizeof(T);
  const int seg0 = blockIdx.x * p.segment, len = min(p.segment, p.vocab - seg0);
  const int row0 = blockIdx.y * p.group, row1 = min(row0 + p.group, p.rows);
  unsigned* place = p.bias_ids ? table + p.segment : nullptr;
  const bool counted = p.history || p.drafted;
  const int tid = threadIdx.x;
  int b = -1, b_end = 0, b_begin = 0;
  float r = 1.f, a = 0.f, f = 0.f;
  for (int row = row0; row < row1; ++row) {
    if (b < 0 || row >= b_end) {          // the next request's tables
      int lo = 0, hi = p.batch - 1;
      while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (p.row_offsets[mid] <= row) lo = mid; else hi = mid - 1;
      }
      b = lo;
      b_begin = max(p.row_offsets[b], 0);
      b_end = p.row_offsets[b + 1];
      if (row < b_begin || row >= b_end) { b = -1; continue; }     // a row of no request stays as it was
      __syncthreads();
      for (int i = tid; i < (place ? 2 * p.segment : p.segment); i += kThreads) table[i] = 0;
      __syncthreads();
      if (p.history) {
        const int h0 = min(max(p.history_offsets[b], 0), p.history_len), h1 = min(max(p.history_offsets[b + 1], h0), p.history_len);
        const int answer = h0 + (p.prompt ? max(p.prompt[b], 0) : 0);
        for (int i = h0 + tid; i < h1; i += kThreads) {
          const unsigned w = (unsigned)(p.history[i] - seg0);
          if (w < (unsigned)len) { if (i < answer) atomicOr(table + w, kSeen); else atomicAdd(table + w, 1u); }
        }
      }
      if (p.drafted)
        for (int i = b_begin + tid; i < row; i += kThreads) {
          const unsigned w = (unsigned)(p.drafted[i] - seg0);
          if (w < (unsigned)len) atomicAdd(table + w, 1u);
        }
      if (place) {
        const int i0 = min(max(p.bias_offsets[b], 0), p.bias_len), i1 = min(max(p.bias_offsets[b + 1], i0), p.bias_len);
        for (int i = i0 + tid; i < i1; i += kThreads) {
          const unsigned w = (unsigned)(p.bias_ids[i] - seg0);
          if (w < (unsigned)len) atomicMax(place + w, (unsigned)i + 1u);
        }
      }
      r = p.repetition ? p.repetition[b] : 1.f;
      a = p.presence ? p.presence[b] : 0.f;
      f = p.frequency ? p.frequency[b] : 0.f;
      __syncthreads();
    }
    const T* z = static_cast<const T*>(p.z) + row * p.ld + seg0;
    T* out = static_cast<T*>(p.out) + row * p.ld + seg0;
    const unsigned char* mask = p.mask ? p.mask + row * p.mask_ld + seg0 / 8 : nullptr;
    for (int i = tid * kVec; i < len; i += kThreads * kVec) {
      uint4 raw = *reinterpret_cast<const uint4*>(z + i);
      T* v = reinterpret_cast<T*>(&raw);
      const unsigned allowed = mask ? mask[i / 8] >> (i % 8) : 0xffu;
#pragma unroll
      for (int k = 0; k < kVec; ++k) {
        const unsigned c = counted ? table[i + k] : 0u, at = place ? place[i + k] : 0u;
        if (c | at) {
          float x = as_float(v[k]);
          if (c) {
            x = x > 0.f ? x / r : x * r;
            const unsigned n = c & ~kSeen;
            x = __fsub_rn(x, __fmul_rn(f, (float)n));
            if (n) x -= a;
          }
          if (at) x += p.bias[at - 1];
          v[k] = rounded<T>(x);
        }
        if (!((allowed >> k) & 1u)) v[k] = rounded<T>(-INFINITY);
      }
      if (i + kVec <= len) {
        *reinterpret_cast<uint4*>(out + i) = raw;
      } else {
        for (int k = 0; i + k < len; ++k) out[i + k] = v[k];
      }
    }
    if (p.drafted && row + 1 < min(b_end, row1)) {     // the next row has this one's token behind it
      __syncthreads();
      const unsigned w = (unsigned)(p.drafted[row] - seg0);
      if (tid == 0 && w < (unsigned)len) table[w] += 1u;
      __syncthreads();
    }
  }
}

}  // namespace edit
}  // namespace covspec
