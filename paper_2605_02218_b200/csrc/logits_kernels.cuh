// Edits of the logits of drafted blocks before they are corrected: penalties for repeated tokens, biases, grammar masks.
//
// For row j of request b, with h the request's history (its first `prompt` tokens the prompt) and y the tokens drafted at the
// rows before j of the same request:
//   seen_w  = w occurs in h or y,   c_w = occurrences of w in h[prompt..) and y
//   x = z_w;  if seen_w: x = x > 0 ? x / r_b : x * r_b;  x = x - f_b c_w;  if c_w > 0: x = x - a_b;  x = x + bias_w;
//   if w is not allowed: x = -inf
// in float32, rounded once to the type of z.  Entries that none of it concerns are copied bit by bit.
#pragma once
#include "cache_kernels.cuh"

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
  int segment;                  // entries of a row that one CTA holds the tables of; a multiple of 256
  int group;                    // rows that one CTA goes through
};

__device__ __forceinline__ float as_float(float v) { return v; }
__device__ __forceinline__ float as_float(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float as_float(__half v) { return __half2float(v); }
template <typename T> __device__ __forceinline__ T rounded(float v);
template <> __device__ __forceinline__ float rounded<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 rounded<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half rounded<__half>(float v) { return __float2half_rn(v); }

// Minus infinity in the halves (or the word) of `v` whose bits of `allowed` are 0.
template <typename T> __device__ __forceinline__ unsigned masked(unsigned v, unsigned allowed) {
  if constexpr (sizeof(T) == 4) {
    return allowed & 1u ? v : 0xff800000u;
  } else {
    constexpr unsigned kLow = __is_same(T, __half) ? 0xfc00u : 0xff80u;
    const unsigned lo = allowed & 1u ? v & 0xffffu : kLow, hi = allowed & 2u ? v & 0xffff0000u : kLow << 16;
    return lo | hi;
  }
}

// One CTA: `segment` entries of `group` rows.  Shared memory: a bit per entry that an edit of the request concerns it; a word with
// what the history says of it; with biases, the place of its bias in the list + 1 (a later place wins over an earlier one,
// whatever the order of the atomics).  Bound by reading and writing the rows; entries with no bit set go through as they are, and a
// vector of which the grammar allows nothing is not read.  1024 rows x 151674 f16 with masks: 172 us, 3.7 TB/s of what reading and
// writing everything once would be; small tables (two vectors of a thread in flight, 4096 entries) let six CTAs share an SM, with four
// vectors and 8192 entries it was 278.
template <typename T>
__global__ void __launch_bounds__(kThreads) edit_kernel(Params p) {
  extern __shared__ __align__(16) unsigned edit_smem[];
  constexpr int kVec = 16 / sizeof(T), kFlight = 2;
  unsigned* bits = edit_smem;                              // [segment / 32]
  unsigned* table = bits + p.segment / 32;
  unsigned* place = p.bias_ids ? table + p.segment : nullptr;
  const unsigned char* bytes = reinterpret_cast<const unsigned char*>(bits);
  const int seg0 = blockIdx.x * p.segment, len = min(p.segment, p.vocab - seg0);
  const int row0 = blockIdx.y * p.group, row1 = min(row0 + p.group, p.rows);
  const int tid = threadIdx.x;
  int b = -1, b_end = 0, b_begin = 0;
  float r = 1.f, a = 0.f, f = 0.f;
  wait_for_previous_kernel();
  auto mask_at = [&](const unsigned char* m, int i) { return !m ? 0xffu : i < len ? (unsigned)m[i / 8] >> (i % 8) : 0u; };
  unsigned ahead[kFlight];                 // the mask of this thread's first vectors of the row to come
#pragma unroll
  for (int j = 0; j < kFlight; ++j) ahead[j] = mask_at(p.mask ? p.mask + row0 * p.mask_ld + seg0 / 8 : nullptr, (tid + j * kThreads) * kVec);
  for (int row = row0; row < row1; ++row) {
    if (b < 0 || row >= b_end) {          // the next request's tables
      b = cache::segment_of(p.row_offsets, p.batch, row);
      b_begin = max(p.row_offsets[b], 0);
      b_end = p.row_offsets[b + 1];
      if (row < b_begin || row >= b_end) {       // a row of no request stays as it was
        b = -1;
        if (row + 1 < row1)
#pragma unroll
          for (int j = 0; j < kFlight; ++j) ahead[j] = mask_at(p.mask ? p.mask + (row + 1) * p.mask_ld + seg0 / 8 : nullptr, (tid + j * kThreads) * kVec);
        continue;
      }
      __syncthreads();
      const int words = p.segment / 32 + p.segment * (place ? 2 : 1);
      for (int i = tid; i < words / 4; i += kThreads) reinterpret_cast<uint4*>(edit_smem)[i] = make_uint4(0u, 0u, 0u, 0u);
      r = p.repetition ? p.repetition[b] : 1.f;
      a = p.presence ? p.presence[b] : 0.f;
      f = p.frequency ? p.frequency[b] : 0.f;
      int h0 = 0, h1 = 0, answer = 0, i0 = 0, i1 = 0;
      if (p.history) {
        h0 = min(max(p.history_offsets[b], 0), p.history_len);
        h1 = min(max(p.history_offsets[b + 1], h0), p.history_len);
        answer = (int)min((long long)h0 + (p.prompt ? max(p.prompt[b], 0) : 0), (long long)h1);
      }
      if (place) {
        i0 = min(max(p.bias_offsets[b], 0), p.bias_len);
        i1 = min(max(p.bias_offsets[b + 1], i0), p.bias_len);
      }
      __syncthreads();
      auto inside = [&](int token) { return (unsigned)token - (unsigned)seg0; };
#pragma unroll 8
      for (int i = h0 + tid; i < answer; i += kThreads)
        if (const unsigned w = inside(p.history[i]); w < (unsigned)len) table[w] = kSeen;
      for (int i = i0 + tid; i < i1; i += kThreads)
        if (const unsigned w = inside(p.bias_ids[i]); w < (unsigned)len) atomicMax(place + w, (unsigned)i + 1u);
      __syncthreads();
#pragma unroll 8
      for (int i = answer + tid; i < h1; i += kThreads)
        if (const unsigned w = inside(p.history[i]); w < (unsigned)len) atomicAdd(table + w, 1u);
      if (p.drafted)
        for (int i = b_begin + tid; i < row; i += kThreads)
          if (const unsigned w = inside(p.drafted[i]); w < (unsigned)len) atomicAdd(table + w, 1u);
      __syncthreads();
      for (int i = tid; i < p.segment; i += kThreads) {
        const unsigned word = __ballot_sync(0xffffffffu, table[i] != 0u || (place && place[i] != 0u));
        if ((tid & 31) == 0) bits[i / 32] = word;
      }
      __syncthreads();
    }
    const T* z = static_cast<const T*>(p.z) + row * p.ld + seg0;
    T* out = static_cast<T*>(p.out) + row * p.ld + seg0;
    const unsigned char* mask = p.mask ? p.mask + row * p.mask_ld + seg0 / 8 : nullptr;
    const bool follows = p.drafted && row + 1 < min(b_end, row1);
    const unsigned drafted = follows ? (unsigned)p.drafted[row] - (unsigned)seg0 : ~0u;
    for (int at = tid * kVec; at < len; at += kThreads * kVec * kFlight) {
      uint4 raw[kFlight];
      unsigned allowed[kFlight];
#pragma unroll
      for (int j = 0; j < kFlight; ++j) {
        const int i = at + j * kThreads * kVec;
        allowed[j] = at == tid * kVec ? ahead[j] : mask_at(mask, i);
      }
      if (at == tid * kVec && mask && row + 1 < row1) {
#pragma unroll
        for (int j = 0; j < kFlight; ++j) ahead[j] = mask_at(mask + p.mask_ld, at + j * kThreads * kVec);
      }
#pragma unroll
      for (int j = 0; j < kFlight; ++j) {
        const int i = at + j * kThreads * kVec;
        raw[j] = make_uint4(0u, 0u, 0u, 0u);
        if (i < len && (allowed[j] & ((1u << kVec) - 1u))) raw[j] = *reinterpret_cast<const uint4*>(z + i);
      }
#pragma unroll
      for (int j = 0; j < kFlight; ++j) {
        const int i = at + j * kThreads * kVec;
        if (i >= len) break;
        const unsigned edits = (unsigned)bytes[i / 8] >> (i % 8) & allowed[j] & ((1u << kVec) - 1u);
        if (edits) {
          T* v = reinterpret_cast<T*>(&raw[j]);
#pragma unroll
          for (int k = 0; k < kVec; ++k) {
            if (!((edits >> k) & 1u)) continue;
            const unsigned c = table[i + k], from = place ? place[i + k] : 0u;
            float x = as_float(v[k]);
            if (c) {
              x = x > 0.f ? x / r : x * r;
              const unsigned n = c & ~kSeen;
              x = __fsub_rn(x, __fmul_rn(f, (float)n));
              if (n) x -= a;
            }
            if (from) x += p.bias[from - 1];
            v[k] = rounded<T>(x);
          }
        }
        if (mask) {
          unsigned* w = reinterpret_cast<unsigned*>(&raw[j]);
#pragma unroll
          for (int k = 0; k < 4; ++k) w[k] = masked<T>(w[k], allowed[j] >> (k * (kVec / 4)));
        }
        if (i + kVec <= len) {
          *reinterpret_cast<uint4*>(out + i) = raw[j];
        } else {
          const T* v = reinterpret_cast<const T*>(&raw[j]);
#pragma unroll
          for (int k = 0; k < kVec; ++k)
            if (i + k < len) out[i + k] = v[k];
        }
      }
    }
    if (drafted < (unsigned)len) {        // the next row has this one's token behind it
      __syncthreads();
      if (tid == 0) {
        table[drafted] += 1u;
        bits[drafted / 32] |= 1u << (drafted % 32);
      }
      __syncthreads();
    }
  }
}

}  // namespace edit
}  // namespace covspec
