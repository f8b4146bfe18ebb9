// Attention of each request's newest tokens over its paged cache: what the kernels share.
//
// Query token i of n of request b stands at position p = length - n + i and attends to the keys max(0, p - window + 1) .. p.
// The group = q_heads / heads query heads of a key head are rows of one tile: row r of a request is token r / group, query head
// h * group + r % group.  A key head's rows are cut into items of `tile_rows` rows, an item's keys into units of `tile_keys`;
// the units of all items, request by request and head by head, form one sequence that the CTAs cut into equal shares, so the
// split follows the lengths on the device and needs no plan from the host.  An item that lies in one share is finished there.
// The others leave their running maxima, sums and unnormalised rows in the workspace, and attend_join_kernel adds them up in the
// order of the shares.
//
// A block one of whose waits gave up marks its share in `open` and leaves; what it has written by then does not matter.  The join makes
// every item that has a unit in such a share NaN: the block that joins an item looks at the marks of all its shares, and a marked
// share's own block goes through the items that begin there.
#pragma once
#include <cuda_fp16.h>

#include "cache_kernels.cuh"
#include "tc_common.cuh"

namespace covspec {
namespace attend {

struct Params {
  cache::Pages c;
  cache::Tokens t;
  const void* q;
  void* out;
  float* lse;                    // or null
  long long q_ld, out_ld;        // elements from token to token
  int n, q_heads, group, window; // window 0: none
  float scale_log2;              // scale * log2(e)
  int rows_over, rows_upto;      // the requests that this launch takes: rows_over < n_b * group <= rows_upto
  int least_units;               // a share is no smaller
  float* part;                   // [2 * grid][tile_rows * (dim + 2)]: rows, maxima, sums of the shares' first and last item
  int4* open;                    // [grid][2]: the item that a share leaves unfinished: first token of its request, head, first
                                 // row, rows; last share of the item, 1 where a wait gave up
  uint32_t polls;                // that a wait makes before it gives up
  int stop_share, stop_unit;     // self-test: the loading warp of this share (-1: none) leaves before this unit
};
// Nothing in these kernels waits for more than what its own CTA has under way.  A wait in vain takes about a second.
constexpr uint32_t kPolls = 1u << 18;

// A wait of the whole warp: its lanes poll together and leave together.  And every lane itself arrives at the barrier without which the one
// that it waits for does not complete again, so that no lane can be left behind by two phases, whatever the compiler makes of the
// warp's convergence: with a loop of its own for each lane, a vote behind it and arrivals by lane 0, lanes left one by one, and in some
// builds lane 0 went on alone and the others waited for a phase that was over.  (One lane that polls for all: 202 us for 138 with 64 single
// tokens over e4m3 caches, 975 for 680 with prompts.)
__device__ __forceinline__ bool warp_wait(uint64_t* bar, uint32_t parity, volatile int* abort_flag, uint32_t polls) {
  for (uint32_t i = 0; i < polls; ++i) {
    if (__all_sync(0xffffffffu, tc::mbar_try_wait(bar, parity))) return true;
    if ((i & 255u) == 255u && __any_sync(0xffffffffu, *abort_flag)) return false;
  }
  *abort_flag = 1;
  return false;
}
// One thread waits for what is under way, whatever has given up.
__device__ __forceinline__ void drain(uint64_t* bar, uint32_t parity) {
  volatile int none = 0;
  tc::mbar_wait_limited(bar, parity, &none, kPolls);
}

// One request as the kernels see it.  Offsets, lengths and positions that make no sense give it no rows or no keys.
struct Request {
  int q0, first, keys, rows;     // first token; its position
};
__device__ __forceinline__ Request load_request(const Params& p, int b) {
  Request r;
  const int length = max(p.t.lengths[b], 0);
  r.q0 = max(p.t.offsets[b], 0);
  const int e = max(p.t.offsets[b + 1], r.q0);         // no end so far before the start that the difference leaves 32 bits
  // a token keeps its position where its request begins before the call's rows or ends behind them; a call has fewer than 2^30 tokens,
  // so what lies further below 0 stays there
  r.first = max(length - (e - r.q0), -(1 << 30));
  r.keys = (int)min((long long)length, (long long)p.t.width << p.c.page_shift);
  r.rows = max(min(e, p.n) - r.q0, 0) * p.group;
  if (r.rows <= p.rows_over || r.rows > p.rows_upto) r.rows = 0;
  return r;
}
struct Range { int lo, hi; };    // keys lo .. hi - 1
template <int ROWS>
__device__ __forceinline__ Range keys_of(const Params& p, const Request& r, int tile) {
  const int first = tile * ROWS / p.group, last = min((tile + 1) * ROWS, r.rows) - 1;
  const int end = r.first + last / p.group + 1;
  Range k;
  k.hi = min(max(end, 0), r.keys);
  k.lo = p.window ? max(r.first + first - p.window + 1, 0) : 0;
  return k;
}
template <int KEYS>
__device__ __forceinline__ int units_of(const Range& k) {
  return k.hi > k.lo ? (k.hi - 1) / KEYS - k.lo / KEYS + 1 : 1;
}

// Place in the sequence of units: the item and the keys of one unit.
template <int ROWS, int KEYS>
struct Cursor {
  Request r;
  Range k;
  int b, h, tile;
  int key, unit, units;          // first key of the unit; its place in the item, the item's units

  __device__ __forceinline__ void open(const Params& p) {
    k = keys_of<ROWS>(p, r, tile);
    units = units_of<KEYS>(k);
    unit = 0;
    key = k.lo / KEYS * KEYS;
  }
  __device__ __forceinline__ void next(const Params& p) {
    key += KEYS;
    if (++unit < units) return;
    if (++tile * ROWS >= r.rows) {
      tile = 0;
      if (++h == p.c.heads) {
        h = 0;
        do {
          if (++b >= p.t.batch) { units = 0x3fffffff; return; }   // behind the last item
          r = load_request(p, b);
        } while (!r.rows);
      }
    }
    open(p);
  }
};

// Share `blockIdx.x` of gridDim.x: its first unit and the number of its units; every thread of the block calls it.  Shares are cut from
// a line on which an item is OPEN steps, what beginning and ending it costs, and then one for each unit; `first` and `per` are
// places on it.  `scratch`: THREADS / 32 + 4 words of shared memory.
template <int ROWS, int KEYS, int THREADS, int OPEN>
__device__ __forceinline__ int find_share(const Params& p, Cursor<ROWS, KEYS>& c, long long& first, long long& per, long long* scratch) {
  long long* sums = scratch;
  long long& place_unit = scratch[THREADS / 32];       // units of the share
  int* place = reinterpret_cast<int*>(scratch + THREADS / 32 + 1);
  const int tid = threadIdx.x, each = (p.t.batch + THREADS - 1) / THREADS;
  const int b0 = min(tid * each, p.t.batch), b1 = min(b0 + each, p.t.batch);
  auto per_head = [&](const Request& r) {
    long long s = 0;
    const int tiles = (r.rows + ROWS - 1) / ROWS;
    for (int t = 0; t < tiles; ++t) s += OPEN + units_of<KEYS>(keys_of<ROWS>(p, r, t));
    return s;
  };
  long long mine = 0;
  for (int b = b0; b < b1; ++b) mine += per_head(load_request(p, b)) * p.c.heads;
  long long scan = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long v = __shfl_up_sync(0xffffffffu, scan, o);
    if ((tid & 31) >= o) scan += v;
  }
  if ((tid & 31) == 31) sums[tid >> 5] = scan;
  __syncthreads();
  long long before = 0;
  long long total = 0;
  for (int w = 0; w < THREADS / 32; ++w) {
    if (w < (tid >> 5)) before += sums[w];
    total += sums[w];
  }
  before += scan - mine;
  per = max((total + gridDim.x - 1) / gridDim.x, (long long)p.least_units);
  first = per * blockIdx.x;
  const long long steps = min(per, total - first);
  if (steps <= 0) return 0;
  if (first >= before && first < before + mine) {
    long long left = first - before;
    int b = b0;
    Request r;
    long long u;
    for (;; ++b) {
      r = load_request(p, b);
      u = per_head(r);
      if (left < u * p.c.heads) break;
      left -= u * p.c.heads;
    }
    const int h = (int)(left / u);
    left -= h * u;
    int tile = 0;
    for (;; ++tile) {
      const int n = OPEN + units_of<KEYS>(keys_of<ROWS>(p, r, tile));
      if (left < n) break;
      left -= n;
    }
    const int unit = max((int)left - OPEN, 0);
    long long count = steps;
    if constexpr (OPEN > 0) {                             // the units among the steps; a share is far below 2^31 of them
      Cursor<ROWS, KEYS> walk;
      walk.b = b; walk.h = h; walk.tile = tile; walk.r = r;
      walk.open(p);
      count = 0;
      for (long long todo = steps, at = left;;) {
        const long long rest = OPEN + walk.units - at;
        if (rest >= todo) {
          count += max(at + todo - OPEN, 0ll) - max(at - OPEN, 0ll);
          break;
        }
        count += walk.units - max(at - OPEN, 0ll);
        todo -= rest;
        at = 0;
        walk.unit = walk.units - 1;
        walk.next(p);
      }
    }
    place[0] = b;
    place[1] = h;
    place[2] = tile;
    place[3] = unit;
    place_unit = count;
  }
  __syncthreads();
  c.b = place[0];
  c.h = place[1];
  c.tile = place[2];
  c.r = load_request(p, c.b);
  c.open(p);
  c.unit = place[3];
  c.key += c.unit * KEYS;
  return (int)place_unit;
}

// Output row of tile row `row` of an item: element offset in a [tokens, q_heads, dim] array and the place in lse.
__device__ __forceinline__ long long token_of(const Params& p, int q0, int row) { return q0 + row / p.group; }
__device__ __forceinline__ int head_of(const Params& p, int h, int row) { return h * p.group + row % p.group; }

template <typename T> __device__ __forceinline__ uint32_t pack2of(float a, float b);
template <> __device__ __forceinline__ uint32_t pack2of<__nv_bfloat16>(float a, float b) { return tc::pack_bf16(a, b); }
template <> __device__ __forceinline__ uint32_t pack2of<__half>(float a, float b) {
  const __half2 t = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&t);
}

// NaN in the rows, and their log-sums, of the items that begin in the block's share.
template <typename T, int ROWS, int KEYS, int OPEN, int DIM>
__device__ __noinline__ void give_up_share(const Params& p) {
  __shared__ long long scratch[128 / 32 + 4];
  Cursor<ROWS, KEYS> at;
  long long first, per;
  const int count = find_share<ROWS, KEYS, 128, OPEN>(p, at, first, per, scratch);
  const int row = blockIdx.y * 4 + warp_index(), lane = threadIdx.x & 31;
  const float nan = __int_as_float(0x7fffffff);
  for (int u = 0; u < count; ++u) {
    const int r = at.tile * ROWS + row;
    if (at.unit == 0 && r < at.r.rows) {
      const long long token = token_of(p, at.r.q0, r);
      const int qh = head_of(p, at.h, r);
      uint32_t* out = reinterpret_cast<uint32_t*>(static_cast<T*>(p.out) + token * p.out_ld + (long long)qh * DIM);
      for (int e = lane; e < DIM / 2; e += 32) out[e] = pack2of<T>(nan, nan);
      if (p.lse && lane == 0) p.lse[token * p.q_heads + qh] = nan;
    }
    if (u + 1 < count) at.next(p);
  }
}

// Joins the shares of the items that no share holds alone: one warp per (item, row).  A share leaves at most one item open, its
// last, which its own slot 1 and slot 0 of the following shares hold.
template <typename T, int ROWS, int KEYS, int OPEN, int DIM>
__global__ void __launch_bounds__(128) attend_join_kernel(const __grid_constant__ Params p) {
  wait_for_previous_kernel();
  const int share = blockIdx.x;
  const int4 item = p.open[2 * share], more = p.open[2 * share + 1];
  const int row = blockIdx.y * 4 + warp_index(), lane = threadIdx.x & 31;
  if (more.y) {
    give_up_share<T, ROWS, KEYS, OPEN, DIM>(p);
    return;
  }
  if (more.x <= share || row >= item.w) return;
  constexpr long long kSlot = (long long)ROWS * (DIM + 2);
  auto slot_of = [&](int s) { return p.part + (2ll * s + (s == share)) * kSlot; };
  float top = -INFINITY;
  int lost = 0;
  for (int s = share + lane; s <= more.x; s += 32) {
    top = fmaxf(top, slot_of(s)[ROWS * DIM + row]);
    lost |= p.open[2 * s + 1].y;
  }
  top = warp_max(top);
  lost = __any_sync(0xffffffffu, lost != 0);
  const float safe = top == -INFINITY ? 0.f : top;
  constexpr int kPer = DIM / 32;
  float o[kPer], sum = 0.f;
#pragma unroll
  for (int e = 0; e < kPer; ++e) o[e] = 0.f;
#pragma unroll 4
  for (int s = share; s <= more.x; ++s) {
    const float* slot = slot_of(s);
    // in two steps: sums of 8-bit caches go on counting where the references are more than 2^126 apart
    const float apart = slot[ROWS * DIM + row] - safe, near = fmaxf(apart, -120.f), rest = exp2f(apart - near);
    float w = exp2f(near);
    sum += w * (slot[ROWS * (DIM + 1) + row] * rest);
    w *= rest;
    const float* x = slot + row * DIM + lane * kPer;
    if constexpr (kPer == 4) {
      const float4 v = *reinterpret_cast<const float4*>(x);
      o[0] += w * v.x; o[1] += w * v.y; o[2] += w * v.z; o[3] += w * v.w;
    } else {
      const float2 v = *reinterpret_cast<const float2*>(x);
      o[0] += w * v.x; o[1] += w * v.y;
    }
  }
  if (lost) sum = __int_as_float(0x7fffffff);
  const float inv = sum > 0.f ? 1.f / sum : (sum == sum ? 0.f : sum);
  const long long token = token_of(p, item.x, item.z + row);
  const int qh = head_of(p, item.y, item.z + row);
  T* out = static_cast<T*>(p.out) + token * p.out_ld + (long long)qh * DIM + lane * kPer;
  uint32_t w[kPer / 2];
#pragma unroll
  for (int e = 0; e < kPer / 2; ++e) w[e] = pack2of<T>(o[2 * e] * inv, o[2 * e + 1] * inv);
  if constexpr (kPer == 4) *reinterpret_cast<uint2*>(out) = make_uint2(w[0], w[1]);
  else *reinterpret_cast<uint32_t*>(out) = w[0];
  if (p.lse && lane == 0) p.lse[token * p.q_heads + qh] = 0.69314718055994531f * (safe + log2f(sum));
}

}  // namespace attend
}  // namespace covspec
