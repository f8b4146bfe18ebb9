// Attention of few rows per key head (single tokens, drafted blocks) over the paged cache: one pass over the keys with running
// maxima and sums.  A tile is 16, 32 or 64 rows (16 a warp; the warps left of four share the keys of a unit) and 64 keys, 128 with
// 8-bit rows and up to 32 rows of queries.  The work is bound by reading the cache, so operands go to the tensor cores through
// registers (mma.sync): shared memory holds the pages' rows as they are in the cache, 8-bit ones are widened in registers.
//
// Warp 4 loads: tiled copies, a box as many rows of one head as a page has (at most a unit's), a box a lane, into a ring of units;
// it tells the others what each unit is, and where not every key is there it clears the values of the rest.  The others go from
// unit to unit each at its own pace and meet at the end of an item only.
//
// Measured (reading the cache once is the floor): 64 single tokens over e4m3 caches of 500-16384 positions, 32 query heads on 8 of 128:
// 138 us, 4.2 TB/s; blocks of 8 tokens over 32 bf16 caches of 300-4096, 28 heads on 4: 44 us, 2.0 TB/s; 24 prompt chunks of up to 700
// tokens over int8 caches, 14 heads on 2 of 64, window 1024: 321 us.  Bound by the chain of instructions of a warp from unit to unit
// (eight computing warps an SM; issue slots 40 % busy, HBM 50 % in the first of these), the last one by mma.sync's rate.
//
// 8-bit rows are exact in float16, so their scales stay outside the products: s_ij = (q_i . k_j) * key scale, and the probability
// takes the value's scale before it is rounded to 16 bits.  So that it cannot leave float16's range, the running maximum is the
// one of s_ij + lift_of(value's scale), whatever the scales are; sums of the probabilities alone may then be as large as 2^93 a key
// (rows of zeros) or as small as 2^-108, and go to a new reference in two steps.
#pragma once
#include <type_traits>

#include "attend_common.cuh"

namespace covspec {
namespace attend {

constexpr int kThreads = 160, kWarps = 4;        // threads of a CTA; its warps that compute
// Units that beginning and ending an item costs.  Without: 155 us for 138 with 64 single tokens over e4m3 caches, 45.2 for 44.0 with blocks
// of 8 tokens, 12.0 for 12.5 with one token over 900 positions (the share's units are counted item by item).
constexpr int kOpen = 2;

template <int STORE, int DIM, int ROWS> struct Layout {
  static constexpr bool k8 = STORE >= cache::kE4M3;
  static constexpr int kKeys = k8 && ROWS < 64 ? 128 : 64;     // of a unit
  static constexpr int kCtas = 2;                              // on an SM
  static constexpr int kRow = DIM * (k8 ? 1 : 2);              // bytes of a key's row
  static constexpr int kChunks = kRow / 16;
  static constexpr int kBlock = kRow < 128 ? kRow : 128;       // bytes of a row in a box; a row of 256 bytes has two
  static constexpr int kBoxes = 16 / (kRow / kBlock);          // of a unit at most: 16 lanes copy keys, 16 values
  static constexpr int kTile = kKeys * kRow;                   // keys, or values
  static constexpr int kScales = k8 ? 2 * kKeys * 4 : 0;       // the keys' and the values'
  static constexpr int kSay = 48;                              // what a unit is, which keys are there
  static constexpr int kStage = 2 * kTile;
  static constexpr int kFixed = 1024 + 256 + 2 * 16 * 8;       // alignment; barriers; maxima and sums of two warps' rows
  static constexpr int kFit = (233472 / kCtas - 1024 - 256 - kFixed) / (kStage + kScales + kSay);   // an SM's shared memory, 1 KB of it a CTA's own
  static constexpr int kStages = kFit < 6 ? kFit : 6;
  static constexpr int kSmem = kStages * (kStage + kScales + kSay) + kFixed;
  static_assert(kStages >= 2 && kKeys / 8 <= kBoxes && (ROWS == 64 || kStage >= 2 * 16 * DIM * 4));
};
// Byte offset of a 16-byte chunk of a row as the tiled copies leave it: chunks are permuted so that eight rows' chunks of one column
// lie in different banks.
template <int ROW, int KEYS> __device__ __forceinline__ int swizzled(int row, int chunk) {
  if constexpr (ROW >= 128) return (chunk >> 3) * (KEYS * 128) + row * 128 + (((chunk & 7) ^ (row & 7)) << 4);
  else return row * ROW + ((chunk ^ ((row >> 1) & 3)) << 4);
}

__device__ __forceinline__ void copy16(uint32_t dst, const void* src, bool there) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copies_close() { asm volatile("cp.async.commit_group;" ::: "memory"); }
__device__ __forceinline__ float ex2(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
// What a value's scale (not negative) adds to the reference: its exponent, near enough to its logarithm, less 13.  A probability times
// its scale is below 2^14 then, and float16 holds it in full down to 2^-27 of the row's largest.  No less than -80 for the exponent (also
// for NaN), so that the sum of 2^30 keys with values of zero stays finite; scales down to 2^-100 still give normal numbers.
__device__ __forceinline__ float lift_of(float x) {
  return __uint_as_float(0x4b000000u | (__float_as_uint(fmaxf(x, 8.271806125530277e-25f)) >> 23)) - (8388608.f + 127.f + 13.f);
}
template <int N> __device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

__device__ __forceinline__ void ldm4(uint32_t (&r)[4], uint32_t a) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(a));
}
__device__ __forceinline__ void ldm4t(uint32_t (&r)[4], uint32_t a) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(a));
}
template <typename T>
__device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  if constexpr (sizeof(T) == 2 && __is_same(T, __half))
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  else
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// Two 8-bit values (bytes `lo` and `hi` of a word) as two float16, exactly.  8-bit keys and values are multiplied in float16
// whatever the type of the queries: both widen to it in fewer instructions than to bfloat16, and probabilities keep three more
// bits.  Queries in bfloat16 are brought to float16 by a power of two for each row (to_half).
//  e4m3: the conversion instruction (half of the pairs by shifts and a product with 2^8 instead, exact too: 64 caches of 500-16384
//        positions, 8 heads of 128, 138 -> 160 us; all of K's 189).
//  int8: the byte becomes the lower bits of 1024 + (v + 128), and 1152 is taken off.
template <int STORE>
__device__ __forceinline__ uint32_t widen(uint32_t bytes, int lo, int hi) {
  uint32_t r;
  if constexpr (STORE == cache::kE4M3) {
    const uint32_t two = lo == 0 && hi == 1 ? bytes : __byte_perm(bytes, 0u, (uint32_t)(lo | hi << 4));
    asm("{\n.reg .b16 h;\ncvt.u16.u32 h, %1;\ncvt.rn.f16x2.e4m3x2 %0, h;\n}" : "=r"(r) : "r"(two));
  } else {
    const uint32_t w = __byte_perm(bytes ^ 0x80808080u, 0x64646464u, (uint32_t)(lo | 4 << 4 | hi << 8 | 4 << 12));
    asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(w), "r"(0x64806480u));
  }
  return r;
}
// The power of two that brings numbers of at most `top` below 2^15 (1 for zero and for what is not finite), and its inverse.
__device__ __forceinline__ float power_for(float top) {
  const int e = (int)(__float_as_uint(top) >> 23);
  return e == 0 || e == 255 ? 1.f : __uint_as_float((uint32_t)min(127 + 14 + 127 - e, 253) << 23);
}
__device__ __forceinline__ float inverse_power(float f) { return __uint_as_float((254u << 23) - __float_as_uint(f)); }
// Two bfloat16 as two float16, times f: exact but for numbers 2^-29 times as small as the row's largest.
__device__ __forceinline__ uint32_t to_half(uint32_t two, float f) {
  const __half2 h = __floats2half2_rn(__uint_as_float(two << 16) * f, __uint_as_float(two & 0xffff0000u) * f);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ float largest_of(uint32_t two, float top) {
  return fmaxf(top, fmaxf(fabsf(__uint_as_float(two << 16)), fabsf(__uint_as_float(two & 0xffff0000u))));
}

// What the loading warp tells the others of a unit: {first key, flags, first token of the request, head}, {first row of the item, rows of
// the request, position of its first token, units of the item behind this one}, which keys are there.
constexpr int kBegins = 1, kEnds = 2, kTwo = 4, kWholeStart = 8;   // first unit of its item in this share; last one of the item; more than
                                                                   // 128 rows; the item's first unit is in this share

__device__ __forceinline__ void tma_load_3d(uint32_t smem_dst, const CUtensorMap* map, int x, int y, int z, uint64_t* bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
      ::"r"(smem_dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(z), "r"(tc::smem_u32(bar))
      : "memory");
}
// A multiple of 16 bytes between 16-byte aligned addresses.
__device__ __forceinline__ void bulk_load(uint32_t smem_dst, const void* src, uint32_t bytes, uint64_t* bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
               ::"r"(smem_dst), "l"(src), "r"(bytes), "r"(tc::smem_u32(bar)) : "memory");
}
__device__ __forceinline__ void fence_async_proxy() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

template <typename T, int STORE, int DIM, int ROWS>
__global__ void __launch_bounds__(kThreads, (Layout<STORE, DIM, ROWS>::kCtas))
attend_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, const Params p) {
  using namespace tc;
  using L = Layout<STORE, DIM, ROWS>;
  constexpr bool k8 = L::k8;
  using M = std::conditional_t<k8, __half, T>;                 // type of the products
  constexpr int kKeys = L::kKeys;
  constexpr int kWarpsM = ROWS / 16, kWarpsK = kWarps / kWarpsM;   // warps along the rows, along the keys of a unit
  constexpr int kMine = kKeys / kWarpsK;                       // keys of a unit that one warp takes
  constexpr int kS = L::kStages;
  extern __shared__ char smem_raw[];
  char* smem = smem_raw + ((0u - smem_u32(smem_raw)) & 1023u);
  char* says = smem + kS * (L::kStage + L::kScales);           // [kS][kSay]
  float2* box_ts = reinterpret_cast<float2*>(says + kS * L::kSay);   // [2][16]
  uint64_t* bars = reinterpret_cast<uint64_t*>(box_ts + 2 * 16);
  uint64_t *full = bars, *empty = bars + 6, *partly = bars + 12, *met = bars + 13;
  volatile int* abort_flag = reinterpret_cast<volatile int*>(bars + 14);
  __shared__ long long scratch[kThreads / 32 + 4];
  const int tid = threadIdx.x, warp = warp_index(), lane = tid & 31;
  if (tid == 0) {
    for (int i = 0; i < kS; ++i) { mbar_init(full + i, 32); mbar_init(empty + i, kWarps * 32); }
    mbar_init(partly, 32);
    mbar_init(met, kWarps * 32);
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  wait_for_previous_kernel();
  const int share = blockIdx.x;
  Cursor<ROWS, kKeys> at;
  long long first, per;
  const int count = find_share<ROWS, kKeys, kThreads, kOpen>(p, at, first, per, scratch);
  if (tid == 0) p.open[2 * share + 1] = make_int4(-1, 0, 0, 0);
  if (count <= 0) {
    launch_dependents_now();
    return;
  }
  __syncthreads();

  if (warp == kWarps) {
    // ---------------- the loading warp ----------------
    const int mask = (1 << p.c.page_shift) - 1, shift = min(p.c.page_shift, kKeys == 128 ? 7 : 6), rows = 1 << shift, boxes = kKeys >> shift;
    const int kv = lane >> 4, box = lane & (L::kBoxes - 1), part = (lane & 15) / L::kBoxes;   // this lane's box of a unit
    int page = -1, stage = 0;
    auto look_up = [&] {                                       // its page in the unit at `at`
      const int key = at.key + (box << shift);
      page = box < boxes && key < at.k.hi && key + rows > at.k.lo ? p.t.table[at.b * p.t.table_ld + (key >> p.c.page_shift)] : -1;
      if ((unsigned)page >= (unsigned)p.c.pages) page = -1;
    };
    bool fresh = true, whole_start = false, loose = false;      // loose: copies under way that no unit has been handed over with
    uint32_t phase = 1, part_phase = 0;
    int filled = 0;                                            // units handed over
    look_up();
    for (int u = 0; u < count; ++u) {
      if (share == p.stop_share && u == p.stop_unit) break;
      if (fresh) whole_start = at.unit == 0;
      const int key0 = at.key, row0 = at.tile * ROWS;
      const bool ends = at.unit + 1 == at.units;
      const int4 say0 = make_int4(key0, (fresh ? kBegins : 0) | (ends ? kEnds : 0) | (whole_start ? kWholeStart : 0), at.r.q0, at.h);
      const int4 say1 = make_int4(row0, at.r.rows, at.r.first, at.units - 1 - at.unit);
      fresh = ends;
      const int page_row = (at.h << p.c.page_shift) + ((key0 + (box << shift)) & mask), box_page = page;
      uint32_t word[kKeys / 32], all = 0xffffffffu;
#pragma unroll
      for (int i = 0; i < kKeys / 32; ++i) {
        const int j = 32 * i + lane, has = __shfl_sync(0xffffffffu, page, j >> shift);
        word[i] = __ballot_sync(0xffffffffu, has >= 0 && key0 + j >= at.k.lo && key0 + j < at.k.hi);
        all &= word[i];
      }
      const bool mine = page >= 0;
      constexpr int kScaleBytes = k8 ? 4 : 0;
      // the first part's lane brings a box's scales too
      const uint32_t bytes = (uint32_t)__popc(__ballot_sync(0xffffffffu, mine)) * rows * (L::kBlock + kScaleBytes);
      if (u + 1 < count) {
        at.next(p);
        look_up();
      }
      if (!warp_wait(empty + stage, phase, abort_flag, p.polls)) break;
      char* base = smem + stage * L::kStage;
      float* sc = reinterpret_cast<float*>(smem + kS * L::kStage) + stage * 2 * kKeys;
      uint64_t* bar = all == 0xffffffffu ? full + stage : partly;
      if (lane == 0) {
        int4* say = reinterpret_cast<int4*>(says + stage * L::kSay);
        say[0] = say0;
        say[1] = say1;
        uint32_t* there = reinterpret_cast<uint32_t*>(say + 2);
#pragma unroll
        for (int i = 0; i < kKeys / 32; ++i) there[i] = word[i];
        mbar_expect_tx(bar, bytes);
      } else {
        mbar_arrive(bar);
      }
      __syncwarp();
      if (mine) {
        tma_load_3d(smem_u32(base + kv * L::kTile + part * (kKeys * 128) + (box << shift) * L::kBlock), kv ? &map_v : &map_k,
                    part * (L::kBlock / (L::kRow / DIM)), page_row, box_page, bar);
        if constexpr (k8)
          bulk_load(smem_u32(sc + kv * kKeys + (box << shift)), (kv ? p.c.v_scale : p.c.k_scale) + ((((long long)box_page * p.c.heads) << p.c.page_shift) + page_row),
                    rows * 4, bar);
      }
      if (all != 0xffffffffu) {                                // values of keys that are not there: zeros, whatever memory holds
        if ((loose = !warp_wait(partly, part_phase, abort_flag, p.polls))) break;
        part_phase ^= 1u;
#pragma unroll
        for (int i = 0; i < kKeys / 32; ++i)
          if (!((word[i] >> lane) & 1u)) {
            for (int c = 0; c < L::kChunks; ++c)
              *reinterpret_cast<uint4*>(base + L::kTile + swizzled<L::kRow, kKeys>(32 * i + lane, c)) = make_uint4(0u, 0u, 0u, 0u);
            if constexpr (k8) sc[kKeys + 32 * i + lane] = 0.f;
          }
        fence_async_proxy();                                   // before copies into the same place
        mbar_arrive(full + stage);
      }
      ++filled;
      if (++stage == kS) { stage = 0; phase ^= 1u; }
    }
    // copies under way end before their memory goes, whether or not the others are still there to wait for them
    if (lane == 0) {
      if (loose) drain(partly, part_phase);
      for (int i = 0; i < min(filled, kS); ++i) drain(full + i, i < stage ? phase ^ 1u : phase);
    }
    __syncwarp();
  } else {
    // ---------------- the computing warps ----------------
    const int wm = warp / kWarpsK, wk = warp % kWarpsK;
    const int g = lane >> 2, tq = lane & 3;
    uint32_t qf[DIM / 16][4];
    float o[DIM / 8][4], top[2], sum[2];
    int pos[2] = {-1, -1};        // position of the thread's two rows; -1 where there is no row
    [[maybe_unused]] float row_scale[2] = {p.scale_log2, p.scale_log2};
    int low = 0, high = 0;        // the lowest of them, the highest before the highest one's window
    int stage = 0;
    uint32_t phase = 0, met_phase = 0;
    int q0 = 0, h = 0, tile_row = 0;  // the item at hand
    auto meet = [&] {
      mbar_arrive(met);
      warp_wait(met, met_phase, abort_flag, p.polls);
      met_phase ^= 1u;
    };
    for (int u = 0; u < count; ++u) {
      if (!warp_wait(full + stage, phase, abort_flag, p.polls)) break;
      const int4* say = reinterpret_cast<const int4*>(says + stage * L::kSay);
      const uint32_t* there = reinterpret_cast<const uint32_t*>(say + 2);
      const int flags = say[0].y;
      if (flags & kBegins) {
        const int4 a = say[0], b = say[1];
        q0 = a.z;
        h = a.w;
        tile_row = b.x;
        low = 0x7fffffff;
        high = -0x7fffffff;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int r = tile_row + wm * 16 + g + 8 * i;
          const bool is = r < b.y;
          const int token = r / p.group;
          pos[i] = is ? b.z + token : -1;
          if (is) {
            low = min(low, pos[i]);
            high = max(high, pos[i] - p.window);
          }
          const T* q = static_cast<const T*>(p.q) + (is ? (long long)(q0 + token) * p.q_ld + (long long)(h * p.group + r - token * p.group) * DIM : 0);
#pragma unroll
          for (int s = 0; s < DIM / 16; ++s) {
            // the order of the products' inner index is free: 8-bit keys come as four neighbours a thread
            const uint32_t* w = reinterpret_cast<const uint32_t*>(q + 16 * s);
            qf[s][i] = is ? w[k8 ? 2 * tq : tq] : 0u;
            qf[s][2 + i] = is ? w[k8 ? 2 * tq + 1 : tq + 4] : 0u;
          }
          if constexpr (!__is_same(M, T)) {
            float most = 0.f;
#pragma unroll
            for (int s = 0; s < DIM / 16; ++s) most = largest_of(qf[s][2 + i], largest_of(qf[s][i], most));
            most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 1));
            most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 2));
            const float f = power_for(most);
#pragma unroll
            for (int s = 0; s < DIM / 16; ++s) { qf[s][i] = to_half(qf[s][i], f); qf[s][2 + i] = to_half(qf[s][2 + i], f); }
            row_scale[i] = p.scale_log2 * inverse_power(f);
          }
          top[i] = -INFINITY;
          sum[i] = 0.f;
        }
#pragma unroll
        for (int j = 0; j < DIM / 8; ++j) o[j][0] = o[j][1] = o[j][2] = o[j][3] = 0.f;
      }
      // ---- scores of this warp's keys ----
      const char* kbase = smem + stage * L::kStage;
      const char* vbase = kbase + L::kTile;
      float s[kMine / 8][4];
#pragma unroll
      for (int j = 0; j < kMine / 8; ++j) {
        s[j][0] = s[j][1] = s[j][2] = s[j][3] = 0.f;
        const int row = wk * kMine + j * 8 + (lane & 7);
#pragma unroll
        for (int c = 0; c < L::kChunks; c += 4) {
          uint32_t kf[4];
          ldm4(kf, smem_u32(kbase + swizzled<L::kRow, kKeys>(row, c + (lane >> 3))));
          if constexpr (k8) {
#pragma unroll
            for (int i = 0; i < 4; ++i) mma<M>(s[j], qf[c + i], widen<STORE>(kf[i], 0, 1), widen<STORE>(kf[i], 2, 3));
          } else {
            mma<M>(s[j], qf[c / 2], kf[0], kf[1]);
            mma<M>(s[j], qf[c / 2 + 1], kf[2], kf[3]);
          }
        }
      }
      // ---- running maxima and sums ----
      const float* sc = reinterpret_cast<const float*>(smem + kS * L::kStage) + stage * 2 * kKeys + wk * kMine;
      uint64_t see_all;                                          // of this warp's keys
      if constexpr (kMine == 64) see_all = *reinterpret_cast<const uint64_t*>(there + wk * 2);
      else see_all = there[wk * kMine / 32] >> (wk * kMine % 32);
      const int key0 = say[0].x + wk * kMine;
      // every row of the warp sees all of its keys
      const bool clear = (kMine == 64 ? see_all == ~0ull : (see_all & ((1ull << (kMine & 63)) - 1)) == (1ull << (kMine & 63)) - 1) &&
                         __all_sync(0xffffffffu, key0 + kMine - 1 <= low && (p.window == 0 || key0 > high));
      float best[2] = {top[0], top[1]};
#pragma unroll
      for (int j = 0; j < kMine / 8; ++j) {
        [[maybe_unused]] float by[2], lift[2];
        if constexpr (k8) {
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            by[i] = sc[j * 8 + 2 * tq + i];
            lift[i] = lift_of(sc[kKeys + j * 8 + 2 * tq + i]);
          }
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int col = j * 8 + 2 * tq + (e & 1), i = e >> 1;
          s[j][e] *= k8 ? by[e & 1] * row_scale[i] : p.scale_log2;
          if (!clear) {
            const int key = key0 + col;
            const bool see = (see_all >> col) & 1u && key <= pos[i] && (p.window == 0 || key > pos[i] - p.window);
            s[j][e] = see ? s[j][e] : -INFINITY;
          }
          best[i] = fmaxf(best[i], k8 ? s[j][e] + lift[e & 1] : s[j][e]);
        }
      }
      float safe[2], shrink[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        best[i] = fmaxf(best[i], __shfl_xor_sync(0xffffffffu, best[i], 1));
        best[i] = fmaxf(best[i], __shfl_xor_sync(0xffffffffu, best[i], 2));
        safe[i] = best[i] == -INFINITY ? 0.f : best[i];
        if constexpr (k8) {                                      // a reference may rise by more than 2^126
          const float part = ex2(0.5f * (top[i] - safe[i]));
          shrink[i] = part * part;
          sum[i] = sum[i] * part * part;
        } else {
          shrink[i] = ex2(top[i] - safe[i]);
          sum[i] *= shrink[i];
        }
        top[i] = best[i];
      }
      if (__any_sync(0xffffffffu, shrink[0] != 1.f || shrink[1] != 1.f)) {
#pragma unroll
        for (int j = 0; j < DIM / 8; ++j) { o[j][0] *= shrink[0]; o[j][1] *= shrink[0]; o[j][2] *= shrink[1]; o[j][3] *= shrink[1]; }
      }
      uint32_t pf[kMine / 16][4];
#pragma unroll
      for (int j = 0; j < kMine / 8; ++j) {
        float e[4];
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          e[x] = ex2(s[j][x] - safe[x >> 1]);
          sum[x >> 1] += e[x];
          if constexpr (k8) e[x] *= sc[kKeys + j * 8 + 2 * tq + (x & 1)];
        }
        pf[j / 2][(j & 1) * 2] = pack2of<M>(e[0], e[1]);
        pf[j / 2][(j & 1) * 2 + 1] = pack2of<M>(e[2], e[3]);
      }
      // ---- values ----
#pragma unroll
      for (int s16 = 0; s16 < kMine / 16; ++s16) {
        const int row0 = wk * kMine + s16 * 16;
        if constexpr (k8) {
#pragma unroll
          for (int c = 0; c < L::kChunks; c += 2) {              // 32 features: chunks c, c + 1 of the 16 keys
            uint32_t vf[4];                                      // [chunk][keys 0-7, 8-15]
            ldm4t(vf, tc::smem_u32(vbase + swizzled<L::kRow, kKeys>(row0 + (lane & 15), c + (lane >> 4))));
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              // a register holds features 2n, 2n + 1 of two keys: the even ones make one tile of eight columns, the odd ones another
              mma<M>(o[2 * (c + h)], pf[s16], widen<STORE>(vf[2 * h], 0, 2), widen<STORE>(vf[2 * h + 1], 0, 2));
              mma<M>(o[2 * (c + h) + 1], pf[s16], widen<STORE>(vf[2 * h], 1, 3), widen<STORE>(vf[2 * h + 1], 1, 3));
            }
          }
        } else {
#pragma unroll
          for (int c = 0; c < L::kChunks; c += 2) {
            uint32_t vf[4];
            ldm4t(vf, tc::smem_u32(vbase + swizzled<L::kRow, kKeys>(row0 + (lane & 15), c + (lane >> 4))));
            mma<M>(o[c], pf[s16], vf[0], vf[1]);
            mma<M>(o[c + 1], pf[s16], vf[2], vf[3]);
          }
        }
      }
      // ---- the item's end, or the share's ----
      const bool last = flags & kEnds;
      if (last || u + 1 == count) {
        const int4 b = say[1];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          sum[i] += __shfl_xor_sync(0xffffffffu, sum[i], 1);
          sum[i] += __shfl_xor_sync(0xffffffffu, sum[i], 2);
        }
        // warps that shared the keys: the upper half hands its rows to the lower one, until one has all; through the unit's own
        // stage, which is not given back before
#pragma unroll
        for (int half = kWarpsK / 2; half > 0; half >>= 1) {
          meet();
          const int which = kWarpsK == 4 ? (wk & (half - 1)) : wm;
          float* box = reinterpret_cast<float*>(smem + stage * L::kStage) + which * 16 * DIM;
          if (wk >= half && wk < 2 * half) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              float* x = box + (g + 8 * i) * DIM;
#pragma unroll
              for (int j = 0; j < DIM / 8; ++j) *reinterpret_cast<float2*>(x + ((j ^ g) * 8 + 2 * tq)) = make_float2(o[j][2 * i], o[j][2 * i + 1]);
              if (tq == 0) box_ts[which * 16 + g + 8 * i] = make_float2(top[i], sum[i]);
            }
          }
          meet();
          if (wk < half) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              const float* x = box + (g + 8 * i) * DIM;
              const float2 ts = box_ts[which * 16 + g + 8 * i];
              const float both = fmaxf(top[i], ts.x), ref = both == -INFINITY ? 0.f : both;
              constexpr float kHalf = k8 ? 0.5f : 1.f;
              float a = ex2(kHalf * (top[i] - ref)), c = ex2(kHalf * (ts.x - ref));
              top[i] = both;
              if constexpr (k8) {
                sum[i] = sum[i] * a * a + ts.y * c * c;
                a *= a;
                c *= c;
              } else {
                sum[i] = sum[i] * a + ts.y * c;
              }
#pragma unroll
              for (int j = 0; j < DIM / 8; ++j) {
                const float2 v = *reinterpret_cast<const float2*>(x + ((j ^ g) * 8 + 2 * tq));
                o[j][2 * i] = o[j][2 * i] * a + v.x * c;
                o[j][2 * i + 1] = o[j][2 * i + 1] * a + v.y * c;
              }
            }
          }
        }
        if (kWarpsK > 1) fence_async_proxy();                  // before copies into the same place
        const bool whole = last && (flags & kWholeStart);
        if (wk == 0) {
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const int in = wm * 16 + g + 8 * i, r = tile_row + in;
            if (r < b.y) {
              if (whole) {
                const float inv = sum[i] > 0.f ? 1.f / sum[i] : (sum[i] == sum[i] ? 0.f : sum[i]);
                const long long token = token_of(p, q0, r);
                const int qh = head_of(p, h, r);
                T* out = static_cast<T*>(p.out) + token * p.out_ld + (long long)qh * DIM;
                if constexpr (k8) {
#pragma unroll
                  for (int j = 0; j < DIM / 8; j += 2)
                    *reinterpret_cast<uint2*>(out + j * 8 + 4 * tq) = make_uint2(pack2of<T>(o[j][2 * i] * inv, o[j + 1][2 * i] * inv),
                                                                                pack2of<T>(o[j][2 * i + 1] * inv, o[j + 1][2 * i + 1] * inv));
                } else {
#pragma unroll
                  for (int j = 0; j < DIM / 8; ++j)
                    *reinterpret_cast<uint32_t*>(out + j * 8 + 2 * tq) = pack2of<T>(o[j][2 * i] * inv, o[j][2 * i + 1] * inv);
                }
                if (p.lse && tq == 0)
                  p.lse[token * p.q_heads + qh] = 0.69314718055994531f * ((top[i] == -INFINITY ? 0.f : top[i]) + log2f(sum[i]));
              } else {
                float* slot = p.part + (2 * share + ((flags & kWholeStart) != 0)) * (long long)(ROWS * (DIM + 2));
                float* x = slot + in * DIM;
                if constexpr (k8) {
#pragma unroll
                  for (int j = 0; j < DIM / 8; j += 2)
                    *reinterpret_cast<float4*>(x + j * 8 + 4 * tq) = make_float4(o[j][2 * i], o[j + 1][2 * i], o[j][2 * i + 1], o[j + 1][2 * i + 1]);
                } else {
#pragma unroll
                  for (int j = 0; j < DIM / 8; ++j) *reinterpret_cast<float2*>(x + j * 8 + 2 * tq) = make_float2(o[j][2 * i], o[j][2 * i + 1]);
                }
                if (tq == 0) {
                  slot[ROWS * DIM + in] = top[i];
                  slot[ROWS * (DIM + 1) + in] = sum[i];
                }
              }
            }
          }
        }
        if (u + 1 == count && tid == 0) {
          const bool open = !last && (flags & kWholeStart);
          p.open[2 * share] = make_int4(q0, h, tile_row, min(ROWS, b.y - tile_row));
          p.open[2 * share + 1].x = open ? (int)((first + per + b.w - 1) / per) : -1;
        }
      }
      mbar_arrive(empty + stage);
      if (++stage == kS) { stage = 0; phase ^= 1u; }
    }
  }
  if (lane == 0 && *abort_flag) p.open[2 * share + 1].y = 1;
  launch_dependents_now();
}

}  // namespace attend
}  // namespace covspec
