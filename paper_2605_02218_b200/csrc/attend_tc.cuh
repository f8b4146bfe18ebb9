// Attention of many rows per key head (chunks of prompts, large blocks) over the paged cache on the tensor cores (tcgen05).
//
// An item is 256 rows of one key head, two tiles of 128 that take turns: while the softmax of one tile runs, the tensor core
// multiplies for the other.  A unit is 128 keys.  TMEM holds S (scores, 128 columns) and O (the rows, `DIM` columns) of both
// tiles; the probabilities overwrite S in 16 bits and are the A operand of the second product from there.  Keys are K-major, values
// MN-major (keys are the inner dimension of the second product), both as rows of 64 features in 128-byte swizzled tiles.
//
// Warps: 0-7 and 8-15 softmax of tile 0 and 1, a row of it two threads in two warps, each half of a unit's keys; a thread of 16
// issues the products (with its warp's other lanes waiting along: 655 us for 668 in the case below, but they arrive nowhere and so could
// be left behind at a wait); 17-19 bring queries, and 17 keys and values, into shared memory: tiled copies, a box as many rows as a page has (at most
// 128), a box a lane.  Where not every key of a unit is there, the values' other rows are cleared before the products may see them.
//
// The running maximum is only a reference that keeps the exponentials in range: a row keeps it
// while a unit's probabilities add up to at most 2^14, so that O is rescaled seldom and one pass over S makes the probabilities.  A
// warp with a row beyond that goes over S again with new references.
//
// 16-bit caches only: 8-bit rows would have to be widened into shared memory first.  The form of this kernel that did so stood still on a
// large call; its waits were of the kind that warp_wait (attend_common.cuh) says of what happened to them.  8-bit caches take the kernel
// for few rows.
//
// Measured: 8 prompts of 2048 tokens over caches of 2048-4096, 32 heads on 8 of 128, bf16: 665-690 us, 0.71-0.73 PFLOP/s (with mma.sync
// 2756).  An SM has 204 units and takes 5200 cycles for one, beginnings and ends of items included: 2330 of products (16 of 128 x 128 x 16
// for each of the two factors; the two tiles' operands take all of shared memory's bandwidth), in the rest the products wait for
// probabilities: 32768 exponentials are 2048 cycles of the special-function units, and the two tiles overlap in part only.
#pragma once
#include "attend_call.cuh"
#include "attend_kernels.cuh"

namespace covspec {
namespace attend {
namespace wide {

using namespace tc;

constexpr int kRows = kWideRows, kKeys = kWideKeys;
constexpr int kThreads = 20 * 32, kSoftmaxWarps = 16;
constexpr int kCopyWarps = 3, kProducers = kCopyWarps * 32;
constexpr int kOpen = 4;                    // units that beginning and ending an item costs (8 prompts of 2048 tokens: 740 us without, 685)
constexpr float kMost = 16384.f;            // a unit's probabilities add up to no more over their reference

template <int STORE, int DIM> struct Layout {
  static_assert(STORE < cache::kE4M3);
  static constexpr int kSlot = kKeys * DIM * 2;                // keys or values of a unit, 16-bit
  static constexpr int kQ = kRows * DIM * 2;
  static constexpr int kSlots = 5;
  static constexpr int kTail = 4 * 16 + 4 * 32                 // which keys of a unit are there, its item; 4 units
                               + 256 + 2 * 128 * 4;            // barriers, TMEM base; exchange, first the scratch of find_share
  static constexpr int kUsed = kQ + kSlots * kSlot + kTail;
  static constexpr int kSmem = kUsed > 120 * 1024 ? kUsed : 120 * 1024;      // one CTA an SM: each takes all of TMEM
  static_assert(kSmem <= 232448);
};

template <typename T> __device__ __forceinline__ uint32_t idesc(int n, bool b_mn) {
  const uint32_t type = __is_same(T, __half) ? 0u : 1u;
  return (1u << 4) | (type << 7) | (type << 10) | ((b_mn ? 1u : 0u) << 16) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);
}
// Values: 64 features of a key are a 128-byte row, eight keys a swizzled block, the next 64 features `kKeys` rows on.
__device__ __forceinline__ uint64_t desc_mn(uint32_t smem_addr) {
  uint64_t d = 0;
  d |= (uint64_t)((smem_addr & 0x3FFFFu) >> 4);
  d |= (uint64_t)((kKeys * 128u) >> 4) << 16;
  d |= (uint64_t)(1024u >> 4) << 32;
  d |= (uint64_t)1 << 46;
  d |= (uint64_t)2 << 61;
  return d;
}
__device__ __forceinline__ void mma_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n"
      ".reg .pred p;\n"
      "setp.ne.b32 p, %4, 0;\n"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n"
      "}\n" ::"r"(d_tmem), "r"(a_tmem), "l"(bdesc), "r"(idesc), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ void tmem_st32(uint32_t taddr, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
      "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
      "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};"
      ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
      "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]),
      "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]),
      "r"(r[30]), "r"(r[31])
      : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

__device__ __forceinline__ f32x2 add2(f32x2 a, f32x2 b) {
  f32x2 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
      ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
      "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}

// Barriers among `n` threads.  Not the aligned forms: those want the warp's lanes together, which nothing after a branch on the lane
// promises.
__device__ __forceinline__ void meet_at(int id, int n) {
  __syncwarp();
  asm volatile("barrier.cta.sync %0, %1;" ::"r"(id), "r"(n) : "memory");
}
// It tells each whether all came with `v`, ...
__device__ __forceinline__ bool barrier_and(int id, int n, bool v) {
  uint32_t r;
  __syncwarp();
  asm volatile(
      "{\n"
      ".reg .pred p, q;\n"
      "setp.ne.u32 p, %3, 0;\n"
      "barrier.cta.red.and.pred q, %1, %2, p;\n"
      "selp.u32 %0, 1, 0, q;\n"
      "}\n"
      : "=r"(r) : "r"(id), "r"(n), "r"((uint32_t)v) : "memory");
  return r != 0;
}

// ... whether one did.
__device__ __forceinline__ bool barrier_or(int id, int n, bool v) {
  uint32_t r;
  __syncwarp();
  asm volatile(
      "{\n"
      ".reg .pred p, q;\n"
      "setp.ne.u32 p, %3, 0;\n"
      "barrier.cta.red.or.pred q, %1, %2, p;\n"
      "selp.u32 %0, 1, 0, q;\n"
      "}\n"
      : "=r"(r) : "r"(id), "r"(n), "r"((uint32_t)v) : "memory");
  return r != 0;
}

// Byte offset of a 16-byte chunk of row `row`, 64 features a block of `rows` rows.
__device__ __forceinline__ int tile_at(int rows, int row, int chunk) {
  return (chunk >> 3) * rows * 128 + row * 128 + (((chunk & 7) ^ (row & 7)) << 4);
}

template <typename T, int STORE, int DIM>
__global__ void __launch_bounds__(kThreads, 1)
attend_wide_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, const Params p) {
  using L = Layout<STORE, DIM>;
  constexpr int kSlots = L::kSlots;
  extern __shared__ __align__(1024) uint8_t wide_smem[];
  uint8_t* smem = wide_smem;
  uint8_t* ring = smem + L::kQ;
  uint8_t* tail = ring + kSlots * L::kSlot;
  uint32_t* there = reinterpret_cast<uint32_t*>(tail);                       // [4][4]
  int4* units = reinterpret_cast<int4*>(tail + 64);                          // [4][2], see below
  uint64_t* bars = reinterpret_cast<uint64_t*>(tail + 192);
  float* exchange = reinterpret_cast<float*>(bars + 32);                     // [2][128]: between the two threads of a row
  uint64_t *full = bars, *empty = bars + 5, *q_full = bars + 10, *q_empty = bars + 11, *s_full = bars + 12, *p_ready = bars + 14,
           *o_full = bars + 16, *drained = bars + 18, *partly = bars + 19;   // 20 barriers
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 20);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  const int tid = threadIdx.x, warp = warp_index(), lane = tid & 31;
  if (tid == 0) {
    for (int i = 0; i < kSlots; ++i) { mbar_init(full + i, 32); mbar_init(empty + i, 1); }
    mbar_init(q_full, kProducers);
    mbar_init(q_empty, 1);
    for (int i = 0; i < 2; ++i) { mbar_init(s_full + i, 1); mbar_init(p_ready + i, 8 * 32); mbar_init(o_full + i, 1); }
    mbar_init(drained, 1);
    mbar_init(partly, 32);
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  wait_for_previous_kernel();
  Cursor<kRows, kKeys> at;
  long long first, per;
  const int count = find_share<kRows, kKeys, kThreads, kOpen>(p, at, first, per, reinterpret_cast<long long*>(exchange));
  const int share = blockIdx.x;
  if (tid == 0) p.open[2 * share + 1] = make_int4(-1, 0, 0, 0);
  if (count <= 0) {
    launch_dependents_now();
    return;
  }
  if (warp == kSoftmaxWarps) tmem_alloc(tmem_slot, 512);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  constexpr uint32_t kO = 256;                                 // first column of O; tile x: S at 128 x, O at kO + 128 x

  if (warp > kSoftmaxWarps) {
    // ---------------- producers ----------------
    const int wp = warp - kSoftmaxWarps - 1;
    int slot = 0;
    uint32_t phase = 1, q_phase = 1;
    bool fresh = true, loose = false;                          // loose: copies under way in a slot that has not been handed over
    int filled = 0;                                            // slots handed over
    auto next_slot = [&] { ++filled; if (++slot == kSlots) { slot = 0; phase ^= 1u; } };
    auto queries = [&] {                                       // of the item at `at`; false: a wait gave up
      if (!warp_wait(q_empty, q_phase, abort_flag, p.polls)) return false;
      q_phase ^= 1u;
      constexpr int kChunks = DIM / 8, kAtOnce = 32 / kChunks, kStep = kCopyWarps * kAtOnce;
      const int chunk = lane % kChunks;
      // token and query head of row r, and how far they go on from one of this thread's rows to the next
      int row = wp * kAtOnce + lane / kChunks;
      int token = (at.tile * kRows + row) / p.group, head = at.tile * kRows + row - token * p.group;
      const int step_token = kStep / p.group, step_head = kStep - step_token * p.group, rows = at.r.rows - at.tile * kRows;
      const T* q0 = static_cast<const T*>(p.q) + at.r.q0 * p.q_ld + (long long)at.h * p.group * DIM + chunk * 8;
#pragma unroll 4
      for (int i = 0; i < (kRows + kStep - 1) / kStep; ++i, row += kStep) {
        const bool in = row < kRows, is = row < min(rows, kRows);
        const T* q = is ? q0 + token * p.q_ld + head * DIM : q0;
        token += step_token;
        head += step_head;
        if (head >= p.group) { head -= p.group; ++token; }
        uint8_t* to = smem + (row >> 7) * (128 * DIM * 2) + tile_at(128, row & 127, chunk);
        if (in) copy16(smem_u32(to), q, is);
      }
      copies_close();
      copies_wait<0>();
      fence_async_proxy();
      mbar_arrive(q_full);
      return true;
    };
    {
      if (wp > 0) {                                            // these two only help with the queries
        for (int u = 0; u < count; ++u) {
          if (fresh && !queries()) break;
          fresh = at.unit + 1 == at.units;
          if (u + 1 < count) at.next(p);
        }
      } else {
        const int mask = (1 << p.c.page_shift) - 1, shift = min(p.c.page_shift, 7), rows = 1 << shift, boxes = kKeys >> shift;
        const int box = lane & 15, part = lane >> 4;           // this lane's box of a unit, and which 64 features of it
        int page = -1;
        auto look_up_box = [&] {                               // page of the box in the unit at `at`
          const int key = at.key + (box << shift);
          page = box < boxes && key < at.k.hi && key + rows > at.k.lo ? p.t.table[at.b * p.t.table_ld + (key >> p.c.page_shift)] : -1;
          if ((unsigned)page >= (unsigned)p.c.pages) page = -1;
        };
        bool whole_start = false;
        uint32_t part_phase = 0;
        look_up_box();
        for (int u = 0; u < count; ++u) {
          if (share == p.stop_share && u == p.stop_unit) break;
          const bool begins = fresh;
          if (begins) {
            if (!queries()) break;
            whole_start = at.unit == 0;
          }
          const int row0 = at.tile * kRows, key0 = at.key, page_row = (at.h << p.c.page_shift) + ((key0 + (box << shift)) & mask);
          fresh = at.unit + 1 == at.units;
          const int4 item[2] = {make_int4(key0, (begins ? kBegins : 0) | (fresh ? kEnds : 0) | (at.r.rows - row0 > 128 ? kTwo : 0) | (whole_start ? kWholeStart : 0), at.r.q0, at.h),
                                make_int4(row0, at.r.rows, at.r.first, at.units - 1 - at.unit)};
          const bool mine = page >= 0 && part < DIM / 64;
          const int box_page = page;
          uint32_t word[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int j = 32 * i + lane;
            const int has = __shfl_sync(0xffffffffu, page, j >> shift);
            word[i] = __ballot_sync(0xffffffffu, has >= 0 && key0 + j >= at.k.lo && key0 + j < at.k.hi);
          }
          const uint32_t bytes = (uint32_t)__popc(__ballot_sync(0xffffffffu, mine)) * rows * 128;
          if (u + 1 < count) {
            at.next(p);
            look_up_box();
          }
          // the words of unit u - 4 have been read: its products are done (the slot that this unit's keys take says so)
          if (!warp_wait(empty + slot, phase, abort_flag, p.polls)) break;
          if (lane == 0) {
            *reinterpret_cast<uint4*>(there + (u & 3) * 4) = make_uint4(word[0], word[1], word[2], word[3]);
            units[(u & 3) * 2] = item[0];
            units[(u & 3) * 2 + 1] = item[1];
            mbar_expect_tx(full + slot, bytes);
          } else {
            mbar_arrive(full + slot);
          }
          __syncwarp();
          if (mine) tma_load_3d(smem_u32(ring + slot * L::kSlot) + part * (kKeys * 128) + (box << shift) * 128, &map_k, part * 64, page_row, box_page, full + slot);
          next_slot();
          if (!warp_wait(empty + slot, phase, abort_flag, p.polls)) break;
          const bool all = (word[0] & word[1] & word[2] & word[3]) == 0xffffffffu;
          uint64_t* bar = all ? full + slot : partly;
          if (lane == 0) mbar_expect_tx(bar, bytes);
          else mbar_arrive(bar);
          __syncwarp();
          if (mine) tma_load_3d(smem_u32(ring + slot * L::kSlot) + part * (kKeys * 128) + (box << shift) * 128, &map_v, part * 64, page_row, box_page, bar);
          if (!all) {                                          // values of keys that are not there: zeros, whatever memory holds
            if ((loose = !warp_wait(partly, part_phase, abort_flag, p.polls))) break;
            part_phase ^= 1u;
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (!((word[i] >> lane) & 1u))
                for (int c = 0; c < DIM / 8; ++c)
                  *reinterpret_cast<uint4*>(ring + slot * L::kSlot + (c >> 3) * (kKeys * 128) + (32 * i + lane) * 128 + (c & 7) * 16) = make_uint4(0u, 0u, 0u, 0u);
            fence_async_proxy();
            mbar_arrive(full + slot);
          }
          next_slot();
        }
        // copies under way end before their memory goes, whether or not the others are still there to wait for them
        if (lane == 0) {
          if (loose) drain(partly, part_phase);
          for (int i = 0; i < min(filled, kSlots); ++i) drain(full + i, i < slot ? phase ^ 1u : phase);
        }
        __syncwarp();
      }
    }
  } else if (warp == kSoftmaxWarps) {
    // ---------------- products ----------------
    if (lane == 0) {
      const uint32_t qk = idesc<T>(kKeys, false), pv = idesc<T>(DIM, true);
      int slot = 0;
      uint32_t phase = 0, q_phase = 0, p_phase = 0;
      bool ok = true;
      auto next_slot = [&] { if (++slot == kSlots) { slot = 0; phase ^= 1u; } };
      auto wait = [&](uint64_t* bar, uint32_t parity) { return ok = ok && mbar_wait_limited(bar, parity, abort_flag, p.polls); };
      auto scores = [&](int x, int s) {
        const uint32_t a0 = smem_u32(smem + x * (128 * DIM * 2)), b0 = smem_u32(ring + s * L::kSlot);
#pragma unroll
        for (int h = 0; h < DIM / 64; ++h) {
          const uint64_t a = umma_desc(a0 + h * 128 * 128), b = umma_desc(b0 + h * kKeys * 128);
#pragma unroll
          for (int k = 0; k < 4; ++k) umma_bf16(tmem + x * 128, a + 2 * k, b + 2 * k, qk, (h | k) != 0);
        }
      };
      auto rows = [&](int x, int s, bool accumulate) {
        const uint64_t b = desc_mn(smem_u32(ring + s * L::kSlot));
#pragma unroll
        for (int k = 0; k < kKeys / 16; ++k)
          mma_ts(tmem + kO + x * 128, tmem + x * 128 + 8 * k, b + k * (16 * 128 / 16), pv, accumulate || k != 0);
      };
      bool opened = false;                                     // the unit's scores are issued
      for (int u = 0; u < count && ok; ++u) {
        if (!opened) {                                         // it begins an item here
          if (!wait(q_full, q_phase) || !wait(full + slot, phase)) break;
          q_phase ^= 1u;
          tc_fence_after();
          scores(0, slot);
          umma_commit(s_full);
          if (units[(u & 3) * 2].y & kTwo) scores(1, slot);
          umma_commit(s_full + 1);                             // also without rows: the warps of the tile go from unit to unit
          umma_commit(empty + slot);
          next_slot();
        }
        const int flags = units[(u & 3) * 2].y;
        const bool two = flags & kTwo, more = u + 1 < count && !(flags & kEnds);
        if (!more) umma_commit(q_empty);
        const int v_slot = slot;
        if (!wait(full + v_slot, phase)) break;
        next_slot();
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          if (!wait(p_ready + x, p_phase) || (x == 0 && more && !wait(full + slot, phase))) break;
          tc_fence_after();
          if (x == 0 || two) {
            rows(x, v_slot, !(flags & kBegins));
            if (!more) umma_commit(o_full + x);
          }
          if (x == 1) umma_commit(empty + v_slot);
          if (more) {
            if (x == 0 || two) scores(x, slot);
            umma_commit(s_full + x);
          }
        }
        p_phase ^= 1u;
        if (more && ok) {
          umma_commit(empty + slot);
          next_slot();
        }
        opened = more;
      }
      // TMEM and the ring are free when every product has ended, also after a wait that gave up
      umma_commit(drained);
      drain(drained, 0);
    }
    __syncwarp();
  } else {
    // ---------------- softmax ----------------
    // tile, which half of the keys (and of the features of O), row
    const int x = warp >> 3, half = (warp >> 2) & 1, row = tid & 127, pair = 2 + x * 4 + (warp & 3);
    const uint32_t lanes = (uint32_t)(warp & 3) << 21;
    const uint32_t s_at = tmem + lanes + x * 128, o_at = tmem + lanes + kO + x * 128 + half * (DIM / 2);
    float* shared = exchange + x * 128 + row;
    float ref = 0.f, sum = 0.f;
    int pos = -1;                                              // position of the row's token
    bool active = false;
    uint32_t s_phase = 0, o_phase = 0;
    for (int u = 0; u < count; ++u) {
      // the two warps of a row go on or give up together: they meet at barriers further down
      if (!barrier_and(pair, 64, warp_wait(s_full + x, s_phase, abort_flag, p.polls))) break;
      s_phase ^= 1u;
      tc_fence_after();
      __syncwarp();
      const int key = units[(u & 3) * 2].x, flags = units[(u & 3) * 2].y;
      if (flags & kBegins) {
        const int4 item = units[(u & 3) * 2 + 1];
        const int r = item.x + x * 128 + row;
        active = x == 0 || (flags & kTwo);
        const bool is = r < item.y;
        pos = is ? item.z + r / p.group : 0x7fffffff;          // no row: nothing to mask, no reference to look for
        ref = is ? -INFINITY : 0.f;
        sum = 0.f;
      }
      if (!active) {
        mbar_arrive(p_ready + x);
      } else {
        const uint4 bits = *reinterpret_cast<const uint4*>(there + (u & 3) * 4);
        // every row of the warp sees all keys of the unit
        const bool clear = (bits.x & bits.y & bits.z & bits.w) == 0xffffffffu &&
                           __all_sync(0xffffffffu, key + kKeys - 1 <= pos && (p.window == 0 || pos == 0x7fffffff || key > pos - p.window));
        const int lowest = p.window && pos != 0x7fffffff ? max(pos - p.window + 1, 0) : 0;
        // bits of 32 keys of this half that the row sees
        auto seen = [&](int c) {
          const int k0 = key + 64 * half + 32 * c;
          uint32_t see = half == 0 ? (c == 0 ? bits.x : bits.y) : (c == 0 ? bits.z : bits.w);
          see &= pos < k0 ? 0u : pos - k0 >= 31 ? 0xffffffffu : (2u << (pos - k0)) - 1u;
          see &= lowest <= k0 ? 0xffffffffu : lowest - k0 > 31 ? 0u : ~((1u << (lowest - k0)) - 1u);
          return see;
        };
        uint32_t packed[32];
        float more;                                            // sum of the probabilities
        bool renew = __any_sync(0xffffffffu, ref == -INFINITY);  // the same in both halves
        for (;;) {
          if (renew) {                                         // new references, from the scores themselves
            float best = ref;
#pragma unroll 1
            for (int c = 0; c < 4; ++c) {
              float v[16];
              tmem_ld16(s_at + 64 * half + 16 * c, v);
              const uint32_t see = seen(c / 2) >> (16 * (c & 1));
#pragma unroll
              for (int e = 0; e < 16; ++e) {
                best = (see >> e) & 1u ? fmaxf(best, v[e] * p.scale_log2) : best;
              }
            }
            if (half) *shared = best;
            meet_at(pair, 64);
            if (!half) *shared = best = fmaxf(best, *shared);
            meet_at(pair, 64);
            if (half) best = *shared;
            const float shrink = ref == -INFINITY ? 0.f : ex2(ref - best);
            ref = best;
            sum *= shrink;
            if (!(flags & kBegins)) {                          // O holds earlier units' rows
#pragma unroll 1
              for (int c = 0; c < DIM / 32; ++c) {
                float v[16];
                tmem_ld16(o_at + 16 * c, v);
                uint32_t w[16];
#pragma unroll
                for (int e = 0; e < 16; ++e) w[e] = __float_as_uint(v[e] * shrink);
                tmem_st16(o_at + 16 * c, w);
              }
              tmem_st_wait();
            }
          }
          const float safe = ref == -INFINITY ? 0.f : ref;
          __syncwarp();
          const f32x2 low = pack2(-safe, -safe), by = pack2(p.scale_log2, p.scale_log2);
          f32x2 sum2[2] = {pack2(0.f, 0.f), pack2(0.f, 0.f)};
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            float v[32];
            tmem_ld32(s_at + 64 * half + 32 * c, v);
#pragma unroll
            for (int e = 0; e < 32; e += 2) {
              const float2 t = unpack2(fma2(pack2(v[e], v[e + 1]), by, low));
              v[e] = t.x;
              v[e + 1] = t.y;
            }
            if (!clear) {
              const uint32_t see = seen(c);
#pragma unroll
              for (int e = 0; e < 32; ++e) v[e] = (see >> e) & 1u ? v[e] : -INFINITY;
            }
#pragma unroll
            for (int e = 0; e < 32; e += 2) {
              const float x = ex2(v[e]), y = ex2(v[e + 1]);
              sum2[e / 2 & 1] = add2(sum2[e / 2 & 1], pack2(x, y));
              packed[16 * c + e / 2] = pack2of<T>(x, y);
            }
          }
          const float2 a = unpack2(add2(sum2[0], sum2[1]));
          more = a.x + a.y;
          // both halves of the rows alike; and both have read their scores, over which the probabilities are written
          const bool over = barrier_or(pair, 64, more > kMost);
          if (renew || !over) break;
          renew = true;
        }
        sum += more;
        __syncwarp();
        tmem_st32(s_at + 32 * half, packed);
        tmem_st_wait();
        tc_fence_before();
        mbar_arrive(p_ready + x);
      }
      if ((flags & kEnds) || u + 1 == count) {
        const int4 item = units[(u & 3) * 2 + 1];
        const bool whole = (flags & kEnds) && (flags & kWholeStart);
        const int q0 = units[(u & 3) * 2].z, h = units[(u & 3) * 2].w;
        if (active) {
          warp_wait(o_full + x, o_phase, abort_flag, p.polls); // both warps of a row go on, whatever it says
          o_phase ^= 1u;
          tc_fence_after();
          const int r = item.x + x * 128 + row;
          const bool is = r < item.y;
          float total = sum;
          if (half) *shared = sum;
          meet_at(pair, 64);
          if (!half) *shared = total = sum + *shared;
          meet_at(pair, 64);
          if (half) total = *shared;
          const float inv = total > 0.f ? 1.f / total : (total == total ? 0.f : total);
          const long long token = is ? token_of(p, q0, r) : 0;
          const int qh = is ? head_of(p, h, r) : 0;
          T* out = static_cast<T*>(p.out) + token * p.out_ld + (long long)qh * DIM + half * (DIM / 2);
          float* slot = p.part + (2 * share + ((flags & kWholeStart) != 0)) * (long long)(kRows * (DIM + 2));
          const int in = x * 128 + row;
#pragma unroll 1
          for (int c = 0; c < DIM / 64; ++c) {
            float v[32];
            tmem_ld32(o_at + 32 * c, v);
            if (is && whole) {
#pragma unroll
              for (int e = 0; e < 32; e += 8)
                *reinterpret_cast<uint4*>(out + 32 * c + e) = make_uint4(pack2of<T>(v[e] * inv, v[e + 1] * inv), pack2of<T>(v[e + 2] * inv, v[e + 3] * inv),
                                                                         pack2of<T>(v[e + 4] * inv, v[e + 5] * inv), pack2of<T>(v[e + 6] * inv, v[e + 7] * inv));
            } else if (is) {
#pragma unroll
              for (int e = 0; e < 32; e += 4) *reinterpret_cast<float4*>(slot + in * DIM + half * (DIM / 2) + 32 * c + e) = make_float4(v[e], v[e + 1], v[e + 2], v[e + 3]);
            }
            __syncwarp();
          }
          if (is && half == 0) {
            if (!whole) {
              slot[kRows * DIM + in] = ref;
              slot[kRows * (DIM + 1) + in] = total;
            } else if (p.lse) {
              p.lse[token * p.q_heads + qh] = 0.69314718055994531f * ((ref == -INFINITY ? 0.f : ref) + log2f(total));
            }
          }
          tc_fence_before();
        }
        if (u + 1 == count && tid == 0) {
          const bool open = !(flags & kEnds) && (flags & kWholeStart);
          p.open[2 * share] = make_int4(q0, h, item.x, min(kRows, item.y - item.x));
          p.open[2 * share + 1].x = open ? (int)((first + per + item.w - 1) / per) : -1;
        }
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == kSoftmaxWarps) tmem_dealloc(tmem, 512);
  if (tid == 0 && *abort_flag) p.open[2 * share + 1].y = 1;
  launch_dependents_now();
}

}  // namespace wide
}  // namespace attend
}  // namespace covspec
