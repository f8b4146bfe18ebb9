// Attention of many rows per key head (chunks of prompts, large blocks) over the paged cache on the tensor cores (tcgen05).
//
// An item is 256 rows of one key head, two tiles of 128 that take turns: while the softmax of one tile runs, the tensor core
// multiplies for the other.  A unit is 128 keys.  TMEM holds S (scores, 128 columns) and O (the rows, `DIM` columns) of both
// tiles; the probabilities overwrite S in 16 bits and are the A operand of the second product from there.  Keys are K-major, values
// MN-major (keys are the inner dimension of the second product), both as rows of 64 features in 128-byte swizzled tiles.
//
// Warps: 0-3 and 4-7 softmax of tile 0 and 1, a row a thread; 8-10 bring queries, keys and values into shared memory, 16-bit rows by
// asynchronous copies, 8-bit ones through registers, where they are widened (attend_kernels.cuh); 11 issues the products.  Twelve
// warps leave each thread 168 registers; with 16 and registers moved between them, some of either kind spilled.
//
// The running maximum is only a reference that keeps the exponentials in range: a row keeps it
// while a unit's probabilities add up to at most 2^14, so that O is rescaled seldom and one pass over S makes the probabilities.  A
// warp with a row beyond that goes over S again with new references.
#pragma once
#include <type_traits>

#include "attend_kernels.cuh"

namespace covspec {
namespace attend {
namespace wide {

using namespace tc;

constexpr int kRows = 256, kKeys = 128;
constexpr int kThreads = 12 * 32;
constexpr int kProducers = 96;
constexpr float kMost = 16384.f;            // a unit's probabilities add up to no more over their reference

template <int STORE, int DIM> struct Layout {
  static constexpr bool k8 = STORE >= cache::kE4M3;
  static constexpr int kSlot = kKeys * DIM * 2;                // keys or values of a unit, 16-bit
  static constexpr int kRow = DIM * (k8 ? 1 : 2);              // bytes of a row in the cache
  static constexpr int kQ = kRows * DIM * 2;
  static constexpr int kSlots = k8 ? 4 : 5;
  static constexpr int kTail = 4 * 16                          // which keys of a unit are there, 4 units
                               + (k8 ? 4 * 2 * kKeys * 4 + 2 * kRows * 4 : 0)   // scales of 4 units; of the query rows of 2 items
                               + 2 * kKeys * 8                 // places of a unit's keys, 2 units
                               + 256;                          // barriers, TMEM base, scratch
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
__device__ __forceinline__ void fence_async_proxy() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

__device__ __forceinline__ f32x2 add2(f32x2 a, f32x2 b) {
  f32x2 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
// 16 columns of this warp's lanes; the registers hold them after tmem_arrived on them.
__device__ __forceinline__ void tmem_fetch(uint32_t taddr, uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
        "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(taddr));
}
__device__ __forceinline__ void tmem_arrived(uint32_t (&r)[16]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]),
                 "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15])::"memory");
}

// Barrier among `n` threads that tells each whether all came with `v`.
__device__ __forceinline__ bool barrier_and(int id, int n, bool v) {
  uint32_t r;
  asm volatile(
      "{\n"
      ".reg .pred p, q;\n"
      "setp.ne.u32 p, %3, 0;\n"
      "barrier.cta.red.and.aligned.pred q, %1, %2, p;\n"
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
__global__ void __launch_bounds__(kThreads, 1) attend_wide_kernel(Params p) {
  using L = Layout<STORE, DIM>;
  constexpr bool k8 = L::k8;
  using M = std::conditional_t<k8, __half, T>;                 // type of the products
  constexpr bool kConvert = !__is_same(M, T);                  // queries to float16
  constexpr int kSlots = L::kSlots;
  extern __shared__ __align__(1024) uint8_t wide_smem[];
  uint8_t* smem = wide_smem;
  uint8_t* ring = smem + L::kQ;
  uint8_t* tail = ring + kSlots * L::kSlot;
  uint32_t* there = reinterpret_cast<uint32_t*>(tail);                       // [4][4]
  float* scales = reinterpret_cast<float*>(tail + 64);                       // [4][2][kKeys]: key scale, value scale
  float* row_scales = scales + 4 * 2 * kKeys;                                // [2][kRows]
  uint32_t* places = reinterpret_cast<uint32_t*>(tail + 64 + (k8 ? 4 * 2 * kKeys * 4 + 2 * kRows * 4 : 0));  // [2][2][kKeys]: keys', values' rows in 16 bytes
  uint64_t* bars = reinterpret_cast<uint64_t*>(places + 4 * kKeys);
  uint64_t *full = bars, *empty = bars + 5, *q_full = bars + 10, *q_empty = bars + 11, *s_full = bars + 12, *p_ready = bars + 14,
           *o_full = bars + 16, *drained = bars + 18;                        // 19 barriers
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 19);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  const int tid = threadIdx.x, warp = warp_index(), lane = tid & 31;
  if (tid == 0) {
    for (int i = 0; i < kSlots; ++i) { mbar_init(full + i, kProducers); mbar_init(empty + i, 1); }
    mbar_init(q_full, kProducers);
    mbar_init(q_empty, 1);
    for (int i = 0; i < 2; ++i) { mbar_init(s_full + i, 1); mbar_init(p_ready + i, 4); mbar_init(o_full + i, 1); }
    mbar_init(drained, 1);
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  wait_for_previous_kernel();
  Cursor<kRows, kKeys> at;
  long long first, per;
  const int count = find_share<kRows, kKeys, kThreads>(p, at, first, per, reinterpret_cast<long long*>(places));
  const int share = blockIdx.x;
  if (count <= 0) {
    if (tid == 0) p.open[2 * share + 1] = make_int4(-1, 0, 0, 0);
    launch_dependents_now();
    return;
  }
  if (warp == 11) tmem_alloc(tmem_slot, 512);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  constexpr uint32_t kO = 256;                                 // first column of O; tile x: S at 128 x, O at kO + 128 x

  if (warp >= 8 && warp < 11) {
    // ---------------- producers ----------------
    const int t = tid - 8 * 32, wp = warp - 8;
    uint64_t* waiting[3] = {nullptr, nullptr, nullptr};        // barriers of copies that are under way, the oldest last
    auto close = [&](uint64_t* bar) {                          // the copies so far belong to `bar`
      copies_close();
      if (waiting[2]) { copies_wait<3>(); fence_async_proxy(); mbar_arrive(waiting[2]); }
      waiting[2] = waiting[1];
      waiting[1] = waiting[0];
      waiting[0] = bar;
    };
    auto flush = [&] {
      copies_wait<0>();
      fence_async_proxy();
#pragma unroll
      for (int i = 2; i >= 0; --i) {
        if (waiting[i]) mbar_arrive(waiting[i]);
        waiting[i] = nullptr;
      }
    };
    // nothing is waited for while copies that the others may need to get on have not been handed over
    auto acquire = [&](uint64_t* bar, uint32_t parity) {
      if (mbar_peek(bar, parity)) return true;
      flush();
      return mbar_wait(bar, parity, abort_flag);
    };
    int slot = 0;
    uint32_t phase = 1, q_phase = 1;
    bool ok = true, fresh = true;
    [[maybe_unused]] int items = 0;
    auto next_slot = [&] { if (++slot == kSlots) { slot = 0; phase ^= 1u; } };
    int page[2] = {-1, -1};
    auto look_up = [&] {                                       // pages of this thread's keys of the unit at `at`
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int key = at.key + t + i * kProducers;
        const bool mine = (i == 0 || wp == 0) && key >= at.k.lo && key < at.k.hi;
        page[i] = mine ? p.t.table[at.b * p.t.table_ld + (key >> p.c.page_shift)] : -1;
      }
    };
    auto spot_of = [&](long long page_ld, int page, int row) {
      return (uint32_t)((unsigned long long)(page * page_ld + (long long)row * DIM) / (16 / (L::kRow / DIM)));
    };
    look_up();
    for (int u = 0; u < count; ++u) {
      if (fresh) {                                             // `at` is at unit u here: its queries
        ok = ok && acquire(q_empty, q_phase);
        q_phase ^= 1u;
        constexpr int kChunks = DIM / 8, kAtOnce = 32 / kChunks;
        const int chunk = lane % kChunks;
#pragma unroll 4
        for (int row0 = wp * kAtOnce; row0 < kRows; row0 += 3 * kAtOnce) {
          const int row = row0 + lane / kChunks, r = at.tile * kRows + row;
          const bool in = row < kRows, is = ok && in && r < at.r.rows;
          const T* q = static_cast<const T*>(p.q) + (is ? token_of(p, at.r.q0, r) * p.q_ld + (long long)head_of(p, at.h, r) * DIM + chunk * 8 : 0);
          uint8_t* to = smem + (row >> 7) * (128 * DIM * 2) + tile_at(128, row & 127, chunk);
          if constexpr (!kConvert) {
            if (in) copy16(smem_u32(to), q, is);
          } else {
            uint4 w = is ? *reinterpret_cast<const uint4*>(q) : make_uint4(0u, 0u, 0u, 0u);
            float most = largest_of(w.x, largest_of(w.y, largest_of(w.z, largest_of(w.w, 0.f))));
#pragma unroll
            for (int o = kChunks / 2; o > 0; o >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
            const float f = power_for(most);
            if (in) {
              *reinterpret_cast<uint4*>(to) = make_uint4(to_half(w.x, f), to_half(w.y, f), to_half(w.z, f), to_half(w.w, f));
              if (chunk == 0) row_scales[items * kRows + row] = inverse_power(f);
            }
          }
        }
        items ^= 1;
        close(q_full);
      }
      // places of the unit's keys: a thread has key t, the first warp the last 32 too; the pages of the next unit's keys are under
      // way meanwhile
      uint32_t* place = places + (u & 1) * 2 * kKeys;
      {
        uint2 spot[2];
        bool is[2];
        [[maybe_unused]] float ks[2] = {0.f, 0.f}, vs[2] = {1.f, 1.f};
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int row = (at.h << p.c.page_shift) + ((at.key + t + i * kProducers) & ((1 << p.c.page_shift) - 1));
          is[i] = (unsigned)page[i] < (unsigned)p.c.pages;
          spot[i] = is[i] ? make_uint2(spot_of(p.c.k_page, page[i], row), spot_of(p.c.v_page, page[i], row)) : make_uint2(kNowhere, kNowhere);
          if constexpr (k8) {
            const long long w = (((long long)page[i] * p.c.heads) << p.c.page_shift) + row;
            if (is[i]) {
              ks[i] = p.c.k_scale[w];
              vs[i] = p.c.v_scale[w];
            }
          }
        }
        fresh = at.unit + 1 == at.units;
        if (u + 1 < count) {
          at.next(p);
          look_up();
        }
        // the words of unit u - 4 have been read: its products are done (the slot that this unit's keys take says so)
        ok = ok && acquire(empty + slot, phase);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int key = t + i * kProducers;
          if (i == 1 && wp != 0) break;
          place[key] = spot[i].x;
          place[kKeys + key] = spot[i].y;
          const uint32_t word = __ballot_sync(0xffffffffu, is[i]);
          if (lane == 0) there[(u & 3) * 4 + (key >> 5)] = word;
          if constexpr (k8) {
            float* sc = scales + (u & 3) * 2 * kKeys;
            sc[key] = ks[i];
            sc[kKeys + key] = vs[i] < cache::kLeastScale ? cache::kLeastScale : vs[i];
          }
        }
      }
      // all of them go on or none: a thread that has left would be waited for at the next barrier
      if (!(ok = barrier_and(1, kProducers, ok))) break;
#pragma unroll
      for (int kv = 0; kv < 2; ++kv) {
        if (kv && !(ok = acquire(empty + slot, phase))) break;
        uint8_t* dst = ring + slot * L::kSlot;
        constexpr int kChunks = L::kRow / 16, kAtOnce = 32 / kChunks, kPer = (kKeys / kAtOnce + 2) / 3;
        const int chunk = lane % kChunks;
        const char* base = static_cast<const char*>(kv ? p.c.v : p.c.k) + chunk * 16;
        auto row_of = [&](int i) { return (wp + 3 * i) * kAtOnce + lane / kChunks; };
        uint32_t spot[kPer];                                   // read ahead: no load passes a copy
#pragma unroll
        for (int i = 0; i < kPer; ++i) spot[i] = row_of(i) < kKeys ? place[kv * kKeys + row_of(i)] : kNowhere;
        if constexpr (!k8) {
          const uint32_t to = smem_u32(dst);
#pragma unroll
          for (int i = 0; i < kPer; ++i) {
            const bool is = spot[i] != kNowhere;
            if (i < kPer - 1 || row_of(i) < kKeys)
              copy16(to + tile_at(kKeys, row_of(i), chunk), base + (is ? (unsigned long long)spot[i] * 16 : 0ull), is);
          }
          close(full + slot);
        } else {
          uint4 raw[kPer];
#pragma unroll
          for (int i = 0; i < kPer; ++i)
            raw[i] = spot[i] != kNowhere ? *reinterpret_cast<const uint4*>(base + (unsigned long long)spot[i] * 16) : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
          for (int i = 0; i < kPer; ++i) {
            const int row = row_of(i);
            if (i == kPer - 1 && row >= kKeys) break;
            const uint32_t w[4] = {raw[i].x, raw[i].y, raw[i].z, raw[i].w};
            uint32_t v[8];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              v[2 * e] = widen<STORE, true>(w[e], 0, 1);
              v[2 * e + 1] = widen<STORE, false>(w[e], 2, 3);
            }
            *reinterpret_cast<uint4*>(dst + tile_at(kKeys, row, 2 * chunk)) = make_uint4(v[0], v[1], v[2], v[3]);
            *reinterpret_cast<uint4*>(dst + tile_at(kKeys, row, 2 * chunk + 1)) = make_uint4(v[4], v[5], v[6], v[7]);
          }
          flush();                                             // the queries' copies, if they are still under way
          mbar_arrive(full + slot);
        }
        next_slot();
      }
    }
    flush();
  } else if (warp == 11) {
    // ---------------- products ----------------
    const uint32_t qk = idesc<M>(kKeys, false), pv = idesc<M>(DIM, true);
    int k_slot = 0, slot = 0;                                  // slot of the keys in S, next slot of the ring
    uint32_t phase = 0, q_phase = 0, p_phase[2] = {0, 0};
    bool ok = true;
    auto next_slot = [&] { if (++slot == kSlots) { slot = 0; phase ^= 1u; } };
    auto scores = [&](int x, int s) {
      const uint32_t a0 = smem_u32(smem + x * (128 * DIM * 2)), b0 = smem_u32(ring + s * L::kSlot);
#pragma unroll
      for (int h = 0; h < DIM / 64; ++h) {
        const uint64_t a = umma_desc(a0 + h * 128 * 128), b = umma_desc(b0 + h * kKeys * 128);
#pragma unroll
        for (int k = 0; k < 4; ++k) umma_bf16(tmem + x * 128, a + 2 * k, b + 2 * k, qk, (h | k) != 0);
      }
      umma_commit(s_full + x);
    };
    auto rows = [&](int x, int s, bool accumulate) {
      const uint64_t b = desc_mn(smem_u32(ring + s * L::kSlot));
#pragma unroll
      for (int k = 0; k < kKeys / 16; ++k)
        mma_ts(tmem + kO + x * 128, tmem + x * 128 + 8 * k, b + k * (16 * 128 / 16), pv, accumulate || k != 0);
    };
    bool fresh = true, opened = false;                         // the next unit begins an item; its scores are issued
    for (int u = 0; u < count && ok; ++u) {
      const bool two = at.r.rows - at.tile * kRows > 128;
      const bool begins = fresh;
      if (!opened) {
        if (fresh) {
          ok = mbar_wait(q_full, q_phase, abort_flag);
          q_phase ^= 1u;
        }
        ok = ok && mbar_wait(full + slot, phase, abort_flag);
        if (!ok) break;
        tc_fence_after();
        if (lane == 0) {
          scores(0, slot);
          if (two) scores(1, slot);
          umma_commit(empty + slot);
        }
        k_slot = slot;
        next_slot();
      }
      (void)k_slot;
      opened = false;
      const bool ends = at.unit + 1 == at.units, more = u + 1 < count && !ends;
      if (!more && lane == 0) umma_commit(q_empty);
      const int v_slot = slot;
      ok = mbar_wait(full + v_slot, phase, abort_flag);
      if (!ok) break;
      next_slot();
      for (int x = 0; x < (two ? 2 : 1) && ok; ++x) {
        ok = mbar_wait(p_ready + x, p_phase[x], abort_flag);
        p_phase[x] ^= 1u;
        if (!ok) break;
        tc_fence_after();
        if (lane == 0) {
          rows(x, v_slot, !begins);
          if (!more) umma_commit(o_full + x);
          if (x == (two ? 1 : 0)) umma_commit(empty + v_slot);
        }
        if (more) {
          if (x == 0) {
            ok = mbar_wait(full + slot, phase, abort_flag);
            if (!ok) break;
            tc_fence_after();
          }
          if (lane == 0) scores(x, slot);
        }
        __syncwarp();
      }
      if (more && ok) {
        if (lane == 0) umma_commit(empty + slot);
        k_slot = slot;
        next_slot();
        opened = true;
      }
      fresh = ends;
      if (u + 1 < count) at.next(p);
      __syncwarp();
    }
    // TMEM and the ring are free when every product has ended, also after a wait that gave up
    if (lane == 0) umma_commit(drained);
    volatile int gave_up = 0;
    mbar_wait(drained, 0, &gave_up);
    __syncwarp();
  } else {
    // ---------------- softmax ----------------
    const int x = warp >> 2, row = tid & 127;
    const uint32_t s_at = tmem + x * 128 + ((uint32_t)(warp & 3) << 21), o_at = s_at + kO;
    float ref = 0.f, sum = 0.f, row_scale = 0.f;
    int items = 1;                                             // items so far, the parity
    bool unread = true;
    int pos = -1;
    int began = 0;                                             // the item's first unit, counted from the share's
    bool fresh = true, ok = true, active = false;
    uint32_t s_phase = 0, o_phase = 0;
    for (int u = 0; u < count; ++u) {
      const int r = at.tile * kRows + x * 128 + row;
      if (fresh) {
        fresh = false;
        began = u - at.unit;
        active = at.r.rows - at.tile * kRows > x * 128;
        const bool is = r < at.r.rows;
        pos = is ? at.r.length - at.r.n + r / p.group : -1;
        ref = is ? -INFINITY : 0.f;                            // rows past the end never ask for a reference
        items ^= 1;
        unread = true;
        sum = 0.f;
      }
      if (active) {
        ok = ok && mbar_wait(s_full + x, s_phase, abort_flag);
        s_phase ^= 1u;
        tc_fence_after();
        const uint4 bits = *reinterpret_cast<const uint4*>(there + (u & 3) * 4);
        const float* sc = scales + (u & 3) * 2 * kKeys;
        if (unread) {                                          // the item's first unit: its queries are there
          row_scale = kConvert ? row_scales[items * kRows + x * 128 + row] * p.scale_log2 : p.scale_log2;
          unread = false;
        }
        // every row of the warp sees all keys of the unit
        const bool clear = (bits.x & bits.y & bits.z & bits.w) == 0xffffffffu &&
                           __all_sync(0xffffffffu, pos < 0 ? r >= at.r.rows : at.key + kKeys - 1 <= pos && (p.window == 0 || at.key > pos - p.window));
        const int lowest = p.window ? max(pos - p.window + 1, 0) : 0;
        // bits of 32 keys that the row sees
        auto seen = [&](int c) {
          const int k0 = at.key + 32 * c;
          uint32_t see = c == 0 ? bits.x : c == 1 ? bits.y : c == 2 ? bits.z : bits.w;
          see &= pos < k0 ? 0u : pos - k0 >= 31 ? 0xffffffffu : (2u << (pos - k0)) - 1u;
          see &= lowest <= k0 ? 0xffffffffu : lowest - k0 > 31 ? 0u : ~((1u << (lowest - k0)) - 1u);
          return see;
        };
        uint32_t packed[64];
        float more = 0.f, most = 0.f;                          // sums of the probabilities, without and with the values' scales
        auto make = [&](float safe, auto masked) {
          const f32x2 low = pack2(-safe, -safe), by = pack2(row_scale, row_scale);
          f32x2 sum2[2] = {pack2(0.f, 0.f), pack2(0.f, 0.f)}, most2 = pack2(0.f, 0.f);
          uint32_t v[2][16];
          tmem_fetch(s_at, v[0]);
          tmem_arrived(v[0]);
          uint32_t see = 0;
#pragma unroll
          for (int c = 0; c < 8; ++c) {
            if (c < 7) tmem_fetch(s_at + 16 * (c + 1), v[(c + 1) & 1]);
            const uint32_t (&w)[16] = v[c & 1];
            if constexpr (decltype(masked)::value) see = c & 1 ? see >> 16 : seen(c / 2);
#pragma unroll
            for (int e = 0; e < 16; e += 4) {
              f32x2 f[2] = {by, by};
              [[maybe_unused]] f32x2 g[2] = {by, by};
              if constexpr (k8) {
                const float4 a = *reinterpret_cast<const float4*>(sc + 16 * c + e), b = *reinterpret_cast<const float4*>(sc + kKeys + 16 * c + e);
                f[0] = mul2(pack2(a.x, a.y), by); f[1] = mul2(pack2(a.z, a.w), by);
                g[0] = pack2(b.x, b.y); g[1] = pack2(b.z, b.w);
              }
#pragma unroll
              for (int i = 0; i < 2; ++i) {
                float2 t = unpack2(fma2(pack2(__uint_as_float(w[e + 2 * i]), __uint_as_float(w[e + 2 * i + 1])), f[i], low));
                if constexpr (decltype(masked)::value) {
                  t.x = (see >> (e + 2 * i)) & 1u ? t.x : -INFINITY;
                  t.y = (see >> (e + 2 * i + 1)) & 1u ? t.y : -INFINITY;
                }
                t.x = ex2(t.x);
                t.y = ex2(t.y);
                f32x2 t2 = pack2(t.x, t.y);
                sum2[i] = add2(sum2[i], t2);
                if constexpr (k8) {
                  t2 = mul2(t2, g[i]);
                  most2 = add2(most2, t2);
                  t = unpack2(t2);
                }
                packed[8 * c + e / 2 + i] = pack2of<M>(t.x, t.y);
              }
            }
            if (c < 7) tmem_arrived(v[(c + 1) & 1]);
          }
          const float2 a = unpack2(add2(sum2[0], sum2[1])), b = unpack2(most2);
          more = a.x + a.y;
          most = k8 ? b.x + b.y : more;
        };
        bool again = __any_sync(0xffffffffu, ref == -INFINITY);
        if (!again) {
          if (clear) make(ref, std::false_type());
          else make(ref, std::true_type());
          again = __any_sync(0xffffffffu, most > kMost);
        }
        if (again) {                                           // new references, from the scores themselves
          float best = ref;
#pragma unroll 1
          for (int c = 0; c < 8; ++c) {
            float v[16];
            tmem_ld16(s_at + 16 * c, v);
            const uint32_t see = seen(c / 2) >> (16 * (c & 1));
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              const int key = 16 * c + e;
              const float t = k8 ? v[e] * (sc[key] * row_scale) + log2f(sc[kKeys + key]) : v[e] * row_scale;
              best = (see >> e) & 1u ? fmaxf(best, t) : best;
            }
          }
          const float shrink = ref == -INFINITY ? 0.f : ex2(ref - best);
          ref = best;
          sum *= shrink;
          if (u > max(began, 0)) {                             // O holds earlier units' rows
#pragma unroll 1
            for (int c = 0; c < DIM / 32; ++c) {
              float v[32];
              tmem_ld32(o_at + 32 * c, v);
              uint32_t w[32];
#pragma unroll
              for (int e = 0; e < 32; ++e) w[e] = __float_as_uint(v[e] * shrink);
              tmem_st32(o_at + 32 * c, w);
            }
            tmem_st_wait();
          }
          make(ref == -INFINITY ? 0.f : ref, std::true_type());
        }
        sum += more;
        tmem_st32(s_at, packed);
        tmem_st32(s_at + 32, packed + 32);
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(p_ready + x);
      }
      const bool last = at.unit + 1 == at.units;
      if (last || u + 1 == count) {
        const bool whole = last && began >= 0;
        if (active) {
          ok = ok && mbar_wait(o_full + x, o_phase, abort_flag);
          o_phase ^= 1u;
          tc_fence_after();
          const bool is = r < at.r.rows;
          // a wait that gave up leaves NaN
          const float inv = !ok ? __int_as_float(0x7fffffff) : sum > 0.f ? 1.f / sum : (sum == sum ? 0.f : sum);
          const long long token = is ? token_of(p, at.r.q0, r) : 0;
          const int qh = is ? head_of(p, at.h, r) : 0;
          T* out = static_cast<T*>(p.out) + token * p.out_ld + (long long)qh * DIM;
          float* slot = p.part + (2 * share + (began >= 0)) * (long long)(kRows * (DIM + 2));
          const int in = x * 128 + row;
#pragma unroll 1
          for (int c = 0; c < DIM / 32; ++c) {
            float v[32];
            tmem_ld32(o_at + 32 * c, v);
            if (is && whole) {
#pragma unroll
              for (int e = 0; e < 32; e += 8)
                *reinterpret_cast<uint4*>(out + 32 * c + e) = make_uint4(pack2of<T>(v[e] * inv, v[e + 1] * inv), pack2of<T>(v[e + 2] * inv, v[e + 3] * inv),
                                                                         pack2of<T>(v[e + 4] * inv, v[e + 5] * inv), pack2of<T>(v[e + 6] * inv, v[e + 7] * inv));
            } else if (is) {
#pragma unroll
              for (int e = 0; e < 32; e += 4) *reinterpret_cast<float4*>(slot + in * DIM + 32 * c + e) = make_float4(v[e], v[e + 1], v[e + 2], v[e + 3]);
            }
            __syncwarp();
          }
          if (is) {
            if (!whole) {
              slot[kRows * DIM + in] = ref;
              slot[kRows * (DIM + 1) + in] = ok ? sum : inv;
            } else if (p.lse) {
              p.lse[token * p.q_heads + qh] = ok ? 0.69314718055994531f * ((ref == -INFINITY ? 0.f : ref) + log2f(sum)) : inv;
            }
          }
          tc_fence_before();
        }
        if (u + 1 == count && tid == 0) {
          const bool open = !last && began >= 0;
          const long long end = first + began + at.units - 1;
          p.open[2 * share] = make_int4(at.r.q0, at.h, at.tile * kRows, min(kRows, at.r.rows - at.tile * kRows));
          p.open[2 * share + 1] = make_int4(open ? (int)(end / per) : -1, 0, 0, 0);
        }
        fresh = true;
      }
      if (u + 1 < count) at.next(p);
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == 11) tmem_dealloc(tmem, 512);
  launch_dependents_now();
}

}  // namespace wide
}  // namespace attend
}  // namespace covspec
