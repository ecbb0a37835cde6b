// Long rows of logits, many of them: one persistent CTA per SM, rows streamed
// through shared memory, so that the copies of the next rows are in flight
// while one is reduced and its gradient written.
//
// Roles of a CTA:
//   warp 0      : copies (one thread): bulk copies of a row's share into a ring
//                 of slots, one mbarrier pair each
//   warp 1      : schedule: finds the CTA's rows and passes them on, with the
//                 row's scalars and slots, through a ring of entries
//   the others  : groups of warps. With a gradient they take the rows in turn, so
//                 that some compute while others wait for their row's sum:
//                 statistics slot by slot; then the group's first warp joins the
//                 warps' sums, works out the row's coefficient and hands it to
//                 the others for the gradient, which they take from the slots.
//                 Without one, one warp joins the sums while the others go on,
//                 and the groups take the slots of long rows in turn.
// A row of up to 76 KB belongs to one CTA; a longer one to a cluster of 2, 4
// or 8, each with an equal share, whose maxima and sums are exchanged through
// distributed shared memory, one message per pair of CTAs and row. The rows are
// dealt out in turn, which spreads the runs of scored rows that masks come in.
//
// The rows' first and last elements that fill no 16 bytes travel with the row's
// entry and are put into their slot by the threads that read it; bulk copies
// move the rest.
//
// A warp's exponentials are relative to a reference that moves only when a
// logit exceeds it by 16, so most slots cost neither a warp-wide maximum nor a
// rescaled sum.
//
// HBM bounds it, with the issue slots at 60% (gradient) and 70% (statistics). Measured
// in bf16, with the time of the bytes at the measured copy rate (6.79 TB/s) in
// brackets, us: gradient 4096 x 50001 133 (121), 8192 x 32000 171 (155), 2048 x 151936
// 193 (183), fp32 2048 x 32000 97 (77); statistics 4096 x 50001 72 (60), 8192 x 32000
// 86 (77), 4096 x 151936 193 (183). Of 8192 x 32000 with 80% of the rows scored at
// random, 169 (139) and 80 (62): some CTAs have more of them than others. The loss
// without its gradient takes 129 us for 8192 x 32000 (77): the slots are given
// back in the pass that would write it.
//
// Every wait is bounded. On expiry the roles of the CTA (and, for want of its
// messages, of its cluster) stop, and when all have, every row of it gets NaN for
// all its results, the gradient too: neither what a buffer held before nor, with
// the gradient in their place, logits are left standing as results.
#include <mutex>

#include "loss_rows.cuh"
#include "meq_mbar.cuh"

namespace meq {
namespace loss {
namespace {

constexpr int kRingBytes = 224 * 1024;
constexpr float kSlack = 16.f;                     // logits above a warp's reference before it moves
// kPieces: a lane's pieces of a warp's unit. With a gradient, where rows stay in
// the ring until it is written, four groups of five warps: while one joins its
// sums and another writes, two take in rows. Groups x warps 4 x 5, 3 x 7, 4 x 6,
// 5 x 4, us: 8192 x 32000 bf16 171, 185, 170, 182; 4096 x 50001 134, 149, 149, 147.
template <bool kPolicy, int kPieces>
struct Cfg {
  static constexpr int kGroups = kPolicy ? 4 : 3, kUserWarps = kPolicy ? 5 : 8;
  static constexpr int kUnit = 32 * kPieces;
  static constexpr int kUsers = kGroups * kUserWarps;
  static constexpr int kThreads = kUsers * 32 + 64;
  static constexpr int kSlot = kUserWarps * kUnit;    // pieces of a slot: one unit per warp
  static constexpr int kSlots = kRingBytes / (kSlot * 16);
};
constexpr int kMostSlots = Cfg<true, 4>::kSlots, kMostUsers = Cfg<false, 4>::kUsers, kMostGroups = Cfg<true, 4>::kGroups;
static_assert(kMostUsers <= 32 && kMostSlots <= 32, "a lane, or a bit, for each");
constexpr int kEntries = 8;
constexpr int kMaxShare = 76 * 1024;               // of a row per CTA: the ring holds 2.8
constexpr int kMaxCtas = 8;
constexpr unsigned long long kWaitNs = 4000000000ull;
// A wait gives up after the limit's time and at least this many polls: time that
// passes while the context is switched out polls nothing.
constexpr uint32_t kLeastPolls = 1024, kMostPolls = 1u << 28;

struct Entry {
  const void* logits;  // of the row
  void* grad;          // NULL: none
  int row;             // -1: no more
  int scored;
  int token;           // kNoToken: beyond the row
  int group;           // that takes it
  int slot;            // its first slot, the phase of it, and the slot's use, counted from the kernel's start
  uint32_t phase, use;
  float weight, old_logp, advantage, ref_logp, zt;
  uint4 head, tail;    // the row's first and last piece, where they do not exist whole
};
// What a group's first warp tells the others of a row.
struct RowResult {
  GradScale scale;
  int ok;
};

// A warp's maximum, its own exponential left out of the sum of the others',
// which is relative to ref.
struct WarpSum {
  float m, rest, ref;
};

struct Limit {
  unsigned long long ns;  // of a wait
  int stop;               // a wait has run out
};

struct StreamShared {
  uint64_t full[kMostSlots], empty[kMostSlots];
  uint64_t entry_full[kEntries], entry_empty[kEntries];
  uint64_t joined[kMostGroups][2], exchange[kMostGroups][2], ready[kMostGroups][2];
  Entry entry[kEntries];
  WarpSum warp[2][kMostUsers];
  MaxSum cta[kMostGroups][2][kMaxCtas];
  RowResult result[kMostGroups][2];
  uint32_t claimed;  // slot uses whose copies are under way
  Limit limit;
};
constexpr int kStreamSmem = kRingBytes + static_cast<int>(sizeof(StreamShared)) + 128;
static_assert(kStreamSmem <= 232448, "shared memory budget of one sm_103a CTA");

struct StreamShape {
  int ctas;    // per row
  int share;   // pieces of a row per CTA, at most
  int rounds;  // slots per share
  int by_slots;  // statistics: 1: the groups take a row's slots in turn, 0: they take the rows in turn
  int pieces;    // of a unit, per lane
  unsigned long long wait_ns;
  int64_t withheld;  // for a test: a row whose first slot is never filled (none: -1)
};

// Whether a wait that began at t0 gives up at poll `it` (looked at in every 128th).
__device__ __forceinline__ bool gives_up(volatile Limit* limit, uint64_t t0, uint32_t it) {
  return limit->stop != 0 || (global_ns() - t0 > limit->ns && it >= kLeastPolls) || it >= kMostPolls;
}
// All lanes of a warp; the same answer in each. False: gave up.
__device__ __forceinline__ bool wait_warp(uint32_t bar, uint32_t parity, volatile Limit* limit) {
  const unsigned FULL = 0xffffffffu;
  if (__all_sync(FULL, mbar_try_wait(bar, parity))) return true;
  const uint64_t t0 = global_ns();
  for (uint32_t it = 1;; ++it) {
    if (__all_sync(FULL, mbar_try_wait(bar, parity))) return true;
    if ((it & 127u) == 0 && __any_sync(FULL, gives_up(limit, t0, it))) {
      limit->stop = 1;
      return false;
    }
  }
}
__device__ __forceinline__ bool wait_one(uint32_t bar, uint32_t parity, volatile Limit* limit) {
  if (mbar_try_wait(bar, parity)) return true;
  const uint64_t t0 = global_ns();
  for (uint32_t it = 1;; ++it) {
    if (mbar_try_wait(bar, parity)) return true;
    if ((it & 127u) == 0 && gives_up(limit, t0, it)) {
      limit->stop = 1;
      return false;
    }
  }
}
// A group may reach a slot before the other group has seen that slot's last
// use filled; its barrier is then still in the phase before, whose parity says
// "complete". So a slot is waited for only once its use has been claimed,
// which the other group's release of it precedes.
__device__ __forceinline__ bool wait_claimed(const uint32_t* claimed, uint32_t use, volatile Limit* limit) {
  const unsigned FULL = 0xffffffffu;
  const uint32_t addr = smem_u32(claimed);
  uint64_t t0 = 0;
  for (uint32_t it = 0;; ++it) {
    uint32_t n;
    asm volatile("ld.acquire.cta.shared::cta.u32 %0, [%1];" : "=r"(n) : "r"(addr) : "memory");
    if (__all_sync(FULL, static_cast<int32_t>(n - use) > 0)) return true;
    if ((it & 127u) == 0) {
      if (it == 0) t0 = global_ns();
      if (__any_sync(FULL, gives_up(limit, t0, it))) {
        limit->stop = 1;
        return false;
      }
    }
  }
}
__device__ __forceinline__ void bulk_copy(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src),
               "r"(bytes), "r"(bar)
               : "memory");
}
// Eight bytes into another CTA's shared memory, as a transaction on its
// barrier, which this call also arms (one arrival).
__device__ __forceinline__ void send(uint32_t addr_cluster, uint32_t bar_cluster, MaxSum v) {
  asm volatile("mbarrier.arrive.expect_tx.relaxed.cluster.shared::cluster.b64 _, [%0], 8;" ::"r"(bar_cluster) : "memory");
  asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.v2.b32 [%0], {%1, %2}, [%3];" ::"r"(addr_cluster),
               "r"(__float_as_uint(v.m)), "r"(__float_as_uint(v.s)), "r"(bar_cluster)
               : "memory");
}

// A warp's running sum of exponentials, each lane's part relative to the same
// reference (-inf before the first finite logit).
template <typename T>
struct Running {
  float ref = -INFINITY, c = 0.f, fix = 1.f, s = 0.f;
  typename Elem<T>::Max top = Elem<T>::none();  // the lane's largest logit
  template <int P>
  __device__ __forceinline__ void add(const uint4 (&q)[P]) {
    constexpr int H = Elem<T>::N / 2;
#pragma unroll
    for (int j = 0; j < P; ++j) top = Elem<T>::max_of(top, q[j]);
    float m = Elem<T>::value(top);
    if (__any_sync(0xffffffffu, m > ref + kSlack)) {
      m = warp_max(m);
      const ExpBase b(fabsf(m) <= kFar ? m : 0.f);
      s = s * fix * exp_diff(ref, m) / b.fix;
      ref = m, c = b.c, fix = b.fix;
    }
    float2 a[P] = {make_float2(s, 0.f)};  // sums side by side: one would be a chain of additions
    if (fabsf(ref) <= kFar || ref == -INFINITY) {
#pragma unroll
      for (int j = 0; j < P; ++j) {
        float2 x[H];
        Elem<T>::unpack(q[j], x);
#pragma unroll
        for (int e = 0; e < H; ++e) {
          const float2 y = fma2(x[e], make_float2(kLog2e, kLog2e), make_float2(-c, -c));
          const float2 z = fma2(x[e], make_float2(kLog2eLo, kLog2eLo), y);
          a[j] = add2(a[j], make_float2(exp2_approx(z.x), exp2_approx(z.y)));
        }
      }
    } else {  // +inf gives NaN
#pragma unroll
      for (int j = 0; j < P; ++j) {
        float2 x[H];
        Elem<T>::unpack(q[j], x);
#pragma unroll
        for (int e = 0; e < H; ++e) a[j] = add2(a[j], make_float2(exp_diff(x[e].x, ref), exp_diff(x[e].y, ref)));
      }
    }
#pragma unroll
    for (int j = 1; j < P; ++j) a[0] = add2(a[0], a[j]);
    s = a[0].x + a[0].y;
  }
  __device__ __forceinline__ WarpSum total() const {  // of the warp, for every lane
    WarpSum t{warp_max(Elem<T>::value(top)), s, ref};
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) t.rest += __shfl_xor_sync(0xffffffffu, t.rest, o);
    if (t.m != -INFINITY) t.rest = (t.rest - (fabsf(ref) <= kFar ? exp_at(t.m, c) : exp_diff(t.m, ref))) * fix;
    return t;
  }
};
// Over the lanes' sums, the same in each lane.
__device__ __forceinline__ MaxSum lanes_join(WarpSum t) {
  MaxSum r{warp_max(t.m), 0.f};
  const float base = finite_or_zero(r.m);
  r.s = fmaf(t.rest, exp_diff(t.ref, base), exp_diff(t.m, base));
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) r.s += __shfl_xor_sync(0xffffffffu, r.s, o);
  return r;
}

// NaN for all results of all rows of the CTA's cluster, of whose gradient it takes its share.
template <typename T, bool kPolicy>
__device__ __forceinline__ void lose_rows(const RowArgs& a, uint32_t ctas) {
  const float nan = __int_as_float(0x7fc00000);
  const uint32_t rank = ctas == 1 ? 0u : cluster_rank();
  for (int64_t row = blockIdx.x / ctas; row < a.rows; row += gridDim.x / ctas) {
    if (rank == 0 && threadIdx.x == 0) {
      a.logp[row] = nan;
      if (a.lse) a.lse[row] = nan;
      if (a.stat) a.stat[row] = make_float2(nan, nan);
      if (a.coef) a.coef[row] = nan;
      if (kPolicy) a.terms[row] = make_float4(nan, nan, nan, nan);
    }
    if (kPolicy && a.grad) {
      T* g = static_cast<T*>(a.grad) + row * a.ld_grad;
      for (int64_t i = static_cast<int64_t>(rank) * blockDim.x + threadIdx.x; i < a.cols; i += static_cast<int64_t>(ctas) * blockDim.x)
        g[i] = Elem<T>::make(nan);
    }
  }
}

template <typename T, bool kPolicy>
__device__ __noinline__ void lose_rows_called(const RowArgs& a, uint32_t ctas) {
  lose_rows<T, kPolicy>(a, ctas);
}

template <typename T, bool kPolicy, int kPieces>
__global__ void __launch_bounds__(Cfg<kPolicy, kPieces>::kThreads, 1) stream_kernel(const __grid_constant__ RowArgs a, const StreamShape shape) {
  using C = Cfg<kPolicy, kPieces>;
  constexpr int kSlots = C::kSlots, kSlot = C::kSlot, kUnit = C::kUnit, kUserWarps = C::kUserWarps, kGroups = C::kGroups;
  static_assert(C::kSlots <= kMostSlots && C::kUsers <= kMostUsers && C::kGroups <= kMostGroups, "");
  const bool by_slots = !kPolicy && shape.by_slots != 0;
  pdl_allow_dependents();
  extern __shared__ uint8_t smem_raw[];
  uint8_t* ring = smem_raw + ((128u - (smem_u32(smem_raw) & 127u)) & 127u);
  StreamShared& sh = *reinterpret_cast<StreamShared*>(ring + kRingBytes);
  const uint32_t ctas = static_cast<uint32_t>(shape.ctas), rank = ctas == 1 ? 0u : cluster_rank();
  const int warp = static_cast<int>(threadIdx.x >> 5), lane = static_cast<int>(threadIdx.x & 31);
  volatile Limit* stop = &sh.limit;
  if (threadIdx.x == 0) {
    for (int i = 0; i < kSlots; ++i) {
      mbar_init(smem_u32(&sh.full[i]), 1);
      mbar_init(smem_u32(&sh.empty[i]), kUserWarps);
    }
    for (int i = 0; i < kEntries; ++i) {
      mbar_init(smem_u32(&sh.entry_full[i]), 1);
      mbar_init(smem_u32(&sh.entry_empty[i]), C::kUsers + 1);
    }
    for (int i = 0; i < 2 * kGroups; ++i) {
      mbar_init(smem_u32(&sh.joined[i / 2][i % 2]), by_slots ? C::kUsers : kUserWarps);
      mbar_init(smem_u32(&sh.exchange[i / 2][i % 2]), ctas);
      mbar_init(smem_u32(&sh.ready[i / 2][i % 2]), 1);
    }
    sh.limit.ns = shape.wait_ns;
    sh.limit.stop = 0;
    sh.claimed = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  __syncthreads();
  if (ctas > 1) cluster_sync_all();
  pdl_wait_predecessor();

  if (warp == 0) {
    if (lane == 0) {
      // ------------------------------------------------------------- copies
      int slot = 0;
      uint32_t phase = 0, filled = 0, filled_phase = 0, use = 0;
      bool ok = true;
      for (int n = 0; ok; ++n) {
        const int i = n % kEntries;
        if (!wait_one(smem_u32(&sh.entry_full[i]), (n / kEntries) & 1, stop)) break;
        const int row = sh.entry[i].row, scored = sh.entry[i].scored;
        const Row<T> r(sh.entry[i].logits, 0, 0, a.cols);
        mbar_arrive_local(smem_u32(&sh.entry_empty[i]));
        if (row < 0) break;
        if (!scored) continue;
        const int lo = static_cast<int>(rank) * shape.share, hi = min(lo + shape.share, r.end);
        for (int c = 0; c < shape.rounds; ++c) {
          if (!wait_one(smem_u32(&sh.empty[slot]), phase ^ 1u, stop)) {
            ok = false;
            break;
          }
          const int c0 = lo + c * kSlot, w0 = max(c0, r.begin), w1 = min(c0 + kSlot, hi);
          const uint32_t bar = smem_u32(&sh.full[slot]);
          const bool withheld = row == shape.withheld && c == 0;
          if (withheld) {
          } else if (w1 > w0) {
            mbar_expect_tx(bar, static_cast<uint32_t>(w1 - w0) * 16u);
            bulk_copy(smem_u32(ring) + static_cast<uint32_t>(slot * kSlot + (w0 - c0)) * 16u, r.p + (w0 * Row<T>::N - r.lead),
                      static_cast<uint32_t>(w1 - w0) * 16u, bar);
          } else {
            mbar_arrive_local(bar);
          }
          ++use;
          asm volatile("st.release.cta.shared::cta.u32 [%0], %1;" ::"r"(smem_u32(&sh.claimed)), "r"(use) : "memory");
          if (!withheld) filled |= 1u << slot;
          filled_phase = (filled_phase & ~(1u << slot)) | (phase << slot);
          if (++slot == kSlots) slot = 0, phase ^= 1u;
        }
      }
      // every copy has landed before the CTA leaves
      Limit own{sh.limit.ns, 0};
      for (int s = 0; s < kSlots; ++s)
        if ((filled >> s) & 1u) wait_one(smem_u32(&sh.full[s]), (filled_phase >> s) & 1u, &own);
    }
    __syncwarp();
  } else if (warp == 1) {
    // -------------------------------------------------------------- schedule
    // Row group + k groups is the k-th of this CTA (or cluster): 32 of them at a
    // time, a lane each, the next ones' targets and weights asked for ahead.
    const int64_t groups = gridDim.x / ctas, group = blockIdx.x / ctas;
    int n = 0, slot = 0;
    uint32_t phase = 0, use = 0, scored_here = 0, others_here = 0;
    bool ok = true;
    int64_t row = group + lane * groups, target = -1;
    float w = 1.f;
    auto fetch = [&]() {
      target = row < a.rows ? a.targets[row] : -1;
      w = row < a.rows && a.weights ? a.weights[row] : 1.f;
    };
    fetch();
    while (ok) {
      Entry e{};
      const bool in = row < a.rows;
      if (in) {
        e.logits = static_cast<const T*>(a.logits) + row * a.ld;
        e.grad = kPolicy && a.grad ? static_cast<T*>(a.grad) + row * a.ld_grad : nullptr;
        e.row = static_cast<int>(row), e.scored = target >= 0 && w != 0.f, e.weight = w;
        e.token = target < a.cols ? static_cast<int>(target) : kNoToken;
        if (e.scored) {
          const Row<T> r(e.logits, 0, 0, a.cols);
          if (r.begin) e.head = r.load_part(0);
          if (r.pieces > r.end) e.tail = r.load_part(r.pieces - 1);
          e.zt = e.token != kNoToken ? Elem<T>::get(static_cast<const T*>(e.logits) + e.token) : __int_as_float(0x7fc00000);
          if (kPolicy) {
            e.old_logp = a.old_logp[row], e.advantage = a.advantages[row];
            if (a.kl != 0.f) e.ref_logp = a.ref_logp[row];
          }
        }
      }
      const int rows_here = __popc(__ballot_sync(0xffffffffu, in));
      row += 32 * groups;
      fetch();
      for (int owner = 0; owner < rows_here; ++owner, ++n) {
        const int i = n % kEntries;
        ok = wait_warp(smem_u32(&sh.entry_empty[i]), ((n / kEntries) & 1) ^ 1, stop);
        if (!ok) break;
        const int on = __shfl_sync(0xffffffffu, e.scored, owner);
        if (lane == owner) {
          e.group = static_cast<int>((on ? scored_here : others_here) % kGroups);
          e.slot = slot, e.phase = phase, e.use = use;
          sh.entry[i] = e;
          mbar_arrive_local(smem_u32(&sh.entry_full[i]));
        }
        __syncwarp();
        if (on) {
          ++scored_here;
          slot += shape.rounds;  // rounds may exceed the ring (statistics of a very long row)
          phase ^= static_cast<uint32_t>(slot / kSlots) & 1u;
          slot %= kSlots;
          use += static_cast<uint32_t>(shape.rounds);
        } else {
          ++others_here;
        }
      }
      if (rows_here < 32) break;
    }
    if (ok) {
      const int i = n % kEntries;
      ok = wait_warp(smem_u32(&sh.entry_empty[i]), ((n / kEntries) & 1) ^ 1, stop);
      if (ok && lane == 0) {
        sh.entry[i].row = -1;
        mbar_arrive_local(smem_u32(&sh.entry_full[i]));
      }
    }
    __syncwarp();
  } else {
    // --------------------------------------------- statistics and gradients
    const int team = (warp - 2) / kUserWarps, uw = (warp - 2) % kUserWarps;
    const int group = by_slots ? 0 : team;  // that shares a row
    const bool first_warp = by_slots ? warp == 2 : uw == 0;
    const float gs = kPolicy && a.grad_scale ? *a.grad_scale : 1.f;
    uint32_t joins = 0;  // scored rows of the group so far
    for (int n = 0;; ++n) {
      const int i = n % kEntries;
      if (!wait_warp(smem_u32(&sh.entry_full[i]), (n / kEntries) & 1, stop)) break;
      const Entry e = sh.entry[i];
      __syncwarp();
      if (lane == 0) mbar_arrive_local(smem_u32(&sh.entry_empty[i]));
      if (e.row < 0) break;
      if (!by_slots && e.group != group) continue;
      const int64_t row = e.row;
      const Row<T> r(e.logits, 0, 0, a.cols);
      const int lo = static_cast<int>(rank) * shape.share, hi = min(lo + shape.share, r.pieces);
      T* g = static_cast<T*>(e.grad);
      const bool same = same_offset(r.p, g);
      // The warp's unit of slot use c: its lane's first piece, and whether its pieces all exist whole.
      auto first_piece = [&](int c) { return lo + c * kSlot + uw * kUnit + lane; };
      auto whole = [&](int k) { return k - lane >= r.begin && k - lane + kUnit <= min(hi, r.end); };
      // f(j, k) for the lane's pieces of the unit that belong to the row's share
      auto store_unit = [&](int k0, auto f) {
        uint4* d = reinterpret_cast<uint4*>(g + (k0 * Row<T>::N - r.lead));
        if (same && whole(k0)) {
#pragma unroll
          for (int j = 0; j < kPieces; ++j) __stcs(d + 32 * j, f(j));
        } else {
#pragma unroll 1
          for (int j = 0; j < kPieces; ++j) {
            const int k = k0 + 32 * j;
            if (k >= hi) break;
            if (same && k >= r.begin && k < r.end) __stcs(d + 32 * j, f(j));
            else r.store_part(g, k, f(j));
          }
        }
      };
      if (!e.scored) {
        if (rank == 0 && first_warp && lane == 0) {
          a.logp[row] = 0.f;
          if (a.lse) a.lse[row] = 0.f;
          if (a.stat) a.stat[row] = make_float2(0.f, 1.f);
          if (a.coef) a.coef[row] = 0.f;
          if (kPolicy) a.terms[row] = make_float4(0.f, 0.f, 0.f, 0.f);
        }
        if (g)
          for (int c = 0; c < shape.rounds; ++c) store_unit(first_piece(c), [](int) { return make_uint4(0u, 0u, 0u, 0u); });
        continue;
      }
      const int b = joins & 1;
      const uint32_t parity = (joins >> 1) & 1u;
      ++joins;
      Running<T> sum;
      int slot = e.slot;
      uint32_t phase = e.phase;
      bool ok = true;
      for (int c = 0; c < shape.rounds; ++c) {
        if (by_slots && (e.use + static_cast<uint32_t>(c)) % kGroups != static_cast<uint32_t>(team)) {
          if (++slot == kSlots) slot = 0, phase ^= 1u;
          continue;
        }
        ok = wait_claimed(&sh.claimed, e.use + static_cast<uint32_t>(c), stop) && wait_warp(smem_u32(&sh.full[slot]), phase, stop);
        if (!ok) break;
        const int k0 = first_piece(c);
        uint4* at = reinterpret_cast<uint4*>(ring) + slot * kSlot + uw * kUnit + lane;
        if (!whole(k0)) {
#pragma unroll 1
          for (int j = 0; j < kPieces; ++j) {
            const int k = k0 + 32 * j;
            if (k >= hi) at[32 * j] = Row<T>::none();
            else if (k < r.begin) at[32 * j] = e.head;
            else if (k >= r.end) at[32 * j] = e.tail;
          }
          // before the slot's next copy, which another proxy writes
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        }
        uint4 q[kPieces];
#pragma unroll
        for (int j = 0; j < kPieces; ++j) q[j] = at[32 * j];
        if (!kPolicy) {
          __syncwarp();
          if (lane == 0) mbar_arrive_local(smem_u32(&sh.empty[slot]));
        }
        sum.template add<kPieces>(q);
        if (++slot == kSlots) slot = 0, phase ^= 1u;
      }
      const WarpSum w = sum.total();
      // statistics alone: the warps run ahead, by at most the two buffers
      if (!kPolicy && joins > 2) ok = ok && wait_warp(smem_u32(&sh.ready[group][b]), parity ^ 1u, stop);
      if (ok && lane == 0) {
        sh.warp[b][warp - 2] = w;
        mbar_arrive_local(smem_u32(&sh.joined[group][b]));
      }
      __syncwarp();
      if (first_warp) {
        ok = ok && wait_warp(smem_u32(&sh.joined[group][b]), parity, stop);
        MaxSum t = lanes_join(lane < (by_slots ? C::kUsers : kUserWarps) ? sh.warp[b][group * kUserWarps + lane]
                                                                        : WarpSum{-INFINITY, 0.f, -INFINITY});
        if (ok && ctas > 1) {
          if (lane < static_cast<int>(ctas))
            send(map_to_rank(smem_u32(&sh.cta[group][b][rank]), lane), map_to_rank(smem_u32(&sh.exchange[group][b]), lane), t);
          __syncwarp();
          ok = wait_warp(smem_u32(&sh.exchange[group][b]), parity, stop);
          t = sh.cta[group][b][0];
          for (uint32_t k = 1; k < ctas; ++k) t = join(t, sh.cta[group][b][k]);
        }
        float rest;
        const float logp = log_prob(e.zt, t, &rest);
        const bool leader = rank == 0 && lane == 0;
        if (leader) a.logp[row] = logp;
        if (!kPolicy) {
          if (leader) {
            if (a.lse) a.lse[row] = -log_prob(0.f, t);
            if (a.stat) a.stat[row] = make_float2(t.m, t.s);
            if (a.coef) a.coef[row] = 0.f;
          }
        } else {
          const TokenLoss l = policy_token(logp, rest, e.old_logp, e.advantage, &e.ref_logp, a.clip_lo, a.clip_hi, a.kl);
          if (leader)
            a.terms[row] = make_float4(e.weight * (l.surrogate + a.kl * l.k3), e.weight * l.surrogate, e.weight * l.k3, e.weight * l.clipped);
          if (lane == 0) {
            sh.result[group][b].scale = GradScale(e.weight * l.slope * gs, t.m, t.s);
            sh.result[group][b].ok = ok;
          }
        }
        __syncwarp();
        if (lane == 0) mbar_arrive_local(smem_u32(&sh.ready[group][b]));
      }
      if (!kPolicy) {
        if (!ok) break;
        continue;
      }
      ok = ok && wait_warp(smem_u32(&sh.ready[group][b]), parity, stop);
      if (!ok || !sh.result[group][b].ok) break;
      const GradScale s = sh.result[group][b].scale;
      const int target_piece = (e.token + r.lead) / Row<T>::N;
      slot = e.slot;
      for (int c = 0; c < shape.rounds; ++c) {
        if (g) {
          const int k0 = first_piece(c);
          const uint4* at = reinterpret_cast<const uint4*>(ring) + slot * kSlot + uw * kUnit + lane;
          if (s.c == 0.f) store_unit(k0, [](int) { return make_uint4(0u, 0u, 0u, 0u); });
          else if (!s.far) store_unit(k0, [&](int j) { return s.template piece<false, T>(at[32 * j]); });
          else store_unit(k0, [&](int j) { return s.template piece<true, T>(at[32 * j]); });
          if (s.c != 0.f && target_piece < hi && holds<T, kPieces>(r, k0, e.token)) g[e.token] = Elem<T>::make(s.at_target(e.zt));
        }
        __syncwarp();
        if (lane == 0) mbar_arrive_local(smem_u32(&sh.empty[slot]));
        if (++slot == kSlots) slot = 0;
      }
    }
    __syncwarp();
  }
  __syncthreads();
  if (ctas > 1) {
    if (stop->stop != 0) __nanosleep(100000);  // messages on their way (a microsecond) have arrived
    if (stop->stop != 0 && threadIdx.x < ctas)
      asm volatile("st.shared::cluster.u32 [%0], 1;" ::"r"(map_to_rank(smem_u32(&sh.limit.stop), threadIdx.x)) : "memory");
    __syncwarp();
    cluster_sync_all();  // no CTA leaves while another may still write to it
  }
  if (stop->stop != 0) {
    // With five pieces a lane has no register to spare: inlined, it spills, 195 -> 206 us for 2048 x 151936 bf16.
    // With four, called instead of inlined, 4096 x 50001 takes 141 us for 134, statistics 74 for 72.5.
    if (kPieces > 4) lose_rows_called<T, kPolicy>(a, ctas);
    else lose_rows<T, kPolicy>(a, ctas);
  }
}

// Of the calling thread's next launches (meq_debug_loss_wait).
thread_local unsigned long long g_wait_ns = kWaitNs;
thread_local int64_t g_withheld = -1;

template <bool kPolicy, int kPieces>
StreamShape shape_with(int64_t row_pieces, int ctas) {
  using C = Cfg<kPolicy, kPieces>;
  const int64_t share = ((row_pieces + ctas - 1) / ctas + C::kUnit - 1) / C::kUnit * C::kUnit;
  const int rounds = static_cast<int>((share + C::kSlot - 1) / C::kSlot);
  // Three groups take a row each where the ring holds one row and more to come,
  // with one join per group and row; a longer row is shared by the groups slot
  // by slot, since waiting for its own slots would idle two of them. Rows -> slots, us:
  // 4096 x 32000 bf16 54 -> 107, x 65000 89 -> 110, x 100000 152 -> 150,
  // 2048 x 151936 111 -> 104.
  return StreamShape{ctas, static_cast<int>(share), rounds, !kPolicy && rounds > C::kSlots ? 1 : 0, kPieces, g_wait_ns, g_withheld};
}
StreamShape shape_for(int64_t cols, int elem_bytes, bool policy) {
  const int n = 16 / elem_bytes;
  const int64_t pieces = (cols + 2 * n - 2) / n;  // of a row that starts anywhere
  if (!policy) return shape_with<false, 4>(pieces, 1);
  int ctas = 1;
  while (ctas < kMaxCtas && (pieces + ctas - 1) / ctas * 16 > kMaxShare) ctas *= 2;
  // Slots of 10 KB, 22 of them; where they hold fewer than three rows, 17 of
  // 12.5 KB, which shares of 70 to 76 KB fill better: at 17 widths of that band
  // (600 MB of logits each) 14 were faster by 1 to 12%, one slower by 4%.
  // 10 -> 12.5 KB, us: bf16 x 36500 221 -> 205, x 38800 201 -> 198, x 72000
  // 211 -> 190, x 75000 207 -> 199, x 155000 210 -> 211, fp32 x 18000 218 -> 213,
  // x 38500 209 -> 197, x 72001 190 -> 197. Outside it: 4096 x 50001 bf16
  // 134 -> 144, x 40000 108 -> 116, 8192 x 32000 171 -> 174.
  const StreamShape s = shape_with<true, 4>(pieces, ctas);
  return 3 * s.rounds > Cfg<true, 4>::kSlots ? shape_with<true, 5>(pieces, ctas) : s;
}

// Clusters of `ctas` CTAs of one kernel that the device holds at a time, asked once per device.
template <typename T, bool kPolicy, int kPieces>
cudaError_t prepared_clusters(int ctas, int* clusters) {
  auto* kernel = stream_kernel<T, kPolicy, kPieces>;
  constexpr int kMaxDevices = 64;
  static std::mutex mu;
  static int known[kMaxDevices][kMaxCtas + 1] = {};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev < 0 || dev >= kMaxDevices) return cudaErrorInvalidDevice;
  std::lock_guard<std::mutex> lock(mu);
  if (!known[dev][ctas]) {
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kStreamSmem);
    if (e != cudaSuccess) return e;
    int most = 0;
    if (ctas == 1) {
      int sms = 0;
      e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
      most = sms;
    } else {
      cudaLaunchConfig_t cfg = {};
      cfg.gridDim = dim3(static_cast<unsigned>(ctas));
      cfg.blockDim = dim3(Cfg<kPolicy, kPieces>::kThreads);
      cfg.dynamicSmemBytes = kStreamSmem;
      cudaLaunchAttribute attr;
      attr.id = cudaLaunchAttributeClusterDimension;
      attr.val.clusterDim.x = static_cast<unsigned>(ctas);
      attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
      cfg.attrs = &attr;
      cfg.numAttrs = 1;
      e = cudaOccupancyMaxActiveClusters(&most, kernel, &cfg);
    }
    if (e != cudaSuccess) return e;
    if (most < 1) return cudaErrorInvalidConfiguration;
    known[dev][ctas] = most;
  }
  *clusters = known[dev][ctas];
  return cudaSuccess;
}

template <typename T, bool kPolicy, int kPieces>
cudaError_t launch(const RowArgs& a, const StreamShape& s, cudaStream_t st) {
  int clusters = 0;
  const cudaError_t e = prepared_clusters<T, kPolicy, kPieces>(s.ctas, &clusters);
  if (e != cudaSuccess) return e;
  if (clusters > a.rows) clusters = static_cast<int>(a.rows);
  return launch_pdl(stream_kernel<T, kPolicy, kPieces>, dim3(static_cast<unsigned>(clusters * s.ctas)),
                    dim3(Cfg<kPolicy, kPieces>::kThreads), kStreamSmem, st, s.ctas, a, s);
}
template <typename T>
cudaError_t launch(const RowArgs& a, bool policy, cudaStream_t st) {
  const StreamShape s = shape_for(a.cols, sizeof(T), policy);
  if (!policy) return launch<T, false, 4>(a, s, st);
  return s.pieces == 4 ? launch<T, true, 4>(a, s, st) : launch<T, true, 5>(a, s, st);
}

}  // namespace

// The other form holds a row in the registers of a CTA or a cluster, one row
// after another per CTA: less to set up for few or short rows, but nothing is
// loaded while a row is reduced and written. Measured, that form -> this one, us:
//   bf16 gradient   4096 x 16000 47.9 -> 59.0, x 24001 86.0 -> 72.9, x 32000 87.7 -> 91.3, x 50001 187 -> 133,
//                   608 x 32000 17.6 -> 20.5, 304 x 50001 17.2 -> 18.2, 608 x 50001 32.4 -> 28.8,
//                   152 x 100000 19.5 -> 20.1
//   fp32 gradient   4096 x 12000 72.1 -> 75.5, x 16000 87.2 -> 98.6, x 18000 112 -> 107, x 32000 187 -> 186
//   bf16 statistics 4096 x 16000 24.9 -> 32.0, x 24001 47.1 -> 41.9, x 32000 51.0 -> 45.6, x 50001 113 -> 72.2,
//                   608 x 32000 8.1 -> 10.4, 1216 x 32000 16.8 -> 16.6, 152 x 100000 11.0 -> 10.2
//   fp32 statistics 4096 x 12000 37.0 -> 34.5, x 16000 42.5 -> 41.7
bool stream_suits(int64_t rows, int64_t cols, int elem_bytes, bool policy) {
  const int64_t row_bytes = cols * elem_bytes;
  if (policy && shape_for(cols, elem_bytes, policy).rounds > Cfg<true, 5>::kSlots) return false;
  const int64_t least = policy && elem_bytes == 4 ? 66000 : 48000;
  return (row_bytes >= least && rows * row_bytes >= 50000000) || (row_bytes >= 192000 && rows >= 128);
}

void stream_wait(unsigned long long ns, int64_t withheld) {
  g_wait_ns = ns ? ns : kWaitNs;
  g_withheld = withheld;
}

cudaError_t launch_stream(const RowArgs& a, int type, bool policy, cudaStream_t st) {
  if (type == MEQ_F32) return launch<float>(a, policy, st);
  if (type == MEQ_BF16) return launch<__nv_bfloat16>(a, policy, st);
  return launch<__half>(a, policy, st);
}

}  // namespace loss
}  // namespace meq
