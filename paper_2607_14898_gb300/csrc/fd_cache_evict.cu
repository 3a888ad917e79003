// Eviction from a bounded cache by accumulated attention weight (fd_op_cache_insert,
// fd_op_cache_compact).
//
// Per list (one KV group of one stream) the n slots that rank first by (class, weight, slot)
// are given up: class 0 empty, 1 unprotected, 2 protected. A slot's rank key is 34 bits, class
// and the weight's bits made monotone; the n-th smallest key T is found by radix selection (class
// with 11 bits, then 11 and 10 bits), and of the slots whose key is T the first e in slot order are
// given up, so equal weights fall to the lowest index. (The first digit reaches two bits into
// the mantissa: with the class as bits of an 11-bit digit it ended at the exponent, most slots fell
// into some twenty counters, and counting them took longer than all else.) Keys are integers and
// counts are sums of integers: the choice does not depend on the order in which threads run. A
// scan of counts then gives every slot that is taken (or kept) its place in slot order, and its
// position, weight and row move, 16 bytes of a row a thread.
//
// One cluster of 1 to 8 CTAs of 1024 threads per list, in two forms:
//   short (up to kShortSlots): every CTA selects from the whole list by itself, keys in registers,
//     and writes its share of the slots. More reads from L2, but no exchange between CTAs,
//     whose steps (a cluster barrier and a round trip through distributed shared memory, four
//     times) take longer than all else in a list this size.
//   long: the list is cut between the CTAs, histograms are summed over the cluster through
//     distributed shared memory. Up to 24 keys a thread in registers; beyond that (196608 slots in 8
//     CTAs) they are read again for every digit.
// For one new token the selection is a minimum over (class, weight, slot) packed into 54 bits: the
// long form, with one exchange.
//
// Bound by memory for long rows (the copied keys and values) and by the latency of the dependent
// steps for short ones: the positions and weights of a list are 8 bytes a slot. Insert of one token
// into 32 lists of 6240 slots (3.2 MB): 5.4 us; of 1560 tokens (29 MB): 11.9 us, 2.4 TB/s; compact of 32
// lists of 32771 slots of 128 elements to 4099 (144 MB): 42 us, 3.4 TB/s, half of it the selection.
#include <cooperative_groups.h>

#include "fd_internal.h"
#include "fd_ptx.cuh"
#include "flashdec_ops.h"

namespace cg = cooperative_groups;

namespace fd {
namespace {

constexpr int kThreads = 1024;
constexpr int kWarps = kThreads / 32;
constexpr int kMaxSlots = 1 << 20;
constexpr int kMaxCluster = 8;
constexpr int kShortSlots = 8 * kThreads;
// Radix digits: class 0 is bin 0 of the first, classes 1 and 2 have 2048 bins each for bits 21..31 (the
// last of them is never used: the largest key, NaN, is below it); then bits 10..20 and 0..9.
constexpr int kBins0 = 4096, kBins1 = 2048, kBins2 = 1024;
constexpr int kHist = kBins0 + kBins1 + kBins2;

struct EvictParams {
  int groups, slots, n;      // slots looked at, slots given up, per list
  int iters;                 // slots of a thread (long form)
  int sinks, recent;
  const int32_t* newest;     // per stream, newest_stride apart: the position recency counts from
  int newest_stride;
  const int32_t* pos;        // list l starts at l * pitch
  const float* weight;
  int64_t pitch;
  int32_t* pos_out;
  float* weight_out;
  int64_t out_pitch;
  int32_t* list;             // slots taken / source slots, per list list_len entries
  int list_len;
  const int32_t* new_pos;    // insert: [streams][n]
  // rows: insert copies row v of new_k to slot list[v] of k, compact slot list[v] to row v
  const uint4 *src_k, *src_v;
  uint4 *dst_k, *dst_v;
  int64_t src_stream, src_group, src_row, dst_stream, dst_group, dst_row;  // in 16-byte units
  int row16;                 // 16-byte units of a row
};

// A slot's class and its weight's bits in ascending order: -0 is +0, NaN is the largest, an empty
// slot's weight does not count. protect >= 0.
struct Rank {
  uint32_t cls, low;
};
__device__ __forceinline__ Rank rank_of(int32_t pos, float w, int sinks, int protect) {
  uint32_t b = __float_as_uint(w);
  if (b == 0x80000000u) b = 0;
  b = w != w ? 0xffc00000u : (b & 0x80000000u ? ~b : b | 0x80000000u);
  if (pos < 0) return {0, 0};
  return {pos < sinks || pos >= protect ? 2u : 1u, b};
}
// The position from which entries are protected as recent (at least 0: below are empty ones).
__device__ __forceinline__ int protect_from(const EvictParams& p, int stream) {
  if (p.newest == nullptr) return 0;
  const int64_t x = static_cast<int64_t>(p.newest[static_cast<int64_t>(stream) * p.newest_stride]) -
                    p.recent;
  return x < 0 ? 0 : static_cast<int>(x);
}
// Once the class of the n-th key is known, 32 bits order the slots: classes before it are 0, it has
// the weight's bits (0 for class 0, never 0 or all ones for the others), classes after it, and
// places past the list's end (class 3), all ones.
__device__ __forceinline__ uint32_t order_of(Rank r, uint32_t cls) {
  return r.cls == cls ? r.low : (r.cls < cls ? 0u : 0xffffffffu);
}

// What has been found: slots with order below `limit` are given up, and of those at it the first
// `ties` in slot order, or all (then `all`). With n = 0: limit 0, no ties.
struct Cut {
  uint32_t cls, limit, ties;
  bool all;
  // whatever the other slots: given up, or (compact) kept
  template <bool COMPACT>
  __device__ __forceinline__ bool sure(uint32_t x, bool in) const {
    if (COMPACT) return in && x > limit;
    return in && (x < limit || (all && x == limit));
  }
  __device__ __forceinline__ bool tie(uint32_t x, bool in) const { return !all && in && x == limit; }
  // list entries among slots with na sure ones and nb ties
  template <bool COMPACT>
  __device__ __forceinline__ uint32_t place(uint32_t na, uint32_t nb) const {
    if (COMPACT) return na + (cls >= 1 && nb > ties ? nb - ties : 0u);
    return na + (nb < ties ? nb : ties);
  }
  template <bool COMPACT>
  __device__ __forceinline__ bool tie_in(uint32_t nb) const {  // nb ties before it
    return COMPACT ? cls >= 1 && nb >= ties : nb < ties;
  }
};

struct Found {
  uint32_t digit, rest, count;  // the bin, what is left to take in it, what it holds
};
// The bin that holds the rest-th item (1-based); c: counts of this thread's PER consecutive bins.
template <int PER>
__device__ __forceinline__ Found find_bin(const uint32_t (&c)[PER], uint32_t rest, uint32_t* sums,
                                          Found* out) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  uint32_t sum = 0;
#pragma unroll
  for (int j = 0; j < PER; ++j) sum += c[j];
  uint32_t x = sum;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const uint32_t y = __shfl_up_sync(0xffffffffu, x, d);
    if (lane >= d) x += y;
  }
  if (lane == 31) sums[warp] = x;
  __syncthreads();
  uint32_t s = sums[lane];
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const uint32_t y = __shfl_up_sync(0xffffffffu, s, d);
    if (lane >= d) s += y;
  }
  const int at = __ffs(__ballot_sync(0xffffffffu, s >= rest)) - 1;  // the warp that has it
  if (warp == at) {
    uint32_t before = __shfl_sync(0xffffffffu, s, at) - sums[at] + x - sum;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      if (before < rest && rest <= before + c[j])
        *out = {static_cast<uint32_t>(threadIdx.x * PER + j), rest - before, c[j]};
      before += c[j];
    }
  }
  __syncthreads();
  return *out;
}

// The three digits. count(pass, high): adds this CTA's slots to the pass's counters; share(): makes all
// CTAs' counters readable; add(h, c): adds the counters h of every CTA to this thread's c;
// settle(cls): called once the class is known.
struct Selector {
  uint32_t* hist;
  uint32_t* sums;
  Found* out;
  template <class Count, class Share, class Add, class Settle>
  __device__ __forceinline__ Cut run(uint32_t n, Count count, Share share, Add add, Settle settle) {
    Cut cut{0, 0, 0, false};
    if (n == 0) {
      settle(0u);
      return cut;
    }
    Found f;
    {
      uint32_t c[4] = {0, 0, 0, 0};
      count(0, 0u);
      share();
      add(hist, c);
      f = find_bin<4>(c, n, sums, out);
    }
    cut.cls = f.digit == 0 ? 0 : 1 + (f.digit - 1) / 2048;
    settle(cut.cls);
    if (cut.cls > 0) {
      uint32_t high = (f.digit - 1) % 2048;
      {
        uint32_t c[2] = {0, 0};
        count(1, high);
        share();
        add(hist + kBins0, c);
        f = find_bin<2>(c, f.rest, sums, out);
      }
      high = (high << 11) | f.digit;
      {
        uint32_t c[1] = {0};
        count(2, high);
        share();
        add(hist + kBins0 + kBins1, c);
        f = find_bin<1>(c, f.rest, sums, out);
      }
      cut.limit = (high << 10) | f.digit;
    }
    cut.all = f.rest == f.count;
    cut.ties = cut.all ? 0 : f.rest;
    // class 0 is all one key; with all of it given up the limit is below every kept slot
    return cut;
  }
};
__device__ __forceinline__ void count_class(uint32_t* hist, Rank r) {
  if (r.cls < 3) atomicAdd(hist + (r.cls == 0 ? 0 : 1 + (r.cls - 1) * 2048 + (r.low >> 21)), 1u);
}
__device__ __forceinline__ void count_order(uint32_t* hist, int pass, uint32_t high, uint32_t x) {
  if ((x >> (pass == 1 ? 21 : 10)) == high && x != 0xffffffffu)
    atomicAdd(hist + (pass == 1 ? kBins0 + ((x >> 10) & 0x7ff) : kBins0 + kBins1 + (x & 0x3ff)), 1u);
}
template <int PER>
__device__ __forceinline__ void add_bins(const uint32_t* h, uint32_t (&c)[PER]) {
  if constexpr (PER == 4) {
    const uint4 x = *reinterpret_cast<const uint4*>(h + 4 * threadIdx.x);
    c[0] += x.x, c[1] += x.y, c[2] += x.z, c[3] += x.w;
  } else if constexpr (PER == 2) {
    const uint2 x = *reinterpret_cast<const uint2*>(h + 2 * threadIdx.x);
    c[0] += x.x, c[1] += x.y;
  } else {
    c[0] += h[threadIdx.x];
  }
}

// Rows of the list entries [first, first + count): 16 bytes of a key and of a value per thread and
// step. slot_of(v): entry v's slot.
template <bool COMPACT, class SlotOf>
__device__ __forceinline__ void copy_rows(const EvictParams& p, int stream, int group,
                                          uint32_t first, uint32_t count, SlotOf slot_of) {
  const int64_t src0 = stream * p.src_stream + group * p.src_group;
  const int64_t dst0 = stream * p.dst_stream + group * p.dst_group;
  const int shift = p.row16 == 8 ? 3 : 4;  // 16-byte units of a row: 8 or 16
  const uint32_t items = count << shift;   // at most 2^24
  constexpr int kUnroll = 4;
  for (uint32_t it0 = threadIdx.x; it0 < items; it0 += kUnroll * kThreads) {
    uint4 xk[kUnroll], xv[kUnroll];
    int64_t to[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const uint32_t it = it0 + u * kThreads;
      if (it >= items) continue;
      const int64_t v = first + (it >> shift);
      const int part = static_cast<int>(it & (p.row16 - 1));
      const int64_t slot = slot_of(static_cast<uint32_t>(v));
      const int64_t from = src0 + (COMPACT ? slot : v) * p.src_row + part;
      to[u] = dst0 + (COMPACT ? v : slot) * p.dst_row + part;
      xk[u] = p.src_k[from];
      xv[u] = p.src_v[from];
    }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      if (it0 + u * kThreads >= items) continue;
      p.dst_k[to[u]] = xk[u];
      p.dst_v[to[u]] = xv[u];
    }
  }
}
// A compacted list's empty end: entries [kept, list_len), shared between the CTAs.
__device__ __forceinline__ void clear_end(const EvictParams& p, int lst, int stream, int group,
                                          uint32_t kept, int rank, int ctas) {
  int32_t* list = p.list + static_cast<int64_t>(lst) * p.list_len;
  const int64_t out_at = static_cast<int64_t>(lst) * p.out_pitch;
  const uint32_t first = kept + rank * kThreads + threadIdx.x;
  for (uint32_t v = first; v < static_cast<uint32_t>(p.list_len); v += ctas * kThreads) {
    list[v] = -1;
    p.pos_out[out_at + v] = -1;
    p.weight_out[out_at + v] = 0.f;
  }
  const int64_t dst0 = stream * p.dst_stream + group * p.dst_group;
  const int64_t end = (static_cast<int64_t>(p.list_len) - kept) * p.row16;
  const uint4 zero = make_uint4(0, 0, 0, 0);
  for (int64_t it = rank * kThreads + threadIdx.x; it < end; it += static_cast<int64_t>(ctas) * kThreads) {
    const int64_t to = dst0 + (kept + it / p.row16) * p.dst_row + it % p.row16;
    p.dst_k[to] = zero;
    p.dst_v[to] = zero;
  }
}

// ---------------------------------------------------------------- short lists
// Round r is slots 32 r .. 32 r + 31: for the selection warp w has rounds w, w + 32, .. of the whole
// list, for the writing CTA c of the cluster has an equal run of them, a warp per round.
template <int KPT, bool COMPACT>
__global__ void __launch_bounds__(kThreads, 1)
    evict_short_kernel(const __grid_constant__ EvictParams p) {
  constexpr int kRounds = KPT * kWarps;
  // counters, then the list of this CTA's share (all slots, where it is alone)
  constexpr int kShared = KPT * kThreads > kHist ? KPT * kThreads : kHist;
  __shared__ alignas(16) uint32_t hist[kShared];
  __shared__ uint32_t sums[kWarps], before_a[kRounds + 1], before_b[kRounds + 1];
  __shared__ Found found;
  cg::cluster_group cluster = cg::this_cluster();
  const int ctas = static_cast<int>(cluster.num_blocks());
  const int rank = static_cast<int>(cluster.block_rank());
  const int lst = blockIdx.x / ctas;
  const int stream = lst / p.groups, group = lst - stream * p.groups;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int64_t at = static_cast<int64_t>(lst) * p.pitch;
  for (int i = tid; i < kHist; i += kThreads) hist[i] = 0;
  grid_dep_wait();
  grid_dep_launch();
  const int protect = protect_from(p, stream);
  uint32_t low[KPT], cls = 0;
  {
    int32_t ps[KPT];
    float ws[KPT];
#pragma unroll
    for (int i = 0; i < KPT; ++i) {
      const int slot = i * kThreads + tid;
      ps[i] = slot < p.slots ? p.pos[at + slot] : 0;
      ws[i] = slot < p.slots ? p.weight[at + slot] : 0.f;
    }
#pragma unroll
    for (int i = 0; i < KPT; ++i) {
      Rank r = rank_of(ps[i], ws[i], p.sinks, protect);
      if (i * kThreads + tid >= p.slots) r.cls = 3;
      low[i] = r.low;
      cls |= r.cls << (2 * i);
    }
  }
  // positions and weights may be written in place: not before every CTA has read them
  __syncthreads();
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  Selector select{hist, sums, &found};
  const Cut cut = select.run(
      static_cast<uint32_t>(p.n),
      [&](int pass, uint32_t high) {
#pragma unroll
        for (int i = 0; i < KPT; ++i) {
          if (pass == 0) count_class(hist, {(cls >> (2 * i)) & 3u, low[i]});
          else count_order(hist, pass, high, low[i]);
        }
      },
      [] { __syncthreads(); }, [](const uint32_t* h, auto& c) { add_bins(h, c); },
      [&](uint32_t c) {
#pragma unroll
        for (int i = 0; i < KPT; ++i) low[i] = order_of({(cls >> (2 * i)) & 3u, low[i]}, c);
      });
  // counts of every round, then of all rounds before it
#pragma unroll
  for (int i = 0; i < KPT; ++i) {
    const bool in = i * kThreads + tid < p.slots;
    const uint32_t a = __ballot_sync(0xffffffffu, cut.sure<COMPACT>(low[i], in));
    const uint32_t b = __ballot_sync(0xffffffffu, cut.tie(low[i], in));
    if (lane == 0) {
      before_a[i * kWarps + warp] = __popc(a);
      before_b[i * kWarps + warp] = __popc(b);
    }
  }
  __syncthreads();
  if (warp == 0) {  // kRounds / 32 entries a lane
    uint32_t a[KPT], b[KPT], sa = 0, sb = 0;
#pragma unroll
    for (int i = 0; i < KPT; ++i) {
      a[i] = before_a[lane * KPT + i];
      b[i] = before_b[lane * KPT + i];
      sa += a[i];
      sb += b[i];
    }
    uint32_t xa = sa, xb = sb;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const uint32_t ya = __shfl_up_sync(0xffffffffu, xa, d), yb = __shfl_up_sync(0xffffffffu, xb, d);
      if (lane >= d) {
        xa += ya;
        xb += yb;
      }
    }
    if (lane == 31) {
      before_a[kRounds] = xa;
      before_b[kRounds] = xb;
    }
    xa -= sa;
    xb -= sb;
#pragma unroll
    for (int i = 0; i < KPT; ++i) {
      before_a[lane * KPT + i] = xa;
      before_b[lane * KPT + i] = xb;
      xa += a[i];
      xb += b[i];
    }
  }
  __syncthreads();
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");

  // ---- this CTA's rounds
  const int rounds = (p.slots + 31) / 32;
  const int r0 = rounds * rank / ctas, r1 = rounds * (rank + 1) / ctas;
  const uint32_t first = cut.place<COMPACT>(before_a[r0], before_b[r0]);
  const uint32_t count = cut.place<COMPACT>(before_a[r1], before_b[r1]) - first;
  const uint32_t kept = cut.place<COMPACT>(before_a[kRounds], before_b[kRounds]);
  const bool copy_pos = p.pos_out != p.pos, copy_weight = p.weight_out != p.weight;
  const int32_t* np = p.new_pos ? p.new_pos + static_cast<int64_t>(stream) * p.n : nullptr;
  int32_t* list = p.list + static_cast<int64_t>(lst) * p.list_len;
  const int64_t out_at = static_cast<int64_t>(lst) * p.out_pitch;
  constexpr int kGroup = 2;
  for (int ra = r0 + warp; ra < r1; ra += kGroup * kWarps) {
    int32_t ps[kGroup];
    float ws[kGroup];
#pragma unroll
    for (int u = 0; u < kGroup; ++u) {
      const int r = ra + u * kWarps, slot = 32 * r + lane;
      const bool in = r < r1 && slot < p.slots;
      ps[u] = in ? p.pos[at + slot] : 0;
      ws[u] = in ? p.weight[at + slot] : 0.f;
    }
#pragma unroll
    for (int u = 0; u < kGroup; ++u) {
      const int r = ra + u * kWarps, slot = 32 * r + lane;
      if (r >= r1) break;
      const bool in = slot < p.slots;
      const uint32_t x = order_of(rank_of(ps[u], ws[u], p.sinks, protect), cut.cls);
      const uint32_t a = __ballot_sync(0xffffffffu, cut.sure<COMPACT>(x, in));
      const uint32_t b = __ballot_sync(0xffffffffu, cut.tie(x, in));
      const uint32_t below = (1u << lane) - 1;
      const uint32_t na = before_a[r] + __popc(a & below), nb = before_b[r] + __popc(b & below);
      const bool take = ((a >> lane) & 1u) || (((b >> lane) & 1u) && cut.tie_in<COMPACT>(nb));
      const uint32_t v = cut.place<COMPACT>(na, nb);
      if (take) {
        list[v] = slot;
        hist[v - first] = slot;
      }
      if (COMPACT) {
        if (take) {
          p.pos_out[out_at + v] = ps[u];
          p.weight_out[out_at + v] = ws[u];
        }
      } else if (in) {
        if (take || copy_pos) p.pos_out[out_at + slot] = take ? np[v] : ps[u];
        if (take || copy_weight) p.weight_out[out_at + slot] = take ? 0.f : ws[u];
      }
    }
  }
  __syncthreads();
  copy_rows<COMPACT>(p, stream, group, first, count,
                     [&](uint32_t v) { return static_cast<int64_t>(hist[v - first]); });
  if (COMPACT) clear_end(p, lst, stream, group, kept, rank, ctas);
}

// ---------------------------------------------------------------- long lists, and one new token
// The keys of a thread: KPT in registers, or (0) read again for every use. Warps hold consecutive
// slots: the thread's i-th is slot0 + 32 i.
struct LongShared {
  alignas(16) uint32_t hist[kHist];
  uint32_t sums[kWarps], warp_a[kWarps], warp_b[kWarps];
  uint64_t warp_min[kWarps], cta_min;
  uint32_t cta_a, cta_b;
  Found found;
};

template <int KPT, bool COMPACT>
__global__ void __launch_bounds__(kThreads, 1)
    evict_long_kernel(const __grid_constant__ EvictParams p) {
  __shared__ LongShared sm;
  cg::cluster_group cluster = cg::this_cluster();
  const int ctas = static_cast<int>(cluster.num_blocks());
  const int rank = static_cast<int>(cluster.block_rank());
  const int lst = blockIdx.x / ctas;
  const int stream = lst / p.groups, group = lst - stream * p.groups;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int iters = p.iters;
  const int slot0 = (rank * kWarps + warp) * 32 * iters + lane;
  const int64_t at = static_cast<int64_t>(lst) * p.pitch;
  for (int i = tid; i < kHist; i += kThreads) sm.hist[i] = 0;
  grid_dep_wait();
  grid_dep_launch();
  const int protect = protect_from(p, stream);
  constexpr int kRegs = KPT > 0 ? KPT : 1, kGroup = KPT >= 4 || KPT == 0 ? 4 : 2;
  uint32_t low[kRegs];
  uint64_t cls = 0;
  if (KPT > 0) {
#pragma unroll
    for (int i0 = 0; i0 < KPT; i0 += kGroup) {
      int32_t ps[kGroup];
      float ws[kGroup];
#pragma unroll
      for (int u = 0; u < kGroup; ++u) {
        const int slot = slot0 + 32 * (i0 + u);
        const bool in = i0 + u < iters && slot < p.slots;
        ps[u] = in ? p.pos[at + slot] : 0;
        ws[u] = in ? p.weight[at + slot] : 0.f;
      }
#pragma unroll
      for (int u = 0; u < kGroup; ++u) {
        const int i = i0 + u;
        Rank r = rank_of(ps[u], ws[u], p.sinks, protect);
        if (i >= iters || slot0 + 32 * i >= p.slots) r.cls = 3;
        low[i % kRegs] = r.low;
        cls |= static_cast<uint64_t>(r.cls) << (2 * i);
      }
    }
  }
  auto rank_at = [&](int i) -> Rank {
    if (KPT > 0) return {static_cast<uint32_t>(cls >> (2 * i)) & 3u, low[i % kRegs]};
    const int slot = slot0 + 32 * i;
    if (slot >= p.slots) return {3, 0};
    return rank_of(p.pos[at + slot], p.weight[at + slot], p.sinks, protect);
  };
#define FOR_KEYS(i) _Pragma("unroll") for (int i = 0; i < (KPT > 0 ? KPT : iters); ++i) if (KPT == 0 || i < iters)
  int32_t* list = p.list + static_cast<int64_t>(lst) * p.list_len;
  const int64_t out_at = static_cast<int64_t>(lst) * p.out_pitch;
  const int32_t* np = p.new_pos ? p.new_pos + static_cast<int64_t>(stream) * p.n : nullptr;
  const bool copy_pos = p.pos_out != p.pos, copy_weight = p.weight_out != p.weight;
  uint32_t first = 0, count = 0, kept = 0;  // this CTA's list entries; all of the list's
  if (!COMPACT && p.n == 1) {
    uint64_t best = ~0ull;
    FOR_KEYS(i) {
      const Rank r = rank_at(i);
      const uint64_t k = (static_cast<uint64_t>(r.cls) << 52) | (static_cast<uint64_t>(r.low) << 20) |
                         static_cast<uint32_t>(slot0 + 32 * i);
      if (r.cls < 3 && k < best) best = k;
    }
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) {
      const uint64_t o = __shfl_xor_sync(0xffffffffu, best, d);
      best = o < best ? o : best;
    }
    if (lane == 0) sm.warp_min[warp] = best;
    __syncthreads();
    if (warp == 0) {
      best = sm.warp_min[lane];
#pragma unroll
      for (int d = 16; d > 0; d >>= 1) {
        const uint64_t o = __shfl_xor_sync(0xffffffffu, best, d);
        best = o < best ? o : best;
      }
      if (lane == 0) sm.cta_min = best;
    }
    cluster.sync();
    best = ~0ull;
#pragma unroll
    for (int c = 0; c < kMaxCluster; ++c)
      if (c < ctas) {
        const uint64_t o = *cluster.map_shared_rank(&sm.cta_min, c);
        best = o < best ? o : best;
      }
    const int only = static_cast<int>(best & (kMaxSlots - 1));
    FOR_KEYS(i) {
      const int slot = slot0 + 32 * i;
      if (slot < p.slots) {
        const bool take = slot == only;
        if (take || copy_pos) p.pos_out[out_at + slot] = take ? np[0] : p.pos[at + slot];
        if (take || copy_weight) p.weight_out[out_at + slot] = take ? 0.f : p.weight[at + slot];
        if (take) list[0] = slot;
      }
    }
    // the CTA that holds the slot moves the row
    const int base = rank * kWarps * 32 * iters;
    if (only >= base && only < base + kWarps * 32 * iters) count = 1;
  } else {
    __syncthreads();
    Selector select{sm.hist, sm.sums, &sm.found};
    uint32_t settled = 0;
    const Cut cut = select.run(
        static_cast<uint32_t>(p.n),
        [&](int pass, uint32_t high) {
          FOR_KEYS(i) {
            if (pass == 0) count_class(sm.hist, rank_at(i));
            else count_order(sm.hist, pass, high, KPT > 0 ? low[i % kRegs] : order_of(rank_at(i), settled));
          }
        },
        [&] { cluster.sync(); },
        [&](const uint32_t* h, auto& c) {
#pragma unroll
          for (int r = 0; r < kMaxCluster; ++r)
            if (r < ctas) add_bins(cluster.map_shared_rank(h, r), c);
        },
        [&](uint32_t c) {
          settled = c;
          if (KPT > 0) FOR_KEYS(i) low[i % kRegs] = order_of(rank_at(i), c);
        });
    auto order_at = [&](int i) -> uint32_t {
      return KPT > 0 ? low[i % kRegs] : order_of(rank_at(i), settled);
    };
    // counts of this warp, of the warps before it, and of the CTAs before this one
    uint32_t a = 0, b = 0;
    FOR_KEYS(i) {
      const bool in = slot0 + 32 * i < p.slots;
      const uint32_t x = order_at(i);
      a += cut.sure<COMPACT>(x, in);
      b += cut.tie(x, in);
    }
    a = __reduce_add_sync(0xffffffffu, a);
    b = __reduce_add_sync(0xffffffffu, b);
    if (lane == 0) {
      sm.warp_a[warp] = a;
      sm.warp_b[warp] = b;
    }
    __syncthreads();
    uint32_t na = sm.warp_a[lane], nb = sm.warp_b[lane];
    const uint32_t ca = __reduce_add_sync(0xffffffffu, na), cb = __reduce_add_sync(0xffffffffu, nb);
    na = __reduce_add_sync(0xffffffffu, lane < warp ? na : 0u);
    nb = __reduce_add_sync(0xffffffffu, lane < warp ? nb : 0u);
    if (tid == 0) {
      sm.cta_a = ca;
      sm.cta_b = cb;
    }
    cluster.sync();
    uint32_t front_a = 0, front_b = 0, all_a = 0, all_b = 0;
#pragma unroll
    for (int r = 0; r < kMaxCluster; ++r)
      if (r < ctas) {
        const uint32_t ra = *cluster.map_shared_rank(&sm.cta_a, r);
        const uint32_t rb = *cluster.map_shared_rank(&sm.cta_b, r);
        front_a += r < rank ? ra : 0;
        front_b += r < rank ? rb : 0;
        all_a += ra;
        all_b += rb;
      }
    first = cut.place<COMPACT>(front_a, front_b);
    count = cut.place<COMPACT>(front_a + ca, front_b + cb) - first;
    kept = cut.place<COMPACT>(all_a, all_b);
    na += front_a;
    nb += front_b;
    // positions and weights a group ahead, so that no load waits for the store before it
#pragma unroll
    for (int i0 = 0; i0 < (KPT > 0 ? KPT : iters); i0 += kGroup) {
      if (i0 >= iters) break;
      int32_t ps[kGroup];
      float ws[kGroup];
      uint32_t xs[kGroup];
#pragma unroll
      for (int u = 0; u < kGroup; ++u) {
        const int i = i0 + u, slot = slot0 + 32 * i;
        const bool in = i < iters && slot < p.slots;
        ps[u] = in && (COMPACT || copy_pos) ? p.pos[at + slot] : 0;
        ws[u] = in && (COMPACT || copy_weight) ? p.weight[at + slot] : 0.f;
        xs[u] = i < iters ? order_at(i) : 0xffffffffu;
      }
#pragma unroll
      for (int u = 0; u < kGroup; ++u) {
        const int i = i0 + u, slot = slot0 + 32 * i;
        if (i >= iters) break;
        const bool in = slot < p.slots;
        const uint32_t ma = __ballot_sync(0xffffffffu, cut.sure<COMPACT>(xs[u], in));
        const uint32_t mb = __ballot_sync(0xffffffffu, cut.tie(xs[u], in));
        const uint32_t below = (1u << lane) - 1;
        const uint32_t la = na + __popc(ma & below), lb = nb + __popc(mb & below);
        const bool take = ((ma >> lane) & 1u) || (((mb >> lane) & 1u) && cut.tie_in<COMPACT>(lb));
        const uint32_t v = cut.place<COMPACT>(la, lb);
        if (take) list[v] = slot;
        if (COMPACT) {
          if (take) {
            p.pos_out[out_at + v] = ps[u];
            p.weight_out[out_at + v] = ws[u];
          }
        } else if (in) {
          if (take || copy_pos) p.pos_out[out_at + slot] = take ? np[v] : ps[u];
          if (take || copy_weight) p.weight_out[out_at + slot] = take ? 0.f : ws[u];
        }
        na += __popc(ma);
        nb += __popc(mb);
      }
    }
  }
#undef FOR_KEYS
  __syncthreads();  // this CTA's part of the list is written
  copy_rows<COMPACT>(p, stream, group, first, count,
                     [&](uint32_t v) { return static_cast<int64_t>(list[v]); });
  if (COMPACT) clear_end(p, lst, stream, group, kept, rank, ctas);
  cluster.sync();  // no CTA leaves while another may still read its shared memory
}

cudaError_t launch_cluster(void (*kernel)(EvictParams), const EvictParams& p, int lists, int ctas,
                           cudaStream_t s) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(lists) * ctas);
  cfg.blockDim = dim3(kThreads);
  cfg.stream = s;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = ctas;
  at[1].val.clusterDim.y = 1;
  at[1].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, kernel, p);
}

// CTAs of a cluster: as many as keep the lists' clusters on the GPU at once, but no fewer than 512
// (short form) or 1024 slots each: below that the cluster's barriers cost more than the shorter loops
// save. Device times in us at 512 / 1024 / 2048 slots each: compact of 4 lists of 2000 slots to 500
// 6.1 / 7.0 / 8.7, of 6240 to 1560 9.0 / 9.0 / 10.4; insert of one into 32 lists of 1500 slots
// 4.9 / 4.2 / 4.8.
// Short form or long, same cases: compact of 2000 7.0 / 14.5, of 6240 9.0 / 21.2, insert of 1560 into 32
// lists of 6240 11.9 / 16.4. Insert of one in the short form: 9.0 for 32 lists of 6240, 5.4 in the
// long one. Keys of a thread: 2 against 8 (short, 2000 slots) 7.0 / 9.2, 2 against 12 (long, insert of
// one into 32 x 6240) 5.4 / 8.5, 12 / 24 / read again (compact of 32 lists of 32771) 42 / 49 / 57.
template <bool COMPACT>
cudaError_t launch(EvictParams& p, int lists, cudaStream_t s) {
  const bool is_short = p.slots <= kShortSlots && (COMPACT || p.n != 1);
  int ctas = 1;
  while (ctas < kMaxCluster && 2 * ctas * static_cast<int64_t>(lists) <= num_sms() &&
         p.slots > (is_short ? 512 : 1024) * ctas)
    ctas *= 2;
  if (is_short) {
    if (p.slots <= 2 * kThreads)
      return launch_cluster(evict_short_kernel<2, COMPACT>, p, lists, ctas, s);
    return launch_cluster(evict_short_kernel<8, COMPACT>, p, lists, ctas, s);
  }
  const int per = kThreads * ctas;
  p.iters = (p.slots + per - 1) / per;
  if (p.iters < 1) p.iters = 1;
  // (one token's insert as a rule; other lists come here from 8193 slots on, 2 a thread in 8 CTAs)
  if constexpr (!COMPACT)
    if (p.iters <= 2) return launch_cluster(evict_long_kernel<2, false>, p, lists, ctas, s);
  if (p.iters <= 12) return launch_cluster(evict_long_kernel<12, COMPACT>, p, lists, ctas, s);
  if (p.iters <= 24) return launch_cluster(evict_long_kernel<24, COMPACT>, p, lists, ctas, s);
  return launch_cluster(evict_long_kernel<0, COMPACT>, p, lists, ctas, s);
}

bool aligned(const void* x, uintptr_t a) { return reinterpret_cast<uintptr_t>(x) % a == 0; }

}  // namespace

bool valid_cache(const fd_cache* c) {
  if (c == nullptr || c->streams < 0 || c->groups < 1 || c->capacity < 0 || c->reserved != 0)
    return false;
  if (c->capacity > kMaxSlots || c->groups > 65536 ||
      static_cast<int64_t>(c->streams) * c->groups > (1 << 24))
    return false;
  if (c->head_dim != 64 && c->head_dim != 128) return false;
  if (c->dtype != FD_DTYPE_BF16 && c->dtype != FD_DTYPE_F16) return false;
  // (lists that share rows have no meaning: an insert would write them twice)
  if (c->slot_stride < c->head_dim || (c->streams > 1 && c->stream_stride < c->head_dim) ||
      (c->groups > 1 && c->group_stride < c->head_dim) || c->stream_stride < 0 ||
      c->group_stride < 0 || c->stream_stride % 8 || c->group_stride % 8 || c->slot_stride % 8)
    return false;
  if (c->streams == 0 || c->capacity == 0) return true;
  return c->k && c->v && c->pos && c->weight && aligned(c->k, 16) && aligned(c->v, 16) &&
         aligned(c->pos, 4) && aligned(c->weight, 4);
}

}  // namespace fd

extern "C" {

fd_status fd_op_cache_insert(const fd_cache* cache, int n_new, const void* k_new,
                             const void* v_new, int64_t new_stream_stride,
                             int64_t new_token_stride, int64_t new_group_stride,
                             const int32_t* new_pos, int sinks, int recent, int32_t* pos_out,
                             float* weight_out, int32_t* slots, void* stream) {
  if (!fd::valid_cache(cache) || n_new < 0 || n_new > cache->capacity || sinks < 0 || recent < 0)
    return FD_ERR_INVALID_ARG;
  const int lists = cache->streams * cache->groups;
  if (lists == 0 || cache->capacity == 0) return FD_OK;
  if (!pos_out || !weight_out || !fd::aligned(pos_out, 4) || !fd::aligned(weight_out, 4))
    return FD_ERR_INVALID_ARG;
  if (n_new > 0 &&
      (!k_new || !v_new || !new_pos || !slots || !fd::aligned(k_new, 16) ||
       !fd::aligned(v_new, 16) || !fd::aligned(new_pos, 4) || !fd::aligned(slots, 4) ||
       new_stream_stride % 8 || new_token_stride % 8 || new_group_stride % 8))
    return FD_ERR_INVALID_ARG;
  if (n_new == 0 && pos_out == cache->pos && weight_out == cache->weight) return FD_OK;
  const fd_status st = fd::check_device();
  if (st != FD_OK) return st;
  fd::EvictParams p{};
  p.groups = cache->groups;
  p.slots = cache->capacity;
  p.n = n_new;
  p.sinks = sinks;
  p.recent = recent;
  p.newest = n_new > 0 ? new_pos : nullptr;
  p.newest_stride = n_new;
  p.pos = cache->pos;
  p.weight = cache->weight;
  p.pitch = cache->capacity;
  p.pos_out = pos_out;
  p.weight_out = weight_out;
  p.out_pitch = cache->capacity;
  p.list = slots;
  p.list_len = n_new;
  p.new_pos = new_pos;
  p.src_k = static_cast<const uint4*>(k_new);
  p.src_v = static_cast<const uint4*>(v_new);
  p.dst_k = static_cast<uint4*>(cache->k);
  p.dst_v = static_cast<uint4*>(cache->v);
  p.src_stream = new_stream_stride / 8;
  p.src_group = new_group_stride / 8;
  p.src_row = new_token_stride / 8;
  p.dst_stream = cache->stream_stride / 8;
  p.dst_group = cache->group_stride / 8;
  p.dst_row = cache->slot_stride / 8;
  p.row16 = cache->head_dim / 8;
  return fd::launch<false>(p, lists, static_cast<cudaStream_t>(stream)) == cudaSuccess
             ? FD_OK
             : FD_ERR_CUDA;
}

fd_status fd_op_cache_compact(const fd_cache* src, int used, const fd_cache* dst,
                              const int32_t* now, int sinks, int recent, int32_t* src_slots,
                              void* stream) {
  if (!fd::valid_cache(src) || !fd::valid_cache(dst) || used < 0 || used > src->capacity ||
      dst->capacity > used || sinks < 0 || recent < 0)
    return FD_ERR_INVALID_ARG;
  if (src->streams != dst->streams || src->groups != dst->groups ||
      src->head_dim != dst->head_dim || src->dtype != dst->dtype)
    return FD_ERR_INVALID_ARG;
  const int lists = src->streams * src->groups;
  if (lists == 0 || dst->capacity == 0) return FD_OK;
  if (!now || !src_slots || !fd::aligned(now, 4) || !fd::aligned(src_slots, 4) ||
      src->k == dst->k || src->v == dst->v || src->pos == dst->pos || src->weight == dst->weight)
    return FD_ERR_INVALID_ARG;
  const fd_status st = fd::check_device();
  if (st != FD_OK) return st;
  fd::EvictParams p{};
  p.groups = src->groups;
  p.slots = used;
  p.n = used - dst->capacity;
  p.sinks = sinks;
  p.recent = recent;
  p.newest = now;
  p.newest_stride = 1;
  p.pos = src->pos;
  p.weight = src->weight;
  p.pitch = src->capacity;
  p.pos_out = dst->pos;
  p.weight_out = dst->weight;
  p.out_pitch = dst->capacity;
  p.list = src_slots;
  p.list_len = dst->capacity;
  p.src_k = static_cast<const uint4*>(src->k);
  p.src_v = static_cast<const uint4*>(src->v);
  p.dst_k = static_cast<uint4*>(dst->k);
  p.dst_v = static_cast<uint4*>(dst->v);
  p.src_stream = src->stream_stride / 8;
  p.src_group = src->group_stride / 8;
  p.src_row = src->slot_stride / 8;
  p.dst_stream = dst->stream_stride / 8;
  p.dst_group = dst->group_stride / 8;
  p.dst_row = dst->slot_stride / 8;
  p.row16 = src->head_dim / 8;
  return fd::launch<true>(p, lists, static_cast<cudaStream_t>(stream)) == cudaSuccess
             ? FD_OK
             : FD_ERR_CUDA;
}

}  // extern "C"
