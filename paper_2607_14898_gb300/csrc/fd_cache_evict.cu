// Eviction from a bounded cache by accumulated attention weight (fd_op_cache_insert,
// fd_op_cache_compact).
//
// Per list (one KV group of one stream) the n slots that rank first by (class, weight, slot)
// are given up: class 0 empty, 1 unprotected, 2 protected. A slot's rank key is 34 bits, class
// and the weight's bits made monotone; the n-th smallest key T is found by radix selection (class
// with 11 bits, then 11 and 10 bits), and of the slots whose key is T the first e in slot order are
// given up, so equal weights fall to the lowest index. (The first digit reaches two bits into
// the mantissa: with the class as bits of the digit it ended at the exponent, most slots fell
// into some twenty counters, and counting them took longer than all else.) Keys are integers and counts are sums of
// integers: the choice does not depend on the order in which threads run.
//
// One cluster of 1 to 8 CTAs per list. Keys are read once into registers, each warp
// holding consecutive slots, and histograms are counted in shared memory. Up to kAloneSlots every
// CTA of the cluster selects from the whole list by itself, and the cluster only shares the
// writing: more reads from L2, but no exchange, whose steps (a cluster barrier and a round
// trip through distributed shared memory, three times) took longer than the rest. Longer lists are
// cut between the CTAs and the histograms summed over the cluster. One scan of counts over
// warps (and CTAs) gives every slot that is taken (or kept) its place in slot order. Then the
// cluster writes the list's positions and weights and moves the rows, 16 bytes a thread. For one
// new token the selection is a minimum over (class, weight, slot) packed into 54 bits, one exchange
// only, so there the list is always cut.
//
// Bound by memory for long rows (the copied keys and values) and by the latency of the dependent steps for
// short ones: the positions and weights of a list are 8 bytes a slot.
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
constexpr int kMaxKeys = 32;  // keys a thread holds in registers
constexpr int kAloneSlots = 8 * kThreads;
// Radix digits: class 0 is bin 0 of the first, classes 1 and 2 have 2048 bins each for bits 21..31 (the
// last of them is never used: the largest key, NaN, is below it); then bits 10..20 and 0..9.
constexpr int kBins0 = 4096, kBins1 = 2048, kBins2 = 1024;
constexpr int kHist = kAloneSlots;  // counters; afterwards the list of a CTA that selects alone
static_assert(kBins0 + kBins1 + kBins2 <= kHist, "counters");

struct EvictParams {
  int groups, slots, n;      // slots looked at, slots given up, per list
  int iters;                 // slots a thread has: kThreads * iters (* cluster size) >= slots
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

// rank key: class in bits 32.., the weight's bits in ascending order below. -0 is +0, NaN is the
// largest; an empty slot's weight does not count.
__device__ __forceinline__ uint64_t rank_key(int32_t pos, float w, int sinks, int64_t protect) {
  if (pos < 0) return 0;
  uint32_t b = __float_as_uint(w);
  if (b == 0x80000000u) b = 0;
  b = w != w ? 0xffc00000u : (b & 0x80000000u ? ~b : b | 0x80000000u);
  const uint64_t cls = pos < sinks || pos >= protect ? 2 : 1;
  return (cls << 32) | b;
}

// The keys of a thread: in registers (KPT > 0), or read again for every use (long lists).
template <int KPT>
struct Keys {
  uint32_t low[KPT];
  uint64_t cls;  // 2 bits each, 3: past the end of the list
  __device__ __forceinline__ void load(const EvictParams& p, int64_t at, int slot0, int64_t protect) {
    cls = ~0ull;
    int32_t ps[KPT];
    float ws[KPT];
#pragma unroll
    for (int i = 0; i < KPT; ++i) {
      const int slot = slot0 + 32 * i;
      const bool in = i < p.iters && slot < p.slots;
      ps[i] = in ? p.pos[at + slot] : 0;
      ws[i] = in ? p.weight[at + slot] : 0.f;
    }
#pragma unroll
    for (int i = 0; i < KPT; ++i) {
      const uint64_t key = rank_key(ps[i], ws[i], p.sinks, protect);
      low[i] = static_cast<uint32_t>(key);
      if (i < p.iters && slot0 + 32 * i < p.slots)
        cls ^= (3ull ^ (key >> 32)) << (2 * i);
    }
  }
  __device__ __forceinline__ uint64_t get(const EvictParams&, int64_t, int, int64_t, int i) const {
    return (((cls >> (2 * i)) & 3ull) << 32) | low[i];
  }
};
template <>
struct Keys<0> {
  __device__ __forceinline__ void load(const EvictParams&, int64_t, int, int64_t) {}
  __device__ __forceinline__ uint64_t get(const EvictParams& p, int64_t at, int slot0,
                                          int64_t protect, int i) const {
    const int slot = slot0 + 32 * i;
    return slot < p.slots ? rank_key(p.pos[at + slot], p.weight[at + slot], p.sinks, protect)
                          : 3ull << 32;
  }
};

struct Shared {
  alignas(16) uint32_t hist[kHist];
  uint32_t warp_a[kWarps], warp_b[kWarps];
  uint64_t warp_min[kWarps];
  uint64_t cta_min;
  uint32_t cta_a, cta_b;
  uint32_t digit, rest, found;  // the radix pass's result
};

// exclusive prefix of v over the block's threads (and the total)
__device__ __forceinline__ uint32_t block_scan(uint32_t v, uint32_t* warp_sums, uint32_t* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  uint32_t x = v;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const uint32_t y = __shfl_up_sync(0xffffffffu, x, d);
    if (lane >= d) x += y;
  }
  if (lane == 31) warp_sums[warp] = x;
  __syncthreads();
  uint32_t s = warp_sums[lane];
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const uint32_t y = __shfl_up_sync(0xffffffffu, s, d);
    if (lane >= d) s += y;
  }
  *total = __shfl_sync(0xffffffffu, s, 31);
  const uint32_t before = __shfl_sync(0xffffffffu, s, warp == 0 ? 0 : warp - 1);
  __syncthreads();
  return (warp == 0 ? 0 : before) + x - v;
}

// COMPACT: the slots that are not given up go to the destination; else the given-up slots are
// taken by new tokens. ALONE: each CTA selects from the whole list, and writes for its share of
// the warps.
template <int KPT, bool COMPACT, bool ALONE>
__global__ void __launch_bounds__(kThreads, 1) evict_kernel(const __grid_constant__ EvictParams p) {
  __shared__ Shared sm;
  cg::cluster_group cluster = cg::this_cluster();
  const int ctas = static_cast<int>(cluster.num_blocks());
  const int rank = static_cast<int>(cluster.block_rank());
  const int lst = blockIdx.x / ctas;
  const int stream = lst / p.groups, group = lst - stream * p.groups;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int iters = p.iters;
  const int slot0 = ((ALONE ? 0 : rank * kWarps) + warp) * 32 * iters + lane;  // i-th: + 32 i
  const int64_t at = static_cast<int64_t>(lst) * p.pitch;

  for (int i = tid; i < kBins0 + kBins1 + kBins2; i += kThreads) sm.hist[i] = 0;
  grid_dep_wait();
  grid_dep_launch();
  const int64_t protect =
      static_cast<int64_t>(p.newest ? p.newest[static_cast<int64_t>(stream) * p.newest_stride] : 0) -
      p.recent;
  Keys<KPT> keys;
  keys.load(p, at, slot0, protect);
  // positions and weights may be written in place: not before every CTA has read them
  if (ALONE) {
    __syncthreads();
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  }
  auto key_of = [&](int i) { return keys.get(p, at, slot0, protect, i); };
#define FOR_KEYS(i) _Pragma("unroll") for (int i = 0; i < (KPT > 0 ? KPT : iters); ++i) if (KPT == 0 || i < iters)

  uint64_t limit = 0;   // T: the n-th smallest key
  uint32_t ties = 0;    // e: so many of the slots with key T are given up
  int only = -1;        // the slot, where a minimum tells it
  if (!COMPACT && !ALONE && p.n == 1) {
    uint64_t best = ~0ull;
    FOR_KEYS(i) {
      const uint64_t k = (key_of(i) << 20) | static_cast<uint32_t>(slot0 + 32 * i);
      if (slot0 + 32 * i < p.slots && k < best) best = k;
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
    only = static_cast<int>(best & (kMaxSlots - 1));
  } else if (p.n > 0) {
    __syncthreads();
    uint32_t rest = static_cast<uint32_t>(p.n);
    uint64_t high = 0;  // the digits found so far, in their places
#pragma unroll
    for (int pass = 0; pass < 3; ++pass) {
      if (pass > 0 && high == 0) break;  // class 0: equal keys
      uint32_t* hist = sm.hist + (pass == 0 ? 0 : pass == 1 ? kBins0 : kBins0 + kBins1);
      FOR_KEYS(i) {
        const uint64_t k = key_of(i);
        const uint32_t cls = static_cast<uint32_t>(k >> 32), low = static_cast<uint32_t>(k);
        if (pass == 0 ? cls < 3 : (k >> (pass == 1 ? 21 : 10)) == high)
          atomicAdd(hist + (pass == 0 ? (cls == 0 ? 0 : 1 + (cls - 1) * 2048 + (low >> 21))
                                      : pass == 1 ? (low >> 10) & 0x7ff : low & 0x3ff), 1u);
      }
      constexpr int kPer[3] = {kBins0 / kThreads, kBins1 / kThreads, kBins2 / kThreads};
      const int per = kPer[pass];  // 4, 2 or 1 bins a thread
      uint32_t c[4] = {0, 0, 0, 0}, sum = 0;
      auto add = [&](const uint32_t* h) {
        if (per == 4) {
          const uint4 x = *reinterpret_cast<const uint4*>(h + 4 * tid);
          c[0] += x.x, c[1] += x.y, c[2] += x.z, c[3] += x.w;
        } else if (per == 2) {
          const uint2 x = *reinterpret_cast<const uint2*>(h + 2 * tid);
          c[0] += x.x, c[1] += x.y;
        } else {
          c[0] += h[tid];
        }
      };
      if (ALONE) {
        __syncthreads();
        add(hist);
      } else {
        cluster.sync();
#pragma unroll
        for (int r = 0; r < kMaxCluster; ++r)
          if (r < ctas) add(cluster.map_shared_rank(hist, r));
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) sum += c[j];
      uint32_t total;
      uint32_t before = block_scan(sum, sm.warp_a, &total);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (j < per && before < rest && rest <= before + c[j]) {
          sm.digit = tid * per + j;
          sm.rest = rest - before;
        }
        before += c[j];
      }
      __syncthreads();
      const uint32_t digit = sm.digit;
      rest = sm.rest;
      if (pass == 0)
        high = digit == 0 ? 0 : (static_cast<uint64_t>(1 + (digit - 1) / 2048) << 11) | ((digit - 1) % 2048);
      else
        high = (high << (pass == 1 ? 11 : 10)) | digit;
      __syncthreads();
    }
    limit = high;
    ties = rest;
  }

  // slots moved by this CTA: list entries [first, first + count)
  uint32_t first = 0, count = 0;
  const int32_t* np = p.new_pos ? p.new_pos + static_cast<int64_t>(stream) * p.n : nullptr;
  int32_t* list = p.list + static_cast<int64_t>(lst) * p.list_len;
  const int64_t out_at = static_cast<int64_t>(lst) * p.out_pitch;
  const bool copy_pos = p.pos_out != p.pos, copy_weight = p.weight_out != p.weight;
  uint32_t kept = 0;  // entries of the whole list
  if (ALONE) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
  if (only >= 0) {
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
    // counts of this warp: slots that are taken (kept) whatever the ties, and ties
    const uint32_t tie_cls = static_cast<uint32_t>(limit >> 32);
    auto sure = [&](uint64_t k) {
      return COMPACT ? k > limit && (k >> 32) >= 1 && (k >> 32) < 3 : k < limit;
    };
    uint32_t a = 0, b = 0;
    FOR_KEYS(i) {
      const uint64_t k = key_of(i);
      a += sure(k);
      b += k == limit;
    }
    a = __reduce_add_sync(0xffffffffu, a);
    b = __reduce_add_sync(0xffffffffu, b);
    if (lane == 0) {
      sm.warp_a[warp] = a;
      sm.warp_b[warp] = b;
    }
    __syncthreads();
    uint32_t wa = sm.warp_a[lane], wb = sm.warp_b[lane];
    const uint32_t ca = __reduce_add_sync(0xffffffffu, wa), cb = __reduce_add_sync(0xffffffffu, wb);
    wa = __reduce_add_sync(0xffffffffu, lane < warp ? wa : 0u);
    wb = __reduce_add_sync(0xffffffffu, lane < warp ? wb : 0u);
    // before this CTA's slots, and in the whole list
    uint32_t before_a = 0, before_b = 0, all_a = ca, all_b = cb;
    if (!ALONE) {
      if (tid == 0) {
        sm.cta_a = ca;
        sm.cta_b = cb;
      }
      cluster.sync();
      all_a = all_b = 0;
#pragma unroll
      for (int r = 0; r < kMaxCluster; ++r)
        if (r < ctas) {
          const uint32_t ra = *cluster.map_shared_rank(&sm.cta_a, r);
          const uint32_t rb = *cluster.map_shared_rank(&sm.cta_b, r);
          before_a += r < rank ? ra : 0;
          before_b += r < rank ? rb : 0;
          all_a += ra;
          all_b += rb;
        }
    }
    // list entries among the slots before a point with na sure ones and nb ties before it
    auto place = [&](uint32_t na, uint32_t nb) -> uint32_t {
      if (COMPACT) return na + (tie_cls >= 1 && nb > ties ? nb - ties : 0u);
      return na + (nb < ties ? nb : ties);
    };
    kept = place(all_a, all_b);
    if (ALONE) {  // an equal share
      first = static_cast<uint32_t>(static_cast<uint64_t>(kept) * rank / ctas);
      count = static_cast<uint32_t>(static_cast<uint64_t>(kept) * (rank + 1) / ctas) - first;
    } else {
      first = place(before_a, before_b);
      count = place(before_a + ca, before_b + cb) - first;
    }
    uint32_t na = before_a + wa, nb = before_b + wb;
    if (ALONE) __syncthreads();  // the counters have been read
    // positions and weights first, so that no load waits for the store before it
    constexpr int kGroup = 4;
#pragma unroll
    for (int i0 = 0; i0 < (KPT > 0 ? KPT : iters); i0 += kGroup) {
      if (i0 >= iters) break;
      int32_t ps[kGroup];
      float ws[kGroup];
#pragma unroll
      for (int u = 0; u < kGroup; ++u) {
        const int i = i0 + u, slot = slot0 + 32 * i;
        // alone: the CTAs write for the warps' rounds in turn
        const bool mine = i < iters && slot < p.slots && (!ALONE || i % ctas == rank);
        ps[u] = mine && (COMPACT || copy_pos) ? p.pos[at + slot] : 0;
        ws[u] = mine && (COMPACT || copy_weight) ? p.weight[at + slot] : 0.f;
      }
#pragma unroll
      for (int u = 0; u < kGroup; ++u) {
        const int i = i0 + u, slot = slot0 + 32 * i;
        if (i >= iters) break;
        const uint64_t k = key_of(KPT > 0 && i >= KPT ? 0 : i);
        const bool is_a = sure(k), is_b = k == limit;
        const uint32_t ma = __ballot_sync(0xffffffffu, is_a), mb = __ballot_sync(0xffffffffu, is_b);
        const uint32_t below = (1u << lane) - 1;
        const uint32_t la = na + __popc(ma & below), lb = nb + __popc(mb & below);
        const bool tie_in = is_b && (COMPACT ? tie_cls >= 1 && lb >= ties : lb < ties);
        const bool take = is_a || tie_in;
        const uint32_t v = place(la, lb);
        if (slot < p.slots) {
          if (ALONE && take) sm.hist[v] = slot;
          if (!ALONE && take) list[v] = slot;
          if (!ALONE || i % ctas == rank) {
            if (COMPACT) {
              if (take) {
                p.pos_out[out_at + v] = ps[u];
                p.weight_out[out_at + v] = ws[u];
              }
            } else {
              if (take || copy_pos) p.pos_out[out_at + slot] = take ? np[v] : ps[u];
              if (take || copy_weight) p.weight_out[out_at + slot] = take ? 0.f : ws[u];
            }
          }
        }
        na += __popc(ma);
        nb += __popc(mb);
      }
    }
    if (COMPACT) {  // the destination's empty end
      for (int v = static_cast<int>(kept) + rank * kThreads + tid; v < p.list_len; v += ctas * kThreads) {
        list[v] = -1;
        p.pos_out[out_at + v] = -1;
        p.weight_out[out_at + v] = 0.f;
      }
    }
  }
#undef FOR_KEYS

  // ---- rows: the entries of this CTA, 16 bytes of a key and of a value per thread and step
  __syncthreads();  // this CTA's part of the list is written
  if (ALONE)
    for (uint32_t v = first + tid; v < first + count; v += kThreads) list[v] = sm.hist[v];
  const int64_t src0 = stream * p.src_stream + group * p.src_group;
  const int64_t dst0 = stream * p.dst_stream + group * p.dst_group;
  const int r16 = p.row16;  // 8 or 16
  const int64_t items = static_cast<int64_t>(count) * r16;
  constexpr int kUnroll = 4;
  for (int64_t it0 = tid; it0 < items; it0 += kUnroll * kThreads) {
    uint4 xk[kUnroll], xv[kUnroll];
    int64_t to[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int64_t it = it0 + u * kThreads;
      if (it >= items) continue;
      const int64_t v = first + it / r16;
      const int part = static_cast<int>(it % r16);
      const int64_t slot = ALONE ? static_cast<int64_t>(sm.hist[v]) : list[v];
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
  if (COMPACT) {
    const uint4 zero = make_uint4(0, 0, 0, 0);
    const int64_t end = static_cast<int64_t>(p.list_len - static_cast<int>(kept)) * r16;
    for (int64_t it = rank * kThreads + tid; it < end; it += static_cast<int64_t>(ctas) * kThreads) {
      const int64_t to = dst0 + (kept + it / r16) * p.dst_row + it % r16;
      p.dst_k[to] = zero;
      p.dst_v[to] = zero;
    }
  }
  if (!ALONE) cluster.sync();  // no CTA leaves while another may still read its shared memory
}

template <int KPT, bool COMPACT, bool ALONE>
cudaError_t launch_evict(const EvictParams& p, int lists, int ctas, cudaStream_t s) {
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
  return cudaLaunchKernelEx(&cfg, evict_kernel<KPT, COMPACT, ALONE>, p);
}

// CTAs of a cluster: as many as keep the lists' clusters on the GPU at once, but no fewer than
// 1024 slots each (below that the cluster's barriers cost more than the shorter loops save).
template <bool COMPACT>
cudaError_t launch(EvictParams& p, int lists, cudaStream_t s) {
  int ctas = 1;
  while (ctas < kMaxCluster && 2 * ctas * static_cast<int64_t>(lists) <= num_sms() &&
         p.slots > 1024 * ctas)
    ctas *= 2;
  const bool alone = p.slots <= kAloneSlots && (COMPACT || p.n != 1);
  const int per = alone ? kThreads : kThreads * ctas;
  p.iters = (p.slots + per - 1) / per;
  if (p.iters < 1) p.iters = 1;
  if (alone)
    return p.iters <= 2 ? launch_evict<2, COMPACT, true>(p, lists, ctas, s)
                        : launch_evict<8, COMPACT, true>(p, lists, ctas, s);
  if (!COMPACT && p.iters <= 2) return launch_evict<2, COMPACT, false>(p, lists, ctas, s);
  if (p.iters <= 12) return launch_evict<12, COMPACT, false>(p, lists, ctas, s);
  if (p.iters <= kMaxKeys) return launch_evict<kMaxKeys, COMPACT, false>(p, lists, ctas, s);
  return launch_evict<0, COMPACT, false>(p, lists, ctas, s);
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
  if (c->stream_stride < 0 || c->group_stride < 0 || c->slot_stride < c->head_dim ||
      c->stream_stride % 8 || c->group_stride % 8 || c->slot_stride % 8)
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
