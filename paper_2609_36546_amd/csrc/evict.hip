// Eviction from the paged cache by gathered attention weight, for gfx950: of a
// sequence's L positions each KV head keeps n, the first n_sink, the last n_recent and
// of the others those of the largest mass (equal masses: the lower position), and they
// move, in order, to positions 0 .. n - 1 of other pages.
//
//   select kernel  one workgroup per (sequence, KV head): the mass of the last position
//                  kept, found by its order number's three digits of 11 bits from the top,
//                  each a histogram in LDS of what the digits before it leave (no more of them
//                  than it takes); then the kept positions by a scan in order, equal masses
//                  counted as they come.
//                  11 us for a sequence of 8000, chains of dependent steps: loads, atomics,
//                  scans, barriers.
//   move kernel    64 kept positions of one (sequence, KV head) per workgroup: keys are
//                  runs of 32 channels per slot, values and masses gathered slot by slot
//                  and stored 16 bytes at a time.  Bound by bytes: kept values lie in every
//                  line of the cache, so those are all read (32 sequences of 2 to 8 Ki positions
//                  to 40%: 835 MB in 171 us).
//
// Whole numbers decide, in an order that does not depend on the atomics', so the same call
// repeats bit for bit.
#include <type_traits>

#include "common.h"
#include "kernels.h"

namespace ipdv {
namespace {

constexpr int kThreads = 1024;     // of the select kernel
constexpr int kWaves = kThreads / kWave;
constexpr int kDigit = 11, kBins = 1 << kDigit;
constexpr int kRun = 16;           // neighbouring positions of a thread: in one page
constexpr int kMove = 64;          // positions of a workgroup of the move kernel

struct EvictParams : EvictLaunch {
  int log2ps, slots, dst_slots;
};

// Masses as unsigned numbers of the same order; NaN below everything, -0 as 0.
__device__ __forceinline__ unsigned order_of(float x) {
  if (x != x) return 0u;
  const unsigned u = __float_as_uint(x == 0.f ? 0.f : x);
  return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}

struct Seq {
  int b, L, n, lo, hi;     // kept without asking: positions below lo, and from hi on
};
__device__ __forceinline__ Seq seq_of(const EvictParams& a, int slot) {
  Seq s;
  s.b = a.seq_ids ? a.seq_ids[slot] : slot;
  s.L = min(max(a.ctx_lens[s.b], 0), a.slots);
  s.n = min(max(a.keep[s.b], 0), min(s.L, a.dst_slots));
  s.lo = min(a.n_sink, s.n);
  s.hi = s.L - min(a.n_recent, s.n - s.lo);
  return s;
}
__device__ __forceinline__ int page_at(const EvictParams& a, const int32_t* table, int width, int pos) {
  return min(max(table[min(pos >> a.log2ps, width - 1)], 0), a.num_pages - 1);
}

// Sums over the threads before this one of two counts (PAIR; else of the first); every thread calls.
// The waves' sums are scanned by the lanes of each wave (one after the other: 0.7 us a call).
template <bool PAIR>
__device__ __forceinline__ int2 scan(int2 v, int2* part, int2* all) {
  static_assert(kWaves <= kWave, "a lane of a wave");
  const int lane = lane_id(), w = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int x = wave_incl_scan_i(v.x), y = PAIR ? wave_incl_scan_i(v.y) : 0;
  __syncthreads();                  // the previous call's readers are done
  if (lane == kWave - 1) part[w] = make_int2(x, y);
  __syncthreads();
  const int2 p = part[lane % kWaves];
  auto over = [&](int mine, int upto, int sum) {       // before this wave, and before the thread in it
    const int s = wave_incl_scan_i(lane < kWaves ? sum : 0);
    return make_int2(upto - mine + (w > 0 ? __builtin_amdgcn_readlane(s, max(w - 1, 0)) : 0),
                     __builtin_amdgcn_readlane(s, kWaves - 1));
  };
  const int2 a = over(v.x, x, p.x), b = PAIR ? over(v.y, y, p.y) : make_int2(0, 0);
  *all = make_int2(a.y, b.y);
  return make_int2(a.x, b.x);
}

// ONE: a round of threads holds all positions, so their masses are read once.
template <bool ONE>
__global__ __launch_bounds__(kThreads) void evict_select_kernel(EvictParams a) {
  // four copies of a bin for four lanes: most masses lie in few bins (0.7 us less)
  __shared__ __attribute__((aligned(16))) int4 s_hist[kBins];
  __shared__ int2 s_part[kWaves];
  __shared__ int s_digit, s_left, s_count;
  typedef __attribute__((__vector_size__(16))) float f32x4;
  const int slot = blockIdx.x / a.Hkv, g = blockIdx.x - slot * a.Hkv, tid = threadIdx.x;
  const int32_t* table = a.page_table + (size_t)(a.seq_ids ? a.seq_ids[slot] : slot) * a.max_pages;
  auto mass_at = [&](int p0) {
    return a.mass + ((size_t)page_at(a, table, a.max_pages, p0) * a.Hkv + g) * (unsigned)a.page_size + (p0 & (a.page_size - 1));
  };
  f32x4 early[kRun / 4];               // asked for before the lengths are known
  if (ONE && tid * kRun < a.slots) {
    const float* m = mass_at(tid * kRun);
#pragma unroll
    for (int i = 0; i < kRun / 4; ++i) early[i] = ld16<f32x4>(m + 4 * i);
  }
  const Seq s = seq_of(a, slot);
  int32_t* kept = a.kept + ((size_t)s.b * a.Hkv + g) * (unsigned)a.dst_slots;
  for (int i = s.n + tid; i < a.dst_slots; i += kThreads) kept[i] = -1;
  if (s.n == 0) return;
  if (s.n == s.L) {
    for (int i = tid; i < s.n; i += kThreads) kept[i] = i;
    return;
  }
  const int rounds = ONE ? 1 : (int)(((long)s.L + kThreads * kRun - 1) / (kThreads * kRun));
  unsigned key[kRun];
  auto load = [&](int round) {
    const int p0 = (round * kThreads + tid) * kRun;
    if (p0 >= s.L) return;
    const float* m = mass_at(p0);
#pragma unroll
    for (int i = 0; i < kRun; i += 4) {
      const f32x4 v = ONE ? early[i / 4] : ld16<f32x4>(m + i);
#pragma unroll
      for (int c = 0; c < 4; ++c) key[i + c] = order_of(v[c]);
    }
  };
  if (ONE) load(0);
  auto candidate = [&](int p) { return p >= s.lo && p < s.hi; };
  // The order number of the last position kept, from its top digit down: `least` so far, its
  // bits below `shift` open; `left` to be kept among those that agree with it above them.
  int left = s.n - s.lo - (s.L - s.hi), shift = 32;
  unsigned least = 0;
  const bool ask = left > 0;        // else nothing beside what is kept unasked
  int* hist = reinterpret_cast<int*>(s_hist) + (tid & 3);
  static_assert(kBins == 2 * kThreads, "two bins of a thread");
  while (ask && shift > 0) {
    const int above = shift;
    shift = max(shift - kDigit, 0);
    s_hist[tid] = s_hist[kThreads + tid] = make_int4(0, 0, 0, 0);
    __syncthreads();
    for (int r = 0; r < rounds; ++r) {
      if (!ONE) load(r);
      const int p0 = (r * kThreads + tid) * kRun;
#pragma unroll
      for (int i = 0; i < kRun; ++i)
        if (candidate(p0 + i) && (above == 32 || (key[i] ^ least) >> above == 0))
          atomicAdd(&hist[4 * ((key[i] >> shift) & (kBins - 1))], 1);
    }
    __syncthreads();
    const int4 h0 = s_hist[2 * (kThreads - 1 - tid)], h1 = s_hist[2 * (kThreads - 1 - tid) + 1];
    const int2 c = make_int2(h0.x + h0.y + h0.z + h0.w, h1.x + h1.y + h1.z + h1.w);      // from the top: .y, then .x
    int2 all;
    const int before = scan<false>(make_int2(c.x + c.y, 0), s_part, &all).x;
    const bool hi = before < left && before + c.y >= left, lo = before + c.y < left && before + c.y + c.x >= left;
    if (hi || lo) {
      s_digit = 2 * (kThreads - 1 - tid) + (hi ? 1 : 0);
      s_left = left - before - (hi ? 0 : c.y);
      s_count = hi ? c.y : c.x;
    }
    __syncthreads();
    least |= (unsigned)s_digit << shift;
    left = s_left;
    if (s_count == left) {          // all of the digit: none of them equals what is just below it
      least -= 1;
      shift = 0;
      left = 0;
    }
    __syncthreads();
  }
  // All above `least` are kept, and the first `left` that equal it.
  int2 base = make_int2(0, 0);
  for (int r = 0; r < rounds; ++r) {
    if (!ONE) load(r);
    const int p0 = (r * kThreads + tid) * kRun;
    int2 mine = make_int2(0, 0);
    unsigned sure = 0, equal = 0;
#pragma unroll
    for (int i = 0; i < kRun; ++i) {
      const int p = p0 + i;
      const bool in = candidate(p);
      sure |= (p < s.L && (!in || (ask && key[i] > least)) ? 1u : 0u) << i;
      equal |= (in && ask && key[i] == least ? 1u : 0u) << i;
    }
    mine.x = __popc(sure);
    mine.y = __popc(equal);
    int2 all;
    const int2 before = scan<true>(mine, s_part, &all);
    int x = base.x + before.x, y = base.y + before.y;
    for (unsigned on = sure | equal; on; on &= on - 1) {
      const int i = __ffs(on) - 1;
      const bool eq = (equal >> i) & 1;
      if (!eq || y < left) kept[x + min(y, left)] = p0 + i;
      x += eq ? 0 : 1;
      y += eq ? 1 : 0;
    }
    base.x += all.x;
    base.y += all.y;
  }
}

template <typename DT, int D>
__global__ __launch_bounds__(256, 4) void evict_move_kernel(EvictParams a) {
  constexpr int EPL = 16 / (int)sizeof(DT);
  typedef __attribute__((__vector_size__(16))) int i32x4;
  __shared__ int s_src[kMove], s_dst[kMove / 16];      // page * page_size + slot; of a 16-slot run
  const int slot = blockIdx.x / a.Hkv, g = blockIdx.x - slot * a.Hkv, tid = threadIdx.x;
  const int i0 = (blockIdx.z * gridDim.y + blockIdx.y) * kMove;
  int p = 0;                                           // asked for before the lengths are known
  if (tid < kMove && i0 + tid < a.dst_slots)
    p = a.kept[((size_t)(a.seq_ids ? a.seq_ids[slot] : slot) * a.Hkv + g) * (unsigned)a.dst_slots + i0 + tid];
  const Seq s = seq_of(a, slot);
  // Not before the selection has ended: new_lens may be ctx_lens or keep, and n stays the same with
  // itself in the place of either.
  if (i0 == 0 && g == 0 && tid == 0) a.new_lens[s.b] = s.n;
  const int n = min(s.n - i0, kMove);
  if (n <= 0) return;
  const int ps = a.page_size;
  if (tid < kMove) {
    int at = 0;
    if (tid < n) {
      at = page_at(a, a.page_table + (size_t)s.b * a.max_pages, a.max_pages, p) * ps + (p & (ps - 1));
    }
    s_src[tid] = at;
  } else if (tid < kMove + kMove / 16) {
    p = i0 + 16 * (tid - kMove);
    s_dst[tid - kMove] = page_at(a, a.dst_table + (size_t)s.b * a.dst_pages, a.dst_pages, p) * ps + (p & (ps - 1));
  }
  __syncthreads();
  auto page = [&](int at) { return (size_t)(at >> a.log2ps) * a.Hkv + g; };
  if (tid < n) {
    const int from = s_src[tid], to = s_dst[tid >> 4] + (tid & 15);
    a.mass[page(to) * ps + (to & (ps - 1))] = a.mass[page(from) * ps + (from & (ps - 1))];
  }
  // keys: 16 bytes of a slot's run of 32 channels.  They, and what is stored, go past the caches'
  // order of use (32 sequences 190 to 185 us); values do not: a line's neighbours come from it.
  constexpr int KPS = 32 / EPL;                        // of a run
  constexpr int KN = kMove * D / EPL / 256;
  const DT* kc = reinterpret_cast<const DT*>(a.k_cache);
  const DT* vc = reinterpret_cast<const DT*>(a.v_cache);
  i32x4 k[KN];
#pragma unroll
  for (int x = 0; x < KN; ++x) {
    const int e = tid + 256 * x, c = e % KPS, i = e / KPS % kMove, sl = e / KPS / kMove;
    if (i < n) {
      const int at = s_src[i];
      k[x] = __builtin_nontemporal_load(reinterpret_cast<const i32x4*>(kc + (page(at) * (D / 32) + sl) * ps * 32 + (at & (ps - 1)) * 32 + EPL * c));
    }
  }
#pragma unroll
  for (int x = 0; x < KN; ++x) {
    const int e = tid + 256 * x, c = e % KPS, i = e / KPS % kMove, sl = e / KPS / kMove;
    if (i < n) {
      const int at = s_dst[i >> 4] + (i & 15);
      DT* dst = reinterpret_cast<DT*>(a.k_cache) + (page(at) * (D / 32) + sl) * ps * 32 + (at & (ps - 1)) * 32 + EPL * c;
      __builtin_nontemporal_store(k[x], reinterpret_cast<i32x4*>(dst));
    }
  }
  // values: a channel's run of EPL slots
  constexpr int RUNS = kMove / EPL, VN = RUNS * D / 256;
  static_assert(RUNS * D % 256 == 0, "whole rounds");
  struct Run { DT e[EPL]; } run[VN];
#pragma unroll
  for (int x = 0; x < VN; ++x) {                       // all asked for before the first is stored
    const int e = tid + 256 * x, i = e % RUNS * EPL, ch = e / RUNS;
#pragma unroll
    for (int c = 0; c < EPL; ++c) {
      const int at = s_src[i + c];                     // behind n: a slot that is there, not used
      run[x].e[c] = vc[(page(at) * D + ch) * ps + (at & (ps - 1))];
    }
  }
#pragma unroll
  for (int x = 0; x < VN; ++x) {
    const int e = tid + 256 * x, i = e % RUNS * EPL, ch = e / RUNS;
    if (i >= n) continue;
    const int to = s_dst[i >> 4] + (i & 15);
    DT* dst = reinterpret_cast<DT*>(a.v_cache) + (page(to) * D + ch) * ps + (to & (ps - 1));
    if (i + EPL <= n) {
      __builtin_nontemporal_store(__builtin_bit_cast(i32x4, run[x]), reinterpret_cast<i32x4*>(dst));
    } else {
#pragma unroll
      for (int c = 0; c < EPL; ++c)
        if (i + c < n) dst[c] = run[x].e[c];
    }
  }
}

}  // namespace

hipError_t launch_kv_evict(const EvictLaunch& L, hipStream_t st) {
  EvictParams p{};
  static_cast<EvictLaunch&>(p) = L;
  p.log2ps = __builtin_ctz(L.page_size);
  p.slots = table_slots(L.max_pages, L.page_size);
  p.dst_slots = table_slots(L.dst_pages, L.page_size);
  const int sg = L.n_seq * L.Hkv;
  trace_begin(st);
  if (p.slots <= kThreads * kRun)
    hipLaunchKernelGGL(evict_select_kernel<true>, dim3(sg), dim3(kThreads), 0, st, p);
  else
    hipLaunchKernelGGL(evict_select_kernel<false>, dim3(sg), dim3(kThreads), 0, st, p);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  trace_mark(st);
  auto move = [&](auto kernel) {
    const int ny = (p.dst_slots + kMove - 1) / kMove, nz = (ny + 65534) / 65535;
    hipLaunchKernelGGL(kernel, dim3(sg, (ny + nz - 1) / nz, nz), dim3(256), 0, st, p);
  };
  if (L.dtype_bf16) {
    if (L.D == 128) move(evict_move_kernel<bf16, 128>); else move(evict_move_kernel<bf16, 64>);
  } else {
    if (L.D == 128) move(evict_move_kernel<float, 128>); else move(evict_move_kernel<float, 64>);
  }
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  trace_mark(st);
  return hipSuccess;
}

}  // namespace ipdv
