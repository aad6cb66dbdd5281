// The filtered draw from logits for gfx950: per row a temperature, top-k, top-p
// and min-p, and one draw by the inverse of the distribution in index order.
//
// With p = softmax(l / T) and the row ordered by logit descending, lower index
// first on equal logits, every filter keeps a prefix of the order:
//   top-k   the first k
//   top-p   as many as it takes for their mass to reach p times the top-k's
//   min-p   those with (l - max l) / T >= ln(min_p)
// and the shortest prefix (one token at least) is what is drawn from.  So the
// kept set is "ordered at or before the cut", a (logit, index) pair, and the
// work is to find the cut, then the token where the kept mass passes u.
//
// Histograms instead of a sort.  With y = 8 l / T, bin = floor(y): a bin spans a
// factor of e^(1/8) in probability, and 255 bins from the maximum's down reach
// e^-31.9 of the top probability.  What lies below is taken as of probability
// zero (at V = 262144 all of it together is below 4e-9 of the mass, less than a
// step of an fp32 u).  An entry adds 2^45 + round(2^30 m) to its bin, m its mass
// against the bin's upper edge: one 64-bit LDS addition counts and sums.  Sums
// of whole numbers do not depend on the order of the atomics, so a call repeats
// bit for bit; m itself is an fp32 exponential of an argument within 1/8, and
// joined sums are in double.  y is in double, for the bins to end where the
// definition puts them.
//
//   chunk kernel  one workgroup per 8192 entries: reads the logits once, into
//                 registers; its histogram below its own maximum (bins are
//                 aligned, since they are floors of y), and a list of its
//                 topmost entries.  Bound by the read of the logits.
//   row kernel    one workgroup per row: adds the histograms up, finds the cut's
//                 bin, orders the bin's entries (from the lists, or from the
//                 logits where a list stops above the bin) and takes the cut;
//                 then the chunk, and in it the entry, where the mass passes u.
//                 Bound by latency: it reads the histograms and one chunk.
// A bin of more entries than fit LDS (equal logits by the thousand) is cut by
// selecting the digits of the logit from the top, reading the row for each.
#include "common.h"
#include "kernels.h"

namespace ipdv {
namespace {

constexpr int kChunk = 8192;      // entries per workgroup of the chunk kernel
constexpr int kBins = 256;
constexpr int kList = 256;        // topmost entries that a chunk lists
constexpr int kSort = 1024;       // entries of one bin that are ordered in LDS
constexpr int kMaxChunks = 32;    // V <= 262144
constexpr double kWidth = 8.0;    // bins per unit of l / T
constexpr int kCountShift = 45;   // 8192 masses of at most 2^30 stay below
constexpr unsigned long long kMassMask = (1ull << kCountShift) - 1;
typedef unsigned long long u64;

struct ChunkHead {
  double floor_max;   // floor(y) of the chunk's maximum, -inf without a finite logit
  float max;
  int bad;            // holds NaN or +inf
  int covered;        // bins that the list holds whole, from the chunk's top bin
  int listed;
};
struct ListEntry {
  float l;
  int v;
};
constexpr size_t kChunkBytes = kBins * sizeof(u64) + kList * sizeof(ListEntry) + 64;
static_assert(sizeof(ChunkHead) <= 64, "chunk record");

struct ChunkRec {
  u64* hist;
  ListEntry* list;
  ChunkHead* head;
};
__device__ __forceinline__ ChunkRec chunk_rec(const SampleLogitsLaunch& p, int n_chunks, int m, int s) {
  char* at = reinterpret_cast<char*>(p.workspace) + ((size_t)m * n_chunks + s) * kChunkBytes;
  return {reinterpret_cast<u64*>(at), reinterpret_cast<ListEntry*>(at + kBins * sizeof(u64)),
          reinterpret_cast<ChunkHead*>(at + kBins * sizeof(u64) + kList * sizeof(ListEntry))};
}

// A row's parameters; greedy (T = 0) is the top entry at temperature 1.
struct Row {
  double width;   // y = l * width
  double temp;
  int k;          // 0: off
  float top_p;    // >= 1: off
  float min_p;    // <= 0: off
  bool bad;
};
__device__ __forceinline__ Row row_of(const SampleLogitsLaunch& p, int m) {
  Row r;
  const float t = p.temperature ? p.temperature[m] : 1.f;
  r.bad = !(t >= 0.f);
  r.temp = t > 0.f ? (double)t : 1.0;
  r.width = kWidth / r.temp;
  r.k = p.top_k ? max(p.top_k[m], 0) : 0;
  r.top_p = p.top_p ? p.top_p[m] : 1.f;
  r.min_p = p.min_p ? p.min_p[m] : 0.f;
  if (!(t > 0.f)) r.k = 1;
  if (!(r.top_p < 1.f)) r.top_p = 1.f;
  if (!(r.min_p > 0.f)) r.min_p = 0.f;
  if (r.min_p > 1.f) {              // no entry passes: the first stays
    r.k = 1;
    r.min_p = 0.f;
  }
  return r;
}

// Bin of a finite logit below `top` = floor(y) of the maximum, and its mass
// against the bin's upper edge in units of 2^-30 (the last bin has none).
__device__ __forceinline__ int classify(float l, double width, double top, unsigned* mass) {
  const double y = (double)l * width;
  const double d = top - floor(y);
  if (!(d < kBins - 1)) {
    *mass = 0;
    return kBins - 1;
  }
  const int bin = (int)d;
  const float t = (float)(y - (top + 1.0 - bin));
  *mass = (unsigned)rintf(fast_exp2(t * (float)(1.4426950408889634 / kWidth)) * 1073741824.f);
  return bin;
}

// Logits as unsigned numbers of the same order, and back to one of equal order.
__device__ __forceinline__ unsigned key_of(float l) {
  const unsigned u = __float_as_uint(l == 0.f ? 0.f : l);   // -0 is +0
  return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}
// Order of entries: logit, then the lower index.
__device__ __forceinline__ u64 order_of(float l, int v) { return ((u64)key_of(l) << 32) | (unsigned)~v; }

template <typename DT>
__device__ __forceinline__ float logit(const SampleLogitsLaunch& p, int m, int v) {
  return to_f32(reinterpret_cast<const DT*>(p.logits)[(size_t)m * p.stride + v]);
}

template <typename DT, bool VEC>
__global__ __launch_bounds__(256) void chunk_kernel(SampleLogitsLaunch p, int n_chunks) {
  constexpr int N = VEC ? 16 / (int)sizeof(DT) : 1;   // entries per load
  constexpr int PER = kChunk / 256;
  __shared__ u64 s_hist[kBins];
  __shared__ float s_max[4];
  __shared__ int s_bad, s_n, s_cover, s_wave[4];
  const int m = blockIdx.x / n_chunks, s = blockIdx.x % n_chunks;
  const int tid = threadIdx.x, lane = lane_id(), w = tid >> 6;
  const int v0 = s * kChunk, n = min(kChunk, p.V - v0);
  const DT* src = reinterpret_cast<const DT*>(p.logits) + (size_t)m * p.stride + v0;
  // entry i of the thread: v0 + (i / N) * 256 N + tid N + i % N
  float x[PER];
#pragma unroll
  for (int i = 0; i < PER; i += N) {
    const int at = (i / N) * 256 * N + tid * N;
    if constexpr (VEC) {            // n is a multiple of N
      if (at < n) {
        typedef __attribute__((__vector_size__(16))) int i32x4;
        const i32x4 raw = ld16<i32x4>(src + at);
        const DT* e = reinterpret_cast<const DT*>(&raw);
#pragma unroll
        for (int c = 0; c < N; ++c) x[i + c] = to_f32(e[c]);
      } else {
#pragma unroll
        for (int c = 0; c < N; ++c) x[i + c] = -INFINITY;
      }
    } else {
      x[i] = at < n ? to_f32(src[at]) : -INFINITY;
    }
  }
  const Row r = row_of(p, m);
  s_hist[tid] = 0;
  if (tid == 0) s_bad = s_n = s_cover = 0;
  float mx = -INFINITY;
  bool bad = false;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    mx = fmaxf(mx, x[i]);
    bad |= !(x[i] < INFINITY);
  }
  mx = wave_max(mx);
  if (lane == 0) s_max[w] = mx;
  __syncthreads();
  if (bad) s_bad = 1;
  mx = fmaxf(fmaxf(s_max[0], s_max[1]), fmaxf(s_max[2], s_max[3]));
  const double top = floor((double)mx * r.width);
  const bool any = mx > -INFINITY && mx < INFINITY;
  if (any) {
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      if (x[i] > -INFINITY) {
        unsigned mass;
        const int bin = classify(x[i], r.width, top, &mass);
        __hip_atomic_fetch_add(&s_hist[bin], (1ull << kCountShift) + mass, __ATOMIC_RELAXED,
                               __HIP_MEMORY_SCOPE_WORKGROUP);
      }
    }
  }
  __syncthreads();
  const ChunkRec rec = chunk_rec(p, n_chunks, m, s);
  rec.hist[tid] = s_hist[tid];
  // The list: whole bins from the top while they fit.
  int cum = wave_incl_scan_i((int)(s_hist[tid] >> kCountShift));
  if (lane == kWave - 1) s_wave[w] = cum;
  __syncthreads();
  for (int i = 0; i < w; ++i) cum += s_wave[i];
  if (cum <= kList) atomicAdd(&s_cover, 1);     // counts never fall, so these are the first bins
  __syncthreads();
  const int cover = s_cover;
  if (any && (r.k > 0 || r.top_p < 1.f || r.min_p > 0.f)) {
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      // entries far below the list's end need no double to be told
      if (x[i] > -INFINITY) {
        unsigned mass;
        if (classify(x[i], r.width, top, &mass) < cover) {
          const int at = atomicAdd(&s_n, 1);
          rec.list[at] = {x[i], v0 + (i / N) * 256 * N + tid * N + i % N};
        }
      }
    }
  }
  __syncthreads();
  if (tid == 0) *rec.head = {any ? top : -INFINITY, mx, s_bad, cover, s_n};
}

// ---- the row kernel ----

constexpr int kRowThreads = 512;

// Sum over the threads before this one, and over all; every thread calls.
template <typename T>
__device__ __forceinline__ T block_scan(T v, T* s_part, T* total) {
  const int lane = lane_id(), w = threadIdx.x >> 6;
  T incl = v;
#pragma unroll
  for (int o = 1; o < kWave; o <<= 1) {
    const T up = __shfl_up(incl, o, kWave);
    if (lane >= o) incl += up;
  }
  __syncthreads();                  // the previous call's readers are done
  if (lane == kWave - 1) s_part[w] = incl;
  __syncthreads();
  T before = 0, all = 0;
#pragma unroll
  for (int i = 0; i < kRowThreads / kWave; ++i) {
    if (i < w) before += s_part[i];
    all += s_part[i];
  }
  *total = all;
  return before + incl - v;
}

struct Shared {
  double edge[kBins];               // e^(-t/8): mass of bin t's upper edge
  double before[kBins];             // mass above bin t
  int count_before[kBins];
  int count[kBins];
  double top;                       // floor(y) of the row's maximum
  int chunk_off[kMaxChunks];        // the chunk's top bin in the row's bins (kBins: none)
  int chunk_cover[kMaxChunks], chunk_listed[kMaxChunks];
  u64 list[kSort], sorted[kSort];   // order numbers of one bin's entries
  double chunk_mass[kMaxChunks];
  u64 part_u[kRowThreads / kWave];
  double part_d[kRowThreads / kWave];
  int part_i[kRowThreads / kWave];
  unsigned digit_count[256];
  u64 digit_mass[256];
  int n, bin, found, chunk, token;
  u64 cut, mass_in;
  unsigned prefix;
  double rest, all;
  u64 digit_before_mass;
  int digit_before;
  float max;
  int bad;
};

__device__ __forceinline__ float logit_of_key(unsigned key) {
  return __uint_as_float((key & 0x80000000u) ? key & 0x7fffffffu : ~key);
}

// What ends a prefix inside a bin: a count of entries, or a mass to be reached.
struct Need {
  bool by_count;
  int count;        // entries of the bin
  double mass;      // mass of the row
};

template <typename DT>
struct RowWork {
  const SampleLogitsLaunch& p;
  Shared& S;
  const Row r;
  const int m, n_chunks, tid;
  const double top;

  // The entries of a bin, into S.list; false when they do not fit.
  __device__ bool collect(int bin) {
    if (S.count[bin] > kSort) return false;
    __syncthreads();
    if (tid == 0) S.n = 0;
    __syncthreads();
    for (int s = 0; s < n_chunks; ++s) {
      const int local = bin - S.chunk_off[s];
      if (local < 0) continue;
      const ChunkRec rec = chunk_rec(p, n_chunks, m, s);
      if ((rec.hist[local] >> kCountShift) == 0) continue;
      if (local < S.chunk_cover[s]) {
        for (int i = tid; i < S.chunk_listed[s]; i += kRowThreads) put(rec.list[i].l, rec.list[i].v, bin);
      } else {
        const int v1 = min((s + 1) * kChunk, p.V);
        for (int v = s * kChunk + tid; v < v1; v += kRowThreads) put(logit<DT>(p, m, v), v, bin);
      }
    }
    __syncthreads();
    return true;
  }
  __device__ void put(float l, int v, int bin) {
    unsigned mass;
    if (l > -INFINITY && classify(l, r.width, top, &mass) == bin) {
      const int at = atomicAdd(&S.n, 1);
      if (at < kSort) S.list[at] = order_of(l, v);
    }
  }
  __device__ u64 mass_of(u64 order) const {
    unsigned mass;
    classify(logit_of_key((unsigned)(order >> 32)), r.width, top, &mass);
    return mass;
  }

  // The cut of a prefix that ends in `bin` (S.cut), and the bin's mass up to
  // it (S.mass_in).
  __device__ void refine(int bin, Need need) {
    if (!collect(bin)) return refine_long(bin, need);
    const int n = min(S.n, kSort);
    for (int i = tid; i < n; i += kRowThreads) {
      const u64 o = S.list[i];
      int rank = 0;
      for (int c = 0; c < n; ++c) rank += S.list[c] > o;
      S.sorted[rank] = o;
    }
    __syncthreads();
    // two neighbouring entries per thread
    const int i0 = 2 * tid;
    const u64 a = i0 < n ? mass_of(S.sorted[i0]) : 0, b = i0 + 1 < n ? mass_of(S.sorted[i0 + 1]) : 0;
    u64 all;
    const u64 pre = block_scan<u64>(a + b, S.part_u, &all);
    const double base = S.before[bin], e = S.edge[bin] * (1.0 / 1073741824.0);
    const bool ka = i0 < n && (need.by_count ? i0 < need.count : i0 == 0 || base + e * (double)pre < need.mass);
    const bool kb = i0 + 1 < n && (need.by_count ? i0 + 1 < need.count : base + e * (double)(pre + a) < need.mass);
    int kept;
    block_scan<int>((int)ka + (int)kb, S.part_i, &kept);
    if (kept == 0) kept = 1;
    if (tid == (kept - 1) / 2) {
      const bool second = (kept - 1) & 1;
      S.cut = S.sorted[kept - 1];
      S.mass_in = pre + a + (second ? b : 0);
    }
    __syncthreads();
  }

  // The same for a bin too long for LDS: the cut's logit from its top digit
  // down, then the index among equal logits.
  __device__ void refine_long(int bin, Need need) {
    const double base = S.before[bin], e = S.edge[bin] * (1.0 / 1073741824.0);
    __syncthreads();
    if (tid == 0) {
      S.prefix = 0;
      S.digit_before = 0;
      S.digit_before_mass = 0;
    }
    for (int shift = 24; shift >= 0; shift -= 8) {
      if (tid < 256) {
        S.digit_count[tid] = 0;
        S.digit_mass[tid] = 0;
      }
      __syncthreads();
      const unsigned prefix = S.prefix;
      for (int v = tid; v < p.V; v += kRowThreads) {
        const float l = logit<DT>(p, m, v);
        unsigned mass;
        if (l > -INFINITY && classify(l, r.width, top, &mass) == bin) {
          const unsigned key = key_of(l);
          if (shift == 24 || (key >> (shift + 8)) == (prefix >> (shift + 8))) {
            atomicAdd(&S.digit_count[(key >> shift) & 255], 1u);
            __hip_atomic_fetch_add(&S.digit_mass[(key >> shift) & 255], (u64)mass, __ATOMIC_RELAXED,
                                   __HIP_MEMORY_SCOPE_WORKGROUP);
          }
        }
      }
      __syncthreads();
      if (tid == 0) {
        int lowest = 0;                                 // the last digit that occurs ends it if none before does
        while (lowest < 255 && S.digit_count[lowest] == 0) ++lowest;
        int cnt = S.digit_before, at = 255;
        u64 mass = S.digit_before_mass;
        for (; at > lowest; --at) {
          if (S.digit_count[at] == 0) continue;
          if (need.by_count ? cnt + (int)S.digit_count[at] >= need.count
                            : base + e * (double)(mass + S.digit_mass[at]) >= need.mass)
            break;
          cnt += S.digit_count[at];
          mass += S.digit_mass[at];
        }
        S.prefix = prefix | ((unsigned)at << shift);
        S.digit_before = cnt;
        S.digit_before_mass = mass;
        S.n = (int)S.digit_count[at];                   // after the last digit: the equal logits
      }
      __syncthreads();
    }
    const unsigned key = S.prefix;
    const int ties = S.n;
    const u64 w = mass_of((u64)key << 32);
    int keep = ties;                                    // the first `keep` of them by index
    if (need.by_count) {
      keep = need.count - S.digit_before;
    } else {
      const double left = need.mass - (base + e * (double)S.digit_before_mass), one = e * (double)w;
      if (one > 0.0 && left < one * ties) keep = (int)ceil(left / one);
    }
    keep = max(1, min(keep, ties));
    // the index of the keep-th: threads take neighbouring entries, so that counts are in index order
    int seen = 0;
    for (int v0 = 0; v0 < p.V; v0 += 8 * kRowThreads) {
      int mine = 0;
      const int a = v0 + 8 * tid, b = min(a + 8, p.V);
      for (int v = a; v < b; ++v) mine += key_of(logit<DT>(p, m, v)) == key;
      int all;
      const int pre = seen + block_scan<int>(mine, S.part_i, &all);
      if (pre < keep && keep <= pre + mine) {
        int c = pre;
        for (int v = a; v < b; ++v)
          if (key_of(logit<DT>(p, m, v)) == key && ++c == keep) {
            S.cut = ((u64)key << 32) | (unsigned)~v;
            S.mass_in = S.digit_before_mass + (u64)keep * w;
          }
      }
      seen += all;
      if (seen >= keep) break;
    }
    __syncthreads();
  }
};

template <typename DT>
__global__ __launch_bounds__(kRowThreads) void row_kernel(SampleLogitsLaunch p, int n_chunks) {
  __shared__ Shared S;
  const int m = blockIdx.x, tid = threadIdx.x;
  const Row r = row_of(p, m);
  if (tid < kWave) {                // a lane per chunk
    double ct = -INFINITY;
    float cm = -INFINITY;
    bool bad = r.bad;
    if (tid < n_chunks) {
      const ChunkHead h = *chunk_rec(p, n_chunks, m, tid).head;
      ct = h.floor_max;
      cm = h.max;
      bad |= h.bad != 0;
      S.chunk_cover[tid] = h.covered;
      S.chunk_listed[tid] = h.listed;
    }
    double all = ct;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) all = fmax(all, __shfl_xor(all, o, kWave));
    const float mx = wave_max(cm);
    if (tid < n_chunks) S.chunk_off[tid] = all - ct < kBins ? (int)(all - ct) : kBins;
    bad = __any(bad) || !(mx > -INFINITY);
    if (tid == 0) {
      S.max = mx;
      S.top = all;
      S.bad = bad;
      S.found = 0;
      S.bin = -1;
    }
  }
  __syncthreads();
  if (S.bad) {
    if (tid == 0) {
      p.token[m] = -1;
      if (p.logp) p.logp[m] = __uint_as_float(0x7fc00000u);
    }
    return;
  }
  const double top = S.top;
  const float mx = S.max;
  // The row's bins: each half of the threads adds up every other chunk's.
  int count = 0;
  u64 mass_u = 0;
  {
    const int t = tid & (kBins - 1);
#pragma unroll 4
    for (int s = tid / kBins; s < n_chunks; s += kRowThreads / kBins) {
      const int local = t - S.chunk_off[s];
      const u64 h = chunk_rec(p, n_chunks, m, s).hist[max(local, 0)];
      count += local >= 0 ? (int)(h >> kCountShift) : 0;
      mass_u += local >= 0 ? h & kMassMask : 0;
    }
    if (tid >= kBins) {
      S.list[t] = mass_u;
      S.count[t] = count;
    }
    __syncthreads();
    if (tid < kBins) {
      mass_u += S.list[t];
      count += S.count[t];
      if (t == kBins - 1) count = 0, mass_u = 0;     // taken as of probability zero
      S.edge[t] = exp(-(double)t / kWidth);
    }
  }
  const double unit = 1.0 / 1073741824.0;
  const double mass = tid < kBins ? (double)mass_u * S.edge[tid] * unit : 0.0;
  double total;
  int n_all;
  const double mass_before = block_scan<double>(mass, S.part_d, &total);
  const int count_before = block_scan<int>(tid < kBins ? count : 0, S.part_i, &n_all);
  if (tid < kBins) {
    S.before[tid] = mass_before;
    S.count_before[tid] = count_before;
    S.count[tid] = count;
  }
  __syncthreads();

  RowWork<DT> work{p, S, r, m, n_chunks, tid, top};
  u64 cut = 0;                      // everything is at or above it
  double kept = total;              // mass of the kept entries
  if (r.k > 0 && r.k < n_all) {     // otherwise nothing that counts is cut
    if (tid < kBins && count_before < r.k && count_before + count >= r.k) S.bin = tid;
    __syncthreads();
    const int bin = S.bin;
    work.refine(bin, {true, r.k - S.count_before[bin], 0.0});
    cut = S.cut;
    kept = S.before[bin] + S.edge[bin] * unit * (double)S.mass_in;
    __syncthreads();
  }
  if (r.top_p < 1.f) {
    const double need = (double)r.top_p * kept;
    if (tid == 0) S.bin = -1;
    __syncthreads();
    // the bin where the mass reaches the need; of nothing, the first
    if (tid < kBins && count > 0 && mass_before + mass >= need && (mass_before < need || count_before == 0))
      S.bin = tid;
    __syncthreads();
    const int bin = S.bin;
    if (bin >= 0) {
      work.refine(bin, {false, 0, need});
      if (S.cut > cut) cut = S.cut;
      __syncthreads();
    }
  }
  // min-p's cut is a logit; the top entry always stays
  double least = -INFINITY;
  if (r.min_p > 0.f) least = log((double)r.min_p);
  // Mass that each chunk keeps: whole bins from its histogram; entry by entry
  // in the cut's bin, or in three around min-p's bound (its bin is known to
  // one, since the bound itself is rounded).
  int bin_cut = kBins - 1;          // bins before it are kept whole
  int bin_end = kBins - 1;          // nothing is kept from here on
  if (cut) {
    unsigned ignore;
    bin_cut = classify(logit_of_key((unsigned)(cut >> 32)), r.width, top, &ignore);
    bin_end = bin_cut + 1;
  }
  if (r.min_p > 0.f) {
    const double d = top - floor(((double)mx + r.temp * least) * r.width) - 1.0;
    const int b = d < 0 ? 0 : d < kBins - 1 ? (int)d : kBins - 1;
    bin_cut = min(bin_cut, b);
    bin_end = min(bin_end, b + 3);
  }
  auto keeps = [&](float l, int v) {
    return l > -INFINITY && order_of(l, v) >= cut &&
           (r.min_p == 0.f || ((double)l - (double)mx) / r.temp >= least);
  };
  const int lane = lane_id(), w = tid >> 6;
  for (int s = w; s < n_chunks; s += kRowThreads / kWave) {
    const ChunkRec rec = chunk_rec(p, n_chunks, m, s);
    const int off = S.chunk_off[s];
    double sum = 0.0;
    for (int g = off + lane; g < bin_cut; g += kWave)
      sum += (double)(rec.hist[g - off] & kMassMask) * S.edge[g];
    u64 some[3] = {0, 0, 0};
    auto add = [&](float l, int v) {
      if (!(l > -INFINITY)) return;
      unsigned ms;
      const int g = classify(l, r.width, top, &ms) - bin_cut;
      if (g >= 0 && g < 3 && keeps(l, v)) {
        if (g == 0) some[0] += ms;
        else if (g == 1) some[1] += ms;
        else some[2] += ms;
      }
    };
    if (bin_cut < bin_end && off < bin_end) {
      if (min(bin_end, kBins - 1) - off <= S.chunk_cover[s]) {
        for (int i = lane; i < S.chunk_listed[s]; i += kWave) add(rec.list[i].l, rec.list[i].v);
      } else {
        const int v1 = min((s + 1) * kChunk, p.V);
        for (int v = s * kChunk + lane; v < v1; v += kWave) add(logit<DT>(p, m, v), v);
      }
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
      sum += __shfl_xor(sum, o, kWave);
#pragma unroll
      for (int i = 0; i < 3; ++i) some[i] += __shfl_xor(some[i], o, kWave);
    }
    if (lane == 0) {
#pragma unroll
      for (int i = 0; i < 3; ++i)
        if (bin_cut + i < kBins) sum += (double)some[i] * S.edge[bin_cut + i];
      S.chunk_mass[s] = sum * unit;
    }
  }
  __syncthreads();
  if (tid == 0) {
    double all = 0.0;
    for (int s = 0; s < n_chunks; ++s) all += S.chunk_mass[s];
    const double goal = (double)p.u[m] * all;
    double at = 0.0;
    int pick = -1, last = 0;
    for (int s = 0; s < n_chunks && pick < 0; ++s) {
      if (S.chunk_mass[s] > 0.0) {
        last = s;
        if (at + S.chunk_mass[s] > goal) pick = s;
        else at += S.chunk_mass[s];
      }
    }
    if (pick < 0) {                 // u at or above 1
      pick = last;
      at -= S.chunk_mass[last];
    }
    S.chunk = pick;
    S.rest = goal - at;
    S.all = all;
    S.token = -1;
  }
  __syncthreads();
  // The entry: threads take neighbouring entries of the chunk.
  constexpr int PER = kChunk / kRowThreads;
  const int v0 = S.chunk * kChunk + tid * PER, v1 = min(v0 + PER, p.V);
  const double goal = S.rest;
  double mine = 0.0;
  int last = -1;
  float x[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int v = v0 + i;
    x[i] = v < v1 ? logit<DT>(p, m, v) : -INFINITY;
    if (keeps(x[i], v)) {
      unsigned ms;
      const int g = classify(x[i], r.width, top, &ms);
      mine += (double)ms * S.edge[g] * unit;
      if (ms) last = v;
    }
  }
  double all;
  const double pre = block_scan<double>(mine, S.part_d, &all);
  if (mine > 0.0 && pre <= goal && pre + mine > goal) {
    double c = pre;
    int tok = last;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int v = v0 + i;
      if (keeps(x[i], v)) {
        unsigned ms;
        const int g = classify(x[i], r.width, top, &ms);
        const double c1 = c + (double)ms * S.edge[g] * unit;
        if (c <= goal && c1 > goal && v <= tok) tok = v;
        c = c1;
      }
    }
    S.token = tok;
  }
  __syncthreads();
  if (S.token < 0) {                // rounding, or u at or above 1: the last entry with a mass
    if (last >= 0) atomicMax(&S.found, last + 1);
    __syncthreads();
    if (tid == 0) S.token = S.found - 1;
    __syncthreads();
  }
  if (tid == 0) {
    const int tok = S.token;
    p.token[m] = tok;
    if (p.logp) {
      float lp = __uint_as_float(0x7fc00000u);
      if (tok >= 0) {
        unsigned ms;
        const int g = classify(logit<DT>(p, m, tok), r.width, top, &ms);
        lp = (float)log((double)ms * S.edge[g] * unit / S.all);
      }
      p.logp[m] = lp;
    }
  }
}

int chunks_of(int V) { return (V + kChunk - 1) / kChunk; }

}  // namespace

size_t sample_logits_workspace(int M, int V) { return (size_t)M * chunks_of(V) * kChunkBytes; }

hipError_t launch_sample_logits(const SampleLogitsLaunch& L, hipStream_t st) {
  const int nc = chunks_of(L.V);
  const int size = L.dtype_bf16 ? 2 : 4;
  const bool vec = ((uintptr_t)L.logits & 15) == 0 && L.stride * size % 16 == 0 && (size_t)L.V * size % 16 == 0;
  trace_begin(st);
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(L.M * nc), dim3(256), 0, st, L, nc); };
  if (L.dtype_bf16) {
    if (vec) go(chunk_kernel<bf16, true>); else go(chunk_kernel<bf16, false>);
  } else {
    if (vec) go(chunk_kernel<float, true>); else go(chunk_kernel<float, false>);
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  trace_mark(st);
  if (L.dtype_bf16) hipLaunchKernelGGL(row_kernel<bf16>, dim3(L.M), dim3(kRowThreads), 0, st, L, nc);
  else hipLaunchKernelGGL(row_kernel<float>, dim3(L.M), dim3(kRowThreads), 0, st, L, nc);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  trace_mark(st);
  return hipSuccess;
}

}  // namespace ipdv
