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
// step of an fp32 u).
// An entry adds 2^45 + 2^30 m to its bin, m its mass against the bin's upper
// edge: one 64-bit LDS addition counts and sums.  Sums of whole numbers do not
// depend on the order of the atomics, so a call repeats bit for bit; m itself is
// an fp32 exponential of an argument of about 1/8, and joined sums are in
// double.  Where exactly a bin ends does not matter, but both kernels must find
// an entry in the same one: it is the floor of y in fp32, a function of the
// logit and T alone, and the rounding of y goes into m.
//
//   chunk kernel  one workgroup per 16384 entries: reads the logits once, into
//                 registers; its histogram below its own maximum (bins are
//                 aligned, since they are floors of y), and its topmost
//                 entries, bin by bin, as far as a cut may lie.
//   row kernel    one workgroup per row: adds the histograms up, finds the cut's
//                 bin, takes the bin's entries from the lists (or from the
//                 logits where a list stops above the bin) and in them the cut;
//                 then the chunk, and in it the entry, where the mass passes u.
//                 Bound by latency, so all histograms are asked for at its start
//                 and stay in registers, and its loops stay rolled where they
//                 can (63 KB of code took 17 us even unfiltered).
//
// At V = 151936: one fp32 row takes 5 us and 11 unfiltered, 8.5 and 17 with top-p
// 0.9; 64 bf16 rows 11 and 11, and 18 and 17.  The chunk kernel is bound by its
// vector instructions (31 to 35 an entry with the list's pass, which issue 81% of
// the time) and LDS atomics, of which it gives rows that need none (an unfiltered
// one: a mass per chunk would do) as many as the others; the row kernel by the
// latency of some ten dependent steps.  Lists that were not in bin order had to be
// searched, and ended higher: a mixed batch of 64 took 58 us where this takes 37.
//
// A bin of many entries (equal logits by the thousand) is narrowed by digits of
// the entries' order numbers until 256 are left, in LDS or, where they do not
// fit there, over the row's logits.
#include <type_traits>

#include "common.h"
#include "kernels.h"

namespace ipdv {
namespace {

constexpr int kChunk = 16384;     // entries per workgroup of the chunk kernel
constexpr int kBins = 256;
constexpr int kList = 2048;       // topmost entries that a chunk lists
constexpr int kHold = 4096;       // entries of one bin that LDS holds
constexpr int kSort = 256;        // entries that are ordered
constexpr int kMaxChunks = 16;    // V <= 262144
constexpr double kWidth = 8.0;    // bins per unit of l / T
constexpr int kCountShift = 45;   // 16384 masses of about 2^30 at most stay below
constexpr unsigned long long kMassMask = (1ull << kCountShift) - 1;
typedef unsigned long long u64;

struct ChunkHead {
  double floor_max;   // floor(y) of the chunk's maximum, -inf without a finite logit
  float max;
  int bad;            // holds NaN or +inf
  int covered;        // bins that the list holds, from the chunk's top bin
};
constexpr size_t kChunkBytes = kBins * (sizeof(u64) + sizeof(int)) + kList * sizeof(u64) + 64;
static_assert(sizeof(ChunkHead) <= 64, "chunk record");

struct ChunkRec {
  u64* hist;
  u64* list;          // order numbers, bin by bin
  int* start;         // [kBins]: where a bin's begin
  ChunkHead* head;
};
__device__ __forceinline__ ChunkRec chunk_rec(const SampleLogitsLaunch& p, int n_chunks, int m, int s) {
  char* at = reinterpret_cast<char*>(p.workspace) + ((size_t)m * n_chunks + s) * kChunkBytes;
  u64* hist = reinterpret_cast<u64*>(at);
  int* start = reinterpret_cast<int*>(hist + kBins + kList);
  return {hist, hist + kBins, start, reinterpret_cast<ChunkHead*>(start + kBins)};
}

// Temperatures below act as this: bins and slopes per unit of logit, 8 / T and
// log2(e) / T, stay finite in fp32.
constexpr float kLeastTemp = 0x1p-124f;

// A row's parameters; greedy (T = 0) is the top entry at temperature 1.
struct Row {
  double width;   // y = l * width
  float hi, lo;   // the same in two terms
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
  r.temp = t > 0.f ? (double)fmaxf(t, kLeastTemp) : 1.0;
  r.width = kWidth / r.temp;
  r.hi = (float)r.width;
  r.lo = (float)(r.width - (double)r.hi);
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

// floor(y) of a finite logit, and what y has above it (a little outside [0, 1)
// where fp32 has rounded y).  Products must not be contracted into the
// differences that follow: what they were rounded to counts.
constexpr float kFar = 16777216.f;      // from here on fp32 has no fraction left, and double takes over
__device__ __forceinline__ float floor_near(const Row& r, float l, float* rest) {
#pragma clang fp contract(off)
  const float y = l * r.hi, f = floorf(y);
  *rest = (y - f) + fmaf(l, r.lo, fmaf(l, r.hi, -y));
  return f;
}
__device__ __forceinline__ double floor_y(const Row& r, float l, float* rest) {
#pragma clang fp contract(off)
  if (fabsf(l * r.hi) < kFar) return (double)floor_near(r, l, rest);
  // A greater logit must not have a lesser floor (bins are differences from the
  // maximum's, and index arrays): fp32 floors reach kFar - 1, and where fp32 has
  // rounded its way up to kFar, z may still lie up to 1.5 below.
  const double z = (double)l * r.width, f = z > 0.0 ? fmax(floor(z), (double)kFar - 1.0) : floor(z);
  *rest = (float)(z - f);
  return f;
}
// 2^30 times the mass against the bin's upper edge: whole, as fp32 has 24 bits.
__device__ __forceinline__ unsigned mass_above(float rest) {
  constexpr float c = (float)(1.4426950408889634 / kWidth);
  return (unsigned)fast_exp2(fmaf(rest, c, 30.f - c));
}

// Bin of a finite logit below `top` = floor(y) of the maximum, and its mass
// against the bin's upper edge in units of 2^-30 (the last bin has none).
__device__ __forceinline__ int classify(const Row& r, float l, double top, unsigned* mass) {
  float x;
  const double d = top - floor_y(r, l, &x);
  if (!(d < kBins - 1)) {
    *mass = 0;
    return kBins - 1;
  }
  *mass = mass_above(x);
  return (int)d;
}

// Logits as unsigned numbers of the same order, and back to one of equal order.
__device__ __forceinline__ unsigned key_of(float l) {
  const unsigned u = __float_as_uint(l == 0.f ? 0.f : l);   // -0 is +0
  return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float logit_of_key(unsigned key) {
  return __uint_as_float((key & 0x80000000u) ? key & 0x7fffffffu : ~key);
}
// Order of entries: logit, then the lower index.
constexpr int kIndexBits = 18;
static_assert(kMaxChunks * kChunk <= 1 << kIndexBits, "an index has 18 bits");
__device__ __forceinline__ u64 order_of(float l, int v) {
  return ((u64)key_of(l) << kIndexBits) | (unsigned)(((1 << kIndexBits) - 1) ^ v);
}
__device__ __forceinline__ float logit_of(u64 order) { return logit_of_key((unsigned)(order >> kIndexBits)); }
__device__ __forceinline__ int index_of(u64 order) {
  return (int)(((1 << kIndexBits) - 1) ^ (unsigned)(order & ((1 << kIndexBits) - 1)));
}

template <typename DT>
__device__ __forceinline__ float logit(const SampleLogitsLaunch& p, int m, int v) {
  return to_f32(reinterpret_cast<const DT*>(p.logits)[(size_t)m * p.stride + v]);
}

constexpr int kThreads = 512;     // of both kernels
constexpr int kWaves = kThreads / kWave;

template <typename DT, bool VEC>
__global__ __launch_bounds__(kThreads, 6) void chunk_kernel(SampleLogitsLaunch p, int n_chunks) {
  constexpr int N = VEC ? 16 / (int)sizeof(DT) : 1;   // entries per load
  constexpr int PER = kChunk / kThreads;
  __shared__ u64 s_hist[kBins];
  __shared__ float s_max[kWaves];
  __shared__ int s_bad, s_cover, s_wave[kBins / kWave], s_at[kBins];
  const int m = blockIdx.x / n_chunks, s = blockIdx.x % n_chunks;
  const int tid = threadIdx.x, lane = lane_id(), w = tid >> 6;
  const int v0 = s * kChunk, n = min(kChunk, p.V - v0);
  const DT* src = reinterpret_cast<const DT*>(p.logits) + (size_t)m * p.stride + v0;
  // entry i of the thread: v0 + (i / N) * kThreads N + tid N + i % N; kept as it
  // came, since bf16 takes half the registers so
  typedef __attribute__((__vector_size__(16))) int i32x4;
  typedef std::conditional_t<VEC, i32x4, DT> Raw;
  Raw raw[PER / N];
#pragma unroll
  for (int i = 0; i < PER / N; ++i) {
    const int at = (i * kThreads + tid) * N;
    if (at < n) {                   // with VEC, n is a multiple of N
      raw[i] = *reinterpret_cast<const Raw*>(src + at);
    } else {
      DT e[N];
#pragma unroll
      for (int c = 0; c < N; ++c) e[c] = from_f32<DT>(-INFINITY);
      raw[i] = __builtin_bit_cast(Raw, e);
    }
  }
  struct Lane { DT e[N]; };
  // makes the compiler take the values as new: it would keep the fp32 forms of
  // one pass for the next, in registers that it does not have
  auto renew = [&] {
#pragma unroll
    for (int i = 0; i < PER / N; ++i) asm volatile("" : "+v"(raw[i]));
  };
  auto x = [&](int i) { return to_f32(__builtin_bit_cast(Lane, raw[i / N]).e[i % N]); };
  const Row r = row_of(p, m);
  if (tid < kBins) s_hist[tid] = 0;
  if (tid == 0) s_bad = s_cover = 0;
  float mx = -INFINITY;
  bool bad = false;
#pragma unroll
  for (int i = 0; i < PER; i += 2) {
    mx = fmaxf(mx, fmaxf(x(i), x(i + 1)));
    bad |= __builtin_isunordered(x(i), x(i + 1));
  }
  renew();
  mx = wave_max(mx);
  if (lane == 0) s_max[w] = mx;
  __syncthreads();
  if (bad) s_bad = 1;
#pragma unroll
  for (int i = 0; i < kWaves; ++i) mx = fmaxf(mx, s_max[i]);
  if (mx == INFINITY) s_bad = 1;
  const bool any = mx > -INFINITY && mx < INFINITY;
  float ignore;
  const double top = any ? floor_y(r, mx, &ignore) : -INFINITY;
  auto add = [&](int bin, unsigned mass) {
    __hip_atomic_fetch_add(&s_hist[bin], (1ull << kCountShift) + mass, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
  };
  const bool near = any && fabs(top) < 0.5 * kFar;      // whatever is not far below is near then
  if (near) {                       // the same without double
    const float ftop = (float)top;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      float rest;
      const float d = ftop - floor_near(r, x(i), &rest);       // infinite for -inf
      if (d < kBins - 1) add((int)d, mass_above(rest));
    }
  } else if (any) {
#pragma unroll 1
    for (int i = 0; i < PER; ++i) {
      float l = x(0);
#pragma unroll
      for (int c = 0; c < PER; ++c) l = c == i ? x(c) : l;
      unsigned mass;
      if (l > -INFINITY) {
        const int bin = classify(r, l, top, &mass);
        if (bin < kBins - 1) add(bin, mass);
      }
    }
  }
  __syncthreads();
  const ChunkRec rec = chunk_rec(p, n_chunks, m, s);
  // The list: whole bins from the top while they fit, and while a cut may lie in
  // them: in none behind k entries, and in none that far below the maximum that
  // min-p lets nothing pass (with top-k and top-p both, top-k's cut counts first).
  int cum = 0, count = 0;
  if (tid < kBins) {
    rec.hist[tid] = s_hist[tid];
    count = (int)(s_hist[tid] >> kCountShift);
    cum = wave_incl_scan_i(count);
    if (lane == kWave - 1) s_wave[w] = cum;
  }
  __syncthreads();
  if (tid < kBins) {
    for (int i = 0; i < w; ++i) cum += s_wave[i];
    s_at[tid] = rec.start[tid] = cum - count;
    bool fits = cum <= kList;
    if (r.k > 0) fits &= cum - count < r.k;
    if (r.min_p > 0.f && !(r.k > 0 && r.top_p < 1.f)) fits &= (float)tid <= 2.f - (float)kWidth * __logf(r.min_p);
    const u64 first = __ballot(fits);             // all three hold for the first bins
    if (lane == 0) atomicAdd(&s_cover, __popcll(first));
  }
  __syncthreads();
  const bool filtered = r.k > 0 || r.top_p < 1.f || r.min_p > 0.f;
  const int cover = any && filtered ? min(s_cover, kBins - 1) : 0;    // the last bin is never listed
  if (tid == 0) *rec.head = {top, mx, s_bad, cover};
  if (cover == 0) return;
  renew();
  const float ftop = (float)top;
  unsigned in = 0;                  // bit i: entry i is listed
  static_assert(PER <= 32, "a bit per entry");
  if (near) {
    const float least = ftop - (float)(cover - 1);       // floor(y) >= this, a whole number, where y is
#pragma unroll
    for (int i = 0; i < PER; ++i) in |= (x(i) * r.hi >= least ? 1u : 0u) << i;
  } else {
#pragma unroll 1
    for (int i = 0; i < PER; ++i) {
      float l = x(0), rest;
#pragma unroll
      for (int c = 0; c < PER; ++c) l = c == i ? x(c) : l;
      in |= (l > -INFINITY && top - floor_y(r, l, &rest) < cover ? 1u : 0u) << i;
    }
  }
  // Few, so a rolled loop, which cannot choose among registers: the cache still has them.
  constexpr int AT = 4;
  while (__any(in != 0)) {
    int v[AT];
    float l[AT];
#pragma unroll
    for (int k = 0; k < AT; ++k) {
      const int i = __ffs(in) - 1;
      v[k] = in ? (i / N * kThreads + tid) * N + i % N : -1;
      in &= in - 1;
      if (v[k] >= 0) l[k] = to_f32(src[v[k]]);
    }
#pragma unroll
    for (int k = 0; k < AT; ++k) {
      if (v[k] < 0) continue;
      float rest;
      const int bin = near ? (int)(ftop - floor_near(r, l[k], &rest)) : (int)(top - floor_y(r, l[k], &rest));
      rec.list[atomicAdd(&s_at[bin], 1)] = order_of(l[k], v0 + v[k]);
    }
  }
}

// ---- the row kernel ----

constexpr double kUnitMass = 1.0 / 1073741824.0;
constexpr int kHeldBins = kMaxChunks * kBins / kThreads;      // histogram bins of a thread

// Sum over the threads before this one; every thread calls.
template <typename T>
__device__ __forceinline__ T block_scan(T v, T* s_part) {
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
  T before = 0;
#pragma unroll
  for (int i = 0; i < kWaves; ++i)
    if (i < w) before += s_part[i];
  return before + incl - v;
}

// Two at once; the doubles also with this thread's, which is the next thread's
// sum before it to the last bit.
__device__ __forceinline__ int block_scan(int a, double b, int* part_a, double* part_b, double* before_b, double* end_b) {
  const int lane = lane_id(), w = threadIdx.x >> 6;
  const int incl_a = wave_incl_scan_i(a);
  double incl_b = b;
#pragma unroll
  for (int o = 1; o < kWave; o <<= 1) {
    const double up = __shfl_up(incl_b, o, kWave);
    if (lane >= o) incl_b += up;
  }
  __syncthreads();
  if (lane == kWave - 1) {
    part_a[w] = incl_a;
    part_b[w] = incl_b;
  }
  __syncthreads();
  int before_a = 0;
  double sum = 0.0;
#pragma unroll
  for (int i = 0; i < kWaves; ++i)
    if (i < w) {
      before_a += part_a[i];
      sum += part_b[i];
    }
  const double left = __shfl_up(incl_b, 1, kWave);
  *before_b = lane > 0 ? sum + left : sum;
  *end_b = sum + incl_b;
  return before_a + incl_a - a;
}

struct Shared {
  double edge[kBins];               // e^(-t/8): mass of bin t's upper edge
  float edge_f[kBins];
  double before[kBins];             // mass above bin t
  int count_before[kBins];
  int count[kBins];
  u64 mass[kBins];
  int off[kMaxChunks];              // the chunk's top bin in the row's bins (kBins: none)
  int cover[kMaxChunks];
  int start[kMaxChunks][kBins];     // where a chunk's list has its bin t
  double chunk_mass[kMaxChunks];
  u64 in_bin[kMaxChunks];           // kept mass of the cut's bin
  double grid[kMaxChunks][kBins + 1];   // mass by chunk and bin, the chunk's top bin first
  u64 hold[kHold];                  // order numbers of one bin's entries
  u64 few[kSort], sorted[kSort];
  int rank[kSort];
  int digit_count[256];
  u64 digit_mass[256];
  u64 part_u[kWaves];
  double part_d[kWaves];
  int part_i[kWaves];
  int n, found, chunk, token, bad;
  int bin[2];                       // where top-k's and top-p's cuts lie
  unsigned from_logits;             // chunks whose list stops above the bin looked for
  float low, high;                  // a bin's logits: [low, high)
  u64 cut, lo, hi, above_mass;
  int above, left;
  double rest, all;
  double top;                       // floor(y) of the row's maximum
  float max;
};

// What ends a prefix: a count of entries, or a mass to be reached.
struct Need {
  bool by_count;
  int count;
  double mass;
};

template <typename DT, bool VEC>
struct RowWork {
  const SampleLogitsLaunch& p;
  Shared& S;
  const Row r;
  const int m, n_chunks, tid;
  const double top;

  // Calls f(l, v) for the logits of the chunks in `chunks` that lie in
  // [low, high); the next chunk's logits are on their way meanwhile.
  template <class F>
  __device__ void scan(unsigned chunks, float low, float high, F f) {
    constexpr int PER = 16, N = VEC ? 16 / (int)sizeof(DT) : 1;      // a half of a chunk at a time
    typedef __attribute__((__vector_size__(16))) int i32x4;
    typedef std::conditional_t<VEC, i32x4, DT> Raw;
    Raw raw[PER / N];
    const DT* row = reinterpret_cast<const DT*>(p.logits) + (size_t)m * p.stride;
    auto load = [&](int v0) {
#pragma unroll
      for (int i = 0; i < PER / N; ++i)
        if (v0 + (i * kThreads + tid) * N < p.V) raw[i] = *reinterpret_cast<const Raw*>(row + v0 + (i * kThreads + tid) * N);
    };
    int half = 0, v0 = chunks ? (__ffs(chunks) - 1) * kChunk : 0;
    if (chunks) load(v0);
    while (chunks) {
      const int now = v0;
      unsigned in = 0;              // bit i: entry i lies in the range
#pragma unroll
      for (int i = 0; i < PER / N; ++i) {
        const DT* e = reinterpret_cast<const DT*>(&raw[i]);
        const bool on = now + (i * kThreads + tid) * N < p.V;
#pragma unroll
        for (int c = 0; c < N; ++c) {
          const float l = to_f32(e[c]);
          in |= (on && l >= low && l < high ? 1u : 0u) << (i * N + c);
        }
      }
      half ^= 1;
      if (!half) chunks &= chunks - 1;
      if (chunks) {
        v0 = (__ffs(chunks) - 1) * kChunk + half * (kChunk / 2);
        load(v0);
      }
      for (; in; in &= in - 1) {    // few, and still in the cache
        const int i = __ffs(in) - 1, v = now + (i / N * kThreads + tid) * N + i % N;
        f(logit<DT>(p, m, v), v);
      }
    }
  }
  static_assert(kChunk == 2 * 16 * kThreads, "two halves of 16 per thread");

  // The logits of a bin: S.low (the least one that is in it or above) and
  // S.high (that of the bin above), two lanes of a search over the floats.
  // Wave 0 calls.
  __device__ void bounds(int bin) {
    const int b = bin - (tid & 1);
    const double goal = top - (double)b;
    const unsigned most = key_of(S.max);
    unsigned lo = key_of(-__FLT_MAX__) - 1u, hi = most;     // the floor is below the goal at lo (taken so), not at hi
    if (b >= 0) {
      const unsigned guess = key_of((float)(goal / r.width));
      float x;
      if (guess - 8u > lo && guess + 8u < hi && guess > 8u) {
        if (floor_y(r, logit_of_key(guess - 8u), &x) < goal) lo = guess - 8u;
        if (floor_y(r, logit_of_key(guess + 8u), &x) >= goal) hi = guess + 8u;
      }
      while (hi - lo > 1u) {
        const unsigned mid = lo + (hi - lo) / 2;
        if (floor_y(r, logit_of_key(mid), &x) >= goal) hi = mid; else lo = mid;
      }
    }
    if (tid == 0) S.low = logit_of_key(hi);
    if (tid == 1) S.high = b >= 0 ? logit_of_key(hi) : INFINITY;
  }

  // The entries of a bin into S.hold; false if they do not fit there.  Where the
  // logits are read for them, or they are too many to be ordered at once, the
  // bin's bounds too: S.low, S.high.
  __device__ bool gather(int bin) {
    const bool fit = S.count[bin] <= kHold;
    __syncthreads();
    if (tid < kWave) {
      bool more = false;
      if (tid < n_chunks) more = S.off[tid] <= bin && bin - S.off[tid] >= S.cover[tid];
      const u64 b = __ballot(more);
      if (b || S.count[bin] > kSort) bounds(bin);
      if (tid == 0) {
        S.from_logits = (unsigned)b;
        S.n = 0;
      }
    }
    __syncthreads();
    if (!fit) return false;
    constexpr int PART = kThreads / kMaxChunks;        // threads of a chunk
    const int s = tid / PART, c = tid % PART;
    int first = 0, n = 0;
    if (s < n_chunks) {
      const int b = bin - S.off[s];
      if (b >= 0 && b < S.cover[s]) {                  // the last bin is never covered
        first = S.start[s][b];
        n = S.start[s][b + 1] - first;
      }
    }
    int at = 0;
    if (c == 0 && n) at = atomicAdd(&S.n, n);
    at = __shfl(at, lane_id() & ~(PART - 1), kWave);
    const u64* list = chunk_rec(p, n_chunks, m, s).list + first;
    for (int i = c; i < n; i += PART) S.hold[at + i] = list[i];
    const unsigned more = S.from_logits;
    if (more)
      scan(more, S.low, S.high, [&](float l, int v) {
        const int to = atomicAdd(&S.n, 1);
        if (to < kHold) S.hold[to] = order_of(l, v);
      });
    __syncthreads();
    return true;
  }

  // Calls f(order) for every entry of the gathered bin.
  template <class F>
  __device__ void each(bool held, F f) {
    if (held) {
      const int n = min(S.n, kHold);
      for (int i = tid; i < n; i += kThreads) f(S.hold[i]);
    } else {
      scan((1u << n_chunks) - 1u, S.low, S.high, [&](float l, int v) { f(order_of(l, v)); });
    }
  }
  __device__ u64 mass_of(u64 order) const {
    unsigned mass;
    classify(r, logit_of(order), top, &mass);
    return mass;
  }

  // The cut of a prefix that ends in the gathered bin: S.cut.
  __device__ void select(int bin, bool held, Need need) {
    const double base = S.before[bin], e = S.edge[bin] * kUnitMass;
    const int first = S.count_before[bin];
    // what is kept: entries with less than the need before them
    auto before = [&](int c, u64 mass) { return need.by_count ? first + c < need.count : base + e * (double)mass < need.mass; };
    if (held && S.count[bin] <= kWave) {       // a wave's: the usual top-k, without the workgroup's barriers
      if (tid < kWave) {
        const int n = S.count[bin];
        const u64 mine = tid < n ? S.hold[tid] : 0;
        int rank = 0;
#pragma unroll 8
        for (int c = 0; c < n; ++c) rank += S.hold[c] > mine;
        if (tid < n) S.sorted[rank] = mine;
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");       // LDS keeps a wave's order: this binds the compiler only
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
        const u64 o = tid < n ? S.sorted[tid] : 0, w = tid < n ? mass_of(o) : 0;
        u64 upto = w;
#pragma unroll
        for (int i = 1; i < kWave; i <<= 1) {
          const u64 up = __shfl_up(upto, i, kWave);
          if (tid >= i) upto += up;
        }
        const bool here = tid < n && (tid == 0 || before(tid, upto - w));
        const bool next = tid + 1 < n && before(tid + 1, upto);
        if (here && !next) S.cut = o;
      }
      __syncthreads();
      return;
    }
    if (tid == 0) {
      S.lo = 0;
      S.hi = ~0ull;
      if (S.count[bin] > kSort) {
        S.lo = (u64)key_of(S.low) << kIndexBits;
        S.hi = ((u64)key_of(S.high < INFINITY ? S.high : S.max) + (S.high < INFINITY ? 0u : 1u)) << kIndexBits;
        S.hi -= 1;
      }
      S.above = 0;
      S.above_mass = 0;
      S.left = S.count[bin];
    }
    __syncthreads();
    while (S.left > kSort) {        // by the highest digit in which lo and hi differ
      const u64 lo = S.lo, hi = S.hi;
      const int shift = max(0, 56 - __clzll((long long)(lo ^ hi)));
      if (tid < 256) {
        S.digit_count[tid] = 0;
        S.digit_mass[tid] = 0;
      }
      if (tid == 0) S.found = -1;
      __syncthreads();
      each(held, [&](u64 o) {
        if (o < lo || o > hi) return;
        const int d = (int)(o >> shift) & 255;
        atomicAdd(&S.digit_count[d], 1);
        __hip_atomic_fetch_add(&S.digit_mass[d], mass_of(o), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
      });
      __syncthreads();
      const int d = 255 - tid;      // from the top
      const int c = tid < 256 ? S.digit_count[d] : 0;
      const u64 w = tid < 256 ? S.digit_mass[d] : 0;
      const int c0 = block_scan<int>(c, S.part_i);
      const u64 w0 = block_scan<u64>(w, S.part_u);
      if (c > 0 && (c0 == 0 || before(S.above + c0, S.above_mass + w0))) atomicMax(&S.found, tid);
      __syncthreads();
      const int a = S.above;
      const u64 am = S.above_mass;
      __syncthreads();
      if (tid == S.found) {
        S.above = a + c0;
        S.above_mass = am + w0;
        S.left = c;
        const u64 low = (((lo >> shift) & ~255ull) | (u64)d) << shift;
        S.lo = max(low, lo);
        S.hi = min(low + ((1ull << shift) - 1), hi);
      }
      __syncthreads();
    }
    // order what is left: every entry's rank, counted by as many threads as there are for it
    if (tid == 0) S.n = min(S.n, kHold);
    if (tid < kSort) S.rank[tid] = 0;
    if (tid == 0) S.found = 0;
    __syncthreads();
    const u64 lo = S.lo, hi = S.hi;
    each(held, [&](u64 o) {
      if (o < lo || o > hi) return;
      const int at = atomicAdd(&S.found, 1);
      if (at < kSort) S.few[at] = o;
    });
    __syncthreads();
    const int n = min(S.found, kSort);
    int span = 64;
    while (span < n) span *= 2;
    const int mine = tid & (span - 1);
    if (mine < n) {
      const u64 o = S.few[mine];
      int rank = 0;
      for (int c = tid / span; c < n; c += kThreads / span) rank += S.few[c] > o;
      atomicAdd(&S.rank[mine], rank);
    }
    __syncthreads();
    if (tid < n) S.sorted[S.rank[tid]] = S.few[tid];
    __syncthreads();
    const u64 o = tid < n ? S.sorted[tid] : 0, w = tid < n ? mass_of(o) : 0;
    const u64 pre = S.above_mass + block_scan<u64>(w, S.part_u);
    const bool here = tid < n && (tid == 0 || before(S.above + tid, pre));
    const bool next = tid + 1 < n && before(S.above + tid + 1, pre + w);
    if (here && !next) S.cut = o;
    __syncthreads();
  }

  // What the chunks keep of the gathered bin, given the cut: into S.in_bin.
  __device__ void record(bool held, u64 cut) {
    each(held, [&](u64 o) {
      if (o >= cut)
        __hip_atomic_fetch_add(&S.in_bin[index_of(o) / kChunk], mass_of(o), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
    });
    __syncthreads();
  }
};

template <typename DT, bool VEC>
__global__ __launch_bounds__(kThreads) void row_kernel(SampleLogitsLaunch p, int n_chunks) {
  __shared__ Shared S;
  const int m = blockIdx.x, tid = threadIdx.x, lane = lane_id(), w = tid >> 6;
  const int t = tid & (kBins - 1), side = tid / kBins;
  // everything that the row is known by: bins t of every other chunk
  u64 hist[kHeldBins];
  int start[kHeldBins];
#pragma unroll
  for (int i = 0; i < kHeldBins; ++i) {
    hist[i] = 0;
    if (2 * i + side < n_chunks) hist[i] = chunk_rec(p, n_chunks, m, 2 * i + side).hist[t];
  }
  const Row r = row_of(p, m);
  const double u = (double)p.u[m];
  const bool filtered = r.k > 0 || r.top_p < 1.f || r.min_p > 0.f;
  if (filtered) {
#pragma unroll
    for (int i = 0; i < kHeldBins; ++i)
      if (2 * i + side < n_chunks) start[i] = chunk_rec(p, n_chunks, m, 2 * i + side).start[t];
  }
  if (tid < kWave) {                // a lane per chunk
    double ct = -INFINITY;
    float cm = -INFINITY;
    bool bad = r.bad;
    if (tid < n_chunks) {
      const ChunkHead h = *chunk_rec(p, n_chunks, m, tid).head;
      ct = h.floor_max;
      cm = h.max;
      bad |= h.bad != 0;
      S.cover[tid] = h.covered;
    }
    double all = ct;
#pragma unroll
    for (int o = kMaxChunks / 2; o > 0; o >>= 1) all = fmax(all, __shfl_xor(all, o, kWave));
    all = __shfl(all, 0, kWave);
    const float mx = wave_max(cm);
    if (tid < n_chunks) S.off[tid] = all - ct < kBins ? (int)(all - ct) : kBins;
    bad = __any(bad) || !(mx > -INFINITY);
    if (tid == 0) {
      S.max = mx;
      S.top = all;
      S.bad = bad;
    }
  }
  if (tid < kBins) {
    S.edge[t] = exp(-(double)t / kWidth);
    S.edge_f[t] = (float)(S.edge[t] * kUnitMass);
    S.mass[t] = 0;
    S.count[t] = 0;
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
  // The row's bins; below the last one nothing counts.
#pragma unroll
  for (int i = 0; i < kHeldBins; ++i) {
    const int s = 2 * i + side;
    if (s >= n_chunks) continue;
    const int g = t + S.off[s];
    S.grid[s][t] = g < kBins ? (double)(hist[i] & kMassMask) * S.edge[g] : 0.0;
    if (filtered && g < kBins - 1 && hist[i]) {
      atomicAdd(&S.count[g], (int)(hist[i] >> kCountShift));
      __hip_atomic_fetch_add(&S.mass[g], hist[i] & kMassMask, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
    }
  }
  u64 cut = 0;                      // everything is at or above it
  int bin_cut = kBins - 1;          // bins before it are kept whole, of later ones nothing
  if (filtered) {
#pragma unroll
    for (int i = 0; i < kHeldBins; ++i)
      if (2 * i + side < n_chunks) S.start[2 * i + side][t] = start[i];
    __syncthreads();
    const int count = tid < kBins ? S.count[t] : 0;
    const double mass = tid < kBins ? (double)S.mass[t] * S.edge[t] * kUnitMass : 0.0;
    double mass_before, mass_end;
    const int count_before = block_scan(count, mass, S.part_i, S.part_d, &mass_before, &mass_end);
    if (tid < kBins) {
      S.before[t] = mass_before;
      S.count_before[t] = count_before;
    }
    if (tid == kBins - 1) S.all = mass_before;         // the last bin has none
    if (tid < 2) S.bin[tid] = kBins - 1;
    __syncthreads();
    RowWork<DT, VEC> work{p, S, r, m, n_chunks, tid, top};
    double kept = S.all;            // mass of what the filters so far leave
    bool held = false;
    u64 bound = 0;                  // min-p's cut is the least logit that passes
    int bin_min = kBins - 1;
    if (r.min_p > 0.f) {
      const double x = log((double)r.min_p), least = (double)mx + (x < 0.0 ? x * r.temp : 0.0);
      float l = (float)least;
      if ((double)l < least) l = nextafterf(l, INFINITY);
      if (l > -INFINITY) {
        unsigned ignore;
        bound = (u64)key_of(l) << kIndexBits;
        bin_min = classify(r, logit_of(bound), top, &ignore);
      }
    }
#pragma unroll 1
    for (int pass = 0; pass < 3; ++pass) {             // top-k, top-p, min-p
      if (pass == 0 ? r.k == 0 : pass == 1 ? r.top_p == 1.f : r.min_p == 0.f) continue;
      const Need need{pass == 0, r.k, (double)r.top_p * kept};
      if (pass == 2 && bound <= cut) continue;
      // the first bin whose end meets the need, of those that hold entries
      const u64 meets = __ballot(pass < 2 && count > 0 && (pass == 0 ? count_before + count >= r.k : mass_end >= need.mass));
      if (lane == 0 && meets) atomicMin(&S.bin[pass], w * kWave + __ffsll((long long)meets) - 1);
      __syncthreads();
      const int bin = pass < 2 ? S.bin[pass] : bin_min;
      if (bin == kBins - 1) continue;                  // nothing that counts is cut
      if (pass < 2 && bin > bin_min && (pass == 1 || r.top_p == 1.f)) continue;      // min-p cuts above it
      if (tid < kMaxChunks) S.in_bin[tid] = 0;         // record's, from here on the last cut's
      if (bin != bin_cut) held = work.gather(bin);
      else if (pass == 2) __syncthreads();
      if (pass < 2) work.select(bin, held, need);
      cut = pass < 2 ? S.cut : bound;                  // at or above the last one
      work.record(held, cut);
      bin_cut = bin;
      u64 in = 0;
      for (int s = 0; s < n_chunks; ++s) in += S.in_bin[s];
      kept = S.before[bin] + S.edge[bin] * kUnitMass * (double)in;
    }
  }
  __syncthreads();
  {
    constexpr int PART = kThreads / kMaxChunks;        // threads of a chunk
    const int s = tid / PART, c = tid % PART;
    double sum = 0.0;
    if (s < n_chunks)
      for (int b = c; b < bin_cut - S.off[s]; b += PART) sum += S.grid[s][b];
#pragma unroll
    for (int o = PART / 2; o > 0; o >>= 1) sum += __shfl_xor(sum, o, kWave);
    if (c == 0) {
      if (bin_cut < kBins - 1 && s < n_chunks) sum += (double)S.in_bin[s] * S.edge[bin_cut];
      S.chunk_mass[s] = sum * kUnitMass;
    }
  }
  __syncthreads();
  if (w == 0) {                     // the chunk where the mass passes u
    const double mine = lane < kMaxChunks ? S.chunk_mass[lane] : 0.0;
    double incl = mine;
#pragma unroll
    for (int o = 1; o < kMaxChunks; o <<= 1) {
      const double up = __shfl_up(incl, o, kWave);
      if (lane >= o) incl += up;
    }
    const double all = __shfl(incl, kMaxChunks - 1, kWave);
    const double goal = u * all;
    const u64 some = __ballot(mine > 0.0);
    u64 hit = __ballot(mine > 0.0 && incl > goal);
    if (hit == 0) hit = 1ull << (63 - __clzll((long long)(some | 1)));      // u at or above 1: the last
    const int pick = __ffsll((long long)hit) - 1;
    if (lane == pick) {
      S.chunk = pick;
      S.rest = goal - (incl - mine);
      S.all = all;
      S.token = kThreads;
      S.found = 0;
    }
  }
  __syncthreads();
  // The entry: threads take neighbouring entries of the chunk.
  constexpr int PER = kChunk / kThreads;
  const int v0 = S.chunk * kChunk + tid * PER;
  const double goal = S.rest;
  float x[PER];
  if (VEC && v0 + PER <= p.V) {
    constexpr int N = 16 / (int)sizeof(DT);
    typedef __attribute__((__vector_size__(16))) int i32x4;
    const DT* src = reinterpret_cast<const DT*>(p.logits) + (size_t)m * p.stride + v0;
#pragma unroll
    for (int i = 0; i < PER; i += N) {
      const i32x4 raw = ld16<i32x4>(src + i);
      const DT* e = reinterpret_cast<const DT*>(&raw);
#pragma unroll
      for (int c = 0; c < N; ++c) x[i + c] = to_f32(e[c]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < PER; ++i) x[i] = v0 + i < p.V ? logit<DT>(p, m, v0 + i) : -INFINITY;
  }
  const float l_cut = cut ? logit_of(cut) : -__FLT_MAX__;
  const int v_cut = cut ? index_of(cut) : p.V;
  // The mass of a kept entry against the upper edge of the maximum's bin, 2^x with
  // x = (l - max) log2(e) / T + what the maximum lies below that edge.  x is off by
  // 2^-24 of itself, which counts where the mass is small only: below 10^-7 of the
  // row's all together.  (By the bin, as the chunk kernel has it, an entry takes 25
  // instructions instead of 10: unfiltered rows took 12.5 us, and take 10.)
  float from_edge;
  floor_y(r, mx, &from_edge);
  constexpr float kPerBin = (float)(1.4426950408889634 / kWidth);
  const float slope = (float)(1.4426950408889634 / r.temp), offset = (from_edge - 1.f) * kPerBin;
  auto weight = [&](float l, int v) -> float {
    const float x = fmaf(fmaxf(l - mx, -__FLT_MAX__), slope, offset);
    const bool kept = l > l_cut || (l == l_cut && v <= v_cut);
    return kept && x > -kBins * kPerBin * 1.000001f ? fast_exp2(x) : 0.f;
  };
  float part = 0.f;                 // a thread's share in fp32: off by 2^-24 of little
#pragma unroll
  for (int i = 0; i < PER; ++i) part += weight(x[i], v0 + i);
  const double mine = (double)part;
  const double pre = block_scan<double>(mine, S.part_d);
  const u64 some = __ballot(mine > 0.0), past = __ballot(mine > 0.0 && pre + mine > goal);
  if (lane == 0 && some) atomicMax(&S.found, w * kWave + 63 - __clzll((long long)some));
  if (lane == 0 && past) atomicMin(&S.token, w * kWave + __ffsll((long long)past) - 1);
  __syncthreads();
  // The first thread whose end passes the goal has it; rounding, or u at or above
  // 1, leave it to the last that holds some.  A lane per entry finds which.
  const int who = S.token < kThreads ? S.token : S.found;
  if (tid == who) S.rest = goal - pre;
  __syncthreads();
  if (w == 0) {
    static_assert(PER <= kWave, "a lane per entry");
    const int v = S.chunk * kChunk + who * PER + lane;
    const float l = lane < PER && v < p.V ? logit<DT>(p, m, v) : -INFINITY;
    const double one = (double)weight(l, v);
    double incl = one;
#pragma unroll
    for (int o = 1; o < PER; o <<= 1) {
      const double up = __shfl_up(incl, o, kWave);
      if (lane >= o) incl += up;
    }
    const u64 some = __ballot(one > 0.0);
    u64 hit = __ballot(one > 0.0 && incl > S.rest);
    if (hit == 0) hit = 1ull << (63 - __clzll((long long)(some | 1)));
    if (lane == __ffsll((long long)hit) - 1) {
      p.token[m] = v;
      if (p.logp) {                 // by the masses that S.all is a sum of: ln 1 is 0 then
        unsigned mass;
        const int g = classify(r, l, top, &mass);
        p.logp[m] = mass ? (float)log((double)((float)mass * S.edge_f[g]) / S.all)
                         : (float)(((double)l * r.width - (top + 1.0)) / kWidth - log(S.all));
      }
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
  auto go = [&](auto kernel, int n) { hipLaunchKernelGGL(kernel, dim3(n), dim3(kThreads), 0, st, L, nc); };
  if (L.dtype_bf16) {
    if (vec) go(chunk_kernel<bf16, true>, L.M * nc); else go(chunk_kernel<bf16, false>, L.M * nc);
  } else {
    if (vec) go(chunk_kernel<float, true>, L.M * nc); else go(chunk_kernel<float, false>, L.M * nc);
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  trace_mark(st);
  if (L.dtype_bf16) {
    if (vec) go(row_kernel<bf16, true>, L.M); else go(row_kernel<bf16, false>, L.M);
  } else {
    if (vec) go(row_kernel<float, true>, L.M); else go(row_kernel<float, false>, L.M);
  }
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  trace_mark(st);
  return hipSuccess;
}

}  // namespace ipdv
