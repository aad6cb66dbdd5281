// The verdict on drafted tokens by the two models' probabilities, for gfx950.  With p and q
// the target's and the draft's (filtered) distributions at a row, x its drafted token:
//
//   accepted while u q(x) < p(x);  at the first row that is not, the token is drawn from
//   max(0, p - q) / sum max(0, p - q), and at a row without a draft from p
//
// so that whatever is emitted is distributed as p.
//
//   stats kernel    one workgroup per row, model and 8192 entries: maximum and mass against
//                   it.  Reads every logit once; bound by their bytes as much as by its
//                   vector instructions.
//   rest kernel     one workgroup per sequence and 8192 entries: the sequence's first row that
//                   ends it, from the rows' masses (every workgroup for itself), and the mass of
//                   max(0, p - q) in the chunk where that row is a rejected draft.
//   draw kernel     one workgroup per sequence: the chunk where the mass passes u, in it
//                   the entry.
//
// Precision.  A token is a whole number next to borders that lie as close as the
// smallest probabilities, and a rejected row's masses are differences: all masses are
// 64-bit floats.  2^y is 2^n (integer added to the exponent) times a polynomial of degree 7 on
// [-1/2, 1/2], fitted to 4e-11 of the result, 14 instructions an entry, at fp32's rate on this
// card.
//
// Filters: sample_logits' kernels find every row's cut first (what is ordered before it
// is not kept).  A row of temperature 0 keeps its first maximum: with no filters the
// stats kernel finds that.
#include <type_traits>

#include "common.h"
#include "kernels.h"
#include "logit_order.h"

namespace ipdv {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kWave;
constexpr int kChunk = 8192;
constexpr int kPer = kChunk / kThreads;
constexpr int kMaxChunks = 32;     // V <= 262144
typedef unsigned long long u64;

// A chunk of one row: its kept mass against its maximum, which it may have none of.
struct Rec {
  double mass;
  u64 top;           // order number of the first maximum (temperature 0 only)
  float max;
  int bad;           // holds NaN or +inf
};
static_assert(sizeof(Rec) == 24, "records");

// One model's logits and what is known of them.
struct Model {
  const void* logits;
  long stride;
  const float* temperature;
  const u64* cuts;   // [T] or null: everything is kept
  Rec* recs;         // [T][chunks]
};
struct DraftParams {
  Model target, draft;       // draft.logits null: the drafts are certain
  int T, V, B, chunks;
  const int32_t* prop_tok;
  const int32_t* cu_q;
  const float* u_accept;
  const float* u_draw;
  int32_t eos_id;
  int32_t* n_acc;
  int32_t* token;
  uint8_t* finished;
  float* p_accept;
  float* logp;
  double* rest;              // [B][chunks]: masses of max(0, p - q)
  int* verdict;              // [B]: what find_end found
};

// 2^y for y <= 0 (and not below -1000).
__device__ __forceinline__ double exp2_of(double d, double slope) {
  const double magic = 6755399441055744.0;         // 1.5 * 2^52: the sum's low bits are the nearest whole number
  const double t = fma(d, slope, magic), f = fma(d, slope, magic - t);
  double p = 1.5201920948780836e-05;
  p = fma(p, f, 0.00015469291124750825);
  p = fma(p, f, 0.001333392256603758);
  p = fma(p, f, 0.009618027253729474);
  p = fma(p, f, 0.05550410353445379);
  p = fma(p, f, 0.2402265119815696);
  p = fma(p, f, 0.693147180728448);
  p = fma(p, f, 0.999999999961681);
  const u64 bits = __builtin_bit_cast(u64, p) + ((u64)__double2loint(t) << 52);
  return __builtin_bit_cast(double, bits);
}

// A row's temperature: log2(e) / T, and the distance from the maximum behind which nothing
// counts (2^-1000 of its mass).  T from 2^100 on acts as that, where an entry of -inf
// still counts for nothing.
constexpr float kMostTemp = 0x1p100f;
struct Scale {
  double slope, far;
  bool first_only, bad;      // T = 0; T negative or NaN
};
__device__ __forceinline__ Scale scale_of(const Model& m, int r) {
  const float t = m.temperature ? m.temperature[r] : 1.f;
  Scale s;
  s.bad = !(t >= 0.f);
  s.first_only = t == 0.f;
  s.slope = 1.4426950408889634 / (t > 0.f ? (double)fminf(fmaxf(t, kLeastTemp), kMostTemp) : 1.0);
  s.far = -1000.0 / s.slope;
  return s;
}
__device__ __forceinline__ double mass_of(float l, float max, double far, double slope) {
  return exp2_of(fmax((double)l - (double)max, far), slope);
}

// What a row is known by once its chunks are joined.
struct RowMass {
  double slope, far, inv;    // 1 / mass against the maximum
  u64 cut;
  float max, l_cut;
  int v_cut;
  bool bad;
  __device__ __forceinline__ bool keeps(float l, int v) const { return l > l_cut || (l == l_cut && v <= v_cut); }
  __device__ __forceinline__ double mass(float l, int v) const {      // the probability
    return keeps(l, v) && l > -INFINITY ? mass_of(l, max, far, slope) * inv : 0.0;
  }
};
// Every lane of a group of 32 calls; all get the result.
__device__ __forceinline__ RowMass join(const DraftParams& p, const Model& m, int r) {
  const int c = lane_id() & 31;
  const Scale sc = scale_of(m, r);
  Rec rec{0.0, 0, -INFINITY, 0};
  if (c < p.chunks) rec = m.recs[(size_t)r * p.chunks + c];
  float mx = rec.max;
  u64 top = rec.top;
  int bad = rec.bad;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    mx = fmaxf(mx, __shfl_xor(mx, o, kWave));
    bad |= __shfl_xor(bad, o, kWave);
    const u64 other = __shfl_xor(top, o, kWave);
    top = other > top ? other : top;
  }
  double mass = rec.max > -INFINITY && rec.mass > 0.0
                    ? rec.mass * mass_of(rec.max, mx, sc.far, sc.slope) : 0.0;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) mass += __shfl_xor(mass, o, kWave);
  RowMass out;
  out.bad = bad || sc.bad || !(mx > -INFINITY);
  out.slope = sc.slope;
  out.far = sc.far;
  out.inv = 1.0 / mass;
  out.max = mx;
  out.cut = m.cuts ? m.cuts[r] : sc.first_only ? top : 0;
  if (sc.first_only) out.inv = 1.0;                // the cut is the maximum's
  out.l_cut = out.cut ? logit_of(out.cut) : -__FLT_MAX__;
  out.v_cut = out.cut ? index_of(out.cut) : p.V;
  return out;
}
template <typename DT> __device__ __forceinline__ float logit(const Model& m, int r, int v) {
  return to_f32(reinterpret_cast<const DT*>(m.logits)[(size_t)r * m.stride + v]);
}
template <typename DT> __device__ __forceinline__ double prob(const DraftParams& p, const Model& m, const RowMass& row, int r, int v) {
  return row.mass(logit<DT>(m, r, v), v);
}

__device__ __forceinline__ double wave_sum_d(double v) {
#pragma unroll
  for (int o = 1; o < kWave; o <<= 1) v += __shfl_xor(v, o, kWave);
  return v;
}
__device__ __forceinline__ double block_sum(double v, double* part) {
  v = wave_sum_d(v);
  __syncthreads();
  if (lane_id() == 0) part[threadIdx.x / kWave] = v;
  __syncthreads();
  v = 0.0;
#pragma unroll
  for (int i = 0; i < kWaves; ++i) v += part[i];
  return v;
}

// A chunk's entries in registers as they came: entry i of the thread is
// (i / N) * kThreads N + tid N + i % N.
typedef __attribute__((__vector_size__(16))) int i32x4;
template <typename DT, bool VEC> struct Entries {
  static constexpr int N = VEC ? 16 / (int)sizeof(DT) : 1;
  typedef std::conditional_t<VEC, i32x4, DT> Raw;
  struct Lane { DT e[N]; };
  Raw raw[kPer / N];
  __device__ __forceinline__ static int at(int i) { return (i / N * kThreads + (int)threadIdx.x) * N + i % N; }
  __device__ __forceinline__ void load(const Model& m, int r, int v0, int V) {
    const DT* src = reinterpret_cast<const DT*>(m.logits) + (size_t)r * m.stride + v0;
    const int n = V - v0;
#pragma unroll
    for (int i = 0; i < kPer / N; ++i) {
      const int to = at(i * N);
      if (to < n) {                                // with VEC, V is a multiple of N
        raw[i] = *reinterpret_cast<const Raw*>(src + to);
      } else {
        Lane e;
#pragma unroll
        for (int c = 0; c < N; ++c) e.e[c] = from_f32<DT>(-INFINITY);
        raw[i] = __builtin_bit_cast(Raw, e);
      }
    }
  }
  __device__ __forceinline__ float get(int i) const { return to_f32(__builtin_bit_cast(Lane, raw[i / N]).e[i % N]); }
};

template <typename DT, bool VEC, bool CUT>
__global__ __launch_bounds__(kThreads) void draft_stats_kernel(DraftParams p, Model m) {
  __shared__ float s_max[kWaves];
  __shared__ double s_part[kWaves];
  __shared__ u64 s_top[kWaves];
  __shared__ int s_bad;
  const int r = blockIdx.x / p.chunks, c = blockIdx.x - r * p.chunks, v0 = c * kChunk, tid = threadIdx.x;
  Entries<DT, VEC> x;
  x.load(m, r, v0, p.V);
  const Scale sc = scale_of(m, r);
  if (tid == 0) s_bad = 0;
  float mx = -INFINITY;
  bool bad = false;
#pragma unroll
  for (int i = 0; i < kPer; i += 2) {
    mx = fmaxf(mx, fmaxf(x.get(i), x.get(i + 1)));
    bad |= __builtin_isunordered(x.get(i), x.get(i + 1));
  }
  mx = wave_max(mx);
  if (lane_id() == 0) s_max[tid / kWave] = mx;
  __syncthreads();
  if (bad) s_bad = 1;
#pragma unroll
  for (int i = 0; i < kWaves; ++i) mx = fmaxf(mx, s_max[i]);
  if (mx == INFINITY) s_bad = 1;
  u64 top = 0;
  double sum = 0.0;
  if (!CUT && sc.first_only) {
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const u64 o = x.get(i) == mx && mx > -INFINITY ? order_of(mx, v0 + Entries<DT, VEC>::at(i)) : 0;
      top = o > top ? o : top;
    }
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) {
      const u64 other = __shfl_xor(top, o, kWave);
      top = other > top ? other : top;
    }
    if (lane_id() == 0) s_top[tid / kWave] = top;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kWaves; ++i) top = s_top[i] > top ? s_top[i] : top;
  } else if (mx > -INFINITY && mx < INFINITY) {
    const u64 cut = CUT ? m.cuts[r] : 0;
    const float l_cut = cut ? logit_of(cut) : -__FLT_MAX__;
    const int v_cut = cut ? index_of(cut) : p.V;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const float l = x.get(i);
      const double e = mass_of(l, mx, sc.far, sc.slope);
      if (CUT) {
        const int v = v0 + Entries<DT, VEC>::at(i);
        sum += l > l_cut || (l == l_cut && v <= v_cut) ? e : 0.0;
      } else {
        sum += e;                                  // of -inf: 2^-1000
      }
    }
  }
  sum = block_sum(sum, s_part);
  if (tid == 0) m.recs[(size_t)r * p.chunks + c] = {sum, top, mx, s_bad};
}

// How a window ends.
enum { kGoesOn = 0, kRejected = 1, kNoDraft = 2, kBad = 3, kEos = 4 };

// The first row of sequence b that ends it, by all threads of the workgroup: in s_end, row * 8 +
// how (INT_MAX: none).  `write`: the rows' p_accept too.
template <typename DT>
__device__ __forceinline__ void find_end(const DraftParams& p, int b, int r0, int k, bool write, int* s_end) {
  if (threadIdx.x == 0) *s_end = 0x7fffffff;
  __syncthreads();
  for (int i0 = 0; i0 < k; i0 += kThreads / 32) {
    const int i = i0 + (int)threadIdx.x / 32, r = r0 + min(i, k - 1);
    const int x = p.prop_tok[r];
    const RowMass t = join(p, p.target, r);
    RowMass d{};
    if (p.draft.logits) d = join(p, p.draft, r);
    if (i < k && (threadIdx.x & 31) == 0) {
      int how = kGoesOn;
      float ratio = 0.f;
      if (t.bad || (x >= 0 && d.bad)) {
        how = kBad;
        ratio = __uint_as_float(0x7fc00000u);
      } else if (x < 0) {
        how = kNoDraft;
      } else {
        double pt = 0.0, pd = p.draft.logits ? 0.0 : 1.0;
        if (x < p.V) {
          pt = prob<DT>(p, p.target, t, r, x);
          if (p.draft.logits) pd = prob<DT>(p, p.draft, d, r, x);
        }
        ratio = pt >= pd ? (pt > 0.0 ? 1.f : 0.f) : (float)(pt / pd);
        how = !((double)p.u_accept[r] * pd < pt) ? kRejected : x == p.eos_id ? kEos : kGoesOn;
      }
      if (write) p.p_accept[r] = ratio;
      if (how != kGoesOn) atomicMin(s_end, 8 * min(i, 0xfffffff) + how);
    }
  }
  __syncthreads();
}

struct Window {
  int r0, k;
};
__device__ __forceinline__ Window window_of(const DraftParams& p, int b) {
  Window w;
  w.r0 = min(max(p.cu_q[b], 0), p.T);
  w.k = min(max(p.cu_q[b + 1] - w.r0, 0), p.T - w.r0);
  return w;
}

// An entry's mass in what a rejected row is drawn from.
__device__ __forceinline__ double rest_of(const RowMass& t, float lt, const RowMass& d, float ld, bool certain, int x, int v) {
  const double m = t.mass(lt, v);
  if (certain) return v == x ? 0.0 : m;
  return fmax(m - d.mass(ld, v), 0.0);
}

template <typename DT, bool VEC>
__global__ __launch_bounds__(kThreads) void draft_rest_kernel(DraftParams p) {
  __shared__ int s_end;
  __shared__ double s_part[kWaves];
  const int b = blockIdx.x / p.chunks, c = blockIdx.x - b * p.chunks;
  const Window w = window_of(p, b);
  find_end<DT>(p, b, w.r0, w.k, c == 0, &s_end);
  const int end = s_end;
  if (c == 0 && threadIdx.x == 0) p.verdict[b] = end;
  if (end == 0x7fffffff || (end & 7) != kRejected) return;
  const int r = w.r0 + (end >> 3), x = p.prop_tok[r], v0 = c * kChunk;
  const bool certain = !p.draft.logits;
  const RowMass t = join(p, p.target, r);
  RowMass d{};
  if (!certain) d = join(p, p.draft, r);
  Entries<DT, VEC> lt, ld;
  lt.load(p.target, r, v0, p.V);
  if (!certain) ld.load(p.draft, r, v0, p.V);
  double sum = 0.0;
#pragma unroll
  for (int i = 0; i < kPer; ++i)
    sum += rest_of(t, lt.get(i), d, certain ? 0.f : ld.get(i), certain, x, v0 + Entries<DT, VEC>::at(i));
  sum = block_sum(sum, s_part);
  if (threadIdx.x == 0) p.rest[(size_t)b * p.chunks + c] = sum;
}

template <typename DT, bool VEC>
__global__ __launch_bounds__(kThreads) void draft_draw_kernel(DraftParams p) {
  __shared__ double s_part[kWaves], s_goal;
  __shared__ int s_chunk, s_hit[2];
  __shared__ double s_before;
  const int b = blockIdx.x, tid = threadIdx.x, lane = lane_id(), wv = tid / kWave;
  const Window w = window_of(p, b);
  const int end = p.verdict[b], how = end == 0x7fffffff ? kGoesOn : end & 7;
  const int n = how == kGoesOn ? w.k : (end >> 3) + (how == kEos ? 1 : 0);
  if (how != kRejected && how != kNoDraft) {
    if (tid == 0) {
      p.n_acc[b] = n;
      p.token[b] = -1;
      p.finished[b] = how == kEos;
      if (p.logp) p.logp[b] = __uint_as_float(0x7fc00000u);
    }
    return;
  }
  const int r = w.r0 + n, x = p.prop_tok[r];
  const RowMass t = join(p, p.target, r);
  const bool certain = !p.draft.logits;
  RowMass d{};
  if (!certain && how == kRejected) d = join(p, p.draft, r);
  // masses of the chunks; a rest of nothing (rounding, a u of 1) leaves p itself
  bool rest = how == kRejected;
  const int c = lane & 31;
  double mine = rest && c < p.chunks ? p.rest[(size_t)b * p.chunks + c] : 0.0;
  double all = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) all += __shfl_xor(all, o, kWave);
  if (!(all > 0.0)) {
    rest = false;
    mine = 0.0;
    if (c < p.chunks) {
      const Rec rec = p.target.recs[(size_t)r * p.chunks + c];
      if (t.cut && !p.target.cuts)                 // temperature 0
        mine = index_of(t.cut) / kChunk == c ? 1.0 : 0.0;
      else if (rec.max > -INFINITY && rec.mass > 0.0)
        mine = rec.mass * mass_of(rec.max, t.max, t.far, t.slope) * t.inv;
    }
  }
  if (wv == 0) {
    double incl = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const double up = __shfl_up(incl, o, 32);
      if (c >= o) incl += up;
    }
    const double goal = (double)p.u_draw[b] * __shfl(incl, 31, 32);
    const unsigned some = (unsigned)__ballot(mine > 0.0);
    unsigned hit = (unsigned)__ballot(mine > 0.0 && incl > goal);
    if (hit == 0) hit = 1u << (31 - __clz((int)(some | 1u)));
    const int pick = __ffs((int)hit) - 1;
    if (lane == pick) {
      s_chunk = pick;
      s_goal = goal - (incl - mine);
      s_hit[0] = kThreads;
      s_hit[1] = 0;
    }
  }
  __syncthreads();
  // threads take neighbouring entries of the chunk
  const int v0 = s_chunk * kChunk + tid * kPer;
  const double goal = s_goal;
  auto weigh = [&](float lt, float ld, int v) { return rest ? rest_of(t, lt, d, ld, certain, x, v) : t.mass(lt, v); };
  auto at = [&](int v) {
    const float lt = logit<DT>(p.target, r, v);
    return weigh(lt, rest && !certain ? logit<DT>(p.draft, r, v) : 0.f, v);
  };
  double sum = 0.0;
  if (VEC && v0 + kPer <= p.V) {
    constexpr int N = 16 / (int)sizeof(DT);
    struct Lane { DT e[N]; };
    const DT* st = reinterpret_cast<const DT*>(p.target.logits) + (size_t)r * p.target.stride + v0;
    const DT* sd = rest && !certain ? reinterpret_cast<const DT*>(p.draft.logits) + (size_t)r * p.draft.stride + v0 : st;
#pragma unroll
    for (int i = 0; i < kPer; i += N) {
      const Lane et = __builtin_bit_cast(Lane, ld16<i32x4>(st + i)), ed = __builtin_bit_cast(Lane, ld16<i32x4>(sd + i));
#pragma unroll
      for (int k = 0; k < N; ++k) sum += weigh(to_f32(et.e[k]), to_f32(ed.e[k]), v0 + i + k);
    }
  } else {
    for (int i = 0; i < kPer && v0 + i < p.V; ++i) sum += at(v0 + i);
  }
  double incl = sum;
#pragma unroll
  for (int o = 1; o < kWave; o <<= 1) {
    const double up = __shfl_up(incl, o, kWave);
    if (lane >= o) incl += up;
  }
  if (lane == kWave - 1) s_part[wv] = incl;
  __syncthreads();
  double before = 0.0;
#pragma unroll
  for (int i = 0; i < kWaves; ++i) before += i < wv ? s_part[i] : 0.0;
  const double left = __shfl_up(incl, 1, kWave);
  const double lo = lane > 0 ? before + left : before, hi = before + incl;
  const u64 some = __ballot(sum > 0.0), past = __ballot(sum > 0.0 && hi > goal);
  if (lane == 0 && some) atomicMax(&s_hit[1], wv * kWave + 63 - __clzll((long long)some));
  if (lane == 0 && past) atomicMin(&s_hit[0], wv * kWave + __ffsll((long long)past) - 1);
  __syncthreads();
  // the first thread whose end passes the goal; rounding, or a u of 1, leave it to the last that holds some
  const int who = s_hit[0] < kThreads ? s_hit[0] : s_hit[1];
  if (tid == who) s_before = goal - lo;
  __syncthreads();
  if (wv != 0) return;
  static_assert(kPer <= kWave, "a lane per entry");
  const int v = s_chunk * kChunk + who * kPer + lane;
  const double one = lane < kPer && v < p.V ? at(v) : 0.0;
  double upto = one;
#pragma unroll
  for (int o = 1; o < kPer; o <<= 1) {
    const double up = __shfl_up(upto, o, kWave);
    if (lane >= o) upto += up;
  }
  const u64 any = __ballot(one > 0.0);
  u64 hit = __ballot(one > 0.0 && upto > s_before);
  if (hit == 0) hit = 1ull << (63 - __clzll((long long)(any | 1)));
  if (lane == __ffsll((long long)hit) - 1) {
    p.n_acc[b] = n;
    p.token[b] = v;
    p.finished[b] = v == p.eos_id;
    if (p.logp) {
      const float l = logit<DT>(p.target, r, v);
      p.logp[b] = (float)(((double)l - (double)t.max) * t.slope * 0.6931471805599453 + log(t.inv));
    }
  }
}

int chunks_of(int V) { return (V + kChunk - 1) / kChunk; }
size_t align(size_t n) { return (n + 255) / 256 * 256; }

}  // namespace

size_t verify_drafts_workspace(int T, int V, int B, bool target_filters, bool draft_filters) {
  const size_t nc = chunks_of(V);
  size_t n = 2 * align(T * nc * sizeof(Rec)) + align(B * nc * sizeof(double)) + align((size_t)B * sizeof(int));
  n += (target_filters ? align((size_t)T * 8) : 0) + (draft_filters ? align((size_t)T * 8) : 0);
  if (target_filters || draft_filters) n += align(sample_logits_workspace(T, V));
  return n;
}

hipError_t launch_verify_drafts(const DraftLaunch& L, hipStream_t st) {
  const int nc = chunks_of(L.V), size = L.dtype_bf16 ? 2 : 4;
  char* ws = static_cast<char*>(L.workspace);
  auto take = [&](size_t n) {
    char* at = ws;
    ws += align(n);
    return at;
  };
  auto filtered = [](const Filters& f) { return f.top_k || f.top_p || f.min_p; };
  DraftParams p{};
  p.target = {L.target, L.target_stride, L.tf.temperature, nullptr, (Rec*)take((size_t)L.T * nc * sizeof(Rec))};
  p.draft = {L.draft, L.draft_stride, L.df.temperature, nullptr, (Rec*)take((size_t)L.T * nc * sizeof(Rec))};
  p.T = L.T;
  p.V = L.V;
  p.B = L.B;
  p.chunks = nc;
  p.prop_tok = L.prop_tok;
  p.cu_q = L.cu_q;
  p.u_accept = L.u_accept;
  p.u_draw = L.u_draw;
  p.eos_id = L.eos_id;
  p.n_acc = L.n_acc;
  p.token = L.token;
  p.finished = L.finished;
  p.p_accept = L.p_accept;
  p.logp = L.logp;
  p.rest = (double*)take((size_t)L.B * nc * sizeof(double));
  p.verdict = (int*)take((size_t)L.B * sizeof(int));
  trace_begin(st);
  u64* cuts[2] = {nullptr, nullptr};
  const bool on[2] = {filtered(L.tf), L.draft && filtered(L.df)};
  for (int i = 0; i < 2; ++i)
    if (on[i]) cuts[i] = (u64*)take((size_t)L.T * 8);
  for (int i = 0; i < 2; ++i) {
    if (!on[i] || L.T == 0) continue;
    const Filters& f = i ? L.df : L.tf;
    SampleLogitsLaunch S{i ? L.draft : L.target, i ? L.draft_stride : L.target_stride, L.T, L.V, nullptr, f.temperature, f.top_k,
                         f.top_p, f.min_p, nullptr, nullptr, L.dtype_bf16, ws, cuts[i]};
    const hipError_t e = launch_logit_cuts(S, st);
    if (e != hipSuccess) return e;
  }
  p.target.cuts = cuts[0];
  p.draft.cuts = cuts[1];
  auto wide = [&](const void* x, int64_t stride) {
    return ((uintptr_t)x & 15) == 0 && stride * size % 16 == 0 && (size_t)L.V * size % 16 == 0;
  };
  const bool vec = wide(L.target, L.target_stride) && (!L.draft || wide(L.draft, L.draft_stride));
  auto with = [&](auto f) {
    if (L.dtype_bf16) {
      if (vec) f(bf16(), std::true_type()); else f(bf16(), std::false_type());
    } else {
      if (vec) f(float(), std::true_type()); else f(float(), std::false_type());
    }
  };
  with([&](auto dt, auto v) {
    using DT = decltype(dt);
    constexpr bool VEC = decltype(v)::value;
    for (int i = 0; i < (L.draft ? 2 : 1) && L.T > 0; ++i) {
      const Model& m = i ? p.draft : p.target;
      if (m.cuts)
        hipLaunchKernelGGL((draft_stats_kernel<DT, VEC, true>), dim3(L.T * nc), dim3(kThreads), 0, st, p, m);
      else
        hipLaunchKernelGGL((draft_stats_kernel<DT, VEC, false>), dim3(L.T * nc), dim3(kThreads), 0, st, p, m);
    }
  });
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  trace_mark(st);
  with([&](auto dt, auto v) {
    hipLaunchKernelGGL((draft_rest_kernel<decltype(dt), decltype(v)::value>), dim3(L.B * nc), dim3(kThreads), 0, st, p);
  });
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  trace_mark(st);
  with([&](auto dt, auto v) {
    hipLaunchKernelGGL((draft_draw_kernel<decltype(dt), decltype(v)::value>), dim3(L.B), dim3(kThreads), 0, st, p);
  });
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  trace_mark(st);
  return hipSuccess;
}

}  // namespace ipdv
