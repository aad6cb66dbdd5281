// The verdict on drafted tokens by the two models' probabilities, for gfx950.  With p and q
// the target's and the draft's (filtered) distributions at a row, x its drafted token:
//
//   accepted while u q(x) < p(x);  at the first row that is not, the token is drawn from
//   max(0, p - q) / sum max(0, p - q), and at a row without a draft from p
//
// so that whatever is emitted is distributed as p.
//
//   stats kernel    one workgroup per row, model and 8192 entries: maximum and mass against
//                   it, by quarters too.  Reads every logit once; its vector instructions
//                   (20 an entry, 8 of them in 64 bits; busy for all of its time) take longer
//                   than its bytes: 512 rows of 151936 bf16 logits of two models 97 us.
//   rest kernel     one workgroup per sequence and 8192 entries: the rows' masses joined, p(x) and
//                   q(x), the first row that ends the window, by each anew (a kernel of its own
//                   took 6 us, and 2.5 of the host's); of a rejected row the masses of max(0, p - q),
//                   by quarters.
//   draw kernel     one workgroup per sequence: the quarter where the mass passes u, in it
//                   the entry.
//
// Precision.  A token is a whole number next to borders that lie as close as the
// smallest probabilities, and a rejected row's masses are differences: all masses are
// 64-bit floats.  2^y is 2^(n + i / 256) from a table in LDS, n added to its exponent, times a
// polynomial of degree 2 of what is left of y, off by 1.1e-10.  (A polynomial of degree 7 alone took
// 5 instructions more, 117 us.)
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
constexpr int kQuarter = kChunk / kWaves;
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
  double* quarters;  // [T][chunks][4]: the record's mass by quarters
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
  double* rest;              // [B][chunks][4]: masses of max(0, p - q)
  int* verdict;              // [B]: 8 * the row that ends the window + how (kNone: none)
};
constexpr int kNone = 0x7fffffff;

// 2^(i / 256), from LDS where a kernel needs many; what i adds to the exponent's sum below is
// taken from the upper words.
constexpr int kPowers = 256;
struct Powers {
  double v[kPowers];
  constexpr Powers() : v() {
    for (int i = 0; i < kPowers; ++i) {
      const double x = 0.69314718055994530942 * i / kPowers;
      double sum = 0.0;
      for (int n = 24; n > 0; --n) sum = (1.0 + sum) * x / n;        // e^x - 1, from the last term
      v[i] = __builtin_bit_cast(double, __builtin_bit_cast(u64, 1.0 + sum) - ((u64)i << 44));
    }
  }
};
__device__ constexpr Powers kPow;
__device__ __forceinline__ void powers_to(double (&lds)[kPowers]) {
  static_assert(kPowers == kThreads, "one of a thread");
  lds[threadIdx.x] = kPow.v[threadIdx.x];
}

// a b + c with c in scalar registers: the compiler would take the form that adds to its operand and
// copy every coefficient for it, two instructions each.
__device__ __forceinline__ double fma_s(double a, double b, double c) {
  double r;
  asm("v_fma_f64 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "s"(c));
  return r;
}
// A mass in two factors, so that a sum takes it in one instruction.
struct Product {
  double base, by;
  __device__ __forceinline__ operator double() const { return base * by; }
  __device__ __forceinline__ void add_to(double& sum) const { sum = fma(base, by, sum); }
};
// 2^(d slope) for d slope <= 0 (and not below -1001): d slope = n + i / 256 + f, |f| <= 2^-9.
__device__ __forceinline__ Product exp2_of(double d, double slope, const double* pow) {
  const double magic = 26388279066624.0;           // 1.5 * 2^44: the sum's low bits count 256ths
  const double t = fma(d, slope, magic), f = fma(d, slope, magic - t);
  const unsigned at = (unsigned)__double2loint(t);
  const double base = pow[at & (kPowers - 1)];
  // 2^f = 1 + ln 2 f + (ln 2 f)^2 / 2, the cubic term levelled: off by 1.1e-10
  const double by = fma(fma_s(f, 0.2402265069591007, 0.6931473393594654), f, 1.0);
  return {__hiloint2double((int)((unsigned)__double2hiint(base) + (at << 12)), __double2loint(base)), by};
}

// A row's temperature: log2(e) / T, and the distance from the maximum behind which an entry has no
// probability (2^-1000 of the maximum's; sums take it for that, since they cannot tell).  T from 2^100
// on acts as that, where an entry of -inf still counts for nothing.
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
  const double at = t > 0.f ? (double)fminf(fmaxf(t, kLeastTemp), kMostTemp) : 1.0;
  s.slope = 1.4426950408889634 / at;
  s.far = -693.14718055994531 * at;
  return s;
}
__device__ __forceinline__ Product mass_of(float l, float max, double far, double slope, const double* pow) {
  // the larger of two that are not positive, to the 20 bits of their upper words
  const double d = (double)l - (double)max;
  const unsigned hi = min((unsigned)__double2hiint(d), (unsigned)__double2hiint(far));
  return exp2_of(__hiloint2double((int)hi, __double2loint(d)), slope, pow);
}

// What a row is known by once its chunks are joined.
struct RowMass {
  double slope, far, inv;    // 1 / mass against the maximum
  u64 cut;
  float max, l_cut;          // what the filters keep, and what has a probability at all
  int v_cut;
  bool bad;
  __device__ __forceinline__ bool keeps(float l, int v) const { return (l > l_cut) | ((l == l_cut) & (v <= v_cut)); }
  __device__ __forceinline__ double mass(float l, int v, const double* pow) const {      // the probability
    const double m = mass_of(l, max, far, slope, pow) * inv;
    return keeps(l, v) ? m : 0.0;
  }
};
template <int CTRL> __device__ __forceinline__ double dpp_move_d(double v) {
  return __hiloint2double(dpp_move_i<CTRL>(__double2hiint(v)), dpp_move_i<CTRL>(__double2loint(v)));
}
// Sum over 32 neighbouring lanes, in all of them.
__device__ __forceinline__ double sum32(double v) {
  v += dpp_move_d<0x140>(v);
  v += dpp_move_d<0x141>(v);
  v += dpp_move_d<0x4E>(v);
  v += dpp_move_d<0xB1>(v);
  return v + __hiloint2double(__float_as_int(lane_xor16(__int_as_float(__double2hiint(v)))),
                              __float_as_int(lane_xor16(__int_as_float(__double2loint(v)))));
}
// Every lane of a group of 32 calls; all get the result.
__device__ __forceinline__ RowMass join(const DraftParams& p, const Model& m, int r) {
  const int c = lane_id() & 31;
  const Scale sc = scale_of(m, r);
  Rec rec{0.0, 0, -INFINITY, 0};
  if (c < p.chunks) rec = m.recs[(size_t)r * p.chunks + c];
  const u64 given = m.cuts ? m.cuts[r] : 0;
  float mx = rec.max;
  mx = fmaxf(mx, dpp_move<0x140>(mx));
  mx = fmaxf(mx, dpp_move<0x141>(mx));
  mx = fmaxf(mx, dpp_move<0x4E>(mx));
  mx = fmaxf(mx, dpp_move<0xB1>(mx));
  mx = fmaxf(mx, lane_xor16(mx));
  const bool bad = (unsigned)(__ballot(rec.bad) >> (lane_id() & 32)) != 0;
  u64 top = rec.top;
  if (__any(sc.first_only && !m.cuts)) {
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const u64 other = __shfl_xor(top, o, kWave);
      top = other > top ? other : top;
    }
  }
  const double mass = sum32(rec.max > -INFINITY && rec.mass > 0.0 ? rec.mass * mass_of(rec.max, mx, sc.far, sc.slope, kPow.v) : 0.0);
  RowMass out;
  out.bad = bad || sc.bad || !(mx > -INFINITY);
  out.slope = sc.slope;
  out.far = sc.far;
  out.inv = sc.first_only ? 1.0 : 1.0 / mass;      // the cut is the maximum's
  out.max = mx;
  out.cut = m.cuts ? given : sc.first_only ? top : 0;
  out.l_cut = out.cut ? logit_of(out.cut) : -__FLT_MAX__;
  out.v_cut = out.cut ? index_of(out.cut) : p.V;
  // a vocabulary masked by a finite fill: a u of 0 must not draw from it
  const float l_far = (float)((double)mx + sc.far);
  if (l_far > out.l_cut) {
    out.l_cut = l_far;
    out.v_cut = p.V;
  }
  return out;
}
template <typename DT> __device__ __forceinline__ float logit(const Model& m, int r, int v) {
  return to_f32(reinterpret_cast<const DT*>(m.logits)[(size_t)r * m.stride + v]);
}
__device__ __forceinline__ double wave_sum_d(double v) {
  v = sum32(v);
  return v + __hiloint2double(lane_xor32(__double2hiint(v)), lane_xor32(__double2loint(v)));
}

// A chunk's entries in registers as they came, a quarter to each wave.
typedef __attribute__((__vector_size__(16))) int i32x4;
template <typename DT, bool VEC> struct Entries {
  static constexpr int N = VEC ? 16 / (int)sizeof(DT) : 1;
  typedef std::conditional_t<VEC, i32x4, DT> Raw;
  struct Lane { DT e[N]; };
  Raw raw[kPer / N];
  __device__ __forceinline__ static int at(int i) {
    return (int)threadIdx.x / kWave * kQuarter + (i / N * kWave + lane_id()) * N + i % N;
  }
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
__global__ __launch_bounds__(kThreads) void draft_stats_kernel(DraftParams p) {
  __shared__ float s_max[kWaves];
  __shared__ double s_part[kWaves];
  __shared__ u64 s_top[kWaves];
  __shared__ int s_bad;
  __shared__ __attribute__((aligned(16))) double s_pow[kPowers];
  const Model& m = blockIdx.y ? p.draft : p.target;
  const int r = blockIdx.x / p.chunks, c = blockIdx.x - r * p.chunks, v0 = c * kChunk, tid = threadIdx.x;
  Entries<DT, VEC> x;
  x.load(m, r, v0, p.V);
  const Scale sc = scale_of(m, r);
  powers_to(s_pow);
  if (tid == 0) s_bad = 0;
  float mx = -INFINITY;
#pragma unroll
  for (int i = 0; i < kPer; i += 2)                // NaN if there is one: v_maximum3_f32
    mx = __builtin_elementwise_maximum(mx, __builtin_elementwise_maximum(x.get(i), x.get(i + 1)));
  const bool bad = mx != mx;
  mx = wave_max(bad ? INFINITY : mx);
  if (lane_id() == 0) s_max[tid / kWave] = mx;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kWaves; ++i) mx = fmaxf(mx, s_max[i]);
  if (mx == INFINITY) s_bad = 1;
  u64 top = 0;
  double sum = 0.0;
  if (sc.first_only && !(CUT && m.cuts)) {
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
    const u64 cut = CUT && m.cuts ? m.cuts[r] : 0;
    const float l_cut = cut ? logit_of(cut) : -__FLT_MAX__;
    const int v_cut = cut ? index_of(cut) : p.V;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const float l = x.get(i);
      if (!CUT) {
        mass_of(l, mx, sc.far, sc.slope, s_pow).add_to(sum);   // of -inf: 2^-1000
      } else if ((l > l_cut) | ((l == l_cut) & (v0 + Entries<DT, VEC>::at(i) <= v_cut))) {      // few: a branch
        mass_of(l, mx, sc.far, sc.slope, s_pow).add_to(sum);
      }
    }
  }
  sum = wave_sum_d(sum);
  const size_t at = (size_t)r * p.chunks + c;
  if (lane_id() == 0) {
    s_part[tid / kWave] = sum;
    m.quarters[at * kWaves + tid / kWave] = sum;
  }
  __syncthreads();
  if (tid == 0) m.recs[at] = {(s_part[0] + s_part[1]) + (s_part[2] + s_part[3]), top, mx, s_bad};
}

// Sums of less come from entries of no probability, which are never drawn.
constexpr double kNothing = 0x1p-900;

// How a window ends.
enum { kGoesOn = 0, kRejected = 1, kNoDraft = 2, kBad = 3, kEos = 4 };

struct Window {
  int r0, k;
};
__device__ __forceinline__ Window window_of(const DraftParams& p, int b) {
  Window w;
  w.r0 = min(max(p.cu_q[b], 0), p.T);
  w.k = min(max(p.cu_q[b + 1] - w.r0, 0), p.T - w.r0);
  return w;
}

// How window b ends, for the whole workgroup: its rows, eight at a time, 32 lanes each.  `tell`:
// what is known of it now goes to the outputs.
template <typename DT> __device__ __forceinline__ int verdict_of(const DraftParams& p, int b, bool tell) {
  __shared__ int s_end;
  if (threadIdx.x == 0) s_end = kNone;
  __syncthreads();
  const Window w = window_of(p, b);
  for (int i0 = 0; i0 < w.k; i0 += kThreads / 32) {
    const int i = i0 + (int)threadIdx.x / 32, r = w.r0 + min(i, w.k - 1);
    const int x = p.prop_tok[r];
    const float u = p.u_accept[r];
    const bool drafted = x >= 0 && x < p.V, given = p.draft.logits != nullptr;
    // asked for before the records are joined
    const float lt = drafted ? logit<DT>(p.target, r, x) : 0.f, ld = drafted && given ? logit<DT>(p.draft, r, x) : 0.f;
    const RowMass t = join(p, p.target, r);
    RowMass d{};
    if (given) d = join(p, p.draft, r);
    if (i < w.k && (threadIdx.x & 31) == 0) {
      int how = kGoesOn;
      float ratio = 0.f;
      if (t.bad || (x >= 0 && d.bad)) {
        how = kBad;
        ratio = __uint_as_float(0x7fc00000u);
      } else if (x < 0) {
        how = kNoDraft;
      } else {
        const double pt = drafted ? t.mass(lt, x, kPow.v) : 0.0, pd = !given ? 1.0 : drafted ? d.mass(ld, x, kPow.v) : 0.0;
        ratio = pt >= pd ? (pt > 0.0 ? 1.f : 0.f) : (float)(pt / pd);
        how = !((double)u * pd < pt) ? kRejected : x == p.eos_id ? kEos : kGoesOn;
      }
      if (tell) p.p_accept[r] = ratio;
      if (how != kGoesOn) atomicMin(&s_end, 8 * i + how);
    }
  }
  __syncthreads();
  const int end = s_end, how = end == kNone ? kGoesOn : end & 7;
  if (tell && threadIdx.x == 0) {
    p.verdict[b] = end;
    if (how != kRejected && how != kNoDraft) {               // else the draw kernel's
      p.n_acc[b] = how == kGoesOn ? w.k : (end >> 3) + (how == kEos ? 1 : 0);
      p.token[b] = -1;
      p.finished[b] = how == kEos;
      if (p.logp) p.logp[b] = __uint_as_float(0x7fc00000u);
    }
  }
  return end;
}

// An entry's mass in what a rejected row is drawn from.
__device__ __forceinline__ double rest_of(const RowMass& t, float lt, const RowMass& d, float ld, bool certain, int x, int v, const double* pow) {
  // both probabilities rounded alike: of equal ones nothing is left
#pragma clang fp contract(off)
  if (!t.keeps(lt, v) || (certain && v == x)) return 0.0;      // filters leave few: a branch
  const double m = t.mass(lt, v, pow);
  return certain ? m : fmax(m - d.mass(ld, v, pow), 0.0);
}

template <typename DT, bool VEC>
__global__ __launch_bounds__(kThreads) void draft_rest_kernel(DraftParams p) {
  const int b = blockIdx.x / p.chunks, c = blockIdx.x - b * p.chunks;
  const int end = verdict_of<DT>(p, b, c == 0);
  if (end == kNone || (end & 7) != kRejected) return;
  const int r = window_of(p, b).r0 + (end >> 3), v0 = c * kChunk;
  const bool certain = !p.draft.logits;
  __shared__ __attribute__((aligned(16))) double s_pow[kPowers];
  Entries<DT, VEC> lt, ld;
  lt.load(p.target, r, v0, p.V);
  if (!certain) ld.load(p.draft, r, v0, p.V);
  const int x = p.prop_tok[r];
  const RowMass t = join(p, p.target, r);
  RowMass d{};
  if (!certain) d = join(p, p.draft, r);
  powers_to(s_pow);
  __syncthreads();
  double sum = 0.0;
  if (t.cut | d.cut | (u64)certain) {
#pragma unroll
    for (int i = 0; i < kPer; ++i)
      sum += rest_of(t, lt.get(i), d, certain ? 0.f : ld.get(i), certain, x, v0 + Entries<DT, VEC>::at(i), s_pow);
  } else {                                         // everything is kept, -inf of 2^-1000
    // both probabilities rounded alike: of equal ones nothing is left
#pragma clang fp contract(off)
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const double m = mass_of(lt.get(i), t.max, t.far, t.slope, s_pow) * t.inv, q = mass_of(ld.get(i), d.max, d.far, d.slope, s_pow) * d.inv;
      sum += fmax(m - q, 0.0);
    }
  }
  sum = wave_sum_d(sum);
  if (lane_id() == 0) p.rest[((size_t)b * p.chunks + c) * kWaves + threadIdx.x / kWave] = sum;
}

// Inclusive sums over the lanes of a wave, in lane order.
__device__ __forceinline__ double wave_scan_d(double v) {
#pragma unroll
  for (int o = 1; o < kWave; o <<= 1) {
    const double up = __shfl_up(v, o, kWave);
    if (lane_id() >= o) v += up;
  }
  return v;
}

template <typename DT, bool VEC>
__global__ __launch_bounds__(kThreads) void draft_draw_kernel(DraftParams p) {
  constexpr int PER = kQuarter / kThreads;         // neighbouring entries of a thread
  constexpr int QN = kMaxChunks * kWaves / kWave;  // quarters of a lane
  __shared__ double s_part[kWaves], s_goal;
  __shared__ int s_quarter, s_hit[2];
  const int b = blockIdx.x, tid = threadIdx.x, lane = lane_id(), wv = tid / kWave;
  const int end = p.verdict[b], how = end == kNone ? kGoesOn : end & 7;
  if (how != kRejected && how != kNoDraft) return;
  const int n = end >> 3, r = window_of(p, b).r0 + n, quarters = p.chunks * kWaves;
  const int x = p.prop_tok[r];
  const float u = p.u_draw[b];
  const bool certain = !p.draft.logits;
  // masses of the quarters, a lane QN neighbours: of the rest, or (a rest of nothing: rounding, a u
  // of 1) of p itself
  double mine[QN], whole[QN];
#pragma unroll
  for (int i = 0; i < QN; ++i) {
    const int q = lane * QN + i;
    mine[i] = how == kRejected && q < quarters ? p.rest[(size_t)b * quarters + q] : 0.0;
    whole[i] = q < quarters ? p.target.quarters[(size_t)r * quarters + q] : 0.0;
  }
  const float chunk_max = lane * QN / kWaves < p.chunks ? p.target.recs[(size_t)r * p.chunks + lane * QN / kWaves].max : -INFINITY;
  static_assert(kWaves % QN == 0, "a lane's quarters lie in one chunk");
  const RowMass t = join(p, p.target, r);
  RowMass d{};
  if (!certain && how == kRejected) d = join(p, p.draft, r);
  double all = 0.0;
#pragma unroll
  for (int i = 0; i < QN; ++i) all += mine[i];
  const bool rest = how == kRejected && wave_sum_d(all) > kNothing;
  if (!rest) {
    const double f = chunk_max > -INFINITY ? mass_of(chunk_max, t.max, t.far, t.slope, kPow.v) * t.inv : 0.0;
#pragma unroll
    for (int i = 0; i < QN; ++i)
      mine[i] = t.cut && !p.target.cuts ? (index_of(t.cut) / kQuarter == lane * QN + i ? 1.0 : 0.0)      // temperature 0
                                        : whole[i] * f;
  }
  if (wv == 0) {
    double part = 0.0;
#pragma unroll
    for (int i = 0; i < QN; ++i) part += mine[i];
    const double upto = wave_scan_d(part);
    const double goal = (double)u * __shfl(upto, kWave - 1, kWave);
    const u64 some = __ballot(part > kNothing);
    u64 hit = __ballot(part > kNothing && upto > goal);
    if (hit == 0) hit = 1ull << (63 - __clzll((long long)(some | 1)));
    if (lane == __ffsll((long long)hit) - 1) {     // its first quarter whose end passes the goal, or its last that holds some
      double before = upto - part;
      int pick = 0;
      bool found = false;
      double at = before;
#pragma unroll
      for (int i = 0; i < QN; ++i) {
        if (!found && mine[i] > kNothing) {
          pick = i;
          at = before;
          found = before + mine[i] > goal;
        }
        before += mine[i];
      }
      s_quarter = lane * QN + pick;
      s_goal = goal - at;
      s_hit[0] = kThreads;
      s_hit[1] = 0;
    }
  }
  __syncthreads();
  const int v0 = s_quarter * kQuarter + tid * PER;
  const double goal = s_goal;
  const bool both = rest && !certain;
  float lt[PER], ld[PER];
  if (VEC && v0 + PER <= p.V) {
    constexpr int N = 16 / (int)sizeof(DT);
    struct Lane { DT e[N]; };
    const DT* st = reinterpret_cast<const DT*>(p.target.logits) + (size_t)r * p.target.stride + v0;
    const DT* sd = both ? reinterpret_cast<const DT*>(p.draft.logits) + (size_t)r * p.draft.stride + v0 : st;
#pragma unroll
    for (int i = 0; i < PER; i += N) {
      const Lane et = __builtin_bit_cast(Lane, ld16<i32x4>(st + i)), ed = __builtin_bit_cast(Lane, ld16<i32x4>(sd + i));
#pragma unroll
      for (int k = 0; k < N; ++k) {
        lt[i + k] = to_f32(et.e[k]);
        ld[i + k] = to_f32(ed.e[k]);
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      lt[i] = v0 + i < p.V ? logit<DT>(p.target, r, v0 + i) : -INFINITY;
      ld[i] = both && v0 + i < p.V ? logit<DT>(p.draft, r, v0 + i) : -INFINITY;
    }
  }
  double m[PER], sum = 0.0;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    m[i] = rest ? rest_of(t, lt[i], d, ld[i], certain, x, v0 + i, kPow.v) : t.mass(lt[i], v0 + i, kPow.v);
    sum += m[i];
  }
  const double incl = wave_scan_d(sum);
  if (lane == kWave - 1) s_part[wv] = incl;
  __syncthreads();
  double before = 0.0;
#pragma unroll
  for (int i = 0; i < kWaves; ++i) before += i < wv ? s_part[i] : 0.0;
  // a thread's end is the next one's beginning, to the last bit
  const double left = __shfl_up(incl, 1, kWave);
  double at = lane > 0 ? before + left : before;
  const double to = before + incl;
  const u64 some = __ballot(sum > 0.0), past = __ballot(sum > 0.0 && to > goal);
  if (lane == 0 && some) atomicMax(&s_hit[1], wv * kWave + 63 - __clzll((long long)some));
  if (lane == 0 && past) atomicMin(&s_hit[0], wv * kWave + __ffsll((long long)past) - 1);
  __syncthreads();
  // the first thread whose end passes the goal; rounding, or a u of 1, leave it to the last that
  // holds some; in it the first entry likewise
  if (tid != (s_hit[0] < kThreads ? s_hit[0] : s_hit[1])) return;
  int pick = 0;
  float l = lt[0];
  bool found = false;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    if (!found && m[i] > 0.0) {
      pick = i;
      l = lt[i];
      found = at + m[i] > goal;
    }
    at += m[i];
  }
  p.n_acc[b] = n;
  p.token[b] = v0 + pick;
  p.finished[b] = v0 + pick == p.eos_id;
  if (p.logp) p.logp[b] = (float)(((double)l - (double)t.max) * t.slope * 0.6931471805599453 + log(t.inv));
}

int chunks_of(int V) { return (V + kChunk - 1) / kChunk; }
size_t align(size_t n) { return (n + 255) / 256 * 256; }

}  // namespace

size_t verify_drafts_workspace(int T, int V, int B, bool target_filters, bool draft_filters) {
  const size_t nc = chunks_of(V);
  size_t n = 2 * (align(T * nc * sizeof(Rec)) + align(T * nc * kWaves * 8)) + align(B * nc * kWaves * 8) + align((size_t)B * sizeof(int));
  n += (target_filters ? align((size_t)T * 8) : 0) + (draft_filters ? align((size_t)T * 8) : 0);
  n += ((target_filters ? 1 : 0) + (draft_filters ? 1 : 0)) * align(sample_logits_workspace(T, V));
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
  auto model = [&](const void* logits, int64_t stride, const float* temperature) {
    const size_t n = (size_t)L.T * nc;
    Rec* recs = (Rec*)take(n * sizeof(Rec));
    return Model{logits, stride, temperature, nullptr, recs, (double*)take(n * kWaves * 8)};
  };
  p.target = model(L.target, L.target_stride, L.tf.temperature);
  p.draft = model(L.draft, L.draft_stride, L.df.temperature);
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
  p.rest = (double*)take((size_t)L.B * nc * kWaves * 8);
  p.verdict = (int*)take((size_t)L.B * sizeof(int));
  trace_begin(st);
  // the cuts of both models in one go
  u64* cuts[2] = {nullptr, nullptr};
  SampleLogitsLaunch S[2];
  int n = 0;
  for (int i = 0; i < (L.draft ? 2 : 1); ++i) {
    const Filters& f = i ? L.df : L.tf;
    if (!filtered(f)) continue;
    cuts[i] = (u64*)take((size_t)L.T * 8);
    S[n++] = SampleLogitsLaunch{i ? L.draft : L.target, i ? L.draft_stride : L.target_stride, L.T, L.V, nullptr, f.temperature,
                                f.top_k, f.top_p, f.min_p, nullptr, nullptr, L.dtype_bf16,
                                take(sample_logits_workspace(L.T, L.V)), cuts[i]};
  }
  if (n > 0 && L.T > 0) {
    const hipError_t e = launch_logit_cuts(S, n, st);
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
  const dim3 all(L.T * nc, L.draft ? 2 : 1);
  with([&](auto dt, auto v) {
    using DT = decltype(dt);
    constexpr bool VEC = decltype(v)::value;
    if (L.T == 0) return;
    if (n > 0)
      hipLaunchKernelGGL((draft_stats_kernel<DT, VEC, true>), all, dim3(kThreads), 0, st, p);
    else
      hipLaunchKernelGGL((draft_stats_kernel<DT, VEC, false>), all, dim3(kThreads), 0, st, p);
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
