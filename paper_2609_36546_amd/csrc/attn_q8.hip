// Attention over the 8-bit cache for gfx950: causal grouped-query attention of
// every window row over the quantised pages of its sequence (kv_q8.hip has the
// format; the window itself has been appended).
//
//   out[i, h] = sum_j p_j V_j / sum_j p_j,  p_j = 2^(c q.K_j - m),  c = scale log2(e)
//
// in one pass over the keys with a running maximum m and sum per row.
//
// Tiles.  The query rows of one (sequence, KV head), k positions x G heads, are
// packed position-major into tiles of 16.  A wave holds QT tiles and walks
// blocks of 64 keys, four 16-slot units:
//
//   S^T[64 keys x 16 rows] = K . Q^T   A = key rows: v_mfma_scale_f32_16x16x128_f8f6f4 in
//                                      bf16 calls, v_mfma_f32_16x16x32_bf16 in fp32 ones
//   O^T[D x 16 rows] += V^T . P^T      v_mfma_f32_16x16x32_bf16, A = value channels, B = P^T in place
//
// The keys' tile t has MFMA row 4 u + e at unit u, slot 4 t + e.  A lane (row
// c16, group j) then ends up with the scores of exactly the 16 slots of unit j,
// and a value load of 16 bytes, one channel's run of unit j, is its operand of
// two PV steps: P never leaves the lane.  Key channels are dealt to the k-steps
// the same way, 16 bytes of a key row at a time.
//
// Precision.  The bf16 call's scores: a query's channels become two e4m3
// numbers each, the first with the scale of the largest, the second what that
// leaves: 8 bits in all, as bf16 has, down to 2^-14 of the largest, where the first
// goes subnormal; below, 2^-21 of the largest.  (Beside a channel of 10^5 one of 1
// is off by up to 3%, beside one of 10^4 by nothing.)  The keys go into the scaled
// fp8 products as they lie in the cache, with their own scale: nothing is rounded or
// converted on the way.  Values times probabilities: an e4m3 value is exact in bf16,
// its scale goes into the probability.  With one row group a probability is two bf16
// terms (16 bits; the second costs 1%, the call being bound by its bytes), else it
// is rounded to bf16 once, as the bf16 cache's attention does (a second term: windows
// of eight 89 to 100 us, prompts 94 to 112; without it the outputs' error, the half
// step of bf16 included, is 0.0021 to 0.0023 instead of 0.0017).  The fp32 call: keys
// and values exact in bf16 (the key's scale in the conversion), queries and
// probabilities split into three bf16 terms (24 bits).  Sums and the running maximum
// are fp32.
//
// Work split.  All steps (a step: the keys that a workgroup takes at once) of
// all items (an item: one row group of one (sequence, KV head)) form one line,
// cut into as many equal spans as there are workgroups, so that ragged contexts,
// single sequences and long contexts all fill the chip.  Items cut by a span's
// end leave partial results, merged by a second kernel.  Where whole items can be
// dealt out about as evenly (prompts), nothing is cut: the longest first, every
// second round backwards.
//
// A workgroup's four waves are RG row groups of QT tiles x KS = 4 / RG key parts,
// merged in LDS at an item's end; plan_of has the choice.  With one row group
// (attn_q8_keys_kernel) every wave streams keys of its own, straight into
// registers.  With more (attn_q8_rows_kernel) the groups share their keys through
// LDS, filled by direct-to-LDS loads that run a step ahead through the span,
// across its items.  (Through the vector cache instead, 64 windows of eight over
// 1024 to 8192 tokens, 32 heads on 4, took 121 us where LDS took 93 then: a second
// request for a line that is still on its way holds the cache up.)
//
// What bounds it, in bf16 at D = 128: one token each of 64 sequences of 1024 to
// 8192 tokens, 16 heads on 8, the bytes (609 MB in 121 us, the rate of a copy);
// windows of eight, 32 heads on 4, the vector instructions beside the loads, 275 per
// wave and 64 keys (313 MB, at a copy's rate 61 us, in 93, of which the merge takes
// 11); prompts, the vector instructions of softmax, masks and conversion, 560 per 64
// keys and 32 rows beside 48 matrix ones (eight of 512 to 1024 tokens in 94 us, 430
// TFLOP/s; vector pipes issuing 58% of the time, and shares that are not even).
#include <algorithm>
#include <type_traits>

#include "common.h"
#include "kernels.h"
#include "q8.h"

namespace ipdv {
namespace {

constexpr int kBlk = 64;                // keys per block
constexpr float kRescaleSlack = 8.0f;   // log2 units a stale running max may lag

// The item that a span begins in.
struct SpanHead {
  long first;          // where it begins on the line (the last entry: the line's length)
  int steps, slot, g, r;
};

struct Q8Params {
  const void* q;
  long q_stride;
  const uint8_t* k_pages;
  const uint8_t* v_pages;
  const uint8_t* scales;
  const int32_t* page_table;
  const int32_t* ctx_lens;
  const int32_t* cu_q;
  const int32_t* seq_ids;
  void* out;
  struct SpanHead* span;   // [grid + 1]: what every span begins in; the last: the line's length
  float* part_o;       // [2 * grid][item rows][D]
  float* part_ml;      // [2 * grid][item rows][2]: maximum, sum
  int max_pages, Hq, Hkv, G, log2g, log2ps, num_pages, n_seq, max_q, slots;   // log2g: of G, or -1
  float scale_log2;
};

typedef __attribute__((__vector_size__(2 * sizeof(__bf16)))) __bf16 bf16x2;

typedef __attribute__((__vector_size__(8 * sizeof(int)))) int i32x8;

// Eight e4m3 values times 2^e, exact.
__device__ __forceinline__ bf16x8 cvt8(unsigned lo, unsigned hi, float scale) {
  const bf16x2 a = __builtin_bit_cast(bf16x2, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false));
  const bf16x2 b = __builtin_bit_cast(bf16x2, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true));
  const bf16x2 c = __builtin_bit_cast(bf16x2, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false));
  const bf16x2 d = __builtin_bit_cast(bf16x2, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true));
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// Values that do not change while a kernel runs, at addresses all lanes share:
// scalar loads, which do not queue behind the vector loads of keys and values.
typedef const __attribute__((address_space(4))) int32_t* ScalarInts;
__device__ __forceinline__ ScalarInts scalar(const int32_t* p) { return (ScalarInts)(uintptr_t)p; }

// (page, head) of the four units of a block, looked up a block ahead.
struct Units {
  int p0, p1, p2, p3;
  __device__ __forceinline__ void look_up(const Q8Params& a, ScalarInts pt, int t0, int g) {
    auto at = [&](int i) {
      return min(max(pt[min((t0 + 16 * i) >> a.log2ps, a.max_pages - 1)], 0), a.num_pages - 1) * a.Hkv + g;
    };
    p0 = at(0);
    p1 = at(1);
    p2 = at(2);
    p3 = at(3);
  }
  __device__ __forceinline__ unsigned of(int u) const {
    const int q0 = p0, q1 = p1, q2 = p2, q3 = p3;   // by value: a choice between variables would go through memory
    const int lo = u & 1 ? q1 : q0, hi = u & 1 ? q3 : q2;
    return (unsigned)(u & 2 ? hi : lo);
  }
};

// One block of 64 keys in registers.
template <int D> struct Block {
  uint4 k[4][D / 64];   // key tile t: 16 channels of one key per load
  uint4 v[D / 16];      // channel tile: one channel's 16 slots of unit j
  uint4 ks, vs;         // scale bytes: the lane's key unit (c16 / 4), its value unit (j)
  __device__ __forceinline__ uint4 key(int t, int h) const { return k[t][h]; }
  __device__ __forceinline__ uint4 key_scales() const { return ks; }
};

// The same block in LDS: every load of 1 KB as the wave that asked for it has
// its lanes, so that the same lane of any wave reads its 16 bytes back; behind
// them the scale bytes of the four units, keys then values.
template <int D> struct LdsBlock {
  static constexpr int kKeys = 4 * (D / 64), kVals = D / 16, kLoads = kKeys + kVals;
  static constexpr int kBytes = (kLoads + 1) * kWave * 16;
  const char* at;
  __device__ __forceinline__ uint4 get(int i) const {
    return *reinterpret_cast<const uint4*>(at + i * (kWave * 16) + lane_id() * 16);
  }
  __device__ __forceinline__ uint4 scales(int i) const {
    return *reinterpret_cast<const uint4*>(at + kLoads * (kWave * 16) + i * 16);
  }
  __device__ __forceinline__ uint4 key(int t, int h) const { return get(4 * h + t); }
  __device__ __forceinline__ uint4 val(int dt) const { return get(kKeys + dt); }
  __device__ __forceinline__ uint4 key_scales() const { return scales((lane_id() & 15) >> 2); }
  __device__ __forceinline__ uint4 val_scales() const { return scales(4 + (lane_id() >> 4)); }
};
template <int N> __device__ __forceinline__ void wait_loads() { asm volatile("s_waitcnt vmcnt(%0)" : : "n"(N) : "memory"); }
// A barrier for what goes through LDS, which leaves loads under way.
__device__ __forceinline__ void lds_barrier() {
  asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" : : : "memory");
}


template <int D>
__device__ __forceinline__ void load_keys(const Q8Params& a, Block<D>& f, int t0, const Units& units) {
  const int lane = lane_id(), c16 = lane & 15, j = lane >> 4;
  const int ps = 1 << a.log2ps, ks0 = (t0 + 16 * (c16 >> 2)) & (ps - 1);
  const unsigned kh = units.of(c16 >> 2);
  const uint8_t* kb = a.k_pages + ((unsigned long)kh * (unsigned)(D * ps) + (unsigned)((ks0 + (c16 & 3) + j * ps) * 16));
#pragma unroll
  for (int h = 0; h < D / 64; ++h) {
#pragma unroll
    for (int t = 0; t < 4; ++t) f.k[t][h] = ld16<uint4>(kb + 64 * t);
    kb += 64 * ps;
  }
  f.ks = ld16<uint4>(a.scales + ((unsigned long)kh * (unsigned)(2 * ps) + (unsigned)ks0));
}
template <int D>
__device__ __forceinline__ void load_values(const Q8Params& a, Block<D>& f, int t0, const Units& units) {
  const int lane = lane_id(), c16 = lane & 15, j = lane >> 4;
  const int ps = 1 << a.log2ps, vs0 = (t0 + 16 * j) & (ps - 1);
  const unsigned vh = units.of(j);
  const uint8_t* vb = a.v_pages + ((unsigned long)vh * (unsigned)(D * ps) + (unsigned)(vs0 + c16 * ps));
  int tile = 16 * ps;                 // a step that the compiler cannot see through: it would keep the
  asm("" : "+s"(tile));               // multiples in registers that it does not have
#pragma unroll
  for (int dt = 0; dt < D / 16; ++dt) {
    f.v[dt] = ld16<uint4>(vb);
    vb += tile;
  }
  f.vs = ld16<uint4>(a.scales + ((unsigned long)vh * (unsigned)(2 * ps) + (unsigned)(ps + vs0)));
}

__device__ __forceinline__ unsigned word(const uint4& v, int i) {
  return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w;
}

// NS bf16 terms of an fp32 value: each takes 8 bits of what is left.
template <int NS> __device__ __forceinline__ void split(float x, __bf16 (&t)[NS]) {
#pragma unroll
  for (int s = 0; s < NS; ++s) {
    t[s] = static_cast<__bf16>(x);
    if (s + 1 < NS) x -= static_cast<float>(t[s]);
  }
}

// The lane's queries: fp32 ones in NS = 3 bf16 terms, bf16 ones in two e4m3
// terms, 32 channels (D = 64: 16, and 16 zeros), with the row's scale bytes.
template <int D, int QT, int NS> struct Queries { bf16x8 q[NS][QT][D / 32]; };
template <int D, int QT> struct Queries<D, QT, 1> {
  i32x8 hi[QT], lo[QT];
  int e_hi[QT], e_lo[QT];
};
// 16 values of a lane from channel tile h: D / 64 such tiles make up its share.
template <int D, int QT>
__device__ __forceinline__ void split_e4m3(Queries<D, QT, 1>& Q, int q, const bf16x8 (&x)[D / 32]) {
  float m = 0.f;
#pragma unroll
  for (int i = 0; i < D / 32; ++i)
#pragma unroll
    for (int k = 0; k < 8; ++k) m = fmaxf(m, fabsf((float)x[i][k]));
  m = fmaxf(m, lane_xor16(m));
  m = fmaxf(m, lane_xor32(m));
  // the scale that kv_q8 would take, but no less than 2^-122: the second's is 2^-4 of it
  const unsigned u = __float_as_uint(m);
  int e = (int)(u >> 23) - 127 - 8 + ((u & 0x7fffffu) > 0x600000u);
  e = min(max(e, -122), 120);                 // a query that is not finite stays so
  const float down = __uint_as_float((unsigned)(127 - e) << 23);
  Q.e_hi[q] = e + 127;
  Q.e_lo[q] = e + 123;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    int hi = 0, lo = 0;
    if (i < D / 16) {
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        const float a = (float)x[i >> 1][4 * (i & 1) + 2 * p] * down, b = (float)x[i >> 1][4 * (i & 1) + 2 * p + 1] * down;
        hi = p ? __builtin_amdgcn_cvt_pk_fp8_f32(a, b, hi, true) : __builtin_amdgcn_cvt_pk_fp8_f32(a, b, hi, false);
        const auto v = p ? __builtin_amdgcn_cvt_pk_f32_fp8(hi, true) : __builtin_amdgcn_cvt_pk_f32_fp8(hi, false);
        const float ra = (a - v[0]) * 16.f, rb = (b - v[1]) * 16.f;
        lo = p ? __builtin_amdgcn_cvt_pk_fp8_f32(ra, rb, lo, true) : __builtin_amdgcn_cvt_pk_fp8_f32(ra, rb, lo, false);
      }
    }
    Q.hi[q][i] = hi;
    Q.lo[q][i] = lo;
  }
}

// Scores of a block: s[q][t][e] of the lane's row of tile q against unit j, slot
// 4 t + e.
template <int D, int QT, int NS, class B>
__device__ __forceinline__ void scores(const B& f, const Queries<D, QT, NS>& Q, floatx4 (&s)[QT][4]) {
  const int c16 = lane_id() & 15;
  const uint4 kscale = f.key_scales();
#pragma unroll
  for (int t = 0; t < 4; ++t) {
#pragma unroll
    for (int q = 0; q < QT; ++q) s[q][t] = floatx4{0.f, 0.f, 0.f, 0.f};
    const unsigned kbyte = (word(kscale, t) >> (8 * (c16 & 3))) & 255u;
    if constexpr (NS == 1) {
      i32x8 kf = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
      for (int h = 0; h < D / 64; ++h) {
        const uint4 w = f.key(t, h);
        kf[4 * h + 0] = (int)w.x;
        kf[4 * h + 1] = (int)w.y;
        kf[4 * h + 2] = (int)w.z;
        kf[4 * h + 3] = (int)w.w;
      }
#pragma unroll
      for (int q = 0; q < QT; ++q)
        s[q][t] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(kf, Q.lo[q], s[q][t], 0, 0, 0, (int)kbyte, 0, Q.e_lo[q]);
#pragma unroll
      for (int q = 0; q < QT; ++q)
        s[q][t] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(kf, Q.hi[q], s[q][t], 0, 0, 0, (int)kbyte, 0, Q.e_hi[q]);
    } else {
      const float ksc = __uint_as_float(kbyte << 23);
#pragma unroll
      for (int h = 0; h < D / 64; ++h) {
        const uint4 kq = f.key(t, h);
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          const bf16x8 kf = cvt8(x ? kq.z : kq.x, x ? kq.w : kq.y, ksc);
#pragma unroll
          for (int n = 0; n < NS; ++n)
#pragma unroll
            for (int q = 0; q < QT; ++q)
              s[q][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, Q.q[n][q][2 * h + x], s[q][t], 0, 0, 0);
        }
      }
    }
  }
}

// The block's probabilities, in PT bf16 terms, and values.  `tail`: some row of the
// wave does not see every key of the block.
template <int D, int QT, int PT>
__device__ __forceinline__ void attend(uint4 (&v)[D / 16], uint4 vscale, floatx4 (&s)[QT][4], float c, bool tail, int t0, int n_keys,
                                       const int (&qlimit)[QT], floatx4 (&acc)[QT][D / 16], float (&m_run)[QT],
                                       float (&l_run)[QT]) {
  const int u0 = t0 + 16 * (lane_id() >> 4);          // unit j's first position
  if (tail) {
    asm volatile("");                // a branch: else every block is masked, 250 of 600 instructions
    // An unseen key's scale byte may be anything, a later row's that of NaN
    // (infinite here, and times a probability of zero NaN): the rows that see
    // such a key get the NaN here, and the scale is taken out.
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const unsigned w = word(vscale, i >> 2), at = 255u << (8 * (i & 3));
      const bool odd = (w & at) == at;
#pragma unroll
      for (int q = 0; q < QT; ++q)
        s[q][i >> 2][i & 3] = u0 + i >= qlimit[q] ? -INFINITY : odd ? __uint_as_float(0x7fc00000u) : s[q][i >> 2][i & 3];
      (i < 4 ? vscale.x : i < 8 ? vscale.y : i < 12 ? vscale.z : vscale.w) = odd ? w & ~at : w;
    }
    auto live = [&](unsigned x, int at) {             // the bytes of slots at .. at + 3: behind the last key may be NaN
      const int n = n_keys - (u0 + at);
      return n >= 4 ? x : n <= 0 ? 0u : x & ((1u << (8 * n)) - 1u);
    };
#pragma unroll
    for (int dt = 0; dt < D / 16; ++dt)
      v[dt] = make_uint4(live(v[dt].x, 0), live(v[dt].y, 4), live(v[dt].z, 8), live(v[dt].w, 12));
  }
  float bm[QT], m_use[QT];
  bool rescale = false;
#pragma unroll
  for (int q = 0; q < QT; ++q) {
    bm[q] = -INFINITY;
#pragma unroll
    for (int i = 0; i < 16; ++i) bm[q] = fmaxf(bm[q], s[q][i >> 2][i & 3]);
  }
#pragma unroll
  for (int q = 0; q < QT; ++q) bm[q] = fmaxf(bm[q], lane_xor16(bm[q]));
#pragma unroll
  for (int q = 0; q < QT; ++q) bm[q] = fmaxf(bm[q], lane_xor32(bm[q]));
#pragma unroll
  for (int q = 0; q < QT; ++q) {
    const float bx = bm[q] * c, m_old = m_run[q];
    const float m_new = (bx > m_old + kRescaleSlack || m_old == -INFINITY) ? fmaxf(bx, m_old) : m_old;
    m_use[q] = m_new == -INFINITY ? 0.f : m_new;
    rescale |= m_new != m_old;
    bm[q] = m_old;
    m_run[q] = m_new;
  }
  if (__any(rescale)) {
#pragma unroll
    for (int q = 0; q < QT; ++q) {
      const float alpha = fast_exp2(bm[q] - m_use[q]);
      l_run[q] *= alpha;
#pragma unroll
      for (int dt = 0; dt < D / 16; ++dt) acc[q][dt] *= alpha;
    }
  }
  bf16x8 pf[PT][QT][2];
#pragma unroll
  for (int i = 0; i < 16; ++i) {           // slot i of unit j
    const float vsc = __uint_as_float(((word(vscale, i >> 2) >> (8 * (i & 3))) & 255u) << 23);
#pragma unroll
    for (int q = 0; q < QT; ++q) {
      const float p = fast_exp2(fmaf(s[q][i >> 2][i & 3], c, -m_use[q]));
      l_run[q] += p;
      __bf16 t[PT];
      split<PT>(p * vsc, t);
#pragma unroll
      for (int n = 0; n < PT; ++n) pf[n][q][i >> 3][i & 7] = t[n];
    }
  }
  __builtin_amdgcn_s_setprio(1);           // matrix work before the other wave's softmax: eight prompts 105 to 98 us
  constexpr int AT = PT == 2 ? 2 : 1;      // channel tiles at once: of one, four products would wait for one another
#pragma unroll
  for (int dt = 0; dt < D / 16; dt += AT) {
#pragma unroll
    for (int st = 0; st < 2; ++st) {       // slots 8 st .. 8 st + 7 of unit j
      bf16x8 vf[AT];
#pragma unroll
      for (int x = 0; x < AT; ++x) {
        const uint4 w = v[dt + x];
        vf[x] = cvt8(st ? w.z : w.x, st ? w.w : w.y, 1.0f);
      }
#pragma unroll
      for (int n = 0; n < PT; ++n)
#pragma unroll
        for (int x = 0; x < AT; ++x)
#pragma unroll
          for (int q = 0; q < QT; ++q)
            acc[q][dt + x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf[x], pf[n][q][st], acc[q][dt + x], 0, 0, 0);
    }
  }
  __builtin_amdgcn_s_setprio(0);
}

// ---- the line of blocks ----

struct Seq {
  int b, L, r0, kb, rows, n_rg;
};
__device__ __forceinline__ Seq seq_of(const Q8Params& a, int slot, int item_rows) {
  Seq s;
  s.b = a.seq_ids ? a.seq_ids[slot] : slot;
  s.L = min(max(a.ctx_lens[s.b], 0), a.slots);
  s.r0 = a.cu_q[s.b];
  s.kb = min(max(a.cu_q[s.b + 1] - s.r0, 0), a.max_q);
  s.rows = s.kb * a.G;
  s.n_rg = (s.rows + item_rows - 1) / item_rows;
  return s;
}
// The same where all lanes ask for one slot: scalar loads.
__device__ __forceinline__ Seq same_seq_of(const Q8Params& a, int slot, int item_rows) {
  Seq s;
  s.b = a.seq_ids ? scalar(a.seq_ids)[slot] : slot;
  s.L = min(max(scalar(a.ctx_lens)[s.b], 0), a.slots);
  s.r0 = scalar(a.cu_q)[s.b];
  s.kb = min(max(scalar(a.cu_q)[s.b + 1] - s.r0, 0), a.max_q);
  s.rows = s.kb * a.G;
  s.n_rg = (s.rows + item_rows - 1) / item_rows;
  return s;
}
// Window row of a packed row.
__device__ __forceinline__ int pos_of(const Q8Params& a, int row) { return a.log2g >= 0 ? row >> a.log2g : row / a.G; }
__device__ __forceinline__ ScalarInts pages_of(const Q8Params& a, int slot) {
  const int b = a.seq_ids ? scalar(a.seq_ids)[slot] : slot;
  return scalar(a.page_table + (size_t)b * a.max_pages);
}
// Steps (of `step` keys) of row group r: up to the last key that its last row sees.
__device__ __forceinline__ int item_steps(const Q8Params& a, const Seq& s, int r, int item_rows, int step) {
  const int last = min((r + 1) * item_rows, s.rows) - 1;
  return (int)((unsigned)(s.L + pos_of(a, last) + step) / (unsigned)step);
}
__device__ __forceinline__ long head_steps(const Q8Params& a, const Seq& s, int item_rows, int step) {
  long n = 0;
  for (int r = 0; r < s.n_rg; ++r) n += item_steps(a, s, r, item_rows, step);
  return n;
}
__device__ __forceinline__ long span_start(long total, long n, long w) { return w * total / n; }
// Spans in use: no more than there are groups of `parts` steps.
__device__ __forceinline__ long spans(long total, int parts, int grid) {
  const long n = (total + parts - 1) / parts;
  return n < grid ? (n > 0 ? n : 1) : grid;
}

// A workgroup's way along its items: the present one's steps j .. end.  Its
// sequence is read again where it is needed: two walks' would take the scalar
// registers that the computation needs.
template <bool DEALT> struct Walk {            // along a span of the line
  int slot, g, r, steps, j, end;
  int span, len;       // the span's number, and its steps
  int first;           // where the item begins, counted from the span's start
  __device__ __forceinline__ bool whole() const { return j == 0 && end == steps; }
  // of the item's part, which no more than two items of a span have
  __device__ __forceinline__ int part() const { return 2 * span + (first >= 0 ? 1 : 0); }
};
template <> struct Walk<true> {                // whole items, dealt out
  int slot, g, r, end;
  static constexpr int j = 0;
  int round, rounds;
  const int* list;           // the rounds' items
  __device__ __forceinline__ bool whole() const { return true; }
  __device__ __forceinline__ int part() const { return 0; }
};

// The next item with steps for this workgroup; false at the end.
template <int ITEM, int STEP>
__device__ __forceinline__ bool advance(const Q8Params& a, Walk<false>& c) {
  if (c.first + c.end >= c.len) return false;
  c.first += c.steps;
  Seq sq = same_seq_of(a, c.slot, ITEM);
  if (++c.r == sq.n_rg) {
    c.r = 0;
    if (++c.g == a.Hkv) {
      c.g = 0;
      do {
        if (++c.slot >= a.n_seq) return false;
        sq = same_seq_of(a, c.slot, ITEM);
      } while (sq.n_rg == 0);
    }
  }
  c.steps = item_steps(a, sq, c.r, ITEM, STEP);
  c.j = 0;
  c.end = min(c.steps, c.len - c.first);
  return true;
}
template <int ITEM, int STEP>
__device__ __forceinline__ bool advance(const Q8Params& a, Walk<true>& c) {
  if (++c.round >= c.rounds) return false;
  c.slot = __builtin_amdgcn_readfirstlane(c.list[3 * c.round]);
  c.g = __builtin_amdgcn_readfirstlane(c.list[3 * c.round + 1]);
  c.r = __builtin_amdgcn_readfirstlane(c.list[3 * c.round + 2]);
  c.end = item_steps(a, same_seq_of(a, c.slot, ITEM), c.r, ITEM, STEP);
  return true;
}

// The line as a workgroup knows it: every one adds it all up, a thread
// neighbouring slots.
struct Line {
  static constexpr int kKept = 1024;
  int steps[kKept];    // a head's steps, of the first slots
  long sum[4], at[2];
  int part[4];
};
struct Share {         // a thread's
  int sl0, sl1;        // its slots
  long at, len;        // where they begin, and their steps
  int most;            // the longest item's
};

// The line's length, of which the merge reads the last: 0 where nothing is cut.
template <int ITEM, int STEP>
__device__ __forceinline__ long add_up(const Q8Params& a, Line& line, Share& mine) {
  const int tid = threadIdx.x, lane = lane_id(), wv = tid >> 6;
  const int per = (a.n_seq + 255) / 256;
  mine.sl0 = min(tid * per, a.n_seq);
  mine.sl1 = min(mine.sl0 + per, a.n_seq);
  mine.len = 0;
  mine.most = 0;
  for (int i = mine.sl0; i < mine.sl1; ++i) {
    const Seq sq = seq_of(a, i, ITEM);
    const long n = head_steps(a, sq, ITEM, STEP);
    if (i < Line::kKept) line.steps[i] = (int)min(n, 0x7fffffffl);
    mine.len += a.Hkv * n;
    if (sq.n_rg > 0) mine.most = max(mine.most, item_steps(a, sq, sq.n_rg - 1, ITEM, STEP));
  }
  long incl = mine.len;
#pragma unroll
  for (int o = 1; o < kWave; o <<= 1) {
    const long up = __shfl_up(incl, o, kWave);
    if (lane >= o) incl += up;
  }
  if (lane == kWave - 1) line.sum[wv] = incl;
  __syncthreads();
  long total = 0;
  mine.at = incl - mine.len;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (i < wv) mine.at += line.sum[i];
    total += line.sum[i];
  }
  if (blockIdx.x == 0 && tid == 0) a.span[gridDim.x].first = total;
  return total;
}

// Sum over the threads before this one; every thread calls.
__device__ __forceinline__ int threads_before(int v, int (&part)[4], int* all = nullptr) {
  const int lane = lane_id(), wv = threadIdx.x >> 6;
  int incl = v;
#pragma unroll
  for (int o = 1; o < kWave; o <<= 1) {
    const int up = __shfl_up(incl, o, kWave);
    if (lane >= o) incl += up;
  }
  __syncthreads();                                  // the previous call's readers are done
  if (lane == kWave - 1) part[wv] = incl;
  __syncthreads();
  int before = 0, sum = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    before += i < wv ? part[i] : 0;
    sum += part[i];
  }
  if (all) *all = sum;
  return before + incl - v;
}

// Items dealt out whole, by falling length in classes of 2^shift steps (256 of
// them at most; within a class by slot, head and row group).  A round gives every
// workgroup one; neighbours in that order, which are a head's, go to one XCD.
struct Deal {
  static constexpr int kRounds = 16, kClasses = 256;
  int above[kClasses + 1];   // items of longer classes
  int list[3 * kRounds];
};
// First row group of at least s steps.
__device__ __forceinline__ int first_of(const Q8Params& a, const Seq& sq, int s, int item_rows, int step) {
  const long x = (long)(s - 1) * step - sq.L;
  if (x <= 0) return 0;
  const long need = x * a.G + 1;
  return need > sq.rows ? sq.n_rg : (int)((need + item_rows - 1) / item_rows) - 1;
}
// Returns whether dealing out is worth it, and if so this workgroup's walk.
template <int ITEM, int STEP>
__device__ __forceinline__ bool deal(const Q8Params& a, Line& line, Deal& d, const Share& mine, long total, Walk<true>& c) {
  const int grid = gridDim.x, tid = threadIdx.x, lane = lane_id();
  if (total < grid || (long)a.n_seq * a.Hkv > (long)Deal::kRounds * grid) return false;
  // the longest item
  int most = mine.most;
#pragma unroll
  for (int o = 1; o < kWave; o <<= 1) most = max(most, __shfl_xor(most, o, kWave));
  __syncthreads();
  if (lane == 0) line.part[tid >> 6] = most;
  d.above[tid] = 0;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 4; ++i) most = max(most, line.part[i]);
  // Cutting costs its partial results, written and read: about 3 steps for 32 rows
  // of an item; less where there are few.  Measured, cut / dealt: prompts of 512 to
  // 1024 tokens, 32 heads on 4, eight of them 163 / 115 us, four 108 / 70; windows
  // of 8 over 1000 tokens, 64 of them (half of the workgroups with an item) 41 / 48;
  // of 128 over 2000 to 4000, eight of them 103 / 181.
  const float mean = (float)((double)total / grid), limit = mean + fminf(0.8f * mean, (float)(ITEM * kBlk * 3 / (32 * STEP)));
  if ((float)most > limit) return false;
  int shift = 0;
  while ((most - 1) >> shift >= Deal::kClasses) ++shift;
  // the classes' items of one head; a slot's row groups to `team` threads
  int team = 1;
  while (team < kWave && 2 * team * a.n_seq <= 256) team *= 2;
  for (int i = tid / team; i < a.n_seq; i += 256 / team) {
    const Seq sq = seq_of(a, i, ITEM);
    for (int r = tid & (team - 1); r < sq.n_rg; r += team)
      atomicAdd(&d.above[(most - item_steps(a, sq, r, ITEM, STEP)) >> shift], 1);
  }
  __syncthreads();
  const int n = d.above[tid] * a.Hkv;
  int items;
  const int before = threads_before(n, line.part, &items);
  if (items > Deal::kRounds * grid) return false;   // then the cuts cost little
  d.above[tid] = before;
  if (tid == 0) d.above[Deal::kClasses] = items;
  __syncthreads();
  // A lane looks up one place: of this workgroup, of the round's first and of its last.
  const int xcd = (blockIdx.x & 7) * (grid >> 3) + (blockIdx.x >> 3);
  const int round = lane / 3, who = lane % 3, p = who == 0 ? xcd : who == 1 ? 0 : grid - 1;
  const int k = round * grid + (round & 1 ? grid - 1 - p : p);
  int cls = 0, hi = Deal::kClasses;                 // above[cls] <= k < above[hi]
  while (hi - cls > 1) {
    const int mid = (cls + hi) / 2;
    if (d.above[mid] <= k) cls = mid; else hi = mid;
  }
  const bool is = round < Deal::kRounds && k < items;
  const float load = is ? (float)(most - (cls << shift)) : 0.f;
  const float worst = fmaxf(wave_sum(who == 1 ? load : 0.f), wave_sum(who == 2 ? load : 0.f));
  if (!(worst <= limit)) return false;
  c.rounds = __popcll(__ballot(is && who == 0));
  for (int i = 0; i < c.rounds; ++i) {
    const int ci = __shfl(cls, 3 * i, kWave), ki = __shfl(k, 3 * i, kWave);
    const int s_hi = most - (ci << shift), s_lo = max(s_hi - (1 << shift) + 1, 1);
    int have = 0;
    for (int sl = mine.sl0; sl < mine.sl1; ++sl) {
      const Seq sq = seq_of(a, sl, ITEM);
      have += (first_of(a, sq, s_hi + 1, ITEM, STEP) - first_of(a, sq, s_lo, ITEM, STEP)) * a.Hkv;
    }
    int at = ki - d.above[ci] - threads_before(have, line.part);
    if (at >= 0 && at < have) {
      for (int sl = mine.sl0; sl < mine.sl1; ++sl) {
        const Seq sq = seq_of(a, sl, ITEM);
        const int r0 = first_of(a, sq, s_lo, ITEM, STEP), m = first_of(a, sq, s_hi + 1, ITEM, STEP) - r0;
        if (at < m * a.Hkv) {
          d.list[3 * i] = sl;
          d.list[3 * i + 1] = at / m;
          d.list[3 * i + 2] = r0 + at % m;
          break;
        }
        at -= m * a.Hkv;
      }
    }
  }
  if (blockIdx.x == 0 && tid == 0) a.span[grid].first = 0;
  __syncthreads();
  c.rounds = __builtin_amdgcn_readfirstlane(c.rounds);
  c.round = -1;
  c.list = d.list;
  return true;
}

// Where the workgroup's walk begins; false when it has none.
template <int ITEM, int STEP>
__device__ __forceinline__ bool begin_walk(const Q8Params& a, Line& line, const Share& mine, long total, int parts,
                                           Walk<false>& c) {
  const long n = spans(total, parts, gridDim.x);
  // Neighbouring spans to one XCD (workgroups go to the 8 XCDs in turn): a
  // prompt's items of one head then find its keys in one L2.  The grid is a
  // multiple of 8, so each of the 8 has workgroups for its `each` spans.
  const int each = (int)((n + 7) / 8), w = (int)(blockIdx.x & 7) * each + (int)(blockIdx.x >> 3);
  if ((int)(blockIdx.x >> 3) >= each || w >= n || total == 0) return false;
  const long p0 = span_start(total, n, w), p1 = span_start(total, n, w + 1);
  if (p0 >= mine.at && p0 < mine.at + mine.len) {
    long at = mine.at;
    for (int i = mine.sl0; i < mine.sl1; ++i) {
      long k = i < Line::kKept ? line.steps[i] : 0x7fffffff;
      if (k == 0x7fffffff) k = head_steps(a, seq_of(a, i, ITEM), ITEM, STEP);
      k *= a.Hkv;
      if (p0 < at + k) {
        line.at[0] = i;
        line.at[1] = at;
        break;
      }
      at += k;
    }
  }
  __syncthreads();
  // the same for all lanes, and known to be
  auto uniform = [](long x) {
    return (long)(((unsigned long)(unsigned)__builtin_amdgcn_readfirstlane((int)(x >> 32)) << 32) |
                  (unsigned)__builtin_amdgcn_readfirstlane((int)x));
  };
  c.span = __builtin_amdgcn_readfirstlane(w);
  const long from = uniform(p0);
  c.len = __builtin_amdgcn_readfirstlane((int)(p1 - p0));
  c.slot = __builtin_amdgcn_readfirstlane((int)line.at[0]);
  long first = uniform(line.at[1]);
  const Seq sq = same_seq_of(a, c.slot, ITEM);
  long hb = c.slot < Line::kKept ? line.steps[c.slot] : 0x7fffffff;
  if (hb == 0x7fffffff) hb = head_steps(a, sq, ITEM, STEP);
  hb = uniform(hb);
  c.g = (int)((from - first) / hb);
  first += c.g * hb;
  c.r = 0;
  c.steps = item_steps(a, sq, 0, ITEM, STEP);
  while (first + c.steps <= from) {
    first += c.steps;
    c.steps = item_steps(a, sq, ++c.r, ITEM, STEP);
  }
  c.first = (int)(first - from);
  c.j = -c.first;
  c.end = min(c.steps, c.len - c.first);
  if (threadIdx.x == 0) a.span[c.span] = {first, c.steps, c.slot, c.g, c.r};
  return true;
}

// What a wave holds of its 16 QT rows while it walks their keys.
template <typename DT, int D, int QT>
struct Rows {
  static constexpr int NS = sizeof(DT) == 2 ? 1 : 3;
  floatx4 acc[QT][D / 16];
  float m_run[QT], l_run[QT];
  Queries<D, QT, NS> Q;
  int qlimit[QT];
  int pr0;         // first packed row of the item's (sequence, head)
  int n_keys;      // keys that some row sees
  int all_see;     // keys below are seen by every row

  template <class W>
  __device__ __forceinline__ void begin(const Q8Params& a, const W& c, int first_row) {
    const int lane = lane_id(), c16 = lane & 15, j = lane >> 4;
    const Seq sq = same_seq_of(a, c.slot, 16 * QT);
    pr0 = first_row;
    n_keys = pr0 < sq.rows ? sq.L + pos_of(a, min(pr0 + 16 * QT, sq.rows) - 1) + 1 : 0;
    all_see = sq.L + pos_of(a, pr0) + 1;
#pragma unroll
    for (int q = 0; q < QT; ++q) {
      m_run[q] = -INFINITY;
      l_run[q] = 0.f;
#pragma unroll
      for (int dt = 0; dt < D / 16; ++dt) acc[q][dt] = floatx4{0.f, 0.f, 0.f, 0.f};
    }
    if (n_keys == 0) return;
#pragma unroll
    for (int q = 0; q < QT; ++q) {
      const int pr = pr0 + 16 * q + c16;
      qlimit[q] = sq.L + pos_of(a, min(pr, sq.rows - 1)) + 1;
      const int row = min(pr, sq.rows - 1), i = pos_of(a, row), hl = row - i * a.G;      // rows behind the last: its copies
      const DT* qr = reinterpret_cast<const DT*>(a.q) + (size_t)(sq.r0 + i) * a.q_stride + (size_t)(c.g * a.G + hl) * D;
      if constexpr (NS == 1) {
        bf16x8 x[D / 32];
#pragma unroll
        for (int i = 0; i < D / 32; ++i) x[i] = ld16<bf16x8>(qr + 16 * (4 * (i >> 1) + j) + 8 * (i & 1));
        split_e4m3<D, QT>(Q, q, x);
      } else {
#pragma unroll
        for (int x = 0; x < D / 32; ++x) {
          const DT* p = qr + 16 * (4 * (x >> 1) + j) + 8 * (x & 1);
          const floatx4 lo = ld16<floatx4>(p), hi = ld16<floatx4>(p + 4);
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            __bf16 t[NS];
            split<NS>(e < 4 ? lo[e & 3] : hi[e & 3], t);
#pragma unroll
            for (int n = 0; n < NS; ++n) Q.q[n][q][x][e] = t[n];
          }
        }
      }
    }
    // The compiler counts its own loads only: the queries have to be here before
    // others are under way, or their wait, inside the walk, would be for those too.
#pragma unroll
    for (int q = 0; q < QT; ++q) {
      if constexpr (NS == 1) {
        asm volatile("" : "+v"(Q.hi[q]), "+v"(Q.lo[q]));
      } else {
#pragma unroll
        for (int n = 0; n < NS; ++n)
#pragma unroll
          for (int x = 0; x < D / 32; ++x) asm volatile("" : "+v"(Q.q[n][q][x]));
      }
    }
  }

  template <class B>
  __device__ __forceinline__ void block(const Q8Params& a, const B& f, int t0) {
    if (t0 >= n_keys) return;
    floatx4 s[QT][4];
    scores<D, QT, NS>(f, Q, s);
    uint4 v[D / 16];                 // asked for now, for they take their time from LDS
#pragma unroll
    for (int dt = 0; dt < D / 16; ++dt) v[dt] = f.val(dt);
    attend<D, QT, NS>(v, f.val_scales(), s, a.scale_log2, t0 + kBlk > all_see, t0, n_keys, qlimit, acc, m_run, l_run);
  }

  // The lanes' sums joined: l_run is the row's from here on.
  __device__ __forceinline__ void join_lanes() {
#pragma unroll
    for (int q = 0; q < QT; ++q) {
      l_run[q] += lane_xor16(l_run[q]);
      l_run[q] += lane_xor32(l_run[q]);
    }
  }

  // One tile to LDS, and one from there merged in: sizeof(floatx4) * (D / 16) *
  // 64 bytes and 32 floats.
  __device__ __forceinline__ void give(int q, floatx4* buf, float* ml) const {
    const int lane = lane_id();
#pragma unroll
    for (int dt = 0; dt < D / 16; ++dt) buf[dt * kWave + lane] = acc[q][dt];
    if (lane < 16) {
      ml[lane] = m_run[q];
      ml[16 + lane] = l_run[q];
    }
  }
  __device__ __forceinline__ void take(int q, const floatx4* buf, const float* ml) {
    const int lane = lane_id(), c16 = lane & 15;
    const float m2 = ml[c16], l2 = ml[16 + c16];
    const float m = fmaxf(m_run[q], m2), mu = m == -INFINITY ? 0.f : m;
    const float x = fast_exp2(m_run[q] - mu), y = fast_exp2(m2 - mu);
    m_run[q] = m;
    l_run[q] = l_run[q] * x + l2 * y;
#pragma unroll
    for (int dt = 0; dt < D / 16; ++dt) acc[q][dt] = acc[q][dt] * x + buf[dt * kWave + lane] * y;
  }

  // The item's rows to the output, or its part of them to the partial results.
  template <class W>
  __device__ __forceinline__ void finish(const Q8Params& a, const W& c, int item_rows, int row0) const {
    const int lane = lane_id(), c16 = lane & 15, j = lane >> 4;
    const Seq sq = same_seq_of(a, c.slot, 16 * QT);
    const bool whole = c.whole();
    const size_t part_row = (size_t)c.part() * item_rows + row0;
#pragma unroll
    for (int q = 0; q < QT; ++q) {
      const int pr = pr0 + 16 * q + c16;
      if (pr >= sq.rows) continue;
      if (whole) {
        const int i = pos_of(a, pr), hl = pr - i * a.G;
        DT* o = reinterpret_cast<DT*>(a.out) + ((size_t)(sq.r0 + i) * a.Hq + c.g * a.G + hl) * D + 4 * j;
        const float inv = 1.f / l_run[q];
#pragma unroll
        for (int dt = 0; dt < D / 16; ++dt) {
          const floatx4 v = acc[q][dt] * inv;
          if constexpr (NS == 1) {
            bf16x4 w;
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = static_cast<bf16>(v[e]);
            *reinterpret_cast<bf16x4*>(o + 16 * dt) = w;
          } else {
            *reinterpret_cast<floatx4*>(o + 16 * dt) = v;
          }
        }
      } else {
        const size_t row = part_row + 16 * q + c16;
#pragma unroll
        for (int dt = 0; dt < D / 16; ++dt)
          *reinterpret_cast<floatx4*>(a.part_o + row * D + 16 * dt + 4 * j) = acc[q][dt];
        if (j == 0) {
          a.part_ml[2 * row] = m_run[q];
          a.part_ml[2 * row + 1] = l_run[q];
        }
      }
    }
  }
};

// One row group: the four waves take parts of the span's keys.
template <typename DT, int D>
__global__ __launch_bounds__(256, 2) void attn_q8_keys_kernel(Q8Params a) {
  constexpr int QT = 1, kItem = 16 * QT, kTile = (D / 16) * kWave;   // of floatx4
  __shared__ floatx4 s_acc[2][kTile];
  __shared__ float s_ml[2][32];
  const int tid = threadIdx.x, wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  __shared__ Line s_line;
  Share mine;
  const long total = add_up<kItem, kBlk>(a, s_line, mine);
  Walk<false> c;
  if (!begin_walk<kItem, kBlk>(a, s_line, mine, total, 4, c)) return;
  do {
    const int j0 = c.j, j1 = c.end;
    Rows<DT, D, QT> R;
    R.begin(a, c, c.r * kItem);
    const int part = (j1 - j0 + 3) / 4, b0 = j0 + wv * part;
    const int b1 = min(min(b0 + part, j1), (R.n_keys + kBlk - 1) / kBlk);
    const ScalarInts pt = pages_of(a, c.slot);
    // the next keys are asked for once the scores have used theirs, the next
    // values once the products have: they are under way in the same registers
    if (b0 < b1) {
      Block<D> f;
      Units units;
      units.look_up(a, pt, b0 * kBlk, c.g);
      load_keys<D>(a, f, b0 * kBlk, units);
      load_values<D>(a, f, b0 * kBlk, units);
      units.look_up(a, pt, (b0 + 1) * kBlk, c.g);
      for (int n = b0; n < b1; ++n) {
        floatx4 s[QT][4];
        scores<D, QT, Rows<DT, D, QT>::NS>(f, R.Q, s);
        const bool more = n + 1 < b1;
        __builtin_amdgcn_sched_barrier(0);          // or the loads move up, into registers of their own
        if (more) load_keys<D>(a, f, (n + 1) * kBlk, units);
        __builtin_amdgcn_sched_barrier(0);
        attend<D, QT, Rows<DT, D, QT>::NS == 1 ? 2 : 3>(f.v, f.vs, s, a.scale_log2, (n + 1) * kBlk > R.all_see, n * kBlk, R.n_keys, R.qlimit,
                                           R.acc, R.m_run, R.l_run);
        __builtin_amdgcn_sched_barrier(0);
        if (more) load_values<D>(a, f, (n + 1) * kBlk, units);
        units.look_up(a, pt, (n + 2) * kBlk, c.g);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    R.join_lanes();
#pragma unroll
    for (int q = 0; q < QT; ++q)
#pragma unroll
      for (int half = 2; half > 0; half >>= 1) {
        if (wv >= half && wv < 2 * half) R.give(q, s_acc[wv - half], s_ml[wv - half]);
        __syncthreads();
        if (wv < half) R.take(q, s_acc[wv], s_ml[wv]);
        __syncthreads();
      }
    if (wv == 0) R.finish(a, c, kItem, 0);
  } while (advance<kItem, kBlk>(a, c));
}

// RG row groups x KS parts of a step's keys.  A step's blocks, one per part, are
// asked for kDepth - 1 steps ahead by the waves of their part together; the
// barrier of a step makes them all arrive, and frees the stage that the step
// before has used.
template <int D, int QT, int RG> struct Ring {
  static constexpr int KS = 4 / RG, kStep = KS * kBlk, kItem = RG * 16 * QT;
  static constexpr int kDepth = KS == 2 ? 2 : 3;                // two workgroups per CU
  static constexpr int kStage = KS * LdsBlock<D>::kBytes;
};
template <typename DT, int D, int QT, int RG, class W>
__device__ __forceinline__ void walk_rows(const Q8Params& a, W c, char* s_ring) {
  typedef Ring<D, QT, RG> G;
  constexpr int KS = G::KS, kStep = G::kStep, WR = 16 * QT, kItem = G::kItem, kDepth = G::kDepth, kStage = G::kStage;
  typedef LdsBlock<D> B;
  constexpr int NL = B::kLoads / RG + 1;                        // loads of a wave per step
  constexpr int kTile = (D / 16) * kWave;
  static_assert(KS == 1 || kStage >= RG * (kTile * 16 + 128), "a merge fits the stage that its item has left");
  const int tid = threadIdx.x, lane = lane_id(), c16 = lane & 15, j = lane >> 4;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6), rg = wv % RG, part = wv / RG;

  // ---- the loads' walk, ahead of the computation's ----
  W e = c;
  int ej = c.j;
  bool more = true;                                 // steps to ask for
  int ahead = 0;                                    // steps asked for and not used yet
  const int ps = 1 << a.log2ps;
  Units units;
  ScalarInts pt = pages_of(a, e.slot);
  auto look_up = [&]() __attribute__((always_inline)) {
    units.look_up(a, pt, ej * kStep + part * kBlk, e.g);
  };
  int fill = 0;                                     // the next stage to fill
  auto issue = [&]() __attribute__((always_inline)) {
    const int t0 = ej * kStep + part * kBlk;
    char* stage = s_ring + fill * kStage + part * B::kBytes;
    const int ku = c16 >> 2, su = lane & 3;
    const uint8_t* kb = a.k_pages + ((unsigned long)units.of(ku) * (unsigned)(D * ps) +
                                     (unsigned)((((t0 + 16 * ku) & (ps - 1)) + (c16 & 3) + j * ps) * 16));
    const uint8_t* vb = a.v_pages + ((unsigned long)units.of(j) * (unsigned)(D * ps) +
                                     (unsigned)(((t0 + 16 * j) & (ps - 1)) + c16 * ps));
    const uint8_t* sb = a.scales + ((unsigned long)units.of(su) * (unsigned)(2 * ps) +
                                    (unsigned)(((t0 + 16 * su) & (ps - 1)) + (lane & 4 ? ps : 0)));
#pragma unroll
    for (int i = 0; i < NL - 1; ++i) {
      const int n = rg + RG * i;
      dma16(n < B::kKeys ? kb + (4 * (n >> 2) * ps + 4 * (n & 3)) * 16 : vb + 16 * (n - B::kKeys) * ps,
            stage + n * kWave * 16);
    }
    dma16(sb, stage + B::kLoads * kWave * 16);
    fill = fill + 1 == kDepth ? 0 : fill + 1;
    ++ahead;
    if (++ej == e.end) {
      more = advance<kItem, kStep>(a, e);
      ej = e.j;
      if (more) pt = pages_of(a, e.slot);
    }
    if (more) look_up();
  };
  look_up();
#pragma unroll 1
  for (int i = 0; i < kDepth - 1 && more; ++i) issue();

  int use = 0;                                      // the next stage to use
  do {
    Rows<DT, D, QT> R;
    R.begin(a, c, c.r * kItem + rg * WR);
    char* stage = nullptr;
    for (int n = c.j; n < c.end; ++n) {
      // steps behind this one that are under way: kDepth - 2, or fewer at the walk's end
      if (kDepth == 2 || --ahead == 0) wait_loads<0>(); else wait_loads<NL>();
      lds_barrier();
      if (more) issue();
      stage = s_ring + use * kStage;
      const B f{stage + part * B::kBytes};
      R.block(a, f, n * kStep + part * kBlk);
      use = use + 1 == kDepth ? 0 : use + 1;
    }
    R.join_lanes();
    if constexpr (KS == 2) {                        // in the stage that was used last: the next to be filled
      floatx4* buf = reinterpret_cast<floatx4*>(stage) + rg * kTile;
      float* ml = reinterpret_cast<float*>(stage + RG * kTile * 16) + rg * 32;
#pragma unroll
      for (int q = 0; q < QT; ++q) {
        lds_barrier();
        if (part) R.give(q, buf, ml);
        lds_barrier();
        if (!part) R.take(q, buf, ml);
      }
    }
    if (part == 0) R.finish(a, c, kItem, rg * WR);
  } while (advance<kItem, kStep>(a, c));
  wait_loads<0>();                                  // none may land after the workgroup has gone
}

template <typename DT, int D, int QT, int RG>
__global__ __launch_bounds__(256, 2) void attn_q8_rows_kernel(Q8Params a) {
  typedef Ring<D, QT, RG> G;
  __shared__ __attribute__((aligned(16))) char s_ring[G::kDepth * G::kStage];
  __shared__ Line s_line;
  __shared__ Deal s_deal;
  Share mine;
  const long total = add_up<G::kItem, G::kStep>(a, s_line, mine);
  Walk<true> items;
  Walk<false> span;
  if (deal<G::kItem, G::kStep>(a, s_line, s_deal, mine, total, items)) {
    if (advance<G::kItem, G::kStep>(a, items)) walk_rows<DT, D, QT, RG>(a, items, s_ring);
  } else if (begin_walk<G::kItem, G::kStep>(a, s_line, mine, total, 2, span)) {
    walk_rows<DT, D, QT, RG>(a, span, s_ring);
  }
}

// Merges the partial results of the items that a span's end has cut: 16 rows per
// workgroup, of the item that span blockIdx.y + 1 is the first to continue.  A
// thread takes four channels of a row: of few pieces all at once, which it weighs
// itself; of more, once the pieces' weights have been found, 16 lanes per row, and
// with few rows every second or fourth of them.
constexpr int kMergeRows = 16, kFewPieces = 4;
template <typename DT, int D>
__global__ __launch_bounds__(256) void attn_q8_merge_kernel(Q8Params a, int item_rows, int parts, int grid) {
  static_assert(kMergeRows == 256 / 16, "16 lanes per row");
  extern __shared__ float s_w[];                     // [kMergeRows][pieces]
  __shared__ floatx4 s_o[256];
  __shared__ float s_inv[kMergeRows];
  const long total = a.span[grid].first;
  const SpanHead item = a.span[blockIdx.y + 1];      // asked for together; not looked at where no span has written it
  const long n_span = spans(total, parts, grid);
  if (blockIdx.y + 1 >= n_span) return;
  const long w0 = blockIdx.y;
  if (item.first >= span_start(total, n_span, w0 + 1) || item.first < span_start(total, n_span, w0)) return;
  const Seq sq = same_seq_of(a, item.slot, item_rows);
  const int r = item.r, g = item.g, row0 = blockIdx.x * kMergeRows;
  const int rows = min(kMergeRows, sq.rows - r * item_rows - row0);
  if (rows <= 0) return;
  const long w1 = ((item.first + item.steps) * n_span - 1) / total;
  const int n = (int)(w1 - w0) + 1;                  // pieces
  // w0 holds the item's start, the others continue it
  auto row_at = [&](int i, int row) { return (size_t)(i ? 2 * (w0 + i) : 2 * w0 + 1) * item_rows + row0 + row; };
  const int tid = threadIdx.x;
  const int units = rows * (D / 4);
  auto put = [&](int e, const floatx4& o, float inv) {
    const int row = e / (D / 4), d = 4 * (e % (D / 4));
    const int pr = r * item_rows + row0 + row, i = pos_of(a, pr), hl = pr - i * a.G;
    DT* out = reinterpret_cast<DT*>(a.out) + ((size_t)(sq.r0 + i) * a.Hq + g * a.G + hl) * D + d;
    typedef DT __attribute__((ext_vector_type(4))) Four;
    Four w;
#pragma unroll
    for (int c = 0; c < 4; ++c) w[c] = from_f32<DT>(o[c] * inv);
    *reinterpret_cast<Four*>(out) = w;
  };
  if (n <= kFewPieces) {
    constexpr int PER = 2;          // units of a thread at a time
    for (int e0 = tid; e0 < units; e0 += PER * 256) {
      floatx4 o[PER][kFewPieces];
      float2 ml[PER][kFewPieces];
#pragma unroll
      for (int u = 0; u < PER; ++u) {
        const int e = min(e0 + 256 * u, units - 1), row = e / (D / 4), d = 4 * (e % (D / 4));
#pragma unroll
        for (int i = 0; i < kFewPieces; ++i)
          if (i < n) {
            const size_t at = row_at(i, row);
            o[u][i] = ld16<floatx4>(a.part_o + at * D + d);
            ml[u][i] = *reinterpret_cast<const float2*>(a.part_ml + 2 * at);
          }
      }
#pragma unroll
      for (int u = 0; u < PER; ++u) {
        if (e0 + 256 * u >= units) continue;
        float m = -INFINITY, l = 0.f;
#pragma unroll
        for (int i = 0; i < kFewPieces; ++i)
          if (i < n) m = fmaxf(m, ml[u][i].x);
        m = m == -INFINITY ? 0.f : m;
        floatx4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < kFewPieces; ++i)
          if (i < n) {
            const float x = fast_exp2(ml[u][i].x - m);
            l += x * ml[u][i].y;
            sum += x * o[u][i];
          }
        put(e0 + 256 * u, sum, 1.f / l);
      }
    }
    return;
  }
  if (const int row = tid >> 4; row < rows) {
    const int c = tid & 15;
    float m = -INFINITY, l = 0.f;
    for (int i = c; i < n; i += 16) {
      const float2 ml = *reinterpret_cast<const float2*>(a.part_ml + 2 * row_at(i, row));
      s_w[row * n + i] = ml.x;
      const float m2 = fmaxf(m, ml.x), mu = m2 == -INFINITY ? 0.f : m2;
      l = l * fast_exp2(m - mu) + ml.y * fast_exp2(ml.x - mu);
      m = m2;
    }
    float all = m;
#pragma unroll
    for (int o = 1; o < 16; o <<= 1) all = fmaxf(all, __shfl_xor(all, o, kWave));
    all = all == -INFINITY ? 0.f : all;
    l *= fast_exp2(m - all);
#pragma unroll
    for (int o = 1; o < 16; o <<= 1) l += __shfl_xor(l, o, kWave);
    for (int i = c; i < n; i += 16) s_w[row * n + i] = fast_exp2(s_w[row * n + i] - all);
    if (c == 0) s_inv[row] = 1.f / l;
  }
  __syncthreads();
  const int split = units <= 64 ? 4 : units <= 128 ? 2 : 1;
  const int team = 256 / split, part = tid / team;
  auto sum = [&](int e) {
    const int row = e / (D / 4), d = 4 * (e % (D / 4));
    floatx4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
    for (int i = part; i < n; i += split) o += s_w[row * n + i] * ld16<floatx4>(a.part_o + row_at(i, row) * D + d);
    return o;
  };
  if (split == 1) {
    for (int e = tid; e < units; e += 256) put(e, sum(e), s_inv[e / (D / 4)]);
    return;
  }
  const int e = tid % team;
  if (e < units) s_o[tid] = sum(e);
  __syncthreads();
  if (part == 0 && e < units) {
    floatx4 o = s_o[tid];
    for (int x = 1; x < split; ++x) o += s_o[tid + x * team];
    put(e, o, s_inv[e / (D / 4)]);
  }
}

struct Q8Plan {
  int qt, rg;          // tiles per wave, row groups
  int item_rows, parts, grid;      // parts: steps per span at least
};
// Row groups share the keys that they load, and leave fewer parts of them to
// merge; but where rows are few they are copies, and their work is wasted.  Two
// tiles per wave share a key's conversion, and halve the waves that a row count
// fills.  Measured (32 heads on 4; 64 windows over 1024 to 8192 tokens; both kernels,
// us) at rg = 1 / 2 / 4 with one tile, for 16, 32 and 64 rows:
//   bf16, D = 128   82 / 78 / 84    109 / 85 / 93     187 / 118 / 99
//   bf16, D = 64    47 / 48 / 63     67 / 54 / 71     112 / 80 / 76
//   fp32, D = 128   83 / 85 / 106   118 / 101 / 135   200 / 162 / 149
//   fp32, D = 64    50 / 54 / 77     75 / 68 / 100    124 / 109 / 105
// (rg = 1 has two terms of each probability in bf16, the others one).  Two tiles, the
// first kernel alone, D = 128: at rg = 2 64 rows take 106; at rg = 4, one tile / two,
// 128 rows 101 / 92, eight prompts 124 / 100.
Q8Plan plan_of(int n_seq, int Hq, int Hkv, int max_q, bool bf16) {
  Q8Plan p;
  const long rows = (long)max_q * (Hq / Hkv);
  p.qt = bf16 && rows > 64 ? 2 : 1;                 // fp32, three terms per query: no registers for two tiles
  p.rg = rows <= 16 ? 1 : rows <= 32 ? 2 : 4;
  p.item_rows = 16 * p.qt * p.rg;
  p.parts = p.rg == 1 ? 4 : 2;
  p.grid = attn_q8_grid(device_cus());
  return p;
}

}  // namespace

// As many workgroups as are resident, alike on every XCD: the same number each.
int attn_q8_grid(int cus) { return std::max(8, 2 * cus / 8 * 8); }

size_t attn_q8_workspace(int n_seq, int Hq, int Hkv, int D, int max_q) {
  size_t most = 0;              // either type
  for (const bool b : {false, true}) {
    const Q8Plan p = plan_of(n_seq, Hq, Hkv, max_q, b);
    const size_t rows = 2 * (size_t)p.grid * p.item_rows;
    const size_t n = rows * (D + 2) * 4 + (p.grid + 1) * sizeof(SpanHead);
    most = std::max(most, (n + 255) / 256 * 256);
  }
  return most;
}

hipError_t launch_attn_q8(const AttnQ8Launch& L, hipStream_t st) {
  const Q8Plan pl = plan_of(L.n_seq, L.Hq, L.Hkv, L.max_q, L.dtype_bf16);
  const size_t rows = 2 * (size_t)pl.grid * pl.item_rows;
  Q8Params p{};
  p.q = L.q;
  p.q_stride = L.q_stride;
  p.k_pages = (const uint8_t*)L.k_pages;
  p.v_pages = (const uint8_t*)L.v_pages;
  p.scales = (const uint8_t*)L.scales;
  p.page_table = L.page_table;
  p.ctx_lens = L.ctx_lens;
  p.cu_q = L.cu_q;
  p.seq_ids = L.seq_ids;
  p.out = L.out;
  p.part_o = (float*)L.workspace;
  p.part_ml = p.part_o + rows * L.D;
  p.span = (SpanHead*)(p.part_ml + 2 * rows);
  p.max_pages = L.max_pages;
  p.Hq = L.Hq;
  p.Hkv = L.Hkv;
  p.G = L.Hq / L.Hkv;
  p.log2g = (p.G & (p.G - 1)) ? -1 : __builtin_ctz(p.G);
  p.log2ps = __builtin_ctz(L.page_size);
  p.num_pages = L.num_pages;
  p.n_seq = L.n_seq;
  p.max_q = L.max_q;
  p.slots = table_slots(L.max_pages, L.page_size);
  p.scale_log2 = L.scale * 1.4426950408889634f;
  trace_begin(st);
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(pl.grid), dim3(256), 0, st, p); };
  auto pick = [&](auto dt, auto dim) {
    using DT = decltype(dt);
    constexpr int D = decltype(dim)::value, QT = sizeof(DT) == 2 ? 2 : 1;
    if (pl.rg == 1) go(attn_q8_keys_kernel<DT, D>);
    else if (pl.rg == 2) go(attn_q8_rows_kernel<DT, D, 1, 2>);
    else if (pl.qt == 1) go(attn_q8_rows_kernel<DT, D, 1, 4>);
    else go(attn_q8_rows_kernel<DT, D, QT, 4>);
  };
  typedef std::integral_constant<int, 64> D64;
  typedef std::integral_constant<int, 128> D128;
  if (L.dtype_bf16) {
    if (L.D == 128) pick(bf16(), D128()); else pick(bf16(), D64());
  } else {
    if (L.D == 128) pick(float(), D128()); else pick(float(), D64());
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  trace_mark(st);
  const dim3 cgrid(pl.item_rows / kMergeRows, pl.grid - 1);
  const size_t lds = (size_t)kMergeRows * pl.grid * 4;      // no item has more pieces than there are spans
  auto merge = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, cgrid, dim3(256), lds, st, p, pl.item_rows, pl.parts, pl.grid);
  };
  if (L.dtype_bf16) {
    if (L.D == 128) merge(attn_q8_merge_kernel<bf16, 128>); else merge(attn_q8_merge_kernel<bf16, 64>);
  } else {
    if (L.D == 128) merge(attn_q8_merge_kernel<float, 128>); else merge(attn_q8_merge_kernel<float, 64>);
  }
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  trace_mark(st);
  return hipSuccess;
}

}  // namespace ipdv
