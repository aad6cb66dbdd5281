// What attn_masked.hip and attn_mass.hip share: a window's rows, what each sees, the
// key operands of a block of 32 keys, and the modified scores.
#pragma once

#include <climits>

#include "common.h"
#include "kernels.h"

namespace ipdv {
namespace {

constexpr int kBlk = 32;                // keys per block

struct WindowParams {
  const void* q;
  long q_stride;
  const void* k_cache;
  const int32_t* page_table;
  const int32_t* ctx_lens;
  const int32_t* cu_q;
  const int32_t* seq_ids;
  const int32_t* first_key;
  const int32_t* end_key;
  const float* slopes;
  int max_pages, Hq, Hkv, G, log2ps, num_pages, n_seq, max_q, slots;
  int log2g;           // of G, or -1
  int window;          // keys that a row sees at most (INT_MAX: all)
  float scale2;        // scale log2(e); with a cap 2 log2(e) scale / cap
  float cap2;          // cap log2(e), 0: no cap
  float cap_scale;     // scale / cap
};
inline WindowParams window_params(const AttnMaskedLaunch& L) {
  WindowParams p{};
  p.q = L.q;
  p.q_stride = L.q_stride;
  p.k_cache = L.k_cache;
  p.page_table = L.page_table;
  p.ctx_lens = L.ctx_lens;
  p.cu_q = L.cu_q;
  p.seq_ids = L.seq_ids;
  p.first_key = L.mod.first_key;
  p.end_key = L.mod.end_key;
  p.slopes = L.mod.slopes;
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
  p.window = L.mod.window > 0 ? L.mod.window : INT_MAX;
  const float log2e = 1.4426950408889634f, cap = L.mod.softcap;
  p.cap2 = cap * log2e;
  p.cap_scale = cap > 0.f ? L.scale / cap : 0.f;
  p.scale2 = cap > 0.f ? 2.f * log2e * (L.scale / cap) : L.scale * log2e;
  return p;
}

// Values that all lanes share and no kernel writes: scalar loads.
typedef const __attribute__((address_space(4))) int32_t* ScalarInts;
__device__ __forceinline__ ScalarInts scalar(const int32_t* p) { return (ScalarInts)(uintptr_t)p; }
__device__ __forceinline__ int uni(int x) { return __builtin_amdgcn_readfirstlane(x); }

struct Seq {
  int b, L, r0, kb, rows;
  int end;             // positions that the table has slots for (all, if the lengths fit it)
};
__device__ __forceinline__ Seq seq_of(const WindowParams& a, int slot) {
  Seq s;
  s.b = a.seq_ids ? scalar(a.seq_ids)[slot] : slot;
  s.L = min(max(scalar(a.ctx_lens)[s.b], 0), a.slots);
  s.r0 = scalar(a.cu_q)[s.b];
  s.kb = min(max(scalar(a.cu_q)[s.b + 1] - s.r0, 0), a.max_q);
  s.rows = s.kb * a.G;
  s.end = min(s.L + s.kb, a.slots);
  return s;
}

// The (sequence slot, head) of workgroup x in row y of a grid whose width is a multiple of 8:
// rows are turned by the heads, since workgroups go to the 8 XCDs in turn.  So the work of one
// sequence, long or short, is shared out over all of them, and what follows on in
// y (tiles that read the same keys) stays on one XCD as far as that allows.  (By x alone, masses of
// eight prompts of 512 to 1024 tokens, 4 heads, kept the CUs busy for 57% of the time.)  -1: none.
__device__ __forceinline__ int slot_head_of(const WindowParams& a, int x, int y, int width) {
  const int at = (int)(((unsigned)x + (unsigned)width - (unsigned)y % (unsigned)width * (unsigned)a.Hkv % (unsigned)width) %
                       (unsigned)width);
  return at < a.n_seq * a.Hkv ? at : -1;
}

// What a row sees, and what biases its scores.
struct RowInfo {
  int lo, hi;          // keys lo .. hi - 1; none: INT_MAX, 0
  int pos;
  float slope2;        // slope log2(e)
};
// What that takes from memory: loaded without branches (any address, where there is
// no array), so that it can be under way while other rows are worked on.
struct RowLoads {
  int first, end;
  float slope;
  // (i and head in a uniform and a lane's part)
  __device__ __forceinline__ void ask(const WindowParams& a, const Seq& s, int i, int head, int lane_i = 0, int lane_h = 0) {
    first = (a.first_key ? a.first_key + s.r0 + i : a.cu_q)[a.first_key ? lane_i : 0];
    end = (a.end_key ? a.end_key + s.r0 + i : a.cu_q)[a.end_key ? lane_i : 0];
    slope = (a.slopes ? a.slopes + head : reinterpret_cast<const float*>(a.cu_q))[a.slopes ? lane_h : 0];
  }
  __device__ __forceinline__ RowInfo info(const WindowParams& a, const Seq& s, int i) const {
    RowInfo r;
    r.pos = s.L + i;
    r.lo = max(a.first_key ? max(first, 0) : 0, r.pos - a.window + 1);
    r.hi = min(a.end_key ? end : r.pos + 1, s.end);
    if (r.lo >= r.hi) {
      r.lo = INT_MAX;
      r.hi = 0;
    }
    r.slope2 = a.slopes ? slope * 1.44269504f : 0.f;
    return r;
  }
};
__device__ __forceinline__ RowInfo row_info(const WindowParams& a, const Seq& s, int i, int head) {
  RowLoads l;
  l.ask(a, s, i, head);
  return l.info(a, s, i);
}
// Window row of a packed row.
__device__ __forceinline__ int row_of(const WindowParams& a, int pr) { return a.log2g >= 0 ? pr >> a.log2g : pr / a.G; }
// Over the wave's rows: what some row sees, and what every row sees.
struct Span {
  int lo, hi, all_lo, all_hi;
  __device__ __forceinline__ bool sees(int t0) const { return t0 + kBlk > lo && t0 < hi; }
  __device__ __forceinline__ bool whole(int t0) const { return t0 >= all_lo && t0 + kBlk <= all_hi; }
};
template <int QT> __device__ __forceinline__ Span span_of(const RowInfo (&row)[QT]) {
  Span s{row[0].lo, row[0].hi, row[0].lo, row[0].hi};
#pragma unroll
  for (int t = 1; t < QT; ++t) {
    s.lo = min(s.lo, row[t].lo);
    s.hi = max(s.hi, row[t].hi);
    s.all_lo = max(s.all_lo, row[t].lo);
    s.all_hi = min(s.all_hi, row[t].hi);
  }
  // the lanes of a group of 16 hold the rows
  auto join = [](int v, auto op) {
    v = op(v, dpp_move_i<0x140>(v));
    v = op(v, dpp_move_i<0x141>(v));
    v = op(v, dpp_move_i<0x4E>(v));
    return uni(op(v, dpp_move_i<0xB1>(v)));
  };
  auto least = [](int x, int y) { return min(x, y); };
  auto most = [](int x, int y) { return max(x, y); };
  return {join(s.lo, least), join(s.hi, most), join(s.all_lo, most), join(s.all_hi, least)};
}

// (page, head) of the two 16-slot parts of a block, and where in the page they
// begin; entries are clamped into the pool.
struct Parts {
  int p0, p1;
  __device__ __forceinline__ void look_up(const WindowParams& a, ScalarInts pt, int t0, int g) {
    auto at = [&](int i) {
      return min(max(pt[min((t0 + 16 * i) >> a.log2ps, a.max_pages - 1)], 0), a.num_pages - 1) * a.Hkv + g;
    };
    p0 = at(0);
    p1 = at(1);
  }
  __device__ __forceinline__ unsigned of(int u) const {
    const int q0 = p0, q1 = p1;
    return (unsigned)(u ? q1 : q0);
  }
};

// ---- operands in registers ----
template <typename DT, int D> struct Frags;
template <int D> struct Frags<bf16, D> {
  bf16x8 k[2][D / 32];
  bf16x8 v[D / 16];
  __device__ __forceinline__ bf16x8 kf(int st, int ks) const { return k[st][ks]; }
  __device__ __forceinline__ bf16x8 vf(int dt) const { return v[dt]; }
};
template <int D> struct Frags<float, D> {
  floatx4 k[2][D / 16];       // lane group j: channels j D / 4 .. of a key
  floatx4 v[D / 16][2];
};

// NT: past the caches' order of use, for what one workgroup reads once: a stream of keys and values
// pushes out nothing else, and arrives at 5.5 TB/s instead of 5.0 (64 sequences of 1 to 8 Ki tokens,
// one row each, 230 to 208 us; 8 of 1 to 2 Ki 17.2 to 15.8).
template <bool NT, typename V, typename T> __device__ __forceinline__ V load16(const T* p) {
  return NT ? __builtin_nontemporal_load(reinterpret_cast<const V*>(p)) : ld16<V>(p);
}
template <typename DT, int D, bool NT = false>
__device__ __forceinline__ void load_keys(const WindowParams& a, Frags<DT, D>& f, int t0, const Parts& parts) {
  const int lane = lane_id(), c16 = lane & 15, j = lane >> 4, ps = 1 << a.log2ps;
  const int kgrp = 8 * (c16 >> 2);               // both sub-tiles' keys lie in one 16-slot part
  const int slot = ((t0 + (kgrp & 16)) & (ps - 1)) + (kgrp & 15) + (c16 & 3);
  const DT* base = reinterpret_cast<const DT*>(a.k_cache) + (size_t)parts.of(kgrp >> 4) * (unsigned)(ps * D);
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    if constexpr (sizeof(DT) == 2) {
#pragma unroll
      for (int ks = 0; ks < D / 32; ++ks) f.k[s][ks] = load16<NT, bf16x8>(base + (unsigned)((ks * ps + slot + 4 * s) * 32 + 8 * j));
    } else {
      const int d0 = j * (D / 4);
#pragma unroll
      for (int c = 0; c < D / 16; ++c)
        f.k[s][c] = load16<NT, floatx4>(base + (unsigned)((d0 / 32 * ps + slot + 4 * s) * 32 + (d0 & 31) + 4 * c));
    }
  }
}
template <typename DT, int D, bool NT = false>
__device__ __forceinline__ void load_values(const WindowParams& a, const void* v_cache, Frags<DT, D>& f, int t0, const Parts& parts) {
  const int lane = lane_id(), c16 = lane & 15, j = lane >> 4, ps = 1 << a.log2ps;
  const int slot = ((t0 + 16 * (j >> 1)) & (ps - 1)) + 8 * (j & 1);
  const DT* base = reinterpret_cast<const DT*>(v_cache) + (size_t)parts.of(j >> 1) * (unsigned)(ps * D);
#pragma unroll
  for (int dt = 0; dt < D / 16; ++dt) {
    const DT* p = base + (unsigned)((16 * dt + c16) * ps + slot);
    if constexpr (sizeof(DT) == 2) {
      f.v[dt] = load16<NT, bf16x8>(p);
    } else {
      f.v[dt][0] = load16<NT, floatx4>(p);
      f.v[dt][1] = load16<NT, floatx4>(p + 4);
    }
  }
}

// ---- one block ----
template <typename DT, int D, int QT> struct Queries;
template <int D, int QT> struct Queries<bf16, D, QT> { bf16x8 q[QT][D / 32]; };
template <int D, int QT> struct Queries<float, D, QT> { floatx4 q[QT][D / 16]; };

template <typename DT, int D, int QT, class F>
__device__ __forceinline__ void scores(const F& f, const Queries<DT, D, QT>& Q, floatx4 (&s)[QT][2]) {
#pragma unroll
  for (int t = 0; t < QT; ++t) s[t][0] = s[t][1] = floatx4{0.f, 0.f, 0.f, 0.f};
  if constexpr (sizeof(DT) == 2) {
#pragma unroll
    for (int ks = 0; ks < D / 32; ++ks)
#pragma unroll
      for (int st = 0; st < 2; ++st) {
        const bf16x8 k = f.kf(st, ks);
#pragma unroll
        for (int t = 0; t < QT; ++t) s[t][st] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, Q.q[t][ks], s[t][st], 0, 0, 0);
      }
  } else {
#pragma unroll
    for (int ks = 0; ks < D / 4; ++ks)
#pragma unroll
      for (int st = 0; st < 2; ++st)
#pragma unroll
        for (int t = 0; t < QT; ++t)
          s[t][st] = __builtin_amdgcn_mfma_f32_16x16x4f32(f.k[st][ks >> 2][ks & 3], Q.q[t][ks >> 2][ks & 3], s[t][st], 0, 0, 0);
  }
}

// tanh(z ln 2 / 2), to 8 2^-24 of itself: near 0 the series up to z^13 (1.8e-7 left out at the seam),
// else 1 - 2 / (2^z + 1).
__device__ __forceinline__ float tanh_of(float z) {
#pragma clang fp contract(off)                   // an fma of two constants holds one in a register of the callers' loops
  constexpr double h = 0.34657359027997264, h2 = h * h;
  const float z2 = z * z;
  float near = z2 * (float)(h * h2 * h2 * h2 * h2 * h2 * h2 * 21844. / 6081075.);
  near = near - (float)(h * h2 * h2 * h2 * h2 * h2 * 1382. / 155925.);
  near = fmaf(z2, near, (float)(h * h2 * h2 * h2 * h2 * 62. / 2835.));
  near = fmaf(z2, near, (float)(h * h2 * h2 * h2 * -17. / 315.));
  near = fmaf(z2, near, (float)(h * h2 * h2 * 2. / 15.));
  near = fmaf(z2, near, (float)(h * h2 * -1. / 3.));
  near = fmaf(z2, near, (float)h) * z;
  asm volatile("" : "+v"(near), "+v"(z));        // one after the other: the callers have no registers for both
  const float far = fmaf(__builtin_amdgcn_rcpf(fast_exp2(z) + 1.f), -2.f, 1.f);
  return fabsf(z) < 1.4426950f ? near : far;
}
// Caps (by log2(e)) up to which bf16 calls take 1 - 2 / (e^2y + 1) everywhere: off by 2^-22 of the cap
// near 0, 2e-5 in a score; with larger ones that would reach every probability (0.09 at a cap of 10^6).
constexpr float kNearCap = 64.f * 1.4426950408889634f;

// Raw products to modified scores in log2 units, plus a number per row.
template <typename DT, int QT>
__device__ __forceinline__ void modify(const WindowParams& a, const RowInfo (&row)[QT], const float (&plus)[QT], int k0, floatx4 (&s)[QT][2]) {
  if (sizeof(DT) == 2 && a.cap2 != 0.f && a.cap2 <= kNearCap) {
    // tanh x = 1 - 2 / (e^2x + 1): infinities give +-1
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      const float top = a.cap2 + plus[t];
#pragma unroll
      for (int i = 0; i < 8; ++i)
        s[t][i >> 2][i & 3] =
            fmaf(__builtin_amdgcn_rcpf(fast_exp2(s[t][i >> 2][i & 3] * a.scale2) + 1.f), -2.f * a.cap2, top);
    }
  } else if (a.cap2 != 0.f) {
#pragma unroll
    for (int t = 0; t < QT; ++t)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float x = s[t][i >> 2][i & 3];
        if constexpr (sizeof(DT) == 2) {
          s[t][i >> 2][i & 3] = fmaf(a.cap2, tanh_of(x * a.scale2), plus[t]);
          __builtin_amdgcn_sched_barrier(0);           // one after the other: no registers for more
        } else {
          s[t][i >> 2][i & 3] = fmaf(a.cap2, tanhf(x * a.cap_scale), plus[t]);
        }
      }
  } else {
#pragma unroll
    for (int t = 0; t < QT; ++t)
#pragma unroll
      for (int i = 0; i < 8; ++i) s[t][i >> 2][i & 3] = fmaf(s[t][i >> 2][i & 3], a.scale2, plus[t]);
  }
  if (a.slopes) {
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      const float d = (float)(row[t].pos - k0);
#pragma unroll
      for (int i = 0; i < 8; ++i)
        s[t][i >> 2][i & 3] = fmaf(-row[t].slope2, fabsf(d - (float)i), s[t][i >> 2][i & 3]);
    }
  }
}

}  // namespace
}  // namespace ipdv
