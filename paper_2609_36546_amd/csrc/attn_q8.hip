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
//   S^T[64 keys x 16 rows] = K . Q^T   v_mfma_f32_16x16x32_bf16, A = key rows
//   O^T[D x 16 rows] += V^T . P^T      A = value channels, B = P^T in place
//
// The keys' tile t has MFMA row 4 u + e at unit u, slot 4 t + e.  A lane (row
// c16, group j) then ends up with the scores of exactly the 16 slots of unit j,
// and a value load of 16 bytes, one channel's run of unit j, is its operand of
// two PV steps: P never leaves the lane.  Key channels are dealt to the k-steps
// the same way, 16 bytes of a key row at a time.
//
// Precision.  An e4m3 value times a power of two is exact in bf16, so keys and
// values enter the bf16 products without a rounding: the key's scale in the
// conversion, the value's in the probability.  Queries are bf16 already; fp32
// queries, and the fp32 call's probabilities, are split into three bf16 terms
// (24 bits), which makes their products exact to fp32 as well.  The bf16 call
// rounds its probabilities to bf16 once, as the bf16 cache's attention does.
// Sums and the running maximum are fp32.
//
// Work split.  All blocks of all items (an item: one row group of one
// (sequence, KV head)) form one line, cut into as many equal spans as there are
// workgroups, so that ragged contexts, single sequences and long prompts all
// fill the chip.  A workgroup's four waves are RG row groups x KS key parts: up
// to 64 rows KS = 4 (each wave its own keys, every byte read and converted
// once), more rows share their keys through the vector cache.  Items cut by a
// span's end leave partial results, merged by a second kernel.
#include <algorithm>

#include "common.h"
#include "kernels.h"
#include "q8.h"

namespace ipdv {
namespace {

constexpr int kBlk = 64;                // keys per block
constexpr float kRescaleSlack = 8.0f;   // log2 units a stale running max may lag

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
  long* head;          // [0] the line's length, then the first block of every item
  float* part_o;       // [2 * grid][item rows][D]
  float* part_ml;      // [2 * grid][item rows][2]: maximum, sum
  int max_pages, Hq, Hkv, G, log2ps, num_pages, n_seq, max_q;
  int n_rg;            // items per (sequence, KV head) at most
  int rg;              // row groups per workgroup: 1, 2 or 4
  float scale_log2;
};

typedef __attribute__((__vector_size__(2 * sizeof(__bf16)))) __bf16 bf16x2;

// Eight e4m3 values times 2^e, exact.
__device__ __forceinline__ bf16x8 cvt8(unsigned lo, unsigned hi, float scale) {
  const bf16x2 a = __builtin_bit_cast(bf16x2, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false));
  const bf16x2 b = __builtin_bit_cast(bf16x2, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true));
  const bf16x2 c = __builtin_bit_cast(bf16x2, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false));
  const bf16x2 d = __builtin_bit_cast(bf16x2, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true));
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// One block of 64 keys as a lane holds it.
template <int D> struct Block {
  uint4 k[4][D / 64];   // key tile t: 16 channels of one key per load
  uint4 v[D / 16];      // channel tile: one channel's 16 slots of unit j
  uint4 ks, vs;         // scale bytes: the lane's key unit (c16 / 4), its value unit (j)
};

template <int D>
__device__ __forceinline__ void load_block(const Q8Params& a, Block<D>& f, int t0, int g, const int* pt_row) {
  const int lane = lane_id(), c16 = lane & 15, j = lane >> 4;
  const int ps = 1 << a.log2ps;
  const int ku = t0 + 16 * (c16 >> 2), vu = t0 + 16 * j;
  const int kpg = min(max(pt_row[min(ku >> a.log2ps, a.max_pages - 1)], 0), a.num_pages - 1);
  const int vpg = min(max(pt_row[min(vu >> a.log2ps, a.max_pages - 1)], 0), a.num_pages - 1);
  const size_t kh = (size_t)kpg * a.Hkv + g, vh = (size_t)vpg * a.Hkv + g;
  const int ks0 = ku & (ps - 1), vs0 = vu & (ps - 1);
  const uint8_t* kb = a.k_pages + kh * D * ps + (size_t)(ks0 + (c16 & 3)) * 16;
#pragma unroll
  for (int h = 0; h < D / 64; ++h)
#pragma unroll
    for (int t = 0; t < 4; ++t) f.k[t][h] = ld16<uint4>(kb + ((4 * h + j) * ps + 4 * t) * 16);
  const uint8_t* vb = a.v_pages + vh * D * ps + vs0;
#pragma unroll
  for (int dt = 0; dt < D / 16; ++dt) f.v[dt] = ld16<uint4>(vb + (16 * dt + c16) * ps);
  f.ks = ld16<uint4>(a.scales + kh * 2 * ps + ks0);
  f.vs = ld16<uint4>(a.scales + vh * 2 * ps + ps + vs0);
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

template <int D, int QT, int NS> struct Queries { bf16x8 q[NS][QT][D / 32]; };

// TAIL: some row of the wave does not see every key of the block.
template <int D, int QT, int NS, bool TAIL>
__device__ __forceinline__ void attend(const Block<D>& f, const Queries<D, QT, NS>& Q, float c, int t0, int n_lim,
                                       const int (&qlimit)[QT], floatx4 (&acc)[QT][D / 16], float (&m_run)[QT],
                                       float (&l_run)[QT]) {
  const int lane = lane_id(), c16 = lane & 15, j = lane >> 4;
  floatx4 s[QT][4];
#pragma unroll
  for (int t = 0; t < 4; ++t) {
#pragma unroll
    for (int q = 0; q < QT; ++q) s[q][t] = floatx4{0.f, 0.f, 0.f, 0.f};
    const float ksc = __uint_as_float(((word(f.ks, t) >> (8 * (c16 & 3))) & 255u) << 23);
#pragma unroll
    for (int h = 0; h < D / 64; ++h)
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const bf16x8 kf = cvt8(x ? f.k[t][h].z : f.k[t][h].x, x ? f.k[t][h].w : f.k[t][h].y, ksc);
#pragma unroll
        for (int n = 0; n < NS; ++n)
#pragma unroll
          for (int q = 0; q < QT; ++q)
            s[q][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, Q.q[n][q][2 * h + x], s[q][t], 0, 0, 0);
      }
  }
  // s[q][t][e]: the lane's row of tile q against unit j, slot 4 t + e
  const int u0 = t0 + 16 * j;
  float bm[QT];
#pragma unroll
  for (int q = 0; q < QT; ++q) {
    bm[q] = -INFINITY;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      if (TAIL && u0 + i >= qlimit[q]) s[q][i >> 2][i & 3] = -INFINITY;
      bm[q] = fmaxf(bm[q], s[q][i >> 2][i & 3]);
    }
  }
#pragma unroll
  for (int q = 0; q < QT; ++q) bm[q] = fmaxf(bm[q], lane_xor16(bm[q]));
#pragma unroll
  for (int q = 0; q < QT; ++q) bm[q] = fmaxf(bm[q], lane_xor32(bm[q]));
  float m_use[QT];
  bool rescale = false;
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
#pragma unroll
  for (int st = 0; st < 2; ++st) {       // slots 8 st .. 8 st + 7 of unit j
    bf16x8 pf[NS][QT];
    float vsc[8];
#pragma unroll
    for (int i = 0; i < 8; ++i)
      vsc[i] = scale_value((word(f.vs, 2 * st + (i >> 2)) >> (8 * (i & 3))) & 255u);
#pragma unroll
    for (int q = 0; q < QT; ++q)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float p = fast_exp2(fmaf(s[q][2 * st + (i >> 2)][i & 3], c, -m_use[q]));
        l_run[q] += p;
        // an unseen key's scale may be anything, a later row's may be NaN
        float pv = p * vsc[i];
        if (TAIL && u0 + 8 * st + i >= qlimit[q]) pv = 0.f;
        __bf16 t[NS];
        split<NS>(pv, t);
#pragma unroll
        for (int n = 0; n < NS; ++n) pf[n][q][i] = t[n];
      }
#pragma unroll
    for (int dt = 0; dt < D / 16; ++dt) {
      unsigned lo = st ? f.v[dt].z : f.v[dt].x, hi = st ? f.v[dt].w : f.v[dt].y;
      if (TAIL) {                        // bytes behind the last key may be NaN
        const int live = n_lim - (u0 + 8 * st);
        lo = live >= 4 ? lo : live <= 0 ? 0u : lo & ((1u << (8 * live)) - 1u);
        hi = live >= 8 ? hi : live <= 4 ? 0u : hi & ((1u << (8 * (live - 4))) - 1u);
      }
      const bf16x8 vf = cvt8(lo, hi, 1.0f);
#pragma unroll
      for (int n = 0; n < NS; ++n)
#pragma unroll
        for (int q = 0; q < QT; ++q)
          acc[q][dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[n][q], acc[q][dt], 0, 0, 0);
    }
  }
}

// ---- the line of blocks ----

struct Seq {
  int b, L, r0, kb, rows, n_rg;
};
__device__ __forceinline__ Seq seq_of(const Q8Params& a, int slot, int item_rows) {
  Seq s;
  s.b = a.seq_ids ? a.seq_ids[slot] : slot;
  s.L = max(a.ctx_lens[s.b], 0);
  s.r0 = a.cu_q[s.b];
  s.kb = min(max(a.cu_q[s.b + 1] - s.r0, 0), a.max_q);
  s.rows = s.kb * a.G;
  s.n_rg = (s.rows + item_rows - 1) / item_rows;
  return s;
}
// Blocks of row group r: up to the last key that its last row sees.
__device__ __forceinline__ int item_blocks(const Q8Params& a, const Seq& s, int r, int item_rows) {
  const int last = min((r + 1) * item_rows, s.rows) - 1;
  return (s.L + last / a.G + kBlk) / kBlk;
}
__device__ __forceinline__ long head_blocks(const Q8Params& a, const Seq& s, int item_rows) {
  long n = 0;
  for (int r = 0; r < s.n_rg; ++r) n += item_blocks(a, s, r, item_rows);
  return n;
}
__device__ __forceinline__ long span_start(long total, long n, long w) { return w * total / n; }
// Spans in use: no more than there are groups of `parts` blocks.
__device__ __forceinline__ long spans(long total, int parts, int grid) {
  const long n = (total + parts - 1) / parts;
  return n < grid ? (n > 0 ? n : 1) : grid;
}

template <typename DT, int D, int QT>
__global__ __launch_bounds__(256) void attn_q8_kernel(Q8Params a) {
  constexpr int NS = sizeof(DT) == 2 ? 1 : 3;
  constexpr int WR = 16 * QT;                       // rows of a wave
  typedef floatx4 Acc[QT][D / 16][kWave];
  __shared__ __attribute__((aligned(16))) char s_acc[2 * sizeof(Acc)];
  __shared__ float s_ml[2][2][WR];
  __shared__ long s_sum[4];
  __shared__ long s_at[2];                          // the span's first slot, and its offset there
  const int tid = threadIdx.x, wv = tid >> 6, lane = lane_id();
  const int c16 = lane & 15, j = lane >> 4;
  const int RG = a.rg, KS = 4 / RG, rg = wv % RG, ks = wv / RG;
  const int item_rows = RG * WR;

  // Every workgroup adds up the whole line: a thread takes neighbouring slots.
  const int per = (a.n_seq + 255) / 256;
  const int sl0 = min(tid * per, a.n_seq), sl1 = min(sl0 + per, a.n_seq);
  long mine = 0;
  for (int i = sl0; i < sl1; ++i) mine += a.Hkv * head_blocks(a, seq_of(a, i, item_rows), item_rows);
  long incl = mine;
#pragma unroll
  for (int o = 1; o < kWave; o <<= 1) {
    const long up = __shfl_up(incl, o, kWave);
    if (lane >= o) incl += up;
  }
  if (lane == kWave - 1) s_sum[wv] = incl;
  __syncthreads();
  long before = 0, total = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (i < wv) before += s_sum[i];
    total += s_sum[i];
  }
  if (blockIdx.x == 0 && tid == 0) a.head[0] = total;
  const long n_span = spans(total, KS, gridDim.x);
  if (blockIdx.x >= n_span || total == 0) return;
  const long sp0 = span_start(total, n_span, blockIdx.x), sp1 = span_start(total, n_span, blockIdx.x + 1);
  {
    const long e0 = before + incl - mine;
    if (sp0 >= e0 && sp0 < e0 + mine) {
      long at = e0;
      for (int i = sl0; i < sl1; ++i) {
        const long n = a.Hkv * head_blocks(a, seq_of(a, i, item_rows), item_rows);
        if (sp0 < at + n) {
          s_at[0] = i;
          s_at[1] = at;
          break;
        }
        at += n;
      }
    }
  }
  __syncthreads();
  int slot = (int)s_at[0];
  long item0 = s_at[1];                             // the item's first block on the line
  Seq sq = seq_of(a, slot, item_rows);
  int g, r = 0;
  {
    const long hb = head_blocks(a, sq, item_rows);
    g = (int)((sp0 - item0) / hb);
    item0 += g * hb;
  }
  int nb = item_blocks(a, sq, 0, item_rows);
  while (item0 + nb <= sp0) {
    item0 += nb;
    nb = item_blocks(a, sq, ++r, item_rows);
  }

  for (long pos = sp0; pos < sp1;) {
    const int jb0 = (int)(pos - item0), jb1 = (int)min((long)nb, sp1 - item0);
    const bool whole = jb0 == 0 && jb1 == nb;
    if (jb0 == 0 && tid == 0) a.head[1 + ((long)slot * a.Hkv + g) * a.n_rg + r] = item0;
    // ---- the wave's rows and keys ----
    const int pr0 = r * item_rows + rg * WR;
    const int* pt_row = a.page_table + (size_t)sq.b * a.max_pages;
    int qlimit[QT];
#pragma unroll
    for (int q = 0; q < QT; ++q) qlimit[q] = sq.L + min(pr0 + 16 * q + c16, sq.rows - 1) / a.G + 1;
    const int n_keys = sq.L + (min(pr0 + WR, sq.rows) - 1) / a.G + 1;   // keys that some row sees
    const int all_see = sq.L + pr0 / a.G + 1;                     // keys below are seen by every row
    floatx4 acc[QT][D / 16];
    float m_run[QT], l_run[QT];
#pragma unroll
    for (int q = 0; q < QT; ++q) {
      m_run[q] = -INFINITY;
      l_run[q] = 0.f;
#pragma unroll
      for (int dt = 0; dt < D / 16; ++dt) acc[q][dt] = floatx4{0.f, 0.f, 0.f, 0.f};
    }
    if (pr0 < sq.rows) {
      Queries<D, QT, NS> Q;
#pragma unroll
      for (int q = 0; q < QT; ++q) {
        const int pr = pr0 + 16 * q + c16;
        const bool on = pr < sq.rows;
        const int i = on ? pr / a.G : 0, hl = on ? pr - i * a.G : 0;
        const DT* qr = reinterpret_cast<const DT*>(a.q) + (size_t)(sq.r0 + i) * a.q_stride + (size_t)(g * a.G + hl) * D;
#pragma unroll
        for (int x = 0; x < D / 32; ++x) {
          const DT* p = qr + 16 * (4 * (x >> 1) + j) + 8 * (x & 1);
          if constexpr (NS == 1) {
            Q.q[0][q][x] = ld16<bf16x8>(p);
          } else {
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
      const int part = (jb1 - jb0 + KS - 1) / KS;
      const int b0 = jb0 + ks * part;
      const int b1 = min(min(b0 + part, jb1), (n_keys + kBlk - 1) / kBlk);
      for (int n = b0; n < b1; ++n) {
        Block<D> f;
        load_block<D>(a, f, n * kBlk, g, pt_row);
        if ((n + 1) * kBlk <= all_see)
          attend<D, QT, NS, false>(f, Q, a.scale_log2, n * kBlk, n_keys, qlimit, acc, m_run, l_run);
        else
          attend<D, QT, NS, true>(f, Q, a.scale_log2, n * kBlk, n_keys, qlimit, acc, m_run, l_run);
      }
    }
#pragma unroll
    for (int q = 0; q < QT; ++q) {
      l_run[q] += lane_xor16(l_run[q]);
      l_run[q] += lane_xor32(l_run[q]);
    }
    // ---- the key parts of a row group, merged in halves ----
    for (int half = KS / 2; half > 0; half >>= 1) {
      if (ks >= half && ks < 2 * half) {
        Acc& buf = *reinterpret_cast<Acc*>(s_acc + ((ks - half) * RG + rg) * sizeof(Acc));
#pragma unroll
        for (int q = 0; q < QT; ++q) {
#pragma unroll
          for (int dt = 0; dt < D / 16; ++dt) buf[q][dt][lane] = acc[q][dt];
          if (j == 0) {
            s_ml[(ks - half) * RG + rg][0][16 * q + c16] = m_run[q];
            s_ml[(ks - half) * RG + rg][1][16 * q + c16] = l_run[q];
          }
        }
      }
      __syncthreads();
      if (ks < half) {
        const Acc& buf = *reinterpret_cast<const Acc*>(s_acc + (ks * RG + rg) * sizeof(Acc));
#pragma unroll
        for (int q = 0; q < QT; ++q) {
          const float m2 = s_ml[ks * RG + rg][0][16 * q + c16], l2 = s_ml[ks * RG + rg][1][16 * q + c16];
          const float m = fmaxf(m_run[q], m2), mu = m == -INFINITY ? 0.f : m;
          const float x = fast_exp2(m_run[q] - mu), y = fast_exp2(m2 - mu);
          m_run[q] = m;
          l_run[q] = l_run[q] * x + l2 * y;
#pragma unroll
          for (int dt = 0; dt < D / 16; ++dt) acc[q][dt] = acc[q][dt] * x + buf[q][dt][lane] * y;
        }
      }
      __syncthreads();
    }
    if (ks == 0) {
      const long ps = 2 * (long)blockIdx.x + (item0 >= sp0 ? 1 : 0);
#pragma unroll
      for (int q = 0; q < QT; ++q) {
        const int pr = pr0 + 16 * q + c16;
        if (pr >= sq.rows) continue;
        if (whole) {
          const int i = pr / a.G, hl = pr - i * a.G;
          DT* o = reinterpret_cast<DT*>(a.out) + ((size_t)(sq.r0 + i) * a.Hq + g * a.G + hl) * D + 4 * j;
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
          const size_t row = (size_t)ps * item_rows + rg * WR + 16 * q + c16;
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
    // ---- the next item ----
    pos = item0 + jb1;
    if (pos >= sp1) break;
    item0 += nb;
    if (++r == sq.n_rg) {
      r = 0;
      if (++g == a.Hkv) {
        g = 0;
        do {                                         // blocks are left, so a slot with rows follows
          if (++slot >= a.n_seq) return;
          sq = seq_of(a, slot, item_rows);
        } while (sq.n_rg == 0);
      }
    }
    nb = item_blocks(a, sq, r, item_rows);
  }
}

// Merges the partial results of an item that a span's end has cut.  A thread
// takes four channels of a row.
template <typename DT, int D>
__global__ __launch_bounds__(256) void attn_q8_combine_kernel(Q8Params a, int item_rows, int parts, int grid) {
  const int r = blockIdx.x, slot = blockIdx.y / a.Hkv, g = blockIdx.y % a.Hkv;
  const Seq sq = seq_of(a, slot, item_rows);
  if (r >= sq.n_rg) return;
  const long total = a.head[0];
  const long n_span = spans(total, parts, grid);
  const long s0 = a.head[1 + ((long)slot * a.Hkv + g) * a.n_rg + r];
  const long s1 = s0 + item_blocks(a, sq, r, item_rows);
  const long w0 = ((s0 + 1) * n_span - 1) / total, w1 = (s1 * n_span - 1) / total;
  if (w0 == w1) return;
  const long first = 2 * w0 + 1;                     // w0 holds the item's start, the others continue it
  const int rows = min(item_rows, sq.rows - r * item_rows);
  for (int e = threadIdx.x; e < rows * (D / 4); e += 256) {
    const int row = e / (D / 4), d = 4 * (e % (D / 4));
    float m = -INFINITY;
    for (long w = w0; w <= w1; ++w)
      m = fmaxf(m, a.part_ml[2 * ((size_t)(w == w0 ? first : 2 * w) * item_rows + row)]);
    floatx4 o = {0.f, 0.f, 0.f, 0.f};
    float l = 0.f;
    const float mu = m == -INFINITY ? 0.f : m;
    for (long w = w0; w <= w1; ++w) {
      const size_t at = (size_t)(w == w0 ? first : 2 * w) * item_rows + row;
      const float x = fast_exp2(a.part_ml[2 * at] - mu);
      l += x * a.part_ml[2 * at + 1];
      o += x * ld16<floatx4>(a.part_o + at * D + d);
    }
    const int pr = r * item_rows + row, i = pr / a.G, hl = pr - i * a.G;
    DT* out = reinterpret_cast<DT*>(a.out) + ((size_t)(sq.r0 + i) * a.Hq + g * a.G + hl) * D + d;
    const float inv = 1.f / l;
#pragma unroll
    for (int c = 0; c < 4; ++c) out[c] = from_f32<DT>(o[c] * inv);
  }
}

struct Q8Plan {
  int qt, rg, n_rg, grid;
};
Q8Plan plan_of(int n_seq, int Hq, int Hkv, int max_q, bool bf16) {
  Q8Plan p;
  const long rows = (long)max_q * (Hq / Hkv);
  if (bf16) {
    p.qt = rows <= 16 ? 1 : rows <= 32 ? 2 : 4;
    p.rg = rows <= 64 ? 1 : rows <= 128 ? 2 : 4;
  } else {                      // three terms per query: fewer rows fit the registers
    p.qt = rows <= 16 ? 1 : 2;
    p.rg = rows <= 32 ? 1 : rows <= 64 ? 2 : 4;
  }
  const int item = 16 * p.qt * p.rg;
  p.n_rg = (int)((rows + item - 1) / item);
  p.grid = device_cus();
  return p;
}

}  // namespace

size_t attn_q8_workspace(int n_seq, int Hq, int Hkv, int D, int max_q) {
  size_t most = 0;              // either type
  for (const bool b : {false, true}) {
    const Q8Plan p = plan_of(n_seq, Hq, Hkv, max_q, b);
    const size_t rows = 2 * (size_t)p.grid * 16 * p.qt * p.rg;
    const size_t n = rows * (D + 2) * 4 + 8 * (1 + (size_t)n_seq * Hkv * p.n_rg);
    most = std::max(most, (n + 255) / 256 * 256);
  }
  return most;
}

hipError_t launch_attn_q8(const AttnQ8Launch& L, hipStream_t st) {
  const Q8Plan pl = plan_of(L.n_seq, L.Hq, L.Hkv, L.max_q, L.dtype_bf16);
  const int item_rows = 16 * pl.qt * pl.rg;
  const size_t rows = 2 * (size_t)pl.grid * item_rows;
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
  p.head = (long*)(p.part_ml + 2 * rows);
  p.max_pages = L.max_pages;
  p.Hq = L.Hq;
  p.Hkv = L.Hkv;
  p.G = L.Hq / L.Hkv;
  p.log2ps = __builtin_ctz(L.page_size);
  p.num_pages = L.num_pages;
  p.n_seq = L.n_seq;
  p.max_q = L.max_q;
  p.n_rg = pl.n_rg;
  p.rg = pl.rg;
  p.scale_log2 = L.scale * 1.4426950408889634f;
  trace_begin(st);
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(pl.grid), dim3(256), 0, st, p); };
  if (L.dtype_bf16) {
    if (L.D == 128) {
      if (pl.qt == 1) go(attn_q8_kernel<bf16, 128, 1>);
      else if (pl.qt == 2) go(attn_q8_kernel<bf16, 128, 2>);
      else go(attn_q8_kernel<bf16, 128, 4>);
    } else {
      if (pl.qt == 1) go(attn_q8_kernel<bf16, 64, 1>);
      else if (pl.qt == 2) go(attn_q8_kernel<bf16, 64, 2>);
      else go(attn_q8_kernel<bf16, 64, 4>);
    }
  } else {
    if (L.D == 128) {
      if (pl.qt == 1) go(attn_q8_kernel<float, 128, 1>); else go(attn_q8_kernel<float, 128, 2>);
    } else {
      if (pl.qt == 1) go(attn_q8_kernel<float, 64, 1>); else go(attn_q8_kernel<float, 64, 2>);
    }
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  trace_mark(st);
  const dim3 cgrid(pl.n_rg, L.n_seq * L.Hkv);
  auto merge = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, cgrid, dim3(256), 0, st, p, item_rows, 4 / pl.rg, pl.grid);
  };
  if (L.dtype_bf16) {
    if (L.D == 128) merge(attn_q8_combine_kernel<bf16, 128>); else merge(attn_q8_combine_kernel<bf16, 64>);
  } else {
    if (L.D == 128) merge(attn_q8_combine_kernel<float, 128>); else merge(attn_q8_combine_kernel<float, 64>);
  }
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  trace_mark(st);
  return hipSuccess;
}

}  // namespace ipdv
