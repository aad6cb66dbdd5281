// The attention weight that every cached key gathers from a window, for gfx950:
//
//   mass[j] = decay mass[j] + sum over rows i and heads h of the KV head of e^(x_ihj - lse_ih)
//
// with x the modified scores and lse their log-sum-exp, as attn_masked.hip has them;
// keys of the window itself start at 0.  With lse in hand a weight needs nothing
// of the row's other keys, so every key's sum belongs to one workgroup: no atomics,
// no partial results, the same bits every time.
//
// Scores are taken as there, S^T[32 keys x 16 rows] = K . Q^T, a lane holding 8 keys of
// one row.  Up to 64 rows (attn_mass_few_kernel) a wave keeps all of them and streams keys; with
// more (attn_mass_many_kernel) it keeps one or two blocks of keys and streams rows, with many
// the 8 waves of a workgroup every 8th tile of them.  Weights are added per lane, over the rows of
// a lane's column, and joined over the 16 columns at the end.
#include <algorithm>
#include <type_traits>

#include "common.h"
#include "kernels.h"
#include "masked.h"

namespace ipdv {
namespace {

constexpr int kWaves = 4;

struct MassParams : WindowParams {
  const float* lse;
  const float* mass_in;
  float* mass_out;
  float decay;
  int per;             // blocks of a workgroup
};

// Sum over the 16 lanes of a group that share a key.
__device__ __forceinline__ float sum16(float v) {
  v += dpp_move<0x140>(v);
  v += dpp_move<0x141>(v);
  v += dpp_move<0x4E>(v);
  return v + dpp_move<0xB1>(v);
}

// Lane 8 j + i (i < 8, of the groups j of 16: lane 16 j + i) writes key t0 + 8 j + i.
__device__ __forceinline__ void put(const MassParams& a, const Seq& s, const Parts& parts, int t0, float sum) {
  const int lane = lane_id(), c16 = lane & 15, j = lane >> 4, key = t0 + 8 * j + c16;
  if (c16 >= 8 || key >= s.end) return;
  const int ps = 1 << a.log2ps;
  const size_t at = (size_t)parts.of(j >> 1) * (unsigned)ps + (unsigned)(key & (ps - 1));
  if (a.mass_in && key < s.L) sum = fmaf(a.decay, a.mass_in[at], sum);
  a.mass_out[at] = sum;
}

// Queries and what else belongs to the lane's row of a tile.
template <typename DT, int D, int QT> struct RowTile {
  Queries<DT, D, QT> Q;
  RowLoads raw[QT];
  float lse[QT];
  RowInfo row[QT];
  float less_lse2[QT]; // -lse log2(e)
  int at[QT];          // window row
  // Asked for; `arrive` makes them what the rest works with.  Behind the last row its copies.
  // Where G is a power of two a whole tile's addresses are a uniform base and an offset that
  // the lane has in every tile (a product of 64 bits costs as much as a score).
  template <bool QUERIES = true>
  __device__ __forceinline__ void ask(const MassParams& a, const Seq& s, int g, int t, int pr0) {
    const int lane = lane_id(), c16 = lane & 15, j = lane >> 4;
    const DT* q = reinterpret_cast<const DT*>(a.q);
    if (a.log2g >= 0 && pr0 + 16 <= s.rows) {
      const int i = pr0 >> a.log2g, h = g * a.G + (pr0 & (a.G - 1)), li = c16 >> a.log2g, lh = c16 & (a.G - 1);
      at[t] = i + li;
      raw[t].ask(a, s, i, h, li, lh);
      lse[t] = (a.lse + (size_t)(s.r0 + i) * a.Hq + h)[li * a.Hq + lh];
      if (QUERIES) load_row(t, q + (size_t)(s.r0 + i) * a.q_stride + (size_t)h * D + ((size_t)li * a.q_stride + lh * D), j);
    } else {
      const int pr = min(pr0 + c16, s.rows - 1), i = row_of(a, pr), h = g * a.G + pr - i * a.G;
      at[t] = i;
      raw[t].ask(a, s, i, h);
      lse[t] = a.lse[(size_t)(s.r0 + i) * a.Hq + h];
      if (QUERIES) load_row(t, q + (size_t)(s.r0 + i) * a.q_stride + (size_t)h * D, j);
    }
  }
  __device__ __forceinline__ void load_row(int t, const DT* qr, int j) {
    if constexpr (sizeof(DT) == 2) {
#pragma unroll
      for (int ks = 0; ks < D / 32; ++ks) Q.q[t][ks] = ld16<bf16x8>(qr + 32 * ks + 8 * j);
    } else {
#pragma unroll
      for (int c = 0; c < D / 16; ++c) Q.q[t][c] = ld16<floatx4>(qr + j * (D / 4) + 4 * c);
    }
  }
  __device__ __forceinline__ void arrive(const MassParams& a, const Seq& s, int t, int pr0) {
    row[t] = raw[t].info(a, s, at[t]);
    less_lse2[t] = pr0 + (lane_id() & 15) < s.rows ? lse[t] * -1.4426950408889634f : -INFINITY;      // copies: of weight 0
  }
  // Adds the tiles' weights of a block's keys.
  __device__ __forceinline__ void add(const MassParams& a, floatx4 (&sc)[QT][2], int t0, bool masked, float (&sum)[8]) const {
    const int k0 = t0 + 8 * (lane_id() >> 4);
    modify<DT, QT>(a, row, less_lse2, k0, sc);
#pragma unroll
    for (int t = 0; t < QT; ++t)
#pragma unroll
      for (int i = 0; i < 8; ++i) sc[t][i >> 2][i & 3] = fast_exp2(sc[t][i >> 2][i & 3]);
    if (masked) {
      asm volatile("");             // a branch: most blocks do without the comparisons
#pragma unroll
      for (int t = 0; t < QT; ++t)
#pragma unroll
        for (int i = 0; i < 8; ++i)
          sc[t][i >> 2][i & 3] = k0 + i >= row[t].lo && k0 + i < row[t].hi ? sc[t][i >> 2][i & 3] : 0.f;
    }
#pragma unroll
    for (int t = 0; t < QT; ++t)
#pragma unroll
      for (int i = 0; i < 8; ++i) sum[i] += sc[t][i >> 2][i & 3];
  }
};

// One of the lane's eight sums, the one that it writes.
__device__ __forceinline__ float pick(const float (&sum)[8]) {
  const int c16 = lane_id() & 15;
  float out = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float v = sum16(sum[i]);
    out = c16 == i ? v : out;
  }
  return out;
}

// The queries of four tiles lie in LDS: in registers they leave room for two waves per SIMD instead
// of four, and each wave would load them all (64 windows of eight by 1 to 8 Ki keys, 64 packed rows:
// 90 us so, 80 from LDS).  Keys, read once, are a stream.
template <typename DT, int D, int QT>
__global__ __launch_bounds__(256, QT == 4 ? 4 : sizeof(DT) == 4 ? 1 : 2) void attn_mass_few_kernel(MassParams a) {
  constexpr bool LDS = QT == 4;
  static_assert(!LDS || (sizeof(DT) == 2 && QT == kWaves), "a tile of a wave");
  __shared__ bf16x8 s_q[LDS ? QT : 1][LDS ? D / 32 : 1][kWave];
  const int sg = slot_head_of(a, blockIdx.x, blockIdx.y, gridDim.x);
  if (sg < 0) return;
  const int slot = sg / a.Hkv, g = sg - slot * a.Hkv;
  const Seq s = seq_of(a, slot);
  const int b0 = blockIdx.y * a.per, b1 = min(b0 + a.per, (s.end + kBlk - 1) / kBlk);
  if (b0 >= b1) return;
  const int wv = uni(threadIdx.x / kWave), first = b0 + wv;
  RowTile<DT, D, QT> R;
  Span span{INT_MAX, 0, INT_MAX, 0};
  if (s.rows > 0) {
    if constexpr (LDS) {
      RowTile<DT, D, 1> mine;
      mine.ask(a, s, g, 0, 16 * wv);
#pragma unroll
      for (int ks = 0; ks < D / 32; ++ks) s_q[wv][ks][lane_id()] = mine.Q.q[0][ks];
    }
#pragma unroll
    for (int t = 0; t < QT; ++t) R.template ask<!LDS>(a, s, g, t, 16 * t);
#pragma unroll
    for (int t = 0; t < QT; ++t) R.arrive(a, s, t, 16 * t);
    span = span_of<QT>(R.row);
  }
  if (LDS) __syncthreads();
  if (first >= b1) return;
  const ScalarInts pt = scalar(a.page_table + (size_t)s.b * a.max_pages);
  Parts parts, next;
  parts.look_up(a, pt, first * kBlk, g);
  Frags<DT, D> f;
  if (span.sees(first * kBlk)) load_keys<DT, D, true>(a, f, first * kBlk, parts);
  next.look_up(a, pt, (first + kWaves) * kBlk, g);
  for (int n = first; n < b1; n += kWaves) {
    const int t0 = n * kBlk;
    float sum[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    const bool seen = span.sees(t0);
    floatx4 sc[QT][2];
    if (seen) {
      if constexpr (LDS) {
        asm volatile("" ::: "memory");           // read anew: there are no registers to keep them
#pragma unroll
        for (int t = 0; t < QT; ++t) sc[t][0] = sc[t][1] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int ks = 0; ks < D / 32; ++ks)
#pragma unroll
          for (int t = 0; t < QT; ++t) {
            const bf16x8 q = s_q[t][ks][lane_id()];
#pragma unroll
            for (int st = 0; st < 2; ++st) sc[t][st] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f.kf(st, ks), q, sc[t][st], 0, 0, 0);
          }
      } else {
        scores<DT, D, QT>(f, R.Q, sc);
      }
    }
    __builtin_amdgcn_sched_barrier(0);
    if (n + kWaves < b1 && span.sees(t0 + kWaves * kBlk)) load_keys<DT, D, true>(a, f, t0 + kWaves * kBlk, next);
    __builtin_amdgcn_sched_barrier(0);
    if (seen) R.add(a, sc, t0, !span.whole(t0), sum);
    put(a, s, parts, t0, pick(sum));
    parts = next;
    next.look_up(a, pt, t0 + 2 * kWaves * kBlk, g);
  }
}

// RS of W waves share NB blocks of keys and take every RS-th tile of rows; the others have
// blocks of their own.  PLAIN: without ranges and slopes, so nothing is loaded for them; in bf16 that
// leaves room for three waves per SIMD (with two, 24 windows of 32, 64 and 100 rows take 43, 73 and 107
// us, so 35, 59 and 86).
template <typename DT, int D, int NB, int RS, int W, bool PLAIN>
__global__ __launch_bounds__(64 * W, RS > 1 ? 1 : PLAIN && sizeof(DT) == 2 ? 3 : 2) void attn_mass_many_kernel(MassParams a) {
  if constexpr (PLAIN) {
    a.first_key = a.end_key = nullptr;
    a.slopes = nullptr;
  }
  constexpr int KS = W / RS;
  __shared__ float s_sum[W][NB][kBlk];
  const int by = blockIdx.z * gridDim.y + blockIdx.y;
  const int sg = slot_head_of(a, blockIdx.x, by, gridDim.x);
  if (sg < 0) return;
  const int slot = sg / a.Hkv, g = sg - slot * a.Hkv;
  const Seq s = seq_of(a, slot);
  const int wv = uni(threadIdx.x / kWave), rs = wv % RS;
  // the first keys, which most rows see, first
  const int t0 = (by * KS + wv / RS) * NB * kBlk;
  if (by * KS * NB * kBlk >= s.end) return;
  const ScalarInts pt = scalar(a.page_table + (size_t)s.b * a.max_pages);
  float sum[NB][8];
#pragma unroll
  for (int n = 0; n < NB; ++n)
#pragma unroll
    for (int i = 0; i < 8; ++i) sum[n][i] = 0.f;
  // rows in front see none of these keys, unless their ranges' ends are given
  const int row0 = a.end_key ? 0 : max(t0 - s.L, 0) * a.G;
  // nor rows that these keys lie in front of the sliding window of
  const long last = (long)t0 + NB * kBlk - 1 + a.window - 1 - s.L;      // the last position that may, counted from L
  const int rows = t0 < s.end ? (int)max(min((long)s.rows, (last + 1) * a.G), 0l) : 0;
  const int tiles = (rows + 15) / 16;
  int tile = row0 / 16 + rs;
  if (tile < tiles) {
    Frags<DT, D> f[NB];
#pragma unroll
    for (int n = 0; n < NB; ++n) {
      Parts parts;
      parts.look_up(a, pt, t0 + n * kBlk, g);
      load_keys<DT, D>(a, f[n], t0 + n * kBlk, parts);
    }
    // two tiles in turn: one is asked for while the other is worked on
    RowTile<DT, D, 1> R[2];
    auto work = [&](RowTile<DT, D, 1>& r, int at) __attribute__((always_inline)) {
      r.arrive(a, s, 0, 16 * at);
#pragma unroll
      for (int n = 0; n < NB; ++n) {
        const int tn = t0 + n * kBlk;
        if (__any(r.row[0].lo < tn + kBlk && r.row[0].hi > tn)) {
          floatx4 sc[1][2];
          scores<DT, D, 1>(f[n], r.Q, sc);
          r.add(a, sc, tn, !__all(r.row[0].lo <= tn && r.row[0].hi >= tn + kBlk), sum[n]);
        }
      }
    };
    R[0].ask(a, s, g, 0, 16 * tile);
    for (;;) {
      R[1].ask(a, s, g, 0, 16 * (tile + RS));     // behind the last tile: its last row, not used
      __builtin_amdgcn_sched_barrier(0);
      work(R[0], tile);
      if ((tile += RS) >= tiles) break;
      __builtin_amdgcn_sched_barrier(0);
      R[0].ask(a, s, g, 0, 16 * (tile + RS));
      __builtin_amdgcn_sched_barrier(0);
      work(R[1], tile);
      if ((tile += RS) >= tiles) break;
      __builtin_amdgcn_sched_barrier(0);
    }
  }
#pragma unroll
  for (int n = 0; n < NB; ++n) {
    float v = pick(sum[n]);
    const int lane = lane_id(), c16 = lane & 15, j = lane >> 4;
    if constexpr (RS > 1) {
      if (c16 < 8) s_sum[wv][n][8 * j + c16] = v;
      __syncthreads();
      if (rs != n % RS) continue;
      v = 0.f;
      if (c16 < 8)
#pragma unroll
        for (int i = 0; i < RS; ++i) v += s_sum[wv - rs + i][n][8 * j + c16];
    }
    Parts parts;
    parts.look_up(a, pt, t0 + n * kBlk, g);
    put(a, s, parts, t0 + n * kBlk, v);
  }
}

}  // namespace

hipError_t launch_attn_mass(const AttnMaskedLaunch& L, hipStream_t st) {
  MassParams p{};
  static_cast<WindowParams&>(p) = window_params(L);
  p.lse = L.lse;
  p.mass_in = L.mass_in;
  p.mass_out = L.mass_out;
  p.decay = L.decay;
  const long rows = (long)L.max_q * p.G, sg = (long)L.n_seq * L.Hkv;
  const long blocks = ((long)p.slots + kBlk - 1) / kBlk;
  const unsigned gx = (unsigned)((sg + 7) / 8 * 8);
  // 64 windows by 1 to 8 Ki keys: of one row 130 us at 32 blocks of a workgroup, 123 at 8 (112 since
  // keys are a stream); of eight (64 packed rows) 83 at either, 80 at 16
  p.per = (int)std::max(std::clamp(sg * blocks / 2048, 4L, rows <= 16 ? 8L : 16L), (blocks + 65534) / 65535);
  trace_begin(st);
  auto pick = [&](auto dt, auto dim) {
    using DT = decltype(dt);
    constexpr int D = decltype(dim)::value;
    auto few = [&](auto kernel) {
      hipLaunchKernelGGL(kernel, dim3(gx, (unsigned)((blocks + p.per - 1) / p.per)), dim3(256), 0, st, p);
    };
    if (rows <= 16) few(attn_mass_few_kernel<DT, D, 1>);
    else if (rows <= 32) few(attn_mass_few_kernel<DT, D, 2>);
    else if (rows <= 64 && sizeof(DT) == 2) {
      if constexpr (sizeof(DT) == 2) few(attn_mass_few_kernel<DT, D, 4>);
    } else {
      auto many = [&](auto kernel, int at_once, int waves) {
        const long ny = (blocks + at_once - 1) / at_once, nz = (ny + 65534) / 65535;
        hipLaunchKernelGGL(kernel, dim3(gx, (unsigned)((ny + nz - 1) / nz), (unsigned)nz), dim3(64 * waves), 0, st, p);
      };
      // two blocks per pass over a bf16 row: 24 windows of 64 rows 98 to 58 us; fp32, which the
      // products bound, has more of waves of one
      constexpr int NB = sizeof(DT) == 4 ? 1 : 2;
      // Waves share blocks where there are too few for all, or the first keys' waves, which have
      // every row, would end last (4 KV heads, G = 8: 8 prompts of 512 to 1024 tokens 358 to 75 us,
      // 64 of them 535 to 442; 24 windows of 100 rows by 500 to 3000 keys take 136 us so, and 85
      // by waves of their own; 16 by 256 to 512 keys 31 and 34).
      const bool shared = rows > 512 && (rows > 4096 || sg * ((blocks + NB - 1) / NB) < 4096);
      const bool plain = !p.first_key && !p.end_key && !p.slopes;
      if (!shared && plain) many(attn_mass_many_kernel<DT, D, NB, 1, 4, true>, 4 * NB, 4);
      else if (!shared) many(attn_mass_many_kernel<DT, D, NB, 1, 4, false>, 4 * NB, 4);
      else if (plain) many(attn_mass_many_kernel<DT, D, NB, 8, 8, true>, NB, 8);
      else many(attn_mass_many_kernel<DT, D, NB, 8, 8, false>, NB, 8);
    }
  };
  typedef std::integral_constant<int, 64> D64;
  typedef std::integral_constant<int, 128> D128;
  if (L.dtype_bf16) {
    if (L.D == 128) pick(bf16(), D128()); else pick(bf16(), D64());
  } else {
    if (L.D == 128) pick(float(), D128()); else pick(float(), D64());
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  trace_mark(st);
  return hipSuccess;
}

}  // namespace ipdv
