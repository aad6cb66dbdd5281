// Attention over the paged cache with the score's modifiers, for gfx950: grouped-
// query attention of every window row over the keys that its range leaves it,
// scores capped by a tanh and biased by distance.
//
//   x_j = scale q.K_j;  x_j = cap tanh(x_j / cap);  x_j -= slope |p - j|
//   out = sum_j e^(x_j - m) V_j / sum_j e^(x_j - m),  first <= j < end;  lse = ln sum_j e^(x_j)
//
// in one pass over the keys with a running maximum m and sum per row, in base 2.
//
// Tiles.  The query rows of one (sequence, KV head), k positions x G heads, are
// packed position-major into tiles of 16, and a wave walks blocks of 32 keys:
//
//   S^T[32 keys x 16 rows] = K . Q^T     v_mfma_f32_16x16x32_bf16 (fp32: 16x16x4), A = key rows
//   O^T[D x 16 rows] += V^T . P^T        A = the channel-major value rows, B = P^T in place
//
// with MFMA row r of sub-tile s dealt key 8 (r / 4) + 4 s + r % 4, so that a lane
// ends up with the 8 neighbouring keys that its operand of the second product needs.
//
// Masks.  A row's range [first, end) is a pair of bounds in its lane.  A wave knows
// the union of its rows' ranges, which it walks, and their intersection: blocks
// inside it need no mask.  In the others a value that is not finite must not reach
// rows that do not see it, and a probability of zero does not keep it out.  So sums that have
// become not finite are taken anew, from the first key, with such values taken out and NaN
// for the rows that see them.  (A branch inside the walk would cost it a copy of the sums: 163
// registers instead of 96 with one tile per wave.)
//
// Work split.  A workgroup takes a piece of the keys of one row tile; tiles of
// a window that has few are cut into more pieces (split_of), joined by a second
// kernel.  Up to 16 rows, and in fp32, its waves walk keys of their own, in registers
// (masked_keys_kernel); with more rows the four hold 16 or 32 rows each and share the
// keys through a ring in LDS (masked_tile_kernel).
#include <algorithm>
#include <type_traits>

#include "common.h"
#include "kernels.h"
#include "masked.h"

namespace ipdv {
namespace {

constexpr int kWaves = 4;
constexpr int kStageValues = 128;       // QT x D up to which there are registers for a block's values
constexpr float kRescaleSlack = 8.0f;   // log2 units a stale running max may lag
constexpr float kLn2 = 0.69314718055994531f;

struct MaskedParams : WindowParams {
  const void* k_new;   // the window's rows, where the attention appends them itself (else null)
  const void* v_new;
  void* v_cache;
  void* out;
  float* lse;
  float* part_o;       // [n_seq * Hkv][units][tile rows][D]
  float2* part_ml;     // [n_seq * Hkv][units][tile rows]: maximum, sum
  int32_t* pieces;     // [n_seq * Hkv][tiles]: pieces of a tile
  int tiles, units;    // row tiles, and tiles x pieces, of a (sequence, head) at most
  int per, walk;       // blocks of a piece at least: per tile of the window, in all
};

// Pieces that a window's tiles are cut into, `np` of `per` blocks each (a tile with
// a shorter range has fewer): a window of many tiles brings as many workgroups by
// itself, and each piece costs it a partial result of all its rows.
struct Split {
  int nt, np, per;
};
__device__ __forceinline__ Split split_of(const MaskedParams& a, const Seq& s, int tile_rows) {
  Split p;
  p.nt = (s.rows + tile_rows - 1) / tile_rows;
  // blocks of a tile at most: up to the window's end, or of the sliding window of
  // the tile's positions (which a range's end may lie behind, if it is given)
  long nb = (s.end + kBlk - 1) / kBlk;
  if (!a.end_key) nb = min(nb, ((long)a.window + tile_rows / a.G + 1 + 2 * kBlk) / kBlk);
  p.per = max(a.per * p.nt, a.walk);
  p.np = (int)((nb + p.per - 1) / p.per);
  return p;
}

// What a wave holds of 16 QT rows while it walks their keys.
template <typename DT, int D, int QT, int PT>
struct Rows {
  floatx4 acc[QT][D / 16];
  float m[QT], l[QT];
  Queries<DT, D, QT> Q;
  RowInfo row[QT];

  __device__ __forceinline__ void begin(const MaskedParams& a, const Seq& s, int g, int pr0, int pr_last) {
    const int lane = lane_id(), c16 = lane & 15, j = lane >> 4;
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      const int pr = min(pr0 + 16 * t + c16, pr_last), i = row_of(a, pr), h = g * a.G + pr - i * a.G;   // behind the last: its copies
      row[t] = row_info(a, s, i, h);
      const DT* qr = reinterpret_cast<const DT*>(a.q) + (size_t)(s.r0 + i) * a.q_stride + (size_t)h * D;
      if constexpr (sizeof(DT) == 2) {
#pragma unroll
        for (int ks = 0; ks < D / 32; ++ks) Q.q[t][ks] = ld16<bf16x8>(qr + 32 * ks + 8 * j);
      } else {
#pragma unroll
        for (int c = 0; c < D / 16; ++c) Q.q[t][c] = ld16<floatx4>(qr + j * (D / 4) + 4 * c);
      }
    }
  }
  // The queries are here from now on: the compiler counts its own loads only, and would wait for
  // them inside the walk, with others under way.
  __device__ __forceinline__ void queries_here() {
#pragma unroll
    for (int t = 0; t < QT; ++t)
#pragma unroll
      for (int ks = 0; ks < (int)(sizeof(Q.q[0]) / 16); ++ks) asm volatile("" : "+v"(Q.q[t][ks]));
  }

  __device__ __forceinline__ void reset() {
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      m[t] = -INFINITY;
      l[t] = 0.f;
#pragma unroll
      for (int dt = 0; dt < D / 16; ++dt) acc[t][dt] = floatx4{0.f, 0.f, 0.f, 0.f};
    }
  }
  // Whether some sum of this lane is not finite.
  __device__ __forceinline__ bool odd() const {
    float x = 0.f;
#pragma unroll
    for (int t = 0; t < QT; ++t)
#pragma unroll
      for (int dt = 0; dt < D / 16; ++dt)
#pragma unroll
        for (int e = 0; e < 4; ++e) x = fmaf(acc[t][dt][e], 0.f, x);
    return x != x;
  }

  // One block.  `masked`: some row does not see all of it.  CAREFUL: its values may be not finite.
  template <bool CAREFUL, class F>
  __device__ __forceinline__ void block(const MaskedParams& a, const F& f, int t0, bool masked) {
    floatx4 s[QT][2];
    scores<DT, D, QT>(f, Q, s);
    if constexpr (QT * D <= kStageValues) {      // asked for before the softmax: LDS takes its time
      Frags<DT, D> r;
#pragma unroll
      for (int dt = 0; dt < D / 16; ++dt) r.v[dt] = f.vf(dt);
      __builtin_amdgcn_sched_barrier(0);
      weigh<CAREFUL>(a, r, s, t0, masked);
    } else {                           // no registers for them
      weigh<CAREFUL>(a, f, s, t0, masked);
    }
  }
  template <bool CAREFUL, class F>
  __device__ __forceinline__ void weigh(const MaskedParams& a, const F& f, floatx4 (&s)[QT][2], int t0, bool masked) {
    const int k0 = t0 + 8 * (lane_id() >> 4);         // the lane's first key
    const float none[QT] = {};
    modify<DT, QT>(a, row, none, k0, s);
    if (masked) {
      asm volatile("");                // a branch: else every block is masked
#pragma unroll
      for (int t = 0; t < QT; ++t)
#pragma unroll
        for (int i = 0; i < 8; ++i)
          s[t][i >> 2][i & 3] = k0 + i >= row[t].lo && k0 + i < row[t].hi ? s[t][i >> 2][i & 3] : -INFINITY;
    }
    float bm[QT], m_use[QT];
    bool rescale = false;
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      bm[t] = -INFINITY;
#pragma unroll
      for (int i = 0; i < 8; ++i) bm[t] = fmaxf(bm[t], s[t][i >> 2][i & 3]);
    }
#pragma unroll
    for (int t = 0; t < QT; ++t) bm[t] = fmaxf(bm[t], lane_xor16(bm[t]));
#pragma unroll
    for (int t = 0; t < QT; ++t) bm[t] = fmaxf(bm[t], lane_xor32(bm[t]));
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      const float m_old = m[t];
      const float m_new = (bm[t] > m_old + kRescaleSlack || m_old == -INFINITY) ? fmaxf(bm[t], m_old) : m_old;
      m_use[t] = m_new == -INFINITY ? 0.f : m_new;
      rescale |= m_new != m_old;
      bm[t] = m_old;
      m[t] = m_new;
    }
    if (__any(rescale)) {
#pragma unroll
      for (int t = 0; t < QT; ++t) {
        const float alpha = fast_exp2(bm[t] - m_use[t]);
        l[t] *= alpha;
#pragma unroll
        for (int dt = 0; dt < D / 16; ++dt) acc[t][dt] *= alpha;
      }
    }
    if constexpr (sizeof(DT) == 2) {
      bf16x8 p[PT][QT];
#pragma unroll
      for (int t = 0; t < QT; ++t)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float x = fast_exp2(s[t][i >> 2][i & 3] - m_use[t]);
          l[t] += x;
          p[0][t][i] = static_cast<bf16>(x);
          if constexpr (PT == 2) p[1][t][i] = static_cast<bf16>(x - static_cast<float>(p[0][t][i]));
        }
      if constexpr (CAREFUL) {
        without_odd(f, p, t0);
        return;
      }
#pragma unroll
      for (int dt = 0; dt < D / 16; ++dt) {
        const bf16x8 v = f.vf(dt);
#pragma unroll
        for (int n = 0; n < PT; ++n)
#pragma unroll
          for (int t = 0; t < QT; ++t) acc[t][dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, p[n][t], acc[t][dt], 0, 0, 0);
      }
    } else {
#pragma unroll
      for (int t = 0; t < QT; ++t)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float x = fast_exp2(s[t][i >> 2][i & 3] - m_use[t]);
          s[t][i >> 2][i & 3] = x;
          l[t] += x;
        }
      if constexpr (CAREFUL) {
        without_odd(f, s, t0);
        return;
      }
#pragma unroll
      for (int dt = 0; dt < D / 16; ++dt)
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
          for (int t = 0; t < QT; ++t)
            acc[t][dt] = __builtin_amdgcn_mfma_f32_16x16x4f32(f.v[dt][i >> 2][i & 3], s[t][i >> 2][i & 3], acc[t][dt], 0, 0, 0);
    }
  }

  // A block with values that are not finite: they are taken out, and what rows that see
  // them have of their channels becomes NaN: those are found by a product of "is not finite" and
  // "is seen", in zeros and ones.
  template <class F, class P> __device__ __forceinline__ void without_odd(const F& f, const P& p, int t0) {
    const int k0 = t0 + 8 * (lane_id() >> 4);
#pragma unroll
    for (int dt = 0; dt < D / 16; ++dt) {
      __builtin_amdgcn_sched_barrier(0);         // one channel tile after the other: registers
      floatx4 odd[QT];
#pragma unroll
      for (int t = 0; t < QT; ++t) odd[t] = floatx4{0.f, 0.f, 0.f, 0.f};
      if constexpr (sizeof(DT) == 2) {
        bf16x8 v = f.vf(dt), o;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float x = static_cast<float>(v[i]);
          const bool is = !(fabsf(x) < INFINITY);
          o[i] = static_cast<bf16>(is ? 1.f : 0.f);
          v[i] = static_cast<bf16>(is ? 0.f : x);
        }
#pragma unroll
        for (int t = 0; t < QT; ++t) {
          bf16x8 see;
#pragma unroll
          for (int i = 0; i < 8; ++i) see[i] = static_cast<bf16>(k0 + i >= row[t].lo && k0 + i < row[t].hi ? 1.f : 0.f);
          odd[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(o, see, odd[t], 0, 0, 0);
#pragma unroll
          for (int n = 0; n < PT; ++n) acc[t][dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, p[n][t], acc[t][dt], 0, 0, 0);
        }
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float x = f.v[dt][i >> 2][i & 3];
          const bool is = !(fabsf(x) < INFINITY);
#pragma unroll
          for (int t = 0; t < QT; ++t) {
            const float see = k0 + i >= row[t].lo && k0 + i < row[t].hi ? 1.f : 0.f;
            odd[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(is ? 1.f : 0.f, see, odd[t], 0, 0, 0);
            acc[t][dt] = __builtin_amdgcn_mfma_f32_16x16x4f32(is ? 0.f : x, p[t][i >> 2][i & 3], acc[t][dt], 0, 0, 0);
          }
        }
      }
#pragma unroll
      for (int t = 0; t < QT; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[t][dt][e] = odd[t][e] > 0.f ? __uint_as_float(0x7fc00000u) : acc[t][dt][e];
    }
  }

  __device__ __forceinline__ void join_lanes() {
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      l[t] += lane_xor16(l[t]);
      l[t] += lane_xor32(l[t]);
    }
  }
  // One tile to LDS, and one from there merged in.
  __device__ __forceinline__ void give(int t, floatx4* buf, float* ml) const {
    const int lane = lane_id();
#pragma unroll
    for (int dt = 0; dt < D / 16; ++dt) buf[dt * kWave + lane] = acc[t][dt];
    if (lane < 16) {
      ml[lane] = m[t];
      ml[16 + lane] = l[t];
    }
  }
  __device__ __forceinline__ void take(int t, const floatx4* buf, const float* ml) {
    const int lane = lane_id(), c16 = lane & 15;
    const float m2 = ml[c16], l2 = ml[16 + c16];
    const float mx = fmaxf(m[t], m2), mu = mx == -INFINITY ? 0.f : mx;
    const float x = fast_exp2(m[t] - mu), y = fast_exp2(m2 - mu);
    m[t] = mx;
    l[t] = l[t] * x + l2 * y;
#pragma unroll
    for (int dt = 0; dt < D / 16; ++dt) acc[t][dt] = acc[t][dt] * x + buf[dt * kWave + lane] * y;
  }

  // The rows to the outputs, or (whole == false) to the partial results.
  __device__ __forceinline__ void finish(const MaskedParams& a, const Seq& s, int g, int pr0, int pr_last, bool whole,
                                         size_t part_row) const {
    const int lane = lane_id(), c16 = lane & 15, j = lane >> 4;
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      const int pr = pr0 + 16 * t + c16;
      if (pr > pr_last) continue;
      if (whole) {
        const int i = row_of(a, pr), h = g * a.G + pr - i * a.G;
        const size_t r = (size_t)(s.r0 + i) * a.Hq + h;
        DT* o = reinterpret_cast<DT*>(a.out) + r * D + 4 * j;
        const float inv = l[t] == 0.f ? 0.f : 1.f / l[t];      // a row without keys: 0
#pragma unroll
        for (int dt = 0; dt < D / 16; ++dt) {
          typedef DT __attribute__((ext_vector_type(4))) Four;
          Four w;
#pragma unroll
          for (int e = 0; e < 4; ++e) w[e] = from_f32<DT>(acc[t][dt][e] * inv);
          *reinterpret_cast<Four*>(o + 16 * dt) = w;
        }
        if (a.lse && j == 0) a.lse[r] = (m[t] + fast_log2(l[t])) * kLn2;
      } else {
        const size_t r = part_row + 16 * t + c16;
#pragma unroll
        for (int dt = 0; dt < D / 16; ++dt) *reinterpret_cast<floatx4*>(a.part_o + r * D + 16 * dt + 4 * j) = acc[t][dt];
        if (j == 0) a.part_ml[r] = make_float2(m[t], l[t]);
      }
    }
  }
};

// What some row of the workgroup sees.
__device__ __forceinline__ Span join_spans(const Span& mine, int (&s_span)[kWaves][2]) {
  if (lane_id() == 0) {
    s_span[threadIdx.x / kWave][0] = mine.lo;
    s_span[threadIdx.x / kWave][1] = mine.hi;
  }
  __syncthreads();
  Span all = mine;
#pragma unroll
  for (int i = 0; i < kWaves; ++i) {
    all.lo = min(all.lo, uni(s_span[i][0]));
    all.hi = max(all.hi, uni(s_span[i][1]));
  }
  return all;
}

// A workgroup's piece: the blocks b0 .. b1 - 1 of a tile.
struct Piece {
  int b0, b1, n;           // n: pieces of the tile
  bool whole;
};
// False if the tile has no such piece.
__device__ __forceinline__ bool piece_of(const Split& sp, const Span& all, int piece, Piece& p) {
  const int blo = all.lo >= all.hi ? 0 : all.lo / kBlk, bhi = all.lo >= all.hi ? 0 : (all.hi + kBlk - 1) / kBlk;
  const int nb = bhi - blo, n = max((nb + sp.per - 1) / sp.per, 1);
  if (piece >= n) return false;
  p.n = n;
  // even pieces: shares of the first nb % n one block more
  const int each = nb / n, more = nb - each * n;
  p.b0 = blo + piece * each + min(piece, more);
  p.b1 = p.b0 + each + (piece < more ? 1 : 0);
  p.whole = n == 1;
  return true;
}
__device__ __forceinline__ void note_pieces(const MaskedParams& a, const Piece& p, int sg, int tile, int piece) {
  if (piece == 0 && threadIdx.x == 0) a.pieces[(size_t)sg * a.tiles + tile] = p.n;
}
__device__ __forceinline__ size_t part_row_of(const MaskedParams& a, const Split& sp, int sg, int tile, int piece, int tile_rows) {
  return ((size_t)sg * a.units + (size_t)tile * sp.np + piece) * tile_rows;
}

// The window's keys and values to their pages, by every workgroup those that it reads
// (several may write the same), by the first of a (sequence, head) all.  A kernel of its own for it
// costs a launch, 2.5 us of the host's and 2 to 6 of the device's; this costs the workgroups at the
// window a round trip (8 windows of eight by 1 to 8 Ki keys 37.0 to 36.1 us, one 23.7 to 22.1; 32
// windows 83.5 and 86, 64 the same).
constexpr int kAppendFew = 16;         // window rows up to which this is done
template <typename DT, int D>
__device__ __forceinline__ void append_own(const MaskedParams& a, const Seq& s, int g, const Piece& p, bool all) {
  if (!a.k_new) return;
  const int from = all ? s.L : max(s.L, p.b0 * kBlk), to = all ? s.end : min(s.end, p.b1 * kBlk);
  if (from >= to) return;
  const int32_t* table = a.page_table + (size_t)s.b * a.max_pages;
  const int ps = 1 << a.log2ps;
  const DT* kn = reinterpret_cast<const DT*>(a.k_new);
  const DT* vn = reinterpret_cast<const DT*>(a.v_new);
  DT* kc = reinterpret_cast<DT*>(const_cast<void*>(a.k_cache));
  DT* vc = reinterpret_cast<DT*>(a.v_cache);
  for (int e = threadIdx.x; e < (to - from) * D; e += blockDim.x) {
    const int pos = from + e / D, d = e % D, sl = pos & (ps - 1);
    const size_t page = (size_t)min(max(table[min(pos >> a.log2ps, a.max_pages - 1)], 0), a.num_pages - 1) * a.Hkv + g;
    const size_t src = ((size_t)(s.r0 + pos - s.L) * a.Hkv + g) * D + d;
    kc[((page * (D / 32) + d / 32) << a.log2ps) * 32 + sl * 32 + (d & 31)] = kn[src];
    vc[((page * D + d) << a.log2ps) + sl] = vn[src];
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");       // written when the others pass the barrier
  __syncthreads();
}

// Operands straight into registers; the W waves take every W-th block of the piece, and join
// their rows at the end.  (In fp32, where a block's products take 2 thousand clocks per 16
// rows, waves with rows of their own left the longest tiles to run alone at the end: 6 prefixes
// of 120 to 700 positions 80 us, 61 so; two windows of 300 rows by 1 to 4.5 Ki keys 995 and 513.)
template <typename DT, int D, int QT, int W>
__global__ __launch_bounds__(64 * W, W == 8 || sizeof(DT) * D > 256 ? 1 : 2) void masked_keys_kernel(MaskedParams a) {
  constexpr bool NT = sizeof(DT) == 2;                 // one tile per window; fp32 may have many (69 to 76 us)
  constexpr int kRows = 16 * QT, kTile = (D / 16) * kWave, PT = sizeof(DT) == 2 ? 2 : 1;
  __shared__ floatx4 s_acc[W / 2][kTile];
  __shared__ float s_ml[W / 2][32];
  const int sg = slot_head_of(a, blockIdx.x, blockIdx.y, gridDim.x);
  if (sg < 0) return;
  const int slot = sg / a.Hkv, g = sg - slot * a.Hkv;
  const Seq s = seq_of(a, slot);
  if (s.rows == 0) return;
  const Split sp = split_of(a, s, kRows);
  const int unit = gridDim.y - 1 - blockIdx.y;         // the last tiles, which see most, first
  const int tile = unit / sp.np, piece = unit - tile * sp.np;
  if (tile >= sp.nt) return;
  const int pr0 = tile * kRows, pr_last = min(pr0 + kRows, s.rows) - 1;
  const int wv = uni(threadIdx.x / kWave);
  Rows<DT, D, QT, PT> R;
  R.begin(a, s, g, pr0, pr_last);
  const Span mine = span_of<QT>(R.row);
  Piece p;
  if (!piece_of(sp, mine, piece, p)) return;
  const ScalarInts pt = scalar(a.page_table + (size_t)s.b * a.max_pages);
  append_own<DT, D>(a, s, g, p, tile == 0 && piece == 0);
  const int first = p.b0 + wv, last = p.b1;
  auto walk = [&](auto careful) __attribute__((always_inline)) {
    constexpr bool CAREFUL = decltype(careful)::value;
    R.reset();
    if (first >= last) return;
    Parts parts;
    parts.look_up(a, pt, first * kBlk, g);
    Frags<DT, D> f;
    load_keys<DT, D, NT>(a, f, first * kBlk, parts);
    load_values<DT, D, NT>(a, a.v_cache, f, first * kBlk, parts);
    parts.look_up(a, pt, (first + W) * kBlk, g);
    for (int n = first; n < last; n += W) {
      const int t0 = n * kBlk;
      // the next keys are asked for once the scores have used theirs, the next
      // values once the products have
      floatx4 sc[QT][2];
      scores<DT, D, QT>(f, R.Q, sc);
      const bool more = n + W < last;
      __builtin_amdgcn_sched_barrier(0);
      if (more) load_keys<DT, D, NT>(a, f, t0 + W * kBlk, parts);
      __builtin_amdgcn_sched_barrier(0);
      R.template weigh<CAREFUL>(a, f, sc, t0, CAREFUL || !mine.whole(t0));
      __builtin_amdgcn_sched_barrier(0);
      if (more) load_values<DT, D, NT>(a, a.v_cache, f, t0 + W * kBlk, parts);
      parts.look_up(a, pt, t0 + 2 * W * kBlk, g);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  R.queries_here();
  walk(std::false_type());
  if (__any(R.odd())) walk(std::true_type());
  note_pieces(a, p, sg, tile, piece);
  R.join_lanes();
#pragma unroll
  for (int t = 0; t < QT; ++t)
#pragma unroll
    for (int half = W / 2; half > 0; half >>= 1) {
      if (wv >= half && wv < 2 * half) R.give(t, s_acc[wv - half], s_ml[wv - half]);
      __syncthreads();
      if (wv < half) R.take(t, s_acc[wv], s_ml[wv]);
      __syncthreads();
    }
  if (wv == 0) R.finish(a, s, g, pr0, pr_last, p.whole, part_row_of(a, sp, sg, tile, piece, kRows));
}

// ---- more rows: keys shared through LDS ----
//
// A unit of the ring is a block's operands, 128 D bytes in pieces of 1 KB, one load
// instruction each: keys [part][32-channel slice][slot][32], values [part][channel]
// [16 slots], or with larger pages (WIDE), whose parts lie side by side, [channel][32
// slots].  Within a piece the 16-byte entries are permuted so that the lanes that a
// 16-byte LDS read serves at once hit distinct banks; a load writes lane l's 16 bytes
// to entry l, so the loading lane fetches what belongs there.
// Two units with a tile per wave (64 windows of eight 155 to 145 us), three with two (packed prompts 57
// us, with two units 59).
constexpr int ring_of(int QT) { return QT == 1 ? 2 : 3; }
// Of the CU's 160 KB more than a quarter: a fourth workgroup would take 64 windows of eight from 145 to
// 160 us, 8 of them from 33 to 40.
constexpr int kLeastLds = 41 * 1024;
__device__ __forceinline__ int key_entry(int slot, int q) { return 4 * slot + (q ^ (((slot >> 1) & 1) | ((slot >> 2) & 2))); }
__device__ __forceinline__ int val_entry(int ch, int h) { return 2 * ch + (h ^ ((ch >> 2) & 1)); }
__device__ __forceinline__ int wide_entry(int ch, int q) {
  const int c4 = (ch >> 2) & 3;
  return 4 * ch + (q ^ (((c4 << 1) ^ (3 * (c4 >> 1))) & 3));
}

template <int D, bool WIDE> struct LdsFrags {
  static constexpr int kStep = WIDE ? 1024 : 512;      // of 16 channels
  const char* at;
  int k0, k1, v0;      // byte offsets of the lane's key of either sub-tile, and of its channel's run
  __device__ __forceinline__ explicit LdsFrags(const char* buf) : at(buf) {
    const int lane = lane_id(), c16 = lane & 15, j = lane >> 4;
    auto key = [&](int st) {
      const int kk = 8 * (c16 >> 2) + 4 * st + (c16 & 3);
      return 1024 * (D / 32) * (kk >> 4) + 16 * key_entry(kk & 15, j);
    };
    k0 = key(0);
    k1 = key(1);
    v0 = 64 * D + (WIDE ? 16 * wide_entry(c16, j) : 32 * D * (j >> 1) + 16 * val_entry(c16, j & 1));
  }
  __device__ __forceinline__ bf16x8 kf(int st, int ks) const {
    return *reinterpret_cast<const bf16x8*>(at + (st ? k1 : k0) + 1024 * ks);
  }
  __device__ __forceinline__ bf16x8 vf(int dt) const { return *reinterpret_cast<const bf16x8*>(at + v0 + kStep * dt); }
};

// Wave t's loads of a unit: pieces t, t + 4, ...
template <int D, bool WIDE> struct Loader {
  static constexpr int kLoads = D / 32, kUnit = 128 * D, kKeys = D / 64;    // loads of keys come first
  unsigned k[kKeys], v[kLoads - kKeys];      // the lane's byte offset in a page of the piece's (page, head)
  __device__ __forceinline__ Loader(int t, int ps) {
    const int lane = lane_id();
#pragma unroll
    for (int i = 0; i < kKeys; ++i) {
      const int slice = (t + 4 * i) % (D / 32), sl = lane >> 2, q = (lane & 3) ^ (key_entry(sl, 0) & 3);
      k[i] = 2u * (unsigned)((slice * ps + sl) * 32 + 8 * q);
    }
#pragma unroll
    for (int i = 0; i < kLoads - kKeys; ++i) {
      const int vp = t + 4 * i;
      if constexpr (WIDE) {
        const int ch = 16 * vp + (lane >> 2), q = (lane & 3) ^ (wide_entry(lane >> 2, 0) & 3);
        v[i] = 2u * (unsigned)(ch * ps + 8 * q);
      } else {
        const int ch = 32 * (vp % (D / 32)) + (lane >> 1), h = (lane & 1) ^ (val_entry(lane >> 1, 0) & 1);
        v[i] = 2u * (unsigned)(ch * ps + 8 * h);
      }
    }
  }
  // `lds`: LDS address of the wave's first piece of the unit.
  template <bool NT>
  __device__ __forceinline__ void issue(const MaskedParams& a, const Parts& parts, int t0, int t, unsigned lds) const {
    const int ps = 1 << a.log2ps;
    const int o0 = t0 & (ps - 1), o1 = (t0 + 16) & (ps - 1);
    // byte offsets of both parts' (page, head), the same in either cache
    const size_t size = (size_t)(unsigned)(2 * D * ps);
    const size_t at0 = (size_t)(unsigned)uni((int)parts.of(0)) * size, at1 = (size_t)(unsigned)uni((int)parts.of(1)) * size;
    const char* kc = reinterpret_cast<const char*>(a.k_cache);
    const char* vc = reinterpret_cast<const char*>(a.v_cache);
    // D = 128: a wave's pieces are of one part after the other; D = 64: of one part
    constexpr int PER = D / 32;                // pieces of a part
#pragma unroll
    for (int i = 0; i < kKeys; ++i) {
      const bool second = PER == 4 ? i : t >= PER;
      load_to<NT>(lds + 4096 * i, kc + (second ? at1 + (unsigned)(64 * o1) : at0 + (unsigned)(64 * o0)), k[i]);
    }
#pragma unroll
    for (int i = 0; i < kLoads - kKeys; ++i) {
      const bool second = !WIDE && (PER == 4 ? i : t >= PER);
      load_to<NT>(lds + 4096 * (i + kKeys), vc + (WIDE ? at0 + (unsigned)(2 * o0) : second ? at1 : at0), v[i]);
    }
  }
  template <bool NT> static __device__ __forceinline__ void load_to(unsigned lds, const char* base, unsigned off) {
    if constexpr (NT)
      asm volatile("s_mov_b32 m0, %0\n\tglobal_load_lds_dwordx4 %1, %2 nt" : : "s"(lds), "v"(off), "s"(base) : "memory", "m0");
    else
      asm volatile("s_mov_b32 m0, %0\n\tglobal_load_lds_dwordx4 %1, %2" : : "s"(lds), "v"(off), "s"(base) : "memory", "m0");
  }
};

// NT: the ring's loads go past the caches' order of use.  A probability is rounded to bf16 once (outputs off
// by 0.0020 to 0.0023 of their size, of which their own rounding is 0.0016); in two terms, as decode rows have
// it, products take twice as long: 64 windows of eight 138 and 146 us, documents 58 and 63, packed prompts 80
// and 96.
template <int D, bool WIDE, int QT, bool NT>
__global__ __launch_bounds__(256, 3) void masked_tile_kernel(MaskedParams a) {
  typedef Loader<D, WIDE> Load;
  constexpr int kRows = 64 * QT, kRing = ring_of(QT);
  __shared__ __attribute__((aligned(1024))) char s_ring[D == 128 && kRing * Load::kUnit < kLeastLds ? kLeastLds : kRing * Load::kUnit];
  __shared__ int s_span[kWaves][2];
  const int sg = slot_head_of(a, blockIdx.x, blockIdx.y, gridDim.x);
  if (sg < 0) return;
  const int slot = sg / a.Hkv, g = sg - slot * a.Hkv;
  const Seq s = seq_of(a, slot);
  if (s.rows == 0) return;
  const Split sp = split_of(a, s, kRows);
  const int unit = gridDim.y - 1 - blockIdx.y;         // the last tiles, which see most, first
  const int tile = unit / sp.np, piece = unit - tile * sp.np;
  if (tile >= sp.nt) return;
  const int t = uni(threadIdx.x / kWave);
  const int pr0 = tile * kRows, pr_last = min(pr0 + kRows, s.rows) - 1, wr0 = pr0 + 16 * QT * t;
  Rows<bf16, D, QT, 1> R;
  R.begin(a, s, g, wr0, pr_last);
  const Span mine = span_of<QT>(R.row);
  Piece p;
  if (!piece_of(sp, join_spans(mine, s_span), piece, p)) return;
  append_own<bf16, D>(a, s, g, p, tile == 0 && piece == 0);
  const bool has_rows = wr0 <= pr_last;
  const ScalarInts pt = scalar(a.page_table + (size_t)s.b * a.max_pages);
  const Load load(t, 1 << a.log2ps);
  const LdsFrags<D, WIDE> lane_at(nullptr);
  const unsigned ring = uni((int)(unsigned)(uintptr_t)(__attribute__((address_space(3))) void*)s_ring + 1024 * t);
  auto walk = [&](auto careful) __attribute__((always_inline)) {
    constexpr bool CAREFUL = decltype(careful)::value;
    R.reset();
    if (p.b0 >= p.b1) return;
    Parts parts;
    // Behind the piece's end its last unit is loaded again, so that every wait has the same count.
    auto look_up = [&](int n) { parts.look_up(a, pt, min(n, p.b1 - 1) * kBlk, g); };
    auto issue = [&](int n, int buf) { load.template issue<NT>(a, parts, min(n, p.b1 - 1) * kBlk, t, ring + buf * Load::kUnit); };
#pragma unroll
    for (int i = 0; i < kRing - 1; ++i) {
      look_up(p.b0 + i);
      issue(p.b0 + i, i);
    }
    look_up(p.b0 + kRing - 1);
    if (!CAREFUL) R.queries_here();                      // only the ring's loads from here on
    int use = 0, fill = kRing - 1;
    for (int n = p.b0; n < p.b1; ++n) {
      // Unit n is there (this wave's loads by the count, the others' by the barrier), and
      // all have read unit n - 1, whose place the next one takes.
      asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(Load::kLoads * (kRing - 2)) : "memory");
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
      issue(n + kRing - 1, fill);
      look_up(n + kRing);
      fill = fill + 1 == kRing ? 0 : fill + 1;
      const int t0 = n * kBlk;
      if (has_rows && mine.sees(t0)) {
        LdsFrags<D, WIDE> f = lane_at;
        f.at = s_ring + use * Load::kUnit;
        R.template block<CAREFUL>(a, f, t0, CAREFUL || !mine.whole(t0));
      }
      use = use + 1 == kRing ? 0 : use + 1;
    }
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");   // none may land after the workgroup has gone
  };
  walk(std::false_type());
  // all waves together, since they share the loads; also the barrier before the ring is filled again
  if (__syncthreads_or(R.odd())) walk(std::true_type());
  note_pieces(a, p, sg, tile, piece);
  R.join_lanes();
  R.finish(a, s, g, wr0, pr_last, p.whole, part_row_of(a, sp, sg, tile, piece, kRows) + 16 * QT * t);
}

// Joins the pieces of every tile that was cut: some neighbouring rows per workgroup, 16
// lanes per row.
template <typename DT, int D>
__global__ __launch_bounds__(256) void masked_merge_kernel(MaskedParams a, int tile_rows, int merge_rows) {
  const int slot = blockIdx.x / a.Hkv, g = blockIdx.x - slot * a.Hkv;
  const Seq s = seq_of(a, slot);
  const int d = ((int)threadIdx.x & 15) * (D / 16);
  constexpr int V = D / 64;                     // of four channels
  const Split sp = split_of(a, s, tile_rows);
  const int last = min((int)(blockIdx.y + 1) * merge_rows, s.rows);
  for (int pr = blockIdx.y * merge_rows + (int)threadIdx.x / 16; pr < last; pr += 16) {
    const int tile = pr / tile_rows;
    const int n = a.pieces[(size_t)blockIdx.x * a.tiles + tile];
    if (n == 1) continue;
    const size_t r0 = part_row_of(a, sp, blockIdx.x, tile, 0, tile_rows) + pr - tile * tile_rows;
    float m = -INFINITY, l = 0.f;
    floatx4 o[V];
#pragma unroll
    for (int i = 0; i < V; ++i) o[i] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int c = 0; c < n; ++c) {
      const size_t r = r0 + (size_t)c * tile_rows;
      const float2 ml = a.part_ml[r];
      floatx4 x[V];
#pragma unroll
      for (int i = 0; i < V; ++i) x[i] = ld16<floatx4>(a.part_o + r * D + d + 4 * i);
      const float mx = fmaxf(m, ml.x), mu = mx == -INFINITY ? 0.f : mx;
      const float u = fast_exp2(m - mu), w = fast_exp2(ml.x - mu);
      m = mx;
      l = l * u + ml.y * w;
#pragma unroll
      for (int i = 0; i < V; ++i) o[i] = o[i] * u + x[i] * w;
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;
    const int i = row_of(a, pr), h = g * a.G + pr - i * a.G;
    const size_t r = (size_t)(s.r0 + i) * a.Hq + h;
    DT* out = reinterpret_cast<DT*>(a.out) + r * D + d;
#pragma unroll
    for (int c = 0; c < V; ++c) {
      typedef DT __attribute__((ext_vector_type(4))) Four;
      Four w;
#pragma unroll
      for (int e = 0; e < 4; ++e) w[e] = from_f32<DT>(o[c][e] * inv);
      *reinterpret_cast<Four*>(out + 4 * c) = w;
    }
    if (a.lse && (threadIdx.x & 15) == 0) a.lse[r] = (m + fast_log2(l)) * kLn2;
  }
}

struct Plan {
  bool shared;                // keys through LDS
  int qt, waves, tile_rows, tiles, units, per, walk;
  bool cut;                   // some tile may be cut
  size_t part_rows;
};
Plan plan_of(int n_seq, int Hq, int Hkv, int max_q, long slots, int window, bool ends, bool bf16) {
  Plan p;
  const long rows = (long)max_q * (Hq / Hkv), sg = (long)n_seq * Hkv;
  p.shared = rows > 16 && bf16;
  p.qt = rows > (bf16 ? 64 : 16) ? 2 : 1;
  p.tile_rows = (p.shared ? 64 : 16) * p.qt;
  p.tiles = (int)((rows + p.tile_rows - 1) / p.tile_rows);
  long nb = (slots + kBlk - 1) / kBlk;
  if (!ends) nb = std::min(nb, ((long)(window > 0 ? window : INT_MAX) + p.tile_rows / (Hq / Hkv) + 1 + 2 * kBlk) / kBlk);
  // pieces of 8 blocks and 16: one window of eight 18 and 22 us, 24 of 13 by 200 to 3000 keys 43 and
  // 49; fp32, of 4 and 8, 24 small ones 26 and 29
  p.per = bf16 ? 8 : 4;
  // With rows enough to fill the chip by themselves, walks of up to 48 blocks stay whole: the
  // merge costs more.
  p.walk = sg * p.tiles >= 512 ? 48 : (int)std::clamp(sg * nb / (p.shared ? 1024 : 512), (long)p.per, 64L);
  p.per = (int)std::max((long)p.per, nb / 16384);      // units stay few under a table for millions of tokens
  p.waves = kWaves;
  // Decode rows of few sequences over short contexts: eight waves walk them whole, which leaves out
  // the merge and its launch (one of 700 tokens 16.2 to 13.8 us; one of 1500 16.5 to 14.7 among other
  // calls, but 30 to 34 alone; 512 sequences and heads 57 to 61).
  if (!p.shared && bf16 && nb <= 32 && sg * p.tiles < 512) {
    p.waves = 8;
    p.walk = 32;
  }
  const int least = std::max(p.per, p.walk);
  p.cut = nb > least;
  // the most units that a window of nt tiles has: nt ceil(nb / max(per nt, walk)), over nt
  long units = p.tiles;
  if (p.cut) {
    const long few = std::min((long)p.tiles, std::max(1L, (long)p.walk / p.per));
    units = std::max(units, few * ((nb + least - 1) / least));
    if (p.tiles > few) units = p.tiles + nb / p.per + 1;
  }
  p.units = (int)units;
  p.part_rows = p.cut ? (size_t)sg * p.units * p.tile_rows : 0;
  return p;
}

}  // namespace

int attn_masked_units(int n_seq, int Hq, int Hkv, int max_q, int max_pages, int page_size, int window, bool ends) {
  int most = 0;
  for (const bool b : {false, true})
    most = std::max(most, plan_of(n_seq, Hq, Hkv, max_q, table_slots(max_pages, page_size), window, ends, b).units);
  return most;
}

size_t attn_masked_workspace(int n_seq, int Hq, int Hkv, int D, int max_q, int max_pages, int page_size, int window, bool ends) {
  size_t most = 0;
  for (const bool b : {false, true}) {
    const Plan p = plan_of(n_seq, Hq, Hkv, max_q, table_slots(max_pages, page_size), window, ends, b);
    most = std::max(most, p.part_rows * (D * 4 + 8) + (size_t)n_seq * Hkv * p.tiles * 4);
  }
  return (most + 255) / 256 * 256;
}

hipError_t launch_attn_masked(const AttnMaskedLaunch& L, hipStream_t st) {
  MaskedParams p{};
  static_cast<WindowParams&>(p) = window_params(L);
  const Plan pl = plan_of(L.n_seq, L.Hq, L.Hkv, L.max_q, p.slots, L.mod.window, L.mod.end_key != nullptr, L.dtype_bf16);
  p.v_cache = L.v_cache;
  p.out = L.out;
  p.lse = L.lse;
  p.part_o = (float*)L.workspace;
  p.part_ml = (float2*)(p.part_o + pl.part_rows * L.D);
  p.pieces = (int32_t*)(p.part_ml + pl.part_rows);
  p.tiles = pl.tiles;
  p.units = pl.units;
  p.per = pl.per;
  p.walk = pl.walk;
  trace_begin(st);
  hipError_t e = hipSuccess;
  if (L.k_new && L.max_q <= kAppendFew) {
    p.k_new = L.k_new;
    p.v_new = L.v_new;
  } else if (L.k_new) {
    e = launch_append_window(L, st);
  }
  if (e != hipSuccess) return e;
  trace_mark(st);
  const int sg = L.n_seq * L.Hkv;
  auto go = [&](auto kernel, int waves = kWaves) {
    hipLaunchKernelGGL(kernel, dim3((sg + 7) / 8 * 8, pl.units), dim3(64 * waves), 0, st, p);
  };
  auto pick = [&](auto dt, auto dim) {
    using DT = decltype(dt);
    constexpr int D = decltype(dim)::value;
    if constexpr (sizeof(DT) == 2) {
      const bool wide = L.page_size > 16;
      if (!pl.shared) { if (pl.waves == 8) go(masked_keys_kernel<DT, D, 1, 8>, 8); else go(masked_keys_kernel<DT, D, 1, 4>); }
      else {
        // One tile of a window reads its keys once.  Less than the 256 MB of the memory-side cache is
        // left to it (4 KV heads, windows of eight by up to 8 Ki keys: 8 of them 33.6 us, 36.1 as a
        // stream; 16 48.4 and 46.4, 64 142 and 132; packed prompts, of many tiles, 86 and 97).
        const bool nt = pl.tiles == 1 && (long)sg * p.slots * D * 4 > 256L << 20;
        auto tile = [&](auto w, auto q) {
          constexpr bool WIDE = decltype(w)::value;
          constexpr int QT = decltype(q)::value;
          if (nt) go(masked_tile_kernel<D, WIDE, QT, true>); else go(masked_tile_kernel<D, WIDE, QT, false>);
        };
        typedef std::integral_constant<int, 1> One;
        typedef std::integral_constant<int, 2> Two;
        if (pl.qt == 1) { if (wide) tile(std::true_type(), One()); else tile(std::false_type(), One()); }
        else { if (wide) tile(std::true_type(), Two()); else tile(std::false_type(), Two()); }
      }
    } else {
      if (pl.qt == 2) go(masked_keys_kernel<DT, D, 2, 4>); else go(masked_keys_kernel<DT, D, 1, 4>);
    }
  };
  typedef std::integral_constant<int, 64> D64;
  typedef std::integral_constant<int, 128> D128;
  if (L.dtype_bf16) {
    if (L.D == 128) pick(bf16(), D128()); else pick(bf16(), D64());
  } else {
    if (L.D == 128) pick(float(), D128()); else pick(float(), D64());
  }
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  trace_mark(st);
  if (pl.cut) {
    auto merge = [&](auto kernel) {
      const int rows = pl.tiles > 8 ? 64 : 16;         // of many tiles, most are whole
      hipLaunchKernelGGL(kernel, dim3(sg, (unsigned)(((long)pl.tiles * pl.tile_rows + rows - 1) / rows)), dim3(256), 0, st, p,
                         pl.tile_rows, rows);
    };
    if (L.dtype_bf16) {
      if (L.D == 128) merge(masked_merge_kernel<bf16, 128>); else merge(masked_merge_kernel<bf16, 64>);
    } else {
      if (L.D == 128) merge(masked_merge_kernel<float, 128>); else merge(masked_merge_kernel<float, 64>);
    }
    e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  trace_mark(st);
  return hipSuccess;
}

}  // namespace ipdv
