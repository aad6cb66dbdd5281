// Rotary positions for gfx950: the pairs of channels of every query and key
// row are turned by the angle position * inverse frequency.
//
//   (x, y) -> s (x cos a - y sin a, x sin a + y cos a),   a = (L_b + i) f_p
//
// for pair p of row i of sequence b; s is the caller's factor, and the inverse
// turns by -a, which with the same s is the transposed map, the gradient.
// Pairs are channels (p, p + R/2) or (2p, 2p + 1) of the first R channels; the
// others pass through.
//
// Angles: position * f is exact in double below position 2^29 (29 + 24 bits) and
// rounded to 2^-53 of itself from there on; its reduction to a fraction of a turn
// adds 2^-52 of the turns, and only the fraction goes to fp32.  In fp32 the angle of
// position 10^5 would be off by 0.004.
//
// Bound by one read and one write of the data, moved in 16-byte pieces where
// the pairs allow it (two pieces R/2 apart, or one piece of whole pairs).  A
// sequence's pieces are dealt out flat over rows, heads and pieces, kPer to a
// thread, so that a few rows of many heads fill as many workgroups as a prompt
// does; a workgroup's rows (two or three at common head counts) have their
// angles computed once, into LDS, while the first pieces are on their way.
// Prompts of 6141 tokens, 36 heads of 128 in bf16: 113 MB in 20 us, the rate of a
// copy; ragged windows in fp32, 17 MB, in 7 (a workgroup per row took 17).
#include "common.h"
#include "kernels.h"

namespace ipdv {
namespace {

constexpr int kPer = 2;         // pieces (pairs of pieces) per thread

typedef __attribute__((__vector_size__(16))) int i32x4;

// VEC: the pairs fall into whole 16-byte pieces (see launch_t).  A row's work:
// per head `turns` units (half: a piece and its partner; interleaved: a piece
// of N / 2 pairs; else a pair), then `pass` pieces behind them.
template <typename DT, bool INTER, bool VEC>
__global__ __launch_bounds__(256) void rope_kernel(RopeLaunch p, int turns, int per_head) {
  extern __shared__ float2 s_cs[];                 // [rows of the workgroup][R / 2] cos, sin
  constexpr int N = VEC ? 16 / (int)sizeof(DT) : 1;
  struct Raw { DT e[N]; };
  const int slot = blockIdx.y;
  const int b = p.seq_ids ? p.seq_ids[slot] : slot;
  const int r0 = p.cu_q[b], kb = min(p.cu_q[b + 1] - r0, p.max_q);
  const int half = p.rot / 2, per_row = per_head * (p.Hq + p.Hkv);
  const long e0 = (long)blockIdx.x * (256 * kPer);
  const long left = (long)max(kb, 0) * per_row - e0;
  if (left <= 0) return;
  const int t0 = (int)(e0 / per_row), in0 = (int)(e0 - (long)t0 * per_row);
  const int n = (int)min(left, (long)(256 * kPer));
  const int n_tok = (in0 + n - 1) / per_row + 1;
  const int pos0 = max(p.ctx_lens[b], 0) + t0;

  const DT* src[kPer];
  DT* dst[kPer];
  int tok[kPer], unit[kPer];
  Raw x[kPer], y[kPer];
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int at = i * 256 + (int)threadIdx.x;
    unit[i] = -1;
    if (at >= n) continue;
    const int e = in0 + at;
    tok[i] = e / per_row;
    const int in_row = e - tok[i] * per_row;
    int h = in_row / per_head;
    unit[i] = in_row - h * per_head;
    const bool is_q = h < p.Hq;
    if (!is_q) h -= p.Hq;
    const size_t row = (size_t)(r0 + t0 + tok[i]);
    src[i] = reinterpret_cast<const DT*>(is_q ? p.q : p.k) + row * (is_q ? p.q_stride : p.k_stride) + (size_t)h * p.D;
    dst[i] = reinterpret_cast<DT*>(is_q ? p.q_out : p.k_out) + row * (is_q ? p.qo_stride : p.ko_stride) + (size_t)h * p.D;
    const int u = unit[i];
    int cx = p.rot + (u - turns) * N, cy = -1;
    if (u < turns) {
      cx = INTER ? (VEC ? u * N : 2 * u) : u * N;
      if (!INTER) cy = cx + half;
      else if (!VEC) cy = cx + 1;
    }
    if constexpr (VEC) {
      x[i] = __builtin_bit_cast(Raw, ld16<i32x4>(src[i] + cx));
      if (cy >= 0) y[i] = __builtin_bit_cast(Raw, ld16<i32x4>(src[i] + cy));
    } else {
      x[i].e[0] = src[i][cx];
      if (cy >= 0) y[i].e[0] = src[i][cy];
    }
  }
  for (int e = threadIdx.x; e < n_tok * half; e += 256) {
    const int t = e / half, c = e - t * half;
    double a = (double)(pos0 + t) * (double)p.inv_freq[c] * 0.15915494309189533577;   // in turns
    a -= rint(a);
    float sn, cs;
    sincospif(2.0f * (float)a, &sn, &cs);
    s_cs[e] = make_float2(cs * p.factor, (p.inverse ? -sn : sn) * p.factor);
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int u = unit[i];
    if (u < 0) continue;
    DT* d = dst[i];
    if (u >= turns) {
      d += p.rot + (u - turns) * N;
    } else if constexpr (INTER && VEC) {
      const float2* cs = s_cs + tok[i] * half + u * (N / 2);
#pragma unroll
      for (int c = 0; c < N; c += 2) {
        const float a = to_f32(x[i].e[c]), b2 = to_f32(x[i].e[c + 1]);
        const float2 w = cs[c / 2];
        x[i].e[c] = from_f32<DT>(a * w.x - b2 * w.y);
        x[i].e[c + 1] = from_f32<DT>(a * w.y + b2 * w.x);
      }
      d += u * N;
    } else {
      const float2* cs = s_cs + tok[i] * half + u * N;
#pragma unroll
      for (int c = 0; c < N; ++c) {
        const float a = to_f32(x[i].e[c]), b2 = to_f32(y[i].e[c]);
        x[i].e[c] = from_f32<DT>(a * cs[c].x - b2 * cs[c].y);
        y[i].e[c] = from_f32<DT>(a * cs[c].y + b2 * cs[c].x);
      }
      d += INTER ? 2 * u : u * N;
      DT* d2 = d + (INTER ? 1 : half);
      if constexpr (VEC) *reinterpret_cast<i32x4*>(d2) = __builtin_bit_cast(i32x4, y[i]);
      else *d2 = y[i].e[0];
    }
    if constexpr (VEC) *reinterpret_cast<i32x4*>(d) = __builtin_bit_cast(i32x4, x[i]);
    else *d = x[i].e[0];
  }
}

template <typename DT>
hipError_t launch_t(const RopeLaunch& L, hipStream_t st) {
  constexpr int W = 16 / (int)sizeof(DT);
  const bool inter = L.interleaved;
  // whole pieces: every row starts on 16 bytes, the pieces of a pair too
  const bool vec = L.al16 && L.D % W == 0 && (inter ? L.rot % W == 0 : (L.rot / 2) % W == 0);
  const int N = vec ? W : 1;
  const int turns = inter ? (vec ? L.rot / N : L.rot / 2) : L.rot / 2 / N;
  const int per_head = turns + (L.D - L.rot) / N, per_row = per_head * (L.Hq + L.Hkv);
  constexpr int kUnits = 256 * kPer;
  const dim3 grid((unsigned)(((long)L.max_q * per_row + kUnits - 1) / kUnits), L.n_seq);
  // rows that a workgroup's units can touch
  const size_t lds = (size_t)((kUnits - 2) / per_row + 2) * (L.rot / 2) * sizeof(float2);
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(256), lds, st, L, turns, per_head); };
  if (inter) {
    if (vec) go(rope_kernel<DT, true, true>); else go(rope_kernel<DT, true, false>);
  } else {
    if (vec) go(rope_kernel<DT, false, true>); else go(rope_kernel<DT, false, false>);
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_rope(const RopeLaunch& L, hipStream_t st) {
  trace_begin(st);
  const hipError_t e = L.dtype_bf16 ? launch_t<bf16>(L, st) : launch_t<float>(L, st);
  if (e != hipSuccess) return e;
  trace_mark(st);
  return hipSuccess;
}

}  // namespace ipdv
