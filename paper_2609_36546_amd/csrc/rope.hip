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
// Angles: position * f is exact in double (31 + 24 bits), and so is its
// reduction to a fraction of a turn to about 1e-16 of the turns; only the
// fraction goes to fp32.  In fp32 the angle of position 10^5 would be off by
// 0.004.  One workgroup takes kRopeTok rows of one sequence with all their
// heads, so an angle is computed once for Hq + Hkv uses and kept in LDS; what
// is left is one read and one write of the data, in 16-byte pieces where the
// pairs allow it (two pieces R/2 apart, or one piece of whole pairs).
#include "common.h"
#include "kernels.h"

namespace ipdv {
namespace {

constexpr int kRopeTok = 4;

typedef __attribute__((__vector_size__(16))) int i32x4;

template <typename DT>
struct Piece {   // 16 bytes of a row
  static constexpr int N = 16 / (int)sizeof(DT);
  DT e[N];
};

template <typename DT>
__device__ __forceinline__ Piece<DT> ld_piece(const DT* p) {
  const i32x4 v = ld16<i32x4>(p);
  return __builtin_bit_cast(Piece<DT>, v);
}
template <typename DT>
__device__ __forceinline__ void st_piece(DT* p, const Piece<DT>& x) {
  *reinterpret_cast<i32x4*>(p) = __builtin_bit_cast(i32x4, x);
}

// VEC: the pairs fall into whole 16-byte pieces (see launch_rope).
template <typename DT, bool INTER, bool VEC>
__global__ __launch_bounds__(256) void rope_kernel(RopeLaunch p) {
  extern __shared__ float2 s_cs[];                 // [kRopeTok][R / 2] cos, sin
  constexpr int N = VEC ? Piece<DT>::N : 1;
  const int slot = blockIdx.y;
  const int b = p.seq_ids ? p.seq_ids[slot] : slot;
  const int r0 = p.cu_q[b], kb = p.cu_q[b + 1] - r0;
  const int i0 = blockIdx.x * kRopeTok;
  if (i0 >= kb) return;
  const int n_tok = min(kRopeTok, kb - i0);
  const int half = p.rot / 2;
  const int pos0 = max(p.ctx_lens[b], 0) + i0;
  for (int e = threadIdx.x; e < n_tok * half; e += 256) {
    const int t = e / half, c = e - t * half;
    double a = (double)(pos0 + t) * (double)p.inv_freq[c] * 0.15915494309189533577;   // in turns
    a -= rint(a);
    float sn, cs;
    sincospif(2.0f * (float)a, &sn, &cs);
    s_cs[e] = make_float2(cs * p.factor, (p.inverse ? -sn : sn) * p.factor);
  }
  __syncthreads();
  // A row's work: `turns` pieces (half: a piece and its partner; interleaved:
  // one piece of N / 2 pairs, or one pair) and `pass` pieces behind them.
  const int turns = INTER ? (VEC ? p.rot / N : half) : half / N;
  const int pass = (p.D - p.rot) / N;
  const int per_head = turns + pass;
  const int per_row = per_head * (p.Hq + p.Hkv);
  for (int e = threadIdx.x; e < n_tok * per_row; e += 256) {
    const int t = e / per_row, in_row = e - t * per_row;
    int h = in_row / per_head;
    const int u = in_row - h * per_head;
    const bool is_q = h < p.Hq;
    if (!is_q) h -= p.Hq;
    const size_t row = (size_t)(r0 + i0 + t);
    const DT* src = reinterpret_cast<const DT*>(is_q ? p.q : p.k) + row * (is_q ? p.q_stride : p.k_stride) + (size_t)h * p.D;
    DT* dst = reinterpret_cast<DT*>(is_q ? p.q_out : p.k_out) + row * (is_q ? p.qo_stride : p.ko_stride) + (size_t)h * p.D;
    const float2* cs = s_cs + t * half;
    if (u >= turns) {
      const int c = p.rot + (u - turns) * N;
      if constexpr (VEC) st_piece(dst + c, ld_piece(src + c));
      else dst[c] = src[c];
    } else if constexpr (!VEC) {
      const int cx = INTER ? 2 * u : u, cy = INTER ? 2 * u + 1 : u + half;
      const float x = to_f32(src[cx]), y = to_f32(src[cy]);
      dst[cx] = from_f32<DT>(x * cs[u].x - y * cs[u].y);
      dst[cy] = from_f32<DT>(x * cs[u].y + y * cs[u].x);
    } else if constexpr (INTER) {
      const int c = u * N;
      Piece<DT> v = ld_piece(src + c);
#pragma unroll
      for (int i = 0; i < N; i += 2) {
        const float x = to_f32(v.e[i]), y = to_f32(v.e[i + 1]);
        const float2 w = cs[(c + i) / 2];
        v.e[i] = from_f32<DT>(x * w.x - y * w.y);
        v.e[i + 1] = from_f32<DT>(x * w.y + y * w.x);
      }
      st_piece(dst + c, v);
    } else {
      const int c = u * N;
      Piece<DT> vx = ld_piece(src + c), vy = ld_piece(src + c + half);
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const float x = to_f32(vx.e[i]), y = to_f32(vy.e[i]);
        const float2 w = cs[c + i];
        vx.e[i] = from_f32<DT>(x * w.x - y * w.y);
        vy.e[i] = from_f32<DT>(x * w.y + y * w.x);
      }
      st_piece(dst + c, vx);
      st_piece(dst + c + half, vy);
    }
  }
}

template <typename DT>
hipError_t launch_t(const RopeLaunch& L, hipStream_t st) {
  constexpr int N = 16 / (int)sizeof(DT);
  const bool inter = L.interleaved;
  // whole pieces: every row starts on 16 bytes, the pieces of a pair too
  const bool vec = L.al16 && L.D % N == 0 && (inter ? L.rot % N == 0 : (L.rot / 2) % N == 0);
  const dim3 grid((L.max_q + kRopeTok - 1) / kRopeTok, L.n_seq);
  const size_t lds = (size_t)kRopeTok * (L.rot / 2) * sizeof(float2);
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(256), lds, st, L); };
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
