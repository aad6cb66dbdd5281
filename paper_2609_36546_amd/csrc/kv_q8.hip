// The 8-bit cache for gfx950: window rows quantised into the pages, and read
// back.  A row (one position of one KV head, keys or values apart) is stored in
// e4m3 with one power-of-two scale:
//
//   e = the least integer >= -126 with max|x| <= 448 2^e   (0 for a zero row)
//   stored = e4m3(x 2^-e), round to nearest even;  scale byte = e + 127
//
// The scale is a power of two because then x 2^-e is exact, the only rounding
// is the one to e4m3, the value that a byte stands for is exact in bf16, and
// the attention can put the scale into its conversion (keys) or its
// probabilities (values) without another rounding.  A finer scale would gain
// nothing but the top half binade: e4m3 is a floating type, its relative step
// does not depend on the scale.  A row with an entry that is not finite is
// stored as NaN as a whole: scale byte 255, key bytes NaN, value bytes zero.
//
// Pages: keys [page][head][D/16][slot][16], values [page][head][D][slot],
// scales [page][head][2][slot] (keys, then values).  A 16-slot unit of a head's
// keys is D/16 runs of 256 bytes, the same unit of its values D runs of 16
// bytes, so both stream in 16-byte lane loads.
//
// One wave per (sequence, head, 16-slot unit), bound by bytes: rows come in
// and go out in 16-byte pieces, values are turned between [slot][channel] and
// [channel][slot] in 2 to 3 KB of LDS per wave.  303 MB read back in 67 us (4.5
// TB/s, seven eighths of a copy's rate); a prompt batch's append, 19 MB, in 10 us
// and a decode step's, 64 rows of 4 heads, in 4.4, which is the latency of its
// chain: lengths, page, rows, row maximum, store.
#include "common.h"
#include "kernels.h"
#include "q8.h"

namespace ipdv {
namespace {

constexpr int kUnit = 16;   // slots per wave

// 8 channels of a row, as the caller holds it.
template <typename DT> __device__ __forceinline__ void ld8(const DT* p, float (&x)[8]);
template <> __device__ __forceinline__ void ld8<bf16>(const bf16* p, float (&x)[8]) {
  const bf16x8 v = ld16<bf16x8>(p);
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = static_cast<float>(v[i]);
}
template <> __device__ __forceinline__ void ld8<float>(const float* p, float (&x)[8]) {
  const floatx4 a = ld16<floatx4>(p), b = ld16<floatx4>(p + 4);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[i] = a[i];
    x[4 + i] = b[i];
  }
}
template <typename DT> __device__ __forceinline__ void st8(DT* p, const float (&x)[8]);
template <> __device__ __forceinline__ void st8<bf16>(bf16* p, const float (&x)[8]) {
  bf16x8 v;
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = static_cast<bf16>(x[i]);
  *reinterpret_cast<bf16x8*>(p) = v;
}
template <> __device__ __forceinline__ void st8<float>(float* p, const float (&x)[8]) {
  floatx4 a, b;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    a[i] = x[i];
    b[i] = x[4 + i];
  }
  *reinterpret_cast<floatx4*>(p) = a;
  *reinterpret_cast<floatx4*>(p + 4) = b;
}

// Maximum over the LPT neighbouring lanes that hold one row (8 or 16).
template <int LPT>
__device__ __forceinline__ float row_max(float v) {
  if constexpr (LPT == 16) v = fmaxf(v, dpp_move<0x140>(v));
  v = fmaxf(v, dpp_move<0x141>(v));
  v = fmaxf(v, dpp_move<0x4E>(v));
  return fmaxf(v, dpp_move<0xB1>(v));
}

// Quantises the row that LPT lanes hold: 8 bytes of this lane, and the scale byte.
template <int LPT>
__device__ __forceinline__ uint2 quantise(const float (&x)[8], bool is_key, int* scale_byte) {
  float am = 0.f, bad = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    am = fmaxf(am, fabsf(x[i]));
    if (!(fabsf(x[i]) < INFINITY)) bad = 1.f;
  }
  am = row_max<LPT>(am);
  bad = row_max<LPT>(bad);
  if (bad != 0.f) {
    *scale_byte = 255;
    const unsigned w = is_key ? 0x7f7f7f7fu : 0u;
    return make_uint2(w, w);
  }
  // am = m 2^x with m in [1, 2): 448 = 1.75 2^8, so e = x - 8, one more above 1.75.
  // A subnormal am has exponent bits 0 and clamps like the smallest normal ones.
  const unsigned u = __float_as_uint(am);
  int e = (int)(u >> 23) - 127 - 8 + ((u & 0x7fffffu) > 0x600000u);
  e = am == 0.f ? 0 : max(e, -126);
  *scale_byte = e + 127;
  const float inv = __uint_as_float((unsigned)(127 - e) << 23);   // 2^-e, e in [-126, 120]
  uint2 r;
  int w = 0;
  w = __builtin_amdgcn_cvt_pk_fp8_f32(x[0] * inv, x[1] * inv, w, false);
  w = __builtin_amdgcn_cvt_pk_fp8_f32(x[2] * inv, x[3] * inv, w, true);
  r.x = w;
  w = __builtin_amdgcn_cvt_pk_fp8_f32(x[4] * inv, x[5] * inv, w, false);
  w = __builtin_amdgcn_cvt_pk_fp8_f32(x[6] * inv, x[7] * inv, w, true);
  r.y = w;
  return r;
}

// Orders a wave's LDS writes before its other lanes' reads (the hardware keeps
// a wave's LDS accesses in order, so this binds the compiler only).
__device__ __forceinline__ void wave_lds_sync() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// The wave's place: false when it has no rows.
struct Place {
  int g, r0, first, n;      // head; batch row of the window's row 0; first live position; live slots' end
  int p0;                   // the unit's first position
  int L;
  size_t page;              // page * Hkv + g
  int s0;                   // the unit's first slot in its page
};
__device__ __forceinline__ bool place(const KvLaunch& p, Place& w) {
  const int sg = blockIdx.y * 4 + (threadIdx.x >> 6);
  if (sg >= p.n_seq * p.Hkv) return false;
  const int slot = sg / p.Hkv;
  w.g = sg - slot * p.Hkv;
  const int b = p.seq_ids ? p.seq_ids[slot] : slot;
  w.L = min(max(p.ctx_lens[b], 0), p.slots);
  w.r0 = p.cu_q[b];
  const int end = w.L + min(p.cu_q[b + 1] - w.r0, p.max_q);
  w.p0 = (w.L & ~(kUnit - 1)) + kUnit * (int)blockIdx.x;
  if (w.p0 >= end) return false;
  w.first = max(w.L, w.p0);
  w.n = min(end, w.p0 + kUnit);
  const int col = min(w.p0 >> p.log2ps, p.max_pages - 1);
  const int pg = p.page_table[(size_t)b * p.max_pages + col];
  w.page = (size_t)min(max(pg, 0), p.num_pages - 1) * p.Hkv + w.g;
  w.s0 = w.p0 & (p.page_size - 1);
  return true;
}

template <typename DT, int D>
__global__ __launch_bounds__(256) void kv_append_kernel(KvLaunch p) {
  constexpr int LPT = D / 8, TPP = kWave / LPT;     // lanes per row, rows per pass
  constexpr int PITCH = kUnit + 4;                  // bytes of a channel's run in LDS
  __shared__ __attribute__((aligned(16))) uint8_t s_t[4][D * PITCH];
  Place w;
  if (!place(p, w)) return;                         // waves are independent: no barrier below
  const int lane = lane_id(), c = lane % LPT, tt = lane / LPT;
  uint8_t* lds = s_t[threadIdx.x >> 6];
  const int ps = p.page_size;
  uint8_t* kp = p.k_pages + w.page * D * ps;
  uint8_t* vp = p.v_pages + w.page * D * ps;
  uint8_t* sc = p.scales + w.page * 2 * ps;
  const bool whole = w.n - w.first == kUnit;
#pragma unroll
  for (int t0 = 0; t0 < kUnit; t0 += TPP) {
    const int o = t0 + tt, pos = w.p0 + o;
    const bool on = pos >= w.first && pos < w.n;
    if (!__any(on)) continue;
    const int row = w.r0 + (on ? pos : w.first) - w.L;
    float x[8];
    int byte;
    ld8<DT>(reinterpret_cast<const DT*>(p.k_in) + (size_t)row * p.k_stride + w.g * D + 8 * c, x);
    const uint2 kq = quantise<LPT>(x, true, &byte);
    if (on) {
      *reinterpret_cast<uint2*>(kp + ((size_t)(c >> 1) * ps + w.s0 + o) * 16 + 8 * (c & 1)) = kq;
      if (c == 0) sc[w.s0 + o] = (uint8_t)byte;
    }
    ld8<DT>(reinterpret_cast<const DT*>(p.v_in) + (size_t)row * p.v_stride + w.g * D + 8 * c, x);
    const uint2 vq = quantise<LPT>(x, false, &byte);
    if (on && c == 0) sc[ps + w.s0 + o] = (uint8_t)byte;
    if (whole) {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        lds[(8 * c + i) * PITCH + o] = (uint8_t)((i < 4 ? vq.x : vq.y) >> (8 * (i & 3)));
    } else if (on) {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        vp[(size_t)(8 * c + i) * ps + w.s0 + o] = (uint8_t)((i < 4 ? vq.x : vq.y) >> (8 * (i & 3)));
    }
  }
  if (!whole) return;
  wave_lds_sync();
  for (int d = lane; d < D; d += kWave) {
    uint4 run;
    const unsigned* s = reinterpret_cast<const unsigned*>(lds + d * PITCH);
    run.x = s[0];
    run.y = s[1];
    run.z = s[2];
    run.w = s[3];
    *reinterpret_cast<uint4*>(vp + (size_t)d * ps + w.s0) = run;
  }
}

template <typename DT, int D>
__global__ __launch_bounds__(256) void kv_read_kernel(KvLaunch p) {
  constexpr int PITCH = D + 8;                      // bytes of a slot's row in LDS
  __shared__ __attribute__((aligned(16))) uint8_t s_t[4][kUnit * PITCH];
  Place w;
  if (!place(p, w)) return;
  const int lane = lane_id();
  uint8_t* lds = s_t[threadIdx.x >> 6];
  const int ps = p.page_size;
  const uint8_t* kp = p.k_pages + w.page * D * ps;
  const uint8_t* vp = p.v_pages + w.page * D * ps;
  const uint8_t* sc = p.scales + w.page * 2 * ps;
  // values: a lane turns one channel's run of 16 slots
#pragma unroll
  for (int d0 = 0; d0 < D; d0 += kWave) {
    const uint4 run = ld16<uint4>(vp + (size_t)(d0 + lane) * ps + w.s0);
    const unsigned r[4] = {run.x, run.y, run.z, run.w};
#pragma unroll
    for (int o = 0; o < kUnit; ++o) lds[o * PITCH + d0 + lane] = (uint8_t)(r[o >> 2] >> (8 * (o & 3)));
  }
  // keys: a lane turns 16 channels of one slot
  constexpr int CH = D / 16;
#pragma unroll
  for (int e0 = 0; e0 < CH * kUnit; e0 += kWave) {
    const int e = e0 + lane, c = e % CH, o = e / CH, pos = w.p0 + o;
    if (pos < w.first || pos >= w.n) continue;
    const uint4 v = ld16<uint4>(kp + ((size_t)c * ps + w.s0 + o) * 16);
    const float f = scale_value(sc[w.s0 + o]);
    DT* dst = reinterpret_cast<DT*>(p.k_out) + (size_t)(w.r0 + pos - w.L) * p.k_stride + w.g * D + 16 * c;
    float x[8];
    values8(v.x, v.y, f, x);
    st8<DT>(dst, x);
    values8(v.z, v.w, f, x);
    st8<DT>(dst + 8, x);
  }
  wave_lds_sync();
  constexpr int LPT = D / 8;
#pragma unroll
  for (int e0 = 0; e0 < LPT * kUnit; e0 += kWave) {
    const int e = e0 + lane, c = e % LPT, o = e / LPT, pos = w.p0 + o;
    if (pos < w.first || pos >= w.n) continue;
    const uint2 v = *reinterpret_cast<const uint2*>(lds + o * PITCH + 8 * c);
    float x[8];
    values8(v.x, v.y, scale_value(sc[ps + w.s0 + o]), x);
    st8<DT>(reinterpret_cast<DT*>(p.v_out) + (size_t)(w.r0 + pos - w.L) * p.v_stride + w.g * D + 8 * c, x);
  }
}

}  // namespace

hipError_t launch_kv_q8(const KvLaunch& L, bool append, hipStream_t st) {
  trace_begin(st);
  // 16-slot units that a window can touch: its start may lie inside one
  const dim3 grid((L.max_q + 2 * (kUnit - 1)) / kUnit, (L.n_seq * L.Hkv + 3) / 4);
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(256), 0, st, L); };
  if (append) {
    if (L.dtype_bf16) {
      if (L.D == 128) go(kv_append_kernel<bf16, 128>); else go(kv_append_kernel<bf16, 64>);
    } else {
      if (L.D == 128) go(kv_append_kernel<float, 128>); else go(kv_append_kernel<float, 64>);
    }
  } else {
    if (L.dtype_bf16) {
      if (L.D == 128) go(kv_read_kernel<bf16, 128>); else go(kv_read_kernel<bf16, 64>);
    } else {
      if (L.D == 128) go(kv_read_kernel<float, 128>); else go(kv_read_kernel<float, 64>);
    }
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  trace_mark(st);
  return hipSuccess;
}

}  // namespace ipdv
