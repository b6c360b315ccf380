// Root-mean-square norm of every query and key head and their rotation by position, in one pass.
//
// A head of D elements is D/8 pairs of four-element pieces: piece p and the one that it is rotated with (half a rotary
// dim on, or right behind it where pairs lie side by side), so a lane rotates what it loaded itself and the only
// exchange is the sum of squares over the lanes of a head.  A wave takes one row: its lanes find the row's angles once
// for all heads.  Bound by HBM: every element is read and written once.
#include "fd_common.h"

namespace fd {

constexpr int RP_WAVES = 4;

typedef __attribute__((ext_vector_type(4))) unsigned short u16x4;
template <typename T> struct Four;
template <> struct Four<bf16_t> {
  static __device__ __forceinline__ void load(const bf16_t* p, float (&x)[4]) {
    const u16x4 w = *reinterpret_cast<const u16x4*>(p);
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = bf16_to_f32(w[e]);
  }
  static __device__ __forceinline__ void store(bf16_t* p, const float (&x)[4]) {
    u16x4 w;
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = f32_to_bf16(x[e]);
    *reinterpret_cast<u16x4*>(p) = w;
  }
};
template <> struct Four<float> {
  static __device__ __forceinline__ void load(const float* p, float (&x)[4]) {
    const f32x4 w = *reinterpret_cast<const f32x4*>(p);
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = w[e];
  }
  static __device__ __forceinline__ void store(float* p, const float (&x)[4]) {
    f32x4 w;
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = x[e];
    *reinterpret_cast<f32x4*>(p) = w;
  }
};

// LPH: lanes of a head (8, 16, 32), D <= 8 LPH.
template <typename T, int LPH, bool INTER>
__global__ __launch_bounds__(RP_WAVES * 64) void qk_norm_rope_kernel(fd_rope_args a, int heads_per_block) {
  __shared__ float2 angles[RP_WAVES][4 * LPH];          // (cos, sin)
  constexpr int AT_ONCE = 64 / LPH;                     // heads a wave takes at once
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int row = blockIdx.x * RP_WAVES + wave;
  const int half = a.rotary_dim / 2;
  const bool there = row < a.total_rows;
  if (there) {
    // The angle in turns, in fp64: positions times frequencies reach 1e6 radians, of which fp32 keeps 1e-1.
    const double pos = half > 0 ? (double)a.positions[row] * 0.15915494309189533577 : 0.0;
    for (int i = lane; i < half; i += 64) {
      double t = pos * (double)a.inv_freq[i];
      t -= rint(t);
      float s, c;
      sincospif(2.f * (float)t, &s, &c);
      angles[wave][i] = make_float2(c, s);
    }
  }
  __syncthreads();
  if (!there) return;
  const int D = a.head_dim, p = lane % LPH, sub = lane / LPH;
  const int rot_pairs = a.rotary_dim / 8;
  const bool active = p < D / 8, rotated = p < rot_pairs;
  // the two pieces of this lane: a rotary pair, or eight elements in a row
  int e0, e1;
  if (INTER || !rotated) { e0 = 8 * p; e1 = e0 + 4; }
  else { e0 = 4 * p; e1 = e0 + half; }
  float c[4], s[4], wq[8], wk[8];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float2 t = rotated ? angles[wave][4 * p + e] : make_float2(1.f, 0.f);
    c[e] = t.x; s[e] = t.y;
  }
  auto weights = [&](const void* w, float (&x)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = 1.f;
    if (!w || !active) return;
    float u[4], v[4];
    Four<T>::load(reinterpret_cast<const T*>(w) + e0, u);
    Four<T>::load(reinterpret_cast<const T*>(w) + e1, v);
#pragma unroll
    for (int e = 0; e < 4; ++e) { x[e] = u[e]; x[4 + e] = v[e]; }
  };
  weights(a.q_weight, wq);
  weights(a.k_weight, wk);
  const int Hq = a.num_q_heads, Hkv = a.num_kv_heads, heads = Hq + Hkv + (a.v ? Hkv : 0);
  const int h_end = min(heads, ((int)blockIdx.y + 1) * heads_per_block);
  const float inv_d = 1.f / (float)D;
  for (int h0 = blockIdx.y * heads_per_block; h0 < h_end; h0 += AT_ONCE) {
    const int h = h0 + sub;
    const bool on = active && h < h_end;
    const int kind = h < Hq ? 0 : h < Hq + Hkv ? 1 : 2;
    const T* src; T* dst;
    if (kind == 0) {
      src = reinterpret_cast<const T*>(a.q) + (long long)row * a.q_stride_row + (long long)h * a.q_stride_head;
      dst = reinterpret_cast<T*>(a.q_out) + ((long long)row * Hq + h) * D;
    } else if (kind == 1) {
      src = reinterpret_cast<const T*>(a.k) + (long long)row * a.k_stride_row + (long long)(h - Hq) * a.k_stride_head;
      dst = reinterpret_cast<T*>(a.k_out) + ((long long)row * Hkv + h - Hq) * D;
    } else {
      src = reinterpret_cast<const T*>(a.v) + (long long)row * a.v_stride_row + (long long)(h - Hq - Hkv) * a.v_stride_head;
      dst = reinterpret_cast<T*>(a.v_out) + ((long long)row * Hkv + h - Hq - Hkv) * D;
    }
    float x[4] = {}, y[4] = {};
    if (on) { Four<T>::load(src + e0, x); Four<T>::load(src + e1, y); }
    float sq = 0.f;
#pragma unroll
    for (int e = 0; e < 4; ++e) sq += x[e] * x[e] + y[e] * y[e];
#pragma unroll
    for (int d = 1; d < LPH; d <<= 1) sq += __shfl_xor(sq, d);
    if (!on) continue;
    if (kind == 2) { Four<T>::store(dst + e0, x); Four<T>::store(dst + e1, y); continue; }
    const bool normed = kind == 0 ? a.q_weight != nullptr : a.k_weight != nullptr;
    if (normed) {
      const float r = 1.f / sqrtf(sq * inv_d + a.eps);
#pragma unroll
      for (int e = 0; e < 4; ++e) { x[e] *= r * (kind == 0 ? wq[e] : wk[e]); y[e] *= r * (kind == 0 ? wq[4 + e] : wk[4 + e]); }
    }
    if (rotated) {
      if (INTER) {
        const float u0 = x[0] * c[0] - x[1] * s[0], u1 = x[1] * c[0] + x[0] * s[0];
        const float u2 = x[2] * c[1] - x[3] * s[1], u3 = x[3] * c[1] + x[2] * s[1];
        const float w0 = y[0] * c[2] - y[1] * s[2], w1 = y[1] * c[2] + y[0] * s[2];
        const float w2 = y[2] * c[3] - y[3] * s[3], w3 = y[3] * c[3] + y[2] * s[3];
        x[0] = u0; x[1] = u1; x[2] = u2; x[3] = u3; y[0] = w0; y[1] = w1; y[2] = w2; y[3] = w3;
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float u = x[e] * c[e] - y[e] * s[e];
          y[e] = y[e] * c[e] + x[e] * s[e];
          x[e] = u;
        }
      }
    }
    Four<T>::store(dst + e0, x);
    Four<T>::store(dst + e1, y);
  }
}

template <typename T, int LPH>
static void launch_rope(const fd_rope_args& a, dim3 grid, int per, hipStream_t st) {
  if (a.interleaved) hipLaunchKernelGGL((qk_norm_rope_kernel<T, LPH, true>), grid, dim3(RP_WAVES * 64), 0, st, a, per);
  else hipLaunchKernelGGL((qk_norm_rope_kernel<T, LPH, false>), grid, dim3(RP_WAVES * 64), 0, st, a, per);
}

hipError_t run_qk_norm_rope(const fd_rope_args& a, hipStream_t st) {
  const int heads = a.num_q_heads + a.num_kv_heads + (a.v ? a.num_kv_heads : 0);
  const int lph = a.head_dim <= 64 ? 8 : a.head_dim <= 128 ? 16 : 32;
  const int at_once = 64 / lph;
  const int blocks = (a.total_rows + RP_WAVES - 1) / RP_WAVES;
  // few rows: the heads of a row are shared out to more work-groups
  int per = (heads + at_once - 1) / at_once * at_once;
  while (per > at_once && (long long)blocks * ((heads + per - 1) / per) < 1024) per -= at_once;
  const dim3 grid(blocks, (heads + per - 1) / per);
  if (a.dtype == FD_BF16) {
    if (lph == 8) launch_rope<bf16_t, 8>(a, grid, per, st);
    else if (lph == 16) launch_rope<bf16_t, 16>(a, grid, per, st);
    else launch_rope<bf16_t, 32>(a, grid, per, st);
  } else {
    if (lph == 8) launch_rope<float, 8>(a, grid, per, st);
    else if (lph == 16) launch_rope<float, 16>(a, grid, per, st);
    else launch_rope<float, 32>(a, grid, per, st);
  }
  return hipGetLastError();
}

}  // namespace fd
