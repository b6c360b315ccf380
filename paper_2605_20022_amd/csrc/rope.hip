// Root-mean-square norm of every query and key head and their rotation by position, in one pass.
//
// A head of D elements is cut into pairs of pieces of E = 8 or 4 elements: a piece and the one that it is rotated with (half a rotary
// dim on, or right behind it where pairs lie side by side), so a lane rotates what it loaded itself and the only
// exchange is the sum of squares over the lanes of a head.  A wave takes one row: its lanes find the row's angles once
// for all heads.  Bound by HBM: every element is read and written once; bf16 pieces of eight are loads of sixteen bytes (8192 rows of
// 40 heads of 128: 38.3 us a call, 4.4 TB/s, where a plain copy reaches 5.1; with pieces of four 40.7).
#include "fd_common.h"

namespace fd {

constexpr int RP_WAVES = 4;

typedef __attribute__((ext_vector_type(4))) unsigned short u16x4;
template <typename T, int E> struct Piece;
template <> struct Piece<bf16_t, 4> {
  u16x4 w;
  __device__ __forceinline__ void load(const bf16_t* p) { w = *reinterpret_cast<const u16x4*>(p); }
  __device__ __forceinline__ void copy(bf16_t* p) const { *reinterpret_cast<u16x4*>(p) = w; }
  __device__ __forceinline__ void get(float (&x)[4]) const {
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
template <> struct Piece<bf16_t, 8> {
  u32x4 w;
  __device__ __forceinline__ void load(const bf16_t* p) { w = *reinterpret_cast<const u32x4*>(p); }
  __device__ __forceinline__ void copy(bf16_t* p) const { *reinterpret_cast<u32x4*>(p) = w; }
  __device__ __forceinline__ void get(float (&x)[8]) const {
#pragma unroll
    for (int e = 0; e < 4; ++e) { x[2 * e] = __uint_as_float(w[e] << 16); x[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u); }
  }
  static __device__ __forceinline__ void store(bf16_t* p, const float (&x)[8]) {
    typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
    typedef __attribute__((ext_vector_type(2))) float f32x2;
    u32x4 w;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const f32x2 f = {x[2 * e], x[2 * e + 1]};
      w[e] = __builtin_bit_cast(unsigned, __builtin_convertvector(f, bf16x2));       // round to nearest even
    }
    *reinterpret_cast<u32x4*>(p) = w;
  }
};
template <> struct Piece<float, 4> {
  f32x4 w;
  __device__ __forceinline__ void load(const float* p) { w = *reinterpret_cast<const f32x4*>(p); }
  __device__ __forceinline__ void copy(float* p) const { *reinterpret_cast<f32x4*>(p) = w; }
  __device__ __forceinline__ void get(float (&x)[4]) const {
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = w[e];
  }
  static __device__ __forceinline__ void store(float* p, const float (&x)[4]) { *reinterpret_cast<f32x4*>(p) = f32x4{x[0], x[1], x[2], x[3]}; }
};

// LPH: lanes of a head (8, 16, 32), D <= 2 E LPH.  AHEAD: heads of a lane that are requested before the first is used.
template <typename T, int E, int LPH, bool INTER>
__global__ __launch_bounds__(RP_WAVES * 64) void qk_norm_rope_kernel(fd_rope_args a, int heads_per_block) {
  __shared__ float2 angles[RP_WAVES][E * LPH];          // (cos, sin)
  constexpr int AT_ONCE = 64 / LPH;                     // heads a wave takes at once
  constexpr int AHEAD = 2;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int row = blockIdx.x * RP_WAVES + wave;
  const int half = a.rotary_dim / 2;
  const bool there = row < a.total_rows;
  const int D = a.head_dim, p = lane % LPH, sub = lane / LPH;
  const bool active = p < D / (2 * E), rotated = p < a.rotary_dim / (2 * E);
  // the two pieces of this lane: a rotary pair, or 2 E elements in a row
  int e0, e1;
  if (INTER || !rotated) { e0 = 2 * E * p; e1 = e0 + E; }
  else { e0 = E * p; e1 = e0 + half; }
  const int Hq = a.num_q_heads, Hkv = a.num_kv_heads, heads = Hq + Hkv + (a.v ? Hkv : 0);
  const int h_first = blockIdx.y * heads_per_block + sub, h_end = min(heads, ((int)blockIdx.y + 1) * heads_per_block);
  typedef Piece<T, E> P;
  P in[AHEAD][2];
  auto request = [&](P (&w)[2], int h) {                // (heads past the end: the first again)
    if (!there || !active) return;
    if (h >= h_end) h = h_first < h_end ? h_first : 0;
    const T* src;
    if (h < Hq) src = reinterpret_cast<const T*>(a.q) + (long long)row * a.q_stride_row + (long long)h * a.q_stride_head;
    else if (h < Hq + Hkv) src = reinterpret_cast<const T*>(a.k) + (long long)row * a.k_stride_row + (long long)(h - Hq) * a.k_stride_head;
    else src = reinterpret_cast<const T*>(a.v) + (long long)row * a.v_stride_row + (long long)(h - Hq - Hkv) * a.v_stride_head;
    w[0].load(src + e0);
    w[1].load(src + e1);
  };
#pragma unroll
  for (int u = 0; u < AHEAD; ++u) request(in[u], h_first + u * AT_ONCE);
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
  float c[E], s[E], wq[2][E], wk[2][E];
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const float2 t = rotated ? angles[wave][E * p + e] : make_float2(1.f, 0.f);
    c[e] = t.x; s[e] = t.y;
  }
  auto weights = [&](const void* w, float (&x)[2][E]) {
#pragma unroll
    for (int e = 0; e < E; ++e) x[0][e] = x[1][e] = 1.f;
    if (!w || !active) return;
    P u;
    u.load(reinterpret_cast<const T*>(w) + e0); u.get(x[0]);
    u.load(reinterpret_cast<const T*>(w) + e1); u.get(x[1]);
  };
  weights(a.q_weight, wq);
  weights(a.k_weight, wk);
  const float inv_d = 1.f / (float)D;
  auto head = [&](const P (&w)[2], int h) {
    const bool on = active && h < h_end, is_q = h < Hq, is_v = h >= Hq + Hkv;
    float x[E], y[E];
    w[0].get(x);
    w[1].get(y);
    float sq = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) sq += x[e] * x[e] + y[e] * y[e];
    if (!active) sq = 0.f;
#pragma unroll
    for (int d = 1; d < LPH; d <<= 1) sq += __shfl_xor(sq, d);
    if (!on) return;
    if (!is_v) {
      if (is_q ? a.q_weight != nullptr : a.k_weight != nullptr) {
        const float r = 1.f / sqrtf(sq * inv_d + a.eps);
#pragma unroll
        for (int e = 0; e < E; ++e) { x[e] *= r * (is_q ? wq[0][e] : wk[0][e]); y[e] *= r * (is_q ? wq[1][e] : wk[1][e]); }
      }
      if (rotated) {
        if (INTER) {
#pragma unroll
          for (int e = 0; e < E; e += 2) {               // angles e / 2 of x's pairs, E / 2 + e / 2 of y's
            const float u = x[e] * c[e / 2] - x[e + 1] * s[e / 2], v = y[e] * c[E / 2 + e / 2] - y[e + 1] * s[E / 2 + e / 2];
            x[e + 1] = x[e + 1] * c[e / 2] + x[e] * s[e / 2];
            y[e + 1] = y[e + 1] * c[E / 2 + e / 2] + y[e] * s[E / 2 + e / 2];
            x[e] = u; y[e] = v;
          }
        } else {
#pragma unroll
          for (int e = 0; e < E; ++e) {
            const float u = x[e] * c[e] - y[e] * s[e];
            y[e] = y[e] * c[e] + x[e] * s[e];
            x[e] = u;
          }
        }
      }
    }
    T* dst;
    if (is_q) dst = reinterpret_cast<T*>(a.q_out) + ((long long)row * Hq + h) * D;
    else if (!is_v) dst = reinterpret_cast<T*>(a.k_out) + ((long long)row * Hkv + h - Hq) * D;
    else {                                               // bit by bit: a conversion makes a signalling NaN a quiet one
      dst = reinterpret_cast<T*>(a.v_out) + ((long long)row * Hkv + h - Hq - Hkv) * D;
      w[0].copy(dst + e0);
      w[1].copy(dst + e1);
      return;
    }
    P::store(dst + e0, x);
    P::store(dst + e1, y);
  };
  for (int h = h_first; h - sub < h_end; h += AHEAD * AT_ONCE)
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      head(in[u], h + u * AT_ONCE);
      request(in[u], h + (u + AHEAD) * AT_ONCE);
    }
}

template <typename T, int E, int LPH>
static void launch_rope(const fd_rope_args& a, dim3 grid, int per, hipStream_t st) {
  if (a.interleaved) hipLaunchKernelGGL((qk_norm_rope_kernel<T, E, LPH, true>), grid, dim3(RP_WAVES * 64), 0, st, a, per);
  else hipLaunchKernelGGL((qk_norm_rope_kernel<T, E, LPH, false>), grid, dim3(RP_WAVES * 64), 0, st, a, per);
}

hipError_t run_qk_norm_rope(const fd_rope_args& a, hipStream_t st) {
  const int heads = a.num_q_heads + a.num_kv_heads + (a.v ? a.num_kv_heads : 0);
  // bf16 in pieces of eight where the head and its rotary part are whole pairs of them and every row is 16-byte aligned
  const bool eight = a.dtype == FD_BF16 && a.head_dim % 16 == 0 && a.rotary_dim % 16 == 0 &&
                     (a.q_stride_row | a.q_stride_head | a.k_stride_row | a.k_stride_head | (a.v ? a.v_stride_row | a.v_stride_head : 0)) % 8 == 0;
  const int lanes = a.head_dim / (eight ? 16 : 8);
  const int lph = lanes <= 8 ? 8 : lanes <= 16 ? 16 : 32;
  const int at_once = 64 / lph;
  const int blocks = (a.total_rows + RP_WAVES - 1) / RP_WAVES;
  // few rows: the heads of a row are shared out to more work-groups
  int per = (heads + at_once - 1) / at_once * at_once;
  while (per > at_once && (long long)blocks * ((heads + per - 1) / per) < 1024) per -= at_once;
  const dim3 grid(blocks, (heads + per - 1) / per);
  if (a.dtype == FD_BF16 && eight) {
    if (lph == 8) launch_rope<bf16_t, 8, 8>(a, grid, per, st);
    else launch_rope<bf16_t, 8, 16>(a, grid, per, st);
  } else if (a.dtype == FD_BF16) {
    if (lph == 8) launch_rope<bf16_t, 4, 8>(a, grid, per, st);
    else if (lph == 16) launch_rope<bf16_t, 4, 16>(a, grid, per, st);
    else launch_rope<bf16_t, 4, 32>(a, grid, per, st);
  } else {
    if (lph == 8) launch_rope<float, 4, 8>(a, grid, per, st);
    else if (lph == 16) launch_rope<float, 4, 16>(a, grid, per, st);
    else launch_rope<float, 4, 32>(a, grid, per, st);
  }
  return hipGetLastError();
}

}  // namespace fd
