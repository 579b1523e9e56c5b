// Decode attention over 4-bit rows: one warp per (sequence, query head), the head dimension spread over the lanes, one slot
// at a time with a running maximum and sum.
#pragma once

#include "q4.cuh"

namespace adore {

template <typename T, int DH>
__global__ void __launch_bounds__(32) q4_attention_simple_kernel(const Q4Rows c, int H, int Hk, int C, int P, float scale, const T* q,
                                                                 const T* k_new, const T* v_new, const int* slot_pos, T* out,
                                                                 float* weights) {
  const int bh = blockIdx.x, b = bh / H, g = (bh % H) / (H / Hk), lane = threadIdx.x;
  const size_t r = size_t(b) * Hk + g;
  constexpr int LPR = DH / 8;
  const int j = lane % LPR;
  const bool on = lane < LPR;
  float qx[8], o[8];
  load8(q + size_t(bh) * DH + 8 * j, qx);
  for (int e = 0; e < 8; ++e) o[e] = 0.f;
  float m = -INFINITY, l = 0.f;
  float* w = weights != nullptr ? weights + size_t(bh) * (size_t(C) + 1) : nullptr;
  for (int s = 0; s <= C; ++s) {
    float kx[8], vx[8];
    bool have;
    if (s < C) {
      have = slot_pos[r * C + s] >= 0;
      if (have) {
        const uint32_t kw = c.k[(r * P + s) * (DH / 8) + q4_k_word<DH>(j)];
        const uint32_t* vp = c.v + (r * (P / 2) + s / 2) * (DH / 4) + q4_v_word<DH>(j);
        const int sh = (s & 1) * 16;
        const uint32_t vw = ((vp[0] >> sh) & 0xffffu) | ((vp[DH / 32] >> sh) << 16);
        const float2 ks = __bfloat1622float2(c.kp[(r * P + s) * (DH / kQ4Group) + (j >> 3)]);
        const float2 vs = __bfloat1622float2(c.vp[(r * P + s) * (DH / kQ4Group) + (j >> 3)]);
        for (int e = 0; e < 8; ++e) {
          kx[e] = fmaf(float((kw >> (4 * e)) & 15u), ks.x, ks.y);
          vx[e] = fmaf(float((vw >> (4 * e)) & 15u), vs.x, vs.y);
        }
      }
    } else {
      have = k_new != nullptr;
      if (have) {
        load8(k_new + r * DH + 8 * j, kx);
        load8(v_new + r * DH + 8 * j, vx);
      }
    }
    float x = -INFINITY;
    if (have) {
      float d = 0.f;
      for (int e = 0; e < 8; ++e) d = fmaf(qx[e], kx[e], d);
      x = warp_sum(on ? d : 0.f) * scale;
      const float now = fmaxf(m, x), f = expf(m - now), p = expf(x - now);
      m = now;
      l = l * f + p;
      for (int e = 0; e < 8; ++e) o[e] = o[e] * f + p * vx[e];
    }
    if (w != nullptr && lane == 0) w[s] = x;
  }
  const float inv = l > 0.f ? 1.f / l : 0.f;
  for (int e = 0; e < 8; ++e) o[e] *= inv;
  if (on) store8(out + size_t(bh) * DH + 8 * j, o);
  __syncwarp();
  if (w != nullptr)
    for (int s = lane; s <= C; s += 32) w[s] = w[s] == -INFINITY ? 0.f : expf(w[s] - m) * inv;
}

}  // namespace adore
