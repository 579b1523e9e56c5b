// Causal attention of packed prompts and the attention weight its tokens receive, on the ALUs in float32.
//
//   s_ij = scale q_i . k_j (j <= i),  lse_i = log sum_j exp s_ij,  out_i = sum_j exp(s_ij - lse_i) v_j
//   acc_j = sum over a group's heads and the queries i >= j of exp(s_ij - lse_i)
//
// One CTA owns 64 query rows of one head (attention) or 64 key rows of one key/value head (weights) and walks over the
// blocks of 64 rows on the other side. 256 threads as 16 x 16, 4 x 4 logits each: the tiles lie transposed in shared memory, so
// that per element of the head dimension a thread reads two 16-byte pieces for 16 multiply-adds. Rows outside the sequence
// are read as zeros and never stored.
#pragma once

#include "packed.cuh"

namespace adore {

constexpr int kPsBlock = 64;
constexpr int kPsThreads = 256;
constexpr int kPsPitch = kPsBlock + 4;     // floats between the rows of a transposed tile

template <int DH>
constexpr size_t prompt_simt_smem() { return size_t(2 * DH * kPsPitch + kPsBlock * DH) * sizeof(float); }
template <int DH>
constexpr size_t prompt_weights_simt_smem() { return size_t(2 * DH * kPsPitch + kPsBlock) * sizeof(float); }

// 64 rows from `row0` of a sequence of `len` rows, transposed to dst[e][row]; lanes of a warp take 8 rows x 4 pieces.
template <typename T, int DH>
__device__ __forceinline__ void load_transposed(float* dst, const T* src, long long row_stride, int row0, int len) {
  for (int i = threadIdx.x; i < kPsBlock * (DH / 4); i += kPsThreads) {
    const int low = i & 31, r = (low & 7) + 8 * ((i >> 5) & 7), c = (low >> 3) + 4 * (i >> 8);
    float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
    if (row0 + r < len) x = load4(src + (row0 + r) * row_stride + 4 * c);
    float* d = dst + 4 * c * kPsPitch + r;
    d[0] = x.x; d[kPsPitch] = x.y; d[2 * kPsPitch] = x.z; d[3 * kPsPitch] = x.w;
  }
}

// 4 x 4 logits of rows 4 ty.. of A against rows 4 tx.. of B, both transposed.
template <int DH>
__device__ __forceinline__ void tile_product(const float* a, const float* b, int ty, int tx, float (&s)[4][4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) s[i][j] = 0.f;
#pragma unroll 8
  for (int e = 0; e < DH; ++e) {
    const float4 x = *reinterpret_cast<const float4*>(a + e * kPsPitch + 4 * ty);
    const float4 y = *reinterpret_cast<const float4*>(b + e * kPsPitch + 4 * tx);
    const float xs[4] = {x.x, x.y, x.z, x.w}, ys[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) s[i][j] = fmaf(xs[i], ys[j], s[i][j]);
  }
}

template <typename T, int DH>
__global__ void __launch_bounds__(kPsThreads, 2) prompt_attention_simt_kernel(const PackedParams p, const T* q, const T* k,
                                                                              const T* v, T* out, float* lse) {
  extern __shared__ __align__(16) float prompt_smem[];
  float* qt = prompt_smem;
  float* kt = qt + DH * kPsPitch;          // later the weights of the block, transposed
  float* vs = kt + DH * kPsPitch;
  __shared__ PackedTile tile;
  __shared__ int found;
  const int h = blockIdx.x % p.H, g = h / p.group;
  if (threadIdx.x < 32) {
    PackedTile t{};
    const bool ok = find_packed_tile<kPsBlock>(p.seq_start, p.S, p.total, blockIdx.x / p.H, p.err, t);
    if (threadIdx.x == 0) { tile = t; found = ok; }
  }
  __syncthreads();
  if (!found) return;
  const int len = tile.len, q0 = tile.index * kPsBlock;
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  const T* qs = q + tile.start * p.q_row + h * p.q_head;
  const T* ks = k + tile.start * p.k_row + g * p.k_head;
  const T* vsrc = v + tile.start * p.v_row + g * p.v_head;
  load_transposed<T, DH>(qt, qs, p.q_row, q0, len);
  constexpr int NV = DH / 64;              // 16-byte pieces of a value row per thread
  float o[4][4 * NV], m[4], l[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    m[i] = -INFINITY;
    l[i] = 0.f;
#pragma unroll
    for (int j = 0; j < 4 * NV; ++j) o[i][j] = 0.f;
  }
  const float c = p.scale * 1.4426950408889634f;      // logits in units of log 2
  for (int kb = 0; kb <= tile.index; ++kb) {
    __syncthreads();
    load_transposed<T, DH>(kt, ks, p.k_row, kb * kPsBlock, len);
    for (int i = threadIdx.x; i < kPsBlock * (DH / 4); i += kPsThreads) {
      const int r = i / (DH / 4), e = i % (DH / 4);
      float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
      if (kb * kPsBlock + r < len) x = load4(vsrc + (kb * kPsBlock + r) * p.v_row + 4 * e);
      *reinterpret_cast<float4*>(vs + r * DH + 4 * e) = x;
    }
    __syncthreads();
    float s[4][4];
    tile_product<DH>(qt, kt, ty, tx, s);
    const bool diagonal = kb == tile.index;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float top = -INFINITY;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        s[i][j] = diagonal && 4 * tx + j > 4 * ty + i ? -INFINITY : s[i][j] * c;
        top = fmaxf(top, s[i][j]);
      }
#pragma unroll
      for (int w = 8; w > 0; w >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, w));
      const float now = fmaxf(m[i], top), f = exp2f(m[i] - now);      // a row's own position is in its block: now is finite
      m[i] = now;
      l[i] *= f;
#pragma unroll
      for (int j = 0; j < 4 * NV; ++j) o[i][j] *= f;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        s[i][j] = exp2f(s[i][j] - now);
        l[i] += s[i][j];
      }
    }
    __syncthreads();                       // every thread has read the key tile
#pragma unroll
    for (int j = 0; j < 4; ++j)
      *reinterpret_cast<float4*>(kt + (4 * tx + j) * kPsPitch + 4 * ty) = make_float4(s[0][j], s[1][j], s[2][j], s[3][j]);
    __syncthreads();
#pragma unroll 4
    for (int r = 0; r < kPsBlock; ++r) {
      const float4 w = *reinterpret_cast<const float4*>(kt + r * kPsPitch + 4 * ty);
      const float ws[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
      for (int n = 0; n < NV; ++n) {
        const float4 x = *reinterpret_cast<const float4*>(vs + r * DH + 64 * n + 4 * tx);
        const float xs[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j) o[i][4 * n + j] = fmaf(ws[i], xs[j], o[i][4 * n + j]);
      }
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
#pragma unroll
    for (int w = 8; w > 0; w >>= 1) l[i] += __shfl_xor_sync(0xffffffffu, l[i], w);
    const int r = q0 + 4 * ty + i;
    if (r >= len) continue;
    const float inv = 1.f / l[i];
    T* dst = out + (tile.start + r) * p.out_row + h * p.out_head;
#pragma unroll
    for (int n = 0; n < NV; ++n)
      store4(dst + 64 * n + 4 * tx, make_float4(o[i][4 * n] * inv, o[i][4 * n + 1] * inv, o[i][4 * n + 2] * inv, o[i][4 * n + 3] * inv));
    if (lse != nullptr && tx == 0) lse[size_t(h) * p.total + tile.start + r] = m[i] * 0.6931471805599453f + logf(l[i]);
  }
}

template <typename T, int DH>
__global__ void __launch_bounds__(kPsThreads, 2) prompt_weights_simt_kernel(const PackedParams p, const T* q, const T* k,
                                                                            const float* lse, int window, float* acc) {
  extern __shared__ __align__(16) float prompt_smem[];
  float* kt = prompt_smem;
  float* qt = kt + DH * kPsPitch;
  float* ls = qt + DH * kPsPitch;
  __shared__ PackedTile tile;
  __shared__ int found;
  const int g = blockIdx.x % p.Hk;
  if (threadIdx.x < 32) {
    PackedTile t{};
    const bool ok = find_packed_tile<kPsBlock>(p.seq_start, p.S, p.total, blockIdx.x / p.Hk, p.err, t);
    if (threadIdx.x == 0) { tile = t; found = ok; }
  }
  __syncthreads();
  if (!found) return;
  const int len = tile.len, blocks = (len + kPsBlock - 1) / kPsBlock;
  const int kb = blocks - 1 - tile.index, k0 = kb * kPsBlock;      // early keys are seen by most queries
  const int first = window > 0 ? max(0, len - window) : 0;         // first query that counts
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  load_transposed<T, DH>(kt, k + tile.start * p.k_row + g * p.k_head, p.k_row, k0, len);
  const float c = p.scale * 1.4426950408889634f;
  float sum[4] = {0.f, 0.f, 0.f, 0.f};
  for (int h = g * p.group; h < (g + 1) * p.group; ++h) {
    const float* lrow = lse + size_t(h) * p.total + tile.start;
    for (int qb = max(kb, first / kPsBlock); qb < blocks; ++qb) {
      const int q0 = qb * kPsBlock;
      __syncthreads();
      load_transposed<T, DH>(qt, q + tile.start * p.q_row + h * p.q_head, p.q_row, q0, len);
      if (threadIdx.x < kPsBlock) {
        const int i = q0 + threadIdx.x;
        ls[threadIdx.x] = i >= first && i < len ? lrow[i] * 1.4426950408889634f : INFINITY;    // infinite: weight 0
      }
      __syncthreads();
      float s[4][4];
      tile_product<DH>(kt, qt, ty, tx, s);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float part = 0.f;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float w = exp2f(fmaf(s[i][j], c, -ls[4 * tx + j]));
          part += qb == kb && 4 * tx + j < 4 * ty + i ? 0.f : w;
        }
        sum[i] += part;
      }
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
#pragma unroll
    for (int w = 8; w > 0; w >>= 1) sum[i] += __shfl_xor_sync(0xffffffffu, sum[i], w);
    const int r = k0 + 4 * ty + i;
    if (tx == 0 && r < len) acc[size_t(g) * p.total + tile.start + r] = sum[i];
  }
}

}  // namespace adore
