// Eviction by accumulated attention weight: the choice of a prompt's kept tokens, their rows in 4 bits, and the step that
// admits one new token.
#pragma once

#include "packed.cuh"
#include "q4.cuh"

namespace adore {

constexpr int kEvictThreads = 512;
constexpr int kEvictWarps = kEvictThreads / 32;

// Order of values: NaN below every number, both zeros equal.
__device__ __forceinline__ uint32_t evict_key(float x) {
  if (x != x) return 0u;
  return float_key(x == 0.f ? 0.f : x);
}

// Exclusive prefix of a flag over the CTA's threads; `total` gets the sum. Two barriers.
__device__ __forceinline__ int block_rank(bool flag, int* warp_counts, int& total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const unsigned b = __ballot_sync(0xffffffffu, flag);
  if (lane == 0) warp_counts[warp] = __popc(b);
  __syncthreads();
  int mine = lane < kEvictWarps ? warp_counts[lane] : 0;
  total = warp_sum(mine);
  const int before = warp_sum(lane < warp ? mine : 0);
  __syncthreads();
  return before + __popc(b & ((1u << lane) - 1u));
}

// Which tokens stay: one CTA per (sequence, key/value head). The threshold is found by a radix select over the older tokens'
// keys, 8 bits a pass; then one pass in ascending position hands out the slots.
__global__ void __launch_bounds__(kEvictThreads) evict_select_kernel(const int* seq_start, int total, int Hk, int C, int recent,
                                                                     const float* acc, int* slot_pos, float* slot_acc, int* length,
                                                                     unsigned* err) {
  __shared__ unsigned hist[256];
  __shared__ unsigned s_prefix, s_need;
  __shared__ int warp_counts[kEvictWarps];
  const int s = blockIdx.x / Hk, g = blockIdx.x % Hk;
  const int n = packed_len(seq_start, s, total, err);
  const float* a = acc + size_t(g) * total + (n > 0 ? seq_start[s] : 0);
  int* pos = slot_pos + size_t(blockIdx.x) * C;
  float* val = slot_acc + size_t(blockIdx.x) * C;
  if (threadIdx.x == 0) length[blockIdx.x] = n;
  const int kept = min(n, C);
  for (int i = kept + threadIdx.x; i < C; i += kEvictThreads) { pos[i] = -1; val[i] = 0.f; }
  if (n <= C) {
    for (int i = threadIdx.x; i < n; i += kEvictThreads) { pos[i] = i; val[i] = a[i]; }
    return;
  }
  const int older = n - recent;                 // n > C >= recent
  unsigned need = unsigned(C - recent), prefix = 0;
  for (int shift = 24; shift >= 0 && need > 0; shift -= 8) {
    if (threadIdx.x < 256) hist[threadIdx.x] = 0;
    __syncthreads();
    const unsigned mask = shift == 24 ? 0u : ~0u << (shift + 8);
    for (int i = threadIdx.x; i < older; i += kEvictThreads) {
      const uint32_t key = evict_key(a[i]);
      if ((key & mask) == prefix) atomicAdd(&hist[(key >> shift) & 255u], 1u);
    }
    __syncthreads();
    if (threadIdx.x == 0) {
      unsigned left = need;
      int d = 255;
      while (d > 0 && hist[d] < left) left -= hist[d--];
      s_need = left;
      s_prefix = prefix | (unsigned(d) << shift);
    }
    __syncthreads();
    need = s_need;
    prefix = s_prefix;
  }
  // keys above `prefix` stay, and of the keys equal to it the first `need`
  const bool any = C > recent;
  int ties = 0, out = 0;
  for (int i0 = 0; i0 < n; i0 += kEvictThreads) {
    const int i = i0 + threadIdx.x;
    const float x = i < n ? a[i] : 0.f;
    const uint32_t key = evict_key(x);
    const bool old = i < older, tie = old && any && key == prefix;
    int sum;
    const int rank = ties + block_rank(tie, warp_counts, sum);
    ties += sum;
    const bool keep = i < n && (!old || (any && key > prefix) || (tie && rank < int(need)));
    const int at = out + block_rank(keep, warp_counts, sum);
    out += sum;
    if (keep && at < C) { pos[at] = i; val[at] = x; }
  }
}

// Rows of the kept tokens in 4 bits; empty slots and the padding behind slot C - 1 get zeros. dh / 8 lanes per row.
template <typename T, int DH>
__global__ void __launch_bounds__(256) evict_pack_kernel(const PackedParams p, const T* k, const T* v, const int* slot_pos,
                                                         const int* length, int C, int P, const Q4Rows c) {
  constexpr int LPR = DH / 8, ROWS = 256 / LPR;
  const size_t r = blockIdx.y;
  const int slot = blockIdx.x * ROWS + threadIdx.x / LPR, j = threadIdx.x % LPR;
  const int s = int(r) / p.Hk, g = int(r) % p.Hk;
  int t = slot < C ? slot_pos[r * C + slot] : -1;
  if (t >= length[r]) t = -1;
  float kx[8], vx[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) kx[e] = vx[e] = 0.f;
  if (t >= 0) {
    const long long row = p.seq_start[s] + t;
    load8(k + row * p.k_row + g * p.k_head + 8 * j, kx);
    load8(v + row * p.v_row + g * p.v_head + 8 * j, vx);
  }
  __nv_bfloat162 kpair, vpair;
  const uint32_t kw = q4_encode8(kx, kpair), vw = q4_encode8(vx, vpair);
  if (slot < P) q4_store_piece<DH>(c, r, P, slot, j, kw, kpair, vw, vpair);
}

// One decode step of one (sequence, key/value head): adds the step's weights, picks the slot, writes the new row.
template <typename T, int DH>
__global__ void __launch_bounds__(256) evict_step_kernel(const float* weights, const T* k_new, const T* v_new, int H, int Hk, int C,
                                                         int P, int recent, const Q4Rows c, int* slot_pos, float* slot_acc, int* length,
                                                         int* admit_slot, int* evicted_pos, unsigned* err) {
  __shared__ unsigned long long best[8];
  const int r = blockIdx.x, b = r / Hk, g = r % Hk, group = H / Hk, lane = threadIdx.x & 31;
  const int now = length[r];
  if (now < 0) {
    if (threadIdx.x == 0) { admit_slot[r] = -1; evicted_pos[r] = -1; }
    return;
  }
  const float* w = weights + (size_t(b) * H + size_t(g) * group) * (size_t(C) + 1);
  int* pos = slot_pos + size_t(r) * C;
  float* val = slot_acc + size_t(r) * C;
  const long long newest = (long long)now - recent;
  // (0, slot) of an empty slot < (1, value, slot) of a token that may go < all others
  unsigned long long mine = ~0ull;
  for (int i = threadIdx.x; i < C; i += 256) {
    const int at = pos[i];
    if (at < 0) { mine = min(mine, (unsigned long long)i); continue; }
    double sum = val[i];
    for (int h = 0; h < group; ++h) sum += w[h * (size_t(C) + 1) + i];
    const float x = float(sum);
    val[i] = x;
    if (at <= newest) mine = min(mine, (1ull << 63) | ((unsigned long long)evict_key(x) << 31) | unsigned(i));
  }
  mine = warp_min(mine);
  if (lane == 0) best[threadIdx.x >> 5] = mine;
  __syncthreads();
  mine = warp_min(best[lane & 7]);
  if (mine == ~0ull) {
    if (threadIdx.x == 0) {
      if (err != nullptr) set_error(err, ERRW_BOUNDS);
      admit_slot[r] = -1;
      evicted_pos[r] = -1;
      length[r] = now + 1;
    }
    return;
  }
  const int slot = int(mine & 0x7fffffffull);
  if (threadIdx.x == 0) {
    double sum = 0.;
    for (int h = 0; h < group; ++h) sum += w[h * (size_t(C) + 1) + C];
    admit_slot[r] = slot;
    evicted_pos[r] = mine >> 63 ? pos[slot] : -1;
    pos[slot] = now;
    val[slot] = float(sum);
    length[r] = now + 1;
  }
  if (threadIdx.x < 32) {
    const int j = threadIdx.x % (DH / 8);
    float kx[8], vx[8];
    load8(k_new + size_t(r) * DH + 8 * j, kx);
    load8(v_new + size_t(r) * DH + 8 * j, vx);
    __nv_bfloat162 kpair, vpair;
    const uint32_t kw = q4_encode8(kx, kpair), vw = q4_encode8(vx, vpair);
    if (threadIdx.x < DH / 8) q4_store_piece<DH>(c, size_t(r), P, slot, j, kw, kpair, vw, vpair);
  }
}

}  // namespace adore
