// Causal attention of packed bfloat16 prompts on the 5th-generation tensor cores (tcgen05 + TMEM).
//
//   S = Q K^T,  P = exp(scale (S - m)),  O = P V / rowsum P,  lse = scale m + log rowsum P
//
// One CTA owns 256 consecutive query rows of one head as two tiles of 128 and walks over the blocks of 128 keys up to the
// diagonal; both tiles use a block while it is in shared memory. Roles (12 warps, two of them idle, one CTA per SM):
//   warp 8     producer: Q tiles once, then K and V blocks by TMA (128-byte swizzle) through a ring of shared-memory stages
//   warp 9     one thread issues the MMAs: S_t = Q_t K^T (both operands in shared memory), O_t += P_t V (P_t in TMEM, V as
//              an N-major operand, so that no transposed copy is needed)
//   warps 0-3  softmax of tile 0, warps 4-7 of tile 1: one row per thread, the whole row of 128 logits in registers
// While one tile's softmax runs, the tensor core works on the other tile: the issue order per block is P V of tile 0, next S
// of tile 0, P V of tile 1, next S of tile 1. P is written over S as bfloat16; the MMAs execute in order, so the next S cannot
// overtake the P V that reads it. TMEM: 2 x 128 columns of S / P and 2 x dh of O.
//
// The row maximum that the weights refer to is raised only when a row's maximum has grown by more than 2^8 (weights of up to 256
// lose nothing in float32 sums and bfloat16 operands); O then has to be rescaled in TMEM, which is rare after the first
// blocks. A weight is rounded to bfloat16 for the product with V (half a step, 2^-8 of its value), the sum takes it unrounded.
//
// Only the last block of a tile (the diagonal) needs a mask: tiles and blocks are aligned alike. Rows behind the end of the
// sequence belong to other sequences or to nobody: their logits are masked there, and their V rows are zeroed in shared memory,
// because 0 times an infinity or NaN would not be 0.
#pragma once

#include "packed.cuh"
#include "tcgen05.cuh"

namespace adore {

constexpr int kPtTile = 128;
constexpr int kPtThreads = 384;           // two softmax warpgroups, one with the producer and the issuer
// 384 threads x 168 registers at launch = 64512; 256 x 208 + 128 x 80 = 63488
constexpr int kPtRegsSoftmax = 208, kPtRegsOther = 80;

template <int DH>
struct PtSmem {
  static constexpr int kStages = DH == 128 ? 5 : 8;
  static constexpr int kTileBytes = kPtTile * DH * 2;
  static constexpr size_t kTotal = size_t(2 + kStages) * kTileBytes + 256 + 1024;    // + barriers + alignment slack
};

__device__ __forceinline__ float pt_exp2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ unsigned long long pt_pack(float a, float b) {
  unsigned long long r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ void pt_unpack(unsigned long long r, float& a, float& b) {
  asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(r));
}
__device__ __forceinline__ unsigned long long pt_fma2(unsigned long long a, unsigned long long b, unsigned long long c) {
  unsigned long long d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
  return d;
}
__device__ __forceinline__ unsigned long long pt_add2(unsigned long long a, unsigned long long b) {
  unsigned long long d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
__device__ __forceinline__ uint32_t pt_bf16x2(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

// One tile of 128 rows x DH elements as DH/64 boxes of 64 elements.
template <int DH>
__device__ __forceinline__ void pt_load_tile(void* dst, const CUtensorMap* map, int head, int row, uint64_t* bar) {
  tc_mbar_expect_tx(bar, uint32_t(PtSmem<DH>::kTileBytes));
#pragma unroll
  for (int i = 0; i < DH / 64; ++i) tc_tma_load_3d(static_cast<unsigned char*>(dst) + i * (kPtTile * 128), map, 64 * i, head, row, bar);
}

// D = A B^T for two K-major tiles of 128 rows x DH.
template <int DH>
__device__ __forceinline__ void pt_mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc) {
#pragma unroll
  for (int k = 0; k < DH / 16; ++k) {
    const uint64_t at = uint64_t((k / 4) * (kPtTile * 128 / 16) + (k % 4) * 2);
    tc_mma_bf16(d, a + at, b + at, idesc, k != 0 ? 1u : 0u);
  }
}

struct PtMaps { CUtensorMap q, k, v; };

template <int DH>
__global__ void __launch_bounds__(kPtThreads, 1)
prompt_attention_tc_kernel(const __grid_constant__ PtMaps maps, const PackedParams p, __nv_bfloat16* out, float* lse) {
  using S = PtSmem<DH>;
  constexpr int kStages = S::kStages;
  extern __shared__ __align__(1024) unsigned char pt_smem_raw[];
  unsigned char* base = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(pt_smem_raw) + 1023) & ~uintptr_t(1023));
  unsigned char* q_tiles = base;
  unsigned char* ring = base + 2 * S::kTileBytes;
  uint64_t* bars = reinterpret_cast<uint64_t*>(ring + size_t(kStages) * S::kTileBytes);
  uint64_t* kv_full = bars;
  uint64_t* kv_empty = kv_full + kStages;
  uint64_t* q_full = kv_empty + kStages;      // per tile
  uint64_t* s_full = q_full + 2;              // logits ready (and every earlier MMA done)
  uint64_t* p_full = s_full + 2;              // weights stored, O rescaled if needed
  uint64_t* o_full = p_full + 2;              // last product done
  uint64_t* drain = o_full + 2;               // after a wait that ran out: every issued MMA done
  __shared__ PackedTile tile;
  __shared__ int found, s_abort;
  __shared__ uint32_t tmem_slot;
  volatile int* abort_flag = &s_abort;

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int h = blockIdx.x % p.H, g = h / p.group;
  if (threadIdx.x == 0) {
    for (int i = 0; i < kStages; ++i) { tc_mbar_init(&kv_full[i], 1u); tc_mbar_init(&kv_empty[i], 1u); }
    for (int t = 0; t < 2; ++t) {
      tc_mbar_init(&q_full[t], 1u);
      tc_mbar_init(&s_full[t], 1u);
      tc_mbar_init(&p_full[t], 4u);
      tc_mbar_init(&o_full[t], 1u);
    }
    tc_mbar_init(drain, 1u);
    s_abort = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 8) {
    PackedTile t{};
    const bool ok = find_packed_tile<2 * kPtTile>(p.seq_start, p.S, p.total, blockIdx.x / p.H, p.err, t);
    if (lane == 0) { tile = t; found = ok; }
  }
  __syncthreads();
  if (!found) return;
  if (warp == 9) { __syncwarp(); tc_alloc(&tmem_slot, 512); }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_slot;
  const uint32_t o_cols = 256;                // S of tile t at column 128 t, O of tile t at 256 + DH t
  const int len = tile.len, q0 = tile.index * 2 * kPtTile;
  const bool two = len > q0 + kPtTile;
  const int n0 = 2 * tile.index + 1, n1 = two ? n0 + 1 : 0, blocks = two ? n1 : n0;

  int issued = 0;                             // producer: ring loads issued

  if (warp >= 8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kPtRegsOther));
    if (warp == 8) {
      // ---------------- producer ----------------
      if (lane == 0) {
        bool ok = true;
        pt_load_tile<DH>(q_tiles, &maps.q, h, tile.start + q0, &q_full[0]);
        // K0 V0 K1 V1 ..
        for (int i = 0; i < 2 * blocks; ++i) {
          const int stage = i % kStages;
          if (i >= kStages && !tc_mbar_wait(&kv_empty[stage], uint32_t(i / kStages - 1) & 1u, abort_flag)) { ok = false; break; }
          pt_load_tile<DH>(ring + size_t(stage) * S::kTileBytes, (i & 1) ? &maps.v : &maps.k, g, tile.start + (i >> 1) * kPtTile, &kv_full[stage]);
          issued = i + 1;
          if (i == 0 && two) pt_load_tile<DH>(q_tiles + S::kTileBytes, &maps.q, h, tile.start + q0 + kPtTile, &q_full[1]);
        }
        if (!ok && !*abort_flag) { if (p.err != nullptr) set_error(p.err, ERRW_TIMEOUT); *abort_flag = 1; }
      }
    } else if (warp == 9) {
      // ---------------- MMA issuer ----------------
      const uint32_t idesc_s = tc_idesc(kPtTile, kPtTile) | (p.scale < 0.f ? kTcIdescNegA : 0u);     // the softmax then takes |scale|
      constexpr uint32_t idesc_o = tc_idesc(kPtTile, DH) | kTcIdescBN;
      bool ok = true;
      const int tail = (len - 1) / kPtTile, tail_rows = len - tail * kPtTile;      // last block of the sequence and its rows
      for (int t = 0; t < (two ? 2 : 1) && ok; ++t) {
        ok = tc_mbar_wait_warp(&q_full[t], 0u, abort_flag) && (t == 1 || tc_mbar_wait_warp(&kv_full[0], 0u, abort_flag));
        if (!ok) break;
        tc_fence_after();
        if (lane == 0) {
          pt_mma_ss<DH>(tmem + 128 * t, tc_smem_desc(q_tiles + t * S::kTileBytes), tc_smem_desc(ring), idesc_s);
          tc_commit(&s_full[t]);
        }
        __syncwarp();
      }
      if (ok && lane == 0) tc_commit(&kv_empty[0]);
      for (int j = 0; j < blocks && ok; ++j) {
        const int vi = 2 * j + 1, vs = vi % kStages, ki = vi + 1, ks = ki % kStages;
        unsigned char* v_tile = ring + size_t(vs) * S::kTileBytes;
        if (!tc_mbar_wait_warp(&kv_full[vs], uint32_t(vi / kStages) & 1u, abort_flag)) { ok = false; break; }
        if (j == tail && tail_rows < kPtTile) {
          constexpr int kPieces = 8 * (DH / 64);                 // 16-byte pieces of a row, in boxes of 8
          for (int i = lane; i < (kPtTile - tail_rows) * kPieces; i += 32) {
            const int r = tail_rows + i / kPieces, c = i % kPieces;
            *reinterpret_cast<uint4*>(v_tile + (c / 8) * (kPtTile * 128) + r * 128 + (c % 8) * 16) = make_uint4(0u, 0u, 0u, 0u);
          }
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          __syncwarp();
        }
        for (int t = 0; t < 2; ++t) {
          const int n = t == 0 ? n0 : n1;
          if (j >= n) continue;
          if (!tc_mbar_wait_warp(&p_full[t], uint32_t(j) & 1u, abort_flag)) { ok = false; break; }
          if (j + 1 < n && !tc_mbar_wait_warp(&kv_full[ks], uint32_t(ki / kStages) & 1u, abort_flag)) { ok = false; break; }
          tc_fence_after();
          if (lane == 0) {
            const uint64_t vd = tc_smem_desc_n(v_tile, kPtTile * 128);
  #pragma unroll
            for (int k = 0; k < kPtTile / 16; ++k)               // 16 keys: 8 columns of P, two groups of 8 rows of V
              tc_mma_bf16_ts(tmem + o_cols + DH * t, tmem + 128 * t + 8 * k, vd + uint64_t(128 * k), idesc_o, (j | k) != 0 ? 1u : 0u);
            if (j + 1 < n) {
              pt_mma_ss<DH>(tmem + 128 * t, tc_smem_desc(q_tiles + t * S::kTileBytes), tc_smem_desc(ring + size_t(ks) * S::kTileBytes), idesc_s);
              tc_commit(&s_full[t]);
            } else {
              tc_commit(&o_full[t]);
            }
          }
          __syncwarp();
        }
        if (ok && lane == 0) {
          tc_commit(&kv_empty[vs]);
          if (j + 1 < blocks) tc_commit(&kv_empty[ks]);
        }
      }
      if (!ok) {
        if (lane == 0) {
          if (!*abort_flag) { if (p.err != nullptr) set_error(p.err, ERRW_TIMEOUT); *abort_flag = 1; }
          tc_commit(drain);
        }
        int never = 0;
        tc_mbar_wait_warp(drain, 0u, &never);
      }
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kPtRegsSoftmax));
    // ---------------- softmax of tile `t`, one row per thread ----------------
    const int t = warp >> 2, quarter = warp & 3;
    const int n = t == 0 ? n0 : n1;
    const int r = quarter * 32 + lane, row = q0 + t * kPtTile + r;
    const uint32_t lanes = uint32_t(quarter * 32) << 16;
    const uint32_t s_at = tmem + lanes + 128 * t, o_at = tmem + lanes + o_cols + DH * t;
    const float c = fabsf(p.scale) * 1.4426950408889634f;      // logits in units of log 2
    float m = -INFINITY, l = 0.f;
    bool ok = true;
    for (int j = 0; j < n; ++j) {
      if (!tc_mbar_wait_warp(&s_full[t], uint32_t(j) & 1u, abort_flag)) { ok = false; break; }
      tc_fence_after();
      uint32_t s[4][32];
      __syncwarp();
#pragma unroll
      for (int i = 0; i < 4; ++i) tc_ld_32x32_start(s_at + 32 * i, s[i]);
#pragma unroll
      for (int i = 0; i < 4; ++i) tc_ld_wait(s[i]);
      if (j == n - 1) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int e = 0; e < 32; ++e)
            if (32 * i + e > r) s[i][e] = 0xff800000u;
      }
      float tops[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        tops[i] = __uint_as_float(s[i][0]);
#pragma unroll
        for (int e = 1; e < 32; ++e) tops[i] = fmaxf(tops[i], __uint_as_float(s[i][e]));
      }
      const float top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
      const bool raise = (top - m) * c > 8.f;                  // also the first block: m = -inf
      if (__any_sync(0xffffffffu, raise)) {
        const float f = raise ? pt_exp2((m - top) * c) : 1.f;
        if (raise) m = top;
        l *= f;
        if (j > 0) {
#pragma unroll 1
          for (int i = 0; i < DH / 32; ++i) {
            uint32_t o[32];
            tc_ld_32x32_start(o_at + 32 * i, o);
            tc_ld_wait(o);
#pragma unroll
            for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
            tc_st_32x32(o_at + 32 * i, o);
          }
        }
      }
      const unsigned long long c2 = pt_pack(c, c), mc2 = pt_pack(-m * c, -m * c);
      unsigned long long sum[2] = {0ull, 0ull};
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        uint32_t w[32];
#pragma unroll
        for (int e = 0; e < 32; ++e) {
          const uint32_t* x = &s[2 * i + e / 16][2 * (e % 16)];
          const unsigned long long y = pt_fma2(pt_pack(__uint_as_float(x[0]), __uint_as_float(x[1])), c2, mc2);
          float a, b;
          pt_unpack(y, a, b);
          a = pt_exp2(a);
          b = pt_exp2(b);
          sum[e & 1] = pt_add2(sum[e & 1], pt_pack(a, b));
          w[e] = pt_bf16x2(a, b);
        }
        tc_st_32x32(s_at + 32 * i, w);
      }
      float a, b;
      pt_unpack(pt_add2(sum[0], sum[1]), a, b);
      l += a + b;
      tc_st_wait();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) tc_mbar_arrive(&p_full[t]);
    }
    if (n > 0 && ok) ok = tc_mbar_wait_warp(&o_full[t], 0u, abort_flag);
    if (n > 0 && ok) {
      tc_fence_after();
      const float inv = 1.f / l;
      const bool mine = row < len;
      __nv_bfloat16* dst = out + (tile.start + row) * p.out_row + h * p.out_head;
#pragma unroll 1
      for (int i = 0; i < DH / 32; ++i) {
        uint32_t o[32];
        __syncwarp();
        tc_ld_32x32_start(o_at + 32 * i, o);
        tc_ld_wait(o);
        if (mine) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            uint32_t w[4];
#pragma unroll
            for (int x = 0; x < 4; ++x)
              w[x] = pt_bf16x2(__uint_as_float(o[8 * e + 2 * x]) * inv, __uint_as_float(o[8 * e + 2 * x + 1]) * inv);
            reinterpret_cast<uint4*>(dst + 32 * i)[e] = make_uint4(w[0], w[1], w[2], w[3]);
          }
        }
      }
      if (mine && lse != nullptr) lse[size_t(h) * p.total + tile.start + row] = (m * c + log2f(l)) * 0.6931471805599453f;
    }
    if (!ok && lane == 0 && !*abort_flag) { if (p.err != nullptr) set_error(p.err, ERRW_TIMEOUT); *abort_flag = 1; }
  }

  tc_fence_before();
  __syncthreads();
  if (*abort_flag) {                          // copies in flight have to land before the CTA ends
    if (warp == 8 && lane == 0) {
      int never = 0;
      for (int i = max(0, issued - kStages); i < issued; ++i) tc_mbar_wait(&kv_full[i % kStages], uint32_t(i / kStages) & 1u, &never);
      tc_mbar_wait(&q_full[0], 0u, &never);
      if (two && issued > 0) tc_mbar_wait(&q_full[1], 0u, &never);
    }
    __syncthreads();
  }
  tc_fence_after();
  if (warp == 9) { __syncwarp(); tc_dealloc(tmem, 512); }
}

}  // namespace adore
