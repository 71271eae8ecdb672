// sp_attn_cross where a sequence's keys are few enough to stay in LDS (attn_cross.hip says what is computed).
//
// Why.  With few keys the work is the queries' way in and the outputs' way out: 2 * head_dim bytes each per query head against
// 4 * head_dim operations per key.  A workgroup of the prefill kernel does one query tile: its lengths, its page ids, its key tiles and its
// queries are a chain of memory round trips of 9 to 10 us behind which nothing else runs on its CU (two waves per SIMD, all registers).
// Here a workgroup brings the sequence's keys and values of one KV head to LDS once and then goes through many query
// tiles: a wave takes 32 columns at a time by itself, without a barrier, and requests the next 32 queries before it works on these.
// Bound: HBM (queries in, outputs out) up to about 100 keys.  Beyond, neither a pipe nor a memory, but a wave's chain of scores, weights and
// products, which the one other wave on its SIMD covers in part: on 8 x 1749 queries on 229 keys at 16q/2kv (56 us, floor 24) the matrix pipe
// is busy in 41 % of the CU cycles and the LDS in 21, on 12 x 957 on 259 at 32q/8kv (87 us, floor 41) in 35 and 19; rows of up to 256 keys
// multiply their weights as hi + lo, half as many operations again.  Measured (query tiles -> here): 13 x 3331 queries on 18 keys at
// 32q/8kv, head_dim 128, 315 -> 146 us (0.71 GB, 4.9 TB/s); 7 x 1901 on 26 88 -> 40; 1 x 57 on 10 at 8q/1kv 10.9 -> 5.8; 14 x 4489 on 90 at
// 16q/2kv, head_dim 64, 96 -> 64.
#include "decode_block.h"
#include "prefill_tile.h"
#include "cross_plan.h"

namespace sp {

template <int D, int WAVES>
__global__ __launch_bounds__(64 * WAVES, 2) void cross_resident_kernel(CrossArgs a, int rounds, int blocks) {
  using G = TileGeom<D>;
  using Z = SwzTile<D>;
  constexpr int ROWB = D * 2, MBYTES = 32 * ROWB, CPR = D / 8;  // a row; 32 keys of K or of V, 16-byte chunks of a row
  constexpr int THREADS = 64 * WAVES;
  extern __shared__ __align__(16) char smem_raw[];
  lds_char *smem = (lds_char *)smem_raw;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 31, half = lane >> 5;
  const int seq = blockIdx.x / a.n_hgroups, hg = blockIdx.x - seq * a.n_hgroups;
  const int q0 = a.cu_q[seq], ncols = (a.cu_q[seq + 1] - q0) << a.gshift;
  const int first = blockIdx.y * (32 * WAVES * rounds) + 32 * w;  // this wave's first column
  if ((int)blockIdx.y * (32 * WAVES * rounds) >= ncols) return;
  const int kv = min(cross_keys(a, a.ctx_lens[seq]), 32 * blocks), nb = (kv + 31) >> 5;
  const int kvh = (hg << a.gshift) / (a.Hq / a.Hkv), gmask = (1 << a.gshift) - 1;
  // Row of q and out of column C; the columns behind the last take its row, and are not stored.
  auto row_off = [&](int C) __attribute__((always_inline)) {
    C = min(C, ncols - 1);
    return ((long)(q0 + (C >> a.gshift)) * a.Hq + ((hg << a.gshift) | (C & gmask))) * ROWB;
  };
  bf16x8 q[1][G::kDSteps], next[G::kDSteps];
  auto request = [&](int c0) __attribute__((always_inline)) {
    const char *row = a.q + row_off(c0 + col) + 16 * half;
#pragma unroll
    for (int s = 0; s < G::kDSteps; ++s) next[s] = *reinterpret_cast<const bf16x8 *>(row + 32 * s);
  };
  request(first);

  // ---- keys and values, 32 at a time in the swizzled layout of SwzTile; zeros behind the last
  const int32_t *bt_row = a.block_table + (long)seq * a.max_pages;
  const size_t page_bytes = (size_t)a.Hkv * (kPage * ROWB), head = (size_t)kvh * (kPage * ROWB);
  constexpr int U = 4;
  for (int i0 = threadIdx.x; i0 < nb * 32 * CPR; i0 += U * THREADS) {
    u32x4 k[U], v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = i0 + u * THREADS, row = i / CPR;
      const int page = min(max(bt_row[min(row, kv - 1) >> 4], 0), a.num_pages - 1);
      const size_t at = (size_t)page * page_bytes + head + (size_t)(min(row, kv - 1) & 15) * ROWB + (i % CPR) * 16;
      k[u] = *reinterpret_cast<const u32x4 *>(a.k_pages + at);
      v[u] = *reinterpret_cast<const u32x4 *>(a.v_pages + at);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = i0 + u * THREADS, row = i / CPR, c = i % CPR;
      if (row >= nb * 32) continue;
      if (row >= kv) k[u] = v[u] = (u32x4){0, 0, 0, 0};
      lds_char *block = smem + (row >> 5) * (2 * MBYTES);
      *(lds_u32x4 *)(block + Z::template offset<false>(row & 31, c)) = k[u];
      *(lds_u32x4 *)(block + MBYTES + Z::template offset<true>(row & 31, c)) = v[u];
    }
  }
  int kofs[G::kDSteps], vofs[G::kDBlocks];
#pragma unroll
  for (int s = 0; s < G::kDSteps; ++s) kofs[s] = Z::template offset<false>(col, 2 * s + half);
  {
    const int n = lane & 15, dg = (lane >> 4) & 1;
#pragma unroll
    for (int db = 0; db < G::kDBlocks; ++db)
      vofs[db] = Z::template offset<true>(4 * half + (n >> 2), 4 * db + 2 * dg + ((n & 3) >> 1)) + 8 * (n & 1);
  }
  __syncthreads();

  for (int r = 0; r < rounds; ++r) {
    const int c0 = first + r * (32 * WAVES);
    if (c0 >= ncols) return;
#pragma unroll
    for (int s = 0; s < G::kDSteps; ++s) q[0][s] = next[s];
    if (r + 1 < rounds) request(c0 + 32 * WAVES);
    f32x16 o[1][G::kDBlocks];
#pragma unroll
    for (int db = 0; db < G::kDBlocks; ++db)
#pragma unroll
      for (int e = 0; e < 16; ++e) o[0][db][e] = 0.f;
    float m[1] = {-INFINITY}, l[1] = {0.f};
    const int lim[1] = {0};
    for (int b = 0; b < nb; ++b) {
      const lds_char *block = smem + b * (2 * MBYTES);
      attend_block<D, false, 1>(block, block + MBYTES, kofs, vofs, q, o, m, l, 32 * b, kv, 0, lim, half, a.sl2e, a.tau, kv <= 256, [] {});
    }
    const float lt = l[0] + other_half(l[0]), inv = nb > 0 ? 1.0f / lt : 0.f;  // no keys: rows of zeros
    // Of 16 channels a lane holds 0..3 and 8..11 (or 4..7 and 12..15); the halves exchange what makes them 0..7 and 8..15, for
    // stores of 16 bytes.
    char *dst = a.out + row_off(c0 + col);
    const bool valid = c0 + col < ncols;
#pragma unroll
    for (int db = 0; db < G::kDBlocks; ++db)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        uint32_t x[2][2];
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            union {
              bf16x2 p;
              uint32_t u;
            } y;
            y.p = __builtin_convertvector((f32x2){o[0][db][8 * h + 4 * t + 2 * e] * inv, o[0][db][8 * h + 4 * t + 2 * e + 1] * inv}, bf16x2);
            x[t][e] = y.u;
          }
        const auto s0 = __builtin_amdgcn_permlane32_swap(x[0][0], x[1][0], false, false);
        const auto s1 = __builtin_amdgcn_permlane32_swap(x[0][1], x[1][1], false, false);
        if (valid) *reinterpret_cast<u32x4 *>(dst + (32 * db + 16 * h + 8 * half) * 2) = (u32x4){s0[0], s1[0], s0[1], s1[1]};
      }
  }
}

template <int D, int WAVES>
static int launch_resident(const CrossArgs &a, const CrossResident &plan, int batch, int max_q_len, hipStream_t stream) {
  static bool done = false;
  const long cols = (long)max_q_len << a.gshift, per = 32L * WAVES * plan.rounds;
  const int smem = plan.blocks * 2 * 32 * D * 2;
  if (int rc = grant_smem((const void *)cross_resident_kernel<D, WAVES>, &done, kResidentLds)) return rc;
  hipLaunchKernelGGL((cross_resident_kernel<D, WAVES>), dim3((unsigned)(batch * a.n_hgroups), (unsigned)((cols + per - 1) / per)), dim3(64 * WAVES),
                     smem, stream, a, plan.rounds, plan.blocks);
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? SP_OK : fail(SP_ERR_HIP, "sp_attn_cross launch: %s", hipGetErrorString(e));
}

int launch_cross_resident(const CrossArgs &a, const CrossResident &plan, int head_dim, int batch, int max_q_len, hipStream_t stream) {
  if (head_dim == 128) return plan.waves == 4 ? launch_resident<128, 4>(a, plan, batch, max_q_len, stream) : launch_resident<128, 8>(a, plan, batch, max_q_len, stream);
  return plan.waves == 4 ? launch_resident<64, 4>(a, plan, batch, max_q_len, stream) : launch_resident<64, 8>(a, plan, batch, max_q_len, stream);
}

}  // namespace sp
