// Queries and keys of the step's new tokens normalised per head and rotated by their positions' angles, the keys and the values
// scattered into their pages (sp_norm_rope_append): everything between the projections and the attention in one pass.
//
//   y = x * rsqrt(mean(x^2) + eps) * weight          per (token, head), fp32
//   (a, b) -> (a cos - b sin, b cos + a sin)         per pair of rotated channels, fp32; then one rounding to bf16
//
// Work decomposition.  A row (one head of one token) belongs to D / 16 lanes, each with two 16-byte chunks of 8 channels.  Where the
// pairs are (i, i + rotary_dim / 2) a lane owns chunk j of either half, so a pair never leaves its lane; the sum of squares is three DPP
// steps (two at head_dim 64).  The angles belong to the token, the weights to the channel: both stay in registers while a
// lane group goes through its rows of the token.
//
// Bound: HBM, 4 * head_dim bytes per (token, head) in and out; small calls by their chain of memory round trips (prefix sums, then
// page id and angles, then the store; rows and weights are requested first).
// Measured (kernel alone): 48703 tokens at 32q/8kv, head_dim 128 (1.2 GB) 206 us, 5.9 TB/s (a plain copy of 2 GiB: 4.9); 4096 at 8q/1kv 5.7;
// 64 at 8q/1kv 3.05; 1 token 2.6 (an empty kernel: 2.2).  Stores that leave no line behind in L2: 218 -> 207 us and 6.7 -> 5.7, and the
// attention behind it takes as long as before.  Rows per lane group: 4 (8: 226 us, 2: 261).
#include "sp_common.h"

namespace sp {

struct NormRopeArgs {
  const char *q, *k, *v;
  char *q_out, *k_pages, *v_pages;
  long q_stride, k_stride, v_stride;  // bytes between tokens
  const char *q_weight, *k_weight;
  const float *cos_sin;
  const int32_t *positions, *cu_new, *ctx_lens, *block_table;
  float eps;
  int num_positions, rotary, batch, max_pages, num_pages, Hq, Hkv, rows, total, gshift;
};

constexpr int kNormThreads = 256;
constexpr int kLensInLds = 1024;  // prefix sums and cached lengths staged in LDS; longer batches search global memory
constexpr int kLensInWave = 4;    // per lane, where a wave keeps those of the batch to itself

// Rows may begin at any element.
typedef u32x4 __attribute__((aligned(2))) row_chunk;
typedef f32x4 __attribute__((aligned(4))) angle_chunk;

__device__ __forceinline__ void widen(u32x4 x, float (&y)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    y[2 * i] = __uint_as_float(x[i] << 16);
    y[2 * i + 1] = __uint_as_float(x[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ u32x4 narrow(const float (&y)[8]) {
  union {
    bf16x2 h[4];
    u32x4 v;
  } u;
#pragma unroll
  for (int i = 0; i < 4; ++i) u.h[i] = __builtin_convertvector((f32x2){y[2 * i], y[2 * i + 1]}, bf16x2);
  return u.v;
}
template <int CTRL>
__device__ __forceinline__ float dpp(float x) {
  return __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), CTRL, 0xF, 0xF, true));
}
// Sum over the 4 or 8 lanes of a row, in all of them: exchange inside pairs, between pairs, between the mirrored quads.
template <int LANES>
__device__ __forceinline__ float row_sum(float x) {
  x += dpp<0xB1>(x);  // quad_perm [1, 0, 3, 2]
  x += dpp<0x4E>(x);  // quad_perm [2, 3, 0, 1]
  if (LANES == 8) x += dpp<0x141>(x);  // row_half_mirror
  return x;
}

enum { kNoRotation, kHalves, kInterleaved };

// U: rows that a lane group has in flight.
template <int D, int ROT, int U>
__global__ __launch_bounds__(kNormThreads) void norm_rope_append_kernel(NormRopeArgs a) {
  constexpr int LANES = D / 16, ROWB = 2 * D;
  constexpr int GROUPS = kNormThreads / LANES;  // lane groups of the workgroup
  __shared__ int32_t s_cu[kLensInLds], s_ctx[kLensInLds];
  const int j = threadIdx.x % LANES, grp = threadIdx.x / LANES;
  const int g = grp & ((1 << a.gshift) - 1);  // which of the token's lane groups this is
  const long tok = (long)blockIdx.x * (GROUPS >> a.gshift) + (grp >> a.gshift);
  const bool live = tok < a.total;
  const int half = a.rotary / 16;  // chunks of half of the rotated channels
  const int c0 = ROT == kHalves && j >= half ? 2 * j : j;
  const int c1 = ROT == kHalves ? (j >= half ? 2 * j + 1 : j + half) : j + LANES;
  const int step = 1 << a.gshift;
  auto row_at = [&](int r) __attribute__((always_inline)) {
    return r < a.Hq ? a.q + tok * a.q_stride + r * ROWB
           : r < a.Hq + a.Hkv ? a.k + tok * a.k_stride + (r - a.Hq) * ROWB : a.v + tok * a.v_stride + (r - a.Hq - a.Hkv) * ROWB;
  };
  u32x4 x[U][2];
  auto load_rows = [&](int r0) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int r = r0 + u * step;
      if (r < a.rows) {
        const char *p = row_at(r);
        x[u][0] = *(const row_chunk *)(p + 16 * c0);
        x[u][1] = *(const row_chunk *)(p + 16 * c1);
      }
    }
  };
  if (live) load_rows(g);
  u32x4 qw[2] = {}, kw[2] = {};
  if (a.q_weight) {
    qw[0] = *(const row_chunk *)(a.q_weight + 16 * c0);
    qw[1] = *(const row_chunk *)(a.q_weight + 16 * c1);
  }
  if (a.k_weight) {
    kw[0] = *(const row_chunk *)(a.k_weight + 16 * c0);
    kw[1] = *(const row_chunk *)(a.k_weight + 16 * c1);
  }
  // The token's sequence s, the largest with cu_new[s] <= tok; tokens outside [cu_new[0], cu_new[batch]) belong to other calls.
  int s, first, end, ctx;
  if (LANES << a.gshift >= 64 && a.batch <= 64 * kLensInWave) {
    // all lanes of a wave have the same token: every wave looks at all prefix sums at once, a few per lane (64 tokens: 3.05 us,
    // with the search below 3.5)
    if (!live) return;
    const int lane = threadIdx.x & 63, u_tok = __builtin_amdgcn_readfirstlane((int)tok);
    int cu[kLensInWave], cx[kLensInWave];
    const int cu0 = a.cu_new[0];
#pragma unroll
    for (int u = 0; u < kLensInWave; ++u) {
      cu[u] = a.cu_new[min(64 * u + lane + 1, a.batch)];
      cx[u] = a.ctx_lens[min(64 * u + lane, a.batch - 1)];
    }
    s = 0;
#pragma unroll
    for (int u = 0; u < kLensInWave; ++u) s += __builtin_popcountll(__builtin_amdgcn_ballot_w64(64 * u + lane < a.batch - 1 && cu[u] <= u_tok));
    first = cu0;
    ctx = end = 0;
#pragma unroll
    for (int u = 0; u < kLensInWave; ++u) {
      if (s - 1 >= 64 * u) first = __builtin_amdgcn_readlane(cu[u], (s - 1) & 63);
      if (s >= 64 * u) ctx = __builtin_amdgcn_readlane(cx[u], s & 63);
      if (a.batch - 1 >= 64 * u) end = __builtin_amdgcn_readlane(cu[u], (a.batch - 1) & 63);
    }
  } else {
    const bool staged = a.batch < kLensInLds;
    if (staged) {
      for (int i = threadIdx.x; i <= a.batch; i += kNormThreads) {
        s_cu[i] = a.cu_new[i];
        if (i < a.batch) s_ctx[i] = a.ctx_lens[i];
      }
      __syncthreads();
    }
    if (!live) return;
    s = 0;
    int hi = a.batch;
    while (hi - s > 1) {
      const int mid = (s + hi) >> 1;
      if ((staged ? s_cu[mid] : a.cu_new[mid]) <= tok) s = mid;
      else hi = mid;
    }
    first = staged ? s_cu[s] : a.cu_new[s];
    end = staged ? s_cu[a.batch] : a.cu_new[a.batch];
    ctx = staged ? s_ctx[s] : a.ctx_lens[s];
  }
  if (tok < first || tok >= end) return;
  const int pos = ctx + (int)(tok - first);
  int page = -1;
  if (a.k && pos >= 0 && (pos >> 4) < a.max_pages) page = a.block_table[(long)s * a.max_pages + (pos >> 4)];
  // this lane's angles: of its pairs in the two halves, or of the four pairs of either chunk
  float cs[8], sn[8];
  bool turn0 = false, turn1 = false;
  if (ROT != kNoRotation) {
    const int at = min(max(a.positions ? a.positions[tok] : pos, 0), a.num_positions - 1);
    const float *cos = a.cos_sin + (long)at * a.rotary, *sin = cos + a.rotary / 2;
    turn0 = ROT == kHalves ? j < half : c0 < 2 * half;
    turn1 = ROT == kHalves ? turn0 : c1 < 2 * half;
    const int from0 = ROT == kHalves ? 8 * j : 4 * c0, from1 = ROT == kHalves ? 8 * j + 4 : 4 * c1;
    if (turn0) {
      *(f32x4 *)cs = *(const angle_chunk *)(cos + from0);
      *(f32x4 *)sn = *(const angle_chunk *)(sin + from0);
    }
    if (turn1) {
      *(f32x4 *)(cs + 4) = *(const angle_chunk *)(cos + from1);
      *(f32x4 *)(sn + 4) = *(const angle_chunk *)(sin + from1);
    }
  }
  const bool stored = page >= 0 && page < a.num_pages;  // bad metadata must not turn into a wild store
  for (int r0 = g;;) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int r = r0 + u * step;
      if (r >= a.rows) break;
      const bool is_q = r < a.Hq, is_v = r >= a.Hq + a.Hkv;
      const bool norm = !is_v && (is_q ? a.q_weight : a.k_weight) != nullptr;
      u32x4 y0 = x[u][0], y1 = x[u][1];
      if (!is_v && (norm || ROT != kNoRotation)) {
        float f0[8], f1[8];
        widen(y0, f0);
        widen(y1, f1);
        if (norm) {
          float sum0 = 0.f, sum1 = 0.f;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            sum0 = __builtin_fmaf(f0[e], f0[e], sum0);
            sum1 = __builtin_fmaf(f1[e], f1[e], sum1);
          }
          const float inv = rsqrtf(row_sum<LANES>(sum0 + sum1) * (1.0f / D) + a.eps);
          float w0[8], w1[8];
          widen(is_q ? qw[0] : kw[0], w0);
          widen(is_q ? qw[1] : kw[1], w1);
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            f0[e] *= inv * w0[e];
            f1[e] *= inv * w1[e];
          }
        }
        if (ROT == kHalves && turn0) {
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float p = f0[e], q = f1[e];
            f0[e] = p * cs[e] - q * sn[e];
            f1[e] = q * cs[e] + p * sn[e];
          }
        }
        if (ROT == kInterleaved) {
          auto turn = [&](float (&f)[8], int k) __attribute__((always_inline)) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float p = f[2 * e], q = f[2 * e + 1];
              f[2 * e] = p * cs[k + e] - q * sn[k + e];
              f[2 * e + 1] = q * cs[k + e] + p * sn[k + e];
            }
          };
          if (turn0) turn(f0, 0);
          if (turn1) turn(f1, 4);
        }
        y0 = narrow(f0);
        y1 = narrow(f1);
      }
      char *to;
      if (is_q) {
        to = a.q_out + (tok * a.Hq + r) * ROWB;
      } else {
        if (!stored) continue;
        const int h = is_v ? r - a.Hq - a.Hkv : r - a.Hq;
        to = (is_v ? a.v_pages : a.k_pages) + (((long)page * a.Hkv + h) * kPage + (pos & 15)) * ROWB;
      }
      __builtin_nontemporal_store((row_chunk)y0, (row_chunk *)(to + 16 * c0));
      __builtin_nontemporal_store((row_chunk)y1, (row_chunk *)(to + 16 * c1));
    }
    r0 += U * step;
    if (r0 >= a.rows) break;
    load_rows(r0);
  }
}

template <int D>
static void launch_norm_rope_d(const NormRopeArgs &a, int rot, dim3 grid, hipStream_t stream) {
  if (rot == kNoRotation) hipLaunchKernelGGL((norm_rope_append_kernel<D, kNoRotation, 4>), grid, dim3(kNormThreads), 0, stream, a);
  else if (rot == kHalves) hipLaunchKernelGGL((norm_rope_append_kernel<D, kHalves, 4>), grid, dim3(kNormThreads), 0, stream, a);
  else hipLaunchKernelGGL((norm_rope_append_kernel<D, kInterleaved, 4>), grid, dim3(kNormThreads), 0, stream, a);
}

int launch_norm_rope_append(const sp_cache_desc &c, const void *q, const void *k, const void *v, long q_stride, long k_stride,
                            long v_stride, void *q_out, const void *q_weight, const void *k_weight, float eps, const sp_rope_desc *rope,
                            const int32_t *positions, const int32_t *cu_new, const int32_t *ctx_lens, const int32_t *block_table,
                            int batch, int max_pages, int total_new, int num_q_heads, hipStream_t stream) {
  NormRopeArgs a;
  a.q = (const char *)q;
  a.k = (const char *)k;
  a.v = (const char *)v;
  a.q_out = (char *)q_out;
  a.k_pages = (char *)c.k_pages;
  a.v_pages = (char *)c.v_pages;
  a.q_stride = 2 * q_stride;
  a.k_stride = 2 * k_stride;
  a.v_stride = 2 * v_stride;
  a.q_weight = (const char *)q_weight;
  a.k_weight = (const char *)k_weight;
  a.eps = eps;
  const int rot = !rope || rope->rotary_dim == 0 ? kNoRotation : rope->interleaved ? kInterleaved : kHalves;
  a.cos_sin = rot == kNoRotation ? nullptr : rope->cos_sin;
  a.num_positions = rot == kNoRotation ? 0 : rope->num_positions;
  a.rotary = rot == kNoRotation ? 0 : rope->rotary_dim;
  a.positions = positions;
  a.cu_new = cu_new;
  a.ctx_lens = ctx_lens;
  a.block_table = block_table;
  a.batch = batch;
  a.max_pages = max_pages;
  a.num_pages = c.num_pages;
  a.Hq = num_q_heads;
  a.Hkv = k ? c.num_kv_heads : 0;
  a.rows = a.Hq + 2 * a.Hkv;
  a.total = total_new;
  const int groups = kNormThreads / (c.head_dim / 16);
  a.gshift = 0;
  while ((1 << a.gshift) < groups && (a.rows + (1 << a.gshift) - 1) >> a.gshift > 4) ++a.gshift;
  while ((1 << a.gshift) < groups && (1 << a.gshift) < a.rows && (long)total_new << a.gshift < 256L * groups) ++a.gshift;
  const long blocks = ((long)total_new + (groups >> a.gshift) - 1) / (groups >> a.gshift);
  if (c.head_dim == 128) launch_norm_rope_d<128>(a, rot, dim3((unsigned)blocks), stream);
  else launch_norm_rope_d<64>(a, rot, dim3((unsigned)blocks), stream);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return fail(SP_ERR_HIP, "norm_rope_append launch: %s", hipGetErrorString(e));
  return SP_OK;
}

}  // namespace sp
