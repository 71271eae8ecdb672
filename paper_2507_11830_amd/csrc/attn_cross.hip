// Attention without a mask over the paged cache (sp_attn_cross): every query token of a sequence sees all of its states, those of an
// encoder of another length.
//
//   out[t] = sum_j p_tj v_j,  p_t = softmax_j(scale q_t . k_j),  j = 0 .. kv_lens[s] - 1; zeros where there are none
//
// Weights go to the second product in bf16, as in the causal calls, where a row has more than 256 keys: each is off by at most 2^-8 of
// itself, and 257 and more of them average that out (error against 64 bits, of unit normal inputs: 0.0019 to 0.0023 of the output's norm, where
// the output's own rounding is 0.0017).  Shorter rows take them as hi + lo, off by 2^-16.  Scores, maxima and sums are fp32.
//
// The kernels are those of the causal calls with another limit on a column's keys (CrossArgs in prefill_tile.h, CROSS in
// decode_stream.h): no tile is masked but a sequence's last, all query tiles of a sequence are equally long, and rows without
// keys are written as zeros.  Bound: bf16 MFMA, 4 * head_dim operations per (query, key) pair and head, for long chunks; HBM, the
// states once for all query heads and tokens, for chunks of a few tokens.
//
// What is chosen from the hints (cross_plan.h says when, and what it measured):
//   - chunks of a few tokens, one column tile of a wave: the decode kernel with equal shares or fixed splits (75 batches of
//     1 to 200 such chunks on 20 to 8000 keys: 22 % faster than query tiles in the mean).  With two column tiles, as in the causal calls,
//     it took 13 % longer than query tiles in pieces (75 batches), but with a workgroup for every column tile it is the faster one
//     up to about a round of workgroups;
//   - few keys, up to 256 or 320: they stay in LDS while a workgroup goes through many queries (attn_cross_resident.hip);
//   - otherwise query tiles of 128 columns in several workgroups a CU, or of 256 (head_dim 128, long key ranges), or of 128 columns
//     whose two wave groups take alternate key tiles, and where even these leave most CUs idle, in pieces of the key range.
#include "decode_stream.h"
#include "prefill_solo.h"
#include "cross_plan.h"

namespace sp {

// ---- chunks of a few tokens, or column tiles of them.  TILES: the tiles of a chunk in neighbouring workgroups.
template <int D, bool TILES>
__global__ __launch_bounds__(64 * kWaves, 2) void cross_stream_kernel(DecodeArgs a) {
  extern __shared__ __align__(16) char smem_raw[];
  lds_char *smem = (lds_char *)smem_raw;
  const int lane = threadIdx.x & 63;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (a.row_splits) {  // fixed splits of a.chunk keys
    const int tiles = TILES ? (int)gridDim.x / a.n_hgroups : 1, seq = blockIdx.y, split = blockIdx.z;
    const int hg = TILES ? (int)blockIdx.x / tiles : (int)blockIdx.x, ct = TILES ? (int)blockIdx.x - hg * tiles : 0;
    const int p0 = split * (a.chunk >> 5);
    const int pages = load_pages(a, seq, p0, 0, w, lane);  // in the same round trip as the lengths
    const int tok = a.cu_q[seq], qn = a.cu_q[seq + 1] - tok, L = cross_keys(a, a.ctx_lens[seq]);
    if (qn <= ct * a.q_cap) return;
    const int p1 = min((L + 31) >> 5, p0 + (a.chunk >> 5)), slot = (seq * a.n_hgroups + hg) * a.row_splits + split;
    if (p1 <= p0) {  // no keys: rows of zeros if there is no other split, else an empty partial
      const int c = ct * a.q_cap * a.geff + threadIdx.x;
      if (a.row_splits > 1) {
        if ((int)threadIdx.x < a.q_cap * a.geff && c < a.cols) *reinterpret_cast<f32x2 *>(a.part_ml + 2 * ((long)slot * a.cols + c)) = (f32x2){-INFINITY, 0.f};
      } else if (ct == 0) {
        zero_chunk<D>(a, tok, qn, hg);
      }
      return;
    }
    row_segment<D, false, true, 1, true>(a, smem, lane, w, seq, hg, L, L - qn, tok, p0, p1, pages, a.row_splits == 1, slot, ct);
    return;
  }
  if constexpr (!TILES) decode_share<D, false, true, 1, true>(a, smem, lane, w, blockIdx.x);
}

template <int D, bool TILES>
static int launch_cross_stream(const DecodeArgs &a, dim3 wgs, int max_pieces, hipStream_t stream) {
  static bool done = false;
  constexpr int smem = kDecodeShareSmem<D, true>;
  if (int rc = grant_smem((const void *)cross_stream_kernel<D, TILES>, &done, smem)) return rc;
  hipLaunchKernelGGL((cross_stream_kernel<D, TILES>), wgs, dim3(64 * kWaves), smem, stream, a);
  if (a.row_splits != 1) launch_decode_combine(a, max_pieces, D, stream);
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? SP_OK : fail(SP_ERR_HIP, "sp_attn_cross launch: %s", hipGetErrorString(e));
}

// ---- longer chunks
template <int D>
static int launch_cross_d(const CrossArgs &a, const CrossShape &shape, int batch, int max_q_len, hipStream_t stream) {
  constexpr size_t smem = kPrefillSmem<D>;
  static bool set[4] = {false, false, false, false};
  if (a.kv_splits > 1) return launch_cfg(prefill_kernel<D, KVT, PFD, true, true, 0, CrossArgs>, &set[0], 2 * smem, 128, a, batch, max_q_len, stream);
  if (shape.halves) return launch_cfg(prefill_kernel<D, KVT, PFD, true, false, 0, CrossArgs>, &set[1], 2 * smem, 128, a, batch, max_q_len, stream);
  if (D == 64 || shape.solo) return launch_cfg(solo_prefill_kernel<CrossArgs, D>, &set[2], kSoloSmemOf<D>, kSoloCols, a, batch, max_q_len, stream, kSoloThreads, kSoloLayers);
  if constexpr (D == 128) return launch_cfg(prefill_kernel<D, KVT, PFD, false, false, 0, CrossArgs>, &set[3], smem, 256, a, batch, max_q_len, stream);
  return SP_OK;
}

static int column_shift(int group) {  // log2 of the heads that share the column dimension
  int gshift = 0;
  if ((group & (group - 1)) == 0)
    while ((1 << gshift) < group && gshift < 5) ++gshift;
  return gshift;
}

// The calling thread's launch overrides (sp_debug_set_tuning) in the place of what cross_shape chooses.
static CrossShape shape_of(int batch, int total_q, int max_q_len, int max_kv_len, int num_q_heads, int num_kv_heads, int head_dim, bool can_cut) {
  const PrefillTuning tune = prefill_tuning();
  const long rows = (long)total_q * num_q_heads;
  const int gshift = column_shift(num_q_heads / num_kv_heads);
  CrossShape s = cross_shape(rows, batch, (long)batch * (num_q_heads >> gshift), 1 << gshift, total_q, max_q_len, max_kv_len, head_dim,
                             can_cut && tune.split == 0);
  if (tune.kv_splits > 0 && can_cut) s.pieces = tune.kv_splits < kv_split_cap(rows) ? tune.kv_splits : kv_split_cap(rows);
  if (tune.split > 0) {
    s.halves = tune.split == 2;
    s.solo = false;
  }
  if (tune.order > 0) s.ranked = tune.order == 2;
  s.ranked = s.ranked && batch <= 64 * kRankSlots;
  return s;
}

static CrossResident resident_of(int batch, int total_q, int max_q_len, int max_kv_len, int num_q_heads, int num_kv_heads, int head_dim) {
  const PrefillTuning tune = prefill_tuning();
  if (tune.split != 0 || tune.kv_splits != 0 || tune.order != 0) return {0, 0, 0};  // the caller asks for query tiles
  const int gshift = column_shift(num_q_heads / num_kv_heads);
  return cross_resident((long)total_q * num_q_heads, (long)batch * (num_q_heads >> gshift), 1 << gshift, max_q_len, max_kv_len, head_dim);
}

static CrossTiles tiles_of(int batch, int max_q_len, int max_kv_len, int num_q_heads, int num_kv_heads, int head_dim, bool can_split) {
  const int cap = decode_route_cap(num_q_heads, num_kv_heads), group = num_q_heads / num_kv_heads;
  const int geff = group < 32 ? group : group % 32 == 0 ? 32 : 1;  // heads of a column tile (set_head_groups)
  return cross_tiles(batch, num_q_heads / geff, cap, max_q_len, max_kv_len, head_dim, can_split);
}

size_t cross_workspace_bytes(int batch, int total_q, int max_q_len, int max_kv_len, int num_q_heads, int num_kv_heads, int head_dim) {
  const long rows = (long)total_q * num_q_heads;
  const bool resident = resident_of(batch, total_q, max_q_len, max_kv_len, num_q_heads, num_kv_heads, head_dim).blocks > 0;
  const int kvs = resident ? 1 : shape_of(batch, total_q, max_q_len, max_kv_len, num_q_heads, num_kv_heads, head_dim, true).pieces;
  const size_t pieces = kvs > 1 ? (size_t)rows * kvs * (head_dim + 2) * sizeof(float) : 0;
  const long streams = (long)batch * (num_q_heads >> column_shift(num_q_heads / num_kv_heads));
  if (resident && cross_resident_for_few(streams, max_kv_len, head_dim)) return 0;
  const size_t few = prefill_tuning().short_chunk == 1 || max_q_len > decode_route_cap(num_q_heads, num_kv_heads) ? 0 : decode_multi_workspace_bytes(batch, total_q, max_q_len, max_kv_len, num_q_heads, num_kv_heads, head_dim);
  const CrossTiles t = tiles_of(batch, max_q_len, max_kv_len, num_q_heads, num_kv_heads, head_dim, true);
  const size_t tiles = resident || prefill_tuning().short_chunk == 1 ? 0 : cross_tiles_bytes(t, batch, num_q_heads, max_q_len, head_dim);
  const size_t more = pieces > few ? pieces : few;
  return more > tiles ? more : tiles;
}

int launch_cross(const sp_cache_desc &c, const void *q, void *out, const int32_t *cu_q, const int32_t *kv_lens, const int32_t *block_table,
                 int batch, int max_pages, int total_q, int max_q_len, int max_kv_len, int num_q_heads, float scale, void *workspace,
                 size_t workspace_bytes, hipStream_t stream) {
  const PrefillTuning tune = prefill_tuning();
  const int gshift = column_shift(num_q_heads / c.num_kv_heads);
  const CrossResident resident = resident_of(batch, total_q, max_q_len, max_kv_len, num_q_heads, c.num_kv_heads, c.head_dim);
  if (tune.short_chunk != 1 && !(resident.blocks > 0 && cross_resident_for_few((long)batch * (num_q_heads >> gshift), max_kv_len, c.head_dim))) {
    DecodeArgs d;
    dim3 wgs;
    int pieces = 0;
    if (plan_decode_cross(d, c, q, out, cu_q, kv_lens, block_table, batch, max_pages, max_q_len, max_kv_len, num_q_heads, scale, workspace, workspace_bytes,
                          &wgs, &pieces))
      return c.head_dim == 128 ? launch_cross_stream<128, false>(d, wgs, pieces, stream) : launch_cross_stream<64, false>(d, wgs, pieces, stream);
  }
  if (tune.short_chunk != 1 && max_pages > 0 && resident.blocks == 0) {
    const CrossTiles t = tiles_of(batch, max_q_len, max_kv_len, num_q_heads, c.num_kv_heads, c.head_dim, workspace != nullptr);
    if (t.tiles > 0 && workspace_bytes >= cross_tiles_bytes(t, batch, num_q_heads, max_q_len, c.head_dim)) {
      DecodeArgs d;
      plan_cross_tiles(d, c, q, out, cu_q, kv_lens, block_table, batch, max_pages, max_q_len, num_q_heads, scale, workspace, t.chunk, t.splits);
      const dim3 wgs((unsigned)(d.n_hgroups * t.tiles), (unsigned)batch, (unsigned)t.splits);
      return c.head_dim == 128 ? launch_cross_stream<128, true>(d, wgs, t.splits, stream) : launch_cross_stream<64, true>(d, wgs, t.splits, stream);
    }
  }
  CrossArgs a = {};
  a.k_pages = (const char *)c.k_pages;
  a.v_pages = (const char *)c.v_pages;
  a.q = (const char *)q;
  a.out = (char *)out;
  a.cu_q = cu_q;
  a.ctx_lens = kv_lens;
  a.block_table = block_table;
  a.max_pages = max_pages;
  a.num_pages = c.num_pages;
  a.Hq = num_q_heads;
  a.Hkv = c.num_kv_heads;
  a.gshift = gshift;
  a.n_hgroups = num_q_heads >> a.gshift;
  a.sl2e = scale * 1.44269504088896340736f;
  a.tau = 8.0f / a.sl2e;
  a.batch = batch;
  a.total_q = total_q;
  const long rows = (long)total_q * num_q_heads;
  if (resident.blocks > 0) return launch_cross_resident(a, resident, c.head_dim, batch, max_q_len, stream);
  CrossShape shape = shape_of(batch, total_q, max_q_len, max_kv_len, num_q_heads, c.num_kv_heads, c.head_dim, workspace != nullptr);
  int kvs = shape.pieces;
  const size_t fit = workspace_bytes / ((size_t)rows * (c.head_dim + 2) * sizeof(float));
  if ((size_t)kvs > fit) {  // fewer pieces, or the shape without any
    kvs = fit > 1 ? (int)fit : 1;
    if (kvs == 1) shape = shape_of(batch, total_q, max_q_len, max_kv_len, num_q_heads, c.num_kv_heads, c.head_dim, false);
  }
  a.kv_splits = kvs;
  a.part_o = (float *)workspace;
  a.part_ml = a.part_o + (size_t)rows * kvs * c.head_dim;
  a.ranked = shape.ranked;
  a.rank_shift = 6;
  while (a.rank_shift < 24 && (((long)max_kv_len + max_q_len) >> a.rank_shift) > 63) ++a.rank_shift;
  const int rc = c.head_dim == 128 ? launch_cross_d<128>(a, shape, batch, max_q_len, stream) : launch_cross_d<64>(a, shape, batch, max_q_len, stream);
  if (rc != SP_OK || kvs == 1) return rc;
  return launch_combine(a.part_o, a.part_ml, out, rows, kvs, c.head_dim, stream, cu_q, batch, num_q_heads);
}

}  // namespace sp
