// Launches of the MFMA decode kernel (decode_mfma_kernel.h) on bf16 caches, the kernels in front of it that order the sequences
// and plan their chunks, and what it takes.  The forms for a cache in 4 bits are compiled in decode_mx4.hip: code objects of
// their own keep these as they were without them (in one, with the same instructions in every kernel, the step of one request took
// 29.1 us instead of 28.6, MLRA-2 on 64 of 8K 131.4 instead of 130.3).
#include "decode_mfma_kernel.h"

namespace mlra {
namespace {

// Sequence ids sorted by length, longest first (rank sort; ties keep index order).  Used when a launch has
// more workgroups than the chip runs at once: workgroups are dispatched in id order, so handing out
// the long sequences first is the longest-processing-time rule and keeps the last round short.
// group > 1 (several query tokens per sequence): entries [i group, i group + group) of seq_lens are the
// queries of one sequence, which read the same cache rows.  Whole sequences are ranked (by their longest
// query) and the queries of the sequence of rank r get the dispatch slots (r / 8) 8 group + 8 q + r % 8:
// the decode kernels put slot k on XCD k % 8 and slots of one run of 8 group side by side in time, so the
// queries of a sequence meet in one L2 and its rows come from HBM once.
__global__ __launch_bounds__(256) void seq_order_kernel(const int32_t* __restrict__ seq_lens,
                                                        int32_t* __restrict__ order, int n_seqs, int group) {
  extern __shared__ int32_t lens[];            // every length once, then the comparisons run out of LDS
  for (int j = threadIdx.x; j < n_seqs; j += 256) lens[j] = seq_lens[(size_t)j * group + group - 1];
  __syncthreads();
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i >= n_seqs) return;
  const int n = lens[i];
  int rank = 0;
  for (int j = 0; j < n_seqs; ++j) {
    const int nj = lens[j];
    rank += (nj > n || (nj == n && j < i)) ? 1 : 0;
  }
  const int full = n_seqs & ~7;                // ranks below this fill whole runs of 8 sequences
  for (int q = 0; q < group; ++q) {
    const int slot = rank < full ? (rank >> 3) * 8 * group + 8 * q + (rank & 7) : full * group + (rank - full) * group + q;
    order[slot] = i * group + q;
  }
}

// Chunk lengths that follow the sequence lengths.  With uniform chunks a ragged batch leaves workgroups
// idle (a sequence half as long as the longest uses half of its chunk slots); here sequence i gets
// S_i ~ target * n_i / sum(n) chunks of ceil(n_i / S_i) tokens (rounded up to the tile, at least
// min_chunk), so that about `target` chunks per block are active in total and they are about equally long.
// unit_tab lists the active (sequence, chunk) pairs, packed as sequence * 1024 + chunk, and -1 after
// them: workgroup ids go round-robin over the XCDs, so the active ones must be contiguous to spread
// evenly (scattered, they leave some XCDs with more work than CUs and others idle).  The pairs are listed
// longest chunk first (for batches of up to 512 sequences): when they need more than one round of
// workgroups, that is the longest-processing-time rule.  With single_if_uniform, a batch whose longest
// sequence is within 25 % of the mean keeps one chunk per sequence (cutting it would only add partials).
__global__ __launch_bounds__(256) void plan_chunks_kernel(const int32_t* __restrict__ seq_lens,
                                                          int32_t* __restrict__ chunk_tab,
                                                          int32_t* __restrict__ unit_tab, int batch, int target,
                                                          int max_slots, int min_chunk, int single_if_uniform) {
  __shared__ float part[4];
  __shared__ int part_max[4], part_count[3][4];
  __shared__ int wave_tot[4];
  extern __shared__ int32_t tab[];             // [batch] lengths, [batch] chunk lengths, [batch] dispatch order
  int32_t* lens = tab;
  int32_t* chunks = tab + batch;
  int32_t* order = tab + 2 * batch;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  float sum = 0.f;
  int longest = 0;
  for (int i = threadIdx.x; i < batch; i += 256) {
    lens[i] = seq_lens[i];
    sum += (float)lens[i];
    longest = max(longest, lens[i]);
  }
  // (lengths are integers below 2^31 and their partial sums are added in one fixed order)
  for (int o = 32; o > 0; o >>= 1) {
    sum += __shfl_xor(sum, o);
    longest = max(longest, __shfl_xor(longest, o));
  }
  if (lane == 0) { part[wave] = sum; part_max[wave] = longest; }
  __syncthreads();
  const float total = (part[0] + part[1]) + (part[2] + part[3]);
  longest = max(max(part_max[0], part_max[1]), max(part_max[2], part_max[3]));
  const bool single = single_if_uniform && (float)longest * (float)batch <= 1.25f * total;
  // Rounding may leave more than `target` chunks, whose surplus would run alone at the end (266 of 256 in 128 sequences of
  // 512 to 8192 tokens: GLA-2 162 -> 140 us, MLRA-2 141 -> 117).  Then the shares are made a little smaller, at most three
  // times.  (Counted are the shares, no less than the chunks that come of them.)
  auto share_of = [&](int n, int share) {
    const int s_i = (total > 0.f && !single) ? (int)((float)share * (float)n / total + 0.5f) : 1;
    return min(max(s_i, 1), max_slots);
  };
  int share = target;
  for (int attempt = 0; single_if_uniform && !single && attempt < 3; ++attempt) {   // (targets that are whole rounds)
    int count = 0;
    for (int i = threadIdx.x; i < batch; i += 256) count += lens[i] > 0 ? share_of(lens[i], share) : 0;
    for (int o = 32; o > 0; o >>= 1) count += __shfl_xor(count, o);
    if (lane == 0) part_count[attempt][wave] = count;
    __syncthreads();
    count = part_count[attempt][0] + part_count[attempt][1] + part_count[attempt][2] + part_count[attempt][3];
    if (count <= target) break;
    share = max(1, share - (count - target));
  }
  for (int i = threadIdx.x; i < batch; i += 256) {
    const int n = lens[i], s_i = share_of(n, share);
    int chunk = (n + s_i - 1) / s_i;
    chunk = max(min_chunk, (chunk + kTile - 1) / kTile * kTile);
    chunks[i] = chunk;         // ceil(n / chunk) <= s_i <= max_slots
    chunk_tab[i] = chunk;
  }
  __syncthreads();
  // dispatch order: rank sort by chunk length, longest first (ties keep index order)
  for (int i = threadIdx.x; i < batch; i += 256) {
    int rank = i;
    if (batch <= 512) {
      const int c = chunks[i];
      rank = 0;
      for (int j = 0; j < batch; ++j) {
        const int cj = chunks[j];
        rank += (cj > c || (cj == c && j < i)) ? 1 : 0;
      }
    }
    order[rank] = i;
  }
  __syncthreads();
  // exclusive scan of the active chunk counts in dispatch order: 256 contiguous segments, one per thread
  const int per = (batch + 255) / 256, lo = min(batch, (int)threadIdx.x * per), hi = min(batch, lo + per);
  int mine = 0;
  for (int r = lo; r < hi; ++r) {
    const int i = order[r];
    mine += (lens[i] + chunks[i] - 1) / chunks[i];
  }
  // (scan over the 256 threads: inside a wave with shuffles, across the four waves through LDS)
  int incl = mine;
  for (int o = 1; o < 64; o <<= 1) {
    const int v = __shfl_up(incl, o);
    if (lane >= o) incl += v;
  }
  if (lane == 63) wave_tot[wave] = incl;
  __syncthreads();
  int u = incl - mine;
  for (int w = 0; w < wave; ++w) u += wave_tot[w];
  const int n_active = wave_tot[0] + wave_tot[1] + wave_tot[2] + wave_tot[3];
  for (int r = lo; r < hi; ++r) {
    const int i = order[r];
    const int active = (lens[i] + chunks[i] - 1) / chunks[i];
    for (int k = 0; k < active; ++k) unit_tab[u++] = i * 1024 + k;
  }
  for (int u = n_active + threadIdx.x; u < batch * max_slots; u += 256) unit_tab[u] = -1;
}

}  // namespace

// Fills a.chunk_tab (workspace) with per-sequence chunk lengths, see plan_chunks_kernel.
int launch_plan_chunks(const DecodeArgs& a) {
  if (!a.chunk_tab || !a.unit_tab || a.plan.target_chunks <= 0) return MLRA_ERR_SHAPE;
  if (a.plan.n_splits > 1023 || a.batch > 2048) return MLRA_ERR_SHAPE;
  plan_chunks_kernel<<<1, 256, 3 * a.batch * sizeof(int32_t), a.stream>>>(
      a.seq_lens, a.chunk_tab, a.unit_tab, a.batch, a.plan.target_chunks, a.plan.n_splits, 128,
      a.plan.single_if_uniform ? 1 : 0);
  return check_launch();
}

// Fills a.seq_order (workspace) with the sequence ids in dispatch order (see seq_order_kernel).
// MLRA_ERR_SHAPE (and nothing enqueued) when the batch is outside what the O(batch^2) rank sort is meant for.
int launch_seq_order(const DecodeArgs& a) {
  const int group = a.q_group > 1 ? a.q_group : 1;
  if (!a.seq_order || a.batch <= 1 || a.batch > 8192 || a.batch % group != 0) return MLRA_ERR_SHAPE;
  const int n_seqs = a.batch / group;
  seq_order_kernel<<<(n_seqs + 255) / 256, 256, n_seqs * sizeof(int32_t), a.stream>>>(a.seq_lens, a.seq_order, n_seqs,
                                                                                     group);
  return check_launch();
}

// (several query tokens per sequence: the order is what brings a sequence's queries together, so it is
// wanted even when one round of workgroups covers the launch)
static bool want_seq_order(const DecodeArgs& a, long long n_wg) {
  return !a.balanced && !a.fitted && (n_wg > a.cus || a.q_group > 1);
}

// Pages of 16 or 32 tokens (a wave's 16 rows of a tile never straddle a page), or whole tiles.  (4 bits: any multiple of 16.)
static bool page_size_ok(int page_size) { return page_size == 16 || page_size == 32 || page_size % kTile == 0; }
// (the kernels form page id x bytes-per-page from 32-bit factors)
static bool page_bytes_ok(const DecodeArgs& a) { return (long long)a.n_blocks * a.page_size * a.d_cb * 2 < (1LL << 32); }

bool decode_mfma_supported(const DecodeArgs& a) {
  // (the query rows are addressed with 32-bit byte offsets from q_abs / q_rope)
  return a.dtype == MLRA_BF16 && a.d_cb == kDcb && a.d_r == kDr &&
         (a.scales ? a.page_size % 16 == 0 : page_size_ok(a.page_size)) && page_bytes_ok(a) &&
         a.plan.chunk_tokens % kTile == 0 &&
         (long long)a.batch * a.n_blocks * a.h * (kDcb * 2) < (1LL << 32) &&
         (long long)a.batch * a.h * a.groups * (kDr * 2) < (1LL << 32);
}

// Blocks that serve at most 64 heads in their last 128-head group leave half of the plain form's waves
// idle; with an even number of blocks in a head group the PAIRED form runs two blocks per workgroup instead (its workgroups
// take the RoPE queries of one group).
bool decode_mfma_paired(int h, int n_blocks, int groups) {
  return n_blocks / groups % 2 == 0 && (h - 1) % kHeadsWG < 64;
}

// GLA-2 shape: latent heads of 256 channels (Section 2.3); 64 heads per workgroup.
bool decode_gla_supported(const DecodeArgs& a) {
  return a.dtype == MLRA_BF16 && a.d_cb == 2 * kDcb && a.d_r == kDr && page_size_ok(a.page_size) && page_bytes_ok(a) &&
         a.plan.chunk_tokens % kTile == 0 &&
         (long long)a.batch * a.n_blocks * a.h * (4 * kDcb) < (1LL << 32) &&
         (long long)a.batch * a.h * a.groups * (kDr * 2) < (1LL << 32);
}

int launch_decode_gla(const DecodeArgs& a) {
  static PerDeviceSetup setup;
  int setup_dev = -1;
  constexpr int kStagesGla = 3;
  const int lds = kStagesGla * (2 * kLatBytes + kRopeBytes) + 4 * 8 * 64 * 16;   // stages + score exchange
  if (setup.needed(&setup_dev)) {
    if (hipFuncSetAttribute((const void*)decode_mfma_kernel<kStagesGla, 2, false>,
                            hipFuncAttributeMaxDynamicSharedMemorySize, lds) != hipSuccess)
      return MLRA_ERR_LAUNCH;
    setup.done(setup_dev);
  }
  MfmaParams p;
  p.latent = (const bf16_t*)a.latent;
  p.rope = (const bf16_t*)a.rope;
  p.page_table = a.page_table;
  p.seq_lens = a.seq_lens;
  p.q_abs = (const bf16_t*)a.q_abs;
  p.q_rope = (const bf16_t*)a.q_rope;
  p.part_z = a.part_z;
  p.part_ml = a.part_ml;
  p.page_size = a.page_size;
  p.max_pages = a.max_pages;
  p.n_blocks = a.n_blocks;
  p.h = a.h;
  p.groups = a.groups;
  p.n_splits = a.plan.n_splits;
  p.chunk = a.plan.chunk_tokens;
  p.batch = a.batch;
  p.scale_log2 = softmax_scale_log2(a.softmax_scale);
  p.rows_bf16 = a.rows_bf16 ? 1 : 0;
  p.chunk_tab = a.balanced ? a.chunk_tab : nullptr;
  p.unit_tab = a.balanced ? a.unit_tab : nullptr;
  p.seq_order = nullptr;
  const long long n_wg = (long long)a.plan.n_splits * a.n_blocks * ((a.h + 63) / 64) * a.batch;
  if (n_wg <= 0 || n_wg > 0x7fffffffLL) return MLRA_ERR_SHAPE;
  if (want_seq_order(a, n_wg) && launch_seq_order(a) == MLRA_OK) p.seq_order = a.seq_order;
  MLRA_LAUNCH_TIMED(a.t_main, (decode_mfma_kernel<kStagesGla, 2, false>), dim3((unsigned)n_wg), dim3(256), lds, a.stream, p);
  return check_launch();
}

int launch_decode_mfma(const DecodeArgs& a) {
  const bool paired = decode_mfma_paired(a.h, a.n_blocks, a.groups);
  MfmaParams p;
  p.latent = (const bf16_t*)a.latent;
  p.scales = (const uint8_t*)a.scales;
  p.rope = (const bf16_t*)a.rope;
  p.page_table = a.page_table;
  p.seq_lens = a.seq_lens;
  p.q_abs = (const bf16_t*)a.q_abs;
  p.q_rope = (const bf16_t*)a.q_rope;
  p.part_z = a.part_z;
  p.part_ml = a.part_ml;
  p.page_size = a.page_size;
  p.max_pages = a.max_pages;
  p.n_blocks = a.n_blocks;
  p.h = a.h;
  p.groups = a.groups;
  p.n_splits = a.plan.n_splits;
  p.chunk = a.plan.chunk_tokens;
  p.batch = a.batch;
  p.scale_log2 = softmax_scale_log2(a.softmax_scale);
  p.rows_bf16 = a.rows_bf16 ? 1 : 0;
  const int n_hg = paired ? (a.h + 63) / 64 : (a.h + kHeadsWG - 1) / kHeadsWG;
  const long long slots = (long long)a.plan.n_splits * a.batch, eights = 8 * a.q_group;
  // (a fitted launch hands its chunks out in runs of eight)
  const long long n_wg = (a.fitted ? (slots + eights - 1) / eights * eights : slots) * (paired ? a.n_blocks / 2 : a.n_blocks) * n_hg;
  if (n_wg <= 0 || n_wg > 0x7fffffffLL) return MLRA_ERR_SHAPE;
  // more than one round of workgroups (one per CU at a time): longest sequences first
  p.seq_order = nullptr;
  p.chunk_tab = a.balanced ? a.chunk_tab : nullptr;
  p.unit_tab = a.balanced ? a.unit_tab : nullptr;
  if (a.fitted) {
    p.fit_min = a.fit_tiles;
    p.fit_group = a.q_group;
    p.cus = a.cus;
    p.chunk_out = a.chunk_tab;
  }
  if (want_seq_order(a, n_wg) && launch_seq_order(a) == MLRA_OK) p.seq_order = a.seq_order;
  if (a.scales) return launch_decode_mx4(a, p, paired, (unsigned)n_wg);
  // (the plain form first: kernels lie in the code object in the order of their first use, and behind the paired form this one is
  // 0.4 us slower, 16 sequences of 16K tokens on one block 41.3 against 40.8 us)
  if (!paired) return launch_form<kStages, 0, false>(a, p, (unsigned)n_wg);
  return launch_form<kStagesPaired, 1, false>(a, p, (unsigned)n_wg);
}

}  // namespace mlra
