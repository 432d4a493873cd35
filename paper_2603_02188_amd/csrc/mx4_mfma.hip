// Decode attention on the latent cache in 4 bits, for every shape: latent blocks of up to 512 channels (multiples of 32), up
// to 128 RoPE channels, any page size, heads and lengths, bf16 and fp32.
//
// One workgroup (4 wavefronts) owns one (context chunk, block, 32 NH heads) and walks the chunk in tiles of 64 tokens.  The
// codes are widened to bf16 on their way into LDS, which is exact, and the tile is key and value at once, as in the kernels
// for the wider caches.  Wave (hw, tw) scores 16 NH heads against 32 of the tile's tokens on v_mfma_f32_16x16x32_bf16:
//   * S^T = K Q^T (16 tokens x 16 heads): lane l holds head l % 16 and tokens 4 (l / 16) + i.  Two such tiles are the B
//     operand of Z^T += V^T P^T if k index 8 q + e means token 4 q + e of the first tile for e < 4 and 4 q + e - 4 of the
//     second one; V^T comes out of the row-major tile through two transpose reads that take the tokens in that order.
//   * fp32: the cached latents are exact in bf16 as they are, so only the other operand needs more than 8 bits.  A query and a
//     probability is the sum of three bf16 numbers (24 bits), a product with the latents three matrix instructions; the RoPE
//     part, fp32 on both sides, takes the six products of terms down to 2^-24.  (The fp32 matrix instructions have a
//     sixteenth of the rate.)
//   * fp32 outputs of a bf16 call (the output itself, or the log-sum-exp) are exact to fp32: cache, queries and weights are exact
//     in bf16 as they come, so that only the probabilities, as three bf16 numbers (two, 2^-17, if the log-sum-exp alone is fp32),
//     and the merge, on the fp32 matrix instructions, differ from a bf16 output's.
//   * the running maximum moves only when a tile outgrows it by more than 2^8; (m, l, Z) is consistent for any reference.
//   * rows are 16 bytes longer than their channels, so that sixteen rows start in sixteen different bank groups.
//   * forms: block width and RoPE width as the tile is padded to (64 to 512, 64 and 128), 32 or 64 heads (mx4_heads_per_wg), terms of a
//     probability, and VEC = false for RoPE widths that are no multiple of four and for tensors that start in between.
//     Registers are spilled in fp32 with 512 and 128 channels only: four in front of the loop, others on the way that computes
//     scores again.
// Bound by the vector instructions of a tile (widening, splitting, softmax: 600 to 700 a wave) and their latency.  fp32, 8
// sequences of 300 to 2048 tokens, 128 heads, four blocks: 32 us, and 17 for the merge; bf16 with an fp32 output, 16 sequences of
// 1000 to 4093, four query tokens: 155 us, and 51 for the merge.
#include "f32_tile.h"
#include "mx4_tile.h"

namespace mlra {
namespace {

using namespace f32_tile;
using mx4_tile::decode8;
using mx4_tile::kGroup;
using mx4_tile::scale_of;
using mx4_tile::u32x4;

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4;
typedef __attribute__((ext_vector_type(4))) short short4v;
typedef __attribute__((ext_vector_type(8))) short short8v;

constexpr int kTile = 64;
constexpr float kNone = -3.0e38f;      // "no token seen yet"
constexpr float kLazy = 8.0f;          // log2 headroom before the reference maximum is moved

struct Mx4Params {
  const uint8_t* latent;
  const uint8_t* scales;
  const void* rope;
  const int32_t* page_table;
  const int32_t* seq_lens;
  const void* q_abs;
  const void* q_rope;
  float* part_z;
  float* part_ml;
  int page_size, max_pages, n_blocks, groups, d_cb, d_r, h, n_splits, chunk, n_hg, batch;
  float scale_log2;
};

template <typename T> struct Terms { static constexpr int n = 3; };      // bf16 terms of a number of type T
template <> struct Terms<bf16_t> { static constexpr int n = 1; };

template <typename T, int DP, int RP>
constexpr int tile_bytes() { return kTile * (DP + 8) * 2 + Terms<T>::n * kTile * (RP + 8) * 2; }
template <typename T, int DP, int RP, int NH>
constexpr size_t lds_bytes() {
  const size_t tile = tile_bytes<T, DP, RP>(), merge = (size_t)4 * NH * (DP / 32) * 64 * 16;
  return (tile > merge ? tile : merge) + 4 * kTile * sizeof(long long) + 2 * 4 * 16 * NH * sizeof(float);
}

// x = t[0] + t[1] + t[2], each a bf16 number (down to 2^-24 |x|; one term: x rounded to bf16)
template <int N>
__device__ __forceinline__ void split(float x, __bf16 (&t)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) {
    t[i] = (__bf16)x;
    x -= (float)t[i];
  }
}

__device__ __forceinline__ short4v read_tr16(const __bf16* p) {
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16(
      (short4v __attribute__((address_space(3)))*)(__attribute__((address_space(3))) const __bf16*)p);
}

// Waves on a SIMD that the registers of the fp32 shapes leave room for, but for the seldom taken ways (0: as it comes)
template <typename T, int DP, int RP, int NH>
constexpr int min_waves() {
  return Terms<T>::n == 1 || DP * NH > 128 || NH * RP > 128 ? 0 : DP == 64 && RP == 64 && NH == 1 ? 3 : 2;
}

// DP, RP: latent and RoPE channels of the tile, at least d_cb and d_r; VEC: RoPE rows and queries in pieces of four elements
// PT: bf16 terms of a probability
template <typename T, int DP, int RP, int NH, bool VEC, int PT>
__global__ __launch_bounds__(256, (min_waves<T, DP, RP, NH>())) void mx4_decode_kernel(Mx4Params p) {
  typedef typename RawOf<T>::type Raw;
  constexpr int N = Terms<T>::n;
  constexpr int LP = DP + 8, PP = RP + 8;                    // elements per row of the latent / RoPE tile
  constexpr int KL = DP / 32, KR = RP / 32, CT = DP / 16;    // k steps over latent and RoPE channels; channel tiles
  constexpr int NG = DP / kGroup, NC = (kTile * NG + 255) / 256, NR = kTile * RP / 4 / 256;
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  __bf16* const lat = (__bf16*)smem;                         // [kTile][LP]
  __bf16* const rop = lat + kTile * LP;                      // [N][kTile][PP]
  constexpr size_t kMain = lds_bytes<T, DP, RP, NH>() - 4 * kTile * sizeof(long long) - 2 * 4 * 16 * NH * sizeof(float);
  long long* const row_at = (long long*)(smem + kMain);      // [2 tiles][latent, rope][kTile] rows in the pools
  float* const mbuf = (float*)(row_at + 4 * kTile);          // [4 waves][16 NH heads]
  float* const lbuf = mbuf + 4 * 16 * NH;

  // workgroup -> (chunk, sequence, block, head group): the head groups of one (chunk, sequence, block) read the same rows
  // and get ids 8 apart, which puts them on one XCD; the chunk is the slowest index.
  int wg = blockIdx.y * gridDim.x + blockIdx.x;
  const int units = p.n_splits * p.batch * p.n_blocks;
  if (wg >= units * p.n_hg) return;
  const int full = units & ~7;
  int u, hg;
  if (wg < full * p.n_hg) {
    const int r = wg >> 3;
    hg = r % p.n_hg;
    u = (r / p.n_hg) * 8 + (wg & 7);
  } else {
    wg -= full * p.n_hg;
    u = full + wg / p.n_hg;
    hg = wg % p.n_hg;
  }
  const int b = u % p.n_blocks, s = u / p.n_blocks % p.batch, split_id = u / p.n_blocks / p.batch;
  const int n = p.seq_lens[s], t0 = split_id * p.chunk;
  if (n <= 0 || (unsigned)t0 >= (unsigned)n) return;         // (slots beyond the capacity)
  const int t1 = t0 + min(n - t0, p.chunk), ntiles = (t1 - t0 + kTile - 1) / kTile;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int q = lane >> 4, r16 = lane & 15, hw = wave & 1, tw = wave >> 1;
  const int d_cb = p.d_cb, d_r = p.d_r;

  // Where the rows of a tile lie: thread i < kTile looks token i's page up one tile before it writes the rows to LDS.  Slots
  // past the chunk repeat its last row: finite wherever the chunk is, and their weight is 0.
  auto page_of = [&](int j) {
    const int tok = t0 + min(j * kTile + tid % kTile, t1 - t0 - 1);
    return p.page_table[(size_t)s * p.max_pages + tok / p.page_size];
  };
  auto row_table = [&](int j, int page_id) {
    if (tid < kTile) {
      const long long page = page_id;
      const int slot = (t0 + min(j * kTile + tid, t1 - t0 - 1)) % p.page_size;
      row_at[(j & 1) * 2 * kTile + tid] = (page * p.n_blocks + b) * p.page_size + slot;
      row_at[(j & 1) * 2 * kTile + kTile + tid] = page * p.page_size + slot;
    }
  };
  // A tile in flight: pieces of a group of 32 channels, and of four RoPE channels.
  u32x4 codes[NC];
  unsigned scale[NC];
  Raw rope[NR];
  auto fetch = [&](int j) {
    const long long* const rows = row_at + (j & 1) * 2 * kTile;
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      const int id = tid + 256 * i, tok = id / NG, g = id % NG;
      const long long row = rows[tok % kTile];
      const int gg = g * kGroup < d_cb ? g : 0;
      codes[i] = *(const u32x4*)(p.latent + row * (d_cb / 2) + gg * (kGroup / 2));
      scale[i] = p.scales[row * (d_cb / kGroup) + gg];
    }
#pragma unroll
    for (int i = 0; i < NR; ++i) {
      const int id = tid + 256 * i, tok = id / (RP / 4), k = id % (RP / 4) * 4;
      const T* const src = (const T*)p.rope + rows[kTile + tok] * d_r;
      if constexpr (VEC) {
        rope[i].load(src + (k < d_r ? k : 0));
      } else {
        rope[i].zero();
#pragma unroll
        for (int e = 0; e < 4; ++e) rope[i].set(e, src[k + e < d_r ? k + e : 0]);
      }
    }
  };
  auto put = [&]() {
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      const int id = tid + 256 * i, tok = id / NG, g = id % NG;
      if (tok < kTile && g * kGroup < d_cb) {
        const float sc = scale_of(scale[i]);
#pragma unroll
        for (int e = 0; e < 4; ++e) *(u32x4*)(lat + tok * LP + g * kGroup + 8 * e) = decode8(codes[i][e], sc);
      }
    }
#pragma unroll
    for (int i = 0; i < NR; ++i) {
      const int id = tid + 256 * i, tok = id / (RP / 4), k = id % (RP / 4) * 4;
      const f32x4 v = rope[i].get();
      bf16x4 t[N];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        __bf16 x[N];
        split(k + e < d_r ? v[e] : 0.f, x);
#pragma unroll
        for (int m = 0; m < N; ++m) t[m][e] = x[m];
      }
#pragma unroll
      for (int m = 0; m < N; ++m) *(bf16x4*)(rop + (m * kTile + tok) * PP + k) = t[m];
    }
  };

  row_table(0, page_of(0));
  row_table(1, page_of(1));
  int page_next = page_of(2);
  // channels past the block's: zero, once
  for (int i = tid; i < kTile * (DP / 8); i += 256)
    if (i % (DP / 8) * 8 >= d_cb) *(u32x4*)(lat + i / (DP / 8) * LP + i % (DP / 8) * 8) = u32x4{0u, 0u, 0u, 0u};
  // queries (a head past the last repeats it and is not stored): k step ks of lane q has channels 32 ks + 8 q .. + 7
  const int head0 = (hg * 2 + hw) * 16 * NH;
  bf16x8 qf[NH][KL + KR][N];
#pragma unroll
  for (int m = 0; m < NH; ++m) {
    const int head = min(head0 + 16 * m + r16, p.h - 1);
    const T* const qa = (const T*)p.q_abs + (((size_t)s * p.n_blocks + b) * p.h + head) * d_cb;
    const T* const qr = (const T*)p.q_rope + ((size_t)s * p.h * p.groups + (b / (p.n_blocks / p.groups)) * p.h + head) * d_r;
#pragma unroll
    for (int ks = 0; ks < KL + KR; ++ks) {
      const T* const src = ks < KL ? qa : qr;
      const int k0 = ks < KL ? 32 * ks + 8 * q : 32 * (ks - KL) + 8 * q, lim = ks < KL ? d_cb : d_r;
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const int k = k0 + 4 * half;
        Raw x;
        if constexpr (VEC) {
          x.load(src + (k < lim ? k : 0));
        } else {
          x.zero();
#pragma unroll
          for (int e = 0; e < 4; ++e) x.set(e, src[k + e < lim ? k + e : 0]);
        }
        const f32x4 v = x.get();
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          __bf16 t[N];
          split(k + e < lim ? v[e] : 0.f, t);
#pragma unroll
          for (int i = 0; i < N; ++i) qf[m][ks][i][4 * half + e] = t[i];
        }
      }
    }
  }
  __syncthreads();
  fetch(0);

  float m_run[NH], l_run[NH];
  f32x4 z[CT][NH];
#pragma unroll
  for (int m = 0; m < NH; ++m) {
    m_run[m] = kNone;
    l_run[m] = 0.f;
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) z[ct][m] = opaque_zero4();
  }
  const int tok0 = 32 * tw;

  for (int j = 0; j < ntiles; ++j) {
    __syncthreads();                    // the tile's readers are done; row tables are visible
    put();
    __syncthreads();
    if (j + 1 < ntiles) {
      row_table(j + 2, page_next);      // into the half that fetch(j) read, two barriers ago
      page_next = page_of(j + 3);
      fetch(j + 1);
    }
    f32x4 sc[NH][2];
#pragma unroll
    for (int m = 0; m < NH; ++m) sc[m][0] = sc[m][1] = opaque_zero4();
#pragma unroll
    for (int ks = 0; ks < KL; ++ks) {
      bf16x8 k[2];
#pragma unroll
      for (int tt = 0; tt < 2; ++tt) k[tt] = *(const bf16x8*)(lat + (tok0 + 16 * tt + r16) * LP + 32 * ks + 8 * q);
#pragma unroll
      for (int i = 0; i < N; ++i)
#pragma unroll
        for (int m = 0; m < NH; ++m)
#pragma unroll
          for (int tt = 0; tt < 2; ++tt)
            sc[m][tt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[tt], qf[m][ks][i], sc[m][tt], 0, 0, 0);
    }
#pragma unroll
    for (int ks = 0; ks < KR; ++ks) {
      bf16x8 k[N][2];
#pragma unroll
      for (int c = 0; c < N; ++c)
#pragma unroll
        for (int tt = 0; tt < 2; ++tt)
          k[c][tt] = *(const bf16x8*)(rop + (c * kTile + tok0 + 16 * tt + r16) * PP + 32 * ks + 8 * q);
#pragma unroll
      for (int c = 0; c < N; ++c)
#pragma unroll
        for (int i = 0; i + c < N; ++i)
#pragma unroll
          for (int m = 0; m < NH; ++m)
#pragma unroll
            for (int tt = 0; tt < 2; ++tt)
              sc[m][tt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[c][tt], qf[m][KL + ks][i], sc[m][tt], 0, 0, 0);
    }
    if constexpr (N > 1) {
      // The lower terms of an infinity, and of a finite number that rounds to one in bf16, are NaN, and so is a score that they
      // are in: it is computed again from the numbers themselves.
      float nan = 0.f;
#pragma unroll
      for (int m = 0; m < NH; ++m)
#pragma unroll
        for (int tt = 0; tt < 2; ++tt) nan += (sc[m][tt][0] + sc[m][tt][1]) + (sc[m][tt][2] + sc[m][tt][3]);
      if (__builtin_expect(__any(nan != nan), 0)) {
#pragma unroll
        for (int m = 0; m < NH; ++m) {
          const int head = min(head0 + 16 * m + r16, p.h - 1);
          const T* const qa = (const T*)p.q_abs + (((size_t)s * p.n_blocks + b) * p.h + head) * d_cb;
          const T* const qr = (const T*)p.q_rope + ((size_t)s * p.h * p.groups + (b / (p.n_blocks / p.groups)) * p.h + head) * d_r;
#pragma unroll
          for (int tt = 0; tt < 2; ++tt)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              if (sc[m][tt][i] == sc[m][tt][i]) continue;
              const int in = tok0 + 16 * tt + 4 * q + i, tok = t0 + min(j * kTile + in, t1 - t0 - 1);
              const long long page = p.page_table[(size_t)s * p.max_pages + tok / p.page_size];
              const T* const kr = (const T*)p.rope + (page * p.page_size + tok % p.page_size) * d_r;
              float sum = 0.f;
#pragma unroll 1
              for (int k = 0; k < d_cb; ++k) sum = fmaf(load_f32(qa, k), (float)lat[in * LP + k], sum);
#pragma unroll 1
              for (int k = 0; k < d_r; ++k) sum = fmaf(load_f32(qr, k), load_f32(kr, k), sum);
              sc[m][tt][i] = sum;
            }
        }
      }
    }
    const int valid = t1 - t0 - j * kTile - tok0;       // tokens of this wave's share that exist
    float mx[NH], lowest = INFINITY;
    bool grown = false;
    if (valid < 32) {                   // (uniform: the chunk's last tile)
#pragma unroll
      for (int m = 0; m < NH; ++m)
#pragma unroll
        for (int tt = 0; tt < 2; ++tt)
#pragma unroll
          for (int i = 0; i < 4; ++i) sc[m][tt][i] = 16 * tt + 4 * q + i < valid ? sc[m][tt][i] : -INFINITY;
    }
#pragma unroll
    for (int m = 0; m < NH; ++m) {
      mx[m] = -INFINITY;
#pragma unroll
      for (int tt = 0; tt < 2; ++tt)
#pragma unroll
        for (int i = 0; i < 4; ++i) mx[m] = fmaxf(mx[m], sc[m][tt][i]);
      mx[m] *= p.scale_log2;
      mx[m] = fmaxf(mx[m], __shfl_xor(mx[m], 16));
      mx[m] = fmaxf(mx[m], __shfl_xor(mx[m], 32));
      grown |= mx[m] > m_run[m] + kLazy;
    }
    if (__any(grown)) {
#pragma unroll
      for (int m = 0; m < NH; ++m) {
        const float m_new = fmaxf(m_run[m], mx[m]), alpha = exp2f(m_run[m] - m_new);
        m_run[m] = m_new;
        l_run[m] *= alpha;
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) z[ct][m] *= alpha;
      }
    }
    bf16x8 pb[NH][PT];
#pragma unroll
    for (int m = 0; m < NH; ++m) {
#pragma unroll
      for (int tt = 0; tt < 2; ++tt)
#pragma unroll
        for (int i = 0; i < 4; ++i) sc[m][tt][i] = __builtin_fmaf(sc[m][tt][i], p.scale_log2, -m_run[m]);
      if constexpr (N > 1) {
        // (the exponential instruction returns zero below 2^-126, exp2f spends a few more on a denormal result: only where
        // there is one, the other bits are the same)
#pragma unroll
        for (int tt = 0; tt < 2; ++tt)
#pragma unroll
          for (int i = 0; i < 4; ++i) lowest = fminf(lowest, sc[m][tt][i]);      // (-inf, no token, among them)
        if (__any(lowest < -126.f)) {
#pragma unroll
          for (int tt = 0; tt < 2; ++tt)
#pragma unroll
            for (int i = 0; i < 4; ++i) sc[m][tt][i] = exp2f(sc[m][tt][i]);
        } else {
#pragma unroll
          for (int tt = 0; tt < 2; ++tt)
#pragma unroll
            for (int i = 0; i < 4; ++i) sc[m][tt][i] = __builtin_amdgcn_exp2f(sc[m][tt][i]);
        }
      } else {
#pragma unroll
        for (int tt = 0; tt < 2; ++tt)
#pragma unroll
          for (int i = 0; i < 4; ++i) sc[m][tt][i] = __builtin_amdgcn_exp2f(sc[m][tt][i]);
      }
#pragma unroll
      for (int tt = 0; tt < 2; ++tt)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          __bf16 t[PT];
          split(sc[m][tt][i], t);
#pragma unroll
          for (int c = 0; c < PT; ++c) pb[m][c][4 * tt + i] = t[c];
          l_run[m] += PT > 1 ? sc[m][tt][i] : (float)t[0];    // (one term: over the weights that the values get)
        }
    }
    const __bf16* const v0 = lat + (tok0 + 4 * q + (r16 >> 2)) * LP + 4 * (r16 & 3);
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
      const short4v lo = read_tr16(v0 + 16 * ct), hi = read_tr16(v0 + 16 * LP + 16 * ct);
      const bf16x8 vt = __builtin_bit_cast(bf16x8, (short8v)__builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
      for (int c = 0; c < PT; ++c)
#pragma unroll
        for (int m = 0; m < NH; ++m) z[ct][m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vt, pb[m][c], z[ct][m], 0, 0, 0);
    }
  }

  // ---- merge the two token halves: wave tw finishes the channel tiles of parity tw and hands the others over.  The partial
  // leaves not normalised, maximum and sum in the log2 domain.
#pragma unroll
  for (int m = 0; m < NH; ++m) {
    l_run[m] += __shfl_xor(l_run[m], 16);
    l_run[m] += __shfl_xor(l_run[m], 32);
  }
  __syncthreads();
  f32x4* const zbuf = (f32x4*)smem;     // [4 waves][NH][CT / 2][64 lanes]
  if (q == 0) {
#pragma unroll
    for (int m = 0; m < NH; ++m) {
      mbuf[(wave * NH + m) * 16 + r16] = m_run[m];
      lbuf[(wave * NH + m) * 16 + r16] = l_run[m];
    }
  }
#pragma unroll
  for (int m = 0; m < NH; ++m)
#pragma unroll
    for (int c2 = 0; c2 < CT / 2; ++c2)
      zbuf[((wave * NH + m) * (CT / 2) + c2) * 64 + lane] = tw == 0 ? z[2 * c2 + 1][m] : z[2 * c2][m];
  __syncthreads();
  const size_t unit = ((size_t)s * p.n_blocks + b) * p.n_splits + split_id;
#pragma unroll
  for (int m = 0; m < NH; ++m) {
    const int at = ((wave ^ 2) * NH + m) * 16 + r16, head = head0 + 16 * m + r16;
    const float mp = mbuf[at], ms = fmaxf(m_run[m], mp), w_own = exp2f(m_run[m] - ms), w_par = exp2f(mp - ms);
    if (head < p.h) {
      const size_t row = unit * p.h + head;
#pragma unroll
      for (int c2 = 0; c2 < CT / 2; ++c2) {
        const f32x4 own = tw == 0 ? z[2 * c2][m] : z[2 * c2 + 1][m];
        const f32x4 got = zbuf[(((wave ^ 2) * NH + m) * (CT / 2) + c2) * 64 + lane];
        const int c = 16 * (2 * c2 + tw) + 4 * q;
        if (c < d_cb) *(f32x4*)(p.part_z + row * d_cb + c) = own * w_own + got * w_par;
      }
      if (tw == 0 && q == 0) {
        p.part_ml[row * 2 + 0] = ms;
        p.part_ml[row * 2 + 1] = l_run[m] * w_own + lbuf[at] * w_par;
      }
    }
  }
}

template <typename T, int DP, int RP, int NH, bool VEC, int PT>
int launch_terms(const DecodeArgs& a, Mx4Params& p) {
  constexpr size_t lds = lds_bytes<T, DP, RP, NH>();
  if (lds > 64 * 1024) {
    static PerDeviceSetup setup;
    int dev = -1;
    if (setup.needed(&dev)) {
      if (hipFuncSetAttribute((const void*)mx4_decode_kernel<T, DP, RP, NH, VEC, PT>,
                              hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds) != hipSuccess)
        return MLRA_ERR_LAUNCH;
      setup.done(dev);
    }
  }
  p.n_hg = (a.h + 32 * NH - 1) / (32 * NH);
  const long long wgs = (long long)a.plan.n_splits * a.n_blocks * a.batch * p.n_hg;
  // A dimension of a launch holds fewer than 2^32 threads (more wrap around without an error): rows of 2^23 workgroups.
  constexpr long long kRow = 1 << 23;
  if (wgs > 0x7fffffffLL - kRow) return MLRA_ERR_LAUNCH;
  const dim3 grid((unsigned)(wgs < kRow ? wgs : kRow), (unsigned)((wgs + kRow - 1) / kRow));
  mx4_decode_kernel<T, DP, RP, NH, VEC, PT><<<grid, 256, lds, a.stream>>>(p);
  return check_launch();
}

template <typename T, int DP, int RP, int NH, bool VEC>
int launch_one(const DecodeArgs& a, Mx4Params& p) {
  if constexpr (Terms<T>::n > 1) return launch_terms<T, DP, RP, NH, VEC, 3>(a, p);
  else return !a.precise ? launch_terms<T, DP, RP, NH, VEC, 1>(a, p)
              : a.out_dtype == MLRA_F32 ? launch_terms<T, DP, RP, NH, VEC, 3>(a, p)
                                        : launch_terms<T, DP, RP, NH, VEC, 2>(a, p);
}

template <typename T, int DP, int RP, bool VEC>
int launch_heads(const DecodeArgs& a, Mx4Params& p) {
  if constexpr (DP > 256 || (DP > 64 && Terms<T>::n > 1)) {
    return launch_one<T, DP, RP, 1, VEC>(a, p);
  } else {
    return mx4_heads_per_wg(a.h, a.d_cb, a.dtype) == 64 ? launch_one<T, DP, RP, 2, VEC>(a, p)
                                                        : launch_one<T, DP, RP, 1, VEC>(a, p);
  }
}

template <typename T, bool VEC>
int launch_typed(const DecodeArgs& a, Mx4Params& p) {
#define MLRA_MX4_RP(DP) return a.d_r <= 64 ? launch_heads<T, DP, 64, VEC>(a, p) : launch_heads<T, DP, 128, VEC>(a, p)
  if (a.d_cb <= 64) MLRA_MX4_RP(64);
  if (a.d_cb <= 128) MLRA_MX4_RP(128);
  if (a.d_cb <= 256) MLRA_MX4_RP(256);
  MLRA_MX4_RP(512);
#undef MLRA_MX4_RP
}

}  // namespace

// Heads per workgroup: 64 share a tile's trip through LDS where the queries and accumulators of 32 heads leave a lane's
// registers room for a second wave on the SIMD.
int mx4_heads_per_wg(int h, int d_cb, int dtype) {
  return h > 32 && d_cb <= (dtype == MLRA_BF16 ? 256 : 64) ? 64 : 32;
}

// (More than two fit for narrow blocks, but their chunks cost the merge more than they save: 8 sequences of 1000 to 4000 tokens
// x 16 heads x 4 blocks of 64 channels 30 us in 512 workgroups, 36 in 1024.)
int mx4_resident(int heads, int d_cb, int dtype) {
  return d_cb <= (dtype == MLRA_BF16 ? (heads == 32 ? 256 : 128) : 128) ? 2 : 1;
}

int launch_mx4_decode(const DecodeArgs& a) {
  Mx4Params p;
  p.latent = (const uint8_t*)a.latent;
  p.scales = (const uint8_t*)a.scales;
  p.rope = a.rope;
  p.page_table = a.page_table;
  p.seq_lens = a.seq_lens;
  p.q_abs = a.q_abs;
  p.q_rope = a.q_rope;
  p.part_z = a.part_z;
  p.part_ml = a.part_ml;
  p.page_size = a.page_size;
  p.max_pages = a.max_pages;
  p.n_blocks = a.n_blocks;
  p.groups = a.groups;
  p.d_cb = a.d_cb;
  p.d_r = a.d_r;
  p.h = a.h;
  p.batch = a.batch;
  p.n_splits = a.plan.n_splits;
  p.chunk = a.plan.chunk_tokens;
  p.scale_log2 = softmax_scale_log2(a.softmax_scale);
  const uintptr_t bases = (uintptr_t)a.rope | (uintptr_t)a.q_abs | (uintptr_t)a.q_rope;
  const bool vec = a.d_r % 4 == 0 && bases % (a.dtype == MLRA_BF16 ? 8 : 16) == 0;
  if (a.dtype == MLRA_BF16) return vec ? launch_typed<bf16_t, true>(a, p) : launch_typed<bf16_t, false>(a, p);
  return vec ? launch_typed<float, true>(a, p) : launch_typed<float, false>(a, p);
}

}  // namespace mlra
