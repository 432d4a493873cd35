// The latent cache in 4 bits: rows written into their pages and read back.
//
// Format (OCP MX, E2M1 elements with E8M0 scales): 32 neighbouring channels of a token share a byte E, a channel is a 4-bit
// code, sign | two exponent bits | one mantissa bit, and stands for +-{0, 0.5, 1, 1.5, 2, 3, 4, 6} 2^(E - 127).
//   E     = clamp(exponent of the largest magnitude as one mantissa bit rounds it - 2, 2, 252): magnitudes from 1.75 2^e on
//           count as 2^(e+1).  Root mean square error on normal channels 0.112; 0.115 with the exponent of the magnitude
//           itself, and with the smallest power of two that cuts nothing off.  The bounds keep every value a normal number
//           of bf16, or zero.
//   codes = x 2^(127 - E) rounded to nearest, ties to the even mantissa, cut off at 6.  The scaling is exact, so the codes
//           are those of the exact quotient.
// A group that holds an infinity or a NaN is stored as E = 255 and zeros, and reads as NaN.
//
// Both kernels are streams, bound by memory: a wavefront takes four tokens, whose pages are scalar, and a lane eight channels
// of each: 16 or 32 bytes on the wide side, 4 on the narrow one, a quarter of a group.  Four tokens keep enough loads in flight (two
// and eight are slower).  Four blocks of 128 channels: written from fp32, 295,000 tokens, 157 us, 5.1 TB/s with what is read;
// read to bf16, 64 x 8192, 180 us, 4.5 TB/s.
#include "mx4_tile.h"

namespace mlra {
namespace {

using namespace mx4_tile;

struct RowsParams {
  uint8_t* latent;        // [num_pages][n_blocks][page_size][d_cb / 2]
  uint8_t* scales;        // [num_pages][n_blocks][page_size][d_cb / 32]
  void* rope;             // [num_pages][page_size][d_r]
  const int32_t* page_table;
  const int32_t* positions;   // [batch] first slot
  const int32_t* row_lens;    // [batch], or null: n_rows each
  void* c_kv;             // [batch][n_rows][n_blocks * d_cb]
  void* k_rope;           // [batch][n_rows][d_r]
  int num_pages, page_size, max_pages, n_blocks, d_cb, d_r, n_rows;
};

constexpr int kTokensWave = 4, kTokensWG = 16;

// eight channels, fp32 or bf16
__device__ __forceinline__ void load8(const float* p, bool aligned, float (&x)[8]) {
  if (aligned) {
    const f32x4 a = *(const f32x4*)p, b = *(const f32x4*)(p + 4);
#pragma unroll
    for (int e = 0; e < 4; ++e) { x[e] = a[e]; x[4 + e] = b[e]; }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = p[e];
  }
}
__device__ __forceinline__ void load8(const bf16_t* p, bool aligned, float (&x)[8]) {
  if (aligned) {
    const u32x4 a = *(const u32x4*)p;
#pragma unroll
    for (int e = 0; e < 4; ++e) { x[2 * e] = __uint_as_float(a[e] << 16); x[2 * e + 1] = __uint_as_float(a[e] & 0xffff0000u); }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = bf16_to_f32(p[e]);
  }
}
__device__ __forceinline__ void store8(float* p, bool aligned, const u32x4& v) {
  float x[8];
#pragma unroll
  for (int e = 0; e < 4; ++e) { x[2 * e] = __uint_as_float(v[e] << 16); x[2 * e + 1] = __uint_as_float(v[e] & 0xffff0000u); }
  if (aligned) {
    __builtin_nontemporal_store(f32x4{x[0], x[1], x[2], x[3]}, (f32x4*)p);
    __builtin_nontemporal_store(f32x4{x[4], x[5], x[6], x[7]}, (f32x4*)(p + 4));
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) p[e] = x[e];
  }
}
__device__ __forceinline__ void store8(bf16_t* p, bool aligned, const u32x4& v) {
  if (aligned) {
    __builtin_nontemporal_store(v, (u32x4*)p);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) { p[2 * e] = (bf16_t)v[e]; p[2 * e + 1] = (bf16_t)(v[e] >> 16); }
  }
}

// The tokens of a wave: where they lie is the same for all lanes.
struct Tokens {
  long long page[kTokensWave];
  int slot[kTokensWave];
  bool ok[kTokensWave];      // the row exists and has a slot in the cache
};
__device__ __forceinline__ Tokens tokens_of(const RowsParams& p, int s, int first) {
  Tokens t;
  const int pos = p.positions[s], rows = p.row_lens ? min(p.row_lens[s], p.n_rows) : p.n_rows;
  const long long at = (long long)pos + first;                     // slot of the first one in the sequence
  const bool any = pos >= 0 && first < rows && at < (long long)p.max_pages * p.page_size;
  unsigned index = any ? (unsigned)at / (unsigned)p.page_size : 0u, slot = any ? (unsigned)at % (unsigned)p.page_size : 0u;
#pragma unroll
  for (int u = 0; u < kTokensWave; ++u) {
    const bool in = any && first + u < rows && index < (unsigned)p.max_pages;
    const int page = __builtin_amdgcn_readfirstlane(in ? p.page_table[(size_t)s * p.max_pages + index] : 0);
    t.ok[u] = in && (unsigned)page < (unsigned)p.num_pages;
    t.page[u] = page;
    t.slot[u] = (int)slot;
    if (++slot == (unsigned)p.page_size) {
      slot = 0;
      ++index;
    }
  }
  return t;
}

// RoPE keys of the wave's tokens, one channel a lane: get and put take an element's index in the pool and in the rows (from
// the wave's first one on).  All tokens' are in flight before the first is stored.
template <typename Get, typename Put>
__device__ __forceinline__ void each_rope(const RowsParams& p, const Tokens& t, Get get, Put put) {
  for (int e = threadIdx.x & 63; e < p.d_r; e += 64) {
    float x[kTokensWave];
#pragma unroll
    for (int u = 0; u < kTokensWave; ++u)
      if (t.ok[u]) x[u] = get((size_t)(t.page[u] * p.page_size + t.slot[u]) * p.d_r + e, (size_t)u * p.d_r + e);
#pragma unroll
    for (int u = 0; u < kTokensWave; ++u)
      if (t.ok[u]) put((size_t)(t.page[u] * p.page_size + t.slot[u]) * p.d_r + e, (size_t)u * p.d_r + e, x[u]);
  }
}

// TS: type of the rows, TC: of the RoPE pool
template <typename TS, typename TC>
__global__ __launch_bounds__(256) void mx4_append_kernel(RowsParams p, bool aligned) {
  const int s = blockIdx.y, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int first = blockIdx.x * kTokensWG + wave * kTokensWave, d_c = p.n_blocks * p.d_cb;
  const Tokens t = tokens_of(p, s, first);
  const long long planes = (long long)p.n_blocks * p.page_size;            // rows of all blocks of a page
  const size_t row0 = (size_t)s * p.n_rows + first;
  const TS* const src = (const TS*)p.c_kv + row0 * d_c;
  const TS* const k_src = (const TS*)p.k_rope + row0 * p.d_r;
  for (int c0 = 0; c0 < d_c; c0 += 512) {
    const int c = c0 + 8 * lane, cc = c < d_c ? c : 0, b = cc / p.d_cb, cb = cc - b * p.d_cb;
    const size_t plane = (size_t)b * p.page_size, code_at = plane * (p.d_cb / 2) + cb / 2,
                 scale_at = plane * (p.d_cb / kGroup) + cb / kGroup;       // of this lane, from row 0 of the page on
    float x[kTokensWave][8];
#pragma unroll
    for (int u = 0; u < kTokensWave; ++u)
      if (t.ok[u]) load8(src + (size_t)u * d_c + cc, aligned, x[u]);
#pragma unroll
    for (int u = 0; u < kTokensWave; ++u) {
      if (!t.ok[u]) continue;
      // the largest magnitude of the group, as bits (of non-negative floats they are ordered like the values)
      unsigned top = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(x[u][e]) & 0x7fffffffu);
      top = max(top, (unsigned)__shfl_xor((int)top, 1));
      top = max(top, (unsigned)__shfl_xor((int)top, 2));
      const unsigned byte = scale_byte(top);
      const unsigned codes = byte == kNaNScale ? 0u : encode8(x[u], byte);
      if (c < d_c) {
        *(unsigned*)(p.latent + (t.page[u] * planes + t.slot[u]) * (p.d_cb / 2) + code_at) = codes;
        if ((lane & 3) == 0) p.scales[(t.page[u] * planes + t.slot[u]) * (p.d_cb / kGroup) + scale_at] = (uint8_t)byte;
      }
    }
  }
  each_rope(p, t, [&](size_t, size_t own) { return load_f32(k_src, own); },
            [&](size_t pool, size_t, float x) { store_f32((TC*)p.rope, pool, x); });
}

template <typename TS, typename TC>
__global__ __launch_bounds__(256) void mx4_read_kernel(RowsParams p, bool aligned) {
  const int s = blockIdx.y, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int first = blockIdx.x * kTokensWG + wave * kTokensWave, d_c = p.n_blocks * p.d_cb;
  const Tokens t = tokens_of(p, s, first);
  const long long planes = (long long)p.n_blocks * p.page_size;            // rows of all blocks of a page
  const size_t row0 = (size_t)s * p.n_rows + first;
  TS* const dst = (TS*)p.c_kv + row0 * d_c;
  TS* const k_dst = (TS*)p.k_rope + row0 * p.d_r;
  for (int c0 = 0; c0 < d_c; c0 += 512) {
    const int c = c0 + 8 * lane, cc = c < d_c ? c : 0, b = cc / p.d_cb, cb = cc - b * p.d_cb;
    const size_t plane = (size_t)b * p.page_size, code_at = plane * (p.d_cb / 2) + cb / 2,
                 scale_at = plane * (p.d_cb / kGroup) + cb / kGroup;       // of this lane, from row 0 of the page on
    unsigned codes[kTokensWave], byte[kTokensWave];
#pragma unroll
    for (int u = 0; u < kTokensWave; ++u)
      if (t.ok[u]) {
        codes[u] = *(const unsigned*)(p.latent + (t.page[u] * planes + t.slot[u]) * (p.d_cb / 2) + code_at);
        byte[u] = p.scales[(t.page[u] * planes + t.slot[u]) * (p.d_cb / kGroup) + scale_at];
      }
#pragma unroll
    for (int u = 0; u < kTokensWave; ++u)
      if (t.ok[u] && c < d_c) store8(dst + (size_t)u * d_c + c, aligned, decode8(codes[u], scale_of(byte[u])));
  }
  each_rope(p, t, [&](size_t pool, size_t) { return load_f32((const TC*)p.rope, pool); },
            [&](size_t, size_t own, float x) { store_f32(k_dst, own, x); });
}

RowsParams rows_params(const mlra_mx4_cache* c, int n_rows, const int32_t* positions, const int32_t* row_lens,
                       const void* c_kv, const void* k_rope) {
  RowsParams p;
  p.latent = (uint8_t*)c->latent;
  p.scales = (uint8_t*)c->scales;
  p.rope = c->rope;
  p.page_table = c->page_table;
  p.positions = positions;
  p.row_lens = row_lens;
  p.c_kv = const_cast<void*>(c_kv);
  p.k_rope = const_cast<void*>(k_rope);
  p.num_pages = c->num_pages;
  p.page_size = c->page_size;
  p.max_pages = c->max_pages_per_seq;
  p.n_blocks = c->n_blocks;
  p.d_cb = c->d_cb;
  p.d_r = c->d_r;
  p.n_rows = n_rows;
  return p;
}

}  // namespace

int launch_mx4_append(const mlra_mx4_cache* c, int batch, int n_rows, const void* c_kv, const void* k_rope, int src_dtype,
                      const int32_t* positions, const int32_t* row_lens, hipStream_t stream) {
  const RowsParams p = rows_params(c, n_rows, positions, row_lens, c_kv, k_rope);
  const bool aligned = (uintptr_t)c_kv % 16 == 0;
  const dim3 grid((n_rows + kTokensWG - 1) / kTokensWG, batch);
#define MLRA_MX4_APPEND(TS, TC) mx4_append_kernel<TS, TC><<<grid, 256, 0, stream>>>(p, aligned)
  if (src_dtype == MLRA_BF16 && c->dtype == MLRA_BF16) MLRA_MX4_APPEND(bf16_t, bf16_t);
  else if (src_dtype == MLRA_BF16) MLRA_MX4_APPEND(bf16_t, float);
  else if (c->dtype == MLRA_BF16) MLRA_MX4_APPEND(float, bf16_t);
  else MLRA_MX4_APPEND(float, float);
#undef MLRA_MX4_APPEND
  return check_launch();
}

int launch_mx4_read(const mlra_mx4_cache* c, int batch, int n_rows, const int32_t* positions, const int32_t* row_lens,
                    void* c_kv, void* k_rope, int dst_dtype, hipStream_t stream) {
  const RowsParams p = rows_params(c, n_rows, positions, row_lens, c_kv, k_rope);
  const bool aligned = (uintptr_t)c_kv % 16 == 0;
  const dim3 grid((n_rows + kTokensWG - 1) / kTokensWG, batch);
#define MLRA_MX4_READ(TS, TC) mx4_read_kernel<TS, TC><<<grid, 256, 0, stream>>>(p, aligned)
  if (dst_dtype == MLRA_BF16 && c->dtype == MLRA_BF16) MLRA_MX4_READ(bf16_t, bf16_t);
  else if (dst_dtype == MLRA_BF16) MLRA_MX4_READ(bf16_t, float);
  else if (c->dtype == MLRA_BF16) MLRA_MX4_READ(float, bf16_t);
  else MLRA_MX4_READ(float, float);
#undef MLRA_MX4_READ
  return check_launch();
}

}  // namespace mlra
