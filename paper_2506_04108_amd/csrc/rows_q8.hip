// Rows into and out of an 8-bit cache: quantisation with one scale for each
// (block, kv head) and the block summaries of the new keys, and the way back.
//
// A wave takes one block of one kv head, for K or for V: lane (r, c) with
// r = lane / 16, c = lane % 16 holds dims [8c, 8c + 8) of rows r, r + 4, ...
// All rows are read before anything is written; the largest magnitude A is a
// maximum of bf16 bit patterns (an integer maximum, which a NaN wins), reduced
// across the wave; scale = max(A, 2^-100) / Q; a code is value / scale rounded
// to nearest even (see snap19). Where the block keeps rows from earlier calls
// the scale can only grow, and the codes that stay are rounded again when it
// does. Both kernels move each byte once and are bound by HBM for prompts
// (512 B in and 256 B out for a row of K and V) and by latency for a decoded
// token: one wave per block, K and V in neighbouring waves, costs it one
// round trip for the lengths and one for the rows. 8 prompts of up to 8180 rows,
// 8 kv heads: 53 us to store (236 MB, 4.4 TB/s), 35 us to load (227 MB, 6.4 TB/s);
// one token of 8 sequences 4.6 and 3.1 us. The same prompts stored, or loaded, again
// and again: 43 - 50 and 34 - 40 us in both formats, contiguous or paged, by blocks of
// 16, 32 and 64.
#include "rows_device.h"

namespace resa {
namespace {

// Items of a wave: blocks that the new rows of a sequence touch. The first 64
// sequences' rows stay in registers, so that up to there the search reads
// memory once.
__device__ __forceinline__ bool find_block(const RowsQ8Args& a, int item, int log2_block, int& bb, int& m, int& first_row,
                                           int& first, int& L) {
  struct Seq {
    int at, n, len;
  };
  const int lane = threadIdx.x & 63, b1 = (1 << log2_block) - 1;
  auto rows_at = [&](int s) -> Seq {
    Seq q;
    packed_rows(a.cu, a.rows, s, q.at, q.n);
    q.len = a.seq_lens[s];
    return q;
  };
  const Seq q0 = lane < a.c.batch ? rows_at(lane) : Seq{0, 0, 0};
  auto count = [&](int s) -> int {
    const Seq q = s < 64 ? q0 : rows_at(s);
    if (q.n == 0 || q.len < q.n || q.len > a.c.capacity) return 0;
    return ((q.len + b1) >> log2_block) - ((q.len - q.n) >> log2_block);
  };
  int rank;
  if (!find_seq(item, a.c.batch, count, bb, rank)) return false;
  const Seq q = bb < 64 ? Seq{__builtin_amdgcn_readlane(q0.at, bb & 63), __builtin_amdgcn_readlane(q0.n, bb & 63),
                              __builtin_amdgcn_readlane(q0.len, bb & 63)}
                        : rows_at(bb);
  first_row = q.at;
  L = q.len;
  first = L - q.n;
  m = (first >> log2_block) + rank;
  return true;
}

template <int kFmt, int BS>
__global__ __launch_bounds__(256) void k_store_rows_q8(RowsQ8Args a) {
  constexpr int kLog2 = BS == 16 ? 4 : BS == 32 ? 5 : 6;
  constexpr int kRows = BS / 4;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int hk = blockIdx.x % a.c.kv_heads;
  const bool is_k = (wave & 1) == 0;
  int bb, m, first_row, first, L;
  if (!find_block(a, (int)(blockIdx.x / a.c.kv_heads) * 2 + (wave >> 1), kLog2, bb, m, first_row, first, L)) return;
  const int64_t row0 = kv_row(a.c, bb, hk, m * BS);
  if (row0 < 0) return;
  const int64_t si = scale_index(a.c, bb, hk, m);
  const int r = lane >> 4, col = (lane & 15) * 8;
  uint8_t* dst = reinterpret_cast<uint8_t*>(const_cast<uint16_t*>(is_k ? a.c.k : a.c.v)) + (size_t)row0 * kHeadDim + col;
  const uint16_t* src = (is_k ? a.k_rows : a.v_rows) + (size_t)hk * kHeadDim + col;
  const int64_t stride = is_k ? a.k_stride : a.v_stride;
  float* scale = (is_k ? a.k_scale : a.v_scale) + si;
  const int keep = max(first - m * BS, 0);          // rows of this block that stay
  const int end = min(L - m * BS, BS);              // rows of this block that exist
  const size_t so = (((size_t)bb * a.c.kv_heads + hk) * a.c.max_blocks + m) * kHeadDim + col;

  U4 x[kRows];
  uint2 old[kRows];
#pragma unroll
  for (int i = 0; i < kRows; ++i) {
    const int row = r + 4 * i;
    // Every lane loads a new row that exists; those of other rows are zeroed.
    const int t = min(max(row, keep), end - 1);
    x[i] = ld16(src + (int64_t)(first_row + m * BS + t - first) * stride);
    if (row < keep || row >= end) x[i] = U4{0, 0, 0, 0};
  }
  float s_old = 0.f;
  U4 lo, hi;
  if (keep > 0) {
    s_old = *scale;
#pragma unroll
    for (int i = 0; i < kRows; ++i) old[i] = *reinterpret_cast<const uint2*>(dst + (size_t)(r + 4 * i) * kHeadDim);
    if (is_k) {
      lo = ld16(a.c.kmin + so);
      hi = ld16(a.c.kmax + so);
    }
  }
  u16x2_t top = {0, 0};
#pragma unroll
  for (int i = 0; i < kRows; ++i) {
    const uint32_t w[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
#pragma unroll
    for (int j = 0; j < 4; ++j) top = __builtin_elementwise_max(top, __builtin_bit_cast(u16x2_t, w[j] & 0x7fff7fffu));
  }
  uint32_t A = max((uint32_t)top[0], (uint32_t)top[1]);
  A = wave_max(A);
  // A block with a value that is not finite has a NaN for its scale.
  float s = A >= 0x7f80u ? __builtin_nanf("") : fmaxf(__uint_as_float(A << 16), kQ8Least) / Q8<kFmt>::kMax;
  if (keep > 0 && !(s_old <= s)) s = s == s ? s_old : s;
  const float inv = 1.f / s;
  if (keep > 0 && s_old != s) {
    const float ratio = s_old * inv;
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
      const int row = r + 4 * i;
      if (row >= keep) continue;
      uint32_t w[2] = {old[i].x, old[i].y};
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        float y[4];
        codes_f32<kFmt>(w[j], y);
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = s == s ? y[e] * ratio : 0.f;
        w[j] = to_codes<kFmt>(y);
      }
      *reinterpret_cast<uint2*>(dst + (size_t)row * kHeadDim) = uint2{w[0], w[1]};
    }
  }
#pragma unroll
  for (int i = 0; i < kRows; ++i) {
    const int row = r + 4 * i;
    const uint32_t w[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
    uint32_t out[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      float y[4] = {bf_lo(w[2 * j]) * inv, bf_hi(w[2 * j]) * inv, bf_lo(w[2 * j + 1]) * inv, bf_hi(w[2 * j + 1]) * inv};
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] = s == s ? y[e] : 0.f;
      out[j] = to_codes<kFmt>(y);
    }
    if (row >= keep && row < end) *reinterpret_cast<uint2*>(dst + (size_t)row * kHeadDim) = uint2{out[0], out[1]};
  }
  if (lane == 0) *scale = s;
  if (is_k) {
    float mn[8], mx[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      mn[j] = __builtin_inff();
      mx[j] = -__builtin_inff();
    }
    if (keep > 0) {
      float unused_mx[8], unused_mn[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        unused_mx[j] = mx[j];
        unused_mn[j] = mn[j];
      }
      fold_minmax(lo, mn, unused_mx);
      fold_minmax(hi, unused_mn, mx);
    }
#pragma unroll
    for (int i = 0; i < kRows; ++i)
      if (r + 4 * i >= keep && r + 4 * i < end) fold_minmax(x[i], mn, mx);
    store_summary(a.c, (size_t)bb * a.c.kv_heads + hk, m, r, col, mn, mx);
  }
}

template <int kFmt, int BS>
__global__ __launch_bounds__(256) void k_load_rows_q8(RowsQ8Args a) {
  constexpr int kLog2 = BS == 16 ? 4 : BS == 32 ? 5 : 6;
  constexpr int kRows = BS / 4;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int hk = blockIdx.x % a.c.kv_heads;
  const bool is_k = (wave & 1) == 0;
  int bb, m, first_row, first, L;
  if (!find_block(a, (int)(blockIdx.x / a.c.kv_heads) * 2 + (wave >> 1), kLog2, bb, m, first_row, first, L)) return;
  const int64_t row0 = kv_row(a.c, bb, hk, m * BS);
  if (row0 < 0) return;
  const int64_t si = scale_index(a.c, bb, hk, m);
  const int r = lane >> 4, col = (lane & 15) * 8;
  const uint8_t* src = reinterpret_cast<const uint8_t*>(is_k ? a.c.k : a.c.v) + (size_t)row0 * kHeadDim + col;
  uint16_t* dst = (is_k ? a.k_out : a.v_out) + (size_t)hk * kHeadDim + col;
  const float s = (is_k ? a.k_scale : a.v_scale)[si];
  const int keep = max(first - m * BS, 0), end = min(L - m * BS, BS);
  uint2 x[kRows];
#pragma unroll
  for (int i = 0; i < kRows; ++i) x[i] = *reinterpret_cast<const uint2*>(src + (size_t)(r + 4 * i) * kHeadDim);
#pragma unroll
  for (int i = 0; i < kRows; ++i) {
    const int row = r + 4 * i;
    if (row < keep || row >= end) continue;
    float y[4], z[4];
    codes_f32<kFmt>(x[i].x, y);
    codes_f32<kFmt>(x[i].y, z);
    st16(dst + (size_t)(first_row + m * BS + row - first) * a.c.kv_heads * kHeadDim,
         U4{pack_bf16(y[0] * s, y[1] * s), pack_bf16(y[2] * s, y[3] * s), pack_bf16(z[0] * s, z[1] * s),
            pack_bf16(z[2] * s, z[3] * s)});
  }
}

template <int kFmt>
hipError_t launch(const RowsQ8Args& a, bool load, hipStream_t stream) {
  // Blocks touched: at most rows / b + 2 a sequence, and one a row.
  const int64_t by_len = a.rows / a.c.block_size + 2 * (int64_t)a.c.batch;
  const int64_t items = by_len < a.rows ? by_len : a.rows;
  const dim3 grid((uint32_t)((items + 1) / 2 * a.c.kv_heads));
  auto go = [&](auto* store, auto* read) {
    if (load)
      hipLaunchKernelGGL(read, grid, dim3(256), 0, stream, a);
    else
      hipLaunchKernelGGL(store, grid, dim3(256), 0, stream, a);
    return hipGetLastError();
  };
  switch (a.c.block_size) {
    case 16: return go(k_store_rows_q8<kFmt, 16>, k_load_rows_q8<kFmt, 16>);
    case 32: return go(k_store_rows_q8<kFmt, 32>, k_load_rows_q8<kFmt, 32>);
    case 64: return go(k_store_rows_q8<kFmt, 64>, k_load_rows_q8<kFmt, 64>);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace

hipError_t launch_store_rows_q8(const RowsQ8Args& a, hipStream_t stream) {
  return a.format == RESA_Q8_INT8 ? launch<RESA_Q8_INT8>(a, false, stream) : launch<RESA_Q8_E4M3>(a, false, stream);
}
hipError_t launch_load_rows_q8(const RowsQ8Args& a, hipStream_t stream) {
  return a.format == RESA_Q8_INT8 ? launch<RESA_Q8_INT8>(a, true, stream) : launch<RESA_Q8_E4M3>(a, true, stream);
}

}  // namespace resa
