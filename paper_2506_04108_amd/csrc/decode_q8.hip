// Block-sparse flash-decoding (Eq. 2; App. A, Alg. 2) over an 8-bit cache, on
// the matrix cores.
//
// As in the bf16 decode, grid (num_splits, kv_heads, batch), a split per
// workgroup of 4 waves, and the splits of a group are merged by log-sum-exp by
// the last of them to finish. A selected block is cut into 16-token halves and
// two halves in a row make a chunk of 32 tokens, the unit that is dealt to the
// splits and their waves. Converting the codes and multiplying them on the
// VALU would cost a multiply-add per code and query head (8 heads: 80 a clock
// and CU at 6 TB/s, more than a CU has), so both products are MFMAs, whose
// operands are bf16: every code (int8, e4m3) is a bf16 value.
//
// Lane (r, c), r = lane / 16, c = lane % 16. Per chunk:
//   S^T = K . Q^T   two halves x four v_mfma_f32_16x16x32_bf16 (tokens x
//                   heads). Lane (r, c) holds 32 bytes of token c: dims
//                   16 r .. + 16 and 64 + 16 r .. + 16 (two 16-byte loads, each
//                   wave-wide load covers 64 bytes of 16 rows); the
//                   contraction runs over the dims in that order, and Q's rows
//                   are held in the same. Lane (r, c) receives the scores of
//                   head c % 8 for tokens 4 r .. + 4 of each half.
//   weights         2^(S ks - m) in fp32, ks the block's key scale times the
//                   softmax scale; times the block's value scale
//   O^T += V^T . P  eight times two v_mfma_f32_16x16x32_bf16 (dims x heads):
//                   the tokens of lane (r, c) are the ones whose weights it
//                   holds, so P needs no exchange between lanes; V rows are
//                   read as 8 bytes a lane (dims 8 c .. + 8 of eight tokens)
//                   and transposed inside the lane, by the choice of the two
//                   values that a packing instruction takes.
// Precision: a weight (fp32) is the exact sum of three bf16 terms (8
// significant bits each). Columns 0 .. 7 of P hold the first terms of the 8
// heads and columns 8 .. 15 the second, so a group of up to 8 heads fills the
// 16 columns, and a second MFMA takes the third terms; products are exact and
// sums fp32. So the result is as exact as with fp32 arithmetic throughout, for
// any range of the scales (they multiply the weight before it is split).
//
// Bound by HBM (256 B a token and kv head); MFMA and VALU take about a third of
// the time that the codes take to arrive.
#include "decode_impl.h"
#include "rows_device.h"

namespace resa {
namespace {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));

constexpr int kDecodeWaves = 4;
// Chunks in flight per wave while one is consumed.
constexpr int kDecodeDepth = 1;

template <int G, int NW>
struct DecodeQ8Lds {
  __attribute__((aligned(16))) float racc[NW][G][kHeadDim];
  float rm[G][NW], rl[G][NW];
  __attribute__((aligned(16))) float own_o[G * kHeadDim];
  float own_l[G];
  int tok[kIdxBatch];   // first token of each half, -1: none
  int row[kIdxBatch];
  __attribute__((aligned(16))) float w[kMaxSplits * G];
  f4_t red[64 * NW];
  uint32_t ticket;
};

struct ChunkQ8 {
  U4 k[2][2];     // [half][bytes 16 r and 64 + 16 r of token c]
  uint2 v[8];     // bytes 8 c of tokens 4 r + j of half 0 (j < 4) and half 1
  float scale;    // lanes of r = 0, 1: key scales of the halves; r = 2, 3: value scales
};

// Eight codes as bf16.
template <int kFmt>
__device__ __forceinline__ bf16x8_t codes_bf16(uint32_t a, uint32_t b) {
  U4 out;
  if constexpr (kFmt == RESA_Q8_INT8) {
    float x[4], y[4];
    codes_f32<kFmt>(a, x);
    codes_f32<kFmt>(b, y);
    out = U4{__builtin_amdgcn_perm(__float_as_uint(x[1]), __float_as_uint(x[0]), 0x07060302u),
             __builtin_amdgcn_perm(__float_as_uint(x[3]), __float_as_uint(x[2]), 0x07060302u),
             __builtin_amdgcn_perm(__float_as_uint(y[1]), __float_as_uint(y[0]), 0x07060302u),
             __builtin_amdgcn_perm(__float_as_uint(y[3]), __float_as_uint(y[2]), 0x07060302u)};
  } else {
    out = U4{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.f, false)),
             __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.f, true)),
             __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.f, false)),
             __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.f, true))};
  }
  return __builtin_bit_cast(bf16x8_t, out);
}

// Dims 4 e .. 4 e + 3 of the lane's eight tokens (words w[0 .. 7]), transposed:
// out[d] holds the eight tokens' values of dim d.
template <int kFmt>
__device__ __forceinline__ void transpose_bf16(const uint32_t (&w)[8], bf16x8_t (&out)[4]) {
  uint32_t o[4][4];
  if constexpr (kFmt == RESA_Q8_INT8) {
#pragma unroll
    for (int t = 0; t < 8; t += 2) {
      float x[4], y[4];
      codes_f32<kFmt>(w[t], x);
      codes_f32<kFmt>(w[t + 1], y);
#pragma unroll
      for (int d = 0; d < 4; ++d)
        o[d][t / 2] = __builtin_amdgcn_perm(__float_as_uint(y[d]), __float_as_uint(x[d]), 0x07060302u);
    }
  } else {
#pragma unroll
    for (int t = 0; t < 8; t += 2) {
      auto pair = [&](int u, bool hi) {
        return hi ? __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[u], 1.f, true))
                  : __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[u], 1.f, false));
      };
      const uint32_t x0 = pair(t, false), x1 = pair(t, true), y0 = pair(t + 1, false), y1 = pair(t + 1, true);
      o[0][t / 2] = __builtin_amdgcn_perm(y0, x0, 0x05040100u);
      o[1][t / 2] = __builtin_amdgcn_perm(y0, x0, 0x07060302u);
      o[2][t / 2] = __builtin_amdgcn_perm(y1, x1, 0x05040100u);
      o[3][t / 2] = __builtin_amdgcn_perm(y1, x1, 0x07060302u);
    }
  }
#pragma unroll
  for (int d = 0; d < 4; ++d) out[d] = __builtin_bit_cast(bf16x8_t, U4{o[d][0], o[d][1], o[d][2], o[d][3]});
}

__device__ __forceinline__ f32x4_t mfma16(bf16x8_t a, bf16x8_t b, f32x4_t c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

template <int G, int BS, int kFmt, int NW, int kDepth>
__device__ __forceinline__ void decode_split_q8(const DecodeArgs& a, const float* k_scale, const float* v_scale, int bb,
                                                int hk, int split, DecodeQ8Lds<G, NW>& lds) {
  constexpr int HPB = BS / 16;  // halves per block
  constexpr int kLog2 = BS == 16 ? 4 : BS == 32 ? 5 : 6;
  constexpr int NT = 64 * NW;
  constexpr int kPer = kIdxBatch / NT;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int S = a.num_splits;
  const size_t grp = (size_t)bb * a.c.kv_heads + hk;
  // The group's chunks are dealt to the splits one by one (split s holds
  // chunks s, s + S, ...), so the id loads do not wait for the count.
  auto half_of = [&](int i) { return 2 * ((i >> 1) * S + split) + (i & 1); };
  auto count_below = [&](int T) { return T > split ? (T - split + S - 1) / S : 0; };
  const int slots = 2 * count_below((a.n_cap * HPB + 1) / 2);
  const int r = lane >> 4, c = lane & 15;
  const int32_t* idx = a.block_idx + grp * a.n_cap;
  int blkv[kPer];
  auto load_ids = [&](int hb) {
    const int lim = min(slots, hb + kIdxBatch) - hb;
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      const int i = tid + j * NT;
      const int at = half_of(hb + i) / HPB;
      blkv[j] = i < lim && at < a.n_cap ? idx[at] : -1;
    }
  };
  load_ids(0);

  // Q (B of S^T): column c is head c % 8, zero past the group.
  bf16x8_t q[4];
  {
    const int head = c & 7;
    const uint16_t* qp = a.q + ((size_t)bb * a.q_heads + (size_t)hk * G + min(head, G - 1)) * kHeadDim + 16 * r;
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      U4 x = ld16(qp + 64 * (s >> 1) + 8 * (s & 1));
      if (head >= G) x = U4{0, 0, 0, 0};
      q[s] = __builtin_bit_cast(bf16x8_t, x);
    }
  }
  const bool paged = a.c.table != nullptr;
  const size_t gbase = paged ? 0 : grp * (size_t)a.c.capacity * kHeadDim;
  const uint8_t* kp = wave_uniform(reinterpret_cast<const uint8_t*>(a.c.k) + gbase);
  const uint8_t* vp = wave_uniform(reinterpret_cast<const uint8_t*>(a.c.v) + gbase);
  // This lane's scale: of half r % 2, the key's or the value's.
  const float* sp = (r < 2 ? k_scale : v_scale) + (paged ? 0 : grp * a.c.max_blocks);
  const float scale = a.scale_log2;
  const float ninf = -__builtin_inff();
  const int n_raw = __hip_atomic_load(a.num_sel + grp, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  const int L = __hip_atomic_load(a.seq_lens + bb, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  uint32_t epoch = __hip_atomic_load(a.epochs + grp, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  const int M = min((L + BS - 1) / BS, a.c.max_blocks);
  const int n = max(0, min(n_raw, a.n_cap));
  const int halves = n * HPB;
  const int valid = 2 * count_below((halves + 1) / 2);  // this split's halves

  auto load_chunk = [&](ChunkQ8& ch, int row0, int row1) __attribute__((always_inline)) {
    constexpr int kBytes = 16 * kHeadDim;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const size_t base = (size_t)(h == 0 ? row0 : row1) * kHeadDim;
      const __amdgpu_buffer_rsrc_t rk =
          __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(kp + base), (short)0, kBytes, kBufWord3);
      const __amdgpu_buffer_rsrc_t rv =
          __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(vp + base), (short)0, kBytes, kBufWord3);
#pragma unroll
      for (int e = 0; e < 2; ++e)
        ch.k[h][e] = __builtin_bit_cast(U4, __builtin_amdgcn_raw_buffer_load_b128(
                                                rk, c * kHeadDim + 16 * r + 64 * e, 0, kPolicyNt));
#pragma unroll
      for (int j = 0; j < 4; ++j)
        ch.v[4 * h + j] = __builtin_bit_cast(uint2, __builtin_amdgcn_raw_buffer_load_b64(
                                                        rv, (4 * r + j) * kHeadDim + 8 * c, 0, kPolicyNt));
    }
    ch.scale = sp[((r & 1) == 0 ? row0 : row1) >> kLog2];
  };

  // Head c % 8: softmax reference m (the same in the four lanes of a column)
  // and this lane's share l of the sum of the weights.
  float m = ninf, l = 0.f;
  f32x4_t o[8];
#pragma unroll
  for (int d = 0; d < 8; ++d) o[d] = f32x4_t{0.f, 0.f, 0.f, 0.f};

  auto consume = [&](ChunkQ8& ch, int t0, int t1) __attribute__((always_inline)) {
    float x[8], vs[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      f32x4_t s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        s = mfma16(codes_bf16<kFmt>(ch.k[h][e].x, ch.k[h][e].y), q[2 * e], s);
        s = mfma16(codes_bf16<kFmt>(ch.k[h][e].z, ch.k[h][e].w), q[2 * e + 1], s);
      }
      const float ks = scale * __builtin_bit_cast(float, __builtin_amdgcn_readlane(__float_as_int(ch.scale), 16 * h));
      vs[h] = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__float_as_int(ch.scale), 32 + 16 * h));
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        // Rounded here, as the reference that is taken of it (a product
        // contracted with the subtraction below could exceed it by far).
        x[4 * h + i] = s[i] * ks;
        __asm__("" : "+v"(x[4 * h + i]));
      }
    }
    // Halves that are none or reach past the sequence: what their rows hold
    // is not used (it may be no number at all).
    const bool partial = t0 < 0 || t1 < 0 || t0 + 16 > L || t1 + 16 > L;
    if (__builtin_expect(partial, 0)) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int t = j < 4 ? t0 : t1;
        if (t < 0 || t + 4 * r + (j & 3) >= L) {
          x[j] = ninf;
          ch.v[j] = uint2{0u, 0u};
        }
      }
      if (t0 < 0) vs[0] = 0.f;
      if (t1 < 0) vs[1] = 0.f;
    }
    float cm = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
    // The reference moves only when a score exceeds it by more than
    // kRefSlack, so the reduction over the column and the rescale are rare.
    if (__any(cm > m + kRefSlack)) {
      const float alpha = move_ref(m, max_xor32(max_xor16(cm)));
      l *= alpha;
#pragma unroll
      for (int d = 0; d < 8; ++d) o[d] *= alpha;
    }
    const float mref = m == ninf ? 0.f : m;
    float p[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) p[j] = fast_exp2(x[j] - mref);
    l += ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
    uint32_t b1[8], b2[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      float w = p[j] * vs[j >> 2];
      if (partial) w = x[j] == ninf ? 0.f : w;
      const float r1 = w - __uint_as_float(__float_as_uint(w) & 0xffff0000u);
      const float r2 = r1 - __uint_as_float(__float_as_uint(r1) & 0xffff0000u);
      b1[j] = __float_as_uint(c < 8 ? w : r1);
      b2[j] = __float_as_uint(c < 8 ? r2 : 0.f);
    }
    U4 f1, f2;
    f1 = U4{__builtin_amdgcn_perm(b1[1], b1[0], 0x07060302u), __builtin_amdgcn_perm(b1[3], b1[2], 0x07060302u),
            __builtin_amdgcn_perm(b1[5], b1[4], 0x07060302u), __builtin_amdgcn_perm(b1[7], b1[6], 0x07060302u)};
    f2 = U4{__builtin_amdgcn_perm(b2[1], b2[0], 0x07060302u), __builtin_amdgcn_perm(b2[3], b2[2], 0x07060302u),
            __builtin_amdgcn_perm(b2[5], b2[4], 0x07060302u), __builtin_amdgcn_perm(b2[7], b2[6], 0x07060302u)};
    const bf16x8_t p1 = __builtin_bit_cast(bf16x8_t, f1), p2 = __builtin_bit_cast(bf16x8_t, f2);
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      uint32_t w[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) w[j] = e == 0 ? ch.v[j].x : ch.v[j].y;
      bf16x8_t vt[4];
      transpose_bf16<kFmt>(w, vt);
#pragma unroll
      for (int d = 0; d < 4; ++d) o[4 * e + d] = mfma16(vt[d], p1, o[4 * e + d]);
#pragma unroll
      for (int d = 0; d < 4; ++d) o[4 * e + d] = mfma16(vt[d], p2, o[4 * e + d]);
    }
  };

  int hb = 0;
  do {
    if (hb > 0) load_ids(hb);
    const int he = min(valid, hb + kIdxBatch);
    const int lim = min(slots, hb + kIdxBatch) - hb;
    int tk[kPer], rw[kPer];
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      const int i = tid + j * NT, hh = half_of(hb + i), blk = blkv[j];
      tk[j] = (i >= lim || hh >= halves || blk < 0 || blk >= M) ? -1 : blk * BS + (hh % HPB) * 16;
      rw[j] = tk[j];
    }
    if (paged) {
      int page[kPer];
#pragma unroll
      for (int j = 0; j < kPer; ++j)
        page[j] = tk[j] >= 0 ? a.c.table[(size_t)bb * a.c.max_blocks + blkv[j]] : -1;
#pragma unroll
      for (int j = 0; j < kPer; ++j) {
        const int hh = half_of(hb + tid + j * NT);
        if (tk[j] >= 0) {
          if ((unsigned)page[j] < (unsigned)a.c.num_pages)
            rw[j] = (page[j] * a.c.kv_heads + hk) * BS + (hh % HPB) * 16;
          else
            tk[j] = -1;
        }
      }
    }
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      const int i = tid + j * NT;
      if (i < lim) {
        lds.tok[i] = tk[j];
        lds.row[i] = tk[j] < 0 ? 0 : rw[j];
      }
    }
    lds_sync();
    // Chunk cc of the pass: halves 2 cc and 2 cc + 1. Wave w takes chunks
    // w, w + NW, ...; kDepth + 1 buffers, as in the bf16 decode.
    const int chunks = (he - hb) / 2;
    auto tok = [&](int cc, int h) -> int {
      return cc < chunks ? __builtin_amdgcn_readfirstlane(lds.tok[2 * cc + h]) : -1;
    };
    auto row = [&](int cc, int h) -> int { return __builtin_amdgcn_readfirstlane(lds.row[2 * cc + h]); };
    ChunkQ8 ring[kDepth + 1];
    int tring[kDepth + 1][2];
    int cc = wave;
#pragma unroll
    for (int k = 0; k <= kDepth; ++k) {
      tring[k][0] = tok(cc + k * NW, 0);
      tring[k][1] = tok(cc + k * NW, 1);
      if (cc + k * NW < chunks) load_chunk(ring[k], row(cc + k * NW, 0), row(cc + k * NW, 1));
    }
    __builtin_amdgcn_sched_barrier(0);
    while (cc < chunks) {
#pragma unroll
      for (int k = 0; k <= kDepth; ++k) {
        if (cc < chunks) {
          consume(ring[k], tring[k][0], tring[k][1]);
          __builtin_amdgcn_sched_barrier(0);
          const int next = cc + (kDepth + 1) * NW;
          tring[k][0] = tok(next, 0);
          tring[k][1] = tok(next, 1);
          if (next < chunks) load_chunk(ring[k], row(next, 0), row(next, 1));
          __builtin_amdgcn_sched_barrier(0);
          cc += NW;
        }
      }
    }
    lds_sync();
    hb += kIdxBatch;
  } while (hb < valid);

  __builtin_amdgcn_s_waitcnt(kWaitVmcnt0);
  uint32_t ticket = 0;
  if (S > 1 && tid == 0)
    ticket = __hip_atomic_fetch_add(a.counters + grp, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);

  // The wave's state to LDS: the three terms' products are added (columns c
  // and c ^ 8), dims 8 (4 r + i) + d.
  const float lt = sum_xor32(sum_xor16(l));
#pragma unroll
  for (int d = 0; d < 8; ++d)
#pragma unroll
    for (int i = 0; i < 4; ++i) o[d][i] += dpp<kDppRor8>(o[d][i]);
  if (c < G) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f4_t* dst = reinterpret_cast<f4_t*>(&lds.racc[wave][c][8 * (4 * r + i)]);
      dst[0] = f4_t{o[0][i], o[1][i], o[2][i], o[3][i]};
      dst[1] = f4_t{o[4][i], o[5][i], o[6][i], o[7][i]};
    }
    if (r == 0) {
      lds.rm[c][wave] = m;
      lds.rl[c][wave] = lt;
    }
  }
  lds_sync();
  constexpr int kItems = (G * 64 + NT - 1) / NT;
  f2_t val[kItems];
  float lg[kItems];
#pragma unroll
  for (int k = 0; k < kItems; ++k) {
    const int it = tid + k * NT;
    val[k] = f2_t{0.f, 0.f};
    lg[k] = ninf;
    if (it < G * 64) {
      const int h = it / 64, d = 2 * (it % 64);
      float mx = ninf;
#pragma unroll
      for (int w = 0; w < NW; ++w) mx = fmaxf(mx, lds.rm[h][w]);
      float ls = 0.f;
      f2_t x = {0.f, 0.f};
#pragma unroll
      for (int w = 0; w < NW; ++w) {
        const float f = lds.rm[h][w] == ninf ? 0.f : fast_exp2(lds.rm[h][w] - mx);
        ls = fmaf(lds.rl[h][w], f, ls);
        x += f * *reinterpret_cast<const f2_t*>(&lds.racc[w][h][d]);
      }
      if (!(ls <= 0.f)) {
        val[k] = x * (1.f / ls);
        lg[k] = mx + fast_log2(ls);
      }
    }
  }
  finish_split<G, NW>(a, grp, split, (size_t)bb * a.q_heads + (size_t)hk * G, ticket, epoch, val, lg, lds);
}

template <int G, int BS, int kFmt>
__global__ __launch_bounds__(64 * kDecodeWaves) void k_decode_q8(DecodeArgs a, const float* k_scale,
                                                                 const float* v_scale) {
  __shared__ DecodeQ8Lds<G, kDecodeWaves> lds;
  decode_split_q8<G, BS, kFmt, kDecodeWaves, kDecodeDepth>(a, k_scale, v_scale, blockIdx.z, blockIdx.y, blockIdx.x, lds);
}

template <int G, int kFmt>
hipError_t launch_g(const DecodeArgs& a, const float* ks, const float* vs, hipStream_t stream) {
  const dim3 grid(a.num_splits, a.c.kv_heads, a.c.batch), block(64 * kDecodeWaves);
  switch (a.c.block_size) {
    case 16: hipLaunchKernelGGL((k_decode_q8<G, 16, kFmt>), grid, block, 0, stream, a, ks, vs); break;
    case 32: hipLaunchKernelGGL((k_decode_q8<G, 32, kFmt>), grid, block, 0, stream, a, ks, vs); break;
    case 64: hipLaunchKernelGGL((k_decode_q8<G, 64, kFmt>), grid, block, 0, stream, a, ks, vs); break;
    default: return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

template <int kFmt>
hipError_t launch_fmt(const DecodeArgs& a, const float* ks, const float* vs, hipStream_t stream) {
  switch (a.group) {
    case 1: return launch_g<1, kFmt>(a, ks, vs, stream);
    case 2: return launch_g<2, kFmt>(a, ks, vs, stream);
    case 3: return launch_g<3, kFmt>(a, ks, vs, stream);
    case 4: return launch_g<4, kFmt>(a, ks, vs, stream);
    case 5: return launch_g<5, kFmt>(a, ks, vs, stream);
    case 6: return launch_g<6, kFmt>(a, ks, vs, stream);
    case 7: return launch_g<7, kFmt>(a, ks, vs, stream);
    case 8: return launch_g<8, kFmt>(a, ks, vs, stream);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace

int32_t decode_q8_auto_splits(int32_t batch, int32_t kv_heads, int32_t n_cap, int32_t block_size) {
  const int64_t groups = (int64_t)batch * kv_heads;
  const int64_t chunks = ((int64_t)n_cap * block_size + 31) / 32;
  int64_t s = (256 + groups - 1) / groups;
  const int64_t most = chunks / kDecodeWaves;
  if (s > most) s = most;
  if (s > 256) s = 256;
  if (s < 1) s = 1;
  return (int32_t)s;
}

hipError_t launch_decode_q8(const DecodeArgs& a, const float* k_scale, const float* v_scale, int32_t format,
                            hipStream_t stream) {
  return format == RESA_Q8_INT8 ? launch_fmt<RESA_Q8_INT8>(a, k_scale, v_scale, stream)
                                : launch_fmt<RESA_Q8_E4M3>(a, k_scale, v_scale, stream);
}

}  // namespace resa
