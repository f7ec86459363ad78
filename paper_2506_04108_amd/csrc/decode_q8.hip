// Block-sparse flash-decoding (Eq. 2; App. A, Alg. 2) over an 8-bit cache, on
// the matrix cores.
//
// As in the bf16 decode, grid (num_splits, kv_heads, batch), a split per
// workgroup of 4 waves, and the splits of a group are merged by log-sum-exp by
// the last of them to finish. A selected block is cut into 16-token halves and
// two halves in a row make a chunk of 32 tokens, the unit that is dealt to the
// splits and their waves. Converting the codes and multiplying them on the
// VALU would cost a multiply-add per code and query head (8 heads: 80 a clock
// and CU at 6 TB/s, more than a CU has), so both products are MFMAs.
//
// Codes go from HBM into a chunk's place a wave in LDS (8 KB, whole kilobytes a
// load and no registers); a wave reads what it needs of a chunk in the layouts of
// the MFMAs, and the next chunk is on its way while it works on this one. Lane
// (r, c), r = lane / 16, c = lane % 16. Per chunk:
//   S^T = K . Q^T   two halves x four v_mfma_f32_16x16x32_bf16 (tokens x
//                   columns): lane (r, c) takes dims 16 r .. + 16 and 64 + 16 r
//                   .. + 16 of token c; the contraction runs over the dims in
//                   that order. Column c is head c % 8: a group has at most 8
//                   heads, and each is there twice. Lane (r, c) receives tokens
//                   4 r .. + 4 of each half.
//   weights         p = 2^(S ks - m) in fp32, ks the block's key scale times the
//                   softmax scale; w = p vs, vs the block's value scale
//   O^T += V^T . w  eight v_mfma_f32_16x16x32_f16 (dims x columns): the tokens of
//                   lane (r, c) are the ones whose weights it holds, so nothing
//                   moves between lanes; it takes dims 8 c .. + 8 of them and
//                   transposes inside the lane, by the choice of the values
//                   that a packing instruction takes.
// Every code is a bf16 and an fp16 value. w is the sum of two fp16 terms (22
// bits, down to 2^-36 of the largest w met), columns 0 .. 7 holding the first
// terms of the 8 heads and columns 8 .. 15 the second; products are exact and
// sums fp32, so results have fp32's precision. The unit 2^-k of w belongs to a
// head: one that sees small values alone keeps their precision whatever the
// others see, and follows the reference: a value that had all the weight until a
// far higher score came does not hold it. Both move rarely (only then are the
// accumulators touched).
//
// Bound by HBM (256 B a token and kv head) and, with few chunks a wave, by the
// latency of a launch, the ids, the first codes and the merge. 64K batch 8 (108
// MB), 256K batch 1 (27 MB), 50K batch 6 paged (40 MB), 4K batch 1: 24.4, 13.3,
// 17.1, 8.5 us (HBM at a large copy's rate: 21, 5.3, 7.8, 0.4, at a large read's: 15,
// 3.8, 5.6, 0.3; with codes through registers, the loads in the MFMAs' layouts:
// 29.3, 15.6, 23.4, 9.0).
// More chunks on their way are slower (two: 26.0, 13.8, 18.0 us, three: 27.5, 15.5,
// 24.6), as in the bf16 decode, and so are 8 waves (25.6, 14.5, 16.9 us, 4K
// 10.0). Both products on int8 digits, with no code converted and half of the
// VALU work, but a longer code for every launch to fetch: 64K 34.4 against 29.3.
#include "decode_impl.h"
#include "rows_device.h"

namespace resa {
namespace {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8_t __attribute__((ext_vector_type(8)));
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));

constexpr int kDecodeWaves = 4;
// Chunks of a wave in LDS or on their way there, beside the one in registers.
constexpr int kRing = 1;
constexpr int kHalfBytes = 16 * kHeadDim;    // codes of 16 tokens
constexpr int kChunkBytes = 4 * kHalfBytes;  // K of two halves, V of two halves
constexpr int kChunkLoads = 8;               // loads of 1 KB

// Chunk lists are staged for this many halves at a time.
constexpr int kListed = 512;

// The ring's memory serves the merges at the end.
template <int G, int NW>
struct DecodeQ8Lds {
  union {
    __attribute__((aligned(1024))) uint8_t ring[NW][kRing][kChunkBytes];
    struct {
      __attribute__((aligned(16))) float racc[NW][G][kHeadDim];
      __attribute__((aligned(16))) float own_o[G * kHeadDim];
      __attribute__((aligned(16))) float w[kMaxSplits * G];
      f4_t red[64 * NW];
      float rm[G][NW], rl[G][NW];
      float own_l[G];
      uint32_t ticket;
    };
  };
  int tok[kListed];   // first token of each half, -1: none
  int row[kListed];
  float ks[kListed], vs[kListed];  // scales of its block (next to each other)
};

// w 2^k: the largest w of a head is made 2^kTop .. 2^(kTop + 1) and may grow to
// 2^kMost (fp16 ends below 2^16) before k changes.
constexpr int kTop = 11, kMost = 15;

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

// Four dims of the lane's eight tokens (words w[0 .. 7]), transposed: out[d]
// holds the eight tokens' values of dim d as fp16.
template <int kFmt>
__device__ __forceinline__ void transpose_f16(const uint32_t (&w)[8], f16x8_t (&out)[4]) {
  uint32_t o[4][4];
#pragma unroll
  for (int t = 0; t < 8; t += 2) {
    if constexpr (kFmt == RESA_Q8_INT8) {
      float x[4], y[4];
      codes_f32<kFmt>(w[t], x);
      codes_f32<kFmt>(w[t + 1], y);
#pragma unroll
      for (int d = 0; d < 4; ++d) o[d][t / 2] = pack_f16_exact(x[d], y[d]);
    } else {
      const uint32_t x0 = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w[t], 1.f, false));
      const uint32_t x1 = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w[t], 1.f, true));
      const uint32_t y0 = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w[t + 1], 1.f, false));
      const uint32_t y1 = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w[t + 1], 1.f, true));
      o[0][t / 2] = __builtin_amdgcn_perm(y0, x0, 0x05040100u);
      o[1][t / 2] = __builtin_amdgcn_perm(y0, x0, 0x07060302u);
      o[2][t / 2] = __builtin_amdgcn_perm(y1, x1, 0x05040100u);
      o[3][t / 2] = __builtin_amdgcn_perm(y1, x1, 0x07060302u);
    }
  }
#pragma unroll
  for (int d = 0; d < 4; ++d) out[d] = __builtin_bit_cast(f16x8_t, U4{o[d][0], o[d][1], o[d][2], o[d][3]});
}

__device__ __forceinline__ f32x4_t mfma16(bf16x8_t a, bf16x8_t b, f32x4_t c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

template <int G, int BS, int kFmt, int NW>
__device__ __forceinline__ void decode_split_q8(const DecodeArgs& a, const float* k_scale, const float* v_scale, int bb,
                                                int hk, int split, DecodeQ8Lds<G, NW>& lds) {
  constexpr int HPB = BS / 16;  // halves per block
  constexpr int kLog2 = BS == 16 ? 4 : BS == 32 ? 5 : 6;
  constexpr int NT = 64 * NW;
  constexpr int kPer = kListed / NT;
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
    const int lim = min(slots, hb + kListed) - hb;
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
  // Scales from the group's (paged: the pool's) first block on.
  const size_t sbase = paged ? 0 : grp * a.c.max_blocks;
  const int sbytes = 4 * (paged ? a.c.num_pages * a.c.kv_heads : a.c.max_blocks);
  const i32x4_t rks = rsrc_words(k_scale + sbase, sbytes), rvs = rsrc_words(v_scale + sbase, sbytes);
  const float scale = a.scale_log2;
  const float ninf = -__builtin_inff();
  const int n_raw = __hip_atomic_load(a.num_sel + grp, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  const int L = __hip_atomic_load(a.seq_lens + bb, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  uint32_t epoch = __hip_atomic_load(a.epochs + grp, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  const int M = min((L + BS - 1) / BS, a.c.max_blocks);
  const int n = max(0, min(n_raw, a.n_cap));
  const int halves = n * HPB;
  const int valid = 2 * count_below((halves + 1) / 2);  // this split's halves

  // A half's codes of K and of V into LDS: 16-byte piece p of row t sits in
  // slot p ^ (t / 2) of K's rows, so that the reads below (one piece of 16
  // rows) meet every bank once, and in slot p of V's (whole rows).
  const uint32_t ring = __builtin_amdgcn_readfirstlane(lds_addr(lds.ring[wave]));
  const int lrow = lane >> 3, lslot = lane & 7;
  const uint32_t k_off = lrow * kHeadDim + 16 * (lslot ^ (lrow >> 1));
  const uint32_t k_off8 = (8 + lrow) * kHeadDim + 16 * (lslot ^ (4 + (lrow >> 1)));
  const uint32_t v_off = 16 * lane;
  // With `there` false nothing is fetched (zeros arrive), so that the number of
  // loads on their way is always the same.
  auto load_chunk = [&](int slot, int row0, int row1, bool there) __attribute__((always_inline)) {
    const uint32_t to = ring + slot * kChunkBytes;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const size_t base = (size_t)(h == 0 ? row0 : row1) * kHeadDim;
      lds_load_rows8<true>(to + h * kHalfBytes, k_off, k_off8, rsrc_words(kp + base, there ? kHalfBytes : 0));
      lds_load_rows8<true>(to + (2 + h) * kHalfBytes, v_off, v_off + 1024, rsrc_words(vp + base, there ? kHalfBytes : 0));
    }
  };

  // Head c % 8: softmax reference m and unit 2^-k of w (the same in the four
  // lanes of a column and in columns c and c ^ 8), and this lane's share l of
  // the sum of the weights.
  float m = ninf, l = 0.f;
  int k = 0;
  float most = 0.f;  // the w that k was last made for, under today's reference
  f32x4_t o[8];      // in units of 2^-k
#pragma unroll
  for (int d = 0; d < 8; ++d) o[d] = f32x4_t{0.f, 0.f, 0.f, 0.f};

  typedef __attribute__((address_space(3))) const u32x4_t lds_u32x4;
  typedef __attribute__((address_space(3))) const u32x2_t lds_u32x2;
  auto consume = [&](const u32x4_t (&kk)[2][2], u32x2_t (&vv)[8], int t0, int t1, float ks0, float ks1, float vs0,
                     float vs1) __attribute__((always_inline)) {
    float x[8], vs[2] = {vs0, vs1};
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      // A scale of the block that is not finite makes its scores NaN.
      const float kscaled = (finite_f(vs[h]) && finite_f(h == 0 ? ks0 : ks1) ? (h == 0 ? ks0 : ks1) : __builtin_nanf("")) * scale;
      f32x4_t s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        s = mfma16(codes_bf16<kFmt>(kk[h][e][0], kk[h][e][1]), q[2 * e], s);
        s = mfma16(codes_bf16<kFmt>(kk[h][e][2], kk[h][e][3]), q[2 * e + 1], s);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        // Rounded here, as the reference that is taken of it (a product
        // contracted with the subtraction below could exceed it by far).
        x[4 * h + i] = s[i] * kscaled;
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
          vv[j] = u32x2_t{0u, 0u};
        }
      }
      if (t0 < 0) vs[0] = 0.f;
      if (t1 < 0) vs[1] = 0.f;
    }
    const float cm = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
    // The reference moves only when a score exceeds it by more than
    // kRefSlack, so the reduction over the column and the rescale are rare.
    const bool moves = __any(cm > m + kRefSlack);
    if (moves) {
      const float alpha = move_ref(m, max_xor32(max_xor16(cm)));
      l *= alpha;
      most *= alpha;
#pragma unroll
      for (int d = 0; d < 8; ++d) o[d] *= alpha;
    }
    const float mref = m == ninf ? 0.f : m;
    float p[8], w[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) p[j] = fast_exp2(x[j] - mref);
    l += ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
    const float f[2] = {__builtin_ldexpf(vs[0], k), __builtin_ldexpf(vs[1], k)};
    float wm = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      w[j] = p[j] * f[j >> 2];
      wm = fmaxf(wm, w[j]);
    }
    // The unit is made anew where a w outgrows it, and where the reference has
    // moved: what the head summed up so far has shrunk beside the weights to come.
    // A scale that is past fp32 in it comes here too.
    if (moves || __any(!(most > 0.f) || wm >= (float)(1 << kMost) || !(f[0] + f[1] < __builtin_inff()))) {
      float y = 0.f;
#pragma unroll
      for (int j = 0; j < 8; ++j) y = fmaxf(y, p[j] * vs[j >> 2]);
      most = fmaxf(most, max_xor32(max_xor16(y)));
      const int to = most > 0.f ? kTop + 127 - (int)((__float_as_uint(most) >> 23) & 0xffu) : k;
#pragma unroll
      for (int d = 0; d < 8; ++d)
#pragma unroll
        for (int i = 0; i < 4; ++i) o[d][i] = __builtin_ldexpf(o[d][i], to - k);
      k = to;
#pragma unroll
      for (int j = 0; j < 8; ++j) w[j] = __builtin_ldexpf(p[j] * vs[j >> 2], k);
    }
    f16x8_t ph;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const _Float16 first = (_Float16)w[j];
      ph[j] = c < 8 ? first : (_Float16)(w[j] - (float)first);
    }
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      uint32_t words[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) words[j] = vv[j][e];
      f16x8_t vt[4];
      transpose_f16<kFmt>(words, vt);
#pragma unroll
      for (int d = 0; d < 4; ++d)
        o[4 * e + d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vt[d], ph, o[4 * e + d], 0, 0, 0);
    }
  };

  int hb = 0;
  do {
    if (hb > 0) load_ids(hb);
    const int he = min(valid, hb + kListed);
    const int lim = min(slots, hb + kListed) - hb;
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
    // Scales straight into their lists (lane i's lands at 4 i), in front of the
    // codes.
    const uint32_t list = __builtin_amdgcn_readfirstlane(lds_addr(lds.ks)) + 4 * 64 * wave;
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      if (j * NT < lim) {
        const uint32_t at = 4 * (tk[j] < 0 ? 0 : rw[j] >> kLog2);
        lds_load_dword(list + 4 * j * NT, at, rks);
        lds_load_dword(list + 4 * (j * NT + kListed), at, rvs);
      }
    }
    lds_sync();
    // Chunk cc of the pass: halves 2 cc and 2 cc + 1. Wave w takes chunks w,
    // w + NW, ...
    const int chunks = (he - hb) / 2;
    auto ask = [&](int slot, int cc) __attribute__((always_inline)) {
      const bool there = cc < chunks;
      const int at = there ? 2 * cc : 0;
      load_chunk(slot, __builtin_amdgcn_readfirstlane(lds.row[at]), __builtin_amdgcn_readfirstlane(lds.row[at + 1]), there);
    };
#pragma unroll
    for (int i = 0; i < kRing; ++i) ask(i, wave + i * NW);
    __builtin_amdgcn_s_waitcnt(wait_vm(kChunkLoads * kRing));
    lds_sync();
    int slot = 0;
#pragma unroll 1
    for (int cc = wave; cc < chunks; cc += NW) {
      const int t0 = __builtin_amdgcn_readfirstlane(lds.tok[2 * cc]), t1 = __builtin_amdgcn_readfirstlane(lds.tok[2 * cc + 1]);
      const float ks0 = lds.ks[2 * cc], ks1 = lds.ks[2 * cc + 1], vs0 = lds.vs[2 * cc], vs1 = lds.vs[2 * cc + 1];
      __builtin_amdgcn_s_waitcnt(wait_vm(kChunkLoads * (kRing - 1)));
      compiler_fence();
      const uint32_t at = ring + slot * kChunkBytes;
      u32x4_t kk[2][2];
      u32x2_t vv[8];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int e = 0; e < 2; ++e)
          kk[h][e] = *(lds_u32x4*)(uintptr_t)(at + h * kHalfBytes + c * kHeadDim + 16 * ((4 * e + r) ^ (c >> 1)));
#pragma unroll
        for (int j = 0; j < 4; ++j)
          vv[4 * h + j] = *(lds_u32x2*)(uintptr_t)(at + (2 + h) * kHalfBytes + (4 * r + j) * kHeadDim + 8 * c);
      }
      __builtin_amdgcn_s_waitcnt(kWaitLgkm0);  // read before the slot is filled again
      compiler_fence();
      ask(slot, cc + kRing * NW);
      consume(kk, vv, t0, t1, ks0, ks1, vs0, vs1);
      slot = slot + 1 == kRing ? 0 : slot + 1;
    }
    __builtin_amdgcn_s_waitcnt(kWaitVmcnt0);
    lds_sync();
    hb += kListed;
  } while (hb < valid);

  __builtin_amdgcn_s_waitcnt(kWaitVmcnt0);
  uint32_t ticket = 0;
  if (S > 1 && tid == 0)
    ticket = __hip_atomic_fetch_add(a.counters + grp, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);

  // The wave's state to LDS: the terms' products are added (columns c and
  // c ^ 8), dims 8 (4 r + i) + d.
  const float lt = sum_xor32(sum_xor16(l));
#pragma unroll
  for (int d = 0; d < 8; ++d)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float y = __builtin_ldexpf(o[d][i], -k);
      o[d][i] = y + dpp<kDppRor8>(y);
    }
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
__global__ __launch_bounds__(64 * kDecodeWaves) __attribute__((amdgpu_waves_per_eu(2, 2))) void k_decode_q8(
    DecodeArgs a, const float* k_scale, const float* v_scale) {
  __shared__ DecodeQ8Lds<G, kDecodeWaves> lds;
  decode_split_q8<G, BS, kFmt, kDecodeWaves>(a, k_scale, v_scale, blockIdx.z, blockIdx.y, blockIdx.x, lds);
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
  // At most a workgroup per CU (6 sequences of 50K, 48 groups: 18.0 us with 5
  // splits, 18.1 with 6, 22.8 with 12), with a chunk per wave at least.
  const int64_t groups = (int64_t)batch * kv_heads;
  const int64_t chunks = ((int64_t)n_cap * block_size + 31) / 32;
  int64_t s = 256 / groups;
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
