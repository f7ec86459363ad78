// Dense causal attention of packed query rows on gfx950 matrix cores: whole
// prompts of different lengths over their own keys (bf16), and the last rows
// of each sequence over an 8-bit cache (rectification, chunked prefill).
//
// Row rho = r * g + h of a (sequence, kv head) group is head h of the
// sequence's packed row r, at position L - n + r; it sees keys up to there. A
// workgroup takes 64, 128 or 256 consecutive rows (a query block) and one split
// of the keys, each wave 32 rows, and walks the keys 64 at a time (a tile):
//   S^T = K . Q^T     v_mfma_f32_32x32x16_bf16 (keys x queries): lane l holds
//                     query l % 32 and keys 8 (i / 4) + 4 (l / 32) + i % 4,
//                     i = 0 .. 15, of each 32
//   weights           2^(S c - m), fp32; their sum is of the fp32 values
//   O^T += V^T . P^T  v_mfma_f32_32x32x16_bf16 (dims x queries), with the
//                     contraction in the order in which the lanes hold the
//                     weights; V^T through the LDS transpose read
// The weights enter the second product as bf16 (8 significant bits, error at
// most 2^-8 each, independent from key to key): the result is rounded to bf16
// itself, and with bf16 operands no V is out of range and V needs no
// conversion, so that K and V rows go from HBM straight into LDS. (With fp16
// weights, V converted on its way and a second pass for what fp16 cannot hold,
// the bf16 cache's rectification runs at 1.02 - 1.16 PFLOP/s.)
//
// A tile's weights are formed while the matrix cores produce the scores of the
// next one (two MFMAs, then the VALU work of a few weights, kept in that order
// by scheduling barriers), then its P.V runs. One barrier a tile, or two. The
// softmax reference is the maximum of the first tile and moves only when the
// weights of a tile sum to more than 2^12 over a lane's keys, so that no tile
// needs its maximum beforehand.
//
// The query blocks are dealt long ones first (every workgroup finds its own by
// a search over the sequences' counts, in one wave's registers), with the kv
// heads of a block next to each other: workgroups go to the 8 XCDs in turn,
// so that with 8 kv heads the blocks of one head share an L2.
//
// 8-bit cache: every code is a bf16 and an fp16 value, so both products are on
// the codes themselves; a block's key scale multiplies the score (inside the fma
// of the weight) and its value scale, over a power of two that all keys share, the
// weight, which is fp16 here (2^-11: the result's own rounding is the larger by
// far). Where the value scales of a split lie more than 2^6 apart, the product of
// each 16 keys is taken by itself, so that a row of small values keeps its bits:
// 8 x 64K 363 -> 548 us, 2033 rows behind 31K 1410 -> 2655. The codes go from HBM into LDS,
// a round later through registers, converted under P.V's MFMAs, into the tiles.
// 8 x 64K, 32 rows of 4 heads each: 402 -> 370 us a call against codes and
// scales held in registers on their way (whose copies from one register to
// another waited for the loads). There the matrix cores are busy 40 % of the
// cycles, the VALU 55 % and the LDS 61 %, at 1.9 GHz; the conversion costs less than
// that suggests: int8, 6 instructions for four codes, 367 us, e4m3, 2, 351. One long
// prompt: matrix cores 61 %, VALU 51 %, LDS 46 %, at 1.8 GHz of 2.4.
//
// Measured: one prompt of 16384 tokens, 32 heads over 8: 1.88 - 1.90 ms, 1.16 - 1.17
// PFLOP/s; 16 prompts of 77 to 2000 tokens, 28 heads over 4: 211 us called again and
// again, 226 - 231 with other inputs each time, 0.72 - 0.79 PFLOP/s; one of 300 tokens 10.0
// us, a chain of latencies. 32 rows of 4 heads behind 8 x 64K codes: 364 - 372 us with
// the stores and the merge, 2.9 - 3.0 TB/s; 2033 rows of 7 behind 31K: 1.41 - 1.43 ms, 0.98
// PFLOP/s (int8 1.45).
//
// Masked keys: scores are replaced, so nothing of a masked K row matters; a
// masked V row meets weights of zero, which only a value that is not finite
// would survive. The tiles that some row of the workgroup masks are searched
// for such values, and a workgroup that finds one takes its range again, a
// tile at a time, with these values apart.
#include <algorithm>
#include <type_traits>

#include "rows_device.h"

namespace resa {
namespace {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8_t __attribute__((ext_vector_type(8)));
typedef short i16x4_t __attribute__((ext_vector_type(4)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));

constexpr int kRowsPerWave = 32;
constexpr int kKT = 64;                    // keys per tile
constexpr int kKT32 = kKT / 32, kKT16 = kKT / 16;
constexpr int kRowBytes = kHeadDim * 2;
constexpr int kCus = 256;
constexpr int kClassKeys = 1024;          // query blocks: a class of costs
constexpr int kShortPrompt = 2560;         // tokens of a prompt on average, that are few
constexpr int64_t kLongSplit = 1024;      // keys of a split that is long
constexpr float kMaxWeightSum = 4096.f;
constexpr int kUnitRange = 7;             // value scales (log2) that share a unit
constexpr int kPacked = -1;                // source of keys: packed bf16 rows, else the format of the 8-bit cache

// Rows of a tile are 256 B; 16-byte piece p of row r sits in slot p ^ swz(r),
// which keeps both the K reads (16 rows, one piece) and the V transpose reads
// (4 aligned rows, four neighbouring pieces) free of bank conflicts.
__host__ __device__ constexpr int swz(int r) { return ((r & 3) << 2) | ((r >> 2) & 3); }

// Rows of a workgroup (64, 128 or 256) and its waves.
__host__ __device__ constexpr int waves_of(int rows) { return rows == 256 ? 8 : 4; }

constexpr int kWaitVm0 = kWaitVmcnt0;

// 1 or 2 KB of codes likewise.
template <int kUnits>
__device__ __forceinline__ void lds_load_codes(uint32_t lds, uint32_t voff, i32x4_t rk) {
  if constexpr (kUnits == 2) {
    lds_load_rows8(lds, voff, voff + 1024, rk);
  } else {
    uint32_t saved;
    __asm__ volatile(
        "s_mov_b32 %0, m0\n\t"
        "s_mov_b32 m0, %1\n\ts_nop 0\n\tbuffer_load_dwordx4 %2, %3, 0 offen lds\n\t"
        "s_mov_b32 m0, %0"
        : "=&s"(saved) : "s"(lds), "v"(voff), "s"(rk) : "memory");
  }
}
__device__ __forceinline__ void bare_barrier() {
  compiler_fence();
  __builtin_amdgcn_s_barrier();
  compiler_fence();
}
__device__ __forceinline__ f32x16_t mfma32(bf16x8_t a, bf16x8_t b, f32x16_t c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x16_t mfma32(f16x8_t a, f16x8_t b, f32x16_t c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}
// x - y, the product x rounded first (never contracted to one operation).
__device__ __forceinline__ float sub_rounded(float x, float y) {
  __asm__ volatile("" : "+v"(x));
  return x - y;
}
// Whether one of the two bf16 values of a word is infinite or NaN.
__device__ __forceinline__ bool not_finite2(uint32_t w) {
  return (w & 0x7f80u) == 0x7f80u || (w & 0x7f800000u) == 0x7f800000u;
}
__device__ __forceinline__ uint32_t finite_or_0(uint32_t w) {
  return ((w & 0x7f80u) == 0x7f80u ? 0u : w & 0xffffu) | ((w & 0x7f800000u) == 0x7f800000u ? 0u : w & 0xffff0000u);
}

// Rows of a sequence as a launch sees them: n rows from packed row `first` on,
// the last of L keys; n = 0 where the call leaves the sequence out.
struct SeqRows {
  int first, n, L;
};
template <int kSrc>
__device__ __forceinline__ SeqRows seq_rows(const RowsArgs& a, int s) {
  SeqRows q;
  packed_rows(a.cu, a.rows, s, q.first, q.n);
  q.L = kSrc == kPacked ? q.n : a.seq_lens[s];
  if (kSrc != kPacked && (q.L < q.n || q.L > a.c.capacity)) q.n = 0;
  return q;
}

// Query block `item`, the longest first. A block's cost is its last row's
// position in units of a block's rows: block b of a sequence with h rows' worth
// of earlier keys costs h + b + 1. The blocks are dealt by classes of cost, of
// kClassKeys keys each, from the highest down, those of a class sequence by
// sequence: workgroups that run together then share the keys of a sequence, in
// the L2, and the last ones are short all the same. Against strictly falling
// costs, all by 256 rows: 16 prompts of up to 2000 tokens, 28 heads over 4, 224 -> 214
// us; 64 of up to 700, 32 over 8, 233 -> 202; 30 of 1000, 8 over 8, whose last class is a
// larger part of the whole, 63.5 -> 67.8. (Blocks of different costs next to each other: 16 prompts 259
// and more.) The first 64 sequences' counts stay in registers, so that up to
// there the search reads memory once.
template <int kSrc, int kPer>
__device__ __forceinline__ bool find_block(const RowsArgs& a, int item, SeqRows& sr, int& seq, int& qblk) {
  const int lane = threadIdx.x & 63;
  const int per = max(kClassKeys * a.group / kPer, 1);  // costs of a class: x per + 1 .. (x + 1) per
  auto earlier = [&](const SeqRows& q) -> int {
    return kSrc == kPacked ? 0 : (int)((int64_t)(q.L - q.n) * a.group / kPer);
  };
  auto blocks = [&](const SeqRows& q) -> int { return (int)(((int64_t)q.n * a.group + kPer - 1) / kPer); };
  auto rows_at = [&](int s) -> SeqRows { return s < a.batch ? seq_rows<kSrc>(a, s) : SeqRows{0, 0, 0}; };
  const SeqRows q0 = rows_at(lane);
  const int h0 = earlier(q0), nb0 = blocks(q0);
  int x = 0, rank = item;
  seq = 0;
  if (a.batch == 1) {
    if (__builtin_amdgcn_readlane(nb0, 0) <= item) return false;
  } else {
    auto of = [&](int h, int nb, int x) -> int { return min(max(h + nb - x * per, 0), nb); };
    auto at_least = [&](int x) -> int {  // blocks of class x and above
      int c = of(h0, nb0, x);
      for (int base = 64; base < a.batch; base += 64) {
        const SeqRows q = rows_at(base + lane);
        c += of(earlier(q), blocks(q), x);
      }
      return wave_total(c);
    };
    int most = nb0 == 0 ? 0 : h0 + nb0, least = nb0 == 0 ? INT32_MAX : h0;
    for (int base = 64; base < a.batch; base += 64) {
      const SeqRows q = rows_at(base + lane);
      const int h = earlier(q), nb = blocks(q);
      if (nb > 0) {
        most = max(most, h + nb);
        least = min(least, h);
      }
    }
    most = (int)wave_max((uint32_t)most);
    if (most == 0) return false;
    x = (int)~wave_max(~(uint32_t)least) / per;
    if (at_least(x) <= item) return false;
    int hi = (most - 1) / per + 1;  // more than `item` blocks of class x and above, not of class hi
    while (hi - x > 1) {
      const int mid = (x + hi) >> 1;
      if (at_least(mid) > item) x = mid;
      else hi = mid;
    }
    auto of_class = [&](int s) -> int {
      const SeqRows q = s < 64 ? q0 : rows_at(s);
      const int h = earlier(q), nb = blocks(q);
      return of(h, nb, x) - of(h, nb, x + 1);
    };
    if (!find_seq(item - at_least(x + 1), a.batch, of_class, seq, rank)) return false;
  }
  sr = seq < 64 ? SeqRows{__builtin_amdgcn_readlane(q0.first, seq & 63), __builtin_amdgcn_readlane(q0.n, seq & 63),
                          __builtin_amdgcn_readlane(q0.L, seq & 63)}
                : seq_rows<kSrc>(a, seq);
  const int h = earlier(sr), last = h + blocks(sr);
  qblk = (a.batch == 1 ? last : min(last, (x + 1) * per)) - rank - h - 1;
  return true;
}

// Keys of a split. Of one length every sequence would take a.chunk; where the
// lengths differ, the longer ones are cut further, as long as all workgroups run
// at once (a.places), into at most a.num_splits: sum of blocks (tiles / t + 1) <=
// places for t = tiles / (places - blocks). 6 sequences of up to 36K, 93 rows of 12
// heads over 2: 165 -> 130 us; 8 of 8K, 100 rows of 32 over 8, for which nothing
// changes but the search, 172 -> 177. `q0` and `nb0` are this lane's sequence
// and its blocks.
template <int kSrc>
__device__ __forceinline__ int split_chunk(const RowsArgs& a, const SeqRows& q0, int nb0) {
  if (a.batch == 1) return a.chunk;
  const int lane = threadIdx.x & 63, shift = __builtin_ctz(a.per);
  int tiles = nb0 * ((q0.L + kKT - 1) / kKT), blocks = nb0, longest = nb0 == 0 ? 0 : q0.L;
  if (nb0 == 0) tiles = 0;
  for (int base = 64; base < a.batch; base += 64) {
    if (base + lane >= a.batch) continue;
    const SeqRows q = seq_rows<kSrc>(a, base + lane);
    const int nb = (q.n * a.group + a.per - 1) >> shift;
    if (nb == 0) continue;
    tiles += nb * ((q.L + kKT - 1) / kKT);
    blocks += nb;
    longest = max(longest, q.L);
  }
  const int free = a.places / a.kv_heads - wave_total(blocks);
  if (free <= 0) return a.chunk;
  const int most = (int)wave_max((uint32_t)longest), sum = wave_total(tiles);
  const int t = max(max((sum + free - 1) / free, (most + kKT * a.num_splits - 1) / (kKT * a.num_splits)), 2);
  return min(a.chunk, t * kKT);
}
template <int kSrc>
__device__ __forceinline__ int splits_of(const RowsArgs& a, int L, int chunk) {
  return min((L + chunk - 1) / chunk, a.num_splits);
}

// Query block and split `item`, sequence by sequence (all splits are about as
// long).
template <int kSrc, int kPer>
__device__ __forceinline__ bool find_split(const RowsArgs& a, int item, SeqRows& sr, int& seq, int& qblk, int& split,
                                           int& chunk) {
  const int lane = threadIdx.x & 63;
  auto rows_at = [&](int s) -> SeqRows { return s < a.batch ? seq_rows<kSrc>(a, s) : SeqRows{0, 0, 0}; };
  auto blocks = [&](const SeqRows& q) -> int { return (q.n * a.group + kPer - 1) / kPer; };
  const SeqRows q0 = rows_at(lane);
  chunk = split_chunk<kSrc>(a, q0, blocks(q0));
  auto count = [&](int s) -> int {
    const SeqRows q = s < 64 ? q0 : rows_at(s);
    const int nb = blocks(q);
    return nb == 0 ? 0 : nb * splits_of<kSrc>(a, q.L, chunk);
  };
  int rank;
  if (!find_seq(item, a.batch, count, seq, rank)) return false;
  sr = seq < 64 ? SeqRows{__builtin_amdgcn_readlane(q0.first, seq & 63), __builtin_amdgcn_readlane(q0.n, seq & 63),
                          __builtin_amdgcn_readlane(q0.L, seq & 63)}
                : seq_rows<kSrc>(a, seq);
  const int S = splits_of<kSrc>(a, sr.L, chunk);
  qblk = rank / S;
  split = rank - qblk * S;
  return true;
}

// LDS of a workgroup: K and V tiles of 16-bit values, tile t in stage t %
// kStages; for an 8-bit cache also the codes of a K and of a V tile on their way
// (each wave's rows in turn; 80 KB with two stages, so that two workgroups fit a
// CU, 144 with four), for packed rows a flag.
template <int kStages, bool kQ8>
struct RowsLds {
  uint8_t k[kStages][kKT * kRowBytes];
  uint8_t v[kStages][kKT * kRowBytes];
  int odd;  // a masked tile holds a V value that is not finite
};
template <int kStages>
struct RowsLds<kStages, true> {
  uint8_t k[kStages][kKT * kRowBytes];
  uint8_t v[kStages][kKT * kRowBytes];
  uint8_t raw[2][kKT * kHeadDim];
};

// A workgroup of kRows rows: 256 and 128 in 8 and 4 waves; 64 in 4 waves, of
// which two share 32 rows, each with its half of every tile's keys, and are
// merged at the end (few rows: a tile takes a wave half as long). With four
// stages of K and V one workgroup fits a CU, with two stages and four waves two
// do. A barrier every kBar tiles, half the stages (2033 rows over 8-bit pages:
// 1454 us with two stages, 1392 with four).
template <int kRows, int kSrc, bool kPaged>
__global__ __launch_bounds__(kRows == 256 ? 512 : 256) __attribute__((amdgpu_waves_per_eu(2, 2)))
void k_rows_attn(RowsArgs a) {
  constexpr bool kQ8 = kSrc != kPacked;
  constexpr int kWaves = waves_of(kRows);
  constexpr bool kHalves = kRows == 64;
  // Keys of a tile that a wave takes, in 32s and 16s.
  constexpr int kMine32 = kHalves ? kKT32 / 2 : kKT32, kMine16 = 2 * kMine32;
  constexpr int kStages = kRows == 256 ? 4 : 2;
  // Weights and V: bf16, or over codes fp16.
  typedef std::conditional_t<kQ8, _Float16, __bf16> Weight;
  typedef std::conditional_t<kQ8, f16x8_t, bf16x8_t> P8;
  constexpr int kBar = kStages / 2;
  constexpr int kLoadRows = kKT / kWaves;  // tile rows whose K and V each wave brings in
  constexpr int kUnits = kLoadRows / 8;
  constexpr int kTileBytes = kKT * kRowBytes;
  typedef RowsLds<kStages, kQ8> Lds;
  __shared__ __attribute__((aligned(1024))) Lds lds;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int rwave = kHalves ? wave & 1 : wave, half = kHalves ? wave >> 1 : 0;
  const int S = a.num_splits, G = a.group;
  const int hk = blockIdx.x % a.kv_heads, item = blockIdx.x / a.kv_heads;
  int seq, qblk, split = 0, chunk = a.chunk;
  SeqRows sr;
  if (kQ8 && S > 1) {
    if (!find_split<kSrc, kRows>(a, item, sr, seq, qblk, split, chunk)) return;
  } else if (!find_block<kSrc, kRows>(a, item, sr, seq, qblk)) {
    return;
  }
  if constexpr (!kQ8) {
    if (tid == 0) lds.odd = 0;
  }
  const int R = sr.n * G, past = sr.L - sr.n;
  const int k0 = split * chunk;
  const int last_row = min(R - 1, (qblk + 1) * kRows - 1);
  const int k1 = min(min(k0 + chunk, sr.L), past + last_row / G + 1);
  if (k1 <= k0) return;  // no key of this split is seen: the merge does not read it
  const int ntiles = (k1 - k0 + kKT - 1) / kKT;
  const float ninf = -__builtin_inff();
  // Softmax scale: a negative one negates the queries, zero clears them.
  const float c = a.scale_log2 == 0.f ? 1.f : fabsf(a.scale_log2);
  const uint32_t q_and = a.scale_log2 == 0.f ? 0u : ~0u, q_xor = a.scale_log2 < 0.f ? 0x80008000u : 0u;
  const int hi = lane >> 5, lq = lane & 31;
  const int row_base = qblk * kRows + rwave * kRowsPerWave;
  const int rho = row_base + lq;
  // Keys past lim are masked. Rows past the last one follow it (their queries
  // are zero and nothing of theirs is stored).
  const int lim = min(past + min(rho, R - 1) / G, k1 - 1);
  // Tiles that reach past `cut` (of the wave) or `wg_cut` (of any wave) mask
  // something.
  const int cut = min(k1, past + min(row_base, R - 1) / G);
  const int wg_cut = past + qblk * kRows / G;

  // Packed rows straight into LDS: lane i fills slot i % 16 of rows i / 16 and
  // + 4 of each eight, fetching the row's piece (i % 16) ^ swz(row).
  const int wrow = kLoadRows * wave;
  const int lrow = lane >> 4, lslot = lane & 15;
  uint32_t koff[kUnits][2], voff[kUnits][2];
#pragma unroll
  for (int u = 0; u < kUnits; ++u)
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const uint32_t piece = 16 * (lslot ^ swz(wrow + 8 * u + 4 * e + lrow));
      koff[u][e] = (uint32_t)(8 * u + 4 * e + lrow) * (uint32_t)(2 * a.k_stride) + piece;
      voff[u][e] = (uint32_t)(8 * u + 4 * e + lrow) * (uint32_t)(2 * a.v_stride) + piece;
    }
  const uint32_t lds0 = lds_addr(&lds);
  const uint32_t lds_k = __builtin_amdgcn_readfirstlane(lds0) + (uint32_t)(wrow * kRowBytes);
  // LDS read addresses (stage, 32-key part and k-step of P.V are immediates).
  // K: row lq, piece (2 ks + hi) ^ swz(lq). V^T by transpose reads, lane c of
  // 16 passing the address of key c / 4, dims 4 (c % 4) .. ; eight rows further
  // the slots differ in bit 1. The pieces of k-step ks and of dims 32 dt are an
  // exclusive or with 32 ks and 64 dt, taken once a round: held in registers
  // they make the kernels spill.
  uint32_t kbase = lds0 + (32 * half + lq) * kRowBytes + 16 * (hi ^ swz(lq));
  uint32_t vbase;
  {
    const int vr = 4 * hi + ((lane & 15) >> 2);
    const int vpiece = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
    vbase = lds0 + (uint32_t)offsetof(Lds, v) + (32 * half + vr) * kRowBytes + 16 * (vpiece ^ swz(vr)) + 8 * (lane & 1);
  }
  auto fresh = [](uint32_t& x) __attribute__((always_inline)) { __asm__ volatile("" : "+v"(x)); };
  typedef __attribute__((address_space(3))) const bf16x8_t lds_bf16x8;
  typedef __attribute__((address_space(3))) i16x4_t lds_i16x4;
  typedef __attribute__((address_space(3))) const u32x4_t lds_u32x4;
  auto read_k = [&](int st, int ks, bf16x8_t (&ka)[kMine32]) __attribute__((always_inline)) {
#pragma unroll
    for (int kt = 0; kt < kMine32; ++kt)
      ka[kt] = *(lds_bf16x8*)(uintptr_t)((kbase ^ (32 * ks)) + st * kTileBytes + kt * 32 * kRowBytes);
  };
  auto read_v32 = [&](int st, int ks, int dt) __attribute__((always_inline)) -> P8 {
    i16x4_t x[2];
#pragma unroll
    for (int e = 0; e < 2; ++e)
      x[e] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
          (lds_i16x4*)(uintptr_t)((vbase ^ (64 * dt + 32 * e)) + 8 * e * kRowBytes + st * kTileBytes + 16 * ks * kRowBytes));
    return __builtin_bit_cast(P8, __builtin_shufflevector(x[0], x[1], 0, 1, 2, 3, 4, 5, 6, 7));
  };
  auto read_v = [&](int st, int ks, P8 (&va)[4]) __attribute__((always_inline)) {
#pragma unroll
    for (int dt = 0; dt < 4; ++dt) va[dt] = read_v32(st, ks, dt);
  };

  // Q^T (B of S^T): lane holds row lq, dims 16 s + 8 hi .. + 8 for k-step s.
  // Rows are read 128 B at a time, eight lanes a row, and change lanes by way of
  // LDS, a half of the dims after the other: 4 KB of the wave's own in stages
  // that nothing has been requested into yet. 16 prompts of up to 77 tokens:
  // 12.4 us with the rows read as the lanes hold them, 32 B each, 11.6 us so.
  bf16x8_t qb[8];
  U4 qx[2][4];
  const int qrow = lane >> 3;
  {
    // Row rel of the block's: a quotient of small numbers, exact in fp32.
    const int r0 = (qblk * kRows) / G, h0 = qblk * kRows - r0 * G;
    const float inv_g = 1.f / (float)G;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int rel = rwave * kRowsPerWave + 8 * j + qrow + h0;
      const int dr = (int)(((float)rel + 0.5f) * inv_g);
      const uint16_t* qp = a.q + (int64_t)(sr.first + min(r0 + dr, sr.n - 1)) * a.q_stride +
                           (hk * G + rel - dr * G) * kHeadDim + 8 * (lane & 7);
#pragma unroll
      for (int p = 0; p < 2; ++p) qx[p][j] = ld16(qp + 64 * p);
    }
  }
  auto exchange_q = [&]() __attribute__((always_inline)) {
    uint8_t* mine = (kQ8 ? lds.k[0] : lds.v[kStages / 2]) + wave * (kRowsPerWave * 128);
#pragma unroll
    for (int p = 0; p < 2; ++p) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int r = 8 * j + qrow;
        const U4 x = qx[p][j];
        st16(mine + r * 128 + 16 * ((lane & 7) ^ ((r >> 1) & 7)),
             row_base + r < R ? U4{(x.x & q_and) ^ q_xor, (x.y & q_and) ^ q_xor, (x.z & q_and) ^ q_xor, (x.w & q_and) ^ q_xor}
                              : U4{0, 0, 0, 0});
      }
#pragma unroll
      for (int s = 0; s < 4; ++s)
        qb[4 * p + s] = __builtin_bit_cast(bf16x8_t, ld16(mine + lq * 128 + 16 * ((2 * s + hi) ^ ((lq >> 1) & 7))));
    }
  };

  // This wave's rows of tile ti: how many exist below k1.
  auto rows_of = [&](int ti) __attribute__((always_inline)) -> int {
    return min(max(k1 - (k0 + ti * kKT + wrow), 0), kLoadRows);
  };
  // Packed keys: K and V of a tile, requested straight into their stages.
  auto issue_packed = [&](const uint16_t* p, int64_t stride, const uint32_t (&off)[kUnits][2], uint32_t to, int ti)
                          __attribute__((always_inline)) {
    const int have = rows_of(ti);
    const int nrec = have > 0 ? (have - 1) * (int)(2 * stride) + kRowBytes : 0;
    const i32x4_t rx = rsrc_words(p + (int64_t)(sr.first + k0 + ti * kKT + wrow) * stride + hk * kHeadDim, nrec);
#pragma unroll
    for (int u = 0; u < kUnits; ++u) lds_load_rows8(to + 8 * u * kRowBytes, off[u][0], off[u][1], rx);
  };
  auto issue_k = [&](int ti, int st) __attribute__((always_inline)) {
    issue_packed(a.k, a.k_stride, koff, lds_k + (uint32_t)(st * kTileBytes), ti);
  };
  auto issue_v = [&](int ti, int st) __attribute__((always_inline)) {
    issue_packed(a.v, a.v_stride, voff, lds_k + (uint32_t)(offsetof(Lds, v) + st * kTileBytes), ti);
  };
  // 8-bit cache. Lane i holds the page and the factors of block i of a window
  // of 64 blocks, which a wave takes with a lane read, with no load in the way;
  // the window moves by 32 blocks, the one after it on its way: the tile at hand
  // lies in its first half, and the blocks of the next four tiles (at most 20
  // further on) in it too. A block with a scale that is no finite number (it was made
  // of rows that held one) is `odd`: it has NaN for its keys, so whoever sees
  // it gets NaN, and for the others its V counts as zero.
  const int mb0 = kQ8 ? k0 >> a.c.log2_block : 0, mlast = kQ8 ? (k1 - 1) >> a.c.log2_block : 0;
  struct Window {
    int page;
    float kf, vf;
  };
  Window win, coming;
  int wbase = 0;      // the window's first block, from mb0 on
  uint64_t odd = 0;   // its odd blocks
  auto load_window = [&](int base) __attribute__((always_inline)) -> Window {
    Window w;
    const int m = min(mb0 + base + lane, mlast);
    int64_t si;
    w.page = 0;
    if constexpr (kPaged) {
      w.page = a.c.table[(size_t)seq * a.c.max_blocks + m];
      if ((unsigned)w.page >= (unsigned)a.c.num_pages) w.page = -1;
      si = (int64_t)max(w.page, 0) * a.kv_heads + hk;
    } else {
      si = ((int64_t)seq * a.kv_heads + hk) * a.c.max_blocks + m;
    }
    w.kf = a.k_scale[si];
    w.vf = a.v_scale[si];
    // A page outside the pool reads as zeros, whatever the page looked at
    // instead belongs to.
    if (kPaged && w.page < 0) {
      w.kf = 1.f;
      w.vf = 0.f;
    }
    return w;
  };
  auto take_window = [&](const Window& w) __attribute__((always_inline)) {
    const bool bad = !finite_f(w.kf) || !finite_f(w.vf);
    odd = __ballot(bad);
    win.page = w.page;
    // Never zero, so that a masked score stays -inf under it.
    win.kf = bad ? c : fmaxf(w.kf * c, 0x1p-126f);
    win.vf = bad ? 0.f : w.vf;
  };
  // Block of key k0 + key (key a multiple of 16) in the window.
  auto block_at = [&](int key) __attribute__((always_inline)) -> int { return (key >> a.c.log2_block) - wbase; };
  auto lane_f = [&](float x, int i) __attribute__((always_inline)) -> float {
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), i));
  };
  // The wave's codes of a tile (its rows lie in one block; 1 or 2 KB, 16 codes
  // of row lane / 8 (and + 8) a lane) into LDS at `to`.
  auto ask = [&](bool key, int ti, uint32_t to) __attribute__((always_inline)) {
    if constexpr (kQ8) {
      const int at = k0 + ti * kKT + wrow;
      int have = rows_of(ti);
      int64_t row;
      if constexpr (kPaged) {
        const int page = __builtin_amdgcn_readlane(win.page, block_at(ti * kKT + (wrow & ~15)));
        if (page < 0) have = 0;
        row = ((int64_t)max(page, 0) * a.kv_heads + hk) * a.c.block_size + (at & (a.c.block_size - 1));
      } else {
        row = ((int64_t)seq * a.kv_heads + hk) * a.c.capacity + at;
      }
      lds_load_codes<kUnits>(to, 16 * lane, rsrc_words(reinterpret_cast<const uint8_t*>(key ? a.c.k : a.c.v) +
                                                       row * kHeadDim, have * kHeadDim));
    }
  };
  const uint32_t raw_of_wave = (uint32_t)(wave * kUnits * 1024);
  auto raw_at = [&](bool key) __attribute__((always_inline)) -> uint32_t {
    if constexpr (kQ8)
      return __builtin_amdgcn_readfirstlane(lds0) + (uint32_t)offsetof(Lds, raw) + (key ? 0 : kKT * kHeadDim) + raw_of_wave;
    else
      return 0;
  };
  // Where this lane's codes go in a tile: pieces 2 (lane % 8) and + 1 of row
  // wrow + lane / 8 (and of row + 8, where slots differ in bit 1).
  const int put_row = wrow + (lane >> 3);
  const uint32_t put0 = put_row * kRowBytes + 16 * ((2 * (lane & 7)) ^ swz(put_row));
  const uint32_t put1 = put_row * kRowBytes + 16 * ((2 * (lane & 7) + 1) ^ swz(put_row));
  // Four codes as 16-bit values: of a key bf16, of a value fp16.
  auto convert = [&](bool key, uint32_t in, uint32_t (&h)[2]) __attribute__((always_inline)) {
    if constexpr (kSrc == RESA_Q8_INT8) {
      float y[4];
      codes_f32<kSrc>(in, y);
#pragma unroll
      for (int u = 0; u < 2; ++u)
        h[u] = key ? __builtin_amdgcn_perm(__float_as_uint(y[2 * u + 1]), __float_as_uint(y[2 * u]), 0x07060302u)
                   : pack_f16_exact(y[2 * u], y[2 * u + 1]);
    } else if (key) {
      h[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(in, 1.f, false));
      h[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(in, 1.f, true));
    } else {
      h[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(in, 1.f, false));
      h[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(in, 1.f, true));
    }
  };
  // The codes of this wave's rows of a tile, arrived in LDS at `from`.
  struct Codes {
    u32x4_t x[kUnits];
  };
  auto codes_at = [&](uint32_t from) __attribute__((always_inline)) -> Codes {
    Codes w;
#pragma unroll
    for (int q = 0; q < kUnits; ++q) w.x[q] = *(lds_u32x4*)(uintptr_t)(from + 16 * lane + 1024 * q);
    return w;
  };
  // Word w (0 .. 4 kUnits - 1) of them converted; every second one stores eight
  // values to stage st (four: those before).
  auto put_word = [&](bool key, const Codes& c8, int w, int st, uint32_t (&four)[2]) __attribute__((always_inline)) {
    uint32_t h[2];
    convert(key, c8.x[w / 4][w % 4], h);
    if (w % 2 == 0) {
      four[0] = h[0];
      four[1] = h[1];
    } else {
      uint8_t* tile = key ? lds.k[st] : lds.v[st];
      st16(tile + 8 * (w / 4) * kRowBytes + ((w % 4 == 1 ? put0 : put1) ^ (32 * (w / 4))), U4{four[0], four[1], h[0], h[1]});
    }
  };
  // Rows of tile ti of an odd block: NaN keys, zero values.
  auto put_odd = [&](bool key, int ti, int st) __attribute__((always_inline)) {
    if constexpr (kQ8) {
      if (__builtin_expect((odd >> block_at(ti * kKT + (wrow & ~15))) & 1, 0)) {
        uint8_t* tile = key ? lds.k[st] : lds.v[st];
        const uint32_t x = key ? 0x7fc07fc0u : 0u;
#pragma unroll
        for (int q = 0; q < kUnits; ++q) {
          st16(tile + 8 * q * kRowBytes + (put0 ^ (32 * q)), U4{x, x, x, x});
          st16(tile + 8 * q * kRowBytes + (put1 ^ (32 * q)), U4{x, x, x, x});
        }
      }
    }
  };
  auto put = [&](bool key, int ti, uint32_t from, int st) __attribute__((always_inline)) {
    if constexpr (kQ8) {
      compiler_fence();
      const Codes w = codes_at(from);
      uint32_t four[2];
#pragma unroll
      for (int i = 0; i < 4 * kUnits; ++i) put_word(key, w, i, st, four);
      put_odd(key, ti, st);
      compiler_fence();  // the codes have been read when the next are asked for
    }
  };

  f32x16_t o[4];
  auto clear_o = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int dt = 0; dt < 4; ++dt)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[dt][i] = 0.f;
  };
  clear_o();
  float m = ninf, l = 0.f;  // l: over this lane's keys; summed across the two halves at the end
  bool guard = false;       // second pass, V values that are not finite left out

  auto mask = [&](int t0, f32x16_t (&s)[kMine32]) __attribute__((always_inline)) {
    const int d = lim - t0 - 32 * half - 4 * hi;
#pragma unroll
    for (int kt = 0; kt < kMine32; ++kt)
#pragma unroll
      for (int i = 0; i < 16; ++i) s[kt][i] = 32 * kt + 8 * (i >> 2) + (i & 3) > d ? ninf : s[kt][i];
  };
  // Factors of a tile's scores and of its weights, for each 16 keys. Those of
  // the scores are read with the K they belong to, a round before their use.
  struct Factors {
    float x[kMine16];
  };
  auto key_factors = [&](int ti) __attribute__((always_inline)) -> Factors {
    Factors f;
#pragma unroll
    for (int i = 0; i < kMine16; ++i) f.x[i] = kQ8 ? lane_f(win.kf, block_at(ti * kKT + 32 * half + 16 * i)) : c;
    return f;
  };
  // fp16 weights carry the value scale over vref, a power of two above the
  // largest one of the split, which the accumulators are in units of. A row may
  // see none of that block, or give it no weight. So this is done only where all
  // scales lie within 2^kUnitRange of vref: a weight then is off by 2^-25
  // 2^kUnitRange at most, where the row's largest is 1 or more. Elsewhere (`apart`)
  // vref is 1 and the product of each block is taken by itself.
  uint32_t vref = 0x3f800000u;  // bits of it
  bool apart = false;
  // The bounds of the split's value scales, found by the waves together: each
  // looks at every kWaves-th 64 blocks and leaves what it finds in LDS that no
  // tile is put into before the second barrier. Blocks of values up to 2^-100
  // (zeros as a rule) and odd ones set no lower bound.
  constexpr uint32_t kNoScale = __builtin_bit_cast(uint32_t, kQ8Least / Q8<kQ8 ? kSrc : 0>::kMax) + 1;
  auto bounds_at = [&]() __attribute__((always_inline)) -> uint32_t* {
    return reinterpret_cast<uint32_t*>((kBar == 1 ? lds.v[kStages - 1] : lds.k[kStages - 1]) + kKT * kHeadDim);
  };
  auto look_at_scales = [&]() __attribute__((always_inline)) {
    if constexpr (kQ8) {
      uint32_t top = 0, low = 0;  // low: of the inverted bits
      auto look = [&](const Window& w) __attribute__((always_inline)) {
        const uint32_t x = __float_as_uint(w.vf);  // in the order of bit patterns: scales are not negative
        if (finite_f(w.vf) && finite_f(w.kf)) {
          top = max(top, x);
          low = max(low, x > kNoScale ? ~x : 0u);
        }
      };
#pragma unroll 4
      for (int base = 64 * wave; base <= mlast - mb0; base += 64 * kWaves) look(load_window(base));
      top = wave_max(top);
      low = wave_max(low);
      if (lane == 0) {
        bounds_at()[2 * wave] = top;
        bounds_at()[2 * wave + 1] = low;
      }
    }
  };
  auto take_bounds = [&]() __attribute__((always_inline)) {
    if constexpr (kQ8) {
      const uint2 mine = *reinterpret_cast<const uint2*>(bounds_at() + 2 * (lane & (kWaves - 1)));
      const uint32_t top = wave_max(mine.x), low = wave_max(mine.y);
      const uint32_t up = (top & 0x7f800000u) + 0x00800000u;
      apart = low != 0 && (~low >> 23) + kUnitRange < up >> 23;
      if (!apart) vref = up;
    }
  };
  auto value_factors = [&](int ti) __attribute__((always_inline)) -> Factors {
    Factors f;
    if constexpr (kQ8) {
      const float inv = __uint_as_float(0x7f000000u - vref);  // 1 / vref
#pragma unroll
      for (int i = 0; i < kMine16; ++i) f.x[i] = lane_f(win.vf, block_at(ti * kKT + 32 * half + 16 * i)) * inv;
    }
    return f;
  };
  auto row_max = [&](const f32x16_t (&s)[kMine32], const Factors& f) __attribute__((always_inline)) {
    float x = ninf;
#pragma unroll
    for (int kt = 0; kt < kMine32; ++kt)
#pragma unroll
      for (int i = 0; i < 16; ++i) x = fmaxf(x, s[kt][i] * f.x[2 * kt + (i >> 3)]);
    return max_xor32(x);
  };
  auto weight = [&](float y, int i, const Factors& g, P8 (&ph)[kMine16], float (&ps)[4]) __attribute__((always_inline)) {
    const float pe = fast_exp2(y);
    ps[i & 3] = i < 4 ? pe : ps[i & 3] + pe;
    if constexpr (kQ8)
      ph[i >> 3][i & 7] = (_Float16)(pe * g.x[i >> 3]);
    else
      ph[i >> 3][i & 7] = (__bf16)pe;
  };
  auto scores = [&](int st, f32x16_t (&s)[kMine32]) __attribute__((always_inline)) {
    bf16x8_t ka[kMine32];
#pragma unroll
    for (int kt = 0; kt < kMine32; ++kt)
#pragma unroll
      for (int i = 0; i < 16; ++i) s[kt][i] = 0.f;
#pragma unroll
    for (int ks = 0; ks < 8; ++ks) {
      read_k(st, ks, ka);
#pragma unroll
      for (int kt = 0; kt < kMine32; ++kt) s[kt] = mfma32(ka[kt], qb[ks], s[kt]);
    }
  };
  // Weights of one tile (scores s) interleaved with the scores of the next
  // (K stage st, into sn).
  auto weights_scores = [&](auto stage, const f32x16_t (&s)[kMine32], f32x16_t (&sn)[kMine32], const Factors& f,
                            const Factors& g, P8 (&ph)[kMine16]) __attribute__((always_inline)) {
    constexpr int st = decltype(stage)::value;
    float ps[4] = {0.f, 0.f, 0.f, 0.f};
    bf16x8_t ka[2][kMine32];
    read_k(st, 0, ka[0]);
#pragma unroll
    for (int kt = 0; kt < kMine32; ++kt)
#pragma unroll
      for (int i = 0; i < 16; ++i) sn[kt][i] = 0.f;
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int ks = 0; ks < 8; ++ks) {
      if (ks < 7) read_k(st, ks + 1, ka[(ks + 1) & 1]);
#pragma unroll
      for (int kt = 0; kt < kMine32; ++kt) {
        sn[kt] = mfma32(ka[ks & 1][kt], qb[ks], sn[kt]);
#pragma unroll
        for (int i = 2 * (kMine32 * ks + kt); i < 2 * (kMine32 * ks + kt) + 2; ++i)
          weight(fmaf(s[i >> 4][i & 15], f.x[i >> 3], -m), i, g, ph, ps);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    __builtin_amdgcn_s_setprio(0);
    return (ps[0] + ps[1]) + (ps[2] + ps[3]);
  };
  // P.V of one tile whose value scales (g) have any sizes: for each 16 keys, which
  // have one scale, the row's weights in units of a power of two that brings the
  // largest to 2^14 .. 2^15 (fp16 ends at 2^16), a product of their own, and that
  // added in fp32 times unit and scale. What a row adds up so is off by 2^-11 of
  // itself, whatever other rows see. Gives the sum of the weights.
  auto products_apart = [&](int st, const f32x16_t (&s)[kMine32], const Factors& f, const Factors& g)
                            __attribute__((always_inline)) -> float {
    constexpr uint32_t kLeastUnit = 15u << 23;  // 2^-112: its inverse is finite
    const float mref = m == ninf ? 0.f : m;
    float sum = 0.f;
#pragma unroll
    for (int ks = 0; ks < kMine16; ++ks) {
      float p[8], pm = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int at = 8 * ks + i;
        p[i] = fast_exp2(sub_rounded(s[at >> 4][at & 15] * f.x[ks], mref));
        pm = fmaxf(pm, p[i]);
        sum += p[i];
      }
      const uint32_t e = max(__float_as_uint(max_xor32(pm)) & 0x7f800000u, kLeastUnit);
      const float up = __uint_as_float((268u << 23) - e);  // 2^14 over the unit e
      const float back = __uint_as_float(e - (14u << 23)) * g.x[ks];
      P8 w;
#pragma unroll
      for (int i = 0; i < 8; ++i) w[i] = (Weight)(p[i] * up);
#pragma unroll
      for (int dt = 0; dt < 4; ++dt) {
        f32x16_t part;
#pragma unroll
        for (int i = 0; i < 16; ++i) part[i] = 0.f;
        part = mfma32(read_v32(st, ks, dt), w, part);
#pragma unroll
        for (int i = 0; i < 16; ++i) o[dt][i] = fmaf(part[i], back, o[dt][i]);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    return sum;
  };
  // The split's tiles one after the other, for value scales of any sizes: the
  // codes of the next tile on their way while one is worked on, K and V tiles in
  // two stages, so that one barrier a tile is enough.
  auto walk_apart = [&]() __attribute__((always_inline)) {
#pragma unroll 1
    for (int ti = 0; ti < ntiles; ++ti) {
      const int st = ti & 1, t0 = k0 + ti * kKT;
      if (block_at(ti * kKT) >= 32) {
        wbase += 32;
        take_window(coming);
        coming = load_window(wbase + 32);
      }
      __builtin_amdgcn_s_waitcnt(kWaitVm0);
      put(true, ti, raw_at(true), st);
      put(false, ti, raw_at(false), st);
      ask(true, ti + 1, raw_at(true));
      ask(false, ti + 1, raw_at(false));
      __builtin_amdgcn_s_waitcnt(kWaitLgkm0);
      bare_barrier();
      f32x16_t s[kMine32];
      fresh(kbase);
      fresh(vbase);
      scores(st, s);
      if (t0 + kKT > cut) mask(t0, s);
      const Factors f = key_factors(ti), g = value_factors(ti);
      const float mn = fmaxf(m, row_max(s, f));
      const float alpha = m == mn ? 1.f : fast_exp2(m - mn);
      m = mn;
#pragma unroll
      for (int dt = 0; dt < 4; ++dt) o[dt] *= alpha;
      l = l * alpha + products_apart(st, s, f, g);
    }
    __builtin_amdgcn_s_waitcnt(kWaitVm0);
    __builtin_amdgcn_s_waitcnt(kWaitLgkm0);
    bare_barrier();
  };
  // One tile: its weights (scores s) with the next tile's scores (sn), then
  // its P.V.
  //
  // Order between the waves, with a barrier before every kBar-th tile p only.
  // Rounds p .. p + kBar - 1 read K(p + 1) .. K(p + kBar) and V(p) .. V(p + kBar
  // - 1). After the barrier the stages of as many tiles before these are free;
  // K(p + kBar + 1) .. K(p + 2 kBar) and V(p + kBar) .. V(p + 2 kBar - 1) are
  // brought into them, and are there at the next barrier, before which every
  // wave has waited for its own.
  auto round = [&](int ti, auto stage, f32x16_t (&s)[kMine32], f32x16_t (&sn)[kMine32], const Factors& f,
                   Factors& fn) __attribute__((always_inline)) {
    constexpr int st = decltype(stage)::value;
    const int t0 = k0 + ti * kKT;
    if constexpr (st % kBar == 0) {
      if constexpr (!kQ8) __builtin_amdgcn_s_waitcnt(kWaitVm0);
      __builtin_amdgcn_s_waitcnt(kWaitLgkm0);
      bare_barrier();
      if constexpr (!kQ8) {
#pragma unroll
        for (int j = 0; j < kBar; ++j) issue_k(ti + kBar + 1 + j, (st + kBar + 1 + j) % kStages);
#pragma unroll
        for (int j = 0; j < kBar; ++j) issue_v(ti + kBar + j, (st + kBar + j) % kStages);
      }
    }
    if constexpr (!kQ8) {
      // What this wave brought of a tile that some row masks: any value that
      // is not finite? In the second pass such values are cleared.
      if (__builtin_expect(guard || t0 + kKT > wg_cut, 0)) {
        bool odd = false;
#pragma unroll
        for (int e = 0; e < 2 * kUnits; ++e) {
          uint8_t* at = lds.v[st] + (wrow + 4 * e) * kRowBytes + 16 * lane;
          const U4 x = ld16(at);
          const bool some = not_finite2(x.x) || not_finite2(x.y) || not_finite2(x.z) || not_finite2(x.w);
          if (guard && some) st16(at, U4{finite_or_0(x.x), finite_or_0(x.y), finite_or_0(x.z), finite_or_0(x.w)});
          odd = odd || some;
        }
        if (__any(odd)) lds.odd = 1;
        if (guard) {
          __builtin_amdgcn_s_waitcnt(kWaitLgkm0);
          bare_barrier();
        }
      }
    }
    if constexpr (kQ8) {
      if (__builtin_expect(block_at(ti * kKT) >= 32, 0)) {
        wbase += 32;
        take_window(coming);
        coming = load_window(wbase + 32);
      }
    }
    const Factors g = value_factors(ti);
    fn = key_factors(ti + 1);
    P8 ph[kMine16];
    fresh(kbase);
    __builtin_amdgcn_sched_barrier(0);
    float ps = weights_scores(std::integral_constant<int, (st + 1) % kStages>{}, s, sn, f, g, ph);
    // Rare: move the reference and form the weights again. A row without one
    // so far (no tile with a finite score) takes this branch too.
    if (__builtin_expect(__any(!(ps <= kMaxWeightSum)), 0)) {
      const float mn = fmaxf(m, row_max(s, f));
      const float alpha = m == mn ? 1.f : fast_exp2(m - mn);
      m = mn;
      l *= alpha;
#pragma unroll
      for (int dt = 0; dt < 4; ++dt) o[dt] *= alpha;
      const float mref = m == ninf ? 0.f : m;
      float pt[4] = {0.f, 0.f, 0.f, 0.f};
      // From the rounded logits that the reference is the maximum of: with
      // logits past 2^31 the unrounded product may exceed it by hundreds.
#pragma unroll
      for (int i = 0; i < 16 * kMine32; ++i) weight(sub_rounded(s[i >> 4][i & 15] * f.x[i >> 3], mref), i, g, ph, pt);
      ps = (pt[0] + pt[1]) + (pt[2] + pt[3]);
    }
    l += ps;
    if (__builtin_expect(t0 + 2 * kKT > cut, 0)) mask(t0 + kKT, sn);
    // The codes of K(ti + kBar + 1) and V(ti + kBar), asked for a round ago.
    Codes wk, wv;
    if constexpr (kQ8) {
      __builtin_amdgcn_s_waitcnt(kWaitVm0);
      compiler_fence();
      wk = codes_at(raw_at(true));
      wv = codes_at(raw_at(false));
    }
    __builtin_amdgcn_sched_barrier(0);
    P8 va[2][4];
    uint32_t four[2];
    fresh(vbase);
    read_v(st, 0, va[0]);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int ks = 0; ks < kMine16; ++ks) {
      if (ks < kMine16 - 1) read_v(st, ks + 1, va[(ks + 1) & 1]);
#pragma unroll
      for (int dt = 0; dt < 4; ++dt) {
        o[dt] = mfma32(va[ks & 1][dt], ph[ks], o[dt]);
        // The words of codes (K's, then V's) shared out under the MFMAs.
        if constexpr (kQ8) {
          constexpr int kWords = 8 * kUnits, kMfmas = 4 * kMine16;
          const int n = 4 * ks + dt;
#pragma unroll
          for (int w = n * kWords / kMfmas; w < (n + 1) * kWords / kMfmas; ++w) {
            if (w < 4 * kUnits) put_word(true, wk, w, (st + kBar + 1) % kStages, four);
            else put_word(false, wv, w - 4 * kUnits, (st + kBar) % kStages, four);
          }
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    if constexpr (kQ8) {
      put_odd(true, ti + kBar + 1, (st + kBar + 1) % kStages);
      put_odd(false, ti + kBar, (st + kBar) % kStages);
      compiler_fence();  // the codes have been read when the next are asked for
      ask(true, ti + kBar + 2, raw_at(true));
      ask(false, ti + kBar + 1, raw_at(false));
    }
    __builtin_amdgcn_sched_barrier(0);
  };

  if constexpr (kQ8) {
    take_window(load_window(0));
    coming = load_window(32);
  }
  // The first tiles of K and V on their way.
  auto request = [&]() __attribute__((always_inline)) {
    if constexpr (!kQ8) {
#pragma unroll
      for (int t = 0; t <= kBar; ++t) issue_k(t, t);
#pragma unroll
      for (int t = 0; t < kBar; ++t) issue_v(t, t);
    }
  };
  request();
  if constexpr (!kQ8) exchange_q();
  for (;;) {
    if constexpr (kQ8) {
      // Beside K(0) and V(0), the first ones by way of the stages that nothing
      // is put into yet.
      const uint32_t spare_v = __builtin_amdgcn_readfirstlane(lds0) + (uint32_t)offsetof(Lds, v[kStages - 1]) + raw_of_wave;
      const uint32_t spare_k = __builtin_amdgcn_readfirstlane(lds0) + (uint32_t)offsetof(Lds, k[kStages - 1]) + raw_of_wave;
      ask(true, 0, raw_at(true));
      ask(false, 0, raw_at(false));
      ask(true, 1, spare_v);
      if constexpr (kBar == 2) {
        ask(true, 2, spare_v + kKT * kHeadDim);
        ask(false, 1, spare_k);
      }
      exchange_q();
      look_at_scales();
      __builtin_amdgcn_s_waitcnt(kWaitVm0);
      __builtin_amdgcn_s_waitcnt(kWaitLgkm0);
      bare_barrier();  // codes go where queries were
      take_bounds();
      if (__builtin_expect(apart, 0)) {
        walk_apart();
        break;
      }
      put(true, 0, raw_at(true), 0);
      put(false, 0, raw_at(false), 0);
      put(true, 1, spare_v, 1);
      if constexpr (kBar == 2) {
        put(true, 2, spare_v + kKT * kHeadDim, 2);
        put(false, 1, spare_k, 1);
      }
      ask(true, kBar + 1, raw_at(true));
      ask(false, kBar, raw_at(false));
    } else {
      __builtin_amdgcn_s_waitcnt(kWaitVm0);
    }
    __builtin_amdgcn_s_waitcnt(kWaitLgkm0);
    bare_barrier();
    f32x16_t sa[kMine32], sb[kMine32];
    scores(0, sa);
    if (k0 + kKT > cut) mask(k0, sa);
    Factors fa = key_factors(0), fb;
    m = row_max(sa, fa);
    for (int ti = 0; ti < ntiles; ti += kStages) {
      round(ti, std::integral_constant<int, 0>{}, sa, sb, fa, fb);
      if (ti + 1 >= ntiles) break;
      round(ti + 1, std::integral_constant<int, 1>{}, sb, sa, fb, fa);
      if constexpr (kStages == 4) {
        if (ti + 2 >= ntiles) break;
        round(ti + 2, std::integral_constant<int, 2>{}, sa, sb, fa, fb);
        if (ti + 3 >= ntiles) break;
        round(ti + 3, std::integral_constant<int, 3>{}, sb, sa, fb, fa);
      }
    }
    // No load may still be writing LDS when the workgroup ends or starts over.
    __builtin_amdgcn_s_waitcnt(kWaitVm0);
    __builtin_amdgcn_s_waitcnt(kWaitLgkm0);
    bare_barrier();
    if constexpr (kQ8) {
      break;
    } else if (guard || __builtin_expect(lds.odd == 0, 1)) {
      break;
    }
    guard = true;
    clear_o();
    l = 0.f;
    request();
  }

  // The halves of the keys: the second waves hand over what they have.
  if constexpr (kHalves) {
    f32x4_t* slot = reinterpret_cast<f32x4_t*>(lds.k[0]) + rwave * (17 * 64) + lane;
    static_assert(2 * 17 * 64 * sizeof(f32x4_t) <= sizeof(Lds::k) + sizeof(Lds::v));
    if (half == 1) {
#pragma unroll
      for (int dt = 0; dt < 4; ++dt)
#pragma unroll
        for (int i4 = 0; i4 < 4; ++i4)
          slot[64 * (4 * dt + i4)] = f32x4_t{o[dt][4 * i4], o[dt][4 * i4 + 1], o[dt][4 * i4 + 2], o[dt][4 * i4 + 3]};
      slot[64 * 16] = f32x4_t{m, l, 0.f, 0.f};
    }
    __builtin_amdgcn_s_waitcnt(kWaitLgkm0);
    bare_barrier();
    if (half == 1) return;
    const f32x4_t ml = slot[64 * 16];
    const float mn = fmaxf(m, ml[0]);
    const float x0 = m == mn ? 1.f : fast_exp2(m - mn), x1 = ml[0] == mn ? 1.f : fast_exp2(ml[0] - mn);
    m = mn;
    l = l * x0 + ml[1] * x1;
#pragma unroll
    for (int dt = 0; dt < 4; ++dt)
#pragma unroll
      for (int i4 = 0; i4 < 4; ++i4) {
        const f32x4_t p = slot[64 * (4 * dt + i4)];
#pragma unroll
        for (int u = 0; u < 4; ++u) o[dt][4 * i4 + u] = o[dt][4 * i4 + u] * x0 + p[u] * x1;
      }
  }

  // V values that are not finite, cleared in the second pass: whoever sees
  // one gets it added. Lane (r, c) looks at 16 bytes of rows r, r + 4, ...
  if constexpr (!kQ8) {
    if (__builtin_expect(guard, 0)) {
      const uint16_t* vb = a.v + (int64_t)sr.first * a.v_stride + hk * kHeadDim;
#pragma unroll 1
      for (int t = k0; t < k1; t += 4) {
        const int mine = t + lrow;
        const U4 x = ld16(vb + (int64_t)min(mine, k1 - 1) * a.v_stride + 8 * lslot);
        uint64_t who = __ballot(mine < k1 && (not_finite2(x.x) || not_finite2(x.y) || not_finite2(x.z) || not_finite2(x.w)));
#pragma unroll 1
        while (who != 0) {
          const int r = __builtin_ctzll(who) >> 4;
          who &= ~(0xffffull << (16 * r));
          const uint16_t* vp = vb + (int64_t)(t + r) * a.v_stride + 4 * hi;
          const bool see = t + r <= lim;
#pragma unroll
          for (int dt = 0; dt < 4; ++dt)
#pragma unroll
            for (int i = 0; i < 16; i += 2) {
              const uint32_t w = *reinterpret_cast<const uint32_t*>(vp + 32 * dt + 8 * (i >> 2) + (i & 3));
              o[dt][i] += see && !finite_f(bf_lo(w)) ? bf_lo(w) : 0.f;
              o[dt][i + 1] += see && !finite_f(bf_hi(w)) ? bf_hi(w) : 0.f;
            }
        }
      }
    }
  }

  const float lt = sum_xor32(l);
  const float inv = lt == 0.f ? 0.f : (kQ8 ? __uint_as_float(vref) : 1.f) / lt;
  if (rho >= R) return;
  const int row = sr.first + rho / G, head = hk * G + rho % G;
  const size_t oi = (size_t)row * a.q_heads + head;
  const float l2 = lt == 0.f ? ninf : m + fast_log2(lt);
  if (S > 1) {
    const size_t pi = (size_t)split * a.rows * a.q_heads + oi;
    float* po = a.part_o + pi * kHeadDim;
#pragma unroll
    for (int dt = 0; dt < 4; ++dt)
#pragma unroll
      for (int i4 = 0; i4 < 4; ++i4)
        *reinterpret_cast<f32x4_t*>(po + 32 * dt + 8 * i4 + 4 * hi) =
            f32x4_t{o[dt][4 * i4] * inv, o[dt][4 * i4 + 1] * inv, o[dt][4 * i4 + 2] * inv, o[dt][4 * i4 + 3] * inv};
    if (hi == 0) a.part_lse[pi] = l2;
    return;
  }
  // Lane (lq, hi) holds dims 32 dt + 8 i4 + 4 hi .. + 4 of its row: a lane
  // swap gives hi = 0 the eight dims of i4 and hi = 1 those of i4 + 1.
  uint16_t* out = a.out + oi * kHeadDim;
#pragma unroll
  for (int dt = 0; dt < 4; ++dt)
#pragma unroll
    for (int i4 = 0; i4 < 4; i4 += 2) {
      uint32_t x[2][2];
#pragma unroll
      for (int e = 0; e < 2; ++e)
#pragma unroll
        for (int u = 0; u < 2; ++u)
          x[e][u] = pack_bf16(o[dt][4 * (i4 + e) + 2 * u] * inv, o[dt][4 * (i4 + e) + 2 * u + 1] * inv);
      const auto s0 = __builtin_amdgcn_permlane32_swap(x[0][0], x[1][0], false, false);
      const auto s1 = __builtin_amdgcn_permlane32_swap(x[0][1], x[1][1], false, false);
      st16(out + 32 * dt + 8 * i4 + 8 * hi, U4{s0[0], s1[0], s0[1], s1[1]});
    }
  if (hi == 0 && a.lse) a.lse[oi] = lt == 0.f ? ninf : l2 * kLn2;
}

// Log-sum-exp merge of the splits (Alg. 2, "Combine"): a wave per (row, query
// head), lane i holding dims 2 i and 2 i + 1. A row reads the splits that hold
// keys it sees; rows of no sequence are left as they are.
template <int kSrc>
__global__ __launch_bounds__(256) void k_rows_combine(RowsArgs a) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t oi = (int64_t)blockIdx.x * 4 + wave;
  const int row = (int)(oi / a.q_heads);
  if (row >= a.rows) return;
  // The sequence whose packed rows hold this row.
  int seq = -1;
  const SeqRows q0 = lane < a.batch ? seq_rows<kSrc>(a, lane) : SeqRows{0, 0, 0};
  for (int base = 0; base < a.batch && seq < 0; base += 64) {
    bool mine = false;
    if (base + lane < a.batch) {
      const SeqRows q = base == 0 ? q0 : seq_rows<kSrc>(a, base + lane);
      mine = row >= q.first && row < q.first + q.n;
    }
    const uint64_t who = __ballot(mine);
    if (who != 0) seq = base + __builtin_ctzll(who);
  }
  if (seq < 0) return;
  const SeqRows sr = seq_rows<kSrc>(a, seq);
  const int keys = sr.L - sr.n + (row - sr.first) + 1;
  const int chunk = split_chunk<kSrc>(a, q0, (q0.n * a.group + a.per - 1) >> __builtin_ctz(a.per));
  const int n = splits_of<kSrc>(a, keys, chunk);
  const size_t stride = (size_t)a.rows * a.q_heads;
  const float ninf = -__builtin_inff();
  float m = ninf, l = 0.f;
  f2_t acc = {0.f, 0.f};
  for (int b = 0; b < n; b += 64) {
    const int cnt = min(64, n - b);
    const float x = lane < cnt ? a.part_lse[(size_t)(b + lane) * stride + oi] : ninf;
    const float mn = fmaxf(m, wave_max_f(x));
    const float e = x == ninf ? 0.f : fast_exp2(x - mn);
    const float alpha = m == ninf ? 0.f : fast_exp2(m - mn);
    l = fmaf(l, alpha, wave_sum_f(e));
    acc *= alpha;
    m = mn;
    for (int q = 0; q < cnt; q += 16) {
      f2_t p[16];
#pragma unroll
      for (int u = 0; u < 16; ++u) {
        p[u] = f2_t{0.f, 0.f};
        if (q + u < cnt)
          p[u] = *reinterpret_cast<const f2_t*>(a.part_o + ((size_t)(b + q + u) * stride + oi) * kHeadDim + 2 * lane);
      }
#pragma unroll
      for (int u = 0; u < 16; ++u)
        acc += __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, e), (q + u) & 63)) * p[u];
    }
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
  reinterpret_cast<uint32_t*>(a.out + oi * kHeadDim)[lane] = pack_bf16(acc.x * inv, acc.y * inv);
  if (lane == 0 && a.lse) a.lse[oi] = l == 0.f ? ninf : (m + fast_log2(l)) * kLn2;
}

// Query blocks of a launch at most: a sequence's last one may not be full.
int64_t most_blocks(const RowsArgs& a, int per) { return (int64_t)a.rows * a.group / per + a.batch; }

template <int kRows, int kSrc, bool kPaged>
hipError_t launch_attn(const RowsArgs& a, hipStream_t stream) {
  // Of one length, every block takes as many splits of a.chunk as the longest.
  int64_t items = most_blocks(a, kRows);
  if (a.num_splits > 1) items = std::max<int64_t>(items * a.even_splits, a.places / a.kv_heads);
  const int64_t grid = items * a.kv_heads;
  if (grid > INT32_MAX) return hipErrorInvalidValue;
  hipLaunchKernelGGL((k_rows_attn<kRows, kSrc, kPaged>), dim3((uint32_t)grid), dim3(64 * waves_of(kRows)), 0, stream, a);
  return hipGetLastError();
}

// Workgroups of `per` rows over one split of the keys.
int64_t rows_wgs(int32_t batch, int32_t kv_heads, int32_t group, int32_t rows, int per) {
  const int64_t each = ((int64_t)((rows + batch - 1) / batch) * group + per - 1) / per;
  return (each < 1 ? 1 : each) * batch * kv_heads;
}
// Splits that fill `slots` places for workgroups once.
int64_t splits_within(int64_t wgs, int64_t slots) { return wgs >= slots ? 1 : slots / wgs; }

// Rows of a workgroup over a cache. Few rows a sequence: as few as hold them
// (32 rows of one head for each of 8 kv heads behind 8 x 32K: 183 us by 128
// rows, 146 by 64; 32 rows of four behind 8 x 64K 381 and 505). More: 256, which
// share the conversion of the codes, where the rows fill three quarters of the
// places (512 rows of 32 heads over 8 behind 32K: 288 us by 256, 320 by 128; 100
// behind 8 x 8K 167 and 181), else 128, two workgroups a CU (54 rows of 40 behind
// 6 x 3.5K 90 and 79; 340 of 16 over 4 behind 8 of up to 3.7K 127 and 114).
int rows_of_block(int32_t batch, int32_t kv_heads, int32_t group, int32_t rows) {
  const int64_t all = (int64_t)rows * group;
  if (all <= (int64_t)64 * batch) return 64;
  if (all <= (int64_t)128 * batch) return 128;
  const int64_t wgs = rows_wgs(batch, kv_heads, group, rows, 256), splits = splits_within(wgs, kCus);
  const int64_t places = wgs * splits > kCus ? wgs * splits : kCus;
  return 4 * all * kv_heads * splits >= 3 * 256 * places ? 256 : 128;
}

// Key splits at most. 256 rows: no more than run at once, one workgroup a CU
// (93 rows of 12 heads over 2 behind 6 of up to 36K: 167 us with 7 splits, 252
// workgroups; with 8, 288 workgroups, 273). Fewer: a workgroup on every CU at
// least, and as many as run at once, two a CU, where a split stays long: every
// split writes its rows' sums and the merge reads them again. 32 rows of 32 heads
// behind 8K: 32.9 us with one workgroup a CU, 40.0 with two; behind 8 x 64K 444
// and 384.
struct RowsPlan {
  int per;
  int64_t splits, places;
};
RowsPlan rows_plan(int32_t batch, int32_t kv_heads, int32_t group, int32_t rows, int32_t max_seq_len) {
  const int per = rows_of_block(batch, kv_heads, group, rows);
  const int64_t wgs = rows_wgs(batch, kv_heads, group, rows, per);
  if (per == 256) return {per, splits_within(wgs, kCus), kCus};
  const int64_t least = wgs >= kCus ? 1 : (kCus + wgs - 1) / wgs;
  const bool is_long = max_seq_len >= kLongSplit * least;
  return {per, is_long ? splits_within(wgs, 2 * kCus) : least, is_long ? 2 * kCus : wgs * least};
}

template <int kSrc, bool kPaged>
hipError_t launch_q8(const RowsArgs& a, hipStream_t stream) {
  const hipError_t e = a.per == 64    ? launch_attn<64, kSrc, kPaged>(a, stream)
                       : a.per == 128 ? launch_attn<128, kSrc, kPaged>(a, stream)
                                      : launch_attn<256, kSrc, kPaged>(a, stream);
  if (e != hipSuccess || a.num_splits == 1) return e;
  const int64_t outs = (int64_t)a.rows * a.q_heads;
  hipLaunchKernelGGL(k_rows_combine<kSrc>, dim3((uint32_t)((outs + 3) / 4)), dim3(256), 0, stream, a);
  return hipGetLastError();
}

}  // namespace

void rows_splits(RowsArgs* a, int32_t max_seq_len) {
  const RowsPlan p = rows_plan(a->batch, a->kv_heads, a->group, a->rows, max_seq_len);
  const int64_t chunk = ((max_seq_len + p.splits - 1) / p.splits + 63) / 64 * 64;
  a->chunk = (int32_t)(chunk < 128 ? 128 : chunk);
  a->per = p.per;
  a->places = (int32_t)p.places;
  a->even_splits = (int32_t)(((int64_t)max_seq_len + a->chunk - 1) / a->chunk);
  a->num_splits = a->even_splits == 1 ? 1 : rows_max_splits(a->batch, a->kv_heads, a->group, a->rows, max_seq_len);
}

// A bound on the splits that never decreases as the length grows: twice those
// of equal lengths, of 128 keys at least.
int32_t rows_max_splits(int32_t batch, int32_t kv_heads, int32_t group, int32_t rows, int32_t max_seq_len) {
  const int64_t most = rows_plan(batch, kv_heads, group, rows, max_seq_len).splits;
  const int64_t by_len = ((int64_t)max_seq_len + 127) / 128;
  if (most == 1 || by_len <= 1) return 1;
  const int64_t s = batch == 1 ? most : 2 * most;
  return (int32_t)(by_len < s ? by_len : s);
}

hipError_t launch_rows_q8(const RowsArgs& a, int32_t format, hipStream_t stream) {
  const bool paged = a.c.table != nullptr;
  if (format == RESA_Q8_INT8) return paged ? launch_q8<RESA_Q8_INT8, true>(a, stream) : launch_q8<RESA_Q8_INT8, false>(a, stream);
  return paged ? launch_q8<RESA_Q8_E4M3, true>(a, stream) : launch_q8<RESA_Q8_E4M3, false>(a, stream);
}

hipError_t launch_prompt(const RowsArgs& a, hipStream_t stream) {
  // Small launches in small workgroups, as long as all of them run at once (two
  // a CU): 1000 tokens of 32 / 8 heads 27.3 us by 128 rows, 24.5 by 64; 8 prompts
  // of up to 250, whose 625 blocks do not, 15.3 and 19.6.
  if (most_blocks(a, 64) * a.kv_heads <= 2 * kCus) return launch_attn<64, kPacked, false>(a, stream);
  // Two workgroups a CU while prompts are short (one computes while the other
  // starts): 30 of 1000 tokens, 8 heads over 8, 67 us by 256 rows, 52 by 128; 64 of up
  // to 700, 32 over 8, 200 and 191; 8 of up to 4000 446 and 437; 4 of 4000, 28 over 4, 452
  // and 458; one of 16384 1912 and 1975.
  return a.rows <= (int64_t)kShortPrompt * a.batch || most_blocks(a, 256) * a.kv_heads < 2 * kCus
             ? launch_attn<128, kPacked, false>(a, stream)
             : launch_attn<256, kPacked, false>(a, stream);
}

}  // namespace resa
