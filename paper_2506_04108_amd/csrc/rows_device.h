// Device helpers of the calls on packed rows and 8-bit caches (gfx950, wave64).
//
// Packed rows: the rows of sequence s are rows [cu[s], cu[s + 1]) of a
// [rows, heads, head_dim] array, and they are the last rows of the sequence,
// positions [L - n, L). Work items (blocks, query blocks) are dealt to the
// sequences in the kernels, from cu and the lengths: the host knows neither,
// and launches an upper bound.
#pragma once

#include "resa_internal.h"

namespace resa {

typedef __bf16 bf16x2v_t __attribute__((ext_vector_type(2)));
typedef unsigned short u16x2_t __attribute__((ext_vector_type(2)));

typedef int32_t i32x4_t __attribute__((ext_vector_type(4)));

// s_waitcnt immediates: LDS operations done; at most n (< 64) vector loads out.
constexpr int kWaitLgkm0 = 0xC07F;
constexpr int wait_vm(int n) { return (n & 15) | ((n >> 4) << 14) | 0x0F70; }

// Words of a buffer resource over `bytes` bytes at p (stride 0, 32-bit format),
// both the same in every lane. Offsets at or past `bytes` read as zero.
__device__ __forceinline__ i32x4_t rsrc_words(const void* p, int bytes) {
  const uint64_t u = reinterpret_cast<uint64_t>(p);
  return i32x4_t{(int32_t)__builtin_amdgcn_readfirstlane((uint32_t)u),
                 (int32_t)(__builtin_amdgcn_readfirstlane((uint32_t)(u >> 32)) & 0xffffu),
                 __builtin_amdgcn_readfirstlane(bytes), kBufWord3};
}
// LDS byte address of an LDS object.
__device__ __forceinline__ uint32_t lds_addr(const void* p) {
  return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void*)p;
}
// A wave's eight rows of a tile straight into LDS: lane i's 16 bytes at offset
// voff0 (voff1) of the resource land at lds + 16 i (lds + 1024 + 16 i). The
// completion is ordered by hand (vmcnt 0, then a barrier). M0 is restored.
template <bool kNt = false>
__device__ __forceinline__ void lds_load_rows8(uint32_t lds, uint32_t voff0, uint32_t voff1, i32x4_t rk) {
  uint32_t saved;
  if constexpr (kNt)
    __asm__ volatile(
        "s_mov_b32 %0, m0\n\t"
        "s_mov_b32 m0, %1\n\ts_nop 0\n\tbuffer_load_dwordx4 %2, %4, 0 offen nt lds\n\t"
        "s_add_i32 m0, %1, 1024\n\ts_nop 0\n\tbuffer_load_dwordx4 %3, %4, 0 offen nt lds\n\t"
        "s_mov_b32 m0, %0"
        : "=&s"(saved) : "s"(lds), "v"(voff0), "v"(voff1), "s"(rk) : "memory", "scc");
  else
    __asm__ volatile(
        "s_mov_b32 %0, m0\n\t"
        "s_mov_b32 m0, %1\n\ts_nop 0\n\tbuffer_load_dwordx4 %2, %4, 0 offen lds\n\t"
        "s_add_i32 m0, %1, 1024\n\ts_nop 0\n\tbuffer_load_dwordx4 %3, %4, 0 offen lds\n\t"
        "s_mov_b32 m0, %0"
        : "=&s"(saved) : "s"(lds), "v"(voff0), "v"(voff1), "s"(rk) : "memory", "scc");
}
// One dword a lane likewise, at offset voff of the resource: lane i's lands at
// lds + 4 i.
__device__ __forceinline__ void lds_load_dword(uint32_t lds, uint32_t voff, i32x4_t rk) {
  uint32_t saved;
  __asm__ volatile(
      "s_mov_b32 %0, m0\n\t"
      "s_mov_b32 m0, %1\n\ts_nop 0\n\tbuffer_load_dword %2, %3, 0 offen lds\n\t"
      "s_mov_b32 m0, %0"
      : "=&s"(saved) : "s"(lds), "v"(voff), "s"(rk) : "memory");
}
// Keeps the compiler from moving memory accesses across this point.
__device__ __forceinline__ void compiler_fence() { __asm__ volatile("" ::: "memory"); }

// Largest magnitude of a code value.
template <int kFmt>
struct Q8 {
  static constexpr float kMax = kFmt == RESA_Q8_INT8 ? 127.f : 448.f;
};
// Least magnitude a block's scale is made of (2^-100): scales stay normal
// numbers, and their reciprocals finite.
constexpr float kQ8Least = 7.888609052210118e-31f;

// Two fp32 values rounded to bf16 (nearest, ties to even), packed.
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  return __builtin_bit_cast(uint32_t, bf16x2v_t{(__bf16)lo, (__bf16)hi});
}

// Two fp32 values that are fp16 values, packed.
__device__ __forceinline__ uint32_t pack_f16_exact(float lo, float hi) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_pkrtz(lo, hi));
}
__device__ __forceinline__ bool finite_f(float x) { return fabsf(x) < __builtin_inff(); }

// The four codes of a word as fp32, exactly.
template <int kFmt>
__device__ __forceinline__ void codes_f32(uint32_t w, float (&x)[4]) {
  if constexpr (kFmt == RESA_Q8_INT8) {
    x[0] = (float)(int8_t)w;
    x[1] = (float)(int8_t)(w >> 8);
    x[2] = (float)(int8_t)(w >> 16);
    x[3] = (float)((int32_t)w >> 24);
  } else {
    const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false);
    const auto hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
    x[0] = lo[0];
    x[1] = lo[1];
    x[2] = hi[0];
    x[3] = hi[1];
  }
}

// A quotient rounded to 19 significant bits. The quotients a code is made of
// are of numbers with 8 and 7 significant bits (a row's bf16 value, the bf16
// magnitude of the scale, a code): one that is no tie between two codes is at
// least 2^-16 of its size away from the tie, so the rounding moves the fp32
// quotient's last bits back onto a tie and never onto one that is none. The
// code then is the exact quotient's, however the division rounds.
__device__ __forceinline__ float snap19(float y) {
  return __uint_as_float((__float_as_uint(y) + 0x10u) & ~0x1fu);
}

// Four quotients to codes (nearest, ties to even), packed.
template <int kFmt>
__device__ __forceinline__ uint32_t to_codes(const float (&y)[4]) {
  if constexpr (kFmt == RESA_Q8_INT8) {
    uint32_t b[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
      b[i] = (uint32_t)(int32_t)__builtin_rintf(fminf(fmaxf(snap19(y[i]), -127.f), 127.f));
    const uint32_t lo = __builtin_amdgcn_perm(b[1], b[0], 0x0c0c0400u);
    const uint32_t hi = __builtin_amdgcn_perm(b[3], b[2], 0x04000c0cu);
    return lo | hi;
  } else {
    float z[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) z[i] = fminf(fmaxf(snap19(y[i]), -448.f), 448.f);
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(z[0], z[1], 0, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(z[2], z[3], w, true);
    return (uint32_t)w;
  }
}

// Rows of sequence s in the packed order, cut to the array: [first, first + n).
__device__ __forceinline__ void packed_rows(const int32_t* cu, int rows, int s, int& first, int& n) {
  first = min(max(cu[s], 0), rows);
  n = max(min(max(cu[s + 1], 0), rows) - first, 0);
}

// The sequence that item i belongs to and its rank among that sequence's
// items; count(s) gives a sequence's items (0 past the last one). A wave takes
// 64 sequences at a time; every lane must be active and i uniform. False when
// there are no more than i items.
template <class Count>
__device__ __forceinline__ bool find_seq(int i, int batch, const Count& count, int& seq, int& rank) {
  const int lane = threadIdx.x & 63;
  for (int base = 0; base < batch; base += 64) {
    const int c = base + lane < batch ? count(base + lane) : 0;
    const int upto = (int)wave_incl_scan((uint32_t)c);
    const int total = __builtin_amdgcn_readlane(upto, 63);
    if (i < total) {
      const int at = __builtin_ctzll(__ballot(upto > i));
      seq = base + at;
      rank = i - __builtin_amdgcn_readlane(upto - c, at);
      return true;
    }
    i -= total;
  }
  return false;
}

// Sum over the 64 lanes, uniform.
__device__ __forceinline__ int wave_total(int x) {
  return __builtin_amdgcn_readlane((int)wave_incl_scan((uint32_t)x), 63);
}

// Maximum over the 64 lanes, uniform.
__device__ __forceinline__ uint32_t wave_max(uint32_t x) {
  x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, kDppXor1, 0xf, 0xf, true));
  x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, kDppXor2, 0xf, 0xf, true));
  x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, kDppHalfMirror, 0xf, 0xf, true));
  x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, kDppMirror, 0xf, 0xf, true));
  return max(max((uint32_t)__builtin_amdgcn_readlane((int)x, 0), (uint32_t)__builtin_amdgcn_readlane((int)x, 16)),
             max((uint32_t)__builtin_amdgcn_readlane((int)x, 32), (uint32_t)__builtin_amdgcn_readlane((int)x, 48)));
}

// The block scale's index of logical block m of (sequence, kv head), or -1
// when the block table sends it outside the pool.
__device__ __forceinline__ int64_t scale_index(const CacheArgs& c, int bb, int hk, int m) {
  if (c.table == nullptr) return ((int64_t)bb * c.kv_heads + hk) * c.max_blocks + m;
  const int page = c.table[(size_t)bb * c.max_blocks + m];
  if ((unsigned)page >= (unsigned)c.num_pages) return -1;
  return (int64_t)page * c.kv_heads + hk;
}

}  // namespace resa
