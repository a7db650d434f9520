// Activations in chunks of 8 elements, and the 8-bit checkpoint format.
//
// Format: a row is cut into groups of 32 values (the last one filled up with zeros).  A group has the
// scale 2^e, e the smallest integer >= -127 with 127 * 2^e >= its largest magnitude, and every value is
// held as the int8 code rint(v / 2^e) (half to even).  With a power of two as the scale
//   * v / 2^e is exact, so the codes depend on the values alone and not on how they were computed, and
//   * code * 2^e has at most 7 significant bits and is exact in bf16, so the tensor cores take it as an
//     operand without a second rounding.
// A linear scale (largest magnitude / 127) would use the codes' range fully (on average 0.7 of it is
// used here) but has neither property.  The scale is kept as the byte e + 127; 255 marks a group that
// holds an Inf or a NaN: it reads back as NaN everywhere, so that a broken activation stays visible.
// At e = 122, the largest, codes end at +-63: what is finite stays finite.
//
// Buffer: codes [rows][32 * groups], then, from the next multiple of 256 bytes, scale bytes
// [rows][groups rounded up to 4] (32-bit loads cover four groups of a row).
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace fa {

using bf16 = __nv_bfloat16;

__host__ __device__ inline long long act8_groups(long long cols) { return (cols + 31) / 32; }
__host__ __device__ inline long long act8_scale_pitch(long long cols) { return (act8_groups(cols) + 3) / 4 * 4; }
__host__ __device__ inline long long act8_scale_offset(long long rows, long long cols) {
  return (rows * act8_groups(cols) * 32 + 255) / 256 * 256;
}

// Part of a checkpoint a kernel works on: `codes` and `scales` point at its first row.
struct Act8 {
  uint8_t* codes;
  uint8_t* scales;
};

// Two floats in one 64-bit register: sm_100 works on both with one instruction.
struct F2 {
  unsigned long long v;
};
__device__ __forceinline__ F2 two(float lo, float hi) {
  F2 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r.v) : "f"(lo), "f"(hi));
  return r;
}
__device__ __forceinline__ F2 two(float both) { return two(both, both); }
__device__ __forceinline__ void apart(F2 a, float* lo, float* hi) {
  asm("mov.b64 {%0, %1}, %2;" : "=f"(*lo), "=f"(*hi) : "l"(a.v));
}
__device__ __forceinline__ F2 fma2(F2 a, F2 b, F2 c) {
  F2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v));
  return r;
}
__device__ __forceinline__ F2 mul2(F2 a, F2 b) {
  F2 r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
  return r;
}
__device__ __forceinline__ F2 add2(F2 a, F2 b) {
  F2 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
  return r;
}
__device__ __forceinline__ float sum_of(F2 a) {
  float lo, hi;
  apart(a, &lo, &hi);
  return lo + hi;
}

// ---- chunks: 8 neighbouring elements of a row per thread, neighbouring lanes holding neighbouring chunks
__device__ __forceinline__ float bf16_lo(uint32_t u) { return __uint_as_float(u << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t u) { return __uint_as_float(u & 0xffff0000u); }
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  __nv_bfloat162 t = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<uint32_t*>(&t);
}
__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(bf16 v) { return __bfloat162float(v); }
template <typename T> __device__ __forceinline__ T from_float(float v);
template <> __device__ __forceinline__ float from_float<float>(float v) { return v; }
template <> __device__ __forceinline__ bf16 from_float<bf16>(float v) { return __float2bfloat16_rn(v); }

template <typename T> struct Raw8;
template <> struct Raw8<bf16> {
  uint4 u;
  __device__ __forceinline__ void zero() { u = make_uint4(0, 0, 0, 0); }
  __device__ __forceinline__ void get(float (&v)[8]) const {
    v[0] = bf16_lo(u.x); v[1] = bf16_hi(u.x); v[2] = bf16_lo(u.y); v[3] = bf16_hi(u.y);
    v[4] = bf16_lo(u.z); v[5] = bf16_hi(u.z); v[6] = bf16_lo(u.w); v[7] = bf16_hi(u.w);
  }
  __device__ __forceinline__ void put(const float (&v)[8]) {
    u = make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
  }
  __device__ __forceinline__ void get(F2 (&v)[4]) const {
    v[0] = two(bf16_lo(u.x), bf16_hi(u.x)); v[1] = two(bf16_lo(u.y), bf16_hi(u.y));
    v[2] = two(bf16_lo(u.z), bf16_hi(u.z)); v[3] = two(bf16_lo(u.w), bf16_hi(u.w));
  }
  __device__ __forceinline__ void put(const F2 (&v)[4]) {
    float f[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) apart(v[i], &f[2 * i], &f[2 * i + 1]);
    put(f);
  }
  // bits of the largest magnitude, as a float's (NaN and Inf on top)
  __device__ __forceinline__ uint32_t top() const {
    const uint32_t k = 0x7FFF7FFFu;
    uint32_t a, b;
    asm("max.u16x2 %0, %1, %2;" : "=r"(a) : "r"(u.x & k), "r"(u.y & k));
    asm("max.u16x2 %0, %1, %2;" : "=r"(b) : "r"(u.z & k), "r"(u.w & k));
    asm("max.u16x2 %0, %1, %2;" : "=r"(a) : "r"(a), "r"(b));
    return max(a & 0xFFFF0000u, a << 16);
  }
  template <int N>
  __device__ __forceinline__ void from_words(const uint32_t (&w)[N]) { u = make_uint4(w[0], w[1], w[2], w[3]); }
  __device__ __forceinline__ void to_words(uint32_t (&w)[4]) const { w[0] = u.x; w[1] = u.y; w[2] = u.z; w[3] = u.w; }
  __device__ __forceinline__ void load(const bf16* p) { u = *reinterpret_cast<const uint4*>(p); }
  __device__ __forceinline__ void store(bf16* p) const { *reinterpret_cast<uint4*>(p) = u; }
};
template <> struct Raw8<float> {
  float4 a, b;
  __device__ __forceinline__ void zero() { a = b = make_float4(0.f, 0.f, 0.f, 0.f); }
  __device__ __forceinline__ void get(float (&v)[8]) const {
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
  }
  __device__ __forceinline__ void put(const float (&v)[8]) {
    a = make_float4(v[0], v[1], v[2], v[3]); b = make_float4(v[4], v[5], v[6], v[7]);
  }
  __device__ __forceinline__ void get(F2 (&v)[4]) const {
    v[0] = two(a.x, a.y); v[1] = two(a.z, a.w); v[2] = two(b.x, b.y); v[3] = two(b.z, b.w);
  }
  __device__ __forceinline__ void put(const F2 (&v)[4]) {
    apart(v[0], &a.x, &a.y); apart(v[1], &a.z, &a.w); apart(v[2], &b.x, &b.y); apart(v[3], &b.z, &b.w);
  }
  __device__ __forceinline__ uint32_t top() const {
    const float v[7] = {a.y, a.z, a.w, b.x, b.y, b.z, b.w};
    float m = fabsf(a.x);
#pragma unroll
    for (int i = 0; i < 7; ++i) asm("max.NaN.f32 %0, %1, %2;" : "=f"(m) : "f"(m), "f"(fabsf(v[i])));
    return __float_as_uint(m);
  }
  template <int N>
  __device__ __forceinline__ void from_words(const uint32_t (&w)[N]) {
    a = make_float4(__uint_as_float(w[0]), __uint_as_float(w[1]), __uint_as_float(w[2]), __uint_as_float(w[3]));
    b = make_float4(__uint_as_float(w[4]), __uint_as_float(w[5]), __uint_as_float(w[6]), __uint_as_float(w[7]));
  }
  __device__ __forceinline__ void to_words(uint32_t (&w)[8]) const {
    w[0] = __float_as_uint(a.x); w[1] = __float_as_uint(a.y); w[2] = __float_as_uint(a.z); w[3] = __float_as_uint(a.w);
    w[4] = __float_as_uint(b.x); w[5] = __float_as_uint(b.y); w[6] = __float_as_uint(b.z); w[7] = __float_as_uint(b.w);
  }
  __device__ __forceinline__ void load(const float* p) {
    a = *reinterpret_cast<const float4*>(p); b = *reinterpret_cast<const float4*>(p + 4);
  }
  __device__ __forceinline__ void store(float* p) const {
    *reinterpret_cast<float4*>(p) = a; *reinterpret_cast<float4*>(p + 4) = b;
  }
};

// The first `valid` elements one by one, zeros behind them.
template <typename T>
__device__ __forceinline__ Raw8<T> load_some(const T* p, int valid) {
  float v[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = j < valid ? to_float(p[j]) : 0.f;
  Raw8<T> r;
  r.put(v);        // exact: the values have T's precision
  return r;
}

// Words w[s / 4] onwards of a window, s in bytes: what lies s bytes into it.  s is a multiple of the element size and
// below 16; OUT + 4 words (OUT for s = 0) are read.
template <int OUT, bool HALVES>
__device__ __forceinline__ void shift_window(uint32_t (&w)[OUT + 4], uint32_t s) {
#pragma unroll
  for (int i = 0; i < OUT + 2; ++i) w[i] = (s & 8) ? w[i + 2] : w[i];
#pragma unroll
  for (int i = 0; i < OUT + 1; ++i) w[i] = (s & 4) ? w[i + 1] : w[i];
  if (HALVES) {
#pragma unroll
    for (int i = 0; i < OUT; ++i) w[i] = __funnelshift_r(w[i], w[i + 1], (s & 2) * 8);
  }
}

// A matrix that is read: `end` is where its last row ends.
template <typename T>
struct Source {
  const T* p;
  long long ld;
  const T* end;
};

// Elements first .. first + 7 of a row of `cols`, zeros past its end: fetched now, put together when they are needed, so
// that a fetch waits for nothing.  VEC: rows start on 16-byte boundaries and cols is a multiple of 8, so a chunk is one
// aligned load (fp32: two), or lies outside.  Otherwise it is cut out of the aligned 16-byte blocks its elements lie in,
// where these are inside the matrix (from its first element to its last; a block may reach over a row's end); the one
// or two chunks of a whole matrix where they are not are read element by element.
template <typename T, bool VEC>
struct Chunk {
  Raw8<T> r;
  // Always a load, of the matrix' first chunk where there is none: around a condition or with a default value the
  // compiler would not keep several under way.
  __device__ __forceinline__ void fetch(const Source<T>& m, const T* row, int first, int cols) {
    r.load(first < cols ? row + first : m.p);
  }
  // `in`: whether there was one (what it was fetched for); without one, zeros
  __device__ __forceinline__ Raw8<T> raw(bool in) const {
    Raw8<T> v = r;
    if (!in) v.zero();
    return v;
  }
};
static __device__ const uint4 kZeroBlocks[3] = {};     // read where there is nothing to read
template <typename T>
struct Chunk<T, false> {
  static constexpr int kOut = 8 * sizeof(T) / 4, kPer = 16 / sizeof(T);     // words of a chunk, elements of a block
  uint32_t w[kOut + 4];
  const T* p;
  int valid;           // elements of the chunk that exist
  bool whole;          // its blocks were read
  __device__ __forceinline__ void fetch(const Source<T>& m, const T* row, int first, int cols) {
    p = row + first;
    valid = cols - first;
    const int before = static_cast<int>((static_cast<uint32_t>(reinterpret_cast<uintptr_t>(p)) & 15u) / sizeof(T));
    const T* a = p - before;
    const int used = before + min(valid, 8);             // elements from the first block's start to the chunk's end
    whole = valid > 0 && a >= m.p && a + (used + kPer - 1) / kPer * kPer <= m.end;
#pragma unroll
    for (int i = 0; i < kOut / 4 + 1; ++i) {
      // (a block without an element of the chunk is not read: behind the row there may be nothing)
      const uint4 t = *(whole && i * kPer < used ? reinterpret_cast<const uint4*>(a) + i : kZeroBlocks + i);
      w[4 * i] = t.x; w[4 * i + 1] = t.y; w[4 * i + 2] = t.z; w[4 * i + 3] = t.w;
    }
  }
  __device__ __forceinline__ Raw8<T> raw(bool) const {
    Raw8<T> r;
    uint32_t v[kOut + 4];
#pragma unroll
    for (int i = 0; i < kOut + 4; ++i) v[i] = w[i];
    shift_window<kOut, sizeof(T) == 2>(v, static_cast<uint32_t>(reinterpret_cast<uintptr_t>(p)) & 15u);
    r.from_words(v);
    if (valid < 8 && valid > 0 && whole) {               // the row ends within the chunk
      float f[8];
      r.get(f);
#pragma unroll
      for (int j = 0; j < 8; ++j) f[j] = j < valid ? f[j] : 0.f;
      r.put(f);
    }
    if (valid > 0 && !whole) r = load_some(p, valid);
    return r;
  }
};

// The reverse.  All 32 lanes call (not VEC: neighbours complete each other's blocks); `live`: there is something to
// store; `prev` / `next`: the lane below / above holds the chunk in front / behind, of the same row and live too.
template <typename T, bool VEC>
__device__ __forceinline__ void store_chunk(T* row, int first, int cols, const Raw8<T>& r, bool live, bool prev, bool next) {
  if constexpr (VEC) {
    if (live && first < cols) r.store(row + first);
  } else {
    constexpr int kOut = 8 * sizeof(T) / 4, kPer = 16 / sizeof(T);
    uint32_t w[kOut + 4];
    uint32_t own[kOut];
    r.to_words(own);
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = __shfl_up_sync(0xffffffffu, own[kOut - 4 + i], 1);
#pragma unroll
    for (int i = 0; i < kOut; ++i) w[4 + i] = own[i];
    T* p = row + first;
    const int valid = cols - first;
    if (!live || valid <= 0) return;
    const uint32_t s = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(p)) & 15u;
    const int before = static_cast<int>(s / sizeof(T));
    float v[8];
    r.get(v);
    if (valid < 8) {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (j < valid) p[j] = from_float<T>(v[j]);
      return;
    }
    if (s == 0) {
      r.store(p);
      return;
    }
    // the blocks that end in this chunk; the first of them begins in the chunk in front
    shift_window<kOut, sizeof(T) == 2>(w, 16 - s);
    uint4* block = reinterpret_cast<uint4*>(p - before);
    if (prev) {
      block[0] = make_uint4(w[0], w[1], w[2], w[3]);
    } else {
#pragma unroll
      for (int j = 0; j < kPer; ++j)
        if (j < kPer - before) p[j] = from_float<T>(v[j]);
    }
    if constexpr (sizeof(T) == 4) block[1] = make_uint4(w[4], w[5], w[6], w[7]);
    // its last elements belong to a block of the chunk behind, if that one is whole
    if (!(next && valid >= 16)) {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (j >= 8 - before) p[j] = from_float<T>(v[j]);
    }
  }
}

// Parameter vectors (weight, bias): type known at run time, one element at a time or 16 bytes at once.
struct ParamVec {
  const void* p;       // null: the constant `none`
  int is_bf16;
  int vec;             // starts on a 16-byte boundary
};
__device__ __forceinline__ void load_param(const ParamVec& w, int first, int cols, float none, float (&v)[8]) {
  if (w.p && w.vec && first + 8 <= cols) {
    if (w.is_bf16) { Raw8<bf16> r; r.load(static_cast<const bf16*>(w.p) + first); r.get(v); }
    else { Raw8<float> r; r.load(static_cast<const float*>(w.p) + first); r.get(v); }
    return;
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const int at = first + j;
    v[j] = none;
    if (w.p && at < cols)
      v[j] = w.is_bf16 ? to_float(static_cast<const bf16*>(w.p)[at]) : static_cast<const float*>(w.p)[at];
  }
}

// ---- encode
__device__ __forceinline__ uint32_t act8_scale_byte(uint32_t amax_bits) {
  // 127 * 2^e = 1.984375 * 2^(e+6): adding 2^17 - 1 carries into the exponent when the mantissa is above that
  const uint32_t k = (amax_bits + 0x1FFFFu) >> 23;
  return amax_bits >= 0x7F800000u ? 255u : (k > 6u ? k - 6u : 0u);
}
__device__ __forceinline__ float act8_scale(uint32_t byte) {
  return byte == 255u ? __uint_as_float(0x7FC00000u) : byte == 0u ? __uint_as_float(0x00400000u) : __uint_as_float(byte << 23);
}

// rint(v * 2^-e) as an int8 in the low byte (1.5 * 2^23 puts it there; the product is exact)
__device__ __forceinline__ uint32_t act8_code(float v, float inv) { return __float_as_uint(fmaf(v, inv, 12582912.f)); }
__device__ __forceinline__ float act8_inverse(uint32_t byte) { return __uint_as_float((254u - byte) << 23); }
// Codes at e = 122 end at +-63 (64 * 2^122 is no float): the value cut to that.
__device__ __forceinline__ float act8_cut(float v) {
  const float top = 63.f * 5.316911983139664e36f;     // 63 * 2^122
  return fminf(fmaxf(v, -top), top);
}

// One chunk of values as they stand in memory (zeros past the row's end) into a checkpoint; the group lies across an
// aligned quad of lanes.  All 32 lanes call; `codes` and `scales` point at the chunk's codes and the group's scale.
// `keep`: the chunk belongs to a row and a group; `pad`: bytes of padding behind the row's last scale, for its lane.
template <typename T>
__device__ __forceinline__ void act8_put(uint8_t* codes, uint8_t* scales, const Raw8<T>& raw, bool first_of_group, int pad,
                                         bool keep) {
  uint32_t m = raw.top();
  m = max(m, __shfl_xor_sync(0xffffffffu, m, 1));
  m = max(m, __shfl_xor_sync(0xffffffffu, m, 2));
  const uint32_t byte = act8_scale_byte(m);
  const float inv = act8_inverse(byte);
  F2 v[4];
  raw.get(v);
  uint32_t q[8];
  const F2 inv2 = two(inv), magic = two(12582912.f);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float lo, hi;
    apart(fma2(v[i], inv2, magic), &lo, &hi);
    q[2 * i] = __float_as_uint(lo);
    q[2 * i + 1] = __float_as_uint(hi);
  }
  if (byte == 249u) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float lo, hi;
      apart(v[i], &lo, &hi);
      q[2 * i] = act8_code(act8_cut(lo), inv);
      q[2 * i + 1] = act8_code(act8_cut(hi), inv);
    }
  }
  uint2 r;
  r.x = __byte_perm(__byte_perm(q[0], q[1], 0x0040), __byte_perm(q[2], q[3], 0x0040), 0x5410);
  r.y = __byte_perm(__byte_perm(q[4], q[5], 0x0040), __byte_perm(q[6], q[7], 0x0040), 0x5410);
  if (byte == 255u) r = make_uint2(0, 0);
  if (!keep) return;
  *reinterpret_cast<uint2*>(codes) = r;
  if (first_of_group) {
    *scales = static_cast<uint8_t>(byte);
    for (int i = 1; i <= pad; ++i) scales[i] = 0;
  }
}

// ---- decode
// A chunk's codes and its group's scale as they lie in memory; the first chunk's if it is not `inside`.
struct RawAct8 {
  uint2 q;
  uint32_t byte;
  __device__ __forceinline__ void load(const Act8& ck, long long code, long long scale, bool inside) {
    q = *reinterpret_cast<const uint2*>(ck.codes + (inside ? code : 0));
    byte = ck.scales[inside ? scale : 0];
  }
  __device__ __forceinline__ void get(F2 (&v)[4]) const {
    const F2 s = two(act8_scale(byte)), off = two(-8388736.f);
    const uint32_t a = q.x ^ 0x80808080u, b = q.y ^ 0x80808080u;   // code + 128 as an unsigned byte
    // 2^23 + (code + 128) by its bits, minus the offset: exact
    auto spread = [](uint32_t w, int i) { return __uint_as_float(__byte_perm(w, 0x4B000000u, 0x7440 + i)); };
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      v[i] = mul2(add2(two(spread(a, 2 * i), spread(a, 2 * i + 1)), off), s);
      v[2 + i] = mul2(add2(two(spread(b, 2 * i), spread(b, 2 * i + 1)), off), s);
    }
  }
};
// ---- division by a number fixed per launch, for 0 <= n < 2^31
struct FastDiv {
  uint32_t d, mul, shift;
  explicit FastDiv(uint32_t div = 1) : d(div), mul(0), shift(0) {
    while ((1ull << shift) < div) ++shift;
    // m = floor(2^32 (2^shift - d) / d) + 1;  n / d = (umulhi(n, m) + n) >> shift
    mul = static_cast<uint32_t>(((1ull << 32) * ((1ull << shift) - div)) / div + 1);
  }
  __device__ __forceinline__ uint32_t div(uint32_t n) const {
    return static_cast<uint32_t>((static_cast<uint64_t>(__umulhi(n, mul)) + n) >> shift);
  }
};

}  // namespace fa
