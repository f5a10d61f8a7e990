// Device helpers of the row operators: 8-element vectors of a row (16 bytes of bf16, 32 of fp32) and the 8-bit
// checkpoint format.
//
// Format: per row, groups of 128 columns (the last one may be shorter) share one binary32 scale.  With a = max |x| of
// the group,
//     scale = a * (1 / 127),   code = rint(x * (127 * (1 / a))),
// (the scale at most kMaxScale, so that 127 codes of the largest finite a do not overflow when they are read back), every
// step one binary32 operation rounded to nearest even (1 / 127 the rounded constant), so that the codes are a function of
// the input alone and any two implementations agree on every bit.  (They are products with rounded reciprocals, as torch takes
// x / 127.0 and 127.0 / x on the GPU too; quotients differ in the last bit of one scale in twenty, and in the code of a value
// half way between two.)  a < 2^-100: the group is stored as zeros (1 / a would overflow on its
// way through the subnormals).  An infinity or a NaN in the group: scale = NaN, the group reads back as NaN.
#pragma once
#include <cuda_bf16.h>
#include <cstdint>

namespace acx {
namespace q8 {

constexpr int kGroup = 128;            // columns that share a scale
constexpr int kVec = 8;                // columns a thread handles at a time
constexpr uint32_t kTinyBits = (127u - 100u) << 23;   // 2^-100
constexpr uint32_t kInfBits = 0x7F800000u, kNanBits = 0x7FFFFFFFu;
constexpr float kMaxScale = 0x1.020406p+121f;   // the largest float whose 127-fold is finite

// Two binary32 operations per instruction, each rounded to nearest even on its own.
__device__ __forceinline__ uint64_t bits2(float2 a) { return (uint64_t(__float_as_uint(a.y)) << 32) | __float_as_uint(a.x); }
__device__ __forceinline__ float2 float2_of(uint64_t b) { return make_float2(__uint_as_float(uint32_t(b)), __uint_as_float(uint32_t(b >> 32))); }
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(bits2(a)), "l"(bits2(b)));
  return float2_of(r);
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(bits2(a)), "l"(bits2(b)));
  return float2_of(r);
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(bits2(a)), "l"(bits2(b)), "l"(bits2(c)));
  return float2_of(r);
}
__device__ __forceinline__ float2 both(float x) { return make_float2(x, x); }

// Loads go through L2 (ld.global.cg), not through the read-only path: a kernel that was launched while the one before it was
// still running may not assume that memory has not changed since its own start.
//
// Eight elements of a row as they are in memory: loads are issued long before the values are needed, and a bf16 vector
// waits for that in four registers instead of eight.
template <typename T>
struct Raw;
template <>
struct Raw<__nv_bfloat16> {
  uint4 u;
  __device__ __forceinline__ void zero() { u = make_uint4(0u, 0u, 0u, 0u); }
  __device__ __forceinline__ void load(const __nv_bfloat16* p) { u = __ldcg(reinterpret_cast<const uint4*>(p)); }
  __device__ __forceinline__ void get(float2 (&v)[4]) const {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = make_float2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xFFFF0000u));
  }
  // Largest magnitude, as the bits of a binary32; a NaN wins over everything.
  __device__ __forceinline__ uint32_t amax_bits() const {
    const uint32_t a = max16x2(max16x2(u.x & 0x7FFF7FFFu, u.y & 0x7FFF7FFFu), max16x2(u.z & 0x7FFF7FFFu, u.w & 0x7FFF7FFFu));
    return max(a << 16, a & 0xFFFF0000u);
  }
  // Both halves' maxima of two pairs of non-negative bf16 values (a NaN wins)
  static __device__ __forceinline__ uint32_t max16x2(uint32_t a, uint32_t b) {
    const __nv_bfloat162 m = __hmax2_nan(*reinterpret_cast<const __nv_bfloat162*>(&a), *reinterpret_cast<const __nv_bfloat162*>(&b));
    return *reinterpret_cast<const uint32_t*>(&m);
  }
};
template <>
struct Raw<float> {
  float4 a, b;
  __device__ __forceinline__ void zero() { a = b = make_float4(0.f, 0.f, 0.f, 0.f); }
  __device__ __forceinline__ void load(const float* p) {
    a = __ldcg(reinterpret_cast<const float4*>(p));
    b = __ldcg(reinterpret_cast<const float4*>(p) + 1);
  }
  __device__ __forceinline__ void get(float2 (&v)[4]) const {
    v[0] = make_float2(a.x, a.y); v[1] = make_float2(a.z, a.w);
    v[2] = make_float2(b.x, b.y); v[3] = make_float2(b.z, b.w);
  }
  // Integer order is the order of magnitudes, with infinity and then NaN on top.
  __device__ __forceinline__ uint32_t amax_bits() const {
    const float v[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(v[i]) & 0x7FFFFFFFu);
    return m;
  }
};

template <typename T>
__device__ __forceinline__ void load8(const T* p, float2 (&v)[4]) {
  Raw<T> r;
  r.load(p);
  r.get(v);
}
__device__ __forceinline__ void store8(__nv_bfloat16* p, const float2 (&v)[4]) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(v[i].x, v[i].y);
    w[i] = *reinterpret_cast<const uint32_t*>(&h);
  }
  *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
}
// One store of 32 bytes where the address allows it (always, unless the matrix starts between two such boundaries): two of 16
// leave every 32-byte sector half written, twice (q8_load of 16384 x 4096: 65 us, 51 us with one; the backward of the gated
// activation of 4096 x 8192: 81 and 72 us).  Loads stay two of 16: as one of 32 they were 3 to 8 % slower in large matrices.
__device__ __forceinline__ void store8(float* p, const float2 (&v)[4]) {
  asm volatile(
      "{\n\t.reg .pred w;\n\t.reg .b64 m;\n\tand.b64 m, %8, 31;\n\tsetp.eq.s64 w, m, 0;\n\t"
      "@w st.global.v8.f32 [%8], {%0, %1, %2, %3, %4, %5, %6, %7};\n\t"
      "@!w st.global.v4.f32 [%8], {%0, %1, %2, %3};\n\t"
      "@!w st.global.v4.f32 [%8 + 16], {%4, %5, %6, %7};\n\t}" ::"f"(v[0].x),
      "f"(v[0].y), "f"(v[1].x), "f"(v[1].y), "f"(v[2].x), "f"(v[2].y), "f"(v[3].x), "f"(v[3].y), "l"(p)
      : "memory");
}

// Largest of a value over LANES consecutive lanes (a power of two).  All lanes of the warp take part.
template <int LANES>
__device__ __forceinline__ uint32_t max_over(uint32_t m) {
#pragma unroll
  for (int o = LANES / 2; o > 0; o >>= 1) m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, o));
  return m;
}

// The same for two values at a time; those of bf16 elements have 16 bits and travel together.
template <typename T, int LANES>
__device__ __forceinline__ void max_pair_over(uint32_t& a, uint32_t& b) {
  if (sizeof(T) == 2) {
    uint32_t m = a | (b >> 16);
#pragma unroll
    for (int o = LANES / 2; o > 0; o >>= 1) m = Raw<__nv_bfloat16>::max16x2(m, __shfl_xor_sync(0xFFFFFFFFu, m, o));
    a = m & 0xFFFF0000u;
    b = m << 16;
  } else {
    a = max_over<LANES>(a);
    b = max_over<LANES>(b);
  }
}

struct GroupScale { float scale, inv; };
__device__ __forceinline__ GroupScale group_scale(uint32_t amax_bits) {
  const float a = __uint_as_float(amax_bits);
  GroupScale g;
  if (amax_bits >= kInfBits) { g.scale = __uint_as_float(kNanBits); g.inv = 0.f; }
  else if (amax_bits < kTinyBits) { g.scale = 0.f; g.inv = 0.f; }
  else { g.scale = fminf(__fmul_rn(a, 1.f / 127.f), kMaxScale); g.inv = __fmul_rn(127.f, __frcp_rn(a)); }
  return g;
}

// Eight codes as two words.  Adding 1.5 * 2^23 rounds a value of magnitude <= 2^22 to a whole number (nearest, ties to
// even) and leaves its two's complement in the low bits of the sum's mantissa: one addition and a byte permutation
// instead of a conversion, whose rate is a quarter.  The product and the sum are rounded separately (no fma), as the
// format says (the additions one at a time: the assembler fuses the two-at-a-time forms of both into one rounding).  A NaN product (0 * inf in a group whose scale is NaN) leaves some byte: it is read back times NaN.
__device__ __forceinline__ uint2 encode8(const float2 (&v)[4], float inv) {
  uint32_t b[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 q = mul2(v[i], both(inv));
    b[2 * i] = __float_as_uint(__fadd_rn(q.x, 12582912.f));
    b[2 * i + 1] = __float_as_uint(__fadd_rn(q.y, 12582912.f));
  }
  uint2 c;
  c.x = __byte_perm(__byte_perm(b[0], b[1], 0x0040), __byte_perm(b[2], b[3], 0x0040), 0x5410);
  c.y = __byte_perm(__byte_perm(b[4], b[5], 0x0040), __byte_perm(b[6], b[7], 0x0040), 0x5410);
  return c;
}

// The values of eight codes.  A byte with its sign bit flipped is code + 128; placed into the mantissa of 2^23 it is the
// float 2^23 + 128 + code, exactly.
__device__ __forceinline__ void decode8(uint2 c, float scale, float2 (&v)[4]) {
  const uint32_t w[2] = {c.x ^ 0x80808080u, c.y ^ 0x80808080u};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t lo = __byte_perm(w[i >> 1], 0x4B000000u, 0x7650 + 2 * (i & 1));   // bytes: 4B 00 00 code
    const uint32_t hi = __byte_perm(w[i >> 1], 0x4B000000u, 0x7651 + 2 * (i & 1));
    v[i] = mul2(add2(make_float2(__uint_as_float(lo), __uint_as_float(hi)), both(-8388736.f)), both(scale));
  }
}

}  // namespace q8
}  // namespace acx
