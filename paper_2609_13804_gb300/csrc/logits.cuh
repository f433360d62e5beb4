// Rows of logits: their 16-byte pieces, running maxima and sums of exponentials, packed fp32 arithmetic.
#pragma once
#include "common.cuh"

namespace sp {

constexpr float kLog2e = 1.44269504088896341f;

SP_DEVINL float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

SP_DEVINL float rcp(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// Running max and sum of exponentials; +infinity counts its occurrences (the limit of the softmax).
struct MaxSum {
  float m, s;
  SP_DEVINL void add(float m2, float s2) {
    const float mn = fmaxf(m, m2);
    if (mn == -INFINITY) return;
    s = (m == mn ? s : s * ex2((m - mn) * kLog2e)) + (m2 == mn ? s2 : s2 * ex2((m2 - mn) * kLog2e));
    m = mn;
  }
};

template <bool F32>
struct Chunk;  // 16 bytes of logits
template <>
struct Chunk<true> {
  static constexpr int N = 4;
  static constexpr uint32_t kNone = 0xff800000u;  // a word of -infinity
  SP_DEVINL static float at(const uint4& u, int k) {
    return __uint_as_float(k == 0 ? u.x : k == 1 ? u.y : k == 2 ? u.z : u.w);
  }
  SP_DEVINL static float top(const uint4& u) {  // (fmaxf passes over NaN)
    return fmaxf(fmaxf(__uint_as_float(u.x), __uint_as_float(u.y)), fmaxf(__uint_as_float(u.z), __uint_as_float(u.w)));
  }
  SP_DEVINL static float one(const void* row, int v) { return __ldg(static_cast<const float*>(row) + v); }
};
template <>
struct Chunk<false> {
  static constexpr int N = 8;
  static constexpr uint32_t kNone = 0xff80ff80u;
  SP_DEVINL static float at(const uint4& u, int k) {
    const uint32_t w = k < 2 ? u.x : k < 4 ? u.y : k < 6 ? u.z : u.w;
    return __uint_as_float((k & 1) ? (w & 0xffff0000u) : (w << 16));
  }
  SP_DEVINL static float top(const uint4& u) {
    const __nv_bfloat162* h = reinterpret_cast<const __nv_bfloat162*>(&u);
    const __nv_bfloat162 m = __hmax2(__hmax2(h[0], h[1]), __hmax2(h[2], h[3]));  // (NaN passed over)
    return fmaxf(__low2float(m), __high2float(m));
  }
  SP_DEVINL static float one(const void* row, int v) {
    return __bfloat162float(static_cast<const __nv_bfloat16*>(row)[v]);
  }
};

// 16 bytes of logits with -infinity for NaN.
template <bool F32>
SP_DEVINL uint4 without_nan(const uint4& u) {
  auto f = [](uint32_t x) -> uint32_t {
    if (F32) return __float_as_uint(fmaxf(__uint_as_float(x), -INFINITY));
    const __nv_bfloat162 m = __hmax2(*reinterpret_cast<const __nv_bfloat162*>(&x), __float2bfloat162_rn(-INFINITY));
    return *reinterpret_cast<const uint32_t*>(&m);
  };
  return make_uint4(f(u.x), f(u.y), f(u.z), f(u.w));
}

// Four logits, which go with 16 bytes of fp32 numbers of the same tokens: a warp's loads of both are contiguous.
template <bool F32>
struct Four;
template <>
struct Four<true> {
  using T = uint4;
  static constexpr int kBytes = 16;
  SP_DEVINL static T none() { return make_uint4(0xff800000u, 0xff800000u, 0xff800000u, 0xff800000u); }
  SP_DEVINL static float at(const T& u, int k) { return Chunk<true>::at(u, k); }
  SP_DEVINL static float top(const T& u) { return Chunk<true>::top(u); }
};
template <>
struct Four<false> {
  using T = uint2;
  static constexpr int kBytes = 8;
  SP_DEVINL static T none() { return make_uint2(0xff80ff80u, 0xff80ff80u); }
  SP_DEVINL static float at(const T& u, int k) {
    const uint32_t w = k < 2 ? u.x : u.y;
    return __uint_as_float((k & 1) ? (w & 0xffff0000u) : (w << 16));
  }
  SP_DEVINL static __nv_bfloat162 pair(uint32_t w) { return *reinterpret_cast<__nv_bfloat162*>(&w); }
  SP_DEVINL static float top(const T& u) {
    const __nv_bfloat162 m = __hmax2(pair(u.x), pair(u.y));
    return fmaxf(__low2float(m), __high2float(m));
  }
};

// Two fp32 numbers as one operand of Blackwell's packed arithmetic
SP_DEVINL unsigned long long pack2(float lo, float hi) {
  unsigned long long r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
  return r;
}
SP_DEVINL void unpack2(unsigned long long v, float& lo, float& hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v)); }
SP_DEVINL unsigned long long add2(unsigned long long a, unsigned long long b) {
  unsigned long long r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
SP_DEVINL unsigned long long mul2(unsigned long long a, unsigned long long b) {
  unsigned long long r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}

}  // namespace sp
