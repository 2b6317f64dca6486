// Sums as pairs of fp32, hi + lo, the error of every addition carried along: good to
// 2^-46 or better, and quicker here than fp64 (the error-free sum of Knuth, TAOCP vol. 2,
// 4.2.2, and Dekker's renormalisation, Numer. Math. 18, 1971).
#pragma once

#include "common.cuh"

namespace fpk {

struct Pair {
  float hi, lo;
};
// a + b, exactly
FP_DEV Pair sum2(float a, float b) {
  const float s = __fadd_rn(a, b), v = __fsub_rn(s, a);
  return {s, __fadd_rn(__fsub_rn(a, __fsub_rn(s, v)), __fsub_rn(b, v))};
}
// hi + lo with hi the nearer fp32 (|hi| >= |lo|)
FP_DEV Pair tidy(float hi, float lo) {
  const float s = __fadd_rn(hi, lo);
  return {s, __fsub_rn(lo, __fsub_rn(s, hi))};
}
FP_DEV Pair add(Pair a, Pair b) {
  const Pair s = sum2(a.hi, b.hi);
  return tidy(s.hi, __fadd_rn(s.lo, __fadd_rn(a.lo, b.lo)));
}
FP_DEV Pair times(Pair a, float r) {
  const float h = __fmul_rn(a.hi, r);
  return tidy(h, __fmaf_rn(a.lo, r, __fmaf_rn(a.hi, r, -h)));
}
FP_DEV bool greater(Pair a, Pair b) {
  const Pair d = sum2(a.hi, -b.hi);
  return __fadd_rn(d.hi, __fadd_rn(d.lo, __fsub_rn(a.lo, b.lo))) > 0.f;
}
// r of a whole sum, 0 <= r < 1, and whether a running sum is past it.  The product's error is as
// small as 2^-48 of it, so both sides are taken times 2^96 where it could underflow (sums of
// weights near the least fp32).
struct Border {
  Pair at;
  float by;
};
FP_DEV Border border_at(Pair total, float r) {
  const float by = total.hi < 0x1p20f ? 0x1p96f : 1.f;
  return {times(Pair{total.hi * by, total.lo * by}, r), by};
}
FP_DEV bool past(Pair upto, Border b) { return greater(Pair{upto.hi * b.by, upto.lo * b.by}, b.at); }
FP_DEV Pair shfl(Pair v, int l) { return {__shfl_sync(0xffffffffu, v.hi, l), __shfl_sync(0xffffffffu, v.lo, l)}; }

// Two fp32 lanes at once: a + b, a b + c.
FP_DEV float2 fp_add2(float2 a, float2 b) {
  float2 d;
  asm("{\n .reg .b64 a, b, d;\n mov.b64 a, {%2, %3};\n mov.b64 b, {%4, %5};\n add.rn.f32x2 d, a, b;\n"
      " mov.b64 {%0, %1}, d;\n}\n"
      : "=f"(d.x), "=f"(d.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return d;
}
FP_DEV float2 fp_fma2(float2 a, float2 b, float2 c) {
  float2 d;
  asm("{\n .reg .b64 a, b, c, d;\n mov.b64 a, {%2, %3};\n mov.b64 b, {%4, %5};\n mov.b64 c, {%6, %7};\n"
      " fma.rn.f32x2 d, a, b, c;\n mov.b64 {%0, %1}, d;\n}\n"
      : "=f"(d.x), "=f"(d.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
  return d;
}

// Inclusive sums over groups of N lanes, lower lanes first.
template <int N>
FP_DEV Pair scan(Pair v, int lane) {
#pragma unroll
  for (int o = 1; o < N; o <<= 1) {
    const Pair f = {__shfl_up_sync(0xffffffffu, v.hi, o, N), __shfl_up_sync(0xffffffffu, v.lo, o, N)};
    if ((lane & (N - 1)) >= o) v = add(f, v);
  }
  return v;
}

}  // namespace fpk
