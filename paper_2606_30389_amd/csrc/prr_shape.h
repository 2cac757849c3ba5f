// Scores with a shape: which keys a token sees, a cap on its logits, a bias that falls with the distance.  The part up to
// the cap needs only int32_t, min and max, so that it can be compiled for the CPU too.
#pragma once

namespace prr {

// What a kernel's instance applies (bits).
constexpr int kShapeSpan = 1, kShapeCap = 2, kShapeSlopes = 4;

struct ShapeArgs {
  const float* slopes;
  const int32_t* prefix;
  const int32_t* first;
  int window;
  float cap, inv, small;  // the cap in the units of q.k, 1 / cap, the logits below which cap_small holds
};

// Keys [lo, hi) of a sequence of kv tokens that the token at position pos (row `row` of the packed tensors) sees; lo = hi:
// none.  pos < kv; 0 <= lo <= hi <= kv whatever the device arrays hold.
struct Span {
  int lo, hi;
};
__device__ __forceinline__ Span span_of(const ShapeArgs& a, int pos, int row, int s, int kv) {
  Span r;
  if (pos < 0) {
    r.lo = r.hi = 0;
    return r;
  }
  r.lo = a.window ? max(pos - a.window + 1, 0) : 0;
  if (a.first) r.lo = max(r.lo, a.first[row]);
  r.hi = pos + 1;
  if (a.prefix) r.hi = min(max(r.hi, a.prefix[s]), kv);
  r.lo = min(r.lo, r.hi);
  return r;
}

#ifdef __HIPCC__

// Logits are held as q.k: a logit's cap and slopes in that unit.
constexpr float kRawPerLogit = 11.313708498984761f;  // sqrt(128)

// cap tanh(s / cap), s in the units of q.k.  Below half the cap: s P((s / cap)^2), P the polynomial of degree 4 closest to
// tanh(x) / x up to 1/2 (least squares with weights moved until the relative error was level): 2^-26 relative before
// rounding, 2^-23 with it.  Seven operations where the other form needs an exponential and a reciprocal, each
// a quarter of an operation's rate.
__device__ __forceinline__ float cap_small(float s, const ShapeArgs& a) {
  const float x = s * a.inv, u = x * x;
  float p = 0.017135007306933403f;
  p = fmaf(p, u, -0.05298607423901558f);
  p = fmaf(p, u, 0.13324779272079468f);
  p = fmaf(p, u, -0.3333306908607483f);
  p = fmaf(p, u, 1.0f);
  return s * p;
}
// Any s: cap (1 - 2 / (1 + e^(2 s / cap))), off by at most cap * 2^-22 (the reciprocal's and the sum's last places);
// infinities give the cap, NaN stays NaN.
__device__ __forceinline__ float cap_large(float s, const ShapeArgs& a) {
  const float e = __builtin_amdgcn_exp2f(s * a.inv * (2.0f * kLog2e));
  return fmaf(-2.0f * a.cap, __builtin_amdgcn_rcpf(1.0f + e), a.cap);
}
__device__ __forceinline__ float cap_any(float s, const ShapeArgs& a) {
  return fabsf(s) < a.small ? cap_small(s, a) : cap_large(s, a);
}

#endif

}  // namespace prr
