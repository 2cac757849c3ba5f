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
  float k[4], k2[4];      // cap_small's coefficients, and in the units of the exponent
  bool wide;              // a cap above kMostCap: cap_wide, in the instances with slopes
};

// Keys [lo, hi) of a sequence of kv tokens that the token at position pos (row `row` of the packed tensors) sees; lo = hi:
// none.  pos < kv; 0 <= lo <= hi <= kv whatever the device arrays hold.
struct Span {
  int lo, hi;
};
// first: where the row's document begins; prefix: the tokens of the sequence's prefix
__device__ __forceinline__ Span span_at(int window, int first, int prefix, int pos, int kv) {
  Span r;
  if (pos < 0) {
    r.lo = r.hi = 0;
    return r;
  }
  r.lo = max(window ? max(pos - window + 1, 0) : 0, first);
  r.hi = min(max(pos + 1, prefix), kv);
  r.lo = min(r.lo, r.hi);
  return r;
}
__device__ __forceinline__ Span span_of(const ShapeArgs& a, int pos, int row, int s, int kv) {
  return span_at(a.window, a.first ? a.first[row] : 0, a.prefix ? a.prefix[s] : 0, pos, kv);
}

// P of cap_small: tanh(x) / x = 1 + t0 x^2 + t1 x^4 + ...
constexpr double kTanh[4] = {-0.33332597508690864, 0.133131166748644, -0.05221180747602632, 0.015612633936512193};
constexpr double kTanhRange = 0.6;
constexpr float kMostCap = 1024.0f;  // of cap_small: above it the last powers of 1 / cap leave float32's range

#ifdef __HIPCC__

// Logits are held as q.k: a logit's cap and slopes in that unit.
constexpr float kRawPerLogit = 11.313708498984761f;  // sqrt(128)

// A query head's slope; instances of caps and slopes serve caps above kMostCap without slopes, too.
template <int SHAPE>
__device__ __forceinline__ float slope_of(const ShapeArgs& a, int head) {
  if ((SHAPE & kShapeCap) && !a.slopes) return 0.0f;
  return a.slopes[head] * kRawPerLogit;
}

// cap tanh(s / cap), s in the units of q.k.  Below 0.6 of the cap: s P((s / cap)^2), P the polynomial of degree 4 closest to
// tanh(x) / x there (least squares with weights moved until the relative error was level): 2^-23.5 relative before
// rounding, 2^-22.4 with it.  k holds P's coefficients times powers of 1 / cap^2, so that s^2 is the argument: six operations
// where the other form needs an exponential and a reciprocal, too, each at half an operation's rate or less.  A tile
// whose logits are all below takes this form alone; in one of both kinds each logit takes its own, so that no result depends
// on the others' logits.  (Up to 1/2, tiles of both kinds are common: nine packed prompts with a cap of 30 and logits of
// standard deviation 4 took 266 us, 214 up to 0.7; degree 5, which that range needs, costs 32768 tokens with a cap
// of 50 another 4%.)
__device__ __forceinline__ float cap_ratio(float s, const float (&k)[4], float one) {
  const float u = s * s;
  return fmaf(fmaf(fmaf(fmaf(k[3], u, k[2]), u, k[1]), u, k[0]), u, one);
}
__device__ __forceinline__ float cap_small(float s, const ShapeArgs& a) { return s * cap_ratio(s, a.k, 1.0f); }
// Any s: cap (1 - 2 / (1 + e^(2 s / cap))); infinities give the cap, NaN stays NaN.  Above 0.6 of the cap, where alone it is
// used, off by less than cap * 2^-21: the argument's four roundings and the exponential's last place make 0.63 * 2^-22 of
// it, the sum's, the reciprocal's and the last one 0.6 * 2^-22.
__device__ __forceinline__ float cap_large(float s, const ShapeArgs& a) {
  const float e = __builtin_amdgcn_exp2f(s * a.inv * (2.0f * kLog2e));
  return fmaf(-2.0f * a.cap, __builtin_amdgcn_rcpf(1.0f + e), a.cap);
}
__device__ __forceinline__ float cap_any(float s, const ShapeArgs& a) {
  return fabsf(s) < a.small ? cap_small(s, a) : cap_large(s, a);
}

// Any s and cap: the polynomial's argument is (s / cap)^2, so that its coefficients need no powers of the cap, for one operation
// more.  Caps above kMostCap are rare: they run the instances with caps and slopes, those of caps alone stay without it.
__device__ __forceinline__ float cap_wide(float s, const ShapeArgs& a) {
  constexpr float k[4] = {(float)kTanh[0], (float)kTanh[1], (float)kTanh[2], (float)kTanh[3]};
  const float x = s * a.inv;
  return fabsf(x) < (float)kTanhRange ? s * cap_ratio(x, k, 1.0f) : cap_large(s, a);
}

// Where memory bounds the kernel: the function itself, to its last places.
__device__ __forceinline__ float cap_exact(float s, const ShapeArgs& a) { return a.cap * tanhf(s * a.inv); }

// Exponents of weights relative to ref: log2(e) z / sqrt(128) - ref of capped logits, with the change of units in k2, so that
// the product with s is the exponent's.  near: every logit of the caller's is below a.small.
__device__ __forceinline__ float cap_exponent(float s, float ref, float scale2, bool near, const ShapeArgs& a) {
  const float x = fmaf(s, cap_ratio(s, a.k2, scale2), -ref);
  if (near) return x;
  return fabsf(s) < a.small ? x : fmaf(cap_large(s, a), scale2, -ref);
}

#endif

}  // namespace prr
