// Activations (adaptcore_activation) and their derivatives, fp32. Included INSIDE
// an unnamed namespace, after hip_runtime.h and adaptcore.h.

// (the hardware's exponential and reciprocal: some units of 2^-24 and |x| 2^-24 of
// the value, against the 2^-12 or more of the 16-bit results; the exact forms are
// a dozen instructions more an element in epilogues that nothing overlaps)
__device__ __forceinline__ float sigmoid(float x) { return __builtin_amdgcn_rcpf(1.0f + __expf(-x)); }
constexpr float GELU_K = 0.7978845608028654f, GELU_A = 0.044715f;  // sqrt(2 / pi)
constexpr float SQRT_HALF = 0.7071067811865476f, INV_SQRT_2PI = 0.3989422804014327f;

__device__ __forceinline__ void act8(int kind, const float (&x)[8], float (&a)[8]) {
  if (kind == AC_ACT_SILU) {
#pragma unroll
    for (int e = 0; e < 8; ++e) a[e] = x[e] * sigmoid(x[e]);
  } else if (kind == AC_ACT_GELU) {
#pragma unroll
    for (int e = 0; e < 8; ++e) a[e] = 0.5f * x[e] * (1.0f + erff(x[e] * SQRT_HALF));
  } else {  // 0.5 (1 + tanh z) = sigmoid(2 z)
#pragma unroll
    for (int e = 0; e < 8; ++e) a[e] = x[e] * sigmoid(2.0f * GELU_K * x[e] * (1.0f + GELU_A * x[e] * x[e]));
  }
}
__device__ __forceinline__ float act1(int kind, float x) {
  if (kind == AC_ACT_SILU) return x * sigmoid(x);
  if (kind == AC_ACT_GELU) return 0.5f * x * (1.0f + erff(x * SQRT_HALF));
  return x * sigmoid(2.0f * GELU_K * x * (1.0f + GELU_A * x * x));
}
// the activation and its derivative
__device__ __forceinline__ void act8_grad(int kind, const float (&x)[8], float (&a)[8], float (&d)[8]) {
  if (kind == AC_ACT_SILU) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float s = sigmoid(x[e]);
      a[e] = x[e] * s;
      d[e] = s * (1.0f + x[e] * (1.0f - s));
    }
  } else if (kind == AC_ACT_GELU) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float c = 0.5f * (1.0f + erff(x[e] * SQRT_HALF));
      a[e] = x[e] * c;
      d[e] = c + x[e] * INV_SQRT_2PI * __expf(-0.5f * x[e] * x[e]);
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      // (bounded: the last factor must not be infinite where s (1 - s) is zero)
      const float x2 = fminf(x[e] * x[e], 1e30f), s = sigmoid(2.0f * GELU_K * x[e] * (1.0f + GELU_A * x2));
      a[e] = x[e] * s;
      d[e] = s + x[e] * s * (1.0f - s) * (2.0f * GELU_K * (1.0f + 3.0f * GELU_A * x2));
    }
  }
}
