// Rows of fp32 or 16-bit elements eight at a time, and sums over a row's waves:
// shared by the kernels that work on whole rows. Included INSIDE an unnamed
// namespace in ac, after hip_runtime.h and adaptcore.h.

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// Eight elements of type T (adaptcore_type) as they are stored.
template <int T>
struct Chunk {
  u32x4 v[T == AC_TYPE_F32 ? 2 : 1];
};
constexpr int elem_bytes(int t) { return t == AC_TYPE_F32 ? 4 : 2; }

template <int T>
__device__ __forceinline__ float elem(const void* p, int64_t i) {
  if constexpr (T == AC_TYPE_F32) return static_cast<const float*>(p)[i];
  const uint16_t h = static_cast<const uint16_t*>(p)[i];
  if constexpr (T == AC_TYPE_F16) return (float)__builtin_bit_cast(_Float16, h);
  return __uint_as_float((uint32_t)h << 16);
}
template <int T>
__device__ __forceinline__ void put(void* p, int64_t i, float f) {
  if constexpr (T == AC_TYPE_F32)
    static_cast<float*>(p)[i] = f;
  else if constexpr (T == AC_TYPE_F16)
    static_cast<uint16_t*>(p)[i] = __builtin_bit_cast(uint16_t, (_Float16)f);
  else
    static_cast<uint16_t*>(p)[i] = __builtin_bit_cast(uint16_t, (__bf16)f);
}

// Elements c .. c+7 of a row of n: whole chunks with 16-byte loads at any
// alignment of the element, the row's last partial one element by element.
template <int T>
__device__ __forceinline__ Chunk<T> load8(const void* row, int c, int n) {
  Chunk<T> r = {};
  const char* p = static_cast<const char*>(row) + (int64_t)c * elem_bytes(T);
  if (c + 8 <= n) {
    __builtin_memcpy(&r, p, sizeof r);
  } else if (c < n) {
    uint32_t h[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      h[e] = 0;
      if (c + e < n) {
        if constexpr (T == AC_TYPE_F32)
          h[e] = reinterpret_cast<const uint32_t*>(p)[e];
        else
          h[e] = reinterpret_cast<const uint16_t*>(p)[e];
      }
    }
    if constexpr (T == AC_TYPE_F32) {
      r.v[0] = u32x4{h[0], h[1], h[2], h[3]};
      r.v[1] = u32x4{h[4], h[5], h[6], h[7]};
    } else {
      r.v[0] = u32x4{h[0] | (h[1] << 16), h[2] | (h[3] << 16), h[4] | (h[5] << 16), h[6] | (h[7] << 16)};
    }
  }
  return r;
}
template <int T>
__device__ __forceinline__ void unpack(const Chunk<T>& r, float (&f)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    if constexpr (T == AC_TYPE_F32)
      f[e] = __uint_as_float(r.v[e >> 2][e & 3]);
    else if constexpr (T == AC_TYPE_F16)
      f[e] = (float)__builtin_bit_cast(_Float16, (uint16_t)(r.v[0][e >> 1] >> (16 * (e & 1))));
    else
      f[e] = __uint_as_float((e & 1) ? r.v[0][e >> 1] & 0xFFFF0000u : r.v[0][e >> 1] << 16);
  }
}
template <int T>
__device__ __forceinline__ void store8(void* row, int c, int n, const float (&f)[8]) {
  if (c + 8 <= n) {
    Chunk<T> r;
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
      if constexpr (T == AC_TYPE_F32) {
        r.v[e >> 2][e & 3] = __float_as_uint(f[e]);
        r.v[e >> 2][(e & 3) + 1] = __float_as_uint(f[e + 1]);
      } else if constexpr (T == AC_TYPE_F16) {
        r.v[0][e >> 1] = (uint32_t)__builtin_bit_cast(uint16_t, (_Float16)f[e]) |
                         ((uint32_t)__builtin_bit_cast(uint16_t, (_Float16)f[e + 1]) << 16);
      } else {
        r.v[0][e >> 1] = (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)f[e]) |
                         ((uint32_t)__builtin_bit_cast(uint16_t, (__bf16)f[e + 1]) << 16);
      }
    }
    __builtin_memcpy(static_cast<char*>(row) + (int64_t)c * elem_bytes(T), &r, sizeof r);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (c + e < n) put<T>(row, c + e, f[e]);
  }
}

// A lane's chunk of a row of n >= 8: the 8 elements from `at` on, of which the
// first `skip` are another lane's (8: all, nothing is loaded).
struct Span {
  int at, skip;
  __device__ __forceinline__ Span(int c, int n) {
    at = min(c, n - 8);
    skip = min(c - at, 8);
  }
};
template <int T>
__device__ __forceinline__ Chunk<T> load_span(const void* row, const Span& s) {
  Chunk<T> r = {};
  if (s.skip < 8) __builtin_memcpy(&r, static_cast<const char*>(row) + (int64_t)s.at * elem_bytes(T), sizeof r);
  return r;
}
template <int T>
__device__ __forceinline__ void store_span(void* row, const Span& s, const float (&f)[8]) {
  if (s.skip < 8) store8<T>(row, s.at, s.at + 8, f);
}

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int m = 32; m >= 1; m >>= 1) v += __shfl_xor(v, m, 64);
  return v;
}

// Sums of a and b over the WPR waves of a row. With WPR > 1 the row's waves
// are the workgroup, and `box` (2 x WPR x 2 floats) alternates between its two
// halves, so that one barrier a reduction is enough: a wave writes a half again
// only after the barrier of the reduction between.
template <int WPR>
__device__ __forceinline__ void row_sum2(float& a, float& b, float* box, int& phase) {
  a = wave_sum(a);
  b = wave_sum(b);
  if constexpr (WPR > 1) {
    float* half = box + phase * (2 * WPR);
    phase ^= 1;
    const int w = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0) {
      half[2 * w] = a;
      half[2 * w + 1] = b;
    }
    __syncthreads();
    a = b = 0.f;
#pragma unroll
    for (int i = 0; i < WPR; ++i) {
      a += half[2 * i];
      b += half[2 * i + 1];
    }
  }
}
