// Activation checkpoints in 8 bits (gfx950).
//
// 32 neighbouring elements share a unit 2^e, the smallest power of two from 2^-126 on in
// which the largest of them rounds to at most 127; an element is the integer x / unit,
// rounded to nearest, ties to even.  2^121 is the largest unit (64 of the next one overflow
// fp32): there the last few values below 2^128 become 127 units.  e + 127 is kept in a byte;
// 255 marks a group with an infinity or a NaN, which comes back as 32 NaN.  Every step is
// exact but the one rounding (products with powers of two, and integers of 7 bits fit a
// bf16's 8), so the result depends on nothing but x, and an unpacked value is off by at most
// half a unit.  That is 2^-7 of the group's largest element or less, but for groups whose largest is
// below 64 units of 2^-126, which may be lost whole; and values above 127 units of 2^121 are off
// by up to one of them.
//
// Both directions move 16 elements to a thread (whole 16-byte pieces of the 8-bit side) and
// are bound by memory: [32768][32][128] bf16, 814 MB packed and unpacked again in 158 us,
// 5.1 TB/s, a large copy's rate.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "attn_common.h"
#include "ckpt8.h"
#include "errors.h"

namespace libra {

typedef int8_t i8x16 __attribute__((ext_vector_type(16)));
constexpr int kPer = 16;   // elements of a thread: half a group

// 16 elements of a row, bf16 or fp32.
__device__ __forceinline__ void load16(const bf16 *p, float (&x)[kPer]) {
  static_for<2>([&](auto h) {
    const bf16x8 v = *reinterpret_cast<const bf16x8 *>(p + 8 * h);
    static_for<8>([&](auto i) { x[8 * h + i] = static_cast<float>(v[int(i)]); });
  });
}
__device__ __forceinline__ void load16(const float *p, float (&x)[kPer]) {
  static_for<4>([&](auto h) {
    const f32x4 v = *reinterpret_cast<const f32x4 *>(p + 4 * h);
    static_for<4>([&](auto i) { x[4 * h + i] = v[int(i)]; });
  });
}
__device__ __forceinline__ void store16(bf16 *p, const float (&x)[kPer]) {
  static_for<2>([&](auto h) {
    bf16x8 v;
    static_for<8>([&](auto i) { v[int(i)] = static_cast<bf16>(x[8 * h + i]); });
    *reinterpret_cast<bf16x8 *>(p + 8 * h) = v;
  });
}
__device__ __forceinline__ void store16(float *p, const float (&x)[kPer]) {
  static_for<4>([&](auto h) {
    f32x4 v;
    static_for<4>([&](auto i) { v[int(i)] = x[4 * h + i]; });
    *reinterpret_cast<f32x4 *>(p + 4 * h) = v;
  });
}
__device__ __forceinline__ float power2(int e) {   // -126 <= e <= 127
  return __uint_as_float((uint32_t)(e + 127) << 23);
}

// Element offset in x of 16-element chunk c; rows of `per` chunks lie ld elements apart
// (per = 0: no gaps).
__device__ __forceinline__ int64_t chunk_at(int64_t c, int64_t per, int64_t ld) {
  if (per == 0) return c * kPer;
  const int64_t row = (c >> 32) || (per >> 32) ? c / per
                                               : (int64_t)((uint32_t)c / (uint32_t)per);
  return row * ld + (c - row * per) * kPer;
}

template <typename T>
__global__ __launch_bounds__(256) void ckpt8_pack_kernel(const T *__restrict__ x, int64_t chunks,
                                                         int64_t per, int64_t ld,
                                                         int8_t *__restrict__ q,
                                                         uint8_t *__restrict__ e) {
  const int64_t step = (int64_t)gridDim.x * 256;
  // an even number of chunks: the two threads of a group stay together
  for (int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x; c < chunks; c += step) {
    float v[kPer], top = 0.f;
    bool bad = false;
    load16(x + chunk_at(c, per, ld), v);
    static_for<kPer>([&](auto i) {
      top = fmaxf(top, fabsf(v[int(i)]));
      bad |= !(fabsf(v[int(i)]) < INFINITY);
    });
    top = fmaxf(top, __shfl_xor(top, 1));
    bad |= __shfl_xor((int)bad, 1) != 0;
    // floor(log2 top) - 6: top / 2^e is in [64, 128); one more if it rounds to 128
    int k = min(max((int)(__float_as_uint(top) >> 23) - 127 - 6, -126), 121);
    if (rintf(top * power2(-k)) > 127.f && k < 121) ++k;
    const float inv = power2(-k);
    i8x16 n;
    static_for<kPer>([&](auto i) {
      const float r = fminf(fmaxf(rintf(v[int(i)] * inv), -127.f), 127.f);
      n[int(i)] = bad ? (int8_t)0 : (int8_t)(int)r;
    });
    *reinterpret_cast<i8x16 *>(q + c * kPer) = n;
    if ((c & 1) == 0) e[c >> 1] = bad ? 255 : (uint8_t)(k + 127);
  }
}

template <typename T>
__device__ __forceinline__ void unpack_chunk(const int8_t *__restrict__ q,
                                             const uint8_t *__restrict__ e, int64_t c, T *x) {
  const i8x16 n = *reinterpret_cast<const i8x16 *>(q + c * kPer);
  const int b = e[c >> 1];
  // units of 2^-126 to 2^121; the byte of any other exponent reads as it would
  const float unit = b == 255 ? __uint_as_float(0x7fc00000u) : __uint_as_float((uint32_t)b << 23);
  float v[kPer];
  static_for<kPer>([&](auto i) { v[int(i)] = (float)n[int(i)] * unit; });
  store16(x, v);
}

template <typename T>
__global__ __launch_bounds__(256) void ckpt8_unpack_kernel(const int8_t *__restrict__ q,
                                                           const uint8_t *__restrict__ e,
                                                           int64_t chunks, int64_t per,
                                                           int64_t ld, T *__restrict__ x) {
  const int64_t step = (int64_t)gridDim.x * 256;
  for (int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x; c < chunks; c += step)
    unpack_chunk(q, e, c, x + chunk_at(c, per, ld));
}

// The four tensors of an attention backward, in one launch.
__global__ __launch_bounds__(256) void ckpt8_unpack4_kernel(Ckpt8Four a) {
  const int64_t total = a.chunks[0] + a.chunks[1] + a.chunks[2] + a.chunks[3];
  const int64_t step = (int64_t)gridDim.x * 256;
  for (int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x; c < total; c += step) {
    int64_t i = c;
    int t = 0;
    while (t < 3 && i >= a.chunks[t]) i -= a.chunks[t++];
    unpack_chunk(a.q[t], a.e[t], i, a.x[t] + i * kPer);
  }
}

static unsigned chunk_blocks(int64_t chunks) {
  return (unsigned)std::min<int64_t>((chunks + 255) / 256, 256 * 64);
}

int launch_ckpt8_pack(const void *x, bool fp32, int64_t rows, int64_t cols, int64_t ld, int8_t *q,
                      uint8_t *e, hipStream_t st) {
  const int64_t chunks = rows * (cols / kPer), per = ld == cols ? 0 : cols / kPer;
  if (fp32)
    hipLaunchKernelGGL(ckpt8_pack_kernel<float>, dim3(chunk_blocks(chunks)), dim3(256), 0, st,
                       static_cast<const float *>(x), chunks, per, ld, q, e);
  else
    hipLaunchKernelGGL(ckpt8_pack_kernel<bf16>, dim3(chunk_blocks(chunks)), dim3(256), 0, st,
                       static_cast<const bf16 *>(x), chunks, per, ld, q, e);
  const hipError_t r = hipGetLastError();
  if (r != hipSuccess) return fail(LIBRA_EHIP, "pack launch failed: %s", hipGetErrorString(r));
  return LIBRA_OK;
}

int launch_ckpt8_unpack(const int8_t *q, const uint8_t *e, int64_t rows, int64_t cols, bool fp32,
                        int64_t ld, void *x, hipStream_t st) {
  const int64_t chunks = rows * (cols / kPer), per = ld == cols ? 0 : cols / kPer;
  if (fp32)
    hipLaunchKernelGGL(ckpt8_unpack_kernel<float>, dim3(chunk_blocks(chunks)), dim3(256), 0, st, q,
                       e, chunks, per, ld, static_cast<float *>(x));
  else
    hipLaunchKernelGGL(ckpt8_unpack_kernel<bf16>, dim3(chunk_blocks(chunks)), dim3(256), 0, st, q,
                       e, chunks, per, ld, static_cast<bf16 *>(x));
  const hipError_t r = hipGetLastError();
  if (r != hipSuccess) return fail(LIBRA_EHIP, "unpack launch failed: %s", hipGetErrorString(r));
  return LIBRA_OK;
}

int launch_ckpt8_unpack4(const Ckpt8Four &a, hipStream_t st) {
  const int64_t total = a.chunks[0] + a.chunks[1] + a.chunks[2] + a.chunks[3];
  if (total == 0) return LIBRA_OK;
  hipLaunchKernelGGL(ckpt8_unpack4_kernel, dim3(chunk_blocks(total)), dim3(256), 0, st, a);
  const hipError_t r = hipGetLastError();
  if (r != hipSuccess) return fail(LIBRA_EHIP, "unpack launch failed: %s", hipGetErrorString(r));
  return LIBRA_OK;
}

}  // namespace libra
