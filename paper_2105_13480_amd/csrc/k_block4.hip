// Values to 4 bits with a shared scale for every 32 of a row, and back.
//
// A block of 32 consecutive values of a row has a scale byte s, 2^(s - 127), and
// codes of 4 bits: the sign and 0, 1/2, 1, 3/2, 2, 3, 4 or 6 times the scale.  With
// 2^x <= a < 2^(x + 1) for the block's largest magnitude a, s = x + 125 (floor: a is
// below 8 scales, and what is above 6 becomes 6) or one more where a > 3/2 2^x (up:
// a is at most 6 scales).  x + 127 is a's exponent field, so s comes from its bits;
// smaller than 2^-127 there is no scale.  Codes are rounded to nearest, ties to the
// even code, by the conversion instructions, which do so for every scale, also where
// values, scale or results are subnormal.  A block that holds an infinity or NaN has
// s = 255 and reads back as NaN.
//
// A lane has 8 values, four lanes a block: 32 or 16 bytes of each in one load, and the
// largest magnitude by two moves among the four.  Bound by memory, each value being read
// and each code written once: 32768 x 2048 from fp32 62 us, 4.9 TB/s, and to bf16 26 us,
// 6.5 TB/s (what was just written is still in the caches); 16384 x 2048 from bf16 18 us,
// 4.7 TB/s; 1001 x 2048 2.7 us each, a launch.
#include "common.h"
#include "routed.h"

namespace cnnlib {

namespace {

constexpr int kUnit = 8;  // values of a lane

// The block's scale byte from the largest magnitude's bits.
__device__ __forceinline__ uint32_t scale_byte(uint32_t top, bool up) {
  if (top >= 0x7f800000u) return 255u;
  const int s = (int)(top >> 23) - 2 + (up && (top & 0x7fffffu) > 0x400000u ? 1 : 0);
  return s > 0 ? (uint32_t)s : 0u;
}
// 2^(s - 127) as the conversions take it (they read the exponent field alone: 0 is
// 2^-127, 255 NaN).
__device__ __forceinline__ float scale_of(uint32_t s) { return __uint_as_float(s << 23); }

template <int CTRL> __device__ __forceinline__ uint32_t quad(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true);
}

template <typename T>
__global__ __launch_bounds__(256) void quantize4(const T* In, uint8_t* Codes, uint8_t* Scales,
                                                 int Nt, int Nc, int up) {
  int t, u;
  const int Nb = (Nc + 31) / 32;
  // a block's four lanes are all there or none
  if (!unit_of_thread(blockIdx.x, threadIdx.x, Nt, 4 * Nb, &t, &u)) return;
  const T* const row = In + (int64_t)t * Nc;
  const int c = kUnit * u;
  float v[kUnit];
  uint32_t raw[4] = {0u, 0u, 0u, 0u};  // bf16 values as they come
  if constexpr (sizeof(T) == 4) {
    if (c + kUnit <= Nc) {
      __builtin_memcpy(v, row + c, 32);
    } else {
#pragma unroll
      for (int i = 0; i < kUnit; ++i) v[i] = c + i < Nc ? row[c + i] : 0.f;
    }
  } else {
    if (c + kUnit <= Nc) {
      __builtin_memcpy(raw, row + c, 16);
    } else {
#pragma unroll
      for (int i = 0; i < kUnit; ++i)
        if (c + i < Nc) raw[i >> 1] |= (uint32_t)row[c + i] << (16 * (i & 1));
    }
#pragma unroll
    for (int i = 0; i < kUnit; ++i)
      v[i] = __uint_as_float(i & 1 ? raw[i >> 1] & 0xffff0000u : raw[i >> 1] << 16);
  }
  uint32_t top = 0u;
#pragma unroll
  for (int i = 0; i < kUnit; ++i) top = max(top, __float_as_uint(v[i]) & 0x7fffffffu);
  top = max(top, quad<0xb1>(top));  // quad_perm 1,0,3,2
  top = max(top, quad<0x4e>(top));  // quad_perm 2,3,0,1
  const uint32_t s = scale_byte(top, up != 0);
  const float scale = scale_of(s);
  uint32_t code = 0u;
#if defined(__HIP_DEVICE_COMPILE__)
  if constexpr (sizeof(T) == 4) {
    code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, v[0], v[1], scale, 0);
    code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, v[2], v[3], scale, 1);
    code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, v[4], v[5], scale, 2);
    code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, v[6], v[7], scale, 3);
  } else {
    typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
    code = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(code, __builtin_bit_cast(bf2, raw[0]), scale, 0);
    code = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(code, __builtin_bit_cast(bf2, raw[1]), scale, 1);
    code = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(code, __builtin_bit_cast(bf2, raw[2]), scale, 2);
    code = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(code, __builtin_bit_cast(bf2, raw[3]), scale, 3);
  }
#endif
  if (s == 255u) code = 0u;
  const int64_t block = (int64_t)t * Nb + (u >> 2);
  __builtin_memcpy(Codes + 16 * block + 4 * (u & 3), &code, 4);
  if ((u & 3) == 0) Scales[block] = (uint8_t)s;
}

template <typename TO>
__global__ __launch_bounds__(256) void dequantize4(const uint8_t* Codes, const uint8_t* Scales, TO* Out,
                                                   int Nt, int Nc) {
  int t, u;
  const int Nb = (Nc + 31) / 32, per = (Nc + kUnit - 1) / kUnit;
  if (!unit_of_thread(blockIdx.x, threadIdx.x, Nt, per, &t, &u)) return;
  const int64_t block = (int64_t)t * Nb + (u >> 2);
  uint32_t code;
  __builtin_memcpy(&code, Codes + 16 * block + 4 * (u & 3), 4);
  const float scale = scale_of(Scales[block]);
  TO* const out = Out + (int64_t)t * Nc + kUnit * u;
  const int left = Nc - kUnit * u;
#if defined(__HIP_DEVICE_COMPILE__)
  if constexpr (sizeof(TO) == 4) {
    typedef float f2 __attribute__((ext_vector_type(2)));
    const f2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, scale, 0);
    const f2 b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, scale, 1);
    const f2 c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, scale, 2);
    const f2 d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, scale, 3);
    const float v[kUnit] = {a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
    if (left >= kUnit) {
      __builtin_memcpy(out, v, 32);
    } else {
#pragma unroll
      for (int i = 0; i < kUnit; ++i)
        if (i < left) out[i] = v[i];
    }
  } else {
    typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
    const bf2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, scale, 0);
    const bf2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, scale, 1);
    const bf2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, scale, 2);
    const bf2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, scale, 3);
    const u32x4_t v = {__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b),
                       __builtin_bit_cast(uint32_t, c), __builtin_bit_cast(uint32_t, d)};
    if (left >= kUnit) {
      __builtin_memcpy(out, &v, 16);
    } else {
#pragma unroll
      for (int i = 0; i < kUnit; ++i)
        if (i < left) out[i] = (bf16_t)(v[i >> 1] >> (16 * (i & 1)));
    }
  }
#else
  (void)code;
  (void)scale;
  (void)out;
  (void)left;
#endif
}

}  // namespace

hipError_t launch_quantize4(const void* In, uint8_t* Codes, uint8_t* Scales, int64_t Nt, int64_t Nc,
                            bool bf16, bool up, hipStream_t stream) {
  const int64_t blocks = (Nt * (4 * ((Nc + 31) / 32)) + 255) / 256;
  const hipError_t e = grid_fits(blocks, 256);
  if (e != hipSuccess) return e;
  const dim3 grid((uint32_t)blocks), block(256);
  if (bf16)
    quantize4<bf16_t><<<grid, block, 0, stream>>>((const bf16_t*)In, Codes, Scales, (int)Nt, (int)Nc, up);
  else
    quantize4<float><<<grid, block, 0, stream>>>((const float*)In, Codes, Scales, (int)Nt, (int)Nc, up);
  return hipGetLastError();
}

hipError_t launch_dequantize4(const uint8_t* Codes, const uint8_t* Scales, void* Out, int64_t Nt,
                              int64_t Nc, bool bf16, hipStream_t stream) {
  const int64_t blocks = (Nt * ((Nc + kUnit - 1) / kUnit) + 255) / 256;
  const hipError_t e = grid_fits(blocks, 256);
  if (e != hipSuccess) return e;
  const dim3 grid((uint32_t)blocks), block(256);
  if (bf16) dequantize4<bf16_t><<<grid, block, 0, stream>>>(Codes, Scales, (bf16_t*)Out, (int)Nt, (int)Nc);
  else dequantize4<float><<<grid, block, 0, stream>>>(Codes, Scales, (float*)Out, (int)Nt, (int)Nc);
  return hipGetLastError();
}

}  // namespace cnnlib
