// Device helpers shared by the kernels: 16-byte row fragments, unpacking, warp reductions.
#ifndef RAZOR_COMMON_CUH_
#define RAZOR_COMMON_CUH_

#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "razor_internal.h"

namespace razor {

// A K or V row is read as 16-byte fragments, one per lane: LPR lanes cover a row, each lane owns
// EPL consecutive dimensions.
template <typename T>
struct Elem;
template <>
struct Elem<float> {
  static constexpr int kEpl = 4;  // elements per 16-byte fragment
  static __device__ __forceinline__ void unpack(const uint4& u, float (&f)[4]) {
    f[0] = __uint_as_float(u.x);
    f[1] = __uint_as_float(u.y);
    f[2] = __uint_as_float(u.z);
    f[3] = __uint_as_float(u.w);
  }
};
template <>
struct Elem<__nv_bfloat16> {
  static constexpr int kEpl = 8;
  // bf16 -> fp32 is a 16-bit shift: the low half of a word is element 2i, the high half 2i+1.
  static __device__ __forceinline__ void unpack(const uint4& u, float (&f)[8]) {
    f[0] = __uint_as_float(u.x << 16);
    f[1] = __uint_as_float(u.x & 0xffff0000u);
    f[2] = __uint_as_float(u.y << 16);
    f[3] = __uint_as_float(u.y & 0xffff0000u);
    f[4] = __uint_as_float(u.z << 16);
    f[5] = __uint_as_float(u.z & 0xffff0000u);
    f[6] = __uint_as_float(u.w << 16);
    f[7] = __uint_as_float(u.w & 0xffff0000u);
  }
};

template <typename T, int D>
struct RowGeom {
  static constexpr int kEpl = Elem<T>::kEpl;
  static constexpr int kRowBytes = D * (int)sizeof(T);
  static constexpr int kLpr = kRowBytes / 16;      // lanes per row
  static constexpr int kRg = 32 / kLpr;            // rows a warp reads per load instruction
  static constexpr int kRowsPerGroup = kPageTokens / kRg;
  static constexpr int kPageBytes = 2 * kPageTokens * kRowBytes;
  static_assert(kLpr == 8 || kLpr == 16 || kLpr == 32, "row must be 128, 256 or 512 bytes");
};

// In-page placement of 16-byte chunks.  A page is stored as [16 K rows][16 V rows]; chunk c of the row
// of token t (t = slot & 15) sits at chunk position c ^ (t & 7).  The page travels to shared memory
// as one flat block, and with this placement eight rows read at the same logical chunk fall into
// eight different bank groups, which is what the matrix-fragment loads of the grouped-query path
// need; row-wise readers just permute their lanes.
__device__ __forceinline__ int swz(int token, int chunk) { return chunk ^ (token & 7); }

__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}

// ---- pages of 8-bit rows.  A row x is held as codes c = round(x * (127 / top)), top its largest magnitude, and one scale
// top / 127 in fp32: the value held is scale * c, off by at most half a step, top / 254, and 2^-22 top (127 / top and its product
// with x move a code by up to 127 2^-23, scale and value round once each).  Quotients, product and rounding are IEEE's, to
// nearest even, so that anybody can compute the same codes.  A page is [16 K rows of D bytes][16 V rows][16 K
// scales][16 V scales]; a code is stored as the byte c + 128.  Chunk placement, chosen for the fragment loads of the decode
// kernel (eight lanes read 16 bytes each at a time): two K rows at four neighbouring chunks, or four V rows at two, meet
// no bank twice (at D = 64 V's do, once: a row is half a line).
constexpr __host__ __device__ int q8_page_bytes(int d) { return 2 * kPageTokens * (d + 4); }
template <int D>
__device__ __forceinline__ int q8_chunk(int kv, int token, int chunk) {
  if (kv == 0) return D == 128 ? chunk ^ ((token & 1) << 2) : chunk;
  return D == 128 ? chunk ^ (token & 7) : chunk ^ ((token >> 1) & 3);
}
template <int D>
struct Q8Row {   // eight elements of a row per lane, D / 8 lanes to a row
  static constexpr int kLpr = D / 8;
  static __device__ __forceinline__ uint8_t* codes(uint8_t* page, int slot, int kv, int lir) {
    const int t = slot & 15;
    return page + (kv * kPageTokens + t) * D + q8_chunk<D>(kv, t, lir >> 1) * 16 + (lir & 1) * 8;
  }
  static __device__ __forceinline__ float* scale(uint8_t* page, int slot, int kv) {
    return (float*)(page + 2 * kPageTokens * D) + kv * kPageTokens + (slot & 15);
  }
  static __device__ __forceinline__ void load(const uint8_t* page, int slot, int kv, int lir, float (&f)[8]) {
    const uint2 u = *(const uint2*)codes((uint8_t*)page, slot, kv, lir);
    const float s = *scale((uint8_t*)page, slot, kv);
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = s * (float)((int)(((i < 4 ? u.x : u.y) >> (8 * (i & 3))) & 0xffu) - 128);
  }
  // The largest magnitude among this lane's eight elements; of the whole row it is the maximum over its kLpr lanes.  NaN if
  // an element is.
  static __device__ __forceinline__ float lane_top(const uint4& raw) {
    float f[8], top = 0.f;
    Elem<__nv_bfloat16>::unpack(raw, f);
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max_nan(top, fabsf(f[i]));
    return top;
  }
  static __device__ __forceinline__ float row_top(const uint4& raw, unsigned lanes) {
    float top = lane_top(raw);
#pragma unroll
    for (int off = kLpr / 2; off > 0; off >>= 1) top = max_nan(top, __shfl_xor_sync(lanes, top, off));
    return top;
  }
  // Quantises the eight bf16 elements `raw` of a row whose largest magnitude is `top`.  w, s: codes and scale, held: the
  // values they stand for.  A row whose largest magnitude is below 2^-100 is held as zeros (127 / top leaves the range of fp32
  // below 2^-121: a bound chosen with room), one with a value that is not finite as NaN.
  static __device__ __forceinline__ void quantise(const uint4& raw, float top, uint32_t (&w)[2], float& s, float (&held)[8]) {
    float f[8];
    Elem<__nv_bfloat16>::unpack(raw, f);
    const bool fine = top < __uint_as_float(0x7f800000u), some = top >= 7.888609052210118e-31f;
    const float inv = fine && some ? __fdiv_rn(127.f, top) : 0.f;
    s = !fine ? __uint_as_float(0x7fc00000u) : (some ? __fdiv_rn(top, 127.f) : 0.f);
    // A product of at most 127 and a bit, plus 1.5 * 2^23: rounded to a whole number, half to even, which is in the low bits.
    // (Conversions to integers take the slow unit; a 32K fill was bound by them and the packing.)
    constexpr float kMagic = 12582912.f;
    uint32_t r[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float x = __fadd_rn(__fmul_rn(f[i], inv), kMagic);
      r[i] = __float_as_uint(x);
      held[i] = s * (x - kMagic);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
      w[i] = __byte_perm(__byte_perm(r[4 * i], r[4 * i + 1], 0x0040), __byte_perm(r[4 * i + 2], r[4 * i + 3], 0x0040), 0x5410) ^ 0x80808080u;
  }
  static __device__ __forceinline__ void store(uint8_t* page, int slot, int kv, int lir, const uint4& raw, float top, float (&held)[8]) {
    uint32_t w[2];
    float s;
    quantise(raw, top, w, s, held);
    *(uint2*)codes(page, slot, kv, lir) = make_uint2(w[0], w[1]);
    if (lir == 0) *scale(page, slot, kv) = s;
  }
};

// Streaming 16-byte load: the KV cache is read once per step, keep it out of L1.
__device__ __forceinline__ uint4 ld_stream(const uint4* p) {
  uint4 v;
  asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
               : "l"(p));
  return v;
}

// Load that must see other SMs' writes from this launch (partial records): L2 only.
__device__ __forceinline__ float ld_cg(const float* p) { return __ldcg(p); }
__device__ __forceinline__ float4 ld_cg4(const float4* p) { return __ldcg(p); }

__device__ __forceinline__ float fast_exp2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// Sum over the kLpr lanes that share a row (butterfly; every lane ends with the total).
template <int LPR>
__device__ __forceinline__ float row_sum(float x) {
#pragma unroll
  for (int off = LPR / 2; off > 0; off >>= 1) x += __shfl_xor_sync(0xffffffffu, x, off);
  return x;
}

// A row of D floats spread over a warp: D/32 consecutive floats per lane.
template <int D>
struct LaneVec;
template <>
struct LaneVec<128> {
  float4 v;
  __device__ __forceinline__ void zero() { v = make_float4(0.f, 0.f, 0.f, 0.f); }
  __device__ __forceinline__ void fma(float c, const LaneVec& o) {
    v.x += c * o.v.x; v.y += c * o.v.y; v.z += c * o.v.z; v.w += c * o.v.w;
  }
  __device__ __forceinline__ void scale(float c) { v.x *= c; v.y *= c; v.z *= c; v.w *= c; }
  __device__ __forceinline__ void load_shared(const float* row, int lane) { v = *(const float4*)(row + lane * 4); }
  __device__ __forceinline__ void load_l2(const float* row, int lane) { v = __ldcg((const float4*)(row + lane * 4)); }
  __device__ __forceinline__ void store(float* row, int lane) const { *(float4*)(row + lane * 4) = v; }
};
template <>
struct LaneVec<64> {
  float2 v;
  __device__ __forceinline__ void zero() { v = make_float2(0.f, 0.f); }
  __device__ __forceinline__ void fma(float c, const LaneVec& o) { v.x += c * o.v.x; v.y += c * o.v.y; }
  __device__ __forceinline__ void scale(float c) { v.x *= c; v.y *= c; }
  __device__ __forceinline__ void load_shared(const float* row, int lane) { v = *(const float2*)(row + lane * 2); }
  __device__ __forceinline__ void load_l2(const float* row, int lane) { v = __ldcg((const float2*)(row + lane * 2)); }
  __device__ __forceinline__ void store(float* row, int lane) const { *(float2*)(row + lane * 2) = v; }
};

}  // namespace razor
#endif
