// Rotary positions: what queries and keys go through between the projection and every attention or cache call of this
// library (the paper's cache holds keys after the rotary transformation: Section 3.2, text below Eq. 4).
//
// Pair i < R / 2 of a row at position p turns by the angle p w_i:
//   y_a = gain (x_a cos - x_b sin),  y_b = gain (x_b cos + x_a sin),   (a, b) = (i, i + R / 2) or (2 i, 2 i + 1);
// the rest of the row (R < D) is carried over.  The inverse takes sin with the other sign: the transposed matrix, which is
// also the gradient with respect to x.
//
// Far positions: p w_i in 32 bits would be off by p 2^-24 radians (0.06 at a million).  Only the fraction of a turn
// matters, so a frequency is kept as a 64-bit fraction of a turn per position, F = w / 2 pi * 2^64, and p F in 64-bit integer
// arithmetic, which drops whole turns by itself, is the phase: off by at most |p| 2^-65 turns (and by what w has lost in its
// own 53 bits).  The sine takes it as half turns in fp32, rounded from all 64 bits: off by 2^-24 of itself, at most 2^-26 turns.
// (Its upper half alone would be cut off at 2^-32 turns: an angle of 1e-6 would have lost a thousandth of itself.)
//
// Bound by memory: every value is read once and written once.  A thread owns a chunk of E pairs (two 16-byte pieces of a
// row), works out its sines and cosines once per token and walks over the heads of queries and keys alike with them, four
// heads' loads in flight; a token's heads are spread over as many threads as it takes to fill the GPU, so a decode step is
// one short pass.  8192 tokens of 32 + 8 heads, bf16: 33.2 us, 5.05 TB/s (0.77 of the measured copy rate); 8004 tokens of 40 + 40
// heads, fp32, half of each turned: 114 us, 5.7 TB/s (0.88).
// (A block that works out its tokens' sines once for all, with four heads to a thread, was tried: 105 us for the latter, but 41
// for the former.)
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <cmath>

#include "razor_common.cuh"

namespace razor {
namespace {

constexpr int kRopeMaxDim = 256;
constexpr int kRopeThreads = 256;

struct RopeSide {   // queries or keys
  const char* in;
  char* out;
  int64_t in_b, in_t, in_h, out_b, out_t, out_h;   // bytes
  int32_t n_heads;
};
struct RopeCall {
  RopeSide side[2];
  const int32_t* positions;   // [batch, n_tokens], NULL: 0, 1, ..
  int64_t rows;               // batch * n_tokens
  int32_t n_tokens, head_dim, rotated, interleaved, inverse;
  int32_t slots;              // threads that share the heads of a token, per column
  int32_t narrow;             // threads are numbered in 32 bits
  float gain;
  uint64_t turn[kRopeMaxDim / 2];   // frequencies in 2^-64 turns per position
};

template <typename T>
__device__ __forceinline__ void pack(const float (&f)[Elem<T>::kEpl], uint4& u);
template <>
__device__ __forceinline__ void pack<float>(const float (&f)[4], uint4& u) {
  u = make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
}
template <>
__device__ __forceinline__ void pack<__nv_bfloat16>(const float (&f)[8], uint4& u) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
    w[i] = *(const uint32_t*)&v;
  }
  u = make_uint4(w[0], w[1], w[2], w[3]);
}

__device__ __forceinline__ void turn_of(const RopeCall& c, int pair, int32_t p, float& cs, float& sn) {
  const uint64_t phase = (uint64_t)(int64_t)p * c.turn[pair];
  // the nearest whole turn dropped: half turns in [-1, 1], rounded once (a small angle keeps its 24 bits)
  sincospif((float)(int64_t)phase * 1.0842021724855044e-19f, &sn, &cs);
  cs *= c.gain;
  sn *= c.inverse ? -c.gain : c.gain;
}

// Where thread `id` of the call works: column, head slot and token.  (A division in 64 bits costs as much as a head's arithmetic.)
struct RopePlace {
  int col, slot;
  int64_t row, b, t;
};
__device__ __forceinline__ RopePlace place(const RopeCall& c, int cols, int64_t id) {
  RopePlace r;
  if (c.narrow) {
    const uint32_t i = (uint32_t)id, rest = i / (uint32_t)cols, row = rest / (uint32_t)c.slots;
    r.col = (int)(i % (uint32_t)cols);
    r.slot = (int)(rest % (uint32_t)c.slots);
    r.row = row;
    r.b = row / (uint32_t)c.n_tokens;
    r.t = row % (uint32_t)c.n_tokens;
  } else {
    const int64_t rest = id / cols;
    r.col = (int)(id % cols);
    r.slot = (int)(rest % c.slots);
    r.row = rest / c.slots;
    r.b = r.row / c.n_tokens;
    r.t = r.row % c.n_tokens;
  }
  return r;
}

__device__ __forceinline__ const char* in_row(const RopeCall& c, int h, int64_t b, int64_t t) {
  const RopeSide& s = c.side[h >= c.side[0].n_heads];
  return s.in + b * s.in_b + t * s.in_t + (h >= c.side[0].n_heads ? h - c.side[0].n_heads : h) * s.in_h;
}
__device__ __forceinline__ char* out_row(const RopeCall& c, int h, int64_t b, int64_t t) {
  const RopeSide& s = c.side[h >= c.side[0].n_heads];
  return s.out + b * s.out_b + t * s.out_t + (h >= c.side[0].n_heads ? h - c.side[0].n_heads : h) * s.out_h;
}

// Rows of 16-byte pieces: head_dim and rotated are multiples of 2 E.  Thread -> (row of tokens, head slot, column); a row
// has head_dim / 2 E columns, the first rotated / 2 E of them turn, the others copy.
template <typename T>
__global__ void __launch_bounds__(kRopeThreads) rope_kernel(const __grid_constant__ RopeCall c) {
  constexpr int E = Elem<T>::kEpl;
  const int cols = c.head_dim / (2 * E);
  const RopePlace at = place(c, cols, (int64_t)blockIdx.x * kRopeThreads + threadIdx.x);
  const int col = at.col, slot = at.slot;
  const int64_t row = at.row, b = at.b, t = at.t;
  if (row >= c.rows) return;
  const int heads = c.side[0].n_heads + c.side[1].n_heads;
  const int turning = c.rotated / (2 * E);
  const bool turns = col < turning;
  // byte offsets of this thread's two pieces
  int lo = 2 * col * 16, hi = lo + 16;
  if (turns && !c.interleaved) {
    lo = col * 16;
    hi = lo + c.rotated / 2 * (int)sizeof(T);
  }
  float cs[E], sn[E];
  if (turns) {
    const int32_t p = c.positions ? c.positions[row] : (int32_t)t;
#pragma unroll
    for (int i = 0; i < E; ++i) turn_of(c, col * E + i, p, cs[i], sn[i]);
  }
  constexpr int U = 4;
  for (int h0 = slot; h0 < heads; h0 += U * c.slots) {
    uint4 x[U], y[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int h = h0 + u * c.slots;
      if (h < heads) {
        const char* src = in_row(c, h, b, t);
        x[u] = *(const uint4*)(src + lo);
        y[u] = *(const uint4*)(src + hi);
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int h = h0 + u * c.slots;
      if (h >= heads) break;
      char* dst = out_row(c, h, b, t);
      if (turns) {
        float f[E], g[E];
        Elem<T>::unpack(x[u], f);
        Elem<T>::unpack(y[u], g);
        if (c.interleaved) {
#pragma unroll
          for (int i = 0; i < E / 2; ++i) {
            const float a0 = f[2 * i], b0 = f[2 * i + 1], a1 = g[2 * i], b1 = g[2 * i + 1];
            f[2 * i] = fmaf(a0, cs[i], -(b0 * sn[i]));
            f[2 * i + 1] = fmaf(b0, cs[i], a0 * sn[i]);
            g[2 * i] = fmaf(a1, cs[E / 2 + i], -(b1 * sn[E / 2 + i]));
            g[2 * i + 1] = fmaf(b1, cs[E / 2 + i], a1 * sn[E / 2 + i]);
          }
        } else {
#pragma unroll
          for (int i = 0; i < E; ++i) {
            const float a = f[i], bb = g[i];
            f[i] = fmaf(a, cs[i], -(bb * sn[i]));
            g[i] = fmaf(bb, cs[i], a * sn[i]);
          }
        }
        pack<T>(f, x[u]);
        pack<T>(g, y[u]);
      }
      *(uint4*)(dst + lo) = x[u];
      *(uint4*)(dst + hi) = y[u];
    }
  }
}

// Any even `rotated` <= head_dim: a thread per pair of values, so accesses of 2 or 4 bytes and one head in flight.  8192 tokens of
// 32 + 8 heads, bf16, 102 of 128 values turned: 74.5 us (0.34 of the measured copy rate); 8004 tokens of 40 + 40 heads, fp32, 58 turned:
// 149 us (0.67).
template <typename T>
__global__ void __launch_bounds__(kRopeThreads) rope_pairs_kernel(const __grid_constant__ RopeCall c) {
  const int cols = c.head_dim / 2;
  const RopePlace at = place(c, cols, (int64_t)blockIdx.x * kRopeThreads + threadIdx.x);
  const int col = at.col, slot = at.slot;
  const int64_t row = at.row, b = at.b, t = at.t;
  if (row >= c.rows) return;
  const int heads = c.side[0].n_heads + c.side[1].n_heads, half = c.rotated / 2;
  const bool turns = col < half;
  int lo = 2 * col, hi = lo + 1;
  if (turns && !c.interleaved) {
    lo = col;
    hi = col + half;
  }
  float cs = 1.f, sn = 0.f;
  if (turns) turn_of(c, col, c.positions ? c.positions[row] : (int32_t)t, cs, sn);
  for (int h = slot; h < heads; h += c.slots) {
    const T* src = (const T*)in_row(c, h, b, t);
    T* dst = (T*)out_row(c, h, b, t);
    const T x = src[lo], y = src[hi];
    if (turns) {
      const float a = (float)x, bb = (float)y;
      dst[lo] = (T)fmaf(a, cs, -(bb * sn));
      dst[hi] = (T)fmaf(bb, cs, a * sn);
    } else {
      dst[lo] = x;
      dst[hi] = y;
    }
  }
}

template <typename T>
cudaError_t launch_rope(RopeCall& c, int n_sms, cudaStream_t s) {
  constexpr int E = Elem<T>::kEpl;
  const bool pieces = c.head_dim % (2 * E) == 0 && c.rotated % (2 * E) == 0;
  const int cols = pieces ? c.head_dim / (2 * E) : c.head_dim / 2;
  const int heads = c.side[0].n_heads + c.side[1].n_heads;
  // Threads that share a token's heads: enough to fill the GPU's 2048 threads per SM (each repeats the sines).
  const int64_t want = ((int64_t)n_sms * 2048 + c.rows * cols - 1) / (c.rows * cols);
  c.slots = (int)std::max<int64_t>(1, std::min<int64_t>(want, heads));
  const int64_t threads = c.rows * cols * c.slots;
  const int64_t blocks = (threads + kRopeThreads - 1) / kRopeThreads;
  if (blocks > 0x7fffffff) return cudaErrorInvalidConfiguration;
  c.narrow = blocks * kRopeThreads < (1LL << 32);
  if (pieces) rope_kernel<T><<<(unsigned)blocks, kRopeThreads, 0, s>>>(c);
  else rope_pairs_kernel<T><<<(unsigned)blocks, kRopeThreads, 0, s>>>(c);
  return cudaGetLastError();
}

// Checks one side and puts it into the call.  Strides that separate nothing are not looked at.
int take_side(const razor_rope_rows_t* r, int batch, int n_tokens, int head_dim, int es, RopeSide& s) {
  if (!r || r->n_heads == 0) {
    s = RopeSide{};
    return RAZOR_OK;
  }
  if (r->n_heads < 0 || r->n_heads > 65536) return RAZOR_E_INVALID_ARG;
  if (n_tokens == 0) return RAZOR_OK;   // (an empty tensor has no address)
  if (!r->in || !r->out) return RAZOR_E_NULL_PTR;
  const int64_t n[3] = {batch, n_tokens, r->n_heads};
  int64_t st[2][3] = {{r->in_stride_b, r->in_stride_t, r->in_stride_h}, {r->out_stride_b, r->out_stride_t, r->out_stride_h}};
  bool misaligned = (((uintptr_t)r->in | (uintptr_t)r->out) & 15) != 0;
  for (int side = 0; side < 2; ++side)
    for (int d = 0; d < 3; ++d) {
      int64_t& x = st[side][d];
      if (n[d] <= 1) x = 0;
      if (x < 0 || x > (1LL << 40) || (x > 0 && n[d] > (1LL << 52) / x)) return RAZOR_E_INVALID_ARG;   // (no such memory)
      // two rows of the output in one place would be written twice (a repeated input row is fine)
      if (side == 1 && n[d] > 1 && x < head_dim) return RAZOR_E_INVALID_ARG;
      misaligned |= ((x * es) & 15) != 0;
    }
  if (misaligned) return RAZOR_E_MISALIGNED;
  // The output's rows must not meet: with its dimensions in the order of their strides, each steps over the one below it.
  {
    int order[3] = {0, 1, 2};
    std::sort(order, order + 3, [&](int a, int b) { return st[1][a] < st[1][b]; });
    int64_t extent = head_dim;
    for (int i = 0; i < 3; ++i) {
      const int d = order[i];
      if (n[d] <= 1) continue;
      if (st[1][d] < extent) return RAZOR_E_INVALID_ARG;
      extent += (n[d] - 1) * st[1][d];
    }
  }
  // In place: the same rows in the same places (a thread reads its pieces before it writes them).
  if (r->in == r->out)
    for (int d = 0; d < 3; ++d)
      if (st[0][d] != st[1][d]) return RAZOR_E_INVALID_ARG;
  s.in = (const char*)r->in;
  s.out = (char*)r->out;
  s.in_b = st[0][0] * es; s.in_t = st[0][1] * es; s.in_h = st[0][2] * es;
  s.out_b = st[1][0] * es; s.out_t = st[1][1] * es; s.out_h = st[1][2] * es;
  s.n_heads = r->n_heads;
  return RAZOR_OK;
}

}  // namespace
}  // namespace razor

extern "C" int razor_rope_frequencies(int32_t rotated, double base, int32_t scaling, double factor, int32_t original_len,
                                      double* inv_freq, float* gain) {
  if (!inv_freq) return RAZOR_E_NULL_PTR;
  if (rotated < 2 || rotated % 2 || rotated > razor::kRopeMaxDim) return RAZOR_E_INVALID_ARG;
  if (!(base > 1.0) || std::isinf(base)) return RAZOR_E_INVALID_ARG;
  if (scaling < RAZOR_ROPE_PLAIN || scaling > RAZOR_ROPE_BANDED) return RAZOR_E_INVALID_ARG;
  if (scaling != RAZOR_ROPE_PLAIN && (!(factor >= 1.0) || std::isinf(factor))) return RAZOR_E_INVALID_ARG;
  if ((scaling == RAZOR_ROPE_YARN || scaling == RAZOR_ROPE_BANDED) && original_len < 1) return RAZOR_E_INVALID_ARG;
  if (scaling == RAZOR_ROPE_NTK && rotated < 4) return RAZOR_E_INVALID_ARG;   // the exponent R / (R - 2) has no value
  const double two_pi = 6.283185307179586476925286766559, R = rotated, L = original_len;
  if (scaling == RAZOR_ROPE_NTK) base *= std::pow(factor, R / (R - 2.0));
  double lo = 0.0, hi = 0.0;
  if (scaling == RAZOR_ROPE_YARN) {   // pairs that make 32 turns and 1 turn over the original length
    lo = std::max(std::floor(R * std::log(L / (two_pi * 32.0)) / (2.0 * std::log(base))), 0.0);
    hi = std::min(std::ceil(R * std::log(L / two_pi) / (2.0 * std::log(base))), R - 1.0);
  }
  for (int i = 0; i < rotated / 2; ++i) {
    const double w = std::pow(base, -2.0 * i / R);
    double out = w;
    if (scaling == RAZOR_ROPE_LINEAR) {
      out = w / factor;
    } else if (scaling == RAZOR_ROPE_YARN) {
      const double ramp = std::min(std::max((i - lo) / std::max(hi - lo, 0.001), 0.0), 1.0);
      out = w / factor * ramp + w * (1.0 - ramp);
    } else if (scaling == RAZOR_ROPE_BANDED) {
      const double smooth = std::min(std::max((L * w / two_pi - 1.0) / (4.0 - 1.0), 0.0), 1.0);
      out = (1.0 - smooth) * w / factor + smooth * w;
    }
    inv_freq[i] = out;
  }
  if (gain) *gain = scaling == RAZOR_ROPE_YARN ? (float)(0.1 * std::log(factor) + 1.0) : 1.f;
  return RAZOR_OK;
}

extern "C" int razor_rope(const razor_rope_rows_t* q, const razor_rope_rows_t* k, const int32_t* positions, int32_t batch,
                          int32_t n_tokens, int32_t head_dim, int32_t rotated, int32_t dtype, const double* inv_freq, float gain,
                          int32_t interleaved, int32_t inverse, void* stream) {
  using namespace razor;
  if (!inv_freq) return RAZOR_E_NULL_PTR;
  if (batch < 1 || n_tokens < 0 || (int64_t)batch * n_tokens > (1LL << 40) || !std::isfinite(gain)) return RAZOR_E_INVALID_ARG;
  if (dtype != RAZOR_F32 && dtype != RAZOR_BF16) return RAZOR_E_UNSUPPORTED_DIM;
  const int es = dtype == RAZOR_BF16 ? 2 : 4;
  if (head_dim < 2 || head_dim > kRopeMaxDim || (head_dim * es) % 16) return RAZOR_E_UNSUPPORTED_DIM;
  if (rotated < 2 || rotated % 2 || rotated > head_dim) return RAZOR_E_INVALID_ARG;
  if ((uintptr_t)positions & 3) return RAZOR_E_MISALIGNED;
  RopeCall c;
  int rc = take_side(q, batch, n_tokens, head_dim, es, c.side[0]);
  if (!rc) rc = take_side(k, batch, n_tokens, head_dim, es, c.side[1]);
  if (rc) return rc;
  for (int i = 0; i < rotated / 2; ++i) {
    if (!std::isfinite(inv_freq[i])) return RAZOR_E_INVALID_ARG;
    // the fraction of a turn per position; whole turns drop out
    long double f = (long double)inv_freq[i] * 0.159154943091895335768883763372514362L;
    if (f < 0.0L || f >= 1.0L) f -= floorl(f);
    f = f * 18446744073709551616.0L + 0.5L;
    c.turn[i] = f >= 18446744073709551616.0L ? 0ull : (uint64_t)f;
  }
  if (n_tokens == 0 || c.side[0].n_heads + c.side[1].n_heads == 0) return RAZOR_OK;
  c.positions = positions;
  c.rows = (int64_t)batch * n_tokens;
  c.n_tokens = n_tokens; c.head_dim = head_dim; c.rotated = rotated;
  c.interleaved = interleaved != 0; c.inverse = inverse != 0; c.gain = gain;
  int dev = 0, sms = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  if (e == cudaSuccess)
    e = dtype == RAZOR_BF16 ? launch_rope<__nv_bfloat16>(c, sms, (cudaStream_t)stream) : launch_rope<float>(c, sms, (cudaStream_t)stream);
  if (e != cudaSuccess) {
    note_cuda_error(e);
    return RAZOR_E_CUDA;
  }
  return RAZOR_OK;
}
