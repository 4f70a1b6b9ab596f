// Rotary positions: Q and K of rows of Q | K | V are rotated pair by pair, by an angle that grows with the token's position.  With
// c = amplitude cos(2 pi p f), n = amplitude sin(2 pi p f) for position p and a pair's frequency f (turns per position):
//   forward (x, y) -> (c x - n y, n x + c y);  backward, the transposed map: (dx, dy) -> (c dx + n dy, c dy - n dx).
//
// Bound by memory: a row is read and written once (in place only what is rotated), 3 flops an element.  The angles are what could
// get in the way: p f needs 64 bits (at position 100000 a product of 32 bits is off by 0.006 turns), its fraction does not.  A wave
// owns a token and a lane one group of a head's pairs, so that a lane's sines and cosines serve the token's heads one after the other.
// 4 x 2048 tokens, 16 heads of 128, bf16: 201 MB in 41 us, 4.95 TB/s; 30011 tokens, 20 + 2 x 4 heads of 160, fp32: 1.08 GB in 210 us, 5.1 TB/s (a copy: 4.9).
#include "common.h"

namespace ptdp {

// V elements, 16 or 8 bytes
template <typename T, int V> struct RotaryVec {
  typedef uint32_t words_t __attribute__((ext_vector_type(V * sizeof(T) / 4)));
  words_t raw;
  __device__ __forceinline__ void load(const T* p) { raw = *reinterpret_cast<const words_t*>(p); }
  __device__ __forceinline__ void store(T* p) const { *reinterpret_cast<words_t*>(p) = raw; }
  __device__ __forceinline__ void unpack(float (&f)[V]) const {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      if constexpr (sizeof(T) == 4) f[i] = __uint_as_float(raw[i]);
      else f[i] = __uint_as_float(i & 1 ? raw[i / 2] & 0xffff0000u : raw[i / 2] << 16);
    }
  }
  __device__ __forceinline__ void pack(const float (&f)[V]) {
#pragma unroll
    for (int i = 0; i < (int)(V * sizeof(T) / 4); ++i) {
      if constexpr (sizeof(T) == 4) raw[i] = __float_as_uint(f[i]);
      else raw[i] = pack_bf16x2(f[2 * i], f[2 * i + 1]);
    }
  }
};

constexpr int kRotaryThreads = 256;
constexpr int kRotaryAhead = 4;   // heads of a lane requested together
// PAIRS: neighbours (2 i, 2 i + 1) form a pair, otherwise (i, i + rot / 2).  V: elements of an access.  A lane's group is V neighbouring
// elements of a head (PAIRS: V / 2 pairs) or V of either half (V pairs).
template <typename T, bool PAIRS, int V>
__global__ void __launch_bounds__(kRotaryThreads)
rotary_kernel(const T* qkv, T* out, const int32_t* __restrict__ positions, const double* __restrict__ turns, uint32_t tokens, int b, int heads,
              int kv_heads, int dh, int rot, float amplitude, float sign) {
  constexpr int NP = PAIRS ? V / 2 : V, NA = PAIRS ? 1 : 2;   // pairs of a group; accesses
  const int lane = threadIdx.x & 63;
  const uint32_t waves = gridDim.x * (kRotaryThreads / 64);
  const int groups = rot / (PAIRS ? V : 2 * V), rotated = heads + kv_heads;
  const int lanes_h = 64 / groups, group = lane % groups, h0 = lane / groups;   // this lane takes heads h0, h0 + lanes_h, ..
  const size_t row = (size_t)(rotated + kv_heads) * dh;
  const bool copy = out != qkv;
  for (uint32_t token = blockIdx.x * (kRotaryThreads / 64) + (threadIdx.x >> 6); token < tokens; token += waves) {
    const T* src = qkv + token * row;
    T* dst = out + token * row;
    const double place = positions ? (double)positions[token] : (double)(token / (uint32_t)b);
    RotaryVec<T, V> x[kRotaryAhead][NA];
    auto load = [&](int h) {
#pragma unroll
      for (int u = 0; u < kRotaryAhead; ++u) {
        const T* p = src + (size_t)min(h + u * lanes_h, rotated - 1) * dh + group * V;
#pragma unroll
        for (int a = 0; a < NA; ++a) x[u][a].load(p + a * (rot / 2));
      }
    };
    float c[NP], n[NP];
    if (h0 < lanes_h) {
      load(h0);
#pragma unroll
      for (int i = 0; i < NP; ++i) {
        const double t = place * turns[group * NP + i];
        float si, co;
        sincospif(2.f * (float)(t - rint(t)), &si, &co);
        c[i] = amplitude * co;
        n[i] = amplitude * sign * si;
      }
      for (int h = h0; h < rotated; h += kRotaryAhead * lanes_h) {
        if (h != h0) load(h);
#pragma unroll
        for (int u = 0; u < kRotaryAhead; ++u) {
          const int head = h + u * lanes_h;
          if (head >= rotated) break;
          float f[NA][V];
#pragma unroll
          for (int a = 0; a < NA; ++a) x[u][a].unpack(f[a]);
#pragma unroll
          for (int i = 0; i < NP; ++i) {
            float& p = PAIRS ? f[0][(2 * i) % V] : f[0][i];
            float& q = PAIRS ? f[0][(2 * i + 1) % V] : f[NA - 1][i];
            const float pr = c[i] * p - n[i] * q, qr = n[i] * p + c[i] * q;
            p = pr;
            q = qr;
          }
          T* to = dst + (size_t)head * dh + group * V;
#pragma unroll
          for (int a = 0; a < NA; ++a) {
            x[u][a].pack(f[a]);
            x[u][a].store(to + a * (rot / 2));
          }
        }
      }
    }
    if (copy) {   // what is not rotated: V, and the rest of every head
      constexpr int N = Vec16<T>::N;
      const int rest = (dh - rot) / N, v0 = rotated * dh;
      for (int i = lane; i < kv_heads * dh / N; i += 64) {
        Vec16<T> w;
        w.load(src + v0 + i * N);
        w.store(dst + v0 + i * N);
      }
      for (int i = lane; i < rotated * rest; i += 64) {
        const int at = (i / rest) * dh + rot + (i % rest) * N;
        Vec16<T> w;
        w.load(src + at);
        w.store(dst + at);
      }
    }
  }
}

template <typename T>
static int rotary_t(int layout, const void* qkv, const int32_t* positions, const double* turns, void* out, int s, int b, int heads, int kv_heads,
                    int dh, int rot, float amplitude, float sign, hipStream_t st) {
  const uint32_t tokens = (uint32_t)s * b;   // below 2^31
  const size_t row = (size_t)(heads + 2 * kv_heads) * dh, moved = out == qkv ? (size_t)(heads + kv_heads) * rot : row;
  Launch L(PTDP_K_OTHER, 2.0 * tokens * moved * sizeof(T), st);
  const uint32_t blocks = (tokens + 3) / 4, cap = 1 << 20;
  const dim3 grid(blocks < cap ? blocks : cap), block(kRotaryThreads);
  constexpr int N = Vec16<T>::N;
#define PTDP_ROTARY(P, V) \
  hipLaunchKernelGGL((rotary_kernel<T, P, V>), grid, block, 0, st, (const T*)qkv, (T*)out, positions, turns, tokens, b, heads, kv_heads, dh, rot, amplitude, sign)
  if (layout == PTDP_ROTARY_PAIRS) PTDP_ROTARY(true, N);
  else if (rot % (2 * N) == 0) PTDP_ROTARY(false, N);
  else PTDP_ROTARY(false, 4);   // bf16 halves that are no whole number of 16 bytes
#undef PTDP_ROTARY
  return L.status();
}

int launch_rotary(int dtype, int layout, const void* qkv, const int32_t* positions, const double* turns, void* out, int s, int b, int heads,
                  int kv_heads, int dh, int rot, float amplitude, bool back, hipStream_t st) {
  const float sign = back ? -1.f : 1.f;
  return dtype == PTDP_BF16 ? rotary_t<bf16_t>(layout, qkv, positions, turns, out, s, b, heads, kv_heads, dh, rot, amplitude, sign, st)
                            : rotary_t<float>(layout, qkv, positions, turns, out, s, b, heads, kv_heads, dh, rot, amplitude, sign, st);
}

}  // namespace ptdp
