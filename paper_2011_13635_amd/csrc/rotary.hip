// Rotary positions of queries and keys, alone or behind the norm of each head, and the gradients.
//
// Pair i turns by pos * f_i.  The angle is kept in turns as a 64-bit fraction: f_i in units of 2^-64 turns times the
// position, modulo 2^64, is the exact fractional turn of the rounded frequency at any position (error pos * 2^-65), where
// an fp32 product would have lost its digits (pos 1e6: 2^-4 radians).  What is left goes to sine and cosine in fp32.
//
// Norm: z = x r g, r = (mean x^2 + eps)^-1/2.  Its gradient, with dz the turned-back gradient of the output:
// dg = sum dz x r;  dx = r (g dz - x r^2 mean(g dz x)).  r is computed again from x, which has to be read anyway.
// All of it in fp32, rounded once on store.
#include "common.h"

namespace mslt {

namespace {

constexpr int MAX_W = 256;

__device__ __forceinline__ float2 turn(const RotaryArgs& a, int pair, int pos) {
  const long long t = (long long)(a.freq[pair] * (unsigned long long)(long long)pos);
  float s, c;
  sincospif((float)(int)(t >> 32) * 0x1p-31f, &s, &c);
  return make_float2(c * a.magnitude, s * a.magnitude);
}

template <typename T>
__device__ __forceinline__ const T* row_ptr(const FormHeads& x, int b, int t, int h) {
  return reinterpret_cast<const T*>(x.p) + (long long)b * x.sb + (long long)t * x.sr + (long long)h * x.sh;
}

// One wavefront per head of a token, any width, any alignment; elements lane, lane + 64, ... of the head.
// grid: token slices x groups of four heads (queries first); a wavefront keeps its head, so the gain's gradient stays in
// registers until the end of its slice.
template <typename T, bool NORM, bool BWD>
__global__ void __launch_bounds__(256) k_rotary_any(RotaryArgs a) {
  __shared__ float row_s[4][MAX_W];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, heads = a.hq + a.hk;
  const int h = blockIdx.y * 4 + wave;
  if (h >= heads) return;                   // (whole wavefronts; the shared row is a wavefront's own)
  const bool isq = h < a.hq;
  const int hh = isq ? h : h - a.hq;
  const FormHeads &in = isq ? a.q : a.k, &go = isq ? a.gq : a.gk, &out = isq ? a.oq : a.ok;
  const float* gain = isq ? a.gain_q : a.gain_k;
  float* const row = row_s[wave];
  float g[4], dg[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int e = lane + 64 * i;
    g[i] = NORM && e < a.w ? gain[(a.per_head ? hh * a.w : 0) + e] : 1.f;
    dg[i] = 0.f;
  }
  const long long tokens = (long long)a.B * a.S;
  const float sign = a.inverse != BWD ? -1.f : 1.f;
  for (long long tok = blockIdx.x; tok < tokens; tok += gridDim.x) {
    const int b = (int)(tok / a.S), t = (int)(tok % a.S), pos = a.positions ? a.positions[tok] : t;
    const T* x = row_ptr<T>(in, b, t, hh);
    T* const y = const_cast<T*>(row_ptr<T>(out, b, t, hh));
    float v[4], r = 1.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = lane + 64 * i < a.w ? ldf(x + lane + 64 * i) : 0.f;
    if constexpr (NORM) {
      float ss = 0.f;
#pragma unroll
      for (int i = 0; i < 4; ++i) ss = fmaf(v[i], v[i], ss);
      r = 1.f / sqrtf(wave_sum(ss) / (float)a.w + a.eps);
    }
    const T* src = BWD ? row_ptr<T>(go, b, t, hh) : x;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int e = lane + 64 * i;
      if (e < a.w) row[e] = BWD ? ldf(src + e) : v[i] * r * g[i];
    }
    __builtin_amdgcn_wave_barrier();
    float z[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int e = lane + 64 * i;
      z[i] = 0.f;
      if (e >= a.w) continue;
      z[i] = row[e];
      if (e >= 2 * a.pairs) continue;
      const int pair = a.interleaved ? e >> 1 : e < a.pairs ? e : e - a.pairs;
      const bool second = a.interleaved ? e & 1 : e >= a.pairs;
      const float other = row[a.interleaved ? e ^ 1 : second ? e - a.pairs : e + a.pairs];
      const float2 cs = turn(a, pair, pos);
      z[i] = fmaf(second ? other : -other, sign * cs.y, z[i] * cs.x);
    }
    __builtin_amdgcn_wave_barrier();
    if constexpr (NORM && BWD) {
      float mean = 0.f;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        dg[i] = fmaf(z[i] * v[i], r, dg[i]);
        mean = fmaf(z[i] * g[i], v[i], mean);
      }
      mean = wave_sum(mean) / (float)a.w * r * r;
#pragma unroll
      for (int i = 0; i < 4; ++i) z[i] = r * fmaf(-v[i], mean, z[i] * g[i]);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (lane + 64 * i < a.w) stf(y + lane + 64 * i, z[i]);
  }
  if constexpr (NORM && BWD) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (lane + 64 * i < a.w) a.partial[((size_t)blockIdx.x * heads + h) * a.w + lane + 64 * i] = dg[i];
  }
}

// Gradient of a gain from the slices' sums, in their order: one workgroup for 64 elements of one head, or of a shared gain.
__global__ void __launch_bounds__(256) k_gain_sums(RotaryArgs a, int slices) {
  __shared__ float sum_s[4][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, heads = a.hq + a.hk, e = blockIdx.x * 64 + lane;
  const int which = blockIdx.y;             // per head: the head; else 0 queries, 1 keys
  const bool isq = a.per_head ? which < a.hq : which == 0;
  const int h0 = a.per_head ? which : isq ? 0 : a.hq, nh = a.per_head ? 1 : isq ? a.hq : a.hk;
  float sum = 0.f;
  if (e < a.w)
    for (int i = wave; i < slices * nh; i += 4) sum += a.partial[((size_t)(i / nh) * heads + h0 + i % nh) * a.w + e];
  sum_s[wave][lane] = sum;
  __syncthreads();
  if (wave == 0 && e < a.w) {
    float* const out = isq ? a.dgain_q : a.dgain_k;
    out[(a.per_head ? (isq ? which : which - a.hq) * a.w : 0) + e] = (sum_s[0][lane] + sum_s[1][lane]) + (sum_s[2][lane] + sum_s[3][lane]);
  }
}

int token_slices(long long tokens) { return (int)(tokens < 512 ? tokens : 512); }

template <typename T>
hipError_t run_t(const RotaryArgs& a, bool backward, hipStream_t s) {
  const int heads = a.hq + a.hk, slices = token_slices((long long)a.B * a.S);
  const dim3 grid((unsigned)slices, (unsigned)((heads + 3) / 4)), block(256);
  if (!a.gain_q) k_rotary_any<T, false, false><<<grid, block, 0, s>>>(a);
  else if (!backward) k_rotary_any<T, true, false><<<grid, block, 0, s>>>(a);
  else {
    k_rotary_any<T, true, true><<<grid, block, 0, s>>>(a);
    k_gain_sums<<<dim3((unsigned)((a.w + 63) / 64), (unsigned)(a.per_head ? heads : a.hk ? 2 : 1)), block, 0, s>>>(a, slices);
  }
  return hipGetLastError();
}

}  // namespace

size_t rotary_partial_floats(long long tokens, int heads, int w) { return (size_t)token_slices(tokens) * heads * w; }
hipError_t rotary_run(int dtype, const RotaryArgs& a, bool backward, hipStream_t s) {
  return dtype ? run_t<bf16>(a, backward, s) : run_t<float>(a, backward, s);
}

}  // namespace mslt
