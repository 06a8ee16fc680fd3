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

// A slice's partial sums of all heads added up for shared gains.  The sums of slice i go to row i of rows of 2 w, behind the
// rows of all heads.
__global__ void __launch_bounds__(256) k_head_sums(RotaryArgs a) {
  const int heads = a.hq + a.hk;
  const float* const row = a.partial + (size_t)blockIdx.x * heads * a.w;
  float* const out = a.partial + (size_t)gridDim.x * heads * a.w + (size_t)blockIdx.x * 2 * a.w;
  for (int i = threadIdx.x; i < 2 * a.w; i += 256) {
    const bool keys = i >= a.w;
    float sum = 0.f;
    for (int h = keys ? a.hq : 0; h < (keys ? heads : a.hq); ++h) sum += row[h * a.w + (keys ? i - a.w : i)];
    out[i] = sum;
  }
}

// The same for heads of whole, aligned 16-byte pieces whose pairs lie in whole pieces too.  A lane takes one piece of one
// head, 2^lg lanes a head; a workgroup takes `group` heads of `abreast` tokens at a time and U such sets in a row, all their
// loads issued first.  Sine and cosine of the tokens are worked out once for all heads, in LDS.  A lane keeps its head and
// piece, so gains and their gradients stay in registers.  Bound by memory: 4x16384 tokens of 16+4 heads of 128, 671 MB, 129 us,
// 5.2 TB/s (a large copy 4.7); with norm and gradients 32x512 tokens of 16+16 heads of 64, 336 MB, 76 us.  One wavefront per
// head (k_rotary_any) takes 628 and 998 us for the same, its sines and cosines worked out by every head.
template <typename T>
struct Piece {
  static constexpr int CH = 16 / (int)sizeof(T);
};
typedef __attribute__((ext_vector_type(4))) uint32_t raw_t;
template <typename T>
__device__ __forceinline__ void unpack(raw_t r, float (&v)[Piece<T>::CH]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(T) == 2) {
      v[2 * i] = __uint_as_float(r[i] << 16);
      v[2 * i + 1] = __uint_as_float(r[i] & 0xffff0000u);
    } else {
      v[i] = __uint_as_float(r[i]);
    }
  }
}
template <typename T>
__device__ __forceinline__ raw_t pack(const float (&v)[Piece<T>::CH]) {
  raw_t r;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(T) == 2) r[i] = pack_bf16x2(v[2 * i], v[2 * i + 1]);
    else r[i] = __float_as_uint(v[i]);
  }
  return r;
}
__device__ __forceinline__ float row_sum(float v, int lg) {
  for (int o = 1 << lg >> 1; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}

constexpr int MAX_THREADS = 512;
// Sets of tokens whose loads go out together.  With the norm, whose gradient reads two tensors, registers for more wavefronts are worth
// more than more loads of each (32x512 tokens of 16+16 heads of 64, forward and backward: four sets 85 us, two 76, one 78).
constexpr int sets_ahead(bool norm) { return norm ? 2 : 4; }
struct RowsPlan {
  int lg, group, abreast, groups, threads, slices;   // grid: slices x groups
  int flat;                                          // tokens lie at one stride across sequences
};

template <typename T, bool NORM, bool BWD, bool INTER>
__global__ void __launch_bounds__(MAX_THREADS) k_rotary_rows(RotaryArgs a, RowsPlan pl) {
  constexpr int CH = Piece<T>::CH, U = sets_ahead(NORM);
  extern __shared__ __attribute__((aligned(16))) float lds[];
  const int tid = threadIdx.x, lane = tid & 63, c = tid & ((1 << pl.lg) - 1), slot = tid >> pl.lg, heads = a.hq + a.hk;
  const int sub = slot / pl.group, h = blockIdx.y * pl.group + slot % pl.group;
  const bool active = sub < pl.abreast && h < heads && c * CH < a.w;
  const bool isq = h < a.hq;
  const int hh = isq ? h : h - a.hq;
  const FormHeads in = isq ? a.q : a.k, go = isq ? a.gq : a.gk, out = isq ? a.oq : a.ok;
  const T* const xb = reinterpret_cast<const T*>(in.p) + (long long)hh * in.sh + c * CH;
  const T* const gb = reinterpret_cast<const T*>(go.p) + (long long)hh * go.sh + c * CH;
  T* const yb = reinterpret_cast<T*>(const_cast<void*>(out.p)) + (long long)hh * out.sh + c * CH;
  // half layout: the piece with the other element of each pair
  const int half = a.pairs / CH;
  // (the table holds the tokens abreast: not so the lanes that only fill the last wavefront)
  const bool turned = sub < pl.abreast && (INTER ? c * CH < 2 * a.pairs : c < 2 * half), second = !INTER && c >= half;
  const int other = turned && !INTER ? lane + (second ? -half : half) : lane;
  const int trig = INTER ? c * (CH / 2) : (second ? c - half : c) * CH;
  const float sign = (a.inverse != 0) != BWD ? -1.f : 1.f;

  float g[CH], gp[CH], dg[CH];
#pragma unroll
  for (int i = 0; i < CH; ++i) g[i] = gp[i] = 1.f, dg[i] = 0.f;
  if (NORM && active) {
    const float* gain = (isq ? a.gain_q : a.gain_k) + (a.per_head ? hh * a.w : 0);
#pragma unroll
    for (int i = 0; i < CH; ++i) g[i] = gain[c * CH + i], gp[i] = gain[(c + other - lane) * CH + i];
  }
  const float inv_w = 1.f / (float)a.w;
  float* const cos_s = lds;
  float* const sin_s = lds + U * pl.abreast * a.pairs;

  const int tokens = a.B * a.S, TB = U * pl.abreast;
  for (int tok0 = blockIdx.x * TB; tok0 < tokens; tok0 += gridDim.x * TB) {
    raw_t x[U], dy[U];
    long long at[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int tok = tok0 + u * pl.abreast + sub;
      x[u] = raw_t{0, 0, 0, 0};
      if (BWD) dy[u] = x[u];
      if (!active || tok >= tokens) continue;
      const int b = pl.flat ? 0 : tok / a.S, t = tok - b * a.S;
      if (!BWD || NORM) x[u] = *reinterpret_cast<const raw_t*>(xb + b * in.sb + t * in.sr);
      if (BWD) dy[u] = *reinterpret_cast<const raw_t*>(gb + b * go.sb + t * go.sr);
      at[u] = b * out.sb + t * out.sr;
    }
    __syncthreads();         // the table before this one has been read
    for (int i = tid; i < TB * a.pairs; i += blockDim.x) {
      const int k = i / a.pairs, tok = tok0 + k;
      // (rows past the last token are worked on as zeros, so that they add zeros to the sums)
      const float2 cs = tok < tokens ? turn(a, i - k * a.pairs, a.positions ? a.positions[tok] : tok % a.S) : make_float2(0.f, 0.f);
      cos_s[i] = cs.x;
      sin_s[i] = sign * cs.y;
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int tok = tok0 + u * pl.abreast + sub;
      float v[CH], z[CH], r = 1.f;
      unpack<T>(x[u], v);
      if constexpr (NORM) {
        float ss = 0.f;
#pragma unroll
        for (int i = 0; i < CH; ++i) ss = fmaf(v[i], v[i], ss);
        // (0 past the last token: rows of zeros have no norm where eps is 0)
        const float square = fmaf(row_sum(ss, pl.lg), inv_w, a.eps);
        r = tok < tokens ? 1.f / sqrtf(square) : 0.f;
      }
      const raw_t src = BWD ? dy[u] : x[u];
      raw_t osrc;
      if constexpr (!INTER) {
#pragma unroll
        for (int i = 0; i < 4; ++i) osrc[i] = (uint32_t)__shfl((int)src[i], other, 64);
      }
      unpack<T>(src, z);
      if constexpr (NORM && !BWD) {
#pragma unroll
        for (int i = 0; i < CH; ++i) z[i] *= r * g[i];
      }
      if (turned) {
        const float* ct = cos_s + (u * pl.abreast + sub) * a.pairs + trig;
        const float* st = sin_s + (u * pl.abreast + sub) * a.pairs + trig;
        if constexpr (INTER) {
#pragma unroll
          for (int i = 0; i < CH / 2; ++i) {
            const float p = z[2 * i], q = z[2 * i + 1];
            z[2 * i] = fmaf(-q, st[i], p * ct[i]);
            z[2 * i + 1] = fmaf(p, st[i], q * ct[i]);
          }
        } else {
          float o[CH];
          unpack<T>(osrc, o);
#pragma unroll
          for (int i = 0; i < CH; ++i) {
            if constexpr (NORM && !BWD) o[i] *= r * gp[i];
            z[i] = fmaf(second ? o[i] : -o[i], st[i], z[i] * ct[i]);
          }
        }
      }
      if constexpr (NORM && BWD) {
        float mean = 0.f;
#pragma unroll
        for (int i = 0; i < CH; ++i) {
          dg[i] = fmaf(z[i] * v[i], r, dg[i]);
          mean = fmaf(z[i] * g[i], v[i], mean);
        }
        mean = row_sum(mean, pl.lg) * inv_w * r * r;
#pragma unroll
        for (int i = 0; i < CH; ++i) z[i] = r * fmaf(-v[i], mean, z[i] * g[i]);
      }
      if (active && tok < tokens) *reinterpret_cast<raw_t*>(yb + at[u]) = pack<T>(z);
    }
  }
  if constexpr (NORM && BWD) {
    // sums of the workgroup, in the order of its slots: per head over the tokens abreast, of a shared gain over its heads too
    __syncthreads();
    if (c * CH < a.w && sub < pl.abreast)
#pragma unroll
      for (int i = 0; i < CH; ++i) lds[slot * a.w + c * CH + i] = active ? dg[i] : 0.f;
    __syncthreads();
    const int n_slots = pl.group * pl.abreast;
    if (a.per_head) {
      for (int i = tid; i < pl.group * a.w; i += blockDim.x) {
        const int hl = i / a.w;
        float sum = 0.f;
        for (int k = hl; k < n_slots; k += pl.group) sum += lds[k * a.w + i - hl * a.w];
        if (blockIdx.y * pl.group + hl < heads) a.partial[((size_t)blockIdx.x * heads + blockIdx.y * pl.group) * a.w + i] = sum;
      }
    } else {
      for (int i = tid; i < 2 * a.w; i += blockDim.x) {
        const bool keys = i >= a.w;
        const int e = keys ? i - a.w : i;
        float sum = 0.f;
        for (int k = 0; k < n_slots; ++k)
          if ((blockIdx.y * pl.group + k % pl.group >= a.hq) == keys) sum += lds[k * a.w + e];
        a.partial[((size_t)blockIdx.y * gridDim.x + blockIdx.x) * 2 * a.w + i] = sum;
      }
    }
  }
}

// Gradients of the gains from `rows` rows of partial sums, in their order: 64 columns a workgroup, its sixteen wavefronts
// taking every sixteenth row.  per head: a column per element of every head; shared: queries' width, then keys' width.
__global__ void __launch_bounds__(1024) k_gain_sums(RotaryArgs a, const float* __restrict__ partial, int rows, int cols) {
  __shared__ float sum_s[16][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, e = blockIdx.x * 64 + lane;
  float sum = 0.f;
  if (e < cols)
#pragma unroll 8
    for (int i = wave; i < rows; i += 16) sum += partial[(size_t)i * cols + e];
  sum_s[wave][lane] = sum;
  __syncthreads();
  if (wave != 0 || e >= cols) return;
  sum = 0.f;
#pragma unroll
  for (int i = 0; i < 16; ++i) sum += sum_s[i][lane];
  const int nq = a.per_head ? a.hq * a.w : a.w;
  if (e < nq) a.dgain_q[e] = sum;
  else a.dgain_k[e - nq] = sum;
}

bool whole_pieces(const FormHeads& x, const RotaryArgs& a, int heads, int esize) {
  if (!x.p) return true;
  const long long unit = 16 / esize;
  return reinterpret_cast<uintptr_t>(x.p) % 16 == 0 && (a.B == 1 || x.sb % unit == 0) && (a.S == 1 || x.sr % unit == 0) &&
         (heads == 1 || x.sh % unit == 0);
}
bool one_stride(const FormHeads& x, const RotaryArgs& a) { return !x.p || a.B == 1 || x.sb == a.S * x.sr; }

// Workgroups a chip of 256 compute units keeps busy; a slice of tokens beyond that is a turn of the loop.  With gradients of the
// gains fewer, three to a unit, as each leaves a row of partial sums (the same case: 512 workgroups 82 us, 768 76, 1280 82).
int most_slices(bool partial) { return partial ? 768 : 4096; }
RowsPlan plan_rows(const RotaryArgs& a, int esize, bool partial) {
  RowsPlan p{};
  const int pieces = a.w * esize / 16, heads = a.hq + a.hk;
  while ((1 << p.lg) < pieces) ++p.lg;
  const int most = MAX_THREADS >> p.lg;
  p.groups = (heads + most - 1) / most;
  p.group = (heads + p.groups - 1) / p.groups;
  const long long tokens = (long long)a.B * a.S;
  p.abreast = (256 >> p.lg) / p.group;
  if (p.abreast < 1) p.abreast = 1;
  while (p.abreast > 1 && (long long)p.abreast > tokens) --p.abreast;
  p.threads = ((p.group * p.abreast << p.lg) + 63) / 64 * 64;
  const int ahead = sets_ahead(a.gain_q != nullptr);
  const long long sets = (tokens + ahead * p.abreast - 1) / (ahead * p.abreast);
  const int limit = most_slices(partial) / p.groups > 1 ? most_slices(partial) / p.groups : 1;
  p.slices = (int)(sets < limit ? sets : limit);
  p.flat = one_stride(a.q, a) && one_stride(a.k, a) && one_stride(a.gq, a) && one_stride(a.gk, a) && one_stride(a.oq, a) && one_stride(a.ok, a);
  return p;
}
int token_slices(long long tokens) { return (int)(tokens < 512 ? tokens : 512); }

template <typename T, bool NORM, bool BWD>
hipError_t rows_t(const RotaryArgs& a, const RowsPlan& p, hipStream_t s) {
  const int trig = 2 * sets_ahead(NORM) * p.abreast * a.pairs, sums = NORM && BWD ? p.group * p.abreast * a.w : 0;
  const int lds = (trig > sums ? trig : sums) * (int)sizeof(float);
  const dim3 grid((unsigned)p.slices, (unsigned)p.groups), block((unsigned)p.threads);
  if (a.interleaved) k_rotary_rows<T, NORM, BWD, true><<<grid, block, lds, s>>>(a, p);
  else k_rotary_rows<T, NORM, BWD, false><<<grid, block, lds, s>>>(a, p);
  return hipGetLastError();
}
template <typename T>
hipError_t run_t(const RotaryArgs& a, bool backward, hipStream_t s) {
  constexpr int E = (int)sizeof(T);
  const int heads = a.hq + a.hk;
  const bool norm = a.gain_q != nullptr, rows = a.w % (16 / E) == 0 && a.pairs % (a.interleaved ? 8 / E : 16 / E) == 0 &&
                    whole_pieces(a.q, a, a.hq, E) && whole_pieces(a.k, a, a.hk, E) && whole_pieces(a.gq, a, a.hq, E) &&
                    whole_pieces(a.gk, a, a.hk, E) && whole_pieces(a.oq, a, a.hq, E) && whole_pieces(a.ok, a, a.hk, E);
  int slices = token_slices((long long)a.B * a.S), sums = slices, cols = heads * a.w;
  size_t first = 0;
  if (rows) {
    const RowsPlan p = plan_rows(a, E, backward);
    const hipError_t e = !norm ? rows_t<T, false, false>(a, p, s) : backward ? rows_t<T, true, true>(a, p, s) : rows_t<T, true, false>(a, p, s);
    if (e != hipSuccess || !backward) return e;
    sums = a.per_head ? p.slices : p.slices * p.groups;
    cols = a.per_head ? cols : 2 * a.w;
  } else {
    const dim3 grid((unsigned)slices, (unsigned)((heads + 3) / 4)), block(256);
    if (!norm) k_rotary_any<T, false, false><<<grid, block, 0, s>>>(a);
    else if (!backward) k_rotary_any<T, true, false><<<grid, block, 0, s>>>(a);
    else k_rotary_any<T, true, true><<<grid, block, 0, s>>>(a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || !backward) return e;
    if (!a.per_head) {        // the heads of a slice first
      k_head_sums<<<dim3((unsigned)slices), block, 0, s>>>(a);
      first = (size_t)slices * cols;
      cols = 2 * a.w;
    }
  }
  k_gain_sums<<<dim3((unsigned)((cols + 63) / 64)), dim3(1024), 0, s>>>(a, a.partial + first, sums, cols);
  return hipGetLastError();
}

}  // namespace

size_t rotary_partial_floats(long long tokens, int heads, int w) {
  // every kernel's rows: per head and slice, behind them two widths a slice, or two widths for each of the slices and groups
  const size_t slices = (size_t)(tokens < most_slices(true) ? tokens : most_slices(true));
  const size_t any = (size_t)token_slices(tokens) * (heads + 2) * w, each = slices * heads * w, rows = (size_t)(most_slices(true) + heads) * 2 * w;
  return any > each ? (any > rows ? any : rows) : (each > rows ? each : rows);
}
hipError_t rotary_run(int dtype, const RotaryArgs& a, bool backward, hipStream_t s) {
  return dtype ? run_t<bf16>(a, backward, s) : run_t<float>(a, backward, s);
}

}  // namespace mslt
