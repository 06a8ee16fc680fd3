// The bf16 kernels of attention_forms.h, and what both precisions share.
#include "attention_forms.h"

namespace mslt {

// Least and largest document entry of every 64 positions, one wavefront each.
__global__ void __launch_bounds__(256) k_doc_ranges(const int32_t* __restrict__ docs, int2* __restrict__ ranges, int B, int S) {
  const int per = (S + 63) / 64, lane = threadIdx.x & 63;
  const long long i = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (i >= (long long)B * per) return;
  const int b = (int)(i / per), at = (int)(i % per) * 64 + lane;
  const int v = docs[(size_t)b * S + min(at, S - 1)];
  const int lo = forms::wave_min_i(v), hi = forms::wave_max_i(v);
  if (lane == 0) ranges[i] = make_int2(lo, hi);
}
hipError_t form_ranges(const FormArgs& a, hipStream_t s) {
  if (!a.docs) return hipSuccess;
  const long long blocks = (long long)a.B * ((a.S + 63) / 64);
  k_doc_ranges<<<dim3((unsigned)((blocks + 3) / 4)), dim3(256), 0, s>>>(a.docs, a.ranges, a.B, a.S);
  return hipGetLastError();
}

// The keys are split only where the workgroups of whole rows leave the chip's 256 compute units short of two each.
int form_splits(int dtype, int B, int n, int S, int nh, int nkv, int w) {
  (void)dtype;
  (void)w;
  const long long rows = (long long)n * (nh / nkv);
  const bool few = rows <= 32;
  const long long blocks = (long long)B * nkv * (few ? 1 : (rows + 127) / 128);
  const int tiles = few ? (S + 127) / 128 : (S + 63) / 64;
  const long long want = (512 + blocks - 1) / blocks, most = few ? tiles : tiles / 8;
  const long long splits = want < most ? want : most;
  return blocks >= 256 || splits < 1 ? 1 : (int)splits;
}

// The key side's workgroups take 128 keys each; below two for each of 256 compute units (causal: the first keys' are the longest)
// the rows are split, as far as every part keeps eight tiles of 64.
int form_row_splits(int B, int n, int S, int nh, int nkv) {
  const long long blocks = (long long)B * nkv * ((S + 127) / 128), tiles = (long long)n * (nh / nkv) / 64;
  const long long want = (512 + blocks - 1) / blocks, most = tiles / 8;
  const long long splits = want < most ? want : most;
  return splits < 1 ? 1 : (int)splits;
}
namespace forms {
bool wide_rows(bool b16, int w, size_t heads, int rows) { return b16 && w > 64 && heads * ((size_t)rows / 256) >= 256; }
}  // namespace forms

hipError_t form_fwd_bf16(const FormArgs& a, hipStream_t s) { return forms::fwd_t<bf16>(a, s); }
hipError_t form_bwd_bf16(const FormArgs& a, hipStream_t s) { return forms::bwd_t<bf16>(a, s); }

}  // namespace mslt
