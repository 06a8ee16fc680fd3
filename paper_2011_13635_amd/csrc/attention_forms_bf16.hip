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
  if (!a.docs || (a.S + 63) / 64 <= FORM_OWN_RANGES) return hipSuccess;
  const long long blocks = (long long)a.B * ((a.S + 63) / 64);
  k_doc_ranges<<<dim3((unsigned)((blocks + 3) / 4)), dim3(256), 0, s>>>(a.docs, a.ranges, a.B, a.S);
  return hipGetLastError();
}

namespace forms {
// 128 rows a workgroup leave 256 compute units idle below 256 of them; 256 rows a workgroup read the keys half as often.
RowMode row_mode(bool wide, size_t heads, int rows) {
  if (heads * (((size_t)rows + 127) / 128) < 256) return ROWS_FEW;
  return wide && heads * ((size_t)rows / 256) >= 256 ? ROWS_EIGHT : ROWS_FOUR;
}
}  // namespace forms

// The keys are split where even 32 rows a workgroup come to fewer than 256 workgroups, as far as every part keeps two tiles.
int form_splits(int B, int n, int S, int nh, int nkv) {
  const long long rows = (long long)n * (nh / nkv), heads = (long long)B * nkv, blocks = heads * ((rows + 31) / 32);
  if (blocks >= 256 || forms::row_mode(false, (size_t)heads, (int)rows) != forms::ROWS_FEW) return 1;
  const long long want = (512 + blocks - 1) / blocks, most = (S + 127) / 256;
  const long long splits = want < most ? want : most;
  return splits < 1 ? 1 : (int)splits;
}
// The key side's workgroups take 128 keys each, or 32; below two for each of 256 compute units the rows are split, as far as every
// part keeps eight tiles (causal: the first keys have the most rows, so that one workgroup for each unit would not do).
int form_row_splits(int B, int n, int S, int nh, int nkv) {
  const bool few = forms::row_mode(false, (size_t)B * nkv, S) == forms::ROWS_FEW;
  const long long blocks = (long long)B * nkv * (few ? (S + 31) / 32 : (S + 127) / 128), tiles = (long long)n * (nh / nkv) / (few ? 128 : 64);
  const long long want = (512 + blocks - 1) / blocks, most = tiles / 8;
  const long long splits = want < most ? want : most;
  return splits < 1 ? 1 : (int)splits;
}

hipError_t form_fwd_bf16(const FormArgs& a, hipStream_t s) { return forms::fwd_t<bf16>(a, s); }
hipError_t form_bwd_bf16(const FormArgs& a, hipStream_t s) { return forms::bwd_t<bf16>(a, s); }

}  // namespace mslt
