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
  // a workgroup's share: where keys are split, whole tiles of 128
  const int most = a.splits > 1 ? 2 * (((a.S + 127) / 128 + a.splits - 1) / a.splits) : (a.S + 63) / 64;
  if (!a.docs || most <= FORM_OWN_RANGES) return hipSuccess;
  const long long blocks = (long long)a.B * ((a.S + 63) / 64);
  k_doc_ranges<<<dim3((unsigned)((blocks + 3) / 4)), dim3(256), 0, s>>>(a.docs, a.ranges, a.B, a.S);
  return hipGetLastError();
}

namespace forms {
// Below so many workgroups of 128 rows (keys) they are dealt out 32 at a time: 128 rows leave compute units idle, or with one
// workgroup and so one wavefront to a SIMD.  Width 64, 1x2048x16 heads (256 workgroups of 128): causal forward 48 -> 35 us, backward
// 113 -> 94, with everything visible 52 -> 56 and 137 -> 140.  At width 128 a workgroup of 32 keys or rows keeps one wavefront to a
// SIMD anyway: 1x2048x16 forward 61 -> 67, 66 -> 109.
RowMode row_mode(bool wide, int w, size_t heads, int rows) {
  if (heads * (((size_t)rows + 127) / 128) < (w <= 64 ? 512u : 256u)) return ROWS_FEW;
  return wide && heads * ((size_t)rows / 256) >= 256 ? ROWS_EIGHT : ROWS_FOUR;
}
// The key side at width 128 can split the rows instead (form_row_splits): 128 workgroups of 128 keys, 4x512x8 heads: 75 us against
// 89 with 32 keys each, 1x4096 over 4: 664 against 872; but 64 workgroups, 1x1024x8 heads: 80 against 70.
// Up to 32 keys there is no more than one block of 32, whatever the batch, and four wavefronts share its rows.
bool few_keys(int w, size_t heads, int keys) { return keys <= FINE || heads * (((size_t)keys + 127) / 128) < (w <= 64 ? 512u : 96u); }
}  // namespace forms

// The keys are split where even 32 rows a workgroup come to fewer than 256 workgroups, as far as every part keeps two tiles.
int form_splits(int B, int n, int S, int nh, int nkv, int w) {
  const long long rows = (long long)n * (nh / nkv), heads = (long long)B * nkv, blocks = heads * ((rows + 31) / 32);
  if (blocks >= 256 || forms::row_mode(false, w, (size_t)heads, (int)rows) != forms::ROWS_FEW) return 1;
  const long long want = (512 + blocks - 1) / blocks, most = (S + 127) / 256;
  const long long splits = want < most ? want : most;
  return splits < 1 ? 1 : (int)splits;
}
// The key side's workgroups take 128 keys each, or 32; below four for each of 256 compute units the rows are split, as far as every
// part keeps eight tiles: with causal the first keys have the most rows (1x4096, 16 heads of 64 over 4: 293 us split to two for
// each unit, 252 to four; 400 and 410 with everything visible).
int form_row_splits(int B, int n, int S, int nh, int nkv, int w) {
  const bool few = forms::few_keys(w, (size_t)B * nkv, S);
  const long long blocks = (long long)B * nkv * (few ? (S + 31) / 32 : (S + 127) / 128), tiles = (long long)n * (nh / nkv) / (few ? 128 : 64);
  const long long want = (1024 + blocks - 1) / blocks, most = tiles / 8;
  const long long splits = want < most ? want : most;
  return splits < 1 ? 1 : (int)splits;
}

hipError_t form_fwd_bf16(const FormArgs& a, hipStream_t s) { return forms::fwd_t<bf16>(a, s); }
hipError_t form_bwd_bf16(const FormArgs& a, hipStream_t s) { return forms::bwd_t<bf16>(a, s); }

}  // namespace mslt
