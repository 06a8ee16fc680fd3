// Attention with a score cap, a distance bias, a document mask and a prefix mask, grouped key/value heads; bf16 and fp32.
//
//   s = scale q.k;  s <- cap tanh(s / cap);  s <- s - slope |pos_q - pos_k|;  p = softmax of s over the visible keys;  o = p v
//
// One pass over the keys with a running maximum and sum, in base 2 (log2 e folded into the factors).  The query heads that
// share a key/value head are rows of the same tile: row R of a kv head is query R / G of head R % G of its group, so a key
// or value is read once for all of them and the gradients of a shared head add up in registers, in a fixed order.
//
// All products are 32 x 32 matrix instructions formed transposed, so that the softmax index sits in a lane's registers:
//   S^T[key, row] = K Q^T, O^T[d, row] = V^T P^T (lane = row);  backward likewise for dQ; for dK, dV lane = key, registers = rows.
// An accumulator is the B operand of the next product as it stands; the A operand (V^T, K^T, Q^T, dO^T) is read transposed
// out of the same LDS tile that the first product reads by rows.
//
// Which tiles a workgroup visits: tiles that no row of it can see are left out.  For documents, the least and largest
// entry of every 64 positions are found first (doc_ranges); each workgroup turns them and the position limits into a
// list of tiles.  A wavefront masks element by element only in tiles that are neither hidden from all its rows nor open
// to all of them.
#pragma once
#include "common.h"

#include <atomic>

namespace mslt {
namespace forms {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8_t;
typedef __attribute__((ext_vector_type(16))) float f32x16_t;
typedef __attribute__((ext_vector_type(4))) float f32x4_t;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4_t;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2_t;
typedef __attribute__((ext_vector_type(4))) short s16x4_t;
typedef __attribute__((address_space(3))) s16x4_t lds_s16x4_t;

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
constexpr int LIST = 256;            // tiles listed at a time, one per thread
constexpr float NO_MAX = -1e30f;     // running maximum before the first visible key: finite, so that differences are
__device__ __forceinline__ f32x16_t zero16() {
  f32x16_t z;
#pragma unroll
  for (int r = 0; r < 16; ++r) z[r] = 0.f;
  return z;
}
// row of a 32-row block that register r of this half-wave holds, without the 4 * half
__device__ __forceinline__ constexpr int acc_row(int r) { return 8 * (r >> 2) + (r & 3); }
// Least and largest of the 64 lanes' values, by moves between neighbouring lanes (a shuffle through LDS takes some 70 cycles, a move
// eight): within four, rows of sixteen, then across the rows; lane 63 holds the result.
template <typename F>
__device__ __forceinline__ int wave_reduce_i(int v, F f) {
  v = f(v, __builtin_amdgcn_update_dpp(v, v, 0x111, 0xf, 0xf, false));     // row_shr:1, 2, 4, 8
  v = f(v, __builtin_amdgcn_update_dpp(v, v, 0x112, 0xf, 0xf, false));
  v = f(v, __builtin_amdgcn_update_dpp(v, v, 0x114, 0xf, 0xf, false));
  v = f(v, __builtin_amdgcn_update_dpp(v, v, 0x118, 0xf, 0xf, false));
  v = f(v, __builtin_amdgcn_update_dpp(v, v, 0x142, 0xa, 0xf, false));     // row_bcast:15, 31
  v = f(v, __builtin_amdgcn_update_dpp(v, v, 0x143, 0xc, 0xf, false));
  return __builtin_amdgcn_readlane(v, 63);
}
__device__ __forceinline__ int wave_min_i(int v) {
  return wave_reduce_i(v, [](int x, int y) { return min(x, y); });
}
__device__ __forceinline__ int wave_max_i(int v) {
  return wave_reduce_i(v, [](int x, int y) { return max(x, y); });
}

// LDS tile of rows of D elements in 16-byte chunks; chunk c of a row sits in place c ^ swz(row).  The order makes both
// ways of reading free of bank conflicts: 16 rows at one chunk (first products), and four consecutive rows at four
// neighbouring chunks (transposed bf16 reads) or two rows four apart at 32 consecutive floats (fp32).
template <typename T, int D>
struct Tile {
  static constexpr int CH = 16 / (int)sizeof(T);
  static constexpr int CPR = D / CH;
  static constexpr int ROWB = D * (int)sizeof(T);
  static constexpr int NS = CPR / 2;     // 16-byte fragments of a row that one half-wave holds
  static __device__ __forceinline__ int swz(int row) {
    if constexpr (sizeof(T) == 4) return (row & 3) | (((row >> 2) & 1) << 3) | (((row >> 3) & 1) << 2);
    else if constexpr (CPR == 8) return (((row >> 1) & 1) << 2) | ((row >> 2) & 3);
    else return ((row & 3) << 2) | ((row >> 2) & 3);
  }
  static __device__ __forceinline__ u32x4_t* at(unsigned char* lds, int row, int chunk) {
    return reinterpret_cast<u32x4_t*>(lds + row * ROWB + 16 * (chunk ^ swz(row)));
  }
};

// a lane's 16-byte pieces of one row: half-wave h holds chunks 2 s + h
template <typename T, int D>
using Frags = u32x4_t[Tile<T, D>::NS];

template <typename T>
__device__ __forceinline__ f32x16_t mma(u32x4_t a, u32x4_t b, f32x16_t acc) {
  if constexpr (sizeof(T) == 2) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), acc, 0, 0, 0);
  } else {
    const f32x4_t x = __builtin_bit_cast(f32x4_t, a), y = __builtin_bit_cast(f32x4_t, b);
#pragma unroll
    for (int j = 0; j < 4; ++j) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(x[j], y[j], acc, 0, 0, 0);
    return acc;
  }
}
// LDS addresses.  A lane's address in a tile is its lane part plus the tile's, and a constant of the step over it (exclusive or,
// where the step changes the chunk; a tile's address is a multiple of its row): one instruction for a read, and two registers
// of addresses in all.  Kept in a register each, the addresses of all steps cost the accumulators' room.
template <typename V>
__device__ __forceinline__ V lds_read(uint32_t addr) {
  return *reinterpret_cast<const __attribute__((address_space(3))) V*>((uintptr_t)addr);
}
__device__ __forceinline__ uint32_t lds_addr(const void* p) {
  return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void*)p;
}
constexpr int TILE_ALIGN = 512;      // of every tile in LDS: the longest row
template <typename T, int D>
struct Lane {
  uint32_t rows, cols;     // parts of a read by rows (first products), and of one by columns (second products)
  __device__ __forceinline__ explicit Lane(int lane) {
    using L = Tile<T, D>;
    const int n = lane & 31, half = lane >> 5;
    rows = n * L::ROWB + 16 * (half ^ L::swz(n));
    if constexpr (sizeof(T) == 2) {
      // sixteen lanes fetch four consecutive rows of sixteen d and receive four rows of one d each
      const int j = lane & 15, blk = (lane >> 4) & 1, row = 4 * half + (j >> 2);
      cols = row * L::ROWB + 16 * ((2 * blk + ((j & 3) >> 1)) ^ L::swz(row)) + 8 * (j & 1);
    } else {
      cols = 4 * half * L::ROWB + 16 * ((n >> 2) ^ (half << 3)) + 4 * (n & 3);
    }
  }
};
// [32 tile rows from row0] x [fragment rows]: lane = fragment row, registers = tile rows
template <typename T, int D>
__device__ __forceinline__ f32x16_t dot_rows(uint32_t tile, int row0, const Frags<T, D>& f, const Lane<T, D>& l, f32x16_t acc = zero16()) {
  const uint32_t at = tile + l.rows;
#pragma unroll
  for (int s = 0; s < Tile<T, D>::NS; ++s) acc = mma<T>(lds_read<u32x4_t>((at ^ (32 * s)) + row0 * Tile<T, D>::ROWB), f[s], acc);
  return acc;
}
// the same with the fragments read out of a second tile's rows
template <typename T, int D>
__device__ __forceinline__ f32x16_t dot_tiles(uint32_t tile, int row0, uint32_t other, const Lane<T, D>& l, f32x16_t acc = zero16()) {
  const uint32_t at = tile + l.rows, to = other + l.rows;
#pragma unroll
  for (int s = 0; s < Tile<T, D>::NS; ++s)
    acc = mma<T>(lds_read<u32x4_t>((at ^ (32 * s)) + row0 * Tile<T, D>::ROWB), lds_read<u32x4_t>(to ^ (32 * s)), acc);
  return acc;
}
// How N times EACH matrix instructions (bf16), each of those fed by READS reads of LDS, are ordered: the reads of the first two go
// out first, then each is followed by those of one further on.  Left to itself the compiler reads right before use where
// registers are short, and a wavefront waits for LDS before every instruction (backward at 1x8192x16 heads of 128: 2.87 ms, so
// 2.57; the forward and width 64 do not care).
template <typename T, int N, int READS, int EACH>
__device__ __forceinline__ void feed() {
  if constexpr (sizeof(T) == 2) {
    constexpr int A = N < 2 ? N : 2;
    __builtin_amdgcn_sched_group_barrier(0x100, A * READS, 0);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x008, EACH, 0);
      if (i + A < N) __builtin_amdgcn_sched_group_barrier(0x100, READS, 0);
    }
  }
}
// registers 8c .. 8c+7 as a B operand
__device__ __forceinline__ bf16x8_t pack_frag(const f32x16_t& p, int c) {
  u32x4_t u;
#pragma unroll
  for (int i = 0; i < 4; ++i) u[i] = pack_bf16x2(p[8 * c + 2 * i], p[8 * c + 2 * i + 1]);
  return __builtin_bit_cast(bf16x8_t, u);
}
// bf16: rows row0 + 16c + 8i + 4half + 0 .. 3, i = 0, 1, of a tile at d = 32 db + lane % 32
template <int D>
__device__ __forceinline__ bf16x8_t frag_transposed(uint32_t tile, int row0, int c, int db, const Lane<bf16, D>& l) {
  const uint32_t at = tile + l.cols;
  s16x4_t v[2];
#pragma unroll
  for (int i = 0; i < 2; ++i)
    v[i] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t*)(uintptr_t)((at ^ (64 * db + 32 * i)) + (row0 + 16 * c + 8 * i) * Tile<bf16, D>::ROWB));
  struct { s16x4_t lo, hi; } w{v[0], v[1]};
  return __builtin_bit_cast(bf16x8_t, w);
}
// acc[d, lane's column] += sum over 32 tile rows from row0 of tile[row][d] * p[row, column].  bf16: p is rounded to bf16
// here, the one rounding between the two products (the sum of a row is taken before it); a term is then off by half a step,
// 2^-8 of itself, as the operands of the first product already are.  Results are off by 2.0e-3 to 2.4e-3 (root of the mean square,
// listed training shapes), of which their own rounding alone is 1.66e-3.  A second part of what is rounded off, as lost() gives it, takes
// them to 1.66e-3 and costs up to a quarter: forward 1x8192x12 heads of 64 390 -> 474 us, 1x8192x16 of 128 353 -> 442, 64x128x16 18.6 -> 21.2;
// backward 1300 -> 1570, 32x512x16 218 -> 251, 64x128x16 45 -> 47.  Callers that need it have fp32 operands.
template <int D>
__device__ __forceinline__ void add_packed(f32x16_t (&acc)[D / 32], uint32_t tile, int row0, const bf16x8_t (&f)[2], const Lane<bf16, D>& l) {
#pragma unroll
  for (int c = 0; c < 2; ++c)
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
      acc[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag_transposed<D>(tile, row0, c, db, l), f[c], acc[db], 0, 0, 0);
}
template <typename T, int D>
__device__ __forceinline__ void add_outer(f32x16_t (&acc)[D / 32], uint32_t tile, int row0, const f32x16_t& p, const Lane<T, D>& l) {
  if constexpr (sizeof(T) == 2) {
    const bf16x8_t f[2] = {pack_frag(p, 0), pack_frag(p, 1)};
    add_packed<D>(acc, tile, row0, f, l);
  } else {
    // The reads of the next two rows are on their way while those at hand are multiplied; left to itself the compiler waits for each
    // read in turn (4x1024x8 heads of 64: forward 96 -> 88 us, backward 322 -> 292).
    const uint32_t at = tile + l.cols;
    float x[2][2][D / 32];
    auto read = [&](int g) {
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int db = 0; db < D / 32; ++db) {
          const int r = 2 * g + i;
          x[g & 1][i][db] = lds_read<float>((at ^ (16 * (8 * db + (r & 3) + ((r >> 2) & 1) * 4))) + (row0 + acc_row(r)) * Tile<T, D>::ROWB);
        }
    };
    read(0);
#pragma unroll
    for (int g = 0; g < 8; ++g) {
      if (g + 1 < 8) read(g + 1);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int db = 0; db < D / 32; ++db) acc[db] = __builtin_amdgcn_mfma_f32_32x32x2f32(x[g & 1][i][db], p[2 * g + i], acc[db], 0, 0, 0);
    }
  }
}
// What rounding to bf16 took off, for a second product.  The roundings of a row's terms average out over many keys; over few, and
// with terms that cancel, the gradient would be off by more than its own rounding.  Sequences of up to 32 keys, whose time is that of
// a launch, take it along (1x32x4 heads of 64, backward: 7.1 -> 7.5 us; 2x4 keys, dQ: 2.5e-3 -> 1.6e-3 off, its own rounding), in
// batches of any size: which kernels may take up to FINE keys have it (SHORT).
constexpr int FINE = 32;
__device__ __forceinline__ f32x16_t lost(const f32x16_t& p) {
  f32x16_t r;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t u = pack_bf16x2(p[2 * i], p[2 * i + 1]);
    r[2 * i] = p[2 * i] - __uint_as_float(u << 16);
    r[2 * i + 1] = p[2 * i + 1] - __uint_as_float(u & 0xffff0000u);
  }
  return r;
}
// two such products of the same tile (bf16)
template <typename T, int D>
__device__ __forceinline__ void add_outer2(f32x16_t (&x)[D / 32], f32x16_t (&y)[D / 32], uint32_t tile, int row0, const f32x16_t& p,
                                           const f32x16_t& q, const Lane<T, D>& l) {
#pragma unroll
  for (int c = 0; c < 2; ++c) {
    const bf16x8_t f = pack_frag(p, c), g = pack_frag(q, c);
#pragma unroll
    for (int db = 0; db < D / 32; ++db) {
      const bf16x8_t t = frag_transposed<D>(tile, row0, c, db, l);
      x[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(t, f, x[db], 0, 0, 0);
      y[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(t, g, y[db], 0, 0, 0);
    }
  }
}

// Score in base 2 from the product x of a query and a key, and what the gradient is multiplied by behind the cap.
// tanh y = 1 - 2 / (1 + e^2y): absolute error a few 2^-24 for any y, and the score's is cap times that.  Up to six tenths of the cap,
// y (c0 + c1 y^2 + .. + c4 y^8) is nearer and faster, six multiply-adds in place of two transcendental instructions (8.4 cycles each
// against 3) and three more; fitted to the least largest error relative to y, 7.4e-8.
// Caps so far above the scale that c4's factor falls below the least fp32: within a twentieth, where c3 y^6 adds less than 2^-29.
// Where a score of a wavefront's block of 32 x 32 lies beyond, each takes its own formula in fp32, so that no score loses digits to its
// neighbours (cap 20 and scores of 6 typically: 4x1024x8 heads of 64, forward 98 -> 102 us, backward 318 -> 329).  In bf16 all take
// the first one as long as its error, 3 2^-24 of a cap below 2^10 in base 2, stays a tenth of the half step that probabilities are
// rounded by (1x8192x12 heads of 64: 452 us, each its own 550).
constexpr float SHARED_CAP = 0x1p10f;
struct Score {
  float a, c;              // no cap: s2 = a x.  cap: s2 = c tanh, exponent a x
  float p[5], reach;       // s2 = x (p0 + p1 x^2 + ...) for |x| <= reach
};
template <bool CAP>
__device__ __forceinline__ Score make_score(float scale, float cap) {
  Score f{scale * LOG2E, 0.f, {0.f, 0.f, 0.f, 0.f, 0.f}, 0.f};
  if constexpr (CAP) {
    constexpr float fit[5] = {0.99999993f, -0.3333231f, 0.13310174f, -0.05210148f, 0.01547543f};
    const float y = scale / cap;
    f.a = 2.f * LOG2E * y;
    f.c = cap * LOG2E;
    float power = f.c * y;
#pragma unroll
    for (int i = 0; i < 5; ++i, power *= y * y) f.p[i] = power * fit[i];
    f.reach = (f.p[4] < 0x1p-126f ? 0.05f : 0.6f) / y;
  }
  return f;
}
__device__ __forceinline__ float near_score(const Score& f, float x) {
  const float u = x * x;
  return x * fmaf(u, fmaf(u, fmaf(u, fmaf(u, f.p[4], f.p[3]), f.p[2]), f.p[1]), f.p[0]);
}
__device__ __forceinline__ float far_score(const Score& f, float x) {
  return f.c * fmaf(-2.f, __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(f.a * x)), 1.f);
}
// 16 scores at once
template <typename T, bool DAMP>
__device__ __forceinline__ void cap_scores(const Score& f, f32x16_t& s, f32x16_t& damp) {
  float top = 0.f;
#pragma unroll
  for (int i = 0; i < 16; ++i) top = fmaxf(top, fabsf(s[i]));
  if (!__any(!(top <= f.reach))) {
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = near_score(f, s[i]);
  } else if (sizeof(T) == 2 && f.c < SHARED_CAP) {
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = far_score(f, s[i]);
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = fabsf(s[i]) <= f.reach ? near_score(f, s[i]) : far_score(f, s[i]);
  }
  if constexpr (DAMP) {      // 1 - tanh^2 to a few 2^-24, from the score (beside the tanh it takes registers: 375 us for 318 at 4x1024x8 heads in fp32)
    const float ic2 = 1.f / (f.c * f.c);
#pragma unroll
    for (int i = 0; i < 16; ++i) damp[i] = fmaf(-ic2 * s[i], s[i], 1.f);
  }
}

// One value of each 64 bytes of a kernel's arguments, fetched before anything else and all at once: where they are needed, one after
// the other, the first use of each 64 bytes would take a trip to memory of its own (1x32x4 heads: forward 6.2 -> 5.7 us).
__device__ __forceinline__ void fetch_args(const FormArgs& a) {
  const int* const p = reinterpret_cast<const int*>(&a);
  int x[(sizeof(FormArgs) + 63) / 64];
#pragma unroll
  for (size_t i = 0; i < sizeof(x) / 4; ++i) x[i] = p[16 * i];
#pragma unroll
  for (size_t i = 0; i < sizeof(x) / 4; ++i) asm volatile("" : : "s"(x[i]));
}
// Least and largest document entry of every 64 positions of a sequence, of which a workgroup needs `most` from block `from` on.  Up
// to 64 it finds them itself, one wavefront a block (a launch of its own takes longer); beyond that k_doc_ranges has.  Called by the
// whole workgroup.
__device__ __forceinline__ const int2* doc_ranges(const FormArgs& a, int b, int2 (&room)[FORM_OWN_RANGES], int tid, int threads, int from, int most) {
  const int blocks = (a.S + 63) / 64;
  if (!a.docs) return nullptr;
  if (most > FORM_OWN_RANGES) return a.ranges + (size_t)b * blocks;
  const int count = min(most, blocks - from), step = threads >> 6;
  for (int i = tid >> 6; i < count; i += 4 * step) {      // four loads at a time (2x4096x8 heads of 64, documents of 128: 17 -> 14 us)
    int v[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = a.docs[(size_t)b * a.S + min(64 * (from + min(i + j * step, count - 1)) + (tid & 63), a.S - 1)];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (i + j * step >= count) break;
      const int lo = wave_min_i(v[j]), hi = wave_max_i(v[j]);
      if ((tid & 63) == 0) room[i + j * step] = make_int2(lo, hi);
    }
  }
  __syncthreads();
  return room - from;
}
__device__ __forceinline__ const int2* doc_ranges(const FormArgs& a, int b, int2 (&room)[FORM_OWN_RANGES], int tid, int threads) {
  return doc_ranges(a, b, room, tid, threads, 0, (a.S + 63) / 64);
}

// Which tile of which kv head a workgroup takes.  Workgroups go round the eight XCDs; the tiles of one kv head are given to one
// XCD, or to 8 / heads of them when there are fewer heads, so that its keys and values stay in few L2s.  uneven (causal): tiles
// differ in work and come longest first; heads that do not divide so are then dealt out tile by tile, as an XCD with the
// first tiles of a head only would finish last (1x8192, 4 kv heads: 492 us when each XCD has a run of tiles, 381 us in turn).
__device__ __forceinline__ void tile_order(int id, int heads, int tiles, bool uneven, int& head, int& tile) {
  const int x = id & 7, i = id >> 3;
  if (heads % 8 == 0) {
    head = x + 8 * (i / tiles);
    tile = i % tiles;
  } else if (8 % heads == 0 && tiles % (8 / heads) == 0) {
    const int share = 8 / heads;
    head = x / share;
    tile = i * share + x % share;
  } else if (uneven) {
    head = id % heads;
    tile = id / heads;
  } else {
    const int total = heads * tiles, q = total >> 3, r = total & 7, at = x * q + min(x, r) + i;
    head = at / tiles;
    tile = at % tiles;
  }
}

struct TileList {
  int tile[LIST], lo[LIST], hi[LIST];
  int count[4];
};
// Lists the tiles of the first 256 threads that ask for it; returns how many there are.  Called by the whole workgroup.
__device__ __forceinline__ int make_list(TileList& l, bool take, int tile, int lo, int hi, int tid) {
  const unsigned long long m = __ballot(take);
  const int wave = tid >> 6, lane = tid & 63;
  __syncthreads();            // the list before this one has been read
  if (lane == 0 && wave < 4) l.count[wave] = __popcll(m);
  __syncthreads();
  int at = __popcll(m & ((1ull << lane) - 1ull)), n = 0;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    if (w < wave) at += l.count[w];
    n += l.count[w];
  }
  if (take) {
    l.tile[at] = tile;
    l.lo[at] = lo;
    l.hi[at] = hi;
  }
  __syncthreads();
  return n;
}

template <typename T>
__device__ __forceinline__ const T* head_ptr(const FormHeads& x, int b, int h) {
  return reinterpret_cast<const T*>(x.p) + (long long)b * x.sb + (long long)h * x.sh;
}
template <typename T>
__device__ __forceinline__ T* head_out(const FormHeads& x, int b, int h) {
  return reinterpret_cast<T*>(const_cast<void*>(x.p)) + (long long)b * x.sb + (long long)h * x.sh;
}

// A lane's row of a [row, d] operand as fragments; rows that are not live and elements past the width are zeros.
template <typename T, int D>
__device__ __forceinline__ void load_frags(Frags<T, D>& f, const T* row, int half, int width, bool live) {
#pragma unroll
  for (int s = 0; s < Tile<T, D>::NS; ++s) {
    const int e = (2 * s + half) * Tile<T, D>::CH;
    f[s] = u32x4_t{0, 0, 0, 0};
    if (live && e < width) f[s] = *reinterpret_cast<const u32x4_t*>(row + e);
  }
}
// Rows go from memory into a tile directly, 64 lanes x 16 bytes an instruction to 1024 consecutive bytes of LDS; which piece a
// lane fetches is free, which is where the swizzle lives.  A lane whose piece is none of the operand's (a row past the end, a
// row of padding, elements past the width) fetches beyond the buffer's end, which writes zeros.
// The load is written out: behind the builtin the compiler lets every transposed read wait for all loads on their way, as it
// cannot tell the tiles apart (1x8192, 16 heads of 128, backward: queries 801 us, 689 written out; keys 1090, 924).  It returns
// nothing to a register; landed() stands between it and the reads.
constexpr uint32_t NOWHERE = 0x80000000u;
struct Source {
  u32x4_t rsrc;
  __device__ __forceinline__ Source(const void* base, uint32_t bytes) {
    const uint64_t p = reinterpret_cast<uint64_t>(base);
    rsrc = u32x4_t{(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)p), (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(p >> 32)) & 0xffffu,
                   (uint32_t)__builtin_amdgcn_readfirstlane((int)bytes), 0x00020000u};
    // a memory instruction may read a scalar register five wait states after a vector instruction wrote it; inside a written
    // out load the compiler does not see to that
    asm volatile("s_nop 4" : "+s"(rsrc));
  }
  // 16 (4) bytes a lane from its offset to LDS address `to` + 16 (4) * lane; `to` the same for the wavefront.  The compiler has M0 to
  // itself and warns when it is named; named it has to be, as it may set M0 once for several uses of its own.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
  __device__ __forceinline__ void load16(uint32_t off, uint32_t to) const {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" : : "s"(to), "v"(off), "s"(rsrc) : "memory", "m0");
  }
  __device__ __forceinline__ void load4(uint32_t off, uint32_t to) const {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, 0 offen lds" : : "s"(to), "v"(off), "s"(rsrc) : "memory", "m0");
  }
#pragma clang diagnostic pop
};
template <typename T, int D, int ROWS, int NW>
struct Loader {
  static constexpr int CPR = Tile<T, D>::CPR, NI = ROWS * CPR / (64 * NW);
  uint32_t voff[NI];
  static __device__ __forceinline__ int row_at(int j, int tid) { return (64 * ((tid >> 6) * NI + j) + (tid & 63)) / CPR; }
  // row r of the tile lies (r / group) * row_bytes + (r % group) * head_bytes behind the base; rows from `used` on are none
  __device__ __forceinline__ void init(int tid, long long row_bytes, int group, long long head_bytes, int used, int width) {
#pragma unroll
    for (int j = 0; j < NI; ++j) {
      const int r = row_at(j, tid), chunk = (tid & (CPR - 1)) ^ Tile<T, D>::swz(r);
      const bool in = chunk * Tile<T, D>::CH < width && r < used;
      voff[j] = in ? (uint32_t)((r / group) * row_bytes + (r % group) * head_bytes) + 16 * chunk : NOWHERE;
    }
  }
  template <typename Keep>
  __device__ __forceinline__ void issue(const T* base, uint32_t tile, int tid, bool guard, Keep keep) const {
    const Source src(base, 0x7fffffffu);
    const uint32_t dst = __builtin_amdgcn_readfirstlane((int)(tile + (tid >> 6) * NI * 1024));
#pragma unroll
    for (int j = 0; j < NI; ++j) {
      uint32_t off = voff[j];
      if (guard && !keep(row_at(j, tid))) off = NOWHERE;
      src.load16(off, dst + j * 1024);
    }
  }
};
__device__ __forceinline__ void meet() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("" ::: "memory");
}
// The loads on their way have landed, this wavefront's and then every one's.
__device__ __forceinline__ void landed() {
  __builtin_amdgcn_s_waitcnt(0x0F70);      // vmcnt(0)
  meet();
}

__device__ __forceinline__ void store4(bf16* p, float a, float b, float c, float d) {
  *reinterpret_cast<u32x2_t*>(p) = u32x2_t{pack_bf16x2(a, b), pack_bf16x2(c, d)};
}
__device__ __forceinline__ void store4(float* p, float a, float b, float c, float d) {
  *reinterpret_cast<f32x4_t*>(p) = f32x4_t{a, b, c, d};
}
// accumulators [d, lane's row] to the row at p
template <typename T, int D>
__device__ __forceinline__ void store_row(T* p, const f32x16_t (&acc)[D / 32], int half, int width, float factor, bool live) {
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const int d = 32 * db + 8 * g + 4 * half;
      if (d >= width) continue;
      float x[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) x[j] = live ? acc[db][4 * g + j] * factor : 0.f;
      store4(p + d, x[0], x[1], x[2], x[3]);
    }
}

// Number of keys, from the first on, among which a query at `pos` may see (of its document): its keys are 0 .. limit-1.
__device__ __forceinline__ int key_limit(const FormArgs& a, int pos, int prefix) {
  return a.causal ? min(a.S, max(pos + 1, prefix)) : a.S;
}

// What a lane that owns a query row knows of it.
struct RowOf {
  int R, qi, head, pos, id, lim;
  bool in, live;       // inside the tensor; sees anything at all
  float slope;         // of the distance, in the scores' unit before score_factor()
};
__device__ __forceinline__ RowOf row_of(const FormArgs& a, int R, int b, int hk, int prefix) {
  RowOf r;
  const int G = a.nh / a.nkv;
  r.R = R;
  r.in = R < a.n * G;
  const int Rc = r.in ? R : 0;
  r.qi = Rc / G;
  r.head = hk * G + Rc % G;
  r.pos = a.S - a.n + r.qi;
  r.id = a.docs ? a.docs[(size_t)b * a.S + r.pos] : 0;
  r.live = r.in && r.id >= 0;
  r.lim = r.live ? key_limit(a, r.pos, prefix) : 0;
  r.slope = a.slopes ? a.slopes[r.head] * (a.cap > 0.f ? LOG2E : 1.f / a.scale) : 0.f;
  return r;
}
// Factors of the gradients of queries and keys.  The softmax of a single score is one whatever the score, its gradient zero.  So it is
// exactly where the position leaves a row one key (causal: the first row), and for the keys where there is one in all.  Where it is
// documents that leave a row one key, the roundings of dp and delta remain, as they do in every row: fp32's, and in bf16 2^-16 of
// the size of dO O, as delta is mended.
__device__ __forceinline__ float query_gradient(const FormArgs& a, const RowOf& r) { return r.lim > 1 ? a.scale : 0.f; }
__device__ __forceinline__ float key_gradient(const FormArgs& a) { return a.S > 1 ? a.scale : 0.f; }

// Limits and document entries of the live rows among R0 .. R0 + count - 1.  Limits grow with the position: the first and the last
// row inside the tensor bound them.
struct Span {
  int lim_lo, lim_hi, id_lo, id_hi;
};
__device__ __forceinline__ void span_limits(const FormArgs& a, Span& s, int R0, int count, int prefix) {
  const int G = a.nh / a.nkv, rows = a.n * G, first = a.S - a.n;
  s.lim_lo = 0x7fffffff;
  s.lim_hi = 0;
  if (R0 >= rows) return;
  s.lim_lo = key_limit(a, first + R0 / G, prefix);
  s.lim_hi = key_limit(a, first + (min(rows, R0 + count) - 1) / G, prefix);
}
__device__ __forceinline__ Span wave_span(const FormArgs& a, const RowOf& r, int R0, int prefix) {
  Span s{0, 0, 0, 0};
  span_limits(a, s, R0, 32, prefix);
  if (a.docs) {
    s.id_lo = wave_min_i(r.live ? r.id : 0x7fffffff);
    s.id_hi = wave_max_i(r.live ? r.id : -1);
    if (s.id_hi < 0) s.lim_hi = 0;
  }
  return s;
}
// of the whole workgroup, whose rows start at R0
template <int NW>
__device__ __forceinline__ Span group_span(const FormArgs& a, const Span& w, int (&shared)[NW][2], int R0, int count, int prefix, int wave, int lane) {
  Span s = w;
  span_limits(a, s, R0, count, prefix);
  if (a.docs) {
    if (lane == 0) {
      shared[wave][0] = w.id_lo;
      shared[wave][1] = w.id_hi;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < NW; ++i) {
      s.id_lo = min(s.id_lo, __builtin_amdgcn_readfirstlane(shared[i][0]));
      s.id_hi = max(s.id_hi, __builtin_amdgcn_readfirstlane(shared[i][1]));
    }
    if (s.id_hi < 0) s.lim_hi = 0;
  }
  return s;
}
// keys k0 .. k0 + count - 1 with entries lo .. hi: 0 hidden from every row of the span, 2 open to every one, 1 neither
__device__ __forceinline__ int tile_state(const FormArgs& a, const Span& s, int k0, int count, int lo, int hi) {
  if (k0 >= s.lim_hi) return 0;
  if (a.docs && (hi < s.id_lo || lo > s.id_hi)) return 0;
  if (k0 + count > s.lim_lo) return 1;
  return a.docs && !(lo == hi && lo == s.id_lo && lo == s.id_hi) ? 1 : 2;
}
// least and largest document entry of the positions p0 .. p1, by whole blocks of 64 of them
__device__ __forceinline__ void positions_range(const int2* r, int p0, int p1, int& lo, int& hi) {
  lo = hi = 0;
  if (!r) return;
  lo = 0x7fffffff;
  hi = -0x7fffffff;
  for (int i = p0 >> 6; i <= p1 >> 6; ++i) {
    lo = min(lo, r[i].x);
    hi = max(hi, r[i].y);
  }
}

// Scores of 32 keys from k0 on (registers) for a lane's row: cap and distance, then the mask.  What comes out times
// score_factor() is the score in base 2; without a cap that leaves the factor to the exponential's own multiply-add.
template <bool CAP>
__device__ __forceinline__ float score_factor(const Score& f) { return CAP ? 1.f : f.a; }
template <typename T, bool CAP, bool SLOPES, bool DAMP>
__device__ __forceinline__ void open_scores(const Score& f, const RowOf& r, int k0, int half, f32x16_t& s, f32x16_t& damp) {
  if constexpr (CAP) cap_scores<T, DAMP>(f, s, damp);
  if constexpr (SLOPES) {
    const float far = (float)(r.pos - k0 - 4 * half);
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = fmaf(-r.slope, fabsf(far - (float)acc_row(i)), s[i]);
  }
}
// the keys that the row does not see get -infinity; limit: the least of the wavefront's rows
__device__ __forceinline__ void hide(const FormArgs& a, const RowOf& r, const int* ids, int k0, int limit, int half, f32x16_t& s) {
  if (k0 + 32 > limit) {
    const int lim = r.lim - k0 - 4 * half;
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = acc_row(i) < lim ? s[i] : -INFINITY;
  }
  if (a.docs) {
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const int4 v = *reinterpret_cast<const int4*>(ids + 8 * g + 4 * half);
      const int id[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
      for (int j = 0; j < 4; ++j) s[4 * g + j] = id[j] == r.id ? s[4 * g + j] : -INFINITY;
    }
  }
}
template <typename T, bool CAP, bool SLOPES, bool DAMP>
__device__ __forceinline__ void scores(const FormArgs& a, const Score& f, const RowOf& r, const int* ids, int k0, int limit, int half, bool mask,
                                       f32x16_t& s, f32x16_t& damp) {
  open_scores<T, CAP, SLOPES, DAMP>(f, r, k0, half, s, damp);
  if (mask) hide(a, r, ids, k0, limit, half, s);
}

// Tiles of keys and values in STAGES stages: while one is worked on, the loads of the next ones are on their way.
template <typename T, int D, int KT, int STAGES, int NW>
struct KeyTiles {
  static constexpr int TILE = KT * Tile<T, D>::ROWB, IDS = 512, STAGE = 2 * TILE + IDS, LDS = STAGES * STAGE;
  static_assert(KT * 4 <= IDS && TILE % TILE_ALIGN == 0, "tiles start on whole rows");
  using Load = Loader<T, D, KT, NW>;
  Load kl, vl;
  const T *k, *v;
  const int32_t* docs;
  int S;
  long long ksr, vsr;
  unsigned char* lds;
  __device__ __forceinline__ void init(const FormArgs& a, int b, int hk, unsigned char* mem, int tid) {
    k = head_ptr<T>(a.k, b, hk);
    v = head_ptr<T>(a.v, b, hk);
    docs = a.docs ? a.docs + (size_t)b * a.S : nullptr;
    S = a.S;
    ksr = a.k.sr;
    vsr = a.v.sr;
    lds = mem;
    kl.init(tid, ksr * (int)sizeof(T), 1, 0, KT, a.w);
    vl.init(tid, vsr * (int)sizeof(T), 1, 0, KT, a.w);
  }
  __device__ __forceinline__ uint32_t keys(int i) const { return lds_addr(lds) + (i & (STAGES - 1)) * STAGE; }
  __device__ __forceinline__ uint32_t values(int i) const { return keys(i) + TILE; }
  __device__ __forceinline__ const int* ids(int i) const { return reinterpret_cast<const int*>(lds + (i & (STAGES - 1)) * STAGE + 2 * TILE); }
  __device__ __forceinline__ void issue(int i, const TileList& list, int tid) const {
    const int k0 = __builtin_amdgcn_readfirstlane(list.tile[i]) * KT;
    const bool guard = k0 + KT > S || __builtin_amdgcn_readfirstlane(list.lo[i]) < 0;      // lo: least entry of the tile's documents
    auto keep = [&](int r) { return k0 + r < S && (docs == nullptr || docs[k0 + r] >= 0); };
    kl.issue(k + k0 * ksr, keys(i), tid, guard, keep);
    vl.issue(v + k0 * vsr, values(i), tid, guard, keep);
    if (docs && tid < KT)        // (entries past the last key are never looked at: positions limit first)
      Source(docs + k0, 4 * (S - k0)).load4(4 * tid, __builtin_amdgcn_readfirstlane((int)(keys(i) + 2 * TILE + (tid >> 6) * 256)));
  }
  // Before the first tile of a list, and before each: its stage has landed, the loads of the one that takes the stage before it begin.
  __device__ __forceinline__ void start(const TileList& list, int count, int tid) const {
    for (int i = 0; i < STAGES - 1 && i < count; ++i) issue(i, list, tid);
  }
  __device__ __forceinline__ void next(int i, const TileList& list, int count, int tid) const {
    if constexpr (STAGES > 1) {
      landed();
      if (i + STAGES - 1 < count) issue(i + STAGES - 1, list, tid);
    } else {
      __syncthreads();
      issue(i, list, tid);
      landed();
    }
  }
};

// ---- forward ----------------------------------------------------------------------------------------------------------
// FEW = false: 32 rows to each of NW wavefronts.  FEW = true (few rows in all): four wavefronts share 32 rows, each takes 32 keys of
// a tile of 128, and they join their results in LDS at the end.
// Few workgroups: the keys are split over a.splits workgroups whose results k_forms_join puts together.
template <typename T, int D, bool CAP, bool FEW, int NW>
struct Fwd {
  static constexpr bool WIDE32 = sizeof(T) == 4 && D == 128;
  static constexpr int KT = FEW ? 128 : 64, ROWS = FEW ? 32 : 32 * NW, TILE = KT * Tile<T, D>::ROWB;
  // One stage where two would leave room for one workgroup of a compute unit (bf16 at width 128, 8x1 queries over 8191 keys: 32.6
  // -> 29.5 us, 2x512x16 heads 21.1 -> 15.6; with a single workgroup to each, 1x1024x8 heads, 16.7 -> 17.5) and the registers do not.
  static constexpr int STAGES = TILE > (WIDE32 ? 32768 : 32767) ? 1 : 2;
  // Wavefronts that share a SIMD: as many as the registers of the accumulators allow (fp32 at width 64, 4x1024x8 heads: 144 us with
  // one, 97 with two; 3x203x12 16.0, 13.5).
  static constexpr int WAVES = WIDE32 ? 1 : sizeof(T) == 2 && D == 64 && !FEW ? (CAP ? 3 : 4) : 2;
  using Keys = KeyTiles<T, D, KT, STAGES, NW>;
  static constexpr int JOIN = FEW ? 4 * 32 * (D + 4) * 4 + 2 * 4 * 32 * 4 : 0;
  static constexpr int LDS = Keys::LDS > JOIN ? Keys::LDS : JOIN;
};

// largest of a lane's 16 scores and of those of the lane that holds the row's other 16
__device__ __forceinline__ float row_top(const f32x16_t& s) {
  float x = fmaxf(fmaxf(s[0], s[1]), s[2]), y = fmaxf(fmaxf(s[3], s[4]), s[5]);
  x = fmaxf(fmaxf(x, s[6]), s[7]);
  y = fmaxf(fmaxf(y, s[8]), s[9]);
  x = fmaxf(fmaxf(x, s[10]), s[11]);
  y = fmaxf(fmaxf(y, s[12]), s[13]);
  x = fmaxf(fmaxf(x, s[14]), s[15]);
  x = fmaxf(x, y);
  const auto w = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(w[0]), __uint_as_float(w[1]));
}

template <typename T, int D, bool CAP, bool SLOPES, bool FEW, int NW>
__global__ void __launch_bounds__(64 * NW, (Fwd<T, D, CAP, FEW, NW>::WAVES)) k_forms_fwd(FormArgs a) {
  fetch_args(a);
  using F = Fwd<T, D, CAP, FEW, NW>;
  static_assert(!FEW || NW == 4, "the wavefronts that share 32 rows");
  constexpr int NK = FEW ? 1 : F::KT / 32;       // blocks of 32 keys of a tile that a wavefront takes
  extern __shared__ __attribute__((aligned(TILE_ALIGN))) unsigned char lds[];
  __shared__ TileList list;
  __shared__ int2 ranges_s[FORM_OWN_RANGES];
  __shared__ int span_s[NW][2];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, half = lane >> 5;
  const int G = a.nh / a.nkv, rows = a.n * G, n_rt = (rows + F::ROWS - 1) / F::ROWS;
  int bh, at;
  tile_order(blockIdx.x, a.B * a.nkv, n_rt * a.splits, a.causal, bh, at);
  const int split = at % a.splits, rt = a.causal ? n_rt - 1 - at / a.splits : at / a.splits;     // the longest rows first
  const int hk = bh % a.nkv, b = bh / a.nkv;

  const int prefix = a.prefix ? a.prefix[b] : 0;
  const int n_tiles = (a.S + F::KT - 1) / F::KT, per = (n_tiles + a.splits - 1) / a.splits;
  const int2* ranges = doc_ranges(a, b, ranges_s, tid, 64 * NW, split * per * (F::KT / 64), per * (F::KT / 64));
  const int R0 = rt * F::ROWS, Rw = __builtin_amdgcn_readfirstlane(R0 + (FEW ? 0 : wave * 32));
  const RowOf r = row_of(a, Rw + (lane & 31), b, hk, prefix);
  const Span ws = wave_span(a, r, Rw, prefix), gs = group_span<NW>(a, ws, span_s, R0, F::ROWS, prefix, wave, lane);
  Frags<T, D> qf;
  load_frags<T, D>(qf, head_ptr<T>(a.q, b, r.head) + (long long)r.qi * a.q.sr, half, a.w, r.live);
  const Score sc = make_score<CAP>(a.scale, a.cap);
  const float factor = score_factor<CAP>(sc);
  const Lane<T, D> ln(lane);
  typename F::Keys kv;
  kv.init(a, b, hk, lds, tid);

  f32x16_t o[D / 32], unused;
#pragma unroll
  for (int i = 0; i < D / 32; ++i) o[i] = zero16();
  float m_run = NO_MAX, l_run = 0.f;
  // The exponentials' reference moves only when a score passes it by 2^8: any reference within that gives the same sums.
  auto refer = [&](float top) {
    if (__any(top > m_run + 8.f)) {
      const float m_new = fmaxf(m_run, top), alpha = __builtin_amdgcn_exp2f(m_run - m_new);
      l_run *= alpha;
      m_run = m_new;
#pragma unroll
      for (int db = 0; db < D / 32; ++db)
#pragma unroll
        for (int j = 0; j < 16; ++j) o[db][j] *= alpha;
    }
  };
  auto powers = [&](f32x16_t& s) {
    float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < 16; ++j) {
      s[j] = __builtin_amdgcn_exp2f(fmaf(s[j], factor, -m_run));
      sum[j & 3] += s[j];
    }
    l_run += (sum[0] + sum[1]) + (sum[2] + sum[3]);
  };
  const int t_end = min(n_tiles, (split + 1) * per);
  for (int base = split * per; base < t_end; base += LIST) {
    const int t = base + tid;
    int lo = 0, hi = 0, take = 0;
    if (tid < LIST && t < t_end) {
      positions_range(ranges, t * F::KT, min(a.S, (t + 1) * F::KT) - 1, lo, hi);
      take = tile_state(a, gs, t * F::KT, F::KT, lo, hi) != 0;
    }
    const int count = make_list(list, take, t, lo, hi, tid);
    // first key of tile i, and whether it has to be masked for this wavefront (a tile hidden from all its rows: like a masked one)
    auto first_key = [&](int i) { return __builtin_amdgcn_readfirstlane(list.tile[i]) * F::KT; };
    auto state_of = [&](int i) {
      return tile_state(a, ws, first_key(i), F::KT, __builtin_amdgcn_readfirstlane(list.lo[i]), __builtin_amdgcn_readfirstlane(list.hi[i]));
    };
    const int kb0 = FEW ? wave : 0;
    kv.start(list, count, tid);
    for (int i = 0; i < count; ++i) {
      kv.next(i, list, count, tid);
      const int k0 = first_key(i), state = state_of(i);
      if (state == 0) continue;
#pragma unroll
      for (int kb = 0; kb < NK; ++kb) {
        const int row0 = 32 * (kb0 + kb);
        f32x16_t s = dot_rows<T, D>(kv.keys(i), row0, qf, ln);
        scores<T, CAP, SLOPES, false>(a, sc, r, kv.ids(i) + row0, k0 + row0, ws.lim_lo, half, state == 1, s, unused);
        refer(factor * row_top(s));
        powers(s);
        add_outer<T, D>(o, kv.values(i), row0, s, ln);
      }
    }
  }
  l_run += __shfl_xor(l_run, 32, 64);

  if constexpr (FEW) {
    // the four wavefronts' results of each row: put onto the largest maximum and added, wavefront by wavefront
    constexpr int LD = D + 4;
    float* const po = reinterpret_cast<float*>(lds);
    float* const pm = po + 4 * 32 * LD;
    float* const pl = pm + 4 * 32;
    __syncthreads();
    if (half == 0) {
      pm[wave * 32 + lane] = m_run;
      pl[wave * 32 + lane] = l_run;
    }
    store_row<float, D>(po + (wave * 32 + (lane & 31)) * LD, o, half, D, 1.f, true);
    __syncthreads();
    // (each wavefront takes 8 rows, 8 lanes a row)
    const int row = wave * 8 + (lane >> 3), R = rt * F::ROWS + row;
    float m = NO_MAX, l = 0.f, e[4];
#pragma unroll
    for (int w = 0; w < 4; ++w) m = fmaxf(m, pm[w * 32 + row]);
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      e[w] = __builtin_amdgcn_exp2f(pm[w * 32 + row] - m);
      l += e[w] * pl[w * 32 + row];
    }
    const RowOf rr = row_of(a, R, b, hk, prefix);
    if (!rr.in) return;
    const bool some = rr.live && l != 0.f;      // (a NaN stays one)
    const size_t prow = ((size_t)split * a.B * a.nkv + (size_t)b * a.nkv + hk) * rows + R;
    const float inv = a.splits > 1 ? 1.f : some ? 1.f / l : 0.f;
    T* const out = head_out<T>(a.o, b, rr.head) + (long long)rr.qi * a.o.sr;
    for (int d = 4 * (lane & 7); d < a.w; d += 32) {
      f32x4_t x = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < 4; ++w) x += *reinterpret_cast<const f32x4_t*>(po + (w * 32 + row) * LD + d) * e[w];
      x *= inv;
      if (a.splits > 1) *reinterpret_cast<f32x4_t*>(a.part + prow * a.w + d) = x;
      else store4(out + d, some ? x[0] : 0.f, some ? x[1] : 0.f, some ? x[2] : 0.f, some ? x[3] : 0.f);
    }
    if ((lane & 7) == 0) {
      if (a.splits > 1) a.part_ml[prow] = make_float2(m, rr.live ? l : 0.f);
      else a.lse[((size_t)b * a.nh + rr.head) * a.n + rr.qi] = some ? (m + __builtin_amdgcn_logf(l)) * LN2 : -INFINITY;
    }
  } else {
    if (!r.in) return;
    const bool some = r.live && l_run != 0.f;      // (a NaN stays one)
    if (a.splits > 1) {
      const size_t prow = ((size_t)split * a.B * a.nkv + (size_t)b * a.nkv + hk) * rows + r.R;
      store_row<float, D>(a.part + prow * a.w, o, half, a.w, 1.f, true);
      if (half == 0) a.part_ml[prow] = make_float2(m_run, r.live ? l_run : 0.f);
    } else {
      store_row<T, D>(head_out<T>(a.o, b, r.head) + (long long)r.qi * a.o.sr, o, half, a.w, some ? 1.f / l_run : 0.f, some);
      if (half == 0) a.lse[((size_t)b * a.nh + r.head) * a.n + r.qi] = some ? (m_run + __builtin_amdgcn_logf(l_run)) * LN2 : -INFINITY;
    }
  }
}

// Results of the workgroups that shared a row's keys: put onto the largest maximum, added in their order.  One wavefront a row;
// its halves take every second workgroup, and lane i of the first ones workgroup i's maximum and sum.
template <typename T>
__global__ void __launch_bounds__(256) k_forms_join(FormArgs a) {
  fetch_args(a);
  __shared__ float e_s[4][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, half = lane >> 5, G = a.nh / a.nkv, rows = a.n * G;
  const size_t total = (size_t)a.B * a.nkv * rows, row = (size_t)blockIdx.x * 4 + wave;
  if (row >= total) return;
  const float2 none = make_float2(NO_MAX, 0.f);
  float m = NO_MAX, l = 0.f;
  f32x4_t x = f32x4_t{0.f, 0.f, 0.f, 0.f};
  const int d = 4 * (lane & 31);
  for (int base = 0; base < a.splits; base += 64) {
    const int n = min(64, a.splits - base);
    const float2 ml = lane < n ? a.part_ml[(size_t)(base + lane) * total + row] : none;
    float top = ml.x;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o, 64));
    const float m_new = fmaxf(m, top), old = __builtin_amdgcn_exp2f(m - m_new), e = ml.y != 0.f ? __builtin_amdgcn_exp2f(ml.x - m_new) : 0.f;
    l = l * old + wave_sum(e * ml.y);
    x *= old;
    m = m_new;
    e_s[wave][lane] = e;
    __builtin_amdgcn_wave_barrier();
    if (d < a.w)
#pragma unroll 8
      for (int s = half; s < n; s += 2) {
        const float f = e_s[wave][s];
        const f32x4_t v = *reinterpret_cast<const f32x4_t*>(a.part + ((size_t)(base + s) * total + row) * a.w + d);
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] = f != 0.f ? fmaf(v[j], f, x[j]) : x[j];
      }
    __builtin_amdgcn_wave_barrier();
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) x[j] += __shfl_xor(x[j], 32, 64);
  const int R = (int)(row % rows), hk = (int)(row / rows) % a.nkv, b = (int)(row / ((size_t)rows * a.nkv));
  const int head = hk * G + R % G, qi = R / G;
  const float inv = l != 0.f ? 1.f / l : 0.f;
  if (half == 0 && d < a.w) store4(head_out<T>(a.o, b, head) + (long long)qi * a.o.sr + d, x[0] * inv, x[1] * inv, x[2] * inv, x[3] * inv);
  if (lane == 0) a.lse[((size_t)b * a.nh + head) * a.n + qi] = l != 0.f ? (m + __builtin_amdgcn_logf(l)) * LN2 : -INFINITY;
}

// Sums of PARTS wavefronts that worked on the same rows (or keys), of which a workgroup has BLOCKS: the others' through LDS onto
// part 0's, in their order.  Called by the whole workgroup.
template <int D, int PARTS, int BLOCKS>
__device__ __forceinline__ void add_parts(f32x16_t (&acc)[D / 32], unsigned char* lds, int part, int blk, int lane) {
  constexpr int FLOATS = 32 * D;
  float* const mine = reinterpret_cast<float*>(lds) + blk * FLOATS + lane * 4;
  __syncthreads();
  if (part > 0)
#pragma unroll
    for (int i = 0; i < D / 32; ++i)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        *reinterpret_cast<f32x4_t*>(mine + (part - 1) * BLOCKS * FLOATS + (4 * i + g) * 256) =
            f32x4_t{acc[i][4 * g], acc[i][4 * g + 1], acc[i][4 * g + 2], acc[i][4 * g + 3]};
  __syncthreads();
  if (part == 0)
#pragma unroll
    for (int p = 0; p < PARTS - 1; ++p)
#pragma unroll
      for (int i = 0; i < D / 32; ++i)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const f32x4_t x = *reinterpret_cast<const f32x4_t*>(mine + p * BLOCKS * FLOATS + (4 * i + g) * 256);
#pragma unroll
          for (int j = 0; j < 4; ++j) acc[i][4 * g + j] += x[j];
        }
}

// ---- backward, query side: delta = sum_d dO O, dQ -----------------------------------------------------------------------
template <typename T>
__device__ __forceinline__ float dot_chunk(u32x4_t x, u32x4_t y) {
  float s = 0.f;
  if constexpr (sizeof(T) == 2) {
    const bf16x8_t u = __builtin_bit_cast(bf16x8_t, x), v = __builtin_bit_cast(bf16x8_t, y);
#pragma unroll
    for (int i = 0; i < 8; ++i) s = fmaf((float)u[i], (float)v[i], s);
  } else {
    const f32x4_t u = __builtin_bit_cast(f32x4_t, x), v = __builtin_bit_cast(f32x4_t, y);
#pragma unroll
    for (int i = 0; i < 4; ++i) s = fmaf(u[i], v[i], s);
  }
  return s;
}

// bf16: the stored output is rounded, so sum_d dO O is not quite the delta that makes a row of p (dp - delta) add up to zero, and
// in rows that look at few keys what is left is of the gradient's own size.  The kernel finds it, rest = sum p (dp - delta),
// and takes it out: delta grows by rest, dQ loses rest * sum p damp k, for which those sums are formed beside dQ.
// bf16 at width 128: the registers of dQ, of those sums and of the queries leave no room for dO's, which stay in LDS (SPARE).  Eight
// wavefronts, two to a SIMD, still spill 5 with a bias and, in the tile loop too, 31 to 33 with a cap; four, one to a SIMD, spill none
// and are slower (cap 20, both sides: 1x8192x16 heads over 4 1458 us against 1597, 32x512x16 534 against 608).
// FEW as in the forward.
template <typename T, int D, bool FEW, int NW>
struct BwdQ {
  static constexpr int KT = FEW ? 128 : 64, ROWS = FEW ? 32 : 32 * NW, TILE = KT * Tile<T, D>::ROWB;
  // wavefronts that share a SIMD (fp32 at width 64, 4x1024x8 heads, both sides: 414 us with one, 369 with two here)
  static constexpr int WAVES = D == 64 || NW == 8 ? 2 : 1, STAGES = TILE > (sizeof(T) == 4 && D == 64 ? 32767 : 32768) ? 1 : 2;
  static constexpr bool MEND = sizeof(T) == 2, SPARE = sizeof(T) == 2 && D == 128;
  using Keys = KeyTiles<T, D, KT, STAGES, NW>;
  static constexpr int LDS = Keys::LDS + (SPARE ? ROWS * Tile<T, D>::ROWB : 0);
  static_assert(!FEW || Keys::LDS >= 3 * 32 * D * 4 + 3 * 256, "the join's room");
};
// A wavefront's 32 rows and 32 keys from k0 on, row0 in the tiles of keys and values: dQ, the sums of p damp k and rest grow.
template <typename T, int D, bool CAP, bool SLOPES, bool MEND, bool SPARE, bool SHORT>
__device__ __forceinline__ void query_block(const FormArgs& a, const Score& sc, const RowOf& r, uint32_t keys, uint32_t values, int row0, const int* ids,
                                            int k0, int limit, bool mask, const Frags<T, D>& qf, const Frags<T, D>& gf, uint32_t grad, const Lane<T, D>& ln,
                                            int half, float l2, float delta, f32x16_t (&dq)[D / 32], f32x16_t (&pk)[MEND ? D / 32 : 1], float& rest) {
  const float factor = score_factor<CAP>(sc);
  f32x16_t s = dot_rows<T, D>(keys, row0, qf, ln), dp, damp;
  if constexpr (SPARE) dp = dot_tiles<T, D>(values, row0, grad, ln);
  else dp = dot_rows<T, D>(values, row0, gf, ln);
  feed<T, Tile<T, D>::NS, 1, 1>();
  feed<T, Tile<T, D>::NS, SPARE ? 2 : 1, 1>();
  scores<T, CAP, SLOPES, true>(a, sc, r, ids, k0, limit, half, mask, s, damp);
#pragma unroll
  for (int j = 0; j < 16; ++j) {
    float p = __builtin_amdgcn_exp2f(fmaf(s[j], factor, -l2)), ds = p * (dp[j] - delta);
    if constexpr (MEND) rest += ds;
    if constexpr (CAP) {
      ds *= damp[j];
      p *= damp[j];
    }
    s[j] = p;
    dp[j] = ds;
  }
  if constexpr (MEND) {
    add_outer2<T, D>(dq, pk, keys, row0, dp, s, ln);
    feed<T, D / 16, 2, 2>();
    if constexpr (SHORT)
      if (a.S <= FINE) add_outer<T, D>(dq, keys, row0, lost(dp), ln);
  } else {
    add_outer<T, D>(dq, keys, row0, dp, ln);
  }
}
template <typename T, int D, bool CAP, bool SLOPES, bool FEW, int NW, bool SHORT>
__global__ void __launch_bounds__(64 * NW, (BwdQ<T, D, FEW, NW>::WAVES)) k_forms_bwd_q(FormArgs a) {
  fetch_args(a);
  using Q = BwdQ<T, D, FEW, NW>;
  static_assert(!FEW || NW == 4, "the wavefronts that share 32 rows");
  constexpr int KT = Q::KT, NK = FEW ? 1 : KT / 32;
  constexpr bool MEND = Q::MEND;
  extern __shared__ __attribute__((aligned(TILE_ALIGN))) unsigned char lds[];
  __shared__ TileList list;
  __shared__ int2 ranges_s[FORM_OWN_RANGES];
  __shared__ int span_s[NW][2];
  unsigned char* const Gs = lds + Q::Keys::LDS;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, half = lane >> 5, part = FEW ? wave : 0, row_blk = FEW ? 0 : wave;
  const int G = a.nh / a.nkv, rows = a.n * G, n_rt = (rows + Q::ROWS - 1) / Q::ROWS;
  int bh, at;
  tile_order(blockIdx.x, a.B * a.nkv, n_rt, a.causal, bh, at);
  const int rt = a.causal ? n_rt - 1 - at : at, hk = bh % a.nkv, b = bh / a.nkv;

  const int prefix = a.prefix ? a.prefix[b] : 0;
  const int2* ranges = doc_ranges(a, b, ranges_s, tid, 64 * NW);
  const int R0 = rt * Q::ROWS, Rw = __builtin_amdgcn_readfirstlane(R0 + row_blk * 32);
  const RowOf r = row_of(a, Rw + (lane & 31), b, hk, prefix);
  const Span ws = wave_span(a, r, Rw, prefix), gs = group_span<NW>(a, ws, span_s, R0, Q::ROWS, prefix, wave, lane);
  const Score sc = make_score<CAP>(a.scale, a.cap);
  const Lane<T, D> ln(lane);
  typename Q::Keys kv;
  kv.init(a, b, hk, lds, tid);

  Frags<T, D> qf, gf;
  const size_t lrow = ((size_t)b * a.nh + r.head) * a.n + r.qi;
  float l2 = INFINITY, delta = 0.f, rest = 0.f;
  if (r.live) {
    l2 = a.lse[lrow] * LOG2E;
    if (l2 == -INFINITY) l2 = INFINITY;       // sees no key: probabilities zero
  }
  load_frags<T, D>(gf, head_ptr<T>(a.g, b, r.head) + (long long)r.qi * a.g.sr, half, a.w, r.live);
  {
    Frags<T, D> of;
    load_frags<T, D>(of, head_ptr<T>(a.o, b, r.head) + (long long)r.qi * a.o.sr, half, a.w, r.live);
#pragma unroll
    for (int s = 0; s < Tile<T, D>::NS; ++s) delta += dot_chunk<T>(gf[s], of[s]);
    delta += __shfl_xor(delta, 32, 64);
  }
  if constexpr (Q::SPARE) {      // (a wavefront reads back what it wrote, or the same that the others write)
#pragma unroll
    for (int s = 0; s < Tile<T, D>::NS; ++s) *Tile<T, D>::at(Gs, row_blk * 32 + (lane & 31), 2 * s + half) = gf[s];
  }
  load_frags<T, D>(qf, head_ptr<T>(a.q, b, r.head) + (long long)r.qi * a.q.sr, half, a.w, r.live);

  f32x16_t dq[D / 32], pk[MEND ? D / 32 : 1];
#pragma unroll
  for (int i = 0; i < D / 32; ++i) dq[i] = zero16();
#pragma unroll
  for (int i = 0; MEND && i < D / 32; ++i) pk[i] = zero16();
  const int n_tiles = (a.S + KT - 1) / KT;
  for (int base = 0; base < n_tiles; base += LIST) {
    const int t = base + tid;
    int lo = 0, hi = 0, take = 0;
    if (tid < LIST && t < n_tiles) {
      positions_range(ranges, t * KT, min(a.S, (t + 1) * KT) - 1, lo, hi);
      take = tile_state(a, gs, t * KT, KT, lo, hi) != 0;
    }
    const int count = make_list(list, take, t, lo, hi, tid);
    kv.start(list, count, tid);
    for (int i = 0; i < count; ++i) {
      kv.next(i, list, count, tid);
      const int k0 = __builtin_amdgcn_readfirstlane(list.tile[i]) * KT;
      const int state = tile_state(a, ws, k0, KT, __builtin_amdgcn_readfirstlane(list.lo[i]), __builtin_amdgcn_readfirstlane(list.hi[i]));
      if (state == 0) continue;
#pragma unroll Q::SPARE ? 1 : NK
      for (int kb = 0; kb < NK; ++kb) {
        const int row0 = 32 * (FEW ? wave : kb);
        query_block<T, D, CAP, SLOPES, MEND, Q::SPARE, SHORT>(a, sc, r, kv.keys(i), kv.values(i), row0, kv.ids(i) + row0, k0 + row0, ws.lim_lo, state == 1, qf, gf,
                                                       lds_addr(Gs) + row_blk * 32 * Tile<T, D>::ROWB, ln, half, l2, delta, dq, pk, rest);
      }
    }
  }
  if constexpr (FEW) {
    // the sums of the other wavefronts' keys onto the first's, through the tiles' room
    float* const rest_s = reinterpret_cast<float*>(lds + 3 * 32 * D * 4);
    add_parts<D, 4, 1>(dq, lds, part, 0, lane);
    if constexpr (MEND) {
      add_parts<D, 4, 1>(pk, lds, part, 0, lane);
      __syncthreads();
      if (part) rest_s[(part - 1) * 64 + lane] = rest;
      __syncthreads();
      if (part == 0) rest = ((rest + rest_s[lane]) + rest_s[64 + lane]) + rest_s[128 + lane];
    }
    if (part) return;
  }
  if constexpr (MEND) {
    rest += __shfl_xor(rest, 32, 64);
    delta += rest;
#pragma unroll
    for (int i = 0; i < D / 32; ++i)
#pragma unroll
      for (int j = 0; j < 16; ++j) dq[i][j] = fmaf(-rest, pk[i][j], dq[i][j]);
  }
  if (!r.in) return;
  if (half == 0) a.delta[lrow] = delta;
  store_row<T, D>(head_out<T>(a.dq, b, r.head) + (long long)r.qi * a.dq.sr, dq, half, a.w, query_gradient(a, r), r.live);
}

// the 16 of 32 rows' values that this half-wave's registers stand for
__device__ __forceinline__ f32x16_t rows_of(const float* x, int half) {
  f32x16_t r;
#pragma unroll
  for (int g = 0; g < 4; ++g) {
    const f32x4_t v = *reinterpret_cast<const f32x4_t*>(x + 8 * g + 4 * half);
#pragma unroll
    for (int j = 0; j < 4; ++j) r[4 * g + j] = v[j];
  }
  return r;
}

// ---- backward, key side: dK, dV ---------------------------------------------------------------------------------------
// What the key side has to know of the rows of a tile.
template <int RT>
struct RowsMeta {
  float l2[RT], delta[RT], slope[RT], pos[RT];      // -log-sum-exp in base 2 (START: over score_factor()), -delta
  int lim[RT], id[RT];
  template <bool START>
  __device__ __forceinline__ void put(int i, const RowOf& r, const Score& sc, float lse, float d) {
    l2[i] = lse == -INFINITY ? -INFINITY : -lse * (START ? LOG2E / sc.a : LOG2E);     // rows that see nothing: probabilities zero
    delta[i] = -d;
    slope[i] = r.slope;
    lim[i] = r.lim;
    id[i] = r.id;
    pos[i] = (float)r.pos;
  }
};
// A wavefront's 32 keys (key: the lane's) and the rows 32 rb .. of the tiles of queries and of output gradients: dK, dV grow.
template <typename T, int D, bool CAP, bool SLOPES, bool SPARE, bool SHORT, int RT>
__device__ __forceinline__ void key_block(const FormArgs& a, const Score& sc, const RowsMeta<RT>& m, uint32_t queries, uint32_t grads, int rb, const Frags<T, D>& kf,
                                          const Frags<T, D>& vf, uint32_t keys, uint32_t values, int key, int kid, bool mask, const Lane<T, D>& ln,
                                          int half, f32x16_t (&dk)[D / 32], f32x16_t (&dv)[D / 32]) {
  constexpr bool START = sizeof(T) == 2 && !CAP, PLAIN = START && !SLOPES;
  // bf16: the products start from what is taken off them, the row's log-sum-exp (no cap) and delta (no slopes either: registers).
  // fp32: not so, as every sum on the way would be rounded at that size (3x203x12 heads: dQ, dK off by 9e-7, not 5e-7).
  f32x16_t s = START ? rows_of(m.l2 + 32 * rb, half) : zero16(), dp = PLAIN ? rows_of(m.delta + 32 * rb, half) : zero16();
  if constexpr (SPARE) {
    s = dot_tiles<T, D>(queries, 32 * rb, keys, ln, s);
    dp = dot_tiles<T, D>(grads, 32 * rb, values, ln, dp);
  } else {
    s = dot_rows<T, D>(queries, 32 * rb, kf, ln, s);
    dp = dot_rows<T, D>(grads, 32 * rb, vf, ln, dp);
  }
  feed<T, Tile<T, D>::NS, SPARE ? 2 : 1, 1>();
  feed<T, Tile<T, D>::NS, SPARE ? 2 : 1, 1>();
  f32x16_t damp;
  if constexpr (CAP) cap_scores<T, true>(sc, s, damp);
  if constexpr (SLOPES) {
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const int at4 = 32 * rb + 8 * g + 4 * half;
      const f32x4_t sl = *reinterpret_cast<const f32x4_t*>(m.slope + at4);
      const f32x4_t pos = *reinterpret_cast<const f32x4_t*>(m.pos + at4);
#pragma unroll
      for (int j = 0; j < 4; ++j) s[4 * g + j] = fmaf(-sl[j], fabsf(pos[j] - (float)key), s[4 * g + j]);
    }
  }
  if (mask) {
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const int at4 = 32 * rb + 8 * g + 4 * half;
      const int4 lm = *reinterpret_cast<const int4*>(m.lim + at4), qi = *reinterpret_cast<const int4*>(m.id + at4);
      const int lim[4] = {lm.x, lm.y, lm.z, lm.w}, qid[4] = {qi.x, qi.y, qi.z, qi.w};
#pragma unroll
      for (int j = 0; j < 4; ++j) s[4 * g + j] = key < lim[j] & (qid[j] == kid) ? s[4 * g + j] : -INFINITY;
    }
  }
#pragma unroll
  for (int g = 0; g < 4; ++g) {
    f32x4_t l2 = f32x4_t{0.f, 0.f, 0.f, 0.f}, dl = l2;
    if constexpr (!START) l2 = *reinterpret_cast<const f32x4_t*>(m.l2 + 32 * rb + 8 * g + 4 * half);
    if constexpr (!PLAIN) dl = *reinterpret_cast<const f32x4_t*>(m.delta + 32 * rb + 8 * g + 4 * half);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float p = __builtin_amdgcn_exp2f(CAP ? s[4 * g + j] + l2[j] : START ? sc.a * s[4 * g + j] : fmaf(sc.a, s[4 * g + j], l2[j]));
      s[4 * g + j] = p;
      dp[4 * g + j] = p * (PLAIN ? dp[4 * g + j] : dp[4 * g + j] + dl[j]) * (CAP ? damp[4 * g + j] : 1.f);
    }
  }
  add_outer<T, D>(dv, grads, 32 * rb, s, ln);
  add_outer<T, D>(dk, queries, 32 * rb, dp, ln);
  feed<T, D / 8, 2, 1>();
  if constexpr (SHORT && sizeof(T) == 2)
    if (a.S <= FINE) {
      add_outer<T, D>(dv, grads, 32 * rb, lost(s), ln);
      add_outer<T, D>(dk, queries, 32 * rb, lost(dp), ln);
    }
}

// BLOCKS times 32 keys, over tiles of as many queries as have their rows (one for each of the G heads of the group) in RT.
// BLOCKS wavefronts take 32 keys each; where there are more, they share the rows of a tile and add up at the end:
//   4 of 4: 128 keys, tiles of 64 rows.  4 of 8 (bf16 at width 128): the same, two wavefronts to 32 keys; keys and values stay in
//   LDS, as the accumulators fill the registers.  1 of 4 (few keys in all): 32 keys, tiles of 128 rows.
// Few workgroups: the rows are split over a.row_splits workgroups, whose sums k_forms_kv_join adds.
template <typename T, int D, int BLOCKS, int NW>
struct BwdKv {
  static constexpr int PARTS = NW / BLOCKS, RT = PARTS == 4 ? 128 : 64, TILE = RT * Tile<T, D>::ROWB, STAGE = 2 * TILE;
  // Wavefronts that share a SIMD.  fp32 at width 64 has one stage for it and spills 9 to 21 vector registers, with a cap 26 to 49, and 38 to
  // 60 scalar ones (4x1024x8 heads, both sides, 369 us with one, 322 with two; 3x203x12, a workgroup to each compute unit, 36 and 37).
  static constexpr int WAVES = D == 64 || NW == 8 ? 2 : 1, BUFS = TILE > (NW == 4 && WAVES == 2 ? 32767 : 32768) ? 1 : 2;
  static constexpr bool SPARE = NW == 8;
  static constexpr int LDS = BUFS * STAGE + (SPARE ? 2 * 128 * Tile<T, D>::ROWB : 0);
  using Meta = RowsMeta<RT>;
  static_assert(BUFS * STAGE >= (PARTS - 1) * BLOCKS * 32 * D * 4, "the sums' room");
};
template <typename T, int D, bool CAP, bool SLOPES, int BLOCKS, int NW>
__global__ void __launch_bounds__(64 * NW, (BwdKv<T, D, BLOCKS, NW>::WAVES)) k_forms_bwd_kv(FormArgs a) {
  fetch_args(a);
  using K = BwdKv<T, D, BLOCKS, NW>;
  constexpr int RT = K::RT, TILE = K::TILE, NR = RT / 32 / K::PARTS, KEYS = 32 * BLOCKS;      // NR: blocks of 32 rows of a tile that a wavefront takes
  extern __shared__ __attribute__((aligned(TILE_ALIGN))) unsigned char lds[];
  __shared__ TileList list;
  __shared__ int2 ranges_s[FORM_OWN_RANGES];
  __shared__ __attribute__((aligned(16))) typename K::Meta meta[K::BUFS];
  unsigned char* const Ks = lds + K::BUFS * K::STAGE;
  unsigned char* const Vs = Ks + 128 * Tile<T, D>::ROWB;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, half = lane >> 5, blk = wave % BLOCKS, part = wave / BLOCKS;
  const int G = a.nh / a.nkv, QT = RT / G, used = QT * G, n_kt = (a.S + KEYS - 1) / KEYS, first = a.S - a.n;
  int bh, at;
  tile_order(blockIdx.x, a.B * a.nkv, n_kt * a.row_splits, a.causal, bh, at);     // (the first keys have the most rows)
  const int kt = at / a.row_splits, split = at % a.row_splits;
  const int hk = bh % a.nkv, b = bh / a.nkv;
  const int prefix = a.prefix ? a.prefix[b] : 0;
  const int32_t* docs = a.docs ? a.docs + (size_t)b * a.S : nullptr;
  const int kw = kt * KEYS + blk * 32, key = kw + (lane & 31);      // this wavefront's keys, this lane's
  const bool in = key < a.S;
  const int kid = docs ? (in ? docs[key] : -1) : 0;
  const bool live = in && kid >= 0;
  const int kid_lo = wave_min_i(live ? kid : 0x7fffffff), kid_hi = wave_max_i(live ? kid : -1);
  const Score sc = make_score<CAP>(a.scale, a.cap);
  const int2* ranges = doc_ranges(a, b, ranges_s, tid, 64 * NW);
  int klo, khi;
  positions_range(ranges, kt * KEYS, min(a.S, kt * KEYS + KEYS) - 1, klo, khi);

  Frags<T, D> kf, vf;
  load_frags<T, D>(kf, head_ptr<T>(a.k, b, hk) + (long long)(in ? key : 0) * a.k.sr, half, a.w, live);
  load_frags<T, D>(vf, head_ptr<T>(a.v, b, hk) + (long long)(in ? key : 0) * a.v.sr, half, a.w, live);
  if constexpr (K::SPARE) {
    if (part == 0)
#pragma unroll
      for (int s = 0; s < Tile<T, D>::NS; ++s) {
        *Tile<T, D>::at(Ks, blk * 32 + (lane & 31), 2 * s + half) = kf[s];
        *Tile<T, D>::at(Vs, blk * 32 + (lane & 31), 2 * s + half) = vf[s];
      }
  }
  f32x16_t dk[D / 32], dv[D / 32];
#pragma unroll
  for (int i = 0; i < D / 32; ++i) dk[i] = dv[i] = zero16();

  const Lane<T, D> ln(lane);
  Loader<T, D, RT, NW> ql, gl;
  ql.init(tid, a.q.sr * (int)sizeof(T), G, a.q.sh * (int)sizeof(T), used, a.w);
  gl.init(tid, a.g.sr * (int)sizeof(T), G, a.g.sh * (int)sizeof(T), used, a.w);
  const T* qbase = head_ptr<T>(a.q, b, hk * G);
  const T* gbase = head_ptr<T>(a.g, b, hk * G);
  auto tiles = [&](int i) { return lds + (K::BUFS > 1 ? (i & 1) * K::STAGE : 0); };
  // queries q0 .. q0 + QT - 1 of all heads of the group; what the mask needs of a row waits in the registers of a thread each
  RowOf mr;
  float ml2 = 0.f, mdelta = 0.f;
  auto issue = [&](int i, int q0, int lo) {
    if (tid < RT) {
      const int R = tid < used ? q0 * G + tid : 0x7fffffff;
      mr = row_of(a, R, b, hk, prefix);
      const size_t lrow = ((size_t)b * a.nh + mr.head) * a.n + mr.qi;
      ml2 = mr.live ? a.lse[lrow] : -INFINITY;
      mdelta = mr.live ? a.delta[lrow] : 0.f;
    }
    const bool guard = q0 + QT > a.n || lo < 0;
    auto keep = [&](int r) { return q0 + r / G < a.n && (docs == nullptr || docs[first + q0 + r / G] >= 0); };
    ql.issue(qbase + q0 * a.q.sr, lds_addr(tiles(i)), tid, guard, keep);
    gl.issue(gbase + q0 * a.g.sr, lds_addr(tiles(i)) + TILE, tid, guard, keep);
  };
  auto commit = [&](int i) {
    if (tid >= RT) return;
    meta[i & (K::BUFS - 1)].template put<sizeof(T) == 2 && !CAP>(tid, mr, sc, ml2, mdelta);
  };

  const int all_tiles = (a.n + QT - 1) / QT, n_tiles = (all_tiles - split + a.row_splits - 1) / a.row_splits;   // every row_splits-th
  for (int base = 0; base < n_tiles; base += LIST) {
    const int t = (base + tid) * a.row_splits + split;
    int lo = 0, hi = 0, take = 0;
    if (tid < LIST && base + tid < n_tiles) {
      const int p0 = first + t * QT, p1 = first + min(a.n, t * QT + QT) - 1;
      positions_range(ranges, p0, p1, lo, hi);
      take = kt * KEYS < key_limit(a, p1, prefix) && (!docs || (hi >= 0 && khi >= 0 && lo <= khi && hi >= klo));
    }
    const int count = make_list(list, take, t, lo, hi, tid);
    auto fetch = [&](int i) { issue(i, __builtin_amdgcn_readfirstlane(list.tile[i]) * QT, __builtin_amdgcn_readfirstlane(list.lo[i])); };
    if (K::BUFS > 1 && count > 0) {
      fetch(0);
      commit(0);
    }
    for (int i = 0; i < count; ++i) {
      const int q0 = __builtin_amdgcn_readfirstlane(list.tile[i]) * QT, p0 = first + q0, p1 = first + min(a.n, q0 + QT) - 1;
      const int lo_t = __builtin_amdgcn_readfirstlane(list.lo[i]), hi_t = __builtin_amdgcn_readfirstlane(list.hi[i]);
      if constexpr (K::BUFS == 1) {
        __syncthreads();
        fetch(i);
        commit(i);
      }
      __builtin_amdgcn_s_waitcnt(0xC07F);       // lgkmcnt(0): what commit() wrote
      landed();
      if (K::BUFS > 1 && i + 1 < count) fetch(i + 1);
      const typename K::Meta& m = meta[i & (K::BUFS - 1)];
      const uint32_t tile = lds_addr(tiles(i));
      const bool hidden = kw >= key_limit(a, p1, prefix) || kid_hi < 0 || (docs && (hi_t < kid_lo || lo_t > kid_hi));
      const bool mask = kw + 32 > key_limit(a, p0, prefix) || (docs && !(lo_t == hi_t && lo_t == kid_lo && lo_t == kid_hi));
      if (!hidden) {
#pragma unroll 1
        for (int rb = part * NR; rb < part * NR + NR; ++rb) {
          key_block<T, D, CAP, SLOPES, K::SPARE, BLOCKS == 1>(a, sc, m, tile, tile + TILE, rb, kf, vf, lds_addr(Ks) + blk * 32 * Tile<T, D>::ROWB,
                                                 lds_addr(Vs) + blk * 32 * Tile<T, D>::ROWB, key, kid, mask, ln, half, dk, dv);
        }
      }
      if (K::BUFS > 1 && i + 1 < count) commit(i + 1);
    }
  }
  if constexpr (K::PARTS > 1) {
    add_parts<D, K::PARTS, BLOCKS>(dk, lds, part, blk, lane);
    add_parts<D, K::PARTS, BLOCKS>(dv, lds, part, blk, lane);
    if (part) return;
  }
  if (!in) return;
  if (a.row_splits > 1) {
    const size_t all = (size_t)a.B * a.nkv * a.S, row = ((size_t)b * a.nkv + hk) * a.S + key;
    float* const out = a.part + ((size_t)split * 2 * all + row) * a.w;
    store_row<float, D>(out, dk, half, a.w, key_gradient(a), live);
    store_row<float, D>(out + all * a.w, dv, half, a.w, 1.f, live);
  } else {
    store_row<T, D>(head_out<T>(a.dk, b, hk) + (long long)key * a.dk.sr, dk, half, a.w, key_gradient(a), live);
    store_row<T, D>(head_out<T>(a.dv, b, hk) + (long long)key * a.dv.sr, dv, half, a.w, 1.f, live);
  }
}

// Sums of the workgroups that shared a key's rows, in their order; four elements a lane.
template <typename T>
__global__ void __launch_bounds__(256) k_forms_kv_join(FormArgs a) {
  const size_t all = (size_t)a.B * a.nkv * a.S * a.w, e = ((size_t)blockIdx.x * 256 + threadIdx.x) * 4;
  if (e >= 2 * all) return;
  f32x4_t x = *reinterpret_cast<const f32x4_t*>(a.part + e);
  for (int s = 1; s < a.row_splits; ++s) x += *reinterpret_cast<const f32x4_t*>(a.part + s * 2 * all + e);
  const bool v = e >= all;
  const size_t i = v ? e - all : e, row = i / a.w;
  const int d = (int)(i % a.w), key = (int)(row % a.S), hk = (int)(row / a.S) % a.nkv, b = (int)(row / ((size_t)a.S * a.nkv));
  const FormHeads& out = v ? a.dv : a.dk;
  store4(head_out<T>(out, b, hk) + (long long)key * out.sr + d, x[0], x[1], x[2], x[3]);
}

// ---- backward of short sequences --------------------------------------------------------------------------------------
// Both sides at once where a head's keys and the rows that see them fit a tile each: every operand is read once, where the two
// kernels read queries, keys, values and output gradients twice, and the two sides' launch and first loads are paid for once.  Each
// wavefront works on 32 rows over all keys, then on 32 keys over all rows; between the two the rows' queries and gradients go from
// registers into the tiles of the keys and values, whose own go into registers.
// 64x128x16 heads of 64, 134 MB: 52 us against 67 of the two kernels.  Its loads and stores alone take 33, each side's products 10
// more: the registers hold two wavefronts a SIMD, too few for loads and products to overlap.  Three, of 168 registers, spill: 54.
// At width 128 and in fp32 the registers hold one: 64x128x8 heads of 128 80 -> 69 us, 16x128x8 52 -> 31, 128x20x16 194 -> 138.
constexpr int ONE = 128;
template <typename T, int D>
struct BwdOne {
  static constexpr int TILE = ONE * Tile<T, D>::ROWB, LDS = 2 * TILE + TILE_ALIGN;
  static constexpr int WAVES = sizeof(T) == 2 && D == 64 ? 2 : 1;      // that share a SIMD: registers
  static constexpr bool MEND = sizeof(T) == 2;
  // Keys and rows up to which it is taken.  fp32: four blocks of 32 one behind the other take longer than on four wavefronts (1x128x8
  // heads of 64: 43 us against 26, 16x128x8 45 and 39; but 56x54x8 50 and 74, 1x20x4 16 and 26).
  static constexpr int MOST = sizeof(T) == 2 ? ONE : 64;
};
template <typename T, int D, bool CAP, bool SLOPES>
__global__ void __launch_bounds__(256, (BwdOne<T, D>::WAVES)) k_forms_bwd_one(FormArgs a) {
  fetch_args(a);
  static_assert(ONE * 4 <= TILE_ALIGN, "the entries' room");
  constexpr int TILE = BwdOne<T, D>::TILE;
  constexpr bool MEND = BwdOne<T, D>::MEND;
  extern __shared__ __attribute__((aligned(TILE_ALIGN))) unsigned char lds[];
  __shared__ int2 ranges_s[FORM_OWN_RANGES];
  __shared__ __attribute__((aligned(16))) RowsMeta<ONE> m;
  const uint32_t first_tile = lds_addr(lds), second_tile = first_tile + TILE;      // keys and values, then queries and gradients
  int* const ids = reinterpret_cast<int*>(lds + 2 * TILE);
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, half = lane >> 5;
  const int G = a.nh / a.nkv, rows = a.n * G, first = a.S - a.n, hk = blockIdx.x % a.nkv, b = blockIdx.x / a.nkv;
  const int prefix = a.prefix ? a.prefix[b] : 0;
  const int32_t* docs = a.docs ? a.docs + (size_t)b * a.S : nullptr;
  const int own = wave * 32 + (lane & 31);                                // the lane's row, then its key

  const RowOf r = row_of(a, own, b, hk, prefix);
  {
    Loader<T, D, ONE, 4> x;
    auto key = [&](int i) { return i < a.S && (docs == nullptr || docs[i] >= 0); };
    x.init(tid, a.k.sr * (int)sizeof(T), 1, 0, a.S, a.w);
    x.issue(head_ptr<T>(a.k, b, hk), first_tile, tid, true, key);
    x.init(tid, a.v.sr * (int)sizeof(T), 1, 0, a.S, a.w);
    x.issue(head_ptr<T>(a.v, b, hk), second_tile, tid, true, key);
  }
  Frags<T, D> qf, gf, of;
  load_frags<T, D>(qf, head_ptr<T>(a.q, b, r.head) + (long long)r.qi * a.q.sr, half, a.w, r.live);
  load_frags<T, D>(gf, head_ptr<T>(a.g, b, r.head) + (long long)r.qi * a.g.sr, half, a.w, r.live);
  load_frags<T, D>(of, head_ptr<T>(a.o, b, r.head) + (long long)r.qi * a.o.sr, half, a.w, r.live);
  const size_t lrow = ((size_t)b * a.nh + r.head) * a.n + r.qi;
  const float lse = r.live ? a.lse[lrow] : -INFINITY;
  const float l2 = lse == -INFINITY ? INFINITY : lse * LOG2E;             // sees no key: probabilities zero
  const bool in = own < a.S;
  const int kid = docs ? (in ? docs[own] : -1) : 0;
  const bool live = in && kid >= 0;
  if (half == 0) ids[own] = kid;
  const int2* ranges = doc_ranges(a, b, ranges_s, tid, 256);
  const int Rw = __builtin_amdgcn_readfirstlane(wave * 32);
  const Span ws = wave_span(a, r, Rw, prefix);
  const int kid_lo = wave_min_i(live ? kid : 0x7fffffff), kid_hi = wave_max_i(live ? kid : -1);
  const Score sc = make_score<CAP>(a.scale, a.cap);
  const Lane<T, D> ln(lane);
  float delta = 0.f, rest = 0.f;
  __builtin_amdgcn_s_waitcnt(0xC07F);       // lgkmcnt(0): the entries
  landed();
#pragma unroll
  for (int s = 0; s < Tile<T, D>::NS; ++s) delta += dot_chunk<T>(gf[s], of[s]);
  delta += __shfl_xor(delta, 32, 64);

  {
    f32x16_t dq[D / 32], pk[MEND ? D / 32 : 1];
#pragma unroll
    for (int i = 0; i < D / 32; ++i) dq[i] = zero16();
#pragma unroll
    for (int i = 0; MEND && i < D / 32; ++i) pk[i] = zero16();
#pragma unroll 1
    for (int k0 = 0; k0 < a.S; k0 += 32) {
      int lo, hi;
      positions_range(ranges, k0, k0, lo, hi);
      const int state = tile_state(a, ws, k0, 32, lo, hi);
      if (state == 0) continue;
      query_block<T, D, CAP, SLOPES, MEND, false, true>(a, sc, r, first_tile, second_tile, k0, ids + k0, k0, ws.lim_lo, state == 1, qf, gf, 0, ln, half, l2, delta, dq, pk, rest);
    }
    if constexpr (MEND) {
      rest += __shfl_xor(rest, 32, 64);
      delta += rest;
#pragma unroll
      for (int i = 0; i < D / 32; ++i)
#pragma unroll
        for (int j = 0; j < 16; ++j) dq[i][j] = fmaf(-rest, pk[i][j], dq[i][j]);
    }
    if (r.in) store_row<T, D>(head_out<T>(a.dq, b, r.head) + (long long)r.qi * a.dq.sr, dq, half, a.w, query_gradient(a, r), r.live);
  }
  if (half == 0) m.template put<sizeof(T) == 2 && !CAP>(own, r, sc, lse, r.live ? delta : 0.f);

  Frags<T, D> kf, vf;      // of the lane's key
#pragma unroll
  for (int s = 0; s < Tile<T, D>::NS; ++s) {
    kf[s] = *Tile<T, D>::at(lds, own, 2 * s + half);
    vf[s] = *Tile<T, D>::at(lds + TILE, own, 2 * s + half);
  }
  __syncthreads();
#pragma unroll
  for (int s = 0; s < Tile<T, D>::NS; ++s) {
    *Tile<T, D>::at(lds, own, 2 * s + half) = qf[s];
    *Tile<T, D>::at(lds + TILE, own, 2 * s + half) = gf[s];
  }
  __syncthreads();
  f32x16_t dk[D / 32], dv[D / 32];
#pragma unroll
  for (int i = 0; i < D / 32; ++i) dk[i] = dv[i] = zero16();
#pragma unroll 1
  for (int R0 = 0; R0 < rows; R0 += 32) {
    const int p0 = first + R0 / G, p1 = first + (min(rows, R0 + 32) - 1) / G;
    int lo, hi;
    positions_range(ranges, p0, p1, lo, hi);
    if (Rw >= key_limit(a, p1, prefix) || kid_hi < 0 || (docs && (hi < kid_lo || lo > kid_hi))) continue;
    const bool mask = Rw + 32 > key_limit(a, p0, prefix) || (docs && !(lo == hi && lo == kid_lo && lo == kid_hi));
    key_block<T, D, CAP, SLOPES, false, true>(a, sc, m, first_tile, second_tile, R0 / 32, kf, vf, 0, 0, own, kid, mask, ln, half, dk, dv);
  }
  if (!in) return;
  store_row<T, D>(head_out<T>(a.dk, b, hk) + (long long)own * a.dk.sr, dk, half, a.w, key_gradient(a), live);
  store_row<T, D>(head_out<T>(a.dv, b, hk) + (long long)own * a.dv.sr, dv, half, a.w, 1.f, live);
}

// ---- launches ---------------------------------------------------------------------------------------------------------
template <auto Kernel>
inline hipError_t launch(int threads, size_t blocks, int lds, const FormArgs& a, hipStream_t s) {
  static std::atomic<bool> allowed[64];      // once per kernel and device: more than 64 KB of LDS has to be asked for
  if (lds > 0) {
    int dev = 0;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return e;
    if (dev < 0 || dev >= 64 || !allowed[dev].load(std::memory_order_relaxed)) {
      e = hipFuncSetAttribute(reinterpret_cast<const void*>(Kernel), hipFuncAttributeMaxDynamicSharedMemorySize, lds);
      if (e != hipSuccess) return e;
      if (dev >= 0 && dev < 64) allowed[dev].store(true, std::memory_order_relaxed);
    }
  }
  Kernel<<<dim3((unsigned)blocks), dim3((unsigned)threads), lds, s>>>(a);
  return hipGetLastError();
}

// How the rows (and, backward, the keys) are dealt out: four wavefronts to 32 rows where there are few, 32 rows to each of eight
// (width 128 in bf16) where there are many; see attention_forms_bf16.hip.
enum RowMode { ROWS_FEW, ROWS_FOUR, ROWS_EIGHT };
RowMode row_mode(bool wide, int w, size_t heads, int rows);
bool few_keys(int w, size_t heads, int keys);

template <typename T, int D, bool CAP, bool SLOPES>
struct Launch {
  static constexpr bool WIDE = sizeof(T) == 2 && D == 128;
  static constexpr int NW = WIDE ? 8 : 4;
  static size_t tiles(int rows, int per) { return ((size_t)rows + per - 1) / per; }
  static hipError_t fwd(const FormArgs& a, hipStream_t s) {
    const int rows = a.n * (a.nh / a.nkv);
    const size_t heads = (size_t)a.B * a.nkv, each = heads * a.splits;
    const RowMode mode = row_mode(WIDE, D, heads, rows);
    hipError_t e;
    if (mode == ROWS_FEW) e = launch<k_forms_fwd<T, D, CAP, SLOPES, true, 4>>(256, each * tiles(rows, 32), Fwd<T, D, CAP, true, 4>::LDS, a, s);
    else if (mode == ROWS_EIGHT) e = launch<k_forms_fwd<T, D, CAP, SLOPES, false, NW>>(64 * NW, each * tiles(rows, 32 * NW), Fwd<T, D, CAP, false, NW>::LDS, a, s);
    else e = launch<k_forms_fwd<T, D, CAP, SLOPES, false, 4>>(256, each * tiles(rows, 128), Fwd<T, D, CAP, false, 4>::LDS, a, s);
    if (e != hipSuccess || a.splits == 1) return e;
    return launch<k_forms_join<T>>(256, (heads * rows + 3) / 4, 0, a, s);
  }
  static hipError_t bwd(const FormArgs& a, hipStream_t s) {
    const int rows = a.n * (a.nh / a.nkv);
    const size_t heads = (size_t)a.B * a.nkv;
    if (a.S <= BwdOne<T, D>::MOST && rows <= BwdOne<T, D>::MOST)
      return launch<k_forms_bwd_one<T, D, CAP, SLOPES>>(256, heads, BwdOne<T, D>::LDS, a, s);
    const RowMode mode = row_mode(WIDE, D, heads, rows);
    hipError_t e;
    // (the lost parts of up to FINE keys in instances of their own where rows are not few: elsewhere they would cost registers)
    constexpr bool PARTS = sizeof(T) == 2;
    if (mode == ROWS_FEW) e = launch<k_forms_bwd_q<T, D, CAP, SLOPES, true, 4, PARTS>>(256, heads * tiles(rows, 32), BwdQ<T, D, true, 4>::LDS, a, s);
    else if (PARTS && a.S <= FINE) e = launch<k_forms_bwd_q<T, D, CAP, SLOPES, false, 4, PARTS>>(256, heads * tiles(rows, 128), BwdQ<T, D, false, 4>::LDS, a, s);
    else if (mode == ROWS_EIGHT) e = launch<k_forms_bwd_q<T, D, CAP, SLOPES, false, NW, false>>(64 * NW, heads * tiles(rows, 32 * NW), BwdQ<T, D, false, NW>::LDS, a, s);
    else e = launch<k_forms_bwd_q<T, D, CAP, SLOPES, false, 4, false>>(256, heads * tiles(rows, 128), BwdQ<T, D, false, 4>::LDS, a, s);
    if (e != hipSuccess) return e;
    if (few_keys(D, heads, a.S))
      e = launch<k_forms_bwd_kv<T, D, CAP, SLOPES, 1, 4>>(256, heads * tiles(a.S, 32) * a.row_splits, BwdKv<T, D, 1, 4>::LDS, a, s);
    else e = launch<k_forms_bwd_kv<T, D, CAP, SLOPES, 4, NW>>(64 * NW, heads * tiles(a.S, 128) * a.row_splits, BwdKv<T, D, 4, NW>::LDS, a, s);
    if (e != hipSuccess || a.row_splits == 1) return e;
    return launch<k_forms_kv_join<T>>(256, (heads * a.S * a.w / 2 + 255) / 256, 0, a, s);
  }
};
template <typename T, int D, typename F>
hipError_t pick_w(const FormArgs& a, F f) {
  if (a.cap > 0.f) return a.slopes ? f(Launch<T, D, true, true>{}) : f(Launch<T, D, true, false>{});
  return a.slopes ? f(Launch<T, D, false, true>{}) : f(Launch<T, D, false, false>{});
}
template <typename T, typename F>
hipError_t pick(const FormArgs& a, F f) {
  return a.w <= 64 ? pick_w<T, 64>(a, f) : pick_w<T, 128>(a, f);
}
template <typename T>
hipError_t fwd_t(const FormArgs& a, hipStream_t s) {
  return pick<T>(a, [&](auto l) { return decltype(l)::fwd(a, s); });
}
template <typename T>
hipError_t bwd_t(const FormArgs& a, hipStream_t s) {
  return pick<T>(a, [&](auto l) { return decltype(l)::bwd(a, s); });
}

}  // namespace forms
}  // namespace mslt
