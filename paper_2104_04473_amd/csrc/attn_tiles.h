// Building blocks of the attention kernels: fragments and sums of the fp32 kernels, tiles, fragments and work assignment of the bf16
// ones.  They know a row pitch, heads' first elements and which rows exist, not which scores are hidden.
#pragma once
#include "common.h"
#include <type_traits>

namespace ptdp {

typedef __attribute__((__vector_size__(8 * sizeof(__bf16)))) __bf16 bf16x8_t;
typedef __attribute__((__vector_size__(16 * sizeof(float)))) float f32x16_t;
typedef __attribute__((__vector_size__(4 * sizeof(float)))) float f32x4_t;

// ------------------------------------------------------------------------------------------------
// fp32 kernels on v_mfma_f32_16x16x4_f32 (fp32 products and sums).  A workgroup of NW waves (four, or eight
// where workgroups are few) owns 16 queries (forward, dQ) or 16 keys (dK, dV) of one head.  The walk over the other side is PARTS
// partial sums, each over every PARTS-th 16-row tile, that meet in LDS in a fixed order (eight instead of four: error against 64
// bits 1 to 13 % smaller).  PARTS follows from s and dh alone and a wave makes PARTS / NW of them one after the other, so that a
// sample's results have the same bits whatever else is in the call.  Operands come from memory straight into fragments: lane (c = lane & 15,
// g = lane >> 4) carries four consecutive dh of row c (elements 16 i + 4 g .. +3 of step i; both factors of a product
// share that order), and the score tile S^T comes out with column c = the workgroup's row and rows 4 g + r = the tile's,
// which is the second product's B operand as it stands.  These are small calls (fp32 is the precision of small
// configurations): what counts is the length of one wave's chain and the number of waves.  128 tokens x 4 heads x 2
// samples, dh 64: forward 68 -> 9 us, backward 155 -> 25 us against one wave per row that reduced every
// score across the wave.
// ND: steps of 16 dh (dh rounded up; the lanes past dh hold zeros).
// ------------------------------------------------------------------------------------------------
constexpr int kF32Rows = 16;
constexpr int kMaxF32Dh = 256;

template <int ND> struct F32Frag { f32x4_t v[ND]; };
// four consecutive dh of one row per step; `row` must be readable
template <int ND> __device__ __forceinline__ void f32_load(F32Frag<ND>& f, const float* __restrict__ row, int g, int dh) {
#pragma unroll
  for (int i = 0; i < ND; ++i) {
    const int d = 16 * i + 4 * g;
    f.v[i] = d < dh ? *reinterpret_cast<const f32x4_t*>(row + d) : f32x4_t{0.f, 0.f, 0.f, 0.f};
  }
}
// 16 x 16 products of rows a (result rows 4 g + r) and rows b (result column c): MFMAs FIRST .. FIRST + N - 1 of 4 dh each
// (of 4 ND), added up as a tree whose leaves are chains of kF32Leaf.
// One chain over dh had up to twice the error of the tree.
template <int ND, int FIRST = 0, int N = 4 * ND>
__device__ __forceinline__ f32x4_t f32_scores(const F32Frag<ND>& a, const F32Frag<ND>& b) {
  constexpr int kF32Leaf = ND > 10 ? 8 : 4;   // (heads beyond 160: a shorter chain's registers would spill)
  if constexpr (N > kF32Leaf) {
    constexpr int kHalf = (N / kF32Leaf + 1) / 2 * kF32Leaf;
    return f32_scores<ND, FIRST, kHalf>(a, b) + f32_scores<ND, FIRST + kHalf, N - kHalf>(a, b);
  } else {
    f32x4_t acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = FIRST; i < FIRST + N; ++i) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(a.v[i / 4][i % 4], b.v[i / 4][i % 4], acc, 0, 0, 0);
    return acc;
  }
}
// acc^T[16 dh rows x 16 columns] += X^T w for the tile rows row0 .. row0 + 15 of X (rows from s on count as zeros; their
// weights are zero).  Register r of acc[t]: dh 16 t + 4 g + r of column c.
// A weight that the causal mask hides is zero, but zero times an infinite or undefined element is not: in a tile on the
// diagonal (`vis`: bit r = row 4 g + r is visible to column c) such elements enter the product as zeros and are added
// afterwards to the columns that see them, so that no bit of the other columns depends on them.
template <int ND>
__device__ __forceinline__ void f32_accumulate(f32x4_t (&acc)[ND], f32x4_t w, const float* __restrict__ X, size_t rs, int row0, int s,
                                               int dh, bool diag, uint32_t vis, int lane) {
  const int c = lane & 15, g = lane >> 4;
  auto at = [&](int t, int r) {
    const int row = row0 + 4 * g + r, d = 16 * t + c;
    const float x = X[(size_t)min(row, s - 1) * rs + min(d, dh - 1)];
    return row < s && d < dh ? x : 0.f;
  };
  if (!diag) {
#pragma unroll
    for (int t = 0; t < ND; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) acc[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(at(t, r), w[r], acc[t], 0, 0, 0);
    return;
  }
  bool finite = true;
#pragma unroll
  for (int t = 0; t < ND; ++t)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const float x = at(t, r);
      const bool ok = fabsf(x) < INFINITY;
      finite = finite && ok;
      acc[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(ok ? x : 0.f, w[r], acc[t], 0, 0, 0);
    }
  if (__all(finite)) return;
#pragma unroll 1
  for (int row = 0; row < 16 && row0 + row < s; ++row) {
    const int src = (row >> 2) * 16 + c, k = row & 3;
    const float wr = __shfl(k & 2 ? (k & 1 ? w[3] : w[2]) : (k & 1 ? w[1] : w[0]), src, 64);
    const bool seen = (__shfl((int)vis, src, 64) >> k) & 1;
    const float* x = X + (size_t)(row0 + row) * rs + 4 * g;
#pragma unroll
    for (int t = 0; t < ND; ++t)
      if (16 * t + 4 * g < dh) {
        const f32x4_t v = *reinterpret_cast<const f32x4_t*>(x + 16 * t);
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (seen && !(fabsf(v[r]) < INFINITY)) acc[t][r] += wr * v[r];
      }
  }
}
// Four waves with a part each: waves 1 .. 3 hand theirs to wave 0 (added in that order); returns true in wave 0.  part: 3 * ND * 64 vectors.
template <int ND> __device__ __forceinline__ bool f32_join(f32x4_t (&acc)[ND], f32x4_t* part, int wave, int lane) {
  __syncthreads();
  if (wave > 0) {
#pragma unroll
    for (int t = 0; t < ND; ++t) part[((wave - 1) * ND + t) * 64 + lane] = acc[t];
  }
  __syncthreads();
  if (wave > 0) return false;
#pragma unroll
  for (int w = 0; w < 3; ++w)
#pragma unroll
    for (int t = 0; t < ND; ++t) acc[t] += part[(w * ND + t) * 64 + lane];
  return true;
}
// Eight parts: part w and part w + 4, then those four sums in order.  Four waves make two parts each: the earlier one waits in the
// wave's own place (f32_set_aside) and f32_add_pair adds it to the later one; of eight waves the upper four hand theirs to the lower.
// place: 4 * ND * 64 vectors per sum.
template <int ND> __device__ __forceinline__ void f32_set_aside(f32x4_t (&acc)[ND], f32x4_t* place, int wave, int lane) {
#pragma unroll
  for (int t = 0; t < ND; ++t) {
    place[(wave * ND + t) * 64 + lane] = acc[t];
    acc[t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  }
}
// (the products are rounded by themselves, or a form might fuse with the sum behind them what another does not)
template <int ND> __device__ __forceinline__ void f32_scale(f32x4_t (&acc)[ND], float f) {
#pragma clang fp contract(off)
#pragma unroll
  for (int t = 0; t < ND; ++t) acc[t] *= f;
}
template <int ND, int NW> __device__ __forceinline__ void f32_add_pair(f32x4_t (&acc)[ND], const f32x4_t* place, float factor, int wave, int lane) {
  if (NW == 8 && wave >= 4) return;
  f32x4_t other[ND];
#pragma unroll
  for (int t = 0; t < ND; ++t) other[t] = place[(wave * ND + t) * 64 + lane];
  if (NW == 4) f32_scale<ND>(other, factor);
#pragma unroll
  for (int t = 0; t < ND; ++t) acc[t] += other[t];
}
// NS sums at once; sum q ends up in wave q.  factor: of the parts set aside (NW = 4)
template <int ND, int NW, int NS>
__device__ __forceinline__ void f32_join_eight(f32x4_t (&acc)[NS][ND], f32x4_t* place, float factor, int wave, int lane) {
  constexpr int kSum = 4 * ND * 64;
  if (NW == 8) {
    if (wave >= 4) {
#pragma unroll
      for (int q = 0; q < NS; ++q) f32_set_aside<ND>(acc[q], place + q * kSum, wave - 4, lane);
    }
    __syncthreads();
  }
#pragma unroll
  for (int q = 0; q < NS; ++q) {
    f32_add_pair<ND, NW>(acc[q], place + q * kSum, factor, wave, lane);
    if (wave < 4 && wave != q) {
#pragma unroll
      for (int t = 0; t < ND; ++t) place[q * kSum + (wave * ND + t) * 64 + lane] = acc[q][t];
    }
  }
  __syncthreads();
#pragma unroll
  for (int q = 0; q < NS; ++q)
    if (wave == q) {
#pragma unroll
      for (int t = 0; t < ND; ++t) {
        f32x4_t sum = q == 0 ? acc[q][t] : place[q * kSum + t * 64 + lane];
#pragma unroll
        for (int w = 1; w < 4; ++w) sum += w == q ? acc[q][t] : place[q * kSum + (w * ND + t) * 64 + lane];
        acc[q][t] = sum;
      }
    }
}
// vectors of LDS for `sums` sums
constexpr int f32_places(int nd, int parts, int sums) { return (parts == 8 ? sums * 4 : 3) * nd * 64; }
template <int ND> __device__ __forceinline__ void f32_store(float* row, const f32x4_t (&acc)[ND], int g, int dh) {
#pragma unroll
  for (int t = 0; t < ND; ++t)
    if (16 * t + 4 * g < dh) *reinterpret_cast<f32x4_t*>(row + 16 * t + 4 * g) = acc[t];
}

// delta = sum_d dctx * ctx of 16 rows (o, dc): the diagonal of ctx dctx^T, summed in the order of dP below: with one visible key
// dP - delta is exactly zero.  Lane (c, g) holds it for row c if the tile's rows are columns, for rows 4 g + r otherwise.
template <int ND> __device__ __forceinline__ float f32_delta_column(const F32Frag<ND>& o, const F32Frag<ND>& dc, int c) {
  const f32x4_t x = f32_scores<ND>(o, dc);
  const float mine = (c & 2) ? ((c & 1) ? x[3] : x[2]) : ((c & 1) ? x[1] : x[0]);
  return __shfl(mine, (c >> 2) * 16 + c, 64);
}
template <int ND> __device__ __forceinline__ f32x4_t f32_delta_rows(const F32Frag<ND>& o, const F32Frag<ND>& dc, int g) {
  const f32x4_t x = f32_scores<ND>(o, dc);
  f32x4_t d;
#pragma unroll
  for (int r = 0; r < 4; ++r) d[r] = __shfl(x[r], 16 * g + 4 * g + r, 64);
  return d;
}

// ------------------------------------------------------------------------------------------------
// bf16 MFMA kernels.  A wave owns 32 queries (forward, dQ) or 32 keys (dK/dV); the other side streams through LDS in
// tiles of 32 or 64 rows kept in memory order [row][dh].  Operands whose contraction index is the tile row (V^T, K^T,
// Q^T, dO^T) are gathered from those same tiles with transposing LDS reads, so nothing is transposed in registers
// and every tile is stored once.
// ------------------------------------------------------------------------------------------------
typedef __attribute__((__vector_size__(4 * sizeof(short)))) short s16x4_t;

// Registers 8*ks .. 8*ks+7 of a 32x32 accumulator as a bf16 B-operand fragment.
__device__ __forceinline__ bf16x8_t pack_frag(const f32x16_t& a, int ks) {
  uint4 t = make_uint4(pack_bf16x2(a[ks * 8 + 0], a[ks * 8 + 1]), pack_bf16x2(a[ks * 8 + 2], a[ks * 8 + 3]),
                       pack_bf16x2(a[ks * 8 + 4], a[ks * 8 + 5]), pack_bf16x2(a[ks * 8 + 6], a[ks * 8 + 7]));
  return *reinterpret_cast<bf16x8_t*>(&t);
}
__device__ __forceinline__ f32x16_t zero16() {
  f32x16_t z;
#pragma unroll
  for (int r = 0; r < 16; ++r) z[r] = 0.f;
  return z;
}
// lane's 8 consecutive dh (k16 step kk) of one token row, as a B-operand fragment straight from HBM
// (`row` must be readable; `ok` false blanks the fragment)
__device__ __forceinline__ bf16x8_t frag_global(const bf16_t* row, bool ok, int kk, int half) {
  const uint4 r = *reinterpret_cast<const uint4*>(row + kk * 16 + half * 8);
  uint4 t = make_uint4(ok ? r.x : 0u, ok ? r.y : 0u, ok ? r.z : 0u, ok ? r.w : 0u);
  return *reinterpret_cast<bf16x8_t*>(&t);
}
// accumulator rows (dh) of lane's column (token) -> 8-byte stores of 4 consecutive dh
template <int NDT>
__device__ __forceinline__ void store_cols(bf16_t* out_row, const f32x16_t (&acc)[NDT], float mul, int half) {
#pragma unroll
  for (int d = 0; d < NDT; ++d)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      uint2 w;
      w.x = pack_bf16x2(acc[d][4 * g] * mul, acc[d][4 * g + 1] * mul);
      w.y = pack_bf16x2(acc[d][4 * g + 2] * mul, acc[d][4 * g + 3] * mul);
      *reinterpret_cast<uint2*>(out_row + d * 32 + 8 * g + 4 * half) = w;
    }
}

// Work assignment.  Workgroups are dealt round-robin to the 8 XCDs, each with its own L2: every block of one
// (sample, head) pair goes to the same XCD so that the pair's K and V stay in that L2, and each XCD
// takes its pairs one after the other - as long as whole rounds of 8 pairs remain.  The last heads * b mod 8 pairs
// are dealt block by block instead (block-major, so that each XCD gets the same share of every block index and
// with it of the causal triangle's work): 20 heads would otherwise leave four XCDs with three pairs and four
// with two.  Returns false for surplus ids.  `blk` counts up within a pair.
__device__ __forceinline__ bool attn_map(int id, int nblk, int heads, int b, int* blk, int* e, int* j) {
  const int xcd = id & 7, local = id >> 3;
  const int pairs = heads * b, whole = pairs >> 3, rest = pairs & 7;
  int pair;
  if (local < whole * nblk) {
    pair = xcd + 8 * (local / nblk);
    *blk = local % nblk;
  } else {
    const int g = (local - whole * nblk) * 8 + xcd;   // index into the remaining pairs' blocks, block-major
    if (g >= rest * nblk) return false;
    pair = 8 * whole + g % rest;
    *blk = g / rest;
  }
  *e = pair % heads;
  *j = pair / heads;
  return true;
}
inline long long attn_grid(long long nblk, int heads, int b) {
  const long long pairs = (long long)heads * b, whole = pairs >> 3, rest = pairs & 7;
  return 8 * (whole * nblk + (rest * nblk + 7) / 8);
}

// The same for the causal kernels on tiles from LDS, whose blocks differ in length: an XCD takes block `blk` of all its pairs
// before block blk + 1 of any, so that the longest walks start first whatever pair they belong to (pair by pair, the last
// pair's longest block starts when most others are done).  Eight block levels at a time; the last heads * b mod 8 pairs
// are dealt block by block.  Fewer than eight blocks: as above.
__device__ __forceinline__ bool attn_map_levels(int id, int nblk, int heads, int b, int* blk, int* e, int* j) {
  if (nblk < 8) return attn_map(id, nblk, heads, b, blk, e, j);
  const int xcd = id & 7, local = id >> 3;
  const int pairs = heads * b, whole = pairs >> 3, rest = pairs & 7;
  const int chunk = local / pairs, r = local % pairs;
  int pair;
  if (r < rest) {
    const int g = (chunk * rest + r) * 8 + xcd;   // index into the remaining pairs' blocks, block-major
    if (g >= rest * nblk) return false;
    pair = 8 * whole + g % rest;
    *blk = g / rest;
  } else {
    *blk = 8 * chunk + (r - rest) / whole;
    if (*blk >= nblk) return false;
    pair = xcd + 8 * ((r - rest) % whole);
  }
  *e = pair % heads;
  *j = pair / heads;
  return true;
}
inline long long attn_grid_levels(long long nblk, int heads, int b) {
  return nblk < 8 ? attn_grid(nblk, heads, b) : (long long)heads * b * (8 * ((nblk + 7) / 8));
}

// ------------------------------------------------------------------------------------------------
// Tiles of 64 rows that travel from memory straight to LDS (buffer_load ... lds), one tile ahead of the arithmetic.
// LDS image: blocks of 32 dh, [block][64 rows][64 bytes]; the 16-byte chunk c of row r sits in slot c ^ ((r >> 2) & 3),
// so that 16 rows of a fragment read and the 8 rows of a transposing read fall into different bank groups.
// ------------------------------------------------------------------------------------------------
typedef uint32_t attn_rsrc_t __attribute__((ext_vector_type(4)));
__device__ __forceinline__ uint32_t attn_lds_offset(const char* p) {
  return (uint32_t)reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) void*)p);
}
// lane i's 16 bytes land at lds + 16 i.  Assembly, because the compiler makes every LDS read wait for all such loads in
// flight; s_nop 4: the descriptor may have been written by the vector ALU just before, which the compiler cannot see here.
__device__ __forceinline__ void attn_load_lds(attn_rsrc_t r, uint32_t lds, uint32_t voff) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" :: "s"(lds), "v"(voff), "s"(r) : "memory", "m0");
}
// A slice is addressed from its first row with 32-bit byte offsets; they reach the end of its sixteenth row up to this pitch.
constexpr bool attn_slice_fits(uint64_t row_elements, int dh) {
  return row_elements < (1ull << 31) && 15 * row_elements * 2 + 2 * (uint64_t)dh <= 0xffffffffull;
}
typedef uint32_t attn_chunk_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) attn_chunk_t lds_chunk_t;
// A group of W waves loads a tile of KT rows; wave w takes the 16-row slices w, w + W, .. of every block.
// WIDE: any row pitch: 64-bit addresses, through registers, to the same places.
template <int DH, int W, int KT, bool WIDE> struct TileDma {
  static_assert(KT / 16 % W == 0, "every wave takes the same slices of every block");
  static constexpr int NDT = DH / 32, kBytes = KT * DH * 2;
  uint32_t off;   // the lane's chunk inside a slice's first block (WIDE: inside the lane's row)
  uint32_t lane;
  size_t rs;
  __device__ __forceinline__ void init(size_t row_elements, int lane_id) {
    rs = row_elements;
    lane = lane_id;
    off = (WIDE ? 0u : (uint32_t)((lane >> 2) * row_elements * 2)) + (((lane & 3) ^ (lane >> 4)) * 16);
  }
  // rows row0 .. row0 + KT - 1 of a head whose row 0 starts at p; rows from s on are zeros
  __device__ __forceinline__ void issue(const bf16_t* __restrict__ p, int row0, int s, uint32_t lds, int w) const {
    if constexpr (WIDE) {
#pragma unroll
      for (int g = 0; g < KT / 16 / W; ++g) {
        const int slice = w + W * g, row = row0 + 16 * slice + (int)(lane >> 2);
        const bool ok = row < s;
        const char* a = reinterpret_cast<const char*>(p + (size_t)min(row, s - 1) * rs) + off;
        const uint32_t to = lds + slice * 1024 + lane * 16;
#pragma unroll
        for (int d = 0; d < NDT; ++d) {
          attn_chunk_t t = {0u, 0u, 0u, 0u};
          if (ok) t = *reinterpret_cast<const attn_chunk_t*>(a + d * 64);
          *(lds_chunk_t*)(uintptr_t)(to + d * (KT * 64)) = t;
        }
      }
      return;
    }
#pragma unroll
    for (int g = 0; g < KT / 16 / W; ++g) {
      const int slice = w + W * g, first = row0 + 16 * slice, rows = min(s - first, 16);
      const uint64_t a = reinterpret_cast<uint64_t>(p + (size_t)first * rs);
      const attn_rsrc_t r = {(uint32_t)a, (uint32_t)(a >> 32) & 0xffffu, rows > 0 ? (uint32_t)((rows - 1) * rs * 2 + DH * 2) : 0u, 0x00020000u};
#pragma unroll
      for (int d = 0; d < NDT; ++d) attn_load_lds(r, lds + d * (KT * 64) + slice * 1024, off + d * 64);
    }
  }
};
typedef __attribute__((address_space(3))) const bf16x8_t lds_frag_t;
typedef __attribute__((address_space(3))) s16x4_t lds_tr_t;
// fragment with the tile row as the MFMA row: row sub * 32 + (lane & 31), eight dh of k16 step kk
template <int KT> struct FragDirect {
  uint32_t base[2];
  __device__ __forceinline__ void init(uint32_t tile, int l31, int half) {
#pragma unroll
    for (int p = 0; p < 2; ++p) base[p] = tile + l31 * 64 + (((2 * p + half) ^ ((l31 >> 2) & 3)) * 16);
  }
  // moved by a stage: the sum is kept in the base registers, so that everything else is in the instructions' offset fields
  __device__ __forceinline__ FragDirect at(uint32_t stage) const {
    FragDirect f{{base[0] + stage, base[1] + stage}};
    asm volatile("" : "+v"(f.base[0]), "+v"(f.base[1]));
    return f;
  }
  __device__ __forceinline__ bf16x8_t get(int sub, int kk, int tile = 0) const {
    return *(lds_frag_t*)(uintptr_t)(base[kk & 1] + (kk >> 1) * (KT * 64) + sub * 2048 + tile);
  }
};
// fragment with dh as the MFMA row (d * 32 + (lane & 31)) and tile rows as the contraction index, in the order of the 32x32
// accumulator rows that feed the other operand: rows 16 * ks + 4 * half + 0..3 and 16 * ks + 8 + 4 * half + 0..3 of
// 32-row half `sub`.  ds_read_b64_tr_b16: within 16 lanes, lane i receives element (i & 3) of the 8-byte rows addressed by
// lanes (i >> 2) + {0, 4, 8, 12}.
template <int KT> struct FragTr {
  uint32_t lo, hi;
  __device__ __forceinline__ void init(uint32_t tile, int lane) {
    const int r = lane & 15, G = lane >> 4, row = 4 * (G >> 1) + (r >> 2), c = (2 * (G & 1) + ((r & 3) >> 1)) ^ (G >> 1);
    lo = tile + row * 64 + c * 16 + (r & 1) * 8;
    hi = tile + (row + 8) * 64 + (c ^ 2) * 16 + (r & 1) * 8;
  }
  __device__ __forceinline__ FragTr at(uint32_t stage) const {
    FragTr f{lo + stage, hi + stage};
    asm volatile("" : "+v"(f.lo), "+v"(f.hi));
    return f;
  }
  __device__ __forceinline__ bf16x8_t get(int d, int sub, int ks, int tile = 0) const {
    const uint32_t o = d * (KT * 64) + sub * 2048 + ks * 1024 + tile;
    const s16x4_t a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_tr_t*)(uintptr_t)(lo + o));
    const s16x4_t b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_tr_t*)(uintptr_t)(hi + o));
    typedef __attribute__((__vector_size__(8 * sizeof(short)))) short s16x8_t;
    const s16x8_t v = __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
    return __builtin_bit_cast(bf16x8_t, v);
  }
};
// every request of this wave has landed, every LDS read has returned, and the same holds for the workgroup's other waves
__device__ __forceinline__ void attn_tiles_ready() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory"); }
// order of a scheduling region's MFMAs and LDS reads: the reads of the first kAhead MFMAs, then one MFMA and the reads of one
template <int MFMAS, int READS> __device__ __forceinline__ void sched_reads_ahead() {
  constexpr int kAhead = 4 < MFMAS ? 4 : MFMAS;
  __builtin_amdgcn_sched_group_barrier(0x100, kAhead * READS, 0);
#pragma unroll
  for (int i = 0; i < MFMAS; ++i) {
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    __builtin_amdgcn_sched_group_barrier(0x100, READS, 0);
  }
}
// MFMAs with the reads of one more and a share of VALU vector instructions behind each
template <int MFMAS, int READS, int VALU> __device__ __forceinline__ void sched_mixed() {
#pragma unroll
  for (int i = 0; i < MFMAS; ++i) {
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    __builtin_amdgcn_sched_group_barrier(0x100, READS, 0);
    __builtin_amdgcn_sched_group_barrier(0x402, (VALU + MFMAS - 1) / MFMAS, 0);
  }
}

template <bool LEVELS> __device__ __forceinline__ bool attn_map_tiles(int id, int nblk, int heads, int b, int* blk, int* e, int* j) {
  if (!(LEVELS ? attn_map_levels(id, nblk, heads, b, blk, e, j) : attn_map(id, nblk, heads, b, blk, e, j))) return false;
  *blk = __builtin_amdgcn_readfirstlane(*blk);
  *e = __builtin_amdgcn_readfirstlane(*e);
  *j = __builtin_amdgcn_readfirstlane(*j);
  return true;
}

// delta = sum_d dctx * ctx of 32 rows, one to a lane and its neighbour 32 lanes on: the diagonal of ctx dctx^T, summed in the order of dP
// in the kernels below (with one visible key dP - D is exactly zero).  `row`: the lane's row of ctx, readable.
template <int DH>
__device__ __forceinline__ float attn_delta_of(const bf16_t* __restrict__ row, const bf16x8_t (&dof)[DH / 16], bool valid, int lane) {
  const int half = lane >> 5, l31 = lane & 31;
  f32x16_t x = zero16();
#pragma unroll
  for (int kk = 0; kk < DH / 16; ++kk) x = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag_global(row, valid, kk, half), dof[kk], x, 0, 0, 0);
  // row l31 of column l31: register (l31 & 3) + 4 * (l31 >> 3) of the lane of half (l31 >> 2) & 1
  float mine = x[0];
#pragma unroll
  for (int r = 1; r < 16; ++r) mine = (l31 & 3) + 4 * (l31 >> 3) == r ? x[r] : mine;
  return __shfl(mine, ((l31 >> 2) & 1) * 32 + l31, 64);
}

inline int attn_compute_units() {
  static std::atomic<int> cached[kMaxDevices];   // per device, looked up once
  const int d = device_slot();
  if (d >= 0 && cached[d].load(std::memory_order_relaxed) > 0) return cached[d].load(std::memory_order_relaxed);
  int dev = 0, cu = 256;
  if (hipGetDevice(&dev) == hipSuccess) {
    int v = 0;
    if (hipDeviceGetAttribute(&v, hipDeviceAttributeMultiprocessorCount, dev) == hipSuccess && v > 0) cu = v;
  }
  if (d >= 0) cached[d].store(cu, std::memory_order_relaxed);
  return cu;
}

}  // namespace ptdp
