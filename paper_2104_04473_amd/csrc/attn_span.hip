// Attention under spans: query i of sample j sees the keys lo <= k < hi of its span and no others.  The causal mask, packed documents,
// prefixes that are read both ways, windows and padding are all intervals of keys, so one pair of integers per query takes the
// place of an s x s mask, and tiles that no query sees are never read.  Scores may be capped, x -> cap tanh(x / cap), and get a bias
// -slope[head] |i - k|; groups of heads / kv_heads query heads share a key/value head.
//
//   x = scale q.k;  c = cap tanh(x / cap);  t = c - slope |i - k|;  p = exp(t - lse);  ctx = sum_k p v
//   dp = dctx.v;  D = dctx.ctx;  dt = p (dp - D);  dx = dt (1 - (c / cap)^2);  dq = scale sum_k dx k;
//   dk = scale sum_i dx q and dv = sum_i p dctx, over the queries of all heads of the group.
// A query whose span is empty gives a row of zeros, lse = -inf and no gradient.
//
// qkv is [s, b, (heads + 2 kv_heads) dh] with columns [Q heads | K heads | V heads].
#include "attn_tiles.h"
#include "gelu.h"

namespace ptdp {

// ------------------------------------------------------------------------------------------------
// Spans in memory: {lo, hi} of every query, [b][s], then of every 32 queries what decides whether a tile of keys is to be read
// (keys before `first` or from `last` on are seen by none) and whether all of it is seen by all (keys from `inner_lo` to `inner_hi`),
// [b][(s + 31) / 32].  An empty span is {kNoKey, 0}: it leaves first and last alone and nothing is seen by all.
// ------------------------------------------------------------------------------------------------
constexpr int kNoKey = 0x7fffffff, kSpanRows = 32;
struct SpanBounds { int first, last, inner_lo, inner_hi; };
struct SpanView {
  const int2* range;           // null: the causal mask, {0, i + 1}
  const SpanBounds* bounds;
};
static size_t span_range_bytes(int s, int b) { return ((size_t)s * b * sizeof(int2) + 15) / 16 * 16; }
size_t attn_spans_bytes(int s, int b) { return span_range_bytes(s, b) + (size_t)b * ((s + kSpanRows - 1) / kSpanRows) * sizeof(SpanBounds); }
static SpanView span_view(const void* spans, int s, int b) {
  if (!spans) return {nullptr, nullptr};
  const char* p = (const char*)spans;
  return {(const int2*)p, (const SpanBounds*)(p + span_range_bytes(s, b))};
}
__device__ __forceinline__ int2 span_of(const SpanView& v, int j, int i, int s) { return v.range ? v.range[(size_t)j * s + i] : make_int2(0, i + 1); }
// of `blocks` blocks of 32 queries from block t on (wave-uniform)
__device__ __forceinline__ SpanBounds bounds_of(const SpanView& v, int j, int t, int blocks, int s) {
  const int nt = (s + kSpanRows - 1) / kSpanRows;
  SpanBounds x = {kNoKey, 0, 0, kNoKey};
  if (!v.range) return {0, min(s, (t + blocks) * kSpanRows), 0, t * kSpanRows + 1};
  for (int w = 0; w < blocks && t + w < nt; ++w) {
    const SpanBounds y = v.bounds[(size_t)j * nt + t + w];
    x = {min(x.first, y.first), max(x.last, y.last), max(x.inner_lo, y.inner_lo), min(x.inner_hi, y.inner_hi)};
  }
  return {__builtin_amdgcn_readfirstlane(x.first), __builtin_amdgcn_readfirstlane(x.last), __builtin_amdgcn_readfirstlane(x.inner_lo),
          __builtin_amdgcn_readfirstlane(x.inner_hi)};
}

// Builds them.  A document is a run of equal ids; a negative id is padding.  One thread per token; where a document begins or ends
// outside the workgroup's tokens, the workgroup looks for it, kSpanStep ids at a time.
constexpr int kSpanThreads = 256, kSpanLook = 16, kSpanStep = kSpanThreads * kSpanLook;
__global__ void __launch_bounds__(kSpanThreads)
attn_spans_kernel(int causal, int window, const int32_t* __restrict__ documents, const int32_t* __restrict__ prefix, int2* __restrict__ range,
                  SpanBounds* __restrict__ bounds, int s, int b) {
  __shared__ unsigned long long starts[kSpanThreads / 64];
  __shared__ int found;
  const int j = blockIdx.y, i0 = blockIdx.x * kSpanThreads, i = i0 + threadIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  auto id = [&](int t) { return documents[(size_t)t * b + j]; };
  int d0 = 0, d1 = s;
  bool gone = false;
  if (documents) {
    const int mine = i < s ? id(i) : 0;
    gone = mine < 0;
    const bool start = i < s && (i == 0 || id(i - 1) != mine);
    const unsigned long long m = __ballot(start);
    if (lane == 0) starts[wave] = m;
    // the last start before the workgroup's tokens
    int before = 0, after = s;
    if (threadIdx.x == 0) found = -1;
    __syncthreads();
    for (int end = i0; end > 0 && !(starts[0] & 1); end -= kSpanStep) {
      int best = -1;
#pragma unroll
      for (int u = 0; u < kSpanLook; ++u) {   // (all of a step's ids are requested at once)
        const int t = end - 1 - (u * kSpanThreads + (int)threadIdx.x);
        const bool differs = id(max(t, 0)) != id(max(t - 1, 0));
        if (t == 0 || (t > 0 && differs)) best = max(best, t);
      }
      if (best >= 0) atomicMax(&found, best);
      __syncthreads();
      before = found;
      __syncthreads();
      if (before >= 0) break;
    }
    // the first start behind them
    if (threadIdx.x == 0) found = s;
    __syncthreads();
    for (int begin = i0 + kSpanThreads; begin < s; begin += kSpanStep) {
      int best = s;
#pragma unroll
      for (int u = 0; u < kSpanLook; ++u) {
        const int t = begin + u * kSpanThreads + (int)threadIdx.x;
        const bool differs = id(min(t, s - 1)) != id(min(t, s) - 1);
        if (t < s && differs) best = min(best, t);
      }
      if (best < s) atomicMin(&found, best);
      __syncthreads();
      after = found;
      __syncthreads();
      if (after < s) break;
    }
    d0 = before;
    d1 = after;
#pragma unroll
    for (int w = 0; w < kSpanThreads / 64; ++w) {   // starts up to this token, the last one wins; behind it, the first one does
      const unsigned long long up_to = w < wave ? ~0ull : w > wave ? 0ull : (lane == 63 ? ~0ull : (2ull << lane) - 1);
      if (starts[w] & up_to) d0 = i0 + 64 * w + 63 - __clzll((long long)(starts[w] & up_to));
      const int v = kSpanThreads / 64 - 1 - w;
      const unsigned long long behind = v > wave ? ~0ull : v < wave ? 0ull : (lane == 63 ? 0ull : ~0ull << (lane + 1));
      if (starts[v] & behind) d1 = i0 + 64 * v + __ffsll((unsigned long long)(starts[v] & behind)) - 1;
    }
  }
  int lo = d0, hi = d1;
  if (causal) {
    hi = i + 1;
    if (prefix && i < s && !gone) hi = max(hi, d0 + min(max(prefix[(size_t)d0 * b + j], 0), d1 - d0));
  }
  if (window > 0) {
    lo = max((long long)lo, (long long)i - window + 1);
    hi = min((long long)hi, (long long)i + window);
  }
  const bool there = i < s;
  if (gone) {
    lo = kNoKey;
    hi = 0;
  }
  if (there) range[(size_t)j * s + i] = make_int2(lo, hi);
  // of every 32 tokens; those behind the last one count for nothing
  int first = there ? lo : kNoKey, last = there ? hi : 0, inner_lo = there ? lo : 0, inner_hi = there ? hi : kNoKey;
#pragma unroll
  for (int d = 1; d < 32; d *= 2) {
    first = min(first, __shfl_xor(first, d, 64));
    last = max(last, __shfl_xor(last, d, 64));
    inner_lo = max(inner_lo, __shfl_xor(inner_lo, d, 64));
    inner_hi = min(inner_hi, __shfl_xor(inner_hi, d, 64));
  }
  if ((lane & 31) == 0 && there) bounds[(size_t)j * ((s + kSpanRows - 1) / kSpanRows) + i / kSpanRows] = {first, last, inner_lo, inner_hi};
}
int launch_attn_spans(int causal, int window, const int32_t* documents, const int32_t* prefix, void* spans, int s, int b, hipStream_t st) {
  Launch L(PTDP_K_OTHER, (double)s * b * 12, st);
  hipLaunchKernelGGL(attn_spans_kernel, dim3((s + kSpanThreads - 1) / kSpanThreads, b), dim3(kSpanThreads), 0, st, causal, window, documents, prefix,
                     (int2*)spans, (SpanBounds*)((char*)spans + span_range_bytes(s, b)), s, b);
  return L.status();
}

// ------------------------------------------------------------------------------------------------
// Scores.  In the bf16 kernels a score is kept in units of 1 / mul of the exponent of two: q.k where there is no cap, tanh(x / cap) where
// there is one, less bias |i - k| in the same units.
// ------------------------------------------------------------------------------------------------
constexpr float kLog2e = 1.4426950408889634f;
struct SpanShape {
  int s, b, heads, kv_heads;
  float scale, cap;
  float mul, steep, per_cap, per_slope;   // exponent of two per unit; 2 log2(e) scale / cap; scale / cap; units of bias per slope
  const float* slopes;           // null: no bias
  __device__ __forceinline__ bool capped() const { return cap > 0.f; }
  bool capped_or_biased() const { return cap > 0.f || slopes; }
  // tanh with the hardware's exponential and reciprocal, as fast_tanh: absolute error 1e-7, of the cap
  __device__ __forceinline__ float tanh(float x) const { return 1.f - 2.f * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(x * steep)); }
  // Where a row has few keys its lse is to have more digits than that leaves: |y| = |x / cap| <= 1/2, as most scores, take y P(y^2), relative error
  // 1.1e-7 (P fitted to tanh(y) / y for the least largest relative error).  The forward kernel does this in tiles that some query does not see all of
  // (in all tiles: 4096 x 20 heads of 160, 158 -> 176 us; so: 160).  Each element's form is its own affair: what others hold, hidden ones above all, does
  // not change a bit of it.
  __device__ __forceinline__ void tanh_to_the_digit(f32x16_t& a) const {
    float most = 0.f;
#pragma unroll
    for (int r = 0; r < 16; ++r) most = fmaxf(most, fabsf(a[r]));
    auto near = [&](float y) {
      const float q = y * y;
      return y * fmaf(q, fmaf(q, fmaf(q, fmaf(q, 0.017135007f, -0.052986074f), 0.13324779f), -0.33333069f), 1.f);
    };
    if (__all(most * per_cap <= 0.5f)) {
#pragma unroll
      for (int r = 0; r < 16; ++r) a[r] = near(a[r] * per_cap);
    } else {
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const float y = a[r] * per_cap;
        float far = tanh(a[r]);
        asm volatile("" : "+v"(far));   // (chosen, not branched to)
        a[r] = fabsf(y) <= 0.5f ? near(y) : far;
      }
    }
  }
  __device__ __forceinline__ float bias(int head) const {   // units per key of distance, in a scalar register
    return __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, slopes ? slopes[head] * per_slope : 0.f)));
  }
};
// row r of a 32 x 32 accumulator, in rows of the lane's half
constexpr int acc_row(int r) { return 8 * (r >> 2) + (r & 3); }
// lane's elements of an accumulator whose rows are keys (queries): those outside [from, from + count) become `fill`
__device__ __forceinline__ void keep_span(f32x16_t& a, int from, uint32_t count, float fill) {
#pragma unroll
  for (int r = 0; r < 16; ++r) a[r] = (uint32_t)(acc_row(r) - from) < count ? a[r] : fill;
}

// A hidden weight is zero, but zero times an infinite or undefined element is not.  The kernels multiply as if all elements were
// finite; where a sum comes out otherwise the workgroup walks again, and in tiles with hidden scores such elements enter the products as
// zeros (finite_only) and are then added to the columns that see them.  (dK and dV have no registers for that: there a key with such a sum
// is made again by itself.)
__device__ __forceinline__ bool bf16_finite(uint32_t v) { return (v & 0x7f80u) != 0x7f80u; }
__device__ __forceinline__ bf16x8_t finite_only(bf16x8_t v) {
  uint4 w = __builtin_bit_cast(uint4, v);
  uint32_t* p = &w.x;
#pragma unroll
  for (int i = 0; i < 4; ++i) p[i] = (bf16_finite(p[i]) ? p[i] & 0xffffu : 0u) | (bf16_finite(p[i] >> 16) ? p[i] & 0xffff0000u : 0u);
  return __builtin_bit_cast(bf16x8_t, w);
}
// acc (rows dh, the lane's column) += w X over the tile's rows row0 .. of X whose elements are not finite; seen(r): whether the lane's
// column sees row row0 + r
template <int NDT, int SUBS, class Seen>
__device__ __forceinline__ void add_nonfinite(f32x16_t (&acc)[NDT], const f32x16_t (&w)[SUBS], const bf16_t* __restrict__ x, size_t rs, int row0, int s,
                                              int lane, Seen seen) {
  const int half = lane >> 5, l31 = lane & 31;
#pragma unroll 1
  for (int r = 0; r < 32 * SUBS && row0 + r < s; ++r) {
    const bf16_t* row = x + (size_t)(row0 + r) * rs;
    bool some = false;
#pragma unroll
    for (int d = 0; d < NDT * 32; d += 64) some |= d + lane < NDT * 32 && !bf16_finite(row[min(d + lane, NDT * 32 - 1)]);
    if (!__any(some)) continue;
    const int at = (r >> 5) * 16 + ((r & 31) >> 3) * 4 + (r & 3);
    float mine = 0.f;
#pragma unroll
    for (int sub = 0; sub < SUBS; ++sub)
#pragma unroll
      for (int k = 0; k < 16; ++k) mine = sub * 16 + k == at ? w[sub][k] : mine;
    const float wr = __shfl(mine, ((r >> 2) & 1) * 32 + l31, 64);
    const bool sees = seen(r);
#pragma unroll
    for (int d = 0; d < NDT; ++d)
#pragma unroll
      for (int k = 0; k < 16; ++k) {
        const uint32_t v = row[d * 32 + acc_row(k) + 4 * half];
        if (sees && !bf16_finite(v)) acc[d][k] += wr * __uint_as_float(v << 16);
        if (k % 4 == 3) asm volatile("" ::: "memory");   // not all of the row's loads at once: this is rare, its registers are dear
      }
  }
}
template <int N> __device__ __forceinline__ bool all_finite(const f32x16_t (&acc)[N]) {
  float t = 0.f;
#pragma unroll
  for (int d = 0; d < N; ++d)
#pragma unroll
    for (int r = 0; r < 16; ++r) t = fmaf(acc[d][r], 0.f, t);
  return t == 0.f;
}
// whether any thread of the workgroup says so; flag: LDS that nothing else uses until the next barrier
__device__ __forceinline__ bool any_of_workgroup(bool mine, int* flag) {
  __syncthreads();
  if (threadIdx.x == 0) *flag = 0;
  __syncthreads();
  if (mine) *flag = 1;
  __syncthreads();
  const bool any = *flag != 0;
  if (any) __syncthreads();   // read by all before the place is used again
  return any;
}

// ------------------------------------------------------------------------------------------------
// Forward, bf16: a workgroup owns 32 QW queries of a head, 32 to a wave; tiles of KT keys stream through two LDS stages, requested one
// tile ahead, with one barrier per tile; NP = 2: two groups of waves take tiles in turn and their results are merged.
// Bound by exponentials and products that wait for each other inside a wave (two waves to a SIMD): 4 x 2048 tokens, 16 heads of 128, causal: 92 us,
// 750 TFLOP/s of the visible pairs; with documents of 400 46 us, where 134 MB in and out would take 27.
// ------------------------------------------------------------------------------------------------
template <int DH, int QW, int NP, int KT>
__global__ void __launch_bounds__(64 * QW * NP, 2)
attn_span_fwd_kernel(const bf16_t* __restrict__ qkv, bf16_t* __restrict__ ctx, float* __restrict__ lse, SpanView view, SpanShape z) {
  constexpr int NKK = DH / 16, NDT = DH / 32, SUBS = KT / 32;
  constexpr uint32_t kTile = TileDma<DH, QW, KT, false>::kBytes, kStage = 2 * kTile;
  extern __shared__ __attribute__((aligned(1024))) char smem_all[];
  const int wave_all = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), grp = NP == 1 ? 0 : wave_all / QW, wave = wave_all % QW;
  const uint32_t lds0 = attn_lds_offset(smem_all) + grp * 2 * kStage;
  const int s = z.s, b = z.b, nqb = (s + 32 * QW - 1) / (32 * QW);
  int qblk, e, j;
  if (!attn_map_tiles<true>(blockIdx.x, nqb, z.heads, b, &qblk, &e, &j)) return;
  qblk = nqb - 1 - qblk;   // long rows first
  const int lane = threadIdx.x & 63, half = lane >> 5, l31 = lane & 31, kve = e / (z.heads / z.kv_heads);
  const size_t row = (size_t)(z.heads + 2 * z.kv_heads) * DH, rs = b * row;
  const bf16_t* sample = qkv + j * row;
  const bf16_t *qb = sample + (size_t)e * DH, *kb = sample + (size_t)(z.heads + kve) * DH, *vb = kb + (size_t)z.kv_heads * DH;
  const int q_first = (qblk * QW + wave) * 32, my_q = q_first + l31;
  const SpanBounds blk = bounds_of(view, j, qblk * QW, QW, s), own = bounds_of(view, j, qblk * QW + wave, 1, s);
  const int kt_first = blk.first / KT, kt_end = blk.last > 0 ? (blk.last + KT - 1) / KT : kt_first;
  TileDma<DH, QW, KT, false> dma;
  dma.init(rs, lane);
  auto request = [&](int kt, uint32_t stage) {
    dma.issue(kb, kt * KT, s, lds0 + stage, wave);
    dma.issue(vb, kt * KT, s, lds0 + stage + kTile, wave);
  };
  const int2 span = my_q < s ? span_of(view, j, my_q, s) : make_int2(kNoKey, 0);
  const uint32_t count = (uint32_t)max(span.y - span.x, 0);
  const float bias = z.bias(e);
  bf16x8_t qf[NKK];
#pragma unroll
  for (int kk = 0; kk < NKK; ++kk) qf[kk] = frag_global(qb + (size_t)min(my_q, s - 1) * rs, my_q < s, kk, half);
  FragDirect<KT> fk;
  FragTr<KT> fv;
  fk.init(lds0, l31, half);
  fv.init(lds0 + kTile, lane);
  f32x16_t o[NDT];
  float m_run, l_run;

  auto walk = [&](auto careful) {   // careful: see add_nonfinite
    constexpr bool CAREFUL = decltype(careful)::value;
    if (kt_first + grp < kt_end) request(kt_first + grp, 0);
#pragma unroll
    for (int d = 0; d < NDT; ++d) o[d] = zero16();
    m_run = -INFINITY;
    l_run = 0.f;
    uint32_t stage = 0;
    // all groups take the same number of steps (the barriers are the workgroup's); a group without a tile idles
    for (int kt0 = kt_first; kt0 < kt_end; kt0 += NP, stage ^= kStage) {
      const int kt = kt0 + grp, key0 = kt * KT;
      attn_tiles_ready();
      if (kt + NP < kt_end) request(kt + NP, stage ^ kStage);
      // (no query of the wave sees a key of the tile)
      if (kt >= kt_end || own.first >= key0 + KT || own.last <= key0) continue;
      const bool full = own.inner_lo <= key0 && own.inner_hi >= key0 + KT;

      f32x16_t sacc[SUBS];
#pragma unroll
      for (int sub = 0; sub < SUBS; ++sub) sacc[sub] = zero16();
      const FragDirect<KT> fks = fk.at(stage);
#pragma unroll
      for (int kk = 0; kk < NKK; ++kk)
#pragma unroll
        for (int sub = 0; sub < SUBS; ++sub) sacc[sub] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fks.get(sub, kk), qf[kk], sacc[sub], 0, 0, 0);
      sched_reads_ahead<SUBS * NKK, 1>();
      __builtin_amdgcn_sched_barrier(0);
      if (z.capped()) {
#pragma unroll
        for (int sub = 0; sub < SUBS; ++sub) {
          if (!full) {
            z.tanh_to_the_digit(sacc[sub]);
          } else {
#pragma unroll
            for (int r = 0; r < 16; ++r) sacc[sub][r] = z.tanh(sacc[sub][r]);
          }
        }
      }
      if (z.slopes) {
        const float ahead = (float)(my_q - key0 - 4 * half);
#pragma unroll
        for (int sub = 0; sub < SUBS; ++sub)
#pragma unroll
          for (int r = 0; r < 16; ++r) sacc[sub][r] = fmaf(-bias, fabsf(ahead - (float)(sub * 32 + acc_row(r))), sacc[sub][r]);
      }
      if (!full) {
#pragma unroll
        for (int sub = 0; sub < SUBS; ++sub) keep_span(sacc[sub], span.x - key0 - sub * 32 - 4 * half, count, -INFINITY);
      }
      float mx = m_run;
#pragma unroll
      for (int sub = 0; sub < SUBS; ++sub)
#pragma unroll
        for (int r = 0; r < 16; ++r) mx = fmaxf(mx, sacc[sub][r]);
      const LaneHalves mh = lane_halves(mx);
      mx = fmaxf(mh.lo, mh.hi);
      const float ref = mx == -INFINITY ? 0.f : mx;   // no key of the row so far: weights of zero, not exp(-inf + inf)
      if (__any(mx > m_run)) {   // some row's maximum moved: rescale what has been accumulated
        const float corr = __builtin_amdgcn_exp2f((m_run - ref) * z.mul);
        m_run = mx;
        l_run *= corr;
#pragma unroll
        for (int d = 0; d < NDT; ++d)
#pragma unroll
          for (int r = 0; r < 16; ++r) o[d][r] *= corr;
      }
      const float mc = ref * z.mul;
      bf16x8_t pf[SUBS][2], vr[2][NDT];
      auto weights = [&](int sub) {
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          sacc[sub][r] = __builtin_amdgcn_exp2f(sacc[sub][r] * z.mul - mc);
          l_run += sacc[sub][r];
        }
        pf[sub][0] = pack_frag(sacc[sub], 0);
        pf[sub][1] = pack_frag(sacc[sub], 1);
      };
      const FragTr<KT> fvs = fv.at(stage);
      auto read_v = [&](int u) {
#pragma unroll
        for (int d = 0; d < NDT; ++d) vr[u & 1][d] = fvs.get(d, u >> 1, u & 1);
      };
      auto multiply = [&](int u) {
#pragma unroll
        for (int d = 0; d < NDT; ++d) o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vr[u & 1][d], pf[u >> 1][u & 1], o[d], 0, 0, 0);
      };
      if (CAREFUL && !full) {
#pragma unroll
        for (int sub = 0; sub < SUBS; ++sub) weights(sub);
#pragma unroll
        for (int u = 0; u < 2 * SUBS; ++u) {
          read_v(u);
#pragma unroll
          for (int d = 0; d < NDT; ++d) vr[u & 1][d] = finite_only(vr[u & 1][d]);
          multiply(u);
        }
        add_nonfinite<NDT, SUBS>(o, sacc, vb, rs, key0, s, lane, [&](int r) { return (uint32_t)(key0 + r - span.x) < count; });
        continue;
      }
      read_v(0);
      weights(0);
      __builtin_amdgcn_sched_barrier(0);
      if constexpr (SUBS == 2) {   // the second half's exponentials between the first half's products
        read_v(1);
        multiply(0);
        read_v(2);
        multiply(1);
        weights(1);
        sched_mixed<2 * NDT, 2, 56>();
        __builtin_amdgcn_sched_barrier(0);
      }
      read_v(2 * SUBS - 1);
      multiply(2 * SUBS - 2);
      multiply(2 * SUBS - 1);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  walk(std::false_type{});
  if (any_of_workgroup(!all_finite(o), reinterpret_cast<int*>(smem_all))) walk(std::true_type{});
  l_run += __shfl_xor(l_run, 32, 64);
  if constexpr (NP > 1) {
    // the second group's partial results join the first's: value v of lane l of wave w at part[w][v][l]
    float* part = reinterpret_cast<float*>(smem_all) + wave * ((2 + NDT * 16) * 64) + lane;
    __syncthreads();   // every wave is done with the tiles
    if (grp == 1) {
      part[0] = m_run;
      part[64] = l_run;
#pragma unroll
      for (int d = 0; d < NDT; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) part[(2 + d * 16 + r) * 64] = o[d][r];
    }
    __syncthreads();
    if (grp == 1) return;
    const float m1 = part[0], l1 = part[64], m = fmaxf(m_run, m1), ref = m == -INFINITY ? 0.f : m;
    const float a0 = __builtin_amdgcn_exp2f((m_run - ref) * z.mul), a1 = __builtin_amdgcn_exp2f((m1 - ref) * z.mul);
    l_run = l_run * a0 + l1 * a1;
    m_run = m;
#pragma unroll
    for (int d = 0; d < NDT; ++d)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[d][r] = o[d][r] * a0 + part[(2 + d * 16 + r) * 64] * a1;
  }
  if (my_q < s) {
    store_cols<NDT>(ctx + ((size_t)my_q * b + j) * z.heads * DH + (size_t)e * DH, o, count ? 1.f / l_run : 0.f, half);
    if (half == 0) lse[((size_t)j * z.heads + e) * s + my_q] = count ? m_run * (z.mul / kLog2e) + __logf(l_run) : -INFINITY;
  }
}

// ------------------------------------------------------------------------------------------------
// Backward, bf16.  dQ: a workgroup owns 32 QW queries and walks their keys as the forward kernel does; it also writes every query's
// lse log2(e) (infinite where nothing is seen) and D = dctx.ctx, which the dK/dV kernel, launched next, reads.  4 x 2048 tokens, 16 heads of
// 128, causal: 127 us, 810 TFLOP/s.
// ctx has been rounded to bf16, and where a softmax is sharp dp - D is a small difference: D from it is off by up to
// 2^-8 |dctx| |ctx| / sqrt(dh).  The rows' sums of p (dp - D), zero by definition, tell by how much: what dK gets
// is the corrected D, and walks of up to kSpanTwice tiles, whose few keys average least out, are made once more with it (dQ's
// relative error against 64 bits with a row's D as it is, s = 2, 8, 100, 2048: 3.9e-3, 4.3e-3, 2.9e-3, 2.6e-3; two roundings alone 2.3e-3).
// ------------------------------------------------------------------------------------------------
constexpr int kSpanTwice = 2;
template <int DH, int QW, int NP, int KT>
__global__ void __launch_bounds__(64 * QW * NP, 2)
attn_span_dq_kernel(const bf16_t* __restrict__ qkv, const bf16_t* __restrict__ ctx, const bf16_t* __restrict__ dctx, const float* __restrict__ lse,
                    float2* __restrict__ stats, bf16_t* __restrict__ dqkv, SpanView view, SpanShape z) {
  constexpr int NKK = DH / 16, NDT = DH / 32, SUBS = KT / 32;
  constexpr uint32_t kTile = TileDma<DH, QW, KT, false>::kBytes, kStage = 2 * kTile;
  extern __shared__ __attribute__((aligned(1024))) char smem_all[];
  const int wave_all = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), grp = NP == 1 ? 0 : wave_all / QW, wave = wave_all % QW;
  const uint32_t lds0 = attn_lds_offset(smem_all) + grp * 2 * kStage;
  const int s = z.s, b = z.b, nqb = (s + 32 * QW - 1) / (32 * QW);
  int qblk, e, j;
  if (!attn_map_tiles<true>(blockIdx.x, nqb, z.heads, b, &qblk, &e, &j)) return;
  qblk = nqb - 1 - qblk;   // long rows first
  const int lane = threadIdx.x & 63, half = lane >> 5, l31 = lane & 31, kve = e / (z.heads / z.kv_heads);
  const size_t row = (size_t)(z.heads + 2 * z.kv_heads) * DH, rs = b * row;
  const bf16_t* sample = qkv + j * row;
  const bf16_t *qb = sample + (size_t)e * DH, *kb = sample + (size_t)(z.heads + kve) * DH, *vb = kb + (size_t)z.kv_heads * DH;
  const int q_first = (qblk * QW + wave) * 32, my_q = q_first + l31;
  const bool valid = my_q < s;
  const SpanBounds blk = bounds_of(view, j, qblk * QW, QW, s), own = bounds_of(view, j, qblk * QW + wave, 1, s);
  const int kt_first = blk.first / KT, kt_end = blk.last > 0 ? (blk.last + KT - 1) / KT : kt_first;
  TileDma<DH, QW, KT, false> dma;
  dma.init(rs, lane);
  auto request = [&](int kt, uint32_t stage) {
    dma.issue(kb, kt * KT, s, lds0 + stage, wave);
    dma.issue(vb, kt * KT, s, lds0 + stage + kTile, wave);
  };
  const int2 span = valid ? span_of(view, j, my_q, s) : make_int2(kNoKey, 0);
  const uint32_t count = (uint32_t)max(span.y - span.x, 0);
  const float bias = z.bias(e);
  const size_t stat = ((size_t)j * z.heads + e) * s + my_q;
  const float L2 = count ? lse[stat] * kLog2e : INFINITY;   // an empty span: weights of zero
  bf16x8_t qf[NKK], dof[NKK];
  const size_t out_row = ((size_t)min(my_q, s - 1) * b + j) * z.heads * DH + (size_t)e * DH;
#pragma unroll
  for (int kk = 0; kk < NKK; ++kk) {
    qf[kk] = frag_global(qb + (size_t)min(my_q, s - 1) * rs, valid, kk, half);
    dof[kk] = frag_global(dctx + out_row, valid, kk, half);
  }
  float D = attn_delta_of<DH>(ctx + out_row, dof, valid, lane), over;   // over: the lane's share of sum_k p (dp - D)
  FragDirect<KT> fk, fv;
  FragTr<KT> ft;
  fk.init(lds0, l31, half);
  fv.init(lds0 + kTile, l31, half);
  ft.init(lds0, lane);
  f32x16_t acc[NDT];

  auto walk = [&](auto careful) {   // careful: see add_nonfinite
    constexpr bool CAREFUL = decltype(careful)::value;
    if (kt_first + grp < kt_end) request(kt_first + grp, 0);
#pragma unroll
    for (int d = 0; d < NDT; ++d) acc[d] = zero16();
    over = 0.f;
    uint32_t stage = 0;
    for (int kt0 = kt_first; kt0 < kt_end; kt0 += NP, stage ^= kStage) {
      const int kt = kt0 + grp, key0 = kt * KT;
      attn_tiles_ready();
      if (kt + NP < kt_end) request(kt + NP, stage ^ kStage);
      if (kt >= kt_end || own.first >= key0 + KT || own.last <= key0) continue;
      const bool full = own.inner_lo <= key0 && own.inner_hi >= key0 + KT;
      const FragDirect<KT> fks = fk.at(stage), fvs = fv.at(stage);
      const FragTr<KT> fts = ft.at(stage);
#pragma unroll
      for (int sub = 0; sub < SUBS; ++sub) {
        f32x16_t sacc = zero16(), dp = zero16();
#pragma unroll
        for (int kk = 0; kk < NKK; ++kk) {
          sacc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fks.get(sub, kk), qf[kk], sacc, 0, 0, 0);
          dp = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fvs.get(sub, kk), dof[kk], dp, 0, 0, 0);
        }
        sched_reads_ahead<2 * NKK, 1>();
        __builtin_amdgcn_sched_barrier(0);
        const float ahead = (float)(my_q - key0 - sub * 32 - 4 * half);
        if (z.capped()) {
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const float th = z.tanh(sacc[r]), t = fmaf(-bias, fabsf(ahead - (float)acc_row(r)), th);
            sacc[r] = __builtin_amdgcn_exp2f(t * z.mul - L2) * (dp[r] - D);
            dp[r] = fmaf(-th, th, 1.f);
          }
        } else {
          if (z.slopes) {
#pragma unroll
            for (int r = 0; r < 16; ++r) sacc[r] = fmaf(-bias, fabsf(ahead - (float)acc_row(r)), sacc[r]);
          }
#pragma unroll
          for (int r = 0; r < 16; ++r) sacc[r] = __builtin_amdgcn_exp2f(sacc[r] * z.mul - L2) * (dp[r] - D);
        }
        if (!full) keep_span(sacc, span.x - key0 - sub * 32 - 4 * half, count, 0.f);
#pragma unroll
        for (int r = 0; r < 16; ++r) over += sacc[r];
        if (z.capped()) {
          if (!full) keep_span(dp, span.x - key0 - sub * 32 - 4 * half, count, 0.f);   // (zero times a hidden NaN)
#pragma unroll
          for (int r = 0; r < 16; ++r) sacc[r] *= dp[r];
        }
        const bf16x8_t dsf[2] = {pack_frag(sacc, 0), pack_frag(sacc, 1)};
        if (CAREFUL && !full) {
#pragma unroll
          for (int ks = 0; ks < 2; ++ks)
#pragma unroll
            for (int d = 0; d < NDT; ++d) acc[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(finite_only(fts.get(d, sub, ks)), dsf[ks], acc[d], 0, 0, 0);
          const f32x16_t w[1] = {sacc};
          add_nonfinite<NDT, 1>(acc, w, kb, rs, key0 + sub * 32, s, lane, [&](int r) { return (uint32_t)(key0 + sub * 32 + r - span.x) < count; });
        } else {
#pragma unroll
          for (int ks = 0; ks < 2; ++ks)
#pragma unroll
            for (int d = 0; d < NDT; ++d) acc[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fts.get(d, sub, ks), dsf[ks], acc[d], 0, 0, 0);
          sched_reads_ahead<2 * NDT, 2>();
          __builtin_amdgcn_sched_barrier(0);
        }
      }
    }
  };
  // the row's sum_k p (dp - D): what D is short of
  auto missing = [&] {
    float v = over + __shfl_xor(over, 32, 64);
    if constexpr (NP == 2) {
      float* other = reinterpret_cast<float*>(smem_all) + wave * 64 + lane;
      __syncthreads();   // every wave is done with the tiles
      other[(grp ^ 1) * QW * 64] = v;
      __syncthreads();
      v = grp == 0 ? v + other[0] : other[grp * QW * 64] + v;   // the first group's share first, in both
      __syncthreads();   // read by all before the place is used again
    }
    return v;
  };
  walk(std::false_type{});
  float miss = missing();
  if (kt_end - kt_first <= kSpanTwice) {
    D += miss;
    walk(std::false_type{});
    miss = missing();
  }
  if (any_of_workgroup(!all_finite(acc), reinterpret_cast<int*>(smem_all))) {
    walk(std::true_type{});
    miss = missing();
  }
  if (grp == 0 && half == 0 && valid) stats[stat] = make_float2(L2, D + miss);
  if constexpr (NP > 1) {
    // the second group's sums join the first's: register r of lane l of wave w at sum[w][r][l]
    float* sum = reinterpret_cast<float*>(smem_all) + wave * (NDT * 16 * 64) + lane;
    __syncthreads();   // every wave is done with the tiles
    if (grp == 1) {
#pragma unroll
      for (int d = 0; d < NDT; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) sum[(d * 16 + r) * 64] = acc[d][r];
    }
    __syncthreads();
    if (grp == 1) return;
#pragma unroll
    for (int d = 0; d < NDT; ++d)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[d][r] += sum[(d * 16 + r) * 64];
  }
  if (valid) store_cols<NDT>(dqkv + (size_t)my_q * rs + j * row + (size_t)e * DH, acc, z.scale, half);
}

// QT queries' eight bytes each from `from` to LDS, zeros from `bytes` on: lane i's four bytes land at lds + 4 i (assembly as attn_load_lds)
template <int QT> __device__ __forceinline__ void span_load_rows(const void* from, int bytes, uint32_t lds, int lane) {
  const uint64_t a = reinterpret_cast<uint64_t>(from);
  const attn_rsrc_t r = {(uint32_t)a, (uint32_t)(a >> 32) & 0xffffu, bytes > 0 ? (uint32_t)bytes : 0u, 0x00020000u};
#pragma unroll
  for (int i = 0; i < QT / 32; ++i)
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dword %1, %2, 0 offen lds" :: "s"(lds + i * 256), "v"(i * 256 + lane * 4), "s"(r) : "memory", "m0");
}

// dK, dV of 32 KW keys of a key/value head: the queries of the group's heads that may see them, head after head, stream through LDS stages
// of QT queries, with their statistics (lse, D) and spans, all of it straight from memory.  Nothing of the next tile passes through vector
// registers: both results, K and V leave none over.
// SPLIT: KW waves keep K and V and make P and dS of a tile, KW waves keep both results and add the tile before it up; the weights go from one
// to the other through LDS as the fragments they are, and three stages hold the tiles.  A SIMD has one wave of each kind, so that exponentials
// run beside products, and no score is made twice.  Heads of 128 and 160, whose results and operands together fill more than a wave's registers;
// dK/dV alone, us, against two halves of which each makes the scores and one result: 4096 x 20 x 160: 243 and 295; capped with 4 key/value heads:
// 300 and 487; 16384 in documents, 8 x 128 on 2: 637 and 784.  Smaller heads: one wave does it all (2048 x 32 x 64: 50, split 58).
template <int DH, int KW, int NP, int QT, bool SPLIT> struct SpanDkvGeom {
  static constexpr int kWaves = SPLIT ? 2 * KW : KW, kThreads = 64 * kWaves;   // of a group
  static constexpr int kTile = QT * DH * 2, kStats = 2 * kTile, kSpans = kStats + 8 * QT, kStage = kSpans + 8 * QT;
  static constexpr int kStages = SPLIT ? 3 : 2, kWeights = kStages * kStage, kWave = QT / 32 * 4096;   // P and dS of a wave's tile
  static constexpr int kGroup = kWeights + (SPLIT ? 2 * KW * kWave : 0);
  static constexpr int kSums = NP > 1 ? KW * 2 * (DH / 2) * 64 * (int)sizeof(float) : 0;
  static constexpr int kBytes = NP * kGroup > kSums ? NP * kGroup : kSums;
  static_assert(kBytes <= 160 * 1024);
};
struct SpanDkvArgs {
  const bf16_t *qkv, *dctx;
  const float2* stats;
  bf16_t* dqkv;
  SpanView view;
  SpanShape z;
  int parts;         // of a key block's walk, each a workgroup's
  float* partial;    // their sums, if there is more than one
};
// where a part's sums of one result (dK or dV) of 32 keys begin: registers 4 g .. 4 g + 3 of acc[d] of lane l are the four at 256 (4 d + g) + 4 l
__device__ __forceinline__ size_t span_partial_at(const SpanShape& z, int part, int j, int kve, int k32, int dk, int dh) {
  return (((((size_t)part * z.b + j) * z.kv_heads + kve) * ((z.s + 31) / 32) + k32) * 2 + dk) * (32 * (size_t)dh);
}
// A key whose dV or dK has a sum that is not finite (`want`: bit 0, bit 1) is made again from the queries that see it and from no others, an
// element to a lane and query after query: a hidden query's zero weight times what is not finite may have got in.  It reads the kernel's
// arguments from where the launch left them and is not inlined: kept for it, they would take the kernel's registers.
template <int DH> __device__ __attribute__((noinline)) void span_dkv_again(const SpanDkvArgs& a, int key, int kve, int j, int want) {
  const SpanShape& z = a.z;
  const int s = z.s, group = z.heads / z.kv_heads, lane = threadIdx.x & 63;
  const size_t row = (size_t)(z.heads + 2 * z.kv_heads) * DH, rs = z.b * row, dors = (size_t)z.b * z.heads * DH;
  const bf16_t *sample = a.qkv + j * row, *kr = sample + (size_t)key * rs + (size_t)(z.heads + kve) * DH, *vr = kr + (size_t)z.kv_heads * DH;
  constexpr int NE = (DH + 63) / 64;
  auto element = [&](const bf16_t* from, int i) { return 64 * i + lane < DH ? bf16_to_f32(from[64 * i + lane]) : 0.f; };
  float ke[NE], ve[NE], dk[NE], dv[NE];
#pragma unroll
  for (int i = 0; i < NE; ++i) {
    ke[i] = element(kr, i);
    ve[i] = element(vr, i);
    dk[i] = dv[i] = 0.f;
  }
#pragma unroll 1
  for (int head = kve * group; head < (kve + 1) * group; ++head) {
    const float bias = z.bias(head);
    const float2* st = a.stats + ((size_t)j * z.heads + head) * s;
#pragma unroll 1
    for (int q = 0; q < s; ++q) {
      const int2 x = span_of(a.view, j, q, s);
      if (!((uint32_t)(key - x.x) < (uint32_t)(x.y - x.x))) continue;
      const bf16_t *qr = sample + (size_t)q * rs + (size_t)head * DH, *dr = a.dctx + (size_t)q * dors + ((size_t)j * z.heads + head) * DH;
      float qe[NE], de[NE], qk = 0.f, dp = 0.f;
#pragma unroll
      for (int i = 0; i < NE; ++i) {
        qe[i] = element(qr, i);
        de[i] = element(dr, i);
        qk = fmaf(qe[i], ke[i], qk);
        dp = fmaf(de[i], ve[i], dp);
      }
      qk = wave_sum(qk);
      dp = wave_sum(dp);
      const float th = z.capped() ? z.tanh(qk) : qk, p = __builtin_amdgcn_exp2f(fmaf(-bias, fabsf((float)(q - key)), th) * z.mul - st[q].x);
      const float ds = p * (dp - st[q].y) * (z.capped() ? fmaf(-th, th, 1.f) : 1.f);
#pragma unroll
      for (int i = 0; i < NE; ++i) {
        dv[i] = fmaf(p, de[i], dv[i]);
        dk[i] = fmaf(ds, qe[i], dk[i]);
      }
    }
  }
  bf16_t* to = a.dqkv + (kr - a.qkv);
#pragma unroll
  for (int i = 0; i < NE; ++i) {
    if (64 * i + lane >= DH) continue;
    if (want & 2) to[64 * i + lane] = f32_to_bf16(dk[i] * z.scale);
    if (want & 1) to[(size_t)z.kv_heads * DH + 64 * i + lane] = f32_to_bf16(dv[i]);
  }
}
// SCORED: there may be a cap or a bias.
template <int DH, int KW, int NP, int QT, bool SPLIT, bool SCORED>
__global__ void __launch_bounds__(64 * KW * (SPLIT ? 2 : 1) * NP, 2)
attn_span_dkv_kernel(SpanDkvArgs a) {
  const SpanView view = a.view;
  const SpanShape& z = a.z;
  using Geom = SpanDkvGeom<DH, KW, NP, QT, SPLIT>;
  constexpr int NKK = DH / 16, NDT = DH / 32, kKeys = 32 * KW, SUBS = QT / 32, GW = Geom::kWaves, kTile = Geom::kTile, kStage = Geom::kStage;
  extern __shared__ __attribute__((aligned(1024))) char smem_all[];
  const int wave_all = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), grp = NP == 1 ? 0 : wave_all / GW, wave = wave_all % GW;
  const int kw = wave % KW;
  static_assert(GW > 1);
  char* smem = smem_all + grp * Geom::kGroup;
  const uint32_t lds0 = attn_lds_offset(smem);
  const int s = z.s, b = z.b, nkb = (s + kKeys - 1) / kKeys, group = z.heads / z.kv_heads;
  int kblk, kve, j;   // the first key blocks see the most queries under the causal mask and start first
  if (!attn_map_tiles<true>(blockIdx.x, nkb, z.kv_heads * a.parts, b, &kblk, &kve, &j)) return;
  const int part = kve % a.parts;
  kve /= a.parts;
  // (which half makes the weights alternates where it takes that to give every SIMD both)
  const bool sums_only = SPLIT && ((wave / KW) ^ (KW == 4 ? 0 : NP == 2 ? grp : (int)(blockIdx.x >> 8))) & 1;
  const int lane = threadIdx.x & 63, half = lane >> 5, l31 = lane & 31;
  const size_t row = (size_t)(z.heads + 2 * z.kv_heads) * DH, rs = b * row, orow = (size_t)z.heads * DH, dors = b * orow;
  const bf16_t* sample = a.qkv + j * row;
  const bf16_t *kb = sample + (size_t)(z.heads + kve) * DH, *vb = kb + (size_t)z.kv_heads * DH;
  const bf16_t *qb = sample + (size_t)kve * group * DH, *dob = a.dctx + j * orow + (size_t)kve * group * DH;
  const size_t stat0 = ((size_t)j * z.heads + (size_t)kve * group) * s;
  const int key_blk = kblk * kKeys, key_first = key_blk + kw * 32, my_key = key_first + l31;
  const bool valid = my_key < s;

  // the tiles of queries that may see a key of the block: from the first to the last block of 32 queries whose bounds meet it
  int qt_first = key_blk / QT, qt_end = (s + QT - 1) / QT;
  const int nt = (s + kSpanRows - 1) / kSpanRows;
  const SpanBounds* bounds = view.bounds + (size_t)j * nt;   // (read if there are spans)
  if (view.range) {
    int* found = reinterpret_cast<int*>(smem_all);
    if (threadIdx.x == 0) {
      found[0] = kNoKey;
      found[1] = -1;
    }
    __syncthreads();
    for (int t = threadIdx.x; t < nt; t += blockDim.x) {
      const SpanBounds y = bounds[t];
      if (y.first < key_blk + kKeys && y.last > key_blk) {
        atomicMin(&found[0], t);
        atomicMax(&found[1], t);
      }
    }
    __syncthreads();
    const int a = __builtin_amdgcn_readfirstlane(found[0]), e = __builtin_amdgcn_readfirstlane(found[1]);
    __syncthreads();
    qt_first = e < 0 ? 0 : a * kSpanRows / QT;
    qt_end = e < 0 ? 0 : e * kSpanRows / QT + 1;
  }
  // tile t of the walk is tile t % nq of head t / nq; a part takes a share of them, one after the other
  const int nq = qt_end - qt_first, share = (group * nq + a.parts - 1) / a.parts, t_first = part * share;
  const int t_end = min(group * nq, t_first + share), steps = t_end > t_first ? (t_end - t_first + NP - 1) / NP : 0;

  // every wave loads a share of both tiles, or one half's first waves Q and the other's dO
  constexpr int kSlices = QT / 16, DW = GW > kSlices ? kSlices : GW;
  TileDma<DH, DW, QT, false> dma_q, dma_do;
  dma_q.init(rs, lane);
  dma_do.init(dors, lane);
  struct Place { int t, head, qt; };   // of the walk; the head of the group; its tile
  auto settle = [&](Place p) {
    while (p.qt >= qt_end) {
      p.qt -= nq;
      ++p.head;
    }
    return p;
  };
  auto request = [&](Place p, uint32_t at) {
    if (GW == DW || wave < DW) dma_q.issue(qb + (size_t)p.head * DH, p.qt * QT, s, lds0 + at, wave % DW);
    if (GW == DW || (wave >= GW / 2 && wave < GW / 2 + DW)) dma_do.issue(dob + (size_t)p.head * DH, p.qt * QT, s, lds0 + at + kTile, wave % DW);
    // eight bytes a query, zeros past the end
    const int q = p.qt * QT, bytes = min(QT, s - q) * 8;
    if (wave == GW - 1) span_load_rows<QT>(a.stats + stat0 + (size_t)p.head * s + q, bytes, lds0 + at + Geom::kStats, lane);
    if (wave == GW - 2 && view.range) span_load_rows<QT>(view.range + (size_t)j * s + q, bytes, lds0 + at + Geom::kSpans, lane);
  };
  // the tile's bounds and bias, from scalar loads: they are a tile's to wait for, not a lane's
  typedef __attribute__((address_space(4))) const int scalar_int_t;
  auto bounds_of_tile = [&](Place p) {
    if (!view.range) return SpanBounds{0, min(s, (p.qt + 1) * QT), 0, p.qt * QT + 1};
    SpanBounds x = {kNoKey, 0, 0, kNoKey};
#pragma unroll
    for (int i = 0; i < SUBS; ++i) {   // (a block past the last one is the last one again)
      const scalar_int_t* y = (scalar_int_t*)(bounds + min(p.qt * SUBS + i, nt - 1));
      x = {min(x.first, y[0]), max(x.last, y[1]), max(x.inner_lo, y[2]), min(x.inner_hi, y[3])};
    }
    return x;
  };
  FragDirect<QT> f0;
  FragTr<QT> t0;
  f0.init(lds0, l31, half);
  t0.init(lds0, lane);
  f32x16_t acc[2][NDT];   // dV and dK

  // the walk of a wave that makes the weights (P and dS), that adds up dV and dK, or that does both
  auto walk = [&](auto weights, auto sums) {
    constexpr bool WEIGHTS = decltype(weights)::value, SUMS = decltype(sums)::value;
    bf16x8_t kf[NKK], vf[NKK];
    if constexpr (WEIGHTS) {
#pragma unroll
      for (int kk = 0; kk < NKK; ++kk) {
        kf[kk] = frag_global(kb + (size_t)min(my_key, s - 1) * rs, valid, kk, half);
        vf[kk] = frag_global(vb + (size_t)min(my_key, s - 1) * rs, valid, kk, half);
      }
    }
    if constexpr (SUMS) {
#pragma unroll
      for (int r = 0; r < 2; ++r)
#pragma unroll
        for (int d = 0; d < NDT; ++d) acc[r][d] = zero16();
    }
    Place at = {t_first + grp, 0, qt_first};
    if (steps > 0) at = settle({at.t, t_first / nq, qt_first + t_first % nq + grp});
    if (at.t < t_end) request(at, 0);
    uint32_t stage = 0, before = 0, slot = Geom::kWeights + kw * Geom::kWave;
    bool had = false;   // the tile before was one to be done
    // all groups take the same number of steps (the barriers are the workgroup's); a group without a tile idles.  Where the work is split
    // the sums are a tile behind the weights.
#pragma unroll 1
    for (int step = 0; step < (SPLIT && steps > 0 ? steps + 1 : steps); ++step) {
      const int q0 = at.qt * QT, head = at.head;
      const SpanBounds bnd = bounds_of_tile(at);
      const float bias = WEIGHTS && SCORED && z.slopes ? ((__attribute__((address_space(4))) const float*)z.slopes)[min(kve * group + head, z.heads - 1)] * z.per_slope : 0.f;
      attn_tiles_ready();
      const Place then = settle({at.t + NP, at.head, at.qt + NP});
      const uint32_t other = stage == (Geom::kStages - 1) * kStage ? 0 : stage + kStage;
      if (then.t < t_end) request(then, other);
      // (skipped if no key of the wave exists or no query of the tile sees one)
      const bool here = at.t < t_end && key_first < s && bnd.first < key_first + 32 && bnd.last > key_first;
      if (WEIGHTS ? here : had) {
        const FragDirect<QT> fs = f0.at(stage);
        const FragTr<QT> ts = t0.at(SPLIT ? before : stage);
        const char *rows = smem + stage + Geom::kStats, *spans = smem + stage + Geom::kSpans;
        const bool full = bnd.inner_lo <= key_first && bnd.inner_hi >= key_first + 32;
#pragma unroll
        for (int sub = 0; sub < SUBS; ++sub) {
          bf16x8_t pf[2], dsf[2];
          // P and dS on their way from one wave to the other: four fragments, each 16 bytes of a lane
          bf16x8_t* way = reinterpret_cast<bf16x8_t*>(smem + slot + sub * 4096) + lane;
          if constexpr (WEIGHTS) {
            f32x16_t sacc = zero16(), dp = zero16();
#pragma unroll
            for (int kk = 0; kk < NKK; ++kk) {
              sacc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fs.get(sub, kk), kf[kk], sacc, 0, 0, 0);
              dp = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fs.get(sub, kk, kTile), vf[kk], dp, 0, 0, 0);
            }
            sched_reads_ahead<2 * NKK, 1>();
            __builtin_amdgcn_sched_barrier(0);
            const float ahead = (float)(my_key - q0 - sub * 32 - 4 * half);
            if (SCORED && z.slopes && !z.capped()) {
#pragma unroll
              for (int r = 0; r < 16; ++r) sacc[r] = fmaf(-bias, fabsf(ahead - (float)acc_row(r)), sacc[r]);
            }
            if (SCORED && z.capped()) {
#pragma unroll
              for (int g = 0; g < 4; ++g) {
                const char* four = rows + (sub * 32 + 8 * g + 4 * half) * 8;   // lse and D of four consecutive queries
                const f32x4_t two[2] = {*reinterpret_cast<const f32x4_t*>(four), *reinterpret_cast<const f32x4_t*>(four + 16)};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                  const int r = 4 * g + i;
                  const float th = z.tanh(sacc[r]), p = __builtin_amdgcn_exp2f(fmaf(-bias, fabsf(ahead - (float)acc_row(r)), th) * z.mul - two[i >> 1][2 * (i & 1)]);
                  sacc[r] = p;
                  dp[r] = p * (dp[r] - two[i >> 1][2 * (i & 1) + 1]) * fmaf(-th, th, 1.f);
                }
              }
            } else {
#pragma unroll
              for (int g = 0; g < 4; ++g) {
                const char* four = rows + (sub * 32 + 8 * g + 4 * half) * 8;
                const f32x4_t two[2] = {*reinterpret_cast<const f32x4_t*>(four), *reinterpret_cast<const f32x4_t*>(four + 16)};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                  const int r = 4 * g + i;
                  const float p = __builtin_amdgcn_exp2f(sacc[r] * z.mul - two[i >> 1][2 * (i & 1)]);
                  sacc[r] = p;
                  dp[r] = p * (dp[r] - two[i >> 1][2 * (i & 1) + 1]);
                }
              }
            }
            if (!full) {
              typedef int i32x4_t __attribute__((ext_vector_type(4)));
              if (view.range) {
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                  const char* four = spans + (sub * 32 + 8 * g + 4 * half) * 8;
                  const i32x4_t two[2] = {*reinterpret_cast<const i32x4_t*>(four), *reinterpret_cast<const i32x4_t*>(four + 16)};
#pragma unroll
                  for (int i = 0; i < 4; ++i) {   // (an empty span, {kNoKey, 0}, has no key either: no key is as far from kNoKey as 0 is)
                    const int lo = two[i >> 1][2 * (i & 1)], hi = two[i >> 1][2 * (i & 1) + 1];
                    const bool seen = (uint32_t)(my_key - lo) < (uint32_t)(hi - lo);
                    sacc[4 * g + i] = seen ? sacc[4 * g + i] : 0.f;
                    dp[4 * g + i] = seen ? dp[4 * g + i] : 0.f;
                  }
                }
              } else {
                const int before = my_key - q0 - sub * 32 - 4 * half;   // local queries below it precede my_key
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                  sacc[r] = acc_row(r) < before ? 0.f : sacc[r];
                  dp[r] = acc_row(r) < before ? 0.f : dp[r];
                }
              }
            }
            pf[0] = pack_frag(sacc, 0);
            pf[1] = pack_frag(sacc, 1);
            dsf[0] = pack_frag(dp, 0);
            dsf[1] = pack_frag(dp, 1);
          }
          if constexpr (SPLIT && WEIGHTS) {
#pragma unroll
            for (int ks = 0; ks < 2; ++ks) {
              way[ks * 64] = pf[ks];
              way[(2 + ks) * 64] = dsf[ks];
            }
          }
          if constexpr (SUMS) {
            if constexpr (SPLIT) {
#pragma unroll
              for (int ks = 0; ks < 2; ++ks) {
                pf[ks] = way[ks * 64];
                dsf[ks] = way[(2 + ks) * 64];
              }
              __builtin_amdgcn_sched_barrier(0);
            }
#pragma unroll
            for (int ks = 0; ks < 2; ++ks)
#pragma unroll
              for (int d = 0; d < NDT; ++d) {
                acc[0][d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ts.get(d, sub, ks, kTile), pf[ks], acc[0][d], 0, 0, 0);
                acc[1][d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ts.get(d, sub, ks), dsf[ks], acc[1][d], 0, 0, 0);
              }
            sched_reads_ahead<4 * NDT, 2>();
          }
          __builtin_amdgcn_sched_barrier(0);
        }
      }
      at = then;
      before = stage;
      stage = other;
      had = here;
      if (WEIGHTS || step > 0) slot = slot < Geom::kWeights + KW * Geom::kWave ? slot + KW * Geom::kWave : slot - KW * Geom::kWave;
    }
    if constexpr (SUMS) {   // whole accumulators up to here: the loop is not to carry the pieces that the stores want
#pragma unroll
      for (int r = 0; r < 2; ++r)
#pragma unroll
        for (int d = 0; d < NDT; ++d) asm volatile("" : "+v"(acc[r][d]));
    }
  };
  if constexpr (!SPLIT) walk(std::true_type{}, std::true_type{});
  if constexpr (SPLIT) {
    if (!sums_only) {
      walk(std::true_type{}, std::false_type{});
      if constexpr (NP > 1) {   // (the barriers below)
        __syncthreads();
        __syncthreads();
      }
      return;
    }
    walk(std::false_type{}, std::true_type{});
  }
  if constexpr (NP > 1) {
    // the second group's sums join the first's: register r of lane l of the wave with keys kw at sum[..][r][l]
    float* sum = reinterpret_cast<float*>(smem_all) + 2 * kw * (NDT * 16 * 64) + lane;
    __syncthreads();   // every wave is done with the tiles
    if (grp == 1) {
#pragma unroll
      for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int d = 0; d < NDT; ++d)
#pragma unroll
          for (int r = 0; r < 16; ++r) sum[((x * NDT + d) * 16 + r) * 64] = acc[x][d][r];
    }
    __syncthreads();
    if (grp == 1) return;
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
      for (int d = 0; d < NDT; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[x][d][r] += sum[((x * NDT + d) * 16 + r) * 64];
  }
  if (a.parts > 1) {
    if (key_first >= s) return;
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      f32x4_t* to = reinterpret_cast<f32x4_t*>(a.partial + span_partial_at(z, part, j, kve, kblk * KW + kw, x, DH)) + lane;
#pragma unroll
      for (int d = 0; d < NDT; ++d)
#pragma unroll
        for (int g = 0; g < 4; ++g) to[(4 * d + g) * 64] = f32x4_t{acc[x][d][4 * g], acc[x][d][4 * g + 1], acc[x][d][4 * g + 2], acc[x][d][4 * g + 3]};
    }
    return;
  }
  bf16_t* out = a.dqkv + (size_t)my_key * rs + j * row + (size_t)(z.heads + kve) * DH;   // dK; dV kv_heads further on
  uint64_t bad[2] = {0, 0};   // keys whose dV, dK has a sum that is not finite
#pragma unroll
  for (int x = 0; x < 2; ++x) {
    const uint64_t m = __ballot(valid && !all_finite(acc[x]));
    bad[x] = (m | m >> 32) & 0xffffffffu;
    if (valid && !(bad[x] >> l31 & 1)) store_cols<NDT>(out + (x == 1 ? 0 : (size_t)z.kv_heads * DH), acc[x], x == 1 ? z.scale : 1.f, half);
  }
  const SpanDkvArgs* kernargs = (const SpanDkvArgs*)(const char*)__builtin_amdgcn_kernarg_segment_ptr();   // (only a kernel knows the place)
#pragma unroll 1
  for (uint64_t left = bad[0] | bad[1]; left; left &= left - 1) {
    const int k = __ffsll((unsigned long long)left) - 1;
    span_dkv_again<DH>(*kernargs, key_first + k, kve, j, (int)(bad[0] >> k & 1) | (int)(bad[1] >> k & 1) << 1);
  }
}

// Adds the parts' sums, in their order: a workgroup has one result of 32 keys, a wave 32 of its columns.
template <int DH>
__global__ void __launch_bounds__(DH * 2)
attn_span_dkv_join_kernel(SpanDkvArgs a) {
  __shared__ uint32_t bad_keys;
  const SpanShape& z = a.z;
  const int nk32 = (z.s + 31) / 32, k32 = blockIdx.x % nk32, pair = blockIdx.x / nk32, kve = pair % z.kv_heads, j = pair / z.kv_heads, dk = blockIdx.y;
  const int d = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, half = lane >> 5, l31 = lane & 31, my_key = k32 * 32 + l31;
  if (threadIdx.x == 0) bad_keys = 0;
  f32x16_t acc[1] = {zero16()};
  for (int part = 0; part < a.parts; ++part) {
    const f32x4_t* from = reinterpret_cast<const f32x4_t*>(a.partial + span_partial_at(z, part, j, kve, k32, dk, DH)) + lane;
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const f32x4_t v = from[(4 * d + g) * 64];
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[0][4 * g + i] += v[i];
    }
  }
  __syncthreads();
  const bool valid = my_key < z.s;
  const uint64_t m = __ballot(valid && !all_finite(acc));
  if (m && lane == 0) atomicOr(&bad_keys, (uint32_t)(m | m >> 32));
  __syncthreads();
  const uint32_t bad = __builtin_amdgcn_readfirstlane(bad_keys);
  const size_t row = (size_t)(z.heads + 2 * z.kv_heads) * DH;
  if (valid && !(bad >> l31 & 1))
    store_cols<1>(a.dqkv + ((size_t)my_key * z.b + j) * row + (size_t)(z.heads + kve + (dk ? 0 : z.kv_heads)) * DH + d * 32, acc, dk ? z.scale : 1.f, half);
  if (d > 0) return;
  const SpanDkvArgs* kernargs = (const SpanDkvArgs*)(const char*)__builtin_amdgcn_kernarg_segment_ptr();
#pragma unroll 1
  for (uint32_t left = bad; left; left &= left - 1) span_dkv_again<DH>(*kernargs, k32 * 32 + __ffs(left) - 1, kve, j, 1 + dk);
}

// ------------------------------------------------------------------------------------------------
// fp32: a workgroup of four waves owns 16 queries (dK/dV: keys); wave w takes every fourth tile of the other side from tile w on, and the
// four sums meet in LDS.
// ------------------------------------------------------------------------------------------------
// over the sixteen lanes of a row (lane & 15)
__device__ __forceinline__ int row_min(int v) {
#pragma unroll
  for (int d = 1; d < 16; d *= 2) v = min(v, __shfl_xor(v, d, 64));
  return __builtin_amdgcn_readfirstlane(v);
}
__device__ __forceinline__ int row_max(int v) {
#pragma unroll
  for (int d = 1; d < 16; d *= 2) v = max(v, __shfl_xor(v, d, 64));
  return __builtin_amdgcn_readfirstlane(v);
}
struct F32Rule {
  float scale, cap, bias;
  __device__ __forceinline__ F32Rule(const SpanShape& z, int head) : scale(z.scale), cap(z.cap), bias(z.slopes ? z.slopes[head] : 0.f) {}
  // t of a product q.k at this distance, and its derivative with respect to scale q.k
  __device__ __forceinline__ float score(float qk, int distance, float* d) const {
    float x = qk * scale;
    *d = 1.f;
    if (cap > 0.f) {
      const float th = tanhf(x / cap);
      *d = fmaf(-th, th, 1.f);
      x = cap * th;
    }
    return fmaf(-bias, fabsf((float)distance), x);
  }
};

template <int ND>
__global__ void __launch_bounds__(256)
attn_span_fwd_f32(const float* __restrict__ qkv, float* __restrict__ ctx, float* __restrict__ lse, SpanView view, SpanShape z, int dh) {
  __shared__ f32x4_t part[3 * ND * 64];
  __shared__ float stat[2][4][16];
  const int e = blockIdx.y, j = blockIdx.z, wave = threadIdx.x >> 6, lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
  const int s = z.s, b = z.b, q0 = ((int)gridDim.x - 1 - (int)blockIdx.x) * kF32Rows, my_q = q0 + c, qr = min(my_q, s - 1);   // long rows first
  const int kve = e / (z.heads / z.kv_heads);
  const size_t row = (size_t)(z.heads + 2 * z.kv_heads) * dh, rs = b * row;
  const float* sample = qkv + j * row;
  const float *kb = sample + (size_t)(z.heads + kve) * dh, *vb = kb + (size_t)z.kv_heads * dh;
  const int2 span = my_q < s ? span_of(view, j, my_q, s) : make_int2(kNoKey, 0);
  const int first = row_min(span.x), last = row_max(span.y), inner_lo = row_max(my_q < s ? span.x : 0), inner_hi = row_min(my_q < s ? span.y : kNoKey);
  const F32Rule rule(z, e);
  F32Frag<ND> q;
  f32_load<ND>(q, sample + (size_t)qr * rs + (size_t)e * dh, g, dh);
  f32x4_t o[ND];
#pragma unroll
  for (int t = 0; t < ND; ++t) o[t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  float l = 0.f, m = -INFINITY;
  if (last > 0)
    for (int kt = first / kF32Rows + wave; kt * kF32Rows < last; kt += 4) {
      const int key0 = kt * kF32Rows;
      F32Frag<ND> k;
      f32_load<ND>(k, kb + (size_t)min(key0 + c, s - 1) * rs, g, dh);
      f32x4_t p = f32_scores<ND>(k, q);
      uint32_t vis = 0;
      float mx = m;
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int key = key0 + 4 * g + r;
        const bool ok = key >= span.x && key < span.y;
        float unused;
        p[r] = ok ? rule.score(p[r], my_q - key, &unused) : -INFINITY;
        vis |= (uint32_t)ok << r;
        mx = fmaxf(mx, p[r]);
      }
      const LaneHalves mr = lane_rows(mx);
      const LaneHalves mh = lane_halves(fmaxf(mr.lo, mr.hi));
      mx = fmaxf(mh.lo, mh.hi);
      const float ref = mx == -INFINITY ? 0.f : mx;   // no key so far: weights of zero, not exp(-inf + inf)
      const float corr = __expf(m - ref);
      m = mx;
      l *= corr;
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        p[r] = __expf(p[r] - ref);
        l += p[r];
      }
#pragma unroll
      for (int t = 0; t < ND; ++t) o[t] *= corr;
      f32_accumulate<ND>(o, p, vb, rs, key0, s, dh, inner_lo > key0 || inner_hi < key0 + kF32Rows, vis, lane);
    }
  l += __shfl_xor(l, 16, 64);
  l += __shfl_xor(l, 32, 64);
  if (g == 0) {
    stat[0][wave][c] = m;
    stat[1][wave][c] = l;
  }
  __syncthreads();
  float mall = stat[0][0][c], lall = 0.f;
#pragma unroll
  for (int w = 1; w < 4; ++w) mall = fmaxf(mall, stat[0][w][c]);
  const float ref = mall == -INFINITY ? 0.f : mall;
#pragma unroll
  for (int w = 0; w < 4; ++w) lall += stat[1][w][c] * __expf(stat[0][w][c] - ref);
  f32_scale<ND>(o, __expf(m - ref));   // a wave without a key: m = -inf, its zeros are multiplied by zero
  f32_join<ND>(o, part, wave, lane);
  if (wave > 0 || my_q >= s) return;
  const bool empty = span.y <= span.x;
#pragma unroll
  for (int t = 0; t < ND; ++t) o[t] = empty ? f32x4_t{0.f, 0.f, 0.f, 0.f} : o[t] / lall;
  f32_store<ND>(ctx + ((size_t)my_q * b + j) * z.heads * dh + (size_t)e * dh, o, g, dh);
  if (g == 0) lse[((size_t)j * z.heads + e) * s + my_q] = empty ? -INFINITY : mall + __logf(lall);
}

template <int ND>
__global__ void __launch_bounds__(256)
attn_span_dq_f32(const float* __restrict__ qkv, const float* __restrict__ ctx, const float* __restrict__ dctx, const float* __restrict__ lse,
                 float* __restrict__ delta, float* __restrict__ dqkv, SpanView view, SpanShape z, int dh) {
  __shared__ f32x4_t part[3 * ND * 64];
  const int e = blockIdx.y, j = blockIdx.z, wave = threadIdx.x >> 6, lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
  const int s = z.s, b = z.b, q0 = ((int)gridDim.x - 1 - (int)blockIdx.x) * kF32Rows, my_q = q0 + c, qr = min(my_q, s - 1);
  const int kve = e / (z.heads / z.kv_heads);
  const size_t row = (size_t)(z.heads + 2 * z.kv_heads) * dh, rs = b * row;
  const float* sample = qkv + j * row;
  const float *kb = sample + (size_t)(z.heads + kve) * dh, *vb = kb + (size_t)z.kv_heads * dh;
  const int2 span = my_q < s ? span_of(view, j, my_q, s) : make_int2(kNoKey, 0);
  const int first = row_min(span.x), last = row_max(span.y), inner_lo = row_max(my_q < s ? span.x : 0), inner_hi = row_min(my_q < s ? span.y : kNoKey);
  const F32Rule rule(z, e);
  const size_t stat = ((size_t)j * z.heads + e) * s + qr, out = ((size_t)qr * b + j) * z.heads * dh + (size_t)e * dh;
  F32Frag<ND> q, dc;
  f32_load<ND>(q, sample + (size_t)qr * rs + (size_t)e * dh, g, dh);
  f32_load<ND>(dc, dctx + out, g, dh);
  float D;
  {
    F32Frag<ND> o;
    f32_load<ND>(o, ctx + out, g, dh);
    D = f32_delta_column<ND>(o, dc, c);
  }
  if (wave == 0 && g == 0 && my_q < s) delta[stat] = D;
  const float L = lse[stat];
  f32x4_t acc[ND];
#pragma unroll
  for (int t = 0; t < ND; ++t) acc[t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  if (last > 0)
    for (int kt = first / kF32Rows + wave; kt * kF32Rows < last; kt += 4) {
      const int key0 = kt * kF32Rows;
      const size_t at = (size_t)min(key0 + c, s - 1) * rs;
      F32Frag<ND> k, v;
      f32_load<ND>(k, kb + at, g, dh);
      f32_load<ND>(v, vb + at, g, dh);
      const f32x4_t sc = f32_scores<ND>(k, q), dp = f32_scores<ND>(v, dc);
      f32x4_t ds;
      uint32_t vis = 0;
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int key = key0 + 4 * g + r;
        const bool ok = key >= span.x && key < span.y;
        float d;
        const float t = rule.score(sc[r], my_q - key, &d);
        ds[r] = ok ? __expf(t - L) * (dp[r] - D) * d * rule.scale : 0.f;
        vis |= (uint32_t)ok << r;
      }
      f32_accumulate<ND>(acc, ds, kb, rs, key0, s, dh, inner_lo > key0 || inner_hi < key0 + kF32Rows, vis, lane);
    }
  f32_join<ND>(acc, part, wave, lane);
  if (wave > 0 || my_q >= s) return;
  f32_store<ND>(dqkv + (size_t)my_q * rs + j * row + (size_t)e * dh, acc, g, dh);
}

template <int ND>
__global__ void __launch_bounds__(256)
attn_span_dkv_f32(const float* __restrict__ qkv, const float* __restrict__ dctx, const float* __restrict__ lse, const float* __restrict__ delta,
                  float* __restrict__ dqkv, SpanView view, SpanShape z, int dh, int parts, float* __restrict__ partial) {
  __shared__ f32x4_t part[3 * ND * 64];
  const int kve = blockIdx.y, j = blockIdx.z, wave = threadIdx.x >> 6, lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
  const int mine_of = blockIdx.x % parts, s = z.s, b = z.b, k0 = blockIdx.x / parts * kF32Rows, my_key = k0 + c, kr = min(my_key, s - 1), group = z.heads / z.kv_heads;
  const size_t row = (size_t)(z.heads + 2 * z.kv_heads) * dh, rs = b * row, orow = (size_t)z.heads * dh, dors = b * orow;
  const float* sample = qkv + j * row;
  const float *kb = sample + (size_t)(z.heads + kve) * dh, *vb = kb + (size_t)z.kv_heads * dh;
  F32Frag<ND> k, v;
  f32_load<ND>(k, kb + (size_t)kr * rs, g, dh);
  f32_load<ND>(v, vb + (size_t)kr * rs, g, dh);
  // the tiles of queries that may see a key of the block
  int qt_first = k0 / kF32Rows, qt_end = (s + kF32Rows - 1) / kF32Rows;
  if (view.range) {
    const int nt = (s + kSpanRows - 1) / kSpanRows;
    int a = kNoKey, z1 = -1;
    for (int t = lane; t < nt; t += 64) {
      const SpanBounds y = view.bounds[(size_t)j * nt + t];
      if (y.first < k0 + kF32Rows && y.last > k0) {
        a = min(a, t);
        z1 = max(z1, t);
      }
    }
#pragma unroll
    for (int d = 16; d < 64; d *= 2) {
      a = min(a, __shfl_xor(a, d, 64));
      z1 = max(z1, __shfl_xor(z1, d, 64));
    }
    a = row_min(a);
    z1 = row_max(z1);
    qt_first = z1 < 0 ? 0 : 2 * a;
    qt_end = z1 < 0 ? 0 : min(qt_end, 2 * z1 + 2);
  }
  const int nq = qt_end - qt_first;
  f32x4_t dk[ND], dv[ND];
#pragma unroll
  for (int t = 0; t < ND; ++t) dk[t] = dv[t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
  for (int at = wave + 4 * mine_of; at < group * nq; at += 4 * parts) {
    const int head = kve * group + at / nq, q0 = (qt_first + at % nq) * kF32Rows, qc = min(q0 + c, s - 1);
    const F32Rule rule(z, head);
    const float *qb = sample + (size_t)head * dh, *dob = dctx + j * orow + (size_t)head * dh;
    const size_t stats = ((size_t)j * z.heads + head) * s;
    f32x4_t sc, dp, p, ds;
    {
      F32Frag<ND> q, dc;
      f32_load<ND>(q, qb + (size_t)qc * rs, g, dh);
      f32_load<ND>(dc, dob + (size_t)qc * dors, g, dh);
      sc = f32_scores<ND>(q, k);
      dp = f32_scores<ND>(dc, v);
    }
    uint32_t vis = 0;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int q = q0 + 4 * g + r, qq = min(q, s - 1);
      const int2 x = span_of(view, j, qq, s);
      const bool ok = q < s && my_key >= x.x && my_key < x.y;
      float d;
      const float t = rule.score(sc[r], q - my_key, &d);
      p[r] = ok ? __expf(t - lse[stats + qq]) : 0.f;
      ds[r] = ok ? p[r] * (dp[r] - delta[stats + qq]) * d * rule.scale : 0.f;
      vis |= (uint32_t)ok << r;
    }
    const bool some = !__all(vis == 15u);
    f32_accumulate<ND>(dv, p, dob, dors, q0, s, dh, some, vis, lane);
    f32_accumulate<ND>(dk, ds, qb, rs, q0, s, dh, some, vis, lane);
  }
  // (a part's sums: [s, b, 2 kv_heads dh])
  float* out = parts > 1 ? partial + (((size_t)mine_of * s + my_key) * b + j) * 2 * z.kv_heads * dh + (size_t)kve * dh
                         : dqkv + (size_t)my_key * rs + j * row + (size_t)(z.heads + kve) * dh;
  const bool mine = f32_join<ND>(dk, part, wave, lane);
  if (mine && my_key < s) f32_store<ND>(out, dk, g, dh);
  if (f32_join<ND>(dv, part, wave, lane) && my_key < s) f32_store<ND>(out + (size_t)z.kv_heads * dh, dv, g, dh);
}

// Adds the parts' sums in their order, four elements to a thread.
__global__ void __launch_bounds__(256) attn_span_dkv_join_f32(const float* __restrict__ partial, float* __restrict__ dqkv, SpanShape z, int dh, int parts) {
  const size_t width = 2 * (size_t)z.kv_heads * dh, n = (size_t)z.s * z.b * width, i = ((size_t)blockIdx.x * 256 + threadIdx.x) * 4;
  if (i >= n) return;
  f32x4_t sum = *reinterpret_cast<const f32x4_t*>(partial + i);
  for (int p = 1; p < parts; ++p) sum += *reinterpret_cast<const f32x4_t*>(partial + p * n + i);
  const size_t r = i / width;
  *reinterpret_cast<f32x4_t*>(dqkv + r * (width + (size_t)z.heads * dh) + (size_t)z.heads * dh + (i - r * width)) = sum;
}

// ------------------------------------------------------------------------------------------------
// host launchers
// ------------------------------------------------------------------------------------------------
bool attn_span_fits(const ptdp_attn_span_cfg* c) {
  const uint64_t pairs = (uint64_t)c->heads * c->b, pitch = (uint64_t)(c->heads + 2ull * c->kv_heads) * c->dh * c->b;
  if (c->dtype == PTDP_F32) return c->heads <= 65535 && c->b <= 65535 && pitch < (1ull << 31);
  return pairs < (1ull << 31) && attn_slice_fits(pitch, c->dh) && attn_grid_levels((c->s + 63) / 64, c->heads, c->b) < (1ll << 32) / 512;
}
static SpanShape span_shape(const ptdp_attn_span_cfg* c, const float* slopes) {
  const bool capped = c->cap > 0.f;
  const float mul = (capped ? c->cap : c->scale) * kLog2e;
  return {c->s, c->b, c->heads, c->kv_heads, c->scale, c->cap, mul, capped ? 2.f * kLog2e * c->scale / c->cap : 0.f,
          capped ? c->scale / c->cap : 0.f, kLog2e / mul, slopes};
}
static long long span_blocks(int s, int heads, int b) { return (long long)((s + 63) / 64) * heads * b; }   // of 64 rows
// Workgroups that share the walk of a key block whose head serves a group of query heads: as many as there are compute units for
// (the walk is up to `tiles` tiles of 64 queries long), and up to eight times as many while each is left kSpanShare tiles - fewer are not worth
// the sums' way through memory.  The workspace holds those sums, so this asks for the chip's units and not for the device's.  dK and dV alone,
// us, 1 part and the parts taken: 2048 tokens, heads 16 to 2 of 128: 307, 71 (8); 32 to 8 of 64: 115, 58 (4); 1024, 20 to 4 of 160: 120, 45 (4);
// 256 x 8, 16 to 2 of 64: 34, 20 (4; 24 with 8); 512 x 8, 16 to 4 of 128: 50 (1; 53 with 2).
constexpr int kSpanUnits = 256, kSpanShare = 32;
static int span_parts(int s, int heads, int kv_heads, int b) {
  const int group = heads / kv_heads;
  const long long blocks = std::max(1ll, span_blocks(s, kv_heads, b)), tiles = (long long)group * ((s + 63) / 64);
  const long long few = kSpanUnits / blocks, many = std::min(8 * kSpanUnits / blocks, tiles / kSpanShare);
  return (int)std::max(1ll, std::min((long long)group, std::max(few, many)));
}
// The same for fp32, whose workgroups of 16 keys take a compute unit or half of one (3 x 187 tokens, 16 heads to 4 of 160, forward and backward: 300 us
// in one part, 240 in three).
constexpr int kSpanUnitsF32 = 2 * kSpanUnits, kSpanShareF32 = 2;   // tiles of 16 queries left to each of four waves
static int span_parts_f32(int s, int heads, int kv_heads, int b) {
  const int group = heads / kv_heads;
  const long long n = (s + kF32Rows - 1) / kF32Rows, blocks = std::max(1ll, n * kv_heads * b);
  return (int)std::max(1ll, std::min({(long long)group, kSpanUnitsF32 / blocks, n * group / (4 * kSpanShareF32)}));
}
static size_t span_delta_bytes(int s, int heads, int b) { return ((size_t)b * heads * s * sizeof(float) + 15) / 16 * 16; }
static size_t span_stats_bytes(int s, int heads, int b) { return ((size_t)b * heads * s * sizeof(float2) + 15) / 16 * 16; }
size_t attn_span_workspace_bytes(const ptdp_attn_span_cfg* c) {
  if (c->dtype == PTDP_F32) {   // D, and the parts' sums
    const int parts = span_parts_f32(c->s, c->heads, c->kv_heads, c->b);
    return span_delta_bytes(c->s, c->heads, c->b) + (parts > 1 ? (size_t)parts * c->s * c->b * 2 * c->kv_heads * c->dh * sizeof(float) : 0);
  }
  const int parts = span_parts(c->s, c->heads, c->kv_heads, c->b);
  const size_t sums = parts > 1 ? (size_t)parts * c->b * c->kv_heads * ((c->s + 31) / 32) * 64 * c->dh * sizeof(float) : 0;
  return span_stats_bytes(c->s, c->heads, c->b) + sums;
}
// the square's visible part is not known to the host: counted as the causal half
static double span_flops(const ptdp_attn_span_cfg* c) { return 2.0 * c->b * c->heads * (double)c->s * c->s * c->dh; }

template <int DH, int QW, int NP, int KT>
static int span_fwd_t(const bf16_t* qkv, bf16_t* ctx, float* lse, const SpanView& view, const SpanShape& z, hipStream_t st) {
  constexpr int tiles = NP * 4 * TileDma<DH, QW, KT, false>::kBytes, part = NP > 1 ? QW * (2 + DH / 2) * 64 * (int)sizeof(float) : 0;
  constexpr int smem = tiles > part ? tiles : part;
  static once_flag_t done[kMaxDevices];
  const auto kernel = attn_span_fwd_kernel<DH, QW, NP, KT>;
  if (set_dynamic_smem(reinterpret_cast<const void*>(kernel), smem, done) != PTDP_OK) return PTDP_E_HIP;
  const dim3 grid(attn_grid_levels((z.s + 32 * QW - 1) / (32 * QW), z.heads, z.b));
  hipLaunchKernelGGL(kernel, grid, dim3(64 * QW * NP), smem, st, qkv, ctx, lse, view, z);
  return PTDP_OK;
}
template <int DH, int QW, int NP, int KT>
static int span_dq_t(const bf16_t* qkv, const bf16_t* ctx, const bf16_t* dctx, const float* lse, float2* stats, bf16_t* dqkv, const SpanView& view,
                     const SpanShape& z, hipStream_t st) {
  constexpr int tiles = NP * 4 * TileDma<DH, QW, KT, false>::kBytes, sums = NP > 1 ? QW * (DH / 2) * 64 * (int)sizeof(float) : 0;
  constexpr int smem = tiles > sums ? tiles : sums;
  static once_flag_t done[kMaxDevices];
  const auto kernel = attn_span_dq_kernel<DH, QW, NP, KT>;
  if (set_dynamic_smem(reinterpret_cast<const void*>(kernel), smem, done) != PTDP_OK) return PTDP_E_HIP;
  const dim3 grid(attn_grid_levels((z.s + 32 * QW - 1) / (32 * QW), z.heads, z.b));
  hipLaunchKernelGGL(kernel, grid, dim3(64 * QW * NP), smem, st, qkv, ctx, dctx, lse, stats, dqkv, view, z);
  return PTDP_OK;
}
template <int DH, int KW, int NP, int QT, bool SPLIT, bool SCORED> static int span_dkv_scored_t(const SpanDkvArgs& a, hipStream_t st) {
  using Geom = SpanDkvGeom<DH, KW, NP, QT, SPLIT>;
  static once_flag_t done[kMaxDevices];
  const auto kernel = attn_span_dkv_kernel<DH, KW, NP, QT, SPLIT, SCORED>;
  if (set_dynamic_smem(reinterpret_cast<const void*>(kernel), Geom::kBytes, done) != PTDP_OK) return PTDP_E_HIP;
  const dim3 grid(attn_grid_levels((a.z.s + 32 * KW - 1) / (32 * KW), a.z.kv_heads * a.parts, a.z.b));
  hipLaunchKernelGGL(kernel, grid, dim3(Geom::kThreads * NP), Geom::kBytes, st, a);
  return PTDP_OK;
}
template <int DH, int KW, int NP, int QT, bool SPLIT> static int span_dkv_t(const SpanDkvArgs& a, hipStream_t st) {
  return a.z.capped_or_biased() ? span_dkv_scored_t<DH, KW, NP, QT, SPLIT, true>(a, st) : span_dkv_scored_t<DH, KW, NP, QT, SPLIT, false>(a, st);
}
// Few key blocks: two groups of waves to each, which take its tiles in turn (2048 tokens, 16 heads of 128, 512 blocks: 62 us, 128 keys to a workgroup
// 76).  Many: 128 keys to a workgroup (4 x 2048: 183 and 235), unless rows are short (8 x 512: 64 keys 42, 128 keys 54; 16 x 512, heads of 32: two groups
// 27, 128 keys 34).
template <int DH> static int span_dkv_dh(const SpanDkvArgs& a, hipStream_t st) {
  const long long ncu = attn_compute_units(), blocks = span_blocks(a.z.s, a.z.kv_heads * a.parts, a.z.b);
  if constexpr (DH > 96) {
    if (blocks <= 2 * ncu) return span_dkv_t<DH, 2, 2, 32, true>(a, st);
    if (a.z.s <= 1024) return span_dkv_t<DH, 2, 1, 32, true>(a, st);
    return span_dkv_t<DH, 4, 1, 32, true>(a, st);
  } else {
    if (blocks <= 4 * ncu || a.z.s <= 1024) return span_dkv_t<DH, 2, 2, 32, false>(a, st);
    return span_dkv_t<DH, 4, 1, 64, false>(a, st);
  }
}

// Few blocks of queries: two groups of waves to each.  Forward, us, two groups and one: 2048 tokens, 16 heads of 128 (512 blocks of 64): 38 and 53;
// 20 of 160 (640): 50 and 58; 32 of 64 (1024): 34 and 37; 2 x 1027, 32 of 64 (1088): 27 and 24.  dQ: 47 and 63 (512); 47 and 49 (1024); 8 x 512,
// 16 of 128 (1024): 37 and 36; 2 x 1027 (1088): 35 and 30.
template <int DH> static int span_fwd_dh(const bf16_t* qkv, bf16_t* ctx, float* lse, const SpanView& view, const SpanShape& z, hipStream_t st) {
  if (span_blocks(z.s, z.heads, z.b) <= 4 * attn_compute_units()) return span_fwd_t<DH, 2, 2, (DH > 128 ? 32 : 64)>(qkv, ctx, lse, view, z, st);
  return span_fwd_t<DH, 4, 1, 64>(qkv, ctx, lse, view, z, st);
}
template <int DH>
static int span_bwd_dh(const bf16_t* qkv, const bf16_t* ctx, const bf16_t* dctx, const float* lse, float2* stats, bf16_t* dqkv, const SpanView& view,
                       const SpanShape& z, hipStream_t st) {
  const long long ncu = attn_compute_units();
  int rc = span_blocks(z.s, z.heads, z.b) <= 3 * ncu ? span_dq_t<DH, 2, 2, 32>(qkv, ctx, dctx, lse, stats, dqkv, view, z, st)
                                                          : span_dq_t<DH, 4, 1, 64>(qkv, ctx, dctx, lse, stats, dqkv, view, z, st);
  if (rc != PTDP_OK) return rc;
  SpanDkvArgs a = {qkv, dctx, stats, dqkv, view, z, span_parts(z.s, z.heads, z.kv_heads, z.b), nullptr};
  a.partial = reinterpret_cast<float*>(reinterpret_cast<char*>(stats) + span_stats_bytes(z.s, z.heads, z.b));
  rc = span_dkv_dh<DH>(a, st);
  if (rc != PTDP_OK || a.parts == 1) return rc;
  hipLaunchKernelGGL(attn_span_dkv_join_kernel<DH>, dim3((z.s + 31) / 32 * z.kv_heads * z.b, 2), dim3(DH * 2), 0, st, a);
  return PTDP_OK;
}

// steps of 16 dh, rounded up to one of the built forms
#define PTDP_SPAN_F32(dh, CALL)     \
  do {                              \
    if ((dh) <= 32) CALL(2);        \
    else if ((dh) <= 64) CALL(4);   \
    else if ((dh) <= 96) CALL(6);   \
    else if ((dh) <= 128) CALL(8);  \
    else if ((dh) <= 160) CALL(10); \
    else CALL(16);                  \
  } while (0)

int launch_attn_span_fwd(const ptdp_attn_span_cfg* c, const void* qkv, const void* spans, const float* slopes, void* ctx, float* lse, hipStream_t st) {
  const SpanView view = span_view(spans, c->s, c->b);
  const SpanShape z = span_shape(c, slopes);
  Launch L(PTDP_K_ATTN_FWD, span_flops(c), st);
  int rc = PTDP_OK;
  if (c->dtype == PTDP_F32) {
    const dim3 grid((c->s + kF32Rows - 1) / kF32Rows, c->heads, c->b);
#define PTDP_CALL(ND) hipLaunchKernelGGL(attn_span_fwd_f32<ND>, grid, dim3(256), 0, st, (const float*)qkv, (float*)ctx, lse, view, z, c->dh)
    PTDP_SPAN_F32(c->dh, PTDP_CALL);
#undef PTDP_CALL
  } else {
#define PTDP_CALL(D) rc = span_fwd_dh<D>((const bf16_t*)qkv, (bf16_t*)ctx, lse, view, z, st)
    if (c->dh == 32) PTDP_CALL(32);
    else if (c->dh == 64) PTDP_CALL(64);
    else if (c->dh == 96) PTDP_CALL(96);
    else if (c->dh == 128) PTDP_CALL(128);
    else PTDP_CALL(160);
#undef PTDP_CALL
  }
  return rc != PTDP_OK ? rc : L.status();
}

int launch_attn_span_bwd(const ptdp_attn_span_cfg* c, const void* qkv, const void* spans, const float* slopes, const void* ctx, const float* lse,
                         const void* dctx, void* dqkv, void* workspace, hipStream_t st) {
  const SpanView view = span_view(spans, c->s, c->b);
  const SpanShape z = span_shape(c, slopes);
  Launch L(PTDP_K_ATTN_BWD, 2.0 * span_flops(c), st);
  int rc = PTDP_OK;
  if (c->dtype == PTDP_F32) {
    const int n = (c->s + kF32Rows - 1) / kF32Rows;
    const float *q = (const float*)qkv, *d = (const float*)dctx;
    float *delta = (float*)workspace, *partial = (float*)((char*)workspace + span_delta_bytes(c->s, c->heads, c->b));
    const int parts = span_parts_f32(c->s, c->heads, c->kv_heads, c->b);
#define PTDP_CALL(ND)                                                                                                                                  \
  do {                                                                                                                                                 \
    hipLaunchKernelGGL(attn_span_dq_f32<ND>, dim3(n, c->heads, c->b), dim3(256), 0, st, q, (const float*)ctx, d, lse, delta, (float*)dqkv, view, z, c->dh); \
    hipLaunchKernelGGL(attn_span_dkv_f32<ND>, dim3(n * parts, c->kv_heads, c->b), dim3(256), 0, st, q, d, lse, (const float*)delta, (float*)dqkv, view, z,  \
                       c->dh, parts, partial);                                                                                                         \
  } while (0)
    PTDP_SPAN_F32(c->dh, PTDP_CALL);
#undef PTDP_CALL
    if (parts > 1)
      hipLaunchKernelGGL(attn_span_dkv_join_f32, dim3((unsigned)(((size_t)c->s * c->b * c->kv_heads * c->dh / 2 + 255) / 256)), dim3(256), 0, st, partial,
                         (float*)dqkv, z, c->dh, parts);
  } else {
#define PTDP_CALL(D) rc = span_bwd_dh<D>((const bf16_t*)qkv, (const bf16_t*)ctx, (const bf16_t*)dctx, lse, (float2*)workspace, (bf16_t*)dqkv, view, z, st)
    if (c->dh == 32) PTDP_CALL(32);
    else if (c->dh == 64) PTDP_CALL(64);
    else if (c->dh == 96) PTDP_CALL(96);
    else if (c->dh == 128) PTDP_CALL(128);
    else PTDP_CALL(160);
#undef PTDP_CALL
  }
  return rc != PTDP_OK ? rc : L.status();
}

}  // namespace ptdp
