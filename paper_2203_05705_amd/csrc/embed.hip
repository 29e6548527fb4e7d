// Embedding: Y[r] = s E[id_r], and its gradient dE[v] = beta dE[v] + s (sum of dY[r] over the r with id_r = v), added in ascending r.
//
// Both passes are bound by bytes.  The gradient first sorts the tokens, stably, so that every row of dE is one sum in a fixed
// order: no atomics on floats, the same bits on every call.
//
// Sorting, one launch: workgroup w owns the ids [w span, (w + 1) span).  All of its wavefronts read their own stretch of the R
// tokens (4 bytes each, from the L2 for all but the first workgroup) and count those it owns by (id, wavefront) in LDS; a
// prefix sum over these counts, ids first, gives every wavefront a place for each id, and a second reading puts the tokens'
// positions there.  R tokens are read 2 x workgroups times, but at 4 bytes against the 2 KB of a position's gradient.
//
// Summing: a row's team of lanes walks its tokens, kInFlight at a time.  Frequent tokens would leave one team behind: a row of more than
// kLong tokens is summed in pieces of kPiece sorted positions each by a launch before, and its team adds the pieces up.
//
// Measured, passes in a row with the forward pass: 8192 tokens, bf16 rows of 1024, an fp32 table of 32768 69 us (launches of 7 + 7 + 15 + 40 us, 2.7 TB/s); 131072 tokens, a table of
// 50000 added to 371 us (96 + 51 + 74 + 152).  Pieces of 128 and two loads of ids ahead took 179 and 489 us in the gradient's launches, these 62 and 277.
// One generation step, 64 tokens: 2.6 us.
#include "rows.hpp"

namespace ard {

constexpr int kSortWaves = 16;     // wavefronts of a sorting workgroup
// workgroups that a table is shared out to, one a compute unit (131072 tokens, 50000 rows of 1024: the gradient's launches 241 us; 64 shares 257, 128 247, 512 254, 1024 286)
constexpr int kShares = 256;
constexpr int kMaxSpan = 1024;     // ids that one may own: counts of span x wavefronts in LDS, 64 KB
constexpr int kPiece = 32;         // sorted positions whose sum is a piece of a long row
constexpr int kLong = 32;          // tokens beyond which a row is summed in pieces (no fewer than kPiece: a piece meets two long rows at most)
constexpr int kAhead = 8;          // loads of ids asked for together
constexpr int kInFlight = 8;       // rows of dY asked for together
constexpr int kMaxGrid = 1 << 20;

// The lanes of a row: `team` of them (a power of two up to a workgroup's 256), 8 neighbouring elements each.
struct Team {
  int lanes, shift;
};
static Team team_of(int D) {
  Team t{1, 0};
  while (t.lanes < 256 && t.lanes * 8 < D) t.lanes *= 2, ++t.shift;
  return t;
}

template <typename T, typename W>
__global__ __launch_bounds__(256) void embed_fwd_kernel(int R, int V, int D, const int32_t* ids, const W* E, int64_t lde, float scale, T* Y, int64_t ldy, int shift) {
  const int team = threadIdx.x >> shift, lane = threadIdx.x - (team << shift), teams = 256 >> shift;
  const int64_t step = (int64_t)gridDim.x * teams;
  for (int64_t r = (int64_t)blockIdx.x * teams + team; r < R; r += step) {
    const int id = ids[r];
    const bool there = id >= 0 && id < V;
    for (int c = lane * 8; c < D; c += 8 << shift) {
      float x[8] = {};
      if (there) load_some<8>(E + id * lde + c, D - c, x);
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = there ? x[j] * scale : 0.0f;
      store_some<8>(Y + r * ldy + c, D - c, x);
    }
  }
}

// sorted[]: the positions r of tokens inside the table, by id and then by r; start[v]: where those of v begin, start[V] their number.
__global__ __launch_bounds__(64 * kSortWaves) void embed_sort_kernel(int R, int V, int span, const int32_t* ids, int32_t* start, int32_t* sorted) {
  __shared__ int32_t at[kMaxSpan * kSortWaves];  // counts, then places, by [id][wavefront]
  __shared__ int32_t sums[kSortWaves], below[kSortWaves];
  const int w = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int lo = blockIdx.x * span, n = imin(V - lo, span);
  for (int i = threadIdx.x; i < n * kSortWaves; i += 64 * kSortWaves) at[i] = 0;
  __syncthreads();
  const int per = ((R + kSortWaves - 1) / kSortWaves + 63) & ~63, r0 = (int)((int64_t)w * per < R ? w * per : R), r1 = R - r0 < per ? R : r0 + per;
  int before = 0;  // tokens of smaller ids
  for (int r = r0; r < r1; r += 64 * kAhead) {
    int id[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) id[k] = r + k * 64 + lane < r1 ? ids[r + k * 64 + lane] : -1;
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      if (id[k] >= lo && id[k] < lo + n) atomicAdd(&at[(id[k] - lo) * kSortWaves + w], 1);
      before += id[k] >= 0 && id[k] < lo;
    }
  }
  __syncthreads();
  // exclusive prefix sums over [id][wavefront], a run of counts a thread
  const int runs = (n * kSortWaves + 64 * kSortWaves - 1) / (64 * kSortWaves), i0 = threadIdx.x * runs, i1 = imin(i0 + runs, n * kSortWaves);
  int mine = 0;
  for (int i = i0; i < i1; ++i) mine += at[i];
  int upto = mine;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const int o = __shfl_up(upto, d);
    if (lane >= d) upto += o;
    before += __shfl_xor(before, d);
  }
  if (lane == 63) sums[w] = upto;
  if (lane == 0) below[w] = before;
  __syncthreads();
  int base = upto - mine;
  for (int k = 0; k < kSortWaves; ++k) base += below[k] + (k < w ? sums[k] : 0);
  for (int i = i0; i < i1; ++i) {
    const int c = at[i];
    at[i] = base;
    if (i % kSortWaves == 0) start[lo + i / kSortWaves] = base;
    base += c;
  }
  if (lo + n == V && i0 < i1 && i1 == n * kSortWaves) start[V] = base;
  __syncthreads();
  for (int r = r0; r < r1; r += 64 * kAhead) {
    int ahead[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) ahead[k] = r + k * 64 + lane < r1 ? ids[r + k * 64 + lane] : -1;
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const int id = ahead[k];
      unsigned long long left = __ballot(id >= lo && id < lo + n);
      while (left) {  // one id at a time: its lanes take places in their order
        const int key = __builtin_amdgcn_readlane(id, __ffsll(left) - 1);
        const unsigned long long same = __ballot(id == key) & left;
        const int cell = (key - lo) * kSortWaves + w, place = at[cell];
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // every lane has read the place before one moves it, and before the next id's is read
        if (id == key) {
          const int rank = __popcll(same & ((1ull << lane) - 1));
          sorted[place + rank] = r + k * 64 + lane;
          if (rank == 0) at[cell] = place + __popcll(same);
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        left &= ~same;
      }
    }
  }
}

// sum of the rows of sorted positions [a, b) at column c, in their order
template <typename T> __device__ __forceinline__ void add_rows(const int32_t* sorted, int a, int b, const T* dY, int64_t ld, int c, int n, float (&sum)[8]) {
  for (int i = a; i < b; i += kInFlight) {
    float x[kInFlight][8];
#pragma unroll
    for (int j = 0; j < kInFlight; ++j)
      if (i + j < b) load_some<8>(dY + sorted[i + j] * ld + c, n, x[j]);
#pragma unroll
    for (int j = 0; j < kInFlight; ++j)
      if (i + j < b) {
#pragma unroll
        for (int e = 0; e < 8; ++e) sum[e] += x[j][e];
      }
  }
}

// pieces[p][0 / 1][D]: what the first / last id of sorted positions [p kPiece, (p + 1) kPiece) has there, if it is a long row's (the
// first where both are the same).
template <typename T>
__global__ __launch_bounds__(256) void embed_pieces_kernel(int V, int D, const int32_t* ids, const int32_t* start, const int32_t* sorted, const T* dY, int64_t lddy,
                                                           float* pieces) {
  const int all = start[V], count = (all + kPiece - 1) / kPiece;
  for (int p = blockIdx.x; p < count; p += gridDim.x) {
    const int a = p * kPiece, b = imin(a + kPiece, all), first = ids[sorted[a]], last = ids[sorted[b - 1]];
#pragma unroll
    for (int side = 0; side < 2; ++side) {
      const int id = side ? last : first;
      if (side && last == first) break;
      const int s = start[id], e = start[id + 1];
      if (e - s <= kLong) continue;
      for (int c = threadIdx.x * 8; c < D; c += 256 * 8) {
        float sum[8] = {};
        add_rows(sorted, imax(a, s), imin(b, e), dY, lddy, c, D - c, sum);
        store_some<8>(pieces + ((int64_t)p * 2 + side) * D + c, D - c, sum);
      }
    }
  }
}

template <typename T, typename W, bool ADD>
__global__ __launch_bounds__(256) void embed_bwd_kernel(int V, int D, const int32_t* start, const int32_t* sorted, const T* dY, int64_t lddy, float scale,
                                                        const float* pieces, W* dE, int64_t lde, int shift) {
  const int team = threadIdx.x >> shift, lane = threadIdx.x - (team << shift), teams = 256 >> shift;
  for (int v = blockIdx.x * teams + team; v < V; v += gridDim.x * teams) {
    const int s = start[v], e = start[v + 1];
    if (ADD && s == e) continue;
    for (int c = lane * 8; c < D; c += 8 << shift) {
      float sum[8] = {}, old[8] = {};
      if (ADD) load_some<8>(dE + v * lde + c, D - c, old);
      if (e - s <= kLong) {
        add_rows(sorted, s, e, dY, lddy, c, D - c, sum);
      } else {
        const int p1 = (e - 1) / kPiece;
        for (int p = s / kPiece; p <= p1; p += kInFlight) {
          float x[kInFlight][8];
#pragma unroll
          for (int j = 0; j < kInFlight; ++j)
            if (p + j <= p1) load_some<8>(pieces + ((int64_t)(p + j) * 2 + ((p + j) * kPiece < s)) * D + c, D - c, x[j]);
#pragma unroll
          for (int j = 0; j < kInFlight; ++j)
            if (p + j <= p1) {
#pragma unroll
              for (int k = 0; k < 8; ++k) sum[k] += x[j][k];
            }
        }
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) sum[j] = ADD ? fmaf(scale, sum[j], old[j]) : s == e ? 0.0f : scale * sum[j];  // (+0.0 without a token, whatever the scale)
      // (32768 x 1024, 8192 tokens, passes in a row 69 us, with stores that stay in the caches 107; with the AdamW step that reads the gradient behind it, passes of the gradient
      // and the step: 50000 rows of 1024 349 and 353, 32768 237 and 239, 8192 61 and 59, 4096 of 512 22.4 and 24.2)
      if (!ADD && D - c >= 8) store_run_past(dE + v * lde + c, sum);
      else store_some<8>(dE + v * lde + c, D - c, sum);
    }
  }
}

// ---- host ---------------------------------------------------------------------
struct EmbedSpace {  // the workspace of the gradient
  size_t start, sorted, pieces, bytes;
};
static EmbedSpace embed_space(int R, int V, int D) {
  EmbedSpace s{};
  s.sorted = align_up((size_t)(V + 1) * 4, 256);
  s.pieces = align_up(s.sorted + (size_t)R * 4, 256);
  s.bytes = s.pieces + (R > kLong ? (size_t)((R + (int64_t)kPiece - 1) / kPiece) * 2 * D * sizeof(float) : 0);
  return s;
}

static int32_t embed_check(int32_t dtype, int32_t wdtype, int32_t R, int32_t V, int32_t D, int64_t lda, int64_t lde, const char* what) {
  if (dtype != ARD_F32 && dtype != ARD_BF16) return fail(ARD_EDTYPE, "unknown dtype %d", dtype);
  if (wdtype != ARD_F32 && wdtype != dtype) return fail(ARD_EDTYPE, "the table's dtype is fp32 or that of the rows (got %d)", wdtype);
  if (R <= 0 || V <= 0 || D <= 0) return fail(ARD_ESHAPE, "R, V and D must be positive (got %d, %d, %d)", R, V, D);
  if (R > 1 << 30 || V > 1 << 28 || D > 1 << 24) return fail(ARD_ESHAPE, "R = %d, V = %d or D = %d is too large", R, V, D);
  if (lda < D || lde < D) return fail(ARD_ESHAPE, "leading dimensions of %s and the table must be at least D", what);
  return ARD_OK;
}

template <class F> static int32_t embed_instance(int32_t dtype, int32_t wdtype, F&& with) {
  if (dtype == ARD_F32) return with(0.0f, 0.0f);
  return wdtype == ARD_F32 ? with((uint16_t)0, 0.0f) : with((uint16_t)0, (uint16_t)0);
}

}  // namespace ard

using namespace ard;

extern "C" size_t ard_embed_workspace_bytes(int32_t R, int32_t V, int32_t D) {
  if (R <= 0 || V <= 0 || D <= 0 || R > 1 << 30 || V > 1 << 28 || D > 1 << 24) return 0;
  return embed_space(R, V, D).bytes;
}

extern "C" int32_t ard_embed_fwd(int32_t dtype, int32_t wdtype, int32_t R, int32_t V, int32_t D, const int32_t* d_ids, const void* E, int64_t lde,
                                 float scale, void* Y, int64_t ldy, void* stream) {
  if (int32_t st = embed_check(dtype, wdtype, R, V, D, ldy, lde, "Y")) return st;
  if (!d_ids || !E || !Y) return fail(ARD_EINVAL, "null tensor pointer");
  const size_t es = dtype == ARD_F32 ? 4 : 2, ws = wdtype == ARD_F32 ? 4 : 2;
  if (misaligned(d_ids, 4) || misaligned(E, ws) || misaligned(Y, es)) return fail(ARD_EINVAL, "a tensor does not start at a whole element");
  const Team t = team_of(D);
  const int64_t groups = ((int64_t)R * t.lanes + 255) / 256;
  const dim3 grid((unsigned)(groups < kMaxGrid ? groups : kMaxGrid));
  hipStream_t st = (hipStream_t)stream;
  return embed_instance(dtype, wdtype, [&](auto a, auto b) {
    using T = decltype(a);
    using W = decltype(b);
    ARD_LAUNCH_NAMED("embed_fwd_kernel", (embed_fwd_kernel<T, W>), grid, dim3(256), 0, st, R, V, D, d_ids, (const W*)E, lde, scale, (T*)Y, ldy, t.shift);
    ARD_LAUNCH_CHECK("embed_fwd_kernel");
    return (int32_t)ARD_OK;
  });
}

extern "C" int32_t ard_embed_bwd(int32_t dtype, int32_t wdtype, int32_t R, int32_t V, int32_t D, const int32_t* d_ids, const void* dY, int64_t lddy,
                                 float scale, float beta, void* dE, int64_t lddE, void* ws, size_t ws_bytes, void* stream) {
  if (int32_t st = embed_check(dtype, wdtype, R, V, D, lddy, lddE, "dY")) return st;
  if (!d_ids || !dY || !dE) return fail(ARD_EINVAL, "null tensor pointer");
  if (beta != 0.0f && beta != 1.0f) return fail(ARD_EINVAL, "beta is 0 or 1 (got %g)", beta);
  const size_t es = dtype == ARD_F32 ? 4 : 2, wsz = wdtype == ARD_F32 ? 4 : 2;
  if (misaligned(d_ids, 4) || misaligned(dY, es) || misaligned(dE, wsz)) return fail(ARD_EINVAL, "a tensor does not start at a whole element");
  const EmbedSpace sp = embed_space(R, V, D);
  if (!ws || ws_bytes < sp.bytes || misaligned(ws, 4)) return fail(ARD_EWORKSPACE, "workspace too small: need %zu bytes, got %zu", sp.bytes, ws ? ws_bytes : 0);
  int32_t *start = (int32_t*)((char*)ws + sp.start), *sorted = (int32_t*)((char*)ws + sp.sorted);
  float* pieces = (float*)((char*)ws + sp.pieces);
  hipStream_t st = (hipStream_t)stream;
  const int span = imin(kMaxSpan, imax(1, ceil_div(V, kShares)));
  ARD_LAUNCH(embed_sort_kernel, dim3(ceil_div(V, span)), dim3(64 * kSortWaves), 0, st, R, V, span, d_ids, start, sorted);
  ARD_LAUNCH_CHECK("embed_sort_kernel");
  const Team t = team_of(D);
  const int64_t groups = ((int64_t)V * t.lanes + 255) / 256;
  const dim3 grid((unsigned)(groups < kMaxGrid ? groups : kMaxGrid));
  return embed_instance(dtype, wdtype, [&](auto a, auto b) {
    using T = decltype(a);
    using W = decltype(b);
    if (R > kLong) {
      const int blocks = imin(ceil_div(R, kPiece), kMaxGrid);
      ARD_LAUNCH_NAMED(launch_instance("embed_pieces_kernel", blocks, kPiece, 256), (embed_pieces_kernel<T>), dim3(blocks), dim3(256), 0, st, V, D, d_ids, start, sorted, (const T*)dY, lddy, pieces);
      ARD_LAUNCH_CHECK("embed_pieces_kernel");
    }
    if (beta == 0.0f)
      ARD_LAUNCH_NAMED("embed_bwd_kernel", (embed_bwd_kernel<T, W, false>), grid, dim3(256), 0, st, V, D, start, sorted, (const T*)dY, lddy, scale, pieces, (W*)dE, lddE, t.shift);
    else
      ARD_LAUNCH_NAMED("embed_bwd_kernel", (embed_bwd_kernel<T, W, true>), grid, dim3(256), 0, st, V, D, start, sorted, (const T*)dY, lddy, scale, pieces, (W*)dE, lddE, t.shift);
    ARD_LAUNCH_CHECK("embed_bwd_kernel");
    return (int32_t)ARD_OK;
  });
}
