// Per-expert counts, the balance loss of the gate and its gradients.
//
// A batch is cut into segments (sequences, or one segment of all tokens) of n_s
// tokens that count.  With c_si the entries of topk_idx that name expert i in
// segment s, A the number of allowed experts, S' the number of segments that hold
// a token, and g the gate's probabilities (Eq. 7, the softmaxes over allowed
// experts and kept groups):
//
//   f_si = c_si / (k n_s),   P_si = (1 / n_s) sum_t g_i(t)
//   L    = coef / S' sum_s A sum_i f_si P_si
//
// which is coef when the experts are used evenly.  The counts are constants of
// the gradient, so with w_si = coef A f_si / (S' n_s), a group's mean wbar_j =
// sum_{i in j} p_local_i w_i and mean = sum_j p_group_j wbar_j,
//
//   dL/dz_i = g_i (w_i - wbar_j),   dL/dm_j = p_group_j (wbar_j - mean)
//
// for the local logits z and the global logits m.  A softmax's gradient does not
// change when a constant is taken from all w, so the integer counts are used less
// their integer mean: exact, and the differences keep their bits.
//
// Where the groups' sizes and number allow it a token is held by L lanes of a warp,
// a chunk of one group's logits in each lane's registers, so nothing but the
// columns' sums passes through shared memory; else a token is a thread's, its row
// of logits in shared memory.  Short batches (is_small) are done by one
// cluster of CTAs in one launch (its CTAs add their histograms and
// their partial sums through distributed shared memory).  Longer ones take four: balance_clear; balance_count, integer histograms
// (atomics on integers, whose order does not matter) and S'; balance_main or
// balance_lanes, each CTA a contiguous range of tokens, one pass over the logits for the
// loss and both gradients; balance_final, the CTAs' partial sums in order.  Bounded by HBM for
// long batches (the logits are read once, their gradients written once), by the
// launches for short ones.  Measured: 1021 tokens of 16 experts 8.2 us; 262144 of 64
// in 64 segments, 158 MB, 45 us, of which main 31 (floor 23).
#include <algorithm>

#include <cuda_runtime.h>

#include "common.cuh"
#include "internal.h"

namespace ec2moe {

// nonzero: an expert id or a segment bound out of range was skipped
__device__ unsigned int g_balance_error;

namespace {

constexpr int TILE = 128;       // tokens per tile
constexpr int NT = 160;         // threads: a token each for TILE of them, 144 columns of logits for the moves
constexpr int COUNT_TOKENS = 256;   // tokens per CTA of balance_count
constexpr int COUNT_WARPS = 8;
constexpr int CL = 8;           // CTAs of the one-launch cluster
// What it takes on: its eight SMs go over the logits, its atomics over the entries of
// topk_idx.  One launch against four, us in a stream (a call that is waited for):
// - lanes, logits T (E + K): 64 experts in 8 groups, Top-6, 74 K 10.4 against 12.4 (23.2,
//   25.6), 147 K 12.4, 12.5 (25.6, 27.5), 295 K 18.6, 12.4 (32.2, 27.7); 8 in 2, Top-1,
//   41 K 10.4, 10.4 (22.2, 23.9), 82 K 12.4, 10.4 (24.6, 24.0); 128 in 16, Top-1, 147 K
//   14.5, 16.5 (26.5, 30.2), 295 K 20.5, 16.5, 2.4 M 107, 20;
// - rows in shared memory, a tile per CTA or more: 96 in 12, 1024 tokens 14.5, 14.5 (27.1,
//   30.5), 2048 22.7, 15.4 (35.6, 30.9); 12 in 3, 1024 10.4, 12.4, 2048 16.6, 12.4.
constexpr long long SMALL_ENTRIES = 16384;
constexpr long long SMALL_LOGITS = 131072;
constexpr int SMALL_TOKENS = CL * TILE;
constexpr int SMALL_CELLS = 4096;   // counts (segments x (experts + 1)) that it keeps on chip

struct Params {
  const float* logits;
  long long ld;
  uint32_t mask_bits[4];
  uint32_t live;      // groups with an allowed expert
  int lane_bits, group_bits;  // lane kernels: lanes of a token and of a group, as powers of two
  int T, E, K, O, k, top_groups, n_allowed;
  const int32_t* topk_idx;
  const uint8_t* valid;
  const int32_t* seg_offsets;
  int n_seg;
  float coef;
  const float* d_loss;
  float* loss;
  int32_t* counts;
  float* d_logits;
  float* d_bias;
  int32_t* n_valid;   // [n_seg] tokens that count
  int32_t* n_live;    // segments that hold one
  double* partial;    // [grid][O + 1]: sums of the gradients, then the loss
  int n_part;
  int lane_steps;     // of a warp of balance_lanes
  int pitch;          // floats per token in shared memory
};

__device__ __forceinline__ bool allowed(const Params& p, int e) { return (p.mask_bits[e >> 5] >> (e & 31)) & 1u; }

// The segment that holds token t, of the segments [lo, hi); -1 when none does.
__device__ __forceinline__ int segment_in(const Params& p, int t, int lo, int hi) {
  if (!p.seg_offsets) return 0;
  // the last s with seg_offsets[s] <= t lies in [lo, hi)
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (p.seg_offsets[mid] <= t) lo = mid;
    else hi = mid;
  }
  return p.seg_offsets[lo] <= t && t < p.seg_offsets[lo + 1] ? lo : -1;
}
__device__ __forceinline__ int segment_of(const Params& p, int t) { return segment_in(p, t, 0, p.n_seg); }
// The segment of token t, where lo and hi are those of tokens before and after it.
__device__ __forceinline__ int segment_between(const Params& p, int t, int lo, int hi) {
  if (lo < 0 || hi < lo) return segment_of(p, t);
  return lo == hi ? lo : segment_in(p, t, lo, hi + 1);
}

// segment_of one token for a warp that asks together: 32 offsets at a time.
__device__ __forceinline__ int segment_by_warp(const Params& p, int t, int lane) {
  if (!p.seg_offsets) return 0;
  int lo = 0, hi = p.n_seg;
  while (hi - lo > 1) {
    const int step = (hi - lo + 31) / 32, i = lo + lane * step;
    const uint32_t before = __ballot_sync(0xffffffffu, i < hi && p.seg_offsets[i] <= t);
    const int n = before == 0xffffffffu ? 32 : __ffs(~before) - 1;
    if (n > 0) lo += (n - 1) * step;
    hi = n > 0 ? min(hi, lo + step) : lo + 1;
  }
  return p.seg_offsets[lo] <= t && t < p.seg_offsets[lo + 1] ? lo : -1;
}

__device__ __forceinline__ void check_segment(const Params& p, int s) {
  if (!p.seg_offsets) return;
  const int a = p.seg_offsets[s], b = p.seg_offsets[s + 1];
  if (a < 0 || b < a || b > p.T) atomicOr(&g_balance_error, 1u);
}

__global__ void __launch_bounds__(256) balance_clear_kernel(Params p) {
  pdl_trigger();
  pdl_wait();
  const long long cells = static_cast<long long>(p.n_seg) * p.E;
  for (long long i = blockIdx.x * 256LL + threadIdx.x; i < cells + p.n_seg + 1; i += gridDim.x * 256LL) {
    if (i < cells) p.counts[i] = 0;
    else if (i < cells + p.n_seg) p.n_valid[i - cells] = 0;
    else *p.n_live = 0;
  }
}

// n > 0 tokens more in segment s; the first ones make it a live segment.
__device__ __forceinline__ void add_tokens(const Params& p, int s, int n) {
  if (atomicAdd(&p.n_valid[s], n) == 0) atomicAdd(p.n_live, 1);
}

__global__ void __launch_bounds__(32 * COUNT_WARPS) balance_count_kernel(Params p) {
  // of the CTA's first and last segment; [E]: its tokens.  Others' entries, of segments
  // that lie inside the CTA's tokens, go to memory one by one (with the last one's
  // too, 262144 tokens of 64 segments took 57 us, without 46).
  __shared__ int hist[COUNT_WARPS][2][128 + 1];
  __shared__ int token_seg[COUNT_TOKENS];  // -1: does not count
  __shared__ int seg[2];
  pdl_trigger();
  constexpr int NTH = 32 * COUNT_WARPS;
  const int t0 = blockIdx.x * COUNT_TOKENS;
  const int t1 = min(t0 + COUNT_TOKENS, p.T);
  const int warp = threadIdx.x / 32;
  const int32_t* ids = p.topk_idx + static_cast<long long>(t0) * p.k;
  const int n = (t1 - t0) * p.k;
  // the entries in order, NTH apart, all of a thread's fetched before the first is used
  constexpr int AHEAD = 8 * COUNT_TOKENS / NTH;
  int id[AHEAD];
#pragma unroll
  for (int u = 0; u < AHEAD; ++u) id[u] = threadIdx.x + u * NTH < n ? ids[threadIdx.x + u * NTH] : 0;
  constexpr int PER = COUNT_TOKENS / NTH;
  bool on[PER];
#pragma unroll
  for (int u = 0; u < PER; ++u) {
    const int t = t0 + threadIdx.x + u * NTH;
    on[u] = t < t1 && !(p.valid && !p.valid[t]);
  }
  for (int i = threadIdx.x; i < COUNT_WARPS * 2 * 129; i += NTH) (&hist[0][0][0])[i] = 0;
  if (warp < 2) {
    const int s = segment_by_warp(p, warp ? t1 - 1 : t0, threadIdx.x & 31);
    if ((threadIdx.x & 31) == 0) seg[warp] = s;
  }
  __syncthreads();
  const int s0 = seg[0], s1 = seg[1];
  pdl_wait();  // the cleared counts
#pragma unroll
  for (int u = 0; u < PER; ++u) {
    const int i = threadIdx.x + u * NTH;
    const int s = on[u] ? segment_between(p, t0 + i, s0, s1) : -1;
    token_seg[i] = s;
    if (s < 0) continue;
    if (s == s0 || s == s1) atomicAdd(&hist[warp][s != s0][p.E], 1);
    else add_tokens(p, s, 1);
  }
  __syncthreads();
  // i / k for i < 8 COUNT_TOKENS by a product: 65536 / k rounded up is at most
  // (k - 1) / k too large, less than 1 / k in all
  static_assert(8 * COUNT_TOKENS * 7 < 65536, "exact quotients");
  const uint32_t per_k = (65536u + p.k - 1) / p.k;
  auto count = [&](int i, int e) {
    const int s = token_seg[(i * per_k) >> 16];
    if (s < 0) return;
    if (e < 0 || e >= p.E) atomicOr(&g_balance_error, 1u);
    else if (s == s0 || s == s1) atomicAdd(&hist[warp][s != s0][e], 1);
    else atomicAdd(&p.counts[static_cast<long long>(s) * p.E + e], 1);
  };
#pragma unroll
  for (int u = 0; u < AHEAD; ++u)
    if (threadIdx.x + u * NTH < n) count(threadIdx.x + u * NTH, id[u]);
  __syncthreads();
  // a segment that is none (-1) has no entries here
  const int half = threadIdx.x / (NTH / 2), s = half ? s1 : s0;
  if (half == 0 || s1 != s0)
    for (int i = threadIdx.x % (NTH / 2); i <= p.E; i += NTH / 2) {
      int v = 0;
#pragma unroll
      for (int w = 0; w < COUNT_WARPS; ++w) v += hist[w][half][i];
      if (v == 0) continue;
      if (i < p.E) atomicAdd(&p.counts[static_cast<long long>(s) * p.E + i], v);
      else add_tokens(p, s, v);
    }
  for (int i = blockIdx.x * NTH + threadIdx.x; i < p.n_seg; i += gridDim.x * NTH) check_segment(p, i);
}

// e^x for x <= 0 (or NaN), within 2^-22 + |x| 2^-24: a term of a softmax that
// weighs e^x is that far off, at most 4e-7 of the sum.
__device__ __forceinline__ float exp_term(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x * 1.4426950408889634f));
  return y;
}

template <int V>
struct alignas(V < 4 ? 4 * V : 16) Chunk {
  float x[V];
};

// One token.  `my` is its row in shared memory: z [E] (masked ones -infinity; then
// e = exp(z - max), then the gradient), m [K] (then p_group, then the gradient),
// 1 / sum e [K], wbar [K].  weight(i): the V centred counts from expert i on.
// Returns the loss less its part from the centre, in units of w per count, and
// leaves the gradients times du.
// ONE: a group is one chunk, gs == V.
template <int V, bool ONE, typename F>
__device__ __forceinline__ float token_gradient(const Params& p, float* my, float du, F weight) {
  const int K = p.K, gs = ONE ? V : p.E / K;
  const uint32_t live = p.live;
  float* pg = my + p.E;
  float* inv = pg + K;
  float* wbar = inv + K;
  // groups that keep their experts: of the live ones the top_groups with the
  // largest global logits, ties to the lower index
  uint32_t kept = live;
  if (p.top_groups > 0 && p.top_groups < __popc(live)) {
    for (int j = 0; j < K; ++j) {
      if (!((live >> j) & 1u)) continue;
      int before = 0;
      for (int i = 0; i < K; ++i)
        if ((live >> i) & 1u) before += pg[i] > pg[j] || (pg[i] == pg[j] && i < j);
      if (before >= p.top_groups) kept &= ~(1u << j);
    }
  }
  float top = -INFINITY;
  for (int j = 0; j < K; ++j) {
    if (!((kept >> j) & 1u)) continue;
    float* z = my + j * gs;
    float mx = -INFINITY;
    Chunk<V> v;
#pragma unroll 1
    for (int i = 0; i < gs; i += V) {
      v = *reinterpret_cast<const Chunk<V>*>(z + i);
#pragma unroll
      for (int u = 0; u < V; ++u) mx = fmaxf(mx, v.x[u]);
    }
    float s2[2] = {0.0f, 0.0f}, d2[2] = {0.0f, 0.0f};  // two chains each
#pragma unroll 1
    for (int i = 0; i < gs; i += V) {
      if (!ONE) v = *reinterpret_cast<const Chunk<V>*>(z + i);
      const Chunk<V> w = weight(j * gs + i);
#pragma unroll
      for (int u = 0; u < V; ++u) {
        v.x[u] = exp_term(v.x[u] - mx);
        s2[u & 1] += v.x[u];
        d2[u & 1] = fmaf(v.x[u], w.x[u], d2[u & 1]);
      }
      *reinterpret_cast<Chunk<V>*>(z + i) = v;
    }
    const float dot = d2[0] + d2[1];
    const float r = __frcp_rn(s2[0] + s2[1]);
    inv[j] = r;
    wbar[j] = dot * r;
    if (K > 1) top = fmaxf(top, pg[j]);
  }
  float sum = 0.0f, mean = 0.0f;
  for (int j = 0; j < K; ++j) {
    float e = 0.0f;
    if ((kept >> j) & 1u) {
      e = K > 1 ? exp_term(pg[j] - top) : 1.0f;
      sum += e;
      mean = fmaf(e, wbar[j], mean);
    }
    pg[j] = e;
  }
  const float pinv = __frcp_rn(sum);
  mean *= pinv;
  for (int j = 0; j < K; ++j) {
    float* z = my + j * gs;
    if (!((kept >> j) & 1u)) {
      for (int i = 0; i < gs; i += V) *reinterpret_cast<Chunk<V>*>(z + i) = Chunk<V>{};
      if (K > 1) pg[j] = 0.0f;
      continue;
    }
    const float pj = pg[j] * pinv * du;
    const float scale = pj * inv[j], c = wbar[j];
#pragma unroll 1
    for (int i = 0; i < gs; i += V) {
      Chunk<V> v = *reinterpret_cast<const Chunk<V>*>(z + i);
      const Chunk<V> w = weight(j * gs + i);
#pragma unroll
      for (int u = 0; u < V; ++u) v.x[u] = scale * v.x[u] * (w.x[u] - c);
      *reinterpret_cast<Chunk<V>*>(z + i) = v;
    }
    if (K > 1) pg[j] = pj * (c - mean);
  }
  return mean;
}

// A chunk at an address that is aligned to ALIGN bytes (16 or 4).
template <int C, int ALIGN>
__device__ __forceinline__ Chunk<C> load_chunk(const float* at) {
  if (ALIGN == 16) return *reinterpret_cast<const Chunk<C>*>(at);
  Chunk<C> v;
#pragma unroll
  for (int u = 0; u < C; ++u) v.x[u] = at[u];
  return v;
}
template <int C, int ALIGN>
__device__ __forceinline__ void store_chunk(float* at, const Chunk<C>& v) {
  if (ALIGN == 16) {
    *reinterpret_cast<Chunk<C>*>(at) = v;
    return;
  }
#pragma unroll
  for (int u = 0; u < C; ++u) at[u] = v.x[u];
}

// Counts and tokens of the segments, in global or shared memory.
struct CountView {
  const int32_t* c;  // counts of segment s at c + s * stride
  int stride;
  const int32_t* n;  // its tokens at n[s * n_stride]
  int n_stride;
};

constexpr int LANE_WARPS = 8;   // of a CTA of the lane kernels
constexpr int LANE_THREADS = 32 * LANE_WARPS;
// per SM: with 4 the eight-logit form's 78 registers are held to 64 (262144 tokens of
// 16 experts 22.6 us, with 3 20.8; of 64 experts 46 and 45)
constexpr int LANE_CTAS = 3;
constexpr int MAX_STEPS = 24;   // of 32 / L tokens each that a warp takes

// Tokens [first, end) in steps of 32 / L, a token on L = 2^lane_bits consecutive
// lanes: lane l of them holds the C logits l C .. l C + C - 1, which lie in one
// group, of which 2^group_bits lanes hold one.  Adds the gradients of the lane's
// columns to col[C] and of its group's global logit to glob, and the loss (once
// per token) to loss.  A step's logits are fetched during the one before; counted()
// is called once, after the first fetch, and before anything of cv is read: it
// returns coef A / (S' k).
template <int C, int ALIGN, typename F>
__device__ __forceinline__ void lane_tokens(const Params& p, int first, int end, const CountView& cv, F counted,
                                            float* col, float& glob, float& loss) {
  const int L = 1 << p.lane_bits, G = 1 << p.group_bits;
  const int lane = threadIdx.x & 31;
  const int part = lane & (L - 1);
  const int j = part >> p.group_bits;  // group
  uint32_t keep = 0;
#pragma unroll
  for (int u = 0; u < C; ++u) keep |= static_cast<uint32_t>(allowed(p, part * C + u)) << u;
  const bool live = (p.live >> j) & 1u;
  const bool prune = p.top_groups > 0 && p.top_groups < __popc(p.live);
  int seg = -2, nv = 0, mean_count = 0, seg_from = 0, seg_to = 0;  // the segment whose counts are in w
  float unit = 0.0f;
  float w[C];
#pragma unroll
  for (int u = 0; u < C; ++u) w[u] = 0.0f;
  const int step = 32 >> p.lane_bits;
  const int mine = lane >> p.lane_bits;
  Chunk<C> z_next = {};
  float m_next = 0.0f;
  bool on_next = false;
  auto fetch = [&](int t) {
    on_next = t < end;
    if (!on_next) return;
    const float* row = p.logits + static_cast<long long>(t) * p.ld;
    z_next = load_chunk<C, ALIGN>(row + part * C);
    if (p.K > 1) m_next = row[p.E + j];
    if (p.valid) on_next = p.valid[t] != 0;
  };
  fetch(first + mine);
  const float per_segment = counted();
  const float upstream = p.d_loss ? *p.d_loss : 1.0f;
  for (int t0 = first; t0 < end; t0 += step) {
    const int t = t0 + mine;
    const bool in = t < end;
    Chunk<C> z = z_next;
    const float m = m_next;
    bool on = on_next;
    fetch(t + step);
    if (on && (seg == -2 || t < seg_from || t >= seg_to)) {
      // another segment: its counts less their mean
      seg = segment_of(p, t);
      seg_from = 0;
      seg_to = p.T;
      nv = 0;
      if (seg >= 0) {
        if (p.seg_offsets) {
          seg_from = p.seg_offsets[seg];
          seg_to = p.seg_offsets[seg + 1];
        }
        nv = cv.n[seg * cv.n_stride];
      } else {
        seg_from = t;  // a token of no segment says nothing of its neighbours
        seg_to = t + 1;
      }
      if (nv > 0) {
        mean_count = static_cast<int>(static_cast<long long>(p.k) * nv / p.n_allowed);
        unit = per_segment / nv / nv;  // w_i = unit * c_i
        const int32_t* c = cv.c + static_cast<long long>(seg) * cv.stride + part * C;
#pragma unroll
        for (int u = 0; u < C; ++u) w[u] = static_cast<float>(c[u] - mean_count);
      }
    }
    on = on && nv > 0;  // no tokens: also where reported bounds made no sense
    // the group's softmax over its allowed experts
    float mx = -INFINITY;
#pragma unroll
    for (int u = 0; u < C; ++u) {
      z.x[u] = (keep >> u) & 1u ? z.x[u] : -INFINITY;
      mx = fmaxf(mx, z.x[u]);
    }
    for (int o = 1; o < G; o <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
    float s2[2] = {0.0f, 0.0f}, d2[2] = {0.0f, 0.0f};  // two chains each
#pragma unroll
    for (int u = 0; u < C; ++u) {
      z.x[u] = exp_term(z.x[u] - mx);
      s2[u & 1] += z.x[u];
      d2[u & 1] = fmaf(z.x[u], w[u], d2[u & 1]);
    }
    float sum = s2[0] + s2[1], dot = d2[0] + d2[1];
    for (int o = 1; o < G; o <<= 1) {
      sum += __shfl_xor_sync(0xffffffffu, sum, o);
      dot += __shfl_xor_sync(0xffffffffu, dot, o);
    }
    const float r = 1.0f / sum;
    const float wbar = dot * r;
    // the groups': of the live ones the top_groups with the largest global logits
    // keep their experts, ties to the lower index
    bool kept = live;
    if (prune) {
      int before = 0;
      for (int i = 0; i < p.K; ++i) {
        const float o = __shfl_sync(0xffffffffu, m, (lane & ~(L - 1)) | (i << p.group_bits));
        if ((p.live >> i) & 1u) before += o > m || (o == m && i < j);
      }
      kept = kept && before < p.top_groups;
    }
    float e = 1.0f;
    if (p.K > 1) {
      float top = kept ? m : -INFINITY;
      for (int o = G; o < L; o <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
      e = kept ? exp_term(m - top) : 0.0f;
    }
    float all = e, mean = kept ? e * wbar : 0.0f;
    for (int o = G; o < L; o <<= 1) {
      all += __shfl_xor_sync(0xffffffffu, all, o);
      mean += __shfl_xor_sync(0xffffffffu, mean, o);
    }
    const float inv = 1.0f / all;
    mean *= inv;
    const float pj = e * inv * unit * upstream;
    const float scale = pj * r;
    float dm = 0.0f;
#pragma unroll
    for (int u = 0; u < C; ++u) z.x[u] = on && kept ? scale * z.x[u] * (w[u] - wbar) : 0.0f;
    if (on && kept) dm = pj * (wbar - mean);
    if (on && part == 0) loss += unit * (mean + mean_count);
#pragma unroll
    for (int u = 0; u < C; ++u) col[u] += z.x[u];
    glob += dm;
    if (in && p.d_logits) {
      float* out = p.d_logits + static_cast<long long>(t) * p.O;
      store_chunk<C, ALIGN>(out + part * C, z);
      if (p.K > 1 && (part & (G - 1)) == 0) out[p.E + j] = dm;
    }
  }
}

// Adds up the CTA's warps: to total[0 .. O] (global or shared) from the lanes'
// columns.  sums: shared [LANE_WARPS][O + 1].  All threads call it.
template <int C>
__device__ __forceinline__ void lane_totals(const Params& p, float* col, float glob, float loss, float* sums,
                                            double* total) {
  const int L = 1 << p.lane_bits, G = 1 << p.group_bits;
  const int lane = threadIdx.x & 31;
  for (int o = L; o < 32; o <<= 1) {
#pragma unroll
    for (int u = 0; u < C; ++u) col[u] += __shfl_xor_sync(0xffffffffu, col[u], o);
    glob += __shfl_xor_sync(0xffffffffu, glob, o);
    loss += __shfl_xor_sync(0xffffffffu, loss, o);
  }
  float* mine = sums + (threadIdx.x >> 5) * (p.O + 1);
  if (lane < L) {
#pragma unroll
    for (int u = 0; u < C; ++u) mine[lane * C + u] = col[u];
    if (p.K > 1 && (lane & (G - 1)) == 0) mine[p.E + (lane >> p.group_bits)] = glob;
    if (lane == 0) mine[p.O] = loss;
  }
  __syncthreads();
  for (int c = threadIdx.x; c <= p.O; c += LANE_THREADS) {
    double v = 0.0;
#pragma unroll
    for (int w = 0; w < LANE_WARPS; ++w) v += sums[w * (p.O + 1) + c];
    total[c] = v;
  }
}

template <int C, int ALIGN>
__global__ void __launch_bounds__(LANE_THREADS, LANE_CTAS) balance_lanes_kernel(Params p) {
  __shared__ float sums[LANE_WARPS * 145];
  pdl_trigger();
  const int per_warp = p.lane_steps * (32 >> p.lane_bits);
  const int first = (blockIdx.x * LANE_WARPS + (threadIdx.x >> 5)) * per_warp;
  float col[C], glob = 0.0f, loss = 0.0f;
#pragma unroll
  for (int u = 0; u < C; ++u) col[u] = 0.0f;
  lane_tokens<C, ALIGN>(
      p, first, min(first + per_warp, p.T), CountView{p.counts, p.E, p.n_valid, 1},
      [&] {
        pdl_wait();
        return p.coef * p.n_allowed / (static_cast<float>(max(1, *p.n_live)) * p.k);
      },
      col, glob, loss);
  lane_totals<C>(p, col, glob, loss, sums, p.partial + static_cast<long long>(blockIdx.x) * (p.O + 1));
}

// Moves of a tile between global and shared memory: a thread keeps a column chunk
// of V logits and takes every SEGS-th row.
template <int V>
struct Mover {
  using Vec = Chunk<V>;
  int col, seg, segs;
  bool on;
  uint32_t keep;  // bit u: column col + u is not a masked expert's
  __device__ __forceinline__ Mover(const Params& p) {
    const int units = (p.O + V - 1) / V;
    segs = NT / units;
    seg = threadIdx.x / units;
    col = (threadIdx.x - seg * units) * V;
    on = seg < segs;
    keep = 0;
    for (int u = 0; u < V; ++u) keep |= static_cast<uint32_t>(col + u >= p.E || allowed(p, col + u)) << u;
  }
  __device__ __forceinline__ void load(const Params& p, float* rows, int t0, int n) const {
    if (!on) return;
#pragma unroll 8
    for (int r = seg; r < n; r += segs) {
      Vec v = *reinterpret_cast<const Vec*>(p.logits + (t0 + r) * p.ld + col);
#pragma unroll
      for (int u = 0; u < V; ++u) v.x[u] = (keep >> u) & 1u ? v.x[u] : -INFINITY;
      *reinterpret_cast<Vec*>(rows + r * p.pitch + col) = v;
    }
  }
  // stores the gradients (out != nullptr) and adds them to sums
  __device__ __forceinline__ void store(const Params& p, const float* rows, int t0, int n, double* sums) const {
    if (!on) return;
    float acc[V] = {};
    float* out = p.d_logits ? p.d_logits + static_cast<long long>(t0) * p.O + col : nullptr;
#pragma unroll 4
    for (int r = seg; r < n; r += segs) {
      const Vec v = *reinterpret_cast<const Vec*>(rows + r * p.pitch + col);
#pragma unroll
      for (int u = 0; u < V; ++u) acc[u] += v.x[u];
      if (out) *reinterpret_cast<Vec*>(out + static_cast<long long>(r) * p.O) = v;
    }
#pragma unroll
    for (int u = 0; u < V; ++u) sums[u] += acc[u];
  }
};

// Adds up the CTA's threads: column sums (through `scratch`, NT * V doubles) and
// loss, to total[0 .. O].  All threads call it.
template <int V>
__device__ __forceinline__ void cta_totals(const Params& p, const Mover<V>& mv, const double* sums, double loss,
                                           double* scratch, double* total) {
  __shared__ double warp_loss[NT / 32];
#pragma unroll
  for (int u = 0; u < V; ++u) scratch[threadIdx.x * V + u] = sums[u];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) loss += __shfl_down_sync(0xffffffffu, loss, o);
  if (threadIdx.x % 32 == 0) warp_loss[threadIdx.x / 32] = loss;
  __syncthreads();
  const int units = (p.O + V - 1) / V;
  for (int c = threadIdx.x; c < p.O; c += NT) {
    double v = 0.0;
    for (int g = 0; g < mv.segs; ++g) v += scratch[(g * units + c / V) * V + c % V];
    total[c] = v;
  }
  if (threadIdx.x == 0) {
    double v = 0.0;
    for (int w = 0; w < NT / 32; ++w) v += warp_loss[w];
    total[p.O] = v;
  }
}

// One tile per CTA: several each would leave the last of them uneven.  Serves groups of
// fewer than four experts, and where their size or number is not a power of two.
template <int V, bool ONE>
__global__ void __launch_bounds__(NT) balance_main_kernel(Params p) {
  constexpr int M = V < 4 ? V : 4;
  extern __shared__ __align__(16) float rows[];  // [TILE][pitch], then the centred counts of one segment [E]
  __shared__ int seg[2];
  float* tab = rows + TILE * p.pitch;
  pdl_trigger();
  const Mover<M> mv(p);
  const int t0 = blockIdx.x * TILE;
  const int n = min(TILE, p.T - t0);
  if (threadIdx.x >= NT - 2) {  // the last warp holds no token
    const int i = threadIdx.x - (NT - 2);
    seg[i] = segment_of(p, i ? t0 + n - 1 : t0);
  }
  mv.load(p, rows, t0, n);
  const int t = t0 + threadIdx.x;
  const bool counts = threadIdx.x < n && !(p.valid && !p.valid[t]);
  pdl_wait();  // what the caller gave is read before, the counts after
  const float upstream = p.d_loss ? *p.d_loss : 1.0f;
  const float per_segment = p.coef * p.n_allowed / (static_cast<float>(max(1, *p.n_live)) * p.k);
  __syncthreads();
  const int s0 = seg[0], s1 = seg[1];
  const bool one = s0 == s1 && s0 >= 0;
  if (one) {
    const int mean = static_cast<int>(static_cast<long long>(p.k) * p.n_valid[s0] / p.n_allowed);
    for (int i = threadIdx.x; i < p.E; i += NT)
      tab[i] = static_cast<float>(p.counts[static_cast<long long>(s0) * p.E + i] - mean);
    __syncthreads();
  }
  double loss = 0.0;
  if (threadIdx.x < n) {
    float* my = rows + threadIdx.x * p.pitch;
    const int s = !counts ? -1 : one ? s0 : segment_of(p, t);
    const int nv = s >= 0 ? p.n_valid[s] : 0;  // 0 also where reported bounds made no sense
    if (nv > 0) {
      const int mean_count = static_cast<int>(static_cast<long long>(p.k) * nv / p.n_allowed);
      const float unit = per_segment / nv / nv;  // w_i = unit * c_i
      float mean;
      if (one) {
        mean = token_gradient<V, ONE>(p, my, unit * upstream,
                                      [&](int i) { return *reinterpret_cast<const Chunk<V>*>(tab + i); });
      } else {
        const int32_t* cnt = p.counts + static_cast<long long>(s) * p.E;
        mean = token_gradient<V, ONE>(p, my, unit * upstream, [&](int i) {
          Chunk<V> w;
#pragma unroll
          for (int u = 0; u < V; ++u) w.x[u] = static_cast<float>(cnt[i + u] - mean_count);
          return w;
        });
      }
      loss = unit * (mean + mean_count);
    } else {
      for (int i = 0; i < p.O; ++i) my[i] = 0.0f;
    }
  }
  __syncthreads();
  double sums[M] = {};
  mv.store(p, rows, t0, n, sums);
  __syncthreads();
  cta_totals<M>(p, mv, sums, loss, reinterpret_cast<double*>(rows), p.partial + static_cast<long long>(blockIdx.x) * (p.O + 1));
}

// ------------------------------------------------------------- short batches
__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_barrier() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// The object at `p` in this CTA's shared memory, in CTA `rank` of the cluster.
template <typename T>
__device__ __forceinline__ T ld_cluster(const T* p, uint32_t rank) {
  uint32_t a;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;"
               : "=r"(a)
               : "r"(static_cast<uint32_t>(__cvta_generic_to_shared(p))), "r"(rank));
  T v;
  if constexpr (sizeof(T) == 8) asm volatile("ld.shared::cluster.f64 %0, [%1];" : "=d"(v) : "r"(a) : "memory");
  else asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(v) : "r"(a) : "memory");
  return v;
}

// The batch's counts and live segments, from those of the cluster's CTAs (mine, cnt:
// [n_seg][E + 1], the last of each row its tokens).  Every thread of every CTA calls
// it after it has counted its tokens in `mine`.
__device__ __forceinline__ void join_counts(const Params& p, uint32_t rank, const int* mine, int* cnt, int* n_live) {
  const int cells = p.n_seg * (p.E + 1);
  if (rank == 0)
    for (int s = threadIdx.x; s < p.n_seg; s += blockDim.x) check_segment(p, s);
  cluster_barrier();
  for (int i = threadIdx.x; i < cells; i += blockDim.x) {
    int v = 0;
#pragma unroll
    for (int c = 0; c < CL; ++c) v += ld_cluster(mine + i, c);
    cnt[i] = v;
    const int s = i / (p.E + 1), e = i - s * (p.E + 1);
    if (e == p.E) {
      if (v > 0) atomicAdd(n_live, 1);
    } else if (rank == 0) {
      p.counts[s * p.E + e] = v;
    }
  }
  __syncthreads();
}
// Counts token t in `mine`.
__device__ __forceinline__ void count_token(const Params& p, int t, int* mine) {
  if (p.valid && !p.valid[t]) return;
  const int s = segment_of(p, t);
  if (s < 0) return;
  int* h = mine + s * (p.E + 1);
  atomicAdd(&h[p.E], 1);
  for (int j = 0; j < p.k; ++j) {
    const int e = p.topk_idx[static_cast<long long>(t) * p.k + j];
    if (e < 0 || e >= p.E) atomicOr(&g_balance_error, 1u);
    else atomicAdd(&h[e], 1);
  }
}
// Adds up the cluster's totals into the results.
__device__ __forceinline__ void join_totals(const Params& p, uint32_t rank, const double* total) {
  cluster_barrier();
  if (rank == 0)
    for (int c = threadIdx.x; c <= p.O; c += blockDim.x) {
      double v = 0.0;
#pragma unroll
      for (int r = 0; r < CL; ++r) v += ld_cluster(total + c, r);
      if (c == p.O) *p.loss = static_cast<float>(v);
      else if (p.d_bias) p.d_bias[c] = static_cast<float>(v);
    }
  cluster_barrier();  // no CTA ends while its totals are read
}

// A cluster of CL CTAs, each an equal range of the tokens, each warp of it too.
template <int C, int ALIGN>
__global__ void __launch_bounds__(LANE_THREADS) balance_small_lanes_kernel(Params p) {
  extern __shared__ __align__(16) float sums[];                          // [LANE_WARPS][O + 1]
  double* total = reinterpret_cast<double*>(sums + LANE_WARPS * (p.O + 1));  // [O + 1]
  int* mine = reinterpret_cast<int*>(total + p.O + 1);
  int* cnt = mine + p.n_seg * (p.E + 1);
  __shared__ int n_live;
  const uint32_t rank = cluster_rank();
  const int per_cta = (p.T + CL - 1) / CL;
  const int c0 = min(static_cast<int>(rank) * per_cta, p.T), c1 = min(c0 + per_cta, p.T);
  for (int i = threadIdx.x; i < p.n_seg * (p.E + 1); i += LANE_THREADS) mine[i] = 0;
  if (threadIdx.x == 0) n_live = 0;
  __syncthreads();
  for (int t = c0 + threadIdx.x; t < c1; t += LANE_THREADS) count_token(p, t, mine);
  const int step = 32 >> p.lane_bits;
  const int per_warp = ((c1 - c0 + LANE_WARPS - 1) / LANE_WARPS + step - 1) / step * step;
  const int first = c0 + (threadIdx.x >> 5) * per_warp;
  float col[C], glob = 0.0f, loss = 0.0f;
#pragma unroll
  for (int u = 0; u < C; ++u) col[u] = 0.0f;
  lane_tokens<C, ALIGN>(
      p, first, min(first + per_warp, c1), CountView{cnt, p.E + 1, cnt + p.E, p.E + 1},
      [&] {
        join_counts(p, rank, mine, cnt, &n_live);
        return p.coef * p.n_allowed / (static_cast<float>(max(1, n_live)) * p.k);
      },
      col, glob, loss);
  lane_totals<C>(p, col, glob, loss, sums, total);
  join_totals(p, rank, total);
}

// A cluster of CL CTAs; CTA c takes the tiles c, c + CL, ...
template <int V, bool ONE>
__global__ void __launch_bounds__(NT) balance_small_kernel(Params p) {
  constexpr int M = V < 4 ? V : 4;
  extern __shared__ __align__(16) float rows[];  // [TILE][pitch]
  double* total = reinterpret_cast<double*>(rows + TILE * p.pitch);                // [O + 1]
  int* mine = reinterpret_cast<int*>(total + p.O + 1);                             // [n_seg][E + 1] of this CTA
  int* cnt = mine + p.n_seg * (p.E + 1);                                           // the same of the batch
  __shared__ int n_live;
  const uint32_t rank = cluster_rank();
  const int cells = p.n_seg * (p.E + 1);
  const Mover<M> mv(p);
  const int tiles = (p.T + TILE - 1) / TILE;
  for (int i = threadIdx.x; i < cells; i += NT) mine[i] = 0;
  if (threadIdx.x == 0) n_live = 0;
  __syncthreads();
  // the first tile's logits travel while its entries are counted
  if (static_cast<int>(rank) < tiles) mv.load(p, rows, rank * TILE, min(TILE, p.T - static_cast<int>(rank) * TILE));
  for (int tile = rank; tile < tiles; tile += CL) {
    const int t = tile * TILE + threadIdx.x;
    if (threadIdx.x < TILE && t < p.T) count_token(p, t, mine);
  }
  join_counts(p, rank, mine, cnt, &n_live);
  const float upstream = p.d_loss ? *p.d_loss : 1.0f;
  const float per_segment = p.coef * p.n_allowed / (static_cast<float>(max(1, n_live)) * p.k);
  double loss = 0.0;
  double sums[M] = {};
  for (int tile = rank; tile < tiles; tile += CL) {
    const int t0 = tile * TILE;
    const int n = min(TILE, p.T - t0);
    if (tile != static_cast<int>(rank)) mv.load(p, rows, t0, n);
    __syncthreads();
    const int t = t0 + threadIdx.x;
    if (threadIdx.x < n) {
      float* my = rows + threadIdx.x * p.pitch;
      const int s = p.valid && !p.valid[t] ? -1 : segment_of(p, t);
      const int* c = cnt + (s >= 0 ? s : 0) * (p.E + 1);
      const int nv = s >= 0 ? c[p.E] : 0;
      if (nv > 0) {
        const int mean_count = static_cast<int>(static_cast<long long>(p.k) * nv / p.n_allowed);
        const float unit = per_segment / nv / nv;  // w_i = unit * c_i
        const float mean = token_gradient<V, ONE>(p, my, unit * upstream, [&](int i) {
          Chunk<V> w;
#pragma unroll
          for (int u = 0; u < V; ++u) w.x[u] = static_cast<float>(c[i + u] - mean_count);
          return w;
        });
        loss += unit * (mean + mean_count);  // the sum over tokens in 64 bits: they are few to a thread
      } else {
        for (int i = 0; i < p.O; ++i) my[i] = 0.0f;
      }
    }
    __syncthreads();
    mv.store(p, rows, t0, n, sums);
    __syncthreads();
  }
  cta_totals<M>(p, mv, sums, loss, reinterpret_cast<double*>(rows), total);
  join_totals(p, rank, total);
}

// One column of the partial sums per CTA, added in a fixed order.
__global__ void __launch_bounds__(256) balance_final_kernel(Params p) {
  __shared__ double part[8];
  pdl_trigger();
  pdl_wait();
  const int c = blockIdx.x;
  double v = 0.0;
#pragma unroll 8
  for (int b = threadIdx.x; b < p.n_part; b += 256) v += p.partial[static_cast<long long>(b) * (p.O + 1) + c];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_down_sync(0xffffffffu, v, o);
  if (threadIdx.x % 32 == 0) part[threadIdx.x / 32] = v;
  __syncthreads();
  if (threadIdx.x > 0) return;
  for (int w = 1; w < 8; ++w) v += part[w];
  if (c == p.O) *p.loss = static_cast<float>(v);
  else if (p.d_bias) p.d_bias[c] = static_cast<float>(v);
}

// CTAs of balance_main at most: no kernel gives one fewer tokens than a tile.
int grid_for(int T) { return (T + TILE - 1) / TILE; }

bool is_small(const Params& p, bool lanes) {
  const long long T = p.T;
  return (lanes ? T * p.O <= SMALL_LOGITS : T <= SMALL_TOKENS) && T * p.k <= SMALL_ENTRIES &&
         static_cast<long long>(p.n_seg) * (p.E + 1) <= SMALL_CELLS;
}

cudaError_t launch_counts(const Params& p, cudaStream_t s) {
  {
    KernelScope ks("balance_clear", s);
    const long long cells = static_cast<long long>(p.n_seg) * (p.E + 1) + 1;
    const long long blocks = (cells + 255) / 256;
    cudaError_t e =
        launch_kernel(balance_clear_kernel, dim3(static_cast<unsigned>(blocks < 1024 ? blocks : 1024)), dim3(256), 0, s, p);
    if (e != cudaSuccess || p.T == 0) return e;
  }
  KernelScope ks("balance_count", s);
  return launch_kernel(balance_count_kernel, dim3((p.T + COUNT_TOKENS - 1) / COUNT_TOKENS), dim3(32 * COUNT_WARPS), 0, s, p);
}

cudaError_t launch_final(const Params& p, cudaStream_t s) {
  KernelScope ks("balance_final", s);
  return launch_kernel(balance_final_kernel, dim3(p.O + 1), dim3(256), 0, s, p);
}

template <int V, bool ONE>
cudaError_t launch_width(const Params& p, cudaStream_t s) {
  cudaError_t e;
  // the totals' scratch, NT doubles per column of a move, fits the tile: rows have 5
  // floats at least, those of chunks 12
  const int tile_bytes = TILE * p.pitch * 4;
  if (is_small(p, false)) {
    const int smem = tile_bytes + (p.O + 1) * 8 + 2 * p.n_seg * (p.E + 1) * 4;
    e = ensure_smem_attr(reinterpret_cast<const void*>(balance_small_kernel<V, ONE>), smem);
    if (e != cudaSuccess) return e;
    KernelScope ks("balance", s);
    return launch_cluster(balance_small_kernel<V, ONE>, 1, CL, NT, (size_t)smem, s, p);
  }
  e = launch_counts(p, s);
  if (e != cudaSuccess) return e;
  if (p.T > 0) {
    const int smem = tile_bytes + p.E * 4;
    e = ensure_smem_attr(reinterpret_cast<const void*>(balance_main_kernel<V, ONE>), smem);
    if (e != cudaSuccess) return e;
    KernelScope ks("balance_main", s);
    e = launch_kernel(balance_main_kernel<V, ONE>, dim3(p.n_part), dim3(NT), (size_t)smem, s, p);
    if (e != cudaSuccess) return e;
  }
  return launch_final(p, s);
}

template <int C, int ALIGN>
cudaError_t launch_lanes(Params p, cudaStream_t s) {
  cudaError_t e;
  if (is_small(p, true)) {
    const int smem = LANE_WARPS * (p.O + 1) * 4 + (p.O + 1) * 8 + 2 * p.n_seg * (p.E + 1) * 4;
    e = ensure_smem_attr(reinterpret_cast<const void*>(balance_small_lanes_kernel<C, ALIGN>), smem);
    if (e != cudaSuccess) return e;
    KernelScope ks("balance", s);
    return launch_cluster(balance_small_lanes_kernel<C, ALIGN>, 1, CL, LANE_THREADS, (size_t)smem, s, p);
  }
  // One wave of CTAs where that leaves a warp at most MAX_STEPS steps, whose sums are
  // fp32, and not fewer tokens than a tile.  64 experts, us, against 8 steps: 16384
  // tokens 16.4 / 20.5, 10^6 in 100 segments 131 / 141.
  const int a_step = LANE_WARPS * (32 >> p.lane_bits);
  const long long wave = static_cast<long long>(sm_count()) * LANE_CTAS * a_step;
  p.lane_steps = static_cast<int>(std::min<long long>((p.T + wave - 1) / wave, MAX_STEPS));
  p.lane_steps = std::max({p.lane_steps, TILE / a_step, 1});
  const int per_cta = a_step * p.lane_steps;
  p.n_part = (p.T + per_cta - 1) / per_cta;
  e = launch_counts(p, s);
  if (e != cudaSuccess) return e;
  if (p.T > 0) {
    KernelScope ks("balance_main", s);
    e = launch_kernel(balance_lanes_kernel<C, ALIGN>, dim3(p.n_part), dim3(LANE_THREADS), 0, s, p);
    if (e != cudaSuccess) return e;
  }
  return launch_final(p, s);
}

bool power_of_two(int x) { return x > 0 && (x & (x - 1)) == 0; }
int log2_of(int x) {
  int b = 0;
  while ((1 << b) < x) ++b;
  return b;
}

size_t align256(size_t x) { return (x + 255) / 256 * 256; }

}  // namespace

size_t balance_bytes(int T, int E, int K, int n_seg) {
  const int O = E + (K > 1 ? K : 0);
  return align256(static_cast<size_t>(grid_for(T)) * (O + 1) * 8) + align256((static_cast<size_t>(n_seg) + 1) * 4);
}

cudaError_t launch_balance(const BalanceArgs& a, cudaStream_t s) {
  Params p;
  p.logits = a.logits;
  p.ld = a.ld;
  for (int i = 0; i < 4; ++i) p.mask_bits[i] = a.mask_bits[i];
  p.live = 0;
  for (int e = 0; e < a.E; ++e)
    if ((a.mask_bits[e >> 5] >> (e & 31)) & 1u) p.live |= 1u << (e / (a.E / a.K));
  p.T = a.T;
  p.E = a.E;
  p.K = a.K;
  p.O = a.E + (a.K > 1 ? a.K : 0);
  p.k = a.k;
  p.top_groups = a.K > 1 ? a.top_groups : 0;
  p.n_allowed = a.n_allowed;
  p.topk_idx = a.topk_idx;
  p.valid = a.valid;
  p.seg_offsets = a.seg_offsets;
  p.n_seg = a.n_seg;
  p.coef = a.coef;
  p.d_loss = a.d_loss;
  p.loss = a.loss;
  p.counts = a.counts;
  p.d_logits = a.d_logits;
  p.d_bias = a.d_bias;
  const int grid = grid_for(a.T);
  uint8_t* ws = static_cast<uint8_t*>(a.workspace);
  p.partial = reinterpret_cast<double*>(ws);
  p.n_valid = reinterpret_cast<int32_t*>(ws + align256(static_cast<size_t>(grid) * (p.O + 1) * 8));
  p.n_live = p.n_valid + a.n_seg;
  p.n_part = grid;
  // Chunks of four floats where every group, row and address allows it; the rows'
  // pitch puts eight rows' chunks (32 rows' floats) into different banks.
  const bool vec = (a.E / a.K) % 4 == 0 && p.O % 4 == 0 && a.ld % 4 == 0 &&
                   (reinterpret_cast<uintptr_t>(a.logits) | reinterpret_cast<uintptr_t>(a.d_logits)) % 16 == 0;
  const int floats = a.E + 3 * a.K;
  p.pitch = vec ? ((floats + 3) / 4 | 1) * 4 : floats | 1;
  const int gs = a.E / a.K;
  cudaError_t e;
  const int chunk = gs % 8 == 0 ? 8 : 4;
  if (gs % 4 == 0 && power_of_two(gs) && power_of_two(a.K) && a.E / chunk <= 16) {
    p.group_bits = log2_of(gs / chunk);
    p.lane_bits = log2_of(a.E / chunk);
    if (chunk == 8) e = vec ? launch_lanes<8, 16>(p, s) : launch_lanes<8, 4>(p, s);
    else e = vec ? launch_lanes<4, 16>(p, s) : launch_lanes<4, 4>(p, s);
  } else if (vec) {
    e = gs % 8 != 0 ? launch_width<4, false>(p, s)
        : gs == 8   ? launch_width<8, true>(p, s)
                    : launch_width<8, false>(p, s);
  } else {
    e = launch_width<1, false>(p, s);
  }
  if (e != cudaSuccess) return e;
  return cudaGetLastError();
}

cudaError_t read_balance_error(unsigned int* word) {
  unsigned int zero = 0;
  cudaError_t e = cudaMemcpyFromSymbol(word, g_balance_error, sizeof(unsigned int));
  if (e != cudaSuccess) return e;
  return cudaMemcpyToSymbol(g_balance_error, &zero, sizeof(unsigned int));
}

}  // namespace ec2moe
