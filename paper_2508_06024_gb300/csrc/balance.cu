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
// balance_count: integer histograms (atomics on integers, whose order does not
// matter) and S'.  balance_main: tiles of 128 tokens in shared memory, a token
// per thread, each CTA a contiguous range of tiles; one pass over the logits gives
// the loss and both gradients.  balance_final adds the CTAs' partial sums in
// order.  Bounded by HBM for long batches (the logits are read once, their
// gradients written once), by the launches for short ones.
#include <cuda_runtime.h>

#include "common.cuh"
#include "internal.h"

namespace ec2moe {

// nonzero: an expert id or a segment bound out of range was skipped
__device__ unsigned int g_balance_error;

namespace {

constexpr int TILE = 128;       // tokens per tile, threads per CTA
constexpr int MAX_GRID = 608;   // CTAs of balance_main
constexpr int COUNT_TOKENS = 1024;  // tokens per CTA of balance_count

struct Params {
  const float* logits;
  long long ld;
  uint32_t mask_bits[4];
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
  int32_t* ticket;
  double* partial;    // [grid][O + 1]: sums of the gradients, then the loss
  int n_part;
  int pitch;          // floats per token in shared memory
};

__device__ __forceinline__ bool allowed(const Params& p, int e) { return (p.mask_bits[e >> 5] >> (e & 31)) & 1u; }

// The segment that holds token t, -1 when none does.
__device__ __forceinline__ int segment_of(const Params& p, int t) {
  if (!p.seg_offsets) return 0;
  int lo = 0, hi = p.n_seg;  // the last s with seg_offsets[s] <= t lies in [lo, hi)
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (p.seg_offsets[mid] <= t) lo = mid;
    else hi = mid;
  }
  return p.seg_offsets[lo] <= t && t < p.seg_offsets[lo + 1] ? lo : -1;
}

__global__ void __launch_bounds__(256) balance_clear_kernel(Params p) {
  pdl_trigger();
  pdl_wait();
  const long long cells = static_cast<long long>(p.n_seg) * p.E;
  for (long long i = blockIdx.x * 256LL + threadIdx.x; i < cells + p.n_seg + 2; i += gridDim.x * 256LL) {
    if (i < cells) p.counts[i] = 0;
    else if (i < cells + p.n_seg) p.n_valid[i - cells] = 0;
    else if (i == cells + p.n_seg) *p.ticket = 0;
    else *p.n_live = 0;
  }
}

__global__ void __launch_bounds__(256) balance_count_kernel(Params p) {
  __shared__ int hist[128 + 1];
  __shared__ int first_seg, last;
  pdl_trigger();
  pdl_wait();
  const int t0 = blockIdx.x * COUNT_TOKENS;
  for (int i = threadIdx.x; i <= p.E; i += 256) hist[i] = 0;
  if (threadIdx.x == 0) first_seg = segment_of(p, t0);
  __syncthreads();
  const int s0 = first_seg;
  for (int t = t0 + threadIdx.x; t < t0 + COUNT_TOKENS && t < p.T; t += 256) {
    if (p.valid && !p.valid[t]) continue;
    const int s = segment_of(p, t);
    if (s < 0) continue;
    if (s == s0) atomicAdd(&hist[p.E], 1);
    else atomicAdd(&p.n_valid[s], 1);
    for (int j = 0; j < p.k; ++j) {
      const int e = p.topk_idx[static_cast<long long>(t) * p.k + j];
      if (e < 0 || e >= p.E) {
        atomicOr(&g_balance_error, 1u);
        continue;
      }
      if (s == s0) atomicAdd(&hist[e], 1);
      else atomicAdd(&p.counts[static_cast<long long>(s) * p.E + e], 1);
    }
  }
  __syncthreads();
  if (s0 >= 0)
    for (int i = threadIdx.x; i <= p.E; i += 256)
      if (hist[i]) atomicAdd(i < p.E ? &p.counts[static_cast<long long>(s0) * p.E + i] : &p.n_valid[s0], hist[i]);
  // the last CTA to arrive counts the segments that hold a token
  __threadfence();
  __syncthreads();
  if (threadIdx.x == 0) last = atomicAdd(p.ticket, 1) == static_cast<int>(gridDim.x) - 1;
  __syncthreads();
  if (!last) return;
  __threadfence();
  int n = 0;
  for (int s = threadIdx.x; s < p.n_seg; s += 256) {
    n += __ldcg(&p.n_valid[s]) > 0;
    if (p.seg_offsets) {
      const int a = p.seg_offsets[s], b = p.seg_offsets[s + 1];
      if (a < 0 || b < a || b > p.T) atomicOr(&g_balance_error, 1u);
    }
  }
  if (n) atomicAdd(p.n_live, n);
}

// Shared row of a token: z [E] (then e = exp(z - max), then the gradient), m [K]
// (then p_group, then the gradient), 1 / sum e [K], wbar [K].
__global__ void __launch_bounds__(TILE) balance_main_kernel(Params p) {
  extern __shared__ float rows[];
  __shared__ double warp_loss[TILE / 32];
  pdl_trigger();
  pdl_wait();
  const int E = p.E, K = p.K, O = p.O, gs = E / K;
  const int tiles = (p.T + TILE - 1) / TILE;
  const int tile0 = static_cast<int>(static_cast<long long>(tiles) * blockIdx.x / gridDim.x);
  const int tile1 = static_cast<int>(static_cast<long long>(tiles) * (blockIdx.x + 1) / gridDim.x);
  const float upstream = p.d_loss ? *p.d_loss : 1.0f;
  const double per_segment = static_cast<double>(p.coef) * p.n_allowed / (static_cast<double>(max(1, *p.n_live)) * p.k);
  int live_groups = 0;
  uint32_t live = 0;
  for (int j = 0; j < K; ++j) {
    bool any = false;
    for (int i = j * gs; i < (j + 1) * gs; ++i) any |= allowed(p, i);
    live |= static_cast<uint32_t>(any) << j;
    live_groups += any;
  }
  const bool prune = p.top_groups > 0 && p.top_groups < live_groups;
  float* my = rows + threadIdx.x * p.pitch;
  float* pg = my + E;
  float* inv = pg + K;
  float* wbar = inv + K;
  double loss = 0.0;
  double sums[2] = {0.0, 0.0};  // columns threadIdx.x and threadIdx.x + TILE
  for (int tile = tile0; tile < tile1; ++tile) {
    const int t0 = tile * TILE;
    const int n = min(TILE, p.T - t0);
    {
      int r = threadIdx.x / O, c = threadIdx.x - r * O;
      const int dr = TILE / O, dc = TILE - dr * O;
#pragma unroll 8
      for (int i = threadIdx.x; i < n * O; i += TILE) {
        rows[r * p.pitch + c] = p.logits[(t0 + r) * p.ld + c];
        r += dr;
        c += dc;
        if (c >= O) {
          c -= O;
          ++r;
        }
      }
    }
    __syncthreads();
    const int t = t0 + threadIdx.x;
    const int s = t < p.T && !(p.valid && !p.valid[t]) ? segment_of(p, t) : -1;
    if (s >= 0) {
      const int32_t* cnt = p.counts + static_cast<long long>(s) * E;
      const int nv = p.n_valid[s];
      const int mean_count = static_cast<int>(static_cast<long long>(p.k) * nv / p.n_allowed);
      const float unit = static_cast<float>(per_segment / (static_cast<double>(nv) * nv));  // w_i = unit * c_i
      // groups that keep their experts: of the live ones the top_groups with the
      // largest global logits, ties to the lower index
      uint32_t kept = live;
      if (prune) {
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
        float mx = -INFINITY;
        for (int i = j * gs; i < (j + 1) * gs; ++i)
          if (allowed(p, i)) mx = fmaxf(mx, my[i]);
        float sum = 0.0f, dot = 0.0f;
        for (int i = j * gs; i < (j + 1) * gs; ++i) {
          float e = 0.0f;
          if (allowed(p, i)) {
            e = expf(my[i] - mx);
            sum += e;
            dot = fmaf(e, static_cast<float>(cnt[i] - mean_count), dot);
          }
          my[i] = e;
        }
        inv[j] = 1.0f / sum;
        wbar[j] = dot / sum;
        if (K > 1) top = fmaxf(top, pg[j]);
      }
      float sum = 0.0f, mean = 0.0f;
      for (int j = 0; j < K; ++j) {
        float e = 0.0f;
        if ((kept >> j) & 1u) {
          e = K > 1 ? expf(pg[j] - top) : 1.0f;
          sum += e;
          mean = fmaf(e, wbar[j], mean);
        }
        pg[j] = e;
      }
      const float pinv = 1.0f / sum;
      mean *= pinv;
      loss += static_cast<double>(unit) * (static_cast<double>(mean) + mean_count);
      const float du = unit * upstream;
      for (int j = 0; j < K; ++j) {
        const bool in = (kept >> j) & 1u;
        const float pj = pg[j] * pinv * du;
        const float scale = in ? pj * inv[j] : 0.0f, w = in ? wbar[j] : 0.0f;
        for (int i = j * gs; i < (j + 1) * gs; ++i)
          my[i] = in && allowed(p, i) ? scale * my[i] * (static_cast<float>(cnt[i] - mean_count) - w) : 0.0f;
        if (K > 1) pg[j] = in ? pj * (w - mean) : 0.0f;
      }
    } else if (t < p.T) {
      for (int i = 0; i < O; ++i) my[i] = 0.0f;
    }
    __syncthreads();
    if (p.d_bias) {
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int c = threadIdx.x + u * TILE;
        if (c < O) {
          float v = 0.0f;
          for (int r = 0; r < n; ++r) v += rows[r * p.pitch + c];
          sums[u] += v;
        }
      }
    }
    if (p.d_logits) {
      int r = threadIdx.x / O, c = threadIdx.x - r * O;
      const int dr = TILE / O, dc = TILE - dr * O;
      float* out = p.d_logits + static_cast<long long>(t0) * O;
#pragma unroll 8
      for (int i = threadIdx.x; i < n * O; i += TILE) {
        out[i] = rows[r * p.pitch + c];
        r += dr;
        c += dc;
        if (c >= O) {
          c -= O;
          ++r;
        }
      }
    }
    __syncthreads();
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) loss += __shfl_down_sync(0xffffffffu, loss, o);
  if (threadIdx.x % 32 == 0) warp_loss[threadIdx.x / 32] = loss;
  __syncthreads();
  double* part = p.partial + static_cast<long long>(blockIdx.x) * (O + 1);
  for (int u = 0; u < 2; ++u)
    if (threadIdx.x + u * TILE < O) part[threadIdx.x + u * TILE] = sums[u];
  if (threadIdx.x == 0) {
    double v = 0.0;
    for (int w = 0; w < TILE / 32; ++w) v += warp_loss[w];
    part[O] = v;
  }
}

// One column of the partial sums per warp, added in a fixed order.
__global__ void __launch_bounds__(32) balance_final_kernel(Params p) {
  pdl_trigger();
  pdl_wait();
  const int c = blockIdx.x;
  double v = 0.0;
#pragma unroll 4
  for (int b = threadIdx.x; b < p.n_part; b += 32) v += p.partial[static_cast<long long>(b) * (p.O + 1) + c];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_down_sync(0xffffffffu, v, o);
  if (threadIdx.x == 0) {
    if (c == p.O) *p.loss = static_cast<float>(v);
    else if (p.d_bias) p.d_bias[c] = static_cast<float>(v);
  }
}

int grid_for(int T) {
  const int tiles = (T + TILE - 1) / TILE;
  return tiles < MAX_GRID ? tiles : MAX_GRID;
}

size_t align256(size_t x) { return (x + 255) / 256 * 256; }

}  // namespace

size_t balance_bytes(int T, int E, int K, int n_seg) {
  const int O = E + (K > 1 ? K : 0);
  return align256(static_cast<size_t>(grid_for(T)) * (O + 1) * 8) + align256((static_cast<size_t>(n_seg) + 2) * 4);
}

cudaError_t launch_balance(const BalanceArgs& a, cudaStream_t s) {
  Params p;
  p.logits = a.logits;
  p.ld = a.ld;
  for (int i = 0; i < 4; ++i) p.mask_bits[i] = a.mask_bits[i];
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
  p.ticket = p.n_valid + a.n_seg;
  p.n_live = p.ticket + 1;
  p.n_part = grid;
  p.pitch = (a.E + 3 * a.K) | 1;
  cudaError_t e;
  {
    KernelScope ks("balance_clear", s);
    const long long cells = static_cast<long long>(a.n_seg) * (a.E + 1) + 2;
    const long long blocks = (cells + 255) / 256;
    e = launch_kernel(balance_clear_kernel, dim3(static_cast<unsigned>(blocks < 1024 ? blocks : 1024)), dim3(256), 0, s, p);
    if (e != cudaSuccess) return e;
  }
  if (a.T > 0) {
    {
      KernelScope ks("balance_count", s);
      e = launch_kernel(balance_count_kernel, dim3((a.T + COUNT_TOKENS - 1) / COUNT_TOKENS), dim3(256), 0, s, p);
      if (e != cudaSuccess) return e;
    }
    const int smem = TILE * p.pitch * 4;
    e = ensure_smem_attr(reinterpret_cast<const void*>(balance_main_kernel), smem);
    if (e != cudaSuccess) return e;
    KernelScope ks("balance_main", s);
    e = launch_kernel(balance_main_kernel, dim3(grid), dim3(TILE), (size_t)smem, s, p);
    if (e != cudaSuccess) return e;
  }
  KernelScope ks("balance_final", s);
  e = launch_kernel(balance_final_kernel, dim3(p.O + 1), dim3(32), 0, s, p);
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
