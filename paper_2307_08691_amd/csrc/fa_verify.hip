// Drafted tokens against the target's probabilities. Draft i of a sequence is accepted iff all before it were and
// u_i q_i(x_i) < p_i(x_i). At the first that is not (or has no token) the sequence goes on with a token drawn from max(p_i - q_i, 0),
// behind k accepted ones with one drawn from p_k: the lowest token whose running sum exceeds u_k times the total.
//
// A running sum over 100 000 probabilities passes a random number at another token if it is off by 1e-7, so everything that is
// summed to draw is held in float64, whatever order it is summed in. The target's logits need their normaliser first: row maxima
// and float32 sums over all rows settle which drafts are accepted; the one row that is drawn from is then summed once more in float64.
//
//   stats   (logits) maximum and sum of every row, in chunks of kChunk tokens
//   sums    per sequence: which drafts are accepted; float64 sums of every chunk of the row that is drawn from
//   draw    per sequence: the chunk in which the running sum passes, then the token in it
#include <hip/hip_runtime.h>

#include "../../include/fa.h"
#include "fa_kernels.h"

namespace fa {

constexpr int kChunk = 4096, kVerifyThreads = 256, kPer = kChunk / kVerifyThreads;

struct ChunkSums {
  // p: sum of the row's weights. above, drafts: sums of p and of q over the tokens where p > q. For logits p and above are sums of
  // exp(inv_t (l - maximum)), to be divided by the row's whole sum.
  double p, above, drafts;
};
struct RowPart {
  float max, sum;
};
__host__ __device__ inline int chunks_of(int V) { return (V + kChunk - 1) / kChunk; }

size_t verify_workspace(int B, int k, int V) {
  return (size_t)B * chunks_of(V) * (sizeof(ChunkSums) + (size_t)(k + 1) * sizeof(RowPart));
}
__device__ __forceinline__ ChunkSums* chunk_sums(const VerifyArgs& a, int b) { return (ChunkSums*)a.ws + (long)b * chunks_of(a.V); }
__device__ __forceinline__ RowPart* row_parts(const VerifyArgs& a, long row) {
  const int n = chunks_of(a.V);
  return (RowPart*)((ChunkSums*)a.ws + (long)a.nseq * n) + row * n;
}

__device__ __forceinline__ float element(const void* p, int type, long i) {
  if (type == FA_TYPE_F32) return ((const float*)p)[i];
  if (type == FA_TYPE_BF16) return (float)((const __bf16*)p)[i];
  return (float)((const _Float16*)p)[i];
}

template <class T>
__device__ __forceinline__ T block_reduce(T x, T* lds, T (*op)(T, T)) {  // the same value in every thread
  for (int o = 32; o; o >>= 1) x = op(x, __shfl_xor(x, o));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = x;
  __syncthreads();
  x = lds[0];
  for (int i = 1; i < kVerifyThreads / 64; ++i) x = op(x, lds[i]);
  return x;
}
template <class T>
__device__ T add(T a, T b) {
  return a + b;
}
__device__ float larger(float a, float b) { return fmaxf(a, b); }

__global__ __launch_bounds__(kVerifyThreads) void verify_stats_kernel(VerifyArgs a) {
  __shared__ float lds[kVerifyThreads / 64];
  const long row = blockIdx.x;
  const int c0 = blockIdx.y * kChunk, end = a.V < c0 + kChunk ? a.V : c0 + kChunk;
  const float t2 = a.inv_t * kLog2e;
  float x[kPer], m = -INFINITY;
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int j = c0 + i * kVerifyThreads + threadIdx.x;
    x[i] = j < end ? element(a.target, a.target_type, row * a.target_stride + j) : -INFINITY;
    m = fmaxf(m, x[i]);
  }
  m = block_reduce(m, lds, larger);
  float z = 0.f;
#pragma unroll
  for (int i = 0; i < kPer; ++i) z += x[i] == -INFINITY ? 0.f : fast_exp2((x[i] - m) * t2);
  z = block_reduce(z, lds, add<float>);
  if (threadIdx.x == 0) row_parts(a, row)[blockIdx.y] = {m, z};
}

// Maximum of a row, and its sum against it.
__device__ __forceinline__ RowPart whole_row(const VerifyArgs& a, long row) {
  const RowPart* part = row_parts(a, row);
  const int n = chunks_of(a.V), lane = threadIdx.x & 63;
  float m = -INFINITY, z = 0.f;
  for (int i = lane; i < n; i += 64) m = fmaxf(m, part[i].max);
  for (int o = 32; o; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
  for (int i = lane; i < n; i += 64) z += part[i].max == -INFINITY ? 0.f : part[i].sum * fast_exp2((part[i].max - m) * a.inv_t * kLog2e);
  for (int o = 32; o; o >>= 1) z += __shfl_xor(z, o);
  return {m, z};
}
// exp(inv_t (l - m)) in float64
__device__ __forceinline__ double weight_of(const VerifyArgs& a, float l, float m) {
  return l == -INFINITY ? 0. : exp((double)a.inv_t * ((double)l - (double)m));
}
__device__ __forceinline__ int draft_token(const VerifyArgs& a, long b, int i) {  // -1: none
  const int x = a.drafts[b * a.k + i];
  return x >= 0 && x < a.V ? x : -1;
}
// How many drafts of sequence b are accepted; `r`: the row that its next token is drawn from.
__device__ __forceinline__ int accepted_drafts(const VerifyArgs& a, long b, RowPart& r) {
  for (int i = 0; i <= a.k; ++i) {
    const long row = b * (a.k + 1) + i;
    r = {0.f, 1.f};
    if (a.logits) r = whole_row(a, row);
    if (i == a.k) break;
    const int x = draft_token(a, b, i);
    if (x < 0) return i;
    const float l = element(a.target, a.target_type, row * a.target_stride + x);
    const double p = a.logits ? weight_of(a, l, r.max) / (double)r.sum : (double)l;
    const double q = a.q ? (double)element(a.q, a.q_type, (b * a.k + i) * a.q_stride + x) : 1.;
    if (!((double)a.uniform[b * (a.k + 1) + i] * q < p)) return i;
  }
  return a.k;
}
// What the draft model gave token j of row (b, i); 0 where nothing is to be taken off.
struct DraftRow {
  const void* q;
  int type, token;  // q == nullptr: all on `token` (-1: nothing)
  long at;
  __device__ __forceinline__ double of(int j) const { return q ? (double)element(q, type, at + j) : (j == token ? 1. : 0.); }
};
__device__ __forceinline__ DraftRow draft_row(const VerifyArgs& a, long b, int i) {
  const int x = i < a.k ? draft_token(a, b, i) : -1;
  if (x < 0 || !a.q) return {nullptr, 0, x, 0};
  return {a.q, a.q_type, x, (b * a.k + i) * a.q_stride};
}

__global__ __launch_bounds__(kVerifyThreads) void verify_sums_kernel(VerifyArgs a) {
  __shared__ double lds[kVerifyThreads / 64];
  const long b = blockIdx.x;
  RowPart r;
  const int i = accepted_drafts(a, b, r);
  const DraftRow q = draft_row(a, b, i);
  const long at = (b * (a.k + 1) + i) * a.target_stride;
  const int c0 = blockIdx.y * kChunk, end = a.V < c0 + kChunk ? a.V : c0 + kChunk;
  const double inv = a.logits ? 1. / (double)r.sum : 1.;
  double sp = 0., sa = 0., sq = 0.;
  for (int j = c0 + threadIdx.x; j < end; j += kVerifyThreads) {
    const float l = element(a.target, a.target_type, at + j);
    const double p = a.logits ? weight_of(a, l, r.max) : (double)l, d = q.of(j);
    sp += p;
    // (r.sum is good to 1e-7: a token at which that decides has p = q to within it, and adds as little either way)
    if (p * inv > d) sa += p, sq += d;
  }
  sp = block_reduce(sp, lds, add<double>);
  sa = block_reduce(sa, lds, add<double>);
  sq = block_reduce(sq, lds, add<double>);
  if (threadIdx.x == 0) chunk_sums(a, b)[blockIdx.y] = {sp, sa, sq};
  if (blockIdx.y == 0) {  // the tokens so far
    if (threadIdx.x == 0) a.accepted[b] = i;
    for (int j = threadIdx.x; j <= a.k; j += kVerifyThreads) a.tokens[b * (a.k + 1) + j] = j < i ? a.drafts[b * a.k + j] : -1;
  }
}

__global__ __launch_bounds__(kVerifyThreads) void verify_draw_kernel(VerifyArgs a) {
  __shared__ double lds[kVerifyThreads / 64];
  __shared__ double before[kVerifyThreads];
  __shared__ int last[kVerifyThreads / 64];
  const long b = blockIdx.x;
  const int tid = threadIdx.x, nc = chunks_of(a.V), i = a.accepted[b];
  const long row = b * (a.k + 1) + i;
  const DraftRow q = draft_row(a, b, i);
  const ChunkSums* part = chunk_sums(a, b);
  // the row's sum, and whether p - q leaves anything
  double z = 0., above = 0., off = 0.;
  for (int c = tid; c < nc; c += kVerifyThreads) z += part[c].p, above += part[c].above, off += part[c].drafts;
  z = block_reduce(z, lds, add<double>);
  above = block_reduce(above, lds, add<double>);
  off = block_reduce(off, lds, add<double>);
  const double inv = a.logits ? 1. / z : 1.;
  const bool residual = above * inv - off > 0.;
  const double total = residual ? above * inv - off : z * inv, want = (double)a.uniform[b * (a.k + 1) + a.k] * total;
  // the first chunk whose end lies past `want`, or else the last one that adds anything
  auto chunk_sum = [&](int c) { return residual ? part[c].above * inv - part[c].drafts : part[c].p * inv; };
  int chunk = -1;
  double sum = 0., base = 0.;
  for (int c = 0; c < nc; ++c) {
    const double x = chunk_sum(c);
    if (x > 0.) chunk = c, base = sum;
    sum += x;
    if (chunk == c && sum > want) break;
  }
  if (chunk < 0) return;  // (nothing to draw from: the token stays -1)
  RowPart r = {0.f, 1.f};
  if (a.logits) r = whole_row(a, row);
  auto weight = [&](int j) {
    const float l = element(a.target, a.target_type, row * a.target_stride + j);
    const double p = (a.logits ? weight_of(a, l, r.max) : (double)l) * inv, d = residual ? q.of(j) : 0.;
    return p > d ? p - d : 0.;
  };
  // each thread: kPer tokens that follow each other
  const int j0 = chunk * kChunk + tid * kPer;
  double x[kPer], mine = 0.;
  int some = -1;  // the last one that adds anything
#pragma unroll
  for (int u = 0; u < kPer; ++u) {
    x[u] = j0 + u < a.V ? weight(j0 + u) : 0.;
    mine += x[u];
    if (x[u] > 0.) some = j0 + u;
  }
  before[tid] = mine;
  for (int o = 32; o; o >>= 1) some = max(some, __shfl_xor(some, o));
  if ((tid & 63) == 0) last[tid >> 6] = some;
  __syncthreads();
  for (int w = 0; w < kVerifyThreads / 64; ++w) some = max(some, last[w]);
  double run = base;
  for (int t = 0; t < tid; ++t) run += before[t];
  int hit = 0x7fffffff;
#pragma unroll
  for (int u = 0; u < kPer; ++u) {
    run += x[u];
    if (x[u] > 0. && run > want && hit == 0x7fffffff) hit = j0 + u;
  }
  for (int o = 32; o; o >>= 1) hit = min(hit, __shfl_xor(hit, o));
  __syncthreads();
  if ((tid & 63) == 0) last[tid >> 6] = hit;
  __syncthreads();
  if (tid == 0) {
    for (int w = 1; w < kVerifyThreads / 64; ++w) hit = min(hit, last[w]);
    a.tokens[row] = hit != 0x7fffffff ? hit : some;
  }
}

hipError_t launch_verify(const VerifyArgs& a, hipStream_t st) {
  const unsigned chunks = (unsigned)chunks_of(a.V);
  if (a.logits) {
    hipLaunchKernelGGL(verify_stats_kernel, dim3((unsigned)(a.nseq * (a.k + 1)), chunks), dim3(kVerifyThreads), 0, st, a);
    if (hipError_t e = hipGetLastError()) return e;
  }
  hipLaunchKernelGGL(verify_sums_kernel, dim3((unsigned)a.nseq, chunks), dim3(kVerifyThreads), 0, st, a);
  if (hipError_t e = hipGetLastError()) return e;
  hipLaunchKernelGGL(verify_draw_kernel, dim3((unsigned)a.nseq), dim3(kVerifyThreads), 0, st, a);
  return hipGetLastError();
}

}  // namespace fa
