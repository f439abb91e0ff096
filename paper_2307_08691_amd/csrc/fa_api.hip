// C ABI of the attention library: argument validation, workspace carving, launches.
#include "../../include/fa.h"
#include "fa_kernels.h"

#include <atomic>
#include <cmath>
#include <cstdlib>

// Scratch of fa_bwd_noalloc: D = rowsum(dO o O) for up to FA_NOALLOC_MAX_ROWS (query row, head)
// pairs, and behind it the most that shares of blocks of keys leave (d = 128). Every GPU the library runs on holds its own copy of this array, at its own address,
// until the process ends. In host code the name below is only a handle for hipGetSymbolAddress.
constexpr size_t kScratchFloats = FA_NOALLOC_MAX_ROWS + (size_t)fa::kShareRows * 2 * 128;
static __device__ __align__(256) float scratch[kScratchFloats];

namespace {

// device address of `scratch` on each GPU, looked up once per device
constexpr int kMaxDevices = 64;
std::atomic<float*> g_scratch[kMaxDevices];

// 0 and the address, or a negative status (and the HIP error kept for fa_last_hip_error)
int scratch_on_current_device(float** out, int* hip_error) {
  int dev = -1;
  hipError_t e = hipGetDevice(&dev);
  if (e == hipSuccess && (dev < 0 || dev >= kMaxDevices)) e = hipErrorInvalidDevice;
  if (e == hipSuccess) {
    float* p = g_scratch[dev].load(std::memory_order_acquire);
    if (!p) {  // first call on this device (two threads racing here look up the same address)
      void* sym = nullptr;
      e = hipGetSymbolAddress(&sym, HIP_SYMBOL(scratch));
      if (e == hipSuccess && !sym) e = hipErrorInvalidSymbol;
      if (e == hipSuccess) {
        p = (float*)sym;
        g_scratch[dev].store(p, std::memory_order_release);
      }
    }
    if (e == hipSuccess) {
      *out = p;
      return FA_OK;
    }
  }
  *hip_error = (int)e;
  return FA_ERR_LAUNCH;
}

thread_local int g_last_hip_error = 0;

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline size_t round_up(size_t x, size_t a) { return (x + a - 1) / a * a; }

// any_d: the entry point also takes head dimensions that the kernels pad on chip
// (multiples of 8 up to 128) and 256, which has kernels of its own; otherwise only the two
// tile widths 64 and 128 themselves.
int check_common(int Hq, int Hkv, int d, float scale, bool any_d = true) {
  if (Hq <= 0 || Hkv <= 0 || d <= 0) return FA_ERR_SHAPE;
  if (Hq % Hkv != 0) return FA_ERR_SHAPE;
  if (!(scale > 0.f) || !std::isfinite(scale)) return FA_ERR_SHAPE;
  if (any_d ? ((d % 8 != 0 || d > 128) && d != 256) : (d != 64 && d != 128)) return FA_ERR_UNSUPPORTED;
  return FA_OK;
}

fa::Problem make_problem(const int32_t* cu, int nseq, int N, int Nk, int Hq, int Hkv, int d, long total, float scale,
                         const int32_t* cu_k = nullptr, int f16 = 0) {
  fa::Problem p;
  p.d = d;
  p.f16 = f16;
  p.drop_thr = 0;
  p.drop_seed = 0;
  p.drop_rp = 1.f;
  p.drop_log2 = 0.f;
  p.mask = nullptr;
  p.mask_bs = p.mask_hs = p.mask_rs = 0;
  p.win_left = p.win_right = -1;
  p.bmask = nullptr;
  p.bmask_bs = p.bmask_hs = 0;
  p.bmask_cols = p.bmask_log2 = 0;
  p.cu_seqlens = cu;
  p.cu_seqlens_k = cu_k;
  p.nseq = nseq;
  p.N = N;
  p.Nk = Nk;
  p.Hq = Hq;
  p.Hkv = Hkv;
  p.G = Hq / Hkv;
  p.total_tokens = (int)total;
  p.lse_seq_stride = cu ? 0 : (long)Hq * N;
  p.lse_head_stride = cu ? total : N;
  p.scale = scale;
  p.scale_log2e = scale * fa::kLog2e;
  return p;
}

size_t ws_bytes(long tokens, int Hq) {
  return round_up((size_t)tokens * Hq * sizeof(float), 256);  // D = rowsum(dO o O)
}
// ... and behind it, where blocks of keys may be taken in shares, the shares' sums of dK and dV
size_t ws_bytes(long tokens, int Hq, int Hkv, int d, long nq, long key_rows) {
  return ws_bytes(tokens, Hq) + (d > 128 ? 0 : round_up((size_t)fa::share_rows(key_rows, Hq, Hkv, nq) * d * 2 * sizeof(float), 256));
}

// dropout: threshold round(256 p) in 0 .. 255 (0: nothing is dropped) and the mixed seed
int set_dropout(fa::Problem& p, float p_drop, uint64_t seed) {
  if (!(p_drop >= 0.f) || !(p_drop < 1.f)) return FA_ERR_SHAPE;
  long t = std::lround(256.0 * (double)p_drop);
  if (t > 255) t = 255;
  p.drop_thr = (uint32_t)t;
  p.drop_seed = (uint32_t)seed ^ ((uint32_t)(seed >> 32) * 0x27D4EB2Fu);
  p.drop_rp = 256.f / (256.f - (float)t);
  p.drop_log2 = 8.f - log2f(256.f - (float)t);
  return FA_OK;
}

// elementwise mask: strides in elements, multiples of 8 (every 16-byte chunk of M aligned)
int set_mask(fa::Problem& p, const void* M, int Nk, long long bs, long long hs, long long rs) {
  if (!M) return FA_ERR_NULL;
  if (!aligned16(M)) return FA_ERR_ALIGN;
  if (bs < 0 || hs < 0 || rs < (((long long)Nk + 7) & ~7LL)) return FA_ERR_SHAPE;
  if (bs % 8 || hs % 8 || rs % 8) return FA_ERR_SHAPE;
  p.mask = (const __bf16*)M;
  p.mask_bs = (long)bs;
  p.mask_hs = (long)hs;
  p.mask_rs = (long)rs;
  return FA_OK;
}

// What an entry point may ask for beyond the plain pass.
struct Options {
  int f16 = 0;                      // element type: 0 bfloat16, 1 IEEE half precision
  bool dropout = false;             // dropout on P with p_drop, seed
  float p_drop = 0.f;
  uint64_t seed = 0;
  bool mask = false;                // elementwise mask M with its three strides
  const void* M = nullptr;
  long long mask_bs = 0, mask_hs = 0, mask_rs = 0;
  bool window = false;              // sliding window (win_left, win_right); a negative bound is no bound
  int win_left = -1, win_right = -1;
  const void* bmask = nullptr;      // block-sparse pattern (with window = true): bytes, two strides, block size
  long long bmask_bs = 0, bmask_hs = 0;
  int block = 0;
  const int32_t* seqlens_k = nullptr;    // key/value cache (split forward only): per-sequence lengths,
  const int32_t* block_table = nullptr;  // page table with its row stride, log2 of the page size
  int page_log2 = 0, table_stride = 0;
  void* dM = nullptr;                    // masked backward: where the gradient of the mask goes, with its strides
  long long dm_bs = 0, dm_hs = 0, dm_rs = 0;
  bool keep_d = false;                   // backward: D has to be in the workspace afterwards (fa_bwd_stages)
};

Options half_precision(int f16) {
  Options o;
  o.f16 = f16;
  return o;
}
Options of_type(Options o, int f16) {
  o.f16 = f16;
  return o;
}
Options with_dropout(float p_drop, uint64_t seed) {
  Options o;
  o.dropout = true;
  o.p_drop = p_drop;
  o.seed = seed;
  return o;
}
Options with_mask(const void* M, long long bs, long long hs, long long rs) {
  Options o;
  o.mask = true;
  o.M = M;
  o.mask_bs = bs;
  o.mask_hs = hs;
  o.mask_rs = rs;
  return o;
}

Options with_window(int left, int right) {
  Options o;
  o.window = true;
  o.win_left = left < 0 ? -1 : left;
  o.win_right = right < 0 ? -1 : right;
  return o;
}

// block-sparse pattern: block a power of two >= 64; the wavefronts' activity bitmaps hold
// kPatternWords * 64 key blocks (forward, dQ) and row tiles (dK/dV: tiles of 32 rows, one per
// query head of a group)
int set_block_pattern(fa::Problem& p, const Options& o) {
  if (!o.bmask) return FA_ERR_NULL;
  if (o.block < 64 || (o.block & (o.block - 1)) || o.bmask_bs < 0 || o.bmask_hs < 0) return FA_ERR_SHAPE;
  const long words = 64L * fa::kPatternWords;
  if (((long)p.Nk + 63) / 64 > words || (((long)p.N + 31) / 32) * p.G > words) return FA_ERR_UNSUPPORTED;
  p.bmask = (const uint8_t*)o.bmask;
  p.bmask_bs = (long)o.bmask_bs;
  p.bmask_hs = (long)o.bmask_hs;
  p.bmask_cols = (p.Nk + o.block - 1) / o.block;
  p.bmask_log2 = __builtin_ctz((unsigned)o.block);
  return FA_OK;
}

int apply_options(fa::Problem& p, const Options& o) {
  if (o.window) {
    p.win_left = o.win_left;
    p.win_right = o.win_right;
    if (o.block)
      if (int e = set_block_pattern(p, o)) return e;
  }
  if (o.dropout)
    if (int e = set_dropout(p, o.p_drop, o.seed)) return e;
  if (o.mask)
    if (int e = set_mask(p, o.M, p.Nk, o.mask_bs, o.mask_hs, o.mask_rs)) return e;
  return FA_OK;
}

int run_fwd(const void* Q, const void* K, const void* V, void* O, float* LSE, const int32_t* cu, int nseq, int N,
            int Nk, long total, int Hq, int Hkv, int d, float scale, int causal, void* stream, int nsplit = 0,
            void* ws = nullptr, const int32_t* cu_k = nullptr, const Options& opt = Options()) {
  fa::FwdArgs a;
  a.nsplit = nsplit;
  a.Opart = (float*)ws;  // [nsplit, tokens, Hq, d], then the partial logsumexps [nsplit, B, Hq, Nq]
  a.Lpart = ws ? (float*)ws + (size_t)nsplit * total * Hq * d : nullptr;
  a.p = make_problem(cu, nseq, N, Nk, Hq, Hkv, d, total, scale, cu_k, opt.f16);
  if (int e = apply_options(a.p, opt)) return e;
  a.seqlens_k = opt.seqlens_k;
  a.block_table = opt.block_table;
  a.page_log2 = opt.page_log2;
  a.table_stride = opt.table_stride;
  a.Q = (const __bf16*)Q;
  a.K = (const __bf16*)K;
  a.V = (const __bf16*)V;
  a.O = (__bf16*)O;
  a.LSE = LSE;
  hipError_t e = fa::launch_fwd(a, d, causal, (hipStream_t)stream);
  if (e != hipSuccess) {
    g_last_hip_error = (int)e;
    return FA_ERR_LAUNCH;
  }
  return FA_OK;
}

int run_bwd(const void* Q, const void* K, const void* V, const void* O, const void* dO, const float* LSE, void* dQ,
            void* dK, void* dV, void* ws, size_t ws_size, const int32_t* cu, int nseq, int N, int Nk, long total, int Hq, int Hkv, int d,
            float scale, int causal, int stages, void* stream, const int32_t* cu_k = nullptr,
            const Options& opt = Options(), long total_k = 0) {
  fa::BwdArgs a;
  a.p = make_problem(cu, nseq, N, Nk, Hq, Hkv, d, total, scale, cu_k, opt.f16);
  if (int e = apply_options(a.p, opt)) return e;
  a.Q = (const __bf16*)Q;
  a.K = (const __bf16*)K;
  a.V = (const __bf16*)V;
  a.O = (const __bf16*)O;
  a.dO = (const __bf16*)dO;
  a.LSE = LSE;
  a.dQ = (__bf16*)dQ;
  a.dK = (__bf16*)dK;
  a.dV = (__bf16*)dV;
  a.Dvec = (float*)ws;
  a.keep_d = opt.keep_d;
  a.shares = 1;
  a.share_turn = 0;
  a.key_rows = cu_k ? total_k : cu ? total : (long)nseq * Nk;
  // (a workspace that holds D alone is enough for the backward without shares)
  a.partial = d <= 128 && !cu_k && ws_size >= ws_bytes(total, Hq, Hkv, d, N, a.key_rows) ? (float*)((char*)ws + ws_bytes(total, Hq)) : nullptr;
  a.dM = (__bf16*)opt.dM;
  a.dm_bs = (long)opt.dm_bs;
  a.dm_hs = (long)opt.dm_hs;
  a.dm_rs = (long)opt.dm_rs;
  hipError_t e = fa::launch_bwd(a, d, causal, stages, (hipStream_t)stream);
  if (e != hipSuccess) {
    g_last_hip_error = (int)e;
    return FA_ERR_LAUNCH;
  }
  return FA_OK;
}

}  // namespace

extern "C" {

int fa_version(void) { return 100; }

const char* fa_status_string(int status) {
  switch (status) {
    case FA_OK: return "ok";
    case FA_ERR_NULL: return "a required pointer is NULL";
    case FA_ERR_SHAPE: return "invalid shape, head grouping, scale or ragged description";
    case FA_ERR_UNSUPPORTED:
      return "unsupported head dimension (multiples of 8 up to 128; dropout, mask and split keys: 64 and 128 only)";
    case FA_ERR_ALIGN: return "a tensor pointer is not 16-byte aligned";
    case FA_ERR_WORKSPACE:
      return "workspace too small (fa_bwd_noalloc: more than FA_NOALLOC_MAX_ROWS (query row, head) pairs)";
    case FA_ERR_LAUNCH: return "the HIP runtime refused a kernel launch";
    default: return "unknown status";
  }
}

int fa_last_hip_error(void) { return g_last_hip_error; }

int fa_fwd(const void* Q, const void* K, const void* V, void* O, float* LSE, int B, int Hq, int Hkv, int N, int d,
           float scale, int causal, void* stream) {
  if (!Q || !K || !V || !O || !LSE) return FA_ERR_NULL;
  if (B <= 0 || N <= 0) return FA_ERR_SHAPE;
  if (int e = check_common(Hq, Hkv, d, scale)) return e;
  if ((long)B * N > 0x7fffffffL) return FA_ERR_SHAPE;
  if (!aligned16(Q) || !aligned16(K) || !aligned16(V) || !aligned16(O) || !aligned16(LSE)) return FA_ERR_ALIGN;
  return run_fwd(Q, K, V, O, LSE, nullptr, B, N, N, (long)B * N, Hq, Hkv, d, scale, causal, stream);
}

size_t fa_bwd_workspace_bytes(int B, int Hq, int Hkv, int N, int d) {
  if (B <= 0 || Hq <= 0 || N <= 0 || d <= 0) return 0;
  return ws_bytes((long)B * N, Hq, Hkv, d, N, (long)B * N);
}

static int dense_bwd(const void* Q, const void* K, const void* V, const void* O, const void* dO, const float* LSE,
                     void* dQ, void* dK, void* dV, void* workspace, size_t workspace_bytes, int B, int Hq, int Hkv, int N,
                     int d, float scale, int causal, int stages, void* stream, const Options& opt = Options()) {
  if (!Q || !K || !V || !O || !dO || !LSE || !dQ || !dK || !dV || !workspace) return FA_ERR_NULL;
  if (B <= 0 || N <= 0) return FA_ERR_SHAPE;
  if (int e = check_common(Hq, Hkv, d, scale)) return e;
  if ((long)B * N > 0x7fffffffL) return FA_ERR_SHAPE;
  if (!aligned16(Q) || !aligned16(K) || !aligned16(V) || !aligned16(O) || !aligned16(dO) || !aligned16(LSE) ||
      !aligned16(dQ) || !aligned16(dK) || !aligned16(dV) || !aligned16(workspace))
    return FA_ERR_ALIGN;
  if (workspace_bytes < ws_bytes((long)B * N, Hq)) return FA_ERR_WORKSPACE;
  if (stages <= 0 || (stages & ~7)) return FA_ERR_SHAPE;
  return run_bwd(Q, K, V, O, dO, LSE, dQ, dK, dV, workspace, workspace_bytes, nullptr, B, N, N, (long)B * N, Hq, Hkv, d, scale, causal,
                 stages, stream, nullptr, opt);
}

int fa_bwd_stages(const void* Q, const void* K, const void* V, const void* O, const void* dO, const float* LSE,
                  void* dQ, void* dK, void* dV, void* workspace, size_t workspace_bytes, int B, int Hq, int Hkv, int N,
                  int d, float scale, int causal, int stages, void* stream) {
  Options opt;
  opt.keep_d = true;
  return dense_bwd(Q, K, V, O, dO, LSE, dQ, dK, dV, workspace, workspace_bytes, B, Hq, Hkv, N, d, scale, causal, stages,
                   stream, opt);
}

int fa_bwd(const void* Q, const void* K, const void* V, const void* O, const void* dO, const float* LSE, void* dQ,
           void* dK, void* dV, void* workspace, size_t workspace_bytes, int B, int Hq, int Hkv, int N, int d,
           float scale, int causal, void* stream) {
  return dense_bwd(Q, K, V, O, dO, LSE, dQ, dK, dV, workspace, workspace_bytes, B, Hq, Hkv, N, d, scale, causal,
                   FA_STAGE_PREP | FA_STAGE_DKDV | FA_STAGE_DQ, stream);
}

int fa_bwd_noalloc(const void* Q, const void* K, const void* V, const void* O, const void* dO, const float* LSE,
                   void* dQ, void* dK, void* dV, int B, int Hq, int Hkv, int N, int d, float scale, int causal,
                   void* stream) {
  // sizes first: a problem that does not fit the static array is refused before anything else happens
  if (B > 0 && Hq > 0 && N > 0 && (long long)B * N * Hq > (long long)FA_NOALLOC_MAX_ROWS) return FA_ERR_WORKSPACE;
  float* ws = nullptr;
  if (int e = scratch_on_current_device(&ws, &g_last_hip_error)) return e;
  return dense_bwd(Q, K, V, O, dO, LSE, dQ, dK, dV, ws, sizeof(float) * kScratchFloats, B, Hq, Hkv, N, d,
                   scale, causal, FA_STAGE_PREP | FA_STAGE_DKDV | FA_STAGE_DQ, stream);
}

static int check_varlen(const int32_t* cu, int nseq, int total_tokens, int max_seqlen) {
  if (!cu) return FA_ERR_NULL;
  if (nseq <= 0 || total_tokens <= 0 || max_seqlen <= 0) return FA_ERR_SHAPE;
  if (max_seqlen > total_tokens) return FA_ERR_SHAPE;
  if ((long)max_seqlen * nseq < (long)total_tokens) return FA_ERR_SHAPE;  // lengths cannot add up
  return FA_OK;
}

static int varlen_fwd(const void* Q, const void* K, const void* V, void* O, float* LSE, const int32_t* cu_seqlens,
                      int nseq, int total_tokens, int max_seqlen, int Hq, int Hkv, int d, float scale, int causal,
                      void* stream, const Options& opt) {
  if (!Q || !K || !V || !O || !LSE) return FA_ERR_NULL;
  if (int e = check_varlen(cu_seqlens, nseq, total_tokens, max_seqlen)) return e;
  if (int e = check_common(Hq, Hkv, d, scale, !(opt.dropout || opt.window))) return e;
  if (!aligned16(Q) || !aligned16(K) || !aligned16(V) || !aligned16(O) || !aligned16(LSE)) return FA_ERR_ALIGN;
  return run_fwd(Q, K, V, O, LSE, cu_seqlens, nseq, max_seqlen, max_seqlen, total_tokens, Hq, Hkv, d, scale, causal,
                 stream, 0, nullptr, nullptr, opt);
}

static int varlen_fwd_any(int f16, const void* Q, const void* K, const void* V, void* O, float* LSE,
                          const int32_t* cu_seqlens, int nseq, int total_tokens, int max_seqlen, int Hq, int Hkv,
                          int d, float scale, int causal, void* stream) {
  return varlen_fwd(Q, K, V, O, LSE, cu_seqlens, nseq, total_tokens, max_seqlen, Hq, Hkv, d, scale, causal, stream,
                    half_precision(f16));
}

int fa_varlen_fwd(const void* Q, const void* K, const void* V, void* O, float* LSE, const int32_t* cu_seqlens,
                  int nseq, int total_tokens, int max_seqlen, int Hq, int Hkv, int d, float scale, int causal,
                  void* stream) {
  return varlen_fwd_any(0, Q, K, V, O, LSE, cu_seqlens, nseq, total_tokens, max_seqlen, Hq, Hkv, d, scale, causal,
                        stream);
}

int fa_varlen_fwd_f16(const void* Q, const void* K, const void* V, void* O, float* LSE, const int32_t* cu_seqlens,
                      int nseq, int total_tokens, int max_seqlen, int Hq, int Hkv, int d, float scale, int causal,
                      void* stream) {
  return varlen_fwd_any(1, Q, K, V, O, LSE, cu_seqlens, nseq, total_tokens, max_seqlen, Hq, Hkv, d, scale, causal,
                        stream);
}

static int varlen_dropout_fwd_any(int f16, const void* Q, const void* K, const void* V, void* O, float* LSE,
                                  const int32_t* cu_seqlens, int nseq, int total_tokens, int max_seqlen, int Hq,
                                  int Hkv, int d, float scale, int causal, float p_drop, uint64_t seed,
                                  void* stream) {
  return varlen_fwd(Q, K, V, O, LSE, cu_seqlens, nseq, total_tokens, max_seqlen, Hq, Hkv, d, scale, causal, stream,
                    of_type(with_dropout(p_drop, seed), f16));
}

int fa_varlen_dropout_fwd(const void* Q, const void* K, const void* V, void* O, float* LSE, const int32_t* cu_seqlens,
                          int nseq, int total_tokens, int max_seqlen, int Hq, int Hkv, int d, float scale, int causal,
                          float p_drop, uint64_t seed, void* stream) {
  return varlen_dropout_fwd_any(0, Q, K, V, O, LSE, cu_seqlens, nseq, total_tokens, max_seqlen, Hq, Hkv, d, scale,
                                causal, p_drop, seed, stream);
}

int fa_varlen_dropout_fwd_f16(const void* Q, const void* K, const void* V, void* O, float* LSE,
                              const int32_t* cu_seqlens, int nseq, int total_tokens, int max_seqlen, int Hq, int Hkv,
                              int d, float scale, int causal, float p_drop, uint64_t seed, void* stream) {
  return varlen_dropout_fwd_any(1, Q, K, V, O, LSE, cu_seqlens, nseq, total_tokens, max_seqlen, Hq, Hkv, d, scale,
                                causal, p_drop, seed, stream);
}

size_t fa_varlen_bwd_workspace_bytes(int total_tokens, int Hq, int Hkv, int d) {
  if (total_tokens <= 0 || Hq <= 0 || d <= 0) return 0;
  return ws_bytes(total_tokens, Hq, Hkv, d, total_tokens, total_tokens);
}

static int varlen_bwd(const void* Q, const void* K, const void* V, const void* O, const void* dO, const float* LSE,
                      void* dQ, void* dK, void* dV, void* workspace, size_t workspace_bytes,
                      const int32_t* cu_seqlens, int nseq, int total_tokens, int max_seqlen, int Hq, int Hkv, int d,
                      float scale, int causal, void* stream, const Options& opt) {
  if (!Q || !K || !V || !O || !dO || !LSE || !dQ || !dK || !dV || !workspace) return FA_ERR_NULL;
  if (int e = check_varlen(cu_seqlens, nseq, total_tokens, max_seqlen)) return e;
  if (int e = check_common(Hq, Hkv, d, scale, !(opt.dropout || opt.window))) return e;
  if (!aligned16(Q) || !aligned16(K) || !aligned16(V) || !aligned16(O) || !aligned16(dO) || !aligned16(LSE) ||
      !aligned16(dQ) || !aligned16(dK) || !aligned16(dV) || !aligned16(workspace))
    return FA_ERR_ALIGN;
  if (workspace_bytes < ws_bytes(total_tokens, Hq)) return FA_ERR_WORKSPACE;
  return run_bwd(Q, K, V, O, dO, LSE, dQ, dK, dV, workspace, workspace_bytes, cu_seqlens, nseq, max_seqlen, max_seqlen, total_tokens, Hq,
                 Hkv, d, scale, causal, 7, stream, nullptr, opt);
}

static int varlen_bwd_any(int f16, const void* Q, const void* K, const void* V, const void* O, const void* dO,
                          const float* LSE, void* dQ, void* dK, void* dV, void* workspace, size_t workspace_bytes,
                          const int32_t* cu_seqlens, int nseq, int total_tokens, int max_seqlen, int Hq, int Hkv,
                          int d, float scale, int causal, void* stream) {
  return varlen_bwd(Q, K, V, O, dO, LSE, dQ, dK, dV, workspace, workspace_bytes, cu_seqlens, nseq, total_tokens,
                    max_seqlen, Hq, Hkv, d, scale, causal, stream, half_precision(f16));
}

int fa_varlen_bwd(const void* Q, const void* K, const void* V, const void* O, const void* dO, const float* LSE,
                  void* dQ, void* dK, void* dV, void* workspace, size_t workspace_bytes, const int32_t* cu_seqlens,
                  int nseq, int total_tokens, int max_seqlen, int Hq, int Hkv, int d, float scale, int causal,
                  void* stream) {
  return varlen_bwd_any(0, Q, K, V, O, dO, LSE, dQ, dK, dV, workspace, workspace_bytes, cu_seqlens, nseq,
                        total_tokens, max_seqlen, Hq, Hkv, d, scale, causal, stream);
}

int fa_varlen_bwd_f16(const void* Q, const void* K, const void* V, const void* O, const void* dO, const float* LSE,
                      void* dQ, void* dK, void* dV, void* workspace, size_t workspace_bytes,
                      const int32_t* cu_seqlens, int nseq, int total_tokens, int max_seqlen, int Hq, int Hkv, int d,
                      float scale, int causal, void* stream) {
  return varlen_bwd_any(1, Q, K, V, O, dO, LSE, dQ, dK, dV, workspace, workspace_bytes, cu_seqlens, nseq,
                        total_tokens, max_seqlen, Hq, Hkv, d, scale, causal, stream);
}

static int varlen_dropout_bwd_any(int f16, const void* Q, const void* K, const void* V, const void* O, const void* dO,
                                  const float* LSE, void* dQ, void* dK, void* dV, void* workspace,
                                  size_t workspace_bytes, const int32_t* cu_seqlens, int nseq, int total_tokens,
                                  int max_seqlen, int Hq, int Hkv, int d, float scale, int causal, float p_drop,
                                  uint64_t seed, void* stream) {
  return varlen_bwd(Q, K, V, O, dO, LSE, dQ, dK, dV, workspace, workspace_bytes, cu_seqlens, nseq, total_tokens,
                    max_seqlen, Hq, Hkv, d, scale, causal, stream, of_type(with_dropout(p_drop, seed), f16));
}

int fa_varlen_dropout_bwd(const void* Q, const void* K, const void* V, const void* O, const void* dO,
                          const float* LSE, void* dQ, void* dK, void* dV, void* workspace, size_t workspace_bytes,
                          const int32_t* cu_seqlens, int nseq, int total_tokens, int max_seqlen, int Hq, int Hkv,
                          int d, float scale, int causal, float p_drop, uint64_t seed, void* stream) {
  return varlen_dropout_bwd_any(0, Q, K, V, O, dO, LSE, dQ, dK, dV, workspace, workspace_bytes, cu_seqlens, nseq,
                                total_tokens, max_seqlen, Hq, Hkv, d, scale, causal, p_drop, seed, stream);
}

int fa_varlen_dropout_bwd_f16(const void* Q, const void* K, const void* V, const void* O, const void* dO,
                              const float* LSE, void* dQ, void* dK, void* dV, void* workspace, size_t workspace_bytes,
                              const int32_t* cu_seqlens, int nseq, int total_tokens, int max_seqlen, int Hq, int Hkv,
                              int d, float scale, int causal, float p_drop, uint64_t seed, void* stream) {
  return varlen_dropout_bwd_any(1, Q, K, V, O, dO, LSE, dQ, dK, dV, workspace, workspace_bytes, cu_seqlens, nseq,
                                total_tokens, max_seqlen, Hq, Hkv, d, scale, causal, p_drop, seed, stream);
}

static int check_cross(int B, int Nq, int Nk, int causal) {
  if (B <= 0 || Nq <= 0 || Nk <= 0) return FA_ERR_SHAPE;
  if (causal && Nq > Nk) return FA_ERR_SHAPE;  // some query would see no key
  if ((long)B * Nq > 0x7fffffffL || (long)B * Nk > 0x7fffffffL) return FA_ERR_SHAPE;
  return FA_OK;
}

// Dense entry points with two lengths: the plain ones, half precision, dropout and mask differ
// only in the options.
// (`rule`: the causal rule is in force although `causal` is 0, because a window instantiation applies it)
static int cross_fwd(const void* Q, const void* K, const void* V, void* O, float* LSE, int B, int Hq, int Hkv, int Nq,
                     int Nk, int d, float scale, int causal, void* stream, const Options& opt, int rule = 0) {
  if (!Q || !K || !V || !O || !LSE) return FA_ERR_NULL;
  if (int e = check_cross(B, Nq, Nk, causal || rule)) return e;
  if (int e = check_common(Hq, Hkv, d, scale, !(opt.dropout || opt.mask || opt.window))) return e;
  if (!aligned16(Q) || !aligned16(K) || !aligned16(V) || !aligned16(O) || !aligned16(LSE)) return FA_ERR_ALIGN;
  return run_fwd(Q, K, V, O, LSE, nullptr, B, Nq, Nk, (long)B * Nq, Hq, Hkv, d, scale, causal, stream, 0, nullptr,
                 nullptr, opt);
}

static int cross_bwd(const void* Q, const void* K, const void* V, const void* O, const void* dO, const float* LSE,
                     void* dQ, void* dK, void* dV, void* workspace, size_t workspace_bytes, int B, int Hq, int Hkv,
                     int Nq, int Nk, int d, float scale, int causal, void* stream, const Options& opt, int rule = 0) {
  if (!Q || !K || !V || !O || !dO || !LSE || !dQ || !dK || !dV || !workspace) return FA_ERR_NULL;
  if (int e = check_cross(B, Nq, Nk, causal || rule)) return e;
  if (int e = check_common(Hq, Hkv, d, scale, !(opt.dropout || opt.mask || opt.window))) return e;
  if (!aligned16(Q) || !aligned16(K) || !aligned16(V) || !aligned16(O) || !aligned16(dO) || !aligned16(LSE) ||
      !aligned16(dQ) || !aligned16(dK) || !aligned16(dV) || !aligned16(workspace))
    return FA_ERR_ALIGN;
  if (workspace_bytes < ws_bytes((long)B * Nq, Hq)) return FA_ERR_WORKSPACE;
  return run_bwd(Q, K, V, O, dO, LSE, dQ, dK, dV, workspace, workspace_bytes, nullptr, B, Nq, Nk, (long)B * Nq, Hq, Hkv, d, scale,
                 causal, FA_STAGE_PREP | FA_STAGE_DKDV | FA_STAGE_DQ, stream, nullptr, opt);
}

int fa_cross_fwd(const void* Q, const void* K, const void* V, void* O, float* LSE, int B, int Hq, int Hkv, int Nq,
                 int Nk, int d, float scale, int causal, void* stream) {
  return cross_fwd(Q, K, V, O, LSE, B, Hq, Hkv, Nq, Nk, d, scale, causal, stream, half_precision(0));
}

int fa_cross_fwd_f16(const void* Q, const void* K, const void* V, void* O, float* LSE, int B, int Hq, int Hkv, int Nq,
                     int Nk, int d, float scale, int causal, void* stream) {
  return cross_fwd(Q, K, V, O, LSE, B, Hq, Hkv, Nq, Nk, d, scale, causal, stream, half_precision(1));
}

size_t fa_cross_bwd_workspace_bytes(int B, int Hq, int Hkv, int Nq, int Nk, int d) {
  if (B <= 0 || Hq <= 0 || Nq <= 0 || Nk <= 0 || d <= 0) return 0;
  return ws_bytes((long)B * Nq, Hq, Hkv, d, Nq, (long)B * Nk);
}

int fa_cross_bwd(const void* Q, const void* K, const void* V, const void* O, const void* dO, const float* LSE,
                 void* dQ, void* dK, void* dV, void* workspace, size_t workspace_bytes, int B, int Hq, int Hkv,
                 int Nq, int Nk, int d, float scale, int causal, void* stream) {
  return cross_bwd(Q, K, V, O, dO, LSE, dQ, dK, dV, workspace, workspace_bytes, B, Hq, Hkv, Nq, Nk, d, scale, causal,
                   stream, half_precision(0));
}

int fa_cross_bwd_f16(const void* Q, const void* K, const void* V, const void* O, const void* dO, const float* LSE,
                     void* dQ, void* dK, void* dV, void* workspace, size_t workspace_bytes, int B, int Hq, int Hkv,
                     int Nq, int Nk, int d, float scale, int causal, void* stream) {
  return cross_bwd(Q, K, V, O, dO, LSE, dQ, dK, dV, workspace, workspace_bytes, B, Hq, Hkv, Nq, Nk, d, scale, causal,
                   stream, half_precision(1));
}

static int dropout_fwd_any(int f16, const void* Q, const void* K, const void* V, void* O, float* LSE, int B, int Hq,
                           int Hkv, int Nq, int Nk, int d, float scale, int causal, float p_drop, uint64_t seed,
                           void* stream) {
  return cross_fwd(Q, K, V, O, LSE, B, Hq, Hkv, Nq, Nk, d, scale, causal, stream,
                   of_type(with_dropout(p_drop, seed), f16));
}

int fa_dropout_fwd(const void* Q, const void* K, const void* V, void* O, float* LSE, int B, int Hq, int Hkv, int Nq,
                   int Nk, int d, float scale, int causal, float p_drop, uint64_t seed, void* stream) {
  return dropout_fwd_any(0, Q, K, V, O, LSE, B, Hq, Hkv, Nq, Nk, d, scale, causal, p_drop, seed, stream);
}

int fa_dropout_fwd_f16(const void* Q, const void* K, const void* V, void* O, float* LSE, int B, int Hq, int Hkv,
                       int Nq, int Nk, int d, float scale, int causal, float p_drop, uint64_t seed, void* stream) {
  return dropout_fwd_any(1, Q, K, V, O, LSE, B, Hq, Hkv, Nq, Nk, d, scale, causal, p_drop, seed, stream);
}

static int dropout_bwd_any(int f16, const void* Q, const void* K, const void* V, const void* O, const void* dO,
                           const float* LSE, void* dQ, void* dK, void* dV, void* workspace, size_t workspace_bytes,
                           int B, int Hq, int Hkv, int Nq, int Nk, int d, float scale, int causal, float p_drop,
                           uint64_t seed, void* stream) {
  return cross_bwd(Q, K, V, O, dO, LSE, dQ, dK, dV, workspace, workspace_bytes, B, Hq, Hkv, Nq, Nk, d, scale, causal,
                   stream, of_type(with_dropout(p_drop, seed), f16));
}

int fa_dropout_bwd(const void* Q, const void* K, const void* V, const void* O, const void* dO, const float* LSE,
                   void* dQ, void* dK, void* dV, void* workspace, size_t workspace_bytes, int B, int Hq, int Hkv,
                   int Nq, int Nk, int d, float scale, int causal, float p_drop, uint64_t seed, void* stream) {
  return dropout_bwd_any(0, Q, K, V, O, dO, LSE, dQ, dK, dV, workspace, workspace_bytes, B, Hq, Hkv, Nq, Nk, d, scale,
                         causal, p_drop, seed, stream);
}

int fa_dropout_bwd_f16(const void* Q, const void* K, const void* V, const void* O, const void* dO, const float* LSE,
                       void* dQ, void* dK, void* dV, void* workspace, size_t workspace_bytes, int B, int Hq, int Hkv,
                       int Nq, int Nk, int d, float scale, int causal, float p_drop, uint64_t seed, void* stream) {
  return dropout_bwd_any(1, Q, K, V, O, dO, LSE, dQ, dK, dV, workspace, workspace_bytes, B, Hq, Hkv, Nq, Nk, d, scale,
                         causal, p_drop, seed, stream);
}

static int mask_fwd_any(int f16, const void* Q, const void* K, const void* V, const void* M, void* O, float* LSE,
                        int B, int Hq, int Hkv, int Nq, int Nk, int d, float scale, int causal,
                        long long mask_batch_stride, long long mask_head_stride, long long mask_row_stride,
                        void* stream) {
  return cross_fwd(Q, K, V, O, LSE, B, Hq, Hkv, Nq, Nk, d, scale, causal, stream,
                   of_type(with_mask(M, mask_batch_stride, mask_head_stride, mask_row_stride), f16));
}

int fa_mask_fwd(const void* Q, const void* K, const void* V, const void* M, void* O, float* LSE, int B, int Hq,
                int Hkv, int Nq, int Nk, int d, float scale, int causal, long long mask_batch_stride,
                long long mask_head_stride, long long mask_row_stride, void* stream) {
  return mask_fwd_any(0, Q, K, V, M, O, LSE, B, Hq, Hkv, Nq, Nk, d, scale, causal, mask_batch_stride, mask_head_stride,
                      mask_row_stride, stream);
}

int fa_mask_fwd_f16(const void* Q, const void* K, const void* V, const void* M, void* O, float* LSE, int B, int Hq,
                    int Hkv, int Nq, int Nk, int d, float scale, int causal, long long mask_batch_stride,
                    long long mask_head_stride, long long mask_row_stride, void* stream) {
  return mask_fwd_any(1, Q, K, V, M, O, LSE, B, Hq, Hkv, Nq, Nk, d, scale, causal, mask_batch_stride, mask_head_stride,
                      mask_row_stride, stream);
}

static int mask_bwd_any(int f16, const void* Q, const void* K, const void* V, const void* M, const void* O,
                        const void* dO, const float* LSE, void* dQ, void* dK, void* dV, void* workspace,
                        size_t workspace_bytes, int B, int Hq, int Hkv, int Nq, int Nk, int d, float scale, int causal,
                        long long mask_batch_stride, long long mask_head_stride, long long mask_row_stride,
                        void* stream) {
  return cross_bwd(Q, K, V, O, dO, LSE, dQ, dK, dV, workspace, workspace_bytes, B, Hq, Hkv, Nq, Nk, d, scale, causal,
                   stream, of_type(with_mask(M, mask_batch_stride, mask_head_stride, mask_row_stride), f16));
}

int fa_mask_bwd(const void* Q, const void* K, const void* V, const void* M, const void* O, const void* dO,
                const float* LSE, void* dQ, void* dK, void* dV, void* workspace, size_t workspace_bytes, int B, int Hq,
                int Hkv, int Nq, int Nk, int d, float scale, int causal, long long mask_batch_stride,
                long long mask_head_stride, long long mask_row_stride, void* stream) {
  return mask_bwd_any(0, Q, K, V, M, O, dO, LSE, dQ, dK, dV, workspace, workspace_bytes, B, Hq, Hkv, Nq, Nk, d, scale,
                      causal, mask_batch_stride, mask_head_stride, mask_row_stride, stream);
}

int fa_mask_bwd_f16(const void* Q, const void* K, const void* V, const void* M, const void* O, const void* dO,
                    const float* LSE, void* dQ, void* dK, void* dV, void* workspace, size_t workspace_bytes, int B,
                    int Hq, int Hkv, int Nq, int Nk, int d, float scale, int causal, long long mask_batch_stride,
                    long long mask_head_stride, long long mask_row_stride, void* stream) {
  return mask_bwd_any(1, Q, K, V, M, O, dO, LSE, dQ, dK, dV, workspace, workspace_bytes, B, Hq, Hkv, Nq, Nk, d, scale,
                      causal, mask_batch_stride, mask_head_stride, mask_row_stride, stream);
}

static int mask_bwd_dmask_any(int f16, const void* Q, const void* K, const void* V, const void* M, const void* O,
                              const void* dO, const float* LSE, void* dQ, void* dK, void* dV, void* dM, void* workspace,
                              size_t workspace_bytes, int B, int Hq, int Hkv, int Nq, int Nk, int d, float scale,
                              int causal, long long mask_batch_stride, long long mask_head_stride,
                              long long mask_row_stride, long long dmask_batch_stride, long long dmask_head_stride,
                              long long dmask_row_stride, void* stream) {
  if (!dM) return FA_ERR_NULL;
  if (!aligned16(dM)) return FA_ERR_ALIGN;
  // every (sequence, head) has rows of its own in dM: strides as for M, none of them zero
  if (dmask_row_stride < (((long long)Nk + 7) & ~7LL) || dmask_row_stride % 8 || dmask_head_stride % 8 ||
      dmask_batch_stride % 8 || dmask_head_stride < dmask_row_stride * Nq ||
      dmask_batch_stride < dmask_head_stride * Hq)
    return FA_ERR_SHAPE;
  Options opt = of_type(with_mask(M, mask_batch_stride, mask_head_stride, mask_row_stride), f16);
  opt.dM = dM;
  opt.dm_bs = dmask_batch_stride;
  opt.dm_hs = dmask_head_stride;
  opt.dm_rs = dmask_row_stride;
  return cross_bwd(Q, K, V, O, dO, LSE, dQ, dK, dV, workspace, workspace_bytes, B, Hq, Hkv, Nq, Nk, d, scale, causal,
                   stream, opt);
}

int fa_mask_bwd_dmask(const void* Q, const void* K, const void* V, const void* M, const void* O, const void* dO,
                      const float* LSE, void* dQ, void* dK, void* dV, void* dM, void* workspace, size_t workspace_bytes,
                      int B, int Hq, int Hkv, int Nq, int Nk, int d, float scale, int causal,
                      long long mask_batch_stride, long long mask_head_stride, long long mask_row_stride,
                      long long dmask_batch_stride, long long dmask_head_stride, long long dmask_row_stride,
                      void* stream) {
  return mask_bwd_dmask_any(0, Q, K, V, M, O, dO, LSE, dQ, dK, dV, dM, workspace, workspace_bytes, B, Hq, Hkv, Nq, Nk, d,
                            scale, causal, mask_batch_stride, mask_head_stride, mask_row_stride, dmask_batch_stride,
                            dmask_head_stride, dmask_row_stride, stream);
}

int fa_mask_bwd_dmask_f16(const void* Q, const void* K, const void* V, const void* M, const void* O, const void* dO,
                          const float* LSE, void* dQ, void* dK, void* dV, void* dM, void* workspace,
                          size_t workspace_bytes, int B, int Hq, int Hkv, int Nq, int Nk, int d, float scale, int causal,
                          long long mask_batch_stride, long long mask_head_stride, long long mask_row_stride,
                          long long dmask_batch_stride, long long dmask_head_stride, long long dmask_row_stride,
                          void* stream) {
  return mask_bwd_dmask_any(1, Q, K, V, M, O, dO, LSE, dQ, dK, dV, dM, workspace, workspace_bytes, B, Hq, Hkv, Nq, Nk, d,
                            scale, causal, mask_batch_stride, mask_head_stride, mask_row_stride, dmask_batch_stride,
                            dmask_head_stride, dmask_row_stride, stream);
}

// Sliding window. Without any bound this is plain attention and with win_right = 0 alone the
// causal rule: both go to the kernels built for them. Otherwise the window instantiations run.
static int window_route(int Nq, int Nk, int& left, int& right, int& causal) {
  if (Nq > Nk) return FA_ERR_SHAPE;  // some query would stand before the first key
  if (left < 0) left = -1;
  if (right < 0) right = -1;
  if (left >= Nk) left = -1;    // a bound no row can reach is no bound
  if (right >= Nk) right = -1;
  causal = left < 0 && right == 0;
  if (causal) right = -1;
  return FA_OK;
}

static int local_fwd_any(int f16, const void* Q, const void* K, const void* V, void* O, float* LSE, int B, int Hq,
                         int Hkv, int Nq, int Nk, int d, float scale, int window_left, int window_right,
                         void* stream) {
  int causal = 0;
  if (B > 0 && Nq > 0 && Nk > 0)
    if (int e = window_route(Nq, Nk, window_left, window_right, causal)) return e;
  const bool none = window_left < 0 && window_right < 0;
  return cross_fwd(Q, K, V, O, LSE, B, Hq, Hkv, Nq, Nk, d, scale, causal, stream,
                   none ? half_precision(f16) : of_type(with_window(window_left, window_right), f16));
}

int fa_local_fwd(const void* Q, const void* K, const void* V, void* O, float* LSE, int B, int Hq, int Hkv, int Nq,
                 int Nk, int d, float scale, int window_left, int window_right, void* stream) {
  return local_fwd_any(0, Q, K, V, O, LSE, B, Hq, Hkv, Nq, Nk, d, scale, window_left, window_right, stream);
}

int fa_local_fwd_f16(const void* Q, const void* K, const void* V, void* O, float* LSE, int B, int Hq, int Hkv, int Nq,
                     int Nk, int d, float scale, int window_left, int window_right, void* stream) {
  return local_fwd_any(1, Q, K, V, O, LSE, B, Hq, Hkv, Nq, Nk, d, scale, window_left, window_right, stream);
}

static int local_bwd_any(int f16, const void* Q, const void* K, const void* V, const void* O, const void* dO,
                         const float* LSE, void* dQ, void* dK, void* dV, void* workspace, size_t workspace_bytes,
                         int B, int Hq, int Hkv, int Nq, int Nk, int d, float scale, int window_left, int window_right,
                         void* stream) {
  int causal = 0;
  if (B > 0 && Nq > 0 && Nk > 0)
    if (int e = window_route(Nq, Nk, window_left, window_right, causal)) return e;
  const bool none = window_left < 0 && window_right < 0;
  return cross_bwd(Q, K, V, O, dO, LSE, dQ, dK, dV, workspace, workspace_bytes, B, Hq, Hkv, Nq, Nk, d, scale, causal,
                   stream, none ? half_precision(f16) : of_type(with_window(window_left, window_right), f16));
}

int fa_local_bwd(const void* Q, const void* K, const void* V, const void* O, const void* dO, const float* LSE,
                 void* dQ, void* dK, void* dV, void* workspace, size_t workspace_bytes, int B, int Hq, int Hkv, int Nq,
                 int Nk, int d, float scale, int window_left, int window_right, void* stream) {
  return local_bwd_any(0, Q, K, V, O, dO, LSE, dQ, dK, dV, workspace, workspace_bytes, B, Hq, Hkv, Nq, Nk, d, scale,
                       window_left, window_right, stream);
}

int fa_local_bwd_f16(const void* Q, const void* K, const void* V, const void* O, const void* dO, const float* LSE,
                     void* dQ, void* dK, void* dV, void* workspace, size_t workspace_bytes, int B, int Hq, int Hkv,
                     int Nq, int Nk, int d, float scale, int window_left, int window_right, void* stream) {
  return local_bwd_any(1, Q, K, V, O, dO, LSE, dQ, dK, dV, workspace, workspace_bytes, B, Hq, Hkv, Nq, Nk, d, scale,
                       window_left, window_right, stream);
}

static Options with_block_pattern(const void* block_mask, int block, long long bs, long long hs, int causal) {
  Options o = with_window(-1, causal ? 0 : -1);  // the causal rule is the window (none, 0)
  o.bmask = block_mask;
  o.bmask_bs = bs;
  o.bmask_hs = hs;
  o.block = block ? block : -1;  // (0 would read as "no pattern")
  return o;
}

static int blocksparse_fwd_any(int f16, const void* Q, const void* K, const void* V, const void* block_mask, void* O,
                               float* LSE, int B, int Hq, int Hkv, int Nq, int Nk, int d, float scale, int causal,
                               int block, long long mask_batch_stride, long long mask_head_stride, void* stream) {
  if (!block_mask) return FA_ERR_NULL;
  return cross_fwd(Q, K, V, O, LSE, B, Hq, Hkv, Nq, Nk, d, scale, 0, stream,
                   of_type(with_block_pattern(block_mask, block, mask_batch_stride, mask_head_stride, causal), f16),
                   causal);
}

int fa_blocksparse_fwd(const void* Q, const void* K, const void* V, const void* block_mask, void* O, float* LSE, int B,
                       int Hq, int Hkv, int Nq, int Nk, int d, float scale, int causal, int block,
                       long long mask_batch_stride, long long mask_head_stride, void* stream) {
  return blocksparse_fwd_any(0, Q, K, V, block_mask, O, LSE, B, Hq, Hkv, Nq, Nk, d, scale, causal, block,
                             mask_batch_stride, mask_head_stride, stream);
}

int fa_blocksparse_fwd_f16(const void* Q, const void* K, const void* V, const void* block_mask, void* O, float* LSE,
                           int B, int Hq, int Hkv, int Nq, int Nk, int d, float scale, int causal, int block,
                           long long mask_batch_stride, long long mask_head_stride, void* stream) {
  return blocksparse_fwd_any(1, Q, K, V, block_mask, O, LSE, B, Hq, Hkv, Nq, Nk, d, scale, causal, block,
                             mask_batch_stride, mask_head_stride, stream);
}

static int blocksparse_bwd_any(int f16, const void* Q, const void* K, const void* V, const void* block_mask,
                               const void* O, const void* dO, const float* LSE, void* dQ, void* dK, void* dV,
                               void* workspace, size_t workspace_bytes, int B, int Hq, int Hkv, int Nq, int Nk, int d,
                               float scale, int causal, int block, long long mask_batch_stride,
                               long long mask_head_stride, void* stream) {
  if (!block_mask) return FA_ERR_NULL;
  return cross_bwd(Q, K, V, O, dO, LSE, dQ, dK, dV, workspace, workspace_bytes, B, Hq, Hkv, Nq, Nk, d, scale, 0, stream,
                   of_type(with_block_pattern(block_mask, block, mask_batch_stride, mask_head_stride, causal), f16),
                   causal);
}

int fa_blocksparse_bwd(const void* Q, const void* K, const void* V, const void* block_mask, const void* O,
                       const void* dO, const float* LSE, void* dQ, void* dK, void* dV, void* workspace,
                       size_t workspace_bytes, int B, int Hq, int Hkv, int Nq, int Nk, int d, float scale, int causal,
                       int block, long long mask_batch_stride, long long mask_head_stride, void* stream) {
  return blocksparse_bwd_any(0, Q, K, V, block_mask, O, dO, LSE, dQ, dK, dV, workspace, workspace_bytes, B, Hq, Hkv,
                             Nq, Nk, d, scale, causal, block, mask_batch_stride, mask_head_stride, stream);
}

int fa_blocksparse_bwd_f16(const void* Q, const void* K, const void* V, const void* block_mask, const void* O,
                           const void* dO, const float* LSE, void* dQ, void* dK, void* dV, void* workspace,
                           size_t workspace_bytes, int B, int Hq, int Hkv, int Nq, int Nk, int d, float scale,
                           int causal, int block, long long mask_batch_stride, long long mask_head_stride,
                           void* stream) {
  return blocksparse_bwd_any(1, Q, K, V, block_mask, O, dO, LSE, dQ, dK, dV, workspace, workspace_bytes, B, Hq, Hkv,
                             Nq, Nk, d, scale, causal, block, mask_batch_stride, mask_head_stride, stream);
}

int fa_fp8_fwd(const void* Q8, const void* K8, const void* Vt8, void* O, float* LSE, int B, int Hq, int Hkv, int Nq,
               int Nk, int d, long long vt_stride, float scale, float descale_q, float descale_k, float descale_v,
               int causal, void* stream) {
  if (!Q8 || !K8 || !Vt8 || !O || !LSE) return FA_ERR_NULL;
  if (int e = check_cross(B, Nq, Nk, causal)) return e;
  if (int e = check_common(Hq, Hkv, d, scale, false)) return e;
  for (float ds : {descale_q, descale_k, descale_v})
    if (!(ds > 0.f) || !std::isfinite(ds)) return FA_ERR_SHAPE;
  if (vt_stride % 64 != 0 || vt_stride < ((long long)Nk + 63) / 64 * 64) return FA_ERR_SHAPE;
  if (!aligned16(Q8) || !aligned16(K8) || !aligned16(Vt8) || !aligned16(O) || !aligned16(LSE)) return FA_ERR_ALIGN;
  fa::Fp8Args a;
  a.p = make_problem(nullptr, B, Nq, Nk, Hq, Hkv, d, (long)B * Nq, scale * descale_q * descale_k);
  a.Q = Q8;
  a.K = K8;
  a.Vt = Vt8;
  a.O = (__bf16*)O;
  a.LSE = LSE;
  a.vt_stride = (long)vt_stride;
  a.descale_v = descale_v;
  hipError_t e = fa::launch_fwd_fp8(a, d, causal, (hipStream_t)stream);
  if (e != hipSuccess) {
    g_last_hip_error = (int)e;
    return FA_ERR_LAUNCH;
  }
  return FA_OK;
}

// Sliding window over a packed ragged batch: the routing of fa_local_fwd with the longest
// sequence standing for both lengths (a bound that reaches past it binds nowhere).
static int varlen_local_fwd_any(int f16, const void* Q, const void* K, const void* V, void* O, float* LSE,
                                const int32_t* cu_seqlens, int nseq, int total_tokens, int max_seqlen, int Hq,
                                int Hkv, int d, float scale, int window_left, int window_right, void* stream) {
  int causal = 0;
  if (max_seqlen > 0)
    if (int e = window_route(max_seqlen, max_seqlen, window_left, window_right, causal)) return e;
  const bool none = window_left < 0 && window_right < 0;
  return varlen_fwd(Q, K, V, O, LSE, cu_seqlens, nseq, total_tokens, max_seqlen, Hq, Hkv, d, scale, causal, stream,
                    none ? half_precision(f16) : of_type(with_window(window_left, window_right), f16));
}

int fa_varlen_local_fwd(const void* Q, const void* K, const void* V, void* O, float* LSE, const int32_t* cu_seqlens,
                        int nseq, int total_tokens, int max_seqlen, int Hq, int Hkv, int d, float scale,
                        int window_left, int window_right, void* stream) {
  return varlen_local_fwd_any(0, Q, K, V, O, LSE, cu_seqlens, nseq, total_tokens, max_seqlen, Hq, Hkv, d, scale,
                              window_left, window_right, stream);
}

int fa_varlen_local_fwd_f16(const void* Q, const void* K, const void* V, void* O, float* LSE,
                            const int32_t* cu_seqlens, int nseq, int total_tokens, int max_seqlen, int Hq, int Hkv,
                            int d, float scale, int window_left, int window_right, void* stream) {
  return varlen_local_fwd_any(1, Q, K, V, O, LSE, cu_seqlens, nseq, total_tokens, max_seqlen, Hq, Hkv, d, scale,
                              window_left, window_right, stream);
}

static int varlen_local_bwd_any(int f16, const void* Q, const void* K, const void* V, const void* O, const void* dO,
                                const float* LSE, void* dQ, void* dK, void* dV, void* workspace,
                                size_t workspace_bytes, const int32_t* cu_seqlens, int nseq, int total_tokens,
                                int max_seqlen, int Hq, int Hkv, int d, float scale, int window_left,
                                int window_right, void* stream) {
  int causal = 0;
  if (max_seqlen > 0)
    if (int e = window_route(max_seqlen, max_seqlen, window_left, window_right, causal)) return e;
  const bool none = window_left < 0 && window_right < 0;
  return varlen_bwd(Q, K, V, O, dO, LSE, dQ, dK, dV, workspace, workspace_bytes, cu_seqlens, nseq, total_tokens,
                    max_seqlen, Hq, Hkv, d, scale, causal, stream,
                    none ? half_precision(f16) : of_type(with_window(window_left, window_right), f16));
}

int fa_varlen_local_bwd(const void* Q, const void* K, const void* V, const void* O, const void* dO, const float* LSE,
                        void* dQ, void* dK, void* dV, void* workspace, size_t workspace_bytes,
                        const int32_t* cu_seqlens, int nseq, int total_tokens, int max_seqlen, int Hq, int Hkv, int d,
                        float scale, int window_left, int window_right, void* stream) {
  return varlen_local_bwd_any(0, Q, K, V, O, dO, LSE, dQ, dK, dV, workspace, workspace_bytes, cu_seqlens, nseq,
                              total_tokens, max_seqlen, Hq, Hkv, d, scale, window_left, window_right, stream);
}

int fa_varlen_local_bwd_f16(const void* Q, const void* K, const void* V, const void* O, const void* dO,
                            const float* LSE, void* dQ, void* dK, void* dV, void* workspace, size_t workspace_bytes,
                            const int32_t* cu_seqlens, int nseq, int total_tokens, int max_seqlen, int Hq, int Hkv,
                            int d, float scale, int window_left, int window_right, void* stream) {
  return varlen_local_bwd_any(1, Q, K, V, O, dO, LSE, dQ, dK, dV, workspace, workspace_bytes, cu_seqlens, nseq,
                              total_tokens, max_seqlen, Hq, Hkv, d, scale, window_left, window_right, stream);
}

static int check_varlen_cross(const int32_t* cu_q, const int32_t* cu_k, int nseq, int total_q, int total_k, int max_q,
                              int max_k) {
  if (int e = check_varlen(cu_q, nseq, total_q, max_q)) return e;
  return check_varlen(cu_k, nseq, total_k, max_k);
}

static int varlen_cross_fwd_any(int f16, const void* Q, const void* K, const void* V, void* O, float* LSE,
                                const int32_t* cu_seqlens_q, const int32_t* cu_seqlens_k, int nseq, int total_q,
                                int total_k, int max_seqlen_q, int max_seqlen_k, int Hq, int Hkv, int d, float scale,
                                int causal, void* stream) {
  if (!Q || !K || !V || !O || !LSE) return FA_ERR_NULL;
  if (int e = check_varlen_cross(cu_seqlens_q, cu_seqlens_k, nseq, total_q, total_k, max_seqlen_q, max_seqlen_k)) return e;
  if (int e = check_common(Hq, Hkv, d, scale)) return e;
  if (!aligned16(Q) || !aligned16(K) || !aligned16(V) || !aligned16(O) || !aligned16(LSE)) return FA_ERR_ALIGN;
  return run_fwd(Q, K, V, O, LSE, cu_seqlens_q, nseq, max_seqlen_q, max_seqlen_k, total_q, Hq, Hkv, d, scale, causal,
                 stream, 0, nullptr, cu_seqlens_k, half_precision(f16));
}

int fa_varlen_cross_fwd(const void* Q, const void* K, const void* V, void* O, float* LSE, const int32_t* cu_seqlens_q,
                        const int32_t* cu_seqlens_k, int nseq, int total_q, int total_k, int max_seqlen_q,
                        int max_seqlen_k, int Hq, int Hkv, int d, float scale, int causal, void* stream) {
  return varlen_cross_fwd_any(0, Q, K, V, O, LSE, cu_seqlens_q, cu_seqlens_k, nseq, total_q, total_k, max_seqlen_q,
                              max_seqlen_k, Hq, Hkv, d, scale, causal, stream);
}

int fa_varlen_cross_fwd_f16(const void* Q, const void* K, const void* V, void* O, float* LSE,
                            const int32_t* cu_seqlens_q, const int32_t* cu_seqlens_k, int nseq, int total_q,
                            int total_k, int max_seqlen_q, int max_seqlen_k, int Hq, int Hkv, int d, float scale,
                            int causal, void* stream) {
  return varlen_cross_fwd_any(1, Q, K, V, O, LSE, cu_seqlens_q, cu_seqlens_k, nseq, total_q, total_k, max_seqlen_q,
                              max_seqlen_k, Hq, Hkv, d, scale, causal, stream);
}

static int varlen_cross_bwd_any(int f16, const void* Q, const void* K, const void* V, const void* O, const void* dO,
                                const float* LSE, void* dQ, void* dK, void* dV, void* workspace,
                                size_t workspace_bytes, const int32_t* cu_seqlens_q, const int32_t* cu_seqlens_k,
                                int nseq, int total_q, int total_k, int max_seqlen_q, int max_seqlen_k, int Hq,
                                int Hkv, int d, float scale, int causal, void* stream) {
  if (!Q || !K || !V || !O || !dO || !LSE || !dQ || !dK || !dV || !workspace) return FA_ERR_NULL;
  if (int e = check_varlen_cross(cu_seqlens_q, cu_seqlens_k, nseq, total_q, total_k, max_seqlen_q, max_seqlen_k)) return e;
  if (int e = check_common(Hq, Hkv, d, scale)) return e;
  if (!aligned16(Q) || !aligned16(K) || !aligned16(V) || !aligned16(O) || !aligned16(dO) || !aligned16(LSE) ||
      !aligned16(dQ) || !aligned16(dK) || !aligned16(dV) || !aligned16(workspace))
    return FA_ERR_ALIGN;
  if (workspace_bytes < ws_bytes(total_q, Hq)) return FA_ERR_WORKSPACE;
  return run_bwd(Q, K, V, O, dO, LSE, dQ, dK, dV, workspace, workspace_bytes, cu_seqlens_q, nseq, max_seqlen_q, max_seqlen_k, total_q,
                 Hq, Hkv, d, scale, causal, 7, stream, cu_seqlens_k, half_precision(f16), total_k);
}

int fa_varlen_cross_bwd(const void* Q, const void* K, const void* V, const void* O, const void* dO, const float* LSE,
                        void* dQ, void* dK, void* dV, void* workspace, size_t workspace_bytes,
                        const int32_t* cu_seqlens_q, const int32_t* cu_seqlens_k, int nseq, int total_q, int total_k,
                        int max_seqlen_q, int max_seqlen_k, int Hq, int Hkv, int d, float scale, int causal,
                        void* stream) {
  return varlen_cross_bwd_any(0, Q, K, V, O, dO, LSE, dQ, dK, dV, workspace, workspace_bytes, cu_seqlens_q,
                              cu_seqlens_k, nseq, total_q, total_k, max_seqlen_q, max_seqlen_k, Hq, Hkv, d, scale,
                              causal, stream);
}

int fa_varlen_cross_bwd_f16(const void* Q, const void* K, const void* V, const void* O, const void* dO,
                            const float* LSE, void* dQ, void* dK, void* dV, void* workspace, size_t workspace_bytes,
                            const int32_t* cu_seqlens_q, const int32_t* cu_seqlens_k, int nseq, int total_q,
                            int total_k, int max_seqlen_q, int max_seqlen_k, int Hq, int Hkv, int d, float scale,
                            int causal, void* stream) {
  return varlen_cross_bwd_any(1, Q, K, V, O, dO, LSE, dQ, dK, dV, workspace, workspace_bytes, cu_seqlens_q,
                              cu_seqlens_k, nseq, total_q, total_k, max_seqlen_q, max_seqlen_k, Hq, Hkv, d, scale,
                              causal, stream);
}

size_t fa_splitkv_fwd_workspace_bytes(int B, int Hq, int Nq, int d, int num_splits) {
  if (B <= 0 || Hq <= 0 || Nq <= 0 || d <= 0 || num_splits <= 0) return 0;
  return round_up((size_t)num_splits * B * Nq * Hq * (d + 1) * sizeof(float), 256);
}

static int splitkv_fwd_any(int f16, const void* Q, const void* K, const void* V, void* O, float* LSE, void* workspace,
                           size_t workspace_bytes, int B, int Hq, int Hkv, int Nq, int Nk, int d, float scale,
                           int causal, int num_splits, void* stream) {
  if (!Q || !K || !V || !O || !LSE || !workspace) return FA_ERR_NULL;
  if (int e = check_cross(B, Nq, Nk, causal)) return e;
  if (int e = check_common(Hq, Hkv, d, scale, false)) return e;
  if (num_splits < 1 || num_splits > FA_SPLITKV_MAX_SPLITS) return FA_ERR_SHAPE;
  if ((long)Nq * (Hq / Hkv) > 0x7fffffffL) return FA_ERR_SHAPE;
  if (!aligned16(Q) || !aligned16(K) || !aligned16(V) || !aligned16(O) || !aligned16(LSE) || !aligned16(workspace))
    return FA_ERR_ALIGN;
  if (workspace_bytes < fa_splitkv_fwd_workspace_bytes(B, Hq, Nq, d, num_splits)) return FA_ERR_WORKSPACE;
  return run_fwd(Q, K, V, O, LSE, nullptr, B, Nq, Nk, (long)B * Nq, Hq, Hkv, d, scale, causal, stream, num_splits,
                 workspace, nullptr, half_precision(f16));
}

int fa_splitkv_fwd(const void* Q, const void* K, const void* V, void* O, float* LSE, void* workspace,
                   size_t workspace_bytes, int B, int Hq, int Hkv, int Nq, int Nk, int d, float scale, int causal,
                   int num_splits, void* stream) {
  return splitkv_fwd_any(0, Q, K, V, O, LSE, workspace, workspace_bytes, B, Hq, Hkv, Nq, Nk, d, scale, causal,
                         num_splits, stream);
}

int fa_splitkv_fwd_f16(const void* Q, const void* K, const void* V, void* O, float* LSE, void* workspace,
                       size_t workspace_bytes, int B, int Hq, int Hkv, int Nq, int Nk, int d, float scale, int causal,
                       int num_splits, void* stream) {
  return splitkv_fwd_any(1, Q, K, V, O, LSE, workspace, workspace_bytes, B, Hq, Hkv, Nq, Nk, d, scale, causal,
                         num_splits, stream);
}

static int kvcache_fwd_any(int f16, const void* Q, const void* Kcache, const void* Vcache, const int32_t* seqlens_k,
                           const int32_t* block_table, void* O, float* LSE, void* workspace, size_t workspace_bytes,
                           int B, int Hq, int Hkv, int Nq, int Nk, int d, int page_size, int pages_per_seq,
                           float scale, int causal, int num_splits, void* stream) {
  if (!Q || !Kcache || !Vcache || !O || !LSE || !workspace) return FA_ERR_NULL;
  if (int e = check_cross(B, Nq, Nk, causal)) return e;
  if (int e = check_common(Hq, Hkv, d, scale, false)) return e;
  if (num_splits < 1 || num_splits > FA_SPLITKV_MAX_SPLITS) return FA_ERR_SHAPE;
  if ((long)Nq * (Hq / Hkv) > 0x7fffffffL) return FA_ERR_SHAPE;
  Options opt = half_precision(f16);
  opt.seqlens_k = seqlens_k;
  if (block_table) {
    if (page_size < 64 || (page_size & (page_size - 1))) return FA_ERR_UNSUPPORTED;  // whole blocks of 64 keys per page
    if (pages_per_seq < 1 || (long)pages_per_seq * page_size < Nk) return FA_ERR_SHAPE;
    opt.block_table = block_table;
    opt.page_log2 = __builtin_ctz((unsigned)page_size);
    opt.table_stride = pages_per_seq;
  }
  if (!aligned16(Q) || !aligned16(Kcache) || !aligned16(Vcache) || !aligned16(O) || !aligned16(LSE) ||
      !aligned16(workspace) || (reinterpret_cast<uintptr_t>(seqlens_k) & 3u) ||
      (reinterpret_cast<uintptr_t>(block_table) & 3u))
    return FA_ERR_ALIGN;
  if (workspace_bytes < fa_splitkv_fwd_workspace_bytes(B, Hq, Nq, d, num_splits)) return FA_ERR_WORKSPACE;
  return run_fwd(Q, Kcache, Vcache, O, LSE, nullptr, B, Nq, Nk, (long)B * Nq, Hq, Hkv, d, scale, causal, stream,
                 num_splits, workspace, nullptr, opt);
}

int fa_kvcache_fwd(const void* Q, const void* Kcache, const void* Vcache, const int32_t* seqlens_k,
                   const int32_t* block_table, void* O, float* LSE, void* workspace, size_t workspace_bytes, int B,
                   int Hq, int Hkv, int Nq, int Nk, int d, int page_size, int pages_per_seq, float scale, int causal,
                   int num_splits, void* stream) {
  return kvcache_fwd_any(0, Q, Kcache, Vcache, seqlens_k, block_table, O, LSE, workspace, workspace_bytes, B, Hq, Hkv,
                         Nq, Nk, d, page_size, pages_per_seq, scale, causal, num_splits, stream);
}

int fa_kvcache_fwd_f16(const void* Q, const void* Kcache, const void* Vcache, const int32_t* seqlens_k,
                       const int32_t* block_table, void* O, float* LSE, void* workspace, size_t workspace_bytes,
                       int B, int Hq, int Hkv, int Nq, int Nk, int d, int page_size, int pages_per_seq, float scale,
                       int causal, int num_splits, void* stream) {
  return kvcache_fwd_any(1, Q, Kcache, Vcache, seqlens_k, block_table, O, LSE, workspace, workspace_bytes, B, Hq, Hkv,
                         Nq, Nk, d, page_size, pages_per_seq, scale, causal, num_splits, stream);
}

// ---- caches that are written, weighed and cut, a prefix that a batch shares, drafts that are verified

static inline bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

static int launched(hipError_t e) {
  if (e == hipSuccess) return FA_OK;
  g_last_hip_error = (int)e;
  return FA_ERR_LAUNCH;
}

// The slots of B sequences (Nk each), in slabs or pages
static int set_cache(fa::CacheView& c, const int32_t* lens, const int32_t* table, int B, int Hkv, int Nk, int d, int page_size, int pages_per_seq) {
  if (B <= 0 || Hkv <= 0 || Nk <= 0) return FA_ERR_SHAPE;
  if (B > (1 << 20) || Hkv > (1 << 20) || (long)B * Hkv > (1 << 20)) return FA_ERR_SHAPE;  // (a grid has room for them)
  if (Nk > FA_CACHE_MAX_SLOTS) return FA_ERR_SHAPE;  // (a slot and the next tile's stay within 32 bits)
  c = {lens, table, 0, pages_per_seq, Nk, Hkv, d};
  if (table) {
    if (page_size < 64 || (page_size & (page_size - 1))) return FA_ERR_UNSUPPORTED;
    if (pages_per_seq < 1 || (long)pages_per_seq * page_size < Nk) return FA_ERR_SHAPE;
    c.page_log2 = __builtin_ctz((unsigned)page_size);
  }
  if (!aligned4(lens) || !aligned4(table)) return FA_ERR_ALIGN;
  return FA_OK;
}

// Head dimensions of the kernels that only move rows
static int check_rows(int d) { return d <= 0 ? FA_ERR_SHAPE : (d % 8 || d > 256 ? FA_ERR_UNSUPPORTED : FA_OK); }

size_t fa_prefix_fwd_workspace_bytes(int B, int Hq, int Hkv, int Nq, int Np, int Nk, int d) {
  if (B <= 0 || Hq <= 0 || Hkv <= 0 || Hq % Hkv || Nq <= 0 || Np < 0 || Nk <= 0 || (d != 64 && d != 128) ||
      (double)B * Nq * Hq > (1 << 26))
    return 0;
  const fa::PrefixPlan p = fa::prefix_plan(B, Hq, Hkv, Nq, Np, Nk, d);
  return round_up((size_t)(p.prefix_shares + p.own_shares) * B * Nq * Hq * (d + 1) * sizeof(float), 256);
}

static int prefix_fwd_any(int f16, const void* Q, const void* Kprefix, const void* Vprefix, const int32_t* prefix_table, const void* Kcache,
                          const void* Vcache, const int32_t* seqlens_k, const int32_t* block_table, void* O, float* LSE, void* workspace,
                          size_t workspace_bytes, int B, int Hq, int Hkv, int Nq, int Np, int Nk, int d, int page_size,
                          int prefix_pages, int pages_per_seq, float scale, int causal, void* stream) {
  if (!Q || !Kcache || !Vcache || !O || !LSE || !workspace || (Np > 0 && (!Kprefix || !Vprefix))) return FA_ERR_NULL;
  if (Nq <= 0 || Np < 0) return FA_ERR_SHAPE;
  if (int e = check_common(Hq, Hkv, d, scale, false)) return e;
  fa::PrefixArgs a;
  if (int e = set_cache(a.own, seqlens_k, block_table, B, Hkv, Nk, d, page_size, pages_per_seq)) return e;
  if (Np > FA_CACHE_MAX_SLOTS || (double)B * Nq * Hq > (1 << 26) || Hkv > (1 << 16)) return FA_ERR_SHAPE;  // (a tile's rows lie within 32 bits of its first)
  if (prefix_table && Np > 0) {
    if (page_size < 64 || (page_size & (page_size - 1))) return FA_ERR_UNSUPPORTED;
    if (prefix_pages < 1 || (long)prefix_pages * page_size < Np) return FA_ERR_SHAPE;
    a.own.page_log2 = __builtin_ctz((unsigned)page_size);
  }
  if (!aligned16(Q) || !aligned16(Kprefix) || !aligned16(Vprefix) || !aligned16(Kcache) || !aligned16(Vcache) || !aligned16(O) ||
      !aligned16(LSE) || !aligned16(workspace) || !aligned4(prefix_table))
    return FA_ERR_ALIGN;
  if (workspace_bytes < fa_prefix_fwd_workspace_bytes(B, Hq, Hkv, Nq, Np, Nk, d)) return FA_ERR_WORKSPACE;
  const fa::PrefixPlan p = fa::prefix_plan(B, Hq, Hkv, Nq, Np, Nk, d);
  a.Q = (const __bf16*)Q;
  a.Kp = (const __bf16*)Kprefix;
  a.Vp = (const __bf16*)Vprefix;
  a.K = (const __bf16*)Kcache;
  a.V = (const __bf16*)Vcache;
  a.prefix_table = prefix_table;
  a.O = (__bf16*)O;
  a.LSE = LSE;
  a.Opart = (float*)workspace;
  a.Lpart = a.Opart + (size_t)(p.prefix_shares + p.own_shares) * B * Nq * Hq * d;
  a.nseq = B;
  a.Nq = Nq;
  a.Np = Np;
  a.Hq = Hq;
  a.Hkv = Hkv;
  a.G = Hq / Hkv;
  a.f16 = f16;
  a.causal = causal != 0;
  a.scale = scale;
  a.scale_log2e = scale * fa::kLog2e;
  return launched(fa::launch_prefix(a, d, (hipStream_t)stream));
}

int fa_prefix_fwd(const void* Q, const void* Kprefix, const void* Vprefix, const int32_t* prefix_table, const void* Kcache,
                  const void* Vcache, const int32_t* seqlens_k, const int32_t* block_table, void* O, float* LSE, void* workspace,
                  size_t workspace_bytes, int B, int Hq, int Hkv, int Nq, int Np, int Nk, int d, int page_size, int prefix_pages,
                  int pages_per_seq, float scale, int causal, void* stream) {
  return prefix_fwd_any(0, Q, Kprefix, Vprefix, prefix_table, Kcache, Vcache, seqlens_k, block_table, O, LSE, workspace, workspace_bytes, B,
                        Hq, Hkv, Nq, Np, Nk, d, page_size, prefix_pages, pages_per_seq, scale, causal, stream);
}

int fa_prefix_fwd_f16(const void* Q, const void* Kprefix, const void* Vprefix, const int32_t* prefix_table, const void* Kcache,
                      const void* Vcache, const int32_t* seqlens_k, const int32_t* block_table, void* O, float* LSE, void* workspace,
                      size_t workspace_bytes, int B, int Hq, int Hkv, int Nq, int Np, int Nk, int d, int page_size,
                      int prefix_pages, int pages_per_seq, float scale, int causal, void* stream) {
  return prefix_fwd_any(1, Q, Kprefix, Vprefix, prefix_table, Kcache, Vcache, seqlens_k, block_table, O, LSE, workspace, workspace_bytes, B,
                        Hq, Hkv, Nq, Np, Nk, d, page_size, prefix_pages, pages_per_seq, scale, causal, stream);
}

int fa_cache_append(const void* Knew, const void* Vnew, void* Kcache, void* Vcache, const int32_t* seqlens_k, const int32_t* block_table,
                    float* weights, int32_t* positions, const int32_t* first_position, int B, int Hkv, int Nq, int Nk, int d,
                    int page_size, int pages_per_seq, void* stream) {
  if (!Knew || !Vnew || !Kcache || !Vcache) return FA_ERR_NULL;
  if (Nq <= 0) return FA_ERR_SHAPE;
  if (int e = check_rows(d)) return e;
  fa::AppendArgs a;
  if (int e = set_cache(a.c, seqlens_k, block_table, B, Hkv, Nk, d, page_size, pages_per_seq)) return e;
  if ((double)B * Nq * Hkv * (d / 8) > (double)(1u << 31)) return FA_ERR_SHAPE;
  if (!aligned16(Knew) || !aligned16(Vnew) || !aligned16(Kcache) || !aligned16(Vcache) || !aligned4(weights) || !aligned4(positions) ||
      !aligned4(first_position))
    return FA_ERR_ALIGN;
  a.Kn = (const __bf16*)Knew;
  a.Vn = (const __bf16*)Vnew;
  a.K = (__bf16*)Kcache;
  a.V = (__bf16*)Vcache;
  a.weights = weights;
  a.positions = positions;
  a.first = first_position;
  a.nseq = B;
  a.Nq = Nq;
  return launched(fa::launch_append(a, (hipStream_t)stream));
}

static int cache_weights_any(int f16, const void* Q, const void* Kcache, const float* LSE, const int32_t* seqlens_k,
                             const int32_t* block_table, const int32_t* queries, float* weights, int B, int Hq, int Hkv, int Nq,
                             int Nk, int d, int page_size, int pages_per_seq, long long lse_bs, long long lse_hs, long long lse_qs, float scale,
                         int causal, void* stream) {
  if (!Q || !Kcache || !LSE || !weights) return FA_ERR_NULL;
  if (Nq <= 0) return FA_ERR_SHAPE;
  if (int e = check_common(Hq, Hkv, d, scale, false)) return e;
  fa::WeightsArgs a;
  if (int e = set_cache(a.c, seqlens_k, block_table, B, Hkv, Nk, d, page_size, pages_per_seq)) return e;
  if ((long)Nq * (Hq / Hkv) > (1 << 30)) return FA_ERR_SHAPE;
  if (!aligned16(Q) || !aligned16(Kcache) || !aligned4(LSE) || !aligned4(weights) || !aligned4(queries)) return FA_ERR_ALIGN;
  a.Q = (const __bf16*)Q;
  a.K = (const __bf16*)Kcache;
  a.LSE = LSE;
  a.weights = weights;
  a.queries = queries;
  a.nseq = B;
  a.Nq = Nq;
  a.Hq = Hq;
  a.G = Hq / Hkv;
  a.f16 = f16;
  a.causal = causal != 0;
  a.lse_bs = (long)lse_bs;
  a.lse_hs = (long)lse_hs;
  a.lse_qs = (long)lse_qs;
  a.scale = scale;
  return launched(fa::launch_weights(a, (hipStream_t)stream));
}

int fa_cache_weights(const void* Q, const void* Kcache, const float* LSE, const int32_t* seqlens_k, const int32_t* block_table,
                     const int32_t* queries, float* weights, int B, int Hq, int Hkv, int Nq, int Nk, int d, int page_size,
                     int pages_per_seq, long long lse_bs, long long lse_hs, long long lse_qs, float scale,
                         int causal, void* stream) {
  return cache_weights_any(0, Q, Kcache, LSE, seqlens_k, block_table, queries, weights, B, Hq, Hkv, Nq, Nk, d, page_size, pages_per_seq,
                           lse_bs, lse_hs, lse_qs, scale, causal, stream);
}

int fa_cache_weights_f16(const void* Q, const void* Kcache, const float* LSE, const int32_t* seqlens_k, const int32_t* block_table,
                         const int32_t* queries, float* weights, int B, int Hq, int Hkv, int Nq, int Nk, int d, int page_size,
                         int pages_per_seq, long long lse_bs, long long lse_hs, long long lse_qs, float scale,
                         int causal, void* stream) {
  return cache_weights_any(1, Q, Kcache, LSE, seqlens_k, block_table, queries, weights, B, Hq, Hkv, Nq, Nk, d, page_size, pages_per_seq,
                           lse_bs, lse_hs, lse_qs, scale, causal, stream);
}

static int evict_room(int Nk, int budget) { return Nk <= budget ? 0 : (Nk - budget < budget ? Nk - budget : budget); }

size_t fa_cache_evict_workspace_bytes(int B, int Hkv, int Nk, int budget) {
  if (B <= 0 || Hkv <= 0 || Nk <= 0 || budget <= 0) return 0;
  return round_up((size_t)B * Hkv * (1 + 2 * (size_t)evict_room(Nk, budget)) * sizeof(int32_t), 256);
}

int fa_cache_evict(void* Kcache, void* Vcache, const float* weights, const int32_t* positions, const int32_t* seqlens_k,
                   const int32_t* block_table, float* weights_out, int32_t* positions_out, int32_t* seqlens_out, void* workspace,
                   size_t workspace_bytes, int B, int Hkv, int Nk, int d, int budget, int sinks, int recent, int page_size,
                   int pages_per_seq, void* stream) {
  if (!Kcache || !Vcache || !weights || !positions || !weights_out || !positions_out || !seqlens_out || !workspace) return FA_ERR_NULL;
  if (budget <= 0 || sinks < 0 || recent < 0 || (long)sinks + recent > budget) return FA_ERR_SHAPE;
  if (int e = check_rows(d)) return e;
  fa::EvictArgs a;
  if (int e = set_cache(a.c, seqlens_k, block_table, B, Hkv, Nk, d, page_size, pages_per_seq)) return e;
  if (!aligned16(Kcache) || !aligned16(Vcache) || !aligned4(weights) || !aligned4(positions) || !aligned4(weights_out) ||
      !aligned4(positions_out) || !aligned4(seqlens_out) || !aligned4(workspace))
    return FA_ERR_ALIGN;
  if (workspace_bytes < fa_cache_evict_workspace_bytes(B, Hkv, Nk, budget)) return FA_ERR_WORKSPACE;
  a.K = (__bf16*)Kcache;
  a.V = (__bf16*)Vcache;
  a.weights = weights;
  a.positions = positions;
  a.weights_out = weights_out;
  a.positions_out = positions_out;
  a.lens_out = seqlens_out;
  a.moves = (int32_t*)workspace;
  a.nseq = B;
  a.budget = budget;
  a.sinks = sinks;
  a.recent = recent;
  a.room = evict_room(Nk, budget);
  return launched(fa::launch_evict(a, (hipStream_t)stream));
}

size_t fa_verify_drafts_workspace_bytes(int B, int k, int V) {
  if (B <= 0 || k < 0 || V <= 0 || V > FA_VERIFY_MAX_VOCAB) return 0;
  return round_up(fa::verify_workspace(B, k, V), 256);
}

int fa_verify_drafts(const int32_t* draft_tokens, const void* draft_probs, const void* target, const float* uniform, int32_t* tokens,
                     int32_t* accepted, void* workspace, size_t workspace_bytes, int B, int k, int V, long long draft_stride,
                     long long target_stride, int draft_type, int target_type, int target_is_logits, float inv_temperature,
                     void* stream) {
  if ((k > 0 && !draft_tokens) || !target || !uniform || !tokens || !accepted || !workspace) return FA_ERR_NULL;
  if (B <= 0 || k < 0 || V <= 0 || V > FA_VERIFY_MAX_VOCAB || (long)B * ((long)k + 1) > (1 << 20)) return FA_ERR_SHAPE;
  if (target_stride < V || (k > 0 && draft_probs && draft_stride < V)) return FA_ERR_SHAPE;
  if (!(inv_temperature > 0.f) || !std::isfinite(inv_temperature)) return FA_ERR_SHAPE;
  auto misplaced = [](const void* p, int type) { return (reinterpret_cast<uintptr_t>(p) & (type == FA_TYPE_F32 ? 3u : 1u)) != 0; };
  if (target_type < FA_TYPE_F32 || target_type > FA_TYPE_F16 || (draft_probs && (draft_type < FA_TYPE_F32 || draft_type > FA_TYPE_F16)))
    return FA_ERR_UNSUPPORTED;
  if (misplaced(target, target_type) || misplaced(draft_probs, draft_type) || !aligned4(draft_tokens) || !aligned4(uniform) ||
      !aligned4(tokens) || !aligned4(accepted) || (reinterpret_cast<uintptr_t>(workspace) & 7u))
    return FA_ERR_ALIGN;
  if (workspace_bytes < fa_verify_drafts_workspace_bytes(B, k, V)) return FA_ERR_WORKSPACE;
  const fa::VerifyArgs a = {draft_tokens, k > 0 ? draft_probs : nullptr, target, uniform, tokens, accepted, workspace, B, k, V, draft_type,
                            target_type, target_is_logits != 0, (long)draft_stride, (long)target_stride, target_is_logits ? inv_temperature : 1.f};
  return launched(fa::launch_verify(a, (hipStream_t)stream));
}

// ---- caches held in 4 or 8 bits, rotary positions

static int set_qcache(fa::QCacheView& c, const void* Kc, const void* Ks, const void* Vc, const void* Vs, const int32_t* lens, const int32_t* table,
                      int B, int Hkv, int Nk, int d, int k_bits, int v_bits, int page_size, int pages_per_seq) {
  if ((k_bits != 4 && k_bits != 8) || (v_bits != 4 && v_bits != 8)) return FA_ERR_UNSUPPORTED;
  if (int e = set_cache(c.c, lens, table, B, Hkv, Nk, d, page_size, pages_per_seq)) return e;
  if (!aligned16(Kc) || !aligned16(Vc) || !aligned4(Ks) || !aligned4(Vs)) return FA_ERR_ALIGN;
  c.Kc = (uint8_t*)Kc;
  c.Ks = (uint8_t*)Ks;
  c.Vc = (uint8_t*)Vc;
  c.Vs = (uint8_t*)Vs;
  c.k_bits = k_bits;
  c.v_bits = v_bits;
  return FA_OK;
}
static int check_blocks(int d) { return d <= 0 ? FA_ERR_SHAPE : (d % 32 || d > 256 ? FA_ERR_UNSUPPORTED : FA_OK); }
static int check_16bit(int type) { return type == FA_TYPE_BF16 || type == FA_TYPE_F16 ? FA_OK : FA_ERR_UNSUPPORTED; }

int fa_qcache_append(const void* Knew, const void* Vnew, void* Kcodes, void* Kscales, void* Vcodes, void* Vscales, void* Kout, void* Vout,
                     const int32_t* seqlens_k, const int32_t* block_table, int B, int Hkv, int Nq, int Nk, int d, int k_bits, int v_bits,
                     int page_size, int pages_per_seq, long long k_batch_stride, long long k_token_stride, long long k_head_stride,
                     long long v_batch_stride, long long v_token_stride, long long v_head_stride, int type, void* stream) {
  if (!Knew || !Vnew || !Kcodes || !Kscales || !Vcodes || !Vscales) return FA_ERR_NULL;
  if (Nq <= 0) return FA_ERR_SHAPE;
  if (int e = check_blocks(d)) return e;
  if (int e = check_16bit(type)) return e;
  fa::QAppendArgs a;
  if (int e = set_qcache(a.c, Kcodes, Kscales, Vcodes, Vscales, seqlens_k, block_table, B, Hkv, Nk, d, k_bits, v_bits, page_size, pages_per_seq))
    return e;
  if ((double)B * Nq * Hkv * (d / 8) > (double)(1u << 30)) return FA_ERR_SHAPE;
  for (long long x : {k_batch_stride, k_token_stride, k_head_stride, v_batch_stride, v_token_stride, v_head_stride})
    if (x < 0 || x % 8) return FA_ERR_SHAPE;
  if (!aligned16(Knew) || !aligned16(Vnew) || !aligned16(Kout) || !aligned16(Vout)) return FA_ERR_ALIGN;
  a.Kn = (const __bf16*)Knew;
  a.Vn = (const __bf16*)Vnew;
  a.Kout = (__bf16*)Kout;
  a.Vout = (__bf16*)Vout;
  a.k_bs = (long)k_batch_stride;
  a.k_ts = (long)k_token_stride;
  a.k_hs = (long)k_head_stride;
  a.v_bs = (long)v_batch_stride;
  a.v_ts = (long)v_token_stride;
  a.v_hs = (long)v_head_stride;
  a.nseq = B;
  a.Nq = Nq;
  a.f16 = type == FA_TYPE_F16;
  return launched(fa::launch_qappend(a, (hipStream_t)stream));
}

int fa_qcache_read(const void* Kcodes, const void* Kscales, const void* Vcodes, const void* Vscales, void* K, void* V,
                   const int32_t* seqlens_k, const int32_t* block_table, const int32_t* first, const int32_t* cu_seqlens, int B, int Hkv, int N,
                   int Nk, int d, int k_bits, int v_bits, int page_size, int pages_per_seq, int type, void* stream) {
  if (!Kcodes || !Kscales || !Vcodes || !Vscales || !K || !V) return FA_ERR_NULL;
  if (N <= 0 || (first && cu_seqlens)) return FA_ERR_SHAPE;
  if (int e = check_blocks(d)) return e;
  if (int e = check_16bit(type)) return e;
  fa::QReadArgs a;
  if (int e = set_qcache(a.c, Kcodes, Kscales, Vcodes, Vscales, seqlens_k, block_table, B, Hkv, Nk, d, k_bits, v_bits, page_size, pages_per_seq))
    return e;
  const long rows = cu_seqlens && Nk < N ? Nk : N;  // (of one sequence, at most)
  if ((double)B * Hkv * ((rows + 63) / 64) >= (double)(1u << 24)) return FA_ERR_SHAPE;  // (threads of a grid are counted in 32 bits)
  if (!aligned16(K) || !aligned16(V) || !aligned4(first) || !aligned4(cu_seqlens)) return FA_ERR_ALIGN;
  a.K = (__bf16*)K;
  a.V = (__bf16*)V;
  a.first = first;
  a.cu = cu_seqlens;
  a.nseq = B;
  a.N = N;
  a.total = N;
  a.f16 = type == FA_TYPE_F16;
  return launched(fa::launch_qread(a, (hipStream_t)stream));
}

static bool qcache_fwd_sizes(int B, int Hq, int Hkv, int Nq, int Nk) {
  if (B <= 0 || Hq <= 0 || Hkv <= 0 || Hq % Hkv || Nq <= 0 || Nk <= 0 || Nk > FA_CACHE_MAX_SLOTS || Hkv > (1 << 16)) return false;
  // (rows as the blocks have them: the merge's grid goes by these, and threads of a grid are counted in 32 bits)
  const long rows = (long)Nq * (Hq / Hkv), block = rows <= 16 ? 16 : (rows <= 64 ? 32 : 128);
  return (double)B * Hkv * (double)((rows + block - 1) / block * block) <= (double)(1 << 26) &&
         (double)B * Hkv * ((double)rows / 16 + 1) * (Nk / 128 + 1) < (double)0x7fffffff;
}

size_t fa_qcache_fwd_workspace_bytes(int B, int Hq, int Hkv, int Nq, int Nk, int d) {
  if (!qcache_fwd_sizes(B, Hq, Hkv, Nq, Nk) || (d != 64 && d != 128)) return 0;
  const fa::QAttendPlan p = fa::qattend_plan(B, Hq, Hkv, Nq, Nk, d, 0);
  if (p.slots == 0) return 0;
  return round_up((size_t)p.slots * p.rows * (d + 1) * sizeof(float) + (size_t)B * Hkv * p.blocks * sizeof(fa::QAttendArgs::Unit), 256);
}

int fa_qcache_fwd(const void* Q, const void* Kcodes, const void* Kscales, const void* Vcodes, const void* Vscales, const int32_t* seqlens_k,
                  const int32_t* block_table, void* O, float* LSE, void* workspace, size_t workspace_bytes, int B, int Hq, int Hkv, int Nq,
                  int Nk, int d, int k_bits, int v_bits, int page_size, int pages_per_seq, float scale, int causal, int type, void* stream) {
  if (!Q || !Kcodes || !Kscales || !Vcodes || !Vscales || !O || !LSE) return FA_ERR_NULL;
  if (int e = check_common(Hq, Hkv, d, scale, false)) return e;
  if (!qcache_fwd_sizes(B, Hq, Hkv, Nq, Nk)) return FA_ERR_SHAPE;
  if (int e = check_16bit(type)) return e;
  fa::QAttendArgs a;
  if (int e = set_qcache(a.c, Kcodes, Kscales, Vcodes, Vscales, seqlens_k, block_table, B, Hkv, Nk, d, k_bits, v_bits, page_size, pages_per_seq))
    return e;
  if (!aligned16(Q) || !aligned16(O) || !aligned4(LSE) || !aligned16(workspace)) return FA_ERR_ALIGN;
  const size_t need = fa_qcache_fwd_workspace_bytes(B, Hq, Hkv, Nq, Nk, d);
  if (need && !workspace) return FA_ERR_NULL;
  if (workspace_bytes < need) return FA_ERR_WORKSPACE;
  const fa::QAttendPlan p = fa::qattend_plan(B, Hq, Hkv, Nq, Nk, d, 0);
  a.Q = (const __bf16*)Q;
  a.O = (__bf16*)O;
  a.LSE = LSE;
  a.Opart = (float*)workspace;
  a.Lpart = a.Opart + (size_t)p.slots * p.rows * d;
  a.units = (fa::QAttendArgs::Unit*)(a.Lpart + (size_t)p.slots * p.rows);
  a.nseq = B;
  a.Nq = Nq;
  a.Hq = Hq;
  a.G = Hq / Hkv;
  a.f16 = type == FA_TYPE_F16;
  a.causal = causal != 0;
  a.scale = scale;
  a.scale_log2e = scale * fa::kLog2e;
  return launched(fa::launch_qattend(a, (hipStream_t)stream));
}

static int rope_any(int inverse, const void* Q, const void* K, void* Qout, void* Kout, const int32_t* positions, const float* inv_freq,
                    const int32_t* axis, int B, int N, int Hq, int Hkv, int d, int pairs, int axes, int neighbours, const long long* strides,
                    long long axis_stride, long long batch_stride, int type, void* stream) {
  if (!Q || !Qout || !positions || !inv_freq || !strides || (K && !Kout)) return FA_ERR_NULL;
  if (type < FA_TYPE_F32 || type > FA_TYPE_F16) return FA_ERR_UNSUPPORTED;
  if (d <= 0) return FA_ERR_SHAPE;
  if (d % 8 || d > 256) return FA_ERR_UNSUPPORTED;
  if (B <= 0 || N <= 0 || (double)B * N > (double)0x7fffffff || Hq <= 0 || (K && Hkv <= 0) || (long)Hq + (K ? Hkv : 0) > (1 << 20) || pairs <= 0 ||
      2 * (long)pairs > d || axes <= 0 || axis_stride < 0 || batch_stride < 0)
    return FA_ERR_SHAPE;
  const int size = type == FA_TYPE_F32 ? 4 : 2;
  const void* at[4] = {Q, Qout, K, Kout};
  // as many elements at once as divide the pairs, the strides and the addresses, 16 bytes at most
  int vec = 16 / size;
  while (pairs % vec) vec /= 2;
  for (int i = 0; i < (K ? 4 : 2); ++i) {
    const uintptr_t p = reinterpret_cast<uintptr_t>(at[i]);
    if (p % size) return FA_ERR_ALIGN;
    while (p % (vec * size)) vec /= 2;
    for (int j = 0; j < 3; ++j) {
      if (strides[3 * i + j] < 0) return FA_ERR_SHAPE;
      while (strides[3 * i + j] % vec) vec /= 2;
    }
  }
  if (!aligned4(positions) || !aligned4(inv_freq) || !aligned4(axis)) return FA_ERR_ALIGN;
  fa::RopeArgs a;
  for (int i = 0; i < 2; ++i) {
    const long long* s = strides + 6 * i;
    if (i && !K) a.t[i] = {nullptr, nullptr, 0, 0, 0, 0, 0, 0, 0};
    else a.t[i] = {at[2 * i], (void*)at[2 * i + 1], i ? Hkv : Hq, (long)s[0], (long)s[1], (long)s[2], (long)s[3], (long)s[4], (long)s[5]};
  }
  a.positions = positions;
  a.inv_freq = inv_freq;
  a.axis = axis;
  a.p_as = (long)axis_stride;
  a.p_bs = (long)batch_stride;
  a.nseq = B;
  a.N = N;
  a.d = d;
  a.pairs = pairs;
  a.axes = axes;
  a.type = type;
  a.neighbours = neighbours != 0;
  a.inverse = inverse;
  a.vec = vec;
  return launched(fa::launch_rope(a, (hipStream_t)stream));
}

int fa_rope_fwd(const void* Q, const void* K, void* Qout, void* Kout, const int32_t* positions, const float* inv_freq, const int32_t* axis,
                int B, int N, int Hq, int Hkv, int d, int pairs, int axes, int neighbours, const long long* strides,
                long long axis_stride, long long batch_stride, int type, void* stream) {
  return rope_any(0, Q, K, Qout, Kout, positions, inv_freq, axis, B, N, Hq, Hkv, d, pairs, axes, neighbours, strides, axis_stride,
                  batch_stride, type, stream);
}

int fa_rope_bwd(const void* dQout, const void* dKout, void* dQ, void* dK, const int32_t* positions, const float* inv_freq, const int32_t* axis,
                int B, int N, int Hq, int Hkv, int d, int pairs, int axes, int neighbours, const long long* strides,
                long long axis_stride, long long batch_stride, int type, void* stream) {
  return rope_any(1, dQout, dKout, dQ, dK, positions, inv_freq, axis, B, N, Hq, Hkv, d, pairs, axes, neighbours, strides, axis_stride,
                  batch_stride, type, stream);
}

size_t fa_mfma_probe_scratch_bytes(void) { return 16 + (size_t)256 * 512 * sizeof(float); }

int fa_mfma_probe(int iters, int random_operands, void* scratch, void* stream) {
  if (!scratch) return FA_ERR_NULL;
  if ((uintptr_t)scratch % 16 != 0) return FA_ERR_ALIGN;
  if (iters < 1) return FA_ERR_SHAPE;
  hipError_t e = fa::launch_mfma_probe((float*)((char*)scratch + 16), (long long*)scratch, 256, iters,
                                       random_operands, (hipStream_t)stream);
  if (e != hipSuccess) {
    g_last_hip_error = (int)e;
    return FA_ERR_LAUNCH;
  }
  return FA_OK;
}

}  // extern "C"
