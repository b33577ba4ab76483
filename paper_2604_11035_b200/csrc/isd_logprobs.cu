// isd_logprobs: log probability of given tokens, entropy and top alternatives of their rows' laws.
// One CTA per entry: a pass for the maximum and the sums, then a pass per alternative.
#include "isd_internal.cuh"

namespace {

struct LogprobsParams {
  const void* logits;
  int64_t logits_rows;
  const int32_t* rows;
  const int32_t* tokens;
  int n, V, top_n, dtype;
  float inv_t;
  float* logprob;
  float* entropy;
  int32_t* top_id;
  float* top_logprob;
  uint32_t* global_status;
};

constexpr int kLpThreads = 256;

template <class T, class Op>
__device__ T block_reduce(T v, T* sm, Op op) {
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) v = op(v, __shfl_xor_sync(0xffffffffu, v, off));
  __syncthreads();
  if ((threadIdx.x & 31) == 0) sm[threadIdx.x >> 5] = v;
  __syncthreads();
  v = sm[0];
#pragma unroll
  for (int w = 1; w < kLpThreads / 32; ++w) v = op(v, sm[w]);
  return v;
}

// order-preserving code of a float (-0 and 0 alike), and the sort key of (value, index): larger value first, then lower index
__device__ __forceinline__ uint32_t order_code(float x) {
  const uint32_t u = __float_as_uint(x + 0.f);
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

__global__ void __launch_bounds__(kLpThreads) logprobs_kernel(const LogprobsParams P) {
  __shared__ float smf[8];
  __shared__ unsigned long long smk[8];
  pdl_wait();
  pdl_launch_dependents();
  const int i = blockIdx.x, tok = P.tokens[i];
  const int64_t row = P.rows ? P.rows[i] : i;
  uint32_t why = 0;
  if (tok >= P.V || (tok >= 0 && (row < 0 || row >= P.logits_rows))) why = ISD_ST_BAD_TOKEN_ID;
  bool skip = tok < 0 || why;
  float m = -INFINITY, s = 0.f, w = 0.f;
  const size_t base = skip ? 0 : (size_t)row * P.V;
  if (!skip) {
    float bad = 0.f;
    for (int v = threadIdx.x; v < P.V; v += kLpThreads) {
      const float x = load_logit(P.logits, P.dtype, base + v);
      if (!(x < INFINITY)) bad = 1.f;
      m = fmaxf(m, x);
    }
    auto fmx = [](float a, float b) { return fmaxf(a, b); };
    bad = block_reduce(bad, smf, fmx);
    m = block_reduce(m, smf, fmx);
    if (bad > 0.f || m == -INFINITY) {
      why = ISD_ST_NONFINITE_LOGIT;
      skip = true;
    }
  }
  if (!skip) {
    for (int v = threadIdx.x; v < P.V; v += kLpThreads) {
      const float d = (load_logit(P.logits, P.dtype, base + v) - m) * P.inv_t;
      const float e = expf(d);
      s += e;
      if (e > 0.f) w = fmaf(e, d, w);
    }
    auto add = [](float a, float b) { return a + b; };
    s = block_reduce(s, smf, add);
    w = block_reduce(w, smf, add);
  }
  const float ls = logf(s);
  if (threadIdx.x == 0) {
    if (why) atomicOr(P.global_status, why);
    P.logprob[i] = skip ? NAN : (load_logit(P.logits, P.dtype, base + tok) - m) * P.inv_t - ls;
    if (P.entropy) P.entropy[i] = skip ? NAN : ls - w / s;
  }
  unsigned long long last = ~0ull;
  for (int k = 0; k < P.top_n; ++k) {
    unsigned long long best = 0;
    if (!skip)
      for (int v = threadIdx.x; v < P.V; v += kLpThreads) {
        const unsigned long long key =
            ((unsigned long long)order_code(load_logit(P.logits, P.dtype, base + v)) << 32) | (0xFFFFFFFFu - (uint32_t)v);
        if (key < last && key > best) best = key;
      }
    best = block_reduce(best, smk, [](unsigned long long a, unsigned long long b) { return a > b ? a : b; });
    last = best;
    if (threadIdx.x == 0) {
      const int id = (int)(0xFFFFFFFFu - (uint32_t)best);
      P.top_id[(size_t)i * P.top_n + k] = skip ? -1 : id;
      P.top_logprob[(size_t)i * P.top_n + k] = skip ? NAN : (load_logit(P.logits, P.dtype, base + id) - m) * P.inv_t - ls;
    }
  }
}

}  // namespace

int isd_logprobs_create(isd_ctx*) { return ISD_OK; }
void isd_logprobs_destroy(isd_ctx*) {}

int isd_launch_logprobs(isd_ctx* ctx, const isd_logprobs_args* a, cudaStream_t stream) {
  LogprobsParams P;
  P.logits = a->logits; P.logits_rows = a->logits_rows; P.rows = a->rows; P.tokens = a->tokens; P.n = a->n;
  P.V = ctx->cfg.vocab; P.top_n = a->top_n; P.dtype = ctx->cfg.logits_dtype; P.inv_t = ctx->cfg.inv_temperature;
  P.logprob = a->logprob; P.entropy = a->entropy; P.top_id = a->top_id; P.top_logprob = a->top_logprob;
  P.global_status = ctx->global_status;
  const cudaError_t e = isd_launch_pdl(logprobs_kernel, dim3(a->n), dim3(kLpThreads), 0, stream, P);
  ctx->launches++;
  return e == cudaSuccess ? ISD_OK : ISD_ERR_CUDA;
}
