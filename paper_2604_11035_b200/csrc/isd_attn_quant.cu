// isd_attn_quant: strict-causal attention of every slot's query block against its paged 4-bit cache (Sec. 3.1 mask).
// One CTA per (slot, kv head), a page at a time, fp32 on the CUDA cores: online softmax with two threads per row.
#include "isd_quant.cuh"

namespace {

struct QuantAttnParams {
  int B, Q, N, Hq, Hkv, G, max_pages;
  float scale2;  // sm_scale * log2(e)
  const int32_t* ctx_len;
  const int32_t* n_ver;
  const uint8_t* active;
  const int32_t* page_table;
  const uint32_t* slot_status;
  const __nv_bfloat16* q;
  __nv_bfloat16* out;
  float* lse;
  const uint8_t* pool;
};

__global__ void __launch_bounds__(256) attn_quant_kernel(const QuantAttnParams P) {
  __shared__ float sk[ISD_PAGE][ISD_HEAD_DIM], sv[ISD_PAGE][ISD_HEAD_DIM], ss[128][ISD_PAGE + 1];
  const int b = blockIdx.x, g = blockIdx.y;
  pdl_wait();
  pdl_launch_dependents();
  if (!P.active[b] || (P.slot_status[b] & (ISD_ST_BAD_PAGE_ID | ISD_ST_SLOT_CAPACITY))) return;
  const int nv = P.n_ver[b];
  if (nv < 0 || nv > P.N - 1) return;
  const int ql = nv + P.N, ctx = P.ctx_len[b];
  const int row = threadIdx.x >> 1, half = threadIdx.x & 1;
  const int r = row / P.G, h = g * P.G + row % P.G;
  const bool ok = r < ql;
  const size_t at = ((size_t)b * P.Q + (ok ? r : 0)) * P.Hq + h;
  float m = -INFINITY, l = 0.f, o[64];
#pragma unroll
  for (int d = 0; d < 64; ++d) o[d] = 0.f;
  for (int pg = 0; pg * ISD_PAGE < ctx + ql; ++pg) {
    const uint8_t* tile = P.pool + ((size_t)P.page_table[(size_t)b * P.max_pages + pg] * P.Hkv + g) * kQTile;
    const __nv_bfloat16* meta = reinterpret_cast<const __nv_bfloat16*>(tile + kQOffMeta);
    __syncthreads();
    for (int i = threadIdx.x; i < ISD_PAGE * ISD_HEAD_DIM; i += 256) {
      const int t = i / ISD_HEAD_DIM, d = i % ISD_HEAD_DIM;
      const uint32_t kw = reinterpret_cast<const uint32_t*>(tile)[(d >> 5) * 64 + t * 4 + ((d >> 3) & 3)];
      const uint32_t vw = reinterpret_cast<const uint32_t*>(tile + kQOffV)[d * 2 + (t >> 3)];
      const int kc = (kw >> (4 * ((d & 7) >> 1) + 16 * (d & 1))) & 15, vc = (vw >> (4 * ((t & 7) >> 1) + 16 * (t & 1))) & 15;
      const bool in = pg * ISD_PAGE + t < ctx + ql;
      sk[t][d] = __bfloat162float(meta[t]) * ((float)kc - (__bfloat162float(meta[16 + t]) - 128.f));
      sv[t][d] = in ? __bfloat162float(meta[32 + t]) * ((float)vc - (__bfloat162float(meta[48 + t]) - 128.f)) : 0.f;
    }
    __syncthreads();
    float s[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) s[j] = 0.f;
    for (int d = 0; d < ISD_HEAD_DIM; ++d) {
      const float x = __bfloat162float(P.q[at * ISD_HEAD_DIM + d]);
#pragma unroll
      for (int j = 0; j < 8; ++j) s[j] = fmaf(x, sk[half * 8 + j][d], s[j]);
    }
    float mx = m;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      s[j] = pg * ISD_PAGE + half * 8 + j <= ctx + r ? s[j] * P.scale2 : -INFINITY;
      mx = fmaxf(mx, s[j]);
    }
    mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
    const float ref = mx == -INFINITY ? 0.f : mx, keep = exp2f(m - ref);
    m = mx;
    l *= keep;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float p = exp2f(s[j] - ref);
      l += p;
      ss[row][half * 8 + j] = p;
    }
    __syncwarp();
#pragma unroll
    for (int d = 0; d < 64; ++d) {
      float a = o[d] * keep;
#pragma unroll 4
      for (int j = 0; j < ISD_PAGE; ++j) a = fmaf(ss[row][j], sv[j][half * 64 + d], a);
      o[d] = a;
    }
  }
  l += __shfl_xor_sync(0xffffffffu, l, 1);
  if (!ok) return;
  for (int d = 0; d < 64; ++d) P.out[at * ISD_HEAD_DIM + half * 64 + d] = __float2bfloat16_rn(o[d] / l);
  if (P.lse && half == 0) P.lse[at] = (m + log2f(l)) * 0.6931471805599453f;
}

}  // namespace

int isd_attn_quant_create(isd_ctx*) { return ISD_OK; }
void isd_attn_quant_destroy(isd_ctx*) {}

int isd_launch_attn_quant(isd_ctx* ctx, const isd_batch_state* st, const void* q, const void*, const void*,
                          void* kv_pool, void* out, float* lse, cudaStream_t stream) {
  const isd_config& c = ctx->cfg;
  QuantAttnParams P;
  P.B = c.batch; P.Q = ctx->Q; P.N = c.stride; P.Hq = c.n_q_heads; P.Hkv = c.n_kv_heads; P.G = ctx->G; P.max_pages = c.max_pages_per_slot;
  P.scale2 = ctx->sm_scale * 1.4426950408889634f;
  P.ctx_len = st->ctx_len; P.n_ver = st->n_ver; P.active = st->active; P.page_table = st->page_table; P.slot_status = st->slot_status;
  P.q = (const __nv_bfloat16*)q; P.out = (__nv_bfloat16*)out; P.lse = lse; P.pool = (const uint8_t*)kv_pool;
  const cudaError_t e = isd_launch_pdl(attn_quant_kernel, dim3(c.batch, c.n_kv_heads), dim3(256), 0, stream, P);
  ctx->launches++;
  return e == cudaSuccess ? ISD_OK : ISD_ERR_CUDA;
}
