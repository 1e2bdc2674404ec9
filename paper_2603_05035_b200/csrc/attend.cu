// Attention of one new token per sequence over a paged key-value cache.
//   o = sum_j p_j v_j,  p_j = exp(s_j - m) / l,  s_j = scale q . k_j,  m = max_j s_j,  l = sum_j exp(s_j - m)
// One pass over the keys and values with the running maximum and sum of the softmax.
// A CTA takes one query head of one sequence; its warps take every eighth position each, lanes hold the components, and the
// warps' sums are joined at the end.
#include "common.cuh"
#include "vec8.cuh"

namespace gelo {

namespace {

constexpr int kWarps = 8;
constexpr int kMaxDim = 256;
constexpr float kNone = -INFINITY;

struct AttendArgs {
    const void *q, *k, *v;
    void* o;
    float* lse;
    const int *len, *table;
    int* status;
    long long page_stride, token_stride, head_stride;
    int ldq, ldo, q_heads, group, dh;
    int pages, page_size, seqs, max_pages, table_ld, window;
    float scale, v_scale;                                     // scale: of the logits, the keys' scale included
};

template <typename T, typename C>
__global__ void __launch_bounds__(32 * kWarps) attend_kernel(const AttendArgs p)
{
    __shared__ float part[kWarps][kMaxDim + 2];
    chain_next();
    chain_wait();
    const int head = blockIdx.x, seq = blockIdx.y, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    long long len = p.len[seq];
    if (len > (long long)p.max_pages * p.page_size) {
        len = (long long)p.max_pages * p.page_size;
        if (threadIdx.x == 0) atomicCAS(p.status, 0, (int)GELO_ERR_INVALID);
    }
    const long long first = p.window && len > p.window ? len - p.window : 0;
    const T* q = static_cast<const T*>(p.q) + (size_t)seq * p.ldq + (size_t)head * p.dh;
    const long long at_head = (head / p.group) * p.head_stride;
    float qr[8], acc[8], m = kNone, l = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        qr[i] = lane + 32 * i < p.dh ? widen_at(q, lane + 32 * i) : 0.0f;
        acc[i] = 0.0f;
    }
    for (long long t = first + warp; t < len; t += kWarps) {
        const int page = p.table[(size_t)seq * p.table_ld + t / p.page_size];
        if (page < 0 || page >= p.pages) {
            if (lane == 0) atomicCAS(p.status, 0, (int)GELO_ERR_INVALID);
            continue;
        }
        const long long at = page * p.page_stride + (t % p.page_size) * p.token_stride + at_head;
        float s = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (lane + 32 * i < p.dh) s = fmaf(qr[i], widen_at(static_cast<const C*>(p.k) + at, lane + 32 * i), s);
#pragma unroll
        for (int off = 16; off > 0; off >>= 1) s += __shfl_xor_sync(0xffffffffu, s, off);
        s *= p.scale;
        const float top = fmaxf(m, s);
        const float base = top == kNone ? 0.0f : top;
        const float keep = expf(m - base), e = expf(s - base);
        m = top;
        l = l * keep + e;
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (lane + 32 * i < p.dh) acc[i] = fmaf(e, widen_at(static_cast<const C*>(p.v) + at, lane + 32 * i), acc[i] * keep);
    }
    if (lane == 0) { part[warp][kMaxDim] = m; part[warp][kMaxDim + 1] = l; }
#pragma unroll
    for (int i = 0; i < 8; ++i) part[warp][lane + 32 * i] = acc[i];
    __syncthreads();
    float top = kNone, sum = 0.0f, o = 0.0f;
    for (int w = 0; w < kWarps; ++w) top = fmaxf(top, part[w][kMaxDim]);
    const float base = top == kNone ? 0.0f : top;
    for (int w = 0; w < kWarps; ++w) {
        const float f = expf(part[w][kMaxDim] - base);
        sum += f * part[w][kMaxDim + 1];
        o += f * part[w][threadIdx.x];
    }
    if (threadIdx.x < p.dh)
        round_to(sum > 0.0f || sum != sum ? o / sum * p.v_scale : 0.0f, static_cast<T*>(p.o) + (size_t)seq * p.ldo + (size_t)head * p.dh + threadIdx.x);
    if (p.lse && threadIdx.x == 0) p.lse[(size_t)seq * p.q_heads + head] = base + logf(sum);
}

template <typename T, typename C>
int launch_as(gelo_ctx* ctx, const AttendArgs& p, cudaStream_t st)
{
    GELO_TRY(launch_chained(ctx, attend_kernel<T, C>, dim3(p.q_heads, p.seqs), 32 * kWarps, 0, st, p));
    return after_launch(ctx);
}

}  // namespace

size_t attend_workspace_bytes() { return 1024; }

int launch_paged_attention(gelo_ctx* ctx, const gelo_kv_cache& kv, const void* q, int ldq, int q_heads, const int* len, float scale, int window,
                           int dtype, void* o, int ldo, float* lse, void* ws, cudaStream_t st)
{
    (void)ws;
    if (kv.seqs > 65535) return GELO_ERR_UNSUPPORTED;
    AttendArgs p;
    p.q = q; p.k = kv.k_dev; p.v = kv.v_dev; p.o = o; p.lse = lse;
    p.len = len; p.table = kv.table_dev; p.status = ctx->status_dev;
    p.page_stride = kv.page_stride; p.token_stride = kv.token_stride; p.head_stride = kv.head_stride;
    p.ldq = ldq; p.ldo = ldo; p.q_heads = q_heads; p.group = q_heads / kv.kv_heads; p.dh = kv.head_dim;
    p.pages = kv.pages; p.page_size = kv.page_size; p.seqs = kv.seqs; p.max_pages = kv.max_pages; p.table_ld = kv.table_ld;
    p.window = window; p.scale = scale * kv.k_scale; p.v_scale = kv.v_scale;
    const bool narrow = kv.dtype == GELO_E4M3;
    if (dtype == GELO_BF16) return narrow ? launch_as<__nv_bfloat16, uint8_t>(ctx, p, st) : launch_as<__nv_bfloat16, __nv_bfloat16>(ctx, p, st);
    if (dtype == GELO_F16) return narrow ? launch_as<__half, uint8_t>(ctx, p, st) : launch_as<__half, __half>(ctx, p, st);
    return launch_as<float, float>(ctx, p, st);
}

}  // namespace gelo
