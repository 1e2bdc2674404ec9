// Rotary positions, and keys and values appended to a paged cache on the way.
//   x_a' = (x_a cos - x_b sin) m,  x_b' = (x_b cos + x_a sin) m,   angle = 2 pi position turns[pair]
// A CTA takes one token: its threads first work out the cosines and sines of all pairs, which all heads share, then stream the heads
// of Q, K and V through.  position * turns is formed and reduced to one circle exactly, as a pair of binary64 (a position times an fp32 frequency is off
// by position * 2^-24); the cosine and sine are binary64 too and then rounded once; the rest is fp32.  Every pair belongs to one thread, which reads both values before it writes either, so Q may be
// rotated in place.  Bound by HBM: Q, K and V in, all three out.  4096 tokens of 32 heads of 128 in bf16, 201 MB: 37.5 us, 82% of a copy's rate; 64 tokens 4 us.
// Threads take the pieces of all heads in a simple loop: a thread that holds several pieces in flight takes the registers of
// the warps that hide the loads (two to four pieces 43 to 66 us), and fewer instructions per piece gain nothing.
// Pieces are eight components wide where the layout allows it (interleaved, or a `rot` of whole sixteens: 112 of 128 43 us), else one (120 of 128 82 us).
#include "common.cuh"
#include "vec8.cuh"

namespace gelo {

namespace {

constexpr int kThreads = 256;
constexpr int kMaxPairs = 128;                                // head_dim <= 256

struct RotateArgs {
    const void *q, *k, *v;
    void *q_out, *k_cache, *v_cache;
    long long page_stride, token_stride, head_stride;
    const double* turns;
    const int *seq, *pos, *table;
    int* status;
    int ldq, ldk, ldv, ldqo;
    int q_heads, kv_heads, dh, rot, interleaved;
    int pages, page_size, seqs, max_pages, table_ld;
    float magnitude, k_scale, v_scale;
};

// Values of a cache element: the storage type itself, or E4M3 codes of value / scale
template <typename T>
__device__ __forceinline__ void put8(T* dst, const float (&v)[8], float)
{
    Eight<T> e;
    e.narrow(v);
    e.store(dst);
}
__device__ __forceinline__ void put8(uint8_t* dst, const float (&v)[8], float scale)
{
    float u[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) u[j] = __fdiv_rn(v[j], scale);
    *reinterpret_cast<uint2*>(dst) = e4m3_codes(u);
}
template <typename T>
__device__ __forceinline__ void put1(T* dst, float v, float) { round_to(v, dst); }
__device__ __forceinline__ void put1(uint8_t* dst, float v, float scale)
{
    *dst = (uint8_t)__nv_cvt_float_to_fp8(__fdiv_rn(v, scale), __NV_SATFINITE, __NV_E4M3);
}

// Both components of a pair; products and sum rounded one by one, so that they do not depend on what the compiler fuses
__device__ __forceinline__ void rotate(float u, float w, float2 cs, float& x, float& y)
{
    x = __fsub_rn(__fmul_rn(u, cs.x), __fmul_rn(w, cs.y));
    y = __fadd_rn(__fmul_rn(w, cs.x), __fmul_rn(u, cs.y));
}

// One piece of a head: kWide pieces are eight components, or eight pairs in the half layout; else one component or pair.
template <typename T, typename C, bool kWide>
__device__ __forceinline__ void rotate_piece(const T* src, C* dst, int piece, const RotateArgs& p, const float2* turn, float scale)
{
    const int half = p.rot >> 1;
    if constexpr (kWide) {
        float a[8], b[8];
        Eight<T> ea, eb;
        if (p.interleaved) {
            const int c0 = 8 * piece;
            ea.load(src + c0);
            ea.widen(a);
#pragma unroll
            for (int j = 0; j < 8; j += 2) {
                if (c0 + j < p.rot) {
                    const float2 cs = turn[(c0 + j) >> 1];
                    const float u = a[j], w = a[j + 1];
                    rotate(u, w, cs, a[j], a[j + 1]);
                }
            }
            put8(dst + c0, a, scale);
        } else if (8 * piece < half) {
            const int c0 = 8 * piece;
            ea.load(src + c0);
            eb.load(src + c0 + half);
            ea.widen(a);
            eb.widen(b);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float2 cs = turn[c0 + j];
                const float u = a[j], w = b[j];
                rotate(u, w, cs, a[j], b[j]);
            }
            put8(dst + c0, a, scale);
            put8(dst + c0 + half, b, scale);
        } else {
            const int c0 = 8 * piece + half;
            ea.load(src + c0);
            ea.widen(a);
            put8(dst + c0, a, scale);
        }
    } else {                                                  // the half layout with a `rot` that is no multiple of 16
        if (piece < half) {
            const float2 cs = turn[piece];
            const float u = widen_at(src, piece), w = widen_at(src, piece + half);
            float x, y;
            rotate(u, w, cs, x, y);
            put1(dst + piece, x, scale);
            put1(dst + piece + half, y, scale);
        } else {
            put1(dst + piece + half, widen_at(src, piece + half), scale);
        }
    }
}

// T: type of Q, K, V; C: of the cache
template <typename T, typename C, bool kWide>
__global__ void __launch_bounds__(kThreads) rotate_append_kernel(const RotateArgs p)
{
    __shared__ float2 turn[kMaxPairs];
    chain_next();
    chain_wait();
    const int token = blockIdx.x;
    const int pos = p.pos[token];
    if (pos < 0) return;
    const int half = p.rot >> 1;
    for (int i = threadIdx.x; i < half; i += kThreads) {
        // (the product's own rounding would be 2^-23 radians at the farthest positions)
        const double turns = p.turns[i], whole = (double)pos * turns, rest = fma((double)pos, turns, -whole);
        double s, c;
        sincospi(2.0 * ((whole - rint(whole)) + rest), &s, &c);
        turn[i] = make_float2((float)c * p.magnitude, (float)s * p.magnitude);
    }
    long long at = -1;                                        // the token's place in the cache
    if (p.k) {
        const int seq = p.seq ? p.seq[token] : token;
        const int column = pos / p.page_size;
        if (seq >= 0 && seq < p.seqs && column < p.max_pages) {
            const int page = p.table[(size_t)seq * p.table_ld + column];
            if (page >= 0 && page < p.pages) at = page * p.page_stride + (pos - column * p.page_size) * p.token_stride;
        }
        if (at < 0 && threadIdx.x == 0) atomicCAS(p.status, 0, (int)GELO_ERR_INVALID);
    }
    __syncthreads();

    const int turned = kWide ? (p.interleaved ? p.dh / 8 : (p.dh - half) / 8) : p.dh - half;   // pieces of a head that is rotated
    const int plain = p.dh / 8;                                                                  // of a head that is copied
    const int n_q = p.q_heads * turned, n_k = at >= 0 ? p.kv_heads * turned : 0, n_v = at >= 0 ? p.kv_heads * plain : 0;
    for (int i = threadIdx.x; i < n_q + n_k + n_v; i += kThreads) {
        if (i < n_q) {
            const int head = i / turned;
            rotate_piece<T, T, kWide>(static_cast<const T*>(p.q) + (size_t)token * p.ldq + (size_t)head * p.dh,
                                      static_cast<T*>(p.q_out) + (size_t)token * p.ldqo + (size_t)head * p.dh, i - head * turned, p, turn, 1.0f);
        } else if (i < n_q + n_k) {
            const int head = (i - n_q) / turned;
            rotate_piece<T, C, kWide>(static_cast<const T*>(p.k) + (size_t)token * p.ldk + (size_t)head * p.dh,
                                      static_cast<C*>(p.k_cache) + at + head * p.head_stride, i - n_q - head * turned, p, turn, p.k_scale);
        } else {
            const int head = (i - n_q - n_k) / plain, c0 = 8 * (i - n_q - n_k - head * plain);
            Eight<T> e;
            float v[8];
            e.load(static_cast<const T*>(p.v) + (size_t)token * p.ldv + (size_t)head * p.dh + c0);
            e.widen(v);
            put8(static_cast<C*>(p.v_cache) + at + head * p.head_stride + c0, v, p.v_scale);
        }
    }
}

template <typename T, typename C>
int launch_cached(gelo_ctx* ctx, const RotateArgs& p, int n, cudaStream_t st)
{
    if (p.interleaved || p.rot % 16 == 0)
        GELO_TRY(launch_chained(ctx, rotate_append_kernel<T, C, true>, dim3(n), kThreads, 0, st, p));
    else
        GELO_TRY(launch_chained(ctx, rotate_append_kernel<T, C, false>, dim3(n), kThreads, 0, st, p));
    return after_launch(ctx);
}

__global__ void rope_turns_kernel(int rot, double base, double factor, double original, double low, double high, double* turns)
{
    chain_next();
    chain_wait();
    const int i = threadIdx.x;
    if (i >= rot / 2) return;
    const double t = pow(base, -2.0 * i / rot) * 0.15915494309189533577;       // 1 / (2 pi)
    const double keep = original > 0.0 ? fmin(fmax((original * t - low) / (high - low), 0.0), 1.0) : 0.0;
    turns[i] = t * (keep + (1.0 - keep) / factor);
}

}  // namespace

int launch_rope_turns(gelo_ctx* ctx, int rot, double base, double factor, double original, double low, double high, double* turns, cudaStream_t st)
{
    GELO_TRY(launch_chained(ctx, rope_turns_kernel, dim3(1), kMaxPairs, 0, st, rot, base, factor, original, low, high, turns));
    return after_launch(ctx);
}

int launch_rotate_append(gelo_ctx* ctx, const gelo_kv_cache* kv, const void* k, int ldk, const void* v, int ldv, const void* q, int ldq, int q_heads,
                         int head_dim, int n, const int* seq, const int* pos, const gelo_rope& rope, int dtype, void* q_out, int ldqo, cudaStream_t st)
{
    RotateArgs p = {};
    p.q = q; p.k = k; p.v = v; p.q_out = q_out;
    p.ldq = ldq; p.ldk = ldk; p.ldv = ldv; p.ldqo = ldqo;
    p.q_heads = q_heads; p.dh = head_dim;
    p.turns = rope.turns_dev; p.rot = rope.rot; p.interleaved = rope.interleaved != 0; p.magnitude = rope.magnitude;
    p.seq = seq; p.pos = pos; p.status = ctx->status_dev;
    if (k) {
        p.k_cache = kv->k_dev; p.v_cache = kv->v_dev; p.table = kv->table_dev;
        p.page_stride = kv->page_stride; p.token_stride = kv->token_stride; p.head_stride = kv->head_stride;
        p.kv_heads = kv->kv_heads;
        p.pages = kv->pages; p.page_size = kv->page_size; p.seqs = kv->seqs; p.max_pages = kv->max_pages; p.table_ld = kv->table_ld;
        p.k_scale = kv->k_scale; p.v_scale = kv->v_scale;
    }
    const bool narrow = k && kv->dtype == GELO_E4M3;
    if (dtype == GELO_BF16) return narrow ? launch_cached<__nv_bfloat16, uint8_t>(ctx, p, n, st) : launch_cached<__nv_bfloat16, __nv_bfloat16>(ctx, p, n, st);
    if (dtype == GELO_F16) return narrow ? launch_cached<__half, uint8_t>(ctx, p, n, st) : launch_cached<__half, __half>(ctx, p, n, st);
    return launch_cached<float, float>(ctx, p, n, st);
}

}  // namespace gelo
