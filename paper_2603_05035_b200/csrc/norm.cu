// Root-mean-square norm with the residual's addition, and an output in E4M3 with a scale per row.
//   h = x + r,  y = h (mean h^2 + eps)^-1/2 w,  scale = max|y| / 448,  code = E4M3(y / scale)
// The maximum of |y| is that of |h w| times the row's factor, so one pass over the row collects the sum of squares and the maximum, with
// the row in registers; the second half writes from there.  Bound by HBM: x and r in, h and y out.  4096 x 4096 bf16, 134 MB: 24.1 us, 86% of a copy's rate;
// 1075 rows to E4M3 6.7 us (71%); 64 rows 2.7 us.
#include <float.h>

#include "common.cuh"
#include "vec8.cuh"

namespace gelo {

namespace {

struct NormArgs {
    const void *x, *r, *w;
    void *r_out, *y;
    uint8_t* codes;
    float* row_scale;
    int ldx, ldr, ldro, ldy, ldc;
    int rows, d;
    float eps;
};

// Sum and maximum over the kThreads threads that share a row
template <int kThreads>
__device__ __forceinline__ void row_reduce(float& sum, float& top)
{
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) {
        sum += __shfl_xor_sync(0xffffffffu, sum, off);
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, off));
    }
    if constexpr (kThreads > 32) {
        __shared__ float2 part[kThreads / 32];
        if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = make_float2(sum, top);
        __syncthreads();
        sum = 0.0f;
#pragma unroll
        for (int i = 0; i < kThreads / 32; ++i) {
            sum += part[i].x;
            top = fmaxf(top, part[i].y);
        }
    }
}

// kVecs groups of eight values per thread stay in registers; kVecs = 0: any width, the row is read a second time (from L2).
// kThreads = 32: four rows per CTA, a warp each.
template <typename T, int kThreads, int kVecs>
__global__ void __launch_bounds__(kThreads == 32 ? 128 : kThreads) rms_norm_kernel(const NormArgs p)
{
    chain_next();
    chain_wait();
    const int row = kThreads == 32 ? blockIdx.x * 4 + (threadIdx.x >> 5) : blockIdx.x;
    const int t = kThreads == 32 ? threadIdx.x & 31 : threadIdx.x;
    if (row >= p.rows) return;                                // whole warps, and no barrier follows for them
    const T* x = static_cast<const T*>(p.x) + (size_t)row * p.ldx;
    const T* r = p.r ? static_cast<const T*>(p.r) + (size_t)row * p.ldr : nullptr;
    const T* w = static_cast<const T*>(p.w);
    const int groups = p.d >> 3;
    constexpr int kKept = kVecs ? kVecs : 1;
    float h[kKept][8];
    float sum = 0.0f, top = 0.0f;

    auto load = [&](int g, float (&v)[8]) {
        Eight<T> a, b;
        a.load(x + 8 * g);
        if (r) b.load(r + 8 * g);
        a.widen(v);
        if (r) {
            float u[8];
            b.widen(u);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] += u[j];
        }
    };
    auto weigh = [&](int g, float (&v)[8]) {                  // v *= w
        if (!w) return;
        Eight<T> a;
        float u[8];
        a.load(w + 8 * g);
        a.widen(u);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] *= u[j];
    };
    auto store = [&](void* to, int ld, int g, const float (&v)[8], float factor) {
        float u[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) u[j] = v[j] * factor;
        Eight<T> a;
        a.narrow(u);
        a.store(static_cast<T*>(to) + (size_t)row * ld + 8 * g);
    };
    auto collect = [&](int g, float (&v)[8]) {                // leaves h w in v
#pragma unroll
        for (int j = 0; j < 8; ++j) sum = fmaf(v[j], v[j], sum);
        weigh(g, v);
        if (p.codes) {
#pragma unroll
            for (int j = 0; j < 8; ++j) top = fmaxf(top, fabsf(v[j]));
        }
    };

    if constexpr (kVecs > 0) {
#pragma unroll
        for (int i = 0; i < kVecs; ++i)
            if (t + i * kThreads < groups) load(t + i * kThreads, h[i]);
#pragma unroll
        for (int i = 0; i < kVecs; ++i) {
            const int g = t + i * kThreads;
            if (g >= groups) continue;
            if (p.r_out) store(p.r_out, p.ldro, g, h[i], 1.0f);       // (x and r of this place have been read, whichever of them it is)
            collect(g, h[i]);
        }
    } else {
        for (int g = t; g < groups; g += kThreads) {
            load(g, h[0]);
            collect(g, h[0]);
        }
    }
    row_reduce<kThreads>(sum, top);
    const float inv = rsqrtf(sum / (float)p.d + p.eps);
    float scale = 1.0f, to_code = 1.0f;
    if (p.codes) {
        const float s = __fdiv_rn(top * inv, 448.0f);
        if (s > 0.0f) scale = s;
        to_code = fminf(__fdiv_rn(inv, scale), FLT_MAX);      // a zero stays zero where the scale is next to nothing
        if (!(sum <= FLT_MAX)) scale = to_code = __int_as_float(0x7fffffff);   // fmaxf passed over a NaN
        if (t == 0) p.row_scale[row] = scale;
    }

    auto emit = [&](int g, float (&v)[8]) {                   // v: h w
        if (p.y) store(p.y, p.ldy, g, v, inv);
        if (p.codes) {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] *= to_code;
            *reinterpret_cast<uint2*>(p.codes + (size_t)row * p.ldc + 8 * g) = e4m3_codes(v);
        }
    };
    if constexpr (kVecs > 0) {
#pragma unroll
        for (int i = 0; i < kVecs; ++i)
            if (t + i * kThreads < groups) emit(t + i * kThreads, h[i]);
    } else {
        for (int g = t; g < groups; g += kThreads) {
            load(g, h[0]);
            if (p.r_out) store(p.r_out, p.ldro, g, h[0], 1.0f);
            weigh(g, h[0]);
            emit(g, h[0]);
        }
    }
}

template <typename T, int kThreads, int kVecs>
int launch_as(gelo_ctx* ctx, const NormArgs& p, cudaStream_t st)
{
    const int grid = kThreads == 32 ? ceil_div(p.rows, 4) : p.rows;
    GELO_TRY(launch_chained(ctx, rms_norm_kernel<T, kThreads, kVecs>, dim3(grid), kThreads == 32 ? 128 : kThreads, 0, st, p));
    return after_launch(ctx);
}

template <typename T>
int launch_typed(gelo_ctx* ctx, const NormArgs& p, cudaStream_t st)
{
    // A warp a row up to 512 values; then as many threads as leave each one or two groups, since a row waits for its slowest thread and more
    // threads in flight read more (4096 rows of 4096 bf16: 256 threads of two groups 24.2 us, 128 of four 26.5, 64 of eight 33, 512 of one 24.8;
    // of 8192: 512 of two 46, 256 of four 49; of 2048: 256 of one 12.8, 128 of two 13.1).
    const int groups = p.d / 8;
    if (groups <= 32) return launch_as<T, 32, 1>(ctx, p, st);
    if (groups <= 64) return launch_as<T, 32, 2>(ctx, p, st);
    if (groups <= 128) return launch_as<T, 128, 1>(ctx, p, st);
    if (groups <= 256) return launch_as<T, 256, 1>(ctx, p, st);
    if (groups <= 512) return launch_as<T, 256, 2>(ctx, p, st);
    if (groups <= 1024) return launch_as<T, 512, 2>(ctx, p, st);
    if (groups <= 2048) return launch_as<T, 512, 4>(ctx, p, st);
    return launch_as<T, 512, 0>(ctx, p, st);
}

}  // namespace

int launch_rms_norm(gelo_ctx* ctx, const void* x, int ldx, const void* r, int ldr, const void* w, int rows, int d, float eps, int dtype,
                    void* r_out, int ldro, void* y, int ldy, void* codes, int ldc, float* row_scale, cudaStream_t st)
{
    NormArgs p;
    p.x = x; p.r = r; p.w = w; p.r_out = r_out; p.y = y;
    p.codes = static_cast<uint8_t*>(codes); p.row_scale = row_scale;
    p.ldx = ldx; p.ldr = ldr; p.ldro = ldro; p.ldy = ldy; p.ldc = ldc;
    p.rows = rows; p.d = d; p.eps = eps;
    if (dtype == GELO_BF16) return launch_typed<__nv_bfloat16>(ctx, p, st);
    if (dtype == GELO_F16) return launch_typed<__half>(ctx, p, st);
    return launch_typed<float>(ctx, p, st);
}

}  // namespace gelo
