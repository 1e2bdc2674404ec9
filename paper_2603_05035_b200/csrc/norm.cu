// Root-mean-square norm with the residual's addition, and an output in E4M3 with a scale per row.
//   h = x + r,  y = h (mean h^2 + eps)^-1/2 w,  scale = max|y| / 448,  code = E4M3(y / scale)
// The maximum of |y| is that of |h w| times the row's factor, so one pass over the row collects the sum of squares and the maximum, with
// the row in registers; the second half writes from there.  Bound by HBM: x and r in, h and y out.  4096 x 4096 bf16, 134 MB: 22.8 us, 90% of a copy's rate
// (8192 wide 43 us, 95%); 1075 rows to E4M3 7.3 us (65%: one wave of CTAs, which load and then convert, and what decides a code on the right side of a middle); 64 rows 2.7 us.
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

// Sum (in S) and maximum over the kThreads threads that share a row
template <int kThreads, typename S>
__device__ __forceinline__ S row_reduce(S sum, float& top)
{
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) {
        sum += __shfl_xor_sync(0xffffffffu, sum, off);
        if (sizeof(S) == 8) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, off));
    }
    if constexpr (kThreads > 32) {
        __shared__ S sums[kThreads / 32];
        __shared__ float tops[kThreads / 32];
        if ((threadIdx.x & 31) == 0) {
            sums[threadIdx.x >> 5] = sum;
            tops[threadIdx.x >> 5] = top;
        }
        __syncthreads();
        sum = 0;
#pragma unroll
        for (int i = 0; i < kThreads / 32; ++i) {
            sum += sums[i];
            if (sizeof(S) == 8) top = fmaxf(top, tops[i]);
        }
    }
    return sum;
}

// Eight values times hi + lo as E4M3 codes of the exact products: where one rounds to the very middle of two codes, what the rounding has left decides.
// (Rows of 16-bit values hold such products by the dozen: their quotients by the largest are short fractions.)
__device__ __forceinline__ uint2 codes_of(const float (&v)[8], float hi, float lo)
{
    constexpr uint32_t kBelow = 0x7ffffu;                     // a middle has five significant bits: these are zero
    float q[8];
    bool middle = false;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        q[j] = fmaf(v[j], hi, v[j] * lo);
        middle |= (__float_as_uint(q[j]) & kBelow) == 0;
    }
    if (middle) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float left = fmaf(v[j], lo, fmaf(v[j], hi, -q[j]));
            const int bits = __float_as_int(q[j]);
            if ((bits & kBelow) == 0 && left != 0.0f && q[j] != 0.0f) q[j] = __int_as_float(bits + (((__float_as_int(left) ^ bits) >> 31) | 1));
        }
    }
    return e4m3_codes(q);
}

// kVecs groups of eight values per thread stay in registers; kVecs = 0: any width, the row is read a second time (from L2).
// kThreads = 32: four rows per CTA, a warp each.
template <typename T, int kThreads, int kVecs, bool kCodes>
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
    double sum64 = 0.0;

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
        // Binary64 where the middles of codes hang on it (codes_of): 1075 x 4096 7.3 us, with fp32 sums of four squares 7.2, but a row all of whose quotients are middles
        // could then be a step off throughout.
        if constexpr (kCodes) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const double wide = (double)v[j];
                sum64 = fma(wide, wide, sum64);
            }
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) sum = fmaf(v[j], v[j], sum);
        }
        weigh(g, v);
        if constexpr (kCodes) {
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
    float inv = 0.0f, to_code = 0.0f, to_code_rest = 0.0f;
    if constexpr (kCodes) {
        // the row's scale and the factor of its codes in binary64, the factor as two floats; a warp works them out for all
        const double squares = row_reduce<kThreads>(sum64, top);
        __shared__ float of_row[3];
        if (t < 32) {
            const double inv64 = rsqrt(squares / p.d + (double)p.eps);
            float scale = 1.0f;
            const float s = (float)((double)top * inv64 * (1.0 / 448.0));
            if (s > 0.0f) scale = s;
            const double f = fmin(inv64 / (double)scale, (double)FLT_MAX);         // a zero stays zero where the scale is next to nothing
            to_code = (float)f;
            to_code_rest = (float)(f - (double)to_code);
            if (!(squares <= FLT_MAX)) scale = to_code = __int_as_float(0x7fffffff);  // fmaxf passed over a NaN
            inv = (float)inv64;
            if (t == 0) {
                p.row_scale[row] = scale;
                if (kThreads > 32) { of_row[0] = inv; of_row[1] = to_code; of_row[2] = to_code_rest; }
            }
        }
        if (kThreads > 32) {
            __syncthreads();
            inv = of_row[0];
            to_code = of_row[1];
            to_code_rest = of_row[2];
        }
    } else {
        inv = rsqrtf(row_reduce<kThreads>(sum, top) / (float)p.d + p.eps);
    }

    auto emit = [&](int g, float (&v)[8]) {                   // v: h w
        if (p.y) store(p.y, p.ldy, g, v, inv);
        if constexpr (kCodes) *reinterpret_cast<uint2*>(p.codes + (size_t)row * p.ldc + 8 * g) = codes_of(v, to_code, to_code_rest);
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

template <typename T, int kThreads, int kVecs, bool kCodes>
int launch_as(gelo_ctx* ctx, const NormArgs& p, cudaStream_t st)
{
    const int grid = kThreads == 32 ? ceil_div(p.rows, 4) : p.rows;
    GELO_TRY(launch_chained(ctx, rms_norm_kernel<T, kThreads, kVecs, kCodes>, dim3(grid), kThreads == 32 ? 128 : kThreads, 0, st, p));
    return after_launch(ctx);
}

template <typename T, bool kCodes>
int launch_typed(gelo_ctx* ctx, const NormArgs& p, cudaStream_t st)
{
    // A warp a row up to 512 values; then as many threads as leave each one or two groups, since a row waits for its slowest thread and more
    // threads in flight read more (4096 rows of 4096 bf16: 256 threads of two groups 22.8 us, 128 of four 24.6, 512 of one 22.9;
    // of 8192: 512 of two 43, 256 of four 46, 1024 of one 48).
    // Rows with codes wait longer between their two halves, so half as many threads, and twice the rows per SM, where the rows are more than
    // a wave of wide ones (five CTAs of 256 threads per SM, two of 512): 1000 rows of 2048 4.8 us against 5.3 with the wide shape, of 8192 16.5 against 18.5, 4096 rows 51.6
    // against 60; few rows the other way, 148 of 2048 3.3 against 2.8, of 8192 4.8 against 4.1.  The thin shape of 4096 needs so many registers that
    // it gains only where its wave of 8 per SM takes all: 1075 rows 7.3 against 8.0, 1480 rows 13.0 against 10.6, 4096 rows 28.3 against 27.5.
    // With the residual stored too, thin and wide: 1075 rows of 2304 6.9, 8.3, of 3584 9.1, 9.7, of 4096 10.1, 10.2 (740 rows 9.1, 7.0; 1500 14.1, 12.9).
    const int groups = p.d / 8, per_sm = ceil_div(p.rows, ctx->sm_count);
    if (groups <= 32) return launch_as<T, 32, 1, kCodes>(ctx, p, st);
    if (groups <= 64) return launch_as<T, 32, 2, kCodes>(ctx, p, st);
    if (groups <= 128) return launch_as<T, 128, 1, kCodes>(ctx, p, st);
    if constexpr (kCodes) {
        if (groups <= 256 && per_sm > 5) return launch_as<T, 128, 2, true>(ctx, p, st);
        if (groups > 256 && groups <= 512 && per_sm > 5 && per_sm <= 8) return launch_as<T, 128, 4, true>(ctx, p, st);
        if (groups > 512 && groups <= 1024 && per_sm > 2) return launch_as<T, 256, 4, true>(ctx, p, st);
    }
    if (groups <= 256) return launch_as<T, 256, 1, kCodes>(ctx, p, st);
    if (groups <= 512) return launch_as<T, 256, 2, kCodes>(ctx, p, st);
    if (groups <= 1024) return launch_as<T, 512, 2, kCodes>(ctx, p, st);
    if (groups <= 2048) return launch_as<T, 512, 4, kCodes>(ctx, p, st);
    return launch_as<T, 512, 0, kCodes>(ctx, p, st);
}

template <typename T>
int launch_codes_or_not(gelo_ctx* ctx, const NormArgs& p, cudaStream_t st)
{
    return p.codes ? launch_typed<T, true>(ctx, p, st) : launch_typed<T, false>(ctx, p, st);
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
    if (dtype == GELO_BF16) return launch_codes_or_not<__nv_bfloat16>(ctx, p, st);
    if (dtype == GELO_F16) return launch_codes_or_not<__half>(ctx, p, st);
    return launch_codes_or_not<float>(ctx, p, st);
}

}  // namespace gelo
