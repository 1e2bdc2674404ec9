// Attention of one new token per sequence over a paged key-value cache.
//   o = sum_j p_j v_j,  p_j = exp(s_j - m) / l,  s_j = scale q . k_j,  m = max_j s_j,  l = sum_j exp(s_j - m)
// One pass over the keys and values with the running maximum and sum of the softmax; every key and value is read once for all query
// heads that share it (up to 16; more heads read them again, from L2).  Bound by HBM: 4 heads-per-group flops per element read.
//
// The work of a call is one line of tiles: sequence after sequence, key-value head after head, 16 or 32 positions a tile.  Every CTA works out
// from the lengths which equal share of that line is its own, so ragged lengths balance and one long sequence fills the GPU.  What of
// a (sequence, head) falls to one CTA is a segment; where a CTA's border cuts one, each side leaves its sums in the workspace and the
// CTA that arrives last adds them up, in the order of the CTAs whoever that is.
// Inside a CTA the warps take the tiles of a segment in turn, each with a ring of its own in shared memory that asynchronous 16-byte copies
// fill, so nothing but a segment's end makes them wait for one another.
#include <limits.h>

#include <type_traits>

#include "common.cuh"
#include "vec8.cuh"

namespace gelo {

namespace {

constexpr int kMaxCtas = 320;
constexpr int kMaxParts = 64;                                 // a head's sums come from no more than about so many CTAs
constexpr int kSlotFloats = 16 * 256 + 32;                    // sums of 16 heads, their maxima, their totals
constexpr float kNone = -INFINITY;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

struct AttendArgs {
    const void *q, *k, *v;
    void* o;
    float *lse, *slots;
    int* arrived;                                             // one counter per CTA, zero between calls
    const int *len, *table;
    int* status;
    long long page_stride, token_stride, head_stride;         // bytes
    int ldq, ldo, q_heads, group, dh;
    int pages, page_size, page_shift, seqs, max_pages, table_ld, window;
    int kv_heads, heads_a_unit, units;                        // units: heads_a_unit query heads of one key-value head each, per sequence
    float scale, v_scale;                                     // scale: of the logits, the keys' scale included
};

// The positions that count of one sequence, and its tiles
struct Span { int first, len, t0, t1; };
template <int kTile>
__device__ __forceinline__ Span span_of(const AttendArgs& p, int seq)
{
    Span s;
    const long long room = (long long)p.max_pages * p.page_size;
    const int cap = room < INT_MAX - kTile ? (int)room : INT_MAX - kTile;             // (a tile's last position is still an int)
    int n = p.len[seq];
    if (n > cap) {
        n = cap;
        atomicCAS(p.status, 0, (int)GELO_ERR_INVALID);
    }
    s.len = n > 0 ? n : 0;
    s.first = p.window && s.len > p.window ? s.len - p.window : 0;
    s.t0 = s.first / kTile;
    s.t1 = max((s.len + kTile - 1) / kTile, s.t0 + 1);        // a sequence without positions has a tile too: its result has to be written
    return s;
}

// A walk over the segments of a CTA's share
template <int kTile>
struct Walk {
    Span s;
    int seq, unit, at, end;                                   // the segment: tiles [at, end) of (seq, unit)
    long long left;                                           // tiles of the share behind it
    __device__ __forceinline__ void begin(const AttendArgs& p, int seq0, long long offset, long long tiles)
    {
        seq = seq0;
        s = span_of<kTile>(p, seq);
        const int n = s.t1 - s.t0;
        unit = (int)(offset / n);
        at = s.t0 + (int)(offset - (long long)unit * n);
        end = at + (int)min((long long)(s.t1 - at), tiles);
        left = tiles - (end - at);
    }
    __device__ __forceinline__ bool next(const AttendArgs& p)
    {
        if (left <= 0) return false;
        if (++unit == p.units) {
            unit = 0;
            s = span_of<kTile>(p, ++seq);
        }
        at = s.t0;
        end = at + (int)min((long long)(s.t1 - at), left);
        left -= end - at;
        return true;
    }
};

__device__ __forceinline__ uint32_t smem_at(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void copy16(uint32_t dst, const void* src, bool there)      // zeros where nothing is there; `src` is not read then
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copies_end() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ void ldmatrix4(uint32_t (&r)[4], uint32_t at)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ void ldmatrix4_t(uint32_t (&r)[4], uint32_t at)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ uint32_t transposed(uint32_t x)
{
    uint32_t y;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
__device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1, __nv_bfloat16)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1, __half)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// 2^x for x <= 0, to two units in the last place; nothing where the result is no normal number
__device__ __forceinline__ float power2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
template <typename M>
__device__ __forceinline__ uint32_t pack2(float lo, float hi)
{
    M e[2];
    round_to(lo, &e[0]);
    round_to(hi, &e[1]);
    return *reinterpret_cast<uint32_t*>(e);
}
// what rounding x to the 16-bit type leaves, rounded to it in turn
template <typename M>
__device__ __forceinline__ float rest(float x)
{
    M e;
    round_to(x, &e);
    return x - widen_at(&e, 0);
}
// four E4M3 codes as halves: the low two, the high two
__device__ __forceinline__ void halves_of_codes(uint32_t four, uint32_t& low, uint32_t& high)
{
    asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, a;\n\tcvt.rn.f16x2.e4m3x2 %1, b;\n\t}" : "=r"(low), "=r"(high) : "r"(four));
}

// Geometry of a kernel instance.  Rows of DH elements of kBytes, 32 of them where that is no more than 8 KB of keys and values, since what a tile
// costs beside its products is the same; the 16-byte pieces of a row are permuted by its number so that eight
// rows' pieces of one column lie in different banks.
template <int DH, int kBytes>
struct Tiles {
    static constexpr int kRow = DH * kBytes;                  // bytes
    static constexpr int kTile = kRow <= 128 ? 32 : 16;       // positions
    static constexpr int kPieces = kRow / 16;                 // of a row
    static constexpr int kHalf = kTile * kRow;                // the keys, or the values
    static constexpr int kStage = 2 * kHalf;
    static constexpr int kWarps = kStage > 16384 ? 2 : 4;
    static constexpr int kStages = kStage >= 8192 ? 3 : 24576 / kStage;
    static constexpr int kCtas = kWarps * kStages * kStage > 98304 ? 1 : 2;            // per SM
    static constexpr int kJoinPitch = DH + 4;
    static constexpr int kJoinHeads = 4;                      // heads whose sums the warps exchange at a time
    static constexpr int kJoin = kWarps * kJoinHeads * kJoinPitch * 4;
    static constexpr int kSmem = kWarps * kStages * kStage + kJoin;
    __device__ static __forceinline__ uint32_t piece(int row, int c)                   // byte offset of piece c of a row
    {
        return kPieces >= 8 ? row * kRow + ((c ^ (row & 7)) << 4) : row * kRow + ((c ^ ((row >> 1) & (kPieces - 1))) << 4);
    }
};

// ---- products of a warp on a 16-bit or E4M3 tile: mma.sync on transposed operands ---------------------------
// S^T = K q^T and O^T = V^T p^T: positions (and components) are the 16 rows of an instruction, up to eight query heads its columns, so a
// single head wastes columns of an otherwise idle unit and no loads.  The matrix rate that this leaves is several times what HBM
// can feed (16 instructions per 8 KB tile of 128 components).  p is handed to the second product as the 16-bit value and what
// that leaves out, i.e. with 16 bits, so the stored result is rounded once; E4M3 caches with bf16 results take it as one half (11 bits).
// E4M3 tiles are widened to half in registers, q is given the same type times a power of two that puts its largest component into [1, 2).
template <typename T, bool kCodes, int DH, int NT>
struct MmaWarp {
    using M = std::conditional_t<kCodes, __half, T>;
    using G = Tiles<DH, kCodes ? 1 : 2>;
    static constexpr bool kPair = !(kCodes && std::is_same_v<T, __nv_bfloat16>);
    static constexpr int kHeads = 8 * NT;
    uint32_t qf[DH / 16][NT][2];
    float acc[DH / 16][NT][4];
    float m[NT][2], l[NT][2], scale[NT][2];

    // heads [0, heads) of the unit; q points at the first one's components
    __device__ __forceinline__ void begin(const AttendArgs& p, const T* q, int heads, int lane)
    {
        const int t = lane & 3;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const int h = 8 * n + (lane >> 2);
            const T* row = q + (size_t)h * p.dh;
            float factor = 1.0f;
            if constexpr (kCodes) {
                float v[DH / 16][4], top = 0.0f;
#pragma unroll
                for (int s = 0; s < DH / 16; ++s)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int c = 16 * s + 4 * t + j;
                        v[s][j] = h < heads && c < p.dh ? widen_at(row, c) : 0.0f;
                        top = fmaxf(top, fabsf(v[s][j]));
                    }
                top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
                top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
                int e = 0;
                if (top > 0.0f && top <= 3.4e38f) e = max(ilogbf(top), -126);
                factor = exp2f((float)e);
                const float down = exp2f((float)-e);
#pragma unroll
                for (int s = 0; s < DH / 16; ++s)
#pragma unroll
                    for (int j = 0; j < 2; ++j) qf[s][n][j] = pack2<M>(v[s][2 * j] * down, v[s][2 * j + 1] * down);
            } else {
#pragma unroll
                for (int s = 0; s < DH / 16; ++s)
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const int c = 16 * s + 2 * t + 8 * j;
                        qf[s][n][j] = h < heads && c < p.dh ? *reinterpret_cast<const uint32_t*>(row + c) : 0u;
                    }
            }
            // columns 2t and 2t + 1 of a product are heads whose q other lanes hold
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                scale[n][j] = p.scale * kLog2e * (kCodes ? __shfl_sync(0xffffffffu, factor, 4 * (2 * t + j)) : 1.0f);
                m[n][j] = kNone;
                l[n][j] = 0.0f;
            }
#pragma unroll
            for (int s = 0; s < DH / 16; ++s)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[s][n][j] = 0.0f;
        }
    }

    __device__ __forceinline__ void tile(uint32_t keys, uint32_t values, uint32_t counts, int lane)
    {
        constexpr int kSub = G::kTile / 16;
        const int r = lane >> 2;
        float c[kSub][NT][4];
#pragma unroll
        for (int b = 0; b < kSub; ++b)
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int j = 0; j < 4; ++j) c[b][n][j] = 0.0f;
        // matrix i of a load comes from the addresses of lanes 8i .. 8i + 7: rows 0-7 and 8-15, then the next piece of both
        const int row = lane & 15, next = lane >> 4;
#pragma unroll
        for (int b = 0; b < kSub; ++b) {
            if constexpr (kCodes) {
#pragma unroll
                for (int s = 0; s < DH / 16; s += 2) {
                    uint32_t x[4];
                    ldmatrix4(x, keys + G::piece(16 * b + row, s + next));
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        uint32_t a[4];
                        halves_of_codes(x[2 * u], a[0], a[2]);
                        halves_of_codes(x[2 * u + 1], a[1], a[3]);
#pragma unroll
                        for (int n = 0; n < NT; ++n) mma(c[b][n], a, qf[s + u][n][0], qf[s + u][n][1], M());
                    }
                }
            } else {
#pragma unroll
                for (int s = 0; s < DH / 16; ++s) {
                    uint32_t a[4];
                    ldmatrix4(a, keys + G::piece(16 * b + row, 2 * s + next));
#pragma unroll
                    for (int n = 0; n < NT; ++n) mma(c[b][n], a, qf[s][n][0], qf[s][n][1], M());
                }
            }
        }
        // positions of this lane: r + 8 i
        bool on[2 * kSub];
#pragma unroll
        for (int i = 0; i < 2 * kSub; ++i) on[i] = (counts >> (r + 8 * i)) & 1u;
        uint32_t ph[kSub][NT][2], pl[kSub][NT][2];
        bool moved = false;
        float keep[NT][2];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            float e[2 * kSub][2];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                float top = kNone;
#pragma unroll
                for (int i = 0; i < 2 * kSub; ++i) {
                    e[i][j] = on[i] ? c[i >> 1][n][2 * (i & 1) + j] * scale[n][j] : kNone;
                    top = fmaxf(top, e[i][j]);
                }
                top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 4));
                top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 8));
                top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 16));
                top = fmaxf(top, m[n][j]);
                const float base = top == kNone ? 0.0f : top;
                keep[n][j] = power2(m[n][j] - base);
                moved |= top > m[n][j];
                m[n][j] = top;
                float sum = 0.0f;
#pragma unroll
                for (int i = 0; i < 2 * kSub; ++i) {
                    e[i][j] = power2(e[i][j] - base);         // (nothing for minus infinity)
                    sum += e[i][j];
                }
                l[n][j] = fmaf(l[n][j], keep[n][j], sum);
            }
#pragma unroll
            for (int i = 0; i < 2 * kSub; ++i) {
                ph[i >> 1][n][i & 1] = transposed(pack2<M>(e[i][0], e[i][1]));
                if constexpr (kPair) pl[i >> 1][n][i & 1] = transposed(pack2<M>(rest<M>(e[i][0]), rest<M>(e[i][1])));
            }
        }
        if (__any_sync(0xffffffffu, moved)) {
#pragma unroll
            for (int s = 0; s < DH / 16; ++s)
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int j = 0; j < 4; ++j) acc[s][n][j] *= keep[n][j & 1];
        }
        const int pos = (lane & 7) + ((lane >> 4) << 3), col = (lane >> 3) & 1;
#pragma unroll
        for (int b = 0; b < kSub; ++b) {
            auto add = [&](int s, const uint32_t (&a)[4]) {
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    mma(acc[s][n], a, ph[b][n][0], ph[b][n][1], M());
                    if constexpr (kPair) mma(acc[s][n], a, pl[b][n][0], pl[b][n][1], M());
                }
            };
            if constexpr (kCodes) {
                // an 8 x 8 transposed load hands out code pairs: components 2r and 2r + 1 of two positions; the first become row r, the second row r + 8
#pragma unroll
                for (int s = 0; s < DH / 16; s += 2) {
                    uint32_t x[4];
                    ldmatrix4_t(x, values + G::piece(16 * b + pos, s + col));
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        uint32_t a[4];
                        halves_of_codes(__byte_perm(x[u], 0, 0x3120), a[0], a[1]);
                        halves_of_codes(__byte_perm(x[2 + u], 0, 0x3120), a[2], a[3]);
                        add(s + u, a);
                    }
                }
            } else {
#pragma unroll
                for (int s = 0; s < DH / 16; ++s) {
                    uint32_t a[4];
                    ldmatrix4_t(a, values + G::piece(16 * b + pos, 2 * s + col));
                    add(s, a);
                }
            }
        }
    }

    // maxima and totals of heads [0, kHeads) into shared memory
    __device__ __forceinline__ void statistics(float* tops, float* totals, int lane)
    {
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                float sum = l[n][j];
#pragma unroll
                for (int off = 4; off < 32; off <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, off);
                if (lane < 4) {
                    tops[8 * n + 2 * lane + j] = m[n][j];
                    totals[8 * n + 2 * lane + j] = sum;
                }
            }
    }
    // sums of heads [h0, h0 + 4) times factor[head], head-major with the join's pitch
    __device__ __forceinline__ void sums(float* out, const float* factor, int h0, int lane)
    {
        const int r = lane >> 2, t = lane & 3;
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int h = 8 * n + 2 * t + j;
                if (h < h0 || h >= h0 + 4) continue;
                const float f = factor[h];
                float* dst = out + (h - h0) * G::kJoinPitch;
#pragma unroll
                for (int s = 0; s < DH / 16; ++s) {
                    dst[16 * s + (kCodes ? 2 * r : r)] = acc[s][n][j] * f;
                    dst[16 * s + (kCodes ? 2 * r + 1 : r + 8)] = acc[s][n][2 + j] * f;
                }
            }
    }
};

// ---- products of a warp on an fp32 tile: multiply-adds ------------------------------------------------------
// Logits: two lanes per position, half the components each, a key's piece in registers for all heads.  Sums: a lane owns DH / 32 components.
template <int DH>
struct FmaWarp {
    using G = Tiles<DH, 4>;
    static constexpr int kHeads = 8;
    static constexpr int kOwn = DH / 32;
    const float* q;
    int heads, dh, group;
    float acc[kHeads][kOwn];
    float m[kHeads], l[kHeads], scale;

    __device__ __forceinline__ void begin(const AttendArgs& p, const float* q_, int heads_, int)
    {
        q = q_; heads = heads_; dh = p.dh; scale = p.scale * kLog2e;
#pragma unroll
        for (int h = 0; h < kHeads; ++h) {
            m[h] = kNone;
            l[h] = 0.0f;
#pragma unroll
            for (int i = 0; i < kOwn; ++i) acc[h][i] = 0.0f;
        }
    }
    __device__ __forceinline__ void tile(uint32_t keys, uint32_t values, uint32_t counts, int lane)
    {
        const int row = lane & 15, side = lane >> 4;
        float s[kHeads];
#pragma unroll
        for (int h = 0; h < kHeads; ++h) s[h] = 0.0f;
        for (int c = side; c < dh / 4; c += 2) {
            float4 k4;
            asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(k4.x), "=f"(k4.y), "=f"(k4.z), "=f"(k4.w) : "r"(keys + G::piece(row, c)) : "memory");
#pragma unroll
            for (int h = 0; h < kHeads; ++h) {
                if (h < heads) {
                    const float4 q4 = *reinterpret_cast<const float4*>(q + (size_t)h * dh + 4 * c);
                    s[h] = fmaf(k4.x, q4.x, fmaf(k4.y, q4.y, fmaf(k4.z, q4.z, fmaf(k4.w, q4.w, s[h]))));
                }
            }
        }
        const bool on = (counts >> row) & 1u;
        float e[kHeads];
#pragma unroll
        for (int h = 0; h < kHeads; ++h) {
            if (h >= heads) break;
            s[h] += __shfl_xor_sync(0xffffffffu, s[h], 16);
            s[h] = on ? s[h] * scale : kNone;
            float top = s[h];
#pragma unroll
            for (int off = 1; off < 16; off <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, off));
            top = fmaxf(top, m[h]);
            const float base = top == kNone ? 0.0f : top;
            const float keep = power2(m[h] - base);
            m[h] = top;
            e[h] = power2(s[h] - base);
            l[h] = l[h] * keep + (side ? 0.0f : e[h]);
#pragma unroll
            for (int i = 0; i < kOwn; ++i) acc[h][i] *= keep;
        }
#pragma unroll 4
        for (int t = 0; t < G::kTile; ++t) {
            float v[kOwn];
            load_own(v, values, t, lane);
#pragma unroll
            for (int h = 0; h < kHeads; ++h) {
                if (h >= heads) break;
                const float w = __shfl_sync(0xffffffffu, e[h], t);
#pragma unroll
                for (int i = 0; i < kOwn; ++i) acc[h][i] = fmaf(w, v[i], acc[h][i]);
            }
        }
    }
    // component i of a lane: 2 lane + i, or 4 lane + i (and 128 further)
    __device__ static __forceinline__ int component(int lane, int i) { return kOwn == 2 ? 2 * lane + i : 4 * lane + (i & 3) + (i >> 2) * 128; }
    __device__ __forceinline__ void load_own(float (&v)[kOwn], uint32_t values, int t, int lane)
    {
        if constexpr (kOwn == 2) {
            asm volatile("ld.shared.v2.f32 {%0, %1}, [%2];" : "=f"(v[0]), "=f"(v[1]) : "r"(values + G::piece(t, lane >> 1) + 8 * (lane & 1)) : "memory");
        } else {
#pragma unroll
            for (int i = 0; i < kOwn; i += 4)
                asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v[i]), "=f"(v[i + 1]), "=f"(v[i + 2]), "=f"(v[i + 3])
                             : "r"(values + G::piece(t, lane + 8 * i)) : "memory");
        }
    }
    __device__ __forceinline__ void statistics(float* tops, float* totals, int lane)
    {
#pragma unroll
        for (int h = 0; h < kHeads; ++h) {
            float sum = l[h];
#pragma unroll
            for (int off = 1; off < 32; off <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, off);
            if (lane == 0) {
                tops[h] = m[h];
                totals[h] = sum;
            }
        }
    }
    __device__ __forceinline__ void sums(float* out, const float* factor, int h0, int lane)
    {
#pragma unroll
        for (int h = 0; h < kHeads; ++h) {
            if (h < h0 || h >= h0 + 4) continue;
#pragma unroll
            for (int i = 0; i < kOwn; ++i) out[(h - h0) * G::kJoinPitch + component(lane, i)] = acc[h][i] * factor[h];
        }
    }
};

template <typename T, typename W>
__device__ __forceinline__ void write_result(const AttendArgs& p, int seq, int head, int c, float sum, float total)
{
    const float o = total > 0.0f || total != total ? sum / total * p.v_scale : 0.0f;
    round_to(o, static_cast<T*>(p.o) + (size_t)seq * p.ldo + (size_t)head * p.dh + c);
}

template <typename T, typename W, int kBytes>
__global__ void __launch_bounds__(32 * W::G::kWarps, W::G::kCtas) attend_kernel(const AttendArgs p)
{
    using G = typename W::G;
    constexpr int kWarps = G::kWarps, kThreads = 32 * kWarps, kStages = G::kStages, kTile = G::kTile;
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ long long scan[kWarps];
    __shared__ long long found_offset;
    __shared__ int found_seq, last;
    __shared__ uint32_t counts[kWarps][kStages];
    __shared__ float tops[kWarps][W::kHeads], totals[kWarps][W::kHeads], factor[kWarps][W::kHeads];
    chain_next();
    chain_wait();
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, cta = blockIdx.x;

    // ---- this CTA's share of the line of tiles ----
    long long x0, tiles, share;
    {
        const int per = (p.seqs + kThreads - 1) / kThreads, s0 = min(tid * per, p.seqs), s1 = min(s0 + per, p.seqs);
        long long mine = 0;
        for (int s = s0; s < s1; ++s) {
            const Span sp = span_of<kTile>(p, s);
            mine += sp.t1 - sp.t0;
        }
        long long upto = mine;
#pragma unroll
        for (int off = 1; off < 32; off <<= 1) {
            const long long u = __shfl_up_sync(0xffffffffu, upto, off);
            if (lane >= off) upto += u;
        }
        if (lane == 31) scan[warp] = upto;
        __syncthreads();
        long long all = 0;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            if (w < warp) upto += scan[w];
            all += scan[w];
        }
        const long long total = all * p.units;
        // a tile for every warp at least, and no head cut into many more than kMaxParts pieces
        share = max(max((total + gridDim.x - 1) / gridDim.x, (long long)kWarps), (all / p.seqs + kMaxParts - 1) / kMaxParts);
        x0 = cta * share;
        tiles = min(share, total - x0);
        if (tiles <= 0) return;
        const long long before = (upto - mine) * p.units;
        if (x0 >= before && x0 < upto * p.units) {
            long long at = before;
            int s = s0;
            for (;;) {
                const Span sp = span_of<kTile>(p, s);
                const long long n = (long long)(sp.t1 - sp.t0) * p.units;
                if (x0 < at + n || s + 1 >= s1) break;
                at += n;
                ++s;
            }
            found_seq = s;
            found_offset = x0 - at;
        }
        __syncthreads();
    }

    // ---- copies: the tiles that this warp will take, in order, kStages - 1 of them ahead ----
    const uint32_t ring = smem_at(smem) + warp * kStages * G::kStage;
    float* const join = reinterpret_cast<float*>(smem + kWarps * kStages * G::kStage);
    Walk<kTile> ahead, walk;
    ahead.begin(p, found_seq, found_offset, tiles);
    walk = ahead;
    int next_tile = ahead.at + warp;
    bool more = true, on = false;                             // `on`: this lane's position (lane % kTile) of the pending tile counts
    int page = -1, in_page = 0;
    const char *keys_of = nullptr, *values_of = nullptr;      // of the pending tile's head
    auto look_up = [&]() {                                    // the pending tile: which page each of its positions is on
        while (more && next_tile >= ahead.end) {
            more = ahead.next(p);
            next_tile = ahead.at + warp;
        }
        on = false;
        if (!more) return;
        const int t = next_tile * kTile + lane % kTile;
        on = t >= ahead.s.first && t < ahead.s.len;
        if (on) {
            const int column = p.page_shift >= 0 ? t >> p.page_shift : t / p.page_size;
            in_page = t - column * p.page_size;
            page = p.table[(size_t)ahead.seq * p.table_ld + column];
        }
        const long long head_at = (ahead.unit / (p.units / p.kv_heads)) * p.head_stride;
        keys_of = static_cast<const char*>(p.k) + head_at;
        values_of = static_cast<const char*>(p.v) + head_at;
        next_tile += kWarps;
    };
    constexpr int kRowsACopy = 32 / G::kPieces ? 32 / G::kPieces : 1;                  // rows that one copy of the warp covers
    const int my_row = lane / G::kPieces, my_piece = lane % G::kPieces;
    const long long my_at = my_row * p.token_stride + 16 * my_piece;
    auto issue = [&](int stage) {
        __syncwarp();                                         // everybody has read what the stage held
        if (on && (page < 0 || page >= p.pages)) {
            on = false;
            atomicCAS(p.status, 0, (int)GELO_ERR_INVALID);
        }
        const uint32_t who = __ballot_sync(0xffffffffu, on);
        if (lane == 0) counts[warp][stage] = who;
        const long long at = on ? page * p.page_stride + in_page * p.token_stride : 0;
        const uint32_t dst = ring + stage * G::kStage;
        if (G::kPieces <= 32 && p.page_size % 16 == 0) {      // sixteen positions are neighbours on one page
            const bool wanted = 16 * my_piece < p.dh * kBytes;
#pragma unroll
            for (int b = 0; b < kTile / 16; ++b) {
                // the page is that of any position that counts; positions before it on the page may not count, but lie there
                const uint32_t half = (who >> (16 * b)) & 0xffffu;
                const int one = half ? __ffs(half) - 1 : 0;
                const long long from = __shfl_sync(0xffffffffu, at, 16 * b + one) - (half ? one * p.token_stride : 0) + my_at;
                const char *k = keys_of + from, *v = values_of + from;
#pragma unroll
                for (int i = 0; i < 16 / kRowsACopy; ++i) {
                    const int row = i * kRowsACopy + my_row;
                    const bool there = wanted && ((half >> row) & 1u);
                    const uint32_t to = dst + G::piece(16 * b + row, my_piece);
                    copy16(to, there ? k : p.k, there);
                    copy16(to + G::kHalf, there ? v : p.v, there);
                    k += kRowsACopy * p.token_stride;
                    v += kRowsACopy * p.token_stride;
                }
            }
        } else {
#pragma unroll
            for (int i = 0; i < kTile * G::kPieces / 32; ++i) {
                const int idx = 32 * i + lane, row = idx / G::kPieces, c = idx % G::kPieces;
                const long long from = __shfl_sync(0xffffffffu, at, row) + 16 * c;
                const bool there = ((who >> row) & 1u) && 16 * c < p.dh * kBytes;
                copy16(dst + G::piece(row, c), there ? keys_of + from : p.k, there);
                copy16(dst + G::kHalf + G::piece(row, c), there ? values_of + from : p.v, there);
            }
        }
    };
    look_up();
#pragma unroll 1
    for (int s = 0; s < kStages - 1; ++s) {
        if (more) issue(s);
        copies_end();
        look_up();
    }

    // ---- segments ----
    W w;
    int put = kStages - 1, get = 0;
    long long x = x0;                                         // where the segment begins
    for (bool go = true; go; x += walk.end - walk.at, go = walk.next(p)) {
        const int part_of_kv = p.units / p.kv_heads;
        const int kv_head = walk.unit / part_of_kv, head0 = (walk.unit - kv_head * part_of_kv) * p.heads_a_unit;
        const int heads = min(p.heads_a_unit, p.group - head0), first_head = kv_head * p.group + head0;
        w.begin(p, static_cast<const T*>(p.q) + (size_t)walk.seq * p.ldq + (size_t)first_head * p.dh, heads, lane);
        for (int t = walk.at + warp; t < walk.end; t += kWarps) {
            if (more) issue(put);
            copies_end();
            look_up();
            copies_wait<kStages - 1>();
            __syncwarp();
            w.tile(ring + get * G::kStage, ring + get * G::kStage + G::kHalf, counts[warp][get], lane);
            put = put + 1 == kStages ? 0 : put + 1;
            get = get + 1 == kStages ? 0 : get + 1;
        }
        // the warps' sums, brought to one maximum
        w.statistics(tops[warp], totals[warp], lane);
        __syncthreads();
        float my_top = kNone, my_total = 0.0f;                // of head tid, where there is one
        if (tid < heads) {
#pragma unroll
            for (int i = 0; i < kWarps; ++i) my_top = fmaxf(my_top, tops[i][tid]);
            const float base = my_top == kNone ? 0.0f : my_top;
#pragma unroll
            for (int i = 0; i < kWarps; ++i) {
                factor[i][tid] = power2(tops[i][tid] - base);
                my_total += factor[i][tid] * totals[i][tid];
            }
            totals[0][tid] = my_total;
        }
        const int n = walk.s.t1 - walk.s.t0;
        const long long unit_at = x - (walk.at - walk.s.t0);
        const bool whole = walk.end - walk.at == n;
        const int first_cta = whole ? cta : (int)(unit_at / share), last_cta = whole ? cta : (int)((unit_at + n - 1) / share);
        float* slot = p.slots + (size_t)(2 * cta + (first_cta == cta ? 1 : 0)) * kSlotFloats;
        if (tid < heads) {
            if (!whole) {
                slot[16 * 256 + tid] = my_top;
                slot[16 * 256 + 16 + tid] = my_total;
            } else if (p.lse) {
                p.lse[(size_t)walk.seq * p.q_heads + first_head + tid] = (my_top == kNone ? 0.0f : my_top * kLn2) + logf(my_total);
            }
        }
        __syncthreads();
        for (int h0 = 0; h0 < heads; h0 += G::kJoinHeads) {
            w.sums(join + warp * G::kJoinHeads * G::kJoinPitch, factor[warp], h0, lane);
            __syncthreads();
            const int some = min(heads - h0, G::kJoinHeads);
            for (int i = tid; i < some * p.dh; i += kThreads) {
                const int h = i / p.dh, c = i - h * p.dh;
                float sum = 0.0f;
#pragma unroll
                for (int j = 0; j < kWarps; ++j) sum += join[(j * G::kJoinHeads + h) * G::kJoinPitch + c];
                if (whole) write_result<T, W>(p, walk.seq, first_head + h0 + h, c, sum, totals[0][h0 + h]);
                else slot[(h0 + h) * 256 + c] = sum;
            }
            __syncthreads();
        }
        if (whole) continue;

        // ---- a head that several CTAs share: the last one to arrive adds up ----
        __threadfence();
        __syncthreads();
        if (tid == 0) {
            const int parts = last_cta - first_cta + 1;
            const int before = atomicAdd(p.arrived + first_cta, 1);
            last = before == parts - 1;
            if (last) p.arrived[first_cta] = 0;
        }
        __syncthreads();
        if (!last) continue;
        __threadfence();
        for (int i = tid; i < heads * (p.dh / 4); i += kThreads) {
            const int h = i / (p.dh / 4), c = 4 * (i - h * (p.dh / 4));
            float top = kNone;
            for (int a = first_cta; a <= last_cta; ++a)
                top = fmaxf(top, __ldcg(p.slots + (size_t)(2 * a + (a == first_cta ? 1 : 0)) * kSlotFloats + 16 * 256 + h));
            const float base = top == kNone ? 0.0f : top;
            float total = 0.0f;
            float4 sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 4
            for (int a = first_cta; a <= last_cta; ++a) {
                const float* from = p.slots + (size_t)(2 * a + (a == first_cta ? 1 : 0)) * kSlotFloats;
                const float f = power2(__ldcg(from + 16 * 256 + h) - base);
                const float4 v = __ldcg(reinterpret_cast<const float4*>(from + h * 256 + c));
                total = fmaf(f, __ldcg(from + 16 * 256 + 16 + h), total);
                sum.x = fmaf(f, v.x, sum.x); sum.y = fmaf(f, v.y, sum.y); sum.z = fmaf(f, v.z, sum.z); sum.w = fmaf(f, v.w, sum.w);
            }
            const float four[4] = {sum.x, sum.y, sum.z, sum.w};
#pragma unroll
            for (int j = 0; j < 4; ++j) write_result<T, W>(p, walk.seq, first_head + h, c + j, four[j], total);
            if (p.lse && c == 0) p.lse[(size_t)walk.seq * p.q_heads + first_head + h] = base * kLn2 + logf(total);
        }
    }
}

template <typename T, typename W, int kBytes>
int launch_as(gelo_ctx* ctx, AttendArgs& p, cudaStream_t st)
{
    using G = typename W::G;
    p.heads_a_unit = W::kHeads < p.group ? W::kHeads : p.group;
    const long long units = (long long)p.kv_heads * ceil_div(p.group, p.heads_a_unit);
    if (units > INT_MAX) return GELO_ERR_UNSUPPORTED;
    p.units = (int)units;
    auto kernel = attend_kernel<T, W, kBytes>;
    GELO_CUDA_OK(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, G::kSmem));
    const int ctas = G::kCtas * ctx->sm_count < kMaxCtas ? G::kCtas * ctx->sm_count : kMaxCtas;
    GELO_TRY(launch_chained(ctx, kernel, dim3(ctas), 32 * G::kWarps, G::kSmem, st, p));
    return after_launch(ctx);
}

template <typename T, bool kCodes>
int launch_mma(gelo_ctx* ctx, AttendArgs& p, cudaStream_t st)
{
    constexpr int kBytes = kCodes ? 1 : 2;
    if (p.group <= 8) {
        if (p.dh <= 64) return launch_as<T, MmaWarp<T, kCodes, 64, 1>, kBytes>(ctx, p, st);
        if (p.dh <= 128) return launch_as<T, MmaWarp<T, kCodes, 128, 1>, kBytes>(ctx, p, st);
        return launch_as<T, MmaWarp<T, kCodes, 256, 1>, kBytes>(ctx, p, st);
    }
    if (p.dh <= 64) return launch_as<T, MmaWarp<T, kCodes, 64, 2>, kBytes>(ctx, p, st);
    if (p.dh <= 128) return launch_as<T, MmaWarp<T, kCodes, 128, 2>, kBytes>(ctx, p, st);
    return launch_as<T, MmaWarp<T, kCodes, 256, 2>, kBytes>(ctx, p, st);
}

}  // namespace

size_t attend_workspace_bytes() { return (size_t)2 * kMaxCtas * kSlotFloats * sizeof(float); }
size_t attend_counter_bytes() { return kMaxCtas * sizeof(int); }

int launch_paged_attention(gelo_ctx* ctx, const gelo_kv_cache& kv, const void* q, int ldq, int q_heads, const int* len, float scale, int window,
                           int dtype, void* o, int ldo, float* lse, void* ws, cudaStream_t st)
{
    AttendArgs p;
    const bool codes = kv.dtype == GELO_E4M3;
    const long long bytes = codes ? 1 : (long long)elem_size(kv.dtype);
    p.q = q; p.k = kv.k_dev; p.v = kv.v_dev; p.o = o; p.lse = lse;
    p.slots = static_cast<float*>(ws); p.arrived = ctx->attend_arrived;
    p.len = len; p.table = kv.table_dev; p.status = ctx->status_dev;
    p.page_stride = kv.page_stride * bytes; p.token_stride = kv.token_stride * bytes; p.head_stride = kv.head_stride * bytes;
    p.ldq = ldq; p.ldo = ldo; p.q_heads = q_heads; p.kv_heads = kv.kv_heads; p.group = q_heads / kv.kv_heads; p.dh = kv.head_dim;
    p.pages = kv.pages; p.page_size = kv.page_size; p.seqs = kv.seqs; p.max_pages = kv.max_pages; p.table_ld = kv.table_ld;
    p.page_shift = -1;
    for (int b = 0; b < 31; ++b)
        if (kv.page_size == 1 << b) p.page_shift = b;
    p.window = window; p.scale = scale * kv.k_scale; p.v_scale = kv.v_scale;
    if (dtype == GELO_BF16) return codes ? launch_mma<__nv_bfloat16, true>(ctx, p, st) : launch_mma<__nv_bfloat16, false>(ctx, p, st);
    if (dtype == GELO_F16) return codes ? launch_mma<__half, true>(ctx, p, st) : launch_mma<__half, false>(ctx, p, st);
    if (p.dh <= 64) return launch_as<float, FmaWarp<64>, 4>(ctx, p, st);
    if (p.dh <= 128) return launch_as<float, FmaWarp<128>, 4>(ctx, p, st);
    return launch_as<float, FmaWarp<256>, 4>(ctx, p, st);
}

}  // namespace gelo
