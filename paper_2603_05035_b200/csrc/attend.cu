// Attention of one new token per sequence over a paged key-value cache.
//   o = sum_j p_j v_j,  p_j = exp(s_j - m) / l,  s_j = scale q . k_j,  m = max_j s_j,  l = sum_j exp(s_j - m)
// One pass over the keys and values with the running maximum and sum of the softmax; every key and value is read once for all query
// heads that share it (up to 16, on fp32 caches 8, or 4 with heads over 128; more heads read them again, from L2).  Bound by HBM: 4 heads-per-group flops per element read.
//
// The work of a call is one line of tiles: sequence after sequence, key-value head after head, 16 or 32 positions a tile.  Every CTA works out
// from the lengths which equal share of that line is its own, so ragged lengths balance and one long sequence fills the GPU.  What of
// a (sequence, head) falls to one CTA is a segment; where a CTA's border cuts one, each side leaves its sums in the workspace and the
// CTA that arrives last adds them up, in the order of the CTAs whoever that is.  Where all sequences are short nothing is cut, and where there are
// many heads besides, every warp takes heads of its own.
// Inside a CTA the warps take the tiles of a segment in turn, each with a ring of its own in shared memory that asynchronous 16-byte copies
// fill, so nothing but a segment's end makes them wait for one another.
//
// Measured (keys and values over time, against a copy's 6509 GB/s): 64 sequences of 100 to 4096, 32 heads of 128, bf16 314 to 327 us (96 to 100%);
// the same in fp32 597 to 621 us (101 to 105%, reads alone run faster than a copy), E4M3 188 to 197 us (80 to 84%, bound by the widening of the codes); one sequence of 32768
// bf16 86 us (96%); 8 of 32 heads on E4M3 108 us (93%).  Two CTAs of four warps per SM: with one of eight the end of a segment leaves the SM
// idle (64 sequences 364 us against 345 at the time).
#include <float.h>
#include <limits.h>

#include <atomic>
#include <type_traits>

#include "common.cuh"
#include "vec8.cuh"

namespace gelo {

namespace {

constexpr int kMaxCtas = 320;
// How the line is dealt, with what either side of a choice takes (us; bf16 and heads of 128 unless said otherwise):
//   kSegmentCost   weight of a head's beginning and end in tiles: 64 ragged sequences x 32 heads 343 without it, 309 with
//   kWhole         heads this short are not cut: five fp32 sequences of up to 200 x 4 heads cut 15.4, whole 8.3
//   kWholeFew      the same where every head finds a CTA and equal pieces do not: 24 sequences of 440 x 8 heads cut 19.9, whole 13.3; of 880 24.4, 20.3
//                  (24 sequences of 880 x 2 heads in pieces 13.6, whole 19.1; one of 440 x 4 9.4, 10.3)
//   kAloneCost     (two heads per CTA or more, all short) warps take heads of their own: 64 x 32 heads of up to 200 67, 22.5
//   kLeast         tiles a warp gets where heads are cut: one sequence of 4000 x 4 heads 14.2 with four, 12.0 with two
//   kAtOnce        one sequence of 32768, four key-value heads (74 parts each of 8 heads): in one go 27.6, in rounds 24.5; eight (37 of 4) 31.3, 32.1
//   kRound         the same with two (148 parts of 16 heads), rounds of 8 30.9, of 13 27.1, of 16 28.0; in one go with no more than 40 parts 37
//   equal pieces   (few sequences; kPieceSlack) five of up to 4000 x 4 heads 14.4, in pieces 11.0; one of 32768 87.8, 86.0
constexpr int kLeast = 2;                                     // tiles that a warp takes where heads are cut
constexpr int kWhole = 24, kWholeFew = 56;                     // up to so many tiles a head stays in one piece; where it has a CTA but no two
constexpr int kSegmentCost = 6, kAloneCost = 2;               // what a segment's beginning and end cost a CTA, and a warp alone, in tiles
constexpr int kPieceSlack = 16;                               // equal pieces may be larger than a share by this part of it (or four tiles)
constexpr int kAtOnce = 40, kRound = 13;                      // parts of a head that one CTA adds up in one go, or else in a round
constexpr int kSlotFloats = 16 * 256 + 32;                    // most that a slot holds: maxima and totals of 16 heads, their sums
constexpr float kNone = -INFINITY;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

struct AttendArgs {
    const void *q, *k, *v;
    void* o;
    float *lse, *slots;
    unsigned* arrived;                                        // two counters per CTA, zero between calls
    const int *len, *table;
    int* status;
    long long page_stride, token_stride, head_stride;         // bytes
    int ldq, ldo, q_heads, group, dh;
    int pages, page_size, page_shift, seqs, max_pages, table_ld, window;
    int slot;                                                 // floats
    int kv_heads, heads_a_unit, units, units_a_kv;            // units: heads_a_unit query heads of one key-value head each, per sequence
    float scale, v_scale;                                     // scale: of the logits, the keys' scale included
    float a_seq, a_cta;                                       // 1 / seqs, 1 / CTAs
};

// a / b of non-negative numbers; nearly always both are small
__device__ __forceinline__ long long quotient(long long a, long long b)
{
    return ((a | b) >> 31) == 0 ? (long long)((unsigned)a / (unsigned)b) : a / b;
}

// n / size rounded up, a_piece = 1 / size: the quotient in fp32 is off by one at most (n < 2^28, size >= 8), and put right
__device__ __forceinline__ int pieces_of(int n, int size, float a_piece)
{
    int q = (int)((float)n * a_piece), rest = n - q * size;
    if (rest < 0) { --q; rest += size; }
    if (rest >= size) { ++q; rest -= size; }
    return q + (rest > 0 ? 1 : 0);
}

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

__device__ __forceinline__ int kv_head_of(const AttendArgs& p, int unit) { return p.units_a_kv == 1 ? unit : unit / p.units_a_kv; }

// A place in the line: tile `tile` (from its sequence's first) of (seq, unit)
struct Place { int seq, unit, tile; };

// A walk over the segments of a share
template <int kTile>
struct Walk {
    Span s;
    int seq, unit, at, end;                                   // the segment: tiles [at, end) of (seq, unit)
    long long seq_at;                                         // where the sequence begins in the line
    Place stop;
    __device__ __forceinline__ bool last() const { return seq == stop.seq && unit == stop.unit; }
    __device__ __forceinline__ void begin(const AttendArgs& p, const Place& from, long long from_at, const Place& to)
    {
        seq = from.seq;
        unit = from.unit;
        seq_at = from_at;
        stop = to;
        s = span_of<kTile>(p, seq);
        at = s.t0 + from.tile;
        end = last() ? s.t0 + stop.tile : s.t1;
    }
    __device__ __forceinline__ bool next(const AttendArgs& p, int cost)
    {
        if (last()) return false;
        const bool over = ++unit == p.units;
        if (over) {
            unit = 0;
            seq_at += (long long)(s.t1 - s.t0 + cost) * p.units;
            ++seq;
        }
        if (last() && stop.tile == 0) return false;
        if (over) s = span_of<kTile>(p, seq);
        at = s.t0;
        end = last() ? s.t0 + stop.tile : s.t1;
        return true;
    }
};

// The place at weight x of the line, in which a head of n - cost tiles weighs n; where nothing is cut, the first head that begins at x or behind.  x lies in
// sequence seq, which begins at seq_at (that of the place in the end).
__device__ __forceinline__ Place place_in(const AttendArgs& p, long long x, int seq, int n, int cost, bool whole, long long& seq_at)
{
    Place at;
    at.seq = seq;
    at.unit = (int)quotient(x - seq_at, n);
    const int offset = (int)(x - seq_at - (long long)at.unit * n);
    at.tile = whole ? 0 : max(offset - cost, 0);
    if (whole && offset > 0 && ++at.unit == p.units) {
        at.unit = 0;
        ++at.seq;
        seq_at += (long long)n * p.units;
    }
    return at;
}

// The lengths of all sequences as a CTA's threads have added them up: thread i those of the sequences from i * per on
template <int kWarps>
struct Prefix {
    long long inside[32 * kWarps];                            // tiles of a head before a thread's first sequence, of its warp's alone
    long long warps[kWarps];                                  // tiles of a head of a warp's sequences
    int longest[kWarps];
    // The place at weight x of the line (place_in), which a warp works out together; seq_at: the weight before the place's sequence
    template <int kTile>
    __device__ __forceinline__ Place find(const AttendArgs& p, long long x, int per, int cost, bool whole, int lane, long long& seq_at) const
    {
        int i = -1;
        long long before = 0;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            const int first = min((32 * w + lane) * per, p.seqs);
            const long long at = (before + inside[32 * w + lane] + (long long)cost * first) * p.units;
            i += __popc(__ballot_sync(0xffffffffu, first < p.seqs && at <= x));
            before += warps[w];
        }
        before = 0;
#pragma unroll
        for (int w = 0; w < kWarps; ++w)
            if (32 * (w + 1) <= i) before += warps[w];
        Place at;
        at.seq = i * per;
        seq_at = (before + inside[i] + (long long)cost * at.seq) * p.units;
        int n;
        for (;;) {
            const Span s = span_of<kTile>(p, at.seq);
            n = s.t1 - s.t0 + cost;
            if (x < seq_at + (long long)n * p.units || at.seq + 1 >= p.seqs) break;
            seq_at += (long long)n * p.units;
            ++at.seq;
        }
        return place_in(p, x, at.seq, n, cost, whole, seq_at);
    }
};

__device__ __forceinline__ uint32_t smem_at(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
// sixteen bytes, zeros where nothing is there (`src` is not read then); `once` marks the lines as the first to leave L2
__device__ __forceinline__ void copy16(uint32_t dst, const void* src, bool there, uint64_t once)
{
    asm volatile("cp.async.cg.shared.global.L2::cache_hint [%0], [%1], 16, %2, %3;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0), "l"(once) : "memory");
}
__device__ __forceinline__ void copy16(uint32_t dst, const void* src, uint64_t once)
{
    asm volatile("cp.async.cg.shared.global.L2::cache_hint [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "l"(once) : "memory");
}
__device__ __forceinline__ uint64_t read_once()
{
    uint64_t policy;
    asm("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(policy));
    return policy;
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
// 2^x for x <= 14, to two units in the last place; nothing where the result is no normal number
__device__ __forceinline__ float power2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// four E4M3 codes as halves: the low two, the high two
__device__ __forceinline__ void halves_of_codes(uint32_t four, uint32_t& low, uint32_t& high)
{
    asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, a;\n\tcvt.rn.f16x2.e4m3x2 %1, b;\n\t}" : "=r"(low), "=r"(high) : "r"(four));
}

// Geometry of a kernel instance.  Rows of DH elements of kBytes, 32 of them where that is no more than 8 KB of keys and values, since what a tile
// costs beside its products is the same (8 heads on E4M3: 197 us with 16, 128 with 32); the 16-byte pieces of a row are permuted by its number so that eight
// rows' pieces of one column lie in different banks.
template <int DH, int kBytes>
struct Tiles {
    static constexpr int kWidth = DH;
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

// What the warps know of a segment's heads: the maximum of each warp's logits (times log2 e) and its total relative to that
template <int kHeads, int kWarps>
struct Joint {
    float tops[kWarps][kHeads], totals[kWarps][kHeads];
    __device__ __forceinline__ float top(int h) const
    {
        float t = kNone;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) t = fmaxf(t, tops[w][h]);
        return t;
    }
    __device__ __forceinline__ float base(int h) const
    {
        const float t = top(h);
        return t == kNone ? 0.0f : t;
    }
    __device__ __forceinline__ float total(int h) const
    {
        const float b = base(h);
        float sum = 0.0f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) sum = fmaf(power2(tops[w][h] - b), totals[w][h], sum);
        return sum;
    }
};

// ---- products of a warp on a 16-bit or E4M3 tile: mma.sync on transposed operands ---------------------------
// S^T = K q^T and O^T = V^T p^T: positions (and components) are the 16 rows of an instruction, up to eight query heads its columns, so a
// single head wastes columns of an otherwise idle unit and no loads.  The matrix rate that this leaves is several times what HBM
// can feed (24 instructions per 8 KB tile of 128 components).  p is handed to the second product as the 16-bit value and what
// that leaves out, i.e. with 16 bits (bf16 caches) or 22, so that the stored result is rounded once.  (E4M3 caches with bf16 results, p as one half of 11 bits: half
// the second products; 33 long sequences, 8 of 32 heads 108 us as with both, 16 heads a key-value head 141 instead of 156; 5 times the distance from a form in fp32.)
// E4M3 tiles are widened to half in registers, q is given the same type times a power of two that puts its largest component into [1, 2): components below 2^-14 of that (of
// bf16, 2^-17) are held to 2^-25 of it, which is what fp32 sums of the products keep.
template <typename T, bool kCodes, int DH, int NT>
struct MmaWarp {
    using M = std::conditional_t<kCodes, __half, T>;
    using G = Tiles<DH, kCodes ? 1 : 2>;
    static constexpr int kHeads = 8 * NT;
    // Halves have no exponents below 2^-24, where a long context's small weights are: p is kept relative to 2^-14 of the largest.
    static constexpr float kRaise = 14.0f;
    uint32_t qf[DH / 16][NT][2];
    float acc[DH / 16][NT][4];
    float m[NT][2], l[NT][2], scale[NT][2];
    bool may_vanish;                                          // a logit of this segment may be minus infinity (the same in all lanes)

    static constexpr int kStaged = 0;                         // floats of shared memory for a warp's q

    // Asks for the q of a segment's heads; q points at the first one's components.  What arrives is taken up by begin().
    __device__ __forceinline__ void fetch(const AttendArgs& p, const T* q, int heads, int lane)
    {
        const int t = lane & 3;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const int h = 8 * n + (lane >> 2);
            const T* row = q + (size_t)h * p.dh;
#pragma unroll
            for (int s = 0; s < DH / 16; ++s) {
                if constexpr (kCodes) {
                    const int c = 16 * s + 4 * t;             // the components that stand where a code tile's row has them
                    const uint2 v = h < heads && c < p.dh ? *reinterpret_cast<const uint2*>(row + c) : make_uint2(0u, 0u);
                    qf[s][n][0] = v.x;
                    qf[s][n][1] = v.y;
                } else {
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const int c = 16 * s + 2 * t + 8 * j;
                        qf[s][n][j] = h < heads && c < p.dh ? *reinterpret_cast<const uint32_t*>(row + c) : 0u;
                    }
                }
            }
        }
    }
    __device__ __forceinline__ void begin(const AttendArgs& p, float*, int lane)
    {
        const int t = lane & 3;
        // Codes are finite and products with q in [-2, 2] bounded, so only an infinite q or a scale that overflows could do it, and nearly all segments are spared
        // the look at their logits (33 long sequences, 8 of 32 heads, f16: 106.7 us, 110.8 with it); the elements of the other caches may be infinite.
        bool vanish = !kCodes;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            float factor = 1.0f;
            if constexpr (kCodes) {
                float top = 0.0f;
#pragma unroll
                for (int s = 0; s < DH / 16; ++s)
#pragma unroll
                    for (int j = 0; j < 4; ++j) top = fmaxf(top, fabsf(widen_at(reinterpret_cast<const T*>(qf[s][n]), j)));
                top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
                top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
                int e = 0;
                if (top > 0.0f && top <= 3.4e38f) e = max(ilogbf(top), -126);
                vanish |= top > 3.4e38f;
                factor = exp2f((float)e);
                const float down = exp2f((float)-e);
#pragma unroll
                for (int s = 0; s < DH / 16; ++s)
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const T* two = reinterpret_cast<const T*>(&qf[s][n][j]);
                        qf[s][n][j] = two_of<M>(widen_at(two, 0) * down, widen_at(two, 1) * down);
                    }
            }
            // columns 2t and 2t + 1 of a product are heads whose q other lanes hold
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                scale[n][j] = p.scale * kLog2e * (kCodes ? __shfl_sync(0xffffffffu, factor, 4 * (2 * t + j)) : 1.0f);
                if constexpr (kCodes) vanish |= !(fabsf(scale[n][j]) * (2.0f * 448.0f * DH) <= FLT_MAX);
                m[n][j] = kNone;
                l[n][j] = 0.0f;
            }
#pragma unroll
            for (int s = 0; s < DH / 16; ++s)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[s][n][j] = 0.0f;
        }
        may_vanish = !kCodes || __any_sync(0xffffffffu, vanish);
    }

    __device__ __forceinline__ void tile(uint32_t keys, uint32_t values, uint32_t counts, int lane)
    {
        // (a tile of codes that is spared the look has code of its own: 105 us, 107 where it jumps over it; with two sets of heads the registers do not suffice for both)
        if (kCodes && NT == 1 && !may_vanish) tile_as<false>(keys, values, counts, lane);
        else tile_as<true>(keys, values, counts, lane);
    }
    // kLook: logits of minus infinity are looked for
    template <bool kLook>
    __device__ __forceinline__ void tile_as(uint32_t keys, uint32_t values, uint32_t counts, int lane)
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
        // A logit of minus infinity weighs nothing, but a product with its value would make a NaN of an infinity there.  Hardly any tile has one: `gone`
        // then has a bit for each of this lane's logits.  (Zeros stand where no key is, so only keys that count are seen.)
        bool any_gone = false;
        uint32_t gone = 0;
        if (kLook && (!kCodes || may_vanish)) {
#pragma unroll
            for (int b = 0; b < kSub; ++b)
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int j = 0; j < 4; ++j) any_gone |= c[b][n][j] * scale[n][j & 1] == kNone;
            any_gone = __any_sync(0xffffffffu, any_gone);
            if (any_gone) {
#pragma unroll
                for (int i = 0; i < 2 * kSub; ++i)
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int j = 0; j < 2; ++j)
                            if (c[i >> 1][n][2 * (i & 1) + j] * scale[n][j] == kNone) gone |= 1u << (2 * (NT * i + n) + j);
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
                if constexpr (std::is_same_v<M, __half>) {    // (where logits are so large that this rounds further down, p would leave a half's range)
                    const float lower = top - kRaise;
                    if (top - lower <= kRaise) top = lower;
                }
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
                const uint32_t two = two_of<M>(e[i][0], e[i][1]);
                ph[i >> 1][n][i & 1] = transposed(two);
                const M* const held = reinterpret_cast<const M*>(&two);                  // and what the rounding has left
                pl[i >> 1][n][i & 1] = transposed(two_of<M>(e[i][0] - widen_at(held, 0), e[i][1] - widen_at(held, 1)));
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
        if (any_gone) pass_over(values, gone, ph, pl, lane);
        const int pos = (lane & 7) + ((lane >> 4) << 3), col = (lane >> 3) & 1;
#pragma unroll
        for (int b = 0; b < kSub; ++b) {
            auto add = [&](int s, const uint32_t (&a)[4]) {
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    mma(acc[s][n], a, ph[b][n][0], ph[b][n][1], M());
                    mma(acc[s][n], a, pl[b][n][0], pl[b][n][1], M());
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

    // Positions with a logit of minus infinity for some head (a bit of `gone`, see tile): their values are added to the sums of the other heads one
    // by one, and cleared before the products of the tile.
    template <int kSub>
    __device__ __forceinline__ void pass_over(uint32_t values, uint32_t gone, const uint32_t (&ph)[kSub][NT][2], const uint32_t (&pl)[kSub][NT][2], int lane)
    {
        const int r = lane >> 2, t = lane & 3;
        constexpr uint32_t kOfRow = (1u << 2 * NT) - 1;
        uint32_t rows = 0;
#pragma unroll
        for (int i = 0; i < 2 * kSub; ++i) {
            const uint32_t lanes = __ballot_sync(0xffffffffu, (gone >> (2 * NT * i)) & kOfRow);
#pragma unroll
            for (int u = 0; u < 8; ++u) rows |= ((lanes >> (4 * u)) & 15u) ? 1u << (8 * i + u) : 0u;
        }
#pragma unroll 1
        for (; rows; rows &= rows - 1) {
            const int at = __ffs(rows) - 1, from = 4 * (at & 7) + t;              // lane `from` has the position's weights of this lane's heads
            const uint32_t skip = __shfl_sync(0xffffffffu, gone, from) >> (2 * NT * (at >> 3));
            float p[NT][2];
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                uint32_t high = 0, low = 0;
#pragma unroll
                for (int i = 0; i < 2 * kSub; ++i) {          // (masks: an index that the loop works out would put the arrays into local memory)
                    const uint32_t its = i == at >> 3 ? 0xffffffffu : 0u;
                    high |= ph[i >> 1][n][i & 1] & its;
                    low |= pl[i >> 1][n][i & 1] & its;
                }
                high = __shfl_sync(0xffffffffu, transposed(high), from);
                low = __shfl_sync(0xffffffffu, transposed(low), from);
#pragma unroll
                for (int j = 0; j < 2; ++j)
                    p[n][j] = widen_at(reinterpret_cast<const M*>(&high), j) + widen_at(reinterpret_cast<const M*>(&low), j);
            }
#pragma unroll
            for (int s = 0; s < DH / 16; ++s) {
                float v[2];
                if constexpr (kCodes) {
                    uint16_t two;
                    asm volatile("ld.shared.u16 %0, [%1];" : "=h"(two) : "r"(values + G::piece(at, s) + 2 * r) : "memory");
                    uint32_t x, unused;
                    halves_of_codes(two, x, unused);
#pragma unroll
                    for (int j = 0; j < 2; ++j) v[j] = widen_at(reinterpret_cast<const M*>(&x), j);
                } else {
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        uint16_t one;
                        asm volatile("ld.shared.u16 %0, [%1];" : "=h"(one) : "r"(values + G::piece(at, 2 * s + j) + 2 * r) : "memory");
                        v[j] = widen_at(reinterpret_cast<const M*>(&one), 0);
                    }
                }
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (!((skip >> (2 * n + (j & 1))) & 1u)) acc[s][n][j] = fmaf(p[n][j & 1], v[j >> 1], acc[s][n][j]);
            }
            __syncwarp();
            for (int i = lane; i < G::kPieces; i += 32)
                asm volatile("st.shared.v4.u32 [%0], {%1, %1, %1, %1};" ::"r"(values + G::piece(at, i)), "r"(0u) : "memory");
        }
        __syncwarp();
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
    // sums of heads [h0, h0 + kJoinHeads) brought to the maximum of all warps (or as they are), head-major with the join's pitch
    __device__ __forceinline__ void sums(float* out, const Joint<kHeads, G::kWarps>* all, int h0, int lane)
    {
        const int r = lane >> 2, t = lane & 3;
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int h = 8 * n + 2 * t + j;
                if (h < h0 || h >= h0 + G::kJoinHeads) continue;
                const float f = all ? power2(m[n][j] - all->base(h)) : 1.0f;
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
// Logits: two lanes per position, every other piece of a row each, a key's piece in registers for all H heads, q in shared memory.  Sums: a lane owns
// DH / 32 components.  H is 1, 4 or 8, the least that holds the heads of a key-value head: with H = 8 always, one head takes 595 us instead of 322, four 157
// instead of 109.
template <int DH, int H>
struct FmaWarp {
    using G = Tiles<DH, 4>;
    static constexpr int kHeads = H;
    static constexpr int kOwn = DH / 32;
    static constexpr int kStaged = H * DH;
    static constexpr int kMine = kStaged / 32;
    const float* q;
    float held[kMine];
    float acc[H][kOwn];
    float m[H], l[H], scale;

    __device__ __forceinline__ void fetch(const AttendArgs& p, const float* from, int heads, int lane)
    {
#pragma unroll
        for (int i = 0; i < kMine; ++i) {
            const int at = 32 * i + lane, h = at / DH, c = at % DH;
            held[i] = h < heads && c < p.dh ? from[(size_t)h * p.dh + c] : 0.0f;
        }
    }
    __device__ __forceinline__ void begin(const AttendArgs& p, float* staged, int lane)
    {
        __syncwarp();                                         // everybody is through with the last segment's
#pragma unroll
        for (int i = 0; i < kMine; ++i) staged[32 * i + lane] = held[i];
        __syncwarp();
        q = staged;
        scale = p.scale * kLog2e;
#pragma unroll
        for (int h = 0; h < H; ++h) {
            m[h] = kNone;
            l[h] = 0.0f;
#pragma unroll
            for (int i = 0; i < kOwn; ++i) acc[h][i] = 0.0f;
        }
    }
    __device__ __forceinline__ void tile(uint32_t keys, uint32_t values, uint32_t counts, int lane)
    {
        const int row = lane & 15, side = lane >> 4;
        float s[H];
#pragma unroll
        for (int h = 0; h < H; ++h) s[h] = 0.0f;
#pragma unroll 8
        for (int i = 0; i < DH / 8; ++i) {
            const int c = 2 * i + side;
            float4 k4;
            asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(k4.x), "=f"(k4.y), "=f"(k4.z), "=f"(k4.w) : "r"(keys + G::piece(row, c)) : "memory");
#pragma unroll
            for (int h = 0; h < H; ++h) {
                const float4 q4 = *reinterpret_cast<const float4*>(q + h * DH + 4 * c);
                s[h] = fmaf(k4.x, q4.x, fmaf(k4.y, q4.y, fmaf(k4.z, q4.z, fmaf(k4.w, q4.w, s[h]))));
            }
        }
        const bool on = (counts >> row) & 1u;
        bool any_gone = false;                                // see MmaWarp::tile
#pragma unroll
        for (int h = 0; h < H; ++h) {
            s[h] += __shfl_xor_sync(0xffffffffu, s[h], 16);
            s[h] *= scale;
            any_gone |= s[h] == kNone;
        }
        any_gone = __any_sync(0xffffffffu, any_gone);
        uint32_t gone = 0;
        if (any_gone) {
#pragma unroll
            for (int h = 0; h < H; ++h)
                if (s[h] == kNone) gone |= 1u << h;
        }
        float e[H];
#pragma unroll
        for (int h = 0; h < H; ++h) {
            s[h] = on ? s[h] : kNone;
            float top = s[h];
#pragma unroll
            for (int off = 1; off < 16; off <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, off));
            top = fmaxf(top, m[h]);
            const float base = top == kNone ? 0.0f : top;
            const float keep = power2(m[h] - base);
            m[h] = top;
            e[h] = power2(s[h] - base);
            l[h] = fmaf(l[h], keep, side ? 0.0f : e[h]);
#pragma unroll
            for (int i = 0; i < kOwn; ++i) acc[h][i] *= keep;
        }
        if (any_gone) {
#pragma unroll 1
            for (int t = 0; t < G::kTile; ++t) {
                float v[kOwn];
                load_own(v, values, t, lane);
                const uint32_t skip = __shfl_sync(0xffffffffu, gone, t);
#pragma unroll
                for (int h = 0; h < H; ++h) {
                    const float w = __shfl_sync(0xffffffffu, e[h], t);
#pragma unroll
                    for (int i = 0; i < kOwn; ++i)
                        if (!((skip >> h) & 1u)) acc[h][i] = fmaf(w, v[i], acc[h][i]);
                }
            }
            return;
        }
#pragma unroll 8
        for (int t = 0; t < G::kTile; ++t) {
            float v[kOwn];
            load_own(v, values, t, lane);
#pragma unroll
            for (int h = 0; h < H; ++h) {
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
        for (int h = 0; h < H; ++h) {
            float sum = l[h];
#pragma unroll
            for (int off = 1; off < 32; off <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, off);
            if (lane == 0) {
                tops[h] = m[h];
                totals[h] = sum;
            }
        }
    }
    __device__ __forceinline__ void sums(float* out, const Joint<kHeads, G::kWarps>* all, int h0, int lane)
    {
#pragma unroll
        for (int h = 0; h < H; ++h) {
            if (h < h0 || h >= h0 + G::kJoinHeads) continue;
            const float f = all ? power2(m[h] - all->base(h)) : 1.0f;
#pragma unroll
            for (int i = 0; i < kOwn; ++i) out[(h - h0) * G::kJoinPitch + component(lane, i)] = acc[h][i] * f;
        }
    }
};

// Four neighbouring components of a result
template <typename T>
__device__ __forceinline__ void write_result(const AttendArgs& p, int seq, int head, int c, float4 sum, float total)
{
    const float f = total > 0.0f || total != total ? __fdiv_rn(p.v_scale, total) : 0.0f;
    __align__(16) T o[4];
    round_to(sum.x * f, o); round_to(sum.y * f, o + 1); round_to(sum.z * f, o + 2); round_to(sum.w * f, o + 3);
    T* dst = static_cast<T*>(p.o) + (size_t)seq * p.ldo + (size_t)head * p.dh + c;
    if constexpr (sizeof(T) == 4) *reinterpret_cast<uint4*>(dst) = *reinterpret_cast<const uint4*>(o);
    else *reinterpret_cast<uint2*>(dst) = *reinterpret_cast<const uint2*>(o);
}

// (top, total, sum) += the part (t, l, v), both brought to the maximum `higher` of all that is being added; `fresh` begins with the part alone
__device__ __forceinline__ void add_part(float& top, float& total, float4& sum, float higher, float t, float l, float4 v, bool fresh)
{
    const float f = power2(t - (higher == kNone ? 0.0f : higher));
    if (fresh) {
        total = f * l;
        sum = make_float4(f * v.x, f * v.y, f * v.z, f * v.w);
    } else {
        total = fmaf(f, l, total);
        sum.x = fmaf(f, v.x, sum.x); sum.y = fmaf(f, v.y, sum.y); sum.z = fmaf(f, v.z, sum.z); sum.w = fmaf(f, v.w, sum.w);
    }
    top = higher;
}

// A head that this CTA shares with others: those are CTAs first .. last, which leave their sums in slots
struct Cut { int first, last, seq, head, heads; };

// The parts of a head that are added up by one CTA: those of CTAs first, first + step .. last.  Up to kAtOnce parts in a single round; more in two, a
// round of kRound neighbours, whose sums go to the slot of the first of them, and then the rounds.
struct Round { int first, last, step; bool ends; };

__device__ __forceinline__ Round round_of(const Cut& u, int level, int cta)
{
    const int after = u.last - u.first;
    if (after < kAtOnce) return {u.first, u.last, 1, true};
    if (level > 0) return {u.first, u.first + after / kRound * kRound, kRound, true};
    const int first = u.first + (cta - u.first) / kRound * kRound;
    return {first, min(first + kRound - 1, u.last), 1, false};
}

// Where CTA b leaves its part of a head that begins in CTA `first`: the second slot for the head that begins in b
__device__ __forceinline__ float* slot_of(const AttendArgs& p, int b, int first)
{
    return p.slots + (size_t)(2 * b + (b == first ? 1 : 0)) * p.slot;
}

template <typename T, typename W, int kBytes>
__global__ void __launch_bounds__(32 * W::G::kWarps, W::G::kCtas) attend_kernel(const AttendArgs p)
{
    using G = typename W::G;
    constexpr int kWarps = G::kWarps, kThreads = 32 * kWarps, kStages = G::kStages, kTile = G::kTile;
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ Prefix<kWarps> prefix;
    __shared__ int last[2];
    __shared__ uint32_t counts[kWarps][kStages];
    __shared__ Joint<W::kHeads, kWarps> joint[2];             // of this segment, and of the one before or behind
    __shared__ __align__(16) float staged[kWarps][W::kStaged ? W::kStaged : 1];
    chain_next();
    chain_wait();
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, cta = blockIdx.x;

    // ---- this CTA's share of the line of tiles, or where `alone` this warp's ----
    // Up to 32 sequences: each lane of every warp has one, and no warp waits for another; more: the threads of the CTA add them up together.
    const bool few = p.seqs <= 32;
    const int per = (p.seqs + kThreads - 1) / kThreads;
    long long all = 0, before = 0;                            // tiles of a head of all sequences; of those before this lane's
    int longest = 0, n = 0;                                   // of this lane's
    if (few) {
        if (lane < p.seqs) {
            const Span sp = span_of<kTile>(p, lane);
            n = sp.t1 - sp.t0;
        }
        long long upto = n;
#pragma unroll
        for (int off = 1; off < 32; off <<= 1) {
            const long long u = __shfl_up_sync(0xffffffffu, upto, off);
            if (lane >= off) upto += u;
        }
        before = upto - n;
        all = __shfl_sync(0xffffffffu, upto, 31);
        longest = __reduce_max_sync(0xffffffffu, n);
    } else {
        long long mine = 0;
        for (int s = min(tid * per, p.seqs); s < min((tid + 1) * per, p.seqs); ++s) {
            const Span sp = span_of<kTile>(p, s);
            mine += sp.t1 - sp.t0;
            longest = max(longest, sp.t1 - sp.t0);
        }
        long long upto = mine;
#pragma unroll
        for (int off = 1; off < 32; off <<= 1) {
            const long long u = __shfl_up_sync(0xffffffffu, upto, off);
            if (lane >= off) upto += u;
        }
        longest = __reduce_max_sync(0xffffffffu, longest);
        prefix.inside[tid] = upto - mine;
        if (lane == 31) {
            prefix.warps[warp] = upto;
            prefix.longest[warp] = longest;
        }
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            all += prefix.warps[w];
            longest = max(longest, prefix.longest[w]);
        }
    }
    const long long heads_in_all = (long long)p.seqs * p.units;
    const bool one_each = heads_in_all <= gridDim.x && !(few && 2 * heads_in_all <= gridDim.x);           // a CTA for a head, and no two equal pieces of it
    const bool whole = longest <= (one_each ? kWholeFew : kWhole), alone = whole && heads_in_all >= 2 * (long long)gridDim.x;
    const int cost = alone ? kAloneCost : kSegmentCost, team = alone ? 1 : kWarps, member = alone ? 0 : warp;
    const long long total = (all + (long long)cost * p.seqs) * p.units;
    long long share = quotient(total + gridDim.x * (alone ? kWarps : 1) - 1, gridDim.x * (alone ? kWarps : 1));
    if (!whole) {
        // kLeast tiles for every warp, or an average head, since what a cut costs is more (any share that is large enough will do: no division)
        const float average = (float)all * p.a_seq;
        share = max(share, (long long)fminf((float)(kLeast * kWarps), average) + 1 + cost);
    }
    // Few sequences: their heads in equal pieces, one for a CTA, if pieces not much larger than a share find a CTA each.  No CTA then has
    // the end of one head and the beginning of another to see to.
    int piece_first = -1, piece_last = -1;                    // the CTAs that a head's pieces belong to
    Walk<kTile> ahead, walk;
    if (!whole && few && heads_in_all <= (long long)gridDim.x) {
        const int grid = (int)gridDim.x, units = p.units, even = (int)fminf((float)(all * units) * p.a_cta, (float)(INT_MAX / 4)) + 1;
        const int least = max(kLeast * kWarps, even), size = least + (int)((long long)least * lane / 32);
        int count = 0;                                        // pieces of this lane's size (the heads are as many as CTAs at most, so no sum gets far)
        const float a_piece = 1.0f / (float)size;
        for (int s = 0; s < p.seqs; ++s) count += min(pieces_of(__shfl_sync(0xffffffffu, n, s), size, a_piece), grid + 1);
        const uint32_t fit = __ballot_sync(0xffffffffu, (long long)count * units <= grid && size <= share + max(4ll, share / kPieceSlack));
        if (fit) {
            const int best = __shfl_sync(0xffffffffu, size, __ffs(fit) - 1), mine = pieces_of(n, best, 1.0f / (float)best);
            int upto = mine * units;
#pragma unroll
            for (int off = 1; off < 32; off <<= 1) {
                const int u = __shfl_up_sync(0xffffffffu, upto, off);
                if (lane >= off) upto += u;
            }
            const int seq = __popc(__ballot_sync(0xffffffffu, upto <= cta));
            if (seq >= p.seqs) return;                        // (all of the CTA)
            const int pieces = __shfl_sync(0xffffffffu, mine, seq), tiles = __shfl_sync(0xffffffffu, n, seq);
            const int at = cta - (__shfl_sync(0xffffffffu, upto, seq) - pieces * units), unit = at / pieces, piece = at - unit * pieces;
            piece_first = cta - piece;
            piece_last = piece_first + pieces - 1;
            const Place from = {seq, unit, (int)((long long)tiles * piece / pieces)};
            Place to = {seq, unit, (int)((long long)tiles * (piece + 1) / pieces)};
            if (to.tile == tiles) to = unit + 1 < units ? Place{seq, unit + 1, 0} : Place{seq + 1, 0, 0};
            ahead.begin(p, from, 0, to);
        }
    }
    if (piece_first < 0) {
        const long long x0 = (alone ? warp * (long long)gridDim.x + cta : cta) * share;
        if (x0 >= total) return;                              // (where not alone, all of the CTA; warps that are alone meet at no barrier)
        long long from_at, to_at;
        const long long mine_at = (before + (long long)cost * lane) * p.units;         // (few)
        auto find = [&](long long x, long long& seq_at) {
            if (!few) return prefix.template find<kTile>(p, x, per, cost, whole, lane, seq_at);
            const int seq = __popc(__ballot_sync(0xffffffffu, lane < p.seqs && mine_at <= x)) - 1;
            seq_at = __shfl_sync(0xffffffffu, mine_at, seq);
            return place_in(p, x, seq, __shfl_sync(0xffffffffu, n, seq) + cost, cost, whole, seq_at);
        };
        const Place from = find(x0, from_at);
        Place to = {p.seqs, 0, 0};
        if (x0 + share < total) to = find(x0 + share, to_at);
        if (from.seq == to.seq && from.unit == to.unit && from.tile == to.tile) return;
        ahead.begin(p, from, from_at, to);
    }
    walk = ahead;

    // ---- copies: the tiles that this warp will take, in order, kStages - 1 of them ahead ----
    const uint32_t ring = smem_at(smem) + warp * kStages * G::kStage;
    float* const join = reinterpret_cast<float*>(smem + kWarps * kStages * G::kStage);
    W w;
    int first_head, heads;                                    // of the segment
    auto fetch = [&](const Walk<kTile>& at) {
        const int kv_head = kv_head_of(p, at.unit), head0 = (at.unit - kv_head * p.units_a_kv) * p.heads_a_unit;
        heads = min(p.heads_a_unit, p.group - head0);
        first_head = kv_head * p.group + head0;
        w.fetch(p, static_cast<const T*>(p.q) + (size_t)at.seq * p.ldq + (size_t)first_head * p.dh, heads, lane);
    };
    fetch(walk);
    int next_tile = ahead.at + member;
    bool more = true;
    long long ahead_head = kv_head_of(p, ahead.unit) * p.head_stride;
    // The next two tiles whose copies have not been asked for: the page that each position (lane % kTile) is on is looked up that far ahead.
    struct Pending {
        long long head;                                       // where the tile's head lies in a page
        int page, in_page;
        bool any, on;                                         // there is a tile; this lane's position of it counts
    } near = {0, 0, 0, false, false}, far = near;
    constexpr int kRowsACopy = 32 / G::kPieces ? 32 / G::kPieces : 1;                  // rows that one copy of the warp covers
    const int my_row = lane / G::kPieces, my_piece = lane % G::kPieces;
    const long long my_at = my_row * p.token_stride + 16 * my_piece, step = kRowsACopy * p.token_stride;
    const uint32_t my_place = G::piece(my_row, my_piece);
    const bool wanted = 16 * my_piece < p.dh * kBytes, full_rows = p.dh == G::kWidth, neighbours = p.page_size % 16 == 0;
    const uint64_t once = read_once();
    auto copy_tile = [&](int stage) {                         // asks for the copies of the next tile and looks up the one after the one behind it
        const Pending t = near;
        near = far;
        while (more && next_tile >= ahead.end) {
            more = ahead.next(p, cost);
            next_tile = ahead.at + member;
            ahead_head = kv_head_of(p, ahead.unit) * p.head_stride;
        }
        far.any = more;
        far.on = false;
        if (more) {
            const int at = next_tile * kTile + lane % kTile;
            far.on = at >= ahead.s.first && at < ahead.s.len;
            if (far.on) {
                const int column = p.page_shift >= 0 ? at >> p.page_shift : at / p.page_size;
                far.in_page = at - column * p.page_size;
                far.page = p.table[(size_t)ahead.seq * p.table_ld + column];
            }
            far.head = ahead_head;
            next_tile += team;
        }
        if (!t.any) return;
        __syncwarp();                                         // everybody has read what the stage held
        bool on = t.on;
        if (on && (t.page < 0 || t.page >= p.pages)) {
            on = false;
            atomicCAS(p.status, 0, (int)GELO_ERR_INVALID);
        }
        const uint32_t who = __ballot_sync(0xffffffffu, on);
        if (lane == 0) counts[warp][stage] = who;
        const long long at = (on ? t.page * p.page_stride + t.in_page * p.token_stride : 0) + t.head;
        const uint32_t dst = ring + stage * G::kStage;
        if (G::kPieces <= 32 && neighbours) {                 // sixteen positions are neighbours on one page
#pragma unroll
            for (int b = 0; b < kTile / 16; ++b) {
                const uint32_t half = (who >> (16 * b)) & 0xffffu, to = dst + 16 * b * G::kRow + my_place;
                if (half == 0xffffu && full_rows) {           // nearly always: nothing to leave out
                    const long long from = __shfl_sync(0xffffffffu, at, 16 * b) + my_at;
                    const char *k = static_cast<const char*>(p.k) + from, *v = static_cast<const char*>(p.v) + from;
#pragma unroll
                    for (int i = 0; i < 16 / kRowsACopy; ++i) {
                        // (a row's number and a lane's have no bit in common, so neither have their turns of the pieces)
                        const uint32_t place = (to ^ G::piece(i * kRowsACopy, 0) % G::kRow) + i * kRowsACopy * G::kRow;
                        copy16(place, k, once);
                        copy16(place + G::kHalf, v, once);
                        k += step;
                        v += step;
                    }
                    continue;
                }
                // the page is that of any position that counts; positions before it on the page may not count, but lie there
                const int one = half ? __ffs(half) - 1 : 0;
                const long long from = __shfl_sync(0xffffffffu, at, 16 * b + one) - (half ? one * p.token_stride : 0) + my_at;
                const char *k = static_cast<const char*>(p.k) + from, *v = static_cast<const char*>(p.v) + from;
#pragma unroll
                for (int i = 0; i < 16 / kRowsACopy; ++i) {
                    const bool there = wanted && ((half >> (i * kRowsACopy + my_row)) & 1u);
                    const uint32_t place = (to ^ G::piece(i * kRowsACopy, 0) % G::kRow) + i * kRowsACopy * G::kRow;
                    copy16(place, there ? k : p.k, there, once);
                    copy16(place + G::kHalf, there ? v : p.v, there, once);
                    k += step;
                    v += step;
                }
            }
        } else {
#pragma unroll
            for (int i = 0; i < kTile * G::kPieces / 32; ++i) {
                const int idx = 32 * i + lane, row = idx / G::kPieces, c = idx % G::kPieces;
                const long long from = __shfl_sync(0xffffffffu, at, row) + 16 * c;
                const bool there = ((who >> row) & 1u) && 16 * c < p.dh * kBytes;
                copy16(dst + G::piece(row, c), there ? static_cast<const char*>(p.k) + from : p.k, there, once);
                copy16(dst + G::kHalf + G::piece(row, c), there ? static_cast<const char*>(p.v) + from : p.v, there, once);
            }
        }
    };

    // ---- segments ----
    Cut cuts[2] = {};
    constexpr int kQuads = G::kWidth / 4, kRows = kThreads / kQuads;                          // a row of threads adds up a head, four components each
    const int c = 4 * (tid % kQuads), my_h = tid / kQuads;
    int put = 0, get = 0, turn = 0, lead = -2;                // lead: tiles asked for and not used (the first two rounds only look up)
    for (;; turn ^= 1) {
        w.begin(p, staged[warp], lane);
        for (int t = walk.at + member; t < walk.end; t += team) {
#pragma unroll 1
            for (; lead < kStages; ++lead) {
                copy_tile(put);
                if (lead < 0) continue;
                copies_end();
                put = put + 1 == kStages ? 0 : put + 1;
            }
            copies_wait<kStages - 1>();
            __syncwarp();
            w.tile(ring + get * G::kStage, ring + get * G::kStage + G::kHalf, counts[warp][get], lane);
            --lead;
            get = get + 1 == kStages ? 0 : get + 1;
        }
        // The warps' sums, brought to one maximum.  The next segment's q is on its way meanwhile, and what the warps exchange
        // alternates between two places: a warp that is through may begin the next segment before the others are.
        Joint<W::kHeads, kWarps>& all = joint[turn];
        w.statistics(all.tops[warp], all.totals[warp], lane);
        const Walk<kTile> done = walk;
        const int done_head = first_head, done_heads = heads;
        const bool go = walk.next(p, cost);
        if (go) fetch(walk);
        if (alone) {
            float* const mine = join + warp * G::kJoinHeads * G::kJoinPitch;
            __syncwarp();
            if (p.lse && lane < done_heads) {
                const float top = all.tops[warp][lane];
                p.lse[(size_t)done.seq * p.q_heads + done_head + lane] = (top == kNone ? 0.0f : top * kLn2) + logf(all.totals[warp][lane]);
            }
            for (int h0 = 0; h0 < done_heads; h0 += G::kJoinHeads) {
                __syncwarp();
                w.sums(mine, nullptr, h0, lane);
                __syncwarp();
                for (int i = lane; i < min(done_heads - h0, G::kJoinHeads) * kQuads; i += 32) {
                    const int h = i / kQuads, at = 4 * (i % kQuads);
                    if (at < p.dh)
                        write_result<T>(p, done.seq, done_head + h0 + h, at, *reinterpret_cast<const float4*>(mine + h * G::kJoinPitch + at), all.totals[warp][h0 + h]);
                }
            }
            __syncwarp();
            if (!go) return;
            continue;
        }
        __syncthreads();
        const int n = done.s.t1 - done.s.t0;
        const bool in_one = done.end - done.at == n;
        const long long unit_at = done.seq_at + (long long)done.unit * (n + cost) + cost;
        const int first_cta = in_one ? cta : piece_first >= 0 ? piece_first : (int)quotient(unit_at, share);
        const int last_cta = in_one ? cta : piece_first >= 0 ? piece_last : (int)quotient(unit_at + n - 1, share);
        float* const slot = slot_of(p, cta, first_cta);
        if (tid < done_heads) {
            const float total = all.total(tid);
            if (!in_one) {
                *reinterpret_cast<float2*>(slot + 2 * tid) = make_float2(all.top(tid), total);
            } else if (p.lse) {
                p.lse[(size_t)done.seq * p.q_heads + done_head + tid] = all.base(tid) * kLn2 + logf(total);
            }
        }
        for (int h0 = 0; h0 < done_heads; h0 += G::kJoinHeads) {
            if (h0 > 0) __syncthreads();
            w.sums(join + warp * G::kJoinHeads * G::kJoinPitch, &all, h0, lane);
            __syncthreads();
            const int some = min(done_heads - h0, G::kJoinHeads);
            for (int h = my_h; h < some && c < p.dh; h += kRows) {
                float4 sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
                for (int j = 0; j < kWarps; ++j) {
                    const float4 v = *reinterpret_cast<const float4*>(join + (j * G::kJoinHeads + h) * G::kJoinPitch + c);
                    sum.x += v.x; sum.y += v.y; sum.z += v.z; sum.w += v.w;
                }
                if (in_one) write_result<T>(p, done.seq, done_head + h0 + h, c, sum, all.total(h0 + h));
                else *reinterpret_cast<float4*>(slot + 32 + (h0 + h) * p.dh + c) = sum;
            }
        }
        if (!in_one) {
            const Cut cut = {first_cta, last_cta, done.seq, done_head, done_heads};
            if (first_cta == cta) cuts[1] = cut;
            else cuts[0] = cut;
        }
        if (!go) break;
    }

    // ---- heads that several CTAs share, the first and the last of this one's at most: who arrives last adds up, in the order of the CTAs ----
#pragma unroll 1
    for (int level = 0; level < 2; ++level) {
        if (cuts[0].heads + cuts[1].heads == 0) return;
        __syncthreads();                                      // what the CTA's threads have written is before the first warp's fence ...
        if (warp == 0) {
            __threadfence();
            if (lane < 2) {
                const Cut u = lane ? cuts[1] : cuts[0];
                bool mine = false;
                if (u.heads > 0) {
                    const Round r = round_of(u, level, cta);
                    const unsigned others = (r.last - r.first) / r.step;
                    // a round of few is counted at its last CTA: no other head has that one in its midst or as its end
                    mine = atomicInc(p.arrived + (r.ends ? u.first : kMaxCtas + r.last), others) == others;        // (the last one leaves a zero)
                }
                last[lane] = mine;
            }
            __threadfence();                                  // ... and what other CTAs wrote before they arrived is before what follows the barrier
        }
        __syncthreads();
        if (!last[0]) cuts[0].heads = 0;
        if (!last[1]) cuts[1].heads = 0;
#pragma unroll 1
        for (int k = 0; k < 2; ++k) {
            const Cut u = k ? cuts[1] : cuts[0];
            if (u.heads == 0) continue;
            const Round r = round_of(u, level, cta);
            // a row of threads takes a head, or where there are more rows than heads every so-manieth part of one
            const int together = min(u.heads, kRows), groups = kRows / together, group = my_h / together;
            for (int h0 = 0; h0 < u.heads; h0 += together) {
                const int h = h0 + my_h % together;
                const bool works = group < groups && h < u.heads && c < p.dh;
                float top = kNone, total = 0.0f;
                float4 sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                if (works) {
                    constexpr int kBatch = kRound;
                    for (int a = r.first + group * r.step; a <= r.last; a += kBatch * groups * r.step) {
                        float2 t[kBatch];
                        float4 v[kBatch];
#pragma unroll
                        for (int i = 0; i < kBatch; ++i) {
                            const float* from = slot_of(p, min(a + i * groups * r.step, r.last), u.first);
                            t[i] = *reinterpret_cast<const float2*>(from + 2 * h);
                            v[i] = *reinterpret_cast<const float4*>(from + 32 + h * p.dh + c);
                        }
                        float higher = top;
#pragma unroll
                        for (int i = 0; i < kBatch; ++i) {
                            if (a + i * groups * r.step > r.last) t[i] = make_float2(kNone, 0.0f);  // a part again: it weighs nothing (no branch, so that all loads fly at once)
                            higher = fmaxf(higher, t[i].x);
                        }
                        add_part(top, total, sum, higher, top, total, sum, true);
#pragma unroll
                        for (int i = 0; i < kBatch; ++i) add_part(top, total, sum, higher, t[i].x, t[i].y, v[i], false);
                    }
                }
                if (groups > 1) {                             // (uniform)
                    float* const row = join + my_h * G::kJoinPitch;
                    __syncthreads();
                    if (works) {
                        *reinterpret_cast<float4*>(row + c) = sum;
                        if (c == 0) { row[G::kWidth] = top; row[G::kWidth + 1] = total; }
                    }
                    __syncthreads();
                    if (works && group == 0) {
                        float higher = kNone;
                        for (int g = 0; g < groups; ++g) higher = fmaxf(higher, join[(my_h + g * together) * G::kJoinPitch + G::kWidth]);
                        top = kNone;
                        for (int g = 0; g < groups; ++g) {
                            const float* const other = join + (my_h + g * together) * G::kJoinPitch;
                            add_part(top, total, sum, higher, other[G::kWidth], other[G::kWidth + 1], *reinterpret_cast<const float4*>(other + c), g == 0);
                        }
                    }
                }
                if (!r.ends) __syncthreads();                 // (uniform) the slot that the sums go to has been read
                if (works && group == 0) {
                    if (r.ends) {
                        write_result<T>(p, u.seq, u.head + h, c, sum, total);
                        if (p.lse && c == 0) p.lse[(size_t)u.seq * p.q_heads + u.head + h] = (top == kNone ? 0.0f : top * kLn2) + logf(total);
                    } else {
                        float* const to = slot_of(p, r.first, u.first);
                        if (c == 0) *reinterpret_cast<float2*>(to + 2 * h) = make_float2(top, total);
                        *reinterpret_cast<float4*>(to + 32 + h * p.dh + c) = sum;
                    }
                }
            }
            if (r.ends) {
                if (k) cuts[1].heads = 0;
                else cuts[0].heads = 0;
            }
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
    p.units_a_kv = ceil_div(p.group, p.heads_a_unit);
    p.slot = 32 + p.heads_a_unit * p.dh;                      // a multiple of 8
    auto kernel = attend_kernel<T, W, kBytes>;
    // once per device: the attribute stays (asking again costs the host a microsecond)
    static std::atomic<uint64_t> allowed{0};
    const uint64_t bit = ctx->device < 64 ? 1ull << ctx->device : 0;
    if (!(allowed.load(std::memory_order_acquire) & bit)) {
        GELO_CUDA_OK(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, G::kSmem));
        allowed.fetch_or(bit, std::memory_order_release);
    }
    const int ctas = G::kCtas * ctx->sm_count < kMaxCtas ? G::kCtas * ctx->sm_count : kMaxCtas;
    p.a_seq = 1.0f / (float)p.seqs;
    p.a_cta = 1.0f / (float)ctas;
    GELO_TRY(launch_chained(ctx, kernel, dim3(ctas), 32 * G::kWarps, G::kSmem, st, p));
    return after_launch(ctx);
}

// Heads padded to 64, 128 or 256 components; up to eight query heads of a key-value head in one set of columns, up to sixteen in two, more in
// units that read the keys and values again (16 heads in two sets 112 us, in two units of eight 166).
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

template <int H>
int launch_fma(gelo_ctx* ctx, AttendArgs& p, cudaStream_t st)
{
    if (p.dh <= 64) return launch_as<float, FmaWarp<64, H>, 4>(ctx, p, st);
    if (p.dh <= 128) return launch_as<float, FmaWarp<128, H>, 4>(ctx, p, st);
    return launch_as<float, FmaWarp<256, H < 4 ? H : 4>, 4>(ctx, p, st);             // (eight would not leave room for their sums in registers)
}

}  // namespace

size_t attend_workspace_bytes() { return (size_t)2 * kMaxCtas * kSlotFloats * sizeof(float); }
size_t attend_counter_bytes() { return 2 * kMaxCtas * sizeof(unsigned); }

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
    if (p.group == 1) return launch_fma<1>(ctx, p, st);
    if (p.group <= 4) return launch_fma<4>(ctx, p, st);
    return launch_fma<8>(ctx, p, st);
}

}  // namespace gelo
