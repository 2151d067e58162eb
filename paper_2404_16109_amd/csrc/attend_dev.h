// Attention over the cache of 8-bit keys and values: the kernels, of kvcache_attention (Args) and, for the keys behind a prefix that a
// batch shares, of kvcache_attention_prefix (its own Args, with its own page_of, first_seen and tiles_of).
//
// With K, V the codes, 2^a and 2^b their pages' scales: s_j = scale * 2^a_j (q . K_j), o = sum_j e^{s_j} 2^b_j V_j / sum_j e^{s_j}
// over the keys j that a query sees.  One pass over the keys with a running maximum:
//   * in units of log2: t_j = s_j log2(e) + b_j, M = max t_j - 14, P_j = 2^(t_j - M).  The scale of V is an exponent and
//     joins the score's, so the weights of all pages enter ONE accumulator of products with the codes as they are, whatever
//     their scales; the sum of the weights is l = sum_j P_j 2^-b_j, in 32 bits.  For the product P is rounded to 11 bits, a
//     16-bit float, as the matrix cores take it beside codes that are exact there: bf16 outputs lose nothing by it (1.6e-3 of their
//     size, the rounding of the output alone), f16 outputs up to 2.8e-4 where that alone is 2.0e-4.  P is at most
//     2^14: it reaches 29 binades below the largest at full precision and 10 more at less.  Exponents lie in [-40, 40], so
//     a score that matters is never below what a 32-bit P holds.
//   * codes become 16-bit floats by putting the byte (with its top bit flipped) under the exponent of 1024 and taking 1152
//     off: exact, five instructions for four codes.  q is scaled by a power of two to just below 2^15, which a 16-bit float
//     holds exactly but for elements 2^-29 of the row's largest.
//   * both products run on the matrix cores, transposed: S^T = K Q^T and O^T = V^T P^T.  What comes out of the first is the
//     second's operand without a move between lanes: a lane gets the scores of tokens that lie side by side, because
//     the rows of K are handed in that order, and V lies in the cache by dimension.
//
// Few rows (up to 32 of a sequence and head of the cache, the query heads that share it among them): the cache is read once,
// straight into registers, a tile ahead of its use, and is what bounds the call.  A wavefront takes 64 tokens at a time: 16
// loads of 1 KiB, so that the eight wavefronts of a CU have 128 KiB on the way.  k_attend_few: four wavefronts share a
// workgroup's part of a sequence, `splits` workgroups the sequence, or eight wavefronts have all of a short one; k_attend_shared:
// as many workgroups as the chip holds share all sequences; k_attend_join adds up.  Measured: one sequence of 131071
// tokens, 8 heads of 128 (268 MB) 59 us, 4.5 TB/s, where a copy of that size reaches 4.8; one of 777 tokens 10.1 us, four workgroups
// to a head and then the join: latency, of the lengths and pages, the keys, the values, and of the parts in a second launch.
// Many rows (k_attend_many: 128 to a workgroup): codes are widened once and shared through LDS, a tile ahead.  A wavefront's 32
// rows and 64 keys take 466 vector instructions (1860 cycles; exponentials, roundings, scales, masks) and 1020 cycles of the matrix
// cores; at two wavefronts to a SIMD little of one hides behind the other: vector ALU 50% busy, matrix cores 26%, LDS 24%.  Row
// tiles are taken with those that see most first, over all heads: 82 us for a prompt of 2048 tokens and 40 heads (43 GFLOP,
// 523 TFLOP/s; head by head it was 160), 600 TFLOP/s for four such prompts.
#pragma once
#include "attend_pieces.h"
#include "kvcache.h"

namespace zkmi {
namespace {

static const float kLog2e = 1.44269504088896341f, kLn2 = 0.693147180559945309f;
static const float kHead = 14.0f;      // P reaches up to 2^14
static const uint32_t kTile = 64;      // tokens
static const uint32_t kWorkgroups = 512;

struct Args {
    static constexpr bool joined = false;  // whether every row is finished by a later launch
    kvcache_i8 cache;
    kv_seqs s;
    const void* q;
    size_t qrow, qhead;
    void* out;
    size_t orow, ohead;
    float* lse;
    float scale;
    uint32_t window, group, page_log, splits, each;  // group: query heads of a head of the cache
    int dtype;
    bool few;   // which kernel leaves the parts
    bool crowd;  // sequences and heads enough for workgroups of four wavefronts
    uint32_t shared;  // workgroups of k_attend_shared, 0 if it is not used
    bool wide;  // q's rows and heads are 16-byte aligned
    float* parts;  // of (sequence, head, split, row): head_dim sums; after all of them (M, l)
    float2* parts_ml;
    uint32_t rows_most;  // rows of a sequence and head at most
};

__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }

// Eight codes as 16-bit floats.
__device__ __forceinline__ v8h widen(uint32_t lo, uint32_t hi) {
    lo ^= 0x80808080u;
    hi ^= 0x80808080u;
    const uint32_t k = 0x64646464u;  // 0x64uu is 1024 + uu
    const v2h bias = {(_Float16)-1152.0f, (_Float16)-1152.0f};
    union {
        v2h p[4];
        v8h v;
    } r;
    r.p[0] = __builtin_bit_cast(v2h, __builtin_amdgcn_perm(k, lo, 0x04010400u)) + bias;
    r.p[1] = __builtin_bit_cast(v2h, __builtin_amdgcn_perm(k, lo, 0x04030402u)) + bias;
    r.p[2] = __builtin_bit_cast(v2h, __builtin_amdgcn_perm(k, hi, 0x04010400u)) + bias;
    r.p[3] = __builtin_bit_cast(v2h, __builtin_amdgcn_perm(k, hi, 0x04030402u)) + bias;
    return r.v;
}

typedef float v2f __attribute__((ext_vector_type(2)));
__device__ __forceinline__ v2h round2(float a, float b) { return __builtin_convertvector((v2f{a, b}), v2h); }  // one instruction

// Maximum / sum over the lane rows (16 lanes each) 2i, 2i + 1, and over the halves of a wavefront.
__device__ __forceinline__ float max_rows(float x) {
    auto r = __builtin_amdgcn_permlane16_swap(float_bits(x), float_bits(x), false, false);
    return fmaxf(bits_float(r[0]), bits_float(r[1]));
}
__device__ __forceinline__ float max_halves(float x) {
    auto r = __builtin_amdgcn_permlane32_swap(float_bits(x), float_bits(x), false, false);
    return fmaxf(bits_float(r[0]), bits_float(r[1]));
}
__device__ __forceinline__ float add_rows(float x) {
    auto r = __builtin_amdgcn_permlane16_swap(float_bits(x), float_bits(x), false, false);
    return bits_float(r[0]) + bits_float(r[1]);
}
__device__ __forceinline__ float add_halves(float x) {
    auto r = __builtin_amdgcn_permlane32_swap(float_bits(x), float_bits(x), false, false);
    return bits_float(r[0]) + bits_float(r[1]);
}

// N consecutive elements of q (16 bits each, N a multiple of 8), as they lie in memory: one wide load for eight where the
// caller's addresses allow it.
template <int N>
__device__ __forceinline__ void load_raw(const void* p, size_t at, bool wide, v4u (&r)[N / 8]) {
    const uint16_t* x = (const uint16_t*)p + at;
    if (wide) {
#pragma unroll
        for (int i = 0; i < N / 8; ++i) r[i] = ((const v4u*)x)[i];
    } else {
#pragma unroll
        for (int i = 0; i < N / 8; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) r[i][e] = (uint32_t)x[8 * i + 2 * e] | ((uint32_t)x[8 * i + 2 * e + 1] << 16);
    }
}

// A row of q, spread over lanes that hold N elements each: scaled to just below 2^15 by a power of two, as 16-bit floats.
// Returns the factor that takes the power back and brings the units of log2; NaN for a row that is not finite.
struct LargestOf2 {
    __device__ __forceinline__ float operator()(float x) const { return max_halves(x); }
};
struct LargestOf4 {
    __device__ __forceinline__ float operator()(float x) const { return max_halves(max_rows(x)); }
};
template <int N, typename Largest>
__device__ __forceinline__ float scale_row(const v4u (&raw)[N / 8], int dtype, float scale, v8h (&out)[N / 8], Largest largest) {
    float x[N], amax = 0.0f;
    if (dtype == ZK_BF16) {
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = half_of<ZK_BF16>(raw[i >> 3][(i & 7) >> 1], i & 1);
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = half_of<ZK_F16>(raw[i >> 3][(i & 7) >> 1], i & 1);
    }
    uint32_t most = 0;  // the bits of |x|: infinities and NaN are above every number
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const uint32_t bits = float_bits(x[i]) & 0x7fffffffu;
        most = bits > most ? bits : most;
    }
    amax = largest(most >= 0x7f800000u ? kInf : bits_float(most));
    const bool fine = amax < kInf;
    int ex = 0;
    if (fine && amax != 0.0f) (void)frexpf(amax, &ex);
#pragma unroll
    for (int i = 0; i < N; ++i) out[i >> 3][i & 7] = fine ? (_Float16)ldexpf(x[i], 15 - ex) : (_Float16)0.0f;
    return fine ? ldexpf(scale * kLog2e, ex - 15) : __builtin_nanf("");
}

__device__ __forceinline__ void put_at(void* p, size_t i, float f, int dtype) {
    const uint16_t b = half_bits<ZK_BF16>(f), h = half_bits<ZK_F16>(f);
    ((uint16_t*)p)[i] = dtype == ZK_BF16 ? b : h;
}

// Where row r of a sequence and head lies in q (or out).
__device__ __forceinline__ size_t row_at(const Args& a, const SeqView& v, uint32_t h, uint32_t r, size_t row, size_t head) {
    const uint32_t token = r / a.group;
    return (size_t)(v.row0 + (int32_t)token) * row + (size_t)(h * a.group + (r - token * a.group)) * head;
}

// The outputs of a sequence that is skipped: NaN, where they lie inside the call's tensors.
__device__ void not_a_number(const Args& a, uint32_t b, uint32_t h) {
    const int64_t from = a.s.cu[b] > 0 ? a.s.cu[b] : 0, end = a.s.cu[b + 1], to = end < (int64_t)a.s.rows ? end : a.s.rows;
    const uint32_t d = a.cache.head_dim;
    if (threadIdx.x == 0) report(a.s, ZK_FAULT_LENGTH);
    for (int64_t row = from; row < to; ++row)
        for (uint32_t i = threadIdx.x; i < a.group * d; i += blockDim.x) {
            const uint32_t head = h * a.group + i / d;
            put_at(a.out, (size_t)row * a.orow + (size_t)head * a.ohead + i % d, __builtin_nanf(""), a.dtype);
            if (a.lse && i % d == 0) a.lse[(size_t)row * (a.cache.kv_heads * a.group) + head] = __builtin_nanf("");
        }
}

// The first key that row i of a sequence sees, or any of the later rows.
__device__ __forceinline__ uint32_t first_seen(const Args& a, const SeqView& v, int32_t i) {
    const int64_t low = a.window ? (int64_t)v.len - v.rows + i - (int64_t)a.window + 1 : 0;
    return low > 0 ? (uint32_t)low : 0;
}

// Where the sums of a sequence and head over a part of its keys lie: those of its first row, the others behind.
__device__ __forceinline__ size_t own_part(const Args& a, const SeqView&, uint32_t b, uint32_t h, uint32_t split) {
    return (((size_t)b * a.cache.kv_heads + h) * a.splits + split) * a.rows_most;
}

// The tile that a sequence's keys begin with, before its lengths are known.
__device__ __forceinline__ uint32_t first_guess(const Args&) { return 0; }

// Tiles [first, end) of the keys that rows [i0, i1] of a sequence see.
struct Tiles {
    uint32_t first, end;
};
__device__ __forceinline__ Tiles tiles_of(const Args& a, const SeqView& v, int32_t i0, int32_t i1) {
    const int64_t last = (int64_t)v.len - v.rows + i1;
    Tiles t;
    t.first = first_seen(a, v, i0) / kTile;
    t.end = last < 0 ? t.first : (uint32_t)(last / kTile) + 1;
    return t;
}

// The same for the 128 rows from r0 on that a workgroup of k_attend_many has.
static const uint32_t kRows = 128;
template <typename A>
__device__ __forceinline__ Tiles tiles_of_rows(const A& a, const SeqView& v, uint32_t r0, uint32_t rows = kRows) {
    const uint32_t R = (uint32_t)v.rows * a.group, last = r0 + rows < R ? r0 + rows - 1 : R - 1;
    return tiles_of(a, v, (int32_t)(r0 / a.group), (int32_t)(last / a.group));
}

// Tiles of a workgroup's part.  The same for all sequences of a call, so that workgroups have like work and short sequences
// fewer of them; more only where a sequence is longer than the caller said.
__device__ __forceinline__ uint32_t part_of(const Args& a, const Tiles& t) {
    const uint32_t need = (t.end - t.first + a.splits - 1) / a.splits;
    return need > a.each ? need : a.each;
}

// The page of a token, as the table has it: what it is worth is looked at when it is used, not while it is on its way.
// Tokens behind the sequence have what the table holds there, or its last entry.
__device__ __forceinline__ uint32_t page_of(const Args& a, uint32_t b, uint32_t token) {
    const uint32_t at = token >> a.page_log, last = a.s.table_pages - 1;
    return (uint32_t)a.s.table[(size_t)b * a.s.table_stride + (at < last ? at : last)];
}
__device__ __forceinline__ uint32_t page_or_0(const Args& a, uint32_t page) { return page < a.cache.pages ? page : 0; }

__device__ __forceinline__ float exponent_value(int e) { return e == ZK_EXP_NAN ? __builtin_nanf("") : (float)e; }

// 2^-b. Of a poisoned page 0: the weights of the keys that a row sees there are NaN by themselves, those of the others 0.
__device__ __forceinline__ float back_of(float b) { return b == b ? exp2_of(-b) : 0.0f; }

// What a row ends with.
__device__ __forceinline__ float lse_of(float m, float l) { return l == 0.0f ? -kInf : (m + __log2f(l)) * kLn2; }

// ---- few rows --------------------------------------------------------------------------------------------------------

// NJ: head_dim in units of 64, rounded up.  RT: tiles of 16 rows.  W: wavefronts.  Lane 16 g + i: row i of a tile, tokens
// 16 g .. 16 g + 15.
template <int NJ, int RT, int W>
struct FewLds {
    static constexpr int row = 64 * NJ + 4;  // of sums, padded
    static size_t bytes(uint32_t rows) { return (2 * (size_t)W * 16 * RT + (size_t)W * rows * row) * sizeof(float); }
};

// The pages of a wavefront's first and second tile, once asked for.
struct Asked {
    uint32_t k, v, k_next, v_next;
};
template <typename A>
__device__ __forceinline__ Asked ask_pages(const A& a, uint32_t b, uint32_t t, uint32_t step) {
    const uint32_t lane = threadIdx.x & 63, k = 16 * ((lane & 15) >> 2), v = 16 * (lane >> 4);
    return Asked{page_of(a, b, t * kTile + k), page_of(a, b, t * kTile + v), page_of(a, b, (t + step) * kTile + k),
                 page_of(a, b, (t + step) * kTile + v)};
}

// Tiles [t_first, t_end) of a sequence and head; `pages` are those of tile t_first + wavefront and the next.  What comes out are
// the rows' outputs if that is all they see, else sums from row part0 of the workspace on.
template <int NJ, int RT, int W, typename A>
__device__ __forceinline__ void attend_part(const A& a, float* sh, const SeqView& v, uint32_t b, uint32_t h, uint32_t t_first, uint32_t t_end,
                                            const Asked& pages, bool whole_row, size_t part0) {
    constexpr int DT = 4 * NJ;  // tiles of 16 dimensions
    const uint32_t tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), g = lane >> 4, i16 = lane & 15, rk = i16 >> 2;
    const uint32_t d = a.cache.head_dim, T = 1u << a.page_log, H = a.cache.kv_heads, R = (uint32_t)v.rows * a.group;
    uint32_t pk_next = pages.k_next, pv_next = pages.v_next;

    v4u raw[RT][2 * NJ];  // q as it lies in memory; asked for first, since loads come back in order
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        const uint32_t r = rt * 16 + i16;
        const size_t at = row_at(a, v, h, r < R ? r : 0, a.qrow, a.qhead);  // rows behind the last: a copy of the first
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
            v4u two[2] = {v4u{0, 0, 0, 0}, v4u{0, 0, 0, 0}};
            if (64 * j + 16 * g < d) load_raw<16>(a.q, at + 64 * j + 16 * g, a.wide, two);
            raw[rt][2 * j] = two[0];
            raw[rt][2 * j + 1] = two[1];
        }
    }

    // Every load is made: tokens behind the sequence read some page, pages that are none page 0, dimensions behind head_dim
    // the row's first (q is 0 there).  All are numbers, and nothing of them is kept.
    const uint32_t len = (uint32_t)v.len, seen_from = first_seen(a, v, 0);  // a tile may begin before what any row sees
    const size_t page_stride = (size_t)T * d;
    v4u kr[4][NJ], vr[DT];
    auto load_k = [&](uint32_t page, uint32_t t) {
        const uint32_t slot = (t * kTile + 16 * rk) & (T - 1);
        const int8_t* at = a.cache.k + ((size_t)page_or_0(a, page) * H + h) * page_stride + (slot + (i16 & 3)) * d;
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
            const uint32_t c = 64 * j + 16 * g < d ? 64 * j + 16 * g : 0;
#pragma unroll
            for (int u = 0; u < 4; ++u) kr[u][j] = *(const v4u*)(at + 4 * u * d + c);
        }
    };
    auto load_v = [&](uint32_t page, uint32_t t) {
        const uint32_t slot = (t * kTile + 16 * g) & (T - 1);
        const int8_t* at = a.cache.v + ((size_t)page_or_0(a, page) * H + h) * page_stride + (i16 << a.page_log) + slot;
#pragma unroll
        for (int c = 0; c < DT; ++c) vr[c] = *(const v4u*)(at + ((16u * c < d ? 16u * c : 0) << a.page_log));
    };
    int ke = 0, ve = 0;  // exponents of the lane's 16 tokens
    bool none = false;   // whether their page is none
    auto load_e = [&](uint32_t page) {
        const size_t at = (size_t)page_or_0(a, page) * H + h;
        ke = a.cache.k_exp[at];
        ve = a.cache.v_exp[at];
        none = page >= a.cache.pages;
    };

    v4f o[RT][DT];
    float m[RT], l[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        m[rt] = -kInf;
        l[rt] = 0.0f;
#pragma unroll
        for (int c = 0; c < DT; ++c) o[rt][c] = v4f{0, 0, 0, 0};
    }

    uint32_t t = t_first + wave;
    if (t < t_end) {
        load_k(pages.k, t);
        load_e(pages.v);
        load_v(pages.v, t);
    }
    // q, scaled by a power of two; qmul takes that back and brings the units of log2
    v8h qf[RT][2 * NJ];
    float qmul[RT];
    int32_t pos[RT];  // the last key that the lane's row sees
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        const uint32_t r = rt * 16 + i16;
        qmul[rt] = scale_row<16 * NJ>(raw[rt], a.dtype, a.scale, qf[rt], LargestOf4());
        pos[rt] = r < R ? v.len - v.rows + (int32_t)(r / a.group) : -1;
    }

    for (; t < t_end; t += W) {
        const bool more = t + W < t_end;
        const uint32_t pk_after = page_of(a, b, (t + 2 * W) * kTile + 16 * rk), pv_after = page_of(a, b, (t + 2 * W) * kTile + 16 * g);
        v4f s[RT][4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) s[rt][u] = v4f{0, 0, 0, 0};
#pragma unroll
            for (int j = 0; j < NJ; ++j) {
                const v8h a0 = widen(kr[u][j][0], kr[u][j][1]), a1 = widen(kr[u][j][2], kr[u][j][3]);
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) {
                    s[rt][u] = __builtin_amdgcn_mfma_f32_16x16x32_f16(a0, qf[rt][2 * j], s[rt][u], 0, 0, 0);
                    s[rt][u] = __builtin_amdgcn_mfma_f32_16x16x32_f16(a1, qf[rt][2 * j + 1], s[rt][u], 0, 0, 0);
                }
            }
        }
        if (more) load_k(pk_next, t + W);
        // a page that is none has a score that is none
        const float kscale = none ? __builtin_nanf("") : exp2_of(exponent_value(ke)), vadd = none ? 0.0f : exponent_value(ve), vback = back_of(vadd);
        if (none && t * kTile + 16 * g < len && t * kTile + 16 * g + 16 > seen_from) report(a.s, ZK_FAULT_PAGE);
        if (more) load_e(pv_next);

        const int32_t base = (int32_t)(t * kTile);
        // whether every row sees all 64 tokens
        const bool whole = base + (int32_t)kTile - 1 <= v.len - v.rows && base > (a.window ? v.len - 1 - (int32_t)a.window : -1);
        v8h p[RT][2];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            const float mul = qmul[rt] * kscale;
#pragma unroll
            for (int u = 0; u < 4; ++u) s[rt][u] = s[rt][u] * mul + vadd;
            if (!whole) {
                const int32_t key0 = base + 16 * (int32_t)g, low = a.window ? pos[rt] - (int32_t)a.window : -1;
#pragma unroll
                for (int u = 0; u < 4; ++u)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int32_t key = key0 + 4 * u + e;
                        if (key > pos[rt] || key <= low) s[rt][u][e] = -kInf;
                    }
            }
            float top = -kInf;
#pragma unroll
            for (int u = 0; u < 4; ++u)
#pragma unroll
                for (int e = 0; e < 4; ++e) top = fmaxf(top, s[rt][u][e]);
            top = max_halves(max_rows(top)) - kHead;
            if (__ballot(top > m[rt])) {
                const float now = fmaxf(m[rt], top), f = exp2_of(now == -kInf ? 0.0f : m[rt] - now);
                m[rt] = now;
                l[rt] *= f;
#pragma unroll
                for (int c = 0; c < DT; ++c) o[rt][c] *= f;
            }
            const float from = m[rt] == -kInf ? 0.0f : m[rt];
            float sum = 0.0f;
#pragma unroll
            for (int u = 0; u < 4; ++u)
#pragma unroll
                for (int e = 0; e < 4; e += 2) {
                    const float x0 = exp2_of(s[rt][u][e] - from), x1 = exp2_of(s[rt][u][e + 1] - from);
                    sum += x0 + x1;
                    const v2h two = round2(x0, x1);
                    p[rt][u >> 1][(u & 1) * 4 + e] = two[0];
                    p[rt][u >> 1][(u & 1) * 4 + e + 1] = two[1];
                }
            l[rt] += sum * vback;
        }
#pragma unroll
        for (int c = 0; c < DT; ++c) {
            const v8h a0 = widen(vr[c][0], vr[c][1]), a1 = widen(vr[c][2], vr[c][3]);
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                o[rt][c] = __builtin_amdgcn_mfma_f32_16x16x32_f16(a0, p[rt][0], o[rt][c], 0, 0, 0);
                o[rt][c] = __builtin_amdgcn_mfma_f32_16x16x32_f16(a1, p[rt][1], o[rt][c], 0, 0, 0);
            }
        }
        if (more) load_v(pv_next, t + W);
        pk_next = pk_after;
        pv_next = pv_after;
    }

    // The wavefronts' sums meet in LDS, each relative to its own maximum.
    constexpr uint32_t D = FewLds<NJ, RT, W>::row;
    float* ms = sh;  // [wave][16 RT]
    float* ls = ms + W * 16 * RT;
    float* sums = ls + W * 16 * RT;  // [wave][R][D]
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        const uint32_t r = rt * 16 + i16;
        l[rt] = add_halves(add_rows(l[rt]));
        if (g == 0) {
            ms[wave * 16 * RT + r] = m[rt];
            ls[wave * 16 * RT + r] = l[rt];
        }
        if (r < R)
#pragma unroll
            for (int c = 0; c < DT; ++c) *(v4f*)(sums + (size_t)(wave * R + r) * D + 16 * c + 4 * g) = o[rt][c];
    }
    __syncthreads();
    const uint32_t quads = d >> 2;
    for (uint32_t i = tid; i < R * quads; i += 64 * W) {
        const uint32_t r = i / quads, c = (i - r * quads) * 4;
        float mw[W], all = -kInf, l_all = 0.0f;
#pragma unroll
        for (int w = 0; w < W; ++w) {
            mw[w] = ms[w * 16 * RT + r];
            all = fmaxf(all, mw[w]);
        }
        const float ref = all == -kInf ? 0.0f : all;
        v4f sum = {0, 0, 0, 0};
#pragma unroll
        for (int w = 0; w < W; ++w) {
            const float f = exp2_of(mw[w] - ref);
            l_all += ls[w * 16 * RT + r] * f;
            sum += *(const v4f*)(sums + (size_t)(w * R + r) * D + c) * f;
        }
        if (whole_row) {
            const size_t at = row_at(a, v, h, r, a.orow, a.ohead) + c;
            const float inv = l_all == 0.0f ? 0.0f : 1.0f / l_all;
#pragma unroll
            for (int e = 0; e < 4; ++e) put_at(a.out, at + e, l_all == 0.0f ? 0.0f : sum[e] * inv, a.dtype);
            if (a.lse && c == 0) a.lse[row_at(a, v, h, r, (size_t)H * a.group, 1)] = lse_of(ref, l_all);
        } else {
            const size_t part = part0 + r;
            *(v4f*)(a.parts + part * d + c) = sum;
            if (c == 0) a.parts_ml[part] = make_float2(all, l_all);
        }
    }
}

// A workgroup's part of a sequence and head.
template <int NJ, int RT, int W, typename A>
__device__ __forceinline__ void attend_few(const A& a, float* sh, uint32_t split, uint32_t h, uint32_t b) {
    const uint32_t wave = uniform(threadIdx.x >> 6);
    // The part begins where the caller's lengths put it, but for windows: its pages are asked for beside the lengths.
    const uint32_t guess = first_guess(a) + split * a.each + wave;
    Asked pages = ask_pages(a, b, guess, W);
    const SeqView v = seq_view(a.s, b, a.page_log);
    if (!v.ok) {
        if (a.splits == 1 && !A::joined) not_a_number(a, b, h);
        return;
    }
    if (v.rows == 0) return;
    const Tiles tiles = tiles_of(a, v, 0, v.rows - 1);
    const uint32_t each = part_of(a, tiles);
    const uint32_t t_first = tiles.first + split * each, t_end = t_first + each < tiles.end ? t_first + each : tiles.end;
    if (a.splits > 1 && t_first >= t_end) return;  // k_attend_join knows
    if (t_first + wave != guess) pages = ask_pages(a, b, t_first + wave, W);
    attend_part<NJ, RT, W>(a, sh, v, b, h, t_first, t_end, pages, a.splits == 1 && !A::joined, own_part(a, v, b, h, split));
}
template <int NJ, int RT, int W>
__global__ __launch_bounds__(64 * W, W == 4 && NJ * RT <= 2 ? 2 : 1) void k_attend_few(Args a) {
    extern __shared__ __attribute__((aligned(16))) float sh[];
    attend_few<NJ, RT, W>(a, sh, blockIdx.x, blockIdx.y, blockIdx.z);
}

// ---- many rows -------------------------------------------------------------------------------------------------------

// Lane 32 h + i: row i of its wavefront's 32, tokens 16 h .. 16 h + 15 of each half of a tile.
// DT: head_dim in units of 32, rounded up.  Rows in LDS are padded by 16 bytes: then those of 16 neighbouring rows lie in
// different banks, whatever DT.
template <int DT>
struct ManyLds {
    static constexpr uint32_t krow = 64 * DT + 16, vrow = 128 + 16, k_bytes = 64 * krow, bytes = k_bytes + 32 * DT * vrow;
};
struct ManyShared {
    float exps[2][2][4];    // [buffer][K, V][16 tokens]
    uint32_t pages[2][4];   // of the next tile
};
// Rows from r0 on, 32 to each of WV wavefronts, of the R of a sequence and head over tiles [first, end); the lane's row sees keys (low, pos], every row of the
// wavefront those up to pos_first, some row of the workgroup pos_last, none those before seen_from.  What comes out are outputs, or
// sums, r's at part0 + r.
// RAW: where all keys of a tile are seen, scores stay products until their exponential is taken, which is one step less for each and rounds
// elsewhere.
template <int DT, bool RAW, int WV, typename A>
__device__ __forceinline__ void attend_rows(const A& a, char* lds, ManyShared& sh, const SeqView& v, uint32_t b, uint32_t h, uint32_t R, uint32_t r0,
                                            const Tiles& tiles, int32_t pos, int32_t pos_first, int32_t pos_last, uint32_t seen_from, bool parts,
                                            size_t part0, float* sums, float2* sums_ml) {
    using L = ManyLds<DT>;
    constexpr uint32_t threads = 64 * WV;
    constexpr int PIECES = (128 * DT + threads - 1) / threads;  // of 16 codes, for a thread, of a tile's K and of its V
    float(&exps)[2][2][4] = sh.exps;
    uint32_t(&pages)[2][4] = sh.pages;
    const uint32_t tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, half = lane >> 5, i32 = lane & 31;
    const uint32_t d = a.cache.head_dim, T = 1u << a.page_log, H = a.cache.kv_heads, r = r0 + wave * 32 + i32;

    // The first tile's pages, then q, then the tile: loads come back in order.
    uint32_t page[4], my_page = 0;  // later tiles' pages are looked up two tiles ahead
    const bool any = tiles.first < tiles.end;
    if (any) {
#pragma unroll
        for (int i = 0; i < 4; ++i) page[i] = page_of(a, b, tiles.first * kTile + 16 * i);
        my_page = page_of(a, b, (tiles.first + 1) * kTile + 16 * (tid & 3));
    }
    v4u raw[2 * DT];
    {
        const size_t at = row_at(a, v, h, r < R ? r : 0, a.qrow, a.qhead);
#pragma unroll
        for (int k = 0; k < 2 * DT; ++k) {
            v4u one[1] = {v4u{0, 0, 0, 0}};
            if (16u * k < d) load_raw<8>(a.q, at + 16 * k + 8 * half, a.wide, one);
            raw[k] = one[0];
        }
    }
    const int32_t low = a.window ? pos - (int32_t)a.window : -1;  // keys in (low, pos] are seen

    // What a thread brings of a tile: of K, pieces of 16 dimensions of a token; of V, of 16 tokens of a dimension.  As in
    // k_attend_few every load is made; what lies outside is not kept.
    uint32_t k_run[PIECES], k_at[PIECES], v_run[PIECES], v_at[PIECES];
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
        const AttendPiece p = attend_piece<DT>(tid, threads, i);
        k_run[i] = p.slot >> 4;
        k_at[i] = (p.slot & 15) * d + (16 * p.c < d ? 16 * p.c : 0);
        v_run[i] = p.run;
        v_at[i] = (p.dim < d ? p.dim : 0) << a.page_log;
    }
    v4u kr[PIECES], vr[PIECES];
    // K's and V's exponents of the tile's runs of 16 tokens, as they are loaded: a float made of one at once would wait for all of
    // the tile.
    int my_exp = 0;
    bool my_none = false, missing = false;  // whether a page is none, and whether such a one was needed
    auto fetch = [&](uint32_t t, const uint32_t(&page)[4]) {
        const uint32_t head = T * d;
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            const uint32_t kp = page_or_0(a, page[k_run[i]]), vp = page_or_0(a, page[v_run[i]]);
            const uint32_t k_slot = (t * kTile + 16 * k_run[i]) & (T - 1), v_slot = (t * kTile + 16 * v_run[i]) & (T - 1);
            kr[i] = *(const v4u*)(a.cache.k + ((size_t)kp * H + h) * head + k_slot * d + k_at[i]);
            vr[i] = *(const v4u*)(a.cache.v + ((size_t)vp * H + h) * head + v_at[i] + v_slot);
        }
        // all threads, like eight of them: a branch here would part the products before it from those behind
        const uint32_t it = page[tid & 3], key = t * kTile + 16 * (tid & 3);
        my_none = it >= a.cache.pages;
        missing |= my_none && t < tiles.end && (int32_t)key <= pos_last && key + 16 > seen_from;
        my_exp = (tid & 4 ? a.cache.v_exp : a.cache.k_exp)[(size_t)page_or_0(a, it) * H + h];
    };
    auto stage = [&](uint32_t buf) {
        char* kb = lds + buf * L::bytes;
        char* vb = kb + L::k_bytes;
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            if (128 * DT % threads != 0 && !attend_piece_kept<DT>(tid, threads, i)) continue;
            const AttendPiece p = attend_piece<DT>(tid, threads, i);
            const uint32_t x = p.slot & 31;
            // the product's rows 8 b + 4 h + j come out in lane half h, as tokens 16 h + 4 b + j
            const uint32_t row = (p.slot & 32) + 8 * ((x >> 2) & 3) + 4 * (x >> 4) + (x & 3);
            v8h* k16 = (v8h*)(kb + row * L::krow + p.c * 32);
            k16[0] = widen(kr[i][0], kr[i][1]);
            k16[1] = widen(kr[i][2], kr[i][3]);
            v8h* v16 = (v8h*)(vb + p.dim * L::vrow + p.run * 32);
            v16[0] = widen(vr[i][0], vr[i][1]);
            v16[1] = widen(vr[i][2], vr[i][3]);
        }
        if (tid < 8) exps[buf][tid >> 2][tid & 3] = my_none ? (tid < 4 ? __builtin_nanf("") : 0.0f) : exponent_value(my_exp);
    };

    const bool idle = r0 + uniform(wave) * 32 >= R;
    v16f o[DT];
#pragma unroll
    for (int c = 0; c < DT; ++c) o[c] = v16f{0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0};
    float m = -kInf, l = 0.0f;
    if (any) fetch(tiles.first, page);
    v8h qf[2 * DT];
    const float qmul = scale_row<16 * DT>(raw, a.dtype, a.scale, qf, LargestOf2());
    for (uint32_t t = tiles.first; t < tiles.end; ++t) {
        const uint32_t buf = (t - tiles.first) & 1;
        stage(buf);
        if (tid < 4) pages[buf][tid] = my_page;
        __syncthreads();
        if (WV > 4 && idle) {  // no rows: it brings its share of the next tile
            my_page = page_of(a, b, (t + 2) * kTile + 16 * (tid & 3));
            fetch(t + 1, pages[buf]);
            continue;
        }
        if (!RAW && t + 1 < tiles.end) {
            my_page = page_of(a, b, (t + 2) * kTile + 16 * (tid & 3));
            fetch(t + 1, pages[buf]);
        }
        const char* kb = lds + buf * L::bytes;
        const char* vb = kb + L::k_bytes;
        const int32_t base = (int32_t)(t * kTile);
        v16f s[2];
        float vback[2], by[2], plus[2];
        float top = -kInf;
        const bool whole = (!RAW || a.scale > 0.0f) && base + (int32_t)kTile - 1 <= pos_first && base > (a.window ? pos_last - (int32_t)a.window : -1);
#pragma unroll
        for (int st = 0; st < 2; ++st) {
            s[st] = v16f{0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0};
            const char* krow = kb + (st * 32 + i32) * L::krow + half * 16;
#pragma unroll
            for (int k = 0; k < 2 * DT; ++k)
                s[st] = __builtin_amdgcn_mfma_f32_32x32x16_f16(*(const v8h*)(krow + 32 * k), qf[k], s[st], 0, 0, 0);
            if (RAW && st == 0) {
                // The next tile is asked for among the products of this one; behind the last one some page is read, and not kept.
                // (431 -> 417 us for 2450 rows behind 32768 tokens; short row tiles lose by it, 82 -> 88 us for a prompt of 2048.)
                my_page = page_of(a, b, (t + 2) * kTile + 16 * (tid & 3));
                fetch(t + 1, pages[buf]);
            }
            const float ke = exps[buf][0][2 * st + half], ve = exps[buf][1][2 * st + half];
            const float mul = qmul * exp2_of(ke);
            vback[st] = back_of(ve);
            by[st] = mul;  // a score is s * by + plus
            plus[st] = ve;
            if (!RAW || !whole) {
                s[st] = s[st] * mul + ve;
                by[st] = 1.0f;
                plus[st] = 0.0f;
            }
            if (!whole) {
                const int32_t key0 = base + 32 * st + 16 * (int32_t)half;
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    if (key0 + e > pos || key0 + e <= low) s[st][e] = -kInf;
            }
            float most = -kInf;
#pragma unroll
            for (int e = 0; e < 16; ++e) most = fmaxf(most, s[st][e]);
            top = fmaxf(top, RAW ? __builtin_fmaf(most, by[st], plus[st]) : most);
        }
        top = max_halves(top) - kHead;
        if (__ballot(top > m)) {
            const float now = fmaxf(m, top), f = exp2_of(now == -kInf ? 0.0f : m - now);
            m = now;
            l *= f;
#pragma unroll
            for (int c = 0; c < DT; ++c) o[c] *= f;
        }
        const float from = m == -kInf ? 0.0f : m;
        v8h p[2][2];
#pragma unroll
        for (int st = 0; st < 2; ++st) {
            float sum = 0.0f;
            const float less = plus[st] - from;
#pragma unroll
            for (int e = 0; e < 16; e += 2) {
                const float x0 = exp2_of(RAW ? __builtin_fmaf(s[st][e], by[st], less) : s[st][e] - from);
                const float x1 = exp2_of(RAW ? __builtin_fmaf(s[st][e + 1], by[st], less) : s[st][e + 1] - from);
                sum += x0 + x1;
                const v2h two = round2(x0, x1);
                p[st][e >> 3][e & 7] = two[0];
                p[st][e >> 3][(e & 7) + 1] = two[1];
            }
            l += sum * vback[st];
        }
#pragma unroll
        for (int c = 0; c < DT; ++c) {
            const char* vrow = vb + (32 * c + i32) * L::vrow + half * 32;
#pragma unroll
            for (int st = 0; st < 2; ++st)
#pragma unroll
                for (int k = 0; k < 2; ++k)
                    o[c] = __builtin_amdgcn_mfma_f32_32x32x16_f16(*(const v8h*)(vrow + 64 * st + 16 * k), p[st][k], o[c], 0, 0, 0);
        }
    }
    if (missing) report(a.s, ZK_FAULT_PAGE);
    l = add_halves(l);
    if (r >= R) return;
    if (parts) {
        const size_t part = part0 + r;
#pragma unroll
        for (int c = 0; c < DT; ++c)
#pragma unroll
            for (int e = 0; e < 16; e += 4) {
                const uint32_t dim = 32 * c + 2 * e + 4 * half;
                if (dim < d) *(v4f*)(sums + part * d + dim) = v4f{o[c][e], o[c][e + 1], o[c][e + 2], o[c][e + 3]};
            }
        if (half == 0) sums_ml[part] = make_float2(m, l);
        return;
    }
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    const size_t at = row_at(a, v, h, r, a.orow, a.ohead);
#pragma unroll
    for (int c = 0; c < DT; ++c)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const uint32_t dim = 32 * c + 8 * (e >> 2) + 4 * half + (e & 3);
            if (dim < d) put_at(a.out, at + dim, l == 0.0f ? 0.0f : o[c][e] * inv, a.dtype);
        }
    if (a.lse && half == 0) a.lse[row_at(a, v, h, r, (size_t)H * a.group, 1)] = lse_of(m == -kInf ? 0.0f : m, l);
}

// A workgroup's rows of a sequence and head, `tile` times as many before its last.
template <int DT, int WV, typename A>
__device__ __forceinline__ void attend_many(const A& a, char* lds, ManyShared& sh, uint32_t tile, uint32_t split, uint32_t h, uint32_t b) {
    constexpr uint32_t rows = 32 * WV;
    const SeqView v = seq_view(a.s, b, a.page_log);
    if (!v.ok) {
        if (tile == 0 && a.splits == 1 && !A::joined) not_a_number(a, b, h);
        return;
    }
    const uint32_t R = (uint32_t)v.rows * a.group, row_tiles = (R + rows - 1) / rows;
    if (tile >= row_tiles) return;
    const uint32_t r0 = (row_tiles - 1 - tile) * rows;  // the rows that see most first, of all heads
    const uint32_t r_last = r0 + rows - 1 < R - 1 ? r0 + rows - 1 : R - 1;
    const int32_t tok0 = (int32_t)(r0 / a.group), tok1 = (int32_t)(r_last / a.group);
    Tiles tiles = tiles_of_rows(a, v, r0, rows);
    if (a.splits > 1) {
        const uint32_t each = part_of(a, tiles);
        tiles.first += split * each;
        if (tiles.first >= tiles.end) return;  // k_attend_join knows
        tiles.end = tiles.first + each < tiles.end ? tiles.first + each : tiles.end;
    }
    const uint32_t r = r0 + (threadIdx.x >> 6) * 32 + (threadIdx.x & 31);
    const int32_t pos = r < R ? v.len - v.rows + (int32_t)(r / a.group) : -1;
    attend_rows<DT, false, WV>(a, lds, sh, v, b, h, R, r0, tiles, pos, v.len - v.rows + tok0, v.len - v.rows + tok1, first_seen(a, v, tok0), a.splits > 1 || A::joined,
                    own_part(a, v, b, h, split), a.parts, a.parts_ml);
}
template <int DT>
__global__ __launch_bounds__(kBlock, DT <= 4 ? 2 : 1) void k_attend_many(Args a) {
    extern __shared__ __attribute__((aligned(16))) char lds[];
    __shared__ ManyShared sh;
    const uint32_t b = blockIdx.z / a.splits;
    attend_many<DT, 4>(a, lds, sh, blockIdx.y, blockIdx.z - b * a.splits, blockIdx.x, b);
}

}  // namespace
}  // namespace zkmi
