// Attention over the cache of 8-bit keys and values.
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
#include "attend_pieces.h"
#include "kvcache.h"

namespace zkmi {
namespace {

static const float kLog2e = 1.44269504088896341f, kLn2 = 0.693147180559945309f;
static const float kHead = 14.0f;      // P reaches up to 2^14
static const uint32_t kTile = 64;      // tokens
static const uint32_t kWorkgroups = 512;

struct Args {
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

__device__ __forceinline__ v2h round2(float a, float b) { return v2h{(_Float16)a, (_Float16)b}; }

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
__device__ __forceinline__ Tiles tiles_of_rows(const Args& a, const SeqView& v, uint32_t r0) {
    const uint32_t R = (uint32_t)v.rows * a.group, last = r0 + kRows < R ? r0 + kRows - 1 : R - 1;
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
__device__ __forceinline__ Asked ask_pages(const Args& a, uint32_t b, uint32_t t, uint32_t step) {
    const uint32_t lane = threadIdx.x & 63, k = 16 * ((lane & 15) >> 2), v = 16 * (lane >> 4);
    return Asked{page_of(a, b, t * kTile + k), page_of(a, b, t * kTile + v), page_of(a, b, (t + step) * kTile + k),
                 page_of(a, b, (t + step) * kTile + v)};
}

// Tiles [t_first, t_end) of a sequence and head; `pages` are those of tile t_first + wavefront and the next.  What comes out are
// the rows' outputs if that is all they see, else sums from row part0 of the workspace on.
template <int NJ, int RT, int W>
__device__ __forceinline__ void attend_part(const Args& a, float* sh, const SeqView& v, uint32_t b, uint32_t h, uint32_t t_first, uint32_t t_end,
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

template <int NJ, int RT, int W>
__global__ __launch_bounds__(64 * W, W == 4 && NJ * RT <= 2 ? 2 : 1) void k_attend_few(Args a) {
    extern __shared__ float sh[];
    const uint32_t split = blockIdx.x, h = blockIdx.y, b = blockIdx.z, wave = uniform(threadIdx.x >> 6);
    // The part begins where the caller's lengths put it, but for windows: its pages are asked for beside the lengths.
    const uint32_t guess = split * a.each + wave;
    Asked pages = ask_pages(a, b, guess, W);
    const SeqView v = seq_view(a.s, b, a.page_log);
    if (!v.ok) {
        if (a.splits == 1) not_a_number(a, b, h);
        return;
    }
    if (v.rows == 0) return;
    const Tiles tiles = tiles_of(a, v, 0, v.rows - 1);
    const uint32_t each = part_of(a, tiles);
    const uint32_t t_first = tiles.first + split * each, t_end = t_first + each < tiles.end ? t_first + each : tiles.end;
    if (a.splits > 1 && t_first >= t_end) return;  // k_attend_join knows
    if (t_first + wave != guess) pages = ask_pages(a, b, t_first + wave, W);
    attend_part<NJ, RT, W>(a, sh, v, b, h, t_first, t_end, pages, a.splits == 1,
                           (((size_t)b * a.cache.kv_heads + h) * a.splits + split) * a.rows_most);
}

// Sequences of unlike lengths: the tiles of all of them and of all heads lie in one row, sequence by sequence, head by head,
// and every workgroup has as many of them, `quota`, wherever they begin and end.  A sequence and head that lies
// in one workgroup is done there; of others a workgroup has an end as its first piece, a beginning as its last, or all it does
// lies within one: two pieces of sums at most.
// A sequence and head counts kPiece tiles more than it has, for what a piece costs however short it is (some 5 us to its first
// scores and from its last, when four tiles take 2.3).
static const uint32_t kMostShared = 256;  // sequences, a thread each
static const uint32_t kPiece = 8;
struct Row {
    uint32_t tiles[kMostShared], before[kMostShared], sums[4];
};
struct Share {
    uint32_t total, quota;
};
__device__ __forceinline__ Share share_out(const Args& a, Row& row) {
    const uint32_t tid = threadIdx.x, lane = tid & 63;
    uint32_t n = 0;
    if (tid < a.s.seqs) {
        const SeqView v = seq_view(a.s, tid, a.page_log);
        if (v.ok && v.rows > 0) {
            const Tiles t = tiles_of(a, v, 0, v.rows - 1);
            n = t.end - t.first;
        }
    }
    const uint32_t cost = n ? n + kPiece : 0;
    uint32_t sum = cost;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const uint32_t other = __shfl_up(sum, o);
        if (lane >= (uint32_t)o) sum += other;
    }
    if (lane == 63) row.sums[tid >> 6] = sum;
    __syncthreads();
    uint32_t before = sum - cost, total = 0;
#pragma unroll
    for (uint32_t w = 0; w < 4; ++w) {
        if (w < tid >> 6) before += row.sums[w];
        total += row.sums[w];
    }
    row.tiles[tid] = n;
    row.before[tid] = before;
    __syncthreads();
    Share s;
    s.total = uniform(total) * a.cache.kv_heads;
    const uint32_t need = (s.total + a.shared - 1) / a.shared;
    s.quota = need < 4 ? 4 : (need + 3) & ~3u;
    return s;
}

template <int NJ, int RT>
__global__ __launch_bounds__(kBlock, NJ * RT <= 2 ? 2 : 1) void k_attend_shared(Args a) {
    extern __shared__ float sh[];
    __shared__ Row row;
    __shared__ uint32_t found;
    const uint32_t tid = threadIdx.x, wave = uniform(tid >> 6), H = a.cache.kv_heads;
    const Share s = share_out(a, row);
    const uint32_t start = blockIdx.x * s.quota, end = start + s.quota < s.total ? start + s.quota : s.total;
    if (start >= end) return;
    const uint32_t first = row.before[tid] * H;
    if (row.tiles[tid] && first <= start && start - first < (row.tiles[tid] + kPiece) * H) found = tid;
    __syncthreads();
    uint32_t b = uniform(found);
    for (uint32_t at = start; at < end;) {
        const uint32_t n = uniform(row.tiles[b]), cost = n + kPiece, in = at - uniform(row.before[b]) * H, h = in / cost, tile = in - h * cost;
        const uint32_t stop = at + (cost - tile) < end ? at + (cost - tile) : end;
        if (tile < n) {
            const uint32_t there = tile + (stop - at) < n ? stop - at : n - tile;
            const SeqView v = seq_view(a.s, b, a.page_log);
            const uint32_t t_first = tiles_of(a, v, 0, v.rows - 1).first + tile;
            attend_part<NJ, RT, 4>(a, sh, v, b, h, t_first, t_first + there, ask_pages(a, b, t_first + wave, 4), there == n,
                                   ((size_t)blockIdx.x * 2 + (at == start ? 0 : 1)) * a.rows_most);
            __syncthreads();
        }
        at = stop;
        if (at < end && in + (cost - tile) == cost * H)  // the last head
            do ++b;
            while (uniform(row.tiles[b]) == 0);
    }
}

// A workgroup: one row of one sequence and head.  Threads hold four dimensions each; what is left of 256 takes parts
// in turn, and LDS adds them up.
static const uint32_t kMostSplits = 256;
__global__ __launch_bounds__(kBlock) void k_attend_join(Args a) {
    __shared__ Row row;
    __shared__ float weight[2 * kMostSplits + 8];
    __shared__ float red[4], red_l[4];
    __shared__ v4f sums[kBlock];
    const uint32_t r = blockIdx.x, h = blockIdx.y, b = blockIdx.z, d = a.cache.head_dim, H = a.cache.kv_heads, tid = threadIdx.x;
    // where the parts of the row lie: the first, the others from `next` on, `stride` apart
    uint32_t used;
    size_t part0, next, stride;
    const SeqView v = seq_view(a.s, b, a.page_log);
    if (!v.ok) {
        if (r == 0) not_a_number(a, b, h);
        return;
    }
    if (r >= (uint32_t)v.rows * a.group) return;
    if (a.shared) {
        const Share s = share_out(a, row);
        const uint32_t n = uniform(row.tiles[b]), from = uniform(row.before[b]) * H + h * (n + kPiece);
        const uint32_t w0 = from / s.quota, w1 = n ? (from + n - 1) / s.quota : w0;
        if (n && w0 == w1) return;  // done where it lies
        used = n ? w1 - w0 + 1 : 0;
        part0 = ((size_t)w0 * 2 + (from == w0 * s.quota ? 0 : 1)) * a.rows_most + r;
        next = (size_t)(w0 + 1) * 2 * a.rows_most + r;
        stride = 2 * (size_t)a.rows_most;
    } else {
        const Tiles tiles = a.few ? tiles_of(a, v, 0, v.rows - 1) : tiles_of_rows(a, v, r / kRows * kRows);
        const uint32_t each = part_of(a, tiles);
        used = (tiles.end - tiles.first + each - 1) / each;
        part0 = ((size_t)b * H + h) * a.splits * a.rows_most + r;
        next = part0 + a.rows_most;
        stride = a.rows_most;
    }
    auto part = [&](uint32_t s) -> size_t { return s ? next + (s - 1) * stride : part0; };
    float top = -kInf;
    for (uint32_t s = tid; s < used; s += kBlock) {
        const float m = a.parts_ml[part(s)].x;
        weight[s] = m;
        top = fmaxf(top, m);
    }
    top = wave_max(top);
    if ((tid & 63) == 0) red[tid >> 6] = top;
    __syncthreads();
    top = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
    const float ref = top == -kInf ? 0.0f : top;
    float l = 0.0f;
    for (uint32_t s = tid; s < used; s += kBlock) {
        const float f = exp2_of(weight[s] - ref);
        weight[s] = f;
        l += a.parts_ml[part(s)].y * f;
    }
    l = wave_add(l);
    if ((tid & 63) == 0) red_l[tid >> 6] = l;
    __syncthreads();
    l = (red_l[0] + red_l[1]) + (red_l[2] + red_l[3]);
    const uint32_t quads = d >> 2, ways = kBlock / quads, way = tid / quads, c = tid - way * quads;
    v4f sum = {0, 0, 0, 0};
    if (way < ways) {
#pragma unroll 8
        for (uint32_t s = way; s < used; s += ways) sum += ((const v4f*)a.parts)[part(s) * quads + c] * weight[s];
    }
    sums[tid] = sum;
    __syncthreads();
    if (way == 0) {
        for (uint32_t w = 1; w < ways; ++w) sum += sums[w * quads + c];
        const size_t at = row_at(a, v, h, r, a.orow, a.ohead) + 4 * c;
#pragma unroll
        for (int e = 0; e < 4; ++e) put_at(a.out, at + e, l == 0.0f ? 0.0f : sum[e] / l, a.dtype);
    }
    if (a.lse && tid == 0) a.lse[row_at(a, v, h, r, (size_t)H * a.group, 1)] = lse_of(ref, l);
}

// ---- many rows -------------------------------------------------------------------------------------------------------

// Lane 32 h + i: row i of its wavefront's 32, tokens 16 h .. 16 h + 15 of each half of a tile.
// DT: head_dim in units of 32, rounded up.  Rows in LDS are padded by 16 bytes: then those of 16 neighbouring rows lie in
// different banks, whatever DT.
template <int DT>
struct ManyLds {
    static constexpr uint32_t krow = 64 * DT + 16, vrow = 128 + 16, k_bytes = 64 * krow, bytes = k_bytes + 32 * DT * vrow;
};
template <int DT>
__global__ __launch_bounds__(kBlock, DT <= 4 ? 2 : 1) void k_attend_many(Args a) {
    using L = ManyLds<DT>;
    constexpr int PIECES = (DT + 1) / 2;  // of 16 codes, for a thread, of a tile's K and of its V
    extern __shared__ char lds[];
    __shared__ float exps[2][2][4];       // [buffer][K, V][16 tokens]
    __shared__ uint32_t pages[2][4];      // of the next tile
    const uint32_t tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, half = lane >> 5, i32 = lane & 31;
    const uint32_t h = blockIdx.x, b = blockIdx.z / a.splits, split = blockIdx.z - b * a.splits;
    const uint32_t d = a.cache.head_dim, T = 1u << a.page_log, H = a.cache.kv_heads;
    const SeqView v = seq_view(a.s, b, a.page_log);
    if (!v.ok) {
        if (blockIdx.y == 0 && a.splits == 1) not_a_number(a, b, h);
        return;
    }
    const uint32_t R = (uint32_t)v.rows * a.group, row_tiles = (R + kRows - 1) / kRows;
    if (blockIdx.y >= row_tiles) return;
    const uint32_t r0 = (row_tiles - 1 - blockIdx.y) * kRows;  // the rows that see most first, of all heads
    const uint32_t r_last = r0 + kRows - 1 < R - 1 ? r0 + kRows - 1 : R - 1;
    const int32_t tok0 = (int32_t)(r0 / a.group), tok1 = (int32_t)(r_last / a.group);
    Tiles tiles = tiles_of_rows(a, v, r0);
    if (a.splits > 1) {
        const uint32_t each = part_of(a, tiles);
        tiles.first += split * each;
        if (tiles.first >= tiles.end) return;  // k_attend_join knows
        tiles.end = tiles.first + each < tiles.end ? tiles.first + each : tiles.end;
    }
    const uint32_t r = r0 + wave * 32 + i32, seen_from = first_seen(a, v, tok0);

    v8h qf[2 * DT];
    float qmul;
    {
        const size_t at = row_at(a, v, h, r < R ? r : 0, a.qrow, a.qhead);
        v4u raw[2 * DT];
#pragma unroll
        for (int k = 0; k < 2 * DT; ++k) {
            v4u one[1] = {v4u{0, 0, 0, 0}};
            if (16u * k < d) load_raw<8>(a.q, at + 16 * k + 8 * half, a.wide, one);
            raw[k] = one[0];
        }
        qmul = scale_row<16 * DT>(raw, a.dtype, a.scale, qf, LargestOf2());
    }
    const int32_t pos = r < R ? v.len - v.rows + (int32_t)(r / a.group) : -1;
    const int32_t low = a.window ? pos - (int32_t)a.window : -1;  // keys in (low, pos] are seen
    const int32_t pos_first = v.len - v.rows + tok0, pos_last = v.len - v.rows + tok1;

    // What a thread brings of a tile: of K, pieces of 16 dimensions of a token; of V, of 16 tokens of a dimension.  As in
    // k_attend_few every load is made; what lies outside is not kept.
    uint32_t k_run[PIECES], k_at[PIECES], v_run[PIECES], v_at[PIECES];
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
        const AttendPiece p = attend_piece<DT>(tid, kBlock, i);
        k_run[i] = p.slot >> 4;
        k_at[i] = (p.slot & 15) * d + (16 * p.c < d ? 16 * p.c : 0);
        v_run[i] = p.run;
        v_at[i] = (p.dim < d ? p.dim : 0) << a.page_log;
    }
    v4u kr[PIECES], vr[PIECES];
    float my_exp = 0.0f;  // threads 0..7: K's and V's exponents of the tile's runs of 16 tokens
    auto fetch = [&](uint32_t t, const uint32_t(&page)[4]) {
        const uint32_t head = T * d;
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            const uint32_t kp = page_or_0(a, page[k_run[i]]), vp = page_or_0(a, page[v_run[i]]);
            const uint32_t k_slot = (t * kTile + 16 * k_run[i]) & (T - 1), v_slot = (t * kTile + 16 * v_run[i]) & (T - 1);
            kr[i] = *(const v4u*)(a.cache.k + ((size_t)kp * H + h) * head + k_slot * d + k_at[i]);
            vr[i] = *(const v4u*)(a.cache.v + ((size_t)vp * H + h) * head + v_at[i] + v_slot);
        }
        if (tid < 8) {
            const uint32_t it = page[tid & 3];
            const bool none = it >= a.cache.pages;
            const uint32_t key = t * kTile + 16 * (tid & 3);
            if (none && (int32_t)key <= pos_last && key + 16 > seen_from) report(a.s, ZK_FAULT_PAGE);
            const size_t at = (size_t)page_or_0(a, it) * H + h;
            my_exp = none ? (tid < 4 ? __builtin_nanf("") : 0.0f) : exponent_value(tid < 4 ? a.cache.k_exp[at] : a.cache.v_exp[at]);
        }
    };
    auto stage = [&](uint32_t buf) {
        char* kb = lds + buf * L::bytes;
        char* vb = kb + L::k_bytes;
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            if (!attend_piece_kept<DT>(tid, kBlock, i)) continue;
            const AttendPiece p = attend_piece<DT>(tid, kBlock, i);
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
        if (tid < 8) exps[buf][tid >> 2][tid & 3] = my_exp;
    };

    v16f o[DT];
#pragma unroll
    for (int c = 0; c < DT; ++c) o[c] = v16f{0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0};
    float m = -kInf, l = 0.0f;
    // pages are looked up two tiles ahead, by threads 0..3
    uint32_t my_page = 0;
    if (tiles.first < tiles.end) {
        uint32_t page[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) page[i] = page_of(a, b, tiles.first * kTile + 16 * i);
        if (tid < 4) my_page = page_of(a, b, (tiles.first + 1) * kTile + 16 * tid);
        fetch(tiles.first, page);
    }
    for (uint32_t t = tiles.first; t < tiles.end; ++t) {
        const uint32_t buf = (t - tiles.first) & 1;
        stage(buf);
        if (tid < 4) pages[buf][tid] = my_page;
        __syncthreads();
        if (t + 1 < tiles.end) {
            if (tid < 4) my_page = page_of(a, b, (t + 2) * kTile + 16 * tid);
            fetch(t + 1, pages[buf]);
        }
        const char* kb = lds + buf * L::bytes;
        const char* vb = kb + L::k_bytes;
        const int32_t base = (int32_t)(t * kTile);
        v16f s[2];
        float vback[2];
        float top = -kInf;
        const bool whole = base + (int32_t)kTile - 1 <= pos_first && base > (a.window ? pos_last - (int32_t)a.window : -1);
#pragma unroll
        for (int st = 0; st < 2; ++st) {
            s[st] = v16f{0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0};
            const char* krow = kb + (st * 32 + i32) * L::krow + half * 16;
#pragma unroll
            for (int k = 0; k < 2 * DT; ++k)
                s[st] = __builtin_amdgcn_mfma_f32_32x32x16_f16(*(const v8h*)(krow + 32 * k), qf[k], s[st], 0, 0, 0);
            const float ke = exps[buf][0][2 * st + half], ve = exps[buf][1][2 * st + half];
            const float mul = qmul * exp2_of(ke);
            vback[st] = back_of(ve);
            s[st] = s[st] * mul + ve;
            if (!whole) {
                const int32_t key0 = base + 32 * st + 16 * (int32_t)half;
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    if (key0 + e > pos || key0 + e <= low) s[st][e] = -kInf;
            }
#pragma unroll
            for (int e = 0; e < 16; ++e) top = fmaxf(top, s[st][e]);
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
#pragma unroll
            for (int e = 0; e < 16; e += 2) {
                const float x0 = exp2_of(s[st][e] - from), x1 = exp2_of(s[st][e + 1] - from);
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
    l = add_halves(l);
    if (r >= R) return;
    if (a.splits > 1) {
        const size_t part = (((size_t)b * H + h) * a.splits + split) * a.rows_most + r;
#pragma unroll
        for (int c = 0; c < DT; ++c)
#pragma unroll
            for (int e = 0; e < 16; e += 4) {
                const uint32_t dim = 32 * c + 2 * e + 4 * half;
                if (dim < d) *(v4f*)(a.parts + part * d + dim) = v4f{o[c][e], o[c][e + 1], o[c][e + 2], o[c][e + 3]};
            }
        if (half == 0) a.parts_ml[part] = make_float2(m, l);
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

// ---- host -------------------------------------------------------------------------------------------------------------

// How many workgroups share a sequence at most, and the tiles of each.
struct Split {
    uint32_t splits, each;
};
bool few_rows(uint64_t rows) { return rows <= 32; }
// Tiles that one workgroup of eight wavefronts does in one launch.  Measured at 8 heads of 128: one sequence of 777 tokens
// 10.7 us that way and 10.2 shared out, of 2000 16.6 and 10.6; 16 sequences of 1000 12.7 and 15.9; 24 of 1000 (four heads) 11.9 and 14.7.
uint32_t short_tiles(uint32_t seqs, uint32_t kv_heads) { return (uint64_t)seqs * kv_heads < 64 ? 8 : 32; }
// rows: of a sequence and head.  With many rows a workgroup is worth four tiles too, and the chip is full with fewer.
uint32_t most_splits(uint32_t seqs, uint32_t kv_heads, uint64_t rows, uint32_t tiles) {
    const uint64_t groups = (uint64_t)seqs * kv_heads * (few_rows(rows) ? 1 : div_up(rows, kRows));
    uint64_t n = groups >= (few_rows(rows) ? kWorkgroups : kWorkgroups / 2) ? 1 : div_up(kWorkgroups, groups);
    if (n > div_up(tiles, 4)) n = div_up(tiles, 4);  // few rows: a tile for each wavefront
    if (n > kMostSplits) n = kMostSplits;
    return n * seqs > 65535 ? 65535 / seqs : (uint32_t)n;
}
Split split_of(uint32_t seqs, uint32_t kv_heads, uint64_t rows, uint32_t tiles) {
    if (few_rows(rows) && tiles <= short_tiles(seqs, kv_heads)) return {1, tiles};
    const uint32_t each = (uint32_t)align_up(div_up(tiles, most_splits(seqs, kv_heads, rows, tiles)), 4);
    return {(uint32_t)div_up(tiles, each), each};
}
uint32_t tiles_for(uint32_t len) { return len ? (uint32_t)div_up(len, kTile) : 1; }

template <int NJ, int RT, int W>
int launch_few(const Args& a, hipStream_t stream) {
    const size_t lds = FewLds<NJ, RT, W>::bytes(a.rows_most);
    if constexpr (W == 4) {
        if (a.shared) {
            if (lds > 60000) ZK_HIP_TRY(hipFuncSetAttribute((const void*)k_attend_shared<NJ, RT>, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds));
            hipLaunchKernelGGL((k_attend_shared<NJ, RT>), dim3(a.shared), dim3(kBlock), lds, stream, a);
        }
    }
    if (!a.shared) {
        if (lds > 65536) ZK_HIP_TRY(hipFuncSetAttribute((const void*)k_attend_few<NJ, RT, W>, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds));
        hipLaunchKernelGGL((k_attend_few<NJ, RT, W>), dim3(a.splits, a.cache.kv_heads, a.s.seqs), dim3(64 * W), lds, stream, a);
    }
    if (a.splits > 1 || a.shared) hipLaunchKernelGGL(k_attend_join, dim3(a.rows_most, a.cache.kv_heads, a.s.seqs), dim3(kBlock), 0, stream, a);
    ZK_HIP_TRY(hipGetLastError());
    return ZK_OK;
}

template <int DT>
int launch_many(const Args& a, hipStream_t stream) {
    const size_t lds = 2 * (size_t)ManyLds<DT>::bytes;
    if (lds > 65536) ZK_HIP_TRY(hipFuncSetAttribute((const void*)k_attend_many<DT>, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds));
    hipLaunchKernelGGL((k_attend_many<DT>), dim3(a.cache.kv_heads, (unsigned)div_up(a.rows_most, kRows), a.s.seqs * a.splits), dim3(kBlock), lds, stream, a);
    if (a.splits > 1) hipLaunchKernelGGL(k_attend_join, dim3(a.rows_most, a.cache.kv_heads, a.s.seqs), dim3(kBlock), 0, stream, a);
    ZK_HIP_TRY(hipGetLastError());
    return ZK_OK;
}

template <int NJ>
int launch(const Args& a, hipStream_t stream) {
    if (a.rows_most <= 16) return a.splits == 1 && !a.shared && !a.crowd ? launch_few<NJ, 1, 8>(a, stream) : launch_few<NJ, 1, 4>(a, stream);
    if (few_rows(a.rows_most)) return launch_few<NJ, 2, 4>(a, stream);
    return a.cache.head_dim > 64 * NJ - 32 ? launch_many<2 * NJ>(a, stream) : launch_many<2 * NJ - 1>(a, stream);
}

// Whether sequences share their workgroups out by tiles, not by parts of like size of each.  Measured, us, shared out and in parts,
// lengths spread evenly up to the longest, 8 heads of 128: 32 sequences of 4096 39.4 and 43.8, 16 of 8000 38.5 and 43.1, 8 of
// 30000 68 and 76, 64 of 4096 65 and 68; 100 of 3000 84 and 83 (800 pairs: not shared out); 32 of 4096 all alike 63 and 59.
bool shared_out(uint32_t seqs, uint32_t kv_heads, uint64_t rows, uint32_t tiles) {
    const uint64_t groups = (uint64_t)seqs * kv_heads;
    return few_rows(rows) && seqs > 1 && seqs <= kMostShared && groups >= 64 && groups <= kWorkgroups && tiles > short_tiles(seqs, kv_heads);
}
size_t parts_bytes(size_t parts, uint32_t head_dim) {
    Carver cv(nullptr, 0);
    cv.take(parts * head_dim * sizeof(float));
    cv.take(parts * sizeof(float2));
    return cv.used();
}

// Rows of a sequence and head at most.
uint64_t rows_most(uint32_t rows, uint32_t max_new, uint32_t group) { return (uint64_t)(max_new < rows ? max_new : rows) * group; }

}  // namespace
}  // namespace zkmi

using namespace zkmi;

extern "C" size_t kvcache_attention_workspace_bytes(uint32_t seqs, uint32_t rows, uint32_t max_new, uint32_t q_heads, uint32_t kv_heads,
                                                    uint32_t head_dim, uint32_t max_len) {
    if (!kv_heads || q_heads % kv_heads || !seqs || !rows || !max_new) return 0;
    const uint64_t most = rows_most(rows, max_new, q_heads / kv_heads);
    const uint32_t tiles = tiles_for(max_len);
    if (few_rows(most) && tiles <= short_tiles(seqs, kv_heads)) return 0;
    // a window makes tiles and workgroups fewer, never more
    const uint32_t splits = most_splits(seqs, kv_heads, most, tiles);
    size_t parts = splits == 1 ? 0 : (size_t)seqs * kv_heads * splits * most;
    if (shared_out(seqs, kv_heads, most, tiles) && parts < 2 * (size_t)kWorkgroups * most) parts = 2 * (size_t)kWorkgroups * most;
    return parts ? parts_bytes(parts, head_dim) : 0;
}

extern "C" int kvcache_attention(const kvcache_i8* cache, const void* q, size_t q_row_stride, size_t q_head_stride, int dtype,
                                 uint32_t q_heads, const kv_seqs* seqs, float scale, uint32_t window, void* out, size_t out_row_stride,
                                 size_t out_head_stride, float* lse, void* ws, size_t ws_bytes, void* stream) {
    if ((dtype != ZK_F16 && dtype != ZK_BF16) || !cache_ok(cache) || !seqs_ok(seqs)) return ZK_E_BADARG;
    if (q_heads == 0 || q_heads % cache->kv_heads || q_heads > 65536 || window >= 0x80000000u || !(scale - scale == 0.0f)) return ZK_E_BADARG;
    if (seqs->rows == 0 || seqs->seqs == 0) return ZK_OK;
    if (!q || !out || !aligned(q, 2) || !aligned(out, 2) || (lse && !aligned(lse, 4))) return ZK_E_BADARG;
    const uint32_t group = q_heads / cache->kv_heads;
    const uint64_t most = rows_most(seqs->rows, seqs->max_new, group);
    if (div_up(most, kRows) > 65535) return ZK_E_BADARG;
    // what a window lets a sequence's rows see, with a tile that it ends in
    const uint64_t seen = window ? (uint64_t)window + seqs->max_new + kTile : seqs->max_len;
    const uint32_t tiles = tiles_for(seen < seqs->max_len ? (uint32_t)seen : seqs->max_len);
    const Split sp = split_of(seqs->seqs, cache->kv_heads, most, tiles);
    // what the table has room for decides whether tiles can be counted in 32 bits: the lengths are on the device
    const bool countable = (uint64_t)seqs->seqs * cache->kv_heads * ((uint64_t)seqs->table_pages * cache->page_tokens / kTile + 2 + kPiece) < 0x7fffffffu;
    const bool shared = countable && shared_out(seqs->seqs, cache->kv_heads, most, tiles);
    Args a = {};
    a.cache = *cache;
    a.s = *seqs;
    a.q = q;
    a.qrow = q_row_stride;
    a.qhead = q_head_stride;
    a.out = out;
    a.orow = out_row_stride;
    a.ohead = out_head_stride;
    a.lse = lse;
    a.scale = scale;
    a.window = window;
    a.group = group;
    a.page_log = (uint32_t)log2_floor(cache->page_tokens);
    a.dtype = dtype;
    a.few = few_rows(most);
    a.wide = aligned(q, 16) && q_row_stride % 8 == 0 && q_head_stride % 8 == 0;
    a.rows_most = (uint32_t)most;
    a.splits = shared ? 1 : sp.splits;
    a.each = sp.each;
    a.shared = shared ? kWorkgroups : 0;
    a.crowd = (uint64_t)seqs->seqs * cache->kv_heads >= kWorkgroups;
    if (shared || sp.splits > 1) {
        const size_t parts = shared ? 2 * (size_t)kWorkgroups * most : (size_t)seqs->seqs * cache->kv_heads * sp.splits * most;
        if (!ws) return ZK_E_BUFSZ;
        Carver cv(ws, ws_bytes);
        a.parts = (float*)cv.take(parts * cache->head_dim * sizeof(float));
        a.parts_ml = (float2*)cv.take(parts * sizeof(float2));
        if (cv.overflow() || !a.parts || !a.parts_ml) return ZK_E_BUFSZ;
    }
    hipStream_t s = as_stream(stream);
    switch ((cache->head_dim + 63) / 64) {
        case 1: return launch<1>(a, s);
        case 2: return launch<2>(a, s);
        case 3: return launch<3>(a, s);
        default: return launch<4>(a, s);
    }
}
