// Attention over the cache of 8-bit keys and values.
//
// With K, V the codes, 2^a and 2^b their pages' scales: s_j = scale * 2^a_j (q . K_j), o = sum_j e^{s_j} 2^b_j V_j / sum_j e^{s_j}
// over the keys j that a query sees.  One pass over the keys with a running maximum:
//   * in units of log2: t_j = s_j log2(e) + b_j, M = max t_j - 14, P_j = 2^(t_j - M).  The scale of V is an exponent and
//     joins the score's, so the weights of all pages enter ONE accumulator of products with the codes as they are, whatever
//     their scales; the sum of the weights is l = sum_j P_j 2^-b_j.  P is at most 2^14: as a 16-bit float with its 11 bits
//     it reaches 29 binades below the largest at full precision and 10 more at less.  Exponents lie in [-40, 40], so a
//     score that matters is never below what a 32-bit P holds.
//   * codes become 16-bit floats by putting the byte (with its top bit flipped) under the exponent of 1024 and taking 1152
//     off: exact, five instructions for four codes.  q is scaled by a power of two to just below 2^15, which a 16-bit float
//     holds exactly but for elements 2^-29 of the row's largest.
//   * both products run on the matrix cores, transposed: S^T = K Q^T and O^T = V^T P^T.  What comes out of the first is the
//     second's operand without a move between lanes: a lane gets the scores of tokens that lie side by side, because
//     the rows of K are handed in that order, and V lies in the cache by dimension.
//
// Few rows (k_attend_few: up to 32 of a sequence and head of the cache, the query heads that share it among them): the
// cache is read once, straight into registers, and is what bounds the call.  A wavefront takes 64 tokens at a time, four
// wavefronts share a workgroup's part of the sequence, and `splits` workgroups the sequence; k_attend_join adds up.
// Many rows (k_attend_many: 128 to a workgroup): codes are widened once and shared through LDS; bound by the
// matrix cores and the exponentials.
#include "kvcache.h"

namespace zkmi {
namespace {

static const float kLog2e = 1.44269504088896341f, kLn2 = 0.693147180559945309f;
static const float kHead = 14.0f;      // P reaches up to 2^14
static const uint32_t kTile = 64;      // tokens

struct Args {
    kvcache_i8 cache;
    kv_seqs s;
    const void* q;
    size_t qrow, qhead;
    void* out;
    size_t orow, ohead;
    float* lse;
    float scale;
    uint32_t window, group, page_log, splits;  // group: query heads of a head of the cache
    int dtype;
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

__device__ __forceinline__ float value_at(const void* p, size_t i, int dtype) {
    return dtype == ZK_BF16 ? load_one<ZK_BF16>(p, i) : load_one<ZK_F16>(p, i);
}
__device__ __forceinline__ void put_at(void* p, size_t i, float f, int dtype) {
    if (dtype == ZK_BF16) store_one<ZK_BF16>(p, i, f);
    else store_one<ZK_F16>(p, i, f);
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

// Tiles [first, end) of the keys that rows [i0, i1] of a sequence see.
struct Tiles {
    uint32_t first, end;
};
__device__ __forceinline__ Tiles tiles_of(const Args& a, const SeqView& v, int32_t i0, int32_t i1) {
    const int64_t past = (int64_t)v.len - v.rows, last = past + i1, low = a.window ? past + i0 - (int64_t)a.window + 1 : 0;
    Tiles t;
    t.first = low > 0 ? (uint32_t)(low / kTile) : 0;
    t.end = last < 0 ? t.first : (uint32_t)(last / kTile) + 1;
    return t;
}

// A page of a sequence: its number (0 where the table names none), and what its exponents are worth.
struct Page {
    uint32_t at;
    bool none;
};
__device__ __forceinline__ Page page_at(const Args& a, uint32_t b, uint32_t token, uint32_t len) {
    Page p = {0, false};
    if (token < len) {
        p.at = (uint32_t)a.s.table[(size_t)b * a.s.table_stride + (token >> a.page_log)];
        p.none = p.at >= a.cache.pages;
        if (p.none) p.at = 0;
    }
    return p;
}
__device__ __forceinline__ float exponent_value(int e) { return e == ZK_EXP_NAN ? __builtin_nanf("") : (float)e; }

// What a row ends with.
__device__ __forceinline__ float lse_of(float m, float l) { return l == 0.0f ? -kInf : (m + __log2f(l)) * kLn2; }

// ---- few rows --------------------------------------------------------------------------------------------------------

// NJ: head_dim in units of 64, rounded up.  RT: tiles of 16 rows.  Lane 16 g + i: row i of a tile, tokens 16 g .. 16 g + 15.
template <int NJ, int RT>
__global__ __launch_bounds__(kBlock, NJ * RT <= 2 ? 2 : 1) void k_attend_few(Args a) {
    constexpr int DT = 4 * NJ;  // tiles of 16 dimensions
    extern __shared__ float sh[];
    const uint32_t tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, g = lane >> 4, i16 = lane & 15;
    const uint32_t split = blockIdx.x, h = blockIdx.y, b = blockIdx.z, d = a.cache.head_dim, T = 1u << a.page_log, H = a.cache.kv_heads;
    const SeqView v = seq_view(a.s, b, a.page_log);
    if (!v.ok) {
        if (a.splits == 1) not_a_number(a, b, h);
        return;
    }
    if (v.rows == 0) return;
    const uint32_t R = (uint32_t)v.rows * a.group;
    const Tiles tiles = tiles_of(a, v, 0, v.rows - 1);
    const uint32_t each = (tiles.end - tiles.first + a.splits - 1) / a.splits;
    const uint32_t t_first = tiles.first + split * each, t_end = t_first + each < tiles.end ? t_first + each : tiles.end;
    if (a.splits > 1 && t_first >= t_end) return;  // k_attend_join knows

    // q, scaled by a power of two; qmul takes that back and brings the units of log2
    v8h qf[RT][NJ][2];
    float qmul[RT];
    int32_t pos[RT];  // the last key that the lane's row sees
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        const uint32_t r = rt * 16 + i16;
        float x[NJ][16], amax = 0.0f;
        const size_t at = r < R ? row_at(a, v, h, r, a.qrow, a.qhead) : 0;
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const uint32_t c = 64 * j + 16 * g + e;
                x[j][e] = r < R && c < d ? value_at(a.q, at + c, a.dtype) : 0.0f;
                // NaN has to come through as infinity does
                amax = fabsf(x[j][e]) <= 3.4028235e38f ? fmaxf(amax, fabsf(x[j][e])) : kInf;
                if (amax == kInf) x[j][e] = 0.0f;
            }
        amax = max_halves(max_rows(amax));
        int ex = 0;
        (void)frexpf(amax, &ex);
        if (amax == 0.0f || amax == kInf) ex = 0;
        qmul[rt] = amax == kInf ? __builtin_nanf("") : ldexpf(a.scale * kLog2e, ex - 15);
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) qf[rt][j][e >> 3][e & 7] = (_Float16)ldexpf(x[j][e], 15 - ex);
        pos[rt] = r < R ? v.len - v.rows + (int32_t)(r / a.group) : -1;
    }

    const uint32_t len = (uint32_t)v.len, rk = i16 >> 2;
    const size_t page_stride = (size_t)T * d;
    v4u kr[4][NJ], vr[DT];
    auto load_k = [&](const Page& p, uint32_t t) {
        const uint32_t token = t * kTile + 16 * rk;
        const int8_t* at = a.cache.k + ((size_t)p.at * H + h) * page_stride + (size_t)((token & (T - 1)) + (i16 & 3)) * d + 16 * g;
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int j = 0; j < NJ; ++j) {
                kr[u][j] = v4u{0, 0, 0, 0};
                if (token < len && 64 * j + 16 * g < d) kr[u][j] = __builtin_nontemporal_load((const v4u*)(at + (size_t)(4 * u) * d + 64 * j));
            }
    };
    auto load_v = [&](const Page& p, uint32_t t) {
        const uint32_t token = t * kTile + 16 * g;
        const int8_t* at = a.cache.v + ((size_t)p.at * H + h) * page_stride + ((size_t)i16 << a.page_log) + (token & (T - 1));
#pragma unroll
        for (int c = 0; c < DT; ++c) {
            vr[c] = v4u{0, 0, 0, 0};
            if (token < len && 16u * c < d) vr[c] = __builtin_nontemporal_load((const v4u*)(at + ((size_t)(16 * c) << a.page_log)));
        }
    };
    float ke = 0.0f, ve = 0.0f;  // exponents of the lane's 16 tokens
    auto load_e = [&](const Page& p) {
        const size_t at = (size_t)p.at * H + h;
        ke = p.none ? __builtin_nanf("") : exponent_value(a.cache.k_exp[at]);
        ve = p.none ? 0.0f : exponent_value(a.cache.v_exp[at]);
        if (p.none) report(a.s, ZK_FAULT_PAGE);
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
    Page pk_next = {0, false}, pv_next = {0, false};
    if (t < t_end) {
        const Page pk = page_at(a, b, t * kTile + 16 * rk, len), pv = page_at(a, b, t * kTile + 16 * g, len);
        load_k(pk, t);
        load_e(pv);
        load_v(pv, t);
        if (t + 4 < t_end) {
            pk_next = page_at(a, b, (t + 4) * kTile + 16 * rk, len);
            pv_next = page_at(a, b, (t + 4) * kTile + 16 * g, len);
        }
    }
    for (; t < t_end; t += 4) {
        const bool more = t + 4 < t_end;
        Page pk_after = {0, false}, pv_after = {0, false};
        if (t + 8 < t_end) {
            pk_after = page_at(a, b, (t + 8) * kTile + 16 * rk, len);
            pv_after = page_at(a, b, (t + 8) * kTile + 16 * g, len);
        }
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
                    s[rt][u] = __builtin_amdgcn_mfma_f32_16x16x32_f16(a0, qf[rt][j][0], s[rt][u], 0, 0, 0);
                    s[rt][u] = __builtin_amdgcn_mfma_f32_16x16x32_f16(a1, qf[rt][j][1], s[rt][u], 0, 0, 0);
                }
            }
        }
        if (more) load_k(pk_next, t + 4);
        const float kscale = exp2_of(ke), vback = exp2_of(-ve), vadd = ve;
        if (more) load_e(pv_next);

        const int32_t base = (int32_t)(t * kTile);
        // whether every row sees all 64 tokens
        const bool whole = base + (int32_t)kTile - 1 <= v.len - v.rows && (!a.window || (int64_t)base > (int64_t)v.len - 1 - a.window);
        v8h p[RT][2];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            const float mul = qmul[rt] * kscale;
            float top = -kInf;
#pragma unroll
            for (int u = 0; u < 4; ++u)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float x = s[rt][u][e] * mul + vadd;
                    if (!whole) {
                        const int32_t key = base + 16 * (int32_t)g + 4 * u + e;
                        const bool seen = key <= pos[rt] && (!a.window || (int64_t)key > (int64_t)pos[rt] - a.window);
                        x = seen ? x : -kInf;
                    }
                    s[rt][u][e] = x;
                    top = fmaxf(top, x);
                }
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
            if (16u * c >= d) continue;
            const v8h a0 = widen(vr[c][0], vr[c][1]), a1 = widen(vr[c][2], vr[c][3]);
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                o[rt][c] = __builtin_amdgcn_mfma_f32_16x16x32_f16(a0, p[rt][0], o[rt][c], 0, 0, 0);
                o[rt][c] = __builtin_amdgcn_mfma_f32_16x16x32_f16(a1, p[rt][1], o[rt][c], 0, 0, 0);
            }
        }
        if (more) load_v(pv_next, t + 4);
        pk_next = pk_after;
        pv_next = pv_after;
    }

    // The wavefronts' sums: relative to one maximum, then two and two in LDS.
    const uint32_t D = 16 * DT + 4;  // a row of sums, padded
    float* ml = sh;                  // [wave][16 RT]
    float* sums = sh + 2 * 4 * 16 * RT;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        l[rt] = add_halves(add_rows(l[rt]));
        if (g == 0) {
            ml[wave * 16 * RT + rt * 16 + i16] = m[rt];
            ml[(4 + wave) * 16 * RT + rt * 16 + i16] = l[rt];
        }
    }
    __syncthreads();
    for (int turn = 0; turn < 2; ++turn) {
        if ((int)(wave >> 1) == turn) {
            float* to = sums + (size_t)(wave & 1) * 16 * RT * D;
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                const float* w = ml + rt * 16 + i16;
                const float all = fmaxf(fmaxf(w[0], w[16 * RT]), fmaxf(w[2 * 16 * RT], w[3 * 16 * RT]));
                const float f = exp2_of(all == -kInf ? 0.0f : m[rt] - all);
#pragma unroll
                for (int c = 0; c < DT; ++c) {
                    v4f* cell = (v4f*)(to + (size_t)(rt * 16 + i16) * D + 16 * c + 4 * g);
                    v4f x = o[rt][c] * f;
                    if (turn) x += *cell;
                    *cell = x;
                }
            }
        }
        __syncthreads();
    }
    for (uint32_t i = tid; i < R * d; i += kBlock) {
        const uint32_t r = i / d, c = i - r * d;
        const float* w = ml + r;
        const float all = fmaxf(fmaxf(w[0], w[16 * RT]), fmaxf(w[2 * 16 * RT], w[3 * 16 * RT])), ref = all == -kInf ? 0.0f : all;
        float ls = 0.0f;
#pragma unroll
        for (int x = 0; x < 4; ++x) ls += w[(4 + x) * 16 * RT] * exp2_of(all == -kInf ? 0.0f : w[x * 16 * RT] - all);
        const float sum = sums[(size_t)r * D + c] + sums[(size_t)(16 * RT + r) * D + c];
        if (a.splits == 1) {
            put_at(a.out, row_at(a, v, h, r, a.orow, a.ohead) + c, ls == 0.0f ? 0.0f : sum / ls, a.dtype);
            if (a.lse && c == 0) a.lse[row_at(a, v, h, r, (size_t)H * a.group, 1)] = lse_of(ref, ls);
        } else {
            const size_t part = (((size_t)b * H + h) * a.splits + split) * a.rows_most + r;
            a.parts[part * d + c] = sum;
            if (c == 0) a.parts_ml[part] = make_float2(all, ls);
        }
    }
}

// A workgroup: one row of one sequence and head; a thread for each dimension.
__global__ __launch_bounds__(kBlock) void k_attend_join(Args a) {
    const uint32_t r = blockIdx.x, h = blockIdx.y, b = blockIdx.z, d = a.cache.head_dim, H = a.cache.kv_heads, c = threadIdx.x;
    const SeqView v = seq_view(a.s, b, a.page_log);
    if (!v.ok) {
        if (r == 0) not_a_number(a, b, h);
        return;
    }
    if (r >= (uint32_t)v.rows * a.group) return;
    const Tiles tiles = tiles_of(a, v, 0, v.rows - 1);
    const uint32_t n = tiles.end - tiles.first, each = (n + a.splits - 1) / a.splits, used = n ? (n + each - 1) / each : 0;
    const size_t part0 = ((size_t)b * H + h) * a.splits * a.rows_most + r;
    float top = -kInf;
    for (uint32_t s = 0; s < used; ++s) top = fmaxf(top, a.parts_ml[part0 + (size_t)s * a.rows_most].x);
    const float ref = top == -kInf ? 0.0f : top;
    float l = 0.0f, sum = 0.0f;
    for (uint32_t s = 0; s < used; ++s) {
        const size_t part = part0 + (size_t)s * a.rows_most;
        const float2 ml = a.parts_ml[part];
        const float f = exp2_of(ml.x - ref);
        l += ml.y * f;
        if (c < d) sum += a.parts[part * d + c] * f;
    }
    if (c < d) put_at(a.out, row_at(a, v, h, r, a.orow, a.ohead) + c, l == 0.0f ? 0.0f : sum / l, a.dtype);
    if (a.lse && c == 0) a.lse[row_at(a, v, h, r, (size_t)H * a.group, 1)] = lse_of(ref, l);
}

// ---- many rows -------------------------------------------------------------------------------------------------------

static const uint32_t kRows = 128;

// Lane 32 h + i: row i of its wavefront's 32, tokens 16 h .. 16 h + 15 of each half of a tile.
template <int NJ>
__global__ __launch_bounds__(kBlock, NJ <= 2 ? 2 : 1) void k_attend_many(Args a) {
    constexpr int DT = 2 * NJ;            // tiles of 32 dimensions
    constexpr uint32_t KROW = 128 * NJ;   // bytes of a row of K in LDS
    constexpr uint32_t BUF = 2 * 64 * KROW;  // K and V
    extern __shared__ char lds[];
    __shared__ float exps[2][2][4];       // [buffer][K, V][16 tokens]
    const uint32_t tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, half = lane >> 5, i32 = lane & 31;
    const uint32_t h = blockIdx.y, b = blockIdx.z, d = a.cache.head_dim, T = 1u << a.page_log, H = a.cache.kv_heads;
    const SeqView v = seq_view(a.s, b, a.page_log);
    if (!v.ok) {
        if (blockIdx.x == 0) not_a_number(a, b, h);
        return;
    }
    const uint32_t R = (uint32_t)v.rows * a.group, row_tiles = (R + kRows - 1) / kRows;
    if (blockIdx.x >= row_tiles) return;
    const uint32_t r0 = (row_tiles - 1 - blockIdx.x) * kRows;  // the rows that see most first
    const uint32_t r_last = r0 + kRows - 1 < R - 1 ? r0 + kRows - 1 : R - 1;
    const int32_t tok0 = (int32_t)(r0 / a.group), tok1 = (int32_t)(r_last / a.group);
    const Tiles tiles = tiles_of(a, v, tok0, tok1);
    const uint32_t r = r0 + wave * 32 + i32, len = (uint32_t)v.len;

    v8h qf[4 * NJ];
    float qmul;
    {
        float x[4 * NJ][8], amax = 0.0f;
        const size_t at = r < R ? row_at(a, v, h, r, a.qrow, a.qhead) : 0;
#pragma unroll
        for (int k = 0; k < 4 * NJ; ++k)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const uint32_t c = 16 * k + 8 * half + e;
                x[k][e] = r < R && c < d ? value_at(a.q, at + c, a.dtype) : 0.0f;
                amax = fabsf(x[k][e]) <= 3.4028235e38f ? fmaxf(amax, fabsf(x[k][e])) : kInf;
                if (amax == kInf) x[k][e] = 0.0f;
            }
        amax = max_halves(amax);
        int ex = 0;
        (void)frexpf(amax, &ex);
        if (amax == 0.0f || amax == kInf) ex = 0;
        qmul = amax == kInf ? __builtin_nanf("") : ldexpf(a.scale * kLog2e, ex - 15);
#pragma unroll
        for (int k = 0; k < 4 * NJ; ++k)
#pragma unroll
            for (int e = 0; e < 8; ++e) qf[k][e] = (_Float16)ldexpf(x[k][e], 15 - ex);
    }
    const int32_t pos = r < R ? v.len - v.rows + (int32_t)(r / a.group) : -1;
    const int32_t pos_first = v.len - v.rows + tok0, pos_last = v.len - v.rows + tok1;

    // Row of K for token x of 32: the product's rows 8 b + 4 h + j come out in lane half h, as tokens 16 h + 4 b + j
    v4u kr[NJ], vr[NJ];
    auto fetch = [&](uint32_t t) {
#pragma unroll
        for (int i = 0; i < NJ; ++i) {
            const uint32_t p = tid + kBlock * i, slot = p / (4 * NJ), c = p % (4 * NJ) * 16, token = t * kTile + slot;
            kr[i] = v4u{0, 0, 0, 0};
            if (c < d && token < len) {
                const Page page = page_at(a, b, token, len);
                kr[i] = *(const v4u*)(a.cache.k + (((size_t)page.at * H + h) * T + (token & (T - 1))) * d + c);
            }
            const uint32_t run = p & 3, dim = p >> 2, vt = t * kTile + 16 * run;
            vr[i] = v4u{0, 0, 0, 0};
            if (dim < d && vt < len) {
                const Page page = page_at(a, b, vt, len);
                vr[i] = *(const v4u*)(a.cache.v + ((((size_t)page.at * H + h) * d + dim) << a.page_log) + (vt & (T - 1)));
            }
        }
    };
    float my_exp = 0.0f;  // threads 0..7: K's and V's exponents of the tile's runs
    auto fetch_exp = [&](uint32_t t) {
        if (tid < 8) {
            const uint32_t token = t * kTile + 16 * (tid & 3);
            const Page page = page_at(a, b, token, len);
            if (page.none) report(a.s, ZK_FAULT_PAGE);
            const size_t at = (size_t)page.at * H + h;
            my_exp = page.none ? (tid < 4 ? __builtin_nanf("") : 0.0f)
                               : token < len ? exponent_value(tid < 4 ? a.cache.k_exp[at] : a.cache.v_exp[at]) : 0.0f;
        }
    };
    auto stage = [&](uint32_t buf) {
        char* kb = lds + buf * BUF;
        char* vb = kb + 64 * KROW;
#pragma unroll
        for (int i = 0; i < NJ; ++i) {
            const uint32_t p = tid + kBlock * i, slot = p / (4 * NJ), c = p % (4 * NJ) * 2, x = slot & 31;
            const uint32_t row = (slot & 32) + 8 * ((x >> 2) & 3) + 4 * (x >> 4) + (x & 3), turn = row & (8 * NJ - 1) & 15;
            *(v8h*)(kb + row * KROW + ((c ^ turn) << 4)) = widen(kr[i][0], kr[i][1]);
            *(v8h*)(kb + row * KROW + (((c + 1) ^ turn) << 4)) = widen(kr[i][2], kr[i][3]);
            const uint32_t run = (p & 3) * 2, dim = p >> 2;
            *(v8h*)(vb + dim * 128 + ((run ^ (dim & 7)) << 4)) = widen(vr[i][0], vr[i][1]);
            *(v8h*)(vb + dim * 128 + (((run + 1) ^ (dim & 7)) << 4)) = widen(vr[i][2], vr[i][3]);
        }
        if (tid < 8) exps[buf][tid >> 2][tid & 3] = my_exp;
    };

    v16f o[DT];
#pragma unroll
    for (int c = 0; c < DT; ++c) o[c] = v16f{0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0};
    float m = -kInf, l = 0.0f;
    if (tiles.first < tiles.end) {
        fetch(tiles.first);
        fetch_exp(tiles.first);
    }
    for (uint32_t t = tiles.first; t < tiles.end; ++t) {
        const uint32_t buf = (t - tiles.first) & 1;
        stage(buf);
        __syncthreads();
        if (t + 1 < tiles.end) {
            fetch(t + 1);
            fetch_exp(t + 1);
        }
        const char* kb = lds + buf * BUF;
        const char* vb = kb + 64 * KROW;
        const int32_t base = (int32_t)(t * kTile);
        v16f s[2];
        float vback[2];
        float top = -kInf;
        const bool whole = base + (int32_t)kTile - 1 <= pos_first && (!a.window || (int64_t)base > (int64_t)pos_last - a.window);
#pragma unroll
        for (int st = 0; st < 2; ++st) {
            s[st] = v16f{0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0};
            const uint32_t row = st * 32 + i32, turn = row & (8 * NJ - 1) & 15;
#pragma unroll
            for (int k = 0; k < 4 * NJ; ++k) {
                if (16u * k >= d) continue;
                const v8h f = *(const v8h*)(kb + row * KROW + (((2 * k + half) ^ turn) << 4));
                s[st] = __builtin_amdgcn_mfma_f32_32x32x16_f16(f, qf[k], s[st], 0, 0, 0);
            }
            const float ke = exps[buf][0][2 * st + half], ve = exps[buf][1][2 * st + half];
            const float mul = qmul * exp2_of(ke);
            vback[st] = exp2_of(-ve);
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                float x = s[st][e] * mul + ve;
                if (!whole) {
                    const int32_t key = base + 32 * st + 16 * (int32_t)half + e;
                    const bool seen = key <= pos && (!a.window || (int64_t)key > (int64_t)pos - a.window);
                    x = seen ? x : -kInf;
                }
                s[st][e] = x;
                top = fmaxf(top, x);
            }
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
            if (32u * c >= d) continue;
            const uint32_t dim = 32 * c + i32;
#pragma unroll
            for (int st = 0; st < 2; ++st)
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const uint32_t chunk = (2 * st + half) * 2 + k;
                    const v8h f = *(const v8h*)(vb + dim * 128 + ((chunk ^ (dim & 7)) << 4));
                    o[c] = __builtin_amdgcn_mfma_f32_32x32x16_f16(f, p[st][k], o[c], 0, 0, 0);
                }
        }
    }
    l = add_halves(l);
    if (r < R) {
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
}

// ---- host -------------------------------------------------------------------------------------------------------------

// How many workgroups share a sequence: enough of them for some four on each of 256 CUs, but not less than a tile for each
// of a workgroup's wavefronts.
uint32_t splits_of(uint32_t seqs, uint32_t kv_heads, uint32_t max_len) {
    const uint64_t tiles = div_up(max_len, kTile), most = div_up(tiles, 4), groups = (uint64_t)seqs * kv_heads;
    uint64_t n = groups >= 1024 ? 1 : div_up(1024, groups ? groups : 1);
    if (n > most) n = most;
    return n < 1 ? 1 : (uint32_t)n;
}

bool few_rows(uint64_t rows) { return rows <= 32; }

template <int NJ, int RT>
int launch_few(const Args& a, hipStream_t stream) {
    const size_t lds = (2 * 4 * 16 * RT + 2 * (size_t)16 * RT * (64 * NJ + 4)) * sizeof(float);
    if (lds > 65536) ZK_HIP_TRY(hipFuncSetAttribute((const void*)k_attend_few<NJ, RT>, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds));
    hipLaunchKernelGGL((k_attend_few<NJ, RT>), dim3(a.splits, a.cache.kv_heads, a.s.seqs), dim3(kBlock), lds, stream, a);
    ZK_HIP_TRY(hipGetLastError());
    if (a.splits > 1) {
        const unsigned threads = (unsigned)align_up(a.cache.head_dim, 64);
        hipLaunchKernelGGL(k_attend_join, dim3(a.rows_most, a.cache.kv_heads, a.s.seqs), dim3(threads), 0, stream, a);
        ZK_HIP_TRY(hipGetLastError());
    }
    return ZK_OK;
}

template <int NJ>
int launch(const Args& a, hipStream_t stream) {
    if (a.rows_most <= 16) return launch_few<NJ, 1>(a, stream);
    if (few_rows(a.rows_most)) return launch_few<NJ, 2>(a, stream);
    const size_t lds = 2 * 2 * 64 * 128 * (size_t)NJ;
    ZK_HIP_TRY(hipFuncSetAttribute((const void*)k_attend_many<NJ>, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds));
    hipLaunchKernelGGL((k_attend_many<NJ>), dim3((unsigned)div_up(a.rows_most, kRows), a.cache.kv_heads, a.s.seqs), dim3(kBlock), lds, stream, a);
    ZK_HIP_TRY(hipGetLastError());
    return ZK_OK;
}

struct Shape {
    uint32_t rows_most, splits;
    size_t parts;  // rows of partial sums
};
Shape shape_of(uint32_t seqs, uint32_t rows, uint32_t max_new, uint32_t q_heads, uint32_t kv_heads, uint32_t max_len) {
    const uint32_t n = max_new < rows ? max_new : rows;
    Shape s;
    s.rows_most = n * (q_heads / kv_heads);
    s.splits = few_rows((uint64_t)n * (q_heads / kv_heads)) ? splits_of(seqs, kv_heads, max_len) : 1;
    s.parts = s.splits > 1 ? (size_t)seqs * kv_heads * s.splits * s.rows_most : 0;
    return s;
}

}  // namespace
}  // namespace zkmi

using namespace zkmi;

extern "C" size_t kvcache_attention_workspace_bytes(uint32_t seqs, uint32_t rows, uint32_t max_new, uint32_t q_heads, uint32_t kv_heads,
                                                    uint32_t head_dim, uint32_t max_len) {
    if (!kv_heads || q_heads % kv_heads || !seqs || !rows || !max_new) return 0;
    const Shape s = shape_of(seqs, rows, max_new, q_heads, kv_heads, max_len);
    if (!s.parts) return 0;
    Carver cv(nullptr, 0);
    cv.take(s.parts * head_dim * sizeof(float));
    cv.take(s.parts * sizeof(float2));
    return cv.used();
}

extern "C" int kvcache_attention(const kvcache_i8* cache, const void* q, size_t q_row_stride, size_t q_head_stride, int dtype,
                                 uint32_t q_heads, const kv_seqs* seqs, float scale, uint32_t window, void* out, size_t out_row_stride,
                                 size_t out_head_stride, float* lse, void* ws, size_t ws_bytes, void* stream) {
    if ((dtype != ZK_F16 && dtype != ZK_BF16) || !cache_ok(cache) || !seqs_ok(seqs)) return ZK_E_BADARG;
    if (q_heads == 0 || q_heads % cache->kv_heads || q_heads > 65536 || window >= 0x80000000u || !(scale - scale == 0.0f)) return ZK_E_BADARG;
    if (seqs->rows == 0 || seqs->seqs == 0) return ZK_OK;
    if (!q || !out || !aligned(q, 2) || !aligned(out, 2) || (lse && !aligned(lse, 4))) return ZK_E_BADARG;
    const uint32_t group = q_heads / cache->kv_heads;
    if ((uint64_t)(seqs->max_new < seqs->rows ? seqs->max_new : seqs->rows) * group >= 0x80000000u) return ZK_E_BADARG;
    const Shape sh = shape_of(seqs->seqs, seqs->rows, seqs->max_new, q_heads, cache->kv_heads, seqs->max_len);
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
    a.rows_most = sh.rows_most;
    a.splits = sh.splits;
    if (sh.parts) {
        if (!ws) return ZK_E_BUFSZ;
        Carver cv(ws, ws_bytes);
        a.parts = (float*)cv.take(sh.parts * cache->head_dim * sizeof(float));
        a.parts_ml = (float2*)cv.take(sh.parts * sizeof(float2));
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
