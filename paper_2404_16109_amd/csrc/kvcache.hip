// Appending to, and reading back, the cache of 8-bit keys and values.
//
// A workgroup has one page that new tokens fall into, one head, and either its keys or its values.  It takes the largest
// magnitude of the new values first (as the integer a float's bits are, which also orders infinities and NaN above every
// number), settles the page's exponent, and writes: new codes, and the old ones where the exponent grew.  Multiplying
// by a power of two is exact, so rint(x * 2^-e) is the only rounding of a new code, and rint(c * 2^-shift) of an old one.
//
// Bound by bytes for prompts (pages that begin are read once, others twice, the second time from the L2, and one byte of each
// value is written; the vector ALU is 81% busy then), by the chain of four dependent loads for single tokens.
// Measured: 7 prompts of up to 2048 tokens, 40 heads of 128 (235 MB) 56 us, 4.2 TB/s; a token of each of 32 sequences 4.5 us.  Pages
// of more than kPageInRegs codes, and rows that no wide load takes, are read a second time and transposed by two-byte loads: 88 us
// where the other way takes 56.
#include "kvcache.h"

namespace zkmi {
namespace {

struct Fresh {
    const void* x;
    size_t row_stride, head_stride;
    bool wide;  // 16 values at a time: everything is 16-byte aligned
};

// The smallest e with |x| <= 127 * 2^e, from the bits of |x|.
__device__ __forceinline__ int exponent_for(uint32_t bits) {
    if (bits >= 0x7f800000u) return ZK_EXP_NAN;
    // |x| = f * 2^(E - 127) with 1 <= f < 2, and 127 * 2^e = (127/64) * 2^(e + 6)
    const int e = (int)(bits >> 23) - 133 + ((bits & 0x7fffffu) > 0x7e0000u ? 1 : 0);
    return e < ZK_EXP_MIN ? ZK_EXP_MIN : e > ZK_EXP_MAX ? ZK_EXP_MAX : e;
}

__device__ __forceinline__ float pow2(int e) { return bits_float((uint32_t)(e + 127) << 23); }
__device__ __forceinline__ int code_of(float x, float step) { return (int)fminf(fmaxf(rintf(x * step), -127.0f), 127.0f); }

// Sixteen consecutive values.
template <int DT>
__device__ __forceinline__ void load16(const Fresh& f, size_t at, float (&v)[16]) {
    if (f.wide) {
        const char* p = (const char*)f.x + at * (DT == ZK_F32 ? 4 : 2);
        if constexpr (DT == ZK_F32) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const v4f r = ((const v4f*)p)[i];
#pragma unroll
                for (int e = 0; e < 4; ++e) v[4 * i + e] = r[e];
            }
        } else {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const v4u r = ((const v4u*)p)[i];
#pragma unroll
                for (int e = 0; e < 8; ++e) v[8 * i + e] = half_of<DT>(r[e >> 1], e & 1);
            }
        }
    } else {
#pragma unroll
        for (int e = 0; e < 16; ++e) v[e] = load_one<DT>(f.x, at + e);
    }
}

// Four codes of a word, rounded to a scale 2^shift times as large (shift <= 0).
__device__ __forceinline__ uint32_t rescale4(uint32_t w, float factor) {
    uint32_t r = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) r |= ((uint32_t)(int)rintf((float)(int8_t)(w >> (8 * e)) * factor) & 255u) << (8 * e);
    return r;
}

// Bytes i of four words as a word, i = 0..3.
__device__ __forceinline__ void transpose4(const uint32_t (&w)[4], uint32_t (&out)[4]) {
    const uint32_t a = __builtin_amdgcn_perm(w[1], w[0], 0x05010400u), b = __builtin_amdgcn_perm(w[3], w[2], 0x05010400u);
    const uint32_t c = __builtin_amdgcn_perm(w[1], w[0], 0x07030602u), d = __builtin_amdgcn_perm(w[3], w[2], 0x07030602u);
    out[0] = __builtin_amdgcn_perm(b, a, 0x05040100u);
    out[1] = __builtin_amdgcn_perm(b, a, 0x07060302u);
    out[2] = __builtin_amdgcn_perm(d, c, 0x05040100u);
    out[3] = __builtin_amdgcn_perm(d, c, 0x07060302u);
}

// A page that begins with this call, its 4 x 8 (tokens x dimensions) pieces held in registers from the first look to the
// codes: kPieces to a thread, pages of at most kPageInRegs codes.  Values go through LDS to lie by dimension.
static const int kPieces = 2;
static const uint32_t kPageInRegs = kPieces * kBlock * 32;
template <int DT>
__device__ void append_page(const Fresh& f, size_t x0, size_t row_stride, int hi, uint32_t T, uint32_t d, bool values, int8_t* codes,
                            int8_t* exps, uint32_t* most, char* lds) {
    constexpr int words = DT == ZK_F32 ? 2 : 1;
    const uint32_t tid = threadIdx.x, d8 = d >> 3, pieces = (T >> 2) * d8;
    v4u raw[kPieces][4][words];
    uint32_t amax = 0;
    auto value = [&](int p, int t, int e) -> float {
        if constexpr (DT == ZK_F32) return bits_float(raw[p][t][e >> 2][e & 3]);
        else return half_of<DT>(raw[p][t][0][e >> 1], e & 1);
    };
#pragma unroll
    for (int p = 0; p < kPieces; ++p) {
        const uint32_t i = tid + kBlock * p, c = i % d8 * 8, t0 = i / d8 * 4;
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int w = 0; w < words; ++w) {
                raw[p][t][w] = v4u{0, 0, 0, 0};
                if (i < pieces && (int)t0 + t < hi)
                    raw[p][t][w] = ((const v4u*)((const char*)f.x + (x0 + (size_t)(t0 + t) * row_stride + c) * (DT == ZK_F32 ? 4 : 2)))[w];
            }
    }
#pragma unroll
    for (int p = 0; p < kPieces; ++p)
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const uint32_t a = float_bits(value(p, t, e)) & 0x7fffffffu;
                amax = a > amax ? a : amax;
            }
    amax = wave_max(amax);
    if ((tid & 63) == 0) most[tid >> 6] = amax;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kBlock / 64; ++w) amax = most[w] > amax ? most[w] : amax;
    const int e = exponent_for(amax);
    if (tid == 0) *exps = (int8_t)e;
    const bool fine = e != ZK_EXP_NAN;
    const float step = fine ? pow2(-e) : 0.0f;
    const uint32_t vrow = T + 4;  // in LDS
#pragma unroll
    for (int p = 0; p < kPieces; ++p) {
        const uint32_t i = tid + kBlock * p, c = i % d8 * 8, t0 = i / d8 * 4;
        if (i >= pieces) continue;
        uint32_t w[2][4];  // [half][token]
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                w[half][t] = 0;
#pragma unroll
                for (int k = 0; k < 4; ++k) w[half][t] |= (fine ? (uint32_t)code_of(value(p, t, 4 * half + k), step) & 255u : 0u) << (8 * k);
            }
        if (!values) {
#pragma unroll
            for (int t = 0; t < 4; ++t) *(uint2*)(codes + (size_t)(t0 + t) * d + c) = make_uint2(w[0][t], w[1][t]);
        } else {
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                uint32_t by[4];
                transpose4(w[half], by);
#pragma unroll
                for (int k = 0; k < 4; ++k) *(uint32_t*)(lds + (c + 4 * half + k) * vrow + t0) = by[k];
            }
        }
    }
    if (!values) return;
    __syncthreads();
    const uint32_t t16 = T >> 4;
    for (uint32_t i = tid; i < d * t16; i += kBlock) {
        const uint32_t* at = (const uint32_t*)(lds + i / t16 * vrow + i % t16 * 16);
        ((v4u*)codes)[i] = v4u{at[0], at[1], at[2], at[3]};
    }
}

// PAGES: calls that may fill pages, 256 threads.  page0: of each sequence's pages, the launch's first.
template <int DT, bool PAGES>
__global__ __launch_bounds__(kBlock) void k_append(kvcache_i8 cache, Fresh fk, Fresh fv, kv_seqs s, uint32_t page_log, uint32_t page0) {
    __shared__ uint32_t most[4];
    const uint32_t tid = threadIdx.x, T = 1u << page_log, d = cache.head_dim, H = cache.kv_heads;
    const bool values = blockIdx.y >= H;
    const uint32_t h = values ? blockIdx.y - H : blockIdx.y, b = blockIdx.z;
    const SeqView q = seq_view(s, b, page_log);
    if (!q.ok) {
        if (tid == 0) report(s, ZK_FAULT_LENGTH);
        return;
    }
    const int32_t first = q.len - q.rows, start = first > 0 ? first : 0;
    const int64_t p = (int64_t)(start >> page_log) + page0 + blockIdx.x;
    const int64_t from = p << page_log, to = from + T;
    const int lo = from > start ? 0 : (int)(start - from), hi = (int)((to < q.len ? to : q.len) - from);  // the page's new slots
    if (hi <= lo) return;
    const uint32_t page = (uint32_t)s.table[(size_t)b * s.table_stride + p];
    if (page >= cache.pages) {
        if (tid == 0) report(s, ZK_FAULT_PAGE);
        return;
    }
    const Fresh& f = values ? fv : fk;
    const size_t at_exp = (size_t)page * H + h;
    int8_t* exps = (values ? cache.v_exp : cache.k_exp) + at_exp;
    int8_t* codes = (values ? cache.v : cache.k) + at_exp * T * d;
    const int held = *exps;
    // row of slot t in the call's tensors, its head's first value
    const size_t x0 = (size_t)h * f.head_stride;
    const int64_t row0 = (int64_t)q.row0 + from - first;
    auto at = [&](int t) -> size_t { return (size_t)(row0 + t) * f.row_stride + x0; };

    if constexpr (PAGES) {
        __shared__ uint32_t lds[(kPageInRegs + 4 * 256) / 4];
        if (lo == 0 && hi >= 16 && f.wide && T * d <= kPageInRegs) {
            append_page<DT>(f, (size_t)row0 * f.row_stride + x0, f.row_stride, hi, T, d, values, codes, exps, most, (char*)lds);
            return;
        }
    }
    const uint32_t d16 = d >> 4;
    uint32_t amax = 0;
    for (uint32_t i = tid; i < (uint32_t)(hi - lo) * d16; i += blockDim.x) {
        float v[16];
        load16<DT>(f, at(lo + (int)(i / d16)) + (i % d16) * 16, v);
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const uint32_t a = float_bits(v[e]) & 0x7fffffffu;
            amax = a > amax ? a : amax;
        }
    }
    amax = wave_max(amax);
    if ((tid & 63) == 0) most[tid >> 6] = amax;
    __syncthreads();
    for (uint32_t w = 0; w < blockDim.x >> 6; ++w) amax = most[w] > amax ? most[w] : amax;

    const bool begins = lo == 0;
    const int need = exponent_for(amax);
    const int e = begins ? need : need == ZK_EXP_NAN || held == ZK_EXP_NAN ? ZK_EXP_NAN : need > held ? need : held;
    if (tid == 0) *exps = (int8_t)e;
    const bool fine = e != ZK_EXP_NAN, grows = !begins && fine && e > held;
    const float step = fine ? pow2(-e) : 0.0f, factor = grows ? pow2(held - e) : 1.0f;
    auto code = [&](float x) -> uint32_t { return fine ? (uint32_t)code_of(x, step) & 255u : 0u; };

    if (!values) {
        // [token][head_dim]: pieces of 16 dimensions
        const int t0 = begins || grows ? 0 : lo, t1 = begins || grows ? (int)T : hi;
        for (uint32_t i = tid; i < (uint32_t)(t1 - t0) * d16; i += blockDim.x) {
            const int t = t0 + (int)(i / d16);
            const uint32_t c = (i % d16) * 16;
            v4u* out = (v4u*)(codes + (size_t)t * d + c);
            v4u r = {0, 0, 0, 0};
            if (t >= lo && t < hi) {
                float v[16];
                load16<DT>(f, at(t) + c, v);
#pragma unroll
                for (int k = 0; k < 16; ++k) r[k >> 2] |= code(v[k]) << (8 * (k & 3));
            } else if (!begins) {
                r = *out;
#pragma unroll
                for (int k = 0; k < 4; ++k) r[k] = rescale4(r[k], factor);
            }
            *out = r;
        }
    } else if (!begins && !grows && hi - lo < 16) {
        // [head_dim][token]: a few tokens are single bytes
        for (uint32_t i = tid; i < (uint32_t)(hi - lo) * d; i += blockDim.x) {
            const int t = lo + (int)(i / d);
            const uint32_t c = i % d;
            codes[((size_t)c << page_log) + t] = (int8_t)code(load_one<DT>(f.x, at(t) + c));
        }
    } else {
        // pieces of 16 tokens; neighbouring threads have neighbouring dimensions
        const int r0 = begins || grows ? 0 : lo >> 4, r1 = begins || grows ? (int)(T >> 4) : (hi + 15) >> 4;
        for (uint32_t i = tid; i < (uint32_t)(r1 - r0) * d; i += blockDim.x) {
            const int t0 = (r0 + (int)(i / d)) * 16;
            const uint32_t c = i % d;
            v4u* out = (v4u*)(codes + ((size_t)c << page_log) + t0);
            v4u r = {0, 0, 0, 0};
            if (!begins && (t0 < lo || t0 + 16 > hi)) {
                r = *out;
                if (grows)
#pragma unroll
                    for (int k = 0; k < 4; ++k) r[k] = rescale4(r[k], factor);
            }
#pragma unroll
            for (int k = 0; k < 16; ++k) {
                const int t = t0 + k;
                if (t >= lo && t < hi) {
                    const uint32_t v = code(load_one<DT>(f.x, at(t) + c));
                    r[k >> 2] = (r[k >> 2] & ~(255u << (8 * (k & 3)))) | (v << (8 * (k & 3)));
                }
            }
            *out = r;
        }
    }
}

// A workgroup: one token, and of more tokens than a grid of them has workgroups the next after as many; keys and values, in order
// of head and dimension.
static const uint32_t kReadGrid = 1u << 20;  // a launch ends at 2^32 threads
__global__ __launch_bounds__(kBlock) void k_read(kvcache_i8 cache, const int32_t* pages, uint32_t page_log, size_t tokens, int32_t* k, int32_t* v,
                                                 uint32_t* fault) {
    const uint32_t T = 1u << page_log, d = cache.head_dim, H = cache.kv_heads;
    for (size_t t = blockIdx.x; t < tokens; t += gridDim.x) {
        const uint32_t slot = (uint32_t)t & (T - 1), page = (uint32_t)pages[t >> page_log];
        const bool ok = page < cache.pages;
        if (!ok && threadIdx.x == 0 && fault) atomicOr(fault, (uint32_t)ZK_FAULT_PAGE);
        for (uint32_t i = threadIdx.x; i < H * d; i += kBlock) {
            const uint32_t h = i / d, c = i % d;
            const size_t at = ((size_t)page * H + h) * T * d;
            k[t * H * d + i] = ok ? cache.k[at + (size_t)slot * d + c] : 0;
            v[t * H * d + i] = ok ? cache.v[at + ((size_t)c << page_log) + slot] : 0;
        }
    }
}

template <int DT>
int append(const kvcache_i8& cache, const Fresh& fk, const Fresh& fv, const kv_seqs& s, hipStream_t stream) {
    const uint32_t T = cache.page_tokens, log = (uint32_t)log2_floor(T);
    const uint32_t span = s.max_new < s.rows ? s.max_new : s.rows;
    const uint32_t pages = (uint32_t)(((size_t)T - 1 + span - 1) / T + 1);  // with the first slot the page's last
    // one wavefront has enough to do with a head of a single token; beyond 16 values to each of its lanes, four
    const unsigned threads = (size_t)(span < T ? span : T) * cache.head_dim <= 1024 ? 64 : kBlock;
    auto* kernel = threads == kBlock ? k_append<DT, true> : k_append<DT, false>;
    const uint32_t most = 1u << 20;  // pages: a launch ends at 2^32 threads across
    for (uint32_t page0 = 0; page0 < pages; page0 += most)
        hipLaunchKernelGGL(kernel, dim3(pages - page0 < most ? pages - page0 : most, 2 * cache.kv_heads, s.seqs), dim3(threads), 0, stream, cache, fk,
                           fv, s, log, page0);
    ZK_HIP_TRY(hipGetLastError());
    return ZK_OK;
}

}  // namespace
}  // namespace zkmi

using namespace zkmi;

extern "C" int kvcache_append(const kvcache_i8* cache, const void* k, size_t k_row_stride, size_t k_head_stride, const void* v,
                              size_t v_row_stride, size_t v_head_stride, int dtype, const kv_seqs* seqs, void* stream) {
    const size_t size = dtype_bytes(dtype);
    if (!size || dtype == ZK_I16 || !cache_ok(cache) || !seqs_ok(seqs)) return ZK_E_BADARG;
    if (seqs->rows == 0 || seqs->seqs == 0) return ZK_OK;
    if (!k || !v || !aligned(k, size) || !aligned(v, size)) return ZK_E_BADARG;
    auto fresh = [&](const void* x, size_t rs, size_t hs) {
        return Fresh{x, rs, hs, aligned(x, 16) && rs * size % 16 == 0 && hs * size % 16 == 0};
    };
    const Fresh fk = fresh(k, k_row_stride, k_head_stride), fv = fresh(v, v_row_stride, v_head_stride);
    hipStream_t s = as_stream(stream);
    if (dtype == ZK_F32) return append<ZK_F32>(*cache, fk, fv, *seqs, s);
    if (dtype == ZK_F16) return append<ZK_F16>(*cache, fk, fv, *seqs, s);
    return append<ZK_BF16>(*cache, fk, fv, *seqs, s);
}

extern "C" int kvcache_read(const kvcache_i8* cache, const int32_t* pages, size_t tokens, int32_t* k_codes, int32_t* v_codes,
                            uint32_t* fault, void* stream) {
    if (!cache_ok(cache) || tokens >= 0x80000000u) return ZK_E_BADARG;
    if (tokens == 0) return ZK_OK;
    if (!pages || !k_codes || !v_codes || !aligned(pages, 4) || !aligned(k_codes, 4) || !aligned(v_codes, 4) || (fault && !aligned(fault, 4)))
        return ZK_E_BADARG;
    hipLaunchKernelGGL(k_read, dim3(tokens < kReadGrid ? (unsigned)tokens : kReadGrid), dim3(kBlock), 0, as_stream(stream), *cache, pages,
                       (uint32_t)log2_floor(cache->page_tokens), tokens, k_codes, v_codes, fault);
    ZK_HIP_TRY(hipGetLastError());
    return ZK_OK;
}
