// Log probabilities of given tokens, with rank, entropy and the first alternatives.
//
// With m the largest of a row's logits x_i, l = sum exp(x_i - m) and t = sum exp(x_i - m) (x_i - m):
//   lse = m + log l,   log p_i = x_i - lse,   -sum p log p = log l - t / l,
// so one pass over the row is enough.  A row is cut into segments; a workgroup holds its segment in registers (32 values
// to a thread), takes the largest first and then the sums relative to it, and leaves (m, l, t), the count for the rank and
// its `top` first values; a wavefront per row joins the segments.
//
// The first `top` of a segment: a wavefront has 64 largest-of-a-thread; the top-th largest of those is a bound that at
// least `top` of its values reach, and so is the largest of the four wavefronts' bounds.  The values that reach it,
// usually about as many as asked for, are put in order by counting, for each, those that come before it.  Order is that
// of 64-bit keys (value, then lower index).  Where too many reach the bound (ties, rows that allow less than `top`
// tokens, NaN) the keys are taken out one after the other instead.
//
// Bound by the bytes of the logits.
#include "serve_dev.h"

namespace zkmi {
namespace {

static const int kPerThread = 32;
static const uint32_t kCandidates = 1024;

struct Part {
    float m, l, t;
    uint32_t before;
};

// Order of the values, larger first: NaN, +inf, ..., -inf; -0 and +0 are equal.
__device__ __forceinline__ uint32_t order_of(float x) {
    const uint32_t b = float_bits(x + 0.0f);
    return x != x ? 0xffffffffu : b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t order) {
    return order == 0xffffffffu ? __builtin_nanf("") : bits_float(order & 0x80000000u ? order ^ 0x80000000u : ~order);
}
__device__ __forceinline__ uint64_t key_of(float x, uint32_t index) { return ((uint64_t)order_of(x) << 32) | (uint32_t)~index; }

__device__ __forceinline__ uint64_t wave_max(uint64_t k) {
#pragma unroll
    for (int o = 32; o; o >>= 1) {
        const uint64_t other = __shfl_xor(k, o);
        k = other > k ? other : k;
    }
    return k;
}
__device__ __forceinline__ float wave_max(float x) {
#pragma unroll
    for (int o = 32; o; o >>= 1) x = fmaxf(x, __shfl_xor(x, o));
    return x;
}
__device__ __forceinline__ float wave_add(float x) {
#pragma unroll
    for (int o = 32; o; o >>= 1) x += __shfl_xor(x, o);
    return x;
}

// exp of a difference to a maximum.
__device__ __forceinline__ float exp_of(float z) { return __builtin_amdgcn_exp2f(z * 1.44269504088896341f); }

struct Results {
    logprobs_out out;
    const int32_t* targets;
    uint32_t top;
};

// What a row's (m, l, t) say; one thread.
__device__ void row_results(const Results& r, size_t row, const Part& p, uint32_t vocab, float xt) {
    const float base = fabsf(p.m) == kInf ? 0.0f : p.m;
    const float logl = logf(p.l);
    const float lse = base + logl;
    const bool none = p.l == 0.0f;
    if (r.out.lse) r.out.lse[row] = lse;
    if (r.out.entropy) r.out.entropy[row] = none ? 0.0f : logl - p.t / p.l;
    if (r.targets) {
        const bool given = (uint32_t)r.targets[row] < vocab;
        r.out.target[row] = !given ? __builtin_nanf("") : none ? -kInf : xt - lse;
        r.out.rank[row] = given ? (int32_t)p.before : -1;
    }
}
__device__ __forceinline__ void top_result(const Results& r, size_t row, uint32_t place, uint64_t key, float m, float l) {
    const float base = fabsf(m) == kInf ? 0.0f : m;
    r.out.top_ids[row * r.top + place] = (int32_t)~(uint32_t)key;
    r.out.top[row * r.top + place] = l == 0.0f ? -kInf : value_of((uint32_t)(key >> 32)) - (base + logf(l));
}

// Workgroup (segment, row) of 256 threads.  A row is read in chunks of 16 bytes that are aligned whatever the row's
// address: chunk c holds the values c * EPC - skew ...  Chunks that lie partly outside the row are read value by value.
template <int DT>
__global__ __launch_bounds__(kBlock) void k_logprobs_part(const void* logits, size_t row_stride, uint32_t vocab, uint32_t chunks_each,
                                                          Results res, Part* parts, uint64_t* keys) {
    constexpr int EPC = DT == ZK_F32 ? 4 : 8;  // values of a chunk
    constexpr int CPT = kPerThread / EPC;      // chunks of a thread
    __shared__ uint64_t cand[kCandidates];
    __shared__ float sh_m[4], sh_l[4], sh_t[4], sh_b[4];
    __shared__ uint32_t sh_n[4], found;
    const size_t row = blockIdx.y;
    const uint32_t seg = blockIdx.x, nseg = gridDim.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const char* at = (const char*)logits + row * row_stride * (DT == ZK_F32 ? 4 : 2);
    const uint32_t skew = (uint32_t)((uintptr_t)at & 15) / (16 / EPC);
    const char* chunk0 = at - skew * (16 / EPC);
    const uint32_t nchunks = (vocab + skew + EPC - 1) / EPC;
    const uint32_t c0 = seg * chunks_each, c1 = c0 + chunks_each < nchunks ? c0 + chunks_each : nchunks;
    const uint32_t target = res.targets ? (uint32_t)res.targets[row] : ~0u;
    const bool given = target < vocab;
    const float xt = given ? load_one<DT>(at, target) : 0.0f;
    if (tid == 0) found = 0;

    v4u raw[CPT];
    const uint32_t fill = DT == ZK_F32 ? 0xff800000u : DT == ZK_BF16 ? 0xff80ff80u : 0xfc00fc00u;  // -inf
#pragma unroll
    for (int i = 0; i < CPT; ++i) {
        const uint32_t c = c0 + tid + i * kBlock;
        raw[i] = v4u{fill, fill, fill, fill};
        if (c < c1) {
            const int64_t first = (int64_t)c * EPC - skew;
            if (first >= 0 && first + EPC <= vocab) {
                raw[i] = __builtin_nontemporal_load((const v4u*)(chunk0 + (size_t)c * 16));
            } else {
#pragma unroll
                for (int e = 0; e < EPC; ++e) {
                    if (first + e < 0 || first + e >= vocab) continue;
                    if constexpr (DT == ZK_F32) {
                        raw[i][e] = ((const uint32_t*)at)[first + e];
                    } else {
                        const uint32_t h = ((const uint16_t*)at)[first + e];
                        raw[i][e >> 1] = e & 1 ? (raw[i][e >> 1] & 0xffffu) | (h << 16) : (raw[i][e >> 1] & 0xffff0000u) | h;
                    }
                }
            }
        }
    }
    auto value = [&](int i, int e) -> float {
        if constexpr (DT == ZK_F32) return bits_float(raw[i][e]);
        else return half_of<DT>(raw[i][e >> 1], e & 1);
    };
    // index of a chunk's first value; chunks of another segment (all -inf here) get one behind every token
    auto index = [&](int i) -> uint32_t {
        const uint32_t c = c0 + tid + i * kBlock;
        return c < c1 ? c * EPC - skew : 0x80000000u;
    };

    float mine = -kInf;
#pragma unroll
    for (int i = 0; i < CPT; ++i)
#pragma unroll
        for (int e = 0; e < EPC; ++e) mine = fmaxf(mine, value(i, e));
    const float wm = wave_max(mine);
    // the bound: the largest v that `top` lanes reach, found bit by bit in the order of the values
    float bound = -kInf;
    if (res.top) {
        const uint32_t o = order_of(mine);
        uint32_t b = 0;
        for (int bit = 31; bit >= 0; --bit) {
            const uint32_t with = b | (1u << bit);
            if ((uint32_t)__builtin_popcountll(__ballot(o >= with)) >= res.top) b = with;
        }
        bound = value_of(b);
    }
    if (lane == 0) {
        sh_m[wave] = wm;
        sh_b[wave] = bound;
    }
    __syncthreads();
    const float m = fmaxf(fmaxf(sh_m[0], sh_m[1]), fmaxf(sh_m[2], sh_m[3]));
    bound = fmaxf(fmaxf(sh_b[0], sh_b[1]), fmaxf(sh_b[2], sh_b[3]));
    const float base = fabsf(m) == kInf ? 0.0f : m;

    // Four sums side by side; 32 values each at most, then lanes and wavefronts pairwise: all in 32 bits.
    float l = 0.0f, t = 0.0f;
    uint32_t before = 0;
#pragma unroll
    for (int i = 0; i < CPT; ++i) {
        const uint32_t first = index(i);
#pragma unroll
        for (int e = 0; e < EPC; ++e) {
            const float x = value(i, e), z = x - base, p = exp_of(z);
            l += p;
            t += p * fmaxf(z, -1000.0f);  // p = 0 there: -inf must not make 0 * inf
            const uint32_t at_index = first + e;
            before += __builtin_popcountll(__ballot(x > xt || (x == xt && at_index < target)));
            if (res.top && x >= bound && at_index < vocab) {
                const uint32_t n = atomicAdd(&found, 1u);
                if (n < kCandidates) cand[n] = key_of(x, at_index);
            }
        }
    }
    // values before the row's start have indexes that wrap round: never below the target
    l = wave_add(l);
    t = wave_add(t);
    if (lane == 0) {
        sh_l[wave] = l;
        sh_t[wave] = t;
        sh_n[wave] = before;
    }
    __syncthreads();
    Part p;
    p.m = m;
    p.l = (sh_l[0] + sh_l[1]) + (sh_l[2] + sh_l[3]);
    p.t = (sh_t[0] + sh_t[1]) + (sh_t[2] + sh_t[3]);
    p.before = given ? sh_n[0] + sh_n[1] + sh_n[2] + sh_n[3] : 0;
    if (tid == 0) {
        if (nseg == 1) row_results(res, row, p, vocab, xt);
        else parts[row * nseg + seg] = p;
    }
    if (res.top == 0) return;
    uint64_t* mykeys = keys ? keys + (row * nseg + seg) * res.top : nullptr;
    auto put = [&](uint32_t place, uint64_t key) {
        if (nseg == 1) top_result(res, row, place, key, p.m, p.l);
        else mykeys[place] = key;
    };
    const uint32_t n = found;
    if (n <= kCandidates && p.l == p.l && n >= res.top) {
        for (uint32_t c = tid; c < n; c += kBlock) {
            const uint64_t key = cand[c];
            uint32_t place = 0;
            for (uint32_t o = 0; o < n; ++o) place += cand[o] > key;
            if (place < res.top) put(place, key);
        }
        return;
    }
    uint64_t last = 0;
    for (uint32_t place = 0; place < res.top; ++place) {
        uint64_t best = 0;
#pragma unroll
        for (int i = 0; i < CPT; ++i)
#pragma unroll
            for (int e = 0; e < EPC; ++e) {
                const uint32_t at_index = index(i) + e;
                const uint64_t key = key_of(value(i, e), at_index);
                if (at_index < vocab && (place == 0 || key < last) && key > best) best = key;
            }
        best = wave_max(best);
        __syncthreads();
        if (lane == 0) cand[wave] = best;
        __syncthreads();
        for (int w = 0; w < 4; ++w) best = cand[w] > best ? cand[w] : best;
        if (tid == 0) put(place, best);  // 0: the segment has no more
        last = best;
        __syncthreads();
    }
}

// A wavefront per row joins its segments: lane i has segments i and 64 + i.
template <int DT>
__global__ __launch_bounds__(kBlock) void k_logprobs_join(const void* logits, size_t row_stride, uint32_t vocab, uint32_t nseg, size_t rows,
                                                          Results res, const Part* parts, const uint64_t* keys) {
    const size_t row = (size_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    const uint32_t lane = threadIdx.x & 63;
    if (row >= rows) return;
    Part p[2];
    uint64_t head[2] = {0, 0};
    uint32_t next[2] = {0, 0};
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const uint32_t seg = lane + 64 * i;
        p[i] = {-kInf, 0.0f, 0.0f, 0};
        if (seg < nseg) {
            p[i] = parts[row * nseg + seg];
            if (res.top) head[i] = keys[(row * nseg + seg) * res.top];
        }
    }
    Part all;
    all.m = wave_max(fmaxf(p[0].m, p[1].m));
    const float base = fabsf(all.m) == kInf ? 0.0f : all.m;
    float l = 0.0f, t = 0.0f;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        // a segment of -inf alone has l = t = 0; what an infinity is the maximum of was summed relative to 0
        // (and a segment far below the maximum, by as much as the type's lowest value, must not make 0 * inf)
        const float own = fabsf(p[i].m) == kInf ? 0.0f : p[i].m, d = fmaxf(own - base, -1000.0f), f = p[i].l == 0.0f ? 0.0f : exp_of(d);
        l += p[i].l * f;
        t += p[i].l == 0.0f ? 0.0f : f * (p[i].t + p[i].l * d);
    }
    all.l = wave_add(l);
    all.t = wave_add(t);
    uint32_t before = p[0].before + p[1].before;
#pragma unroll
    for (int o = 32; o; o >>= 1) before += __shfl_xor(before, o);
    all.before = before;
    if (lane == 0) {
        const uint32_t target = res.targets ? (uint32_t)res.targets[row] : ~0u;
        const float xt = target < vocab ? load_one<DT>((const char*)logits + row * row_stride * (DT == ZK_F32 ? 4 : 2), target) : 0.0f;
        row_results(res, row, all, vocab, xt);
    }
    for (uint32_t place = 0; place < res.top; ++place) {
        const uint64_t best = wave_max(head[0] > head[1] ? head[0] : head[1]);
        if (lane == 0) top_result(res, row, place, best, all.m, all.l);
#pragma unroll
        for (int i = 0; i < 2; ++i)
            if (best && head[i] == best) head[i] = ++next[i] < res.top ? keys[(row * nseg + lane + 64 * i) * res.top + next[i]] : 0;
    }
}

struct Plan {
    uint32_t nseg, chunks_each;
};
// Few rows are cut finer than the registers need, until there are some 512 workgroups or a thread has one chunk.
Plan plan_of(size_t rows, size_t vocab, int dtype) {
    const uint32_t epc = dtype == ZK_F32 ? 4 : 8, cpt = kPerThread / epc;
    const uint32_t chunks = (uint32_t)(vocab + epc - 1 + epc - 1) / epc;  // with the most skew
    const uint32_t need = (uint32_t)div_up(chunks, (size_t)kBlock * cpt), most = (uint32_t)div_up(chunks, kBlock);
    uint32_t nseg = need;
    if (rows * nseg < 512) nseg = (uint32_t)div_up(512, rows);
    if (nseg > most) nseg = most;
    if (nseg > 64) nseg = 64;
    if (nseg < need) nseg = need;
    Plan p;
    p.chunks_each = (uint32_t)div_up(chunks, nseg);
    p.nseg = (uint32_t)div_up(chunks, p.chunks_each);
    return p;
}

bool shape_ok(size_t rows, size_t vocab, uint32_t top) {
    return vocab >= 1 && vocab <= ((size_t)1 << 19) && top <= LOGPROBS_MAX_TOP && top <= vocab && rows <= 0xffffffffu;
}

template <int DT>
int run(const void* logits, size_t row_stride, size_t rows, uint32_t vocab, const Results& res, Plan plan, Part* parts, uint64_t* keys,
        hipStream_t stream) {
    // the grid's second dimension ends at 65535
    for (size_t r0 = 0; r0 < rows; r0 += 65535) {
        const size_t n = rows - r0 < 65535 ? rows - r0 : 65535;
        Results r = res;
        if (r.targets) {
            r.targets += r0;
            r.out.target += r0;
            r.out.rank += r0;
        }
        if (r.out.lse) r.out.lse += r0;
        if (r.out.entropy) r.out.entropy += r0;
        if (r.top) {
            r.out.top_ids += r0 * r.top;
            r.out.top += r0 * r.top;
        }
        const char* at = (const char*)logits + r0 * row_stride * (DT == ZK_F32 ? 4 : 2);
        hipLaunchKernelGGL((k_logprobs_part<DT>), dim3(plan.nseg, (unsigned)n), dim3(kBlock), 0, stream, at, row_stride, vocab,
                           plan.chunks_each, r, parts, keys);
        if (plan.nseg > 1)
            hipLaunchKernelGGL((k_logprobs_join<DT>), dim3((unsigned)div_up(n, 4)), dim3(kBlock), 0, stream, at, row_stride, vocab,
                               plan.nseg, n, r, parts, keys);
    }
    ZK_HIP_TRY(hipGetLastError());
    return ZK_OK;
}

}  // namespace
}  // namespace zkmi

using namespace zkmi;

extern "C" size_t logprobs_workspace_bytes(size_t rows, size_t vocab, uint32_t top) {
    if (!shape_ok(rows, vocab, top) || rows == 0) return 0;
    // the type is not known here: 32-bit logits have the most segments where the registers decide, and few rows the same number
    size_t most = 0;
    for (int dtype : {ZK_F32, ZK_BF16}) {
        const Plan p = plan_of(rows, vocab, dtype);
        const size_t n = (rows < 65535 ? rows : 65535) * p.nseg;
        Carver cv(nullptr, 0);
        cv.take(n * sizeof(Part));
        cv.take(n * top * sizeof(uint64_t));
        if (p.nseg > 1 && cv.used() > most) most = cv.used();
    }
    return most;
}

extern "C" int logprobs(const void* logits, size_t row_stride, int dtype, size_t rows, size_t vocab, const int32_t* targets,
                        uint32_t top, const logprobs_out* out, void* ws, size_t ws_bytes, void* stream) {
    const size_t size = dtype_bytes(dtype);
    if (!size || dtype == ZK_I16 || !out || !shape_ok(rows, vocab, top) || (rows > 1 && row_stride < vocab)) return ZK_E_BADARG;
    if (rows == 0) return ZK_OK;
    if (!logits || !aligned(logits, size)) return ZK_E_BADARG;
    if (targets && (!out->target || !out->rank)) return ZK_E_BADARG;
    if (top && (!out->top_ids || !out->top)) return ZK_E_BADARG;
    const Plan plan = plan_of(rows, vocab, dtype);
    Part* parts = nullptr;
    uint64_t* keys = nullptr;
    if (plan.nseg > 1) {
        const size_t n = (rows < 65535 ? rows : 65535) * plan.nseg;
        if (!ws) return ZK_E_BUFSZ;
        Carver cv(ws, ws_bytes);
        parts = (Part*)cv.take(n * sizeof(Part));
        keys = (uint64_t*)cv.take(n * top * sizeof(uint64_t));
        if (cv.overflow() || !parts || (top && !keys)) return ZK_E_BUFSZ;
    }
    const Results res = {*out, targets, top};
    hipStream_t s = as_stream(stream);
    if (dtype == ZK_F32) return run<ZK_F32>(logits, row_stride, rows, (uint32_t)vocab, res, plan, parts, keys, s);
    if (dtype == ZK_F16) return run<ZK_F16>(logits, row_stride, rows, (uint32_t)vocab, res, plan, parts, keys, s);
    return run<ZK_BF16>(logits, row_stride, rows, (uint32_t)vocab, res, plan, parts, keys, s);
}
