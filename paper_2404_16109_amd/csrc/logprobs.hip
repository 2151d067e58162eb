// Log probabilities of given tokens, with rank, entropy and the first alternatives.
//
// With m the largest of a row's logits x_i, l = sum exp(x_i - m) and t = sum exp(x_i - m) (x_i - m):
//   lse = m + log l,   log p_i = (x_i - m) - log l,   -sum p log p = log l - t / l,
// so one pass over the row is enough (and what all logits have in common costs log p no bits).  A row is cut into segments; a
// workgroup holds its segment in registers (128 bytes to a thread), takes the largest first and then the sums relative to it, and
// leaves (m, l, t), the count for the rank and its `top` first values; a wavefront per row joins the segments.
//
// The first `top` of a segment: of W wavefronts each finds, among its 64 largest-of-a-thread, the (top / W)-th largest; at
// least `top` values reach the smallest of these bounds.  The values that reach it,
// usually not many more than asked for, are put in order by counting, for each, those that come before it.  Order is that
// of 64-bit keys (value, then lower index).  Where too many reach the bound (ties, rows that allow less than `top`
// tokens, NaN) the keys are taken out one after the other instead.
//
// Bound by the vector ALU, 91% busy (31 instructions a value with 20 alternatives of 32-bit logits), the more so for 16-bit ones, of
// half the bytes.  Measured: 2048 rows of 50257 floats, 20 alternatives (412 MB) 112 us, 3.7 TB/s (a copy: 4.8), but 550 where all
// but 50 of a row's tokens are -inf, and the keys are taken out one after the other; 4096 rows of 32001 bf16 106 us with 5
// alternatives, 81 without; 8 rows of 32001, one launch, 8.4 us, the latency of a dozen dependent steps.
#include "serve_dev.h"

namespace zkmi {
namespace {

static const uint32_t kCandidates = 1024;
static const size_t kManyRows = 128;

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

__device__ __forceinline__ uint64_t key_max(uint64_t k) {
#pragma unroll
    for (int o = 32; o; o >>= 1) {
        const uint64_t other = __shfl_xor(k, o);
        k = other > k ? other : k;
    }
    return k;
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
    const bool none = p.l == 0.0f;
    if (r.out.lse) r.out.lse[row] = base + logl;
    if (r.out.entropy) r.out.entropy[row] = none ? 0.0f : logl - p.t / p.l;
    if (r.targets) {
        const bool given = (uint32_t)r.targets[row] < vocab;
        r.out.target[row] = !given ? __builtin_nanf("") : none ? -kInf : (xt - base) - logl;
        r.out.rank[row] = given ? (int32_t)p.before : -1;
    }
}
__device__ __forceinline__ void top_result(const Results& r, size_t row, uint32_t place, uint64_t key, float m, float l) {
    const float base = fabsf(m) == kInf ? 0.0f : m;
    r.out.top_ids[row * r.top + place] = (int32_t)~(uint32_t)key;
    r.out.top[row * r.top + place] = l == 0.0f ? -kInf : (value_of((uint32_t)(key >> 32)) - base) - logf(l);
}

// Workgroup (segment, row); CPT: chunks of a thread.  A row is read in chunks of 16 bytes that are aligned whatever the row's address: chunk c holds
// the values c * EPC - skew ...  Chunks that lie partly outside the row are read value by value.
template <int DT, int THREADS, int CPT>
__global__ __launch_bounds__(THREADS) void k_logprobs_part(const void* logits, size_t row_stride, uint32_t vocab, uint32_t chunks_each,
                                                           Results res, Part* parts, uint64_t* keys) {
    constexpr int EPC = DT == ZK_F32 ? 4 : 8;  // values of a chunk
    constexpr int W = THREADS / 64;
    __shared__ uint64_t cand[kCandidates];
    __shared__ float sh_m[W], sh_l[W], sh_t[W], sh_b[W];
    __shared__ uint32_t sh_n[W], found;
    const size_t row = blockIdx.y;
    const uint32_t seg = blockIdx.x, nseg = gridDim.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const char* at = (const char*)logits + row * row_stride * (DT == ZK_F32 ? 4 : 2);
    const uint32_t skew = (uint32_t)((uintptr_t)at & 15) / (16 / EPC);
    const char* chunk0 = at - skew * (16 / EPC);
    const uint32_t nchunks = (vocab + skew + EPC - 1) / EPC;
    const uint32_t c0 = seg * chunks_each, c1 = c0 + chunks_each < nchunks ? c0 + chunks_each : nchunks;
    if (tid == 0) found = 0;

    v4u raw[CPT];
    const uint32_t fill = DT == ZK_F32 ? 0xff800000u : DT == ZK_BF16 ? 0xff80ff80u : 0xfc00fc00u;  // -inf
#pragma unroll
    for (int i = 0; i < CPT; ++i) {
        const uint32_t c = c0 + tid + i * THREADS;
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
    // the token asked for, while the row is on its way
    const uint32_t target = res.targets ? (uint32_t)res.targets[row] : ~0u;
    const bool given = target < vocab;
    const float xt = given ? load_one<DT>(at, target) : 0.0f;
    auto value = [&](int i, int e) -> float {
        if constexpr (DT == ZK_F32) return bits_float(raw[i][e]);
        else return half_of<DT>(raw[i][e >> 1], e & 1);
    };
    // index of a chunk's first value; chunks of another segment (all -inf here) get one behind every token.  Values before
    // the row's start have indexes that wrap round.
    auto index = [&](int i) -> uint32_t {
        const uint32_t c = c0 + tid + i * THREADS;
        return c < c1 ? c * EPC - skew : 0x80000000u;
    };

    float top[CPT], mine = -kInf;  // the largest of each chunk
#pragma unroll
    for (int i = 0; i < CPT; ++i) {
        top[i] = value(i, 0);
#pragma unroll
        for (int e = 1; e < EPC; ++e) top[i] = fmaxf(top[i], value(i, e));
        mine = fmaxf(mine, top[i]);
    }
    const float wm = wave_max(mine);
    // A bound that at least `top` values reach: each wavefront's `share`-th largest of its lanes', found bit by bit in the order
    // of the values (the upper half of the bits will do: what is left out makes it lower), and of those the `of`-th largest.
    const uint32_t share = (res.top + W - 1) / W, of = share ? (res.top + share - 1) / share : 0;
    float bound = -kInf;
    if (res.top) {
        const uint32_t o = order_of(mine);
        uint32_t b = 0;
        for (int bit = 31; bit >= 16; --bit) {
            const uint32_t with = b | (1u << bit);
            if ((uint32_t)__builtin_popcountll(__ballot(o >= with)) >= share) b = with;
        }
        bound = value_of(b);
    }
    if (lane == 0) {
        sh_m[wave] = wm;
        sh_b[wave] = bound;
    }
    __syncthreads();
    float m = sh_m[0];
#pragma unroll
    for (int w = 1; w < W; ++w) m = fmaxf(m, sh_m[w]);
    if (res.top) {
        const float b = sh_b[lane & (W - 1)];
        uint32_t above = 0;
#pragma unroll
        for (int w = 0; w < W; ++w) above += sh_b[w] > b || (sh_b[w] == b && w < (int)lane) ? 1 : 0;
        const uint64_t it = __ballot(lane < W && above == of - 1);  // one lane, unless a bound is no number
        bound = it ? bits_float((uint32_t)__builtin_amdgcn_readlane((int)float_bits(b), __builtin_ctzll(it))) : -kInf;
    }
    const float base = fabsf(m) == kInf ? 0.0f : m;

    // 32 or 64 values each at most, then lanes and wavefronts: all in 32 bits.  In the chunks before the target's an equal value
    // comes before it: those are compared with the next smaller number.
    const bool lowest = xt == -kInf;  // nothing is below it: its equals are counted apart
    const float below = xt > 0.0f ? bits_float(float_bits(xt) - 1) : lowest ? xt : xt < 0.0f ? bits_float(float_bits(xt) + 1) : -1.4e-45f;
    float l = 0.0f, t = 0.0f;
    uint32_t before = 0;
#pragma unroll
    for (int i = 0; i < CPT; ++i) {
        const uint32_t first = index(i);
        const float limit = first + EPC <= target ? below : xt;
#pragma unroll
        for (int e = 0; e < EPC; ++e) {
            const float x = value(i, e), z = x - base, p = exp_of(z);
            l += p;
            t += p * fmaxf(z, -1000.0f);  // p = 0 there: -inf must not make 0 * inf
            before += x > limit ? 1 : 0;
        }
    }
#pragma unroll
    for (int i = 0; i < CPT; ++i) {
        const uint32_t first = index(i);
        if (lowest || ((int32_t)first <= (int32_t)target && (int32_t)target < (int32_t)(first + EPC)))
#pragma unroll
            for (int e = 0; e < EPC; ++e) before += value(i, e) == xt && first + e < target && (lowest || first + EPC > target) ? 1 : 0;
        if (res.top && top[i] >= bound)
#pragma unroll
            for (int e = 0; e < EPC; ++e) {
                if (!(value(i, e) >= bound) || first + e >= vocab) continue;
                const uint32_t n = atomicAdd(&found, 1u);
                if (n < kCandidates) cand[n] = key_of(value(i, e), first + e);
            }
    }
    l = wave_add(l);
    t = wave_add(t);
    before = wave_add(before);
    if (lane == 0) {
        sh_l[wave] = l;
        sh_t[wave] = t;
        sh_n[wave] = before;
    }
    __syncthreads();
    Part p = {m, 0.0f, 0.0f, 0};
#pragma unroll
    for (int w = 0; w < W; ++w) {
        p.l += sh_l[w];
        p.t += sh_t[w];
        p.before += sh_n[w];
    }
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
        for (uint32_t c = tid; c < n; c += THREADS) {
            const uint64_t key = cand[c];
            uint32_t place = 0;
#pragma unroll 4
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
        best = key_max(best);
        __syncthreads();
        if (lane == 0) cand[wave] = best;
        __syncthreads();
        for (int w = 0; w < W; ++w) best = cand[w] > best ? cand[w] : best;
        if (tid == 0) put(place, best);  // 0: the segment has no more
        last = best;
        __syncthreads();
    }
}

// A wavefront (and workgroup) per row joins its segments: lane i has segments i and 64 + i.
static const uint32_t kMostKeys = 65 * LOGPROBS_MAX_TOP;
template <int DT>
__global__ __launch_bounds__(64) void k_logprobs_join(const void* logits, size_t row_stride, uint32_t vocab, uint32_t nseg, Results res,
                                                      const Part* parts, const uint64_t* keys) {
    __shared__ uint64_t all_keys[kMostKeys];
    const size_t row = blockIdx.x;
    const uint32_t lane = threadIdx.x, n = nseg * res.top;
    Part p[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) p[i] = lane + 64 * i < nseg ? parts[row * nseg + lane + 64 * i] : Part{-kInf, 0.0f, 0.0f, 0};
    for (uint32_t i = lane; i < n; i += 64) all_keys[i] = keys[row * n + i];
    const uint32_t target = res.targets ? (uint32_t)res.targets[row] : ~0u;
    const float xt = target < vocab ? load_one<DT>((const char*)logits + row * row_stride * (DT == ZK_F32 ? 4 : 2), target) : 0.0f;
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
    all.before = wave_add(p[0].before + p[1].before);
    if (lane == 0) row_results(res, row, all, vocab, xt);
    __syncthreads();
    if (n <= 320) {
        // each key's place: how many come before it (keys that stand for nothing are all 0, behind every other)
        for (uint32_t i = lane; i < n; i += 64) {
            const uint64_t key = all_keys[i];
            uint32_t place = 0;
#pragma unroll 4
            for (uint32_t o = 0; o < n; ++o) place += all_keys[o] > key;
            if (key && place < res.top) top_result(res, row, place, key, all.m, all.l);
        }
        return;
    }
    uint32_t next[2] = {0, 0};
    uint64_t head[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) head[i] = lane + 64 * i < nseg ? all_keys[(lane + 64 * i) * res.top] : 0;
    for (uint32_t place = 0; place < res.top; ++place) {
        const uint64_t best = key_max(head[0] > head[1] ? head[0] : head[1]);
        if (lane == 0) top_result(res, row, place, best, all.m, all.l);
#pragma unroll
        for (int i = 0; i < 2; ++i)
            if (best && head[i] == best) head[i] = ++next[i] < res.top ? all_keys[(lane + 64 * i) * res.top + next[i]] : 0;
    }
}

// Workgroups of 1024 threads for few rows: a vocabulary of 2^15 is then one segment, and nothing has to be joined.  Of 256 for
// many: several of them to a CU, so that some load while others compute.
struct Plan {
    uint32_t threads, chunks_most, nseg, chunks_each;
};
Plan plan_of(size_t rows, size_t vocab, int dtype) {
    const uint32_t epc = dtype == ZK_F32 ? 4 : 8;
    const uint32_t chunks = (uint32_t)(vocab + epc - 1 + epc - 1) / epc;  // with the most skew
    Plan p;
    p.threads = rows < kManyRows && chunks > 1024 ? 1024 : 256;
    p.chunks_most = p.threads == 1024 && chunks <= 4096 ? 4 : 8;
    p.nseg = (uint32_t)div_up(chunks, p.threads * p.chunks_most);
    p.chunks_each = (uint32_t)div_up(chunks, p.nseg);
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
        auto* part = plan.threads == 256 ? k_logprobs_part<DT, 256, 8> : plan.chunks_most == 4 ? k_logprobs_part<DT, 1024, 4> : k_logprobs_part<DT, 1024, 8>;
        hipLaunchKernelGGL(part, dim3(plan.nseg, (unsigned)n), dim3(plan.threads), 0, stream, at, row_stride, vocab, plan.chunks_each, r, parts,
                           keys);
        if (plan.nseg > 1)
            hipLaunchKernelGGL((k_logprobs_join<DT>), dim3((unsigned)n), dim3(64), 0, stream, at, row_stride, vocab, plan.nseg, r, parts, keys);
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
