// What stands between two blocks of a layer, and activations as 8-bit codes.
//
//   t = norm(z) * post_gain + post_bias, r = alpha x + gate t, h = norm(r) * gain + bias; h as it is or as codes with a scale.
//
// One workgroup has a row and keeps it in registers: every tensor is read once and written once, which is what bounds the
// call.  Statistics are sums in 64 bits (at the rate of 32 here) and are rounded to 32 bits once; from there on every step is one
// operation of 32 bits with its own rounding, so nothing is contracted below: the codes are the integers of a proof, and whoever
// computes the definition gets the same ones.  The definition's sums are exact; those here are rounded in an order that the spread of a row
// over threads decides (its width, how many rows there are, addresses).  So a statistic is looked at before it is used: where roundings might
// have moved it over the middle between two floats, its row is added up again without any (Ziv's test).
//
// Measured: 8192 rows of 5120 bf16 through two norms and a gate to codes (378 MB) 88 us, 4.3 TB/s where a copy reaches 5.1, the vector
// ALU 61% busy (3 us of it for the look at statistics); 777 rows of 4097 floats, which no 16-byte load takes, 14.9 us, 3.4 TB/s; 4096 of 5120 floats, two
// norms and a gate to codes (357 MB), 79 us, 4.5 TB/s; 1024 of 20000 bf16 in LDS 78 us, 1.8 TB/s; codes of 8192 x 13824 f16 59 us, 5.8 TB/s (part of it
// stays in the last cache); one row 3.8 us in a graph, latency, where a launch of nothing is 1.7.
// A row whose mean is added up again takes 1.7 us more: layer norms of 8192 x 5120 bf16, of which one in 40 is, 46 us (42 if none were looked at), 4096 of
// 5120 floats that were centred before, of which all are, 53 (35).
#include "serve_dev.h"

#pragma clang fp contract(off)

namespace zkmi {
namespace {

static const uint32_t kMostDim = 32768;   // of a row in registers: 1024 threads of 32 elements
static const uint32_t kMostThreads = 1024;
static const float kLeast = 0x1p-100f;    // rows whose largest magnitude is below it are zeros: 127 / amax has to be a number

struct NormArgs {
    block_norm_args a;
    int dtype;
    uint32_t dim;
    size_t rows;
};
// A launch holds fewer than 2^32 threads in a direction: workgroups of many rows lie in two.
static const size_t kRowsAcross = (size_t)1 << 20;
dim3 grid_of(size_t rows) { return rows <= kRowsAcross ? dim3((unsigned)rows) : dim3((unsigned)kRowsAcross, (unsigned)div_up(rows, kRowsAcross)); }
__device__ __forceinline__ size_t row_of_block() { return (size_t)blockIdx.y * kRowsAcross + blockIdx.x; }

// An element of 16 or 32 bits, as it lies in memory.
template <int DT>
struct Element {
    using type = uint16_t;
    static constexpr int wide = 8;  // elements to 16 bytes
};
template <>
struct Element<ZK_F32> {
    using type = uint32_t;
    static constexpr int wide = 4;
};

// Which elements of a row a thread has.  WIDE: runs of 16 bytes, so that every load is one; else single ones, side by side
// across the threads, which takes any alignment and length.
template <int DT, int E, bool WIDE>
struct Place {
    static constexpr int W = Element<DT>::wide;
    uint32_t tid, threads, dim;
    __device__ __forceinline__ uint32_t at(int i) const {
        return WIDE ? (tid + (uint32_t)(i / W) * threads) * W + (uint32_t)(i % W) : tid + (uint32_t)i * threads;
    }
    __device__ __forceinline__ bool in(int i) const { return at(WIDE ? i / W * W : i) < dim; }
};

// Two elements of 16 bits, each rounded to nearest.
typedef float v2f __attribute__((ext_vector_type(2)));
typedef __bf16 v2b __attribute__((ext_vector_type(2)));
template <int DT>
__device__ __forceinline__ uint32_t pair_bits(float a, float b) {
    if constexpr (DT == ZK_BF16) return __builtin_bit_cast(uint32_t, __builtin_convertvector((v2f{a, b}), v2b));
    else return __builtin_bit_cast(uint32_t, __builtin_convertvector((v2f{a, b}), v2h));
}

// A thread's elements of a row, as they lie in memory: asked for long before they are used.  Zeros behind the row's end.
template <int DT, int E, bool WIDE>
struct Raw {
    static constexpr int W = Element<DT>::wide;
    uint32_t word[WIDE ? E / W * 4 : E];
    __device__ __forceinline__ void load(const void* p, size_t row, const Place<DT, E, WIDE>& at) {
        const typename Element<DT>::type* x = (const typename Element<DT>::type*)p + row;
        if constexpr (WIDE) {
#pragma unroll
            for (int v = 0; v < E / W; ++v) {
                v4u q = {0, 0, 0, 0};
                if (at.in(v * W)) q = *(const v4u*)(x + at.at(v * W));
#pragma unroll
                for (int k = 0; k < 4; ++k) word[4 * v + k] = q[k];
            }
        } else {
#pragma unroll
            for (int i = 0; i < E; ++i) word[i] = at.in(i) ? (uint32_t)x[at.at(i)] : 0u;
        }
    }
    __device__ __forceinline__ float get(int i) const {
        if constexpr (DT == ZK_F32) return bits_float(word[i]);
        else if constexpr (WIDE) return half_of<DT>(word[i >> 1], i & 1);
        else return half_of<DT>(word[i], 0);
    }
    // f, rounded to the type
    __device__ __forceinline__ void set(const float (&f)[E]) {
#pragma unroll
        for (int i = 0; i < E; ++i) {
            if constexpr (!WIDE) word[i] = half_bits<DT>(as_it_is(f[i]));
            else if (i & 1) word[i >> 1] = pair_bits<DT>(as_it_is(f[i - 1]), as_it_is(f[i]));
        }
    }
    __device__ __forceinline__ void store(void* p, size_t row, const Place<DT, E, WIDE>& at) const {
        typename Element<DT>::type* y = (typename Element<DT>::type*)p + row;
        if constexpr (WIDE) {
#pragma unroll
            for (int v = 0; v < E / W; ++v)
                if (at.in(v * W)) *(v4u*)(y + at.at(v * W)) = v4u{word[4 * v], word[4 * v + 1], word[4 * v + 2], word[4 * v + 3]};
        } else {
#pragma unroll
            for (int i = 0; i < E; ++i)
                if (at.in(i)) y[at.at(i)] = (typename Element<DT>::type)word[i];
        }
    }
};

template <int DT>
__device__ __forceinline__ float rounded(float f) {
    if constexpr (DT == ZK_F32) return f;
    return half_of<DT>(half_bits<DT>(as_it_is(f)), 0);
}

// A thread's elements of a row of 32 bits.
template <int E, bool WIDE>
__device__ __forceinline__ void store_floats(void* p, size_t row, const Place<ZK_F32, E, WIDE>& at, const float (&f)[E]) {
    float* y = (float*)p + row;
    if constexpr (WIDE) {
#pragma unroll
        for (int v = 0; v < E; v += 4)
            if (at.in(v)) *(v4f*)(y + at.at(v)) = v4f{f[v], f[v + 1], f[v + 2], f[v + 3]};
    } else {
#pragma unroll
        for (int i = 0; i < E; ++i)
            if (at.in(i)) y[at.at(i)] = as_it_is(f[i]);
    }
}

static const uint32_t kDigits = 10, kCopies = 16;  // of 32 bits, from 2^-149 on: what 2^15 floats add up to; copies, so that few lanes meet

// Over a workgroup, in every thread.  LDS slots are used in turn, so that one barrier is enough between two sums.
struct Scratch {
    double sums[2][kMostThreads / 64], lost[2][kMostThreads / 64];
    unsigned long long digits[kDigits][kCopies];
    uint32_t most[kMostThreads / 64];
};
template <int CTRL, int ROWS>
__device__ __forceinline__ double partner(double x) {  // 0 where a lane has none
    const uint64_t b = __builtin_bit_cast(uint64_t, x);
    const uint32_t lo = from_lane<CTRL, ROWS>(0u, (uint32_t)b), hi = from_lane<CTRL, ROWS>(0u, (uint32_t)(b >> 32));
    return __builtin_bit_cast(double, ((uint64_t)hi << 32) | lo);
}
template <int CTRL, int ROWS>
__device__ __forceinline__ double add_from(double x) {
    return x + partner<CTRL, ROWS>(x);
}
__device__ __forceinline__ double wave_add64(double x) {  // the same moves as over_wave; in lane 63
    x = add_from<0x111, 0xf>(x);
    x = add_from<0x112, 0xf>(x);
    x = add_from<0x114, 0xf>(x);
    x = add_from<0x118, 0xf>(x);
    x = add_from<0x142, 0xa>(x);
    return add_from<0x143, 0xc>(x);
}
__device__ __forceinline__ double all_add(double x, Scratch& s, int turn, uint32_t waves) {
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    x = wave_add64(x);
    if (lane == 63) s.sums[turn & 1][wave] = x;
    __syncthreads();
    double sum = 0.0;
    for (uint32_t w = 0; w < waves; ++w) sum += s.sums[turn & 1][w];
    return sum;
}

// A lane's value, for all.
__device__ __forceinline__ double one_for_all(double x, int lane = 0) {
    const uint64_t b = __builtin_bit_cast(uint64_t, x);
    const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)b, lane), hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(b >> 32), lane);
    return __builtin_bit_cast(double, ((uint64_t)hi << 32) | lo);
}

// What a norm takes off and multiplies by.
struct Stats {
    float mean, rstd;
};
__device__ __forceinline__ double rstd_of(double variance, float eps) { return 1.0 / sqrt(variance + (double)eps); }

// A sum and what its additions have lost (Knuth's two-sum): together exact to some 2^-90 of the summands' sizes.
struct Whole {
    double sum = 0.0, lost = 0.0;
    __device__ __forceinline__ void add(double x) {
        const double s = sum + x, b = s - sum;
        lost += (sum - (s - b)) + (x - b);
        sum = s;
    }
    __device__ __forceinline__ void add_square(double v, double mean) {  // (v - mean)^2: v - mean is d + less, d^2 is square and its own loss
        const double d = v - mean, b = d - v, less = (v - (d - b)) - (mean + b), square = d * d;
        add(square);
        lost += __builtin_fma(d, d, -square) + 2.0 * d * less;
    }
    template <int CTRL, int ROWS>
    __device__ __forceinline__ void add_partner() {
        const double other = partner<CTRL, ROWS>(sum), also = partner<CTRL, ROWS>(lost);
        add(other);
        lost += also;
    }
};
__device__ __forceinline__ Whole all_add(Whole x, Scratch& s, int turn, uint32_t waves) {
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    x.add_partner<0x111, 0xf>();
    x.add_partner<0x112, 0xf>();
    x.add_partner<0x114, 0xf>();
    x.add_partner<0x118, 0xf>();
    x.add_partner<0x142, 0xa>();
    x.add_partner<0x143, 0xc>();
    if (lane == 63) {
        s.sums[turn & 1][wave] = x.sum;
        s.lost[turn & 1][wave] = x.lost;
    }
    __syncthreads();
    const bool has = (lane & 15) < waves;  // 16 wavefronts at most, whose sums a row of lanes adds up
    x = {has ? s.sums[turn & 1][lane & 15] : 0.0, has ? s.lost[turn & 1][lane & 15] : 0.0};
    x.add_partner<0x111, 0xf>();
    x.add_partner<0x112, 0xf>();
    x.add_partner<0x114, 0xf>();
    x.add_partner<0x118, 0xf>();
    return {one_for_all(x.sum, 15), one_for_all(x.lost, 15)};
}

// A sum of floats that cancels, in fixed point: a float's 24 bits lie in two digits, which integers add up in any order.
__device__ __forceinline__ void add_digits(Scratch& s, float v) {
    const uint32_t bits = float_bits(v), e = (bits >> 23) & 0xff, at = e ? e - 1 : 0;
    const uint64_t x = (uint64_t)((bits & 0x7fffffu) | (e ? 0x800000u : 0u)) << (at & 31);
    const uint64_t lo = (uint32_t)x, hi = x >> 32;
    unsigned long long* digit = &s.digits[at >> 5][threadIdx.x % kCopies];
    atomicAdd(digit, bits >> 31 ? 0 - lo : lo);
    atomicAdd(digit + kCopies, bits >> 31 ? 0 - hi : hi);
}
// What they come to, rounded once; by one thread, which leaves them in another form.
__device__ __forceinline__ double digits_value(Scratch& s) {
    int64_t carry = 0;
#pragma unroll 1
    for (uint32_t k = 0; k < kDigits; ++k) {  // each to 32 bits
        carry += (int64_t)s.digits[k][0];
        s.digits[k][0] = (uint32_t)carry;
        carry >>= 32;
    }
    const bool negative = carry < 0;
    if (negative) {
        carry = 1;
#pragma unroll 1
        for (uint32_t k = 0; k < kDigits; ++k) {
            carry += (uint32_t)~s.digits[k][0];
            s.digits[k][0] = (uint32_t)carry;
            carry >>= 32;
        }
    }
    int top = (int)kDigits - 1;
#pragma unroll 1
    while (top > 0 && s.digits[top][0] == 0) --top;
    if (s.digits[top][0] == 0) return 0.0;
    // the highest 64 bits, in the lowest of them whether anything lies below
    uint64_t most = (s.digits[top][0] << 32) | (top > 0 ? s.digits[top - 1][0] : 0), rest = top > 1 ? s.digits[top - 2][0] << 32 : 0;
    const int zeros = __builtin_clzll(most);
    if (zeros) {
        most = (most << zeros) | (rest >> (64 - zeros));
        rest <<= zeros;
    }
#pragma unroll 1
    for (int k = 0; k < top - 2; ++k) rest |= s.digits[k][0];
    const double value = ldexp((double)(most | (rest ? 1 : 0)), 32 * (top - 1) - zeros - 149);
    return negative ? -value : value;
}

// Whether two sums of the same row in other orders might come to statistics that differ in 32 bits.  A summand goes through `each` additions
// (at most 32) of its thread, 6 of its wavefront and those of the workgroup's, so that a sum is within as many times 2^-53 of its summands' sizes,
// whose mean is at most |mean| + sqrt(variance) (Cauchy).  For one root in some 2^20 they might, and for one mean in some 2^17 of 32 bits, of 16 bits in 40 (in
// the very middle), oftener where it is small beside its row; then the row is added up again.  What is given is the same in every thread.
enum { kMeanOpen = 1, kRstdOpen = 2 };
__device__ __forceinline__ uint32_t undecided(int kind, double mean, double variance, double rstd, float eps, uint32_t each, uint32_t waves) {
    // within 2^-45 of the middle between two floats, or below the normal ones
    const uint64_t bits = __builtin_bit_cast(uint64_t, rstd);
    const uint32_t low = ((uint32_t)bits - (0x10000000u - 256u)) & 0x1fffffffu, high = (uint32_t)(bits >> 32);
    uint32_t open = low < 512u || high - 1u < 0x38100000u - 1u ? kRstdOpen : 0;
    if (kind == ZK_NORM_LAYER) {
        const double by = (double)(each + waves + 10) * 0x1.01p-53 * (__builtin_fabs(mean) + __builtin_amdgcn_sqrt(variance));  // the root to some 2^-20
        if (__ballot((float)(mean - by) < (float)(mean + by))) open |= kMeanOpen;
        // around a mean that is off by as much the squares come to by^2 more
        if (__ballot(by * by * 0x1p47 > variance + (double)eps)) open |= kRstdOpen;
    }
    return open;
}
// The statistics st of a row of which some are undecided, mean and variance as they were before.  `over` hands each of the thread's elements on, and
// whether it is one of the row.  The mean of numbers of 16 bits often lies in the very middle, but nothing is lost when they are added up; where
// something is, and two numbers of 64 bits leave the mean open too, it cancels and is taken in fixed point.
template <typename Over>
__device__ __forceinline__ void decide(Stats& st, uint32_t open, int kind, double mean, double variance, double n, float eps, Scratch& s, int& turn, uint32_t waves,
                                       Over over) {
    if (kind == ZK_NORM_LAYER) {
        Whole sum;
        over([&](float v, bool in) { sum.add(in ? (double)v : 0.0); });
        const Whole all = all_add(sum, s, turn++, waves);
        const double by = 0x1p-85 * (__builtin_fabs(mean) + __builtin_amdgcn_sqrt(variance));
        mean = (all.sum + all.lost) / n;
        if (__ballot(all.lost != 0.0 && (float)(mean - by) < (float)(mean + by))) {
            const int slot = turn++ & 1;
            for (uint32_t k = threadIdx.x; k < kDigits * kCopies; k += blockDim.x) s.digits[0][k] = 0;
            __syncthreads();
            over([&](float v, bool in) { add_digits(s, in ? v : 0.0f); });
            __syncthreads();
            if (threadIdx.x < kDigits)
                for (uint32_t c = 1; c < kCopies; ++c) s.digits[threadIdx.x][0] += s.digits[threadIdx.x][c];
            __syncthreads();
            if (threadIdx.x == 0) s.sums[slot][0] = digits_value(s);
            __syncthreads();
            mean = s.sums[slot][0] / n;
        }
        st.mean = (float)mean;
    }
    if (open & kRstdOpen) {
        Whole squares;
        over([&](float v, bool in) { squares.add_square(in ? (double)v : mean, mean); });
        const Whole all = all_add(squares, s, turn++, waves);
        st.rstd = (float)rstd_of((all.sum + all.lost) / n, eps);
    }
}
__device__ __forceinline__ float normed(float v, int kind, const Stats& st) {
    if (kind == ZK_NORM_LAYER) v = v - st.mean;
    return kind == ZK_NORM_NONE ? v : v * st.rstd;
}

// v = (v - mean) * rstd * gain + bias, statistics over the workgroup's row.  `turn` counts the sums.
template <int DT, int E, bool WIDE>
__device__ __forceinline__ void normalise(float (&v)[E], int kind, float eps, const Raw<DT, E, WIDE>& gain, bool has_gain,
                                          const Raw<DT, E, WIDE>& bias, bool has_bias, const Place<DT, E, WIDE>& at, Scratch& s, int& turn,
                                          uint32_t waves) {
    if (kind != ZK_NORM_NONE) {
        const double n = (double)at.dim;
        double mean = 0.0, sum = 0.0;
        if (kind == ZK_NORM_LAYER) {
#pragma unroll
            for (int i = 0; i < E; ++i) sum += (double)v[i];  // zeros behind the row's end
            mean = one_for_all(all_add(sum, s, turn++, waves) / n);
            sum = 0.0;
#pragma unroll
            for (int i = 0; i < E; ++i) {
                const double d = at.in(i) ? (double)v[i] - mean : 0.0;
                sum = __builtin_fma(d, d, sum);
            }
        } else {
#pragma unroll
            for (int i = 0; i < E; ++i) sum = __builtin_fma((double)v[i], (double)v[i], sum);
        }
        const double variance = all_add(sum, s, turn++, waves) / n, rstd = one_for_all(rstd_of(variance, eps));
        Stats st = {(float)mean, (float)rstd};
        const uint32_t open = undecided(kind, mean, variance, rstd, eps, E, waves);
        if (__builtin_expect(open, 0))
            decide(st, open, kind, mean, variance, n, eps, s, turn, waves, [&](auto take) {
#pragma unroll
                for (int i = 0; i < E; ++i) take(v[i], at.in(i));
            });
#pragma unroll
        for (int i = 0; i < E; ++i) v[i] = normed(v[i], kind, st);
    }
    if (has_gain) {
#pragma unroll
        for (int i = 0; i < E; ++i) v[i] = v[i] * gain.get(i);
    }
    if (has_bias) {
#pragma unroll
        for (int i = 0; i < E; ++i) v[i] = v[i] + bias.get(i);
    }
}

// scale = amax / 127, codes rint(h * (127 / amax)); the sum with 1.5 * 2^23 has the rounded integer in its lowest bits.
__device__ __forceinline__ bool code_scale(uint32_t most, float& scale, float& inv) {
    const float amax = bits_float(most);
    const bool fine = most < 0x7f800000u, some = fine && amax >= kLeast;
    scale = some ? amax / 127.0f : fine ? 0.0f : __builtin_nanf("");
    inv = some ? 127.0f / amax : 0.0f;
    return some;
}
__device__ __forceinline__ uint32_t code_of(float h, float inv) { return float_bits(h * inv + 12582912.0f); }  // the lowest byte

__device__ __forceinline__ uint32_t all_most(uint32_t most, Scratch& s, uint32_t waves) {
    most = wave_max(most);
    if (waves > 1) {
        if ((threadIdx.x & 63) == 0) s.most[threadIdx.x >> 6] = most;
        __syncthreads();
        for (uint32_t w = 0; w < waves; ++w) most = s.most[w] > most ? s.most[w] : most;
    }
    return most;
}

// Behind the row's end everything is zero and stays so (gains and biases are zeros there), but for what a mean was taken off.
template <int DT, int E, bool WIDE>
__device__ __forceinline__ void zeros_behind(float (&v)[E], int kind, const Place<DT, E, WIDE>& at) {
    if (kind != ZK_NORM_LAYER) return;
#pragma unroll
    for (int i = 0; i < E; ++i) v[i] = at.in(i) ? v[i] : 0.0f;
}

template <int DT, int E, bool WIDE>
__device__ __forceinline__ void store_codes(int8_t* codes, size_t row, float* scale_at, const Place<DT, E, WIDE>& at, const float (&h)[E], Scratch& s,
                                            uint32_t waves) {
    constexpr int W = Element<DT>::wide;
    uint32_t most = 0;  // the bits of |h|: infinities and NaN are above every number
#pragma unroll
    for (int i = 0; i < E; ++i) {
        const uint32_t bits = float_bits(h[i]) & 0x7fffffffu;  // zeros behind the row's end
        most = bits > most ? bits : most;
    }
    float scale, inv;
    const bool some = code_scale(all_most(most, s, waves), scale, inv);
    if (threadIdx.x == 0) *scale_at = scale;
    int8_t* y = codes + row;
    if constexpr (WIDE) {
#pragma unroll
        for (int v = 0; v < E / W; ++v) {
            uint32_t q[W / 4];
#pragma unroll
            for (int k = 0; k < W / 4; ++k) {
                const float* f = h + v * W + 4 * k;  // the lowest byte of each
                const uint32_t lo = __builtin_amdgcn_perm(code_of(f[1], inv), code_of(f[0], inv), 0x0c0c0400u);
                const uint32_t hi = __builtin_amdgcn_perm(code_of(f[3], inv), code_of(f[2], inv), 0x0c0c0400u);
                q[k] = some ? __builtin_amdgcn_perm(hi, lo, 0x05040100u) : 0u;
            }
            if (at.in(v * W)) {
                if constexpr (W == 8) *(uint2*)(y + at.at(v * W)) = make_uint2(q[0], q[1]);
                else *(uint32_t*)(y + at.at(v * W)) = q[0];
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < E; ++i)
            if (at.in(i)) y[at.at(i)] = some ? (int8_t)code_of(h[i], inv) : (int8_t)0;
    }
}

// Eight wavefronts to a SIMD where eight elements do: 777 rows of 4097 floats 16.3 -> 14.6 us, though registers spill (13 words of a thread's
// where no 16-byte load is taken, 5 of floats in whole runs, most of them on the way of rows that are undecided); five with 16 elements of 16 bits, which would be four with the registers that the
// second sums ask for (8192 rows of 5120 bf16 90 us, 114 with four).
template <int DT, int E, bool WIDE>
__global__ __launch_bounds__(kMostThreads, E <= 8 ? 8 : DT == ZK_F32 ? 4 : 5) void k_block_norm(NormArgs n) {
    __shared__ Scratch s;
    const block_norm_args& a = n.a;
    const size_t row = row_of_block();
    if (row >= n.rows) return;
    const uint32_t waves = blockDim.x >> 6;
    const Place<DT, E, WIDE> at = {threadIdx.x, blockDim.x, n.dim};
    Raw<DT, E, WIDE> z, x, gate, gain, bias, post_gain, post_bias;
    if (a.z) z.load(a.z, row * a.z_row_stride, at);
    x.load(a.x, row * a.x_row_stride, at);
    if (a.gate) gate.load(a.gate, row * a.gate_row_stride, at);
    int turn = 0;
    float v[E];
    if (a.z) {
        if (a.post_gain) post_gain.load(a.post_gain, 0, at);
        if (a.post_bias) post_bias.load(a.post_bias, 0, at);
#pragma unroll
        for (int i = 0; i < E; ++i) v[i] = z.get(i);
        normalise(v, a.post_norm, a.eps, post_gain, a.post_gain != nullptr, post_bias, a.post_bias != nullptr, at, s, turn, waves);
        zeros_behind(v, a.post_norm, at);
        if (a.gate) {
#pragma unroll
            for (int i = 0; i < E; ++i) v[i] = gate.get(i) * v[i];
        }
#pragma unroll
        for (int i = 0; i < E; ++i) v[i] = a.alpha * x.get(i) + v[i];
    } else {
#pragma unroll
        for (int i = 0; i < E; ++i) v[i] = a.alpha * x.get(i);
    }
    if (a.gain) gain.load(a.gain, 0, at);
    if (a.bias) bias.load(a.bias, 0, at);
    if constexpr (DT == ZK_F32) {
        if (a.r) store_floats(a.r, row * a.r_row_stride, at, v);
        if (!a.h && !a.codes) return;
#pragma unroll
        for (int i = 0; i < E; ++i) v[i] = WIDE || at.in(i) ? v[i] : 0.0f;
    } else {
        Raw<DT, E, WIDE> out;
        out.set(v);
        if (a.r) out.store(a.r, row * a.r_row_stride, at);
        if (!a.h && !a.codes) return;
#pragma unroll
        for (int i = 0; i < E; ++i) v[i] = out.get(i);  // what the next block sees is what is stored
    }
    normalise(v, a.norm, a.eps, gain, a.gain != nullptr, bias, a.bias != nullptr, at, s, turn, waves);
    if (a.h) {
        if constexpr (DT == ZK_F32) {
            store_floats(a.h, row * a.h_row_stride, at, v);
        } else {
            Raw<DT, E, WIDE> out;
            out.set(v);
            out.store(a.h, row * a.h_row_stride, at);
        }
        return;
    }
    zeros_behind(v, a.norm, at);
    store_codes<DT, E, WIDE>(a.codes, row * a.codes_row_stride, a.scales + row, at, v, s, waves);
}

// Rows of more than 16 elements to a thread (or of eight that no 16-byte load takes): the row lies in LDS, in 32 bits, each element
// read and written by the thread that brought it.  In registers, with the gains beside, they would spill (100 us for one row).
template <int DT>
__global__ __launch_bounds__(kMostThreads, 8) void k_block_norm_long(NormArgs n) {
    extern __shared__ __attribute__((aligned(16))) float line[];
    __shared__ Scratch s;
    const block_norm_args& a = n.a;
    const size_t row = row_of_block();
    if (row >= n.rows) return;
    const uint32_t waves = kMostThreads / 64, dim = n.dim;
    int turn = 0;
    auto statistics = [&](int kind) {
        Stats st = {0.0f, 1.0f};
        if (kind == ZK_NORM_NONE) return st;
        double mean = 0.0, sum = 0.0;
        if (kind == ZK_NORM_LAYER) {
            for (uint32_t i = threadIdx.x; i < dim; i += kMostThreads) sum += (double)line[i];
            mean = all_add(sum, s, turn++, waves) / (double)dim;
            sum = 0.0;
        }
        for (uint32_t i = threadIdx.x; i < dim; i += kMostThreads) {
            const double d = (double)line[i] - mean;
            sum = __builtin_fma(d, d, sum);
        }
        const double variance = all_add(sum, s, turn++, waves) / (double)dim, rstd = one_for_all(rstd_of(variance, a.eps));
        st.rstd = (float)rstd;
        st.mean = (float)mean;
        const uint32_t open = undecided(kind, mean, variance, rstd, a.eps, 32, waves);
        if (__builtin_expect(open, 0))
            decide(st, open, kind, mean, variance, (double)dim, a.eps, s, turn, waves, [&](auto take) {
                for (uint32_t i = threadIdx.x; i < dim; i += kMostThreads) take(line[i], true);
            });
        return st;
    };
    auto finished = [&](float v, int kind, const Stats& st, const void* gain, const void* bias, uint32_t i) {
        v = normed(v, kind, st);
        if (gain) v = v * load_one<DT>(gain, i);
        return bias ? v + load_one<DT>(bias, i) : v;
    };
    if (a.z) {
        for (uint32_t i = threadIdx.x; i < dim; i += kMostThreads) line[i] = load_one<DT>(a.z, row * a.z_row_stride + i);
        const Stats st = statistics(a.post_norm);
        for (uint32_t i = threadIdx.x; i < dim; i += kMostThreads) {
            float t = finished(line[i], a.post_norm, st, a.post_gain, a.post_bias, i);
            if (a.gate) t = load_one<DT>(a.gate, row * a.gate_row_stride + i) * t;
            line[i] = a.alpha * load_one<DT>(a.x, row * a.x_row_stride + i) + t;
        }
    } else {
        for (uint32_t i = threadIdx.x; i < dim; i += kMostThreads) line[i] = a.alpha * load_one<DT>(a.x, row * a.x_row_stride + i);
    }
    for (uint32_t i = threadIdx.x; i < dim; i += kMostThreads) {
        const float v = line[i];
        if (a.r) store_one<DT>(a.r, row * a.r_row_stride + i, as_it_is(v));
        line[i] = rounded<DT>(v);
    }
    if (!a.h && !a.codes) return;
    const Stats st = statistics(a.norm);
    uint32_t most = 0;
    for (uint32_t i = threadIdx.x; i < dim; i += kMostThreads) {
        const float h = finished(line[i], a.norm, st, a.gain, a.bias, i);
        if (a.h) store_one<DT>(a.h, row * a.h_row_stride + i, as_it_is(h));
        line[i] = h;
        const uint32_t bits = float_bits(h) & 0x7fffffffu;
        most = bits > most ? bits : most;
    }
    if (!a.codes) return;
    float scale, inv;
    const bool some = code_scale(all_most(most, s, waves), scale, inv);
    if (threadIdx.x == 0) a.scales[row] = scale;
    for (uint32_t i = threadIdx.x; i < dim; i += kMostThreads) a.codes[row * a.codes_row_stride + i] = some ? (int8_t)code_of(line[i], inv) : (int8_t)0;
}

template <int DT, int E, bool WIDE>
__global__ __launch_bounds__(kMostThreads) void k_quantise(int8_t* codes, size_t codes_row, float* scales, const void* x, size_t x_row, uint32_t dim,
                                                         size_t rows) {
    __shared__ Scratch s;
    const size_t row = row_of_block();
    if (row >= rows) return;
    const Place<DT, E, WIDE> at = {threadIdx.x, blockDim.x, dim};
    Raw<DT, E, WIDE> raw;
    raw.load(x, row * x_row, at);
    float v[E];
#pragma unroll
    for (int i = 0; i < E; ++i) v[i] = raw.get(i);
    store_codes<DT, E, WIDE>(codes, row * codes_row, scales + row, at, v, s, blockDim.x >> 6);
}

// Rows longer than the registers of a workgroup: read twice, the second time from a cache that holds them.
template <int DT>
__global__ __launch_bounds__(kMostThreads) void k_quantise_long(int8_t* codes, size_t codes_row, float* scales, const void* x, size_t x_row, uint32_t dim,
                                                              size_t rows) {
    __shared__ Scratch s;
    const size_t row = row_of_block(), from = row * x_row;
    if (row >= rows) return;
    uint32_t most = 0;
    for (uint32_t i = threadIdx.x; i < dim; i += kMostThreads) {
        const uint32_t bits = float_bits(load_one<DT>(x, from + i)) & 0x7fffffffu;
        most = bits > most ? bits : most;
    }
    float scale, inv;
    const bool some = code_scale(all_most(most, s, kMostThreads / 64), scale, inv);
    if (threadIdx.x == 0) scales[row] = scale;
    for (uint32_t i = threadIdx.x; i < dim; i += kMostThreads)
        codes[row * codes_row + i] = some ? (int8_t)code_of(load_one<DT>(x, from + i), inv) : (int8_t)0;
}

// ---- host -------------------------------------------------------------------------------------------------------------

bool float_type(int dtype) { return dtype == ZK_F32 || dtype == ZK_F16 || dtype == ZK_BF16; }
bool norm_kind(int kind) { return kind == ZK_NORM_NONE || kind == ZK_NORM_RMS || kind == ZK_NORM_LAYER; }

// How a row is spread: elements of a thread, and threads.  As few elements as 1024 threads allow; of many rows 16, which takes fewer steps
// to add up a row and to bring gains: 8192 rows of 5120 bf16 104 -> 89 us (one row 3.7 -> 4.1, so not of few).
struct Spread {
    int each;
    uint32_t threads;
};
Spread spread_of(int dtype, uint32_t dim, size_t rows, bool wide) {
    int each = dtype == ZK_F32 ? 4 : 8;
    if (each == 8 && wide && rows >= 1024 && dim >= 1024) each = 16;
    while (each < 32 && div_up(dim, each) > kMostThreads) each *= 2;
    return {each, (uint32_t)align_up(div_up(dim, each), 64)};
}

template <int DT, int E, bool WIDE>
int launch_norm(const NormArgs& n, uint32_t threads, hipStream_t s) {
    hipLaunchKernelGGL((k_block_norm<DT, E, WIDE>), grid_of(n.rows), dim3(threads), 0, s, n);
    return ZK_OK;
}
template <int DT>
int launch_long(const NormArgs& n, hipStream_t s) {
    const size_t lds = n.dim * sizeof(float);
    if (lds > 60000) ZK_HIP_TRY(hipFuncSetAttribute((const void*)k_block_norm_long<DT>, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds));
    hipLaunchKernelGGL((k_block_norm_long<DT>), grid_of(n.rows), dim3(kMostThreads), lds, s, n);
    return ZK_OK;
}
template <int DT, bool WIDE>
int spread_norm(const NormArgs& n, hipStream_t s) {
    const Spread p = spread_of(DT, n.dim, n.rows, WIDE);
    if constexpr (DT == ZK_F32)
        if (p.each == 4) return launch_norm<DT, 4, WIDE>(n, p.threads, s);
    if (p.each == 8) return launch_norm<DT, 8, WIDE>(n, p.threads, s);
    if constexpr (WIDE)
        if (p.each == 16) return launch_norm<DT, 16, WIDE>(n, p.threads, s);
    return launch_long<DT>(n, s);
}

struct QuantiseArgs {
    int8_t* codes;
    size_t codes_row;
    float* scales;
    const void* x;
    size_t x_row;
    uint32_t dim;
    size_t rows;
};
template <int DT, int E, bool WIDE>
void launch_quantise(const QuantiseArgs& q, uint32_t threads, hipStream_t s) {
    hipLaunchKernelGGL((k_quantise<DT, E, WIDE>), grid_of(q.rows), dim3(threads), 0, s, q.codes, q.codes_row, q.scales, q.x, q.x_row, q.dim, q.rows);
}
template <int DT, bool WIDE>
void spread_quantise(const QuantiseArgs& q, hipStream_t s) {
    const Spread p = spread_of(DT, q.dim, q.rows, WIDE);
    if constexpr (DT == ZK_F32)
        if (p.each == 4) return launch_quantise<DT, 4, WIDE>(q, p.threads, s);
    if (p.each == 8) return launch_quantise<DT, 8, WIDE>(q, p.threads, s);
    if (p.each == 16) return launch_quantise<DT, 16, WIDE>(q, p.threads, s);
    launch_quantise<DT, 32, WIDE>(q, p.threads, s);
}
template <int DT>
void quantise_of(const QuantiseArgs& q, bool wide, hipStream_t s) {
    if (q.dim > kMostDim) hipLaunchKernelGGL((k_quantise_long<DT>), grid_of(q.rows), dim3(kMostThreads), 0, s, q.codes, q.codes_row, q.scales, q.x, q.x_row, q.dim, q.rows);
    else if (wide) spread_quantise<DT, true>(q, s);
    else spread_quantise<DT, false>(q, s);
}

// A matrix of the call: rows far enough apart, aligned to its elements.  With one row the stride says nothing.
bool rows_ok(const void* p, size_t stride, size_t bytes, size_t rows, size_t dim) {
    return aligned(p, bytes) && (rows <= 1 || stride >= dim) && stride <= (size_t)1 << 40;
}

}  // namespace
}  // namespace zkmi

using namespace zkmi;

extern "C" int block_norm(const block_norm_args* args, int dtype, size_t rows, size_t dim, void* stream) {
    if (!args || !float_type(dtype) || dim == 0 || dim > kMostDim || rows >= 0x80000000u) return ZK_E_BADARG;
    block_norm_args a = *args;
    const size_t bytes = dtype_bytes(dtype);
    if (!norm_kind(a.norm) || !norm_kind(a.post_norm) || !(a.alpha - a.alpha == 0.0f)) return ZK_E_BADARG;
    if ((a.norm != ZK_NORM_NONE || a.post_norm != ZK_NORM_NONE) && !(a.eps > 0.0f && a.eps - a.eps == 0.0f)) return ZK_E_BADARG;
    if (rows == 0) return ZK_OK;
    if (!a.z && (a.gate || a.post_gain || a.post_bias || a.post_norm != ZK_NORM_NONE)) return ZK_E_BADARG;
    if ((a.h && a.codes) || (!a.codes != !a.scales)) return ZK_E_BADARG;
    if (!a.x || (!a.r && !a.h && !a.codes)) return ZK_E_BADARG;
    if (!rows_ok(a.x, a.x_row_stride, bytes, rows, dim) || (a.z && !rows_ok(a.z, a.z_row_stride, bytes, rows, dim)) ||
        (a.gate && a.gate_row_stride && !rows_ok(a.gate, a.gate_row_stride, bytes, rows, dim)) || (a.r && !rows_ok(a.r, a.r_row_stride, bytes, rows, dim)) ||
        (a.h && !rows_ok(a.h, a.h_row_stride, bytes, rows, dim)) || (a.codes && !rows_ok(a.codes, a.codes_row_stride, 1, rows, dim)))
        return ZK_E_BADARG;
    for (const void* p : {a.gate, a.gain, a.bias, a.post_gain, a.post_bias, (const void*)a.scales})
        if (p && !aligned(p, p == a.scales ? 4 : bytes)) return ZK_E_BADARG;
    const size_t run = 16 / bytes;
    bool wide = dim % run == 0;
    const struct {
        const void* p;
        size_t stride;
    } tensors[] = {{a.x, a.x_row_stride}, {a.z, a.z_row_stride}, {a.gate, a.gate_row_stride}, {a.r, a.r_row_stride}, {a.h, a.h_row_stride},
                   {a.gain, 0}, {a.bias, 0}, {a.post_gain, 0}, {a.post_bias, 0}};
    for (const auto& t : tensors) wide = wide && (!t.p || (aligned(t.p, 16) && (rows == 1 || t.stride % run == 0)));
    wide = wide && (!a.codes || (aligned(a.codes, run) && (rows == 1 || a.codes_row_stride % run == 0)));
    const NormArgs n = {a, dtype, (uint32_t)dim, rows};
    hipStream_t s = as_stream(stream);
    if (dtype == ZK_F32) ZK_TRY((wide ? spread_norm<ZK_F32, true>(n, s) : spread_norm<ZK_F32, false>(n, s)));
    else if (dtype == ZK_F16) ZK_TRY((wide ? spread_norm<ZK_F16, true>(n, s) : spread_norm<ZK_F16, false>(n, s)));
    else ZK_TRY((wide ? spread_norm<ZK_BF16, true>(n, s) : spread_norm<ZK_BF16, false>(n, s)));
    ZK_HIP_TRY(hipGetLastError());
    return ZK_OK;
}

extern "C" int i8_quantise(int8_t* codes, size_t codes_row_stride, float* scales, const void* x, size_t x_row_stride, int dtype, size_t rows,
                           size_t k, void* stream) {
    if (!float_type(dtype) || k == 0 || k > I8_MAX_K || rows >= 0x80000000u) return ZK_E_BADARG;
    if (rows == 0) return ZK_OK;
    const size_t bytes = dtype_bytes(dtype), run = 16 / bytes;
    if (!codes || !scales || !x || !aligned(scales, 4) || !rows_ok(x, x_row_stride, bytes, rows, k) || !rows_ok(codes, codes_row_stride, 1, rows, k))
        return ZK_E_BADARG;
    const bool wide = k % run == 0 && aligned(x, 16) && aligned(codes, run) && (rows == 1 || (x_row_stride % run == 0 && codes_row_stride % run == 0));
    const QuantiseArgs q = {codes, codes_row_stride, scales, x, x_row_stride, (uint32_t)k, rows};
    hipStream_t s = as_stream(stream);
    if (dtype == ZK_F32) quantise_of<ZK_F32>(q, wide, s);
    else if (dtype == ZK_F16) quantise_of<ZK_F16>(q, wide, s);
    else quantise_of<ZK_BF16>(q, wide, s);
    ZK_HIP_TRY(hipGetLastError());
    return ZK_OK;
}
