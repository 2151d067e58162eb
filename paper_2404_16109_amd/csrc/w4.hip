// Products of a few vectors with a matrix of 4-bit weights, a scale for each group of inputs.
//
//   y[m][n] = unit * sum_g s[n][g] * sum_{k in g} c[n][k] x[m][k],   c = u - 8,  u a half byte.
//
// The sums over a group run on the matrix cores (16 x 16 x 32).  The first operand is x, a column of it to a row of the
// operand; the second holds 16 outputs' weights.  For 16-bit x a half byte becomes a 16-bit float without a table or a
// subtraction: put into the top of the mantissa of 8.0 it is 8 + u/2 = (c + 24) / 2, exact in both 16-bit types, and -12 sum x
// is added by one more matrix instruction whose second operand is the constant -12.  A term c x is then carried at up to
// (|c| + 24) |x| in 32-bit sums, which leaves up to 1e-5 of the results' size as error (measured at 5120 positive inputs, codes
// of deviation 1.5) where a 16-bit output itself rounds to 2.4e-4 (f16) or 2e-3 (bf16).  A 32-bit output would show it: there
// weights are widened to 16 c, without an offset, for twice the vector instructions; the error is 1.3e-7 then, whatever
// the codes and the inputs (a library's product of 32-bit floats: 1.1e-6).  Types:
//   ZK_F16   x as it is.            ZK_BF16  x as it is.
//   ZK_F32   x as the sum of three bf16 (8 + 8 + 8 bits: exact, whatever stands beside it), three columns.  (Two f16 of a
//            vector scaled to its largest are fewer columns, but miss 2^-40 of the largest in every element: more than a
//            rounding where an outlier meets small weights.)
//   ZK_I16   x = 256 h + l, two columns of whole numbers below 2^8; a group's sums are below 2^20 halves, exact in 32
//            bits, and everything after that is in 64-bit integers.
//
// Layout.  A lane loads 16 bytes, 32 inputs of one output: lane 16 g + i has output i, inputs 32 g .. 32 g + 31 of a step
// of 128.  An instruction wants inputs 8 g .. 8 g + 7 of ONE block of 32 in lane row g, so that what it adds up belongs
// to one group: four exchanges of lane rows transpose the 4 x 4 words.  Of a word's eight half bytes i and i + 4 come to
// lie in one register, so x is kept in the order 0 4 1 5 2 6 3 7.
//
// Bound by the weights' bytes where they are many and the vectors few, by latency below some 20 MB.  For many columns nothing is
// full (96 columns of 32-bit vectors: vector ALU 50% busy, matrix cores 29%, LDS 25%): two wavefronts to a SIMD, in step with each
// other, hide little.  Measured: one vector of bf16 by 5120 x 5120 (13.5 MB) 7.5 us, by 32001 x 5120 (84 MB) 22 us, 3.8 TB/s; 8 of
// 16-bit integers by 4096 x 11008 14.7 us; 64 of bf16 by 32001 x 5120 45 us, 465 TFLOP/s; 32 of 32 bits 51 us; 512 of bf16 by 5120
// x 5120 78 us, 346 TFLOP/s, of 16-bit integers 141.
#include "serve_dev.h"

namespace zkmi {
namespace {

static const int kStep = 128;                      // inputs a wavefront takes at a time
static const int kWaves = 8;
static const uint32_t kStageHalves = 32768;        // 64 KiB of x in LDS
static const size_t kMostRows = (size_t)1 << 20;    // 32768 blocks of columns at most, those of 32-bit floats
// More columns than 16: blocks of 16 that each read the weights again (out of the caches), or the kernel for many columns, whose
// workgroups have 64 or 128 outputs and are too few for a short matrix.  Measured, the first against the second, us: 32
// vectors of bf16 by 4096 x 11008 18.7 and 34.8, by 5120 x 5120 15.0 and 18.7, by 8192 x 4096 18.4 and 16.2, by 9000 x 5120 (24
// of them) 23.2 and 19.3, by 13824 x 5120 30 and 19.5; 64 by 5120 x 5120 21 and 29, by 13824 x 5120 49 and 30; 100 by 4096 x
// 4096 28 and 25.
static const uint32_t kManyOutputs = 8192, kBlocksOfFew = 6;
// Of 32-bit vectors, whose blocks of 16 columns are five vectors, four blocks and more lose against the other kernel sooner, if that
// makes up for few outputs with blocks of two tiles, ten vectors.  Measured, us, blocks of five against blocks of ten (and of 32):
// 16 vectors by 5120 x 5120 22.6 and 18.3 (25.2), 32 33.9 and 27.9 (33.2), 32 by 4096 x 11008 48.8 and 36.2 (68.8), 20 by 8000 x 4096 31.6
// and 15.8 (21.2), 32 by 3000 x 5120 24.3 and 18.8 (33.0); but 16 by 2000 x 8192 16.5 and 24.9, 32 by 1000 x 5120 13.3 and 18.1, and 6
// by 5120 x 5120 15.5 and 17.6.
static const uint32_t kTens = 10, kTensOutputs = 2560;
// What a CU has of LDS.  The kernel for few columns keeps the scales of all groups there, 32 bytes to a group: of more inputs than
// 163840 (groups of 32), 327680 (64) or 655360 (128) a call of whatever rows goes to the kernel for many columns, which keeps
// those of a chunk.
static const size_t kMostLds = 163840;
// Outputs from which a workgroup of the kernel for many columns has 128, not 64.  Measured, 128 and 64, us: 64 vectors of bf16 by
// 13824 x 5120 38 and 30, by 20000 x 5120 38.4 and 39.7, by 32001 x 5120 45 and 49; 32 of 32 bits by 32001 x 5120 52 and 67, 10 of
// them 29 and 32.  But 64 for six tiles of columns and groups of 32, whose sums do not fit the registers with 128: 96 vectors of
// bf16 by 32001 x 5120 192 and 92, 70 by 20000 x 4096 140 and 67, 40 of 16-bit integers by it 149 and 79, 32 of 32 bits by 32001 x
// 5120 153 and 80.
static const uint32_t kWide = 16384;

template <int DT>
struct Kind {
    static constexpr bool wide = DT == ZK_F32;                              // 32 bits to a value of x
    static constexpr int parts = DT == ZK_F32 ? 3 : DT == ZK_I16 ? 2 : 1;  // columns of a vector
    static constexpr int vectors = 16 / parts;                             // vectors of a call's 16 columns
    static constexpr bool f16 = DT == ZK_F16;
    static constexpr bool offset = DT != ZK_F32;                            // weights enter as (c + 24) / 2, else as 16 c
    static constexpr float step = offset ? 2.0f : 0.0625f;                  // what takes that back
};

template <int DT>
__device__ __forceinline__ v4f product(v4u a, v4u b, v4f c) {
    if constexpr (Kind<DT>::f16) return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8h, a), __builtin_bit_cast(v8h, b), c, 0, 0, 0);
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8b, a), __builtin_bit_cast(v8b, b), c, 0, 0, 0);
}

// Eight half bytes as 8 + u/2, or as 16 c: with its top bit flipped a half byte is c in two's complement, in the upper half of a
// byte 16 c, which converts to a float whose lower 16 bits are zero.
template <int DT>
__device__ __forceinline__ v4u widen(uint32_t w) {
    if constexpr (!Kind<DT>::offset) {
        const uint32_t t = w ^ 0x88888888u, even = (t << 4) & 0xf0f0f0f0u, odd = t & 0xf0f0f0f0u;
        auto two = [](uint32_t x, int at) {  // of bytes at and at + 2
            const float lo = (float)(int8_t)(x >> (8 * at)), hi = (float)(int8_t)(x >> (8 * at + 16));
            return __builtin_amdgcn_perm(float_bits(hi), float_bits(lo), 0x07060302u);
        };
        return v4u{two(even, 0), two(odd, 0), two(even, 1), two(odd, 1)};
    }
    if constexpr (Kind<DT>::f16) {
        const uint32_t mask = 0x03c003c0u, eight = 0x48004800u;
        return v4u{((w << 6) & mask) | eight, ((w << 2) & mask) | eight, ((w >> 2) & mask) | eight, ((w >> 6) & mask) | eight};
    }
    const uint32_t mask = 0x00780078u, eight = 0x41004100u;
    return v4u{((w << 3) & mask) | eight, ((w >> 1) & mask) | eight, ((w >> 5) & mask) | eight, ((w >> 9) & mask) | eight};
}

// Lane row g has words r[0..3] of block g; afterwards r[q] is word g of block q.
__device__ __forceinline__ void transpose_rows(v4u& r) {
    auto a = __builtin_amdgcn_permlane32_swap(r[0], r[2], false, false);
    auto b = __builtin_amdgcn_permlane32_swap(r[1], r[3], false, false);
    auto c = __builtin_amdgcn_permlane16_swap(a[0], b[0], false, false);
    auto d = __builtin_amdgcn_permlane16_swap(a[1], b[1], false, false);
    r = v4u{(uint32_t)c[0], (uint32_t)c[1], (uint32_t)d[0], (uint32_t)d[1]};
}

// Inputs k .. k+7 of a vector as they lie in memory, and as its columns' operands, in the order 0 4 1 5 2 6 3 7.
template <int DT>
struct Eight {
    static constexpr int words = Kind<DT>::wide ? 2 : 1;
    v4u r[words];
};
template <int DT>
__device__ __forceinline__ Eight<DT> load_eight(const void* x, size_t at) {
    Eight<DT> e;
    const v4u* p = (const v4u*)((const char*)x + at * (Kind<DT>::wide ? 4 : 2));
#pragma unroll
    for (int i = 0; i < Eight<DT>::words; ++i) e.r[i] = p[i];
    return e;
}
template <int DT>
__device__ __forceinline__ void columns_of(const Eight<DT>& x, v4u (&out)[Kind<DT>::parts]) {
    if constexpr (DT == ZK_F16 || DT == ZK_BF16) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t lo = x.r[0][i >> 1], hi = x.r[0][2 + (i >> 1)];  // elements i and i + 4
            out[0][i] = __builtin_amdgcn_perm(hi, lo, i & 1 ? 0x07060302u : 0x05040100u);
        }
    } else if constexpr (DT == ZK_I16) {
        auto part = [&](int e, int p) -> uint32_t {
            const int v = (int16_t)(x.r[0][e >> 1] >> (16 * (e & 1)));
            return half_bits<ZK_BF16>((float)(p == 0 ? v >> 8 : v & 255));
        };
#pragma unroll
        for (int p = 0; p < 2; ++p)
#pragma unroll
            for (int i = 0; i < 4; ++i) out[p][i] = part(i, p) | (part(i + 4, p) << 16);
    } else {
        float r[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) r[e] = bits_float(x.r[e >> 2][e & 3]);
#pragma unroll
        for (int p = 0; p < 3; ++p)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t lo = half_bits<ZK_BF16>(r[i]), hi = half_bits<ZK_BF16>(r[i + 4]);
                out[p][i] = lo | (hi << 16);
                r[i] -= bits_float(lo << 16);
                r[i + 4] -= bits_float(hi << 16);
            }
    }
}

// Weights are read through a buffer descriptor of a workgroup's outputs: a load behind its end comes back as 0 and costs
// nothing, so that loads can be asked for ahead without a branch (a branch makes the compiler wait for all of them).
// Steps behind the last input, and outputs behind the last, read nothing that way.
typedef __amdgpu_buffer_rsrc_t Buffer;
__device__ __forceinline__ Buffer buffer_of(const void* p, size_t bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, bytes < 0xffffff00u ? (int)bytes : (int)0xffffff00u, 0x00020000);
}
static const uint32_t kNowhere = 0xfffffff0u;
__device__ __forceinline__ v4u load16(Buffer b, uint32_t at) { return __builtin_bit_cast(v4u, __builtin_amdgcn_raw_buffer_load_b128(b, (int)at, 0, 0)); }

// Where a lane finds the weights of an output: 16 bytes (32 inputs) of each of its steps.
struct Row {
    uint32_t at, steps;
};
__device__ __forceinline__ Row row_of(uint32_t out, uint32_t k, uint32_t g) {
    return Row{out * (k >> 1) + g * 16, k / kStep + (g * 32 < k % kStep ? 1 : 0)};
}
__device__ __forceinline__ v4u fetch(Buffer b, const Row& w, uint32_t j) { return load16(b, j < w.steps ? w.at + j * (kStep / 2) : kNowhere); }
// A workgroup's weights, from output n0 on.
__device__ __forceinline__ Buffer weights_of(const uint8_t* codes, uint32_t n, uint32_t k, uint32_t n0, uint32_t outputs) {
    const uint32_t there = n - n0 < outputs ? n - n0 : outputs;
    return buffer_of(codes + (size_t)n0 * (k >> 1), (size_t)there * (k >> 1));
}

// ---- few columns -----------------------------------------------------------------------------------------------------

// How a workgroup of 512 brings x into LDS: `across` threads to a vector, each eight inputs at a time.
__host__ __device__ __forceinline__ uint32_t threads_across(uint32_t vectors) { return vectors == 1 ? 512 : vectors == 2 ? 256 : 128; }
// Workgroup: 16 outputs, up to 16 columns; its eight wavefronts share out the steps and add up at the end.  x comes from
// LDS where all of it fits there (STAGED), else from `xf`, where k_w4_columns has laid out the operands [k / 8][16]: a
// wavefront then reads a kilobyte of them for each instruction, out of the L2, and nothing waits for anything in the loop.
template <int DT, bool STAGED, int GL>
__global__ __launch_bounds__(kWaves * 64) void k_w4_few(void* y, size_t ystride, const void* x, size_t xstride, const v4u* xf, size_t rows,
                                                        const uint8_t* codes, const uint16_t* scales, uint32_t n, uint32_t k,
                                                        float step_unit) {
    constexpr int parts = Kind<DT>::parts;
    constexpr uint32_t group_log = GL;
    extern __shared__ v4u shared[];
    const uint32_t tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), g = lane >> 4, i16 = lane & 15;
    const uint32_t n0 = blockIdx.x * 16;
    const size_t m0 = (size_t)blockIdx.y * Kind<DT>::vectors;
    const uint32_t vectors = rows - m0 < (size_t)Kind<DT>::vectors ? (uint32_t)(rows - m0) : Kind<DT>::vectors;
    const uint32_t cols = vectors * parts;
    const uint32_t steps = (k + kStep - 1) / kStep, groups = (k + (1u << group_log) - 1) >> group_log, all_groups = steps * kStep >> group_log;
    v4u* xs = shared;                                                            // [k / 8][cols]
    uint16_t* ss = (uint16_t*)(shared + (STAGED ? (size_t)steps * (kStep / 8) * cols : 0));  // [group][16]
    const uint32_t col = i16 < cols ? i16 : cols - 1;                            // rows of the operand behind the last column: not stored

    // Loads come back in the order they were asked for: what is waited for first comes first.
    constexpr int early = 4;
    uint16_t sc[early];
    const uint32_t out = n0 + (tid & 15) < n ? n0 + (tid & 15) : n - 1;
#pragma unroll
    for (int i = 0; i < early; ++i) {
        const uint32_t at = (tid >> 4) + 32 * i;
        sc[i] = scales[(size_t)out * groups + (at < groups ? at : groups - 1)];
    }
    // Pieces of x, of eight inputs: the thread's first two are asked for before the weights, others (of several vectors, or
    // long ones) when those are stored.
    const uint32_t across = threads_across(vectors), first = tid & (across - 1), apart = 512 / across;
    const uint32_t rounds = (steps * (kStep / 8) + across - 1) / across, need = rounds * ((vectors + apart - 1) / apart);
    struct Place {
        uint32_t k8, m;
    };
    auto place = [&](uint32_t p) -> Place { return {first + across * (p % rounds), tid / across + apart * (p / rounds)}; };
    auto ask = [&](uint32_t p) -> Eight<DT> {
        const Place at = place(p);
        if (p < need && at.m < vectors && at.k8 * 8 < k) return load_eight<DT>(x, (m0 + at.m) * xstride + at.k8 * 8);
        return Eight<DT>{};
    };
    auto keep = [&](uint32_t p, const Eight<DT>& raw) {
        const Place at = place(p);
        if (p >= need || at.m >= vectors || at.k8 >= steps * (kStep / 8)) return;
        v4u c[parts];
        columns_of<DT>(raw, c);
#pragma unroll
        for (int q = 0; q < parts; ++q) xs[at.k8 * cols + at.m * parts + q] = c[q];
    };
    Eight<DT> raw[2];
    if constexpr (STAGED) {
        raw[0] = ask(0);
        raw[1] = ask(1);
    }
    const Row row = row_of(i16, k, g);
    const Buffer weights = weights_of(codes, n, k, n0, 16);
    constexpr int ahead = STAGED ? 3 : 2;
    v4u w[ahead], xa[ahead][4];
    const Buffer operands = buffer_of(xf + (size_t)blockIdx.y * steps * 256, STAGED ? 0 : (size_t)steps * 4096);
    auto fetch_x = [&](uint32_t j, v4u(&to)[4]) {
#pragma unroll
        for (int q = 0; q < 4; ++q) to[q] = load16(operands, j * 4096 + q * 1024 + lane * 16);
    };
#pragma unroll
    for (int p = 0; p < ahead; ++p) {
        w[p] = fetch(weights, row, wave + p * kWaves);
        if constexpr (!STAGED) fetch_x(wave + p * kWaves, xa[p]);
    }
#pragma unroll
    for (int i = 0; i < early; ++i) {
        const uint32_t at = (tid >> 4) + 32 * i;
        if (at < all_groups) ss[at * 16 + (tid & 15)] = at < groups ? sc[i] : (uint16_t)0;
    }
    for (uint32_t at = (tid >> 4) + 32 * early; at < all_groups; at += 32)
        ss[at * 16 + (tid & 15)] = at < groups ? scales[(size_t)out * groups + at] : (uint16_t)0;
    if constexpr (STAGED) {
        keep(0, raw[0]);
        keep(1, raw[1]);
        for (uint32_t p = 2; p < need; p += 2) {
            const Eight<DT> r0 = ask(p), r1 = ask(p + 1);
            keep(p, r0);
            keep(p + 1, r1);
        }
    }
    __syncthreads();

    v4f total = {0, 0, 0, 0};
    int64_t itotal[2] = {0, 0};
    const uint32_t minus12 = Kind<DT>::f16 ? 0xca00ca00u : 0xc140c140u;
    const v4u back = {minus12, minus12, minus12, minus12};
    auto add_group = [&](const v4f& acc, uint32_t group) {
        const uint32_t s = ss[group * 16 + i16];
        if constexpr (DT == ZK_I16) {
#pragma unroll
            for (int v = 0; v < 2; ++v) itotal[v] += (int64_t)((int)(acc[2 * v] * 2.0f) * 256 + (int)(acc[2 * v + 1] * 2.0f)) * (int64_t)s;
        } else {
            total += acc * (float)s;
        }
    };
    auto step = [&](uint32_t j, v4u& wr, v4u(&xr)[4]) {
        v4u r = wr, a[4];
        if constexpr (STAGED) {
            const v4u* at = xs + (j * (kStep / 8) + g) * cols + col;
#pragma unroll
            for (int q = 0; q < 4; ++q) a[q] = at[q * 4 * cols];
        } else {
#pragma unroll
            for (int q = 0; q < 4; ++q) a[q] = xr[q];
        }
        wr = fetch(weights, row, j + ahead * kWaves);
        if constexpr (!STAGED) fetch_x(j + ahead * kWaves, xr);
        transpose_rows(r);
        // two halves of a step side by side: their instructions do not wait for each other
        v4f acc[2];
        const uint32_t gr = j * kStep >> group_log;
        if (group_log == 5) {
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                v4f p = {0, 0, 0, 0};
                if constexpr (Kind<DT>::offset) p = product<DT>(a[q], back, p);
                add_group(product<DT>(a[q], widen<DT>(r[q]), p), gr + q);
            }
        } else {
#pragma unroll
            for (int f = 0; f < 2; ++f) {
                acc[f] = v4f{0, 0, 0, 0};
#pragma unroll
                for (int q = 2 * f; q < 2 * f + 2; ++q) {
                    if constexpr (Kind<DT>::offset) acc[f] = product<DT>(a[q], back, acc[f]);
                    acc[f] = product<DT>(a[q], widen<DT>(r[q]), acc[f]);
                }
            }
            if (group_log == 6) {
                add_group(acc[0], gr);
                add_group(acc[1], gr + 1);
            } else {
                add_group(acc[0] + acc[1], gr);
            }
        }
    };
    uint32_t j = wave;
    for (; j + (ahead - 1) * kWaves < steps; j += ahead * kWaves)
#pragma unroll
        for (int p = 0; p < ahead; ++p) step(j + p * kWaves, w[p], xa[p]);
#pragma unroll
    for (int p = 0; p < ahead - 1; ++p)
        if (j + p * kWaves < steps) step(j + p * kWaves, w[p], xa[p]);

    __syncthreads();
    if constexpr (DT == ZK_I16) {
        int64_t* red = (int64_t*)shared;  // [wave][vector][16]
#pragma unroll
        for (int v = 0; v < 2; ++v) red[(wave * 8 + 2 * g + v) * 16 + i16] = itotal[v];
        __syncthreads();
        if (tid < 128) {
            const uint32_t m = tid >> 4, o = tid & 15;
            int64_t sum = 0;
#pragma unroll
            for (int v = 0; v < kWaves; ++v) sum += red[(v * 8 + m) * 16 + o];
            if (m < vectors && n0 + o < n) ((int64_t*)y)[(m0 + m) * ystride + n0 + o] = sum;
        }
    } else {
        float* red = (float*)shared;  // [wave][column][16]
#pragma unroll
        for (int e = 0; e < 4; ++e) red[(wave * 16 + 4 * g + e) * 16 + i16] = total[e];
        __syncthreads();
        if (tid < 256) {
            const uint32_t m = tid >> 4, o = tid & 15;
            if (m < vectors && n0 + o < n) {
                float sum = 0.0f;
#pragma unroll
                for (int p = 0; p < parts; ++p)
#pragma unroll
                    for (int v = 0; v < kWaves; ++v) sum += red[(v * 16 + m * parts + p) * 16 + o];
                store_one<DT>(y, (m0 + m) * ystride + n0 + o, sum * step_unit);
            }
        }
    }
}

// x as operands: xf[block][k / 8][columns of a block], zero behind the last column and the last input (up to a step's end);
// with sums, -12 times the sum over each group of inputs, [block][group][columns of a block].  A block has `vectors`
// vectors.  Workgroup: one group, or eight of 16 bytes where nobody asks for sums.
template <int DT>
__global__ __launch_bounds__(kBlock) void k_w4_columns(v4u* xf, float* sums, const void* x, size_t xstride, size_t rows, uint32_t k,
                                                       uint32_t k8_all, uint32_t columns, uint32_t vectors, uint32_t group_log) {
    constexpr int parts = Kind<DT>::parts;
    const uint32_t block = blockIdx.y, per = sums ? 1u << (group_log - 3) : 8;  // pieces of eight inputs of a workgroup, 4, 8 or 16
    const uint32_t sub = threadIdx.x & (per - 1), k8 = blockIdx.x * per + sub;
    const size_t m0 = (size_t)block * vectors;
    for (uint32_t m = threadIdx.x / per; m * parts < columns; m += kBlock / per) {
        v4u c[parts];
#pragma unroll
        for (int p = 0; p < parts; ++p) c[p] = v4u{0, 0, 0, 0};
        if (m < vectors && m0 + m < rows && k8 * 8 < k)
            columns_of<DT>(load_eight<DT>(x, (m0 + m) * xstride + k8 * 8), c);
#pragma unroll
        for (int p = 0; p < parts; ++p) {
            const uint32_t col = m * parts + p;
            if (col >= columns) continue;
            if (k8 < k8_all) xf[((size_t)block * k8_all + k8) * columns + col] = c[p];
            if (!sums) continue;
            float sum = 0.0f;
#pragma unroll
            for (int i = 0; i < 4; ++i) sum += half_of<Kind<DT>::f16 ? ZK_F16 : ZK_BF16>(c[p][i], 0) + half_of<Kind<DT>::f16 ? ZK_F16 : ZK_BF16>(c[p][i], 1);
            for (uint32_t o = 1; o < per; o <<= 1) sum += __shfl_xor(sum, (int)o);
            if (sub == 0) sums[((size_t)block * (k8_all / per) + blockIdx.x) * columns + col] = -12.0f * sum;
        }
    }
}

// ---- many columns ----------------------------------------------------------------------------------------------------

// Workgroup: 64 NT outputs by 16 CT columns, chunks of two steps.  Wavefront w: outputs 16 NT (w mod 4) .., step w / 4 of a
// chunk.  Operands and sums come from k_w4_columns through registers, one or two chunks ahead, into LDS.
template <int CT, int NT, bool OFFSET>
struct ManyLds {
    static constexpr uint32_t C = 16 * CT, N = 64 * NT, x = 32 * C * 16, sums = OFFSET ? 8 * C * 4 : 0, scales = 8 * N * 2, bytes = x + sums + scales;
    static constexpr uint32_t meet = 4 * NT * CT * 64 * 16;  // also the outputs, C * N floats
    static constexpr uint32_t all = 2 * bytes > meet ? 2 * bytes : meet;
};
template <int DT, int CT, int NT, int GL>
__global__ __launch_bounds__(512) void k_w4_many(void* y, size_t ystride, const v4u* xf, const float* sums, size_t rows, const uint8_t* codes,
                                                 const uint16_t* scales, uint32_t n, uint32_t k, uint32_t vectors, float step_unit) {
    constexpr uint32_t group_log = GL;
    constexpr bool offset = Kind<DT>::offset;
    using L = ManyLds<CT, NT, offset>;
    constexpr uint32_t C = L::C, N = L::N;
    extern __shared__ v4u shared[];
    char* lds = (char*)shared;
    const uint32_t tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), g = lane >> 4, i16 = lane & 15, nw = wave & 3, kw = wave >> 2;
    const uint32_t n0 = blockIdx.x * N, block = blockIdx.y;
    const uint32_t steps = (k + kStep - 1) / kStep, k8_all = steps * (kStep / 8), chunks = (steps + 1) / 2;
    const uint32_t groups = (k + (1u << group_log) - 1) >> group_log, all_groups = k8_all >> (group_log - 3), each = 256u >> group_log;

    // What a thread brings of a chunk lies in a row with what its neighbours bring; behind the last input everything reads as 0.
    const Buffer operands = buffer_of(xf + (size_t)block * k8_all * C, (size_t)k8_all * C * 16);
    const Buffer offsets = buffer_of(sums + (offset ? (size_t)block * all_groups * C : 0), offset ? (size_t)all_groups * C * 4 : 0);
    const Buffer factors = buffer_of(scales + (size_t)n0 * groups, (size_t)(n - n0 < N ? n - n0 : N) * groups * 2);
    struct Load {
        v4u x[CT];
        float b[2];
        uint16_t s[NT];
    };
    // Chunks under way ahead of the one at work.  Two and one, us, 32001 x 5120: 32 vectors of bf16 33.3 and 38.5, 64 45.6 and
    // 44.7 (groups of 32: 66 and 50, registers spill): with four tiles the work is the longer part.
    constexpr int D = CT <= 2 ? 2 : 1;
    Load load[D];
    auto ask = [&](Load& to, uint32_t chunk) {
#pragma unroll
        for (int i = 0; i < CT; ++i) to.x[i] = load16(operands, (chunk * 32 * C + tid + 512 * i) * 16);
#pragma unroll
        for (int i = 0; offset && i < 2; ++i)
            to.b[i] = bits_float((uint32_t)__builtin_amdgcn_raw_buffer_load_b32(offsets, (int)((chunk * each * C + tid + 512 * i) * 4), 0, 0));
#pragma unroll
        for (int i = 0; i < NT; ++i) {
            const uint32_t p = tid + 512 * i, gr = chunk * each + p / N;
            to.s[i] = (uint16_t)__builtin_amdgcn_raw_buffer_load_b16(factors, (int)(gr < groups ? (p % N * groups + gr) * 2 : kNowhere), 0, 0);
        }
    };
    auto put = [&](const Load& from, uint32_t buf) {
        char* at = lds + buf * L::bytes;
#pragma unroll
        for (int i = 0; i < CT; ++i) ((v4u*)at)[tid + 512 * i] = from.x[i];
#pragma unroll
        for (int i = 0; offset && i < 2; ++i)
            if (tid + 512 * i < each * C) ((float*)(at + L::x))[tid + 512 * i] = from.b[i];
#pragma unroll
        for (int i = 0; i < NT; ++i)
            if (tid + 512 * i < each * N) ((uint16_t*)(at + L::x + L::sums))[tid + 512 * i] = from.s[i];
    };
    Row row[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) row[t] = row_of((nw * NT + t) * 16 + i16, k, g);
    const Buffer weights = weights_of(codes, n, k, n0, N);
    v4u w[D][NT];
#pragma unroll
    for (int p = 0; p < D; ++p) {
        ask(load[p], p);
#pragma unroll
        for (int t = 0; t < NT; ++t) w[p][t] = fetch(weights, row[t], kw + 2 * p);
        __builtin_amdgcn_sched_barrier(0);
    }

    v4f total[NT][CT];
    int64_t itotal[NT][CT][2];
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int c = 0; c < CT; ++c) {
            total[t][c] = v4f{0, 0, 0, 0};
            itotal[t][c][0] = itotal[t][c][1] = 0;
        }
    auto work = [&](uint32_t chunk, const int buf) {
        put(load[buf % D], buf);
        __syncthreads();
        ask(load[buf % D], chunk + D);
        v4u r[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            // moved, not renamed: the next load's registers are then the loop's own, and nothing waits for it at the loop's end
#pragma unroll
            for (int i = 0; i < 4; ++i) asm("v_mov_b32 %0, %1" : "=v"(r[t][i]) : "v"(w[buf % D][t][i]));
            w[buf % D][t] = fetch(weights, row[t], (chunk + D) * 2 + kw);
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int t = 0; t < NT; ++t) transpose_rows(r[t]);
        const char* at = lds + buf * L::bytes;
        const v4u* xs = (const v4u*)at + (kw * 16 + g) * C + i16;
        const float* bs = (const float*)(at + L::x) + 4 * g;
        const uint16_t* ss = (const uint16_t*)(at + L::x + L::sums) + nw * 16 * NT + i16;
        v4f acc[NT][CT];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const uint32_t gr = (kw * kStep + q * 32) >> group_log;
            if (q == 0 || (q == 2 && group_log <= 6) || group_log == 5) {
                // a group's sums start at what the codes' offset takes off
#pragma unroll
                for (int c = 0; c < CT; ++c) {
                    if constexpr (offset) acc[0][c] = *(const v4f*)(bs + gr * C + 16 * c);
                    else acc[0][c] = v4f{0, 0, 0, 0};
#pragma unroll
                    for (int t = 1; t < NT; ++t) acc[t][c] = acc[0][c];
                }
            }
            v4u f[NT];
#pragma unroll
            for (int t = 0; t < NT; ++t) f[t] = widen<DT>(r[t][q]);
#pragma unroll
            for (int c = 0; c < CT; ++c) {
                const v4u x = xs[q * 4 * C + 16 * c];
#pragma unroll
                for (int t = 0; t < NT; ++t) acc[t][c] = product<DT>(x, f[t], acc[t][c]);
            }
            if (q == 3 || (q & 1 && group_log <= 6) || group_log == 5) {
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    const uint32_t s = ss[gr * N + 16 * t];
#pragma unroll
                    for (int c = 0; c < CT; ++c) {
                        if constexpr (DT == ZK_I16) {
#pragma unroll
                            for (int v = 0; v < 2; ++v)
                                itotal[t][c][v] += (int64_t)((int)(acc[t][c][2 * v] * 2.0f) * 256 + (int)(acc[t][c][2 * v + 1] * 2.0f)) * (int64_t)s;
                        } else {
                            total[t][c] += acc[t][c] * (float)s;
                        }
                    }
                }
            }
        }
    };
    // in pairs, without a question between them (what is behind the last chunk is zeros), so that a wait names its own loads
    for (uint32_t chunk = 0; chunk < chunks; chunk += 2) {
        work(chunk, 0);
        work(chunk + 1, 1);
    }

    // the two halves of the inputs, then the columns of a vector
    __syncthreads();
    v4u* meet = shared + (size_t)nw * NT * CT * 64 + lane;
    if (kw == 1)
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int c = 0; c < CT; ++c)
                meet[(t * CT + c) * 64] = DT == ZK_I16 ? __builtin_bit_cast(v4u, itotal[t][c]) : __builtin_bit_cast(v4u, total[t][c]);
    __syncthreads();
    const size_t m0 = (size_t)block * vectors;
    if constexpr (DT == ZK_I16) {
        if (kw == 0)
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int c = 0; c < CT; ++c) {
                    struct Two {
                        int64_t v[2];
                    };
                    const Two other = __builtin_bit_cast(Two, meet[(t * CT + c) * 64]);
                    const uint32_t o = n0 + (nw * NT + t) * 16 + i16;
#pragma unroll
                    for (int v = 0; v < 2; ++v) {
                        const uint32_t m = 8 * c + 2 * g + v;
                        if (m < vectors && m0 + m < rows && o < n) ((int64_t*)y)[(m0 + m) * ystride + o] = itotal[t][c][v] + other.v[v];
                    }
                }
    } else {
        if (kw == 0)
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int c = 0; c < CT; ++c) total[t][c] += __builtin_bit_cast(v4f, meet[(t * CT + c) * 64]);
        __syncthreads();
        float* tile = (float*)shared;  // [column][output]
        if (kw == 0)
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int c = 0; c < CT; ++c)
#pragma unroll
                    for (int e = 0; e < 4; ++e) tile[(16 * c + 4 * g + e) * N + (nw * NT + t) * 16 + i16] = total[t][c][e];
        __syncthreads();
        for (uint32_t i = tid; i < vectors * N; i += 512) {
            const uint32_t m = i / N, o = i % N;
            if (m0 + m >= rows || n0 + o >= n) continue;
            float sum = 0.0f;
#pragma unroll
            for (int p = 0; p < Kind<DT>::parts; ++p) sum += tile[(m * Kind<DT>::parts + p) * N + o];
            store_one<DT>(y, (m0 + m) * ystride + n0 + o, sum * step_unit);
        }
    }
}

__global__ __launch_bounds__(kBlock) void k_w4_expand(int16_t* W, const uint8_t* codes, const uint16_t* scales, uint32_t n, uint32_t k,
                                                      uint32_t group_log) {
    // a thread: one output, eight inputs; consecutive threads are consecutive outputs, whose entries lie side by side in W
    const uint32_t out = blockIdx.x * kBlock + threadIdx.x;
    if (out >= n) return;
    const uint32_t groups = (k + (1u << group_log) - 1) >> group_log;
    for (uint32_t k8 = blockIdx.y; k8 < k >> 3; k8 += gridDim.y) {
        const uint32_t w = *(const uint32_t*)(codes + (size_t)out * (k >> 1) + k8 * 4);
        const int s = scales[(size_t)out * groups + ((k8 * 8) >> group_log)];
#pragma unroll
        for (int e = 0; e < 8; ++e) W[(size_t)(k8 * 8 + e) * n + out] = (int16_t)(((int)((w >> (4 * e)) & 15) - 8) * s);
    }
}

// How a call goes: its columns in blocks, and how x gets to them.
struct Way {
    bool staged;                // few columns, x in LDS
    uint32_t blocks, vectors;   // of columns, and the vectors of each
    uint32_t tiles;             // of 16 columns of a block; 1: few columns
    uint32_t k8;                // pieces of eight inputs, whole steps
    size_t operands, sums;      // in the workspace, bytes
};
size_t scales_bytes(uint32_t k8, uint32_t group_log) { return (size_t)(k8 >> (group_log - 3)) * 32; }  // of 16 outputs
template <int DT>
Way way_of(size_t rows, uint32_t n, uint32_t k, uint32_t group_log) {
    constexpr uint32_t parts = Kind<DT>::parts;
    Way w = {};
    w.k8 = (uint32_t)align_up(k, kStep) / 8;
    const bool between = n < kManyOutputs && rows * parts <= 16 * kBlocksOfFew;
    const bool tens = DT == ZK_F32 && between && rows > kTens && n >= kTensOutputs;
    if (scales_bytes(w.k8, group_log) <= kMostLds && (rows <= (size_t)Kind<DT>::vectors || (between && !tens))) {
        w.tiles = 1;
        w.vectors = Kind<DT>::vectors;
        w.blocks = (uint32_t)div_up(rows, w.vectors);
        w.staged = w.blocks == 1 && (size_t)w.k8 * 8 * rows * parts <= kStageHalves;
    } else {
        // blocks of at most 96 columns, as like as they can be, two, four or six tiles each
        const size_t most = tens ? kTens : 96 / parts;
        const size_t blocks = div_up(rows, most), v = div_up(rows, blocks);
        w.tiles = v * parts <= 32 ? 2 : v * parts <= 64 ? 4 : 6;
        w.vectors = (uint32_t)v;
        w.blocks = (uint32_t)div_up(rows, v);
    }
    if (!w.staged) w.operands = (size_t)w.blocks * w.k8 * w.tiles * 256;
    if (w.tiles > 1 && Kind<DT>::offset) w.sums = (size_t)w.blocks * (w.k8 / 4) * w.tiles * 64;  // of the shortest groups
    return w;
}
size_t way_bytes(const Way& w) {
    Carver cv(nullptr, 0);
    cv.take(w.operands);
    cv.take(w.sums);
    return w.operands ? cv.used() : 0;
}

struct Call {
    void* y;
    size_t ystride;
    const void* x;
    size_t xstride, rows;
    const uint8_t* codes;
    const uint16_t* scales;
    uint32_t n, k, group_log;
    float unit;
    void* ws;
    size_t ws_bytes;
    hipStream_t stream;
};

template <int DT, int CT, int NT, int GL>
int run_many(const Call& c, const Way& w, const v4u* xf, const float* sums) {
    const size_t lds = ManyLds<CT, NT, Kind<DT>::offset>::all;
    auto* kernel = k_w4_many<DT, CT, NT, GL>;
    if (lds > 65536) ZK_HIP_TRY(hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds));
    hipLaunchKernelGGL(kernel, dim3((unsigned)div_up(c.n, 64 * NT), w.blocks), dim3(512), lds, c.stream, c.y, c.ystride, xf, sums, c.rows,
                       c.codes, c.scales, c.n, c.k, w.vectors, c.unit * Kind<DT>::step);
    ZK_HIP_TRY(hipGetLastError());
    return ZK_OK;
}
template <int DT, int CT, int NT>
int run_many(const Call& c, const Way& w, const v4u* xf, const float* sums) {
    if constexpr (CT < 6)
        if (c.group_log == 5) return run_many<DT, CT, NT, 5>(c, w, xf, sums);
    return c.group_log == 6 ? run_many<DT, CT, NT, 6>(c, w, xf, sums) : run_many<DT, CT, NT, 7>(c, w, xf, sums);
}
template <int DT, int CT>
int run_many(const Call& c, const Way& w, const v4u* xf, const float* sums) {
    if constexpr (CT == 6)
        if (c.group_log == 5) return run_many<DT, CT, 1, 5>(c, w, xf, sums);
    return c.n >= kWide ? run_many<DT, CT, 2>(c, w, xf, sums) : run_many<DT, CT, 1>(c, w, xf, sums);
}

template <int DT>
int run(const Call& c) {
    const Way w = way_of<DT>(c.rows, c.n, c.k, c.group_log);
    v4u* xf = nullptr;
    float* sums = nullptr;
    if (w.operands) {
        if (!c.ws) return ZK_E_BUFSZ;
        Carver cv(c.ws, c.ws_bytes);
        xf = (v4u*)cv.take(w.operands);
        if (w.sums) sums = (float*)cv.take(w.sums);
        if (cv.overflow() || !xf || (w.sums && !sums)) return ZK_E_BUFSZ;
        const uint32_t per = sums ? 1u << (c.group_log - 3) : 8;
        hipLaunchKernelGGL((k_w4_columns<DT>), dim3((unsigned)div_up(w.k8, per), w.blocks), dim3(kBlock), 0, c.stream, xf, sums, c.x, c.xstride,
                           c.rows, c.k, w.k8, w.tiles * 16, w.vectors, c.group_log);
        ZK_HIP_TRY(hipGetLastError());
    }
    if (w.tiles == 1) {
        const uint32_t cols = (uint32_t)c.rows * Kind<DT>::parts;  // of a call that stages x
        size_t lds = (w.staged ? (size_t)w.k8 * cols * 16 : 0) + scales_bytes(w.k8, c.group_log);
        if (lds < 8192) lds = 8192;  // the sums at the end
        const dim3 grid((unsigned)div_up(c.n, 16), w.blocks);
        auto* kernel = w.staged ? (c.group_log == 5 ? k_w4_few<DT, true, 5> : c.group_log == 6 ? k_w4_few<DT, true, 6> : k_w4_few<DT, true, 7>)
                                : (c.group_log == 5 ? k_w4_few<DT, false, 5> : c.group_log == 6 ? k_w4_few<DT, false, 6> : k_w4_few<DT, false, 7>);
        if (lds > 65536) ZK_HIP_TRY(hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds));
        hipLaunchKernelGGL(kernel, grid, dim3(kWaves * 64), lds, c.stream, c.y, c.ystride, c.x, c.xstride, xf, c.rows, c.codes, c.scales, c.n,
                           c.k, c.unit * Kind<DT>::step);
        ZK_HIP_TRY(hipGetLastError());
        return ZK_OK;
    }
    return w.tiles == 2 ? run_many<DT, 2>(c, w, xf, sums) : w.tiles == 4 ? run_many<DT, 4>(c, w, xf, sums) : run_many<DT, 6>(c, w, xf, sums);
}

bool inputs_ok(size_t k) { return k >= 32 && k <= ((size_t)1 << 20) && k % 32 == 0; }
bool weights_ok(const uint8_t* codes, const uint16_t* scales, size_t n, size_t k, uint32_t group) {
    return codes && scales && aligned(codes, 16) && aligned(scales, 2) && n >= 1 && n <= ((size_t)1 << 24) && inputs_ok(k) &&
           (group == 32 || group == 64 || group == 128);
}

}  // namespace
}  // namespace zkmi

using namespace zkmi;

namespace {
template <int DT>
size_t workspace(size_t rows, uint32_t k) {  // whatever the number of outputs and the groups
    size_t most = 0;
    for (uint32_t n : {1u, kTensOutputs, 1u << 24})
        for (uint32_t group_log : {5u, 7u}) {  // where scales are the longest and the shortest
            const size_t need = way_bytes(way_of<DT>(rows, n, k, group_log));
            most = need > most ? need : most;
        }
    return most;
}
}  // namespace

extern "C" size_t w4_matvec_workspace_bytes(int dtype, size_t rows, size_t k) {
    if (!dtype_bytes(dtype) || rows == 0 || rows > kMostRows || !inputs_ok(k)) return 0;
    switch (dtype) {
        case ZK_F32: return workspace<ZK_F32>(rows, (uint32_t)k);
        case ZK_F16: return workspace<ZK_F16>(rows, (uint32_t)k);
        case ZK_BF16: return workspace<ZK_BF16>(rows, (uint32_t)k);
        default: return workspace<ZK_I16>(rows, (uint32_t)k);
    }
}

extern "C" int w4_matvec(void* y, size_t y_row_stride, const void* x, size_t x_row_stride, int dtype, size_t rows, const uint8_t* codes,
                         const uint16_t* scales, size_t n, size_t k, uint32_t group, float unit, void* ws, size_t ws_bytes, void* stream) {
    const size_t size = dtype_bytes(dtype);
    if (!size || !weights_ok(codes, scales, n, k, group) || rows > kMostRows) return ZK_E_BADARG;
    if (rows == 0) return ZK_OK;
    if (!x || !y || !aligned(x, 16) || !aligned(y, dtype == ZK_I16 ? 8 : size)) return ZK_E_BADARG;
    if (rows > 1 && (x_row_stride < k || y_row_stride < n || x_row_stride * size % 16)) return ZK_E_BADARG;
    const Call c = {y, y_row_stride, x, x_row_stride, rows, codes, scales, (uint32_t)n, (uint32_t)k, group == 32 ? 5u : group == 64 ? 6u : 7u,
                    unit, ws, ws_bytes, as_stream(stream)};
    switch (dtype) {
        case ZK_F32: return run<ZK_F32>(c);
        case ZK_F16: return run<ZK_F16>(c);
        case ZK_BF16: return run<ZK_BF16>(c);
        default: return run<ZK_I16>(c);
    }
}

extern "C" int w4_expand_i16(int16_t* W, const uint8_t* codes, const uint16_t* scales, size_t n, size_t k, uint32_t group, void* stream) {
    if (!W || !aligned(W, 2) || !weights_ok(codes, scales, n, k, group)) return ZK_E_BADARG;
    const uint32_t gl = group == 32 ? 5 : group == 64 ? 6 : 7;
    const unsigned across = (unsigned)div_up(n, kBlock), k8 = (unsigned)(k >> 3);
    hipLaunchKernelGGL(k_w4_expand, dim3(across, k8 < 65535 ? k8 : 65535), dim3(kBlock), 0, as_stream(stream), W, codes, scales,
                       (uint32_t)n, (uint32_t)k, gl);
    ZK_HIP_TRY(hipGetLastError());
    return ZK_OK;
}
