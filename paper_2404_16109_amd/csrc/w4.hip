// Products of a few vectors with a matrix of 4-bit weights, a scale for each group of inputs.
//
//   y[m][n] = unit * sum_g s[n][g] * sum_{k in g} c[n][k] x[m][k],   c = u - 8,  u a half byte.
//
// The sums over a group run on the matrix cores (16 x 16 x 32).  The first operand is x, a column of it to a row of the
// operand; the second holds 16 outputs' weights.  A half byte becomes a 16-bit float without a table or a subtraction:
// put into the top of the mantissa of 8.0 it is 8 + u/2 = (c + 24) / 2, exact in both 16-bit types, and -12 sum x is
// added by one more matrix instruction whose second operand is the constant -12.  What is accumulated is three times the
// size of the result's terms at most, so nothing is lost of 32-bit sums.  Types:
//   ZK_F16   x as it is.            ZK_BF16  x as it is.
//   ZK_F32   x as the sum of three bf16 (8 + 8 + 8 bits: exact), three columns.
//   ZK_I16   x = 256 h + l, two columns of whole numbers below 2^8; a group's sums are below 2^20 halves, exact in 32
//            bits, and everything after that is in 64-bit integers.
//
// Layout.  A lane loads 16 bytes, 32 inputs of one output: lane 16 g + i has output i, inputs 32 g .. 32 g + 31 of a step
// of 128.  An instruction wants inputs 8 g .. 8 g + 7 of ONE block of 32 in lane row g, so that what it adds up belongs
// to one group: four exchanges of lane rows transpose the 4 x 4 words.  Of a word's eight half bytes i and i + 4 come to
// lie in one register, so x is kept in the order 0 4 1 5 2 6 3 7.
#include "serve_dev.h"

namespace zkmi {
namespace {

static const int kStep = 128;                      // inputs a wavefront takes at a time
static const int kWaves = 8;
static const uint32_t kStageHalves = 16384;        // 32 KiB of x in LDS

template <int DT>
struct Kind {
    static constexpr int parts = DT == ZK_F32 ? 3 : DT == ZK_I16 ? 2 : 1;  // columns of a vector
    static constexpr int vectors = 16 / parts;                             // vectors of a call's 16 columns
    static constexpr bool f16 = DT == ZK_F16;
};

template <int DT>
__device__ __forceinline__ v4f product(v4u a, v4u b, v4f c) {
    if constexpr (Kind<DT>::f16) return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8h, a), __builtin_bit_cast(v8h, b), c, 0, 0, 0);
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8b, a), __builtin_bit_cast(v8b, b), c, 0, 0, 0);
}

// Eight half bytes as 8 + u/2.
template <int DT>
__device__ __forceinline__ v4u widen(uint32_t w) {
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

// Inputs k .. k+7 of a vector as its columns' operands, in the order 0 4 1 5 2 6 3 7.
template <int DT>
__device__ __forceinline__ void columns_of(const void* x, size_t at, v4u (&out)[Kind<DT>::parts]) {
    if constexpr (DT == ZK_F16 || DT == ZK_BF16) {
        const v4u r = *(const v4u*)((const uint16_t*)x + at);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t lo = r[i >> 1], hi = r[2 + (i >> 1)];  // elements i and i + 4
            out[0][i] = i & 1 ? (lo >> 16) | (hi & 0xffff0000u) : (lo & 0xffffu) | (hi << 16);
        }
    } else if constexpr (DT == ZK_I16) {
        const v4u r = *(const v4u*)((const uint16_t*)x + at);
        auto part = [&](int e, int p) -> uint32_t {
            const int v = (int16_t)(r[e >> 1] >> (16 * (e & 1)));
            return half_bits<ZK_BF16>((float)(p == 0 ? v >> 8 : v & 255));
        };
#pragma unroll
        for (int p = 0; p < 2; ++p)
#pragma unroll
            for (int i = 0; i < 4; ++i) out[p][i] = part(i, p) | (part(i + 4, p) << 16);
    } else {
        const v4f* f = (const v4f*)((const float*)x + at);
        v4f r[2] = {f[0], f[1]};
#pragma unroll
        for (int p = 0; p < 3; ++p)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t a = half_bits<ZK_BF16>(r[0][i]), b = half_bits<ZK_BF16>(r[1][i]);
                out[p][i] = a | (b << 16);
                r[0][i] -= bits_float(a << 16);
                r[1][i] -= bits_float(b << 16);
            }
    }
}

// Workgroup: 16 outputs, up to 16 columns; its eight wavefronts share out the steps and add up at the end.
template <int DT>
__global__ __launch_bounds__(kWaves * 64) void k_w4_few(void* y, size_t ystride, const void* x, size_t xstride, size_t rows,
                                                        const uint8_t* codes, const uint16_t* scales, uint32_t n, uint32_t k,
                                                        uint32_t group_log, uint32_t chunk, float unit2) {
    constexpr int parts = Kind<DT>::parts;
    extern __shared__ v4u shared[];
    const uint32_t tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, g = lane >> 4, i16 = lane & 15;
    const uint32_t n0 = blockIdx.x * 16;
    const size_t m0 = (size_t)blockIdx.y * Kind<DT>::vectors;
    const uint32_t vectors = rows - m0 < (size_t)Kind<DT>::vectors ? (uint32_t)(rows - m0) : Kind<DT>::vectors;
    const uint32_t cols = vectors * parts;
    v4u* xs = shared;                                                // [chunk / 8][cols]
    uint16_t* ss = (uint16_t*)(shared + (size_t)(chunk >> 3) * cols);  // [chunk / group][16]
    const uint32_t groups = (k + (1u << group_log) - 1) >> group_log, chunk_groups = chunk >> group_log;
    const uint32_t col = i16 < cols ? i16 : cols - 1;                // rows of the operand behind the last column: not stored

    const uint32_t out = n0 + i16 < n ? n0 + i16 : n - 1;
    const uint8_t* wrow = codes + (size_t)out * (k >> 1) + g * 16;
    const uint32_t steps = (k + kStep - 1) / kStep;
    auto fetch = [&](uint32_t j) -> v4u {
        if (j < steps && j * kStep + g * 32 < k) return __builtin_nontemporal_load((const v4u*)(wrow + (size_t)j * (kStep / 2)));
        return v4u{0, 0, 0, 0};
    };
    constexpr int ahead = 4;
    v4u w[ahead];
#pragma unroll
    for (int p = 0; p < ahead; ++p) w[p] = fetch(wave + p * kWaves);

    v4f total = {0, 0, 0, 0};
    int64_t itotal[2] = {0, 0};
    const uint32_t minus12 = Kind<DT>::f16 ? 0xca00ca00u : 0xc140c140u;
    for (uint32_t k0 = 0; k0 < k; k0 += chunk) {
        if (k0) __syncthreads();
        for (uint32_t t = tid; t < (chunk >> 3) * vectors; t += kWaves * 64) {
            const uint32_t k8 = t % (chunk >> 3), m = t / (chunk >> 3);
            v4u c[parts];
#pragma unroll
            for (int p = 0; p < parts; ++p) c[p] = v4u{0, 0, 0, 0};
            if (k0 + k8 * 8 < k) columns_of<DT>(x, (m0 + m) * xstride + k0 + k8 * 8, c);
#pragma unroll
            for (int p = 0; p < parts; ++p) xs[k8 * cols + m * parts + p] = c[p];
        }
        for (uint32_t t = tid; t < chunk_groups * 16; t += kWaves * 64) {
            const uint32_t gr = t % chunk_groups, o = t / chunk_groups, at = (k0 >> group_log) + gr;
            ss[gr * 16 + o] = at < groups && n0 + o < n ? scales[(size_t)(n0 + o) * groups + at] : (uint16_t)0;
        }
        __syncthreads();
        const uint32_t last = (k0 + chunk < k ? k0 + chunk : k);
#pragma unroll 4
        for (uint32_t j = k0 / kStep + wave; j * kStep < last; j += kWaves) {
            v4u r = w[0];
#pragma unroll
            for (int p = 0; p + 1 < ahead; ++p) w[p] = w[p + 1];
            w[ahead - 1] = fetch(j + ahead * kWaves);
            transpose_rows(r);
            const uint32_t kk = j * kStep - k0;
            v4f acc = {0, 0, 0, 0};
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const v4u a = xs[((kk >> 3) + q * 4 + g) * cols + col];
                acc = product<DT>(a, v4u{minus12, minus12, minus12, minus12}, acc);
                acc = product<DT>(a, widen<DT>(r[q]), acc);
                if (q == 3 || (q & 1 && group_log <= 6) || group_log == 5) {
                    const uint32_t s = ss[((kk + q * 32) >> group_log) * 16 + i16];
                    if constexpr (DT == ZK_I16) {
#pragma unroll
                        for (int v = 0; v < 2; ++v)
                            itotal[v] += (int64_t)((int)(acc[2 * v] * 2.0f) * 256 + (int)(acc[2 * v + 1] * 2.0f)) * (int64_t)s;
                    } else {
                        total += acc * (float)s;
                    }
                    acc = v4f{0, 0, 0, 0};
                }
            }
        }
    }

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
                store_one<DT>(y, (m0 + m) * ystride + n0 + o, sum * unit2);
            }
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

template <int DT>
int run(void* y, size_t ystride, const void* x, size_t xstride, size_t rows, const uint8_t* codes, const uint16_t* scales, uint32_t n,
        uint32_t k, uint32_t group_log, float unit, hipStream_t stream) {
    constexpr int vectors = Kind<DT>::vectors, parts = Kind<DT>::parts;
    const uint32_t cols = (uint32_t)(rows < (size_t)vectors ? rows : vectors) * parts;
    uint32_t chunk = kStageHalves / cols / (kStep * kWaves) * (kStep * kWaves);  // at most 16 columns: at least one step each
    const uint32_t whole = (uint32_t)align_up(k, kStep * kWaves);
    if (chunk > whole) chunk = whole;
    size_t lds = (size_t)(chunk >> 3) * cols * 16 + (size_t)(chunk >> group_log) * 32;
    if (lds < 8192) lds = 8192;  // the sums at the end
    for (size_t r0 = 0; r0 < rows; r0 += (size_t)65535 * vectors) {  // the grid's second dimension ends there
        const size_t r = rows - r0 < (size_t)65535 * vectors ? rows - r0 : (size_t)65535 * vectors;
        hipLaunchKernelGGL((k_w4_few<DT>), dim3((unsigned)div_up(n, 16), (unsigned)div_up(r, vectors)), dim3(kWaves * 64), lds, stream,
                           (char*)y + r0 * ystride * (DT == ZK_I16 ? 8 : dtype_bytes(DT)), ystride,
                           (const char*)x + r0 * xstride * dtype_bytes(DT), xstride, r, codes, scales, n, k, group_log, chunk, unit * 2.0f);
    }
    ZK_HIP_TRY(hipGetLastError());
    return ZK_OK;
}

bool weights_ok(const uint8_t* codes, const uint16_t* scales, size_t n, size_t k, uint32_t group) {
    return codes && scales && aligned(codes, 16) && aligned(scales, 2) && n >= 1 && n <= ((size_t)1 << 24) && k >= 32 &&
           k <= ((size_t)1 << 24) && k % 32 == 0 && (group == 32 || group == 64 || group == 128);
}

}  // namespace
}  // namespace zkmi

using namespace zkmi;

extern "C" size_t w4_matvec_workspace_bytes(int dtype, size_t rows, size_t k) {
    (void)dtype;
    (void)rows;
    (void)k;
    return 0;
}

extern "C" int w4_matvec(void* y, size_t y_row_stride, const void* x, size_t x_row_stride, int dtype, size_t rows, const uint8_t* codes,
                         const uint16_t* scales, size_t n, size_t k, uint32_t group, float unit, void* ws, size_t ws_bytes, void* stream) {
    (void)ws;
    (void)ws_bytes;
    const size_t size = dtype_bytes(dtype);
    if (!size || !weights_ok(codes, scales, n, k, group)) return ZK_E_BADARG;
    if (rows == 0) return ZK_OK;
    if (!x || !y || !aligned(x, 16) || !aligned(y, dtype == ZK_I16 ? 8 : size)) return ZK_E_BADARG;
    if (rows > 1 && (x_row_stride < k || y_row_stride < n || x_row_stride * size % 16)) return ZK_E_BADARG;
    const uint32_t gl = group == 32 ? 5 : group == 64 ? 6 : 7;
    hipStream_t s = as_stream(stream);
    switch (dtype) {
        case ZK_F32: return run<ZK_F32>(y, y_row_stride, x, x_row_stride, rows, codes, scales, (uint32_t)n, (uint32_t)k, gl, unit, s);
        case ZK_F16: return run<ZK_F16>(y, y_row_stride, x, x_row_stride, rows, codes, scales, (uint32_t)n, (uint32_t)k, gl, unit, s);
        case ZK_BF16: return run<ZK_BF16>(y, y_row_stride, x, x_row_stride, rows, codes, scales, (uint32_t)n, (uint32_t)k, gl, unit, s);
        default: return run<ZK_I16>(y, y_row_stride, x, x_row_stride, rows, codes, scales, (uint32_t)n, (uint32_t)k, gl, unit, s);
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
