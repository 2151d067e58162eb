// Products of 8-bit integers: y[m][i] = (sum_j x[m][j] w[i][j]) * x_scales[m] * w_scales[i], or the sums themselves.
//
// Sums are exact in 32 bits (|x w| <= 2^14, k < 2^17), in whatever order: parts of k may be added up anywhere.
//
// Few rows (k_few: up to 32): the weights are read once, straight into registers, and bound the call.  A workgroup has 16 to 64
// outputs, its eight wavefronts share k in steps of 128, so that every row of weights is read in whole lines.  Measured, weights from HBM:
// one row by 13824 x 5120 16.8 us, 4.2 TB/s; 32 rows 20 us.  One row by 5120 x 5120 8.4 us where the bytes alone take 5.1: latency.
// Many rows (k_tiles): tiles of x and w come through LDS, put there by loads that pass no register, a step of 128 ahead; 16-byte
// pieces lie in LDS at piece ^ ((row / 2) & 7): rows of 128 bytes lie in one half of the banks or the other, so 16 neighbouring rows
// answer from all of them (no conflict is counted).  One barrier a step, before its last quarter, the loads among that quarter's
// products.  Measured: 8192 x 13824 x 5120 520 us, 2.2 P operations/s, 8192^3 2.4 (a library's product 2.2 and 2.4): the matrix cores are
// 61% busy at 1.84 GHz, to which the card's power brings the clock.  Stages of 64 of k, four or five ahead, took 645 us where this took 584.
// Where there are fewer tiles than the chip holds, workgroups share k and k_join adds up (333 rows by 5120 x 13824: 33 us and 6).
#include "i8_plan.h"
#include "serve_dev.h"

#pragma clang fp contract(off)

namespace zkmi {
namespace {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef int v16i __attribute__((ext_vector_type(16)));

struct Args {
    void* y;
    size_t yrow;
    const int8_t* x;
    size_t xrow;
    const float* xs;
    const int8_t* w;
    const float* ws;
    uint32_t rows, n, k;
    uint32_t splits, each;  // of k: steps of kStep to a part
    int32_t* parts;         // [split][row][n_pad]
    uint32_t n_pad;
    bool quads, wide;       // y takes four outputs, or 16 bytes, at once
};

// Four outputs of a row, from n0 on: those below n are stored.
template <int Y>
__device__ __forceinline__ void put_quad(const Args& a, uint32_t row, uint32_t n0, v4i s) {
    if (n0 >= a.n) return;
    const size_t at = (size_t)row * a.yrow + n0;
    if constexpr (Y == ZK_I32) {
        int32_t* y = (int32_t*)a.y + at;
        if (a.quads && n0 + 4 <= a.n) *(v4i*)y = s;
        else
            for (uint32_t e = 0; e < 4 && n0 + e < a.n; ++e) y[e] = s[e];
    } else {
        const float xs = a.xs[row];
        float f[4];
#pragma unroll
        for (uint32_t e = 0; e < 4; ++e) f[e] = as_it_is((float)s[e] * xs * (n0 + e < a.n ? a.ws[n0 + e] : 0.0f));
        if (a.quads && n0 + 4 <= a.n) {
            if constexpr (Y == ZK_F32) *(v4f*)((float*)a.y + at) = v4f{f[0], f[1], f[2], f[3]};
            else
                *(uint2*)((uint16_t*)a.y + at) = make_uint2((uint32_t)half_bits<Y>(f[0]) | ((uint32_t)half_bits<Y>(f[1]) << 16),
                                                            (uint32_t)half_bits<Y>(f[2]) | ((uint32_t)half_bits<Y>(f[3]) << 16));
        } else {
            for (uint32_t e = 0; e < 4 && n0 + e < a.n; ++e) store_one<Y>(a.y, at + e, f[e]);
        }
    }
}
template <int Y>
__device__ __forceinline__ void finish_quad(const Args& a, uint32_t split, uint32_t row, uint32_t n0, v4i s) {
    if (a.splits == 1) return put_quad<Y>(a, row, n0, s);
    if (n0 < a.n) *(v4i*)(a.parts + ((size_t)split * a.rows + row) * a.n_pad + n0) = s;
}

// ---- few rows --------------------------------------------------------------------------------------------------------

// RT: tiles of 16 rows; NT: of 16 outputs.  Lane 16 g + i: row (output) i of a tile, bytes 16 g .. 16 g + 15 of 64.
static const int kAhead = 3;
template <int RT, int NT, int Y>
__global__ __launch_bounds__(64 * kWaves) void k_few(Args a) {
    __shared__ v4i red[kWaves][RT * NT][64];
    const uint32_t tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), g = lane >> 4, i16 = lane & 15;
    const uint32_t n0 = blockIdx.x * 16 * NT, split = blockIdx.y;
    const uint32_t steps = (a.k + kStep - 1) / kStep, first = split * a.each, last = first + a.each < steps ? first + a.each : steps;
    const int8_t* w[NT];
    const int8_t* x[RT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const uint32_t o = n0 + 16 * t + i16;
        w[t] = a.w + (size_t)(o < a.n ? o : a.n - 1) * a.k;
    }
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        const uint32_t r = 16 * t + i16;
        x[t] = a.x + (size_t)(r < a.rows ? r : a.rows - 1) * a.xrow;
    }
    v4i acc[RT][NT];
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int t = 0; t < NT; ++t) acc[r][t] = v4i{0, 0, 0, 0};
    v4i wr[kAhead][NT][2], xr[kAhead][RT][2];
    // Every load is made: bytes behind k are the row's first, and zeros of x.
    auto load = [&](uint32_t s, v4i(&wp)[NT][2], v4i(&xp)[RT][2]) {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const uint32_t j = s * kStep + 64 * u + 16 * g;
            const uint32_t at = j < a.k ? j : 0;
#pragma unroll
            for (int t = 0; t < NT; ++t) wp[t][u] = *(const v4i*)(w[t] + at);
#pragma unroll
            for (int t = 0; t < RT; ++t) xp[t][u] = *(const v4i*)(x[t] + at);
        }
    };
    auto multiply = [&](uint32_t s, const v4i(&wp)[NT][2], const v4i(&xp)[RT][2]) {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const bool in = s * kStep + 64 * u + 16 * g < a.k;
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                const v4i q = in ? xp[r][u] : v4i{0, 0, 0, 0};
#pragma unroll
                for (int t = 0; t < NT; ++t) acc[r][t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wp[t][u], q, acc[r][t], 0, 0, 0);
            }
        }
    };
#pragma unroll
    for (int p = 0; p < kAhead; ++p)
        if (first + wave + p * kWaves < last) load(first + wave + p * kWaves, wr[p], xr[p]);
    for (uint32_t s = first + wave; s < last; s += kAhead * kWaves) {
#pragma unroll
        for (int p = 0; p < kAhead; ++p) {
            if (s + p * kWaves < last) {
                multiply(s + p * kWaves, wr[p], xr[p]);
                if (s + (p + kAhead) * kWaves < last) load(s + (p + kAhead) * kWaves, wr[p], xr[p]);
            }
        }
    }
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int t = 0; t < NT; ++t) red[wave][r * NT + t][lane] = acc[r][t];
    __syncthreads();
    for (uint32_t i = tid; i < RT * NT * 64; i += 64 * kWaves) {
        const uint32_t q = i >> 6, l = i & 63, row = 16 * (q / NT) + (l & 15);
        if (row >= a.rows) continue;
        v4i sum = red[0][q][l];
#pragma unroll
        for (int v = 1; v < kWaves; ++v) sum += red[v][q][l];
        finish_quad<Y>(a, split, row, n0 + 16 * (q % NT) + 4 * (l >> 4), sum);
    }
}

// ---- many rows -------------------------------------------------------------------------------------------------------

typedef __attribute__((address_space(3))) void lds_void;
#define kOutside 0xfffffff0u  // an offset that no tile reaches: loads from there give zeros

// What lanes of a wavefront have written to LDS is there for its other lanes, and what they have read may be written over.
__device__ __forceinline__ void lanes_meet() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// A wavefront's outputs, from the accumulators (lane: one row, four outputs side by side) through LDS to memory (16 bytes of a row a lane).
template <int Y, int MO, int NR>
__device__ __forceinline__ void store_tile(const Args& a, const v16i (&acc)[MO][NR], int8_t* corner, const float* scales, uint32_t row0, uint32_t n0, void* to,
                                           size_t stride, bool wide) {
    constexpr int size = Y == ZK_I32 || Y == ZK_F32 ? 4 : 2, G = 8 / size < MO ? 8 / size : MO;  // tiles of 32 outputs at a time
    constexpr uint32_t row_bytes = 32 * G * size, pitch = row_bytes + 16, lanes = row_bytes / 16, each = 16 / size;
    const uint32_t lane = threadIdx.x & 63, half = lane >> 5, i32 = lane & 31;
#pragma unroll
    for (int r = 0; r < NR; ++r) {
        float xs = 0.0f;
        if constexpr (Y != ZK_I32) {
            const uint32_t row = row0 + 32 * r + i32;
            xs = a.xs[row < a.rows ? row : a.rows - 1];
        }
#pragma unroll
        for (int g = 0; g < MO; g += G) {
#pragma unroll
            for (int o = 0; o < G; ++o)
#pragma unroll
                for (int e = 0; e < 16; e += 4) {
                    const uint32_t out = 32 * o + 2 * e + 4 * half;
                    const v4i s = {acc[g + o][r][e], acc[g + o][r][e + 1], acc[g + o][r][e + 2], acc[g + o][r][e + 3]};
                    int8_t* at = corner + i32 * pitch + out * size;
                    if constexpr (Y == ZK_I32) *(v4i*)at = s;
                    else {
                        const v4f ws = *(const v4f*)(scales + 32 * g + out);
                        v4f f;
#pragma unroll
                        for (int q = 0; q < 4; ++q) f[q] = as_it_is((float)s[q] * xs * ws[q]);
                        if constexpr (Y == ZK_F32) *(v4f*)at = f;
                        else
                            *(uint2*)at = make_uint2((uint32_t)half_bits<Y>(f[0]) | ((uint32_t)half_bits<Y>(f[1]) << 16),
                                                     (uint32_t)half_bits<Y>(f[2]) | ((uint32_t)half_bits<Y>(f[3]) << 16));
                    }
                }
            lanes_meet();
#pragma unroll
            for (uint32_t q = 0; q < 32 * lanes / 64; ++q) {
                const uint32_t in = q * (64 / lanes) + lane / lanes, row = row0 + 32 * r + in, c = lane % lanes, out = n0 + 32 * g + c * each;
                const v4u v = *(const v4u*)(corner + in * pitch + c * 16);
                if (row >= a.rows || out >= a.n) continue;
                const size_t at = (size_t)row * stride + out;
                if (wide && out + each <= a.n) {
                    *(v4u*)((int8_t*)to + at * size) = v;
                } else {
#pragma unroll
                    for (uint32_t e = 0; e < each; ++e) {
                        if (out + e >= a.n) continue;
                        if constexpr (size == 4) ((uint32_t*)to)[at + e] = v[e];
                        else ((uint16_t*)to)[at + e] = (uint16_t)(v[e >> 1] >> (16 * (e & 1)));
                    }
                }
            }
            lanes_meet();
        }
    }
}

// MO, NR: tiles of 32 outputs and of 32 rows that a wavefront has; WO x WR wavefronts.
template <int MO, int NR, int WO, int WR, int Y>
__global__ __launch_bounds__(64 * WO * WR) void k_tiles(Args a, uint32_t row_tiles, uint32_t out_tiles) {
#if defined(__HIP_DEVICE_COMPILE__)  // the host has no type for a buffer's descriptor
    constexpr uint32_t waves = WO * WR, outs = 32 * MO * WO, rows = 32 * NR * WR;
    constexpr int loads_w = outs / 8 / waves, loads_x = rows / 8 / waves;  // of a wavefront in a step: eight rows each
    __shared__ __attribute__((aligned(16))) int8_t s0[(outs + rows) * kStep];
    __shared__ __attribute__((aligned(16))) int8_t s1[(outs + rows) * kStep];
    __shared__ __attribute__((aligned(16))) float scales[outs];  // of the tile's outputs
    const uint32_t lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), half = lane >> 5, i32 = lane & 31;
    const uint32_t wo = wave % WO, wr = wave / WO, split = blockIdx.y;

    // Workgroups go to the eight XCDs in turn; each gets tiles that lie together, eight row tiles by as many of outputs as come.
    uint32_t id = blockIdx.x;
    {
        const uint32_t total = row_tiles * out_tiles, q = total >> 3, rest = total & 7, xcd = id & 7, in = id >> 3;
        id = xcd * q + (xcd < rest ? xcd : rest) + in;
    }
    const uint32_t band = id / (8 * out_tiles), in_band = id - band * 8 * out_tiles;
    const uint32_t band_rows = row_tiles - band * 8 < 8 ? row_tiles - band * 8 : 8;
    const uint32_t r0 = (band * 8 + in_band % band_rows) * rows, o0 = in_band / band_rows * outs;

    const uint32_t steps = (a.k + kStep - 1) / kStep, first = split * a.each, last = first + a.each < steps ? first + a.each : steps;
    const uint32_t w_rows = a.n - o0 < outs ? a.n - o0 : outs, x_rows = a.rows - r0 < rows ? a.rows - r0 : rows;
    __amdgpu_buffer_rsrc_t wb = __builtin_amdgcn_make_buffer_rsrc((void*)(a.w + (size_t)o0 * a.k), 0, (w_rows - 1) * a.k + a.k, 0x00020000);
    __amdgpu_buffer_rsrc_t xb = __builtin_amdgcn_make_buffer_rsrc((void*)(a.x + (size_t)r0 * a.xrow), 0, (x_rows - 1) * (uint32_t)a.xrow + a.k, 0x00020000);
    // A lane brings one piece of row lane / 8 of each eight; which eight of 16 they are is the same in all of its loads.
    static_assert(waves % 2 == 0, "");
    const uint32_t sub = lane >> 3, piece = ((lane & 7) ^ (4 * (wave & 1) + (sub >> 1))) * 16;
    uint32_t w_at[loads_w], x_at[loads_x];
#pragma unroll
    for (int i = 0; i < loads_w; ++i) {
        const uint32_t r = (i * waves + wave) * 8 + sub;
        w_at[i] = r < w_rows ? r * a.k + piece : kOutside;
    }
#pragma unroll
    for (int i = 0; i < loads_x; ++i) {
        const uint32_t r = (i * waves + wave) * 8 + sub;
        x_at[i] = r < x_rows ? r * (uint32_t)a.xrow + piece : kOutside;
    }
    const uint32_t k_end = last * kStep < a.k ? last * kStep : a.k;
    // Before the loads of a step that reaches behind the part: pieces there are zeros, from then on.
    auto trim = [&](uint32_t step) {
        if ((step + 1) * kStep > k_end && step * kStep + piece >= k_end) {
#pragma unroll
            for (int i = 0; i < loads_w; ++i) w_at[i] = kOutside;
#pragma unroll
            for (int i = 0; i < loads_x; ++i) x_at[i] = kOutside;
        }
    };
    auto load = [&](uint32_t step, int8_t* to, int i) {
        const uint32_t j = step * kStep < k_end ? step * kStep : 0;
        if (i < loads_w) __builtin_amdgcn_raw_ptr_buffer_load_lds(wb, (lds_void*)(to + (i * waves + wave) * 1024), 16, w_at[i < loads_w ? i : 0], j, 0, 0);
        else __builtin_amdgcn_raw_ptr_buffer_load_lds(xb, (lds_void*)(to + outs * kStep + ((i - loads_w) * waves + wave) * 1024), 16, x_at[i < loads_w ? 0 : i - loads_w], j, 0, 0);
    };
    auto fetch = [&](uint32_t step, int8_t* to) {
        trim(step);
#pragma unroll
        for (int i = 0; i < loads_w + loads_x; ++i) load(step, to, i);
    };
    v16i acc[MO][NR];
#pragma unroll
    for (int o = 0; o < MO; ++o)
#pragma unroll
        for (int r = 0; r < NR; ++r) acc[o][r] = v16i{0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0};
    const uint32_t w_row = (wo * MO * 32 + i32) * kStep, x_row = outs * kStep + (wr * NR * 32 + i32) * kStep;
    // Operands are read a quarter of a step ahead of the products that take them, those of the next step's first quarter too: the
    // wait for that step and for everybody to be done with this one lies before the last quarter's products.
    v4i w[2][MO], x[2][NR];
    auto read = [&](const int8_t* from, int q) {
        const uint32_t at = ((2 * q + half) ^ ((i32 >> 1) & 7)) * 16;
#pragma unroll
        for (int r = 0; r < NR; ++r) x[q & 1][r] = *(const v4i*)(from + x_row + r * 32 * kStep + at);
#pragma unroll
        for (int o = 0; o < MO; ++o) w[q & 1][o] = *(const v4i*)(from + w_row + o * 32 * kStep + at);
    };
    auto multiply = [&](int q, auto between) {
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int o = 0; o < MO; ++o)
#pragma unroll
            for (int r = 0; r < NR; ++r) {
                acc[o][r] = __builtin_amdgcn_mfma_i32_32x32x32_i8(w[q & 1][o], x[q & 1][r], acc[o][r], 0, 0, 0);
                between(o * NR + r);
            }
        __builtin_amdgcn_sched_barrier(0);
    };
    const auto nothing = [](int) {};
    // Every operand of a step is in registers, and what is on its way to LDS has come.
    auto turn = [] {
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        __syncthreads();
    };
    auto step = [&](uint32_t s, int8_t* from, const int8_t* other) {
        read(from, 1);
        multiply(0, nothing);
        read(from, 2);
        multiply(1, nothing);
        read(from, 3);
        multiply(2, nothing);
        turn();
        read(other, 0);
        trim(s + 2);
        multiply(3, [&](int m) {  // the loads among the products
            constexpr int each = (loads_w + loads_x + MO * NR - 1) / (MO * NR);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = m * each; i < (m + 1) * each && i < loads_w + loads_x; ++i) load(s + 2, from, i);
            __builtin_amdgcn_sched_barrier(0);
        });
    };
    if (Y != ZK_I32 && a.splits == 1)
        for (uint32_t i = threadIdx.x; i < outs; i += 64 * waves) scales[i] = a.ws[o0 + i < a.n ? o0 + i : a.n - 1];
    fetch(first, s0);
    turn();
    read(s0, 0);
    fetch(first + 1, s1);
#pragma unroll 1
    for (uint32_t s = first; s < last; s += 2) {
        step(s, s0, s1);
        step(s + 1, s1, s0);
    }
    // Nothing is on its way to LDS any more, and nobody reads there: each wavefront turns its outputs over in a corner of its own, so
    // that a row's lie side by side and leave in whole lines.  (Stored from the accumulators, eight bytes to a lane, they took a fifth
    // of the call: 8192 x 13824 x 5120 590 us, 460 without any.)
    turn();
    int8_t* corner = (wave & 1 ? s1 : s0) + (wave >> 1) * (32 * (256 + 16));
    static_assert((waves / 2) * 32 * (256 + 16) <= sizeof(s0), "");
    if (a.splits == 1) store_tile<Y, MO, NR>(a, acc, corner, scales + wo * MO * 32, r0 + wr * NR * 32, o0 + wo * MO * 32, a.y, a.yrow, a.wide);
    else store_tile<ZK_I32, MO, NR>(a, acc, corner, scales, r0 + wr * NR * 32, o0 + wo * MO * 32, a.parts + (size_t)split * a.rows * a.n_pad, a.n_pad, true);
#endif
}

template <int Y>
__global__ __launch_bounds__(kBlock) void k_join(Args a) {
    const uint32_t quads = a.n_pad >> 2;
    const size_t i = (size_t)blockIdx.x * kBlock + threadIdx.x;
    const size_t row = i / quads;
    if (row >= a.rows) return;
    const uint32_t n0 = (uint32_t)(i - row * quads) * 4;
    v4i s = {0, 0, 0, 0};
#pragma unroll 4
    for (uint32_t p = 0; p < a.splits; ++p) s += *(const v4i*)(a.parts + ((size_t)p * a.rows + row) * a.n_pad + n0);
    put_quad<Y>(a, (uint32_t)row, n0, s);
}

// ---- host -------------------------------------------------------------------------------------------------------------

template <int RT, int Y>
void launch_few(const Args& a, const I8Plan& p, hipStream_t s) {
    const dim3 grid(p.groups, p.splits), block(64 * kWaves);
    if (p.nt == 1) hipLaunchKernelGGL((k_few<RT, 1, Y>), grid, block, 0, s, a);
    else if (p.nt == 2) hipLaunchKernelGGL((k_few<RT, 2, Y>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((k_few<RT, 4, Y>), grid, block, 0, s, a);
}
template <int Y>
int launch(const Args& a, const I8Plan& p, hipStream_t s) {
    const dim3 grid(p.groups, p.splits);
    const I8Shape& t = kShapes[p.tile];
    const uint32_t rt = p.tile == kFew ? 0 : (uint32_t)div_up(a.rows, t.rows), nt = p.tile == kFew ? 0 : (uint32_t)div_up(a.n, t.outs);
    if (p.tile == kFew) a.rows <= 16 ? launch_few<1, Y>(a, p, s) : launch_few<2, Y>(a, p, s);
    else if (p.tile == kShort) hipLaunchKernelGGL((k_tiles<2, 1, 2, 2, Y>), grid, dim3(256), 0, s, a, rt, nt);
    else if (p.tile == kMid) hipLaunchKernelGGL((k_tiles<2, 2, 2, 2, Y>), grid, dim3(256), 0, s, a, rt, nt);
    else if (p.tile == kWide) hipLaunchKernelGGL((k_tiles<2, 3, 4, 2, Y>), grid, dim3(512), 0, s, a, rt, nt);
    else hipLaunchKernelGGL((k_tiles<4, 2, 2, 4, Y>), grid, dim3(512), 0, s, a, rt, nt);
    if (p.splits > 1) hipLaunchKernelGGL((k_join<Y>), dim3((unsigned)div_up((size_t)a.rows * (a.n_pad >> 2), kBlock)), dim3(kBlock), 0, s, a);
    ZK_HIP_TRY(hipGetLastError());
    return ZK_OK;
}

bool sizes_ok(size_t rows, size_t n, size_t k) {
    return rows <= (size_t)1 << 24 && n >= 1 && n <= (size_t)1 << 24 && k >= 16 && k % 16 == 0 && k <= I8_MAX_K;
}

}  // namespace
}  // namespace zkmi

using namespace zkmi;

extern "C" size_t i8_matmul_workspace_bytes(size_t rows, size_t n, size_t k) {
    if (rows == 0 || !sizes_ok(rows, n, k)) return 0;
    const I8Plan p = i8_plan(rows, n, k);
    if (p.splits == 1) return 0;
    Carver cv(nullptr, 0);
    cv.take((size_t)p.splits * rows * align_up(n, 4) * sizeof(int32_t));
    return cv.used();
}

extern "C" int i8_matmul(void* y, size_t y_row_stride, int y_dtype, const int8_t* x, size_t x_row_stride, const float* x_scales, size_t rows,
                         const int8_t* w, const float* w_scales, size_t n, size_t k, void* ws, size_t ws_bytes, void* stream) {
    const size_t bytes = y_dtype == ZK_I32 ? 4 : y_dtype == ZK_I16 ? 0 : dtype_bytes(y_dtype);
    if (!bytes || !sizes_ok(rows, n, k)) return ZK_E_BADARG;
    if (rows == 0) return ZK_OK;
    if (!y || !x || !w || !aligned(y, bytes) || !aligned(x, 16) || !aligned(w, 16)) return ZK_E_BADARG;
    if (rows > 1 && (x_row_stride < k || x_row_stride % 16 || x_row_stride > (size_t)1 << 23 || y_row_stride < n)) return ZK_E_BADARG;
    if (y_dtype != ZK_I32 && (!x_scales || !w_scales || !aligned(x_scales, 4) || !aligned(w_scales, 4))) return ZK_E_BADARG;
    const I8Plan p = i8_plan(rows, n, k);
    if (p.tile != kFew && (uint64_t)div_up(rows, kShapes[p.tile].rows) * div_up(n, kShapes[p.tile].outs) >= (uint64_t)1 << 23) return ZK_E_BADARG;
    Args a = {};
    a.y = y;
    a.yrow = y_row_stride;
    a.x = x;
    a.xrow = rows > 1 ? x_row_stride : k;
    a.xs = x_scales;
    a.w = w;
    a.ws = w_scales;
    a.rows = (uint32_t)rows;
    a.n = (uint32_t)n;
    a.k = (uint32_t)k;
    a.splits = p.splits;
    a.each = p.each;
    a.n_pad = (uint32_t)align_up(n, 4);
    a.quads = aligned(y, 4 * bytes) && (rows == 1 || y_row_stride % 4 == 0);
    a.wide = aligned(y, 16) && (rows == 1 || y_row_stride * bytes % 16 == 0);
    if (p.splits > 1) {
        if (!ws) return ZK_E_BUFSZ;
        Carver cv(ws, ws_bytes);
        a.parts = (int32_t*)cv.take((size_t)p.splits * rows * a.n_pad * sizeof(int32_t));
        if (cv.overflow() || !a.parts) return ZK_E_BUFSZ;
    }
    hipStream_t s = as_stream(stream);
    switch (y_dtype) {
        case ZK_I32: return launch<ZK_I32>(a, p, s);
        case ZK_F32: return launch<ZK_F32>(a, p, s);
        case ZK_F16: return launch<ZK_F16>(a, p, s);
        default: return launch<ZK_BF16>(a, p, s);
    }
}
