// kvcache_attention_prefix: attention for a batch whose sequences all begin with the same tokens.
//
// The keys of a row are those of the prefix and its sequence's own.  With (M, l, o) the maximum, the sum of weights and
// the weighted values over a part of the keys, parts join by e^(M - max M): so the prefix is one part, or several, for ALL rows
// of the batch at once, and its codes are read once for so many rows where they would be read once for each sequence.
// k_prefix: workgroups of two kinds in one launch.  The first have 128 or 256 rows of the whole batch over tiles of the prefix, which the
// vector ALU bounds; those behind have a sequence's own keys, which latency bounds, and run beside them.  k_prefix_join adds up.
//
// Measured, 8 heads of 128 and 40 of queries, whole calls in a graph: a step of 64 sequences behind 8192 tokens 37 us (11.1 GFLOP, 54 MB: of
// it 15 are latency, a prefix of one page takes as long, 15 the tiles, 1.2 each, and the rest parts on their way to memory and back); 16 questions
// of up to 64 tokens behind 32768 377 to 388 us, 820 to 843 TFLOP/s, on one card, 416 on another (vector ALU 55% and matrix cores 41% busy in a run under the
// profiler, whose kernels took 422 and 17 us); a prompt's next 2048 tokens beside 127 single ones behind 8192 0.87 ms.
// Registers: kernels of two tiles of rows to a sequence spill, 107 of a thread's for heads beyond 192, 16 for those of 65 to 128 with eight
// wavefronts; no others do.
#include "attend_dev.h"
#include "prefix_plan.h"

namespace zkmi {
namespace {

static_assert(kPrefixTile == kTile && kPrefixWorkgroups == kWorkgroups, "");
static const uint32_t kMostJoins = 1 << 20;  // workgroups of k_prefix_join in a direction of the launch

struct PrefixArgs : Args {
    static constexpr bool joined = true;
    const int32_t* front;      // the prefix's pages
    uint32_t front_tokens;     // a multiple of the page
    uint32_t front_tiles;      // whole tiles of it; what is left is read with each sequence's own
    uint32_t front_splits, front_each, front_groups, row_tile;
    uint32_t joins;  // workgroups of k_prefix_join that a head's rows have, in a direction of the launch
    float seqs_per_row;
};
// Sums lie by the rows of the batch, so that what is kept does not go by how many rows other sequences have: those of the prefix as
// [head][part][row], behind them the own ones as [part][sequence][head][row], which workgroups that run side by side write side by side.
__device__ __forceinline__ size_t front_part(const PrefixArgs& a, uint32_t h, uint32_t part) {
    return ((size_t)h * a.front_splits + part) * (a.s.rows * a.group);
}
__device__ __forceinline__ size_t own_part(const PrefixArgs& a, const SeqView& v, uint32_t, uint32_t h, uint32_t part) {
    const size_t H = a.cache.kv_heads, R = a.s.rows * a.group;
    return (a.front_splits + part) * H * R + ((size_t)v.row0 * H + (size_t)v.rows * h) * a.group;
}

// As for a sequence alone, but that its first tokens lie in the prefix's pages, and its first tiles are not its own.
__device__ __forceinline__ uint32_t page_of(const PrefixArgs& a, uint32_t b, uint32_t token) {
    const uint32_t at = token >> a.page_log, last = a.s.table_pages - 1;
    const int32_t* p = token < a.front_tokens ? a.front + at : a.s.table + (size_t)b * a.s.table_stride + (at < last ? at : last);
    return (uint32_t)*p;
}
__device__ __forceinline__ uint32_t first_seen(const PrefixArgs& a, const SeqView&, int32_t) { return a.front_tiles * kTile; }
__device__ __forceinline__ uint32_t first_guess(const PrefixArgs& a) { return a.front_tiles; }
__device__ __forceinline__ Tiles tiles_of(const PrefixArgs& a, const SeqView& v, int32_t, int32_t i1) {
    const int64_t last = (int64_t)v.len - v.rows + i1;
    const uint32_t end = last < 0 ? 0 : (uint32_t)(last / kTile) + 1;
    return Tiles{a.front_tiles, end > a.front_tiles ? end : a.front_tiles};
}

template <int WV>
struct FrontShared {
    ManyShared many;
    int32_t place[32 * WV], least, most;  // positions of the tokens that the rows belong to, -1: nobody's
};
// A part of the prefix's whole tiles for a workgroup's rows of the batch.
template <int DT, int WV>
__device__ __forceinline__ void attend_front(const PrefixArgs& a, char* lds, FrontShared<WV>& sh, uint32_t h, uint32_t tile, uint32_t split) {
    constexpr uint32_t rows = 32 * WV, threads = 64 * WV;
    const uint32_t r0 = tile * rows, tid = threadIdx.x, R = a.s.rows * a.group, r_last = r0 + rows - 1 < R - 1 ? r0 + rows - 1 : R - 1;
    const int32_t tok0 = (int32_t)(r0 / a.group), tok1 = (int32_t)(r_last / a.group);
    if (tid < rows) sh.place[tid] = -1;
    if (tid == 0) {
        sh.least = 0x7fffffff;
        sh.most = -1;
    }
    __syncthreads();
    for (uint32_t b = tid; b < a.s.seqs; b += threads) {
        const SeqView v = seq_view(a.s, b, a.page_log);
        if (!v.ok || v.rows == 0) continue;
        const int32_t from = v.row0 > tok0 ? v.row0 : tok0, to = v.row0 + v.rows - 1 < tok1 ? v.row0 + v.rows - 1 : tok1;
        for (int32_t t = from; t <= to; ++t) sh.place[t - tok0] = v.len - v.rows + (t - v.row0);
    }
    __syncthreads();
    if ((int32_t)tid <= tok1 - tok0 && sh.place[tid] >= 0) {  // rows without a token get no answer: what they come to does not matter
        atomicMin(&sh.least, sh.place[tid]);
        atomicMax(&sh.most, sh.place[tid]);
    }
    __syncthreads();
    const int32_t least = (int32_t)uniform((uint32_t)sh.least), most = (int32_t)uniform((uint32_t)sh.most);
    if (most < 0) return;  // no row of theirs sees a key, and k_prefix_join does not ask
    Tiles tiles = {split * a.front_each, (split + 1) * a.front_each};
    if (tiles.end > a.front_tiles) tiles.end = a.front_tiles;
    const uint32_t r = r0 + (tid >> 6) * 32 + (tid & 31);
    const int32_t pos = r < R ? sh.place[r / a.group - (uint32_t)tok0] : -1;
    const SeqView all = {0, (int32_t)a.s.rows, 0, true};
    attend_rows<DT, true, WV>(a, lds, sh.many, all, 0, h, R, r0, tiles, pos, least, most, 0, true, front_part(a, h, split), a.parts, a.parts_ml);
}

// RT: tiles of 16 rows that a sequence and head has, 0: many rows.  Workgroups of one head lie eight apart where there are eight heads, so
// that an XCD reads the prefix of its own.
template <int DT, int RT, int WV>
__global__ __launch_bounds__(64 * WV, WV == 8 || (DT <= 4 && RT < 2) ? 2 : 1) void k_prefix(PrefixArgs a) {
    extern __shared__ __attribute__((aligned(16))) char lds[];
    __shared__ FrontShared<WV> sh;
    const uint32_t H = a.cache.kv_heads;
    if (blockIdx.x < a.front_groups) {
        const uint32_t id = blockIdx.x, h = id % H, at = id / H, tile = at / a.front_splits;
        return attend_front<DT, WV>(a, lds, sh, h, tile, at - tile * a.front_splits);
    }
    uint32_t id = blockIdx.x - a.front_groups;
    const uint32_t h = id % H;
    id /= H;
    const uint32_t split = id % a.splits;
    id /= a.splits;
    if constexpr (RT != 0) attend_few<(DT + 1) / 2, RT, WV>(a, (float*)lds, split, h, id);
    else {
        const uint32_t tiles = (a.rows_most + a.row_tile - 1) / a.row_tile, b = id / tiles;
        attend_many<DT, WV>(a, lds, sh.many, id - b * tiles, split, h, b);
    }
}

// The sequence that has a row of the batch, for a wavefront; one that is not ok where none has it.  64 are looked at at once: those about where it
// lies if all have as many rows, then those that a search of cu comes to, then all, if cu says that there is one (and does not rise).
__device__ __forceinline__ SeqView seq_of(const PrefixArgs& a, int32_t token) {
    const uint32_t n = a.s.seqs, lane = threadIdx.x & 63, most = n > 64 ? n - 64 : 0;
    const int32_t about = (int32_t)((float)token * a.seqs_per_row) - 32;
    uint32_t b0 = about <= 0 ? 0 : (uint32_t)about < most ? (uint32_t)about : most;
    for (uint32_t turn = 0;; ++turn) {
        const uint32_t b = b0 + lane < n ? b0 + lane : n - 1;
        const int32_t from = a.s.cu[b], end = a.s.cu[b + 1], len = a.s.lens[b];
        const uint64_t has = __ballot(from <= token && token < end);
        if (has) {
            const int at = __ffsll((long long)has) - 1;
            return seq_view(a.s, a.page_log, __builtin_amdgcn_readlane(from, at), __builtin_amdgcn_readlane(end, at), __builtin_amdgcn_readlane(len, at));
        }
        if (n <= 64 || (turn == 0 && token >= a.s.cu[n]) || turn * 64 >= n + 128) return SeqView{0, 0, 0, false};
        if (turn == 0) {
            b0 = 0;
            for (uint32_t left = n; left > 64;) {
                const uint32_t step = (left + 63) / 64, k = b0 + lane * step;
                const uint64_t below = __ballot(lane * step < left && a.s.cu[k < n ? k : n - 1] <= token);
                const uint32_t at = below ? (63 - (uint32_t)__builtin_clzll(below)) * step : 0;
                b0 += at;
                left = left - at < step ? left - at : step;
            }
        } else {
            b0 = (turn - 1) * 64;
        }
    }
}

// A wavefront: one row of the batch and a head.  Lanes hold four dimensions each; the lanes left of 64 take parts in turn.
__device__ __forceinline__ void join_row(const PrefixArgs& a, uint32_t h, uint32_t row) {
    const uint32_t H = a.cache.kv_heads, d = a.cache.head_dim, lane = threadIdx.x & 63, token = row / a.group;
    const SeqView v = seq_of(a, (int32_t)token);
    if (!v.ok) {  // nobody's, or one of a sequence that is skipped
        if (v.rows == 0) return;
        const size_t head = h * a.group + (row - token * a.group);
        for (uint32_t i = lane; i < d; i += 64) put_at(a.out, token * a.orow + head * a.ohead + i, __builtin_nanf(""), a.dtype);
        if (a.lse && lane == 0) a.lse[(size_t)token * H * a.group + head] = __builtin_nanf("");
        return;
    }
    const uint32_t r = row - (uint32_t)v.row0 * a.group;
    const int32_t pos = v.len - v.rows + (int32_t)(r / a.group);
    // parts of the prefix come first; a row that sees no key has none
    const uint32_t front = pos >= 0 ? a.front_splits : 0;
    const Tiles tiles = a.few ? tiles_of(a, v, 0, v.rows - 1) : tiles_of_rows(a, v, r / a.row_tile * a.row_tile, a.row_tile);
    const uint32_t each = part_of(a, tiles), n = tiles.end - tiles.first, own = pos >= 0 && n ? (n + each - 1) / each : 0, parts = front + own;
    const size_t R = a.s.rows * a.group, front0 = front_part(a, h, 0) + row, own0 = own_part(a, v, 0, h, 0) + r;
    const size_t own_less = own0 - front * R * H;
    const auto at = [&](uint32_t p) { return (p < front ? front0 : own_less) + p * (p < front ? R : R * H); };
    float m = -kInf, l = 0.0f;
    if (lane < parts) {
        const float2 ml = a.parts_ml[at(lane)];
        m = ml.x;
        l = ml.y;
    }
    const uint32_t quads = d >> 2, ways = 64 / quads, way = lane / quads, c = lane - way * quads;
    v4f sum = {0, 0, 0, 0};
    float weight = 0.0f, ref = 0.0f;
    // eight parts of a lane are on their way at once, the first beside the maxima
    for (uint32_t p0 = 0; p0 < parts || p0 == 0; p0 += 8 * ways) {
        v4f x[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            const uint32_t p = p0 + u * ways + way;
            x[u] = v4f{0, 0, 0, 0};
            if (way < ways && p < parts) x[u] = ((const v4f*)a.parts)[at(p) * quads + c];
        }
        if (p0 == 0) {
            const float top = wave_max(m);
            ref = top == -kInf ? 0.0f : top;
            weight = exp2_of(m - ref);
            l = wave_add(l * weight);
        }
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            const uint32_t p = p0 + u * ways + way;
            const float w = bits_float((uint32_t)__shfl((int)float_bits(weight), (int)(p & 63)));
            if (way < ways && p < parts) sum += x[u] * w;
        }
    }
    for (uint32_t w = 1; w < ways; ++w) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float other = bits_float((uint32_t)__shfl((int)float_bits(sum[e]), (int)((lane + w * quads) & 63)));
            if (way == 0) sum[e] += other;
        }
    }
    if (way == 0) {
        const size_t to = row_at(a, v, h, r, a.orow, a.ohead) + 4 * c;
        const float inv = l == 0.0f ? 0.0f : 1.0f / l;
#pragma unroll
        for (int e = 0; e < 4; ++e) put_at(a.out, to + e, l == 0.0f ? 0.0f : sum[e] * inv, a.dtype);
    }
    if (a.lse && lane == 0) a.lse[row_at(a, v, h, r, (size_t)H * a.group, 1)] = lse_of(ref, l);
}
// Workgroups behind those that join look the sequences over.
__global__ __launch_bounds__(kBlock) void k_prefix_join(PrefixArgs a) {
    if (blockIdx.x >= a.joins) {
        const uint32_t b = (blockIdx.x - a.joins) * kBlock + threadIdx.x;
        if (blockIdx.y + blockIdx.z == 0 && b < a.s.seqs && !seq_view(a.s, b, a.page_log).ok) report(a.s, ZK_FAULT_LENGTH);
        return;
    }
    const uint32_t row = uniform((blockIdx.z * a.joins + blockIdx.x) * (kBlock / 64) + (threadIdx.x >> 6));
    if (row < a.s.rows * a.group) join_row(a, blockIdx.y, row);
}

// ---- host -------------------------------------------------------------------------------------------------------------

// What lies in the workspace; with a null base the bytes alone.
size_t carve(Carver& cv, const PrefixPlan& p, uint64_t rows, uint32_t kv_heads, uint32_t head_dim, PrefixArgs* a) {
    const size_t parts = (size_t)kv_heads * (p.front_splits + p.splits) * rows;
    void* at[2] = {cv.take(parts * head_dim * sizeof(float)), cv.take(parts * sizeof(float2))};
    if (a) {
        a->parts = (float*)at[0];
        a->parts_ml = (float2*)at[1];
    }
    return cv.used();
}

template <int DT, int RT, int WV>
int launch(const PrefixArgs& a, uint64_t own, hipStream_t s) {
    size_t lds = 2 * (size_t)ManyLds<DT>::bytes;
    if constexpr (RT != 0) {
        const size_t few = FewLds<(DT + 1) / 2, RT, WV>::bytes(a.rows_most);
        if (few > lds) lds = few;
    }
    if (lds > 60000) ZK_HIP_TRY(hipFuncSetAttribute((const void*)k_prefix<DT, RT, WV>, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds));
    hipLaunchKernelGGL((k_prefix<DT, RT, WV>), dim3((unsigned)(a.front_groups + own)), dim3(64 * WV), lds, s, a);
    hipLaunchKernelGGL(k_prefix_join, dim3(a.joins + (unsigned)div_up(a.s.seqs, kBlock), a.cache.kv_heads, (unsigned)div_up(div_up((size_t)a.s.rows * a.group, kBlock / 64), a.joins)),
                       dim3(kBlock), 0, s, a);
    ZK_HIP_TRY(hipGetLastError());
    return ZK_OK;
}
template <int DT, int WV>
int launch(const PrefixArgs& a, uint64_t own, hipStream_t s) {
    switch (prefix_row_tiles(a.rows_most)) {
        case 1: return launch<DT, 1, WV>(a, own, s);
        case 2: return launch<DT, 2, WV>(a, own, s);
        default: return launch<DT, 0, WV>(a, own, s);
    }
}
template <int DT>
int launch(const PrefixArgs& a, uint64_t own, hipStream_t s) {
    if constexpr (DT <= 4)
        if (a.row_tile == 256) return launch<DT, 8>(a, own, s);
    return launch<DT, 4>(a, own, s);
}

// Rows of a sequence and head at most.
uint64_t rows_most(uint32_t rows, uint32_t max_new, uint32_t group) { return (uint64_t)(max_new < rows ? max_new : rows) * group; }

}  // namespace
}  // namespace zkmi

using namespace zkmi;

extern "C" size_t kvcache_attention_prefix_workspace_bytes(uint32_t seqs, uint32_t rows, uint32_t max_new, uint32_t q_heads, uint32_t kv_heads,
                                                           uint32_t head_dim, uint32_t prefix_tokens, uint32_t max_len) {
    if (!kv_heads || q_heads == 0 || q_heads % kv_heads || !seqs || seqs > 65535 || !rows || !max_new) return 0;
    const uint32_t group = q_heads / kv_heads;
    const uint64_t all = (uint64_t)rows * group, most = rows_most(rows, max_new, group);
    Carver cv(nullptr, 0);
    return carve(cv, prefix_plan(seqs, all, most, kv_heads, head_dim, prefix_tokens, max_len), all, kv_heads, head_dim, nullptr);
}

extern "C" int kvcache_attention_prefix(const kvcache_i8* cache, const void* q, size_t q_row_stride, size_t q_head_stride, int dtype,
                                        uint32_t q_heads, const kv_seqs* seqs, const int32_t* prefix, uint32_t prefix_pages, float scale, void* out,
                                        size_t out_row_stride, size_t out_head_stride, float* lse, void* ws, size_t ws_bytes, void* stream) {
    if ((dtype != ZK_F16 && dtype != ZK_BF16) || !cache_ok(cache) || !seqs_ok(seqs)) return ZK_E_BADARG;
    if (q_heads == 0 || q_heads % cache->kv_heads || q_heads > 65536 || !(scale - scale == 0.0f)) return ZK_E_BADARG;
    if ((uint64_t)prefix_pages * cache->page_tokens >= 0x80000000u || (prefix_pages && (!prefix || !aligned(prefix, 4)))) return ZK_E_BADARG;
    if (seqs->rows == 0 || seqs->seqs == 0) return ZK_OK;
    if (!q || !out || !aligned(q, 2) || !aligned(out, 2) || (lse && !aligned(lse, 4))) return ZK_E_BADARG;
    const uint32_t group = q_heads / cache->kv_heads;
    const uint64_t rows = (uint64_t)seqs->rows * group, most = rows_most(seqs->rows, seqs->max_new, group);
    if (rows >= 0x7fffff00u || most * cache->kv_heads > ((uint64_t)1 << 26) - 4) return ZK_E_BADARG;
    PrefixArgs a = {};
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
    a.group = group;
    a.page_log = (uint32_t)log2_floor(cache->page_tokens);
    a.dtype = dtype;
    a.few = prefix_few(most);
    a.wide = aligned(q, 16) && q_row_stride % 8 == 0 && q_head_stride % 8 == 0;
    a.rows_most = (uint32_t)most;
    a.front = prefix;
    a.front_tokens = prefix_pages * cache->page_tokens;
    const PrefixPlan p = prefix_plan(seqs->seqs, rows, most, cache->kv_heads, cache->head_dim, a.front_tokens, seqs->max_len);
    a.front_tiles = p.front_tiles;
    a.row_tile = p.row_tile;
    a.front_splits = p.front_splits;
    a.front_each = p.front_each;
    a.splits = p.splits;
    a.each = p.each;
    const uint64_t front = (uint64_t)cache->kv_heads * p.front_splits * div_up(rows, p.row_tile);
    const uint64_t own = (uint64_t)seqs->seqs * cache->kv_heads * p.splits * (a.few ? 1 : div_up(most, p.row_tile));
    if (front + own >= (uint64_t)1 << 23) return ZK_E_BADARG;  // a launch holds fewer than 2^32 threads
    a.front_groups = (uint32_t)front;
    const size_t joins = div_up(rows, kBlock / 64);
    a.joins = (uint32_t)(joins < kMostJoins ? joins : kMostJoins);
    a.seqs_per_row = (float)seqs->seqs / (float)seqs->rows;
    if (!ws) return ZK_E_BUFSZ;
    Carver cv(ws, ws_bytes);
    carve(cv, p, rows, cache->kv_heads, cache->head_dim, &a);
    if (cv.overflow()) return ZK_E_BUFSZ;
    hipStream_t s = as_stream(stream);
    switch ((cache->head_dim + 31) / 32) {
        case 1: return launch<1>(a, own, s);
        case 2: return launch<2>(a, own, s);
        case 3: return launch<3>(a, own, s);
        case 4: return launch<4>(a, own, s);
        case 5: return launch<5>(a, own, s);
        case 6: return launch<6>(a, own, s);
        case 7: return launch<7>(a, own, s);
        default: return launch<8>(a, own, s);
    }
}
