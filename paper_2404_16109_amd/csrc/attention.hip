// kvcache_attention: how a call is spread, workgroups that share out sequences of unlike lengths, and the join of parts.  The kernels for
// few and for many rows, and what they measured: attend_dev.h.
#include "attend_dev.h"

namespace zkmi {
namespace {

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
    extern __shared__ __attribute__((aligned(16))) float sh[];
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
