// pf_prefix.cu -- single-token attention of sequences that share prefixes.
//
//   out = sum_t w_t V_t / sum_t w_t,  t over the prefix of the sequence's group and over its own tokens,  w_t = exp(sm q . K_t)
//
// A group's rows (sequences times query heads of a key head) are cut into tiles of 256, and such a tile goes through the group's prefix once:
// the cache is read once for all of them.  All (tile of rows, tile of 128 tokens) pairs of all groups and key heads form one list, which is cut into
// equal pieces; a piece leaves partial results (reference z, sum, weighted values) of each of its tiles of rows.  The sequences' own tokens go
// through the kernel of pf_decode_attention, and a third kernel joins the parts of every row in a fixed order.
#include <math.h>

#include "pf_attention.cuh"

namespace pf {

constexpr int kRows = 256;               // rows of a task
constexpr int kTok = 128;                // tokens of a tile
constexpr int kMostTiles = 512;          // tiles of a piece at most: 32-bit sums do not run over more than 65536 tokens
constexpr int kLeastTiles = 4;           // a piece takes no fewer while others have none

struct PrefixArgs {
    AttnArgs a;
    const int32_t *cu, *plen, *ptable;
    int n_groups, pcols;
    long long n_slots;
    float *slots;                        // [n_slots] x (kRows x HD values, kRows references, kRows sums)
};

struct Group { int first, rows, row_tiles, len, tiles; };
__device__ __forceinline__ Group group_of(const PrefixArgs &P, int g)
{
    const AttnArgs &A = P.a;
    Group r;
    r.first = P.cu ? min(max(P.cu[g], 0), A.n_seq) : 0;      // without offsets: one group of all
    const int last = P.cu ? min(max(P.cu[g + 1], r.first), A.n_seq) : A.n_seq;
    r.rows = (last - r.first) * A.group;
    r.row_tiles = (r.rows + kRows - 1) / kRows;
    const long long cap = (long long)P.pcols * A.c.page;
    r.len = max(0, P.plen[g]);
    if (r.len > cap) r.len = (int)cap;
    r.tiles = (r.len + kTok - 1) / kTok;
    return r;
}

// Tiles and tasks of the groups in front of each group, by the whole block.  units, tasks: n_groups + 1 words
__device__ __forceinline__ void group_prefix(const PrefixArgs &P, long long *units, int *tasks)
{
    __shared__ long long warp_units[32];
    __shared__ int warp_tasks[32];
    const int nt = blockDim.x, tid = threadIdx.x, lane = tid & 31, nw = (nt + 31) >> 5;
    long long base_u = 0;
    int base_t = 0;
    if (tid == 0) units[0] = 0, tasks[0] = 0;
    for (int g0 = 0; g0 < P.n_groups; g0 += nt) {
        long long u = 0;
        int t = 0;
        if (g0 + tid < P.n_groups) {
            const Group r = group_of(P, g0 + tid);
            t = r.tiles ? r.row_tiles * P.a.c.n_kv : 0;
            u = (long long)t * r.tiles;
        }
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long pu = __shfl_up_sync(0xFFFFFFFFu, u, o);
            const int pt = __shfl_up_sync(0xFFFFFFFFu, t, o);
            if (lane >= o) u += pu, t += pt;
        }
        __syncthreads();
        if (lane == 31) warp_units[tid >> 5] = u, warp_tasks[tid >> 5] = t;
        __syncthreads();
        long long add_u = base_u;
        int add_t = base_t;
        for (int i = 0; i < nw; i++) {
            if (i < (tid >> 5)) add_u += warp_units[i], add_t += warp_tasks[i];
            base_u += warp_units[i];
            base_t += warp_tasks[i];
        }
        if (g0 + tid < P.n_groups) units[g0 + tid + 1] = add_u + u, tasks[g0 + tid + 1] = add_t + t;
    }
    __syncthreads();
}
// pieces that the list is cut into: one a block, or as many more as keep them at kMostTiles
__device__ __forceinline__ int pieces_of(long long total, int blocks)
{
    const long long few = (total + kLeastTiles - 1) / kLeastTiles;
    if (few < blocks) return (int)few;
    const long long per = (total + (long long)blocks * kMostTiles - 1) / ((long long)blocks * kMostTiles);
    return (int)(per * blocks);
}
// the last entry of a rising list of n + 1 words whose value is at most x
template <typename V>
__device__ __forceinline__ int last_at(const V *list, int n, V x)
{
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (list[mid] <= x) lo = mid; else hi = mid;
    }
    return lo;
}

// A stretch of one task: tiles [tile, end) of task `task` (number `no` within its group)
struct Stretch {
    Group g;
    int kv, row0, rows, tile, end, group;
    long long slot;
};

template <typename T, int HD>
__global__ void __launch_bounds__(512, 1) prefix_kernel(const __grid_constant__ PrefixArgs P)
{
    const AttnArgs &A = P.a;
    extern __shared__ __align__(128) uint8_t smem[];
    float *ks = reinterpret_cast<float *>(smem), *vs = ks + 32 * HD, *lv = vs + 32 * HD;
    long long *units = reinterpret_cast<long long *>(lv + 32);
    int *tasks = reinterpret_cast<int *>(units + P.n_groups + 1);
    group_prefix(P, units, tasks);
    const long long total = units[P.n_groups];
    if (total == 0) return;
    const int n_pieces = pieces_of(total, gridDim.x);
    const int row = threadIdx.x >> 1, part = threadIdx.x & 1;
    constexpr int D = HD / 2;
    for (int piece = blockIdx.x; piece < n_pieces; piece += gridDim.x) {
        long long u = first_tile(total, n_pieces, piece);
        const long long u_end = first_tile(total, n_pieces, piece + 1);
        while (u < u_end) {
            const int gi = last_at(units, P.n_groups, u);
            const Group g = group_of(P, gi);
            const long long r = u - units[gi];
            const int no = (int)(r / g.tiles), tile0 = (int)(r - (long long)no * g.tiles);
            const int end = (int)min((long long)g.tiles, tile0 + (u_end - u));
            const int kv = no / g.row_tiles, rt = no - kv * g.row_tiles;
            const int at = rt * kRows + row;
            const bool live = at < g.rows;
            float q[D], o[D], z = -INFINITY, l = 0.f;
#pragma unroll
            for (int i = 0; i < D; i++) q[i] = 0.f, o[i] = 0.f;
            if (live) {
                const uint16_t *src = A.q + (int64_t)(g.first + at / A.group) * A.qs + (int64_t)(kv * A.group + at % A.group) * HD + part * D;
#pragma unroll
                for (int i = 0; i < D; i += 2) {
                    const float2 f = pair_to_f32<T>(*reinterpret_cast<const uint32_t *>(src + i));
                    q[i] = f.x * A.scale_log2;
                    q[i + 1] = f.y * A.scale_log2;
                }
            }
            for (int tok0 = tile0 * kTok; tok0 < min(g.len, end * kTok); tok0 += 32) {
                __syncthreads();
                for (int i = threadIdx.x; i < 32 * HD / 4; i += blockDim.x) {
                    const int t = i / (HD / 4), e = i % (HD / 4) * 4, tok = tok0 + t;
                    int page = tok < g.len ? P.ptable[(int64_t)gi * P.pcols + tok / A.c.page] : -1;
                    if (page >= A.c.n_pages) page = -1;
                    const int64_t ph = (int64_t)page * A.c.n_kv + kv, from = (ph * A.c.page + tok % A.c.page) * HD + e;
                    const uint32_t k = page < 0 ? 0u : *reinterpret_cast<const uint32_t *>(A.c.d_k + from), v = page < 0 ? 0u : *reinterpret_cast<const uint32_t *>(A.c.d_v + from);
                    const float fk = page < 0 ? 0.f : A.c.d_k_scale[ph], fv = page < 0 ? 0.f : A.c.d_v_scale[ph];
                    const float2 k0 = f32x2_of_f16x2(f16x2_of_e4m3x2(k)), k1 = f32x2_of_f16x2(f16x2_of_e4m3x2(k >> 16));
                    const float2 v0 = f32x2_of_f16x2(f16x2_of_e4m3x2(v)), v1 = f32x2_of_f16x2(f16x2_of_e4m3x2(v >> 16));
                    *reinterpret_cast<float4 *>(ks + t * HD + e) = make_float4(k0.x * fk, k0.y * fk, k1.x * fk, k1.y * fk);
                    *reinterpret_cast<float4 *>(vs + t * HD + e) = make_float4(v0.x * fv, v0.y * fv, v1.x * fv, v1.y * fv);
                    if (e == 0) lv[t] = page < 0 ? -INFINITY : 0.f;
                }
                __syncthreads();
                for (int t = 0; t < 32; t++) {
                    float s = 0.f;
#pragma unroll
                    for (int i = 0; i < D; i++) s = fmaf(q[i], ks[t * HD + part * D + i], s);
                    s += __shfl_xor_sync(0xFFFFFFFFu, s, 1);
                    s += lv[t];
                    const float n = fmaxf(z, s);
                    const float f = n == -INFINITY ? 1.f : exp2f(z - n), p = exp2f(s - (n == -INFINITY ? 0.f : n));
                    z = n;
                    l = fmaf(l, f, p);
#pragma unroll
                    for (int i = 0; i < D; i++) o[i] = fmaf(o[i], f, p * vs[t * HD + part * D + i]);
                }
            }
            const long long slot = tasks[gi] + no + piece;
            if (live && slot < P.n_slots) {
                float *to = P.slots + slot * (kRows * (HD + 2));
#pragma unroll
                for (int i = 0; i < D; i++) to[row * HD + part * D + i] = o[i];
                if (part == 0) {
                    to[kRows * HD + row] = z;
                    to[kRows * (HD + 1) + row] = l;
                }
            }
            u += end - tile0;
        }
    }
}

// ------------------------------------------------------------------ the join
// A warp joins the parts of one row: what its own tokens left (one part where a single block finished them, else one of each block), and
// one of each piece that goes through the prefix.
template <typename T, int HD, int NB>
__global__ void __launch_bounds__(256) prefix_join_kernel(const __grid_constant__ PrefixArgs P, const int own_grid, const int prefix_grid)
{
    using S = AttnShape<HD, NB>;
    constexpr int V = HD / 32;
    const AttnArgs &A = P.a;
    extern __shared__ __align__(128) uint8_t smem[];
    long long *units = reinterpret_cast<long long *>(smem);
    int *tasks = reinterpret_cast<int *>(units + P.n_groups + 1);
    int *prefix = tasks + P.n_groups + 1;
    __shared__ int warp_sum[8];
    group_prefix(P, units, tasks);
    tile_prefix(A, prefix, warp_sum);
    const int lane = threadIdx.x & 31;
    const long long total = units[P.n_groups], own_total = (long long)prefix[A.n_seq] * A.jobs_per_seq;
    const int n_pieces = total ? pieces_of(total, prefix_grid) : 0, own_blocks = blocks_used(own_total, own_grid);
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const float *blocks = A.part + (int64_t)own_grid * S::kWarps * S::kPartFloats;
    const long long n_rows = (long long)A.n_seq * A.n_heads;
    for (long long row = (long long)blockIdx.x * 8 + (threadIdx.x >> 5); row < n_rows; row += (long long)gridDim.x * 8) {
        const int b = (int)(row / A.n_heads), head = (int)(row - (long long)b * A.n_heads);
        const int kv = head / A.group, gh = head - kv * A.group;
        // parts of its own tokens
        int w0 = 0, n_own = 0, own_row = 0;
        const int own_tiles = prefix[b + 1] - prefix[b];
        if (own_tiles) {
            const int rb = gh / S::kHeads;
            own_row = gh - rb * S::kHeads;
            const long long begin = (long long)prefix[b] * A.jobs_per_seq + (long long)(kv * A.row_blocks + rb) * own_tiles;
            w0 = piece_of(own_total, own_blocks, begin);
            n_own = piece_of(own_total, own_blocks, begin + own_tiles - 1) - w0 + 1;
        }
        // parts of its group's prefix
        long long slot = 0;
        int n_pre = 0, at = 0;
        if (total) {
            const int gi = P.cu ? last_at(P.cu, P.n_groups, b) : 0;
            const Group g = group_of(P, gi);
            if (g.tiles && b >= g.first && b < g.first + g.rows / A.group) {
                at = (b - g.first) * A.group + gh;
                const int no = kv * g.row_tiles + at / kRows;
                at %= kRows;
                const long long begin = units[gi] + (long long)no * g.tiles;
                const int p0 = piece_of(total, n_pieces, begin);
                n_pre = piece_of(total, n_pieces, begin + g.tiles - 1) - p0 + 1;
                slot = (long long)tasks[gi] + no + p0;
                if (slot + n_pre > P.n_slots) n_pre = 0;
            }
        }
        const int n = n_own + n_pre;
        float top = -INFINITY, sum = 0.f, v[V];
#pragma unroll
        for (int k = 0; k < V; k++) v[k] = 0.f;
        for (int i0 = 0; i0 < n; i0 += 32) {
            const int i = i0 + lane;
            const float *from = nullptr;          // lane k: values of part i0 + k
            float z = -INFINITY, l = 0.f;
            if (i < n_own && n_own == 1) {
                from = A.own_v + row * HD;
                z = A.own_z[row];
                l = A.own_l[row];
            } else if (i < n_own) {               // a job begins in slot 1 of its first block and goes on in slot 0 of the others
                const float *p = blocks + ((int64_t)(w0 + i) * 2 + (i == 0 ? 1 : 0)) * S::kPartFloats;
                from = p + own_row * HD;
                z = p[S::kHeads * HD + own_row];
                l = p[S::kHeads * (HD + 1) + own_row];
            } else if (i < n) {
                const float *p = P.slots + (slot + i - n_own) * (kRows * (HD + 2));
                from = p + at * HD;
                z = p[kRows * HD + at];
                l = p[kRows * (HD + 1) + at];
            }
            float most = fmaxf(top, z);
#pragma unroll
            for (int x = 16; x; x >>= 1) most = fmaxf(most, __shfl_xor_sync(0xFFFFFFFFu, most, x));
            const float ref = most == -INFINITY ? 0.f : most, old = exp2f(top - ref), f = exp2f(z - ref);
            float add = l * f;
#pragma unroll
            for (int x = 16; x; x >>= 1) add += __shfl_xor_sync(0xFFFFFFFFu, add, x);
            top = most;
            sum = fmaf(sum, old, add);
#pragma unroll
            for (int k = 0; k < V; k++) v[k] *= old;
            const int count = min(32, n - i0);
            for (int k = 0; k < count; k++) {
                const float *p = (const float *)__shfl_sync(0xFFFFFFFFu, (unsigned long long)from, k) + lane * V;
                const float w = __shfl_sync(0xFFFFFFFFu, f, k);
#pragma unroll
                for (int j = 0; j < V; j++) v[j] = fmaf(p[j], w, v[j]);
            }
        }
        const float inv = sum == 0.f ? 0.f : 1.f / sum;      // (a sum that is not a number stays one)
        uint32_t *dst = reinterpret_cast<uint32_t *>(A.out + b * A.os + (int64_t)head * HD) + lane * V / 2;
#pragma unroll
        for (int k = 0; k < V; k += 2) dst[k / 2] = pair_of_f32<T>(v[k] * inv, v[k + 1] * inv);
        if (A.lse && lane == 0) A.lse[row] = sum == 0.f ? -INFINITY : (top + log2f(sum)) * kLn2;
    }
}

// ------------------------------------------------------------------ host
struct PrefixSizes {
    size_t own_v, own_z, own_l, slots, bytes;      // offsets in the workspace, and its size
    long long n_slots;
};
static PrefixSizes prefix_sizes(int hd, int page, int n_kv, int n_seq, int n_heads, int n_groups, int pcols, int sms)
{
    PrefixSizes s;
    auto up = [](size_t x) { return (x + 255) & ~(size_t)255; };
    const size_t rows = (size_t)n_seq * n_heads;
    s.own_v = up(attention_workspace_bytes(hd, sms));
    s.own_z = s.own_v + up(rows * hd * 4);
    s.own_l = s.own_z + up(rows * 4);
    s.slots = s.own_l + up(rows * 4);
    const long long tiles = ((long long)pcols * page + kTok - 1) / kTok;
    const long long tasks = (long long)n_kv * (((long long)n_seq * (n_heads / n_kv)) / kRows + n_groups);
    const long long per = (tasks * tiles + (long long)sms * kMostTiles - 1) / ((long long)sms * kMostTiles);
    s.n_slots = tasks + (per > 1 ? per : 1) * sms;
    s.bytes = s.slots + (size_t)s.n_slots * kRows * (hd + 2) * 4;
    return s;
}

template <typename T, int HD, int NB>
static int prefix_launch(PrefixArgs p, int device, int sms, cudaStream_t st)
{
    using S = AttnShape<HD, NB>;
    AttnArgs &a = p.a;
    a.row_blocks = (a.group + S::kHeads - 1) / S::kHeads;
    a.jobs_per_seq = a.c.n_kv * a.row_blocks;
    const size_t groups = (size_t)(p.n_groups + 1) * 12, own = ((size_t)a.n_seq + 1) * 4;
    const size_t smem0 = 2 * 32 * HD * 4 + 128 + groups, smem1 = (size_t)S::kWarps * S::kWarpBytes + own, smem2 = groups + own;
    PF_CUDA_TRY(ensure_dynamic_smem((const void *)prefix_kernel<T, HD>, device, smem0), "prefix_kernel shared memory");
    PF_CUDA_TRY(ensure_dynamic_smem((const void *)attention_kernel<T, HD, NB, true>, device, smem1), "attention_kernel shared memory");
    PF_CUDA_TRY(ensure_dynamic_smem((const void *)prefix_join_kernel<T, HD, NB>, device, smem2), "prefix_join_kernel shared memory");
    prefix_kernel<T, HD><<<sms, 512, smem0, st>>>(p);
    PF_CUDA_TRY(cudaGetLastError(), "prefix_kernel launch");
    count_launch();
    PF_CUDA_TRY(launch_chained(attention_kernel<T, HD, NB, true>, dim3(sms), dim3(S::kWarps * 32), smem1, st, a), "attention_kernel launch");
    count_launch();
    const long long blocks = ((long long)a.n_seq * a.n_heads + 7) / 8;
    PF_CUDA_TRY(launch_chained(prefix_join_kernel<T, HD, NB>, dim3((unsigned)(blocks < 4 * sms ? blocks : 4 * sms)), dim3(256), smem2, st, p, sms, sms),
                "prefix_join_kernel launch");
    count_launch();
    return PF_OK;
}
template <typename T>
static int prefix_launch(const PrefixArgs &p, int device, int sms, cudaStream_t st)
{
    if (p.a.c.hd == 64) return p.a.group <= 8 ? prefix_launch<T, 64, 1>(p, device, sms, st) : prefix_launch<T, 64, 2>(p, device, sms, st);
    return p.a.group <= 8 ? prefix_launch<T, 128, 1>(p, device, sms, st) : prefix_launch<T, 128, 2>(p, device, sms, st);
}

}  // namespace pf

using namespace pf;

extern "C" size_t pf_prefix_attention_workspace(const pf_kv_cache_t *cache, int32_t n_seq, int32_t n_heads, int32_t n_groups, int32_t prefix_cols)
{
    int device, sms;
    if (!cache || cache->n_kv <= 0 || cache->page <= 0 || n_seq <= 0 || n_heads <= 0 || n_groups < 0 || prefix_cols < 0 || current_sm_count(&device, &sms) != PF_OK) return 256;
    return prefix_sizes(cache->hd, cache->page, cache->n_kv, n_seq, n_heads, n_groups, prefix_cols, sms).bytes;
}

extern "C" int pf_prefix_attention(const pf_kv_cache_t *cache, int32_t dtype, int32_t n_seq, int32_t n_heads, const void *d_q, int64_t q_stride,
                                   const int32_t *d_len, const int32_t *d_table, int32_t table_cols, int32_t n_groups, const int32_t *d_cu_seqs,
                                   const int32_t *d_prefix_len, const int32_t *d_prefix_table, int32_t prefix_cols, float sm_scale, void *d_out,
                                   int64_t out_stride, float *d_lse, void *d_workspace, size_t workspace_bytes, void *stream)
{
    if (!kv_cache_ok(cache) || (dtype != PF_DT_BF16 && dtype != PF_DT_F16)) return PF_EINVAL;
    if (n_seq < 0 || n_seq > PF_ATTN_MAX_SEQ || n_heads < 0 || table_cols < 0 || (int64_t)table_cols * cache->page >= (1ll << 31)) return PF_ERANGE;
    if (n_groups < 0 || n_groups > PF_PREFIX_MAX_GROUPS || prefix_cols < 0 || (int64_t)prefix_cols * cache->page >= (1ll << 31)) return PF_ERANGE;
    const int64_t tiles = ((int64_t)table_cols * cache->page + kTile - 1) / kTile;      // as in pf_decode_attention
    if ((int64_t)n_seq * tiles >= (1ll << 31)) return PF_ERANGE;
    if ((int64_t)n_seq * n_heads >= (1ll << 30)) return PF_ERANGE;
    if (n_heads % cache->n_kv != 0 || !isfinite(sm_scale)) return PF_EINVAL;
    if (n_seq == 0 || n_heads == 0) return PF_OK;
    if (!d_q || !d_out || !d_len || (!d_table && table_cols > 0) || !aligned16(d_q) || !aligned16(d_out)) return PF_EINVAL;
    if (n_groups > 0 && ((!d_cu_seqs && n_groups > 1) || !d_prefix_len || (!d_prefix_table && prefix_cols > 0))) return PF_EINVAL;
    if ((uintptr_t)d_len % 4 || (uintptr_t)d_table % 4 || (uintptr_t)d_lse % 4 || (uintptr_t)d_cu_seqs % 4 || (uintptr_t)d_prefix_len % 4 || (uintptr_t)d_prefix_table % 4)
        return PF_EINVAL;
    const int64_t row = (int64_t)n_heads * cache->hd;
    if (q_stride < row || out_stride < row || q_stride % 8 || out_stride % 8) return PF_EINVAL;
    if (n_groups == 0 || prefix_cols == 0)
        return pf_decode_attention(cache, dtype, n_seq, n_heads, d_q, q_stride, d_len, d_table, table_cols, sm_scale, d_out, out_stride, d_lse, d_workspace,
                                   workspace_bytes, stream);
    int device, sms;
    if (int rc = current_sm_count(&device, &sms)) return rc;
    const PrefixSizes z = prefix_sizes(cache->hd, cache->page, cache->n_kv, n_seq, n_heads, n_groups, prefix_cols, sms);
    if (!d_workspace || ((uintptr_t)d_workspace & 255) != 0 || workspace_bytes < z.bytes) return PF_EWORKSPACE;
    uint8_t *ws = (uint8_t *)d_workspace;
    PrefixArgs p;
    AttnArgs &a = p.a;
    a.c = *cache;
    a.q = (const uint16_t *)d_q; a.out = (uint16_t *)d_out; a.lse = d_lse;
    a.len = d_len; a.table = d_table;
    a.qs = q_stride; a.os = out_stride;
    a.n_seq = n_seq; a.n_heads = n_heads; a.group = n_heads / cache->n_kv; a.cols = table_cols;
    a.scale_log2 = sm_scale * kLog2e;
    a.part = (float *)ws;
    a.own_v = (float *)(ws + z.own_v); a.own_z = (float *)(ws + z.own_z); a.own_l = (float *)(ws + z.own_l);
    p.cu = d_cu_seqs; p.plen = d_prefix_len; p.ptable = d_prefix_table;
    p.n_groups = n_groups; p.pcols = prefix_cols; p.n_slots = z.n_slots;
    p.slots = (float *)(ws + z.slots);
    cudaStream_t st = (cudaStream_t)stream;
    return dtype == PF_DT_BF16 ? prefix_launch<Bf16>(p, device, sms, st) : prefix_launch<F16>(p, device, sms, st);
}
