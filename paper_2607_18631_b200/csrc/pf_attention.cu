// pf_attention.cu -- one query token per sequence against the 8-bit paged cache.
//
//   out = sum_t w_t V_t / sum_t w_t,   w_t = exp(sm q . K_t),   K_t = ks[page] * k8_t,   V_t = vs[page] * v8_t
//
// The cache is read once and dominates the traffic, so the kernel is built around keeping HBM busy:
//  - Work is cut into tiles of 32 tokens of one key / value head (2 * 32 * HD bytes).  All tiles of all sequences and heads
//    form one list, and each warp of the grid takes an equal, contiguous piece of it, whatever the lengths are.  A warp
//    works by itself: no barrier is needed in the loop.
//  - A warp keeps kStages tiles in flight with 16-byte asynchronous copies into shared memory of its own, across the
//    borders between sequences and heads.  16-byte chunks are permuted (chunk ^ line) so that reads have no bank conflicts.
//  - A (sequence, head) cut over several warps leaves partial results (running maximum, sum, weighted values) in the
//    workspace; a second kernel joins them in a fixed order.
// The query heads that share a key head are the 16 rows of the matrix instruction (16 at most per job; more heads make
// several jobs over the same tiles, which the L2 serves).  Bytes are widened to fp16, which is exact; queries are scaled by a
// power of two into fp16's range.  Scores, maxima and sums are fp32.
// The value scale joins the exponent: with p_t = exp2(s_t + log2 vs - m) in [0, 1], the values' sum is plain and the
// denominator is sum p_t / vs, one multiplication per page, so a page's scale costs nothing per element.  p is rounded to
// fp16 (11 bits) for the second product.
#include <math.h>

#include "pf_ops.cuh"

namespace pf {

constexpr int kTile = 32;                // tokens per tile
constexpr int kAttnWarps = 8;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

struct AttnArgs {
    pf_kv_cache_t c;
    const uint16_t *q;
    uint16_t *out;
    float *lse;
    const int32_t *len, *table;
    int64_t qs, os;
    int n_seq, n_heads, group, cols, row_blocks, jobs_per_seq;   // jobs_per_seq = n_kv * row_blocks
    int n_warps;                                                 // warps that share the list of tiles
    float scale_log2;                                            // sm_scale * log2(e)
    float *part;                                                 // [2 n_warps] x (16 x HD values, 16 maxima, 16 sums)
};

// length of sequence b as the kernel counts it: no negative, none past the table
__device__ __forceinline__ int seq_len(const AttnArgs &A, int b)
{
    const long long cap = (long long)A.cols * A.c.page;
    const int n = max(0, A.len[b]);
    return (long long)n < cap ? n : (int)cap;
}
__device__ __forceinline__ long long first_tile(const AttnArgs &A, long long total, int w) { return total * w / A.n_warps; }
// the warp whose piece holds tile t: the largest w with total * w / n_warps <= t
__device__ __forceinline__ int warp_of_tile(const AttnArgs &A, long long total, long long t)
{
    return (int)(((t + 1) * A.n_warps - 1) / total);
}

// prefix[b] = tiles of one job of sequences 0 .. b - 1, for b = 0 .. n_seq, by the whole block
__device__ __forceinline__ void tile_prefix(const AttnArgs &A, int *prefix, int *warp_sum)
{
    const int nt = blockDim.x, tid = threadIdx.x, lane = tid & 31, nw = nt >> 5;
    int base = 0;
    if (tid == 0) prefix[0] = 0;
    for (int b0 = 0; b0 < A.n_seq; b0 += nt) {
        int v = b0 + tid < A.n_seq ? (seq_len(A, b0 + tid) + kTile - 1) / kTile : 0;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int u = __shfl_up_sync(0xFFFFFFFFu, v, o);
            if (lane >= o) v += u;
        }
        __syncthreads();
        if (lane == 31) warp_sum[tid >> 5] = v;
        __syncthreads();
        int add = base, all = 0;
        for (int i = 0; i < nw; i++) {
            if (i < (tid >> 5)) add += warp_sum[i];
            all += warp_sum[i];
        }
        if (b0 + tid < A.n_seq) prefix[b0 + tid + 1] = add + v;
        base += all;
    }
    __syncthreads();
}
// the sequence whose tiles hold tile t of the list (prefix * jobs_per_seq is its offset); 0 <= t < total
__device__ __forceinline__ int seq_of_tile(const AttnArgs &A, const int *prefix, long long t)
{
    int lo = 0, hi = A.n_seq;       // prefix[lo] * J <= t < prefix[hi] * J
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if ((long long)prefix[mid] * A.jobs_per_seq <= t) lo = mid; else hi = mid;
    }
    return lo;
}

struct TileCursor {
    int b, job, tile, n_tiles, len; // tile of job of sequence b, whose length is len
    __device__ __forceinline__ void seek(const AttnArgs &A, const int *prefix, long long t)
    {
        b = seq_of_tile(A, prefix, t);
        n_tiles = prefix[b + 1] - prefix[b];
        len = seq_len(A, b);
        const long long r = t - (long long)prefix[b] * A.jobs_per_seq;
        job = (int)(r / n_tiles);
        tile = (int)(r - (long long)job * n_tiles);
    }
    __device__ __forceinline__ void next(const AttnArgs &A, const int *prefix)
    {
        if (++tile < n_tiles) return;
        tile = 0;
        if (++job < A.jobs_per_seq) return;
        job = 0;
        do {
            b++;
            n_tiles = b < A.n_seq ? prefix[b + 1] - prefix[b] : 1;
        } while (n_tiles == 0);
        len = b < A.n_seq ? seq_len(A, b) : 0;
    }
};

// byte offset of 16-byte chunk c of token row r inside a [kTile][HD] tile in shared memory: the eight chunks of a 128-byte line are
// permuted by the line's number
template <int HD>
__device__ __forceinline__ uint32_t chunk_at(int r, int c)
{
    const int at = r * (HD / 16) + c, line = at >> 3;
    return (uint32_t)(line * 128 + (((at & 7) ^ (line & 7)) << 4));
}

template <int HD>
struct AttnShape {
    static constexpr int kTileBytes = kTile * HD;                  // keys or values of a tile
    static constexpr int kStageBytes = 2 * kTileBytes + 16;        // and its scales: ks, vs of two 16-token halves
    static constexpr int kStages = HD == 128 ? 3 : 6;
    static constexpr int kWarpBytes = kStages * kStageBytes;
    static constexpr int kPartFloats = 16 * HD + 32;
};

template <typename T, int HD>
__global__ void __launch_bounds__(kAttnWarps * 32, 1) attention_kernel(const __grid_constant__ AttnArgs A)
{
    using S = AttnShape<HD>;
    constexpr int KS = HD / 16;               // summed steps of the first product
    constexpr int NT = HD / 8;                // 8-dim column blocks of the second
    constexpr int DG = HD / 8;                // neighbouring dims of a lane group's column set
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ int warp_sum[kAttnWarps];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
    int *prefix = reinterpret_cast<int *>(smem + kAttnWarps * S::kWarpBytes);
    tile_prefix(A, prefix, warp_sum);

    // rows without a token: zeros (their jobs have no tile)
    for (int b = blockIdx.x; b < A.n_seq; b += gridDim.x) {
        if (prefix[b + 1] != prefix[b]) continue;
        for (int i = threadIdx.x; i < A.n_heads * HD / 2; i += blockDim.x) reinterpret_cast<uint32_t *>(A.out + b * A.os)[i] = 0u;
        if (A.lse)
            for (int i = threadIdx.x; i < A.n_heads; i += blockDim.x) A.lse[(int64_t)b * A.n_heads + i] = -INFINITY;
    }

    const long long total = (long long)prefix[A.n_seq] * A.jobs_per_seq;
    const int w = warp * gridDim.x + blockIdx.x;       // neighbouring pieces on different SMs
    if (w >= A.n_warps || total == 0) return;
    const long long t_begin = first_tile(A, total, w), t_end = first_tile(A, total, w + 1);
    if (t_begin == t_end) return;

    const uint32_t ring = smem_addr(smem) + warp * S::kWarpBytes;
    const int half_pages = A.c.page == 16 ? 2 : 1;     // pages per tile

    // ---- the copying side: a cursor that runs kStages tiles ahead, its page numbers fetched one tile earlier still
    TileCursor ld;
    ld.seek(A, prefix, t_begin);
    long long t_load = t_begin;
    int page0 = -1, page1 = -1;
    auto fetch_pages = [&]() {
        const int32_t *row = A.table + (int64_t)ld.b * A.cols;
        const int at = ld.tile * kTile / A.c.page;
        page0 = row[at];
        page1 = half_pages == 2 && at + 1 < A.cols ? row[at + 1] : -1;
    };                                                  // the numbers are looked at when the next tile is loaded
    fetch_pages();
    int slot_ld = 0;
    auto load_tile = [&]() {                            // always commits a group, an empty one past the end
        if (t_load < t_end) {
            const uint32_t dst = ring + slot_ld * S::kStageBytes;
            const int h = ld.job / A.row_blocks;
            const int tok = ld.tile * kTile, left = ld.len - tok;                 // tokens of the tile that exist
            if (page0 >= A.c.n_pages) page0 = -1;
            if (half_pages == 1) page1 = page0;
            else if (page1 >= A.c.n_pages) page1 = -1;
            const int slot = tok & (A.c.page - 1);
            constexpr int LPR = HD / 16;                // lanes per token row
#pragma unroll
            for (int i = 0; i < kTile * LPR / 32; i++) {
                const int r = i * (32 / LPR) + lane / LPR, c = lane % LPR;
                const int page = r < 16 ? page0 : page1;
                const uint32_t take = (r < left && page >= 0) ? 16u : 0u;
                const int in_page = half_pages == 2 ? (r & 15) : slot + r;
                const int64_t off = take ? (((int64_t)page * A.c.n_kv + h) * A.c.page + in_page) * HD + c * 16 : 0;
                copy16(dst + chunk_at<HD>(r, c), A.c.d_k + off, take);
                copy16(dst + S::kTileBytes + chunk_at<HD>(r, c), A.c.d_v + off, take);
            }
            if (lane < 4) {                             // words: ks half 0, ks half 1, vs half 0, vs half 1
                const int page = (lane & 1) ? page1 : page0;
                const uint32_t at = dst + 2 * S::kTileBytes + lane * 4;
                if (page >= 0) copy4(at, (lane < 2 ? A.c.d_k_scale : A.c.d_v_scale) + (int64_t)page * A.c.n_kv + h);
                else asm volatile("st.shared.f32 [%0], %1;" ::"r"(at), "f"(-1.f) : "memory");
            }
            t_load++;
            slot_ld = slot_ld + 1 == S::kStages ? 0 : slot_ld + 1;
            ld.next(A, prefix);
            if (t_load < t_end) fetch_pages();
        }
        copy_commit();
    };
#pragma unroll
    for (int i = 0; i < S::kStages; i++) load_tile();

    // ---- the computing side
    TileCursor cur;
    cur.seek(A, prefix, t_begin);
    long long t = t_begin;
    int slot = 0;
    while (t < t_end) {
        // one job: rows g and g + 8 of 16 query heads
        const int b = cur.b, h = cur.job / A.row_blocks, rb = cur.job - h * A.row_blocks;
        const int rows = min(16, A.group - rb * 16);
        const int head0 = h * A.group + rb * 16;
        const int len = cur.len;
        uint32_t qa[KS][4];
        float q_scale;
        {
            // lane q of a row holds dims HD/4 * q + 4 s + {0, 1, 2, 3} at step s
            const uint16_t *q0 = A.q + b * A.qs + (int64_t)(head0 + g) * HD + q * (HD / 4);
            uint32_t raw[KS][4];
            float m = 0.f;
#pragma unroll
            for (int i = 0; i < KS / 2; i++) {
                uint4 lo = make_uint4(0, 0, 0, 0), hi = lo;
                if (g < rows) lo = *reinterpret_cast<const uint4 *>(q0 + 8 * i);
                if (g + 8 < rows) hi = *reinterpret_cast<const uint4 *>(q0 + 8 * HD + 8 * i);
                raw[2 * i][0] = lo.x; raw[2 * i][2] = lo.y; raw[2 * i + 1][0] = lo.z; raw[2 * i + 1][2] = lo.w;
                raw[2 * i][1] = hi.x; raw[2 * i][3] = hi.y; raw[2 * i + 1][1] = hi.z; raw[2 * i + 1][3] = hi.w;
            }
#pragma unroll
            for (int s = 0; s < KS; s++)
#pragma unroll
                for (int i = 0; i < 4; i++) {
                    const float2 f = pair_to_f32<T>(raw[s][i]);
                    m = fmaxf(m, fmaxf(fabsf(f.x), fabsf(f.y)));
                }
#pragma unroll
            for (int o = 16; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, o));
            // the largest query element goes to [2^13, 2^14): elements down to 2^-28 of it stay exact in fp16
            int e = (m > 0.f && m < INFINITY) ? ((int)(__float_as_uint(m) >> 23) - 127) : 0;
            e = max(-100, e) - 13;
            const float down = exp2f((float)-e);
            q_scale = exp2f((float)e);
#pragma unroll
            for (int s = 0; s < KS; s++)
#pragma unroll
                for (int i = 0; i < 4; i++) {
                    const float2 f = pair_to_f32<T>(raw[s][i]);
                    qa[s][i] = f16x2_of(f.x * down, f.y * down);
                }
        }
        const float score_scale = A.scale_log2 * q_scale;
        float o[NT][4], m0 = -INFINITY, m1 = -INFINITY, l0 = 0.f, l1 = 0.f;
#pragma unroll
        for (int j = 0; j < NT; j++) o[j][0] = o[j][1] = o[j][2] = o[j][3] = 0.f;
        const int tile0 = cur.tile;

        do {
            copy_wait<S::kStages - 1>();
            __syncwarp();
            const uint32_t kt = ring + slot * S::kStageBytes, vt = kt + S::kTileBytes;
            float s[4][4];
#pragma unroll
            for (int n = 0; n < 4; n++) {
                s[n][0] = s[n][1] = s[n][2] = s[n][3] = 0.f;
#pragma unroll
                for (int i = 0; i < HD / 64; i++) {
                    const uint4 v = lds128(kt + chunk_at<HD>(n * 8 + g, (HD / 64) * q + i));
                    const uint32_t word[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                    for (int j = 0; j < 4; j++)
                        mma16<F16>(s[n], qa[4 * i + j][0], qa[4 * i + j][1], qa[4 * i + j][2], qa[4 * i + j][3],
                                   f16x2_of_e4m3x2(word[j]), f16x2_of_e4m3x2(word[j] >> 16));
                }
            }
            const uint4 sc = lds128(kt + 2 * S::kTileBytes);
            const float ks[2] = {__uint_as_float(sc.x), __uint_as_float(sc.y)}, vs[2] = {__uint_as_float(sc.z), __uint_as_float(sc.w)};
            float lv[2], ivs[2];
#pragma unroll
            for (int i = 0; i < 2; i++) {
                const float v = fmaxf(vs[i], 8.673617379884035e-19f);     // 2^-60
                lv[i] = vs[i] < 0.f ? -INFINITY : __log2f(v);
                ivs[i] = 1.f / v;
            }
            const int left = len - cur.tile * kTile;
            float t0 = -INFINITY, t1 = -INFINITY;
#pragma unroll
            for (int n = 0; n < 4; n++) {
                const float f = score_scale * ks[n >> 1], add = lv[n >> 1];
#pragma unroll
                for (int i = 0; i < 4; i++) {
                    s[n][i] = fmaf(s[n][i], f, add);
                    if (n * 8 + 2 * q + (i & 1) >= left) s[n][i] = -INFINITY;
                }
                t0 = fmaxf(t0, fmaxf(s[n][0], s[n][1]));
                t1 = fmaxf(t1, fmaxf(s[n][2], s[n][3]));
            }
#pragma unroll
            for (int x = 1; x < 4; x <<= 1) {
                t0 = fmaxf(t0, __shfl_xor_sync(0xFFFFFFFFu, t0, x));
                t1 = fmaxf(t1, __shfl_xor_sync(0xFFFFFFFFu, t1, x));
            }
            const float n0 = fmaxf(m0, t0), n1 = fmaxf(m1, t1);
            const float z0 = n0 == -INFINITY ? 0.f : n0, z1 = n1 == -INFINITY ? 0.f : n1;
            const float a0 = exp2f(m0 - z0), a1 = exp2f(m1 - z1);
            m0 = n0;
            m1 = n1;
            l0 *= a0;
            l1 *= a1;
            if (__any_sync(0xFFFFFFFFu, a0 != 1.f || a1 != 1.f)) {
#pragma unroll
                for (int j = 0; j < NT; j++) {
                    o[j][0] *= a0;
                    o[j][1] *= a0;
                    o[j][2] *= a1;
                    o[j][3] *= a1;
                }
            }
            uint32_t p[4][2];
#pragma unroll
            for (int n = 0; n < 4; n++) {
                const float e0 = exp2f(s[n][0] - z0), e1 = exp2f(s[n][1] - z0), e2 = exp2f(s[n][2] - z1), e3 = exp2f(s[n][3] - z1);
                l0 = fmaf(e0 + e1, ivs[n >> 1], l0);
                l1 = fmaf(e2 + e3, ivs[n >> 1], l1);
                p[n][0] = f16x2_of(e0, e1);
                p[n][1] = f16x2_of(e2, e3);
            }
#pragma unroll
            for (int k = 0; k < 2; k++) {
                const int r = 16 * k + 2 * q;           // token rows r, r + 1, r + 8, r + 9
                uint32_t v[4][DG / 4];
#pragma unroll
                for (int i = 0; i < 4; i++) {
                    const int row = r + (i & 1) + (i >> 1) * 8;
                    if (HD == 128) {
                        const uint4 u = lds128(vt + chunk_at<HD>(row, g));
                        v[i][0] = u.x; v[i][1] = u.y; v[i][2 % (DG / 4)] = u.z; v[i][3 % (DG / 4)] = u.w;
                    } else {
                        const uint2 u = lds64(vt + chunk_at<HD>(row, g >> 1) + (g & 1) * 8);
                        v[i][0] = u.x; v[i][1] = u.y;
                    }
                }
#pragma unroll
                for (int i = 0; i < DG / 4; i++) {
                    // bytes of tokens (r, r + 1) and (r + 8, r + 9) side by side, dim by dim
                    const uint32_t x0 = __byte_perm(v[0][i], v[1][i], 0x5140), x1 = __byte_perm(v[0][i], v[1][i], 0x7362);
                    const uint32_t y0 = __byte_perm(v[2][i], v[3][i], 0x5140), y1 = __byte_perm(v[2][i], v[3][i], 0x7362);
#pragma unroll
                    for (int d = 0; d < 4; d++) {
                        const uint32_t b0 = f16x2_of_e4m3x2((d < 2 ? x0 : x1) >> (16 * (d & 1)));
                        const uint32_t b1 = f16x2_of_e4m3x2((d < 2 ? y0 : y1) >> (16 * (d & 1)));
                        mma16<F16>(o[4 * i + d], p[2 * k][0], p[2 * k][1], p[2 * k + 1][0], p[2 * k + 1][1], b0, b1);
                    }
                }
            }
            __syncwarp();                               // every lane has read the slot that is filled again
            load_tile();
            slot = slot + 1 == S::kStages ? 0 : slot + 1;
            t++;
            cur.tile++;
        } while (t < t_end && cur.tile < cur.n_tiles);

#pragma unroll
        for (int x = 1; x < 4; x <<= 1) {
            l0 += __shfl_xor_sync(0xFFFFFFFFu, l0, x);
            l1 += __shfl_xor_sync(0xFFFFFFFFu, l1, x);
        }
        // a lane's columns 2q, 2q + 1 of block j are dims DG * 2q + j and DG * (2q + 1) + j: 2 * DG neighbouring dims
        const bool whole = tile0 == 0 && cur.tile == cur.n_tiles;
        if (whole) {
#pragma unroll
            for (int hi = 0; hi < 2; hi++) {
                const int row = g + 8 * hi;
                if (row >= rows) continue;
                const float l = hi ? l1 : l0, inv = l > 0.f ? 1.f / l : 0.f;
                uint4 *dst = reinterpret_cast<uint4 *>(A.out + b * A.os + (int64_t)(head0 + row) * HD + q * 2 * DG);
#pragma unroll
                for (int c = 0; c < 2; c++)
#pragma unroll
                    for (int j = 0; j < DG; j += 8)
                        dst[(c * DG + j) / 8] = make_uint4(pair_of_f32<T>(o[j][2 * hi + c] * inv, o[j + 1][2 * hi + c] * inv),
                                                           pair_of_f32<T>(o[j + 2][2 * hi + c] * inv, o[j + 3][2 * hi + c] * inv),
                                                           pair_of_f32<T>(o[j + 4][2 * hi + c] * inv, o[j + 5][2 * hi + c] * inv),
                                                           pair_of_f32<T>(o[j + 6][2 * hi + c] * inv, o[j + 7][2 * hi + c] * inv));
                if (A.lse && q == 0)
                    A.lse[(int64_t)b * A.n_heads + head0 + row] = l > 0.f ? ((hi ? m1 : m0) + log2f(l)) * kLn2 : -INFINITY;
            }
        } else {
            // slot 0: a job that began before this warp's piece; slot 1: one that begins inside it
            float *part = A.part + ((int64_t)w * 2 + (tile0 == 0 ? 1 : 0)) * S::kPartFloats;
#pragma unroll
            for (int hi = 0; hi < 2; hi++) {
                const int row = g + 8 * hi;
                if (row >= rows) continue;
                float4 *dst = reinterpret_cast<float4 *>(part + row * HD + q * 2 * DG);
#pragma unroll
                for (int c = 0; c < 2; c++)
#pragma unroll
                    for (int j = 0; j < DG; j += 4)
                        dst[(c * DG + j) / 4] = make_float4(o[j][2 * hi + c], o[j + 1][2 * hi + c], o[j + 2][2 * hi + c], o[j + 3][2 * hi + c]);
                if (q == 0) {
                    part[16 * HD + row] = hi ? m1 : m0;
                    part[16 * HD + 16 + row] = hi ? l1 : l0;
                }
            }
        }
        if (cur.tile == cur.n_tiles) {
            cur.tile--;
            cur.next(A, prefix);
        }
    }
    copy_wait<0>();
}

// Joins the partial results of the jobs that were cut: block (w, y) looks at the border between pieces w and w + 1; the block
// whose border is its job's first joins the job's rows y, y + gridDim.y, ...
template <typename T, int HD>
__global__ void __launch_bounds__(128) attention_join_kernel(const __grid_constant__ AttnArgs A)
{
    using S = AttnShape<HD>;
    constexpr int LANES = HD / 4;                    // float4 lanes of a row
    constexpr int STEP = 128 / LANES;                // pieces read side by side
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ int warp_sum[4];
    __shared__ float4 acc[128];
    __shared__ float2 ml[STEP];
    int *prefix = reinterpret_cast<int *>(smem);
    tile_prefix(A, prefix, warp_sum);
    const long long total = (long long)prefix[A.n_seq] * A.jobs_per_seq;
    if (total == 0) return;
    const int w = blockIdx.x;
    const long long border = first_tile(A, total, w + 1);
    if (border >= total || border == first_tile(A, total, w)) return;
    TileCursor c;
    c.seek(A, prefix, border);
    if (c.tile == 0) return;                         // the border lies between two jobs
    const long long job_begin = border - c.tile, job_end = job_begin + c.n_tiles;
    const int w0 = warp_of_tile(A, total, job_begin), w1 = warp_of_tile(A, total, job_end - 1);
    // pieces may be empty when there are fewer tiles than warps; the first border inside the job is the one behind w0
    if (first_tile(A, total, w0 + 1) != border || w != w0) return;
    const int h = c.job / A.row_blocks, rb = c.job - h * A.row_blocks;
    const int rows = min(16, A.group - rb * 16);
    const int sub = threadIdx.x / LANES, lane = threadIdx.x % LANES;
    const int slot0 = 1;                             // w0 holds the job's beginning
    for (int row = blockIdx.y; row < rows; row += gridDim.y) {
        float m = -INFINITY, l = 0.f;
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int i = w0 + sub; i <= w1; i += STEP) {
            if (first_tile(A, total, i) == first_tile(A, total, i + 1)) continue;
            const float *part = A.part + ((int64_t)i * 2 + (i == w0 ? slot0 : 0)) * S::kPartFloats;
            const float pm = part[16 * HD + row], pl = part[16 * HD + 16 + row];
            const float4 pv = reinterpret_cast<const float4 *>(part + row * HD)[lane];
            const float nm = fmaxf(m, pm), z = nm == -INFINITY ? 0.f : nm;
            const float a = exp2f(m - z), c2 = exp2f(pm - z);
            m = nm;
            l = l * a + pl * c2;
            v.x = v.x * a + pv.x * c2;
            v.y = v.y * a + pv.y * c2;
            v.z = v.z * a + pv.z * c2;
            v.w = v.w * a + pv.w * c2;
        }
        __syncthreads();
        acc[threadIdx.x] = v;
        if (lane == 0) ml[sub] = make_float2(m, l);
        __syncthreads();
        if (sub == 0) {
            float top = -INFINITY;
#pragma unroll
            for (int i = 0; i < STEP; i++) top = fmaxf(top, ml[i].x);
            const float z = top == -INFINITY ? 0.f : top;
            float sum = 0.f;
            float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int i = 0; i < STEP; i++) {
                const float f = exp2f(ml[i].x - z);
                const float4 x = acc[i * LANES + lane];
                sum += ml[i].y * f;
                s.x += x.x * f;
                s.y += x.y * f;
                s.z += x.z * f;
                s.w += x.w * f;
            }
            const float inv = sum > 0.f ? 1.f / sum : 0.f;
            const int head = h * A.group + rb * 16 + row;
            reinterpret_cast<uint2 *>(A.out + c.b * A.os + (int64_t)head * HD)[lane] =
                make_uint2(pair_of_f32<T>(s.x * inv, s.y * inv), pair_of_f32<T>(s.z * inv, s.w * inv));
            if (A.lse && lane == 0) A.lse[(int64_t)c.b * A.n_heads + head] = sum > 0.f ? (top + log2f(sum)) * kLn2 : -INFINITY;
        }
    }
}

template <typename T, int HD>
static int attention_launch(const AttnArgs &a, int device, int sms, cudaStream_t st)
{
    using S = AttnShape<HD>;
    const size_t smem = (size_t)kAttnWarps * S::kWarpBytes + ((size_t)a.n_seq + 1) * 4;
    PF_CUDA_TRY(ensure_dynamic_smem((const void *)attention_kernel<T, HD>, device, smem), "attention_kernel shared memory");
    attention_kernel<T, HD><<<sms, kAttnWarps * 32, smem, st>>>(a);
    PF_CUDA_TRY(cudaGetLastError(), "attention_kernel launch");
    count_launch();
    const int rows = a.group < 16 ? a.group : 16;
    const size_t jsmem = ((size_t)a.n_seq + 1) * 4;
    attention_join_kernel<T, HD><<<dim3(a.n_warps, rows), 128, jsmem, st>>>(a);
    PF_CUDA_TRY(cudaGetLastError(), "attention_join_kernel launch");
    count_launch();
    return PF_OK;
}

static size_t attention_workspace_bytes(int hd, int n_warps)
{
    return (size_t)n_warps * 2 * (16 * (size_t)hd + 32) * sizeof(float);
}

}  // namespace pf

using namespace pf;

extern "C" size_t pf_decode_attention_workspace(const pf_kv_cache_t *cache, int32_t n_seq, int32_t n_heads)
{
    int device, sms;
    if (!cache || n_seq <= 0 || n_heads <= 0 || current_sm_count(&device, &sms) != PF_OK) return 256;
    return attention_workspace_bytes(cache->hd, sms * kAttnWarps);
}

extern "C" int pf_decode_attention(const pf_kv_cache_t *cache, int32_t dtype, int32_t n_seq, int32_t n_heads, const void *d_q,
                                   int64_t q_stride, const int32_t *d_len, const int32_t *d_table, int32_t table_cols, float sm_scale,
                                   void *d_out, int64_t out_stride, float *d_lse, void *d_workspace, size_t workspace_bytes,
                                   void *stream)
{
    if (!kv_cache_ok(cache) || (dtype != PF_DT_BF16 && dtype != PF_DT_F16)) return PF_EINVAL;
    if (n_seq < 0 || n_seq > PF_ATTN_MAX_SEQ || n_heads < 0 || table_cols < 0 || (int64_t)table_cols * cache->page >= (1ll << 31)) return PF_ERANGE;
    if (n_heads % cache->n_kv != 0 || !isfinite(sm_scale)) return PF_EINVAL;
    if (n_seq == 0 || n_heads == 0) return PF_OK;
    if (!d_q || !d_out || !d_len || !d_table || !aligned16(d_q) || !aligned16(d_out)) return PF_EINVAL;
    if ((uintptr_t)d_len % 4 || (uintptr_t)d_table % 4 || (uintptr_t)d_lse % 4) return PF_EINVAL;
    const int64_t row = (int64_t)n_heads * cache->hd;
    if (q_stride < row || out_stride < row || q_stride % 8 || out_stride % 8) return PF_EINVAL;
    int device, sms;
    if (int rc = current_sm_count(&device, &sms)) return rc;
    AttnArgs a;
    a.c = *cache;
    a.q = (const uint16_t *)d_q; a.out = (uint16_t *)d_out; a.lse = d_lse;
    a.len = d_len; a.table = d_table;
    a.qs = q_stride; a.os = out_stride;
    a.n_seq = n_seq; a.n_heads = n_heads; a.group = n_heads / cache->n_kv; a.cols = table_cols;
    a.row_blocks = (a.group + 15) / 16;
    a.jobs_per_seq = cache->n_kv * a.row_blocks;
    a.n_warps = sms * kAttnWarps;
    a.scale_log2 = sm_scale * kLog2e;
    a.part = (float *)d_workspace;
    if (!d_workspace || ((uintptr_t)d_workspace & 255) != 0 || workspace_bytes < attention_workspace_bytes(cache->hd, a.n_warps)) return PF_EWORKSPACE;
    cudaStream_t st = (cudaStream_t)stream;
    if (dtype == PF_DT_BF16) return cache->hd == 64 ? attention_launch<Bf16, 64>(a, device, sms, st) : attention_launch<Bf16, 128>(a, device, sms, st);
    return cache->hd == 64 ? attention_launch<F16, 64>(a, device, sms, st) : attention_launch<F16, 128>(a, device, sms, st);
}
