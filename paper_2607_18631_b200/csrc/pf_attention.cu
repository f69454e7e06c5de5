// pf_attention.cu -- one query token per sequence against the 8-bit paged cache.
//
//   out = sum_t w_t V_t / sum_t w_t,   w_t = exp(sm q . K_t),   K_t = ks[page] * k8_t,   V_t = vs[page] * v8_t
//
// The cache is read once and dominates the traffic, so the kernel is built around keeping HBM busy:
//  - Work is cut into tiles of 32 tokens of one key / value head (2 * 32 * HD bytes).  All tiles of all sequences and heads
//    form one list; each block, and within it each warp, takes an equal, contiguous piece of it, whatever the lengths are.  A
//    warp works by itself: no barrier is needed in the loop.
//  - A warp keeps kStages tiles in flight with 16-byte asynchronous copies into shared memory of its own, across the
//    borders between sequences and heads.  16-byte chunks are permuted (chunk ^ line) so that reads have no bank conflicts.
//  - A (sequence, head) cut over several warps leaves partial results (running maximum, sum, weighted values).  A block joins
//    those of its warps, and a second kernel those of the blocks, in a fixed order.  (Joining all warps' parts in the second kernel took
//    17 us instead of 5 for one sequence of 131071 tokens.)  The second kernel is let in when the first one's loops end, and finds its
//    job before it waits for the parts: 1.2 us less.  (Let in at the start, its waiting blocks cost the first kernel that much.)
// The first product is K q^T: 16 tokens of a tile are the rows of the matrix instruction, 8 query heads that share the key head its
// columns (16 heads as two column blocks; more make several jobs over the same tiles, which the L2 serves).  The second is V^T p^T: 16 dims
// are the rows.  So with up to 8 heads a key head, and with one, no more than the unused columns is computed in vain (heads as rows: twice
// the products, accumulators and exponentials, 62 us instead of 53 for one sequence of 131071 tokens, 8 key and 64 query heads of 128).
// Measured (one B200, device time of both kernels): that sequence (269 MB) 57 us, of which the copies alone take 45; 48 ragged sequences up to 8192
// tokens, 32 / 8 heads (418 MB) 86 us, copies alone 68; 64 / 4 heads (209 MB) 71 us; 777 tokens, 16 heads of 64: 9.6 us.
// Bytes are widened to fp16, which is exact; queries are scaled by a power of two a head into fp16's range.  Scores, maxima and
// sums are fp32.
// The value scale joins the exponent: with p_t = exp2(s_t + log2 vs - z), the values' sum is plain and the denominator
// is sum p_t / vs, one multiplication per page, so a page's scale costs nothing per element.  p is rounded to fp16 for the
// second product, and z lies 15 below the maximum (rounded up, so that p <= 2^15 whatever the scores' size): weights keep
// 11 bits down to 2^-29 of the largest and count down to 2^-40 of it.  (With p <= 1 it was 2^-14 and 2^-25: behind one
// token of nearly all the weight, 100,000 others lost up to a sixth of theirs.)
#include <math.h>

#include "pf_ops.cuh"

namespace pf {

constexpr int kTile = 32;                // tokens per tile
constexpr int kBlockTiles = 8;           // a block takes no fewer tiles while others have none
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kLift = 15.f;            // log2 of the largest weight in the second product

struct AttnArgs {
    pf_kv_cache_t c;
    const uint16_t *q;
    uint16_t *out;
    float *lse;
    const int32_t *len, *table;
    int64_t qs, os;
    int n_seq, n_heads, group, cols, row_blocks, jobs_per_seq;   // jobs_per_seq = n_kv * row_blocks, row_blocks of 8 NB heads
    float scale_log2;                                            // sm_scale * log2(e)
    float *part;                                                 // [warps] x (8 NB x HD values, 8 NB references z, 8 NB sums), then [2 blocks] of the same
};

// length of sequence b as the kernel counts it: no negative, none past the table
__device__ __forceinline__ int seq_len(const AttnArgs &A, int b)
{
    const long long cap = (long long)A.cols * A.c.page;
    const int n = max(0, A.len[b]);
    return (long long)n < cap ? n : (int)cap;
}
// `total` tiles are cut into n equal pieces: the first tile of piece i, and the piece that holds tile t
__device__ __forceinline__ long long first_tile(long long total, int n, int i) { return total * i / n; }
__device__ __forceinline__ int piece_of(long long total, int n, long long t) { return (int)(((t + 1) * n - 1) / total); }
// blocks that share the list: few tiles are spread over many SMs, but not one by one
__device__ __forceinline__ int blocks_used(long long total, int sms)
{
    const long long n = (total + kBlockTiles - 1) / kBlockTiles;
    return n < sms ? (int)n : sms;
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

template <int HD, int NB>
struct AttnShape {
    static constexpr int kTileBytes = kTile * HD;                  // keys or values of a tile
    static constexpr int kStageBytes = 2 * kTileBytes + 16;        // and its scales: ks, vs of two 16-token halves
    // 8 warps with 16 KB in flight each.  Measured for 131071 tokens (us, first kernel): 6 warps 53.0, 8: 50.8, 10: 55.5, 12: 54.1; three
    // stages 53.5: more copies in flight than HBM needs only lengthen its queues.
    static constexpr int kWarps = 8;
    static constexpr int kStages = 2 * (128 / HD);
    static constexpr int kWarpBytes = kStages * kStageBytes;
    static constexpr int kHeads = 8 * NB;
    static constexpr int kPartFloats = kHeads * (HD + 2);
};

// four e4m3 bytes -> two fp16 pairs
__device__ __forceinline__ void widen4(uint32_t w, uint32_t &lo, uint32_t &hi)
{
    asm("{\n.reg .b16 l, h;\nmov.b32 {l, h}, %2;\ncvt.rn.f16x2.e4m3x2 %0, l;\ncvt.rn.f16x2.e4m3x2 %1, h;\n}" : "=r"(lo), "=r"(hi) : "r"(w));
}
// 8 x 8 fp16 matrix, a row's neighbouring pair per lane -> its transpose in the same form
__device__ __forceinline__ uint32_t transpose8(uint32_t v)
{
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
    return r;
}
__device__ __forceinline__ float ex2(float x)      // 2^x, results below the normals to zero
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// A warp joins one row of up to 32 partial results at a time: lane k holds the pointer to part k (NULL: none, not for lane 0) of `count`.  Largest
// reference, sum and values (V = HD / 32 neighbouring ones a lane) are carried from call to call.
template <int HD, int NB>
struct RowJoin {
    static constexpr int V = HD / 32;
    float top, sum, v[V];
    __device__ __forceinline__ void clear()
    {
        top = -INFINITY;
        sum = 0.f;
#pragma unroll
        for (int k = 0; k < V; k++) v[k] = 0.f;
    }
    __device__ __forceinline__ void add(const float *part, int row, int count)
    {
        constexpr int H = AttnShape<HD, NB>::kHeads;
        const int lane = threadIdx.x & 31;
        const float m = part ? part[H * HD + row] : -INFINITY, l = part ? part[H * (HD + 1) + row] : 0.f;
        float n = fmaxf(top, m);
#pragma unroll
        for (int x = 16; x; x >>= 1) n = fmaxf(n, __shfl_xor_sync(0xFFFFFFFFu, n, x));
        const float z = n == -INFINITY ? 0.f : n, old = exp2f(top - z), f = exp2f(m - z);
        float add = l * f;
#pragma unroll
        for (int x = 16; x; x >>= 1) add += __shfl_xor_sync(0xFFFFFFFFu, add, x);
        top = n;
        sum = fmaf(sum, old, add);
#pragma unroll
        for (int k = 0; k < V; k++) v[k] *= old;
        // a missing part, and what the unrolled loop reads past the last, is part 0 with weight 0: no branch between the loads
        const unsigned long long any = __shfl_sync(0xFFFFFFFFu, (unsigned long long)part, 0);
        const unsigned long long mine = part ? (unsigned long long)part : any;
#pragma unroll 8
        for (int i = 0; i < (count + 7) / 8 * 8; i++) {
            const float *from = (const float *)__shfl_sync(0xFFFFFFFFu, mine, i);
            const float w = __shfl_sync(0xFFFFFFFFu, f, i);
            if (V == 4) {
                const float4 y = *reinterpret_cast<const float4 *>(from + row * HD + lane * V);
                v[0] = fmaf(y.x, w, v[0]);
                v[1] = fmaf(y.y, w, v[1]);
                v[2 % V] = fmaf(y.z, w, v[2 % V]);
                v[3 % V] = fmaf(y.w, w, v[3 % V]);
            } else {
                const float2 y = *reinterpret_cast<const float2 *>(from + row * HD + lane * V);
                v[0] = fmaf(y.x, w, v[0]);
                v[1] = fmaf(y.y, w, v[1]);
            }
        }
    }
    template <typename T>
    __device__ __forceinline__ void write(const AttnArgs &A, int b, int head)
    {
        const int lane = threadIdx.x & 31;
        const float inv = sum == 0.f ? 0.f : 1.f / sum;      // (a sum that is not a number stays one)
        uint32_t *dst = reinterpret_cast<uint32_t *>(A.out + b * A.os + (int64_t)head * HD) + lane * V / 2;
#pragma unroll
        for (int k = 0; k < V; k += 2) dst[k / 2] = pair_of_f32<T>(v[k] * inv, v[k + 1] * inv);
        if (A.lse && lane == 0) A.lse[(int64_t)b * A.n_heads + head] = sum == 0.f ? -INFINITY : (top + log2f(sum)) * kLn2;
    }
};

template <typename T, int HD, int NB>
__global__ void __launch_bounds__(AttnShape<HD, NB>::kWarps * 32, 1) attention_kernel(const __grid_constant__ AttnArgs A)
{
    using S = AttnShape<HD, NB>;
    constexpr int KS = HD / 16;               // summed steps of the first product
    constexpr int MT = HD / 16;               // 16-dim row blocks of the second
    constexpr int DG = HD / 8;                // neighbouring dims of a lane group
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ int warp_sum[S::kWarps];
    __shared__ long long seg_job[2 * S::kWarps];       // cut jobs: the list's tile where each begins, -1 for none
    __shared__ int seg_b[2 * S::kWarps], seg_no[2 * S::kWarps], seg_tiles[2 * S::kWarps];
    __shared__ const float *seg_part[2 * S::kWarps];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
    int *prefix = reinterpret_cast<int *>(smem + S::kWarps * S::kWarpBytes);
    tile_prefix(A, prefix, warp_sum);

    // rows without a token: zeros (their jobs have no tile)
    for (int b = blockIdx.x; b < A.n_seq; b += gridDim.x) {
        if (prefix[b + 1] != prefix[b]) continue;
        for (int i = threadIdx.x; i < A.n_heads * HD / 2; i += blockDim.x) reinterpret_cast<uint32_t *>(A.out + b * A.os)[i] = 0u;
        if (A.lse)
            for (int i = threadIdx.x; i < A.n_heads; i += blockDim.x) A.lse[(int64_t)b * A.n_heads + i] = -INFINITY;
    }

    const long long total = (long long)prefix[A.n_seq] * A.jobs_per_seq;
    if (total == 0) return;
    const int n_blocks = blocks_used(total, gridDim.x);
    if ((int)blockIdx.x >= n_blocks) return;
    const long long block_begin = first_tile(total, n_blocks, blockIdx.x), block_end = first_tile(total, n_blocks, blockIdx.x + 1);
    const long long t_begin = block_begin + first_tile(block_end - block_begin, S::kWarps, warp);
    const long long t_end = block_begin + first_tile(block_end - block_begin, S::kWarps, warp + 1);
    if (lane < 2) seg_job[2 * warp + lane] = -1;
    __syncwarp();

    const uint32_t ring = smem_addr(smem) + warp * S::kWarpBytes;
    const bool two_pages = A.c.page == 16;             // a tile of two pages

    // ---- the copying side: a cursor that runs kStages tiles ahead, its page numbers fetched one tile earlier still
    TileCursor ld;
    if (t_begin < t_end) ld.seek(A, prefix, t_begin);
    long long t_load = t_begin;
    int page0 = -1, page1 = -1;
    auto fetch_pages = [&]() {
        const int32_t *row = A.table + (int64_t)ld.b * A.cols;
        const int at = ld.tile * kTile / A.c.page;
        page0 = row[at];
        page1 = two_pages && at + 1 < A.cols ? row[at + 1] : -1;
    };                                                  // the numbers are looked at when the next tile is loaded
    if (t_begin < t_end) fetch_pages();
    int slot_ld = 0;
    // a lane's places in a tile: rows lane / LPR + i * (32 / LPR), chunk lane % LPR
    constexpr int LPR = HD / 16, RPI = 32 / LPR, COPIES = kTile / RPI;
    const int lr = lane / LPR, lc = lane % LPR;
    auto load_tile = [&]() {                            // always commits a group, an empty one past the end
        if (t_load < t_end) {
            const uint32_t dst = ring + slot_ld * S::kStageBytes;
            const int h = ld.job / A.row_blocks;
            const int tok = ld.tile * kTile, left = ld.len - tok;                 // tokens of the tile that exist
            if (page0 >= A.c.n_pages) page0 = -1;
            if (!two_pages) page1 = page0;
            else if (page1 >= A.c.n_pages) page1 = -1;
            const int64_t ph0 = (int64_t)page0 * A.c.n_kv + h, ph1 = (int64_t)page1 * A.c.n_kv + h;
            if (left >= kTile && page0 >= 0 && !two_pages) {
                const int64_t at = (ph0 * A.c.page + (tok & (A.c.page - 1)) + lr) * HD + lc * 16;
                const uint8_t *k = A.c.d_k + at, *v = A.c.d_v + at;
#pragma unroll
                for (int i = 0; i < COPIES; i++) {
                    const uint32_t to = dst + chunk_at<HD>(lr + i * RPI, lc);
                    copy16(to, k + i * RPI * HD, 16u);
                    copy16(to + S::kTileBytes, v + i * RPI * HD, 16u);
                }
            } else {
#pragma unroll
                for (int i = 0; i < COPIES; i++) {
                    const int r = lr + i * RPI;
                    const uint32_t take = (r < left && (r < 16 ? page0 : page1) >= 0) ? 16u : 0u;
                    const int in_page = two_pages ? (r & 15) : (tok & (A.c.page - 1)) + r;
                    const int64_t at = take ? ((r < 16 ? ph0 : ph1) * A.c.page + in_page) * HD + lc * 16 : 0;
                    const uint32_t to = dst + chunk_at<HD>(r, lc);
                    copy16(to, A.c.d_k + at, take);
                    copy16(to + S::kTileBytes, A.c.d_v + at, take);
                }
            }
            if (lane < 4) {                             // words: ks half 0, ks half 1, vs half 0, vs half 1
                const uint32_t to = dst + 2 * S::kTileBytes + lane * 4;
                if (((lane & 1) ? page1 : page0) >= 0) copy4(to, (lane < 2 ? A.c.d_k_scale : A.c.d_v_scale) + ((lane & 1) ? ph1 : ph0));
                else asm volatile("st.shared.f32 [%0], %1;" ::"r"(to), "f"(-1.f) : "memory");
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
    if (t_begin < t_end) cur.seek(A, prefix, t_begin);
    long long t = t_begin;
    int slot = 0;
    while (t < t_end) {
        // one job: 8 NB query heads of one key head; lane 4 g + q holds head g (of each block) of q, and heads 2q, 2q + 1 of sums
        const int b = cur.b, h = cur.job / A.row_blocks, rb = cur.job - h * A.row_blocks;
        const int heads = min(S::kHeads, A.group - rb * S::kHeads);
        const int head0 = h * A.group + rb * S::kHeads;
        uint32_t qb[NB][KS][2];
        float score_scale[NB][2];
        // lane q of a head holds dims HD/4 * q + 4 s + {0, 1, 2, 3} at step s
#pragma unroll
        for (int nb = 0; nb < NB; nb++) {
            const uint16_t *src = A.q + b * A.qs + (int64_t)(head0 + nb * 8 + g) * HD + q * (HD / 4);
#pragma unroll
            for (int i = 0; i < KS / 2; i++) {
                uint4 v = make_uint4(0, 0, 0, 0);
                if (nb * 8 + g < heads) v = *reinterpret_cast<const uint4 *>(src + 8 * i);
                qb[nb][2 * i][0] = v.x; qb[nb][2 * i][1] = v.y; qb[nb][2 * i + 1][0] = v.z; qb[nb][2 * i + 1][1] = v.w;
            }
            // A head's largest finite element goes to [2^13, 2^14): elements down to 2^-28 of it stay exact in fp16.  Each head has its own power
            // of two: what one head's query holds, infinities included, is nothing to the others.
            float top = 0.f;
#pragma unroll
            for (int s = 0; s < KS; s++)
#pragma unroll
                for (int i = 0; i < 2; i++) {
                    const float2 f = pair_to_f32<T>(qb[nb][s][i]);
                    top = fmaxf(top, fmaxf(fabsf(f.x) < INFINITY ? fabsf(f.x) : 0.f, fabsf(f.y) < INFINITY ? fabsf(f.y) : 0.f));
                }
            top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
            top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
            int e = top > 0.f ? ((int)(__float_as_uint(top) >> 23) - 127) : 0;
            e = max(-100, e) - 13;
            const float down = exp2f((float)-e), up = A.scale_log2 * exp2f((float)e);
            score_scale[nb][0] = __shfl_sync(0xFFFFFFFFu, up, 8 * q);        // of heads 2q and 2q + 1
            score_scale[nb][1] = __shfl_sync(0xFFFFFFFFu, up, 8 * q + 4);
#pragma unroll
            for (int s = 0; s < KS; s++)
#pragma unroll
                for (int i = 0; i < 2; i++) {
                    const float2 f = pair_to_f32<T>(qb[nb][s][i]);
                    qb[nb][s][i] = f16x2_of(f.x * down, f.y * down);
                }
        }
        // m: the references z; l: the denominators, in two levels: 32 tiles are added up in l32 first, since the weights of a long
        // sequence may each lie below the last bit of a sum that holds a large one
        float o[NB][MT][4], m[NB][2], l[NB][2], l32[NB][2];
#pragma unroll
        for (int nb = 0; nb < NB; nb++) {
            m[nb][0] = m[nb][1] = -INFINITY;
            l[nb][0] = l[nb][1] = l32[nb][0] = l32[nb][1] = 0.f;
#pragma unroll
            for (int j = 0; j < MT; j++) o[nb][j][0] = o[nb][j][1] = o[nb][j][2] = o[nb][j][3] = 0.f;
        }
        const int tile0 = cur.tile;

        do {
            copy_wait<S::kStages - 1>();
            __syncwarp();
            const uint32_t kt = ring + slot * S::kStageBytes, vt = kt + S::kTileBytes;
            // s[mt][nb]: tokens 16 mt + g and + 8, heads 8 nb + 2q and + 1
            float s[2][NB][4];
#pragma unroll
            for (int mt = 0; mt < 2; mt++) {
#pragma unroll
                for (int nb = 0; nb < NB; nb++) s[mt][nb][0] = s[mt][nb][1] = s[mt][nb][2] = s[mt][nb][3] = 0.f;
#pragma unroll
                for (int i = 0; i < HD / 64; i++) {
                    const uint4 u = lds128(kt + chunk_at<HD>(mt * 16 + g, (HD / 64) * q + i));
                    const uint4 v = lds128(kt + chunk_at<HD>(mt * 16 + g + 8, (HD / 64) * q + i));
                    const uint32_t wu[4] = {u.x, u.y, u.z, u.w}, wv[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                    for (int j = 0; j < 4; j++) {
                        uint32_t a0, a1, a2, a3;
                        widen4(wu[j], a0, a2);
                        widen4(wv[j], a1, a3);
#pragma unroll
                        for (int nb = 0; nb < NB; nb++) mma16<F16>(s[mt][nb], a0, a1, a2, a3, qb[nb][4 * i + j][0], qb[nb][4 * i + j][1]);
                    }
                }
            }
            const uint4 sc = lds128(kt + 2 * S::kTileBytes);
            const float ks[2] = {__uint_as_float(sc.x), __uint_as_float(sc.y)}, vs[2] = {__uint_as_float(sc.z), __uint_as_float(sc.w)};
            float lv[2], ivs[2];
#pragma unroll
            for (int i = 0; i < 2; i++) {
                const float v = fmaxf(vs[i], 8.673617379884035e-19f);     // 2^-60
                lv[i] = vs[i] < 0.f ? -INFINITY : __log2f(v);
                ivs[i] = __fdividef(1.f, v);
            }
            const int left = cur.len - cur.tile * kTile;
            uint32_t p[2][NB][2];
#pragma unroll
            for (int nb = 0; nb < NB; nb++) {
                float t0 = -INFINITY, t1 = -INFINITY;           // the tile's largest scores, then the references they ask for
#pragma unroll
                for (int mt = 0; mt < 2; mt++) {
                    const float f[2] = {score_scale[nb][0] * ks[mt], score_scale[nb][1] * ks[mt]};
#pragma unroll
                    for (int i = 0; i < 4; i++) s[mt][nb][i] = fmaf(s[mt][nb][i], f[i & 1], lv[mt]);
                }
                if (left < kTile) {
#pragma unroll
                    for (int mt = 0; mt < 2; mt++)
#pragma unroll
                        for (int i = 0; i < 4; i++)
                            if (mt * 16 + g + (i >> 1) * 8 >= left) s[mt][nb][i] = -INFINITY;
                }
#pragma unroll
                for (int mt = 0; mt < 2; mt++) {
                    t0 = fmaxf(t0, fmaxf(s[mt][nb][0], s[mt][nb][2]));
                    t1 = fmaxf(t1, fmaxf(s[mt][nb][1], s[mt][nb][3]));
                }
                t0 = __fsub_ru(t0, kLift);
                t1 = __fsub_ru(t1, kLift);
                // a lane looks at its own tokens first: in most tiles no head has a new maximum
                if (__any_sync(0xFFFFFFFFu, t0 > m[nb][0] || t1 > m[nb][1])) {
#pragma unroll
                    for (int x = 4; x < 32; x <<= 1) {
                        t0 = fmaxf(t0, __shfl_xor_sync(0xFFFFFFFFu, t0, x));
                        t1 = fmaxf(t1, __shfl_xor_sync(0xFFFFFFFFu, t1, x));
                    }
                    const float n0 = fmaxf(m[nb][0], t0), n1 = fmaxf(m[nb][1], t1);
                    const float a0 = n0 == -INFINITY ? 1.f : ex2(m[nb][0] - n0), a1 = n1 == -INFINITY ? 1.f : ex2(m[nb][1] - n1);
                    m[nb][0] = n0;
                    m[nb][1] = n1;
                    l[nb][0] *= a0;
                    l[nb][1] *= a1;
                    l32[nb][0] *= a0;
                    l32[nb][1] *= a1;
#pragma unroll
                    for (int j = 0; j < MT; j++) {
                        o[nb][j][0] *= a0;
                        o[nb][j][1] *= a1;
                        o[nb][j][2] *= a0;
                        o[nb][j][3] *= a1;
                    }
                }
                const float z0 = m[nb][0] == -INFINITY ? 0.f : m[nb][0], z1 = m[nb][1] == -INFINITY ? 0.f : m[nb][1];
#pragma unroll
                for (int mt = 0; mt < 2; mt++) {
                    const float e0 = ex2(s[mt][nb][0] - z0), e1 = ex2(s[mt][nb][1] - z1), e2 = ex2(s[mt][nb][2] - z0), e3 = ex2(s[mt][nb][3] - z1);
                    l32[nb][0] = fmaf(e0 + e2, ivs[mt], l32[nb][0]);
                    l32[nb][1] = fmaf(e1 + e3, ivs[mt], l32[nb][1]);
                    // heads as columns, tokens as rows -> the second product's other way round
                    p[mt][nb][0] = transpose8(f16x2_of(e0, e1));
                    p[mt][nb][1] = transpose8(f16x2_of(e2, e3));
                }
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
                for (int i = 0; i < DG / 4; i++)
#pragma unroll
                    for (int d = 0; d < 2; d++) {
                        // bytes of tokens (r, r + 1) and (r + 8, r + 9) side by side: dims 4 i + 2 d and 4 i + 2 d + 1 of the lane group
                        const uint32_t sel = d ? 0x7362 : 0x5140;
                        uint32_t a0, a1, a2, a3;
                        widen4(__byte_perm(v[0][i], v[1][i], sel), a0, a1);
                        widen4(__byte_perm(v[2][i], v[3][i], sel), a2, a3);
#pragma unroll
                        for (int nb = 0; nb < NB; nb++) mma16<F16>(o[nb][2 * i + d], a0, a1, a2, a3, p[k][nb][0], p[k][nb][1]);
                    }
            }
            __syncwarp();                               // every lane has read the slot that is filled again
            load_tile();
            slot = slot + 1 == S::kStages ? 0 : slot + 1;
            t++;
            cur.tile++;
            if ((cur.tile & 31) == 0 || t == t_end || cur.tile == cur.n_tiles) {
#pragma unroll
                for (int nb = 0; nb < NB; nb++)
#pragma unroll
                    for (int c = 0; c < 2; c++) {
                        l[nb][c] += l32[nb][c];
                        l32[nb][c] = 0.f;
                    }
            }
        } while (t < t_end && cur.tile < cur.n_tiles);

        // a lane has heads 8 nb + 2q, + 1 and dims DG * g .. + DG - 1: row block j's rows are dims 2 j and 2 j + 1 of these
        const bool whole = tile0 == 0 && cur.tile == cur.n_tiles;
        // slot 0: a job that began before this warp's piece; slot 1: one that begins inside it
        const int seg = 2 * warp + (tile0 == 0 ? 1 : 0);
        // a warp's last segment goes to its own stages, which are done with
        static_assert(S::kPartFloats * 4 <= S::kWarpBytes, "a partial result fits a warp's stages");
        float *part = t == t_end ? reinterpret_cast<float *>(smem + warp * S::kWarpBytes) : A.part + ((int64_t)blockIdx.x * S::kWarps + warp) * S::kPartFloats;
        if (!whole && lane == 0) {
            seg_job[seg] = t - cur.tile;                // t stands behind the job's last tile here
            seg_b[seg] = b;
            seg_no[seg] = cur.job;
            seg_tiles[seg] = cur.n_tiles;
            seg_part[seg] = part;
        }
#pragma unroll
        for (int nb = 0; nb < NB; nb++)
#pragma unroll
            for (int c = 0; c < 2; c++) {
                float sum = l[nb][c];
#pragma unroll
                for (int x = 4; x < 32; x <<= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, x);
                const int row = nb * 8 + 2 * q + c;
                if (row >= heads) continue;
                if (whole) {
                    const float inv = sum == 0.f ? 0.f : 1.f / sum;      // (a sum that is not a number stays one)
                    uint4 *dst = reinterpret_cast<uint4 *>(A.out + b * A.os + (int64_t)(head0 + row) * HD + g * DG);
#pragma unroll
                    for (int j = 0; j < MT; j += 4)
                        dst[j / 4] = make_uint4(pair_of_f32<T>(o[nb][j][c] * inv, o[nb][j][c + 2] * inv),
                                                pair_of_f32<T>(o[nb][j + 1][c] * inv, o[nb][j + 1][c + 2] * inv),
                                                pair_of_f32<T>(o[nb][j + 2][c] * inv, o[nb][j + 2][c + 2] * inv),
                                                pair_of_f32<T>(o[nb][j + 3][c] * inv, o[nb][j + 3][c + 2] * inv));
                    if (A.lse && g == 0) A.lse[(int64_t)b * A.n_heads + head0 + row] = sum == 0.f ? -INFINITY : (m[nb][c] + log2f(sum)) * kLn2;
                } else {
                    float4 *dst = reinterpret_cast<float4 *>(part + row * HD + g * DG);
#pragma unroll
                    for (int j = 0; j < MT; j += 2)
                        dst[j / 2] = make_float4(o[nb][j][c], o[nb][j][c + 2], o[nb][j + 1][c], o[nb][j + 1][c + 2]);
                    if (g == 0) {
                        part[S::kHeads * HD + row] = m[nb][c];
                        part[S::kHeads * (HD + 1) + row] = sum;
                    }
                }
            }
        if (cur.tile == cur.n_tiles) {
            cur.tile--;
            cur.next(A, prefix);
        }
    }
    copy_wait<0>();
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    __syncthreads();

    // ---- the block's cut jobs, whose segments follow one another: a warp per row
    int task = 0;
    for (int i = 0; i < 2 * S::kWarps;) {
        const long long job_begin = seg_job[i];
        if (job_begin < 0) {
            i++;
            continue;
        }
        const int first = i, b = seg_b[i], job = seg_no[i], n_tiles = seg_tiles[i];
        for (i++; i < 2 * S::kWarps && (seg_job[i] < 0 || seg_job[i] == job_begin); i++) {}
        const int h = job / A.row_blocks, rb = job - h * A.row_blocks;
        const int heads = min(S::kHeads, A.group - rb * S::kHeads);
        const bool begins = job_begin >= block_begin, complete = begins && job_begin + n_tiles <= block_end;
        const float *part = first + lane < i && seg_job[first + lane] >= 0 ? seg_part[first + lane] : nullptr;
        float *to = A.part + ((int64_t)gridDim.x * S::kWarps + 2 * blockIdx.x + (begins ? 1 : 0)) * S::kPartFloats;
        for (int row = 0; row < heads; row++) {
            if (task++ % S::kWarps != warp) continue;
            RowJoin<HD, NB> r;
            r.clear();
            r.add(part, row, i - first);
            if (complete) {
                r.template write<T>(A, b, h * A.group + rb * S::kHeads + row);
                continue;
            }
#pragma unroll
            for (int k = 0; k < HD / 32; k++) to[row * HD + lane * (HD / 32) + k] = r.v[k];
            if (lane == 0) {
                to[S::kHeads * HD + row] = r.top;
                to[S::kHeads * (HD + 1) + row] = r.sum;
            }
        }
    }
}

// Joins the blocks' partial results of the jobs that were cut between blocks, a row (head) per warp.  With no more jobs than borders
// between blocks, block x looks at job x; otherwise at border x, and the first border inside a job has it joined.
constexpr int kJoinWarps = 8;
template <typename T, int HD, int NB>
__global__ void __launch_bounds__(kJoinWarps * 32) attention_join_kernel(const __grid_constant__ AttnArgs A, const int grid)
{
    using S = AttnShape<HD, NB>;
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ int warp_sum[kJoinWarps];
    int *prefix = reinterpret_cast<int *>(smem);
    tile_prefix(A, prefix, warp_sum);
    // Which job, by the lengths alone, which no kernel of this call writes; every block then waits for the first kernel to end, those without work
    // too: what follows on the stream waits for this kernel only.
    const long long total = (long long)prefix[A.n_seq] * A.jobs_per_seq;
    const int n = blocks_used(total, grid), lane = threadIdx.x & 31;
    TileCursor c;
    long long job_begin = 0;
    int w0 = 0, w1 = 0;
    auto find = [&]() {
        if (total == 0) return;
        if (gridDim.x == (unsigned)A.n_seq * (unsigned)A.jobs_per_seq) {
            c.b = blockIdx.x / A.jobs_per_seq;
            c.job = blockIdx.x - c.b * A.jobs_per_seq;
            c.n_tiles = prefix[c.b + 1] - prefix[c.b];
            if (c.n_tiles == 0) return;
            job_begin = (long long)prefix[c.b] * A.jobs_per_seq + (long long)c.job * c.n_tiles;
        } else {
            if ((int)blockIdx.x + 1 >= n) return;
            const long long border = first_tile(total, n, blockIdx.x + 1);
            c.seek(A, prefix, border);
            if (c.tile == 0) return;                     // the border lies between two jobs
            job_begin = border - c.tile;
            if (piece_of(total, n, job_begin) != (int)blockIdx.x) return;      // not the job's first border
        }
        w0 = piece_of(total, n, job_begin);
        w1 = piece_of(total, n, job_begin + c.n_tiles - 1);
    };
    find();
    asm volatile("griddepcontrol.wait;" ::: "memory");
    if (w0 == w1) return;                            // no job, or one written by its block
    const int h = c.job / A.row_blocks, rb = c.job - h * A.row_blocks;
    const int heads = min(S::kHeads, A.group - rb * S::kHeads);
    const float *from = A.part + (int64_t)grid * S::kWarps * S::kPartFloats;
    for (int row = threadIdx.x >> 5; row < heads; row += kJoinWarps) {
        RowJoin<HD, NB> r;
        r.clear();
        for (int i0 = w0; i0 <= w1; i0 += 32) {      // a job begins in slot 1 of its first block and goes on in slot 0 of the others
            const int i = i0 + lane;
            r.add(i <= w1 ? from + ((int64_t)i * 2 + (i == w0 ? 1 : 0)) * S::kPartFloats : nullptr, row, min(32, w1 - i0 + 1));
        }
        r.template write<T>(A, c.b, h * A.group + rb * S::kHeads + row);
    }
}

template <typename T, int HD, int NB>
static int attention_launch(AttnArgs a, int device, int sms, cudaStream_t st)
{
    using S = AttnShape<HD, NB>;
    a.row_blocks = (a.group + S::kHeads - 1) / S::kHeads;
    a.jobs_per_seq = a.c.n_kv * a.row_blocks;
    const size_t table = ((size_t)a.n_seq + 1) * 4, smem = (size_t)S::kWarps * S::kWarpBytes + table;
    PF_CUDA_TRY(ensure_dynamic_smem((const void *)attention_kernel<T, HD, NB>, device, smem), "attention_kernel shared memory");
    attention_kernel<T, HD, NB><<<sms, S::kWarps * 32, smem, st>>>(a);
    PF_CUDA_TRY(cudaGetLastError(), "attention_kernel launch");
    count_launch();
    const long long jobs = (long long)a.n_seq * a.jobs_per_seq;
    PF_CUDA_TRY(launch_chained(attention_join_kernel<T, HD, NB>, dim3((unsigned)(jobs < sms ? jobs : sms)), dim3(kJoinWarps * 32), table, st, a, sms),
                "attention_join_kernel launch");
    count_launch();
    return PF_OK;
}
template <typename T, int HD>
static int attention_launch(const AttnArgs &a, int device, int sms, cudaStream_t st)
{
    return a.group <= 8 ? attention_launch<T, HD, 1>(a, device, sms, st) : attention_launch<T, HD, 2>(a, device, sms, st);
}

// a slot per warp and two per block, of 16 heads at most
static size_t attention_workspace_bytes(int hd, int sms)
{
    return (size_t)sms * 10 * 16 * ((size_t)hd + 2) * sizeof(float);
}

}  // namespace pf

using namespace pf;

extern "C" size_t pf_decode_attention_workspace(const pf_kv_cache_t *cache, int32_t n_seq, int32_t n_heads)
{
    int device, sms;
    if (!cache || n_seq <= 0 || n_heads <= 0 || current_sm_count(&device, &sms) != PF_OK) return 256;
    return attention_workspace_bytes(cache->hd, sms);
}

extern "C" int pf_decode_attention(const pf_kv_cache_t *cache, int32_t dtype, int32_t n_seq, int32_t n_heads, const void *d_q,
                                   int64_t q_stride, const int32_t *d_len, const int32_t *d_table, int32_t table_cols, float sm_scale,
                                   void *d_out, int64_t out_stride, float *d_lse, void *d_workspace, size_t workspace_bytes,
                                   void *stream)
{
    if (!kv_cache_ok(cache) || (dtype != PF_DT_BF16 && dtype != PF_DT_F16)) return PF_EINVAL;
    if (n_seq < 0 || n_seq > PF_ATTN_MAX_SEQ || n_heads < 0 || table_cols < 0 || (int64_t)table_cols * cache->page >= (1ll << 31)) return PF_ERANGE;
    // the kernels count a job's tiles of all sequences in 32 bits, and the lengths, which the host does not see, are bounded by the table only
    const int64_t tiles = ((int64_t)table_cols * cache->page + kTile - 1) / kTile;
    if ((int64_t)n_seq * tiles >= (1ll << 31)) return PF_ERANGE;
    if (n_heads % cache->n_kv != 0 || !isfinite(sm_scale)) return PF_EINVAL;
    if (n_seq == 0 || n_heads == 0) return PF_OK;
    if (!d_q || !d_out || !d_len || (!d_table && table_cols > 0) || !aligned16(d_q) || !aligned16(d_out)) return PF_EINVAL;
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
    a.scale_log2 = sm_scale * kLog2e;
    a.part = (float *)d_workspace;
    if (!d_workspace || ((uintptr_t)d_workspace & 255) != 0 || workspace_bytes < attention_workspace_bytes(cache->hd, sms)) return PF_EWORKSPACE;
    cudaStream_t st = (cudaStream_t)stream;
    if (dtype == PF_DT_BF16) return cache->hd == 64 ? attention_launch<Bf16, 64>(a, device, sms, st) : attention_launch<Bf16, 128>(a, device, sms, st);
    return cache->hd == 64 ? attention_launch<F16, 64>(a, device, sms, st) : attention_launch<F16, 128>(a, device, sms, st);
}
