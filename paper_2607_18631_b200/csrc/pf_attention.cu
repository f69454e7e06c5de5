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
#include "pf_attention.cuh"

namespace pf {

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
