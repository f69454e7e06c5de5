// pf_kvcache.cu -- new keys and values into the 8-bit paged cache.
//
//   s = max(old s if the page holds earlier tokens, least 2^e >= max|x| / 448),  bytes = e4m3(x / s)
//
// A unit of work is one page of one head of one sequence, keys or values: its new tokens' maximum has to be known before
// the first byte is written.  Powers of two make the scale change exact: bytes already in the page are multiplied by
// 2^-n, which loses nothing but what underflows e4m3, so the cache does not depend on how a sequence was cut into calls
// beyond that.  A unit is worked on by R rows of HD / 8 lanes, a lane holding 8 neighbouring elements (one 16-byte load,
// one 8-byte store): R = 1 for single tokens (16 to 32 units a block), R = 128 / (HD / 8) for prompts (a unit a block).  The values are
// read twice, the second time from the caches: keeping them in registers cost more blocks than it saved (27.6 us instead of 21.1 for 6 prompts of up to
// 4096 tokens, 94 MB).  256 single tokens of 32 heads of 128: 6.2 us, a chain of four reads.
#include "pf_ops.cuh"

namespace pf {

struct AppendArgs {
    pf_kv_cache_t c;
    const uint16_t *x[2];
    int64_t xs[2];
    const int32_t *cu, *len, *table;
    int n_seq, cols, max_new, units_per_seq;
    int64_t n_new;
    int64_t units;    // n_seq * units_per_seq * n_kv * 2
};

template <typename T, int HD, int R>
__global__ void __launch_bounds__(R == 1 ? 256 : 128) append_kernel(const AppendArgs A)
{
    constexpr int LANES = HD / 8;                 // lanes per token row
    constexpr int UNITS = R == 1 ? 256 / LANES : 1;
    static_assert(R == 1 || R * LANES == 128, "one unit per block of 128 threads");
    __shared__ float part[4];
    const int lane = threadIdx.x % LANES, r = R == 1 ? 0 : threadIdx.x / LANES;
    int64_t u = (int64_t)blockIdx.x * UNITS + (R == 1 ? threadIdx.x / LANES : 0);
    const bool in_range = u < A.units;
    if (!in_range) u = A.units - 1;               // whole warps stay for the shuffles; nothing is written
    const int which = (int)(u & 1);
    u >>= 1;
    const int h = (int)(u % A.c.n_kv);
    u /= A.c.n_kv;
    const int j = (int)(u % A.units_per_seq), b = (int)(u / A.units_per_seq);
    const int P = A.c.page;
    // tokens [t0, t1) of the call go to slots [s0, ..) of the page
    const int64_t cu0 = A.cu[b];
    int64_t n = min((int64_t)A.cu[b + 1], A.n_new) - cu0;          // tokens outside the call's rows are not written
    n = cu0 < 0 ? 0 : max((int64_t)0, min((int64_t)A.max_new, n));
    const int64_t start = max(0, A.len[b]);
    const int64_t col = start / P + j;
    const int64_t lo = max(start, col * P), hi = min(start + n, (col + 1) * P);   // positions
    int page = -1;
    if (in_range && lo < hi && col < A.cols) page = A.table[(int64_t)b * A.cols + col];
    const int64_t t0 = cu0 + (lo - start);
    int cnt = (int)(hi - lo);
    const int s0 = (int)(lo - col * P);
    if (page < 0 || page >= A.c.n_pages) cnt = 0;
    const uint16_t *x = A.x[which] + t0 * A.xs[which] + h * HD + lane * 8;
    const int64_t xs = A.xs[which];
    float m = 0.f;
    for (int t = r; t < cnt; t += R) {
        const uint4 v = *reinterpret_cast<const uint4 *>(x + t * xs);
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const float2 f = pair_to_f32<T>(w[i]);
            m = fmaxf(m, fmaxf(fabsf(f.x), fabsf(f.y)));
        }
    }
#pragma unroll
    for (int o = (R == 1 ? LANES : 32) / 2; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, o));
    if (R > 1) {
        if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = m;
        __syncthreads();
        m = fmaxf(fmaxf(part[0], part[1]), fmaxf(part[2], part[3]));
    }
    if (cnt <= 0) return;
    const int64_t ph = (int64_t)page * A.c.n_kv + h;
    float *scale = (which ? A.c.d_v_scale : A.c.d_k_scale) + ph;
    uint8_t *bytes = (which ? A.c.d_v : A.c.d_k) + ph * P * HD + lane * 8;
    const float fresh = pow2f(scale_exponent(m));
    float s = fresh;
    if (s0 > 0) {
        const float old = *scale;
        s = fmaxf(old, fresh);
        if (s > old) {
            const float f = old / s;
            for (int t = r; t < s0; t += R) {
                uint2 *p = reinterpret_cast<uint2 *>(bytes + t * HD);
                const uint2 v = *p;
                uint32_t o[2];
                const uint32_t in[2] = {v.x, v.y};
#pragma unroll
                for (int i = 0; i < 2; i++) {
                    const float2 a = f32x2_of_f16x2(f16x2_of_e4m3x2(in[i])), c = f32x2_of_f16x2(f16x2_of_e4m3x2(in[i] >> 16));
                    o[i] = e4m3x4(a.x * f, a.y * f, c.x * f, c.y * f);
                }
                *p = make_uint2(o[0], o[1]);
            }
        }
    }
    if (R > 1) __syncthreads();                   // every thread has read the old scale
    else __syncwarp((0xFFFFFFFFu >> (32 - LANES)) << ((threadIdx.x & 31) / LANES * LANES));
    if (lane == 0 && r == 0) *scale = s;
    const float inv = 1.f / s;                    // exact: powers of two (an older scale of any other value is rounded once)
    for (int t = r; t < cnt; t += R) {
        const uint4 v = *reinterpret_cast<const uint4 *>(x + t * xs);
        const float2 a = pair_to_f32<T>(v.x), c = pair_to_f32<T>(v.y), d = pair_to_f32<T>(v.z), e = pair_to_f32<T>(v.w);
        *reinterpret_cast<uint2 *>(bytes + (s0 + t) * HD) =
            make_uint2(e4m3x4(a.x * inv, a.y * inv, c.x * inv, c.y * inv), e4m3x4(d.x * inv, d.y * inv, e.x * inv, e.y * inv));
    }
}

template <typename T, int HD>
static void append_launch(const AppendArgs &a, cudaStream_t st)
{
    // One unit per HD / 8 lanes for calls of a few tokens a sequence, one per block otherwise: with one token a block of 128 threads would leave
    // all but 16 idle, and with many a row of lanes would read a page's tokens one after another.
    if (a.max_new <= 4) {
        constexpr int UNITS = 256 / (HD / 8);
        append_kernel<T, HD, 1><<<(unsigned)((a.units + UNITS - 1) / UNITS), 256, 0, st>>>(a);
    } else {
        append_kernel<T, HD, 128 / (HD / 8)><<<(unsigned)a.units, 128, 0, st>>>(a);
    }
}

}  // namespace pf

using namespace pf;

extern "C" int pf_kv_append(const pf_kv_cache_t *cache, int32_t dtype, int32_t n_seq, int64_t n_new, int32_t max_new, const void *d_k,
                            int64_t k_stride, const void *d_v, int64_t v_stride, const int32_t *d_cu_new, const int32_t *d_len,
                            const int32_t *d_table, int32_t table_cols, void *stream)
{
    if (!kv_cache_ok(cache) || (dtype != PF_DT_BF16 && dtype != PF_DT_F16)) return PF_EINVAL;
    if (n_seq < 0 || n_new < 0 || n_new >= (1ll << 31) || max_new < 0 || table_cols < 0) return PF_ERANGE;
    if (n_seq == 0 || n_new == 0 || max_new == 0 || table_cols == 0) return PF_OK;
    if (!d_k || !d_v || !d_cu_new || !d_len || !d_table || !aligned16(d_k) || !aligned16(d_v)) return PF_EINVAL;
    if ((uintptr_t)d_cu_new % 4 || (uintptr_t)d_len % 4 || (uintptr_t)d_table % 4) return PF_EINVAL;
    const int64_t row = (int64_t)cache->n_kv * cache->hd;
    if (k_stride < row || v_stride < row || k_stride % 8 || v_stride % 8) return PF_EINVAL;
    AppendArgs a;
    a.c = *cache;
    a.x[0] = (const uint16_t *)d_k; a.x[1] = (const uint16_t *)d_v;
    a.xs[0] = k_stride; a.xs[1] = v_stride;
    a.cu = d_cu_new; a.len = d_len; a.table = d_table;
    a.n_seq = n_seq; a.cols = table_cols;
    a.max_new = (int32_t)(max_new < n_new ? max_new : n_new);
    a.n_new = n_new;
    // the most pages that max_new tokens behind any start can touch
    a.units_per_seq = (int)(((int64_t)cache->page - 1 + a.max_new + cache->page - 1) / cache->page);
    if (a.units_per_seq > table_cols) a.units_per_seq = table_cols;
    a.units = (int64_t)n_seq * a.units_per_seq * cache->n_kv * 2;
    if (a.units >= (1ll << 31)) return PF_ERANGE;
    cudaStream_t st = (cudaStream_t)stream;
    if (dtype == PF_DT_BF16) cache->hd == 64 ? append_launch<Bf16, 64>(a, st) : append_launch<Bf16, 128>(a, st);
    else cache->hd == 64 ? append_launch<F16, 64>(a, st) : append_launch<F16, 128>(a, st);
    PF_CUDA_TRY(cudaGetLastError(), "append_kernel launch");
    count_launch();
    return PF_OK;
}
