// pf_norm.cu -- residual addition, root-mean-square norm and 8-bit output in one pass.
//
//   a = x + r,  y = a * rsqrt(mean(a^2) + eps) * w,  s_g = max_g |y| / 448,  q = e4m3(y / s_g)
//
// A block works on a row at a time: the row is read once and stays in registers (fp32) between the sum of squares, the maxima and
// the stores, so the traffic is what the outputs need and nothing else: the kernel is bound by HBM for many rows and by the
// chain load -> reduce -> store for few.  A thread owns runs of 8 neighbouring elements (16-byte loads of 16-bit types,
// 8-byte stores of q); 16 lanes own one 128-element scale group, so its maximum takes four shuffles and no barrier.  With many
// rows a block goes through several and has the next one's loads in flight while it reduces and stores.
// 8192 rows of 7168, bf16, residual, all outputs (530 MB): 92 us, 0.88 of the copy rate, with one block of 1024 threads an SM and a run a thread;
// (before the divisions were replaced by products: 96; 110 with two blocks of 512 and two runs, 119 with a row a block of 256:
// more rows under way at once mix reads and writes worse).  The schedulers issue in 64 % of the cycles.
#include <math.h>

#include "pf_ops.cuh"

namespace pf {

struct NormArgs {
    const void *x, *res, *w;
    void *sum, *y;
    uint8_t *q;
    float *scale;
    int64_t xs, rs, ss, ys;   // row strides, elements
    int64_t rows;
    int H, groups;            // groups: scales per row
    float eps, inv_H;
};

// 8 elements as they lie in memory
template <typename T> struct Raw8 { uint4 w[sizeof(T) / 2]; };
template <typename T>
__device__ __forceinline__ void fetch(const T *p, Raw8<T> &r)      // read once: not to be kept in caches
{
#pragma unroll
    for (int i = 0; i < (int)(sizeof(T) / 2); i++) r.w[i] = __ldcs(reinterpret_cast<const uint4 *>(p) + i);
}
template <typename T>
__device__ __forceinline__ void widen(const Raw8<T> &r, float (&v)[8])
{
    const uint32_t w[4] = {r.w[0].x, r.w[0].y, r.w[0].z, r.w[0].w};
#pragma unroll
    for (int i = 0; i < 4; i++) {
        const float2 f = pair_to_f32<T>(w[i]);
        v[2 * i] = f.x;
        v[2 * i + 1] = f.y;
    }
}
template <>
__device__ __forceinline__ void widen<float>(const Raw8<float> &r, float (&v)[8])
{
    v[0] = __uint_as_float(r.w[0].x); v[1] = __uint_as_float(r.w[0].y); v[2] = __uint_as_float(r.w[0].z); v[3] = __uint_as_float(r.w[0].w);
    v[4] = __uint_as_float(r.w[1].x); v[5] = __uint_as_float(r.w[1].y); v[6] = __uint_as_float(r.w[1].z); v[7] = __uint_as_float(r.w[1].w);
}
template <typename T> __device__ __forceinline__ float one(const T *p) { return pair_to_f32<T>((uint32_t)p->bits).x; }
template <> __device__ __forceinline__ float one<float>(const float *p) { return *p; }
template <typename T, bool ALIGNED>
__device__ __forceinline__ void load8(const T *p, int n, float (&v)[8])
{
    if (ALIGNED) {
        Raw8<T> r;
#pragma unroll
        for (int i = 0; i < (int)(sizeof(T) / 2); i++) r.w[i] = __ldg(reinterpret_cast<const uint4 *>(p) + i);
        widen<T>(r, v);
    } else {
#pragma unroll
        for (int i = 0; i < 8; i++) v[i] = i < n ? one<T>(p + i) : 0.f;
    }
}
template <typename T, bool ALIGNED>
__device__ __forceinline__ void store8(T *p, int n, const float (&v)[8])
{
    if (ALIGNED) {
        *reinterpret_cast<uint4 *>(p) = make_uint4(pair_of_f32<T>(v[0], v[1]), pair_of_f32<T>(v[2], v[3]),
                                                   pair_of_f32<T>(v[4], v[5]), pair_of_f32<T>(v[6], v[7]));
    } else {
#pragma unroll
        for (int i = 0; i < 8; i++)
            if (i < n) p[i].bits = (uint16_t)pair_of_f32<T>(v[i], 0.f);
    }
}
template <>
__device__ __forceinline__ void store8<float, true>(float *p, int, const float (&v)[8])
{
    reinterpret_cast<float4 *>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
    reinterpret_cast<float4 *>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
}
template <>
__device__ __forceinline__ void store8<float, false>(float *p, int n, const float (&v)[8])
{
#pragma unroll
    for (int i = 0; i < 8; i++)
        if (i < n) p[i] = v[i];
}

template <bool MAX>
__device__ __forceinline__ float warp_all(float v)
{
#pragma unroll
    for (int m = 16; m; m >>= 1) {
        const float o = __shfl_xor_sync(0xFFFFFFFFu, v, m);
        v = MAX ? fmaxf(v, o) : v + o;
    }
    return v;
}
// every thread gets the block's sum / maximum; `part` holds one word per warp and is used once per call site
template <int THREADS, bool MAX>
__device__ __forceinline__ float block_all(float v, float *part)
{
    v = warp_all<MAX>(v);
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = v;
    __syncthreads();
    const int lane = threadIdx.x & 31;
    return warp_all<MAX>(lane < THREADS / 32 ? part[lane] : 0.f);
}

// MIN_BLOCKS: blocks of an SM that the registers have to leave room for
template <typename T, int THREADS, int NV, bool ALIGNED, int MIN_BLOCKS>
__global__ void __launch_bounds__(THREADS, MIN_BLOCKS) norm_kernel(const NormArgs A)
{
    __shared__ float parts[2][2][32];      // by row parity: a row's barrier lies between two uses of the same words
    Raw8<T> nx[NV], nr[NV];                // the next row
    auto fetch_row = [&](int64_t row) {
#pragma unroll
        for (int i = 0; i < NV; i++) {
            const int e = 8 * (threadIdx.x + i * THREADS);
            if (e >= A.H) continue;
            fetch<T>((const T *)A.x + row * A.xs + e, nx[i]);
            if (A.res) fetch<T>((const T *)A.res + row * A.rs + e, nr[i]);
        }
    };
    if (ALIGNED) fetch_row(blockIdx.x);
    int turn = 0;
    for (int64_t row = blockIdx.x; row < A.rows; row += gridDim.x, turn ^= 1) {
        float (&part)[2][32] = parts[turn];
        float a[NV][8];
        float ss = 0.f;
#pragma unroll
        for (int i = 0; i < NV; i++) {
            const int e = 8 * (threadIdx.x + i * THREADS), n = A.H - e;
#pragma unroll
            for (int j = 0; j < 8; j++) a[i][j] = 0.f;
            if (n <= 0) continue;
            float r[8];
            if (ALIGNED) widen<T>(nx[i], a[i]);
            else load8<T, false>((const T *)A.x + row * A.xs + e, n, a[i]);
            if (!A.res) continue;
            if (ALIGNED) widen<T>(nr[i], r);
            else load8<T, false>((const T *)A.res + row * A.rs + e, n, r);
#pragma unroll
            for (int j = 0; j < 8; j++) a[i][j] += r[j];
        }
        if (ALIGNED && row + gridDim.x < A.rows) fetch_row(row + gridDim.x);
#pragma unroll
        for (int i = 0; i < NV; i++) {
            const int e = 8 * (threadIdx.x + i * THREADS), n = A.H - e;
            if (A.sum && n > 0) store8<T, ALIGNED>((T *)A.sum + row * A.ss + e, n, a[i]);
#pragma unroll
            for (int j = 0; j < 8; j++) ss = fmaf(a[i][j], a[i][j], ss);
        }
        const float rstd = rsqrtf(block_all<THREADS, false>(ss, part[0]) * A.inv_H + A.eps);
        float row_max = 0.f;
#pragma unroll
        for (int i = 0; i < NV; i++) {
            const int e = 8 * (threadIdx.x + i * THREADS), n = A.H - e;
            float w[8];
            if (A.w && n > 0) load8<T, ALIGNED>((const T *)A.w + e, n, w);
#pragma unroll
            for (int j = 0; j < 8; j++) {
                a[i][j] *= rstd;
                if (A.w && n > 0) a[i][j] *= w[j];
            }
            if (A.y && n > 0) store8<T, ALIGNED>((T *)A.y + row * A.ys + e, n, a[i]);
            if (!A.q) continue;
            float m = 0.f;
#pragma unroll
            for (int j = 0; j < 8; j++)
                if (j < n) m = fmaxf(m, fabsf(a[i][j]));
            if (A.groups == 1) {
                row_max = fmaxf(row_max, m);
                continue;
            }
#pragma unroll
            for (int o = 8; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, o));
            if (n <= 0) continue;
            const float s = m > 0.f ? fmaxf(m * (1.f / kE4m3Max), kMinScale) : 1.f;
            if ((threadIdx.x & 15) == 0) A.scale[row * A.groups + e / PF_SCALE_GROUP] = s;
            const float inv = __fdividef(1.f, s);      // within 2 units: far below e4m3's
            uint8_t *q = A.q + row * A.H + e;
            const uint32_t lo = e4m3x4(a[i][0] * inv, a[i][1] * inv, a[i][2] * inv, a[i][3] * inv);
            const uint32_t hi = e4m3x4(a[i][4] * inv, a[i][5] * inv, a[i][6] * inv, a[i][7] * inv);
            if (ALIGNED) {
                *reinterpret_cast<uint2 *>(q) = make_uint2(lo, hi);
            } else {
#pragma unroll
                for (int j = 0; j < 8; j++)
                    if (j < n) q[j] = (uint8_t)((j < 4 ? lo : hi) >> (8 * (j & 3)));
            }
        }
        if (!A.q || A.groups != 1) continue;
        const float m = block_all<THREADS, true>(row_max, part[1]);
        const float s = m > 0.f ? fmaxf(m * (1.f / kE4m3Max), kMinScale) : 1.f, inv = __fdividef(1.f, s);
        if (threadIdx.x == 0) A.scale[row] = s;
#pragma unroll
        for (int i = 0; i < NV; i++) {
            const int e = 8 * (threadIdx.x + i * THREADS), n = A.H - e;
            if (n <= 0) continue;
            uint8_t *q = A.q + row * A.H + e;
            const uint32_t lo = e4m3x4(a[i][0] * inv, a[i][1] * inv, a[i][2] * inv, a[i][3] * inv);
            const uint32_t hi = e4m3x4(a[i][4] * inv, a[i][5] * inv, a[i][6] * inv, a[i][7] * inv);
            if (ALIGNED) {
                *reinterpret_cast<uint2 *>(q) = make_uint2(lo, hi);
            } else {
#pragma unroll
                for (int j = 0; j < 8; j++)
                    if (j < n) q[j] = (uint8_t)((j < 4 ? lo : hi) >> (8 * (j & 3)));
            }
        }
    }
}

template <typename T, int THREADS, int NV, bool ALIGNED, int MIN_BLOCKS>
static void norm_run(const NormArgs &a, int sms, cudaStream_t st)
{
    // rows that fit the GPU at once have a block each; of more, a block takes several
    const int64_t room = (int64_t)sms * MIN_BLOCKS;
    norm_kernel<T, THREADS, NV, ALIGNED, MIN_BLOCKS><<<(unsigned)(a.rows < room ? a.rows : room), THREADS, 0, st>>>(a);
}
template <typename T, bool ALIGNED>
static void norm_launch(const NormArgs &a, int sms, cudaStream_t st)
{
    constexpr int W = sizeof(T) == 4 ? 1 : 2;      // fp32 rows take twice the registers
    // up to a row an SM: the most threads for each (1 x 7168: 2.9 us)
    if (a.rows <= sms && a.H > 2048) {
        if (a.H <= 8192) norm_run<T, 1024, 1, ALIGNED, 1>(a, sms, st);
        else norm_run<T, 1024, 2, ALIGNED, 1>(a, sms, st);
        return;
    }
    if (a.H <= 1024) norm_run<T, 128, 1, ALIGNED, 8>(a, sms, st);
    else if (a.H <= 2048) norm_run<T, 256, 1, ALIGNED, 4>(a, sms, st);
    else if (a.H <= 4096) norm_run<T, 512, 1, ALIGNED, 2>(a, sms, st);
    // 512 threads and two runs a thread against 1024 and one, us at 148 SMs.  16-bit types (two blocks of 512 an SM): 149 x 5120 4.2, 4.7 and 200 x
    // 5120 4.5, 4.9 with a scale a row, 149 x 7168 4.5, 4.6 and 200 x 7168 4.9, 4.8 with a scale a group; 296 x 7168 5.6, 4.9; 592 x 5120
    // 8.4, 7.1; 2000 x 7168 32, 24.  fp32 (one block): 149 x 7168 6.4, 6.9; 592 x 7168 13.1, 13.6; 1184 x 7168 27.8, 24.9.
    else if (a.H <= 8192 && 2 * a.rows <= (sizeof(T) == 4 ? 8 : 3) * sms) norm_run<T, 512, 2, ALIGNED, W>(a, sms, st);
    else if (a.H <= 8192) norm_run<T, 1024, 1, ALIGNED, 1>(a, sms, st);
    else norm_run<T, 1024, 2, ALIGNED, 1>(a, sms, st);
}

}  // namespace pf

using namespace pf;

extern "C" int pf_add_rms_norm(int32_t dtype, int64_t rows, int32_t H, const void *d_x, int64_t x_stride, const void *d_residual,
                               int64_t residual_stride, const void *d_weight, float eps, int32_t group, void *d_sum,
                               int64_t sum_stride, void *d_y, int64_t y_stride, uint8_t *d_q, float *d_scale, void *stream)
{
    if (dtype != PF_DT_BF16 && dtype != PF_DT_F16 && dtype != PF_DT_F32) return PF_EINVAL;
    if (group != 0 && group != PF_SCALE_GROUP) return PF_EINVAL;
    if (!(eps >= 0.f) || isinf(eps)) return PF_EINVAL;
    if (H < 1 || H > PF_NORM_MAX_H || rows < 0 || rows >= (1ll << 31)) return PF_ERANGE;
    if (rows == 0) return PF_OK;
    if (!d_sum && !d_y && !d_q) return PF_EINVAL;
    if (d_q && !d_scale) return PF_EINVAL;
    if (x_stride < H || (d_residual && residual_stride < H) || (d_sum && sum_stride < H) || (d_y && y_stride < H)) return PF_EINVAL;
    if (!d_x) return PF_EINVAL;
    const int esize = dtype == PF_DT_F32 ? 4 : 2;
    if ((uintptr_t)d_x % esize || (uintptr_t)d_residual % esize || (uintptr_t)d_weight % esize || (uintptr_t)d_sum % esize ||
        (uintptr_t)d_y % esize || (uintptr_t)d_scale % 4)
        return PF_EINVAL;
    const int per16 = 16 / esize;
    const bool aligned = H % 8 == 0 && aligned16(d_x) && x_stride % per16 == 0 && aligned16(d_weight) &&
                         (!d_residual || (aligned16(d_residual) && residual_stride % per16 == 0)) &&
                         (!d_sum || (aligned16(d_sum) && sum_stride % per16 == 0)) &&
                         (!d_y || (aligned16(d_y) && y_stride % per16 == 0)) && (uintptr_t)d_q % 8 == 0;
    int device, sms;
    if (int rc = current_sm_count(&device, &sms)) return rc;
    NormArgs a;
    a.x = d_x; a.res = d_residual; a.w = d_weight; a.sum = d_sum; a.y = d_y; a.q = d_q; a.scale = d_scale;
    a.xs = x_stride; a.rs = residual_stride; a.ss = sum_stride; a.ys = y_stride;
    a.rows = rows; a.H = H; a.groups = group ? (H + group - 1) / group : 1; a.eps = eps; a.inv_H = 1.f / (float)H;
    cudaStream_t st = (cudaStream_t)stream;
    // a row of at most one group takes the row path: one scale either way
    if (dtype == PF_DT_BF16) aligned ? norm_launch<Bf16, true>(a, sms, st) : norm_launch<Bf16, false>(a, sms, st);
    else if (dtype == PF_DT_F16) aligned ? norm_launch<F16, true>(a, sms, st) : norm_launch<F16, false>(a, sms, st);
    else aligned ? norm_launch<float, true>(a, sms, st) : norm_launch<float, false>(a, sms, st);
    PF_CUDA_TRY(cudaGetLastError(), "norm_kernel launch");
    count_launch();
    return PF_OK;
}
