// pf_rope.cu -- rotary positions: heads rotated by themselves, and on their way into the 8-bit paged cache.
//
//   pair i of a head at position p turns by theta = p f_i:  (a, b) -> m (a cos - b sin, b cos + a sin)
//
// Angles.  f_i is held as a fraction of a turn in 64 bits, F_i = f_i / (2 pi) * 2^64, so that the angle modulo a turn is the product
// p F_i modulo 2^64: two 32-bit multiplications, exact for every 32-bit position, where a product of 32-bit floats would be off by
// p 2^-24 radians (0.06 at 2^20).  Its upper 32 bits, signed, are half turns in [-1, 1).
#include <math.h>

#include "pf_ops.cuh"

namespace pf {

struct Rot {
    const uint64_t *phase;
    int rot;                  // rotated elements of a head
    float amp, flip;          // m, and -1 where the transposed rotation is asked for
};

// Cosine and sine of a pair's angle, each within 2^-23 of its own size, so that an element next to a zero of its sine or cosine is as exact as the others.  The angle is taken apart into
// quarter turns and the rest, an integer of 30 bits between -1/8 and 1/8 of a turn.  Of the rest u (in eighths) the sine is u S(u^2), the cosine C(u^2), of the least degrees whose
// nearest polynomials (by exchange, relative) are off by less than 2^-28; the sine's first coefficient, pi / 4, is two numbers.  8192 tokens of 40 heads of 128: 31.5 us, with the
// special-function unit 30.9, which is off by up to 2^-21.4 of the pair's length whatever the element's size.
// FAST, for results in 8 bits: the unit's.  At the page's scale e4m3's least half step is 2^-18.8 of the largest element, and an element is off by 2^-20.4 of it at most.
template <bool FAST>
__device__ __forceinline__ void turn_of(const Rot &r, int pair, int32_t pos, float &c, float &s)
{
    const uint64_t f = __ldg(r.phase + pair);
    const int32_t t = (int32_t)(uint32_t)(((uint64_t)(int64_t)pos * f) >> 32);
    if (FAST) {
        const float x = (float)t * 1.4629180792671596e-9f;              // pi 2^-31
        c = __cosf(x);
        s = __sinf(x);
    } else {
        const uint32_t quarter = ((uint32_t)t + 0x20000000u) >> 30;
        const float u = (float)(int32_t)((uint32_t)t - (quarter << 30)) * 1.862645149230957e-9f, v = u * u;      // 2^-29
        const float sine = fmaf(u, 0.7853981852531433f, u * fmaf(fmaf(fmaf(-3.59504520019982e-5f, v, 2.49000103212893e-3f), v, -0.08074543625116348f), v, -2.1855694e-8f));
        const float cosine = fmaf(fmaf(fmaf(fmaf(3.52876168108196e-6f, v, -3.259365039411932e-4f), v, 0.015854323282837868f), v, -0.3084251284599304f), v, 1.f);
        const bool swap = quarter & 1;
        c = __uint_as_float(__float_as_uint(swap ? sine : cosine) ^ ((quarter + 1) & 2) << 30);
        s = __uint_as_float(__float_as_uint(swap ? cosine : sine) ^ (quarter & 2) << 30);
    }
    c *= r.amp;
    s *= r.amp * r.flip;
}

// A thread's 16 elements of a head are two runs of 8, and the runs of neighbouring threads are neighbours: where a head's halves turn with one another, the
// runs that do so; where neighbours do, a run of either half of the head.
template <bool HALF>
struct Runs {
    int a, b;                 // where they begin
    bool turns_a, turns_b;
    __device__ __forceinline__ Runs(int chunk, int rot, int hd)
    {
        if (!HALF || rot == 0) {
            a = 8 * chunk;
            b = hd / 2 + 8 * chunk;
            turns_a = a < rot;
            turns_b = b < rot;
        } else {
            const int k = chunk - rot / 16;
            turns_a = turns_b = k < 0;
            a = turns_a ? 8 * chunk : rot + 8 * k;
            b = turns_a ? rot / 2 + 8 * chunk : rot + (hd - rot) / 2 + 8 * k;
        }
    }
    template <bool FAST>
    __device__ __forceinline__ void angles(const Rot &r, int32_t pos, float (&c)[8], float (&s)[8]) const
    {
#pragma unroll
        for (int j = 0; j < 8; j++) {
            if (HALF) {
                if (turns_a) turn_of<FAST>(r, a + j, pos, c[j], s[j]);
            } else if (j < 4 ? turns_a : turns_b) {
                turn_of<FAST>(r, (j < 4 ? a : b) / 2 + (j & 3), pos, c[j], s[j]);
            }
        }
    }
    __device__ __forceinline__ void turn(float (&x)[8], float (&y)[8], const float (&c)[8], const float (&s)[8]) const
    {
        if (HALF) {
            if (!turns_a) return;
#pragma unroll
            for (int j = 0; j < 8; j++) {
                const float u = x[j], v = y[j];
                x[j] = fmaf(u, c[j], -v * s[j]);
                y[j] = fmaf(v, c[j], u * s[j]);
            }
        }
#pragma unroll
        for (int j = 0; j < 8 && !HALF; j++) {
            if (!(j < 4 ? turns_a : turns_b)) continue;
            float &u = j < 4 ? x[2 * (j & 3)] : y[2 * (j & 3)], &v = j < 4 ? x[2 * (j & 3) + 1] : y[2 * (j & 3) + 1];
            const float p = u, q = v;
            u = fmaf(p, c[j], -q * s[j]);
            v = fmaf(q, c[j], p * s[j]);
        }
    }
};

// 8 neighbouring elements as they lie in memory, read and written once: not to be kept in caches
template <typename T> struct Run8 {
    uint4 w;
    __device__ __forceinline__ void load(const T *p) { w = __ldcs(reinterpret_cast<const uint4 *>(p)); }
    __device__ __forceinline__ void get(float (&v)[8]) const
    {
        const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const float2 f = pair_to_f32<T>(u[i]);
            v[2 * i] = f.x;
            v[2 * i + 1] = f.y;
        }
    }
};
template <> struct Run8<float> {
    float4 a, b;
    __device__ __forceinline__ void load(const float *p) { a = __ldcs(reinterpret_cast<const float4 *>(p)); b = __ldcs(reinterpret_cast<const float4 *>(p) + 1); }
    __device__ __forceinline__ void get(float (&v)[8]) const
    {
        v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
        v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
    }
};
template <typename T> __device__ __forceinline__ void get8(const T *p, float (&v)[8])      // to be read again
{
    Run8<T> r;
    r.w = *reinterpret_cast<const uint4 *>(p);
    r.get(v);
}
template <typename T> __device__ __forceinline__ void put8(T *p, const float (&v)[8])
{
    __stcs(reinterpret_cast<uint4 *>(p),
        make_uint4(pair_of_f32<T>(v[0], v[1]), pair_of_f32<T>(v[2], v[3]), pair_of_f32<T>(v[4], v[5]), pair_of_f32<T>(v[6], v[7])));
}
template <> __device__ __forceinline__ void put8<float>(float *p, const float (&v)[8])
{
    reinterpret_cast<float4 *>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
    reinterpret_cast<float4 *>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
}
template <typename T> __device__ __forceinline__ float get1(const T *p) { return pair_to_f32<T>((uint32_t)p->bits).x; }
template <> __device__ __forceinline__ float get1<float>(const float *p) { return *p; }
template <typename T> __device__ __forceinline__ void put1(T *p, float v) { p->bits = (uint16_t)pair_of_f32<T>(v, 0.f); }
template <> __device__ __forceinline__ void put1<float>(float *p, float v) { *p = v; }

// ------------------------------------------------------------------ heads by themselves
struct RopeArgs {
    Rot r;
    const void *x;
    void *y;
    int64_t xt, xh, yt, yh;   // strides of a token and of a head, elements
    const int32_t *pos;
    int64_t units;            // threads with work
    int heads, hd, per, groups;   // heads a thread takes, and groups of so many
};

// 16 elements of each of `n` heads of one token, B heads at a time
template <typename T, bool HALF, int B>
__device__ __forceinline__ void rope_heads(const Rot &r, int32_t pos, int hd, int chunk, const T *x, int64_t xh, T *y, int64_t yh, int n)
{
    const Runs<HALF> run(chunk, r.rot, hd);
    float c[8], s[8];
    run.template angles<false>(r, pos, c, s);
    // x and y may be one tensor, so the loads of a few heads are asked for before the first store
    for (int h = 0; h < n; h += B) {
        Run8<T> in[B][2];
#pragma unroll
        for (int i = 0; i < B; i++)
            if (h + i < n) {
                in[i][0].load(x + (h + i) * xh + run.a);
                in[i][1].load(x + (h + i) * xh + run.b);
            }
#pragma unroll
        for (int i = 0; i < B; i++)
            if (h + i < n) {
                float a[8], b[8];
                in[i][0].get(a);
                in[i][1].get(b);
                run.turn(a, b, c, s);
                put8<T>(y + (h + i) * yh + run.a, a);
                put8<T>(y + (h + i) * yh + run.b, b);
            }
    }
}

template <typename T, bool HALF>
__global__ void __launch_bounds__(256) rope_kernel(const RopeArgs A)
{
    int64_t u = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (u >= A.units) return;
    const int chunks = A.hd / 16;
    const int chunk = (int)(u % chunks);
    u /= chunks;
    const int first = (int)(u % A.groups) * A.per;
    const int64_t t = u / A.groups;
    // (8192 tokens of 40 heads: four heads' loads under way, with two 7 us more; in 32 bits 61 us)
    rope_heads<T, HALF, sizeof(T) == 4 ? 2 : 4>(A.r, A.pos[t], A.hd, chunk, (const T *)A.x + t * A.xt + first * A.xh, A.xh, (T *)A.y + t * A.yt + first * A.yh, A.yh,
                        min(A.per, A.heads - first));
}

// any size, alignment and even `rot`: a thread takes a pair, or one element that stays.  Bound by what a thread does for its few bytes (two 64-bit divisions, an angle, a sine and a cosine a
// pair and head): 8192 tokens of 40 heads of 80, 40 of them turned, 110 us for 105 MB; heads of 128 that begin 2 bytes past a boundary 123 us, where the kernel above takes 31.
template <typename T, bool HALF>
__global__ void __launch_bounds__(256) rope_any_kernel(const RopeArgs A)
{
    int64_t u = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (u >= A.units) return;
    const int pairs = A.r.rot / 2, items = A.hd - pairs;
    const int i = (int)(u % items);
    u /= items;
    const int h = (int)(u % A.heads);
    const int64_t t = u / A.heads;
    const T *x = (const T *)A.x + t * A.xt + h * A.xh;
    T *y = (T *)A.y + t * A.yt + h * A.yh;
    if (i >= pairs) {
        y[i + pairs] = x[i + pairs];
        return;
    }
    float c, s;
    turn_of<false>(A.r, i, A.pos[t], c, s);
    const int a = HALF ? i : 2 * i, b = HALF ? i + pairs : 2 * i + 1;
    const float p = get1<T>(x + a), q = get1<T>(x + b);
    put1<T>(y + a, fmaf(p, c, -q * s));
    put1<T>(y + b, fmaf(q, c, p * s));
}

template <typename T>
static void rope_launch(const RopeArgs &a, bool half, bool wide, cudaStream_t st)
{
    const unsigned grid = (unsigned)((a.units + 255) / 256);
    if (wide) half ? rope_kernel<T, true><<<grid, 256, 0, st>>>(a) : rope_kernel<T, false><<<grid, 256, 0, st>>>(a);
    else half ? rope_any_kernel<T, true><<<grid, 256, 0, st>>>(a) : rope_any_kernel<T, false><<<grid, 256, 0, st>>>(a);
}

// ------------------------------------------------------------------ into the cache
// A unit of work is a page of one head of one sequence, keys or values, as in the append without rotation: the largest element of what is
// written there has to be known before the first byte.  Keys are rotated in 32 bits and rounded once, to e4m3; they are rotated twice, once for the
// maximum and once for the bytes.  A unit is worked on by R rows of HD / 16 lanes.  Queries are rotated by the blocks behind the units'.
struct AppendRopeArgs {
    pf_kv_cache_t c;
    Rot r;
    const void *q, *k, *v;
    void *qo;
    int64_t qs, qos, ks, vs;
    const int32_t *cu, *len, *table, *pos;
    int n_seq, cols, max_new, units_per_seq, n_heads, per, groups;
    int64_t n_new, units, unit_blocks, q_units;
};

// tokens of sequence b in this call
__device__ __forceinline__ int64_t new_tokens(const AppendRopeArgs &A, int b, int64_t &cu0)
{
    cu0 = A.cu[b];
    const int64_t n = min((int64_t)A.cu[b + 1], A.n_new) - cu0;    // tokens outside the call's rows are not there
    return cu0 < 0 ? 0 : max((int64_t)0, min((int64_t)A.max_new, n));
}

template <typename T, int HD, bool HALF>
__device__ __forceinline__ void append_query(const AppendRopeArgs &A, int64_t u)
{
    if (u >= A.q_units) return;
    constexpr int CHUNKS = HD / 16;
    const int chunk = (int)(u % CHUNKS);
    u /= CHUNKS;
    const int first = (int)(u % A.groups) * A.per;
    int64_t t = u / A.groups, cu0;
    int b;
    if (A.max_new <= 4) {                     // a few tokens each: by sequence
        b = (int)(t / A.max_new);
        const int64_t j = t - (int64_t)b * A.max_new;
        if (j >= new_tokens(A, b, cu0)) return;
        t = cu0 + j;
    } else {                                  // by row: the last sequence that begins at or before it
        int lo = 0, hi = A.n_seq;
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (A.cu[mid] <= t) lo = mid; else hi = mid;
        }
        b = lo;
        const int64_t n = new_tokens(A, b, cu0);
        if (t < cu0 || t >= cu0 + n) return;
    }
    const int32_t pos = A.pos ? A.pos[t] : (int32_t)((int64_t)max(0, A.len[b]) + (t - cu0));
    // two heads at a time: the registers of four would leave the units' blocks fewer places (six prompts of up to 4096 tokens: 70 us instead of 76)
    rope_heads<T, HALF, 2>(A.r, pos, HD, chunk, (const T *)A.q + t * A.qs + first * HD, HD, (T *)A.qo + t * A.qos + first * HD, HD, min(A.per, A.n_heads - first));
}

template <typename T, int HD, int R, bool HALF>
__global__ void __launch_bounds__(R == 1 ? 256 : 128) append_rope_kernel(const AppendRopeArgs A)
{
    constexpr int LANES = HD / 16;                // lanes per token row
    constexpr int THREADS = R == 1 ? 256 : 128;
    constexpr int UNITS = R == 1 ? THREADS / LANES : 1;
    static_assert(R == 1 || R * LANES == THREADS, "one unit per block");
    __shared__ float part[4];
    if ((int64_t)blockIdx.x >= A.unit_blocks) {
        append_query<T, HD, HALF>(A, ((int64_t)blockIdx.x - A.unit_blocks) * THREADS + threadIdx.x);
        return;
    }
    const int lane = threadIdx.x % LANES, r = R == 1 ? 0 : threadIdx.x / LANES;
    int64_t u = (int64_t)blockIdx.x * UNITS + (R == 1 ? threadIdx.x / LANES : 0);
    const bool in_range = u < A.units;
    if (!in_range) u = A.units - 1;               // whole warps stay for the shuffles; nothing is written
    const int which = (int)(u & 1);               // 0: keys
    u >>= 1;
    const int h = (int)(u % A.c.n_kv);
    u /= A.c.n_kv;
    const int j = (int)(u % A.units_per_seq), b = (int)(u / A.units_per_seq);
    const int P = A.c.page;
    // tokens [t0, t0 + cnt) of the call go to slots [s0, ..) of the page
    int64_t cu0;
    const int64_t n = new_tokens(A, b, cu0);
    const int64_t start = max(0, A.len[b]);
    const int64_t col = start / P + j;
    const int64_t lo = max(start, col * P), hi = min(start + n, (col + 1) * P);   // places in the sequence
    int page = -1;
    if (in_range && lo < hi && col < A.cols) page = A.table[(int64_t)b * A.cols + col];
    const int64_t t0 = cu0 + (lo - start);
    int cnt = (int)(hi - lo);
    const int s0 = (int)(lo - col * P);
    if (page < 0 || page >= A.c.n_pages) cnt = 0;
    const int64_t xs = which ? A.vs : A.ks;
    const T *x = (const T *)(which ? A.v : A.k) + t0 * xs + h * HD;
    const Runs<HALF> run(lane, which ? 0 : A.r.rot, HD);
    float f[8], g[8];
    auto fetch = [&](int t) {
        get8<T>(x + t * xs + run.a, f);
        get8<T>(x + t * xs + run.b, g);
        float c[8], s[8];
        run.template angles<true>(A.r, A.pos ? A.pos[t0 + t] : (int32_t)(lo + t), c, s);
        run.turn(f, g, c, s);
    };
    float m = 0.f;
    for (int t = r; t < cnt; t += R) {
        fetch(t);
#pragma unroll
        for (int i = 0; i < 8; i++) m = fmaxf(m, fmaxf(fabsf(f[i]), fabsf(g[i])));
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
    uint8_t *bytes = (which ? A.c.d_v : A.c.d_k) + ph * P * HD;
    const float fresh = pow2f(scale_exponent(m));
    float s = fresh;
    if (s0 > 0) {
        const float old = *scale;
        s = fmaxf(old, fresh);
        if (s > old) {
            const float down = old / s;
            for (int t = r; t < s0; t += R) {
                uint4 *p = reinterpret_cast<uint4 *>(bytes + t * HD + lane * 16);
                const uint4 v = *p;
                const uint32_t in[4] = {v.x, v.y, v.z, v.w};
                uint32_t o[4];
#pragma unroll
                for (int i = 0; i < 4; i++) {
                    const float2 a = f32x2_of_f16x2(f16x2_of_e4m3x2(in[i])), c = f32x2_of_f16x2(f16x2_of_e4m3x2(in[i] >> 16));
                    o[i] = e4m3x4(a.x * down, a.y * down, c.x * down, c.y * down);
                }
                *p = make_uint4(o[0], o[1], o[2], o[3]);
            }
        }
    }
    if (R > 1) __syncthreads();                   // every thread has read the old scale
    else __syncwarp((0xFFFFFFFFu >> (32 - LANES)) << ((threadIdx.x & 31) / LANES * LANES));
    if (lane == 0 && r == 0) *scale = s;
    const float inv = 1.f / s;                    // exact: powers of two (an older scale of any other value is rounded once)
    for (int t = r; t < cnt; t += R) {
        if (cnt > R) fetch(t);                    // else the thread's one token is still here
        uint8_t *to = bytes + (s0 + t) * HD;
        *reinterpret_cast<uint2 *>(to + run.a) = make_uint2(e4m3x4(f[0] * inv, f[1] * inv, f[2] * inv, f[3] * inv), e4m3x4(f[4] * inv, f[5] * inv, f[6] * inv, f[7] * inv));
        *reinterpret_cast<uint2 *>(to + run.b) = make_uint2(e4m3x4(g[0] * inv, g[1] * inv, g[2] * inv, g[3] * inv), e4m3x4(g[4] * inv, g[5] * inv, g[6] * inv, g[7] * inv));
    }
}

template <typename T, int HD, bool HALF>
static void append_rope_launch(AppendRopeArgs a, cudaStream_t st)
{
    constexpr int LANES = HD / 16;
    // units of few tokens share a block, as in the append without rotation
    const int threads = a.max_new <= 4 ? 256 : 128;
    a.unit_blocks = a.max_new <= 4 ? (a.units + 256 / LANES - 1) / (256 / LANES) : a.units;
    const unsigned grid = (unsigned)(a.unit_blocks + (a.q_units + threads - 1) / threads);
    if (a.max_new <= 4) append_rope_kernel<T, HD, 1, HALF><<<grid, 256, 0, st>>>(a);
    else append_rope_kernel<T, HD, 128 / LANES, HALF><<<grid, 128, 0, st>>>(a);
}

// Heads a thread takes: its eight angles serve all of them, but not at the price of idle SMs (`threads`: with one head each)
static int heads_per_thread(int64_t threads, int heads)
{
    int per = 1;
    while (per < 8 && per < heads && threads / (2 * per) >= 148 * 1024) per *= 2;
    return per;
}

static bool rotary_ok(const pf_rotary_t *r, int hd)
{
    return r && r->rot >= 0 && r->rot % 2 == 0 && r->rot <= hd && (r->layout == PF_ROPE_HALF || r->layout == PF_ROPE_INTERLEAVED) &&
           isfinite(r->amplitude) && (r->rot == 0 || (r->d_phase && (uintptr_t)r->d_phase % 8 == 0));
}

}  // namespace pf

using namespace pf;

extern "C" int pf_rotary_phases(int32_t n, const double *freq, uint64_t *phase)
{
    if (n < 0) return PF_ERANGE;
    if (n > 0 && (!freq || !phase)) return PF_EINVAL;
    for (int32_t i = 0; i < n; i++) {
        if (!isfinite(freq[i])) return PF_EINVAL;
        const long double turns = (long double)freq[i] / 6.283185307179586476925286766559L;
        const long double whole = 18446744073709551616.0L, part = roundl((turns - floorl(turns)) * whole);
        phase[i] = part < whole ? (uint64_t)part : 0;      // (a fraction that is rounded up to a turn: a tiny negative frequency)
    }
    return PF_OK;
}

extern "C" int pf_rope(const pf_rotary_t *rotary, int32_t transposed, int32_t dtype, int64_t tokens, int32_t heads, int32_t hd, const void *d_x,
                       int64_t x_token, int64_t x_head, const int32_t *d_pos, void *d_y, int64_t y_token, int64_t y_head, void *stream)
{
    if (dtype != PF_DT_BF16 && dtype != PF_DT_F16 && dtype != PF_DT_F32) return PF_EINVAL;
    if (tokens < 0 || tokens >= (1ll << 31) || heads < 0 || heads > PF_ROPE_MAX_HEADS || hd < 1 || hd > PF_ROPE_MAX_HD) return PF_ERANGE;
    if (!rotary_ok(rotary, hd)) return PF_EINVAL;
    if (tokens == 0 || heads == 0) return PF_OK;
    const int esize = dtype == PF_DT_F32 ? 4 : 2;
    if (!d_x || !d_y || !d_pos || (uintptr_t)d_x % esize || (uintptr_t)d_y % esize || (uintptr_t)d_pos % 4) return PF_EINVAL;
    // rows of heads that lie one behind the other, tokens inside heads or heads inside tokens
    auto apart = [&](int64_t t, int64_t h) { return (heads == 1 || h >= hd) && (tokens == 1 || t >= hd) &&
                                                    (heads == 1 || tokens == 1 || t >= (int64_t)heads * h || h >= tokens * t); };
    if (!apart(x_token, x_head) || !apart(y_token, y_head)) return PF_EINVAL;
    RopeArgs a;
    a.r = Rot{rotary->d_phase, rotary->rot, rotary->amplitude, transposed ? -1.f : 1.f};
    a.x = d_x; a.y = d_y; a.xt = x_token; a.xh = x_head; a.yt = y_token; a.yh = y_head; a.pos = d_pos;
    a.heads = heads; a.hd = hd;
    const int per16 = 16 / esize;
    const bool wide = hd % 16 == 0 && rotary->rot % 16 == 0 && aligned16(d_x) && aligned16(d_y) && x_token % per16 == 0 && x_head % per16 == 0 &&
                      y_token % per16 == 0 && y_head % per16 == 0;
    if (wide) {
        a.per = heads_per_thread(tokens * heads * (hd / 16), heads);
        a.groups = (heads + a.per - 1) / a.per;
        a.units = tokens * a.groups * (hd / 16);
    } else {
        a.per = a.groups = 1;
        a.units = tokens * heads * (hd - rotary->rot / 2);
    }
    if ((a.units + 255) / 256 >= (1ll << 31)) return PF_ERANGE;
    cudaStream_t st = (cudaStream_t)stream;
    const bool half = rotary->layout == PF_ROPE_HALF;
    if (dtype == PF_DT_BF16) rope_launch<Bf16>(a, half, wide, st);
    else if (dtype == PF_DT_F16) rope_launch<F16>(a, half, wide, st);
    else rope_launch<float>(a, half, wide, st);
    PF_CUDA_TRY(cudaGetLastError(), "rope_kernel launch");
    count_launch();
    return PF_OK;
}

extern "C" int pf_kv_append_rope(const pf_kv_cache_t *cache, const pf_rotary_t *rotary, int32_t dtype, int32_t n_seq, int64_t n_new, int32_t max_new,
                                 int32_t n_heads, const void *d_q, int64_t q_stride, void *d_q_out, int64_t q_out_stride, const void *d_k,
                                 int64_t k_stride, const void *d_v, int64_t v_stride, const int32_t *d_cu_new, const int32_t *d_len,
                                 const int32_t *d_table, int32_t table_cols, const int32_t *d_pos, void *stream)
{
    if (!kv_cache_ok(cache) || (dtype != PF_DT_BF16 && dtype != PF_DT_F16)) return PF_EINVAL;
    if (n_seq < 0 || n_new < 0 || n_new >= (1ll << 31) || max_new < 0 || table_cols < 0 || n_heads < 0 || n_heads > PF_ROPE_MAX_HEADS) return PF_ERANGE;
    if (!rotary_ok(rotary, cache->hd) || rotary->rot % 16 != 0) return PF_EINVAL;
    if (n_seq == 0 || n_new == 0 || max_new == 0) return PF_OK;
    if (!d_k || !d_v || !d_cu_new || !d_len || (!d_table && table_cols > 0) || !aligned16(d_k) || !aligned16(d_v)) return PF_EINVAL;
    if ((uintptr_t)d_cu_new % 4 || (uintptr_t)d_len % 4 || (uintptr_t)d_table % 4 || (uintptr_t)d_pos % 4) return PF_EINVAL;
    const int hd = cache->hd;
    const int64_t row = (int64_t)cache->n_kv * hd, q_row = (int64_t)n_heads * hd;
    if (k_stride < row || v_stride < row || k_stride % 8 || v_stride % 8) return PF_EINVAL;
    if (n_heads > 0 && (!d_q || !d_q_out || !aligned16(d_q) || !aligned16(d_q_out) || q_stride < q_row || q_out_stride < q_row || q_stride % 8 || q_out_stride % 8))
        return PF_EINVAL;
    AppendRopeArgs a;
    a.c = *cache;
    a.r = Rot{rotary->d_phase, rotary->rot, rotary->amplitude, 1.f};
    a.q = d_q; a.qo = d_q_out; a.k = d_k; a.v = d_v;
    a.qs = q_stride; a.qos = q_out_stride; a.ks = k_stride; a.vs = v_stride;
    a.cu = d_cu_new; a.len = d_len; a.table = d_table; a.pos = d_pos;
    a.n_seq = n_seq; a.cols = table_cols; a.n_new = n_new; a.n_heads = n_heads;
    a.max_new = (int32_t)(max_new < n_new ? max_new : n_new);
    // the most pages that max_new tokens behind any start can touch
    a.units_per_seq = (int)(((int64_t)cache->page - 1 + a.max_new + cache->page - 1) / cache->page);
    if (a.units_per_seq > table_cols) a.units_per_seq = table_cols;
    a.units = (int64_t)n_seq * a.units_per_seq * cache->n_kv * 2;
    const int64_t rows = a.max_new <= 4 ? (int64_t)n_seq * a.max_new : n_new;
    a.per = a.groups = 1;
    a.q_units = 0;
    if (n_heads > 0) {
        a.per = heads_per_thread(rows * n_heads * (hd / 16), n_heads);
        a.groups = (n_heads + a.per - 1) / a.per;
        a.q_units = rows * a.groups * (hd / 16);
    }
    if (a.units + a.q_units / 128 + 2 >= (1ll << 31)) return PF_ERANGE;
    if (a.units == 0 && a.q_units == 0) return PF_OK;
    cudaStream_t st = (cudaStream_t)stream;
    const bool half = rotary->layout == PF_ROPE_HALF;
    auto go = [&](auto t) {
        using T = decltype(t);
        if (hd == 64) half ? append_rope_launch<T, 64, true>(a, st) : append_rope_launch<T, 64, false>(a, st);
        else half ? append_rope_launch<T, 128, true>(a, st) : append_rope_launch<T, 128, false>(a, st);
    };
    dtype == PF_DT_BF16 ? go(Bf16{}) : go(F16{});
    PF_CUDA_TRY(cudaGetLastError(), "append_rope_kernel launch");
    count_launch();
    return PF_OK;
}
