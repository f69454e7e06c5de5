// pf_moe.cu -- a whole mixture-of-experts layer for a few tokens in two kernels.
//
//   l = x R^T,  (e_1 .. e_K) = the K largest,  w = softmax(l_e),  out = sum_k w_k D_e (silu(G_e x) * (U_e x)) + shared
//
// With few tokens the layer is a stream: every chosen expert's three matrices are read once, each element takes part in as
// many multiplications as tokens chose the expert.  HBM bounds it, so the kernels are built to keep weight bytes in flight:
//  - pf_moe_pack lays the matrices out once in the order in which the lanes of a warp hold them for the matrix
//    instruction (m16n8k16: 16 weight rows times up to 8 tokens), so a warp's copies are contiguous and no lane
//    needs another lane's bytes.
//  - moe_route_kernel: router logits (partial sums over slices of H), and the tokens as the second kernel's products take them.
//  - moe_kernel: one block per SM, launched cooperatively, does everything else.  Its blocks choose the experts, then run
//    through the row tiles of the chosen experts' gate and up matrices, meet, run through the tiles of the down matrices,
//    meet, and add up each token's parts in a fixed order.  Four warps of a block copy (bulk copies into a ring of 3 to
//    5 stages of 32 KB of weights, completion on an mbarrier), sixteen multiply; a multiplying warp waits for nothing but its stage.
//    While the blocks meet, the ring already fills with the down matrices' first stages, which do not depend on the meeting.
//  - Every wait has a limit.  Where one runs out (a block that never comes to a meeting, a copy that never arrives) the layer's work goes on as far
//    as it goes, so that all waits of the block end and nothing is in flight when it does; the status is 1, and every block that knows of it
//    writes NaN instead of its part of the output.
//  - 8 gate rows and the same 8 up rows form one 16-row tile: a lane's accumulators hold both factors of its products.
// Sums are fp32.  bf16 weights multiply bf16 tokens; the hidden activations (fp32) enter the second product as the
// sum of two bf16 numbers (16 bits of mantissa).  e4m3 weights are widened to fp16, which is exact; tokens and hidden activations
// are scaled by a power of two per row and rounded to fp16 (11 bits); a weight block's scale is applied to the fp32 sum of
// its 128 columns.  A hidden row's power of two has to be known before the row is: |h_f| <= |g_f . x| |u_f . x| <= |x|^2 max|g| max|u|
// (Cauchy-Schwarz; |silu(a)| <= |a|), the maxima over blocks of 128 hidden units, whose sizes pf_moe_pack has evened out.  The bound may lie
// 2^29 above an |h| before fp16's least step costs it any of its 11 bits; with random weights it lies a factor H above, which leaves
// 2^16 for gate and up rows of a block that are larger than its others.
// The legacy matrix instruction is enough: at full HBM speed a scheduler gets a 2 KB slice every 333 cycles, and its products take 70 for up to
// 8 tokens an expert.  Beyond 16 tokens an expert the reads of token rows from shared memory (4 per product) bound the kernel.
// Measured (one B200, device time): 1 token, bf16, 6 + 2 of 64 experts of 4096 x 1408 (277 MB): 66 us; 16 tokens, e4m3, 8 of 128, 32 here, 5120 x
// 1536 (511 MB): 122 us; 128 tokens, e4m3, 8 of 256, 32 here, 7168 x 2048 (1436 MB): 337 us.  Of the 66 us the streams of the two products take 44
// (6.3 TB/s), the router's kernel 5, the choice and the sorting of pairs 5, the meetings 8.
#include <atomic>
#include <type_traits>

#include "pf_ops.cuh"

namespace pf {

constexpr int kMoeWarps = 16, kMoeThreads = kMoeWarps * 32;   // that multiply
constexpr int kCopyWarps = 4;                                // that copy
constexpr int kMoeBlock = kMoeThreads + kCopyWarps * 32;
constexpr int kSliceBytes = 2048;          // 16 rows x KW elements, KW = 64 (bf16) or 128 (e4m3)
constexpr size_t kMoeSmem = 227 * 1024 - 1024;   // dynamic shared memory of a block, beside its static variables
constexpr unsigned kMeetLimit = 1u << 21;  // polls of a meeting before it gives up (a poll takes about a microsecond)
std::atomic<unsigned> g_meet_limit{kMeetLimit}, g_meet_missing{0};      // host: what the next calls wait for (pf_moe_meeting)
constexpr unsigned kRanOut = 1u << 31;
constexpr unsigned kRingLimit = 1u << 20;  // waits of up to a microsecond for a stage before they give up

struct MoeArgs {
    pf_moe_t m;
    int T, choices;                        // choices = top_k + n_shared: a token's (token, expert) pairs
    int n_sets;                            // n_local + n_shared
    int f_tiles, h_tiles, ks_up, ks_down;  // row tiles and column slices of the packed matrices
    int Fp;                                // 8 * f_tiles
    int Hk, Fk;                            // H and F rounded up to whole slices: row lengths of the products' inputs
    size_t set_bytes, down_at;             // packed bytes per expert, offset of its down part
    size_t n_up_scales, n_down_scales;     // block scales of one expert's gate (or up) and down matrices
    size_t packed_bytes;                   // matrices, then gate, up and down scales, then bounds
    const uint16_t *x;
    int64_t xs;
    const uint8_t *xq;
    const float *xscale;
    const uint16_t *router;
    const uint8_t *packed;
    const float *gs, *us, *ds;             // block scales and bounds, behind the packed matrices (e4m3 weights)
    const float *row_max;                  // [n_sets][2] squares whose roots' product bounds a hidden unit's size over |x|^2
    uint16_t *out;
    int32_t *ids;
    float *weights;
    int32_t *status;
    // workspace
    unsigned *ctl;                         // arrivals, and kRanOut once a wait ran out
    float *logits;                         // [h_splits][T][n_experts]
    uint16_t *xh;                          // [T][Hk] tokens, zero behind H: bf16, or fp16 times a power of two (e4m3 weights)
    float *xh_scale;                       // [T] that power of two
    float *x_norm2;                        // [T] |x|^2 (e4m3 weights)
    uint16_t *hop;                         // zero behind F; bf16: [pairs][2][Fk] high and low parts; e4m3: [pairs][Fk] fp16
    float *y;                              // [pairs][H]
    int h_splits, e_tiles, t_chunks;       // router grid
    unsigned meet_limit, meet_missing;     // polls of a meeting; arrivals that it waits for and nobody makes (0 but in a test of the limit)
};

// ------------------------------------------------------------------ weight layout
// Slice s of row tile r holds 16 rows x KW columns as four chunks of 512 bytes, 16 bytes a lane.  bf16: chunk c is one step of the
// matrix instruction, columns k = 64 s + 32 (c / 2) + 8 q + 4 (c % 2) + {0, 1 | 2, 3}; e4m3: chunk c is two steps, columns
// k = 128 s + 32 c + 8 q + 4 step + {0, 1 | 2, 3}.  Within a step: (row g, first pair), (row g + 8, first pair), (row g, second pair),
// (row g + 8, second pair).
template <bool E4M3>
__global__ void __launch_bounds__(256) moe_pack_kernel(const pf_moe_t m, int n_sets, int f_tiles, int ks_up, int ks_down, size_t set_bytes,
                                                       size_t down_at, const uint8_t *gate, const uint8_t *up, const uint8_t *down,
                                                       uint8_t *packed)
{
    constexpr int ES = E4M3 ? 1 : 2, KW = E4M3 ? 128 : 64;
    const size_t per_set = set_bytes / 16;
    const size_t total = per_set * (size_t)n_sets;
    for (size_t i = (size_t)blockIdx.x * blockDim.x + threadIdx.x; i < total; i += (size_t)gridDim.x * blockDim.x) {
        const size_t set = i / per_set, in_set = i - set * per_set;
        const bool is_down = in_set * 16 >= down_at;
        const size_t u = is_down ? in_set - down_at / 16 : in_set;
        const int lane = (int)(u & 31), chunk = (int)((u >> 5) & 3), g = lane >> 2, q = lane & 3;
        const size_t slice = u >> 7;
        const int ks = is_down ? ks_down : ks_up, tile = (int)(slice / ks), s = (int)(slice % ks);
        const int rows = is_down ? m.H : m.F, cols = is_down ? m.F : m.H;
        uint32_t w[4] = {0, 0, 0, 0};
        uint8_t *b = reinterpret_cast<uint8_t *>(w);
#pragma unroll
        for (int j = 0; j < 16 / ES; j++) {
            const int step = j / 8, r = (j >> 1) & 1, pair = (j >> 2) & 1, one = j & 1;
            const int k = s * KW + (E4M3 ? chunk * 32 + 8 * q + 4 * step : (chunk >> 1) * 32 + 8 * q + 4 * (chunk & 1)) + 2 * pair + one;
            const int row = is_down ? tile * 16 + g + 8 * r : tile * 8 + g;
            const uint8_t *src = is_down ? down : (r ? up : gate);
            if (row < rows && k < cols) {
                const uint8_t *p = src + ((set * rows + row) * (size_t)cols + k) * ES;
#pragma unroll
                for (int x = 0; x < ES; x++) b[j * ES + x] = p[x];
            }
        }
        reinterpret_cast<uint4 *>(packed)[i] = make_uint4(w[0], w[1], w[2], w[3]);
    }
}

// A block of 128 hidden units of an expert (e4m3): its units' sizes are bounded by |x|^2 p, p the product of the block's largest gate and up row
// norms.  The block's up scales are multiplied by 2^-b and its down scales by 2^b, p = 1.m * 2^b, so that the activations of all
// blocks come out below 2 |x|^2 and one block's outlier rows take no bits off the others' fp16 numbers.  What is left of the
// bound, squared (1.m^2, more where b is clamped), goes to the expert's largest.
__global__ void __launch_bounds__(256) moe_block_norm_kernel(const pf_moe_t m, const uint8_t *gate, const uint8_t *up, const float *gs, float *us, float *ds,
                                                             float *bound2)
{
    __shared__ float part[2][8];
    const int kb = (m.H + 127) / 128, fb = (m.F + 127) / 128, set = blockIdx.x / fb, block = blockIdx.x - set * fb;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, rows = min(128, m.F - block * 128);
    float *su = us + ((size_t)set * fb + block) * kb, *sd = ds + (size_t)set * kb * fb + block;
    float top[2] = {0.f, 0.f};
    bool nan = false;
    for (int r = warp; r < rows; r += 8)
#pragma unroll
        for (int which = 0; which < 2; which++) {
            const uint8_t *w = (which ? up : gate) + ((size_t)set * m.F + block * 128 + r) * m.H;
            const float *sc = which ? su : gs + ((size_t)set * fb + block) * kb;
            float ss = 0.f;
            for (int k = lane * 16; k < m.H; k += 512) {
                const uint4 v = *reinterpret_cast<const uint4 *>(w + k);
                const uint32_t c[4] = {v.x, v.y, v.z, v.w};
                float sum = 0.f;
#pragma unroll
                for (int i = 0; i < 4; i++) {
                    const float2 f = f32x2_of_f16x2(f16x2_of_e4m3x2(c[i])), g = f32x2_of_f16x2(f16x2_of_e4m3x2(c[i] >> 16));
                    sum = fmaf(f.x, f.x, fmaf(f.y, f.y, fmaf(g.x, g.x, fmaf(g.y, g.y, sum))));
                }
                const float s = sc[k / 128];
                ss = fmaf(sum * s, s, ss);
            }
#pragma unroll
            for (int o = 16; o; o >>= 1) ss += __shfl_xor_sync(0xFFFFFFFFu, ss, o);
            top[which] = fmaxf(top[which], ss);
            nan |= ss != ss;
        }
    if (lane == 0) {
        part[0][warp] = nan ? __int_as_float(0x7FFFFFFF) : top[0];
        part[1][warp] = top[1];
    }
    __syncthreads();
    float g2 = 0.f, u2 = 0.f;
    nan = false;
#pragma unroll
    for (int i = 0; i < 8; i++) {
        nan |= part[0][i] != part[0][i];
        g2 = fmaxf(g2, part[0][i]);
        u2 = fmaxf(u2, part[1][i]);
    }
    float p = sqrtf(g2) * sqrtf(u2);
    const int b = p > 0.f && p < INFINITY && !nan ? max(-64, min(64, (int)(__float_as_uint(p) >> 23) - 127)) : 0;
    const float down = __uint_as_float((uint32_t)(127 - b) << 23), lift = __uint_as_float((uint32_t)(127 + b) << 23);
    p *= down;
    if (threadIdx.x == 0 && !nan) atomicMax(reinterpret_cast<unsigned *>(bound2 + set * 2), __float_as_uint(p * p));   // not negative: bits in the order of the values
    if (threadIdx.x == 0 && block == 0) bound2[set * 2 + 1] = 1.f;
    for (int k = threadIdx.x; k < kb; k += 256) {
        su[k] *= down;
        sd[(size_t)k * fb] *= lift;
    }
}

// ------------------------------------------------------------------ router logits, tokens as fp16
// exponent that brings a row's largest magnitude into [2^13, 2^14): what is 2^-27 of it keeps 11 bits in fp16
__device__ __forceinline__ int fp16_exponent(float amax)
{
    const int e = (amax > 0.f && amax < INFINITY) ? (int)(__float_as_uint(amax) >> 23) - 127 : 0;
    return max(-100, e) - 13;
}
__device__ __forceinline__ float exp2i(int e) { return __uint_as_float((uint32_t)(min(127, max(-126, e)) + 127) << 23); }

// a hidden row's exponent: 2^-e brings |x|^2 |g| |u| (squares of the norms given), and so the row, below 2^15.  2 % cover the tokens' rounding.
__device__ __forceinline__ int hidden_exponent(float x2, float g2, float u2)
{
    const float b = 1.02f * x2 * sqrtf(g2) * sqrtf(u2);
    if (!(b > 0.f)) return 0;
    return max(-112, min(112, (int)(__float_as_uint(b) >> 23) - 127 + 1 - 15));
}

constexpr int kRouteSplits = 8, kRouteWarps = 8, kRouteThreads = kRouteWarps * 32;
template <bool E4M3, int JT>
__global__ void __launch_bounds__(kRouteThreads) moe_route_kernel(const __grid_constant__ MoeArgs A)
{
    constexpr int kTokens = 8 * JT;                          // of a block: route_tokens() on the host
    __shared__ float red[kRouteWarps][16][kTokens + 1];
    __shared__ float part[2][kRouteWarps];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, q = lane & 3;
    const int n_gemm = A.e_tiles * A.h_splits * A.t_chunks;
    const int H = A.m.H, E = A.m.n_experts;
    if (blockIdx.x == 0) {
        if (tid == 0) *A.ctl = 0u;
        if (tid == 0 && A.status) *A.status = 0;
    }
    if ((int)blockIdx.x < n_gemm) {
        const int et = blockIdx.x % A.e_tiles, r = blockIdx.x / A.e_tiles, hs = r % A.h_splits, tc = r / A.h_splits;
        const int groups = (H + 31) / 32;                    // 32 columns at a time
        const int k_lo = (int)((long long)groups * hs / A.h_splits), k_hi = (int)((long long)groups * (hs + 1) / A.h_splits);
        const int t0 = tc * kTokens, n = min(kTokens, A.T - t0);
        float c[JT][4];
#pragma unroll
        for (int j = 0; j < JT; j++) c[j][0] = c[j][1] = c[j][2] = c[j][3] = 0.f;
        const int r0 = et * 16 + g, r1 = r0 + 8;
#pragma unroll 4
        for (int kg = k_lo + warp; kg < k_hi; kg += kRouteWarps) {
            const int k = kg * 32 + q * 8;
            const uint4 zero = make_uint4(0, 0, 0, 0);
            const uint4 a = k < H && r0 < E ? __ldg(reinterpret_cast<const uint4 *>(A.router + (int64_t)r0 * H + k)) : zero;
            const uint4 b = k < H && r1 < E ? __ldg(reinterpret_cast<const uint4 *>(A.router + (int64_t)r1 * H + k)) : zero;
            uint4 x[JT];
#pragma unroll
            for (int j = 0; j < JT; j++)
                x[j] = k < H && j * 8 + g < n ? __ldg(reinterpret_cast<const uint4 *>(A.x + (int64_t)(t0 + j * 8 + g) * A.xs + k)) : zero;
#pragma unroll
            for (int j = 0; j < JT; j++) {
                mma16<Bf16>(c[j], a.x, b.x, a.y, b.y, x[j].x, x[j].y);
                mma16<Bf16>(c[j], a.z, b.z, a.w, b.w, x[j].z, x[j].w);
            }
        }
#pragma unroll
        for (int j = 0; j < JT; j++) {
            red[warp][g][j * 8 + 2 * q] = c[j][0];
            red[warp][g][j * 8 + 2 * q + 1] = c[j][1];
            red[warp][g + 8][j * 8 + 2 * q] = c[j][2];
            red[warp][g + 8][j * 8 + 2 * q + 1] = c[j][3];
        }
        __syncthreads();
        for (int i = tid; i < 16 * n; i += kRouteThreads) {
            const int e = i & 15, t = i >> 4;
            float s = 0.f;
#pragma unroll
            for (int wv = 0; wv < kRouteWarps; wv++) s += red[wv][e][t];
            if (et * 16 + e < E) A.logits[((int64_t)hs * A.T + t0 + t) * E + et * 16 + e] = s;
        }
        return;
    }
    const int t = blockIdx.x - n_gemm;
    if constexpr (!E4M3) {
        for (int k = tid * 8; k < A.Hk; k += kRouteThreads * 8)
            *reinterpret_cast<uint4 *>(A.xh + (size_t)t * A.Hk + k) =
                k < H ? *reinterpret_cast<const uint4 *>(A.x + (int64_t)t * A.xs + k) : make_uint4(0, 0, 0, 0);
    } else {
    // token t as fp16 times a power of two
    const int groups = (H + PF_SCALE_GROUP - 1) / PF_SCALE_GROUP;
    auto value8 = [&](int k, float (&v)[8]) {
        if (A.xq) {
            const uint2 b = *reinterpret_cast<const uint2 *>(A.xq + (int64_t)t * H + k);
            const float s = A.xscale[t * groups + k / PF_SCALE_GROUP];
            const uint32_t w[4] = {b.x & 0xFFFFu, b.x >> 16, b.y & 0xFFFFu, b.y >> 16};
#pragma unroll
            for (int i = 0; i < 4; i++) {
                const float2 f = f32x2_of_f16x2(f16x2_of_e4m3x2(w[i]));
                v[2 * i] = f.x * s;
                v[2 * i + 1] = f.y * s;
            }
        } else {
            const uint4 b = *reinterpret_cast<const uint4 *>(A.x + (int64_t)t * A.xs + k);
            const uint32_t w[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
            for (int i = 0; i < 4; i++) {
                const float2 f = f32x2_of_bf16x2(w[i]);
                v[2 * i] = f.x;
                v[2 * i + 1] = f.y;
            }
        }
    };
    float m = 0.f, ss = 0.f;
    for (int k = tid * 8; k < H; k += kRouteThreads * 8) {
        float v[8];
        value8(k, v);
#pragma unroll
        for (int i = 0; i < 8; i++) {
            m = fmaxf(m, fabsf(v[i]));
            ss = fmaf(v[i], v[i], ss);
        }
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) {
        m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, o));
        ss += __shfl_xor_sync(0xFFFFFFFFu, ss, o);
    }
    if (lane == 0) {
        part[0][warp] = m;
        part[1][warp] = ss;
    }
    __syncthreads();
    ss = 0.f;
#pragma unroll
    for (int i = 0; i < kRouteWarps; i++) {
        m = fmaxf(m, part[0][i]);
        ss += part[1][i];
    }
    const int e = fp16_exponent(m);
    const float down = exp2i(-e);
    if (tid == 0) {
        A.xh_scale[t] = exp2i(e);
        A.x_norm2[t] = ss;
    }
    for (int k = tid * 8; k < A.Hk; k += kRouteThreads * 8) {
        float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (k < H) value8(k, v);
        *reinterpret_cast<uint4 *>(A.xh + (size_t)t * A.Hk + k) =
            make_uint4(f16x2_of(v[0] * down, v[1] * down), f16x2_of(v[2] * down, v[3] * down), f16x2_of(v[4] * down, v[5] * down),
                       f16x2_of(v[6] * down, v[7] * down));
    }
    }
}

// ------------------------------------------------------------------ the layer
__device__ __forceinline__ void wait_ran_out(const MoeArgs &A)
{
    atomicOr(A.ctl, kRanOut);
    if (A.status) *A.status = 1;
}
// All blocks of the (cooperative) grid meet, each represented by one thread; false where this or any wait before it ran out, here or in a
// block whose word has come through.
__device__ __forceinline__ bool arrive_and_poll(const MoeArgs &A, unsigned round, bool arrive)
{
    if (arrive) {
        __threadfence();
        atomicAdd(A.ctl, 1u);
    }
    unsigned seen = 0, polls = 0;
    do {
        asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(seen) : "l"(A.ctl) : "memory");
    } while (seen < round + A.meet_missing && ++polls < A.meet_limit);      // (kRanOut is above any number of arrivals)
    __threadfence();
    return seen >= round + A.meet_missing && !(seen & kRanOut);
}
template <int ID, int THREADS> __device__ __forceinline__ void bar()
{
    asm volatile("bar.sync %0, %1;" ::"n"(ID), "n"(THREADS) : "memory");
}
// the multiplying threads (or, before the roles part, all threads) of the block meet the other blocks'
template <int ID, int THREADS>
__device__ __forceinline__ bool meet(const MoeArgs &A, unsigned &round, int *ok)
{
    round += gridDim.x;
    asm volatile("fence.proxy.async;" ::: "memory");      // what was written is read by bulk copies
    bar<ID, THREADS>();
    if (threadIdx.x == 0) {
        *ok = arrive_and_poll(A, round, true);
        if (!*ok) wait_ran_out(A);
    }
    bar<ID, THREADS>();
    return *ok != 0;
}

// ---- mbarriers in shared memory
__device__ __forceinline__ void mbar_init(uint32_t b, unsigned count) { asm volatile("mbarrier.init.shared.b64 [%0], %1;" ::"r"(b), "r"(count) : "memory"); }
__device__ __forceinline__ void mbar_arrive(uint32_t b) { asm volatile("mbarrier.arrive.shared.b64 _, [%0];" ::"r"(b) : "memory"); }
__device__ __forceinline__ void mbar_expect(uint32_t b, uint32_t bytes)
{
    asm volatile("mbarrier.arrive.expect_tx.shared.b64 _, [%0], %1;" ::"r"(b), "r"(bytes) : "memory");
}
// waits for the phase of the given parity to end; false where the wait ran out
__device__ __forceinline__ bool mbar_wait(uint32_t b, unsigned parity)
{
    for (unsigned i = 0; i < kRingLimit; i++) {
        uint32_t done;
        asm volatile("{\n.reg .pred p;\nmbarrier.try_wait.parity.shared.b64 p, [%1], %2, %3;\nselp.u32 %0, 1, 0, p;\n}"
                     : "=r"(done) : "r"(b), "r"(parity), "r"(1000u) : "memory");
        if (done) return true;
    }
    return false;
}
__device__ __forceinline__ void bulk_copy(uint32_t dst, const void *src, uint32_t bytes, uint32_t mbar)
{
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes), "r"(mbar) : "memory");
}

// One warp chooses token t's experts: `keep` ([T][top_k], may be NULL) gets the indices, and the outputs too where `write`.
template <int KEYS>
__device__ __forceinline__ void choose(const MoeArgs &A, int t, int *keep, bool write)
{
    const int lane = threadIdx.x & 31, T = A.T, K = A.m.top_k, E = A.m.n_experts;
    float v[KEYS];
    uint32_t key[KEYS];
#pragma unroll
    for (int i = 0; i < KEYS; i++) v[i] = 0.f;
#pragma unroll
    for (int hs = 0; hs < kRouteSplits; hs++)                   // added in a fixed order
#pragma unroll
        for (int i = 0; i < KEYS; i++) {
            const int e = i * 32 + lane;
            v[i] += hs < A.h_splits && e < E ? A.logits[((int64_t)hs * T + t) * E + e] : 0.f;
        }
#pragma unroll
    for (int i = 0; i < KEYS; i++) {
        const uint32_t b = v[i] == v[i] ? __float_as_uint(v[i]) : 0xFF800000u;
        key[i] = i * 32 + lane < E ? ((b >> 31) ? ~b : (b | 0x80000000u)) : 0u;      // order of the floats; 0 = not there, or taken
    }
    float top = 0.f, sum = 0.f, mine = 0.f;
    int my_id = 0;
    for (int j = 0; j < K; j++) {
        uint32_t best = 0u, at = 0xFFFFFFFFu;
#pragma unroll
        for (int i = 0; i < KEYS; i++) best = max(best, key[i]);
        const uint32_t all = __reduce_max_sync(0xFFFFFFFFu, best);
#pragma unroll
        for (int i = KEYS - 1; i >= 0; i--)
            if (key[i] == all) at = i * 32 + lane;
        at = __reduce_min_sync(0xFFFFFFFFu, at);
#pragma unroll
        for (int i = 0; i < KEYS; i++)
            if (at == (uint32_t)(i * 32 + lane)) key[i] = 0u;
        const float l = __uint_as_float((all >> 31) ? all & 0x7FFFFFFFu : ~all);
        if (j == 0) top = l;
        const float w = expf(l - top);
        sum += w;
        if (lane == j) {
            mine = w;
            my_id = (int)at;
        }
    }
    if (lane < K) {
        if (keep) keep[t * K + lane] = my_id;
        if (write) {
            A.ids[t * K + lane] = my_id;
            A.weights[t * K + lane] = mine / sum;
        }
    }
}

template <bool E4M3, int NT, int STAGES_>
struct MoeShape {
    static constexpr int KW = E4M3 ? 128 : 64;
    static constexpr int PLANES = E4M3 ? 1 : 2;               // of the hidden activations
    static constexpr int LWK = NT == 16 && !E4M3 ? 2 : 1;     // log2 of the fewest warps that share a row tile
    static constexpr int TM = kMoeWarps >> LWK;               // row tiles of an item, at most
    static constexpr int A_BYTES = kMoeWarps * kSliceBytes;
    // a stage's token row, for 2^lwk slices; 64 mod 128: two rows' quarters use all banks
    static constexpr __host__ __device__ int pitch(int lwk) { return (KW * 2 << lwk) + 64; }
    static constexpr int B_BYTES = NT * PLANES * ((KW * 2 << LWK) + 64);
    static constexpr int STAGE = A_BYTES + B_BYTES;
    static constexpr int PASS = NT < 16 ? NT : 16;            // tokens whose partial sums meet at a time
    static constexpr int RED = kMoeWarps * 16 * PASS * 4;
    static constexpr int STAGES = STAGES_;
    static constexpr int FIXED = STAGES * STAGE + RED;
};

template <bool E4M3, int NT, int STAGES_>
__global__ void __launch_bounds__(kMoeBlock, 1) moe_kernel(const __grid_constant__ MoeArgs A)
{
    using S = MoeShape<E4M3, NT, STAGES_>;
    using MT = typename std::conditional<E4M3, F16, Bf16>::type;
    constexpr int kStages = S::STAGES;
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ __align__(8) uint64_t bars[2 * kStages];
    __shared__ int meet_ok;
    __shared__ int n_active_s;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, q = lane & 3;
    const int T = A.T, K = A.m.top_k, C = A.choices, E = A.m.n_experts, H = A.m.H;
    uint8_t *ring_p = smem;
    const uint32_t ring = smem_addr(ring_p);
    float *red = reinterpret_cast<float *>(smem + kStages * S::STAGE);
    int *cnt = reinterpret_cast<int *>(smem + S::FIXED);      // [n_sets] tokens per expert, then running offsets
    int *off = cnt + A.n_sets;                                                       // [n_sets] first list entry
    int *act = off + A.n_sets;                                                       // [n_sets] experts with tokens
    int *cum = act + A.n_sets;                                                       // [n_sets + 1] token chunks before an active expert
    uint16_t *list = reinterpret_cast<uint16_t *>(cum + A.n_sets + 1);               // [T * C] pairs by expert
    unsigned *local = reinterpret_cast<unsigned *>(list + (T * C + 1) / 2 * 2);      // [T] which of a token's choices are here
    unsigned round = 0;

    // ---- the choice: one warp per token.  For few tokens each block makes all of it by itself, which saves a meeting.
    const bool by_itself = T <= kMoeWarps;
    // the block's part of the output, four elements a thread, where a wait ran out
    auto spoil = [&]() {
        if (tid >= kMoeThreads) return;
        for (int i = blockIdx.x * kMoeThreads + tid; i < T * (H / 4); i += gridDim.x * kMoeThreads)
            reinterpret_cast<uint2 *>(A.out)[i] = make_uint2(0x7FFF7FFFu, 0x7FFF7FFFu);
    };
    if (tid == 0) {
        for (int i = 0; i < kStages; i++) {
            mbar_init(smem_addr(bars + i), 2 * kCopyWarps);      // full: each copying warp's announcements of weights and of tokens, and their bytes
            mbar_init(smem_addr(bars + kStages + i), kMoeWarps);   // empty: the multiplying warps
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp < kMoeWarps) {
        const int t0 = by_itself ? warp : warp * (int)gridDim.x + (int)blockIdx.x, dt = by_itself ? kMoeWarps : kMoeWarps * (int)gridDim.x;
        int *keep = by_itself ? reinterpret_cast<int *>(red) : nullptr;
        const bool write = !by_itself || blockIdx.x == 0;
        for (int t = t0; t < T; t += dt) {
            if (E <= 64) choose<2>(A, t, keep, write);
            else if (E <= 128) choose<4>(A, t, keep, write);
            else if (E <= 256) choose<8>(A, t, keep, write);
            else choose<16>(A, t, keep, write);
        }
    }
    if (by_itself) __syncthreads();
    else if (!meet<0, kMoeBlock>(A, round, &meet_ok)) return spoil();      // the choices are not there: nothing can be run

    // ---- pairs by expert, in pair order within each: off and cnt of every expert (cnt: the end of its pairs), the experts that
    // have any, the chunks of NT tokens before each of those, and which of a token's choices are here.  All blocks arrive at the same.
    const int P = T * C;
    // The experts of all tokens come first in the list, so that what is left for its end, cut into small pieces, has few tokens.
    auto set_of = [&](int t, int j) {        // place of the expert of token t's choice j among this GPU's, n_sets if it lives elsewhere
        if (j >= K) return j - K;
        const int e = (by_itself ? reinterpret_cast<const int *>(red)[t * K + j] : A.ids[t * K + j]) - A.m.first;
        return e >= 0 && e < A.m.n_local ? A.m.n_shared + e : A.n_sets;
    };
    // offsets, experts with pairs and chunks from the counts in cnt: a scan by warp 0; cnt becomes `begin` ? off : the pairs' end
    auto scan = [&](bool begin) {
        int o = 0, a = 0, c = 0;
        for (int i0 = 0; i0 < A.n_sets; i0 += 32) {
            const int i = i0 + lane, n = i < A.n_sets ? cnt[i] : 0, ch = (n + NT - 1) / NT;
            int so = n, sc = ch;
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const int u = __shfl_up_sync(0xFFFFFFFFu, so, d), v = __shfl_up_sync(0xFFFFFFFFu, sc, d);
                if (lane >= d) {
                    so += u;
                    sc += v;
                }
            }
            const unsigned live = __ballot_sync(0xFFFFFFFFu, n > 0);
            if (i < A.n_sets) {
                off[i] = o + so - n;
                cnt[i] = begin ? o + so - n : o + so;
            }
            if (n > 0) {
                const int at = a + __popc(live & ((1u << lane) - 1u));
                act[at] = i;
                cum[at + 1] = c + sc;
            }
            o += __shfl_sync(0xFFFFFFFFu, so, 31);
            c += __shfl_sync(0xFFFFFFFFu, sc, 31);
            a += __popc(live);
        }
        if (lane == 0) {
            cum[0] = 0;
            n_active_s = a;
        }
    };
    if (P <= kMoeBlock) {
        // a thread for each pair: its rank within its warp, and before it the pairs of the warps in front
        uint16_t *before = reinterpret_cast<uint16_t *>(ring_p);      // [warps][n_sets]; the ring is not in use yet
        const int used = (P + 31) / 32;
        for (int i = tid; i < used * A.n_sets; i += kMoeBlock) before[i] = 0;
        if (tid < T) local[tid] = 0u;
        __syncthreads();
        int s = A.n_sets, rank = 0;
        if (warp < used) {
            if (tid < P) {
                const int t = tid / C, j = tid - t * C;
                s = set_of(t, j);
                if (s < A.n_sets) atomicOr(local + t, 1u << j);
            }
            const unsigned same = __match_any_sync(0xFFFFFFFFu, s);
            rank = __popc(same & ((1u << lane) - 1u));
            if (s < A.n_sets && rank == 0) before[warp * A.n_sets + s] = (uint16_t)__popc(same);
        }
        __syncthreads();
        for (int i = tid; i < A.n_sets; i += kMoeBlock) {
            int c = 0;
            for (int w = 0; w < used; w++) {
                const int n = before[w * A.n_sets + i];
                before[w * A.n_sets + i] = (uint16_t)c;
                c += n;
            }
            cnt[i] = c;
        }
        __syncthreads();
        if (warp == 0) scan(false);
        __syncthreads();
        if (s < A.n_sets) list[off[s] + before[warp * A.n_sets + s] + rank] = (uint16_t)tid;
        __syncthreads();
    } else {
        uint16_t *set_at = reinterpret_cast<uint16_t *>(ring_p), *dealt = set_at + P;
        for (int i = tid; i < A.n_sets; i += kMoeBlock) cnt[i] = 0;
        __syncthreads();
        for (int t = tid; t < T; t += kMoeBlock) {
            unsigned mask = 0u;
            for (int j = 0; j < C; j++) {
                const int s = set_of(t, j);
                if (s == A.n_sets) continue;
                atomicAdd(cnt + s, 1);
                mask |= 1u << j;
            }
            local[t] = mask;
        }
        __syncthreads();
        if (warp == 0) scan(true);
        __syncthreads();
        // dealt out in any order, then ranked by pair number within each expert
        for (int t = tid; t < T; t += kMoeBlock)
            for (int j = 0; j < C; j++) {
                const int s = set_of(t, j);
                if (s == A.n_sets) continue;
                const int at = atomicAdd(cnt + s, 1);
                dealt[at] = (uint16_t)(t * C + j);
                set_at[at] = (uint16_t)s;
            }
        __syncthreads();                     // now cnt[s] is the end of expert s's pairs
        for (int i = tid; i < (n_active_s ? cnt[act[n_active_s - 1]] : 0); i += kMoeBlock) {
            const int s = set_at[i], p = dealt[i], lo = off[s], hi = cnt[s];
            int rank = lo;
            for (int k = lo; k < hi; k++) rank += dealt[k] < p;
            list[rank] = (uint16_t)p;
        }
        __syncthreads();
    }
    auto weights_of = [&](int place) { return place < A.m.n_shared ? A.m.n_local + place : place - A.m.n_shared; };      // index in the weight tensors
    const int n_active = n_active_s, n_chunks = cum[n_active];

    // ---- The work of a product is a list: for every chunk of up to NT tokens of an expert, that expert's row tiles.  Blocks take TM
    // tiles of it in turn, so that each gets its part of the chunks that cost more (more tokens), as long as there are TM for every
    // block; what is left is cut into equal pieces.  (Equal contiguous pieces of the whole list: the blocks that held the experts of all
    // tokens took 1.6 times as long as the average.)  A matrix that several chunks read comes from HBM once and then from the L2.
    // An item's row tiles are dealt to groups of 2^lwk warps, which split the columns: with few tiles left a group is larger, as far as
    // the stage holds its token rows, so that the warps and the stages stay full.
    auto shape_of = [&](int tiles, int rows, int ks) {
        int lwk = tiles > 4 ? 1 : tiles > 2 ? 2 : tiles > 1 ? 3 : 4;
        while (lwk > S::LWK && (rows * S::pitch(lwk) > S::B_BYTES || (1 << lwk) >= 2 * ks)) lwk--;
        return max(lwk, S::LWK);
    };
    struct Cursor {
        int at, end, part, a, c, tile, n, tokens, lwk, stages, stage;   // tiles at .. end - 1 of the list are this block's part number `part`;
                                                                // item: tiles tile .. tile + n - 1 of chunk c (of `tokens`) of active expert a
    };
    auto item = [&](bool second, Cursor &c) {
        const int ks = second ? A.ks_down : A.ks_up;
        c.n = min((second ? A.h_tiles : A.f_tiles) - c.tile, c.end - c.at);
        c.tokens = min(NT, cnt[act[c.a]] - off[act[c.a]] - c.c * NT);
        c.lwk = shape_of(c.n, second ? c.tokens * S::PLANES : c.tokens, ks);
        c.stages = (ks + (1 << c.lwk) - 1) >> c.lwk;
        c.stage = 0;
    };
    auto take = [&](bool second, Cursor &c) {                   // the next part, if there is one
        const int tiles = second ? A.h_tiles : A.f_tiles, all = n_chunks * tiles, grid = gridDim.x, turns = all / (grid * S::TM);
        if (c.part < turns) {
            c.at = (c.part * grid + blockIdx.x) * S::TM;
            c.end = c.at + S::TM;
        } else {
            const int done = turns * grid * S::TM, left = all - done;           // left < grid * TM
            c.at = done + left * (int)blockIdx.x / grid;
            c.end = c.part == turns ? done + left * ((int)blockIdx.x + 1) / grid : c.at;
        }
        c.part++;
        if (c.at >= c.end) return;
        const int v = c.at / tiles;
        c.tile = c.at - v * tiles;
        while (cum[c.a + 1] <= v) c.a++;
        c.c = v - cum[c.a];
        item(second, c);
    };
    auto begin = [&](bool second, Cursor &c) {
        c.part = c.a = 0;
        take(second, c);
    };
    auto more = [](const Cursor &c) { return c.at < c.end; };
    auto next = [&](bool second, Cursor &c) {
        c.at += c.n;
        if (c.at >= c.end) return take(second, c);
        c.tile = 0;                                             // a part that runs into the next chunk
        if (++c.c == cum[c.a + 1] - cum[c.a]) {
            c.c = 0;
            c.a++;
        }
        item(second, c);
    };
    const int grid = gridDim.x;

    // ---- the stream: a position per stage, those of the first product and then those of the second; position p uses ring slot p % kStages
    const uint32_t full = smem_addr(bars), empty = full + kStages * 8;
    asm volatile("fence.proxy.async;" ::: "memory");            // the ring held `dealt`: bulk copies write it from here on
    __syncthreads();                                            // barriers are set up; `red` held the ids

    if (warp >= kMoeWarps) {                                    // ================= the copying warps
        // Issuing a copy takes a warp 100 to 200 cycles, and at full HBM speed a stage lasts 1400: one warp alone held the stream at
        // 5.4 TB/s.  So the copies of a stage (TM runs of weights, a row for each token) are dealt to kCopyWarps warps, and what
        // belongs to an item is worked out once.
        const int cw = warp - kMoeWarps;
        constexpr int TILES = (S::TM + kCopyWarps - 1) / kCopyWarps;                              // tiles cw, cw + kCopyWarps, ..
        constexpr int ROWS = (NT * S::PLANES + 32 * kCopyWarps - 1) / (32 * kCopyWarps);          // rows cw + kCopyWarps * (lane + 32 i)
        struct Feed {
            Cursor c;
            const uint8_t *weights;              // of tile cw, this stage
            const uint16_t *row[ROWS];           // this stage
            int tiles, rows;                     // this warp's share
        };
        auto set_up = [&](bool second, Feed &f) {
            const Cursor &c = f.c;
            if (!more(c)) return;
            const int e = act[c.a], first = off[e] + c.c * NT, n = c.tokens;
            f.weights = A.packed + (size_t)weights_of(e) * A.set_bytes + (second ? A.down_at : 0) + (size_t)(c.tile + cw) * (second ? A.ks_down : A.ks_up) * kSliceBytes;
            f.tiles = (c.n + kCopyWarps - 1 - cw) / kCopyWarps;
            f.rows = ((second ? n * S::PLANES : n) + kCopyWarps - 1 - cw) / kCopyWarps;
#pragma unroll
            for (int i = 0; i < ROWS; i++) {
                if (i * 32 + lane >= f.rows) continue;
                const int r = cw + kCopyWarps * (i * 32 + lane);
                const int p = list[first + (second ? r / S::PLANES : r)];
                f.row[i] = second ? A.hop + ((size_t)p * S::PLANES + r % S::PLANES) * A.Fk : A.xh + (size_t)(p / C) * A.Hk;
            }
        };
        auto advance = [&](bool second, Feed &f) {
            if (++f.c.stage < f.c.stages) {
                f.weights += kSliceBytes << f.c.lwk;
#pragma unroll
                for (int i = 0; i < ROWS; i++) f.row[i] += S::KW << f.c.lwk;
                return;
            }
            next(second, f.c);
            set_up(second, f);
        };
        // full barrier of a stage: each copying warp announces its weights' bytes in one arrival and its tokens' in another
        auto load_weights = [&](bool second, const Feed &f, int slot) {
            if (lane != 0) return;
            const int ks = second ? A.ks_down : A.ks_up;
            const uint32_t bytes = (uint32_t)(min(1 << f.c.lwk, ks - (f.c.stage << f.c.lwk)) * kSliceBytes);
            mbar_expect(full + slot * 8, f.tiles * bytes);
#pragma unroll
            for (int i = 0; i < TILES; i++)
                if (i < f.tiles)
                    bulk_copy(ring + slot * S::STAGE + ((cw + i * kCopyWarps) * kSliceBytes << f.c.lwk), f.weights + (size_t)(i * kCopyWarps) * ks * kSliceBytes,
                              bytes, full + slot * 8);
        };
        auto load_tokens = [&](bool second, const Feed &f, int slot) {
            const uint32_t bytes = (uint32_t)(min(1 << f.c.lwk, (second ? A.ks_down : A.ks_up) - (f.c.stage << f.c.lwk)) * S::KW * 2);
            if (lane == 0) mbar_expect(full + slot * 8, f.rows * bytes);
            __syncwarp();
#pragma unroll
            for (int i = 0; i < ROWS; i++)
                if (i * 32 + lane < f.rows)
                    bulk_copy(ring + slot * S::STAGE + S::A_BYTES + (cw + kCopyWarps * (i * 32 + lane)) * S::pitch(f.c.lwk), f.row[i], bytes, full + slot * 8);
        };
        bool ok = true;
        int pos = 0, slot = 0;
        unsigned round_of = 1;                                  // parity of the phase in which the slot was last emptied
        auto next_slot = [&]() {                                // position pos may be filled
            if (pos >= kStages) ok = mbar_wait(empty + slot * 8, round_of);
            return ok;
        };
        auto filled = [&]() {
            pos++;
            if (++slot == kStages) {
                slot = 0;
                round_of ^= 1u;
            }
        };
        Feed f;
        begin(false, f.c);
        set_up(false, f);
        while (more(f.c) && next_slot()) {
            load_weights(false, f, slot);
            load_tokens(false, f, slot);
            filled();
            advance(false, f);
        }
        begin(true, f.c);
        set_up(true, f);
        Feed late = f;                                          // tokens of the second product follow the meeting
        const int n1 = pos;                                     // (after a failed wait it does not matter)
        int pos_b = pos, slot_b = slot;
        while (ok && more(f.c) && pos < n1 + kStages && next_slot()) {
            load_weights(true, f, slot);
            filled();
            advance(true, f);
        }
        const unsigned target = round + gridDim.x;
        // (where it fails the tokens' rows are copied all the same: the ring's stages stay complete, and the output is spoilt)
        if (ok && more(late.c) && !arrive_and_poll(A, target, false) && lane == 0) wait_ran_out(A);
        __syncwarp();
        asm volatile("fence.proxy.async;" ::: "memory");
        for (; ok && pos_b < pos; pos_b++) {
            load_tokens(true, late, slot_b);
            advance(true, late);
            slot_b = slot_b + 1 == kStages ? 0 : slot_b + 1;
        }
        while (ok && more(f.c) && next_slot()) {
            load_weights(true, f, slot);
            load_tokens(true, f, slot);
            filled();
            advance(true, f);
        }
        // Nothing may be in flight when the block ends.  After a wait that ran out (no stage was emptied: the multiplying warps have given up)
        // the stages without tokens are closed first.
        if (!ok) {
            for (; pos_b < pos; pos_b++) {
                if (lane == 0) mbar_arrive(full + slot_b * 8);
                slot_b = slot_b + 1 == kStages ? 0 : slot_b + 1;
            }
            if (lane == 0) wait_ran_out(A);
        }
        for (int i = max(0, pos - kStages); i < pos && mbar_wait(full + (i % kStages) * 8, (unsigned)(i / kStages) & 1u); i++) {}
        return;
    }

    // ===================================================== the multiplying warps
    float acc[NT / 8][4], scale0 = 0.f, scale1 = 0.f;
    int slot = 0;
    unsigned parity = 0;
    bool ok = true;
    // This warp's slice of the stage into acc, JT column blocks of tokens; what is known at compile time leaves no branch between the
    // loads and the products.
    auto multiply = [&](auto second_, auto jt_, const Cursor &c) {
        constexpr bool second = decltype(second_)::value;
        constexpr int JT = decltype(jt_)::value, CH = E4M3 && JT <= 2 ? 2 : 1;
        const int ks = second ? A.ks_down : A.ks_up, wm = warp >> c.lwk, wk = warp & ((1 << c.lwk) - 1), s = (c.stage << c.lwk) + wk;
        const bool live = wm < c.n && s < ks;
        float s0 = 1.f, s1 = 1.f;
        if (E4M3) {
            if (c.stage % 32 == 0) {                            // block scales of 32 stages, a stage a lane
                const int mine = ((c.stage + lane) << c.lwk) + wk, tile = c.tile + wm;
                const bool any = wm < c.n && mine < ks;
                const int kb_n = second ? (A.m.F + 127) / 128 : (H + 127) / 128;
                if (second) {
                    scale0 = any ? __ldg(A.ds + ((size_t)weights_of(act[c.a]) * ((H + 127) / 128) + tile / 8) * kb_n + mine) : 0.f;
                } else {
                    const size_t at = ((size_t)weights_of(act[c.a]) * ((A.m.F + 127) / 128) + tile / 16) * kb_n + mine;
                    scale0 = any ? __ldg(A.gs + at) : 0.f;
                    scale1 = any ? __ldg(A.us + at) : 0.f;
                }
            }
            s0 = __shfl_sync(0xFFFFFFFFu, scale0, c.stage % 32);
            s1 = second ? s0 : __shfl_sync(0xFFFFFFFFu, scale1, c.stage % 32);
        }
        if (ok) ok = mbar_wait(full + slot * 8, parity);
        if (live && ok) {
            constexpr int planes = second ? S::PLANES : 1;
            const int pitch = S::pitch(c.lwk);
            const uint32_t wa = ring + slot * S::STAGE + warp * kSliceBytes + lane * 16;
            // a column without a token reads the last token's row: nothing outside the stage's rows is touched, nobody reads its sums
            uint32_t tb[JT];
#pragma unroll
            for (int j = 0; j < JT; j++)
                tb[j] = ring + slot * S::STAGE + S::A_BYTES + min(j * 8 + g, c.tokens - 1) * planes * pitch + wk * S::KW * 2 + q * 16;
            float sub[CH][NT / 8][4];                           // a block scale's part
            float (&sum)[NT / 8][4] = E4M3 ? sub[0] : acc, (&sum2)[NT / 8][4] = E4M3 ? sub[CH - 1] : acc;
            if (E4M3)
#pragma unroll
            for (int x = 0; x < CH; x++)
#pragma unroll
                for (int j = 0; j < JT; j++) sub[x][j][0] = sub[x][j][1] = sub[x][j][2] = sub[x][j][3] = 0.f;
#pragma unroll
            for (int kg = 0; kg < S::KW / 32; kg++) {
                uint32_t a[2][4];
                if (E4M3) {
                    const uint4 v = lds128(wa + kg * 512);
                    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                    for (int i = 0; i < 4; i++) {
                        a[i >> 1][2 * (i & 1)] = f16x2_of_e4m3x2(w[i]);
                        a[i >> 1][2 * (i & 1) + 1] = f16x2_of_e4m3x2(w[i] >> 16);
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < 2; i++) {
                        const uint4 v = lds128(wa + (2 * kg + i) * 512);
                        a[i][0] = v.x; a[i][1] = v.y; a[i][2] = v.z; a[i][3] = v.w;
                    }
                }
#pragma unroll
                for (int j = 0; j < JT; j++)
#pragma unroll
                    for (int pl = 0; pl < planes; pl++) {
                        const uint4 b = lds128(tb[j] + pl * pitch + kg * 64);
                        mma16<MT>(sum[j], a[0][0], a[0][1], a[0][2], a[0][3], b.x, b.y);
                        mma16<MT>(sum2[j], a[1][0], a[1][1], a[1][2], a[1][3], b.z, b.w);
                    }
            }
            if (E4M3)
#pragma unroll
            for (int x = 0; x < CH; x++)
#pragma unroll
                for (int j = 0; j < JT; j++)
#pragma unroll
                    for (int i = 0; i < 4; i++) acc[j][i] = fmaf(sub[x][j][i], i < 2 ? s0 : s1, acc[j][i]);
        }
        __syncwarp();
        if (lane == 0 && ok) mbar_arrive(empty + slot * 8);     // a warp that gave up empties no stage: the copies stop
        if (++slot == kStages) {
            slot = 0;
            parity ^= 1u;
        }
    };
    auto run_item = [&](auto second_, Cursor &c, int n) {       // an item's stages, for as many column blocks as it has tokens
#pragma unroll
        for (int j = 0; j < NT / 8; j++) acc[j][0] = acc[j][1] = acc[j][2] = acc[j][3] = 0.f;
        if (NT == 8 || n <= 8) {
            for (; c.stage < c.stages; c.stage++) multiply(second_, std::integral_constant<int, 1>(), c);
        } else if (NT == 16 || n <= 16) {
            for (; c.stage < c.stages; c.stage++) multiply(second_, std::integral_constant<int, (NT < 16 ? 1 : 2)>(), c);
        } else if (n <= 24) {
            for (; c.stage < c.stages; c.stage++) multiply(second_, std::integral_constant<int, (NT < 32 ? 1 : 3)>(), c);
        } else {
            for (; c.stage < c.stages; c.stage++) multiply(second_, std::integral_constant<int, NT / 8>(), c);
        }
    };
    // The warps' partial sums meet in `red` ([warp][row][token]), PASS tokens at a time, and all warps finish an item.  (Two buffers, two
    // halves of the warps finishing items in turn: 349 us instead of 339 for 128 tokens, e4m3, 7168 x 2048.)
    auto finish = [&](int n, auto &&each) {                     // each(first token, tokens) once their sums are in `red`
#pragma unroll
        for (int ps = 0; ps < NT / S::PASS; ps++) {
            if (ps * S::PASS >= n) break;
            bar<2, kMoeThreads>();                              // everyone has read what was there before
#pragma unroll
            for (int j = 0; j < S::PASS / 8; j++) {
                float *r = red + (warp * 16 + g) * S::PASS + j * 8 + 2 * q;
                const float (&v)[4] = acc[ps * (S::PASS / 8) + j];
                r[0] = v[0];
                r[1] = v[1];
                r[8 * S::PASS] = v[2];
                r[8 * S::PASS + 1] = v[3];
            }
            bar<1, kMoeThreads>();
            each(ps * S::PASS, min(S::PASS, n - ps * S::PASS));
        }
    };
    auto total = [&](int lwk, int tile, int row, int col) {     // row of the item's tile, token of the pass
        float v = 0.f;
        for (int i = 0; i < (1 << lwk); i++) v += red[(((tile << lwk) + i) * 16 + row) * S::PASS + col];
        return v;
    };

    Cursor c;
    for (begin(false, c); more(c); next(false, c)) {
        const int e = act[c.a], first = off[e] + c.c * NT, n = c.tokens;
        run_item(std::false_type(), c, n);
        constexpr int FR = 8 * S::TM;                           // hidden units of the item
        float g2 = 0.f, u2 = 0.f;
        if (E4M3) {
            g2 = __ldg(A.row_max + weights_of(e) * 2);
            u2 = __ldg(A.row_max + weights_of(e) * 2 + 1);
        }
        finish(n, [&](int t0, int nt) {
            for (int i = tid; i < FR * nt; i += kMoeThreads) {
                const int col = i / FR, fr = i - col * FR, f = c.tile * 8 + fr;
                if (fr >= c.n * 8) continue;
                const int p = list[first + t0 + col];
                float gate = total(c.lwk, fr >> 3, fr & 7, col), up = total(c.lwk, fr >> 3, (fr & 7) + 8, col);
                if (E4M3) {
                    const float xs = A.xh_scale[p / C];
                    gate *= xs;
                    up *= xs;
                }
                const float h = gate / (1.f + expf(-gate)) * up;
                if (E4M3) {
                    A.hop[(size_t)p * A.Fk + f] = (uint16_t)f16x2_of(h * exp2i(-hidden_exponent(A.x_norm2[p / C], g2, u2)), 0.f);
                } else {
                    const uint32_t hi = bf16x2_of(h, 0.f) & 0xFFFFu;
                    uint16_t *dst = A.hop + (size_t)p * 2 * A.Fk + f;
                    dst[0] = (uint16_t)hi;
                    dst[A.Fk] = (uint16_t)bf16x2_of(h - __uint_as_float(hi << 16), 0.f);
                }
            }
        });
        if (c.tile + c.n == A.f_tiles) {                // zeros behind F
            const int pad = A.Fk - A.Fp, rows = n * S::PLANES;
            for (int i = tid; i < pad * rows; i += kMoeThreads) {
                const int r = i / pad;
                A.hop[((size_t)list[first + r / S::PLANES] * S::PLANES + r % S::PLANES) * A.Fk + A.Fp + i - r * pad] = 0;
            }
        }
    }

    // ---- all hidden activations are there (or a wait ran out, which the last meeting hears of)
    if (!ok && lane == 0) wait_ran_out(A);
    meet<3, kMoeThreads>(A, round, &meet_ok);

    // ---- second product
    for (begin(true, c); more(c); next(true, c)) {
        const int e = act[c.a], first = off[e] + c.c * NT, n = c.tokens;
        run_item(std::true_type(), c, n);
        constexpr int HR = 16 * S::TM;
        float g2 = 0.f, u2 = 0.f;
        if (E4M3) {
            g2 = __ldg(A.row_max + weights_of(e) * 2);
            u2 = __ldg(A.row_max + weights_of(e) * 2 + 1);
        }
        finish(n, [&](int t0, int nt) {
            for (int i = tid; i < HR * nt; i += kMoeThreads) {
                const int col = i / HR, row = i - col * HR;
                if (row >= c.n * 16) continue;
                const int p = list[first + t0 + col];
                float v = total(c.lwk, row >> 4, row & 15, col);
                if (E4M3) v *= exp2i(hidden_exponent(A.x_norm2[p / C], g2, u2));
                A.y[(size_t)p * H + c.tile * 16 + row] = v;
            }
        });
    }
    if (!ok && lane == 0) wait_ran_out(A);
    if (!meet<3, kMoeThreads>(A, round, &meet_ok)) return spoil();

    // ---- a token's parts, in the order of its choices
    const int quads = H / 4;
    for (int i = blockIdx.x * kMoeThreads + tid; i < T * quads; i += grid * kMoeThreads) {
        const int t = i / quads, h = (i - t * quads) * 4;
        float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
        for (unsigned rest = local[t]; rest; rest &= rest - 1u) {
            const int j = __ffs(rest) - 1;
            const float w = j < K ? A.weights[t * K + j] : 1.f;
            const float4 v = *reinterpret_cast<const float4 *>(A.y + (size_t)(t * C + j) * H + h);
            s.x = fmaf(w, v.x, s.x);
            s.y = fmaf(w, v.y, s.y);
            s.z = fmaf(w, v.z, s.z);
            s.w = fmaf(w, v.w, s.w);
        }
        *reinterpret_cast<uint2 *>(A.out + (size_t)t * H + h) = make_uint2(bf16x2_of(s.x, s.y), bf16x2_of(s.z, s.w));
    }
}

// ------------------------------------------------------------------ host
static bool moe_ok(const pf_moe_t *m)
{
    return m && m->H >= 16 && m->H % 16 == 0 && m->H <= (1 << 20) && m->F >= 1 && m->F <= (1 << 20) && m->n_experts >= 1 &&
           m->n_experts <= PF_MOE_MAX_EXPERTS && m->first >= 0 && m->n_local >= 0 && m->n_local <= m->n_experts &&
           m->first <= m->n_experts - m->n_local && m->n_shared >= 0 && m->n_shared <= PF_MOE_MAX_CHOICES && m->top_k >= 1 && m->top_k <= m->n_experts &&
           m->top_k + m->n_shared <= PF_MOE_MAX_CHOICES && m->n_local + m->n_shared >= 1 &&
           (m->wtype == PF_DT_BF16 || m->wtype == PF_DT_E4M3);
}
static void moe_layout(const pf_moe_t *m, MoeArgs &a)
{
    const int kw = m->wtype == PF_DT_E4M3 ? 128 : 64;
    a.m = *m;
    a.choices = m->top_k + m->n_shared;
    a.n_sets = m->n_local + m->n_shared;
    a.f_tiles = (m->F + 7) / 8;
    a.h_tiles = m->H / 16;
    a.ks_up = (m->H + kw - 1) / kw;
    a.Fp = a.f_tiles * 8;
    a.ks_down = (a.Fp + kw - 1) / kw;
    a.Hk = a.ks_up * kw;
    a.Fk = a.ks_down * kw;
    a.down_at = (size_t)a.f_tiles * a.ks_up * kSliceBytes;
    a.set_bytes = a.down_at + (size_t)a.h_tiles * a.ks_down * kSliceBytes;
    const size_t fb = (m->F + 127) / 128, hb = (m->H + 127) / 128, n = a.n_sets;
    a.n_up_scales = a.n_down_scales = fb * hb;
    a.packed_bytes = a.set_bytes * n;
    if (m->wtype == PF_DT_E4M3) a.packed_bytes += (n * (2 * a.n_up_scales + a.n_down_scales) + 2 * n) * sizeof(float);
}
static void moe_point(MoeArgs &a, const void *packed)
{
    a.packed = (const uint8_t *)packed;
    a.gs = (const float *)(a.packed + a.set_bytes * (size_t)a.n_sets);
    a.us = a.gs + a.n_up_scales * a.n_sets;
    a.ds = a.us + a.n_up_scales * a.n_sets;
    a.row_max = a.ds + a.n_down_scales * a.n_sets;
}
static size_t take(size_t &at, size_t bytes)
{
    const size_t here = at;
    at += (bytes + 255) & ~(size_t)255;
    return here;
}
// tokens of a block of the router: whole column blocks of the matrix instruction
static int route_tokens(int T) { return T <= 8 ? 8 : T <= 16 ? 16 : 32; }
// carves the workspace; sms: number of SMs (sizes the router's grid).  Returns its size; `base` may be NULL.
static size_t moe_carve(MoeArgs &a, int T, int sms, uint8_t *base)
{
    const pf_moe_t &m = a.m;
    const bool e4m3 = m.wtype == PF_DT_E4M3;
    a.T = T;
    a.e_tiles = (m.n_experts + 15) / 16;
    const int tokens = route_tokens(T);
    a.t_chunks = (T + tokens - 1) / tokens;
    // router: about one block per SM, at least 256 columns (32 per warp) for each
    const int most = (m.H + 255) / 256, want = sms / (a.e_tiles * a.t_chunks);
    a.h_splits = want < 1 ? 1 : (want < most ? want : most);
    if (a.h_splits > kRouteSplits) a.h_splits = kRouteSplits;
    const size_t pairs = (size_t)T * a.choices;
    size_t at = 0;
    a.ctl = (unsigned *)(base + take(at, 256));
    a.logits = (float *)(base + take(at, (size_t)a.h_splits * T * m.n_experts * 4));
    a.xh = (uint16_t *)(base + take(at, (size_t)T * a.Hk * 2));
    a.xh_scale = (float *)(base + take(at, (size_t)T * 4));
    a.x_norm2 = (float *)(base + take(at, (size_t)T * 4));
    a.hop = (uint16_t *)(base + take(at, pairs * a.Fk * 2 * (e4m3 ? 1 : 2)));
    a.y = (float *)(base + take(at, pairs * m.H * 4));
    return at;
}

template <bool E4M3, int NT, int STAGES_>
static int moe_launch(const MoeArgs &a, int device, int sms, cudaStream_t st)
{
    using S = MoeShape<E4M3, NT, STAGES_>;
    const size_t lists = ((size_t)a.n_sets * 4 + 1) * 4 + ((size_t)a.T * a.choices + 1) / 2 * 4 + (size_t)a.T * 4, smem = S::FIXED + lists;
    // one stage less where the lists of pairs and experts do not leave room for it; the shortest ring fits with the longest lists
    if constexpr (STAGES_ > 3)
        if (smem > kMoeSmem) return moe_launch<E4M3, NT, STAGES_ - 1>(a, device, sms, st);
    PF_CUDA_TRY(ensure_dynamic_smem((const void *)moe_kernel<E4M3, NT, STAGES_>, device, smem), "moe_kernel shared memory");
    const int n_route = a.e_tiles * a.h_splits * a.t_chunks + a.T;
    switch (route_tokens(a.T)) {
    case 8: moe_route_kernel<E4M3, 1><<<n_route, kRouteThreads, 0, st>>>(a); break;
    case 16: moe_route_kernel<E4M3, 2><<<n_route, kRouteThreads, 0, st>>>(a); break;
    default: moe_route_kernel<E4M3, 4><<<n_route, kRouteThreads, 0, st>>>(a); break;
    }
    PF_CUDA_TRY(cudaGetLastError(), "moe_route_kernel launch");
    count_launch();
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(sms);
    cfg.blockDim = dim3(kMoeBlock);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeCooperative;
    at[0].val.cooperative = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    PF_CUDA_TRY(cudaLaunchKernelEx(&cfg, moe_kernel<E4M3, NT, STAGES_>, a), "moe_kernel launch");
    count_launch();
    return PF_OK;
}

}  // namespace pf

using namespace pf;

extern "C" size_t pf_moe_packed_bytes(const pf_moe_t *m)
{
    if (!moe_ok(m)) return 0;
    MoeArgs a;
    moe_layout(m, a);
    return a.packed_bytes;
}

extern "C" int pf_moe_pack(const pf_moe_t *m, const void *d_gate, const void *d_up, const void *d_down, const float *d_gate_scale,
                           const float *d_up_scale, const float *d_down_scale, void *d_packed, void *stream)
{
    if (!moe_ok(m) || !d_gate || !d_up || !d_down || !d_packed) return PF_EINVAL;
    if (!aligned16(d_gate) || !aligned16(d_up) || !aligned16(d_down) || ((uintptr_t)d_packed & 255)) return PF_EINVAL;
    const bool e4m3 = m->wtype == PF_DT_E4M3;
    if (e4m3 ? (!d_gate_scale || !d_up_scale || !d_down_scale) : (d_gate_scale || d_up_scale || d_down_scale)) return PF_EINVAL;
    if ((uintptr_t)d_gate_scale % 4 || (uintptr_t)d_up_scale % 4 || (uintptr_t)d_down_scale % 4) return PF_EINVAL;
    MoeArgs a;
    moe_layout(m, a);
    moe_point(a, d_packed);
    const size_t units = a.set_bytes * (size_t)a.n_sets / 16, n = a.n_sets;
    const unsigned grid = (unsigned)((units + 255) / 256 < 65536 ? (units + 255) / 256 : 65536);
    cudaStream_t st = (cudaStream_t)stream;
    if (!e4m3) {
        moe_pack_kernel<false><<<grid, 256, 0, st>>>(*m, a.n_sets, a.f_tiles, a.ks_up, a.ks_down, a.set_bytes, a.down_at, (const uint8_t *)d_gate,
                                                     (const uint8_t *)d_up, (const uint8_t *)d_down, (uint8_t *)d_packed);
        PF_CUDA_TRY(cudaGetLastError(), "moe_pack_kernel launch");
        count_launch();
        return PF_OK;
    }
    PF_CUDA_TRY(cudaMemcpyAsync((void *)a.gs, d_gate_scale, n * a.n_up_scales * 4, cudaMemcpyDeviceToDevice, st), "scale copy");
    PF_CUDA_TRY(cudaMemcpyAsync((void *)a.us, d_up_scale, n * a.n_up_scales * 4, cudaMemcpyDeviceToDevice, st), "scale copy");
    PF_CUDA_TRY(cudaMemcpyAsync((void *)a.ds, d_down_scale, n * a.n_down_scales * 4, cudaMemcpyDeviceToDevice, st), "scale copy");
    PF_CUDA_TRY(cudaMemsetAsync((void *)a.row_max, 0, n * 2 * 4, st), "row norms");
    moe_pack_kernel<true><<<grid, 256, 0, st>>>(*m, a.n_sets, a.f_tiles, a.ks_up, a.ks_down, a.set_bytes, a.down_at, (const uint8_t *)d_gate,
                                                (const uint8_t *)d_up, (const uint8_t *)d_down, (uint8_t *)d_packed);
    PF_CUDA_TRY(cudaGetLastError(), "moe_pack_kernel launch");
    moe_block_norm_kernel<<<(unsigned)(n * ((m->F + 127) / 128)), 256, 0, st>>>(*m, (const uint8_t *)d_gate, (const uint8_t *)d_up, a.gs, (float *)a.us,
                                                                                (float *)a.ds, (float *)a.row_max);
    PF_CUDA_TRY(cudaGetLastError(), "moe_block_norm_kernel launch");
    count_launch();
    count_launch();
    return PF_OK;
}

extern "C" size_t pf_moe_workspace(const pf_moe_t *m, int32_t T)
{
    int device, sms;
    if (!moe_ok(m) || T <= 0 || T > PF_MOE_MAX_TOKENS || current_sm_count(&device, &sms) != PF_OK) return 256;
    MoeArgs a;
    moe_layout(m, a);
    return moe_carve(a, T, sms, nullptr);
}

extern "C" int pf_moe_forward(const pf_moe_t *m, int32_t T, const void *d_x, int64_t x_stride, const uint8_t *d_xq, const float *d_xscale,
                              const void *d_router, const void *d_packed, void *d_out, int32_t *d_ids, float *d_weights, int32_t *d_status,
                              void *d_workspace, size_t workspace_bytes, void *stream)
{
    if (!moe_ok(m)) return PF_EINVAL;
    if (T < 0 || T > PF_MOE_MAX_TOKENS) return PF_ERANGE;
    if (T == 0) return PF_OK;
    const bool e4m3 = m->wtype == PF_DT_E4M3;
    if (!d_x || !d_router || !d_packed || !d_out || !d_ids || !d_weights) return PF_EINVAL;
    if (!aligned16(d_x) || x_stride < m->H || x_stride % 8 || !aligned16(d_router) || ((uintptr_t)d_packed & 255) || (uintptr_t)d_out % 8) return PF_EINVAL;
    if ((uintptr_t)d_ids % 4 || (uintptr_t)d_weights % 4 || (uintptr_t)d_status % 4) return PF_EINVAL;
    if ((d_xq != nullptr) != (d_xscale != nullptr) || (d_xq && (!e4m3 || (uintptr_t)d_xq % 8 || (uintptr_t)d_xscale % 4))) return PF_EINVAL;
    int device, sms;
    if (int rc = current_sm_count(&device, &sms)) return rc;
    MoeArgs a;
    moe_layout(m, a);
    if (!d_workspace || ((uintptr_t)d_workspace & 255) != 0 || workspace_bytes < moe_carve(a, T, sms, (uint8_t *)d_workspace)) return PF_EWORKSPACE;
    a.x = (const uint16_t *)d_x; a.xs = x_stride; a.xq = d_xq; a.xscale = d_xscale;
    a.router = (const uint16_t *)d_router;
    moe_point(a, d_packed);
    a.out = (uint16_t *)d_out; a.ids = d_ids; a.weights = d_weights; a.status = d_status;
    a.meet_limit = g_meet_limit; a.meet_missing = g_meet_missing;
    cudaStream_t st = (cudaStream_t)stream;
    // Tokens an item takes at most: 8 (a column block of the matrix instruction) where no expert can have more, then 16, and 32 with more
    // than 8 an expert on average: a stage's token rows take room from the ring, and an expert with more tokens than an item is read again,
    // mostly from the L2.  Measured with 16 and 32 (us) on either side of the rule's border.  6 + 2 of 64 experts, 4096 x 1408, border at 85 tokens: e4m3
    // 24 tokens 216, 224; 64: 264, 265; 96: 310, 308; 256: 619, 519; bf16 24: 341, 347; 256: 850, 658.  8 + 1 of 256, 32 here, 7168 x 2048, border
    // 256: e4m3 32: 200, 222; 128: 328, 328; 256: 445, 433.  8 + 1 of 128, 32 here, 5120 x 1536, border 128: e4m3 32: 152, 157; 192: 277, 259.  2 of
    // 8, 1024 x 2816, border 32: e4m3 24: 39, 37; 48: 48, 45; 64: 55, 55; 256: 116, 113; bf16 64: 63, 76, the one place where it costs; 192: 116, 103.
    if (T <= 8) return e4m3 ? moe_launch<true, 8, 5>(a, device, sms, st) : moe_launch<false, 8, 5>(a, device, sms, st);
    if ((long long)T * m->top_k <= 8ll * m->n_experts)
        return e4m3 ? moe_launch<true, 16, 5>(a, device, sms, st) : moe_launch<false, 16, 4>(a, device, sms, st);
    return e4m3 ? moe_launch<true, 32, 4>(a, device, sms, st) : moe_launch<false, 32, 4>(a, device, sms, st);
}

extern "C" int pf_moe_meeting(uint32_t polls, uint32_t missing)
{
    if (polls > kMeetLimit || missing > 1) return PF_ERANGE;
    g_meet_limit = polls ? polls : kMeetLimit;
    g_meet_missing = missing;
    return PF_OK;
}
