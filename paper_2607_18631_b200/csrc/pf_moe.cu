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
//    meet, and add up each token's parts in a fixed order.  One warp of a block copies (bulk copies into a ring of a few
//    stages, completion on an mbarrier), eight multiply; a multiplying warp waits for nothing but its stage.  While the blocks
//    meet, the ring already fills with the down matrices' first stages, which do not depend on the meeting.
//  - 8 gate rows and the same 8 up rows form one 16-row tile: a lane's accumulators hold both factors of its products.
// Sums are fp32.  bf16 weights multiply bf16 tokens; the hidden activations (fp32) enter the second product as the
// sum of two bf16 numbers (16 bits of mantissa).  e4m3 weights are widened to fp16, which is exact; tokens and hidden activations
// are scaled by a power of two per row and rounded to fp16 (11 bits); a weight block's scale is applied to the fp32 sum of
// its 128 columns.  Two products in bf16 or fp16 cost less than half of the matrix rate at full HBM speed for 32 tokens a tile.
#include "pf_ops.cuh"

namespace pf {

constexpr int kMoeWarps = 8, kMoeThreads = kMoeWarps * 32;   // that multiply
constexpr int kMoeBlock = kMoeThreads + 32;                  // and one warp that copies
constexpr int kSliceBytes = 2048;          // 16 rows x KW elements, KW = 64 (bf16) or 128 (e4m3)
constexpr unsigned kMeetLimit = 1u << 21;  // polls of a meeting before it gives up (a poll takes about a microsecond)
constexpr unsigned kRingLimit = 1u << 20;  // waits of up to a microsecond for a stage before they give up

struct MoeArgs {
    pf_moe_t m;
    int T, choices;                        // choices = top_k + n_shared: a token's (token, expert) pairs
    int n_sets;                            // n_local + n_shared
    int f_tiles, h_tiles, ks_up, ks_down;  // row tiles and column slices of the packed matrices
    int Fp;                                // 8 * f_tiles
    int Hk, Fk;                            // H and F rounded up to whole slices: row lengths of the products' inputs
    size_t set_bytes, down_at;             // packed bytes per expert, offset of its down part
    const uint16_t *x;
    int64_t xs;
    const uint8_t *xq;
    const float *xscale;
    const uint16_t *router;
    const uint8_t *packed;
    const float *gs, *us, *ds;
    uint16_t *out;
    int32_t *ids;
    float *weights;
    int32_t *status;
    // workspace
    unsigned *ctl;                         // [0] arrivals, [1] a meeting failed
    unsigned *h_max;                       // [pairs] bits of max |h| (e4m3 weights)
    float *logits;                         // [h_splits][T][n_experts]
    uint16_t *xh;                          // [T][Hk] tokens, zero behind H: bf16, or fp16 times a power of two (e4m3 weights)
    float *xh_scale;                       // [T] power of two
    float *h32;                            // [pairs][Fp] (e4m3 weights)
    uint16_t *hop;                         // zero behind F; bf16: [pairs][2][Fk] high and low parts; e4m3: [pairs][Fk] fp16
    float *y;                              // [pairs][H]
    int h_splits, e_tiles, t_chunks;       // router grid
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

// ------------------------------------------------------------------ router logits, tokens as fp16
// exponent that brings a row's largest magnitude into [2^13, 2^14): what is 2^-27 of it keeps 11 bits in fp16
__device__ __forceinline__ int fp16_exponent(float amax)
{
    const int e = (amax > 0.f && amax < INFINITY) ? (int)(__float_as_uint(amax) >> 23) - 127 : 0;
    return max(-100, e) - 13;
}
__device__ __forceinline__ float exp2i(int e) { return __uint_as_float((uint32_t)(min(127, max(-126, e)) + 127) << 23); }

constexpr int kRouteTokens = 32, kRouteSplits = 8;
template <bool E4M3>
__global__ void __launch_bounds__(kMoeThreads) moe_route_kernel(const __grid_constant__ MoeArgs A)
{
    __shared__ float red[kMoeWarps][16][kRouteTokens + 1];
    __shared__ float part[kMoeWarps];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, q = lane & 3;
    const int n_gemm = A.e_tiles * A.h_splits * A.t_chunks;
    const int H = A.m.H, E = A.m.n_experts;
    if (blockIdx.x == 0) {
        if (tid < 2) A.ctl[tid] = 0u;
        if (tid == 0 && A.status) *A.status = 0;
    }
    if ((int)blockIdx.x < n_gemm) {
        const int et = blockIdx.x % A.e_tiles, r = blockIdx.x / A.e_tiles, hs = r % A.h_splits, tc = r / A.h_splits;
        const int groups = (H + 31) / 32;                    // 32 columns at a time
        const int k_lo = (int)((long long)groups * hs / A.h_splits), k_hi = (int)((long long)groups * (hs + 1) / A.h_splits);
        const int t0 = tc * kRouteTokens, n = min(kRouteTokens, A.T - t0);
        float c[kRouteTokens / 8][4];
#pragma unroll
        for (int j = 0; j < kRouteTokens / 8; j++) c[j][0] = c[j][1] = c[j][2] = c[j][3] = 0.f;
        const int r0 = et * 16 + g, r1 = r0 + 8;
#pragma unroll 4
        for (int kg = k_lo + warp; kg < k_hi; kg += kMoeWarps) {
            const int k = kg * 32 + q * 8;
            uint4 a = make_uint4(0, 0, 0, 0), b = a;
            if (k < H) {
                if (r0 < E) a = __ldg(reinterpret_cast<const uint4 *>(A.router + (int64_t)r0 * H + k));
                if (r1 < E) b = __ldg(reinterpret_cast<const uint4 *>(A.router + (int64_t)r1 * H + k));
            }
#pragma unroll
            for (int j = 0; j < kRouteTokens / 8; j++) {
                if (j * 8 >= n) break;
                uint4 x = make_uint4(0, 0, 0, 0);
                if (k < H && j * 8 + g < n) x = __ldg(reinterpret_cast<const uint4 *>(A.x + (int64_t)(t0 + j * 8 + g) * A.xs + k));
                mma16<Bf16>(c[j], a.x, b.x, a.y, b.y, x.x, x.y);
                mma16<Bf16>(c[j], a.z, b.z, a.w, b.w, x.z, x.w);
            }
        }
#pragma unroll
        for (int j = 0; j < kRouteTokens / 8; j++) {
            red[warp][g][j * 8 + 2 * q] = c[j][0];
            red[warp][g][j * 8 + 2 * q + 1] = c[j][1];
            red[warp][g + 8][j * 8 + 2 * q] = c[j][2];
            red[warp][g + 8][j * 8 + 2 * q + 1] = c[j][3];
        }
        __syncthreads();
        for (int i = tid; i < 16 * n; i += kMoeThreads) {
            const int e = i & 15, t = i >> 4;
            float s = 0.f;
#pragma unroll
            for (int wv = 0; wv < kMoeWarps; wv++) s += red[wv][e][t];
            if (et * 16 + e < E) A.logits[((int64_t)hs * A.T + t0 + t) * E + et * 16 + e] = s;
        }
        return;
    }
    const int t = blockIdx.x - n_gemm;
    if constexpr (!E4M3) {
        for (int k = tid * 8; k < A.Hk; k += kMoeThreads * 8)
            *reinterpret_cast<uint4 *>(A.xh + (size_t)t * A.Hk + k) =
                k < H ? *reinterpret_cast<const uint4 *>(A.x + (int64_t)t * A.xs + k) : make_uint4(0, 0, 0, 0);
    } else {
    // token t as fp16 times a power of two; its pairs' maxima start at zero
    for (int j = tid; j < A.choices; j += kMoeThreads) A.h_max[t * A.choices + j] = 0u;
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
    float m = 0.f;
    for (int k = tid * 8; k < H; k += kMoeThreads * 8) {
        float v[8];
        value8(k, v);
#pragma unroll
        for (int i = 0; i < 8; i++) m = fmaxf(m, fabsf(v[i]));
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, o));
    if (lane == 0) part[warp] = m;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kMoeWarps; i++) m = fmaxf(m, part[i]);
    const int e = fp16_exponent(m);
    const float down = exp2i(-e);
    if (tid == 0) A.xh_scale[t] = exp2i(e);
    for (int k = tid * 8; k < A.Hk; k += kMoeThreads * 8) {
        float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (k < H) value8(k, v);
        *reinterpret_cast<uint4 *>(A.xh + (size_t)t * A.Hk + k) =
            make_uint4(f16x2_of(v[0] * down, v[1] * down), f16x2_of(v[2] * down, v[3] * down), f16x2_of(v[4] * down, v[5] * down),
                       f16x2_of(v[6] * down, v[7] * down));
    }
    }
}

// ------------------------------------------------------------------ the layer
// All blocks of the (cooperative) grid meet, each represented by one thread; false where the wait ran out.
__device__ __forceinline__ bool arrive_and_poll(unsigned *ctl, unsigned round, bool arrive)
{
    if (arrive) {
        __threadfence();
        atomicAdd(ctl, 1u);
    }
    unsigned seen = 0, polls = 0;
    do {
        asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(seen) : "l"(ctl) : "memory");
    } while (seen < round && ++polls < kMeetLimit);
    __threadfence();
    return seen >= round;
}
template <int ID, int THREADS> __device__ __forceinline__ void bar()
{
    asm volatile("bar.sync %0, %1;" ::"n"(ID), "n"(THREADS) : "memory");
}
template <int ID, int THREADS> __device__ __forceinline__ void bar_arrive()
{
    asm volatile("bar.arrive %0, %1;" ::"n"(ID), "n"(THREADS) : "memory");
}
// the multiplying threads (or, before the roles part, all threads) of the block meet the other blocks'
template <int ID, int THREADS>
__device__ __forceinline__ bool meet(unsigned *ctl, unsigned &round, int *ok)
{
    round += gridDim.x;
    asm volatile("fence.proxy.async;" ::: "memory");      // what was written is read by bulk copies
    bar<ID, THREADS>();
    if (threadIdx.x == 0) *ok = arrive_and_poll(ctl, round, true);
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

template <bool E4M3, int WM, int WK, int MI, int NT>
struct MoeShape {
    static constexpr int KW = E4M3 ? 128 : 64;
    static constexpr int PLANES = E4M3 ? 1 : 2;               // of the hidden activations
    static constexpr int TM = WM * MI;                        // row tiles of an item
    static constexpr int A_BYTES = kMoeWarps * MI * kSliceBytes;
    static constexpr int PITCH = WK * KW * 2 + 64;            // a token row; 64 mod 128: two rows' quarters use all banks
    static constexpr int B_BYTES = NT * PLANES * PITCH;
    static constexpr int STAGE = A_BYTES + B_BYTES;
    static constexpr int RED = WK * TM * 16 * NT * 4;         // one item's partial sums
    static constexpr int BUFS = RED > 16384 ? 1 : 2;
    static constexpr int STAGES = NT == 8 ? 4 : 3;            // what 227 KB hold beside the partial sums and the longest list of pairs
    static constexpr int FIXED = STAGES * STAGE + BUFS * RED;
    static_assert(WM * WK == kMoeWarps, "one slice per warp and stage");
};

template <bool E4M3, int WM, int WK, int MI, int NT>
__global__ void __launch_bounds__(kMoeBlock, 1) moe_kernel(const __grid_constant__ MoeArgs A)
{
    using S = MoeShape<E4M3, WM, WK, MI, NT>;
    using MT = typename std::conditional<E4M3, F16, Bf16>::type;
    constexpr int kStages = S::STAGES;
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ __align__(8) uint64_t bars[2 * kStages];
    __shared__ int meet_ok;
    __shared__ int n_active_s;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, q = lane & 3;
    const int wm = warp / WK, wk = warp % WK;
    const int T = A.T, K = A.m.top_k, C = A.choices, E = A.m.n_experts, H = A.m.H;
    uint8_t *ring_p = smem;
    const uint32_t ring = smem_addr(ring_p);
    float *red = reinterpret_cast<float *>(smem + kStages * S::STAGE);
    int *cnt = reinterpret_cast<int *>(smem + S::FIXED);      // [n_sets] tokens per expert, then running offsets
    int *off = cnt + A.n_sets;                                                       // [n_sets] first list entry
    int *act = off + A.n_sets;                                                       // [n_sets] experts with tokens
    int *cum = act + A.n_sets;                                                       // [n_sets + 1] token chunks before an active expert
    uint16_t *list = reinterpret_cast<uint16_t *>(cum + A.n_sets + 1);               // [T * C] pairs by expert
    unsigned round = 0;

    // ---- the choice: one warp per token.  For few tokens each block makes all of it by itself, which saves a meeting.
    const bool by_itself = T <= 2 * kMoeWarps;
    if (tid == 0) {
        for (int i = 0; i < kStages; i++) {
            mbar_init(smem_addr(bars + i), 2);                   // full: the weights' and the tokens' announcements, and their bytes
            mbar_init(smem_addr(bars + kStages + i), kMoeWarps);   // empty: the multiplying warps
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp < kMoeWarps)
    for (int t = by_itself ? warp : warp * (int)gridDim.x + (int)blockIdx.x; t < T; t += by_itself ? kMoeWarps : kMoeWarps * (int)gridDim.x) {
        uint32_t key[PF_MOE_MAX_EXPERTS / 32];
#pragma unroll
        for (int i = 0; i < PF_MOE_MAX_EXPERTS / 32; i++) {
            key[i] = 0u;
            const int e = i * 32 + lane;
            if (i * 32 < E && e < E) {
                float v[kRouteSplits], s = 0.f;                 // all in flight, added in a fixed order
#pragma unroll
                for (int hs = 0; hs < kRouteSplits; hs++) v[hs] = hs < A.h_splits ? A.logits[((int64_t)hs * T + t) * E + e] : 0.f;
#pragma unroll
                for (int hs = 0; hs < kRouteSplits; hs++) s += v[hs];
                const uint32_t b = s == s ? __float_as_uint(s) : 0xFF800000u;
                key[i] = (b >> 31) ? ~b : (b | 0x80000000u);      // order of the floats; 0 = taken
            }
        }
        float top = 0.f, sum = 0.f, mine = 0.f;
        int my_id = 0;
        for (int j = 0; j < K; j++) {
            uint32_t best = 0u;
#pragma unroll
            for (int i = 0; i < PF_MOE_MAX_EXPERTS / 32; i++) best = max(best, key[i]);
            const uint32_t all = __reduce_max_sync(0xFFFFFFFFu, best);
            uint32_t at = 0xFFFFFFFFu;
#pragma unroll
            for (int i = PF_MOE_MAX_EXPERTS / 32 - 1; i >= 0; i--)
                if (key[i] == all) at = i * 32 + lane;
            at = __reduce_min_sync(0xFFFFFFFFu, at);
#pragma unroll
            for (int i = 0; i < PF_MOE_MAX_EXPERTS / 32; i++)
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
            if (by_itself) {
                reinterpret_cast<int *>(red)[t * K + lane] = my_id;
            }
            if (!by_itself || blockIdx.x == 0) {
                A.ids[t * K + lane] = my_id;
                A.weights[t * K + lane] = mine / sum;
            }
        }
    }
    if (by_itself) __syncthreads();
    else if (!meet<0, kMoeBlock>(A.ctl, round, &meet_ok)) {
        if (tid == 0 && A.status) *A.status = 1;
        return;
    }

    // ---- pairs by expert
    for (int i = tid; i < A.n_sets; i += kMoeBlock) cnt[i] = 0;
    __syncthreads();
    auto set_of = [&](int p) {               // expert of pair p on this GPU, -1 if it lives elsewhere
        const int t = p / C, j = p - t * C;
        if (j >= K) return A.m.n_local + j - K;
        const int e = (by_itself ? reinterpret_cast<const int *>(red)[t * K + j] : A.ids[t * K + j]) - A.m.first;
        return e >= 0 && e < A.m.n_local ? e : -1;
    };
    for (int p = tid; p < T * C; p += kMoeBlock) {
        const int s = set_of(p);
        if (s >= 0) atomicAdd(cnt + s, 1);
    }
    __syncthreads();
    if (warp == 0) {                         // offsets, active experts, chunks: a scan by one warp
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
            if (i < A.n_sets) off[i] = o + so - n;
            if (n > 0) {
                const int at = a + __popc(live & ((1u << lane) - 1u));
                act[at] = i;
                cum[at] = c + sc - ch;
            }
            o += __shfl_sync(0xFFFFFFFFu, so, 31);
            c += __shfl_sync(0xFFFFFFFFu, sc, 31);
            a += __popc(live);
        }
        if (lane == 0) {
            cum[a] = c;
            n_active_s = a;
        }
    }
    __syncthreads();
    // All blocks need the same order (a block takes some of an expert's chunks), so what the atomics dealt out in any order is
    // ranked by pair number within each expert.
    for (int i = tid; i < A.n_sets; i += kMoeBlock) cnt[i] = off[i];
    __syncthreads();
    uint16_t *dealt = reinterpret_cast<uint16_t *>(ring_p), *set_at = dealt + T * C;      // the ring is not in use yet
    for (int p = tid; p < T * C; p += kMoeBlock) {
        const int s = set_of(p);
        if (s < 0) continue;
        const int at = atomicAdd(cnt + s, 1);
        dealt[at] = (uint16_t)p;
        set_at[at] = (uint16_t)s;
    }
    __syncthreads();                         // now cnt[s] is the end of expert s's pairs
    for (int i = tid; i < (n_active_s ? cnt[act[n_active_s - 1]] : 0); i += kMoeBlock) {
        const int s = set_at[i], p = dealt[i];
        int rank = off[s];
        for (int k = off[s]; k < cnt[s]; k++) rank += dealt[k] < p;
        list[rank] = (uint16_t)p;
    }
    __syncthreads();
    const int n_active = n_active_s, n_chunks = cum[n_active];

    // ---- row tiles: item = (expert, group of WM row tiles, chunk of NT tokens), chunks fastest so that a tile's second reading hits the L2
    struct Cursor {
        int item, a, r, c, chunks, stage;
        __device__ __forceinline__ void at(int i, int groups, const int *cum, int n_active)
        {
            item = i;
            while (a < n_active && i >= groups * cum[a + 1]) a++;
            if (a >= n_active) return;
            chunks = cum[a + 1] - cum[a];
            const int rest = i - groups * cum[a];
            r = rest / chunks;
            c = rest - r * chunks;
        }
    };
    const int groups1 = (A.f_tiles + S::TM - 1) / S::TM, groups2 = (A.h_tiles + S::TM - 1) / S::TM;
    const int stages1 = (A.ks_up + WK - 1) / WK, stages2 = (A.ks_down + WK - 1) / WK;
    const int items1 = groups1 * n_chunks, items2 = groups2 * n_chunks;
    const int grid = gridDim.x;

    // ---- the stream: positions 0 .. n1 - 1 are stages of the first product, n1 .. n1 + n2 - 1 of the second; position p uses
    // ring slot p % kStages
    const int mine1 = items1 > (int)blockIdx.x ? (items1 - (int)blockIdx.x + grid - 1) / grid : 0;
    const int mine2 = items2 > (int)blockIdx.x ? (items2 - (int)blockIdx.x + grid - 1) / grid : 0;
    const int n1 = mine1 * stages1, n2 = mine2 * stages2;
    const uint32_t full = smem_addr(bars), empty = full + kStages * 8;
    asm volatile("fence.proxy.async;" ::: "memory");            // the ring held `dealt`: bulk copies write it from here on
    __syncthreads();                                            // barriers are set up; `red` held the ids

    if (warp == kMoeWarps) {                                    // ================= the copying warp
        // What a stage costs this warp bounds the whole stream, so everything that belongs to an item is worked out once: where its
        // tiles begin, and for each lane its (up to ROWS) token rows.
        constexpr int ROWS = (NT * S::PLANES + 31) / 32;
        struct Feed {
            Cursor c;
            const uint8_t *weights;
            const uint16_t *row[ROWS];
            int tiles, rows;
        };
        auto set_up = [&](bool second, Feed &f) {
            const Cursor &c = f.c;
            if (c.a >= n_active) return;
            const int e = act[c.a], first = off[e] + c.c * NT, n = min(NT, cnt[e] - first);
            f.weights = A.packed + (size_t)e * A.set_bytes + (second ? A.down_at : 0) + (size_t)(c.r * S::TM) * (second ? A.ks_down : A.ks_up) * kSliceBytes;
            f.tiles = min(S::TM, (second ? A.h_tiles : A.f_tiles) - c.r * S::TM);
            f.rows = second ? n * S::PLANES : n;
#pragma unroll
            for (int i = 0; i < ROWS; i++) {
                const int r = i * 32 + lane;
                if (r >= f.rows) continue;
                const int p = list[first + (second ? r / S::PLANES : r)];
                f.row[i] = second ? A.hop + ((size_t)p * S::PLANES + r % S::PLANES) * A.Fk : A.xh + (size_t)(p / C) * A.Hk;
            }
        };
        auto begin = [&](bool second, Feed &f) {
            f.c.a = f.c.stage = 0;
            f.c.at(blockIdx.x, second ? groups2 : groups1, cum, n_active);
            set_up(second, f);
        };
        auto advance = [&](bool second, Feed &f) {
            if (++f.c.stage < (second ? stages2 : stages1)) return;
            f.c.stage = 0;
            f.c.at(f.c.item + grid, second ? groups2 : groups1, cum, n_active);
            set_up(second, f);
        };
        // full barrier of a stage: one arrival announces the weights' bytes, one the tokens'
        auto load_weights = [&](bool second, const Feed &f, int slot) {
            if (lane != 0) return;
            const int ks = second ? A.ks_down : A.ks_up, s0 = f.c.stage * WK;
            const uint32_t bytes = (uint32_t)(min(WK, ks - s0) * kSliceBytes);
            mbar_expect(full + slot * 8, f.tiles * bytes);
#pragma unroll
            for (int i = 0; i < S::TM; i++)
                if (i < f.tiles)
                    bulk_copy(ring + slot * S::STAGE + i * WK * kSliceBytes, f.weights + ((size_t)i * ks + s0) * kSliceBytes, bytes, full + slot * 8);
        };
        auto load_tokens = [&](bool second, const Feed &f, int slot) {
            const int s0 = f.c.stage * WK;
            const uint32_t bytes = (uint32_t)(min(WK, (second ? A.ks_down : A.ks_up) - s0) * S::KW * 2);
            if (lane == 0) mbar_expect(full + slot * 8, f.rows * bytes);
            __syncwarp();
#pragma unroll
            for (int i = 0; i < ROWS; i++)
                if (i * 32 + lane < f.rows)
                    bulk_copy(ring + slot * S::STAGE + S::A_BYTES + (i * 32 + lane) * S::PITCH, f.row[i] + s0 * S::KW, bytes, full + slot * 8);
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
        begin(false, f);
        while (pos < n1 && next_slot()) {
            load_weights(false, f, slot);
            load_tokens(false, f, slot);
            filled();
            advance(false, f);
        }
        begin(true, f);
        Feed late = f;                                          // tokens of the second product follow the meeting
        int pos_b = pos, slot_b = slot;
        while (ok && pos < n1 + n2 && pos < n1 + kStages && next_slot()) {
            load_weights(true, f, slot);
            filled();
            advance(true, f);
        }
        const unsigned target = round + gridDim.x * (E4M3 ? 2u : 1u);
        if (ok && n2 > 0) ok = arrive_and_poll(A.ctl, target, false);
        __syncwarp();
        asm volatile("fence.proxy.async;" ::: "memory");
        for (; ok && pos_b < pos; pos_b++) {
            load_tokens(true, late, slot_b);
            advance(true, late);
            slot_b = slot_b + 1 == kStages ? 0 : slot_b + 1;
        }
        while (ok && pos < n1 + n2 && next_slot()) {
            load_weights(true, f, slot);
            load_tokens(true, f, slot);
            filled();
            advance(true, f);
        }
        // nothing may be in flight when the block ends; after a wait that ran out, the stages without tokens are closed first
        if (!ok) {
            for (; pos_b < pos && pos_b >= n1; pos_b++) {
                if (lane == 0) mbar_arrive(full + slot_b * 8);
                slot_b = slot_b + 1 == kStages ? 0 : slot_b + 1;
            }
            for (int i = max(0, pos - kStages); i < pos; i++) mbar_wait(full + (i % kStages) * 8, (unsigned)(i / kStages) & 1u);
            if (lane == 0 && A.status) *A.status = 1;
        }
        return;
    }

    // ===================================================== the multiplying warps
    float acc[MI][NT / 8][4], scale0[MI], scale1[MI];
    int slot = 0;
    unsigned parity = 0;
    bool ok = true;
    auto clear = [&](float (&v)[MI][NT / 8][4]) {
#pragma unroll
        for (int i = 0; i < MI; i++)
#pragma unroll
            for (int j = 0; j < NT / 8; j++) v[i][j][0] = v[i][j][1] = v[i][j][2] = v[i][j][3] = 0.f;
    };
    auto multiply = [&](bool second, const Cursor &c, int n) {  // this warp's slices of the stage into acc
        const int tiles = second ? A.h_tiles : A.f_tiles, ks = second ? A.ks_down : A.ks_up;
        const int tile = c.r * S::TM + wm * MI, s = c.stage * WK + wk;
        const bool live = tile < tiles && s < ks;               // a second tile past the end multiplies old bytes of the ring; nobody reads the rows
        float s0[MI], s1[MI];
        if (E4M3) {
            if (c.stage % 32 == 0) {                            // block scales of 32 stages, a stage a lane
                const int mine = (c.stage + lane) * WK + wk;
                const int kb_n = second ? (A.m.F + 127) / 128 : (H + 127) / 128;
#pragma unroll
                for (int i = 0; i < MI; i++) {
                    const bool any = tile + i < tiles && mine < ks;
                    if (second) {
                        scale0[i] = any ? __ldg(A.ds + ((size_t)act[c.a] * ((H + 127) / 128) + (tile + i) / 8) * kb_n + mine) : 0.f;
                    } else {
                        const size_t at = ((size_t)act[c.a] * ((A.m.F + 127) / 128) + (tile + i) / 16) * kb_n + mine;
                        scale0[i] = any ? __ldg(A.gs + at) : 0.f;
                        scale1[i] = any ? __ldg(A.us + at) : 0.f;
                    }
                }
            }
#pragma unroll
            for (int i = 0; i < MI; i++) {
                s0[i] = __shfl_sync(0xFFFFFFFFu, scale0[i], c.stage % 32);
                s1[i] = second ? s0[i] : __shfl_sync(0xFFFFFFFFu, scale1[i], c.stage % 32);
            }
        }
        if (ok) ok = mbar_wait(full + slot * 8, parity);
        if (live && ok) {
            const uint32_t wa = ring + slot * S::STAGE + (wm * MI * WK + wk) * kSliceBytes + lane * 16;
            const int planes = second ? S::PLANES : 1;
            const uint32_t tb = ring + slot * S::STAGE + S::A_BYTES + g * (planes * S::PITCH) + wk * S::KW * 2 + q * 16;
            float sub[MI][NT / 8][4];
            if (E4M3) clear(sub);
            float (&sum)[MI][NT / 8][4] = E4M3 ? sub : acc;
#pragma unroll
            for (int kg = 0; kg < S::KW / 32; kg++) {
                uint32_t a[MI][2][4];
#pragma unroll
                for (int t = 0; t < MI; t++) {
                    if (E4M3) {
                        const uint4 v = lds128(wa + t * WK * kSliceBytes + kg * 512);
                        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                        for (int i = 0; i < 4; i++) {
                            a[t][i >> 1][2 * (i & 1)] = f16x2_of_e4m3x2(w[i]);
                            a[t][i >> 1][2 * (i & 1) + 1] = f16x2_of_e4m3x2(w[i] >> 16);
                        }
                    } else {
#pragma unroll
                        for (int i = 0; i < 2; i++) {
                            const uint4 v = lds128(wa + t * WK * kSliceBytes + (2 * kg + i) * 512);
                            a[t][i][0] = v.x; a[t][i][1] = v.y; a[t][i][2] = v.z; a[t][i][3] = v.w;
                        }
                    }
                }
#pragma unroll
                for (int j = 0; j < NT / 8; j++) {
                    if (NT > 8 && j * 8 >= n) break;
                    for (int pl = 0; pl < planes; pl++) {
                        const uint4 b = lds128(tb + (j * 8 * planes + pl) * S::PITCH + kg * 64);
#pragma unroll
                        for (int t = 0; t < MI; t++) mma16<MT>(sum[t][j], a[t][0][0], a[t][0][1], a[t][0][2], a[t][0][3], b.x, b.y);
#pragma unroll
                        for (int t = 0; t < MI; t++) mma16<MT>(sum[t][j], a[t][1][0], a[t][1][1], a[t][1][2], a[t][1][3], b.z, b.w);
                    }
                }
            }
            if (E4M3) {
#pragma unroll
                for (int j = 0; j < NT / 8; j++) {
                    if (NT > 8 && j * 8 >= n) break;
#pragma unroll
                    for (int t = 0; t < MI; t++) {
                        acc[t][j][0] = fmaf(sub[t][j][0], s0[t], acc[t][j][0]);
                        acc[t][j][1] = fmaf(sub[t][j][1], s0[t], acc[t][j][1]);
                        acc[t][j][2] = fmaf(sub[t][j][2], s1[t], acc[t][j][2]);
                        acc[t][j][3] = fmaf(sub[t][j][3], s1[t], acc[t][j][3]);
                    }
                }
            }
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(empty + slot * 8);
        if (++slot == kStages) {
            slot = 0;
            parity ^= 1u;
        }
    };
    // The WK warps' partial sums meet in `red` ([wk][row][token]).  Where two buffers fit, two halves of the warps take turns: one
    // finishes an item while the other already multiplies the next.  A warp puts its sums into a buffer again only after it has waited for,
    // or finished, the item in between, and that item's barrier has seen every warp finish with the buffer.  With one buffer
    // all warps finish every item.
    constexpr int FINISH = S::BUFS == 2 ? kMoeThreads / 2 : kMoeThreads;
    const int half = warp / (kMoeWarps / 2), htid = tid % FINISH;
    int turn = 0;
    const float *r_get = red;
    auto put_partials = [&]() {                                 // true: this warp finishes the item, with FINISH - 1 other threads
        float *buf = red + turn * (S::RED / 4);
        if (S::BUFS == 1) bar<2, kMoeThreads>();                // everyone has finished the item before
#pragma unroll
        for (int t = 0; t < MI; t++)
#pragma unroll
            for (int j = 0; j < NT / 8; j++) {
                float *r = buf + ((wk * S::TM + wm * MI + t) * 16 + g) * NT + j * 8 + 2 * q;
                r[0] = acc[t][j][0];
                r[1] = acc[t][j][1];
                r[8 * NT] = acc[t][j][2];
                r[8 * NT + 1] = acc[t][j][3];
            }
        r_get = buf;
        if (S::BUFS == 1) {
            bar<1, kMoeThreads>();
            return true;
        }
        const bool mine = turn == half;
        if (turn == 0) {
            if (mine) bar<1, kMoeThreads>(); else bar_arrive<1, kMoeThreads>();
        } else {
            if (mine) bar<2, kMoeThreads>(); else bar_arrive<2, kMoeThreads>();
        }
        turn ^= 1;
        return mine;
    };
    auto total = [&](int row, int col) {
        float v = 0.f;
#pragma unroll
        for (int i = 0; i < WK; i++) v += r_get[(i * S::TM * 16 + row) * NT + col];
        return v;
    };

    Cursor c;
    c.a = c.stage = 0;
    c.at(blockIdx.x, groups1, cum, n_active);
    for (int it = 0; it < mine1; it++) {
        const int e = act[c.a], first = off[e] + c.c * NT, n = min(NT, cnt[e] - first);
        clear(acc);
        for (c.stage = 0; c.stage < stages1; c.stage++) multiply(false, c, n);
        constexpr int FR = 8 * S::TM;                              // hidden units of the item
        const bool mine = put_partials();
        for (int i = htid; mine && i < (FR * n + 31) / 32 * 32; i += FINISH) {
            const int col = i / FR, fr = i - col * FR, f = c.r * FR + fr;
            float h = 0.f;
            int p = 0;
            if (col < n) {
                const int row = (fr >> 3) * 16 + (fr & 7);
                p = list[first + col];
                float gate = total(row, col), up = total(row + 8, col);
                if (E4M3) {
                    const float xs = A.xh_scale[p / C];
                    gate *= xs;
                    up *= xs;
                }
                if (f < A.Fp) {
                    h = gate / (1.f + expf(-gate)) * up;
                    if (E4M3) {
                        A.h32[(size_t)p * A.Fp + f] = h;
                    } else {
                        const uint32_t hi = bf16x2_of(h, 0.f) & 0xFFFFu;
                        uint16_t *dst = A.hop + (size_t)p * 2 * A.Fk + f;
                        dst[0] = (uint16_t)hi;
                        dst[A.Fk] = (uint16_t)bf16x2_of(h - __uint_as_float(hi << 16), 0.f);
                    }
                }
            }
            if (E4M3) {
                unsigned m = __float_as_uint(h) & 0x7FFFFFFFu;  // order of the magnitudes, infinity and NaN above all
#pragma unroll
                for (int o = (FR < 32 ? FR : 32) / 2; o; o >>= 1) m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, o));
                if (fr % 32 == 0 && col < n) atomicMax(A.h_max + p, m);   // a maximum: the order does not matter
            }
        }
        if (!E4M3 && mine && c.r == groups1 - 1) {              // zeros behind F
            const int pad = A.Fk - A.Fp;
            for (int i = htid; i < pad * n * 2; i += FINISH)
                A.hop[((size_t)list[first + i / (2 * pad)] * 2 + i / pad % 2) * A.Fk + A.Fp + i % pad] = 0;
        }
        c.at(c.item + grid, groups1, cum, n_active);
    }

    // ---- all hidden activations are there
    ok = meet<3, kMoeThreads>(A.ctl, round, &meet_ok) && ok;
    if (E4M3) {                                                 // as fp16 times a power of two per pair
        const int quads = A.Fk / 4, n_pairs = n_active ? cnt[act[n_active - 1]] : 0;
        for (long long i = (long long)blockIdx.x * kMoeThreads + tid; i < (long long)n_pairs * quads; i += (long long)grid * kMoeThreads) {
            const int p = list[i / quads], f = (int)(i % quads) * 4;
            float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
            if (f < A.Fp) v = *reinterpret_cast<const float4 *>(A.h32 + (size_t)p * A.Fp + f);
            const float d = exp2i(-fp16_exponent(__uint_as_float(A.h_max[p])));
            *reinterpret_cast<uint2 *>(A.hop + (size_t)p * A.Fk + f) = make_uint2(f16x2_of(v.x * d, v.y * d), f16x2_of(v.z * d, v.w * d));
        }
        ok = meet<3, kMoeThreads>(A.ctl, round, &meet_ok) && ok;
    }

    // ---- second product
    c.a = c.stage = 0;
    c.at(blockIdx.x, groups2, cum, n_active);
    for (int it = 0; it < mine2; it++) {
        const int e = act[c.a], first = off[e] + c.c * NT, n = min(NT, cnt[e] - first);
        clear(acc);
        for (c.stage = 0; c.stage < stages2; c.stage++) multiply(true, c, n);
        constexpr int HR = 16 * S::TM;
        const bool mine = put_partials();
        for (int i = htid; mine && i < HR * n; i += FINISH) {
            const int col = i / HR, row = i - col * HR, hr = c.r * HR + row;
            const int p = list[first + col];
            if (hr < H) {
                float v = total(row, col);
                if (E4M3) v *= exp2i(fp16_exponent(__uint_as_float(A.h_max[p])));
                A.y[(size_t)p * H + hr] = v;
            }
        }
        c.at(c.item + grid, groups2, cum, n_active);
    }
    ok = meet<3, kMoeThreads>(A.ctl, round, &meet_ok) && ok;
    if (!ok) {
        if (lane == 0 && A.status) *A.status = 1;
        return;
    }

    // ---- a token's parts, in the order of its choices
    const int quads = H / 4;
    for (int i = blockIdx.x * kMoeThreads + tid; i < T * quads; i += grid * kMoeThreads) {
        const int t = i / quads, h = (i - t * quads) * 4;
        float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int j = 0; j < C; j++) {
            float w = 1.f;
            if (j < K) {
                const int e = A.ids[t * K + j] - A.m.first;
                if (e < 0 || e >= A.m.n_local) continue;
                w = A.weights[t * K + j];
            }
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
}
static size_t take(size_t &at, size_t bytes)
{
    const size_t here = at;
    at += (bytes + 255) & ~(size_t)255;
    return here;
}
// carves the workspace; sms: number of SMs (sizes the router's grid).  Returns its size; `base` may be NULL.
static size_t moe_carve(MoeArgs &a, int T, int sms, uint8_t *base)
{
    const pf_moe_t &m = a.m;
    const bool e4m3 = m.wtype == PF_DT_E4M3;
    a.T = T;
    a.e_tiles = (m.n_experts + 15) / 16;
    a.t_chunks = (T + kRouteTokens - 1) / kRouteTokens;
    // router: about one block per SM, at least 256 columns (32 per warp) for each
    const int most = (m.H + 255) / 256, want = sms / (a.e_tiles * a.t_chunks);
    a.h_splits = want < 1 ? 1 : (want < most ? want : most);
    if (a.h_splits > kRouteSplits) a.h_splits = kRouteSplits;
    const size_t pairs = (size_t)T * a.choices;
    size_t at = 0;
    a.ctl = (unsigned *)(base + take(at, 256));
    a.h_max = (unsigned *)(base + take(at, pairs * 4));
    a.logits = (float *)(base + take(at, (size_t)a.h_splits * T * m.n_experts * 4));
    a.xh = (uint16_t *)(base + take(at, (size_t)T * a.Hk * 2));
    a.xh_scale = (float *)(base + take(at, (size_t)T * 4));
    a.h32 = (float *)(base + take(at, e4m3 ? pairs * a.Fp * 4 : 0));
    a.hop = (uint16_t *)(base + take(at, pairs * a.Fk * 2 * (e4m3 ? 1 : 2)));
    a.y = (float *)(base + take(at, pairs * m.H * 4));
    return at;
}

template <bool E4M3, int WM, int WK, int MI, int NT>
static int moe_launch(const MoeArgs &a, int device, int sms, cudaStream_t st)
{
    using S = MoeShape<E4M3, WM, WK, MI, NT>;
    const size_t smem = (size_t)S::FIXED + ((size_t)a.n_sets * 4 + 1) * 4 + (size_t)a.T * a.choices * 2;
    PF_CUDA_TRY(ensure_dynamic_smem((const void *)moe_kernel<E4M3, WM, WK, MI, NT>, device, smem), "moe_kernel shared memory");
    const int n_route = a.e_tiles * a.h_splits * a.t_chunks + a.T;
    moe_route_kernel<E4M3><<<n_route, kMoeThreads, 0, st>>>(a);
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
    PF_CUDA_TRY(cudaLaunchKernelEx(&cfg, moe_kernel<E4M3, WM, WK, MI, NT>, a), "moe_kernel launch");
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
    return a.set_bytes * (size_t)a.n_sets;
}

extern "C" int pf_moe_pack(const pf_moe_t *m, const void *d_gate, const void *d_up, const void *d_down, void *d_packed, void *stream)
{
    if (!moe_ok(m) || !d_gate || !d_up || !d_down || !d_packed) return PF_EINVAL;
    if (!aligned16(d_gate) || !aligned16(d_up) || !aligned16(d_down) || ((uintptr_t)d_packed & 255)) return PF_EINVAL;
    MoeArgs a;
    moe_layout(m, a);
    const size_t units = a.set_bytes * (size_t)a.n_sets / 16;
    const unsigned grid = (unsigned)((units + 255) / 256 < 65536 ? (units + 255) / 256 : 65536);
    cudaStream_t st = (cudaStream_t)stream;
    if (m->wtype == PF_DT_E4M3)
        moe_pack_kernel<true><<<grid, 256, 0, st>>>(*m, a.n_sets, a.f_tiles, a.ks_up, a.ks_down, a.set_bytes, a.down_at, (const uint8_t *)d_gate,
                                                    (const uint8_t *)d_up, (const uint8_t *)d_down, (uint8_t *)d_packed);
    else
        moe_pack_kernel<false><<<grid, 256, 0, st>>>(*m, a.n_sets, a.f_tiles, a.ks_up, a.ks_down, a.set_bytes, a.down_at, (const uint8_t *)d_gate,
                                                     (const uint8_t *)d_up, (const uint8_t *)d_down, (uint8_t *)d_packed);
    PF_CUDA_TRY(cudaGetLastError(), "moe_pack_kernel launch");
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
                              const void *d_router, const void *d_packed, const float *d_gate_scale, const float *d_up_scale,
                              const float *d_down_scale, void *d_out, int32_t *d_ids, float *d_weights, int32_t *d_status,
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
    if (e4m3 && (!d_gate_scale || !d_up_scale || !d_down_scale)) return PF_EINVAL;
    int device, sms;
    if (int rc = current_sm_count(&device, &sms)) return rc;
    MoeArgs a;
    moe_layout(m, a);
    if (!d_workspace || ((uintptr_t)d_workspace & 255) != 0 || workspace_bytes < moe_carve(a, T, sms, (uint8_t *)d_workspace)) return PF_EWORKSPACE;
    a.x = (const uint16_t *)d_x; a.xs = x_stride; a.xq = d_xq; a.xscale = d_xscale;
    a.router = (const uint16_t *)d_router; a.packed = (const uint8_t *)d_packed;
    a.gs = d_gate_scale; a.us = d_up_scale; a.ds = d_down_scale;
    a.out = (uint16_t *)d_out; a.ids = d_ids; a.weights = d_weights; a.status = d_status;
    cudaStream_t st = (cudaStream_t)stream;
    // Up to 8 tokens an expert never has more than one 8-token column block: tiles of 32 rows, the columns split over the
    // warps, fill the GPU with the fewest experts.  Beyond, 64 rows share a stage's tokens, up to 16 of them, and with more than 8 tokens an
    // expert on average 128 rows share up to 32.
    if (T <= 8) return e4m3 ? moe_launch<true, 1, 8, 2, 8>(a, device, sms, st) : moe_launch<false, 1, 8, 2, 8>(a, device, sms, st);
    if ((long long)T * m->top_k <= 8ll * m->n_experts)
        return e4m3 ? moe_launch<true, 2, 4, 2, 16>(a, device, sms, st) : moe_launch<false, 2, 4, 2, 16>(a, device, sms, st);
    return e4m3 ? moe_launch<true, 4, 2, 2, 32>(a, device, sms, st) : moe_launch<false, 4, 2, 2, 32>(a, device, sms, st);
}
