// pf_topk.cuh -- block top-k in shared memory.  Only warp and block collectives of the language are used, so the code also
// compiles for the host over an emulation of these (tests/topk_emulation.cpp runs it under arbitrary warp orders).
#pragma once

namespace pf {

constexpr int kTopkCap = 2048;       // shared-memory candidate buffer per block (2 * PF_K_MAX)

// ------------------------------------------------------------------ block top-k in shared memory
// buf[kTopkCap] holds candidate keys, *count the number of valid ones, *thr the current admission
// threshold (the k-th best key once k are held, else 0).  All functions are block-collective unless
// noted; the block may have any multiple of 32 threads.

// Descending bitonic sort of buf[0, n_sort); n_sort a power of two <= kTopkCap; buf has room for 64 keys at
// least.  PAIRS = kTopkCap / 2 / blockDim.x.  Each thread owns adjacent elements (2p, 2p+1) for its pair
// numbers p = tid, tid + blockDim, ...; a warp therefore owns a 64-element window.  All compare-exchanges
// with stride <= 32 stay inside that window: they run on registers with warp shuffles.  Only the wider
// strides (>= 64) go through shared memory with block barriers.
template <int PAIRS>
__device__ inline void tk_sort_desc(unsigned long long *buf, int n_sort)
{
    const int tid = threadIdx.x, nt = blockDim.x, lane = tid & 31;
    const int n_eff = n_sort < 64 ? 64 : n_sort;   // whole warps take part; missing elements are zeros
    unsigned long long r0[PAIRS], r1[PAIRS];
    __syncthreads();
#pragma unroll
    for (int t = 0; t < PAIRS; t++) {
        const int i0 = 2 * (tid + t * nt);
        r0[t] = i0 < n_sort ? buf[i0] : 0ull;
        r1[t] = i0 + 1 < n_sort ? buf[i0 + 1] : 0ull;
    }
    for (int size = 2; size <= n_eff; size <<= 1) {
        int stride = size >> 1;
        if (stride >= 64) {
#pragma unroll
            for (int t = 0; t < PAIRS; t++) {
                const int i0 = 2 * (tid + t * nt);
                if (i0 < n_eff) {
                    buf[i0] = r0[t];
                    buf[i0 + 1] = r1[t];
                }
            }
            for (; stride >= 64; stride >>= 1) {
                __syncthreads();
                for (int i = tid; i < n_eff / 2; i += nt) {
                    const int lo = 2 * i - (i & (stride - 1)), hi = lo + stride;
                    const bool desc = (lo & size) == 0;
                    const unsigned long long a = buf[lo], b = buf[hi];
                    if (desc ? (a < b) : (a > b)) {
                        buf[lo] = b;
                        buf[hi] = a;
                    }
                }
            }
            __syncthreads();
#pragma unroll
            for (int t = 0; t < PAIRS; t++) {
                const int i0 = 2 * (tid + t * nt);
                if (i0 < n_eff) {
                    r0[t] = buf[i0];
                    r1[t] = buf[i0 + 1];
                }
            }
        }
        for (; stride >= 1; stride >>= 1) {
#pragma unroll
            for (int t = 0; t < PAIRS; t++) {
                const int i0 = 2 * (tid + t * nt);
                if (i0 >= n_eff) continue;   // whole warps only: n_eff / 2 is a multiple of 32
                const bool desc = (i0 & size) == 0;
                if (stride == 1) {
                    const unsigned long long a = r0[t], b = r1[t];
                    if (desc ? (a < b) : (a > b)) {
                        r0[t] = b;
                        r1[t] = a;
                    }
                } else {
                    const int lm = stride >> 1;
                    const unsigned long long o0 = __shfl_xor_sync(0xFFFFFFFFu, r0[t], lm);
                    const unsigned long long o1 = __shfl_xor_sync(0xFFFFFFFFu, r1[t], lm);
                    const bool keep_max = ((lane & lm) == 0) == desc;
                    r0[t] = keep_max ? (r0[t] > o0 ? r0[t] : o0) : (r0[t] < o0 ? r0[t] : o0);
                    r1[t] = keep_max ? (r1[t] > o1 ? r1[t] : o1) : (r1[t] < o1 ? r1[t] : o1);
                }
            }
        }
    }
#pragma unroll
    for (int t = 0; t < PAIRS; t++) {
        const int i0 = 2 * (tid + t * nt);
        if (i0 < n_eff) {
            buf[i0] = r0[t];
            buf[i0 + 1] = r1[t];
        }
    }
    __syncthreads();
}

// Keep the best k: sort what is held (padded to a power of two), clamp the count, refresh the threshold.
template <int PAIRS>
__device__ inline void tk_prune(unsigned long long *buf, int *count, unsigned long long *thr, int k)
{
    __syncthreads();
    int c = *count;
    if (c > kTopkCap) c = kTopkCap;
    int n_sort = 32;
    while (n_sort < c) n_sort <<= 1;
    for (int i = c + threadIdx.x; i < n_sort; i += blockDim.x) buf[i] = 0ull;
    tk_sort_desc<PAIRS>(buf, n_sort);
    if (threadIdx.x == 0) {
        int n = c < k ? c : k;
        *count = n;
        *thr = (n == k) ? buf[k - 1] : 0ull;
    }
    __syncthreads();
}

// Append the block's held keys that are >= min_key (after tk_prune: sorted, c of them) to a compact global
// key list.  s_base: two shared ints of scratch.  Block-collective.
__device__ inline void tk_flush(const unsigned long long *buf, int c, unsigned long long min_key, int *s_base,
                                unsigned long long *out_keys, unsigned int *out_count)
{
    if (threadIdx.x == 0) s_base[1] = 0;
    __syncthreads();
    // the buffer is sorted descending: the cut is the last position whose key is still >= min_key
    for (int i = threadIdx.x; i < c; i += blockDim.x)
        if (buf[i] >= min_key && (i + 1 == c || buf[i + 1] < min_key)) s_base[1] = i + 1;
    __syncthreads();
    const int keep = s_base[1];
    if (threadIdx.x == 0) s_base[0] = keep > 0 ? (int)atomicAdd(out_count, (unsigned int)keep) : 0;
    __syncthreads();
    unsigned long long *out = out_keys + s_base[0];
    for (int i = threadIdx.x; i < keep; i += blockDim.x) out[i] = buf[i];
}

// Append this thread's key if it beats the threshold.  Warp-collective (all 32 lanes must call); the
// caller guarantees room for one key per thread of the block.
__device__ __forceinline__ void tk_push(unsigned long long *buf, int *count, unsigned long long thr, bool has,
                                        unsigned long long key)
{
    bool take = has && key > thr;
    unsigned mask = __ballot_sync(0xFFFFFFFFu, take);
    if (mask == 0) return;
    int lane = threadIdx.x & 31;
    int leader = __ffs(mask) - 1;
    int base = 0;
    if (lane == leader) base = atomicAdd(count, __popc(mask));
    base = __shfl_sync(0xFFFFFFFFu, base, leader);
    if (take) {
        int pos = base + __popc(mask & ((1u << lane) - 1u));
        if (pos < kTopkCap) buf[pos] = key;
    }
}

// Walk through in[lo, hi) a tile of blockDim.x keys at a time, admitting only keys above the running k-th best, and
// leave the k best in buf (sorted, *count of them; *count and *thr start at zero).  A tile's admissions are counted
// before they are appended, so the buffer is pruned only when it would really overflow.  Whether it would is decided
// on the count as it was before anyone appends: read behind the counting barrier instead, a slow warp would see
// what faster warps have appended already, could decide otherwise than they did, and the block's warps would wait at
// different barriers.
template <int PAIRS>
__device__ inline void tk_walk(const unsigned long long *in, unsigned int lo, unsigned int hi, unsigned long long *buf,
                               int *count, unsigned long long *thr, int k)
{
    for (unsigned int pos = lo; pos < hi; pos += blockDim.x) {
        const unsigned int i = pos + threadIdx.x;
        const unsigned long long key = i < hi ? in[i] : 0ull;
        unsigned long long t = *thr;
        const int held = *count;
        const int takers = __syncthreads_count(key > t);
        if (held + takers > kTopkCap) {
            tk_prune<PAIRS>(buf, count, thr, k);
            t = *thr;
        }
        tk_push(buf, count, t, key != 0ull, key);
        __syncthreads();
    }
    tk_prune<PAIRS>(buf, count, thr, k);
}

}  // namespace pf
