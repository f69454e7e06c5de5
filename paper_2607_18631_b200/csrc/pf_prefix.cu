// pf_prefix.cu -- single-token attention of sequences that share prefixes.
//
//   out = sum_t w_t V_t / sum_t w_t,  t over the prefix of the sequence's group and over its own tokens,  w_t = exp(sm q . K_t)
//
// A group's rows (sequences times query heads of a key head) are cut into tiles of 256, and such a tile goes through the group's prefix once:
// the cache is read once for all of them.  All (tile of rows, tile of 128 tokens) pairs of all groups and key heads form one list, which is cut into
// equal pieces, one a block; a piece leaves partial results (reference z, sum, weighted values) of each of its tiles of rows.  The sequences' own tokens
// go through the kernel of pf_decode_attention on the SMs that the prefixes leave, and a third kernel joins the parts of every row in a fixed order.
//
// Both products are the fifth generation's matrix instruction: scores = Q K^T, 128 rows by 128 tokens, both operands in shared memory; values += P V, the
// weights P in tensor memory, where the threads that own the rows put them over the scores.  The cache's e4m3 is widened to fp16 in between (exact), as in the kernel of the own
// tokens, so queries keep all their bits and weights 11; scores, references, sums and values are fp32.  The value scale joins the exponent, as there.
// A block has two streams of 128 rows, so that the products of one are under way while the other's weights are computed; with no more than 128 rows both
// go through the same ones and take turns with the tiles.  A row's reference lies 15 below the largest score when it is set, and stays until a weight would pass
// 2^15.9: tensor memory's values are scaled anew in the first tiles of a piece for the most part.  Warps have one role each and meet at barriers in shared memory:
//   plan -> copy (bulk, half tiles) -> widen -> products <-> rows.
// What bounds it.  Many rows: 128 x 128 scores take the products 1024 cycles, the special-function unit 768 (a quarter of the powers are polynomials) and shared memory
// 1280 (operands 768, the cache's bytes in, out and widened 1024 a tile that two streams share), and the chain scores -> largest -> powers -> products of a stream some 4000, of which the
// other stream fills a half: 256 sequences of 64 / 8 heads of 128 behind 32768 tokens 336 us (825 TFLOP/s; behind 8192 the tensor pipe is 36 % active, issue slots 45 %).  Few rows: a tile's way
// through copy, widen and products, some 2350 cycles against 1400 from HBM: 3 such sequences behind 262143 tokens 162 us (3.3 TB/s).
// Measured on the way there (us, these two): rows' scores read twice, one widening role that also loads: 594, 442; scores kept in registers, registers moved to the groups that need
// them: 394, 198; a whole warp in the products' loop: 373; packed arithmetic, polynomials, half tiles of weights handed over: 353; bulk copies, roles apart: 344, 177; own tokens
// beside the prefixes: 322; less code in what every tile goes through: 171; whole tiles widened without a look at their pages: 161 (few rows); references 15 below the largest score instead of
// 7, for the small weights' bits, and a way for scores at which fp32 is coarse: 336, 162.  Not kept: 16 warps for the rows (two a row, 350), two warps for the products (386), eight
// warps that widen (344), four places for half tiles where few rows leave room (360, 207), few rows several times over for a part of a tile each (332, 211).
#include <math.h>

#include <atomic>
#include <type_traits>

#include "pf_attention.cuh"
#include "pf_tcgen.cuh"

namespace pf {

constexpr int kMostTiles = 512;          // tiles of a piece: tensor memory's 32-bit sums do not run over more than 65536 tokens
constexpr int kMostPieces = 64;          // of a block, though: lists of more than 64 x 512 tiles a block (some 80 ms) have longer ones
constexpr int kAhead = 4;                // tiles that are under way from HBM to the L2
constexpr int kLeastTiles = 1;           // a piece takes no fewer while others have none
constexpr unsigned kWaitLimit = 500000, kDrainLimit = 500000;      // polls of 2 us: a second
std::atomic<unsigned> g_wait_limit{kWaitLimit}, g_wait_lost{0};      // host: what the next calls do (pf_prefix_waits)
constexpr float kCoarse = 131072.f;      // references from here on: a unit in the last place is 2^-6 or more
// log2 of the largest weight when a row's reference is set (kLift, as in the kernel of the own tokens: weights keep 11 bits down to 2^-29 of the largest and count down
// to 2^-40 of it), and what it may grow to before the reference is set anew: fp16 ends at 2^15.9999
constexpr float kMostLift = 15.9f;

struct PrefixArgs {
    AttnArgs a;
    const int32_t *ptable;
    unsigned wait_limit, wait_lost;      // polls of a wait inside the kernel; whether a block waits for what does not come (a test of the limit)
    long long n_rows;                    // rows of partial results
    uint32_t *status;                    // [blocks], written by those with work
    float *part_v, *part_z, *part_l;     // [n_rows] x HD values, references, sums
    int32_t *report;                     // the call's status, or NULL
};

// Partial results.  A task (a tile of a group's rows of a key head) takes as many rows as it has, twice as many where both streams go through the same ones, and each piece of the list leaves
// those of its tasks `piece_rows` further on than the piece in front, which is no less than any task takes: neighbours on the list are apart.
__host__ __device__ __forceinline__ int task_rows(int rows) { return rows <= 128 ? 2 * rows : rows; }
__host__ __device__ __forceinline__ int piece_rows(int n_seq, int group) { return n_seq * (long long)group < kRows / 2 ? 2 * n_seq * group : kRows; }
// rows of a group's tasks of one key head
__device__ __forceinline__ int head_rows(const Group &g) { return (g.row_tiles - 1) * kRows + task_rows(g.rows - (g.row_tiles - 1) * kRows); }

// Tiles, and rows of partial results, of the groups in front of each group, by the whole block.  units, rows: n_groups + 1 words; scratch: 64
__device__ __forceinline__ void group_prefix(const PrefixArgs &P, long long *units, long long *rows, long long *scratch)
{
    long long *warp_rows = scratch, *warp_units = scratch + 32;
    const int nt = blockDim.x, tid = threadIdx.x, lane = tid & 31, nw = (nt + 31) >> 5;
    long long base_u = 0, base_r = 0;
    if (tid == 0) units[0] = rows[0] = 0;
    for (int g0 = 0; g0 < P.a.n_groups; g0 += nt) {
        long long u = 0, r = 0;
        if (g0 + tid < P.a.n_groups) {
            const Group g = group_of(P.a, g0 + tid);
            if (g.tiles && g.row_tiles) {
                u = (long long)g.row_tiles * P.a.c.n_kv * g.tiles;
                r = (long long)head_rows(g) * P.a.c.n_kv;
            }
        }
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long pu = __shfl_up_sync(0xFFFFFFFFu, u, o), pr = __shfl_up_sync(0xFFFFFFFFu, r, o);
            if (lane >= o) u += pu, r += pr;
        }
        __syncthreads();
        if (lane == 31) warp_units[tid >> 5] = u, warp_rows[tid >> 5] = r;
        __syncthreads();
        long long add_u = base_u, add_r = base_r;
        for (int i = 0; i < nw; i++) {
            if (i < (tid >> 5)) add_u += warp_units[i], add_r += warp_rows[i];
            base_u += warp_units[i];
            base_r += warp_rows[i];
        }
        if (g0 + tid < P.a.n_groups) units[g0 + tid + 1] = add_u + u, rows[g0 + tid + 1] = add_r + r;
    }
    __syncthreads();
}
// pieces that the list is cut into: one a block, or as many more as keep them at kMostTiles
__device__ __forceinline__ int pieces_of(long long total, int blocks)
{
    const long long few = (total + kLeastTiles - 1) / kLeastTiles;
    if (few < blocks) return (int)few;
    const long long per = (total + (long long)blocks * kMostTiles - 1) / ((long long)blocks * kMostTiles);
    return (int)(per < kMostPieces ? per : kMostPieces) * blocks;
}
// pieces of a block, which follow one another
__device__ __forceinline__ int pieces_each(int n_pieces, int blocks) { return (n_pieces + blocks - 1) / blocks; }
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

// A stretch of tiles [tile, end) of one task: what the roles of a block work on together
struct __align__(16) Stretch {
    int group, first, members, len;      // the group, its first sequence, its rows, and its tokens
    int kv, row0, rows, tile;            // the task's rows are row0 .. row0 + rows - 1 of the group
    int end, pad;                        // (end = tile: there are no more)
    long long at;                        // the first of its rows of partial results
    // few rows: both streams go through the same rows, and take turns with the tiles
    __device__ __forceinline__ bool turns() const { return rows <= 128; }
    __device__ __forceinline__ int tiles_of(int stream) const { return turns() ? (end - tile + 1 - stream) / 2 : end - tile; }
};
static_assert(sizeof(Stretch) == 48, "as the roles read it");

// Four groups of four warps: two streams that own the rows, one that widens the cache's bytes, and one of which a warp issues the products, two copy
// from the cache and one plans.  Registers go where they are needed: 256 x 184 + 128 x 96 + 128 x 48 = 512 x 128, what the block is launched with.
constexpr int kSoftWarps = 8, kWidenWarps = 4;
constexpr int kPrefixThreads = 512, kSoftRegs = 184, kWidenRegs = 96, kProductRegs = 48;
static_assert(kSoftRegs * 256 + kWidenRegs * 128 + kProductRegs * 128 <= kPrefixThreads * 128, "no group waits for registers that nobody gives back");
template <int N> __device__ __forceinline__ void take_registers() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N> __device__ __forceinline__ void leave_registers() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }
template <int HD> struct PrefixShape {
    static constexpr int kHalves = HD / 64;             // 128-byte columns of an fp16 row
    static constexpr int kOperand = kHalves * 16384;    // 128 rows of HD fp16
    static constexpr int kQ = 0, kK = 2 * kOperand, kV = 4 * kOperand;
    static constexpr int kRing = 6 * kOperand;          // bytes of the cache under way: a tile of keys and one of values
    static constexpr int kScales = kRing + 2 * kTok * HD;        // of eight tiles, for each 16 tokens: key scale, log2 and inverse of the value scale
    static constexpr int kHave = kScales + 8 * 128;     // which runs of a half tile were copied, of keys and of values
    static constexpr int kPlan = kHave + 16;            // two stretches
    static constexpr int kBars = kPlan + 2 * 48, kBytes = kBars + 288;
    static_assert(kBytes <= 227 * 1024, "fits an SM");
};
constexpr uint32_t kTmem = 0;            // tensor memory: a block takes all 512 columns, which begin at 0
// barriers, 8 bytes each
enum {
    B_KFULL = 0, B_KEMPTY = 2, B_VFULL = 4, B_VEMPTY = 6,                       // two tiles of operands, widened and given back
    B_QFULL = 8, B_SFULL = 10, B_PHALF = 12, B_PFULL = 14, B_OFULL = 16,        // of either stream: queries, scores, half and all of the weights, values
    B_DRAIN = 18,
    B_KRAW = 19, B_VRAW = 21, B_KREAD = 23, B_VREAD = 25,                       // either half of a tile's bytes, copied and read
    B_PLAN = 27, B_DONE = 29,                                                   // two stretches
    B_COUNT = 31
};

// 16-byte chunk c of row r of an operand's 128-byte column
__device__ __forceinline__ uint32_t operand_at(int r, int c) { return (uint32_t)(r * 128 + ((c ^ (r & 7)) << 4)); }
__device__ __forceinline__ void sts128(uint32_t a, uint32_t x, uint32_t y, uint32_t z, uint32_t w)
{
    asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(a), "r"(x), "r"(y), "r"(z), "r"(w) : "memory");
}

struct PrefixRoom {                     // what the roles share
    uint32_t smem, bars, gave_up;
    unsigned limit;
    int run_log2;
    __device__ __forceinline__ bool wait(int bar, unsigned parity) const { return bar_wait(bars + 8 * bar, parity & 1u, limit, gave_up); }
    __device__ __forceinline__ bool wait_warp(int bar, unsigned parity) const { return __all_sync(0xFFFFFFFFu, wait(bar, parity)); }      // one answer for all lanes
    __device__ __forceinline__ void arrive(int bar) const { bar_arrive(bars + 8 * bar); }
    // the run-th stretch, by a whole warp, which says done() of it afterwards; false: there is none
    __device__ __forceinline__ bool next(const Stretch *plan, unsigned run, Stretch &s) const
    {
        if (!wait_warp(B_PLAN + (run & 1), run >> 1)) return false;
        s = plan[run & 1];
        return s.end > s.tile;
    }
    __device__ __forceinline__ void done(unsigned run) const
    {
        __syncwarp();
        if ((threadIdx.x & 31) == 0) arrive(B_DONE + (run & 1));
    }
};

// ---- one thread finds the block's stretches, one ahead: pieces follow one another, so where the first begins is looked up once (`units`, `rows`: before the others
// overwrite them), and from there it goes on by itself
struct Walk {
    Group g;
    int group, no, tile, piece, last, n_pieces;         // no: of the group's tasks
    long long total, row;                               // row: the group's first of partial results
    __device__ __forceinline__ bool begin(const PrefixArgs &P, const long long *units, const long long *rows, int blocks)
    {
        total = units[P.a.n_groups];
        n_pieces = total ? pieces_of(total, blocks) : 0;
        const int per = pieces_each(n_pieces, blocks);
        piece = blockIdx.x * per;
        last = min(n_pieces, piece + per);
        if (piece >= last) return false;
        const long long u = first_tile(total, n_pieces, piece);
        group = last_at(units, P.a.n_groups, u);
        g = group_of(P.a, group);
        row = rows[group];
        no = (int)((u - units[group]) / g.tiles);
        tile = (int)((u - units[group]) - (long long)no * g.tiles);
        return true;
    }
};
__device__ __forceinline__ void plan_role(const PrefixArgs &P, const PrefixRoom &R, Walk k, Stretch *plan)
{
    unsigned run = 0;
    auto room = [&]() { return R.wait(B_DONE + (run & 1), (run >> 1) ^ 1u); };
    for (; k.piece < k.last; k.piece++) {
        int left = (int)(first_tile(k.total, k.n_pieces, k.piece + 1) - first_tile(k.total, k.n_pieces, k.piece));
        while (left > 0) {
            while (k.no >= (k.g.tiles ? k.g.row_tiles * P.a.c.n_kv : 0)) {
                if (k.g.tiles && k.g.row_tiles) k.row += (long long)head_rows(k.g) * P.a.c.n_kv;
                k.no = 0;
                if (++k.group >= P.a.n_groups) return;    // (not reached: the list ends with the last piece)
                k.g = group_of(P.a, k.group);
            }
            Stretch s;
            s.group = k.group; s.first = k.g.first; s.members = k.g.rows; s.len = k.g.len;
            s.kv = k.no / k.g.row_tiles;
            s.row0 = (k.no - s.kv * k.g.row_tiles) * kRows;
            s.rows = min(kRows, k.g.rows - s.row0);
            s.tile = k.tile;
            s.end = min(k.g.tiles, k.tile + left);
            s.pad = 0;
            s.at = k.row + (long long)s.kv * head_rows(k.g) + s.row0 + (long long)k.piece * piece_rows(P.a.n_seq, P.a.group);
            left -= s.end - s.tile;
            k.tile = s.end;
            if (k.tile == k.g.tiles) {
                k.tile = 0;
                k.no++;
            }
            if (!room()) return;
            plan[run & 1] = s;
            R.arrive(B_PLAN + (run & 1));
            run++;
        }
    }
    if (!room()) return;
    plan[run & 1].tile = plan[run & 1].end = 0;
    R.arrive(B_PLAN + (run & 1));
}

// ---- the cache's bytes on their way: a warp for keys, one for values.  Half a tile at a time is copied in bulk into one of two places, as soon as what was there has
// been read; tiles further on are asked for from HBM into the L2, so that a copy has the L2's latency only.
// (Tried instead: pieces in the registers of those who widen them, whose loads a warp waits for all together; 16-byte copies, of which a warp issues one in some 100 cycles.)
template <int HD>
__device__ __forceinline__ void copy_role(const PrefixArgs &P, const PrefixRoom &R, const Stretch *plan, const int values)
{
    using S = PrefixShape<HD>;
    const AttnArgs &A = P.a;
    const int lane = threadIdx.x & 31;
    const uint8_t *cache = values ? A.c.d_v : A.c.d_k;
    const uint32_t ring = R.smem + S::kRing + values * kTok * HD, have_at = R.smem + S::kHave + values * 8;
    const int raw = values ? B_VRAW : B_KRAW, read = values ? B_VREAD : B_KREAD;
    // a run: tokens of half a tile that lie side by side in the cache.  (A copy takes the warp some 100 cycles, whatever its size.)
    const int page_log2 = 31 - __clz(A.c.page), run_log2 = min(page_log2, 6), runs = kTok >> run_log2;
    unsigned n = 0, asked[2] = {0, 0};                  // tiles so far, and of either half those that were asked for
    bool good = true;
    Stretch s;
    for (unsigned run = 0; good && R.next(plan, run, s); R.done(run), run++) {
        const int32_t *row = P.ptable + (int64_t)s.group * P.a.pcols;
        auto page_of = [&](int tile) {                  // lane i: page of the tile's i-th run, negative: none
            const int tok = tile * kTok + (lane << run_log2);
            return lane < runs && tile < s.end && tok < s.len ? row[tok >> page_log2] : -1;
        };
        auto there = [&](int page) { return page >= 0 && page < A.c.n_pages; };
        auto place_of = [&](int page) { return cache + (((int64_t)page * A.c.n_kv + s.kv) * A.c.page + ((lane << run_log2) & (A.c.page - 1))) * HD; };
        auto ahead = [&](int page) {
            if (there(page)) asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(place_of(page)), "r"(HD << run_log2) : "memory");
        };
        // The keys' warp also leaves the tile's scales.  Missing pages and 16 tokens behind the end: log2 -infinity, inverse 0.
        float ks = 1.f, vs = -1.f;
        auto scales_of = [&](int pages) {
            const int page = __shfl_sync(0xFFFFFFFFu, pages, (lane & 7) >> (run_log2 - 4));
            const int64_t ph = (int64_t)page * A.c.n_kv + s.kv;
            ks = there(page) ? __ldg(A.c.d_k_scale + ph) : 1.f;
            vs = there(page) ? __ldg(A.c.d_v_scale + ph) : -1.f;
        };
        int page = page_of(s.tile), next = page_of(s.tile + 1), far = page_of(s.tile + kAhead);
        if (!values) scales_of(page);
        for (int t = s.tile; good && t < s.end; t++, n++) {
            const uint8_t *from = place_of(page);
            const int bytes = there(page) ? min(1 << run_log2, s.len - t * kTok - (lane << run_log2)) * HD : 0;
            const unsigned have = __ballot_sync(0xFFFFFFFFu, bytes > 0);
            if (!values) {
                // Eight tiles' places: what lies in tile n's, the scales of tile n - 8, has been read when the keys of tile n - 1 are being widened
                if (lane < 8) {
                    const float v = fmaxf(vs, 8.673617379884035e-19f);      // 2^-60
                    asm volatile("st.shared.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(R.smem + S::kScales + (n & 7) * 128 + lane * 16), "f"(ks),
                                 "f"(vs < 0.f ? -INFINITY : __log2f(v)), "f"(vs < 0.f ? 0.f : __fdividef(1.f, v)), "f"(0.f) : "memory");
                }
                __syncwarp();
                scales_of(next);
            }
#pragma unroll 1
            for (int h = 0; h < 2; h++) {
                const bool mine = lane >> (6 - run_log2) == h && bytes > 0;
                const int all = __reduce_add_sync(0xFFFFFFFFu, mine ? bytes : 0);
                good = good && R.wait_warp(read + h, (n & 1u) ^ 1u);
                if (!good) break;
                if (lane == 0) {
                    asm volatile("st.shared.u32 [%0], %1;" ::"r"(have_at + 4 * h), "r"(have) : "memory");
                    bar_expect(R.bars + 8 * (raw + h), all);
                }
                if (h) asked[1]++;
                else asked[0]++;
                __syncwarp();
                if (mine) bulk_in(ring + (lane << run_log2) * HD, from, bytes, R.bars + 8 * (raw + h));
            }
            page = next;
            next = page_of(t + 2);
            ahead(far);
            far = page_of(t + 1 + kAhead);
        }
        if (!good) break;
    }
    for (int h = 0; h < 2; h++)                         // what is under way arrives before the block may end
        if (asked[h]) bar_wait(R.bars + 8 * (raw + h), (asked[h] - 1) & 1u, kDrainLimit, R.gave_up + 4);
}

// ---- the cache's bytes -> fp16 operands.  Two warps widen keys, two values.  Eight neighbouring lanes have four pieces of 16 bytes of each of two rows, so that neither their
// loads nor their stores meet a bank twice.
template <int HD>
__device__ __forceinline__ void widen_role(const PrefixRoom &R, const Stretch *plan)
{
    using S = PrefixShape<HD>;
    constexpr int ROWS = 64 / (HD / 16);                // rows of a pass of both warps
    constexpr int N = 64 / ROWS, B = N < 8 ? N : 8;     // passes of half a tile, and of them at a time
    const int lane = threadIdx.x & 31, w = threadIdx.x / 32 - kSoftWarps, values = w >> 1;
    // HD 128: lanes 0 - 3 row 0 pieces 0 - 3, 4 - 7 row 1 pieces 4 - 7, 8 - 11 row 0 pieces 4 - 7, 12 - 15 row 1 pieces 0 - 3, 16 - 31 rows 2 and 3 likewise
    const int c = HD == 128 ? (lane & 3) + 4 * (((lane >> 2) ^ (lane >> 3)) & 1) : lane & 3;
    const int r0 = (w & 1) * (ROWS / 2) + (HD == 128 ? ((lane >> 2) & 1) + 2 * (lane >> 4) : lane >> 2);
    const uint32_t to = R.smem + (values ? S::kV : S::kK) + (uint32_t)(c >> 2) * 16384u;
    const uint32_t to0 = to + operand_at(r0, 2 * (c & 3)), to1 = to + operand_at(r0, 2 * (c & 3) + 1);
    const uint32_t own = R.smem + S::kRing + values * kTok * HD + r0 * HD + c * 16, have_at = R.smem + S::kHave + values * 8;
    const int full = values ? B_VFULL : B_KFULL, empty = values ? B_VEMPTY : B_KEMPTY, raw = values ? B_VRAW : B_KRAW, read = values ? B_VREAD : B_KREAD;
    const int run_log2 = R.run_log2, runs = kTok >> run_log2;
    unsigned n = 0;                                     // tiles so far
    Stretch s;
    for (unsigned run = 0; R.next(plan, run, s); R.done(run), run++) {
        for (int t = s.tile; t < s.end; t++, n++) {
            const int stage = n & 1, left = s.len - t * kTok;
            if (!R.wait_warp(empty + stage, ((n >> 1) & 1u) ^ 1u)) return;
#pragma unroll 1
            for (int h = 0; h < 2; h++) {
                if (!R.wait_warp(raw + h, n)) return;
                uint32_t have;                          // runs of the tile that were copied
                asm volatile("ld.shared.u32 %0, [%1];" : "=r"(have) : "r"(have_at + 4 * h) : "memory");
                const bool whole = have == (1u << runs) - 1 && left >= kTok;
#pragma unroll
                for (int q = 0; q < N; q += B) {
                    uint4 x[B];
#pragma unroll
                    for (int i = 0; i < B; i++) x[i] = lds128(own + (h * 64 + (q + i) * ROWS) * HD);
                    if (!whole) {
#pragma unroll
                        for (int i = 0; i < B; i++) {
                            const int at = h * 64 + (q + i) * ROWS + r0;
                            if (at >= left || !(have >> (at >> run_log2) & 1u)) x[i] = make_uint4(0u, 0u, 0u, 0u);
                        }
                    }
#pragma unroll
                    for (int i = 0; i < B; i++) {
                        uint32_t v[8];
                        widen4(x[i].x, v[0], v[1]);
                        widen4(x[i].y, v[2], v[3]);
                        widen4(x[i].z, v[4], v[5]);
                        widen4(x[i].w, v[6], v[7]);
                        const uint32_t on = stage * S::kOperand + (h * 64 + (q + i) * ROWS) * 128;
                        sts128(to0 + on, v[0], v[1], v[2], v[3]);
                        sts128(to1 + on, v[4], v[5], v[6], v[7]);
                    }
                }
                __syncwarp();
                if (lane == 0) R.arrive(read + h);
            }
            publish_shared();
            __syncwarp();
            if (lane == 0) R.arrive(full + stage);
        }
    }
}

// ---- the products, by one warp, of which one thread issues them; the others go the same way, so that the operands' addresses are a warp's, not a thread's.
// (With one thread going through all this, their computation took longer than the products.)
// Tensor memory: 128 columns of scores of either stream, which weights replace, then HD columns of values of either
template <int HD>
__device__ __forceinline__ void product_role(const PrefixArgs &P, const PrefixRoom &R, const Stretch *plan)
{
    using S = PrefixShape<HD>;
    constexpr uint32_t kScores = mma_shape(kTok, false), kValues = mma_shape(HD, true);
    const uint32_t tmem = kTmem, smem = R.smem, bars = R.bars;
    const bool one = elected();
    if (P.wait_lost && blockIdx.x == 0 && !R.wait_warp(B_DRAIN, 0)) return;      // nothing arrives there before the end
    unsigned n = 0, runs = 0, weights[2] = {0, 0};      // tiles and stretches so far; each stream's tiles of weights
    auto commit = [&](int bar) {
        if (one) mma_commit(bars + 8 * bar);
    };
    auto scores = [&](int j, int stage) {
        const uint32_t q = operand_along(smem + S::kQ + j * S::kOperand), k = operand_along(smem + S::kK + stage * S::kOperand), d = tmem + j * 128;
        if (one) {
#pragma unroll
            for (int i = 0; i < HD / 16; i++) {
                const uint32_t on = (i / 4) * 1024 + (i % 4) * 2;        // in 16 bytes
                mma_shared(d, q + on, k + on, kScores, i > 0);
            }
            mma_commit(bars + 8 * (B_SFULL + j));
        }
    };
    // a stream's values, as soon as either half of its weights is there
    auto values = [&](int j, int stage, bool first) {
        const uint32_t v = operand_across(smem + S::kV + stage * S::kOperand, 16384u), d = tmem + 256 + j * HD, w = tmem + j * 128;
        const unsigned turn = j ? weights[1]++ : weights[0]++;
        if (!R.wait_warp(B_PHALF + j, turn)) return false;
        tmem_after_sync();
        if (one) {
#pragma unroll
            for (int i = 0; i < kTok / 32; i++) mma_tmem(d, w + 8 * i, v + i * 128, kValues, i > 0 || !first);
        }
        if (!R.wait_warp(B_PFULL + j, turn)) return false;
        tmem_after_sync();
        if (one) {
#pragma unroll
            for (int i = kTok / 32; i < kTok / 16; i++) mma_tmem(d, w + 8 * i, v + i * 128, kValues, 1);
        }
        return true;
    };
    Stretch s;
    for (; R.next(plan, runs, s); R.done(runs), runs++) {
        const int m = s.end - s.tile;
        const bool turns = s.turns();
        if (!R.wait_warp(B_QFULL, runs) || !R.wait_warp(B_QFULL + 1, runs)) return;
        const unsigned base = n;
        const int lag = turns ? 2 : 1;
        // step i: the scores of tile i, behind the values of the tile `lag` in front, whose weights lie where the scores go
        for (int i = 0; i < m + lag; i++) {
            const unsigned kt = base + i, vt = base + i - lag;
            if (i < m && !R.wait_warp(B_KFULL + (kt & 1), kt >> 1)) return;
            if (i >= lag && !R.wait_warp(B_VFULL + (vt & 1), vt >> 1)) return;
            for (int j = turns ? i & 1 : 0; j < (turns ? (i & 1) + 1 : 2); j++) {
                if (i >= lag) {
                    if (!values(j, vt & 1, i < 2 * lag)) return;
                    if (i >= m) commit(B_OFULL + j);
                }
                if (i < m) scores(j, kt & 1);
            }
            if (i >= lag) commit(B_VEMPTY + (vt & 1));
            if (i < m) commit(B_KEMPTY + (kt & 1));
        }
        if (turns && m == 1) commit(B_OFULL + 1);       // a stream without a tile keeps step too
        n += m;
    }
}

// ---- two fp32 numbers at a time: half the instructions
struct Two { uint64_t v; };
__device__ __forceinline__ Two two(float lo, float hi) { Two r; asm("mov.b64 %0, {%1, %2};" : "=l"(r.v) : "f"(lo), "f"(hi)); return r; }
__device__ __forceinline__ void apart(Two a, float &lo, float &hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(a.v)); }
__device__ __forceinline__ Two fma2(Two a, Two b, Two c) { Two r; asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v)); return r; }
// (what lies below the normals counts as 0)
__device__ __forceinline__ Two add2(Two a, Two b) { Two r; asm("add.rn.ftz.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v)); return r; }
// 2^a without the special-function unit, which computes 16 a cycle and SM where a tile asks for 16384: a = n + f, n whole, |f| <= 1/2, and the
// polynomial of degree 5 that is nearest to 2^f there (found by exchange; in 32 bits 2^-22 relative, as the unit's).  Below 2^-126 (-infinity) a
// number below the normals comes out, which add2 and the conversion to fp16 take as 0: value scales reach 2^118, so 2^-126 times an inverse scale could outweigh the sum.  No NaN comes out.
__device__ __forceinline__ void pow2_two(Two a, float &lo, float &hi)
{
    float x, y;
    apart(a, x, y);
    a = two(fmaxf(x, -126.75f), fmaxf(y, -126.75f));      // n = -127, f = 1/4
    const float big = 12582912.f;                       // 1.5 * 2^23: what is added to it is rounded to a whole number
    const Two m = add2(a, two(big, big)), n = add2(m, two(-big, -big)), f = fma2(n, two(-1.f, -1.f), a);
    Two r = fma2(f, two(0.0013276472454890609f, 0.0013276472454890609f), two(0.009675540961325169f, 0.009675540961325169f));
    r = fma2(r, f, two(0.05550713092088699f, 0.05550713092088699f));
    r = fma2(r, f, two(0.24022120237350464f, 0.24022120237350464f));
    r = fma2(r, f, two(0.6931469440460205f, 0.6931469440460205f));
    r = fma2(r, f, two(1.0000001192092896f, 1.0000001192092896f));
    float mx, my;
    apart(m, mx, my);
    apart(r, x, y);
    lo = __uint_as_float(__float_as_uint(x) + (__float_as_uint(mx) << 23));
    hi = __uint_as_float(__float_as_uint(y) + (__float_as_uint(my) << 23));
}
// largest of three, NaN if one of them is
__device__ __forceinline__ float max3(float a, float b, float c)
{
    float r;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
__device__ __forceinline__ float score_of(const uint32_t (&x)[8][16], int k) { return __uint_as_float(x[k / 16][k % 16]); }

// ---- the rows: thread r of a stream owns row r of its 128
template <typename T, int HD>
__device__ __forceinline__ bool rows_run(const PrefixArgs &P, const PrefixRoom &R, const Stretch &s, int j, unsigned first, unsigned &tiles, float (&zl)[2])
{
    using S = PrefixShape<HD>;
    const AttnArgs &A = P.a;
    const int warp = threadIdx.x / 32 % 4, lane = threadIdx.x & 31, r = 32 * warp + lane;
    const int at = s.row0 + (s.turns() ? 0 : 128 * j) + r;
    const bool live = at < s.members;
    const bool any = s.row0 + (s.turns() ? 0 : 128 * j) + 32 * warp < s.members;       // of the warp
    const int count = s.tiles_of(j);
    const uint32_t lanes = (uint32_t)(32 * warp) << 16, score = kTmem + lanes + j * 128, value = kTmem + lanes + 256 + j * HD;
    // The query row, as in the kernel of a sequence's own tokens: its largest finite element goes to [2^13, 2^14), and the power of two and the sign of
    // sm_scale to the factor of the scores.
    float up;
    {
        const uint16_t *src = A.q + (int64_t)(s.first + at / A.group) * A.qs + (int64_t)(s.kv * A.group + at % A.group) * HD;
        float top = 0.f;
#pragma unroll 2
        for (int i = 0; i < HD / 8; i++) {
            const uint4 raw = live ? *reinterpret_cast<const uint4 *>(src + 8 * i) : make_uint4(0u, 0u, 0u, 0u);
            const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
            for (int x = 0; x < 4; x++) {
                const float2 f = pair_to_f32<T>(w[x]);
                top = fmaxf(top, fmaxf(fabsf(f.x) < INFINITY ? fabsf(f.x) : 0.f, fabsf(f.y) < INFINITY ? fabsf(f.y) : 0.f));
            }
        }
        int e = top > 0.f ? ((int)(__float_as_uint(top) >> 23) - 127) : 0;
        e = max(-100, e) - 13;
        const float down = A.scale_log2 < 0.f ? -exp2f((float)-e) : exp2f((float)-e);
        up = fabsf(A.scale_log2) * exp2f((float)e);
        const uint32_t q = R.smem + S::kQ + j * S::kOperand;
#pragma unroll 2
        for (int i = 0; i < HD / 8; i++) {
            const uint4 raw = live ? *reinterpret_cast<const uint4 *>(src + 8 * i) : make_uint4(0u, 0u, 0u, 0u);
            const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
            uint32_t o[4];
#pragma unroll
            for (int x = 0; x < 4; x++) {
                const float2 f = pair_to_f32<T>(w[x]);
                o[x] = f16x2_of(f.x * down, f.y * down);
            }
            sts128(q + (i / 8) * 16384 + operand_at(r, i % 8), o[0], o[1], o[2], o[3]);
        }
        publish_shared();
        __syncwarp();
        if (lane == 0) R.arrive(B_QFULL + j);
    }
    float &z = zl[0], &l = zl[1];
    float l32 = 0.f;                                    // sums in two levels, as there
    z = -INFINITY;
    l = 0.f;
    const int step = s.turns() ? 2 : 1;
    int left = s.len - s.tile * kTok;                 // tokens of the tile that exist
    if (s.turns()) left -= j * kTok;
    unsigned place = first + (s.turns() ? j : 0);       // the tile's number
    for (int i = 0; i < count; i++, tiles++, place += step, left -= step * kTok) {
        const uint32_t scales = R.smem + S::kScales + (place & 7) * 128;
        auto scale_of = [&](int g) {
            float4 v;
            asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(scales + 16 * g) : "memory");
            v.x = fmaxf(v.x * up, 1.1754944e-38f);      // never 0, which times -infinity would be no number
            return v;
        };
        if (!R.wait_warp(B_SFULL + j, tiles)) return false;
        tmem_after_sync();
        if (any) {
            if (left < kTok) {
                // a last tile: -infinity, so weight 0, for what lies behind the end.  In a loop of its own: what a tile goes through has to fit the instruction cache
#pragma unroll 1
                for (int c = left > 0 ? left / 16 : 0; c < 8; c++) {
                    uint32_t y[16];
                    tmem_ld16(score + 16 * c, y);
                    tmem_wait_ld(y);
#pragma unroll
                    for (int k = 0; k < 16; k++)
                        if (16 * c + k >= left) y[k] = 0xFF800000u;
                    tmem_st16(score + 16 * c, y);
                }
                tmem_wait_st();
            }
            uint32_t x[8][16];                          // the row's scores
            auto read_scores = [&]() {
#pragma unroll
                for (int c = 0; c < 8; c++) tmem_ld16(score + 16 * c, x[c]);
                tmem_wait_ld(x[0]);
#pragma unroll
                for (int c = 1; c < 8; c++) tmem_named(x[c]);
            };
            read_scores();
            float top = -INFINITY;
#pragma unroll
            for (int g = 0; g < 8; g++) {
                float m0 = score_of(x, 16 * g), m1 = score_of(x, 16 * g + 1);
#pragma unroll
                for (int k = 2; k < 14; k += 4) {
                    m0 = max3(m0, score_of(x, 16 * g + k), score_of(x, 16 * g + k + 1));
                    m1 = max3(m1, score_of(x, 16 * g + k + 2), score_of(x, 16 * g + k + 3));
                }
                m0 = max3(m0, m1, score_of(x, 16 * g + 14));
                m0 = max3(m0, m0, score_of(x, 16 * g + 15));
                const float4 sc = scale_of(g);
                top = max3(top, top, fmaf(m0, sc.x, sc.y));
            }
            // a score that is no number, or infinite, makes the row NaN, whichever way its weight is computed
            if (!(top < INFINITY)) l = __int_as_float(0x7FC00000);
            // A new reference where a weight would pass 2^15.9; it brings the largest to 2^15.  (Less, with more room to the next time, costs the small weights their bits: with 2^14
            // 1 to 2 % less time, with 2^7 3 to 5 %.  Moving the other rows of the warp along would save 0.7 %, but a row's bits would depend on its neighbours.)
            if (__any_sync(0xFFFFFFFFu, __fsub_ru(top, kMostLift) > z)) {
                const float n = __fsub_ru(top, kMostLift) > z ? __fsub_ru(top, kLift) : z;
                const float a = n == -INFINITY ? 1.f : ex2(z - n);
                z = n;
                l *= a;
                l32 *= a;
                if (i > 0) {                            // this stream's products in front are done: their end came before the scores'
                    constexpr int N = HD / 32;          // half of the columns at a time (all at once, 3 behind 262143 with heads of 64: 156 us, not 143)
#pragma unroll 1
                    for (int c = 0; c < HD / (16 * N); c++) {
                        uint32_t o[N][16];
#pragma unroll
                        for (int h = 0; h < N; h++) tmem_ld16(value + 16 * (N * c + h), o[h]);
                        tmem_wait_ld(o[0]);
#pragma unroll
                        for (int h = 1; h < N; h++) tmem_named(o[h]);
#pragma unroll
                        for (int h = 0; h < N; h++) {
#pragma unroll
                            for (int k = 0; k < 16; k++) o[h][k] = __float_as_uint(__uint_as_float(o[h][k]) * a);
                            tmem_st16(value + 16 * (N * c + h), o[h]);
                        }
                    }
                    read_scores();                      // again: their registers were needed (16 columns at a time without: 342 us, not 336, for 256 behind 32768)
                }
            }
            const float ref = z == -INFINITY ? 0.f : z;
            // weights of tokens 32 c .. 32 c + 31 (two groups of scores), over scores that have been read
            auto weigh = [&](auto any_coarse, bool coarse, const uint32_t (&y0)[16], const uint32_t (&y1)[16], int c) {
                uint32_t w[16];
#pragma unroll
                for (int h = 0; h < 2; h++) {
                    const uint32_t(&y)[16] = h ? y1 : y0;
                    const float4 sc = scale_of(2 * c + h);
                    const bool first = decltype(any_coarse)::value && coarse;
                    const float times = first ? 1.f : sc.x, shift = first ? -ref : sc.y - ref;
                    const Two ff = two(times, times), ss = two(shift, shift);
                    Two sum = two(0.f, 0.f);
#pragma unroll
                    for (int k = 0; k < 8; k++) {
                        float p = __uint_as_float(y[2 * k]), q = __uint_as_float(y[2 * k + 1]);
                        if (first) p = fmaf(p, sc.x, sc.y), q = fmaf(q, sc.x, sc.y);
                        const Two a = fma2(two(p, q), ff, ss);
                        float e0, e1;
                        if (k % 4 == 3) {               // a quarter: the special-function unit and the others take about as long
                            pow2_two(a, e0, e1);
                        } else {
                            apart(a, e0, e1);
                            e0 = ex2(e0);
                            e1 = ex2(e1);
                        }
                        sum = add2(sum, two(e0, e1));
                        w[8 * h + k] = f16x2_of(e0, e1);
                    }
                    float s0, s1;
                    apart(sum, s0, s1);
                    l32 = fmaf(s0 + s1, sc.z, l32);
                }
                tmem_st16(score + 16 * c, w);
                if (c == 1) {                           // half of the weights: their products may begin
                    tmem_wait_st();
                    tmem_before_sync();
                    __syncwarp();
                    if (lane == 0) R.arrive(B_PHALF + j);
                }
            };
            // A weight is 2^(score x scale + (log2 - reference)), the product not rounded.  Where fp32 is coarse at the reference's size the rounding of that sum could lift it by
            // any amount, so there the score is rounded first, as for the reference itself: no weight is above what the reference allows then.
            const bool coarse = fabsf(ref) >= kCoarse;
            if (!__any_sync(0xFFFFFFFFu, coarse)) {
#pragma unroll
                for (int c = 0; c < 4; c++) weigh(std::false_type{}, false, x[2 * c], x[2 * c + 1], c);
            } else {
#pragma unroll 1
                for (int c = 0; c < 4; c++) {           // rare, so little code: the scores are read anew
                    uint32_t y0[16], y1[16];
                    tmem_ld16(score + 32 * c, y0);
                    tmem_ld16(score + 32 * c + 16, y1);
                    tmem_wait_ld(y0);
                    tmem_named(y1);
                    weigh(std::true_type{}, coarse, y0, y1, c);
                }
            }
            tmem_wait_st();
            if ((i & 31) == 31) {
                l += l32;
                l32 = 0.f;
            }
        } else if (lane == 0) {
            R.arrive(B_PHALF + j);
        }
        tmem_before_sync();
        __syncwarp();
        if (lane == 0) R.arrive(B_PFULL + j);
    }
    l += l32;
    return true;
}

template <typename T, int HD>
__device__ __forceinline__ void rows_role(const PrefixArgs &P, const PrefixRoom &R, const Stretch *plan)
{
    const int j = threadIdx.x / 128, warp = threadIdx.x / 32 % 4, lane = threadIdx.x & 31, r = 32 * warp + lane;
    unsigned runs = 0, tiles = 0, all = 0;              // stretches, tiles of this stream and of both, so far
    Stretch s;
    for (; R.next(plan, runs, s); R.done(runs), runs++) {
        float zl[2];
        const int count = s.tiles_of(j);
        if (!rows_run<T, HD>(P, R, s, j, all, tiles, zl) || !R.wait_warp(B_OFULL + j, runs)) return;
        all += s.end - s.tile;
        const int row = s.turns() ? r : 128 * j + r;
        const long long place = s.at + (s.turns() ? j * s.rows : 128 * j) + r;
        const bool live = row < s.rows && place < P.n_rows;
        float *to = P.part_v + place * HD;
        if (live) {
            P.part_z[place] = zl[0];
            P.part_l[place] = zl[1];
        }
        if (count) {
            tmem_after_sync();
#pragma unroll 1
            for (int c = 0; c < HD / 16; c++) {
                uint32_t x[16];
                tmem_ld16(kTmem + ((uint32_t)(32 * warp) << 16) + 256 + j * HD + 16 * c, x);
                tmem_wait_ld(x);
                if (live)
#pragma unroll
                    for (int k = 0; k < 16; k += 4) *reinterpret_cast<uint4 *>(to + 16 * c + k) = make_uint4(x[k], x[k + 1], x[k + 2], x[k + 3]);
            }
            tmem_before_sync();
        } else if (live) {
#pragma unroll 1
            for (int k = 0; k < HD; k += 4) *reinterpret_cast<uint4 *>(to + k) = make_uint4(0u, 0u, 0u, 0u);
        }
    }
}

template <typename T, int HD>
__global__ void __launch_bounds__(kPrefixThreads, 1) prefix_kernel(const __grid_constant__ PrefixArgs P)
{
    using S = PrefixShape<HD>;
    extern __shared__ __align__(1024) uint8_t prefix_smem[];
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    // the groups' prefix sums lie where operands come later
    long long *units = reinterpret_cast<long long *>(prefix_smem);
    long long *rows = units + PF_PREFIX_MAX_GROUPS + 1;
    group_prefix(P, units, rows, rows + PF_PREFIX_MAX_GROUPS + 1);
    const int blocks = prefix_share(units[P.a.n_groups], own_tiles(P.a, rows + PF_PREFIX_MAX_GROUPS + 1), gridDim.x);
    Walk walk;
    if (!walk.begin(P, units, rows, blocks)) return;
    uint32_t *words = reinterpret_cast<uint32_t *>(prefix_smem + S::kBars + 8 * B_COUNT);
    uint32_t *gave_up = words + 1;
    Stretch *plan = reinterpret_cast<Stretch *>(prefix_smem + S::kPlan);
    const int warp = threadIdx.x >> 5;
    const PrefixRoom R{smem_addr(prefix_smem), smem_addr(prefix_smem) + S::kBars, smem_addr(gave_up), P.wait_limit, min(31 - __clz(P.a.c.page), 6)};
    if (threadIdx.x == 0) {
        words[1] = words[2] = 0;
        for (int i = 0; i < 2; i++) {
            bar_init(R.bars + 8 * (B_KFULL + i), kWidenWarps / 2);
            bar_init(R.bars + 8 * (B_VFULL + i), kWidenWarps / 2);
            bar_init(R.bars + 8 * (B_KEMPTY + i), 1);
            bar_init(R.bars + 8 * (B_VEMPTY + i), 1);
            bar_init(R.bars + 8 * (B_KRAW + i), 1);
            bar_init(R.bars + 8 * (B_VRAW + i), 1);
            bar_init(R.bars + 8 * (B_KREAD + i), kWidenWarps / 2);
            bar_init(R.bars + 8 * (B_VREAD + i), kWidenWarps / 2);
            bar_init(R.bars + 8 * (B_PLAN + i), 1);
            bar_init(R.bars + 8 * (B_DONE + i), kSoftWarps + kWidenWarps + 3);
            bar_init(R.bars + 8 * (B_QFULL + i), 4);
            bar_init(R.bars + 8 * (B_SFULL + i), 1);
            bar_init(R.bars + 8 * (B_PHALF + i), 4);
            bar_init(R.bars + 8 * (B_PFULL + i), 4);
            bar_init(R.bars + 8 * (B_OFULL + i), 1);
        }
        bar_init(R.bars + 8 * B_DRAIN, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == kSoftWarps + kWidenWarps) tmem_alloc(smem_addr(words), 512);
    tmem_before_sync();
    __syncthreads();
    tmem_after_sync();
    if (warp < kSoftWarps) {
        take_registers<kSoftRegs>();
        rows_role<T, HD>(P, R, plan);
    } else if (warp < kSoftWarps + kWidenWarps) {
        leave_registers<kWidenRegs>();
        widen_role<HD>(R, plan);
    } else {
        leave_registers<kProductRegs>();
        if (warp == kSoftWarps + kWidenWarps + 3) {
            product_role<HD>(P, R, plan);
            // whatever was begun is done before the block gives its memory back
            __syncwarp();
            if (elected()) mma_commit(R.bars + 8 * B_DRAIN);
            const uint32_t alone = smem_addr(words + 2);
            bar_wait(R.bars + 8 * B_DRAIN, 0, kDrainLimit, alone);
        } else if (threadIdx.x == 32 * (kSoftWarps + kWidenWarps)) {
            plan_role(P, R, walk, plan);
        } else if (warp > kSoftWarps + kWidenWarps) {
            copy_role<HD>(P, R, plan, warp & 1);
        }
        __syncwarp();
    }
    tmem_before_sync();
    __syncthreads();
    if (warp == kSoftWarps + kWidenWarps) tmem_free(words[0], 512);
    if (threadIdx.x == 0) P.status[blockIdx.x] = words[1];      // a wait that ran out: the join makes NaN of what this block had to do
}

// ------------------------------------------------------------------ the join
// A warp joins the parts of one row: what its own tokens left (one part where a single block finished them, else one of each block), and
// one of each piece that goes through the prefix.
// (Four blocks an SM, so 64 registers: with 48, which the compiler takes for more of them, 2 us more for 4 behind 777 and 6 for 3 behind 262143.)
template <typename T, int HD, int NB>
__global__ void __launch_bounds__(256, 4) prefix_join_kernel(const __grid_constant__ PrefixArgs P, const int own_grid, const int prefix_grid)
{
    using S = AttnShape<HD, NB>;
    constexpr int V = HD / 32;
    const AttnArgs &A = P.a;
    extern __shared__ __align__(128) uint8_t smem[];
    long long *units = reinterpret_cast<long long *>(smem);
    long long *rows = units + P.a.n_groups + 1;
    int *prefix = reinterpret_cast<int *>(rows + P.a.n_groups + 1);
    __shared__ int warp_sum[8];
    __shared__ long long scratch[64];
    group_prefix(P, units, rows, scratch);
    tile_prefix(A, prefix, warp_sum);
    const int lane = threadIdx.x & 31;
    const long long total = units[P.a.n_groups], own_total = (long long)prefix[A.n_seq] * A.jobs_per_seq;
    const int share = prefix_share(total, own_total, prefix_grid), n_pieces = total ? pieces_of(total, share) : 0;
    const int each = share ? pieces_each(n_pieces, share) : 1, own_blocks = own_total ? blocks_used(own_total, own_grid - share) : 1;
    const int next = piece_rows(A.n_seq, A.group);
    bool waited = false;                          // where a warp's first row has its parts follows from the lengths alone
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
        long long at = 0;                         // the first's row; the other stream's is `apart` further on, the next piece's `next`
        int n_pre = 0, p0 = 0, both = 1, apart = 0;      // both: parts of a piece
        if (total) {
            const int gi = P.a.cu ? last_at(P.a.cu, P.a.n_groups, b) : 0;
            const Group g = group_of(P.a, gi);
            if (g.tiles && b >= g.first && b < g.first + g.rows / A.group) {
                const int r = (b - g.first) * A.group + gh, no = kv * g.row_tiles + r / kRows;
                apart = g.rows - r / kRows * kRows;
                both = apart <= 128 ? 2 : 1;
                const long long begin = units[gi] + (long long)no * g.tiles;
                p0 = piece_of(total, n_pieces, begin);
                n_pre = piece_of(total, n_pieces, begin + g.tiles - 1) - p0 + 1;
                at = rows[gi] + (long long)kv * head_rows(g) + r + (long long)p0 * next;
                if (at + (long long)(n_pre - 1) * next + (both == 2 ? apart : 0) >= P.n_rows) n_pre = 0;
                n_pre *= both;
            }
        }
        if (!waited) asm volatile("griddepcontrol.wait;" ::: "memory");
        waited = true;
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
                const int no = i - n_own, piece = both == 2 ? no >> 1 : no;
                const long long place = at + (long long)piece * next + (both == 2 && (no & 1) ? apart : 0);
                from = P.part_v + place * HD;
                z = P.part_z[place];
                l = P.status[(p0 + piece) / each] ? __int_as_float(0x7FC00000) : P.part_l[place];
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
            // what the unrolled loop reads past the last part is the first one, with weight 0: no branch between the loads
            const int count = min(32, n - i0);
            const unsigned long long any = __shfl_sync(0xFFFFFFFFu, (unsigned long long)from, 0), mine = from ? (unsigned long long)from : any;
            const float weight = from ? f : 0.f;
#pragma unroll 8
            for (int k = 0; k < (count + 7) / 8 * 8; k++) {
                const float *p = (const float *)__shfl_sync(0xFFFFFFFFu, mine, k) + lane * V;
                const float w = __shfl_sync(0xFFFFFFFFu, weight, k);
                if (V == 4) {
                    const float4 y = *reinterpret_cast<const float4 *>(p);
                    v[0] = fmaf(y.x, w, v[0]);
                    v[1] = fmaf(y.y, w, v[1]);
                    v[2 % V] = fmaf(y.z, w, v[2 % V]);
                    v[3 % V] = fmaf(y.w, w, v[3 % V]);
                } else {
                    const float2 y = *reinterpret_cast<const float2 *>(p);
                    v[0] = fmaf(y.x, w, v[0]);
                    v[1] = fmaf(y.y, w, v[1]);
                }
            }
        }
        const float inv = sum == 0.f ? 0.f : 1.f / sum;      // (a sum that is not a number stays one)
        uint32_t *dst = reinterpret_cast<uint32_t *>(A.out + b * A.os + (int64_t)head * HD) + lane * V / 2;
#pragma unroll
        for (int k = 0; k < V; k += 2) dst[k / 2] = pair_of_f32<T>(v[k] * inv, v[k + 1] * inv);
        if (A.lse && lane == 0) A.lse[row] = sum == 0.f ? -INFINITY : (top + log2f(sum)) * kLn2;
    }
    if (!waited) asm volatile("griddepcontrol.wait;" ::: "memory");      // what follows on the stream waits for this kernel only
    if (P.report && blockIdx.x == 0 && threadIdx.x < 32) {
        unsigned lost = 0;
        for (int i = lane; i < (n_pieces + each - 1) / each; i += 32) lost |= P.status[i];      // of the blocks with work
        lost = __any_sync(0xFFFFFFFFu, lost != 0);
        if (lane == 0) *P.report = (int)lost;
    }
}

// ------------------------------------------------------------------ host
struct PrefixSizes {
    size_t own_v, own_z, own_l, status, part_v, part_z, part_l, bytes;      // offsets in the workspace, and its size
    long long n_rows;
};
static PrefixSizes prefix_sizes(int hd, int page, int n_kv, int n_seq, int n_heads, int n_groups, int pcols, int sms)
{
    PrefixSizes s;
    auto up = [](size_t x) { return (x + 255) & ~(size_t)255; };
    const size_t rows = (size_t)n_seq * n_heads;
    s.own_v = up(attention_workspace_bytes(hd, sms));
    s.own_z = s.own_v + up(rows * hd * 4);
    s.own_l = s.own_z + up(rows * 4);
    s.status = s.own_l + up(rows * 4);
    s.part_v = s.status + up((size_t)sms * 4);
    const long long tiles = ((long long)pcols * page + kTok - 1) / kTok;
    const long long tasks = (long long)n_kv * (((long long)n_seq * (n_heads / n_kv)) / kRows + n_groups);
    const long long wanted = tasks * tiles / kMostTiles + sms, pieces = wanted < (long long)kMostPieces * sms ? wanted : (long long)kMostPieces * sms;
    // all tasks' rows (of n_groups unknown sizes), and what the pieces are apart
    const long long all = 2 * (long long)rows < tasks * kRows ? 2 * (long long)rows : tasks * kRows;
    s.n_rows = all + pieces * piece_rows(n_seq, n_heads / n_kv);
    s.part_z = s.part_v + up((size_t)s.n_rows * hd * 4);
    s.part_l = s.part_z + up((size_t)s.n_rows * 4);
    s.bytes = s.part_l + up((size_t)s.n_rows * 4);
    return s;
}

template <typename T, int HD, int NB>
static int prefix_launch(PrefixArgs p, int device, int sms, cudaStream_t st)
{
    using S = AttnShape<HD, NB>;
    AttnArgs &a = p.a;
    a.row_blocks = (a.group + S::kHeads - 1) / S::kHeads;
    a.jobs_per_seq = a.c.n_kv * a.row_blocks;
    const size_t groups = (size_t)(p.a.n_groups + 1) * 16, own = ((size_t)a.n_seq + 1) * 4;
    const size_t smem0 = PrefixShape<HD>::kBytes, smem1 = (size_t)S::kWarps * S::kWarpBytes + own, smem2 = groups + own;
    PF_CUDA_TRY(ensure_dynamic_smem((const void *)prefix_kernel<T, HD>, device, smem0), "prefix_kernel shared memory");
    PF_CUDA_TRY(ensure_dynamic_smem((const void *)attention_kernel<T, HD, NB, true>, device, smem1), "attention_kernel shared memory");
    PF_CUDA_TRY(ensure_dynamic_smem((const void *)prefix_join_kernel<T, HD, NB>, device, smem2), "prefix_join_kernel shared memory");
    prefix_kernel<T, HD><<<sms, kPrefixThreads, smem0, st>>>(p);
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

extern "C" int pf_prefix_attention_status(const pf_kv_cache_t *cache, int32_t dtype, int32_t n_seq, int32_t n_heads, const void *d_q, int64_t q_stride,
                                          const int32_t *d_len, const int32_t *d_table, int32_t table_cols, int32_t n_groups, const int32_t *d_cu_seqs,
                                          const int32_t *d_prefix_len, const int32_t *d_prefix_table, int32_t prefix_cols, float sm_scale, void *d_out,
                                          int64_t out_stride, float *d_lse, int32_t *d_status, void *d_workspace, size_t workspace_bytes, void *stream)
{
    cudaStream_t st = (cudaStream_t)stream;
    auto complete = [&]() -> int {                      // calls without a wait inside
        if (d_status) PF_CUDA_TRY(cudaMemsetAsync(d_status, 0, 4, st), "pf_prefix_attention status");
        return PF_OK;
    };
    if (!kv_cache_ok(cache) || (dtype != PF_DT_BF16 && dtype != PF_DT_F16)) return PF_EINVAL;
    if (n_seq < 0 || n_seq > PF_ATTN_MAX_SEQ || n_heads < 0 || table_cols < 0 || (int64_t)table_cols * cache->page >= (1ll << 31)) return PF_ERANGE;
    if (n_groups < 0 || n_groups > PF_PREFIX_MAX_GROUPS || prefix_cols < 0) return PF_ERANGE;
    if ((int64_t)prefix_cols * cache->page > PF_PREFIX_MAX_TOKENS) return PF_ERANGE;      // tile numbers times 128, a few tiles past the end, fit 32 bits
    const int64_t tiles = ((int64_t)table_cols * cache->page + kTile - 1) / kTile;      // as in pf_decode_attention
    if ((int64_t)n_seq * tiles >= (1ll << 31)) return PF_ERANGE;
    if ((int64_t)n_seq * n_heads >= (1ll << 30)) return PF_ERANGE;
    if (n_heads % cache->n_kv != 0 || !isfinite(sm_scale) || (uintptr_t)d_status % 4) return PF_EINVAL;
    if (n_seq == 0 || n_heads == 0) return complete();
    if (!d_q || !d_out || !d_len || (!d_table && table_cols > 0) || !aligned16(d_q) || !aligned16(d_out)) return PF_EINVAL;
    if (n_groups > 0 && ((!d_cu_seqs && n_groups > 1) || !d_prefix_len || (!d_prefix_table && prefix_cols > 0))) return PF_EINVAL;
    if ((uintptr_t)d_len % 4 || (uintptr_t)d_table % 4 || (uintptr_t)d_lse % 4 || (uintptr_t)d_cu_seqs % 4 || (uintptr_t)d_prefix_len % 4 || (uintptr_t)d_prefix_table % 4)
        return PF_EINVAL;
    const int64_t row = (int64_t)n_heads * cache->hd;
    if (q_stride < row || out_stride < row || q_stride % 8 || out_stride % 8) return PF_EINVAL;
    if (n_groups == 0 || prefix_cols == 0) {
        const int rc = pf_decode_attention(cache, dtype, n_seq, n_heads, d_q, q_stride, d_len, d_table, table_cols, sm_scale, d_out, out_stride, d_lse, d_workspace,
                                           workspace_bytes, stream);
        return rc == PF_OK ? complete() : rc;
    }
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
    a.cu = d_cu_seqs; a.plen = d_prefix_len; p.ptable = d_prefix_table;
    a.n_groups = n_groups; a.pcols = prefix_cols; p.n_rows = z.n_rows;
    p.status = (uint32_t *)(ws + z.status);
    p.part_v = (float *)(ws + z.part_v); p.part_z = (float *)(ws + z.part_z); p.part_l = (float *)(ws + z.part_l);
    p.wait_limit = g_wait_limit;
    p.wait_lost = g_wait_lost;
    p.report = d_status;
    return dtype == PF_DT_BF16 ? prefix_launch<Bf16>(p, device, sms, st) : prefix_launch<F16>(p, device, sms, st);
}

extern "C" int pf_prefix_attention(const pf_kv_cache_t *cache, int32_t dtype, int32_t n_seq, int32_t n_heads, const void *d_q, int64_t q_stride,
                                   const int32_t *d_len, const int32_t *d_table, int32_t table_cols, int32_t n_groups, const int32_t *d_cu_seqs,
                                   const int32_t *d_prefix_len, const int32_t *d_prefix_table, int32_t prefix_cols, float sm_scale, void *d_out,
                                   int64_t out_stride, float *d_lse, void *d_workspace, size_t workspace_bytes, void *stream)
{
    return pf_prefix_attention_status(cache, dtype, n_seq, n_heads, d_q, q_stride, d_len, d_table, table_cols, n_groups, d_cu_seqs, d_prefix_len, d_prefix_table,
                                      prefix_cols, sm_scale, d_out, out_stride, d_lse, nullptr, d_workspace, workspace_bytes, stream);
}

extern "C" int pf_prefix_waits(uint32_t polls, uint32_t lost)
{
    if (polls > (1u << 21) || lost > 1) return PF_ERANGE;
    g_wait_limit = polls ? polls : kWaitLimit;
    g_wait_lost = lost;
    return PF_OK;
}
