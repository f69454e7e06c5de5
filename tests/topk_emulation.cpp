// Runs the block top-k of pf_topk.cuh on the host: every thread of the block is a coroutine, which runs until it meets a
// collective; the next one to run is drawn at random, now and then with some warps held back as long as others can
// go on.  So threads see each other's writes to shared memory in orders that a GPU produces seldom.  A barrier that is
// completed by threads that stand at different places of the source ends the run: on a GPU that is undefined.
//
// topk_walk(keys, n, k, seed, out): the k best of n distinct keys into out, by a block of 1024 threads.  Returns how many, or
// -1 for a barrier met at different places, -2 for a collective that not all of its threads reach.
#include <ucontext.h>

#include <cstdint>
#include <cstring>
#include <random>
#include <vector>

namespace emu {
constexpr int kThreads = 1024, kWarps = kThreads / 32;
constexpr size_t kStack = 32768;
struct Dim { unsigned int x; };
struct Thread {
    ucontext_t at;
    std::vector<char> stack;
    int place = 0;                    // line of the collective it waits in, 0: runnable, -1: done
    bool block_wide = false;
    unsigned long long in = 0, out = 0;
};
std::vector<Thread> threads;
ucontext_t scheduler;
int current = 0, failure = 0;
Dim tid, dim{kThreads};

// wait in a collective with a value; what it gives back
unsigned long long collective(int line, bool block_wide, unsigned long long in)
{
    Thread &t = threads[current];
    t.place = line;
    t.block_wide = block_wide;
    t.in = in;
    swapcontext(&t.at, &scheduler);
    return t.out;
}
enum { kBarrier, kCount, kBallot, kShfl, kShflXor };
int kind_of_line[4096], arg_of_thread[kThreads];
unsigned long long call(int kind, int line, bool block_wide, unsigned long long in, int arg = 0)
{
    kind_of_line[line] = kind;
    arg_of_thread[current] = arg;
    return collective(line, block_wide, in);
}
void finish(int first, int n)         // all n threads from `first` on wait in the same collective: serve it
{
    const int kind = kind_of_line[threads[first].place];
    unsigned long long count = 0, mask = 0;
    for (int i = 0; i < n; i++) {
        count += threads[first + i].in != 0;
        if (n == 32 && threads[first + i].in) mask |= 1ull << i;
    }
    for (int i = 0; i < n; i++) {
        Thread &t = threads[first + i];
        const int arg = arg_of_thread[first + i];
        t.out = kind == kCount ? count : kind == kBallot ? mask : kind == kShfl ? threads[first + arg].in : kind == kShflXor ? threads[first + (i ^ arg)].in : 0;
    }
    for (int i = 0; i < n; i++) threads[first + i].place = 0;
}
}  // namespace emu

#define threadIdx emu::tid
#define blockDim emu::dim
#define __device__
#define __forceinline__ inline
#define __syncthreads() ((void)emu::call(emu::kBarrier, __LINE__, true, 0))
#define __syncthreads_count(p) ((int)emu::call(emu::kCount, __LINE__, true, (p) ? 1 : 0))
#define __ballot_sync(m, p) ((unsigned)emu::call(emu::kBallot, __LINE__, false, (p) ? 1 : 0))
#define __shfl_sync(m, v, l) ((decltype((v) + 0))emu::call(emu::kShfl, __LINE__, false, (unsigned long long)(v), (l)))
#define __shfl_xor_sync(m, v, l) ((decltype((v) + 0))emu::call(emu::kShflXor, __LINE__, false, (v), (l)))
static int __ffs(unsigned v) { return __builtin_ffs((int)v); }
static int __popc(unsigned v) { return __builtin_popcount(v); }
template <typename T> static T atomicAdd(T *p, T v)
{
    const T old = *p;
    *p = old + v;
    return old;
}

#include "pf_topk.cuh"

namespace {
const unsigned long long *g_in;
unsigned int g_n;
int g_k, g_count;
unsigned long long g_thr, g_buf[pf::kTopkCap];

void body()
{
    pf::tk_walk<pf::kTopkCap / 2 / emu::kThreads>(g_in, 0u, g_n, g_buf, &g_count, &g_thr, g_k);
    emu::threads[emu::current].place = -1;
    swapcontext(&emu::threads[emu::current].at, &emu::scheduler);
}
}  // namespace

extern "C" int topk_walk(const unsigned long long *keys, unsigned int n, int k, unsigned int seed, unsigned long long *out)
{
    using namespace emu;
    std::mt19937 rng(seed);
    g_in = keys;
    g_n = n;
    g_k = k;
    g_count = 0;
    g_thr = 0;
    threads.clear();
    threads.resize(kThreads);
    for (Thread &t : threads) {
        t.stack.resize(kStack);
        getcontext(&t.at);
        t.at.uc_stack.ss_sp = t.stack.data();
        t.at.uc_stack.ss_size = kStack;
        t.at.uc_link = &scheduler;
        makecontext(&t.at, body, 0);
    }
    auto serve_warp = [&](int w) {    // a warp whose 32 threads wait in one warp collective
        const int line = threads[w * 32].place;
        if (line <= 0 || threads[w * 32].block_wide) return false;
        for (int i = 1; i < 32; i++)
            if (threads[w * 32 + i].place != line) return false;
        finish(w * 32, 32);
        return true;
    };
    std::vector<int> ready;
    uint32_t held = 0;                // warps that run only when no other can
    for (;;) {
        ready.clear();
        for (int pass = 0; pass < 2 && ready.empty(); pass++)
            for (int w = 0; w < kWarps; w++) {
                if (pass == 0 && ((held >> w) & 1u)) continue;
                bool runnable = false;
                for (int i = 0; i < 32; i++) runnable |= threads[w * 32 + i].place == 0;
                if (runnable || serve_warp(w)) ready.push_back(w);
            }
        if (ready.empty()) {
            int done = 0, waiting = 0, line = 0;
            bool alike = true;
            for (Thread &t : threads) {
                done += t.place == -1;
                if (t.place <= 0) continue;
                if (!t.block_wide) return -2;
                waiting++;
                alike &= line == 0 || line == t.place;
                line = t.place;
            }
            if (done == kThreads) break;
            if (!alike) return -1;
            if (waiting != kThreads) return -2;
            finish(0, kThreads);
            held = rng() % 4 ? rng() : 0u;
            continue;
        }
        const int w = ready[rng() % ready.size()];
        for (int i = 0; i < 32; i++) {
            Thread &t = threads[w * 32 + i];
            if (t.place != 0) continue;
            current = w * 32 + i;
            tid.x = (unsigned int)current;
            swapcontext(&scheduler, &t.at);
        }
    }
    memcpy(out, g_buf, sizeof(unsigned long long) * (size_t)g_count);
    return g_count;
}
