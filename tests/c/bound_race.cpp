// A workgroup's bound of the k best (bound_of_groups in csrc/gs_scores.hip, whose text
// BOUND_SOURCE holds) with a thread for each lane: barriers and ballots order the threads as they
// do on the GPU, nothing else does, so that ThreadSanitizer sees an access to LDS that only luck orders.
#include <pthread.h>

#include <cstdint>
#include <cstdio>
#include <thread>
#include <type_traits>
#include <vector>

#define __device__
#define __forceinline__ inline
constexpr int kWave = 64, kThreads = 256;

static pthread_barrier_t all_meet, wave_meet;
static int votes[2][kWave];
struct Index {
    int x;
};
static thread_local Index threadIdx;
static thread_local int ballots;

static void __syncthreads() { pthread_barrier_wait(&all_meet); }
static unsigned long long __ballot(bool on)  // (of the first wave)
{
    int *mine = votes[ballots++ % 2];
    mine[threadIdx.x] = on;
    pthread_barrier_wait(&wave_meet);
    unsigned long long v = 0;
    for (int i = 0; i < kWave; i++) v |= (unsigned long long)mine[i] << i;
    return v;
}
static int __popcll(unsigned long long v) { return __builtin_popcountll(v); }
template <int L, class Op> uint32_t group_fold_u(uint32_t v, Op &&) { return v; }  // (of four times as many threads)

constexpr int kTopGroups = 256, kTopKeep = 2880;
typedef unsigned long long u64;
#include BOUND_SOURCE

static WideLds<kThreads> lds;
static uint32_t key_of(int thread, int call) { return 1000u * (call + 1) + (uint32_t)(thread * 37 % kThreads); }

int main()
{
    constexpr int kCalls = 12, kBest = 20;
    pthread_barrier_init(&all_meet, nullptr, kThreads);
    pthread_barrier_init(&wave_meet, nullptr, kWave);
    std::vector<int> wrong(kThreads);
    std::vector<std::thread> threads;
    for (int t = 0; t < kThreads; t++)
        threads.emplace_back([&, t] {
            threadIdx.x = t;
            // one call behind the other, as a row's first parts make them; the keys are a permutation of 0 .. 255
            for (int c = 0; c < kCalls; c++)
                wrong[t] += bound_of_groups<kThreads>(key_of(t, c), kBest, lds) != 1000u * (c + 1) + kThreads - kBest;
        });
    for (auto &t : threads) t.join();
    for (int w : wrong)
        if (w) return 1;
    std::puts("bound ok");
    return 0;
}
