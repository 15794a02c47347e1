// Kernels on the CPU: a work-group's threads run one at a time, from one barrier (or exchange between the lanes of a wave)
// to the next, in an order that the caller chooses. Whatever two threads do to one place between two barriers then shows as
// a result that depends on the order. Work-groups run one after the other. Stands in for the HIP headers of a source file
// that is compiled for the host; what it does not define, a test does not need.
#pragma once

#include <math.h>
#include <stdint.h>
#include <string.h>
#include <ucontext.h>

#include <algorithm>
#include <functional>
#include <random>
#include <vector>

#define __global__
#define __device__
#define __host__
#define __forceinline__ inline
#define __launch_bounds__(...)
#define __shared__ static

typedef int hipError_t;
typedef void* hipStream_t;
typedef void* hipEvent_t;
constexpr hipError_t hipSuccess = 0;
struct dim3 {
    unsigned x, y, z;
    constexpr dim3(unsigned x_ = 1, unsigned y_ = 1, unsigned z_ = 1) : x(x_), y(y_), z(z_) {}
};
struct int4 { int x, y, z, w; };
struct float2 { float x, y; };
inline hipError_t hipExtLaunchKernel(const void*, dim3, dim3, void**, size_t, hipStream_t, hipEvent_t, hipEvent_t, int) { return 1; }

namespace simt {

constexpr unsigned kLanes = 64;
constexpr size_t kStack = 64 << 10;

enum State { kReady, kAtBarrier, kAtWave, kDone };
struct Thread {
    ucontext_t at;
    State state;
    std::vector<char> stack;
};
inline std::vector<Thread> threads;
inline ucontext_t scheduler;
inline unsigned current, order_seed;  // 0: ascending, 1: descending, else shuffled by the seed
inline uint64_t wave_value[2048];
inline int any_acc, any_result;
inline bool dry;                   // launches are noted, not run
inline unsigned long long most;    // threads in a row of the largest launch noted, 0 from a launch of too many rows on
inline std::function<void()> body;

inline void wait(State s) {
    Thread& t = threads[current];
    t.state = s;
    swapcontext(&t.at, &scheduler);
}
inline void enter() {
    body();
    threads[current].state = kDone;
    swapcontext(&threads[current].at, &scheduler);
}

}  // namespace simt

inline dim3 threadIdx, blockIdx;

namespace simt {

inline void run_group(unsigned n, std::mt19937& rng) {
    if (threads.size() < n) threads.resize(n);
    for (unsigned i = 0; i < n; ++i) {
        Thread& t = threads[i];
        t.stack.resize(kStack);
        getcontext(&t.at);
        t.at.uc_stack.ss_sp = t.stack.data();
        t.at.uc_stack.ss_size = kStack;
        t.at.uc_link = nullptr;
        t.state = kReady;
        makecontext(&t.at, enter, 0);
    }
    std::vector<unsigned> order(n);
    for (;;) {
        for (unsigned i = 0; i < n; ++i) order[i] = order_seed == 1 ? n - 1 - i : i;
        if (order_seed > 1) std::shuffle(order.begin(), order.end(), rng);
        for (unsigned i : order)
            if (threads[i].state == kReady) {
                current = i;
                threadIdx = dim3(i);
                swapcontext(&scheduler, &threads[i].at);
            }
        unsigned live = 0, at_barrier = 0;
        for (unsigned i = 0; i < n; ++i) {
            live += threads[i].state != kDone;
            at_barrier += threads[i].state == kAtBarrier;
        }
        if (live == 0) return;
        bool moved = false;
        for (unsigned w = 0; w < n; w += kLanes) {  // a wave exchanges once all of its threads are there
            bool all = true, some = false;
            for (unsigned i = w; i < w + kLanes && i < n; ++i) {
                all &= threads[i].state == kAtWave || threads[i].state == kDone;
                some |= threads[i].state == kAtWave;
            }
            if (all && some) {
                moved = true;
                for (unsigned i = w; i < w + kLanes && i < n; ++i)
                    if (threads[i].state == kAtWave) threads[i].state = kReady;
            }
        }
        if (at_barrier == live) {
            moved = true;
            any_result = any_acc;
            any_acc = 0;
            for (unsigned i = 0; i < n; ++i)
                if (threads[i].state == kAtBarrier) threads[i].state = kReady;
        }
        if (!moved) __builtin_trap();  // a barrier that some threads never reach
    }
}

template <typename T>
inline T exchange(T v, unsigned from) {
    static_assert(sizeof(T) <= 8, "one value a lane");
    memcpy(&wave_value[current], &v, sizeof(T));
    wait(kAtWave);
    T r;
    memcpy(&r, &wave_value[current / kLanes * kLanes + from], sizeof(T));
    wait(kAtWave);
    return r;
}

}  // namespace simt

inline void __syncthreads() { simt::wait(simt::kAtBarrier); }
inline int __syncthreads_or(int x) {
    simt::any_acc |= x != 0;
    simt::wait(simt::kAtBarrier);
    return simt::any_result;
}
template <typename T>
inline T __shfl_up(T v, unsigned by, int) {
    const unsigned lane = simt::current % simt::kLanes;
    return simt::exchange(v, lane >= by ? lane - by : lane);
}
template <typename T>
inline T __shfl_xor(T v, unsigned mask, int) { return simt::exchange(v, (simt::current % simt::kLanes) ^ mask); }
template <typename T>
inline T __shfl(T v, unsigned from, int) { return simt::exchange(v, from % simt::kLanes); }

template <typename T, typename U>
inline T atomicOr(T* p, U v) { const T old = *p; *p = old | static_cast<T>(v); return old; }
template <typename T, typename U>
inline T atomicAnd(T* p, U v) { const T old = *p; *p = old & static_cast<T>(v); return old; }
template <typename T, typename U>
inline T atomicAdd(T* p, U v) { const T old = *p; *p = old + static_cast<T>(v); return old; }
template <typename T, typename U>
inline T atomicMax(T* p, U v) { const T old = *p; *p = std::max(old, static_cast<T>(v)); return old; }
template <typename T, typename U>
inline T atomicMin(T* p, U v) { const T old = *p; *p = std::min(old, static_cast<T>(v)); return old; }
inline float __uint_as_float(uint32_t v) { float r; memcpy(&r, &v, 4); return r; }
inline uint32_t __float_as_uint(float v) { uint32_t r; memcpy(&r, &v, 4); return r; }
inline float __fsub_rn(float x, float y) { return x - y; }
inline float __fmul_rn(float x, float y) { return x * y; }
inline double __dsub_rn(double x, double y) { return x - y; }
inline double __dmul_rn(double x, double y) { return x * y; }
inline float __double2float_rn(double x) { return static_cast<float>(x); }

// In place of the library's launch_kernel, which kernels.h has under another name.
#define launch_kernel launch_kernel_of_the_gpu
#include "kernels.h"
#undef launch_kernel

namespace elis {

template <typename... P, typename... A>
inline hipError_t launch_kernel(void (*kernel)(P...), dim3 grid, dim3 block, uint32_t, hipStream_t, A... a) {
    if (simt::dry) {
        const unsigned long long row = static_cast<unsigned long long>(grid.x) * block.x;
        simt::most = simt::most == 0 || grid.y > 65535 ? 0 : std::max(simt::most, row);
        return hipSuccess;
    }
    std::mt19937 rng(simt::order_seed);
    simt::body = [&] { kernel(static_cast<P>(a)...); };
    std::vector<unsigned> groups(grid.x);
    for (unsigned i = 0; i < grid.x; ++i) groups[i] = simt::order_seed == 1 ? grid.x - 1 - i : i;
    if (simt::order_seed > 1) std::shuffle(groups.begin(), groups.end(), rng);
    for (unsigned y = 0; y < grid.y; ++y)
        for (unsigned x : groups) {
            blockIdx = dim3(x, y);
            simt::run_group(block.x, rng);
        }
    return hipSuccess;
}

inline bool launch_timing_events(hipEvent_t*, hipEvent_t*) { return false; }

}  // namespace elis
