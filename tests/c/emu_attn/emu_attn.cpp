// emu_attn.cpp -- workgroups of the CPU build of the cache kernels (kvio_lane.h
// beside it): all threads of a workgroup are coroutines.
#include <setjmp.h>
#include <stdio.h>
#include <stdlib.h>
#include <string.h>
#include <ucontext.h>

#include <vector>

#include "kvio_lane.h"

namespace {

constexpr size_t kStack = 1 << 20;
constexpr const char *kBarrier = "barrier";

struct Thread {
    ucontext_t start;
    jmp_buf at;
    char *stack = nullptr;
    bool fresh, done;
    const char *what;
    int phase;
    char value[2][64];
};
std::vector<Thread> threads;
std::vector<char> joined[2];                 // [wave][lane][64]
int current = 0;
jmp_buf back;
const std::function<void()> *body = nullptr;
unsigned orders = 0;

[[noreturn]] void die(const char *why, const char *what) {
    fprintf(stderr, "emulated workgroup: %s at %s\n", why, what);
    abort();
}
void enter() {
    (*body)();
    threads[size_t(current)].done = true;
    _longjmp(back, 1);
}
void meet(const char *what) {
    Thread &t = threads[size_t(current)];
    t.what = what;
    if (_setjmp(t.at) == 0) _longjmp(back, 1);
}
void resume(int i) {
    current = i;
    threadIdx.x = static_cast<unsigned>(i);
    Thread &t = threads[size_t(i)];
    if (_setjmp(back) == 0) {
        if (t.fresh) {
            t.fresh = false;
            getcontext(&t.start);
            t.start.uc_stack.ss_sp = t.stack;
            t.start.uc_stack.ss_size = kStack;
            t.start.uc_link = nullptr;
            makecontext(&t.start, enter, 0);
            setcontext(&t.start);
        } else {
            _longjmp(t.at, 1);
        }
    }
}
// Run a wave up to the next barrier; whether it ended.
bool run_wave(int first) {
    for (;;) {
        int ended = 0;
        for (int l = 0; l < 64; ++l) {
            resume(first + l);
            ended += threads[size_t(first + l)].done;
        }
        if (ended == 64) return true;
        const Thread &a = threads[size_t(first)];
        if (ended != 0) die("some lanes ended while others wait", "the end");
        for (int l = 1; l < 64; ++l) {
            const Thread &t = threads[size_t(first + l)];
            if (strcmp(t.what, a.what) != 0 || t.phase != a.phase) die("lanes wait at different operations", t.what);
        }
        if (a.what == kBarrier) return false;
        for (int l = 0; l < 64; ++l)
            memcpy(&joined[0][size_t(first + l) * 64], threads[size_t(first + l)].value[(a.phase - 1) & 1], 64);
    }
}

}  // namespace

const char *emu_attn_join(const void *mine, size_t bytes, const char *what) {
    Thread &t = threads[size_t(current)];
    if (bytes > 64) die("too much", what);
    memcpy(t.value[t.phase++ & 1], mine, bytes);
    meet(what);
    return &joined[0][size_t(current & ~63) * 64];
}
void emu_attn_barrier() { meet(kBarrier); }
int emu_attn_lane() { return current & 63; }

namespace kvio {
int wave_first(int v) {
    const char *all = emu_attn_join(&v, sizeof v, "wave_first");
    for (int l = 0; l < 64; ++l)
        if (memcmp(all + l * 64, &v, sizeof v) != 0) die("a value taken as wave-uniform is not", "wave_first");
    return v;
}
uint64_t wave_ballot(bool v) {
    const char *all = emu_attn_join(&v, sizeof v, "wave_ballot");
    uint64_t m = 0;
    for (int l = 0; l < 64; ++l) m |= uint64_t(all[l * 64] != 0) << l;
    return m;
}
}  // namespace kvio

void emu_attn_launch(dim3 grid, dim3 block, const std::function<void()> &lane) {
    const int n = static_cast<int>(block.x);
    if (n == 0 || n % 64 != 0 || n > 1024 || grid.x == 0 || grid.y == 0 || grid.z == 0 || block.y != 1 || block.z != 1) die("launch shape", "launch");
    while (static_cast<int>(threads.size()) < n) {
        threads.emplace_back();
        threads.back().stack = static_cast<char *>(malloc(kStack));
    }
    joined[0].resize(size_t(n) * 64);
    gridDim = grid;
    blockDim = block;
    body = &lane;
    // Workgroups run last to first, waves in an order that changes: nothing may depend on either.
    for (unsigned z = grid.z; z-- > 0;)
        for (unsigned y = grid.y; y-- > 0;)
            for (unsigned x = grid.x; x-- > 0;) {
                blockIdx.x = x, blockIdx.y = y, blockIdx.z = z;
                for (int i = 0; i < n; ++i) {
                    threads[size_t(i)].fresh = true;
                    threads[size_t(i)].done = false;
                    threads[size_t(i)].phase = 0;
                }
                std::vector<bool> ended(size_t(n) / 64, false);
                for (bool any = true; any;) {
                    any = false;
                    const unsigned turn = orders++;
                    for (int k = 0; k < n / 64; ++k) {
                        const int w = static_cast<int>((turn & 1 ? n / 64 - 1 - k : k) + turn / 2) % (n / 64);
                        if (ended[size_t(w)]) continue;
                        if (run_wave(w * 64)) ended[size_t(w)] = true;
                        else any = true;
                    }
                }
            }
}
