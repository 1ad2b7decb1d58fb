// Runs the lanes of a workgroup on one CPU thread (hip/hip_runtime.h). A wavefront's lanes are taken up to where they meet (a move across lanes, a ballot), then on together; a
// wavefront is taken up to a barrier before another one is, the first one first (lanes_order 0) or the last one (1); or any of them takes a few such steps, at random (others: the seed).
#include "hip/hip_runtime.h"
#undef asm

#include <limits.h>
#include <setjmp.h>
#include <stdio.h>
#include <stdlib.h>
#include <sys/mman.h>
#include <ucontext.h>

#include <map>
#include <string>

dim3 lanes::thread, lanes::block, lanes::threads, lanes::blocks;

namespace {

using namespace lanes;

constexpr int MOST = 1024;
constexpr size_t STACK = 128 << 10;

struct Lane {
    ucontext_t first;
    jmp_buf at;
    bool begun, failed;
    Op op;
    int with, rows;
    uint64_t said, heard;
};

Lane lane[MOST];
char *stacks;
jmp_buf scheduler;
int now;
bool failed;
uint64_t order = 0, seed = 1;
const std::function<void()> *kernel;
std::map<std::string, long> launches;
char message[300];

uint64_t next_random() { return seed = seed * 6364136223846793005ull + 1442695040888963407ull, seed >> 33; }

void fail(const char *what)
{
    failed = true;
    snprintf(message, sizeof message, "%s: workgroup %u, lane %d, line %d", what, block.x, now, lane[now].with);
}

void enter()
{
    (*kernel)();
    lane[now].op = DONE;
    _longjmp(scheduler, 1);
}

void run(int i)      // up to where the lane next meets others
{
    now = i;
    thread = dim3(i, 0, 0);
    lane[i].op = NONE;
    if (_setjmp(scheduler)) return;
    if (lane[i].begun) _longjmp(lane[i].at, 1);
    lane[i].begun = true;
    getcontext(&lane[i].first);
    lane[i].first.uc_stack.ss_sp = stacks + i * STACK;
    lane[i].first.uc_stack.ss_size = STACK;
    lane[i].first.uc_link = nullptr;
    makecontext(&lane[i].first, enter, 0);
    setcontext(&lane[i].first);
}

// the lane that a move's control names, -1: none
int source(int l, int control)
{
    if (control >= 0x1000) return l ^ (control - 0x1000);
    if (control < 0x100) return (l & ~3) | (control >> 2 * (l & 3) & 3);
    if (control > 0x110 && control < 0x120) return (l & 15) >= control - 0x110 ? l - (control - 0x110) : -1;
    if (control == 0x140) return l ^ 15;
    if (control == 0x141) return l ^ 7;
    if (control == 0x142) return l >= 16 ? (l & ~15) - 1 : -1;
    if (control == 0x143) return l >= 32 ? 31 : -1;
    fail("a move that is not known here");
    return -1;
}

// a wavefront, up to a barrier or its end, or for some steps; whether it is there
bool run_wave(int from, int to, int steps)
{
    for (; !failed; --steps) {
        for (int i = from; i < to && !failed; ++i) if (lane[i].op == NONE) run(i);
        int here[DONE + 1] = {};
        for (int i = from; i < to; ++i) ++here[lane[i].op];
        if (here[BARRIER] + here[DONE] == to - from) return true;
        if (!steps) return false;
        // lanes that have left a loop wait behind it, where all of them meet
        Op op = here[ANY] ? ANY : NONE;
        if (op == NONE) {
            for (int o = BALLOT; o <= FENCE; ++o) if (here[o]) op = (Op)o;
            if (here[op] + here[DONE] != to - from || (here[DONE] && op != BALLOT)) {
                fail("lanes of a wavefront are apart");
                return true;
            }
        }
        uint64_t all = 0;
        for (int i = from; i < to; ++i) if (lane[i].op == op && lane[i].said) all |= 1ull << (i - from);
        for (int i = from; i < to; ++i) {
            Lane &l = lane[i];
            if (l.op != op) continue;
            if (op == ANY) l.heard = all != 0;
            else if (op == BALLOT) l.heard = all;
            else if (op == READ) l.heard = lane[from + l.with].said;
            else if (op == MOVE) {
                const int of = source(i - from, l.with);
                l.heard = of < 0 || !(l.rows >> ((i - from) / 16) & 1) ? 0 : lane[from + of].said;
            }
        }
        for (int i = from; i < to; ++i) if (lane[i].op == op) lane[i].op = NONE;
    }
    return true;
}

void run_block(int n)
{
    for (int i = 0; i < n; ++i) { lane[i].begun = false; lane[i].op = NONE; }
    const int waves = (n + 63) / 64;
    std::vector<int> turn;
    while (!failed) {
        turn.clear();
        for (int w = 0; w < waves; ++w) turn.push_back(order == 0 ? waves - 1 - w : w);
        while (!turn.empty()) {
            const size_t k = order > 1 ? next_random() % turn.size() : turn.size() - 1;
            const int w = turn[k];
            if (run_wave(w * 64, std::min(n, w * 64 + 64), order > 1 ? 1 + (int)(next_random() % 8) : INT_MAX)) turn.erase(turn.begin() + (long)k);
        }
        if (failed) return;
        int line = -1;
        for (int i = 0; i < n; ++i) {
            if (lane[i].op == DONE) continue;
            if (line >= 0 && lane[i].with != line) {
                now = i;
                fail("wavefronts are at different barriers");
                return;
            }
            line = lane[i].with;
            lane[i].op = NONE;
        }
        if (line < 0) return;
    }
}

}  // namespace

uint64_t lanes::meet(Op op, uint64_t say, int with, int rows)
{
    Lane &l = lane[now];
    l.op = op; l.said = say; l.with = with; l.rows = rows;
    if (!_setjmp(l.at)) _longjmp(scheduler, 1);
    return lane[now].heard;
}

void lanes::launch(const char *name, dim3 grid, dim3 size, std::function<void()> f)
{
    ++launches[name];
    if (size.x > MOST || failed) { failed = true; return; }
    if (!stacks) stacks = (char *)mmap(nullptr, MOST * STACK, PROT_READ | PROT_WRITE, MAP_PRIVATE | MAP_ANONYMOUS | MAP_NORESERVE, -1, 0);
    kernel = &f;
    threads = size;
    blocks = grid;
    for (unsigned b = 0; b < grid.x && !failed; ++b) {
        block = dim3(b, 0, 0);
        run_block((int)size.x);
    }
}

hipError_t hipGetLastError()
{
    const bool was = failed;
    failed = false;
    return was ? hipErrorLaunchFailure : hipSuccess;
}

extern "C" {

void lanes_order(uint64_t o) { order = o; seed = o; message[0] = 0; }
const char *lanes_message() { return message; }
// launches of kernels whose names have `part` in them, since the last call with NULL
long lanes_launches(const char *part)
{
    if (!part) { launches.clear(); return 0; }
    long n = 0;
    for (const auto &l : launches) if (l.first.find(part) != std::string::npos) n += l.second;
    return n;
}

}
