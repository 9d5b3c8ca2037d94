// The launch emulation for the kernels of fla_seq.h: a launch runs its blocks one after another; the work
// items of a block are coroutines of one host thread, which change over at barriers (over the block, or over
// the 64 lanes of a wave around an exchange of operands).  A block in which no item can go on ends the run.
#include <cstdlib>
#include <memory>
#include <vector>

#include <sanitizer/common_interface_defs.h>

#include "fla_seq_internal.h"

// saves the callee-saved registers and the stack pointer at *from, and goes on where `to` was saved (x86-64)
extern "C" void emu_switch(void** from, void* to);
asm(R"(
    .text
    .globl emu_switch
    .hidden emu_switch
    .type emu_switch, @function
emu_switch:
    pushq %rbp
    pushq %rbx
    pushq %r12
    pushq %r13
    pushq %r14
    pushq %r15
    movq %rsp, (%rdi)
    movq %rsi, %rsp
    popq %r15
    popq %r14
    popq %r13
    popq %r12
    popq %rbx
    popq %rbp
    ret
    .size emu_switch, .-emu_switch
)");

thread_local emu_index threadIdx, blockIdx, gridDim;

namespace {
constexpr unsigned kEmuMaxWaves = 16;
constexpr size_t kStack = 256 << 10;
enum State { kRuns, kAtWave, kAtBlock, kEnded };
struct Item {
    void* sp;
    std::unique_ptr<unsigned char[]> stack;
    State state;
    unsigned exchanges;   // of this lane so far: every lane of a wave counts the same
    void* fake_stack;
};
std::vector<Item> g_items(64 * kEmuMaxWaves);
void* g_main;
const void* g_main_stack;
size_t g_main_size;
unsigned g_now;
const void* g_kernel;
void** g_args;
alignas(64) unsigned char g_wave_slots[kEmuMaxWaves][2][4096];

// back to the scheduler, in the given state
void leave(State s) {
    Item& it = g_items[g_now];
    it.state = s;
    __sanitizer_start_switch_fiber(s == kEnded ? nullptr : &it.fake_stack, g_main_stack, g_main_size);
    emu_switch(&it.sp, g_main);
    __sanitizer_finish_switch_fiber(it.fake_stack, &g_main_stack, &g_main_size);
}
}  // namespace

void __syncthreads() { leave(kAtBlock); }
unsigned emu_lane_id() { return threadIdx.x & 63u; }
void emu_wave_barrier() { leave(kAtWave); }
unsigned char* emu_wave_slots() { return g_wave_slots[g_now >> 6][g_items[g_now].exchanges++ & 1u]; }

hipError_t hipGetDevice(int* device) {
    *device = 0;
    return hipSuccess;
}
hipError_t hipGetDeviceProperties(hipDeviceProp_t* prop, int) {
    std::strcpy(prop->gcnArchName, "gfx950:sramecc+:xnack-");
    prop->multiProcessorCount = 2;   // so that ordinary problems take several rows, tokens and chunks per workgroup
    return hipSuccess;
}
hipError_t hipGetLastError() { return hipSuccess; }

// which argument struct the kernels of the next call take, and whether launches fail
extern "C" {
int emu_kernel_args = 0;
int emu_fail_launch = 0;
int emu_launches = 0;
}

template <typename A>
static void call(const void* fn, void** args) {
    reinterpret_cast<void (*)(A)>(const_cast<void*>(fn))(*static_cast<A*>(args[0]));
}

static void item_main() {
    __sanitizer_finish_switch_fiber(nullptr, &g_main_stack, &g_main_size);
    switch (emu_kernel_args) {
        case 0: call<fla::NormArgs>(g_kernel, g_args); break;
        case 1: call<fla::NormBwdArgs>(g_kernel, g_args); break;
        case 2: call<fla::RotaryArgs>(g_kernel, g_args); break;
        case 3: call<fla::ScanArgs>(g_kernel, g_args); break;
        case 4: call<fla::ScanBwdArgs>(g_kernel, g_args); break;
        default: std::abort();
    }
    leave(kEnded);
}

static void run_block(unsigned n) {
    for (unsigned t = 0; t < n; ++t) {
        Item& it = g_items[t];
        if (!it.stack) it.stack.reset(new unsigned char[kStack]);
        // six registers, then where the first switch returns to, with the stack as a call leaves it
        void** top = reinterpret_cast<void**>((reinterpret_cast<uintptr_t>(it.stack.get()) + kStack) & ~uintptr_t(15)) - 1;
        *--top = reinterpret_cast<void*>(&item_main);
        for (int r = 0; r < 6; ++r) *--top = nullptr;
        it.sp = top;
        it.state = kRuns;
        it.exchanges = 0;
        it.fake_stack = nullptr;
    }
    for (unsigned ended = 0; ended < n;) {
        for (unsigned t = 0; t < n; ++t) {
            Item& it = g_items[t];
            if (it.state != kRuns) continue;
            g_now = t;
            threadIdx = {t, 0, 0};
            void* fake = nullptr;
            __sanitizer_start_switch_fiber(&fake, it.stack.get(), kStack);
            emu_switch(&g_main, it.sp);
            __sanitizer_finish_switch_fiber(fake, nullptr, nullptr);
            ended += it.state == kEnded;
        }
        // a wave whose lanes have all come to the exchange goes on, a block whose items are all at the barrier too
        bool moved = ended == n, all = true;
        for (unsigned w = 0; w < n; w += 64) {
            unsigned waits = 0, live = 0;
            for (unsigned t = w; t < w + 64; ++t) {
                live += g_items[t].state != kEnded;
                waits += g_items[t].state == kAtWave;
                all = all && (g_items[t].state == kEnded || g_items[t].state == kAtBlock);
            }
            if (live == 0 || waits != live) continue;
            moved = true;
            for (unsigned t = w; t < w + 64; ++t)
                if (g_items[t].state == kAtWave) g_items[t].state = kRuns;
        }
        if (all)
            for (unsigned t = 0; t < n; ++t)
                if (g_items[t].state == kAtBlock) {
                    g_items[t].state = kRuns;
                    moved = true;
                }
        if (!moved) std::abort();
    }
}

hipError_t hipLaunchKernel(const void* fn, dim3 grid, dim3 block, void** args, size_t, hipStream_t) {
    if (emu_fail_launch) return hipErrorInvalidValue;
    ++emu_launches;
    if (block.x > 64 * kEmuMaxWaves || block.x % 64 || grid.y != 1 || grid.z != 1 || block.y != 1 || block.z != 1)
        std::abort();
    g_kernel = fn;
    g_args = args;
    gridDim = {grid.x, 1, 1};
    for (unsigned b = 0; b < grid.x; ++b) {
        blockIdx = {b, 0, 0};
        run_block(block.x);
    }
    return hipSuccess;
}
