// Every address that the 4-bit product reads and writes, on the CPU: bgmf_mx.hip is
// built for it (KERNELS: the source without its asm statements), and each argument and
// the workspace, of exactly the bytes that the call asks for, ends (then begins) at a
// page that faults.
#include <signal.h>
#include <stdio.h>
#include <stdlib.h>
#include <sys/mman.h>
#include <ucontext.h>
#include <unistd.h>

#include <functional>
#include <vector>

#include "hip/hip_runtime.h"

namespace {

// A workgroup's threads, each until its next __syncthreads() in turn.
constexpr unsigned kMostThreads = 256;
constexpr size_t kStack = 128 << 10;
ucontext_t g_main, g_thread[kMostThreads];
std::vector<char> g_stacks(kMostThreads * kStack);
bool g_done[kMostThreads];
unsigned g_now;
const std::function<void()> *g_kernel;

void thread_main() {
  (*g_kernel)();
  g_done[g_now] = true;
}

void run_group(unsigned threads, const std::function<void()> &kernel) {
  g_kernel = &kernel;
  for (unsigned t = 0; t < threads; ++t) {
    getcontext(&g_thread[t]);
    g_thread[t].uc_stack.ss_sp = &g_stacks[t * kStack];
    g_thread[t].uc_stack.ss_size = kStack;
    g_thread[t].uc_link = &g_main;
    makecontext(&g_thread[t], thread_main, 0);
    g_done[t] = false;
  }
  for (unsigned left = threads; left > 0;) {
    for (g_now = 0; g_now < threads; ++g_now) {
      if (g_done[g_now]) continue;
      threadIdx = dim3(g_now);
      swapcontext(&g_main, &g_thread[g_now]);
      left -= g_done[g_now];
    }
  }
}

template <class... Parameters, class... Arguments>
void launched(void (*kernel)(Parameters...), dim3 grid, dim3 block, Arguments... arguments) {
  if (block.x > kMostThreads || block.y != 1 || block.z != 1) abort();
  gridDim = grid;
  const std::function<void()> one = [&] { kernel(arguments...); };
  for (unsigned z = 0; z < grid.z; ++z)
    for (unsigned y = 0; y < grid.y; ++y)
      for (unsigned x = 0; x < grid.x; ++x) {
        blockIdx = dim3(x, y, z);
        run_group(block.x, one);
      }
}

}  // namespace

void __syncthreads() {
  swapcontext(&g_thread[g_now], &g_main);
  threadIdx = dim3(g_now);
}

#define hipLaunchKernelGGL(kernel, grid, block, lds, stream, ...) \
  launched(kernel, grid, block, __VA_ARGS__)

namespace bgmfk {
int fail_call(int code, const char *fmt, ...) {
  fprintf(stderr, "refused: %s\n", fmt);
  return code;
}
}  // namespace bgmfk

#include KERNELS

namespace {

char g_case[256];
void on_fault(int, siginfo_t *info, void *) {
  printf("%s: a fault at %p\n", g_case, info->si_addr);
  fflush(stdout);
  _exit(1);
}

// `bytes` bytes with a page that faults right after them (or right before).
struct Guarded {
  char *map;
  size_t all;
  void *data;
  Guarded(size_t bytes, bool before) {
    const size_t page = 4096, inner = (bytes + page - 1) / page * page;
    all = inner + 2 * page;
    map = static_cast<char *>(
        mmap(nullptr, all, PROT_READ | PROT_WRITE, MAP_PRIVATE | MAP_ANONYMOUS, -1, 0));
    if (map == MAP_FAILED) abort();
    mprotect(map, page, PROT_NONE);
    mprotect(map + page + inner, page, PROT_NONE);
    data = before ? map + page : map + page + inner - bytes;
  }
  ~Guarded() { munmap(map, all); }
};

}  // namespace

// Lines of: type (0 fp32, 1 bf16, 4 users in 4 bits) rows items k out_type
int main() {
  struct sigaction act = {};
  act.sa_sigaction = on_fault;
  act.sa_flags = SA_SIGINFO | SA_ONSTACK;
  std::vector<char> stack(1 << 16);
  stack_t alternative = {stack.data(), 0, stack.size()};
  sigaltstack(&alternative, nullptr);
  sigaction(SIGSEGV, &act, nullptr);
  sigaction(SIGBUS, &act, nullptr);
  int type, out_type;
  long long rows, items, k;
  while (scanf("%d %lld %lld %lld %d", &type, &rows, &items, &k, &out_type) == 5) {
    snprintf(g_case, sizeof g_case, "type %d, %lld x %lld, k = %lld, to type %d", type, rows, items,
             k, out_type);
    const int64_t blocks = (k + 31) / 32;
    const bool own = type != BGMF_TYPE_MX4;
    for (const bool before : {false, true}) {
      const int64_t x_stride = own ? k : blocks * 16;
      const Guarded x((size_t)(rows * x_stride * (own ? bgmfk::type_bytes(type) : 1)), before);
      const Guarded row_scale((size_t)(rows * blocks), before);
      const Guarded w((size_t)(items * blocks * 16), before), scale((size_t)(items * blocks), before);
      const Guarded out((size_t)(rows * items * bgmfk::type_bytes(out_type)), before);
      const int64_t need = bgmf_mx_scores_workspace(rows, items, k, type);
      const Guarded ws((size_t)need, before);
      const int rc = bgmf_mx_scores(
          x.data, type, rows, k, x_stride, own ? nullptr : static_cast<uint8_t *>(row_scale.data),
          blocks, static_cast<uint8_t *>(w.data), items, blocks * 16,
          static_cast<uint8_t *>(scale.data), blocks, out.data, out_type, items, ws.data, need,
          nullptr);
      if (rc != BGMF_OK) {
        printf("%s: refused\n", g_case);
        return 1;
      }
    }
    printf("%s: in bounds\n", g_case);
    fflush(stdout);
  }
  return 0;
}
