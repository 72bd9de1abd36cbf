// Drives the chunk attention's host code on stand-ins of the HIP runtime's entries
// (which the library finds here before the runtime's own): launches only move the
// launch tables, and whether an upload is ever seen to end is up to the scenario.
//
//   table_slots_host <libcas.so> <scenario>
#include <dlfcn.h>
#include <stdint.h>
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

#include <atomic>
#include <map>
#include <mutex>
#include <string>
#include <thread>
#include <vector>

#include "cas.h"

namespace {

struct Dim3 {
  uint32_t x, y, z;
};
struct Config {
  Dim3 grid, block;
  size_t shared;
  void *stream;
};

std::mutex mu;
std::map<const void *, std::string> kernels;
thread_local Config config;
thread_local int device = 0;
std::atomic<bool> stuck[2];          // uploads on that device never end
std::atomic<int> fail_uploads{0};    // so many uploads fail to launch
std::atomic<int> by_slot{0}, by_argument{0}, attention{0};

}  // namespace

extern "C" {

void **__hipRegisterFatBinary(const void *) {
  static void *handle;
  return &handle;
}
void __hipUnregisterFatBinary(void **) {}
void __hipRegisterFunction(void **, const void *host, char *, const char *name, unsigned, void *, void *, void *, void *, int *) {
  std::lock_guard<std::mutex> lk(mu);
  kernels[host] = name;
}
void __hipRegisterVar(void **, void *, char *, const char *, int, size_t, int, int) {}
int __hipPushCallConfiguration(Dim3 grid, Dim3 block, size_t shared, void *stream) {
  config = Config{grid, block, shared, stream};
  return 0;
}
int __hipPopCallConfiguration(Dim3 *grid, Dim3 *block, size_t *shared, void **stream) {
  *grid = config.grid;
  *block = config.block;
  *shared = config.shared;
  *stream = config.stream;
  return 0;
}
int hipGetDevice(int *d) {
  *d = device;
  return 0;
}
int hipDeviceGetAttribute(int *v, int, int) {
  *v = 256;
  return 0;
}
int hipGetLastError(void) { return 0; }
const char *hipGetErrorString(int) { return "made up"; }
int hipStreamIsCapturing(void *, int *status) {
  *status = 0;
  return 0;
}
int hipHostMalloc(void **p, size_t n, unsigned) {
  n = (n + 4095) & ~(size_t)4095;
  *p = aligned_alloc(4096, n);
  if (*p) memset(*p, 0, n);
  return *p ? 0 : 2;
}
int hipHostFree(void *p) {
  free(p);
  return 0;
}
int hipLaunchKernel(const void *f, Dim3 grid, Dim3 block, void **args, size_t, void *) {
  std::string name;
  {
    std::lock_guard<std::mutex> lk(mu);
    name = kernels[f];
  }
  if (name.find("table_flag_kernel") != std::string::npos) {
    if (fail_uploads.load() > 0) {
      --fail_uploads;
      return 719;
    }
    ++by_slot;
    memcpy(*(void **)args[0], *(void **)args[1], (size_t) * (int64_t *)args[2] * 16);
    for (uint32_t i = 0; i < grid.x && !stuck[device]; ++i)
      __atomic_store_n(*(uint32_t **)args[3] + i, *(uint32_t *)args[4], __ATOMIC_RELEASE);
  } else if (name.find("table_args_kernel") != std::string::npos) {
    ++by_argument;
    const char *data = (const char *)args[0];   // block.x pieces of 16 bytes, the destination, their count
    memcpy(*(void *const *)(data + block.x * 16), data, (size_t) * (const uint32_t *)(data + block.x * 16 + 8) * 16);
  } else if (name.find("chunk_bf16_kernel") != std::string::npos) {
    ++attention;
  }
  return 0;
}

}  // extern "C"

namespace {

decltype(&cas_paged_chunk_plan_create) plan_create;
decltype(&cas_paged_chunk_run) chunk_run;
decltype(&cas_last_error_message) last_error;

#define CHECK(x)                                                                         \
  do {                                                                                   \
    if (!(x)) {                                                                          \
      fprintf(stderr, "line %d: %s (%s)\n", __LINE__, #x, last_error ? last_error() : ""); \
      exit(1);                                                                           \
    }                                                                                    \
  } while (0)

struct Case {
  std::vector<int32_t> q{0}, kv, po{0}, ids;
  cas_decode_problem_t p;
  cas_chunk_plan_t *plan = nullptr;
  size_t bytes = 0, tables = 0;   // of the workspace, and of its start, which holds the tables
  std::vector<char> first;        // that start after the first call

  Case(int batch, int keys) {
    for (int b = 0; b < batch; ++b) {
      q.push_back(q.back() + 300);
      kv.push_back(keys + b);
      for (int i = 0; i < (keys + b + 15) / 16; ++i) ids.push_back((int32_t)ids.size());
      po.push_back((int32_t)ids.size());
    }
    p = cas_decode_problem_t{};
    p.batch = batch;
    p.num_kv_heads = 8;
    p.group_size = 4;
    p.head_dim = 128;
    p.softmax_scale = 0.1f;
    p.page_size = 16;
    p.num_pages = (int32_t)ids.size();
    p.q_offsets = q.data();
    p.kv_lens = kv.data();
    p.page_offsets = po.data();
    p.page_ids = ids.data();
    CHECK(plan_create(&p, &plan, &bytes) == CAS_OK && bytes > 4096);
    tables = bytes < (512 << 10) ? bytes : 512 << 10;
  }
  // One call on the current device; its workspace holds the same tables as after the first call.
  cas_status_t call() {
    thread_local std::map<const Case *, std::vector<char>> workspaces;
    std::vector<char> &ws = workspaces[this];
    if (ws.empty()) ws.resize(bytes + 256);
    char *at = (char *)(((uintptr_t)ws.data() + 255) & ~(uintptr_t)255);
    memset(at, 0, tables);
    const uintptr_t far = (uintptr_t)1 << 44;   // (never touched)
    const cas_status_t s = chunk_run(plan, (void *)far, (void *)(2 * far), (void *)(3 * far), (void *)(4 * far), nullptr, at, bytes,
                                     (void *)0x10);
    if (s == CAS_OK) {
      std::lock_guard<std::mutex> lk(mu);
      if (first.empty()) first.assign(at, at + tables);
      CHECK(memcmp(first.data(), at, tables) == 0);
    }
    return s;
  }
};

}  // namespace

int main(int argc, char **argv) {
  CHECK(argc == 3);
  void *lib = dlopen(argv[1], RTLD_NOW | RTLD_GLOBAL);
  if (!lib) fprintf(stderr, "%s\n", dlerror());
  CHECK(lib);
  plan_create = (decltype(plan_create))dlsym(lib, "cas_paged_chunk_plan_create");
  chunk_run = (decltype(chunk_run))dlsym(lib, "cas_paged_chunk_run");
  last_error = (decltype(last_error))dlsym(lib, "cas_last_error_message");
  CHECK(plan_create && chunk_run && last_error);
  const std::string scenario = argv[2];
  Case small(20, 1000), large(60, 20000);   // (tables of about 12 KB and 330 KB)
  if (scenario == "usual") {
    // Every upload ends: slots, again and again.
    for (int i = 0; i < 100; ++i) CHECK(small.call() == CAS_OK);
    for (int i = 0; i < 40; ++i) CHECK(large.call() == CAS_OK);
    CHECK(by_slot == 140 && by_argument == 0 && attention == 140);
  } else if (scenario == "never") {
    // No upload ends (a device error, or a stream that waits for work still to be enqueued).
    stuck[0] = true;
    for (int i = 0; i < 40; ++i) CHECK(small.call() == CAS_OK);
    CHECK(by_slot == 16 && by_argument > 24 && attention == 40);
    // Larger tables: the slots that are on their way are no obstacle.
    for (int i = 0; i < 20; ++i) CHECK(large.call() == CAS_OK);
    CHECK(by_slot == 32 && attention == 60);
  } else if (scenario == "failing") {
    // Uploads that could not be launched: their slots are free again.
    CHECK(small.call() == CAS_OK);
    for (int i = 0; i < 20; ++i) {
      fail_uploads = 1;
      CHECK(small.call() == CAS_ERR_HIP);
    }
    for (int i = 0; i < 40; ++i) CHECK(small.call() == CAS_OK);
    CHECK(by_slot == 41 && by_argument == 0);
  } else if (scenario == "devices") {
    // One device whose uploads never end does not hold up another (100 calls there take a few ms, the
    // waiting thread's 10 ms each).
    stuck[0] = true;
    std::atomic<int> calls{0};
    std::atomic<bool> full{false}, done{false};
    std::thread waiting([&] {
      for (; calls < 400 && !done; ++calls) {
        CHECK(small.call() == CAS_OK);
        full = calls >= 20;
      }
    });
    while (!full) std::this_thread::yield();
    const int before = calls;
    device = 1;
    for (int i = 0; i < 100; ++i) CHECK(small.call() == CAS_OK);
    const int after = calls;
    done = true;
    waiting.join();
    CHECK(after - before < 50);
  } else {
    CHECK(!"a known scenario");
  }
  printf("%s ok\n", scenario.c_str());
  return 0;
}
