// A plan that cannot get its device memory, on the CPU over the stand-in runtime of fake_hip.h: whichever allocation fails,
// nothing has been copied or cleared by then (the runtime makes what its copies need at the first one, and with the
// device's memory taken it may not find the room), all that was taken is given back, and the error is DR_ENOMEM.
// Exit status 0 when everything holds.
#include <hip/hip_runtime.h>

#define hipMalloc fake_hipMalloc
#define hipMemcpy fake_hipMemcpy
#define hipMemset fake_hipMemset
#include "fake_hip.h"
#undef hipMalloc
#undef hipMemcpy
#undef hipMemset

#include <string>

#include "dr_internal.h"
#include "kernels.h"

static int errors = 0, allocations = 0, fails = 0, moves = 0, move_fails = 0, moves_in_need = 0;
#define CHECK(c, ...)                                   \
  do {                                                  \
    if (!(c)) {                                         \
      std::fprintf(stderr, "FAIL %s: ", #c);            \
      std::fprintf(stderr, __VA_ARGS__);                \
      std::fprintf(stderr, "\n");                       \
      ++errors;                                         \
    }                                                   \
  } while (0)

extern "C" {
hipError_t hipMalloc(void** p, size_t n) {
  if (++allocations == fails) {
    moves_in_need = moves;
    return hipErrorOutOfMemory;
  }
  return fake_hipMalloc(p, n);
}
hipError_t hipMemcpy(void* d, const void* s, size_t n, hipMemcpyKind kind) {
  return ++moves == move_fails ? hipErrorOutOfMemory : fake_hipMemcpy(d, s, n, kind);
}
hipError_t hipMemset(void* p, int v, size_t n) { return ++moves == move_fails ? hipErrorOutOfMemory : fake_hipMemset(p, v, n); }
}

namespace dr {
hipError_t launch_stage_kernel(const StageLaunch&, hipStream_t) { return hipSuccess; }
hipError_t launch_stage_relay(const StageLaunch&, const Reload&, hipStream_t) { return hipSuccess; }
hipError_t launch_chunk_sums(const ChunkSum&, uint32_t, uint32_t, hipStream_t) { return hipSuccess; }
hipError_t launch_zero_words(uint64_t*, uint64_t, hipStream_t) { return hipSuccess; }
hipError_t launch_reshard_kernel(const ReshardLaunch&, hipStream_t) { return hipSuccess; }
hipError_t launch_reshard_relay(const ReshardLaunch&, const Reload&, hipStream_t) { return hipSuccess; }
int scratch_on(int, uint64_t** out) { return *out = nullptr, DR_OK; }
}  // namespace dr

static int create(bool reshard, dr_plan** p) {
  const dr_model m = {2, 256, 4, 2, 64, 688, 2048};
  dr_layout l{};
  l.train_shards = 4, l.tp = 2, l.chunk_bytes = 1 << 18, l.moment_chunk_bytes = 1 << 18;
  allocations = moves = moves_in_need = 0;
  return reshard ? dr_reshard_plan_create(&m, 4, 3, 1 << 18, p) : dr_plan_create(&m, &l, p);
}

static void check_freed(const char* what, int n) {
  for (auto& [p, a] : fake::allocs) CHECK(!a.alive, "%zu bytes kept after %s %d failed", a.bytes, what, n);
  fake::release_for_good();
}

int main() {
  for (bool reshard : {false, true}) {
    dr_plan* p = nullptr;
    fails = move_fails = 0;
    CHECK(create(reshard, &p) == DR_OK, "%s", dr_last_error());
    const int all = allocations, all_moves = moves;
    dr_plan_destroy(p);
    fake::release_for_good();
    CHECK(all >= 4 && all_moves >= 4, "%d allocations, %d copies", all, all_moves);
    for (fails = 1; fails <= all; ++fails) {
      p = reinterpret_cast<dr_plan*>(1);
      const int rc = create(reshard, &p);
      CHECK(rc == DR_ENOMEM && !p && std::string(dr_last_error()).find("hipMalloc") != std::string::npos, "allocation %d: %d, %s", fails, rc, dr_last_error());
      CHECK(moves_in_need == 0 && moves == 0, "%d copies before allocation %d failed", moves_in_need, fails);
      check_freed("allocation", fails);
    }
    fails = 0;
    for (move_fails = 1; move_fails <= all_moves; ++move_fails) {
      p = reinterpret_cast<dr_plan*>(1);
      const int rc = create(reshard, &p);
      CHECK(rc == DR_ENOMEM && !p, "copy %d without memory: %d, %s", move_fails, rc, dr_last_error());
      check_freed("copy", move_fails);
    }
    move_fails = 0;
    CHECK(create(reshard, &p) == DR_OK, "%s", dr_last_error());
    dr_plan_destroy(p);
    fake::release_for_good();
  }
  std::printf("plan memory: %d errors\n", errors);
  return errors != 0;
}
