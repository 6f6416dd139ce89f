// Host-only driver for the argument checks of the adapters and checkpoints (csrc/adapter_api.hip), built with -fsanitize=address,undefined for
// the host pass and run on the CPU by tests/test_adapter_sanitizers.py.  Every call must be refused before anything is launched: the launch
// functions below abort.  What is exercised is the arithmetic on sizes near the 64-bit and 32-bit limits.
#include <cstdarg>
#include <cstdint>
#include <cstdio>
#include <cstdlib>

#include "../../paper_2409_09099_amd/csrc/adapter.h"

namespace sste {
static char message[512];
int fail(int status, const char* fmt, ...) {
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(message, sizeof message, fmt, ap);
  va_end(ap);
  return status;
}
void clear_error() { message[0] = 0; }
[[noreturn]] static void reached(const char* what) {
  std::printf("launch function reached: %s\n", what);
  std::abort();
}
hipError_t launch_adapter_apply(const AdapterApply&, hipStream_t) { reached("adapter_apply"); }
hipError_t launch_adapter_wgrad(const AdapterSegments&, int, const AdapterOuter&, const AdapterOuter&, int, void*, hipStream_t) { reached("adapter_wgrad"); }
size_t adapter_apply_workspace_bytes(int64_t T, int, int R, int64_t, int64_t) { return (size_t)T * (size_t)R * 16; }
size_t adapter_wgrad_workspace_bytes(int64_t T, int segments, int R, int64_t I, int64_t O) { return (size_t)(T / 128 + segments + 2) * (size_t)R * (size_t)(I + O) * 4; }
hipError_t launch_checkpoint_pack(const void*, int64_t, int64_t, int64_t, void*, int64_t, void*, int64_t, hipStream_t) { reached("checkpoint_pack"); }
hipError_t launch_checkpoint_backward(const void*, const void*, int64_t, int64_t, int64_t, int64_t, int, void*, int64_t, const void*, int64_t, void*, int64_t, hipStream_t) {
  reached("checkpoint_backward");
}
}  // namespace sste

static int failures = 0;
#define EXPECT(call, want)                                                                              \
  do {                                                                                                  \
    int got_ = (call);                                                                                  \
    if (got_ != (want)) {                                                                               \
      std::printf("line %d: status %d, expected %d (%s)\n", __LINE__, got_, (want), sste::message);     \
      failures++;                                                                                       \
    }                                                                                                   \
  } while (0)

int main() {
  void* fake = reinterpret_cast<void*>(0x1000);
  float* f = reinterpret_cast<float*>(0x1000);
  const int32_t* seg = reinterpret_cast<const int32_t*>(0x1000);
  const int64_t huge = INT64_MAX / 2, wide = 1ll << 23, most = (1ll << 27) - 1;
  auto fwd = [&](int64_t T, int64_t I, int64_t ldx, int64_t segments, int64_t lda, int64_t adapters, int64_t R, int64_t O, int64_t ldz) {
    return sste_adapter_fwd(fake, T, I, ldx, SSTE_BF16, 1.f, seg, segments, seg, fake, lda, fake, O, f, adapters, R, O, fake, ldz, fake, ldz, f, R, nullptr, 0, nullptr);
  };
  EXPECT(fwd(huge, 64, 64, 1, 64, 1, 8, 64, 64), SSTE_ERR_UNSUPPORTED);
  EXPECT(fwd(4, huge - huge % 8, huge - huge % 8, 1, huge - huge % 8, 1, 8, 64, 64), SSTE_ERR_UNSUPPORTED);
  EXPECT(fwd(4, 64, huge - huge % 8, 1, 64, 1, 8, 64, 64), SSTE_ERR_UNSUPPORTED);
  EXPECT(fwd(4, 64, 64, huge, 64, 1, 8, 64, 64), SSTE_ERR_UNSUPPORTED);
  EXPECT(fwd(4, 64, 64, 1, 64, huge, 8, 64, 64), SSTE_ERR_UNSUPPORTED);
  EXPECT(fwd(4, 64, 64, 1, 64, 1, huge - huge % 8, 64, 64), SSTE_ERR_UNSUPPORTED);
  EXPECT(fwd(4, 64, 64, 1, 64, 1, 8, huge - huge % 8, huge - huge % 8), SSTE_ERR_UNSUPPORTED);
  EXPECT(fwd(most, wide, wide, 1, wide, 65535, 128, wide, wide), SSTE_ERR_UNSUPPORTED);      // more than 2^40 elements
  EXPECT(fwd(64, wide, wide, 1 << 20, huge - huge % 8, 65535, 128, wide, wide), SSTE_ERR_UNSUPPORTED);
  EXPECT(fwd(1 << 16, 8, 8, 1 << 20, 8, 1, 8, wide, wide), SSTE_ERR_UNSUPPORTED);             // more than 2^24 tiles
  EXPECT(fwd(INT64_MIN, 64, 64, 1, 64, 1, 8, 64, 64), SSTE_ERR_SHAPE);
  auto wgrad = [&](int64_t T, int64_t I, int64_t O, int64_t segments, int64_t adapters, int64_t R, int64_t ldda, size_t bytes) {
    return sste_adapter_wgrad(fake, T, O, O, SSTE_BF16, 1.f, fake, I, I, SSTE_BF16, 1.f, nullptr, 0, f, R, f, R, seg, segments, seg, adapters, R, f, ldda, f, O, 0, fake, bytes, nullptr);
  };
  EXPECT(wgrad(huge, 64, 64, 1, 1, 8, 64, 1 << 20), SSTE_ERR_UNSUPPORTED);
  EXPECT(wgrad(4, wide, wide, 1, 65535, 128, wide, 1 << 20), SSTE_ERR_UNSUPPORTED);
  EXPECT(wgrad(1 << 15, wide, wide, 1 << 20, 1, 128, wide, 1 << 20), SSTE_ERR_UNSUPPORTED);
  EXPECT(wgrad(4, 64, 64, 1, 1, 8, huge - huge % 4, 1 << 20), SSTE_ERR_UNSUPPORTED);
  EXPECT(wgrad(1024, 64, 64, 1, 1, 8, 64, 16), SSTE_ERR_WORKSPACE);
  if (sste_adapter_wgrad_workspace_bytes(huge, huge, huge, huge, huge) != 0) failures++;
  if (sste_adapter_workspace_bytes(huge, 1, 8, 64, 64) != 0 || sste_adapter_workspace_bytes(4, 1, 8, huge, 64) != 0) failures++;
  (void)sste_adapter_wgrad_workspace_bytes(most, 1 << 20, 128, wide, wide);                   // a number of bytes, whatever it is
  EXPECT(sste_checkpoint_pack(fake, huge, 64, 64, fake, 64, fake, 2, nullptr), SSTE_ERR_UNSUPPORTED);
  EXPECT(sste_checkpoint_pack(fake, 4, huge - huge % 16, huge - huge % 16, fake, huge - huge % 16, fake, huge, nullptr), SSTE_ERR_UNSUPPORTED);
  EXPECT(sste_checkpoint_pack(fake, 4, 64, 64, fake, huge - huge % 16, fake, 2, nullptr), SSTE_ERR_UNSUPPORTED);
  EXPECT(sste_checkpoint_pack(fake, 4, 64, 64, fake, 64, fake, huge, nullptr), SSTE_ERR_UNSUPPORTED);
  EXPECT(sste_checkpoint_backward(fake, fake, INT64_MAX, 64, 64, 2, 1, fake, 64, fake, 64, fake, 64, nullptr), SSTE_ERR_UNSUPPORTED);
  EXPECT(sste_checkpoint_backward(fake, fake, 4, 64, 64, 2, 1, fake, huge - huge % 8, fake, 64, fake, 64, nullptr), SSTE_ERR_UNSUPPORTED);
  EXPECT(sste_checkpoint_backward(fake, fake, INT64_MIN, 64, 64, 2, 1, fake, 64, fake, 64, fake, 64, nullptr), SSTE_ERR_SHAPE);

  std::printf(failures ? "FAILED: %d\n" : "adapter driver ok%.0d\n", failures);
  return failures ? 1 : 0;
}
