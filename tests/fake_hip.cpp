// The HIP calls that the host side of the cache operators makes, without a
// GPU: they are written to a log with the device that is current, memory is
// addresses that nothing reads, and a test says what a stream's capture
// status is and which call fails.  Launches are logged too.
#include <hip/hip_runtime.h>

#include <stdio.h>
#include <string.h>

#include <map>
#include <string>

#include "cache.h"

namespace {
struct Block {
  size_t size;
  int device;
};
std::map<uintptr_t, Block> memory;
std::map<std::string, int> fails;  // call -> error it returns
uintptr_t next_address;
int device, capturing;
hipStream_t captured;
std::string trace;

hipError_t made(const char *call, const char *more = "") {
  trace += std::string(call) + more + " on " + std::to_string(device) + "\n";
  const auto f = fails.find(call);
  return f == fails.end() ? hipSuccess : (hipError_t)f->second;
}
std::map<uintptr_t, Block>::iterator find(const void *p) {
  auto it = memory.upper_bound((uintptr_t)p);
  if (it == memory.begin()) return memory.end();
  --it;
  return (uintptr_t)p < it->first + it->second.size ? it : memory.end();
}
}  // namespace

extern "C" {
void fake_reset() {
  memory.clear();
  fails.clear();
  next_address = (uintptr_t)1 << 40;
  device = capturing = 0;
  captured = nullptr;
  trace.clear();
}
uintptr_t fake_memory(size_t size, int on) {
  const uintptr_t p = next_address;
  memory[p] = {size, on};
  next_address += (size + 4096) / 4096 * 4096 + 4096;
  return p;
}
void fake_fail(const char *call, int error) {
  if (error) fails[call] = error;
  else fails.erase(call);
}
void fake_capture(int on, void *stream) {
  capturing = on;
  captured = (hipStream_t)stream;
}
void fake_device(int d) { device = d; }
const char *fake_log() {
  static std::string out;
  out.swap(trace);
  trace.clear();
  return out.c_str();
}

hipError_t hipGetLastError() { return hipSuccess; }
const char *hipGetErrorString(hipError_t e) {
  static char text[32];
  snprintf(text, sizeof text, "error %d", (int)e);
  return text;
}
hipError_t hipSetDevice(int d) {
  device = d;
  return made("hipSetDevice");
}
hipError_t hipMalloc(void **p, size_t n) {
  const hipError_t e = made("hipMalloc");
  if (e == hipSuccess) *p = (void *)fake_memory(n, device);
  return e;
}
hipError_t hipFree(void *p) {
  memory.erase((uintptr_t)p);
  return made("hipFree");
}
hipError_t hipMemset(void *, int, size_t) { return made("hipMemset"); }
hipError_t hipMemsetAsync(void *, int, size_t, hipStream_t) { return made("hipMemsetAsync"); }
hipError_t hipMemcpyAsync(void *to, const void *, size_t n, hipMemcpyKind, hipStream_t) {
  memset(to, 0, n);
  return made("hipMemcpyAsync");
}
hipError_t hipDeviceSynchronize() { return made("hipDeviceSynchronize"); }
hipError_t hipStreamSynchronize(hipStream_t s) {
  char text[32];
  snprintf(text, sizeof text, " of stream %zu", (size_t)s);
  return made("hipStreamSynchronize", text);
}
hipError_t hipStreamIsCapturing(hipStream_t s, hipStreamCaptureStatus *status) {
  *status = capturing && s == captured ? hipStreamCaptureStatusActive : hipStreamCaptureStatusNone;
  return made("hipStreamIsCapturing");
}
hipError_t hipPointerGetAttributes(hipPointerAttribute_t *a, const void *p) {
  const auto it = find(p);
  if (it == memory.end()) return hipErrorInvalidValue;
  a->type = hipMemoryTypeDevice;
  a->device = it->second.device;
  return hipSuccess;
}
hipError_t hipMemGetAddressRange(hipDeviceptr_t *base, size_t *size, hipDeviceptr_t p) {
  const auto it = find(p);
  if (it == memory.end()) return hipErrorInvalidValue;
  *base = (hipDeviceptr_t)it->first;
  *size = it->second.size;
  return hipSuccess;
}
}  // extern "C"

namespace gr {
hipError_t launch_attend(uint32_t, bool, const AttendArgs &, hipStream_t) { return made("attend"); }
hipError_t launch_attend_join(bool, const AttendArgs &, uint32_t, hipStream_t) { return made("join"); }
hipError_t launch_attend_weights(bool, const AttendArgs &, hipStream_t) { return made("weights"); }
hipError_t launch_attend_ids(bool, const IdsArgs &, hipStream_t) { return made("ids"); }
hipError_t launch_append(const AppendArgs &, hipStream_t) { return made("append"); }
hipError_t launch_evict(const EvictArgs &, hipStream_t) { return made("evict"); }
}  // namespace gr
