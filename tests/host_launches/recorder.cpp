// A stand-in for the HIP runtime that launches nothing and writes down what it is asked for: built and loaded before libdta.so by
// tests/test_host_launches.py, so that the library's own host code decides and the test reads what it decided.
// Streams finish nothing by themselves: a test says when one has (rec_finish).  The handle hipStreamPerThread is another stream in
// every thread, as it is for the runtime.
#define __HIP_PLATFORM_AMD__ 1
#include <hip/hip_runtime_api.h>

#include <cstdio>
#include <cstdlib>
#include <map>
#include <mutex>
#include <string>
#include <thread>
#include <utility>

namespace {

std::mutex mu;
std::string book, taken;
std::map<const void*, std::string> kernels;
hipError_t last_error = hipSuccess;
int fail_in = 0;   // the launch that fails, counted from the next; 0: none
bool capturing = false;

typedef std::pair<hipStream_t, std::thread::id> Key;
struct Line {   // of work on a stream
  long issued = 0, finished = 0;
};
std::map<Key, Line> lines;
Line& line_of(hipStream_t s) { return lines[Key(s, s == hipStreamPerThread ? std::this_thread::get_id() : std::thread::id())]; }

struct Event {
  Line* line = nullptr;   // null: never recorded
  long at = 0;
};

struct {
  dim3 grid, block;
  size_t shared;
  hipStream_t stream;
} pushed;

hipError_t note(hipError_t e) {
  if (e != hipSuccess) last_error = e;
  return e;
}

hipError_t launch(const void* f, dim3 grid, dim3 block, hipStream_t stream, hipEvent_t stop) {
  std::lock_guard<std::mutex> lock(mu);
  const bool refused = (uint64_t)grid.x * block.x >= (uint64_t)1 << 32 || !grid.x || (fail_in && --fail_in == 0);
  char text[64];
  snprintf(text, sizeof text, " %u %u %d\n", grid.x, block.x, (int)!refused);
  book += "launch " + kernels[f] + text;
  if (refused) return note(hipErrorInvalidConfiguration);
  Line& line = line_of(stream);
  ++line.issued;
  if (stop) *(Event*)stop = Event{&line, line.issued};
  return hipSuccess;
}

}  // namespace

extern "C" {

// for the test
const char* rec_take() {
  std::lock_guard<std::mutex> lock(mu);
  taken.swap(book);
  book.clear();
  return taken.c_str();
}
const char* rec_kernels() {   // all that the library has
  std::lock_guard<std::mutex> lock(mu);
  taken.clear();
  for (const auto& k : kernels) taken += k.second + "\n";
  return taken.c_str();
}
void rec_fail(int nth) { fail_in = nth; }
void rec_capture(int on) { capturing = on; }
void rec_finish(void* stream) {   // what the calling thread sees as that stream has run
  std::lock_guard<std::mutex> lock(mu);
  Line& line = line_of((hipStream_t)stream);
  line.finished = line.issued;
}

// the runtime, as far as the library uses it
void** __hipRegisterFatBinary(const void*) {
  static void* one;
  return &one;
}
void __hipUnregisterFatBinary(void**) {}
void __hipRegisterFunction(void**, const void* host, char*, const char* name, unsigned, void*, void*, void*, void*, int*) {
  kernels[host] = name;
}
void __hipRegisterVar(void**, void*, char*, char*, int, size_t, int, int) {}
hipError_t __hipPushCallConfiguration(dim3 grid, dim3 block, size_t shared, hipStream_t stream) {
  pushed = {grid, block, shared, stream};
  return hipSuccess;
}
hipError_t __hipPopCallConfiguration(dim3* grid, dim3* block, size_t* shared, hipStream_t* stream) {
  *grid = pushed.grid;
  *block = pushed.block;
  *shared = pushed.shared;
  *stream = pushed.stream;
  return hipSuccess;
}
hipError_t hipLaunchKernel(const void* f, dim3 grid, dim3 block, void**, size_t, hipStream_t stream) {
  return launch(f, grid, block, stream, nullptr);
}
hipError_t hipExtLaunchKernel(const void* f, dim3 grid, dim3 block, void**, size_t, hipStream_t stream, hipEvent_t, hipEvent_t stop,
                              int) {
  return launch(f, grid, block, stream, stop);
}
hipError_t hipGetLastError() {
  const hipError_t e = last_error;
  last_error = hipSuccess;
  return e;
}
hipError_t hipPeekAtLastError() { return last_error; }
const char* hipGetErrorString(hipError_t) { return "refused by the test"; }
hipError_t hipGetDevice(int* dev) {
  *dev = 0;
  return hipSuccess;
}
hipError_t hipStreamIsCapturing(hipStream_t, hipStreamCaptureStatus* status) {
  *status = capturing ? hipStreamCaptureStatusActive : hipStreamCaptureStatusNone;
  return hipSuccess;
}
hipError_t hipStreamCreateWithFlags(hipStream_t* s, unsigned) {
  static char streams[64];
  static int n;
  *s = (hipStream_t)&streams[n++];
  return hipSuccess;
}
hipError_t hipStreamSynchronize(hipStream_t s) {
  rec_finish((void*)s);
  return hipSuccess;
}
hipError_t hipStreamWaitEvent(hipStream_t, hipEvent_t, unsigned) { return hipSuccess; }
hipError_t hipEventCreateWithFlags(hipEvent_t* e, unsigned) {
  *e = (hipEvent_t) new Event();
  return hipSuccess;
}
hipError_t hipEventDestroy(hipEvent_t e) {
  delete (Event*)e;
  return hipSuccess;
}
hipError_t hipEventRecord(hipEvent_t e, hipStream_t s) {
  std::lock_guard<std::mutex> lock(mu);
  Line& line = line_of(s);
  *(Event*)e = Event{&line, line.issued};
  book += "record\n";
  return hipSuccess;
}
hipError_t hipEventQuery(hipEvent_t e) {
  std::lock_guard<std::mutex> lock(mu);
  const Event& ev = *(Event*)e;
  return !ev.line || ev.line->finished >= ev.at ? hipSuccess : note(hipErrorNotReady);
}
hipError_t hipEventSynchronize(hipEvent_t) { return hipSuccess; }
hipError_t hipMalloc(void** p, size_t bytes) {   // addresses that nothing follows
  static uintptr_t next = (uintptr_t)1 << 44;
  std::lock_guard<std::mutex> lock(mu);
  *p = (void*)next;
  next += (bytes + 4095) / 4096 * 4096 + 4096;
  return hipSuccess;
}
hipError_t hipFree(void*) { return hipSuccess; }
hipError_t hipMemcpyAsync(void* dst, const void*, size_t bytes, hipMemcpyKind, hipStream_t s) {
  std::lock_guard<std::mutex> lock(mu);
  ++line_of(s).issued;
  char text[96];
  snprintf(text, sizeof text, "copy %llu %zu\n", (unsigned long long)(uintptr_t)dst, bytes);
  book += text;
  return hipSuccess;
}
hipError_t hipGetSymbolAddress(void** p, const void*) {
  *p = (void*)((uintptr_t)1 << 43);
  return hipSuccess;
}

}  // extern "C"
