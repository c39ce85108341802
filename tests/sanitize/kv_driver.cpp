// Host side of the cache in four bits against a runtime that only writes down what it is asked for, from a script on stdin, one line
// of output per command: the command, the status that the call returned, and the runtime calls that it made, in their order.  No GPU: the
// runtime's functions and the kernels' launches are defined here, and the cache's memory is a heap block of exactly its size.
//
//   create                     a cache (8 query and 2 key heads of 64, 10 blocks, 4 rows, 100 tokens a step)
//   extend <stream> <T>        4 requests;  keeps the step as the latest
//   release <stream>
//   store | attend <stream> <which>   with the latest step (which 0), or the one before it (1)
//   read | poll <stream>
//   destroy
//   capture <stream> <0|1>     the stream is being captured from now on, or no longer
//   end <stream>               the caller has destroyed it
//   fail <name>                the next call of that name fails
//
// Names in the output: record s (the event, on stream s), wait s, device_wait, stream_wait s, fill, copy, plan, release, heads, attend, read; a
// failing one has a "!" behind it.  Streams are numbers; 0 is the default stream.
#include "../../paper_2602_24044_amd/csrc/kv/kv_api.hip"

#include <cstdio>
#include <cstdlib>
#include <iostream>
#include <set>
#include <sstream>
#include <string>

namespace {

std::ostringstream trace;
std::set<long> captured, ended;
std::string failing;

long number(hipStream_t s) { return reinterpret_cast<long>(s) / 64; }
hipStream_t stream(long n) { return reinterpret_cast<hipStream_t>(n * 64); }

hipError_t did(const std::string& name, const std::string& what = "", hipError_t e = hipSuccess)
{
    if (failing == name) {
        failing.clear();
        e = hipErrorUnknown;
    }
    trace << ' ' << name << what << (e == hipSuccess ? "" : "!");
    return e;
}
hipError_t on(const std::string& name, hipStream_t s)
{
    return did(name, std::to_string(number(s)), ended.count(number(s)) ? hipErrorInvalidHandle : hipSuccess);
}

}  // namespace

extern "C" {
hipError_t hipGetDevice(int* d) { *d = 0; return hipSuccess; }
hipError_t hipSetDevice(int) { return hipSuccess; }
hipError_t hipDeviceGetAttribute(int* v, hipDeviceAttribute_t, int) { *v = 256; return hipSuccess; }
hipError_t hipGetLastError() { return hipSuccess; }
hipError_t hipDeviceSynchronize() { return did("device_wait"); }
hipError_t hipEventCreateWithFlags(hipEvent_t* e, unsigned) { *e = reinterpret_cast<hipEvent_t>(64); return hipSuccess; }
hipError_t hipEventDestroy(hipEvent_t) { return hipSuccess; }
hipError_t hipEventRecord(hipEvent_t, hipStream_t s) { return on("record", s); }
hipError_t hipStreamWaitEvent(hipStream_t s, hipEvent_t, unsigned) { return on("wait", s); }
hipError_t hipStreamSynchronize(hipStream_t s) { return on("stream_wait", s); }
hipError_t hipStreamIsCapturing(hipStream_t s, hipStreamCaptureStatus* c)
{
    if (ended.count(number(s))) return hipErrorInvalidHandle;
    *c = captured.count(number(s)) ? hipStreamCaptureStatusActive : hipStreamCaptureStatusNone;
    return hipSuccess;
}
hipError_t hipMemcpyAsync(void* to, const void* from, size_t n, hipMemcpyKind, hipStream_t)
{
    std::memcpy(to, from, n);
    return did("copy");
}
}

namespace lora {
bool note_hip_failure(hipError_t e, const char*) { return e != hipSuccess; }
hipError_t launch_fill_i32(int32_t* p, int32_t v, size_t n, hipStream_t)
{
    for (size_t i = 0; i < n; ++i) p[i] = v;
    return did("fill");
}
namespace kv {
hipError_t launch_plan(const PlanArgs&, hipStream_t s) { return on("plan", s); }
hipError_t launch_release(const Tables&, int, const int32_t*, const int32_t*, hipStream_t s) { return on("release", s); }
hipError_t launch_heads(const HeadsArgs&, int, hipStream_t s) { return on("heads", s); }
hipError_t launch_read(const ReadArgs&, int, hipStream_t s) { return on("read", s); }
hipError_t launch_attend(const AttendArgs&, int, int, hipStream_t s) { return on("attend", s); }
}  // namespace kv
}  // namespace lora

int main()
{
    lora_kv_config cfg = {2, 8, 2, 64, 10, 4, 200, 100, nullptr, 0};
    void* const there = reinterpret_cast<void*>(1 << 20);                      // (an address that nothing follows)
    lora_kv* kv = nullptr;
    lora_kv_step steps[2] = {};
    std::string line;
    while (std::getline(std::cin, line)) {
        std::istringstream in(line);
        std::string cmd;
        long s = 0, x = 0;
        in >> cmd;
        if (cmd == "fail") {
            in >> failing;
            continue;
        }
        in >> s >> x;
        trace.str("");
        int st = -1;
        if (cmd == "create") {
            cfg.slab_bytes = lora_kv_slab_bytes(&cfg);
            if (!cfg.slab) cfg.slab = std::aligned_alloc(256, cfg.slab_bytes);
            st = lora_kv_create(&cfg, &kv);
        } else if (cmd == "capture") {
            if (x) captured.insert(s);
            else captured.erase(s);
            continue;
        } else if (cmd == "end") {
            ended.insert(s);
            continue;
        } else if (cmd == "extend") {
            const int32_t* d = static_cast<const int32_t*>(there);
            lora_kv_step step = {};
            st = lora_kv_extend(kv, 4, d, d, d, (int32_t)x, (int32_t)x, &step, stream(s));
            if (st == LORA_OK) {
                steps[1] = steps[0];
                steps[0] = step;
            }
        } else if (cmd == "release") {
            st = lora_kv_release(kv, 1, static_cast<const int32_t*>(there), nullptr, stream(s));
        } else if (cmd == "store") {
            lora_heads h = {};
            h.d_k = h.d_v = there;
            st = lora_kv_store(kv, 0, &steps[x], &h, stream(s));
        } else if (cmd == "attend") {
            st = lora_kv_attend(kv, 0, &steps[x], 1.f, there, 0, static_cast<char*>(there) + 65536, 0, stream(s));
        } else if (cmd == "read") {
            st = lora_kv_read(kv, 0, 1, static_cast<const int32_t*>(there), static_cast<const int32_t*>(there), nullptr, nullptr, stream(s));
        } else if (cmd == "poll") {
            st = lora_kv_poll_flags(kv, nullptr, stream(s));
        } else if (cmd == "destroy") {
            st = lora_kv_destroy(kv);
            kv = nullptr;
        }
        std::printf("%s %d%s\n", cmd.c_str(), st, trace.str().c_str());
    }
    if (kv) lora_kv_destroy(kv);
    std::free(cfg.slab);
    return 0;
}
