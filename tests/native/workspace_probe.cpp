// Drives csrc/workspace.cpp without a GPU: the HIP calls that it makes are
// replaced by a record of which addresses are allocated.  Each scenario prints
// one line; the exit status is 0 when all of them hold.
#include <hip/hip_runtime_api.h>
#include <stdint.h>
#include <stdio.h>
#include <stdlib.h>

#include <new>
#include <set>

#include "plan.hpp"

namespace {
std::set<void *> g_live;
int g_synced = 0;
hipStreamCaptureStatus g_capture = hipStreamCaptureStatusNone;
bool g_memory = true;   // false: host allocations fail
}  // namespace

void *operator new(size_t n)
{
    void *p = g_memory ? malloc(n) : nullptr;
    if (!p) throw std::bad_alloc();
    return p;
}
void operator delete(void *p) noexcept { free(p); }
void operator delete(void *p, size_t) noexcept { free(p); }

extern "C" {
hipError_t hipGetDevice(int *d)
{
    *d = 0;
    return hipSuccess;
}
hipError_t hipGetLastError(void) { return hipSuccess; }
hipError_t hipStreamIsCapturing(hipStream_t, hipStreamCaptureStatus *s)
{
    *s = g_capture;
    return hipSuccess;
}
hipError_t hipStreamSynchronize(hipStream_t)
{
    ++g_synced;
    return hipSuccess;
}
hipError_t hipMalloc(void **p, size_t)
{
    static uintptr_t next = 1 << 12;   // no address comes twice
    *p = reinterpret_cast<void *>(next += 1 << 12);
    g_live.insert(*p);
    return hipSuccess;
}
hipError_t hipFree(void *p)
{
    return g_live.erase(p) ? hipSuccess : hipErrorInvalidValue;
}
hipError_t hipMemsetAsync(void *, int, size_t, hipStream_t) { return hipSuccess; }
}

namespace {

struct Got {
    gett_status_t status;
    void *tiles, *counters;
};
Got ask(uintptr_t stream, uint64_t counters, uint64_t bytes, bool capturing = false)
{
    g_capture = capturing ? hipStreamCaptureStatusActive : hipStreamCaptureStatusNone;
    gett::Partials p;
    const gett_status_t st =
        gett::stream_workspace(reinterpret_cast<hipStream_t>(stream), counters, bytes, p);
    return {st, p.tiles, p.counters};
}
bool live(void *p) { return g_live.count(p) == 1; }

int g_failed = 0;
void check(const char *what, bool ok)
{
    printf("%s %s\n", ok ? "ok" : "FAILED", what);
    g_failed += !ok;
}

}  // namespace

int main()
{
    // without a capture, growth frees the old buffers after a synchronisation
    Got a = ask(1, 8, 1 << 20);
    Got b = ask(1, 1 << 16, 1 << 24);
    check("growth of eager buffers frees them",
          a.status == GETT_SUCCESS && b.status == GETT_SUCCESS && !live(a.tiles) &&
              !live(a.counters) && live(b.tiles) && live(b.counters) && g_synced == 1);

    // buffers that a capture took outlive a larger eager call on the stream
    Got eager = ask(2, 8, 1 << 20), graph = ask(2, 8, 1 << 20, true);
    check("a capture takes the eager call's buffers",
          graph.status == GETT_SUCCESS && graph.tiles == eager.tiles &&
              graph.counters == eager.counters);
    Got larger = ask(2, 1 << 16, 1 << 24);
    check("growth leaves a graph its slots", larger.tiles != graph.tiles && live(graph.tiles));
    check("growth leaves a graph its counters",
          larger.counters != graph.counters && live(graph.counters));

    // ... only those that it took: the next growth frees the eager buffers
    Got larger2 = ask(2, 1 << 18, 1 << 26);
    check("buffers of no graph are freed", larger2.status == GETT_SUCCESS && !live(larger.tiles) &&
                                               !live(larger.counters));

    // a second capture, of the grown buffers, keeps them too
    Got graph2 = ask(2, 1 << 18, 1 << 26, true), larger3 = ask(2, 1 << 20, 1 << 28);
    check("a second graph keeps its own",
          larger3.status == GETT_SUCCESS && live(graph2.tiles) && live(graph2.counters) &&
              live(graph.tiles) && live(graph.counters));

    // a capture that takes slots only does not keep the counters, nor the reverse
    ask(3, 8, 1 << 20);
    Got slots = ask(3, 0, 1 << 20, true), more = ask(3, 1 << 16, 1 << 24);
    check("kept by use", more.status == GETT_SUCCESS && live(slots.tiles) && !live(slots.counters));

    // growth inside a capture is refused, with everything as it was
    Got refused = ask(3, 8, 1 << 26, true), same = ask(3, 8, 1 << 24);
    check("growth inside a capture is refused", refused.status == GETT_ERROR_NOT_SUPPORTED &&
                                                    same.tiles == more.tiles && live(same.tiles));

    // no host memory for a new stream's entry: a status, not an exception
    gett_status_t none = GETT_SUCCESS;
    g_memory = false;
    try {
        none = ask(4, 8, 1 << 20).status;
    } catch (...) {
    }
    g_memory = true;
    check("no host memory is a status", none == GETT_ERROR_ALLOC);
    return g_failed != 0;
}
