// workspace.cpp -- device workspace for the partial tiles of K slices and of
// the stream-K tail (kernel.hpp: a tile's pieces are saved and summed in
// piece order by the last to finish; direct.hpp: summed by a second launch).
//
// One pair of buffers per (device, stream): per-tile counters, zeroed when
// allocated and left at zero by every launch that uses them, and the
// partial-tile slots, which need no initial value.  Launches on one stream
// run in order and a call holds the pair until its launches are enqueued, so
// they can share it; launches on different streams get different pairs.
//
// A buffer grows when a call needs more: the stream is synchronised first
// (queued work may still use the old one) and the old buffer freed.  Growth is
// refused (GETT_ERROR_NOT_SUPPORTED, nothing enqueued) while the stream is
// capturing a graph -- an eager call on that stream beforehand allocates what
// the captured calls use.  A buffer that a captured call was given belongs to
// that graph from then on, whose kernels hold its address: when the stream needs
// a larger one it is left allocated, until the process ends (when the last graph
// that holds it goes cannot be seen from here).
#include <hip/hip_runtime_api.h>
#include <stdint.h>

#include <map>
#include <mutex>
#include <utility>

#include "plan.hpp"

namespace gett {
namespace {

struct Buffer {
    void *p = nullptr;
    uint64_t bytes = 0;
    bool inGraph = false;   // a captured call was given it
};
struct Buffers {
    Buffer counters, tiles;
    std::mutex use;   // held by the call that is enqueuing its launches
};

std::mutex g_mutex;   // of the map; its entries stay where they are
std::map<std::pair<int, hipStream_t>, Buffers> g_buffers;

uint64_t round_up(uint64_t n) { return (n + 4095) / 4096 * 4096; }

// A new buffer in place of one that nothing enqueued uses any more.
gett_status_t grow(Buffer &b, uint64_t bytes)
{
    if (b.p && !b.inGraph && hipFree(b.p) != hipSuccess) return GETT_ERROR_HIP;
    b = Buffer{};
    const uint64_t n = round_up(bytes);
    if (hipMalloc(&b.p, n) != hipSuccess) {
        b.p = nullptr;
        return GETT_ERROR_HIP;
    }
    b.bytes = n;
    return GETT_SUCCESS;
}

}  // namespace

gett_status_t stream_workspace(hipStream_t stream, uint64_t counters, uint64_t tileBytes,
                               Partials &out)
{
    int dev = 0;
    if (hipGetDevice(&dev) != hipSuccess) return GETT_ERROR_HIP;
    Buffers *found;
    try {   // (a new entry takes host memory)
        std::lock_guard<std::mutex> lock(g_mutex);
        found = &g_buffers[{dev, stream}];
    } catch (...) {
        return GETT_ERROR_ALLOC;
    }
    Buffers &b = *found;
    out.hold = std::unique_lock<std::mutex>(b.use);
    const uint64_t cBytes = counters * sizeof(int);
    const bool growC = cBytes > b.counters.bytes, growT = tileBytes > b.tiles.bytes;
    hipStreamCaptureStatus cap = hipStreamCaptureStatusNone;
    if (hipStreamIsCapturing(stream, &cap) != hipSuccess) {
        if (growC || growT) return GETT_ERROR_HIP;
        (void)hipGetLastError();   // no capture of this stream; its launches say the rest
        cap = hipStreamCaptureStatusNone;
    }
    const bool capturing = cap != hipStreamCaptureStatusNone;
    if (capturing && (growC || growT)) return GETT_ERROR_NOT_SUPPORTED;
    if ((growC && b.counters.p) || (growT && b.tiles.p)) {
        // queued launches on this stream may still use the old buffers
        if (hipStreamSynchronize(stream) != hipSuccess) return GETT_ERROR_HIP;
    }
    if (growC) {
        const gett_status_t st = grow(b.counters, cBytes);
        if (st != GETT_SUCCESS) return st;
        // ordered before the launches that follow on this stream
        if (hipMemsetAsync(b.counters.p, 0, b.counters.bytes, stream) != hipSuccess) {
            b.counters.bytes = 0;   // (not zeroed: never handed out)
            return GETT_ERROR_HIP;
        }
    }
    if (growT) {
        const gett_status_t st = grow(b.tiles, tileBytes);
        if (st != GETT_SUCCESS) return st;
    }
    if (capturing) {
        b.counters.inGraph |= cBytes > 0;
        b.tiles.inGraph |= tileBytes > 0;
    }
    out.counters = static_cast<int *>(b.counters.p);
    out.tiles = b.tiles.p;
    return GETT_SUCCESS;
}

}  // namespace gett
