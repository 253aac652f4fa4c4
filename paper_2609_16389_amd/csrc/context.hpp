// The handle and its workspace, shared by the library's translation units.
#pragma once

#include <hip/hip_runtime.h>

#include <stddef.h>
#include <stdint.h>

#include <vector>

#include "xgemm.h"

struct Workspace {
    void *p;
    size_t bytes;
};

struct xgemm_ctx {
    int device;
    int cu_count;
    // The workspace of the call being enqueued: that of calls which run at
    // once, or that of calls which a stream capture records.  A recorded call
    // keeps its workspace's address for every replay, so that buffer is never
    // freed before the handle is (one that a larger call replaces is kept in
    // ws_old), and calls that run at once have a buffer of their own, whatever
    // stream a graph is replayed on.
    void *workspace;
    Workspace ws_direct, ws_record;
    std::vector<void *> ws_old;
    bool recording;         // `workspace` is ws_record's
    bool record_clears;     // ws_record was allocated within a capture: each recorded call clears its counters
    // Direct calls that share the workspace never overlap, whichever streams they
    // are enqueued on.  While a handle's calls all come on one stream, the
    // stream's order is enough and nothing is recorded (an event record
    // between two GEMMs leaves the GPU idle for about 10 us).  The first
    // call on another stream waits for the device to drain (the previous
    // stream may no longer exist), and from then on every call records
    // ws_event on its stream after its last launch, and a call on another
    // stream makes its stream wait for that event.  The workspace is only
    // freed (to grow it) once its last user has completed.  Recorded calls take
    // no part in this: their graphs' replays are ordered by the program.
    hipEvent_t ws_event;
    hipStream_t ws_stream;  // stream of the last call that used the workspace
    bool ws_used;           // ws_stream is set
    bool ws_recorded;       // ws_event follows the last use on ws_stream
    bool ws_multi;          // calls have come on more than one stream
    size_t ws_limit;        // largest workspace the handle may allocate (0: no limit)
    bool persistent;        // the selected plans may use the persistent kernel
    void *scratch;          // this device's `scratch` array (xgemm_run_noalloc)
    struct PlanCache *plans;  // selections already made (sizes and layout flags only)
    char last_error[256];
};

namespace xgemm_host {

// Counter words that calls share: the first bytes of every workspace, zero
// when the workspace is allocated and zero again after every call that uses
// them (the persistent kernel's split tiles, joins of split rows); the other
// workspace users start after them.
constexpr size_t kWsPrefix = 4096;

constexpr int64_t kMaxDim = (int64_t)1 << 31;

__attribute__((visibility("hidden"))) void set_error(xgemm_ctx *h, const char *what, hipError_t e);

// Make `bytes` of workspace after the counter prefix available at h->workspace
// to work enqueued (or recorded) on stream s, and mark the end of the users
// just enqueued.
__attribute__((visibility("hidden"))) int acquire_workspace(xgemm_ctx *h, size_t bytes, hipStream_t s);
__attribute__((visibility("hidden"))) int release_workspace(xgemm_ctx *h, hipStream_t s);

}  // namespace xgemm_host
