// What the host sides of the entry points share: the context behind a symb_handle, its error text, and the way a call's descriptors reach the device.
#pragma once
#include <hip/hip_runtime.h>

#include <algorithm>
#include <atomic>
#include <cstdarg>
#include <cstdint>
#include <cstdio>
#include <cstring>
#include <initializer_list>
#include <new>
#include <string>
#include <utility>
#include <vector>

#include "../../include/symb.h"
#include "symb_ring.hpp"

namespace symb {

inline thread_local std::string g_tls_error;

constexpr size_t kSlotBytes = (size_t)2 << 20;  // capacity of one descriptor blob

inline size_t align_up(size_t v, size_t a) { return (v + a - 1) / a * a; }

struct HipRuntime {                             // what the descriptor ring asks of HIP
    using Stream = hipStream_t;
    using Event = hipEvent_t;
    using Status = hipError_t;
    static Status record(Event ev, Stream st) {
        const hipError_t e = hipEventRecord(ev, st);
        if (e != hipSuccess) (void)hipGetLastError();
        return e;
    }
    static Status wait(Event ev) { return hipEventSynchronize(ev); }
    static Status wait_all() { return hipDeviceSynchronize(); }
    static bool done(Event ev) {
        if (hipEventQuery(ev) == hipSuccess) return true;
        (void)hipGetLastError();                // (not ready yet is no error of this call)
        return false;
    }
    static StreamState state(Stream st, uint64_t* capture) {
        hipStreamCaptureStatus s = hipStreamCaptureStatusNone;
        unsigned long long id = 0;
        const hipError_t e = hipStreamGetCaptureInfo(st, &s, &id);
        if (e == hipSuccess) {
            *capture = s == hipStreamCaptureStatusNone ? 0 : id + 1;
            return StreamState::Known;
        }
        (void)hipGetLastError();
        return e == hipErrorStreamCaptureImplicit ? StreamState::Unsure : StreamState::Gone;     // (HIP looks the handle up among its live streams)
    }
    static uint64_t thread(Stream st) {
        if (st != hipStreamPerThread) return 0;
        static std::atomic<uint64_t> threads{0};
        thread_local const uint64_t mine = ++threads;
        return mine;
    }
};
constexpr int kSlots = DescRing<HipRuntime>::kSlots;

}  // namespace symb

struct symb_context {
    int device = 0;
    unsigned char* host_ring = nullptr;   // pinned, kSlots * kSlotBytes
    unsigned char* dev_ring = nullptr;    // device, kSlots * kSlotBytes
    symb::DescRing<symb::HipRuntime> ring;
    symb::HipRuntime rt;
    int64_t desc_sent = 0, desc_in_place = 0;
    int call_slot = -1;                   // the slot this call's descriptors went to (-1: none yet)
    std::string error;
    // measurement switches (symb_debug_set_option); all on by default
    bool opt_desc_reuse = true, opt_k_split = true, opt_small_rows = true, opt_skinny_deep = true;
    // Whether workgroup id mod 8 names the XCD a workgroup runs on, measured at creation: the K-split of
    // the GEMM keeps all parts of a tile on one XCD (behind one L2) and is used only if this holds.
    bool xcd_rule = false;
    int xcc_of_residue[8] = {-1, -1, -1, -1, -1, -1, -1, -1};
    unsigned char* static_scratch = nullptr;     // this device's copy of the file-scope scratch array
    std::vector<const void*> lds_attr_set;       // kernels whose dynamic-LDS limit was raised on this context's device
    // measurement hook: event pairs around GEMM launches
    bool timing = false;
    std::vector<hipEvent_t> tev;                 // 2 * kMaxTimed events, created on first enable
    struct Timed { int variant; double flops; };
    std::vector<Timed> timed;
};

namespace symb {

inline symb_status fail(symb_handle h, symb_status st, const char* fmt, ...) {
    char buf[512];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(buf, sizeof buf, fmt, ap);
    va_end(ap);
    if (h) h->error = buf;
    g_tls_error = buf;
    return st;
}

#define SYMB_HIP(h, call)                                                                      \
    do {                                                                                       \
        hipError_t e_ = (call);                                                                \
        if (e_ != hipSuccess)                                                                  \
            return fail(h, SYMB_ERR_DEVICE, "%s failed: %s", #call, hipGetErrorString(e_));    \
    } while (0)

inline bool misaligned16(const void* p) { return ((uintptr_t)p & 15) != 0; }

// ---- descriptor blob -------------------------------------------------------------------------
struct Blob {
    std::vector<unsigned char> bytes;
    template <class T>
    size_t add(const T* p, size_t n) {
        const size_t off = align_up(bytes.size(), 16);
        bytes.resize(off + std::max<size_t>(n, 1) * sizeof(T));
        if (n) memcpy(bytes.data() + off, p, n * sizeof(T));
        return off;
    }
};

inline symb_status upload(symb_handle h, const Blob& blob, hipStream_t st, unsigned char** dev_base) {
    if (blob.bytes.size() > kSlotBytes)
        return fail(h, SYMB_ERR_UNSUPPORTED, "batch descriptors need %zu bytes, capacity is %zu", blob.bytes.size(), kSlotBytes);
    // The kernels only read a slot's device copy (the K-split arrival counters are back at zero when
    // a launch ends), so a batch that comes again with the same offsets, adapters and buffers -- the
    // next decode step of the same clients, the same projection in the next training step -- finds
    // its descriptors in place.  The pinned copy of a slot is what its device copy holds.
    const size_t n = blob.bytes.size();
    uint64_t hash = 0x9E3779B97F4A7C15ull ^ n;
    {
        size_t i = 0;
        for (; i + 8 <= n; i += 8) {
            uint64_t w;
            memcpy(&w, blob.bytes.data() + i, 8);
            hash = (hash ^ w) * 0x100000001B3ull;
            hash ^= hash >> 29;
        }
        for (; i < n; ++i) hash = (hash ^ blob.bytes[i]) * 0x100000001B3ull;
    }
    h->ring.begin(h->rt, st);
    const int in_place = h->opt_desc_reuse ? h->ring.find(n, hash, [&](int j) { return memcmp(h->host_ring + (size_t)j * kSlotBytes, blob.bytes.data(), n) == 0; }) : -1;
    if (in_place >= 0) {
        h->call_slot = in_place;
        ++h->desc_in_place;
        *dev_base = h->dev_ring + (size_t)in_place * kSlotBytes;
        return SYMB_OK;
    }
    SYMB_HIP(h, h->ring.take(h->rt));
    const int slot = h->call_slot = h->ring.cur;
    unsigned char* hp = h->host_ring + (size_t)slot * kSlotBytes;
    unsigned char* dp = h->dev_ring + (size_t)slot * kSlotBytes;
    memcpy(hp, blob.bytes.data(), n);
    SYMB_HIP(h, hipMemcpyAsync(dp, hp, n, hipMemcpyHostToDevice, st));
    ++h->desc_sent;
    SYMB_HIP(h, h->ring.sent(h->rt, n, hash));
    *dev_base = dp;
    return SYMB_OK;
}

// A call that fails after its descriptors went to a slot may leave that slot's device copy in a state
// no later call should take over (a GEMM that never ran has not put its K-split counters back to zero, a
// launch may be half enqueued): unless the call completes, its slot is never matched again.
struct CallGuard {
    symb_handle h;
    bool completed = false;
    explicit CallGuard(symb_handle h_) : h(h_) { h->call_slot = -1; }
    ~CallGuard() {
        if (!completed && h->call_slot >= 0) h->ring.slot[h->call_slot].size = SIZE_MAX;
    }
};

inline symb_status seal_slot(symb_handle h) {
    SYMB_HIP(h, h->ring.seal(h->rt));
    return SYMB_OK;
}

inline symb_status check_handle(symb_handle h) {
    if (!h) return fail(nullptr, SYMB_ERR_INVALID_ARG, "handle is null");
    if (hipSetDevice(h->device) != hipSuccess) return fail(h, SYMB_ERR_DEVICE, "hipSetDevice(%d) failed", h->device);
    return SYMB_OK;
}

// Nothing throws across the C boundary: the work lists are the only allocations.
template <class F>
symb_status guarded(symb_handle h, F&& f) {
    try {
        return f();
    } catch (const std::bad_alloc&) {
        return fail(h, SYMB_ERR_UNSUPPORTED, "out of host memory for the batch's work lists");
    }
}

inline symb_status check_segments(symb_handle h, int32_t S, const int32_t* off) {
    if (S < 0) return fail(h, SYMB_ERR_INVALID_ARG, "num_segments is negative");
    if (!off) return fail(h, SYMB_ERR_INVALID_ARG, "seg_offsets is null");
    if (off[0] != 0) return fail(h, SYMB_ERR_BAD_SEGMENTS, "seg_offsets[0] must be 0");
    for (int i = 0; i < S; ++i)
        if (off[i + 1] < off[i]) return fail(h, SYMB_ERR_BAD_SEGMENTS, "seg_offsets decrease at segment %d", i);
    return SYMB_OK;
}

// The size of a Blob of these lists: what the workspace queries refuse as the calls do.
inline size_t blob_bytes(std::initializer_list<std::pair<size_t, size_t>> lists) {              // (entries, bytes of one)
    size_t n = 0;
    for (const auto& l : lists) n = align_up(n, 16) + std::max<size_t>(l.first, 1) * l.second;
    return n;
}

}  // namespace symb
