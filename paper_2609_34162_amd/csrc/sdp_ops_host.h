// Host code that the entry points of the training operators share (sdp_ops.hip has
// it; sdp_layer.hip uses it too): checks of their buffers, the context's workspace
// for them, and exceptions kept inside.  Not installed; not part of the ABI.
#pragma once

#include <utility>
#include <vector>

#include "sdp_ops.h"
#include "sdp_ops_plan.h"
#include "sdp_rt.h"

namespace sdpops {

// ---- checks -----------------------------------------------------------------

inline bool is_float_type(int t) { return t == SDP_TYPE_F32 || t == SDP_TYPE_BF16; }
inline bool is_int_type(int t) { return t == SDP_TYPE_I32 || t == SDP_TYPE_I64; }
inline int64_t type_size(int t) { return t == SDP_TYPE_BF16 ? 2 : t == SDP_TYPE_I64 ? 8 : 4; }

// A buffer of a call: where it lies, and whether the call writes it.
struct Tensor {
    const char *what;
    const void *p;
    Layout layout;
    int64_t size;  // of an element
    bool written;
};

inline Tensor dense(const char *what, const void *p, int64_t n, int64_t size, bool written) {
    return {what, p, Layout{{1, 1, 1}, {0, 0, 0}, n}, size, written};
}
inline Tensor rows_of(const char *what, const void *p, int64_t rows, int64_t stride, int64_t cols, int64_t size, bool written) {
    return {what, p, Layout{{1, rows, 1}, {0, rows > 1 ? stride : 0, 0}, cols}, size, written};
}

// Every buffer lies in device memory of the context's GPU, aligned to its
// elements; no output overlaps itself or another buffer, except that a pair of
// in_place (indexes into ts) may be the very same tensor.
int check_tensors(const sdp_ctx *ctx, const char *call, const std::vector<Tensor> &ts,
                  const std::vector<std::pair<int, int>> &in_place);

// ---- workspace ----------------------------------------------------------------

// The workspace for a call, which then runs after the last one that used it.  A
// captured graph would keep the workspace's address after it has grown, and the
// context's event would become part of the capture, so such a call is refused.
int take_ops_space(sdp_ctx *ctx, const char *call, size_t bytes, hipStream_t s);
// After the last launch of a call that took the workspace.
int ops_mark(sdp_ctx *ctx, hipStream_t s);

// ---- entry points ---------------------------------------------------------------

// No C++ exception leaves a C entry point: what allocates here is the host's
// own bookkeeping.
template <class F>
int guarded(F &&body) {
    sdprt::t_err.clear();
    try {
        return body();
    } catch (const std::bad_alloc &) {
        return sdprt::fail(SDP_ERR_OUT_OF_MEMORY, "out of host memory");
    } catch (const std::exception &e) {
        return sdprt::fail(SDP_ERR_INVALID_ARGUMENT, "%s", e.what());
    }
}

}  // namespace sdpops
