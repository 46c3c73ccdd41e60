// The arguments of kvb_accept's kernels and how a row is split.
#ifndef KVB_ACCEPT_DEVICE_H
#define KVB_ACCEPT_DEVICE_H

#include "kvb_scan_device.h"

namespace kvb_impl {

// Where the walk ended, as scalars: drafts accepted on the way and drafts rejected at the end (bit i: draft i), both in the order
// of the drafts.
struct AcceptWalk {
    int place;
    uint32_t accepted, rejected;
};

struct AcceptArgs {
    const int32_t *n_drafts;   // [B] or nullptr: T
    const int32_t *parent;     // [B][T] or nullptr: a chain
    const int32_t *tokens;     // [B][T]
    const void *target;        // [B][T + 1][stride]
    const void *draft;         // [B][T][stride] or nullptr: certain drafts
    const float *u, *s;        // [B][T], [B]
    int32_t *path, *accepted, *token;
    double *sums;              // [B][segments]
    AcceptWalk *walks;         // [B]
    int64_t stride;
    int32_t B, T, V, segments, segment;
};

// Segments of a row, each a workgroup.
inline int accept_segments(int B, int V)
{
    const int most = V / 8192;
    const int want = 1024 / (B < 1 ? 1 : B);
    return most < 2 || want < 2 ? 1 : want < most ? want : most;
}
inline int accept_segment(int V, int segments) { return ((V + segments - 1) / segments + 2047) / 2048 * 2048; }

void launch_accept(int dtype, const AcceptArgs &a, hipStream_t stream);   // kvb_accept.hip

}  // namespace kvb_impl
#endif  // KVB_ACCEPT_DEVICE_H
