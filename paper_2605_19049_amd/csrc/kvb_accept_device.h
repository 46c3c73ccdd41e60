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

// Segments of a row, each a workgroup; 1: the whole of a request by one workgroup, in one launch instead of two.  A row is split where one
// workgroup would read it for longer than a launch takes and the requests alone do not fill the card.  us, split against whole rows, 4 drafts,
// fp32, nothing in the caches: 1 request of 32000 tokens 11.1 / 8.9, of 40000 10.7 / 10.5; 64 requests of 32000 15.5 / 11.0, of 65537 16.2 / 17.9, of
// 150001 22.5 / 31.8; 128 of 65537 21.5 / 18.5, of 150001 35.7 / 38.5; 256 of 150001, bf16, 48.5 / 41.3.  Segments of at least 8192 (16384: 32
// of 150001 18.3, against 16.2), about 1024 in all.
inline int accept_split_most(int V) { return V < 32768 ? 0 : V < 131072 ? 64 : 128; }   // requests up to which rows are split; grows with V
inline int accept_segments(int B, int V)
{
    if (B > accept_split_most(V))
        return 1;
    const int most = V / 8192, want = 1024 / (B < 1 ? 1 : B);
    return want < most ? want : most;
}
inline int accept_segment(int V, int segments) { return ((V + segments - 1) / segments + 2047) / 2048 * 2048; }

// Bytes of workspace: the most that a call of up to B requests and up to V tokens needs, so that one of this size serves smaller calls
// too.  (One of fewer requests may need more than one of B, whose rows are not split.)  A sum for each segment, of which there are at most V / 8192 a
// request and 1024 in all, and a walk for each request whose row is split.
inline int64_t accept_work_bytes(int B, int V)
{
    const int64_t most = accept_split_most(V), split = B < most ? B : most, sums = split * (V / 8192) < 1024 ? split * (V / 8192) : 1024;
    const int64_t need = 8 * sums + 16 * split;
    return need > 8 * (int64_t)B ? need : 8 * (int64_t)B;
}
static_assert(sizeof(AcceptWalk) <= 16);

void launch_accept(int dtype, const AcceptArgs &a, hipStream_t stream);   // kvb_accept.hip

}  // namespace kvb_impl
#endif  // KVB_ACCEPT_DEVICE_H
