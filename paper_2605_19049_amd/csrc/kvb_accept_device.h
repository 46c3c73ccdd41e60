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
// workgroup would take longer for it than a launch does and the requests alone do not fill the card.  That goes by tokens, not bytes: what a
// workgroup takes is the work and latency for each, 150001 tokens of bf16 38 us and of fp32 37.  us, split against whole rows, 4 drawn drafts, nothing in
// the caches, fp32: 1 request of 32768 tokens 11.7 / 9.8, of 40000 10.7 / 10.5, of 65537 13.4 / 14.1, of 150001 14.2 / 22.0; 64 of 32768 15.3 / 13.5, of
// 65537 18.6 / 20.8, of 150001 26.2 / 37.3; 96 of 65537 21.2 / 21.8, of 100003 25.5 / 28.4; 128 of 65537 24.8 / 22.8, of 100003 30.7 / 29.6, of 150001 38.5 / 41.5;
// 160 of 150001 47.1 / 44.3.  bf16: 64 of 65537 19.9 / 21.8; 128 of 65537 21.9 / 22.6, of 150001 32.3 / 40.5; 160 of 150001 37.7 / 41.0; 200 42.1 / 42.6; 256
// 51.5 / 43.6.  So the bounds are those of fp32, and on the low side for 16 bits; around 32768 tokens a split costs up to 2 us.  Segments of at
// least 8192 (16384: 32 of 150001 18.3, against 16.2), about 1024 in all.
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
