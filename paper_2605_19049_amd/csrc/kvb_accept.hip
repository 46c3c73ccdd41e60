// kvb_accept: which drafted tokens the target's probabilities accept, and the token that follows.
//
// The walk down the drafts needs single probabilities.  What has to be read as a whole is one row of the target (and the draft's row
// that was rejected there): the token that follows is drawn from what is left of it.  Weights are whole multiples of 2^-48, held as fp64
// integers, so sums of up to 32 are exact in any order (probabilities sum to 1) and the token does not depend on how
// the row was split; rows that sum to more get one of their tokens.  All comparisons are in fp32, each operation rounded by itself (no contraction): p and q of 16 bits are exact.
//   few, long rows     kvb_accept_sum_kernel walks and sums a row's segments side by side, kvb_accept_find_kernel looks for the token
//   otherwise          kvb_accept_row_kernel does both, a workgroup a request
//   trees with draft probabilities: after a rejection the next sibling is tested against the sum of what is left, a whole row;
//                      a workgroup a request, which reads the target's row and those of all drafts rejected there once more for each sum.
//                      8 siblings, fp32, 150001 tokens: 1 request 81 us with 1.4 of them rejected, 245 with 6.2; 64 requests 430 and 473
// Bounded by reading the rows where there are many: 128 requests of 150001 tokens, 4 drafts, fp32, 146 MB, 35.6 us or 4.1 TB/s; few are bounded by
// the chain launch, walk (two loads), sum, search: 1 request of 32000 tokens 9 us.  Rows are read twice, to sum and to find, the second time
// only the part of a row that holds the token: which weight the random number falls on is known only after the sum.
#include "kvb_accept_device.h"

namespace kvb_impl {

#pragma clang fp contract(off)

namespace {

using Walk = AcceptWalk;
template <typename T>
struct Probs {
    const T *p;              // the place's row of the target
    const T *q;              // the request's draft rows, or nullptr
    const int32_t *tokens;   // the request's
    const float *mass;       // the sum of what was left before each draft that was rejected there (in LDS)
    int64_t stride;
};
template <typename T>
__device__ __forceinline__ Probs<T> probs_of(const AcceptArgs &a, int b, int place, const float *mass)
{
    return Probs<T>{static_cast<const T *>(a.target) + ((int64_t)b * (a.T + 1) + place + 1) * a.stride,
                    a.draft ? static_cast<const T *>(a.draft) + (int64_t)b * a.T * a.stride : nullptr, a.tokens + (int64_t)b * a.T, mass, a.stride};
}

// what is left of r when as much as `taken` is not there
__device__ __forceinline__ float less(float r, float taken)
{
    const float t = r - taken;
    return t < 0.0f ? 0.0f : t;
}
// What is left of the place's probabilities r of N tokens from j on.  A chain rejects one draft at most, with nothing lost before.
template <bool TREE, int N, typename T, typename Get>
__device__ __forceinline__ void leave(const Probs<T> &rows, const Walk &w, int j, float (&r)[N], Get &&get)
{
    for (uint32_t bits = w.rejected; bits; bits &= bits - 1) {
        const int m = __builtin_ctz(bits);
        if (rows.q) {
            float q[N];
            get(rows.q + m * rows.stride + j, q);
            const float mass = TREE ? rows.mass[m] : 1.0f;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float taken = mass * q[i];
                r[i] = less(r[i], taken);
            }
        } else {
            const int x = rows.tokens[m] - j;
#pragma unroll
            for (int i = 0; i < N; ++i)
                r[i] = x == i ? 0.0f : r[i];
        }
        if constexpr (!TREE)
            break;
    }
}
// a probability as a whole number of 2^-48
__device__ __forceinline__ double weight(float r)
{
    const float w = r > 0.0f ? fminf(r, 1.0f) : 0.0f;
    return (double)truncf(w * 0x1p48f);
}

__device__ __forceinline__ double wave_sum(double x)
{
#pragma unroll
    for (int s = 32; s > 0; s /= 2)
        x += __shfl_xor(x, s);
    return x;
}

// N elements at any element's address
template <int N, typename T>
__device__ __forceinline__ void load_any(const T *p, float (&x)[N])
{
    struct __attribute__((packed, aligned(sizeof(T)))) Any { T t[N]; };
    const Any a = *reinterpret_cast<const Any *>(p);
#pragma unroll
    for (int i = 0; i < N; ++i)
        x[i] = to_f32(a.t[i]);
}
template <bool TREE, int N, typename T>
__device__ __forceinline__ void left_at(const Probs<T> &rows, const Walk &w, int j, float (&r)[N])
{
    load_any(rows.p + j, r);
    leave<TREE>(rows, w, j, r, [](const T *p, float (&q)[N]) { load_any(p, q); });
}

// Sum of the weights of tokens lo .. hi-1 over the lanes of a wave; all lanes get it
template <bool TREE, typename T>
__device__ double sum_range(const Probs<T> &rows, const Walk &w, int lo, int hi)
{
    double s = 0.0;
    int j = lo + 8 * (int)(threadIdx.x % 64);
#pragma unroll 4
    for (; j + 8 <= hi; j += 512) {
        float r[8];
        left_at<TREE>(rows, w, j, r);
#pragma unroll
        for (int i = 0; i < 8; ++i)
            s += weight(r[i]);
    }
    for (; j < hi; ++j) {   // (what one lane has of a last, short step)
        float r[1];
        left_at<TREE>(rows, w, j, r);
        s += weight(r[0]);
    }
    return wave_sum(s);
}

// Sum over the whole row by all waves of the workgroup (part: one double a wave in LDS; all threads call it and get the sum).
// Wave v has the range bounds(v) .. bounds(v + 1).
__device__ __forceinline__ int bound_of(int lo, int hi, int v, int waves)
{
    const int each = ((hi - lo + waves - 1) / waves + 511) / 512 * 512;
    return min(hi, lo + v * each);
}
template <bool TREE, int WAVES, typename T>
__device__ double sum_row(const Probs<T> &rows, const Walk &w, int lo, int hi, double *part)
{
    const int wave = threadIdx.x / 64;
    const double s = sum_range<TREE>(rows, w, bound_of(lo, hi, wave, WAVES), bound_of(lo, hi, wave + 1, WAVES));
    __syncthreads();
    if (threadIdx.x % 64 == 0)
        part[wave] = s;
    __syncthreads();
    double total = 0.0;
    for (int v = 0; v < WAVES; ++v)
        total += part[v];
    return total;
}

// Sums of weights up to here are exact.  Only rows that are no probabilities reach it, and then an aim may fall between two sums of the
// same tokens that were rounded differently: the search takes care of that (where told so; 0.5 us otherwise).
constexpr double EXACT_SUM = 0x1p53;
// The first of n ranges, with sums at(0) .. at(n - 1) of which one at least is not zero, whose running sum exceeds aim; aim becomes what is
// left of it there.  rounded: an aim that passes the last one gets the last range with anything in it, and so on inside.
template <typename At>
__device__ __forceinline__ int pick(int n, double &aim, bool rounded, At &&at)
{
    if (!rounded) {
        int v = 0;
        for (; v + 1 < n && at(v) <= aim; ++v)
            aim -= at(v);
        return v;
    }
    int last = 0;
    for (int v = 0; v < n; ++v) {
        const double s = at(v);
        if (aim < s)
            return v;
        aim -= s;
        last = s > 0.0 ? v : last;
    }
    aim = __builtin_huge_val();
    return last;
}
// The first token of lo .. hi-1 whose running sum exceeds aim (as in pick), hi - lo some hundreds: a few neighbours
// a thread.  The thread that has it writes it.
template <bool TREE, int WAVES, typename T>
__device__ void find_in(const Probs<T> &rows, const Walk &w, int lo, int hi, double aim, bool rounded, double *part, int32_t *to)
{
    const int wave = threadIdx.x / 64, lane = threadIdx.x % 64, each = (hi - lo + 64 * WAVES - 1) / (64 * WAVES);
    const int from = min(hi, lo + (int)threadIdx.x * each), end = min(hi, from + each);
    auto at = [&](int j) {
        float r[1];
        left_at<TREE>(rows, w, j, r);
        return weight(r[0]);
    };
    double own = 0.0;
    for (int j = from; j < end; ++j)
        own += at(j);
    double upto = own;
#pragma unroll
    for (int s = 1; s < 64; s *= 2) {
        const double x = __shfl_up(upto, s);
        upto += lane >= s ? x : 0.0;
    }
    __syncthreads();
    if (lane == 63)
        part[wave] = upto;
    __syncthreads();
    if (rounded) {
        if (wave != pick(WAVES, aim, true, [&](int v) { return part[v]; }))
            return;
        const uint64_t some = __ballot(own > 0.0), past = __ballot(own > 0.0 && aim < upto);
        if (lane != (past ? __builtin_ctzll(past) : 63 - __builtin_clzll(some | 1)))
            return;
        double run = upto - own;
        for (int j = from; j < end; ++j) {
            const double x = at(j);
            if (x > 0.0) {
                *to = j;
                run += x;
                if (aim < run)
                    break;
            }
        }
        return;
    }
    for (int v = 0; v < wave; ++v)
        upto += part[v];
    double run = upto - own;
    if (run <= aim && aim < upto)
        for (int j = from; j < end; ++j) {
            run += at(j);
            if (aim < run) {
                *to = j;
                break;
            }
        }
}
// The same for a range of any length whose waves' sums are in `part`: on to the wave's range that has it, until that is short.
template <bool TREE, int WAVES, typename T>
__device__ void find_long(const Probs<T> &rows, const Walk &w, int lo, int hi, double aim, bool rounded, double *part, int32_t *to)
{
    for (;;) {
        const int v = pick(WAVES, aim, rounded, [&](int i) { return part[i]; });
        const int from = bound_of(lo, hi, v, WAVES), end = bound_of(lo, hi, v + 1, WAVES);
        lo = from;
        hi = end;
        if (hi - lo <= 128 * WAVES)
            break;
        sum_row<TREE, WAVES>(rows, w, lo, hi, part);
    }
    find_in<TREE, WAVES>(rows, w, lo, hi, aim, rounded, part, to);
}

// floor(s total), below total
__device__ __forceinline__ double aim_of(float s, double total)
{
    const float in = s > 0.0f ? fminf(s, 0x1.fffffep-1f) : 0.0f;
    return floor((double)in * total);
}

// lane i's word, for a scalar i
__device__ __forceinline__ int of_lane(int x, int i) { return __builtin_amdgcn_readlane(x, i); }
__device__ __forceinline__ float of_lane(float x, int i) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), i)); }

// Walks down the drafts of request b.  All waves do, with the same result.  A draft's place is its parent, so every probability
// that a test may need is known ahead: lane 8 m + i loads draft i's token, its target's and its own probability and what draft m's
// row gives it, at once; the walk itself touches no memory.  FULL: the sums of what rejections left are needed on
// the way (trees of drafts with probabilities); all threads of the workgroup then take part.
template <bool TREE, bool FULL, int WAVES, typename T>
__device__ Walk walk(const AcceptArgs &a, int b, Probs<T> &rows, float *mass_at, double *part)
{
    const int lane = threadIdx.x % 64, i0 = min(lane % 8, a.T - 1), m0 = min(lane / 8, a.T - 1);
    const T *target = static_cast<const T *>(a.target) + (int64_t)b * (a.T + 1) * a.stride;
    rows = probs_of<T>(a, b, -1, mass_at);
    const int n = __builtin_amdgcn_readfirstlane(a.n_drafts ? min(max(a.n_drafts[b], 0), a.T) : a.T);
    const int x = rows.tokens[i0], up = TREE && a.parent ? a.parent[(int64_t)b * a.T + i0] : i0 - 1;
    const float u = a.u[(int64_t)b * a.T + i0];
    const int parent = up < -1 || up >= i0 ? -1 : up, known = x >= 0 && x < a.V, xs = known ? x : 0;
    const float pt = to_f32(target[(parent + 1) * a.stride + xs]), p = pt == pt ? pt : 0.0f;   // (no number: nothing, and what is left loses nothing)
    const float q = rows.q ? to_f32(rows.q[m0 * a.stride + xs]) : 1.0f;   // of token i in row m

    Walk w{-1, 0, 0};
    float mass = 1.0f;
    float lost[KVB_MAX_DRAFTS];
#pragma unroll
    for (int i = 0; i < KVB_MAX_DRAFTS; ++i) {
        lost[i] = mass;
        if (i < n && of_lane(parent, i) == w.place) {
            const int xi = of_lane(x, i);
            float r = of_lane(p, i);
#pragma unroll
            for (int m = 0; m < i; ++m)
                if (w.rejected >> m & 1) {
                    if (rows.q) {
                        const float taken = lost[m] * of_lane(q, 8 * m + i);
                        r = less(r, taken);
                    } else {
                        r = of_lane(x, m) == xi ? 0.0f : r;
                    }
                }
            const float uq = of_lane(u, i) * of_lane(q, 9 * i);
            const bool there = of_lane(known, i) != 0;
            if (there && uq * mass < r) {
                w.accepted |= 1u << i;
                w.rejected = 0;
                w.place = i;
                mass = 1.0f;
            } else {
                w.rejected |= 1u << i;
                if (!rows.q) {
                    mass = there ? less(mass, r) : mass;
                } else if constexpr (FULL) {
                    bool more = false;
#pragma unroll
                    for (int k = i + 1; k < KVB_MAX_DRAFTS; ++k)
                        more |= k < n && of_lane(parent, k) == w.place;
                    if (threadIdx.x == 0)
                        mass_at[i] = lost[i];
                    if (more) {
                        __syncthreads();
                        rows.p = target + (w.place + 1) * a.stride;
                        mass = (float)(sum_row<TREE, WAVES>(rows, w, 0, a.V, part) * 0x1p-48);
                    }
                }
            }
        }
    }
    rows.p = target + (w.place + 1) * a.stride;
    if constexpr (FULL)
        __syncthreads();   // (mass_at)
    return w;
}

__device__ __forceinline__ void write_walk(const AcceptArgs &a, int b, const Walk &w)
{
    const int i = threadIdx.x;
    if (i < a.T) {   // the i-th accepted draft
        uint32_t bits = w.accepted;
        for (int k = 0; k < i; ++k)
            bits &= bits - 1;
        a.path[(int64_t)b * a.T + i] = bits ? __builtin_ctz(bits) : -1;
    }
    if (i == 0)
        a.accepted[b] = __popc(w.accepted);
}

// Looks for the token when the whole row's wave sums are in `part` and its total is known (0: falls back on the target's row,
// and on no token if that sums to nothing either).
template <bool TREE, int WAVES, typename T>
__device__ void find_row(const AcceptArgs &a, int b, const Probs<T> &rows, Walk &w, double total, double *part)
{
    if (total == 0.0 && w.rejected) {
        w.rejected = 0;
        total = sum_row<TREE, WAVES>(rows, w, 0, a.V, part);
    }
    if (total == 0.0) {
        if (threadIdx.x == 0)
            a.token[b] = -1;
        return;
    }
    find_long<TREE, WAVES>(rows, w, 0, a.V, aim_of(a.s[b], total), total >= EXACT_SUM, part, a.token + b);
}

}  // namespace

// The whole of a request by one workgroup
template <typename T, bool TREE, bool FULL>
__global__ __launch_bounds__(1024) void kvb_accept_row_kernel(const AcceptArgs a)
{
    __shared__ double part[16];
    __shared__ float mass[KVB_MAX_DRAFTS];
    const int b = blockIdx.x;
    Probs<T> rows;
    Walk w = walk<TREE, FULL, 16>(a, b, rows, mass, part);
    write_walk(a, b, w);
    const double total = sum_row<TREE, 16>(rows, w, 0, a.V, part);
    find_row<TREE, 16>(a, b, rows, w, total, part);
}

// One segment of a request's row: its sum goes to sums[b][segment]
template <typename T, bool TREE>
__global__ __launch_bounds__(256) void kvb_accept_sum_kernel(const AcceptArgs a)
{
    __shared__ double part[4];
    const int b = blockIdx.x / a.segments, s = blockIdx.x - b * a.segments;
    Probs<T> rows;
    const Walk w = walk<TREE, false, 4>(a, b, rows, nullptr, part);
    const double sum = sum_row<TREE, 4>(rows, w, min(a.V, s * a.segment), min(a.V, (s + 1) * a.segment), part);
    if (threadIdx.x == 0) {
        a.sums[(int64_t)b * a.segments + s] = sum;
        if (s == 0)
            a.walks[b] = w;
    }
    if (s == 0)
        write_walk(a, b, w);
}

// The token from the segments' sums
template <typename T, bool TREE>
__global__ __launch_bounds__(1024) void kvb_accept_find_kernel(const AcceptArgs a)
{
    __shared__ double part[16];
    const int b = blockIdx.x;
    Walk w = a.walks[b];
    Probs<T> rows = probs_of<T>(a, b, w.place, nullptr);
    const double *sums = a.sums + (int64_t)b * a.segments;
    double total = 0.0;
    for (int s = 0; s < a.segments; ++s)
        total += sums[s];
    if (total == 0.0) {
        find_row<TREE, 16>(a, b, rows, w, total, part);
        return;
    }
    double aim = aim_of(a.s[b], total);
    const bool rounded = total >= EXACT_SUM;
    const int s = pick(a.segments, aim, rounded, [&](int i) { return sums[i]; });
    const int lo = min(a.V, s * a.segment), hi = min(a.V, (s + 1) * a.segment);
    sum_row<TREE, 16>(rows, w, lo, hi, part);
    find_long<TREE, 16>(rows, w, lo, hi, aim, rounded, part, a.token + b);
}

namespace {

template <typename T, bool TREE>
void launch_split(const AcceptArgs &a, hipStream_t stream)
{
    if (a.segments == 1) {
        launch_part(kvb_accept_row_kernel<T, TREE, false>, true, true, a.B, 1024, stream, a);
    } else {
        launch_part(kvb_accept_sum_kernel<T, TREE>, true, false, (int64_t)a.B * a.segments, 256, stream, a);
        launch_part(kvb_accept_find_kernel<T, TREE>, false, true, a.B, 1024, stream, a);
    }
}
template <typename T>
void launch_accept_typed(const AcceptArgs &a, hipStream_t stream)
{
    if (a.draft && a.parent)
        launch_part(kvb_accept_row_kernel<T, true, true>, true, true, a.B, 1024, stream, a);
    else if (a.parent)
        launch_split<T, true>(a, stream);
    else
        launch_split<T, false>(a, stream);
}

}  // namespace

void launch_accept(int dtype, const AcceptArgs &a, hipStream_t stream)
{
    if (dtype == KVB_F32)
        launch_accept_typed<float>(a, stream);
    else if (dtype == KVB_BF16)
        launch_accept_typed<bf16_t>(a, stream);
    else
        launch_accept_typed<f16_t>(a, stream);
}

}  // namespace kvb_impl
