// Rows of streams (rh_state_rows) cut into pieces of work, which workgroups find by themselves: the offsets lie in device memory.
#pragma once
#include "seq_common.h"

#define STREAMS_T 256            // threads of the workgroups that do

struct streams_args {
    const int32_t *offsets, *slots, *into, *past;
    int32_t n_streams, n_rows, n_slots;
};

// the rows of stream b, in [0, n_rows) whatever the offsets say; false where the offsets descend
__device__ __forceinline__ bool streams_rows(const streams_args& r, int b, int32_t& begin, int32_t& end)
{
    auto clipped = [&](int32_t v) { return v < 0 ? 0 : v > r.n_rows ? r.n_rows : v; };
    begin = clipped(r.offsets[b]); end = clipped(r.offsets[b + 1]);
    return begin <= end;
}
// the slot that a stream's state is read from, -1 where it is zeros; and the one it goes to, -1 where it goes nowhere
__device__ __forceinline__ int32_t streams_slot(const streams_args& r, int b)
{
    const int32_t s = r.slots[b];
    return s < 0 || s >= r.n_slots || (r.past && r.past[b] <= 0) ? -1 : s;
}
__device__ __forceinline__ int32_t streams_into(const streams_args& r, int b)
{
    const int32_t s = r.into[b];
    return s < 0 || s >= r.n_slots ? -1 : s;
}

// For every stream the sum of count(rows) over the streams before it, in s[0 .. n_streams], the last being the sum of all.  False, for every thread, where any
// offsets descend: every workgroup of a call then finds the same and leaves everything as it is, counters between workgroups among it.
template <typename F>
__device__ __forceinline__ bool streams_sums(const streams_args& r, int32_t* s, int32_t* s_wave, F count)
{
    constexpr int PER = RH_SEQ_MAX_STREAMS / STREAMS_T;
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6, per = (r.n_streams + STREAMS_T - 1) / STREAMS_T, b0 = t * per;
    int32_t n[PER], mine = 0;
    bool ascend = true;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        n[i] = 0;
        if (i >= per || b0 + i >= r.n_streams) continue;
        int32_t begin, end;
        if (!streams_rows(r, b0 + i, begin, end)) { ascend = false; continue; }
        n[i] = count(end - begin);
        mine += n[i];
    }
    int32_t before = seq_scan(mine);
    ascend = __all(ascend);
    if (lane == 63) s_wave[wave] = ascend ? before : -1;     // sums of counts are below 2^31 where offsets ascend
    __syncthreads();
    before -= mine;
#pragma unroll
    for (int w = 0; w < STREAMS_T / 64; ++w) { ascend = ascend && s_wave[w] >= 0; if (w < wave) before += s_wave[w]; }
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        if (i >= per || b0 + i >= r.n_streams) continue;
        s[b0 + i] = before;
        before += n[i];
    }
    if (t == STREAMS_T - 1) s[r.n_streams] = before;         // it has the last streams, or none behind them
    __syncthreads();
    return ascend;
}
// The same of up to 64 streams, a stream a lane: its rows, and the sum over the streams before it.
struct streams_lane { int32_t begin, end, before, count; };
template <typename F>
__device__ __forceinline__ bool streams_few(const streams_args& r, F count, streams_lane& s, int32_t& all)
{
    const int lane = threadIdx.x & 63;
    s.begin = s.end = 0;
    const bool ascend = lane >= r.n_streams || streams_rows(r, lane, s.begin, s.end);
    s.count = ascend ? count(s.end - s.begin) : 0;
    const int32_t upto = seq_scan(s.count);
    all = __builtin_amdgcn_readlane(upto, 63);
    s.before = upto - s.count;
    return __all(ascend);
}
// Largest b in [0, n) with s[b] <= q; s ascending, s[0] = 0 <= q.
__device__ __forceinline__ int streams_find(const int32_t* s, int n, int32_t q)
{
    int lo = 0;
    for (int hi = n; hi - lo > 1;) { const int mid = (lo + hi) >> 1; if (s[mid] <= q) lo = mid; else hi = mid; }
    return lo;
}

// v / (1 + exp(-v)) within (|v| + 8) 2^-24 of itself: the power's argument is rounded once, and power and reciprocal are the hardware's
__device__ __forceinline__ float seq_silu(float v) { return v * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(v * -1.44269504089f)); }

// refusals of a call's rows; `name` is the call's
rh_status streams_check(rh_ctx* ctx, const char* name, const rh_state_rows* r, streams_args* a);
