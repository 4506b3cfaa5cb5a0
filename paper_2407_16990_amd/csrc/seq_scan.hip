// rh_state_scan: the entry, and the scan of bf16 rows.
#include "seq_scan.h"

hipError_t scan_launch_f32(rh_ctx* ctx, scan_args& a, rh_status* failed);

extern "C" rh_status rh_state_scan(rh_ctx* ctx, const rh_state_rows* rows, const rh_scan_inputs* in, float* state, void* y, int64_t y_stride)
{
    if (!ctx) return RH_E_INVALID;
    if (!rows || !in) RH_FAIL(ctx, RH_E_INVALID, "rh_state_scan: null argument");
    scan_args a;
    const rh_status st = streams_check(ctx, "rh_state_scan", rows, &a.r);
    if (st != RH_OK) return st;
    if (in->type != RH_T_F32 && in->type != RH_T_BF16) RH_FAIL(ctx, RH_E_INVALID, "rh_state_scan: rows of type %d", in->type);
    if (in->channels < 1 || in->channels > RH_SEQ_MAX_CHANNELS) RH_FAIL(ctx, RH_E_SHAPE, "rh_state_scan: %d channels (1 to %d)", in->channels, RH_SEQ_MAX_CHANNELS);
    if (in->groups < 1 || in->channels % in->groups) RH_FAIL(ctx, RH_E_SHAPE, "rh_state_scan: %d channels in %d groups", in->channels, in->groups);
    if (in->n < 1 || in->n > RH_SEQ_MAX_STATE) RH_FAIL(ctx, RH_E_SHAPE, "rh_state_scan: a state of %d (1 to %d)", in->n, RH_SEQ_MAX_STATE);
    if (in->x_stride < in->channels || in->dt_stride < in->channels || (in->gate && in->gate_stride < in->channels) || y_stride < in->channels)
        RH_FAIL(ctx, RH_E_SHAPE, "rh_state_scan: a row stride below %d", in->channels);
    if (in->b_stride < (int64_t)in->groups * in->n || in->c_stride < (int64_t)in->groups * in->n)
        RH_FAIL(ctx, RH_E_SHAPE, "rh_state_scan: a row stride of b or c below %lld", (long long)in->groups * in->n);
    if (rows->n_rows == 0 || rows->n_streams == 0) return RH_OK;
    if (!in->x || !in->dt || !in->b || !in->c || !in->a || !y || (rows->n_slots && !state)) RH_FAIL(ctx, RH_E_INVALID, "rh_state_scan: null argument");
    a.x = in->x; a.dt = in->dt; a.gate = in->gate; a.b = in->b; a.c = in->c; a.a = in->a; a.dt_bias = in->dt_bias; a.skip = in->skip;
    a.state = state; a.ws = nullptr; a.y = y; a.x_stride = in->x_stride; a.dt_stride = in->dt_stride; a.gate_stride = in->gate_stride;
    a.b_stride = in->b_stride; a.c_stride = in->c_stride; a.y_stride = y_stride; a.per = seq_make_div((uint32_t)(in->channels / in->groups));
    a.channels = in->channels; a.n = in->n; a.softplus = in->softplus != 0;
    rh_status failed = RH_OK;
    const hipError_t e = in->type == RH_T_F32 ? scan_launch_f32(ctx, a, &failed) : launch_scan<__bf16>(ctx, a, &failed);
    if (failed != RH_OK) return failed;
    RH_HIP(ctx, e);
    return RH_OK;
}
