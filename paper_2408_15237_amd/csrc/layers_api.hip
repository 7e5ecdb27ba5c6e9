// The C ABI of the layer operators (ssmv_layers.h): argument validation on the host, before any HIP call, and kernel launches.
#include "api_checks.h"
#include "layers_internal.h"

using namespace ssmv;

namespace {

int check_layer_stride(int64_t *stride, long packed, const char *name)
{
    TRY(check_stride(stride, packed, name));
    if (*stride > SSMV_LAYER_STRIDE_MAX) return fail(SSMV_EUNSUPPORTED, "%s %lld > %d", name, (long long)*stride, SSMV_LAYER_STRIDE_MAX);
    return SSMV_OK;
}

int check_io_opt(const void *p, int io, const char *name) { return p ? check_io(p, io, name) : SSMV_OK; }
int check_f32_opt(const void *p, const char *name) { return p ? check_f32(p, name) : SSMV_OK; }

// a gradient of something that was not there
int check_no(const void *grad, const void *of, const char *name)
{
    return grad && !of ? fail(SSMV_EINVAL, "%s: there is no input that it is the gradient of", name) : SSMV_OK;
}

// in place is possible with one stride only
int check_alias(const void *out, int64_t out_stride, const void *in, int64_t in_stride, const char *what)
{
    return out && out == in && out_stride != in_stride ? fail(SSMV_EINVAL, "%s are one tensor with two strides", what) : SSMV_OK;
}

int check_norm_sizes(int rows, int channels)
{
    if (rows < 1 || channels < 1) return fail(SSMV_EINVAL, "rows %d and channels %d must be >= 1", rows, channels);
    if (channels > SSMV_BLOCK_NORM_MAX) return fail(SSMV_EUNSUPPORTED, "channels %d > %d", channels, SSMV_BLOCK_NORM_MAX);
    // a launch counts its threads with 32 bits: 64 for every 512 channels of a row
    if ((double)rows * ((channels + 511) / 512) * 64 > 4.0e9) return fail(SSMV_EUNSUPPORTED, "%d rows of %d channels: feed them in pieces", rows, channels);
    return SSMV_OK;
}

// what the forward and the backward call have in common
template <typename Args>
int check_norm(Args &a)
{
    TRY(check_io_type(a.io_dtype));
    TRY(check_io_type(a.res_dtype));
    if (a.res_dtype != a.io_dtype && a.res_dtype != SSMV_F32) return fail(SSMV_EINVAL, "res_dtype must be io_dtype or fp32");
    TRY(check_norm_sizes(a.rows, a.channels));
    if (!(a.eps >= 0.f)) return fail(SSMV_EINVAL, "eps must be >= 0");
    TRY(check_layer_stride(&a.x_stride, a.channels, "x_stride"));
    TRY(check_layer_stride(&a.z_stride, a.channels, "z_stride"));
    TRY(check_layer_stride(&a.res_stride, a.channels, "res_stride"));
    if (!a.x && !a.res) return fail(SSMV_EINVAL, "x and res are both NULL");
    if (!a.x && (a.z || a.post_wgt || a.ch_scale)) return fail(SSMV_EINVAL, "without x there is no z, post_wgt or ch_scale");
    TRY(check_io_opt(a.x, a.io_dtype, "x"));
    TRY(check_io_opt(a.z, a.io_dtype, "z"));
    TRY(check_io_opt(a.res, a.res_dtype, "res"));
    TRY(check_f32_opt(a.post_wgt, "post_wgt"));
    TRY(check_f32_opt(a.ch_scale, "ch_scale"));
    TRY(check_f32_opt(a.pre_wgt, "pre_wgt"));
    return SSMV_OK;
}

int check_gated_sizes(int batch, int channels, int L)
{
    if (batch < 1 || channels < 1 || L < 1) return fail(SSMV_EINVAL, "batch %d, channels %d and L %d must be >= 1", batch, channels, L);
    if (batch > 65535) return fail(SSMV_EUNSUPPORTED, "batch %d > 65535", batch);
    if (channels > (1 << 22) || L > (1 << 30)) return fail(SSMV_EUNSUPPORTED, "more than 2^22 channels or 2^30 tokens");
    return SSMV_OK;
}

template <typename Args>
int check_gated(Args &a)
{
    TRY(check_io_type(a.io_dtype));
    TRY(check_gated_sizes(a.batch, a.channels, a.L));
    if (a.form != SSMV_GATED_LRU && a.form != SSMV_GATED_MIX) return fail(SSMV_EINVAL, "form %d unknown", a.form);
    TRY(check_layer_stride(&a.x_stride, a.channels, "x_stride"));
    TRY(check_layer_stride(&a.f_stride, a.channels, "f_stride"));
    TRY(check_layer_stride(&a.i_stride, a.channels, "i_stride"));
    TRY(check_layer_stride(&a.z_stride, a.channels, "z_stride"));
    TRY(check_io(a.x, a.io_dtype, "x"));
    TRY(check_io(a.f, a.io_dtype, "f"));
    TRY(check_io_opt(a.i, a.io_dtype, "i"));
    TRY(check_io_opt(a.z, a.io_dtype, "z"));
    if (a.form == SSMV_GATED_LRU) TRY(check_f32(a.A, "A"));
    else if (a.A) return fail(SSMV_EINVAL, "A must be NULL in form SSMV_GATED_MIX");
    TRY(check_f32_opt(a.f_bias, "f_bias"));
    TRY(check_f32_opt(a.i_bias, "i_bias"));
    if (a.i_bias && !a.i) return fail(SSMV_EINVAL, "i_bias without i");
    if (!aligned_to(a.seq_len, 4)) return fail(SSMV_EALIGN, "seq_len is not 4-byte aligned");
    return SSMV_OK;
}

// two [batch][segments][C] arrays, each rounded to whole 16 bytes
size_t gated_segments(int batch, int channels, const GatedPlan &plan)
{
    return plan.seg_count == 1 ? 0 : ((size_t)batch * plan.seg_count * channels * sizeof(float) + 15) / 16 * 16;
}

}  // namespace

extern "C" {

int ssmv_block_norm(const ssmv_block_norm_args *args, void *hip_stream)
{
    if (!args) return fail(SSMV_EINVAL, "args is NULL");
    ssmv_block_norm_args a = *args;
    TRY(check_norm(a));
    TRY(check_layer_stride(&a.r_stride, a.channels, "r_stride"));
    TRY(check_layer_stride(&a.n_stride, a.channels, "n_stride"));
    TRY(check_io_opt(a.r_out, a.res_dtype, "r_out"));
    TRY(check_io_opt(a.n_out, a.io_dtype, "n_out"));
    if (!a.r_out && !a.n_out) return fail(SSMV_EINVAL, "r_out and n_out are both NULL");
    if (!a.x && a.r_out) return fail(SSMV_EINVAL, "without x r is res: r_out must be NULL");
    TRY(check_alias(a.r_out, a.r_stride, a.res, a.res_stride, "r_out and res"));
    if ((a.x && (a.r_out == a.x || a.n_out == a.x)) || (a.z && (a.r_out == a.z || a.n_out == a.z)) || (a.n_out && (a.n_out == a.res || a.n_out == a.r_out)))
        return fail(SSMV_EINVAL, "an output is an input or another output; only r_out may be res");
    BlockNormParams p{};
    p.x = a.x; p.z = a.z; p.res = a.res; p.post = a.post_wgt; p.scale = a.ch_scale; p.pre = a.pre_wgt; p.r_out = a.r_out; p.n_out = a.n_out;
    p.x_stride = a.x_stride; p.z_stride = a.z_stride; p.res_stride = a.res_stride; p.r_stride = a.r_stride; p.n_stride = a.n_stride;
    p.rows = a.rows; p.C = a.channels; p.io = a.io_dtype; p.res_io = a.res_dtype; p.eps = a.eps; p.alpha = a.res_scale;
    const int hc = launch_block_norm(p, (hipStream_t)hip_stream);
    return hc == 0 ? SSMV_OK : hip_fail(hc, "ssmv_block_norm");
}

int ssmv_block_norm_backward_workspace(int32_t rows, int32_t channels, size_t *out_bytes)
{
    TRY(check_norm_sizes(rows, channels));
    if (!out_bytes) return fail(SSMV_EINVAL, "out_bytes is NULL");
    *out_bytes = ((size_t)norm_parts(rows) * 3 * channels * sizeof(float) + 15) / 16 * 16;
    return SSMV_OK;
}

int ssmv_block_norm_backward(const ssmv_block_norm_grad_args *args, void *hip_stream)
{
    if (!args) return fail(SSMV_EINVAL, "args is NULL");
    ssmv_block_norm_grad_args a = *args;
    TRY(check_norm(a));
    TRY(check_layer_stride(&a.dr_stride, a.channels, "dr_stride"));
    TRY(check_layer_stride(&a.dn_stride, a.channels, "dn_stride"));
    TRY(check_layer_stride(&a.dx_stride, a.channels, "dx_stride"));
    TRY(check_layer_stride(&a.dz_stride, a.channels, "dz_stride"));
    TRY(check_layer_stride(&a.dres_stride, a.channels, "dres_stride"));
    TRY(check_io_opt(a.dr, a.res_dtype, "dr"));
    TRY(check_io_opt(a.dn, a.io_dtype, "dn"));
    if (!a.dr && !a.dn) return fail(SSMV_EINVAL, "dr and dn are both NULL");
    TRY(check_io_opt(a.dx, a.io_dtype, "dx"));
    TRY(check_io_opt(a.dz, a.io_dtype, "dz"));
    TRY(check_io_opt(a.dres, a.res_dtype, "dres"));
    TRY(check_f32_opt(a.dpost_wgt, "dpost_wgt"));
    TRY(check_f32_opt(a.dch_scale, "dch_scale"));
    TRY(check_f32_opt(a.dpre_wgt, "dpre_wgt"));
    TRY(check_no(a.dx, a.x, "dx"));
    TRY(check_no(a.dz, a.z, "dz"));
    TRY(check_no(a.dres, a.res, "dres"));
    TRY(check_no(a.dpost_wgt, a.post_wgt, "dpost_wgt"));
    TRY(check_no(a.dch_scale, a.ch_scale, "dch_scale"));
    TRY(check_no(a.dpre_wgt, a.pre_wgt, "dpre_wgt"));
    TRY(check_alias(a.dres, a.dres_stride, a.dr, a.dr_stride, "dres and dr"));
    TRY(check_alias(a.dx, a.dx_stride, a.dn, a.dn_stride, "dx and dn"));
    for (const void *out : {(const void *)a.dx, (const void *)a.dz, (const void *)a.dres})
        if (out && (out == a.x || out == a.z || out == a.res)) return fail(SSMV_EINVAL, "a gradient may not overwrite an input of the forward call");
    if ((a.dz && (a.dz == a.dr || a.dz == a.dn || a.dz == a.dx || a.dz == a.dres)) || (a.dx && (a.dx == a.dr || a.dx == a.dres)) || (a.dres && a.dres == a.dn))
        return fail(SSMV_EINVAL, "only dres may be dr, and dx dn");
    const bool vectors = a.dpost_wgt || a.dch_scale || a.dpre_wgt;
    if (vectors) TRY(check_ptr(a.workspace, "workspace"));
    BlockNormGradParams p{};
    p.x = a.x; p.z = a.z; p.res = a.res; p.post = a.post_wgt; p.scale = a.ch_scale; p.pre = a.pre_wgt; p.dr = a.dr; p.dn = a.dn;
    p.dx = a.dx; p.dz = a.dz; p.dres = a.dres; p.dpost = a.dpost_wgt; p.dscale = a.dch_scale; p.dpre = a.dpre_wgt;
    p.partial = vectors ? static_cast<float *>(a.workspace) : nullptr;
    p.x_stride = a.x_stride; p.z_stride = a.z_stride; p.res_stride = a.res_stride; p.dr_stride = a.dr_stride; p.dn_stride = a.dn_stride;
    p.dx_stride = a.dx_stride; p.dz_stride = a.dz_stride; p.dres_stride = a.dres_stride;
    p.rows = a.rows; p.C = a.channels; p.io = a.io_dtype; p.res_io = a.res_dtype; p.eps = a.eps; p.alpha = a.res_scale;
    const int hc = launch_block_norm_backward(p, (hipStream_t)hip_stream);
    return hc == 0 ? SSMV_OK : hip_fail(hc, "ssmv_block_norm_backward");
}

int ssm_gated_recurrence_workspace(int32_t batch, int32_t channels, int32_t L, size_t *out_bytes)
{
    TRY(check_gated_sizes(batch, channels, L));
    if (!out_bytes) return fail(SSMV_EINVAL, "out_bytes is NULL");
    *out_bytes = 0;                                                 // enough for either type
    for (int io : {SSMV_F32, SSMV_BF16}) {
        const size_t n = 2 * gated_segments(batch, channels, gated_plan(batch, channels, L, io, false));
        if (n > *out_bytes) *out_bytes = n;
    }
    return SSMV_OK;
}

int ssm_gated_recurrence(const ssmv_gated_args *args, void *hip_stream)
{
    if (!args) return fail(SSMV_EINVAL, "args is NULL");
    ssmv_gated_args a = *args;
    TRY(check_gated(a));
    TRY(check_layer_stride(&a.y_stride, a.channels, "y_stride"));
    TRY(check_rows(&a.rows_in, a.batch, a.src_row));
    TRY(check_io(a.y_out, a.io_dtype, "y_out"));
    TRY(check_f32_opt(a.h_in, "h_in"));
    TRY(check_f32_opt(a.h_out, "h_out"));
    TRY(check_f32_opt(a.states, "states"));
    if (a.src_row && a.h_out && a.h_out == a.h_in) return fail(SSMV_EINVAL, "h_out may be h_in only without src_row");
    if (a.y_out == a.x || a.y_out == a.f || a.y_out == a.i || a.y_out == a.z) return fail(SSMV_EINVAL, "y_out may not be an input");
    if (a.states && (a.states == a.h_in || a.states == a.h_out)) return fail(SSMV_EINVAL, "states may be neither h_in nor h_out");
    GatedParams p{};
    const GatedPlan plan = gated_plan(a.batch, a.channels, a.L, a.io_dtype, false);
    p.wide = plan.wide; p.seg_len = plan.seg_len; p.seg_count = plan.seg_count;
    if (const size_t each = gated_segments(a.batch, a.channels, plan)) {
        TRY(check_ptr(a.workspace, "workspace (these sequences are cut: ssm_gated_recurrence_workspace)"));
        p.seg_p = static_cast<float *>(a.workspace);
        p.seg_h = p.seg_p + each / sizeof(float);
    }
    p.x = a.x; p.f = a.f; p.i = a.i; p.z = a.z; p.A = a.A; p.f_bias = a.f_bias; p.i_bias = a.i_bias; p.h_in = a.h_in; p.src_row = a.src_row; p.seq_len = a.seq_len;
    p.y = a.y_out; p.h_out = a.h_out; p.states = a.states;
    p.x_stride = a.x_stride; p.f_stride = a.f_stride; p.i_stride = a.i_stride; p.z_stride = a.z_stride; p.y_stride = a.y_stride;
    p.batch = a.batch; p.rows_in = a.rows_in; p.C = a.channels; p.L = a.L; p.io = a.io_dtype; p.lru = a.form == SSMV_GATED_LRU;
    const int hc = launch_gated_recurrence(p, (hipStream_t)hip_stream);
    return hc == 0 ? SSMV_OK : hip_fail(hc, "ssm_gated_recurrence");
}

// the segments' pairs, then the sums of the vectors' gradients
static size_t gated_backward_layout(int batch, int channels, const GatedPlan &plan, size_t *sums_at)
{
    *sums_at = 2 * gated_segments(batch, channels, plan);
    return *sums_at + ((size_t)batch * plan.seg_count * 3 * channels * sizeof(float) + 15) / 16 * 16;
}

int ssm_gated_recurrence_backward_workspace(int32_t batch, int32_t channels, int32_t L, size_t *out_bytes)
{
    TRY(check_gated_sizes(batch, channels, L));
    if (!out_bytes) return fail(SSMV_EINVAL, "out_bytes is NULL");
    size_t at;
    *out_bytes = 0;
    for (int io : {SSMV_F32, SSMV_BF16}) {
        const size_t n = gated_backward_layout(batch, channels, gated_plan(batch, channels, L, io, true), &at);
        if (n > *out_bytes) *out_bytes = n;
    }
    return SSMV_OK;
}

int ssm_gated_recurrence_backward(const ssmv_gated_grad_args *args, void *hip_stream)
{
    if (!args) return fail(SSMV_EINVAL, "args is NULL");
    ssmv_gated_grad_args a = *args;
    TRY(check_gated(a));
    TRY(check_layer_stride(&a.dy_stride, a.channels, "dy_stride"));
    TRY(check_layer_stride(&a.dx_stride, a.channels, "dx_stride"));
    TRY(check_layer_stride(&a.df_stride, a.channels, "df_stride"));
    TRY(check_layer_stride(&a.di_stride, a.channels, "di_stride"));
    TRY(check_layer_stride(&a.dz_stride, a.channels, "dz_stride"));
    TRY(check_f32(a.states, "states"));
    TRY(check_io(a.dy, a.io_dtype, "dy"));
    TRY(check_f32_opt(a.dh_out, "dh_out"));
    TRY(check_io_opt(a.dx, a.io_dtype, "dx"));
    TRY(check_io_opt(a.df, a.io_dtype, "df"));
    TRY(check_io_opt(a.di, a.io_dtype, "di"));
    TRY(check_io_opt(a.dz, a.io_dtype, "dz"));
    TRY(check_f32_opt(a.dA, "dA"));
    TRY(check_f32_opt(a.df_bias, "df_bias"));
    TRY(check_f32_opt(a.di_bias, "di_bias"));
    TRY(check_f32_opt(a.dh_in, "dh_in"));
    TRY(check_no(a.di, a.i, "di"));
    TRY(check_no(a.dz, a.z, "dz"));
    TRY(check_no(a.dA, a.A, "dA"));
    TRY(check_no(a.df_bias, a.f_bias, "df_bias"));
    TRY(check_no(a.di_bias, a.i_bias, "di_bias"));
    for (const void *out : {(const void *)a.dx, (const void *)a.df, (const void *)a.di, (const void *)a.dz})
        if (out && (out == a.x || out == a.f || out == a.i || out == a.z || out == a.dy)) return fail(SSMV_EINVAL, "a gradient may not be an input");
    if ((a.dx && (a.dx == a.df || a.dx == a.di || a.dx == a.dz)) || (a.df && (a.df == a.di || a.df == a.dz)) || (a.di && a.di == a.dz))
        return fail(SSMV_EINVAL, "two gradients are one tensor");
    if (a.dh_in && (a.dh_in == a.dh_out || a.dh_in == a.states)) return fail(SSMV_EINVAL, "dh_in may be neither dh_out nor states");
    const GatedPlan plan = gated_plan(a.batch, a.channels, a.L, a.io_dtype, true);
    size_t sums_at;
    gated_backward_layout(a.batch, a.channels, plan, &sums_at);
    const bool vectors = a.dA || a.df_bias || a.di_bias;
    if (vectors || plan.seg_count > 1) TRY(check_ptr(a.workspace, "workspace"));
    GatedGradParams p{};
    p.wide = plan.wide; p.seg_len = plan.seg_len; p.seg_count = plan.seg_count;
    p.seg_p = static_cast<float *>(a.workspace);
    p.seg_r = p.seg_p + sums_at / 2 / sizeof(float);
    p.partial = vectors ? p.seg_p + sums_at / sizeof(float) : nullptr;
    p.x = a.x; p.f = a.f; p.i = a.i; p.z = a.z; p.dy = a.dy; p.A = a.A; p.f_bias = a.f_bias; p.i_bias = a.i_bias; p.states = a.states; p.dh_out = a.dh_out;
    p.seq_len = a.seq_len; p.dx = a.dx; p.df = a.df; p.di = a.di; p.dz = a.dz; p.dA = a.dA; p.df_bias = a.df_bias; p.di_bias = a.di_bias; p.dh_in = a.dh_in;
    p.x_stride = a.x_stride; p.f_stride = a.f_stride; p.i_stride = a.i_stride; p.z_stride = a.z_stride; p.dy_stride = a.dy_stride;
    p.dx_stride = a.dx_stride; p.df_stride = a.df_stride; p.di_stride = a.di_stride; p.dz_stride = a.dz_stride;
    p.batch = a.batch; p.C = a.channels; p.L = a.L; p.io = a.io_dtype; p.lru = a.form == SSMV_GATED_LRU;
    const int hc = launch_gated_backward(p, (hipStream_t)hip_stream);
    return hc == 0 ? SSMV_OK : hip_fail(hc, "ssm_gated_recurrence_backward");
}

int ssmv_logit_rules(const ssmv_rules_args *args, void *hip_stream)
{
    if (!args) return fail(SSMV_EINVAL, "args is NULL");
    ssmv_rules_args a = *args;
    TRY(check_io_type(a.io_dtype));
    if (a.rows < 1 || a.vocab < 1) return fail(SSMV_EINVAL, "rows %d and vocab %d must be >= 1", a.rows, a.vocab);
    if (a.rows > 65535) return fail(SSMV_EUNSUPPORTED, "rows %d > 65535", a.rows);
    if (a.vocab > 1 << 24) return fail(SSMV_EUNSUPPORTED, "vocab %d > 2^24", a.vocab);
    TRY(check_layer_stride(&a.row_stride, a.vocab, "row_stride"));
    TRY(check_layer_stride(&a.out_stride, a.vocab, "out_stride"));
    TRY(check_io(a.logits, a.io_dtype, "logits"));
    TRY(check_io(a.out, a.io_dtype, "out"));
    TRY(check_alias(a.out, a.out_stride, a.logits, a.row_stride, "out and logits"));
    if (a.hist) {
        TRY(check_f32(a.hist, "hist"));
        TRY(check_f32(a.hist_len, "hist_len"));
        TRY(check_rows(&a.rows_in, a.rows, a.src_row));
        if (a.hist_stride < 1) return fail(SSMV_EINVAL, "hist_stride %d < 1", a.hist_stride);
        if (a.hist_stride > SSMV_RULES_HISTORY_MAX) return fail(SSMV_EUNSUPPORTED, "hist_stride %d > %d", a.hist_stride, SSMV_RULES_HISTORY_MAX);
        TRY(check_f32_opt(a.token, "token"));
        TRY(check_f32_opt(a.prompt_len, "prompt_len"));
        TRY(check_f32_opt(a.repetition, "repetition"));
        TRY(check_f32_opt(a.frequency, "frequency"));
        TRY(check_f32_opt(a.presence, "presence"));
        if (!a.hist_out != !a.hist_len_out) return fail(SSMV_EINVAL, "hist_out and hist_len_out come together");
        TRY(check_f32_opt(a.hist_out, "hist_out"));
        TRY(check_f32_opt(a.hist_len_out, "hist_len_out"));
        if (a.hist_out && a.hist_out == a.hist && a.src_row) return fail(SSMV_EINVAL, "hist_out may be hist only without src_row");
        if (a.hist_len_out && a.hist_len_out == a.hist_len) return fail(SSMV_EINVAL, "hist_len_out may not be hist_len: other workgroups read it");
    } else if (a.hist_len || a.src_row || a.token || a.prompt_len || a.repetition || a.frequency || a.presence || a.hist_out || a.hist_len_out) {
        return fail(SSMV_EINVAL, "without hist there is nothing that its arguments and the penalties could mean");
    }
    if (a.bias_token) {
        if (a.bias_n < 1) return fail(SSMV_EINVAL, "bias_n %d < 1", a.bias_n);
        if (a.bias_n > SSMV_RULES_BIAS_MAX) return fail(SSMV_EUNSUPPORTED, "bias_n %d > %d", a.bias_n, SSMV_RULES_BIAS_MAX);
        TRY(check_f32(a.bias_token, "bias_token"));
        TRY(check_f32(a.bias, "bias"));
    } else if (a.bias) {
        return fail(SSMV_EINVAL, "bias without bias_token");
    }
    if (a.mask) {
        TRY(check_f32(a.mask, "mask"));
        TRY(check_f32_opt(a.mask_row, "mask_row"));
        if (a.mask_rows < 1) return fail(SSMV_EINVAL, "mask_rows %d < 1", a.mask_rows);
        if (!a.mask_row && a.mask_rows < a.rows) return fail(SSMV_EINVAL, "mask_rows %d < %d rows, and no mask_row", a.mask_rows, a.rows);
        TRY(check_layer_stride(&a.mask_stride, ((long)a.vocab + 31) / 32, "mask_stride"));
    } else if (a.mask_row) {
        return fail(SSMV_EINVAL, "mask_row without mask");
    }
    RulesParams p{};
    p.logits = a.logits; p.hist = a.hist; p.hist_len = a.hist_len; p.src_row = a.src_row; p.token = a.token; p.prompt_len = a.prompt_len;
    p.repetition = a.repetition; p.frequency = a.frequency; p.presence = a.presence; p.bias_token = a.bias_token; p.bias = a.bias;
    p.mask = a.mask; p.mask_row = a.mask_row; p.out = a.out; p.hist_out = a.hist_out; p.hist_len_out = a.hist_len_out;
    p.row_stride = a.row_stride; p.out_stride = a.out_stride; p.mask_stride = a.mask_stride;
    p.rows = a.rows; p.rows_in = a.rows_in; p.V = a.vocab; p.io = a.io_dtype; p.room = a.hist_stride; p.bias_n = a.bias_n; p.mask_rows = a.mask_rows;
    const int hc = launch_logit_rules(p, (hipStream_t)hip_stream);
    return hc == 0 ? SSMV_OK : hip_fail(hc, "ssmv_logit_rules");
}

}  // extern "C"
