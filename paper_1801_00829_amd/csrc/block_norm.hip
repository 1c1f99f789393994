// Norms around a block: checks, launch shapes and C entry points (kernels: block_norm.h).
#include "block_norm.h"

namespace fuse {
FUSE_NORM_TYPE(extern, double)
FUSE_NORM_TYPE(extern, float)
FUSE_NORM_TYPE(extern, __bf16)
FUSE_NORM_TYPE(extern, _Float16)
}  // namespace fuse

namespace {

using namespace fuse;

int each_of(const fuse_block *b) { return dtype_size(b->dtype) == 2 ? kEach<__bf16> : kEach<float>; }

// Steps per row, and threads per row: whole waves, as few as that takes.  Blocks of 512 threads leave a thread 256 registers, which hold
// a gradient call's sums and two rows of one step each; the longest rows take 1024.
int steps_for(const fuse_block *b)
{
    const int64_t one = 512 * each_of(b);
    return b->cols <= one ? 1 : b->cols <= 2 * one ? 2 : b->cols <= 4 * one && one == 2048 ? 4 : 32 / each_of(b);
}

int group_for(const fuse_block *b)
{
    const int64_t per = 64 * each_of(b) * steps_for(b);
    return (int)((b->cols + per - 1) / per) * 64;
}

// Threads per block: as many groups as 512 hold, at least one.
int threads_for(const fuse_block *b)
{
    const int g = group_for(b);
    return g >= 512 ? g : 512 / g * g;
}

int grad_blocks(const fuse_block *b)
{
    const int64_t per = threads_for(b) / group_for(b), want = (b->rows + per - 1) / per;
    return (int)(want < 1 ? 1 : want > kGradBlocks ? kGradBlocks : want);
}

#define FUSE_BY_DTYPE(dtype, call, ...)                                                                                    \
    do {                                                                                                                  \
        switch (dtype) {                                                                                                  \
        case FUSE_F64: call<double>(__VA_ARGS__); break;                                                                  \
        case FUSE_F32: call<float>(__VA_ARGS__); break;                                                                   \
        case FUSE_BF16: call<__bf16>(__VA_ARGS__); break;                                                                 \
        default: call<_Float16>(__VA_ARGS__); break;                                                                      \
        }                                                                                                                 \
    } while (0)

int check_block(const fuse_block *b)
{
    if (!b)
        return report(FUSE_EINVAL, "block is NULL");
    if (!known_dtype(b->dtype))
        return report(FUSE_EINVAL, "dtype is not a fuse_dtype");
    if (b->norm != FUSE_NORM_RMS && b->norm != FUSE_NORM_LAYER)
        return report(FUSE_EINVAL, "norm is not a fuse_norm_kind");
    if (b->rows < 0 || b->cols < 1)
        return report(FUSE_EINVAL, "rows must not be negative and cols must be positive");
    if (b->cols > kMaxCols)
        return report(FUSE_EUNSUPPORTED, "cols " + std::to_string(b->cols) + " > " + std::to_string(kMaxCols));
    if (b->rows > (INT64_C(1) << 40))
        return report(FUSE_EUNSUPPORTED, "rows " + std::to_string(b->rows) + " > 2^40");
    if (!(b->eps >= 0.0))
        return report(FUSE_EINVAL, "eps must not be negative");
    if (!b->z && (b->post_weight || b->gate_kind != FUSE_GATE_NONE))
        return report(FUSE_EINVAL, "a norm after the block and a gate need the block's result z");
    if (b->norm == FUSE_NORM_RMS && (b->post_bias || b->pre_bias))
        return report(FUSE_EINVAL, "a bias needs FUSE_NORM_LAYER");
    if ((b->post_bias && !b->post_weight) || (b->pre_bias && !b->pre_weight))
        return report(FUSE_EINVAL, "a bias needs its norm's weight");
    if (b->gate_kind != FUSE_GATE_NONE && b->gate_kind != FUSE_SIDE_ROWVEC && b->gate_kind != FUSE_SIDE_COLVEC &&
        b->gate_kind != FUSE_SIDE_MATRIX)
        return report(FUSE_EINVAL, "gate_kind is none of FUSE_GATE_NONE, FUSE_SIDE_ROWVEC, FUSE_SIDE_COLVEC, FUSE_SIDE_MATRIX");
    if (b->gate_kind != FUSE_GATE_NONE && !b->gate)
        return report(FUSE_EINVAL, "gate is NULL");
    return FUSE_OK;
}

int check_ld(const fuse_block *b, const void *p, int64_t ld, const char *what)
{
    return p && b->rows > 1 && ld < b->cols ? report(FUSE_ESHAPE, std::string(what) + ": leading dimension < cols") : FUSE_OK;
}

int gate_code(const fuse_block *b)
{
    return b->gate_kind == FUSE_GATE_NONE ? 0 : b->gate_kind == FUSE_SIDE_ROWVEC ? 1 : b->gate_kind == FUSE_SIDE_COLVEC ? 2 : 3;
}

// 16-byte loads: whole rows of vectors, every row of every matrix on 16 bytes.
bool rows_on_16(const fuse_block *b, const void *p, int64_t ld)
{
    return !p || (on_16_bytes(p) && (b->rows <= 1 || (ld * (int64_t)dtype_size(b->dtype)) % 16 == 0));
}

bool block_on_16(const fuse_block *b)
{
    return b->cols % 8 == 0 && rows_on_16(b, b->z, b->z_ld) && on_16_bytes(b->post_weight) && on_16_bytes(b->post_bias) &&
           on_16_bytes(b->pre_weight) && on_16_bytes(b->pre_bias) &&
           (b->gate_kind == FUSE_GATE_NONE || b->gate_kind == FUSE_SIDE_COLVEC ||
            (b->gate_kind == FUSE_SIDE_ROWVEC ? on_16_bytes(b->gate) : rows_on_16(b, b->gate, b->gate_ld)));
}

int check_gate_ld(const fuse_block *b)
{
    if (b->gate_kind == FUSE_SIDE_MATRIX)
        return check_ld(b, b->gate, b->gate_ld, "gate");
    if (b->gate_kind == FUSE_SIDE_COLVEC && b->rows > 1 && b->gate_ld < 1)
        return report(FUSE_ESHAPE, "gate: stride < 1");
    return FUSE_OK;
}

int norm_impl(const fuse_block *b, const void *x, int64_t x_ld, void *h, int64_t h_ld, void *y, int64_t y_ld, void *stream)
{
    report(FUSE_OK, "");
    int rc = check_block(b);
    if (rc)
        return rc;
    if (b->pre_weight ? !y : y != nullptr)
        return report(FUSE_EINVAL, "y goes with pre_weight: both or neither");
    if (!b->z && h)
        return report(FUSE_EINVAL, "h needs the block's result z: without one it is x");
    if (!h && !y)
        return report(FUSE_EINVAL, "neither h nor y is asked for");
    if (!x && b->rows > 0)
        return report(FUSE_EINVAL, "x is NULL");
    if ((rc = check_ld(b, x, x_ld, "x")) || (rc = check_ld(b, b->z, b->z_ld, "z")) || (rc = check_ld(b, h, h_ld, "h")) ||
        (rc = check_ld(b, y, y_ld, "y")) || (rc = check_gate_ld(b)))
        return rc;
    if (b->rows == 0)
        return FUSE_OK;
    FwdArgs a;
    a.x = x, a.z = b->z, a.post_w = b->post_weight, a.post_b = b->post_bias, a.pre_w = b->pre_weight, a.pre_b = b->pre_bias;
    a.h = h, a.y = y;
    a.x_ld = x_ld, a.z_ld = b->z_ld, a.h_ld = h_ld, a.y_ld = y_ld, a.rows = b->rows;
    a.cols = (int)b->cols, a.group = group_for(b);
    a.gate = {gate_code(b), b->gate, b->gate_ld};
    a.eps = b->eps, a.scale = b->scale;
    const bool vec = block_on_16(b) && rows_on_16(b, x, x_ld) && rows_on_16(b, h, h_ld) && rows_on_16(b, y, y_ld);
    const int threads = threads_for(b), per = threads / a.group;
    const int64_t want = (b->rows + per - 1) / per;
    const unsigned blocks = (unsigned)(want > 65536 ? 65536 : want);
    FUSE_BY_DTYPE(b->dtype, launch_fwd, a, b->norm == FUSE_NORM_LAYER, steps_for(b), vec, blocks, threads, (hipStream_t)stream);
    return launched("block_norm_kernel");
}

size_t grad_bytes(const fuse_block *b)
{
    return (size_t)5 * grad_blocks(b) * b->cols * (b->dtype == FUSE_F64 ? 8 : 4);
}

int norm_grad_impl(const fuse_block *b, const void *dh, int64_t dh_ld, const void *dy, int64_t dy_ld, const void *h, int64_t h_ld,
                   const fuse_block_grads *g, void *workspace, size_t workspace_bytes, void *stream)
{
    report(FUSE_OK, "");
    int rc = check_block(b);
    if (rc)
        return rc;
    if (!g)
        return report(FUSE_EINVAL, "grads is NULL");
    if (!dh && !dy)
        return report(FUSE_EINVAL, "neither dh nor dy is given");
    if (dy && !b->pre_weight)
        return report(FUSE_EINVAL, "dy needs the norm that made y: pre_weight is NULL");
    if (dy && !h && b->rows > 0)
        return report(FUSE_EINVAL, "h is NULL");
    if (!b->z && g->dz)
        return report(FUSE_EINVAL, "dz needs z");
    if ((g->dgate && b->gate_kind == FUSE_GATE_NONE) || (g->dpost_weight && !b->post_weight) || (g->dpre_weight && !b->pre_weight) ||
        (g->dpost_bias && !b->post_bias) || (g->dpre_bias && !b->pre_bias))
        return report(FUSE_EINVAL, "a gradient is asked for whose input is not given");
    if ((rc = check_ld(b, dh, dh_ld, "dh")) || (rc = check_ld(b, dy, dy_ld, "dy")) || (rc = check_ld(b, h, h_ld, "h")) ||
        (rc = check_ld(b, b->z, b->z_ld, "z")) || (rc = check_ld(b, g->dx, g->dx_ld, "dx")) || (rc = check_ld(b, g->dz, g->dz_ld, "dz")) ||
        (rc = check_gate_ld(b)) ||
        (rc = b->gate_kind == FUSE_SIDE_MATRIX ? check_ld(b, g->dgate, g->dgate_ld, "dgate") : FUSE_OK))
        return rc;
    if (b->gate_kind == FUSE_SIDE_COLVEC && g->dgate && b->rows > 1 && g->dgate_ld < 1)
        return report(FUSE_ESHAPE, "dgate: stride < 1");
    if (!workspace || !on_16_bytes(workspace) || workspace_bytes < grad_bytes(b))
        return report(FUSE_EINVAL, "workspace: " + std::to_string(grad_bytes(b)) + " bytes on 16 are needed");
    BwdArgs a;
    a.dh = dh, a.dy = dy, a.h = h, a.z = b->z, a.post_w = b->post_weight, a.post_b = b->post_bias, a.pre_w = b->pre_weight;
    a.dx = g->dx, a.dz = g->dz, a.dgate = g->dgate, a.partial = workspace;
    a.dh_ld = dh_ld, a.dy_ld = dy_ld, a.h_ld = h_ld, a.z_ld = b->z_ld, a.dx_ld = g->dx_ld, a.dz_ld = g->dz_ld, a.dgate_ld = g->dgate_ld;
    a.rows = b->rows, a.cols = (int)b->cols, a.group = group_for(b);
    a.gate = {gate_code(b), b->gate, b->gate_ld};
    a.eps = b->eps, a.scale = b->scale;
    // (without dy or rows the sums are those of nothing: zeros)
    a.want_dpre_w = g->dpre_weight != nullptr, a.want_dpre_b = g->dpre_bias != nullptr;
    a.want_dpost_w = g->dpost_weight != nullptr, a.want_dpost_b = g->dpost_bias != nullptr;
    const bool vec = block_on_16(b) && rows_on_16(b, dh, dh_ld) && rows_on_16(b, dy, dy_ld) && rows_on_16(b, h, h_ld) &&
                     rows_on_16(b, g->dx, g->dx_ld) && rows_on_16(b, g->dz, g->dz_ld) &&
                     (b->gate_kind != FUSE_SIDE_MATRIX || rows_on_16(b, g->dgate, g->dgate_ld));
    const int blocks = grad_blocks(b);
    FUSE_BY_DTYPE(b->dtype, launch_bwd, a, b->norm == FUSE_NORM_LAYER, steps_for(b), vec, blocks, threads_for(b), (hipStream_t)stream);
    rc = launched("block_norm_grad_kernel");
    SumArgs sa;
    sa.partial = workspace, sa.blocks = blocks, sa.cols = (int)b->cols;
    sa.out[0] = g->dpre_weight, sa.out[1] = g->dpost_weight;
    sa.out[2] = b->gate_kind == FUSE_SIDE_ROWVEC ? g->dgate : nullptr;
    sa.out[3] = g->dpre_bias, sa.out[4] = g->dpost_bias;
    if (rc || (!sa.out[0] && !sa.out[1] && !sa.out[2] && !sa.out[3] && !sa.out[4]))
        return rc;
    FUSE_BY_DTYPE(b->dtype, launch_sums, sa, (hipStream_t)stream);
    rc = launched("block_norm_sums_kernel");
    if (!rc)
        set_last_kernel("block_norm_grad_kernel");
    return rc;
}

}  // namespace

extern "C" {

int fuse_block_norm(const fuse_block *block, const void *x, int64_t x_ld, void *h, int64_t h_ld, void *y, int64_t y_ld, void *stream)
{
    return fuse::guard([&] { return norm_impl(block, x, x_ld, h, h_ld, y, y_ld, stream); });
}

size_t fuse_block_norm_backward_bytes(const fuse_block *block)
{
    if (!block || !known_dtype(block->dtype) || block->rows < 0 || block->cols < 1 || block->cols > kMaxCols)
        return 0;
    return grad_bytes(block);
}

int fuse_block_norm_backward(const fuse_block *block, const void *dh, int64_t dh_ld, const void *dy, int64_t dy_ld, const void *h,
                             int64_t h_ld, const fuse_block_grads *grads, void *workspace, size_t workspace_bytes, void *stream)
{
    return fuse::guard([&] { return norm_grad_impl(block, dh, dh_ld, dy, dy_ld, h, h_ld, grads, workspace, workspace_bytes, stream); });
}

}  // extern "C"
