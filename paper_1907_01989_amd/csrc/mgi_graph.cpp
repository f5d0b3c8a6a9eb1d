// Graph building, validation and error reporting of the C ABI.
//
// Each add call checks its operands the way the paper's delegate checks that
// an operator is supported before taking it over (Sec. 3.1); there is no CPU
// fallback, an unsupported operator is reported as MGI_ERR_UNSUPPORTED.
#include <climits>
#include <cmath>
#include <cstdio>
#include <cstring>
#include <new>

#include "mgi_internal.h"

namespace mgi {

static thread_local std::string g_last_error;

mgi_status fail(mgi_status s, const std::string &msg) {
    g_last_error = msg;
    return s;
}

}  // namespace mgi

using namespace mgi;

extern "C" const char *mgi_status_str(int s) {
    switch (s) {
        case MGI_OK: return "MGI_OK";
        case MGI_ERR_INVALID_ARG: return "MGI_ERR_INVALID_ARG";
        case MGI_ERR_SHAPE: return "MGI_ERR_SHAPE";
        case MGI_ERR_UNSUPPORTED: return "MGI_ERR_UNSUPPORTED";
        case MGI_ERR_STATE: return "MGI_ERR_STATE";
        case MGI_ERR_WORKSPACE: return "MGI_ERR_WORKSPACE";
        case MGI_ERR_HIP: return "MGI_ERR_HIP";
        case MGI_ERR_OOM_HOST: return "MGI_ERR_OOM_HOST";
        case MGI_ERR_INTERNAL: return "MGI_ERR_INTERNAL";
    }
    return "MGI_ERR_UNKNOWN";
}

extern "C" const char *mgi_last_error(void) { return g_last_error.c_str(); }

extern "C" mgi_status mgi_graph_create(mgi_graph **g) {
    MGI_ABI_TRY
    if (!g) return fail(MGI_ERR_INVALID_ARG, "mgi_graph_create: null out pointer");
    *g = new (std::nothrow) mgi_graph();
    if (!*g) return fail(MGI_ERR_OOM_HOST, "mgi_graph_create: out of host memory");
    return MGI_OK;
    MGI_ABI_CATCH("mgi_graph_create")
}

extern "C" mgi_status mgi_graph_destroy(mgi_graph *g) {
    MGI_ABI_TRY
    delete g;
    return MGI_OK;
    MGI_ABI_CATCH("mgi_graph_destroy")
}

namespace {

bool valid_act(int a) { return a == MGI_ACT_NONE || a == MGI_ACT_RELU || a == MGI_ACT_RELU6; }

mgi_status check_tensor(const mgi_graph *g, int id, const char *who) {
    if (!g) return fail(MGI_ERR_INVALID_ARG, std::string(who) + ": null graph");
    if (id < 0 || id >= (int)g->ops.size())
        return fail(MGI_ERR_INVALID_ARG, std::string(who) + ": tensor id " + std::to_string(id) +
                                             " does not exist");
    return MGI_OK;
}

bool is_index(const GOp &op) {
    return op.kind == OpKind::TopK || op.kind == OpKind::Argmax ||
           (op.kind == OpKind::Input && op.in_dtype == MGI_DTYPE_INT32);
}

// an 8-bit tensor: only the 8-bit layer reads one
bool is_8bit(const GOp &op) { return op.kind == OpKind::Quantize || (op.kind == OpKind::RmsNorm && op.to8); }

// an operand that holds values: not the indices of topk or of an index input
mgi_status check_values(const mgi_graph *g, int id, const char *who) {
    const mgi_status s = check_tensor(g, id, who);
    if (s) return s;
    if (is_8bit(g->ops[id]))
        return fail(MGI_ERR_UNSUPPORTED, std::string(who) + ": tensor " + std::to_string(id) + " is held in 8 bits");
    if (is_index(g->ops[id]) && g->ops[id].kind != OpKind::Argmax)   // (argmax: finalize says so)
        return fail(MGI_ERR_UNSUPPORTED, std::string(who) + ": tensor " + std::to_string(id) + " holds indices");
    return MGI_OK;
}

// the operand of topk, log_prob and entropy
mgi_status check_rows(const mgi_graph *g, int id, const char *who) {
    const mgi_status s = check_values(g, id, who);
    if (s) return s;
    if (g->ops[id].kind == OpKind::Argmax)
        return fail(MGI_ERR_UNSUPPORTED, std::string(who) + ": tensor " + std::to_string(id) + " holds indices");
    const Shape x = g->ops[id].out;
    if (x.c > kern::kMaxAnswerCols || x.pixels() > (size_t)INT_MAX / 8)
        return fail(MGI_ERR_UNSUPPORTED, std::string(who) + ": at most 2^19 channels and 2^28 - 1 pixels");
    return MGI_OK;
}

// the operand of an attention block's operator, whose kernels count 16-byte
// elements in an int
mgi_status check_tokens(const mgi_graph *g, int id, const char *who) {
    const mgi_status s = check_values(g, id, who);
    if (s) return s;
    if (is_index(g->ops[id]))
        return fail(MGI_ERR_UNSUPPORTED, std::string(who) + ": tensor " + std::to_string(id) + " holds indices");
    return MGI_OK;
}

// ... and whether a tensor of that shape can be counted so
bool countable(const Shape &x) {
    const unsigned __int128 e = (unsigned __int128)x.n * x.h * x.w;
    return e <= INT_MAX && e * (((size_t)x.c + 127) / 128 * 16) <= INT_MAX;
}

mgi_status push(mgi_graph *g, GOp &&op, int *out) {
    try {
        g->ops.push_back(std::move(op));
    } catch (const std::bad_alloc &) {
        return fail(MGI_ERR_OOM_HOST, "out of host memory");
    }
    *out = (int)g->ops.size() - 1;
    return MGI_OK;
}

// Validates window attributes shared by conv2d and depthwise and computes the
// output size.
mgi_status conv_geometry(const Shape &x, const mgi_conv_desc *d, const char *who, int *oh, int *ow) {
    if (!d) return fail(MGI_ERR_INVALID_ARG, std::string(who) + ": null descriptor");
    if (d->kh <= 0 || d->kw <= 0 || d->stride_h <= 0 || d->stride_w <= 0 || d->dil_h <= 0 ||
        d->dil_w <= 0 || d->pad_t < 0 || d->pad_b < 0 || d->pad_l < 0 || d->pad_r < 0)
        return fail(MGI_ERR_INVALID_ARG, std::string(who) + ": window, stride and dilation must "
                                                            "be positive and pads non-negative");
    if (!valid_act(d->act)) return fail(MGI_ERR_INVALID_ARG, std::string(who) + ": bad activation");
    long eh = (long)x.h + d->pad_t + d->pad_b - (long)d->dil_h * (d->kh - 1) - 1;
    long ew = (long)x.w + d->pad_l + d->pad_r - (long)d->dil_w * (d->kw - 1) - 1;
    if (eh < 0 || ew < 0)
        return fail(MGI_ERR_SHAPE, std::string(who) + ": window larger than the padded input");
    *oh = (int)(eh / d->stride_h + 1);
    *ow = (int)(ew / d->stride_w + 1);
    return MGI_OK;
}

}  // namespace

extern "C" mgi_status mgi_graph_add_input(mgi_graph *g, int n, int h, int w, int c, int dtype,
                                          int *out) {
    MGI_ABI_TRY
    if (!g || !out) return fail(MGI_ERR_INVALID_ARG, "mgi_graph_add_input: null pointer");
    if (n <= 0 || h <= 0 || w <= 0 || c <= 0)
        return fail(MGI_ERR_INVALID_ARG, "mgi_graph_add_input: sizes must be positive");
    if (dtype != MGI_DTYPE_FP32 && dtype != MGI_DTYPE_FP16 && dtype != MGI_DTYPE_BF16)
        return fail(MGI_ERR_UNSUPPORTED, "mgi_graph_add_input: inputs are fp32, fp16 or bf16");
    GOp op;
    op.kind = OpKind::Input;
    op.out = {n, h, w, c};
    op.in_dtype = dtype;
    mgi_status s = push(g, std::move(op), out);
    if (s == MGI_OK) g->inputs.push_back(*out);
    return s;
    MGI_ABI_CATCH("mgi_graph_add_input")
}

extern "C" mgi_status mgi_graph_add_conv2d(mgi_graph *g, int in, const mgi_conv_desc *d,
                                           const float *w, const float *bias, int *out) {
    MGI_ABI_TRY
    mgi_status s = check_values(g, in, "mgi_graph_add_conv2d");
    if (s) return s;
    if (!out || !w) return fail(MGI_ERR_INVALID_ARG, "mgi_graph_add_conv2d: null pointer");
    const Shape x = g->ops[in].out;
    int oh, ow;
    if ((s = conv_geometry(x, d, "mgi_graph_add_conv2d", &oh, &ow))) return s;
    if (d->cout <= 0) return fail(MGI_ERR_INVALID_ARG, "mgi_graph_add_conv2d: cout must be positive");
    GOp op;
    op.kind = OpKind::Conv2d;
    op.in = {in};
    op.conv = *d;
    op.act = d->act;
    op.out = {x.n, oh, ow, d->cout};
    size_t wn = (size_t)d->cout * d->kh * d->kw * x.c;
    try {
        op.w.assign(w, w + wn);
        if (bias) op.b.assign(bias, bias + d->cout); else op.b.assign(d->cout, 0.0f);
    } catch (const std::bad_alloc &) {
        return fail(MGI_ERR_OOM_HOST, "mgi_graph_add_conv2d: out of host memory");
    }
    return push(g, std::move(op), out);
    MGI_ABI_CATCH("mgi_graph_add_conv2d")
}

extern "C" mgi_status mgi_graph_add_depthwise(mgi_graph *g, int in, const mgi_conv_desc *d,
                                              const float *w, const float *bias, int *out) {
    MGI_ABI_TRY
    mgi_status s = check_values(g, in, "mgi_graph_add_depthwise");
    if (s) return s;
    if (!out || !w) return fail(MGI_ERR_INVALID_ARG, "mgi_graph_add_depthwise: null pointer");
    const Shape x = g->ops[in].out;
    int oh, ow;
    if ((s = conv_geometry(x, d, "mgi_graph_add_depthwise", &oh, &ow))) return s;
    GOp op;
    op.kind = OpKind::Depthwise;
    op.in = {in};
    op.conv = *d;
    op.conv.cout = x.c;
    op.act = d->act;
    op.out = {x.n, oh, ow, x.c};
    size_t wn = (size_t)x.c * d->kh * d->kw;
    try {
        op.w.assign(w, w + wn);
        if (bias) op.b.assign(bias, bias + x.c); else op.b.assign(x.c, 0.0f);
    } catch (const std::bad_alloc &) {
        return fail(MGI_ERR_OOM_HOST, "mgi_graph_add_depthwise: out of host memory");
    }
    return push(g, std::move(op), out);
    MGI_ABI_CATCH("mgi_graph_add_depthwise")
}

static bool same_shape(const Shape &a, const Shape &b) {
    return a.n == b.n && a.h == b.h && a.w == b.w && a.c == b.c;
}

extern "C" mgi_status mgi_graph_add_add(mgi_graph *g, int a, int b, int act, int *out) {
    MGI_ABI_TRY
    mgi_status s;
    if ((s = check_values(g, a, "mgi_graph_add_add")) || (s = check_values(g, b, "mgi_graph_add_add")))
        return s;
    if (!out) return fail(MGI_ERR_INVALID_ARG, "mgi_graph_add_add: null pointer");
    if (!valid_act(act)) return fail(MGI_ERR_INVALID_ARG, "mgi_graph_add_add: bad activation");
    if (!same_shape(g->ops[a].out, g->ops[b].out))
        return fail(MGI_ERR_SHAPE, "mgi_graph_add_add: operand shapes differ");
    GOp op;
    op.kind = OpKind::Add;
    op.in = {a, b};
    op.act = act;
    op.out = g->ops[a].out;
    return push(g, std::move(op), out);
    MGI_ABI_CATCH("mgi_graph_add_add")
}

extern "C" mgi_status mgi_graph_add_activation(mgi_graph *g, int in, int act, int *out) {
    MGI_ABI_TRY
    mgi_status s = check_values(g, in, "mgi_graph_add_activation");
    if (s) return s;
    if (!out) return fail(MGI_ERR_INVALID_ARG, "mgi_graph_add_activation: null pointer");
    if (!valid_act(act)) return fail(MGI_ERR_INVALID_ARG, "mgi_graph_add_activation: bad activation");
    GOp op;
    op.kind = OpKind::Activation;
    op.in = {in};
    op.act = act;
    op.out = g->ops[in].out;
    return push(g, std::move(op), out);
    MGI_ABI_CATCH("mgi_graph_add_activation")
}

extern "C" mgi_status mgi_graph_add_pad(mgi_graph *g, int in, int pad_t, int pad_b, int pad_l,
                                        int pad_r, int *out) {
    MGI_ABI_TRY
    mgi_status s = check_values(g, in, "mgi_graph_add_pad");
    if (s) return s;
    if (!out) return fail(MGI_ERR_INVALID_ARG, "mgi_graph_add_pad: null pointer");
    if (pad_t < 0 || pad_b < 0 || pad_l < 0 || pad_r < 0)
        return fail(MGI_ERR_INVALID_ARG, "mgi_graph_add_pad: pads must be non-negative");
    GOp op;
    op.kind = OpKind::Pad;
    op.in = {in};
    op.pads[0] = pad_t;
    op.pads[1] = pad_b;
    op.pads[2] = pad_l;
    op.pads[3] = pad_r;
    op.out = g->ops[in].out;
    op.out.h += pad_t + pad_b;
    op.out.w += pad_l + pad_r;
    return push(g, std::move(op), out);
    MGI_ABI_CATCH("mgi_graph_add_pad")
}

extern "C" mgi_status mgi_graph_add_global_avgpool(mgi_graph *g, int in, int *out) {
    MGI_ABI_TRY
    mgi_status s = check_values(g, in, "mgi_graph_add_global_avgpool");
    if (s) return s;
    if (!out) return fail(MGI_ERR_INVALID_ARG, "mgi_graph_add_global_avgpool: null pointer");
    GOp op;
    op.kind = OpKind::GlobalAvgPool;
    op.in = {in};
    const Shape x = g->ops[in].out;
    op.out = {x.n, 1, 1, x.c};
    return push(g, std::move(op), out);
    MGI_ABI_CATCH("mgi_graph_add_global_avgpool")
}

extern "C" mgi_status mgi_graph_add_fc(mgi_graph *g, int in, int cout, const float *w,
                                       const float *bias, int *out) {
    MGI_ABI_TRY
    mgi_status s = check_values(g, in, "mgi_graph_add_fc");
    if (s) return s;
    if (!out || !w) return fail(MGI_ERR_INVALID_ARG, "mgi_graph_add_fc: null pointer");
    if (cout <= 0) return fail(MGI_ERR_INVALID_ARG, "mgi_graph_add_fc: cout must be positive");
    const Shape x = g->ops[in].out;
    if (x.h != 1 || x.w != 1)
        return fail(MGI_ERR_UNSUPPORTED, "mgi_graph_add_fc: input must be 1x1 spatially");
    GOp op;
    op.kind = OpKind::FC;
    op.in = {in};
    op.cout = cout;
    op.out = {x.n, 1, 1, cout};
    try {
        op.w.assign(w, w + (size_t)cout * x.c);
        if (bias) op.b.assign(bias, bias + cout); else op.b.assign(cout, 0.0f);
    } catch (const std::bad_alloc &) {
        return fail(MGI_ERR_OOM_HOST, "mgi_graph_add_fc: out of host memory");
    }
    return push(g, std::move(op), out);
    MGI_ABI_CATCH("mgi_graph_add_fc")
}

extern "C" mgi_status mgi_graph_add_softmax(mgi_graph *g, int in, int *out) {
    MGI_ABI_TRY
    mgi_status s = check_values(g, in, "mgi_graph_add_softmax");
    if (s) return s;
    if (!out) return fail(MGI_ERR_INVALID_ARG, "mgi_graph_add_softmax: null pointer");
    GOp op;
    op.kind = OpKind::Softmax;
    op.in = {in};
    op.out = g->ops[in].out;
    return push(g, std::move(op), out);
    MGI_ABI_CATCH("mgi_graph_add_softmax")
}

extern "C" mgi_status mgi_graph_add_concat(mgi_graph *g, const int *ins, int count, int *out) {
    MGI_ABI_TRY
    if (!g || !ins || !out) return fail(MGI_ERR_INVALID_ARG, "mgi_graph_add_concat: null pointer");
    if (count < 1 || count > 8)
        return fail(count < 1 ? MGI_ERR_INVALID_ARG : MGI_ERR_UNSUPPORTED,
                    "mgi_graph_add_concat: 1 to 8 inputs");
    Shape o{};
    for (int i = 0; i < count; ++i) {
        mgi_status s = check_values(g, ins[i], "mgi_graph_add_concat");
        if (s) return s;
        const Shape x = g->ops[ins[i]].out;
        if (i == 0) o = x, o.c = 0;
        if (x.n != o.n || x.h != o.h || x.w != o.w)
            return fail(MGI_ERR_SHAPE, "mgi_graph_add_concat: inputs differ in n, h or w");
        o.c += x.c;
    }
    GOp op;
    op.kind = OpKind::Concat;
    op.in.assign(ins, ins + count);
    op.out = o;
    return push(g, std::move(op), out);
    MGI_ABI_CATCH("mgi_graph_add_concat")
}

extern "C" mgi_status mgi_graph_add_resize_bilinear(mgi_graph *g, int in, int oh, int ow,
                                                    int align_corners, int *out) {
    MGI_ABI_TRY
    mgi_status s = check_values(g, in, "mgi_graph_add_resize_bilinear");
    if (s) return s;
    if (!out) return fail(MGI_ERR_INVALID_ARG, "mgi_graph_add_resize_bilinear: null pointer");
    if (oh <= 0 || ow <= 0)
        return fail(MGI_ERR_INVALID_ARG, "mgi_graph_add_resize_bilinear: sizes must be positive");
    GOp op;
    op.kind = OpKind::ResizeBilinear;
    op.in = {in};
    op.oh = oh;
    op.ow = ow;
    op.align_corners = align_corners ? 1 : 0;
    const Shape x = g->ops[in].out;
    op.out = {x.n, oh, ow, x.c};
    return push(g, std::move(op), out);
    MGI_ABI_CATCH("mgi_graph_add_resize_bilinear")
}

extern "C" mgi_status mgi_graph_add_argmax(mgi_graph *g, int in, int *out) {
    MGI_ABI_TRY
    mgi_status s = check_values(g, in, "mgi_graph_add_argmax");
    if (s) return s;
    if (!out) return fail(MGI_ERR_INVALID_ARG, "mgi_graph_add_argmax: null pointer");
    GOp op;
    op.kind = OpKind::Argmax;
    op.in = {in};
    const Shape x = g->ops[in].out;
    op.out = {x.n, x.h, x.w, 1};
    return push(g, std::move(op), out);
    MGI_ABI_CATCH("mgi_graph_add_argmax")
}

extern "C" mgi_status mgi_graph_add_fc_int4(mgi_graph *g, int in, int cout, int group,
                                            const unsigned char *codes, const float *scales,
                                            const unsigned char *zeros, const float *bias, int *out) {
    MGI_ABI_TRY
    const char *who = "mgi_graph_add_fc_int4";
    mgi_status s = check_values(g, in, who);
    if (s) return s;
    if (!out || !codes || !scales) return fail(MGI_ERR_INVALID_ARG, std::string(who) + ": null pointer");
    if (cout <= 0) return fail(MGI_ERR_INVALID_ARG, std::string(who) + ": cout must be positive");
    if (group <= 0) return fail(MGI_ERR_INVALID_ARG, std::string(who) + ": group must be positive");
    if (group % 32 != 0) return fail(MGI_ERR_UNSUPPORTED, std::string(who) + ": group must be a multiple of 32");
    const Shape x = g->ops[in].out;
    if (x.h != 1 || x.w != 1)
        return fail(MGI_ERR_UNSUPPORTED, std::string(who) + ": input must be 1x1 spatially");
    if (x.n > kern::kMaxFcInt4Rows)
        return fail(MGI_ERR_UNSUPPORTED, std::string(who) + ": at most " + std::to_string(kern::kMaxFcInt4Rows) + " images");
    const size_t groups = ((size_t)x.c + group - 1) / group, n = (size_t)cout * groups;
    for (size_t i = 0; i < n; ++i)
        if (!std::isfinite(scales[i])) return fail(MGI_ERR_INVALID_ARG, std::string(who) + ": scales must be finite");
    for (size_t i = 0; zeros && i < n; ++i)
        if (zeros[i] > 15) return fail(MGI_ERR_INVALID_ARG, std::string(who) + ": zero points are 0..15");
    GOp op;
    op.kind = OpKind::FcInt4;
    op.in = {in};
    op.cout = cout;
    op.group = group;
    op.out = {x.n, 1, 1, cout};
    try {
        op.codes.assign(codes, codes + (size_t)cout * ((x.c + 1) / 2));
        op.w.assign(scales, scales + n);
        if (zeros) op.zeros.assign(zeros, zeros + n);
        if (bias) op.b.assign(bias, bias + cout); else op.b.assign(cout, 0.0f);
    } catch (const std::bad_alloc &) {
        return fail(MGI_ERR_OOM_HOST, std::string(who) + ": out of host memory");
    }
    return push(g, std::move(op), out);
    MGI_ABI_CATCH("mgi_graph_add_fc_int4")
}

extern "C" mgi_status mgi_graph_add_index_input(mgi_graph *g, int n, int h, int w, int c, int *out) {
    MGI_ABI_TRY
    if (!g || !out) return fail(MGI_ERR_INVALID_ARG, "mgi_graph_add_index_input: null pointer");
    if (n <= 0 || h <= 0 || w <= 0 || c <= 0)
        return fail(MGI_ERR_INVALID_ARG, "mgi_graph_add_index_input: sizes must be positive");
    GOp op;
    op.kind = OpKind::Input;
    op.out = {n, h, w, c};
    op.in_dtype = MGI_DTYPE_INT32;
    mgi_status s = push(g, std::move(op), out);
    if (s == MGI_OK) g->inputs.push_back(*out);
    return s;
    MGI_ABI_CATCH("mgi_graph_add_index_input")
}

extern "C" mgi_status mgi_graph_add_topk(mgi_graph *g, int in, int k, int *out) {
    MGI_ABI_TRY
    mgi_status s = check_rows(g, in, "mgi_graph_add_topk");
    if (s) return s;
    if (!out) return fail(MGI_ERR_INVALID_ARG, "mgi_graph_add_topk: null pointer");
    if (k <= 0) return fail(MGI_ERR_INVALID_ARG, "mgi_graph_add_topk: k must be positive");
    const Shape x = g->ops[in].out;
    if (k > x.c) return fail(MGI_ERR_SHAPE, "mgi_graph_add_topk: k exceeds the channels");
    if (k > kern::kMaxTopK)
        return fail(MGI_ERR_UNSUPPORTED, "mgi_graph_add_topk: k is at most " + std::to_string(kern::kMaxTopK));
    GOp op;
    op.kind = OpKind::TopK;
    op.in = {in};
    op.k = k;
    op.out = {x.n, x.h, x.w, k};
    return push(g, std::move(op), out);
    MGI_ABI_CATCH("mgi_graph_add_topk")
}

extern "C" mgi_status mgi_graph_add_log_prob(mgi_graph *g, int in, int index, int *out) {
    MGI_ABI_TRY
    mgi_status s = check_rows(g, in, "mgi_graph_add_log_prob");
    if (s || (s = check_tensor(g, index, "mgi_graph_add_log_prob"))) return s;
    if (!out) return fail(MGI_ERR_INVALID_ARG, "mgi_graph_add_log_prob: null pointer");
    const GOp &ix = g->ops[index];
    if (!is_index(ix))
        return fail(MGI_ERR_INVALID_ARG, "mgi_graph_add_log_prob: index is an index input or the output of topk or argmax");
    const Shape x = g->ops[in].out;
    if (ix.out.n != x.n || ix.out.h != x.h || ix.out.w != x.w)
        return fail(MGI_ERR_SHAPE, "mgi_graph_add_log_prob: index differs in n, h or w");
    GOp op;
    op.kind = OpKind::LogProb;
    op.in = {in, index};
    op.out = ix.out;
    return push(g, std::move(op), out);
    MGI_ABI_CATCH("mgi_graph_add_log_prob")
}

extern "C" mgi_status mgi_graph_add_entropy(mgi_graph *g, int in, int *out) {
    MGI_ABI_TRY
    mgi_status s = check_rows(g, in, "mgi_graph_add_entropy");
    if (s) return s;
    if (!out) return fail(MGI_ERR_INVALID_ARG, "mgi_graph_add_entropy: null pointer");
    GOp op;
    op.kind = OpKind::Entropy;
    op.in = {in};
    op.out = g->ops[in].out;
    op.out.c = 1;
    return push(g, std::move(op), out);
    MGI_ABI_CATCH("mgi_graph_add_entropy")
}

namespace {

mgi_status check_8bit_source(const mgi_graph *g, int in, const char *who) {
    const mgi_status s = check_tokens(g, in, who);
    if (s) return s;
    const Shape x = g->ops[in].out;
    if (x.c > kern::kMaxNormChannels)
        return fail(MGI_ERR_UNSUPPORTED, std::string(who) + ": at most " + std::to_string(kern::kMaxNormChannels) + " channels");
    if (!countable(x)) return fail(MGI_ERR_UNSUPPORTED, std::string(who) + ": tensor too large");
    return MGI_OK;
}

mgi_status check_index_input(const mgi_graph *g, int id, const char *who, const char *what) {
    const mgi_status s = check_tensor(g, id, who);
    if (s) return s;
    const GOp &ix = g->ops[id];
    if (ix.kind != OpKind::Input || ix.in_dtype != MGI_DTYPE_INT32)
        return fail(MGI_ERR_INVALID_ARG, std::string(who) + ": " + what + " is an index input");
    return MGI_OK;
}

}  // namespace

extern "C" mgi_status mgi_graph_add_rms_norm(mgi_graph *g, int in, const float *weight, float eps, int to8, int *out) {
    MGI_ABI_TRY
    const char *who = "mgi_graph_add_rms_norm";
    const mgi_status s = check_8bit_source(g, in, who);
    if (s) return s;
    if (!out) return fail(MGI_ERR_INVALID_ARG, std::string(who) + ": null pointer");
    if (!std::isfinite(eps) || eps < 0.0f) return fail(MGI_ERR_INVALID_ARG, std::string(who) + ": eps is at least 0 and finite");
    if (to8 != 0 && to8 != 1) return fail(MGI_ERR_INVALID_ARG, std::string(who) + ": to8 is 0 or 1");
    GOp op;
    op.kind = OpKind::RmsNorm;
    op.in = {in};
    op.out = g->ops[in].out;
    op.eps = eps;
    op.to8 = to8 != 0;
    try {
        if (weight) op.w.assign(weight, weight + op.out.c); else op.w.assign(op.out.c, 1.0f);
    } catch (const std::bad_alloc &) {
        return fail(MGI_ERR_OOM_HOST, std::string(who) + ": out of host memory");
    }
    return push(g, std::move(op), out);
    MGI_ABI_CATCH("mgi_graph_add_rms_norm")
}

extern "C" mgi_status mgi_graph_add_quantize(mgi_graph *g, int in, int *out) {
    MGI_ABI_TRY
    const char *who = "mgi_graph_add_quantize";
    const mgi_status s = check_8bit_source(g, in, who);
    if (s) return s;
    if (!out) return fail(MGI_ERR_INVALID_ARG, std::string(who) + ": null pointer");
    GOp op;
    op.kind = OpKind::Quantize;
    op.in = {in};
    op.out = g->ops[in].out;
    return push(g, std::move(op), out);
    MGI_ABI_CATCH("mgi_graph_add_quantize")
}

extern "C" mgi_status mgi_graph_add_pointwise_fp8(mgi_graph *g, int in, int cout, const unsigned char *codes,
                                                  const float *scales, const float *bias, int act, int *out) {
    MGI_ABI_TRY
    const char *who = "mgi_graph_add_pointwise_fp8";
    const mgi_status s = check_tensor(g, in, who);
    if (s) return s;
    if (!out || !codes || !scales) return fail(MGI_ERR_INVALID_ARG, std::string(who) + ": null pointer");
    if (cout <= 0) return fail(MGI_ERR_INVALID_ARG, std::string(who) + ": cout must be positive");
    if (!valid_act(act)) return fail(MGI_ERR_INVALID_ARG, std::string(who) + ": bad activation");
    if (!is_8bit(g->ops[in]))
        return fail(MGI_ERR_UNSUPPORTED, std::string(who) + ": tensor " + std::to_string(in) + " is not held in 8 bits");
    const Shape x = g->ops[in].out;
    Shape y = x;
    y.c = cout;
    if (cout > (1 << 24) || !countable(y)) return fail(MGI_ERR_UNSUPPORTED, std::string(who) + ": tensor too large");
    const size_t n = (size_t)cout * x.c, ns = (((size_t)cout + 127) / 128) * (((size_t)x.c + 127) / 128);
    for (size_t i = 0; i < ns; ++i)
        if (!std::isfinite(scales[i])) return fail(MGI_ERR_INVALID_ARG, std::string(who) + ": scales must be finite");
    for (size_t i = 0; i < n; ++i)
        if ((codes[i] & 0x7f) == 0x7f) return fail(MGI_ERR_INVALID_ARG, std::string(who) + ": a code is NaN");
    GOp op;
    op.kind = OpKind::PointwiseFp8;
    op.in = {in};
    op.cout = cout;
    op.act = act;
    op.out = y;
    try {
        op.codes.assign(codes, codes + n);
        op.w.assign(scales, scales + ns);
        if (bias) op.b.assign(bias, bias + cout); else op.b.assign(cout, 0.0f);
    } catch (const std::bad_alloc &) {
        return fail(MGI_ERR_OOM_HOST, std::string(who) + ": out of host memory");
    }
    return push(g, std::move(op), out);
    MGI_ABI_CATCH("mgi_graph_add_pointwise_fp8")
}

extern "C" mgi_status mgi_graph_add_rotary(mgi_graph *g, int in, const mgi_rotary_desc *d, const int *axes,
                                           const double *freqs, int positions, int *out) {
    MGI_ABI_TRY
    const char *who = "mgi_graph_add_rotary";
    mgi_status s = check_tokens(g, in, who);
    if (s) return s;
    if (!out || !d) return fail(MGI_ERR_INVALID_ARG, std::string(who) + ": null pointer");
    if (d->heads <= 0 || d->head_dim <= 0 || d->from < 0 || d->pairs < 0 || (d->adjacent != 0 && d->adjacent != 1))
        return fail(MGI_ERR_INVALID_ARG, std::string(who) + ": heads and head_dim are positive, from and pairs at least 0, adjacent 0 or 1");
    if (d->head_dim % 8 || d->from % 8)
        return fail(MGI_ERR_UNSUPPORTED, std::string(who) + ": head_dim and from are multiples of 8");
    if (d->pairs > d->head_dim / 2) return fail(MGI_ERR_SHAPE, std::string(who) + ": more pairs than half a head's channels");
    if (d->pairs > 0 && (!axes || !freqs)) return fail(MGI_ERR_INVALID_ARG, std::string(who) + ": null pointer");
    const Shape x = g->ops[in].out;
    if ((long)d->from + (long)d->heads * d->head_dim > x.c)
        return fail(MGI_ERR_SHAPE, std::string(who) + ": heads past the last channel");
    int n_axes = 3;
    if (positions != -1) {
        if ((s = check_index_input(g, positions, who, "positions"))) return s;
        const Shape ps = g->ops[positions].out;
        if (ps.n != x.n || ps.h != x.h || ps.w != x.w)
            return fail(MGI_ERR_SHAPE, std::string(who) + ": positions differ in n, h or w");
        if (ps.c > kern::kMaxAxes)
            return fail(MGI_ERR_UNSUPPORTED, std::string(who) + ": at most " + std::to_string(kern::kMaxAxes) + " axes");
        n_axes = ps.c;
    }
    for (int i = 0; i < d->pairs; ++i) {
        if (axes[i] < 0 || axes[i] >= n_axes) return fail(MGI_ERR_INVALID_ARG, std::string(who) + ": no such axis");
        if (!std::isfinite(freqs[i])) return fail(MGI_ERR_INVALID_ARG, std::string(who) + ": freqs must be finite");
    }
    GOp op;
    op.kind = OpKind::Rotary;
    op.in = {in};
    if (positions != -1) op.in.push_back(positions);
    op.out = x;
    op.out.c = d->heads * d->head_dim;
    if (!countable(x) || !countable(op.out)) return fail(MGI_ERR_UNSUPPORTED, std::string(who) + ": tensor too large");
    op.rotary = *d;
    try {
        op.axes.assign(axes, axes + d->pairs);
        op.freqs.assign(freqs, freqs + d->pairs);
    } catch (const std::bad_alloc &) {
        return fail(MGI_ERR_OOM_HOST, std::string(who) + ": out of host memory");
    }
    return push(g, std::move(op), out);
    MGI_ABI_CATCH("mgi_graph_add_rotary")
}

extern "C" mgi_status mgi_graph_add_attention(mgi_graph *g, int q, int k, int v, const mgi_attention_desc *d,
                                              int bounds, int k_bounds, int *out) {
    MGI_ABI_TRY
    const char *who = "mgi_graph_add_attention";
    mgi_status s;
    for (int t : {q, k, v})
        if ((s = check_tokens(g, t, who))) return s;
    if (!out || !d) return fail(MGI_ERR_INVALID_ARG, std::string(who) + ": null pointer");
    if (d->heads <= 0 || d->kv_heads <= 0 || d->head_dim <= 0 || d->heads % d->kv_heads)
        return fail(MGI_ERR_INVALID_ARG, std::string(who) + ": heads, kv_heads and head_dim are positive, heads a multiple of kv_heads");
    if (d->q_from < 0 || d->k_from < 0 || d->v_from < 0 || (d->causal != 0 && d->causal != 1) || !std::isfinite(d->scale))
        return fail(MGI_ERR_INVALID_ARG, std::string(who) + ": first channels are at least 0, causal 0 or 1, scale finite");
    if (d->head_dim % 8 || d->head_dim > kern::kMaxHeadDim || d->q_from % 8 || d->k_from % 8 || d->v_from % 8)
        return fail(MGI_ERR_UNSUPPORTED, std::string(who) + ": head_dim and first channels are multiples of 8, head_dim at most " +
                                             std::to_string(kern::kMaxHeadDim));
    const Shape xq = g->ops[q].out, xk = g->ops[k].out, xv = g->ops[v].out;
    const long dim = d->head_dim;
    if (d->q_from + d->heads * dim > xq.c || d->k_from + d->kv_heads * dim > xk.c || d->v_from + d->kv_heads * dim > xv.c)
        return fail(MGI_ERR_SHAPE, std::string(who) + ": heads past the last channel");
    if (xk.n != xv.n || xk.h != xv.h || xk.w != xv.w)
        return fail(MGI_ERR_SHAPE, std::string(who) + ": k and v differ in n, h or w");
    GOp op;
    op.kind = OpKind::Attention;
    op.in = {q, k, v};
    op.out = xq;
    op.out.c = (int)(d->heads * dim);
    if (!countable(xq) || !countable(xk) || !countable(xv) || !countable(op.out))
        return fail(MGI_ERR_UNSUPPORTED, std::string(who) + ": tensor too large");
    if (bounds == -1) {
        if (k_bounds != -1) return fail(MGI_ERR_INVALID_ARG, std::string(who) + ": k_bounds without bounds");
        if (xq.n != xk.n) return fail(MGI_ERR_SHAPE, std::string(who) + ": q and k differ in n");
    } else {
        if ((s = check_index_input(g, bounds, who, "bounds"))) return s;
        const size_t nb = g->ops[bounds].out.elems();
        if (nb < 2) return fail(MGI_ERR_SHAPE, std::string(who) + ": at least two bounds");
        if (nb > (size_t)kern::kMaxSequences + 1)
            return fail(MGI_ERR_UNSUPPORTED, std::string(who) + ": at most " + std::to_string(kern::kMaxSequences) + " sequences");
        op.in.push_back(bounds);
        if (k_bounds != -1) {
            if ((s = check_index_input(g, k_bounds, who, "k_bounds"))) return s;
            if (g->ops[k_bounds].out.elems() != nb) return fail(MGI_ERR_SHAPE, std::string(who) + ": as many k_bounds as bounds");
            op.in.push_back(k_bounds);
        } else if (xq.pixels() != xk.pixels()) {
            return fail(MGI_ERR_SHAPE, std::string(who) + ": q and k differ in pixels, and there are no k_bounds");
        }
    }
    op.attention = *d;
    // (the kernel counts query rows of a group of heads in an int)
    if ((unsigned __int128)xq.pixels() * (d->heads / d->kv_heads) > INT_MAX / 2)
        return fail(MGI_ERR_UNSUPPORTED, std::string(who) + ": too many queries");
    // (... and a launch has fewer than 2^24 workgroups of 256 threads)
    const kern::AttentionGeom geo = kern::attention_geom((int)xq.pixels(), (int)xk.pixels(), xq.n,
                                                         bounds == -1 ? 0 : (int)g->ops[bounds].out.elems() - 1,
                                                         d->heads / d->kv_heads, d->kv_heads, d->head_dim / 8);
    if ((uint64_t)geo.tiles * d->kv_heads * geo.chunks >= 1u << 24)
        return fail(MGI_ERR_UNSUPPORTED, std::string(who) + ": too many sequences and heads");
    return push(g, std::move(op), out);
    MGI_ABI_CATCH("mgi_graph_add_attention")
}

namespace {

mgi_status mark_output(mgi_graph *g, int id, int dtype, const char *who) {
    mgi_status s = check_tensor(g, id, who);
    if (s) return s;
    if (g->ops[id].kind == OpKind::Input)
        return fail(MGI_ERR_UNSUPPORTED, std::string(who) + ": a graph input cannot be an output");
    for (int t : g->outputs)
        if (t == id) return fail(MGI_ERR_INVALID_ARG, std::string(who) + ": already an output");
    g->outputs.push_back(id);
    g->output_dtypes.push_back(dtype);
    return MGI_OK;
}

}  // namespace

extern "C" mgi_status mgi_graph_mark_output(mgi_graph *g, int id) {
    MGI_ABI_TRY
    return mark_output(g, id, MGI_DTYPE_FP32, "mgi_graph_mark_output");
    MGI_ABI_CATCH("mgi_graph_mark_output")
}

extern "C" mgi_status mgi_graph_mark_output_as(mgi_graph *g, int id, int dtype) {
    MGI_ABI_TRY
    const char *who = "mgi_graph_mark_output_as";
    if (dtype != MGI_DTYPE_FP32 && dtype != MGI_DTYPE_FP16 && dtype != MGI_DTYPE_BF16)
        return fail(MGI_ERR_UNSUPPORTED, std::string(who) + ": outputs are fp32, fp16 or bf16");
    mgi_status s = check_tensor(g, id, who);
    if (s) return s;
    const OpKind k = g->ops[id].kind;
    if (dtype != MGI_DTYPE_FP32 && (k == OpKind::FC || k == OpKind::FcInt4 || k == OpKind::Softmax || k == OpKind::Argmax ||
                                    k == OpKind::TopK || k == OpKind::LogProb || k == OpKind::Entropy))
        return fail(MGI_ERR_UNSUPPORTED, std::string(who) + ": tensor " + std::to_string(id) + " is not stored in 16 bits");
    return mark_output(g, id, dtype, who);
    MGI_ABI_CATCH("mgi_graph_mark_output_as")
}

extern "C" void mgi_options_default(mgi_options *o) {
    if (!o) return;
    o->planner = MGI_PLANNER_GREEDY;
    o->fuse = 1;
    o->materialize_all = 0;
    o->dtype = MGI_DTYPE_FP16;
    o->fuse_dwpw = 0;
    o->fuse_pwdw = 1;
    o->fuse_stemdw = 1;
    o->fuse_pool = 1;
    o->fuse_softmax = 1;
    o->fuse_irb = 0;
}
