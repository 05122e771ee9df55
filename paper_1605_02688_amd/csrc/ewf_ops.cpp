// The operators of sequence models: argument checks and layouts.  The kernels are in ewf_norm.hip, ewf_act8.hip,
// ewf_recurrence.hip, ewf_logprobs.hip and ewf_distill.hip; everything that they assume about their operands is established here.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstring>
#include <initializer_list>

#include "ewf_internal.h"
#include "ewf_ops.h"

using namespace ewf;

namespace {

constexpr int64_t kMaxCols = (int64_t)1 << 30;
constexpr int64_t kMaxNormCols = (int64_t)1 << 24;      // what one workgroup's sums are accurate for
constexpr int64_t kMaxRows = ((int64_t)1 << 31) - 1;
constexpr int64_t kMaxStepBytes = (int64_t)32 << 20;

int float_size(int t) { return t == EWF_F32 ? 4 : 2; }
bool is_float(int t) { return t == EWF_F32 || t == EWF_F16 || t == EWF_BF16; }
bool is_code(int t) { return t == EWF_I8 || t == EWF_E4M3; }
bool present(const ewf_tensor &t) { return t.ptr || t.shape; }

struct Operand8 {
    const char *name;
    const ewf_tensor *t;
    RawView view;
    bool out;
    uint64_t begin = 0, end = 0;         // of its bytes; equal where it has no elements
};

// The tensors of one call, checked one by one as they are added.
struct Call {
    // (no heap: the checks are made on every call)
    Operand8 ops[16];
    size_t n = 0;
    ewf_status status = EWF_OK;

    ewf_status fail(ewf_status s) { return status = s; }

    // Adds tensor `t` of `rank` axes; `shape` are the extents it must have.  Absent tensors are skipped
    // (a required one is an error).  Returns whether the tensor is there and sound.
    bool add(const char *name, const ewf_tensor &t, int isz, int rank, const int64_t *shape, bool out, bool required)
    {
        if (status != EWF_OK) return false;
        if (!present(t)) {
            if (required) { set_error("%s is needed", name); fail(EWF_EINVAL); }
            return false;
        }
        if (rank > 0 && (!t.shape || !t.strides)) { set_error("%s: null shape or strides", name); fail(EWF_EINVAL); return false; }
        Operand8 o{name, &t, RawView{(uint64_t)(uintptr_t)t.ptr, isz, {0}, {0}, rank}, out};
        bool empty = false;
        double span = 1;
        uint64_t reach = 1;
        for (int d = 0; d < rank; d++) {
            if (t.shape[d] != shape[d]) {
                set_error("%s: dimension %d has extent %lld, expected %lld", name, d, (long long)t.shape[d], (long long)shape[d]);
                fail(EWF_ESHAPE);
                return false;
            }
            if (t.strides[d] < 0) { set_error("%s: negative strides are not supported", name); fail(EWF_EINVAL); return false; }
            if (t.shape[d] == 0) empty = true;
            o.view.ext[d] = t.shape[d];
            o.view.str[d] = t.shape[d] > 1 ? t.strides[d] : 0;
            if (t.shape[d] > 1) {
                span += (double)(t.shape[d] - 1) * (double)t.strides[d];
                reach += (uint64_t)(t.shape[d] - 1) * (uint64_t)t.strides[d];
            }
        }
        if (empty) { ops[n++] = o; return true; }
        if (!t.ptr) { set_error("%s: null pointer", name); fail(EWF_EINVAL); return false; }
        if ((uintptr_t)t.ptr % (unsigned)isz) { set_error("%s: the pointer is not aligned to its element", name); fail(EWF_EINVAL); return false; }
        if (span * isz >= 0x1p62) { set_error("%s: its extents and strides reach beyond the address space", name); fail(EWF_ESHAPE); return false; }
        o.begin = o.view.addr;
        o.end = o.begin + reach * (uint64_t)isz;
        // (each axis steps over what the axes behind it span: the usual case, found without sorting)
        int64_t behind = 0;
        bool apart = true;
        for (int d = rank - 1; out && apart && d >= 0; d--) {
            if (o.view.ext[d] <= 1) continue;
            apart = o.view.str[d] > behind;
            behind += (o.view.ext[d] - 1) * o.view.str[d];
        }
        if (out && !apart && !self_disjoint(o.view)) { set_error("%s: two of its elements share memory", name); fail(EWF_EALIAS); return false; }
        ops[n++] = o;
        return true;
    }
    bool add(const char *name, const ewf_tensor &t, int isz, std::initializer_list<int64_t> shape, bool out, bool required)
    {
        return add(name, t, isz, (int)shape.size(), shape.begin(), out, required);
    }

    // The last axis must be contiguous.
    ewf_status unit_last(const ewf_tensor &t, const char *name, int rank)
    {
        if (status != EWF_OK || !present(t) || rank == 0) return status;
        if (t.shape[rank - 1] > 1 && t.strides[rank - 1] != 1) {
            set_error("%s: the last axis must be contiguous (its stride is %lld)", name, (long long)t.strides[rank - 1]);
            return fail(EWF_EUNSUPPORTED);
        }
        return status;
    }

    // Results overlap nothing, but for results that lie exactly over one of the operands they may lie over.
    ewf_status check_results(std::initializer_list<std::pair<const char *, const char *>> allowed)
    {
        if (status != EWF_OK) return status;
        for (size_t o = 0; o < n; o++) {
            if (!ops[o].out) continue;
            for (size_t k = 0; k < n; k++) {
                if (k == o || (ops[k].out && k > o) || ops[k].end <= ops[o].begin || ops[o].end <= ops[k].begin) continue;
                if (!views_overlap(ops[k].view, ops[o].view)) continue;
                bool ok = false;
                for (auto &p : allowed)
                    ok = ok || (!ops[k].out && !strcmp(p.first, ops[o].name) && !strcmp(p.second, ops[k].name) &&
                                ops[k].view.rank == ops[o].view.rank && same_view(ops[k].view, ops[o].view));
                if (ok) continue;
                set_error("%s overlaps %s", ops[o].name, ops[k].name);
                return fail(EWF_EALIAS);
            }
        }
        return status;
    }
};

// The axes before the last of the row tensors, merged into at most two that all of them share.
struct RowLayout {
    static constexpr int kMaxRowTensors = 12;
    struct Entry { const ewf_tensor *t; RowStride *to; };
    Entry e[kMaxRowTensors];
    size_t n = 0;
    void add(const ewf_tensor &t, RowStride *to) { if (present(t)) e[n++] = {&t, to}; }

    ewf_status merge(const int64_t *shape, int lead, Rows &r)
    {
        double total = 1;
        for (int d = 0; d < lead; d++) total *= (double)shape[d];
        if (total > (double)kMaxRows) { set_error("%.0f rows: fewer than 2^31 are supported", total); return EWF_ESHAPE; }
        if (total == 0) { r.rows = 0; r.n1 = 1; return EWF_OK; }
        struct Axis { int64_t ext, st[kMaxRowTensors]; } axes[kMaxDims];
        int naxes = 0;
        for (int d = 0; d < lead; d++) {
            if (shape[d] == 1) continue;
            Axis &a = axes[naxes];
            a.ext = shape[d];
            for (size_t k = 0; k < n; k++) a.st[k] = e[k].t->strides[d];
            bool ok = naxes > 0;
            for (size_t k = 0; ok && k < n; k++) ok = axes[naxes - 1].st[k] == a.st[k] * a.ext;
            if (!ok) { naxes++; continue; }
            a.ext *= axes[naxes - 1].ext;
            axes[naxes - 1] = a;
        }
        if (naxes > 2) { set_error("the axes before the last do not merge into two that all tensors share"); return EWF_EUNSUPPORTED; }
        r.rows = (uint32_t)total;
        r.n1 = naxes ? (uint32_t)axes[naxes - 1].ext : 1;
        for (size_t k = 0; k < n; k++) {
            e[k].to->inner = naxes ? axes[naxes - 1].st[k] : 0;
            e[k].to->outer = naxes == 2 ? axes[0].st[k] : 0;
        }
        return EWF_OK;
    }
};

// Shape of the tensor that the others of a call are measured by.
ewf_status base_shape(const char *name, const ewf_tensor &t, int32_t ndim, int64_t *shape)
{
    if (ndim < 1 || ndim > EWF_MAX_DIMS) { set_error("bad rank"); return EWF_EINVAL; }
    if (!present(t)) { set_error("%s is needed", name); return EWF_EINVAL; }
    if (!t.shape || !t.strides) { set_error("%s: null shape or strides", name); return EWF_EINVAL; }
    for (int d = 0; d < ndim; d++) {
        if (t.shape[d] < 0) { set_error("%s: negative extent", name); return EWF_EINVAL; }
        shape[d] = t.shape[d];
    }
    return EWF_OK;
}

// Launches, and says what came of it (an error that an earlier call of the program's has left unread is not this one's).
template <typename F>
ewf_status launched(const char *what, F &&launch)
{
    (void)hipGetLastError();
    launch();
    hipError_t he = hipGetLastError();
    if (he == hipSuccess) return EWF_OK;
    set_error("%s: %s", what, hipGetErrorString(he));
    return EWF_EHIP;
}

ewf_status workspace_fits(size_t need, void *workspace, size_t bytes)
{
    if (need == 0) return EWF_OK;
    if (!workspace || bytes < need) { set_error("workspace of %zu bytes needed, %zu given", need, workspace ? bytes : (size_t)0); return EWF_ENOMEM; }
    if ((uintptr_t)workspace & 15) { set_error("workspace must be 16-byte aligned"); return EWF_EINVAL; }
    return EWF_OK;
}

// codes and scales, both or neither.
ewf_status kept_pair(Call &c, RowLayout &l, const ewf_tensor &codes, const ewf_tensor &scales, int code_dtype, const int64_t *shape, int nd,
                     bool out, bool required, RowStride *sc, RowStride *ss)
{
    if (c.status != EWF_OK) return c.status;
    if (present(codes) != present(scales)) { set_error("codes and scales come together"); return c.fail(EWF_EINVAL); }
    if (present(codes) && !is_code(code_dtype)) { set_error("codes are int8 or e4m3"); return c.fail(EWF_ETYPE); }
    int64_t ks[kMaxDims];
    for (int d = 0; d < nd; d++) ks[d] = shape[d];
    ks[nd - 1] = (shape[nd - 1] + kKeepBlock - 1) / kKeepBlock;
    c.add("codes", codes, 1, nd, shape, out, required);
    c.add("scales", scales, 1, nd, ks, out, required);
    c.unit_last(codes, "codes", nd);
    c.unit_last(scales, "scales", nd);
    l.add(codes, sc);
    l.add(scales, ss);
    return c.status;
}

// ------------------------------------------------------------------ layer normalisation

ewf_status norm_layout(const ewf_layer_norm_args *a, bool grad, NormLaunch &n)
{
    if (!a) { set_error("null arguments"); return EWF_EINVAL; }
    if (a->reserved) { set_error("reserved must be 0"); return EWF_EINVAL; }
    if (!is_float(a->dtype)) { set_error("tensors are float32, float16 or bfloat16"); return EWF_ETYPE; }
    const bool params = present(a->weight) || (grad ? present(a->dweight) || present(a->dbias) : present(a->bias));
    if (params && a->param_dtype != a->dtype && a->param_dtype != EWF_F32) { set_error("parameters have the tensors' type or float32"); return EWF_ETYPE; }
    int64_t shape[kMaxDims];
    const int nd = a->ndim;
    ewf_status st = grad ? base_shape("dy", a->dy, nd, shape) : base_shape("x", a->x, nd, shape);
    if (st != EWF_OK) return st;
    const int64_t cols = shape[nd - 1];
    if (cols < 1 || cols > kMaxNormCols) { set_error("rows of %lld elements: 1 to 2^24 are supported", (long long)cols); return EWF_ESHAPE; }
    if (!grad && !(a->eps >= 0)) { set_error("eps must not be negative"); return EWF_EINVAL; }
    const int isz = float_size(a->dtype), psz = float_size(a->param_dtype);
    Call c;
    RowLayout l;
    n = NormLaunch();
    n.dtype = a->dtype; n.param_dtype = a->param_dtype; n.code_dtype = a->code_dtype; n.eps = a->eps;
    auto full = [&](const char *name, const ewf_tensor &t, bool out, bool required, RowStride *to) {
        if (!c.add(name, t, isz, nd, shape, out, required)) return;
        c.unit_last(t, name, nd);
        l.add(t, to);
    };
    auto stat = [&](const char *name, const ewf_tensor &t, bool out, bool required, RowStride *to) {
        if (c.add(name, t, 4, nd - 1, shape, out, required)) l.add(t, to);
    };
    auto param = [&](const char *name, const ewf_tensor &t, bool out) {
        if (c.add(name, t, psz, {cols}, out, false)) c.unit_last(t, name, 1);
    };
    param("weight", a->weight, false);
    if (!grad) {
        param("bias", a->bias, false);
        full("x", a->x, false, true, &n.sx);
        full("y", a->y, true, true, &n.sy);
        stat("mean", a->mean, true, false, &n.smean);
        stat("rstd", a->rstd, true, false, &n.srstd);
        kept_pair(c, l, a->codes, a->scales, a->code_dtype, shape, nd, true, false, &n.scodes, &n.sscales);
        c.check_results({{"y", "x"}});
    } else {
        full("dy", a->dy, false, true, &n.sdy);
        stat("rstd", a->rstd, false, true, &n.srstd);
        if (c.status == EWF_OK && present(a->x) == present(a->codes)) { set_error("either x and mean or codes and scales are needed"); return EWF_EINVAL; }
        if (c.status == EWF_OK && present(a->x)) {
            full("x", a->x, false, true, &n.sx);
            stat("mean", a->mean, false, true, &n.smean);
        } else {
            kept_pair(c, l, a->codes, a->scales, a->code_dtype, shape, nd, false, true, &n.scodes, &n.sscales);
        }
        full("dx", a->dx, true, true, &n.sdx);
        param("dweight", a->dweight, true);
        param("dbias", a->dbias, true);
        c.check_results({{"dx", "dy"}, {"dx", "x"}});
    }
    if (c.status != EWF_OK) return c.status;
    st = l.merge(shape, nd - 1, n.r);
    if (st != EWF_OK) return st;
    n.r.cols = (int32_t)cols;
    n.x = a->x.ptr; n.weight = a->weight.ptr; n.bias = a->bias.ptr; n.y = a->y.ptr; n.dy = a->dy.ptr; n.dx = a->dx.ptr;
    n.dweight = a->dweight.ptr; n.dbias = a->dbias.ptr;
    n.mean = (float *)a->mean.ptr; n.rstd = (float *)a->rstd.ptr;
    n.codes = (uint8_t *)a->codes.ptr; n.scales = (uint8_t *)a->scales.ptr;
    if (grad && n.codes) { n.x = nullptr; n.mean = nullptr; }
    if (grad) plan_layer_norm_grad(n, device_cu_count());
    return EWF_OK;
}

size_t norm_workspace(const NormLaunch &n)
{
    return n.dweight || n.dbias ? (size_t)n.blocks * 2 * (size_t)n.padded * sizeof(float) : 0;
}

// ------------------------------------------------------------------ activations in 8 bits

enum class ActCall { Forward, Grad, Read };

ewf_status act_layout(const ewf_activation_args *a, ActCall call, ActLaunch &n)
{
    if (!a) { set_error("null arguments"); return EWF_EINVAL; }
    if (!is_float(a->dtype)) { set_error("tensors are float32, float16 or bfloat16"); return EWF_ETYPE; }
    if ((int)a->act < 0 || a->act >= EWF_ACT_COUNT) { set_error("unknown activation"); return EWF_EINVAL; }
    int64_t shape[kMaxDims];
    const int nd = a->ndim;
    ewf_status st = call == ActCall::Grad ? base_shape("dy", a->dy, nd, shape) : base_shape("x", a->x, nd, shape);
    if (st != EWF_OK) return st;
    const int64_t cols = shape[nd - 1];
    if (cols > kMaxCols) { set_error("rows of %lld elements: at most 2^30 are supported", (long long)cols); return EWF_ESHAPE; }
    const int isz = float_size(a->dtype);
    Call c;
    RowLayout l;
    n = ActLaunch();
    n.dtype = a->dtype; n.code_dtype = a->code_dtype; n.act = a->act;
    auto full = [&](const char *name, const ewf_tensor &t, bool out, bool required, RowStride *to) {
        if (!c.add(name, t, isz, nd, shape, out, required)) return;
        c.unit_last(t, name, nd);
        l.add(t, to);
    };
    if (call == ActCall::Forward) {
        if (!present(a->y) && !present(a->codes)) { set_error("y, or codes and scales, are needed"); return EWF_EINVAL; }
        full("x", a->x, false, true, &n.sx);
        full("y", a->y, true, false, &n.sy);
        kept_pair(c, l, a->codes, a->scales, a->code_dtype, shape, nd, true, false, &n.scodes, &n.sscales);
        c.check_results({{"y", "x"}});
        n.x = a->x.ptr; n.y = a->y.ptr;
    } else if (call == ActCall::Grad) {
        full("dy", a->dy, false, true, &n.sdy);
        kept_pair(c, l, a->codes, a->scales, a->code_dtype, shape, nd, false, true, &n.scodes, &n.sscales);
        full("dx", a->dx, true, true, &n.sdx);
        c.check_results({{"dx", "dy"}});
        n.dy = a->dy.ptr; n.dx = a->dx.ptr;
    } else {
        kept_pair(c, l, a->codes, a->scales, a->code_dtype, shape, nd, false, true, &n.scodes, &n.sscales);
        full("x", a->x, true, true, &n.sdx);
        c.check_results({});
        n.dx = a->x.ptr;
        n.act = EWF_IDENTITY;
    }
    if (c.status != EWF_OK) return c.status;
    st = l.merge(shape, nd - 1, n.r);
    if (st != EWF_OK) return st;
    n.r.cols = (int32_t)cols;
    n.codes = (uint8_t *)a->codes.ptr; n.scales = (uint8_t *)a->scales.ptr;
    return EWF_OK;
}

// ------------------------------------------------------------------ recurrence

ewf_status rec_layout(const ewf_recurrence_args *a, bool grad, RecLaunch &n)
{
    if (!a) { set_error("null arguments"); return EWF_EINVAL; }
    if (a->reserved) { set_error("reserved must be 0"); return EWF_EINVAL; }
    if (!is_float(a->dtype)) { set_error("tensors are float32, float16 or bfloat16"); return EWF_ETYPE; }
    int64_t s[kMaxDims];
    ewf_status st = base_shape("u", a->u, 3, s);
    if (st != EWF_OK) return st;
    // (steps and channels are counted in 32 bits, to the end of the last tile)
    if ((double)s[0] * (double)s[2] > (double)kMaxRows - 64 || s[1] > ((int64_t)1 << 30)) {
        set_error("at most 2^30 steps, and fewer than 2^31 sequences times channels, are supported");
        return EWF_ESHAPE;
    }
    const int isz = float_size(a->dtype);
    Call c;
    n = RecLaunch();
    n.dtype = a->dtype; n.batch = s[0]; n.steps = s[1]; n.channels = s[2];
    auto seq = [&](const char *name, const ewf_tensor &t, bool out, bool required, RecTensor &to) {
        if (!c.add(name, t, isz, {s[0], s[1], s[2]}, out, required)) return;
        c.unit_last(t, name, 3);
        to.p = t.ptr;
        to.batch = s[0] > 1 ? t.strides[0] : 0;
        to.step = s[1] > 1 ? t.strides[1] : 0;
        // (the kernels reach 32 steps with offsets of 31 bits)
        if (to.step > kMaxStepBytes / isz) {
            set_error("%s: steps that are %lld elements apart: at most 32 MiB are supported", name, (long long)to.step);
            c.fail(EWF_EUNSUPPORTED);
        }
    };
    auto state = [&](const char *name, const ewf_tensor &t, bool out, RecTensor &to) {
        if (!c.add(name, t, 4, {s[0], s[2]}, out, false)) return;
        c.unit_last(t, name, 2);
        to.p = t.ptr;
        to.batch = s[0] > 1 ? t.strides[0] : 0;
    };
    seq("u", a->u, false, true, n.u);
    seq("v", a->v, false, true, n.v);
    seq("w", a->w, false, false, n.w);
    state("h0", a->h0, false, n.h0);
    if (c.add("lengths", a->lengths, 4, {s[0]}, false, false)) {
        n.lengths = (const int32_t *)a->lengths.ptr;
        n.lengths_stride = s[0] > 1 ? a->lengths.strides[0] : 0;
    }
    seq("h", a->h, !grad, true, n.h);
    if (!grad) {
        state("last", a->last, true, n.last);
        c.check_results({{"h", "u"}, {"h", "v"}, {"h", "w"}, {"last", "h0"}});
    } else {
        seq("dh", a->dh, false, true, n.dh);
        state("dlast", a->dlast, false, n.dlast);
        seq("du", a->du, true, true, n.du);
        seq("dv", a->dv, true, true, n.dv);
        if (c.status == EWF_OK && present(a->w) != present(a->dw)) { set_error("dw comes with w"); return EWF_EINVAL; }
        seq("dw", a->dw, true, false, n.dw);
        state("dh0", a->dh0, true, n.dh0);
        c.check_results({{"du", "u"}, {"du", "v"}, {"du", "w"}, {"du", "dh"}, {"dv", "u"}, {"dv", "v"}, {"dv", "w"}, {"dv", "dh"},
                         {"dw", "u"}, {"dw", "v"}, {"dw", "w"}, {"dw", "dh"}, {"dh0", "dlast"}});
    }
    if (c.status != EWF_OK) return c.status;
    return EWF_OK;
}

ewf_status rec_workspace(const ewf_recurrence_args *a, bool grad, size_t *bytes)
{
    if (!bytes) { set_error("null argument"); return EWF_EINVAL; }
    RecLaunch n;
    ewf_status st = rec_layout(a, grad, n);
    if (st == EWF_OK) *bytes = recurrence_workspace(n, grad, device_cu_count());
    return st;
}

ewf_status rec_run(const ewf_recurrence_args *a, bool grad, void *workspace, size_t bytes, void *stream)
{
    RecLaunch n;
    ewf_status st = rec_layout(a, grad, n);
    if (st != EWF_OK) return st;
    const int units = device_cu_count();
    st = workspace_fits(recurrence_workspace(n, grad, units), workspace, bytes);
    if (st != EWF_OK) return st;
    if (n.batch == 0 || n.channels == 0) return EWF_OK;
    n.workspace = workspace;
    return launched(grad ? "recurrence, backward" : "recurrence", [&] { launch_recurrence(n, grad, units, (hipStream_t)stream); });
}

// ------------------------------------------------------------------ rows of logits

constexpr int64_t kMaxVocab = (int64_t)1 << 24;

// What the operators over a vocabulary have in common: their logits, scale and results by row.
struct VocabCall {
    Call c;
    RowLayout l;
    VocabLaunch &n;
    int64_t shape[kMaxDims];
    int nd = 0;

    explicit VocabCall(VocabLaunch &n) : n(n) { n = VocabLaunch(); }

    ewf_status begin(const ewf_tensor &logits, int32_t dtype, int32_t ndim, float scale)
    {
        if (!is_float(dtype)) { set_error("tensors are float32, float16 or bfloat16"); return c.fail(EWF_ETYPE); }
        ewf_status st = base_shape("logits", logits, ndim, shape);
        if (st != EWF_OK) return c.fail(st);
        nd = ndim;
        if (shape[nd - 1] < 1 || shape[nd - 1] > kMaxVocab) {
            set_error("rows of %lld logits: 1 to 2^24 are supported", (long long)shape[nd - 1]);
            return c.fail(EWF_ESHAPE);
        }
        if (!(scale >= 0x1p-64f && scale <= 0x1p64f)) { set_error("scale: 2^-64 to 2^64 are supported"); return c.fail(EWF_EINVAL); }
        n.dtype = dtype;
        n.scale = scale;
        n.c = scale * 1.44269504f;
        n.lag = 8.f / n.c;
        full("logits", logits, false, true, &n.slogits);
        n.logits = logits.ptr;
        return c.status;
    }
    void full(const char *name, const ewf_tensor &t, bool out, bool required, RowStride *to)
    {
        if (!c.add(name, t, float_size(n.dtype), nd, shape, out, required)) return;
        c.unit_last(t, name, nd);
        l.add(t, to);
    }
    // A number a row: 4 bytes.
    template <typename P> void column(const char *name, const ewf_tensor &t, bool out, bool required, RowStride *to, P *&p)
    {
        if (!c.add(name, t, 4, nd - 1, shape, out, required)) return;
        l.add(t, to);
        p = (P *)t.ptr;
    }
    // `count` elements a row; count is the first such tensor's.
    bool few(const char *name, const ewf_tensor &t, int isz, bool out, int &count, RowStride *to)
    {
        if (c.status != EWF_OK) return false;
        if (!present(t)) { set_error("%s is needed", name); c.fail(EWF_EINVAL); return false; }
        if (!t.shape || !t.strides) { set_error("%s: null shape or strides", name); c.fail(EWF_EINVAL); return false; }
        int64_t s[kMaxDims];
        for (int d = 0; d < nd; d++) s[d] = shape[d];
        s[nd - 1] = count ? count : t.shape[nd - 1];
        if (s[nd - 1] < 1 || s[nd - 1] > kMaxTop) {
            set_error("%s: %lld a row: 1 to %d are supported", name, (long long)s[nd - 1], kMaxTop);
            c.fail(EWF_ESHAPE);
            return false;
        }
        if (!c.add(name, t, isz, nd, s, out, true)) return false;
        if (c.unit_last(t, name, nd) != EWF_OK) return false;
        count = (int)s[nd - 1];
        l.add(t, to);
        return true;
    }
    ewf_status end()
    {
        if (c.status != EWF_OK) return c.status;
        ewf_status st = l.merge(shape, nd - 1, n.r);
        n.r.cols = (int32_t)shape[nd - 1];
        return st;
    }
};

ewf_status logprobs_layout(const ewf_token_logprobs_args *a, bool grad, VocabLaunch &n)
{
    if (!a) { set_error("null arguments"); return EWF_EINVAL; }
    if (a->reserved) { set_error("reserved must be 0"); return EWF_EINVAL; }
    VocabCall v(n);
    if (v.begin(a->logits, a->dtype, a->ndim, a->scale) != EWF_OK) return v.c.status;
    v.column("tokens", a->tokens, false, false, &n.stokens, n.tokens);
    if (!grad) {
        if (v.c.status == EWF_OK && present(a->logprob) && !present(a->tokens)) { set_error("logprob comes with tokens"); return EWF_EINVAL; }
        v.column("logprob", a->logprob, true, false, &n.slogprob, n.logprob);
        v.column("peak", a->peak, true, false, &n.speak, n.peak);
        v.column("logsum", a->logsum, true, false, &n.slogsum, n.logsum);
        v.column("entropy", a->entropy, true, false, &n.sentropy, n.entropy);
        if (v.c.status == EWF_OK && present(a->top_values) != present(a->top_indices)) {
            set_error("top_values and top_indices come together");
            return EWF_EINVAL;
        }
        if (present(a->top_values)) {
            v.few("top_values", a->top_values, 4, true, n.top, &n.stop_values);
            v.few("top_indices", a->top_indices, 4, true, n.top, &n.stop_indices);
            n.top_values = (float *)a->top_values.ptr;
            n.top_indices = (int32_t *)a->top_indices.ptr;
        }
        if (v.c.status == EWF_OK && !present(a->logprob) && !present(a->peak) && !present(a->logsum) && !present(a->entropy) && !n.top) {
            set_error("a result is needed: logprob, peak, logsum, entropy or top_values and top_indices");
            return EWF_EINVAL;
        }
        v.c.check_results({});
    } else {
        if (v.c.status == EWF_OK && !present(a->dlogprob) && !present(a->dentropy)) { set_error("dlogprob or dentropy is needed"); return EWF_EINVAL; }
        if (v.c.status == EWF_OK && present(a->dlogprob) && !present(a->tokens)) { set_error("dlogprob comes with tokens"); return EWF_EINVAL; }
        v.column("peak", a->peak, false, true, &n.speak, n.peak);
        v.column("logsum", a->logsum, false, true, &n.slogsum, n.logsum);
        v.column("dlogprob", a->dlogprob, false, false, &n.sdlogprob, n.dlogprob);
        v.column("dentropy", a->dentropy, false, false, &n.sdentropy, n.dentropy);
        v.column("entropy", a->entropy, false, present(a->dentropy), &n.sentropy, n.entropy);
        v.full("dlogits", a->dlogits, true, true, &n.sdlogits);
        n.dlogits = a->dlogits.ptr;
        v.c.check_results({{"dlogits", "logits"}});
    }
    ewf_status st = v.end();
    if (st == EWF_OK) plan_vocab(n, device_cu_count());
    return st;
}

ewf_status distill_layout(const ewf_distill_args *a, bool grad, VocabLaunch &n)
{
    if (!a) { set_error("null arguments"); return EWF_EINVAL; }
    if (a->reserved) { set_error("reserved must be 0"); return EWF_EINVAL; }
    VocabCall v(n);
    if (v.begin(a->logits, a->dtype, a->ndim, a->scale) != EWF_OK) return v.c.status;
    if (a->teacher_dtype != a->dtype && a->teacher_dtype != EWF_F32) { set_error("the teacher's values have the logits' type or float32"); return EWF_ETYPE; }
    if (!(a->teacher_scale >= 0x1p-64f && a->teacher_scale <= 0x1p64f)) { set_error("teacher_scale: 2^-64 to 2^64 are supported"); return EWF_EINVAL; }
    n.teacher_dtype = a->teacher_dtype;
    n.teacher_scale = a->teacher_scale;
    n.with_tail = present(a->tail);
    if (v.few("teacher_values", a->teacher_values, float_size(a->teacher_dtype), false, n.entries, &n.steacher_values))
        v.few("teacher_indices", a->teacher_indices, 4, false, n.entries, &n.steacher_indices);
    n.teacher_values = a->teacher_values.ptr;
    n.teacher_indices = (const int32_t *)a->teacher_indices.ptr;
    if (!grad) v.column("loss", a->loss, true, true, &n.sloss, n.loss);
    v.column("peak", a->peak, !grad, grad, &n.speak, n.peak);
    v.column("logsum", a->logsum, !grad, grad, &n.slogsum, n.logsum);
    v.column("tail", a->tail, !grad, false, &n.stail, n.tail);
    if (v.c.status == EWF_OK && !grad && present(a->dloss) && !present(a->dlogits)) { set_error("dloss comes with dlogits"); return EWF_EINVAL; }
    v.column("dloss", a->dloss, false, false, &n.sdloss, n.dloss);
    v.full("dlogits", a->dlogits, true, grad, &n.sdlogits);
    n.dlogits = a->dlogits.ptr;
    v.c.check_results({{"dlogits", "logits"}});
    ewf_status st = v.end();
    if (st == EWF_OK) plan_vocab(n, device_cu_count());
    return st;
}

// The parts of rows that several workgroups share, their largest logits, and what a gradient in a launch of its own needs.
size_t vocab_workspace(VocabLaunch &n, void *workspace)
{
    size_t bytes = 0;
    auto take = [&](size_t more) {
        void *at = workspace ? (char *)workspace + bytes : nullptr;
        bytes += (more + 15) / 16 * 16;
        return at;
    };
    const size_t rows = n.r.rows, parts = rows * (size_t)n.splits;
    if (n.splits > 1 || n.top) n.parts = (float *)take(parts * 4 * sizeof(float));
    if (n.pieces_per_part) n.pieces = (float *)take(parts * (size_t)n.pieces_per_part * sizeof(float));
    if (n.entries && n.dlogits && !n.held) n.prepared = take(rows * (kPreparedBytes + (size_t)n.entries * kPreparedEntryBytes));
    return bytes;
}

}  // namespace

extern "C" {

ewf_status ewf_token_logprobs_workspace(const ewf_token_logprobs_args *a, size_t *workspace_bytes)
{
    return guarded([&]() -> ewf_status {
        if (!workspace_bytes) { set_error("null argument"); return EWF_EINVAL; }
        VocabLaunch n;
        ewf_status st = logprobs_layout(a, false, n);
        if (st == EWF_OK) *workspace_bytes = vocab_workspace(n, nullptr);
        return st;
    });
}

ewf_status ewf_token_logprobs(const ewf_token_logprobs_args *a, void *workspace, size_t workspace_bytes, void *hip_stream)
{
    return guarded([&]() -> ewf_status {
        VocabLaunch n;
        ewf_status st = logprobs_layout(a, false, n);
        if (st != EWF_OK) return st;
        st = workspace_fits(vocab_workspace(n, workspace), workspace, workspace_bytes);
        if (st != EWF_OK || n.r.rows == 0) return st;
        return launched("log probabilities", [&] { launch_token_logprobs(n, (hipStream_t)hip_stream); });
    });
}

ewf_status ewf_token_logprobs_grad(const ewf_token_logprobs_args *a, void *hip_stream)
{
    return guarded([&]() -> ewf_status {
        VocabLaunch n;
        ewf_status st = logprobs_layout(a, true, n);
        if (st != EWF_OK || n.r.rows == 0) return st;
        return launched("log probabilities, backward", [&] { launch_token_logprobs_grad(n, (hipStream_t)hip_stream); });
    });
}

ewf_status ewf_distill_workspace(const ewf_distill_args *a, size_t *workspace_bytes)
{
    return guarded([&]() -> ewf_status {
        if (!workspace_bytes) { set_error("null argument"); return EWF_EINVAL; }
        VocabLaunch n;
        ewf_status st = distill_layout(a, false, n);
        if (st == EWF_OK) *workspace_bytes = vocab_workspace(n, nullptr);
        return st;
    });
}

ewf_status ewf_distill(const ewf_distill_args *a, void *workspace, size_t workspace_bytes, void *hip_stream)
{
    return guarded([&]() -> ewf_status {
        VocabLaunch n;
        ewf_status st = distill_layout(a, false, n);
        if (st != EWF_OK) return st;
        st = workspace_fits(vocab_workspace(n, workspace), workspace, workspace_bytes);
        if (st != EWF_OK || n.r.rows == 0) return st;
        return launched("distillation", [&] { launch_distill(n, (hipStream_t)hip_stream); });
    });
}

ewf_status ewf_distill_grad_workspace(const ewf_distill_args *a, size_t *workspace_bytes)
{
    return guarded([&]() -> ewf_status {
        if (!workspace_bytes) { set_error("null argument"); return EWF_EINVAL; }
        VocabLaunch n;
        ewf_status st = distill_layout(a, true, n);
        if (st == EWF_OK) *workspace_bytes = vocab_workspace(n, nullptr);
        return st;
    });
}

ewf_status ewf_distill_grad(const ewf_distill_args *a, void *workspace, size_t workspace_bytes, void *hip_stream)
{
    return guarded([&]() -> ewf_status {
        VocabLaunch n;
        ewf_status st = distill_layout(a, true, n);
        if (st != EWF_OK) return st;
        st = workspace_fits(vocab_workspace(n, workspace), workspace, workspace_bytes);
        if (st != EWF_OK || n.r.rows == 0) return st;
        return launched("distillation, backward", [&] { launch_distill_grad(n, (hipStream_t)hip_stream); });
    });
}

ewf_status ewf_layer_norm(const ewf_layer_norm_args *a, void *hip_stream)
{
    return guarded([&]() -> ewf_status {
        NormLaunch n;
        ewf_status st = norm_layout(a, false, n);
        if (st != EWF_OK) return st;
        if (n.r.rows == 0) return EWF_OK;
        return launched("layer normalisation", [&] { launch_layer_norm(n, device_cu_count(), (hipStream_t)hip_stream); });
    });
}

ewf_status ewf_layer_norm_grad_workspace(const ewf_layer_norm_args *a, size_t *workspace_bytes)
{
    return guarded([&]() -> ewf_status {
        if (!workspace_bytes) { set_error("null argument"); return EWF_EINVAL; }
        NormLaunch n;
        ewf_status st = norm_layout(a, true, n);
        if (st == EWF_OK) *workspace_bytes = norm_workspace(n);
        return st;
    });
}

ewf_status ewf_layer_norm_grad(const ewf_layer_norm_args *a, void *workspace, size_t workspace_bytes, void *hip_stream)
{
    return guarded([&]() -> ewf_status {
        NormLaunch n;
        ewf_status st = norm_layout(a, true, n);
        if (st != EWF_OK) return st;
        const size_t need = norm_workspace(n);
        st = workspace_fits(need, workspace, workspace_bytes);
        if (st != EWF_OK) return st;
        if (n.r.rows == 0 && !n.dweight && !n.dbias) return EWF_OK;
        // (a workspace that the call does not need is not looked at, neither its size nor its alignment, and not written)
        n.partials = need ? (float *)workspace : nullptr;
        return launched("layer normalisation, backward", [&] { launch_layer_norm_grad(n, (hipStream_t)hip_stream); });
    });
}

ewf_status ewf_activation(const ewf_activation_args *a, void *hip_stream)
{
    return guarded([&]() -> ewf_status {
        ActLaunch n;
        ewf_status st = act_layout(a, ActCall::Forward, n);
        if (st != EWF_OK) return st;
        if (n.r.rows == 0 || n.r.cols == 0) return EWF_OK;
        return launched("activation", [&] { launch_activation(n, (hipStream_t)hip_stream); });
    });
}

ewf_status ewf_activation_grad(const ewf_activation_args *a, void *hip_stream)
{
    return guarded([&]() -> ewf_status {
        ActLaunch n;
        ewf_status st = act_layout(a, ActCall::Grad, n);
        if (st != EWF_OK) return st;
        if (n.r.rows == 0 || n.r.cols == 0) return EWF_OK;
        return launched("activation, backward", [&] { launch_activation_grad(n, (hipStream_t)hip_stream); });
    });
}

ewf_status ewf_read8(const ewf_activation_args *a, void *hip_stream)
{
    return guarded([&]() -> ewf_status {
        ActLaunch n;
        ewf_status st = act_layout(a, ActCall::Read, n);
        if (st != EWF_OK) return st;
        if (n.r.rows == 0 || n.r.cols == 0) return EWF_OK;
        return launched("reading 8 bits", [&] { launch_read8(n, (hipStream_t)hip_stream); });
    });
}

ewf_status ewf_recurrence_workspace(const ewf_recurrence_args *a, size_t *workspace_bytes)
{
    return guarded([&]() -> ewf_status { return rec_workspace(a, false, workspace_bytes); });
}

ewf_status ewf_recurrence(const ewf_recurrence_args *a, void *workspace, size_t workspace_bytes, void *hip_stream)
{
    return guarded([&]() -> ewf_status { return rec_run(a, false, workspace, workspace_bytes, hip_stream); });
}

ewf_status ewf_recurrence_grad_workspace(const ewf_recurrence_args *a, size_t *workspace_bytes)
{
    return guarded([&]() -> ewf_status { return rec_workspace(a, true, workspace_bytes); });
}

ewf_status ewf_recurrence_grad(const ewf_recurrence_args *a, void *workspace, size_t workspace_bytes, void *hip_stream)
{
    return guarded([&]() -> ewf_status { return rec_run(a, true, workspace, workspace_bytes, hip_stream); });
}

}  // extern "C"
