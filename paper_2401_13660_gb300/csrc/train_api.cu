// C ABI of the operators that a training step runs around the scan: host-side
// validation, then the launches on the caller's stream. Declarations and the
// contract of every entry point are in include/mbscan.h.
#include <cuda_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <memory>
#include <new>

#include "../../include/mbscan.h"
#include "checks.h"
#include "internal.h"

using mbscan::aligned16;
using mbscan::from_cuda;
using mbscan::kMaxTokens;
using mbscan::overlap;
using mbscan::Range;
using mbscan::range_of;

namespace {

int64_t elem_size(int32_t dtype) { return dtype == MB_BF16 ? 2 : 4; }

// Bytes spanned by `rows` rows of `width` elements, `stride` elements apart.
int64_t strided_bytes(int64_t rows, int64_t width, int64_t stride, int64_t es) {
    return rows > 0 && width > 0 ? ((rows - 1) * stride + width) * es : 0;
}

// A row stride in elements: 0 (contiguous), or at least the width and whole 16-byte groups.
bool stride_ok(int64_t stride, int64_t width, int64_t es) {
    return stride == 0 || (stride >= width && stride <= INT32_MAX && (stride * es) % 16 == 0);
}

// Scratch of a workspace: what follows its status block.
bool ws_ok(const void *ws, size_t ws_bytes, size_t need) {
    return ws != nullptr && ws_bytes >= need && (reinterpret_cast<uintptr_t>(ws) & 255u) == 0;
}
template <typename P> P *scratch_of(void *ws) {
    return reinterpret_cast<P *>(static_cast<char *>(ws) + mbscan::kStatusBytes);
}

// Sizes and strides of a convolution: sets *any when there is something to do.
mb_status check_conv(const mb_conv1d_args *a, bool *any) {
    *any = false;
    if (!a || a->batch < 0 || a->seqlen < 0 || a->width < 0) return MB_ERR_INVALID_ARG;
    if (a->batch > kMaxTokens || a->seqlen > kMaxTokens || a->width > kMaxTokens) return MB_ERR_INVALID_ARG;
    if (a->dtype != MB_F32 && a->dtype != MB_BF16) return MB_ERR_INVALID_ARG;
    if (a->width % 8 != 0) return MB_ERR_UNSUPPORTED;
    if (!stride_ok(a->x_stride, a->width, elem_size(a->dtype))) return MB_ERR_INVALID_ARG;
    if (a->batch * a->width == 0) return MB_OK;
    if (a->batch > kMaxTokens / a->width) return MB_ERR_INVALID_ARG;
    if (a->seqlen > 0 && a->batch * a->width > kMaxTokens / a->seqlen) return MB_ERR_INVALID_ARG;
    if ((a->seqlen > 0 && !a->x) || !a->w) return MB_ERR_INVALID_ARG;
    for (const void *p : {a->x, a->state, static_cast<const void *>(a->w), static_cast<const void *>(a->bias)})
        if (!aligned16(p)) return MB_ERR_INVALID_ARG;
    *any = true;
    return MB_OK;
}

mbscan::ConvParams to_conv(const mb_conv1d_args *a) {
    mbscan::ConvParams p{};
    p.batch = a->batch; p.seqlen = a->seqlen; p.width = a->width;
    p.x_stride = a->x_stride ? a->x_stride : a->width;
    p.x = a->x; p.state = a->state; p.w = a->w; p.bias = a->bias;
    return p;
}

bool dtype_ok(int32_t dtype) { return dtype == MB_F32 || dtype == MB_BF16; }

// Bytes of a token id; 0 for a type that is none.
int64_t token_size(int32_t type) {
    return type == MB_TOKEN_U8 ? 1 : type == MB_TOKEN_I32 ? 4 : type == MB_TOKEN_I64 ? 8 : 0;
}
bool aligned_to(const void *p, int64_t size) { return reinterpret_cast<uintptr_t>(p) % (uintptr_t)size == 0; }

constexpr int64_t kMaxEmbedWidth = (int64_t)1 << 20;

mb_status check_embed(int64_t n, int64_t vocab, int64_t width) {
    if (n < 0 || vocab < 0 || width < 0 || n > kMaxTokens || vocab >= kMaxTokens) return MB_ERR_INVALID_ARG;
    if (width % 8 != 0 || width > kMaxEmbedWidth) return MB_ERR_UNSUPPORTED;
    if (width > 0 && (n > kMaxTokens / width || vocab > kMaxTokens / width)) return MB_ERR_INVALID_ARG;
    return MB_OK;
}

constexpr int64_t kMaxNumel = (int64_t)1 << 40;

mb_status check_list(const mb_tensor *list, int64_t count) {
    if (count < 0 || (count > 0 && !list)) return MB_ERR_INVALID_ARG;
    for (int64_t i = 0; i < count; ++i) {
        const mb_tensor &t = list[i];
        if (t.numel < 0 || t.numel > kMaxNumel || !dtype_ok(t.dtype) || t.reserved != 0) return MB_ERR_INVALID_ARG;
        if (t.numel > 0 && (!t.data || !aligned_to(t.data, elem_size(t.dtype)))) return MB_ERR_INVALID_ARG;
    }
    return MB_OK;
}
Range tensor_range(const mb_tensor &t) { return range_of(t.data, t.numel * elem_size(t.dtype)); }

// Outputs that lie in the order of the list, those of each type by themselves, and away from everything else, as slices of
// one buffer per type do: a look at every tensor shows it (532 tensors 0.8 us of a call, sorted and searched 5).
bool plainly_apart(const mb_tensor *list, const mb_tensor *out, int64_t count) {
    Range all[2] = {};   // of the outputs of a type
    for (int64_t i = 0; i < count; ++i) {
        if (out[i].numel == 0) continue;
        const Range r = tensor_range(out[i]);
        Range &a = all[out[i].dtype == MB_BF16];
        if (r.lo < a.hi) return false;
        if (a.lo == 0) a.lo = r.lo;
        a.hi = r.hi;
    }
    if (overlap(all[0], all[1])) return false;
    for (int64_t i = 0; i < count; ++i) {
        if (list[i].numel == 0 || (out[i].data == list[i].data && out[i].dtype == list[i].dtype)) continue;
        const Range r = tensor_range(list[i]);
        if (overlap(r, all[0]) || overlap(r, all[1])) return false;
    }
    return true;
}

// Whether each out[i] shares no memory with another output, nor with any tensor of the list but list[i] where it is
// list[i] itself.
mb_status check_apart(const mb_tensor *list, const mb_tensor *out, int64_t count) {
    if (plainly_apart(list, out, count)) return MB_OK;
    constexpr int64_t kFew = 128;
    Range few[kFew];
    std::unique_ptr<Range[]> many;
    if (count > kFew) {
        many.reset(new (std::nothrow) Range[count]);
        if (!many) return MB_ERR_CUDA;   // out of host memory
    }
    Range *const outs = count > kFew ? many.get() : few;
    Range *end = outs;
    for (int64_t i = 0; i < count; ++i)
        if (out[i].numel > 0) *end++ = tensor_range(out[i]);
    std::sort(outs, end, [](const Range &a, const Range &b) { return a.lo < b.lo; });
    for (Range *r = outs; r + 1 < end; ++r)
        if (r->hi > r[1].lo) return MB_ERR_INVALID_ARG;
    for (int64_t i = 0; i < count; ++i) {
        if (list[i].numel == 0 || (out[i].data == list[i].data && out[i].dtype == list[i].dtype)) continue;
        const Range in = tensor_range(list[i]);
        const Range *r = std::upper_bound(outs, end, in.lo, [](uintptr_t lo, const Range &o) { return lo < o.hi; });
        if (r < end && r->lo < in.hi) return MB_ERR_INVALID_ARG;
    }
    return MB_OK;
}

}  // namespace

extern "C" {

mb_status mb_conv1d(const mb_conv1d_args *args, void *out, void *state_out, void *stream) {
    bool any;
    if (const mb_status st = check_conv(args, &any); st != MB_OK || !any) return st;
    if ((args->seqlen > 0 && !out) || !aligned16(out) || !aligned16(state_out)) return MB_ERR_INVALID_ARG;
    const int64_t es = elem_size(args->dtype), rows = args->batch * args->seqlen;
    mbscan::ConvParams p = to_conv(args);
    const int64_t window = 3 * args->batch * args->width * es;
    const Range ro = range_of(out, rows * args->width * es), rw = range_of(state_out, window);
    const Range ins[] = {range_of(args->x, strided_bytes(rows, args->width, p.x_stride, es)),
                         range_of(args->w, args->width * 16), range_of(args->bias, args->width * 4)};
    const Range rs = range_of(args->state, window);
    for (const Range &r : ins)
        if (overlap(ro, r) || overlap(rw, r)) return MB_ERR_INVALID_ARG;
    if (overlap(ro, rw) || overlap(ro, rs) || (state_out != args->state && overlap(rw, rs))) return MB_ERR_INVALID_ARG;
    if (args->seqlen == 0 && !state_out) return MB_OK;
    p.out = out;
    p.state_out = state_out;
    return from_cuda(mbscan::launch_conv(p, args->dtype == MB_BF16, (cudaStream_t)stream));
}

size_t mb_conv1d_backward_workspace_size(int64_t batch, int64_t seqlen, int64_t width) {
    mb_conv1d_args a{};
    a.batch = batch; a.seqlen = seqlen; a.width = width;
    a.x = a.w = reinterpret_cast<const float *>(mbscan::kStatusBytes);   // only the sizes are looked at
    bool any;
    if (check_conv(&a, &any) != MB_OK) return 0;
    return mbscan::kStatusBytes + (any ? mbscan::conv_backward_scratch(batch, seqlen, width) : 0);
}

mb_status mb_conv1d_backward(const mb_conv1d_args *args, const void *dout, const void *dstate_out,
                             const mb_conv1d_grads *grads, void *ws, size_t ws_bytes, void *stream) {
    bool any;
    if (const mb_status st = check_conv(args, &any); st != MB_OK) return st;
    if (!grads) return MB_ERR_INVALID_ARG;
    const int64_t es = elem_size(args->dtype), rows = args->batch * args->seqlen, width = args->width;
    const mb_conv1d_grads &g = *grads;
    if (!stride_ok(g.dx_stride, width, es)) return MB_ERR_INVALID_ARG;
    if (width == 0) return MB_OK;
    if (!g.dw || (rows > 0 && (!dout || !g.dx))) return MB_ERR_INVALID_ARG;
    for (const void *q : {dout, dstate_out, static_cast<const void *>(g.dx), static_cast<const void *>(g.dstate),
                          static_cast<const void *>(g.dw), static_cast<const void *>(g.dbias)})
        if (!aligned16(q)) return MB_ERR_INVALID_ARG;
    mbscan::ConvParams p = to_conv(args);
    p.dx_stride = g.dx_stride ? g.dx_stride : width;
    p.dout = dout; p.dstate_out = dstate_out;
    p.dx = g.dx; p.dstate = g.dstate; p.dw = g.dw; p.dbias = g.dbias;
    const size_t need = mb_conv1d_backward_workspace_size(args->batch, args->seqlen, width);
    if (!ws_ok(ws, ws_bytes, need)) return MB_ERR_INVALID_ARG;
    const int64_t window = 3 * args->batch * width * es;
    const Range outs[] = {range_of(g.dx, strided_bytes(rows, width, p.dx_stride, es)), range_of(g.dstate, window),
                          range_of(g.dw, width * 16), range_of(g.dbias, width * 4), range_of(ws, (int64_t)need)};
    const Range ins[] = {range_of(args->x, strided_bytes(rows, width, p.x_stride, es)), range_of(args->state, window),
                         range_of(args->w, width * 16), range_of(args->bias, width * 4),
                         range_of(dout, rows * width * es), range_of(dstate_out, window)};
    constexpr int kOuts = sizeof(outs) / sizeof(outs[0]);
    for (int i = 0; i < kOuts; ++i) {
        for (const Range &r : ins)
            if (overlap(outs[i], r)) return MB_ERR_INVALID_ARG;
        for (int j = i + 1; j < kOuts; ++j)
            if (overlap(outs[i], outs[j])) return MB_ERR_INVALID_ARG;
    }
    return from_cuda(mbscan::launch_conv_backward(p, args->dtype == MB_BF16, scratch_of<float>(ws), (cudaStream_t)stream));
}

mb_status mb_embed(const void *tokens, int32_t token_type, const void *table, int32_t table_dtype, float scale,
                   void *out, int32_t out_dtype, int64_t n, int64_t vocab, int64_t width, void *stream) {
    const int64_t ts = token_size(token_type);
    if (ts == 0 || !dtype_ok(table_dtype) || !dtype_ok(out_dtype)) return MB_ERR_INVALID_ARG;
    if (const mb_status st = check_embed(n, vocab, width); st != MB_OK) return st;
    if (n * width == 0) return MB_OK;
    if (!tokens || !out || (vocab > 0 && !table)) return MB_ERR_INVALID_ARG;
    if (!aligned_to(tokens, ts) || !aligned16(table) || !aligned16(out)) return MB_ERR_INVALID_ARG;
    const Range ro = range_of(out, n * width * elem_size(out_dtype));
    if (overlap(ro, range_of(tokens, n * ts)) || overlap(ro, range_of(table, vocab * width * elem_size(table_dtype))))
        return MB_ERR_INVALID_ARG;
    return from_cuda(mbscan::launch_embed(tokens, token_type, table, table_dtype == MB_BF16, scale, out,
                                          out_dtype == MB_BF16, n, (int)vocab, width, (cudaStream_t)stream));
}

size_t mb_embed_backward_workspace_size(int64_t n, int64_t vocab, int64_t width) {
    if (check_embed(n, vocab, width) != MB_OK) return 0;
    if (n == 0 || vocab == 0 || width == 0) return mbscan::kStatusBytes;   // nothing to sort or add
    return mbscan::kStatusBytes + mbscan::embed_backward_scratch(n, width);
}

mb_status mb_embed_backward(const void *tokens, int32_t token_type, const void *dout, int32_t dtype, float scale,
                            int32_t accumulate, float *dtable, int64_t n, int64_t vocab, int64_t width, void *ws,
                            size_t ws_bytes, void *stream) {
    const int64_t ts = token_size(token_type);
    if (ts == 0 || !dtype_ok(dtype)) return MB_ERR_INVALID_ARG;
    if (const mb_status st = check_embed(n, vocab, width); st != MB_OK) return st;
    if (vocab * width == 0) return MB_OK;
    if (!dtable || (n > 0 && (!tokens || !dout))) return MB_ERR_INVALID_ARG;
    if (!aligned_to(tokens, ts) || !aligned16(dout) || !aligned16(dtable)) return MB_ERR_INVALID_ARG;
    const size_t need = mb_embed_backward_workspace_size(n, vocab, width);
    if (!ws_ok(ws, ws_bytes, need)) return MB_ERR_INVALID_ARG;
    const Range rd = range_of(dtable, vocab * width * 4), rw = range_of(ws, (int64_t)need);
    const Range ins[] = {range_of(tokens, n * ts), range_of(dout, n * width * elem_size(dtype))};
    for (const Range &r : ins)
        if (overlap(rd, r) || overlap(rw, r)) return MB_ERR_INVALID_ARG;
    if (overlap(rd, rw)) return MB_ERR_INVALID_ARG;
    return from_cuda(mbscan::launch_embed_backward(tokens, token_type, dout, dtype == MB_BF16, scale, accumulate != 0,
                                                   dtable, n, (int)vocab, width, scratch_of<char>(ws),
                                                   (cudaStream_t)stream));
}

mb_status mb_cross_entropy(const void *logits, int32_t dtype, const void *targets, int32_t token_type,
                           const float *weight, float scale, float *loss, void *dlogits, int64_t n, int64_t vocab,
                           void *stream) {
    const int64_t ts = token_size(token_type);
    if (ts == 0 || !dtype_ok(dtype)) return MB_ERR_INVALID_ARG;
    if (n < 0 || n > kMaxTokens || vocab < 1 || vocab > kMaxTokens / 2 || n > kMaxTokens / vocab) return MB_ERR_INVALID_ARG;
    if (n == 0) return MB_OK;
    if (!logits || !targets || !loss) return MB_ERR_INVALID_ARG;
    if (!aligned16(logits) || !aligned16(dlogits) || !aligned_to(targets, ts) || !aligned_to(weight, 4) ||
        !aligned_to(loss, 4))
        return MB_ERR_INVALID_ARG;
    const int64_t bytes = n * vocab * elem_size(dtype);
    const Range rl = range_of(logits, bytes), rd = range_of(dlogits, bytes), ro = range_of(loss, n * 4);
    const Range ins[] = {range_of(targets, n * ts), range_of(weight, n * 4)};
    for (const Range &r : ins)
        if (overlap(rd, r) || overlap(ro, r)) return MB_ERR_INVALID_ARG;
    if (overlap(ro, rl) || overlap(ro, rd) || (dlogits != logits && overlap(rd, rl))) return MB_ERR_INVALID_ARG;
    return from_cuda(mbscan::launch_cross_entropy(logits, dtype == MB_BF16, targets, token_type, weight, scale, loss,
                                                  dlogits, n, (int)vocab, (cudaStream_t)stream));
}

size_t mb_grad_norm_workspace_size(void) { return mbscan::kStatusBytes + mbscan::grad_norm_scratch(); }

mb_status mb_grad_norm(const mb_tensor *list, int64_t count, float *norm, void *ws, size_t ws_bytes, void *stream) {
    if (const mb_status st = check_list(list, count); st != MB_OK) return st;
    if (!norm || !aligned_to(norm, 4)) return MB_ERR_INVALID_ARG;
    const size_t need = mb_grad_norm_workspace_size();
    if (!ws_ok(ws, ws_bytes, need)) return MB_ERR_INVALID_ARG;
    const Range rn = range_of(norm, 4), rw = range_of(ws, (int64_t)need);
    if (overlap(rn, rw)) return MB_ERR_INVALID_ARG;
    for (int64_t i = 0; i < count; ++i)
        if (overlap(tensor_range(list[i]), rn) || overlap(tensor_range(list[i]), rw)) return MB_ERR_INVALID_ARG;
    return from_cuda(mbscan::launch_grad_norm(list, count, norm, static_cast<mbscan::StatusBlock *>(ws), scratch_of<char>(ws),
                                              (cudaStream_t)stream));
}

mb_status mb_grad_clip(const mb_tensor *list, const mb_tensor *out, int64_t count, const float *norm,
                       float max_norm, void *stream) {
    if (const mb_status st = check_list(list, count); st != MB_OK) return st;
    if (!norm || !aligned_to(norm, 4) || !(max_norm > 0.f)) return MB_ERR_INVALID_ARG;
    const Range rn = range_of(norm, 4);
    if (out) {
        if (const mb_status st = check_list(out, count); st != MB_OK) return st;
        for (int64_t i = 0; i < count; ++i)
            if (out[i].numel != list[i].numel) return MB_ERR_INVALID_ARG;
    }
    if (const mb_status st = check_apart(list, out ? out : list, count); st != MB_OK) return st;
    for (int64_t i = 0; i < count; ++i)
        if (overlap(tensor_range((out ? out : list)[i]), rn)) return MB_ERR_INVALID_ARG;
    return from_cuda(mbscan::launch_grad_clip(list, out, count, norm, max_norm, (cudaStream_t)stream));
}

}  // extern "C"
