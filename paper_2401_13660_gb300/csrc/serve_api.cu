// C ABI of decoding on 8-bit projections and of drawing tokens: host-side
// validation, then the launches on the caller's stream. Declarations and the
// contract of every entry point are in include/mbscan.h.
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/mbscan.h"
#include "checks.h"
#include "internal.h"
#include "matmul_plan.h"

using mbscan::aligned16;
using mbscan::from_cuda;
using mbscan::kMaxTokens;
using mbscan::kQuantBlock;
using mbscan::overlap;
using mbscan::Range;
using mbscan::range_of;

namespace {

int64_t elem_size(int32_t dtype) { return dtype == MB_BF16 ? 2 : 4; }
bool dtype_ok(int32_t dtype) { return dtype == MB_F32 || dtype == MB_BF16; }
bool aligned_to(const void *p, int64_t size) { return reinterpret_cast<uintptr_t>(p) % (uintptr_t)size == 0; }

// Sizes of a matrix in 8 bits.
mb_status check_size(int64_t rows, int64_t width) {
    if (rows < 0 || width < 0 || rows > kMaxTokens || width > kMaxTokens) return MB_ERR_INVALID_ARG;
    if (width % 16 != 0) return MB_ERR_UNSUPPORTED;
    if (width > 0 && rows > kMaxTokens / width) return MB_ERR_INVALID_ARG;
    return MB_OK;
}
int64_t scale_rows(int64_t rows, int32_t block_rows) { return (rows + block_rows - 1) / block_rows; }
bool block_rows_ok(int32_t block_rows) { return block_rows == 1 || block_rows == kQuantBlock; }

// Sizes of a product of two of them, and its type.
mb_status check_product(int64_t rows, int64_t n_out, int64_t width, int32_t out_dtype) {
    for (const int64_t n : {rows, n_out})
        if (const mb_status st = check_size(n, width); st != MB_OK) return st;
    if (!dtype_ok(out_dtype)) return MB_ERR_INVALID_ARG;
    if (n_out % 8 != 0) return MB_ERR_UNSUPPORTED;
    if (n_out > 0 && rows > kMaxTokens / n_out) return MB_ERR_INVALID_ARG;
    return MB_OK;
}

Range scales_range(const void *scales, int64_t rows, int32_t block_rows, int64_t width) {
    return range_of(scales, scale_rows(rows, block_rows) * mbscan::quant_stride(width));
}

// Whether no range of `outs` shares memory with another of them or with one of `ins`.
template <int kO, int kI> bool apart(const Range (&outs)[kO], const Range (&ins)[kI]) {
    for (int i = 0; i < kO; ++i) {
        for (int j = 0; j < kI; ++j)
            if (overlap(outs[i], ins[j])) return false;
        for (int j = i + 1; j < kO; ++j)
            if (overlap(outs[i], outs[j])) return false;
    }
    return true;
}

}  // namespace

extern "C" {

int64_t mb_q8_scale_stride(int64_t width) {
    return width < 0 || width > kMaxTokens || width % 16 != 0 ? 0 : mbscan::quant_stride(width);
}

mb_status mb_rmsnorm_q8(const void *add, int32_t dtype, float *residual, const float *w, float eps, uint8_t *q, uint8_t *scales,
                        int64_t rows, int64_t width, void *stream) {
    if (const mb_status st = check_size(rows, width); st != MB_OK) return st;
    if (!dtype_ok(dtype)) return MB_ERR_INVALID_ARG;
    if (rows * width == 0) return MB_OK;
    if (!(eps >= 0.f)) return MB_ERR_INVALID_ARG;
    if (!residual || !w || !q || !scales) return MB_ERR_INVALID_ARG;
    if (!aligned16(residual) || !aligned16(w) || !aligned16(q) || !aligned16(add) || !aligned_to(scales, 4)) return MB_ERR_INVALID_ARG;
    const Range outs[] = {range_of(residual, rows * width * 4), range_of(q, rows * width), scales_range(scales, rows, 1, width)};
    const Range ins[] = {range_of(add, rows * width * elem_size(dtype)), range_of(w, width * 4)};
    if (!apart(outs, ins)) return MB_ERR_INVALID_ARG;
    return from_cuda(mbscan::launch_rmsnorm_q8(add, dtype == MB_BF16, residual, w, eps, q, scales, rows, width, (cudaStream_t)stream));
}

mb_status mb_quantize_q8(const void *x, int32_t dtype, int64_t x_stride, int32_t block_rows, uint8_t *q, uint8_t *scales,
                         int64_t rows, int64_t width, void *stream) {
    if (const mb_status st = check_size(rows, width); st != MB_OK) return st;
    if (!dtype_ok(dtype) || !block_rows_ok(block_rows)) return MB_ERR_INVALID_ARG;
    const int64_t es = elem_size(dtype), stride = x_stride ? x_stride : width;
    if (stride < width || stride > INT32_MAX || (stride * es) % 16 != 0) return MB_ERR_INVALID_ARG;
    if (rows * width == 0) return MB_OK;
    if (!x || !q || !scales || !aligned16(x) || !aligned16(q) || !aligned_to(scales, 4)) return MB_ERR_INVALID_ARG;
    const Range outs[] = {range_of(q, rows * width), scales_range(scales, rows, block_rows, width)};
    const Range ins[] = {range_of(x, ((rows - 1) * stride + width) * es)};
    if (!apart(outs, ins)) return MB_ERR_INVALID_ARG;
    return from_cuda(mbscan::launch_quantize(x, dtype == MB_BF16, stride, block_rows != 1, q, scales, rows, width, (cudaStream_t)stream));
}

mb_status mb_dequantize_q8(const uint8_t *q, const uint8_t *scales, int32_t block_rows, void *out, int32_t dtype, int64_t rows,
                           int64_t width, void *stream) {
    if (const mb_status st = check_size(rows, width); st != MB_OK) return st;
    if (!dtype_ok(dtype) || !block_rows_ok(block_rows)) return MB_ERR_INVALID_ARG;
    if (rows * width == 0) return MB_OK;
    if (!q || !scales || !out || !aligned16(q) || !aligned16(out) || !aligned_to(scales, 4)) return MB_ERR_INVALID_ARG;
    const Range outs[] = {range_of(out, rows * width * elem_size(dtype))};
    const Range ins[] = {range_of(q, rows * width), scales_range(scales, rows, block_rows, width)};
    if (!apart(outs, ins)) return MB_ERR_INVALID_ARG;
    return from_cuda(mbscan::launch_dequantize(q, scales, block_rows != 1, out, dtype == MB_BF16, rows, width, (cudaStream_t)stream));
}

mb_status mb_matmul_q8(const uint8_t *a, const uint8_t *a_scales, const uint8_t *w, const uint8_t *w_scales, void *out,
                       int32_t out_dtype, int64_t rows, int64_t n_out, int64_t width, int64_t part, void *ws, size_t ws_bytes,
                       void *stream) {
    if (const mb_status st = check_product(rows, n_out, width, out_dtype); st != MB_OK) return st;
    if (part == 0) part = n_out;
    if (part != n_out && (part < 0 || part % kQuantBlock != 0 || n_out % part != 0)) return MB_ERR_INVALID_ARG;
    if (ws && (ws_bytes < mbscan::kStatusBytes || (reinterpret_cast<uintptr_t>(ws) & 255u) != 0)) return MB_ERR_INVALID_ARG;
    if (rows * n_out == 0) return MB_OK;
    const int64_t es = elem_size(out_dtype);
    if (!out || !aligned16(out)) return MB_ERR_INVALID_ARG;
    if (width == 0) return from_cuda(cudaMemsetAsync(out, 0, (size_t)(rows * n_out * es), (cudaStream_t)stream));   // a sum of nothing
    if (!a || !a_scales || !w || !w_scales) return MB_ERR_INVALID_ARG;
    if (!aligned16(a) || !aligned16(w) || !aligned_to(a_scales, 4) || !aligned_to(w_scales, 4)) return MB_ERR_INVALID_ARG;
    const Range outs[] = {range_of(out, rows * n_out * es), range_of(ws, mbscan::kStatusBytes)};
    const Range ins[] = {range_of(a, rows * width), scales_range(a_scales, rows, 1, width), range_of(w, n_out * width),
                         scales_range(w_scales, n_out, kQuantBlock, width)};
    if (!apart(outs, ins)) return MB_ERR_INVALID_ARG;
    mbscan::MatmulParams p{a, a_scales, w, w_scales, out, rows, n_out, width, part, static_cast<mbscan::StatusBlock *>(ws)};
    return from_cuda(mbscan::launch_matmul_q8(p, out_dtype == MB_BF16, (cudaStream_t)stream));
}

mb_status mb_matmul_q8_form(int64_t rows, int64_t n_out, int64_t width, int32_t out_dtype, int64_t form[5]) {
    if (!form) return MB_ERR_INVALID_ARG;
    if (const mb_status st = check_product(rows, n_out, width, out_dtype); st != MB_OK) return st;
    for (int i = 0; i < 5; ++i) form[i] = 0;
    if (rows * n_out == 0 || width == 0) return MB_OK;   // no product runs
    mbscan::MatmulPlan p;
    if (!mbscan::plan_matmul_here(rows, n_out, width, out_dtype == MB_BF16, &p)) return MB_ERR_CUDA;
    const int64_t tiles = (int64_t)p.t.features * p.t.rows;
    const int64_t v[5] = {p.ctas, p.t.split, p.t.height, p.t.deep, (tiles + p.teams - 1) / p.teams};
    for (int i = 0; i < 5; ++i) form[i] = v[i];
    return MB_OK;
}

mb_status mb_sample(const void *logits, int32_t dtype, const float *u, const float *temperature, const int32_t *top_k,
                    const float *top_p, const float *min_p, void *tokens, int32_t token_type, float *prob, int64_t n,
                    int64_t vocab, void *stream) {
    if (!dtype_ok(dtype) || (token_type != MB_TOKEN_I32 && token_type != MB_TOKEN_I64)) return MB_ERR_INVALID_ARG;
    if (n < 0 || n > kMaxTokens || vocab < 1 || vocab > kMaxTokens / 2 || n > kMaxTokens / vocab) return MB_ERR_INVALID_ARG;
    if (n == 0) return MB_OK;
    const int64_t ts = token_type == MB_TOKEN_I64 ? 8 : 4;
    if (!logits || !u || !tokens) return MB_ERR_INVALID_ARG;
    if (!aligned16(logits) || !aligned_to(tokens, ts)) return MB_ERR_INVALID_ARG;
    for (const void *p : {static_cast<const void *>(u), static_cast<const void *>(temperature), static_cast<const void *>(top_k),
                          static_cast<const void *>(top_p), static_cast<const void *>(min_p), static_cast<const void *>(prob)})
        if (!aligned_to(p, 4)) return MB_ERR_INVALID_ARG;
    const Range outs[] = {range_of(tokens, n * ts), range_of(prob, n * 4)};
    const Range ins[] = {range_of(logits, n * vocab * elem_size(dtype)), range_of(u, n * 4), range_of(temperature, n * 4),
                         range_of(top_k, n * 4), range_of(top_p, n * 4), range_of(min_p, n * 4)};
    if (!apart(outs, ins)) return MB_ERR_INVALID_ARG;
    mbscan::SampleParams p{logits, u, temperature, top_k, top_p, min_p, tokens, token_type == MB_TOKEN_I64, prob, n, (int)vocab};
    return from_cuda(mbscan::launch_sample(p, dtype == MB_BF16, (cudaStream_t)stream));
}

}  // extern "C"
