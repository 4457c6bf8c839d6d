// Attention over the paged 8-bit key/value cache.
#include "entro_kv_attention.cuh"

#include "entro_kv_tokens.cuh"

namespace entro {
namespace {

// One warp per row and query head, token after token: a lane holds dim / 32 of the values.
template <typename T, int kDim>
__global__ void __launch_bounds__(128) attention_simple_kernel(Kv kv, KvBatch batch, Query qq)
{
    constexpr int kPer = kDim / 32;
    const uint32_t row = blockIdx.x, lane = threadIdx.x & 31u, head = blockIdx.y * 4u + (threadIdx.x >> 5);
    int b = (int)row;
    if (batch.row_start) b = block_find(batch.n, row, [&](uint32_t i) { return (uint32_t)batch.first(i); });
    if (head >= qq.heads || b < 0 || (int)row >= batch.first(b) + batch.count(b)) return;
    const int slot = batch.slot(b, kv.slots);
    const int len = slot >= 0 ? __ldg(kv.lens + slot) : 0;
    const int position = len - batch.count(b) + ((int)row - batch.first(b));
    const uint32_t kv_head = head / qq.group;
    float q[kPer], o[kPer];
    const T* qp = (const T*)(qq.q + row * qq.q_row + head * qq.q_head);
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        q[i] = (float)qp[lane + 32 * i];
        o[i] = 0.f;
    }
    float top = -INFINITY, sum = 0.f;
    for (int j = 0; j <= position; ++j) {
        if (qq.window && (int64_t)j <= (int64_t)position - qq.window && (uint32_t)j >= qq.sinks) continue;
        const int page = kv_page(kv, slot, (uint32_t)j >> kv.page_shift);
        if (page < 0) continue;
        const uint8_t* k = kv.codes + (uint64_t)page * kv.page_bytes() + kv_head * kv.head_bytes() +
                           ((uint32_t)j & (kv.page() - 1u)) * kDim;
        const uint8_t* v = k + kv.heads * kv.head_bytes();
        const float ks = kv.scales[(uint64_t)page * 2u * kv.heads + kv_head];
        const float vs = kv.scales[((uint64_t)page * 2u + 1u) * kv.heads + kv_head];
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < kPer; ++i) s = fmaf(q[i], (float)((int)k[lane + 32 * i] - ENTRO_KV_ZERO_POINT), s);
#pragma unroll
        for (int m = 16; m; m >>= 1) s += __shfl_xor_sync(0xffffffffu, s, m);
        s *= ks * qq.scale;
        const float up = fmaxf(top, s);
        const float keep = top == up ? 1.f : expf(top - up), p = expf(s - up);
        sum = sum * keep + p;
        top = up;
#pragma unroll
        for (int i = 0; i < kPer; ++i)
            o[i] = o[i] * keep + p * vs * (float)((int)v[lane + 32 * i] - ENTRO_KV_ZERO_POINT);
    }
    T* op = (T*)(qq.out + row * qq.out_row + head * qq.out_head);
#pragma unroll
    for (int i = 0; i < kPer; ++i) op[lane + 32 * i] = (T)(sum == 0.f ? 0.f : o[i] / sum);
    if (qq.lse && lane == 0) qq.lse[(uint64_t)row * qq.heads + head] = sum == 0.f ? -INFINITY : top + logf(sum);
}

template <typename T>
entro_status launch_attention(const Kv& kv, const KvBatch& batch, const Query& q, uint32_t max_rows, cudaStream_t s)
{
    Workspace* ws;
    {
        Guard g;
        ws = workspace();
    }
    if (!ws) return ENTRO_ERR_CUDA;
    const uint64_t rows = (uint64_t)(batch.row_start ? (max_rows ? max_rows : batch.rows) : 1u) * q.group;
    if (rows <= kTokenRows) {
        float* partials = (float*)kv.region;
        cudaError_t e = kv.dim == 64   ? launch_tokens<T, 64>(kv, batch, q, (uint32_t)rows, (uint32_t)ws->sm_count, partials, s)
                        : kv.dim == 96 ? launch_tokens<T, 96>(kv, batch, q, (uint32_t)rows, (uint32_t)ws->sm_count, partials, s)
                                       : launch_tokens<T, 128>(kv, batch, q, (uint32_t)rows, (uint32_t)ws->sm_count, partials, s);
        ENTRO_CUDA(e);
    } else {
        const dim3 grid(batch.rows, (q.heads + 3u) / 4u);
        if (kv.dim == 64)
            attention_simple_kernel<T, 64><<<grid, 128, 0, s>>>(kv, batch, q);
        else if (kv.dim == 96)
            attention_simple_kernel<T, 96><<<grid, 128, 0, s>>>(kv, batch, q);
        else
            attention_simple_kernel<T, 128><<<grid, 128, 0, s>>>(kv, batch, q);
        ENTRO_CUDA(cudaGetLastError());
    }
    count_launch();
    return ENTRO_OK;
}

}  // namespace
}  // namespace entro

using namespace entro;

extern "C" entro_status entro_kv_attention(const entro_kv_cache* cache, const entro_kv_batch* b, const entro_kv_query* a,
                                           void* cuda_stream)
{
    Kv kv;
    KvBatch batch;
    if (entro_status e = kv_check(cache, &kv)) return e;
    if (entro_status e = kv_check(cache, b, &batch)) return e;
    if (batch.n == 0 || batch.rows == 0) return ENTRO_OK;
    if (!a || !a->q_dev || !a->out_dev || !aligned(a->q_dev, 16) || !aligned(a->out_dev, 16) || !aligned(a->lse_dev, 4))
        return ENTRO_ERR_INVALID_ARG;
    if (a->type != ENTRO_FLOAT16 && a->type != ENTRO_BFLOAT16) return ENTRO_ERR_INVALID_ARG;
    if (!kv_strides_ok(a->q_row_stride, a->q_head_stride) || !kv_strides_ok(a->out_row_stride, a->out_head_stride))
        return ENTRO_ERR_INVALID_ARG;
    if (a->q_heads == 0 || a->q_heads % kv.heads || a->q_heads > 65536u) return ENTRO_ERR_INVALID_ARG;
    if (!(a->softmax_scale >= 0.f && a->softmax_scale <= 3.4e38f)) return ENTRO_ERR_INVALID_ARG;
    Query q;
    q.q = (const unsigned char*)a->q_dev;
    q.out = (unsigned char*)a->out_dev;
    q.lse = a->lse_dev;
    q.q_row = 2 * a->q_row_stride;
    q.q_head = 2 * a->q_head_stride;
    q.out_row = 2 * a->out_row_stride;
    q.out_head = 2 * a->out_head_stride;
    q.heads = a->q_heads;
    q.group = a->q_heads / kv.heads;
    q.window = a->window;
    q.sinks = a->sinks;
    q.scale = a->softmax_scale > 0.f ? a->softmax_scale : 1.f / sqrtf((float)kv.dim);
    return a->type == ENTRO_FLOAT16 ? launch_attention<__half>(kv, batch, q, a->max_rows, (cudaStream_t)cuda_stream)
                                    : launch_attention<__nv_bfloat16>(kv, batch, q, a->max_rows, (cudaStream_t)cuda_stream);
}
