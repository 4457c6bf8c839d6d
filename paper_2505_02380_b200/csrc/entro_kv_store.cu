// Writing rows into the paged 8-bit key/value cache and reading them back.
#include "entro_kv_common.cuh"

namespace entro {
namespace {

constexpr float kScaleFloor = 8.673617379884035e-19f;   // 2^-60: no scale is 0, so the attention kernels may divide by one

struct Rows {
    const unsigned char* base[2];   // keys, values
    int64_t row[2], head[2];        // strides in bytes
};

// Work items of a ragged batch: sequence b's touched pages are items f(b) + 0, 1, ... with
// f(b) = row_start[b] / page + 2 b.  A sequence of r rows touches at most ceil((r - 1) / page) + 1
// pages, which is no more than f(b + 1) - f(b), so the places never collide and need no scan over
// lengths that only the device knows.
__host__ __device__ inline uint32_t item_of(uint32_t first_row, uint32_t b, uint32_t page_shift)
{
    return (first_row >> page_shift) + 2u * b;
}

// A work item as found by a block: the tokens [lo, hi) of one block of a sequence that are new.
struct Item {
    int page;         // -1: nothing to do
    int row0;         // row of token lo
    uint32_t lo, hi;  // inside the page
};

__device__ __forceinline__ Item find_item(const Kv& kv, const KvBatch& batch, uint32_t item)
{
    Item it;
    it.page = -1;
    int b, k = 0;
    if (batch.row_start) {
        b = block_find(batch.n, item, [&](uint32_t i) { return item_of((uint32_t)batch.first(i), i, kv.page_shift); });
        if (b < 0) return it;
        k = (int)(item - item_of((uint32_t)batch.first(b), b, kv.page_shift));
    } else {
        b = (int)item;
    }
    const int slot = batch.slot(b, kv.slots);
    if (slot < 0) return it;
    const int len = __ldg(kv.lens + slot), rows = batch.count(b);
    const int begin = max(0, len - rows);
    if (rows == 0 || len <= 0) return it;
    const int block = (begin >> kv.page_shift) + k;
    const int from = max(begin, block << kv.page_shift), to = min(len, (block + 1) << kv.page_shift);
    if (from >= to) return it;
    it.page = kv_page(kv, slot, (uint32_t)block);
    it.row0 = batch.first(b) + (from - (len - rows));
    it.lo = (uint32_t)(from - (block << kv.page_shift));
    it.hi = (uint32_t)(to - (block << kv.page_shift));
    return it;
}

// One block per (touched page, head, keys or values).  Bound by memory: a new value is read once
// (2 bytes) and written once (1 byte); it waits in registers for the page's maximum.  Old tokens
// of the page are only touched when its scale grows.
template <typename T, int kVec>
__global__ void __launch_bounds__(256) append_kernel(Kv kv, KvBatch batch, Rows rows)
{
    const Item it = find_item(kv, batch, blockIdx.x);
    const uint32_t head = blockIdx.y, which = blockIdx.z;
    if (it.page < 0) return;
    const uint32_t per_token = kv.dim / 8u;
    uint8_t* codes = kv.codes + (uint64_t)it.page * kv.page_bytes() + (which * kv.heads + head) * kv.head_bytes();
    float* scale_at = kv.scales + ((uint64_t)it.page * 2u + which) * kv.heads + head;
    const float old_scale = it.lo ? *scale_at : 0.f;

    uint4 x[kVec];
    float top = 0.f;
    bool odd = false;
#pragma unroll
    for (int j = 0; j < kVec; ++j) {
        const uint32_t i = threadIdx.x + 256u * j, token = i / per_token, part = i - token * per_token;
        x[j] = make_uint4(0u, 0u, 0u, 0u);
        if (token >= it.lo && token < it.hi) {
            const int64_t row = it.row0 + (int)(token - it.lo);
            x[j] = __ldg((const uint4*)(rows.base[which] + row * rows.row[which] + head * rows.head[which]) + part);
        }
    }
#pragma unroll
    for (int j = 0; j < kVec; ++j) {
        const uint32_t w[4] = {x[j].x, x[j].y, x[j].z, x[j].w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float2 f = to_float2<T>(w[e]);
            const float a = fabsf(f.x), b = fabsf(f.y);
            const bool fa = a <= 3.402823466e38f, fb = b <= 3.402823466e38f;   // false for infinities and NaN
            top = fmaxf(top, fmaxf(fa ? a : 0.f, fb ? b : 0.f));
            odd |= !(fa && fb);
        }
    }
#pragma unroll
    for (int s = 16; s; s >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, s));
    __shared__ float tops[8];
    if ((threadIdx.x & 31u) == 0) tops[threadIdx.x >> 5] = top;
    if (__syncthreads_or(odd) && threadIdx.x == 0) atomicOr(&kv.head->status, kKvStatNonfinite);
#pragma unroll
    for (int w = 0; w < 8; ++w) top = fmaxf(top, tops[w]);
    const float scale = fmaxf(fmaxf(old_scale, __fdiv_rn(top, 127.f)), kScaleFloor);
    const bool grown = it.lo && scale != old_scale;
    const float ratio = __fdiv_rn(old_scale, scale);
#pragma unroll
    for (int j = 0; j < kVec; ++j) {
        const uint32_t i = threadIdx.x + 256u * j, token = i / per_token;
        uint2* at = (uint2*)codes + i;
        if (token >= it.lo && token < it.hi) {
            const uint32_t w[4] = {x[j].x, x[j].y, x[j].z, x[j].w};
            uint32_t out[2] = {0u, 0u};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float2 f = to_float2<T>(w[e]);
#pragma unroll
                for (int p = 0; p < 2; ++p) {
                    const float v = p ? f.y : f.x;
                    // an infinity divides to an infinity and is clamped; the maximum is finite, so no NaN arises from it
                    float q = rintf(__fdiv_rn(v, scale));
                    q = v == v ? fminf(fmaxf(q, -127.f), 127.f) : 0.f;
                    out[e >> 1] |= (uint32_t)((int)q + ENTRO_KV_ZERO_POINT) << (16 * (e & 1) + 8 * p);
                }
            }
            *at = make_uint2(out[0], out[1]);
        } else if (grown && token < it.lo) {
            const uint2 old = *at;
            const uint32_t w[2] = {old.x, old.y};
            uint32_t out[2] = {0u, 0u};
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float q = (float)((int)(w[e >> 2] >> (8 * (e & 3)) & 0xffu) - ENTRO_KV_ZERO_POINT);
                const float r = fminf(fmaxf(rintf(__fmul_rn(q, ratio)), -128.f), 127.f);
                out[e >> 2] |= (uint32_t)((int)r + ENTRO_KV_ZERO_POINT) << (8 * (e & 3));
            }
            *at = make_uint2(out[0], out[1]);
        }
    }
    if (threadIdx.x == 0) *scale_at = scale;
}

// One block per row; a thread takes eight values at a time.
template <typename T>
__global__ void __launch_bounds__(256) read_kernel(Kv kv, KvBatch batch, Rows rows)
{
    const uint32_t row = blockIdx.x;
    int b = (int)row;
    if (batch.row_start) {
        b = block_find(batch.n, row, [&](uint32_t i) { return (uint32_t)batch.first(i); });
        if (b < 0 || (int)row >= batch.first(b) + batch.count(b)) return;
    }
    const int slot = batch.slot(b, kv.slots);
    const int len = slot >= 0 ? __ldg(kv.lens + slot) : 0;
    const int position = len - batch.count(b) + ((int)row - batch.first(b));
    const int page = position >= 0 && slot >= 0 ? kv_page(kv, slot, (uint32_t)position >> kv.page_shift) : -1;
    const uint32_t token = (uint32_t)position & (kv.page() - 1u), per_token = kv.dim / 8u, per_side = kv.heads * per_token;
    for (uint32_t i = threadIdx.x; i < 2u * per_side; i += blockDim.x) {
        const uint32_t which = i >= per_side, head = (i - which * per_side) / per_token, part = i - which * per_side - head * per_token;
        uint4 out = make_uint4(0u, 0u, 0u, 0u);
        if (page >= 0) {
            const uint8_t* codes = kv.codes + (uint64_t)page * kv.page_bytes() + (which * kv.heads + head) * kv.head_bytes();
            const uint2 c = __ldg((const uint2*)codes + token * per_token + part);
            const float s = __ldg(kv.scales + ((uint64_t)page * 2u + which) * kv.heads + head);
            const uint32_t w[2] = {c.x, c.y};
            uint32_t o[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const uint32_t two = w[e >> 1] >> (16 * (e & 1));
                o[e] = from_float2<T>(__fmul_rn(s, (float)((int)(two & 0xffu) - ENTRO_KV_ZERO_POINT)),
                                      __fmul_rn(s, (float)((int)(two >> 8 & 0xffu) - ENTRO_KV_ZERO_POINT)));
            }
            out = make_uint4(o[0], o[1], o[2], o[3]);
        }
        *((uint4*)(const_cast<unsigned char*>(rows.base[which]) + (int64_t)row * rows.row[which] + head * rows.head[which]) + part) = out;
    }
}

entro_status check_rows(const entro_kv_rows* r, Rows* out)
{
    if (!r || !r->k_dev || !r->v_dev || r->reserved) return ENTRO_ERR_INVALID_ARG;
    if (r->type != ENTRO_FLOAT16 && r->type != ENTRO_BFLOAT16) return ENTRO_ERR_INVALID_ARG;
    if (!aligned(r->k_dev, 16) || !aligned(r->v_dev, 16) || !kv_strides_ok(r->k_row_stride, r->k_head_stride) ||
        !kv_strides_ok(r->v_row_stride, r->v_head_stride))
        return ENTRO_ERR_INVALID_ARG;
    *out = Rows{{(const unsigned char*)r->k_dev, (const unsigned char*)r->v_dev},
                {2 * r->k_row_stride, 2 * r->v_row_stride},
                {2 * r->k_head_stride, 2 * r->v_head_stride}};
    return ENTRO_OK;
}

template <typename T>
void launch_append(const Kv& kv, const KvBatch& batch, const Rows& rows, dim3 grid, cudaStream_t s)
{
    const uint32_t vectors = kv.page() * kv.dim / 8u;
    if (vectors <= 256u)
        append_kernel<T, 1><<<grid, 256, 0, s>>>(kv, batch, rows);
    else if (vectors <= 512u)
        append_kernel<T, 2><<<grid, 256, 0, s>>>(kv, batch, rows);
    else if (vectors <= 1024u)
        append_kernel<T, 4><<<grid, 256, 0, s>>>(kv, batch, rows);
    else
        append_kernel<T, 8><<<grid, 256, 0, s>>>(kv, batch, rows);
}

}  // namespace
}  // namespace entro

using namespace entro;

extern "C" entro_status entro_kv_append(const entro_kv_cache* cache, const entro_kv_batch* b, const entro_kv_rows* r,
                                        void* cuda_stream)
{
    Kv kv;
    KvBatch batch;
    Rows rows;
    if (entro_status e = kv_check(cache, &kv)) return e;
    if (entro_status e = kv_check(cache, b, &batch)) return e;
    if (batch.n == 0 || batch.rows == 0) return ENTRO_OK;
    if (entro_status e = check_rows(r, &rows)) return e;
    const uint32_t items = batch.row_start ? item_of(batch.rows, batch.n, kv.page_shift) : batch.n;
    const dim3 grid(items, kv.heads, 2);
    if (r->type == ENTRO_FLOAT16)
        launch_append<__half>(kv, batch, rows, grid, (cudaStream_t)cuda_stream);
    else
        launch_append<__nv_bfloat16>(kv, batch, rows, grid, (cudaStream_t)cuda_stream);
    count_launch();
    ENTRO_CUDA(cudaGetLastError());
    return ENTRO_OK;
}

extern "C" entro_status entro_kv_read(const entro_kv_cache* cache, const entro_kv_batch* b, const entro_kv_rows* r,
                                      void* cuda_stream)
{
    Kv kv;
    KvBatch batch;
    Rows rows;
    if (entro_status e = kv_check(cache, &kv)) return e;
    if (entro_status e = kv_check(cache, b, &batch)) return e;
    if (batch.n == 0 || batch.rows == 0) return ENTRO_OK;
    if (entro_status e = check_rows(r, &rows)) return e;
    if (r->type == ENTRO_FLOAT16)
        read_kernel<__half><<<batch.rows, 256, 0, (cudaStream_t)cuda_stream>>>(kv, batch, rows);
    else
        read_kernel<__nv_bfloat16><<<batch.rows, 256, 0, (cudaStream_t)cuda_stream>>>(kv, batch, rows);
    count_launch();
    ENTRO_CUDA(cudaGetLastError());
    return ENTRO_OK;
}
