// Attention of few rows per sequence (a token step): the cache is read once, at memory speed.
//
// A unit is a sequence and a key/value head: its rows (new tokens times query heads of the group,
// at most 8 * kTiles) against all tokens they see, in slices of 16 tokens.  All slices of all units
// form one line that is cut into equal shares, one per block, whatever the lengths; a unit that is
// cut leaves partial results (M, L, sums) that the block arriving last joins, in the order of the
// shares, so results do not depend on who came first.
//
// Inside a block every warp takes slices of its own (8 warps, every eighth slice) with statistics of
// its own, joined at the unit's end.  Products run on m16n8k16 with the tokens as rows, so that eight
// query heads fill a tile:  S^T[16 tokens, 8] = K' Q^T and O^T[dim, 8] += V'^T P^T.  The matrix unit is
// far from busy: the bound is memory, then the byte-to-fp16 conversion (1 to 1.25 instructions per
// code).  Any permutation of the inner index is allowed if both operands share it, so a thread's 16
// consecutive bytes of a key row serve four products, and a thread's 16 bytes of four value rows eight.
// Each warp keeps a ring of slices of its own in shared memory, filled by asynchronous 16-byte copies
// two slices ahead; rows are 16 bytes longer there than in the cache, which spreads the four value rows
// of a load over the banks.  No barrier until the unit's end.
#pragma once

#include "entro_kv_attention.cuh"

namespace entro {
namespace {

constexpr uint32_t kTokenWarps = 8, kTokenThreads = 32 * kTokenWarps;
constexpr uint32_t kTokenRows = 16;             // most rows of a unit
constexpr uint32_t kTokenBlocks = 512;          // most blocks of a launch
constexpr uint32_t kTokenMinSlices = 16;        // a share is not made smaller than this
// Starting and ending a unit costs a block about as much time as this many slices; on the line a unit
// is that much longer than its slices, or a block with many short sequences would be last by far.
constexpr uint32_t kTokenUnitCost = 12;

static_assert(kKvPartialBytes >= 4ull * kTokenBlocks * 2 * kTokenRows * 130, "a block leaves at most two partial results");

__device__ __forceinline__ void mma_16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose_8x8(uint32_t a)
{
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(a));
    return r;
}
__device__ __forceinline__ void copy16(uint32_t to, const uint8_t* from)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
}
__device__ __forceinline__ void copy4(uint32_t to, const void* from)
{
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(to), "l"(from) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int kLeft>
__device__ __forceinline__ void copies_wait()
{
    asm volatile("cp.async.wait_group %0;" ::"n"(kLeft) : "memory");
}
__device__ __forceinline__ uint4 lds16(uint32_t a)
{
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a) : "memory");
    return v;
}
__device__ __forceinline__ uint2 lds8(uint32_t a)
{
    uint2 v;
    asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(a) : "memory");
    return v;
}
__device__ __forceinline__ uint32_t lds4(uint32_t a)
{
    uint32_t v;
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(a) : "memory");
    return v;
}

// First of the four inner indices (dims) that word i of a lane's key row and of its query row stands for.
template <int kDim>
__device__ __forceinline__ uint32_t key_dim(int i, uint32_t t)
{
    return kDim == 96 ? 32u * (i / 2) + 8u * t + 4u * (i % 2) : 16u * (t + 4u * (i / 4)) + 4u * (i % 4);
}
template <int kDim>
__device__ __forceinline__ void load_key_row(uint32_t row, uint32_t t, uint32_t (&w)[kDim / 16])
{
    if constexpr (kDim == 96) {
#pragma unroll
        for (int c = 0; c < 3; ++c) {
            const uint2 v = lds8(row + 32u * c + 8u * t);
            w[2 * c] = v.x;
            w[2 * c + 1] = v.y;
        }
    } else {
#pragma unroll
        for (int c = 0; c < kDim / 64; ++c) {
            const uint4 v = lds16(row + 16u * (t + 4u * c));
            w[4 * c] = v.x;
            w[4 * c + 1] = v.y;
            w[4 * c + 2] = v.z;
            w[4 * c + 3] = v.w;
        }
    }
}
// First of the four dims that word i of a lane's value rows stands for.
template <int kDim>
__device__ __forceinline__ uint32_t value_dim(int i, uint32_t g)
{
    return kDim == 128 ? 16u * g + 4u * i : kDim == 64 || i < 2 ? 8u * g + 4u * i : 64u + 4u * g;
}
template <int kDim>
__device__ __forceinline__ void load_value_row(uint32_t row, uint32_t g, uint32_t (&w)[kDim / 32])
{
    if constexpr (kDim == 128) {
        const uint4 v = lds16(row + 16u * g);
        w[0] = v.x;
        w[1] = v.y;
        w[2] = v.z;
        w[3] = v.w;
    } else {
        const uint2 v = lds8(row + 8u * g);
        w[0] = v.x;
        w[1] = v.y;
        if constexpr (kDim == 96) w[2] = lds4(row + 64u + 4u * g);
    }
}

// A ring stage: 16 key rows, 16 value rows, the two scales.  Two blocks of 8 warps (one tile) or one (two tiles) share
// the SM's 227 KB.
template <int kDim>
constexpr uint32_t kTokenRowBytes = kDim + 16;
template <int kDim>
constexpr uint32_t kTokenStageBytes = 32 * kTokenRowBytes<kDim> + 16;
template <int kDim, int kTiles>
constexpr int kTokenStages = kDim == 64 ? 5 : kTiles == 1 ? 3 : 5;

// A sequence as the kernel handles it.
struct TokenSeq {
    int slot, len, rows, row0;       // slot -1: no tokens
    uint32_t slices;                 // per unit; 0: not this kernel's
};

__device__ __forceinline__ TokenSeq token_seq(const Kv& kv, const KvBatch& batch, const Query& q, uint32_t b, uint32_t most_rows,
                                              Span* span)
{
    TokenSeq s;
    s.rows = batch.count(b);
    s.row0 = batch.first(b);
    s.slot = batch.slot(b, kv.slots);
    s.len = s.slot >= 0 ? max(0, __ldg(kv.lens + s.slot)) : 0;
    *span = Span{0u, 0u, 1u};        // nothing to see: one masked slice, so that the rows are written
    if (s.len > 0) *span = span_of(max(0, s.len - s.rows), s.len - 1, q.window, q.sinks, 4u);
    s.slices = s.rows > 0 && (uint32_t)s.rows * q.group <= most_rows ? span->count : 0u;
    return s;
}

template <typename T, int kDim, int kTiles>
__global__ void __launch_bounds__(kTokenThreads, kTiles == 1 ? 2 : 1)
    token_attention_kernel(Kv kv, KvBatch batch, Query q, float* partials)
{
    constexpr uint32_t kCols = 8 * kTiles;
    constexpr int kSteps = kDim / 16;            // products of a slice's first matrix product; words of a key row
    constexpr int kWords = kDim / 32;            // words of a value row
    constexpr uint32_t kStride = kDim + 4;
    constexpr int kStages = kTokenStages<kDim, kTiles>;
    constexpr uint32_t kRow = kTokenRowBytes<kDim>, kStage = kTokenStageBytes<kDim>;
    extern __shared__ __align__(16) float joined[];              // [warps][cols][stride], where the rings lie until then
    const uint32_t ring = (uint32_t)__cvta_generic_to_shared(joined) + (threadIdx.x >> 5) * kStages * kStage;
    __shared__ float stat_m[kTokenWarps][kCols], stat_l[kTokenWarps][kCols];
    __shared__ uint32_t found_b, found_before, is_last, warp_sums[kTokenWarps];
    const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3u;

    // ---- this block's share of the line of slices
    auto slices_of = [&](uint32_t b) {
        Span span;
        const uint32_t n = token_seq(kv, batch, q, b, kCols, &span).slices;
        return n ? (n + kTokenUnitCost) * kv.heads : 0u;
    };
    uint32_t mine = 0;
    for (uint32_t b = threadIdx.x; b < batch.n; b += kTokenThreads) mine += slices_of(b);
#pragma unroll
    for (int s = 16; s; s >>= 1) mine += __shfl_xor_sync(0xffffffffu, mine, s);
    if (lane == 0) warp_sums[warp] = mine;
    __syncthreads();
    uint32_t all = 0;
#pragma unroll
    for (uint32_t w = 0; w < kTokenWarps; ++w) all += warp_sums[w];
    const uint32_t parts = min(gridDim.x, (all + kTokenMinSlices - 1u) / kTokenMinSlices);
    if (blockIdx.x >= parts) return;
    const Shares shares(all, parts);
    uint32_t x = shares.start(blockIdx.x);
    const uint32_t x_end = shares.start(blockIdx.x + 1u);
    // sequence that slice x belongs to
    for (uint32_t base = 0, before = 0; base < batch.n; base += kTokenThreads) {
        const uint32_t b = base + threadIdx.x;
        const uint32_t w = b < batch.n ? slices_of(b) : 0u;
        uint32_t sum = w;
#pragma unroll
        for (int s = 1; s < 32; s <<= 1) {
            const uint32_t y = __shfl_up_sync(0xffffffffu, sum, s);
            if (lane >= (uint32_t)s) sum += y;
        }
        __syncthreads();
        if (lane == 31u) warp_sums[warp] = sum;
        __syncthreads();
        uint32_t chunk = 0;
#pragma unroll
        for (uint32_t i = 0; i < kTokenWarps; ++i) {
            if (i < warp) sum += warp_sums[i];
            chunk += warp_sums[i];
        }
        const uint32_t from = before + sum - w;
        if (x >= from && x < from + w) {
            found_b = b;
            found_before = from;
        }
        before += chunk;
        if (x < before) break;       // the same for all threads
    }
    __syncthreads();
    uint32_t b = found_b, seq_start = found_before;

    Span span;
    TokenSeq seq = token_seq(kv, batch, q, b, kCols, &span);
    while (x < x_end) {
        const uint32_t of_unit = seq.slices ? seq.slices + kTokenUnitCost : 0u, of_seq = of_unit * kv.heads;
        if (x >= seq_start + of_seq) {
            seq_start += of_seq;
            seq = token_seq(kv, batch, q, ++b, kCols, &span);
            continue;
        }
        // the unit's place on the line: its cost, then its slices
        const uint32_t head = (x - seq_start) / of_unit, unit_end = seq_start + (head + 1u) * of_unit;
        const uint32_t unit_start = unit_end - seq.slices, stop = min(unit_end, x_end);
        x = max(x, unit_start);
        if (x >= stop) {             // the share ends before the unit's first slice
            x = stop;
            continue;
        }
        const uint32_t rows = (uint32_t)seq.rows * q.group;
        const int first = seq.len - seq.rows;                    // position of the first row

        // ---- the rows as the second operand; columns 2t, 2t + 1 of each tile are this lane's
        uint32_t qf[kTiles][kSteps][2];
        float factor[kTiles][2];                                 // power of two taken out of the row, times scale * log2 e
        int position[kTiles][2];
#pragma unroll
        for (int n = 0; n < kTiles; ++n) {
            const uint32_t r = 8u * n + g;
            int e = 0;
            uint2 raw[kSteps];
            if (r < rows) {
                const unsigned char* p = q.q + (int64_t)(seq.row0 + (int)(r / q.group)) * q.q_row +
                                         (int64_t)(head * q.group + r % q.group) * q.q_head;
#pragma unroll
                for (int i = 0; i < kSteps; ++i) raw[i] = __ldg((const uint2*)(p + 2u * key_dim<kDim>(i, t)));
            } else {
#pragma unroll
                for (int i = 0; i < kSteps; ++i) raw[i] = make_uint2(0u, 0u);
            }
            if constexpr (sizeof(T) == 2 && !__is_same(T, __half)) {
                float top = 0.f;
#pragma unroll
                for (int i = 0; i < kSteps; ++i) {
                    const float2 a = to_float2<T>(raw[i].x), c = to_float2<T>(raw[i].y);
                    top = fmaxf(fmaxf(fmaxf(fabsf(a.x), fabsf(a.y)), fmaxf(fabsf(c.x), fabsf(c.y))), top);
                }
                top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
                top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
                e = row_exponent(top);
                const float up = power_of_two(e);
#pragma unroll
                for (int i = 0; i < kSteps; ++i) {
                    const float2 a = to_float2<T>(raw[i].x), c = to_float2<T>(raw[i].y);
                    raw[i] = make_uint2(from_float2<__half>(a.x * up, a.y * up), from_float2<__half>(c.x * up, c.y * up));
                }
            }
#pragma unroll
            for (int i = 0; i < kSteps; ++i) {
                qf[n][i][0] = raw[i].x;
                qf[n][i][1] = raw[i].y;
            }
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                const int col = 2 * (int)t + c;
                const int ec = __shfl_sync(0xffffffffu, e, col * 4);       // lanes of row g = col hold its exponent
                factor[n][c] = q.scale * kLog2e * power_of_two(-ec);
                position[n][c] = first + (int)((8u * n + (uint32_t)col) / q.group);
            }
        }

        float o[kSteps][kTiles][4];
        float m[kTiles][2], l[kTiles][2];
#pragma unroll
        for (int n = 0; n < kTiles; ++n) {
#pragma unroll
            for (int i = 0; i < kSteps; ++i) o[i][n][0] = o[i][n][1] = o[i][n][2] = o[i][n][3] = 0.f;
            m[n][0] = m[n][1] = -INFINITY;
            l[n][0] = l[n][1] = 0.f;
        }

        // ---- slices x + warp, x + warp + 8, ...
        const int last = seq.len - 1;
        const int64_t open_from = q.window ? (int64_t)last - (int64_t)q.window : -1;   // later positions are in every row's window
        uint32_t i = x + warp - unit_start;
        const uint32_t i_end = seq.len > 0 ? stop - unit_start : 0u;
        const int32_t* table_row = kv.table + (uint64_t)max(seq.slot, 0) * kv.width;
        const uint64_t page_bytes = kv.page_bytes(), to_values = (uint64_t)kv.heads * kv.head_bytes();
        const uint8_t* lane_codes = kv.codes + head * kv.head_bytes() + lane * 16u;
        const float* lane_scales = kv.scales + head + (lane & 1u) * kv.heads;
        const uint32_t in_page = kv.page() / 16u - 1u, to_block = kv.page_shift - 4u;
        auto page_at = [&](uint32_t idx) -> int {
            if (idx >= i_end) return -1;
            const uint32_t block = span.piece(idx) >> to_block;
            if (block >= kv.width) return -1;
            const int p = __ldg(table_row + block);
            return (uint32_t)p < kv.pages ? p : -1;
        };
        // slice idx, whose page is `page`, into a stage; one commit group per call
        auto fetch = [&](int page, uint32_t idx, uint32_t stage) {
            if (page >= 0) {
                const uint8_t* k = lane_codes + (uint64_t)(uint32_t)page * page_bytes + (span.piece(idx) & in_page) * (16u * kDim);
#pragma unroll
                for (int c = 0; c < kDim / 32; ++c) {
                    const uint32_t chunk = lane + 32u * c, at = chunk / (kDim / 16u) * kRow + chunk % (kDim / 16u) * 16u;
                    copy16(stage + at, k + 512u * c);
                    copy16(stage + 16u * kRow + at, k + to_values + 512u * c);
                }
                if (lane < 2u) copy4(stage + 32u * kRow + lane * 4u, lane_scales + (uint64_t)(uint32_t)page * 2u * kv.heads);
            }
            copies_commit();
        };
        const float ref = value_reference(kv, seq.slot, span.piece(0) >> to_block, head), by_ref = __frcp_rn(ref);
        int pages[kStages];          // of the slices in the ring and, last, of the next one to fetch
#pragma unroll
        for (int c = 0; c < kStages; ++c) pages[c] = page_at(i + c * kTokenWarps);
#pragma unroll
        for (int c = 0; c < kStages - 1; ++c) fetch(pages[c], i + c * kTokenWarps, ring + c * kStage);
        uint32_t stage = ring, stage_in = ring + (kStages - 1) * kStage;
        for (; i < i_end; i += kTokenWarps) {
            copies_wait<kStages - 2>();
            __syncwarp();            // every lane's copies of this slice are in place, and the stage before it has been read
            const int page = pages[0];
            fetch(pages[kStages - 1], i + (kStages - 1) * kTokenWarps, stage_in);
#pragma unroll
            for (int c = 0; c + 1 < kStages; ++c) pages[c] = pages[c + 1];
            pages[kStages - 1] = page_at(i + kStages * kTokenWarps);

            float s[kTiles][4];
#pragma unroll
            for (int n = 0; n < kTiles; ++n) s[n][0] = s[n][1] = s[n][2] = s[n][3] = 0.f;
            {
                uint32_t kw[2][kSteps];
                load_key_row<kDim>(stage + g * kRow, t, kw[0]);
                load_key_row<kDim>(stage + (g + 8u) * kRow, t, kw[1]);
#pragma unroll
                for (int j = 0; j < kSteps; ++j) {
                    const uint32_t a[4] = {codes_low(kw[0][j]), codes_low(kw[1][j]), codes_high(kw[0][j]), codes_high(kw[1][j])};
#pragma unroll
                    for (int n = 0; n < kTiles; ++n) mma_16816(s[n], a, qf[n][j][0], qf[n][j][1]);
                }
            }
            const int j0 = (int)(span.piece(i) * 16u);
            const bool there = page >= 0;
            const bool whole = there && j0 + 15 <= first && (j0 > open_from || (uint32_t)j0 + 15u < q.sinks);
            const float key_scale = __uint_as_float(lds4(stage + 32u * kRow));
            const float rel = there ? relative_scale(__uint_as_float(lds4(stage + 32u * kRow + 4u)), by_ref) : 1.f;
            const float lv = lg2(rel), inv = rcp(rel);

            uint32_t pb[kTiles][2];
            float shrink[kTiles][2];
            bool moved = false;
#pragma unroll
            for (int n = 0; n < kTiles; ++n) {
                float u[4];
#pragma unroll
                for (int c = 0; c < 4; ++c) u[c] = fmaf(s[n][c], key_scale * factor[n][c & 1], lv);
                if (!whole) {
#pragma unroll
                    for (int c = 0; c < 4; ++c)
                        if (!there || !sees(position[n][c & 1], j0 + (int)g + 8 * (c >> 1), q.window, q.sinks)) u[c] = -INFINITY;
                }
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    float top = fmaxf(u[c], u[c + 2]);
                    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 4));
                    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 8));
                    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 16));
                    const float up = fmaxf(m[n][c], top);
                    const float base = up == -INFINITY ? 0.f : up;
                    moved |= up != m[n][c];
                    shrink[n][c] = ex2(m[n][c] - base);
                    m[n][c] = up;
                    u[c] = ex2(u[c] - base);
                    u[c + 2] = ex2(u[c + 2] - base);
                    l[n][c] = fmaf(u[c] + u[c + 2], inv, l[n][c] * shrink[n][c]);
                }
                pb[n][0] = transpose_8x8(from_float2<__half>(u[0], u[1]));
                pb[n][1] = transpose_8x8(from_float2<__half>(u[2], u[3]));
            }
            if (__any_sync(0xffffffffu, moved)) {
#pragma unroll
                for (int n = 0; n < kTiles; ++n)
#pragma unroll
                    for (int j = 0; j < kSteps; ++j) {
                        o[j][n][0] *= shrink[n][0];
                        o[j][n][1] *= shrink[n][1];
                        o[j][n][2] *= shrink[n][0];
                        o[j][n][3] *= shrink[n][1];
                    }
            }
            uint32_t vw[4][kWords];
            load_value_row<kDim>(stage + (16u + 2u * t) * kRow, g, vw[0]);
            load_value_row<kDim>(stage + (17u + 2u * t) * kRow, g, vw[1]);
            load_value_row<kDim>(stage + (24u + 2u * t) * kRow, g, vw[2]);
            load_value_row<kDim>(stage + (25u + 2u * t) * kRow, g, vw[3]);
#pragma unroll
            for (int w = 0; w < kWords; ++w) {
                // two tokens' bytes side by side, then two dims (rows g, g + 8 of a product) at a time
                const uint32_t lo01 = __byte_perm(vw[0][w], vw[1][w], 0x5140), hi01 = __byte_perm(vw[0][w], vw[1][w], 0x7362);
                const uint32_t lo23 = __byte_perm(vw[2][w], vw[3][w], 0x5140), hi23 = __byte_perm(vw[2][w], vw[3][w], 0x7362);
                const uint32_t a0[4] = {codes_low(lo01), codes_high(lo01), codes_low(lo23), codes_high(lo23)};
                const uint32_t a1[4] = {codes_low(hi01), codes_high(hi01), codes_low(hi23), codes_high(hi23)};
#pragma unroll
                for (int n = 0; n < kTiles; ++n) {
                    mma_16816(o[2 * w][n], a0, pb[n][0], pb[n][1]);
                    mma_16816(o[2 * w + 1][n], a1, pb[n][0], pb[n][1]);
                }
            }
            stage_in = stage;
            stage = stage + kStage == ring + kStages * kStage ? ring : stage + kStage;
        }

        // ---- the warps' results become the block's
#pragma unroll
        for (int n = 0; n < kTiles; ++n)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                float sum = l[n][c];
                sum += __shfl_xor_sync(0xffffffffu, sum, 4);
                sum += __shfl_xor_sync(0xffffffffu, sum, 8);
                sum += __shfl_xor_sync(0xffffffffu, sum, 16);
                if (g == 0) {
                    stat_m[warp][8 * n + 2 * t + c] = m[n][c];
                    stat_l[warp][8 * n + 2 * t + c] = sum;
                }
            }
        __syncthreads();
#pragma unroll
        for (int n = 0; n < kTiles; ++n)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                const uint32_t col = 8u * n + 2u * t + c;
                float top = -INFINITY;
#pragma unroll
                for (uint32_t w = 0; w < kTokenWarps; ++w) top = fmaxf(top, stat_m[w][col]);
                const float f = top == -INFINITY ? 0.f : ex2(m[n][c] - top);
                float* to = joined + (warp * kCols + col) * kStride;
#pragma unroll
                for (int w = 0; w < kWords; ++w)
                    *(float4*)(to + value_dim<kDim>(w, g)) =
                        make_float4(o[2 * w][n][c] * f, o[2 * w][n][c + 2] * f, o[2 * w + 1][n][c] * f, o[2 * w + 1][n][c + 2] * f);
            }
        __syncthreads();
        const bool complete = x == unit_start && stop == unit_end;
        // of a block's two places the first is for a unit that began in another block, the second for one that goes on in the next
        const uint32_t row_floats = kCols * (kDim + 2u);
        float* partial = partials + (uint64_t)(blockIdx.x * 2u + (x == unit_start ? 1u : 0u)) * row_floats;
        auto finish = [&](uint32_t r, uint32_t d, float4 v, float top, float sum) {
            const float by = sum == 0.f ? 0.f : ref * __frcp_rn(sum);
            const int64_t row = seq.row0 + (int)(r / q.group);
            const uint32_t query_head = head * q.group + r % q.group;
            uint2 two = make_uint2(from_float2<T>(v.x * by, v.y * by), from_float2<T>(v.z * by, v.w * by));
            *(uint2*)(q.out + row * q.out_row + (int64_t)query_head * q.out_head + 2u * d) = two;
            if (d == 0 && q.lse) q.lse[(uint64_t)row * q.heads + query_head] = sum == 0.f ? -INFINITY : kLn2 * (top + log2f(sum));
        };
        for (uint32_t e = threadIdx.x; e < rows * (kDim / 4u); e += kTokenThreads) {
            const uint32_t r = e / (kDim / 4u), d = 4u * (e - r * (kDim / 4u));
            float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
            float top = -INFINITY, sum = 0.f;
#pragma unroll
            for (uint32_t w = 0; w < kTokenWarps; ++w) top = fmaxf(top, stat_m[w][r]);
#pragma unroll
            for (uint32_t w = 0; w < kTokenWarps; ++w) {
                sum += stat_l[w][r] * (top == -INFINITY ? 0.f : ex2(stat_m[w][r] - top));
                const float4 a = *(const float4*)(joined + (w * kCols + r) * kStride + d);
                v.x += a.x;
                v.y += a.y;
                v.z += a.z;
                v.w += a.w;
            }
            if (complete) {
                finish(r, d, v, top, sum);
            } else {
                __stcg((float4*)(partial + r * kDim + d), v);
                if (d == 0) {
                    __stcg(partial + kCols * kDim + r, top);
                    __stcg(partial + kCols * kDim + kCols + r, sum);
                }
            }
        }
        if (!complete) {
            // the unit's shares: blocks c0 .. c1; the last one to arrive joins them in that order
            const uint32_t c0 = shares.owner(unit_start), c1 = shares.owner(unit_end - 1u);
            __threadfence();
            __syncthreads();
            if (threadIdx.x == 0) {
                const uint32_t before = atomicAdd(&kv.head->arrived[c0], 1u);
                is_last = before == c1 - c0;
                if (is_last) kv.head->arrived[c0] = 0u;
            }
            __syncthreads();
            if (is_last) {
                __threadfence();
                const float* from0 = partials + (uint64_t)(c0 * 2u + 1u) * row_floats;
                const float* from1 = partials + (uint64_t)((c0 + 1u) * 2u) * row_floats;
                const uint32_t others = c1 - c0;
                for (uint32_t e = threadIdx.x; e < rows * (kDim / 4u); e += kTokenThreads) {
                    const uint32_t r = e / (kDim / 4u), d = 4u * (e - r * (kDim / 4u));
                    const float m0 = __ldcg(from0 + kCols * kDim + r);
                    float top = m0;
#pragma unroll 8
                    for (uint32_t c = 0; c < others; ++c)
                        top = fmaxf(top, __ldcg(from1 + (uint64_t)c * 2u * row_floats + kCols * kDim + r));
                    const float base = top == -INFINITY ? 0.f : top;
                    float f = ex2(m0 - base);
                    float sum = __ldcg(from0 + kCols * kDim + kCols + r) * f;
                    float4 v = __ldcg((const float4*)(from0 + r * kDim + d));
                    v = make_float4(v.x * f, v.y * f, v.z * f, v.w * f);
#pragma unroll 8
                    for (uint32_t c = 0; c < others; ++c) {
                        const float* p = from1 + (uint64_t)c * 2u * row_floats;
                        const float mc = __ldcg(p + kCols * kDim + r), lc = __ldcg(p + kCols * kDim + kCols + r);
                        const float4 a = __ldcg((const float4*)(p + r * kDim + d));
                        f = ex2(mc - base);
                        sum = fmaf(lc, f, sum);
                        v.x = fmaf(a.x, f, v.x);
                        v.y = fmaf(a.y, f, v.y);
                        v.z = fmaf(a.z, f, v.z);
                        v.w = fmaf(a.w, f, v.w);
                    }
                    finish(r, d, v, top, sum);
                }
            }
        }
        __syncthreads();             // shared memory is free for the next unit
        x = stop;
    }
}

template <typename T, int kDim>
cudaError_t launch_tokens(const Kv& kv, const KvBatch& batch, const Query& q, uint32_t most_rows, uint32_t sm_count, float* partials,
                          cudaStream_t s)
{
    // at most 8 rows: one tile of columns, 128 registers, two blocks per SM; else two tiles and one block
    const bool one = most_rows <= 8;
    auto* kernel = one ? token_attention_kernel<T, kDim, 1> : token_attention_kernel<T, kDim, 2>;
    const uint32_t smem = kTokenWarps * kTokenStageBytes<kDim> * (one ? kTokenStages<kDim, 1> : kTokenStages<kDim, 2>);
    static_assert(kTokenStageBytes<kDim> * kTokenStages<kDim, 1> >= 8u * (kDim + 4u) * 4u &&
                      kTokenStageBytes<kDim> * kTokenStages<kDim, 2> >= 16u * (kDim + 4u) * 4u,
                  "the joined sums fit where the rings were");
    if (smem > 48u * 1024u) {        // per device, so not remembered here
        cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
        if (e != cudaSuccess) return e;
    }
    const uint32_t blocks = min(kTokenBlocks, (one ? 2u : 1u) * sm_count);
    kernel<<<blocks, kTokenThreads, smem, s>>>(kv, batch, q, partials);
    return cudaGetLastError();
}

}  // namespace
}  // namespace entro
