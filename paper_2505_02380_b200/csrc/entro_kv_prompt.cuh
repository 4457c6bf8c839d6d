// Attention of many rows per sequence (prompts) on the fifth-generation tensor cores.
//
// A unit is a sequence, a key/value head and a tile of 256 rows (row r = new token r / group, query
// head r % group: the group's heads share every key and value that is fetched and converted).  It runs
// against all tokens its rows see, in pieces of 128 tokens.  As for single tokens, all pieces of all
// units form one line that is cut into equal shares, one per SM, and units that are cut are joined by
// whoever arrives last.
//
// One block per SM, warp-specialised around mbarriers:
//   warps 0 - 3, 4 - 7   softmax of rows 0 - 127 and 128 - 255, one thread per row: reads S from tensor
//                        memory, writes P over it as fp16, rescales the output sum when its row's
//                        maximum has grown by more than 2^8, writes results
//   warps 8 - 11         bytes of the cache to fp16 in shared memory (keys and values, two pieces each)
//   warp 12, one thread  issues tcgen05.mma:  S = Q K'^T (both in shared memory) and O += P V' (P in
//                        tensor memory); order QK0(j), PV1(j-1), QK1(j), PV0(j), so that one half's
//                        products run under the other half's softmax
// Keys lie [token][dim] and are a K-major operand; values lie [token][dim] too, which is an MN-major
// operand, so both are stored alike: 128-byte rows of 64 dims, 16-byte units XORed with the row (the
// 128-byte swizzle of the matrix descriptors).
// Tensor memory: S0, S1, O0, O1 of 128 columns each.
#pragma once

#include "entro_kv_attention.cuh"

namespace entro {
namespace {

constexpr uint32_t kPromptThreads = 416;
constexpr uint32_t kPromptRows = 256;            // rows of a unit
constexpr uint32_t kPromptBlocks = 160;          // most blocks of a launch
constexpr uint32_t kPromptMinPieces = 2;         // a share is not made smaller than this
constexpr uint32_t kPromptUnitCost = 2;          // starting and ending a unit, in pieces
constexpr uint32_t kSlabBytes = 128 * 128;       // 128 rows of 64 fp16 numbers
constexpr uint32_t kWaitLimit = 1u << 20;        // tries of a barrier wait (each may suspend) before the kernel gives up
constexpr float kGrowth = 8.f;                   // P stays below 2^8: the output sum is rescaled when the maximum grows by more
constexpr uint32_t kPromptArrived = 512;         // first counter of KvWorkHeader::arrived that is this kernel's

template <int kDim>
constexpr uint32_t kPromptSlabs = kDim == 64 ? 1 : 2;
template <int kDim>
constexpr uint32_t kPromptSmem = 1024 + 6 * kPromptSlabs<kDim> * kSlabBytes + 1024;

static_assert(kKvPartialBytes >= 4ull * kPromptBlocks * 2 * kPromptRows * 130, "a block leaves at most two partial results");

struct PromptShared {
    uint64_t q_full[2], k_full[2], k_empty[2], v_full[2], v_empty[2], s_full[2], p_full[2], o_full[2], scale_full[4];
    uint64_t joint[2], drained;                  // the warps of a half meet; products of a run that was given up
    float4 scales[4][8];                         // ring of pieces: per 16 tokens key factor, log2 of the value scale, its inverse
    uint32_t tmem, dead, last[2];
};
static_assert(sizeof(PromptShared) <= 1024, "fits behind the tiles");

// ---------------------------------------------------------------------------------- barriers, tensor memory

__device__ __forceinline__ uint32_t shared_address(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void bar_init(uint64_t* b, uint32_t count)
{
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(shared_address(b)), "r"(count) : "memory");
}
__device__ __forceinline__ void bar_arrive(uint64_t* b)
{
    asm volatile("mbarrier.arrive.release.cta.shared::cta.b64 _, [%0];" ::"r"(shared_address(b)) : "memory");
}
// One thread's wait; false when it ran out of tries here or in another warp: the caller leaves its loop.
__device__ __forceinline__ bool bar_wait_one(uint64_t* b, uint32_t parity, PromptShared& sh)
{
    const uint32_t a = shared_address(b);
    for (uint32_t i = 0; i < kWaitLimit; ++i) {
        uint32_t done;
        asm volatile(
            "{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.acquire.cta.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
            : "=r"(done)
            : "r"(a), "r"(parity)
            : "memory");
        if (done) return true;
        if ((i & 63u) == 63u && *(volatile uint32_t*)&sh.dead) return false;
    }
    *(volatile uint32_t*)&sh.dead = 1u;
    return false;
}
// A whole warp's wait, the same answer for all lanes.
__device__ __forceinline__ bool bar_wait(uint64_t* b, uint32_t parity, PromptShared& sh)
{
    return __all_sync(0xffffffffu, bar_wait_one(b, parity, sh));
}
__device__ __forceinline__ void tc_commit(uint64_t* b)
{
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(shared_address(b)) : "memory");
}
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void proxy_fence() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

__device__ __forceinline__ void tm_load32(uint32_t at, uint32_t (&r)[32])
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
          "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]),
          "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]),
          "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(at));
}
__device__ __forceinline__ void tm_store32(uint32_t at, const uint32_t (&r)[32])
{
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
        "{%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};" ::"r"(
            at),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
        "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]),
        "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]),
        "r"(r[31])
        : "memory");
}
__device__ __forceinline__ void tm_store16(uint32_t at, const uint32_t (&r)[16])
{
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(at), "r"(r[0]),
        "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]),
        "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
        : "memory");
}
__device__ __forceinline__ void tm_wait_load() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tm_wait_store() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// Matrix descriptor of a tile stored as 128-byte rows with the 128-byte swizzle: address, leading offset, 1024 bytes
// from one group of eight rows to the next (all in 16-byte units), version 1, swizzle mode 2.
__device__ __forceinline__ uint64_t tile_descriptor(uint32_t address, uint32_t leading_bytes)
{
    return (uint64_t)((address >> 4) & 0x3fffu) | (uint64_t)((leading_bytes >> 4) & 0x3fffu) << 16 | (uint64_t)(1024u >> 4) << 32 |
           (uint64_t)1u << 46 | (uint64_t)2u << 61;
}
// Instruction descriptor: fp16 operands, fp32 sums, 128 rows, `n` columns, second operand K-major or MN-major.
__device__ __forceinline__ constexpr uint32_t product_descriptor(uint32_t n, bool mn_major)
{
    return 1u << 4 | (mn_major ? 1u << 16 : 0u) | (n >> 3) << 17 | (128u >> 4) << 24;
}
__device__ __forceinline__ void tc_product_shared(uint32_t d, uint64_t a, uint64_t b, uint32_t what, uint32_t add)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a),
        "l"(b), "r"(what), "r"(add)
        : "memory");
}
__device__ __forceinline__ void tc_product_tensor(uint32_t d, uint32_t a, uint64_t b, uint32_t what, uint32_t add)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d), "r"(a),
        "l"(b), "r"(what), "r"(add)
        : "memory");
}

// ---------------------------------------------------------------------------------- the line of pieces

struct PromptSeq {
    int slot, len, rows, row0;
    uint32_t tiles;                  // tiles of 256 rows per head; 0: not this kernel's
};

__device__ __forceinline__ PromptSeq prompt_seq(const Kv& kv, const KvBatch& batch, const Query& q, uint32_t b, uint32_t few_rows)
{
    PromptSeq s;
    s.rows = batch.count(b);
    s.row0 = batch.first(b);
    s.slot = batch.slot(b, kv.slots);
    s.len = s.slot >= 0 ? max(0, __ldg(kv.lens + s.slot)) : 0;
    const uint32_t r = (uint32_t)s.rows * q.group;
    s.tiles = r > few_rows ? (r + kPromptRows - 1u) / kPromptRows : 0u;
    return s;
}

// What the rows of one tile see; a tile that sees nothing gets one masked piece, so that its rows are written.
__device__ __forceinline__ Span prompt_span(const PromptSeq& s, const Query& q, uint32_t tile)
{
    const int first = s.len - s.rows, from = first + (int)(tile * kPromptRows / q.group);
    const int to = first + (int)(min((uint32_t)s.rows * q.group - 1u, tile * kPromptRows + kPromptRows - 1u) / q.group);
    if (s.len == 0 || to < 0) return Span{0u, 0u, 1u};
    return span_of(max(0, from), to, q.window, q.sinks, 7u);
}

// Line length of a sequence for one head; the lanes of a warp share the tiles.
__device__ __forceinline__ uint32_t prompt_weight(const PromptSeq& s, const Query& q)
{
    uint32_t w = 0;
    for (uint32_t tile = threadIdx.x & 31u; tile < s.tiles; tile += 32u) w += kPromptUnitCost + prompt_span(s, q, tile).count;
#pragma unroll
    for (int d = 16; d; d >>= 1) w += __shfl_xor_sync(0xffffffffu, w, d);
    return w;
}

// A block's way along its share; every warp keeps one of its own and they all take the same steps.
struct PromptWalk {
    uint32_t x, end;                 // what is left of the share
    uint32_t b, head, tile, begin;   // the current unit and where it begins on the line
    PromptSeq seq;
    // of the unit that next() returned
    Span span;
    uint32_t from, to;               // pieces of this block
    uint32_t unit_first, unit_end;   // line places of the unit's first piece and of its end
    uint32_t unit_head, unit_tile;
    PromptSeq unit_seq;
    bool two;                        // more than 128 rows

    __device__ __forceinline__ bool next(const Kv& kv, const KvBatch& batch, const Query& q, uint32_t few_rows)
    {
        while (x < end) {
            if (seq.tiles == 0) {
                seq = prompt_seq(kv, batch, q, ++b, few_rows);
                continue;
            }
            span = prompt_span(seq, q, tile);
            unit_first = begin + kPromptUnitCost;
            unit_end = unit_first + span.count;
            const uint32_t a = max(x, unit_first), e = min(end, unit_end);
            const bool some = a < e;
            unit_head = head;
            unit_tile = tile;
            unit_seq = seq;
            if (some) {
                from = a - unit_first;
                to = e - unit_first;
                two = (uint32_t)seq.rows * q.group - tile * kPromptRows > 128u;
            }
            x = max(x, e);
            if (x >= unit_end) {
                begin = unit_end;
                if (++tile == seq.tiles) {
                    tile = 0;
                    if (++head == kv.heads) {
                        head = 0;
                        if (x < end) seq = prompt_seq(kv, batch, q, ++b, few_rows);
                    }
                }
            }
            if (some) return true;
        }
        return false;
    }
};

template <typename T, int kDim>
__global__ void __launch_bounds__(kPromptThreads, 1)
    prompt_attention_kernel(Kv kv, KvBatch batch, Query q, float* partials, uint32_t few_rows)
{
    constexpr uint32_t kSlabs = kPromptSlabs<kDim>, kTile = kSlabs * kSlabBytes;
    constexpr int kUnits = kDim / 8;             // 16-byte units of a row
    extern __shared__ unsigned char raw_shared[];
    unsigned char* tiles = raw_shared + ((1024u - (shared_address(raw_shared) & 1023u)) & 1023u);
    unsigned char* const q_tile = tiles;                     // [2] tiles
    unsigned char* const k_tile = tiles + 2 * kTile;         // [2] stages
    unsigned char* const v_tile = tiles + 4 * kTile;         // [2] stages
    PromptShared& sh = *(PromptShared*)(tiles + 6 * kTile);
    __shared__ uint32_t seq_weight[64];
    const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5;
    constexpr uint32_t kWarps = kPromptThreads / 32u;

    // ---- this block's share of the line
    uint32_t all = 0;
    for (uint32_t base = 0; base < batch.n; base += 64u) {
        __syncthreads();
        for (uint32_t i = warp; i < 64u && base + i < batch.n; i += kWarps) {
            const uint32_t w = prompt_weight(prompt_seq(kv, batch, q, base + i, few_rows), q);
            if (lane == 0) seq_weight[i] = w * kv.heads;
        }
        __syncthreads();
        uint32_t sum = 0;
        for (uint32_t i = lane; i < 64u && base + i < batch.n; i += 32u) sum += seq_weight[i];
#pragma unroll
        for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
        all += sum;
    }
    const uint32_t parts = min(gridDim.x, (all + kPromptMinPieces + kPromptUnitCost - 1u) / (kPromptMinPieces + kPromptUnitCost));
    if (blockIdx.x >= parts) return;
    const Shares shares(all, parts);
    PromptWalk walk;
    walk.x = shares.start(blockIdx.x);
    walk.end = shares.start(blockIdx.x + 1u);
    for (uint32_t base = 0, before = 0; base < batch.n; base += 64u) {
        if (batch.n > 64u) {
            __syncthreads();
            for (uint32_t i = warp; i < 64u && base + i < batch.n; i += kWarps) {
                const uint32_t w = prompt_weight(prompt_seq(kv, batch, q, base + i, few_rows), q);
                if (lane == 0) seq_weight[i] = w * kv.heads;
            }
            __syncthreads();
        }
        uint32_t b = base;
        for (; b < batch.n && b < base + 64u; ++b) {
            const uint32_t w = seq_weight[b - base];
            if (walk.x < before + w) break;
            before += w;
        }
        if (b < batch.n && b < base + 64u) {
            // head and tile inside the sequence
            const PromptSeq s = prompt_seq(kv, batch, q, b, few_rows);
            const uint32_t per_head = seq_weight[b - base] / kv.heads, head = (walk.x - before) / per_head;
            uint32_t at = before + head * per_head, tile = 0;
            for (uint32_t t0 = 0; t0 < s.tiles; t0 += 32u) {
                const uint32_t mine = t0 + lane < s.tiles ? kPromptUnitCost + prompt_span(s, q, t0 + lane).count : 0u;
                uint32_t sum = mine;
#pragma unroll
                for (int d = 1; d < 32; d <<= 1) {
                    const uint32_t y = __shfl_up_sync(0xffffffffu, sum, d);
                    if (lane >= (uint32_t)d) sum += y;
                }
                const uint32_t in = __ballot_sync(0xffffffffu, t0 + lane < s.tiles && walk.x < at + sum);
                if (in) {
                    const int l = __ffs(in) - 1;
                    tile = t0 + l;
                    at += __shfl_sync(0xffffffffu, sum - mine, l);
                    break;
                }
                at += __shfl_sync(0xffffffffu, sum, 31);
            }
            walk.b = b;
            walk.head = head;
            walk.tile = tile;
            walk.begin = at;
            walk.seq = s;
            break;
        }
    }

    // ---- barriers and tensor memory
    if (threadIdx.x == 0) {
        for (int i = 0; i < 2; ++i) {
            bar_init(&sh.q_full[i], 4);
            bar_init(&sh.k_full[i], 4);
            bar_init(&sh.k_empty[i], 1);
            bar_init(&sh.v_full[i], 4);
            bar_init(&sh.v_empty[i], 1);
            bar_init(&sh.s_full[i], 1);
            bar_init(&sh.p_full[i], 4);
            bar_init(&sh.o_full[i], 1);
            bar_init(&sh.joint[i], 4);
        }
        for (int i = 0; i < 4; ++i) bar_init(&sh.scale_full[i], 4);
        bar_init(&sh.drained, 1);
        sh.dead = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 12u) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(shared_address(&sh.tmem)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        tc_fence_before();
    }
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = sh.tmem;

    if (warp < 8u) {
        // =============================================================== softmax, one thread per row
        const uint32_t half = warp >> 2, row = threadIdx.x & 127u;
        const uint32_t lanes = (warp & 3u) << 21;            // lane field of a tensor memory address
        const uint32_t s_at = tmem + lanes + half * 128u, o_at = tmem + lanes + 256u + half * 128u;
        unsigned char* my_q = q_tile + half * kTile + row * 128u;
        uint32_t piece_count = 0, s_count = 0, unit_count = 0;   // pieces of the walk, of this half, units of this half
        uint32_t joints = 0;                                     // times this half's warps have met
        bool ok = true;
        auto meet = [&]() {
            __syncwarp();
            if (lane == 0) bar_arrive(&sh.joint[half]);
            return bar_wait(&sh.joint[half], joints++ & 1u, sh);
        };
        while (ok && walk.next(kv, batch, q, few_rows)) {
            const uint32_t pieces = walk.to - walk.from;
            if (half && !walk.two) {
                piece_count += pieces;
                continue;
            }
            const PromptSeq& seq = walk.unit_seq;
            const uint32_t r = walk.unit_tile * kPromptRows + half * 128u + row, rows = (uint32_t)seq.rows * q.group;
            const bool real = r < rows;
            const int first = seq.len - seq.rows;
            const int position = real ? first + (int)(r / q.group) : -1;
            const int64_t out_row = seq.row0 + (int)(r / q.group);
            const uint32_t query_head = walk.unit_head * q.group + r % q.group;
            // positions of the first and last row of this half
            const uint32_t r0 = walk.unit_tile * kPromptRows + half * 128u;
            const int low_position = first + (int)(r0 / q.group), high_position = first + (int)(min(rows - 1u, r0 + 127u) / q.group);

            // the row into shared memory, as fp16
            float row_factor = q.scale * kLog2e;
            {
                const uint4* from = (const uint4*)(q.q + out_row * q.q_row + (int64_t)query_head * q.q_head);
                float up = 1.f;
                if constexpr (!__is_same(T, __half)) {
                    float top = 0.f;
                    if (real) {
#pragma unroll
                        for (int u = 0; u < kUnits; ++u) {
                            const uint4 v = __ldg(from + u);
                            const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                const float2 f = to_float2<T>(w[e]);
                                top = fmaxf(top, fmaxf(fabsf(f.x), fabsf(f.y)));
                            }
                        }
                    }
                    const int e = row_exponent(top);
                    up = power_of_two(e);
                    row_factor *= power_of_two(-e);
                }
#pragma unroll
                for (int u = 0; u < kUnits; ++u) {
                    uint4 v = real ? __ldg(from + u) : make_uint4(0u, 0u, 0u, 0u);
                    if constexpr (!__is_same(T, __half)) {
                        uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const float2 f = to_float2<T>(w[e]);
                            w[e] = from_float2<__half>(f.x * up, f.y * up);
                        }
                        v = make_uint4(w[0], w[1], w[2], w[3]);
                    }
                    *(uint4*)(my_q + (u >> 3) * kSlabBytes + (((uint32_t)u & 7u) ^ (row & 7u)) * 16u) = v;
                }
                proxy_fence();
                __syncwarp();
                if (lane == 0) bar_arrive(&sh.q_full[half]);
            }

            float m = -INFINITY, l = 0.f;
            for (uint32_t j = 0; j < pieces; ++j, ++piece_count, ++s_count) {
                __syncwarp();
                const uint32_t ring = piece_count & 3u;
                const int t0 = (int)(walk.span.piece(walk.from + j) * 128u);
                const bool whole = t0 + 127 <= low_position &&
                                   (q.window == 0u || (int64_t)t0 > (int64_t)high_position - (int64_t)q.window || (uint32_t)t0 + 127u < q.sinks);
                // columns that this row sees: up to `upto`, and behind `after` or before `sinks`
                const int upto = max(-1, min(127, position - t0));
                const int after = q.window ? (int)max((int64_t)-1, min((int64_t)127, (int64_t)position - (int64_t)q.window - t0)) : -1;
                const int kept = (int)max((int64_t)0, min((int64_t)128, (int64_t)q.sinks - t0));
                ok = bar_wait(&sh.scale_full[ring], (piece_count >> 2) & 1u, sh) && bar_wait(&sh.s_full[half], s_count & 1u, sh);
                if (!ok) break;
                tc_fence_after();
                uint32_t s[32];
                float top = -INFINITY;
#pragma unroll 1
                for (int c = 0; c < 4; ++c) {
                    tm_load32(s_at + 32u * c, s);
                    tm_wait_load();
                    if (!whole) {
#pragma unroll
                        for (int e = 0; e < 32; ++e) {
                            const int col = 32 * c + e;
                            if (!(col <= upto && (col > after || col < kept))) s[e] = 0xff800000u;
                        }
                    }
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const float4 sc = sh.scales[ring][2 * c + h];
                        float best = __uint_as_float(s[16 * h]);
#pragma unroll
                        for (int e = 1; e < 16; ++e) best = fmaxf(best, __uint_as_float(s[16 * h + e]));
                        // a factor of 0 times minus infinity would be NaN
                        top = fmaxf(top, best == -INFINITY ? -INFINITY : fmaf(best, sc.x * row_factor, sc.y));
                    }
                }
                if (top > m + kGrowth || (m == -INFINITY && top > -INFINITY)) {
                    // handled below: the maximum moves
                } else {
                    top = m;
                }
                const float shrink = top == m ? 1.f : ex2(m - top);
                if (__any_sync(0xffffffffu, top != m) && j > 0) {
#pragma unroll 1
                    for (int c = 0; c < kDim / 32; ++c) {
                        tm_load32(o_at + 32u * c, s);
                        tm_wait_load();
#pragma unroll
                        for (int e = 0; e < 32; ++e) s[e] = __float_as_uint(__uint_as_float(s[e]) * shrink);
                        tm_store32(o_at + 32u * c, s);
                    }
                }
                l *= shrink;
                m = top;
                const float base = m == -INFINITY ? 0.f : m;
#pragma unroll 1
                for (int c = 0; c < 4; ++c) {
                    tm_load32(s_at + 32u * c, s);
                    tm_wait_load();
                    if (!whole) {
#pragma unroll
                        for (int e = 0; e < 32; ++e) {
                            const int col = 32 * c + e;
                            if (!(col <= upto && (col > after || col < kept))) s[e] = 0xff800000u;
                        }
                    }
                    uint32_t p[16];
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const float4 sc = sh.scales[ring][2 * c + h];
                        const float f = fmaxf(sc.x * row_factor, 1e-37f), add = sc.y - base;   // not 0, for the masked ones' sake
                        float sum = 0.f;
#pragma unroll
                        for (int e = 0; e < 16; e += 2) {
                            const float a = ex2(fmaf(__uint_as_float(s[16 * h + e]), f, add));
                            const float b = ex2(fmaf(__uint_as_float(s[16 * h + e + 1]), f, add));
                            sum += a + b;
                            p[8 * h + e / 2] = from_float2<__half>(a, b);
                        }
                        l = fmaf(sum, sc.z, l);
                    }
                    tm_store16(s_at + 16u * c, p);
                }
                tm_wait_store();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) bar_arrive(&sh.p_full[half]);
            }
            if (!ok) break;
            ok = bar_wait(&sh.o_full[half], unit_count & 1u, sh);
            if (!ok) break;
            tc_fence_after();
            ++unit_count;

            // ---- results
            const bool complete = pieces == walk.span.count;
            const float ref = value_reference(kv, seq.slot, walk.span.piece(0) << (7u - kv.page_shift), walk.unit_head);
            constexpr uint32_t kPartial = kPromptRows * (kDim + 2u);
            float* mine = partials + (uint64_t)(blockIdx.x * 2u + (walk.from == 0u ? 1u : 0u)) * kPartial + (half * 128u + row) * kDim;
            float* mine_stat = mine - (half * 128u + row) * kDim + kPromptRows * kDim + (half * 128u + row) * 2u;
            unsigned char* out = q.out + out_row * q.out_row + (int64_t)query_head * q.out_head;
            float* lse = q.lse && real ? q.lse + (uint64_t)out_row * q.heads + query_head : nullptr;
            const float by = l == 0.f ? 0.f : ref * __frcp_rn(l);
            uint32_t o[32];
#pragma unroll 1
            for (int c = 0; c < kDim / 32; ++c) {
                __syncwarp();
                tm_load32(o_at + 32u * c, o);
                tm_wait_load();
                if (complete && real) {
#pragma unroll
                    for (int e = 0; e < 32; e += 8) {
                        uint4 v;
                        v.x = from_float2<T>(__uint_as_float(o[e]) * by, __uint_as_float(o[e + 1]) * by);
                        v.y = from_float2<T>(__uint_as_float(o[e + 2]) * by, __uint_as_float(o[e + 3]) * by);
                        v.z = from_float2<T>(__uint_as_float(o[e + 4]) * by, __uint_as_float(o[e + 5]) * by);
                        v.w = from_float2<T>(__uint_as_float(o[e + 6]) * by, __uint_as_float(o[e + 7]) * by);
                        *(uint4*)(out + 64u * c + 2u * e) = v;
                    }
                } else if (real) {
#pragma unroll
                    for (int e = 0; e < 32; e += 4)
                        __stcg((float4*)(mine + 32u * c + e), make_float4(__uint_as_float(o[e]), __uint_as_float(o[e + 1]),
                                                                          __uint_as_float(o[e + 2]), __uint_as_float(o[e + 3])));
                }
            }
            __syncwarp();
            tc_fence_before();
            if (complete) {
                if (lse) *lse = l == 0.f ? -INFINITY : kLn2 * (m + log2f(l));
                continue;
            }
            if (real) __stcg((float2*)mine_stat, make_float2(m, l));
            const uint32_t c0 = shares.owner(walk.unit_first), c1 = shares.owner(walk.unit_end - 1u);
            __threadfence();
            ok = meet();
            if (!ok) break;
            if (row == 0) {
                uint32_t* counter = &kv.head->arrived[kPromptArrived + 2u * c0 + half];
                const uint32_t was = atomicAdd(counter, 1u);
                sh.last[half] = was == c1 - c0;
                if (was == c1 - c0) *counter = 0u;
            }
            ok = meet();
            if (!ok) break;
            if (*(volatile uint32_t*)&sh.last[half] && real) {
                __threadfence();
                // block c0 left the unit's beginning in its second place, the others theirs in the first
                auto place = [&](uint32_t c) { return partials + (uint64_t)(c * 2u + (c == c0 ? 1u : 0u)) * kPartial; };
                const uint32_t at = half * 128u + row;
                float top = -INFINITY, sum = 0.f;
                for (uint32_t c = c0; c <= c1; ++c) top = fmaxf(top, __ldcg(place(c) + kPromptRows * kDim + at * 2u));
                const float base = top == -INFINITY ? 0.f : top;
                for (uint32_t c = c0; c <= c1; ++c) {
                    const float2 ml = __ldcg((const float2*)(place(c) + kPromptRows * kDim + at * 2u));
                    sum = fmaf(ml.y, ex2(ml.x - base), sum);
                }
                const float f = sum == 0.f ? 0.f : ref * __frcp_rn(sum);
#pragma unroll 1
                for (int d = 0; d < kDim; d += 8) {
                    float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
                    for (uint32_t c = c0; c <= c1; ++c) {
                        const float* p = place(c);
                        const float w = ex2(__ldcg(p + kPromptRows * kDim + at * 2u) - base);
                        const float4 a = __ldcg((const float4*)(p + at * kDim + d)), b = __ldcg((const float4*)(p + at * kDim + d + 4));
                        v[0] = fmaf(a.x, w, v[0]);
                        v[1] = fmaf(a.y, w, v[1]);
                        v[2] = fmaf(a.z, w, v[2]);
                        v[3] = fmaf(a.w, w, v[3]);
                        v[4] = fmaf(b.x, w, v[4]);
                        v[5] = fmaf(b.y, w, v[5]);
                        v[6] = fmaf(b.z, w, v[6]);
                        v[7] = fmaf(b.w, w, v[7]);
                    }
                    *(uint4*)(out + 2u * d) = make_uint4(from_float2<T>(v[0] * f, v[1] * f), from_float2<T>(v[2] * f, v[3] * f),
                                                         from_float2<T>(v[4] * f, v[5] * f), from_float2<T>(v[6] * f, v[7] * f));
                }
                if (lse) *lse = sum == 0.f ? -INFINITY : kLn2 * (top + log2f(sum));
            }
            ok = meet();             // last[] has been read
        }
    } else if (warp < 12u) {
        // =============================================================== cache bytes to fp16 tiles
        const uint32_t w = warp - 8u;
        // eight lanes of a quarter warp write rows {0, 1, 4, 5} or {2, 3, 6, 7} of two neighbouring chunks: under the
        // swizzle that is eight different 16-byte bank groups
        const uint32_t sub_row = (lane >> 1 & 1u) | (lane >> 2 & 1u) << 2 | (lane >> 3 & 1u) << 1;
        const uint32_t chunk = (lane & 1u) | (lane >> 4) << 1;
        constexpr int kHalves = kDim == 64 ? 1 : 2;                              // 64-byte parts of a cache row
        const bool in_second = kDim != 96 || chunk < 2u;
        uint32_t count = 0;                                                      // pieces of the walk
        bool ok = true;
        uint4 kb[4][kHalves], vb[4][kHalves];
        float key_scale = 0.f, value_scale = 0.f;
        int page[2] = {-1, -1};
        uint32_t inside[2] = {0u, 0u};
        auto find = [&](uint32_t piece) {
            const PromptSeq& seq = walk.unit_seq;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint32_t token = piece * 128u + w * 32u + h * 16u;
                page[h] = seq.slot >= 0 && token < (uint32_t)seq.len ? kv_page(kv, seq.slot, token >> kv.page_shift) : -1;
                inside[h] = token & (kv.page() - 1u);
            }
        };
        auto load = [&](uint4(&to)[4][kHalves], uint32_t which) {
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int p = page[g >> 1];
                const uint8_t* at = kv.codes + (uint64_t)(uint32_t)max(p, 0) * kv.page_bytes() +
                                    (uint64_t)(which * kv.heads + walk.unit_head) * kv.head_bytes() +
                                    (inside[g >> 1] + 8u * (g & 1) + sub_row) * kDim + chunk * 16u;
#pragma unroll
                for (int h = 0; h < kHalves; ++h)
                    to[g][h] = p >= 0 && (h == 0 || in_second) ? __ldg((const uint4*)(at + 64u * h))
                                                               : make_uint4(0x80808080u, 0x80808080u, 0x80808080u, 0x80808080u);
            }
        };
        auto store = [&](const uint4(&from)[4][kHalves], unsigned char* tile) {
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const uint32_t r = w * 32u + 8u * g + sub_row;
#pragma unroll
                for (int h = 0; h < kHalves; ++h) {
                    if (h == 1 && !in_second) continue;
                    unsigned char* to = tile + h * kSlabBytes + r * 128u;
                    const uint4 c = from[g][h];
                    *(uint4*)(to + ((2u * chunk) ^ (r & 7u)) * 16u) = make_uint4(codes_low(c.x), codes_high(c.x), codes_low(c.y), codes_high(c.y));
                    *(uint4*)(to + ((2u * chunk + 1u) ^ (r & 7u)) * 16u) = make_uint4(codes_low(c.z), codes_high(c.z), codes_low(c.w), codes_high(c.w));
                }
            }
            proxy_fence();
            __syncwarp();
        };
        while (ok && walk.next(kv, batch, q, few_rows)) {
            const float by_ref =
                __frcp_rn(value_reference(kv, walk.unit_seq.slot, walk.span.piece(0) << (7u - kv.page_shift), walk.unit_head));
            for (uint32_t j = walk.from; j < walk.to; ++j, ++count) {
                find(walk.span.piece(j));
                load(kb, 0u);
                load(vb, 1u);
                if (lane < 2u) {
                    const int p = lane ? page[1] : page[0];
                    if (p >= 0) {
                        const float* at = kv.scales + (uint64_t)(uint32_t)p * 2u * kv.heads + walk.unit_head;
                        key_scale = __ldg(at);
                        value_scale = __ldg(at + kv.heads);
                    }
                }
                const uint32_t stage = count & 1u, parity = (count >> 1 & 1u) ^ 1u;
                ok = bar_wait(&sh.k_empty[stage], parity, sh);
                if (!ok) break;
                if (lane < 2u) {
                    // the scales of a piece four places back are no longer read: its S tiles have been followed by newer ones
                    const int p = lane ? page[1] : page[0];
                    const float rel = relative_scale(value_scale, by_ref);
                    sh.scales[count & 3u][2u * w + lane] =
                        p >= 0 ? make_float4(key_scale, lg2(rel), rcp(rel), 0.f) : make_float4(0.f, -INFINITY, 0.f, 0.f);
                }
                store(kb, k_tile + stage * kTile);
                if (lane == 0) {
                    bar_arrive(&sh.scale_full[count & 3u]);
                    bar_arrive(&sh.k_full[stage]);
                }
                ok = bar_wait(&sh.v_empty[stage], parity, sh);
                if (!ok) break;
                store(vb, v_tile + stage * kTile);
                if (lane == 0) bar_arrive(&sh.v_full[stage]);
            }
        }
    } else {
        // =============================================================== products, one thread
        if (lane == 0) {
            const uint32_t q_at = shared_address(q_tile), k_at = shared_address(k_tile), v_at = shared_address(v_tile);
            auto scores = [&](uint32_t half, uint32_t stage) {
#pragma unroll
                for (int k = 0; k < kDim / 16; ++k) {
                    const uint32_t off = (uint32_t)(k >> 2) * kSlabBytes + (uint32_t)(k & 3) * 32u;
                    tc_product_shared(tmem + half * 128u, tile_descriptor(q_at + half * kTile + off, 16u),
                                      tile_descriptor(k_at + stage * kTile + off, 16u), product_descriptor(128u, false), k > 0);
                }
            };
            auto outputs = [&](uint32_t half, uint32_t stage, bool add) {
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    tc_product_tensor(tmem + 256u + half * 128u, tmem + half * 128u + 8u * k,
                                      tile_descriptor(v_at + stage * kTile + 2048u * k, kSlabBytes), product_descriptor(kDim, true),
                                      k > 0 || add);
            };
            uint32_t count = 0, s_count[2] = {0u, 0u}, units[2] = {0u, 0u};
            bool ok = true;
            while (ok && walk.next(kv, batch, q, few_rows)) {
                const uint32_t pieces = walk.to - walk.from;
                const bool two = walk.two;
                ok = bar_wait_one(&sh.q_full[0], units[0]++ & 1u, sh) && (!two || bar_wait_one(&sh.q_full[1], units[1]++ & 1u, sh));
                for (uint32_t j = 0; ok && j < pieces; ++j, ++count) {
                    const uint32_t stage = count & 1u, parity = count >> 1 & 1u;
                    ok = bar_wait_one(&sh.k_full[stage], parity, sh);
                    if (!ok) break;
                    tc_fence_after();
                    scores(0u, stage);
                    tc_commit(&sh.s_full[0]);
                    if (two) {
                        if (j > 0) {
                            ok = bar_wait_one(&sh.p_full[1], s_count[1]++ & 1u, sh);
                            if (!ok) break;
                            tc_fence_after();
                            outputs(1u, stage ^ 1u, j > 1);
                            tc_commit(&sh.v_empty[stage ^ 1u]);
                        }
                        scores(1u, stage);
                        tc_commit(&sh.s_full[1]);
                    }
                    tc_commit(&sh.k_empty[stage]);
                    ok = bar_wait_one(&sh.v_full[stage], parity, sh) && bar_wait_one(&sh.p_full[0], s_count[0]++ & 1u, sh);
                    if (!ok) break;
                    tc_fence_after();
                    outputs(0u, stage, j > 0);
                    if (!two) tc_commit(&sh.v_empty[stage]);
                    if (j + 1u == pieces) tc_commit(&sh.o_full[0]);
                }
                if (ok && two) {
                    ok = bar_wait_one(&sh.p_full[1], s_count[1]++ & 1u, sh);
                    if (!ok) break;
                    tc_fence_after();
                    outputs(1u, (count - 1u) & 1u, pieces > 1u);
                    tc_commit(&sh.v_empty[(count - 1u) & 1u]);
                    tc_commit(&sh.o_full[1]);
                }
            }
            if (!ok) {               // given up: say so, and let the products that were issued end
                atomicOr(&kv.head->status, kKvStatInternal);
                sh.dead = 0;
                tc_commit(&sh.drained);
                bar_wait_one(&sh.drained, 0u, sh);
            }
        }
        __syncwarp();
    }
    // every product has been waited for by the warps that read its result, or above
    __syncthreads();
    if (warp == 12u) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem));
    }
}

template <typename T, int kDim>
cudaError_t launch_prompt(const Kv& kv, const KvBatch& batch, const Query& q, uint32_t few_rows, uint32_t sm_count, float* partials,
                          cudaStream_t s)
{
    auto* kernel = prompt_attention_kernel<T, kDim>;
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kPromptSmem<kDim>);
    if (e != cudaSuccess) return e;
    kernel<<<min(kPromptBlocks, sm_count), kPromptThreads, kPromptSmem<kDim>, s>>>(kv, batch, q, partials, few_rows);
    return cudaGetLastError();
}

}  // namespace
}  // namespace entro
