// Weight gradient of the first dense stage of an LC model on a mini-batch of rows (the stage: lc_layer.cu):
//
//   dWt[h][f] = sum_k sum_i dZ_k[i][h] X_k[batch[i]][f],   dZ_k = dY_k where Y_k > 0 (hops with ReLU), dY_k (the others)
//
// One pass over dY, Y and the gathered rows of X; neither dZ nor the gathered rows exist as matrices.  A product whose sum runs
// over the batch: a CTA takes a tile of 128 x up to 128 of dWt and a share of the batch of all hops, and leaves its sums in the
// workspace, which a second kernel adds up in a fixed order.
//
//   warps 0-7    add up.  They read finished accumulators out of tensor memory and add them, rounded to nearest, to sums in
//                registers (the tensor core cuts what an addition drops, so long sums in one accumulator come out too small).
//   warps 8-11   operand A = dZ^T: a lane has one column h and reads it in the 32 rows of a chunk, masks, splits, and stores it to
//                tensor memory, where a lane is a row of A.
//   warps 12-15  operand B = the gathered rows of X: split and laid down in shared memory as they lie, rows along K.
//   warps 16-19  copy chunks of dY, Y and the gathered rows into shared memory, asynchronously and as many chunks ahead as there is
//                room for: no register holds what is in flight, and zeros fill what does not exist.  (Read by the splitting warps
//                themselves, 32 rows at a time: 9.2 us a chunk, 28.6 ms for 2.4 M rows x 3 hops, F = 100, hidden 256.)
//   warp 20      issues the products.
//
// Numbers.  An fp32 operand is the sum of three bf16 numbers, cut one after the other from its 24 bits, so nothing is lost and any
// scale fits; of the nine products the six largest are taken, which drops less than 2^-23 of |dZ||X| per term.  (Two fp16 numbers
// and three products would need a scale known before the data is read.)
//
// Tensor memory: two accumulators of 128 columns in turn, then 48 columns (three parts of 16: two elements of K per column) for each
// of five chunks of A.  What A takes there it neither writes to nor is read from shared memory, whose bandwidth B alone then
// needs.
#include <algorithm>
#include <atomic>

#include "dense.cuh"
#include "tensor_core.cuh"

namespace gnnpre {
namespace {

constexpr int kGradTile = 128;        // rows (h) of a tile, columns (f) at most
constexpr int kGradChunk = 32;        // batch rows per stage
constexpr int kGradRaw = 3;           // chunks being copied or split
constexpr int kGradStages = 3;        // chunks split
constexpr int kGradSlice = 2;         // chunks whose products share an accumulator
constexpr int kGradSumWarps = 8, kGradBWarp = 12, kGradCopyWarp = 16, kGradMmaWarp = 20, kGradWarps = 24;
constexpr int kGradThreads = 32 * kGradWarps;            // (whole warpgroups, for the registers they hand on)
constexpr uint32_t kGradMatrix = kGradChunk * kGradTile * 4;  // a chunk of dY, Y or X as copied: 32 rows of 512 bytes
constexpr uint32_t kGradRawStage = 3 * kGradMatrix;
constexpr uint32_t kGradPart = 2 * kGradChunk * 128;     // one part of B's chunk: two blocks of 64 columns, 32 rows of 128 bytes
constexpr uint32_t kGradStage = 3 * kGradPart;
constexpr uint32_t kGradTmem = 512, kGradTmemA = 256, kGradTmemStage = 48;
constexpr int kGradSmem = kGradStages * (int)kGradStage + kGradRaw * (int)kGradRawStage + 1024;
// Registers per thread: 768 threads start with 80, 61,440 in all; 2 x 128 x 104 + 128 x (96 + 80 + 56 + 24) = 59,392.
constexpr int kRegsSum = 104, kRegsA = 96, kRegsCopy = 56, kRegsMma = 24;

struct GradArgs {
    const float* hop[GNNPRE_MAX_HOPS];
    int64_t ldh, n;
    int32_t feat_dim, hidden, num_hops;
    const int32_t* batch;
    int64_t batch_size;
    const float* dy;
    int64_t lddy, dy_hop;
    const float* y;
    int64_t ldy, y_hop;
    uint64_t relu_mask;
    int32_t tiles_f, width;     // tiles of `width` features (a multiple of 16)
    int32_t tiles;              // of dWt
    int32_t splits;
    int64_t chunks_per_hop, chunks;
    float* parts;               // [splits][hidden][part_ld]
    int64_t part_ld;
    int32_t* error;
    uint32_t spin_limit;
    int32_t wide;               // rows of dY and Y start on 16-byte boundaries
    int32_t drop;               // self-test: chunks that are complete are not announced
};

// v = h + m + l, each with the upper 16 bits of an fp32 number only.
struct Parts {
    uint32_t h, m, l;
};
__device__ __forceinline__ Parts cut(float v) {
    Parts p;
    p.h = __float_as_uint(v);
    const float r = v - __uint_as_float(p.h & 0xffff0000u);
    p.m = __float_as_uint(r);
    p.l = __float_as_uint(r - __uint_as_float(p.m & 0xffff0000u));
    return p;
}
// The upper halves of two numbers, the first one low.
__device__ __forceinline__ uint32_t pack(uint32_t a, uint32_t b) { return __byte_perm(a, b, 0x7632); }

template <int REGS>
__device__ __forceinline__ void more_registers() {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(REGS));
}
template <int REGS>
__device__ __forceinline__ void fewer_registers() {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(REGS));
}

// BYTES bytes global -> shared without passing through registers, or as many zeros.
template <int BYTES>
__device__ __forceinline__ void grad_copy(uint32_t dst, const float* src, bool live) {
    const int size = live ? BYTES : 0;
    if (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(size) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(size) : "memory");
}

__device__ __forceinline__ float4 grad_read4(uint32_t at) {
    float4 v;
    asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(at) : "memory");
    return v;
}
__device__ __forceinline__ float grad_read(uint32_t at) {
    float v;
    asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v) : "r"(at) : "memory");
    return v;
}

__global__ void __launch_bounds__(kGradThreads, 1) k_lc_grad(const __grid_constant__ GradArgs a) {
    extern __shared__ unsigned char grad_smem[];
    __shared__ __align__(8) unsigned long long bars[2 * kGradStages + 2 * kGradRaw + 5];
    __shared__ uint32_t tmem_slot;
    __shared__ int abort_word;
    volatile int* abort_flag = &abort_word;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t base = (tc_smem(grad_smem) + 1023u) & ~1023u;
    const uint32_t raw0 = base + kGradStages * kGradStage;
    const uint32_t bar0 = tc_smem(&bars[0]);
    auto full = [&](int s) { return bar0 + 8u * s; };
    auto empty = [&](int s) { return bar0 + 8u * (kGradStages + s); };
    auto raw_full = [&](int s) { return bar0 + 8u * (2 * kGradStages + s); };
    auto raw_empty = [&](int s) { return bar0 + 8u * (2 * kGradStages + kGradRaw + s); };
    constexpr int kRest = 2 * kGradStages + 2 * kGradRaw;
    auto acc_full = [&](int b) { return bar0 + 8u * (kRest + b); };
    auto acc_empty = [&](int b) { return bar0 + 8u * (kRest + 2 + b); };
    const uint32_t drained = bar0 + 8u * (kRest + 4);
    if (threadIdx.x == 0) {
        for (int s = 0; s < kGradStages; ++s) {
            tc_bar_init(full(s), 8 + (a.drop ? 1 : 0));  // a lane of each splitting warp
            tc_bar_init(empty(s), 1);
        }
        for (int s = 0; s < kGradRaw; ++s) {
            tc_bar_init(raw_full(s), 128);               // every copying thread, once its copies have landed
            tc_bar_init(raw_empty(s), 8);
        }
        for (int b = 0; b < 2; ++b) {
            tc_bar_init(acc_full(b), 1);
            tc_bar_init(acc_empty(b), kGradSumWarps);
        }
        tc_bar_init(drained, 1);
        abort_word = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == kGradMmaWarp) tc_alloc(tc_smem(&tmem_slot), kGradTmem);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_slot;

    // neighbouring CTAs take the tiles of one share of the batch, whose rows they then find in the L2
    const int tile = blockIdx.x % a.tiles, split = blockIdx.x / a.tiles;
    const int h0 = tile / a.tiles_f * kGradTile, f0 = tile % a.tiles_f * a.width;
    const int64_t first = a.chunks * split / a.splits, last = a.chunks * (split + 1) / a.splits;
    const int count = (int)(last - first), slices = (count + kGradSlice - 1) / kGradSlice;
    auto hop_of = [&](int64_t chunk) { return (int)(chunk / a.chunks_per_hop); };

    if (warp < kGradSumWarps) {
        more_registers<kRegsSum>();
        const int q = warp & 3, half = warp >> 2;
        constexpr int kCols = kGradTile / 2;
        float sum[kCols];
#pragma unroll
        for (int j = 0; j < kCols; ++j) sum[j] = 0.f;
        const uint32_t taddr = tmem + ((uint32_t)(32 * q) << 16) + half * kCols;
        bool ok = true;
        for (int i = 0; i < slices; ++i) {
            ok = tc_wait_warp(acc_full(i & 1), (uint32_t)(i >> 1) & 1u, abort_flag, a.error, a.spin_limit);
            if (!ok) break;
            tc_fence_after();
#pragma unroll
            for (int part = 0; part < kCols / 32; ++part) {
                if (half * kCols + 32 * part >= a.width) continue;
                uint32_t v[32];
                tc_load32(taddr + (uint32_t)(i & 1) * kGradTile + 32 * part, v);
                tc_load_wait();
#pragma unroll
                for (int j = 0; j < 32; ++j) sum[32 * part + j] += __uint_as_float(v[j]);
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) tc_bar_arrive(acc_empty(i & 1));
        }
        const int h = h0 + 32 * q + lane;
        if (ok && h < a.hidden) {
            float* dst = a.parts + ((int64_t)split * a.hidden + h) * a.part_ld + f0 + half * kCols;
#pragma unroll
            for (int j = 0; j < kCols; j += 4)  // (rows of parts have room for whole tiles)
                if (half * kCols + j < a.width)
                    *reinterpret_cast<float4*>(dst + j) = make_float4(sum[j], sum[j + 1], sum[j + 2], sum[j + 3]);
        }
    } else if (warp < kGradBWarp) {
        more_registers<kRegsA>();
        const int q = warp & 3;
        const uint32_t column = 4u * (32 * q + lane);
        for (int c = 0; c < count; ++c) {
            const int s = c % kGradStages, r0 = c % kGradRaw;
            const bool relu = (a.relu_mask >> hop_of(first + c)) & 1u;
            if (!tc_wait_warp(raw_full(r0), (uint32_t)(c / kGradRaw) & 1u, abort_flag, a.error, a.spin_limit)) break;
            const uint32_t dy = raw0 + r0 * kGradRawStage + column, y = dy + kGradMatrix;
            float v[kGradChunk];
#pragma unroll
            for (int r = 0; r < kGradChunk; ++r) v[r] = grad_read(dy + 4u * kGradTile * r);
            if (relu) {
#pragma unroll
                for (int r = 0; r < kGradChunk; ++r) v[r] = grad_read(y + 4u * kGradTile * r) > 0.f ? v[r] : 0.f;
            }
            __syncwarp();
            if (lane == 0) tc_bar_arrive(raw_empty(r0));
            if (!tc_wait_warp(empty(s), ((uint32_t)(c / kGradStages) & 1u) ^ 1u, abort_flag, a.error, a.spin_limit)) break;
            tc_fence_after();
            uint32_t p[3][16];
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                const Parts e = cut(v[2 * j]), o = cut(v[2 * j + 1]);
                p[0][j] = pack(e.h, o.h);
                p[1][j] = pack(e.m, o.m);
                p[2][j] = pack(e.l, o.l);
            }
            const uint32_t to = tmem + ((uint32_t)(32 * q) << 16) + kGradTmemA + kGradTmemStage * s;
#pragma unroll
            for (int i = 0; i < 3; ++i) tc_store16(to + 16 * i, p[i]);
            tc_store_wait();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) tc_bar_arrive(full(s));
        }
    } else if (warp < kGradCopyWarp) {
        const int w = warp - kGradBWarp, col = 4 * lane;  // of the tile
        constexpr int kRows = kGradChunk / 4;
        for (int c = 0; c < count; ++c) {
            const int s = c % kGradStages, r0 = c % kGradRaw;
            if (!tc_wait_warp(raw_full(r0), (uint32_t)(c / kGradRaw) & 1u, abort_flag, a.error, a.spin_limit)) break;
            const uint32_t from = raw0 + r0 * kGradRawStage + 2 * kGradMatrix + 16u * lane;
            float4 v[kRows];
#pragma unroll
            for (int i = 0; i < kRows; ++i) v[i] = grad_read4(from + 4u * kGradTile * (w * kRows + i));
            __syncwarp();
            if (lane == 0) tc_bar_arrive(raw_empty(r0));
            if (!tc_wait_warp(empty(s), ((uint32_t)(c / kGradStages) & 1u) ^ 1u, abort_flag, a.error, a.spin_limit)) break;
            const uint32_t to = base + (uint32_t)s * kGradStage + (col / 64) * (kGradChunk * 128) + (col % 8) * 2;
#pragma unroll
            for (int i = 0; i < kRows; ++i) {
                const int k = w * kRows + i;
                const Parts x = cut(v[i].x), y = cut(v[i].y), z = cut(v[i].z), u = cut(v[i].w);
                const uint32_t at = to + 128u * k + ((uint32_t)((col % 64 / 8) ^ (k & 7)) << 4);
                asm volatile("st.shared.v2.b32 [%0], {%1, %2};" ::"r"(at), "r"(pack(x.h, y.h)), "r"(pack(z.h, u.h)) : "memory");
                asm volatile("st.shared.v2.b32 [%0], {%1, %2};" ::"r"(at + kGradPart), "r"(pack(x.m, y.m)), "r"(pack(z.m, u.m)) : "memory");
                asm volatile("st.shared.v2.b32 [%0], {%1, %2};" ::"r"(at + 2 * kGradPart), "r"(pack(x.l, y.l)), "r"(pack(z.l, u.l)) : "memory");
            }
            tc_fence_async();
            __syncwarp();
            if (lane == 0) tc_bar_arrive(full(s));
        }
    } else if (warp < kGradMmaWarp) {
        fewer_registers<kRegsCopy>();
        const int w = warp - kGradCopyWarp;
        constexpr int kRows = kGradChunk / 4;
        const int col = 4 * lane;  // of the tile
        const int left = col < a.width ? a.feat_dim - f0 - col : 0;  // features from here on
        const bool column = h0 + col < a.hidden;                     // (hidden is a multiple of 16)
        // the hop matrix's row of this lane's row of a chunk; -1: there is none
        auto row_index = [&](int64_t chunk) {
            const int64_t pos = (chunk - hop_of(chunk) * a.chunks_per_hop) * kGradChunk + lane;
            if (pos >= a.batch_size) return -1;
            const int64_t r = a.batch ? (int64_t)__ldg(a.batch + pos) : pos;
            return r >= 0 && r < a.n ? (int)r : -1;
        };
        int row = count > 0 ? row_index(first) : -1;
        for (int c = 0; c < count; ++c) {
            const int next = c + 1 < count ? row_index(first + c + 1) : -1;  // a chunk ahead
            const int64_t chunk = first + c;
            const int hop = hop_of(chunk), r0 = c % kGradRaw;
            const int64_t row0 = (chunk - hop * a.chunks_per_hop) * kGradChunk + w * kRows;
            const bool relu = (a.relu_mask >> hop) & 1u;
            if (!tc_wait_warp(raw_empty(r0), ((uint32_t)(c / kGradRaw) & 1u) ^ 1u, abort_flag, a.error, a.spin_limit)) break;
            const uint32_t to = raw0 + r0 * kGradRawStage + 4u * kGradTile * (w * kRows);
            const float* x = a.hop[hop] + f0 + col;
            auto copy_rows = [&](uint32_t dst, const float* src, int64_t ld) {
                if (a.wide) {
                    src += h0 + col;
#pragma unroll
                    for (int i = 0; i < kRows; ++i) {
                        const bool there = __shfl_sync(0xffffffffu, row, w * kRows + i) >= 0, live = there && column;
                        grad_copy<16>(dst + 4u * kGradTile * i + 16u * lane, live ? src + i * ld : a.dy, live);
                    }
                } else {
                    src += h0 + lane;
#pragma unroll
                    for (int i = 0; i < kRows; ++i) {
                        const bool there = __shfl_sync(0xffffffffu, row, w * kRows + i) >= 0;
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const bool live = there && h0 + 32 * j + lane < a.hidden;
                            grad_copy<4>(dst + 4u * kGradTile * i + 128u * j + 4u * lane, live ? src + i * ld + 32 * j : a.dy, live);
                        }
                    }
                }
            };
            copy_rows(to, a.dy + hop * a.dy_hop + row0 * a.lddy, a.lddy);
            if (relu) copy_rows(to + kGradMatrix, a.y + hop * a.y_hop + row0 * a.ldy, a.ldy);
#pragma unroll
            for (int i = 0; i < kRows; ++i) {
                const int r = __shfl_sync(0xffffffffu, row, w * kRows + i);
                const uint32_t dst = to + 2 * kGradMatrix + 4u * kGradTile * i + 16u * lane;
                const float* src = x + (int64_t)max(r, 0) * a.ldh;
                if (left >= 4 || left <= 0) {
                    grad_copy<16>(dst, left > 0 && r >= 0 ? src : a.hop[hop], left > 0 && r >= 0);
                } else {  // the last features, without what lies behind them
#pragma unroll
                    for (int j = 0; j < 4; ++j) grad_copy<4>(dst + 4u * j, j < left && r >= 0 ? src + j : a.hop[hop], j < left && r >= 0);
                }
            }
            asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(raw_full(r0)) : "memory");
            row = next;
        }
        asm volatile("cp.async.wait_all;" ::: "memory");  // nothing may land after this CTA has left
    } else {
        fewer_registers<kRegsMma>();
        if (warp == kGradMmaWarp) {
            const uint32_t instr = tc_instr(kGradTile, a.width, true, true);
            bool ok = true;
            for (int i = 0, c = 0; i < slices && ok; ++i) {
                ok = tc_wait_warp(acc_empty(i & 1), ((uint32_t)(i >> 1) & 1u) ^ 1u, abort_flag, a.error, a.spin_limit);
                for (const int start = c; ok && c < min(start + kGradSlice, count); ++c) {
                    const int s = c % kGradStages;
                    ok = tc_wait_warp(full(s), (uint32_t)(c / kGradStages) & 1u, abort_flag, a.error, a.spin_limit);
                    if (!ok) break;
                    tc_fence_after();
                    const uint32_t d = tmem + (uint32_t)(i & 1) * kGradTile, am = tmem + kGradTmemA + kGradTmemStage * s;
                    const uint32_t at = base + (uint32_t)s * kGradStage;
                    const uint64_t b[3] = {tc_desc_mn(at, kGradChunk * 128), tc_desc_mn(at + kGradPart, kGradChunk * 128),
                                           tc_desc_mn(at + 2 * kGradPart, kGradChunk * 128)};
                    // the small terms first
                    constexpr int kA[6] = {1, 2, 0, 1, 0, 0}, kB[6] = {1, 0, 2, 0, 1, 0};
#pragma unroll
                    for (int t = 0; t < 6; ++t)
#pragma unroll
                        for (int j = 0; j < kGradChunk / 16; ++j)
                            tc_mma_ta(d, am + 16 * kA[t] + 8 * j, b[kB[t]] + (2048 >> 4) * j, instr, c != start || t != 0 || j != 0);
                    tc_commit(empty(s));
                }
                if (ok) tc_commit(acc_full(i & 1));
            }
            tc_commit(drained);
            for (uint32_t i = 0; i < kTcSpinLimit; ++i)
                if (tc_bar_test(drained, 0)) break;
            __syncwarp();
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == kGradMmaWarp) {
        tc_fence_after();
        tc_free(tmem, kGradTmem);
    }
}

// Sums of the splits' parts, in their order within each of eight interleaved groups, the groups in theirs.
constexpr int kJoinGroups = 8;
__global__ void __launch_bounds__(32 * kJoinGroups) k_lc_grad_join(const float* parts, int64_t part_ld, int32_t splits, int32_t hidden,
                                                                   int32_t feat_dim, int32_t accumulate, float* dw, int64_t ldw) {
    wait_previous_kernel();
    __shared__ float4 room[kJoinGroups][32];
    const int lane = threadIdx.x & 31, group = threadIdx.x >> 5;
    const int h = blockIdx.y, f = (blockIdx.x * 32 + lane) * 4;
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
    if (f < feat_dim)
#pragma unroll 4
        for (int p = group; p < splits; p += kJoinGroups) {
            const float4 v = *reinterpret_cast<const float4*>(parts + ((int64_t)p * hidden + h) * part_ld + f);
            s.x += v.x;
            s.y += v.y;
            s.z += v.z;
            s.w += v.w;
        }
    room[group][lane] = s;
    __syncthreads();
    if (group != 0 || f >= feat_dim) return;
#pragma unroll
    for (int g = 1; g < kJoinGroups; ++g) {
        const float4 v = room[g][lane];
        s.x += v.x;
        s.y += v.y;
        s.z += v.z;
        s.w += v.w;
    }
    float* dst = dw + (int64_t)h * ldw + f;
    const float o[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (f + e < feat_dim) dst[e] = accumulate ? dst[e] + o[e] : o[e];
}

struct GradShape {
    int32_t tiles_f, width, tiles, splits;
    int64_t chunks_per_hop, chunks, part_ld, bytes;
};

// As many shares of the batch as the SMs have room for beside the tiles, each of at least one chunk.
GradShape grad_shape(int64_t num_hops, int64_t batch_size, int64_t feat_dim, int64_t hidden, int sms) {
    GradShape g{};
    const int64_t tiles_h = (hidden + kGradTile - 1) / kGradTile;
    g.tiles_f = (int32_t)((feat_dim + kGradTile - 1) / kGradTile);
    g.width = (int32_t)(((feat_dim + g.tiles_f - 1) / g.tiles_f + 15) / 16 * 16);
    g.tiles_f = (int32_t)((feat_dim + g.width - 1) / g.width);
    g.tiles = (int32_t)(tiles_h * g.tiles_f);
    g.chunks_per_hop = (batch_size + kGradChunk - 1) / kGradChunk;
    g.chunks = num_hops * g.chunks_per_hop;
    g.splits = (int32_t)std::max<int64_t>(1, std::min<int64_t>(g.chunks, sms / g.tiles));
    g.part_ld = (int64_t)g.tiles_f * g.width;
    g.bytes = (int64_t)4 * g.splits * hidden * g.part_ld;
    return g;
}

// More than any device of this architecture has, for a size that does not depend on the device.
constexpr int kMostSms = 192;

int check_grad(int64_t num_hops, int64_t batch_size, int64_t feat_dim, int64_t hidden) {
    if (num_hops < 1 || num_hops > GNNPRE_MAX_HOPS || batch_size < 0 || batch_size > INT32_MAX || feat_dim < 1 || feat_dim > (1 << 20))
        return GNNPRE_ERR_INVALID_ARG;
    if (hidden < 16 || hidden > 256 || hidden % 16 != 0) return GNNPRE_ERR_INVALID_ARG;
    return GNNPRE_OK;
}

int grad_launch(const float* const* hops, int32_t num_hops, int64_t n, int64_t feat_dim, int64_t ldh, const int32_t* batch,
                int64_t batch_size, const float* dY, int64_t lddy, int64_t dy_hop, const float* Y, int64_t ldy, int64_t y_hop,
                uint64_t relu_mask, int64_t hidden, int32_t accumulate, float* dWt, int64_t ldw, void* workspace, int64_t workspace_bytes,
                int32_t* error_flag, void* stream, bool drop = false, uint32_t polls = kTcSpinLimit) {
    GNNPRE_TRY(check_grad(num_hops, batch_size, feat_dim, hidden));
    if (!hops || n < 1 || n > INT32_MAX || !dWt || ldw < feat_dim || ldh < feat_dim) return GNNPRE_ERR_INVALID_ARG;
    const uint64_t used = relu_mask & (num_hops == 64 ? ~0ull : (1ull << num_hops) - 1);
    if (batch_size > 0 && (!dY || !workspace || (used && !Y) || lddy < hidden || (used && ldy < hidden))) return GNNPRE_ERR_INVALID_ARG;
    if (!batch && batch_size > n) return GNNPRE_ERR_INVALID_ARG;
    if (dy_hop < 0 || (used && y_hop < 0)) return GNNPRE_ERR_INVALID_ARG;
    if (ldh % 4 != 0 || reinterpret_cast<uintptr_t>(dY) % 4 || reinterpret_cast<uintptr_t>(Y) % 4 || reinterpret_cast<uintptr_t>(dWt) % 4 ||
        reinterpret_cast<uintptr_t>(workspace) % 256 || reinterpret_cast<uintptr_t>(batch) % 4)
        return GNNPRE_ERR_ALIGN;
    for (int32_t k = 0; k < num_hops; ++k) {
        if (!hops[k]) return GNNPRE_ERR_INVALID_ARG;
        if (reinterpret_cast<uintptr_t>(hops[k]) % 16) return GNNPRE_ERR_ALIGN;
    }
    const int64_t dw_span = (hidden - 1) * ldw + feat_dim;
    const auto meets = [&](const void* p, int64_t floats) { return arrays_overlap(dWt, 1, dw_span, 1, 4, p, 1, floats, 1, 4); };
    if (batch_size > 0) {
        const int64_t rows = (batch_size - 1);
        if (meets(dY, (num_hops - 1) * dy_hop + rows * lddy + hidden) || (used && meets(Y, (num_hops - 1) * y_hop + rows * ldy + hidden)) ||
            (batch && meets(batch, batch_size)))
            return GNNPRE_ERR_INVALID_ARG;
        const int64_t room = grad_shape(num_hops, batch_size, feat_dim, hidden, kMostSms).bytes;
        if (workspace_bytes < room || meets(workspace, room / 4)) return GNNPRE_ERR_INVALID_ARG;
        for (int32_t k = 0; k < num_hops; ++k)
            if (meets(hops[k], (n - 1) * ldh + feat_dim)) return GNNPRE_ERR_INVALID_ARG;
    }
    int sms = 0;
    const bool empty = batch_size == 0;
    GradShape g{};
    if (!empty) {
        GNNPRE_TRY(device_sms(&sms));
        g = grad_shape(num_hops, batch_size, feat_dim, hidden, std::min(sms, kMostSms));
    } else {
        GNNPRE_TRY(check_device());
        if (accumulate) return GNNPRE_OK;
    }
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (!empty) {
        static std::atomic<bool> opted_in[kMaxDevices];
        int dev = 0;
        GNNPRE_CUDA(cudaGetDevice(&dev));
        if (dev >= kMaxDevices || !opted_in[dev].load(std::memory_order_relaxed)) {
            GNNPRE_CUDA(cudaFuncSetAttribute(k_lc_grad, cudaFuncAttributeMaxDynamicSharedMemorySize, kGradSmem));
            if (dev < kMaxDevices) opted_in[dev].store(true, std::memory_order_relaxed);
        }
        GradArgs a{};
        for (int32_t k = 0; k < num_hops; ++k) a.hop[k] = hops[k];
        a.ldh = ldh;
        a.n = n;
        a.feat_dim = (int32_t)feat_dim;
        a.hidden = (int32_t)hidden;
        a.num_hops = num_hops;
        a.batch = batch;
        a.batch_size = batch_size;
        a.dy = dY;
        a.lddy = lddy;
        a.dy_hop = dy_hop;
        a.y = Y;
        a.ldy = ldy;
        a.y_hop = y_hop;
        a.relu_mask = used;
        a.tiles_f = g.tiles_f;
        a.width = g.width;
        a.tiles = g.tiles;
        a.splits = g.splits;
        a.chunks_per_hop = g.chunks_per_hop;
        a.chunks = g.chunks;
        a.parts = static_cast<float*>(workspace);
        a.part_ld = g.part_ld;
        a.error = error_flag;
        a.spin_limit = polls;
        a.drop = drop;
        a.wide = ((reinterpret_cast<uintptr_t>(dY) | (uintptr_t)(lddy * 4) | (uintptr_t)(dy_hop * 4)) % 16 == 0) &&
                 (!used || (reinterpret_cast<uintptr_t>(Y) | (uintptr_t)(ldy * 4) | (uintptr_t)(y_hop * 4)) % 16 == 0);
        k_lc_grad<<<(unsigned)((int64_t)g.tiles * g.splits), kGradThreads, kGradSmem, st>>>(a);
        GNNPRE_CUDA(cudaGetLastError());
    }
    return launch_after(k_lc_grad_join, dim3((unsigned)((feat_dim + 127) / 128), (unsigned)hidden), 32 * kJoinGroups, 0, !empty, st,
                        (const float*)workspace, g.part_ld, g.splits, (int32_t)hidden, (int32_t)feat_dim, (int32_t)(accumulate != 0), dWt, ldw);
}

}  // namespace
}  // namespace gnnpre

using namespace gnnpre;

extern "C" int64_t gnnpre_lc_first_layer_grad_workspace(int32_t num_hops, int64_t batch_size, int64_t feat_dim, int64_t hidden) {
    if (check_grad(num_hops, batch_size, feat_dim, hidden) != GNNPRE_OK) return GNNPRE_ERR_INVALID_ARG;
    return batch_size == 0 ? 0 : grad_shape(num_hops, batch_size, feat_dim, hidden, kMostSms).bytes;
}

extern "C" int gnnpre_lc_first_layer_grad(const float* const* hops, int32_t num_hops, int64_t n, int64_t feat_dim, int64_t ldh,
                                          const int32_t* batch, int64_t batch_size, const float* dY, int64_t lddy, int64_t dy_hop_stride,
                                          const float* Y, int64_t ldy, int64_t y_hop_stride, uint64_t relu_mask, int64_t hidden,
                                          int32_t accumulate, float* dWt, int64_t ldw, void* workspace, int64_t workspace_bytes,
                                          int32_t* error_flag, void* stream) {
    return grad_launch(hops, num_hops, n, feat_dim, ldh, batch, batch_size, dY, lddy, dy_hop_stride, Y, ldy, y_hop_stride, relu_mask, hidden,
                       accumulate, dWt, ldw, workspace, workspace_bytes, error_flag, stream);
}

// Failure-detection self-test: see include/gnnpre.h.
extern "C" int gnnpre_lc_grad_selftest_wait_timeout(const float* hop, int64_t n, int64_t feat_dim, int64_t ldh, const float* dY, int64_t lddy,
                                                    int64_t hidden, float* dWt, int64_t ldw, void* workspace, int64_t workspace_bytes,
                                                    int32_t* error_flag, uint32_t polls, void* stream) {
    if (!error_flag || polls == 0 || polls > 100000u) return GNNPRE_ERR_INVALID_ARG;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const float* hops[1] = {hop};
    GNNPRE_CUDA(cudaMemsetAsync(error_flag, 0, sizeof(int32_t), st));
    GNNPRE_TRY(grad_launch(hops, 1, n, feat_dim, ldh, nullptr, n, dY, lddy, 0, nullptr, 0, 0, 0, hidden, 0, dWt, ldw, workspace, workspace_bytes,
                           error_flag, stream, true, polls));
    GNNPRE_CUDA(cudaStreamSynchronize(st));
    int32_t flag = 0;
    GNNPRE_CUDA(cudaMemcpy(&flag, error_flag, sizeof(flag), cudaMemcpyDeviceToHost));
    return flag ? GNNPRE_ERR_TIMEOUT : GNNPRE_OK;
}
