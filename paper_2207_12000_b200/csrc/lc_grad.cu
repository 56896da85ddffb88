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
//   warps 8-15   operand A = dZ^T: a lane has one column h and reads it in the 16 rows of a chunk, masks, splits, and stores it to
//                tensor memory, where a lane is a row of A.
//   warps 16-23  operand B = the gathered rows of X: split and laid down in shared memory as they lie, rows along K.
//                Splitting a chunk is a chain of waits, reads, splits and stores, so either kind has two groups of four warps that
//                take the chunks in turn.
//   warps 24-26  have the copy engine bring chunks into shared memory, as many ahead as there is room for: 24 and 25, in turn, gathered
//                rows of X (four per instruction), 26 tiles of dY and Y.  One warp issues a chunk's copies in some 1,200 cycles, of
//                which the copies' own instructions are the least; read by the splitting warps themselves the rows took 9.2 us a
//                chunk of 32, 16-byte copies by four warps (cp.async) 1.7 us.  Rows of dY or Y that do not start on 16-byte
//                boundaries take 4-byte copies by warps 24 and 25.
//   warp 27      issues the products.
//
// Numbers.  An fp32 operand is the sum of three bf16 numbers h + m + l, each what is left rounded to nearest, so nothing is lost and
// any scale fits; of the nine products the six largest are taken.  |m| <= 2^-8 and |l| <= 2^-17 of the operand, so those left out come to
// 2^-24 of |dZ||X| per term at most, of either sign.  (Parts cut from the 24 bits, at the same number of instructions, leave out up to
// 2^-21, and all of it has the product's sign.  Two fp16 numbers and three products would need a scale known before the data is read.)
//
// Tensor memory: two accumulators of 128 columns in turn, then 24 columns (three parts of 8: two elements of K per column) for each of
// six chunks of A.  What A takes there it neither writes to nor is read from shared memory, whose bandwidth B alone then needs.
//
// Measured: 2.4 M rows x 3 hops, F = 100, hidden 256: 4.35 ms in long runs (3.6 TB/s, 55 % of the copy rate; 3.7 ms on a cool device),
// 7.35 M rows' products at 86 TFLOP/s, six times that on the tensor cores.  A chunk takes some 1,000 cycles, its products 384.
// At 72 registers a thread before they are handed on, 64 bytes spill.
#include <algorithm>
#include <atomic>

#include "dense.cuh"
#include "tensor_core.cuh"

namespace gnnpre {
namespace {

constexpr int kGradTile = 128;        // rows (h) of a tile, columns (f) at most
constexpr int kGradChunk = 16;        // batch rows per stage
constexpr int kGradMaxHops = 8;       // hops per launch
constexpr int kGradRaw = 6;           // chunks being copied or split
constexpr int kGradStages = 6;        // chunks split
constexpr int kGradSlice = 4;         // chunks whose products share an accumulator
// Of two groups that take chunks in turn each must have its own places of a ring: one that meets a place's barrier only every other
// phase cannot tell by its parity whether the phase before the awaited one is over.
static_assert(kGradRaw % 2 == 0 && kGradStages % 2 == 0, "a place belongs to one group");
constexpr int kGradSumWarps = 8, kGradBWarp = 16, kGradCopyWarp = 24, kGradTileWarp = 26, kGradMmaWarp = 27, kGradWarps = 28;
constexpr int kGradThreads = 32 * kGradWarps;            // (whole warpgroups, for the registers they hand on)
constexpr uint32_t kGradAllRows = (1u << kGradChunk) - 1;
constexpr uint32_t kGradMatrix = kGradChunk * kGradTile * 4;  // a chunk of dY, Y or X as copied: rows of 512 bytes
constexpr uint32_t kGradRawStage = 3 * kGradMatrix;
constexpr uint32_t kGradPart = 2 * kGradChunk * 128;     // one part of B's chunk: two blocks of 64 columns, rows of 128 bytes
constexpr uint32_t kGradStage = 3 * kGradPart;
constexpr uint32_t kGradTmem = 512, kGradTmemA = 256, kGradTmemStage = 24;
constexpr int kGradSmem = kGradStages * (int)kGradStage + kGradRaw * (int)kGradRawStage + 1024;
// Registers per thread: 896 threads start with 72, 64,512 in all = 256 x (104 + 72 + 48) + 128 x 56.
constexpr int kRegsSum = 104, kRegsB = 48, kRegsRest = 56;

struct GradMaps {
    CUtensorMap x[kGradMaxHops];  // [n, F] hop matrices, box [1, 128]
    CUtensorMap dy, y;            // [hops, batch_size, hidden], box [1, 16, 128]
};

struct GradArgs {
    int64_t n;
    int32_t feat_dim, hidden;
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
    int32_t chunks_per_hop;
    int64_t chunks;
    float* parts;               // [splits][hidden][part_ld]
    int64_t part_ld;
    int32_t* error;
    uint32_t spin_limit;
    int32_t wide;               // rows of dY and Y start on 16-byte boundaries
    int32_t drop;               // self-test: chunks that are complete are not announced
};

// Two numbers in three bf16 parts each, the first one's in the lower halves.  Every part is rounded to nearest, and the third one holds
// what is left exactly.
struct Parts {
    uint32_t h, m, l;
};
__device__ __forceinline__ uint32_t round2(float v, float w) {
    uint32_t p;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(p) : "f"(w), "f"(v));
    return p;
}
__device__ __forceinline__ Parts split2(float v, float w) {
    Parts p;
    // (saturated: the largest fp32 numbers would round to infinity; of an infinity the second part is one and the third NaN)
    asm("cvt.rn.satfinite.bf16x2.f32 %0, %1, %2;" : "=r"(p.h) : "f"(w), "f"(v));
    v -= __uint_as_float(p.h << 16);
    w -= __uint_as_float(p.h & 0xffff0000u);
    p.m = round2(v, w);
    p.l = round2(v - __uint_as_float(p.m << 16), w - __uint_as_float(p.m & 0xffff0000u));
    return p;
}

template <int REGS>
__device__ __forceinline__ void more_registers() {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(REGS));
}
template <int REGS>
__device__ __forceinline__ void fewer_registers() {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(REGS));
}

// Four bytes global -> shared without passing through registers, or as many zeros.
__device__ __forceinline__ void grad_copy(uint32_t dst, const float* src, bool live) {
    const int size = live ? 4 : 0;
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(size) : "memory");
}

// Four rows of X, and a chunk of dY or Y; what lies outside the matrices comes as zeros.
__device__ __forceinline__ void grad_gather4(uint32_t dst, const CUtensorMap* map, int x0, int r0, int r1, int r2, int r3, uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cluster.global.tile::gather4.mbarrier::complete_tx::bytes"
        " [%0], [%1, {%3, %4, %5, %6, %7}], [%2];" ::"r"(dst),
        "l"(reinterpret_cast<uint64_t>(map)), "r"(bar), "r"(x0), "r"(r0), "r"(r1), "r"(r2), "r"(r3)
        : "memory");
}
__device__ __forceinline__ void grad_tile(uint32_t dst, const CUtensorMap* map, int x0, int y0, int z0, uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
        " [%0], [%1, {%3, %4, %5}], [%2];" ::"r"(dst),
        "l"(reinterpret_cast<uint64_t>(map)), "r"(bar), "r"(x0), "r"(y0), "r"(z0)
        : "memory");
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

__global__ void __launch_bounds__(kGradThreads, 1) k_lc_grad(const __grid_constant__ GradMaps maps, const __grid_constant__ GradArgs a) {
    extern __shared__ unsigned char grad_smem[];
    __shared__ __align__(8) unsigned long long bars[2 * kGradStages + 2 * kGradRaw + 5];
    __shared__ uint32_t tmem_slot;
    __shared__ int abort_word;
    __shared__ uint32_t rows_of[kGradRaw];  // of a chunk as copied: the rows that exist
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
            tc_bar_init(raw_full(s), a.wide ? 2 : 1 + 32);  // X and the tiles, or X and every thread that copies
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
    // the share's first chunk; the others follow one by one
    int hop = (int)(first / a.chunks_per_hop);
    int in_hop = (int)(first - (int64_t)hop * a.chunks_per_hop);
    auto advance = [&](int& k, int& c) {
        if (++c == a.chunks_per_hop) {
            c = 0;
            ++k;
        }
    };

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
        const int q = warp & 3, group = (warp - kGradSumWarps) >> 2;
        const uint32_t column = 4u * (32 * q + lane);
        if (group) advance(hop, in_hop);
        for (int c = group; c < count; c += 2) {
            const int s = c % kGradStages, r0 = c % kGradRaw;
            const bool relu = (a.relu_mask >> hop) & 1u;
            advance(hop, in_hop);
            advance(hop, in_hop);
            if (!tc_wait_warp(raw_full(r0), (uint32_t)(c / kGradRaw) & 1u, abort_flag, a.error, a.spin_limit)) break;
            const uint32_t dy = raw0 + r0 * kGradRawStage + column, y = dy + kGradMatrix, rows = rows_of[r0];
            float v[kGradChunk];
#pragma unroll
            for (int r = 0; r < kGradChunk; ++r) v[r] = grad_read(dy + 4u * kGradTile * r);
            if (relu) {
                float m[kGradChunk];
#pragma unroll
                for (int r = 0; r < kGradChunk; ++r) m[r] = grad_read(y + 4u * kGradTile * r);
#pragma unroll
                for (int r = 0; r < kGradChunk; ++r) v[r] = m[r] > 0.f ? v[r] : 0.f;
            }
            __syncwarp();
            if (lane == 0) tc_bar_arrive(raw_empty(r0));
            if (rows != kGradAllRows) {
#pragma unroll
                for (int r = 0; r < kGradChunk; ++r) v[r] = rows >> r & 1u ? v[r] : 0.f;
            }
            uint32_t p[3][kGradChunk / 2];
#pragma unroll
            for (int j = 0; j < kGradChunk / 2; ++j) {
                const Parts two = split2(v[2 * j], v[2 * j + 1]);
                p[0][j] = two.h;
                p[1][j] = two.m;
                p[2][j] = two.l;
            }
            if (!tc_wait_warp(empty(s), ((uint32_t)(c / kGradStages) & 1u) ^ 1u, abort_flag, a.error, a.spin_limit)) break;
            tc_fence_after();
            const uint32_t to = tmem + ((uint32_t)(32 * q) << 16) + kGradTmemA + kGradTmemStage * s;
#pragma unroll
            for (int i = 0; i < 3; ++i) tc_store8(to + kGradChunk / 2 * i, p[i]);
            tc_store_wait();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) tc_bar_arrive(full(s));
        }
    } else if (warp < kGradCopyWarp) {
        fewer_registers<kRegsB>();
        constexpr int kRows = kGradChunk / 4;
        const int col = 4 * lane, first_row = (warp & 3) * kRows, group = (warp - kGradBWarp) >> 2;  // of the tile, of the chunk
        for (int c = group; c < count; c += 2) {
            const int s = c % kGradStages, r0 = c % kGradRaw;
            if (!tc_wait_warp(raw_full(r0), (uint32_t)(c / kGradRaw) & 1u, abort_flag, a.error, a.spin_limit)) break;
            const uint32_t from = raw0 + r0 * kGradRawStage + 2 * kGradMatrix + 16u * lane + 4u * kGradTile * first_row;
            const uint32_t rows = rows_of[r0];
            float4 v[kRows];
#pragma unroll
            for (int i = 0; i < kRows; ++i) v[i] = grad_read4(from + 4u * kGradTile * i);
            __syncwarp();
            if (lane == 0) tc_bar_arrive(raw_empty(r0));
            if (rows != kGradAllRows) {
#pragma unroll
                for (int i = 0; i < kRows; ++i)
                    if (!(rows >> (first_row + i) & 1u)) v[i] = make_float4(0.f, 0.f, 0.f, 0.f);
            }
            if (!tc_wait_warp(empty(s), ((uint32_t)(c / kGradStages) & 1u) ^ 1u, abort_flag, a.error, a.spin_limit)) break;
            const uint32_t to = base + (uint32_t)s * kGradStage + (col / 64) * (kGradChunk * 128) + (col % 8) * 2;
#pragma unroll
            for (int i = 0; i < kRows; ++i) {
                const int k = first_row + i;
                const Parts x = split2(v[i].x, v[i].y), z = split2(v[i].z, v[i].w);
                const uint32_t at = to + 128u * k + ((uint32_t)((col % 64 / 8) ^ (k & 7)) << 4);
                asm volatile("st.shared.v2.b32 [%0], {%1, %2};" ::"r"(at), "r"(x.h), "r"(z.h) : "memory");
                asm volatile("st.shared.v2.b32 [%0], {%1, %2};" ::"r"(at + kGradPart), "r"(x.m), "r"(z.m) : "memory");
                asm volatile("st.shared.v2.b32 [%0], {%1, %2};" ::"r"(at + 2 * kGradPart), "r"(x.l), "r"(z.l) : "memory");
            }
            tc_fence_async();
            __syncwarp();
            if (lane == 0) tc_bar_arrive(full(s));
        }
    } else {
        fewer_registers<kRegsRest>();
    }
    // nothing may land after this CTA has left: the last copies of the ring's places t, t + step, ...
    auto landed = [&](int issued, int t, int step) {
        for (; t < min(issued, kGradRaw); t += step)
            for (uint32_t i = 0; i < kTcSpinLimit; ++i)
                if (tc_bar_test(raw_full(t), (uint32_t)((issued - t + kGradRaw - 1) / kGradRaw - 1) & 1u)) break;
    };
    if (warp == kGradCopyWarp || warp == kGradCopyWarp + 1) {
        const int w = warp - kGradCopyWarp, n = (int)a.n, rows_in = (int)a.batch_size;
        // This lane's row of the hop matrix in a chunk, -1 or another row outside for none.  Asked for kAhead of the warp's chunks
        // ahead: with one, copies were issued no faster than one load from memory after the other.
        constexpr int kAhead = 4;
        auto ask = [&](int c) {
            const int64_t pos = (int64_t)c * kGradChunk + lane;
            if (lane >= kGradChunk || pos >= rows_in) return -1;
            return a.batch ? __ldg(a.batch + pos) : (int)pos;
        };
        if (w == 1) advance(hop, in_hop);
        int asked[kAhead], ask_hop = hop, ask_in = in_hop;
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            asked[j] = w + 2 * j < count ? ask(ask_in) : -1;
            advance(ask_hop, ask_in);
            advance(ask_hop, ask_in);
        }
        const int first4 = 4 * (lane & (kGradChunk / 4 - 1));
        int place = w, issued = 0;  // issued: chunks up to this warp's last
        uint32_t ph = 1;
        bool ok = true;
        for (int c0 = w; c0 < count && ok; c0 += 2 * kAhead)
#pragma unroll
            for (int j = 0; j < kAhead; ++j) {
                const int c = c0 + 2 * j, row = asked[j];
                if (c >= count || !ok) continue;
                if (c + 2 * kAhead < count) asked[j] = ask(ask_in);
                advance(ask_hop, ask_in);
                advance(ask_hop, ask_in);
                // (rows that do not exist are fetched from row 0 and left out when the chunk is split)
                const bool exists = row >= 0 && row < n;
                const uint32_t rows = __ballot_sync(0xffffffffu, exists);
                const int from = exists ? row : 0;
                const int q0 = __shfl_sync(0xffffffffu, from, first4), q1 = __shfl_sync(0xffffffffu, from, first4 + 1),
                          q2 = __shfl_sync(0xffffffffu, from, first4 + 2), q3 = __shfl_sync(0xffffffffu, from, first4 + 3);
                ok = tc_wait_warp(raw_empty(place), ph, abort_flag, a.error, a.spin_limit);
                if (!ok) continue;
                const uint32_t to = raw0 + place * kGradRawStage, bar = raw_full(place);
                if (lane == 0) {
                    rows_of[place] = rows;
                    tc_bar_expect(bar, kGradMatrix);
                }
                __syncwarp();
                if (lane < kGradChunk / 4) grad_gather4(to + 2 * kGradMatrix + 4u * kGradTile * first4, &maps.x[hop], f0, q0, q1, q2, q3, bar);
                if (!a.wide) {
                    const int row0 = in_hop * kGradChunk;
                    auto copy_rows = [&](uint32_t dst, const float* src, int64_t ld) {
                        for (int i = 0; i < kGradChunk; ++i)
#pragma unroll
                            for (int k = 0; k < 4; ++k) {
                                const bool live = row0 + i < rows_in && h0 + 32 * k + lane < a.hidden;
                                grad_copy(dst + 4u * kGradTile * i + 128u * k + 4u * lane, live ? src + (int64_t)(row0 + i) * ld + h0 + 32 * k + lane : a.dy, live);
                            }
                    };
                    copy_rows(to, a.dy + hop * a.dy_hop, a.lddy);
                    if (a.relu_mask >> hop & 1u) copy_rows(to + kGradMatrix, a.y + hop * a.y_hop, a.ldy);
                    asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(bar) : "memory");
                }
                advance(hop, in_hop);
                advance(hop, in_hop);
                issued = c + 1;
                place += 2;
                if (place >= kGradRaw) {
                    place -= kGradRaw;
                    ph ^= 1u;
                }
            }
        asm volatile("cp.async.wait_all;" ::: "memory");
        landed(issued, w, 2);
    } else if (warp == kGradTileWarp) {
        if (lane == 0 && a.wide) {
            int place = 0, issued = 0;
            uint32_t ph = 1;
            for (; issued < count; ++issued) {
                if (!tc_wait(raw_empty(place), ph, abort_flag, a.error, a.spin_limit)) break;
                const bool relu = a.relu_mask >> hop & 1u;
                const uint32_t to = raw0 + place * kGradRawStage, bar = raw_full(place);
                tc_bar_expect(bar, kGradMatrix * (1 + relu));
                grad_tile(to, &maps.dy, h0, in_hop * kGradChunk, hop, bar);
                if (relu) grad_tile(to + kGradMatrix, &maps.y, h0, in_hop * kGradChunk, hop, bar);
                advance(hop, in_hop);
                if (++place == kGradRaw) {
                    place = 0;
                    ph ^= 1u;
                }
            }
            landed(issued, 0, 1);
        }
        __syncwarp();
    } else if (warp == kGradMmaWarp) {
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
                        tc_mma_ta(d, am + kGradChunk / 2 * kA[t] + 8 * j, b[kB[t]] + (2048 >> 4) * j, instr, c != start || t != 0 || j != 0);
                tc_commit(empty(s));
            }
            if (ok) tc_commit(acc_full(i & 1));
        }
        tc_commit(drained);
        for (uint32_t i = 0; i < kTcSpinLimit; ++i)
            if (tc_bar_test(drained, 0)) break;
        __syncwarp();
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

int encode_map(const float* base, int rank, const cuuint64_t* dims, const cuuint64_t* strides, const cuuint32_t* box, CUtensorMap* out) {
    typedef CUresult (*encode_fn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                  const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion,
                                  CUtensorMapFloatOOBfill);
    static std::atomic<encode_fn> cached{nullptr};  // threads may race to fill it; they all store the same pointer
    encode_fn encode = cached.load(std::memory_order_acquire);
    if (!encode) {
        void* fn = nullptr;
        cudaDriverEntryPointQueryResult q;
        GNNPRE_CUDA(cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &q));
        if (q != cudaDriverEntryPointSuccess || !fn) return GNNPRE_ERR_CUDA;
        encode = reinterpret_cast<encode_fn>(fn);
        cached.store(encode, std::memory_order_release);
    }
    const cuuint32_t elem[3] = {1u, 1u, 1u};
    const CUresult r = encode(out, CU_TENSOR_MAP_DATA_TYPE_FLOAT32, (cuuint32_t)rank, const_cast<float*>(base), dims, strides, box, elem,
                              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) {
        set_last_cuda_error(cudaErrorInvalidValue, "cuTensorMapEncodeTiled", __FILE__, __LINE__);
        return GNNPRE_ERR_CUDA;
    }
    return GNNPRE_OK;
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
    if (batch_size > 0) {
        const int64_t rows = batch_size - 1, room = grad_shape(num_hops, batch_size, feat_dim, hidden, kMostSms).bytes;
        if (workspace_bytes < room) return GNNPRE_ERR_INVALID_ARG;
        // what is written, the sums and the shares' sums before them, lies apart from what is read and from one another
        const auto meets = [&](const void* p, int64_t floats) {
            return arrays_overlap(dWt, 1, dw_span, 1, 4, p, 1, floats, 1, 4) || arrays_overlap(workspace, 1, room, 1, 1, p, 1, floats, 1, 4);
        };
        if (meets(dY, (num_hops - 1) * dy_hop + rows * lddy + hidden) || (used && meets(Y, (num_hops - 1) * y_hop + rows * ldy + hidden)) ||
            (batch && meets(batch, batch_size)) || arrays_overlap(dWt, 1, dw_span, 1, 4, workspace, 1, room, 1, 1))
            return GNNPRE_ERR_INVALID_ARG;
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
    const auto join = [&](int32_t splits, bool add, bool after) {
        return launch_after(k_lc_grad_join, dim3((unsigned)((feat_dim + 127) / 128), (unsigned)hidden), 32 * kJoinGroups, 0, after, st,
                            (const float*)workspace, g.part_ld, splits, (int32_t)hidden, (int32_t)feat_dim, (int32_t)add, dWt, ldw);
    };
    if (!empty) {
        static std::atomic<bool> opted_in[kMaxDevices];
        int dev = 0;
        GNNPRE_CUDA(cudaGetDevice(&dev));
        if (dev >= kMaxDevices || !opted_in[dev].load(std::memory_order_relaxed)) {
            GNNPRE_CUDA(cudaFuncSetAttribute(k_lc_grad, cudaFuncAttributeMaxDynamicSharedMemorySize, kGradSmem));
            if (dev < kMaxDevices) opted_in[dev].store(true, std::memory_order_relaxed);
        }
        GradArgs a{};
        a.n = n;
        a.feat_dim = (int32_t)feat_dim;
        a.hidden = (int32_t)hidden;
        a.batch = batch;
        a.batch_size = batch_size;
        a.lddy = lddy;
        a.dy_hop = dy_hop;
        a.ldy = ldy;
        a.y_hop = y_hop;
        a.tiles_f = g.tiles_f;
        a.width = g.width;
        a.tiles = g.tiles;
        a.chunks_per_hop = (int32_t)g.chunks_per_hop;
        a.parts = static_cast<float*>(workspace);
        a.part_ld = g.part_ld;
        a.error = error_flag;
        a.spin_limit = polls;
        a.drop = drop;
        for (int32_t k0 = 0; k0 < num_hops; k0 += kGradMaxHops) {  // further hops are added to the first ones' sum
            const int32_t kn = std::min(kGradMaxHops, num_hops - k0);
            const GradShape now = grad_shape(kn, batch_size, feat_dim, hidden, std::min(sms, kMostSms));
            a.relu_mask = used >> k0 & ((1ull << kn) - 1);
            a.dy = dY + k0 * dy_hop;
            a.y = a.relu_mask ? Y + k0 * y_hop : nullptr;
            a.splits = now.splits;
            a.chunks = now.chunks;
            const auto tiled = [&](const float* p, int64_t ld, int64_t hop) {
                return (reinterpret_cast<uintptr_t>(p) | (uintptr_t)(ld * 4)) % 16 == 0 && ld < ((int64_t)1 << 36) &&
                       (kn == 1 || (hop > 0 && hop % 4 == 0 && hop < ((int64_t)1 << 36)));
            };
            a.wide = tiled(a.dy, lddy, dy_hop) && (!a.relu_mask || tiled(a.y, ldy, y_hop));
            GradMaps maps{};
            for (int32_t k = 0; k < kn; ++k) {
                const cuuint64_t dims[2] = {(cuuint64_t)feat_dim, (cuuint64_t)n}, strides[1] = {(cuuint64_t)ldh * 4};
                const cuuint32_t box[2] = {kGradTile, 1u};
                GNNPRE_TRY(encode_map(hops[k0 + k], 2, dims, strides, box, &maps.x[k]));
            }
            if (a.wide) {
                const cuuint64_t dims[3] = {(cuuint64_t)hidden, (cuuint64_t)batch_size, (cuuint64_t)kn};
                const cuuint32_t box[3] = {kGradTile, kGradChunk, 1u};
                const cuuint64_t dy_strides[2] = {(cuuint64_t)lddy * 4, kn > 1 ? (cuuint64_t)dy_hop * 4 : (cuuint64_t)16};
                GNNPRE_TRY(encode_map(a.dy, 3, dims, dy_strides, box, &maps.dy));
                const cuuint64_t y_strides[2] = {(cuuint64_t)ldy * 4, kn > 1 ? (cuuint64_t)y_hop * 4 : (cuuint64_t)16};
                if (a.relu_mask) GNNPRE_TRY(encode_map(a.y, 3, dims, y_strides, box, &maps.y));
            }
            k_lc_grad<<<(unsigned)((int64_t)g.tiles * now.splits), kGradThreads, kGradSmem, st>>>(maps, a);
            GNNPRE_CUDA(cudaGetLastError());
            GNNPRE_TRY(join(now.splits, accumulate || k0 > 0, true));
        }
        return GNNPRE_OK;
    }
    return join(0, false, false);
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
