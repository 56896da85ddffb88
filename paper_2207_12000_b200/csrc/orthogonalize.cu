// An update orthogonalised by Newton-Schulz products:
//
//   X_0 = G / (||G||_F + eps),   A = X X^T,   X <- (a I + b A + c A^2) X   `steps` times,   out = scale X
//
// on the smaller side of G (X is [r, n] with r <= n, G or its transpose).  Everything is matrix products, on the tensor cores.
//
// Numbers.  ||X_0||_F <= 1, so every singular value starts in [0, 1] and the polynomial's coefficients bound all that follows
// (computed on the host; coefficients under which the iterates may grow without such a bound are refused).  A matrix with a known
// bound is held as 2^e times itself in two fp16 numbers, high and low part, e chosen so that the bound just fits: 22 significant
// bits of entries down to some 2^-16 of the bound, and of smaller ones an absolute error of 2^-39 of it, far below that of fp32 sums of
// that size.  (An update whose norm is far below eps starts far below one: the device finds bounds for it from its norm.)  A product
// takes three tensor-core products (high x high, high x low, low x high) into one fp32 accumulator; what is dropped is below 2^-22 of
// the operands.  fp16 carries 11 bits where tf32 carries as many at half the rate and bf16 carries 8: one fp16 product in place of
// the three would lose the small singular values, which a step multiplies by a (3.4) and with them the rounding errors of the large
// ones.  (Plain fp32 has 24 bits: it is off by 1.7e-6 on [256, 128] where this is by 1.9e-6, and by 4.6e-6 on [2048, 4096], whose long
// sums it rounds more often, where this is by 1.6e-6.)
//
// Order of the products.  The polynomials of a few steps commute and are polynomials of the first A, so they can be multiplied
// together before X: with P = aI + bA + cA^2, X <- P X makes A <- P A P.  A segment of g steps is
//     A = X X^T;   g times { P = aI + bA + cA^2;  T = A P;  A = T P;  Q = Q P };   X = Q X
// (the last step needs no T and A, the first no Q).  The r x r products are symmetric: only the lower tiles are computed.  That
// saves work on matrices that are not square, at the price of an error of A that grows by a^2 per step where an A formed anew has
// none of it: [256, 128] with six strong directions is off by 1.8e-6 in steps by themselves (as plain fp32 is) and by 2.0e-4 in
// segments of three.  So segments have three steps at most for bf16 outputs (one rounding: 1.7e-3), two for fp16, one for fp32.
//
// Measured, us, five steps: 256 x 128 59 (one CTA, from shared memory; 56-58 in a graph), three of 256 x 602 144 (a cluster of 16
// CTAs each), 2,048 x 4,096 1,220 (a launch per product; 164-183 TFLOP/s of the least work, three times that on the tensor cores).
//
// Layout.  Operands are stored as the tensor core reads them: blocks of 128 rows x 64 columns of K in the 128-byte swizzle, the
// high parts' 16 KB and then the low parts', so an operand tile is one contiguous copy and needs no tensor map.
#include <algorithm>
#include <atomic>
#include <cmath>

#include "dense.cuh"
#include "tensor_core.cuh"

namespace gnnpre {
namespace {

constexpr int kBlockRows = 128, kBlockCols = 64;
constexpr int kHalfBytes = kBlockRows * kBlockCols * 2;  // one part of a block
constexpr int kBlockBytes = 2 * kHalfBytes;
constexpr int kPipeBytes = 192 * 1024;
constexpr int kSumWarps = 8, kCopyWarp = 8, kMmaWarp = 9;
constexpr int kProductThreads = 320;
constexpr int kAccs = 4;                                 // accumulators that take turns
constexpr int kSliceChunks = 1;                          // chunks of 64 of K in one accumulator
constexpr int kMaxSteps = 64;
constexpr float kMostSpectral = 16.f;    // bound of X under which coefficients are accepted
constexpr int64_t kMaxSide = 1 << 16;

// A split matrix [rows, cols], both padded: block (rb, kb) of a batch entry.
struct Split {
    unsigned char* p;
    int64_t batch_bytes;
    int32_t kblocks;
    __device__ __forceinline__ unsigned char* block(int64_t batch, int rb, int kb) const {
        return p + batch * batch_bytes + ((int64_t)rb * kblocks + kb) * kBlockBytes;
    }
};

// Byte of element (row, col) of a block's part.
__device__ __forceinline__ uint32_t block_byte(int row, int col) {
    return (uint32_t)(row * 128 + ((((col >> 3) ^ (row & 7)) & 7) << 4) + (col & 7) * 2);
}

// v in two fp16 numbers, eight of them at a time.  The high part is rounded to nearest: cut from v's upper bits (two conversions less,
// no faster here) it leaves a low part of v's sign, whose squares, which are not computed, then add up in A's diagonal: 3.1e-6 off
// on [256, 128] for 1.9e-6.
__device__ __forceinline__ void split8(const float (&v)[8], uint4& hi, uint4& lo) {
    uint32_t h[4], l[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __half2 hh = __floats2half2_rn(v[2 * i], v[2 * i + 1]);
        const float2 back = __half22float2(hh);
        const __half2 ll = __floats2half2_rn(v[2 * i] - back.x, v[2 * i + 1] - back.y);
        h[i] = *reinterpret_cast<const uint32_t*>(&hh);
        l[i] = *reinterpret_cast<const uint32_t*>(&ll);
    }
    hi = make_uint4(h[0], h[1], h[2], h[3]);
    lo = make_uint4(l[0], l[1], l[2], l[3]);
}

// ------------------------------------------------------------------------------------------------ exponents

struct Coeffs {
    float a, b, c;
};

constexpr double kLeastSpectral = 0x1p-90;  // what lies below is held as if it were as large (its squares leave fp32 at 2^-63)
constexpr double kOwnBounds = 0.25;         // norms of X_0 from here on cost at most two of the 22 bits: the coefficients' bounds do

// 2^e with which a matrix of this bound fits fp16 with room to spare.
__host__ __device__ inline int exponent_for(double bound) { return 14 - ilogb(fmax(bound, 1e-200)); }

// Of c A + b I, A's second form, where X has this bound.
__host__ __device__ inline int second_exponent(const Coeffs& c, double x) { return exponent_for(fabs((double)c.c) * x * x + fabs((double)c.b)); }

// Bounds of |P| and of the next X where X's bound x is its own and lies below the one that the coefficients give, which says `all_p` and
// `all_next`.
__device__ inline void own_bounds(const Coeffs& c, double x, double all_p, double all_next, double* p, double* next) {
    const double t = x * x;
    *p = fmin(all_p, fabs((double)c.a) + (fabs((double)c.b) + fabs((double)c.c) * t) * t);
    *next = fmax(fmin(all_next, x * *p * (1.0 + 1e-4)), kLeastSpectral);
}

// Bound of an X_0 of this norm.
__device__ inline double first_bound(double norm_of_x) { return fmax(norm_of_x * (1.0 + 1e-4), kLeastSpectral); }

// What the products of a step are multiplied by, between the exponents of what goes in and of what comes out.
struct StepFactors {
    float gram;           // A = X X^T
    float gram2, diag2;   // its second form (k_ns_chip: of c A A and b A in P)
    float p, p_diag;      // P
    float apply;          // X = P X
    float out;            // the caller's matrix = P X
};

// `ex`: X's exponent, and then the next X's.
__host__ __device__ inline StepFactors step_factors(const Coeffs& c, bool chip, float scale, double x, double p, double next, int* ex) {
    const int ea = exponent_for(x * x), ep = exponent_for(p), e2 = chip ? ep : second_exponent(c, x), en = exponent_for(next);
    StepFactors f;
    f.gram = (float)ldexp(1.0, ea - 2 * *ex);
    f.gram2 = (float)ldexp((double)c.c, chip ? ep - 2 * ea : e2 - 2 * *ex);
    f.diag2 = (float)ldexp((double)c.b, chip ? ep - ea : e2);
    f.p = (float)ldexp(1.0, ep - ea - e2);
    f.p_diag = (float)ldexp((double)c.a, ep);
    f.apply = (float)ldexp(1.0, en - ep - *ex);
    f.out = (float)ldexp((double)scale, -ep - *ex);
    *ex = en;
    return f;
}

// The coefficients' bounds: of X before a step, of |P| in it.
struct AllBounds {
    Coeffs c;
    double x[kMaxSteps + 1], p[kMaxSteps];
};

// ------------------------------------------------------------------------------------------------ norm and first split

struct Source {
    const void* g;
    int64_t ldg, batch_stride;
    int32_t rows, cols;      // of G
    int32_t dtype;
    int32_t tall;            // rows > cols: X is G's transpose
    double eps;
    double* partial;         // [batch][kNormBlocks]
    float factor;            // 2^e of X
    Split x, xt;
};

constexpr int kNormBlocks = 256;
constexpr int kNormThreads = 256;

// f with G as what it is.
template <typename F>
__device__ __forceinline__ void with_type(const Source& s, int64_t batch, F f) {
    const int64_t at = batch * s.batch_stride;
    if (s.dtype == GNNPRE_F32) f(static_cast<const float*>(s.g) + at);
    else if (s.dtype == GNNPRE_BF16) f(static_cast<const __nv_bfloat16*>(s.g) + at);
    else f(static_cast<const __half*>(s.g) + at);
}

// Squares in 64 bits: neither tiny nor huge updates lose their norm.
__global__ void __launch_bounds__(kNormThreads) k_ns_norm(const Source s) {
    __shared__ double room[kNormThreads / 32];
    double sum = 0;
    with_type(s, blockIdx.y, [&](const auto* g) {
        for (int64_t i = blockIdx.x; i < s.rows; i += gridDim.x) {
            // (what lies beyond a row's end is its last element again, so that the loads do not wait for a condition)
            constexpr int kAtOnce = 8;
            for (int j0 = threadIdx.x; j0 < s.cols; j0 += kAtOnce * kNormThreads) {
                float v[kAtOnce];
#pragma unroll
                for (int u = 0; u < kAtOnce; ++u) v[u] = to_f32(g[i * s.ldg + min(j0 + u * kNormThreads, s.cols - 1)]);
#pragma unroll
                for (int u = 0; u < kAtOnce; ++u)
                    if (j0 + u * kNormThreads < s.cols) sum += (double)v[u] * v[u];
            }
        }
    });
#pragma unroll
    for (int d = 16; d > 0; d /= 2) sum += __shfl_xor_sync(0xffffffffu, sum, d);
    if ((threadIdx.x & 31) == 0) room[threadIdx.x >> 5] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < kNormThreads / 32; ++w) sum += room[w];
        s.partial[blockIdx.y * kNormBlocks + blockIdx.x] = sum;
    }
}

// Of a launch per product: how much larger than the coefficients' exponents a matrix's own ones are, for each kind of operand and step.
enum { kOfX, kOfA, kOfA2, kOfP, kOfQ, kOfT, kKinds };
constexpr int kSlots = kKinds * (kMaxSteps + 1);
__host__ __device__ inline int slot(int kind, int step) { return kind * (kMaxSteps + 1) + step; }

struct Own {
    AllBounds all;
    int32_t steps, segment;  // (Q is the product of the P of a segment so far)
    int32_t* by;             // [batch][kSlots]
};

// One thread's work; small: X_0's norm lies below kOwnBounds.
__device__ inline void own_exponents(const Own& o, double norm_of_x, int32_t* by) {
    double x = first_bound(norm_of_x), all_q = 1, q = 1;
    for (int k = 0; k <= o.steps; ++k) {
        const double all_x = o.all.x[k];
        by[slot(kOfX, k)] = exponent_for(x) - exponent_for(all_x);
        if (k == o.steps) break;
        const double all_p = o.all.p[k];
        double p, next;
        own_bounds(o.all.c, x, all_p, o.all.x[k + 1], &p, &next);
        all_q = k % o.segment ? all_q * all_p : all_p;
        q = k % o.segment ? q * p : p;
        by[slot(kOfA, k)] = exponent_for(x * x) - exponent_for(all_x * all_x);
        by[slot(kOfA2, k)] = second_exponent(o.all.c, x) - second_exponent(o.all.c, all_x);
        by[slot(kOfP, k)] = exponent_for(p) - exponent_for(all_p);
        by[slot(kOfQ, k)] = exponent_for(q) - exponent_for(all_q);
        by[slot(kOfT, k)] = exponent_for(x * x * p) - exponent_for(all_x * all_x * all_p);
        x = next;
    }
}

// X and its transpose, split: a CTA takes [64, 64] of X.
__global__ void __launch_bounds__(256) k_ns_split(const Source s, const int32_t norm_blocks, const __grid_constant__ Own own) {
    __shared__ float tile[64][65];
    __shared__ double inverse;
    const int64_t batch = blockIdx.z;
    const int i0 = blockIdx.y * 64, j0 = blockIdx.x * 64;  // of X
    const int fast = threadIdx.x & 63, gi0 = (s.tall ? j0 : i0) + (threadIdx.x >> 6), gj = (s.tall ? i0 : j0) + fast;
    // neighbouring threads, neighbouring elements of G (nothing before this kernel writes them)
    float v[16];
    with_type(s, batch, [&](const auto* g) {
#pragma unroll
        for (int u = 0; u < 16; ++u) v[u] = to_f32(g[(int64_t)min(gi0 + 4 * u, s.rows - 1) * s.ldg + min(gj, s.cols - 1)]);
    });
    wait_previous_kernel();
    if (threadIdx.x < 32) {  // the blocks' sums in a fixed order
        double sum = 0;
        for (int b = threadIdx.x; b < norm_blocks; b += 32) sum += s.partial[batch * kNormBlocks + b];
#pragma unroll
        for (int d = 16; d > 0; d /= 2) sum += __shfl_xor_sync(0xffffffffu, sum, d);
        const double norm = sqrt(sum), over = 1.0 / (norm + s.eps), norm_of_x = norm * over;
        const bool small = norm_of_x < kOwnBounds;
        if (threadIdx.x == 0) inverse = over * (small ? ldexp(1.0, exponent_for(first_bound(norm_of_x))) : (double)s.factor);
        if (blockIdx.x == 0 && blockIdx.y == 0) {
            int32_t* by = own.by + batch * kSlots;
            if (!small) {
                for (int i = threadIdx.x; i < kSlots; i += 32) by[i] = 0;
            } else if (threadIdx.x == 0) {
                own_exponents(own, norm_of_x, by);
            }
        }
    }
    __syncthreads();
    const double scale = inverse;
#pragma unroll
    for (int u = 0; u < 16; ++u) {
        const int slow = (threadIdx.x >> 6) + 4 * u;
        const float o = gi0 + 4 * u < s.rows && gj < s.cols ? (float)((double)v[u] * scale) : 0.f;
        if (s.tall) tile[fast][slow] = o;
        else tile[slow][fast] = o;
    }
    __syncthreads();
    for (int c = threadIdx.x; c < 64 * 8; c += 256) {
        const int row = c >> 3, chunk = c & 7;
        float v[8];
        uint4 hi, lo;
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = tile[row][8 * chunk + e];
        split8(v, hi, lo);
        unsigned char* d = s.x.block(batch, (i0 + row) / kBlockRows, j0 / kBlockCols) + block_byte((i0 + row) % kBlockRows, 8 * chunk);
        *reinterpret_cast<uint4*>(d) = hi;
        *reinterpret_cast<uint4*>(d + kHalfBytes) = lo;
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = tile[8 * chunk + e][row];
        split8(v, hi, lo);
        d = s.xt.block(batch, (j0 + row) / kBlockRows, i0 / kBlockCols) + block_byte((j0 + row) % kBlockRows, 8 * chunk);
        *reinterpret_cast<uint4*>(d) = hi;
        *reinterpret_cast<uint4*>(d + kHalfBytes) = lo;
    }
}

// ------------------------------------------------------------------------------------------------ products

// D = alpha * (A B^T) + diag * I over the stored (scaled) numbers.  Where D is a new A, its second form c A + b I is written too:
// P = a I + A (c A + b I) then needs no A beside its accumulator (read from memory there it took 4.5 us of a product's 7.5).
struct Job {
    Split a, b, d, dt, d2;
    float alpha, diag, alpha2, diag2;
    int32_t k_chunks;
    int32_t write_t, write_2;  // write_t: D's transpose as well
    int32_t of_a, of_b, of_d, of_d2;  // whose exponents they have: slots of `by`
};

struct Product {
    Job job[2];
    int32_t jobs;
    const int32_t* by;   // a matrix's own exponents
    int32_t tiles_n;     // of BN columns
    int32_t symmetric;   // D = D^T: only tiles on and below the diagonal, the others by their transposes
    int32_t* error;
    uint32_t spin_limit;
    int32_t drop;        // self-test: the copies' bytes are not announced
    // the last product writes the caller's matrix instead
    void* out;           // nullptr: it does not
    int64_t ldo, out_batch;
    int32_t out_dtype, out_rows, out_cols;
    float out_factor;
};

// One tile of 128 x BN per CTA.  Warps 0-7 add up and store: warps w and w + 4 share the accumulator's lanes 32 (w & 3) .. and
// take a half of the columns each; warp 8 copies, warp 9 multiplies.
//
// The tensor core cuts, not rounds, a sum that it adds a product to: over K = 4000 in one accumulator the sums of squares in A
// came out 1e-5 too small (750 additions, half of 2^-23 each).  So an accumulator takes one chunk only, its small terms first, so
// that four cuts count; four take turns (two of 256 columns), and their sums are added up in registers, rounded to nearest, while the next ones form.
// What bounds a wide product is shared memory: per 64 of K a 128 x 128 tile writes 64 KB and the twelve products read 96 KB, 1,280 cycles at
// 128 bytes a cycle for 840 of the tensor core; 128 x 256 takes 1,920 for twice the work.
template <int BN>
__global__ void __launch_bounds__(kProductThreads, 1) k_ns_product(const __grid_constant__ Product a) {
    constexpr uint32_t kBBytes = BN * 128;                  // one part of B's chunk
    constexpr uint32_t kStage = kBlockBytes + 2 * kBBytes;
    constexpr int kStages = kPipeBytes / kStage;
    constexpr int kCols = BN / 2;                           // of a thread
    constexpr int kTurns = BN == 256 ? 2 : kAccs;           // accumulators that fit tensor memory
    extern __shared__ unsigned char ns_smem[];
    __shared__ __align__(8) unsigned long long bars[2 * kStages + 2 * kTurns + 1];
    __shared__ uint32_t tmem_slot;
    __shared__ int abort_word;
    __shared__ float alphas[2], diags[2], out_factor;  // of D's forms, with the matrices' own exponents
    volatile int* abort_flag = &abort_word;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t base = (tc_smem(ns_smem) + 1023u) & ~1023u;
    unsigned char* const base_p = ns_smem + (base - tc_smem(ns_smem));
    const uint32_t bar0 = tc_smem(&bars[0]);
    auto full = [&](int s) { return bar0 + 8u * s; };
    auto empty = [&](int s) { return bar0 + 8u * (kStages + s); };
    auto acc_full = [&](int b) { return bar0 + 8u * (2 * kStages + b); };
    auto acc_empty = [&](int b) { return bar0 + 8u * (2 * kStages + kTurns + b); };
    const uint32_t drained = bar0 + 8u * (2 * kStages + 2 * kTurns);
    const Job& job = a.job[blockIdx.z % a.jobs];
    const int64_t batch = blockIdx.z / a.jobs;
    int bi, bj;  // tile row (of 128), tile column (of BN)
    if (a.symmetric) {
        bi = (int)((sqrtf(8.f * blockIdx.x + 1.f) - 1.f) * 0.5f);
        while ((bi + 1) * (bi + 2) / 2 <= (int)blockIdx.x) ++bi;
        while (bi * (bi + 1) / 2 > (int)blockIdx.x) --bi;
        bj = blockIdx.x - bi * (bi + 1) / 2;
    } else {
        bi = blockIdx.x / a.tiles_n;
        bj = blockIdx.x % a.tiles_n;
    }
    if (threadIdx.x == 0) {
        for (int s = 0; s < kStages; ++s) {
            tc_bar_init(full(s), 1 + (a.drop ? 1 : 0));
            tc_bar_init(empty(s), 1);
        }
        for (int b = 0; b < kTurns; ++b) {
            tc_bar_init(acc_full(b), 1);
            tc_bar_init(acc_empty(b), kSumWarps);
        }
        tc_bar_init(drained, 1);
        abort_word = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == kMmaWarp) tc_alloc(tc_smem(&tmem_slot), kTurns * BN);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_slot;
    wait_previous_kernel();

    const int slices = (job.k_chunks + kSliceChunks - 1) / kSliceChunks;
    float sum[kCols];
    bool ok = true;
    if (warp < kSumWarps) {
        if (threadIdx.x == 0) {  // (read after the products)
            const int32_t* by = a.by + batch * kSlots;
            const int in = by[job.of_a] + by[job.of_b], d = by[job.of_d], d2 = by[job.of_d2];
            alphas[0] = ldexpf(job.alpha, d - in);
            alphas[1] = ldexpf(job.alpha2, d2 - in);
            diags[0] = ldexpf(job.diag, d);
            diags[1] = ldexpf(job.diag2, d2);
            out_factor = ldexpf(a.out_factor, -in);
        }
#pragma unroll
        for (int j = 0; j < kCols; ++j) sum[j] = 0.f;
        const uint32_t taddr = tmem + ((uint32_t)(32 * (warp & 3)) << 16) + (warp >> 2) * kCols;
        for (int i = 0; i < slices; ++i) {
            ok = tc_wait_warp(acc_full(i % kTurns), (uint32_t)(i / kTurns) & 1u, abort_flag, a.error, a.spin_limit);
            if (!ok) break;
            tc_fence_after();
#pragma unroll
            for (int part = 0; part < kCols / 32; ++part) {
                uint32_t v[32];
                tc_load32(taddr + (uint32_t)(i % kTurns) * BN + 32 * part, v);
                tc_load_wait();
#pragma unroll
                for (int j = 0; j < 32; ++j) sum[32 * part + j] += __uint_as_float(v[j]);
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) tc_bar_arrive(acc_empty(i % kTurns));
        }
    } else if (warp == kCopyWarp) {
        if (lane == 0) {
            int s = 0, issued = 0;
            uint32_t ph = 0;
            const int rows0 = bj * BN % kBlockRows, rb = bj * BN / kBlockRows;
            for (int kc = 0; kc < job.k_chunks; ++kc, ++issued) {
                ok = tc_wait(empty(s), ph ^ 1u, abort_flag, a.error, a.spin_limit);
                if (!ok) break;
                const uint32_t to = base + (uint32_t)s * kStage;
                const unsigned char* b = job.b.block(batch, rb, kc);
                tc_bar_expect(full(s), kStage);
                tc_bulk_load(to, job.a.block(batch, bi, kc), kBlockBytes, full(s));
                if (BN == kBlockRows) {
                    tc_bulk_load(to + kBlockBytes, b, kBlockBytes, full(s));
                } else if (BN > kBlockRows) {  // two blocks of rows, their high parts behind one another
#pragma unroll
                    for (int h = 0; h < BN / kBlockRows; ++h) {
                        const unsigned char* rows = job.b.block(batch, rb + h, kc);
                        tc_bulk_load(to + kBlockBytes + h * kHalfBytes, rows, kHalfBytes, full(s));
                        tc_bulk_load(to + kBlockBytes + kBBytes + h * kHalfBytes, rows + kHalfBytes, kHalfBytes, full(s));
                    }
                } else {
                    tc_bulk_load(to + kBlockBytes, b + rows0 * 128, kBBytes, full(s));
                    tc_bulk_load(to + kBlockBytes + kBBytes, b + kHalfBytes + rows0 * 128, kBBytes, full(s));
                }
                if (++s == kStages) {
                    s = 0;
                    ph ^= 1u;
                }
            }
            // Every copy has landed before this CTA's memory is used again or given up.  (A self-test's barriers wait for one
            // more arrival: theirs is made up for once the waits have run out.)
            if (a.drop) {
                for (uint32_t i = 0; i < 4 * a.spin_limit && !*abort_flag; ++i) __nanosleep(kTcSuspendNs);
                *abort_flag = 1;
            }
            for (int t = 0; t < min(issued, kStages); ++t) {
                const int uses = (issued - t + kStages - 1) / kStages;
                if (a.drop) tc_bar_arrive(full(t));
                for (uint32_t i = 0; i < kTcSpinLimit; ++i)
                    if (tc_bar_test(full(t), (uint32_t)(uses - 1) & 1u)) break;
            }
        }
        __syncwarp();
    } else if (warp == kMmaWarp) {
        const uint32_t instr = tc_instr(kBlockRows, BN, false);
        int s = 0;
        uint32_t ph = 0;
        for (int i = 0, kc = 0; i < slices && ok; ++i) {
            ok = tc_wait_warp(acc_empty(i % kTurns), ((uint32_t)(i / kTurns) & 1u) ^ 1u, abort_flag, a.error, a.spin_limit);
            for (int first = kc; ok && kc < min(first + kSliceChunks, job.k_chunks); ++kc) {
                ok = tc_wait_warp(full(s), ph, abort_flag, a.error, a.spin_limit);
                if (!ok) break;
                tc_fence_after();
                const uint32_t at = base + (uint32_t)s * kStage, d = tmem + (uint32_t)(i % kTurns) * BN;
                const uint64_t ah = tc_desc_k(at), al = tc_desc_k(at + kHalfBytes), bh = tc_desc_k(at + kBlockBytes),
                               bl = tc_desc_k(at + kBlockBytes + kBBytes);
#pragma unroll
                for (int j = 0; j < kBlockCols / 16; ++j) {  // the small terms first
                    tc_mma(d, al + 2 * j, bh + 2 * j, instr, kc != first || j != 0);
                    tc_mma(d, ah + 2 * j, bl + 2 * j, instr, 1u);
                }
#pragma unroll
                for (int j = 0; j < kBlockCols / 16; ++j) tc_mma(d, ah + 2 * j, bh + 2 * j, instr, 1u);
                tc_commit(empty(s));
                if (++s == kStages) {
                    s = 0;
                    ph ^= 1u;
                }
            }
            if (ok) tc_commit(acc_full(i % kTurns));
        }
        // tensor memory is freed, and shared memory used again, when the tensor core is done
        tc_commit(drained);
        for (uint32_t i = 0; i < kTcSpinLimit; ++i)
            if (tc_bar_test(drained, 0)) break;
        __syncwarp();
    }
    ok = __syncthreads_and(ok);
    const int q = warp & 3, half = (warp >> 2) & 1, row = 32 * q + lane;
    if (ok && a.out) {
        float* line = reinterpret_cast<float*>(base_p) + warp * (32 * 33);
        const float factor = out_factor;
        if (warp < kSumWarps)
#pragma unroll
            for (int part = 0; part < kCols / 32; ++part) {
#pragma unroll
                for (int j = 0; j < 32; ++j) line[lane * 33 + j] = sum[32 * part + j] * factor;
                __syncwarp();
                const int col = bj * BN + half * kCols + 32 * part + lane;
                if (col < a.out_cols)
                    for (int r = 0; r < 32; ++r) {
                        const int64_t i = (int64_t)bi * kBlockRows + 32 * q + r;
                        if (i >= a.out_rows) break;
                        const int64_t at = batch * a.out_batch + i * a.ldo + col;
                        const float o = line[r * 33 + lane];
                        if (a.out_dtype == GNNPRE_F32) static_cast<float*>(a.out)[at] = o;
                        else if (a.out_dtype == GNNPRE_BF16) static_cast<__nv_bfloat16*>(a.out)[at] = __float2bfloat16_rn(o);
                        else static_cast<__half*>(a.out)[at] = __float2half_rn(o);
                    }
                __syncwarp();
            }
    } else if (ok) {
        // D's blocks of 64 columns lie behind one another in shared memory, then its transpose's blocks of 64 columns (a row of
        // those is a column of the tile); both go out as they lie.
        const bool transposed = job.write_t || (a.symmetric && bi != bj);
        // (a wide tile and its transpose take shared memory one after the other)
        constexpr bool kApart = 2 * (BN / kBlockCols) * kBlockBytes > kPipeBytes;
        constexpr uint32_t kTransposed = kApart ? 0u : BN / kBlockCols * kBlockBytes;
        unsigned char* const tile_t = base_p + kTransposed;
        const int passes = (1 + job.write_2) * (kApart && transposed ? 2 : 1);
        for (int pass = 0; pass < passes; ++pass) {
            const int form = kApart && transposed ? pass / 2 : pass;
            const bool plain = !kApart || !transposed || pass % 2 == 0, turned = transposed && (!kApart || pass % 2 == 1);
            const Split& to = form ? job.d2 : job.d;
            const float alpha = alphas[form], on_diag = diags[form];
            if (pass) __syncthreads();  // (the pass before's copies have read their tiles: thread 0 has waited)
            if (warp < kSumWarps)
#pragma unroll
                for (int part = 0; part < kCols / 32; ++part) {
                    const int c0 = half * kCols + 32 * part;
                    const int diag = bi * kBlockRows + row - (bj * BN + c0);  // the column of these 32 that lies on the diagonal
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        float o[8];
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            o[e] = alpha * sum[32 * part + 8 * j + e];
                            if (8 * j + e == diag) o[e] += on_diag;
                        }
                        uint4 hi, lo;
                        split8(o, hi, lo);
                        unsigned char* d = base_p + c0 / kBlockCols * kBlockBytes + block_byte(row, c0 % kBlockCols + 8 * j);
                        if (plain) {
                            *reinterpret_cast<uint4*>(d) = hi;
                            *reinterpret_cast<uint4*>(d + kHalfBytes) = lo;
                        }
                        if (turned) {
                            const __half* h = reinterpret_cast<const __half*>(&hi);
                            const __half* l = reinterpret_cast<const __half*>(&lo);
#pragma unroll
                            for (int e = 0; e < 8; ++e) {
                                unsigned char* t = tile_t + row / kBlockCols * (2 * kBBytes) + block_byte(c0 + 8 * j + e, row % kBlockCols);
                                *reinterpret_cast<__half*>(t) = h[e];
                                *reinterpret_cast<__half*>(t + kBBytes) = l[e];
                            }
                        }
                    }
                }
            tc_fence_async();
            __syncthreads();
            if (threadIdx.x == 0) {
                if (plain)
#pragma unroll
                    for (int b = 0; b < BN / kBlockCols; ++b)
                        tc_bulk_store(to.block(batch, bi, bj * (BN / kBlockCols) + b), base + b * kBlockBytes, kBlockBytes);
                if (turned) {
                    const Split& to_t = job.write_t ? job.dt : to;
                    const int rows0 = bj * BN % kBlockRows;
                    constexpr uint32_t kPiece = kBBytes < kHalfBytes ? kBBytes : kHalfBytes;  // rows of one block
#pragma unroll
                    for (int b = 0; b < 2; ++b)
#pragma unroll
                        for (uint32_t h = 0; h < kBBytes / kPiece; ++h) {
                            unsigned char* t = to_t.block(batch, bj * BN / kBlockRows + (int)h, 2 * bi + b) + rows0 * 128;
                            const uint32_t from = base + kTransposed + b * 2 * kBBytes + h * kPiece;
                            tc_bulk_store(t, from, kPiece);
                            tc_bulk_store(t + kHalfBytes, from + kBBytes, kPiece);
                        }
                }
                asm volatile("cp.async.bulk.commit_group;" ::: "memory");
                if (pass + 1 < passes) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
                else asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
            }
        }
    }
    if (warp == kMmaWarp) {
        tc_fence_after();
        tc_free(tmem, kTurns * BN);
    }
}

// ------------------------------------------------------------------------------------------------ small matrices, one launch

// All of it for one matrix by one cluster of CTAs, which share out the tiles of each product, exchange them through the L2 and wait
// for one another between products (three per step).  A product by itself takes some 7.5 us as a launch of its own: its CTAs
// start, set up barriers and tensor memory, wait for the first copies, and leave.
struct Steps {
    StepFactors by_all[kMaxSteps];  // with the coefficients' bounds
    AllBounds all;
    float scale;
};

struct Cluster {
    Source src;
    Split a, a2, p, xt[2];   // (x and xt[0] are the source's)
    int32_t rp, np, k_r, k_n, steps;
    void* out;
    int64_t ldo, out_batch;
    int32_t* error;
    uint32_t spin_limit;
    int32_t drop;
    Steps s;
};

constexpr int kClusterTile = 64;                                         // columns of a tile
constexpr uint32_t kClusterStage = kBlockBytes + kClusterTile * 128 * 2; // a chunk of A's 128 rows and B's 64
constexpr int kClusterStages = 3;
constexpr int kClusterStaging = 2 * kBlockBytes;                         // a tile and its transpose
constexpr int kClusterSmem = kClusterStages * (int)kClusterStage + kClusterStaging + 1024;
constexpr int kClusterSourceTiles = (kClusterSmem - 1024) / (64 * 65 * 4);
constexpr int kMostClusterTiles = 32;   // tiles of X in a product, at most
static_assert(2 * kMostClusterTiles / 8 <= kClusterSourceTiles, "the [64, 64] tiles of X that a CTA reads fit");

__device__ __forceinline__ void ns_cluster_sync() {
    // what either proxy has written is seen by either proxy of the others
    asm volatile("fence.proxy.async;" ::: "memory");
    __syncwarp();
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
    asm volatile("fence.proxy.async;" ::: "memory");
}

__device__ __forceinline__ void ns_sum_warps_sync() { asm volatile("bar.sync 1, 256;" ::: "memory"); }

__global__ void __launch_bounds__(kProductThreads, 1) k_ns_cluster(const __grid_constant__ Cluster a) {
    constexpr int BN = kClusterTile, kCols = BN / 2;
    constexpr uint32_t kBBytes = BN * 128;
    extern __shared__ unsigned char ns_smem[];
    __shared__ __align__(8) unsigned long long bars[2 * kClusterStages + 2 * kAccs + 1];
    __shared__ uint32_t tmem_slot;
    __shared__ int abort_word;
    __shared__ double room[kProductThreads / 32];
    volatile int* abort_flag = &abort_word;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    uint32_t rank, ctas;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    asm("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(ctas));
    const int64_t batch = blockIdx.x / ctas;
    const uint32_t base = (tc_smem(ns_smem) + 1023u) & ~1023u;
    unsigned char* const base_p = ns_smem + (base - tc_smem(ns_smem));
    const uint32_t bar0 = tc_smem(&bars[0]);
    auto full = [&](int s) { return bar0 + 8u * s; };
    auto empty = [&](int s) { return bar0 + 8u * (kClusterStages + s); };
    auto acc_full = [&](int b) { return bar0 + 8u * (2 * kClusterStages + b); };
    auto acc_empty = [&](int b) { return bar0 + 8u * (2 * kClusterStages + kAccs + b); };
    const uint32_t drained = bar0 + 8u * (2 * kClusterStages + 2 * kAccs);
    if (threadIdx.x == 0) {
        for (int s = 0; s < kClusterStages; ++s) {
            tc_bar_init(full(s), 1 + (a.drop ? 1 : 0));
            tc_bar_init(empty(s), 1);
        }
        for (int b = 0; b < kAccs; ++b) {
            tc_bar_init(acc_full(b), 1);
            tc_bar_init(acc_empty(b), kSumWarps);
        }
        tc_bar_init(drained, 1);
        abort_word = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == kMmaWarp) tc_alloc(tc_smem(&tmem_slot), kAccs * BN);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_slot;

    // G, read once: this CTA's [64, 64] tiles of X go to shared memory, their squares to the norm
    const Source& src = a.src;
    const int side_tiles = a.np / 64, tiles = side_tiles * (a.rp / 64);
    float(*const tile)[64][65] = reinterpret_cast<float(*)[64][65]>(base_p);
    double sum2 = 0;
    for (int t = rank, k = 0; t < tiles; t += ctas, ++k) {
        const int i0 = t / side_tiles * 64, j0 = t % side_tiles * 64, fast = threadIdx.x & 63;
        if (warp >= kSumWarps) continue;
        const int gi0 = (src.tall ? j0 : i0) + (threadIdx.x >> 6), gj = (src.tall ? i0 : j0) + fast;
        float v[16];
        with_type(src, batch, [&](const auto* g) {
#pragma unroll
            for (int u = 0; u < 16; ++u) v[u] = to_f32(g[(int64_t)min(gi0 + 4 * u, src.rows - 1) * src.ldg + min(gj, src.cols - 1)]);
        });
#pragma unroll
        for (int u = 0; u < 16; ++u) {
            const int slow = (threadIdx.x >> 6) + 4 * u;
            const float o = gi0 + 4 * u < src.rows && gj < src.cols ? v[u] : 0.f;
            tile[k][src.tall ? fast : slow][src.tall ? slow : fast] = o;
            sum2 += (double)o * o;
        }
    }
#pragma unroll
    for (int d = 16; d > 0; d /= 2) sum2 += __shfl_xor_sync(0xffffffffu, sum2, d);
    if (lane == 0) room[warp] = sum2;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < kSumWarps; ++w) sum2 += room[w];
        src.partial[batch * kNormBlocks + rank] = sum2;
    }
    ns_cluster_sync();
    if (threadIdx.x < 32) {  // the CTAs' sums, in their order
        double v = lane < (int)ctas ? __ldcg(src.partial + batch * kNormBlocks + lane) : 0.0, total = 0;
        for (int c = 0; c < (int)ctas; ++c) total += __shfl_sync(0xffffffffu, v, c);
        if (lane == 0) {
            room[0] = 1.0 / (sqrt(total) + src.eps);
            room[1] = sqrt(total) * room[0];
        }
    }
    __syncthreads();
    const double norm_of_x = room[1];
    const bool small = norm_of_x < kOwnBounds;
    double bound = first_bound(norm_of_x);  // of X, where it goes by its own; and X's exponent
    int ex = exponent_for(bound);
    const double scale = room[0] * (small ? ldexp(1.0, ex) : (double)src.factor);
    StepFactors f;
    for (int t = rank, k = 0; t < tiles; t += ctas, ++k) {
        const int i0 = t / side_tiles * 64, j0 = t % side_tiles * 64;
        for (int c = threadIdx.x; c < 64 * 8; c += kProductThreads) {
            const int row = c >> 3, chunk = c & 7;
            float v[8];
            uint4 hi, lo;
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = (float)((double)tile[k][row][8 * chunk + e] * scale);
            split8(v, hi, lo);
            unsigned char* d = src.x.block(batch, (i0 + row) / kBlockRows, j0 / kBlockCols) + block_byte((i0 + row) % kBlockRows, 8 * chunk);
            *reinterpret_cast<uint4*>(d) = hi;
            *reinterpret_cast<uint4*>(d + kHalfBytes) = lo;
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = (float)((double)tile[k][8 * chunk + e][row] * scale);
            split8(v, hi, lo);
            d = src.xt.block(batch, (j0 + row) / kBlockRows, i0 / kBlockCols) + block_byte((j0 + row) % kBlockRows, 8 * chunk);
            *reinterpret_cast<uint4*>(d) = hi;
            *reinterpret_cast<uint4*>(d + kHalfBytes) = lo;
        }
    }
    ns_cluster_sync();

    // chunks copied or multiplied, accumulators filled or added up so far: each role counts for itself
    int chunk = 0, issued = 0;
    bool ok = true;
    const uint32_t instr = tc_instr(kBlockRows, BN, false);
    unsigned char* const staging_p = base_p + kClusterStages * kClusterStage;
    const uint32_t staging = base + kClusterStages * kClusterStage;
    bool stored = false;
    for (int stage = 0; stage < 3 * a.steps; ++stage) {
        const int step = stage / 3, kind = stage % 3;
        const bool last = stage == 3 * a.steps - 1, tall = last && src.tall;
        if (kind == 0) {
            f = a.s.by_all[step];
            if (small) {
                double p, next;
                own_bounds(a.s.all.c, bound, a.s.all.p[step], a.s.all.x[step + 1], &p, &next);
                f = step_factors(a.s.all.c, false, a.s.scale, bound, p, next, &ex);
                bound = next;
            }
        }
        const Split& xt = a.xt[step & 1];
        const Split& sa = kind == 0 ? src.x : kind == 1 ? a.a : tall ? xt : a.p;
        const Split& sb = kind == 0 ? src.x : kind == 1 ? a.a2 : tall ? a.p : xt;
        const int rows = tall ? a.np : a.rp, cols = kind < 2 || tall ? a.rp : a.np;
        const int k_chunks = kind == 0 ? a.k_n : a.k_r, tiles_n = cols / BN, all = rows / kBlockRows * tiles_n;
        for (int t = rank; t < all; t += ctas) {
            const int bi = t / tiles_n, bj = t % tiles_n;
            if (warp < kSumWarps) {
                float sum[kCols];
#pragma unroll
                for (int j = 0; j < kCols; ++j) sum[j] = 0.f;
                const int q = warp & 3, half = warp >> 2, row = 32 * q + lane;
                for (int i = 0; i < k_chunks; ++i, ++chunk) {
                    ok = ok && tc_wait_warp(acc_full(chunk % kAccs), (uint32_t)(chunk / kAccs) & 1u, abort_flag, a.error, a.spin_limit);
                    if (!ok) break;
                    tc_fence_after();
                    uint32_t v[32];
                    tc_load32(tmem + ((uint32_t)(32 * q) << 16) + half * kCols + (uint32_t)(chunk % kAccs) * BN, v);
                    tc_load_wait();
#pragma unroll
                    for (int j = 0; j < 32; ++j) sum[j] += __uint_as_float(v[j]);
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) tc_bar_arrive(acc_empty(chunk % kAccs));
                }
                if (last) {
                    if (!ok) continue;
                    float* line = reinterpret_cast<float*>(staging_p) + warp * (32 * 33);
#pragma unroll
                    for (int j = 0; j < 32; ++j) line[lane * 33 + j] = sum[j] * f.out;
                    __syncwarp();
                    const int col = bj * BN + half * kCols + lane;
                    if (col < src.cols)
                        for (int r = 0; r < 32; ++r) {
                            const int64_t i = (int64_t)bi * kBlockRows + 32 * q + r;
                            if (i >= src.rows) break;
                            const int64_t at = batch * a.out_batch + i * a.ldo + col;
                            const float o = line[r * 33 + lane];
                            if (src.dtype == GNNPRE_F32) static_cast<float*>(a.out)[at] = o;
                            else if (src.dtype == GNNPRE_BF16) static_cast<__nv_bfloat16*>(a.out)[at] = __float2bfloat16_rn(o);
                            else static_cast<__half*>(a.out)[at] = __float2half_rn(o);
                        }
                    __syncwarp();
                    continue;
                }
                const int c0 = half * kCols, diag = bi * kBlockRows + row - (bj * BN + c0);
                // the staging is free when the last tile's copies have read it
                if (threadIdx.x == 0 && stored) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
                ns_sum_warps_sync();
                auto stage_tile = [&](unsigned char* to, float alpha, float on_diag, bool transpose) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        float o[8];
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            o[e] = alpha * sum[8 * j + e];
                            if (8 * j + e == diag) o[e] += on_diag;
                        }
                        uint4 hi, lo;
                        split8(o, hi, lo);
                        unsigned char* d = to + block_byte(row, c0 + 8 * j);
                        *reinterpret_cast<uint4*>(d) = hi;
                        *reinterpret_cast<uint4*>(d + kHalfBytes) = lo;
                        if (transpose) {
                            const __half* h = reinterpret_cast<const __half*>(&hi);
                            const __half* l = reinterpret_cast<const __half*>(&lo);
#pragma unroll
                            for (int e = 0; e < 8; ++e) {
                                unsigned char* u = staging_p + kBlockBytes + row / kBlockCols * (2 * kBBytes) + block_byte(c0 + 8 * j + e, row % kBlockCols);
                                *reinterpret_cast<__half*>(u) = h[e];
                                *reinterpret_cast<__half*>(u + kBBytes) = l[e];
                            }
                        }
                    }
                };
                if (kind == 0) {
                    stage_tile(staging_p, f.gram, 0.f, false);
                    stage_tile(staging_p + kBlockBytes, f.gram2, f.diag2, false);
                } else if (kind == 1) {
                    stage_tile(staging_p, f.p, f.p_diag, false);
                } else {
                    stage_tile(staging_p, f.apply, 0.f, true);
                }
                tc_fence_async();
                ns_sum_warps_sync();
                if (threadIdx.x == 0) {
                    tc_bulk_store((kind == 0 ? a.a : kind == 1 ? a.p : src.x).block(batch, bi, bj), staging, kBlockBytes);
                    if (kind == 0) tc_bulk_store(a.a2.block(batch, bi, bj), staging + kBlockBytes, kBlockBytes);
                    if (kind == 2) {
                        const int rows0 = bj * BN % kBlockRows;
#pragma unroll
                        for (int b = 0; b < 2; ++b) {
                            unsigned char* u = a.xt[(step & 1) ^ 1].block(batch, bj * BN / kBlockRows, 2 * bi + b) + rows0 * 128;
                            tc_bulk_store(u, staging + kBlockBytes + b * 2 * kBBytes, kBBytes);
                            tc_bulk_store(u + kHalfBytes, staging + kBlockBytes + b * 2 * kBBytes + kBBytes, kBBytes);
                        }
                    }
                    asm volatile("cp.async.bulk.commit_group;" ::: "memory");
                    stored = true;
                }
            } else if (warp == kCopyWarp) {
                if (lane == 0) {
                    const int rows0 = bj * BN % kBlockRows, rb = bj * BN / kBlockRows;
                    for (int kc = 0; kc < k_chunks && ok; ++kc) {
                        const int s = chunk % kClusterStages;
                        ok = tc_wait(empty(s), ((uint32_t)(chunk / kClusterStages) & 1u) ^ 1u, abort_flag, a.error, a.spin_limit);
                        if (!ok) break;
                        const uint32_t to = base + (uint32_t)s * kClusterStage;
                        const unsigned char* b = sb.block(batch, rb, kc);
                        tc_bar_expect(full(s), kClusterStage);
                        tc_bulk_load(to, sa.block(batch, bi, kc), kBlockBytes, full(s));
                        tc_bulk_load(to + kBlockBytes, b + rows0 * 128, kBBytes, full(s));
                        tc_bulk_load(to + kBlockBytes + kBBytes, b + kHalfBytes + rows0 * 128, kBBytes, full(s));
                        ++chunk;
                        ++issued;
                    }
                }
                __syncwarp();
            } else {
                for (int kc = 0; kc < k_chunks && ok; ++kc) {
                    const int s = chunk % kClusterStages;
                    ok = tc_wait_warp(acc_empty(chunk % kAccs), ((uint32_t)(chunk / kAccs) & 1u) ^ 1u, abort_flag, a.error, a.spin_limit) &&
                         tc_wait_warp(full(s), (uint32_t)(chunk / kClusterStages) & 1u, abort_flag, a.error, a.spin_limit);
                    if (!ok) break;
                    tc_fence_after();
                    const uint32_t at = base + (uint32_t)s * kClusterStage, d = tmem + (uint32_t)(chunk % kAccs) * BN;
                    const uint64_t ah = tc_desc_k(at), al = tc_desc_k(at + kHalfBytes), bh = tc_desc_k(at + kBlockBytes),
                                   bl = tc_desc_k(at + kBlockBytes + kBBytes);
#pragma unroll
                    for (int j = 0; j < kBlockCols / 16; ++j) {
                        tc_mma(d, al + 2 * j, bh + 2 * j, instr, j != 0);
                        tc_mma(d, ah + 2 * j, bl + 2 * j, instr, 1u);
                    }
#pragma unroll
                    for (int j = 0; j < kBlockCols / 16; ++j) tc_mma(d, ah + 2 * j, bh + 2 * j, instr, 1u);
                    tc_commit(empty(s));
                    tc_commit(acc_full(chunk % kAccs));
                    ++chunk;
                }
            }
        }
        if (!last) {
            if (threadIdx.x == 0 && stored) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
            ns_cluster_sync();  // (given up or not: every CTA comes here as often)
        }
    }
    if (warp == kCopyWarp && lane == 0) {
        // every copy has landed before this CTA leaves (a self-test's barriers: see k_ns_product)
        if (a.drop) {
            for (uint32_t i = 0; i < 4 * a.spin_limit && !*abort_flag; ++i) __nanosleep(kTcSuspendNs);
            *abort_flag = 1;
        }
        for (int t = 0; t < min(issued, kClusterStages); ++t) {
            if (a.drop) tc_bar_arrive(full(t));
            for (uint32_t i = 0; i < kTcSpinLimit; ++i)
                if (tc_bar_test(full(t), (uint32_t)((issued - t + kClusterStages - 1) / kClusterStages - 1) & 1u)) break;
        }
    }
    if (warp == kMmaWarp) {
        tc_commit(drained);
        for (uint32_t i = 0; i < kTcSpinLimit; ++i)
            if (tc_bar_test(drained, 0)) break;
    }
    tc_fence_before();
    __syncthreads();
    if (warp == kMmaWarp) {
        tc_fence_after();
        tc_free(tmem, kAccs * BN);
    }
}

// ------------------------------------------------------------------------------------------------ r <= 128: on the chip

// With r <= 128 all r x r matrices are one tile, and X (or, of a long one, a CTA's share of its columns) stays in shared memory
// from the first step to the last.  It serves A = X X^T as both operands, rows along K, and P X as operand B as it lies: a row
// of X is a row along K there (MN-major).  The CTAs of a cluster add up their shares' A, in the order of their ranks, and each
// computes P for itself.  The sixteen warps read the accumulators: warps w, w + 4, w + 8 and w + 12 share lanes 32 (w & 3) .., and take
// 32-column pieces in turn; A stays in their registers for P.  (With eight warps reading, splitting and storing took 13,000 of a
// step's 21,000 cycles on [256, 128], with the products, 96 of them, at the tensor core's rate in the rest.)  As each K-chunk's
// large terms have an accumulator of their own, four cuts of the tensor core meet in a sum.
constexpr int kChipThreads = 512;
constexpr int kChipCols = 256;                       // columns of X in a CTA
constexpr int kChipMaxCtas = 8;
constexpr int kChipSmem = (kChipCols / kBlockCols + 3) * kBlockBytes + 1024;  // X, A or P, and room for half of a sum over the CTAs

struct Chip {
    Source src;          // (x, xt: unused)
    int32_t cols;        // of X per CTA, a multiple of 64
    int32_t steps;
    void* out;
    int64_t ldo, out_batch;
    int32_t* error;
    uint32_t spin_limit;
    int32_t drop;
    Steps s;
};

__device__ __forceinline__ float4 ns_read_peer(uint32_t addr, uint32_t rank) {
    float4 v;
    asm volatile(
        "{\n\t.reg .b32 remote;\n\t"
        "mapa.shared::cluster.u32 remote, %4, %5;\n\t"
        "ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [remote];\n\t}"
        : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w)
        : "r"(addr), "r"(rank)
        : "memory");
    return v;
}

__global__ void __launch_bounds__(kChipThreads, 1) k_ns_chip(const __grid_constant__ Chip a) {
    extern __shared__ unsigned char ns_smem[];
    __shared__ __align__(8) unsigned long long bars[2];
    __shared__ uint32_t tmem_slot;
    __shared__ int abort_word;
    __shared__ double room[kChipThreads / 32];
    __shared__ StepFactors f;  // of a step
    __shared__ double bound;   // of X where it goes by its own, else 0; and X's exponent (one thread keeps them and f)
    __shared__ int ex;
    volatile int* abort_flag = &abort_word;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    uint32_t rank, ctas;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    asm("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(ctas));
    const int64_t batch = blockIdx.x / ctas;
    const uint32_t base = (tc_smem(ns_smem) + 1023u) & ~1023u;
    unsigned char* const base_p = ns_smem + (base - tc_smem(ns_smem));
    const uint32_t xs = base, as = base + kChipCols / kBlockCols * kBlockBytes;       // X's blocks; A's, later P's two
    unsigned char* const as_p = base_p + kChipCols / kBlockCols * kBlockBytes;
    const uint32_t done = tc_smem(&bars[0]), drained = tc_smem(&bars[1]);
    if (threadIdx.x == 0) {
        tc_bar_init(done, 1);
        tc_bar_init(drained, 1);
        abort_word = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 0) tc_alloc(tc_smem(&tmem_slot), 512);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_slot;
    const Source& src = a.src;
    const int r = src.tall ? src.cols : src.rows, n = src.tall ? src.rows : src.cols;
    const int j0 = (int)rank * a.cols, blocks = a.cols / kBlockCols;
    const int q = warp & 3, piece = warp >> 2, row = 32 * q + lane;  // this thread's lane of the accumulators, its piece of 128 columns

    {
        // G is read along its rows and laid down as fp32 where X will be: rows of 64 16-byte pieces, turned by the row.  Then every thread
        // takes 64 columns of a row of X, and once all have theirs, X in two parts takes the place.  The squares are added up in 64 bits
        // between the loads, which hide them (in a pass of its own over the registers: 1.3 us more on [256, 128]).
        constexpr int kWarps = kChipThreads / 32;
        auto place = [&](int i, int j) { return base_p + i * (kChipCols * 4) + (((j >> 2) ^ (i & 31)) << 4) + (j & 3) * 4; };
        double sum2 = 0, odd2 = 0;
        auto keep = [&](int i, int j, int k, float v) {
            *reinterpret_cast<float*>(place(i, j)) = v;
            double& to = k & 1 ? odd2 : sum2;
            to = fma((double)v, (double)v, to);
        };
        auto load = [&](auto* p) {
            p += batch * src.batch_stride;
            if (src.tall) {  // a row of G is a column of X: lanes are rows of X
#pragma unroll 4
                for (int j = warp; j < a.cols; j += kWarps)
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const int i = 32 * k + lane;
                        const float v = to_f32(p[(int64_t)min(j0 + j, n - 1) * src.ldg + min(i, r - 1)]);
                        keep(i, j, k, i < r && j0 + j < n ? v : 0.f);
                    }
            } else {
#pragma unroll 2
                for (int i = warp; i < 128; i += kWarps)
#pragma unroll
                    for (int k = 0; k < kChipCols / 32; ++k) {
                        const int j = 32 * k + lane;
                        const float v = to_f32(p[(int64_t)min(i, r - 1) * src.ldg + min(j0 + j, n - 1)]);
                        keep(i, j, k, i < r && j < a.cols && j0 + j < n ? v : 0.f);
                    }
            }
        };
        if (src.dtype == GNNPRE_F32) load(static_cast<const float*>(src.g));
        else if (src.dtype == GNNPRE_BF16) load(static_cast<const __nv_bfloat16*>(src.g));
        else load(static_cast<const __half*>(src.g));
        sum2 += odd2;
#pragma unroll
        for (int d = 16; d > 0; d /= 2) sum2 += __shfl_xor_sync(0xffffffffu, sum2, d);
        if (lane == 0) room[warp] = sum2;
        __syncthreads();
        constexpr int kGroups = kChipCols / 32;  // of eight columns
        float g[kGroups][8];
#pragma unroll
        for (int k = 0; k < kGroups; ++k) {
            const int c = 8 * (4 * k + piece);
            if (c >= a.cols) continue;
            const float4 u = *reinterpret_cast<const float4*>(place(row, c)), w = *reinterpret_cast<const float4*>(place(row, c + 4));
            g[k][0] = u.x, g[k][1] = u.y, g[k][2] = u.z, g[k][3] = u.w;
            g[k][4] = w.x, g[k][5] = w.y, g[k][6] = w.z, g[k][7] = w.w;
        }
        // the warps' sums and then the CTAs', in their order
        sum2 = room[0];
        for (int w = 1; w < kWarps; ++w) sum2 += room[w];
        if (ctas > 1) {
            if (threadIdx.x == 0) src.partial[batch * kNormBlocks + rank] = sum2;
            ns_cluster_sync();
            sum2 = 0;
            for (uint32_t c = 0; c < ctas; ++c) sum2 += __ldcg(src.partial + batch * kNormBlocks + c);
        }
        __syncthreads();
        // entries are brought to size one first: neither tiny nor huge ones leave fp32's range
        const double size = sqrt(sum2), over = 1.0 / (size + src.eps), norm_of_x = size * over;
        const bool small = norm_of_x < kOwnBounds;
        const double first = small ? first_bound(norm_of_x) : 0.0;
        const float to_fp16 = small ? ldexpf(1.f, exponent_for(first)) : src.factor;
        if (threadIdx.x == kChipThreads - 32) {
            bound = first;
            ex = exponent_for(first);
        }
        const int exponent = min(max(ilogb(size), -126), 126);
        const float to_one = ldexpf(1.f, -exponent), scale = (float)ldexp(over * (double)to_fp16, exponent);
#pragma unroll
        for (int k = 0; k < kGroups; ++k) {
            const int c = 8 * (4 * k + piece);
            if (c >= a.cols) continue;
            float v[8];
            uint4 hi, lo;
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = g[k][e] * to_one * scale;
            split8(v, hi, lo);
            unsigned char* d = base_p + c / kBlockCols * kBlockBytes + block_byte(row, c % kBlockCols);
            *reinterpret_cast<uint4*>(d) = hi;
            *reinterpret_cast<uint4*>(d + kHalfBytes) = lo;
        }
    }

    bool ok = true;
    uint32_t ph = 0;
    const uint32_t square = tc_instr(kBlockRows, 128, false), wide = tc_instr(kBlockRows, a.cols, false, true);
    // operands written by this CTA's threads, seen by the tensor core
    auto publish = [&] {
        tc_fence_async();
        tc_fence_before();
        __syncthreads();
        tc_fence_after();
    };
    // the products issued since, complete for everybody or given up by everybody
    auto finish = [&] {
        if (warp == 0 && !a.drop) tc_commit(done);
        ok = __syncthreads_and(ok && tc_wait_warp(done, ph, abort_flag, a.error, a.spin_limit));
        ph ^= 1u;
        tc_fence_after();
    };
    // sums of `accs` accumulators `apart` columns apart, 32 columns from `col`
    auto read32 = [&](int col, int accs, int apart, float (&sum)[32]) {
        uint32_t v[32];
        tc_load32(tmem + ((uint32_t)(32 * q) << 16) + (uint32_t)col, v);
        tc_load_wait();
#pragma unroll
        for (int j = 0; j < 32; ++j) sum[j] = __uint_as_float(v[j]);
        for (int k = 1; k < accs; ++k) {
            tc_load32(tmem + ((uint32_t)(32 * q) << 16) + (uint32_t)(k * apart + col), v);
            tc_load_wait();
#pragma unroll
            for (int j = 0; j < 32; j += 2) {
                const float2 two = __fadd2_rn(make_float2(sum[j], sum[j + 1]), make_float2(__uint_as_float(v[j]), __uint_as_float(v[j + 1])));
                sum[j] = two.x;
                sum[j + 1] = two.y;
            }
        }
    };
    auto times = [&](float (&o)[32], float f) {
#pragma unroll
        for (int j = 0; j < 32; j += 2) {
            const float2 two = __fmul2_rn(make_float2(o[j], o[j + 1]), make_float2(f, f));
            o[j] = two.x;
            o[j + 1] = two.y;
        }
    };
    // 32 of this thread's numbers to columns col.. of the blocks at p
    auto write32 = [&](unsigned char* p, int col, const float (&o)[32]) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            float v[8];
            uint4 hi, lo;
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = o[8 * j + e];
            split8(v, hi, lo);
            unsigned char* d = p + col / kBlockCols * kBlockBytes + block_byte(row, col % kBlockCols + 8 * j);
            *reinterpret_cast<uint4*>(d) = hi;
            *reinterpret_cast<uint4*>(d + kHalfBytes) = lo;
        }
    };
    for (int step = 0; step < a.steps; ++step) {
        // A = X X^T of this share: the small terms of all chunks and the large ones of the first in one accumulator, those of the
        // others in one each
        publish();
        if (warp == 0 && ok) {
            for (int b = 0; b < blocks; ++b) {
                const uint64_t h = tc_desc_k(xs + b * kBlockBytes), l = tc_desc_k(xs + b * kBlockBytes + kHalfBytes);
#pragma unroll
                for (int j = 0; j < kBlockCols / 16; ++j) {
                    tc_mma(tmem, l + 2 * j, h + 2 * j, square, b != 0 || j != 0);
                    tc_mma(tmem, h + 2 * j, l + 2 * j, square, 1u);
                }
            }
            for (int b = 0; b < blocks; ++b) {
                const uint64_t h = tc_desc_k(xs + b * kBlockBytes);
#pragma unroll
                for (int j = 0; j < kBlockCols / 16; ++j) tc_mma(tmem + 128 * b, h + 2 * j, h + 2 * j, square, b == 0 || j != 0);
            }
        }
        if (threadIdx.x == kChipThreads - 32) {  // (everybody has done with the last step's, and nobody reads these before finish)
            if (bound > 0.0) {
                double p, next;
                own_bounds(a.s.all.c, bound, a.s.all.p[step], a.s.all.x[step + 1], &p, &next);
                f = step_factors(a.s.all.c, true, a.s.scale, bound, p, next, &ex);
                bound = next;
            } else {
                f = a.s.by_all[step];
            }
        }
        __syncwarp();
        finish();
        float av[32];
        read32(32 * piece, blocks, 128, av);
        times(av, f.gram);
        if (ctas > 1) {
            // The shares' sums, laid down where A will be: rows of 32 pieces of 16 bytes, turned by the row.  Half of the rows at a time
            // the CTAs' are read piece by piece as they lie, neighbouring lanes neighbouring pieces (a lane to a row: 40 us a step
            // with four CTAs), and added up in a place of their own.
#pragma unroll
            for (int j = 0; j < 8; ++j)
                *reinterpret_cast<float4*>(as_p + row * 512 + ((8 * piece + j) ^ (row & 31)) * 16) =
                    make_float4(av[4 * j], av[4 * j + 1], av[4 * j + 2], av[4 * j + 3]);
            ns_cluster_sync();
            unsigned char* const sum_p = as_p + 2 * kBlockBytes;
            for (int part = 0; part < 2; ++part) {
                constexpr int kPieces = kBlockBytes / 16 / kChipThreads;  // of a thread
                float4 sum[kPieces];
                for (uint32_t c = 0; c < ctas; ++c) {
                    float4 v[kPieces];
#pragma unroll
                    for (int j = 0; j < kPieces; ++j) v[j] = ns_read_peer(as + (uint32_t)(part * kBlockBytes + (j * kChipThreads + (int)threadIdx.x) * 16), c);
#pragma unroll
                    for (int j = 0; j < kPieces; ++j)
                        sum[j] = c == 0 ? v[j] : make_float4(sum[j].x + v[j].x, sum[j].y + v[j].y, sum[j].z + v[j].z, sum[j].w + v[j].w);
                }
#pragma unroll
                for (int j = 0; j < kPieces; ++j) *reinterpret_cast<float4*>(sum_p + (j * kChipThreads + threadIdx.x) * 16) = sum[j];
                __syncthreads();
                if (row / 64 == part)
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const float4 v = *reinterpret_cast<const float4*>(sum_p + row % 64 * 512 + ((8 * piece + j) ^ (row & 31)) * 16);
                        av[4 * j] = v.x;
                        av[4 * j + 1] = v.y;
                        av[4 * j + 2] = v.z;
                        av[4 * j + 3] = v.w;
                    }
                __syncthreads();
            }
            ns_cluster_sync();
        }
        write32(as_p, 32 * piece, av);
        publish();
        // A A, then P = a I + b A + c A A over it
        if (warp == 0 && ok) {
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                const uint64_t h = tc_desc_k(as + b * kBlockBytes), l = tc_desc_k(as + b * kBlockBytes + kHalfBytes);
#pragma unroll
                for (int j = 0; j < kBlockCols / 16; ++j) {
                    tc_mma(tmem, l + 2 * j, h + 2 * j, square, b != 0 || j != 0);
                    tc_mma(tmem, h + 2 * j, l + 2 * j, square, 1u);
                }
            }
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                const uint64_t h = tc_desc_k(as + b * kBlockBytes);
#pragma unroll
                for (int j = 0; j < kBlockCols / 16; ++j) tc_mma(tmem + 128 * b, h + 2 * j, h + 2 * j, square, b == 0 || j != 0);
            }
        }
        finish();
        {
            const int col = 32 * piece;
            float o[32];
            read32(col, 2, 128, o);
            times(o, f.gram2);
            const float2 b = make_float2(f.diag2, f.diag2);
#pragma unroll
            for (int j = 0; j < 32; j += 2) {
                const float2 two = __ffma2_rn(b, make_float2(av[j], av[j + 1]), make_float2(o[j], o[j + 1]));
                o[j] = two.x;
                o[j + 1] = two.y;
            }
            if (piece == q) {  // the diagonal's warps
#pragma unroll
                for (int j = 0; j < 32; ++j)
                    if (j == lane) o[j] += f.p_diag;
            }
            write32(as_p, col, o);
        }
        publish();
        // P X: K is r here, a row of X a row along K
        if (warp == 0 && ok) {
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                const uint64_t h = tc_desc_k(as + b * kBlockBytes), l = tc_desc_k(as + b * kBlockBytes + kHalfBytes);
                const uint64_t xh = tc_desc_mn(xs + b * 64 * 128, kBlockBytes), xl = tc_desc_mn(xs + kHalfBytes + b * 64 * 128, kBlockBytes);
#pragma unroll
                for (int j = 0; j < kBlockCols / 16; ++j) {
                    tc_mma(tmem, l + 2 * j, xh + (2048 >> 4) * j, wide, b != 0 || j != 0);
                    tc_mma(tmem, h + 2 * j, xl + (2048 >> 4) * j, wide, 1u);
                }
            }
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                const uint64_t h = tc_desc_k(as + b * kBlockBytes), xh = tc_desc_mn(xs + b * 64 * 128, kBlockBytes);
#pragma unroll
                for (int j = 0; j < kBlockCols / 16; ++j) tc_mma(tmem + 256 * b, h + 2 * j, xh + (2048 >> 4) * j, wide, b == 0 || j != 0);
            }
        }
        finish();
        const bool last = step + 1 == a.steps;
        for (int col = 32 * piece; col < a.cols; col += 128) {
            float o[32];
            read32(col, 2, 256, o);
            if (!last) {
                times(o, f.apply);
                write32(base_p, col, o);
                continue;
            }
            if (!ok) continue;
            auto store = [&](int64_t i, int64_t j, float v) {
                const int64_t at = batch * a.out_batch + i * a.ldo + j;
                if (src.dtype == GNNPRE_F32) static_cast<float*>(a.out)[at] = v;
                else if (src.dtype == GNNPRE_BF16) static_cast<__nv_bfloat16*>(a.out)[at] = __float2bfloat16_rn(v);
                else static_cast<__half*>(a.out)[at] = __float2half_rn(v);
            };
            if (src.tall) {  // neighbouring lanes are neighbours in out's rows
#pragma unroll
                for (int j = 0; j < 32; ++j)
                    if (row < r && j0 + col + j < n) store(j0 + col + j, row, o[j] * f.out);
            } else {
                float* line = reinterpret_cast<float*>(as_p) + warp * (32 * 32);  // (P has been read); columns turned by the row
#pragma unroll
                for (int j = 0; j < 32; ++j) line[lane * 32 + (j ^ lane)] = o[j] * f.out;
                __syncwarp();
                if (j0 + col + lane < n)
                    for (int i = 0; i < 32 && 32 * q + i < r; ++i) store(32 * q + i, j0 + col + lane, line[i * 32 + (lane ^ i)]);
                __syncwarp();
            }
        }
        tc_fence_before();
    }
    if (warp == 0) {
        tc_commit(drained);
        for (uint32_t i = 0; i < kTcSpinLimit; ++i)
            if (tc_bar_test(drained, 0)) break;
    }
    if (ctas > 1) ns_cluster_sync();  // nobody reads this CTA's memory any more
    tc_fence_before();
    __syncthreads();
    if (warp == 0) {
        tc_fence_after();
        tc_free(tmem, 512);
    }
}

// ------------------------------------------------------------------------------------------------ host

// How large the polynomials can make the singular values, which start in [0, 1]; false: beyond kMostSpectral.
bool bounds_of(const float* coeffs, int32_t steps, AllBounds* out) {
    const double a = coeffs[0], b = coeffs[1], c = coeffs[2];
    out->c = Coeffs{coeffs[0], coeffs[1], coeffs[2]};
    if (!std::isfinite(a) || !std::isfinite(b) || !std::isfinite(c)) return false;
    double r = 1.0;
    for (int32_t k = 0; k < steps; ++k) {
        r = std::max(r * (1.0 + 1e-4), kLeastSpectral);  // (what rounding adds)
        out->x[k] = r;
        const double u1 = r * r;
        const auto p = [&](double u) { return std::fabs(a + b * u + c * u * u); };
        const auto x = [&](double u) { return std::sqrt(u) * p(u); };
        double mp = std::max(p(0), p(u1)), mx = x(u1);
        const auto inside = [&](double u, bool slope) {
            if (!(u > 0 && u < u1)) return;
            if (slope) mx = std::max(mx, x(u));
            else mp = std::max(mp, p(u));
        };
        if (c != 0) inside(-b / (2 * c), false);
        // d/ds (a s + b s^3 + c s^5) = a + 3 b u + 5 c u^2,  u = s^2
        if (c != 0) {
            const double d = 9 * b * b - 20 * a * c;
            if (d >= 0) {
                inside((-3 * b + std::sqrt(d)) / (10 * c), true);
                inside((-3 * b - std::sqrt(d)) / (10 * c), true);
            }
        } else if (b != 0) {
            inside(-a / (3 * b), true);
        }
        out->p[k] = mp;
        r = mx;
        if (!(r <= kMostSpectral) || !(mp <= 1024.0)) return false;
    }
    out->x[steps] = std::max(r, kLeastSpectral);
    return true;
}

struct NsShape {
    int64_t r, n, rp, np, batch;
    int32_t segment;  // steps at most between two X
    int32_t ctas;     // of the cluster that does all of a matrix; 0: a launch per product
    bool chip;        // ... from shared memory
    int64_t side, square;  // bytes of one split [rp, np], [rp, rp]
    int64_t xt[2], x, a, a2, t, p, q[2], partial, by, total;
};

// Steps of a segment at most (see above).
int32_t most_segment_steps(int32_t dtype) { return dtype == GNNPRE_BF16 ? 3 : dtype == GNNPRE_F16 ? 2 : 1; }

NsShape ns_shape(int64_t batch, int64_t rows, int64_t cols, int32_t steps, int32_t most) {
    NsShape s{};
    s.batch = batch;
    s.r = std::min(rows, cols);
    s.n = std::max(rows, cols);
    s.rp = (s.r + 127) / 128 * 128;
    s.np = (s.n + 127) / 128 * 128;
    // multiplications per step of a segment of g steps, in units of r^2: n + 2 n for its ends, (4 g - 3) r between
    const auto cost = [&](int g) { return (3.0 * s.np + (4.0 * g - 3.0) * s.rp) / g; };
    // One cluster per matrix where the square products leave a CTA one tile (r <= 256, eight tiles) and those of X few, and where all
    // matrices' clusters run at once: seven of 16 CTAs, fourteen of 8.  us, fp32, five steps, 16 CTAs / 8 / a launch per product:
    // one of 200 x 384 110 / 127 / 121, 256 x 512 117 / 137 / 128, 256 x 1,024 165 / 204 / 160; seven of them 111 / 128 / 126, 118 / 137 /
    // 135, 166 / 205 / 182; ten of 256 x 512 234 / 138 / 150, sixteen 350 / 273 / 155; one of 130 x 130 90 / 93 / 100.  Beyond: 256 x 1,536
    // 213 / 271 / 192, 384 x 384 194 / 266 / 138, 300 x 1,000 276 / 421 / 169.
    const int64_t tiles = s.rp / 128 * (s.np / kClusterTile);
    const bool ever_cluster = s.rp <= 256 && tiles <= kMostClusterTiles;  // (for some number of matrices)
    s.ctas = !ever_cluster || batch > 14 ? 0 : tiles > 8 && batch <= 7 ? 16 : 8;
    // On the chip where a matrix fits, and where eight CTAs are needed while all matrices' clusters run at once (else as above).  us, on
    // the chip / a launch per product: one of 64 x 64 35 / 77, 128 x 256 54 / 96, 128 x 1,000 101 / 144, 128 x 2,048 176 / 207; fourteen of
    // the last 199 / 269, eighteen 361 / 275; a hundred of 128 x 256 56 / 198, of 128 x 1,000 421 / 478.
    s.chip = s.r <= 128 && s.n <= kChipCols * kChipMaxCtas && (batch <= 14 || 2 * s.n <= kChipCols * kChipMaxCtas);
    if (s.chip)
        for (s.ctas = 1; s.ctas * kChipCols < s.n;) s.ctas *= 2;
    s.segment = 1;
    if (s.ctas) most = 1;
    for (int g = 2; g <= std::min(most, steps); ++g)
        if (cost(g) < 0.99 * cost(s.segment)) s.segment = g;
    s.side = s.rp * s.np * 4;
    s.square = s.rp * s.rp * 4;
    int64_t at = 0;
    const auto take = [&](int64_t bytes) {
        const int64_t here = at;
        at += (bytes * batch + 1023) / 1024 * 1024;
        return here;
    };
    if (s.chip) {
        s.partial = take((int64_t)sizeof(double) * kNormBlocks);
        s.total = at;
        return s;
    }
    s.x = take(s.side);
    s.xt[0] = take(s.side);
    // (where a cluster may do it, as much for a launch per product: a kept workspace serves fewer matrices than it was made for)
    s.xt[1] = steps > s.segment || ever_cluster ? take(s.side) : s.xt[0];
    s.a = take(s.square);
    s.a2 = take(s.square);
    s.p = take(s.square);
    s.q[0] = s.segment > 1 ? take(s.square) : s.p;
    s.q[1] = s.segment > 1 ? take(s.square) : s.p;
    s.t = s.segment > 1 ? take(s.square) : s.p;
    s.partial = take((int64_t)sizeof(double) * kNormBlocks);
    if (!s.ctas) s.by = take((int64_t)sizeof(int32_t) * kSlots);
    s.total = at;
    return s;
}

struct NsSelfTest {
    int32_t drop;
    uint32_t polls;
};

// One cluster of `ctas` CTAs per matrix.
template <typename Args>
int launch_clusters(void (*kernel)(Args), unsigned threads, int smem, int32_t ctas, int64_t batch, cudaStream_t st, const Args& args) {
    static std::atomic<bool> opted_in[kMaxDevices];  // (per kernel: their arguments' types differ)
    int dev = 0;
    GNNPRE_CUDA(cudaGetDevice(&dev));
    if (dev >= kMaxDevices || !opted_in[dev].load(std::memory_order_relaxed)) {
        GNNPRE_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
        GNNPRE_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1));
        if (dev < kMaxDevices) opted_in[dev].store(true, std::memory_order_relaxed);
    }
    cudaLaunchAttribute attr{};
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = (unsigned)ctas;
    attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(batch * ctas));
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = (size_t)smem;
    cfg.stream = st;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    GNNPRE_CUDA(cudaLaunchKernelEx(&cfg, kernel, args));
    return GNNPRE_OK;
}

template <int BN>
int launch_product_n(const Product& a, int64_t tiles_m, int64_t batch, cudaStream_t st) {
    constexpr int kSmem = kPipeBytes + 1024;
    static std::atomic<bool> opted_in[kMaxDevices];
    int dev = 0;
    GNNPRE_CUDA(cudaGetDevice(&dev));
    if (dev >= kMaxDevices || !opted_in[dev].load(std::memory_order_relaxed)) {
        GNNPRE_CUDA(cudaFuncSetAttribute(k_ns_product<BN>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem));
        if (dev < kMaxDevices) opted_in[dev].store(true, std::memory_order_relaxed);
    }
    const int64_t tiles = a.symmetric ? tiles_m * (tiles_m + 1) / 2 : tiles_m * a.tiles_n;
    return launch_after(k_ns_product<BN>, dim3((unsigned)tiles, 1, (unsigned)(batch * a.jobs)), kProductThreads, kSmem, true, st, a);
}

// D has rows x cols elements.
int launch_product(Product& a, int64_t rows, int64_t cols, int64_t batch, bool symmetric, int sms, cudaStream_t st) {
    const int64_t tiles_m = rows / 128;
    // Tiles of 128 x 64 while they fit the machine; symmetric products need square ones to leave any out.  us, one matrix, never / so /
    // up to twice as many: 500 x 1,000 262 / 195 / 195, 1,000 x 1,000 341 / 264 / 264, 1,024 x 2,048 420 / 352 / 411, 1,500 x 1,500 466 / 466 / 710.
    const bool narrow = tiles_m * (cols / 64) * batch * a.jobs <= sms;
    a.symmetric = symmetric && !narrow && tiles_m > 1;
    // Tiles of 128 x 256 where they give every SM one (2,048 x 4,096, five steps: 1,340 us without them, 1,216 with).
    const bool wide = !narrow && !a.symmetric && cols % 256 == 0 && tiles_m * (cols / 256) * batch * a.jobs >= sms;
    a.tiles_n = (int32_t)(narrow ? cols / 64 : wide ? cols / 256 : cols / 128);
    if (wide) return launch_product_n<256>(a, tiles_m, batch, st);
    return narrow ? launch_product_n<64>(a, tiles_m, batch, st) : launch_product_n<128>(a, tiles_m, batch, st);
}

// Whether a matrix of out lies on one of G that is not its own: matrices are done side by side, so one may be written before another
// is read.  out may be G itself.
bool updates_meet(const void* G, int64_t ldg, int64_t g_stride, const void* out, int64_t ldo, int64_t o_stride, int64_t batch, int64_t rows,
                  int64_t cols, int64_t es) {
    if (G == out && (ldg == ldo || rows == 1) && (batch == 1 || g_stride == o_stride)) return false;
    const char *g = static_cast<const char*>(G), *o = static_cast<const char*>(out);
    if (batch == 1) return arrays_overlap(g, rows, cols, ldg, es, o, rows, cols, ldo, es);
    const int64_t span = (rows - 1) * std::max(ldg, ldo) + cols;
    if (!arrays_overlap(g, 1, (batch - 1) * g_stride + span, 1, es, o, 1, (batch - 1) * o_stride + span, 1, es)) return false;
    if (g_stride != o_stride) return true;
    for (int64_t k = 1 - batch; k < batch; ++k)  // matrices of one buffer, as many apart
        if (arrays_overlap(g, rows, cols, ldg, es, o + k * o_stride * es, rows, cols, ldo, es)) return true;
    return false;
}

int ns_launch(const void* G, int64_t rows, int64_t cols, int64_t ldg, int64_t g_stride, int64_t batch, int32_t dtype, int32_t steps,
              const float* coeffs, float eps, float scale, void* out, int64_t ldo, int64_t o_stride, void* workspace,
              int64_t workspace_bytes, int32_t* error_flag, void* stream, const NsSelfTest* test = nullptr) {
    if (!is_dtype(dtype) || rows < 1 || cols < 1 || rows > kMaxSide || cols > kMaxSide || batch < 0 || batch > 16384) return GNNPRE_ERR_INVALID_ARG;
    if (steps < 1 || steps > kMaxSteps || !coeffs || !(eps >= 0.f) || !std::isfinite(eps)) return GNNPRE_ERR_INVALID_ARG;
    Own own{};
    AllBounds& all = own.all;
    if (!bounds_of(coeffs, steps, &all)) return GNNPRE_ERR_INVALID_ARG;
    if (batch == 0) return GNNPRE_OK;
    if (!G || !out || !workspace || ldg < cols || ldo < cols) return GNNPRE_ERR_INVALID_ARG;
    if (batch > 1 && (g_stride < 0 || o_stride < (rows - 1) * ldo + cols)) return GNNPRE_ERR_INVALID_ARG;
    const int64_t es = dtype_bytes(dtype);
    if (reinterpret_cast<uintptr_t>(G) % es || reinterpret_cast<uintptr_t>(out) % es || reinterpret_cast<uintptr_t>(workspace) % 256)
        return GNNPRE_ERR_ALIGN;
    const NsShape s = ns_shape(batch, rows, cols, steps, most_segment_steps(dtype));
    if (workspace_bytes < s.total) return GNNPRE_ERR_INVALID_ARG;
    const int64_t span_g = (batch - 1) * g_stride + (rows - 1) * ldg + cols, span_o = (batch - 1) * o_stride + (rows - 1) * ldo + cols;
    if (arrays_overlap(workspace, 1, s.total, 1, 1, G, 1, span_g, 1, es) || arrays_overlap(workspace, 1, s.total, 1, 1, out, 1, span_o, 1, es))
        return GNNPRE_ERR_INVALID_ARG;
    if (updates_meet(G, ldg, g_stride, out, ldo, o_stride, batch, rows, cols, es)) return GNNPRE_ERR_INVALID_ARG;
    int sms = 0;
    GNNPRE_TRY(device_sms(&sms));
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    unsigned char* w = static_cast<unsigned char*>(workspace);
    const auto side = [&](int64_t at) { return Split{w + at, s.side, (int32_t)(s.np / 64)}; };
    const auto side_t = [&](int64_t at) { return Split{w + at, s.side, (int32_t)(s.rp / 64)}; };
    const auto square = [&](int64_t at) { return Split{w + at, s.square, (int32_t)(s.rp / 64)}; };

    int ex = exponent_for(all.x[0]);
    Source src{G, ldg, g_stride, (int32_t)rows, (int32_t)cols, dtype, rows > cols, (double)eps, reinterpret_cast<double*>(w + s.partial),
               (float)std::ldexp(1.0, ex), side(s.x), side_t(s.xt[0])};
    Steps factors{};
    factors.all = all;
    factors.scale = scale;
    if (s.ctas)
        for (int32_t k = 0; k < steps; ++k)
            factors.by_all[k] = step_factors(all.c, s.chip, scale, all.x[k], all.p[k], all.x[k + 1], &ex);
    if (s.chip) {
        const int64_t cols = ((s.n + s.ctas - 1) / s.ctas + 63) / 64 * 64;
        const Chip c{src, (int32_t)cols, steps, out, ldo, o_stride, error_flag, test ? test->polls : kTcSpinLimit, test ? test->drop : 0, factors};
        return launch_clusters(k_ns_chip, kChipThreads, kChipSmem, s.ctas, batch, st, c);
    }
    if (s.ctas) {
        Cluster c{};
        c.src = src;
        c.a = square(s.a);
        c.a2 = square(s.a2);
        c.p = square(s.p);
        c.xt[0] = side_t(s.xt[0]);
        c.xt[1] = side_t(s.xt[1]);
        c.rp = (int32_t)s.rp;
        c.np = (int32_t)s.np;
        c.k_r = (int32_t)((s.r + 63) / 64);
        c.k_n = (int32_t)((s.n + 63) / 64);
        c.steps = steps;
        c.out = out;
        c.ldo = ldo;
        c.out_batch = o_stride;
        c.error = error_flag;
        c.spin_limit = test ? test->polls : kTcSpinLimit;
        c.drop = test ? test->drop : 0;
        c.s = factors;
        return launch_clusters(k_ns_cluster, kProductThreads, kClusterSmem, s.ctas, batch, st, c);
    }
    own.steps = steps;
    own.segment = s.segment;
    own.by = reinterpret_cast<int32_t*>(w + s.by);
    const int norm_blocks = (int)std::min<int64_t>(kNormBlocks, rows);
    k_ns_norm<<<dim3((unsigned)norm_blocks, (unsigned)batch), kNormThreads, 0, st>>>(src);
    GNNPRE_CUDA(cudaGetLastError());
    GNNPRE_TRY(launch_after(k_ns_split, dim3((unsigned)(s.np / 64), (unsigned)(s.rp / 64), (unsigned)batch), 256, 0, true, st, src, norm_blocks, own));

    Product base{};
    base.error = error_flag;
    base.spin_limit = test ? test->polls : kTcSpinLimit;
    base.drop = test ? test->drop : 0;
    base.jobs = 1;
    base.by = own.by;
    const int32_t k_r = (int32_t)((s.r + 63) / 64), k_n = (int32_t)((s.n + 63) / 64);
    int xt = 0;
    for (int32_t k = 0; k < steps;) {
        const int32_t g = std::min(s.segment, steps - k);
        int ea = exponent_for(all.x[k] * all.x[k]), e2 = second_exponent(all.c, all.x[k]);
        // a new A from an accumulator that holds 2^acc of it
        const auto new_a = [&](Job& job, int32_t step, int acc) {
            job.d = square(s.a);
            job.of_d = slot(kOfA, step);
            job.of_d2 = slot(kOfA2, step);
            job.alpha = (float)std::ldexp(1.0, ea - acc);
            job.d2 = square(s.a2);
            job.alpha2 = (float)std::ldexp((double)coeffs[2], e2 - acc);
            job.diag2 = (float)std::ldexp((double)coeffs[1], e2);
            job.write_2 = 1;
        };
        const auto operands = [](const Split& x, int of_x, const Split& y, int of_y, int32_t chunks) {
            Job job{};
            job.a = x;
            job.b = y;
            job.of_a = of_x;
            job.of_b = of_y;
            job.k_chunks = chunks;
            return job;
        };
        Product m = base;
        m.job[0] = operands(side(s.x), slot(kOfX, k), side(s.x), slot(kOfX, k), k_n);
        new_a(m.job[0], k, 2 * ex);
        GNNPRE_TRY(launch_product(m, s.rp, s.rp, batch, true, sms, st));
        int eq = 0, q = 0;
        double q_bound = 1;
        for (int32_t j = 0; j < g; ++j) {
            // P = a I + A (c A + b I)
            const int ep = exponent_for(all.p[k + j]);
            const Split p = square(j == 0 ? s.q[0] : s.p);
            m = base;
            const int of_p = slot(kOfP, k + j);
            m.job[0] = operands(square(s.a), slot(kOfA, k + j), square(s.a2), slot(kOfA2, k + j), k_r);
            m.job[0].d = p;
            m.job[0].of_d = of_p;
            m.job[0].alpha = (float)std::ldexp(1.0, ep - ea - e2);
            m.job[0].diag = (float)std::ldexp((double)coeffs[0], ep);
            GNNPRE_TRY(launch_product(m, s.rp, s.rp, batch, true, sms, st));
            q_bound *= all.p[k + j];
            const int eq_new = j == 0 ? ep : exponent_for(q_bound);
            Job more = operands(square(s.q[q]), slot(kOfQ, k + j - 1), p, of_p, k_r);  // (from the second step on)
            more.d = square(s.q[q ^ 1]);
            more.of_d = slot(kOfQ, k + j);
            more.alpha = (float)std::ldexp(1.0, eq_new - eq - ep);
            m = base;
            if (j + 1 < g) {
                // T = A P, then the next A = T P beside Q = Q P
                const int et = exponent_for(all.x[k + j] * all.x[k + j] * all.p[k + j]);
                m.job[0] = operands(square(s.a), slot(kOfA, k + j), p, of_p, k_r);
                m.job[0].d = square(s.t);
                m.job[0].of_d = slot(kOfT, k + j);
                m.job[0].alpha = (float)std::ldexp(1.0, et - ea - ep);
                GNNPRE_TRY(launch_product(m, s.rp, s.rp, batch, true, sms, st));
                ea = exponent_for(all.x[k + j + 1] * all.x[k + j + 1]);
                e2 = second_exponent(all.c, all.x[k + j + 1]);
                m = base;
                m.job[0] = operands(square(s.t), slot(kOfT, k + j), p, of_p, k_r);
                new_a(m.job[0], k + j + 1, et + ep);
                if (j > 0) {
                    m.job[1] = more;
                    m.jobs = 2;
                }
                GNNPRE_TRY(launch_product(m, s.rp, s.rp, batch, true, sms, st));
            } else if (j > 0) {
                m.job[0] = more;
                GNNPRE_TRY(launch_product(m, s.rp, s.rp, batch, true, sms, st));
            }
            if (j > 0) q ^= 1;
            eq = eq_new;
        }
        const int of_q = slot(kOfQ, k + g - 1), of_x = slot(kOfX, k);
        k += g;
        m = base;
        if (k < steps) {
            const int ex_new = exponent_for(all.x[k]);
            m.job[0] = operands(square(s.q[q]), of_q, side_t(s.xt[xt]), of_x, k_r);
            m.job[0].d = side(s.x);
            m.job[0].of_d = slot(kOfX, k);
            m.job[0].dt = side_t(s.xt[xt ^ 1]);
            m.job[0].write_t = 1;
            m.job[0].alpha = (float)std::ldexp(1.0, ex_new - eq - ex);
            GNNPRE_TRY(launch_product(m, s.rp, s.np, batch, false, sms, st));
            ex = ex_new;
            xt ^= 1;
            continue;
        }
        m.out = out;
        m.ldo = ldo;
        m.out_batch = o_stride;
        m.out_dtype = dtype;
        m.out_rows = (int32_t)rows;
        m.out_cols = (int32_t)cols;
        m.out_factor = (float)std::ldexp((double)scale, -eq - ex);
        // Q is symmetric: the transpose of Q X is X^T Q
        const bool tall = rows > cols;
        m.job[0] = tall ? operands(side_t(s.xt[xt]), of_x, square(s.q[q]), of_q, k_r) : operands(square(s.q[q]), of_q, side_t(s.xt[xt]), of_x, k_r);
        GNNPRE_TRY(launch_product(m, tall ? s.np : s.rp, tall ? s.rp : s.np, batch, false, sms, st));
    }
    return GNNPRE_OK;
}

}  // namespace
}  // namespace gnnpre

using namespace gnnpre;

extern "C" int64_t gnnpre_orthogonalize_workspace(int64_t batch, int64_t rows, int64_t cols, int32_t steps) {
    if (rows < 1 || cols < 1 || rows > kMaxSide || cols > kMaxSide || batch < 0 || batch > 16384 || steps < 1 || steps > kMaxSteps) return GNNPRE_ERR_INVALID_ARG;
    if (batch == 0) return 0;
    int64_t total = 0;
    for (int32_t most = 1; most <= 3; ++most) total = std::max(total, ns_shape(batch, rows, cols, steps, most).total);
    return total;
}

extern "C" int gnnpre_orthogonalize(const void* G, int64_t rows, int64_t cols, int64_t ldg, int64_t g_stride, int64_t batch, int32_t dtype,
                                    int32_t steps, const float* coeffs, float eps, float scale, void* out, int64_t ldo, int64_t o_stride,
                                    void* workspace, int64_t workspace_bytes, int32_t* error_flag, void* stream) {
    return ns_launch(G, rows, cols, ldg, g_stride, batch, dtype, steps, coeffs, eps, scale, out, ldo, o_stride, workspace, workspace_bytes,
                     error_flag, stream);
}

// Failure-detection self-test: see include/gnnpre.h.
extern "C" int gnnpre_orthogonalize_selftest_wait_timeout(const float* G, int64_t rows, int64_t cols, float* out, void* workspace,
                                                          int64_t workspace_bytes, int32_t* error_flag, uint32_t polls, void* stream) {
    if (!error_flag || polls == 0 || polls > 100000u) return GNNPRE_ERR_INVALID_ARG;
    const float coeffs[3] = {1.5f, -0.5f, 0.f};
    const NsSelfTest test{1, polls};
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    GNNPRE_CUDA(cudaMemsetAsync(error_flag, 0, sizeof(int32_t), st));
    GNNPRE_TRY(ns_launch(G, rows, cols, cols, 0, 1, GNNPRE_F32, 1, coeffs, 1e-7f, 1.f, out, cols, 0, workspace, workspace_bytes, error_flag, stream, &test));
    GNNPRE_CUDA(cudaStreamSynchronize(st));
    int32_t flag = 0;
    GNNPRE_CUDA(cudaMemcpy(&flag, error_flag, sizeof(flag), cudaMemcpyDeviceToHost));
    return flag ? GNNPRE_ERR_TIMEOUT : GNNPRE_OK;
}
