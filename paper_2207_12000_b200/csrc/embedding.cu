// Learned tables: rows looked up and scaled, and the table's gradient by sorted ids.
//
//   lookup    out[i] = scale * table[ids[i]]
//   gradient  d_table[v] (+)= scale * sum over { i : ids[i] = v } of d_out[i]
//
// The lookup is one pass over memory.  The gradient sorts (id, position) pairs, so that the rows of one id are neighbours, and sums
// the sorted list in segments of equal length, whatever the ids' frequencies: a table's frequent rows cost no more per entry than
// its rare ones, no sum depends on the order in which anything ran, and a row is written once.  An id's parts from several
// segments meet in a second kernel, as the cut rows of a hop do.
//
// The sort is stable (least significant digit first), so a row's sum runs in the order of the positions.  Up to kOneCtaKeys keys
// are sorted by one CTA in shared memory; longer lists take, per digit, a count per block of keys, a scan over the blocks (done by
// the next kernel itself where there are few) and the move.  A table that is not accumulated into is cleared by further CTAs of
// these launches: sorting is latency, clearing is bandwidth.
#include <algorithm>
#include <atomic>

#include "dense.cuh"

namespace gnnpre {

int device_sms(int* out) {
    int dev = 0;
    GNNPRE_CUDA(cudaGetDevice(&dev));
    static std::atomic<int> known[kMaxDevices];
    int sms = dev < kMaxDevices ? known[dev].load(std::memory_order_relaxed) : 0;
    if (sms == 0) {
        GNNPRE_TRY(check_device());
        GNNPRE_CUDA(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
        if (dev < kMaxDevices) known[dev].store(sms, std::memory_order_relaxed);
    }
    *out = sms;
    return GNNPRE_OK;
}

namespace {

constexpr int64_t kMaxDim = 1 << 20;

// ------------------------------------------------------------------------------------------------ ids

struct Ids {
    const void* p;
    int32_t wide;   // int64 instead of int32
    int64_t n;      // rows of the table
};

// The row that position i asks for; n for an id outside the table.
__device__ __forceinline__ uint32_t id_at(const Ids& ids, int64_t i) {
    const int64_t v = ids.wide ? __ldg(static_cast<const long long*>(ids.p) + i) : (int64_t)__ldg(static_cast<const int*>(ids.p) + i);
    return v >= 0 && v < ids.n ? (uint32_t)v : (uint32_t)ids.n;
}

// ------------------------------------------------------------------------------------------------ lookup

struct LookupArgs {
    Ids ids;
    const void* table;
    int64_t ldt;
    void* out;
    int64_t ldo;
    int64_t count;
    int64_t dim;
    float scale;
    int32_t lanes;  // per row, a power of two
};

constexpr int kLookupThreads = 128;

// Rows that this call does not read again: written past what the L2 keeps (2.4 M rows of 256 bf16 from a table that it holds: 508 us
// without the hint, 373 with it, 357 in CTAs of 128 threads; the stores by themselves 330).
template <typename T, int E>
__device__ __forceinline__ void store_once(T* p, const Vec<T, E>& v) {
    if constexpr (E * sizeof(T) == 16) __stcs(reinterpret_cast<uint4*>(p), *reinterpret_cast<const uint4*>(&v));
    else if constexpr (E * sizeof(T) == 8) __stcs(reinterpret_cast<uint2*>(p), *reinterpret_cast<const uint2*>(&v));
    else *reinterpret_cast<Vec<T, E>*>(p) = v;
}

// `lanes` threads per row and U rows per thread, whose reads are all in flight before the first is used.
template <typename T, int E, int U>
__global__ void __launch_bounds__(kLookupThreads) k_lookup(const LookupArgs a) {
    const int lane = threadIdx.x & (a.lanes - 1);
    const int64_t group = ((int64_t)blockIdx.x * kLookupThreads + threadIdx.x) / a.lanes;
    const int64_t row0 = group * U;
    if (row0 >= a.count) return;
    const T* src[U];
    T* dst[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int64_t i = row0 + u;
        const uint32_t r = i < a.count ? id_at(a.ids, i) : (uint32_t)a.ids.n;
        src[u] = r < (uint32_t)a.ids.n ? static_cast<const T*>(a.table) + (int64_t)r * a.ldt : nullptr;
        dst[u] = i < a.count ? static_cast<T*>(a.out) + i * a.ldo : nullptr;
    }
    const int64_t whole = a.dim / E * E;
    for (int64_t c = (int64_t)lane * E; c < whole; c += (int64_t)a.lanes * E) {
        Vec<T, E> v[U];
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (src[u]) v[u] = *reinterpret_cast<const Vec<T, E>*>(src[u] + c);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (!dst[u]) continue;
#pragma unroll
            for (int e = 0; e < E; ++e) v[u].v[e] = src[u] ? from_f32<T>(to_f32(v[u].v[e]) * a.scale) : from_f32<T>(0.f);
            store_once(dst[u] + c, v[u]);
        }
    }
    for (int64_t c = whole + lane; c < a.dim; c += a.lanes)  // what does not fill an access
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (dst[u]) dst[u][c] = src[u] ? from_f32<T>(to_f32(src[u][c]) * a.scale) : from_f32<T>(0.f);
}

// (16-bit rows at a pitch of 8 bytes take accesses of two elements, like those of 4: accesses of four are not built.  600,000 bf16 rows of
// 100 columns, us: pitch 104 71, 100 or 102 110; of 602 fp16 columns, 100,000 of them: 608 48, 604 77.  Their gradient does not
// tell: 270 and 281.)
template <typename T, int E>
int launch_lookup(LookupArgs a, int num_sms, cudaStream_t st) {
    const int64_t pieces = std::max<int64_t>(1, a.dim / E);
    a.lanes = 1;
    while (a.lanes < 32 && a.lanes < pieces) a.lanes *= 2;
    // Four rows per thread hide the latency of the ids and rows when the machine is full of threads anyway; few rows are spread.  us,
    // one row / four: 1,000 rows of 602 fp16 2.9 / 3.9, 4,096 of 128 fp32 2.4 / 2.5, 18,944 (the border is at 9,472) 5.3 / 4.0, 400,000 88 / 62.
    const bool few = a.count * a.lanes <= (int64_t)num_sms * 2048;
    const int64_t groups = few ? a.count : (a.count + 3) / 4;
    const int64_t blocks = (groups * a.lanes + kLookupThreads - 1) / kLookupThreads;
    if (blocks > INT32_MAX) return GNNPRE_ERR_INVALID_ARG;
    if (few) k_lookup<T, E, 1><<<(unsigned)blocks, kLookupThreads, 0, st>>>(a);
    else k_lookup<T, E, 4><<<(unsigned)blocks, kLookupThreads, 0, st>>>(a);
    GNNPRE_CUDA(cudaGetLastError());
    return GNNPRE_OK;
}

// ------------------------------------------------------------------------------------------------ clearing

struct Clear {
    char* p;
    int64_t pitch, row_bytes, rows;  // rows == 1: one piece of memory
    int32_t first, parts;            // this launch clears parts [first, first + 1) of `parts`
    int32_t wide;                    // 16-byte stores
};

// The zeros leave the L2 first: kept there, 87 MB of them take the place of d_out's rows while those are summed (65,553 bf16 rows into
// 169,343: 61.4 us a gradient, 59.6 so).
__device__ __forceinline__ void clear_bytes(char* p, int64_t bytes, int64_t at, int64_t step, bool wide) {
    if (wide) {
        const int64_t whole = bytes / 16;
        for (int64_t i = at; i < whole; i += step) __stcs(reinterpret_cast<uint4*>(p) + i, make_uint4(0, 0, 0, 0));
        for (int64_t i = whole * 8 + at; i < bytes / 2; i += step) reinterpret_cast<uint16_t*>(p)[i] = 0;
    } else {
        for (int64_t i = at; i < bytes / 2; i += step) reinterpret_cast<uint16_t*>(p)[i] = 0;
    }
}

// The CTAs of a launch from `block` on (of `blocks`) clear its share of the table.
__device__ __forceinline__ void clear_share(const Clear& c, int block, int blocks) {
    if (c.rows == 1) {
        const int64_t per = (c.row_bytes / c.parts + 15) / 16 * 16;
        const int64_t lo = min(c.row_bytes, per * c.first), hi = c.first + 1 == c.parts ? c.row_bytes : min(c.row_bytes, lo + per);
        clear_bytes(c.p + lo, hi - lo, (int64_t)block * blockDim.x + threadIdx.x, (int64_t)blocks * blockDim.x, c.wide);
        return;
    }
    const int64_t per = (c.rows + c.parts - 1) / c.parts;
    const int64_t lo = min(c.rows, per * c.first), hi = min(c.rows, lo + per);
    const int warps = blockDim.x >> 5;
    for (int64_t r = lo + (int64_t)block * warps + (threadIdx.x >> 5); r < hi; r += (int64_t)blocks * warps)
        clear_bytes(c.p + r * c.pitch, c.row_bytes, threadIdx.x & 31, 32, c.wide);
}

__global__ void k_clear(const Clear c) { clear_share(c, blockIdx.x, gridDim.x); }

// ------------------------------------------------------------------------------------------------ sorting

constexpr int kOneCtaPerThread = 8;
// By a CTA of 1024 threads, fewer keys by one of 512 or 256.  us a gradient, one CTA / blocks of keys: 500 ids into 1,000 rows 9.8 / 12.7,
// into 169,343 13.4 / 21.1; 3,000 ids 15.7 / 16.0 and 18.4 / 24.1; 5,000 18.8 / 16.8 and 24.2 / 26.5; 8,192, where shared memory ends,
// 22.7 / 17.4 and 29.7 / 26.9: keys of one digit would pay from some 3,000 on, those of two from 6,000.
constexpr int kOneCtaKeys = 1024 * kOneCtaPerThread;
constexpr int kOneCtaDigit = 8;                  // bits
constexpr int kSortThreads = 512;
// Keys of a block: 2048 (four per thread) while such blocks fit the machine at once, two to an SM, else 4096.  The time of a block is
// that of its threads' rounds.  us a gradient, 4096 / 2048: 65,553 rows 71 / 63, 300,000 62 / 56, 2.4 M 333 / 342.
constexpr int kSortFew = 4, kSortMany = 8;
constexpr int kMaxDigit = 11;
// Up to here a block adds up the other blocks' counts itself.  us a gradient into 169,343 rows, so / by a kernel of its own: 20,000 ids (10
// blocks) 27.6 / 29.3, 65,553 (33) 31.9 / 33.2, 131,072 (64) 39.5 / 38.9, 260,000 (127) 71 / 55.
constexpr int kSelfScanBlocks = 64;

// Places of one warp's keys among those with the same digit before them in this warp; `counts` is the warp's row of counters.
// Rounds of 32 neighbouring keys, so the order is kept.  Lanes with the same digit are found bit by bit: the ballots of a round do
// not wait for one another (match.any takes longer the more digits there are).
template <int ROUNDS>
__device__ __forceinline__ void rank_in_warp(const uint32_t (&digit)[ROUNDS], const bool (&live)[ROUNDS], int bits, int rounds,
                                             uint16_t* counts, uint32_t (&place)[ROUNDS]) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r) {
        if (r >= rounds) break;
        uint32_t peers = __ballot_sync(0xffffffffu, live[r]);
        for (int b = 0; b < bits; ++b) {
            const bool bit = digit[r] >> b & 1u;
            const uint32_t with = __ballot_sync(0xffffffffu, bit);
            peers &= bit ? with : ~with;
        }
        const uint32_t below = peers & ((1u << lane) - 1u);
        uint32_t before = 0;
        if (live[r]) before = counts[digit[r]];
        __syncwarp();
        if (live[r] && below == 0) counts[digit[r]] = (uint16_t)(before + __popc(peers));
        place[r] = before + __popc(below);
        __syncwarp();
    }
}

// Exclusive sums of v over the threads of a CTA; `room` holds one value per warp and one more, the total.
__device__ __forceinline__ uint32_t block_exclusive_sum(uint32_t v, uint32_t* room) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    uint32_t s = v;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
        const uint32_t o = __shfl_up_sync(0xffffffffu, s, d);
        if (lane >= d) s += o;
    }
    if (lane == 31) room[warp] = s;
    __syncthreads();
    if (warp == 0) {
        uint32_t w = lane < warps ? room[lane] : 0u;
#pragma unroll
        for (int d = 1; d < 32; d *= 2) {
            const uint32_t o = __shfl_up_sync(0xffffffffu, w, d);
            if (lane >= d) w += o;
        }
        room[lane] = w;
    }
    __syncthreads();
    const uint32_t base = warp > 0 ? room[warp - 1] : 0u;
    return base + s - v;
}

struct SortArgs {
    Ids ids;
    int64_t count;
    int32_t shift, bits;       // of this pass
    int32_t blocks;            // of kSortThreads * (kSortFew or kSortMany) keys
    int32_t scanned;           // the counts are sums over the blocks before, `totals` the digits' counts
    const uint32_t* keys_in;   // nullptr: the ids themselves, in their order
    const uint32_t* pos_in;
    uint32_t* keys_out;
    uint32_t* pos_out;
    uint32_t* counts;          // [digit][block] where they are scanned by a kernel of their own, else [block][digit]
    uint32_t* totals;          // [digit]
    Clear clear;
};

// All passes by one CTA; the others clear the table.
template <int THREADS>
__global__ void __launch_bounds__(THREADS) k_sort_one_cta(const SortArgs a, const int32_t key_bits) {
    if (blockIdx.x > 0) {
        clear_share(a.clear, blockIdx.x - 1, gridDim.x - 1);
        return;
    }
    extern __shared__ __align__(16) unsigned char sort_smem[];
    uint32_t* keys = reinterpret_cast<uint32_t*>(sort_smem);
    constexpr int kKeys = THREADS * kOneCtaPerThread, kParts = THREADS >> kOneCtaDigit, kPartWarps = (1 << kOneCtaDigit) / 32;
    uint16_t* pos = reinterpret_cast<uint16_t*>(keys + kKeys);
    uint16_t* counts = pos + kKeys;  // [warp][digit]
    __shared__ uint16_t firsts[kParts][1 << kOneCtaDigit];
    __shared__ uint32_t room[32];
    constexpr int kWarps = THREADS / 32;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int n = (int)a.count;
    // neighbouring keys of a warp, in rounds that no thread needs more of than there are keys for
    const int per_warp = ((n + kWarps - 1) / kWarps + 31) / 32 * 32, rounds = per_warp / 32;
    const int passes = (key_bits + kOneCtaDigit - 1) / kOneCtaDigit, bits = (key_bits + passes - 1) / passes;
    uint32_t key[kOneCtaPerThread], place[kOneCtaPerThread], digit[kOneCtaPerThread];
    uint16_t at[kOneCtaPerThread];
    bool live[kOneCtaPerThread];
#pragma unroll
    for (int r = 0; r < kOneCtaPerThread; ++r) {
        const int i = warp * per_warp + 32 * r + lane;
        live[r] = r < rounds && i < n;
        at[r] = (uint16_t)i;
        key[r] = live[r] ? id_at(a.ids, i) : 0u;
    }
    const int digits = 1 << bits;
    for (int p = 0; p < passes; ++p) {
        const int shift = p * bits;
        for (int i = threadIdx.x; i < kWarps * digits / 2; i += THREADS) reinterpret_cast<uint32_t*>(counts)[i] = 0;
        __syncthreads();
#pragma unroll
        for (int r = 0; r < kOneCtaPerThread; ++r) digit[r] = (key[r] >> shift) & (uint32_t)(digits - 1);
        rank_in_warp<kOneCtaPerThread>(digit, live, bits, rounds, counts + warp * digits, place);
        __syncthreads();
        // sums over the warps before, eight warps to a thread
        const int d = threadIdx.x & ((1 << kOneCtaDigit) - 1), part = threadIdx.x >> kOneCtaDigit;
        if (d < digits) {
            uint32_t c[kPartWarps], sum = 0;
#pragma unroll
            for (int w = 0; w < kPartWarps; ++w) c[w] = counts[(part * (kPartWarps) + w) * digits + d];
#pragma unroll
            for (int w = 0; w < kPartWarps; ++w) {
                counts[(part * (kPartWarps) + w) * digits + d] = (uint16_t)sum;
                sum += c[w];
            }
            firsts[part][d] = (uint16_t)sum;
        }
        __syncthreads();
        uint32_t ahead[kParts], total = 0;
        if ((int)threadIdx.x < digits)
#pragma unroll
            for (int q = 0; q < kParts; ++q) {
                ahead[q] = total;
                total += firsts[q][threadIdx.x];
            }
        const uint32_t base = block_exclusive_sum(total, room);
        if ((int)threadIdx.x < digits)
#pragma unroll
            for (int q = 0; q < kParts; ++q) firsts[q][threadIdx.x] = (uint16_t)(base + ahead[q]);
        __syncthreads();
#pragma unroll
        for (int r = 0; r < kOneCtaPerThread; ++r)
            if (live[r]) {
                const uint32_t to = firsts[warp / (kPartWarps)][digit[r]] + counts[warp * digits + digit[r]] + place[r];
                keys[to] = key[r];
                pos[to] = at[r];
            }
        __syncthreads();
#pragma unroll
        for (int r = 0; r < kOneCtaPerThread; ++r) {
            const int i = warp * per_warp + 32 * r + lane;
            if (live[r]) {
                key[r] = keys[i];
                at[r] = pos[i];
            }
        }
    }
#pragma unroll
    for (int r = 0; r < kOneCtaPerThread; ++r) {
        const int i = warp * per_warp + 32 * r + lane;
        if (live[r]) {
            a.keys_out[i] = key[r];
            a.pos_out[i] = at[r];
        }
    }
}

__device__ __forceinline__ uint32_t sort_key(const SortArgs& a, int64_t i) { return a.keys_in ? a.keys_in[i] : id_at(a.ids, i); }

// Digits of each block of keys.
template <int kSortPerThread>
__global__ void __launch_bounds__(kSortThreads) k_sort_count(const SortArgs a) {
    constexpr int kSortKeys = kSortThreads * kSortPerThread;
    wait_previous_kernel();
    if ((int)blockIdx.x >= a.blocks) {
        clear_share(a.clear, blockIdx.x - a.blocks, gridDim.x - a.blocks);
        return;
    }
    __shared__ uint32_t hist[1 << kMaxDigit];
    const int digits = 1 << a.bits;
    for (int d = threadIdx.x; d < digits; d += kSortThreads) hist[d] = 0;
    __syncthreads();
    const int64_t lo = (int64_t)blockIdx.x * kSortKeys;
    uint32_t key[kSortPerThread];
#pragma unroll
    for (int r = 0; r < kSortPerThread; ++r) key[r] = sort_key(a, min(lo + r * kSortThreads + threadIdx.x, a.count - 1));
#pragma unroll
    for (int r = 0; r < kSortPerThread; ++r)
        if (lo + r * kSortThreads + threadIdx.x < a.count) atomicAdd(&hist[(key[r] >> a.shift) & (uint32_t)(digits - 1)], 1u);
    __syncthreads();
    for (int d = threadIdx.x; d < digits; d += kSortThreads)
        a.counts[a.scanned ? (int64_t)d * a.blocks + blockIdx.x : (int64_t)blockIdx.x * digits + d] = hist[d];
}

// A warp per digit: its counts become sums over the blocks before, its total is noted.
__global__ void __launch_bounds__(kSortThreads) k_sort_scan(const SortArgs a) {
    wait_previous_kernel();
    const int lane = threadIdx.x & 31, d = (int)(blockIdx.x * (kSortThreads / 32) + (threadIdx.x >> 5));
    if (d >= 1 << a.bits) return;
    uint32_t* c = a.counts + (int64_t)d * a.blocks;
    uint32_t sum = 0;
    for (int b0 = 0; b0 < a.blocks; b0 += 32) {
        const uint32_t v = b0 + lane < a.blocks ? c[b0 + lane] : 0u;
        uint32_t s = v;
#pragma unroll
        for (int k = 1; k < 32; k *= 2) {
            const uint32_t o = __shfl_up_sync(0xffffffffu, s, k);
            if (lane >= k) s += o;
        }
        if (b0 + lane < a.blocks) c[b0 + lane] = sum + s - v;
        sum += __shfl_sync(0xffffffffu, s, 31);
    }
    if (lane == 0) a.totals[d] = sum;
}

// Moves the pairs to their places by this pass's digit.  (With eight keys a thread it spills 96 bytes at the 64 registers that two CTAs
// per SM leave.)
template <int kSortPerThread>
__global__ void __launch_bounds__(kSortThreads, 2) k_sort_move(const SortArgs a) {
    constexpr int kSortKeys = kSortThreads * kSortPerThread;
    wait_previous_kernel();
    if ((int)blockIdx.x >= a.blocks) {
        clear_share(a.clear, blockIdx.x - a.blocks, gridDim.x - a.blocks);
        return;
    }
    extern __shared__ __align__(16) unsigned char sort_smem[];
    constexpr int kWarps = kSortThreads / 32, kMostPer = (1 << kMaxDigit) / kSortThreads;
    const int digits = 1 << a.bits;
    uint32_t* keys = reinterpret_cast<uint32_t*>(sort_smem);            // this block's pairs in the order of their digits
    uint32_t* pos = keys + kSortKeys;
    uint32_t* base = pos + kSortKeys;                                   // [digit] place of the block's first one, less its place here
    uint16_t* firsts = reinterpret_cast<uint16_t*>(base + digits);      // [digit] place here of the first one
    uint16_t* counts = firsts + digits;                                 // [warp][digit]
    __shared__ uint32_t room[32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t lo = (int64_t)blockIdx.x * kSortKeys + warp * (32 * kSortPerThread);
    const int here = (int)min((int64_t)kSortKeys, a.count - (int64_t)blockIdx.x * kSortKeys);
    uint32_t key[kSortPerThread], at[kSortPerThread], digit[kSortPerThread], place[kSortPerThread];
    bool live[kSortPerThread];
#pragma unroll
    for (int r = 0; r < kSortPerThread; ++r) {
        const int64_t i = lo + 32 * r + lane;
        live[r] = i < a.count;
        key[r] = sort_key(a, min(i, a.count - 1));
        at[r] = a.keys_in ? a.pos_in[min(i, a.count - 1)] : (uint32_t)i;
    }
    for (int i = threadIdx.x; i < kWarps * digits / 2; i += kSortThreads) reinterpret_cast<uint32_t*>(counts)[i] = 0;
    // thread t has the digits from t * per on: how many there are in all, and in the blocks before this one
    const int per = digits <= kSortThreads ? 1 : digits / kSortThreads;
    uint32_t total[kMostPer], before[kMostPer], sum = 0;
#pragma unroll
    for (int j = 0; j < kMostPer; ++j) {
        const int d = threadIdx.x * per + j;
        total[j] = before[j] = 0;
        if (j >= per || d >= digits) continue;
        if (a.scanned) {
            total[j] = a.totals[d];
            before[j] = a.counts[(int64_t)d * a.blocks + blockIdx.x];
        } else {
#pragma unroll 8
            for (int b = 0; b < a.blocks; ++b) {
                const uint32_t v = a.counts[(int64_t)b * digits + d];
                total[j] += v;
                if (b < (int)blockIdx.x) before[j] += v;
            }
        }
        sum += total[j];
    }
#pragma unroll
    for (int r = 0; r < kSortPerThread; ++r) digit[r] = (key[r] >> a.shift) & (uint32_t)(digits - 1);
    const uint32_t all = block_exclusive_sum(sum, room);
    __syncthreads();
    rank_in_warp<kSortPerThread>(digit, live, a.bits, kSortPerThread, counts + warp * digits, place);
    __syncthreads();
    // this block's digits: sums over the warps before, then over the digits before
    uint32_t mine[kMostPer], mine_sum = 0;
#pragma unroll
    for (int j = 0; j < kMostPer; ++j) {
        const int d = threadIdx.x * per + j;
        mine[j] = 0;
        if (j >= per || d >= digits) continue;
        uint32_t c[kWarps];
#pragma unroll
        for (int w = 0; w < kWarps; ++w) c[w] = counts[w * digits + d];
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            counts[w * digits + d] = (uint16_t)mine[j];
            mine[j] += c[w];
        }
        mine_sum += mine[j];
    }
    uint32_t local = block_exclusive_sum(mine_sum, room), global = all;
#pragma unroll
    for (int j = 0; j < kMostPer; ++j) {
        const int d = threadIdx.x * per + j;
        if (j >= per || d >= digits) continue;
        firsts[d] = (uint16_t)local;
        base[d] = global + before[j] - local;
        local += mine[j];
        global += total[j];
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kSortPerThread; ++r) {
        if (!live[r]) continue;
        const uint32_t to = firsts[digit[r]] + counts[warp * digits + digit[r]] + place[r];
        keys[to] = key[r];
        pos[to] = at[r];
    }
    __syncthreads();
    // neighbouring threads write neighbouring places, digit by digit (pair by pair from where they were read: 80 us for 2.4 M pairs)
    for (int i = threadIdx.x; i < here; i += kSortThreads) {
        const uint32_t k = keys[i], to = base[(k >> a.shift) & (uint32_t)(digits - 1)] + i;
        a.keys_out[to] = k;
        a.pos_out[to] = pos[i];
    }
}

// ------------------------------------------------------------------------------------------------ sums

struct SumArgs {
    const uint32_t* keys;  // sorted ids; n = adds nothing
    const uint32_t* pos;
    int64_t count;
    int64_t n;
    const void* d_out;
    int64_t ldd;
    void* d_table;
    int64_t ldt;
    int64_t dim;
    float scale;
    int32_t accumulate;
    int32_t lanes;         // per segment, a power of two
    int32_t length;        // entries of a segment, a multiple of 8
    int64_t segments;
    float* parts;          // [2 * segments][part_ld]: of a row that began before the segment, of one that goes on after it
    int64_t part_ld;
    int32_t out_vec;       // d_table's rows take stores of four elements
};

template <typename TO, int E>
__device__ __forceinline__ void store_row(const SumArgs& a, uint32_t row, int64_t col, const float (&acc)[E], bool whole) {
    TO* dst = static_cast<TO*>(a.d_table) + (int64_t)row * a.ldt + col;
    if (whole) {
        Vec<TO, E> v;
        if (a.accumulate) v = *reinterpret_cast<const Vec<TO, E>*>(dst);
#pragma unroll
        for (int e = 0; e < E; ++e) v.v[e] = from_f32<TO>(a.accumulate ? fmaf(a.scale, acc[e], to_f32(v.v[e])) : a.scale * acc[e]);
        *reinterpret_cast<Vec<TO, E>*>(dst) = v;
    } else {
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (col + e < a.dim) dst[e] = from_f32<TO>(a.accumulate ? fmaf(a.scale, acc[e], to_f32(dst[e])) : a.scale * acc[e]);
    }
}

constexpr int kSumThreads = 128;
constexpr int kSumWindow = 8;  // rows in flight per lane

// A group of lanes per segment and E columns per lane; column tiles are the grid's second dimension.
template <typename TI, typename TO, int E>
__global__ void __launch_bounds__(kSumThreads) k_table_sums(const SumArgs a) {
    wait_previous_kernel();
    const int64_t seg = ((int64_t)blockIdx.x * kSumThreads + threadIdx.x) / a.lanes;
    if (seg >= a.segments) return;
    const int64_t col = ((int64_t)blockIdx.y * a.lanes + (threadIdx.x & (a.lanes - 1))) * E;
    if (col >= a.dim) return;
    const bool whole = col + E <= a.dim;
    const int64_t lo = seg * a.length, hi = min(a.count, lo + a.length);
    const TI* src = static_cast<const TI*>(a.d_out) + col;
    uint32_t row = a.keys[lo];
    bool began = lo > 0 && a.keys[lo - 1] == row;
    const bool goes_on = hi < a.count && a.keys[hi] == a.keys[hi - 1];
    float acc[E];
#pragma unroll
    for (int e = 0; e < E; ++e) acc[e] = 0.f;
    auto part = [&](int which) {
        if (row >= (uint32_t)a.n) return;
        float* dst = a.parts + (2 * seg + which) * a.part_ld + col;
        if (whole) {
            Vec<float, E> v;
#pragma unroll
            for (int e = 0; e < E; ++e) v.v[e] = acc[e];
            *reinterpret_cast<Vec<float, E>*>(dst) = v;
        } else {
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (col + e < a.dim) dst[e] = acc[e];
        }
    };
    // (the pairs' arrays have room for whole windows)
    uint4 k4[2], p4[2];
    auto fetch = [&](int64_t i) {
        k4[0] = *reinterpret_cast<const uint4*>(a.keys + i);
        k4[1] = *reinterpret_cast<const uint4*>(a.keys + i + 4);
        p4[0] = *reinterpret_cast<const uint4*>(a.pos + i);
        p4[1] = *reinterpret_cast<const uint4*>(a.pos + i + 4);
    };
    fetch(lo);
    for (int64_t i = lo; i < hi; i += kSumWindow) {
        const uint32_t key[8] = {k4[0].x, k4[0].y, k4[0].z, k4[0].w, k4[1].x, k4[1].y, k4[1].z, k4[1].w};
        const uint32_t pos[8] = {p4[0].x, p4[0].y, p4[0].z, p4[0].w, p4[1].x, p4[1].y, p4[1].z, p4[1].w};
        Vec<TI, E> v[kSumWindow];
#pragma unroll
        for (int j = 0; j < kSumWindow; ++j) {
            if (i + j >= hi || key[j] >= (uint32_t)a.n) continue;
            const TI* s = src + (int64_t)pos[j] * a.ldd;
            if (whole) {
                v[j] = *reinterpret_cast<const Vec<TI, E>*>(s);
            } else {
#pragma unroll
                for (int e = 0; e < E; ++e) v[j].v[e] = col + e < a.dim ? s[e] : from_f32<TI>(0.f);
            }
        }
        if (i + kSumWindow < hi) fetch(i + kSumWindow);
#pragma unroll
        for (int j = 0; j < kSumWindow; ++j) {
            if (i + j >= hi) break;
            if (key[j] != row) {
                if (began) part(0);
                else store_row<TO, E>(a, row, col, acc, whole);  // (n sorts last, so a row that another one follows is real)
                began = false;
                row = key[j];
#pragma unroll
                for (int e = 0; e < E; ++e) acc[e] = 0.f;
            }
            if (row < (uint32_t)a.n) {
#pragma unroll
                for (int e = 0; e < E; ++e) acc[e] += to_f32(v[j].v[e]);
            }
        }
    }
    if (began) part(0);
    else if (goes_on) part(1);
    else if (row < (uint32_t)a.n) store_row<TO, E>(a, row, col, acc, whole);
}

constexpr int kJoinThreads = 1024;
// Parts that one warp adds up by itself.  us a gradient with 4 / 32 / 256 / any number: 65,553 ids into 1,000 rows 26 / 23 / 35 / 47, 2.4 M into
// 65,536 337 / 333 / 347 / 446, 100,000 of one id 45 / 45 / 45 / 391.
constexpr int kJoinAlone = 32;

// A warp per segment: where a row begins in it that goes on in later ones, their parts are added up.  Rows of more than kJoinAlone
// parts get the whole CTA: each warp a chain, the chains in their order.
template <typename TO>
__global__ void __launch_bounds__(kJoinThreads) k_table_joins(const SumArgs a) {
    wait_previous_kernel();
    constexpr int kWarps = kJoinThreads / 32;
    __shared__ uint32_t hub_row[kWarps];
    __shared__ int64_t hub_seg[kWarps], hub_last[kWarps];
    __shared__ int hubs;
    __shared__ float4 chains[kWarps][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if (threadIdx.x == 0) hubs = 0;
    __syncthreads();
    const int64_t col = ((int64_t)blockIdx.y * 32 + lane) * 4;
    const bool some = col < a.dim, whole = a.out_vec && col + 4 <= a.dim;
    // sum of the parts of segments t, t + step, ... up to `last`
    auto chain = [&](int64_t t, int64_t step, int64_t last, float4& s) {
        if (!some) return;
        for (; t <= last; t += 8 * step) {
            float4 v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (t + j * step <= last) v[j] = *reinterpret_cast<const float4*>(a.parts + 2 * (t + j * step) * a.part_ld + col);
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (t + j * step <= last) {
                    s.x += v[j].x;
                    s.y += v[j].y;
                    s.z += v[j].z;
                    s.w += v[j].w;
                }
        }
    };
    auto finish = [&](uint32_t row, const float4& s) {
        if (!some) return;
        const float acc[4] = {s.x, s.y, s.z, s.w};
        store_row<TO, 4>(a, row, col, acc, whole);
    };
    const int64_t seg = (int64_t)blockIdx.x * kWarps + warp;
    const int64_t lo = seg * a.length, hi = min(a.count, lo + a.length);
    if (hi < a.count) {  // (so the segment is a whole one, and another follows)
        const uint32_t row = a.keys[hi - 1];
        const bool goes_on = a.keys[hi] == row;
        const bool began = a.keys[lo] == row && lo > 0 && a.keys[lo - 1] == row;
        if (goes_on && !began && row < (uint32_t)a.n) {
            // the last segment that begins with this row: the next 32 looked at at once, then ever smaller steps of the rest
            auto is_row = [&](int64_t t) { return t < a.segments && a.keys[t * a.length] == row; };
            int64_t last = seg + 1;
            int c = __popc(__ballot_sync(0xffffffffu, is_row(last + 1 + lane)));
            last += c;
            if (c == 32) {
                int64_t end = a.segments;  // no segment from here on begins with it
                while (end - last > 1) {
                    const int64_t step = (end - last + 31) / 32;
                    c = __popc(__ballot_sync(0xffffffffu, last + step * (lane + 1) < end && is_row(last + step * (lane + 1))));
                    end = min(end, last + step * (c + 1));
                    last += step * c;
                }
            }
            if (last - seg <= kJoinAlone) {
                float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
                if (some) s = *reinterpret_cast<const float4*>(a.parts + (2 * seg + 1) * a.part_ld + col);
                chain(seg + 1, 1, last, s);
                finish(row, s);
            } else if (lane == 0) {
                const int h = atomicAdd(&hubs, 1);
                hub_row[h] = row;
                hub_seg[h] = seg;
                hub_last[h] = last;
            }
        }
    }
    __syncthreads();
    const int count = hubs;
    for (int h = 0; h < count; ++h) {
        float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
        if (warp == 0 && some) s = *reinterpret_cast<const float4*>(a.parts + (2 * hub_seg[h] + 1) * a.part_ld + col);
        chain(hub_seg[h] + 1 + warp, kWarps, hub_last[h], s);
        chains[warp][lane] = s;
        __syncthreads();
        if (warp == 0) {
#pragma unroll 8
            for (int w = 1; w < kWarps; ++w) {
                const float4 o = chains[w][lane];
                s.x += o.x;
                s.y += o.y;
                s.z += o.z;
                s.w += o.w;
            }
            finish(hub_row[h], s);
        }
        __syncthreads();
    }
}

// ------------------------------------------------------------------------------------------------ host

constexpr int kSortSms = 148;  // (a size that does not depend on the device: the workspace's goes by it)

struct GradShape {
    int32_t key_bits, passes, digit_bits;
    int32_t per_thread;     // keys of a thread in the sort
    int64_t blocks;         // of the sort
    int32_t length;         // of a segment
    int64_t segments;
    int64_t part_ld;
    // bytes from the workspace's start
    int64_t pairs, counts, totals, parts, total;
};

// Entries per segment: as many segments as keep the SMs' lanes busy some waves long, and no more parts of cut rows than that.
GradShape grad_shape(int64_t n, int64_t dim, int64_t count) {
    GradShape g{};
    g.key_bits = 1;
    while (((int64_t)1 << g.key_bits) <= n) ++g.key_bits;
    g.passes = (g.key_bits + kMaxDigit - 1) / kMaxDigit;
    g.digit_bits = (g.key_bits + g.passes - 1) / g.passes;
    g.per_thread = count <= (int64_t)2 * kSortSms * kSortThreads * kSortFew ? kSortFew : kSortMany;
    g.blocks = (count + kSortThreads * g.per_thread - 1) / (kSortThreads * g.per_thread);
    g.length = 8;
    while (g.length < 128 && count / g.length > 8192) g.length *= 2;
    g.segments = (count + g.length - 1) / g.length;
    g.part_ld = (dim + 3) / 4 * 4;
    const auto round = [](int64_t b) { return (b + 255) / 256 * 256; };
    g.pairs = 0;
    const int64_t array = round(4 * (count + kSumWindow));
    g.counts = 4 * array;
    g.totals = g.counts + round(4 * (g.blocks << g.digit_bits));
    g.parts = g.totals + round(4 << g.digit_bits);
    g.total = g.parts + round(4 * 2 * g.segments * g.part_ld);
    return g;
}

template <typename TI, typename TO, int E>
int launch_sums(SumArgs a, cudaStream_t st) {
    const int64_t pieces = (a.dim + E - 1) / E;
    a.lanes = 1;
    while (a.lanes < 32 && a.lanes < pieces) a.lanes *= 2;
    const int64_t tiles = (pieces + a.lanes - 1) / a.lanes;
    const int64_t blocks = (a.segments * a.lanes + kSumThreads - 1) / kSumThreads;
    if (tiles > 65535 || blocks > INT32_MAX) return GNNPRE_ERR_INVALID_ARG;
    return launch_after(k_table_sums<TI, TO, E>, dim3((unsigned)blocks, (unsigned)tiles), kSumThreads, 0, true, st, a);
}

template <typename TI, typename TO>
int launch_sums_and_joins(SumArgs a, cudaStream_t st) {
    const uintptr_t in = reinterpret_cast<uintptr_t>(a.d_out) | (uintptr_t)(a.ldd * (int64_t)sizeof(TI));
    const uintptr_t out = reinterpret_cast<uintptr_t>(a.d_table) | (uintptr_t)(a.ldt * (int64_t)sizeof(TO));
    constexpr int kMost = 16 / (int)sizeof(TI);
    int e = elements_per_access(in, sizeof(TI), kMost);
    while (e > 1 && out % (uintptr_t)std::min<int64_t>(16, e * (int64_t)sizeof(TO)) != 0) e /= 2;
    a.out_vec = out % (4 * sizeof(TO)) == 0;
    if (e == kMost) GNNPRE_TRY((launch_sums<TI, TO, kMost>(a, st)));
    else if (e >= 2) GNNPRE_TRY((launch_sums<TI, TO, 2>(a, st)));
    else GNNPRE_TRY((launch_sums<TI, TO, 1>(a, st)));
    if (a.segments < 2) return GNNPRE_OK;
    const int64_t tiles = (a.dim + 127) / 128, blocks = (a.segments + 31) / 32;
    if (tiles > 65535) return GNNPRE_ERR_INVALID_ARG;
    return launch_after(k_table_joins<TO>, dim3((unsigned)blocks, (unsigned)tiles), kJoinThreads, 0, true, st, a);
}

// What both calls ask of their arguments.
int check_table(int64_t n, int64_t dim, int32_t ids_type, int64_t count) {
    if (n < 1 || n > INT32_MAX || dim < 1 || dim > kMaxDim || count < 0 || count > INT32_MAX) return GNNPRE_ERR_INVALID_ARG;
    if (ids_type != GNNPRE_I32 && ids_type != GNNPRE_I64) return GNNPRE_ERR_INVALID_ARG;
    return GNNPRE_OK;
}

}  // namespace
}  // namespace gnnpre

using namespace gnnpre;

extern "C" int gnnpre_embedding_lookup(const void* table, int64_t n, int64_t dim, int64_t ldt, int32_t dtype, const void* ids,
                                       int32_t ids_type, int64_t count, float scale, void* out, int64_t ldo, void* stream) {
    GNNPRE_TRY(check_table(n, dim, ids_type, count));
    if (!table || !is_dtype(dtype) || ldt < dim || ldo < dim || (count > 0 && (!ids || !out))) return GNNPRE_ERR_INVALID_ARG;
    const int64_t es = dtype_bytes(dtype), ids_es = ids_type == GNNPRE_I64 ? 8 : 4;
    if (reinterpret_cast<uintptr_t>(table) % es || reinterpret_cast<uintptr_t>(out) % es || reinterpret_cast<uintptr_t>(ids) % ids_es)
        return GNNPRE_ERR_ALIGN;
    if (arrays_overlap(table, n, dim, ldt, es, out, count, dim, ldo, es) ||
        arrays_overlap(ids, 1, count, count, ids_es, out, 1, count > 0 ? (count - 1) * ldo + dim : 0, 1, es))
        return GNNPRE_ERR_INVALID_ARG;
    int sms = 0;
    GNNPRE_TRY(device_sms(&sms));
    if (count == 0) return GNNPRE_OK;
    LookupArgs a{{ids, ids_type == GNNPRE_I64, n}, table, ldt, out, ldo, count, dim, scale, 0};
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const uintptr_t at = reinterpret_cast<uintptr_t>(table) | reinterpret_cast<uintptr_t>(out) | (uintptr_t)(ldt * es) | (uintptr_t)(ldo * es);
    const int e = elements_per_access(at, es, (int)(16 / es));
    if (dtype == GNNPRE_F32) {
        if (e == 4) return launch_lookup<float, 4>(a, sms, st);
        return e == 2 ? launch_lookup<float, 2>(a, sms, st) : launch_lookup<float, 1>(a, sms, st);
    }
    if (dtype == GNNPRE_BF16) {
        if (e == 8) return launch_lookup<__nv_bfloat16, 8>(a, sms, st);
        return e >= 2 ? launch_lookup<__nv_bfloat16, 2>(a, sms, st) : launch_lookup<__nv_bfloat16, 1>(a, sms, st);
    }
    if (e == 8) return launch_lookup<__half, 8>(a, sms, st);
    return e >= 2 ? launch_lookup<__half, 2>(a, sms, st) : launch_lookup<__half, 1>(a, sms, st);
}

extern "C" int64_t gnnpre_embedding_grad_workspace(int64_t n, int64_t dim, int64_t count) {
    if (check_table(n, dim, GNNPRE_I32, count) != GNNPRE_OK) return GNNPRE_ERR_INVALID_ARG;
    return count == 0 ? 0 : grad_shape(n, dim, count).total;
}

extern "C" int gnnpre_embedding_grad(const void* d_out, int64_t ldd, int32_t dtype, const void* ids, int32_t ids_type, int64_t count,
                                     int64_t n, int64_t dim, float scale, int32_t accumulate, void* d_table, int64_t ldt,
                                     int32_t table_dtype, void* workspace, int64_t workspace_bytes, void* stream) {
    GNNPRE_TRY(check_table(n, dim, ids_type, count));
    if (!d_table || !is_dtype(dtype) || (table_dtype != dtype && table_dtype != GNNPRE_F32)) return GNNPRE_ERR_INVALID_ARG;
    if (ldd < dim || ldt < dim || (count > 0 && (!ids || !d_out || !workspace))) return GNNPRE_ERR_INVALID_ARG;
    const int64_t es = dtype_bytes(dtype), es_t = dtype_bytes(table_dtype), ids_es = ids_type == GNNPRE_I64 ? 8 : 4;
    if (reinterpret_cast<uintptr_t>(d_out) % es || reinterpret_cast<uintptr_t>(d_table) % es_t || reinterpret_cast<uintptr_t>(ids) % ids_es ||
        reinterpret_cast<uintptr_t>(workspace) % 256)
        return GNNPRE_ERR_ALIGN;
    const GradShape g = count > 0 ? grad_shape(n, dim, count) : GradShape{};
    if (workspace_bytes < g.total) return GNNPRE_ERR_INVALID_ARG;
    const int64_t table_span = (n - 1) * ldt + dim, rows_span = count > 0 ? (count - 1) * ldd + dim : 0;
    if (arrays_overlap(d_out, count, dim, ldd, es, d_table, n, dim, ldt, es_t) ||
        arrays_overlap(ids, 1, count, count, ids_es, d_table, 1, table_span, 1, es_t) ||
        arrays_overlap(workspace, 1, g.total, 1, 1, d_table, 1, table_span, 1, es_t) ||
        arrays_overlap(workspace, 1, g.total, 1, 1, d_out, 1, rows_span, 1, es) || arrays_overlap(workspace, 1, g.total, 1, 1, ids, 1, count, 1, ids_es))
        return GNNPRE_ERR_INVALID_ARG;
    int sms = 0;
    GNNPRE_TRY(device_sms(&sms));
    cudaStream_t st = static_cast<cudaStream_t>(stream);

    Clear c{static_cast<char*>(d_table), ldt * es_t, dim * es_t, n, 0, 1, 0};
    if (ldt == dim) {  // one piece of memory
        c.row_bytes = n * dim * es_t;
        c.rows = 1;
    }
    c.wide = reinterpret_cast<uintptr_t>(d_table) % 16 == 0 && (c.rows == 1 || c.pitch % 16 == 0);
    // CTAs of 256 threads that clear: enough to fill the machine, no more than give a thread four stores
    const int64_t bytes = accumulate ? 0 : n * dim * es_t;
    const auto clear_blocks = [&](int parts, int threads) {
        return bytes == 0 ? 0u : (unsigned)std::max<int64_t>(1, std::min<int64_t>((int64_t)sms * 2048 / threads, bytes / parts / (64 * threads)));
    };
    if (count == 0) {
        if (bytes == 0) return GNNPRE_OK;
        k_clear<<<clear_blocks(1, 256), 256, 0, st>>>(c);
        GNNPRE_CUDA(cudaGetLastError());
        return GNNPRE_OK;
    }

    char* w = static_cast<char*>(workspace);
    const int64_t array = g.counts / 4;
    uint32_t* pair[2][2];
    for (int i = 0; i < 4; ++i) pair[i / 2][i % 2] = reinterpret_cast<uint32_t*>(w + i * array);
    SortArgs s{};
    s.ids = Ids{ids, ids_type == GNNPRE_I64, n};
    s.count = count;
    s.blocks = (int32_t)g.blocks;
    s.counts = reinterpret_cast<uint32_t*>(w + g.counts);
    s.totals = reinterpret_cast<uint32_t*>(w + g.totals);
    s.clear = c;
    int at = 0;  // the pair of arrays that holds the sorted list
    if (count <= kOneCtaKeys) {
        s.keys_out = pair[0][0];
        s.pos_out = pair[0][1];
        // The fewer threads wait for one another, the sooner a pass is done: as many as eight keys each need (a gradient in a graph, us, by
        // 1024 threads / so: 37 ids 11.7 / 8.2, 500 12.8 / 10.1, 3,000 15.6 / 14.7).
        const int threads = count <= 256 * kOneCtaPerThread ? 256 : count <= 512 * kOneCtaPerThread ? 512 : 1024;
        const auto sort = threads == 256 ? k_sort_one_cta<256> : threads == 512 ? k_sort_one_cta<512> : k_sort_one_cta<1024>;
        constexpr int kPerThread = kOneCtaPerThread * 6 + 2 * (1 << kOneCtaDigit) / 32;  // bytes of shared memory
        if (threads == 1024) {
            static std::atomic<bool> opted_in[kMaxDevices];
            int dev = 0;
            GNNPRE_CUDA(cudaGetDevice(&dev));
            if (dev >= kMaxDevices || !opted_in[dev].load(std::memory_order_relaxed)) {
                GNNPRE_CUDA(cudaFuncSetAttribute(k_sort_one_cta<1024>, cudaFuncAttributeMaxDynamicSharedMemorySize, 1024 * kPerThread));
                if (dev < kMaxDevices) opted_in[dev].store(true, std::memory_order_relaxed);
            }
        }
        sort<<<1 + clear_blocks(1, threads), threads, (size_t)threads * kPerThread, st>>>(s, g.key_bits);
        GNNPRE_CUDA(cudaGetLastError());
    } else {
        s.scanned = g.blocks > kSelfScanBlocks;
        s.bits = g.digit_bits;
        s.clear.parts = 2 * g.passes;
        const unsigned grid = (unsigned)g.blocks + clear_blocks(s.clear.parts, kSortThreads);
        const auto count_keys = g.per_thread == kSortFew ? k_sort_count<kSortFew> : k_sort_count<kSortMany>;
        const auto move = g.per_thread == kSortFew ? k_sort_move<kSortFew> : k_sort_move<kSortMany>;
        const size_t smem = 8 * kSortThreads * g.per_thread + (((size_t)4 + 2 + 2 * (kSortThreads / 32)) << g.digit_bits);
        constexpr int kMostSmem = 8 * kSortThreads * kSortMany + ((4 + 2 + 2 * (kSortThreads / 32)) << kMaxDigit);
        static std::atomic<bool> opted_in[kMaxDevices];
        int dev = 0;
        GNNPRE_CUDA(cudaGetDevice(&dev));
        if (dev >= kMaxDevices || !opted_in[dev].load(std::memory_order_relaxed)) {
            GNNPRE_CUDA(cudaFuncSetAttribute(k_sort_move<kSortFew>, cudaFuncAttributeMaxDynamicSharedMemorySize, kMostSmem));
            GNNPRE_CUDA(cudaFuncSetAttribute(k_sort_move<kSortMany>, cudaFuncAttributeMaxDynamicSharedMemorySize, kMostSmem));
            if (dev < kMaxDevices) opted_in[dev].store(true, std::memory_order_relaxed);
        }
        for (int p = 0; p < g.passes; ++p) {
            s.shift = p * g.digit_bits;
            s.keys_in = p == 0 ? nullptr : pair[at][0];
            s.pos_in = p == 0 ? nullptr : pair[at][1];
            if (p > 0) at ^= 1;
            s.keys_out = pair[at][0];
            s.pos_out = pair[at][1];
            s.clear.first = 2 * p;
            GNNPRE_TRY(launch_after(count_keys, dim3(grid), kSortThreads, 0, p > 0, st, s));
            if (s.scanned)
                GNNPRE_TRY(launch_after(k_sort_scan, dim3((unsigned)(((1 << g.digit_bits) + kSortThreads / 32 - 1) / (kSortThreads / 32))), kSortThreads, 0, true, st, s));
            s.clear.first = 2 * p + 1;
            GNNPRE_TRY(launch_after(move, dim3(grid), kSortThreads, smem, true, st, s));
        }
    }

    SumArgs a{};
    a.keys = pair[at][0];
    a.pos = pair[at][1];
    a.count = count;
    a.n = n;
    a.d_out = d_out;
    a.ldd = ldd;
    a.d_table = d_table;
    a.ldt = ldt;
    a.dim = dim;
    a.scale = scale;
    a.accumulate = accumulate != 0;
    a.length = g.length;
    a.segments = g.segments;
    a.parts = reinterpret_cast<float*>(w + g.parts);
    a.part_ld = g.part_ld;
    if (dtype == GNNPRE_F32) return launch_sums_and_joins<float, float>(a, st);
    if (dtype == GNNPRE_BF16)
        return table_dtype == GNNPRE_F32 ? launch_sums_and_joins<__nv_bfloat16, float>(a, st) : launch_sums_and_joins<__nv_bfloat16, __nv_bfloat16>(a, st);
    return table_dtype == GNNPRE_F32 ? launch_sums_and_joins<__half, float>(a, st) : launch_sums_and_joins<__half, __half>(a, st);
}
