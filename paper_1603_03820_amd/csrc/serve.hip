// Answering with a trained factor model on gfx950 (MI355X): the C ABI of include/als_serve.h plus its kernels.
//
//   k_quantize    rows to 8-bit integers with one scale a row (k_quantize_long: rows of over 8,192 fp32 values)
//   k_score_tiles scores of users against items from 8-bit rows, by integer matrix instructions on tiles in LDS
//                 (k_pack lays rows of other strides and alignments out for it, in the workspace)
//   k_sample      one column a row from its scores: temperature, top-k, top-p, min-p, columns left out; a workgroup a
//                 row, which stays in registers
//   k_long_*      the same for rows past 65,536 columns, in segments
//
// The draw's arithmetic: a weight is a whole number, 2^40 times the exponential rounded down, and sums of
// weights are 64-bit integers.  So every sum is exact and may be taken in any order, by any number of threads and by
// atomics, and the set that top-p keeps and the column that a uniform number meets do not depend on how a row is
// held.  The rounding down costs a column at most 2^-40 of the best one's weight.

#include <hip/hip_bf16.h>
#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>

#include <atomic>
#include <cmath>
#include <cstdint>
#include <cstring>
#include <mutex>
#include <new>
#include <type_traits>

#include "als_serve.h"

namespace {

typedef int i4 __attribute__((ext_vector_type(4)));

constexpr int kWave = 64;

struct F16 { uint16_t bits; };
struct BF16 { uint16_t bits; };

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(F16 v) {
    return (float)__builtin_bit_cast(_Float16, v.bits);
}
__device__ __forceinline__ float to_float(BF16 v) {
    return __builtin_bit_cast(float, (uint32_t)v.bits << 16);
}
// The nearest value of the type, ties to even.
__device__ __forceinline__ void from_float(float v, float* out) { *out = v; }
__device__ __forceinline__ void from_float(float v, F16* out) {
    *out = F16{__builtin_bit_cast(uint16_t, (_Float16)v)};
}
__device__ __forceinline__ void from_float(float v, BF16* out) {
    *out = BF16{__builtin_bit_cast(uint16_t, (__bf16)v)};
}

// ------------------------------------------------------------------------------ quantize --

constexpr int kQuantThreads = 256;

// A row's scale from the bits of its largest magnitude (NaN where the row is not finite).
struct RowScale {
    float largest, inverse;
    bool finite, far;      // far: 127 x overflows, or the inverse does
    __device__ __forceinline__ explicit RowScale(uint32_t bits) {
        largest = __builtin_bit_cast(float, bits);
        finite = bits < 0x7F800000u;
        far = largest > 1e36f || largest < 1e-36f;
        inverse = 1.f / largest;
    }
    __device__ __forceinline__ float scale() const { return finite ? largest * (1.f / 127.f) : NAN; }
    // rint(127 x / a).  The product with 1 / a is within 2^-15 of the quotient, so it rounds to the same whole number
    // unless it lies that near to a half; a division takes ten instructions, and about one wave in twenty takes it.
    __device__ __forceinline__ int of(float x) const {
        const float y = x * 127.f, p = y * inverse;
        float r = rintf(p);
        if (far || !(fabsf(fabsf(p - r) - 0.5f) > 0x1p-14f)) {
            if (!finite || largest == 0.f) return 0;
            // past the largest float: a power of two off both sides changes no quotient
            const float down = largest > 1e36f ? 0x1p-8f : 1.f;
            r = rintf((x * down) * 127.f / (largest * down));
        }
        return (int)r;
    }
};

template <int N>
__device__ __forceinline__ uint32_t max_of_lanes(uint32_t v) {     // over N neighbouring lanes, to each
#pragma unroll
    for (int d = N / 2; d > 0; d >>= 1) v = max(v, (uint32_t)__shfl_xor(v, d));
    return v;
}

// `v` values of a row (of f) from k on as the bits of their magnitudes and as values, 0 past f.
template <typename T, int V>
__device__ __forceinline__ uint32_t load_row(const T* row, int k, int f, float (&x)[V]) {
    T t[V];
    if (k + V <= f) {
        __builtin_memcpy(t, row + k, sizeof t);
#pragma unroll
        for (int i = 0; i < V; ++i) x[i] = to_float(t[i]);
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) x[i] = k + i < f ? to_float(row[k + i]) : 0.f;
    }
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < V; ++i) most = max(most, __builtin_bit_cast(uint32_t, x[i]) & 0x7FFFFFFFu);
    return most;
}

// The values' whole numbers at k, as far as `end` (f, or with its padding).
template <int V>
__device__ __forceinline__ void store_row(int8_t* row, int k, int end, const RowScale& s, const float (&x)[V]) {
    if (k >= end) return;
    int8_t v[V];
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = (int8_t)s.of(x[i]);
    if (k + V <= end) {
        __builtin_memcpy(row + k, v, V);
    } else {
        for (int i = 0; i < V; ++i)
            if (k + i < end) row[k + i] = v[i];
    }
}

// G lanes a row (or, G = 256, a workgroup), 16 bytes a lane and load, E loads, all of which stay in registers between
// the largest magnitude and the quotients: each row is read once.  Bound by memory: 625,000 x 100 fp32 in 61 us
// (5.1 TB/s), 8,192 x 8,192 bf16 in 46 us (4.3 TB/s); in 16 bits, short rows by their conversions and quotients
// (625,000 x 100 bf16 in 66 us, 2.9 TB/s).
template <typename T, int G, int E>
__global__ __launch_bounds__(kQuantThreads) void k_quantize(const T* __restrict__ x, int64_t of, int64_t ldx,
                                                            const int32_t* __restrict__ users, int64_t rows,
                                                            int f, int8_t* __restrict__ q, int64_t ldq, int end,
                                                            float* __restrict__ scale) {
    constexpr int V = 16 / sizeof(T);
    __shared__ uint32_t of_waves[kQuantThreads / kWave];
    const int lane = threadIdx.x % G;
    const int64_t row = (int64_t)blockIdx.x * (kQuantThreads / G) + threadIdx.x / G;
    int64_t src = row;
    if (users) src = row < rows ? (int64_t)users[row] : -1;
    const bool there = row < rows && src >= 0 && src < of;
    const T* xr = x + (there ? src * ldx : 0);
    float v[E][V];
    uint32_t most = there ? 0 : 0x7FC00000u;
#pragma unroll
    for (int e = 0; e < E; ++e) most = max(most, load_row<T, V>(xr, (e * G + lane) * V, there ? f : 0, v[e]));
    most = max_of_lanes<(G < kWave ? G : kWave)>(most);
    if (G == kQuantThreads) {
        if (lane % kWave == 0) of_waves[lane / kWave] = most;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kQuantThreads / kWave; ++w) most = max(most, of_waves[w]);
    }
    if (row >= rows) return;
    const RowScale s(most);
#pragma unroll
    for (int e = 0; e < E; ++e) store_row<V>(q + row * ldq, (e * G + lane) * V, end, s, v[e]);
    if (lane == 0) scale[row] = s.scale();
}

// Rows that no workgroup's registers hold: a workgroup a row, the second read from the cache.
template <typename T>
__global__ __launch_bounds__(kQuantThreads) void k_quantize_long(const T* __restrict__ x, int64_t of, int64_t ldx,
                                                                 const int32_t* __restrict__ users, int64_t rows,
                                                                 int f, int8_t* __restrict__ q, int64_t ldq, int end,
                                                                 float* __restrict__ scale) {
    constexpr int V = 16 / sizeof(T);
    __shared__ uint32_t of_waves[kQuantThreads / kWave];
    const int64_t row = blockIdx.x;
    const int64_t src = users ? (int64_t)users[row] : row;
    const bool there = src >= 0 && src < of;
    const T* xr = x + (there ? src * ldx : 0);
    uint32_t m = there ? 0 : 0x7FC00000u;
    float v[V];
    for (int k = threadIdx.x * V; k < f; k += kQuantThreads * V) m = max(m, load_row<T, V>(xr, k, there ? f : 0, v));
    m = max_of_lanes<kWave>(m);
    if (threadIdx.x % kWave == 0) of_waves[threadIdx.x / kWave] = m;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kQuantThreads / kWave; ++w) m = max(m, of_waves[w]);
    const RowScale s(m);
    for (int k = threadIdx.x * V; k < end; k += kQuantThreads * V) {
        load_row<T, V>(xr, k, there ? f : 0, v);
        store_row<V>(q + row * ldq, k, end, s, v);
    }
    if (threadIdx.x == 0) scale[row] = s.scale();
}

// --------------------------------------------------------------------------------- score --

// Sixteen values of a row from column k on, zeros past column f (any alignment).
__device__ __forceinline__ i4 load16(const int8_t* row, int k, int f) {
    i4 v = {0, 0, 0, 0};
    if (k + 16 <= f) {
        __builtin_memcpy(&v, row + k, 16);
    } else if (k < f) {
        uint32_t w[4] = {0, 0, 0, 0};
        for (int b = 0; b < 16; ++b)
            if (k + b < f) w[b >> 2] |= (uint32_t)(uint8_t)row[k + b] << (8 * (b & 3));
        v = i4{(int)w[0], (int)w[1], (int)w[2], (int)w[3]};
    }
    return v;
}

// The product in tiles: a workgroup of WU x WI waves holds a tile of users x items, each wave FU x FI
// fragments of 16 x 16, and walks f in steps of 128.  A step's rows of both sides lie in LDS, 128 bytes a row, while
// the next steps' (STAGES - 1 of them) arrive straight from memory beside them (buffer_load ... lds: no
// registers, no instructions but the load).  The 16-byte group c of row r lies in slot c ^ s(r), so that the 16 rows of
// one operand read spread over all banks: s is r / 2 % 8 where an operand's rows are neighbours.  For
// outputs of 16 bits an item operand takes rows 0..3 of every 8 of 32, or 4..7 (so that a lane's four items of two
// fragments are neighbours and go out as 16 bytes), and s is r / 2 % 2 + 2 (r / 8 % 4).
// v_mfma_i32_16x16x64_i8 with the items as the first operand: a lane holds four neighbouring items of one user.  Items
// and users past the end, and values past f, are multiplied too: their results are not written, or one side is 0.
// 8,192^3 in 435 us, 2.5 Pop/s.  A step of a 256 x 256 tile brings 64 KB from memory and its eight waves read 192 KB of
// LDS for 16.8 Mop; counters: the matrix units are busy in 58% of the cycles, at about 2.0 GHz under this load (2.4 is
// the most), LDS without bank conflicts, waits for LDS in 2% of the waves' time.  At f <= 128 the scores' way out bounds
// it: 1,024 x 17,770 to fp32 in 16.3 us (4.6 TB/s), 4,096 x 40,000 in 150 us (4.4 TB/s; a kernel that only writes so takes
// 125), to bf16 in 91 us into two buffers in turn and 112 into fresh ones (3.6 and 3.0 TB/s).  Few users and wide rows are
// bound by the items' bytes: 5 x 8,192 x 8,192 in 14.7 us (4.6 TB/s).
constexpr int kStep = 128;
constexpr int64_t kTileStride = 1 << 22;        // row strides below it keep a tile's offsets below 2^30 ...
constexpr uint32_t kPastEnd = 0x7FFFFFF0u;      // ... and this past every tile's end

template <int WU, int WI, int FU, int FI, int STAGES>
struct Tiles {
    static constexpr int kWaves = WU * WI;
    static constexpr int kUsers = WU * FU * 16, kItems = WI * FI * 16;
    static constexpr int kRows = kUsers + kItems;
    static constexpr int kUserLoads = kUsers / 8 / kWaves, kItemLoads = kItems / 8 / kWaves;   // 1 KB, a wave and step
    static constexpr int kStage = kRows * kStep;           // bytes
    static constexpr int kStages = STAGES;
    static_assert(kUsers % (8 * kWaves) == 0 && kItems % (8 * kWaves) == 0, "whole loads");
    static_assert(FI % 2 == 0, "pairs of item fragments");
    static_assert((STAGES - 2) * (kUserLoads + kItemLoads) < 64, "loads that can be counted");
};

// A buffer of `bytes` bytes from `base` on (both the same in every lane).
__device__ __forceinline__ i4 buffer_of(const void* base, uint32_t bytes) {
    const uint64_t b = (uint64_t)base;
    i4 r;
    r[0] = __builtin_amdgcn_readfirstlane((uint32_t)b);
    r[1] = __builtin_amdgcn_readfirstlane((uint32_t)(b >> 32) & 0xFFFFu);
    r[2] = __builtin_amdgcn_readfirstlane(bytes);
    r[3] = 0x00020000;
    return r;
}

// 16 bytes a lane from buffer + voffset + soffset to LDS at `lds` + 16 lane.  Inline assembly: the compiler would
// wait for every load to LDS before any LDS read.  It has no result register; the caller waits
// (settle) before the data are read.  M0 needs one wait state.  (M0 is reserved and cannot be named as clobbered: a
// kernel with these loads must have nothing else that reads or keeps it, such as registers picked by an index.)
__device__ __forceinline__ void load_to_lds(i4 buffer, uint32_t voffset, uint32_t soffset, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %3\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, %2 offen lds"
                 :
                 : "v"(voffset), "s"(buffer), "s"(soffset), "s"(lds)
                 : "memory");
}
// A load reads a scalar register that a vector instruction wrote (readfirstlane) no sooner than five wait states
// later; the compiler keeps them for the loads it knows.
__device__ __forceinline__ void buffer_settle(i4 a, i4 b) { asm volatile("s_nop 4" : : "s"(a), "s"(b)); }
// All of this wave's loads but the last LEFT have arrived, and its LDS reads are done.
template <int LEFT>
__device__ __forceinline__ void settle() {
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" : : "n"(LEFT) : "memory");
}

// The bytes of the group at k that lie before f.
__device__ __forceinline__ i4 keep_bytes(i4 v, int k, int f) {
    const int left = f - k;
#pragma unroll
    for (int d = 0; d < 4; ++d) {
        const int bytes = left - 4 * d;
        v[d] &= bytes >= 4 ? -1 : (bytes > 0 ? (1 << (8 * bytes)) - 1 : 0);
    }
    return v;
}

// Tile t of a grid of tu x ti: the eight dies take workgroups in turn, so each gets a run of tiles of its own, and
// runs go down eight tiles of users before the next of items (their rows stay in the die's L2).
__device__ __forceinline__ void tile_of(uint32_t t, uint32_t tu, uint32_t ti, uint32_t* u, uint32_t* i) {
    const uint32_t total = tu * ti, per = total / 8;
    if (t < per * 8) t = (t % 8) * per + t / 8;
    const uint32_t band = 8 * ti, b = t / band, left = t % band;
    const uint32_t high = tu - 8 * b < 8 ? tu - 8 * b : 8;
    *u = 8 * b + left % high;
    *i = left / high;
}

template <typename T, int WU, int WI, int FU, int FI, int STAGES>
__global__ __launch_bounds__(64 * WU * WI) void k_score_tiles(
    const int8_t* __restrict__ xq, int64_t ldx, const float* __restrict__ xs, int64_t m,
    const int8_t* __restrict__ tq, int64_t ldt, const float* __restrict__ ts, int64_t n, int f,
    T* __restrict__ out, int64_t ldo, uint32_t tu, uint32_t ti) {
    using C = Tiles<WU, WI, FU, FI, STAGES>;
    constexpr bool kPairs = sizeof(T) == 2;
    extern __shared__ __align__(1024) unsigned char lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    uint32_t tile_u, tile_i;
    tile_of(blockIdx.x, tu, ti, &tile_u, &tile_i);
    const int64_t u0 = (int64_t)tile_u * C::kUsers, i0 = (int64_t)tile_i * C::kItems;

    // what the buffers hold: the tile's rows, the last up to the end of its last group
    const int64_t users = m - u0 < C::kUsers ? m - u0 : C::kUsers, items = n - i0 < C::kItems ? n - i0 : C::kItems;
    const int whole = (f + 15) / 16 * 16;
    const i4 from_u = buffer_of(xq + u0 * ldx, (uint32_t)((users - 1) * ldx + whole));
    const i4 from_i = buffer_of(tq + i0 * ldt, (uint32_t)((items - 1) * ldt + whole));
    buffer_settle(from_u, from_i);
    const int first_u = wave * C::kUserLoads * 8, first_i = wave * C::kItemLoads * 8;   // this wave's rows
    const auto spread_u = [](int r) { return r >> 1 & 7; };
    const auto spread_i = [](int r) { return kPairs ? (r >> 1 & 1) | (r >> 3 & 3) << 1 : r >> 1 & 7; };
    const auto group_u = [&](int r) { return 16 * ((lane & 7) ^ spread_u(r)); };
    const auto group_i = [&](int r) { return 16 * ((lane & 7) ^ spread_i(r)); };
    uint32_t of_u[C::kUserLoads], of_i[C::kItemLoads];
#pragma unroll
    for (int l = 0; l < C::kUserLoads; ++l) {
        const int r = first_u + 8 * l + (lane >> 3);
        of_u[l] = (uint32_t)(r * ldx) + group_u(r);
    }
#pragma unroll
    for (int l = 0; l < C::kItemLoads; ++l) {
        const int r = first_i + 8 * l + (lane >> 3);
        of_i[l] = (uint32_t)(r * ldt) + group_i(r);
    }
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)lds;
    const int steps = (f + kStep - 1) / kStep;
    // groups past f are not read: their offset is past the buffer's end
    const auto fetch = [&](int step, int stage, auto tail) {
        const uint32_t to = lds0 + stage * C::kStage;
#pragma unroll
        for (int l = 0; l < C::kUserLoads; ++l) {
            const int r = first_u + 8 * l;
            const bool in = !tail.value || step * kStep + group_u(r + (lane >> 3)) < f;
            load_to_lds(from_u, in ? of_u[l] : kPastEnd, step * kStep,
                        __builtin_amdgcn_readfirstlane(to + r * kStep));
        }
#pragma unroll
        for (int l = 0; l < C::kItemLoads; ++l) {
            const int r = first_i + 8 * l;
            const bool in = !tail.value || step * kStep + group_i(r + (lane >> 3)) < f;
            load_to_lds(from_i, in ? of_i[l] : kPastEnd, step * kStep,
                        __builtin_amdgcn_readfirstlane(to + (C::kUsers + r) * kStep));
        }
    };
    const auto fetch_any = [&](int step, int stage) {
        if (step + 1 < steps) fetch(step, stage, std::false_type());
        else fetch(step, stage, std::true_type());
    };

    const int wu = wave / WI, wi = wave % WI;
    const int row = lane & 15, group = lane >> 4;
    i4 acc[FU][FI];
#pragma unroll
    for (int u = 0; u < FU; ++u)
#pragma unroll
        for (int i = 0; i < FI; ++i) acc[u][i] = i4{0, 0, 0, 0};

    // the first item of fragment i's rows 4 x (of a lane's results: 4 group), and the row of the operand's row x
    const auto item_of = [&](int i, int x) {
        return kPairs ? (wi * FI + (i & ~1)) * 16 + 8 * x + 4 * (i & 1) : (wi * FI + i) * 16 + 4 * x;
    };
    const auto multiply = [&](int step, int stage, auto tail) {
        const unsigned char* at = lds + stage * C::kStage;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            i4 a[FI], b[FU];
#pragma unroll
            for (int i = 0; i < FI; ++i) {
                const int r = item_of(i, row >> 2) + (row & 3);
                a[i] = *(const i4*)(at + (C::kUsers + r) * kStep + 16 * ((4 * h + group) ^ spread_i(r)));
            }
#pragma unroll
            for (int u = 0; u < FU; ++u) {
                const int r = (wu * FU + u) * 16 + row;
                b[u] = *(const i4*)(at + r * kStep + 16 * ((4 * h + group) ^ spread_u(r)));
                if (tail.value) b[u] = keep_bytes(b[u], step * kStep + 64 * h + 16 * group, f);
            }
#pragma unroll
            for (int u = 0; u < FU; ++u)
#pragma unroll
                for (int i = 0; i < FI; ++i)
                    acc[u][i] = __builtin_amdgcn_mfma_i32_16x16x64_i8(a[i], b[u], acc[u][i], 0, 0, 0);
        }
    };

#pragma unroll
    for (int p = 0; p < STAGES - 1; ++p)
        if (p < steps) fetch_any(p, p);
    // the scales, here rather than where they are used: there, each load would be waited for
    float s[FU], t[FI][4];
#pragma unroll
    for (int u = 0; u < FU; ++u) {
        const int64_t user = u0 + (wu * FU + u) * 16 + row;
        s[u] = xs[user < m ? user : m - 1];
    }
#pragma unroll
    for (int i = 0; i < FI; ++i) {
        const int64_t item = i0 + item_of(i, group);
        if (item + 4 <= n) __builtin_memcpy(t[i], ts + item, 16);
        else
            for (int r = 0; r < 4; ++r) t[i][r] = ts[item + r < n ? item + r : n - 1];
    }
    // a step: its rows are there and the last step's are done with (one barrier for both), whose place the rows
    // STAGES - 1 steps on take
    int stage = 0;
    const auto after = [](int x) { return x + 1 == STAGES ? 0 : x + 1; };
    int step = 0;
    for (; step + STAGES - 1 < steps; ++step) {
        settle<(STAGES - 2) * (C::kUserLoads + C::kItemLoads)>();
        __builtin_amdgcn_s_barrier();
        fetch_any(step + STAGES - 1, stage == 0 ? STAGES - 1 : stage - 1);
        multiply(step, stage, std::false_type());
        stage = after(stage);
    }
    settle<0>();
    __builtin_amdgcn_s_barrier();
    for (; step + 1 < steps; ++step) {
        multiply(step, stage, std::false_type());
        stage = after(stage);
    }
    multiply(step, stage, std::true_type());

#pragma unroll
    for (int u = 0; u < FU; ++u) {
        const int64_t user = u0 + (wu * FU + u) * 16 + row;
        if (user >= m) continue;
        T* o = out + user * ldo;
        constexpr int kTogether = kPairs ? 2 : 1;
#pragma unroll
        for (int i = 0; i < FI; i += kTogether) {
            const int64_t item = i0 + item_of(i, group);
            T v[4 * kTogether];
#pragma unroll
            for (int r = 0; r < 4 * kTogether; ++r)
                from_float((float)acc[u][i + r / 4][r % 4] * s[u] * t[i + r / 4][r % 4], &v[r]);
            if (item + 4 * kTogether <= n) {
                __builtin_memcpy(o + item, v, sizeof v);
            } else {
                for (int r = 0; r < 4 * kTogether; ++r)
                    if (item + r < n) o[item + r] = v[r];
            }
        }
    }
}

// Rows of any stride and alignment to rows of a stride that is a multiple of 16, zeros past f: anew in every call, so rows
// that are scored again and again are better held so.  With it and without, us: 1,024 x 17,770 x 100 23 and 16,
// 1 x 625,000 x 100 45 and 14, 8,192^3 461 and 418.
__global__ __launch_bounds__(256) void k_pack(const int8_t* __restrict__ from, int64_t ld, int64_t rows, int f,
                                              int8_t* __restrict__ to, int64_t groups) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= rows * groups) return;
    const int64_t r = i / groups;
    const i4 v = load16(from + r * ld, (int)(i - r * groups) * 16, f);
    *(i4*)(to + i * 16) = v;
}

// -------------------------------------------------------------------------------- sample --

constexpr int kSampleThreads = 1024;
constexpr int kSampleWaves = kSampleThreads / kWave;
constexpr int kBins = 2048;
constexpr int kList = 1024;              // candidates that are ranked one against another
constexpr int kChunk = 1 << 19;          // columns whose left-out bits are held at a time (64 KB)

struct Limits {
    const float* temperature;
    const int32_t* top_k;
    const float* top_p;
    const float* min_p;
    float temperature_all;
    int32_t top_k_all;
    float top_p_all;
    float min_p_all;
};

// Larger scores have larger keys; -0 has +0's.
__device__ __forceinline__ uint32_t key_of(float z) {
    const uint32_t b = __builtin_bit_cast(uint32_t, z + 0.f);
    return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float score_of(uint32_t key) {
    const uint32_t b = key & 0x80000000u ? key ^ 0x80000000u : ~key;
    return __builtin_bit_cast(float, b);
}

__device__ __forceinline__ float unit_of(float u) { return u > 0.f ? fminf(u, 1.f - 0x1p-24f) : 0.f; }

// floor(total part / 2^24), part <= 2^24, total < 2^62.
__device__ __forceinline__ uint64_t share_of(uint64_t total, uint32_t part) {
    return (total >> 24) * part + (((total & 0xFFFFFFu) * part) >> 24);
}

// One of the wave's DPP moves of a 64-bit value: lanes without a source get 0.
template <int CTRL, int ROWS>
__device__ __forceinline__ uint64_t dpp64(uint64_t v) {
    const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)v, CTRL, ROWS, 0xF, false);
    const uint32_t hi = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)(v >> 32), CTRL, ROWS, 0xF, false);
    return (uint64_t)hi << 32 | lo;
}
template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t dpp32(uint32_t v) {
    return __builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xF, false);
}
// Inclusive sums over the wave: within rows of 16 lanes, then across rows.
__device__ __forceinline__ uint64_t scan64(uint64_t v) {
    v += dpp64<0x111, 0xF>(v);   // row_shr:1, 2, 4, 8
    v += dpp64<0x112, 0xF>(v);
    v += dpp64<0x114, 0xF>(v);
    v += dpp64<0x118, 0xF>(v);
    v += dpp64<0x142, 0xA>(v);   // row_bcast:15 into rows 1 and 3
    v += dpp64<0x143, 0xC>(v);   // row_bcast:31 into rows 2 and 3
    return v;
}
__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
    v = max(v, dpp32<0x111, 0xF>(v));
    v = max(v, dpp32<0x112, 0xF>(v));
    v = max(v, dpp32<0x114, 0xF>(v));
    v = max(v, dpp32<0x118, 0xF>(v));
    v = max(v, dpp32<0x142, 0xA>(v));
    v = max(v, dpp32<0x143, 0xC>(v));
    return __builtin_amdgcn_readlane(v, 63);
}
__device__ __forceinline__ float wave_max(float v) {      // NaN-free
    const uint32_t least = __builtin_bit_cast(uint32_t, -INFINITY);
#define ALS_STEP(CTRL, ROWS)                                                                                        \
    v = fmaxf(v, __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(                                             \
                     (int)least, (int)__builtin_bit_cast(uint32_t, v), CTRL, ROWS, 0xF, false)))
    ALS_STEP(0x111, 0xF);
    ALS_STEP(0x112, 0xF);
    ALS_STEP(0x114, 0xF);
    ALS_STEP(0x118, 0xF);
    ALS_STEP(0x142, 0xA);
    ALS_STEP(0x143, 0xC);
#undef ALS_STEP
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), 63));
}
__device__ __forceinline__ uint64_t last64(uint64_t v) {
    return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((uint32_t)(v >> 32), 63) << 32 |
           (uint32_t)__builtin_amdgcn_readlane((uint32_t)v, 63);
}

// What a row asks for, and its best score: all that a weight depends on.
struct Asked {
    float top, inv_t;   // the best score, 1 / T (both finite: see Held::plain)
    float least;        // 2^40 min_p
    float t;
    __device__ __forceinline__ Asked(float best, float t_, float least_)
        : top(best), inv_t(1.f / t_), least(least_), t(t_) {}

    // 2^40 exp((z - top) / T), z <= top, of the exponential rounded to fp32: 2 to the nearest whole number of
    // x log2(e), held in two parts, times 2 to the rest.  Where that is 1 or more it equals 2^40 expf(x) in every bit
    // for all but 2 of the 1.1e9 such x (tested one by one), at half its instructions: x ends at -64, where no weight
    // is left (nor where a difference or product is not a number), so that nothing overflows.  (The reduction by log2(e)
    // in two parts is Cody and Waite's; the result falls with x over all those floats, tested too.)  The whole number comes
    // by adding 1.5 2^23 (+ 40), whose sum has it in its last bits; they go to the exponent.  No product may be
    // fused into a sum here but the two that are written so.
    __device__ __forceinline__ float scaled(float z) const {
#pragma clang fp contract(off)
        const float x = fmaxf((z - top) * inv_t, -64.f);
        const float high = x * 0x1.715476p+0f;
        const float low = fmaf(x, 0x1.4ae0cp-26f, fmaf(x, 0x1.715476p+0f, -high));
        const float shifted = high + (0x1.8p23f + 40.f);
        const float part = __builtin_amdgcn_exp2f((high - (shifted - (0x1.8p23f + 40.f))) + low);
        return __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, part) +
                                             (__builtin_bit_cast(uint32_t, shifted) << 23));
    }
    // Whether the formula holds: with a best score of +inf, or 1 / T past the largest float, the best columns weigh
    // 2^40 each and all others nothing.
    __device__ __forceinline__ bool is_plain() const { return top < INFINITY && inv_t < INFINITY; }
    // The weight, a whole number of at most 24 significant bits.
    __device__ __forceinline__ float weight_of(float z) const { return floorf(scaled(z)); }
};

__device__ __forceinline__ uint64_t whole_of(float w) {      // of a weight
    const uint32_t high = (uint32_t)(w * 0x1p-20f);
    return ((uint64_t)high << 20) + (uint32_t)fmaf((float)high, -0x1p20f, w);
}
// 53 bits hold the sum of a thread's weights.
__device__ __forceinline__ uint64_t whole_of(double w) {
    const uint32_t high = (uint32_t)(w * 0x1p-32);
    return ((uint64_t)high << 32) + (uint32_t)fma((double)high, -0x1p32, w);
}

// A place in the order (score descending, position ascending): what stands up to it, itself included, stays.
struct Cut {
    float z = -INFINITY;        // every allowed score is larger
    int position = -1;
    __device__ __forceinline__ bool keeps(float v, uint32_t p) const {
        return v > z || (v == z && (int)p <= position);
    }
};

// One row in the registers of a workgroup: K scores a thread (-inf: not allowed), four neighbours at a time, a
// wave's positions in one run.  The loops over them stay loops (a register is picked by a uniform index): unrolled,
// a row's passes are one long run of code that no instruction cache holds, at four times the time.
// Bins and list are LDS: a cut is found by a histogram over the scores, then by ranking the columns of the one bin
// in which it falls.  LDS sums are of integers, so their order does not matter.
template <int K, int BINS>
struct Held {
    static constexpr int kScores = K, kBins = BINS, kList = BINS < 1024 ? BINS / 2 : 1024, kMaxWaves = 16;
    static constexpr int kRanked = BINS / 2 < 256 ? BINS / 2 : 256;      // columns that are ranked one against another
    typedef float Scores __attribute__((ext_vector_type(K < 32 ? K : 32)));
    static_assert(K % 4 == 0 && K <= 64, "scores a thread");    // (its weights add up below 2^53)
    struct Shared {
        uint64_t bin[kBins];
        float list_z[kList];
        uint32_t list_position[kList];
        uint64_t wave_sum[kMaxWaves];
        float wave_a[kMaxWaves], wave_b[kMaxWaves];
        uint32_t wave_c[kMaxWaves];
        uint64_t found_before;
        uint32_t found_bin, listed;
        float cut_z;
        uint32_t cut_position;
        uint32_t low, high;
    };
    Scores z[(K + 31) / 32];
    Shared* sh;
    int threads, waves;      // of the workgroup

    static __device__ __forceinline__ int lane() { return threadIdx.x & (kWave - 1); }
    static __device__ __forceinline__ int wave() { return __builtin_amdgcn_readfirstlane(threadIdx.x / kWave); }
    // of the first of a thread's four scores v
    static __device__ __forceinline__ uint32_t position(int v) {
        return (uint32_t)(wave() * (K / 4) + v) * (4 * kWave) + 4 * lane();
    }
    __device__ __forceinline__ void sync() const {
        if (waves > 1) __syncthreads();
        else __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
    // Where the weights' formula does not hold (the best columns weigh 2^40 each and all others nothing), scores for
    // which it does: 0 for the best, none for the others.
    __device__ __forceinline__ void plain(Asked& ask) {
        if (ask.is_plain()) return;
#pragma unroll
        for (int v = 0; v < K; ++v) z[v / 32][v % 32] = z[v / 32][v % 32] == ask.top ? 0.f : -INFINITY;
        ask = Asked(0.f, 1.f, ask.least);
    }
    // fn(score, position) for every held score.
    template <typename Fn>
    __device__ __forceinline__ void each(Fn fn) const {
#pragma unroll
        for (int h = 0; h < (K + 31) / 32; ++h) {
            uint32_t p = position(8 * h);
#pragma nounroll
            for (int v = 0; v < (K < 32 ? K : 32); v += 4, p += 4 * kWave)
#pragma unroll
                for (int c = 0; c < 4; ++c) fn(z[h][v + c], p + c);
        }
    }

    // The same without a loop, for passes of a few instructions a score.
    template <typename Fn>
    __device__ __forceinline__ void each_at_once(Fn fn) const {
#pragma unroll
        for (int v = 0; v < K; v += 4)
#pragma unroll
            for (int c = 0; c < 4; ++c) fn(z[v / 32][v % 32 + c], position(v / 4) + c);
    }

    // Of the waves' sums: their sum, and the sum of those before this wave's.
    __device__ __forceinline__ uint64_t sum(uint64_t mine, uint64_t* before_wave) {
        sync();
        if (lane() == 0) sh->wave_sum[wave()] = mine;
        sync();
        uint64_t total = 0;
        *before_wave = 0;
        for (int w = 0; w < waves; ++w) {
            if (w == wave()) *before_wave = total;
            total += sh->wave_sum[w];
        }
        return total;
    }

    // A thread's largest score, and the workgroup's.
    __device__ __forceinline__ float largest(float* best) {
        float mine = -INFINITY;
        each_at_once([&](float k, uint32_t) { mine = fmaxf(mine, k); });
        float hi = wave_max(mine);
        if (waves > 1) {
            if (lane() == 0) sh->wave_a[wave()] = hi;
            sync();
            for (int w = 0; w < waves; ++w) hi = fmaxf(hi, sh->wave_a[w]);
        }
        *best = hi;
        return mine;
    }
    // The least allowed score of every fourth column: near enough to the least for bins.
    __device__ __forceinline__ float near_least() {
        float lo = -INFINITY;    // its negative
#pragma unroll
        for (int v = 0; v < K; v += 4) {
            const float k = z[v / 32][v % 32];
            lo = fmaxf(lo, k > -INFINITY ? -k : -INFINITY);
        }
        lo = wave_max(lo);
        if (waves > 1) {
            sync();
            if (lane() == 0) sh->wave_b[wave()] = lo;
            sync();
            lo = -INFINITY;
            for (int w = 0; w < waves; ++w) lo = fmaxf(lo, sh->wave_b[w]);
        }
        return -lo;
    }

    // A value that at least k of those reach that `values(fn)` hands this thread, and few more: the k-th largest, as
    // near below it as bins tell.  -inf: there are fewer than k.  `best` is the largest.
    template <typename Values>
    __device__ __forceinline__ float reached_by(uint32_t k, float best, Values values) {
        constexpr int kCoarse = kBins < 256 ? kBins : 256;
        float low = -INFINITY;      // the least one's negative
        values([&](float v) { low = fmaxf(low, v > -INFINITY ? -v : -INFINITY); });
        low = wave_max(low);
        sync();
        if (lane() == 0) sh->wave_b[wave()] = low;
        for (int b = threadIdx.x; b < kCoarse; b += threads) sh->bin[b] = 0;
        if (threadIdx.x == 0) sh->found_bin = kCoarse;
        sync();
        for (int w = 0; w < waves; ++w) low = fmaxf(low, sh->wave_b[w]);
        const float per = best + low > 0.f ? (float)(kCoarse - 1) / (best + low) : 0.f;
        const auto bin_of = [&](float v) {
            const float x = (best - v) * per;
            return v == best ? 0 : (x < (float)(kCoarse - 1) ? (int)x : kCoarse - 1);
        };
        values([&](float v) {
            if (v > -INFINITY) atomicAdd((unsigned long long*)&sh->bin[bin_of(v)], 1ull);
        });
        search_bins([&](uint64_t) { return (uint64_t)k; }, kCoarse);
        const int found = (int)sh->found_bin;
        low = -INFINITY;
        values([&](float v) { low = fmaxf(low, v > -INFINITY && bin_of(v) <= found ? -v : -INFINITY); });
        low = wave_max(low);
        if (lane() == 0) sh->wave_a[wave()] = low;
        sync();
        for (int w = 0; w < waves; ++w) low = fmaxf(low, sh->wave_a[w]);
        return found == kCoarse ? -INFINITY : -low;
    }

    // put(i, score, position) for the columns that `take(score)` picks, i counting them by position, where they
    // are no more than `most`; how many there are.
    template <typename Take, typename Put>
    __device__ __forceinline__ uint32_t collect(uint32_t most, Take take, Put put) {
        uint32_t mine = 0;
        each_at_once([&](float k, uint32_t) { mine += (uint32_t)__popcll(__ballot(take(k))); });
        sync();
        if (lane() == 0) sh->wave_c[wave()] = mine;
        sync();
        uint32_t total = 0, at = 0;
        for (int w = 0; w < waves; ++w) {
            if (w == wave()) at = total;
            total += sh->wave_c[w];
        }
        sync();
        if (total > most) return total;
#pragma unroll
        for (int v = 0; v < K; v += 4) {
            uint64_t takes[4];
            uint32_t all = 0;
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                takes[c] = __ballot(take(z[v / 32][v % 32 + c]));
                all += __popcll(takes[c]);
            }
            if (all) {
                uint32_t mine = at;
#pragma unroll
                for (int c = 0; c < 4; ++c)
                    mine = __builtin_amdgcn_mbcnt_hi((uint32_t)(takes[c] >> 32),
                                                     __builtin_amdgcn_mbcnt_lo((uint32_t)takes[c], mine));
#pragma unroll
                for (int c = 0; c < 4; ++c)
                    if (takes[c] >> lane() & 1) put(mine++, z[v / 32][v % 32 + c], position(v / 4) + c);
                at += all;
            }
        }
        sync();
        return total;
    }

    // The first position at which the running sum of measure(score, position), a whole number, exceeds t (the
    // sum over all does).
    template <typename Fn>
    __device__ __forceinline__ uint32_t find(uint64_t t, uint64_t mine, uint64_t before_wave, Fn measure) {
        // `mine`: this wave's sum; exactly one wave holds the place
        if (t >= before_wave && t - before_wave < mine) {
            uint64_t left = t - before_wave;
            bool open = true;
#pragma unroll
            for (int h = 0; h < (K + 31) / 32; ++h) {
                uint32_t p = position(8 * h);
#pragma nounroll
                for (int v = 0; open && v < (K < 32 ? K : 32); v += 4, p += 4 * kWave) {
                    uint64_t s = 0;
#pragma unroll
                    for (int c = 0; c < 4; ++c) s += whole_of(measure(z[h][v + c], p + c));
                    const uint64_t upto = scan64(s), all = last64(upto);
                    if (left < all) {
                        uint64_t at = upto - s;
#pragma nounroll
                        for (int c = 0; c < 4; ++c) {
                            const uint64_t w = whole_of(measure(z[h][v + c], p + c));
                            if (left >= at && left < at + w) sh->cut_position = p + c;
                            at += w;
                        }
                        open = false;
                    } else {
                        left -= all;
                    }
                }
            }
        }
        sync();
        const uint32_t p = sh->cut_position;
        sync();
        return p;
    }

    // The bin of a score: linear from the best one down, the last bin for all that is the range or more below it.
    struct Scale { float top, per; };
    // Down to `least` (or some score near the least: the last bin has all that is below), but no further than 28 T
    // below the best, where a weight is 0 (clipped).
    static __device__ __forceinline__ Scale scale_of(float top, float least, float t, bool* clipped) {
        const float all = top - least;
        *clipped = all > 28.f * t;
        const float range = *clipped ? 28.f * t : all;
        return Scale{top, range > 1e-30f ? (float)(kBins - 1) / range : 0.f};
    }
    __device__ __forceinline__ int bin_of(float k, const Scale& c) const {
        return (int)fminf((c.top - k) * c.per, (float)(kBins - 1));
    }
    __device__ __forceinline__ void add_to_bin(uint32_t bin, bool by_mass, float k, const Asked& ask) {
        const uint64_t w = by_mass ? whole_of(ask.weight_of(k)) : 1;
        if (w) atomicAdd((unsigned long long*)&sh->bin[bin], (unsigned long long)w);
    }

    // The least score of bins 0 .. b (of all scores above -inf): bins fall with the score, so the wave cuts the range
    // of keys into 64 until it is one key.
    __device__ __forceinline__ float least_of_bins(int b, const Scale& c) const {
        uint32_t no = key_of(-INFINITY), yes = key_of(c.top);      // the last key above the bins, the first within
        while (yes - no > 1) {
            const uint32_t step = (yes - no - 1) / kWave + 1;
            const uint64_t at = (uint64_t)no + (uint64_t)step * (lane() + 1);
            const uint64_t in = __ballot(at >= yes || bin_of(score_of((uint32_t)at), c) <= b);
            const int first = in ? __ffsll((unsigned long long)in) - 1 : kWave;
            const uint64_t next = (uint64_t)no + (uint64_t)step * (first + 1);
            no += step * first;
            yes = next < yes ? (uint32_t)next : yes;
        }
        return score_of(yes);
    }

    // Adds up the bins in their order: the first at which the sum reaches the target (found_bin,
    // found_before).  target(total) is asked once the total is known.
    template <typename Fn>
    __device__ __forceinline__ void search_bins(Fn target, int bins = kBins) {
        sync();
        const int per = (bins + threads - 1) / threads, first = per * threadIdx.x;
        const int end = first + per < bins ? first + per : bins;
        uint64_t s = 0, before;
        for (int b = first; b < end; ++b) s += sh->bin[b];
        const uint64_t upto = scan64(s);
        if (lane() == 63) sh->wave_sum[wave()] = upto;
        if (threadIdx.x == 0) sh->listed = 0;
        sync();
        uint64_t total = 0;
        for (int w = 0; w < waves; ++w) {
            if (w == wave()) before = total;
            total += sh->wave_sum[w];
        }
        uint64_t at = before + upto - s;
        const uint64_t goal = target(total);
        if (at < goal && goal <= at + s)
            for (int b = first; b < end; ++b) {
                const uint64_t v = sh->bin[b];
                if (at < goal && goal <= at + v) {
                    sh->found_bin = b;
                    sh->found_before = at;
                }
                at += v;
            }
        sync();
    }

    // The columns that `take` picks and their measures, in the bins' place (which are done with), as far as kRanked go;
    // how many there are.  An entry is a number that orders the columns, and the measure.
    template <typename Fn>
    __device__ __forceinline__ uint32_t make_list(bool by_mass, const Asked& ask, Fn take) {
        each([&](float k, uint32_t p) {
            if (take(k, p)) {
                const uint32_t at = atomicAdd(&sh->listed, 1u);
                if (at < (uint32_t)kRanked) {
                    sh->bin[2 * at] = (uint64_t)~key_of(k) << 32 | p;
                    sh->bin[2 * at + 1] = by_mass ? whole_of(ask.weight_of(k)) : 1;
                }
            }
        });
        sync();
        return sh->listed;
    }

    // Among the listed columns, the last with less than `goal` of the measure before it.
    __device__ __forceinline__ Cut rank_list(uint32_t count, uint64_t before, uint64_t goal) {
        for (uint32_t i = threadIdx.x; i < count; i += threads) {
            const uint64_t key = sh->bin[2 * i], own = sh->bin[2 * i + 1];
            uint64_t front = before;
#pragma unroll 4
            for (uint32_t j = 0; j < count; ++j) front += sh->bin[2 * j] < key ? sh->bin[2 * j + 1] : 0;
            if (front < goal && goal <= front + own) {
                sh->cut_z = score_of(~(uint32_t)(key >> 32));
                sh->cut_position = (uint32_t)key;
            }
        }
        sync();
        Cut cut;
        cut.z = sh->cut_z;
        cut.position = (int)sh->cut_position;
        sync();
        return cut;
    }

    // The last column, in the order, with less than the target of the measure before it, among the columns
    // that `within` keeps.  by_mass: the measure is the weight and the target share_of(its sum, part), at least 1;
    // else the target is `part` columns; all stay where there are fewer.
    // (`given`, where it is not 0, is the target itself.)
    __device__ __forceinline__ Cut select(bool by_mass, Cut within, float least, uint32_t part, const Asked& ask,
                                          uint64_t given = 0) {
        sync();
        for (int b = threadIdx.x; b < kBins; b += threads) sh->bin[b] = 0;
        if (threadIdx.x == 0) sh->found_bin = kBins;
        sync();
        bool clipped;
        const Scale scale = scale_of(ask.top, least, ask.t, &clipped);
        each([&](float k, uint32_t p) {
            if (within.keeps(k, p)) add_to_bin(bin_of(k, scale), by_mass, k, ask);
        });
        uint64_t goal;
        search_bins([&](uint64_t total) {
            goal = given ? given : (by_mass ? share_of(total, part) : part);
            if (goal < 1) goal = 1;
            return goal;
        });
        const int bin = sh->found_bin;
        uint64_t before = sh->found_before;
        if (bin == kBins) return within;                               // fewer columns than asked for
        if (!by_mass && clipped && bin == kBins - 1) return within;   // what would go has no weight
        uint32_t listed =
            make_list(by_mass, ask, [&](float k, uint32_t p) { return within.keeps(k, p) && bin_of(k, scale) == bin; });
        if (listed <= (uint32_t)kRanked) return rank_list(listed, before, goal);

        // Many columns crowd the bin (equal scores, or some far from the others): bins of its keys, narrowed until
        // the rest can be ranked or is one score.
        const uint32_t best = key_of(ask.top);
        uint32_t lo = 0, hi = 0;     // distances of keys from the best
        for (bool keys = false;; keys = true) {
            const auto in = [&](float k, uint32_t p) {
                const uint32_t d = best - key_of(k);
                return within.keeps(k, p) && (keys ? d >= lo && d <= hi : bin_of(k, scale) == bin);
            };
            uint32_t far = 0, near = 0;        // the largest distance, the least one's complement
            each([&](float k, uint32_t p) {
                const uint32_t d = best - key_of(k);
                if (in(k, p)) { far = max(far, d); near = max(near, ~d); }
            });
            far = wave_max(far);
            near = wave_max(near);
            sync();
            if (threadIdx.x == 0) { sh->high = 0; sh->low = 0; }
            for (int b = threadIdx.x; b < kBins; b += threads) sh->bin[b] = 0;
            sync();
            if (lane() == 0) { atomicMax(&sh->high, far); atomicMax(&sh->low, near); }
            sync();
            lo = ~sh->low;
            hi = sh->high;
            if (lo != hi) {
                int shift = 0;
                while (((hi - lo) >> shift) >= (uint32_t)kBins) ++shift;
                each([&](float k, uint32_t p) {
                    const uint32_t d = best - key_of(k) - lo;
                    if (d <= hi - lo && within.keeps(k, p)) add_to_bin(d >> shift, by_mass, k, ask);
                });
                search_bins([&](uint64_t) { return goal - before; });
                before += sh->found_before;
                lo += sh->found_bin << shift;
                const uint32_t end = lo + ((1u << shift) - 1);
                hi = end < hi ? end : hi;
            }
            if (lo == hi) {     // equal scores: as many of them, by position, as reach the goal
                Cut cut;
                cut.z = score_of(best - lo);
                const uint64_t own = by_mass ? whole_of(ask.weight_of(cut.z)) : 1;
                const uint64_t more = (goal - before + own - 1) / own;
                const auto same = [&](float k, uint32_t p) { return k == cut.z && within.keeps(k, p) ? 1.f : 0.f; };
                float count = 0.f;
                each([&](float k, uint32_t p) { count += same(k, p); });
                const uint64_t mine = last64(scan64((uint64_t)(uint32_t)count));
                uint64_t before_wave;
                sum(mine, &before_wave);
                cut.position = (int)find(more - 1, mine, before_wave, same);
                return cut;
            }
            listed = make_list(by_mass, ask, [&](float k, uint32_t p) {
                return best - key_of(k) - lo <= hi - lo && within.keeps(k, p);
            });
            if (listed <= (uint32_t)kRanked) return rank_list(listed, before, goal);
        }
    }

    // The draw: the position, and the logarithm of its probability (to every thread).
    struct Drawn { uint32_t position; float log; };
    template <typename Wanted>
    __device__ __forceinline__ Drawn draw(const Wanted& want, const Asked& ask) {
        const int top_k = want.top_k;
        const float top_p = want.top_p;
        Cut cut;
        float least = 0.f;
        if (top_k > 0 || top_p < 1.f) least = near_least();
#pragma nounroll
        for (int by_mass = 0; by_mass < 2; ++by_mass) {     // one copy of the code for both cuts
            if (by_mass ? !(top_p < 1.f) : top_k <= 0) continue;
            cut = select(by_mass != 0, cut, least, by_mass ? want.part() : (uint32_t)top_k, ask);
        }
        const auto weight = [&](float k, uint32_t p) {
            const float e = ask.scaled(k);
            return cut.keeps(k, p) && e >= ask.least ? floorf(e) : 0.f;
        };
        double thread = 0.0;
        if (cut.position < 0 && !(ask.least > 0.f)) each([&](float k, uint32_t) { thread += (double)ask.weight_of(k); });
        else each([&](float k, uint32_t p) { thread += (double)weight(k, p); });
        const uint64_t mine = last64(scan64(whole_of(thread)));
        uint64_t before_wave;
        const uint64_t total = sum(mine, &before_wave);
        const uint32_t p = find(share_of(total, (uint32_t)(want.u * 0x1p24f)), mine, before_wave, weight);
        each([&](float k, uint32_t at) { if (at == p) sh->cut_z = k; });
        sync();
        const float k = sh->cut_z;
        const float x = (k - ask.top) * ask.inv_t;
        return Drawn{p, x - logf((float)total * 0x1p-40f)};
    }

    // The first position of the best score.
    __device__ __forceinline__ uint32_t first_of(float best) {
        uint32_t p = 0;
        each([&](float k, uint32_t at) { if (k == best) p = max(p, ~at); });
        p = wave_max(p);
        if (waves > 1) {
            sync();
            if (lane() == 0) sh->wave_c[wave()] = p;
            sync();
            for (int w = 0; w < waves; ++w) p = max(p, sh->wave_c[w]);
        }
        return ~p;
    }
};

__device__ __forceinline__ float limit_of(const float* each, float all, int64_t r) { return each ? each[r] : all; }

// A row's CSR row of columns to leave out.
struct Rated {
    const int64_t* ptr;
    const int32_t* idx;
    const int32_t* users;
    int64_t of;
    // false: the row's user does not exist
    __device__ __forceinline__ bool row(int64_t r, const int32_t** list, int64_t* count) const {
        *list = nullptr;
        *count = 0;
        if (!ptr) return true;
        const int64_t u = users ? (int64_t)users[r] : r;
        if (u < 0 || u >= of) return false;
        const int64_t first = ptr[u];
        *list = idx + first;
        *count = ptr[u + 1] - first;
        return true;
    }
};

// Four neighbouring scores as they lie in memory.
template <typename T>
struct Four { uint32_t word[sizeof(T)]; };
__device__ __forceinline__ void less_than_all(float* v) { *v = -INFINITY; }
__device__ __forceinline__ void less_than_all(F16* v) { *v = F16{0xFC00}; }
__device__ __forceinline__ void less_than_all(BF16* v) { *v = BF16{0xFF80}; }

// Columns base .. base + n of a row on their way into registers (-inf past them).
template <typename H, typename T>
__device__ __forceinline__ void fetch_columns(const H& h, const T* row, uint32_t base, uint32_t n,
                                              Four<T> (&raw)[H::kScores / 4]) {
#pragma unroll
    for (int v = 0; v < H::kScores / 4; ++v) {
        const uint32_t c = h.position(v);
        if (c + 4 <= n) {
            __builtin_memcpy(&raw[v], row + base + c, sizeof raw[v]);
        } else {
            T t[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                less_than_all(&t[i]);
                if (c + i < n) t[i] = row[base + c + i];
            }
            __builtin_memcpy(&raw[v], t, sizeof raw[v]);
        }
    }
}

// The fetched columns without those on the row's list (a NaN stays: no comparison holds for it); `bits` is LDS, one
// a column.  `there`: the row's user exists.  (Between fetch and here, a kernel finds out what to do with them.)
template <typename H, typename T>
__device__ __forceinline__ void take_columns(H& h, const Four<T> (&raw)[H::kScores / 4], uint32_t base, uint32_t n,
                                             const Rated& rated, int64_t r, uint32_t* bits, bool* there) {
    constexpr int K = H::kScores;
    const int32_t* list;
    int64_t listed;
    *there = rated.row(r, &list, &listed);
    const bool some = *there && listed > 0;
    if (some) {
        for (uint32_t w = threadIdx.x; w < (n + 31) / 32; w += h.threads) bits[w] = 0;
        h.sync();
        for (int64_t k = threadIdx.x; k < listed; k += h.threads) {
            const uint32_t c = (uint32_t)list[k] - base;
            if (c < n) atomicOr(&bits[c >> 5], 1u << (c & 31));
        }
        h.sync();
    }
#pragma unroll
    for (int v = 0; v < K / 4; ++v) {
        T t[4];
        __builtin_memcpy(t, &raw[v], sizeof t);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            h.z[v / 8][v % 8 * 4 + i] = to_float(t[i]);
        }
    }
    if (some) {
#pragma unroll
        for (int v = 0; v < K / 4; ++v) {
            const uint32_t c = h.position(v);
            const uint32_t four = c < n ? bits[c >> 5] >> (c & 31) & 15 : 0;
            if (four) {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    h.z[v / 8][v % 8 * 4 + i] = four >> i & 1 ? -INFINITY : h.z[v / 8][v % 8 * 4 + i];
            }
        }
        h.sync();
    }
}

// What row r asks for.
struct Wanted {
    float t, top_p, least, u;
    int top_k;
    __device__ __forceinline__ Wanted(const Limits& lim, const float* u_, int64_t r) {
        t = limit_of(lim.temperature, lim.temperature_all, r);
        top_p = limit_of(lim.top_p, lim.top_p_all, r);
        const float min_p = limit_of(lim.min_p, lim.min_p_all, r);
        least = min_p > 0.f ? fminf(min_p, 1.f) * 0x1p40f : 0.f;
        top_k = lim.top_k ? lim.top_k[r] : lim.top_k_all;
        u = unit_of(u_[r]);
    }
    __device__ __forceinline__ uint32_t part() const { return top_p > 0.f ? (uint32_t)(top_p * 0x1p24f) : 0; }
};

// The draw among held columns that are some columns of a row, `column` being theirs.
template <typename Few>
__device__ __forceinline__ void draw_held(Few& few, const uint32_t (&column)[Few::kScores], const Wanted& want,
                                          const Asked& ask, int64_t r, int32_t* index, float* log) {
    const auto d = few.draw(want, ask);
#pragma unroll
    for (int i = 0; i < Few::kScores; ++i)
        if (few.position(i / 4) + i % 4 == d.position) {
            index[r] = (int32_t)column[i];
            if (log) log[r] = d.log;
        }
}

// The draw among the columns on a list (in LDS, by column), by the workgroup's first `waves` waves.  The list's place is
// free once they have it.
template <typename Few, typename Shared>
__device__ __forceinline__ void draw_listed(Few few, Shared* sh, uint32_t count, int waves, const Wanted& want,
                                            const Asked& ask, int64_t r, int32_t* index, float* log) {
    constexpr int K = Few::kScores;
    static_assert(sizeof(typename Few::Shared) <= sizeof(Shared) && K <= 32, "the list's own place");
    few.sh = (typename Few::Shared*)sh;
    few.threads = waves * kWave;
    few.waves = waves;
    uint32_t column[K];
#pragma unroll
    for (int i = 0; i < K; ++i) {
        const uint32_t at = few.position(i / 4) + i % 4;
        few.z[0][i] = at < count ? sh->list_z[at] : -INFINITY;
        column[i] = at < count ? sh->list_position[at] : 0;
    }
    few.sync();
    draw_held(few, column, want, ask, r, index, log);
}

// A workgroup a row, the row in registers from its one read on.  1,024 x 17,770 fp32 scores (13.9 us of reading), us:
// the best column 21, temperature 44, top-k 200 48, with top-p 0.9 51, with 208 columns left out 58; top-p alone 97.
// Bound by vector instructions and by waits between a row's short passes: 15 instructions an exponential, about 30 a
// score and pass that weighs all of them; four to five waves a SIMD.
template <int K, int BINS, typename T>
__global__ __launch_bounds__(1024, K <= 8 ? 8 : (K <= 32 ? 6 : 4)) void k_sample(
    const T* __restrict__ z, int64_t row0, uint32_t n, int64_t ldz, Limits lim, const float* __restrict__ u, Rated rated,
    int32_t* __restrict__ index, float* __restrict__ log) {
    using H = Held<K, BINS>;
    extern __shared__ __align__(16) unsigned char shared[];
    H h;
    h.sh = (typename H::Shared*)shared;
    h.threads = blockDim.x;
    h.waves = blockDim.x / kWave;
    uint32_t* bits = (uint32_t*)(shared + sizeof(typename H::Shared));   // the columns left out, one bit each
    const int64_t r = row0 + blockIdx.x;
    bool there;
    Four<T> raw[K / 4];
    fetch_columns(h, z + r * ldz, 0, n, raw);
    take_columns<H, T>(h, raw, 0, n, rated, r, bits, &there);
    if (!there) {
        if (threadIdx.x == 0) { index[r] = -1; if (log) log[r] = NAN; }
        return;
    }
    float best;
    const float mine = h.largest(&best);
    if (!(best > -INFINITY)) {
        if (threadIdx.x == 0) { index[r] = -1; if (log) log[r] = -INFINITY; }
        return;
    }
    const Wanted want(lim, u, r);
    const int top_k = want.top_k;
    if (!(want.t > 0.f)) {
        const uint32_t p = h.first_of(best);
        if (threadIdx.x == 0) { index[r] = (int32_t)p; if (log) log[r] = 0.f; }
        return;
    }
    Asked ask(best, want.t, want.least);
    const bool odd = !ask.is_plain();
    h.plain(ask);
    // A few best columns are looked for among the few that reach a score which enough threads' largest ones reach:
    // the passes over the row are then two comparisons a score, and all else is done on a list.
    if (!odd && h.waves > 1 && top_k > 0 && top_k <= h.threads * 3 / 4) {
        const float reached = h.reached_by((uint32_t)top_k, best, [&](auto fn) { fn(mine); });
        const uint32_t most = H::kList;
        static_assert(H::kList <= 16 * kWave, "one wave holds the list");
        const uint32_t count = !(reached > -INFINITY) ? most + 1 : h.collect(
            most, [&](float v) { return v >= reached; },
            [&](uint32_t i, float v, uint32_t position) {
                h.sh->list_z[i] = v;
                h.sh->list_position[i] = position;
            });
        if (count <= most) {     // one wave: no barriers
            if (h.wave() != 0) return;
            if (count <= 512u) draw_listed(Held<8, 256>(), h.sh, count, 1, want, ask, r, index, log);
            else draw_listed(Held<16, 256>(), h.sh, count, 1, want, ask, r, index, log);
            return;
        }
    }
    const auto d = h.draw(want, ask);
    if (threadIdx.x == 0) { index[r] = (int32_t)d.position; if (log) log[r] = d.log; }
}

enum RowKind { kRowNone, kRowBest, kRowFew, kRowShare, kRowRest, kRowSlow };

// What a long row's kernels tell one another.
struct RowPlan {
    int kind;
    float best;
    int bin;                // the bin in which the cut falls,
    float from, to;         // and its scores: from <= z < to
    uint64_t before, goal;
};

struct SampleShared {
    uint64_t mass[kBins];
    uint32_t count[kBins];
    uint32_t list_d[kList];
    uint32_t list_i[kList];
    uint64_t wave64[kSampleWaves + 1];
    uint32_t wave_a[kSampleWaves], wave_b[kSampleWaves], wave_c[kSampleWaves];
    uint32_t found_bin, found_count, listed;
    uint64_t found_before;
    uint32_t cut_d, cut_i;
    uint64_t before;
    uint32_t bits[1];   // the columns left out, one bit each
};

// One row in the hands of one workgroup.
template <typename T>
struct Row {
    const T* z;
    int64_t n;
    const int32_t* rated;
    int64_t rated_count;
    SampleShared* sh;
    uint32_t best;      // the largest key
    Asked ask{0.f, 1.f, 0.f};
    bool odd, one_chunk;      // odd: the weights' formula does not hold

    // Marks the left-out columns of [c0, c1).
    __device__ void mark(int64_t c0, int64_t c1) {
        __syncthreads();
        for (int64_t w = threadIdx.x; w < (c1 - c0 + 31) / 32; w += kSampleThreads) sh->bits[w] = 0;
        __syncthreads();
        for (int64_t k = threadIdx.x; k < rated_count; k += kSampleThreads) {
            const int64_t c = rated[k];
            if (c >= c0 && c < c1) atomicOr(&sh->bits[(c - c0) >> 5], 1u << ((c - c0) & 31));
        }
        __syncthreads();
    }

    // fn(column, key) for every allowed column.
    template <typename Fn>
    __device__ void each(Fn fn) {
        for (int64_t c0 = 0; c0 < n; c0 += kChunk) {
            const int64_t c1 = c0 + kChunk < n ? c0 + kChunk : n;
            if (rated_count > 0 && !one_chunk) mark(c0, c1);
            for (int64_t c = c0 + threadIdx.x; c < c1; c += kSampleThreads) {
                const float v = to_float(z[c]);
                if (!(v > -INFINITY)) continue;
                if (rated_count > 0 && (sh->bits[(c - c0) >> 5] >> ((c - c0) & 31) & 1)) continue;
                fn(c, key_of(v));
            }
        }
    }

    __device__ float scaled(uint32_t d) const {
        return odd ? (d == 0 ? 0x1p40f : 0.f) : ask.scaled(score_of(best - d));
    }
    __device__ uint64_t weight_of(uint32_t d) const { return whole_of(floorf(scaled(d))); }
};

// Sums over the workgroup, to every thread.
__device__ uint64_t block_sum(uint64_t v, SampleShared* sh) {
    const uint64_t s = scan64(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 63) sh->wave64[threadIdx.x >> 6] = s;
    __syncthreads();
    uint64_t total = 0;
    for (int w = 0; w < kSampleWaves; ++w) total += sh->wave64[w];
    return total;
}

// A place in the order (score descending, column ascending): columns up to and with (d, column).
struct LongCut {
    uint32_t d;
    uint32_t column;
    __device__ bool keeps(uint32_t dd, int64_t c) const {
        return dd < d || (dd == d && (uint32_t)c <= column);
    }
};

// The first column, by column number, at which the running sum of measure(column, d) exceeds t (the sum
// over all columns does).
template <typename T, typename Fn>
__device__ uint32_t find_column(Row<T>& row, uint64_t t, Fn measure) {
    SampleShared* sh = row.sh;
    uint64_t before = 0;
    for (int64_t c0 = 0; c0 < row.n; c0 += kChunk) {
        const int64_t c1 = c0 + kChunk < row.n ? c0 + kChunk : row.n;
        if (row.rated_count > 0 && !row.one_chunk) row.mark(c0, c1);
        for (int64_t b0 = c0; b0 < c1; b0 += kSampleThreads) {
            const int64_t c = b0 + threadIdx.x;
            uint64_t v = 0;
            if (c < c1) {
                const float z = to_float(row.z[c]);
                if (z > -INFINITY &&
                    !(row.rated_count > 0 && (sh->bits[(c - c0) >> 5] >> ((c - c0) & 31) & 1)))
                    v = measure(c, row.best - key_of(z));
            }
            const uint64_t s = scan64(v);
            __syncthreads();
            if ((threadIdx.x & 63) == 63) sh->wave64[threadIdx.x >> 6] = s;
            if (threadIdx.x == 0) sh->cut_i = 0xFFFFFFFFu;
            __syncthreads();
            uint64_t mine = before;
            for (int w = 0; w < kSampleWaves; ++w) {
                if (w == (int)(threadIdx.x >> 6)) mine = before;
                before += sh->wave64[w];
            }
            if (v > 0 && mine + s > t && mine + s - v <= t) sh->cut_i = (uint32_t)c;
            __syncthreads();
            if (sh->cut_i != 0xFFFFFFFFu) return sh->cut_i;
        }
    }
    return 0xFFFFFFFFu;
}

// The last column, in the order, with less than `target` of the measure before it; among the columns that
// `within` keeps.  BY_MASS: the measure is the weight, else 1.  target >= 1 and at most the sum.
template <bool BY_MASS, typename T>
__device__ LongCut select_cut(Row<T>& row, LongCut within, uint32_t widest, uint64_t target) {
    SampleShared* sh = row.sh;
    uint64_t before = 0;                       // measure in front of the range
    uint32_t lo = 0, hi = widest;              // the range of distances
    for (;;) {
        int shift = 0;
        while (((hi - lo) >> shift) >= kBins) ++shift;
        __syncthreads();
        for (int b = threadIdx.x; b < kBins; b += kSampleThreads) { sh->mass[b] = 0; sh->count[b] = 0; }
        __syncthreads();
        row.each([&](int64_t c, uint32_t key) {
            const uint32_t d = row.best - key;
            if (d < lo || d > hi || !within.keeps(d, c)) return;
            const uint32_t b = (d - lo) >> shift;
            atomicAdd(&sh->count[b], 1u);
            if (BY_MASS) {
                const uint64_t w = row.weight_of(d);
                if (w) atomicAdd((unsigned long long*)&sh->mass[b], (unsigned long long)w);
            }
        });
        __syncthreads();
        // the bin in which the measure reaches the target: two bins a thread
        const int b = 2 * threadIdx.x;
        const uint64_t v0 = BY_MASS ? sh->mass[b] : sh->count[b], v1 = BY_MASS ? sh->mass[b + 1] : sh->count[b + 1];
        const uint64_t s = scan64(v0 + v1);
        if ((threadIdx.x & 63) == 63) sh->wave64[threadIdx.x >> 6] = s;
        __syncthreads();
        uint64_t at = before;
        for (int w = 0; w < (int)(threadIdx.x >> 6); ++w) at += sh->wave64[w];
        at += s - (v0 + v1);
        if (at < target && target <= at + v0) {
            sh->found_bin = b; sh->found_before = at; sh->found_count = sh->count[b];
        } else if (at + v0 < target && target <= at + v0 + v1) {
            sh->found_bin = b + 1; sh->found_before = at + v0; sh->found_count = sh->count[b + 1];
        }
        if (threadIdx.x == 0) sh->listed = 0;
        __syncthreads();
        before = sh->found_before;
        lo = lo + (sh->found_bin << shift);
        const uint32_t end = shift ? lo + ((1u << shift) - 1) : lo;
        hi = end < hi && end >= lo ? end : hi;
        const uint32_t count = sh->found_count;
        if (count <= kList) {
            row.each([&](int64_t c, uint32_t key) {
                const uint32_t d = row.best - key;
                if (d < lo || d > hi || !within.keeps(d, c)) return;
                const uint32_t at = atomicAdd(&sh->listed, 1u);
                sh->list_d[at] = d;
                sh->list_i[at] = (uint32_t)c;
            });
            __syncthreads();
            if (threadIdx.x < count) {
                const uint32_t d = sh->list_d[threadIdx.x], i = sh->list_i[threadIdx.x];
                uint64_t front = before;
                for (uint32_t k = 0; k < count; ++k) {
                    const uint32_t dk = sh->list_d[k];
                    if (dk < d || (dk == d && sh->list_i[k] < i)) front += BY_MASS ? row.weight_of(dk) : 1;
                }
                const uint64_t own = BY_MASS ? row.weight_of(d) : 1;
                if (front < target && target <= front + own) { sh->cut_d = d; sh->cut_i = i; }
            }
            __syncthreads();
            const LongCut cut{sh->cut_d, sh->cut_i};
            __syncthreads();
            return cut;
        }
        if (lo == hi) {    // equal scores: as many of them, by column, as reach the target
            const uint64_t own = BY_MASS ? row.weight_of(lo) : 1;
            const uint64_t keep = (target - before + own - 1) / own;
            const uint32_t d = lo;
            const uint32_t c = find_column(row, keep - 1, [&](int64_t cc, uint32_t dd) -> uint64_t {
                return dd == d && within.keeps(dd, cc) ? 1 : 0;
            });
            __syncthreads();
            return LongCut{d, c};
        }
    }
}

// Rows that no workgroup's registers hold, in segments of 16,384 columns, a workgroup each; what the segments find
// out goes through the workspace from one kernel to the next, and each kernel reads the scores again
// (from the cache that all dies share, where they fit it):
//   k_long_stats  a segment's best and (nearly) least score, and the best scores of groups of its columns
//   k_long_parts  top-k: the segment's columns with a score that k groups' best ones reach; top-p: a histogram of
//                 weights over the row's scores; neither: the segment's weight
//   k_long_rows   a workgroup a row.  top-k: the draw, among what the segments listed; top-p: the bin in which the cut
//                 falls; neither: the draw
//   k_long_cut    top-p: the segment's columns in that bin, and the weight of those above it
//   k_long_draw   top-p: the cut, by ranking the listed columns, and the draw
// Rows whose lists do not hold what they should are drawn by the last of these kernels alone, one workgroup that reads
// the row again for every pass (sample_slowly): with a top_k above 7/8 of the groups (2,184 of 2,496 groups at 625,000
// columns, 2,240 at 70,000, 3,584 at most); a top_k whose best columns stand side by side (sorted rows: over 2,048
// listed in one segment); over 2,048 columns of a segment, or 16,384 of the row, in the bin of a top-p cut (bf16 scores
// close to one another); a best score of +inf.
// 64 x 625,000 bf16 scores (15.3 us of reading), us: the best column 33, temperature 61, top-k 200 66, top-p 0.9 149
// (two sets of inputs in turn; 132 over one), by kernel 19 (memory), 45 (vector instructions: a weight a score), 13 (a
// workgroup a row: waits), 37 and 39 (waits).  By sample_slowly, 1 and 64 such rows: top-k 5,000 930 and 1,980; sorted
// fp32 rows with top-k 200 1,030 and 1,560; scores of 4 +- 0.2 with top-p 0.9 2,120 and 2,930; +inf in fp32 300 and 560.
constexpr int kSegWaves = 8, kSegThreads = kSegWaves * kWave, kSegColumns = kSegThreads * 32;
constexpr int kSegMax = ALS_SERVE_N_MAX / kSegColumns;
constexpr int kSlab = 2048;              // columns a segment lists
constexpr int kFew = 16384;              // columns a row's workgroup takes from its lists
constexpr int kGroups = 4096;            // most groups of a row
using Segment = Held<32, 1024>;
using FewOfRow = Held<16, 2048>;
using SegmentOfRow = Held<16, 2048>;      // (more waves than the segment's own workgroup)
constexpr int kRowThreads = kFew / 16;
static_assert(kSegColumns <= 16 * kRowThreads, "a segment in a row's workgroup");
static_assert(kSegMax <= kSegThreads && kSegMax <= kRowThreads && kRowThreads == kSampleThreads, "a thread a segment");

struct SegStat {
    float best, least;      // the least: near it
    uint64_t mass;
    uint32_t listed;
};
// A batch's part of the workspace.  Segment s of the batch's row b is number b segments + s.
struct LongWork {
    RowPlan* plan;
    SegStat* stat;
    float* groups;              // kSegThreads / group a segment
    uint64_t* bins;             // Segment::kBins a segment
    float* list_z;              // kSlab a segment
    uint32_t* list_column;
    uint32_t segments, group;   // group: threads (of 32 columns each) that publish one best score
    int64_t row0;               // the batch's first row
};
template <typename T>
struct LongArgs {
    const T* z;
    int64_t n, ldz;
    Limits lim;
    const float* u;
    Rated rated;
    int32_t* index;
    float* log;
    LongWork work;
    __device__ __forceinline__ uint32_t columns(uint32_t seg) const {
        const int64_t left = n - (int64_t)seg * kSegColumns;
        return left < kSegColumns ? (uint32_t)left : kSegColumns;
    }
};

// A whole row by one workgroup of kSampleThreads, which reads it again for every pass.
template <typename T>
__device__ __forceinline__ void sample_slowly(const LongArgs<T>& a, int64_t r, unsigned char* shared) {
    SampleShared* sh = (SampleShared*)shared;
    const Limits& lim = a.lim;
    const float* u = a.u;
    int32_t* index = a.index;
    float* log = a.log;
    Row<T> row;
    row.z = a.z + r * a.ldz;
    row.n = a.n;
    row.sh = sh;
    row.one_chunk = a.n <= kChunk;
    if (!a.rated.row(r, &row.rated, &row.rated_count)) return;     // (has no allowed column, and is not slow)
    __syncthreads();
    if (row.rated_count > 0 && row.one_chunk) row.mark(0, a.n);
    // the largest and the least key, and the number of allowed columns
    uint32_t hi = 0, lo = 0xFFFFFFFFu, count = 0;
    row.each([&](int64_t, uint32_t key) { hi = max(hi, key); lo = min(lo, key); ++count; });
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) {
        hi = max(hi, (uint32_t)__shfl_xor(hi, d));
        lo = min(lo, (uint32_t)__shfl_xor(lo, d));
        count += __shfl_xor(count, d);
    }
    __syncthreads();
    if ((threadIdx.x & 63) == 0) {
        const int w = threadIdx.x >> 6;
        sh->wave_a[w] = hi; sh->wave_b[w] = lo; sh->wave_c[w] = count;
    }
    __syncthreads();
    hi = 0; lo = 0xFFFFFFFFu; count = 0;
    for (int w = 0; w < kSampleWaves; ++w) {
        hi = max(hi, sh->wave_a[w]); lo = min(lo, sh->wave_b[w]); count += sh->wave_c[w];
    }
    if (count == 0) {
        if (threadIdx.x == 0) { index[r] = -1; if (log) log[r] = -INFINITY; }
        return;
    }
    const Wanted want(lim, u, r);
    const bool greedy = !(want.t > 0.f);
    row.best = hi;
    row.ask = Asked(score_of(hi), greedy ? 1.f : want.t, want.least);
    row.odd = !row.ask.is_plain();
    const int k = want.top_k;
    const uint32_t widest = hi - lo;
    LongCut cut{widest, 0xFFFFFFFFu};
    if (greedy) {
        const uint32_t c = find_column(row, 0, [](int64_t, uint32_t d) -> uint64_t { return d == 0; });
        if (threadIdx.x == 0) { index[r] = (int32_t)c; if (log) log[r] = 0.f; }
        return;
    }
    if (k > 0 && (uint32_t)k < count) cut = select_cut<false>(row, cut, cut.d, (uint64_t)k);
    if (want.top_p < 1.f) {
        uint64_t sum = 0;
        row.each([&](int64_t c, uint32_t key) {
            if (cut.keeps(hi - key, c)) sum += row.weight_of(hi - key);
        });
        sum = block_sum(sum, sh);
        uint64_t target = share_of(sum, want.part());
        if (target < 1) target = 1;
        cut = select_cut<true>(row, cut, cut.d, target);
    }
    auto weight = [&](int64_t c, uint32_t d) -> uint64_t {
        if (!cut.keeps(d, c)) return 0;
        const float e = row.scaled(d);
        return e >= want.least ? whole_of(floorf(e)) : 0;
    };
    uint64_t sum = 0;
    row.each([&](int64_t c, uint32_t key) { sum += weight(c, hi - key); });
    sum = block_sum(sum, sh);
    const uint32_t c = find_column(row, share_of(sum, (uint32_t)(want.u * 0x1p24f)), weight);
    if (threadIdx.x == 0) {
        index[r] = (int32_t)c;
        if (log) {
            const float v = to_float(row.z[c]);
            const float x = row.odd ? 0.f : (v - row.ask.top) * row.ask.inv_t;
            log[r] = x - logf((float)sum * 0x1p-40f);
        }
    }
}


// Best and (nearly) least score of a row, from its segments; by the whole workgroup.
template <typename H>
__device__ __forceinline__ void row_stats(H& h, const SegStat* stat, uint32_t segments, float* best, float* least) {
    const bool mine = threadIdx.x < segments;
    float hi = mine ? stat[threadIdx.x].best : -INFINITY, lo = mine ? -stat[threadIdx.x].least : -INFINITY;
    hi = wave_max(hi);
    lo = wave_max(lo);
    if (h.lane() == 0) { h.sh->wave_a[h.wave()] = hi; h.sh->wave_b[h.wave()] = lo; }
    h.sync();
    hi = lo = -INFINITY;
    for (int w = 0; w < h.waves; ++w) {
        hi = fmaxf(hi, h.sh->wave_a[w]);
        lo = fmaxf(lo, h.sh->wave_b[w]);
    }
    h.sync();
    *best = hi;
    *least = -lo;
}

__device__ __forceinline__ int kind_of(const Wanted& want, float best, int64_t n, uint32_t groups) {
    if (!(best > -INFINITY)) return kRowNone;
    if (!(want.t > 0.f)) return kRowBest;
    if (!Asked(best, want.t, 0.f).is_plain()) return kRowSlow;
    if (want.top_k > 0 && want.top_k < n) return (uint32_t)want.top_k <= groups / 8 * 7 ? kRowFew : kRowSlow;
    return want.top_p < 1.f ? kRowShare : kRowRest;
}

template <typename T>
__global__ __launch_bounds__(kSegThreads, 8) void k_long_stats(LongArgs<T> a) {
    __shared__ Segment::Shared sh;
    __shared__ uint32_t bits[kSegColumns / 32];
    Segment h;
    h.sh = &sh;
    h.threads = kSegThreads;
    h.waves = kSegWaves;
    const LongWork& w = a.work;
    const uint32_t b = blockIdx.x / w.segments, seg = blockIdx.x % w.segments;
    const int64_t r = w.row0 + b;
    bool there;
    Four<T> raw[Segment::kScores / 4];
    fetch_columns(h, a.z + r * a.ldz, seg * kSegColumns, a.columns(seg), raw);
    take_columns<Segment, T>(h, raw, seg * kSegColumns, a.columns(seg), a.rated, r, bits, &there);
    float best;
    float mine = h.largest(&best);
    const float least = h.near_least();
    if (threadIdx.x == 0) {
        SegStat& s = w.stat[blockIdx.x];
        s.best = there ? best : -INFINITY;
        s.least = least;
    }
    for (uint32_t d = 1; d < w.group; d <<= 1) mine = fmaxf(mine, __shfl_xor(mine, d));
    if (threadIdx.x % w.group == 0)
        w.groups[(int64_t)blockIdx.x * (kSegThreads / w.group) + threadIdx.x / w.group] = mine;
}

template <typename T>
__global__ __launch_bounds__(kSegThreads) void k_long_parts(LongArgs<T> a) {
    __shared__ Segment::Shared sh;
    __shared__ uint32_t bits[kSegColumns / 32];
    Segment h;
    h.sh = &sh;
    h.threads = kSegThreads;
    h.waves = kSegWaves;
    const LongWork& w = a.work;
    const uint32_t b = blockIdx.x / w.segments, seg = blockIdx.x % w.segments;
    const int64_t r = w.row0 + b;
    Four<T> raw[Segment::kScores / 4];
    fetch_columns(h, a.z + r * a.ldz, seg * kSegColumns, a.columns(seg), raw);
    float best, least;
    row_stats(h, w.stat + (int64_t)b * w.segments, w.segments, &best, &least);
    const Wanted want(a.lim, a.u, r);
    const uint32_t per = kSegThreads / w.group, groups = w.segments * per;
    const int kind = kind_of(want, best, a.n, groups);
    if (kind != kRowFew && kind != kRowShare && kind != kRowRest) return;
    Asked ask(best, want.t, want.least);
    bool there;
    take_columns<Segment, T>(h, raw, seg * kSegColumns, a.columns(seg), a.rated, r, bits, &there);
    if (kind == kRowFew) {
        const float* all = w.groups + (int64_t)b * groups;
        float z[kGroups / kSegThreads];
#pragma unroll
        for (int i = 0; i < kGroups / kSegThreads; ++i) {
            const uint32_t at = i * kSegThreads + threadIdx.x;
            z[i] = at < groups ? all[at] : -INFINITY;
        }
        const float reached = h.reached_by((uint32_t)want.top_k, best, [&](auto fn) {
#pragma unroll
            for (int i = 0; i < kGroups / kSegThreads; ++i) fn(z[i]);
        });
        // (fewer than k groups hold an allowed column: the list cannot be told to be long enough)
        const uint32_t listed = !(reached > -INFINITY) ? kSlab + 1 : h.collect(
            kSlab, [&](float v) { return v >= reached; },
            [&](uint32_t i, float v, uint32_t position) {
                w.list_z[(int64_t)blockIdx.x * kSlab + i] = v;
                w.list_column[(int64_t)blockIdx.x * kSlab + i] = seg * kSegColumns + position;
            });
        if (threadIdx.x == 0) w.stat[blockIdx.x].listed = listed;
    } else if (kind == kRowShare) {
        for (int i = threadIdx.x; i < Segment::kBins; i += kSegThreads) sh.bin[i] = 0;
        h.sync();
        bool clipped;
        const auto scale = Segment::scale_of(best, least, want.t, &clipped);
        h.each([&](float v, uint32_t) {
            if (v > -INFINITY) h.add_to_bin(h.bin_of(v, scale), true, v, ask);
        });
        h.sync();
        for (int i = threadIdx.x; i < Segment::kBins; i += kSegThreads)
            w.bins[(int64_t)blockIdx.x * Segment::kBins + i] = sh.bin[i];
    } else {
        double thread = 0.0;
        h.each([&](float v, uint32_t) {
            const float e = ask.scaled(v);
            thread += v > -INFINITY && e >= ask.least ? (double)floorf(e) : 0.0;
        });
        uint64_t before;
        const uint64_t mass = h.sum(last64(scan64(whole_of(thread))), &before);
        if (threadIdx.x == 0) w.stat[blockIdx.x].mass = mass;
    }
}

struct RowShared {
    SegmentOfRow::Shared held;
    uint32_t first[kSegMax + 1];         // of a segment's list, on the row's
    uint64_t mass[kSegMax];
    uint32_t bits[kSegColumns / 32];
    uint32_t found, cut_column;
    float cut_z;
    uint64_t before;
};
static_assert(sizeof(FewOfRow::Shared) == sizeof(SegmentOfRow::Shared), "one place for both");

// Where the segments' lists lie on the row's; false: some list, or all of them, are too long.
template <typename H>
__device__ __forceinline__ bool place_lists(H& h, const SegStat* stat, uint32_t segments, RowShared* sh) {
    const uint32_t mine = threadIdx.x < segments ? stat[threadIdx.x].listed : 0;
    const float longest = wave_max((float)mine);
    const uint64_t upto = scan64(mine);
    h.sync();
    if (h.lane() == 63) { sh->held.wave_sum[h.wave()] = upto; sh->held.wave_a[h.wave()] = longest; }
    h.sync();
    uint64_t before = 0, total = 0;
    bool fits = true;
    for (int w = 0; w < h.waves; ++w) {
        if (w == h.wave()) before = total;
        total += sh->held.wave_sum[w];
        fits = fits && sh->held.wave_a[w] <= (float)kSlab;
    }
    if (threadIdx.x < segments) sh->first[threadIdx.x] = (uint32_t)(before + upto - mine);
    if (threadIdx.x == segments) sh->first[segments] = (uint32_t)total;
    h.sync();
    return fits && total <= (uint64_t)kFew;
}

// The row's listed columns, by column, four neighbours a thread and time; `column` are theirs.
template <typename Few>
__device__ __forceinline__ void take_lists(Few& few, const LongWork& w, uint32_t b, const RowShared* sh,
                                           uint32_t (&column)[Few::kScores]) {
    const uint32_t total = sh->first[w.segments];
#pragma unroll
    for (int v = 0; v < Few::kScores / 4; ++v)
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            const uint32_t i = few.position(v) + c;
            float z = -INFINITY;
            uint32_t at = 0;
            if (i < total) {
                uint32_t lo = 0, hi = w.segments;      // the last segment whose list starts at or before i
                while (hi - lo > 1) {
                    const uint32_t mid = (lo + hi) / 2;
                    if (sh->first[mid] <= i) lo = mid;
                    else hi = mid;
                }
                const int64_t from = ((int64_t)b * w.segments + lo) * kSlab + (i - sh->first[lo]);
                z = w.list_z[from];
                at = w.list_column[from];
            }
            few.z[0][4 * v + c] = z;
            column[4 * v + c] = at;
        }
}

// The row's listed columns into LDS, by column (there are at most kList).
__device__ __forceinline__ void gather_lists(const LongWork& w, uint32_t b, RowShared* sh) {
    for (uint32_t seg = threadIdx.x / kWave; seg < w.segments; seg += kRowThreads / kWave) {
        const uint32_t first = sh->first[seg], count = sh->first[seg + 1] - first;
        const int64_t from = ((int64_t)b * w.segments + seg) * kSlab;
        for (uint32_t i = threadIdx.x % kWave; i < count; i += kWave) {
            sh->held.list_z[first + i] = w.list_z[from + i];
            sh->held.list_position[first + i] = w.list_column[from + i];
        }
    }
    __syncthreads();
}

// The draw from the segments' weights (sh->mass), the columns being those that `cut` (by column) keeps.
template <typename T>
__device__ __forceinline__ void draw_from_segments(SegmentOfRow& h, const LongArgs<T>& a, uint32_t b, const Wanted& want,
                                                   const Asked& ask, const Cut& cut, RowShared* sh) {
    const LongWork& w = a.work;
    const int64_t r = w.row0 + b;
    h.sync();
    const uint64_t mine = threadIdx.x < w.segments ? sh->mass[threadIdx.x] : 0;
    const uint64_t upto = scan64(mine);
    uint64_t before;
    const uint64_t total = h.sum(last64(upto), &before);
    const uint64_t t = share_of(total, (uint32_t)(want.u * 0x1p24f)), at = before + upto - mine;
    if (t >= at && t - at < mine) { sh->found = threadIdx.x; sh->before = at; }
    h.sync();
    const uint32_t seg = sh->found, base = seg * kSegColumns;
    bool there;
    Four<T> raw[SegmentOfRow::kScores / 4];
    fetch_columns(h, a.z + r * a.ldz, base, a.columns(seg), raw);
    take_columns<SegmentOfRow, T>(h, raw, base, a.columns(seg), a.rated, r, sh->bits, &there);
    const auto weight = [&](float k, uint32_t p) {
        const float e = ask.scaled(k);
        return cut.keeps(k, base + p) && e >= ask.least ? floorf(e) : 0.f;
    };
    double thread = 0.0;
    h.each([&](float k, uint32_t p) { thread += (double)weight(k, p); });
    const uint64_t of_wave = last64(scan64(whole_of(thread)));
    uint64_t before_wave;
    h.sum(of_wave, &before_wave);
    const uint32_t p = h.find(t - sh->before, of_wave, before_wave, weight);
    h.each([&](float k, uint32_t i) {
        if (i == p) {
            a.index[r] = (int32_t)(base + p);
            const float x = (k - ask.top) * ask.inv_t;
            if (a.log) a.log[r] = x - logf((float)total * 0x1p-40f);
        }
    });
}

template <typename T>
__global__ __launch_bounds__(kRowThreads) void k_long_rows(LongArgs<T> a) {
    extern __shared__ __align__(16) unsigned char shared[];
    RowShared* sh = (RowShared*)shared;
    SegmentOfRow h;
    h.sh = &sh->held;
    h.threads = kRowThreads;
    h.waves = kRowThreads / kWave;
    const LongWork& w = a.work;
    const uint32_t b = blockIdx.x;
    const int64_t r = w.row0 + b;
    const SegStat* stat = w.stat + (int64_t)b * w.segments;
    float best, least;
    row_stats(h, stat, w.segments, &best, &least);
    const Wanted want(a.lim, a.u, r);
    int kind = kind_of(want, best, a.n, w.segments * (kSegThreads / w.group));
    Asked ask(best, want.t, want.least);
    RowPlan plan{kind, best, 0, 0.f, 0.f, 0, 0};
    if (kind == kRowNone) {
        const int32_t* list;
        int64_t listed;
        if (threadIdx.x == 0) {
            a.index[r] = -1;
            if (a.log) a.log[r] = a.rated.row(r, &list, &listed) ? -INFINITY : NAN;
        }
    } else if (kind == kRowBest) {
        if (threadIdx.x == 0) sh->found = w.segments;
        h.sync();
        if (threadIdx.x < w.segments && stat[threadIdx.x].best == best) atomicMin(&sh->found, threadIdx.x);
        h.sync();
        const uint32_t seg = sh->found;
        bool there;
        Four<T> raw[SegmentOfRow::kScores / 4];
        fetch_columns(h, a.z + r * a.ldz, seg * kSegColumns, a.columns(seg), raw);
        take_columns<SegmentOfRow, T>(h, raw, seg * kSegColumns, a.columns(seg), a.rated, r, sh->bits, &there);
        const uint32_t p = h.first_of(best);
        if (threadIdx.x == 0) { a.index[r] = (int32_t)(seg * kSegColumns + p); if (a.log) a.log[r] = 0.f; }
    } else if (kind == kRowFew) {
        if (!place_lists(h, stat, w.segments, sh)) {
            kind = kRowSlow;
        } else if (sh->first[w.segments] <= (uint32_t)SegmentOfRow::kList) {
            gather_lists(w, b, sh);
            if (h.wave() == 0)
                draw_listed(Held<16, 256>(), &sh->held, sh->first[w.segments], 1, want, ask, r, a.index, a.log);
        } else {
            FewOfRow few;
            few.sh = (FewOfRow::Shared*)&sh->held;
            few.threads = h.threads;
            few.waves = h.waves;
            uint32_t column[FewOfRow::kScores];
            take_lists(few, w, b, sh, column);
            draw_held(few, column, want, ask, r, a.index, a.log);
        }
    } else if (kind == kRowShare) {
        // the segments' histograms: two bins a thread, every second segment
        for (int i = threadIdx.x; i < SegmentOfRow::kBins; i += kRowThreads) sh->held.bin[i] = 0;
        h.sync();
        constexpr uint32_t kHalf = Segment::kBins / 2;
        static_assert(kRowThreads == 2 * kHalf, "two bins a thread");
        const uint32_t i = threadIdx.x % kHalf;
        const ulonglong2* two = (const ulonglong2*)(w.bins + (int64_t)b * w.segments * Segment::kBins) + i;
        uint64_t s0 = 0, s1 = 0;
#pragma unroll 10
        for (uint32_t seg = threadIdx.x / kHalf; seg < w.segments; seg += 2) {
            const ulonglong2 v = two[(int64_t)seg * kHalf];
            s0 += v.x;
            s1 += v.y;
        }
        if (s0) atomicAdd((unsigned long long*)&sh->held.bin[2 * i], (unsigned long long)s0);
        if (s1) atomicAdd((unsigned long long*)&sh->held.bin[2 * i + 1], (unsigned long long)s1);
        h.search_bins([&](uint64_t total) {
            const uint64_t goal = share_of(total, want.part());
            plan.goal = goal < 1 ? 1 : goal;
            return plan.goal;
        });
        bool clipped;
        const auto scale = Segment::scale_of(best, least, want.t, &clipped);
        Segment bins;
        const int bin = (int)sh->held.found_bin;
        plan.bin = bin;
        plan.from = bins.least_of_bins(bin, scale);
        plan.to = bin == 0 ? INFINITY : bins.least_of_bins(bin - 1, scale);
        plan.before = sh->held.found_before;
    } else if (kind == kRowRest) {
        if (threadIdx.x < w.segments) sh->mass[threadIdx.x] = stat[threadIdx.x].mass;
        draw_from_segments(h, a, b, want, ask, Cut(), sh);
    }
    if (kind == kRowSlow) sample_slowly(a, r, shared);
    if (threadIdx.x == 0) w.plan[b] = plan;
}

template <typename T>
__global__ __launch_bounds__(kSegThreads) void k_long_cut(LongArgs<T> a) {
    __shared__ Segment::Shared sh;
    __shared__ uint32_t bits[kSegColumns / 32];
    Segment h;
    h.sh = &sh;
    h.threads = kSegThreads;
    h.waves = kSegWaves;
    const LongWork& w = a.work;
    const uint32_t b = blockIdx.x / w.segments, seg = blockIdx.x % w.segments;
    const int64_t r = w.row0 + b;
    Four<T> raw[Segment::kScores / 4];
    fetch_columns(h, a.z + r * a.ldz, seg * kSegColumns, a.columns(seg), raw);
    const RowPlan plan = w.plan[b];
    if (plan.kind != kRowShare) return;
    const Wanted want(a.lim, a.u, r);
    Asked ask(plan.best, want.t, want.least);
    bool there;
    take_columns<Segment, T>(h, raw, seg * kSegColumns, a.columns(seg), a.rated, r, bits, &there);
    const auto above = [&](float v) { return v >= plan.to; };
    const uint32_t listed = h.collect(
        kSlab, [&](float v) { return v >= plan.from && !above(v); },
        [&](uint32_t i, float v, uint32_t position) {
            w.list_z[(int64_t)blockIdx.x * kSlab + i] = v;
            w.list_column[(int64_t)blockIdx.x * kSlab + i] = seg * kSegColumns + position;
        });
    // the weight above the bin is in the histogram, unless min_p takes some of it
    uint64_t thread = 0;
    if (plan.bin == 0 || ask.scaled(plan.to) >= ask.least) {
        for (int i = threadIdx.x; i < plan.bin; i += kSegThreads)
            thread += w.bins[(int64_t)blockIdx.x * Segment::kBins + i];
    } else {
        double sum = 0.0;
        h.each([&](float v, uint32_t) {
            if (above(v)) {
                const float e = ask.scaled(v);
                sum += e >= ask.least ? (double)floorf(e) : 0.0;
            }
        });
        thread = whole_of(sum);
    }
    uint64_t before;
    const uint64_t mass = h.sum(last64(scan64(thread)), &before);
    if (threadIdx.x == 0) {
        w.stat[blockIdx.x].listed = listed;
        w.stat[blockIdx.x].mass = mass;
    }
}

// The cut among the segments' listed columns (of the bin in which it falls), by the workgroup's first `waves` waves.
template <typename Few, typename T>
__device__ __forceinline__ void cut_listed(Few few, const LongArgs<T>& a, uint32_t b, const Asked& ask,
                                           const RowPlan& plan, int waves, RowShared* sh) {
    few.sh = (typename Few::Shared*)&sh->held;
    few.threads = waves * kWave;
    few.waves = waves;
    uint32_t column[Few::kScores];
    if (waves == 1) {
        const uint32_t count = sh->first[a.work.segments];
#pragma unroll
        for (int i = 0; i < Few::kScores; ++i) {
            const uint32_t at = few.position(i / 4) + i % 4;
            few.z[0][i] = at < count ? sh->held.list_z[at] : -INFINITY;
            column[i] = at < count ? sh->held.list_position[at] : 0;
        }
        few.sync();
    } else {
        take_lists(few, a.work, b, sh, column);
    }
    const Cut place = few.select(true, Cut(), few.near_least(), 0, ask, plan.goal - plan.before);
#pragma unroll
    for (int i = 0; i < Few::kScores; ++i) {
        const float k = few.z[0][i];
        const uint32_t at = few.position(i / 4) + i % 4;
        if (at == (uint32_t)place.position) { sh->cut_column = column[i]; sh->cut_z = place.z; }
        if (place.keeps(k, at)) {
            const float e = ask.scaled(k);
            if (e >= ask.least)
                atomicAdd((unsigned long long*)&sh->mass[column[i] / kSegColumns],
                          (unsigned long long)whole_of(floorf(e)));
        }
    }
}

template <typename T>
__global__ __launch_bounds__(kRowThreads) void k_long_draw(LongArgs<T> a) {
    extern __shared__ __align__(16) unsigned char shared[];
    RowShared* sh = (RowShared*)shared;
    SegmentOfRow h;
    h.sh = &sh->held;
    h.threads = kRowThreads;
    h.waves = kRowThreads / kWave;
    const LongWork& w = a.work;
    const uint32_t b = blockIdx.x;
    const int64_t r = w.row0 + b;
    const RowPlan plan = w.plan[b];
    if (plan.kind != kRowShare) return;
    const SegStat* stat = w.stat + (int64_t)b * w.segments;
    const Wanted want(a.lim, a.u, r);
    Asked ask(plan.best, want.t, want.least);
    if (!place_lists(h, stat, w.segments, sh)) {
        sample_slowly(a, r, shared);
        return;
    }
    if (threadIdx.x < w.segments) sh->mass[threadIdx.x] = stat[threadIdx.x].mass;
    h.sync();
    // the cut, by column; what it keeps of the lists counts for its segments
    if (sh->first[w.segments] <= (uint32_t)SegmentOfRow::kList) {
        gather_lists(w, b, sh);
        if (h.wave() == 0) cut_listed(Held<16, 256>(), a, b, ask, plan, 1, sh);
    } else {
        cut_listed(FewOfRow(), a, b, ask, plan, h.waves, sh);
    }
    h.sync();
    Cut cut;
    cut.z = sh->cut_z;
    cut.position = (int)sh->cut_column;
    draw_from_segments(h, a, b, want, ask, cut, sh);
}

// ---------------------------------------------------------------------------------- host --

bool aligned(const void* p, size_t a) { return ((uintptr_t)p & (a - 1)) == 0; }

size_t type_bytes(int dtype) { return dtype == ALS_F32 ? 4 : 2; }

// Bytes from the first element of a strided matrix to past its last.
uint64_t span_of(int64_t rows, int64_t cols, int64_t ld, size_t bytes) {
    return rows <= 0 || cols <= 0 ? 0 : ((uint64_t)(rows - 1) * (uint64_t)ld + (uint64_t)cols) * bytes;
}

bool overlap(const void* a, uint64_t an, const void* b, uint64_t bn) {
    if (!a || !b || an == 0 || bn == 0) return false;
    const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
    return x < y + bn && y < x + an;
}

struct DeviceGuard {
    int prev = -1;
    bool ok = false;
    explicit DeviceGuard(int dev) {
        if (hipGetDevice(&prev) != hipSuccess) prev = -1;
        ok = (prev == dev) || hipSetDevice(dev) == hipSuccess;
    }
    ~DeviceGuard() {
        int cur = -1;
        if (prev >= 0 && hipGetDevice(&cur) == hipSuccess && cur != prev) (void)hipSetDevice(prev);
    }
};

// What a device is: asked for once per device and process.
constexpr int kMaxDevices = 64;
struct DeviceInfo {
    std::mutex mu;
    bool known = false;
    int cus = 0;
};
DeviceInfo g_device[kMaxDevices];

int query_device(int device, int* cus) {
    int count = 0;
    if (hipGetDeviceCount(&count) != hipSuccess || device < 0 || device >= count || device >= kMaxDevices)
        return ALS_ERR_DEVICE;
    DeviceInfo& d = g_device[device];
    std::lock_guard<std::mutex> lock(d.mu);
    if (!d.known) {
        hipDeviceProp_t prop;
        if (hipGetDeviceProperties(&prop, device) != hipSuccess) return ALS_ERR_DEVICE;
        if (strncmp(prop.gcnArchName, "gfx950", 6) != 0) return ALS_ERR_DEVICE;
        d.cus = prop.multiProcessorCount;
        d.known = true;
    }
    *cus = d.cus;
    return ALS_OK;
}

constexpr size_t kWorkspaceBytes = 128u << 20, kWorkspaceMost = (size_t)1 << 34;   // (what a launch can walk)

}  // namespace

struct als_serve_ctx {
    int device;
    int cus;
    unsigned char* ws;
    size_t ws_bytes;
    int last_hip;
};

namespace {

// Lets a kernel use all of a CU's LDS; once per kernel and device.
template <typename Kernel>
void whole_lds(Kernel kernel, int device, std::atomic<uint64_t>* done) {
    if (done->load(std::memory_order_acquire) >> device & 1) return;
    if (hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, 160 * 1024) == hipSuccess)
        done->fetch_or(1ull << device, std::memory_order_release);
}

// A launch counts its threads in 32 bits: one of 2^32 or more fails or, worse, runs only what is left of the count and
// reports nothing.  fn(first, count) for parts of `total` rows, `most` at a time.
constexpr int64_t kMaxThreads = UINT32_MAX;
template <typename Fn>
void in_parts(int64_t total, int64_t most, Fn fn) {
    for (int64_t first = 0; first < total; first += most) fn(first, total - first < most ? total - first : most);
}

struct ScoreArgs {
    const int8_t* xq;
    int64_t ldx;
    const float* xs;
    int64_t m;
    const int8_t* tq;
    int64_t ldt;
    const float* ts;
    int64_t n;
    int f;
    void* out;
    int64_t ldo;
    hipStream_t stream;
    int device;
};

template <typename T, int WU, int WI, int FU, int FI, int STAGES>
void launch_tiles(const ScoreArgs& a) {
    using C = Tiles<WU, WI, FU, FI, STAGES>;
    static std::atomic<uint64_t> done{0};
    auto* kernel = k_score_tiles<T, WU, WI, FU, FI, STAGES>;
    const int64_t tu = (a.m + C::kUsers - 1) / C::kUsers, ti = (a.n + C::kItems - 1) / C::kItems;
    const int steps = (a.f + kStep - 1) / kStep;
    whole_lds(kernel, a.device, &done);
    hipLaunchKernelGGL(kernel, dim3((unsigned)(tu * ti)), dim3(64 * C::kWaves),
                       (steps < STAGES ? steps : STAGES) * C::kStage, a.stream, a.xq, a.ldx, a.xs, a.m, a.tq, a.ldt,
                       a.ts, a.n, a.f, (T*)a.out, a.ldo, (uint32_t)tu, (uint32_t)ti);
}

// The tile: the largest that still gives every CU enough of them.  A large tile reads the rows fewer times, which
// counts where f is large; with few tiles, CUs stand idle (256 x 8,192 x 8,192, us: 256 x 256 tiles 90, 128 x 128
// 42, 64 x 128 37, 64 x 64 in four stages 27).  Measured (us, users x items x f):
//   8,192 x 8,192 x 8,192      256 x 256: 445    128 x 128: 489    64 x 128: 589
//   1,024 x 8,192 x 8,192      256 x 256: 99     128 x 128: 64     64 x 128: 87
//   2,048 x 2,048 x 1,024      128 x 128: 9.6    64 x 128: 8.4     64 x 64: 11.0
//   512 x 512 x 4,096          64 x 128: 14.7    64 x 64: 10.2     16 x 64: 8.6
//   5 x 8,192 x 8,192          64 x 128: 34      64 x 64: 18       16 x 64: 15
// Up to f = 128 there is one step and the scores' way out counts (into two buffers in turn):
//   fp32   4,096 x 40,000 x 128    128 x 128: 150    64 x 128: 170    32 x 256: 186
//          6,000 x 6,000 x 100     128 x 128: 26.7   64 x 128: 26.0   32 x 256: 27.3
//   bf16   4,096 x 40,000 x 128    128 x 128: 102    64 x 128: 111    32 x 256: 91      (f16 101, 108, 90)
//          4,096 x 40,000 x 100    128 x 128: 99     64 x 128: 108    32 x 256: 88
//          1,024 x 17,770 x 100    128 x 128: 12.7   64 x 128: 12.3   32 x 256: 13.2
//          2,100 x 8,200 x 100     128 x 128: 12.7   64 x 128: 11.8   32 x 256: 12.8
//          8,192 x 12,000 x 64     128 x 128: 44.5   64 x 128: 45.8   32 x 256: 49.8
//          6,000 x 6,000 x 16      128 x 128: 17.8   64 x 128: 19.1   32 x 256: 19.7
// So 32 x 256 gains a tenth on outputs larger than the card's cache and loses as much on those that fit it.
template <typename T>
void score_tiles(const ScoreArgs& a, int cus) {
    const auto tiles = [&](int64_t users, int64_t items) {
        return ((a.m + users - 1) / users) * ((a.n + items - 1) / items);
    };
    if (a.m > 16) {
        if (a.f <= kStep) {
            if (sizeof(T) == 2 && tiles(32, 256) >= 8 * cus) return launch_tiles<T, 1, 4, 2, 4, 2>(a);
            if (sizeof(T) == 4 && tiles(128, 128) >= 8 * cus) return launch_tiles<T, 2, 2, 4, 4, 2>(a);
        } else {
            if (a.f >= 1024 && tiles(256, 256) >= cus) return launch_tiles<T, 2, 4, 8, 4, 2>(a);
            if (tiles(128, 128) >= 2 * cus) return launch_tiles<T, 2, 2, 4, 4, 2>(a);
        }
        if (tiles(64, 128) >= 2 * cus) return launch_tiles<T, 2, 2, 2, 4, 2>(a);
        if (tiles(64, 64) >= cus) return launch_tiles<T, 2, 2, 2, 2, 4>(a);
    }
    return launch_tiles<T, 1, 2, 1, 2, 4>(a);
}

int finish(als_serve_ctx* ctx) {
    const hipError_t e = hipGetLastError();
    if (e == hipSuccess) return ALS_OK;
    ctx->last_hip = (int)e;
    return ALS_ERR_HIP;
}

}  // namespace

extern "C" {

size_t als_serve_workspace_bytes(int device) {
    int cus = 0;
    return query_device(device, &cus) == ALS_OK ? kWorkspaceBytes : 0;
}

int als_serve_init(als_serve_ctx** out, int device, void* workspace, size_t workspace_bytes) {
    if (!out) return ALS_ERR_INVALID_ARG;
    *out = nullptr;
    if (!workspace) return ALS_ERR_WORKSPACE;
    if (!aligned(workspace, 256)) return ALS_ERR_ALIGN;
    int cus = 0;
    if (const int rc = query_device(device, &cus); rc != ALS_OK) return rc;
    if (workspace_bytes < kWorkspaceBytes) return ALS_ERR_WORKSPACE;
    als_serve_ctx* ctx = new (std::nothrow) als_serve_ctx();
    if (!ctx) return ALS_ERR_INVALID_ARG;
    ctx->device = device;
    ctx->cus = cus;
    ctx->ws = (unsigned char*)workspace;
    ctx->ws_bytes = workspace_bytes < kWorkspaceMost ? workspace_bytes : kWorkspaceMost;
    ctx->last_hip = 0;
    *out = ctx;
    return ALS_OK;
}

int als_serve_destroy(als_serve_ctx* ctx) {
    delete ctx;
    return ALS_OK;
}

int als_serve_last_hip_error(const als_serve_ctx* ctx) { return ctx ? ctx->last_hip : 0; }

int als_quantize(als_serve_ctx* ctx, const void* x, int32_t dtype, int64_t of, int64_t ldx, const int32_t* users,
                 int64_t rows, int32_t f, int8_t* q, int64_t ldq, float* scale, void* stream) {
    const int64_t pad = ((int64_t)f + 15) / 16 * 16;
    return als_quantize_into(ctx, x, dtype, of, ldx, users, rows, f, q, ldq, (int32_t)(pad < ldq ? pad : ldq), scale,
                             stream);
}

int als_quantize_into(als_serve_ctx* ctx, const void* x, int32_t dtype, int64_t of, int64_t ldx, const int32_t* users,
                      int64_t rows, int32_t f, int8_t* q, int64_t ldq, int32_t width, float* scale, void* stream) {
    if (!ctx || of < 0 || rows < 0 || dtype < ALS_F32 || dtype > ALS_BF16) return ALS_ERR_INVALID_ARG;
    if (f < 1 || f > ALS_SERVE_F_MAX) return ALS_ERR_UNSUPPORTED_F;
    const int64_t pad = ((int64_t)f + 15) / 16 * 16;
    if (ldx < f || ldq < f || width < f || width > ldq || width > pad || (!users && rows > of)) return ALS_ERR_INVALID_ARG;
    if (rows == 0) return ALS_OK;
    if (!q || !scale || (of > 0 && !x)) return ALS_ERR_INVALID_ARG;
    if (!aligned(x, type_bytes(dtype)) || !aligned(users, 4) || !aligned(scale, 4)) return ALS_ERR_ALIGN;
    const uint64_t xn = span_of(of, f, ldx, type_bytes(dtype));
    const uint64_t qn = span_of(rows, width, ldq, 1), sn = (uint64_t)rows * 4;
    if (overlap(q, qn, x, xn) || overlap(scale, sn, x, xn) || overlap(q, qn, scale, sn) ||
        overlap(q, qn, users, sn) || overlap(scale, sn, users, sn))
        return ALS_ERR_ALIAS;
    DeviceGuard guard(ctx->device);
    if (!guard.ok) return ALS_ERR_DEVICE;
    // kernel(x, of, users, rows, q, scale) for parts of the rows, a workgroup taking `per` of them
    const auto rows_by = [&](auto* p, int64_t per, auto kernel) {
        in_parts(rows, kMaxThreads / kQuantThreads * per, [&](int64_t r, int64_t some) {
            hipLaunchKernelGGL(kernel, dim3((unsigned)((some + per - 1) / per)), dim3(kQuantThreads), 0,
                               (hipStream_t)stream, users ? p : p + r * ldx, users ? of : of - r, ldx,
                               users ? users + r : users, some, f, q + r * ldq, ldq, width, scale + r);
        });
    };
    const auto go = [&](auto* p, auto lanes, auto loads) {
        using T = std::remove_cv_t<std::remove_pointer_t<decltype(p)>>;
        constexpr int G = decltype(lanes)::value, E = decltype(loads)::value;
        rows_by(p, kQuantThreads / G, k_quantize<T, G, E>);
    };
    // Two loads a lane and the fewest lanes that hold the row so, up to a wave; then more loads, then a workgroup.
    // 625,000 x 100 fp32: 16 lanes of 2 loads 61 us, 8 of 4 65, 32 of 1 100, 32 of 2 94 (half the lanes idle);
    // 200,000 x 256: 32 of 2 44, 16 of 4 49, 64 of 1 56; 1,000,000 x 16: 4 of 2 17, 8 of 1 30, 16 of 1 58.
    const auto launch = [&](auto* p) {
        using T = std::remove_cv_t<std::remove_pointer_t<decltype(p)>>;
        using std::integral_constant;
        using Two = integral_constant<int, 2>;
        const int groups = (int)((pad + 16 / sizeof(T) - 1) / (16 / sizeof(T)));      // loads of a row
        if (groups <= 8) go(p, integral_constant<int, 4>(), Two());
        else if (groups <= 16) go(p, integral_constant<int, 8>(), Two());
        else if (groups <= 32) go(p, integral_constant<int, 16>(), Two());
        else if (groups <= 64) go(p, integral_constant<int, 32>(), Two());
        else if (groups <= 128) go(p, integral_constant<int, 64>(), Two());
        else if (groups <= 256) go(p, integral_constant<int, 64>(), integral_constant<int, 4>());
        else if (groups <= 512) go(p, integral_constant<int, 256>(), Two());
        else if (groups <= 1024) go(p, integral_constant<int, 256>(), integral_constant<int, 4>());
        else if (groups <= 2048) go(p, integral_constant<int, 256>(), integral_constant<int, 8>());
        else rows_by(p, 1, k_quantize_long<T>);
    };
    if (dtype == ALS_F32) launch((const float*)x);
    else if (dtype == ALS_F16) launch((const F16*)x);
    else launch((const BF16*)x);
    return finish(ctx);
}

int als_score(als_serve_ctx* ctx, const int8_t* xq, int64_t ldx, const float* xs, int64_t m, const int8_t* tq,
              int64_t ldt, const float* ts, int64_t n, int32_t f, void* out, int32_t dtype, int64_t ldo,
              void* stream) {
    if (!ctx || m < 0 || n < 0 || dtype < ALS_F32 || dtype > ALS_BF16) return ALS_ERR_INVALID_ARG;
    if (f < 1 || f > ALS_SERVE_F_MAX) return ALS_ERR_UNSUPPORTED_F;
    if (ldx < f || ldt < f || ldo < n) return ALS_ERR_INVALID_ARG;
    if (m == 0 || n == 0) return ALS_OK;
    if (!xq || !xs || !tq || !ts || !out) return ALS_ERR_INVALID_ARG;
    if (!aligned(xs, 4) || !aligned(ts, 4) || !aligned(out, type_bytes(dtype))) return ALS_ERR_ALIGN;
    const uint64_t on = span_of(m, n, ldo, type_bytes(dtype));
    if (overlap(out, on, xq, span_of(m, f, ldx, 1)) || overlap(out, on, tq, span_of(n, f, ldt, 1)) ||
        overlap(out, on, xs, (uint64_t)m * 4) || overlap(out, on, ts, (uint64_t)n * 4))
        return ALS_ERR_ALIAS;
    DeviceGuard guard(ctx->device);
    if (!guard.ok) return ALS_ERR_DEVICE;
    const hipStream_t st = (hipStream_t)stream;
    // rows that a tile's loads cannot take are first laid out anew in the workspace, half of it for either side, as many
    // at a time as it holds (512 at least)
    const int64_t whole = ((int64_t)f + 15) / 16 * 16, half = (int64_t)(ctx->ws_bytes / 2), fit = half / whole;
    const auto direct = [](const int8_t* q, int64_t ld) { return aligned(q, 16) && ld % 16 == 0 && ld < kTileStride; };
    const bool x_direct = direct(xq, ldx), t_direct = direct(tq, ldt);
    int64_t users = x_direct || m < fit ? m : fit, items = t_direct || n < fit ? n : fit;
    // no launch of more than 2^31 threads: the most a tile takes is 128 of them for 16 users and 64 items (half the
    // limit: the larger tiles' last rows); the narrower side stays whole, and parts are whole tiles
    const int64_t most = kMaxThreads / 128 / 2, tu = (users + 15) / 16, ti = (items + 63) / 64;
    if (tu > most / ti) {
        if (tu > 4096 && ti > 4096) items = 4096 * 64;
        if (tu <= 4096) items = most / tu / 4 * 4 * 64;
        else users = most / ((items + 63) / 64) / 16 * 16 * 16;
    }
    const auto pack = [&](const int8_t* q, int64_t ld, int64_t rows, unsigned char* to) {
        const int64_t groups = whole / 16, blocks = (rows * groups + 255) / 256;
        hipLaunchKernelGGL(k_pack, dim3((unsigned)blocks), dim3(256), 0, st, q, ld, rows, f, (int8_t*)to, groups);
        return (const int8_t*)to;
    };
    for (int64_t i = 0; i < m; i += users) {
        const int64_t mi = m - i < users ? m - i : users;
        const int8_t* x = x_direct ? xq + i * ldx : pack(xq + i * ldx, ldx, mi, ctx->ws);
        for (int64_t j = 0; j < n; j += items) {
            const int64_t nj = n - j < items ? n - j : items;
            const int8_t* t = (const int8_t*)(ctx->ws + half);
            if (t_direct) t = tq + j * ldt;
            else if (i == 0 || items < n) pack(tq + j * ldt, ldt, nj, ctx->ws + half);      // else all items are there
            const ScoreArgs args{x, x_direct ? ldx : whole, xs + i, mi, t, t_direct ? ldt : whole, ts + j, nj, f,
                                 (char*)out + (i * ldo + j) * type_bytes(dtype), ldo, st, ctx->device};
            if (dtype == ALS_F32) score_tiles<float>(args, ctx->cus);
            else if (dtype == ALS_F16) score_tiles<F16>(args, ctx->cus);
            else score_tiles<BF16>(args, ctx->cus);
        }
    }
    return finish(ctx);
}

int als_sample(als_serve_ctx* ctx, const void* z, int32_t dtype, int64_t rows, int64_t n, int64_t ldz,
               const als_sample_limits* limits, const float* u, const int64_t* rated_ptr,
               const int32_t* rated_idx, const int32_t* users, int64_t of, int32_t* index, float* log,
               void* stream) {
    if (!ctx || !limits || rows < 0 || n < 0 || n > ALS_SERVE_N_MAX || dtype < ALS_F32 || dtype > ALS_BF16 ||
        ldz < n || of < 0)
        return ALS_ERR_INVALID_ARG;
    if (rows == 0) return ALS_OK;
    if (!u || !index || (n > 0 && !z) || rows > INT32_MAX) return ALS_ERR_INVALID_ARG;
    if (!rated_ptr != !rated_idx || (users && !rated_ptr) || (rated_ptr && !users && of < rows))
        return ALS_ERR_INVALID_ARG;
    const als_sample_limits& l = *limits;
    if (!aligned(z, type_bytes(dtype)) || !aligned(u, 4) || !aligned(rated_ptr, 8) || !aligned(rated_idx, 4) ||
        !aligned(users, 4) || !aligned(index, 4) || !aligned(log, 4) || !aligned(l.temperature, 4) ||
        !aligned(l.top_k, 4) || !aligned(l.top_p, 4) || !aligned(l.min_p, 4))
        return ALS_ERR_ALIGN;
    const uint64_t rn = (uint64_t)rows * 4;
    const void* outs[2] = {index, log};
    for (const void* o : outs)
        if (overlap(o, rn, z, span_of(rows, n, ldz, type_bytes(dtype))) || overlap(o, rn, u, rn) ||
            overlap(o, rn, rated_ptr, ((uint64_t)of + 1) * 8) || overlap(o, rn, users, rn) ||
            overlap(o, rn, l.temperature, rn) || overlap(o, rn, l.top_k, rn) || overlap(o, rn, l.top_p, rn) ||
            overlap(o, rn, l.min_p, rn))
            return ALS_ERR_ALIAS;
    if (overlap(index, rn, log, rn)) return ALS_ERR_ALIAS;
    DeviceGuard guard(ctx->device);
    if (!guard.ok) return ALS_ERR_DEVICE;
    const Limits lim{l.temperature, l.top_k, l.top_p, l.min_p, l.temperature_all, l.top_k_all, l.top_p_all,
                     l.min_p_all};
    const Rated rated{rated_ptr, rated_idx, users, of};
    const auto held = [&](auto h, auto* p) {
        using H = decltype(h);
        using T = std::remove_cv_t<std::remove_pointer_t<decltype(p)>>;
        auto* kernel = k_sample<H::kScores, H::kBins, T>;
        const size_t lds = sizeof(typename H::Shared) + (rated_ptr ? (size_t)(n + 31) / 32 * 4 : 0);
        static std::atomic<uint64_t> done{0};
        whole_lds(kernel, ctx->device, &done);
        const int64_t a_wave = kWave * H::kScores, waves = n < a_wave ? 1 : (n + a_wave - 1) / a_wave;
        in_parts(rows, kMaxThreads / (kWave * waves), [&](int64_t row0, int64_t some) {
            hipLaunchKernelGGL(kernel, dim3((unsigned)some), dim3((unsigned)(kWave * waves)), lds, (hipStream_t)stream, p,
                               row0, (uint32_t)n, ldz, lim, u, rated, index, log);
        });
    };
    const auto launch = [&](auto* p) {
        using T = std::remove_cv_t<std::remove_pointer_t<decltype(p)>>;
        // Few rows: few scores a thread, as a row's passes are what is waited for.  More rows than CUs: more scores a
        // thread and fewer waves, up to one, which needs no barrier.  Top-k 200, top-p 0.9 and left-out columns, us,
        // by scores a thread: 1 x 500 4 12.6, 8 15.6; 1 x 1,000 4 13, 16 19; 2,048 x 1,000 4 29, 16 25; 2,048 x 2,000 8
        // 41, 16 31; 2,048 x 4,000 8 38, 16 49; 2,000 x 8,000 8 83, 16 48, 32 89; 1 x 16,000 by top-p alone 16 21, 32 28;
        // 2,000 x 16,000 16 108, 32 68.
        if (rows <= ctx->cus) {
            if (n <= 1024) return held(Held<4, 256>(), p);
            if (n <= 4096) return held(Held<8, 1024>(), p);
            if (n <= 16384) return held(Held<16, 1024>(), p);
        } else {
            if (n <= 512) return held(Held<8, 256>(), p);
            if (n <= 2048) return held(Held<16, 512>(), p);
            if (n <= 4096) return held(Held<8, 1024>(), p);     // (enough threads for a top-k of some hundreds)
            if (n <= 8192) return held(Held<16, 1024>(), p);
        }
        if (n <= 32768) return held(Held<32, 2048>(), p);
        if (n <= ALS_SERVE_HELD_MAX) return held(Held<64, 4096>(), p);
        // in batches of as many rows as the workspace holds
        const int64_t segments = (n + kSegColumns - 1) / kSegColumns;
        uint32_t group = 1;
        while (segments * (kSegThreads / group) > kGroups) group *= 2;
        const size_t a_segment = sizeof(SegStat) + kSegThreads / group * sizeof(float) + Segment::kBins * 8 + kSlab * 8;
        const int64_t batch = (int64_t)(ctx->ws_bytes / (a_segment * segments + sizeof(RowPlan)));
        const hipStream_t st = (hipStream_t)stream;
        const int64_t bits = rated_ptr ? (n < kChunk ? n : kChunk) : 0;
        const size_t slow_lds = sizeof(SampleShared) + (size_t)((bits + 31) / 32) * 4;
        const size_t row_lds = sizeof(RowShared) > slow_lds ? sizeof(RowShared) : slow_lds;
        static std::atomic<uint64_t> of_rows{0}, of_draw{0};
        whole_lds(k_long_rows<T>, ctx->device, &of_rows);
        whole_lds(k_long_draw<T>, ctx->device, &of_draw);
        const bool shares = l.top_p || l.top_p_all < 1.f;
        for (int64_t row0 = 0; row0 < rows; row0 += batch) {
            const int64_t some = rows - row0 < batch ? rows - row0 : batch;
            LongArgs<T> args{p, n, ldz, lim, u, rated, index, log, {}};
            LongWork& w = args.work;
            unsigned char* at = ctx->ws;        // the widest types first
            w.bins = (uint64_t*)at;
            at += some * segments * Segment::kBins * 8;
            w.stat = (SegStat*)at;
            at += some * segments * sizeof(SegStat);
            w.plan = (RowPlan*)at;
            at += some * sizeof(RowPlan);
            w.groups = (float*)at;
            at += some * segments * (kSegThreads / group) * sizeof(float);
            w.list_z = (float*)at;
            at += some * segments * kSlab * 4;
            w.list_column = (uint32_t*)at;
            w.segments = (uint32_t)segments;
            w.group = group;
            w.row0 = row0;
            const dim3 parts((unsigned)(some * segments)), whole((unsigned)some);
            hipLaunchKernelGGL(k_long_stats<T>, parts, dim3(kSegThreads), 0, st, args);
            hipLaunchKernelGGL(k_long_parts<T>, parts, dim3(kSegThreads), 0, st, args);
            hipLaunchKernelGGL(k_long_rows<T>, whole, dim3(kRowThreads), row_lds, st, args);
            if (shares) {
                hipLaunchKernelGGL(k_long_cut<T>, parts, dim3(kSegThreads), 0, st, args);
                hipLaunchKernelGGL(k_long_draw<T>, whole, dim3(kRowThreads), row_lds, st, args);
            }
        }
    };
    if (dtype == ALS_F32) launch((const float*)z);
    else if (dtype == ALS_F16) launch((const F16*)z);
    else launch((const BF16*)z);
    return finish(ctx);
}

}  // extern "C"
