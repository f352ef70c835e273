// How probable items are under a trained factor model, on gfx950 (MI355X): the C ABI of include/als_predict.h plus its
// kernels.
//
//   k_product_lds predictions from 16-bit rows at multiples of 16 bytes, which arrive in LDS straight from memory
//   k_product     predictions from any other rows, which pass through registers into LDS; fp32 rows as three bf16
//                 parts (k_join: the products' parts along f into one, where few tiles are cut along it)
//   k_row         a row of scores, or a segment of one, as a distribution: statistics, given columns, best columns
//                 (k_row_join: a row's segments into one)
//   k_gradient    the gradient with respect to scores and offsets (k_columns: the offsets' from its parts)

#include <new>

#include "als_predict.h"
#include "common.h"

namespace {

typedef float f4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf8 __attribute__((ext_vector_type(8)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));
typedef int i4 __attribute__((ext_vector_type(4)));

// Two values to 16 bits each by one instruction, where the type has one.
typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
typedef float f2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t two_bf16(float a, float b) {
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f2{a, b}), bf2));
}
template <int N, typename T>
__device__ __forceinline__ void from_floats(const float* v, T (&out)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) from_float(v[i], &out[i]);
}
template <int N>
__device__ __forceinline__ void from_floats(const float* v, BF16 (&out)[N]) {
    uint32_t w[N / 2];
#pragma unroll
    for (int i = 0; i < N / 2; ++i) w[i] = two_bf16(v[2 * i], v[2 * i + 1]);
    __builtin_memcpy(out, w, sizeof out);
}

// A barrier for what the workgroup's waves write to LDS and read there: __syncthreads() would also wait for the loads and
// stores that are on their way to or from memory.
__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// ------------------------------------------------------------------------------- product --

// What follows a product: its offsets, activation and residual, and where it goes.
struct Epilogue {
    const float* user_offset;
    const float* item_offset;
    const void* residual;
    int64_t ldr;
    void* out;
    int64_t ldo;
    float low, high;
    int activation;
    int type;      // of residual and out
};

struct Product {
    const void* x;
    int64_t of, ldx;
    const int32_t* users;
    int64_t m;
    const void* theta;
    int64_t n, ldt;
    int f, tail;             // values of a row, and those of them behind the last whole step (see k_product)
    uint32_t tu, ti;         // tiles of users and of items
    uint32_t height;         // tiles of users that follow one another
    int steps;               // along f in one part of it
    Epilogue end;
    float* parts;            // where f is cut: parts x m x n sums; else NULL

    // The row of X that row i of the result is for; -1: there is none.
    __device__ __forceinline__ int64_t user_of(int64_t i) const {
        const int64_t u = users ? (int64_t)users[i] : i;
        return u >= 0 && u < of ? u : -1;
    }
};

// exp(x + low), x in [-300, 0] and low of its last bits: a product with log2(e) in two parts, as the whole exponent's
// rounding would cost |x| units.
__device__ __forceinline__ float exp_of(float x, float low) {
    const float high = x * 0x1.715476p+0f;
    const float rest = fmaf(x, 0x1.715476p+0f, -high) + fmaf(x, 0x1.4ae0cp-26f, low * 0x1.715476p+0f);
    const float e = __builtin_amdgcn_exp2f(high);
    return fmaf(e, rest * 0x1.62e43p-1f, e);
}
// 1 / d, d in [1, 2^30], to half a unit and a little.
__device__ __forceinline__ float inverse_of(float d) {
    const float r = __builtin_amdgcn_rcpf(d);
    return fmaf(fmaf(-d, r, 1.f), r, r);
}
// 1 / (1 + exp(-y)) by exp(-|y|), which does not overflow and keeps the small values down to 2^-126, below which an
// exponential is 0 (y < -87.3).
__device__ __forceinline__ float sigmoid(float y) {
    const float e = exp_of(-fminf(fabsf(y), 126.f), 0.f), r = inverse_of(1.f + e);
    return y != y ? y : (y < 0.f ? e * r : r);
}
// y erfc(-y / sqrt 2) / 2.  With a = |y| / sqrt 2 and t = 1 / (1 + 0.3 a), erfc(a) exp(a^2) / t is a polynomial in t
// (fitted by least squares, weighted towards the largest error, to scipy's erfcx); with these coefficients it is off by
// 4.3e-8 of its value up to |y| = 13.  In fp32 GELU was off by at most 5.3e-7 of its value (2 million arguments each in
// [-13.1, -12], [-12, -0.001], [-1, -0.001], [-0.001, 0] and [0, 12]), also where it is small: 1 + erf(y / sqrt 2) would lose
// it.  Below y = -13.2, where the exponential is below 2^-126, it is -0.
__device__ __forceinline__ float gelu(float y) {
    const float a = fminf(fabsf(y), 18.f), t = inverse_of(fmaf(a, 0.212132034f, 1.f));
    float q = -0.12925273f;
    q = fmaf(q, t, 0.48429954f);
    q = fmaf(q, t, -0.5097682f);
    q = fmaf(q, t, 0.5449625f);
    q = fmaf(q, t, -0.092823245f);
    q = fmaf(q, t, 0.21418034f);
    q = fmaf(q, t, 0.14852151f);
    q = fmaf(q, t, 0.1706909f);
    q = fmaf(q, t, 0.16918935f);
    const float square = a * a, half = 0.5f * fminf(fmaxf(y, -30.f), 30.f);
    const float tail = t * q * exp_of(-0.5f * square, -0.5f * fmaf(a, a, -square));
    return y < 0.f ? half * tail : fmaf(-half, tail, y);
}

// For results of 16 bits, whose half a unit is 2^-11 or more of them: exponentials of arguments rounded to fp32 (a few
// units of 2^-24, times the exponent's size), and for GELU a polynomial (in t = 1 / (1 + 0.44 a)) to 5.2e-6 of its value
// up to |y| = 13 (7.5e-6 at 18, where the value is 0 in every type).
__device__ __forceinline__ float sigmoid16(float y) {
    return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(y * -0x1.715476p+0f));
}
__device__ __forceinline__ float gelu16(float y) {
    const float a = fminf(fabsf(y), 18.f), t = __builtin_amdgcn_rcpf(fmaf(a, 0.31112698f, 1.f));
    float q = -0.14610672f;
    q = fmaf(q, t, 0.35065565f);
    q = fmaf(q, t, 0.040727474f);
    q = fmaf(q, t, 0.26358837f);
    q = fmaf(q, t, 0.242569f);
    q = fmaf(q, t, 0.24856107f);
    const float half = 0.5f * fminf(fmaxf(y, -30.f), 30.f);
    const float tail = t * q * __builtin_amdgcn_exp2f(a * a * -0.72134752f);
    return y < 0.f ? half * tail : fmaf(-half, tail, y);
}

// The activations, and those of results of 16 bits.
enum { kSigmoid16 = 16, kSilu16, kGelu16 };
template <int ACT>
__device__ __forceinline__ float activated(float y, const Epilogue& e) {
    if constexpr (ACT == ALS_ACT_CLIP) {
        y = y < e.low ? e.low : y;
        return y > e.high ? e.high : y;
    }
    if constexpr (ACT == ALS_ACT_RELU) return y < 0.f ? 0.f : y;
    if constexpr (ACT == ALS_ACT_GELU) return gelu(y);
    if constexpr (ACT == ALS_ACT_SILU) return fmaxf(y, -126.f) * sigmoid(y);
    if constexpr (ACT == ALS_ACT_SIGMOID) return sigmoid(y);
    if constexpr (ACT == ALS_ACT_TANH) return tanhf(y);
    if constexpr (ACT == kGelu16) return gelu16(y);
    if constexpr (ACT == kSilu16) return fmaxf(y, -126.f) * sigmoid16(y);
    if constexpr (ACT == kSigmoid16) return sigmoid16(y);
    return y;
}
// fn(the activation as a constant): once for many values, as a choice for each takes longer than most of them do
template <typename Fn>
__device__ __forceinline__ void by_activation(const Epilogue& e, Fn fn) {
    using std::integral_constant;
    const bool fine = e.type == ALS_F32;
    switch (e.activation) {
        case ALS_ACT_CLIP: return fn(integral_constant<int, ALS_ACT_CLIP>());
        case ALS_ACT_RELU: return fn(integral_constant<int, ALS_ACT_RELU>());
        case ALS_ACT_GELU: return fine ? fn(integral_constant<int, ALS_ACT_GELU>()) : fn(integral_constant<int, kGelu16>());
        case ALS_ACT_SILU: return fine ? fn(integral_constant<int, ALS_ACT_SILU>()) : fn(integral_constant<int, kSilu16>());
        case ALS_ACT_SIGMOID:
            return fine ? fn(integral_constant<int, ALS_ACT_SIGMOID>()) : fn(integral_constant<int, kSigmoid16>());
        case ALS_ACT_TANH: return fn(integral_constant<int, ALS_ACT_TANH>());
        default: return fn(integral_constant<int, ALS_ACT_NONE>());
    }
}
template <typename Fn>
__device__ __forceinline__ void by_out_type(int type, Fn fn) {
    if (type == ALS_F32) fn((float*)nullptr);
    else if (type == ALS_F16) fn((F16*)nullptr);
    else fn((BF16*)nullptr);
}

// Four neighbouring values of a row, as far as `left` of them are there.  (As a vector of the elements' alignment: of four
// values the compiler takes apart what both branches do, and the whole four are no longer one access.)
template <typename T>
struct Vector4;
template <>
struct Vector4<float> { typedef uint32_t Type __attribute__((ext_vector_type(4), aligned(4))); };
template <>
struct Vector4<F16> { typedef uint16_t Type __attribute__((ext_vector_type(4), aligned(2))); };
template <>
struct Vector4<BF16> { typedef uint16_t Type __attribute__((ext_vector_type(4), aligned(2))); };

template <typename T>
__device__ __forceinline__ void load4(const T* p, int left, float (&v)[4]) {
    using Vector = typename Vector4<T>::Type;
    T t[4];
    if (left >= 4) {
        const Vector w = *(const Vector*)p;
        __builtin_memcpy(t, &w, sizeof t);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = to_float(t[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = i < left ? to_float(p[i]) : 0.f;
    }
}
template <typename T>
__device__ __forceinline__ void store4(T* p, int left, const float (&v)[4]) {
    using Vector = typename Vector4<T>::Type;
    T t[4];
    from_floats<4>(v, t);
    if (left >= 4) {
        Vector w;
        __builtin_memcpy(&w, t, sizeof t);
        *(Vector*)p = w;
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < left) p[i] = t[i];
    }
}

// What user i's results have added: its offset; NaN for a user that there is not.
__device__ __forceinline__ float own_offset(const Product& a, int64_t i) {
    const int64_t u = i < a.m ? a.user_of(i) : -1;
    return u < 0 ? NAN : (a.end.user_offset ? a.end.user_offset[u] : 0.f);
}

// How many of the four items from `item` on there are.
__device__ __forceinline__ int items_left(const Product& a, int64_t item) {
    const int64_t left = a.n - item;
    return left >= 4 ? 4 : (left > 0 ? (int)left : 0);
}

// Of N rows of results, from the sums of four neighbouring items each: the residuals first, all of them on their way
// together; then what follows a product.  The rows lie `row[k]` (the same in every lane, so that no lane multiplies by a
// row stride) past the user whose results are at out_at and residuals at residual_at; `left[k]` of the four are there.
template <int N, int ACT>
__device__ __forceinline__ void finish(const Product& a, int64_t out_at, int64_t residual_at, const int (&row)[N],
                                       const int (&left)[N], float (&v)[N][4], const float (&own)[N],
                                       const float (&offset)[4]) {
    const Epilogue& e = a.end;
    float r[N][4];
    if (e.residual)
        by_out_type(e.type, [&](auto* p) {
#pragma unroll
            for (int k = 0; k < N; ++k) load4((decltype(p))e.residual + row[k] * e.ldr + residual_at, left[k], r[k]);
        });
#pragma unroll
    for (int k = 0; k < N; ++k)
#pragma unroll
        for (int i = 0; i < 4; ++i) v[k][i] = activated<ACT>(v[k][i] + own[k] + offset[i], e);
    if (e.residual) {
#pragma unroll
        for (int k = 0; k < N; ++k)
#pragma unroll
            for (int i = 0; i < 4; ++i) v[k][i] += r[k][i];
    }
    by_out_type(e.type, [&](auto* p) {
#pragma unroll
        for (int k = 0; k < N; ++k) store4((decltype(p))e.out + row[k] * e.ldo + out_at, left[k], v[k]);
    });
}

// Tile t of a grid of tu x ti: the eight dies take workgroups in turn, so each gets a run of tiles of its own, and
// runs go down `height` tiles of users before the next of items (their rows stay in the die's L2).
__device__ __forceinline__ void tile_of(uint32_t t, uint32_t tu, uint32_t ti, uint32_t height, uint32_t* u, uint32_t* i) {
    const uint32_t total = tu * ti, per = total / 8;
    if (t < per * 8) t = (t % 8) * per + t / 8;
    const uint32_t band = height * ti, b = t / band, left = t % band;
    const uint32_t high = tu - height * b < height ? tu - height * b : height;
    *u = height * b + left % high;
    *i = left / high;
}

// Matrix instructions of eight values a lane, by the type of the parts that are multiplied.
__device__ __forceinline__ f4 multiply8(u4 a, u4 b, f4 c, BF16) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf8, a), __builtin_bit_cast(bf8, b), c, 0, 0, 0);
}
__device__ __forceinline__ f4 multiply8(u4 a, u4 b, f4 c, F16) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8, a), __builtin_bit_cast(h8, b), c, 0, 0, 0);
}

// A type's rows as they are multiplied: `kParts` parts of 16 bits a value.
template <typename T>
struct Parts {
    static constexpr int kParts = 1;
    static constexpr int kValues = 64;       // of a row in a step
    using Part = T;
    // eight values, zeros past `left`
    static __device__ __forceinline__ void load(const T* p, int left, u4 (&v)[1]) {
        if (left >= 8) {
            __builtin_memcpy(&v[0], p, 16);
        } else {
            uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < left) w[i / 2] |= (uint32_t)p[i].bits << (i % 2 * 16);
            v[0] = u4{w[0], w[1], w[2], w[3]};
        }
    }
    static __device__ __forceinline__ void split(const u4 (&raw)[1], u4 (&part)[1]) { part[0] = raw[0]; }
    static constexpr int kRaw = 1;
};

template <>
struct Parts<float> {
    static constexpr int kParts = 3;
    static constexpr int kValues = 32;
    using Part = BF16;
    static constexpr int kRaw = 2;
    static __device__ __forceinline__ void load(const float* p, int left, u4 (&v)[2]) {
        using Vector = Vector4<float>::Type;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            v[h] = u4{0, 0, 0, 0};
            if (left >= 4 * h + 4) v[h] = *(const Vector*)(p + 4 * h);
            else if (left > 4 * h)
#pragma unroll
                for (int i = 0; i < 3; ++i)
                    if (4 * h + i < left) v[h][i] = __builtin_bit_cast(uint32_t, p[4 * h + i]);
        }
    }
    // x = high + mid + low: the upper 16 bits of x (cut off, so that the largest floats stay finite), then what is left
    // rounded to bf16 twice; |mid| < 2^-7 |x|, |low| <= 2^-16 |x|, and what is left after it is 0.
    static __device__ __forceinline__ void split(const u4 (&raw)[2], u4 (&part)[3]) {
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const uint32_t b0 = raw[w / 2][w % 2 * 2], b1 = raw[w / 2][w % 2 * 2 + 1];
            part[0][w] = __builtin_amdgcn_perm(b1, b0, 0x07060302u);
            const float r0 = __builtin_bit_cast(float, b0) - __builtin_bit_cast(float, b0 & 0xFFFF0000u);
            const float r1 = __builtin_bit_cast(float, b1) - __builtin_bit_cast(float, b1 & 0xFFFF0000u);
            const uint32_t mid = two_bf16(r0, r1);
            part[1][w] = mid;
            part[2][w] = two_bf16(r0 - __builtin_bit_cast(float, mid << 16),
                                  r1 - __builtin_bit_cast(float, mid & 0xFFFF0000u));
        }
    }
};

constexpr int kHead = 1024;      // of LDS: a tile's users' offsets

template <typename T, int WU, int WI, int FU, int FI>
struct Staged {
    using P = Parts<T>;
    static constexpr int kThreads = 64 * WU * WI;
    static constexpr int kUsers = WU * FU * 16, kItems = WI * FI * 16, kRows = kUsers + kItems;
    static constexpr int kRowBytes = 2 * P::kValues, kGroups = P::kValues / 8;      // of a part of a row
    static constexpr int kPart = kRows * kRowBytes, kStage = P::kParts * kPart;
    static constexpr int kUnits = kRows * kGroups, kLoads = (kUnits + kThreads - 1) / kThreads;
    // the way out: so many fragments of users at a time, rows of items four values apart from one bank
    static constexpr int kOut = FU < 2 ? 1 : 2, kOutRows = WU * kOut * 16, kOutStride = kItems + 4;
    static constexpr int kBoth = kStage + (P::kParts == 3 ? kRows * 32 : 0);      // with the values behind whole steps
    static constexpr int kLds = kBoth > kOutRows * kOutStride * 4 ? kBoth : kOutRows * kOutStride * 4;
    static_assert(FU % kOut == 0, "whole passes");
    static_assert(kUsers * 4 <= kHead && kHead + kLds <= 160 * 1024, "LDS");
};

// What a tile's results have added: the users' offsets in LDS, and those of this thread's four items.  Asked for once the
// first rows are on their way, so that neither they nor the results wait for it.
template <typename C>
__device__ __forceinline__ void fetch_offsets(const Product& a, float* own, float (&offset)[4], int64_t u0, int64_t i0) {
#pragma unroll
    for (int i = 0; i < 4; ++i) offset[i] = 0.f;
    if (a.parts) return;
    const int64_t item = i0 + 4 * (threadIdx.x % (C::kItems / 4));
    if (a.end.item_offset) load4(a.end.item_offset + item, items_left(a, item), offset);
    for (int r = threadIdx.x; r < C::kUsers; r += C::kThreads) own[r] = own_offset(a, u0 + r);
}

// The products of a tile on their way out, through LDS, so that a wave writes whole lines and what follows a product
// is there once in the code.  A lane holds four neighbouring items (of group lane / 16) of one user (lane % 16).
template <typename C, int WU, int WI, int FU, int FI>
__device__ __forceinline__ void write_tile(const Product& a, const f4 (&acc)[FU][FI], float* lds, const float* own,
                                           const float (&offset)[4], int64_t u0, int64_t i0, int wu, int wi, int part) {
    const int lane = threadIdx.x & 63;
    constexpr int kFours = C::kItems / 4, kAtOnce = C::kThreads / kFours, kRuns = C::kOutRows / kAtOnce;
    constexpr int N = kRuns < 4 ? kRuns : 4;
    static_assert(16 * C::kOut % kAtOnce == 0 && kRuns % N == 0, "whole runs of rows, each of one wave's users");
    const int four = threadIdx.x % kFours, first = threadIdx.x / kFours;
    const int64_t item = i0 + 4 * four, user0 = u0 + first;
    const int items = items_left(a, item), users = a.m - u0 < C::kUsers ? (int)(a.m - u0) : C::kUsers;
    const int64_t out_at = user0 * a.end.ldo + item, residual_at = user0 * a.end.ldr + item, parts_at = (part * a.m + user0) * a.n + item;
    const auto rows = [&](int pass, auto go) {
#pragma unroll 1
        for (int run = 0; run < kRuns; run += N) {
            float v[N][4], mine[N];
            int row[N], left[N];
#pragma unroll
            for (int k = 0; k < N; ++k) {
                const int r = (run + k) * kAtOnce;
                row[k] = (r / (16 * C::kOut) * FU + pass * C::kOut) * 16 + r % (16 * C::kOut);
                left[k] = first + row[k] < users ? items : 0;
                mine[k] = own[first + row[k]];
                const f4 s = *(const f4*)(lds + (first + r) * C::kOutStride + 4 * four);
#pragma unroll
                for (int i = 0; i < 4; ++i) v[k][i] = s[i];
            }
            go(row, left, v, mine);
        }
    };
#pragma unroll 1
    for (int pass = 0; pass < FU / C::kOut; ++pass) {
        lds_barrier();
#pragma unroll
        for (int u = 0; u < FU; ++u) {
            if (u / C::kOut != pass) continue;
#pragma unroll
            for (int i = 0; i < FI; ++i)
                *(f4*)(lds + ((wu * C::kOut + u % C::kOut) * 16 + (lane & 15)) * C::kOutStride + (wi * FI + i) * 16 +
                       4 * (lane >> 4)) = acc[u][i];
        }
        lds_barrier();
        if (a.parts)
            rows(pass, [&](auto& row, auto& left, auto& v, auto&) {
#pragma unroll
                for (int k = 0; k < N; ++k) store4(a.parts + row[k] * a.n + parts_at, left[k], v[k]);
            });
        else
            by_activation(a.end, [&](auto act) {
                rows(pass, [&](auto& row, auto& left, auto& v, auto& mine) {
                    finish<N, act.value>(a, out_at, residual_at, row, left, v, mine, offset);
                });
            });
    }
}

// The product in tiles, rows through registers: a workgroup of WU x WI waves holds a tile of users x items, each wave
// FU x FI fragments of 16 x 16, and walks f in steps of 32 fp32 or 64 16-bit values.  While a step is multiplied
// from LDS the next one's rows arrive in registers; fp32 values are split there, once for all that they meet.
// The 16-byte group c of a part of row r lies in slot c ^ s(r), so that the 16 rows of an operand read spread
// over all banks: s is r / 2 % 8 for rows of 128 bytes, and 0, 2, 3, 1 by r / 4 % 4 for 64 (with 0, 1, 2, 3 the sixteen
// lanes that read at a time, which are not neighbours, met in pairs).
// Of fp32, up to eight values behind whole steps are multiplied as they are, by fp32 matrix instructions, four at a time
// from places of their own in LDS: a step for them would cost as much as any other (1,024 x 17,770 x 100: 44 us, 46 without).
// (Rows whose stride is a multiple of 128 bytes are the fastest: a step of a row at 400 bytes lies in two lines, and f = 96
// takes 34 us, f = 128 41.)
// 1,024 x 17,770 x 100 fp32 in 39 to 44 us (1.8 TB/s out, 93 Tflop/s): its vector instructions issue in 20 us (splits a third,
// the way out a fifth), its matrix instructions in 12, and barriers and loads keep them from running side by side.
template <typename T, int WU, int WI, int FU, int FI>
__global__ __launch_bounds__(64 * WU * WI) void k_product(Product a) {
    using C = Staged<T, WU, WI, FU, FI>;
    using P = Parts<T>;
    extern __shared__ __align__(1024) unsigned char shared[];
    float* own = (float*)shared;
    unsigned char* lds = shared + kHead;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    uint32_t tile_u, tile_i;
    tile_of(blockIdx.x, a.tu, a.ti, a.height, &tile_u, &tile_i);
    const int64_t u0 = (int64_t)tile_u * C::kUsers, i0 = (int64_t)tile_i * C::kItems;
    const auto slot = [](int r, int g) { return C::kRowBytes == 64 ? g ^ (0x78 >> (r >> 1 & 6) & 3) : g ^ (r >> 1 & 7); };

    const int whole = a.f - a.tail;
    const auto row_of = [&](int r) -> const T* {      // of the tile's rows, users first
        if (r < C::kUsers) {
            const int64_t u = u0 + r < a.m ? a.user_of(u0 + r) : -1;
            return u >= 0 ? (const T*)a.x + u * a.ldx : nullptr;
        }
        return i0 + r - C::kUsers < a.n ? (const T*)a.theta + (i0 + r - C::kUsers) * a.ldt : nullptr;
    };
    // this thread's groups of eight values: a row each, at the same place in every step
    const T* from[C::kLoads];
    int to[C::kLoads];
    int at[C::kLoads];
#pragma unroll
    for (int l = 0; l < C::kLoads; ++l) {
        const int unit = threadIdx.x + l * C::kThreads, r = unit / C::kGroups, g = unit % C::kGroups;
        at[l] = 8 * g;
        to[l] = unit < C::kUnits ? r * C::kRowBytes + 16 * slot(r, g) : -1;
        from[l] = unit < C::kUnits ? row_of(r) : nullptr;
    }
    u4 raw[C::kLoads][P::kRaw];
    const auto fetch = [&](int step) {
#pragma unroll
        for (int l = 0; l < C::kLoads; ++l) {
            const int k = step * P::kValues + at[l];
            P::load(from[l] + k, from[l] ? whole - k : 0, raw[l]);
        }
    };
    const auto stage = [&]() {
#pragma unroll
        for (int l = 0; l < C::kLoads; ++l) {
            u4 part[P::kParts];
            P::split(raw[l], part);
            if (to[l] < 0) continue;
#pragma unroll
            for (int p = 0; p < P::kParts; ++p) *(u4*)(lds + p * C::kPart + to[l]) = part[p];
        }
    };

    const int wu = wave / WI, wi = wave % WI, row = lane & 15, group = lane >> 4;
    f4 acc[FU][FI];
#pragma unroll
    for (int u = 0; u < FU; ++u)
#pragma unroll
        for (int i = 0; i < FI; ++i) acc[u][i] = f4{0.f, 0.f, 0.f, 0.f};
    const auto read = [&](int r, int h, u4 (&v)[P::kParts]) {
#pragma unroll
        for (int p = 0; p < P::kParts; ++p)
            v[p] = *(const u4*)(lds + p * C::kPart + r * C::kRowBytes + 16 * slot(r, 4 * h + group));
    };
    const auto multiply = [&]() {
#pragma unroll
        for (int h = 0; h < P::kValues / 32; ++h) {
            u4 t[FI][P::kParts];
#pragma unroll
            for (int i = 0; i < FI; ++i) read(C::kUsers + (wi * FI + i) * 16 + row, h, t[i]);
#pragma unroll
            for (int u = 0; u < FU; ++u) {
                u4 x[P::kParts];
                read((wu * FU + u) * 16 + row, h, x);
                // the smallest products first; of nine, those of mid x low and below are left out
                const auto add = [&](int p, int q) {
#pragma unroll
                    for (int i = 0; i < FI; ++i) acc[u][i] = multiply8(t[i][p], x[q], acc[u][i], typename P::Part());
                };
                if constexpr (P::kParts == 3) {
                    add(2, 0);
                    add(0, 2);
                    add(1, 1);
                    add(1, 0);
                    add(0, 1);
                }
                add(0, 0);
            }
        }
    };

    const int steps = (whole + P::kValues - 1) / P::kValues, begin = blockIdx.y * a.steps;
    const int end = begin + a.steps < steps ? begin + a.steps : steps;
    fetch(begin);
    float offset[4];
    fetch_offsets<C>(a, own, offset, u0, i0);
    float* tails = (float*)(lds + C::kStage);
    const bool with_tail = P::kParts == 3 && a.tail > 0 && end == steps;
    if (with_tail)
        for (int r = threadIdx.x; r < C::kRows; r += C::kThreads) {
            const float* p = (const float*)row_of(r) + whole;
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                float v[4];
                load4(p + 4 * c, row_of(r) ? a.tail - 4 * c : 0, v);
#pragma unroll
                for (int i = 0; i < 4; ++i) v[i] += v[i] - v[i];      // an infinity gives NaN, as it does in parts
                *(f4*)(tails + (c * C::kRows + r) * 4) = f4{v[0], v[1], v[2], v[3]};
            }
        }
    for (int step = begin; step < end; ++step) {
        stage();
        lds_barrier();
        if (step + 1 < end) fetch(step + 1);
        multiply();
        if (step + 1 < end) lds_barrier();
    }
    if (with_tail) {
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            if (4 * c >= a.tail) continue;
            const auto value = [&](int r) { return tails[(c * C::kRows + r) * 4 + group]; };
            float t[FI];
#pragma unroll
            for (int i = 0; i < FI; ++i) t[i] = value(C::kUsers + (wi * FI + i) * 16 + row);
#pragma unroll
            for (int u = 0; u < FU; ++u) {
                const float x = value((wu * FU + u) * 16 + row);
#pragma unroll
                for (int i = 0; i < FI; ++i) acc[u][i] = __builtin_amdgcn_mfma_f32_16x16x4f32(t[i], x, acc[u][i], 0, 0, 0);
            }
        }
    }
    write_tile<C, WU, WI, FU, FI>(a, acc, (float*)lds, own, offset, u0, i0, wu, wi, blockIdx.y);
}

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
// wait for every load to LDS before any LDS read.  It has no result register; the caller waits (settle) before the data
// are read.  M0 needs one wait state, and is these loads' alone in their kernels (it cannot be named as clobbered).
__device__ __forceinline__ void load_to_lds(i4 buffer, uint32_t voffset, uint32_t soffset, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %3\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, %2 offen lds"
                 :
                 : "v"(voffset), "s"(buffer), "s"(soffset), "s"(lds)
                 : "memory");
}
// A load reads a scalar register that a vector instruction wrote (readfirstlane) no sooner than five wait states
// later; the compiler keeps them for the loads it knows.
__device__ __forceinline__ void buffer_settle(i4 a, i4 b) { asm volatile("s_nop 4" : : "s"(a), "s"(b)); }
// All of each wave's loads but its last LEFT have arrived, and its LDS reads are done.
template <int LEFT>
__device__ __forceinline__ void settle() {
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" : : "n"(LEFT) : "memory");
}

// The values of a group of eight 16-bit ones of which `left` are there, zeros in the others' place.
__device__ __forceinline__ u4 keep_values(u4 v, int left) {
#pragma unroll
    for (int d = 0; d < 4; ++d) v[d] &= left >= 2 * d + 2 ? 0xFFFFFFFFu : (left == 2 * d + 1 ? 0xFFFFu : 0u);
    return v;
}

constexpr int64_t kNear = 1 << 21;              // row strides below it (4 MiB) keep a tile's offsets below 2^30 ...
constexpr uint32_t kPastEnd = 0x7FFFFFF0u;      // ... and this past every buffer's end

template <int WU, int WI, int FU, int FI, int STEP, int STAGES>
struct Direct {
    static constexpr int kStep = STEP, kStepBytes = 2 * STEP, kGroups = STEP / 8;      // a row's in a step
    static constexpr int kWaves = WU * WI, kThreads = 64 * kWaves;
    static constexpr int kUsers = WU * FU * 16, kItems = WI * FI * 16, kRows = kUsers + kItems;
    static constexpr int kAtOnce = 64 / kGroups;      // rows that a wave's load of 1 KB takes
    static constexpr int kUserLoads = kUsers / kAtOnce / kWaves, kItemLoads = kItems / kAtOnce / kWaves;
    static constexpr int kStage = kRows * kStepBytes;
    static constexpr int kOut = FU < 2 ? 1 : 2, kOutRows = WU * kOut * 16, kOutStride = kItems + 4;
    static constexpr int kOutBytes = kOutRows * kOutStride * 4;
    static_assert(kUsers % (kAtOnce * kWaves) == 0 && kItems % (kAtOnce * kWaves) == 0, "whole loads");
    static_assert((STAGES - 2) * (kUserLoads + kItemLoads) < 64, "loads that can be counted");
    static_assert(kUsers * 4 <= kHead && kHead + STAGES * kStage <= 160 * 1024 && kHead + kOutBytes <= 160 * 1024, "LDS");
};

// The product in tiles as k_product has them, of 16-bit rows at multiples of 16 bytes: a step's rows of both sides lie
// in LDS, 2 STEP bytes a row, while the next steps' (STAGES - 1 of them) arrive straight from memory beside them
// (buffer_load ... lds: no registers, no instructions but the load).  Items and users past the end read as zeros; in the
// last step values past f are masked on both sides, as what lies in their place may be no number.
// 4,096 x 8,192 x 8,192 in 425 us without activation and residual (1.29 Pflop/s; the library's product 406), with GELU and
// residual 456 to 484 by card: one workgroup is on a CU, and nothing runs beside its way out.  4,096 x 40,000 x 128 in 124 us
// without activation, with a sigmoid in 132 to 140 (2.5 TB/s): loads, products and stores of a tile follow one another, and
// the four workgroups of a CU do not hide all of it (stores alone took 95 us, where a fill of as many bytes takes 48).
// 5 x 8,192 x 8,192 with its join in 24.5 us where the last level of cache holds the weights (5.5 TB/s), in 35 where they come
// from memory (3.8 TB/s).
template <typename T, int WU, int WI, int FU, int FI, int STEP, int STAGES>
__global__ __launch_bounds__(64 * WU * WI) void k_product_lds(Product a) {
    using C = Direct<WU, WI, FU, FI, STEP, STAGES>;
    constexpr int kStep = C::kStep, kStepBytes = C::kStepBytes, kAtOnce = C::kAtOnce;
    extern __shared__ __align__(1024) unsigned char shared[];
    float* own = (float*)shared;
    unsigned char* lds = shared + kHead;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    uint32_t tile_u, tile_i;
    tile_of(blockIdx.x, a.tu, a.ti, a.height, &tile_u, &tile_i);
    const int64_t u0 = (int64_t)tile_u * C::kUsers, i0 = (int64_t)tile_i * C::kItems;

    // what the buffers hold: the tile's rows (all of X where users are taken by index; one at least), the last up to the
    // end of its last group.  A load's offset is compared with the bytes less the scalar offset, which a buffer
    // without rows would take below 0 and so past kPastEnd.
    const int64_t users = a.m - u0 < C::kUsers ? a.m - u0 : C::kUsers, items = a.n - i0 < C::kItems ? a.n - i0 : C::kItems;
    const int64_t from = a.users ? 0 : u0, rows = a.users ? a.of : users;
    const int whole = (a.f + 7) / 8 * 16;
    const i4 from_u = buffer_of((const T*)a.x + from * a.ldx, (uint32_t)((rows - 1) * a.ldx * 2 + whole));
    const i4 from_i = buffer_of((const T*)a.theta + i0 * a.ldt, (uint32_t)((items - 1) * a.ldt * 2 + whole));
    buffer_settle(from_u, from_i);
    const int first_u = wave * C::kUserLoads * kAtOnce, first_i = wave * C::kItemLoads * kAtOnce;   // this wave's rows
    const auto slot = [](int r, int g) { return kStepBytes == 64 ? g ^ (0x78 >> (r >> 1 & 6) & 3) : g ^ (r >> 1 & 7); };
    const auto group_of = [&](int r) { return 16 * slot(r, lane % C::kGroups); };
    uint32_t of_u[C::kUserLoads], of_i[C::kItemLoads];
#pragma unroll
    for (int l = 0; l < C::kUserLoads; ++l) {
        const int r = first_u + kAtOnce * l + lane / C::kGroups;
        const int64_t u = u0 + r < a.m ? a.user_of(u0 + r) : -1;
        of_u[l] = u < 0 ? kPastEnd : (uint32_t)((u - from) * a.ldx * 2) + group_of(r);
    }
#pragma unroll
    for (int l = 0; l < C::kItemLoads; ++l) {
        const int r = first_i + kAtOnce * l + lane / C::kGroups;
        of_i[l] = (uint32_t)(r * a.ldt * 2) + group_of(r);
    }
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)lds;
    const int steps = (a.f + kStep - 1) / kStep, begin = blockIdx.y * a.steps;
    const int end = begin + a.steps < steps ? begin + a.steps : steps;
    // groups past f are not read: their offset is past the buffer's end
    const auto fetch = [&](int step, int stage) {
        const uint32_t to = lds0 + stage * C::kStage;
        const int left = 2 * a.f - step * kStepBytes;
#pragma unroll
        for (int l = 0; l < C::kUserLoads; ++l) {
            const int r = first_u + kAtOnce * l;
            load_to_lds(from_u, group_of(r + lane / C::kGroups) < left ? of_u[l] : kPastEnd, step * kStepBytes,
                        __builtin_amdgcn_readfirstlane(to + r * kStepBytes));
        }
#pragma unroll
        for (int l = 0; l < C::kItemLoads; ++l) {
            const int r = first_i + kAtOnce * l;
            load_to_lds(from_i, group_of(r + lane / C::kGroups) < left ? of_i[l] : kPastEnd, step * kStepBytes,
                        __builtin_amdgcn_readfirstlane(to + (C::kUsers + r) * kStepBytes));
        }
    };

    const int wu = wave / WI, wi = wave % WI;
    const int row = lane & 15, group = lane >> 4;
    f4 acc[FU][FI];
#pragma unroll
    for (int u = 0; u < FU; ++u)
#pragma unroll
        for (int i = 0; i < FI; ++i) acc[u][i] = f4{0.f, 0.f, 0.f, 0.f};
    const auto multiply = [&](int step, int stage, auto tail) {
        const unsigned char* at = lds + stage * C::kStage;
#pragma unroll
        for (int h = 0; h < kStep / 32; ++h) {
            u4 t[FI], x[FU];
            const int left = a.f - step * kStep - 32 * h - 8 * group;
            const auto read = [&](int r) {
                const u4 v = *(const u4*)(at + r * kStepBytes + 16 * slot(r, 4 * h + group));
                return tail.value ? keep_values(v, left) : v;
            };
#pragma unroll
            for (int i = 0; i < FI; ++i) t[i] = read(C::kUsers + (wi * FI + i) * 16 + row);
#pragma unroll
            for (int u = 0; u < FU; ++u) x[u] = read((wu * FU + u) * 16 + row);
            __builtin_amdgcn_s_setprio(1);      // (these before another wave's reads: 1% at 4,096 x 8,192 x 8,192)
#pragma unroll
            for (int u = 0; u < FU; ++u)
#pragma unroll
                for (int i = 0; i < FI; ++i) acc[u][i] = multiply8(t[i], x[u], acc[u][i], T());
            __builtin_amdgcn_s_setprio(0);
        }
    };

#pragma unroll
    for (int p = 0; p < STAGES - 1; ++p)
        if (begin + p < end) fetch(begin + p, p);
    float offset[4];
    fetch_offsets<C>(a, own, offset, u0, i0);
    // a step: its rows are there and the last step's are done with (settle says both), whose place the rows
    // STAGES - 1 steps on take
    int stage = 0;
    const auto after = [](int x) { return x + 1 == STAGES ? 0 : x + 1; };
    int step = begin;
    for (; step + STAGES - 1 < end; ++step) {
        settle<(STAGES - 2) * (C::kUserLoads + C::kItemLoads)>();
        fetch(step + STAGES - 1, stage == 0 ? STAGES - 1 : stage - 1);
        multiply(step, stage, std::false_type());
        stage = after(stage);
    }
    settle<0>();
    for (; step + 1 < end; ++step) {
        multiply(step, stage, std::false_type());
        stage = after(stage);
    }
    multiply(step, stage, std::true_type());
    write_tile<C, WU, WI, FU, FI>(a, acc, (float*)lds, own, offset, u0, i0, wu, wi, blockIdx.y);
}

// The sums of the parts of f into one, in their order, and what follows a product.
__global__ __launch_bounds__(256) void k_join(Product a, int count) {
    const int64_t fours = (a.n + 3) / 4, at = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int64_t i = at / fours, item = at % fours * 4;
    if (i >= a.m) return;
    const int left = items_left(a, item);
    float v[1][4], offset[4] = {0.f, 0.f, 0.f, 0.f};
    load4(a.parts + i * a.n + item, left, v[0]);
#pragma unroll 4
    for (int p = 1; p < count; ++p) {
        float w[4];
        load4(a.parts + (p * a.m + i) * a.n + item, left, w);
#pragma unroll
        for (int k = 0; k < 4; ++k) v[0][k] += w[k];
    }
    if (a.end.item_offset) load4(a.end.item_offset + item, left, offset);
    const float own = own_offset(a, i);
    by_activation(a.end, [&](auto act) {
        finish<1, act.value>(a, i * a.end.ldo + item, i * a.end.ldr + item, {0}, {left}, v, {own}, offset);
    });
}

// --------------------------------------------------------------------------- distribution --

__device__ __forceinline__ float wave_sum(float v) {
#define ALS_STEP(CTRL, ROWS) v += __builtin_bit_cast(float, dpp32<CTRL, ROWS>(__builtin_bit_cast(uint32_t, v)))
    ALS_STEP(0x111, 0xF);
    ALS_STEP(0x112, 0xF);
    ALS_STEP(0x114, 0xF);
    ALS_STEP(0x118, 0xF);
    ALS_STEP(0x142, 0xA);
    ALS_STEP(0x143, 0xC);
#undef ALS_STEP
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), 63));
}

constexpr float kLog2E = 1.44269504f, kLn2 = 0.693147181f;
constexpr float kNothing = -200.f;       // 2 to it is 0 in fp32

// Some scores' best one, their weights' sum and the sum of weight times exponent; weights are 2^((z - best) c),
// c = log2(e) / T.
struct Mass {
    float best, sum, spread;
};

// (z - best) c, from -200 up; what is not a number (NaN scores, +inf less +inf) weighs nothing
__device__ __forceinline__ float exponent(float z, float best, float c) { return fmaxf((z - best) * c, kNothing); }

// The masses that the wave's lanes hold as one (best -inf, sums 0: nothing).
__device__ __forceinline__ Mass joined(Mass a, float c) {
    Mass all;
    all.best = wave_max(a.best);
    const float x = a.best == all.best ? 0.f : exponent(a.best, all.best, c);
    const float w = __builtin_amdgcn_exp2f(x) * a.sum;
    all.sum = wave_sum(w);
    all.spread = wave_sum(__builtin_amdgcn_exp2f(x) * a.spread + w * x);
    return all;
}

// log2(e) / T, finite.
__device__ __forceinline__ float rate_of(float t) { return fminf((float)(1.4426950408889634 / (double)t), 3.402823466e38f); }

// A row's distribution as its results need it.
struct Law {
    float best, t, size;     // size: log of the weights' sum
    uint32_t first;          // the first best column, where T is not above 0 (else unused)
    bool there;              // the row's user exists
    __device__ __forceinline__ bool greedy() const { return !(t > 0.f); }
    __device__ __forceinline__ bool none() const { return best == -INFINITY; }
    // log p of an allowed column
    __device__ __forceinline__ float log_of(float z, uint32_t column) const {
        if (!there) return NAN;
        if (!(z > -INFINITY)) return -INFINITY;
        if (greedy()) return column == first ? 0.f : -INFINITY;
        const float d = z - best;
        return z == best ? -size : (d > -INFINITY ? d / t - size : -INFINITY);
    }
};

template <typename T>
struct RowArgs {
    const T* z;
    int64_t row0, rows, n, ldz;
    const float* temperature;
    float temperature_all;
    Rated rated;
    als_given given;
    float* log;
    float* stats;
    float* entropy;
    int top;
    int32_t* top_index;
    float* top_log;
    // rows in segments
    uint32_t segments, columns;     // of a row; of a segment
    struct SegMass* mass;           // rows x segments
    uint64_t* keys;                 // rows x segments x top

    __device__ __forceinline__ void entries(int64_t r, int64_t* begin, int64_t* end) const {
        if (given.ptr) {
            const int64_t b = given.ptr[r], e = given.ptr[r + 1];
            *begin = b < 0 ? 0 : b;
            *end = e > given.entries ? given.entries : e;
        } else {
            *begin = r * given.each;
            *end = *begin + given.each;
        }
    }
};

struct SegMass {
    Mass mass;
    uint32_t first;
};

// Order of columns: higher scores first, then lower columns; 0 is no column.
__device__ __forceinline__ uint64_t place_of(float z, uint32_t column) {
    return z > -INFINITY ? (uint64_t)key_of(z) << 32 | (0xFFFFFFFFu - column) : 0;
}
__device__ __forceinline__ float score_at(uint64_t place) { return score_of((uint32_t)(place >> 32)); }
__device__ __forceinline__ uint32_t column_at(uint64_t place) { return 0xFFFFFFFFu - (uint32_t)place; }

__device__ __forceinline__ uint64_t wave_max64(uint64_t v) {
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) {
        const uint64_t o = (uint64_t)__shfl_xor((unsigned long long)v, d);
        v = o > v ? o : v;
    }
    return v;
}

constexpr int kMaxWaves = 16;
constexpr int kGroups = 256;
constexpr int kList = 1024;

struct RowShared {
    Mass mass[kMaxWaves];
    uint64_t place[kMaxWaves];
    uint32_t first;
    uint32_t cut, count;
    uint32_t group[kGroups];
    uint64_t list[kList];
};

// The first `top` places in their order, for few that are given: emit(rank, place) for each, by some thread; how many
// there are is the result.  A score that `top` groups of threads have reached at their best is below none of the first
// `top`; the columns from it on are listed (random rows: hardly more than `top`, as the groups' best are mostly of
// different groups) and each one's rank is counted among them.  Where the list does not hold them (the best columns stand
// in few groups, or many are equal) they are taken one at a time.
//   offer     each thread's best key (0: none); then a barrier
//   decide    by the first wave, while the others go on with something else; then a barrier
//   finish    each(cut, fn) calls fn(place) for all of a thread's places whose key is at least the cut
struct Top {
    RowShared* sh;
    int top;

    __device__ __forceinline__ void offer(uint32_t key) const {
        int d = 0;
        if (blockDim.x > kGroups) {
            key = max(key, (uint32_t)__builtin_amdgcn_mov_dpp((int)key, 0xB1, 0xF, 0xF, true));     // lanes 1, 0, 3, 2
            d = 1;
        }
        if (blockDim.x > 2 * kGroups) {
            key = max(key, (uint32_t)__builtin_amdgcn_mov_dpp((int)key, 0x4E, 0xF, 0xF, true));     // lanes 2, 3, 0, 1
            d = 2;
        }
        if ((threadIdx.x & ((1 << d) - 1)) == 0) sh->group[threadIdx.x >> d] = key;
        if (threadIdx.x == 0) sh->count = 0;
    }

    __device__ __forceinline__ void decide() const {
        if (threadIdx.x < kWave) {
            const int d = blockDim.x > 2 * kGroups ? 2 : (blockDim.x > kGroups ? 1 : 0), groups = blockDim.x >> d;
            uint32_t key[kGroups / kWave];
#pragma unroll
            for (int k = 0; k < kGroups / kWave; ++k) {
                const int at = k * kWave + threadIdx.x;
                key[k] = at < groups ? sh->group[at] : 0;
            }
            uint32_t cut = 0;
            for (uint32_t bit = 1u << 31; bit != 0; bit >>= 1) {
                int reached = 0;
#pragma unroll
                for (int k = 0; k < kGroups / kWave; ++k) reached += __popcll(__ballot(key[k] >= (cut | bit)));
                if (reached >= top) cut |= bit;
                if (reached == top) break;
            }
            if (threadIdx.x == 0) sh->cut = cut < 1 ? 1 : cut;
        }
    }

    template <typename Each, typename Below, typename Emit>
    __device__ __forceinline__ int finish(uint32_t own, Each each, Below below, Emit emit) const {
        const uint32_t cut = sh->cut;
        if (own >= cut)
            each(cut, [&](uint64_t place) {
                const uint32_t at = atomicAdd(&sh->count, 1u);
                if (at < kList) sh->list[at] = place;
            });
        lds_barrier();
        const int count = sh->count;
        if (count <= kList) {
            for (int i = threadIdx.x; i < count; i += blockDim.x) {
                const uint64_t mine = sh->list[i];
                int rank = 0;
#pragma unroll 4
                for (int j = 0; j < count; ++j) rank += sh->list[j] > mine;
                if (rank < top) emit(rank, mine);
            }
            return count < top ? count : top;
        }
        const int wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
        uint64_t limit = ~0ull;
        int found = 0;
        for (; found < top; ++found) {
            uint64_t p = wave_max64(below(limit));
            lds_barrier();
            if ((threadIdx.x & 63) == 0) sh->place[wave] = p;
            lds_barrier();
            for (int w = 0; w < waves; ++w) p = sh->place[w] > p ? sh->place[w] : p;
            if (p == 0) break;
            if (threadIdx.x == 0) emit(found, p);
            limit = p;
        }
        return found;
    }
};

// What a row's distribution gives, but its log p of given columns; called by all of the workgroup's threads.
template <typename T>
__device__ __forceinline__ void write_law(const RowArgs<T>& a, int64_t r, const Law& law, const Mass& mass) {
    if (threadIdx.x != 0) return;
    if (a.stats) {
        const bool as_is = law.there && !law.none();
        a.stats[2 * r] = law.there ? law.best : NAN;
        a.stats[2 * r + 1] = as_is ? (law.greedy() ? 0.f : law.size) : (law.there ? -INFINITY : NAN);
    }
    if (a.entropy) {
        float h = law.size - kLn2 * (mass.spread / mass.sum);
        if (law.none() || law.greedy()) h = 0.f;
        a.entropy[r] = law.there ? h : NAN;
    }
}

template <typename T>
__device__ __forceinline__ void write_top(const RowArgs<T>& a, int64_t r, const Law& law, int rank, uint64_t place) {
    if (a.top_index) a.top_index[r * a.top + rank] = law.there ? (int32_t)column_at(place) : -1;
    if (a.top_log) a.top_log[r * a.top + rank] = law.log_of(score_at(place), column_at(place));
}
template <typename T>
__device__ __forceinline__ void write_no_top(const RowArgs<T>& a, int64_t r, const Law& law, int from) {
    for (int k = from + threadIdx.x; k < a.top; k += blockDim.x) {
        if (a.top_index) a.top_index[r * a.top + k] = -1;
        if (a.top_log) a.top_log[r * a.top + k] = law.there ? -INFINITY : NAN;
    }
}

// A row, or a segment of one, of up to E scores a thread, which stay in registers from their one read on: the best one of
// a wave, then weights relative to it (a wave's sums need no barrier), then the waves' masses joined.  H comes from the
// same pass: with x = log2 w, H = log S - ln 2 sum(w x) / S, whose terms are all of one sign.
// 1,024 x 17,770 fp32 in 19.5 us, with the 20 best 25 to 26 (73 MB: 3.8 and 2.9 TB/s); 64 x 625,000 bf16 with the join in 29
// and 41 where the last level of cache holds the rows, in 33 and 46 where not.  Bound by waits: a workgroup's loads, lists, sums
// and its best columns follow one another, and most workgroups are at the same one.  40 scores a thread past 16,384 took the
// least time (1,024 x 17,770 with the best: 32 a thread 36 us, 40 27, 48 29, 64 42 at the time).  At 80 registers a SIMD has
// six of its waves, so a CU three rows of 17,770 (seven waves each), and 1,024 rows take two rounds, the second a third full.
// Segments of 20,480 columns (64 x 625,000 bf16: 45.8 us; 8,192 49.0, 16,384 49.4, 32,768 59.0); fewer rows have segments as
// long, and leave CUs idle: one row of 625,000 is 31 workgroups.
template <typename T, int E>
__global__ __launch_bounds__(1024, E <= 16 || sizeof(T) == 2 ? 8 : 6) void k_row(RowArgs<T> a) {
    constexpr int V = E * sizeof(T) < 16 ? E : 16 / sizeof(T);
    __shared__ RowShared sh;
    extern __shared__ uint32_t bits[];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
    const uint32_t segment = blockIdx.x % a.segments;
    const int64_t local = blockIdx.x / a.segments, r = a.row0 + local;
    const uint32_t base = segment * a.columns;
    const uint32_t n = (uint32_t)a.n - base < a.columns ? (uint32_t)a.n - base : a.columns;
    const T* row = a.z + r * a.ldz + base;
    const auto position = [&](int v) { return (uint32_t)(v * blockDim.x + threadIdx.x) * V; };

    // the lists' first entries before the scores, as loads come back in their order
    const int32_t* list;
    int64_t listed, begin, end;
    Law law;
    law.there = a.rated.row(r, &list, &listed);
    law.t = limit_of(a.temperature, a.temperature_all, r);
    a.entries(r, &begin, &end);
    const bool some = law.there && listed > 0;
    const uint32_t out0 = some && threadIdx.x < listed ? (uint32_t)list[threadIdx.x] - base : ~0u;
    const bool asked = begin + threadIdx.x < end;
    const uint32_t column0 = asked ? (uint32_t)a.given.idx[begin + threadIdx.x] : ~0u;
    // (scores of 16 bits are quiet from here on, fp32 ones once they have arrived: a loop here would wait for each load)
    const auto score = [](T t) { return sizeof(T) == 2 ? quiet(to_float(t)) : to_float(t); };
    float z[E];
#pragma unroll
    for (int v = 0; v < E / V; ++v) {
        const uint32_t c = position(v);
        T t[V];
        if (c + V <= n) {
            __builtin_memcpy(t, row + c, sizeof t);
#pragma unroll
            for (int i = 0; i < V; ++i) z[v * V + i] = score(t[i]);
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i) z[v * V + i] = c + i < n ? score(row[c + i]) : -INFINITY;
        }
    }
    const float score0 = column0 - base < n ? to_float(row[column0 - base]) : 0.f;
    if (threadIdx.x == 0) sh.first = ~0u;
    if (some) {
        for (uint32_t w = threadIdx.x; w < (n + 31) / 32; w += blockDim.x) bits[w] = 0;
        lds_barrier();
        const auto mark = [&](uint32_t c) {
            if (c < n) atomicOr(&bits[c >> 5], 1u << (c & 31));
        };
        mark(out0);
        for (int64_t k = threadIdx.x + blockDim.x; k < listed; k += blockDim.x) mark((uint32_t)list[k] - base);
    }
    lds_barrier();
    const auto left_out = [&](uint32_t c) { return some && (bits[c >> 5] >> (c & 31) & 1); };
    if (some) {
#pragma unroll
        for (int v = 0; v < E / V; ++v) {
            const uint32_t c = position(v);
            if (c >= n) continue;
            const uint32_t w = bits[c >> 5] >> (c & 31);      // V divides 32
#pragma unroll
            for (int i = 0; i < V; ++i) z[v * V + i] = w >> i & 1 ? -INFINITY : z[v * V + i];
        }
    }

    const float c = law.greedy() ? 1.f : rate_of(law.t);
    Mass mass{-INFINITY, 0.f, 0.f};
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int e = 0; e < E; ++e) z[e] = quiet(z[e]);
    }
#pragma unroll
    for (int e = 0; e < E; ++e) mass.best = fmaxf(mass.best, z[e]);
    const uint32_t own = mass.best > -INFINITY ? key_of(mass.best) : 0;
    const Top top{&sh, a.top};
    if (a.top) {
        top.offer(own);
        lds_barrier();
        top.decide();
    }
    mass.best = wave_max(mass.best);
#pragma unroll
    for (int e = 0; e < E; ++e) {
        const float x = exponent(z[e], mass.best, c), w = __builtin_amdgcn_exp2f(x);
        mass.sum += w;
        mass.spread = fmaf(w, x, mass.spread);
    }
    if (mass.best == INFINITY) {
        mass.sum = mass.spread = 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) mass.sum += z[e] == INFINITY ? 1.f : 0.f;
    }
    mass.sum = wave_sum(mass.sum);
    mass.spread = wave_sum(mass.spread);
    if (lane == 0) sh.mass[wave] = mass;
    lds_barrier();
    mass = joined(lane < waves ? sh.mass[lane] : Mass{-INFINITY, 0.f, 0.f}, c);
    law.best = mass.best;
    law.size = logf(mass.sum);
    if (law.greedy()) {
        uint32_t first = ~0u;
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (z[e] == mass.best && z[e] > -INFINITY) {
                const uint32_t at = position(e / V) + e % V;
                first = at < first ? at : first;
            }
        if (first != ~0u) atomicMin(&sh.first, base + first);
        lds_barrier();
    }
    law.first = sh.first;

    const bool whole = a.segments == 1;
    const auto answer = [&](int64_t e, uint32_t column, float s) {
        const uint32_t at = column - base;
        if (at < n) {
            const float v = left_out(at) ? -INFINITY : s;
            a.log[e] = whole ? law.log_of(v, column) : v;
        } else if (column >= (uint32_t)a.n && segment == 0) {
            a.log[e] = law.there ? -INFINITY : NAN;
        }
    };
    if (asked) answer(begin + threadIdx.x, column0, score0);
    for (int64_t e = begin + threadIdx.x + blockDim.x; e < end; e += blockDim.x) {
        const uint32_t column = (uint32_t)a.given.idx[e], at = column - base;
        answer(e, column, at < n ? to_float(row[at]) : 0.f);
    }
    const auto below = [&](uint64_t limit) {      // (from memory, so that no key is kept in a register)
        uint64_t best = 0;
        for (uint32_t at = threadIdx.x; at < n; at += blockDim.x) {
            const uint64_t p = left_out(at) ? 0 : place_of(to_float(row[at]), base + at);
            best = p < limit && p > best ? p : best;
        }
        return best;
    };
    const auto each = [&](uint32_t cut, auto fn) {
        const float least = fmaxf(score_of(cut < 0x00800000u ? 0x00800000u : cut), -3.402823466e38f);
        // (eight at a time: a branch for each score that is below the cut would take longer than the comparison)
#pragma unroll
        for (int g = 0; g < E / 8; ++g) {
            float most = z[8 * g];
#pragma unroll
            for (int i = 1; i < 8; ++i) most = fmaxf(most, z[8 * g + i]);
            if (!__any(most >= least)) continue;
#pragma unroll
            for (int e = 8 * g; e < 8 * g + 8; ++e)
                if (z[e] >= least) fn(place_of(z[e], base + position(e / V) + e % V));
        }
    };
    if (whole) {
        write_law(a, r, law, mass);
        if (a.top == 0) return;
        const int found = top.finish(own, each, below, [&](int k, uint64_t p) { write_top(a, r, law, k, p); });
        write_no_top(a, r, law, found);
    } else {
        const int64_t part = local * a.segments + segment;
        if (threadIdx.x == 0) a.mass[part] = SegMass{mass, law.first};
        if (a.top == 0) return;
        uint64_t* keys = a.keys + part * a.top;
        const int found = top.finish(own, each, below, [&](int k, uint64_t p) { keys[k] = p; });
        for (int k = found + threadIdx.x; k < a.top; k += blockDim.x) keys[k] = 0;
    }
}

// A row's segments into one.
constexpr int kJoinThreads = 256;
template <typename T>
__global__ __launch_bounds__(kJoinThreads) void k_row_join(RowArgs<T> a) {
    __shared__ RowShared sh;
    const int64_t local = blockIdx.x, r = a.row0 + local;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    // all that can be asked for at once: the segments' best places (the first four a thread), masses, and given columns
    const uint64_t* keys = a.keys + local * a.segments * a.top;
    const uint32_t count = a.segments * a.top;
    uint64_t held[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const uint32_t k = j * kJoinThreads + threadIdx.x;
        held[j] = k < count ? keys[k] : 0;
    }
    const auto each_key = [&](auto fn) {
#pragma unroll
        for (int j = 0; j < 4; ++j) fn(held[j]);
        for (uint32_t k = 4 * kJoinThreads + threadIdx.x; k < count; k += kJoinThreads) fn(keys[k]);
    };
    int64_t begin, end;
    a.entries(r, &begin, &end);
    const bool asked = begin + threadIdx.x < end;
    const uint32_t column0 = asked ? (uint32_t)a.given.idx[begin + threadIdx.x] : ~0u;
    const float log0 = asked ? a.log[begin + threadIdx.x] : 0.f;
    const int32_t* list;
    int64_t listed;
    Law law;
    law.there = a.rated.row(r, &list, &listed);
    law.t = limit_of(a.temperature, a.temperature_all, r);
    const float c = law.greedy() ? 1.f : rate_of(law.t);
    if (threadIdx.x == 0) sh.first = ~0u;
    Mass mass{-INFINITY, 0.f, 0.f};
    uint32_t first = ~0u;
    if (threadIdx.x < a.segments) {
        const SegMass s = a.mass[local * a.segments + threadIdx.x];
        mass = s.mass;
        first = s.first;
    }
    const float own = mass.best;
    mass = joined(mass, c);
    if (lane == 0) sh.mass[wave] = mass;
    const Top top{&sh, a.top};
    uint32_t most = 0;
    if (a.top) {
        each_key([&](uint64_t p) { most = max(most, (uint32_t)(p >> 32)); });
        top.offer(most);
        lds_barrier();
        top.decide();
    }
    lds_barrier();
    mass = joined(lane < kJoinThreads / 64 ? sh.mass[lane] : Mass{-INFINITY, 0.f, 0.f}, c);
    law.best = mass.best;
    law.size = logf(mass.sum);
    if (law.greedy()) {
        if (own == mass.best && first != ~0u) atomicMin(&sh.first, first);
        lds_barrier();
    }
    law.first = sh.first;
    if (asked && column0 < (uint32_t)a.n) a.log[begin + threadIdx.x] = law.log_of(log0, column0);
    for (int64_t e = begin + threadIdx.x + kJoinThreads; e < end; e += kJoinThreads) {
        const uint32_t column = (uint32_t)a.given.idx[e];
        if (column < (uint32_t)a.n) a.log[e] = law.log_of(a.log[e], column);
    }
    write_law(a, r, law, mass);
    if (a.top == 0) return;
    const auto each = [&](uint32_t cut, auto fn) {
        each_key([&](uint64_t p) {
            if ((uint32_t)(p >> 32) >= cut) fn(p);
        });
    };
    const auto below = [&](uint64_t limit) {
        uint64_t best = 0;
        each_key([&](uint64_t p) { best = p < limit && p > best ? p : best; });
        return best;
    };
    const int found = top.finish(most, each, below, [&](int k, uint64_t p) { write_top(a, r, law, k, p); });
    write_no_top(a, r, law, found);
}

// ------------------------------------------------------------------------------- gradient --

template <typename T>
struct GradArgs {
    const T* z;
    int64_t rows, n, ldz;
    float temperature_all;
    int64_t of;                  // rows of the left-out columns
    int64_t entries, each;
    T* grad;
    int64_t ldg;
    float* parts;                // groups x n sums of rows
    uint32_t chunks, groups;     // of a row's columns; of rows
};

constexpr int kGradThreads = 256;
template <bool COLUMNS>
struct Grad {
    static constexpr int kEach = COLUMNS ? 8 : 16;       // columns a lane
    static constexpr int kRun = kWave * kEach, kChunk = kGradThreads * kEach;      // of a wave, of a workgroup
};

// A chunk of a row's columns, and of the rows that follow it `groups` apart, each wave having a run of them.  The
// left-out columns are marked in LDS by all of the workgroup (three rows' marks in turn: one is cleared while one is read,
// so a row takes one barrier).  The given columns each wave looks through for itself: what lies in its run goes to the
// lane that has it, in the list's order, so that sums of repeated columns are the same on every run.
// 1,024 x 17,770 fp32 in 29 us (5.0 TB/s read and written), 64 x 625,000 bf16 in 40 to 42 (3.9 TB/s): memory.  Where the last
// level of cache holds the rows, 27 (5.5 TB/s) and 33 (4.9).  With the columns' sums alone 28 + 6 us (2.1 TB/s): 8 columns a
// lane, as the sums and the next row's scores take registers (34.7 us with k_columns, 16 a lane 44), and a third of its
// instructions are a row's, not a column's.
template <typename T, bool COLUMNS>
__global__ __launch_bounds__(kGradThreads, COLUMNS ? 6 : 5) void k_gradient(
    GradArgs<T> a, const float* __restrict__ temperature, const int64_t* __restrict__ rated_ptr,
    const int32_t* __restrict__ rated_idx, const int32_t* __restrict__ users, const int64_t* __restrict__ given_ptr,
    const int32_t* __restrict__ given_idx, const float* __restrict__ log, const float* __restrict__ stats,
    const float* __restrict__ entropy, const float* __restrict__ grad_log, const float* __restrict__ grad_entropy) {
    constexpr int E = Grad<COLUMNS>::kEach, V = 16 / sizeof(T), kMarks = Grad<COLUMNS>::kChunk / 32;
    constexpr uint32_t kRun = Grad<COLUMNS>::kRun, kChunk = Grad<COLUMNS>::kChunk;
    __shared__ uint32_t marks[3 * kMarks];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t chunk = blockIdx.x % a.chunks, group = blockIdx.x / a.chunks;
    const uint32_t start = chunk * kChunk, base = start + wave * kRun, n = (uint32_t)a.n;
    const auto position = [&](int v) { return base + (uint32_t)(v * kWave + lane) * V; };
    const bool inside = base + kRun <= n;

    // What a row needs, in the order in which it can be asked for: where its lists lie, then their first entries
    // and the scores.
    struct Place {
        int64_t rated, rated_end, begin, end;
        bool there;
    };
    struct Fetched {
        T z[E];
        uint32_t rated, given;
        float g, log;
        float t, best, size, h, spread;
    };
    const auto place_of_row = [&](int64_t r) {
        Place p{0, 0, r * a.each, (r + 1) * a.each, true};
        if (rated_ptr) {
            const int64_t u = users ? (int64_t)users[r] : r;
            p.there = u >= 0 && u < a.of;
            if (p.there) {
                p.rated = rated_ptr[u];
                p.rated_end = rated_ptr[u + 1];
            }
        }
        if (given_ptr) {
            p.begin = given_ptr[r];
            p.end = given_ptr[r + 1];
            p.begin = p.begin < 0 ? 0 : p.begin;
            p.end = p.end > a.entries ? a.entries : p.end;
        }
        return p;
    };
    const auto fetch = [&](int64_t r, const Place& p) {
        Fetched f;
        const T* row = a.z + r * a.ldz;
#pragma unroll
        for (int v = 0; v < E / V; ++v) {
            const uint32_t c = position(v);
            if (inside) {
                __builtin_memcpy(&f.z[v * V], row + c, V * sizeof(T));
            } else {
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    from_float(-INFINITY, &f.z[v * V + i]);
                    if (c + i < n) f.z[v * V + i] = row[c + i];
                }
            }
        }
        f.rated = p.rated + threadIdx.x < p.rated_end ? (uint32_t)rated_idx[p.rated + threadIdx.x] : ~0u;
        const bool in = p.begin + lane < p.end;
        f.given = in ? (uint32_t)given_idx[p.begin + lane] : ~0u;
        f.g = in ? grad_log[p.begin + lane] : 0.f;
        f.log = in ? log[p.begin + lane] : -INFINITY;
        f.t = limit_of(temperature, a.temperature_all, r);
        f.best = stats[2 * r];
        f.size = stats[2 * r + 1];
        f.h = grad_entropy ? grad_entropy[r] : 0.f;
        f.spread = grad_entropy ? entropy[r] : 0.f;
        return f;
    };
    float total[E];
#pragma unroll
    for (int e = 0; e < E; ++e) total[e] = 0.f;
    int turn = 0;
    if (rated_ptr) {
        for (int w = threadIdx.x; w < 3 * kMarks; w += kGradThreads) marks[w] = 0;
        lds_barrier();
    }
    // with the columns' sums a workgroup has several rows: the next one's values and the places after it are on their
    // way while a row is worked on
    const auto after = [&](int64_t r) { return r + a.groups < a.rows ? r + a.groups : r; };
    Place place = place_of_row(group), place_after = COLUMNS ? place_of_row(after(group)) : Place{};
    Fetched now = fetch(group, place);
    for (int64_t r = group; r < a.rows; r += a.groups) {
        const Place p = place;
        const Fetched f = now;
        if (COLUMNS) {
            now = fetch(after(r), place_after);
            place = place_after;
            place_after = place_of_row(after(after(r)));
        }
        const bool there = p.there;
        const int64_t begin = p.begin, end = p.end;
        const float t = f.t, best = f.best, size = f.size, h = f.h, spread = f.spread;
        const bool some = there && t > 0.f && best > -INFINITY;
        if (rated_ptr) {
            if (some) {
                const auto mark = [&](uint32_t column) {
                    const uint32_t at = column - start;
                    if (at < kChunk) atomicOr(&marks[turn * kMarks + (at >> 5)], 1u << (at & 31));
                };
                mark(f.rated);
                for (int64_t k = p.rated + threadIdx.x + kGradThreads; k < p.rated_end; k += kGradThreads)
                    mark((uint32_t)rated_idx[k]);
            }
            lds_barrier();
        }
        const uint32_t* marked = marks + turn * kMarks;
        if (rated_ptr) {
            turn = turn == 2 ? 0 : turn + 1;
            const int clear = turn == 2 ? 0 : turn + 1;
            for (int w = threadIdx.x; w < kMarks; w += kGradThreads) marks[clear * kMarks + w] = 0;
        }
        float d[E];
        if (some) {
            // (1 / T of the smallest T overflows: the rest of it then comes as a power of two)
            const float boost = t < 0x1p-100f ? 0x1p64f : 1.f, inverse = 1.f / (t * boost);
            float sum = 0.f;
#pragma unroll
            for (int e = 0; e < E; ++e) d[e] = 0.f;
            for (int64_t k0 = begin; k0 < end; k0 += kWave) {
                uint32_t column = f.given;
                float g = f.g, entry = f.log;
                if (k0 != begin) {
                    const bool in = k0 + lane < end;
                    column = in ? (uint32_t)given_idx[k0 + lane] : ~0u;
                    g = in ? grad_log[k0 + lane] : 0.f;
                    entry = in ? log[k0 + lane] : -INFINITY;
                }
                const bool counts = entry > -INFINITY;
                const uint32_t at = counts ? column - base : ~0u;
                const float w = counts ? g : 0.f;
                sum += w;
                uint64_t in = __ballot(at < kRun);
                while (in) {
                    const int l = __builtin_ctzll(in);
                    in &= in - 1;
                    const uint32_t to = __builtin_amdgcn_readlane(at, l), place = to / (V * kWave) * V + to % V;
                    const float more = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, w), l));
                    if (lane == to / V % kWave) {
#pragma unroll
                        for (int e = 0; e < E; ++e) d[e] += e == place ? more : 0.f;
                    }
                }
            }
            sum = wave_sum(sum);
            const float c = fminf(kLog2E / t, 3.402823466e38f), shift = size * kLog2E;
            const float constant = fmaf(h, spread, sum) * inverse, slope = h * kLn2 * inverse;
            const auto each = [&](auto endless) {
#pragma unroll
                for (int v = 0; v < E / V; ++v) {
                    const uint32_t at = position(v) - start;
                    const uint32_t out = rated_ptr ? marked[at >> 5] >> (at & 31) : 0;      // V divides 32
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        const int e = v * V + i;
                        // a left-out score becomes NaN, which weighs nothing
                        const float s = __builtin_bit_cast(
                            float, __builtin_bit_cast(uint32_t, to_float(f.z[e])) | (uint32_t)((int32_t)(out << (31 - i)) >> 31));
                        // (of equal best scores +inf: their difference is 0, of a finite one and +inf -inf)
                        const float x = fmaxf(fmaf(endless.value ? (s == best ? 0.f : -INFINITY) : s - best, c, -shift), kNothing);
                        d[e] = fmaf(d[e], inverse, -(__builtin_amdgcn_exp2f(x) * fmaf(slope, x, constant)));
                    }
                }
            };
            if (best == INFINITY) each(std::true_type());
            else each(std::false_type());
            if (boost != 1.f) {
#pragma unroll
                for (int e = 0; e < E; ++e) d[e] *= boost;
            }
        } else {
            const float all = there && !(best != best) ? 0.f : NAN;
#pragma unroll
            for (int e = 0; e < E; ++e) d[e] = all;
        }
        if (COLUMNS) {
#pragma unroll
            for (int e = 0; e < E; ++e) total[e] += d[e];
        }
        if (a.grad) {
            T* to = a.grad + r * a.ldg;
#pragma unroll
            for (int v = 0; v < E / V; ++v) {
                const uint32_t c = position(v);
                T w[V];
                from_floats<V>(&d[v * V], w);
                if (inside) {
                    __builtin_memcpy(to + c, w, sizeof w);
                } else {
#pragma unroll
                    for (int i = 0; i < V; ++i)
                        if (c + i < n) to[c + i] = w[i];
                }
            }
        }
        if (!COLUMNS && r + a.groups < a.rows) {
            place = place_of_row(r + a.groups);
            now = fetch(r + a.groups, place);
        }
    }
    if (COLUMNS) {
        float* to = a.parts + (int64_t)group * n;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const uint32_t c = position(e / V) + e % V;
            if (c < n) to[c] = total[e];
        }
    }
}

// The groups' sums into one: runs of groups, eight at a time, then across the runs.
constexpr int kRuns = 16;
__global__ __launch_bounds__(kRuns * kWave) void k_columns(const float* __restrict__ parts, uint32_t groups, int64_t n,
                                                           float* __restrict__ columns) {
    __shared__ float runs[kRuns][kWave];
    const int lane = threadIdx.x & 63, run = threadIdx.x >> 6;
    const int64_t c = (int64_t)blockIdx.x * kWave + lane;
    float sum = 0.f;
    if (c < n) {
        for (uint32_t g = run; g < groups; g += 8 * kRuns) {
            float v[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = g + k * kRuns < groups ? parts[(g + k * kRuns) * n + c] : 0.f;
#pragma unroll
            for (int k = 0; k < 8; ++k) sum += v[k];
        }
    }
    runs[run][lane] = sum;
    __syncthreads();
    if (run == 0 && c < n) {
#pragma unroll
        for (int k = 1; k < kRuns; ++k) sum += runs[k][lane];
        columns[c] = sum;
    }
}

constexpr size_t kWorkspaceBytes = 128u << 20, kWorkspaceMost = (size_t)1 << 34;

}  // namespace

struct als_predict_ctx {
    int device;
    int cus;
    unsigned char* ws;
    size_t ws_bytes;
    int last_hip;
};

namespace {

int finish(als_predict_ctx* ctx) {
    const hipError_t e = hipGetLastError();
    if (e == hipSuccess) return ALS_OK;
    ctx->last_hip = (int)e;
    return ALS_ERR_HIP;
}

// fn(a null pointer to the type)
template <typename Fn>
void by_type(int dtype, Fn fn) {
    if (dtype == ALS_F32) fn((const float*)nullptr);
    else if (dtype == ALS_F16) fn((const F16*)nullptr);
    else fn((const BF16*)nullptr);
}
template <typename P>
using Type = std::remove_cv_t<std::remove_pointer_t<P>>;

constexpr int64_t kCache = 256 << 20;      // of the last level

// The product's tiles in one launch, and where there are few of them f in parts of 4 steps at least, as many as give every CU
// two workgroups and the workspace holds.
template <typename Kernel>
void launch_product(const als_predict_ctx* ctx, Kernel kernel, Product a, int users, int items, int values, int threads,
                    int lds, hipStream_t st) {
    a.tu = (uint32_t)((a.m + users - 1) / users);
    a.ti = (uint32_t)((a.n + items - 1) / items);
    // Where the results' bytes count (f up to 128) and no cache holds them, rows of tiles next to one another write what lies
    // side by side: 4,096 x 40,000 x 128 bf16 150 us at height 2, 159 at 4, 179 at 8; 1,024 x 17,770 21.7, 20.6, 20.8.
    a.height = a.f <= 128 && a.m * a.n * (a.end.type == ALS_F32 ? 4 : 2) > kCache ? 2 : 8;
    const int64_t steps = (a.f - a.tail + values - 1) / values, tiles = (int64_t)a.tu * a.ti;
    int64_t parts = 2 * ctx->cus / tiles;
    if (parts > steps / 4) parts = steps / 4;
    const int64_t fit = (int64_t)(ctx->ws_bytes / 4) / (a.m * a.n);
    if (parts > fit) parts = fit;
    if (parts < 1) parts = 1;
    a.steps = (int)((steps + parts - 1) / parts);
    parts = (steps + a.steps - 1) / a.steps;
    a.parts = parts > 1 ? (float*)ctx->ws : nullptr;
    hipLaunchKernelGGL(kernel, dim3((unsigned)tiles, (unsigned)parts), dim3(threads), kHead + lds, st, a);
    if (parts > 1) {
        const int64_t fours = a.m * ((a.n + 3) / 4);
        hipLaunchKernelGGL(k_join, dim3((unsigned)((fours + 255) / 256)), dim3(256), 0, st, a, (int)parts);
    }
}

template <typename T, int WU, int WI, int FU, int FI>
void staged(const als_predict_ctx* ctx, Product a, hipStream_t st) {
    using C = Staged<T, WU, WI, FU, FI>;
    static std::atomic<uint64_t> done{0};
    auto* kernel = k_product<T, WU, WI, FU, FI>;
    whole_lds(kernel, ctx->device, &done);
    if (sizeof(T) == 4 && a.f > C::P::kValues && a.f % C::P::kValues <= 8) a.tail = a.f % C::P::kValues;
    launch_product(ctx, kernel, a, C::kUsers, C::kItems, C::P::kValues, C::kThreads, C::kLds, st);
}

template <typename T, int WU, int WI, int FU, int FI, int STEP, int STAGES>
void direct(const als_predict_ctx* ctx, const Product& a, hipStream_t st) {
    using C = Direct<WU, WI, FU, FI, STEP, STAGES>;
    static std::atomic<uint64_t> done{0};
    auto* kernel = k_product_lds<T, WU, WI, FU, FI, STEP, STAGES>;
    whole_lds(kernel, ctx->device, &done);
    const int steps = (a.f + STEP - 1) / STEP, rows = (steps < STAGES ? steps : STAGES) * C::kStage;
    launch_product(ctx, kernel, a, C::kUsers, C::kItems, STEP, C::kThreads, rows > C::kOutBytes ? rows : C::kOutBytes, st);
}

// The tile.  Few users: as few rows for them as hold them.  Otherwise the largest that still gives every CU enough of them, and
// up to f = 128, where the results' way out counts, a smaller one, of which a CU holds more at a time.  Tiles come in rounds of
// as many as the CUs hold at once, so what a shape costs goes by its rounds' whole area (`rounds`), filled or not.  Measured (us,
// users x items x f):
//   bf16   4,096 x 8,192 x 8,192      256 x 256 427 (the library's product 406)
//          310 x 38,418 x 2,568       256 x 256 155 (two rounds, the second all but empty), 128 x 128 119, 64 x 128 133
//          1,024 x 8,192 x 8,192      256 x 256 153, 128 x 128 135, 64 x 128 198
//          1,000 x 9,000 x 1,000      256 x 256 69, 128 x 128 41, 64 x 128 37, 64 x 64 45
//          600 x 5,000 x 2,000        128 x 128 29, 64 x 128 28, 64 x 64 36
//          2,048 x 2,048 x 1,024      128 x 128 24, 64 x 128 14, 64 x 64 18
//          4,096 x 40,000 x 128       64 x 128 in steps of 32 values 139, of 64 153; 128 x 128 of 32 135, of 64 160
//          1,024 x 17,770 x 128       64 x 128 in steps of 32 values 19.9, of 64 20.9; 128 x 128 of 32 20.6, of 64 24.5
//          25 x 100,000 x 1,000       128 x 128 78, 64 x 128 54, 64 x 64 49, 32 x 128 50
//          5 x 8,192 x 8,192          16 x 64 25.5 (the library's product 23; both with the weights in the last-level cache)
//   fp32   1,024 x 17,770 x 100       64 x 128 45, 64 x 64 46, 128 x 64 47, 128 x 128 51 (before the values behind steps)
//          2,000 x 9,000 x 500        64 x 128 122, 64 x 64 134, 128 x 128 128
//          500 x 9,000 x 1,000        64 x 128 78, 64 x 64 85, 128 x 128 93
//          100 x 50,000 x 200         64 x 128 33 (14 of 782 tiles are left for a second round), 64 x 64 27, 128 x 128 27
//          25 x 221,853 x 80          64 x 128 33, 64 x 64 31, 32 x 128 26, 32 x 64 24
template <typename T>
void product(const als_predict_ctx* ctx, const Product& a, hipStream_t st) {
    const auto tiles = [&](int64_t users, int64_t items) {
        return ((a.m + users - 1) / users) * ((a.n + items - 1) / items);
    };
    const auto rounds = [&](int64_t users, int64_t items, int64_t on_a_cu) {
        const int64_t at_once = ctx->cus * on_a_cu;
        return (double)((tiles(users, items) + at_once - 1) / at_once * at_once) * (double)(users * items);
    };
    if constexpr (sizeof(T) == 2) {
        const auto near = [](const void* p, int64_t ld) { return aligned(p, 16) && ld % 8 == 0 && ld < kNear; };
        // (an X without rows, whose users all do not exist, is k_product's, which loads nothing for them)
        if (a.of > 0 && near(a.x, a.ldx) && near(a.theta, a.ldt) && (!a.users || a.of < (int64_t)(kPastEnd / 2) / a.ldx)) {
            if (a.m <= 16) return direct<T, 1, 2, 1, 2, 64, 4>(ctx, a, st);
            if (a.f > 128) {
                if (a.m <= 32) return direct<T, 1, 4, 2, 2, 64, 3>(ctx, a, st);
                if (a.f >= 512 && tiles(256, 256) >= ctx->cus && rounds(256, 256, 1) <= 1.4 * rounds(128, 128, 2))
                    return direct<T, 2, 4, 8, 4, 64, 2>(ctx, a, st);
                if (a.m > 64 && tiles(128, 128) >= 2 * ctx->cus) return direct<T, 2, 2, 4, 4, 64, 2>(ctx, a, st);
                if (2 * tiles(64, 128) >= 3 * ctx->cus) return direct<T, 2, 2, 2, 4, 64, 2>(ctx, a, st);
            } else if (tiles(64, 128) >= 2 * ctx->cus) {
                return direct<T, 2, 2, 2, 4, 32, 3>(ctx, a, st);
            }
            return direct<T, 2, 2, 2, 2, 64, 4>(ctx, a, st);
        }
    }
    if (a.m <= 16) return staged<T, 1, 4, 1, 1>(ctx, a, st);
    if (a.m <= 32) return staged<T, 1, 4, 2, 1>(ctx, a, st);
    const double wide = 1.2 * rounds(64, 128, 3), narrow = 1.15 * rounds(64, 64, 4);
    if (a.f > 128 && a.m > 64 && rounds(128, 128, 2) <= wide && rounds(128, 128, 2) <= narrow)
        return staged<T, 2, 2, 4, 4>(ctx, a, st);
    if (wide <= narrow) return staged<T, 2, 2, 2, 4>(ctx, a, st);
    return staged<T, 2, 2, 2, 2>(ctx, a, st);
}

// A row's registers: as many scores a thread as E; longer rows in segments.
constexpr int64_t kHeld = 32 * 1024;
constexpr int64_t kSegment = 20480;
static_assert(ALS_PREDICT_N_MAX <= kSegment * kJoinThreads, "a thread a segment");

int check_scores(const als_scores* s, const als_given* g) {
    if (!s || !g || s->rows < 0 || s->n < 0 || s->n > ALS_PREDICT_N_MAX || s->dtype < ALS_F32 || s->dtype > ALS_BF16 ||
        s->ldz < s->n || s->of < 0 || s->rows > INT32_MAX || g->entries < 0 || g->each < 0)
        return ALS_ERR_INVALID_ARG;
    if (!s->rated_ptr != !s->rated_idx || (s->users && !s->rated_ptr) || (s->rated_ptr && !s->users && s->of < s->rows))
        return ALS_ERR_INVALID_ARG;
    // (without entries each is 0; a quotient, as the product may not fit)
    if (!g->ptr && (s->rows == 0 || g->each == 0 ? g->entries != 0
                                                 : g->entries % s->rows != 0 || g->entries / s->rows != g->each))
        return ALS_ERR_INVALID_ARG;
    if ((s->rows > 0 && s->n > 0 && !s->z) || (g->entries > 0 && !g->idx)) return ALS_ERR_INVALID_ARG;
    if (!aligned(s->z, type_bytes(s->dtype)) || !aligned(s->temperature, 4) || !aligned(s->rated_ptr, 8) ||
        !aligned(s->rated_idx, 4) || !aligned(s->users, 4) || !aligned(g->ptr, 8) || !aligned(g->idx, 4))
        return ALS_ERR_ALIGN;
    return ALS_OK;
}

// Whether an output lies on one of the inputs (but on the scores, where `beside_scores` says so).
bool on_inputs(const void* o, uint64_t bytes, const als_scores* s, const als_given* g, bool beside_scores = false) {
    const uint64_t rn = (uint64_t)s->rows * 4;
    return (!beside_scores && overlap(o, bytes, s->z, span_of(s->rows, s->n, s->ldz, type_bytes(s->dtype)))) ||
           overlap(o, bytes, s->temperature, rn) || overlap(o, bytes, s->rated_ptr, ((uint64_t)s->of + 1) * 8) ||
           overlap(o, bytes, s->users, rn) || overlap(o, bytes, g->ptr, ((uint64_t)s->rows + 1) * 8) ||
           overlap(o, bytes, g->idx, (uint64_t)g->entries * 4);
}

template <typename T>
RowArgs<T> row_args(const als_scores* s, const als_given* g) {
    RowArgs<T> a{};
    a.z = (const T*)s->z;
    a.rows = s->rows;
    a.n = s->n;
    a.ldz = s->ldz;
    a.temperature = s->temperature;
    a.temperature_all = s->temperature_all;
    a.rated = Rated{s->rated_ptr, s->rated_idx, s->users, s->of};
    a.given = *g;
    a.segments = 1;
    a.columns = (uint32_t)(s->n > 0 ? s->n : 1);
    return a;
}

}  // namespace

extern "C" {

size_t als_predict_workspace_bytes(int device) {
    int cus = 0;
    return query_device(device, &cus) == ALS_OK ? kWorkspaceBytes : 0;
}

int als_predict_init(als_predict_ctx** out, int device, void* workspace, size_t workspace_bytes) {
    if (!out) return ALS_ERR_INVALID_ARG;
    *out = nullptr;
    if (!workspace) return ALS_ERR_WORKSPACE;
    if (!aligned(workspace, 256)) return ALS_ERR_ALIGN;
    int cus = 0;
    if (const int rc = query_device(device, &cus); rc != ALS_OK) return rc;
    if (workspace_bytes < kWorkspaceBytes) return ALS_ERR_WORKSPACE;
    als_predict_ctx* ctx = new (std::nothrow) als_predict_ctx();
    if (!ctx) return ALS_ERR_INVALID_ARG;
    ctx->device = device;
    ctx->cus = cus;
    ctx->ws = (unsigned char*)workspace;
    ctx->ws_bytes = workspace_bytes < kWorkspaceMost ? workspace_bytes : kWorkspaceMost;
    ctx->last_hip = 0;
    *out = ctx;
    return ALS_OK;
}

int als_predict_destroy(als_predict_ctx* ctx) {
    delete ctx;
    return ALS_OK;
}

int als_predict_last_hip_error(const als_predict_ctx* ctx) { return ctx ? ctx->last_hip : 0; }

int als_predict(als_predict_ctx* ctx, const void* x, int64_t of, int64_t ldx, const int32_t* users, int64_t m,
                const void* theta, int64_t n, int64_t ldt, int32_t dtype, int32_t f, const float* user_offset,
                const float* item_offset, int32_t activation, float low, float high, const void* residual,
                int64_t ldr, void* out, int64_t ldo, int32_t out_dtype, void* stream) {
    if (!ctx || of < 0 || m < 0 || n < 0 || dtype < ALS_F32 || dtype > ALS_BF16 || out_dtype < ALS_F32 ||
        out_dtype > ALS_BF16 || activation < ALS_ACT_NONE || activation > ALS_ACT_TANH)
        return ALS_ERR_INVALID_ARG;
    if (f < 1 || f > ALS_PREDICT_F_MAX) return ALS_ERR_UNSUPPORTED_F;
    if (ldx < f || ldt < f || ldo < n || (residual && ldr < n) || (!users && m > of) ||
        (activation == ALS_ACT_CLIP && !(low <= high)))
        return ALS_ERR_INVALID_ARG;
    if (m == 0 || n == 0) return ALS_OK;
    if (!theta || !out || (of > 0 && !x)) return ALS_ERR_INVALID_ARG;
    const size_t in = type_bytes(dtype), each = type_bytes(out_dtype);
    if (!aligned(x, in) || !aligned(theta, in) || !aligned(users, 4) || !aligned(user_offset, 4) ||
        !aligned(item_offset, 4) || !aligned(residual, each) || !aligned(out, each))
        return ALS_ERR_ALIGN;
    const uint64_t on = span_of(m, n, ldo, each);
    if (overlap(out, on, x, span_of(of, f, ldx, in)) || overlap(out, on, theta, span_of(n, f, ldt, in)) ||
        overlap(out, on, users, (uint64_t)m * 4) || overlap(out, on, user_offset, (uint64_t)of * 4) ||
        overlap(out, on, item_offset, (uint64_t)n * 4) ||
        (!(residual == out && ldr == ldo) && overlap(out, on, residual, span_of(m, n, ldr, each))))
        return ALS_ERR_ALIAS;
    DeviceGuard guard(ctx->device);
    if (!guard.ok) return ALS_ERR_DEVICE;
    const hipStream_t st = (hipStream_t)stream;
    // Launches of at most 2^31 threads (a tile takes 256 for 16 users and 64 items at least): the users in parts of
    // whole tiles, and the items where one row of tiles is too long already.
    const int64_t most = (kMaxThreads / 2) / 256;
    const int64_t items = (n + 63) / 64 < most ? n : most * 64;
    const int64_t fit = most / ((items + 63) / 64) * 16, users_at_once = m < fit ? m : (fit >= 128 ? fit / 128 * 128 : fit);
    by_type(dtype, [&](auto* p) {
        using T = Type<decltype(p)>;
        for (int64_t i = 0; i < m; i += users_at_once)
            for (int64_t j = 0; j < n; j += items) {
                Product a{};
                a.x = users ? x : (const T*)x + i * ldx;
                a.of = users ? of : of - i;
                a.ldx = ldx;
                a.users = users ? users + i : nullptr;
                a.m = m - i < users_at_once ? m - i : users_at_once;
                a.theta = (const T*)theta + j * ldt;
                a.n = n - j < items ? n - j : items;
                a.ldt = ldt;
                a.f = f;
                a.end = Epilogue{user_offset ? user_offset + (users ? 0 : i) : nullptr,
                                 item_offset ? item_offset + j : nullptr,
                                 residual ? (const char*)residual + (i * ldr + j) * each : nullptr, ldr,
                                 (char*)out + (i * ldo + j) * each, ldo, low, high, activation, out_dtype};
                product<T>(ctx, a, st);
            }
    });
    return finish(ctx);
}

int als_log_prob(als_predict_ctx* ctx, const als_scores* scores, const als_given* given, float* log, float* stats,
                 float* entropy, int32_t top, int32_t* top_index, float* top_log, void* stream) {
    if (!ctx) return ALS_ERR_INVALID_ARG;
    if (const int rc = check_scores(scores, given); rc != ALS_OK) return rc;
    const als_scores& s = *scores;
    if (top < 0 || top > ALS_PREDICT_TOP_MAX || (given->entries > 0 && !log)) return ALS_ERR_INVALID_ARG;
    if (!aligned(log, 4) || !aligned(stats, 4) || !aligned(entropy, 4) || !aligned(top_index, 4) || !aligned(top_log, 4))
        return ALS_ERR_ALIGN;
    const uint64_t rn = (uint64_t)s.rows * 4;
    const void* outs[5] = {log, stats, entropy, top_index, top_log};
    const uint64_t bytes[5] = {(uint64_t)given->entries * 4, 2 * rn, rn, rn * top, rn * top};
    for (int i = 0; i < 5; ++i) {
        if (on_inputs(outs[i], bytes[i], scores, given)) return ALS_ERR_ALIAS;
        for (int j = 0; j < i; ++j)
            if (overlap(outs[i], bytes[i], outs[j], bytes[j])) return ALS_ERR_ALIAS;
    }
    if (s.rows == 0) return ALS_OK;
    DeviceGuard guard(ctx->device);
    if (!guard.ok) return ALS_ERR_DEVICE;
    by_type(s.dtype, [&](auto* p) {
        using T = Type<decltype(p)>;
        RowArgs<T> a = row_args<T>(scores, given);
        a.log = log;
        a.stats = stats;
        a.entropy = entropy;
        a.top = top_index || top_log ? top : 0;
        a.top_index = top_index;
        a.top_log = top_log;
        const auto go = [&](auto each, int64_t rows) {
            constexpr int E = decltype(each)::value;
            const int64_t threads = ((int64_t)a.columns + E - 1) / E, waves = (threads + kWave - 1) / kWave;
            const size_t lds = s.rated_ptr ? (size_t)(a.columns + 31) / 32 * 4 : 0;
            const int64_t row0 = a.row0;
            in_parts(rows, kMaxThreads / (kWave * waves * a.segments), [&](int64_t first, int64_t some) {
                a.row0 = row0 + first;
                hipLaunchKernelGGL((k_row<T, E>), dim3((unsigned)(some * a.segments)), dim3((unsigned)(kWave * waves)),
                                   lds, (hipStream_t)stream, a);
            });
            a.row0 = row0;
        };
        using std::integral_constant;
        if (s.n <= kHeld) {
            if (s.n <= 1024) return go(integral_constant<int, 8>(), s.rows);
            if (s.n <= 16384) return go(integral_constant<int, 16>(), s.rows);
            return go(integral_constant<int, 40>(), s.rows);
        }
        a.segments = (uint32_t)((s.n + kSegment - 1) / kSegment);
        a.columns = kSegment;
        const size_t a_row = a.segments * (sizeof(SegMass) + a.top * sizeof(uint64_t));
        int64_t batch = (int64_t)(ctx->ws_bytes / a_row);
        const int64_t most = kMaxThreads / (1024 * a.segments);
        if (batch > most) batch = most;
        a.keys = (uint64_t*)ctx->ws;
        for (int64_t row0 = 0; row0 < s.rows; row0 += batch) {
            const int64_t some = s.rows - row0 < batch ? s.rows - row0 : batch;
            a.mass = (SegMass*)(ctx->ws + some * a.segments * a.top * sizeof(uint64_t));
            a.row0 = row0;
            go(integral_constant<int, 40>(), some);
            hipLaunchKernelGGL(k_row_join<T>, dim3((unsigned)some), dim3(kJoinThreads), 0, (hipStream_t)stream, a);
        }
    });
    return finish(ctx);
}

int als_log_prob_grad(als_predict_ctx* ctx, const als_scores* scores, const als_given* given, const float* log,
                      const float* stats, const float* entropy, const float* grad_log, const float* grad_entropy,
                      void* grad, int64_t ldg, float* columns, void* stream) {
    if (!ctx) return ALS_ERR_INVALID_ARG;
    if (const int rc = check_scores(scores, given); rc != ALS_OK) return rc;
    const als_scores& s = *scores;
    if ((given->entries > 0 && (!log || !grad_log)) || (s.rows > 0 && !stats) ||
        (s.rows > 0 && grad_entropy && !entropy) || (grad && ldg < s.n))
        return ALS_ERR_INVALID_ARG;
    const size_t each = type_bytes(s.dtype);
    if (!aligned(log, 4) || !aligned(stats, 4) || !aligned(entropy, 4) || !aligned(grad_log, 4) ||
        !aligned(grad_entropy, 4) || !aligned(grad, each) || !aligned(columns, 4))
        return ALS_ERR_ALIGN;
    const uint64_t rn = (uint64_t)s.rows * 4, en = (uint64_t)given->entries * 4, cn = (uint64_t)s.n * 4;
    const uint64_t gn = grad ? span_of(s.rows, s.n, ldg, each) : 0;
    const bool in_place = grad == s.z && ldg == s.ldz;
    const auto on_more = [&](const void* o, uint64_t bytes) {
        return overlap(o, bytes, log, en) || overlap(o, bytes, stats, 2 * rn) || overlap(o, bytes, entropy, rn) ||
               overlap(o, bytes, grad_log, en) || overlap(o, bytes, grad_entropy, rn);
    };
    if (on_inputs(grad, gn, scores, given, in_place) || on_inputs(columns, cn, scores, given) || on_more(grad, gn) ||
        on_more(columns, cn) || overlap(grad, gn, columns, cn))
        return ALS_ERR_ALIAS;
    if (s.n == 0 || (!grad && !columns) || (s.rows == 0 && !columns)) return ALS_OK;
    DeviceGuard guard(ctx->device);
    if (!guard.ok) return ALS_ERR_DEVICE;
    const hipStream_t st = (hipStream_t)stream;
    // a workgroup takes one row's chunk, or with the columns' sums as many rows as leave every CU eight workgroups (it has six
    // of them at a time, at 80 registers, so that at 1,024 x 17,770 the last quarter is a round of its own)
    int64_t groups = 0;
    by_type(s.dtype, [&](auto* p) {
        using T = Type<decltype(p)>;
        const int64_t chunk = columns ? Grad<true>::kChunk : Grad<false>::kChunk, chunks = (s.n + chunk - 1) / chunk;
        groups = s.rows;
        if (columns) {
            const int64_t wanted = (8 * ctx->cus + chunks - 1) / chunks, fit = (int64_t)(ctx->ws_bytes / 4) / s.n;
            groups = groups < wanted ? groups : wanted;
            groups = groups < fit ? groups : fit;
        }
        const int64_t most = kMaxThreads / kGradThreads / chunks;
        groups = groups < most ? groups : most;
        if (groups == 0) return;
        const GradArgs<T> g{(const T*)s.z, s.rows, s.n, s.ldz, s.temperature_all, s.of, given->entries, given->each,
                            (T*)grad, ldg, (float*)ctx->ws, (uint32_t)chunks, (uint32_t)groups};
        const auto go = [&](auto* kernel) {
            hipLaunchKernelGGL(kernel, dim3((unsigned)(chunks * groups)), dim3(kGradThreads), 0, st, g, s.temperature,
                               s.rated_ptr, s.rated_idx, s.users, given->ptr, given->idx, log, stats, entropy, grad_log,
                               grad_entropy);
        };
        if (columns) go(k_gradient<T, true>);
        else go(k_gradient<T, false>);
    });
    if (columns)
        hipLaunchKernelGGL(k_columns, dim3((unsigned)((s.n + kWave - 1) / kWave)), dim3(kRuns * kWave), 0, st,
                           (const float*)ctx->ws, (uint32_t)groups, s.n, columns);
    return finish(ctx);
}

}  // extern "C"
