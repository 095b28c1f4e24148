// lba_layer_device.h -- what the operators of lba_layer.h share on the device: element types in registers, 8-bit codes,
// activations, the dropout generator and sums over a wave.
#ifndef LBA_LAYER_DEVICE_H_
#define LBA_LAYER_DEVICE_H_

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "lba_layer.h"

namespace lba {

typedef __bf16 bf16_t;

// vectors of the element's own alignment: rows start anywhere, and the memory system takes unaligned vectors
template <typename T, int V> struct Vec { typedef T type __attribute__((ext_vector_type(V), aligned(sizeof(T)))); };
template <typename T> struct Vec<T, 1> { typedef T type; };

// an output format of 8-bit codes as the encoder uses it
struct CodeFmt {
    float scale;             // 2^(bias - canonical bias)
    float top;               // largest value at the canonical bias
    float sub;               // 2^(emin - man + 23): adding it rounds to the subnormal grid
    float norm;              // 2^emin, the smallest normal number
    int32_t sh;              // 23 - man_bits
    int32_t off;             // (127 - canonical bias) << man_bits
    int32_t e4m3;            // 1: exp_bits 4, the hardware conversion rounds as the format does
};

inline CodeFmt make_code_fmt(const lba_infmt& f) {
    CodeFmt c;
    const int bc = (1 << (f.exp_bits - 1)) - 1, emin = 1 - bc;
    c.scale = __builtin_ldexpf(1.0f, f.bias - bc);
    c.e4m3 = f.exp_bits == 4 ? 1 : 0;
    c.top = c.e4m3 ? 448.0f : __builtin_ldexpf(2.0f - __builtin_ldexpf(1.0f, -f.man_bits), (1 << f.exp_bits) - 1 - bc);
    c.sub = __builtin_ldexpf(1.0f, emin - f.man_bits + 23);
    c.norm = __builtin_ldexpf(1.0f, emin);
    c.sh = 23 - f.man_bits;
    c.off = (127 - bc) << f.man_bits;
    return c;
}

__device__ __forceinline__ uint32_t code_one(float v, const CodeFmt& c) {
    const uint32_t sign = (__float_as_uint(v) >> 24) & 0x80u;
    const float u = fabsf(v) * c.scale;
    const uint32_t b = __float_as_uint(u > c.top ? c.top : u);
    uint32_t code = ((b + ((1u << (c.sh - 1)) - 1u) + ((b >> c.sh) & 1u)) >> c.sh) - (uint32_t)c.off;
    if (u < c.norm) code = __float_as_uint(u + c.sub) - __float_as_uint(c.sub);
    if (u != u) code = 0x7Fu;
    return code | sign;
}

// four values -> four codes of one word, the first in the low byte
__device__ __forceinline__ uint32_t code_four(float a, float b, float c, float d, const CodeFmt& f) {
    if (f.e4m3) {
        const float v[4] = {a, b, c, d};
        float s[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            // these keep a NaN, for which the conversion writes 0x7f or 0xff
            s[j] = __builtin_elementwise_minimum(__builtin_elementwise_maximum(v[j] * f.scale, -448.0f), 448.0f);
        }
        int w = __builtin_amdgcn_cvt_pk_fp8_f32(s[0], s[1], 0, false);
        return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(s[2], s[3], w, true);
    }
    return code_one(a, f) | (code_one(b, f) << 8) | (code_one(c, f) << 16) | (code_one(d, f) << 24);
}

// V consecutive elements <-> float registers
template <int V> __device__ __forceinline__ void load_vec(const float* p, float (&v)[V]) {
    const typename Vec<float, V>::type x = *(const typename Vec<float, V>::type*)p;
#pragma unroll
    for (int j = 0; j < V; ++j) v[j] = x[j];
}
template <int V> __device__ __forceinline__ void load_vec(const bf16_t* p, float (&v)[V]) {
    const typename Vec<uint16_t, V>::type x = *(const typename Vec<uint16_t, V>::type*)p;
#pragma unroll
    for (int j = 0; j < V; ++j) v[j] = __uint_as_float((uint32_t)x[j] << 16);
}
template <int V> __device__ __forceinline__ void store_vec(float* p, const float (&v)[V], const CodeFmt&) {
    typename Vec<float, V>::type x;
#pragma unroll
    for (int j = 0; j < V; ++j) x[j] = v[j];
    *(typename Vec<float, V>::type*)p = x;
}
template <int V> __device__ __forceinline__ void store_vec(bf16_t* p, const float (&v)[V], const CodeFmt&) {
    typename Vec<bf16_t, V>::type x;
#pragma unroll
    for (int j = 0; j < V; ++j) x[j] = (bf16_t)v[j];
    *(typename Vec<bf16_t, V>::type*)p = x;
}
template <int V> __device__ __forceinline__ void store_vec(uint8_t* p, const float (&v)[V], const CodeFmt& f) {
    typedef uint32_t words __attribute__((ext_vector_type(V / 4), aligned(1)));
    words x;
#pragma unroll
    for (int j = 0; j < V / 4; ++j) x[j] = code_four(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3], f);
    *(words*)p = x;
}
__device__ __forceinline__ float load_one(const float* p) { return *p; }
__device__ __forceinline__ float load_one(const bf16_t* p) { return (float)*p; }
__device__ __forceinline__ void store_one(float* p, float v, const CodeFmt&) { *p = v; }
__device__ __forceinline__ void store_one(bf16_t* p, float v, const CodeFmt&) { *p = (bf16_t)v; }
__device__ __forceinline__ void store_one(uint8_t* p, float v, const CodeFmt& f) { *p = (uint8_t)code_one(v, f); }

// the first `n` of V elements (n >= V: all); what is past them reads as `fill`
template <int V, typename T> __device__ __forceinline__ void load_some(const T* p, int n, float (&v)[V], float fill = 0.0f) {
    if (n >= V) { load_vec<V>(p, v); return; }
#pragma unroll
    for (int j = 0; j < V; ++j) v[j] = j < n ? load_one(p + j) : fill;
}
template <int V, typename T> __device__ __forceinline__ void store_some(T* p, int n, const float (&v)[V], const CodeFmt& f) {
    if (n >= V) { store_vec<V>(p, v, f); return; }
#pragma unroll
    for (int j = 0; j < V; ++j)
        if (j < n) store_one(p + j, v[j], f);
}

// a vector as it comes from memory: converted where it is used, so that nothing waits for a load that is under way
template <typename T, int V> struct Raw { typename Vec<T, V>::type v; };
template <int V> __device__ __forceinline__ float raw_at(const Raw<float, V>& r, int j) { return r.v[j]; }
template <int V> __device__ __forceinline__ float raw_at(const Raw<uint16_t, V>& r, int j) { return __uint_as_float((uint32_t)r.v[j] << 16); }
template <typename T> struct Bits { typedef uint16_t type; };
template <> struct Bits<float> { typedef float type; };
template <typename T, int V> __device__ __forceinline__ Raw<T, V> load_raw(const T* p, int n) {
    Raw<T, V> r;
    if (n >= V) {
        r.v = *(const typename Vec<T, V>::type*)p;
    } else {
#pragma unroll
        for (int j = 0; j < V; ++j) r.v[j] = j < n ? p[j] : (T)0;
    }
    return r;
}

// ---- activations ----------------------------------------------------------------------------

// e^x to 1.5 ulp: 2^t of the rounded product t = x log2 e, corrected by what the rounding left off.  Beyond float32's range the
// correction must not meet an infinity: arguments under it are taken as one whose result is flushed, above it infinity is returned.
__device__ __forceinline__ float exp_near(float x) {
    const float y = fminf(fmaxf(x, -104.0f), 88.72f);
    const float t = y * 1.44269502f;
    const float left = fmaf(y, 1.44269502f, -t) + y * 1.92596303e-8f;
    const float e = __builtin_amdgcn_exp2f(t);
    return x > 88.72f ? __builtin_inff() : fmaf(e, left * 0.693147181f, e);
}

// The normal distribution's tail Phi(-a) for a = |z|, and its density phi.  Phi(-a) = phi(a) * h(t) with t = 1 / (1 + 0.28 a); h is smooth and is
// taken as a polynomial of degree 6 without a constant term, fitted to (1 + a) * Phi in the largest error (1.5e-8).  With it z * Phi(z) is
// max(z, 0) - a * Phi(-a) for either sign: nothing cancels in the tail, and nothing is chosen by a comparison.  `a` is at most 64, where
// the tail is 0 as a float32 number, so that an infinity does not meet that zero; a NaN comes through the exponential.
__device__ __forceinline__ float normal_tail(float z, float& a, float& phi) {
    a = fminf(fabsf(z), 64.0f);
    const float t = __builtin_amdgcn_rcpf(fmaf(0.28f, a, 1.0f));
    phi = __builtin_amdgcn_exp2f(fmaf(z * z, -0.72134752f, -1.32574809f));
    float h = fmaf(t, -0.267091841f, 0.985024333f);
    h = fmaf(t, h, -0.606841385f);
    h = fmaf(t, h, 0.684532404f);
    h = fmaf(t, h, 0.164927423f);
    h = fmaf(t, h, 0.292763114f);
    return phi * (t * h);
}
__device__ __forceinline__ float logistic(float z) { return __builtin_amdgcn_rcpf(1.0f + exp_near(-z)); }

template <int ACT> __device__ __forceinline__ float act_value(float z) {
    if constexpr (ACT == LBA_ACT_RELU) return z > 0.0f ? z : (z != z ? z : 0.0f);
    if constexpr (ACT == LBA_ACT_GELU) {
        float a, phi;
        const float q = normal_tail(z, a, phi);
        return fmaf(-a, q, fmaxf(z, 0.0f));
    }
    if constexpr (ACT == LBA_ACT_SILU) return z * logistic(z);
    return z;
}
// act(z) and its derivative
template <int ACT> __device__ __forceinline__ void act_both(float z, float& value, float& slope) {
    if constexpr (ACT == LBA_ACT_RELU) {
        value = z > 0.0f ? z : (z != z ? z : 0.0f);
        slope = z > 0.0f ? 1.0f : 0.0f;
    } else if constexpr (ACT == LBA_ACT_GELU) {
        float a, phi;
        const float q = normal_tail(z, a, phi);
        value = fmaf(-a, q, fmaxf(z, 0.0f));
        slope = fmaf(copysignf(a, z), phi, z < 0.0f ? q : 1.0f - q);
    } else if constexpr (ACT == LBA_ACT_SILU) {
        const float h = logistic(z);
        value = z * h;
        slope = h * (1.0f + z * (1.0f - h));
    } else {
        value = z;
        slope = 1.0f;
    }
}
// a number known when compiling, as an argument
template <int V> struct Known { static constexpr int value = V; };
// f(Known<act>): one branch around what is done with the activation, not one an element
template <typename F> __device__ __forceinline__ void with_act(int act, F f) {
    if (act == LBA_ACT_NONE) f(Known<LBA_ACT_NONE>{});
    else if (act == LBA_ACT_RELU) f(Known<LBA_ACT_RELU>{});
    else if (act == LBA_ACT_GELU) f(Known<LBA_ACT_GELU>{});
    else f(Known<LBA_ACT_SILU>{});
}

// ---- dropout --------------------------------------------------------------------------------

struct DropParams {
    uint64_t seed, stream;
    const uint64_t* step;
    uint32_t on;             // 0: nothing is dropped (T = 0)
    uint32_t above;          // 65536 T - 1: an element stays iff its 16 bits, in the high half of a word, are above it
    float keep_scale;        // 65536 / (65536 - threshold); 0 where everything is dropped
};

constexpr uint64_t kGolden = 0x9E3779B97F4A7C15ull;

__host__ __device__ __forceinline__ uint64_t mix64(uint64_t z) {
    z = (z ^ (z >> 30)) * 0xBF58476D1CE4E5B9ull;
    z = (z ^ (z >> 27)) * 0x94D049BB133111EBull;
    return z ^ (z >> 31);
}
__device__ __forceinline__ uint64_t drop_base(const DropParams& d) {
    const uint64_t s = d.stream + (d.step ? *d.step : 0ull);
    return mix64(mix64(d.seed * 2 + 1) ^ ((s * 2 + 1) * kGolden));
}
// 32-bit halves of the generator's words, two elements each -> which of the elements stay
template <int V> __device__ __forceinline__ void kept_of(const uint32_t (&h)[V / 2], const DropParams& d, bool (&keep)[V]) {
#pragma unroll
    for (int j = 0; j < V; ++j) keep[j] = (j % 2 ? h[j / 2] : h[j / 2] << 16) > d.above;           // what is below the high half decides nothing
}
// The halves from element `i % 4` of the first word on: `h` has two more halves than come out.  In 32-bit steps: a 64-bit shift whose amount is
// a register read its amount wrong on gfx950 where that was the last one of the wave's allocation (8192 x 4107 bfloat16 elements with GELU:
// thousands of wrong bits, others from run to run), and the compiler does not keep it off that register.
template <int H> __device__ __forceinline__ void halves_from(uint64_t i, const uint32_t (&h)[H + 2], uint32_t (&out)[H]) {
    const uint32_t later = 0u - (((uint32_t)i >> 1) & 1u);                           // all ones: one half further (by masks: a choice of
    const uint32_t bits = ((uint32_t)i & 1u) * 16;
    uint32_t s[H + 1];
#pragma unroll
    for (int j = 0; j <= H; ++j) s[j] = (h[j + 1] & later) | (h[j] & ~later);        // elements would put them into scratch memory)
#pragma unroll
    for (int j = 0; j < H; ++j) out[j] = __builtin_amdgcn_alignbit(s[j + 1], s[j], bits);
}
// Which of V consecutive elements from index i on stay.  `whole`: i is a multiple of 4 (uniform: where rows are multiples of 4); else the
// elements' bits are cut out of one more word.
template <int V> __device__ __forceinline__ void drop_keeps(uint64_t i, uint64_t base, const DropParams& d, bool whole, bool (&keep)[V]) {
    static_assert(V % 4 == 0, "whole words");
    uint64_t z = (i >> 2) * kGolden + base;
    uint32_t h[V / 2 + 2], out[V / 2];
#pragma unroll
    for (int q = 0; q < V / 4; ++q, z += kGolden) {
        const uint64_t u = mix64(z);
        out[2 * q] = h[2 * q] = (uint32_t)u;
        out[2 * q + 1] = h[2 * q + 1] = (uint32_t)(u >> 32);
    }
    if (!whole) {
        const uint64_t last = mix64(z);
        h[V / 2] = (uint32_t)last;
        h[V / 2 + 1] = (uint32_t)(last >> 32);
        halves_from<V / 2>(i, h, out);
    }
    kept_of<V>(out, d, keep);
}
// The same for a wave whose 64 lanes hold neighbouring groups of 8 elements of one row, the first of index `first` (uniform): the word behind a lane's two
// is its neighbour's first, and the last lane's is made once for the wave.
__device__ __forceinline__ void drop_keeps_wave(uint64_t first, uint64_t base, const DropParams& d, bool whole, bool (&keep)[8]) {
    const uint64_t row = (first >> 2) * kGolden + base;  // uniform
    const uint64_t z = row + (uint64_t)(2 * (threadIdx.x & 63)) * kGolden, u0 = mix64(z), u1 = mix64(z + kGolden);
    uint32_t out[4] = {(uint32_t)u0, (uint32_t)(u0 >> 32), (uint32_t)u1, (uint32_t)(u1 >> 32)};
    if (!whole) {
        const uint64_t last = mix64(row + 128 * kGolden);
        const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp((int)(uint32_t)last, (int)out[0], 0x130, 0xF, 0xF, false);
        const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp((int)(last >> 32), (int)out[1], 0x130, 0xF, 0xF, false);
        const uint32_t h[6] = {out[0], out[1], out[2], out[3], lo, hi};
        halves_from<4>(first, h, out);
    }
    kept_of<8>(out, d, keep);
}

// ---- sums over a wave -----------------------------------------------------------------------

template <int CTRL, int ROWS> __device__ __forceinline__ float dpp_zero(float v) {
    return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), CTRL, ROWS, 0xF, true));
}
// the sum of the wave's 64 values, the same in every lane; every lane takes part
__device__ __forceinline__ float wave_sum(float v) {
    v += dpp_zero<0x111, 0xF>(v);                        // within rows of 16: shifted by 1, 2, 4, 8
    v += dpp_zero<0x112, 0xF>(v);
    v += dpp_zero<0x114, 0xF>(v);
    v += dpp_zero<0x118, 0xF>(v);
    v += dpp_zero<0x142, 0xA>(v);                        // rows 0 and 2 into 1 and 3, then the lower half into the upper
    v += dpp_zero<0x143, 0xC>(v);
    return __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(v), 63));
}

template <int CTRL, int ROWS> __device__ __forceinline__ double dpp_zero(double v) {
    const uint64_t b = __builtin_bit_cast(uint64_t, v);
    const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)b, CTRL, ROWS, 0xF, true);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(b >> 32), CTRL, ROWS, 0xF, true);
    return __builtin_bit_cast(double, ((uint64_t)hi << 32) | lo);
}
__device__ __forceinline__ double wave_sum(double v) {
    v += dpp_zero<0x111, 0xF>(v);
    v += dpp_zero<0x112, 0xF>(v);
    v += dpp_zero<0x114, 0xF>(v);
    v += dpp_zero<0x118, 0xF>(v);
    v += dpp_zero<0x142, 0xA>(v);
    v += dpp_zero<0x143, 0xC>(v);
    const uint64_t b = __builtin_bit_cast(uint64_t, v);
    const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)b, 63), hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(b >> 32), 63);
    return __builtin_bit_cast(double, ((uint64_t)hi << 32) | lo);
}

// ---- column sums ----------------------------------------------------------------------------

// out0[n] = sum over `parts` rows of part[row * ld + n], and with out1 out1[n] that of part[row * ld + N + n] (out0 may be null then),
// always in the same order; columns from `split` on have `parts2` rows
void launch_column_sum(const float* part, int64_t parts, int64_t ld, float* out0, float* out1, int64_t N, hipStream_t st, int64_t split = INT64_MAX,
                       int64_t parts2 = 0);
// zeros (an even number of bytes; a kernel, so that it can be captured)
void launch_zero(void* out, int64_t bytes, hipStream_t st);

// ---- host checks ----------------------------------------------------------------------------

inline int check_float_type(int32_t t) { return t == LBA_F32 || t == LBA_BF16 ? LBA_OK : LBA_ERR_UNSUPPORTED; }
int check_out_type(int32_t t, const lba_infmt& f);
int check_drop(const lba_drop& d, DropParams* out);
int check_rows(int64_t M, int64_t N);
inline int check_act(int32_t a) { return a >= LBA_ACT_NONE && a <= LBA_ACT_SILU ? LBA_OK : LBA_ERR_UNSUPPORTED; }

constexpr size_t align256(size_t b) { return (b + 255) & ~(size_t)255; }

}  // namespace lba
#endif
