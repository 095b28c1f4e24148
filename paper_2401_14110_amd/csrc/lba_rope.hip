// lba_rope.hip -- rotary positions and their gradient.
//
// A pair (a, b) of a row at position m is turned by the angle m f, the same for all heads of the row: a workgroup takes a few rows, works out
// their cosines and sines once, one a lane, into LDS, and then streams over the heads, every lane with 16 bytes of either half (interleaved: 16
// bytes of pairs) at a time.  The angle is a float64 product in turns, m * (f / 2 pi), from which whole quarter turns are taken before anything
// is rounded to float32: positions of 10^6 are off by 2^-33 of a turn.  What is left is at most an eighth of a turn, where the series of cosine and sine
// are taken to the terms of x^10 and x^9, under 2^-28 off.
// Bound by memory: one read and one write of the tensor (16384 rows of 40 heads of 128 in bfloat16, 336 MB: 68 us, 4.9 TB/s; a copy's 5.2).
#include "lba_attn_device.h"

namespace lba {

struct RopeParams {
    const void* X;
    void* Y;
    const void* positions;
    const double* freq;
    lba_strides x, y;
    int32_t T, H, D, pairs;
    int32_t wide;            // positions of 64 bits
    int32_t rows;            // rows of a workgroup at a time
    float gain, sign;
};

constexpr int kRopeAngles = 512;                         // cosines and sines in LDS: rows * pairs are at most this

// gain * (cos, sign * sin) of m * f
__device__ __forceinline__ float2 turn_of(double m, double f, float gain, float sign) {
    const double t = m * (f * 0.15915494309189533577);   // turns
    const double u = (t - __builtin_rint(t)) * 4.0;      // quarter turns, -2 .. 2; exact
    const double q = __builtin_rint(u);
    const float x = (float)(u - q) * 1.57079632679489662f, s = x * x;
    float sn = fmaf(s, 2.7557319e-6f, -1.9841270e-4f);
    sn = fmaf(s, sn, 8.3333333e-3f);
    sn = fmaf(s, sn, -0.16666667f);
    sn = fmaf(s * sn, x, x);
    float cs = fmaf(s, -2.7557319e-7f, 2.4801587e-5f);
    cs = fmaf(s, cs, -1.3888889e-3f);
    cs = fmaf(s, cs, 4.1666667e-2f);
    cs = fmaf(s, cs, -0.5f);
    cs = fmaf(s, cs, 1.0f);
    const int k = (int)q & 3;
    const float a = k & 1 ? sn : cs, b = k & 1 ? cs : sn;
    return {gain * (k == 1 || k == 2 ? -a : a), gain * sign * (k >= 2 ? -b : b)};
}

// the first n of V elements as they are
template <int V, typename B> __device__ __forceinline__ void copy_some(const B* x, B* y, int n) {
    const Raw<B, V> r = load_raw<B, V>(x, n);
    if (n >= V) {
        *(typename Vec<B, V>::type*)y = r.v;
    } else {
#pragma unroll
        for (int j = 0; j < V; ++j)
            if (j < n) y[j] = r.v[j];
    }
}

template <typename T, bool INTERLEAVED>
__global__ __launch_bounds__(256) void rope_kernel(RopeParams p) {
    constexpr int V = 16 / sizeof(T), PV = INTERLEAVED ? V / 2 : V;                  // elements of a load, pairs of an item
    __shared__ float2 angle[kRopeAngles];
    const T* X = (const T*)p.X;
    T* Y = (T*)p.Y;
    const CodeFmt none = {};
    const int turned = (p.pairs + PV - 1) / PV, copied = (p.D - 2 * p.pairs + V - 1) / V, items = turned + copied;
    for (int64_t t0 = (int64_t)blockIdx.x * p.rows; t0 < p.T; t0 += (int64_t)gridDim.x * p.rows) {
        const int rows = (int)min((int64_t)p.rows, p.T - t0);
        __syncthreads();
        for (int i = threadIdx.x; i < rows * p.pairs; i += 256) {
            const int64_t t = t0 + i / p.pairs;
            const double m = p.wide ? (double)((const int64_t*)p.positions)[t] : (double)((const int32_t*)p.positions)[t];
            angle[i] = turn_of(m, p.freq[i % p.pairs], p.gain, p.sign);
        }
        __syncthreads();
        for (int i = threadIdx.x; i < rows * p.H * items; i += 256) {
            const int c = i % items, rh = i / items, h = rh % p.H, r = rh / p.H;
            const T* x = X + (t0 + r) * p.x.row + (int64_t)h * p.x.head;
            T* y = Y + (t0 + r) * p.y.row + (int64_t)h * p.y.head;
            if (c >= turned) {
                const int d = 2 * p.pairs + (c - turned) * V;
                copy_some<V>((const typename Bits<T>::type*)x + d, (typename Bits<T>::type*)y + d, p.D - d);
                continue;
            }
            const float2* w = angle + r * p.pairs + c * PV;
            const int left = p.pairs - c * PV;           // pairs from here on
            if constexpr (INTERLEAVED) {
                float v[V], o[V];
                load_some<V>(x + c * V, 2 * left, v);
#pragma unroll
                for (int j = 0; j < PV; ++j) {
                    const float2 cs = w[j < left ? j : 0];
                    o[2 * j] = v[2 * j] * cs.x - v[2 * j + 1] * cs.y;
                    o[2 * j + 1] = v[2 * j + 1] * cs.x + v[2 * j] * cs.y;
                }
                store_some<V>(y + c * V, 2 * left, o, none);
            } else {
                float a[V], b[V], o[V], q[V];
                load_some<V>(x + c * V, left, a);
                load_some<V>(x + p.pairs + c * V, left, b);
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    const float2 cs = w[j < left ? j : 0];
                    o[j] = a[j] * cs.x - b[j] * cs.y;
                    q[j] = b[j] * cs.x + a[j] * cs.y;
                }
                store_some<V>(y + c * V, left, o, none);
                store_some<V>(y + p.pairs + c * V, left, q, none);
            }
        }
    }
}

static int rope(const void* X, lba_strides x_at, int32_t type, const void* positions, int32_t pos_bits, const double* freq, int64_t pairs,
                int32_t interleaved, float gain, float sign, void* Y, lba_strides y_at, int64_t T, int64_t H, int64_t D, hipStream_t st) {
    int rc = check_heads(T, H, D);
    if (rc == LBA_OK) rc = check_strides(x_at);
    if (rc == LBA_OK) rc = check_strides(y_at);
    if (rc == LBA_OK && (pairs < 0 || 2 * pairs > D)) rc = LBA_ERR_SHAPE;
    if (rc == LBA_OK) rc = check_float_type(type);
    if (rc == LBA_OK && pos_bits != 32 && pos_bits != 64) rc = LBA_ERR_UNSUPPORTED;
    if (rc != LBA_OK) return rc;
    if (T == 0 || H == 0 || D == 0) return LBA_OK;
    if (!X || !Y || (pairs > 0 && (!positions || !freq))) return LBA_ERR_NULL;
    RopeParams p = {};
    p.X = X; p.Y = Y; p.positions = positions; p.freq = freq; p.x = x_at; p.y = y_at;
    p.T = (int32_t)T; p.H = (int32_t)H; p.D = (int32_t)D; p.pairs = (int32_t)pairs; p.wide = pos_bits == 64;
    p.gain = gain; p.sign = sign;
    // (the angles of four rows at once, but where there are few rows one a workgroup: 9 rows of 40 heads 6.8 us by fours)
    p.rows = pairs > 256 ? 1 : pairs > 64 ? 2 : 4;
    if (T < 256 * p.rows) p.rows = 1;
    const int64_t blocks = (T + p.rows - 1) / p.rows;
    const dim3 grid((unsigned)(blocks < (1 << 20) ? blocks : (1 << 20)));
    if (type == LBA_F32) {
        if (interleaved) hipLaunchKernelGGL((rope_kernel<float, true>), grid, dim3(256), 0, st, p);
        else hipLaunchKernelGGL((rope_kernel<float, false>), grid, dim3(256), 0, st, p);
    } else {
        if (interleaved) hipLaunchKernelGGL((rope_kernel<bf16_t, true>), grid, dim3(256), 0, st, p);
        else hipLaunchKernelGGL((rope_kernel<bf16_t, false>), grid, dim3(256), 0, st, p);
    }
    return hipGetLastError() == hipSuccess ? LBA_OK : LBA_ERR_LAUNCH;
}

}  // namespace lba

using namespace lba;

extern "C" {

int lba_rope(const void* X, lba_strides x_at, int32_t type, const void* positions, int32_t pos_bits, const double* freq, int64_t pairs,
             int32_t interleaved, float gain, void* Y, lba_strides y_at, int64_t T, int64_t H, int64_t D, void* hip_stream) {
    return rope(X, x_at, type, positions, pos_bits, freq, pairs, interleaved, gain, 1.0f, Y, y_at, T, H, D, (hipStream_t)hip_stream);
}

int lba_rope_bwd(const void* G, lba_strides g_at, int32_t type, const void* positions, int32_t pos_bits, const double* freq, int64_t pairs,
                 int32_t interleaved, float gain, void* dX, lba_strides dx_at, int64_t T, int64_t H, int64_t D, void* hip_stream) {
    return rope(G, g_at, type, positions, pos_bits, freq, pairs, interleaved, gain, -1.0f, dX, dx_at, T, H, D, (hipStream_t)hip_stream);
}

}  // extern "C"
