// lba_norm.hip -- layer norm over rows and its gradients (include/lba_layer.h).
//
// Forward: a row is read once into registers; mean = sum / N, then the sum of squared differences from that mean, both in float32 (in 64 bits
// where codes come out) over the same registers, so nothing cancels.  Backward: with n = (x - mean) * rstd and h = g * gamma the row sums of
// h and h * n come from registers too, and the column sums of g * n and g, which dgamma and dbeta are, stay in the registers of the lanes
// that own the columns while a workgroup walks over its rows; one row of partial sums per workgroup goes to the workspace, and
// a second launch adds them in a fixed order.
// Both are bound by memory: every element is moved once.  A row belongs to a wave where four vectors of 16 bytes a lane hold it (two of
// bfloat16), else to a workgroup of 256, 512 or 1024 lanes; rows beyond 16384 elements are read again from cache for each pass, which is a plain
// loop: 1024 x 65536 bfloat16 take 269 us forward and 271 + 131 backward, where their bytes would take 52 and 77.
// Measured (bytes that have to move over the time; a copy of 1 GiB reaches 5.2 TB/s): 16384 x 4096 bfloat16, forward, backward and column sums
// together 137 us, 4.9 TB/s; 4096 x 768 float32 to codes 9.2 us, backward 9.8 + 3.7; 1024 x 16384 float32 forward 27, backward 38 + 11; one row
// of 768: 3 us, a launch.
#include "lba_layer_device.h"
#include "lba_internal.h"

namespace lba {

// sums of K values over the T lanes that share a row (T = 64: a wave; else the whole workgroup)
template <int T, int K, typename W> __device__ __forceinline__ void row_sums(W (&v)[K], W* lds, int turn) {
#pragma unroll
    for (int k = 0; k < K; ++k) v[k] = wave_sum(v[k]);
    if (T == 64) return;
    constexpr int WAVES = T / 64;
    W* at = lds + (turn & 1) * (K * WAVES);              // two sets: a wave that is ahead writes the other one
    if ((threadIdx.x & 63) == 0) {
#pragma unroll
        for (int k = 0; k < K; ++k) at[k * WAVES + threadIdx.x / 64] = v[k];
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < K; ++k) {
        W s = 0;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) s += at[k * WAVES + w];
        v[k] = s;
    }
}

// What a row is worked on in.  Codes have four significant bits: a float32 result next to the middle of two codes falls on the wrong side once in
// a million (3 of 3.1 M codes), so codes are made in 64 bits and none does.  It takes 9.2 us instead of 6.3 on 4096 x 768 float32, 68 us on 16384 x
// 4096 bfloat16 where bfloat16 numbers take 44, and nothing on a single row; keeping the elements in 64 bits gained nothing.
template <typename TY> struct Work { typedef float type; };
template <> struct Work<uint8_t> { typedef double type; };
// 64 bits -> 32, cut off, and the last bit set where something was: rounding that again to fewer bits is rounding once.  The bit is set before
// the conversion, which then is exact or, beyond float32, an infinity.
__device__ __forceinline__ float to_odd(double d) {
    const uint64_t b = __builtin_bit_cast(uint64_t, d);
    const uint32_t lo = (uint32_t)b, rest = lo & 0x1FFFFFFFu;                        // float32 has 29 bits less
    const uint32_t kept = (lo | (rest < 1u ? rest : 1u) << 29) & 0xE0000000u;
    return (float)__builtin_bit_cast(double, (b >> 32 << 32) | kept);
}
__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(double v) { return to_odd(v); }

struct NormParams {
    const void* X;
    const void* G;
    const float* gamma;
    const float* beta;
    void* Y;                 // forward: y; backward: dx
    float* mean;
    float* rstd;
    float* part;             // backward: [blocks][2][N] partial sums, or null
    int64_t M;
    int32_t N;
    float eps, n;             // n: N, which sums are divided by (a rounded 1 / N would give a constant row another mean)
    CodeFmt fmt;
};

// A lane group walks over rows: gamma and beta stay in registers and the next row is loaded while this one is worked on (two sets of registers,
// so that none is moved while in flight).
template <typename TX, typename TY, int T, int NV>
__global__ __launch_bounds__(T < 256 ? 256 : T) void norm_fwd_kernel(NormParams p) {
    constexpr int V = 16 / sizeof(TX), RPB = T < 256 ? 256 / T : 1;
    typedef typename Bits<TX>::type BX;
    typedef typename Work<TY>::type W;
    __shared__ W lds[2 * (T / 64)];
    const int t = threadIdx.x % T, sub = __builtin_amdgcn_readfirstlane(threadIdx.x / T);
    struct Row { Raw<BX, V> x[NV]; };
    auto load = [&](int64_t row, Row& r) {
        const BX* x = (const BX*)p.X + row * p.N;
#pragma unroll
        for (int i = 0; i < NV; ++i) r.x[i] = load_raw<BX, V>(x + (i * T + t) * V, p.N - (i * T + t) * V);
    };
    const int64_t step = (int64_t)gridDim.x * RPB;
    int64_t row = (int64_t)blockIdx.x * RPB + sub;
    Row a;
    if (row < p.M) load(row, a);
    constexpr bool KEEP = T < 1024 || sizeof(W) == 4;    // else 128 registers hold neither gamma and beta nor a second row
    float ga[KEEP ? NV : 1][V], be[KEEP ? NV : 1][V];
    auto columns = [&](int i, float (&g)[V], float (&b)[V]) {
        const int c = (i * T + t) * V;
#pragma unroll
        for (int j = 0; j < V; ++j) {
            g[j] = 1.0f;
            b[j] = 0.0f;
        }
        if (p.gamma) load_some<V>(p.gamma + c, p.N - c, g);
        if (p.beta) load_some<V>(p.beta + c, p.N - c, b);
    };
    if constexpr (KEEP) {
#pragma unroll
        for (int i = 0; i < NV; ++i) columns(i, ga[i], be[i]);
    }
    auto work = [&](int64_t at, const Row& r) {
        W s[1] = {0};
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int j = 0; j < V; ++j) s[0] += (W)raw_at(r.x[i], j);                // 0 beyond the row
        row_sums<T, 1>(s, lds, 0);
        const W mean = s[0] / (W)p.n;
        s[0] = 0;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (i * T + t) * V;
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const W d = (W)raw_at(r.x[i], j) - mean;
                if (c + j < p.N) s[0] = fma(d, d, s[0]);
            }
        }
        row_sums<T, 1>(s, lds, 1);
        const W rstd = 1 / sqrt(s[0] / (W)p.n + (W)p.eps);
        if (t == 0) {
            if (p.mean) p.mean[at] = (float)mean;
            if (p.rstd) p.rstd[at] = (float)rstd;
        }
        TY* y = (TY*)p.Y + at * p.N;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (i * T + t) * V;
            if (c >= p.N) break;
            float v[V];
            if (!KEEP) columns(i, ga[0], be[0]);
            constexpr int EVERY = KEEP ? 1 : 0;
#pragma unroll
            for (int j = 0; j < V; ++j) v[j] = to_float(fma(((W)raw_at(r.x[i], j) - mean) * rstd, (W)ga[i * EVERY][j], (W)be[i * EVERY][j]));
            store_some<V>(y + c, p.N - c, v, p.fmt);
        }
    };
    if constexpr (!KEEP) {
        while (row < p.M) {
            work(row, a);
            row += step;
            if (row < p.M) load(row, a);
        }
    } else {
        Row b;
        for (; row < p.M; row += 2 * step) {
            const bool more = row + step < p.M;
            if (more) load(row + step, b);
            work(row, a);
            if (!more) break;
            if (row + 2 * step < p.M) load(row + 2 * step, a);
            work(row + step, b);
        }
    }
}

// rows that do not fit the registers of 1024 lanes
template <typename TX, typename TY>
__global__ __launch_bounds__(1024) void norm_fwd_long_kernel(NormParams p) {
    constexpr int V = 16 / sizeof(TX), T = 1024;
    __shared__ float lds[2 * (T / 64)];
    for (int64_t row = blockIdx.x; row < p.M; row += gridDim.x) {
    const TX* x = (const TX*)p.X + row * p.N;
    float s[1] = {0.0f}, v[V];
    for (int c = threadIdx.x * V; c < p.N; c += T * V) {
        load_some<V>(x + c, p.N - c, v);
#pragma unroll
        for (int j = 0; j < V; ++j) s[0] += v[j];
    }
    row_sums<T, 1>(s, lds, 0);
    const float mean = s[0] / p.n;
    s[0] = 0.0f;
    for (int c = threadIdx.x * V; c < p.N; c += T * V) {
        load_some<V>(x + c, p.N - c, v, mean);
#pragma unroll
        for (int j = 0; j < V; ++j) s[0] = fmaf(v[j] - mean, v[j] - mean, s[0]);
    }
    row_sums<T, 1>(s, lds, 1);
    const float rstd = 1.0f / sqrtf(s[0] / p.n + p.eps);
    if (threadIdx.x == 0) {
        if (p.mean) p.mean[row] = mean;
        if (p.rstd) p.rstd[row] = rstd;
    }
    TY* y = (TY*)p.Y + row * p.N;
    for (int c = threadIdx.x * V; c < p.N; c += T * V) {
        load_some<V>(x + c, p.N - c, v);
#pragma unroll
        for (int j = 0; j < V; ++j) {
            float o = (v[j] - mean) * rstd;
            if (c + j < p.N) {
                if (p.gamma) o *= p.gamma[c + j];
                if (p.beta) o += p.beta[c + j];
            }
            v[j] = o;
        }
        store_some<V>(y + c, p.N - c, v, p.fmt);
    }
    }
}

// The next row of a lane group is loaded while this one is worked on, but for
// workgroups of 1024 lanes, whose 128 registers do not hold both.
template <typename TG, typename TX, int T, int NV>
__global__ __launch_bounds__(T < 256 ? 256 : T) void norm_bwd_kernel(NormParams p) {
    constexpr int V = 16 / sizeof(TX), RPB = T < 256 ? 256 / T : 1;
    typedef typename Bits<TX>::type BX;
    typedef typename Bits<TG>::type BG;
    __shared__ float lds[4 * (T / 64)];
    const int t = threadIdx.x % T, sub = __builtin_amdgcn_readfirstlane(threadIdx.x / T);
    float ga[NV][V], dga[NV][V], dbe[NV][V];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (i * T + t) * V;
        if (p.gamma) load_some<V>(p.gamma + c, p.N - c, ga[i]);
#pragma unroll
        for (int j = 0; j < V; ++j) {
            if (!p.gamma) ga[i][j] = 1.0f;
            dga[i][j] = dbe[i][j] = 0.0f;
        }
    }
    struct Row { Raw<BX, V> x[NV]; Raw<BG, V> g[NV]; float mean, rstd; };
    auto load = [&](int64_t row, Row& r) {
        const BX* x = (const BX*)p.X + row * p.N;
        const BG* g = (const BG*)p.G + row * p.N;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (i * T + t) * V;
            r.x[i] = load_raw<BX, V>(x + c, p.N - c);
            r.g[i] = load_raw<BG, V>(g + c, p.N - c);
        }
        r.mean = p.mean[row];
        r.rstd = p.rstd[row];
    };
    int turn = 0;
    auto work = [&](int64_t row, const Row& r) {
        float s[2] = {0.0f, 0.0f}, n[NV][V];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (i * T + t) * V;
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float g = raw_at(r.g[i], j);
                n[i][j] = c + j < p.N ? (raw_at(r.x[i], j) - r.mean) * r.rstd : 0.0f;
                const float h = g * ga[i][j];
                dga[i][j] = fmaf(g, n[i][j], dga[i][j]);
                dbe[i][j] += g;
                s[0] += h;
                s[1] = fmaf(h, n[i][j], s[1]);
            }
        }
        if (!p.Y) return;
        row_sums<T, 2>(s, lds, turn++);
        const float mh = s[0] / p.n, mhn = s[1] / p.n;
        TX* dx = (TX*)p.Y + row * p.N;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (i * T + t) * V;
            if (c >= p.N) break;
#pragma unroll
            for (int j = 0; j < V; ++j) n[i][j] = r.rstd * (raw_at(r.g[i], j) * ga[i][j] - fmaf(n[i][j], mhn, mh));
            store_some<V>(dx + c, p.N - c, n[i], p.fmt);
        }
    };
    const int64_t step = (int64_t)gridDim.x * RPB;
    int64_t row = (int64_t)blockIdx.x * RPB + sub;
    Row a;
    if constexpr (T >= 1024) {
        for (; row < p.M; row += step) {
            load(row, a);
            work(row, a);
        }
    } else {
        Row b;
        if (row < p.M) load(row, a);
        for (; row < p.M; row += 2 * step) {
            const bool more = row + step < p.M;
            if (more) load(row + step, b);
            work(row, a);
            if (!more) break;
            if (row + 2 * step < p.M) load(row + 2 * step, a);
            work(row + step, b);
        }
    }
    if (!p.part) return;
    if (RPB > 1) {                                       // the workgroup's rows first: one after the other into LDS
        __shared__ float acc[RPB > 1 ? 2 * T * NV * V : 1];
        for (int r = 0; r < RPB; ++r) {
            if (sub == r) {
#pragma unroll
                for (int i = 0; i < NV; ++i)
#pragma unroll
                    for (int j = 0; j < V; ++j) {
                        float* at = acc + (i * V + j) * T + t;
                        at[0] = r ? at[0] + dga[i][j] : dga[i][j];
                        at[T * NV * V] = r ? at[T * NV * V] + dbe[i][j] : dbe[i][j];
                    }
            }
            __syncthreads();
        }
        if (sub != 0) return;
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int j = 0; j < V; ++j) {
                dga[i][j] = acc[(i * V + j) * T + t];
                dbe[i][j] = acc[(i * V + j) * T + t + T * NV * V];
            }
    }
    float* out = p.part + (int64_t)blockIdx.x * 2 * p.N;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (i * T + t) * V;
        if (c >= p.N) break;
        store_some<V>(out + c, p.N - c, dga[i], p.fmt);
        store_some<V>(out + p.N + c, p.N - c, dbe[i], p.fmt);
    }
}

// dx of rows that do not fit the registers of 1024 lanes
template <typename TG, typename TX>
__global__ __launch_bounds__(1024) void norm_bwd_long_kernel(NormParams p) {
    constexpr int V = 16 / sizeof(TX), T = 1024;
    __shared__ float lds[4 * (T / 64)];
    int turn = 0;                                        // a row has one barrier: a wave that is ahead must not write the set that others read
    for (int64_t row = blockIdx.x; row < p.M; row += gridDim.x) {
    const TX* x = (const TX*)p.X + row * p.N;
    const TG* gr = (const TG*)p.G + row * p.N;
    const float mean = p.mean[row], rstd = p.rstd[row];
    float s[2] = {0.0f, 0.0f}, n[V], g[V];
    for (int c = threadIdx.x * V; c < p.N; c += T * V) {
        load_some<V>(x + c, p.N - c, n);
        load_some<V>(gr + c, p.N - c, g);
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const float h = c + j < p.N && p.gamma ? g[j] * p.gamma[c + j] : g[j];
            s[0] += h;
            if (c + j < p.N) s[1] = fmaf(h, (n[j] - mean) * rstd, s[1]);
        }
    }
    row_sums<T, 2>(s, lds, turn++);
    const float mh = s[0] / p.n, mhn = s[1] / p.n;
    TX* dx = (TX*)p.Y + row * p.N;
    for (int c = threadIdx.x * V; c < p.N; c += T * V) {
        load_some<V>(x + c, p.N - c, n);
        load_some<V>(gr + c, p.N - c, g);
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const float h = c + j < p.N && p.gamma ? g[j] * p.gamma[c + j] : g[j];
            n[j] = rstd * (h - fmaf((n[j] - mean) * rstd, mhn, mh));
        }
        store_some<V>(dx + c, p.N - c, n, p.fmt);
    }
    }
}

// and the partial column sums of such rows: a workgroup owns 256 * V columns of a slice of the rows
template <typename TG, typename TX>
__global__ __launch_bounds__(256) void norm_bwd_long_params_kernel(NormParams p) {
    constexpr int V = 16 / sizeof(TX);
    const int c = (blockIdx.y * 256 + threadIdx.x) * V;
    if (c >= p.N) return;
    float dga[V], dbe[V], n[V], g[V];
#pragma unroll
    for (int j = 0; j < V; ++j) dga[j] = dbe[j] = 0.0f;
    for (int64_t row = blockIdx.x; row < p.M; row += gridDim.x) {
        const float mean = p.mean[row], rstd = p.rstd[row];
        load_some<V>((const TX*)p.X + row * p.N + c, p.N - c, n);
        load_some<V>((const TG*)p.G + row * p.N + c, p.N - c, g);
#pragma unroll
        for (int j = 0; j < V; ++j) {
            dga[j] = fmaf(g[j], (n[j] - mean) * rstd, dga[j]);
            dbe[j] += g[j];
        }
    }
    float* out = p.part + (int64_t)blockIdx.x * 2 * p.N;
    store_some<V>(out + c, p.N - c, dga, p.fmt);
    store_some<V>(out + p.N + c, p.N - c, dbe, p.fmt);
}

// ---- column sums ----------------------------------------------------------------------------

// A workgroup takes 16 columns: thread t adds every 64th row of column t % 16, eight loads in flight, then the 64 sums of a column are added
// in a fixed order.  (One lane a column and four rows in flight left the loads' latency bare: 1024 rows of 1536 columns took 23 us.)
__global__ __launch_bounds__(1024) void column_sum_kernel(const float* part, int64_t parts, int64_t ld, float* out0, float* out1, int64_t N, int64_t split,
                                                         int64_t parts2) {
    __shared__ float lds[16][16];
    const int c = threadIdx.x & 15;
    const int64_t n = (int64_t)blockIdx.x * 16 + c;
    const int64_t cols = out1 ? 2 * N : N;
    if (n >= split) parts = parts2;
    float s = 0.0f;
    if (n < cols) {
        int64_t r = threadIdx.x / 16;
        for (; r + 448 < parts; r += 512) {
            float v[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = part[(r + 64 * k) * ld + n];
            s += ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7]));
        }
        float v[7];
#pragma unroll
        for (int k = 0; k < 7; ++k) v[k] = r + 64 * k < parts ? part[(r + 64 * k) * ld + n] : 0.0f;
        s += ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + v[6]);
    }
    s += __shfl_xor(s, 16);
    s += __shfl_xor(s, 32);
    if ((threadIdx.x & 48) == 0) lds[threadIdx.x / 64][c] = s;
    __syncthreads();
    if (threadIdx.x >= 16 || n >= cols) return;
    float total = 0.0f;
#pragma unroll
    for (int w = 0; w < 16; ++w) total += lds[w][c];
    if (n >= N) out1[n - N] = total;
    else if (out0) out0[n] = total;
}

void launch_column_sum(const float* part, int64_t parts, int64_t ld, float* out0, float* out1, int64_t N, hipStream_t st, int64_t split, int64_t parts2) {
    const int64_t cols = out1 ? 2 * N : N;
    hipLaunchKernelGGL(column_sum_kernel, dim3((unsigned)((cols + 15) / 16)), dim3(1024), 0, st, part, parts, ld, out0, out1, N, split, parts2);
}

__global__ __launch_bounds__(256) void zero_kernel(uint16_t* out, int64_t n) {
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) out[i] = 0;
}
void launch_zero(void* out, int64_t bytes, hipStream_t st) {
    const int64_t n = bytes / 2, blocks = (n + 255) / 256;
    if (n > 0) hipLaunchKernelGGL(zero_kernel, dim3((unsigned)(blocks < 65536 ? blocks : 65536)), dim3(256), 0, st, (uint16_t*)out, n);
}

// ---- launchers ------------------------------------------------------------------------------

// lanes that share a row and vectors of 16 bytes a lane holds: the least that hold N elements (0 lanes: none does)
struct RowShape { int lanes, vecs; };
static RowShape row_shape(int64_t N, int v) {
    static const RowShape all[] = {{64, 1}, {64, 2}, {64, 4}, {256, 2}, {256, 4}, {512, 2}, {512, 4}, {1024, 2}, {1024, 4}};
    for (const RowShape& r : all)
        if (N <= (int64_t)r.lanes * r.vecs * v && r.vecs * v <= 16) return r;
    return {0, 0};
}

// lanes of a forward launch: as many as the chip holds at a time, each of which walks over rows
constexpr int64_t kNormLanes = 256 * 2048;
// Workgroups for rows beyond the registers, which walk over the rows beyond: a launch holds fewer than 2^32 lanes.  (4096 of them, four rows each,
// took 16384 rows of 20000 bfloat16 elements 1290 us forward instead of 1262.)
static unsigned long_blocks(int64_t M) { return (unsigned)(M < 65536 ? M : 65536); }

template <typename TX, typename TY> static void norm_fwd(const NormParams& p, hipStream_t st) {
    const RowShape r = row_shape(p.N, 16 / (int)sizeof(TX));
    const int lanes = r.lanes < 256 ? 256 : r.lanes;
    const int64_t groups = r.lanes == 64 ? (p.M + 3) / 4 : p.M, most = kNormLanes / lanes;
    const dim3 grid((unsigned)(groups < most ? groups : most));
#define LBA_NORM_FWD(T, NV) \
    if (r.lanes == T && r.vecs == NV) { hipLaunchKernelGGL((norm_fwd_kernel<TX, TY, T, NV>), grid, dim3(T < 256 ? 256 : T), 0, st, p); return; }
    LBA_NORM_FWD(64, 1)
    LBA_NORM_FWD(64, 2)
    LBA_NORM_FWD(256, 2)
    LBA_NORM_FWD(512, 2)
    LBA_NORM_FWD(1024, 2)
    if constexpr (sizeof(TX) == 4) {
        LBA_NORM_FWD(64, 4)
        LBA_NORM_FWD(256, 4)
        LBA_NORM_FWD(512, 4)
        LBA_NORM_FWD(1024, 4)
    }
#undef LBA_NORM_FWD
    hipLaunchKernelGGL((norm_fwd_long_kernel<TX, TY>), dim3(long_blocks(p.M)), dim3(1024), 0, st, p);
}

// Workgroups of the backward pass, each of which writes a row of partial sums: enough to fill the chip, few enough that these rows stay a
// small part of the traffic
static int64_t norm_bwd_blocks(int64_t M, int64_t N) {
    const int64_t groups = N <= 1024 ? (M + 3) / 4 : M;                              // rows that workgroups take at a time
    const int64_t most = groups >= 4096 || N <= 1024 ? 512 : 256;                    // few long rows: half of the partial sums
    return groups < most ? groups : most;
}

template <typename TG, typename TX> static void norm_bwd(NormParams p, hipStream_t st) {
    const RowShape r = row_shape(p.N, 16 / (int)sizeof(TX));
    const unsigned blocks = (unsigned)norm_bwd_blocks(p.M, p.N);
#define LBA_NORM_BWD(T, NV) \
    if (r.lanes == T && r.vecs == NV) { \
        hipLaunchKernelGGL((norm_bwd_kernel<TG, TX, T, NV>), dim3(blocks), dim3(T < 256 ? 256 : T), 0, st, p); \
        return; \
    }
    LBA_NORM_BWD(64, 1)
    LBA_NORM_BWD(64, 2)
    LBA_NORM_BWD(256, 2)
    LBA_NORM_BWD(512, 2)
    LBA_NORM_BWD(1024, 2)
    if constexpr (sizeof(TX) == 4) {
        LBA_NORM_BWD(64, 4)
        LBA_NORM_BWD(256, 4)
        LBA_NORM_BWD(512, 4)
        LBA_NORM_BWD(1024, 4)
    }
#undef LBA_NORM_BWD
    constexpr int V = 16 / sizeof(TX);
    if (p.part)
        hipLaunchKernelGGL((norm_bwd_long_params_kernel<TG, TX>), dim3(blocks, (unsigned)((p.N + 256 * V - 1) / (256 * V))), dim3(256), 0, st, p);
    if (p.Y) hipLaunchKernelGGL((norm_bwd_long_kernel<TG, TX>), dim3(long_blocks(p.M)), dim3(1024), 0, st, p);
}

int check_out_type(int32_t t, const lba_infmt& f) {
    if (t == LBA_F32 || t == LBA_BF16) return LBA_OK;
    if (t != LBA_CODE8) return LBA_ERR_UNSUPPORTED;
    if (f.exp_bits < 2 || f.exp_bits > 5 || f.man_bits != 7 - f.exp_bits || f.bias < -32 || f.bias > 32) return LBA_ERR_FORMAT;
    return LBA_OK;
}
int check_drop(const lba_drop& d, DropParams* out) {
    if (!(d.p >= 0.0 && d.p <= 1.0)) return LBA_ERR_FORMAT;
    out->seed = d.seed; out->stream = d.stream; out->step = d.step;
    const uint32_t t = (uint32_t)(d.p * 65536.0 + 0.5);
    out->on = t > 0 ? 1 : 0;
    out->above = t * 65536u - 1u;                        // all ones for T = 65536: nothing is above
    out->keep_scale = t >= 65536u ? 0.0f : (float)(65536.0 / (65536.0 - t));
    return LBA_OK;
}
int check_rows(int64_t M, int64_t N) {
    if (M < 0 || N < 0 || M > 2147483647LL || N > ((int64_t)1 << 21)) return LBA_ERR_SHAPE;
    return LBA_OK;
}

}  // namespace lba

using namespace lba;

extern "C" {

int lba_layernorm(const void* X, int32_t x_type, const float* gamma, const float* beta, float eps,
                  void* Y, int32_t y_type, lba_infmt y_fmt, float* mean, float* rstd,
                  int64_t M, int64_t N, void* hip_stream) {
    int rc = check_rows(M, N);
    if (rc == LBA_OK) rc = check_float_type(x_type);
    if (rc == LBA_OK) rc = check_out_type(y_type, y_fmt);
    if (rc != LBA_OK) return rc;
    if (M == 0 || (N == 0 && !mean && !rstd)) return LBA_OK;
    if (N > 0 && (!X || !Y)) return LBA_ERR_NULL;        // rows of no elements: the kernel reads none, and their mean is 0 / 0
    NormParams p = {};
    p.X = X; p.gamma = gamma; p.beta = beta; p.Y = Y; p.mean = mean; p.rstd = rstd;
    p.M = M; p.N = (int32_t)N; p.eps = eps; p.n = (float)N;
    if (y_type == LBA_CODE8) p.fmt = make_code_fmt(y_fmt);
    const hipStream_t st = (hipStream_t)hip_stream;
    if (x_type == LBA_F32) {
        if (y_type == LBA_F32) norm_fwd<float, float>(p, st);
        else if (y_type == LBA_BF16) norm_fwd<float, bf16_t>(p, st);
        else norm_fwd<float, uint8_t>(p, st);
    } else {
        if (y_type == LBA_F32) norm_fwd<bf16_t, float>(p, st);
        else if (y_type == LBA_BF16) norm_fwd<bf16_t, bf16_t>(p, st);
        else norm_fwd<bf16_t, uint8_t>(p, st);
    }
    return hipGetLastError() == hipSuccess ? LBA_OK : LBA_ERR_LAUNCH;
}

size_t lba_layernorm_bwd_workspace_bytes(int64_t M, int64_t N) {
    if (check_rows(M, N) != LBA_OK || M == 0 || N == 0) return 0;
    return align256((size_t)norm_bwd_blocks(M, N) * 2 * (size_t)N * sizeof(float));
}

int lba_layernorm_bwd(const void* G, int32_t g_type, const void* X, int32_t x_type, const float* gamma,
                      const float* mean, const float* rstd, void* dX, float* dgamma, float* dbeta,
                      int64_t M, int64_t N, void* workspace, size_t workspace_bytes, void* hip_stream) {
    int rc = check_rows(M, N);
    if (rc == LBA_OK) rc = check_float_type(g_type);
    if (rc == LBA_OK) rc = check_float_type(x_type);
    if (rc != LBA_OK) return rc;
    if (N == 0) return LBA_OK;
    const hipStream_t st = (hipStream_t)hip_stream;
    if (M == 0) {                                        // dX holds nothing: its address may be null
        if (!dgamma && !dbeta) return LBA_OK;
        if (dgamma) launch_zero(dgamma, N * 4, st);
        if (dbeta) launch_zero(dbeta, N * 4, st);
        return hipGetLastError() == hipSuccess ? LBA_OK : LBA_ERR_LAUNCH;
    }
    if (!dX && !dgamma && !dbeta) return LBA_ERR_NULL;
    if (!G || !X || !mean || !rstd) return LBA_ERR_NULL;
    const bool params = dgamma || dbeta;
    if (params) {
        if (!workspace) return LBA_ERR_NULL;
        if ((uintptr_t)workspace % 256 != 0) return LBA_ERR_ALIGN;
        if (workspace_bytes < lba_layernorm_bwd_workspace_bytes(M, N)) return LBA_ERR_SHAPE;
    }
    NormParams p = {};
    p.X = X; p.G = G; p.gamma = gamma; p.Y = dX; p.mean = (float*)mean; p.rstd = (float*)rstd;
    p.part = params ? (float*)workspace : nullptr;
    p.M = M; p.N = (int32_t)N; p.n = (float)N;
    if (g_type == LBA_F32) {
        if (x_type == LBA_F32) norm_bwd<float, float>(p, st); else norm_bwd<float, bf16_t>(p, st);
    } else {
        if (x_type == LBA_F32) norm_bwd<bf16_t, float>(p, st); else norm_bwd<bf16_t, bf16_t>(p, st);
    }
    if (params) launch_column_sum(p.part, norm_bwd_blocks(M, N), 2 * N, dgamma, dbeta, N, st);
    return hipGetLastError() == hipSuccess ? LBA_OK : LBA_ERR_LAUNCH;
}

}  // extern "C"
