// lba_dropout.hip -- dropout with bias, activation and residual, and its gradients (include/lba_layer.h).
//
// The mask is a function of (seed, stream, element index): 16 bits of a splitmix64 word for each element, four elements a word, so the
// backward pass makes it again and nothing of it is stored.  A word is two 64-bit products; on four elements that is less than
// the memory time of a bfloat16 element.
// A lane owns one vector of 16 bytes' worth of columns and walks over rows, so a bias is loaded once and the column sums of the
// backward pass, dbias, stay in registers; a workgroup writes one row of partial sums, and a second launch adds them in a fixed order.
// Columns beyond the last full strip of 64 vectors have lanes of their own: as many rows side by side in a wave as they fit.
// Measured, memory the bound: 4096 x 768 float32 with bias and residual 8.0 us, 4.7 TB/s; 16411 x 4099 bfloat16 with GELU forward 61 us,
// 4.4 TB/s, backward with the column sums 88 + 5 us, 4.4 TB/s (95 + 5 without the next row under way; a tenth fewer instructions changed
// nothing).
#include "lba_layer_device.h"
#include "lba_internal.h"

namespace lba {

struct DropoutParams {
    const void* X;
    const void* G;
    const void* R;
    const float* bias;
    void* Y;                 // forward: y; backward: dx
    float* part;             // backward: [chunks][N] partial sums, or null
    int64_t M;
    int32_t N;
    int32_t r_type;
    float scale;
    int32_t strips;          // full strips of 64 vectors; workgroups below main_blocks belong to them
    int32_t main_blocks, main_chunks, tail_chunks;
    int64_t main_rows, tail_rows;     // rows of a chunk
    int32_t tail_log;        // log2 of the lanes that share a row of the tail
    DropParams drop;
    CodeFmt fmt;
};

// where a lane stands: its columns, its first row, the step to its next one and the end of its chunk
struct LanePlace { int col, cols; int64_t row, end; int step, chunk, lanes_log; };
template <int V> __device__ __forceinline__ LanePlace lane_place(const DropoutParams& p) {
    LanePlace q;
    const int lane = threadIdx.x & 63, wave = threadIdx.x / 64;
    const bool tail = (int)blockIdx.x >= p.main_blocks;
    const int b = tail ? (int)blockIdx.x - p.main_blocks : (int)blockIdx.x;
    q.lanes_log = tail ? p.tail_log : 6;
    const int strip = tail ? p.strips : b % p.strips;
    q.chunk = tail ? b : b / p.strips;
    q.col = strip * 64 * V + (lane & ((1 << q.lanes_log) - 1)) * V;
    q.cols = p.N - q.col;
    const int64_t rows = tail ? p.tail_rows : p.main_rows;
    q.row = q.chunk * rows + (wave << (6 - q.lanes_log)) + (lane >> q.lanes_log);
    q.end = q.chunk * rows + rows < p.M ? q.chunk * rows + rows : p.M;
    q.step = 4 << (6 - q.lanes_log);
    return q;
}

// A row's vector of a lane: in a full strip whole, and the wave's lanes, all of which take part, share the words of the generator.
template <bool FULL, int V, typename T> __device__ __forceinline__ void load_part(const T* at, int n, float (&v)[V]) {
    if constexpr (FULL) load_vec<V>(at, v);
    else load_some<V>(at, n, v);
}
template <bool FULL, typename T, int V> __device__ __forceinline__ Raw<T, V> raw_part(const T* at, int n) {
    return load_raw<T, V>(at, FULL ? V : n);
}
// a lane's rows, the next one under way while one is worked on (two sets of registers, so that none is moved while in flight)
template <typename Row, typename Load, typename Work> __device__ __forceinline__ void walk(const LanePlace& q, const Load& load, const Work& work) {
    Row a, b;
    int64_t row = q.row;
    if (row < q.end) load(row, a);
#pragma unroll 1
    for (; row < q.end; row += 2 * q.step) {
        const bool more = row + q.step < q.end;
        if (more) load(row + q.step, b);
        work(row, a);
        if (!more) break;
        if (row + 2 * q.step < q.end) load(row + 2 * q.step, a);
        work(row + q.step, b);
    }
}
template <bool FULL, int V> __device__ __forceinline__ void keeps(const DropoutParams& p, const LanePlace& q, int64_t row, int64_t i, uint64_t base, bool (&keep)[V]) {
    if constexpr (FULL && V == 8) {
        const int64_t first = (int64_t)__builtin_amdgcn_readfirstlane((int)row) * p.N + __builtin_amdgcn_readfirstlane(q.col);
        drop_keeps_wave((uint64_t)first, base, p.drop, (p.N & 3) == 0, keep);
    } else {
        drop_keeps<V>((uint64_t)i, base, p.drop, (p.N & 3) == 0, keep);
    }
}

template <typename TX, typename TY, int ACT>
__global__ __launch_bounds__(256) void dropout_fwd_kernel(DropoutParams p) {
    constexpr int V = 16 / sizeof(TX);
    const LanePlace q = lane_place<V>(p);
    if (q.cols <= 0) return;
    const uint64_t base = drop_base(p.drop);
    float bias[V];
#pragma unroll
    for (int j = 0; j < V; ++j) bias[j] = 0.0f;
    if (p.bias) load_some<V>(p.bias + q.col, q.cols, bias);
    auto rows = [&](auto full) {
        constexpr bool FULL = decltype(full)::value != 0;
        // (The next row under way, as in the backward pass, did not pay here, with four times its workgroups: 61 us became 70.)
#pragma unroll 1
        for (int64_t row = q.row; row < q.end; row += q.step) {
            const int64_t i = row * p.N + q.col;
            float x[V], r[V];
            bool keep[V];
            load_part<FULL, V>((const TX*)p.X + i, q.cols, x);
            if (p.R && p.r_type == LBA_F32) load_part<FULL, V>((const float*)p.R + i, q.cols, r);
            else if (p.R) load_part<FULL, V>((const bf16_t*)p.R + i, q.cols, r);
            if (p.drop.on) keeps<FULL, V>(p, q, row, i, base, keep);
#pragma unroll
            for (int j = 0; j < V; ++j) x[j] = act_value<ACT>(fmaf(x[j], p.scale, bias[j]));
            if (p.drop.on) {
#pragma unroll
                for (int j = 0; j < V; ++j) x[j] = keep[j] ? x[j] * p.drop.keep_scale : 0.0f;
            }
            if (p.R) {
#pragma unroll
                for (int j = 0; j < V; ++j) x[j] += r[j];
            }
            if constexpr (FULL) store_vec<V>((TY*)p.Y + i, x, p.fmt);
            else store_some<V>((TY*)p.Y + i, q.cols, x, p.fmt);
        }
    };
    if ((int)blockIdx.x < p.main_blocks) rows(Known<1>{});
    else rows(Known<0>{});
}

template <typename TG, typename TX, int ACT>
__global__ __launch_bounds__(256) void dropout_bwd_kernel(DropoutParams p) {
    constexpr int V = 16 / sizeof(TX);
    typedef typename Bits<TX>::type BX;
    typedef typename Bits<TG>::type BG;
    const LanePlace q = lane_place<V>(p);
    const uint64_t base = drop_base(p.drop);
    float bias[V], sum[V];
#pragma unroll
    for (int j = 0; j < V; ++j) bias[j] = sum[j] = 0.0f;
    constexpr bool read_x = ACT != LBA_ACT_NONE;
    const float keep_scale = p.drop.on ? p.drop.keep_scale : 1.0f, dx_scale = p.scale * keep_scale;
    if (p.bias && read_x) load_some<V>(p.bias + q.col, q.cols, bias);
    auto rows = [&](auto full) {
        constexpr bool FULL = decltype(full)::value != 0;
        struct Row { Raw<BG, V> g; Raw<BX, V> x; };
        auto load = [&](int64_t row, Row& w) {
            const int64_t i = row * p.N + q.col;
            w.g = raw_part<FULL, BG, V>((const BG*)p.G + i, q.cols);
            if (read_x) w.x = raw_part<FULL, BX, V>((const BX*)p.X + i, q.cols);
        };
        auto work = [&](int64_t row, const Row& w) {
            const int64_t i = row * p.N + q.col;
            float g[V];
            bool keep[V];
            if (p.drop.on) keeps<FULL, V>(p, q, row, i, base, keep);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                g[j] = raw_at(w.g, j);
                if (read_x) {
                    float value, slope;
                    act_both<ACT>(fmaf(raw_at(w.x, j), p.scale, bias[j]), value, slope);
                    g[j] *= slope;
                }
            }
            if (p.drop.on) {
#pragma unroll
                for (int j = 0; j < V; ++j) g[j] = keep[j] ? g[j] : 0.0f;
            }
#pragma unroll
            for (int j = 0; j < V; ++j) {
                sum[j] += g[j];                          // what is kept is scaled once, at the end
                g[j] *= dx_scale;
            }
            if (p.Y) {
                if constexpr (FULL) store_vec<V>((TX*)p.Y + i, g, p.fmt);
                else store_some<V>((TX*)p.Y + i, q.cols, g, p.fmt);
            }
        };
        walk<Row>(q, load, work);
    };
    if ((int)blockIdx.x < p.main_blocks) rows(Known<1>{});
    else if (q.cols > 0) rows(Known<0>{});
    if (!p.part) return;
    // the lanes that own the same columns: within the wave, then its four sums
    const int lanes = 1 << q.lanes_log;
    for (int d = lanes; d < 64; d *= 2) {
#pragma unroll
        for (int j = 0; j < V; ++j) sum[j] += __shfl_xor(sum[j], d);
    }
    __shared__ float lds[4][64 * V];
#pragma unroll
    for (int j = 0; j < V; ++j) lds[threadIdx.x / 64][j * 64 + (threadIdx.x & 63)] = sum[j];
    __syncthreads();
    if ((int)threadIdx.x >= lanes || q.cols <= 0) return;
#pragma unroll
    for (int j = 0; j < V; ++j) {
        const int at = j * 64 + threadIdx.x;
        sum[j] = ((lds[0][at] + lds[1][at]) + (lds[2][at] + lds[3][at])) * keep_scale;
    }
    store_some<V>(p.part + (int64_t)q.chunk * p.N + q.col, q.cols, sum, p.fmt);
}

// ---- launchers ------------------------------------------------------------------------------

// How rows and columns are cut.  A chunk is a multiple of the rows a workgroup has in flight; the chip holds about 2048 workgroups of
// four waves, and the backward pass writes a row of sums for each chunk, so it takes fewer of them.
static int64_t chunk_rows(int64_t M, int64_t step, int64_t strips, int64_t most) {
    const int64_t chunks = most / (strips < 1 ? 1 : strips) < 1 ? 1 : most / (strips < 1 ? 1 : strips);
    const int64_t rows = (M + chunks - 1) / chunks;
    return (rows + step - 1) / step * step;
}

constexpr int64_t kFwdBlocks = 8192, kBwdBlocks = 2048;

// both passes' cut for vectors of v elements; the number of chunks that write partial sums is the larger of the two
static unsigned dropout_cut(DropoutParams* p, int v, int64_t most) {
    p->strips = p->N / (64 * v);
    const int tail_cols = p->N - p->strips * 64 * v;
    int64_t blocks = 0;
    p->main_blocks = p->main_chunks = p->tail_chunks = 0;
    if (p->strips > 0) {
        p->main_rows = chunk_rows(p->M, 4, p->strips, most);
        p->main_chunks = (int32_t)((p->M + p->main_rows - 1) / p->main_rows);
        p->main_blocks = p->main_chunks * p->strips;
        blocks = p->main_blocks;
    }
    if (tail_cols > 0) {
        p->tail_log = 0;
        while ((v << p->tail_log) < tail_cols) ++p->tail_log;
        // as many chunks as the strips beside it have, or as fill the chip alone
        const int64_t share = p->strips > 0 ? p->main_chunks : most;
        p->tail_rows = chunk_rows(p->M, 4 << (6 - p->tail_log), 1, share);
        p->tail_chunks = (int32_t)((p->M + p->tail_rows - 1) / p->tail_rows);
        blocks += p->tail_chunks;
    }
    return (unsigned)blocks;
}

}  // namespace lba

using namespace lba;

extern "C" {

int lba_dropout(const void* X, int32_t x_type, float scale, const float* bias, int32_t act, lba_drop drop,
                const void* residual, int32_t r_type, void* Y, int32_t y_type, lba_infmt y_fmt,
                int64_t M, int64_t N, void* hip_stream) {
    DropoutParams p = {};
    int rc = check_rows(M, N);
    if (rc == LBA_OK) rc = check_float_type(x_type);
    if (rc == LBA_OK && residual) rc = check_float_type(r_type);
    if (rc == LBA_OK) rc = check_out_type(y_type, y_fmt);
    if (rc == LBA_OK) rc = check_act(act);
    if (rc == LBA_OK) rc = check_drop(drop, &p.drop);
    if (rc != LBA_OK) return rc;
    if (M == 0 || N == 0) return LBA_OK;
    if (!X || !Y) return LBA_ERR_NULL;
    p.X = X; p.R = residual; p.bias = bias; p.Y = Y; p.M = M; p.N = (int32_t)N; p.r_type = r_type; p.scale = scale;
    if (y_type == LBA_CODE8) p.fmt = make_code_fmt(y_fmt);
    const dim3 grid(dropout_cut(&p, x_type == LBA_F32 ? 4 : 8, kFwdBlocks));
    const hipStream_t st = (hipStream_t)hip_stream;
#define LBA_DROPOUT(TX, TY) \
    do { \
        if (act == LBA_ACT_NONE) hipLaunchKernelGGL((dropout_fwd_kernel<TX, TY, LBA_ACT_NONE>), grid, dim3(256), 0, st, p); \
        else if (act == LBA_ACT_RELU) hipLaunchKernelGGL((dropout_fwd_kernel<TX, TY, LBA_ACT_RELU>), grid, dim3(256), 0, st, p); \
        else if (act == LBA_ACT_GELU) hipLaunchKernelGGL((dropout_fwd_kernel<TX, TY, LBA_ACT_GELU>), grid, dim3(256), 0, st, p); \
        else hipLaunchKernelGGL((dropout_fwd_kernel<TX, TY, LBA_ACT_SILU>), grid, dim3(256), 0, st, p); \
    } while (0)
    if (x_type == LBA_F32) {
        if (y_type == LBA_F32) LBA_DROPOUT(float, float);
        else if (y_type == LBA_BF16) LBA_DROPOUT(float, bf16_t);
        else LBA_DROPOUT(float, uint8_t);
    } else {
        if (y_type == LBA_F32) LBA_DROPOUT(bf16_t, float);
        else if (y_type == LBA_BF16) LBA_DROPOUT(bf16_t, bf16_t);
        else LBA_DROPOUT(bf16_t, uint8_t);
    }
#undef LBA_DROPOUT
    return hipGetLastError() == hipSuccess ? LBA_OK : LBA_ERR_LAUNCH;
}

size_t lba_dropout_bwd_workspace_bytes(int64_t M, int64_t N) {
    if (check_rows(M, N) != LBA_OK || M == 0 || N == 0) return 0;
    size_t most = 0;
    for (int v = 4; v <= 8; v += 4) {                    // either type of X
        DropoutParams p = {};
        p.M = M; p.N = (int32_t)N;
        dropout_cut(&p, v, kBwdBlocks);
        const size_t chunks = (size_t)(p.main_chunks > p.tail_chunks ? p.main_chunks : p.tail_chunks);
        if (chunks > most) most = chunks;
    }
    return align256(most * (size_t)N * sizeof(float));
}

int lba_dropout_bwd(const void* G, int32_t g_type, const void* X, int32_t x_type, float scale, const float* bias,
                    int32_t act, lba_drop drop, void* dX, float* dbias, int64_t M, int64_t N,
                    void* workspace, size_t workspace_bytes, void* hip_stream) {
    DropoutParams p = {};
    int rc = check_rows(M, N);
    if (rc == LBA_OK) rc = check_float_type(g_type);
    if (rc == LBA_OK) rc = check_float_type(x_type);
    if (rc == LBA_OK) rc = check_act(act);
    if (rc == LBA_OK) rc = check_drop(drop, &p.drop);
    if (rc != LBA_OK) return rc;
    if (N == 0) return LBA_OK;
    const hipStream_t st = (hipStream_t)hip_stream;
    if (M == 0) {                                        // dX holds nothing: its address may be null
        if (!dbias) return LBA_OK;
        launch_zero(dbias, N * 4, st);
        return hipGetLastError() == hipSuccess ? LBA_OK : LBA_ERR_LAUNCH;
    }
    if (!dX && !dbias) return LBA_ERR_NULL;
    if (!G || (act != LBA_ACT_NONE && !X)) return LBA_ERR_NULL;
    if (dbias) {
        if (!workspace) return LBA_ERR_NULL;
        if ((uintptr_t)workspace % 256 != 0) return LBA_ERR_ALIGN;
        if (workspace_bytes < lba_dropout_bwd_workspace_bytes(M, N)) return LBA_ERR_SHAPE;
    }
    p.X = X; p.G = G; p.bias = bias; p.Y = dX; p.part = dbias ? (float*)workspace : nullptr;
    p.M = M; p.N = (int32_t)N; p.scale = scale;
    const dim3 grid(dropout_cut(&p, x_type == LBA_F32 ? 4 : 8, kBwdBlocks));
#define LBA_DROPOUT(TG, TX) \
    do { \
        if (act == LBA_ACT_NONE) hipLaunchKernelGGL((dropout_bwd_kernel<TG, TX, LBA_ACT_NONE>), grid, dim3(256), 0, st, p); \
        else if (act == LBA_ACT_RELU) hipLaunchKernelGGL((dropout_bwd_kernel<TG, TX, LBA_ACT_RELU>), grid, dim3(256), 0, st, p); \
        else if (act == LBA_ACT_GELU) hipLaunchKernelGGL((dropout_bwd_kernel<TG, TX, LBA_ACT_GELU>), grid, dim3(256), 0, st, p); \
        else hipLaunchKernelGGL((dropout_bwd_kernel<TG, TX, LBA_ACT_SILU>), grid, dim3(256), 0, st, p); \
    } while (0)
    if (g_type == LBA_F32) {
        if (x_type == LBA_F32) LBA_DROPOUT(float, float); else LBA_DROPOUT(float, bf16_t);
    } else {
        if (x_type == LBA_F32) LBA_DROPOUT(bf16_t, float); else LBA_DROPOUT(bf16_t, bf16_t);
    }
#undef LBA_DROPOUT
    if (dbias) {
        // full strips and the tail are cut into chunks of their own number
        const int64_t full = (int64_t)p.strips * 64 * (x_type == LBA_F32 ? 4 : 8);
        launch_column_sum(p.part, p.main_chunks, N, dbias, nullptr, N, st, full, p.tail_chunks);
    }
    return hipGetLastError() == hipSuccess ? LBA_OK : LBA_ERR_LAUNCH;
}

}  // extern "C"
