// lba_dense.hip -- the dense product's plan, its operands' copies, the joining of sliced sums, and the entry points.
//
// Operands whose rows the tile cannot read where they are (rows off 16 bytes, codes of five exponent bits, sums over rows) are laid out once
// per call in the workspace: a pass over one byte an element beside a product of K (or N) operations on each.
#include "lba_dense.h"
#include "lba_internal.h"

namespace lba {

constexpr int64_t up_to(int64_t x, int64_t m) { return (x + m - 1) / m * m; }

// ---- operands laid out for the tile ---------------------------------------------------------

struct RowsParams {
    const uint8_t* src;      // [R, K] codes
    uint8_t* dst;            // rows of ld bytes, zeros behind K
    int64_t R, ld;
    int32_t K;
    CodeBits bits;
};

// 16 bytes of output a lane: codes as they are, or as bfloat16 numbers
template <bool BF16> __global__ __launch_bounds__(256) void dense_rows_kernel(RowsParams p) {
    constexpr int PER = BF16 ? 8 : 16;
    const int64_t per_row = p.ld / 16, total = p.R * per_row;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        const int64_t r = i / per_row;
        const int k = (int)(i - r * per_row) * PER;
        const uint8_t* s = p.src + r * p.K + k;
        uint32_t w[PER / 4];
        if (k + PER <= p.K) {
            typedef uint32_t words __attribute__((ext_vector_type(PER / 4), aligned(1)));
            const words x = *(const words*)s;
#pragma unroll
            for (int j = 0; j < PER / 4; ++j) w[j] = x[j];
        } else {
#pragma unroll
            for (int j = 0; j < PER / 4; ++j) w[j] = 0;
#pragma unroll
            for (int j = 0; j < PER; ++j)
                if (k + j < p.K) w[j / 4] |= (uint32_t)s[j] << (8 * (j % 4));
        }
        i32x4 o;
        if (BF16) {
            uint32_t lo, hi;
            code_bf16(w[0], p.bits, lo, hi); o[0] = (int32_t)lo; o[1] = (int32_t)hi;
            code_bf16(w[1], p.bits, lo, hi); o[2] = (int32_t)lo; o[3] = (int32_t)hi;
        } else {
            for (int j = 0; j < 4; ++j) o[j] = (int32_t)w[j % (PER / 4)];
        }
        *(i32x4*)(p.dst + r * p.ld + (int64_t)(i - r * per_row) * 16) = o;
    }
}

struct TransposedParams {
    const uint8_t* src;      // [R, K] codes
    bf16_t* dst;             // [K][ld], R columns and zeros up to `wide`, a multiple of 8
    int64_t R, ld, wide;
    int32_t K;
    int32_t tiles_k;
    CodeBits bits;
};

// 64 x 64 codes through LDS: read along k, written along the rows as bfloat16
__global__ __launch_bounds__(256) void dense_transposed_kernel(TransposedParams p) {
    __shared__ uint8_t t[64][68];
    const int64_t r0 = (int64_t)(blockIdx.x / p.tiles_k) * 64;
    const int k0 = (int)(blockIdx.x % p.tiles_k) * 64;
    for (int i = threadIdx.x; i < 64 * 16; i += 256) {
        const int r = i / 16, k = (i % 16) * 4;
        uint32_t w = 0;
        if (r0 + r < p.R) {
            const uint8_t* s = p.src + (r0 + r) * p.K + k0 + k;
            typedef uint32_t word_any __attribute__((aligned(1)));
            if (k0 + k + 4 <= p.K) w = *(const word_any*)s;
            else
                for (int j = 0; j < 4; ++j)
                    if (k0 + k + j < p.K) w |= (uint32_t)s[j] << (8 * j);
        }
        *(uint32_t*)&t[r][k] = w;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < 64 * 8; i += 256) {
        const int k = i / 8, r = (i % 8) * 8;
        if (k0 + k >= p.K || r0 + r >= p.wide) continue;
        i32x4 o;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t a = __float_as_uint(code_value(t[r + 2 * j][k], p.bits)), b = __float_as_uint(code_value(t[r + 2 * j + 1][k], p.bits));
            o[j] = (int32_t)__builtin_amdgcn_perm(b, a, 0x07060302u);
        }
        *(i32x4*)(p.dst + (int64_t)(k0 + k) * p.ld + r0 + r) = o;
    }
}

// adds the slices of a product's sums, in order, and finishes the outputs
template <bool GATED> __global__ __launch_bounds__(256) void dense_join_kernel(EpiParams e, const float* split, int32_t slices, int32_t cols) {
    const int64_t quads = (e.N + 3) / 4, total = quads * e.M, plane = (int64_t)e.M * cols;
    const uint64_t base = e.drop.threshold ? drop_base(e.drop) : 0;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        const int64_t m = i / quads;
        const int n = (int)(i - m * quads) * 4;
        float z[4] = {0.0f, 0.0f, 0.0f, 0.0f}, u[4] = {0.0f, 0.0f, 0.0f, 0.0f}, v[4];
        const float* s = split + m * cols + n;
        for (int q = 0; q < slices; ++q) {
            load_some<4>(s + q * plane, e.N - n, v);
#pragma unroll
            for (int j = 0; j < 4; ++j) z[j] += v[j];
            if (GATED) {
                load_some<4>(s + q * plane + e.N, e.N - n, v);
#pragma unroll
                for (int j = 0; j < 4; ++j) u[j] += v[j];
            }
        }
        float r[4];
        load_extra(e, e.R, e.r_type, (int)m, n, r);
        finish_forward<GATED>(e, columns_of<GATED>(e, n), base, (int)m, z, u, r);
    }
}

// ---- plan -----------------------------------------------------------------------------------

static unsigned grid_of(int64_t items) {
    const int64_t blocks = (items + 255) / 256;
    return (unsigned)(blocks < 1 ? 1 : blocks < 65536 ? blocks : 65536);
}

// tile and slices of a product of rows x cols outputs over `steps` steps
struct TilePlan { int tile, slices, per_slice; int64_t split_floats; };
static TilePlan plan_tile(int64_t rows, int64_t cols, bool gated, int64_t steps, bool may_split) {
    (void)may_split;
    TilePlan t = {TILE_64, 1, (int)steps, 0};
    const int64_t c = gated ? cols / 2 * 2 : cols;
    auto tiles = [&](int b) { return ((rows + b - 1) / b) * ((c + b - 1) / b); };
    if (tiles(256) >= 192) t.tile = TILE_256;
    else if (tiles(128) >= 192) t.tile = TILE_128;
    return t;
}

static int check_infmt(const lba_infmt& f) {
    return f.exp_bits < 2 || f.exp_bits > 5 || f.man_bits != 7 - f.exp_bits || f.bias < -32 || f.bias > 32 ? LBA_ERR_FORMAT : LBA_OK;
}
static int check_dense(int64_t M, int64_t N, int64_t K, const lba_infmt& fa, const lba_infmt& fb) {
    if (M < 0 || N < 0 || K < 0 || M > ((int64_t)1 << 30) || N > ((int64_t)1 << 20) || K > ((int64_t)1 << 30)) return LBA_ERR_SHAPE;
    return check_infmt(fa) != LBA_OK ? LBA_ERR_FORMAT : check_infmt(fb);
}

// where everything stands in the workspace
struct DensePlan {
    int elem;
    bool in_place, token;
    int64_t cols;            // rows of B
    int64_t ld;              // bytes of a laid-out row
    int64_t steps, chunks;
    TilePlan fwd;
    size_t copy_a, copy_b, split, bytes;
};

static DensePlan plan_forward(int64_t M, int64_t N, int64_t K, const lba_infmt& fa, const lba_infmt& fb, bool gated, bool aligned) {
    DensePlan d = {};
    d.elem = elem_of(fa, fb);
    d.token = M <= kTokenRows;
    d.cols = gated ? 2 * N : N;
    d.in_place = d.token || (d.elem != ELEM_BF16 && K % 16 == 0 && aligned);
    d.ld = d.elem != ELEM_BF16 ? up_to(K, 16) : 2 * up_to(K, 8);
    d.chunks = d.ld / 16;
    d.steps = (d.ld + 127) / 128;
    size_t at = 0;
    if (!d.in_place) {
        d.copy_a = at; at += align256((size_t)(M * d.ld));
        d.copy_b = at; at += align256((size_t)(d.cols * d.ld));
    }
    d.fwd = plan_tile(M, d.cols, gated, d.steps, true);
    d.split = at; at += align256((size_t)d.fwd.split_floats * 4);
    d.bytes = d.token ? 0 : at;
    return d;
}

struct BwdPlan {
    DensePlan f;             // the sums computed again
    bool sums;               // whether they are
    int pieces;
    int64_t ldp, ldt;        // elements of a row of the gradient matrix and of its transpose
    TilePlan da, db;
    int64_t part_rows;
    size_t p, pt, at, bt, part, split, bytes;
};

static BwdPlan plan_backward(int64_t M, int64_t N, int64_t K, const lba_infmt& fa, const lba_infmt& fb, bool gated, int act, int g_type, bool aligned) {
    BwdPlan b = {};
    b.sums = act != LBA_ACT_NONE || gated;
    b.f = plan_forward(M, N, K, fa, fb, gated, aligned);
    DensePlan& f = b.f;
    // the sums again, always by the tile: few rows as well
    f.token = false;
    f.in_place = f.elem != ELEM_BF16 && K % 16 == 0 && aligned;
    f.fwd = plan_tile(M, f.cols, gated, f.steps, false);
    size_t at = 0;
    if (b.sums && !f.in_place) {
        f.copy_a = at; at += align256((size_t)(M * f.ld));
        f.copy_b = at; at += align256((size_t)(f.cols * f.ld));
    }
    b.pieces = g_type == LBA_F32 ? 3 : 1;
    b.ldp = (gated ? 2 : 1) * up_to(N, 8);
    b.ldt = up_to(M, 8);
    b.p = at; at += align256((size_t)(b.pieces * M * b.ldp) * 2);
    b.pt = at; at += align256((size_t)(b.pieces * f.cols * b.ldt) * 2);
    b.at = at; at += align256((size_t)(K * b.ldt) * 2);
    b.bt = at; at += align256((size_t)(K * b.ldp) * 2);
    const TileShape s = tile_shape(f.fwd.tile);
    b.part_rows = (M + s.bm - 1) / s.bm * s.wm;
    b.part = at; at += align256((size_t)(b.part_rows * f.cols) * 4);
    b.da = plan_tile(M, K, false, (b.ldp * 2 + 127) / 128 * b.pieces, true);
    b.db = plan_tile(f.cols, K, false, (b.ldt * 2 + 127) / 128 * b.pieces, true);
    const int64_t most = b.da.split_floats > b.db.split_floats ? b.da.split_floats : b.db.split_floats;
    b.split = at; at += align256((size_t)most * 4);
    b.bytes = at;
    return b;
}

static bool fits_a_launch(int64_t rows, int64_t cols, const TilePlan& t) {
    const TileShape s = tile_shape(t.tile);
    const int64_t tiles = ((rows + s.bm - 1) / s.bm) * ((cols + s.bn / 2 - 1) / (s.bn / 2));
    return tiles < ((int64_t)1 << 22);                   // fewer than 2^32 lanes
}

static void lay_rows(const uint8_t* src, uint8_t* dst, int64_t R, int64_t K, int64_t ld, int elem, const lba_infmt& f, hipStream_t st) {
    if (R == 0 || ld == 0) return;
    RowsParams p = {src, dst, R, ld, (int32_t)K, make_code_bits(f)};
    const dim3 grid(grid_of(R * (ld / 16)));
    if (elem != ELEM_BF16) hipLaunchKernelGGL(dense_rows_kernel<false>, grid, dim3(256), 0, st, p);
    else hipLaunchKernelGGL(dense_rows_kernel<true>, grid, dim3(256), 0, st, p);
}

static void lay_transposed(const uint8_t* src, bf16_t* dst, int64_t R, int64_t K, int64_t ld, const lba_infmt& f, hipStream_t st) {
    if (K == 0 || ld == 0) return;
    TransposedParams p = {src, dst, R, ld, up_to(R, 8), (int32_t)K, (int32_t)((K + 63) / 64), make_code_bits(f)};
    hipLaunchKernelGGL(dense_transposed_kernel, dim3((unsigned)(p.tiles_k * ((R + 63) / 64))), dim3(256), 0, st, p);
}

static void run_product(GemmParams& g, const TilePlan& t, int elem, bool gated, int epi, float* split, hipStream_t st) {
    g.slices = t.slices;
    g.per_slice = t.per_slice;
    g.split = t.slices > 1 ? split : nullptr;
    if (elem == ELEM_E4M3) launch_dense_e4m3(g, t.tile, gated, epi, st);
    else if (elem == ELEM_F16) launch_dense_f16(g, t.tile, gated, epi, st);
    else launch_dense_bf16(g, t.tile, gated, epi, st);
    if (t.slices > 1) {
        const dim3 grid(grid_of((int64_t)g.e.M * ((g.e.N + 3) / 4)));
        if (gated) hipLaunchKernelGGL(dense_join_kernel<true>, grid, dim3(256), 0, st, g.e, split, t.slices, g.rows_b);
        else hipLaunchKernelGGL(dense_join_kernel<false>, grid, dim3(256), 0, st, g.e, split, t.slices, g.rows_b);
    }
}

static int check_workspace(const void* ws, size_t have, size_t need) {
    if (need == 0) return LBA_OK;
    if (!ws) return LBA_ERR_NULL;
    if ((uintptr_t)ws % 256 != 0) return LBA_ERR_ALIGN;
    return have < need ? LBA_ERR_SHAPE : LBA_OK;
}

static bool aligned16(const void* a, const void* b) { return ((uintptr_t)a | (uintptr_t)b) % 16 == 0; }

}  // namespace lba

using namespace lba;

extern "C" {

size_t lba_dense_workspace_bytes(int64_t M, int64_t N, int64_t K, lba_infmt fmt_a, lba_infmt fmt_b, int32_t gated, int32_t aligned) {
    if (check_dense(M, N, K, fmt_a, fmt_b) != LBA_OK || M == 0 || N == 0) return 0;
    return plan_forward(M, N, K, fmt_a, fmt_b, gated != 0, aligned != 0).bytes;
}

int lba_dense(const uint8_t* A, const uint8_t* B, int64_t M, int64_t N, int64_t K, lba_infmt fmt_a, lba_infmt fmt_b, int32_t gated,
              const float* bias, int32_t act, lba_drop drop, const void* residual, int32_t r_type,
              void* Y, int32_t y_type, lba_infmt y_fmt, void* workspace, size_t workspace_bytes, void* hip_stream) {
    EpiParams e = {};
    int rc = check_dense(M, N, K, fmt_a, fmt_b);
    if (rc == LBA_OK && residual) rc = check_float_type(r_type);
    if (rc == LBA_OK) rc = check_out_type(y_type, y_fmt);
    if (rc == LBA_OK) rc = check_act(act);
    if (rc == LBA_OK) rc = check_drop(drop, &e.drop);
    if (rc != LBA_OK) return rc;
    if (M == 0 || N == 0) return LBA_OK;
    if (!Y || (K > 0 && (!A || !B))) return LBA_ERR_NULL;
    const bool two = gated != 0;
    const DensePlan d = plan_forward(M, N, K, fmt_a, fmt_b, two, aligned16(A, B));
    if (!d.token && !fits_a_launch(M, d.cols, d.fwd)) return LBA_ERR_SHAPE;
    rc = check_workspace(workspace, workspace_bytes, d.bytes);
    if (rc != LBA_OK) return rc;
    const ElemFmt ea = make_elem(fmt_a, d.elem), eb = make_elem(fmt_b, d.elem);
    e.scale = ea.factor * eb.factor;
    e.bias = bias; e.act = act; e.M = (int32_t)M; e.N = (int32_t)N;
    e.R = residual; e.r_type = r_type; e.Y = Y; e.y_type = y_type;
    if (y_type == LBA_CODE8) e.fmt = make_code_fmt(y_fmt);
    const hipStream_t st = (hipStream_t)hip_stream;
    if (d.token) {
        TokenParams t = {A, B, (int32_t)M, (int32_t)K, (int32_t)d.cols, (int32_t)N, ea, eb, make_code_bits(fmt_a), make_code_bits(fmt_b), e};
        launch_dense_token(t, d.elem, two, st);
        return hipGetLastError() == hipSuccess ? LBA_OK : LBA_ERR_LAUNCH;
    }
    uint8_t* ws = (uint8_t*)workspace;
    GemmParams g = {};
    g.A = A; g.B = B; g.lda = g.ldb = d.ld;
    if (!d.in_place) {
        lay_rows(A, ws + d.copy_a, M, K, d.ld, d.elem, fmt_a, st);
        lay_rows(B, ws + d.copy_b, d.cols, K, d.ld, d.elem, fmt_b, st);
        g.A = ws + d.copy_a; g.B = ws + d.copy_b;
    }
    g.pieces = 1; g.rows_a = (int32_t)M; g.rows_b = (int32_t)d.cols; g.half = (int32_t)N;
    g.chunks = (int32_t)d.chunks; g.steps = (int32_t)d.steps;
    g.shift_a = ea.shift; g.shift_b = eb.shift; g.keep_a = ea.keep; g.keep_b = eb.keep;
    g.e = e;
    run_product(g, d.fwd, d.elem, two, EPI_FORWARD, (float*)(ws + d.split), st);
    return hipGetLastError() == hipSuccess ? LBA_OK : LBA_ERR_LAUNCH;
}

size_t lba_dense_bwd_workspace_bytes(int64_t M, int64_t N, int64_t K, lba_infmt fmt_a, lba_infmt fmt_b, int32_t gated, int32_t act,
                                     int32_t g_type, int32_t aligned) {
    if (check_dense(M, N, K, fmt_a, fmt_b) != LBA_OK || check_act(act) != LBA_OK || check_float_type(g_type) != LBA_OK || M == 0 || N == 0) return 0;
    return plan_backward(M, N, K, fmt_a, fmt_b, gated != 0, act, g_type, aligned != 0).bytes;
}

int lba_dense_bwd(const void* G, int32_t g_type, const uint8_t* A, const uint8_t* B, int64_t M, int64_t N, int64_t K,
                  lba_infmt fmt_a, lba_infmt fmt_b, int32_t gated, const float* bias, int32_t act, lba_drop drop,
                  void* dA, void* dB, float* dbias, void* workspace, size_t workspace_bytes, void* hip_stream) {
    EpiParams e = {};
    int rc = check_dense(M, N, K, fmt_a, fmt_b);
    if (rc == LBA_OK) rc = check_float_type(g_type);
    if (rc == LBA_OK) rc = check_act(act);
    if (rc == LBA_OK) rc = check_drop(drop, &e.drop);
    if (rc != LBA_OK) return rc;
    if (!dA && !dB && !dbias) return LBA_ERR_NULL;
    const hipStream_t st = (hipStream_t)hip_stream;
    const bool two = gated != 0;
    const int64_t cols = two ? 2 * N : N, size = g_type == LBA_F32 ? 4 : 2;
    if (M == 0 || N == 0) {                              // sums of nothing
        if (dA) launch_zero(dA, M * K * size, st);
        if (dB) launch_zero(dB, cols * K * size, st);
        if (dbias) launch_zero(dbias, cols * 4, st);
        return hipGetLastError() == hipSuccess ? LBA_OK : LBA_ERR_LAUNCH;
    }
    const BwdPlan b = plan_backward(M, N, K, fmt_a, fmt_b, two, act, g_type, aligned16(A, B));
    if (!G || (K > 0 && (((dA || b.sums) && !B) || ((dB || b.sums) && !A)))) return LBA_ERR_NULL;
    if (!fits_a_launch(M, cols, b.f.fwd) || !fits_a_launch(M, K, b.da) || !fits_a_launch(cols, K, b.db)) return LBA_ERR_SHAPE;
    rc = check_workspace(workspace, workspace_bytes, b.bytes);
    if (rc != LBA_OK) return rc;
    uint8_t* ws = (uint8_t*)workspace;
    bf16_t* P = (bf16_t*)(ws + b.p);
    bf16_t* PT = (bf16_t*)(ws + b.pt);

    // the gradient of the sums
    const ElemFmt ea = make_elem(fmt_a, b.f.elem), eb = make_elem(fmt_b, b.f.elem);
    e.scale = ea.factor * eb.factor;
    e.bias = b.sums ? bias : nullptr; e.act = act; e.M = (int32_t)M; e.N = (int32_t)N;
    e.G = G; e.g_type = g_type; e.pieces = b.pieces;
    e.P = dA ? P : nullptr; e.PT = dB ? PT : nullptr;
    e.ldp = b.ldp; e.ldt = b.ldt; e.wide = (int32_t)up_to(N, 8); e.p_piece = M * b.ldp; e.pt_piece = cols * b.ldt;
    e.part = dbias ? (float*)(ws + b.part) : nullptr;
    GemmParams g = {};
    g.A = A; g.B = B; g.lda = g.ldb = b.f.ld;
    if (b.sums && !b.f.in_place) {
        lay_rows(A, ws + b.f.copy_a, M, K, b.f.ld, b.f.elem, fmt_a, st);
        lay_rows(B, ws + b.f.copy_b, cols, K, b.f.ld, b.f.elem, fmt_b, st);
        g.A = ws + b.f.copy_a; g.B = ws + b.f.copy_b;
    }
    g.pieces = 1; g.rows_a = (int32_t)M; g.rows_b = (int32_t)cols; g.half = (int32_t)N;
    g.chunks = b.sums ? (int32_t)b.f.chunks : 0; g.steps = b.sums ? (int32_t)b.f.steps : 0;
    g.shift_a = ea.shift; g.shift_b = eb.shift; g.keep_a = ea.keep; g.keep_b = eb.keep;
    g.e = e;
    run_product(g, b.f.fwd, b.f.elem, two, EPI_BACKWARD, nullptr, st);
    if (dbias) launch_column_sum(e.part, b.part_rows, cols, dbias, nullptr, cols, st);

    // the two products of it
    EpiParams o = {};
    o.y_type = g_type;
    GemmParams q = {};
    q.pieces = b.pieces;
    q.rows_b = (int32_t)K; q.half = (int32_t)K;
    if (dA && K > 0) {
        lay_transposed(B, (bf16_t*)(ws + b.bt), N, K, b.ldp, fmt_b, st);
        if (two) lay_transposed(B + N * K, (bf16_t*)(ws + b.bt) + e.wide, N, K, b.ldp, fmt_b, st);
        q.A = (const uint8_t*)P; q.B = ws + b.bt; q.lda = q.ldb = b.ldp * 2; q.a_piece = e.p_piece * 2;
        q.rows_a = (int32_t)M; q.chunks = (int32_t)(b.ldp / 8); q.steps = (int32_t)((b.ldp * 2 + 127) / 128 * b.pieces);
        o.scale = make_elem(fmt_b, ELEM_BF16).factor; o.M = (int32_t)M; o.N = (int32_t)K; o.Y = dA;
        q.e = o;
        run_product(q, b.da, ELEM_BF16, false, EPI_FORWARD, (float*)(ws + b.split), st);
    }
    if (dB && K > 0) {
        lay_transposed(A, (bf16_t*)(ws + b.at), M, K, b.ldt, fmt_a, st);
        q.A = (const uint8_t*)PT; q.B = ws + b.at; q.lda = q.ldb = b.ldt * 2; q.a_piece = e.pt_piece * 2;
        q.rows_a = (int32_t)cols; q.chunks = (int32_t)(b.ldt / 8); q.steps = (int32_t)((b.ldt * 2 + 127) / 128 * b.pieces);
        o.scale = make_elem(fmt_a, ELEM_BF16).factor; o.M = (int32_t)cols; o.N = (int32_t)K; o.Y = dB;
        q.e = o;
        run_product(q, b.db, ELEM_BF16, false, EPI_FORWARD, (float*)(ws + b.split), st);
    }
    return hipGetLastError() == hipSuccess ? LBA_OK : LBA_ERR_LAUNCH;
}

}  // extern "C"
