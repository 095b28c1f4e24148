// lba_dense.hip -- the dense product's plan, its operands' copies, the joining of sliced sums, and the entry points.
//
// Operands whose rows the tile cannot read where they are (rows off 16 bytes, codes of five exponent bits, sums over rows) are laid out once
// per call in the workspace: a pass over one byte an element beside a product of K (or N) operations on each.  What the gradient products read is
// laid out by workgroups beside those of the gradient of the sums (12 M codes: 10 us in a launch of their own, none beside 105 us of sums);
// what the sums themselves read takes a launch before them (6 M codes: 5 us).
#include "lba_dense.h"
#include "lba_internal.h"

namespace lba {

constexpr int64_t up_to(int64_t x, int64_t m) { return (x + m - 1) / m * m; }

__global__ __launch_bounds__(256) void dense_lay_kernel(LayJobs jobs) {
    __shared__ uint32_t t[kLayWords];
    lay_block(jobs, blockIdx.x, t);
}

// adds the slices of a product's sums, in order, and finishes the outputs: of one product or of two
struct JoinPart { EpiParams e; const float* split; int32_t slices, cols; };
struct JoinPair { JoinPart p[2]; int32_t blocks; };
template <bool GATED> __global__ __launch_bounds__(256) void dense_join_kernel(JoinPair both) {
    const bool second = (int)blockIdx.x >= both.blocks;
    const JoinPart& p = both.p[second];
    const EpiParams& e = p.e;
    const int64_t first = second ? (int64_t)blockIdx.x - both.blocks : (int64_t)blockIdx.x, blocks = second ? (int64_t)gridDim.x - both.blocks : (int64_t)both.blocks;
    const int64_t quads = (e.N + 3) / 4, total = quads * e.M, plane = (int64_t)e.M * p.cols;
    const uint64_t base = e.drop.on ? drop_base(e.drop) : 0;
    for (int64_t i = first * 256 + threadIdx.x; i < total; i += blocks * 256) {
        const int64_t m = i / quads;
        const int n = (int)(i - m * quads) * 4;
        float z[4] = {0.0f, 0.0f, 0.0f, 0.0f}, u[4] = {0.0f, 0.0f, 0.0f, 0.0f}, r[4], v[4], w[4];
        const float* s = p.split + m * p.cols + n;
        load_extra<4>(e, (int)m, n, r);
#pragma unroll 4
        for (int q = 0; q < p.slices; ++q) {
            load_some<4>(s + q * plane, e.N - n, v);
            if (GATED) load_some<4>(s + q * plane + e.N, e.N - n, w);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                z[j] += v[j];
                if (GATED) u[j] += w[j];
            }
        }
        const Columns<GATED, 4> cols = columns_of<GATED, 4>(e, n);
        with_act(e.act, [&](auto act) { finish_forward<GATED, false, decltype(act)::value, 4>(e, cols, base, (int)m, At{m * e.N + n, 0}, z, u, r); });
    }
}

// ---- plan -----------------------------------------------------------------------------------

static int32_t join_blocks(const EpiParams& e) {
    const int64_t blocks = ((int64_t)e.M * ((e.N + 3) / 4) + 255) / 256;
    return (int32_t)(blocks < 16384 ? blocks : 16384);
}

// A product of rows x cols outputs over `steps` steps, and how it is cut.
struct Product { int64_t rows, cols, steps; int slices; int64_t per_slice; };
static int64_t tiles_of(const Product& p, int tile) {
    const TileShape s = tile_shape(tile);
    return ((p.rows + s.bm - 1) / s.bm) * ((p.cols + s.bn - 1) / s.bn);
}
static void cut(Product& p, int64_t slices) {
    p.per_slice = (p.steps + slices - 1) / slices;
    p.slices = p.per_slice > 0 ? (int)((p.steps + p.per_slice - 1) / p.per_slice) : 1;
    if (p.slices < 1) p.slices = 1;
}
// A launch holds fewer than 2^32 lanes.  Beside backward sums and gradient products run workgroups of their own: of at most three transposed
// copies, (R + 64) (K + 128) / 8192 <= 2^20 each, or 2^17 of column sums.
enum { PLAN_FORWARD = 0, PLAN_BACKWARD = 1 };             // with the backward epilogue only small tiles, and no slices
constexpr int64_t kBeside = (int64_t)1 << 22;
static bool fits_a_launch(const Product* p, int n, int tile, int kind) {
    int64_t tiles = n > 1 || kind == PLAN_BACKWARD ? kBeside : 0;
    for (int i = 0; i < n; ++i) tiles += tiles_of(p[i], tile) * p[i].slices;
    return tiles * tile_shape(tile).threads < (int64_t)1 << 32;
}
static size_t split_bytes(const Product& p) { return p.slices > 1 ? align256((size_t)(p.slices * p.rows * p.cols) * 4) : 0; }

// What a launch takes, in microseconds: a tile's workgroup needs `fixed` and `step` for each step where every CU holds `per_cu` of them, and
// `fixed1` and `step1` where it has the CU to itself.  Measured on grids of 1 to 8 rounds and 1 to 64 steps (4096 x 4096 and 1024 x 1024 outputs,
// K = 128 to 4096); a step of codes is 128 long, of bfloat16 rows 64.  The sums were stored as they are: what an epilogue adds is not in it, 4 us
// (tiles of 64) to 14 (256) for GELU, dropout and a float32 residual on 3985 x 770 x 768, whose sums take 13.2 us (11.5 here).  It did not change
// which tile is the fastest: 64 there, 128 on 8192 x 1024 x 1024 (22.5 and 29.4 us; 64: 25.9, 31.0), 256 on 4096 x 4096 x 1024 (38.4 and 47.9;
// 128: 40.2, 53.9), and backward 64, 128 and 128, as the costs have it.
// `f16`: what a step of codes that become FP16 numbers takes, whose conversions are five instructions for E4M3's two, and the more of them the
// smaller a wave's part of the tile is.
struct TileCost { int tile, per_cu; float fixed, step, fixed1, step1, f16; };
static const TileCost kCodes[] = {
    {TILE_256, 1, 9.0f, 2.45f, 9.0f, 2.3f, 1.2f}, {TILE_192, 1, 7.0f, 1.9f, 7.0f, 1.85f, 1.25f},
    {TILE_128, 2, 4.0f, 1.45f, 2.7f, 0.95f, 1.33f}, {TILE_64, 4, 2.6f, 0.95f, 0.6f, 0.47f, 1.5f}};
static const TileCost kRows[] = {
    {TILE_256, 1, 9.0f, 2.0f, 9.0f, 1.75f, 1.0f}, {TILE_128, 2, 4.0f, 0.97f, 2.7f, 0.85f, 1.0f}, {TILE_128_DEEP, 1, 3.0f, 0.75f, 3.0f, 0.6f, 1.0f},
    {TILE_64, 4, 2.6f, 0.62f, 0.6f, 0.55f, 1.0f}, {TILE_64_DEEP, 2, 1.4f, 0.5f, 0.6f, 0.42f, 1.0f}};
static const TileCost kThree[] = {                         // three pieces of A: steps of 64 bytes
    {TILE_256_THREE, 1, 9.0f, 2.4f, 9.0f, 2.4f, 1.0f}, {TILE_128_THREE, 2, 4.0f, 1.42f, 2.7f, 0.8f, 1.0f}, {TILE_64_THREE, 4, 2.6f, 1.1f, 0.6f, 0.5f, 1.0f}};
constexpr float kLaunch = 4.5f, kJoinRate = 5e6f;         // a launch alone; bytes a microsecond that the join moves
constexpr int kCus = 256;

// the end of `a` workgroups of duration da and then `b` of db on `slots` places, da >= db
static double finish_of(int64_t a, double da, int64_t b, double db, int64_t slots) {
    const int64_t rounds = a / slots, rest = a % slots;
    const double at = (double)rounds * da;
    if (b == 0) return at + (rest ? da : 0.0);
    if (rest == 0) return at + (double)((b + slots - 1) / slots) * db;
    const int64_t beside = (slots - rest) * (int64_t)(da / db);                      // of the second kind, beside the first's last round
    if (b <= beside) return at + da;
    return at + da + (double)((b - beside + slots - 1) / slots) * db;
}

static double cost_of(const Product* p, const int64_t* tiles, int n, const TileCost& c, float step_scale, float fixed_scale) {
    int64_t wgs[2] = {0, 0};
    double t = kLaunch, d[2] = {0.0, 0.0};
    int64_t all = 0;
    for (int i = 0; i < n; ++i) all += wgs[i] = tiles[i] * p[i].slices;
    const bool alone = all <= kCus;
    for (int i = 0; i < n; ++i) {
        d[i] = (alone ? c.fixed1 : c.fixed) * fixed_scale + (double)p[i].per_slice * (alone ? c.step1 : c.step) * step_scale;
        if (p[i].slices > 1) t += (p[i].slices + 1.0) * (double)p[i].rows * (double)p[i].cols * 4.0 / kJoinRate;
    }
    if (p[0].slices > 1 || (n > 1 && p[1].slices > 1)) t += kLaunch;
    const int x = n > 1 && d[1] > d[0] ? 1 : 0;
    const int64_t slots = (int64_t)kCus * c.per_cu;
    // between one and all places of a CU taken, a round is between the two durations
    if (!alone && all < slots && c.per_cu > 1) {
        const double share = (double)(all - kCus) / (double)(slots - kCus);
        for (int i = 0; i < n; ++i) {
            const double d1 = c.fixed1 * fixed_scale + (double)p[i].per_slice * c.step1 * step_scale;
            d[i] = d1 + (d[i] - d1) * share;
        }
    }
    return t + finish_of(wgs[x], d[x], wgs[1 - x], n > 1 ? d[1 - x] : 1.0, slots);
}

// Chooses the tile of a product, or of two that share a launch, and their slices: the least cost of those whose workgroups fit a launch.
static int plan_tile(Product* p, int n, int elem, int kind, bool gated, int pieces = 1) {
    const TileCost* all = pieces == 3 ? kThree : elem == ELEM_BF16 ? kRows : kCodes;
    const size_t bytes = pieces == 3 ? sizeof(kThree) : elem == ELEM_BF16 ? sizeof(kRows) : sizeof(kCodes);
    const int count = (int)(bytes / sizeof(TileCost));
    static const int kSlices[] = {1, 2, 3, 4, 5, 6, 8, 12, 16};
    int best = all[count - 1].tile;
    double least = 1e300;
    Product cut_best[2] = {p[0], n > 1 ? p[1] : p[0]};   // (where no tile fits a launch, which the entry points refuse)
    for (Product& q : cut_best) cut(q, 1);
    for (int t = 0; t < count; ++t) {
        const float step_scale = elem == ELEM_F16 ? all[t].f16 : 1.0f;
        if (kind == PLAN_BACKWARD && all[t].tile != TILE_128 && all[t].tile != TILE_64) continue;
        if (gated && (all[t].tile == TILE_128_DEEP || all[t].tile == TILE_64_DEEP)) continue;          // built for plain products
        if (!fits_a_launch(p, n, all[t].tile, kind)) continue;
        const int64_t slots = (int64_t)kCus * all[t].per_cu;
        int64_t tiles[2] = {tiles_of(p[0], all[t].tile), n > 1 ? tiles_of(p[1], all[t].tile) : 0};
        // slices as long as they are four steps or more and the chip has room for them
        auto may = [&](int i, int s) { return s == 1 || (kind == PLAN_FORWARD && p[i].steps >= 4 * s && tiles[i] * s <= 2 * slots); };
        for (int s0 : kSlices) {
            if (!may(0, s0)) break;
            for (int s1 : kSlices) {
                if (n > 1 ? !may(1, s1) : s1 > 1) break;
                Product q[2] = {p[0], n > 1 ? p[1] : p[0]};
                cut(q[0], s0);
                if (n > 1) cut(q[1], s1);
                const double c = cost_of(q, tiles, n, all[t], step_scale, kind == PLAN_BACKWARD ? 3.0f : 1.0f);
                if (c < least) {
                    least = c;
                    best = all[t].tile;
                    cut_best[0] = q[0];
                    cut_best[1] = q[1];
                }
            }
        }
    }
    for (int i = 0; i < n; ++i) p[i] = cut_best[i];
    return best;
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
    Product fwd;
    int tile;
    size_t copy_a, copy_b, split, bytes;
};

// Bytes from row to row of a copy of rows of `bytes`: whole cache lines but for short rows.  (The gradient products of 3985 x 770 x 771, whose steps
// of 64 or 128 bytes straddled two lines, took 53 us instead of 41.)
static int64_t pitch(int64_t bytes) { return bytes < 512 ? bytes : up_to(bytes, 128); }

static void lay_out(DensePlan& d, int64_t N, int64_t K, const lba_infmt& fa, const lba_infmt& fb, bool gated, bool aligned) {
    d.elem = elem_of(fa, fb);
    d.cols = gated ? 2 * N : N;
    d.in_place = d.elem != ELEM_BF16 && K % 16 == 0 && aligned;
    const int64_t bytes = d.elem != ELEM_BF16 ? up_to(K, 16) : 2 * up_to(K, 8);
    d.ld = d.in_place ? K : pitch(bytes);
    d.chunks = bytes / 16;
    d.steps = (bytes + 127) / 128;
}

static DensePlan plan_forward(int64_t M, int64_t N, int64_t K, const lba_infmt& fa, const lba_infmt& fb, bool gated, bool aligned) {
    DensePlan d = {};
    lay_out(d, N, K, fa, fb, gated, aligned);
    d.token = M <= kTokenRows;
    if (d.token) return d;                               // reads its operands where they are
    size_t at = 0;
    if (!d.in_place) {
        d.copy_a = at; at += align256((size_t)(M * d.ld));
        d.copy_b = at; at += align256((size_t)(d.cols * d.ld));
    }
    d.fwd = {M, d.cols, d.steps, 1, d.steps};
    d.tile = plan_tile(&d.fwd, 1, d.elem, PLAN_FORWARD, gated);
    d.split = at; at += split_bytes(d.fwd);
    d.bytes = at;
    return d;
}

struct BwdPlan {
    DensePlan f;             // the sums computed again
    bool sums;               // whether they are
    int pieces;
    int64_t np, mp;          // columns of the gradient matrix and of its transpose, with the zeros up to multiples of 8
    int64_t ldp, ldt;        // elements from row to row of them
    Product out[2];          // dA and dB, in one launch
    int tile;
    int64_t part_rows;
    size_t p, pt, at, bt, part, split_a, split_b, bytes;
};

static BwdPlan plan_backward(int64_t M, int64_t N, int64_t K, const lba_infmt& fa, const lba_infmt& fb, bool gated, int act, int g_type, bool aligned) {
    BwdPlan b = {};
    b.sums = act != LBA_ACT_NONE || gated;
    DensePlan& f = b.f;
    lay_out(f, N, K, fa, fb, gated, aligned);            // the sums again, always by the tile: few rows as well
    f.fwd = {M, f.cols, b.sums ? f.steps : 0, 1, 0};
    f.tile = plan_tile(&f.fwd, 1, f.elem, PLAN_BACKWARD, gated);
    size_t at = 0;
    if (b.sums && !f.in_place) {
        f.copy_a = at; at += align256((size_t)(M * f.ld));
        f.copy_b = at; at += align256((size_t)(f.cols * f.ld));
    }
    b.pieces = g_type == LBA_F32 ? 3 : 1;
    b.np = (gated ? 2 : 1) * up_to(N, 8);
    b.mp = up_to(M, 8);
    b.ldp = pitch(b.np * 2) / 2;
    b.ldt = pitch(b.mp * 2) / 2;
    b.p = at; at += align256((size_t)(b.pieces * M * b.ldp) * 2);
    b.pt = at; at += align256((size_t)(b.pieces * f.cols * b.ldt) * 2);
    b.at = at; at += align256((size_t)(K * b.ldt) * 2);
    b.bt = at; at += align256((size_t)(K * b.ldp) * 2);
    const TileShape s = tile_shape(f.tile);
    b.part_rows = (M + s.bm - 1) / s.bm * s.wm;
    b.part = at; at += align256((size_t)(b.part_rows * f.cols) * 4);
    const int64_t step = b.pieces == 3 ? 64 : 128;
    b.out[0] = {M, K, (b.np * 2 + step - 1) / step, 1, 0};
    b.out[1] = {f.cols, K, (b.mp * 2 + step - 1) / step, 1, 0};
    b.tile = plan_tile(b.out, 2, ELEM_BF16, PLAN_FORWARD, false, b.pieces);
    b.split_a = at; at += split_bytes(b.out[0]);
    b.split_b = at; at += split_bytes(b.out[1]);
    b.bytes = at;
    return b;
}

static void add_job(LayJobs& jobs, uint32_t& blocks, const uint8_t* src, void* dst, int64_t R, int64_t K, int64_t ld, int kind, const lba_infmt& f) {
    if (R == 0 || K == 0) return;
    LayJob& j = jobs.job[jobs.n++];
    j.src = src; j.dst = (uint8_t*)dst; j.R = R; j.ld = ld; j.K = (int32_t)K; j.kind = kind; j.first = blocks; j.bits = make_code_bits(f);
    j.wide = (int32_t)up_to(R, 8);
    j.tiles_k = (int32_t)((K + kLayK - 1) / kLayK);
    blocks += (uint32_t)(kind == LAY_TRANSPOSED ? j.tiles_k * ((R + 63) / 64) : (R * (ld / 16) + 255) / 256);
}
// a job's workgroups take 2048 codes or more: five jobs stay under 2^32 lanes
static bool lay_fits(int64_t R, int64_t K) { return (R + 64) * (K + 64) <= ((int64_t)1 << 32); }

// one product, or two that share a launch
static int run_products(GemmParams* g, const Product* p, int n, const Beside* side, int tile, int elem, bool gated, int epi, hipStream_t st) {
    JoinPair join = {};
    int sliced = 0;
    for (int i = 0; i < n; ++i) {
        g[i].slices = p[i].slices;
        g[i].per_slice = (int32_t)p[i].per_slice;
        if (p[i].slices > 1) join.p[sliced++] = {g[i].e, g[i].split, p[i].slices, g[i].rows_b};
    }
    const int x = n > 1 && p[1].per_slice > p[0].per_slice ? 1 : 0;                  // the longer workgroups first
    const GemmParams* second = n > 1 ? &g[1 - x] : nullptr;
    int rc;
    if (elem == ELEM_E4M3) rc = launch_dense_e4m3(g[x], second, side, tile, gated, epi, st);
    else if (elem == ELEM_F16) rc = launch_dense_f16(g[x], second, side, tile, gated, epi, st);
    else rc = launch_dense_bf16(g[x], second, side, tile, gated, epi, st);
    if (rc != LBA_OK || !sliced) return rc;
    join.blocks = join_blocks(join.p[0].e);
    const dim3 grid((unsigned)(join.blocks + (sliced > 1 ? join_blocks(join.p[1].e) : 0)));
    if (gated) hipLaunchKernelGGL(dense_join_kernel<true>, grid, dim3(256), 0, st, join);
    else hipLaunchKernelGGL(dense_join_kernel<false>, grid, dim3(256), 0, st, join);
    return LBA_OK;
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
    if (!d.token && (!fits_a_launch(&d.fwd, 1, d.tile, PLAN_FORWARD) || (!d.in_place && (!lay_fits(M, K) || !lay_fits(d.cols, K))))) return LBA_ERR_SHAPE;
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
        LayJobs jobs = {};
        uint32_t blocks = 0;
        const int kind = d.elem == ELEM_BF16 ? LAY_BF16 : LAY_CODES;
        add_job(jobs, blocks, A, ws + d.copy_a, M, K, d.ld, kind, fmt_a);
        add_job(jobs, blocks, B, ws + d.copy_b, d.cols, K, d.ld, kind, fmt_b);
        if (jobs.n) hipLaunchKernelGGL(dense_lay_kernel, dim3(blocks), dim3(256), 0, st, jobs);
        g.A = ws + d.copy_a; g.B = ws + d.copy_b;
    }
    g.rows_a = (int32_t)M; g.rows_b = (int32_t)d.cols; g.half = (int32_t)N;
    g.chunks = (int32_t)d.chunks; g.steps = (int32_t)d.steps;
    g.shift_a = ea.shift; g.shift_b = eb.shift; g.keep_a = ea.keep; g.keep_b = eb.keep;
    g.e = e;
    g.split = (float*)(ws + d.split);
    rc = run_products(&g, &d.fwd, 1, nullptr, d.tile, d.elem, two, EPI_FORWARD, st);
    if (rc != LBA_OK) return rc;
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
    const hipStream_t st = (hipStream_t)hip_stream;
    const bool two = gated != 0;
    const int64_t cols = two ? 2 * N : N, size = g_type == LBA_F32 ? 4 : 2;
    const bool nothing = !dA && !dB && !dbias;           // which asks for nothing only where none of them has elements
    if (nothing && (K == 0 || M == 0 || N == 0)) return LBA_OK;
    if (nothing) return LBA_ERR_NULL;
    if (M == 0 || N == 0) {                              // sums of nothing
        if (dA) launch_zero(dA, M * K * size, st);
        if (dB) launch_zero(dB, cols * K * size, st);
        if (dbias) launch_zero(dbias, cols * 4, st);
        return hipGetLastError() == hipSuccess ? LBA_OK : LBA_ERR_LAUNCH;
    }
    const BwdPlan b = plan_backward(M, N, K, fmt_a, fmt_b, two, act, g_type, aligned16(A, B));
    if (!G || (K > 0 && (((dA || b.sums) && !B) || ((dB || b.sums) && !A)))) return LBA_ERR_NULL;
    if (!fits_a_launch(&b.f.fwd, 1, b.f.tile, PLAN_BACKWARD) || !fits_a_launch(b.out, 2, b.tile, PLAN_FORWARD) || !lay_fits(M, K) || !lay_fits(cols, K)) return LBA_ERR_SHAPE;
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
    const int32_t wide = (int32_t)up_to(N, 8);
    Beside side = {};
    if (b.sums && !b.f.in_place) {                       // what the sums read, before them
        LayJobs jobs = {};
        uint32_t blocks = 0;
        const int kind = b.f.elem == ELEM_BF16 ? LAY_BF16 : LAY_CODES;
        add_job(jobs, blocks, A, ws + b.f.copy_a, M, K, b.f.ld, kind, fmt_a);
        add_job(jobs, blocks, B, ws + b.f.copy_b, cols, K, b.f.ld, kind, fmt_b);
        if (jobs.n) hipLaunchKernelGGL(dense_lay_kernel, dim3(blocks), dim3(256), 0, st, jobs);
        g.A = ws + b.f.copy_a; g.B = ws + b.f.copy_b;
    }
    if (dA) {                                            // what the gradient products read, beside them
        add_job(side.jobs, side.job_blocks, B, ws + b.bt, N, K, b.ldp * 2, LAY_TRANSPOSED, fmt_b);
        if (two) add_job(side.jobs, side.job_blocks, B + N * K, ws + b.bt + wide * 2, N, K, b.ldp * 2, LAY_TRANSPOSED, fmt_b);
    }
    if (dB) add_job(side.jobs, side.job_blocks, A, ws + b.at, M, K, b.ldt * 2, LAY_TRANSPOSED, fmt_a);
    g.rows_a = (int32_t)M; g.rows_b = (int32_t)cols; g.half = (int32_t)N;
    g.chunks = b.sums ? (int32_t)b.f.chunks : 0; g.steps = b.sums ? (int32_t)b.f.steps : 0;
    g.shift_a = ea.shift; g.shift_b = eb.shift; g.keep_a = ea.keep; g.keep_b = eb.keep;
    g.e = e;
    rc = run_products(&g, &b.f.fwd, 1, &side, b.f.tile, b.f.elem, two, EPI_BACKWARD, st);
    if (rc != LBA_OK) return rc;

    // the two products of it, and dbias beside them
    if (K == 0 || (!dA && !dB)) {
        if (dbias) launch_column_sum(e.part, b.part_rows, cols, dbias, nullptr, cols, st);
        return hipGetLastError() == hipSuccess ? LBA_OK : LBA_ERR_LAUNCH;
    }
    if (dbias) side.sums = {e.part, dbias, (int32_t)b.part_rows, (int32_t)cols};
    GemmParams q[2] = {};
    Product parts[2];
    int n = 0;
    if (dA) {
        GemmParams& a = q[n];
        a.A = (const uint8_t*)P; a.B = ws + b.bt; a.lda = a.ldb = b.ldp * 2; a.a_piece = e.p_piece * 2;
        a.rows_a = (int32_t)M; a.chunks = (int32_t)(b.np / 8); a.split = (float*)(ws + b.split_a);
        a.e.scale = make_elem(fmt_b, ELEM_BF16).factor; a.e.M = (int32_t)M; a.e.Y = dA;
        parts[n++] = b.out[0];
    }
    if (dB) {
        GemmParams& a = q[n];
        a.A = (const uint8_t*)PT; a.B = ws + b.at; a.lda = a.ldb = b.ldt * 2; a.a_piece = e.pt_piece * 2;
        a.rows_a = (int32_t)cols; a.chunks = (int32_t)(b.mp / 8); a.split = (float*)(ws + b.split_b);
        a.e.scale = make_elem(fmt_a, ELEM_BF16).factor; a.e.M = (int32_t)cols; a.e.Y = dB;
        parts[n++] = b.out[1];
    }
    for (int i = 0; i < n; ++i) {
        q[i].rows_b = q[i].half = (int32_t)K;
        q[i].steps = (int32_t)parts[i].steps;
        q[i].e.N = (int32_t)K; q[i].e.y_type = g_type;
    }
    rc = run_products(q, parts, n, &side, b.tile, ELEM_BF16, false, EPI_FORWARD, st);
    if (rc != LBA_OK) return rc;
    return hipGetLastError() == hipSuccess ? LBA_OK : LBA_ERR_LAUNCH;
}

}  // extern "C"
