// Which kernel runs a product of 8-bit integers, and copies of operands whose rows are not
// multiples of 16 bytes.
#include "api_state.h"
#include "emu_internal.h"
#include "moe.h"
#include "moe_common.h"

namespace emu {
namespace {

constexpr int64_t OFFSETS = (int64_t)1 << 32;        // what a copy's 32-bit offset spans
constexpr int64_t MOST_COPIED = (int64_t)1 << 33;    // bytes of workspace for copies
constexpr int64_t MOST_TILES = (int64_t)1 << 28;     // a workgroup of 256 takes 32: fewer than 2^32 threads

bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
int64_t up(int64_t n, int64_t unit) { return (n + unit - 1) / unit * unit; }

// A matrix (or one for each expert) of 8-bit integers as the copy has it: rows x ld, ld a
// multiple of 16, zeros behind the entries that exist.
struct Copied {
    const int8_t *src;
    int64_t lds, stride, src_rows;
    int cols;
    const int *map;                 // row r is row map[r] of the source (zeros if it has none); or null
    int mats;
    const int *offsets;             // matrix e is copied if expert e has rows; or null
    int64_t R;                      // of offsets
    int64_t rows, ld;
    int64_t bytes() const { return mats * rows * ld; }
};

// Four times 16 bytes a thread: unaligned loads, aligned stores; `per_x` workgroups for X,
// then `per_w` for each matrix of W.  Bound by bytes.
constexpr int COPY = 4;
__global__ __launch_bounds__(256) void q8_copy_kernel(Copied x, int8_t *__restrict__ to_x, unsigned per_x, Copied w,
                                                      int8_t *__restrict__ to_w, unsigned per_w) {
    const bool is_x = blockIdx.x < per_x;
    const unsigned b = is_x ? blockIdx.x : blockIdx.x - per_x;
    const Copied m = is_x ? x : w;
    const int e = is_x ? 0 : (int)(b / per_w);
    if (m.offsets) {
        int64_t lo, hi;
        expert_rows(m.offsets, m.mats, m.R, e, lo, hi);
        if (lo == hi) return;
    }
    const unsigned i0 = (is_x ? b : b % per_w) * (256 * COPY) + threadIdx.x, per_row = (unsigned)(m.ld / 16);
    int8_t *const dst = (is_x ? to_x : to_w) + e * m.rows * m.ld;
    i32x4 v[COPY];
#pragma unroll
    for (int j = 0; j < COPY; ++j) {
        const unsigned i = i0 + 256 * j;
        const int64_t row = i / per_row;
        const int c = (int)(i % per_row) * 16;
        v[j] = i32x4{};
        if (row >= m.rows) continue;
        const int64_t at = m.map ? m.map[row] : row;
        if (at < 0 || at >= m.src_rows) continue;
        v[j] = load_bytes16(m.src + e * m.stride + at * m.lds, c, m.cols);
    }
#pragma unroll
    for (int j = 0; j < COPY; ++j) {
        const unsigned i = i0 + 256 * j;
        if (i / per_row < m.rows) *reinterpret_cast<i32x4 *>(dst + (int64_t)i * 16) = v[j];
    }
}
hipError_t copy(const Copied &x, char *to_x, const Copied &w, char *to_w, hipStream_t s) {
    auto blocks = [](const Copied &m) { return (unsigned)((m.rows * m.ld / 16 + 256 * COPY - 1) / (256 * COPY)); };
    const unsigned per_x = x.mats * blocks(x), per_w = blocks(w);
    q8_copy_kernel<<<per_x + w.mats * per_w, 256, 0, s>>>(x, reinterpret_cast<int8_t *>(to_x), per_x, w,
                                                         reinterpret_cast<int8_t *>(to_w), per_w);
    return hipGetLastError();
}

// The kernel of q8_tiles.h: rows of whole 16-byte chunks, offsets of 32 bits, and a launch that fits.
bool fits_tiles(const Q8Gemm &g) {
    return g.K > 0 && g.K % 16 == 0 && g.E > 0 && aligned16(g.X) && aligned16(g.W) && g.ldx % 16 == 0 &&
           g.ldw % 16 == 0 && g.sw % 16 == 0 && (g.rows ? g.xrows : 256) * g.ldx < OFFSETS && 256 * g.ldw < OFFSETS &&
           (!g.rows || g.xrows > 0) && row_blocks_bound(g.R, g.E, 128) * ((g.N + 127) / 128) <= MOST_TILES;
}

// Times, us, that the choice between the two kernels goes by.  Measured, that for few rows
// and that of tiles: 16 rows of 8192 x 8192 20 and 30; 64 rows of 4096 x 4096 14 and 18, 128 rows
// 17 and 19; 100 rows of 8192 x 4096 22 and 18, 300 rows 57 and 21; 64 experts of 2048 x 2048,
// 8 rows 10 and 16, 32 rows 25 and 19, 128 rows 47 and 38, 4096 rows 144 and 50; 13 of 1501 x 777,
// 100 rows 10 and 24 (with the copies); 64 of 1280 x 1081, 854 rows 67 and 50.
int64_t tiles_of(const Q8Gemm &g, int64_t t) { return row_blocks_expected(g.R, g.E, t) * ((g.N + t - 1) / t); }
// The kernel for few rows: its waves read X and W at 7 to 8 TB/s, the matrices come at 6 TB/s,
// a workgroup takes 1024 indices in 0.7 to 2.5 us, by its loads, and 6 us beside; rows that are
// not whole words take half as much again.
double time_of_few(const Q8Gemm &g, int splits = 1) {
    const Q8FewShape f = q8_few_shape(g);
    const double cus = (double)device_cu_count(), loads = f.mt + f.nt, more = f.words ? 1 : 1.5;
    const double rounds = (double)(up(g.K, Q8_FEW_ROUND * splits) / (Q8_FEW_ROUND * splits));
    double t = ceil(f.tiles * splits / (f.per_cu * cus)) * (6 + (0.1 + 0.3 * loads) * rounds * more) - 6;
    t = fmax(t, f.tiles * g.K * 16 * loads * more / (g.E > 1 ? 7e6 : 8e6));
    t = fmax(t, experts_reached(g.R, g.E) * g.N * g.K * more / 6e6);
    return (g.E > 1 ? 8 : 5) + t;
}
// Tiles of 128 take 0.45 us for a k-block (copies to LDS at 64 bytes a cycle and the reads of
// fragments), all of them the matrices' bytes at 6 TB/s.
double time_of_tiles(const Q8Gemm &g, int splits = 1) {
    const int64_t cus = device_cu_count(), blocks = ((g.K + 127) / 128 + splits - 1) / splits;
    const double copies =
        (g.E > 1 || splits > 1 ? 8 : 4) + (double)((tiles_of(g, 128) * splits + cus - 1) / cus) * blocks * 0.45;
    const double bytes = 1 + experts_reached(g.R, g.E) * g.N * g.K / 6e6;
    return copies > bytes ? copies : bytes;
}
// Sums of splits of a long reduction: written, read and joined at 4.5 TB/s by a kernel of
// its own, one launch more.
double time_of_join(const Q8Gemm &g, int splits) { return 7 + (double)g.R * g.N * 8 * splits / 4.5e6; }

// Y from the sums of the splits (R x ld each): one matrix, four columns to a thread.
template <typename T>
__global__ __launch_bounds__(256) void q8_join_kernel(Q8Gemm g, const int *__restrict__ sums, int64_t ld,
                                                      int splits) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, per_row = ld / 4, r = i / per_row;
    const int c = (int)(i - r * per_row) * 4;
    if (r >= g.R) return;
    int64_t lo, hi;
    expert_rows(g.offsets, 1, g.R, 0, lo, hi);
    const int64_t at = g.rows ? g.rows[r] : r;
    const bool there = r < hi && at >= 0 && at < g.xrows;
    i32x4 sum = {};
    for (int k = 0; k < splits; ++k) sum += *reinterpret_cast<const i32x4 *>(sums + (k * g.R + r) * ld + c);
    const float x = there ? g.xs[at] : 0.0f;
    T *const y = static_cast<T *>(g.Y) + r * g.ldy + c;
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (c + j < g.N) y[j] = there ? (T)q8_result(sum[j], g.ws[c + j], x) : (T)0.0f;
}

// Times, us, of rounds of one tile of 256 on a CU, of two of 128 (or of one, where half the
// places stay empty), and of one of 128 in four stages: those of its k-blocks, and of its
// start and its stores.  Measured: 8192 x 8192 x 8192 449, 521 and 603 us; 2048 x 4096 x 4096
// 52, 40 and 43; 300 rows of 8192 x 4096 49, 27 and 21; 4999 over 13 experts of 1501 x 784 in
// float32 35, 28 and 30; 200 over 8 of 2048 x 1024 SMALL 9, DEEP 12.
hipError_t run_tiles_kernel(const Q8Gemm &g, hipStream_t s) {
    const int64_t cus = device_cu_count(), small = tiles_of(g, 128), rest = small % (2 * cus);
    const double blocks = (double)((g.K + 127) / 128);
    auto rounds = [&](int64_t tiles) { return (double)((tiles + cus - 1) / cus); };
    const double large = rounds(tiles_of(g, 256)) * (blocks * 1.65 + (g.dtype == EMU_F32 ? 18 : 10));
    const double two = blocks * 0.96 + 6, one = blocks * 0.7 + 4;
    const double pairs = (double)(small / (2 * cus)) * two + (rest > cus ? two : (rest > 0 ? one : 0));
    const double deep = rounds(small) * (blocks * 0.45 + 8);
    const Q8Tiles how = large <= pairs && large <= deep ? Q8Tiles::LARGE
                                                        : (pairs <= deep ? Q8Tiles::SMALL : Q8Tiles::DEEP);
    if (g.dtype == EMU_F32) return launch_q8_tiles_f32(g, how, s);
    return g.dtype == EMU_BF16 ? launch_q8_tiles_bf16(g, how, s) : launch_q8_tiles_f16(g, how, s);
}

}  // namespace

// A product of one matrix whose reduction is split, if that is faster than `time` us: *done,
// or else nothing was launched.
// 294 rows of 2176 x 8128: 33 us in one piece, 23 in four; 512 of 4096 x 16384 59 and, in two,
// 49; 39 of 64 x 6656 16 and, in four, 11; 16 of 2048 x 16384 17 and, in 16, 23.
static int split_gemm(const Q8Gemm &g, double time, hipStream_t s, bool *done) {
    *done = false;
    if (g.E != 1 || g.K < 1024) return EMU_OK;
    const bool fits = fits_tiles(g), narrow = q8_few_shape(g).nt == 1;
    int splits = 1;
    bool few = true;
    for (int n = 2; n <= 16; n *= 2) {
        const double join = time_of_join(g, n);
        if (narrow && g.K >= 1024 * n && time_of_few(g, n) + join < time) {
            time = time_of_few(g, n) + join;
            splits = n;
            few = true;
        }
        if (fits && g.K >= 512 * n && time_of_tiles(g, n) + join < time) {
            time = time_of_tiles(g, n) + join;
            splits = n;
            few = false;
        }
    }
    if (splits == 1) return EMU_OK;
    const int64_t ld = up(g.N, 4), bytes = splits * g.R * ld * 4;
    if (bytes > MOST_COPIED) return EMU_OK;
    char *at = nullptr;
    if (int rc = api_try_workspace(bytes, &at)) return rc;
    if (!at) return EMU_OK;
    *done = true;
    Q8Gemm d = g;
    d.Y = at;
    d.ldy = ld;
    d.part = (int)up((g.K + splits - 1) / splits, 128);
    const int n = (g.K + d.part - 1) / d.part;
    hipError_t e = few ? launch_q8_few_sums(d, n, s) : launch_q8_tiles_sums(d, n, s);
    if (e == hipSuccess)
        with_type(g.dtype, [&](auto z) {
            q8_join_kernel<decltype(z)><<<(unsigned)((g.R * (ld / 4) + 255) / 256), 256, 0, s>>>(
                g, reinterpret_cast<const int *>(at), ld, n);
        });
    return api_done(e == hipSuccess ? hipGetLastError() : e, "q8_gemm");
}

// The product on copies of the operands that the kernel of q8_tiles.h cannot take: d, with the
// copies to be made (to workspace that d does not have yet).
struct OnCopies {
    Copied x, w;
    Q8Gemm d;
    bool possible;
    int64_t xb() const { return up(x.bytes(), 256); }
    int64_t bytes() const { return xb() + w.bytes(); }
    double time() const { return 4 + bytes() * 2 / 6e6 + time_of_tiles(d); }
};
static OnCopies on_copies(const Q8Gemm &g) {
    OnCopies c = {};
    // the rows of X through their numbers into the copy, where those are fewer
    const int *const map = g.rows && g.xrows > g.R ? g.rows : nullptr;
    const int64_t K = up(g.K, 16), xr = g.rows && !map ? g.xrows : g.R;
    const bool pad = K != g.K, x = pad || !aligned16(g.X) || g.ldx % 16 || (map && g.xrows * g.ldx >= OFFSETS);
    const bool w = pad || !aligned16(g.W) || g.ldw % 16 || g.sw % 16;
    const int mats = g.sw == 0 ? 1 : g.E;                       // one matrix for all experts
    c.x = {g.X, g.ldx, 0, g.xrows, g.K, map, x ? 1 : 0, nullptr, 0, xr, K};
    c.w = {g.W, g.ldw, g.sw, g.N, g.K, nullptr, w ? mats : 0, g.sw == 0 ? nullptr : g.offsets, g.R, g.N, K};
    c.d = g;
    c.d.K = (int)K;
    if (x) {
        c.d.X = nullptr;
        c.d.ldx = K;
        if (map) c.d.rows = nullptr;
    }
    if (w) {
        c.d.W = nullptr;
        c.d.ldw = K;
        c.d.sw = g.sw == 0 ? 0 : c.w.rows * K;
    }
    c.possible = fits_tiles(c.d) && c.bytes() <= MOST_COPIED;
    return c;
}

int launch_q8_gemm(const Q8Gemm &g, hipStream_t s) {
    // the sums of rows without entries, or without any row to read, are zeros
    if (g.K == 0 || g.E == 0 || g.xrows == 0) return api_done(launch_q8_few(g, s), "q8_gemm");
    const bool fits = fits_tiles(g);
    OnCopies c = {};
    if (!fits) c = on_copies(g);
    const double few = time_of_few(g), tiles = fits ? time_of_tiles(g) : (c.possible ? c.time() : few);
    bool done;
    if (int rc = split_gemm(g, few < tiles ? few : tiles, s, &done)) return rc;
    if (done) return EMU_OK;
    if (fits && tiles < few) return api_done(run_tiles_kernel(g, s), "q8_gemm");
    char *at = nullptr;
    if (!fits && tiles < few)
        if (int rc = api_try_workspace(c.bytes(), &at)) return rc;
    if (!at) return api_done(launch_q8_few(g, s), "q8_gemm");
    if (c.x.mats > 0) c.d.X = reinterpret_cast<int8_t *>(at);
    if (c.w.mats > 0) c.d.W = reinterpret_cast<int8_t *>(at + c.xb());
    hipError_t e = copy(c.x, at, c.w, at + c.xb(), s);
    if (e == hipSuccess) e = run_tiles_kernel(c.d, s);
    return api_done(e, "q8_gemm");
}

}  // namespace emu
