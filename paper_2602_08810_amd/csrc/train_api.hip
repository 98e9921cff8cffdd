// C ABI of the short causal convolution, the loss over a vocabulary, and the norm and clipping of gradients: argument checks, layout of workspaces, launches.
// Nothing here allocates, frees or synchronises; see include/lrnnx.h for the contract.
#include "../../include/lrnnx.h"
#include "conv.hpp"
#include "grad_clip.hpp"
#include "vocab_loss.hpp"

#include <cstdlib>
#include <initializer_list>

using namespace lrnnx;

namespace {

inline int64_t up(int64_t x, int64_t m) { return (x + m - 1) / m * m; }
inline bool on(const void *p, size_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }
inline size_t elem(int dtype) { return dtype == LRNNX_BF16 ? 2 : 4; }
inline bool io_type(int dtype) { return dtype == LRNNX_F32 || dtype == LRNNX_BF16; }
inline int status(hipError_t e) { return e == hipSuccess ? LRNNX_OK : LRNNX_ERR_LAUNCH; }

// Memory of a tensor: up to two axes of rows, steps and row in bytes.
struct Area {
    const char *p = nullptr;
    int64_t row = 0, n[2] = {1, 1}, step[2] = {0, 0};
    Area(const void *p, int64_t row, int64_t n0 = 1, int64_t step0 = 0, int64_t n1 = 1, int64_t step1 = 0) : p(static_cast<const char *>(p)), row(row) {
        const bool turned = n1 > 1 && (n0 <= 1 || std::abs(step1) < std::abs(step0));          // the axis of smaller steps first
        n[0] = turned ? n1 : n0; step[0] = turned ? step1 : step0;
        n[1] = turned ? n0 : n1; step[1] = turned ? step0 : step1;
        for (int k = 0; k < 2; ++k) if (n[k] <= 1) { n[k] = 1; step[k] = 0; }
    }
    int64_t low() const { return (step[0] < 0 ? step[0] * (n[0] - 1) : 0) + (step[1] < 0 ? step[1] * (n[1] - 1) : 0); }
    int64_t high() const { return (step[0] > 0 ? step[0] * (n[0] - 1) : 0) + (step[1] > 0 ? step[1] * (n[1] - 1) : 0) + row; }
};
// Whether two tensors share an element.  Exact for views of the same shape and steps whose rows do not overlap themselves (parts of the channels of a wider tensor); of others it is
// enough that their extents do.
bool meet(const Area &a, const Area &b) {
    if (!a.p || !b.p) return false;
    const int64_t apart = (int64_t)(reinterpret_cast<uintptr_t>(b.p) - reinterpret_cast<uintptr_t>(a.p));
    if (a.high() <= apart + b.low() || apart + b.high() <= a.low()) return false;
    int64_t span = a.row;
    bool same = a.row == b.row;
    for (int k = 0; k < 2; ++k) {
        same = same && a.n[k] == b.n[k] && a.step[k] == b.step[k] && (a.n[k] == 1 || a.step[k] >= span);
        span += a.step[k] * (a.n[k] - 1);
    }
    if (!same) return true;
    // rows i of a and j of b lie `apart` + step (j - i) apart: below a row's length for one of the two differences next to it of either axis, or for none
    const auto near = [](int64_t d, int64_t step, int k) { return step ? (d >= 0 ? d / step : -((-d + step - 1) / step)) + k : 0; };
    for (int i = 0; i < 2; ++i) {
        const int64_t c1 = near(apart, a.step[1], i);
        if (std::abs(c1) >= a.n[1]) continue;
        const int64_t left = apart - c1 * a.step[1];
        for (int j = 0; j < 2; ++j) {
            const int64_t c0 = near(left, a.step[0], j);
            if (std::abs(c0) < a.n[0] && std::abs(left - c0 * a.step[0]) < a.row) return true;
        }
    }
    return false;
}
bool meet(const Area &a, std::initializer_list<Area> others) {
    for (const Area &b : others) if (meet(a, b)) return true;
    return false;
}

// ---------------------------------------------------------------- short causal convolution
template <class A> int conv_checks(const A *a) {
    if (a->B < 1 || a->D < 1 || a->L < 1 || a->W < 1 || a->act < 0 || a->act > 1 || a->time_last < 0 || a->time_last > 1 || !io_type(a->io_dtype)) return LRNNX_ERR_INVALID_ARG;
    if (a->W < 2 || a->W > 4 || a->D > 65536 || a->B > 65535) return LRNNX_ERR_UNSUPPORTED;
    // elements stay countable in tiles of four steps, which are counted in 32 bits
    if (a->L > ((int64_t)1 << 32) / (a->cu_seqlens ? 1 : a->B)) return LRNNX_ERR_UNSUPPORTED;
    return LRNNX_OK;
}
template <class A> bool conv_inputs(const A *a) {
    const size_t es = elem(a->io_dtype);
    return a->x && a->weight && on(a->x, es) && on(a->weight, 4) && on(a->bias, 4) && on(a->x0, es) && on(a->cu_seqlens, 8);
}
template <class A> ConvParams conv_params(const A *a, bool backward) {
    ConvParams p{};
    p.seqs = a->B; p.B = a->cu_seqlens ? 1 : a->B; p.D = a->D; p.W = a->W; p.L = a->L;
    p.io = a->io_dtype == LRNNX_BF16; p.act = a->act; p.time_last = a->time_last; p.cu = a->cu_seqlens;
    p.x = a->x; p.x_b = a->x_stride_b;
    p.x_l = a->time_last ? 1 : a->x_stride_s; p.x_d = a->time_last ? a->x_stride_s : 1;
    p.w = a->weight; p.bias = a->bias; p.x0 = a->x0;
    plan_conv(p, backward);
    return p;
}
// [B,L,D] or [B,D,L] with these strides; [B,W-1,D]; the inputs that both passes have
template <class A> Area conv_rows(const A *a, const void *p, int64_t sb, int64_t ss) {
    const int64_t es = elem(a->io_dtype);
    return Area(p, (a->time_last ? a->L : a->D) * es, a->time_last ? a->D : a->L, ss * es, a->cu_seqlens ? 1 : a->B, sb * es);
}
template <class A> Area conv_state(const A *a, const void *p) { return Area(p, (int64_t)a->B * (a->W - 1) * a->D * (int64_t)elem(a->io_dtype)); }
template <class A> bool over_inputs(const A *a, const Area &out) {
    return meet(out, {conv_rows(a, a->x, a->x_stride_b, a->x_stride_s), Area(a->weight, (int64_t)a->D * a->W * 4), Area(a->bias, (int64_t)a->D * 4), conv_state(a, a->x0), Area(a->cu_seqlens, ((int64_t)a->B + 1) * 8)});
}
size_t conv_sums_bytes(const ConvParams &p) { return (size_t)p.blocks * (p.W + 1) * p.D * sizeof(float); }

}  // namespace

extern "C" {

int lrnnx_short_conv_fwd(const lrnnx_conv_fwd_args *a) {
    if (!a || a->struct_size != sizeof(lrnnx_conv_fwd_args)) return LRNNX_ERR_INVALID_ARG;
    if (const int e = conv_checks(a)) return e;
    const size_t es = elem(a->io_dtype);
    if (!conv_inputs(a) || !a->y || !on(a->y, es) || !on(a->x_last, es)) return LRNNX_ERR_INVALID_ARG;
    const Area y = conv_rows(a, a->y, a->y_stride_b, a->y_stride_s), last = conv_state(a, a->x_last);
    if (over_inputs(a, y) || over_inputs(a, last) || meet(y, last)) return LRNNX_ERR_INVALID_ARG;
    ConvParams p = conv_params(a, false);
    p.y = a->y; p.y_b = a->y_stride_b; p.y_l = a->time_last ? 1 : a->y_stride_s; p.y_d = a->time_last ? a->y_stride_s : 1;
    p.x_last = a->x_last;
    const hipStream_t s = reinterpret_cast<hipStream_t>(a->stream);
    return status(a->time_last ? launch_conv_time(p, false, s) : launch_conv_rows(p, false, s));
}

size_t lrnnx_short_conv_bwd_workspace_bytes(const lrnnx_conv_bwd_args *a) {
    if (!a || a->struct_size != sizeof(lrnnx_conv_bwd_args) || conv_checks(a) != LRNNX_OK) return 0;
    return conv_sums_bytes(conv_params(a, true));
}

int lrnnx_short_conv_bwd(const lrnnx_conv_bwd_args *a) {
    if (!a || a->struct_size != sizeof(lrnnx_conv_bwd_args)) return LRNNX_ERR_INVALID_ARG;
    if (const int e = conv_checks(a)) return e;
    const size_t es = elem(a->io_dtype);
    if (!conv_inputs(a) || !a->dy || !a->dx || !a->dweight || (a->dbias && !a->bias)) return LRNNX_ERR_INVALID_ARG;
    if (!on(a->dy, es) || !on(a->dx, es) || !on(a->dx_last, es) || !on(a->dx0, es) || !on(a->dweight, 4) || !on(a->dbias, 4) || !on(a->workspace, 16)) return LRNNX_ERR_INVALID_ARG;
    ConvParams p = conv_params(a, true);
    if (!a->workspace || a->workspace_bytes < conv_sums_bytes(p)) return LRNNX_ERR_WORKSPACE;
    const Area dx = conv_rows(a, a->dx, a->dx_stride_b, a->dx_stride_s), dx0 = conv_state(a, a->dx0), dw(a->dweight, (int64_t)a->D * a->W * 4), db(a->dbias, (int64_t)a->D * 4);
    const Area dy = conv_rows(a, a->dy, a->dy_stride_b, a->dy_stride_s), dx_last = conv_state(a, a->dx_last);
    for (const Area &out : {dx, dx0, dw, db}) if (over_inputs(a, out) || meet(out, {dy, dx_last})) return LRNNX_ERR_INVALID_ARG;
    if (meet(dx, {dx0, dw, db}) || meet(dx0, {dw, db}) || meet(dw, db)) return LRNNX_ERR_INVALID_ARG;
    p.dy = a->dy; p.dy_b = a->dy_stride_b; p.dy_l = a->time_last ? 1 : a->dy_stride_s; p.dy_d = a->time_last ? a->dy_stride_s : 1;
    p.dx = a->dx; p.y_b = a->dx_stride_b; p.y_l = a->time_last ? 1 : a->dx_stride_s; p.y_d = a->time_last ? a->dx_stride_s : 1;
    p.dx_last = a->dx_last; p.dx0 = a->dx0; p.dw = a->dweight; p.db = a->dbias;
    p.sums = reinterpret_cast<float *>(a->workspace);
    const hipStream_t s = reinterpret_cast<hipStream_t>(a->stream);
    if ((a->time_last ? launch_conv_time(p, true, s) : launch_conv_rows(p, true, s)) != hipSuccess) return LRNNX_ERR_LAUNCH;
    return status(launch_conv_sums(p, s));
}

int lrnnx_short_conv_step(const lrnnx_conv_step_args *a) {
    if (!a || a->struct_size != sizeof(lrnnx_conv_step_args)) return LRNNX_ERR_INVALID_ARG;
    if (a->B < 1 || a->D < 1 || a->W < 1 || a->act < 0 || a->act > 1 || !io_type(a->io_dtype)) return LRNNX_ERR_INVALID_ARG;
    if (a->W < 2 || a->W > 4 || a->D > 65536 || a->B > 65535) return LRNNX_ERR_UNSUPPORTED;
    const size_t es = elem(a->io_dtype);
    if (!a->x || !a->weight || !a->state || !a->y || !on(a->x, es) || !on(a->state, es) || !on(a->y, es) || !on(a->weight, 4) || !on(a->bias, 4)) return LRNNX_ERR_INVALID_ARG;
    // (y may be x: a thread has read what it writes)
    const int64_t bytes = (int64_t)es;
    const Area x(a->x, bytes, a->D, a->x_stride_d * bytes, a->B, a->x_stride_b * bytes), y(a->y, bytes, a->D, a->y_stride_d * bytes, a->B, a->y_stride_b * bytes);
    const Area state(a->state, bytes * a->B * (a->W - 1) * a->D), w(a->weight, (int64_t)a->D * a->W * 4), bias(a->bias, (int64_t)a->D * 4);
    const bool in_place = a->x == a->y && (a->B == 1 || a->x_stride_b == a->y_stride_b) && (a->D == 1 || a->x_stride_d == a->y_stride_d);
    if (meet(state, {x, y, w, bias}) || meet(y, {w, bias}) || (!in_place && meet(y, x))) return LRNNX_ERR_INVALID_ARG;
    ConvStepParams p{};
    p.B = a->B; p.D = a->D; p.W = a->W; p.io = a->io_dtype == LRNNX_BF16; p.act = a->act;
    p.x = a->x; p.x_b = a->x_stride_b; p.x_d = a->x_stride_d; p.w = a->weight; p.bias = a->bias; p.state = a->state;
    p.y = a->y; p.y_b = a->y_stride_b; p.y_d = a->y_stride_d;
    return status(launch_conv_step(p, reinterpret_cast<hipStream_t>(a->stream)));
}

}  // extern "C"

// ---------------------------------------------------------------- loss over a vocabulary
namespace {

template <class A> int vocab_checks(const A *a) {
    if (a->T < 1 || a->V < 1 || a->K < 1 || !io_type(a->io_dtype)) return LRNNX_ERR_INVALID_ARG;
    if (a->T > (1 << 27) || a->V > (1 << 27) || a->K > (1 << 20)) return LRNNX_ERR_UNSUPPORTED;
    if (((a->V + kVocabTile - 1) / kVocabTile) * ((a->T + kVocabTile - 1) / kVocabTile) > (1 << 30)) return LRNNX_ERR_UNSUPPORTED;     // workgroups of a launch
    return LRNNX_OK;
}
template <class A> bool vocab_inputs(const A *a) {
    const size_t es = elem(a->io_dtype);
    return a->h && a->weight && a->target && on(a->h, es) && on(a->weight, es) && on(a->target, 8);
}
// Rows that the matrix kernels can read as they lie: whole 16-byte pieces at 16-byte steps, 256 of them within 31 bits.
bool rows_in_place(const void *p, int64_t ld, int K, int io) { return io == LRNNX_BF16 && on(p, 16) && K % 8 == 0 && ld % 8 == 0 && ld >= K && ld <= 1 << 21; }
// What is split where it is read, an element a load if need be.
bool wide_in_place(int64_t ld, int K) { return ld >= K && ld <= 1 << 21; }
bool wide_pieces(const void *p, int64_t ld, int K) { return on(p, 16) && K % 4 == 0 && ld % 4 == 0; }

struct Layout {
    char *base;
    size_t at = 0;
    template <class T> T *take(int64_t count) {
        const size_t here = (at + 255) / 256 * 256;
        at = here + (size_t)count * sizeof(T);
        return base ? reinterpret_cast<T *>(base + here) : nullptr;
    }
};

struct VocabPlan {
    VocabParams p;
    VocabPack h, w;                      // copies; src null: read in place
    VocabRows rows;
    int64_t each;                        // words of a piece
    size_t bytes;
};

// Float32 inputs of so few rows: the weight is split where it is read, instead of once, into a copy.  The products then take a fifth longer (168 for 210 TFLOP/s), the copy is 10 bytes an
// element; forward it is for one product, backward for two.  (100 rows, 56617 words, 1472 terms: z, dz and dh 156, 163 and 141 us, from a copy 193, 196 and 171 and twice 140 to make it.  Split, over
// a copy, of 5000 to 150000 words and 332 to 4096 terms: forward, 576 rows 0.70 to 0.96, 768 0.71 to 1.05, 896 0.90 to 1.17; backward, 576 rows 0.87 to 1.03, 704 0.90 to 1.06, 896 0.98 to 1.15.
// Where terms are few the copy is small beside what comes of z: 150000 words of 64 1.06 of 450 rows, 1.11 of 576, 1.24 of 768.)
int64_t vocab_few(int64_t K, bool backward) { return K < 256 ? 512 : backward ? 576 : 768; }
// The vocabulary is taken in as few pieces as lie in 1 GiB of workspace (a piece's dz; of a copied vocabulary its copy): of whole tiles.
constexpr int64_t kVocabRoom = (int64_t)1 << 30;
int64_t piece_of(int64_t words, int64_t bytes_each) {
    int64_t n = bytes_each > 0 ? kVocabRoom / bytes_each / kVocabTile * kVocabTile : words;
    if (n > 1 << 21) n = 1 << 21;
    if (n < kVocabTile) n = kVocabTile;
    return n < words ? n : words;
}

// First side of a product's tiles and the stretches of its terms that are taken side by side (of 512 terms at least; of z, whose parts are larger than what comes of them, of 256, and only where all fit one turn): what takes the least time.  Tiles are
// 256 x 256 or 128 x 128, two a compute unit; of three planes 256 x 128 or 128 x 64, two a compute unit; of a wide factor 128 x 64 or 64 x 64, two.  A whole turn of the smaller
// tiles takes 0.67 of the larger ones' time; 0.6 of three planes; 0.8 of a wide factor.  (z of 997 rows, 5003 words, 771 terms in float32: 73 us with the larger ones, 87 with the smaller;
// of 200 rows, 15179 words, 768 terms 67 and 51; in bfloat16 of 300 rows, 32000 words, 1024 terms 34 and 38, of 100, 32768, 2048 61 and 42.)
int64_t side_n(int planes, int side) { return planes == 1 ? side : side == kVocabTile ? 128 : 64; }
struct VocabShape { int side, splits; };
VocabShape shape_of(int planes, bool wide, int64_t m, int64_t n, int64_t terms, bool z) {
    const int large = wide ? kVocabTile / 2 : kVocabTile, units = wide ? 512 : 256;
    const double part = wide ? 0.8 : planes == 1 ? 0.67 : 0.6;
    VocabShape best{};
    double least = 0;
    for (int side = large; side >= large / 2; side /= 2) {
        const int64_t across = side_n(planes, side), tiles = up(m, side) / side * (up(n, across) / across), at_once = side == large ? units : 512;
        for (int64_t s = 1; s == 1 || (z ? tiles * s <= at_once && s * 256 <= terms : s <= 256 && s * 512 <= terms); ++s) {
            // (of z two more launches, as long as 256 terms, and its parts from memory)
            const double time = (z && s > 1 ? 256 + 1e-4 * (double)(s * m * n) : 0) + (side == large ? 1.0 : part) * vocab_time(tiles, s, at_once, terms);
            if (!best.side || time < least) { least = time; best = {side, (int)s}; }
        }
    }
    return best;
}

// Blocks of words over which the elements of dz are added where they are made: a wavefront's part of a tile, or a thread's eight of z's parts.
int64_t sum_blocks(const VocabParams &p, int64_t words) { return p.splits_z > 1 ? (words + 7) / 8 : up(words, p.side_z) / p.side_z * 2; }

template <class A> VocabPlan plan_vocab(const A *a, char *ws, bool backward) {
    VocabPlan f{};
    const int io = a->io_dtype == LRNNX_BF16, planes = io ? 1 : 3;
    // rows of a copy start on 128 bytes, and not all in the same channel of memory
    const int64_t Kp = up(a->K, 8), ldd = up(a->K, 64) + 64;
    Layout l{ws};
    VocabParams &p = f.p;
    p.T = a->T; p.K = a->K; p.Kp = Kp; p.planes = planes; p.io = io; p.words = a->V; p.target = a->target;
    p.wide = !io && a->T <= vocab_few(a->K, backward);
    auto copy = [&](VocabPack &k, VocabFactor &to, const void *src, int64_t ld, int64_t rows, int planes, bool must) {
        if (!must) { to = {reinterpret_cast<const uint16_t *>(src), 0, ld}; return; }
        k.src = src; k.ld = ld; k.rows = rows; k.ldd = ldd; k.plane = rows * ldd; k.K = a->K; k.Kp = (int)Kp; k.io = io; k.planes = planes;
        k.dst = l.take<uint16_t>((planes ? planes : 2) * k.plane);
        to = {k.dst, k.plane, ldd};
    };
    const bool copied = !(p.wide ? wide_in_place(a->weight_stride, a->K) : rows_in_place(a->weight, a->weight_stride, a->K, a->io_dtype));
    p.any = p.wide && !copied && !wide_pieces(a->weight, a->weight_stride, a->K);
    int64_t each = piece_of(a->V, copied ? (p.wide ? 2 : planes) * ldd * 2 : 0);
    if (backward) {
        const int64_t of_dz = piece_of(a->V, planes * a->T * 2);
        each = of_dz < each ? of_dz : each;
    }
    f.each = p.each = each;
    p.ldz = up(each, 8);
    copy(f.h, p.h, a->h, a->h_stride, a->T, planes, backward || !rows_in_place(a->h, a->h_stride, a->K, a->io_dtype));
    copy(f.w, p.w, a->weight, a->weight_stride, each, p.wide ? 0 : planes, copied);
    const VocabShape z = shape_of(planes, p.wide, each, a->T, a->K, true);
    p.side_z = z.side; p.splits_z = z.splits;
    if (z.splits > 1) p.z_part = l.take<float>(z.splits * a->T * p.ldz);
    if (!backward) {
        p.parts = p.splits_z > 1 ? (a->V + each - 1) / each : up(a->V, p.side_z) / p.side_z;
        p.part = l.take<float>(2 * p.parts * a->T);
        p.hit = l.take<float>(a->T);
    } else {
        const VocabShape dh = shape_of(planes, p.wide, a->K, a->T, each, false), dw = shape_of(planes, false, a->K, each, a->T, false);
        p.side_h = dh.side; p.splits = dh.splits;
        p.side_w = dw.side; p.splits_w = dw.splits;
        // whole tiles, and rows that do not all start in the same channel of memory
        p.dz.ld = up(each, kVocabTile) + 128; p.dz.plane = a->T * p.dz.ld;
        p.dz.p = l.take<uint16_t>(planes * p.dz.plane);
        f.rows.index = l.take<int>(a->T);
        f.rows.place = l.take<int>(a->T);
        f.rows.count = l.take<int>(2);
        f.rows.row_lse = l.take<float>(a->T);
        f.rows.row_scale = l.take<float>(a->T);
        f.rows.row_target = l.take<int>(a->T);
        if (io) {
            p.rests = l.take<VocabRest>(a->T * kVocabRests);
            f.rows.row_others = p.row_others = l.take<int>(a->T);
            p.row_key = l.take<int>(a->T);
            p.row_sum = l.take<float>(a->T);
            p.row_left = l.take<float2>(a->T);
            p.sum_part = l.take<float>(a->T * sum_blocks(p, each));
        }
        if (p.splits_w > 1) p.dw_part = l.take<float>(p.splits_w * each * Kp);
        p.dh_part = l.take<float>(p.splits * a->T * Kp);
        p.count = f.rows.count; p.row_lse = f.rows.row_lse; p.row_scale = f.rows.row_scale; p.row_target = f.rows.row_target;
        f.h.index = f.rows.index; f.h.count = f.rows.count;
        f.rows.side = (int)side_n(planes, p.side_h); f.rows.across = (int)(up(a->K, p.side_h) / p.side_h);
        f.rows.at_once = p.side_h == kVocabTile ? 256 : 512;
        f.rows.units = f.rows.across * (up(a->T, f.rows.side) / f.rows.side) * p.splits; f.rows.each = each; f.rows.splits = p.splits;
        f.rows.T = a->T; f.rows.V = a->V; f.rows.target = a->target;
    }
    f.bytes = l.at;
    return f;
}
// The piece of the vocabulary from word v0 on, copied if it has to be.
int vocab_piece(VocabPlan &f, const void *weight, int64_t stride, int64_t v0, hipStream_t s) {
    VocabParams &p = f.p;
    p.v0 = v0;
    p.V = p.words - v0 < f.each ? p.words - v0 : f.each;
    p.first = v0 == 0;
    p.sum_blocks = (int)sum_blocks(p, p.V);
    const char *from = reinterpret_cast<const char *>(weight) + v0 * stride * (p.io ? 2 : 4);
    if (!f.w.src) { p.w.p = reinterpret_cast<const uint16_t *>(from); return LRNNX_OK; }
    f.w.src = from; f.w.rows = p.V;
    return status(launch_vocab_pack(f.w, s));
}

}  // namespace

extern "C" {

size_t lrnnx_vocab_loss_fwd_workspace_bytes(const lrnnx_vocab_fwd_args *a) {
    if (!a || a->struct_size != sizeof(lrnnx_vocab_fwd_args) || vocab_checks(a) != LRNNX_OK) return 0;
    return plan_vocab(a, nullptr, false).bytes;
}

int lrnnx_vocab_loss_fwd(const lrnnx_vocab_fwd_args *a) {
    if (!a || a->struct_size != sizeof(lrnnx_vocab_fwd_args)) return LRNNX_ERR_INVALID_ARG;
    if (const int e = vocab_checks(a)) return e;
    if (!vocab_inputs(a) || !a->loss || !a->lse || !on(a->loss, 4) || !on(a->lse, 4) || !on(a->workspace, 256)) return LRNNX_ERR_INVALID_ARG;
    VocabPlan f = plan_vocab(a, reinterpret_cast<char *>(a->workspace), false);
    if (!a->workspace || a->workspace_bytes < f.bytes) return LRNNX_ERR_WORKSPACE;
    const hipStream_t s = reinterpret_cast<hipStream_t>(a->stream);
    if (f.h.src && launch_vocab_pack(f.h, s) != hipSuccess) return LRNNX_ERR_LAUNCH;
    for (int64_t v0 = 0; v0 < a->V; v0 += f.each) {
        if (const int e = vocab_piece(f, a->weight, a->weight_stride, v0, s)) return e;
        if (launch_vocab_logits(f.p, false, s) != hipSuccess) return LRNNX_ERR_LAUNCH;
    }
    const VocabLoss end{a->T, a->V, f.p.parts, a->target, f.p.part, f.p.hit, a->loss, a->lse};
    return status(launch_vocab_loss(end, s));
}

size_t lrnnx_vocab_loss_bwd_workspace_bytes(const lrnnx_vocab_bwd_args *a) {
    if (!a || a->struct_size != sizeof(lrnnx_vocab_bwd_args) || vocab_checks(a) != LRNNX_OK) return 0;
    return plan_vocab(a, nullptr, true).bytes;
}

int lrnnx_vocab_loss_bwd(const lrnnx_vocab_bwd_args *a) {
    if (!a || a->struct_size != sizeof(lrnnx_vocab_bwd_args)) return LRNNX_ERR_INVALID_ARG;
    if (const int e = vocab_checks(a)) return e;
    const size_t es = elem(a->io_dtype);
    if (!vocab_inputs(a) || !a->lse || !a->dloss || (!a->dh && !a->dweight)) return LRNNX_ERR_INVALID_ARG;
    if (!on(a->lse, 4) || !on(a->dloss, 4) || !on(a->dh, es) || !on(a->dweight, es) || !on(a->workspace, 256)) return LRNNX_ERR_INVALID_ARG;
    VocabPlan f = plan_vocab(a, reinterpret_cast<char *>(a->workspace), true);
    if (!a->workspace || a->workspace_bytes < f.bytes) return LRNNX_ERR_WORKSPACE;
    const hipStream_t s = reinterpret_cast<hipStream_t>(a->stream);
    // the words are read again for dh when dweight is there
    const int64_t bytes = (int64_t)es;
    const Area words(a->weight, a->K * bytes, a->V, a->weight_stride * bytes), dh(a->dh, a->T * a->K * bytes), dweight(a->dweight, a->V * a->K * bytes);
    if (meet(words, {dh, dweight}) || meet(dh, dweight)) return LRNNX_ERR_INVALID_ARG;
    f.rows.lse = a->lse; f.rows.dloss = a->dloss; f.rows.dloss_stride = a->dloss_stride;
    if (launch_vocab_rows(f.rows, s) != hipSuccess || launch_vocab_pack(f.h, s) != hipSuccess) return LRNNX_ERR_LAUNCH;
    f.p.dw = a->dweight;
    for (int64_t v0 = 0; v0 < a->V; v0 += f.each) {
        if (const int e = vocab_piece(f, a->weight, a->weight_stride, v0, s)) return e;
        if (launch_vocab_logits(f.p, true, s) != hipSuccess) return LRNNX_ERR_LAUNCH;
        if (f.p.io && launch_vocab_rests(f.p, s) != hipSuccess) return LRNNX_ERR_LAUNCH;
        if (a->dh && launch_vocab_dh(f.p, s) != hipSuccess) return LRNNX_ERR_LAUNCH;
        if (!a->dweight) continue;
        if (launch_vocab_dw(f.p, s) != hipSuccess) return LRNNX_ERR_LAUNCH;
        if (f.p.splits_w == 1) continue;
        const VocabAdd parts{f.p.V, f.p.V * f.p.Kp, a->K, (int)f.p.Kp, f.p.io, f.p.splits_w, f.p.dw_part, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, 0, reinterpret_cast<char *>(a->dweight) + v0 * a->K * (int64_t)es};
        if (launch_vocab_add(parts, s) != hipSuccess) return LRNNX_ERR_LAUNCH;
    }
    if (!a->dh) return LRNNX_OK;
    const VocabAdd end{a->T, a->T * f.p.Kp, a->K, (int)f.p.Kp, f.p.io, f.p.splits, f.p.dh_part, f.rows.place, f.rows.count, f.p.row_key, f.p.row_left, f.p.rests, a->weight, a->weight_stride, a->dh};
    return status(launch_vocab_add(end, s));
}

}  // extern "C"

// ---------------------------------------------------------------- norm and clipping
namespace {

constexpr int64_t kGradMost = (int64_t)1 << 44;        // elements in all
// Elements of a piece: about `many` pieces in all, of 8192 elements at least.  The more there are, the less the end of a launch waits for the last; one workgroup adds up the norm's. (290
// tensors, 4e8 elements, with 4096, 16384, 32768 of the norm: 181, 171 and 170 us, 4.6, 4.6 and 6.8 to add them; with 4096, 16384, 32768, 65536 of the scale: 313, 292, 285, 280.)
constexpr int64_t kNormPieces = 16384, kScalePieces = 65536;
int64_t grad_piece(const int64_t *numel, int64_t count, int64_t many, int64_t &pieces) {
    int64_t total = 0;
    for (int64_t i = 0; i < count; ++i) total += numel[i];
    int64_t n = up(total / many, 2048);
    n = n < 8192 ? 8192 : n > 1 << 24 ? 1 << 24 : n;
    pieces = 0;
    for (int64_t i = 0; i < count; ++i) pieces += (numel[i] + n - 1) / n;
    return n;
}
template <class A> int grad_checks(const A *a) {
    if (a->count < 1 || !a->grads || !a->numel || !a->dtype) return LRNNX_ERR_INVALID_ARG;
    int64_t total = 0;
    for (int64_t i = 0; i < a->count; ++i) {
        if (a->numel[i] < 0 || !io_type(a->dtype[i])) return LRNNX_ERR_INVALID_ARG;
        if (a->numel[i] > kGradMost || (total += a->numel[i]) > kGradMost) return LRNNX_ERR_UNSUPPORTED;
        if (a->numel[i] && (!a->grads[i] || !on(a->grads[i], elem(a->dtype[i])))) return LRNNX_ERR_INVALID_ARG;
    }
    return LRNNX_OK;
}
// `launch` on lists of the tensors that have elements; false if it fails
template <class A, class F> bool grad_lists(const A *a, void *const *out, const int32_t *out_dtype, int64_t piece, F launch) {
    GradList l;
    l.count = 0; l.piece = (int)piece; l.base = 0; l.first[0] = 0;
    for (int64_t i = 0; i < a->count; ++i) {
        if (a->numel[i]) {
            const int k = l.count++;
            l.g[k] = a->grads[i];
            l.out[k] = out ? out[i] : const_cast<void *>(static_cast<const void *>(a->grads[i]));
            l.n[k] = a->numel[i];
            l.io[k] = (uint8_t)((a->dtype[i] == LRNNX_BF16 ? 1 : 0) | ((out ? out_dtype[i] : a->dtype[i]) == LRNNX_BF16 ? 2 : 0));
            l.first[k + 1] = l.first[k] + (uint32_t)((a->numel[i] + piece - 1) / piece);
        }
        if (l.count == kGradTensors || (i + 1 == a->count && l.count)) {
            if (launch(l) != hipSuccess) return false;
            l.base += l.first[l.count];
            l.count = 0;
        }
    }
    return true;
}

}  // namespace

extern "C" {

size_t lrnnx_grad_norm_workspace_bytes(const lrnnx_grad_norm_args *a) {
    if (!a || a->struct_size != sizeof(lrnnx_grad_norm_args) || a->count < 1 || !a->numel) return 0;
    int64_t pieces, total = 0;
    for (int64_t i = 0; i < a->count; ++i)
        if (a->numel[i] < 0 || a->numel[i] > kGradMost || (total += a->numel[i]) > kGradMost) return 0;
    grad_piece(a->numel, a->count, kNormPieces, pieces);
    return (size_t)pieces * sizeof(double);
}

int lrnnx_grad_norm(const lrnnx_grad_norm_args *a) {
    if (!a || a->struct_size != sizeof(lrnnx_grad_norm_args)) return LRNNX_ERR_INVALID_ARG;
    if (const int e = grad_checks(a)) return e;
    if (!a->norm || !on(a->norm, 4) || !on(a->workspace, 16)) return LRNNX_ERR_INVALID_ARG;
    int64_t pieces;
    const int64_t piece = grad_piece(a->numel, a->count, kNormPieces, pieces);
    if (pieces && (!a->workspace || a->workspace_bytes < (size_t)pieces * sizeof(double))) return LRNNX_ERR_WORKSPACE;
    const hipStream_t s = reinterpret_cast<hipStream_t>(a->stream);
    double *sums = reinterpret_cast<double *>(a->workspace);
    if (!grad_lists(a, nullptr, nullptr, piece, [&](const GradList &l) { return launch_grad_squares(l, sums, s); })) return LRNNX_ERR_LAUNCH;
    return status(launch_grad_total(sums, (uint32_t)pieces, a->norm, s));
}

int lrnnx_grad_clip(const lrnnx_grad_clip_args *a) {
    if (!a || a->struct_size != sizeof(lrnnx_grad_clip_args)) return LRNNX_ERR_INVALID_ARG;
    if (const int e = grad_checks(a)) return e;
    if (!a->norm || !on(a->norm, 4) || !(a->max_norm >= 0.0f) || !(a->eps >= 0.0f) || (a->out && !a->out_dtype)) return LRNNX_ERR_INVALID_ARG;
    if (a->out)
        for (int64_t i = 0; i < a->count; ++i) {
            if (a->out_dtype[i] != LRNNX_F32 && a->out_dtype[i] != a->dtype[i]) return LRNNX_ERR_INVALID_ARG;
            if (a->numel[i] && (!a->out[i] || !on(a->out[i], elem(a->out_dtype[i])))) return LRNNX_ERR_INVALID_ARG;
        }
    // every workgroup reads the norm: no result may lie there
    for (int64_t i = 0; i < a->count; ++i) {
        const int32_t type = a->out ? a->out_dtype[i] : a->dtype[i];
        if (a->numel[i] && meet(Area(a->norm, 4), Area(a->out ? a->out[i] : a->grads[i], a->numel[i] * (int64_t)elem(type)))) return LRNNX_ERR_INVALID_ARG;
    }
    int64_t pieces;
    const int64_t piece = grad_piece(a->numel, a->count, kScalePieces, pieces);
    const hipStream_t s = reinterpret_cast<hipStream_t>(a->stream);
    return grad_lists(a, a->out, a->out_dtype, piece, [&](const GradList &l) { return launch_grad_scale(l, a->norm, a->max_norm, a->eps, !a->out, s); }) ? LRNNX_OK : LRNNX_ERR_LAUNCH;
}

}  // extern "C"
