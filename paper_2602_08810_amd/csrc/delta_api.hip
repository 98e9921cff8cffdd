// C ABI of the gated delta rule and of the norms around a block: argument checks, layout of workspace and saved data, launches.
// Nothing here allocates, frees or synchronises; see include/lrnnx.h for the contract.
#include "../../include/lrnnx.h"
#include "delta.hpp"
#include "block_norm.hpp"

using namespace lrnnx;

namespace {

inline int64_t up(int64_t x, int64_t m) { return (x + m - 1) / m * m; }
inline bool on16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline bool on_elem(const void *p, size_t es) { return (reinterpret_cast<uintptr_t>(p) & (es - 1)) == 0; }
inline size_t elem(int dtype) { return dtype == LRNNX_BF16 ? 2 : 4; }

// What the forward and the backward call have in common.
struct Shape {
    int B, Hk, Hv, dk, dv, dkp, dvp, bf16, planes;       // planes: bfloat16 numbers that an input is the sum of
    int exact;                                           // a gradient of the gates is float32, and so what it comes from
    int64_t L, rows, nslots, slots_each;
};

template <class A> int common_checks(const A *a) {
    if (a->B < 1 || a->Hk < 1 || a->Hv < 1 || a->dk < 1 || a->dv < 1 || a->L < 1) return LRNNX_ERR_INVALID_ARG;
    if (a->Hv % a->Hk) return LRNNX_ERR_INVALID_ARG;
    if (a->io_dtype != LRNNX_F32 && a->io_dtype != LRNNX_BF16) return LRNNX_ERR_INVALID_ARG;
    if (a->gate_dtype != LRNNX_F32 && a->gate_dtype != a->io_dtype) return LRNNX_ERR_INVALID_ARG;
    if (a->dk > 128 || a->dv > 256 || a->B > 65535 || a->Hv > 65535) return LRNNX_ERR_UNSUPPORTED;
    // rows, slots and their arrays stay countable; a slot and head is a workgroup of one launch
    if (a->L > ((int64_t)1 << 40)) return LRNNX_ERR_UNSUPPORTED;
    const int64_t slots = a->cu_seqlens ? a->L / kDeltaSlot + a->B : a->B * ((a->L + kDeltaSlot - 1) / kDeltaSlot);
    if (slots > (int64_t)0x0fffffff / a->Hv) return LRNNX_ERR_UNSUPPORTED;
    return LRNNX_OK;
}
template <class A> Shape shape_of(const A *a) {
    Shape s;
    s.B = a->B; s.Hk = a->Hk; s.Hv = a->Hv; s.dk = a->dk; s.dv = a->dv; s.L = a->L;
    s.dkp = a->dk > 64 ? 128 : 64; s.dvp = (int)up(a->dv, 32);
    s.bf16 = a->io_dtype == LRNNX_BF16; s.planes = s.bf16 ? 1 : 3; s.exact = a->gate_dtype == LRNNX_F32;
    s.rows = (a->cu_seqlens ? 1 : (int64_t)a->B) * a->L;
    s.slots_each = (a->L + kDeltaSlot - 1) / kDeltaSlot;
    s.nslots = a->cu_seqlens ? a->L / kDeltaSlot + a->B : a->B * s.slots_each;
    return s;
}
inline int adjoint_planes(const Shape &s, bool s0) { return s.exact || s0 ? 3 : 2; }

// Rows that do not overlap and of which 32 span less than 2 GB.
bool rows_near(const Shape &s, int width, int64_t sl) { return s.L == 1 || (sl >= width && sl < (int64_t)1 << 24); }
// Strided rows of `width` elements that the matrix kernels can read as they lie.
bool rows_in_place(const Shape &s, const void *p, int width, int padded, int64_t sb, int64_t sl, int64_t sh, bool one_batch, int H) {
    return s.bf16 && width == padded && on16(p) && rows_near(s, width, sl) && (one_batch || s.B == 1 || sb % 8 == 0) && (s.L == 1 || sl % 8 == 0) && (H == 1 || sh % 8 == 0);
}

// Lays arrays out one after the other, 256-byte aligned; with a null base it only counts.
struct Layout {
    char *base;
    size_t at = 0;
    template <class T> T *take(int64_t count) {
        const size_t here = (at + 255) / 256 * 256;
        at = here + (size_t)count * sizeof(T);
        return base ? reinterpret_cast<T *>(base + here) : nullptr;
    }
};
inline int64_t mats(const Shape &s) { return s.nslots * s.Hv * 2; }
inline int a_planes(const Shape &s) { return s.bf16 ? 2 : 3; }

// States by slot and rows by step, float32 or 16 bits with the units of their blocks.
void lay_kept(const Shape &s, Layout &l, void *&states, void *&rows, float *&units) {
    const int64_t size = s.exact ? 4 : 2;
    states = l.take<char>(s.nslots * s.Hv * s.dkp * s.dvp * size);
    rows = l.take<char>(s.rows * s.Hv * s.dvp * size);
    if (!s.exact) units = l.take<float>(s.nslots * s.Hv * 6 * (s.dvp / 16));
}
void lay_saved(const Shape &s, bool s0, Layout &l, DeltaParams &p) {
    lay_kept(s, l, p.states, p.err, p.units);
    p.mats_adj = l.take<uint16_t>(mats(s) * chunk_words(adjoint_planes(s, s0), adjoint_planes(s, s0)));
}

DeltaRows lay_rows(const Shape &s, Layout &l, const void *src, int H, int width, int padded, int64_t sb, int64_t sl, int64_t sh, bool one_batch, bool &copied) {
    copied = !rows_in_place(s, src, width, padded, sb, sl, sh, one_batch, H);
    DeltaRows r;
    if (!copied) {
        r.p = reinterpret_cast<const uint16_t *>(src); r.plane = 0; r.sb = sb; r.sl = s.L == 1 ? padded : sl; r.sh = sh;
        return r;
    }
    r.plane = s.rows * H * padded;
    r.p = l.take<uint16_t>(s.planes * r.plane);
    r.sb = s.L * H * padded; r.sl = (int64_t)H * padded; r.sh = padded;
    return r;
}
void add_pack(const Shape &s, DeltaPacks &all, const DeltaRows &r, const void *src, int H, int width, int padded, int64_t sb, int64_t sl, int64_t sh, bool one_batch) {
    DeltaPack &k = all.p[all.n++];
    k.src = src; k.sb = sb; k.sl = sl; k.sh = sh;
    k.dst = const_cast<uint16_t *>(r.p); k.plane = r.plane;
    k.H = H; k.d = width; k.dp = padded;
    const int64_t each = s.bf16 ? 8 : 4;                  // elements of 16 bytes
    k.vec = on16(src) && (one_batch || s.B == 1 || sb % each == 0) && (s.L == 1 || sl % each == 0) && (H == 1 || sh % each == 0);
    k.items = (unsigned)(H * (padded / 8));
    k.rows = k.items < 256 ? 256 / k.items : 1;
    k.by_items = Divider(k.items); k.by_head = Divider((unsigned)(padded / 8));
    all.B = one_batch ? 1 : s.B; all.planes = s.planes; all.io = s.bf16; all.L = s.L;
}

template <class A> void set_inputs(const A *a, const Shape &s, DeltaParams &p) {
    p.B = s.B; p.Hk = s.Hk; p.Hv = s.Hv; p.dk = s.dk; p.dv = s.dv; p.dvp = s.dvp;
    p.L = s.L; p.nslots = s.nslots; p.slots_each = s.slots_each; p.scale = a->scale;
    p.io = s.bf16; p.gate_io = a->gate_dtype == LRNNX_BF16; p.exact = s.exact; p.cu = a->cu_seqlens;
    p.v = a->v; p.g = a->g; p.beta = a->beta;
    p.v_sb = a->v_stride_b; p.v_sl = a->v_stride_l; p.v_sh = a->v_stride_h;
    p.g_sb = a->g_stride_b; p.g_sl = a->g_stride_l; p.g_sh = a->g_stride_h;
    p.be_sb = a->beta_stride_b; p.be_sl = a->beta_stride_l; p.be_sh = a->beta_stride_h;
    p.s0 = a->s0;
}

// Segments of the time axis: walked side by side where the heads alone leave the chip part empty, at the price of a walk with dk more columns before and
// of chaining (4 us a segment).  32768 steps of 8 heads of 128 x 128, bfloat16: 1640 us in one walk, 16 segments 149 + 62 + 144.
// Taken where both walks (the first over as many turns of the chip as its workgroups need, each chunk 1.15 times a single walk's, in float32 1.25) and the
// chaining, counted in chunks, come to less than one walk's chunks.  Whole calls for prompts, one walk / segments, us, of 128 x 128 in bfloat16: 8 heads 768
// steps 54 / 61 (one), 1024 68 / 65, 2048 122 / 83; 40 heads 1024 steps 73 / 94 (one), 2048 131 / 136 (one), 4096 246 / 231; float32 8 heads 1024 steps
// 120 / 97, 40 heads 137 / 178 (one), 4096 575 / 576; 64 x 64 of 64 heads 768 steps 51 / 53 (one), 2048 111 / 86, of 84 heads in float32 4096 steps
// 469 / 487 (one).
void plan_segments(const Shape &s, bool packed, Layout &l, DeltaParams &p) {
    p.nseg = 1; p.seg_chunks = 0; p.entry = nullptr; p.trans = nullptr;
    const int64_t heads = (int64_t)s.B * s.Hv, wgs = heads * ((s.dvp + 63) / 64), slots = s.slots_each;
    if (packed) return;
    int64_t n = 256 / wgs;                            // a workgroup a compute unit
    if (n > slots / 4) n = slots / 4;                 // of 256 steps at least (8 heads of 128 x 128, 1024 steps: 4 segments 65 us, 8 of 128 steps 71)
    if (n < 2) return;
    const int64_t each = (slots + n - 1) / n, segs = (slots + each - 1) / each;
    const double turns = (double)(heads * (segs - 1) * ((s.dvp + s.dkp + 63) / 64)) / (s.bf16 && s.dkp == 64 ? 512 : 256);
    if ((1 + (turns > 1 ? turns : 1)) * 2 * each * (s.bf16 ? 1.15 : 1.25) + 2 * segs + 3 >= 2 * slots) return;
    p.nseg = (int)segs; p.seg_chunks = (int)(2 * each);
    p.entry = l.take<float>(heads * p.nseg * s.dkp * s.dvp);
    p.trans = l.take<uint16_t>(heads * (p.nseg - 1) * p.np * s.dkp * s.dkp);
}

struct DeltaFwdPlan { DeltaParams p; bool copy_q, copy_k, copy_v; size_t bytes, saved; };
DeltaFwdPlan plan_fwd(const lrnnx_delta_fwd_args *a, const Shape &s, char *ws, char *saved) {
    DeltaFwdPlan f{};
    set_inputs(a, s, f.p);
    const bool one = a->cu_seqlens != nullptr;
    f.p.np = s.exact || a->s0 || a->s_last ? 3 : 2;
    f.p.np_adjoint = adjoint_planes(s, a->s0 != nullptr);
    Layout l{ws}, sv{saved};
    f.p.q = lay_rows(s, l, a->q, s.Hk, s.dk, s.dkp, a->q_stride_b, a->q_stride_l, a->q_stride_h, one, f.copy_q);
    f.p.k = lay_rows(s, l, a->k, s.Hk, s.dk, s.dkp, a->k_stride_b, a->k_stride_l, a->k_stride_h, one, f.copy_k);
    f.copy_v = !rows_near(s, s.dv, a->v_stride_l);
    if (f.copy_v) {                                   // v of rows that overlap or lie far apart, one after the other
        f.p.v = l.take<char>(s.rows * s.Hv * s.dv * (int64_t)elem(a->io_dtype));
        f.p.v_sb = s.L * s.Hv * s.dv; f.p.v_sl = (int64_t)s.Hv * s.dv; f.p.v_sh = s.dv;
    } else if (s.L == 1) f.p.v_sl = s.dv;
    f.p.mats = l.take<uint16_t>(mats(s) * chunk_words(f.p.np, a_planes(s)));
    if (a->saved || !ws) lay_saved(s, a->s0 != nullptr, sv, f.p);
    plan_segments(s, one, l, f.p);
    f.bytes = l.at; f.saved = sv.at;
    return f;
}

struct DeltaBwdPlan { DeltaParams p; bool copy_q, copy_k, copy_d; size_t bytes, saved; };
DeltaBwdPlan plan_bwd(const lrnnx_delta_bwd_args *a, const Shape &s, char *ws, char *saved) {
    DeltaBwdPlan f{};
    set_inputs(a, s, f.p);
    const bool one = a->cu_seqlens != nullptr;
    f.p.np = adjoint_planes(s, a->s0 != nullptr);
    Layout l{ws}, sv{saved};
    f.p.q = lay_rows(s, l, a->q, s.Hk, s.dk, s.dkp, a->q_stride_b, a->q_stride_l, a->q_stride_h, one, f.copy_q);
    f.p.k = lay_rows(s, l, a->k, s.Hk, s.dk, s.dkp, a->k_stride_b, a->k_stride_l, a->k_stride_h, one, f.copy_k);
    f.p.dout = lay_rows(s, l, a->dout, s.Hv, s.dv, s.dvp, a->dout_stride_b, a->dout_stride_l, a->dout_stride_h, one, f.copy_d);
    lay_saved(s, a->s0 != nullptr, sv, f.p);
    lay_kept(s, l, f.p.dstates, f.p.z, f.p.dunits);
    if (s.Hv > s.Hk) f.p.part = l.take<float>(2 * s.rows * s.Hv * s.dkp);
    plan_segments(s, one, l, f.p);
    f.bytes = l.at; f.saved = sv.at;
    return f;
}

template <class A> bool inputs_given(const A *a) { return a->q && a->k && a->v && a->g && a->beta; }
template <class A> bool inputs_on_elements(const A *a) {
    const size_t es = elem(a->io_dtype), gs = elem(a->gate_dtype);
    return on_elem(a->q, es) && on_elem(a->k, es) && on_elem(a->v, es) && on_elem(a->g, gs) && on_elem(a->beta, gs) && on_elem(a->s0, 4) &&
           on_elem(a->cu_seqlens, 8);
}

}  // namespace

extern "C" {

size_t lrnnx_gated_delta_fwd_workspace_bytes(const lrnnx_delta_fwd_args *a) {
    if (!a || a->struct_size != sizeof(lrnnx_delta_fwd_args) || common_checks(a) != LRNNX_OK) return 0;
    return plan_fwd(a, shape_of(a), nullptr, nullptr).bytes;
}
size_t lrnnx_gated_delta_saved_bytes(const lrnnx_delta_fwd_args *a) {
    if (!a || a->struct_size != sizeof(lrnnx_delta_fwd_args) || common_checks(a) != LRNNX_OK) return 0;
    return plan_fwd(a, shape_of(a), nullptr, nullptr).saved;
}

int lrnnx_gated_delta_fwd(const lrnnx_delta_fwd_args *a) {
    if (!a || a->struct_size != sizeof(lrnnx_delta_fwd_args)) return LRNNX_ERR_INVALID_ARG;
    if (const int e = common_checks(a)) return e;
    if (!inputs_given(a) || !a->o) return LRNNX_ERR_INVALID_ARG;
    const size_t es = elem(a->io_dtype);
    if (!inputs_on_elements(a) || !on_elem(a->o, es) || !on_elem(a->s_last, 4) || !on16(a->saved) || !on16(a->workspace)) return LRNNX_ERR_INVALID_ARG;
    const Shape s = shape_of(a);
    DeltaFwdPlan f = plan_fwd(a, s, reinterpret_cast<char *>(a->workspace), reinterpret_cast<char *>(a->saved));
    if (!a->workspace || a->workspace_bytes < f.bytes || (a->saved && a->saved_bytes < f.saved)) return LRNNX_ERR_WORKSPACE;
    DeltaParams &p = f.p;
    p.o = a->o; p.o_sb = a->o_stride_b; p.o_sl = a->o_stride_l; p.o_sh = a->o_stride_h; p.s_last = a->s_last;
    const bool one = a->cu_seqlens != nullptr;
    p.o_vec = (reinterpret_cast<uintptr_t>(a->o) & (4 * es - 1)) == 0 && (one || s.B == 1 || a->o_stride_b % 4 == 0) &&
              (s.L == 1 || a->o_stride_l % 4 == 0) && (s.Hv == 1 || a->o_stride_h % 4 == 0);
    const hipStream_t st = reinterpret_cast<hipStream_t>(a->stream);
    DeltaPacks packs;
    if (f.copy_q) add_pack(s, packs, p.q, a->q, s.Hk, s.dk, s.dkp, a->q_stride_b, a->q_stride_l, a->q_stride_h, one);
    if (f.copy_k) add_pack(s, packs, p.k, a->k, s.Hk, s.dk, s.dkp, a->k_stride_b, a->k_stride_l, a->k_stride_h, one);
    if (packs.n && launch_delta_pack(packs, st) != hipSuccess) return LRNNX_ERR_LAUNCH;
    if (f.copy_v) {
        DeltaGather k{};
        k.src = a->v; k.sb = a->v_stride_b; k.sl = a->v_stride_l; k.sh = a->v_stride_h;
        k.dst = const_cast<void *>(p.v);
        k.B = one ? 1 : s.B; k.H = s.Hv; k.d = s.dv; k.io = s.bf16; k.L = s.L;
        if (launch_delta_gather(k, st) != hipSuccess) return LRNNX_ERR_LAUNCH;
    }
    if (launch_delta_prep(p, st) != hipSuccess) return LRNNX_ERR_LAUNCH;
    return launch_delta_scan(p, st) == hipSuccess ? LRNNX_OK : LRNNX_ERR_LAUNCH;
}

size_t lrnnx_gated_delta_bwd_workspace_bytes(const lrnnx_delta_bwd_args *a) {
    if (!a || a->struct_size != sizeof(lrnnx_delta_bwd_args) || common_checks(a) != LRNNX_OK) return 0;
    return plan_bwd(a, shape_of(a), nullptr, nullptr).bytes;
}

int lrnnx_gated_delta_bwd(const lrnnx_delta_bwd_args *a) {
    if (!a || a->struct_size != sizeof(lrnnx_delta_bwd_args)) return LRNNX_ERR_INVALID_ARG;
    if (const int e = common_checks(a)) return e;
    if (!inputs_given(a) || !a->dout || !a->saved || !a->dq || !a->dkey || !a->dval || !a->dg || !a->dbeta) return LRNNX_ERR_INVALID_ARG;
    const size_t es = elem(a->io_dtype), gs = elem(a->gate_dtype);
    if (!inputs_on_elements(a) || !on_elem(a->dout, es) || !on_elem(a->ds_last, 4) || !on16(a->saved) || !on_elem(a->dq, es) || !on_elem(a->dkey, es) ||
        !on_elem(a->dval, es) || !on_elem(a->dg, gs) || !on_elem(a->dbeta, gs) || !on_elem(a->ds0, 4) || !on16(a->workspace))
        return LRNNX_ERR_INVALID_ARG;
    const Shape s = shape_of(a);
    DeltaBwdPlan f = plan_bwd(a, s, reinterpret_cast<char *>(a->workspace), reinterpret_cast<char *>(const_cast<void *>(a->saved)));
    if (!a->workspace || a->workspace_bytes < f.bytes || a->saved_bytes != f.saved) return LRNNX_ERR_WORKSPACE;      // (its layout goes by its size)
    DeltaParams &p = f.p;
    p.ds_last = a->ds_last; p.ds0 = a->ds0;
    auto on4 = [&](const void *q) { return (reinterpret_cast<uintptr_t>(q) & (4 * es - 1)) == 0; };
    p.o_vec = s.dv % 4 == 0 && on4(a->dval) && on4(a->dq) && on4(a->dkey);
    p.dq = a->dq; p.dkk = a->dkey; p.dvv = a->dval; p.dg = a->dg; p.dbeta = a->dbeta;
    const bool one = a->cu_seqlens != nullptr;
    const hipStream_t st = reinterpret_cast<hipStream_t>(a->stream);
    DeltaPacks packs;
    if (f.copy_q) add_pack(s, packs, p.q, a->q, s.Hk, s.dk, s.dkp, a->q_stride_b, a->q_stride_l, a->q_stride_h, one);
    if (f.copy_k) add_pack(s, packs, p.k, a->k, s.Hk, s.dk, s.dkp, a->k_stride_b, a->k_stride_l, a->k_stride_h, one);
    if (f.copy_d) add_pack(s, packs, p.dout, a->dout, s.Hv, s.dv, s.dvp, a->dout_stride_b, a->dout_stride_l, a->dout_stride_h, one);
    if (packs.n && launch_delta_pack(packs, st) != hipSuccess) return LRNNX_ERR_LAUNCH;
    if (launch_delta_adjoint(p, st) != hipSuccess) return LRNNX_ERR_LAUNCH;
    return launch_delta_grads(p, st) == hipSuccess ? LRNNX_OK : LRNNX_ERR_LAUNCH;
}

int lrnnx_gated_delta_step(const lrnnx_delta_step_args *a) {
    if (!a || a->struct_size != sizeof(lrnnx_delta_step_args)) return LRNNX_ERR_INVALID_ARG;
    if (a->B < 1 || a->Hk < 1 || a->Hv < 1 || a->dk < 1 || a->dv < 1 || a->Hv % a->Hk) return LRNNX_ERR_INVALID_ARG;
    if (a->io_dtype != LRNNX_F32 && a->io_dtype != LRNNX_BF16) return LRNNX_ERR_INVALID_ARG;
    if (a->gate_dtype != LRNNX_F32 && a->gate_dtype != a->io_dtype) return LRNNX_ERR_INVALID_ARG;
    if (a->dk > 128 || a->dv > 256 || a->B > 65535 || a->Hv > 65535) return LRNNX_ERR_UNSUPPORTED;
    if (!a->q || !a->k || !a->v || !a->g || !a->beta || !a->state || !a->o) return LRNNX_ERR_INVALID_ARG;
    const size_t es = elem(a->io_dtype), gs = elem(a->gate_dtype);
    if (!on_elem(a->q, es) || !on_elem(a->k, es) || !on_elem(a->v, es) || !on_elem(a->o, es) || !on_elem(a->g, gs) || !on_elem(a->beta, gs) ||
        !on_elem(a->state, 4))
        return LRNNX_ERR_INVALID_ARG;
    DeltaStepParams p{};
    p.B = a->B; p.Hk = a->Hk; p.Hv = a->Hv; p.dk = a->dk; p.dv = a->dv; p.gate_io = a->gate_dtype == LRNNX_BF16; p.scale = a->scale;
    p.q = a->q; p.k = a->k; p.v = a->v; p.g = a->g; p.beta = a->beta; p.state = a->state; p.o = a->o;
    p.q_sb = a->q_stride_b; p.q_sh = a->q_stride_h; p.k_sb = a->k_stride_b; p.k_sh = a->k_stride_h; p.v_sb = a->v_stride_b; p.v_sh = a->v_stride_h;
    p.g_sb = a->g_stride_b; p.g_sh = a->g_stride_h; p.be_sb = a->beta_stride_b; p.be_sh = a->beta_stride_h; p.o_sb = a->o_stride_b; p.o_sh = a->o_stride_h;
    return launch_delta_step(p, a->io_dtype == LRNNX_BF16, reinterpret_cast<hipStream_t>(a->stream)) == hipSuccess ? LRNNX_OK : LRNNX_ERR_LAUNCH;
}

}  // extern "C"

namespace {

template <class A> int norm_checks(const A *a) {
    if (a->M < 1 || a->D < 1 || a->groups < 1 || a->D % a->groups || a->gate_act < 0 || a->gate_act > 1) return LRNNX_ERR_INVALID_ARG;
    if (a->io_dtype != LRNNX_F32 && a->io_dtype != LRNNX_BF16) return LRNNX_ERR_INVALID_ARG;
    if (a->res_dtype != LRNNX_F32 && a->res_dtype != a->io_dtype) return LRNNX_ERR_INVALID_ARG;
    if (!(a->eps >= 0.0f) || !a->x) return LRNNX_ERR_INVALID_ARG;
    if (a->D > 8192 || a->M > ((int64_t)1 << 40)) return LRNNX_ERR_UNSUPPORTED;
    const size_t es = elem(a->io_dtype), rs = elem(a->res_dtype);
    if (!on_elem(a->x, es) || !on_elem(a->gate, es) || !on_elem(a->residual, rs) || !on_elem(a->post_weight, 4) || !on_elem(a->res_scale, 4) ||
        !on_elem(a->pre_weight, 4))
        return LRNNX_ERR_INVALID_ARG;
    return LRNNX_OK;
}
template <class A> NormParams norm_params(const A *a) {
    NormParams p{};
    p.M = a->M; p.D = a->D; p.groups = a->groups; p.width = a->D / a->groups; p.post_shared = a->post_shared != 0 && a->groups > 1;
    p.io = a->io_dtype == LRNNX_BF16; p.res_io = a->res_dtype == LRNNX_BF16; p.gate_act = a->gate_act; p.eps = a->eps;
    p.x = a->x; p.gate = a->gate; p.res = a->residual;
    p.x_s = a->x_stride; p.gate_s = a->gate_stride; p.res_s = a->residual_stride;
    p.post = a->post_weight; p.scale = a->res_scale; p.pre = a->pre_weight;
    return p;
}

}  // namespace

extern "C" {

int lrnnx_block_norm_fwd(const lrnnx_norm_fwd_args *a) {
    if (!a || a->struct_size != sizeof(lrnnx_norm_fwd_args)) return LRNNX_ERR_INVALID_ARG;
    if (const int e = norm_checks(a)) return e;
    if (!a->h || (a->pre_weight != nullptr) != (a->y != nullptr)) return LRNNX_ERR_INVALID_ARG;
    if (!on_elem(a->h, elem(a->res_dtype)) || !on_elem(a->y, elem(a->io_dtype))) return LRNNX_ERR_INVALID_ARG;
    NormParams p = norm_params(a);
    p.h = a->h; p.y = a->y;
    return launch_norm_fwd(p, reinterpret_cast<hipStream_t>(a->stream)) == hipSuccess ? LRNNX_OK : LRNNX_ERR_LAUNCH;
}

size_t lrnnx_block_norm_bwd_workspace_bytes(int64_t M, int64_t D) {
    if (M < 1 || D < 1 || D > 8192) return 0;
    return (size_t)norm_bwd_blocks(M, (int)D) * 3 * (size_t)D * sizeof(float);
}

int lrnnx_block_norm_bwd(const lrnnx_norm_bwd_args *a) {
    if (!a || a->struct_size != sizeof(lrnnx_norm_bwd_args)) return LRNNX_ERR_INVALID_ARG;
    if (const int e = norm_checks(a)) return e;
    if (!a->dx || (!a->dh && !a->dy) || (a->dy && !a->pre_weight)) return LRNNX_ERR_INVALID_ARG;
    if ((a->dgate && !a->gate) || (a->dresidual && !a->residual) || (a->dpost_weight && !a->post_weight) || (a->dres_scale && !a->res_scale) ||
        (a->dpre_weight && !a->pre_weight))
        return LRNNX_ERR_INVALID_ARG;
    const size_t es = elem(a->io_dtype), rs = elem(a->res_dtype);
    if (!on_elem(a->dh, rs) || !on_elem(a->dy, es) || !on_elem(a->dx, es) || !on_elem(a->dgate, es) || !on_elem(a->dresidual, rs) ||
        !on_elem(a->dpost_weight, 4) || !on_elem(a->dres_scale, 4) || !on_elem(a->dpre_weight, 4) || !on16(a->workspace))
        return LRNNX_ERR_INVALID_ARG;
    if (!a->workspace || a->workspace_bytes < lrnnx_block_norm_bwd_workspace_bytes(a->M, a->D)) return LRNNX_ERR_WORKSPACE;
    NormParams p = norm_params(a);
    p.dh = a->dh; p.dy = a->dy; p.dh_s = a->dh_stride; p.dy_s = a->dy_stride;
    p.dx = a->dx; p.dgate = a->dgate; p.dres = a->dresidual;
    p.dpost = a->dpost_weight; p.dscale = a->dres_scale; p.dpre = a->dpre_weight;
    p.sums = reinterpret_cast<float *>(a->workspace); p.blocks = norm_bwd_blocks(a->M, a->D);
    return launch_norm_bwd(p, reinterpret_cast<hipStream_t>(a->stream)) == hipSuccess ? LRNNX_OK : LRNNX_ERR_LAUNCH;
}

}  // extern "C"
