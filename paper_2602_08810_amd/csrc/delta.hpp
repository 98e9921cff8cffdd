// Host-visible parameter block and launcher declarations of the gated delta rule.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>
#include "kernels.hpp"

namespace lrnnx {

constexpr int kDeltaSlot = 64;           // steps between saved states; a slot holds two chunks
constexpr int kDeltaChunk = 32;          // steps whose corrections are solved for together

// The matrices of a chunk, in 16-bit words: T, then A, of np and npa planes (the adjoint's of the same number), of planes each two tiles of 16 rows, first the one of whose two 16 x 16 blocks one is zero (the
// other block alone, 256 a plane), then the whole one (512 a plane); then exp(G), exp(G_end - G), beta (3 x 32 floats).
constexpr int chunk_words(int np, int npa) { return (np + npa) * 768 + 192; }

// Rows of a matrix operand in bfloat16: element (plane, batch, step, head, column) at plane * plane_stride + b * sb + t * sl + h * sh + column,
// rows 16-byte aligned and zero beyond the head's width up to the padded one.  A float32 operand is the sum of three planes.
struct DeltaRows {
    const uint16_t *p;
    int64_t plane, sb, sl, sh;
};

struct DeltaParams {
    int B, Hk, Hv, dk, dv, dvp;          // dvp: dv padded to whole matrix tiles (32)
    int64_t L, nslots, slots_each;       // slots in all; of one sequence (batch form)
    float scale;
    int io, gate_io;                     // 1: bfloat16 inputs; gate_io: g and beta in the I/O type
    const int64_t *cu;
    DeltaRows q, k, dout;
    const void *v, *g, *beta;
    int64_t v_sb, v_sl, v_sh, g_sb, g_sl, g_sh, be_sb, be_sl, be_sh;
    const float *s0;
    void *o;
    int64_t o_sb, o_sl, o_sh;
    int o_vec;                           // rows of o take stores of four elements
    float *s_last;
    uint16_t *mats;                      // per slot, head and chunk: (I + N beta)^-1 and A as matrix operands, and the gates (chunk_words)
    uint16_t *mats_adj;                  // the same for the adjoint: ((I + beta N)^-1)^T and A^T; null: not wanted
    int exact;                           // what is saved is float32; else 16-bit floating point
    void *states, *err;                  // saved for the backward pass, by slot and head a column to a row [nslots,Hv,dvp,dkp], by step [rows,Hv,dvp]; null: not wanted
    float *units;                        // and in 16 bits the powers of two of their blocks of 16 columns: S0 (2 halves of its rows by G), E (4 times 16 steps by G) of a slot's head
    // backward
    const float *ds_last;
    float *ds0;
    void *dstates, *z;
    float *dunits;                       // likewise S1's (2 G), Z's (4 G)
    void *dq, *dkk, *dvv, *dg, *dbeta;
    float *part;                         // with shared key heads: [2,rows,Hv,dkp] every value head's share of dq and of dk
    int np, np_adjoint;                  // planes of the state chain, of its adjoint
    // segments of the time axis that are walked side by side (one sequence of a batch entry alone does not fill the chip); 1: none
    int nseg, seg_chunks, groups;        // segments, chunks of one (even); groups of columns (workgroups) of a head
    float *entry;                        // [B,Hv,nseg,dkp,dvp] state entering each segment (adjoint: of the segment's end)
    uint16_t *trans;                     // [B,Hv,nseg-1,planes,dkp,dkp] what a segment makes of the state that enters it
};

struct DeltaPack {                       // a strided operand copied into planes, [B,L,H,dp]
    const void *src;
    int64_t sb, sl, sh;
    uint16_t *dst;
    int64_t plane;
    int H, d, dp, vec;                   // vec: eight elements at a time may be read as 16-byte pieces
    unsigned items, rows;                // pieces of eight elements a step, steps a workgroup takes at once
    Divider by_items, by_head;
};
struct DeltaPacks {                      // all operands of a call that need it
    DeltaPack p[3];
    int n = 0, B, planes, io;
    int64_t L;
};
struct DeltaGather {                     // rows copied one after the other as they are
    const void *src;
    int64_t sb, sl, sh;
    void *dst;
    int B, H, d, io;
    int64_t L;
};

hipError_t launch_delta_pack(const DeltaPacks &p, hipStream_t s);
hipError_t launch_delta_gather(const DeltaGather &p, hipStream_t s);
hipError_t launch_delta_prep(const DeltaParams &p, hipStream_t s);
hipError_t launch_delta_scan(const DeltaParams &p, hipStream_t s);
hipError_t launch_delta_adjoint(const DeltaParams &p, hipStream_t s);
hipError_t launch_delta_join(const DeltaParams &p, bool adjoint, hipStream_t s);
hipError_t launch_delta_grads(const DeltaParams &p, hipStream_t s);

struct DeltaStepParams {
    int B, Hk, Hv, dk, dv, gate_io;
    float scale;
    const void *q, *k, *v, *g, *beta;
    int64_t q_sb, q_sh, k_sb, k_sh, v_sb, v_sh, g_sb, g_sh, be_sb, be_sh, o_sb, o_sh;
    float *state;
    void *o;
};
hipError_t launch_delta_step(const DeltaStepParams &p, int io, hipStream_t s);

}  // namespace lrnnx
