// Host-visible parameter blocks and launcher declarations of the loss over a vocabulary.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace lrnnx {

constexpr int kVocabTile = 256;          // rows and columns of a product's largest tile
// With bfloat16 inputs, what rounding takes from a row's elements of dz: the target's, and those of other words whose p is over kVocabLikely (fewer than kVocabRests).
constexpr int kVocabRests = 9;
constexpr float kVocabLikely = 0.125f;
struct VocabRest { int word; float rest; };
// A row's target and the number of its other rests in one number; -1: a target beyond the vocabulary
constexpr int kVocabWordBits = 27;

// A factor of a matrix product in bfloat16, `planes` numbers to an element (a float32 element is the sum of three): element (plane, row, column) at
// plane * plane_stride + row * ld + column.  16-byte aligned rows of whole 16-byte pieces.
struct VocabFactor {
    const uint16_t *p;
    int64_t plane, ld;
};

struct VocabParams {
    int64_t T, V, K, Kp;                 // V: words of this piece; Kp: K up to whole 16-byte pieces
    int side_z, side_h, side_w;          // first side of a tile of z, dh, dw
    bool wide, any;                      // w is float32, split where it is read; in rows that are no 16-byte pieces at 16-byte steps
    int planes, io;                      // io 1: bfloat16
    const int *count;                    // device: rows that have a target (null: all T); stretches of dh's words
    VocabFactor h, w, dz;                // [T,K], [V,K], [T,V]
    int64_t v0, words, each;             // first word of this piece, words in all, of a piece
    float *z_part;                       // [splits_z,T,ldz], if there are several
    int splits_z;
    int64_t ldz;
    // forward
    float *part;                         // [T, tiles (or pieces) of all words, 2]: largest, sum
    int64_t parts;
    float *hit;                          // [T] z of the target
    const int64_t *target;
    // backward, by row among those that have a target
    const float *row_lse, *row_scale;
    const int *row_target;               // -1: beyond the vocabulary
    VocabRest *rests;                    // [T,kVocabRests], the target's first, the others' by word; bfloat16 only, as the next six
    int *row_others;                     // how many others have been found
    int *row_key;
    float *sum_part;                     // sums of the stored dz over blocks of words: [blocks,T], of z in stretches [T,blocks]
    int sum_blocks;
    float *row_sum;                      // of the row's stored dz, all pieces so far
    float2 *row_left;                    // what is missing to the sum of its dz with all rests, which is 0; by how much its p are too small for that, relative to them
    float *dh_part;                      // [stretches, rows that have a target, Kp], within [splits,T,Kp]
    int splits, first;                   // first piece: the parts are set, not added to
    float *dw_part;                      // [splits_w,V,Kp], if there are several
    int splits_w;
    void *dw;                            // [words,K]
};
hipError_t launch_vocab_logits(const VocabParams &p, bool backward, hipStream_t s);
hipError_t launch_vocab_rests(const VocabParams &p, hipStream_t s);
hipError_t launch_vocab_dh(const VocabParams &p, hipStream_t s);
hipError_t launch_vocab_dw(const VocabParams &p, hipStream_t s);

// [rows,K] strided elements as a factor with Kp columns in rows of ldd, zeros behind the K-th (no planes: in float32); `index`: the source's row of each (and `count` rows)
struct VocabPack {
    const void *src; int64_t ld;
    uint16_t *dst; int64_t plane, ldd, rows;
    int K, Kp, io, planes;
    const int *index, *count;
};
hipError_t launch_vocab_pack(const VocabPack &p, hipStream_t s);

// What a product of so many tiles takes, in so many stretches of its terms: turns of the workgroups that there are at once; a tile's start and end take about as long as 256 terms,
// and every part is added once more.
__host__ __device__ inline float vocab_time(int64_t tiles, int64_t splits, int64_t at_once, int64_t terms) {
    return (float)((tiles * splits + at_once - 1) / at_once) * ((float)((terms + splits - 1) / splits) + 256.0f) * (1.0f + 0.01f * (float)splits);
}

struct VocabRows {
    int64_t T, V;
    const int64_t *target;
    const float *lse, *dloss; int64_t dloss_stride;
    int *index, *place, *count;          // row of the T that the i-th with a target is; place: the other way, -1: none
    float *row_lse, *row_scale;
    int *row_target;
    int *row_others;                     // set to 0, or null
    // for dh: tiles along K, rows of a tile, workgroups at once and in the launch; words of a piece; stretches that there is room for with all rows
    int across, side, at_once;
    int64_t units, each, splits;
};
hipError_t launch_vocab_rows(const VocabRows &p, hipStream_t s);

struct VocabLoss {
    int64_t T, V, parts;
    const int64_t *target;
    const float *part, *hit;
    float *loss, *lse;
};
hipError_t launch_vocab_loss(const VocabLoss &p, hipStream_t s);

struct VocabAdd {
    int64_t rows, plane;                 // rows of the result; elements from part to part
    int K, Kp, io, splits;
    const float *part;
    const int *place;                    // or null
    const int *count;                    // or null; device: rows of a part, parts
    const int *key;                      // by row of the parts, or null: as in VocabParams, with what is to be added
    const float2 *left;
    const VocabRest *rests;
    const void *w; int64_t w_ld;
    void *out;                           // [rows,K]
};
hipError_t launch_vocab_add(const VocabAdd &p, hipStream_t s);

}  // namespace lrnnx
