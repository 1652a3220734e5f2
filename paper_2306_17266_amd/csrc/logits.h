// Operators on rows of logits (sample.hip, top_logits.hip, distill.hip): what their launchers take.
//
// The order of a row: value descending, index ascending; a NaN counts as -inf, and what is -inf belongs to no order.
// The weight of a logit: exp((z - max z) / T).
#pragma once

#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>

namespace sushi {

constexpr int LOGITS_MAX_CLASSES = 1 << 20;  // (so that sums of weights fit 64-bit fixed point, and indexes of 16-byte pieces an int)
constexpr int LOGITS_MAX_TOP = 1024;

struct LogitRows {
    const void *x;  // float32 or bf16
    long stride;    // elements from row to row
    int rows, n;    // n logits in a row
    bool bf16;
};

struct SampleArgs {
    LogitRows in;
    const float *uniform;      // [rows]
    const float *temperature;  // [rows] or null (1); this and the next three
    const int32_t *top_k;      // (null, <= 0: all)
    const float *top_p;        // (null, >= 1, NaN: all)
    const float *min_p;        // (null, <= 0, NaN: all)
    int32_t *classes;          // [rows]
    float *log_prob;           // [rows] or null
};

struct TopArgs {
    LogitRows in;
    int k;
    float temperature;  // of `rest`
    float *values;      // [rows][k]
    int32_t *classes;   // [rows][k]
    float *rest;        // [rows] or null
};

struct DistillArgs {
    LogitRows in;
    const float *values;     // [rows][k]
    const int32_t *classes;  // [rows][k]
    const float *rest;       // [rows] or null (0)
    const float *weight;     // [rows] or null (1)
    int k;
    float temperature;
    float *loss;       // [rows] or null
    void *grad;        // type of the logits, or null
    long grad_stride;  // elements from row to row
};

// Rows are read in pieces of 16 bytes.  A row that fits the registers of a workgroup is one workgroup's, who reads it once; longer
// rows, and long ones where there are few, are read in parts, a workgroup each, whose results a workgroup per row joins.
constexpr int LOGITS_PART_PIECES = 2048;
constexpr int LOGITS_SMALL_PART_PIECES = 512;  // where few rows would leave compute units without a part
constexpr int LOGITS_MOST_SMALL_PARTS = 1024;  // of all rows
constexpr int LOGITS_MOST_PARTS = LOGITS_MAX_CLASSES / (4 * LOGITS_PART_PIECES) + 1;  // of a row
inline int logits_pieces(int n, bool bf16) {  // (a row may start inside its first piece)
    const int per = bf16 ? 8 : 4;
    return (n + 2 * per - 2) / per;
}
inline int logits_parts(int pieces, int part_pieces) { return (pieces + part_pieces - 1) / part_pieces; }

// Whether rows are held.  Measured, in parts against held, in us:
//                                                   rows = 16                    rows = 256
//   float32 x  16000: sample, its plain form      25.1 - 17.8, 10.0 - 11.1     34.4 - 18.1, 14.2 - 11.4
//                     top, loss, loss + gradient  18.7 - 11.5, 10.2 - 7.5, 14.3 - 8.6
//   float32 x  32000: sample, its plain form      25.4 - 20.7,  9.8 - 16.5     42.7 - 23.5, 19.3 - 18.0
//                     top, loss, loss + gradient  19.1 - 14.1, 10.1 - 9.8, 14.0 - 11.9
//   bf16    x  32000: sample, its plain form      26.7 - 27.9, 10.0 - 18.1     41.7 - 27.0, 20.1 - 18.5
//   bf16    x  64000: sample, its plain form      28.0 - 31.5, 10.4 - 27.9     55.2 - 33.1, 27.7 - 29.1
//                     top, loss, loss + gradient  21.4 - 21.1, 10.1 - 14.6, 13.9 - 18.4 (37.9 - 23.8, 20.8 - 15.9, 32.6 - 23.5)
// The plain form of sampling (no top_k, top_p, min_p) computes an exponential for each logit and little else, and gains by more
// compute units sooner.
constexpr int LOGITS_HELD_PIECES = 8192, LOGITS_HELD_PLAIN_PIECES = 4096;
constexpr int LOGITS_HELD_FEW = 32000, LOGITS_HELD_PLAIN_FEW = 16000, LOGITS_MANY_ROWS = 192;
inline bool held_rows(const LogitRows &in) {
    return logits_pieces(in.n, in.bf16) <= LOGITS_HELD_PIECES && (in.n <= LOGITS_HELD_FEW || in.rows >= LOGITS_MANY_ROWS);
}
inline bool held_plain_rows(const LogitRows &in) {
    return logits_pieces(in.n, in.bf16) <= LOGITS_HELD_PLAIN_PIECES && (in.n <= LOGITS_HELD_PLAIN_FEW || in.rows >= LOGITS_MANY_ROWS);
}
// Whether the parts are small: as long as they are few, of all rows and of each (what joins the row's parts takes longer with more).
// Measured, large parts against small ones, in us: 1 x 131071 in bf16 loss 11.8 - 10.2, loss and gradient 18.3 - 14.3, plain
// sampling 16.9 - 10.2; sampling with a histogram from each part 33.5 - 30.8 there (33 small parts), 30.6 - 33.5 in float32 (64),
// and 30.5 - 39.1 for 1 x 250007 in float32 (123).
constexpr int LOGITS_FEW_PARTS = 48;
inline bool small_parts(const LogitRows &in, int most) {
    const int parts = logits_parts(logits_pieces(in.n, in.bf16), LOGITS_SMALL_PART_PIECES);
    return parts <= most && (long)in.rows * parts <= LOGITS_MOST_SMALL_PARTS;
}
// Rows that go out in one launch in parts (for both types alike): what a call needs of the workspace stays bounded.
inline long rows_of_slice(int n) {
    const long rows = 8192 / logits_parts(logits_pieces(n, false), LOGITS_PART_PIECES);
    return rows > 1 ? rows : 1;
}
// Of the workspace: bytes that an operator needs for each part, and for each row.
size_t top_logits_part_bytes();
size_t sample_part_bytes();
size_t sample_row_bytes();
size_t distill_part_bytes();
size_t distill_row_bytes();

// Bytes of scratch memory that every operator gets by with on rows of n logits.
size_t logits_workspace_bytes(int rows, int n);

// Return hipSuccess or the launch error.  ws: logits_workspace_bytes() bytes, 16-byte aligned.
hipError_t launch_sample(const SampleArgs &a, void *ws, hipStream_t s);
hipError_t launch_top_logits(const TopArgs &a, void *ws, hipStream_t s);
hipError_t launch_distill(const DistillArgs &a, void *ws, hipStream_t s);

}  // namespace sushi
