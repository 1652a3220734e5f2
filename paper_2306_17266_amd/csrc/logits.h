// Operators on rows of logits (row_order.hip, distill.hip): what their launchers take.
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

// Rows are read in pieces of 16 bytes.  A row that fits the registers of a workgroup is one workgroup's; longer rows, and long ones
// where there are few, are read in parts, a workgroup each, whose results a workgroup per row joins.
constexpr int LOGITS_PART_PIECES = 2048;
constexpr int LOGITS_SMALL_PART_PIECES = 512;  // where few rows would leave compute units without a part
constexpr int LOGITS_MOST_SMALL_PARTS = 1024;  // of all rows
constexpr int LOGITS_MOST_PARTS = LOGITS_MAX_CLASSES / (4 * LOGITS_PART_PIECES) + 1;  // of a row
inline int logits_pieces(int n, bool bf16) {  // (a row may start inside its first piece)
    const int per = bf16 ? 8 : 4;
    return (n + 2 * per - 2) / per;
}
inline int logits_parts(int pieces, int part_pieces) { return (pieces + part_pieces - 1) / part_pieces; }
inline bool held_rows(const LogitRows &in) {
    const int pieces = logits_pieces(in.n, in.bf16);
    return pieces <= 1024 || (pieces <= 8192 && in.rows >= 192);
}
inline bool small_parts(const LogitRows &in) {
    const int parts = logits_parts(logits_pieces(in.n, in.bf16), LOGITS_SMALL_PART_PIECES);
    return parts <= LOGITS_MOST_PARTS && (long)in.rows * parts <= LOGITS_MOST_SMALL_PARTS;
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
