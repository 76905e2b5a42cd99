// Internal declarations of the attention of K workers (norms of heads with rotation, windowed attention, learned bias by buckets),
// shared by its host API (grawa_attention.cpp) and its kernels (grawa_heads.hip, grawa_attend.hip, grawa_attend_back.hip).
#ifndef GRAWA_ATTENTION_H
#define GRAWA_ATTENTION_H

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "grawa.h"
#include "grawa_sublayer.h"

struct grawa_attention_plan {
    int K, device;
    int64_t N, S;           // most sequences of a worker, most tokens of a sequence
    int H, G, D;            // heads of queries, of keys and values; width of a head
    grawa_dtype_t dtype;
    float scale;
    int window, sinks;      // window: GRAWA_NO_WINDOW where there is none
    int rotary, interleaved;
    int buckets, distances; // 0: no bias
    // one device allocation, carved up:
    char *ws;
    double *turns;          // [rotary / 2] turns a position
    int *bucket_of;         // [distances]
    float *rows;            // two of [K N][H][S rounded up to 256]: log2 of the sum of exponentials, -do . o
    float *norm_part;       // [K][norm_blocks][2][D] sums of the weights' gradients
    float *bias_part;       // [K N][H][blocks of queries][buckets]
    float *part;            // outputs and sums of blocks that share them
    int64_t part_floats;
    int norm_blocks;
};

constexpr int GRAWA_NO_WINDOW = 1 << 30;

// Queries of a block that forms dq and sums for dbias.
constexpr int grawa_dq_queries(bool bf16) { return bf16 ? 128 : 64; }

// Rows of D elements behind a pointer, strides in bytes.
struct GrawaHeads {
    char *p;
    int64_t worker, seq, token, head;
};

// What a call of the attention has; the backward pass has all of it, the forward pass q, k, v and o.
struct GrawaAttend {
    GrawaHeads q, k, v, o, go, dq, dk, dv;
    const int *starts, *lengths; // [K][N] or null
    float *lse;                  // [K][N][H][Sq] or null
    GrawaMat bias, dbias;        // [H][buckets] of every worker
    const int *bucket_of;
    float *row_lse, *row_dot;    // [K N][H][row_pitch]: log2 of the sum of exponentials (infinity: the row counts for nothing), -do . o
    float *bias_part, *part;
    int64_t row_pitch;           // Sq rounded up to 256
    int K, N, H, G, D, Sq, Sk, share; // share = H / G
    int window, sinks, buckets, distances;
    float scale;
    int blocks, splits;          // blocks of queries of a head; blocks that share one's keys
    int accumulate, by_xcd;
    // dk and dv: blocks of keys; the first of them, which all queries see, and how many blocks share their queries; places in `part` for
    // a group's blocks that share
    int key_blocks, sink_blocks, sink_splits, slots;
};

static inline int64_t grawa_round256(int64_t n) { return (n + 255) & ~(int64_t)255; }
static inline int grawa_padded_width(int D) { return D <= 64 ? 64 : 128; }

int grawa_head_norm_blocks(const grawa_attention_plan *s);

hipError_t grawa_launch_head_norm(const grawa_attention_plan *s, int64_t N, int64_t S, GrawaHeads q, GrawaHeads k, GrawaMat qw, GrawaMat kw, float eps,
                                  const int *starts, GrawaHeads qo, GrawaHeads ko, hipStream_t st);
hipError_t grawa_launch_head_norm_backward(const grawa_attention_plan *s, int64_t N, int64_t S, GrawaHeads dqo, GrawaHeads dko, GrawaHeads q, GrawaHeads k,
                                           GrawaMat qw, GrawaMat kw, float eps, const int *starts, GrawaHeads dq, GrawaHeads dk, GrawaMat dqw,
                                           GrawaMat dkw, int accumulate, hipStream_t st);
hipError_t grawa_launch_attend(const grawa_attention_plan *s, GrawaAttend a, hipStream_t st);
hipError_t grawa_launch_attend_backward(const grawa_attention_plan *s, GrawaAttend a, hipStream_t st);

#endif
