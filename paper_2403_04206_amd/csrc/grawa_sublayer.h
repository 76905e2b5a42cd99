// Internal declarations of the feed-forward sublayer (layer norm, gated feed-forward block, dropout) of K workers, shared by its
// host API (grawa_sublayer.cpp) and its kernels (grawa_layernorm.hip, grawa_dropout.hip, grawa_ffn.hip).
#ifndef GRAWA_SUBLAYER_H
#define GRAWA_SUBLAYER_H

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "grawa.h"
#include "grawa_philox.h"

struct grawa_sublayer {
    int K, device;
    int64_t T;          // most tokens of a worker
    int64_t d, f;       // model width; inner width of the feed-forward block, 0: none
    int64_t dp, fp;     // rounded up to 64 elements: pitches of what the library lays out itself, so that a row's tiles are whole lines
    grawa_dtype_t dtype;
    grawa_act_t act;
    int planes;         // bfloat16 terms that a matrix element is held in: 1, or 3 for float32
    int norm_blocks;    // most blocks of a worker in the backward norm
    // one device allocation, carved up:
    char *ws;
    float *norm_part;                // [K][norm_blocks][2][d] sums of dweight and dbias
    char *x, *dy;                    // [planes][K][T][dp] copies of x and dy where they cannot be read in place
    char *wg, *wu, *wd;              // the same of the matrices, [planes][K][f][dp] and [planes][K][d][fp]
    char *h, *dg, *du;               // [planes][K][T][fp]
    float *part;                     // sums of a product split over its long axis
    int64_t part_floats;
};

// [K][T][width] elements behind a pointer: worker k's row t starts at p + k * worker + t * row elements.
struct GrawaRows {
    char *p;
    int64_t worker, row;
};

// K matrices, or K vectors, each without gaps, `worker` elements apart.
struct GrawaMat {
    char *p;
    int64_t worker;
};

static inline int64_t grawa_round64(int64_t n) { return (n + 63) & ~(int64_t)63; }

static inline int64_t grawa_round16(int64_t n) { return (n + 15) & ~(int64_t)15; }

constexpr int GRAWA_FEW = 64; // tokens of a worker up to which a forward pass may take the kernels of grawa_few.h

// The buffer that a training forward leaves to its backward: gate and up before the activation, in fragments of 16 x 16; then
// their product in bfloat16 planes, [planes][K][T][fp]; then with float32, unless the tokens are few, the planes of x and of the
// three matrices, [3][K][T][dp], 2 x [3][K][f][dp], [3][K][d][fp].  All parts are multiples of 16 bytes.
static inline int64_t grawa_kept_bytes(const grawa_sublayer *s) { return s->planes == 1 ? 6 : 8; } // of a gate and an up, see grawa_ffn.hip
static inline int64_t grawa_save_bytes_own(const grawa_sublayer *s, int64_t T)
{
    return (int64_t)s->K * (grawa_round16(T) * grawa_round16(s->f) * grawa_kept_bytes(s) + T * s->fp * 2 * s->planes);
}
static inline bool grawa_keeps_copies(const grawa_sublayer *s, int64_t T) { return s->planes == 3 && T > GRAWA_FEW; }
static inline int64_t grawa_save_bytes(const grawa_sublayer *s, int64_t T)
{
    return grawa_save_bytes_own(s, T) + (grawa_keeps_copies(s, T) ? 6 * (int64_t)s->K * (T * s->dp + 2 * s->f * s->dp + s->d * s->fp) : 0);
}

hipError_t grawa_launch_layer_norm(const grawa_sublayer *s, int64_t T, GrawaRows x, GrawaMat w, GrawaMat b, float eps, GrawaRows y,
                                   float *stats, hipStream_t st);
hipError_t grawa_launch_layer_norm_backward(const grawa_sublayer *s, int64_t T, GrawaRows dy, GrawaRows x, GrawaMat w, const float *stats,
                                            GrawaRows add, GrawaRows dx, GrawaMat dw, GrawaMat db, int accumulate, hipStream_t st);
int grawa_norm_blocks(int K, int64_t T, int64_t d);
hipError_t grawa_launch_dropout(int K, int64_t T, int64_t d, grawa_dtype_t dtype, GrawaRows x, GrawaRows residual, GrawaDrop drop,
                                GrawaRows y, hipStream_t st);
int64_t grawa_ffn_part_floats(const grawa_sublayer *s);
hipError_t grawa_launch_ffn(const grawa_sublayer *s, int64_t T, GrawaRows x, GrawaMat wg, GrawaMat wu, GrawaMat wd, GrawaRows residual,
                            GrawaDrop drop, GrawaRows y, char *save, hipStream_t st);
hipError_t grawa_launch_ffn_backward(const grawa_sublayer *s, int64_t T, GrawaRows dy, GrawaRows x, GrawaMat wg, GrawaMat wu, GrawaMat wd,
                                     const char *save, GrawaRows dx, GrawaMat dwg, GrawaMat dwu, GrawaMat dwd, int accumulate,
                                     hipStream_t st);

#endif
