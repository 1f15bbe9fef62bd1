// Internal declarations of what surrounds an encoder's layers in training
// (layer norm, embedding table, dropout, cross entropy): host launchers.
#pragma once

#include "encoder.h"

namespace gpic {

// --------------------------------------------------------------- norm.hip
struct Norm {
    int64_t n, k, ldx, ldy;    // ldy: of Y (backward: of dY)
    float eps;
    int dtype;
};
size_t norm_ws(const Norm &p);             // of the backward pass
hipError_t run_norm(const Norm &p, const void *X, const void *w, const void *b, void *Y,
                    float *stats, hipStream_t st);
hipError_t run_norm_backward(const Norm &p, const void *dY, const void *X, const void *w,
                             const float *stats, void *dX, void *dW, void *db, void *ws,
                             hipStream_t st);

// ------------------------------------------------------------ dropout.hip
struct Dropout {
    int64_t n, m, ldx, ldr, ldy;
    uint64_t seed, offset;
    uint32_t limit;            // of 2^16: a value stays from here on
    int dtype;
};
hipError_t run_dropout(const Dropout &p, const void *X, const void *R, const int64_t *step,
                       void *Y, hipStream_t st);

// ---------------------------------------------------------- embedding.hip
struct Embedding {
    int64_t n, k, rows, ldt, ldy;
    float scale;
    int dtype;
    bool wide;                 // 64-bit ids
    bool accumulate;
};
size_t embedding_ws(const Embedding &p);   // of the backward pass
// Whether every launch of the backward pass stays below a grid's 2^32 threads.
bool embedding_fits(const Embedding &p);
hipError_t run_embedding(const Embedding &p, const void *ids, const void *T, void *Y,
                         hipStream_t st);
hipError_t run_embedding_backward(const Embedding &p, const void *dY, const void *ids, void *dT,
                                  void *ws, hipStream_t st);

// ---------------------------------------------------------- loss_thin.hip
// Gradients of up to kThinRows rows from D [n][v] and a contiguous X, both float32
// whatever the matrices' type; part: thin_ws bytes.
constexpr int64_t kThinRows = 64;
size_t thin_ws(int64_t n, int64_t k, int64_t v);
hipError_t run_thin_gradients(const float *D, const float *X, const void *W, int64_t n, int64_t k,
                              int64_t v, int64_t ldw, int dtype, void *dX, void *dW, void *db,
                              float *part, hipStream_t st);

// --------------------------------------------------------------- loss.hip
struct Loss {
    int64_t n, k, v, ldx, ldw;
    int dtype;
    bool wide;                 // 64-bit targets
    bool aligned16;            // X and W start on 16 bytes
};
size_t loss_ws(const Loss &p, bool backward);
// Whether every launch of a call stays below a grid's 2^32 threads.
bool loss_fits(const Loss &p, bool backward);
hipError_t run_loss(const Loss &p, const void *X, const void *W, const void *bias,
                    const void *targets, float *loss, float *lse, void *ws, hipStream_t st);
hipError_t run_loss_backward(const Loss &p, const float *dloss, const void *X, const void *W,
                             const void *bias, const void *targets, const float *loss,
                             const float *lse, void *dX, void *dW, void *db, void *ws,
                             hipStream_t st);

} // namespace gpic
