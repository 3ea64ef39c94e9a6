/* The library's functions that csrc/sdl_training.c calls, for a run of it on the CPU: each reads the views and numbers that it is told of. */
#include "sdl.h"

static int64_t read_view(const sdl_view_t* v) { return (int64_t)(uintptr_t)v->data ^ v->stride_batch ^ v->stride_token ^ v->stride_head; }
static int some(int64_t x) { return x == 1; }

int sdl_embedding(const void* table, int64_t stride, uint32_t vocab, uint32_t width, sdl_dtype_t td, const void* tokens, sdl_index_t index, uint32_t b, uint32_t t,
                  float scale, const sdl_view_t* out, sdl_dtype_t d, void* stream)
{ return some(read_view(out) ^ stride); }
int sdl_embedding_backward(const sdl_view_t* d_out, sdl_dtype_t d, const void* tokens, sdl_index_t index, uint32_t b, uint32_t t, float scale, void* d_table,
                           int64_t stride, uint32_t vocab, uint32_t width, sdl_dtype_t td, void* space, size_t bytes, void* stream)
{ return some(read_view(d_out) ^ stride); }
int sdl_cross_entropy(const sdl_view_t* x, uint32_t b, uint32_t t, uint32_t vocab, sdl_dtype_t d, const void* targets, sdl_index_t index, float smoothing, float z,
                      float* loss, float* lse, const float* d_loss, const sdl_view_t* d_x, void* stream)
{ return some(read_view(x) ^ (d_x ? read_view(d_x) : 0)); }
int sdl_cross_entropy_backward(const sdl_view_t* x, uint32_t b, uint32_t t, uint32_t vocab, sdl_dtype_t d, const void* targets, sdl_index_t index, float smoothing, float z,
                               const float* lse, const float* d_loss, const sdl_view_t* d_x, void* stream)
{ return some(read_view(x) ^ (d_x ? read_view(d_x) : 0)); }
int sdl_orthogonalize(const sdl_view_t* x, uint32_t b, uint32_t r, uint32_t c, sdl_dtype_t d, const float* coefficients, uint32_t steps, float eps, float scale,
                      const sdl_view_t* out, sdl_dtype_t od, void* space, size_t bytes, void* stream)
{
    float sum = 0;
    for (uint32_t i = 0; i < 3 * steps; ++i) sum += coefficients[i];
    return some(read_view(x) ^ read_view(out) ^ (sum == 1.0f));
}
