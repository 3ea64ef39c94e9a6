/* The library's functions that csrc/sdl_operators.c calls, for a run of it on the CPU: each reads the views that it is told of. */
#include "sdl.h"

static int64_t read_view(const sdl_view_t* v) { return (int64_t)(uintptr_t)v->data ^ v->stride_batch ^ v->stride_token ^ v->stride_head; }
static int some(int64_t x) { return x == 1; }

int sdl_layer_norm(const sdl_view_t* x, uint32_t b, uint32_t t, uint32_t h, uint32_t w, sdl_dtype_t d, const void* weight, const void* bias, sdl_dtype_t pd,
                   float eps, const sdl_view_t* y, float* mean, float* rstd, void* stream)
{ return some(read_view(x) ^ read_view(y)); }
int sdl_layer_norm_backward(const sdl_view_t* dy, const sdl_view_t* x, uint32_t b, uint32_t t, uint32_t h, uint32_t w, sdl_dtype_t d, const void* weight,
                            sdl_dtype_t pd, const float* mean, const float* rstd, const sdl_view_t* dx, void* dweight, void* dbias, void* space, size_t bytes,
                            void* stream)
{ return some(read_view(dy) ^ read_view(x) ^ read_view(dx)); }
int sdl_rotary(const sdl_view_t* x, uint32_t b, uint32_t t, uint32_t h, uint32_t w, sdl_dtype_t d, uint32_t rot, sdl_rotary_layout_t layout,
               const int32_t* positions, int32_t first, const double* f, float scale, int inverse, const sdl_view_t* out, void* stream)
{ return some(read_view(x) ^ read_view(out)); }
int sdl_attention(const sdl_view_t* q, const sdl_view_t* k, const sdl_view_t* v, uint32_t b, uint32_t queries, uint32_t keys, uint32_t h, uint32_t g, uint32_t w,
                  sdl_dtype_t d, float scale, int causal, const int32_t* q_len, const int32_t* k_len, const sdl_view_t* out, float* lse, void* space, size_t bytes,
                  void* stream)
{ return some(read_view(q) ^ read_view(k) ^ read_view(v) ^ read_view(out)); }
int sdl_attention_backward(const sdl_view_t* d_out, const sdl_view_t* q, const sdl_view_t* k, const sdl_view_t* v, const sdl_view_t* out, const float* lse,
                           uint32_t b, uint32_t queries, uint32_t keys, uint32_t h, uint32_t g, uint32_t w, sdl_dtype_t d, float scale, int causal,
                           const int32_t* q_len, const int32_t* k_len, const sdl_view_t* dq, const sdl_view_t* dk, const sdl_view_t* dv, void* space, size_t bytes,
                           void* stream)
{ return some(read_view(d_out) ^ read_view(q) ^ read_view(k) ^ read_view(v) ^ read_view(out) ^ read_view(dq) ^ read_view(dk) ^ read_view(dv)); }
