// [batch][tokens][heads][dim] tensors of the operators on token sequences.
#pragma once

#include <stdint.h>

#include "layout.h"

namespace elasto {

struct View {  // strides in bytes
  char* p;
  int64_t sb, st, sh;
};

inline bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

// *v from t, for elements of es bytes; an axis of no elements needs no tensor.
// False, with the thread's error message set, where t is refused.
inline bool take_view(const char* op, const char* name, const elasto_heads_t* t, int64_t batch,
                      int64_t tokens, int64_t heads, int64_t dim, int es, bool written, View* v) {
  *v = View{nullptr, 0, 0, 0};
  if (batch == 0 || tokens == 0 || heads == 0) return true;
  if (!t || !t->data) return fail(ELASTO_ERR_INVALID_ARG, "%s: %s is NULL", op, name), false;
  if (!aligned(t->data, 16) || t->batch_stride * es % 16 || t->token_stride * es % 16 ||
      t->head_stride * es % 16)
    return fail(ELASTO_ERR_INVALID_ARG, "%s: %s and its strides must be multiples of 16 bytes", op, name), false;
  if (t->batch_stride < 0 || t->token_stride < 0 || t->head_stride < 0)
    return fail(ELASTO_ERR_INVALID_ARG, "%s: %s has a negative stride", op, name), false;
  if (written && ((batch > 1 && t->batch_stride < dim) || (tokens > 1 && t->token_stride < dim) ||
                  (heads > 1 && t->head_stride < dim)))
    return fail(ELASTO_ERR_INVALID_ARG, "%s: rows of %s overlap", op, name), false;
  *v = View{static_cast<char*>(t->data), t->batch_stride * es, t->token_stride * es, t->head_stride * es};
  return true;
}

}  // namespace elasto
