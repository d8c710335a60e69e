// Strided tensors [batch, heads, rows, d] of the C ABI: their checks on the host and what a kernel takes of them.
#pragma once
#include "common.h"

namespace dfs {

// A dfs_view as kernels take it: strides in bytes, 0 along axes of one entry.
struct View {
  char* data;
  int64_t batch, head, row;
  __device__ __forceinline__ char* at(int64_t b, int64_t h, int64_t r) const { return data + b * batch + h * head + r * row; }
};

// Checks a view of batch x heads x rows rows of d elements and fills `out`.
inline int check_view(const char* call, const char* name, const dfs_view* v, int dtype, int64_t batch, int64_t heads, int64_t rows, int d,
                      bool output, View* out) {
  if (!v) return fail(DFS_EINVAL, "%s: %s is NULL", call, name);
  *out = View{};
  if (batch == 0 || heads == 0 || rows == 0) return DFS_OK;              // no memory, wherever it points
  out->data = static_cast<char*>(v->data);
  if (!v->data) return fail(DFS_EINVAL, "%s: %s has no memory", call, name);
  const int e = elem_size(dtype);
  const int64_t n[3] = {batch, heads, rows}, s[3] = {v->batch, v->head, v->row};
  int64_t used[3];
  for (int i = 0; i < 3; ++i) {
    used[i] = n[i] > 1 ? s[i] : 0;
    if (used[i] < 0 || used[i] > (int64_t(1) << 44) / n[i]) return fail(DFS_EINVAL, "%s: %s has a stride of %lld", call, name, (long long)s[i]);
    if (used[i] * e % 16) return fail(DFS_EINVAL, "%s: rows of %s must start on 16-byte boundaries (stride %lld)", call, name, (long long)s[i]);
  }
  if (misaligned(16, {v->data})) return fail(DFS_EINVAL, "%s: %s must be 16-byte aligned", call, name);
  if (output) {                                      // axes from the closest entries to the widest: none may reach into the next
    int order[3] = {0, 1, 2};
    for (int i = 0; i < 3; ++i)
      for (int j = i + 1; j < 3; ++j)
        if (used[order[j]] < used[order[i]]) { const int t = order[i]; order[i] = order[j]; order[j] = t; }
    int64_t span = d;
    for (int i : order) {
      if (n[i] == 1) continue;
      if (used[i] < span) return fail(DFS_EINVAL, "%s: rows of %s overlap", call, name);
      span += used[i] * (n[i] - 1);
    }
  }
  out->batch = used[0] * e;
  out->head = used[1] * e;
  out->row = used[2] * e;
  return DFS_OK;
}

// Refuses outputs that begin where another tensor of the call does.  (Overlap in general is the caller's to avoid: parts of one buffer interleave.)
struct Named { const char* name; const View* v; };
inline int check_apart(const char* call, std::initializer_list<Named> outputs, std::initializer_list<Named> inputs) {
  for (const Named& o : outputs) {
    if (!o.v->data) continue;
    for (const auto* list : {&outputs, &inputs})
      for (const Named& x : *list)
        if (x.v != o.v && x.v->data == o.v->data) return fail(DFS_EINVAL, "%s: %s and %s are the same memory", call, o.name, x.name);
  }
  return DFS_OK;
}
// Whether an output is its own input with other strides.
inline bool moved(const View& in, const View& out) {
  return in.data && in.data == out.data && (in.batch != out.batch || in.head != out.head || in.row != out.row);
}

}  // namespace dfs
