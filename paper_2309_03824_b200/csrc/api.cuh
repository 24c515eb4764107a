// What the files of entry points share: argument checks, the path in force and the debug mode.
#pragma once
#include "common.cuh"

namespace lrd {

lrd_status_t check_arch();
bool elem_aligned(const void* p, int dtype);
lrd_status_t check_ws(const void* ws, size_t have, size_t need);
int current_path();                                          // lrd_set_path's (an lrd_path_t)
// In the debug mode (LRD_DEBUG): waits for the call's work and returns what went wrong in it; else `st`.
lrd_status_t debug_checked(lrd_status_t st, void* cuda_stream);

#define LRD_TRY(expr)                          \
    do {                                       \
        lrd_status_t st__ = (expr);            \
        if (st__ != LRD_OK) return st__;       \
    } while (0)

}  // namespace lrd
