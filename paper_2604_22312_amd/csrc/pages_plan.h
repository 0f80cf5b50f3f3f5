// pages_plan.h -- argument checks, workspace and launch shapes of the page
// step. Plain C++ with no HIP dependency, so the library and a sanitizer build
// on the CPU compile the same code.
#ifndef GVR_PAGES_PLAN_H
#define GVR_PAGES_PLAN_H

#include <stddef.h>
#include <stdint.h>

#include "gvr_pages.h"

namespace gvr_pages {

constexpr int64_t kMaxCount = ((int64_t)1 << 31) - 16;
constexpr int kMaxRequests = 1 << 20;
constexpr int kThreads = 1024;     // of the workgroup that adds up the requests
constexpr int kTokenThreads = 256;
constexpr int kArrays = 6;         // numbers of a request that the step's parts hand over
constexpr int kHeader = 4;         // 64-bit totals ahead of them

inline int64_t workspace_bytes(int requests) {
    if (requests < 0 || requests > kMaxRequests) return -1;
    return 8 * kHeader + (int64_t)kArrays * 4 * ((requests + 1 + 3) & ~3);
}

inline gvr_status check(const gvr_page_pool* p, const gvr_page_step_args* a, const void* ws, size_t ws_bytes) {
    if (!p || !a) return GVR_ERR_INVALID_ARG;
    if (p->requests < 0 || p->width < 0 || p->pages < 0 || a->T < 0 || (a->dense && a->ld < 0)) return GVR_ERR_INVALID_ARG;
    if (p->page_size < 1 || p->page_size > 65536 || (p->page_size & (p->page_size - 1))) return GVR_ERR_INVALID_ARG;
    if (p->requests > kMaxRequests || p->width > kMaxCount || p->width * p->page_size > kMaxCount ||
        p->pages > kMaxCount || a->T > kMaxCount || (a->dense && a->ld > kMaxCount))
        return GVR_ERR_TOO_LONG;
    if (((uintptr_t)p->block_table | (uintptr_t)p->ctx_len | (uintptr_t)p->free_pages | (uintptr_t)p->free_count |
         (uintptr_t)a->new_len | (uintptr_t)a->keep | (uintptr_t)a->q_start | (uintptr_t)a->taken |
         (uintptr_t)a->positions | (uintptr_t)a->row_len) & 3)
        return GVR_ERR_INVALID_ARG;
    if (((uintptr_t)a->slots | (uintptr_t)a->dense) & 7) return GVR_ERR_INVALID_ARG;
    if (p->requests > 0 && (!p->ctx_len || !p->free_count || !a->new_len || (p->width > 0 && !p->block_table) ||
                            (p->pages > 0 && !p->free_pages)))
        return GVR_ERR_INVALID_ARG;
    if (!ws || ((uintptr_t)ws & 15)) return GVR_ERR_INVALID_ARG;
    if (ws_bytes < (size_t)workspace_bytes(p->requests)) return GVR_ERR_WORKSPACE;
    return GVR_OK;
}

// One workgroup does the whole step where it has at most this many requests and
// rows, else it adds up the requests and two more kernels move the pages and fill
// the rows (one workgroup and three kernels: 64 requests and 128 rows 4.4 us and 9.5, 1024
// and 2048 9.1 and 11.5, 300 and 4096 10.5 both, 300 and 16384 22.6 and 10.5).
constexpr int kSmallRequests = 1024, kSmallRows = 2048;
inline bool small_step(int requests, int64_t T) { return requests <= kSmallRequests && T <= kSmallRows; }

}  // namespace gvr_pages

#endif  // GVR_PAGES_PLAN_H
