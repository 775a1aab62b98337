// A context of the library and what every entry point does with it: the workspace's arena, error messages, kernel timing.
#pragma once

#include <cstdarg>
#include <cstdio>
#include <map>
#include <string>
#include <vector>

#include "../../include/gmeta.h"
#include "gm_internal.h"

struct Arena {
    char* base = nullptr;
    size_t cap = 0, off = 0;
    bool overflow = false;
    template <typename T>
    T* get(size_t n) {
        const size_t bytes = (n * sizeof(T) + 255) / 256 * 256;
        if (off + bytes > cap) {
            overflow = true;
            off += bytes;
            return nullptr;
        }
        T* p = base ? reinterpret_cast<T*>(base + off) : nullptr;
        off += bytes;
        return p;
    }
};

struct ProfEntry {
    int64_t launches = 0;
    double ms = 0, bytes = 0, flops = 0;
};
struct ProfPending {
    std::string name;
    hipEvent_t e0, e1;
    double bytes, flops;
};

struct gm_ctx {
    int F = 0, D = 0, n_dense = 0, L = 0, mlp_dtype = 0;
    std::vector<int64_t> rows, field_base;
    std::vector<int> dims, ld;
    std::vector<int64_t> offW, offb;    // fp32 theta layout
    std::vector<int64_t> offWb;         // bf16 theta layout: W_l as stored ([d_in, d_out]), l = 1..L-1
    int64_t n_theta = 0, n_theta_b = 0;
    int FD = 0, row_pad = 1;
    int device = 0;
    hipStream_t stream = nullptr;
    char* ws = nullptr;
    size_t ws_bytes = 0;
    size_t persistent = 0;
    int64_t* d_field_base = nullptr;
    u32* d_status = nullptr;
    u32* d_status_side = nullptr;   // status words of the work on the side stream
    // The ordering of the lookups by row depends on the indices only: it runs on a stream of its own beside the dense
    // computation (same priority) and is joined before the segment reduction.
    hipStream_t side = nullptr;
    hipEvent_t ev_side = nullptr, ev_main = nullptr, ev_go = nullptr;
    // The pair-count matrices depend on the indices only and are first read by the first row hop: counting them on the
    // side stream lets the prefetch and the first forward / backward pass (bound by memory traffic) run beside a kernel
    // that is bound by latency and instruction issue.
    hipEvent_t ev_pairs_go = nullptr, ev_pairs = nullptr;
    int overlap_pairs = 0;
    int overlap_sort = 0;   // measured: 1-1.5 % (both streams contend for the same memory system), so off unless asked for
    std::string err;
    int pair_tile_rows = 0;
    int adapt_rows = 1;   // 0: the inner loop adapts the dense parameters only (embedding rows are read, not updated)
    int gemm_tile_n = 0;
    int wgrad_wide = 1;      // weight gradients over runs of tasks in 256 x 256 tiles where the shape allows
    int chain_factors = 0;   // the second-order chain's direction on a task's hidden layers: 0 by size, 1 matrices, 2 factors where they can be (see factor_rows)
    int theta_from_meta = 1; // bf16, several inner steps: a step's weights from theta and all steps' gradients, in first order where tasks are small
    int coarse_groups = 0;   // runs of tasks for the products only summed over tasks (0: chosen by shape)
    int n_cus = 256;
    int row_path = 0;   // task-local row arithmetic: 0 = choose per wave, 1 = sparse two-hop kernel, 2 = pair-count matrices
    int sort_fields = 1; // with index_path's row order: 1 = the keys are laid out field after field and every field's range sorted by row alone (fewer radix passes), 0 = one sort on (field, row)
    int index_path = 0; // per-(task, field) dictionaries: 0 = choose per wave, 1 = sorted per (task, field) in LDS, 2 = read off the wave's (task, field, row) order
    int max_wave_tasks = 0;   // 0: as many tasks per wave as the workspace holds
    char* static_scratch = nullptr;   // this device's copy of the static scratch array (gm_meta_step_static)
    // the calls on histories (gm_seq_*)
    int wait = 1;                     // 0: they return once enqueued, and gm_wait says what the device found
    u32* seq_status = nullptr;        // pinned host words (SEQ_*) that their kernels set
    // optional kernel timing
    bool prof_on = false;
    std::vector<ProfPending> prof_pending;
    std::vector<hipEvent_t> prof_free;
    std::map<std::string, ProfEntry> prof;
    std::string prof_text;
};

static inline int fail(gm_ctx* c, int code, const char* fmt, ...) {
    char buf[512];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(buf, sizeof buf, fmt, ap);
    va_end(ap);
    if (c) c->err = buf;
    return code;
}

#define HIPCHK(c, call)                                                                            \
    do {                                                                                           \
        hipError_t e_ = (call);                                                                    \
        if (e_ != hipSuccess) return fail(c, GM_ERR_HIP, "%s: %s", #call, hipGetErrorString(e_)); \
    } while (0)

// Brackets the launches issued during its lifetime with two events on the context's stream.
struct Prof {
    gm_ctx* c;
    ProfPending p;
    bool on;
    hipStream_t st;
    Prof(gm_ctx* c_, const char* name, double bytes, double flops, hipStream_t st_ = nullptr, bool use_st = false)
        : c(c_), on(c_->prof_on), st(use_st ? st_ : c_->stream) {
        if (!on) return;
        p.name = name;
        p.bytes = bytes;
        p.flops = flops;
        for (hipEvent_t* e : {&p.e0, &p.e1}) {
            if (!c->prof_free.empty()) {
                *e = c->prof_free.back();
                c->prof_free.pop_back();
            } else if (hipEventCreate(e) != hipSuccess) {
                on = false;
                return;
            }
        }
        (void)hipEventRecord(p.e0, st);
    }
    ~Prof() {
        if (!on) return;
        (void)hipEventRecord(p.e1, st);
        c->prof_pending.push_back(p);
    }
};

static inline void prof_drain(gm_ctx* c) {  // after the stream has been synchronised
    for (ProfPending& p : c->prof_pending) {
        float ms = 0.f;
        if (hipEventElapsedTime(&ms, p.e0, p.e1) == hipSuccess) {
            ProfEntry& e = c->prof[p.name];
            e.launches += 1;
            e.ms += ms;
            e.bytes += p.bytes;
            e.flops += p.flops;
        }
        c->prof_free.push_back(p.e0);
        c->prof_free.push_back(p.e1);
    }
    c->prof_pending.clear();
}
