// A gated linear recurrence over histories, channel by channel:
//   a_t = sigmoid(g_t),  h_t = a_t h_{t-1} + (1 - a_t) x_t
// A step is the map h -> A h + B; maps compose as (A2, B2) after (A1, B1) = (A2 A1, A2 B1 + B2), so that a run of steps may be
// combined in pieces: lanes hold pieces of SCAN_U steps, a wave combines its lanes' pieces, and where few histories are long the chunks
// of one history are combined by a launch of their own.
// The gradient runs from the last row to the first:
//   c_T = d last,  d_t = dh_t + c_{t+1},  dx_t = (1 - a_t) d_t,  dg_t = d_t (h_{t-1} - x_t) a_t (1 - a_t),  c_t = a_t d_t,  dh0 = c_0
// which is the same kind of recurrence in c.  All of it is held in fp32; 1 - a is computed as sigmoid(-g) (a close to one leaves
// nothing of 1 - a in the difference).
#include <algorithm>

#include "gm_internal.h"

// sigmoid(g) = 1 / (1 + e), sigmoid(-g) = e / (1 + e), e = exp(-g); e stays below 2^126, where the first is 0 beside anything (NaN goes through).
__device__ __forceinline__ void gate_of(float g, float& a, float& na) {
    const float e = __builtin_amdgcn_exp2f(__builtin_elementwise_minimum(-1.44269504088896f * g, 126.f));
    a = __builtin_amdgcn_rcpf(1.f + e);
    na = e * a;
}

enum { SCAN_WHOLE = 0, SCAN_AGG = 1, SCAN_APPLY = 2 };

// A wave takes one history (or chunk of one) and a block of CT * V channels; its 64 / CT lanes along the time axis hold U rows each.
// Bound: memory.  1,024 users of 64 to 512 events, 256 channels, bf16: 106 us (455 MB, 4.3 TB/s); the gradient of 4 of up to 40,000 events 80 us, two launches
// (23 + 57) of which the first reads two of the six arrays once more; 201 users of up to 243 events, 100 channels, fp32: the gradient 24 us, by then the latency of
// a history's eight tiles one after the other.
template <typename T, int V, int CT, int U, int DEPTH, bool GRAD, int MODE, bool STREAM>
__global__ __launch_bounds__(256) void seq_scan_kernel(SeqScanArgs a) {
    constexpr int TT = 64 / CT, TILE = TT * U;
    const int lane = threadIdx.x & 63, tr = lane / CT;
    const int cbs = (a.channels + CT * V - 1) / (CT * V);
    int64_t unit = (int64_t)workgroup() * 4 + (threadIdx.x >> 6);
    const int c = (int)(unit % cbs) * CT * V + (lane % CT) * V;
    unit /= cbs;
    const int v = MODE == SCAN_WHOLE ? 0 : (int)(unit % a.chunks);   // the chunk's number in the order of the recurrence
    const int64_t s = MODE == SCAN_WHOLE ? unit : unit / a.chunks;
    if (s >= a.v.n_seqs) return;
    const int64_t o0 = a.v.offsets[s], o1 = a.v.offsets[s + 1];
    if (!seq_inside(o0, o1, a.v.n_rows, a.v.longest) || (s == 0 && o0 != 0) || (s + 1 == a.v.n_seqs && o1 != a.v.n_rows)) {
        seq_flag(a.v.status, SEQ_BAD_OFFSETS);
        return;
    }
    const int64_t len = o1 - o0, first = MODE == SCAN_WHOLE ? 0 : v * a.chunk, left = len - first;
    if (MODE != SCAN_WHOLE && v > 0 && left <= 0) return;
    const int64_t n = MODE == SCAN_WHOLE ? len : min(left, a.chunk);   // steps of this wave
    const bool last_chunk = MODE == SCAN_WHOLE || left <= a.chunk;
    if (MODE == SCAN_AGG && last_chunk) return;                         // (nobody reads it)
    const bool on = c < a.channels;
    const int cc = on ? c : 0;   // (lanes past the last channel read the first ones and write nothing)
    // step i of the wave is row o0 + first + i, or counted from the end
    auto row = [&](int64_t i) { return GRAD ? o1 - 1 - (first + i) : o0 + first + i; };

    float carry[V];
    {
        const float* init = GRAD ? a.tail : a.start;
#pragma unroll
        for (int e = 0; e < V; ++e) carry[e] = MODE != SCAN_AGG && init ? init[s * a.channels + cc + e] : 0.f;
    }
    // combines the lanes' pieces along time: (A, B) becomes what lies in front of the lane's piece; returns the whole in (wa, wb)
    auto across = [&](float (&A)[V], float (&B)[V], float (&wa)[V], float (&wb)[V]) {
#pragma unroll
        for (int d = 1; d < TT; d *= 2)
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float pa = __shfl_up(A[e], d * CT), pb = __shfl_up(B[e], d * CT);
                if (tr >= d) {
                    B[e] = fmaf(A[e], pb, B[e]);
                    A[e] *= pa;
                }
            }
#pragma unroll
        for (int e = 0; e < V; ++e) {
            wa[e] = __shfl(A[e], 64 - CT + lane % CT);
            wb[e] = __shfl(B[e], 64 - CT + lane % CT);
            const float pa = __shfl_up(A[e], CT), pb = __shfl_up(B[e], CT);
            A[e] = tr ? pa : 1.f;
            B[e] = tr ? pb : 0.f;
        }
    };
    const int64_t plane = a.v.n_seqs * a.chunks * (int64_t)a.channels;
    if constexpr (MODE == SCAN_APPLY) {   // the chunks in front of this one
        if (v > 0) {
            float A[V], B[V], wa[V], wb[V];
#pragma unroll
            for (int e = 0; e < V; ++e) { A[e] = 1.f; B[e] = 0.f; }
            const int per = (v + TT - 1) / TT, lo = min(tr * per, v), hi = min(lo + per, v);
            const float* p = a.agg + (s * a.chunks + lo) * a.channels + cc;
            for (int i = lo; i < hi; ++i, p += a.channels)
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    B[e] = fmaf(p[e], B[e], p[plane + e]);
                    A[e] *= p[e];
                }
            across(A, B, wa, wb);
#pragma unroll
            for (int e = 0; e < V; ++e) carry[e] = fmaf(wa[e], carry[e], wb[e]);
        }
    }
    float total[V];   // SCAN_AGG: the product of all a
#pragma unroll
    for (int e = 0; e < V; ++e) total[e] = 1.f;

    typedef Pack<T, V> P;
    auto read_rows = [&](const T* p) { return STREAM && MODE != SCAN_AGG ? stream_in<P>(p) : *reinterpret_cast<const P*>(p); };
    auto write_rows = [&](T* p, const P& x) {
        if (STREAM) stream_out(p, x);
        else *reinterpret_cast<P*>(p) = x;
    };
    struct Tile { P x[U], g[U], h[U], d[U]; };
    auto load = [&](Tile& t, int64_t i0) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t i = i0 + tr * U + u, r = row(min(i, n - 1));
            t.g[u] = read_rows((const T*)a.gate + r * a.ldg + cc);
            if (!GRAD || MODE != SCAN_AGG) t.x[u] = read_rows((const T*)a.x + r * a.ldx + cc);
            if (GRAD) {
                t.d[u] = read_rows((const T*)a.dh + r * a.lddh + cc);
                if (MODE != SCAN_AGG && r > o0) t.h[u] = *reinterpret_cast<const P*>((const T*)a.h + (r - 1) * a.ldh + cc);
            }
        }
    };
    Tile ring[DEPTH];
#pragma unroll
    for (int d = 0; d < DEPTH; ++d)
        if (d * TILE < n) load(ring[d], d * TILE);
    auto tile = [&](Tile& t, int64_t i0) {
        float ca[U][V], cb[U][V], k1[U][V], k2[U][V];   // coefficients; the gradient's factors of d
        if (i0 + TILE > n) {   // rows behind the end: a = 1, and nothing is added
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (i0 + tr * U + u >= n) {
                    float inf[V], zero[V];
#pragma unroll
                    for (int e = 0; e < V; ++e) { inf[e] = INFINITY; zero[e] = 0.f; }
                    t.g[u].put(inf);
                    if (GRAD) t.d[u].put(zero);
                    if (!GRAD || MODE != SCAN_AGG) t.x[u].put(zero);
                }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t i = i0 + tr * U + u, r = row(min(i, n - 1));
#pragma unroll
            for (int e = 0; e < V; ++e) {
                float ga, na;
                gate_of(t.g[u].get(e), ga, na);
                ca[u][e] = ga;
                if (!GRAD) cb[u][e] = na * t.x[u].get(e);
                else {
                    cb[u][e] = t.d[u].get(e);
                    if (MODE != SCAN_AGG) {
                        const float hp = r > o0 ? t.h[u].get(e) : a.start ? a.start[s * a.channels + cc + e] : 0.f;
                        k1[u][e] = na;
                        k2[u][e] = (hp - t.x[u].get(e)) * (ga * na);
                    }
                }
            }
        }
        if (i0 + DEPTH * TILE < n) load(t, i0 + DEPTH * TILE);   // (later rows, while these are combined)
        float A[V], B[V], wa[V], wb[V];
#pragma unroll
        for (int e = 0; e < V; ++e) { A[e] = 1.f; B[e] = 0.f; }
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int e = 0; e < V; ++e) {
                B[e] = GRAD ? ca[u][e] * (B[e] + cb[u][e]) : fmaf(ca[u][e], B[e], cb[u][e]);
                A[e] *= ca[u][e];
            }
        across(A, B, wa, wb);
        if constexpr (MODE == SCAN_AGG) {
#pragma unroll
            for (int e = 0; e < V; ++e) {
                carry[e] = fmaf(wa[e], carry[e], wb[e]);
                total[e] *= wa[e];
            }
        } else {
            float h[V];
#pragma unroll
            for (int e = 0; e < V; ++e) h[e] = fmaf(A[e], carry[e], B[e]);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int64_t i = i0 + tr * U + u;
                float y[V], y2[V];
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    if (!GRAD) y[e] = h[e] = fmaf(ca[u][e], h[e], cb[u][e]);
                    else {
                        const float d = cb[u][e] + h[e];
                        y[e] = k1[u][e] * d;
                        y2[e] = k2[u][e] * d;
                        h[e] = ca[u][e] * d;
                    }
                }
                if (i < n && on) {
                    P p;
                    p.put(y);
                    write_rows((T*)a.out + row(i) * a.ldo + c, p);
                    if (GRAD) {
                        p.put(y2);
                        write_rows((T*)a.out2 + row(i) * a.ldo2 + c, p);
                    }
                }
            }
#pragma unroll
            for (int e = 0; e < V; ++e) carry[e] = __shfl(h[e], 64 - CT + lane % CT);
        }
    };
    for (int64_t i0 = 0; i0 < n; i0 += DEPTH * TILE)
#pragma unroll
        for (int d = 0; d < DEPTH; ++d)
            if (i0 + d * TILE < n) tile(ring[d], i0 + d * TILE);
    if (tr || !on) return;
    if constexpr (MODE == SCAN_AGG) {
        float* p = a.agg + (s * a.chunks + v) * a.channels + c;
#pragma unroll
        for (int e = 0; e < V; ++e) {
            p[e] = total[e];
            p[plane + e] = carry[e];
        }
    } else if (a.end && last_chunk) {
#pragma unroll
        for (int e = 0; e < V; ++e) a.end[s * a.channels + c + e] = carry[e];
    }
}

// Channels of a wave: whole 128-byte lines of a row where it has them.
static int scan_block(int bf16) { return bf16 ? 64 : 32; }
// Few histories: their time axis is split over two launches, the first of which reads two arrays (of the gradient's: two of six) once more.  us, whole / split,
// bf16, 256 channels, forward and gradient: 64 histories (256 waves) of 400 steps 28 / 20, 61 / 26; 128 of 200 17 / 20, 34 / 25, of 400 28 / 29, 61 / 41, of
// 1,000 72 / 64, 164 / 92; 200 of 400 29 / 46, 70 / 70, of 1,000 76 / 101, 173 / 161; fp32: 64 (512 waves) of 400 19 / 23, 34 / 30, 128 of 1,000 58 / 86, 129 / 144.
SeqSplit seq_scan_split(int64_t n_seqs, int64_t longest, int channels, int bf16, int grad, int64_t room) {
    const int64_t waves = n_seqs * ((channels + scan_block(bf16) - 1) / scan_block(bf16));
    const int64_t tile = 64, enough = longest >= 1000 ? (grad ? 1024 : 640) : (grad ? 640 : 512);
    if (waves >= enough || longest <= 2 * tile || waves <= 0) return {1, std::max<int64_t>(longest, 1)};
    const int64_t want = std::min<int64_t>({(longest + tile - 1) / tile, std::max<int64_t>(1, 4096 / waves), 256, room / (2 * n_seqs * channels)});
    if (want <= 1) return {1, longest};
    const int64_t chunk = ((longest + want - 1) / want + tile - 1) / tile * tile;
    return {(int)((longest + chunk - 1) / chunk), chunk};
}

template <typename T, int V, int CT, bool GRAD, bool STREAM>
static void scan_modes(hipStream_t st, const SeqScanArgs& a) {
    // Consecutive rows of a lane (the gradient holds more arrays), and tiles on their way: two of bf16 (1,024 users 114 -> 106 us), one of fp32, which has
    // half as many channels in as many registers (two: 200 users of 400 steps 42 -> 47 us).
    constexpr int U = GRAD ? 4 : 8, DEPTH = sizeof(T) == 2 ? 2 : 1;
    const int64_t units = a.v.n_seqs * a.chunks * ((a.channels + CT * V - 1) / (CT * V));
    const dim3 grid = workgroups((units + 3) / 4);
    if (a.chunks == 1) {
        hipLaunchKernelGGL((seq_scan_kernel<T, V, CT, U, DEPTH, GRAD, SCAN_WHOLE, STREAM>), grid, dim3(256), 0, st, a);
    } else {
        hipLaunchKernelGGL((seq_scan_kernel<T, V, CT, U, DEPTH, GRAD, SCAN_AGG, false>), grid, dim3(256), 0, st, a);
        hipLaunchKernelGGL((seq_scan_kernel<T, V, CT, U, DEPTH, GRAD, SCAN_APPLY, STREAM>), grid, dim3(256), 0, st, a);
    }
}
// Elements a lane moves at once: four.  (bf16 with eight, 16 bytes: twice the registers, one wave a SIMD and as many exchanges along the time axis for half the rows;
// 1,024 users 122 us instead of 115.  fp32 with two: 201 ragged users' gradient 30 us instead of 24.)
static int scan_vector(const SeqScanArgs& a, int bf16, int grad) {
    const int elem = bf16 ? 2 : 4, bytes = 4 * elem;
    auto ok = [&](const void* p, int64_t ld) { return (uintptr_t)p % bytes == 0 && (ld * elem) % bytes == 0; };
    return a.channels % 4 == 0 && ok(a.x, a.ldx) && ok(a.gate, a.ldg) && ok(a.out, a.ldo) &&
                   (!grad || (ok(a.h, a.ldh) && ok(a.dh, a.lddh) && ok(a.out2, a.ldo2)))
               ? 4 : 1;
}
void launch_seq_scan(hipStream_t st, const SeqScanArgs& a, int bf16, int grad) {
    if (a.v.n_seqs <= 0) return;
    const int v = scan_vector(a, bf16, grad);
    // Past the caches where the arrays take most of the last of them or more (455 MB: 115 -> 112 us; 225 MB in two passes: 87 -> 83; 66 MB: 32 -> 41, so not there).
    const bool stream = (double)a.v.n_rows * a.channels * (bf16 ? 2 : 4) * (grad ? 6 : 3) > 192e6;
#define SCAN(T_, V_, CT_)                                                                                                   \
    do {                                                                                                                    \
        if (grad && stream) scan_modes<T_, V_, CT_, true, (V_ > 1)>(st, a);                                                 \
        else if (grad) scan_modes<T_, V_, CT_, true, false>(st, a);                                                         \
        else if (stream) scan_modes<T_, V_, CT_, false, (V_ > 1)>(st, a);                                                   \
        else scan_modes<T_, V_, CT_, false, false>(st, a);                                                                  \
    } while (0)
    if (bf16) { if (v == 4) SCAN(bf16_t, 4, 16); else SCAN(bf16_t, 1, 32); }
    else { if (v == 4) SCAN(float, 4, 8); else SCAN(float, 1, 32); }
#undef SCAN
}

// One row of every sequence: the state, fp32, in place.  Bound: latency (512 users x 256 channels, 2 MB: 2 of the call's 8.6 us are the kernel's).
template <typename T, int V>
__global__ __launch_bounds__(256) void seq_scan_step_kernel(int64_t n_seqs, int channels, const T* __restrict__ x, int64_t ldx, const T* __restrict__ gate,
                                                            int64_t ldg, float* state, T* h, int64_t ldh) {
    const int per = channels / V;
    const int64_t i = (int64_t)workgroup() * 256 + threadIdx.x, s = i / per;
    if (s >= n_seqs) return;
    const int c = (int)(i % per) * V;
    const Pack<T, V> px = *reinterpret_cast<const Pack<T, V>*>(x + s * ldx + c), pg = *reinterpret_cast<const Pack<T, V>*>(gate + s * ldg + c);
    Pack<float, V>* ps = reinterpret_cast<Pack<float, V>*>(state + s * channels + c);
    const Pack<float, V> old = *ps;
    float y[V];
#pragma unroll
    for (int e = 0; e < V; ++e) {
        float a, na;
        gate_of(pg.get(e), a, na);
        y[e] = fmaf(a, old.get(e), na * px.get(e));
    }
    Pack<float, V> ns;
    ns.put(y);
    *ps = ns;
    if (h) {
        Pack<T, V> ph;
        ph.put(y);
        *reinterpret_cast<Pack<T, V>*>(h + s * ldh + c) = ph;
    }
}
void launch_seq_scan_step(hipStream_t st, int64_t n_seqs, int channels, int bf16, const void* x, int64_t ldx, const void* gate, int64_t ldg,
                          float* state, void* h, int64_t ldh) {
    if (n_seqs <= 0) return;
    const int elem = bf16 ? 2 : 4;
    auto ok = [&](const void* p, int64_t ld) { return (uintptr_t)p % (4 * elem) == 0 && (ld * elem) % (4 * elem) == 0; };
    const bool wide = channels % 4 == 0 && ok(x, ldx) && ok(gate, ldg) && (!h || ok(h, ldh)) && (uintptr_t)state % 16 == 0;
    const dim3 grid = workgroups((n_seqs * (channels / (wide ? 4 : 1)) + 255) / 256);
#define STEP(T_, V_) hipLaunchKernelGGL((seq_scan_step_kernel<T_, V_>), grid, dim3(256), 0, st, n_seqs, channels, (const T_*)x, ldx, (const T_*)gate, ldg, state, (T_*)h, ldh)
    if (bf16) { if (wide) STEP(bf16_t, 4); else STEP(bf16_t, 1); }
    else { if (wide) STEP(float, 4); else STEP(float, 1); }
#undef STEP
}
