// The calls on histories without a GPU: the runtime's entry points that they use are defined here (a program's own definitions come before a library's), a launch is looked at
// instead of run.  Each call gets a context whose workspace has just the size that the library names for it, or for a call of no less of anything; it must be taken, and what its
// launches are told to write must end with the workspace.  Nothing is allocated on a device; the pointers are numbers.
#include <dlfcn.h>

#include <algorithm>
#include <cstring>
#include <random>

#include "../paper_2401_04338_amd/csrc/gm_context.h"

static char* const WS = reinterpret_cast<char*>((uintptr_t)1 << 40);
static void* const DATA = reinterpret_cast<void*>((uintptr_t)1 << 44);
static float* const FLOATS = static_cast<float*>(DATA);
static gm_ctx ctx;
static u32 words[SEQ_WORDS];
static std::string what;        // the call, for messages
static int bf16, n_failed = 0;
static int64_t n_calls = 0, n_launches = 0;

static void failed(const char* fmt, ...) {
    if (++n_failed > 20) return;
    va_list ap;
    va_start(ap, fmt);
    printf("%s: ", what.c_str());
    vprintf(fmt, ap);
    printf("\n");
    va_end(ap);
}
// `count` elements of `size` bytes from p on lie in the workspace
static void inside(const char* name, const void* p, int64_t count, int64_t size) {
    const char* from = static_cast<const char*>(p);
    if (from < WS || from + count * size > WS + ctx.ws_bytes)
        failed("%s: [%lld, %lld) of a workspace of %lld bytes", name, (long long)(from - WS), (long long)(from - WS + count * size), (long long)ctx.ws_bytes);
}
static void launched(const char* kernel, dim3 grid, void** args) {
    const int64_t groups = (int64_t)grid.x * grid.y, elem = bf16 ? 2 : 4;
    ++n_launches;
    auto is = [&](const char* part) { return strstr(kernel, part) != nullptr; };
    if (is("seq_norm_grad_kernel") || is("seq_norm_columns_kernel")) {
        const SeqNormArgs& a = *static_cast<SeqNormArgs*>(args[0]);
        if (groups < a.blocks) failed("%s: %lld workgroups for %d", kernel, (long long)groups, a.blocks);
        if (a.dweight && a.blocks > 1) inside(kernel, a.partial, (int64_t)a.blocks * 2 * ((a.channels + 3) / 4 * 4), 4);
    } else if (is("sum_blocks_kernel")) {
        const SumBlocks& a = *static_cast<SumBlocks*>(args[0]);
        inside(kernel, a.partial, a.blocks * 2 * a.half_stride, 4);
    } else if (is("seq_glu_slope") || is("seq_glu_dx") || is("seq_glu_dw") || is("seq_glu_join")) {
        const SeqGluArgs& a = *static_cast<SeqGluArgs*>(args[0]);
        inside(kernel, a.d, a.n * 2 * a.d_out, elem);
        if (a.splits > 1) inside("pieces of the weights' gradients", a.partial, (int64_t)a.splits * a.d_in * 2 * a.d_out, 4);
        if (a.dx_splits > 1) inside("pieces of dx", a.dx_partial, a.dx_splits * a.n * a.d_in, 4);
        if (a.dbg && a.blocks > 1) inside("sums of the biases", a.colpart, (int64_t)a.blocks * 2 * a.d_out, 4);
        if (is("seq_glu_slope") && groups < a.blocks) failed("%s: %lld workgroups for %d", kernel, (long long)groups, a.blocks);
    } else if (is("seq_attend_kernel") || is("seq_attend_wide_kernel") || is("seq_attend_join_kernel")) {
        const SeqAttendArgs& a = *static_cast<SeqAttendArgs*>(args[0]);
        const int64_t n = a.splits * a.n_queries * a.kv_heads * a.group;
        if (a.splits > 1) inside(kernel, a.part_o, n * a.dim, 4);
        if (a.splits > 1) inside(kernel, a.part_ml, n * 2, 4);
    }
}

static struct { dim3 grid, block; size_t lds; hipStream_t stream; } config;   // of the launch that is being made
extern "C" {
hipError_t __hipPushCallConfiguration(dim3 grid, dim3 block, size_t lds, hipStream_t stream) {
    config = {grid, block, lds, stream};
    return hipSuccess;
}
hipError_t __hipPopCallConfiguration(dim3* grid, dim3* block, size_t* lds, hipStream_t* stream) {
    *grid = config.grid; *block = config.block; *lds = config.lds; *stream = config.stream;
    return hipSuccess;
}
hipError_t hipLaunchKernel(const void* f, dim3 grid, dim3, void** args, size_t, hipStream_t) {
    Dl_info info;
    if (!dladdr(f, &info) || !info.dli_sname) failed("a launch of no name");
    else launched(info.dli_sname, grid, args);
    return hipSuccess;
}
hipError_t hipSetDevice(int) { return hipSuccess; }
hipError_t hipGetLastError() { return hipSuccess; }
hipError_t hipFuncSetAttribute(const void*, hipFuncAttribute, int) { return hipSuccess; }
}

static void taken(int rc) {
    ++n_calls;
    if (rc != GM_OK) failed("refused (%d): %s", rc, ctx.err.c_str());
}
template <typename... A> static void say(const char* fmt, A... a) {
    char buf[256];
    snprintf(buf, sizeof buf, fmt, a...);
    what = buf;
}
static std::mt19937_64 rng(7);
static int64_t uniform(int64_t lo, int64_t hi) { return std::uniform_int_distribution<int64_t>(lo, hi)(rng); }
static int64_t spread(int64_t lo, int64_t hi) {   // evenly over the logarithm
    const double x = std::uniform_real_distribution<double>(std::log((double)lo), std::log((double)hi + 1))(rng);
    return std::min(hi, std::max(lo, (int64_t)std::exp(x)));
}
static int64_t below(int64_t lo, int64_t hi) { return rng() % 3 ? spread(lo, hi) : hi; }   // often the largest

static void norm(int64_t room_rows, int room_channels, int64_t n, int channels) {
    ctx.ws_bytes = gm_seq_norm_grad_bytes(room_rows, room_channels);
    say("layer norm's gradient, %lld rows of %d, %s, room for %lld of %d", (long long)n, channels, bf16 ? "bf16" : "fp32", (long long)room_rows, room_channels);
    if (!ctx.ws_bytes) failed("no size");
    const int64_t ld = channels + (int64_t)(rng() % 3 ? 0 : uniform(0, 9));
    taken(gm_seq_norm_grad(&ctx, n, channels, bf16, DATA, ld, DATA, ld, FLOATS, rng() % 2 ? FLOATS : nullptr, rng() % 2 ? DATA : nullptr, ld, DATA, ld, FLOATS, FLOATS));
}
static void norms() {
    for (bf16 = 0; bf16 < 2; ++bf16) {
        for (int channels : {1, 7, 8, 32, 33, 64, 100, 128, 255, 256, 257, 512, 513, 845, 1023, 1024, 1025, 1030, 1500, 2047, 2048, 2049, 3000, 4095, 4096, 4097, 8191, 8192, 8193, 20000, 65536})
            for (int64_t n : {1, 2, 3, 4, 5, 7, 8, 15, 16, 17, 31, 32, 33, 100, 255, 256, 257, 1000, 1023, 1024, 1025, 2047, 2048, 3000, 4000, 4095, 4096, 4097, 5000, 70000, 1 << 20})
                norm(n, channels, n, channels);
        for (int i = 0; i < 100000; ++i) {
            const int64_t n = spread(1, 20000), channels = spread(1, 12000);
            norm(n, (int)channels, below(1, n), (int)below(1, channels));
        }
    }
}

static void glu(int64_t room_rows, int room_in, int room_out, int64_t n, int d_in, int d_out) {
    ctx.ws_bytes = gm_seq_glu_grad_bytes(&ctx, room_rows, room_in, room_out, bf16);
    say("gated feed-forward's gradient, %lld rows, %d to 2 x %d, %s, room for %lld, %d to 2 x %d", (long long)n, d_in, d_out, bf16 ? "bf16" : "fp32", (long long)room_rows, room_in, room_out);
    if (!ctx.ws_bytes) failed("no size");
    float* bias = rng() % 4 ? FLOATS : nullptr;
    taken(gm_seq_glu_grad(&ctx, n, d_in, d_out, bf16, (int)(rng() % 4), DATA, d_out, DATA, d_in, DATA, d_out, DATA, d_out, DATA, d_out, DATA, d_out, DATA, d_in, DATA, d_out, DATA,
                          d_out, bias, bias));
}
static void glus() {
    for (bf16 = 0; bf16 < 2; ++bf16) {
        const int unit = bf16 ? 8 : 4;
        for (int d_out : {8, 64, 256, 264, 504, 512, 520, 1024, 1536, 2048, 4096, 8192, 16384, 65536})
            for (int d_in : {8, 64, 136, 512, 1024, 4096})
                for (int64_t n : {0, 1, 3, 4, 5, 16, 64, 127, 128, 400, 817, 1000, 2048, 3001, 8192, 8193, 20000, 65536}) glu(n, d_in, d_out, n, d_in, d_out);
        for (int i = 0; i < 100000; ++i) {
            const int64_t n = spread(1, 70000), k = spread(1, 4096 / unit), m = spread(1, 16384 / unit);
            glu(n, (int)k * unit, (int)m * unit, below(1, n), (int)below(1, k) * unit, (int)below(1, m) * unit);
        }
    }
}

static void attend(int64_t users, int64_t queries, int64_t keys, int heads, int kv_heads, int dim, int64_t room_users, int64_t room_queries, int64_t room_keys) {
    const gm_seq_heads hd{heads, kv_heads, dim, bf16, 0.125f};
    auto seqs = [](int64_t n, int64_t longest) { return gm_seq{n, n * longest, longest, static_cast<const int64_t*>(DATA), nullptr}; };
    const gm_seq rq = seqs(room_users, room_queries), rk = seqs(room_users, room_keys), q = seqs(users, queries), k = seqs(users, keys);
    ctx.ws_bytes = gm_seq_attend_bytes(&ctx, &rq, &rk, &hd, 0);
    say("attention, %lld of %lld queries, %lld keys, %d heads over %d of %d, %s, room for %lld of %lld, %lld", (long long)users, (long long)queries, (long long)keys, heads, kv_heads, dim,
        bf16 ? "bf16" : "fp32", (long long)room_users, (long long)room_queries, (long long)room_keys);
    const int64_t ldq = (int64_t)heads * dim, ldk = (int64_t)kv_heads * dim;
    const uint8_t* mask = rng() % 2 ? static_cast<const uint8_t*>(DATA) : nullptr;
    // a call of up to 32 rows a key head lies on one wave, in either order: the pieces of 32 rows that the device holds
    const int64_t slots = (bf16 ? 2 : 1) * ctx.n_cus, order = 2 * 256 * 4;
    if (room_queries * (heads / kv_heads) <= 32 && (int64_t)ctx.ws_bytes > order + 2 * 256 + slots * 32 * (dim + 2) * 4) failed("%lld bytes named", (long long)ctx.ws_bytes);
    taken(gm_seq_attend(&ctx, &q, &k, &hd, DATA, ldq, DATA, ldk, DATA, ldk, mask, DATA, ldq, FLOATS));
    taken(gm_seq_attend_causal(&ctx, &q, &k, &hd, DATA, ldq, DATA, ldk, DATA, ldk, mask, DATA, ldq, FLOATS));
}
static void attends() {
    for (bf16 = 0; bf16 < 2; ++bf16)
        for (int i = 0; i < 100000; ++i) {
            const int kv_heads = (int)uniform(1, 4), heads = kv_heads * (int)spread(1, 16), dim = 8 * (int)uniform(1, 16);
            const int64_t users = spread(1, 400), queries = spread(1, 300), keys = spread(1, 20000);
            attend(below(1, users), below(1, queries), below(1, keys), heads, kv_heads, dim, users, queries, keys);
        }
}

int main(int argc, char** argv) {
    const std::string which = argc > 1 ? argv[1] : "";
    ctx.ws = WS;
    ctx.seq_status = words;
    ctx.wait = 0;
    if (which == "norm") norms();
    else if (which == "glu") glus();
    else if (which == "attend") attends();
    else return 2;
    printf("%lld calls, %lld launches, %d failed\n", (long long)n_calls, (long long)n_launches, n_failed);
    return n_failed || !n_launches ? 1 : 0;
}
