// Forks and cuts over a fake device: the host code of paper_2505_18610_amd/csrc/kvq_moves.hip, which is included here, with kvq_host.cpp and a HIP
// runtime that is stubbed below.  A launch does to the page tables what the kernel does to them and checks what the kernel would read
// and write.  tests/test_moves_stub.py builds it with sanitizers on the host side; argument: the scenario.  Exit code 0 = pass.  No GPU
// and no HIP library is involved.
#include "../paper_2505_18610_amd/csrc/kvq_moves.hip"

#include <sys/mman.h>

#include <cstdio>
#include <cstdlib>
#include <functional>
#include <map>
#include <random>
#include <set>
#include <string>
#include <utility>

namespace {

int failures = 0;
#define CHECK(cond, ...)                                                                                                        \
    do {                                                                                                                        \
        if (!(cond)) { ++failures; printf("line %d: %s: ", __LINE__, #cond); printf(__VA_ARGS__); printf("\n"); fflush(stdout); } \
    } while (0)

int launches = 0, fail_launch = -1;  // the launch with this number fails
hipError_t last_error = hipSuccess;
hipError_t launched() { return launches++ == fail_launch ? hipErrorLaunchFailure : hipSuccess; }

struct Arena {
    uint64_t bytes;
    int units, tpp;
};
std::map<const uint8_t*, Arena> arenas;

using Span = std::pair<uint64_t, uint64_t>;
void add_spans(std::vector<Span>& spans, const Arena& a, const KvqPageDesc& d, bool meta) {
    const uint64_t code = (uint64_t)d.code_off256 * 256, m = (uint64_t)d.meta_off256 * 256;
    spans.push_back({code, code + 1024ull * d.bits * a.tpp * a.units});
    if (meta) spans.push_back({m, m + 1024ull * a.tpp * a.units});
}
void check_apart(std::vector<Span> spans, uint64_t bytes) {
    std::sort(spans.begin(), spans.end());
    for (size_t i = 0; i < spans.size(); ++i) {
        CHECK(spans[i].second <= bytes, "a page ends at %llu of %llu", (unsigned long long)spans[i].second, (unsigned long long)bytes);
        CHECK(i == 0 || spans[i - 1].second <= spans[i].first, "pages overlap");
    }
}
bool has_meta(const KvqPageDesc& d) { return d.bits < 16 || d.int16; }

void fork_launched(const ForkArgs& A, dim3 grid) {
    const Arena &src = arenas.at(A.src), &dst = arenas.at(A.dst);
    CHECK(src.tpp == A.tpp && dst.tpp == A.tpp && src.units == A.src_batch * A.n_kv && dst.units == A.dst_batch * A.n_kv, "shapes");
    CHECK((uint64_t)grid.x == (uint64_t)A.groups * dst.units * A.n_here && A.groups * KVQ_FORK_TILES >= A.tpp, "%u workgroups", grid.x);
    CHECK(A.page0 >= 0 && A.n_here > 0 && A.n_here <= KVQ_FORK_ARG_PAGES && A.page0 + A.n_here <= A.n_pages, "%d + %d of %d pages", A.page0, A.n_here, A.n_pages);
    CHECK(A.last_tiles >= 1 && A.last_tiles <= A.tpp, "%d tiles in the last page", A.last_tiles);
    std::vector<Span> to;
    for (int i = 0; i < A.n_here; ++i) {
        const KvqPageDesc from = A.src_table[A.page0 + i];
        CHECK(from.bits == 16 || from.bits == 8 || from.bits == 4 || from.bits == 2, "page %d has %u bits", A.page0 + i, from.bits);
        KvqPageDesc d = from;
        d.code_off256 = A.code_off256[i];
        d.meta_off256 = A.meta_off256[i];
        add_spans(to, dst, d, has_meta(d));
        if (A.in_place) add_spans(to, src, from, has_meta(from));  // what is read is not written over
        else A.dst_table[A.page0 + i] = d;
    }
    check_apart(to, dst.bytes);
    if (A.map)
        for (int b = 0; b < A.dst_batch; ++b) (void)*const_cast<const volatile int32_t*>(A.map + b);
}
void table_launched(const ForkArgs& A) {
    for (int i = 0; i < A.n_here; ++i) {
        A.dst_table[A.page0 + i].code_off256 = A.code_off256[i];
        A.dst_table[A.page0 + i].meta_off256 = A.meta_off256[i];
    }
}

// the call configuration of a launch, as the compiler's stubs hand it on
struct Config { dim3 grid, block; size_t shared; hipStream_t stream; } config;

}  // namespace

// ---- the HIP runtime, as far as the host code uses it
extern "C" {
void** __hipRegisterFatBinary(const void*) { static void* handle; return &handle; }
void __hipRegisterFunction(void**, const void*, char*, const char*, unsigned, void*, void*, void*, void*, int*) {}
void __hipRegisterVar(void**, void*, char*, char*, int, size_t, int, int) {}
void __hipUnregisterFatBinary(void**) {}
hipError_t __hipPushCallConfiguration(dim3 grid, dim3 block, size_t shared, hipStream_t stream) { config = {grid, block, shared, stream}; return hipSuccess; }
hipError_t __hipPopCallConfiguration(dim3* grid, dim3* block, size_t* shared, hipStream_t* stream) {
    *grid = config.grid; *block = config.block; *shared = config.shared; *stream = config.stream;
    return hipSuccess;
}
hipError_t hipLaunchKernel(const void* f, dim3 grid, dim3 block, void** args, size_t, hipStream_t) {
    // a launch has less than 2^32 threads
    if ((uint64_t)grid.x * block.x >> 32) return last_error = hipErrorInvalidConfiguration;
    const hipError_t e = launched();
    if (e != hipSuccess) return last_error = e;
    const auto is = [&](auto kernel) { return f == reinterpret_cast<const void*>(kernel); };
    if (is(&kvq_fork_kernel<true>) || is(&kvq_fork_kernel<false>)) fork_launched(*static_cast<const ForkArgs*>(args[0]), grid);
    else if (is(&kvq_fork_table_kernel)) table_launched(*static_cast<const ForkArgs*>(args[0]));
    else if (is(&kvq_clear_tail_kernel)) CHECK(*static_cast<const int*>(args[3]) >= 0 && *static_cast<const int*>(args[3]) < *static_cast<const int*>(args[2]), "tile");
    else CHECK(is(&kvq_read_kernel), "another kernel");
    return hipSuccess;
}
hipError_t hipGetLastError() { const hipError_t e = last_error; last_error = hipSuccess; return e; }
hipError_t hipHostMalloc(void** p, size_t n, unsigned int) { *p = aligned_alloc(256, (n + 255) / 256 * 256); return hipSuccess; }
hipError_t hipHostFree(void* p) { free(p); return hipSuccess; }
hipError_t hipHostGetDevicePointer(void** d, void* h, unsigned int) { *d = h; return hipSuccess; }
hipError_t hipEventCreateWithFlags(hipEvent_t* e, unsigned) { *e = nullptr; return hipSuccess; }
hipError_t hipEventDestroy(hipEvent_t) { return hipSuccess; }
hipError_t hipEventRecord(hipEvent_t, hipStream_t) { return hipSuccess; }
hipError_t hipEventSynchronize(hipEvent_t) { return hipSuccess; }
hipError_t hipStreamSynchronize(hipStream_t) { return hipSuccess; }
hipError_t hipMemcpyAsync(void* d, const void* s, size_t n, hipMemcpyKind, hipStream_t) { memcpy(d, s, n); return hipSuccess; }
hipError_t hipGetDevice(int* d) { *d = 0; return hipSuccess; }
hipError_t hipGetDevicePropertiesR0600(hipDeviceProp_tR0600* p, int) { memset(p, 0, sizeof *p); p->multiProcessorCount = 256; return hipSuccess; }
}

// ---- the launches of the library's other translation units
hipError_t kvq_launch_append(int, uint8_t*, KvqPageDesc* table, const void*, const void*, int, int, int, int, const KvqAppendPages& ap, KvqVMark, int,
                             const float*, int, const float*, bool, hipStream_t) {
    const hipError_t e = launched();
    if (e != hipSuccess) return e;
    for (int i = ap.fresh; i < ap.n; ++i) table[ap.first_page + i] = KvqPageDesc{ap.code_off256[i], ap.meta_off256[i], ap.bits, ap.int16};
    return hipSuccess;
}
static hipError_t requant(int to, KvqPageDesc* table, const KvqRequantJob* dev, const KvqRequantJob* host, int n) {
    const hipError_t e = launched();
    if (e != hipSuccess) return e;
    for (int i = 0; i < n; ++i) {
        const KvqRequantJob& j = host ? host[i] : dev[i];
        table[j.tiles_page >> 11] = KvqPageDesc{j.dst_code_off256, j.meta_off256, (uint32_t)to, 0u};
    }
    return hipSuccess;
}
hipError_t kvq_launch_shrink(int to, int, uint8_t*, KvqPageDesc* table, const KvqRequantJob* dev, const KvqRequantJob* host, int n, int, int, KvqVMark,
                             hipStream_t) { return requant(to, table, dev, host, n); }
hipError_t kvq_launch_quant16(int to, uint8_t*, KvqPageDesc* table, const KvqRequantJob* dev, const KvqRequantJob* host, int n, int, int, KvqVMark, int,
                              hipStream_t) { return requant(to, table, dev, host, n); }
hipError_t kvq_launch_reparam_store(const float*, float*, int, hipStream_t) { return launched(); }
hipError_t kvq_launch_calibrate(const void*, int, int, int, float, float, float*, hipStream_t) { return launched(); }
int kvq_error_workgroups(int, int) { return 1; }
hipError_t kvq_launch_error(bool, const uint8_t*, const KvqPageDesc*, const void*, const void*, const float*, const float*, int, int, int, double*,
                            hipStream_t) { return launched(); }
hipError_t kvq_launch_stream_read(const void*, size_t, int, uint32_t*, hipStream_t) { return launched(); }
hipError_t kvq_launch_fill_u32(uint32_t* dst, uint32_t value, size_t n, hipStream_t) {
    const hipError_t e = launched();
    if (e == hipSuccess) std::fill_n(dst, n, value);
    return e;
}
hipError_t kvq_static_scratch(unsigned char** ptr) { *ptr = nullptr; return hipErrorUnknown; }
hipError_t kvq_launch_attention(const KvqAttnParams& p, int, hipStream_t) {
    const hipError_t e = launched();
    if (e == hipSuccess && p.app_page >= 0) const_cast<KvqPageDesc*>(p.table)[p.app_page] = p.app_desc;
    return e;
}
hipError_t kvq_launch_merge(const KvqAttnParams&, int, hipStream_t) { return launched(); }
hipError_t kvq_launch_attention_batch(const KvqAttnParams*, const KvqAttnParams*, const int*, int, hipStream_t) { return launched(); }

namespace {

uint16_t input[16];  // never read
struct Cache {
    kvq_cache_t* c = nullptr;
    kvq_config_t cfg{};
    uint8_t* arena = nullptr;
    uint64_t bytes = 0, whole = 0;
    // pages: how many of 16 bits the arena holds; device: false for an accounting-only cache
    Cache(int batch, int kv, int page, int max_tokens, int pages, int policy, int window, int tier16, uint64_t budget, bool device, int layers = 1) {
        cfg.n_layers = layers; cfg.batch = batch; cfg.n_kv_heads = kv; cfg.n_q_heads = kv; cfg.head_dim = 128; cfg.group = 32;
        cfg.max_tokens = max_tokens; cfg.page_tokens = page; cfg.policy = policy; cfg.window = window; cfg.count_metadata_in_budget = 1;
        const std::vector<uint64_t> budgets((size_t)layers, budget);
        const std::vector<uint8_t> fbits((size_t)layers, 2);
        bytes = kvq_arena_bytes(&cfg, (uint64_t)pages * 512 * page * batch * kv);
        if (device) {
            void* const p = mmap(nullptr, bytes, PROT_READ | PROT_WRITE, MAP_PRIVATE | MAP_ANONYMOUS | MAP_NORESERVE, -1, 0);
            if (p == MAP_FAILED) { printf("no address space for %llu bytes\n", (unsigned long long)bytes); exit(77); }
            arena = static_cast<uint8_t*>(p);
            arenas[arena] = Arena{bytes, batch * kv, page / 32};
        }
        const kvq_status_t st = kvq_cache_create(&cfg, budgets.data(), fbits.data(), arena, bytes, &c);
        CHECK(st == KVQ_OK, "create: %s", kvq_status_string(st));
        if (tier16) CHECK(kvq_cache_set_option(c, KVQ_OPT_TIER16, 1) == KVQ_OK, "tier");
        whole = kvq_cache_arena_free_bytes(c);
    }
    ~Cache() {
        kvq_cache_destroy(c);
        if (arena) { arenas.erase(arena); munmap(arena, bytes); }
    }
    Cache(const Cache&) = delete;
    int tokens(int layer = 0) const { int T = -1; kvq_cache_describe(c, layer, nullptr, 0, nullptr, nullptr, &T, nullptr); return T; }
    std::vector<int> widths(int layer = 0) const {
        std::vector<kvq_segment_info_t> s(512);
        int n = 0;
        kvq_cache_describe(c, layer, s.data(), 512, &n, nullptr, nullptr, nullptr);
        std::vector<int> w;
        for (int i = 0; i < n; ++i) w.insert(w.end(), (size_t)(s[(size_t)i].token_end - s[(size_t)i].token_begin), s[(size_t)i].bits);
        return w;
    }
    // the table's entries are the pages that the blocks hold, the blocks' pages lie apart, and the arena's free bytes are the others
    void check(const std::set<int>& unusable = {}) const {
        std::vector<Span> spans;
        uint64_t held = 0;
        for (int l = 0; l < cfg.n_layers; ++l) {
            const kvq_host::Layer& L = c->layers[(size_t)l];
            int t = 0;
            for (size_t i = 0; i < L.pages.size(); ++i) {
                const Page& p = L.pages[i];
                const KvqPageDesc d = c->desc(p);
                CHECK(p.n > 0 && p.n <= cfg.page_tokens && (i + 1 == L.pages.size() || p.n == cfg.page_tokens), "page %zu holds %d tokens", i, p.n);
                t += p.n;
                held += (uint64_t)(p.bits == 16 ? 16 : p.bits == 8 ? 8 : p.bits == 4 ? 4 : 2) + (c->has_meta(p.bits) ? 1 : 0);
                add_spans(spans, Arena{bytes, c->units, c->tpp}, d, c->has_meta(p.bits));
                if (arena && !unusable.count(l)) CHECK(std::memcmp(&d, c->table_dev(l) + i, sizeof d) == 0, "entry %zu of block %d", i, l);
            }
            CHECK(t == L.T, "%d tokens in pages, %d in the block", t, L.T);
        }
        check_apart(spans, bytes);
        CHECK(kvq_cache_arena_free_bytes(c) == whole - held * c->unit_bytes, "free bytes");
    }
};

// Random calls on three caches, launches that fail now and then: refused calls change nothing, a block whose launch failed is refused until it is
// emptied, and everything else goes on.
void random_calls(bool device) {
    for (int seed = 0; seed < 120; ++seed) {
        std::mt19937 rng((unsigned)seed);
        const auto R = [&](int lo, int hi) { return lo + (int)(rng() % (unsigned)(hi - lo + 1)); };
        const int kv = R(1, 2), page = 32 * R(1, 3), tier16 = R(0, 1), layers = R(1, 2);
        std::vector<std::unique_ptr<Cache>> caches;
        for (int i = 0; i < 3; ++i)
            caches.emplace_back(new Cache(R(1, 3), kv, page, page * R(3, 30), R(2, 14), R(0, 1), page * R(0, 1), tier16,
                                          (uint64_t)R(20, 4000) * kv * 576, device, layers));
        std::vector<std::set<int>> unusable(3);
        std::vector<int32_t> map{0, 1, 2};
        for (int op = 0; op < 150; ++op) {
            const int i = R(0, 2), k = R(0, 2), layer = R(0, layers - 1);
            Cache &a = *caches[(size_t)i], &b = *caches[(size_t)k];
            const int what = R(0, 9), old = a.tokens(layer);
            const auto before = a.widths(layer);
            const uint64_t free = kvq_cache_arena_free_bytes(a.c);
            if (R(0, 11) == 0) fail_launch = launches + R(0, 2);
            kvq_status_t st = KVQ_OK;
            bool refused_changes_nothing = true;
            if (what < 4) {
                st = kvq_quantize_append(a.c, layer, input, input, R(1, 3 * page), R(0, 3) ? 0 : 2 << R(0, 3), nullptr);
                if (st == KVQ_E_BUDGET) {
                    fail_launch = -1;
                    int done = 0;
                    kvq_progressive_requant(a.c, layer, -1, page, nullptr, &done);
                    refused_changes_nothing = false;
                }
            } else if (what < 7) {
                const int n = R(0, 2) ? -1 : R(-2, b.tokens(layer) + 2);
                st = kvq_cache_fork(a.c, b.c, layer, R(0, 3) ? map.data() : nullptr, n, nullptr);
                if (st == KVQ_OK) {
                    auto w = b.widths(layer);
                    if (i == k) w = before;
                    if (n >= 0) w.resize((size_t)n);
                    CHECK(a.widths(layer) == w, "widths behind a fork");
                }
            } else if (what == 7) {
                const int n = R(-1, old + 1);
                st = kvq_cache_truncate(a.c, layer, n, nullptr);
                if (st == KVQ_OK) {
                    auto w = before;
                    w.resize((size_t)n);
                    CHECK(a.widths(layer) == w, "widths behind a cut");
                }
            } else if (what == 8 && device) {
                st = kvq_cache_read(a.c, layer, 0, R(0, old + 1), input, input, R(0, 1), nullptr);
            } else if (R(0, 3) == 0) {
                CHECK(kvq_cache_reset(a.c, layer) == KVQ_OK, "reset");
                unusable[(size_t)i].erase(layer);
                refused_changes_nothing = false;
            }
            const bool failed = fail_launch >= 0 && launches > fail_launch;
            fail_launch = -1;
            CHECK(st != KVQ_E_HIP || failed, "a failure without a failing launch");
            if (unusable[(size_t)i].count(layer)) CHECK(st != KVQ_OK || refused_changes_nothing == false || what >= 8, "a block that is unusable");
            if (st == KVQ_E_HIP && a.c->layers[(size_t)layer].poisoned) unusable[(size_t)i].insert(layer);
            if (st != KVQ_OK && st != KVQ_E_HIP && refused_changes_nothing)
                CHECK(a.widths(layer) == before && kvq_cache_arena_free_bytes(a.c) == free, "a refused call (%s) has changed the block", kvq_status_string(st));
            for (int x = 0; x < 3; ++x) caches[(size_t)x]->check(unusable[(size_t)x]);
            if (failures) { printf("seed %d call %d what %d\n", seed, op, what); return; }
        }
        for (auto& c : caches) {
            CHECK(kvq_cache_reset(c->c, -1) == KVQ_OK && kvq_cache_arena_free_bytes(c->c) == c->whole, "an emptied cache holds its arena");
        }
    }
}

// One prompt of 35,840 tokens into 8,191 sequences: fewer pages go into a launch, which has less than 2^32 threads.
void many_units() {
    Cache src(1, 8, 256, 256 * 150, 30, KVQ_POLICY_PAPER, 0, 0, ~0ull >> 1, true), dst(8191, 8, 256, 256 * 150, 30, KVQ_POLICY_PAPER, 0, 0, ~0ull >> 1, true);
    CHECK(kvq_quantize_append(src.c, 0, input, input, 256 * 140, 2, nullptr) == KVQ_OK, "append");
    const kvq_status_t st = kvq_cache_fork(dst.c, src.c, 0, nullptr, -1, nullptr);
    CHECK(st == KVQ_OK && dst.tokens() == 256 * 140, "%s, %d tokens", kvq_status_string(st), dst.tokens());
    dst.check();
    // read-back of more tiles than a launch takes is refused with nothing enqueued
    const int before = launches;
    CHECK(kvq_cache_read(dst.c, 0, 0, 256 * 100, input, input, 0, nullptr) == KVQ_E_INVALID && launches == before, "read");
    CHECK(kvq_cache_read(dst.c, 0, 0, 256 * 60, input, input, 0, nullptr) == KVQ_OK, "read");
}

}  // namespace

int main(int argc, char** argv) {
    const std::string what = argc > 1 ? argv[1] : "";
    if (what == "random_calls") random_calls(true);
    else if (what == "random_calls_without_a_device") random_calls(false);
    else if (what == "many_units") many_units();
    else return 2;
    if (failures) return 1;
    printf("ok\n");
    return 0;
}
