// Host-only driver (tests/test_host_threads.py): calls from several host
// threads on one stream.  The HIP calls and the kernel launchers are stand-ins:
// a call of several launches writes its own number into the stream's workspace
// ("the first launch"), rests, and looks whether it is still there ("the
// second").  Between the two no other call may have enqueued on the stream.
#include <atomic>
#include <chrono>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <mutex>
#include <thread>
#include <vector>

#include "tl_internal.h"
#include "tl_serve.h"

extern "C" {
hipError_t hipGetDevice(int* d) { *d = 0; return hipSuccess; }
hipError_t hipSetDevice(int) { return hipSuccess; }
hipError_t hipMalloc(void** p, size_t n) { *p = std::malloc(n); return *p ? hipSuccess : hipErrorOutOfMemory; }
hipError_t hipFree(void* p) { std::free(p); return hipSuccess; }
hipError_t hipStreamSynchronize(hipStream_t) { return hipSuccess; }
hipError_t hipMemcpy(void* d, const void* s, size_t n, hipMemcpyKind) { std::memcpy(d, s, n); return hipSuccess; }
hipError_t hipMemcpyAsync(void* d, const void* s, size_t n, hipMemcpyKind, hipStream_t) { std::memcpy(d, s, n); return hipSuccess; }
hipError_t hipStreamIsCapturing(hipStream_t, hipStreamCaptureStatus* s) { *s = hipStreamCaptureStatusNone; return hipSuccess; }
hipError_t hipDeviceGetAttribute(int*, hipDeviceAttribute_t, int) { return hipErrorInvalidValue; }
}

static std::atomic<int> bad{0}, inside{0}, most_inside{0}, calls{0}, arrivals{0};
#define CHECK(x) do { if (!(x)) { if (bad++ < 20) std::printf("%s:%d: %s\n", __FILE__, __LINE__, #x); } } while (0)

// Two launches of a call on stream 'stream' over the workspace 'ws' (1 MB at least).
static hipError_t two_launches(void* ws, hipStream_t stream) {
    static std::atomic<int> last[16];               // of a stream: the call that enqueued last
    const int me = ++calls, now = ++inside;
    for (int seen = most_inside; now > seen && !most_inside.compare_exchange_weak(seen, now);) {}
    std::atomic<int>& on = last[(reinterpret_cast<uintptr_t>(stream) >> 42) & 15];
    auto* words = static_cast<std::atomic<int>*>(ws);
    on = me;
    for (int i = 0; i < 4096; ++i) words[i * 64].store(me);
    std::this_thread::sleep_for(std::chrono::microseconds(300));
    CHECK(on == me);
    bool mine = true;
    for (int i = 0; i < 4096; ++i) mine = mine && words[i * 64].load() == me;
    CHECK(mine);
    --inside;
    return hipSuccess;
}

namespace tl {
hipError_t launch_repack(const void*, void*, int64_t, int64_t, const Layout&, bool, hipStream_t) { std::abort(); }
// K splits in two launches, or summed inside one: the sets of counters are used in turn, in the order of the launches
hipError_t launch_decode(const DecodeLaunch& d, hipStream_t stream) {
    if (!d.arrive) return d.split_k > 1 ? two_launches(d.ws, stream) : hipSuccess;
    static std::mutex mu;
    static const unsigned* next[16];
    std::this_thread::sleep_for(std::chrono::microseconds(50));
    std::lock_guard<std::mutex> lock(mu);
    const unsigned*& want = next[(reinterpret_cast<uintptr_t>(stream) >> 42) & 15];
    CHECK(!want || want == d.arrive);
    want = d.arrive + d.arrive_clear;
    ++arrivals;
    return hipSuccess;
}
hipError_t launch_splitk_reduce(const DecodeLaunch&, hipError_t, hipStream_t) { std::abort(); }
hipError_t launch_lgms(const DecodeLaunch&, int64_t, int, hipStream_t) { std::abort(); }
int lgms_ctas_per_cu(int) { std::abort(); }
hipError_t launch_prefill(const PrefillLaunch& q, hipStream_t stream) { return two_launches(q.ws, stream); }
hipError_t launch_view_load(const uint8_t*, int64_t, const ViewProgram&, uint8_t*, hipStream_t) { std::abort(); }
hipError_t launch_zero_u64(unsigned long long* p, hipStream_t) { std::memset(p, 0, kStateWords * sizeof *p); return hipSuccess; }
hipError_t launch_stream_read(const uint8_t*, int64_t, unsigned*, hipStream_t) { std::abort(); }
hipError_t scratch_address(float**) { std::abort(); }
int64_t kv_append_workgroups(const KvAppendLaunch&, int) { std::abort(); }
int64_t kv_read_workgroups(const KvView&, int, int64_t) { std::abort(); }
hipError_t launch_kv_append(const KvAppendLaunch&, int, int, hipStream_t) { std::abort(); }
hipError_t launch_kv_read(const KvView&, int, int, const int32_t*, int64_t, uint16_t*, uint16_t*, hipStream_t) { std::abort(); }
hipError_t launch_kv_keep(const KvKeepLaunch&, int, int, hipStream_t) { std::abort(); }
hipError_t launch_attn(const AttnLaunch& a, int, int, hipStream_t stream) {
    CHECK(a.split && a.ws);
    return two_launches(a.ws, stream);
}
int64_t verify_workspace_bytes(int64_t vocab, int64_t total, int, int) { return vocab * total; }
hipError_t launch_verify(const VerifyLaunch& a, hipStream_t stream) { return two_launches(a.ws, stream); }
}  // namespace tl

using namespace tl;

template <typename T = void>
static T* dp(int i) { return reinterpret_cast<T*>(uintptr_t(i) << 42); }

static void attn(int64_t len, int stream) {
    const tl_kv_cache c = {dp(1), dp(2), dp<uint8_t>(3), dp<uint8_t>(4), 1000, 64, 1, 128, 1};
    CHECK(tl_attn(dp(5), 128, &c, dp<int32_t>(6), 4096, dp<int32_t>(7), dp<int32_t>(8), nullptr, 0, 1, 1, 1, len, 1, 0.1f, dp(9), dp(stream)) == TL_OK);
}
static void verify(int64_t vocab, int stream) {
    CHECK(tl_verify(dp(10), TL_OUT_F32, vocab, dp<int32_t>(11), dp<int32_t>(12), dp<int32_t>(13), 1, 40, 40, nullptr, 0, dp<float>(14),
                    dp<float>(15), dp<float>(16), dp<int32_t>(17), dp<int32_t>(18), dp<int32_t>(19), dp(stream)) == TL_OK);
}
static void gemm(int64_t M, int64_t N, int64_t K, int S, int stream) {
    tl_layout_desc d = {};
    d.kind = TL_LAYOUT_TILE;
    d.elem_bytes = 2;
    d.G = 4096;
    d.block_rows = 32;
    d.split_k = S;
    CHECK(tl_gemm(dp(20), dp(21), dp(22), M, N, K, &d, TL_FETCH_BLOCK, dp(stream)) == TL_OK);
}

static void together(int threads, void (*work)(int)) {
    std::atomic<int> ready{0};
    std::vector<std::thread> all;
    for (int t = 0; t < threads; ++t)
        all.emplace_back([&, t] {
            for (++ready; ready < threads;) std::this_thread::yield();
            work(t);
        });
    for (std::thread& t : all) t.join();
}

int main() {
    // one stream, calls of several launches, workspaces that grow meanwhile
    together(4, [](int t) {
        for (int i = 0; i < 40; ++i) {
            if (t == 0) attn(4096 + i, 1);
            if (t == 1) verify(1000 + i * 40000, 1);
            if (t == 2) gemm(8, 10240, 8192, 0, 1);
            if (t == 3) gemm(128, 1024, 2048 + 64 * i, 0, 1);
        }
    });
    CHECK(calls == 160);
    CHECK(most_inside == 1);
    // one stream, counters used in turn
    together(4, [](int) {
        for (int i = 0; i < 40; ++i) gemm(1, 1024, 1024, 0, 2);
    });
    CHECK(arrivals == 160);
    // a release between calls: they keep what they use
    together(4, [](int t) {
        for (int i = 0; i < 40; ++i) {
            if (t == 0) tl_release();
            else if (t == 1) verify(500000, 3);
            std::this_thread::sleep_for(std::chrono::microseconds(100));
        }
    });
    // streams of their own do not wait for one another
    most_inside = 0;
    together(4, [](int t) {
        for (int i = 0; i < 40; ++i) verify(500000, 4 + t);
    });
    CHECK(most_inside > 1);
    tl_release();
    std::printf("host threads driver: %d unexpected results\n", bad.load());
    return bad ? 1 : 0;
}
