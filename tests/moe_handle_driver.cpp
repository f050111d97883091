// Host checks of the expert layer's handle (csrc/esp_moe.cu) without a GPU: the CUDA runtime is a fake that follows
// which work is ordered after which, which streams are being captured, and which memory a captured graph names. The
// kernels' launchers are stubs that record a piece of work.
//
//   moe_handle_driver NAME     runs the check NAME; exit code 0 and "ok", or a line for each fault

#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <map>
#include <set>
#include <string>
#include <vector>

#include "esp_moe_impl.h"

namespace {

struct Stream {
    bool capturing = false;
    bool broken = false;      // its capture was ended by a call that cannot be captured
    std::set<int> before;     // eager work that what comes next on the stream runs after
};

struct Event {
    std::set<int> before;
};

struct Work {
    bool captured;
    const void *ws;
};

Stream legacy;
std::vector<Work> works;
std::set<int> finished;                  // work that the host has waited for
std::map<const void *, size_t> memory;   // live blocks
std::set<const void *> in_graph;         // blocks that captured work names
std::vector<std::string> faults;
cudaStreamCaptureMode mode = cudaStreamCaptureModeGlobal;   // of the calling thread

void fault(const std::string &what)
{
    faults.push_back(what);
}

Stream &of(cudaStream_t s)
{
    return s ? *reinterpret_cast<Stream *>(s) : legacy;
}

std::vector<Stream *> streams;

cudaStream_t new_stream()
{
    streams.push_back(new Stream());
    return reinterpret_cast<cudaStream_t>(streams.back());
}

bool any_capturing()
{
    for (Stream *s : streams)
        if (s->capturing)
            return true;
    return false;
}

// An allocation or a release now: a capture forbids it, and is ended by it, unless the thread has relaxed that.
bool breaks_captures()
{
    if (!any_capturing() || mode == cudaStreamCaptureModeRelaxed)
        return false;
    for (Stream *s : streams)
        s->broken = s->broken || s->capturing;
    return true;
}

// A kernel queued on the handle's stream that uses its work space and counters.
cudaError_t work(esp_moe *m)
{
    Stream &s = of(m->stream);
    const int id = (int)works.size();
    works.push_back(Work{s.capturing, m->ws});
    if (m->ws && !memory.count(m->ws))
        fault("work " + std::to_string(id) + " uses freed memory");
    if (s.capturing) {
        in_graph.insert(m->ws);
        return cudaSuccess;
    }
    for (int i = 0; i < id; ++i)
        if (!works[i].captured && !s.before.count(i) && !finished.count(i))
            fault("work " + std::to_string(id) + " shares the work space with " + std::to_string(i) + " without order");
    s.before.insert(id);
    return cudaSuccess;
}

}  // namespace

// ---- the CUDA runtime that csrc/esp_moe.cu calls

extern "C" {

cudaError_t cudaGetLastError() { return cudaSuccess; }
cudaError_t cudaGetDevice(int *d)
{
    *d = 0;
    return cudaSuccess;
}
cudaError_t cudaSetDevice(int) { return cudaSuccess; }
cudaError_t cudaGetDeviceCount(int *n)
{
    *n = 1;
    return cudaSuccess;
}
cudaError_t cudaDeviceGetAttribute(int *v, cudaDeviceAttr a, int)
{
    *v = a == cudaDevAttrComputeCapabilityMajor ? 10 : a == cudaDevAttrComputeCapabilityMinor ? 3 : 152;
    return cudaSuccess;
}
cudaError_t cudaMalloc(void **p, size_t n)
{
    if (breaks_captures())
        return cudaErrorStreamCaptureUnsupported;
    *p = calloc(1, n < 4096 ? n : 4096);
    memory[*p] = n;
    return cudaSuccess;
}
cudaError_t cudaFree(void *p)
{
    if (breaks_captures())
        return cudaErrorStreamCaptureUnsupported;
    if (in_graph.count(p))
        fault("memory that a captured graph names is freed");
    if (!memory.erase(p))
        fault("memory is freed twice");
    for (size_t i = 0; i < works.size(); ++i)
        finished.insert((int)i);
    free(p);
    return cudaSuccess;
}
cudaError_t cudaHostAlloc(void **p, size_t n, unsigned int)
{
    if (breaks_captures())
        return cudaErrorStreamCaptureUnsupported;
    *p = calloc(1, n);
    return cudaSuccess;
}
cudaError_t cudaFreeHost(void *p)
{
    if (breaks_captures())
        return cudaErrorStreamCaptureUnsupported;
    free(p);
    return cudaSuccess;
}
cudaError_t cudaHostGetDevicePointer(void **d, void *h, unsigned int)
{
    *d = h;
    return cudaSuccess;
}
cudaError_t cudaMemset(void *p, int v, size_t n)
{
    memset(p, v, n);
    return cudaSuccess;
}
cudaError_t cudaStreamSynchronize(cudaStream_t s)
{
    if (of(s).capturing) {
        of(s).broken = true;
        return cudaErrorStreamCaptureUnsupported;
    }
    finished.insert(of(s).before.begin(), of(s).before.end());
    return cudaSuccess;
}
cudaError_t cudaStreamIsCapturing(cudaStream_t s, cudaStreamCaptureStatus *st)
{
    *st = of(s).capturing ? cudaStreamCaptureStatusActive : cudaStreamCaptureStatusNone;
    return cudaSuccess;
}
cudaError_t cudaThreadExchangeStreamCaptureMode(cudaStreamCaptureMode *m)
{
    std::swap(mode, *m);
    return cudaSuccess;
}
cudaError_t cudaEventCreateWithFlags(cudaEvent_t *e, unsigned int)
{
    *e = reinterpret_cast<cudaEvent_t>(new Event());
    return cudaSuccess;
}
cudaError_t cudaEventDestroy(cudaEvent_t e)
{
    delete reinterpret_cast<Event *>(e);
    return cudaSuccess;
}
cudaError_t cudaEventRecord(cudaEvent_t e, cudaStream_t s)
{
    if (of(s).capturing) {
        of(s).broken = true;
        return cudaErrorStreamCaptureUnsupported;
    }
    reinterpret_cast<Event *>(e)->before = of(s).before;
    return cudaSuccess;
}
cudaError_t cudaStreamWaitEvent(cudaStream_t s, cudaEvent_t e, unsigned int)
{
    if (of(s).capturing) {
        of(s).broken = true;
        return cudaErrorStreamCaptureIsolation;
    }
    const Event *ev = reinterpret_cast<Event *>(e);
    of(s).before.insert(ev->before.begin(), ev->before.end());
    return cudaSuccess;
}

}  // extern "C"

// ---- the launchers

namespace esp_moe_impl {

size_t route_hist_ints(int64_t T, int32_t E, int32_t) { return (size_t)(T * E); }
cudaError_t launch_route(esp_moe *m, int32_t, const RouteArgs &) { return work(m); }
int64_t balance_slots(int64_t T, int32_t B) { return T + B; }
cudaError_t launch_balance(esp_moe *m, int32_t, const BalanceArgs &) { return work(m); }
cudaError_t launch_route_backward(esp_moe *, int32_t, const RouteBackwardArgs &) { return cudaSuccess; }
cudaError_t launch_step_prices(esp_moe *, int32_t, const int64_t *, double, double, float *) { return cudaSuccess; }
cudaError_t launch_combine(esp_moe *, int32_t, const CombineArgs &) { return cudaSuccess; }
cudaError_t launch_combine_backward(esp_moe *, int32_t, const CombineArgs &) { return cudaSuccess; }
cudaError_t launch_quant_rows(esp_moe *m, int32_t, const QuantRowsArgs &) { return work(m); }
cudaError_t launch_pick_rows(esp_moe *m, const PickRowsArgs &) { return work(m); }
cudaError_t launch_quant_cols(esp_moe *m, int32_t, const QuantColsArgs &) { return work(m); }
cudaError_t launch_quant_weight(esp_moe *, int32_t, const void *, int64_t, const esp_moe_weight &) { return cudaSuccess; }
size_t gemm_partial_floats(const esp_moe *) { return 1024; }
cudaError_t launch_gemm_rows(esp_moe *m, int32_t, const GemmRowsArgs &) { return work(m); }
cudaError_t launch_gemm_cols(esp_moe *m, const GemmColsArgs &) { return work(m); }

}  // namespace esp_moe_impl

// ---- checks

namespace {

esp_moe *open(cudaStream_t s)
{
    esp_moe *m = nullptr;
    if (esp_moe_create(&m, 0, s) != ESP_OK)
        fault("create");
    return m;
}

// Work space grows with T.
esp_status route(esp_moe *m, int64_t T)
{
    static int32_t idx[1];
    static float weight[1], logits[1];
    static int64_t counts[1];
    const esp_moe_gate gate = {ESP_MOE_SOFTMAX, 1, 1.0f};
    return esp_moe_route(m, &gate, ESP_MOE_F32, T, 8, 1, 8, logits, nullptr, nullptr, idx, weight, counts, nullptr,
                         nullptr, nullptr);
}

void want(esp_status got, esp_status expected, const char *what)
{
    if (got != expected)
        fault(std::string(what) + ": status " + std::to_string((int)got));
}

// A graph is captured, then a larger call makes the work space grow: the graph's block stays.
void graph_keeps_its_block()
{
    cudaStream_t s = new_stream();
    esp_moe *m = open(s);
    want(route(m, 10), ESP_OK, "small call");
    of(s).capturing = true;
    want(route(m, 10), ESP_OK, "captured call");
    of(s).capturing = false;
    want(route(m, 1000), ESP_OK, "larger call");
    of(s).capturing = true;
    want(route(m, 1000), ESP_OK, "captured larger call");
    of(s).capturing = false;
    want(route(m, 5000), ESP_OK, "largest call");
    want(route(m, 9000), ESP_OK, "larger still");   // a block that no graph names goes at once
    if (memory.size() != 4)                         // the counters, two kept, the present one
        fault("blocks alive: " + std::to_string(memory.size()));
    in_graph.clear();                               // the graphs end before the handle
    esp_moe_destroy(m);
    if (!memory.empty())
        fault("memory left after the handle's end");
}

// A captured call that needs more work space gets it without touching the capture or the block in use.
void growing_while_captured()
{
    for (int64_t before : {0, 10}) {
        cudaStream_t s = new_stream();
        esp_moe *m = open(s);
        if (before)
            want(route(m, before), ESP_OK, "call before");
        of(s).capturing = true;
        want(route(m, 1000), ESP_OK, "captured call that grows");
        want(route(m, 3000), ESP_OK, "captured call that grows again");
        if (of(s).broken)
            fault("the capture is broken");
        of(s).capturing = false;
        want(route(m, 9000), ESP_OK, "call after");
        cudaStream_t other = new_stream();   // a capture that is not the handle's
        of(other).capturing = true;
        want(route(m, 20000), ESP_OK, "call beside a capture");
        if (of(other).broken)
            fault("the other capture is broken");
        of(other).capturing = false;
        if (mode != cudaStreamCaptureModeGlobal)
            fault("the thread's capture mode is left changed");
        in_graph.clear();
        esp_moe_destroy(m);
    }
}

// A handle made or destroyed (by a garbage collector, say) while some stream is being captured.
void handles_beside_a_capture()
{
    cudaStream_t s = new_stream(), other = new_stream();
    esp_moe *before = open(s);
    want(route(before, 10), ESP_OK, "call");
    of(other).capturing = true;
    esp_moe *m = open(s);
    if (m)
        esp_moe_destroy(m);
    esp_moe_destroy(before);
    if (of(other).broken)
        fault("the capture is broken");
    if (!memory.empty())
        fault("memory left after the handles' end");
    if (mode != cudaStreamCaptureModeGlobal)
        fault("the thread's capture mode is left changed");
}

// Work before a capture and work after it share the work space in order, whichever stream comes after.
void order_across_a_capture()
{
    for (int stay = 0; stay < 2; ++stay) {
        cudaStream_t a = new_stream(), b = new_stream(), c = new_stream();
        esp_moe *m = open(a);
        want(route(m, 10), ESP_OK, "call");
        of(b).capturing = true;
        want(esp_moe_set_stream(m, b), ESP_OK, "to the captured stream");
        want(route(m, 10), ESP_OK, "captured call");
        of(b).capturing = false;
        if (!stay)
            want(esp_moe_set_stream(m, c), ESP_OK, "to another stream");
        want(route(m, 10), ESP_OK, "call after");
        want(esp_moe_set_stream(m, a), ESP_OK, "back");
        want(route(m, 10), ESP_OK, "last call");
        in_graph.clear();
        esp_moe_destroy(m);
    }
}

// A capture that began on the handle's own stream, after work of the handle there: no order can be had until it ends.
void order_after_a_capture_in_place()
{
    cudaStream_t a = new_stream(), b = new_stream();
    esp_moe *m = open(a);
    want(route(m, 10), ESP_OK, "call");
    of(a).capturing = true;
    want(route(m, 10), ESP_OK, "captured call");
    want(esp_moe_set_stream(m, b), ESP_ERR_STATE, "to another stream during the capture");
    want(route(m, 10), ESP_OK, "captured call after the refusal");
    of(b).capturing = true;
    want(esp_moe_set_stream(m, b), ESP_OK, "to a captured stream");
    want(route(m, 10), ESP_OK, "call captured there");
    of(b).capturing = false;
    want(route(m, 10), ESP_ERR_STATE, "a call there that nothing orders");
    of(a).capturing = false;
    if (of(a).broken || of(b).broken)
        fault("a capture is broken");
    want(route(m, 10), ESP_OK, "call after");
    in_graph.clear();
    esp_moe_destroy(m);
}

// Waiting for the handle reaches work on the stream before a capture, and is refused during one.
void synchronize_across_a_capture()
{
    cudaStream_t a = new_stream(), b = new_stream();
    esp_moe *m = open(a);
    want(route(m, 10), ESP_OK, "call");
    of(b).capturing = true;
    want(esp_moe_set_stream(m, b), ESP_OK, "to the captured stream");
    want(route(m, 10), ESP_OK, "captured call");
    want(esp_moe_synchronize(m), ESP_ERR_STATE, "waiting during the capture");
    if (of(b).broken)
        fault("the capture is broken");
    of(b).capturing = false;
    want(esp_moe_synchronize(m), ESP_OK, "waiting");
    if (!finished.count(0))
        fault("work before the capture was not waited for");
    in_graph.clear();
    esp_moe_destroy(m);
}

// A wait that ran out is reported by the next call of any kind, once; then the handle refuses work.
void timeout_is_reported_by_the_next_call()
{
    for (int way = 0; way < 3; ++way) {
        cudaStream_t a = new_stream(), b = new_stream();
        esp_moe *m = open(a);
        want(route(m, 10), ESP_OK, "call");
        *m->d_err = 1u;   // as a kernel does
        want(way == 0 ? route(m, 10) : way == 1 ? esp_moe_set_stream(m, b) : esp_moe_synchronize(m), ESP_ERR_TIMEOUT,
             "next call");
        want(route(m, 10), ESP_ERR_STATE, "call after");
        want(esp_moe_synchronize(m), ESP_ERR_STATE, "waiting after");
        esp_moe_destroy(m);
    }
}

const std::map<std::string, void (*)()> checks = {
    {"growing_while_captured", growing_while_captured},
    {"graph_keeps_its_block", graph_keeps_its_block},
    {"handles_beside_a_capture", handles_beside_a_capture},
    {"order_across_a_capture", order_across_a_capture},
    {"order_after_a_capture_in_place", order_after_a_capture_in_place},
    {"synchronize_across_a_capture", synchronize_across_a_capture},
    {"timeout_is_reported_by_the_next_call", timeout_is_reported_by_the_next_call},
};

}  // namespace

int main(int argc, char **argv)
{
    const auto it = argc == 2 ? checks.find(argv[1]) : checks.end();
    if (it == checks.end()) {
        for (const auto &c : checks)
            printf("%s\n", c.first.c_str());
        return 2;
    }
    it->second();
    for (const std::string &f : faults)
        printf("%s\n", f.c_str());
    for (Stream *s : streams)
        delete s;
    if (faults.empty())
        printf("ok\n");
    return faults.empty() ? 0 : 1;
}
