// Host side of the encoder's layers (ifvs_layers_* and the operators declared
// with them in include/ifvs.h): the handle, argument checks, workspace and
// stream order.
#include <math.h>
#include <stdlib.h>
#include <string.h>

#include <new>

#include "layers.cuh"
#include "scan_common.cuh"

using namespace ifvs;

thread_local int ifvs::launches_to_failure = 0;

namespace {
// A workspace that a captured graph may still use
struct Retired {
    uint8_t* p;
    Retired* next;
};
}  // namespace

struct ifvs_layers {
    int device = 0, num_sms = 0;
    cudaStream_t own = nullptr;
    cudaEvent_t done = nullptr;     // after the last enqueued call that used the workspace
    uint8_t* work = nullptr;
    size_t work_bytes = 0;
    bool work_captured = false;     // a captured graph holds its address
    bool may_stall = false;         // waits may be made to run out
    bool may_fail = false;          // launches may be made to fail
    Retired* retired = nullptr;
    int* err_host = nullptr;        // the error words, page-locked
    int* err = nullptr;             // their device address
};

namespace {

int fail(cudaError_t e, const char* what, int line) {
    cudaGetLastError();
    return report_error(e == cudaErrorMemoryAllocation ? IFVS_ERR_OOM : IFVS_ERR_CUDA, "%s failed: %s (layers.cu:%d)",
                        what, cudaGetErrorString(e), line);
}

#define CUDA_TRY(x)                                               \
    do {                                                          \
        const cudaError_t e_ = (x);                               \
        if (e_ != cudaSuccess) return fail(e_, #x, __LINE__);     \
    } while (0)

#define TRY(x)                    \
    do {                          \
        const int rc_ = (x);      \
        if (rc_ != 0) return rc_; \
    } while (0)

// What the kernels found since the last look, the gravest first.  A word is read
// and cleared in one step: kernels of other streams may still store.
int take_error(ifvs_layers* L) {
    int e[kErrWords];
    for (int i = 0; i < kErrWords; ++i) e[i] = __atomic_exchange_n(L->err_host + i, 0, __ATOMIC_ACQ_REL);
    if (e[kErrWait]) return report_error(IFVS_ERR_TIMEOUT, "a bounded wait inside a kernel ran out");
    if (e[kErrId]) return report_error(IFVS_ERR_ARG, "a token id is outside -1..V-1");
    if (e[kErrOffsets]) return report_error(IFVS_ERR_ARG, "offsets must start at 0, end at T and not decrease");
    return IFVS_OK;
}

// One call's place in the handle's order: begin, the launches, end.
struct Call {
    ifvs_layers* L;
    DeviceGuard guard;
    cudaStream_t s;
    bool waits, ordered = false;

    Call(ifvs_layers* l, void* stream)
        : L(l), guard(l->device), s(stream ? (cudaStream_t)stream : l->own), waits(stream == nullptr) {}

    // bytes: of workspace (0: the call has no place in the order of those that use it)
    int begin(size_t bytes) {
        if (!guard.ok) return report_error(IFVS_ERR_CUDA, "device %d cannot be made current", L->device);
        const char* n = L->may_fail ? getenv("IFVS_FAIL_LAUNCH") : nullptr;
        launches_to_failure = n ? atoi(n) : 0;
        if (bytes == 0) return 0;
        cudaStreamCaptureStatus st = cudaStreamCaptureStatusNone;
        if (!waits) CUDA_TRY(cudaStreamIsCapturing(s, &st));
        // in a capture the order of the graph's launches is the caller's
        ordered = st == cudaStreamCaptureStatusNone;
        if (bytes > L->work_bytes) {
            if (!ordered) return report_error(IFVS_ERR_STATE, "the workspace would have to grow during a stream capture");
            CUDA_TRY(cudaEventSynchronize(L->done));
            if (L->work && L->work_captured) {
                Retired* r = new (std::nothrow) Retired{L->work, L->retired};
                if (!r) return report_error(IFVS_ERR_OOM, "out of host memory");
                L->retired = r;
            } else if (L->work) {
                cudaFree(L->work);
            }
            L->work = nullptr;
            L->work_bytes = 0;
            L->work_captured = false;
            void* p = nullptr;
            const cudaError_t e = device_malloc(&p, bytes);
            if (e != cudaSuccess) {
                cudaGetLastError();
                return report_error(IFVS_ERR_OOM, "device allocation of %zu bytes failed: %s", bytes,
                                    cudaGetErrorString(e));
            }
            L->work = (uint8_t*)p;
            L->work_bytes = bytes;
        }
        if (ordered)
            CUDA_TRY(cudaStreamWaitEvent(s, L->done, 0));
        else
            L->work_captured = true;
        return 0;
    }
    // launched: of the call's launches.  Kernels enqueued before one that failed use
    // the workspace and the arrays like those of a whole call.
    int end(cudaError_t launched) {
        const int rc = launched == cudaSuccess ? IFVS_OK : fail(launched, "a launch", __LINE__);
        cudaError_t e = ordered ? cudaEventRecord(L->done, s) : cudaSuccess;
        if (e == cudaSuccess && waits) e = cudaStreamSynchronize(s);
        if (rc != IFVS_OK) return rc;
        if (e != cudaSuccess) return fail(e, "the call's end", __LINE__);
        return waits ? take_error(L) : IFVS_OK;
    }
};

bool aligned(const void* p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

// Waits run out after half a second; those that a test makes run out, after 32 ms.
// Looking for the test's variable takes 0.5 us: only handles that were created
// while it was there do, in every call.
Waits waits_of(const ifvs_layers* L) {
    if (L->may_stall && stall_copies_for_tests()) return {L->err, 16u, 1ll << 26};
    return {L->err, 0u, kWaitCycles};
}

int check_type(int type) {
    if (type != IFVS_T_F32 && type != IFVS_T_F16 && type != IFVS_T_BF16)
        return report_error(IFVS_ERR_ARG, "unknown element type %d", type);
    return 0;
}
int check_tokens(int64_t T) {
    if (T < 0 || T > 0x7FFFFFFFLL) return report_error(IFVS_ERR_ARG, "T = %lld outside 0..2^31 - 1", (long long)T);
    return 0;
}
int check_width(int D) {
    if (D < 1 || D > IFVS_MAX_WIDTH) return report_error(IFVS_ERR_ARG, "D = %d outside 1..%d", D, IFVS_MAX_WIDTH);
    return 0;
}
// an array that has to be there, aligned to `to` bytes
int check_array(const void* p, size_t to, const char* name) {
    if (!p) return report_error(IFVS_ERR_ARG, "%s is NULL", name);
    if (!aligned(p, to)) return report_error(IFVS_ERR_ARG, "%s is not aligned to %zu bytes", name, to);
    return 0;
}
int check_optional(const void* p, size_t to, const char* name) { return p ? check_array(p, to, name) : 0; }

int embed_check(const ifvs_layers* L, const int32_t* ids, int64_t T, int64_t V, int D, int type, float scale,
                EmbedArgs* a) {
    if (!L) return report_error(IFVS_ERR_ARG, "the handle is NULL");
    TRY(check_type(type));
    TRY(check_tokens(T));
    TRY(check_width(D));
    if (V < 1 || V > 0x7FFFFFFFLL) return report_error(IFVS_ERR_ARG, "V = %lld outside 1..2^31 - 1", (long long)V);
    if (!isfinite(scale)) return report_error(IFVS_ERR_ARG, "scale is not finite");
    if (T > 0) TRY(check_array(ids, 4, "ids"));
    *a = EmbedArgs{ids, T, V, D, type, scale, waits_of(L), L->num_sms};
    return 0;
}

int join_check(const ifvs_layers* L, const ifvs_join_params* p, bool block, JoinArgs* a) {
    if (!L || !p) return report_error(IFVS_ERR_ARG, "the handle or params is NULL");
    TRY(check_type(p->type));
    TRY(check_tokens(p->T));
    TRY(check_width(p->D));
    const size_t e = elem_bytes(p->type);
    if (p->n_seq < 1 || p->n_seq > 0x7FFFFFFFLL)
        return report_error(IFVS_ERR_ARG, "n_seq = %lld outside 1..2^31 - 1", (long long)p->n_seq);
    if (!p->offsets && p->n_seq != 1) return report_error(IFVS_ERR_ARG, "offsets is NULL with n_seq = %lld", (long long)p->n_seq);
    TRY(check_optional(p->offsets, 8, "offsets"));
    if (!(p->eps > 0.f) || !isfinite(p->eps)) return report_error(IFVS_ERR_ARG, "eps must be positive and finite");
    if (!isfinite(p->res_scale)) return report_error(IFVS_ERR_ARG, "res_scale is not finite");
    TRY(check_optional(p->gate, e, "gate"));
    TRY(check_optional(p->w_pre, e, "w_pre"));
    if (block)
        TRY(check_array(p->w_post, e, "w_post"));
    else if (p->w_post || p->gate)
        return report_error(IFVS_ERR_ARG, "w_post and gate must be NULL without y");
    *a = JoinArgs{p->T, p->n_seq, p->D, p->type, p->n_seq == 1 ? nullptr : p->offsets, p->offsets, p->gate, p->w_post, p->w_pre,
                  block ? p->res_scale : 1.f, p->eps, waits_of(L), L->num_sms};
    return 0;
}

int ffn_check(const ifvs_layers* L, const ifvs_ffn_params* p, FfnArgs* a) {
    if (!L || !p) return report_error(IFVS_ERR_ARG, "the handle or params is NULL");
    TRY(check_type(p->type));
    TRY(check_tokens(p->T));
    TRY(check_width(p->D));
    if (p->F < 1 || p->F > IFVS_MAX_HIDDEN) return report_error(IFVS_ERR_ARG, "F = %d outside 1..%d", p->F, IFVS_MAX_HIDDEN);
    if (p->act != IFVS_ACT_SILU && p->act != IFVS_ACT_GELU && p->act != IFVS_ACT_RELU)
        return report_error(IFVS_ERR_ARG, "unknown activation %d", p->act);
    if (p->type == IFVS_T_F32) return report_error(IFVS_ERR_UNSUPPORTED, "the feed-forward block takes 16-bit types only");
    if (p->D % 8 || p->F % 8)
        return report_error(IFVS_ERR_UNSUPPORTED, "D = %d and F = %d must be multiples of 8", p->D, p->F);
    TRY(check_array(p->w_in, 16, "w_in"));
    TRY(check_array(p->w_out, 16, "w_out"));
    *a = FfnArgs{p->T, p->D, p->F, p->type, p->act, p->w_in, p->w_out, waits_of(L), L->num_sms};
    return 0;
}

}  // namespace

extern "C" {

int ifvs_layers_create(ifvs_layers** out, int32_t device) {
    if (!out) return report_error(IFVS_ERR_ARG, "out is NULL");
    *out = nullptr;
    int ndev = 0;
    if (cudaGetDeviceCount(&ndev) != cudaSuccess || ndev == 0) {
        cudaGetLastError();
        return report_error(IFVS_ERR_CUDA, "no CUDA device is available");
    }
    if (device < 0 || device >= ndev) return report_error(IFVS_ERR_ARG, "device %d outside 0..%d", device, ndev - 1);
    DeviceGuard guard(device);
    ifvs_layers* L = new (std::nothrow) ifvs_layers;
    if (!L) return report_error(IFVS_ERR_OOM, "out of host memory");
    L->device = device;
    L->may_stall = getenv("IFVS_TEST_STALL_COPIES") != nullptr;
    L->may_fail = getenv("IFVS_FAIL_LAUNCH") != nullptr;
    void *h = nullptr, *d = nullptr;
    cudaError_t e = cudaDeviceGetAttribute(&L->num_sms, cudaDevAttrMultiProcessorCount, device);
    // blocking: ordered after the caller's work on the legacy default stream
    if (e == cudaSuccess) e = cudaStreamCreateWithFlags(&L->own, cudaStreamDefault);
    if (e == cudaSuccess) e = cudaEventCreateWithFlags(&L->done, cudaEventDisableTiming);
    if (e == cudaSuccess) e = cudaHostAlloc(&h, kErrWords * sizeof(int), cudaHostAllocMapped | cudaHostAllocPortable);
    if (e == cudaSuccess) {
        L->err_host = (int*)h;
        memset(h, 0, kErrWords * sizeof(int));
        e = cudaHostGetDevicePointer(&d, h, 0);
        L->err = (int*)d;
    }
    if (e != cudaSuccess) {
        ifvs_layers_free(L);
        return fail(e, "ifvs_layers_create", __LINE__);
    }
    *out = L;
    return IFVS_OK;
}

void ifvs_layers_free(ifvs_layers* L) {
    if (!L) return;
    DeviceGuard guard(L->device);
    cudaDeviceSynchronize();        // kernels may still write the error words
    if (L->done) cudaEventDestroy(L->done);
    if (L->work) cudaFree(L->work);
    while (Retired* r = L->retired) {
        L->retired = r->next;
        cudaFree(r->p);
        delete r;
    }
    if (L->own) cudaStreamDestroy(L->own);
    if (L->err_host) cudaFreeHost(L->err_host);
    cudaGetLastError();
    delete L;
}

int ifvs_layers_status(ifvs_layers* L) {
    if (!L) return report_error(IFVS_ERR_ARG, "the handle is NULL");
    DeviceGuard guard(L->device);
    CUDA_TRY(cudaDeviceSynchronize());
    return take_error(L);
}

int ifvs_embed(ifvs_layers* L, const void* table, int64_t V, int32_t D, int32_t type, const int32_t* ids, int64_t T,
               float scale, void* out, void* stream) {
    EmbedArgs a;
    TRY(embed_check(L, ids, T, V, D, type, scale, &a));
    TRY(check_array(table, elem_bytes(type), "table"));
    if (T > 0) TRY(check_array(out, elem_bytes(type), "out"));
    Call c(L, stream);
    TRY(c.begin(0));
    return c.end(T > 0 ? launch_embed(a, table, out, c.s) : cudaSuccess);
}

int ifvs_embed_grad(ifvs_layers* L, const void* d_out, const int32_t* ids, int64_t T, int64_t V, int32_t D, int32_t type,
                    float scale, void* d_table, void* stream) {
    EmbedArgs a;
    TRY(embed_check(L, ids, T, V, D, type, scale, &a));
    if (T > 0) TRY(check_array(d_out, elem_bytes(type), "d_out"));
    TRY(check_array(d_table, elem_bytes(type), "d_table"));
    Call c(L, stream);
    TRY(c.begin(embed_grad_bytes(a)));
    return c.end(launch_embed_grad(a, d_out, d_table, L->work, c.s));
}

int ifvs_norm_join(ifvs_layers* L, const ifvs_join_params* p, const void* x, const void* y, void* x_out, void* n_out) {
    JoinArgs a;
    TRY(join_check(L, p, y != nullptr, &a));
    const size_t e = elem_bytes(a.type);
    if ((n_out == nullptr) != (a.w_pre == nullptr)) return report_error(IFVS_ERR_ARG, "n_out and w_pre go together");
    if ((x_out == nullptr) != (y == nullptr)) return report_error(IFVS_ERR_ARG, "x_out and y go together");
    if (!y && !n_out) return report_error(IFVS_ERR_ARG, "nothing to compute: y and n_out are NULL");
    TRY(check_optional(y, e, "y"));
    TRY(check_optional(x_out, e, "x_out"));
    TRY(check_optional(n_out, e, "n_out"));
    TRY(check_array(x, e, "x"));
    Call c(L, p->stream);
    TRY(c.begin(0));
    return c.end(launch_norm_join(a, x, y, x_out, n_out, c.s));
}

int ifvs_norm_join_grad(ifvs_layers* L, const ifvs_join_params* p, const void* x_out, const void* y, const void* d_x_out,
                        const void* d_n, void* dx, void* dy, void* d_gate, void* d_w_post, void* d_w_pre) {
    JoinArgs a;
    TRY(join_check(L, p, y != nullptr, &a));
    const size_t e = elem_bytes(a.type);
    if (!d_x_out && !d_n) return report_error(IFVS_ERR_ARG, "d_x_out and d_n are NULL");
    if ((d_n == nullptr) != (d_w_pre == nullptr)) return report_error(IFVS_ERR_ARG, "d_n and d_w_pre go together");
    if (d_n && !a.w_pre) return report_error(IFVS_ERR_ARG, "d_n needs w_pre");
    if ((y == nullptr) != (dy == nullptr) || (y == nullptr) != (d_w_post == nullptr))
        return report_error(IFVS_ERR_ARG, "y, dy and d_w_post go together");
    if (d_gate && (!y || !a.gate)) return report_error(IFVS_ERR_ARG, "d_gate needs y and gate");
    TRY(check_array(x_out, e, "x_out"));
    TRY(check_array(dx, e, "dx"));
    TRY(check_optional(y, e, "y"));
    TRY(check_optional(d_x_out, e, "d_x_out"));
    TRY(check_optional(d_n, e, "d_n"));
    TRY(check_optional(dy, e, "dy"));
    TRY(check_optional(d_gate, e, "d_gate"));
    TRY(check_optional(d_w_post, e, "d_w_post"));
    TRY(check_optional(d_w_pre, e, "d_w_pre"));
    Call c(L, p->stream);
    TRY(c.begin(norm_join_grad_bytes(a)));
    const JoinGrads g{x_out, y, d_x_out, d_n, dx, dy, d_gate, d_w_post, d_w_pre};
    return c.end(launch_norm_join_grad(a, g, L->work, c.s));
}

int ifvs_ffn(ifvs_layers* L, const ifvs_ffn_params* p, const void* x, void* y) {
    FfnArgs a;
    TRY(ffn_check(L, p, &a));
    if (a.T > 0) {
        TRY(check_array(x, 16, "x"));
        TRY(check_array(y, 16, "y"));
    }
    Call c(L, p->stream);
    TRY(c.begin(ffn_bytes(a)));
    return c.end(a.T > 0 ? launch_ffn(a, x, y, L->work, c.s) : cudaSuccess);
}

int ifvs_ffn_grad(ifvs_layers* L, const ifvs_ffn_params* p, const void* x, const void* dy, void* dx, void* d_w_in,
                  void* d_w_out) {
    FfnArgs a;
    TRY(ffn_check(L, p, &a));
    if (a.T > 0) {
        TRY(check_array(x, 16, "x"));
        TRY(check_array(dy, 16, "dy"));
        TRY(check_array(dx, 16, "dx"));
    }
    TRY(check_array(d_w_in, 16, "d_w_in"));
    TRY(check_array(d_w_out, 16, "d_w_out"));
    Call c(L, p->stream);
    TRY(c.begin(ffn_grad_bytes(a)));
    return c.end(launch_ffn_grad(a, x, dy, dx, d_w_in, d_w_out, L->work, c.s));
}

}  // extern "C"
