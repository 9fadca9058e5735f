// C ABI of the 16-bit attention (declared in include/sna.h): checks of arguments and the choice of kernels.
#include <algorithm>

#include "sna_attend.cuh"

namespace sna {
namespace attend {
namespace {

bool multiple_of_8(const sna_tensor_t& t) { return ((uintptr_t)t.data & 15u) == 0 && ((t.batch | t.head | t.lat | t.lon) & 7) == 0; }

// One stride for all points of a tensor; false if they do not lie in one line.
bool view_of(const sna_tensor_t& t, int nlat, int nlon, View& view) {
    view = View{t.data, t.batch, t.head, nlon > 1 ? t.lon : t.lat};
    return nlat <= 1 || nlon <= 1 || t.lat == nlon * t.lon;
}

sna_status_t describe(const sna_attention_t* a, sna_dtype_t dtype, bool backward, Problem& p) {
    if (a == nullptr) return fail(SNA_ERR_INVALID_ARG, "the problem is NULL");
    if (dtype != SNA_BFLOAT16 && dtype != SNA_FLOAT16) return fail(SNA_ERR_UNSUPPORTED, "dtype %d unsupported (bfloat16 or float16)", (int)dtype);
    if (a->B < 0 || a->Hq < 0 || a->Hk < 0 || a->nlat_q < 0 || a->nlon_q < 0 || a->nlat_k < 0 || a->nlon_k < 0) return fail(SNA_ERR_INVALID_ARG, "sizes must not be negative");
    if (a->C < 8 || a->C > 128 || a->C % 8 != 0) return fail(SNA_ERR_UNSUPPORTED, "C=%d unsupported (a multiple of 8 between 8 and 128)", a->C);
    if (a->Hk > 0 ? a->Hq % a->Hk != 0 : a->Hq != 0) return fail(SNA_ERR_INVALID_ARG, "Hq=%d must be a multiple of Hk=%d", a->Hq, a->Hk);
    if (!(a->scale > -1e30f && a->scale < 1e30f)) return fail(SNA_ERR_INVALID_ARG, "scale must be finite");
    const int64_t Nq = (int64_t)a->nlat_q * a->nlon_q, Nk = (int64_t)a->nlat_k * a->nlon_k, most = (int64_t)1 << 30;
    if (Nq >= most || Nk >= most || (int64_t)a->Hq * Nq >= most || (int64_t)a->Hk * Nk >= most || (int64_t)a->B * a->Hq * Nq >= 64 * most || (int64_t)a->B * a->Hk * Nk >= 64 * most ||
        (int64_t)a->B * a->Hq >= most)
        return fail(SNA_ERR_UNSUPPORTED, "problem too large: heads * points must be less than 2^30, and 2^36 over the batch");
    p = Problem{};
    p.B = a->B; p.Hq = a->Hq; p.Hk = a->Hk; p.G = a->Hk > 0 ? a->Hq / a->Hk : 1; p.Nq = (int)Nq; p.Nk = (int)Nk; p.C = a->C;
    p.scale = a->scale; p.scale_log2 = a->scale * LOG2E;
    p.lse = a->lse; p.log_weights = a->log_weights; p.log_weights_batch = a->log_weights_batch;
    if (((uintptr_t)a->lse | (uintptr_t)a->log_weights) & 3u) return fail(SNA_ERR_INVALID_ARG, "lse and log_weights must be 4-byte aligned");
    struct { const sna_tensor_t& t; View& view; bool used, query; } tensors[] = {
        {a->q, p.q, true, true},          {a->k, p.k, true, false},       {a->v, p.v, true, false},       {a->out, p.out, true, true},
        {a->out_rest, p.rest, a->out_rest.data != nullptr, true},
        {a->dout, p.dout, backward, true}, {a->dq, p.dq, backward, true}, {a->dk, p.dk, backward, false}, {a->dv, p.dv, backward, false}};
    for (const auto& x : tensors) {
        if (!x.used) continue;
        if (!multiple_of_8(x.t)) return fail(SNA_ERR_INVALID_ARG, "data pointers and strides must be multiples of 8 elements");
        if (!view_of(x.t, x.query ? a->nlat_q : a->nlat_k, x.query ? a->nlon_q : a->nlon_k, x.view)) return fail(SNA_ERR_INVALID_ARG, "the points of a tensor must lie in one line (lat = nlon * lon)");
        const int64_t elements = (int64_t)a->B * (x.query ? a->Hq * Nq : a->Hk * Nk);
        if (elements > 0 && x.t.data == nullptr) return fail(SNA_ERR_INVALID_ARG, "a tensor's data is NULL");
    }
    if (backward && rows_of(p) > 0 && a->lse == nullptr) return fail(SNA_ERR_INVALID_ARG, "lse must not be NULL");
    return SNA_OK;
}

sna_status_t check_workspace(const void* workspace, size_t bytes, size_t need) {
    if (need == 0) return SNA_OK;
    if (workspace == nullptr || ((uintptr_t)workspace & 255u)) return fail(SNA_ERR_INVALID_ARG, "workspace must be non-NULL and 256-byte aligned");
    if (bytes < need) return fail(SNA_ERR_WORKSPACE, "workspace too small: %zu < %zu bytes", bytes, need);
    return SNA_OK;
}

// Which kernels: those on tcgen05 unless there are few queries (whose tiles of 128 and 256 rows per head would be nearly empty, while the mma.sync kernels stack
// the heads of a group) or few points.  us, mma.sync : tcgen05, bf16, C = 64, forward and (in brackets) with the backward pass: 32 heads, 32 x 1024
// 15.8 : 12.1 (56 : 41), 17 x 8192 41.8 : 27.0 (280 : 148), 65 x 128 7.7 : 6.9 (27 : 26); 128 heads, 512 x 64 20 : 16 (77 : 61), 128 x 64 7.5 : 7.9 (28 : 27);
// 4 heads, 64 x 8192 14.6 : 20.2 (193 : 57).
// On the other side of both limits the gradients are slow: the mma.sync kernels do not cut a walk over many keys (dq) or many queries (dk, dv) into pieces as their
// forward pass and the tcgen05 kernels do.  us, forward (and with the backward pass), B = 2, 8 and 2 heads of 64: 16 queries, 361x720 points 121 (6780), 17 queries
// 250 (926); 361x720 queries, 63 points 921 (60500), 64 points 743 (3100).
// The tcgen05 kernels find a row's maximum before the scores are scaled, and hold weights divided by the scale: it has to be positive, and not so small that
// a point left out could be taken for one with a low weight.
// (Without query heads there is no tile of queries, and dk and dv are zeros.)
bool on_tensor_memory(const Problem& p) { return p.G > 0 && p.Nq > 16 && p.Nk >= 64 && p.scale >= 0x1p-20f && p.scale <= 0x1p20f; }
// Pieces of a workspace, or with a null pointer their sizes alone.
struct Pieces {
    char* at;
    size_t bytes = 0;
    char* take(size_t size) {
        char* here = at == nullptr ? nullptr : at + bytes;
        bytes += align256(size);
        return here;
    }
    Selection selection(const Problem& p) {
        Selection sel{};
        if (!on_tensor_memory(p) || !selects(p)) return sel;
        const size_t copies = (size_t)p.B * p.Hk * p.Nk * p.C * 2;
        sel.taken = reinterpret_cast<int*>(take((size_t)p.B * sizeof(int)));
        sel.index = reinterpret_cast<int*>(take((size_t)p.B * p.Nk * sizeof(int)));
        sel.weights = reinterpret_cast<float*>(take((size_t)p.B * p.Nk * sizeof(float)));
        sel.k = take(copies);
        sel.v = take(copies);
        return sel;
    }
};

// What the forward pass needs to hold partial results, on either path (the tcgen05 kernels fall back where the driver refuses a tensor).
struct ForwardWorkspace {
    float* partials;
    Selection selection;
    size_t bytes;
};
ForwardWorkspace forward_workspace(const Problem& p, void* workspace, int sms) {
    Pieces pieces{static_cast<char*>(workspace)};
    const int splits = forward_splits(p, sms);
    const size_t simple = splits > 1 ? (size_t)splits * rows_of(p) * (1 + p.C) : 0;
    ForwardWorkspace w{};
    w.partials = reinterpret_cast<float*>(pieces.take(sizeof(float) * (on_tensor_memory(p) ? std::max(simple, partial_floats(p, Kernel::FORWARD, sms)) : simple)));
    w.selection = pieces.selection(p);
    w.bytes = pieces.bytes;
    return w;
}

struct BackwardWorkspace {
    Stats stats;
    Selection selection;
    float *dq_partials, *dkdv_partials;
    size_t bytes;
};
BackwardWorkspace backward_workspace(const Problem& p, void* workspace, int sms) {
    BackwardWorkspace w{};
    Pieces pieces{static_cast<char*>(workspace)};
    auto take = [&](size_t bytes) { return pieces.take(bytes); };
    const int64_t weight_blocks = weight_blocks_of(p, on_tensor_memory(p) && selects(p));
    w.stats.extra = reinterpret_cast<uint4*>(take((size_t)query_blocks_of(p) * 2 * STATS_BLOCK * sizeof(uint4)));
    w.stats.weights = reinterpret_cast<uint4*>(take((size_t)weight_blocks * STATS_BLOCK * sizeof(uint4)));
    w.stats.gone = reinterpret_cast<uint2*>(take((size_t)weight_blocks * sizeof(uint2)));
    w.stats.lse2 = reinterpret_cast<float*>(take((size_t)rows_of(p) * sizeof(float)));
    w.stats.D = reinterpret_cast<float*>(take((size_t)rows_of(p) * sizeof(float)));
    w.stats.norms = reinterpret_cast<uint32_t*>(take((size_t)p.B * p.Hk * 2 * sizeof(uint32_t)));
    w.dq_partials = reinterpret_cast<float*>(take(on_tensor_memory(p) ? sizeof(float) * partial_floats(p, Kernel::DQ, sms) : 0));
    w.dkdv_partials = reinterpret_cast<float*>(take(on_tensor_memory(p) ? sizeof(float) * partial_floats(p, Kernel::DKDV, sms) : 0));
    w.selection = pieces.selection(p);
    w.bytes = pieces.bytes;
    return w;
}

}  // namespace
}  // namespace attend
}  // namespace sna

using namespace sna::attend;

extern "C" {

size_t sna_attention_forward_workspace_bytes(const sna_attention_t* a, sna_dtype_t dtype) {
    Problem p;
    if (describe(a, dtype, false, p) != SNA_OK) return 0;
    const int sms = sna::sms_of_current_device();
    return sms == 0 ? 0 : forward_workspace(p, nullptr, sms).bytes;
}

sna_status_t sna_attention_forward(const sna_attention_t* a, sna_dtype_t dtype, void* workspace, size_t workspace_bytes, void* cuda_stream) {
    Problem p;
    sna_status_t st = describe(a, dtype, false, p);
    if (st != SNA_OK) return st;
    if (rows_of(p) == 0) return SNA_OK;
    const int sms = sna::sms_of_current_device();
    if (sms == 0) return sna::fail(SNA_ERR_CUDA, "no CUDA device");
    const ForwardWorkspace w = forward_workspace(p, workspace, sms);
    st = check_workspace(workspace, workspace_bytes, w.bytes);
    if (st != SNA_OK) return st;
    cudaStream_t stream = (cudaStream_t)cuda_stream;
    float* partials = w.partials;
    cudaError_t e = cudaSuccess;
    if (!on_tensor_memory(p) || !forward_tc(p, w.selection, dtype, sms, partials, stream, e)) {
        const int splits = forward_splits(p, sms);
        e = launch_forward(p, dtype, splits, partials, stream);
        if (e == cudaSuccess && splits > 1) e = launch_join(p, dtype, splits, partials, stream);
    }
    if (e != cudaSuccess) return sna::fail(SNA_ERR_CUDA, "attention launch: %s", cudaGetErrorString(e));
    return SNA_OK;
}

size_t sna_attention_backward_workspace_bytes(const sna_attention_t* a, sna_dtype_t dtype) {
    Problem p;
    if (describe(a, dtype, true, p) != SNA_OK) return 0;
    const int sms = sna::sms_of_current_device();
    return sms == 0 ? 0 : backward_workspace(p, nullptr, sms).bytes;
}

sna_status_t sna_attention_backward(const sna_attention_t* a, sna_dtype_t dtype, void* workspace, size_t workspace_bytes, void* cuda_stream) {
    Problem p;
    sna_status_t st = describe(a, dtype, true, p);
    if (st != SNA_OK) return st;
    const bool queries = rows_of(p) > 0, keys = (int64_t)p.B * p.Hk * p.Nk > 0;
    if (!queries && !keys) return SNA_OK;
    const int sms = sna::sms_of_current_device();
    if (sms == 0) return sna::fail(SNA_ERR_CUDA, "no CUDA device");
    const BackwardWorkspace w = backward_workspace(p, workspace, sms);
    st = check_workspace(workspace, workspace_bytes, w.bytes);
    if (st != SNA_OK) return st;
    cudaStream_t stream = (cudaStream_t)cuda_stream;
    const Stats& s = w.stats;
    cudaError_t e = launch_statistics(p, s, w.selection, dtype, stream);
    // (on_tensor_memory: there are queries and keys)
    if (e == cudaSuccess && on_tensor_memory(p) && backward_tc(p, s, w.selection, dtype, sms, w.dq_partials, w.dkdv_partials, stream, e)) {
        if (e == cudaSuccess) e = join_backward(p, w.selection, dtype, sms, w.dq_partials, w.dkdv_partials, stream);
    } else {
        if (e == cudaSuccess && queries) e = launch_backward_dq(p, s, dtype, stream);
        if (e == cudaSuccess && keys) e = launch_backward_dkdv(p, s, dtype, stream);
    }
    if (e != cudaSuccess) return sna::fail(SNA_ERR_CUDA, "attention backward launch: %s", cudaGetErrorString(e));
    return SNA_OK;
}

sna_status_t sna_debug_exercise_layer_wait(void* cuda_stream) {
    if (sna::sms_of_current_device() == 0) return sna::fail(SNA_ERR_CUDA, "no CUDA device");
    const cudaError_t e = launch_wait_probe((cudaStream_t)cuda_stream);
    if (e != cudaSuccess) return sna::fail(SNA_ERR_CUDA, "probe launch: %s", cudaGetErrorString(e));
    return SNA_OK;
}

sna_status_t sna_layer_check(void) {
    int status = 0;
    const cudaError_t e = read_status(&status);
    if (e != cudaSuccess) return sna::fail(SNA_ERR_CUDA, "reading the status word: %s", cudaGetErrorString(e));
    if (status != 0) return sna::fail(SNA_ERR_CUDA, "a kernel gave up on a bounded wait; its outputs are incomplete");
    return SNA_OK;
}

}  // extern "C"
