// Rows of scores as distributions (hr_scores.h): log probabilities of given entries, entropy, best alternatives, a teacher's
// list, and the gradients of all of them.  A workgroup takes a row.
//
// Mathematics.  With s the scale, m the largest score of a row and t_i = exp(s (z_i - m)):  S0 = sum t_i >= 1,  S1 = sum s (z_i - m) t_i <= 0,
//   ln p_i = s (z_i - m) - ln S0,      entropy = ln S0 - S1 / S0  (two terms that are not negative: nothing cancels).
// Every thread keeps m, S0, S1 of the chunks it has seen (float32; a larger maximum rescales the sums) and the threads' are
// merged in a fixed order at the end.  Exponents are counted in base 2: one multiplication by s / ln 2 serves scale and base.
#include "entry.h"
#include "row_math.h"

namespace hr {

// ---- best k of a row: keys of (score, entry) in one 64-bit number, larger is better, no two alike
__device__ __forceinline__ uint64_t entry_key(float z, int i) { return (uint64_t)order_key(z) << 32 | (uint32_t)~i; }
constexpr uint64_t kNoKey = (uint64_t)kNoCandidate << 32 | 0xffffffffu;      // every candidate's is larger

template <int THREADS>
struct TopBuffer {
    static constexpr int kCap = 1024;
    uint64_t key[kCap];
    int fill, valid;
    uint64_t bound;                     // key of the k-th best seen so far
};

// The best k of the first `fill` keys go to the front, best first (ranked by counting); returns how many there are.
template <int THREADS>
__device__ int rank_best(TopBuffer<THREADS>& b, int fill, int k)
{
    uint64_t mine[TopBuffer<THREADS>::kCap / THREADS];
    int rank[TopBuffer<THREADS>::kCap / THREADS];
    __syncthreads();
    for (int r = 0; r * THREADS < fill; ++r) {
        const int i = r * THREADS + threadIdx.x;
        mine[r] = i < fill ? b.key[i] : 0;
        rank[r] = i < fill ? 0 : TopBuffer<THREADS>::kCap;
        for (int j = 0; j < fill; ++j) rank[r] += b.key[j] > mine[r];
    }
    __syncthreads();
    for (int r = 0; r * THREADS < fill; ++r)
        if (rank[r] < k) b.key[rank[r]] = mine[r];
    __syncthreads();
    return fill < k ? fill : k;
}

// Offers the chunk [c, c + THREADS) of the row, a chunk per thread, to the buffer.
template <typename T, int THREADS>
__device__ void offer_chunks(const Row<T>& row, int c, TopBuffer<THREADS>& b, int k)
{
    float v[Row<T>::E];
    int first = 0;
    bool pending = c + (int)threadIdx.x < row.nchunks;
    if (pending) first = row.load(c + threadIdx.x, v);
    for (;;) {
        if (threadIdx.x == 0) b.valid = TopBuffer<THREADS>::kCap;
        __syncthreads();
        int cnt = 0;
        if (pending)
            for (int e = 0; e < Row<T>::E; ++e) cnt += entry_key(v[e], first + e) > b.bound;
        if (pending && cnt == 0) pending = false;
        if (pending) {
            int pos = atomicAdd(&b.fill, cnt);
            if (pos + cnt <= TopBuffer<THREADS>::kCap) {
                for (int e = 0; e < Row<T>::E; ++e) {
                    const uint64_t key = entry_key(v[e], first + e);
                    if (key > b.bound) b.key[pos++] = key;
                }
                pending = false;
            } else {
                atomicMin(&b.valid, pos);
            }
        }
        // (a chunk that found no room: the best k are kept, the k-th is the new bound, and it is offered again)
        if (!__syncthreads_or(pending)) return;
        const int kept = rank_best(b, b.valid < b.fill ? b.valid : b.fill, k);
        if (threadIdx.x == 0) {
            b.fill = kept;
            if (kept == k) b.bound = b.key[k - 1];
        }
        __syncthreads();
    }
}

template <typename T, int THREADS>
__global__ __launch_bounds__(THREADS) void k_logprobs(LogprobsArgs a)
{
    __shared__ RowShared<THREADS> sh;
    __shared__ TopBuffer<THREADS> buf;
    const float c2 = a.scale * kLog2e;
    for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const Row<T> row(a.logits, r * a.ld, a.n);
        const RowStat st = row_stats<T, THREADS>(row, c2, sh);
        const float logsum = st.log_sum();
        if (threadIdx.x == 0) {
            if (a.norm) { a.norm[2 * r] = st.top(); a.norm[2 * r + 1] = logsum; }
            if (a.entropy) a.entropy[r] = st.entropy(logsum);
        }
        for (int j = threadIdx.x; j < a.ngiven; j += THREADS)
            a.logprobs[r * a.ngiven + j] = st.log_p(row.at(a.given[r * a.ngiven + j]), a.scale, logsum);
        if (a.k > 0) {
            if (threadIdx.x == 0) { buf.fill = 0; buf.bound = kNoKey; }
            __syncthreads();
            const bool some = logsum == logsum;
            for (int c = 0; some && c < row.nchunks; c += THREADS) offer_chunks<T, THREADS>(row, c, buf, a.k);
            const int found = some ? rank_best(buf, buf.fill, a.k) : 0;
            for (int j = threadIdx.x; j < a.k; j += THREADS) {
                const bool there = j < found;
                const float z = there ? order_value((uint32_t)(buf.key[j] >> 32)) : -INFINITY;
                a.top_ids[r * a.k + j] = there ? (int64_t)(uint32_t)~(uint32_t)buf.key[j] : -1;
                a.top_logprobs[r * a.k + j] = some ? st.log_p(z, a.scale, logsum) : NAN;
            }
            __syncthreads();
        }
    }
}

// ---- gradients:  g_i = p_i (A + B ln p_i) + sum of the list's c_j with id_j = i
template <typename T, int THREADS>
__device__ void row_gradient(const Row<T>& row, T* out, float m, float logsum, float scale, float A, float B, bool zero, int count,
                             ListShared& list)
{
    // scores of listed entries are read before anything is written: the gradient may take the place of the scores
    __syncthreads();
    for (int j = threadIdx.x; j < count; j += THREADS) list.z[j] = list.id[j] >= 0 ? row.at(list.id[j]) : -INFINITY;
    __syncthreads();
    // The exponential instruction gives 0 below 2^-126, but p times ln p and the coefficients may be above that: it is taken of x + 32
    // (p is 0 from 2^-158 on) and the product brought back.
    const float c2 = scale * kLog2e, l2 = logsum * kLog2e - 32.0f, b2 = B * kLn2, a2 = A - 32.0f * b2;
    auto grad = [&](float z) {
        const float x = (z - m) * c2 - l2;
        return __builtin_amdgcn_exp2f(x) * fmaf(b2, fmaxf(x, kLowest2), a2) * 0x1p-32f;
    };
    for (int c = threadIdx.x; c < row.nchunks; c += THREADS) {
        float v[Row<T>::E];
        const int first = row.load(c, v);
        for (int e = 0; e < Row<T>::E; ++e) v[e] = zero ? 0.0f : grad(v[e]);
        store_chunk<T>(out, row.n, first, v);
    }
    if (zero) return;
    __syncthreads();
    for (int j = threadIdx.x; j < count; j += THREADS) {
        const int id = list.id[j];
        if (id < 0) continue;
        float c = list.c[j];
        bool first = true;
        for (int i = 0; i < count; ++i)
            if (i != j && list.id[i] == id) { c += list.c[i]; first &= i > j; }
        if (first) out[id] = (T)(list.z[j] == -INFINITY ? 0.0f : grad(list.z[j]) + c);
    }
}

template <typename T, int THREADS>
__global__ __launch_bounds__(THREADS) void k_logprobs_backward(LogprobsBackwardArgs a)
{
    __shared__ RowShared<THREADS> sh;
    __shared__ ListShared list;
    for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const Row<T> row(a.logits, r * a.ld, a.n);
        __syncthreads();
        float sum = 0.0f;
        for (int j = threadIdx.x; j < a.ngiven; j += THREADS) {
            const int64_t id = a.given[r * a.ngiven + j];
            const bool there = row.at(id) != -INFINITY;
            const float g = there ? a.grad_logprobs[r * a.ngiven + j] : 0.0f;
            list.id[j] = there ? (int)id : -1;
            list.c[j] = g * a.scale;
            sum += g;
        }
        sum = group_sum<THREADS>(sum, sh);
        const float gh = a.grad_entropy ? a.grad_entropy[r] : 0.0f;
        const float A = -a.scale * (sum + (gh != 0.0f ? gh * a.entropy[r] : 0.0f));
        const float m = a.norm[2 * r];
        row_gradient<T, THREADS>(row, (T*)a.grad + r * a.ldg, m, a.norm[2 * r + 1], a.scale, A, -a.scale * gh, m == -INFINITY, a.ngiven, list);
    }
}

// ---- a teacher's list
// q of the entries that count into list.c (0 for the others), their ids into list.id (-1 for the others); returns the loss
template <typename T, int THREADS>
__device__ float teacher_list(const Row<T>& row, const int64_t* ids, const float* teacher, int k, float scale, const RowStat& st, float logsum,
                              ListShared& list, RowShared<THREADS>& sh, bool& some)
{
    __syncthreads();
    float top = -FLT_MAX;
    int n = 0;
    for (int j = threadIdx.x; j < k; j += THREADS) {
        const float z = row.at(ids[j]), t = teacher[j];
        const bool counts = z != -INFINITY && t != -INFINITY;
        list.id[j] = counts ? (int)ids[j] : -1;
        list.z[j] = z;
        if (counts) { top = fmaxf(top, t); n = 1; }
    }
    top = group_max<THREADS>(top, sh);
    some = __syncthreads_or(n);
    float sum = 0.0f;
    for (int j = threadIdx.x; j < k; j += THREADS) {
        const float e = list.id[j] >= 0 ? expf((teacher[j] - top) * scale) : 0.0f;
        list.c[j] = e;
        sum += e;
    }
    sum = group_sum<THREADS>(sum, sh);
    const float logq = logf(sum);
    float loss = 0.0f;
    for (int j = threadIdx.x; j < k; j += THREADS) {
        if (list.id[j] < 0) continue;
        const float q = list.c[j] / sum;
        list.c[j] = q;
        // q (ln q - ln p), the part of ln p that may not fit float32 multiplied by q first (a student's mask of the lowest value)
        if (q != 0.0f) loss += fmaf(q * scale, st.m - list.z[j], q * ((teacher[j] - top) * scale - logq + logsum));
    }
    return group_sum<THREADS>(loss, sh);
}

template <typename T, int THREADS, bool STEP>
__global__ __launch_bounds__(THREADS) void k_distill(DistillArgs a)
{
    __shared__ RowShared<THREADS> sh;
    __shared__ ListShared list;
    for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const Row<T> row(a.logits, r * a.ld, a.n);
        const RowStat st = row_stats<T, THREADS>(row, a.scale * kLog2e, sh);
        const float logsum = st.log_sum();
        bool some;
        const float loss = teacher_list<T, THREADS>(row, a.ids + r * a.k, a.teacher + r * a.k, a.k, a.scale, st, logsum, list, sh, some);
        if (threadIdx.x == 0) {
            a.loss[r] = loss;
            if (a.norm) { a.norm[2 * r] = st.top(); a.norm[2 * r + 1] = logsum; }
        }
        for (int j = threadIdx.x; a.q && j < a.k; j += THREADS) a.q[r * a.k + j] = list.c[j];
        if (STEP) {
            const float w = (a.weights ? a.weights[r] : 1.0f) * a.scale;
            for (int j = threadIdx.x; j < a.k; j += THREADS) list.c[j] *= -w;
            row_gradient<T, THREADS>(row, (T*)a.grad + r * a.ldg, st.top(), logsum, a.scale, w, 0.0f, !some || w == 0.0f, a.k, list);
        }
    }
}

template <typename T, int THREADS>
__global__ __launch_bounds__(THREADS) void k_distill_backward(DistillArgs a)
{
    __shared__ ListShared list;
    for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const Row<T> row(a.logits, r * a.ld, a.n);
        const float w = (a.weights ? a.weights[r] : 1.0f) * a.scale;
        __syncthreads();
        int some = 0;
        for (int j = threadIdx.x; j < a.k; j += THREADS) {
            const float q = a.q[r * a.k + j];
            const int64_t id = a.ids[r * a.k + j];
            const bool counts = q != 0.0f && id >= 0 && id < a.n;
            list.id[j] = counts ? (int)id : -1;
            list.c[j] = -w * q;
            some |= counts;
        }
        some = __syncthreads_or(some);
        row_gradient<T, THREADS>(row, (T*)a.grad + r * a.ldg, a.norm[2 * r], a.norm[2 * r + 1], a.scale, w, 0.0f, !some || w == 0.0f, a.k, list);
    }
}

// ---- launches
constexpr int kRowThreads = 256;
static unsigned row_grid(int64_t rows) { return (unsigned)(rows < (1 << 20) ? rows : 1 << 20); }      // (a launch may not have 2^32 threads)

#define HR_ROWS_LAUNCH(kernel, dtype, ...)                                                                                        \
    switch (dtype) {                                                                                                              \
    case HR_F32: hipLaunchKernelGGL((kernel<float, kRowThreads __VA_ARGS__>), dim3(row_grid(a.rows)), dim3(kRowThreads), 0, s, a); break;   \
    case HR_F16: hipLaunchKernelGGL((kernel<_Float16, kRowThreads __VA_ARGS__>), dim3(row_grid(a.rows)), dim3(kRowThreads), 0, s, a); break; \
    default: hipLaunchKernelGGL((kernel<__bf16, kRowThreads __VA_ARGS__>), dim3(row_grid(a.rows)), dim3(kRowThreads), 0, s, a); break;      \
    }                                                                                                                             \
    return hipGetLastError()

static hipError_t launch_logprobs(int dtype, const LogprobsArgs& a, hipStream_t s) { HR_ROWS_LAUNCH(k_logprobs, dtype); }
static hipError_t launch_logprobs_backward(int dtype, const LogprobsBackwardArgs& a, hipStream_t s) { HR_ROWS_LAUNCH(k_logprobs_backward, dtype); }
static hipError_t launch_distill(int dtype, const DistillArgs& a, hipStream_t s) { HR_ROWS_LAUNCH(k_distill, dtype, , false); }
static hipError_t launch_distill_step(int dtype, const DistillArgs& a, hipStream_t s) { HR_ROWS_LAUNCH(k_distill, dtype, , true); }
static hipError_t launch_distill_backward(int dtype, const DistillArgs& a, hipStream_t s) { HR_ROWS_LAUNCH(k_distill_backward, dtype); }

}  // namespace hr

// ---- C entry points
using namespace hr;

static int check_rows(const void* logits, int64_t ld, int32_t dtype, int64_t rows, int64_t n, float scale)
{
    if (dtype != HR_F32 && dtype != HR_F16 && dtype != HR_BF16) return fail(HR_ERR_ARG, "unknown dtype %d", dtype);
    if (rows < 0 || rows > (1 << 24)) return fail(HR_ERR_ARG, "rows=%lld out of range", (long long)rows);
    if (n < 1 || n > HR_ROW_MAX) return fail(HR_ERR_ARG, "n=%lld must be in 1..%d", (long long)n, HR_ROW_MAX);
    if (ld < n || ld > (1LL << 40)) return fail(HR_ERR_ARG, "ld=%lld: rows of %lld scores overlap or are too far apart", (long long)ld, (long long)n);
    if (!(scale > 0.0f) || scale > FLT_MAX) return fail(HR_ERR_ARG, "scale=%g must be positive and finite", (double)scale);
    if (rows > 0 && !logits) return fail(HR_ERR_ARG, "logits is null");
    if ((uintptr_t)logits % element_bytes(dtype)) return fail(HR_ERR_ARG, "logits is not aligned to its elements");
    return HR_OK;
}

static int check_gradient(const void* logits, int64_t ld, int32_t dtype, int64_t n, const void* grad, int64_t ldg)
{
    if (!grad) return fail(HR_ERR_ARG, "grad_logits is null");
    if (ldg < n || ldg > (1LL << 40)) return fail(HR_ERR_ARG, "ldg=%lld: rows of %lld scores overlap or are too far apart", (long long)ldg, (long long)n);
    if ((uintptr_t)grad % element_bytes(dtype)) return fail(HR_ERR_ARG, "grad_logits is not aligned to its elements");
    if (grad == logits && ldg != ld) return fail(HR_ERR_ARG, "grad_logits is logits, but ldg=%lld is not ld=%lld", (long long)ldg, (long long)ld);
    return HR_OK;
}

extern "C" {

size_t hr_logprobs_workspace_bytes(int64_t rows, int64_t n, int32_t k)
{
    if (rows < 0 || rows > (1 << 24) || n < 1 || n > HR_ROW_MAX || k < 0 || k > HR_K_MAX) {
        fail(HR_ERR_ARG, "rows=%lld, n=%lld or k=%d out of range", (long long)rows, (long long)n, k);
        return 0;
    }
    return HR_WORKSPACE_ALIGN;
}

int hr_logprobs(const void* logits, int64_t ld, int32_t dtype, int64_t rows, int64_t n, float scale, const int64_t* given,
                int32_t ngiven, int32_t k, float* out_logprobs, float* out_entropy, float* out_norm, int64_t* out_top_ids,
                float* out_top_logprobs, void* workspace, size_t workspace_bytes, void* stream)
{
    if (int rc = check_rows(logits, ld, dtype, rows, n, scale)) return rc;
    if (ngiven < 0 || ngiven > HR_LIST_MAX) return fail(HR_ERR_ARG, "ngiven=%d must be in 0..%d", ngiven, HR_LIST_MAX);
    if (k < 0 || k > HR_K_MAX) return fail(HR_ERR_ARG, "k=%d must be in 0..%d", k, HR_K_MAX);
    if (rows == 0) return HR_OK;
    if (ngiven > 0 && (!given || !out_logprobs)) return fail(HR_ERR_ARG, "given / out_logprobs is null");
    if (k > 0 && (!out_top_ids || !out_top_logprobs)) return fail(HR_ERR_ARG, "out_top_ids / out_top_logprobs is null");
    if (int rc = check_workspace(workspace, workspace_bytes, hr_logprobs_workspace_bytes(rows, n, k))) return rc;
    LogprobsArgs a{logits, ld, rows, (int)n, scale, given, ngiven, k, out_logprobs, out_entropy, out_norm, out_top_ids, out_top_logprobs};
    HR_HIP(launch_logprobs(dtype, a, (hipStream_t)stream));
    return HR_OK;
}

int hr_logprobs_backward(const void* logits, int64_t ld, int32_t dtype, int64_t rows, int64_t n, float scale, const int64_t* given,
                         int32_t ngiven, const float* entropy, const float* norm, const float* grad_logprobs,
                         const float* grad_entropy, void* grad_logits, int64_t ldg, void* stream)
{
    if (int rc = check_rows(logits, ld, dtype, rows, n, scale)) return rc;
    if (ngiven < 0 || ngiven > HR_LIST_MAX) return fail(HR_ERR_ARG, "ngiven=%d must be in 0..%d", ngiven, HR_LIST_MAX);
    if (rows == 0) return HR_OK;
    if (int rc = check_gradient(logits, ld, dtype, n, grad_logits, ldg)) return rc;
    if (!norm) return fail(HR_ERR_ARG, "norm is null");
    if (grad_logprobs && ngiven > 0 && !given) return fail(HR_ERR_ARG, "given is null");
    if (grad_entropy && !entropy) return fail(HR_ERR_ARG, "entropy is null");
    LogprobsBackwardArgs a{logits, ld, rows, (int)n, scale, given, grad_logprobs ? ngiven : 0, entropy, norm, grad_logprobs, grad_entropy, grad_logits, ldg};
    HR_HIP(launch_logprobs_backward(dtype, a, (hipStream_t)stream));
    return HR_OK;
}

size_t hr_distill_workspace_bytes(int64_t rows, int64_t n, int32_t k)
{
    if (rows < 0 || rows > (1 << 24) || n < 1 || n > HR_ROW_MAX || k < 1 || k > HR_LIST_MAX) {
        fail(HR_ERR_ARG, "rows=%lld, n=%lld or k=%d out of range", (long long)rows, (long long)n, k);
        return 0;
    }
    return HR_WORKSPACE_ALIGN;
}

int hr_distill_forward(const void* logits, int64_t ld, int32_t dtype, int64_t rows, int64_t n, float scale, const int64_t* ids,
                       const float* teacher, int32_t k, float* out_loss, float* out_norm, float* out_q, void* workspace,
                       size_t workspace_bytes, void* stream)
{
    if (int rc = check_rows(logits, ld, dtype, rows, n, scale)) return rc;
    if (k < 1 || k > HR_LIST_MAX) return fail(HR_ERR_ARG, "k=%d must be in 1..%d", k, HR_LIST_MAX);
    if (rows == 0) return HR_OK;
    if (!ids || !teacher || !out_loss) return fail(HR_ERR_ARG, "ids / teacher / out_loss is null");
    if (int rc = check_workspace(workspace, workspace_bytes, hr_distill_workspace_bytes(rows, n, k))) return rc;
    DistillArgs a{logits, ld, rows, (int)n, scale, ids, teacher, k, nullptr, out_loss, out_norm, out_q, nullptr, 0};
    HR_HIP(launch_distill(dtype, a, (hipStream_t)stream));
    return HR_OK;
}

int hr_distill_backward(const void* logits, int64_t ld, int32_t dtype, int64_t rows, int64_t n, float scale, const int64_t* ids,
                        const float* q, int32_t k, const float* norm, const float* weights, void* grad_logits, int64_t ldg, void* stream)
{
    if (int rc = check_rows(logits, ld, dtype, rows, n, scale)) return rc;
    if (k < 1 || k > HR_LIST_MAX) return fail(HR_ERR_ARG, "k=%d must be in 1..%d", k, HR_LIST_MAX);
    if (rows == 0) return HR_OK;
    if (!ids || !q || !norm) return fail(HR_ERR_ARG, "ids / q / norm is null");
    if (int rc = check_gradient(logits, ld, dtype, n, grad_logits, ldg)) return rc;
    DistillArgs a{logits, ld, rows, (int)n, scale, ids, nullptr, k, weights, nullptr, (float*)norm, (float*)q, grad_logits, ldg};
    HR_HIP(launch_distill_backward(dtype, a, (hipStream_t)stream));
    return HR_OK;
}

int hr_distill_step(const void* logits, int64_t ld, int32_t dtype, int64_t rows, int64_t n, float scale, const int64_t* ids,
                    const float* teacher, int32_t k, const float* weights, float* out_loss, float* out_norm, float* out_q,
                    void* grad_logits, int64_t ldg, void* workspace, size_t workspace_bytes, void* stream)
{
    if (int rc = check_rows(logits, ld, dtype, rows, n, scale)) return rc;
    if (k < 1 || k > HR_LIST_MAX) return fail(HR_ERR_ARG, "k=%d must be in 1..%d", k, HR_LIST_MAX);
    if (rows == 0) return HR_OK;
    if (!ids || !teacher || !out_loss) return fail(HR_ERR_ARG, "ids / teacher / out_loss is null");
    if (int rc = check_gradient(logits, ld, dtype, n, grad_logits, ldg)) return rc;
    if (int rc = check_workspace(workspace, workspace_bytes, hr_distill_workspace_bytes(rows, n, k))) return rc;
    DistillArgs a{logits, ld, rows, (int)n, scale, ids, teacher, k, weights, out_loss, out_norm, out_q, grad_logits, ldg};
    HR_HIP(launch_distill_step(dtype, a, (hipStream_t)stream));
    return HR_OK;
}

}  // extern "C"
