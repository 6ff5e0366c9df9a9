// Rows of scores as distributions (hr_scores.h): log probabilities of given entries, entropy, best alternatives, a teacher's
// list, and the gradients of all of them.  A workgroup takes a row.
//
// Mathematics.  With s the scale, m the largest score of a row and t_i = exp(s (z_i - m)):  S0 = sum t_i >= 1,  S1 = sum s (z_i - m) t_i <= 0,
//   ln p_i = s (z_i - m) - ln S0,      entropy = ln S0 - S1 / S0  (two terms that are not negative: nothing cancels).
// Every thread keeps such sums of the chunks it has seen (float32) and the threads' are brought to the largest maximum and added
// in a fixed order at the end.  Exponents are counted in base 2: one multiplication by s / ln 2 serves scale and base.
#include <algorithm>
#include <type_traits>

#include "entry.h"
#include "row_math.h"

namespace hr {

// entries of a row's list that a thread looks after
template <int THREADS> constexpr int kListPer = (HR_LIST_MAX + THREADS - 1) / THREADS;

// ---- best k of a row
// The pass over the row keeps the largest score of every slot.  A few slots of a thread (or of two neighbours) make a group, and the
// k-th largest of 512 groups' maxima is a bound that k entries reach: only slots that reach it are read again (about k of
// them), their entries that reach it are collected and ranked.  Keys of (score, entry) are 64-bit numbers, larger is better, no two
// alike: equal scores go by entry.  Where a score at the bound is that of very many entries (masks of the lowest value, rows all
// alike) the better ones are collected first, then the first of the equal ones in the order of the row.
__device__ __forceinline__ uint64_t entry_key(float z, int i) { return (uint64_t)order_key(z) << 32 | (uint32_t)~i; }

template <int THREADS>
struct TopShared {
    // (one wave has 7 KB, 22 of them share a compute unit; a chunk has to fit in beside kMost kept entries)
    static constexpr int kMost = HR_K_MAX, kCap = THREADS >= 256 ? 1024 : 384;
    static constexpr int kAll = kCap + 1, kGroups = 512;
    Slots<THREADS> slots;
    uint16_t picked[Slots<THREADS>::kPer * THREADS];
    uint64_t key[kCap];
    uint64_t best[kMost];
    uint64_t bound;                     // entries at or below it are not among the best
    uint32_t group[THREADS == 64 ? 1 : kGroups];         // (with 64 threads every slot is a group)
    int wave[THREADS / 64];
    int npicked, fill, ties;
    int valid[2];                       // by turns: keys that there was room for, or kAll where that was all of a round's
};

// A lower bound, as an order_key, of the k-th largest of 64 N keys, N of which every lane of a wave holds, such that few more
// than k reach it where they differ (the range between the smallest and the largest is cut until k .. 1.5 k + 8 are left;
// ties: more than that reach it).  Keys at or below kNoCandidate are none; with fewer than k others all of those reach the bound.
template <int N>
__device__ __forceinline__ uint32_t bound_of(const uint32_t* mine, int k, bool& ties)
{
    uint32_t least = 0xffffffffu, largest = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        if (mine[i] > kNoCandidate) least = min(least, mine[i]);
        largest = max(largest, mine[i]);
    }
    least = wave_min(least);
    largest = wave_fold(largest, [](uint32_t x, uint32_t y) { return x > y ? x : y; });
    ties = false;
    // lo is reached by k or more, hi + 1 by fewer
    uint32_t lo = kNoCandidate + 1, hi = largest;
    if (least > largest) return lo;
    const int enough = k + k / 2 + 8;
    int reached = 0;
    for (bool once = true; lo < hi || once; once = false) {
        // three bounds at once split what is left in four; the first time the smallest key is the lowest of them
        const uint32_t from = once ? least : lo + 1, part = (hi - from) / (once ? 3 : 4) + 1;
        const uint32_t b1 = once ? from : min(lo + part, hi), b2 = min(b1 + part, hi), b3 = min(b2 + part, hi);
        int n1 = 0, n2 = 0, n3 = 0;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            n1 += __popcll(__ballot(mine[i] >= b1));
            n2 += __popcll(__ballot(mine[i] >= b2));
            n3 += __popcll(__ballot(mine[i] >= b3));
        }
        if (n3 >= k) { lo = b3; reached = n3; }
        else if (n2 >= k) { lo = b2; hi = b3 - 1; reached = n2; }
        else if (n1 >= k) { lo = b1; hi = b2 - 1; reached = n1; }
        else if (once) return lo;
        else { hi = b1 - 1; continue; }
        if (reached <= enough) return lo;
    }
    ties = true;
    return lo;
}

// The best k of the first `fill` keys, best first, in t.best; returns how many there are.
template <int THREADS>
__device__ int rank_best(TopShared<THREADS>& t, int fill, int k)
{
    if (fill > k + k / 2 + 64) {
        // Most of them need not be ranked: a bound among their scores, or among the entries of equal scores, and those that
        // reach it go to the front.
        constexpr int N = TopShared<THREADS>::kCap / 64, PER = TopShared<THREADS>::kCap / THREADS;
        uint32_t part[N];
#pragma unroll
        for (int i = 0; i < N; ++i) part[i] = i * 64 + lane_id() < fill ? (uint32_t)(t.key[i * 64 + lane_id()] >> 32) : 0;
        bool ties;
        const uint32_t score = bound_of<N>(part, k, ties);
        uint64_t least = (uint64_t)score << 32;
        if (ties) {
            int better = 0;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                better += __popcll(__ballot(part[i] > score));
                part[i] = part[i] == score ? (uint32_t)t.key[i * 64 + lane_id()] : 0;      // (~entry, above kNoCandidate: entries are below 2^30)
            }
            bool none;
            least |= bound_of<N>(part, k - better, none);
        }
        uint64_t mine[PER];
#pragma unroll
        for (int i = 0; i < PER; ++i) mine[i] = i * THREADS + (int)threadIdx.x < fill ? t.key[i * THREADS + threadIdx.x] : 0;
        __syncthreads();
        if (threadIdx.x == 0) t.fill = 0;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < PER; ++i)
            if (mine[i] >= least) t.key[atomicAdd(&t.fill, 1)] = mine[i];
        __syncthreads();
        fill = t.fill;
    }
    // Up to 256 threads: each has a key (one wave's up to four) and counts how many beat it, all lanes reading the same four of them at a
    // time.  With 1024 sixteen lanes count for a key, one round for 64 of them.  (That way with fewer threads 16 times as much LDS is read
    // for a key: 4096 rows of 4096 float32 k 32 28.8 us, 24.7 now, k 64 44.8 and 32.8; 2048 of 32000 bfloat16 k 128 70 and 56; one row of 32003
    // with 1024 threads k 32 11.0, and 11.7 this way.)
    if constexpr (THREADS <= 256) {
        constexpr int kWays = THREADS == 64 ? 4 : 1;
        static_assert(HR_K_MAX + HR_K_MAX / 2 + 64 <= kWays * THREADS && HR_K_MAX + HR_K_MAX / 2 + 68 <= TopShared<THREADS>::kCap);
        if (threadIdx.x < 4) t.key[fill + threadIdx.x] = 0;
        __syncthreads();
        auto rank = [&](auto ways) __attribute__((always_inline)) {
            constexpr int N = decltype(ways)::value;
            uint64_t mine[N];
            int beaten[N] = {};
#pragma unroll
            for (int i = 0; i < N; ++i) mine[i] = i * THREADS + (int)threadIdx.x < fill ? t.key[i * THREADS + threadIdx.x] : 0;
            for (int j = 0; j < fill; j += 4) {
                uint64_t other[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) other[e] = t.key[j + e];
#pragma unroll
                for (int e = 0; e < 4; ++e)
#pragma unroll
                    for (int i = 0; i < N; ++i) beaten[i] += other[e] > mine[i];
            }
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (i * THREADS + (int)threadIdx.x < fill && beaten[i] < k) t.best[beaten[i]] = mine[i];
        };
        using std::integral_constant;
        if (THREADS > 64 || fill <= 64) {
            if ((int)threadIdx.x / 64 * 64 < fill) rank(integral_constant<int, 1>{});
        } else if (fill <= 128) {
            rank(integral_constant<int, 2>{});
        } else {
            rank(integral_constant<int, kWays>{});
        }
    } else {
        const int sub = threadIdx.x & 15;
        for (int i = threadIdx.x / 16; i < fill; i += THREADS / 16) {
            const uint64_t mine = t.key[i];
            int n = 0;
            for (int j = sub; j < fill; j += 16) n += t.key[j] > mine;
            n += __builtin_amdgcn_update_dpp(0, n, 0xb1, 0xf, 0xf, false);      // lanes ^ 1, ^ 2, the other four, the other eight
            n += __builtin_amdgcn_update_dpp(0, n, 0x4e, 0xf, 0xf, false);
            n += __builtin_amdgcn_update_dpp(0, n, 0x141, 0xf, 0xf, false);
            n += __builtin_amdgcn_update_dpp(0, n, 0x140, 0xf, 0xf, false);
            if (sub == 0 && n < k) t.best[n] = mine;
        }
    }
    __syncthreads();
    return fill < k ? fill : k;
}

// Offers chunk c of the row (-1: none), one of every thread, to the buffer: entries above t.bound are appended.  Where there is
// no room for a chunk's, the best k of what the buffer holds are kept, the k-th is the new bound, and the chunk is offered again:
// there is room for one at least.  turn: a number that changes from call to call: what a round leaves in t.valid is read behind its
// barrier, when the next round may already write the other one.
template <typename T, int THREADS>
__device__ __forceinline__ void offer(const Row<T>& row, int c, TopShared<THREADS>& t, int k, int turn)
{
    constexpr int E = Row<T>::E;
    float v[E];
    bool pending = c >= 0;
    const int first = pending ? row.load(c, v) : 0;
    for (;;) {
        int cnt = 0;
        const uint64_t above = t.bound;
        if (pending) {
#pragma unroll
            for (int e = 0; e < E; ++e) cnt += entry_key(v[e], first + e) > above;
        }
        pending = pending && cnt > 0;
        if (pending) {
            int pos = atomicAdd(&t.fill, cnt);
            if (pos + cnt <= TopShared<THREADS>::kCap) {
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const uint64_t key = entry_key(v[e], first + e);
                    if (key > above) t.key[pos++] = key;
                }
                pending = false;
            } else {
                atomicMin(&t.valid[turn & 1], pos);
            }
        }
        __syncthreads();
        const int valid = t.valid[turn & 1];
        if (valid == TopShared<THREADS>::kAll) return;
        const int kept = rank_best(t, valid, k);
        for (int j = threadIdx.x; j < kept; j += THREADS) t.key[j] = t.best[j];
        __syncthreads();
        if (threadIdx.x == 0) {
            t.fill = kept;
            t.valid[turn & 1] = TopShared<THREADS>::kAll;
            if (kept == k) t.bound = t.best[k - 1];
        }
        __syncthreads();
    }
}

// Appends the first of the entries with this score, in the order of the row, until the buffer holds k.
template <typename T, int THREADS>
__device__ void append_equal(const Row<T>& row, uint32_t score, TopShared<THREADS>& t, int k)
{
    constexpr int E = Row<T>::E;
    int have = t.fill;
    for (int c0 = 0; c0 < row.nchunks && have < k; c0 += THREADS) {
        const int c = c0 + threadIdx.x;
        float v[E];
        int first = 0, cnt = 0;
        if (c < row.nchunks) {
            first = row.load(c, v);
#pragma unroll
            for (int e = 0; e < E; ++e) cnt += order_key(v[e]) == score;
        }
        // places of a thread's behind those of the threads before it
        int pos = wave_prefix_sum(cnt);
        __syncthreads();
        if (lane_id() == 63) t.wave[threadIdx.x / 64] = pos;
        __syncthreads();
        pos += have - cnt;
        for (int w = 0; w < THREADS / 64; ++w) {
            if (w < (int)threadIdx.x / 64) pos += t.wave[w];
            have += t.wave[w];
        }
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (c < row.nchunks && order_key(v[e]) == score && pos < k) t.key[pos++] = entry_key(v[e], first + e);
    }
    __syncthreads();
    if (threadIdx.x == 0) t.fill = min(have, k);
    __syncthreads();
}

// The best k of a row whose slots are filled, best first, in t.best; returns how many there are.  Slot s: the chunks that thread
// s % WIDTH of WIDTH threads has read in its steps from s / WIDTH * span on.
template <typename T, int THREADS, int WIDTH>
__device__ int best_entries(const Row<T>& row, int span, int k, TopShared<THREADS>& t)
{
    constexpr int PER = Slots<THREADS>::kPer;
    static_assert(THREADS == 64 || THREADS == 256 || THREADS == 1024);
    uint32_t mine[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) mine[i] = t.slots.key[i][threadIdx.x];          // slot i THREADS + this thread
    // the groups' maxima: a thread's slots one by one, four of them, or all of two neighbours
    if (THREADS > 64) {
        uint32_t a = max(max(mine[0], mine[1]), max(mine[2], mine[3]));
        if (THREADS == 1024) {
            a = max(a, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)a, 0xb1, 0xf, 0xf, false));      // lane ^ 1
            t.group[threadIdx.x / 2] = a;
        } else {
            t.group[threadIdx.x] = a;
            t.group[(256 + threadIdx.x) % TopShared<THREADS>::kGroups] = max(max(mine[PER - 4], mine[PER - 3]), max(mine[PER - 2], mine[PER - 1]));
        }
    }
    __syncthreads();
    if (threadIdx.x < 64) {
        constexpr int N = TopShared<THREADS>::kGroups / 64;
        uint32_t g[N];
#pragma unroll
        for (int i = 0; i < N; ++i) g[i] = THREADS == 64 ? mine[i % PER] : t.group[i * 64 + lane_id()];
        bool ties;
        // (256 groups are enough for few)
        uint32_t bound;
        if (k <= 32) {
            uint32_t h[N / 2];
#pragma unroll
            for (int i = 0; i < N / 2; ++i) h[i] = max(g[2 * i], g[2 * i + 1]);
            bound = bound_of<N / 2>(h, k, ties);
        } else {
            bound = bound_of<N>(g, k, ties);
        }
        if (threadIdx.x == 0) {
            t.bound = ((uint64_t)(bound + ties) << 32) - 1;
            t.ties = ties;
            t.fill = t.npicked = 0;
            t.valid[0] = t.valid[1] = TopShared<THREADS>::kAll;
        }
    }
    __syncthreads();
    const uint32_t bound = (uint32_t)(t.bound >> 32) + 1;
#pragma unroll
    for (int i = 0; i < PER; ++i)
        if (mine[i] >= bound) t.picked[atomicAdd(&t.npicked, 1)] = (uint16_t)(i * THREADS + threadIdx.x);
    __syncthreads();
    // chunks of the picked slots, then the edges
    // (numbers of chunks, also of those that slots have behind the row's end, are below 2^30)
    const uint32_t chunks = (uint32_t)t.npicked * span, all = chunks + (row.edges() ? 2 : 0);
    int turn = 0;
    for (uint32_t c0 = 0; c0 < all; c0 += THREADS) {
        const uint32_t i = c0 + threadIdx.x;
        int c = -1;
        if (i < chunks) {
            const uint32_t j = span == 1 ? i : i / (uint32_t)span, p = t.picked[j];
            const uint32_t at = ((p / WIDTH) * span + (i - j * span)) * WIDTH + p % WIDTH;
            if ((int)at >= row.lo && (int)at < row.hi) c = (int)at;
        } else if (i < all) {
            c = i == chunks ? (row.lo > 0 ? 0 : -1) : (row.hi < row.nchunks && row.hi >= row.lo ? row.hi : -1);
        }
        offer<T, THREADS>(row, c, t, k, turn++);
    }
    if (t.ties && t.fill < k) append_equal<T, THREADS>(row, bound - 1, t, k);
    return rank_best(t, t.fill, k);
}

// Sums (and with SLOTS the largest score that each thread has seen) of part blockIdx.x of row blockIdx.y.
template <typename T, bool ENTROPY, bool SLOTS>
__global__ __launch_bounds__(kPartThreads) void k_row_parts(const void* logits, int64_t ld, int n, float scale, Parts parts)
{
    constexpr int THREADS = kPartThreads;
    __shared__ RowShared<THREADS> sh;
    __shared__ std::conditional_t<SLOTS, Slots<THREADS>, char> slots;
    const int64_t r = blockIdx.y, part = r * parts.n + blockIdx.x;
    const Row<T> row(logits, r * ld, n);
    const int begin = (int)blockIdx.x * parts.len, end = blockIdx.x + 1 == gridDim.x ? row.nchunks : begin + parts.len;
    Held<4, T> held;
    Slots<THREADS>* mine = nullptr;
    if constexpr (SLOTS) mine = &slots;
    const RowStat st = row_stats<T, THREADS, ENTROPY, SLOTS>(row, begin, end, scale * kLog2e, sh, mine, 1 << 30, held, [] {});
    if (threadIdx.x == 0) *(floatx4*)(parts.stats + part * 4) = floatx4{st.m, st.s0, st.s1, 0.0f};
    if constexpr (SLOTS) parts.slots[part * THREADS + threadIdx.x] = slots.key[0][threadIdx.x];
}

// PARTS: the sums and slots come from k_row_parts
template <typename T, int THREADS, bool TOP, bool PARTS>
__global__ __launch_bounds__(THREADS) void k_logprobs(LogprobsArgs a)
{
    __shared__ RowShared<THREADS> sh;
    __shared__ std::conditional_t<TOP, TopShared<THREADS>, char> top_;
    const float c2 = a.scale * kLog2e;
    for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const Row<T> row(a.logits, r * a.ld, a.n);
        Slots<THREADS>* slots = nullptr;
        int span = 0;
        if constexpr (TOP) {
            slots = &top_.slots;
            span = Slots<THREADS>::span_for(row.nchunks);
        }
        float z[kListPer<THREADS>];
        auto read_given = [&] {
#pragma unroll
            for (int i = 0; i < kListPer<THREADS>; ++i) {
                const int j = i * THREADS + threadIdx.x;
                if (i * THREADS < a.ngiven) z[i] = j < a.ngiven ? row.at(a.given[r * a.ngiven + j]) : 0.0f;
            }
        };
        RowStat st;
        if constexpr (PARTS) {
            read_given();
            if constexpr (TOP) {
                span = a.parts.len / kPartThreads;
#pragma unroll
                for (int i = 0; i < Slots<THREADS>::kPer; ++i) {
                    const int s = i * THREADS + threadIdx.x;
                    slots->key[i][threadIdx.x] = s < a.parts.n * kPartThreads ? a.parts.slots[r * a.parts.n * kPartThreads + s] : 0;
                }
            }
            st = joined_stats(a.parts, r, c2);
        } else {
            Held<4, T> held;
            st = row_stats<T, THREADS, true, TOP>(row, 0, row.nchunks, c2, sh, slots, span, held, read_given);
        }
        const float logsum = st.log_sum();
        if (threadIdx.x == 0) {
            if (a.norm) { a.norm[2 * r] = st.top(); a.norm[2 * r + 1] = logsum; }
            if (a.entropy) a.entropy[r] = st.entropy(logsum);
        }
#pragma unroll
        for (int i = 0; i < kListPer<THREADS>; ++i) {
            const int j = i * THREADS + threadIdx.x;
            if (j < a.ngiven) a.logprobs[r * a.ngiven + j] = st.log_p(z[i], a.scale, logsum);
        }
        if constexpr (TOP) {
            const bool some = logsum == logsum;
            const int found = some ? best_entries<T, THREADS, PARTS ? kPartThreads : THREADS>(row, span, a.k, top_) : 0;
            for (int j = threadIdx.x; j < a.k; j += THREADS) {
                const bool there = j < found;
                const float z = there ? order_value((uint32_t)(top_.best[j] >> 32)) : -INFINITY;
                a.top_ids[r * a.k + j] = there ? (int64_t)(uint32_t)~(uint32_t)top_.best[j] : -1;
                a.top_logprobs[r * a.k + j] = some ? st.log_p(z, a.scale, logsum) : NAN;
            }
            __syncthreads();
        }
    }
}

// ---- gradients:  g_i = p_i (A + B ln p_i) + sum of the list's c_j with id_j = i
// With x = log2 p_i = (z_i - m) s / ln 2 - log2 S0 rounded as it is: a likely entry's is near 0, and A + B ln p_i, which cancels for a row that is sure of
// an entry, keeps all of its bits.  The exponential instruction gives 0 below 2^-126, where p times a large coefficient, or p in float32
// itself, is not 0 yet: an entry with x < -126 takes the square of 2^(x / 2), of which only one factor meets the coefficient before the other (products
// with p down to 2^-252; what is lost beyond is below 2^-124 whatever the coefficient).
struct Coefficients {
    float m, l2, c2, a, b2;
    bool zero;                          // the row takes no part
    static constexpr float kNormal = -126.0f;

    __device__ __forceinline__ void set(float m_, float logsum, float scale, float A, float B, bool zero_)
    {
        m = m_;
        c2 = scale * kLog2e;
        l2 = logsum * kLog2e;
        a = A;
        b2 = B * kLn2;
        zero = zero_;
    }
    __device__ __forceinline__ float exponent(float z) const { return fmaf(z - m, c2, -l2); }
    // of an exponent that is not below kNormal
    template <bool ENTROPY>
    __device__ __forceinline__ float near(float x) const
    {
        const float p = __builtin_amdgcn_exp2f(x);
        return ENTROPY ? p * fmaf(b2, x, a) : p * a;
    }
    // of any: where it is not, the same bits
    template <bool ENTROPY>
    __device__ __forceinline__ float any(float x) const
    {
        const bool low = x < kNormal;
        const float e = __builtin_amdgcn_exp2f(low ? 0.5f * x : x), g = ENTROPY ? e * fmaf(b2, fmaxf(x, kLowest2), a) : e * a;
        return low ? (e == 0.0f ? 0.0f : e * g) : g;
    }
    template <bool ENTROPY>
    __device__ __forceinline__ float grad(float z) const { return any<ENTROPY>(exponent(z)); }
    // of a chunk: few have entries that low
    template <bool ENTROPY, int E, typename V>
    __device__ __forceinline__ void grads(const V& z, float* v) const
    {
        float least = 0.0f;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            v[e] = exponent((float)z[e]);
            least = fminf(least, v[e]);
        }
        if (least >= kNormal) {
#pragma unroll
            for (int e = 0; e < E; ++e) v[e] = near<ENTROPY>(v[e]);
        } else {
#pragma unroll
            for (int e = 0; e < E; ++e) v[e] = any<ENTROPY>(v[e]);
        }
    }
};

// held: chunks of the row that the thread has already, from held->at on (null: none).  first() is called once while the first
// chunks are on their way: it fills k (Coefficients) and the list: entries (-1: none), coefficients, scores, which have to be read before anything is
// written (the gradient may take the place of the scores), with a barrier at its end.
template <typename T, int THREADS, bool ENTROPY, typename G>
__device__ __forceinline__ void row_gradient(const Row<T>& row, int begin, int end, T* out, const Coefficients& k, int count, ListShared& list, const Held<4, T>* held, G&& first)
{
    constexpr int E = Row<T>::E;
    auto chunk = [&](const typename Row<T>::V& raw, int c, bool in) __attribute__((always_inline)) {
        float v[E];
        if (k.zero) {
#pragma unroll
            for (int e = 0; e < E; ++e) v[e] = 0.0f;
        } else {
            k.template grads<ENTROPY, E>(raw, v);
        }
        if (in) store_chunk<T>(out + row.first(c), v);
    };
    Held<4, T> rest;
    if (held) {
        first();
        for_held<THREADS>(row, begin, end, *held, chunk);
        const int left = min(held->at, end);
        if (left > begin) for_chunks<THREADS>(row, begin, left, rest, chunk, [] {});
    } else {
        for_chunks<THREADS>(row, begin, end, rest, chunk, first);
    }
    if (begin == 0 && row.edges()) {
        const int i = row.edge(threadIdx.x);
        if (i >= 0) out[i] = (T)(k.zero ? 0.0f : k.template grad<ENTROPY>((float)row.z[i]));
    }
    if (k.zero) return;
    __syncthreads();
    for (int j = threadIdx.x; j < count; j += THREADS) {
        const int id = list.id[j];
        if (id < 0) continue;
        // (an entry may be listed more than once: the first of them writes the sum)
        float c = list.c[j];
        bool leads = true;
        for (int i = 0; i < count; i += 4) {
            const intx4 other = *(const intx4*)(list.id + i);         // (behind the last one: -1)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (other[e] == id && i + e != j) {
                    c += list.c[i + e];
                    leads &= i + e > j;
                }
        }
        if (leads) out[id] = (T)(list.z[j] == -INFINITY ? 0.0f : k.template grad<ENTROPY>(list.z[j]) + c);
    }
}

// Chunks that workgroup blockIdx.y of a row takes: the first has the edges too, wherever they are.
template <typename T>
struct Slice {
    int begin, end;
    __device__ __forceinline__ Slice(const Row<T>& row, int len)
    {
        begin = (int)blockIdx.y * len;
        end = min(begin + len, row.nchunks);
    }
    __device__ __forceinline__ bool has(const Row<T>& row, int64_t id) const
    {
        if (id < 0 || id >= row.n) return false;
        const int c = (int)((id + row.before) / Row<T>::E);
        return c < row.lo || c >= row.hi ? begin == 0 : c >= begin && c < end;
    }
};

template <typename T, int THREADS>
__global__ __launch_bounds__(THREADS) void k_logprobs_backward(LogprobsBackwardArgs a)
{
    __shared__ RowShared<THREADS> sh;
    __shared__ ListShared list;
    for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const Row<T> row(a.logits, r * a.ld, a.n);
        const Slice<T> slice(row, a.slice);
        const float m = a.norm[2 * r], logsum = a.norm[2 * r + 1], gh = a.grad_entropy ? a.grad_entropy[r] : 0.0f;
        const float entropy = gh != 0.0f ? a.entropy[r] : 0.0f;
        Coefficients k;
        row_gradient<T, THREADS, true>(row, slice.begin, slice.end, (T*)a.grad + r * a.ldg, k, a.ngiven, list, nullptr, [&] {
            __syncthreads();                            // (the list of the row before is no longer read)
            float sum = 0.0f;
            for (int j = threadIdx.x; j < (a.ngiven + 3) / 4 * 4; j += THREADS) {
                const int64_t id = j < a.ngiven ? a.given[r * a.ngiven + j] : -1;
                const float z = row.at(id);
                const bool there = z != -INFINITY;
                const float g = there ? a.grad_logprobs[r * a.ngiven + j] : 0.0f;
                list.id[j] = there && slice.has(row, id) ? (int)id : -1;
                list.c[j] = g * a.scale;
                list.z[j] = z;
                sum += g;
            }
            if (a.ngiven > 0) {
                sum = group_sum<THREADS>(sum, sh);
                __syncthreads();
            }
            k.set(m, logsum, a.scale, -a.scale * (sum + gh * entropy), -a.scale * gh, m == -INFINITY);
        });
    }
}

// ---- a teacher's list
// What a thread holds of it: read() while the row's first chunks are on their way, finish() with the row's sums.
template <typename T, int THREADS>
struct Teacher {
    static constexpr int PER = kListPer<THREADS>;
    int id[PER];                        // -1: does not count
    float t[PER], z[PER];

    __device__ __forceinline__ void read(const Row<T>& row, const int64_t* ids, const float* teacher, int k)
    {
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int j = i * THREADS + threadIdx.x;
            id[i] = -1;
            t[i] = z[i] = -INFINITY;
            if (i * THREADS < k && j < k) {
                const int64_t at = ids[j];
                t[i] = teacher[j];
                z[i] = row.at(at);
                id[i] = (int)at;
            }
        }
    }
    // q of the entries that count into list.c, their entries and scores into list.id, list.z (0, -1 for the others), the loss and
    // whether any counts into list.loss, list.some: for all to read behind a barrier.  A list of 64 entries is the first wave's alone.
    __device__ __forceinline__ void finish(int k, float scale, const RowStat& st, float logsum, ListShared& list, RowShared<THREADS>& sh)
    {
        const bool one = k <= 64;
        if (one && threadIdx.x >= 64) return;
        auto all_max = [&](float v) { return one ? lanes_max(v) : group_max<THREADS>(v, sh); };
        auto all_sum = [&](float v) { return one ? lanes_sum(v) : group_sum<THREADS>(v, sh); };
        float top = -INFINITY;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            if (z[i] == -INFINITY || t[i] == -INFINITY) id[i] = -1;
            // (a NaN counts, and makes the loss NaN)
            if (id[i] >= 0) top = fmaxf(top, t[i] == t[i] ? t[i] : -FLT_MAX);
        }
        top = all_max(top);
        float sum = 0.0f, e[PER];
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            e[i] = id[i] >= 0 ? expf((t[i] - top) * scale) : 0.0f;
            sum += e[i];
        }
        sum = all_sum(sum);
        const float logq = logf(sum);
        float loss = 0.0f;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int j = i * THREADS + threadIdx.x;
            const float q = id[i] >= 0 ? e[i] / sum : 0.0f;
            // q (ln q - ln p), the part of ln p that may not fit float32 multiplied by q first (a student's mask of the lowest value)
            if (q != 0.0f) loss += fmaf(q * scale, st.m - z[i], q * ((t[i] - top) * scale - logq + logsum));
            if (j < (k + 3) / 4 * 4) { list.id[j] = id[i]; list.c[j] = q; list.z[j] = z[i]; }
        }
        loss = all_sum(loss);
        if (threadIdx.x == 0) {
            list.loss = loss;
            list.some = top != -INFINITY;
        }
    }
};

template <typename T, int THREADS, bool STEP, bool PARTS>
__global__ __launch_bounds__(THREADS) void k_distill(DistillArgs a)
{
    __shared__ RowShared<THREADS> sh;
    __shared__ ListShared list;
    for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const Row<T> row(a.logits, r * a.ld, a.n);
        Teacher<T, THREADS> teacher;
        auto read_teacher = [&] { teacher.read(row, a.ids + r * a.k, a.teacher + r * a.k, a.k); };
        Held<4, T> held;
        RowStat st;
        if constexpr (PARTS) {
            read_teacher();
            st = joined_stats(a.parts, r, a.scale * kLog2e);
        } else {
            st = row_stats<T, THREADS, false, false>(row, 0, row.nchunks, a.scale * kLog2e, sh, nullptr, 0, held, read_teacher);
        }
        const float logsum = st.log_sum();
        __syncthreads();                                 // (the list of the row before is no longer read)
        teacher.finish(a.k, a.scale, st, logsum, list, sh);
        __syncthreads();
        if (threadIdx.x == 0) {
            a.loss[r] = list.loss;
            if (a.norm) { a.norm[2 * r] = st.top(); a.norm[2 * r + 1] = logsum; }
        }
        for (int j = threadIdx.x; a.q && j < a.k; j += THREADS) a.q[r * a.k + j] = list.c[j];
        if (STEP) {
            const float w = (a.weights ? a.weights[r] : 1.0f) * a.scale;
            Coefficients k;
            k.set(st.top(), logsum, a.scale, w, 0.0f, !list.some || w == 0.0f);
            // (a thread scales its own entries, which are read behind the next barrier)
            for (int j = threadIdx.x; j < a.k; j += THREADS) list.c[j] *= -w;
            row_gradient<T, THREADS, false>(row, 0, row.nchunks, (T*)a.grad + r * a.ldg, k, a.k, list, &held, [] {});
        }
    }
}

template <typename T, int THREADS>
__global__ __launch_bounds__(THREADS) void k_distill_backward(DistillArgs a)
{
    __shared__ ListShared list;
    for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const Row<T> row(a.logits, r * a.ld, a.n);
        const Slice<T> slice(row, a.slice);
        const float m = a.norm[2 * r], logsum = a.norm[2 * r + 1], w = (a.weights ? a.weights[r] : 1.0f) * a.scale;
        Coefficients k;
        row_gradient<T, THREADS, false>(row, slice.begin, slice.end, (T*)a.grad + r * a.ldg, k, a.k, list, nullptr, [&] {
            __syncthreads();                            // (the list of the row before is no longer read)
            int some = 0;
            for (int j = threadIdx.x; j < (a.k + 3) / 4 * 4; j += THREADS) {
                const float q = j < a.k ? a.q[r * a.k + j] : 0.0f;
                const int64_t id = j < a.k ? a.ids[r * a.k + j] : -1;
                const bool counts = q != 0.0f && id >= 0 && id < a.n, mine = counts && slice.has(row, id);
                list.id[j] = mine ? (int)id : -1;
                list.c[j] = -w * q;
                list.z[j] = mine ? (float)row.z[id] : 0.0f;             // (other slices' scores may be gradients by now)
                some |= counts;
            }
            some = __syncthreads_or(some);
            k.set(m, logsum, a.scale, w, 0.0f, !some || w == 0.0f);
        });
    }
}

// ---- launches
static unsigned row_grid(int64_t rows) { return (unsigned)(rows < (1 << 20) ? rows : 1 << 20); }      // (a launch may not have 2^32 threads)

// Threads of the workgroup that takes a row (us a call with 64, 256, 1024 threads):
//   64    many short rows: what a row takes besides its scores is least with one wave, and with 256 threads the alternatives leave room for
//         1024 rows at a time.  float32, 10 alternatives: 4096 rows of 4096 21.5, 40, -, 1400 of 4000 13.0, 19.4, -, 1024 of 4000 12.1, 12.6, -;
//         128 of them: 4096 of 4096 51, 73, -, 2000 of 8000 49, 42, -  (the rule does not know how many are wanted: with that many, such rows
//         would be quicker with 256)
//   1024  few long rows: each has a compute unit for itself.  20 alternatives: one row of 131072 float32 101, 27, 17.5, 64 rows 105, 29, 18; 256
//         of 32768 35, 14, 14
//   256   the others: 1024 rows of 131072 139, 103, 120
static int row_threads(int dtype, int64_t rows, int64_t n)
{
    const int64_t chunks = n * (int64_t)element_bytes(dtype) / 16;
    if (chunks <= 2048 && rows > 1024) return 64;
    return chunks >= 4096 && rows < 256 ? 1024 : 256;
}

// f(element, threads) with the type and the number as compile-time values
template <typename F>
static void with_row_type(int dtype, int threads, F&& f)
{
    auto type = [&](auto e) {
        using std::integral_constant;
        if (threads == 64) f(e, integral_constant<int, 64>{});
        else if (threads == 256) f(e, integral_constant<int, 256>{});
        else f(e, integral_constant<int, 1024>{});
    };
    if (dtype == HR_F32) type(float{});
    else if (dtype == HR_F16) type(_Float16{});
    else type(__bf16{});
}

#define HR_ROWS_LAUNCH(kernel) hipLaunchKernelGGL(kernel, dim3(row_grid(a.rows)), dim3(decltype(threads)::value), 0, s, a)
#define HR_SLICES_LAUNCH(kernel) hipLaunchKernelGGL(kernel, dim3(row_grid(a.rows), slices), dim3(decltype(threads)::value), 0, s, a)

static int64_t row_chunks(int dtype, int64_t n) { return (n * (int64_t)element_bytes(dtype) + 15) / 16 + 1; }        // (at most)

// Parts of few long rows: 16, 1024 in all, of 1024 chunks at least, for rows of 192 KB and more (us a call, whole rows and in parts: one row of 131072
// bfloat16 with 20 alternatives 16.4, 10.9, gradient 15.2, 7.2, 65 rows of 600001 44, 21 without alternatives; 64 rows of 32768 float32, 128 KB, 11.7, 11.4, a step 12.4, 14.4: where one row of such a length or shorter would start to gain has not been measured).
constexpr int64_t kPartsInAll = 1024, kPartRow = 12288, kPartRows = 255;
static Parts row_parts(int dtype, int64_t rows, int64_t n)
{
    const int64_t chunks = row_chunks(dtype, n);
    Parts p{0, 0, nullptr, nullptr};
    if (rows < 1 || rows > kPartRows || chunks < kPartRow) return p;
    const int64_t parts = std::min({(int64_t)kMostParts, kPartsInAll / rows, chunks / 1024});
    p.len = (int)((chunks + parts * kPartThreads - 1) / (parts * kPartThreads) * kPartThreads);
    p.n = (int)((chunks + p.len - 1) / p.len);
    return p;
}
// places for the parts of any number of rows up to this one
static int64_t part_places(int64_t rows) { return std::min(rows * kMostParts, kPartsInAll); }
static size_t stats_bytes(int64_t rows) { return (size_t)part_places(rows) * 16; }
static size_t slots_bytes(int64_t rows) { return (size_t)part_places(rows) * kPartThreads * 4; }

// Slices of a row that workgroups write the gradient of, 1024 in all or rows with at least 1024 chunks each.
static int gradient_slices(int dtype, int64_t rows, int64_t n, int threads, int& slice)
{
    const int64_t chunks = row_chunks(dtype, n), want = std::max((int64_t)1, std::min((int64_t)1024 / rows, chunks / 1024));
    slice = (int)((chunks + want - 1) / want + threads - 1) / threads * threads;
    return (int)((chunks + slice - 1) / slice);
}

template <bool ENTROPY>
static void launch_parts(int dtype, const void* logits, int64_t ld, int64_t rows, int n, float scale, const Parts& parts, hipStream_t s)
{
    with_row_type(dtype, kPartThreads, [&](auto e, auto) {
        using T = decltype(e);
        const dim3 grid(parts.n, (unsigned)rows), block(kPartThreads);
        if (ENTROPY && parts.slots) hipLaunchKernelGGL((k_row_parts<T, ENTROPY, ENTROPY>), grid, block, 0, s, logits, ld, n, scale, parts);
        else hipLaunchKernelGGL((k_row_parts<T, ENTROPY, false>), grid, block, 0, s, logits, ld, n, scale, parts);
    });
}

static hipError_t launch_logprobs(int dtype, const LogprobsArgs& a, hipStream_t s)
{
    if (a.parts.n > 1) {
        launch_parts<true>(dtype, a.logits, a.ld, a.rows, a.n, a.scale, a.parts, s);
        with_row_type(dtype, 1024, [&](auto e, auto) {
            const std::integral_constant<int, 1024> threads;
            if (a.k > 0) HR_ROWS_LAUNCH((k_logprobs<decltype(e), 1024, true, true>));
            else HR_ROWS_LAUNCH((k_logprobs<decltype(e), 1024, false, true>));
        });
        return hipGetLastError();
    }
    with_row_type(dtype, row_threads(dtype, a.rows, a.n), [&](auto e, auto threads) {
        if (a.k > 0) HR_ROWS_LAUNCH((k_logprobs<decltype(e), decltype(threads)::value, true, false>));
        else HR_ROWS_LAUNCH((k_logprobs<decltype(e), decltype(threads)::value, false, false>));
    });
    return hipGetLastError();
}
static hipError_t launch_logprobs_backward(int dtype, LogprobsBackwardArgs a, hipStream_t s)
{
    // In the place of the scores a row has one workgroup: each looks at the scores of all given entries.
    const int few = row_threads(dtype, a.rows, a.n), chosen = a.grad == a.logits ? few : std::min(few, 256);
    int slices = 1;
    if (a.grad == a.logits) a.slice = (int)row_chunks(dtype, a.n);
    else slices = gradient_slices(dtype, a.rows, a.n, chosen, a.slice);
    with_row_type(dtype, chosen, [&](auto e, auto threads) { HR_SLICES_LAUNCH((k_logprobs_backward<decltype(e), decltype(threads)::value>)); });
    return hipGetLastError();
}
static hipError_t launch_distill(int dtype, const DistillArgs& a, hipStream_t s)
{
    if (a.parts.n > 1) {
        launch_parts<false>(dtype, a.logits, a.ld, a.rows, a.n, a.scale, a.parts, s);
        with_row_type(dtype, 256, [&](auto e, auto) {
            const std::integral_constant<int, 256> threads;
            HR_ROWS_LAUNCH((k_distill<decltype(e), 256, false, true>));
        });
        return hipGetLastError();
    }
    with_row_type(dtype, row_threads(dtype, a.rows, a.n), [&](auto e, auto threads) { HR_ROWS_LAUNCH((k_distill<decltype(e), decltype(threads)::value, false, false>)); });
    return hipGetLastError();
}
static hipError_t launch_distill_backward(int dtype, DistillArgs a, hipStream_t s)
{
    const int chosen = std::min(row_threads(dtype, a.rows, a.n), 256), slices = gradient_slices(dtype, a.rows, a.n, chosen, a.slice);
    with_row_type(dtype, chosen, [&](auto e, auto threads) { HR_SLICES_LAUNCH((k_distill_backward<decltype(e), decltype(threads)::value>)); });
    return hipGetLastError();
}
static hipError_t launch_distill_step(int dtype, const DistillArgs& a, hipStream_t s)
{
    if (a.parts.n > 1) {
        if (hipError_t e = launch_distill(dtype, a, s)) return e;
        return launch_distill_backward(dtype, a, s);
    }
    int chosen = row_threads(dtype, a.rows, a.n);
    // Rows are read again but for the eight chunks that each thread still holds, 32 KB of a row with 256 threads.  From 192 KB on twice as many
    // take it: half as many rows are under way, and of each twice as much is held (4096 rows of 131072 bfloat16 522, with 512 threads 496, with 1024 535;
    // 2048 rows 273, 240, 253; 1024 rows of 65536 float32 137, 128, 124; shorter ones, 2048 rows of 65537 binary16, 132, 133, 155).
    if (chosen == 256 && row_chunks(dtype, a.n) >= 12288) {
        with_row_type(dtype, 256, [&](auto e, auto) {
            const std::integral_constant<int, 512> threads;
            HR_ROWS_LAUNCH((k_distill<decltype(e), 512, true, false>));
        });
        return hipGetLastError();
    }
    with_row_type(dtype, chosen, [&](auto e, auto threads) { HR_ROWS_LAUNCH((k_distill<decltype(e), decltype(threads)::value, true, false>)); });
    return hipGetLastError();
}

}  // namespace hr

// ---- C entry points
using namespace hr;

static int check_rows(const void* logits, int64_t ld, int32_t dtype, int64_t rows, int64_t n, float scale)
{
    if (dtype != HR_F32 && dtype != HR_F16 && dtype != HR_BF16) return fail(HR_ERR_ARG, "unknown dtype %d", dtype);
    if (rows < 0 || rows > (1 << 24)) return fail(HR_ERR_ARG, "rows=%lld out of range", (long long)rows);
    if (n < 1 || n > HR_ROW_MAX) return fail(HR_ERR_ARG, "n=%lld must be in 1..%d", (long long)n, HR_ROW_MAX);
    if (ld < n || ld > (1LL << 40)) return fail(HR_ERR_ARG, "ld=%lld: rows of %lld scores overlap or are too far apart", (long long)ld, (long long)n);
    if (!(scale > 0.0f) || scale > 1e30f) return fail(HR_ERR_ARG, "scale=%g must be positive, at most 1e30", (double)scale);
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
    // (float32 has the most chunks; without alternatives no slots)
    if (row_chunks(HR_F32, n) < kPartRow) return HR_WORKSPACE_ALIGN;
    return aligned(stats_bytes(rows)) + (k > 0 ? slots_bytes(rows) : 0) + HR_WORKSPACE_ALIGN;
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
    LogprobsArgs a{logits, ld, rows, (int)n, scale, given, ngiven, k, out_logprobs, out_entropy, out_norm, out_top_ids, out_top_logprobs, row_parts(dtype, rows, n)};
    a.parts.stats = (float*)workspace;
    if (k > 0) a.parts.slots = (uint32_t*)((char*)workspace + aligned(stats_bytes(rows)));
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
    LogprobsBackwardArgs a{logits, ld, rows, (int)n, scale, given, grad_logprobs ? ngiven : 0, entropy, norm, grad_logprobs, grad_entropy, grad_logits, ldg, 0};
    HR_HIP(launch_logprobs_backward(dtype, a, (hipStream_t)stream));
    return HR_OK;
}

size_t hr_distill_workspace_bytes(int64_t rows, int64_t n, int32_t k)
{
    if (rows < 0 || rows > (1 << 24) || n < 1 || n > HR_ROW_MAX || k < 1 || k > HR_LIST_MAX) {
        fail(HR_ERR_ARG, "rows=%lld, n=%lld or k=%d out of range", (long long)rows, (long long)n, k);
        return 0;
    }
    if (row_chunks(HR_F32, n) < kPartRow) return HR_WORKSPACE_ALIGN;
    // (with rows in parts a step keeps what the backward call needs: there are few of them)
    const int64_t few = std::min(rows, kPartRows);
    return aligned(stats_bytes(rows)) + aligned((size_t)few * 8) + aligned((size_t)few * k * 4) + HR_WORKSPACE_ALIGN;
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
    DistillArgs a{logits, ld, rows, (int)n, scale, ids, teacher, k, nullptr, out_loss, out_norm, out_q, nullptr, 0, row_parts(dtype, rows, n), 0};
    a.parts.stats = (float*)workspace;
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
    DistillArgs a{logits, ld, rows, (int)n, scale, ids, nullptr, k, weights, nullptr, (float*)norm, (float*)q, grad_logits, ldg, {0, 0, nullptr, nullptr}, 0};
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
    DistillArgs a{logits, ld, rows, (int)n, scale, ids, teacher, k, weights, out_loss, out_norm, out_q, grad_logits, ldg, row_parts(dtype, rows, n), 0};
    a.parts.stats = (float*)workspace;
    if (a.parts.n > 1) {
        char* room = (char*)workspace + aligned(stats_bytes(rows));
        if (!a.norm) a.norm = (float*)room;
        if (!a.q) a.q = (float*)(room + aligned((size_t)rows * 8));
    }
    HR_HIP(launch_distill_step(dtype, a, (hipStream_t)stream));
    return HR_OK;
}

}  // extern "C"
