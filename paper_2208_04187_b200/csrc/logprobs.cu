// Log probabilities of given tokens, entropies, the most probable tokens, and the gradient of the logits.
//
//   m = max x,  s = sum exp(x - m),  t = sum (x - m) exp(x - m)          (one pass: running values, rescaled when m grows)
//   log p_j = (x_j - m) - log s,     entropy = log s - t / s
//   dx_j = dlp ([j = target] - p_j) - dH p_j (log p_j + H)
// m and log s are kept apart: their sum would lose log s next to a large m.
//
// Forward is bound by memory where the vocabulary is long (one reading of the logits), by the exponentials next (16 a clock and SM).  A
// cluster of 1 to 8 CTAs takes a row; a thread takes 16-byte pieces of it, LP_THREADS apart, 4 of them under way together, and
// joins its sums with the others' in a fixed order.  Additions and products go two at a time (f32x2).
//
// The most probable tokens come from the same pass.  The k-th largest of the 64 maxima of the CTA's groups of 4 threads is a bound that
// at least k logits reach; few others do (k-th of 64 groups: the N best logits lie in about 64 (1 - exp(-N/64)) groups, so that 20 groups
// are reached by 24).  Threads whose own maximum reaches it have their pieces read again, out of L2, by whole warps, and what
// reaches the bound is collected and ranked by counting.  Where more than LP_THREADS logits reach it (many equal ones, sorted rows,
// NaN) each warp keeps a sorted list across its lanes instead, and the lists are ranked.
#include "mx.cuh"

namespace divk {

constexpr uint32_t LP_THREADS = 256, LP_WARPS = LP_THREADS / 32, LP_MAX_TOP = 32, LP_MAX_CLUSTER = 8;
constexpr float LP_LOG2E = 1.4426950408889634f;
constexpr uint32_t LP_RESIDENT = 6, LP_SMEM = 228u * 1024u;      // CTAs of an SM; its shared memory
constexpr uint32_t LP_AT_ONCE = 4;              // pieces of a thread under way together
constexpr float LP_LEAST = -1000.f;             // exp of it is 0, and 0 times it is no NaN

struct LogprobParams {
    const void* x;
    uint64_t stride;
    uint32_t rows, vocab;
    const int64_t* targets;
    uint32_t top, split;
    float *logprobs, *entropy, *stats, *top_logprobs;
    int64_t* top_indices;
};

struct Running {
    float m, s, t;
};
__device__ __forceinline__ float max_nan(float a, float b) {
    float v;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(v) : "f"(a), "f"(b));
    return v;
}
__device__ __forceinline__ float exp2_fast(float a) {
    float v;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(v) : "f"(a));
    return v;
}
// brings r to a larger maximum
__device__ __forceinline__ void rescale(Running& r, float m) {
    if (m > r.m) {
        if (r.m != -INFINITY) {                        // (else nothing has been summed)
            const float d = max_nan(r.m - m, LP_LEAST), c = exp2_fast(d * LP_LOG2E);
            r.t = c * fmaf(r.s, d, r.t);
            r.s = c * r.s;
        }
        r.m = m;
    }
}
__device__ __forceinline__ Running join(Running a, const Running& b) {
    Running c = b;
    rescale(a, c.m);
    rescale(c, a.m);
    a.s += c.s;
    a.t += c.t;
    return a;
}
// two numbers in one register pair
__device__ __forceinline__ uint64_t two(float a, float b) {
    uint64_t v;
    asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(a), "f"(b));
    return v;
}
__device__ __forceinline__ void one_each(uint64_t v, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ uint64_t add_two(uint64_t a, uint64_t b) {
    uint64_t v;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(v) : "l"(a), "l"(b));
    return v;
}
__device__ __forceinline__ uint64_t mul_two(uint64_t a, uint64_t b) {
    uint64_t v;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(v) : "l"(a), "l"(b));
    return v;
}
__device__ __forceinline__ uint64_t fma_two(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t v;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(v) : "l"(a), "l"(b), "l"(c));
    return v;
}
// a thread's sums, in two halves
struct Sums {
    float m;
    uint64_t s, t;
    __device__ __forceinline__ void raise(float to) {
        if (to > m) {
            if (m != -INFINITY) {
                const float d = max_nan(m - to, LP_LEAST), c = exp2_fast(d * LP_LOG2E);
                t = mul_two(two(c, c), fma_two(s, two(d, d), t));
                s = mul_two(two(c, c), s);
            }
            m = to;
        }
    }
    // two numbers, neither above m (base: m, or 0 where nothing but -inf has come yet)
    __device__ __forceinline__ void take(uint64_t x, uint64_t minus_base) {
        float a, b;
        one_each(add_two(x, minus_base), a, b);
        a = max_nan(a, LP_LEAST);
        b = max_nan(b, LP_LEAST);
        const uint64_t ab = two(a, b);
        one_each(mul_two(ab, two(LP_LOG2E, LP_LOG2E)), a, b);
        const uint64_t e = two(exp2_fast(a), exp2_fast(b));
        s = add_two(s, e);
        t = fma_two(e, ab, t);
    }
    __device__ __forceinline__ Running whole() const {
        Running r;
        float s1, t1;
        r.m = m;
        one_each(s, r.s, s1);
        one_each(t, r.t, t1);
        r.s += s1;
        r.t += t1;
        return r;
    }
};
// 16 bytes of the row: their largest, and their pairs in 32 bits
template <typename T> struct Quad;
template <> struct Quad<float> {
    static __device__ __forceinline__ float largest(const uint4& q) {
        return fmaxf(fmaxf(__uint_as_float(q.x), __uint_as_float(q.y)), fmaxf(__uint_as_float(q.z), __uint_as_float(q.w)));
    }
    static __device__ __forceinline__ void take(Sums& r, const uint4& q, uint64_t minus_base) {
        r.take(two(__uint_as_float(q.x), __uint_as_float(q.y)), minus_base);
        r.take(two(__uint_as_float(q.z), __uint_as_float(q.w)), minus_base);
    }
};
template <> struct Quad<__nv_bfloat16> {
    static __device__ __forceinline__ float largest(const uint4& q) {
        const __nv_bfloat162 *a = reinterpret_cast<const __nv_bfloat162*>(&q);
        const __nv_bfloat162 m = __hmax2(__hmax2(a[0], a[1]), __hmax2(a[2], a[3]));
        return fmaxf(__low2float(m), __high2float(m));
    }
    static __device__ __forceinline__ void take(Sums& r, const uint4& q, uint64_t minus_base) {
        const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) r.take(two(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xFFFF0000u)), minus_base);
    }
};
template <> struct Quad<__half> {
    static __device__ __forceinline__ float largest(const uint4& q) {
        const __half2* a = reinterpret_cast<const __half2*>(&q);
        const __half2 m = __hmax2(__hmax2(a[0], a[1]), __hmax2(a[2], a[3]));
        return fmaxf(__low2float(m), __high2float(m));
    }
    static __device__ __forceinline__ void take(Sums& r, const uint4& q, uint64_t minus_base) {
        const __half2* a = reinterpret_cast<const __half2*>(&q);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 f = __half22float2(a[i]);
            r.take(two(f.x, f.y), minus_base);
        }
    }
};

// ---------------------------------------------------------------------------------------------
// 16-byte pieces of a row that may begin anywhere: piece 0 ends at the first multiple of 16 bytes
// ---------------------------------------------------------------------------------------------
template <typename T> struct Pieces {
    static constexpr uint32_t N = 16u / sizeof(T);
    const T* row;
    uint32_t first, count, vocab;                // numbers before the first whole piece (0..N-1); pieces in all
    __device__ __forceinline__ Pieces(const T* r, uint32_t v) : row(r), vocab(v) {
        first = (uint32_t)((16u - (reinterpret_cast<uintptr_t>(r) & 15u)) & 15u) / (uint32_t)sizeof(T);
        if (first > v) first = v;
        count = (first ? 1u : 0u) + (v - first + N - 1u) / N;
    }
    // index of the first number of a piece, and how many it has
    __device__ __forceinline__ uint32_t begin(uint32_t piece) const { return first ? (piece ? first + (piece - 1u) * N : 0u) : piece * N; }
    __device__ __forceinline__ uint32_t size(uint32_t piece) const {
        const uint32_t b = begin(piece), full = first && piece == 0 ? first : N;
        return min(full, vocab - b);
    }
    // numbers that are not there are -inf
    __device__ __forceinline__ void get(uint32_t piece, float (&v)[N]) const {
        const T* p = row + begin(piece);
        const uint32_t n = size(piece);
        if (n == N) {
            unpack(*reinterpret_cast<const uint4*>(p), v);
        } else {
#pragma unroll
            for (uint32_t i = 0; i < N; ++i) v[i] = i < n ? to_f32(p[i]) : -INFINITY;
        }
    }
    static __device__ __forceinline__ void unpack(const uint4& q, float (&v)[N]) {
        const uint32_t w[4] = {q.x, q.y, q.z, q.w};
        if (sizeof(T) == 4) {
#pragma unroll
            for (uint32_t i = 0; i < N; ++i) v[i] = __uint_as_float(w[i]);
        } else {
#pragma unroll
            for (uint32_t i = 0; i < N; ++i) {
                const unsigned short h = (unsigned short)(w[i >> 1] >> (16u * (i & 1u)));
                v[i] = to_f32(*reinterpret_cast<const T*>(&h));
            }
        }
    }
};

// ---------------------------------------------------------------------------------------------
// the most probable tokens: (key, index) pairs, larger keys first, then smaller indices
// ---------------------------------------------------------------------------------------------
__device__ __forceinline__ uint32_t order_key(float x) { return x != x ? 0xFFFFFFFFu : float_key(x + 0.f); }     // (-0 is 0; key 0 is nobody's)
__device__ __forceinline__ float key_value(uint32_t k) { return k == 0xFFFFFFFFu ? __uint_as_float(0x7FC00000u) : key_float(k); }
// a logit and its index as one number: larger logits are larger, of equal ones the smaller index; 0 is nobody's
__device__ __forceinline__ uint64_t entry(uint32_t key, uint32_t index) { return (uint64_t)key << 32 | (0xFFFFFFFFu - index); }
__device__ __forceinline__ uint32_t entry_key(uint64_t e) { return (uint32_t)(e >> 32); }
__device__ __forceinline__ uint32_t entry_index(uint64_t e) { return 0xFFFFFFFFu - (uint32_t)e; }

struct TopList {            // across the lanes of a warp, best first
    uint64_t mine, last;    // last: the top-th
    __device__ __forceinline__ void offer(bool have, uint64_t e, uint32_t top) {
        const uint32_t lane = threadIdx.x & 31u;
        uint32_t who = __ballot_sync(0xFFFFFFFFu, have && e > last);
        while (who) {
            const uint32_t src = (uint32_t)__ffs((int)who) - 1u;
            who &= who - 1u;
            const uint64_t c = __shfl_sync(0xFFFFFFFFu, e, src);
            if (c <= last) continue;
            const uint32_t at = (uint32_t)__popc(__ballot_sync(0xFFFFFFFFu, mine > c));
            const uint64_t up = __shfl_up_sync(0xFFFFFFFFu, mine, 1);
            mine = lane == at ? c : lane > at ? up : mine;
            last = __shfl_sync(0xFFFFFFFFu, mine, top - 1u);
        }
    }
};

constexpr uint32_t LP_GROUPS = LP_THREADS / 4;
struct LogprobShared {
    alignas(16) uint32_t maxima[LP_GROUPS];         // keys of the groups' maxima
    Running warps[LP_WARPS];
    Running cta;
    uint32_t bound, n_again, n_found;
    uint32_t again[LP_THREADS];                     // threads whose pieces are read again
    alignas(16) uint64_t found[LP_THREADS];          // what reaches the bound; the warps' lists; (of rank 0) the cluster's
    uint64_t best[LP_MAX_TOP];
};
static_assert(LP_WARPS * LP_MAX_TOP == LP_THREADS && LP_MAX_CLUSTER * LP_MAX_TOP <= LP_THREADS, "a list entry for each thread");

__device__ __forceinline__ uint32_t lp_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ uint32_t lp_peer(uint32_t local, uint32_t rank) {
    uint32_t at, v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(local), "r"(rank));
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(at) : "memory");
    return v;
}
__device__ __forceinline__ uint64_t lp_peer_entry(uint32_t local, uint32_t rank) {
    uint32_t at;
    uint64_t v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(local), "r"(rank));
    asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(at) : "memory");
    return v;
}
// the `top` best of the first n entries of sh.found go to sh.best (n even or followed by a 0); all threads together
__device__ __forceinline__ void lp_rank_entries(LogprobShared& sh, uint32_t n, uint32_t top) {
    if (threadIdx.x < n) {
        const uint64_t mine = sh.found[threadIdx.x];
        uint32_t better = 0;
        for (uint32_t j = 0; j < n; j += 2u) {
            const ulonglong2 two_of = *reinterpret_cast<const ulonglong2*>(&sh.found[j]);
            better += (two_of.x > mine ? 1u : 0u) + (two_of.y > mine ? 1u : 0u);
        }
        if (mine != 0u && better < top) sh.best[better] = mine;
    }
}

// (8 pieces of a thread under way together, of 2 to 4 CTAs an SM, took longer than 4 of 6: 37 rows of 131072 bf16 with 5 alternatives 14.5
// and 9.5 us.)
template <typename XT, bool TOP>
__global__ void __launch_bounds__(LP_THREADS, LP_RESIDENT)
logprob_forward_kernel(const __grid_constant__ LogprobParams p) {
    typedef Pieces<XT> P;
    __shared__ LogprobShared sh;
    const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5;
    const uint32_t row = blockIdx.x / p.split, rank = p.split > 1u ? lp_rank() : 0u;
    griddep_wait();
    griddep_launch();
    const P pieces(static_cast<const XT*>(p.x) + row * p.stride, p.vocab);
    const uint32_t from = (uint32_t)((uint64_t)pieces.count * rank / p.split), to = (uint32_t)((uint64_t)pieces.count * (rank + 1u) / p.split);

    Sums sums = {-INFINITY, 0ull, 0ull};
    // whole pieces: all but perhaps the row's first and its last
    const uint32_t w0 = max(from, pieces.first ? 1u : 0u), w1 = min(to, pieces.count - (pieces.size(pieces.count - 1u) < P::N ? 1u : 0u));
    const uint4* quads = reinterpret_cast<const uint4*>(pieces.row + pieces.first) - (pieces.first ? 1 : 0);       // (piece 0 is not read there)
    uint32_t piece = from + threadIdx.x;
    if (piece < w0) piece += LP_THREADS;
    for (; piece + (LP_AT_ONCE - 1u) * LP_THREADS < w1; piece += LP_AT_ONCE * LP_THREADS) {
        uint4 q[LP_AT_ONCE];
#pragma unroll
        for (uint32_t u = 0; u < LP_AT_ONCE; ++u) q[u] = quads[piece + u * LP_THREADS];
        float m = Quad<XT>::largest(q[0]);
#pragma unroll
        for (uint32_t u = 1; u < LP_AT_ONCE; ++u) m = fmaxf(m, Quad<XT>::largest(q[u]));
        sums.raise(m);
        const float base = sums.m == -INFINITY ? 0.f : sums.m;
        const uint64_t minus = two(-base, -base);
#pragma unroll
        for (uint32_t u = 0; u < LP_AT_ONCE; ++u) Quad<XT>::take(sums, q[u], minus);
    }
    {
        // the rest, still all under way together
        uint4 q[LP_AT_ONCE];
#pragma unroll
        for (uint32_t u = 0; u < LP_AT_ONCE; ++u)
            if (piece + u * LP_THREADS < w1) q[u] = quads[piece + u * LP_THREADS];
#pragma unroll
        for (uint32_t u = 0; u < LP_AT_ONCE; ++u) {
            if (piece + u * LP_THREADS < w1) {
                sums.raise(Quad<XT>::largest(q[u]));
                const float base = sums.m == -INFINITY ? 0.f : sums.m;
                Quad<XT>::take(sums, q[u], two(-base, -base));
            }
        }
    }
    // the first and the last piece, if cut: by the thread whose they are
    for (uint32_t end = 0; end < 2u; ++end) {
        const uint32_t cut = end ? pieces.count - 1u : 0u;
        if (cut >= from && cut < to && (cut < w0 || cut >= w1) && (end == 0u || cut != 0u) && (cut - from) % LP_THREADS == threadIdx.x) {
            float v[P::N];
            pieces.get(cut, v);
#pragma unroll
            for (uint32_t i = 0; i < P::N; i += 2u) {
                sums.raise(fmaxf(v[i], v[i + 1u]));
                const float base = sums.m == -INFINITY ? 0.f : sums.m;
                sums.take(two(v[i], v[i + 1u]), two(-base, -base));
            }
        }
    }
    Running r = sums.whole();
    const float thread_max = r.m;
#pragma unroll
    for (int d = 16; d; d >>= 1) {
        Running o;
        o.m = __shfl_xor_sync(0xFFFFFFFFu, r.m, d);
        o.s = __shfl_xor_sync(0xFFFFFFFFu, r.s, d);
        o.t = __shfl_xor_sync(0xFFFFFFFFu, r.t, d);
        // (both lanes of a pair join in the same order, so that they agree to the bit)
        const bool low = (lane & d) == 0;
        r = join(low ? r : o, low ? o : r);
    }
    if (lane == 0) sh.warps[warp] = r;
    const uint32_t mine = TOP && from + threadIdx.x < to ? order_key(thread_max) : 0u;
    if (TOP) {
        const uint32_t pair = max(mine, __shfl_xor_sync(0xFFFFFFFFu, mine, 1)), group = max(pair, __shfl_xor_sync(0xFFFFFFFFu, pair, 2));
        if ((lane & 3u) == 0) sh.maxima[threadIdx.x >> 2] = group;
        if (threadIdx.x == 0) sh.n_again = sh.n_found = 0;
    }
    __syncthreads();
    r = sh.warps[0];
    for (uint32_t w = 1; w < LP_WARPS; ++w) r = join(r, sh.warps[w]);
    if (threadIdx.x == 0) sh.cta = r;

    if (TOP) {
        // the top-th largest of the groups' maxima; 0 (everything) where not that many groups had a piece.  A sum that is NaN may come
        // from a NaN, which no maximum shows: everything is read again.  (4 threads count for a group, a quarter of the others each.)
        const uint32_t group = sh.maxima[threadIdx.x >> 2];
        uint32_t above = 0, reach = 0;
#pragma unroll
        for (uint32_t j = 0; j < LP_GROUPS / 4u; j += 4u) {
            const uint4 k = *reinterpret_cast<const uint4*>(&sh.maxima[(lane & 3u) * (LP_GROUPS / 4u) + j]);
            above += (k.x > group) + (k.y > group) + (k.z > group) + (k.w > group);
            reach += (k.x >= group) + (k.y >= group) + (k.z >= group) + (k.w >= group);
        }
        uint32_t both = above << 16 | reach;
        both += __shfl_xor_sync(0xFFFFFFFFu, both, 1);
        both += __shfl_xor_sync(0xFFFFFFFFu, both, 2);
        if ((both >> 16) < p.top && (both & 0xFFFFu) >= p.top) sh.bound = group;       // (all that write, write the same)
        if (threadIdx.x < LP_MAX_TOP) sh.best[threadIdx.x] = 0u;        // (a CTA of a cluster may hold fewer than `top`)
        __syncthreads();
        const uint32_t bound = r.s != r.s ? 0u : sh.bound;
        if (from + threadIdx.x < to && mine >= bound) sh.again[atomicAdd(&sh.n_again, 1u)] = threadIdx.x;
        __syncthreads();
        const uint32_t each = (to - from + LP_THREADS - 1u) / LP_THREADS;          // pieces of a thread, at most
        const uint32_t items = sh.n_again * each;
        for (uint32_t item = threadIdx.x; item < items; item += LP_THREADS) {
            if (*(volatile uint32_t*)&sh.n_found > LP_THREADS) break;                // (lists are the way then)
            const uint32_t at = from + sh.again[item / each] + item % each * LP_THREADS;
            if (at < to) {
                float v[P::N];
                pieces.get(at, v);
                const uint32_t n = pieces.size(at), first = pieces.begin(at);
#pragma unroll
                for (uint32_t i = 0; i < P::N; ++i) {
                    const uint32_t k = order_key(v[i]);
                    if (i < n && k >= bound) {
                        const uint32_t slot = atomicAdd(&sh.n_found, 1u);
                        if (slot < LP_THREADS) sh.found[slot] = entry(k, first + i);
                    }
                }
            }
        }
        __syncthreads();
        uint32_t n = sh.n_found;
        __syncthreads();                                   // (nobody writes entries before all have seen the count)
        if (n > LP_THREADS) {
            TopList list = {0u, 0u};
            const uint32_t rounds = (items + LP_THREADS - 1u) / LP_THREADS;
            for (uint32_t round = 0; round < rounds; ++round) {
                const uint32_t item = round * LP_THREADS + threadIdx.x, at = item < items ? from + sh.again[item / each] + item % each * LP_THREADS : to;
                float v[P::N];
#pragma unroll
                for (uint32_t i = 0; i < P::N; ++i) v[i] = -INFINITY;
                const uint32_t have = at < to ? pieces.size(at) : 0u, first = at < to ? pieces.begin(at) : 0u;
                if (have) pieces.get(at, v);
#pragma unroll
                for (uint32_t i = 0; i < P::N; ++i) {
                    const uint32_t k = order_key(v[i]);
                    list.offer(i < have && k >= bound, entry(k, first + i), p.top);
                }
            }
            __syncthreads();
            sh.found[threadIdx.x] = lane < p.top ? list.mine : 0u;
            n = LP_THREADS;
        } else if (threadIdx.x == 0 && n < LP_THREADS) {
            sh.found[n] = 0u;
        }
        __syncthreads();
        lp_rank_entries(sh, n, p.top);
    }
    if (p.split > 1u) {
        asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
        if (rank == 0) {
            // a lane to a CTA of the cluster, then one after another
            const uint32_t at = (uint32_t)__cvta_generic_to_shared(&sh.cta), from_cta = lane < p.split ? lane : 0u;
            Running o;
            o.m = __uint_as_float(lp_peer(at, from_cta));
            o.s = __uint_as_float(lp_peer(at + 4u, from_cta));
            o.t = __uint_as_float(lp_peer(at + 8u, from_cta));
            uint64_t e = 0u;
            if (TOP && threadIdx.x < p.split * p.top)
                e = lp_peer_entry((uint32_t)__cvta_generic_to_shared(&sh.best[threadIdx.x % p.top]), threadIdx.x / p.top);
            for (uint32_t c = 1; c < p.split; ++c) {
                Running q;
                q.m = __shfl_sync(0xFFFFFFFFu, o.m, c);
                q.s = __shfl_sync(0xFFFFFFFFu, o.s, c);
                q.t = __shfl_sync(0xFFFFFFFFu, o.t, c);
                r = join(r, q);
            }
            if (TOP) {
                __syncthreads();
                sh.found[threadIdx.x] = e;
                __syncthreads();
                lp_rank_entries(sh, p.split * p.top, p.top);        // (even: split is)
            }
        }
        asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
        if (rank != 0) return;
    }
    if (TOP) __syncthreads();
    const bool empty = r.m == -INFINITY && r.s == 0.f;
    const float m = empty ? 0.f : r.m, log_s = empty ? INFINITY : logf(r.s);
    if (threadIdx.x == 0) {
        const int64_t target = p.targets[row];
        float lp = 0.f;
        if (target >= (int64_t)p.vocab) lp = __uint_as_float(0x7FC00000u);
        else if (target >= 0) lp = (to_f32(pieces.row[target]) - m) - log_s;
        p.logprobs[row] = lp;
        p.entropy[row] = empty ? 0.f : log_s - r.t / r.s;
        p.stats[2ull * row] = m;
        p.stats[2ull * row + 1u] = log_s;
    }
    if (TOP && threadIdx.x < p.top) {
        p.top_logprobs[(uint64_t)row * p.top + threadIdx.x] = (key_value(entry_key(sh.best[threadIdx.x])) - m) - log_s;
        p.top_indices[(uint64_t)row * p.top + threadIdx.x] = (int64_t)entry_index(sh.best[threadIdx.x]);
    }
}

struct LogprobBackParams {
    const void* x;
    uint64_t stride;
    uint32_t rows, vocab;
    const int64_t* targets;
    const float *stats, *entropy, *dlogprobs, *dentropy;
    void* dx;
    uint32_t chunks;            // CTAs of a row
};
constexpr uint32_t LP_BACK_EACH = 4;          // pieces of a thread

// pairs of dlogits -> 16 bytes
template <typename T> struct Pack;
template <> struct Pack<float> {
    static __device__ __forceinline__ void put(uint4& q, int pair, float a, float b) {
        if (pair == 0) q.x = __float_as_uint(a), q.y = __float_as_uint(b);
        else q.z = __float_as_uint(a), q.w = __float_as_uint(b);
    }
    static __device__ __forceinline__ uint64_t get(const uint4& q, int pair) {
        return pair == 0 ? two(__uint_as_float(q.x), __uint_as_float(q.y)) : two(__uint_as_float(q.z), __uint_as_float(q.w));
    }
};
template <> struct Pack<__nv_bfloat16> {
    static __device__ __forceinline__ void put(uint4& q, int pair, float a, float b) { reinterpret_cast<__nv_bfloat162*>(&q)[pair] = __floats2bfloat162_rn(a, b); }
    static __device__ __forceinline__ uint64_t get(const uint4& q, int pair) {
        const uint32_t w = reinterpret_cast<const uint32_t*>(&q)[pair];
        return two(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
    }
};
template <> struct Pack<__half> {
    static __device__ __forceinline__ void put(uint4& q, int pair, float a, float b) { reinterpret_cast<__half2*>(&q)[pair] = __floats2half2_rn(a, b); }
    static __device__ __forceinline__ uint64_t get(const uint4& q, int pair) {
        const float2 f = __half22float2(reinterpret_cast<const __half2*>(&q)[pair]);
        return two(f.x, f.y);
    }
};
struct Slope {                                // of a row
    float m, log_s, dent, c0, dlp;
    // -p (dent log p + c0) of two logits
    __device__ __forceinline__ void apply(uint64_t x, float& a, float& b) const {
        one_each(add_two(add_two(x, two(-m, -m)), two(-log_s, -log_s)), a, b);
        const uint64_t lp = two(max_nan(a, LP_LEAST), max_nan(b, LP_LEAST));
        one_each(mul_two(lp, two(LP_LOG2E, LP_LOG2E)), a, b);
        const uint64_t p = two(-exp2_fast(a), -exp2_fast(b));
        one_each(mul_two(p, fma_two(two(dent, dent), lp, two(c0, c0))), a, b);
    }
};

// A thread takes LP_BACK_EACH pieces, their reads under way together; the target's number is stored once more by the thread whose it is.
// Bound by memory: one reading, one writing.
template <typename XT>
__global__ void __launch_bounds__(LP_THREADS)
logprob_backward_kernel(const __grid_constant__ LogprobBackParams p) {
    typedef Pieces<XT> P;
    griddep_wait();
    griddep_launch();
    const uint32_t row = blockIdx.x / p.chunks, chunk = blockIdx.x % p.chunks;
    const P pieces(static_cast<const XT*>(p.x) + row * p.stride, p.vocab);
    XT* out = static_cast<XT*>(p.dx) + (uint64_t)row * p.vocab;
    const bool same = ((reinterpret_cast<uintptr_t>(out) ^ reinterpret_cast<uintptr_t>(pieces.row)) & 15u) == 0;      // pieces begin alike
    const uint32_t c0 = chunk * LP_THREADS * LP_BACK_EACH, first = c0 + threadIdx.x;
    // all pieces of the CTA are whole ones, and written as they are read
    const bool plain = same && c0 + LP_THREADS * LP_BACK_EACH < pieces.count && (c0 != 0u || pieces.first == 0u);
    uint4 q[LP_BACK_EACH];
    if (plain) {
#pragma unroll
        for (uint32_t u = 0; u < LP_BACK_EACH; ++u) q[u] = __ldcs(reinterpret_cast<const uint4*>(pieces.row + pieces.begin(first + u * LP_THREADS)));
    }
    Slope s;
    s.m = p.stats[2ull * row];
    s.log_s = p.stats[2ull * row + 1u];
    const int64_t target = p.targets[row];
    s.dlp = p.dlogprobs ? p.dlogprobs[row] : 0.f;
    if (target < 0 || s.log_s == INFINITY) s.dlp = 0.f;
    else if (target >= (int64_t)p.vocab) s.dlp = __uint_as_float(0x7FC00000u);
    s.dent = p.dentropy ? p.dentropy[row] : 0.f;
    s.c0 = p.dentropy ? fmaf(s.dent, p.entropy[row], s.dlp) : s.dlp;
    const uint32_t hit = target >= 0 && target < (int64_t)p.vocab ? (uint32_t)target : 0xFFFFFFFFu;
    if (plain) {
#pragma unroll
        for (uint32_t u = 0; u < LP_BACK_EACH; ++u) {
            const uint32_t begin = pieces.begin(first + u * LP_THREADS);
            uint4 d;
#pragma unroll
            for (int i = 0; i < (int)P::N / 2; ++i) {
                float a, b;
                s.apply(Pack<XT>::get(q[u], i), a, b);
                Pack<XT>::put(d, i, a, b);
            }
            __stcs(reinterpret_cast<uint4*>(out + begin), d);
        }
    } else {
        for (uint32_t u = 0; u < LP_BACK_EACH; ++u) {
            const uint32_t piece = first + u * LP_THREADS;
            if (piece >= pieces.count) break;
            const uint32_t begin = pieces.begin(piece), n = pieces.size(piece);
            float v[P::N];
            pieces.get(piece, v);
#pragma unroll
            for (uint32_t i = 0; i < P::N; i += 2u) {
                float a, b;
                s.apply(two(v[i], v[i + 1u]), a, b);
                if (i < n) out[begin + i] = from_f32<XT>(a);
                if (i + 1u < n) out[begin + i + 1u] = from_f32<XT>(b);
            }
        }
    }
    if (hit != 0xFFFFFFFFu) {
        const uint32_t piece = pieces.first ? (hit < pieces.first ? 0u : 1u + (hit - pieces.first) / P::N) : hit / P::N;
        if (piece >= c0 && piece - c0 < LP_THREADS * LP_BACK_EACH && (piece - c0) % LP_THREADS == threadIdx.x) {
            float a, b;
            s.apply(two(to_f32(pieces.row[hit]), 0.f), a, b);
            out[hit] = from_f32<XT>(a + s.dlp);
        }
    }
}

}  // namespace divk

namespace {
using namespace divk;
inline bool aligned_to(const void* p, uintptr_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }
}  // namespace

extern "C" {

div_status div_token_logprobs_forward(const void* logits_dev, int64_t row_stride, int64_t rows, int64_t vocab, int32_t dtype, const int64_t* targets_dev,
                                      int32_t top, float* logprobs_dev, float* entropy_dev, float* stats_dev, float* top_logprobs_dev,
                                      int64_t* top_indices_dev, void* cuda_stream) {
    if (!logits_dev || !targets_dev || !logprobs_dev || !entropy_dev || !stats_dev || (top > 0 && (!top_logprobs_dev || !top_indices_dev))) return DIV_ERR_NULL;
    if (!lm_size_ok(rows) || !lm_size_ok(vocab) || (rows > 1 && row_stride < vocab)) return DIV_ERR_SHAPE;
    if (!lm_dtype_ok(dtype) || top < 0 || top > (int32_t)LP_MAX_TOP || top > vocab) return DIV_ERR_PARAM;
    if (!aligned_to(logits_dev, lm_dtype_bytes(dtype)) || !aligned_to(targets_dev, 8) || !aligned_to(logprobs_dev, 4) || !aligned_to(entropy_dev, 4) ||
        !aligned_to(stats_dev, 4) || !aligned_to(top_logprobs_dev, 4) || !aligned_to(top_indices_dev, 8))
        return DIV_ERR_ALIGN;
    LogprobParams p;
    p.x = logits_dev;
    p.stride = (uint64_t)row_stride;
    p.rows = (uint32_t)rows;
    p.vocab = (uint32_t)vocab;
    p.targets = targets_dev;
    p.top = (uint32_t)top;
    p.logprobs = logprobs_dev;
    p.entropy = entropy_dev;
    p.stats = stats_dev;
    p.top_logprobs = top_logprobs_dev;
    p.top_indices = top_indices_dev;
    // few rows: a cluster each, as long as every thread of it has a piece
    const uint64_t pieces = (uint64_t)vocab * lm_dtype_bytes(dtype) / 16u;
    uint32_t split = 1;
    while (split < LP_MAX_CLUSTER && (uint64_t)rows * split < 296u && pieces >= 2ull * split * LP_THREADS) split *= 2u;
    p.split = split;
    if ((uint64_t)rows * split >= (1ull << 31) - 512u) return DIV_ERR_SHAPE;
    return with_type(dtype, [&](auto* t) {
        typedef std::remove_pointer_t<decltype(t)> XT;
        auto kern = top ? logprob_forward_kernel<XT, true> : logprob_forward_kernel<XT, false>;
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3((uint32_t)rows * split);
        cfg.blockDim = dim3(LP_THREADS);
        cfg.stream = (cudaStream_t)cuda_stream;
        // Fewer CTAs than places: some SMs would get 6 while others get 2.  Shared memory that nobody uses leaves as many places as an even
        // share takes.  For 16-bit types and shares of 4 and 5 only: 131072 bf16 with 5 alternatives, 260 rows in clusters of two 27.7 -> 22.2 us,
        // 450 rows 45.4 -> 35.5, 600 46.7 -> 42.9, 740 42.2 -> 45.7; of 32000 260 14.4 -> 11.6, 592 12.4 -> 12.8.  With shares of 2 and 3 it gives
        // nothing (300 rows 27.2 and 28.0, 400 29.2 and 29.4), and float32 takes longer with any (50257 numbers, 300 rows 18.3 and 22.4, 500 26.1
        // and 30.8, 650 28.9 and 40.0).
        const uint32_t share = ((uint32_t)rows * split + 147u) / 148u;
        if (sizeof(XT) == 2 && split <= 2u && share < LP_RESIDENT && share > 3u) {
            static SmemAllowed allowed[2];
            cfg.dynamicSmemBytes = LP_SMEM / share - 5u * 1024u;              // (what a CTA has besides: its own 3.7 KB, the system's 1 KB)
            if (!allowed[top ? 1 : 0]((const void*)kern, LP_SMEM / 4u)) return DIV_ERR_CUDA;
        }
        cudaLaunchAttribute at[2];
        at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        at[0].val.programmaticStreamSerializationAllowed = 1;
        at[1].id = cudaLaunchAttributeClusterDimension;
        at[1].val.clusterDim.x = split;
        at[1].val.clusterDim.y = 1;
        at[1].val.clusterDim.z = 1;
        cfg.attrs = at;
        cfg.numAttrs = 2;
        if (cudaLaunchKernelEx(&cfg, kern, p) != cudaSuccess) {
            cudaGetLastError();
            return DIV_ERR_CUDA;
        }
        return DIV_OK;
    });
}

div_status div_token_logprobs_backward(const void* logits_dev, int64_t row_stride, int64_t rows, int64_t vocab, int32_t dtype, const int64_t* targets_dev,
                                       const float* stats_dev, const float* entropy_dev, const float* dlogprobs_dev, const float* dentropy_dev,
                                       void* dlogits_dev, void* cuda_stream) {
    if (!logits_dev || !targets_dev || !stats_dev || (dentropy_dev && !entropy_dev) || !dlogits_dev) return DIV_ERR_NULL;
    if (!lm_size_ok(rows) || !lm_size_ok(vocab) || (rows > 1 && row_stride < vocab)) return DIV_ERR_SHAPE;
    if (!lm_dtype_ok(dtype)) return DIV_ERR_PARAM;
    if (!aligned_to(logits_dev, lm_dtype_bytes(dtype)) || !aligned_to(targets_dev, 8) || !aligned_to(stats_dev, 4) || !aligned_to(entropy_dev, 4) ||
        !aligned_to(dlogprobs_dev, 4) || !aligned_to(dentropy_dev, 4) || !aligned_to(dlogits_dev, lm_dtype_bytes(dtype)))
        return DIV_ERR_ALIGN;
    LogprobBackParams p;
    p.x = logits_dev;
    p.stride = (uint64_t)row_stride;
    p.rows = (uint32_t)rows;
    p.vocab = (uint32_t)vocab;
    p.targets = targets_dev;
    p.stats = stats_dev;
    p.entropy = entropy_dev;
    p.dlogprobs = dlogprobs_dev;
    p.dentropy = dentropy_dev;
    p.dx = dlogits_dev;
    const uint64_t each = 16u / lm_dtype_bytes(dtype), most = ((uint64_t)vocab + 2u * each - 2u) / each;      // pieces, wherever a row begins
    const uint64_t chunks = (most + LP_THREADS * LP_BACK_EACH - 1u) / (LP_THREADS * LP_BACK_EACH);
    p.chunks = (uint32_t)chunks;
    if ((uint64_t)rows * chunks >= (1ull << 31)) return DIV_ERR_SHAPE;
    return with_type(dtype, [&](auto* t) {
        typedef std::remove_pointer_t<decltype(t)> XT;
        return launch_pdl(logprob_backward_kernel<XT>, dim3((uint32_t)(rows * chunks)), LP_THREADS, 0, (cudaStream_t)cuda_stream, p);
    });
}

}  // extern "C"
