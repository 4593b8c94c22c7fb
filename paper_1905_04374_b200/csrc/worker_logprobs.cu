// Token log probabilities with entropy and top alternatives, and their gradient (gar_worker.h).
//
// Forward.  Every thread runs the softmax recurrence over its share of a row: with m the largest
// value so far, s = sum e^(x-m) and u = sum e^(x-m) (x-m) log2(e); a larger m' rescales
//     f = e^(m-m'),  u <- f (u + s (m-m') log2(e)),  s <- f s.
// x - m is formed before the product with log2(e), so large logits lose nothing to cancellation.  A
// masked entry (-inf) must add e = 0 and 0 to u, not 0 * inf: where a tile holds one, the exponents
// are kept above -1e4.  Shares are joined by the same rescaling: lanes, warps, then (rows split over
// a cluster) CTAs through distributed shared memory.
//
// The k best entries cost that loop one store: the maximum of every tile of a thread's share (32 bytes
// to 16 KB).  With j = ceil(k / warps), the j-th largest of the tile maxima of a warp (two of each thread
// count), taken as the least over the warps, has at least k entries not below it; only the tiles whose maximum reaches it are read
// again, about two k of them, and of those the entries that reach it are ranked by counting.  A 64-bit
// key (value in an order-preserving code, complement of the index) makes the order total: equal values
// go to the lowest index.  If more entries qualify than the list holds (rows with many equal values,
// such as heavily masked ones) the k best are extracted one by one instead.
#include <cooperative_groups.h>

#include "worker_common.cuh"

namespace cg = cooperative_groups;

namespace gar {
namespace worker {
namespace {

constexpr int LP_THREADS = 256;
constexpr int LP_WARPS = LP_THREADS / 32;
constexpr int LP_UNROLL = 4;            // 16-byte slots of a thread's turn (find_top's shift counts on 4)
constexpr int LP_TILES = 16;            // tiles of a thread's share
constexpr int LP_MAX_CLUSTER = 8;
constexpr int LP_WARP_VOCAB = 16384;    // longest row that one warp takes
constexpr float LP_FLOOR = -1e4f;       // exponents below this are 0 in fp32
constexpr float LP_HUGE = 1e30f;        // between -LP_HUGE and LP_HUGE no exponent overflows

struct Softmax {
    float m, s, u;
};
__device__ __forceinline__ float centre(float m) { return m == -CUDART_INF_F ? 0.f : m; }

__device__ __forceinline__ void raise(Softmax& a, float m) {
    if (a.m == -CUDART_INF_F) {          // nothing but masked (or NaN) entries so far: they have added 0 (or NaN)
        a.m = m;
        return;
    }
    const float d = (a.m - m) * kLog2e, f = ex2(d);
    // f == 0 drops the old sums; d may be -inf then
    a.u = f > 0.f ? f * (a.u + a.s * d) : (a.u + a.s) * 0.f;
    a.s = a.s * f;
    a.m = m;
}
__device__ __forceinline__ void join(Softmax& a, Softmax b) {
    if (b.m > a.m) raise(a, b.m);
    else if (a.m > b.m) raise(b, a.m);
    a.s += b.s;
    a.u += b.u;
}
__device__ __forceinline__ void add_one(Softmax& a, float x) {
    if (x > a.m) raise(a, x);
    const float t = max_nan((x - centre(a.m)) * kLog2e, LP_FLOOR), e = ex2(t);
    a.s += e;
    a.u += e * t;
}

// Order-preserving code of a value: larger value, larger code; -0 = +0; NaN lowest.
__device__ __forceinline__ unsigned code_of(float x) {
    if (x != x) return 0u;
    const unsigned b = __float_as_uint(x + 0.f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(unsigned c) {
    if (c == 0u) return CUDART_NAN_F;
    return __uint_as_float(c & 0x80000000u ? c & 0x7fffffffu : ~c);
}
__device__ __forceinline__ unsigned long long key_of(float x, unsigned idx) {
    return (static_cast<unsigned long long>(code_of(x)) << 32) | (0xffffffffu - idx);
}

__device__ __forceinline__ unsigned long long shfl_xor64(unsigned long long v, int o) {
    return __shfl_xor_sync(0xffffffffu, v, o);
}

// What a row comes to, from its joined sums.  A NaN or +inf in the row has made s a NaN, and with it
// everything here.  An empty row gets m = 0 and log s = +inf: every log probability is then -inf.
struct RowResult {
    float lse, lse_lo, entropy, log_s, m;
};
__device__ __forceinline__ RowResult finish(const Softmax& a) {
    RowResult r;
    r.m = a.m;
    r.log_s = logf(a.s);
    r.lse = __fadd_rn(a.m, r.log_s);
    // the rounding error of m + log s, exactly (two-sum)
    const float part = __fsub_rn(r.lse, a.m);
    r.lse_lo = __fadd_rn(__fsub_rn(a.m, __fsub_rn(r.lse, part)), __fsub_rn(r.log_s, part));
    r.entropy = r.log_s - (a.u / a.s) * 0.69314718055994531f;
    if (a.m == -CUDART_INF_F && a.s == 0.f) {
        r.m = 0.f;
        r.log_s = CUDART_INF_F;
        r.lse = -CUDART_INF_F;
        r.lse_lo = r.entropy = 0.f;
    }
    return r;
}
__device__ __forceinline__ float logprob_of(const RowResult& r, float x) { return (x - r.m) - r.log_s; }

template <typename T>
__device__ __forceinline__ float load_one(const T* row, int64_t j) { return Elem<T>::widen(row[j]); }

struct ForwardArgs {
    const void*    logits;
    int64_t        rows, vocab, ld;
    const int64_t* targets;
    float *        logprobs, *entropy, *lse, *lse_lo, *top_logprobs;
    int64_t*       top_index;
    int            top;
};

// The target's logit, asked for before the row is worked on.
struct Target {
    int64_t index;               // < 0: none
    float   x;
};
template <typename T>
__device__ __forceinline__ Target read_target(const ForwardArgs& a, int64_t row) {
    Target t{-1, 0.f};
    if (a.logprobs) {
        t.index = a.targets[row];
        if (t.index >= 0 && t.index < a.vocab) t.x = load_one(static_cast<const T*>(a.logits) + row * a.ld, t.index);
    }
    return t;
}
__device__ __forceinline__ void store_row(const ForwardArgs& a, int64_t row, const RowResult& r, const Target& t) {
    if (a.lse) a.lse[row] = r.lse;
    if (a.lse_lo) a.lse_lo[row] = r.lse_lo;
    if (a.entropy) a.entropy[row] = r.entropy;
    if (a.logprobs) a.logprobs[row] = t.index < 0 ? 0.f : t.index >= a.vocab ? CUDART_NAN_F : logprob_of(r, t.x);
}
__device__ __forceinline__ void store_top(const ForwardArgs& a, int64_t row, int rank, unsigned long long key, const RowResult& r) {
    a.top_logprobs[row * a.top + rank] = logprob_of(r, value_of(unsigned(key >> 32)));
    a.top_index[row * a.top + rank] = int64_t(0xffffffffu - unsigned(key));
}

// ---- rows of up to 256 entries: L lanes hold a row in registers, EPL entries each ----------------
template <typename T, int L, int EPL>
__global__ void __launch_bounds__(LP_THREADS) logprobs_small_kernel(const ForwardArgs a) {
    const int lane = threadIdx.x % L;
    const int64_t row = (int64_t(blockIdx.x) * LP_THREADS + threadIdx.x) / L;
    const bool live = row < a.rows;
    const T* x = static_cast<const T*>(a.logits) + (live ? row : 0) * a.ld;
    const int vocab = int(a.vocab);
    float v[EPL];
#pragma unroll
    for (int i = 0; i < EPL; ++i) {
        const int j = lane + i * L;
        v[i] = j < vocab ? load_one(x, j) : -CUDART_INF_F;
    }
    const Target target = live && lane == 0 ? read_target<T>(a, row) : Target{-1, 0.f};
    Softmax st{-CUDART_INF_F, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < EPL; ++i) st.m = fmaxf(st.m, v[i]);
#pragma unroll
    for (int o = L / 2; o; o >>= 1) st.m = fmaxf(st.m, __shfl_xor_sync(0xffffffffu, st.m, o));
    const float c = centre(st.m);
#pragma unroll
    for (int i = 0; i < EPL; ++i) {
        const float t = max_nan((v[i] - c) * kLog2e, LP_FLOOR), e = ex2(t);
        st.s += e;
        st.u += e * t;
    }
#pragma unroll
    for (int o = L / 2; o; o >>= 1) {
        st.s += __shfl_xor_sync(0xffffffffu, st.s, o);
        st.u += __shfl_xor_sync(0xffffffffu, st.u, o);
    }
    const RowResult r = finish(st);
    if (live && lane == 0) store_row(a, row, r, target);
    if (a.top == 0) return;
    // a.top rounds: the largest code left, of equal ones the lowest index (an entry that is not there or is
    // taken has code 0 and index -1)
    unsigned code[EPL];
#pragma unroll
    for (int i = 0; i < EPL; ++i) code[i] = code_of(v[i]);
    unsigned gone = 0;
    for (int k = 0; k < a.top; ++k) {
        unsigned best = 0, at = 0xffffffffu;
#pragma unroll
        for (int i = EPL - 1; i >= 0; --i)
            if (lane + i * L < vocab && !(gone >> i & 1u) && code[i] >= best) {
                best = code[i];
                at = unsigned(lane + i * L);
            }
        if (L == 32) {
            const unsigned top = __reduce_max_sync(0xffffffffu, best);
            at = __reduce_min_sync(0xffffffffu, best == top ? at : 0xffffffffu);
            best = top;
        } else {
#pragma unroll
            for (int o = L / 2; o; o >>= 1) {
                const unsigned c2 = __shfl_xor_sync(0xffffffffu, best, o), a2 = __shfl_xor_sync(0xffffffffu, at, o);
                if (c2 > best || (c2 == best && a2 < at)) {
                    best = c2;
                    at = a2;
                }
            }
        }
        if (int(at % L) == lane) gone |= 1u << (at / L);
        if (live && lane == 0) store_top(a, row, k, (static_cast<unsigned long long>(best) << 32) | (0xffffffffu - at), r);
    }
}

// ---- longer rows: a team of WARPS warps per row: one warp, a CTA (eight), or a cluster of up to eight CTAs
template <int WARPS> struct ForwardShared {
    static constexpr int LIST = WARPS == 1 ? 256 : 512;         // candidate entries
    static constexpr int SHARES = WARPS == 1 ? 192 : 256;       // tiles that are read again
    float              tile_max[LP_TILES][32 * WARPS];
    Softmax            part[WARPS];
    Softmax            total;                      // of this CTA: read by the cluster's first
    unsigned           warp_code[WARPS];
    int                shares[SHARES];             // thread + threads * tile
    int                nshares, nlist;
    unsigned long long list[LIST];
    unsigned long long top[GAR_MAX_TOP];           // this CTA's best, in order (0: none): read by the cluster's first
    unsigned long long warp_key[WARPS];
};
// Threads of a CTA whose teams have WARPS warps: eight teams of a warp, or one team.
__host__ __device__ constexpr int cta_threads(int warps) { return warps == 1 ? 256 : 32 * warps; }
template <int WARPS> __device__ __forceinline__ void team_sync() {
    if (WARPS == 1) __syncwarp();
    else __syncthreads();
}

// A row as 16-byte slots: slot i holds elements [i E - head, (i + 1) E - head); the row's first and
// last slot may be incomplete and are then read by element ("edge" entries).
template <typename T> struct RowView {
    const T* x;              // the row
    const T* base;           // x - head: 16-byte aligned
    int      head;           // elements of slot 0 before the row
    int64_t  vocab;
    int64_t  first, last;    // this CTA's complete slots [first, last)
    int64_t  lead, tail;     // edge entries of this CTA: [0, lead) and [vocab - tail, vocab)
};
template <typename T>
__device__ __forceinline__ RowView<T> view_row(const T* x, int64_t vocab, unsigned rank, unsigned parts) {
    constexpr int E = Elem<T>::PER16;
    RowView<T> v;
    v.x = x;
    v.vocab = vocab;
    v.head = int((reinterpret_cast<uintptr_t>(x) & 15) / sizeof(T));
    v.base = x - v.head;
    const int64_t whole_first = v.head ? 1 : 0, whole_last = (vocab + v.head) / E;       // complete slots
    const int64_t n = whole_last > whole_first ? whole_last - whole_first : 0;
    v.first = parts == 1 ? whole_first : whole_first + n * rank / parts;
    v.last = parts == 1 ? whole_first + n : whole_first + n * (rank + 1) / parts;
    v.lead = v.tail = 0;
    if (rank == 0 && v.head) v.lead = E - v.head;
    if (rank == parts - 1) v.tail = (vocab + v.head) - whole_last * E;
    return v;
}
// the edge entry of a thread (at most 14 of them), or -1
template <typename T>
__device__ __forceinline__ int64_t edge_entry(const RowView<T>& v, int tid) {
    if (tid < v.lead) return tid;
    if (tid >= 16 && tid - 16 < v.tail) return v.vocab - v.tail + (tid - 16);
    return -1;
}

template <int WARPS>
__device__ __forceinline__ void offer(ForwardShared<WARPS>& sh, float x, int64_t idx) {
    const int at = atomicAdd(&sh.nlist, 1);
    if (at < sh.LIST) sh.list[at] = key_of(x, unsigned(idx));
}

// best key below `bound` in a thread's share
template <typename T, int THREADS>
__device__ unsigned long long best_below(const RowView<T>& v, int tid, unsigned long long bound) {
    constexpr int E = Elem<T>::PER16;
    unsigned long long best = 0;
    for (int64_t slot = v.first + tid; slot < v.last; slot += THREADS) {
        float f[E];
        widen16B(*reinterpret_cast<const uint4*>(v.base + slot * E), f, static_cast<const T*>(nullptr));
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const unsigned long long key = key_of(f[e], unsigned(slot * E + e - v.head));
            if (key < bound && key > best) best = key;
        }
    }
    const int64_t j = edge_entry(v, tid);
    if (j >= 0) {
        const unsigned long long key = key_of(load_one(v.x, j), unsigned(j));
        if (key < bound && key > best) best = key;
    }
    return best;
}

// The CTA's `top` best entries of its part of the row into sh.top, in order (zeros beyond what there
// is).  `first`, `second`: the thread's two largest tile maxima; tiles of (1 << shift) slots.
template <typename T, int WARPS>
__device__ void find_top(ForwardShared<WARPS>& sh, const RowView<T>& v, float first, float second, int top, int shift) {
    constexpr int E = Elem<T>::PER16, THREADS = 32 * WARPS;
    const int tid = threadIdx.x % THREADS, warp = tid / 32, lane = tid % 32;
    if (tid == 0) sh.nshares = sh.nlist = 0;
    if (tid < GAR_MAX_TOP) sh.top[tid] = 0;
    // warps whose 32 threads all have a slot (a team of one warp may have idle lanes: they count as 0); a share without a number or with masked entries only counts as 0
    const int64_t slots = v.last - v.first;
    const int full = WARPS == 1 ? 1 : slots >= THREADS ? WARPS : int(slots / 32);
    const unsigned own = first == -CUDART_INF_F ? 0u : code_of(first);
    unsigned least = 0xffffffffu;
    if (warp < full) {
        unsigned rest = own, again = second == -CUDART_INF_F ? 0u : code_of(second);
        for (int j = (top + full - 1) / full; j > 0; --j) {
            least = __reduce_max_sync(0xffffffffu, rest);
            if (lane == __ffs(__ballot_sync(0xffffffffu, rest == least)) - 1) {
                rest = again;
                again = 0u;
            }
        }
    }
    if (lane == 0) sh.warp_code[warp] = least;
    team_sync<WARPS>();
    unsigned low = full ? sh.warp_code[0] : 0u;
    for (int w = 1; w < full; ++w) low = min(low, sh.warp_code[w]);
    if (own >= low) {
        const int tiles = int((slots - tid + THREADS - 1) / THREADS + (1 << shift) - 1) >> shift;      // of this thread
        for (int i = 0; i < tiles; ++i)
            if (low == 0u || code_of(sh.tile_max[i][tid]) >= low) {
                const int at = atomicAdd(&sh.nshares, 1);
                if (at < sh.SHARES) sh.shares[at] = tid + THREADS * i;
            }
    }
    const int64_t edge = edge_entry(v, tid);
    if (edge >= 0) {
        const float f = load_one(v.x, edge);
        if (code_of(f) >= low) offer(sh, f, edge);
    }
    team_sync<WARPS>();
    const int nshares = sh.nshares;
    if (nshares <= sh.SHARES) {
        for (int i = tid; i < nshares << shift; i += THREADS) {
            const int share = sh.shares[i >> shift];
            const int64_t slot = v.first + share % THREADS + int64_t(((share / THREADS) << shift) + (i & ((1 << shift) - 1))) * THREADS;
            if (slot < v.last) {
                float f[E];
                widen16B(*reinterpret_cast<const uint4*>(v.base + slot * E), f, static_cast<const T*>(nullptr));
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if (code_of(f[e]) >= low) offer(sh, f[e], slot * E + e - v.head);
            }
        }
    }
    team_sync<WARPS>();
    const int nlist = sh.nlist;
    if (nshares <= sh.SHARES && nlist <= sh.LIST) {
        for (int i = tid; i < nlist; i += THREADS) {
            const unsigned long long key = sh.list[i];
            int rank = 0;
            for (int j = 0; j < nlist; ++j) rank += sh.list[j] > key;
            if (rank < top) sh.top[rank] = key;
        }
        team_sync<WARPS>();
        return;
    }
    // too many equal values for the list: one by one
    unsigned long long cur = best_below<T, THREADS>(v, tid, ~0ull);
    for (int k = 0; k < top; ++k) {
        unsigned long long best = cur;
#pragma unroll
        for (int o = 16; o; o >>= 1) {
            const unsigned long long other = shfl_xor64(best, o);
            if (other > best) best = other;
        }
        if (lane == 0) sh.warp_key[warp] = best;
        team_sync<WARPS>();
        best = sh.warp_key[0];
#pragma unroll
        for (int w = 1; w < WARPS; ++w) best = sh.warp_key[w] > best ? sh.warp_key[w] : best;
        if (tid == 0) sh.top[k] = best;
        if (best != 0 && cur == best) cur = best_below<T, THREADS>(v, tid, best);
        team_sync<WARPS>();
    }
}

// Largest value (NaN entries do not count) of a tile, and whether a masked entry (-inf, or so low that the
// exponent may overflow) may be in it.
__device__ __forceinline__ void tile_range(const uint4 (&raw)[LP_UNROLL], float& top, bool& masked, const float*) {
    top = -CUDART_INF_F;
#pragma unroll
    for (int i = 0; i < LP_UNROLL; ++i)
        top = fmaxf(fmaxf(fmaxf(top, __uint_as_float(raw[i].x)), fmaxf(__uint_as_float(raw[i].y), __uint_as_float(raw[i].z))), __uint_as_float(raw[i].w));
    masked = true;                       // four entries per 16 bytes: keeping the exponents in range costs less than asking
}
template <typename H2, typename From, typename Max, typename Min>
__device__ __forceinline__ void tile_range_16(const uint4 (&raw)[LP_UNROLL], float& top, bool& masked, From from, Max mx, Min mn) {
    H2 hi = from(raw[0].x), lo = hi;
#pragma unroll
    for (int i = 0; i < LP_UNROLL; ++i) {
        const unsigned w[4] = {raw[i].x, raw[i].y, raw[i].z, raw[i].w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            hi = mx(hi, from(w[j]));
            lo = mn(lo, from(w[j]));
        }
    }
    top = fmaxf(fmaxf(-CUDART_INF_F, float(hi.x)), float(hi.y));     // a tile of NaN: -inf
    masked = !(float(lo.x) >= -LP_HUGE && float(lo.y) >= -LP_HUGE);
}
__device__ __forceinline__ void tile_range(const uint4 (&raw)[LP_UNROLL], float& top, bool& masked, const __nv_bfloat16*) {
    tile_range_16<__nv_bfloat162>(raw, top, masked, [](unsigned w) { return *reinterpret_cast<const __nv_bfloat162*>(&w); },
                                  [](__nv_bfloat162 a, __nv_bfloat162 b) { return __hmax2(a, b); },
                                  [](__nv_bfloat162 a, __nv_bfloat162 b) { return __hmin2(a, b); });
}
__device__ __forceinline__ void tile_range(const uint4 (&raw)[LP_UNROLL], float& top, bool& masked, const __half*) {
    tile_range_16<__half2>(raw, top, masked, [](unsigned w) { return *reinterpret_cast<const __half2*>(&w); },
                           [](__half2 a, __half2 b) { return __hmax2(a, b); }, [](__half2 a, __half2 b) { return __hmin2(a, b); });
}
// 16 bytes of -inf
template <typename T> __device__ __forceinline__ uint4 nothing() {
    const unsigned w = sizeof(T) == 4 ? 0xff800000u : std::is_same<T, __half>::value ? 0xfc00fc00u : 0xff80ff80u;
    return make_uint4(w, w, w, w);
}
template <typename T, bool MASKED>
__device__ __forceinline__ void add_tile(const uint4 (&raw)[LP_UNROLL], float centre_at, f32x2& s2, f32x2& u2) {
    constexpr int E = Elem<T>::PER16;
    const f32x2 nc = pack2(-centre_at, -centre_at), scale = pack2(kLog2e, kLog2e);
#pragma unroll
    for (int i = 0; i < LP_UNROLL; ++i) {
        float f[E];
        widen16B(raw[i], f, static_cast<const T*>(nullptr));
#pragma unroll
        for (int e = 0; e < E; e += 2) {
            f32x2 t = mul2(add2(pack2(f[e], f[e + 1]), nc), scale);
            float t0, t1;
            unpack2(t, t0, t1);
            if (MASKED) {
                t0 = max_nan(t0, LP_FLOOR);
                t1 = max_nan(t1, LP_FLOOR);
                t = pack2(t0, t1);
            }
            const f32x2 ex = pack2(ex2(t0), ex2(t1));
            s2 = add2(s2, ex);
            u2 = fma2(ex, t, u2);
        }
    }
}

// Per entry one exponential (of 16 a cycle and SM; the memory's rate asks for 11.6 entries of 16 bits) and
// five instructions.  The next turn's loads are in flight while a turn is worked on.  Measured: 4096 x
// 131072 bf16 200 us without alternatives, 233 to 244 with 20 (1.07 GB: 5.4 and 4.5 TB/s, copy peak 6.5;
// under the profiler issue slots 67 % busy, exponential unit 60 %), fp32 170 us for
// 2048 x 131072 (6.3 TB/s).  The alternatives cost the row's end: two barriers, a second read of some 40
// tiles, 10 % more DRAM traffic; it hides behind the other rows of the SM, which is why a row gets a warp up
// to 16384 entries (16384 x 8192 bf16: 55 us, by CTAs of eight warps 123) and four warps beyond while the
// rows last (4096 x 32768, 20 alternatives: 76 us, by eight warps 99).  4 x 32768: 8.5 us, latency.
template <typename T, int WARPS>
__global__ void __launch_bounds__(cta_threads(WARPS), 1024 / cta_threads(WARPS)) logprobs_kernel(const ForwardArgs a, int parts) {
    constexpr int E = Elem<T>::PER16, THREADS = 32 * WARPS, TEAMS = cta_threads(WARPS) / THREADS;
    __shared__ __align__(16) ForwardShared<WARPS> shared[TEAMS];
    ForwardShared<WARPS>& sh = shared[threadIdx.x / THREADS];
    const int tid = threadIdx.x % THREADS, warp = tid / 32, lane = tid % 32;
    if (WARPS == 1) parts = 1;                                   // a cluster has CTAs for teams
    const unsigned rank = WARPS == 1 ? 0u : blockIdx.x % unsigned(parts);
    const int64_t row = int64_t(WARPS == 1 ? blockIdx.x : blockIdx.x / unsigned(parts)) * TEAMS + threadIdx.x / THREADS;
    if (TEAMS > 1 && row >= a.rows) return;
    const RowView<T> v = view_row(static_cast<const T*>(a.logits) + row * a.ld, a.vocab, rank, unsigned(parts));

    // turns of LP_UNROLL slots per thread; a tile is (1 << turn_shift) turns
    const int turns = int((v.last - v.first + LP_UNROLL * THREADS - 1) / (LP_UNROLL * THREADS));
    int turn_shift = 0;
    while ((turns + (1 << turn_shift) - 1) >> turn_shift > LP_TILES) ++turn_shift;

    Softmax st{-CUDART_INF_F, 0.f, 0.f};
    f32x2 s2 = pack2(0.f, 0.f), u2 = pack2(0.f, 0.f);
    const T* at = v.base + (v.first + tid) * E;
    int64_t left = v.last - v.first - tid;                       // slots from `at` on, at a stride of THREADS
    auto fetch = [&](uint4 (&raw)[LP_UNROLL]) {
#pragma unroll
        for (int i = 0; i < LP_UNROLL; ++i)
            raw[i] = left > i * THREADS ? load_stream(at + i * THREADS * E) : nothing<T>();
        at += LP_UNROLL * THREADS * E;
        left -= LP_UNROLL * THREADS;
    };
    uint4 raw[LP_UNROLL], next[LP_UNROLL];
    float tile_top = -CUDART_INF_F, first = -CUDART_INF_F, second = -CUDART_INF_F;
    if (turns > 0) fetch(raw);
    const Target target = tid == 0 && rank == 0 ? read_target<T>(a, row) : Target{-1, 0.f};      // behind the first loads
    for (int turn = 0; turn < turns; ++turn) {
        if (turn + 1 < turns) fetch(next);
        float top;
        bool masked;
        tile_range(raw, top, masked, static_cast<const T*>(nullptr));
        if (a.top) {
            tile_top = (turn & ((1 << turn_shift) - 1)) ? fmaxf(tile_top, top) : top;
            sh.tile_max[turn >> turn_shift][tid] = tile_top;
            if (turn + 1 == turns || ((turn + 1) & ((1 << turn_shift) - 1)) == 0) {      // the tile's last turn
                second = fmaxf(second, fminf(first, tile_top));
                first = fmaxf(first, tile_top);
            }
        }
        if (top > st.m) {
            float s0, s1, u0, u1;
            unpack2(s2, s0, s1);
            unpack2(u2, u0, u1);
            st.s = s0 + s1;
            st.u = u0 + u1;
            raise(st, top);
            s2 = pack2(st.s, 0.f);
            u2 = pack2(st.u, 0.f);
        }
        if (masked || st.m > LP_HUGE) add_tile<T, true>(raw, centre(st.m), s2, u2);
        else add_tile<T, false>(raw, centre(st.m), s2, u2);
#pragma unroll
        for (int i = 0; i < LP_UNROLL; ++i) raw[i] = next[i];
    }
    {
        float s0, s1, u0, u1;
        unpack2(s2, s0, s1);
        unpack2(u2, u0, u1);
        st.s = s0 + s1;
        st.u = u0 + u1;
    }
    const int64_t edge = edge_entry(v, tid);
    if (edge >= 0) add_one(st, load_one(v.x, edge));
    // the warp's sums about the warp's maximum
    const float warp_m = value_of(__reduce_max_sync(0xffffffffu, code_of(st.m)));
    if (warp_m > st.m) raise(st, warp_m);
#pragma unroll
    for (int o = 16; o; o >>= 1) {
        st.s += __shfl_xor_sync(0xffffffffu, st.s, o);
        st.u += __shfl_xor_sync(0xffffffffu, st.u, o);
    }
    Softmax total = st;
    if (WARPS > 1) {
        if (lane == 0) sh.part[warp] = st;
        __syncthreads();
        total = Softmax{sh.part[0].m, 0.f, 0.f};
#pragma unroll
        for (int w = 1; w < WARPS; ++w) total.m = fmaxf(total.m, sh.part[w].m);
#pragma unroll
        for (int w = 0; w < WARPS; ++w) {
            Softmax b = sh.part[w];
            if (total.m > b.m) raise(b, total.m);
            total.s += b.s;
            total.u += b.u;
        }
        __syncthreads();
    }
    if (a.top) find_top<T, WARPS>(sh, v, first, second, a.top, turn_shift + 2);

    if (WARPS == 1 || parts == 1) {
        const RowResult r = finish(total);
        if (tid == 0) store_row(a, row, r, target);
        if (tid < a.top) store_top(a, row, tid, sh.top[tid], r);
        return;
    }
    // the cluster's first CTA joins the others' results
    cg::cluster_group cluster = cg::this_cluster();
    if (tid == 0) sh.total = total;
    cluster.sync();
    if (rank == 0) {
        for (int p = 1; p < parts; ++p) join(total, cluster.map_shared_rank(&sh, p)->total);
        const RowResult r = finish(total);
        if (tid == 0) store_row(a, row, r, target);
        if (a.top) {
            const int n = parts * a.top;               // at most 256 = one entry per thread
            unsigned long long key = 0;
            if (tid < n) key = cluster.map_shared_rank(&sh, tid / a.top)->top[tid % a.top];
            if (tid < n) sh.list[tid] = key;
            __syncthreads();
            if (key != 0) {
                int at = 0;
                for (int j = 0; j < n; ++j) at += sh.list[j] > key;
                if (at < a.top) store_top(a, row, at, key, r);
            }
        }
    }
    cluster.sync();
}

template <typename T>
cudaError_t forward(const ForwardArgs& a, int sm_count, cudaStream_t stream) {
    if (a.vocab <= 256) {
        const int lanes = a.vocab <= 16 ? 4 : a.vocab <= 64 ? 8 : 32;
        const int64_t blocks = (a.rows + LP_THREADS / lanes - 1) / (LP_THREADS / lanes);
        if (blocks > 0x7fffffff) return cudaErrorInvalidConfiguration;
        const unsigned n = unsigned(blocks);
        if (a.vocab <= 16) logprobs_small_kernel<T, 4, 4><<<n, LP_THREADS, 0, stream>>>(a);
        else if (a.vocab <= 64) logprobs_small_kernel<T, 8, 8><<<n, LP_THREADS, 0, stream>>>(a);
        else if (a.vocab <= 128) logprobs_small_kernel<T, 32, 4><<<n, LP_THREADS, 0, stream>>>(a);
        else logprobs_small_kernel<T, 32, 8><<<n, LP_THREADS, 0, stream>>>(a);
        return cudaGetLastError();
    }
    // A warp per row has no barriers: it is the faster team as long as the rows give every SM eight of
    // them, or the row is no more than a turn.
    if (a.vocab <= 1024 || (a.vocab <= LP_WARP_VOCAB && a.rows >= 8 * int64_t(sm_count))) {
        const int64_t blocks = (a.rows + LP_WARPS - 1) / LP_WARPS;
        if (blocks > 0x7fffffff) return cudaErrorInvalidConfiguration;
        logprobs_kernel<T, 1><<<unsigned(blocks), LP_THREADS, 0, stream>>>(a, 1);
        return cudaGetLastError();
    }
    // Long rows, enough of them: half a CTA's worth of threads per row, so that twice as many rows are in
    // work on an SM and the end of one (reductions, the top alternatives) hides behind the others
    if (a.rows >= 4 * int64_t(sm_count)) {
        if (a.rows > 0x7fffffff) return cudaErrorInvalidConfiguration;
        logprobs_kernel<T, 4><<<unsigned(a.rows), cta_threads(4), 0, stream>>>(a, 1);
        return cudaGetLastError();
    }
    // A row is split over a cluster while that still leaves SMs without work and every CTA a tile
    // of its own (LP_UNROLL slots per thread).
    int parts = 1;
    const int64_t slots = a.vocab / Elem<T>::PER16;
    while (parts < LP_MAX_CLUSTER && a.rows * parts < 2 * sm_count && slots >= int64_t(2 * parts) * LP_THREADS * LP_UNROLL) parts *= 2;
    if (a.rows * parts > 0x7fffffff) return cudaErrorInvalidConfiguration;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(unsigned(a.rows * parts));
    cfg.blockDim = dim3(LP_THREADS);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = unsigned(parts);
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = parts > 1 ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, logprobs_kernel<T, LP_WARPS>, a, parts);
}

// ---- gradient --------------------------------------------------------------------------------
struct BackwardArgs {
    const void*    logits;
    void*          dlogits;
    int64_t        rows, vocab, ld, ldo;
    const int64_t* targets;
    const float *  lse, *lse_lo, *entropy;
    const int64_t* top_index;
    const float *  grad_logprobs, *grad_entropy, *grad_top;
    int            top;
};

// A row's constants, and this lane's special entry (one of the top alternatives).
struct RowGrad {
    float   lse, lse_lo, entropy, c, sum;  // sum = a + sum_i b_i
    bool    empty;
    float   a;                             // gradient of the target's log probability
    int64_t target;                        // -1: none
    int64_t at;                            // lane i: top_index[i], -1 beyond the list
    float   b;                             // its gradient
};
// What grad_at reads, from the sums: dx = p (c' log p + sum'), c' = -c, sum' = -(sum + c H).  An empty row
// (lse = -inf) gets lse = +inf, so that every p is 0, and c' = sum' = 0: the gradients at its results, which are
// infinite themselves, may be infinities or NaN.
__device__ __forceinline__ void settle(RowGrad& r) {
    r.empty = r.lse == -CUDART_INF_F;
    if (r.empty) r.lse = CUDART_INF_F;
    r.sum = r.empty ? 0.f : -fmaf(r.c, r.entropy, r.sum);
    r.c = r.empty ? 0.f : -r.c;
}
// All 32 lanes of a warp call.
__device__ __forceinline__ RowGrad row_grad(const BackwardArgs& g, int64_t row, int lane) {
    RowGrad r;
    r.lse = g.lse[row];
    r.lse_lo = g.lse_lo ? g.lse_lo[row] : 0.f;
    r.c = g.grad_entropy ? g.grad_entropy[row] : 0.f;
    r.entropy = g.grad_entropy ? g.entropy[row] : 0.f;
    r.target = -1;
    r.a = 0.f;
    if (g.grad_logprobs) {
        const int64_t t = g.targets[row];
        if (t >= g.vocab) r.a = CUDART_NAN_F;
        else if (t >= 0) {
            r.target = t;
            r.a = g.grad_logprobs[row];
        }
    }
    r.at = -1;
    r.b = 0.f;
    if (lane < g.top) {
        r.at = g.top_index[row * g.top + lane];
        r.b = g.grad_top[row * g.top + lane];
        if (r.at < 0 || r.at >= g.vocab) {
            r.at = -1;
            r.b = CUDART_NAN_F;
        }
    }
    r.sum = r.b;
    if (g.top) {
#pragma unroll
        for (int o = 16; o; o >>= 1) r.sum += __shfl_xor_sync(0xffffffffu, r.sum, o);
    }
    r.sum += r.a;
    settle(r);
    return r;
}
__device__ __forceinline__ float grad_at(const RowGrad& r, float x) {
    const float lp = max_nan((x - r.lse) - r.lse_lo, LP_FLOOR);
    return ex2(lp * kLog2e) * fmaf(r.c, lp, r.sum);
}
// the same for two entries
__device__ __forceinline__ void grad_at2(const RowGrad& r, float& x0, float& x1) {
    float a, b;
    unpack2(add2(add2(pack2(x0, x1), pack2(-r.lse, -r.lse)), pack2(-r.lse_lo, -r.lse_lo)), a, b);
    a = max_nan(a, LP_FLOOR);
    b = max_nan(b, LP_FLOOR);
    const f32x2 lp = pack2(a, b);
    unpack2(mul2(lp, pack2(kLog2e, kLog2e)), a, b);
    unpack2(mul2(pack2(ex2(a), ex2(b)), fma2(pack2(r.c, r.c), lp, pack2(r.sum, r.sum))), x0, x1);
}

// The special entries of a row: their logits, read before anything is written (dx may be x), and their
// gradients, written over the plain ones.  A place that occurs more than once gets every term, in one
// order, whoever writes it.  Entries outside [lo, hi) are somebody else's.
struct Special {
    float x, x_target;
};
template <typename T>
__device__ __forceinline__ Special read_special(const RowGrad& r, const T* x, int64_t lo, int64_t hi) {
    Special s{0.f, 0.f};
    if (r.at >= lo && r.at < hi) s.x = load_one(x, r.at);
    if (r.target >= lo && r.target < hi) s.x_target = load_one(x, r.target);
    return s;
}
template <typename T>
__device__ __forceinline__ void write_special(const BackwardArgs& g, const RowGrad& r, const Special& s, T* dx, int64_t lo, int64_t hi, int lane) {
    const bool here = (r.at >= lo && r.at < hi) || (r.target >= lo && r.target < hi);
    if (r.empty || !__any_sync(0xffffffffu, here)) return;
    float own = grad_at(r, s.x), target = grad_at(r, s.x_target);
    for (int j = 0; j < g.top; ++j) {
        const int64_t at = __shfl_sync(0xffffffffu, r.at, j);
        const float b = __shfl_sync(0xffffffffu, r.b, j);
        if (at == r.at) own += b;
        if (at == r.target) target += b;
    }
    if (r.at == r.target) own += r.a;
    target += r.a;
    if (r.at >= 0 && r.at >= lo && r.at < hi) dx[r.at] = Elem<T>::narrow(own);
    if (lane == 0 && r.target >= 0 && r.target >= lo && r.target < hi) dx[r.target] = Elem<T>::narrow(target);
}

// Rows of up to 64 entries: eight lanes per row, plain accesses; every lane adds the special terms to
// its own entries.
template <typename T>
__global__ void __launch_bounds__(LP_THREADS) logprobs_backward_small_kernel(const BackwardArgs g) {
    constexpr int L = 8, EPL = 8;
    const int lane = threadIdx.x % L;
    const int64_t row = (int64_t(blockIdx.x) * LP_THREADS + threadIdx.x) / L;
    if (row >= g.rows) return;
    const T* x = static_cast<const T*>(g.logits) + row * g.ld;
    T* dx = static_cast<T*>(g.dlogits) + row * g.ldo;
    const int vocab = int(g.vocab);
    float v[EPL], extra[EPL];
#pragma unroll
    for (int i = 0; i < EPL; ++i) {
        v[i] = lane + i * L < vocab ? load_one(x, lane + i * L) : 0.f;
        extra[i] = 0.f;
    }
    RowGrad r;
    r.lse = g.lse[row];
    r.lse_lo = g.lse_lo ? g.lse_lo[row] : 0.f;
    r.c = g.grad_entropy ? g.grad_entropy[row] : 0.f;
    r.entropy = g.grad_entropy ? g.entropy[row] : 0.f;
    r.sum = 0.f;
    auto term = [&](int64_t at, float value) {
        r.sum += at < vocab ? value : CUDART_NAN_F;
#pragma unroll
        for (int i = 0; i < EPL; ++i)
            if (at == lane + i * L) extra[i] += value;
    };
    for (int j = 0; j < g.top; ++j) {
        const int64_t at = g.top_index[row * g.top + j];
        term(at < 0 ? vocab : at, g.grad_top[row * g.top + j]);
    }
    if (g.grad_logprobs && g.targets[row] >= 0) term(g.targets[row], g.grad_logprobs[row]);
    settle(r);
#pragma unroll
    for (int i = 0; i < EPL; ++i)
        if (lane + i * L < vocab) dx[lane + i * L] = Elem<T>::narrow(r.empty ? 0.f : grad_at(r, v[i]) + extra[i]);
}

// Longer rows: a team of WARPS warps takes LPB_SLOTS 16-byte slots per thread of a row at a time: a
// CTA one such chunk, a warp (a row of its own) one after the other.  Bound by memory: 4096 x 131072 bf16
// 325 us = 6.6 TB/s, 2048 x 32000 43 us, 300 x 50001 fp32 (odd rows) 22.6 us = 5.3 TB/s.
constexpr int LPB_SLOTS = 4;

template <typename T, int WARPS>
__global__ void __launch_bounds__(LP_THREADS) logprobs_backward_kernel(const BackwardArgs g, unsigned chunks) {
    constexpr int E = Elem<T>::PER16, THREADS = 32 * WARPS, TEAMS = LP_THREADS / THREADS;
    const int tid = threadIdx.x % THREADS, lane = threadIdx.x % 32;
    const int64_t row = TEAMS > 1 ? int64_t(blockIdx.x) * TEAMS + threadIdx.x / THREADS : blockIdx.x / chunks;
    if (TEAMS > 1 && row >= g.rows) return;
    const unsigned first = TEAMS > 1 ? 0u : blockIdx.x % chunks, last = TEAMS > 1 ? chunks : first + 1u;
    const T* x = static_cast<const T*>(g.logits) + row * g.ld;
    T* dx = static_cast<T*>(g.dlogits) + row * g.ldo;
    const int head = int((reinterpret_cast<uintptr_t>(x) & 15) / sizeof(T));
    const bool together = ((reinterpret_cast<uintptr_t>(x) ^ reinterpret_cast<uintptr_t>(dx)) & 15) == 0;
    // slot i: elements [i E - head, (i + 1) E - head)
    const int64_t lo = int64_t(first) * (THREADS * LPB_SLOTS * E) - head;
    const int64_t hi = min(int64_t(last) * (THREADS * LPB_SLOTS * E) - head, g.vocab);

    uint4 raw[LPB_SLOTS];
    bool whole[LPB_SLOTS];
    auto fetch = [&](unsigned chunk) {
        const int64_t slot0 = int64_t(chunk) * (THREADS * LPB_SLOTS) + tid;
#pragma unroll
        for (int i = 0; i < LPB_SLOTS; ++i) {
            const int64_t j = (slot0 + i * THREADS) * E - head;
            whole[i] = together && j >= 0 && j + E <= g.vocab;
            if (whole[i]) raw[i] = load_stream(x + j);
        }
    };
    fetch(first);
    const RowGrad r = row_grad(g, row, lane);
    const bool last_word = threadIdx.x % THREADS < 32;            // the warp that writes the special entries
    const Special s = last_word ? read_special<T>(r, x, lo, hi) : Special{0.f, 0.f};
    if (WARPS == 1) __syncwarp();
    else __syncthreads();                 // read before anything is written: dx may be x
    for (unsigned chunk = first; chunk < last; ++chunk) {
        if (chunk > first) fetch(chunk);
        const int64_t slot0 = int64_t(chunk) * (THREADS * LPB_SLOTS) + tid;
#pragma unroll
        for (int i = 0; i < LPB_SLOTS; ++i) {
            const int64_t j = (slot0 + i * THREADS) * E - head;
            if (whole[i]) {
                float f[E];
                widen16B(raw[i], f, static_cast<const T*>(nullptr));
#pragma unroll
                for (int e = 0; e < E; e += 2) grad_at2(r, f[e], f[e + 1]);
                store_stream(dx + j, narrow16B(f, static_cast<const T*>(nullptr)));
            } else if (j < g.vocab) {
                for (int e = 0; e < E; ++e)
                    if (j + e >= 0 && j + e < g.vocab) dx[j + e] = Elem<T>::narrow(grad_at(r, load_one(x, j + e)));
            }
        }
    }
    if (WARPS == 1) __syncwarp();
    else __syncthreads();
    if (last_word) write_special<T>(g, r, s, dx, lo, hi, lane);
}

template <typename T>
cudaError_t backward(const BackwardArgs& g, int sm_count, cudaStream_t stream) {
    if (g.vocab <= 64) {
        const int64_t blocks = (g.rows + LP_THREADS / 8 - 1) / (LP_THREADS / 8);
        if (blocks > 0x7fffffff) return cudaErrorInvalidConfiguration;
        logprobs_backward_small_kernel<T><<<unsigned(blocks), LP_THREADS, 0, stream>>>(g);
        return cudaGetLastError();
    }
    constexpr int E = Elem<T>::PER16;
    const int64_t slots = (g.vocab + E - 1) / E + 1;                          // with the largest head
    if (g.vocab <= 1024 || (g.vocab <= LP_WARP_VOCAB / 4 && g.rows >= 8 * int64_t(sm_count))) {
        const int64_t blocks = (g.rows + LP_WARPS - 1) / LP_WARPS;
        if (blocks > 0x7fffffff) return cudaErrorInvalidConfiguration;
        logprobs_backward_kernel<T, 1><<<unsigned(blocks), LP_THREADS, 0, stream>>>(g, unsigned((slots + 32 * LPB_SLOTS - 1) / (32 * LPB_SLOTS)));
        return cudaGetLastError();
    }
    const int64_t chunks = (slots + LP_THREADS * LPB_SLOTS - 1) / (LP_THREADS * LPB_SLOTS);
    if (g.rows * chunks > 0x7fffffff) return cudaErrorInvalidConfiguration;
    logprobs_backward_kernel<T, LP_WARPS><<<unsigned(g.rows * chunks), LP_THREADS, 0, stream>>>(g, unsigned(chunks));
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_logprobs(const gar_logprobs_params_t& p, int64_t ld, int sm_count) {
    const ForwardArgs a{p.logits, p.rows, p.vocab, ld, p.targets, p.logprobs, p.entropy, p.lse, p.lse_lo, p.top_logprobs, p.top_index, p.top};
    cudaStream_t s = static_cast<cudaStream_t>(p.stream);
    if (p.dtype == GAR_F32) return forward<float>(a, sm_count, s);
    if (p.dtype == GAR_BF16) return forward<__nv_bfloat16>(a, sm_count, s);
    return forward<__half>(a, sm_count, s);
}

cudaError_t launch_logprobs_backward(const gar_logprobs_grad_params_t& p, int64_t ld, int64_t ldo, int sm_count) {
    const BackwardArgs g{p.logits, p.dlogits, p.rows, p.vocab, ld, ldo, p.targets, p.lse, p.lse_lo, p.entropy, p.top_index,
                         p.grad_logprobs, p.grad_entropy, p.grad_top, p.top};
    cudaStream_t s = static_cast<cudaStream_t>(p.stream);
    if (p.dtype == GAR_F32) return backward<float>(g, sm_count, s);
    if (p.dtype == GAR_BF16) return backward<__nv_bfloat16>(g, sm_count, s);
    return backward<__half>(g, sm_count, s);
}

}  // namespace worker
}  // namespace gar
