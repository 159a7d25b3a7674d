// Embedding lookup with scaling and its gradient (ifvs_embed, ifvs_embed_grad).
//
// Lookup: out[t] = scale table[ids[t]], a copy of rows: bound by memory (163847
// tokens x 960 of bfloat16 66 us, 6.0 TB/s).  Rows that do not begin on 16 bytes go
// element by element (ids drawn evenly: 960 columns 86 us, 998 or 999 293).
//
// Gradient: d_table[v] = scale (sum of d_out[t] over the tokens with id v).  The
// tokens are sorted by id (stable, so a row's sum runs over its tokens in
// order), and the sorted order is cut into parts of equal length, whatever ids
// they hold: a few ids have most of the tokens.  A warp adds the rows of its
// part for a slice of the columns, run by run: a run inside the part goes to its
// row, the two that may reach beyond it are left as float32 partial sums, which
// k_embed_join adds in the order of the parts.  Rows that no token names are
// found by a search in the sorted ids and set to zero.  Every row is written
// once, no order depends on timing.  Measured: 17408 tokens x 128 of float32 into
// 3760 rows 25 us, 14 of them the sort; 400009 x 384 of bfloat16 into 50021 rows 102
// us, 60 for the rows' sums and 35 for the sort's six launches.  Rows that do not
// begin on 16 bytes are loaded element by element (ids drawn evenly: 384 columns 96
// us, 385 or 386 204).
#include "layers.cuh"
#include "scan_common.cuh"

namespace ifvs {

namespace {

inline bool vectors(const EmbedArgs& a, const void* p, const void* q) {
    return a.D * elem_bytes(a.type) % 16 == 0 && ((uintptr_t)p | (uintptr_t)q) % 16 == 0;
}

// out[t] = scale table[ids[t]].  A thread copies kEmbedPieces pieces of a row, 256
// pieces apart: that is `rows` rows and `pieces` pieces further, so that one
// division per thread places all (a division per piece kept the SMs' issue slots
// 68 % busy).
constexpr int kEmbedPieces = 4;

template <class T, int N>
__global__ void __launch_bounds__(256)
k_embed(const T* __restrict__ table, EmbedArgs a, int per_row, int rows, int pieces, T* __restrict__ out) {
    using F = typename Pack<T, N>::F;
    const int64_t first = (int64_t)blockIdx.x * (256 * kEmbedPieces) + threadIdx.x;
    int64_t t = first <= 0xFFFFFFFFll ? (int64_t)((uint32_t)first / (uint32_t)per_row) : first / per_row;
    int col = (int)(first - t * per_row);
    Pack<T, N> v[kEmbedPieces];
    int id[kEmbedPieces];
#pragma unroll
    for (int i = 0; i < kEmbedPieces; ++i) {
        id[i] = -1;
        if (t < a.T) {
            id[i] = __ldg(a.ids + t);
            if (id[i] < -1 || id[i] >= a.V) {
                if (col == 0) a.waits.err[kErrId] = 1;
                id[i] = -1;
            }
            if (id[i] >= 0) v[i].load(table + (int64_t)id[i] * a.D + col * N);
        }
        col += pieces;
        t += rows;
        if (col >= per_row) {
            col -= per_row;
            ++t;
        }
    }
    const int64_t n = a.T * per_row;
#pragma unroll
    for (int i = 0; i < kEmbedPieces; ++i) {
        const int64_t at = first + i * 256;
        if (at >= n) continue;
#pragma unroll
        for (int j = 0; j < Pack<T, N>::kF; ++j) v[i].set(j, id[i] >= 0 ? mul_(both<F>(a.scale), v[i].get(j)) : both<F>(0.f));
        v[i].store_stream(out + at * N);     // the table's rows stay in L2
    }
}

// ---- sort by id ------------------------------------------------------------------
// Least significant digit first, digits of equal width of at most 9 bits (tables
// below 2^18 rows in two passes; a pass costs three launches); the key of a
// token without a row is V.
constexpr int kDigitBits = 9, kBins = 1 << kDigitBits;
constexpr int kSortRounds = 8;                       // keys per lane, at most

struct SortPlan {
    int passes, bits;
    __host__ __device__ uint32_t digit(uint32_t key, int pass) const {
        return (key >> (pass * bits)) & ((1u << bits) - 1u);
    }
};
SortPlan sort_plan(int64_t V) {
    int bits = 1;
    while ((1ll << bits) <= V) ++bits;               // keys 0..V
    const int passes = (bits + kDigitBits - 1) / kDigitBits;
    return {passes, (bits + passes - 1) / passes};
}

struct Pairs {
    uint32_t *key, *pos;
};

__device__ __forceinline__ uint32_t key_of(const EmbedArgs& a, int64_t i) {
    const int id = __ldg(a.ids + i);
    if (id >= 0 && id < a.V) return (uint32_t)id;
    if (id != -1) a.waits.err[kErrId] = 1;
    return (uint32_t)a.V;
}

// The keys of a warp's R x 32 places from `first` (absent beyond n),
// with their rank among the warp's earlier keys of the same digit; counts in
// hist [kBins].  Lanes of equal digits find each other by a ballot per bit.
template <int R>
struct WarpKeys {
    uint32_t key[R], pos[R];
    uint16_t rank[R];
};
template <int R>
__device__ __forceinline__ void load_keys(WarpKeys<R>& k, const EmbedArgs& a, Pairs in, int64_t first, int64_t left, int lane) {
#pragma unroll
    for (int j = 0; j < R; ++j) {
        const int64_t i = first + j * 32 + lane;
        k.key[j] = k.pos[j] = 0;
        if (j * 32 + lane >= left) continue;
        if (in.key) {
            // written by this kernel's cluster or an earlier kernel: not through the read-only path
            k.key[j] = __ldcg(in.key + i);
            k.pos[j] = __ldcg(in.pos + i);
        } else {
            k.key[j] = key_of(a, i);
            k.pos[j] = (uint32_t)i;
        }
    }
}
template <int R>
__device__ __forceinline__ void rank_keys(WarpKeys<R>& k, const SortPlan& plan, int pass, int64_t left, int lane,
                                          uint32_t* hist) {
    uint32_t same[R];
#pragma unroll
    for (int j = 0; j < R; ++j) same[j] = __ballot_sync(0xFFFFFFFFu, j * 32 + lane < left);
    // bit by bit over all rounds: the ballots of a bit do not wait for each other
    for (int b = 0; b < plan.bits; ++b) {
        const int at = pass * plan.bits + b;
#pragma unroll
        for (int j = 0; j < R; ++j) {
            const bool bit = k.key[j] >> at & 1u;
            const uint32_t set = __ballot_sync(0xFFFFFFFFu, bit);
            same[j] &= bit ? set : ~set;
        }
    }
#pragma unroll
    for (int j = 0; j < R; ++j) {
        if (j * 32 >= left) break;
        const bool in = j * 32 + lane < left;
        const uint32_t d = plan.digit(k.key[j], pass);
        const uint32_t before = in ? hist[d] : 0u;
        k.rank[j] = (uint16_t)(before + __popc(same[j] & ((1u << lane) - 1u)));
        __syncwarp();
        if (in && (same[j] >> lane) == 1u) hist[d] = before + __popc(same[j]);    // the last of its digit
        __syncwarp();
    }
}

// Exclusive sums of kBins values, two neighbours for each of the first kBins / 2
// threads (the whole block calls): the sum before the first of the two.
constexpr int kScanThreads = kBins / 2;
__device__ __forceinline__ uint32_t scan_bins(uint32_t v0, uint32_t v1, uint32_t* warp_sums) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint32_t v = v0 + v1;
    uint32_t s = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint32_t u = __shfl_up_sync(0xFFFFFFFFu, s, o);
        if (lane >= o) s += u;
    }
    if (lane == 31 && warp < kScanThreads / 32) warp_sums[warp] = s;
    __syncthreads();
    uint32_t base = 0;
    for (int i = 0; i < min(warp, kScanThreads / 32); ++i) base += warp_sums[i];
    return base + s - v;
}

// In each bin of a block's W histograms the counts of the warps before, from
// `start`; returns the bin's total
template <int W>
__device__ __forceinline__ uint32_t stack_counts(uint32_t (*hist)[kBins], int bin, uint32_t start) {
    uint32_t n[W], sum = start;
#pragma unroll
    for (int w = 0; w < W; ++w) n[w] = hist[w][bin];
#pragma unroll
    for (int w = 0; w < W; ++w) {
        hist[w][bin] = sum;
        sum += n[w];
    }
    return sum - start;
}

// Up to 65536 tokens: one cluster sorts them in one launch.  Each of its CTAs owns
// a segment of the order, in shared memory between the passes; the digits'
// counts and the pairs pass through distributed shared memory (through global
// memory a pass of 17408 tokens took 7 us instead of 5).
constexpr int kClusterMax = 8;
constexpr int64_t cluster_tokens(int warps) { return (int64_t)kClusterMax * warps * 32 * kSortRounds; }   // 65536 at 32

__device__ __forceinline__ uint32_t cluster_size() {
    uint32_t v;
    asm("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(v));
    return v;
}
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// two neighbours at this CTA's address p, from another CTA
__device__ __forceinline__ uint2 load_of(const uint32_t* p, uint32_t cta) {
    uint32_t at;
    uint2 v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(cta));
    asm volatile("ld.shared::cluster.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(at) : "memory");
    return v;
}
__device__ __forceinline__ void store_to(uint32_t at, uint32_t cta, uint32_t a, uint32_t b) {
    uint32_t q;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(q) : "r"(at), "r"(cta));
    asm volatile("st.shared::cluster.v2.u32 [%0], {%1, %2};" ::"r"(q), "r"(a), "r"(b) : "memory");
}

// W warps a CTA, 16 where they suffice.  magic: 2^32 / segment, rounded up.
constexpr size_t cluster_smem(int warps, int rounds) {
    return sizeof(uint32_t) * warps * kBins + 2 * sizeof(uint2) * warps * 32 * rounds;
}
template <int W>
__global__ void __launch_bounds__(W * 32, 1)
k_sort_cluster(EmbedArgs a, SortPlan plan, Pairs out, int rounds, uint32_t magic) {
    extern __shared__ __align__(16) uint32_t sort_smem[];
    uint32_t(*hist)[kBins] = reinterpret_cast<uint32_t(*)[kBins]>(sort_smem);      // [W]
    const int segment = W * 32 * rounds;
    uint2* held = reinterpret_cast<uint2*>(sort_smem + W * kBins);                  // [2][segment] keys and positions
    __shared__ __align__(8) uint32_t total[kBins];
    __shared__ uint32_t base[kBins], warp_sums[kScanThreads / 32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, bins = 1 << plan.bits;
    const uint32_t cta = blockIdx.x, ctas = cluster_size();
    const int64_t first = (int64_t)cta * segment + warp * 32 * rounds;
    const int64_t left = min(a.T - first, (int64_t)32 * rounds);
    start_dependents();
    for (int pass = 0; pass < plan.passes; ++pass) {
        for (int i = lane; i < bins; i += 32) hist[warp][i] = 0;
        WarpKeys<kSortRounds> k;
        if (pass == 0) {
            load_keys(k, a, Pairs{nullptr, nullptr}, first, left, lane);
        } else {
#pragma unroll
            for (int j = 0; j < kSortRounds; ++j) {
                uint2 v = make_uint2(0, 0);
                if (j * 32 + lane < left) v = held[(pass & 1) * segment + (warp * rounds + j) * 32 + lane];
                k.key[j] = v.x;
                k.pos[j] = v.y;
            }
        }
        __syncwarp();
        rank_keys(k, plan, pass, left, lane, hist[warp]);
        __syncthreads();
        for (int d = threadIdx.x; d < bins; d += W * 32) total[d] = stack_counts<W>(hist, d, 0);
        cluster_sync();
        uint32_t all[2] = {0, 0}, before[2] = {0, 0};
        const int d0 = threadIdx.x * 2;
        if (d0 < bins) {
            uint2 n[kClusterMax];        // all loads are issued before the first is used
#pragma unroll
            for (uint32_t c = 0; c < kClusterMax; ++c) n[c] = load_of(&total[d0], min(c, ctas - 1u));
#pragma unroll
            for (uint32_t c = 0; c < kClusterMax; ++c) {
                before[0] += c < cta ? n[c].x : 0u;
                before[1] += c < cta ? n[c].y : 0u;
                all[0] += c < ctas ? n[c].x : 0u;
                all[1] += c < ctas ? n[c].y : 0u;
            }
        }
        const uint32_t start = scan_bins(all[0], all[1], warp_sums);
        if (d0 < bins) {
            base[d0] = start + before[0];
            base[d0 + 1] = start + all[0] + before[1];
        }
        __syncthreads();
        const bool last = pass + 1 == plan.passes;
        const uint32_t to = (uint32_t)__cvta_generic_to_shared(held) + ((pass + 1) & 1) * segment * 8u;
#pragma unroll
        for (int j = 0; j < kSortRounds; ++j)
            if (j * 32 + lane < left) {
                const uint32_t g = plan.digit(k.key[j], pass), at = base[g] + hist[warp][g] + k.rank[j];
                if (last) {
                    out.key[at] = k.key[j];
                    out.pos[at] = k.pos[j];
                } else {
                    const uint32_t c = __umulhi(at, magic);
                    store_to(to + (at - c * segment) * 8u, c, k.key[j], k.pos[j]);
                }
            }
        cluster_sync();      // the pairs are there, and every CTA has read the totals
    }
}

// More tokens: per pass the digits' counts of every tile of kTileTokens, their
// sums over the tiles before, and the scatter.
constexpr int kTileWarps = 8;
constexpr int kTileRounds = 4;
constexpr int kTileTokens = kTileWarps * 32 * kTileRounds;   // 1024: more CTAs, each a chain of latencies

// counts [kBins][tiles]
__global__ void __launch_bounds__(kTileWarps * 32)
k_sort_count(EmbedArgs a, SortPlan plan, int pass, Pairs in, uint32_t* __restrict__ counts, int tiles) {
    __shared__ uint32_t hist[kBins];
    for (int d = threadIdx.x; d < kBins; d += kTileWarps * 32) hist[d] = 0;
    __syncthreads();
    start_dependents();
    if (pass > 0) wait_before();
    const int64_t first = (int64_t)blockIdx.x * kTileTokens;
#pragma unroll
    for (int j = 0; j < kTileRounds; ++j) {
        const int64_t i = first + j * (kTileWarps * 32) + threadIdx.x;
        if (i < a.T) atomicAdd(&hist[plan.digit(in.key ? __ldcg(in.key + i) : key_of(a, i), pass)], 1u);
    }
    __syncthreads();
    for (int d = threadIdx.x; d < 1 << plan.bits; d += kTileWarps * 32) counts[(int64_t)d * tiles + blockIdx.x] = hist[d];
}

// a warp per digit: exclusive sums over the tiles, and the digit's total
__global__ void __launch_bounds__(256)
k_sort_scan(uint32_t* __restrict__ counts, int bins, int tiles, uint32_t* __restrict__ totals) {
    start_dependents();
    wait_before();
    const int lane = threadIdx.x & 31, d = blockIdx.x * 8 + (threadIdx.x >> 5);
    if (d >= bins) return;
    uint32_t* c = counts + (int64_t)d * tiles;
    uint32_t sum = 0;
    for (int i0 = 0; i0 < tiles; i0 += 32) {
        const int i = i0 + lane;
        const uint32_t v = i < tiles ? __ldcg(c + i) : 0u;
        uint32_t s = v;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t u = __shfl_up_sync(0xFFFFFFFFu, s, o);
            if (lane >= o) s += u;
        }
        if (i < tiles) c[i] = sum + s - v;
        sum += __shfl_sync(0xFFFFFFFFu, s, 31);
    }
    if (lane == 0) totals[d] = sum;
}

__global__ void __launch_bounds__(kTileWarps * 32)
k_sort_scatter(EmbedArgs a, SortPlan plan, int pass, Pairs in, Pairs out, const uint32_t* __restrict__ counts,
               int tiles, const uint32_t* __restrict__ totals) {
    __shared__ uint32_t hist[kTileWarps][kBins], warp_sums[kScanThreads / 32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, bins = 1 << plan.bits;
    start_dependents();
    for (int i = lane; i < bins; i += 32) hist[warp][i] = 0;
    const int64_t first = (int64_t)blockIdx.x * kTileTokens + warp * (32 * kTileRounds);
    wait_before();
    const int d0 = threadIdx.x * 2;
    uint32_t all[2] = {0, 0}, before[2] = {0, 0};
    if (d0 < bins)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            all[j] = __ldcg(totals + d0 + j);
            before[j] = __ldcg(counts + (int64_t)(d0 + j) * tiles + blockIdx.x);
        }
    WarpKeys<kTileRounds> k;
    const int64_t left = a.T - first;
    load_keys(k, a, in, first, left, lane);
    __syncwarp();
    rank_keys(k, plan, pass, left, lane, hist[warp]);
    const uint32_t start = scan_bins(all[0], all[1], warp_sums);     // with a barrier: every warp has ranked
    if (d0 < bins) {
        stack_counts<kTileWarps>(hist, d0, start + before[0]);
        stack_counts<kTileWarps>(hist, d0 + 1, start + all[0] + before[1]);
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kTileRounds; ++j)
        if (j * 32 + lane < left) {
            const uint32_t at = hist[warp][plan.digit(k.key[j], pass)] + k.rank[j];
            out.key[at] = k.key[j];
            out.pos[at] = k.pos[j];
        }
}

// ---- sums by id --------------------------------------------------------------------
struct SumPlan {
    int part;            // tokens per part (a multiple of 32)
    int64_t parts;
    int slices, width;   // of the columns, columns per slice
    int64_t sum_warps;   // parts x slices
    int64_t zero_warps;  // of 32 rows of the table
};

// Clears the rows that no token names: a lane looks for its row of the 32 from
// v0 in the sorted ids, the warp clears.
template <class T, int N>
__device__ __forceinline__ void clear_absent(const EmbedArgs& a, Pairs sorted, int64_t v0, T* __restrict__ d_table) {
    const int lane = threadIdx.x & 31;
    const int64_t v = v0 + lane;
    bool absent = false;
    if (v < a.V) {
        int64_t lo = 0, hi = a.T;                    // the first place with a key >= v
        while (lo < hi) {
            const int64_t m = (lo + hi) >> 1;
            if (__ldcg(sorted.key + m) < (uint32_t)v)
                lo = m + 1;
            else
                hi = m;
        }
        absent = lo == a.T || __ldcg(sorted.key + lo) != (uint32_t)v;
    }
    uint32_t rows = __ballot_sync(0xFFFFFFFFu, absent);
    Pack<T, N> zero;
#pragma unroll
    for (int j = 0; j < Pack<T, N>::kF; ++j) zero.set(j, both<typename Pack<T, N>::F>(0.f));
    for (; rows; rows &= rows - 1u) {
        T* row = d_table + (v0 + __ffs(rows) - 1) * a.D;
        for (int c = lane * N; c < a.D; c += 32 * N) zero.store(row + c);
    }
}

// One warp's sums over its part: NV accesses of N columns from `col`, 32 N apart,
// below `limit`.
// Partial sums [parts][2][D]: of the run that reaches into the part from before
// (0) and of the one that begins in it and goes on (1).
constexpr uint32_t kNoKey = 0xFFFFFFFFu;

template <class T, int N, int NV>
struct RunSums {
    using F = typename Pack<T, N>::F;
    static constexpr int kF = Pack<T, N>::kF;
    F sum[NV][kF];
    int64_t part;
    uint32_t run = kNoKey, last;        // the run's key; the key before the next token
    bool head = false;
    int col, limit;

    __device__ __forceinline__ void start(const EmbedArgs& a, Pairs sorted, int64_t part_, int64_t begin, int col_, int limit_) {
        part = part_;
        col = col_;
        limit = limit_;
        last = begin > 0 ? __ldcg(sorted.key + begin - 1) : kNoKey;
    }
    __device__ __forceinline__ void flush(const EmbedArgs& a, bool goes_on, float* partial, T* d_table) {
        if (run == kNoKey) return;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = col + i * 32 * N;
            if (c >= limit) continue;
            if (head || goes_on) {
                float* to = partial + (part * 2 + (head ? 0 : 1)) * a.D + c;
#pragma unroll
                for (int j = 0; j < kF; ++j) *reinterpret_cast<F*>(to + j * (N / kF)) = sum[i][j];
            } else {
                Pack<T, N> v;
#pragma unroll
                for (int j = 0; j < kF; ++j) v.set(j, mul_(both<F>(a.scale), sum[i][j]));
                v.store(d_table + (int64_t)run * a.D + c);
            }
        }
    }
    // Of 32 tokens with these keys (sorted; kNoKey beyond the part): which begin a
    // run of this part (bit per token), and how many have a row.
    __device__ __forceinline__ uint32_t starts(const EmbedArgs& a, uint32_t key, bool first, int* rows) {
        const int lane = threadIdx.x & 31;
        uint32_t prev = __shfl_up_sync(0xFFFFFFFFu, key, 1);
        if (lane == 0) prev = first ? kNoKey : last;
        const uint32_t some = __ballot_sync(0xFFFFFFFFu, key < a.V);
        *rows = __popc(some);
        return __ballot_sync(0xFFFFFFFFu, key != prev) & some;
    }
    // the row of token i of the 32
    __device__ __forceinline__ void add(const EmbedArgs& a, uint32_t starts, uint32_t key, int i, bool first,
                                        const Pack<T, N> (&v)[NV], float* partial, T* d_table) {
        if (starts >> i & 1u) {
            flush(a, false, partial, d_table);
            run = __shfl_sync(0xFFFFFFFFu, key, i);
            head = first && i == 0 && last == run;
#pragma unroll
            for (int k = 0; k < NV; ++k)
#pragma unroll
                for (int j = 0; j < kF; ++j) sum[k][j] = v[k].get(j);
        } else {
#pragma unroll
            for (int k = 0; k < NV; ++k)
#pragma unroll
                for (int j = 0; j < kF; ++j) sum[k][j] = add_(sum[k][j], v[k].get(j));
        }
    }
};

// Rows on 16 bytes: a warp has 16 / NV rows (of its slice) on their way into each
// of two halves of its shared memory, a bulk copy per lane and row, while it adds
// those of the other.  Measured at 400009 rows of 768 bytes: loads into registers,
// 8 in flight a warp, 87 us; the same as a ring of 8, 179 us (a use waits for
// the loads after its own too).
constexpr int kSumWarps = 4;
constexpr int kSliceBytes = 512;         // per NV

template <class T, int NV>
__global__ void __launch_bounds__(kSumWarps * 32)
k_embed_sum_rows(const T* __restrict__ d_out, EmbedArgs a, SumPlan p, Pairs sorted, float* __restrict__ partial,
                 T* __restrict__ d_table) {
    constexpr int N = 16 / (int)sizeof(T), HALF = 16 / NV, GROUPS = 32 / HALF, ROW = kSliceBytes * NV;
    extern __shared__ __align__(16) uint8_t halves[];        // [kSumWarps][2][HALF][ROW]
    __shared__ __align__(8) uint64_t bars[kSumWarps][2];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t job = (int64_t)blockIdx.x * kSumWarps + warp;
    start_dependents();
    if (lane < 2) mbar_init((uint32_t)__cvta_generic_to_shared(&bars[warp][lane]), 1);
    fence_mbar_init();
    __syncwarp();
    wait_before();
    if (job >= p.sum_warps) {
        if (job - p.sum_warps < p.zero_warps) clear_absent<T, N>(a, sorted, (job - p.sum_warps) * 32, d_table);
        return;
    }
    const int64_t part = job / p.slices, begin = part * p.part, end = min(a.T, begin + p.part);
    const int c0 = (int)(job - part * p.slices) * p.width;
    RunSums<T, N, NV> r;
    r.start(a, sorted, part, begin, c0 + lane * N, min(a.D, c0 + p.width));
    const uint32_t bytes = (uint32_t)(r.limit - c0) * (uint32_t)sizeof(T);
    uint8_t* mine = halves + warp * (2 * HALF * ROW);
    const uint32_t mine_at = (uint32_t)__cvta_generic_to_shared(mine), bar = (uint32_t)__cvta_generic_to_shared(bars[warp]);
    const uint64_t once = policy_evict_first();
    auto keys_at = [&](int64_t b) { return b + lane < end ? __ldcg(sorted.key + b + lane) : kNoKey; };
    auto places_at = [&](int64_t b) { return b + lane < end ? __ldcg(sorted.pos + b + lane) : 0u; };
    // the rows of group g of the 32 tokens whose keys and places these are, to half g & 1
    auto fetch = [&](int g, uint32_t key, uint32_t pos) {
        const bool its = lane / HALF == g && key < a.V;
        const uint32_t rows = __popc(__ballot_sync(0xFFFFFFFFu, its)), to = bar + 8 * (g & 1);
        if (lane == 0) mbar_arrive_expect_tx(to, rows * bytes + a.waits.extra);
        __syncwarp();
        if (its) bulk_g2s(mine_at + lane % (2 * HALF) * ROW, d_out + (int64_t)pos * a.D + c0, bytes, to, once);
    };
    uint32_t key = keys_at(begin), pos = places_at(begin), next_key = keys_at(begin + 32), next_pos = places_at(begin + 32);
    fetch(0, key, pos);
    fetch(1, key, pos);
    uint32_t parity = 0;
    for (int64_t b = begin; b < end; b += 32) {
        int rows;
        const uint32_t starts = r.starts(a, key, b == begin, &rows);
#pragma unroll 1
        for (int g = 0; g < GROUPS; ++g) {
            // a wait that runs out is reported and ends the warp's work: no barrier is
            // armed again; the copies of this half and of the other, if it has been
            // armed, are waited for once more, bounded
            if (!mbar_wait_warp(bar + 8 * (g & 1), parity, a.waits.cycles)) {
                if (lane == 0) a.waits.err[kErrWait] = 1;
                mbar_wait_warp(bar + 8 * (g & 1), parity, a.waits.cycles);
                if (g + 1 < GROUPS || b + 32 < end) mbar_wait_warp(bar + 8 * (~g & 1), parity ^ ((uint32_t)g & 1u), a.waits.cycles);
                return;
            }
            parity ^= (uint32_t)g & 1u;
            auto row = [&](Pack<T, N>(&v)[NV], int i) {
#pragma unroll
                for (int k = 0; k < NV; ++k)
                    v[k].w = *reinterpret_cast<const uint4*>(mine + i % (2 * HALF) * ROW + (k * 32 + lane) * 16);
            };
#pragma unroll 1
            for (int i0 = g * HALF; i0 < min(rows, (g + 1) * HALF); i0 += 8) {
                if (i0 + 8 <= rows) {
                    Pack<T, N> v[8][NV];
#pragma unroll
                    for (int u = 0; u < 8; ++u) row(v[u], i0 + u);
#pragma unroll
                    for (int u = 0; u < 8; ++u) r.add(a, starts, key, i0 + u, b == begin, v[u], partial, d_table);
                } else {
#pragma unroll 1
                    for (int i = i0; i < rows; ++i) {
                        Pack<T, N> v[NV];
                        row(v, i);
                        r.add(a, starts, key, i, b == begin, v, partial, d_table);
                    }
                }
            }
            fence_proxy_async_smem();
            __syncwarp();
            if (g + 2 < GROUPS)
                fetch(g + 2, key, pos);
            else if (b + 32 < end)
                fetch(g + 2 - GROUPS, next_key, next_pos);
        }
        r.last = __shfl_sync(0xFFFFFFFFu, key, 31);
        key = next_key;
        pos = next_pos;
        next_key = keys_at(b + 64);
        next_pos = places_at(b + 64);
    }
    r.flush(a, end < a.T && __ldcg(sorted.key + end) == r.run, partial, d_table);
}

// Rows of any alignment: element loads into registers, kAhead rows at a time
template <class T>
__global__ void __launch_bounds__(256, 2)
k_embed_sum(const T* __restrict__ d_out, EmbedArgs a, SumPlan p, Pairs sorted, float* __restrict__ partial,
            T* __restrict__ d_table) {
    constexpr int NV = 8, kAhead = 4;
    const int lane = threadIdx.x & 31;
    const int64_t job = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
    start_dependents();
    wait_before();
    if (job >= p.sum_warps) {
        if (job - p.sum_warps < p.zero_warps) clear_absent<T, 1>(a, sorted, (job - p.sum_warps) * 32, d_table);
        return;
    }
    const int64_t part = job / p.slices, begin = part * p.part, end = min(a.T, begin + p.part);
    RunSums<T, 1, NV> r;
    r.start(a, sorted, part, begin, (int)(job - part * p.slices) * p.width + lane, a.D);
    for (int64_t b = begin; b < end; b += 32) {
        const bool in = b + lane < end;
        const uint32_t key = in ? __ldcg(sorted.key + b + lane) : kNoKey;
        const uint32_t pos = in ? __ldcg(sorted.pos + b + lane) : 0u;
        int rows;
        const uint32_t starts = r.starts(a, key, b == begin, &rows);
        for (int i0 = 0; i0 < rows; i0 += kAhead) {
            Pack<T, 1> v[kAhead][NV];
            // without conditions, so that all loads are issued before the first is
            // used: places without a row read another, columns beyond D the last
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const T* row = d_out + (int64_t)__shfl_sync(0xFFFFFFFFu, pos, i0 + u) * a.D;
#pragma unroll
                for (int i = 0; i < NV; ++i) v[u][i].load(row + min(r.col + i * 32, a.D - 1));
            }
#pragma unroll
            for (int u = 0; u < kAhead; ++u)
                if (i0 + u < rows) r.add(a, starts, key, i0 + u, b == begin, v[u], partial, d_table);
        }
        r.last = __shfl_sync(0xFFFFFFFFu, key, 31);
    }
    r.flush(a, end < a.T && __ldcg(sorted.key + end) == r.run, partial, d_table);
}

// Runs over several parts: a warp per part in which one begins (and 128 columns)
// adds its partial sums; the CTA together those of long runs.
constexpr int kWarpParts = 8;            // parts that a warp adds by itself (17408 tokens: 28 us; 31 with 32)

template <class T>
__global__ void __launch_bounds__(256)
k_embed_join(EmbedArgs a, SumPlan p, Pairs sorted, const float* __restrict__ partial, T* __restrict__ d_table) {
    __shared__ float part_sum[8][128];
    __shared__ uint32_t long_run[8];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c0 = blockIdx.y * 128;
    wait_before();
    float sum[4];
    auto add = [&](const float* from) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int c = c0 + j * 32 + lane;
            if (c < a.D) sum[j] += __ldcg(from + c);
        }
    };
    // the first partial sums of parts first, first + by, ... <= last
    auto add_parts = [&](int64_t first, int64_t last, int by) {
        for (int64_t r = first; r <= last; r += 8 * by) {
            float q[8][4];               // eight parts' loads are issued before the first is added
#pragma unroll
            for (int u = 0; u < 8; ++u)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    q[u][j] = 0.f;
                    if (r + u * by <= last && c0 + j * 32 + lane < a.D)
                        q[u][j] = __ldcg(partial + (r + u * by) * 2 * a.D + c0 + j * 32 + lane);
                }
#pragma unroll
            for (int u = 0; u < 8; ++u)
#pragma unroll
                for (int j = 0; j < 4; ++j) sum[j] += q[u][j];
        }
    };
    auto key_at = [&](int64_t i) { return __ldcg(sorted.key + i); };
    const int64_t part = (int64_t)blockIdx.x * 8 + warp;
    uint32_t its = kNoKey;               // the run that begins in this part and goes on
    if (part + 1 < p.parts) {            // parts but the last are whole
        const int64_t begin = part * p.part, end = begin + p.part;
        const uint32_t run = key_at(end - 1), next = key_at(end), first = key_at(begin), before = key_at(max(begin - 1, (int64_t)0));
        if (run < a.V && next == run && !(begin > 0 && first == run && before == run)) its = run;
    }
    // the parts after the next that begin with the run
    int more = 1;
    if (its != kNoKey) {
        const int64_t q = part + 2 + lane;
        more += __popc(__ballot_sync(0xFFFFFFFFu, q < p.parts && key_at(q * p.part) == its));
    }
    const bool alone = more <= kWarpParts;
    if (lane == 0) long_run[warp] = alone ? kNoKey : its;
    if (its != kNoKey && alone) {
#pragma unroll
        for (int j = 0; j < 4; ++j) sum[j] = 0.f;
        add(partial + (part * 2 + 1) * a.D);
        add_parts(part + 1, part + more, 1);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int c = c0 + j * 32 + lane;
            if (c < a.D) d_table[(int64_t)its * a.D + c] = from_f32<T>(a.scale * sum[j]);
        }
    }
    __syncthreads();
    for (int w = 0; w < 8; ++w) {
        const uint32_t run = long_run[w];
        if (run == kNoKey) continue;
        const int64_t k = (int64_t)blockIdx.x * 8 + w;
        int64_t many = 1;
        for (;;) {
            const int64_t q = k + 1 + many + threadIdx.x;
            const int n = __syncthreads_count(q < p.parts && key_at(q * p.part) == run);
            many += n;
            if (n < 256) break;
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) sum[j] = 0.f;
        if (warp == 0) add(partial + (k * 2 + 1) * a.D);
        add_parts(k + 1 + warp, k + many, 8);
#pragma unroll
        for (int j = 0; j < 4; ++j) part_sum[warp][j * 32 + lane] = sum[j];
        __syncthreads();
        const int c = c0 + threadIdx.x;
        if (threadIdx.x < 128 && c < a.D) {
            float all = 0.f;
            for (int v = 0; v < 8; ++v) all += part_sum[v][threadIdx.x];
            d_table[(int64_t)run * a.D + c] = from_f32<T>(a.scale * all);
        }
        __syncthreads();
    }
}

// Parts long enough that their partial sums are few against the rows, short
// enough that every SM has `warps` of them
SumPlan sum_plan(const EmbedArgs& a, int most_columns, int multiple, int warps) {
    SumPlan p;
    p.slices = (a.D + most_columns - 1) / most_columns;
    p.width = ((a.D + p.slices - 1) / p.slices + multiple - 1) / multiple * multiple;
    p.part = 32;
    while (p.part < 256 && a.T / (2 * p.part) * p.slices >= (int64_t)warps * a.num_sms) p.part *= 2;
    p.parts = (a.T + p.part - 1) / p.part;
    p.sum_warps = p.parts * p.slices;
    p.zero_warps = (a.V + 31) / 32;
    return p;
}

size_t padded(size_t n) { return (n + 255) / 256 * 256; }
int64_t sort_tiles(const EmbedArgs& a) { return (a.T + kTileTokens - 1) / kTileTokens; }

cudaError_t sort_by_id(const EmbedArgs& a, Pairs p0, Pairs p1, uint32_t* counts, cudaStream_t s, Pairs* sorted) {
    const SortPlan plan = sort_plan(a.V);
    *sorted = p0;
    auto in_cluster = [&](auto warps) {
        const auto kernel = k_sort_cluster<warps()>;
        // the work of a pass is in its ranks: spread over the cluster's SMs
        int ctas = 1;
        while (ctas < kClusterMax && (int64_t)ctas * warps() * 64 < a.T) ctas *= 2;
        const int rounds = (int)((a.T + ctas * warps() * 32 - 1) / (ctas * warps() * 32));
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3((unsigned)ctas);
        cfg.blockDim = dim3(warps() * 32);
        cfg.dynamicSmemBytes = cluster_smem(warps(), rounds);
        const cudaError_t e = allow_smem(kernel, cfg.dynamicSmemBytes);
        if (e != cudaSuccess) return e;
        cfg.stream = s;
        cudaLaunchAttribute attr[1];
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim = {(unsigned)ctas, 1u, 1u};
        cfg.attrs = attr;
        cfg.numAttrs = 1;
        const uint32_t magic = (uint32_t)((1ull << 32) / (unsigned)(warps() * 32 * rounds) + 1);
        const cudaError_t n = next_launch();
        return n != cudaSuccess ? n : cudaLaunchKernelEx(&cfg, kernel, a, plan, p0, rounds, magic);
    };
    if (a.T <= cluster_tokens(16)) return in_cluster(std::integral_constant<int, 16>());
    if (a.T <= cluster_tokens(32)) return in_cluster(std::integral_constant<int, 32>());
    *sorted = plan.passes & 1 ? p0 : p1;
    const int tiles = (int)sort_tiles(a);
    uint32_t* totals = counts + (int64_t)kBins * tiles;
    // No launch after one that failed: the scatter writes where the counts say.
    for (int pass = 0; pass < plan.passes; ++pass) {
        const Pairs in = pass == 0 ? Pairs{nullptr, nullptr} : (pass & 1 ? p0 : p1);
        const Pairs out = pass & 1 ? p1 : p0;
        cudaError_t e = launch_next(k_sort_count, dim3(tiles), dim3(kTileWarps * 32), 0, pass > 0, s, a, plan, pass, in, counts, tiles);
        if (e == cudaSuccess)
            e = launch_next(k_sort_scan, dim3((unsigned)(((1 << plan.bits) + 7) / 8)), dim3(256), 0, true, s, counts, 1 << plan.bits,
                            tiles, totals);
        if (e == cudaSuccess)
            e = launch_next(k_sort_scatter, dim3(tiles), dim3(kTileWarps * 32), 0, true, s, a, plan, pass, in, out,
                            (const uint32_t*)counts, tiles, (const uint32_t*)totals);
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

template <class T>
cudaError_t sum_by_id(const EmbedArgs& a, const void* d_out, Pairs sorted, float* partial, void* d_table, cudaStream_t s) {
    const bool rows = vectors(a, d_out, d_table), wide = a.D * sizeof(T) > kSliceBytes;
    constexpr int N = 16 / (int)sizeof(T);
    const SumPlan p = rows ? sum_plan(a, kSliceBytes * (wide ? 2 : 1) / (int)sizeof(T), N, 16) : sum_plan(a, 256, 256, 16);
    const int64_t warps = p.sum_warps + p.zero_warps;
    cudaError_t e;
    if (rows) {
        const size_t smem = (size_t)kSumWarps * 2 * 16 * kSliceBytes;
        const auto kernel = wide ? k_embed_sum_rows<T, 2> : k_embed_sum_rows<T, 1>;
        e = allow_smem(kernel, smem);
        if (e == cudaSuccess)
            e = launch_next(kernel, dim3((unsigned)((warps + kSumWarps - 1) / kSumWarps)), dim3(kSumWarps * 32), smem, true, s,
                              (const T*)d_out, a, p, sorted, partial, (T*)d_table);
    } else {
        e = launch_next(k_embed_sum<T>, dim3((unsigned)((warps + 7) / 8)), dim3(256), 0, true, s, (const T*)d_out, a, p, sorted,
                          partial, (T*)d_table);
    }
    if (e == cudaSuccess && p.parts > 1)
        e = launch_next(k_embed_join<T>, dim3((unsigned)((p.parts + 7) / 8), (unsigned)((a.D + 127) / 128)), dim3(256), 0, true, s,
                          a, p, sorted, (const float*)partial, (T*)d_table);
    return e;
}

}  // namespace

cudaError_t launch_embed(const EmbedArgs& a, const void* table, void* out, cudaStream_t s) {
    return with_type(a.type, [&](auto z) {
        using T = decltype(z);
        constexpr int N = 16 / (int)sizeof(T);
        const bool vec = vectors(a, table, out);
        const int per_row = a.D / (vec ? N : 1), rows = 256 / per_row, pieces = 256 % per_row;
        const int64_t n = a.T * per_row;
        const unsigned grid = (unsigned)((n + 256 * kEmbedPieces - 1) / (256 * kEmbedPieces));
        const cudaError_t e = next_launch();
        if (e != cudaSuccess) return e;
        if (vec)
            k_embed<T, N><<<grid, 256, 0, s>>>((const T*)table, a, per_row, rows, pieces, (T*)out);
        else
            k_embed<T, 1><<<grid, 256, 0, s>>>((const T*)table, a, per_row, rows, pieces, (T*)out);
        return cudaGetLastError();
    });
}

// two sets of pairs, the tiles' counts, the partial sums of the shortest parts
size_t embed_grad_bytes(const EmbedArgs& a) {
    return 4 * padded((size_t)a.T * 4) + padded((size_t)(sort_tiles(a) + 1) * kBins * 4) +
           (size_t)((a.T + 31) / 32) * 2 * a.D * 4;
}

cudaError_t launch_embed_grad(const EmbedArgs& a, const void* d_out, void* d_table, uint8_t* work, cudaStream_t s) {
    if (a.T == 0) return cudaMemsetAsync(d_table, 0, (size_t)a.V * a.D * elem_bytes(a.type), s);
    auto take = [&](size_t bytes) {
        uint8_t* p = work;
        work += padded(bytes);
        return (uint32_t*)p;
    };
    const size_t n = (size_t)a.T * 4;
    const Pairs p0{take(n), take(n)}, p1{take(n), take(n)};
    uint32_t* counts = take((size_t)(sort_tiles(a) + 1) * kBins * 4);
    float* partial = (float*)work;
    Pairs sorted;
    const cudaError_t e = sort_by_id(a, p0, p1, counts, s, &sorted);
    if (e != cudaSuccess) return e;
    return with_type(a.type, [&](auto z) {
        using T = decltype(z);
        return sum_by_id<T>(a, d_out, sorted, partial, d_table, s);
    });
}

}  // namespace ifvs
