// The norm after a block, its gate, the residual and the norm before the next
// block in one pass, and the gradients (ifvs_norm_join, ifvs_norm_join_grad).
//
//   u = y / rms(y), x' = rho x + gate_b w_post u, n = w_pre x' / rms(x')
//
// with g = dL/dx' (d_x_out plus what comes through n):
//   z = d_n w_pre, i = 1 / rms(x'), g = d_x_out + i (z - x' i^2 mean(z x'))
//   dx = rho g, du = gate_b w_post g, dy = (du - u mean(du u)) / rms(y)
//   S_b = sum over sequence b of g u, d_gate_b = w_post S_b,
//   d_w_post = sum of gate_b g u, d_w_pre = sum of d_n x' i over all tokens
//
// Both are bound by memory: two rows read and two written per token, four and
// two.  A team of 1 to 16 warps takes tokens that follow each other, through a ring
// of two places in shared memory that bulk copies fill ahead: each row is
// read once from memory, whatever the norms need of it, and a team's loads go on
// while it reduces.  A place holds the bytes of a few tokens (they follow each
// other in memory, so that rows need no alignment).  The sequence of a team's
// first token is searched, the others' follow, and the gradient keeps its sums
// over tokens in registers.  A sequence inside a team's tokens has its gate's
// gradient written at once; one that reaches beyond them leaves float32 partial
// sums that k_join_finish adds in order, as it does with the norms' weights.  No
// result depends on timing.  Measured: 163847 tokens x 960 of bfloat16 227 us,
// 5.6 TB/s; the gradient of 131101 x 1024 289 us, 5.6 TB/s.  Rows that do not begin
// on 16 bytes go by 8, 4 or 2: 100003 x 960, 964, 962 and 961 of bfloat16 141, 168,
// 237 and 463 us (more accesses a row; of two elements and of one, with spilled
// registers), the gradient of 100003 x 1024 and 1023 242 and 713.
#include "layers.cuh"
#include "places.h"
#include "scan_common.cuh"

namespace ifvs {

namespace {

// A team's reductions: warps of one team meet at a named barrier; two sets of
// slots, so that a set is not written again before all have read it.
struct Team {
    int warps, warp, id;        // warps of the team, this one's place, the team's number in the CTA
    float* slots;               // [2][all warps of the CTA][4], 16-byte aligned
    int turn, all;
    __device__ __forceinline__ void sync() const {
        if (warps == 1)
            __syncwarp();
        else
            asm volatile("barrier.cta.sync %0, %1;" ::"r"(1 + id), "r"(warps * 32) : "memory");
    }
    // both sums hold a barrier of the team
    __device__ __forceinline__ float sum(float v) {
        v = warp_sum(v);
        if (warps == 1) {
            __syncwarp();
            return v;
        }
        float* s = slots + (turn * all + id * warps) * 4;
        turn ^= 1;
        if ((threadIdx.x & 31) == 0) s[warp * 4] = v;
        sync();
        v = s[0];
        for (int w = 1; w < warps; ++w) v += s[w * 4];
        return v;
    }
    // three sums at once: lanes that differ in bit 0 share the first two, in bit 1
    // those and the third, so that three more exchanges end all of them
    __device__ __forceinline__ float3 sum3(float x, float y, float z) {
        const int lane = threadIdx.x & 31;
        const bool odd = lane & 1, third = lane & 2;
        float v = (odd ? y : x) + __shfl_xor_sync(0xFFFFFFFFu, odd ? x : y, 1);
        z += __shfl_xor_sync(0xFFFFFFFFu, z, 1);
        v = (third ? z : v) + __shfl_xor_sync(0xFFFFFFFFu, third ? v : z, 2);
#pragma unroll
        for (int o = 4; o < 32; o <<= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
        if (warps == 1)
            return make_float3(__shfl_sync(0xFFFFFFFFu, v, 0), __shfl_sync(0xFFFFFFFFu, v, 1), __shfl_sync(0xFFFFFFFFu, v, 2));
        float* s = slots + (turn * all + id * warps) * 4;
        turn ^= 1;
        if (lane < 4) s[warp * 4 + lane] = v;
        sync();
        float4 t = *reinterpret_cast<const float4*>(s);
        for (int w = 1; w < warps; ++w) {
            const float4 q = *reinterpret_cast<const float4*>(s + w * 4);
            t.x += q.x;
            t.y += q.y;
            t.z += q.z;
        }
        return make_float3(t.x, t.y, t.z);
    }
};

// The sequence of a team's next token, given that of an earlier one
struct Sequence {
    const int64_t* offsets;
    int B, T, b, end;           // end: offsets[b + 1], within 0..T whatever the offsets hold
    __device__ __forceinline__ int offset(int i) const { return (int)max((int64_t)0, min((int64_t)T, __ldg(offsets + i))); }
    __device__ __forceinline__ void start(int t) {
        b = (int)sequence_of(offsets, B, t);
        end = offsets ? offset(b + 1) : T;
    }
    // whether the sequence changes at token t
    __device__ __forceinline__ bool moved(int t) const { return t >= end && b + 1 < B; }
    __device__ __forceinline__ void move(int t) {
        ++b;
        end = offset(b + 1);
        if (t >= end && b + 1 < B) start(t);     // past empty sequences
    }
    __device__ __forceinline__ int begin() const { return offsets ? offset(b) : 0; }
};

constexpr int kStages = 2;               // places of a ring (1: no copies ahead)

extern __shared__ __align__(16) uint8_t join_smem[];

// tokens per place: about 1 KB of an array, at most 8
__host__ __device__ constexpr int place_tokens(int row_bytes) {
    return row_bytes >= 1024 ? 1 : (row_bytes <= 128 ? 8 : 1024 / row_bytes);
}

// After a wait that ran out: waits for the copies of place number `at`, which
// begins with token t, and of the places filled after it, once more and bounded
// together.  Out of line: inside the token loop it costs the gradient registers
// (131101 tokens x 1024: 297 us, 287 so).
template <int S>
__device__ __noinline__ void drain_places(uint32_t bars, int at, uint32_t parity, int t, int end, int per, long long cycles) {
    const long long t0 = clock64();
    for (int i = 0; i < S; ++i) {
        if (place_count(t, end, per, i))
            while (!mbar_try_wait(bars + 8u * at, parity) && clock64() - t0 < cycles) {
            }
        if (++at == S) {
            at = 0;
            parity ^= 1u;
        }
    }
}

// A team's ring: per place the rows of `per` tokens of A arrays (absent ones are
// null), from the 16-byte boundary before them to the one after.  Where that
// boundary lies outside the array, the row's bytes beside it are copied by
// plain loads: no byte outside an array is read.
template <class T, int N, int A, int S = kStages>
struct Rows {
    const T* p[A];
    uint32_t ring;              // S x A x stride bytes of join_smem
    uint32_t bars;              // address of S mbarriers and two 32-bit words: a wait for a place ran out, by turns
    Waits waits;
    int T_, D;                  // tokens of the arrays, their width
    int per, stride, place = 0;
    uint32_t parity = 0;
    uint32_t off[A];            // of the current token's rows in the ring

    static __host__ __device__ int stride_of(int D) {
        return (place_tokens(D * (int)sizeof(T)) * D * (int)sizeof(T) + 32 + 15) / 16 * 16;
    }
    __device__ __forceinline__ Rows(uint64_t* bars_, const JoinArgs& a, int team)
        : ring(team * S * A * stride_of(a.D)),
          bars((uint32_t)__cvta_generic_to_shared(bars_ + team * (S + 1))), waits(a.waits), T_((int)a.T), D(a.D),
          per(place_tokens(a.D * (int)sizeof(T))), stride(stride_of(a.D)) {}

    // tokens [t, t + n); the team's earlier reads of the place lie before a barrier of the team
    __device__ __forceinline__ void fill(const Team& team, int place_, int t, int n) const {
        if (team.warp != 0) return;
        const int lane = threadIdx.x & 31;
        const uint32_t to = (uint32_t)__cvta_generic_to_shared(join_smem) + ring + place_ * A * stride;
        if constexpr (N * sizeof(T) == 16) {        // rows begin and end on 16 bytes
            if (!elect_one()) return;
            const uint32_t len = n * D * (uint32_t)sizeof(T);
            const int64_t at = (int64_t)t * D;
            uint32_t arrays = 0;
#pragma unroll
            for (int k = 0; k < A; ++k) arrays += p[k] != nullptr;
            mbar_arrive_expect_tx(bars + 8u * place_, arrays * len + waits.extra);
            const uint64_t once = policy_evict_first();
#pragma unroll
            for (int k = 0; k < A; ++k)
                if (p[k]) bulk_g2s(to + k * stride, p[k] + at, len, bars + 8u * place_, once);
            return;
        }
        const int64_t o = (int64_t)t * D * (int)sizeof(T), rest = (int64_t)(T_ - t - n) * D * (int)sizeof(T);
        const uint32_t len = n * D * (uint32_t)sizeof(T), bar = bars + 8u * place_;
        // of array k: bytes of the copy before and after the rows, and whether they lie in the array
        auto copy = [&](int k, bool issue, uint64_t policy) -> uint32_t {
            const uint8_t* lo = reinterpret_cast<const uint8_t*>(p[k]) + o;
            const uint32_t before = (uint32_t)(reinterpret_cast<uintptr_t>(lo)) & 15u, after = (0u - before - len) & 15u;
            const uint32_t skip = before > o ? 16u : 0u, cut = after > rest ? 16u : 0u;
            const uint32_t all = before + len + after;
            const uint32_t bytes = all > skip + cut ? all - skip - cut : 0u;
            if (!issue) return bytes;
            if (skip | cut)
                for (uint32_t q = before + lane * 2; q < before + len; q += 64)
                    if (q < skip || q >= skip + bytes)
                        asm volatile("st.shared.u16 [%0], %1;" ::"r"(to + k * stride + q),
                                     "h"(__ldg(reinterpret_cast<const uint16_t*>(lo - before + q)))
                                     : "memory");
            if (bytes && elect_one())
                bulk_g2s(to + k * stride + skip, lo - before + skip, bytes, bar, policy);
            return bytes;
        };
        uint32_t all = 0;
#pragma unroll
        for (int k = 0; k < A; ++k)
            if (p[k]) all += copy(k, false, 0);
        if (elect_one()) mbar_arrive_expect_tx(bar, all + waits.extra);
        const uint64_t once = policy_evict_first();
#pragma unroll
        for (int k = 0; k < A; ++k)
            if (p[k]) copy(k, true, once);
    }
    // fills the ring for tokens [t, end)
    __device__ __forceinline__ void start(const Team& team, int t, int end) const {
        for (int i = 0; i < S; ++i)
            if (const int n = place_count(t, end, per, i)) fill(team, i, t + i * per, n);
        team.sync();
    }
    // the word of the current place: another one than that of the place before
    __device__ __forceinline__ uint32_t late() const {
        static_assert(S <= 2, "places take turns");
        return bars + 8u * S + 4u * (S == 2 ? (uint32_t)place : parity);
    }
    // The place's rows are there, for the whole team; t is its first token.  A wait
    // that runs out is reported and ends the team's work where it leaves the place.
    __device__ __forceinline__ void enter(const Team& team, int t) {
        const uint32_t bar = bars + 8u * place;
        if (!mbar_try_wait(bar, parity)) {
            const long long t0 = clock64();
            while (!mbar_try_wait(bar, parity))
                if (clock64() - t0 > waits.cycles) {
                    asm volatile("st.shared.u32 [%0], %1;" ::"r"(late()), "r"(1) : "memory");
                    waits.err[kErrWait] = 1;
                    break;
                }
        }
        if (S == 1) team.sync();         // plain loads of the fill just before
#pragma unroll
        for (int k = 0; k < A; ++k) {
            off[k] = ring + (uint32_t)((place * A + k) * stride);
            if (N * sizeof(T) != 16) off[k] += (uint32_t)reinterpret_cast<uintptr_t>(p[k] + (int64_t)t * D) & 15u;
        }
    }
    __device__ __forceinline__ Pack<T, N> get(int k, int col) const {
        Pack<T, N> v;
        v.w = *reinterpret_cast<const typename Pack<T, N>::Word*>(join_smem + off[k] + col * (uint32_t)sizeof(T));
        return v;
    }
    __device__ __forceinline__ void next() {
#pragma unroll
        for (int k = 0; k < A; ++k) off[k] += D * sizeof(T);
    }
    // This thread has read the place (before a barrier of the team, then leave).
    __device__ __forceinline__ void done() const { fence_proxy_async_smem(); }
    // The place that begins with token t is read by the whole team: fills it with
    // what comes S places later.  False, for the whole team alike, where a wait for
    // the place ran out: no barrier is armed again and no copy issued, and the team
    // goes to drain.  (Between the word's stores, in enter, and this look at it lies
    // a barrier of the team; before it can be stored again lie those of the next
    // place, which has the other word.)
    __device__ __forceinline__ bool leave(const Team& team, int t, int end) {
        uint32_t ran_out;
        asm volatile("ld.shared.u32 %0, [%1];" : "=r"(ran_out) : "r"(late()) : "memory");
        if (ran_out) return false;
        if (const int n = place_count(t, end, per, S)) fill(team, place, t + S * per, n);
        if (++place == S) {
            place = 0;
            parity ^= 1u;
        }
        return true;
    }
    __device__ __forceinline__ void drain(int t, int end) const {
        drain_places<S>(bars, place, parity, t, end, per, waits.cycles);
    }
};

// one thread: the barriers and words of `teams` teams
template <int S>
__device__ __forceinline__ void init_bars(uint64_t* bars, int teams) {
    for (int i = 0; i < teams; ++i, bars += S + 1) {
        for (int k = 0; k < S; ++k) mbar_init((uint32_t)__cvta_generic_to_shared(bars + k), 1);
        bars[S] = 0;
    }
    fence_mbar_init();
}

constexpr int kJoinThreads = 256;
// Columns a warp holds at most: 512 and three CTAs an SM, 1024 and two where 512 a
// warp need more warps than a CTA has.  512 against 1024, 100003 tokens of bfloat16:
// 960 columns 141 us and 144, 964 168 and 163, 962 237 and 281, 961 463 and 511;
// 50003 of float32: 960 133 and 146, 961 248 and 478.
constexpr int join_columns(int D) { return D <= kJoinThreads / 32 * 512 ? 512 : 1024; }
constexpr int join_ctas(int columns) { return columns > 512 ? 2 : 3; }       // per SM, by registers

// Shared memory of a kernel whose `teams` teams have rings of A rows a place
template <class T, int N, int A, int S = kStages>
size_t ring_bytes(int teams, int D) {
    return (size_t)teams * S * A * Rows<T, N, A, S>::stride_of(D);
}

// Without tokens: what the other kernels look at on their way
__global__ void __launch_bounds__(256) k_check_offsets(JoinArgs a) { check_offsets(a.given, a.B, a.T, a.waits.err); }

// Tokens [chunk team, chunk (team + 1)) of team number `team`
template <class T, int N, int NV>
__global__ void __launch_bounds__(kJoinThreads, join_ctas(32 * N * NV))
k_norm_join(JoinArgs a, int team_warps, int64_t chunk, const T* __restrict__ x, const T* __restrict__ y,
            T* __restrict__ xo, T* __restrict__ no) {
    __shared__ __align__(16) float slots[2 * kJoinThreads / 32 * 4];
    __shared__ __align__(8) uint64_t bars[kJoinThreads / 32 * (kStages + 1)];
    check_offsets(a.given, a.B, a.T, a.waits.err);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    Team team{team_warps, warp % team_warps, warp / team_warps, slots, 0, kJoinThreads / 32};
    const int64_t number = (int64_t)blockIdx.x * (kJoinThreads / 32 / team_warps) + team.id;
    const int t0 = (int)min(a.T, number * chunk), t1 = (int)min(a.T, number * chunk + chunk);
    const int col = (team.warp * 32 + lane) * N, step = team_warps * 32 * N;
    const float inv_d = 1.f / (float)a.D;
    const T* gate = (const T*)a.gate;
    const T* wp = (const T*)a.w_post;
    const T* wn = (const T*)a.w_pre;
    Rows<T, N, 2> rows(bars, a, team.id);
    rows.p[0] = x;
    rows.p[1] = y;
    if (threadIdx.x == 0) init_bars<kStages>(bars, kJoinThreads / 32);
    __syncthreads();
    if (t0 >= t1) return;
    rows.start(team, t0, t1);
    using F = typename Pack<T, N>::F;
    constexpr int kF = Pack<T, N>::kF;
    Sequence seq{a.offsets, (int)a.B, (int)a.T, 0, 0};
    F gw[NV][kF];                    // gate * w_post of the sequence
    auto load_gate = [&] {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = col + i * step;
            if (c >= a.D) continue;
            Pack<T, N> w, g;
            w.load(wp + c);
            if (gate) g.load(gate + (int64_t)seq.b * a.D + c);
#pragma unroll
            for (int j = 0; j < kF; ++j) gw[i][j] = gate ? mul_(g.get(j), w.get(j)) : w.get(j);
        }
    };
    if (gate) seq.start(t0);
    if (y) load_gate();
    const F rho = both<F>(a.rho);
    int first = t0;                                        // token of the place
    for (int t = t0; t < t1; ++t) {
        F v[NV][kF], q = both<F>(0.f);
        if (gate && seq.moved(t)) {
            seq.move(t);
            load_gate();
        }
        if (t == first) rows.enter(team, t);
        if (y) {
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int c = col + i * step;
                if (c >= a.D) continue;
                const Pack<T, N> r = rows.get(1, c);
#pragma unroll
                for (int j = 0; j < kF; ++j) {
                    v[i][j] = r.get(j);
                    q = fma_(v[i][j], v[i][j], q);
                }
            }
            const F iy = both<F>(rsqrtf(fmaf(team.sum(total(q)), inv_d, a.eps)));
            q = both<F>(0.f);
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int c = col + i * step;
                if (c >= a.D) continue;
                const Pack<T, N> r = rows.get(0, c);
                Pack<T, N> o;
#pragma unroll
                for (int j = 0; j < kF; ++j) {
                    v[i][j] = fma_(mul_(v[i][j], iy), gw[i][j], mul_(rho, r.get(j)));
                    q = fma_(v[i][j], v[i][j], q);
                    o.set(j, v[i][j]);
                }
                o.store(xo + (int64_t)t * a.D + c);
            }
        } else {
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int c = col + i * step;
                if (c >= a.D) continue;
                const Pack<T, N> r = rows.get(0, c);
#pragma unroll
                for (int j = 0; j < kF; ++j) {
                    v[i][j] = r.get(j);
                    q = fma_(v[i][j], v[i][j], q);
                }
            }
        }
        rows.next();
        const bool last = ends_place(t, first, t1, rows.per);
        if (last) rows.done();
        const float square = team.sum(total(q));           // with a barrier
        if (last) {
            if (!rows.leave(team, first, t1)) {
                rows.drain(first, t1);
                break;
            }
            first = t + 1;
        }
        if (!no) continue;
        const F ix = both<F>(rsqrtf(fmaf(square, inv_d, a.eps)));
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = col + i * step;
            if (c >= a.D) continue;
            Pack<T, N> w, o;
            w.load(wn + c);
#pragma unroll
            for (int j = 0; j < kF; ++j) o.set(j, mul_(w.get(j), mul_(v[i][j], ix)));
            o.store(no + (int64_t)t * a.D + c);
        }
    }
}

// ---- gradient ------------------------------------------------------------------
// 16 warps a CTA; two places of four rows each in shared memory at 512 columns of
// 16 bits a warp (more warps per token repeat its sums and waits: 410 us with
// 256 columns, 360 with 512, 131101 tokens x 1024), 256 of float32.  Float32
// rows beyond 4096 take 512 and a single place.
constexpr int kGradWarps = 16;
constexpr int kGradStages = kStages;     // 293 us, 331 with 3 (131101 tokens x 1024): what is left is L1 for the weights
constexpr int grad_columns(int type, int D) { return type == IFVS_T_F32 && D <= kGradWarps * 256 ? 256 : 512; }

struct GradPlan {
    int team_warps, ctas;
    int64_t teams, chunk;
    float* gates;        // [teams][2][D]: sums of the sequence that reaches into the team's tokens from
                         // before, and of the one that begins in them and goes on
    float* weights;      // [ctas][2][D]: d_w_post, d_w_pre
    int2* open;          // [teams]: the sequence that begins in the team's tokens and goes on (-1: none), its end
};

// ALL: y, d_x_out, d_n and the gate are there
template <class T, int N, int NV, int S, bool ALL>
__global__ void __launch_bounds__(kGradWarps * 32, 1) k_norm_join_grad(JoinArgs a, JoinGrads g, GradPlan p) {
    using Ring = Rows<T, N, 4, S>;
    constexpr int WARPS = kGradWarps;
    __shared__ __align__(16) float slots[2 * WARPS * 4];
    __shared__ __align__(8) uint64_t bars[WARPS * (S + 1)];
    check_offsets(a.given, a.B, a.T, a.waits.err);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    Team team{p.team_warps, warp % p.team_warps, warp / p.team_warps, slots, 0, WARPS};
    const int cta_teams = WARPS / p.team_warps;
    const int64_t number = (int64_t)blockIdx.x * cta_teams + team.id;
    const int t0 = (int)min(a.T, number * p.chunk), t1 = (int)min(a.T, number * p.chunk + p.chunk);
    const int col = (team.warp * 32 + lane) * N, step = p.team_warps * 32 * N;
    const float inv_d = 1.f / (float)a.D;
    const T *x = (const T*)g.x_out, *y = (const T*)g.y, *dxo = (const T*)g.d_x_out, *dn = (const T*)g.d_n;
    const T *gate = (const T*)a.gate, *wp = (const T*)a.w_post, *wn = (const T*)a.w_pre;
    Ring rows(bars, a, team.id);
    rows.p[0] = x;
    rows.p[1] = y;
    rows.p[2] = dxo;
    rows.p[3] = dn;
    if (threadIdx.x == 0) init_bars<S>(bars, WARPS);
    __syncthreads();
    rows.start(team, t0, t1);
    using F = typename Pack<T, N>::F;
    constexpr int kF = Pack<T, N>::kF;
    F s_gate[NV][kF], s_post[NV][kF], s_pre[NV][kF];
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < kF; ++j) s_gate[i][j] = s_post[i][j] = s_pre[i][j] = both<F>(0.f);
    Sequence seq{a.offsets, (int)a.B, (int)a.T, 0, 0};
    F gw[NV][kF];                                          // gate * w_post of the sequence
    auto load_gate = [&] {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = col + i * step;
            if (c >= a.D) continue;
            Pack<T, N> w, k;
            w.load(wp + c);
            if (ALL || gate) k.load(gate + (int64_t)seq.b * a.D + c);
#pragma unroll
            for (int j = 0; j < kF; ++j) gw[i][j] = ALL || gate ? mul_(k.get(j), w.get(j)) : w.get(j);
        }
    };
    // s_gate, the sum of g u over the tokens of seq.b among this team's, goes to
    // its place and, times the gate, to s_post
    int2 open = make_int2(-1, 0);
    auto flush = [&] {
        const bool head = seq.begin() < t0, goes_on = seq.end > t1;
        if (goes_on && !head) open = make_int2(seq.b, seq.end);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = col + i * step;
            if (c >= a.D) continue;
            if (g.d_gate) {
                if (head || goes_on) {
                    float* to = p.gates + (number * 2 + (head ? 0 : 1)) * a.D + c;
#pragma unroll
                    for (int j = 0; j < kF; ++j) *reinterpret_cast<F*>(to + j * (N / kF)) = s_gate[i][j];
                } else {
                    Pack<T, N> w, o;
                    w.load(wp + c);
#pragma unroll
                    for (int j = 0; j < kF; ++j) o.set(j, mul_(w.get(j), s_gate[i][j]));
                    o.store((T*)g.d_gate + (int64_t)seq.b * a.D + c);
                }
            }
            Pack<T, N> k;
            if (ALL || gate) k.load(gate + (int64_t)seq.b * a.D + c);
#pragma unroll
            for (int j = 0; j < kF; ++j) {
                s_post[i][j] = fma_(ALL || gate ? k.get(j) : both<F>(1.f), s_gate[i][j], s_post[i][j]);
                s_gate[i][j] = both<F>(0.f);
            }
        }
    };
    if (t0 < t1 && (ALL || gate)) seq.start(t0);
    if (t0 < t1 && (ALL || y)) load_gate();
    const F rho = both<F>(a.rho);
    int first = t0;                                        // token of the place
    for (int t = t0; t < t1; ++t) {
        const int64_t at = (int64_t)t * a.D;
        if ((ALL || gate) && seq.moved(t)) {
            flush();
            seq.move(t);
            load_gate();
        }
        if (t == first) rows.enter(team, t);
        F qx = both<F>(0.f), qz = both<F>(0.f), qy = both<F>(0.f);      // x'^2, z x', y^2
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = col + i * step;
            if (c >= a.D) continue;
            if (ALL || dn) {
                const Pack<T, N> r = rows.get(0, c), n = rows.get(3, c);
                Pack<T, N> w;
                w.load(wn + c);
#pragma unroll
                for (int j = 0; j < kF; ++j) {
                    const F x_ = r.get(j);
                    qx = fma_(x_, x_, qx);
                    qz = fma_(mul_(n.get(j), w.get(j)), x_, qz);
                }
            }
            if (ALL || y) {
                const Pack<T, N> r = rows.get(1, c);
#pragma unroll
                for (int j = 0; j < kF; ++j) qy = fma_(r.get(j), r.get(j), qy);
            }
        }
        const float3 q = team.sum3(total(qx), total(qz), total(qy));
        const float ix_ = ALL || dn ? rsqrtf(fmaf(q.x, inv_d, a.eps)) : 0.f, iy_ = rsqrtf(fmaf(q.z, inv_d, a.eps));
        // the mean first: of a row of zeros it is 0, and the cube of its 1 / rms may
        // lie beyond float32 (from eps = 2e-26 down)
        const F ix = both<F>(ix_), along = both<F>(-(q.y * inv_d * ix_) * ix_ * ix_), iy = both<F>(iy_);
        F v[NV][kF], m = both<F>(0.f);                     // du / rms(y); du u
        Pack<T, N> ry[NV];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = col + i * step;
            if (c >= a.D) continue;
            if (ALL || dxo) {
                const Pack<T, N> r = rows.get(2, c);
#pragma unroll
                for (int j = 0; j < kF; ++j) v[i][j] = r.get(j);
            } else {
#pragma unroll
                for (int j = 0; j < kF; ++j) v[i][j] = both<F>(0.f);
            }
            if (ALL || dn) {
                const Pack<T, N> r = rows.get(0, c), n = rows.get(3, c);
                Pack<T, N> w;
                w.load(wn + c);
#pragma unroll
                for (int j = 0; j < kF; ++j) {
                    const F x_ = r.get(j), n_ = mul_(n.get(j), ix);
                    v[i][j] = fma_(x_, along, fma_(n_, w.get(j), v[i][j]));
                    s_pre[i][j] = fma_(n_, x_, s_pre[i][j]);
                }
            }
            Pack<T, N> o;
#pragma unroll
            for (int j = 0; j < kF; ++j) o.set(j, mul_(rho, v[i][j]));
            o.store((T*)g.dx + at + c);
            if (ALL || y) {
                ry[i] = rows.get(1, c);
#pragma unroll
                for (int j = 0; j < kF; ++j) {
                    const F y_ = ry[i].get(j), gi = mul_(v[i][j], iy);
                    s_gate[i][j] = fma_(gi, y_, s_gate[i][j]);
                    v[i][j] = mul_(gi, gw[i][j]);
                    m = fma_(v[i][j], y_, m);
                }
            }
        }
        rows.next();
        const bool last = ends_place(t, first, t1, rows.per);
        if (last) rows.done();
        const float along_u = team.sum(total(m));          // with a barrier
        if (last) {
            if (!rows.leave(team, first, t1)) {
                rows.drain(first, t1);
                break;
            }
            first = t + 1;
        }
        if (!ALL && !y) continue;
        const F back = both<F>(-(along_u * inv_d * iy_) * iy_);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = col + i * step;
            if (c >= a.D) continue;
            Pack<T, N> o;
#pragma unroll
            for (int j = 0; j < kF; ++j) o.set(j, fma_(ry[i].get(j), back, v[i][j]));
            o.store((T*)g.dy + at + c);
        }
    }
    if (t0 < t1 && (ALL || y)) flush();
    if (g.d_gate && team.warp == 0 && lane == 0) p.open[number] = open;
    // the CTA's sums for the norms' weights, teams in order
    float* sums = reinterpret_cast<float*>(join_smem);     // [teams of the CTA][D]
    auto gather = [&](const F (&s)[NV][kF], float* to) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int j = 0; j < kF; ++j)
                if (col + i * step < a.D)
                    *reinterpret_cast<F*>(sums + team.id * a.D + col + i * step + j * (N / kF)) = s[i][j];
        __syncthreads();
        for (int c = threadIdx.x; c < a.D; c += WARPS * 32) {
            float v = 0.f;
            for (int k = 0; k < cta_teams; ++k) v += sums[k * a.D + c];
            to[c] = v;
        }
    };
    if (ALL || y) gather(s_post, p.weights + (int64_t)blockIdx.x * 2 * a.D);
    if (ALL || dn) gather(s_pre, p.weights + ((int64_t)blockIdx.x * 2 + 1) * a.D);
}

// CTAs (128 columns each along y) of three kinds along x: 0 and 1 add the norms'
// weights over the CTAs before; the next ones, for 32 teams each, add the
// partial sums of sequences that begin among a team's tokens and go on (a warp
// per team, or for long ones the CTA); the rest clear the gradients of empty
// sequences' gates.
constexpr int kFinishWarps = 32;         // teams per CTA too
constexpr int kClearRows = kFinishWarps * 32;
constexpr int kWarpRows = 16;            // partial sums that a warp adds by itself

template <class T>
__global__ void __launch_bounds__(kFinishWarps * 32) k_join_finish(JoinArgs a, JoinGrads g, GradPlan p) {
    __shared__ float part[kFinishWarps][128];
    __shared__ int2 long_run[kFinishWarps];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int c0 = blockIdx.y * 128;
    wait_before();
    // v[j] += sum over rows first, first + by, ... <= last of from[row * stride + c0 + 32 j + lane]
    auto add_rows = [&](float (&v)[4], const float* from, int64_t stride, int64_t first, int64_t last, int by) {
        for (int64_t r = first; r <= last; r += 8 * by) {
            float q[8][4];               // eight rows' loads are issued before the first is added
#pragma unroll
            for (int u = 0; u < 8; ++u)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    q[u][j] = 0.f;
                    if (r + u * by <= last && c0 + j * 32 + lane < a.D)
                        q[u][j] = __ldcg(from + (r + u * by) * stride + c0 + j * 32 + lane);
                }
#pragma unroll
            for (int u = 0; u < 8; ++u)
#pragma unroll
                for (int j = 0; j < 4; ++j) v[j] += q[u][j];
        }
    };
    // the same with rows spread over the CTA's warps: column threadIdx.x < 128
    auto cta_rows = [&](const float* from, int64_t stride, int64_t first, int64_t last) {
        float v[4] = {0.f, 0.f, 0.f, 0.f};
        add_rows(v, from, stride, first + warp, last, kFinishWarps);
        __syncthreads();
#pragma unroll
        for (int j = 0; j < 4; ++j) part[warp][j * 32 + lane] = v[j];
        __syncthreads();
        float sum = 0.f;
        if (threadIdx.x < 128)
            for (int w = 0; w < kFinishWarps; ++w) sum += part[w][threadIdx.x];
        return sum;
    };
    const int c = c0 + threadIdx.x;
    if (blockIdx.x < 2) {
        T* out = (T*)(blockIdx.x == 0 ? g.d_w_post : g.d_w_pre);
        if (!out) return;
        const float v = cta_rows(p.weights + blockIdx.x * a.D, 2 * a.D, 0, p.ctas - 1);
        if (threadIdx.x < 128 && c < a.D) out[c] = from_f32<T>(v);
        return;
    }
    const int64_t group = (int64_t)blockIdx.x - 2, groups = (p.teams + kFinishWarps - 1) / kFinishWarps;
    const T* wp = (const T*)a.w_post;
    if (group < groups) {
        const int64_t k = group * kFinishWarps + warp;
        int2 open = k < p.teams ? __ldcg(p.open + k) : make_int2(-1, 0);
        open.y = (int)min(p.teams - 1, (int64_t)((open.y - 1) / (int)p.chunk));       // the last team with tokens of it
        const int64_t b = open.x, last = open.x < 0 ? -1 : open.y;
        // this team's second row, then the first row of those that follow
        const bool alone = last - k <= kWarpRows;
        if (lane == 0) long_run[warp] = alone ? make_int2(-1, 0) : open;
        if (last >= 0 && alone) {
            float v[4] = {0.f, 0.f, 0.f, 0.f};
            add_rows(v, p.gates + a.D, 2 * a.D, k, k, 1);
            add_rows(v, p.gates, 2 * a.D, k + 1, last, 1);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int e = c0 + j * 32 + lane;
                if (e < a.D) ((T*)g.d_gate)[b * a.D + e] = from_f32<T>(to_f32(wp[e]) * v[j]);
            }
        }
        __syncthreads();
        for (int w = 0; w < kFinishWarps; ++w) {
            if (long_run[w].x < 0) continue;
            const int64_t kw = group * kFinishWarps + w, bw = long_run[w].x;
            const float v = cta_rows(p.gates, 2 * a.D, kw + 1, long_run[w].y);
            if (threadIdx.x < 128 && c < a.D)
                ((T*)g.d_gate)[bw * a.D + c] = from_f32<T>(to_f32(wp[c]) * (__ldcg(p.gates + (kw * 2 + 1) * a.D + c) + v));
        }
        return;
    }
    const int64_t b0 = (group - groups) * kClearRows + warp * 32;
    uint32_t empty = __ballot_sync(0xFFFFFFFFu, b0 + lane < a.B && __ldg(a.offsets + b0 + lane) == __ldg(a.offsets + b0 + lane + 1));
    for (; empty; empty &= empty - 1u)
        for (int e = c0 + lane; e < min(a.D, c0 + 128); e += 32)
            ((T*)g.d_gate)[(b0 + __ffs(empty) - 1) * a.D + e] = from_f32<T>(0.f);
}

// ---- host ------------------------------------------------------------------------

cudaError_t check_without_tokens(const JoinArgs& a, cudaStream_t s) {
    if (!a.given) return cudaSuccess;
    const int64_t want = (a.B + 255) / 256, most = 8 * a.num_sms;
    return launch_next(k_check_offsets, dim3((unsigned)(want < most ? want : most)), dim3(256), 0, false, s, a);
}

// Elements per access: of 16, 8 or 4 bytes where every row of every array begins on
// a multiple of that, else one
template <class... P>
int access_elems(const JoinArgs& a, P... arrays) {
    uintptr_t all = (uintptr_t)a.gate | (uintptr_t)a.w_post | (uintptr_t)a.w_pre;
    const uintptr_t each[] = {(uintptr_t)arrays...};
    for (uintptr_t p : each) all |= p;
    const int e = (int)elem_bytes(a.type);
    all |= (uintptr_t)(a.D * e);
    return all % 16 == 0 ? 16 / e : (all % 8 == 0 ? 8 / e : (all % 4 == 0 ? 4 / e : 1));
}

// Warps per team and accesses per lane for rows of D, N elements an access, at
// most `most` columns a warp
struct Shape {
    int warps, accesses;
};
Shape team_shape(int D, int N, int most) {
    Shape s;
    s.warps = 1;
    while (s.warps * most < D) s.warps *= 2;
    s.accesses = (D + s.warps * 32 * N - 1) / (s.warps * 32 * N);
    return s;
}

// f(T, N, accesses) with the smallest compiled count of accesses >= n
template <class T, int N, int... NV, class Fn>
cudaError_t pick(int n, std::integer_sequence<int, NV...>, const Fn& f) {
    cudaError_t e = cudaErrorInvalidValue;
    bool done = false;
    ((!done && n <= NV ? (done = true, e = f(T(), std::integral_constant<int, N>(), std::integral_constant<int, NV>()))
                       : e),
     ...);
    return e;
}
template <int N>
using Count = std::integral_constant<int, N>;
template <int... NV>
using Counts = std::integer_sequence<int, NV...>;

}  // namespace

cudaError_t launch_norm_join(const JoinArgs& a, const void* x, const void* y, void* x_out, void* n_out,
                             cudaStream_t s) {
    if (a.T == 0) return check_without_tokens(a, s);
    const int N = access_elems(a, x, y, x_out, n_out);
    const Shape sh = team_shape(a.D, N, join_columns(a.D));
    auto go = [&](auto t, auto n, auto nv) {
        using T = decltype(t);
        const int cta_teams = kJoinThreads / 32 / sh.warps;
        const size_t smem = ring_bytes<T, n(), 2>(cta_teams, a.D);
        cudaError_t e = allow_smem(k_norm_join<T, n(), nv()>, smem);
        if (e == cudaSuccess) e = next_launch();
        if (e != cudaSuccess) return e;
        // as many CTAs as run at once; fewer tokens: one per team
        const int64_t want = (a.T + cta_teams - 1) / cta_teams, by_smem = 226 * 1024 / ((int64_t)smem + 2048);
        const int64_t regs = join_ctas(32 * n() * nv()), most = a.num_sms * (by_smem < regs ? by_smem : regs);
        const int64_t ctas = want < most ? want : most, chunk = (a.T + ctas * cta_teams - 1) / (ctas * cta_teams);
        k_norm_join<T, n(), nv()><<<(unsigned)ctas, kJoinThreads, smem, s>>>(a, sh.warps, chunk, (const T*)x, (const T*)y,
                                                                           (T*)x_out, (T*)n_out);
        return cudaGetLastError();
    };
    auto of16 = [&](auto t) {
        using T = decltype(t);
        if (N == 8) return pick<T, 8>(sh.accesses, Counts<1, 2, 4>(), go);
        if (N == 4) return pick<T, 4>(sh.accesses, Counts<1, 4, 8>(), go);
        if (N == 2) return pick<T, 2>(sh.accesses, Counts<2, 8, 16>(), go);
        return pick<T, 1>(sh.accesses, Counts<4, 16, 32>(), go);
    };
    if (a.type == IFVS_T_F16) return of16(__half());
    if (a.type == IFVS_T_BF16) return of16(__nv_bfloat16());
    if (N == 4) return pick<float, 4>(sh.accesses, Counts<1, 2, 4, 8>(), go);
    if (N == 2) return pick<float, 2>(sh.accesses, Counts<2, 8, 16>(), go);
    return pick<float, 1>(sh.accesses, Counts<4, 16, 32>(), go);
}

namespace {
GradPlan grad_plan(const JoinArgs& a) {
    GradPlan p{};
    p.team_warps = 1;
    while (p.team_warps * grad_columns(a.type, a.D) < a.D) p.team_warps *= 2;
    const int64_t cta_teams = kGradWarps / p.team_warps;
    const int64_t want = (a.T + cta_teams - 1) / cta_teams;
    p.ctas = (int)(want < a.num_sms ? want : a.num_sms);
    p.teams = p.ctas * cta_teams;
    p.chunk = p.teams ? (a.T + p.teams - 1) / p.teams : 1;
    return p;
}
}  // namespace

size_t norm_join_grad_bytes(const JoinArgs& a) {
    const GradPlan p = grad_plan(a);
    return (size_t)p.teams * sizeof(int2) + (size_t)(p.teams + p.ctas) * 2 * a.D * sizeof(float);
}

cudaError_t launch_norm_join_grad(const JoinArgs& a, const JoinGrads& g, uint8_t* work, cudaStream_t s) {
    const int N = access_elems(a, g.x_out, g.y, g.d_x_out, g.d_n, g.dx, g.dy, g.d_gate);
    const Shape sh = team_shape(a.D, N, grad_columns(a.type, a.D));
    GradPlan p = grad_plan(a);
    p.open = (int2*)work;
    p.gates = (float*)(p.open + p.teams);
    p.weights = p.gates + p.teams * 2 * a.D;
    auto go = [&](auto t, auto n, auto nv) {
        using T = decltype(t);
        auto rows = [&](auto places) {
            const bool all = g.y && g.d_x_out && g.d_n && a.gate;
            const auto kernel = all ? k_norm_join_grad<T, n(), nv(), places(), true> : k_norm_join_grad<T, n(), nv(), places(), false>;
            const int cta_teams = kGradWarps / p.team_warps;
            size_t smem = ring_bytes<T, n(), 4, places()>(cta_teams, a.D);
            const size_t sums = (size_t)cta_teams * a.D * sizeof(float);
            smem = smem > sums ? smem : sums;
            const cudaError_t r = allow_smem(kernel, smem);
            if (r != cudaSuccess) return r;
            return launch_next(kernel, dim3((unsigned)p.ctas), dim3(kGradWarps * 32), smem, false, s, a, g, p);
        };
        cudaError_t e = cudaSuccess;
        if (a.T > 0) {
            if constexpr (sizeof(T) == 4 && n() * nv() == 16)
                e = rows(Count<1>());
            else
                e = rows(Count<kGradStages>());
        }
        if (e != cudaSuccess) return e;
        const int64_t teams = g.d_gate ? p.teams : 0, clears = g.d_gate && a.offsets ? (a.B + kClearRows - 1) / kClearRows : 0;
        GradPlan q = p;
        q.teams = teams;
        return launch_next(k_join_finish<T>, dim3((unsigned)(2 + (teams + kFinishWarps - 1) / kFinishWarps + clears), (unsigned)((a.D + 127) / 128)),
                             dim3(kFinishWarps * 32), 0, true, s, a, g, q);
    };
    auto of16 = [&](auto t) {
        using T = decltype(t);
        if (N == 8) return pick<T, 8>(sh.accesses, Counts<1, 2>(), go);
        if (N == 4) return pick<T, 4>(sh.accesses, Counts<1, 2, 4>(), go);
        if (N == 2) return pick<T, 2>(sh.accesses, Counts<2, 4, 8>(), go);
        return pick<T, 1>(sh.accesses, Counts<4, 8, 16>(), go);
    };
    if (a.T == 0) {                 // no team: the gates' gradients are all zeros
        cudaError_t e = check_without_tokens(a, s);
        if (e == cudaSuccess && g.d_gate) e = cudaMemsetAsync(g.d_gate, 0, (size_t)a.B * a.D * elem_bytes(a.type), s);
        if (e != cudaSuccess) return e;
    }
    if (a.type == IFVS_T_F16) return of16(__half());
    if (a.type == IFVS_T_BF16) return of16(__nv_bfloat16());
    if (N == 4) return pick<float, 4>(sh.accesses, Counts<1, 2, 4>(), go);
    if (N == 2) return pick<float, 2>(sh.accesses, Counts<2, 4, 8>(), go);
    return pick<float, 1>(sh.accesses, Counts<4, 8, 16>(), go);
}

}  // namespace ifvs
