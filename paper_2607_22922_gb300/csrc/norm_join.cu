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
// two.  A team of 1 to 16 warps takes a token's rows through a ring of kStages
// places in shared memory, filled ahead by bulk copies, or by 4-byte
// asynchronous copies where rows do not begin on 16 bytes: each row is read
// once from memory, whatever the norms need of it, and a team's loads go on
// while it reduces.  A team takes tokens that follow each other: the sequence of
// the first is searched, the others' follow, and the gradient keeps its sums
// over tokens in registers.  A sequence inside a team's tokens has its gate's
// gradient written at once; one that reaches beyond them leaves float32 partial
// sums that k_join_finish adds in order, as it does with the norms' weights.  No
// result depends on timing.
#include "layers.cuh"
#include "scan_common.cuh"

namespace ifvs {

namespace {

// A team's reductions: warps of one team meet at a named barrier; two sets of
// slots, so that a set is not written again before all have read it.
struct Team {
    int warps, warp, id;        // warps of the team, this one's place, the team's number in the CTA
    float4* slots;              // [2][all warps of the CTA]
    int turn, all;
    __device__ __forceinline__ void sync() const {
        if (warps == 1)
            __syncwarp();
        else
            asm volatile("barrier.cta.sync %0, %1;" ::"r"(1 + id), "r"(warps * 32) : "memory");
    }
    __device__ __forceinline__ float4 sum(float4 v) {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            v.x += __shfl_xor_sync(0xFFFFFFFFu, v.x, o);
            v.y += __shfl_xor_sync(0xFFFFFFFFu, v.y, o);
            v.z += __shfl_xor_sync(0xFFFFFFFFu, v.z, o);
        }
        if (warps == 1) return v;
        float4* s = slots + turn * all + id * warps;
        turn ^= 1;
        if ((threadIdx.x & 31) == 0) s[warp] = v;
        sync();
        v = s[0];
        for (int w = 1; w < warps; ++w) {
            v.x += s[w].x;
            v.y += s[w].y;
            v.z += s[w].z;
        }
        return v;
    }
};

// The sequence of a team's next token, given that of an earlier one
struct Sequence {
    const int64_t* offsets;
    int64_t B, T, b, end;       // offsets[b + 1]
    __device__ __forceinline__ void start(int64_t t) {
        b = sequence_of(offsets, B, t);
        end = offsets ? __ldg(offsets + b + 1) : T;
    }
    // whether the sequence changes at token t
    __device__ __forceinline__ bool moved(int64_t t) const { return t >= end && b + 1 < B; }
    __device__ __forceinline__ void move(int64_t t) {
        ++b;
        end = __ldg(offsets + b + 1);
        if (t >= end && b + 1 < B) start(t);     // past empty sequences
    }
    __device__ __forceinline__ int64_t begin() const { return offsets ? __ldg(offsets + b) : 0; }
};

constexpr int kStages = 3;               // places of a ring (1: no copies ahead)

// A team's ring of rows: A arrays per place (absent ones are null).  Bulk copies
// (one thread, completion on an mbarrier) where rows begin on 16 bytes;
// otherwise 4-byte copies by all lanes, from the 4-byte word that holds the
// row's first element, so that a row lies `shift` bytes into its place.
template <class T, int N, int A, int S = kStages>
struct Rows {
    static constexpr bool kBulk = N * sizeof(T) == 16;
    const T* p[A];
    uint8_t* ring;              // S x A x stride bytes
    uint64_t* bars;             // S
    volatile int* dead;
    int* err;
    int D, stride, place = 0;
    uint32_t parity = 0;

    static __host__ __device__ int stride_of(int D) { return (D * (int)sizeof(T) + 4 + 15) / 16 * 16; }
    __device__ __forceinline__ uint8_t* at(int place_, int k) const { return ring + (place_ * A + k) * stride; }
    __device__ __forceinline__ uint32_t shift(int k, int64_t t) const {
        return kBulk ? 0u : (uint32_t)(reinterpret_cast<uintptr_t>(p[k] + t * D) & 3u);
    }
    // the whole team; its earlier reads of the place lie before a barrier of the team
    __device__ __forceinline__ void fill(const Team& team, int place_, int64_t t) const {
        const int lane = threadIdx.x & 31;
        if constexpr (kBulk) {
            if (team.warp == 0 && lane == 0) {
                const uint32_t bar = (uint32_t)__cvta_generic_to_shared(bars + place_), bytes = D * sizeof(T);
                int n = 0;
#pragma unroll
                for (int k = 0; k < A; ++k) n += p[k] != nullptr;
                mbar_arrive_expect_tx(bar, n * bytes);
                const uint64_t once = policy_evict_first();
#pragma unroll
                for (int k = 0; k < A; ++k)
                    if (p[k]) bulk_g2s((uint32_t)__cvta_generic_to_shared(at(place_, k)), p[k] + t * D, bytes, bar, once);
            }
        } else {
#pragma unroll
            for (int k = 0; k < A; ++k) {
                if (!p[k]) continue;
                const uint8_t* row = reinterpret_cast<const uint8_t*>(p[k] + t * D);
                const uint32_t s = shift(k, t), end = s + D * sizeof(T);
                const uint32_t dst = (uint32_t)__cvta_generic_to_shared(at(place_, k));
                for (uint32_t w = (team.warp * 32 + lane) * 4; w < end; w += team.warps * 128) {
                    if (w >= s && w + 4 <= end) {
                        asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst + w), "l"(row - s + w) : "memory");
                    } else {                // a word of which the row has one half: no byte beside the row is read
                        const uint32_t h = w < s ? s : w;
                        *reinterpret_cast<uint16_t*>(at(place_, k) + h) = __ldg(reinterpret_cast<const uint16_t*>(row - s + h));
                    }
                }
            }
        }
    }
    __device__ __forceinline__ void close() const {      // after every fill, taken place or not
        if constexpr (!kBulk) asm volatile("cp.async.commit_group;" ::: "memory");
    }
    // the place's rows are there, for the whole team.  A wait that runs out marks
    // the CTA: later waits return at once, the team goes on and its results are
    // reported as incomplete
    __device__ __forceinline__ void wait(const Team& team) const {
        if constexpr (kBulk) {
            const uint32_t bar = (uint32_t)__cvta_generic_to_shared(bars + place);
            if (!mbar_try_wait(bar, parity)) {
                const long long t0 = clock64();
                while (!mbar_try_wait(bar, parity) && !*dead)
                    if (clock64() - t0 > kWaitCycles) {
                        *dead = 1;
                        *err = kErrWait;
                    }
            }
        } else {
            asm volatile("cp.async.wait_group %0;" ::"n"(S - 1) : "memory");
            team.sync();
        }
    }
    __device__ __forceinline__ Pack<T, N> get(int k, int64_t t, int col) const {
        Pack<T, N> v;
        const uint8_t* q = at(place, k) + shift(k, t) + col * sizeof(T);
        v.w = *reinterpret_cast<const typename Pack<T, N>::Word*>(q);
        return v;
    }
    // this place is read by the whole team: orders the reads before its next fill
    __device__ __forceinline__ void leave(const Team& team, int64_t t, int64_t end) {
        if constexpr (kBulk) fence_proxy_async_smem();
        team.sync();
        if (t + S < end) fill(team, place, t + S);
        close();
        if (++place == S) {
            place = 0;
            parity ^= 1u;
        }
    }
    __device__ __forceinline__ void start(const Team& team, int64_t t0, int64_t t1) const {
        for (int i = 0; i < S; ++i) {
            if (t0 + i < t1) fill(team, i, t0 + i);
            close();
        }
    }
    // copies in flight after a wait that ran out: bounded
    __device__ __forceinline__ void drain() const {
        if constexpr (kBulk) {
            if (!*dead) return;
            for (int i = 0; i < S; ++i) {
                const long long t0 = clock64();
                while (!mbar_try_wait((uint32_t)__cvta_generic_to_shared(bars + i), parity ^ (i < place ? 1u : 0u)) &&
                       clock64() - t0 < kWaitCycles) {
                }
            }
        }
    }
};

constexpr int kJoinThreads = 256;
constexpr int kJoinColumns = 1024;       // columns a warp holds at most

// Shared memory of a kernel whose `teams` teams have rings of A rows a place
template <class T, int N, int A, int S = kStages>
size_t ring_bytes(int teams, int D) {
    return (size_t)teams * S * A * Rows<T, N, A>::stride_of(D);
}

// Tokens [chunk team, chunk (team + 1)) of team number `team`
template <class T, int N, int NV>
__global__ void __launch_bounds__(kJoinThreads, 2)
k_norm_join(JoinArgs a, int team_warps, int64_t chunk, const T* __restrict__ x, const T* __restrict__ y,
            T* __restrict__ xo, T* __restrict__ no) {
    extern __shared__ __align__(16) uint8_t rings[];
    __shared__ float4 slots[2 * kJoinThreads / 32];
    __shared__ __align__(8) uint64_t bars[kJoinThreads / 32 * kStages];
    __shared__ int dead;
    check_offsets(a.offsets, a.B, a.T, a.err);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    Team team{team_warps, warp % team_warps, warp / team_warps, slots, 0, kJoinThreads / 32};
    const int64_t number = (int64_t)blockIdx.x * (kJoinThreads / 32 / team_warps) + team.id;
    const int64_t t0 = number * chunk, t1 = min(a.T, t0 + chunk);
    const int col = (team.warp * 32 + lane) * N, step = team_warps * 32 * N;
    const float inv_d = 1.f / (float)a.D;
    const T* gate = (const T*)a.gate;
    const T* wp = (const T*)a.w_post;
    const T* wn = (const T*)a.w_pre;
    Rows<T, N, 2> rows{{x, y}, rings + team.id * kStages * 2 * Rows<T, N, 2>::stride_of(a.D), bars + team.id * kStages,
                       &dead, a.err, a.D, Rows<T, N, 2>::stride_of(a.D)};
    if (threadIdx.x == 0) {
        for (int i = 0; i < kJoinThreads / 32 * kStages; ++i) mbar_init((uint32_t)__cvta_generic_to_shared(bars + i), 1);
        dead = 0;
        fence_mbar_init();
    }
    __syncthreads();
    if (t0 >= t1) return;
    rows.start(team, t0, t1);
    using F = typename Pack<T, N>::F;
    constexpr int kF = Pack<T, N>::kF;
    Sequence seq{a.offsets, a.B, a.T, 0, 0};
    F gw[NV][kF];                    // gate * w_post of the sequence
    auto load_gate = [&] {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = col + i * step;
            if (c >= a.D) continue;
            Pack<T, N> w, g;
            w.load(wp + c);
            if (gate) g.load(gate + seq.b * a.D + c);
#pragma unroll
            for (int j = 0; j < kF; ++j) gw[i][j] = gate ? mul_(g.get(j), w.get(j)) : w.get(j);
        }
    };
    if (gate) seq.start(t0);
    if (y) load_gate();
    const F rho = both<F>(a.rho);
    for (int64_t t = t0; t < t1; ++t) {
        F v[NV][kF], q = both<F>(0.f);
        if (gate && seq.moved(t)) {
            seq.move(t);
            load_gate();
        }
        rows.wait(team);
        if (y) {
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int c = col + i * step;
                if (c >= a.D) continue;
                const Pack<T, N> r = rows.get(1, t, c);
#pragma unroll
                for (int j = 0; j < kF; ++j) {
                    v[i][j] = r.get(j);
                    q = fma_(v[i][j], v[i][j], q);
                }
            }
            const F iy = both<F>(rsqrtf(fmaf(team.sum(make_float4(total(q), 0.f, 0.f, 0.f)).x, inv_d, a.eps)));
            q = both<F>(0.f);
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int c = col + i * step;
                if (c >= a.D) continue;
                const Pack<T, N> r = rows.get(0, t, c);
                Pack<T, N> o;
#pragma unroll
                for (int j = 0; j < kF; ++j) {
                    v[i][j] = fma_(mul_(v[i][j], iy), gw[i][j], mul_(rho, r.get(j)));
                    q = fma_(v[i][j], v[i][j], q);
                    o.set(j, v[i][j]);
                }
                o.store(xo + t * a.D + c);
            }
        } else {
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int c = col + i * step;
                if (c >= a.D) continue;
                const Pack<T, N> r = rows.get(0, t, c);
#pragma unroll
                for (int j = 0; j < kF; ++j) {
                    v[i][j] = r.get(j);
                    q = fma_(v[i][j], v[i][j], q);
                }
            }
        }
        rows.leave(team, t, t1);
        if (!no) continue;
        const F ix = both<F>(rsqrtf(fmaf(team.sum(make_float4(total(q), 0.f, 0.f, 0.f)).x, inv_d, a.eps)));
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = col + i * step;
            if (c >= a.D) continue;
            Pack<T, N> w, o;
            w.load(wn + c);
#pragma unroll
            for (int j = 0; j < kF; ++j) o.set(j, mul_(w.get(j), mul_(v[i][j], ix)));
            o.store(no + t * a.D + c);
        }
    }
    rows.drain();
}

// ---- gradient ------------------------------------------------------------------
// 16 warps of 16-bit rows, 8 of float32 rows: three places of four rows each fit
// the shared memory at 512 columns a warp.  One row of float32 beyond 4096 takes
// 16 warps, and a single place.
constexpr int grad_warps(int type, int D) { return type == IFVS_T_F32 && D <= 8 * 512 ? 8 : 16; }
constexpr int kGradColumns = 512;        // columns a warp holds at most

struct GradPlan {
    int team_warps, ctas;
    int64_t teams, chunk;
    float* gates;        // [teams][2][D]: sums of the sequence that reaches into the team's tokens from
                         // before, and of the one that begins in them and goes on
    float* weights;      // [ctas][2][D]: d_w_post, d_w_pre
};

template <class T, int N, int NV, int WARPS, int S>
__global__ void __launch_bounds__(WARPS * 32, 1) k_norm_join_grad(JoinArgs a, JoinGrads g, GradPlan p) {
    using Ring = Rows<T, N, 4, S>;
    __shared__ float4 slots[2 * WARPS];
    __shared__ __align__(8) uint64_t bars[WARPS * S];
    __shared__ int dead;
    extern __shared__ __align__(16) uint8_t rings[];     // after the tokens: [teams of the CTA][D] sums
    check_offsets(a.offsets, a.B, a.T, a.err);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    Team team{p.team_warps, warp % p.team_warps, warp / p.team_warps, slots, 0, WARPS};
    const int cta_teams = WARPS / p.team_warps;
    const int64_t number = (int64_t)blockIdx.x * cta_teams + team.id;
    const int64_t t0 = min(a.T, number * p.chunk), t1 = min(a.T, t0 + p.chunk);
    const int col = (team.warp * 32 + lane) * N, step = p.team_warps * 32 * N;
    const float inv_d = 1.f / (float)a.D;
    const T *x = (const T*)g.x_out, *y = (const T*)g.y, *dxo = (const T*)g.d_x_out, *dn = (const T*)g.d_n;
    const T *gate = (const T*)a.gate, *wp = (const T*)a.w_post, *wn = (const T*)a.w_pre;
    Ring rows{{x, y, dxo, dn}, rings + team.id * S * 4 * Ring::stride_of(a.D), bars + team.id * S, &dead, a.err, a.D,
              Ring::stride_of(a.D)};
    if (threadIdx.x == 0) {
        for (int i = 0; i < WARPS * S; ++i) mbar_init((uint32_t)__cvta_generic_to_shared(bars + i), 1);
        dead = 0;
        fence_mbar_init();
    }
    __syncthreads();
    rows.start(team, t0, t1);
    using F = typename Pack<T, N>::F;
    constexpr int kF = Pack<T, N>::kF;
    F s_gate[NV][kF], s_post[NV][kF], s_pre[NV][kF];
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < kF; ++j) s_gate[i][j] = s_post[i][j] = s_pre[i][j] = both<F>(0.f);
    Sequence seq{a.offsets, a.B, a.T, 0, 0};
    F gw[NV][kF];                                          // gate * w_post of the sequence
    auto load_gate = [&] {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = col + i * step;
            if (c >= a.D) continue;
            Pack<T, N> w, k;
            w.load(wp + c);
            if (gate) k.load(gate + seq.b * a.D + c);
#pragma unroll
            for (int j = 0; j < kF; ++j) gw[i][j] = gate ? mul_(k.get(j), w.get(j)) : w.get(j);
        }
    };
    // s_gate, the sum of g u over the tokens of seq.b among this team's, goes to
    // its place and, times the gate, to s_post
    auto flush = [&] {
        const bool head = seq.begin() < t0, goes_on = seq.end > t1;
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
                    o.store((T*)g.d_gate + seq.b * a.D + c);
                }
            }
            Pack<T, N> k;
            if (gate) k.load(gate + seq.b * a.D + c);
#pragma unroll
            for (int j = 0; j < kF; ++j) {
                s_post[i][j] = fma_(gate ? k.get(j) : both<F>(1.f), s_gate[i][j], s_post[i][j]);
                s_gate[i][j] = both<F>(0.f);
            }
        }
    };
    if (t0 < t1 && gate) seq.start(t0);
    if (t0 < t1 && y) load_gate();
    const F rho = both<F>(a.rho);
    for (int64_t t = t0; t < t1; ++t) {
        const int64_t at = t * a.D;
        if (gate && seq.moved(t)) {
            flush();
            seq.move(t);
            load_gate();
        }
        rows.wait(team);
        F qx = both<F>(0.f), qz = both<F>(0.f), qy = both<F>(0.f);      // x'^2, z x', y^2
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = col + i * step;
            if (c >= a.D) continue;
            if (dn) {
                const Pack<T, N> r = rows.get(0, t, c), n = rows.get(3, t, c);
                Pack<T, N> w;
                w.load(wn + c);
#pragma unroll
                for (int j = 0; j < kF; ++j) {
                    const F x_ = r.get(j);
                    qx = fma_(x_, x_, qx);
                    qz = fma_(mul_(n.get(j), w.get(j)), x_, qz);
                }
            }
            if (y) {
                const Pack<T, N> r = rows.get(1, t, c);
#pragma unroll
                for (int j = 0; j < kF; ++j) qy = fma_(r.get(j), r.get(j), qy);
            }
        }
        const float4 q = team.sum(make_float4(total(qx), total(qz), total(qy), 0.f));
        const float ix_ = dn ? rsqrtf(fmaf(q.x, inv_d, a.eps)) : 0.f, iy_ = rsqrtf(fmaf(q.z, inv_d, a.eps));
        const F ix = both<F>(ix_), along = both<F>(-ix_ * ix_ * ix_ * (q.y * inv_d)), iy = both<F>(iy_);
        F v[NV][kF], m = both<F>(0.f);                     // du / rms(y); du u
        Pack<T, N> ry[NV];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = col + i * step;
            if (c >= a.D) continue;
            if (dxo) {
                const Pack<T, N> r = rows.get(2, t, c);
#pragma unroll
                for (int j = 0; j < kF; ++j) v[i][j] = r.get(j);
            } else {
#pragma unroll
                for (int j = 0; j < kF; ++j) v[i][j] = both<F>(0.f);
            }
            if (dn) {
                const Pack<T, N> r = rows.get(0, t, c), n = rows.get(3, t, c);
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
            if (y) {
                ry[i] = rows.get(1, t, c);
#pragma unroll
                for (int j = 0; j < kF; ++j) {
                    const F y_ = ry[i].get(j), gi = mul_(v[i][j], iy);
                    s_gate[i][j] = fma_(gi, y_, s_gate[i][j]);
                    v[i][j] = mul_(gi, gw[i][j]);
                    m = fma_(v[i][j], y_, m);
                }
            }
        }
        rows.leave(team, t, t1);
        if (!y) continue;
        const F back = both<F>(-iy_ * iy_ * (team.sum(make_float4(total(m), 0.f, 0.f, 0.f)).x * inv_d));
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
    rows.drain();
    if (t0 < t1 && y) flush();
    // the CTA's sums for the norms' weights, teams in order
    float* sums = reinterpret_cast<float*>(rings);
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
    if (y) gather(s_post, p.weights + (int64_t)blockIdx.x * 2 * a.D);
    if (dn) gather(s_pre, p.weights + ((int64_t)blockIdx.x * 2 + 1) * a.D);
}

// CTAs (128 columns each along y) of three kinds along x: 0 and 1 add the norms'
// weights over the CTAs before; the next ones, for 32 teams each, add the
// partial sums of sequences that begin among a team's tokens and go on (a warp
// per team, or for long ones the CTA); the rest clear the gradients of empty
// sequences' gates.
constexpr int kFinishWarps = 32;         // teams per CTA too
constexpr int kClearRows = 1024;
constexpr int kWarpRows = 16;            // partial sums that a warp adds by itself

template <class T>
__global__ void __launch_bounds__(kFinishWarps * 32) k_join_finish(JoinArgs a, JoinGrads g, GradPlan p) {
    __shared__ float part[kFinishWarps][128];
    __shared__ int64_t long_last[kFinishWarps];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int c0 = blockIdx.y * 128;
    wait_before();
    // v[j] += sum over rows first, first + by, ... <= last of from[row * stride + c0 + 32 j + lane]
    auto add_rows = [&](float (&v)[4], const float* from, int64_t stride, int64_t first, int64_t last, int by) {
#pragma unroll 4
        for (int64_t r = first; r <= last; r += by)
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (c0 + j * 32 + lane < a.D) v[j] += __ldcg(from + r * stride + c0 + j * 32 + lane);
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
        const int64_t k = group * kFinishWarps + warp, t0 = k * p.chunk, t1 = t0 + p.chunk;
        int64_t last = -1, b = 0;
        if (k < p.teams && t1 < a.T) {
            b = sequence_of(a.offsets, a.B, t1 - 1);
            const int64_t begin = a.offsets ? __ldg(a.offsets + b) : 0;
            const int64_t end = a.offsets ? min(a.T, __ldg(a.offsets + b + 1)) : a.T;
            if (begin >= t0 && end > t1) last = min(p.teams - 1, (end - 1) / p.chunk);
        }
        // this team's second row, then the first row of those that follow
        const bool alone = last - k <= kWarpRows;
        if (lane == 0) long_last[warp] = alone ? -1 : last;
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
            if (long_last[w] < 0) continue;
            const int64_t kw = group * kFinishWarps + w, bw = sequence_of(a.offsets, a.B, kw * p.chunk + p.chunk - 1);
            const float v = cta_rows(p.gates, 2 * a.D, kw + 1, long_last[w]);
            if (threadIdx.x < 128 && c < a.D)
                ((T*)g.d_gate)[bw * a.D + c] = from_f32<T>(to_f32(wp[c]) * (__ldcg(p.gates + (kw * 2 + 1) * a.D + c) + v));
        }
        return;
    }
    const int64_t b0 = (group - groups) * kClearRows;
    for (int64_t b = b0 + warp; b < min(a.B, b0 + kClearRows); b += kFinishWarps)
        if (__ldg(a.offsets + b) == __ldg(a.offsets + b + 1))
            for (int e = c0 + lane; e < min(a.D, c0 + 128); e += 32) ((T*)g.d_gate)[b * a.D + e] = from_f32<T>(0.f);
}

// ---- host ------------------------------------------------------------------------

// Elements per access: 16 bytes where every row of every array begins on 16,
// 4 bytes for even widths of the 16-bit types
template <class... P>
int access_elems(const JoinArgs& a, P... arrays) {
    uintptr_t all = (uintptr_t)a.gate | (uintptr_t)a.w_post | (uintptr_t)a.w_pre;
    const uintptr_t each[] = {(uintptr_t)arrays...};
    for (uintptr_t p : each) all |= p;
    const int e = (int)elem_bytes(a.type);
    all |= (uintptr_t)(a.D * e);
    return all % 16 == 0 ? 16 / e : (all % 4 == 0 ? 4 / e : 1);
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
    const int N = access_elems(a, x, y, x_out, n_out);
    const Shape sh = team_shape(a.D, N, kJoinColumns);
    auto go = [&](auto t, auto n, auto nv) {
        using T = decltype(t);
        const int cta_teams = kJoinThreads / 32 / sh.warps;
        const size_t smem = ring_bytes<T, n(), 2>(cta_teams, a.D);
        const cudaError_t e = cudaFuncSetAttribute(k_norm_join<T, n(), nv()>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
        if (e != cudaSuccess) return e;
        // as many CTAs as run at once; fewer tokens: one per team
        const int64_t want = (a.T + cta_teams - 1) / cta_teams, most = (int64_t)a.num_sms * (smem > 110 * 1024 ? 1 : 2);
        const int64_t ctas = want < most ? want : most, chunk = (a.T + ctas * cta_teams - 1) / (ctas * cta_teams);
        k_norm_join<T, n(), nv()><<<(unsigned)ctas, kJoinThreads, smem, s>>>(a, sh.warps, chunk, (const T*)x, (const T*)y,
                                                                           (T*)x_out, (T*)n_out);
        return cudaGetLastError();
    };
    auto of16 = [&](auto t) {
        using T = decltype(t);
        if (N == 8) return pick<T, 8>(sh.accesses, Counts<1, 2, 4>(), go);
        if (N == 2) return pick<T, 2>(sh.accesses, Counts<2, 8, 16>(), go);
        return pick<T, 1>(sh.accesses, Counts<4, 16, 32>(), go);
    };
    if (a.type == IFVS_T_F16) return of16(__half());
    if (a.type == IFVS_T_BF16) return of16(__nv_bfloat16());
    return N == 4 ? pick<float, 4>(sh.accesses, Counts<1, 2, 4, 8>(), go)
                  : pick<float, 1>(sh.accesses, Counts<4, 16, 32>(), go);
}

namespace {
GradPlan grad_plan(const JoinArgs& a) {
    GradPlan p{};
    p.team_warps = 1;
    while (p.team_warps * kGradColumns < a.D) p.team_warps *= 2;
    const int64_t cta_teams = grad_warps(a.type, a.D) / p.team_warps;
    const int64_t want = (a.T + cta_teams - 1) / cta_teams;
    p.ctas = (int)(want < a.num_sms ? want : a.num_sms);
    p.teams = p.ctas * cta_teams;
    p.chunk = p.teams ? (a.T + p.teams - 1) / p.teams : 1;
    return p;
}
}  // namespace

size_t norm_join_grad_bytes(const JoinArgs& a) {
    const GradPlan p = grad_plan(a);
    return (size_t)(p.teams + p.ctas) * 2 * a.D * sizeof(float);
}

cudaError_t launch_norm_join_grad(const JoinArgs& a, const JoinGrads& g, uint8_t* work, cudaStream_t s) {
    const int N = access_elems(a, g.x_out, g.y, g.d_x_out, g.d_n, g.dx, g.dy, g.d_gate);
    const Shape sh = team_shape(a.D, N, kGradColumns);
    GradPlan p = grad_plan(a);
    p.gates = (float*)work;
    p.weights = p.gates + p.teams * 2 * a.D;
    auto go = [&](auto t, auto n, auto nv) {
        using T = decltype(t);
        auto rows = [&](auto warps, auto places) {
            const auto kernel = k_norm_join_grad<T, n(), nv(), warps(), places()>;
            const int cta_teams = warps() / p.team_warps;
            size_t smem = ring_bytes<T, n(), 4, places()>(cta_teams, a.D);
            const size_t sums = (size_t)cta_teams * a.D * sizeof(float);
            smem = smem > sums ? smem : sums;
            const cudaError_t r = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
            if (r != cudaSuccess) return r;
            kernel<<<(unsigned)p.ctas, warps() * 32, smem, s>>>(a, g, p);
            return cudaGetLastError();
        };
        cudaError_t e = cudaSuccess;
        if (a.T == 0) {
        } else if constexpr (sizeof(T) == 2) {
            e = rows(Count<16>(), Count<kStages>());
        } else if (grad_warps(a.type, a.D) == 8) {
            e = rows(Count<8>(), Count<kStages>());
        } else if constexpr (n() * nv() == 16) {
            e = rows(Count<16>(), Count<1>());
        }
        if (e != cudaSuccess) return e;
        const int64_t teams = g.d_gate ? p.teams : 0, clears = g.d_gate && a.offsets ? (a.B + kClearRows - 1) / kClearRows : 0;
        GradPlan q = p;
        q.teams = teams;
        return launch_kernel(k_join_finish<T>, dim3((unsigned)(2 + (teams + kFinishWarps - 1) / kFinishWarps + clears), (unsigned)((a.D + 127) / 128)),
                             dim3(kFinishWarps * 32), 0, true, s, a, g, q);
    };
    auto of16 = [&](auto t) {
        using T = decltype(t);
        if (N == 8) return pick<T, 8>(sh.accesses, Counts<1, 2>(), go);
        if (N == 2) return pick<T, 2>(sh.accesses, Counts<2, 8>(), go);
        return pick<T, 1>(sh.accesses, Counts<4, 16>(), go);
    };
    if (a.T == 0 && g.d_gate) {     // no team: the gates' gradients are all zeros
        const cudaError_t e = cudaMemsetAsync(g.d_gate, 0, (size_t)a.B * a.D * elem_bytes(a.type), s);
        if (e != cudaSuccess) return e;
    }
    if (a.type == IFVS_T_F16) return of16(__half());
    if (a.type == IFVS_T_BF16) return of16(__nv_bfloat16());
    return N == 4 ? pick<float, 4>(sh.accesses, Counts<1, 2, 4>(), go) : pick<float, 1>(sh.accesses, Counts<4, 16>(), go);
}

}  // namespace ifvs
