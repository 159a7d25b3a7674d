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
// two.  A team of 1 to 16 warps holds a token's rows in registers, so that each
// is read once whatever the norms need of it.  A team takes tokens that follow
// each other: the sequence of the first is searched, the others' follow, and
// the gradient keeps its sums over tokens in registers.  A sequence inside a
// team's tokens has its gate's gradient written at once; one that reaches
// beyond them leaves float32 partial sums that k_join_finish adds in order, as
// it does with the norms' weights.  No result depends on timing.
#include "layers.cuh"

namespace ifvs {

namespace {

// A team's reductions: warps of one team meet at a named barrier; two sets of
// slots, so that a set is not written again before all have read it.
struct Team {
    int warps, warp, id;        // warps of the team, this one's place, the team's number in the CTA
    float4* slots;              // [2][all warps of the CTA]
    int turn, all;
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
        asm volatile("barrier.cta.sync %0, %1;" ::"r"(1 + id), "r"(warps * 32) : "memory");
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

template <class T, int N, int NV>
struct Row {
    Pack<T, N> v[NV];
    // p: the row; columns beyond D read as zeros
    __device__ __forceinline__ void load(const T* p, int col, int step, int D) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            v[i].w = {};
            if (col + i * step < D) v[i].load(p + col + i * step);
        }
    }
    __device__ __forceinline__ float get(int i, int j) const { return v[i].get(j); }
};

constexpr int kJoinThreads = 256;

// Tokens [chunk team, chunk (team + 1)) of team number `team`
template <class T, int N, int NV>
__global__ void __launch_bounds__(kJoinThreads, N * NV > 16 ? 3 : 4)
k_norm_join(JoinArgs a, int team_warps, int64_t chunk, const T* __restrict__ x, const T* __restrict__ y,
            T* __restrict__ xo, T* __restrict__ no) {
    __shared__ float4 slots[2 * kJoinThreads / 32];
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
    if (t0 >= t1) return;
    Sequence seq{a.offsets, a.B, a.T, 0, 0};
    if (gate) seq.start(t0);
    for (int64_t t = t0; t < t1; ++t) {
        Row<T, N, NV> rx, ry;
        rx.load(x + t * a.D, col, step, a.D);
        float v[NV][N];
        float q = 0.f;
        if (y) {
            ry.load(y + t * a.D, col, step, a.D);
            if (gate && seq.moved(t)) seq.move(t);
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int j = 0; j < N; ++j) q = fmaf(ry.get(i, j), ry.get(i, j), q);
            const float iy = rsqrtf(fmaf(team.sum(make_float4(q, 0.f, 0.f, 0.f)).x, inv_d, a.eps));
            q = 0.f;
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int c = col + i * step;
                if (c >= a.D) continue;
                Pack<T, N> w, g, o;
                w.load(wp + c);
                if (gate) g.load(gate + seq.b * a.D + c);
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    const float post = w.get(j) * (ry.get(i, j) * iy);
                    v[i][j] = fmaf(a.rho, rx.get(i, j), gate ? g.get(j) * post : post);
                    q = fmaf(v[i][j], v[i][j], q);
                    o.set(j, v[i][j]);
                }
                o.store(xo + t * a.D + c);
            }
        } else {
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    v[i][j] = rx.get(i, j);
                    q = fmaf(v[i][j], v[i][j], q);
                }
        }
        if (!no) continue;
        const float ix = rsqrtf(fmaf(team.sum(make_float4(q, 0.f, 0.f, 0.f)).x, inv_d, a.eps));
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = col + i * step;
            if (c >= a.D) continue;
            Pack<T, N> w, o;
            w.load(wn + c);
#pragma unroll
            for (int j = 0; j < N; ++j) o.set(j, w.get(j) * (v[i][j] * ix));
            o.store(no + t * a.D + c);
        }
    }
}

// ---- gradient ------------------------------------------------------------------
constexpr int kGradThreads = 512;
constexpr int kGradWarps = kGradThreads / 32;
constexpr int kGradColumns = 512;        // columns a warp holds at most

struct GradPlan {
    int team_warps, ctas;
    int64_t teams, chunk;
    float* gates;        // [teams][2][D]: sums of the sequence that reaches into the team's tokens from
                         // before, and of the one that begins in them and goes on
    float* weights;      // [ctas][2][D]: d_w_post, d_w_pre
};

template <class T, int N, int NV>
__global__ void __launch_bounds__(kGradThreads, 1) k_norm_join_grad(JoinArgs a, JoinGrads g, GradPlan p) {
    __shared__ float4 slots[2 * kGradWarps];
    extern __shared__ float sums[];          // [teams of the CTA][D]
    check_offsets(a.offsets, a.B, a.T, a.err);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    Team team{p.team_warps, warp % p.team_warps, warp / p.team_warps, slots, 0, kGradWarps};
    const int cta_teams = kGradWarps / p.team_warps;
    const int64_t number = (int64_t)blockIdx.x * cta_teams + team.id;
    const int64_t t0 = min(a.T, number * p.chunk), t1 = min(a.T, t0 + p.chunk);
    const int col = (team.warp * 32 + lane) * N, step = p.team_warps * 32 * N;
    const float inv_d = 1.f / (float)a.D;
    const T *x = (const T*)g.x_out, *y = (const T*)g.y, *dxo = (const T*)g.d_x_out, *dn = (const T*)g.d_n;
    const T *gate = (const T*)a.gate, *wp = (const T*)a.w_post, *wn = (const T*)a.w_pre;
    float s_gate[NV][N], s_post[NV][N], s_pre[NV][N];
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < N; ++j) s_gate[i][j] = s_post[i][j] = s_pre[i][j] = 0.f;
    Sequence seq{a.offsets, a.B, a.T, 0, 0};
    // the sums of the tokens of seq.b among this team's
    auto flush = [&] {
        const bool head = seq.begin() < t0, goes_on = seq.end > t1;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = col + i * step;
            if (c >= a.D) continue;
            if (head || goes_on) {
                float* to = p.gates + (number * 2 + (head ? 0 : 1)) * a.D + c;
#pragma unroll
                for (int j = 0; j < N; ++j) to[j] = s_gate[i][j];
            } else {
                Pack<T, N> w, o;
                w.load(wp + c);
#pragma unroll
                for (int j = 0; j < N; ++j) o.set(j, w.get(j) * s_gate[i][j]);
                o.store((T*)g.d_gate + seq.b * a.D + c);
            }
#pragma unroll
            for (int j = 0; j < N; ++j) s_gate[i][j] = 0.f;
        }
    };
    if (t0 < t1 && gate) seq.start(t0);
    for (int64_t t = t0; t < t1; ++t) {
        const int64_t at = t * a.D;
        Row<T, N, NV> rx, ry, rd, rn;
        rx.load(x + at, col, step, a.D);
        if (dn) rn.load(dn + at, col, step, a.D);
        if (y) ry.load(y + at, col, step, a.D);
        if (dxo) rd.load(dxo + at, col, step, a.D);
        if (gate && seq.moved(t)) {
            if (g.d_gate) flush();
            seq.move(t);
        }
        float4 q = make_float4(0.f, 0.f, 0.f, 0.f);        // x'^2, z x', y^2
        float v[NV][N];                                    // z, then g
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = col + i * step;
            Pack<T, N> w;
            w.w = {};
            if (dn && c < a.D) w.load(wn + c);
#pragma unroll
            for (int j = 0; j < N; ++j) {
                v[i][j] = dn ? rn.get(i, j) * w.get(j) : 0.f;
                q.x = fmaf(rx.get(i, j), rx.get(i, j), q.x);
                q.y = fmaf(v[i][j], rx.get(i, j), q.y);
                if (y) q.z = fmaf(ry.get(i, j), ry.get(i, j), q.z);
            }
        }
        q = team.sum(q);
        const float ix = dn ? rsqrtf(fmaf(q.x, inv_d, a.eps)) : 0.f, iy = rsqrtf(fmaf(q.z, inv_d, a.eps));
        const float along = ix * ix * (q.y * inv_d);
        float m = 0.f;                                     // du u
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = col + i * step;
            if (c >= a.D) continue;
            Pack<T, N> w, k, o;
            if (y) w.load(wp + c);
            if (gate) k.load(gate + seq.b * a.D + c);
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const float xv = rx.get(i, j);
                float gv = ix * (v[i][j] - xv * along);
                if (dxo) gv += rd.get(i, j);
                if (dn) s_pre[i][j] = fmaf(rn.get(i, j) * ix, xv, s_pre[i][j]);
                o.set(j, a.rho * gv);
                if (y) {
                    const float gu = gv * (ry.get(i, j) * iy), gk = gate ? k.get(j) : 1.f;
                    s_gate[i][j] += gu;
                    s_post[i][j] = fmaf(gk, gu, s_post[i][j]);
                    v[i][j] = gk * w.get(j) * gv;          // du
                    m = fmaf(v[i][j], ry.get(i, j) * iy, m);
                }
            }
            o.store((T*)g.dx + at + c);
        }
        if (!y) continue;
        m = team.sum(make_float4(m, 0.f, 0.f, 0.f)).x * inv_d;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = col + i * step;
            if (c >= a.D) continue;
            Pack<T, N> o;
#pragma unroll
            for (int j = 0; j < N; ++j) o.set(j, iy * (v[i][j] - (ry.get(i, j) * iy) * m));
            o.store((T*)g.dy + at + c);
        }
    }
    if (t0 < t1 && g.d_gate) flush();
    // the CTA's sums for the norms' weights, teams in order
    auto gather = [&](const float (&s)[NV][N], float* to) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int j = 0; j < N; ++j)
                if (col + i * step < a.D) sums[team.id * a.D + col + i * step + j] = s[i][j];
        __syncthreads();
        for (int c = threadIdx.x; c < a.D; c += kGradThreads) {
            float v = 0.f;
            for (int k = 0; k < cta_teams; ++k) v += sums[k * a.D + c];
            to[c] = v;
        }
    };
    if (y) gather(s_post, p.weights + (int64_t)blockIdx.x * 2 * a.D);
    if (dn) gather(s_pre, p.weights + ((int64_t)blockIdx.x * 2 + 1) * a.D);
}

// CTAs (32 columns each along y) of three kinds along x: 0 and 1 add the norms'
// weights over the CTAs before; the next ones, one per team, add the partial sums
// of a sequence that begins among the team's tokens and goes on; the rest clear
// the gradients of empty sequences' gates.
constexpr int kClearRows = 256;

template <class T>
__global__ void __launch_bounds__(256) k_join_finish(JoinArgs a, JoinGrads g, GradPlan p) {
    __shared__ float part[8][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int c = blockIdx.y * 32 + lane;
    wait_before();
    // sum over rows first + warp, first + warp + 8, ... <= last of p[row * stride + c]
    auto column_sum = [&](const float* from, int64_t stride, int64_t first, int64_t last) {
        float v = 0.f;
        if (c < a.D)
#pragma unroll 4
            for (int64_t r = first + warp; r <= last; r += 8) v += __ldcg(from + r * stride + c);
        part[warp][lane] = v;
        __syncthreads();
        v = 0.f;
        for (int w = 0; w < 8; ++w) v += part[w][lane];
        return v;
    };
    if (blockIdx.x < 2) {
        T* out = (T*)(blockIdx.x == 0 ? g.d_w_post : g.d_w_pre);
        if (!out) return;
        const float v = column_sum(p.weights + blockIdx.x * a.D, 2 * a.D, 0, p.ctas - 1);
        if (warp == 0 && c < a.D) out[c] = from_f32<T>(v);
        return;
    }
    const int64_t k = (int64_t)blockIdx.x - 2;
    if (k < p.teams) {
        const int64_t t0 = k * p.chunk, t1 = t0 + p.chunk;
        if (t1 >= a.T) return;
        const int64_t b = sequence_of(a.offsets, a.B, t1 - 1);
        const int64_t begin = a.offsets ? __ldg(a.offsets + b) : 0, end = a.offsets ? min(a.T, __ldg(a.offsets + b + 1)) : a.T;
        if (begin < t0 || end <= t1) return;
        const int64_t last = min(p.teams - 1, (end - 1) / p.chunk);
        // this team's second row, then the first row of those that follow
        float v = column_sum(p.gates, 2 * a.D, k + 1, last);
        if (warp == 0 && c < a.D) {
            v = __ldcg(p.gates + (k * 2 + 1) * a.D + c) + v;
            ((T*)g.d_gate)[b * a.D + c] = from_f32<T>(to_f32(((const T*)a.w_post)[c]) * v);
        }
        return;
    }
    if (c >= a.D) return;
    const int64_t b0 = (k - p.teams) * kClearRows;
    for (int64_t b = b0 + warp; b < min(a.B, b0 + kClearRows); b += 8)
        if (__ldg(a.offsets + b) == __ldg(a.offsets + b + 1)) ((T*)g.d_gate)[b * a.D + c] = from_f32<T>(0.f);
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
template <int... NV>
using Counts = std::integer_sequence<int, NV...>;

}  // namespace

cudaError_t launch_norm_join(const JoinArgs& a, const void* x, const void* y, void* x_out, void* n_out,
                             cudaStream_t s) {
    const int N = access_elems(a, x, y, x_out, n_out);
    const Shape sh = team_shape(a.D, N, 1024);
    auto go = [&](auto t, auto n, auto nv) {
        using T = decltype(t);
        constexpr int E = n() * nv();
        const int64_t cta_teams = kJoinThreads / 32 / sh.warps;
        const int64_t want = (a.T + cta_teams - 1) / cta_teams, most = (int64_t)a.num_sms * (E > 16 ? 3 : 4);
        const int64_t ctas = want < most ? want : most, chunk = (a.T + ctas * cta_teams - 1) / (ctas * cta_teams);
        k_norm_join<T, n(), nv()><<<(unsigned)ctas, kJoinThreads, 0, s>>>(a, sh.warps, chunk, (const T*)x, (const T*)y,
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
GradPlan grad_plan(const JoinArgs& a, int warps) {
    GradPlan p{};
    p.team_warps = warps;
    const int64_t cta_teams = kGradWarps / warps, want = (a.T + cta_teams - 1) / cta_teams;
    p.ctas = (int)(want < a.num_sms ? want : a.num_sms);
    p.teams = p.ctas * cta_teams;
    p.chunk = p.teams ? (a.T + p.teams - 1) / p.teams : 1;
    return p;
}
}  // namespace

// the team's shape depends on the arrays' alignment: room for teams of one warp
size_t norm_join_grad_bytes(const JoinArgs& a) {
    int warps = 1;
    while (warps * kGradColumns < a.D) warps *= 2;
    const GradPlan p = grad_plan(a, warps);
    return (size_t)(p.teams + p.ctas) * 2 * a.D * sizeof(float);
}

cudaError_t launch_norm_join_grad(const JoinArgs& a, const JoinGrads& g, uint8_t* work, cudaStream_t s) {
    const int N = access_elems(a, g.x_out, g.y, g.d_x_out, g.d_n, g.dx, g.dy, g.d_gate);
    const Shape sh = team_shape(a.D, N, kGradColumns);
    GradPlan p = grad_plan(a, sh.warps);
    p.gates = (float*)work;
    p.weights = p.gates + p.teams * 2 * a.D;
    auto go = [&](auto t, auto n, auto nv) {
        using T = decltype(t);
        const size_t smem = (size_t)(kGradWarps / sh.warps) * a.D * sizeof(float);     // at most 32 KB
        if (a.T > 0)
            k_norm_join_grad<T, n(), nv()><<<(unsigned)p.ctas, kGradThreads, smem, s>>>(a, g, p);
        cudaError_t e = cudaGetLastError();
        if (e != cudaSuccess) return e;
        const int64_t teams = g.d_gate ? p.teams : 0, clears = g.d_gate && a.offsets ? (a.B + kClearRows - 1) / kClearRows : 0;
        GradPlan q = p;
        q.teams = teams;
        return launch_kernel(k_join_finish<T>, dim3((unsigned)(2 + teams + clears), (unsigned)((a.D + 31) / 32)), dim3(256), 0,
                             true, s, a, g, q);
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
