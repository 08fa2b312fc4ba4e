// Layer norm and the residual tail on rows of up to ROW_MOST features: a row stays in the registers of a team of threads.
//
// Every array passes once.  A team is 4, 8, 16 or 32 lanes of a warp, or a few warps; a thread holds ITEMS pieces of 16 bytes of its
// row.  Pieces begin at multiples of 16 bytes of the array, not of the row: where rows begin anywhere (EDGES), a team's rows are
// those that begin at the same place inside a piece, so that a thread's features are the same ones in each of its rows.  It therefore
// keeps their weights, and in a VJP the sums of their gradients, in registers; the teams of a block add those sums up at
// its end, and weight_grads (prior_norm.cuh) adds up the blocks.
#pragma once
#include "prior_common.cuh"

namespace gleam {
namespace prior {

constexpr int ROW_TEAMS_THREADS = 512;

__device__ __forceinline__ void team_barrier(int team, int threads) { asm volatile("bar.sync %0, %1;" ::"r"(team + 1), "r"(threads) : "memory"); }

// Where a thread stands: its team (in the block and in the grid), its place in it, and its features.
template <class T, int TEAM, int ITEMS, bool EDGES>
struct RowPlace {
    int width, team, t, first;           // threads of a team, team in the block, thread in the team, feature of its first piece
    long long row, rows_apart;
    __device__ __forceinline__ RowPlace(const Args& a, int warps, int teams) {
        width = TEAM ? TEAM : warps * 32;
        team = threadIdx.x / width;
        t = threadIdx.x - team * width;
        row = (long long)blockIdx.x * teams + team;
        rows_apart = (long long)gridDim.x * teams;
        int phase = 0;
        if (EDGES) phase = (int)(row % VEC<T>) * (int)(a.features % VEC<T>) % VEC<T>;
        first = t * VEC<T> - phase;
    }
    __device__ __forceinline__ int feature(int k) const { return first + k * width * VEC<T>; }
};

// One piece of a row: whole, or the features of it that lie in the row (others become 0).
template <class T, bool EDGES>
__device__ __forceinline__ Pack<T> load_piece(const T* row, int c, int n, bool packed) {
    Pack<T> p;
    if (EDGES ? packed && c >= 0 && c + VEC<T> <= n : c < n) {
        p = load_pack(row + c);
    } else {
#pragma unroll
        for (int j = 0; j < VEC<T>; ++j) p.e[j] = EDGES && (unsigned)(c + j) < (unsigned)n ? row[c + j] : from_float<T>(0.f);
    }
    return p;
}
template <class T, bool EDGES>
__device__ __forceinline__ void store_piece(T* row, int c, int n, bool packed, const Pack<T>& p) {
    if (EDGES ? packed && c >= 0 && c + VEC<T> <= n : c < n) {
        store_pack(row + c, p);
    } else if (EDGES) {
#pragma unroll
        for (int j = 0; j < VEC<T>; ++j)
            if ((unsigned)(c + j) < (unsigned)n) row[c + j] = p.e[j];
    }
}
template <class T, int ITEMS, bool EDGES, class Place>
__device__ __forceinline__ void load_weights(const void* w, int f32, float missing, const Place& at, int n, float (&v)[ITEMS][VEC<T>]) {
#pragma unroll
    for (int k = 0; k < ITEMS; ++k)
#pragma unroll
        for (int j = 0; j < VEC<T>; ++j) {
            const int c = at.feature(k) + j;
            v[k][j] = !w ? missing : (unsigned)c < (unsigned)n ? weight_at<T>(w, f32, c) : 0.f;
        }
}

template <int TEAM>
__device__ __forceinline__ float lanes_sum(float v) {
#pragma unroll
    for (int o = (TEAM && TEAM < 32 ? TEAM : 32) / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// What the warps of a team exchange: three numbers each, in two sets that take turns, so that one barrier is enough.
struct Exchange {
    float* at; int warps, warp, team, turn;
    __device__ __forceinline__ Exchange(float* shared, int warps_, int team_, int t) : warps(warps_), warp(t >> 5), team(team_), turn(0) {
        at = shared + team_ * 2 * 3 * warps_;
    }
    __device__ __forceinline__ const float* put(float a, float b, float c, int t) {
        float* set = at + turn * 3 * warps;
        if ((t & 31) == 0) { set[3 * warp] = a; set[3 * warp + 1] = b; set[3 * warp + 2] = c; }
        team_barrier(team, warps * 32);
        turn ^= 1;
        return set;
    }
};

template <class T, int TEAM, int ITEMS, bool EDGES, bool TAIL>
__global__ void __launch_bounds__(ROW_TEAMS_THREADS, ITEMS * VEC<T> > 8 ? 1 : 2) row_team_forward(const __grid_constant__ Args a, int warps, int teams) {
    grid_dependency_wait();
    extern __shared__ float shared[];
    constexpr int V = VEC<T>;
    const RowPlace<T, TEAM, ITEMS, EDGES> at(a, warps, teams);
    Exchange exchange(shared, warps, at.team, at.t);
    const Mask mask(a);
    const int n = (int)a.features;
    const bool packed = a.aligned;
    const float count = (float)n;
    float w[ITEMS][V], b[ITEMS][V];
    load_weights<T, ITEMS, EDGES>(a.weight, a.weight_f32, 1.f, at, n, w);
    load_weights<T, ITEMS, EDGES>(a.bias, a.weight_f32, 0.f, at, n, b);
    // the lanes of a warp go on together
    const long long lead = TEAM && TEAM < 32 ? (threadIdx.x & 31) / TEAM : 0;
    for (long long r = at.row; r - lead < a.outer; r += at.rows_apart) {
        const bool live = !TEAM || TEAM == 32 || r < a.outer;
        float v[ITEMS][V];
        if (live) {
            const T* x = static_cast<const T*>(a.x) + r * a.px;
            if (!TAIL) {
#pragma unroll
                for (int k = 0; k < ITEMS; ++k) unpack(load_piece<T, EDGES>(x, at.feature(k), n, packed), v[k]);
            } else {
                const T* res = static_cast<const T*>(a.res) + r * a.pres;
                T* sum = static_cast<T*>(a.out2) + r * a.pout2;
                Pack<T> px[ITEMS], pr[ITEMS];
#pragma unroll
                for (int k = 0; k < ITEMS; ++k) {
                    px[k] = load_piece<T, EDGES>(x, at.feature(k), n, packed);
                    pr[k] = load_piece<T, EDGES>(res, at.feature(k), n, packed);
                }
#pragma unroll
                for (int k = 0; k < ITEMS; ++k) {
                    const int c = at.feature(k);
                    uint4 words[V / 4];
                    if (a.dropping) {
#pragma unroll
                        for (int q = 0; q < V / 4; ++q) words[q] = mask.words((uint64_t)(r * n + c) / 4 + q);
                    }
                    float xs[V], rs[V];
                    unpack(px[k], xs);
                    unpack(pr[k], rs);
#pragma unroll
                    for (int j = 0; j < V; ++j) {
                        const float kept = fmaf(xs[j], a.scale, rs[j]);
                        rs[j] = a.dropping && mask.dropped(words[j / 4], j % 4) ? rs[j] : kept;
                    }
                    const Pack<T> stored = pack<T>(rs);
                    unpack(stored, v[k]);
                    store_piece<T, EDGES>(sum, c, n, packed, stored);
                }
            }
        }
        // features of the row in this thread's pieces; the others are 0 in v
        auto inside = [&](int k, int j) { return live && (EDGES ? (unsigned)(at.feature(k) + j) < (unsigned)n : at.feature(k) < n); };
        float s = 0.f;
#pragma unroll
        for (int k = 0; k < ITEMS; ++k)
#pragma unroll
            for (int j = 0; j < V; ++j) s += inside(k, j) ? v[k][j] : 0.f;
        s = lanes_sum<TEAM>(s);
        float mean, q = 0.f;
        if (TEAM) {
            mean = s / count;
#pragma unroll
            for (int k = 0; k < ITEMS; ++k)
#pragma unroll
                for (int j = 0; j < V; ++j) { const float d = v[k][j] - mean; q += inside(k, j) ? d * d : 0.f; }
            q = lanes_sum<TEAM>(q);
        } else {
            // every warp's mean and squared deviations from it; then sum (d_w + m_w - m)^2 = sum d_w^2 + n_w (m_w - m)^2
            int here = 0;
#pragma unroll
            for (int k = 0; k < ITEMS; ++k) {
                const int c = at.feature(k);
                here += max(0, min(c + V, n) - max(c, 0));
            }
            const float nw = (float)__reduce_add_sync(0xffffffffu, here), mw = nw > 0.f ? s / nw : 0.f;
#pragma unroll
            for (int k = 0; k < ITEMS; ++k)
#pragma unroll
                for (int j = 0; j < V; ++j) { const float d = v[k][j] - mw; q += inside(k, j) ? d * d : 0.f; }
            q = lanes_sum<TEAM>(q);
            const float* set = exchange.put(s, q, nw, at.t);
            s = 0.f;
            for (int u = 0; u < warps; ++u) s += set[3 * u];
            mean = s / count;
            q = 0.f;
            for (int u = 0; u < warps; ++u) {
                const float m = set[3 * u + 2] > 0.f ? set[3 * u] / set[3 * u + 2] - mean : 0.f;
                q += fmaf(set[3 * u + 2] * m, m, set[3 * u + 1]);
            }
        }
        const float rstd = 1.f / sqrtf(q / count + a.eps);
        if (!live) continue;
        T* y = static_cast<T*>(a.out) + r * a.pout;
#pragma unroll
        for (int k = 0; k < ITEMS; ++k) {
#pragma unroll
            for (int j = 0; j < V; ++j) v[k][j] = fmaf((v[k][j] - mean) * rstd, w[k][j], b[k][j]);
            store_piece<T, EDGES>(y, at.feature(k), n, packed, pack<T>(v[k]));
        }
        if (at.t == 0) {
            if (a.mean) a.mean[r] = mean;
            if (a.rstd) a.rstd[r] = rstd;
        }
    }
}

template <class T, int TEAM, int ITEMS, bool EDGES, bool TAIL>
__global__ void __launch_bounds__(ROW_TEAMS_THREADS, 1) row_team_vjp(const __grid_constant__ Args a, int warps, int teams) {
    grid_dependency_wait();
    extern __shared__ float shared[];
    constexpr int V = VEC<T>;
    const RowPlace<T, TEAM, ITEMS, EDGES> at(a, warps, teams);
    Exchange exchange(shared, warps, at.team, at.t);
    const Mask mask(a);
    const int n = (int)a.features;
    const bool packed = a.aligned;
    const float count = (float)n;
    float w[ITEMS][V], gw[ITEMS][V], gb[ITEMS][V];
    load_weights<T, ITEMS, EDGES>(a.weight, a.weight_f32, 1.f, at, n, w);
#pragma unroll
    for (int k = 0; k < ITEMS; ++k)
#pragma unroll
        for (int j = 0; j < V; ++j) gw[k][j] = gb[k][j] = 0.f;
    const long long lead = TEAM && TEAM < 32 ? (threadIdx.x & 31) / TEAM : 0;
    for (long long r = at.row; r - lead < a.outer; r += at.rows_apart) {
        const bool live = !TEAM || TEAM == 32 || r < a.outer;
        Pack<T> pg[ITEMS], pv[ITEMS], ps[ITEMS];
        float mean = 0.f, rstd = 0.f;
        const bool added = TAIL && a.gsum;
        if (live) {
            mean = a.mean[r]; rstd = a.rstd[r];
#pragma unroll
            for (int k = 0; k < ITEMS; ++k) {
                const int c = at.feature(k);
                pg[k] = load_piece<T, EDGES>(static_cast<const T*>(a.x) + r * a.px, c, n, packed);
                pv[k] = load_piece<T, EDGES>(static_cast<const T*>(a.res) + r * a.pres, c, n, packed);
                if (added) ps[k] = load_piece<T, EDGES>(static_cast<const T*>(a.gsum) + r * a.pgsum, c, n, packed);
            }
        }
        float s1 = 0.f, s2 = 0.f;
#pragma unroll
        for (int k = 0; k < ITEMS; ++k) {
            if (!live) break;
            float g[V], v[V];
            unpack(pg[k], g);
            unpack(pv[k], v);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                // a feature beyond the row has g = 0
                const float h = (v[j] - mean) * rstd, d = g[j] * w[k][j];
                gw[k][j] = fmaf(g[j], h, gw[k][j]);
                gb[k][j] += g[j];
                s1 += d;
                s2 = fmaf(d, h, s2);
            }
        }
        s1 = lanes_sum<TEAM>(s1);
        s2 = lanes_sum<TEAM>(s2);
        if (!TEAM) {
            const float* set = exchange.put(s1, s2, 0.f, at.t);
            s1 = s2 = 0.f;
            for (int u = 0; u < warps; ++u) { s1 += set[3 * u]; s2 += set[3 * u + 1]; }
        }
        if (!live) continue;
        s1 /= count; s2 /= count;
        T* out = static_cast<T*>(a.out) + r * a.pout;
        T* out2 = TAIL ? static_cast<T*>(a.out2) + r * a.pout2 : nullptr;
#pragma unroll
        for (int k = 0; k < ITEMS; ++k) {
            const int c = at.feature(k);
            float g[V], v[V];
            unpack(pg[k], g);
            unpack(pv[k], v);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float h = (v[j] - mean) * rstd;
                v[j] = rstd * (g[j] * w[k][j] - s1 - h * s2);
            }
            if (TAIL) {
                if (added) {
                    unpack(ps[k], g);
#pragma unroll
                    for (int j = 0; j < V; ++j) v[j] += g[j];
                }
                store_piece<T, EDGES>(out2, c, n, packed, pack<T>(v));
                if (a.dropping) {
#pragma unroll
                    for (int q = 0; q < V / 4; ++q) {
                        const uint4 words = mask.words((uint64_t)(r * n + c) / 4 + q);
#pragma unroll
                        for (int j = 0; j < 4; ++j) v[4 * q + j] = mask.dropped(words, j) ? 0.f : v[4 * q + j] * a.scale;
                    }
                }
            }
            store_piece<T, EDGES>(out, c, n, packed, pack<T>(v));
        }
    }
    if (!a.gw && !a.gb) return;
    auto put = [&](int c, int which, float v) {
        if (gridDim.x > 1) a.part[((long long)blockIdx.x * 2 + which) * n + c] = v;
        else if (which ? a.gb : a.gw) store_weight_grad<T>(which ? a.gb : a.gw, a.weight_f32, c, v);
    };
    if (teams == 1) {
#pragma unroll
        for (int k = 0; k < ITEMS; ++k)
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const int c = at.feature(k) + j;
                if ((unsigned)c < (unsigned)n) { put(c, 0, gw[k][j]); put(c, 1, gb[k][j]); }
            }
        return;
    }
    // sums over the block's teams, one team after another
    __syncthreads();
    float* total = shared;
    for (int c = threadIdx.x; c < 2 * n; c += blockDim.x) total[c] = 0.f;
    for (int u = 0; u < teams; ++u) {
        __syncthreads();
        if (at.team != u) continue;
#pragma unroll
        for (int k = 0; k < ITEMS; ++k)
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const int c = at.feature(k) + j;
                if ((unsigned)c < (unsigned)n) { total[c] += gw[k][j]; total[n + c] += gb[k][j]; }
            }
    }
    __syncthreads();
    for (int c = threadIdx.x; c < n; c += blockDim.x) { put(c, 0, total[c]); put(c, 1, total[n + c]); }
}

}  // namespace prior
}  // namespace gleam
