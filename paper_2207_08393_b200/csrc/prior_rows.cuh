// Layer norm and the residual tail on rows: a row stays with a team of threads that passes over every array once.
//
// A team is 4, 8, 16 or 32 lanes of a warp, or a few warps; a thread has ITEMS pieces of 16 bytes of its row.  Pieces begin at
// multiples of 16 bytes of the array, not of the row: where rows begin anywhere (EDGES), a team's rows are those that begin at
// the same place inside a piece, so that a thread's features are the same ones in each of its rows, and so are their weights
// and, in a VJP, the sums of their gradients, which it keeps in registers.  The teams of a block add those sums up at its
// end, and weight_grads (prior_norm.cuh) adds up the blocks.
//
// Bound by memory where a thread has many features.  What a row costs each thread apart from its features (about a
// hundred instructions: the sums across lanes, the ring, the statistics) counts with few: with eight features a thread and a
// team of four warps, rows of 1024 in bf16 were bound by issue at 47 instructions a feature.  So a thread takes up to 32
// features before a second warp joins its team.
#pragma once
#include "prior_common.cuh"

namespace gleam {
namespace prior {

constexpr int ROW_BLOCK = 256, ROW_BLOCK_WARPS = ROW_BLOCK / 32, ROW_FEATURES = 32;    // threads a block, features a thread at most

__device__ __forceinline__ void team_barrier(int team, int threads) { asm volatile("bar.sync %0, %1;" ::"r"(team + 1), "r"(threads) : "memory"); }
__device__ __forceinline__ void copy16(uint32_t to, const void* from) { asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory"); }
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int LEFT> __device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(LEFT) : "memory"); }

// s / n for a whole n with inv = 1 / n: the product, corrected by its residual (exact where the quotient is representable).
__device__ __forceinline__ float quotient(float s, float n, float inv) {
    const float q = s * inv, r = fmaf(-q, n, s);
    return r == r ? fmaf(r, inv, q) : q;
}
// 1 / sqrt(x) with one Newton step on the approximation.
__device__ __forceinline__ float inverse_root(float x) {
    const float r = rsqrtf(x), e = fmaf(-x * r, r, 1.f);
    return e == e ? fmaf(0.5f * r, e, r) : r;
}

// Where a thread stands: its team (in the block and in the grid), its place in it, and its features.
template <class T, int TEAM, int ITEMS, bool EDGES>
struct RowPlace {
    static constexpr int V = VEC<T>;
    int width, team, t, phase;           // threads of a team, team in the block, thread in the team, where its rows begin in a piece
    long long row, rows_apart;
    __device__ __forceinline__ RowPlace(const Args& a, int warps, int teams) {
        width = TEAM ? TEAM : warps * 32;
        team = threadIdx.x / width;
        t = threadIdx.x - team * width;
        rows_apart = (long long)gridDim.x * teams;
        // several pieces a thread: all rows of a block lie alike, for its teams share the weights
        if (EDGES && ITEMS > 1) row = blockIdx.x % V + (long long)V * ((long long)(blockIdx.x / V) * teams + team);
        else row = (long long)blockIdx.x * teams + team;
        phase = EDGES ? (int)(row % V) * (int)(a.features % V) % V : 0;
    }
    __device__ __forceinline__ int piece(int k) const { return t + k * width; }
    __device__ __forceinline__ int feature(int k) const { return piece(k) * V - phase; }
};

// What is left of a piece with its first feature at c in a row of n: all of it, or some.
template <class T, bool EDGES>
__device__ __forceinline__ bool whole(int c, int n) { return EDGES ? c >= 0 && c + VEC<T> <= n : c < n; }
template <class T, bool EDGES>
__device__ __forceinline__ bool partly(int c, int n) { return EDGES && c < n && c + VEC<T> > 0; }

template <class T, bool EDGES>
__device__ __forceinline__ void store_piece(T* row, int c, int n, bool packed, const Pack<T>& p) {
    if (whole<T, EDGES>(c, n) && (!EDGES || packed)) {
        store_pack(row + c, p);
    } else if (partly<T, EDGES>(c, n)) {
#pragma unroll
        for (int j = 0; j < VEC<T>; ++j)
            if ((unsigned)(c + j) < (unsigned)n) row[c + j] = p.e[j];
    }
}
// The numbers of a piece; those beyond the row are 0.
template <class T, bool EDGES>
__device__ __forceinline__ void take(const Pack<T>& p, int c, int n, float (&v)[VEC<T>]) {
    unpack(p, v);
    if (!whole<T, EDGES>(c, n)) {
#pragma unroll
        for (int j = 0; j < VEC<T>; ++j) v[j] = EDGES && (unsigned)(c + j) < (unsigned)n ? v[j] : 0.f;
    }
}

template <int TEAM>
__device__ __forceinline__ float lanes_sum(float v) {
#pragma unroll
    for (int o = (TEAM && TEAM < 32 ? TEAM : 32) / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// A vector of the weights as the team's pieces hold it: with one piece a thread in registers, else in shared memory, where the
// quarters of the pieces lie one behind another (no bank conflicts).  The threads of a block fill it together.
template <class T, int TEAM, int ITEMS, bool EDGES>
struct Weights {
    static constexpr int V = VEC<T>;
    float own[V];
    const float4* shared;
    int pieces;
    template <class Place>
    __device__ __forceinline__ Weights(const void* w, const Args& a, float missing, const Place& at, float* room) : shared(nullptr), pieces(at.width * ITEMS) {
        const int n = (int)a.features;
        auto one = [&](int c) { return (unsigned)c >= (unsigned)n ? 0.f : w ? weight_at<T>(w, a.weight_f32, c) : missing; };
        if (ITEMS == 1) {
#pragma unroll
            for (int j = 0; j < V; ++j) own[j] = one(at.feature(0) + j);
        } else {
            for (int i = threadIdx.x; i < pieces * V; i += blockDim.x)
                room[((i % V) / 4 * pieces + i / V) * 4 + i % 4] = one(i - at.phase);
            shared = reinterpret_cast<const float4*>(room);
        }
    }
    __device__ __forceinline__ void get(int piece, float (&v)[V]) const {
        if (ITEMS == 1) {
#pragma unroll
            for (int j = 0; j < V; ++j) v[j] = own[j];
        } else {
#pragma unroll
            for (int q = 0; q < V / 4; ++q) {
                const float4 f = shared[q * pieces + piece];
                v[4 * q] = f.x; v[4 * q + 1] = f.y; v[4 * q + 2] = f.z; v[4 * q + 3] = f.w;
            }
        }
    }
};

// What the warps of a team exchange: four numbers each, in two sets that take turns, so that one barrier is enough.
struct Exchange {
    float4* at; int warps, warp, team, turn;
    __device__ __forceinline__ Exchange(float* shared, int warps_, int team_, int t) : warps(warps_), warp(t >> 5), team(team_), turn(0) {
        at = reinterpret_cast<float4*>(shared) + team_ * 2 * warps_;
    }
    __device__ __forceinline__ const float4* put(float4 v, int t) {
        float4* set = at + turn * warps;
        if ((t & 31) == 0) set[warp] = v;
        team_barrier(team, warps * 32);
        turn ^= 1;
        return set;
    }
};
constexpr int EXCHANGE_BYTES = 2 * ROW_BLOCK_WARPS * sizeof(float4);

// A thread's pieces of the rows to come, in shared memory: copied there by the thread itself, STAGES - 1 rows ahead, and read
// by it alone, so that no barrier is needed.  (Rows of 1024 in bf16, forward and VJP, teams of four warps: 216 us with loads into
// registers, 177 with the ring.)
template <class T, int ARRAYS, int ITEMS, int STAGES, bool EDGES>
struct Ring {
    Pack<T>* base;
    uint32_t address;
    __device__ __forceinline__ explicit Ring(void* shared) {
        base = static_cast<Pack<T>*>(shared) + threadIdx.x;
        address = (uint32_t)__cvta_generic_to_shared(base);
    }
    __device__ __forceinline__ int place(int stage, int array, int k) const { return ((stage * ARRAYS + array) * ITEMS + k) * (int)blockDim.x; }
    __device__ __forceinline__ Pack<T> get(int stage, int array, int k) const { return base[place(stage, array, k)]; }
    // Piece k of row r of an array, its first feature at c.  A piece over the row's ends is copied whole, with its neighbours'
    // elements, where the array has them.
    __device__ __forceinline__ void fetch(int stage, int array, int k, const void* from, long long pitch, long long r, int c, const Args& a) {
        const int n = (int)a.features;
        if (!whole<T, EDGES>(c, n) && !partly<T, EDGES>(c, n)) return;
        const T* row = static_cast<const T*>(from) + r * pitch;
        if (!EDGES || (a.aligned && r * pitch + c >= 0 && r * pitch + c + VEC<T> <= (a.outer - 1) * pitch + n)) {
            copy16(address + 16u * place(stage, array, k), row + c);
        } else {
            Pack<T> p;
#pragma unroll
            for (int j = 0; j < VEC<T>; ++j) p.e[j] = (unsigned)(c + j) < (unsigned)n ? row[c + j] : from_float<T>(0.f);
            base[place(stage, array, k)] = p;
        }
    }
};

// Blocks on an SM (registers) and rows in the ring: four, or as many as the shared memory holds beside the weights.
template <class T, bool VJP, int ITEMS> constexpr int row_blocks() { return VJP ? 2 : 3; }
template <class T, bool VJP, bool TAIL, int ITEMS>
constexpr int row_stages() {
    const int stage = ROW_BLOCK * 16 * ITEMS * ((VJP ? 2 : 1) + TAIL), room = 196 * 1024 / row_blocks<T, VJP, ITEMS>();
    return room / stage >= 4 ? 4 : room / stage >= 3 ? 3 : 2;
}

template <class T, int TEAM, int ITEMS, bool EDGES, bool TAIL>
__global__ void __launch_bounds__(ROW_BLOCK, row_blocks<T, false, ITEMS>()) row_team_forward(const __grid_constant__ Args a, int warps, int teams) {
    grid_dependency_wait();
    extern __shared__ __align__(16) float shared[];
    constexpr int V = VEC<T>, STAGES = row_stages<T, false, TAIL, ITEMS>(), ARRAYS = TAIL ? 2 : 1;
    const RowPlace<T, TEAM, ITEMS, EDGES> at(a, warps, teams);
    Exchange exchange(shared, warps, at.team, at.t);
    float* room = shared + EXCHANGE_BYTES / 4;
    Ring<T, ARRAYS, ITEMS, STAGES, EDGES> ring(room);
    room += ARRAYS * ITEMS * STAGES * 4 * blockDim.x;
    const Mask mask(a);
    const int n = (int)a.features;
    const bool packed = a.aligned;
    const float count = (float)n, inv_count = 1.f / count;
    auto fetch = [&](long long r, int stage) {
        if (r < a.outer) {
#pragma unroll
            for (int k = 0; k < ITEMS; ++k) {
                ring.fetch(stage, 0, k, a.x, a.px, r, at.feature(k), a);
                if (TAIL) ring.fetch(stage, 1, k, a.res, a.pres, r, at.feature(k), a);
            }
        }
        copies_commit();
    };
#pragma unroll
    for (int i = 0; i < STAGES - 1; ++i) fetch(at.row + i * at.rows_apart, i);
    const Weights<T, TEAM, ITEMS, EDGES> weight(a.weight, a, 1.f, at, room), bias(a.bias, a, 0.f, at, room + at.width * ITEMS * V);
    if (ITEMS > 1) __syncthreads();
    float here = 0.f;                              // features of the row that this warp has
    if (!TEAM) {
        int mine = 0;
#pragma unroll
        for (int k = 0; k < ITEMS; ++k) mine += max(0, min(at.feature(k) + V, n) - max(at.feature(k), 0));
        here = (float)__reduce_add_sync(0xffffffffu, mine);
    }
    const float inv_here = here > 0.f ? 1.f / here : 0.f;
    // the lanes of a warp go on together
    const long long lead = TEAM && TEAM < 32 ? (threadIdx.x & 31) / TEAM : 0;
    int stage = 0;
    for (long long r = at.row; r - lead < a.outer; r += at.rows_apart) {
        const bool live = !TEAM || TEAM == 32 || r < a.outer;
        fetch(r + (STAGES - 1) * at.rows_apart, stage == 0 ? STAGES - 1 : stage - 1);
        copies_wait<STAGES - 1>();
        float v[ITEMS][V];
#pragma unroll
        for (int k = 0; k < ITEMS; ++k) {
            const int c = at.feature(k);
            if (!TAIL) {
                take<T, EDGES>(ring.get(stage, 0, k), c, live ? n : 0, v[k]);
            } else {
                float xs[V], rs[V];
                uint4 words[V / 4];
                if (a.dropping) {
#pragma unroll
                    for (int q = 0; q < V / 4; ++q) words[q] = mask.words((uint64_t)((r * n - at.phase) / 4) + (uint32_t)(at.piece(k) * (V / 4) + q));
                }
                unpack(ring.get(stage, 0, k), xs);
                unpack(ring.get(stage, 1, k), rs);
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    const float kept = fmaf(xs[j], a.scale, rs[j]);
                    rs[j] = a.dropping && mask.dropped(words[j / 4], j % 4) ? rs[j] : kept;
                }
                const Pack<T> stored = pack<T>(rs);
                take<T, EDGES>(stored, c, live ? n : 0, v[k]);
                if (live) store_piece<T, EDGES>(static_cast<T*>(a.out2) + r * a.pout2, c, n, packed, stored);
            }
        }
        stage = stage + 1 == STAGES ? 0 : stage + 1;
        float s = 0.f;
#pragma unroll
        for (int k = 0; k < ITEMS; ++k)
#pragma unroll
            for (int j = 0; j < V; ++j) s += v[k][j];
        s = lanes_sum<TEAM>(s);
        auto deviations = [&](float m) {
            float q = 0.f;
#pragma unroll
            for (int k = 0; k < ITEMS; ++k) {
                const int c = at.feature(k);
                if (whole<T, EDGES>(c, n)) {
#pragma unroll
                    for (int j = 0; j < V; ++j) { const float d = v[k][j] - m; q = fmaf(d, d, q); }
                } else if (partly<T, EDGES>(c, n)) {
#pragma unroll
                    for (int j = 0; j < V; ++j) { const float d = (unsigned)(c + j) < (unsigned)n ? v[k][j] - m : 0.f; q = fmaf(d, d, q); }
                }
            }
            return lanes_sum<TEAM>(q);
        };
        float mean, q;
        if (TEAM) {
            mean = quotient(s, count, inv_count);
            q = deviations(mean);
        } else {
            // every warp's mean m_w and squared deviations from it; the sum of (d + m_w - m)^2 is that of d^2 and n_w (m_w - m)^2
            const float mw = s * inv_here;
            const float4* set = exchange.put(make_float4(s, deviations(mw), mw, here), at.t);
            s = q = 0.f;
            for (int u = 0; u < warps; ++u) s += set[u].x;
            mean = quotient(s, count, inv_count);
            for (int u = 0; u < warps; ++u) { const float4 f = set[u]; const float d = f.z - mean; q += fmaf(f.w * d, d, f.y); }
        }
        const float rstd = inverse_root(q * inv_count + a.eps);
        if (!live) continue;
        T* y = static_cast<T*>(a.out) + r * a.pout;
#pragma unroll
        for (int k = 0; k < ITEMS; ++k) {
            float w[V], b[V];
            weight.get(at.piece(k), w);
            bias.get(at.piece(k), b);
#pragma unroll
            for (int j = 0; j < V; ++j) v[k][j] = fmaf((v[k][j] - mean) * rstd, w[j], b[j]);
            store_piece<T, EDGES>(y, at.feature(k), n, packed, pack<T>(v[k]));
        }
        if (at.t == 0) {
            if (a.mean) a.mean[r] = mean;
            if (a.rstd) a.rstd[r] = rstd;
        }
    }
}

template <class T, int TEAM, int ITEMS, bool EDGES, bool TAIL>
__global__ void __launch_bounds__(ROW_BLOCK, row_blocks<T, true, ITEMS>()) row_team_vjp(const __grid_constant__ Args a, int warps, int teams) {
    grid_dependency_wait();
    extern __shared__ __align__(16) float shared[];
    constexpr int V = VEC<T>, STAGES = row_stages<T, true, TAIL, ITEMS>(), ARRAYS = TAIL ? 3 : 2;
    const RowPlace<T, TEAM, ITEMS, EDGES> at(a, warps, teams);
    Exchange exchange(shared, warps, at.team, at.t);
    float* room = shared + EXCHANGE_BYTES / 4;
    Ring<T, ARRAYS, ITEMS, STAGES, EDGES> ring(room);
    room += ARRAYS * ITEMS * STAGES * 4 * blockDim.x;
    const Mask mask(a);
    const int n = (int)a.features;
    const bool packed = a.aligned, added = TAIL && a.gsum;
    const float inv_count = 1.f / (float)n;
    auto fetch = [&](long long r, int stage) {
        if (r < a.outer) {
#pragma unroll
            for (int k = 0; k < ITEMS; ++k) {
                ring.fetch(stage, 0, k, a.x, a.px, r, at.feature(k), a);
                ring.fetch(stage, 1, k, a.res, a.pres, r, at.feature(k), a);
                if (added) ring.fetch(stage, 2, k, a.gsum, a.pgsum, r, at.feature(k), a);
            }
        }
        copies_commit();
    };
#pragma unroll
    for (int i = 0; i < STAGES - 1; ++i) fetch(at.row + i * at.rows_apart, i);
    float mean_next = 0.f, rstd_next = 0.f;
    if (at.row < a.outer) { mean_next = a.mean[at.row]; rstd_next = a.rstd[at.row]; }
    const Weights<T, TEAM, ITEMS, EDGES> weight(a.weight, a, 1.f, at, room);
    if (ITEMS > 1) __syncthreads();
    float gw[ITEMS][V], gb[ITEMS][V];
#pragma unroll
    for (int k = 0; k < ITEMS; ++k)
#pragma unroll
        for (int j = 0; j < V; ++j) gw[k][j] = gb[k][j] = 0.f;
    const long long lead = TEAM && TEAM < 32 ? (threadIdx.x & 31) / TEAM : 0;
    int stage = 0;
    for (long long r = at.row; r - lead < a.outer; r += at.rows_apart) {
        const bool live = !TEAM || TEAM == 32 || r < a.outer;
        fetch(r + (STAGES - 1) * at.rows_apart, stage == 0 ? STAGES - 1 : stage - 1);
        const float mean = mean_next, rstd = rstd_next;
        if (r + at.rows_apart < a.outer) { mean_next = a.mean[r + at.rows_apart]; rstd_next = a.rstd[r + at.rows_apart]; }
        copies_wait<STAGES - 1>();
        const int used = stage;
        stage = stage + 1 == STAGES ? 0 : stage + 1;
        float s1 = 0.f, s2 = 0.f;
#pragma unroll
        for (int k = 0; k < ITEMS; ++k) {
            const int c = at.feature(k);
            if (!live || !(whole<T, EDGES>(c, n) || partly<T, EDGES>(c, n))) continue;
            float g[V], v[V], w[V];
            take<T, EDGES>(ring.get(used, 0, k), c, n, g);
            take<T, EDGES>(ring.get(used, 1, k), c, n, v);
            weight.get(at.piece(k), w);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                // beyond the row g is 0
                const float h = (v[j] - mean) * rstd, d = g[j] * w[j];
                gw[k][j] = fmaf(g[j], h, gw[k][j]);
                gb[k][j] += g[j];
                s1 += d;
                s2 = fmaf(d, h, s2);
            }
        }
        s1 = lanes_sum<TEAM>(s1);
        s2 = lanes_sum<TEAM>(s2);
        if (!TEAM) {
            const float4* set = exchange.put(make_float4(s1, s2, 0.f, 0.f), at.t);
            s1 = s2 = 0.f;
            for (int u = 0; u < warps; ++u) { s1 += set[u].x; s2 += set[u].y; }
        }
        if (!live) continue;
        // rstd (g w - mean(g w) - h mean(g w h))
        const float c1 = -rstd * (s1 * inv_count), c2 = -rstd * (s2 * inv_count);
        T* out = static_cast<T*>(a.out) + r * a.pout;
        T* out2 = TAIL ? static_cast<T*>(a.out2) + r * a.pout2 : nullptr;
#pragma unroll
        for (int k = 0; k < ITEMS; ++k) {
            const int c = at.feature(k);
            float g[V], v[V], w[V];
            unpack(ring.get(used, 0, k), g);
            unpack(ring.get(used, 1, k), v);
            weight.get(at.piece(k), w);
#pragma unroll
            for (int j = 0; j < V; ++j) v[j] = fmaf((v[j] - mean) * rstd, c2, fmaf(g[j] * w[j], rstd, c1));
            if (TAIL) {
                if (added) {
                    unpack(ring.get(used, 2, k), g);
#pragma unroll
                    for (int j = 0; j < V; ++j) v[j] += g[j];
                }
                store_piece<T, EDGES>(out2, c, n, packed, pack<T>(v));
                if (a.dropping) {
#pragma unroll
                    for (int q = 0; q < V / 4; ++q) {
                        const uint4 words = mask.words((uint64_t)((r * n - at.phase) / 4) + (uint32_t)(at.piece(k) * (V / 4) + q));
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
