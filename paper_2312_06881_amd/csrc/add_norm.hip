// h = x_scale x + y_scale gate * drop(post(y)),  out = norm(h): a block's output joins the
// residual stream, and the next block's input is normed, in one pass over the rows; and the
// gradients.  Everything is memory traffic: each operand is read once, each result written
// once, and a row lives in registers between the sums over it.
//
// norm(v) = (v - mean) r w + b with r = 1 / sqrt(mean((v - mean)^2) + eps) (layer), or
// v r w + b with r = 1 / sqrt(mean(v^2) + eps) (rms).  Sums are fp32, the mean taken out
// before squaring.  out is the norm of the fp32 sum h, not of h as rounded to the stream's
// type: one rounding fewer, and no dependence of out on that type.
//
// Backward, with u = (h - mean) r and d = dout w:
//   g    = dh + r (d - mean(d) - u mean(d u))      (rms: without mean(d))
//   dx   = x_scale g
//   dz   = y_scale g gate, zero where dropped, else scaled;  dgate = sum y_scale g drop(z)
//   dy   = dz, or through the post norm as above with its own u and d = dz pw
//   dw   = sum dout u,  db = sum dout;  dpw = sum dz u_y,  dpb = sum dz
// The sums over rows are kept in registers over a workgroup's rows, written as fp32 partials
// and added by a second kernel in a fixed order, so results repeat bit by bit.
//
// A team of TPR threads takes a row, NV vectors of 8 columns a thread; up to 1024 columns a
// team is a wave, which needs no barrier.
#include "lm_internal.h"
#include "philox.h"
#include "row_io.h"

namespace dyad {

namespace {

struct Norm {
    AddNormPass p;
    DropArgs d;
    int n, octets, npad;
    int64_t rows_per_gate;       // M when there is one gate row, or none
    bool drop;
    // backward
    int64_t units, per_group;    // units of rows; those of one gate row
    int64_t unit_rows;           // rows of a gate row (or M), split into per_group units
    float *part[4];              // dw, db, dpw, dpb: [workgroups][npad]; null: not wanted
    float *gpart;                // [units][npad]
};

constexpr int threads_of(int tpr) { return tpr < 256 ? (tpr == 64 ? 256 : tpr) : tpr; }
constexpr int teams_of(int tpr) { return threads_of(tpr) / tpr; }

template <bool RAG>
__device__ __forceinline__ void load_param(const void *base, bool f32, int64_t row, int c, int n, float (&v)[8]) {
    if (f32) load_row<RAG>(static_cast<const float *>(base) + row * n, c, n, v);
    else load_row<RAG>(static_cast<const uint16_t *>(base) + row * n, c, n, v);
}

// Sums of a and b over a team, the same bits in each of its threads.
template <int TPR>
struct TeamSum {
    float2 *lds;     // [2][TPR / 64] for teams of several waves
    int parity;      // of the buffer: a wave is at most one sum ahead of another
    __device__ __forceinline__ void operator()(float &a, float &b) {
#pragma unroll
        for (int m = 32; m > 0; m >>= 1) {
            a += __shfl_xor(a, m);
            b += __shfl_xor(b, m);
        }
        if constexpr (TPR > 64) {
            float2 *buf = lds + parity * (TPR / 64);
            parity ^= 1;
            if ((threadIdx.x & 63) == 0) buf[threadIdx.x / 64] = make_float2(a, b);
            __syncthreads();
            a = b = 0.f;
#pragma unroll
            for (int w = 0; w < TPR / 64; ++w) {
                const float2 t = buf[w];
                a += t.x;
                b += t.y;
            }
        }
    }
};

// Mean (zero for rms) and 1 / deviation of a row held as v[NV][8].
template <int TPR, int NV>
__device__ __forceinline__ float2 row_stats(const float (&v)[NV][8], int kind, const Norm &a, int c0, TeamSum<TPR> &sum) {
    const float inv = 1.f / (float)a.n;
    float s = 0.f, unused = 0.f, mean = 0.f;
    if (kind == kNormLayer) {
#pragma unroll
        for (int q = 0; q < NV; ++q)
#pragma unroll
            for (int e = 0; e < 8; ++e) s += v[q][e];      // columns past n hold zero
        sum(s, unused);
        mean = s * inv;
    }
    s = 0.f;
#pragma unroll
    for (int q = 0; q < NV; ++q)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float t = v[q][e] - mean;
            s += c0 + q * 8 * TPR + e < a.n ? t * t : 0.f;
        }
    sum(s, unused);
    return make_float2(mean, 1.f / sqrtf(s * inv + a.p.eps));
}

template <class TS, class TB, int TPR, int NV, bool RAG>
__global__ void __launch_bounds__(threads_of(TPR)) add_norm_kernel(Norm a) {
    __shared__ float2 lds[TPR > 64 ? 2 * (TPR / 64) : 1];
    TeamSum<TPR> sum{lds, 0};
    const int lane = threadIdx.x % TPR, n = a.n, c0 = lane * 8;
    const bool pf32 = a.p.param_dtype == kF32;
    const uint64_t offset = a.drop ? drop_offset(a.d) : 0;
    for (int64_t row = (int64_t)blockIdx.x * teams_of(TPR) + threadIdx.x / TPR; row < a.p.M;
         row += (int64_t)gridDim.x * teams_of(TPR)) {
        float h[NV][8];
        const TS *xr = static_cast<const TS *>(a.p.x) + row * n;
        float x[NV][8];
#pragma unroll
        for (int q = 0; q < NV; ++q) load_row<RAG>(xr, c0 + q * 8 * TPR, n, x[q]);
        if (a.p.y) {
            const TB *yr = static_cast<const TB *>(a.p.y) + row * n;
#pragma unroll
            for (int q = 0; q < NV; ++q) load_row<RAG>(yr, c0 + q * 8 * TPR, n, h[q]);
            if (a.p.post != kNormNone) {
                const float2 st = row_stats<TPR, NV>(h, a.p.post, a, c0, sum);
                if (a.p.post_stats && lane == 0) reinterpret_cast<float2 *>(a.p.post_stats)[row] = st;
#pragma unroll
                for (int q = 0; q < NV; ++q) {
                    float w[8], b[8];
                    const int c = c0 + q * 8 * TPR;
#pragma unroll
                    for (int e = 0; e < 8; ++e) h[q][e] = (h[q][e] - st.x) * st.y;
                    if (a.p.pw) {
                        load_param<RAG>(a.p.pw, pf32, 0, c, n, w);
#pragma unroll
                        for (int e = 0; e < 8; ++e) h[q][e] *= w[e];
                    }
                    if (a.p.pb) {
                        load_param<RAG>(a.p.pb, pf32, 0, c, n, b);
#pragma unroll
                        for (int e = 0; e < 8; ++e) h[q][e] += b[e];
                    }
                }
            }
            const int64_t grow = a.p.gate && a.p.groups > 1 ? row / a.rows_per_gate : 0;
#pragma unroll
            for (int q = 0; q < NV; ++q) {
                const int c = c0 + q * 8 * TPR;
                if (a.drop && c < n)
                    apply_drop(h[q], keep_bits(philox(a.d.seed, offset, (uint64_t)(row * a.octets + (c >> 3))), a.d.thr),
                               a.d.scale);
                if (a.p.gate) {
                    float g[8];
                    load_param<RAG>(a.p.gate, pf32, grow, c, n, g);
#pragma unroll
                    for (int e = 0; e < 8; ++e) h[q][e] *= g[e];
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) h[q][e] = c + e < n ? fmaf(h[q][e], a.p.y_scale, x[q][e] * a.p.x_scale) : 0.f;
            }
        } else {
#pragma unroll
            for (int q = 0; q < NV; ++q)
#pragma unroll
                for (int e = 0; e < 8; ++e) h[q][e] = x[q][e] * a.p.x_scale;
        }
        if (a.p.h) {
            TS *hr = static_cast<TS *>(a.p.h) + row * n;
#pragma unroll
            for (int q = 0; q < NV; ++q) store_cols<RAG>(hr, c0 + q * 8 * TPR, n, h[q]);
        }
        if (a.p.norm == kNormNone) continue;
        const float2 st = row_stats<TPR, NV>(h, a.p.norm, a, c0, sum);
        if (a.p.stats && lane == 0) reinterpret_cast<float2 *>(a.p.stats)[row] = st;
        TB *o = static_cast<TB *>(a.p.out) + row * n;
#pragma unroll
        for (int q = 0; q < NV; ++q) {
            const int c = c0 + q * 8 * TPR;
            float w[8], b[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) h[q][e] = (h[q][e] - st.x) * st.y;
            if (a.p.w) {
                load_param<RAG>(a.p.w, pf32, 0, c, n, w);
#pragma unroll
                for (int e = 0; e < 8; ++e) h[q][e] *= w[e];
            }
            if (a.p.b) {
                load_param<RAG>(a.p.b, pf32, 0, c, n, b);
#pragma unroll
                for (int e = 0; e < 8; ++e) h[q][e] += b[e];
            }
            store_cols<RAG>(o, c, n, h[q]);
        }
    }
}

// The gradient through a norm: d[q][e] (already times the weight) becomes the gradient of the
// normed values, u being their unit form.
template <int TPR, int NV>
__device__ __forceinline__ void norm_grad(float (&d)[NV][8], const float (&u)[NV][8], float r, int kind, int n,
                                          TeamSum<TPR> &sum) {
    float s = 0.f, t = 0.f;
#pragma unroll
    for (int q = 0; q < NV; ++q)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            s += d[q][e];
            t = fmaf(d[q][e], u[q][e], t);
        }
    sum(s, t);
    const float inv = 1.f / (float)n;
    s = kind == kNormLayer ? s * inv : 0.f;
    t *= inv;
#pragma unroll
    for (int q = 0; q < NV; ++q)
#pragma unroll
        for (int e = 0; e < 8; ++e) d[q][e] = r * (d[q][e] - s - u[q][e] * t);
}

// A workgroup's sums of one kind over its teams, in team order, to dst [npad]; clears them.
template <int TPR, int NV>
__device__ __forceinline__ void flush(float (&acc)[NV][8], float *dst, int npad, float *buf) {
    const int lane = threadIdx.x % TPR, team = threadIdx.x / TPR;
    if constexpr (teams_of(TPR) > 1) {
        for (int t = 0; t < teams_of(TPR); ++t) {
            __syncthreads();
            if (t == team) {
#pragma unroll
                for (int q = 0; q < NV; ++q)
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        float *b = buf + (q * 8 + e) * TPR + lane;
                        if (t > 0) acc[q][e] += *b;
                        *b = acc[q][e];
                    }
            }
        }
    }
    if (team == teams_of(TPR) - 1) {
#pragma unroll
        for (int q = 0; q < NV; ++q) {
            const int c = (lane + q * TPR) * 8;
            if (c < npad) store8(dst + c, acc[q]);
        }
    }
#pragma unroll
    for (int q = 0; q < NV; ++q)
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[q][e] = 0.f;
}

template <class TS, class TB, int NV>
struct Row {
    Raw<TS> h[NV], dh[NV];
    Raw<TB> g[NV], y[NV];
    float2 st, ps;
};

// FULL: there is a post norm or a gate whose gradient is wanted.  h is read, or with x given
// formed again from x and y: as rounded to a bf16 stream it would put 2^-8 of each of its values
// into u, and so into dw (2.5e-3 off 64 bits in place of bf16's own 1.7e-3, or with fp32
// parameters 1.7e-3 in place of 1e-7).  16384 tokens of 768 in bf16: 37 us for the 151 MB of dh,
// dout, x, y, dx, dy (29 us at a large copy's rate); rows loaded one ahead and kept as they lie in
// memory, 71 us without.
template <class TS, class TB, int TPR, int NV, bool FULL, bool RAG>
__global__ void __launch_bounds__(threads_of(TPR)) add_norm_grad_kernel(Norm a) {
    __shared__ float2 lds[TPR > 64 ? 2 * (TPR / 64) : 1];
    __shared__ float buf[teams_of(TPR) > 1 ? NV * 8 * TPR : 1];
    TeamSum<TPR> sum{lds, 0};
    const int lane = threadIdx.x % TPR, team = threadIdx.x / TPR, n = a.n, c0 = lane * 8;
    const bool pf32 = a.p.param_dtype == kF32;
    const bool again = a.p.x != nullptr, reads_y = FULL || (again && a.p.y != nullptr && a.p.dout != nullptr);
    const uint64_t offset = a.drop ? drop_offset(a.d) : 0;
    const auto fetch = [&](int64_t row) __attribute__((always_inline)) {
        Row<TS, TB, NV> r;
#pragma unroll
        for (int q = 0; q < NV; ++q) {
            const int c = c0 + q * 8 * TPR;
            if (a.p.dout) {
                r.h[q] = load_raw<RAG>(static_cast<const TS *>(again ? a.p.x : a.p.h) + row * n, c, n);
                r.g[q] = load_raw<RAG>(static_cast<const TB *>(a.p.dout) + row * n, c, n);
            }
            if (reads_y) r.y[q] = load_raw<RAG>(static_cast<const TB *>(a.p.y) + row * n, c, n);
            if (a.p.dh) r.dh[q] = load_raw<RAG>(static_cast<const TS *>(a.p.dh) + row * n, c, n);
            else r.dh[q] = Raw<TS>{};
        }
        if (a.p.dout) r.st = reinterpret_cast<const float2 *>(a.p.stats)[row];
        if (FULL && a.p.post != kNormNone) r.ps = reinterpret_cast<const float2 *>(a.p.post_stats)[row];
        return r;
    };
    // the parameters stay in registers: loads return in order, so one in the loop would wait for
    // the next row's (8192 rows of 4096, post norm and gate: 163 us with such loads, 143 without).
    // Sixteen waves have 128 registers each and cannot: with a post norm they load rows and
    // parameters as they come to them and keep four of the sums in LDS, where each thread adds to
    // words of its own (4096 rows of 8192, fp32 stream, post norm and gate: 165 us, 3.7 TB/s).
    constexpr bool kKeep = TPR < 1024, kAhead = TPR < 1024 || !FULL, kLdsSums = TPR == 1024 && FULL && NV == 1;
    __shared__ f32x4_t lsum[kLdsSums ? 8 * TPR : 1];
    const auto param = [&](const void *base, int64_t row, float missing, int q, float (&v)[8]) __attribute__((always_inline)) {
        if (base) {
            load_param<RAG>(base, pf32, row, c0 + q * 8 * TPR, n, v);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = missing;
        }
    };
    float w[kKeep ? NV : 1][8], gate[kKeep ? NV : 1][8], pw[kKeep && FULL ? NV : 1][8], pb[kKeep && FULL ? NV : 1][8];
    if constexpr (kKeep) {
#pragma unroll
        for (int q = 0; q < NV; ++q) {
            param(a.p.w, 0, 1.f, q, w[q]);
            if constexpr (FULL) {
                param(a.p.pw, 0, 1.f, q, pw[q]);
                param(a.p.pb, 0, 0.f, q, pb[q]);
            }
            param(a.p.gate, 0, 1.f, q, gate[q]);
        }
    }
    // v times a parameter's eight columns (kept ones in t)
    const auto times = [&](float (&v)[8], const void *base, int64_t row, int q, const auto &kept) __attribute__((always_inline)) {
        float t[8];
        if constexpr (kKeep) {
#pragma unroll
            for (int e = 0; e < 8; ++e) t[e] = kept[q][e];
        } else {
            param(base, row, 1.f, q, t);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] *= t[e];
    };
    if constexpr (kLdsSums) {
#pragma unroll
        for (int k = 0; k < 8; ++k) lsum[k * TPR + lane] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    }
    // sum k (0 dw, 1 db, 2 dpw, 3 dpb) of eight columns
    const auto add = [&](int k, float (&acc)[8], const float (&v)[8]) __attribute__((always_inline)) {
        if constexpr (kLdsSums) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                f32x4_t t = lsum[(2 * k + h) * TPR + lane];
#pragma unroll
                for (int e = 0; e < 4; ++e) t[e] += v[4 * h + e];
                lsum[(2 * k + h) * TPR + lane] = t;
            }
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) acc[e] += v[e];
        }
    };
    int64_t gate_row = 0;
    float dw[NV][8] = {}, db[NV][8] = {};
    float dpw[FULL ? NV : 1][8] = {}, dpb[FULL ? NV : 1][8] = {}, dgate[FULL ? NV : 1][8] = {};
    const int64_t u1 = (int64_t)(blockIdx.x + 1) * a.units / gridDim.x;
    for (int64_t unit = (int64_t)blockIdx.x * a.units / gridDim.x; unit < u1; ++unit) {
        const int64_t group = unit / a.per_group, piece = unit - group * a.per_group;
        const int64_t first = group * a.unit_rows + piece * a.unit_rows / a.per_group;
        const int64_t last = group * a.unit_rows + (piece + 1) * a.unit_rows / a.per_group;
        // a row's operands are loaded while the row before it is worked on, and wait as they lie in memory
        Row<TS, TB, NV> next;
        if (first + team < last) next = fetch(first + team);
        for (int64_t row = first + team; row < last; row += teams_of(TPR)) {
            const Row<TS, TB, NV> cur = next;
            if constexpr (kAhead) next = fetch(row + teams_of(TPR) < last ? row + teams_of(TPR) : row);
            float g[NV][8], u[NV][8];
            uint32_t keep[NV];
            if (a.p.groups > 1 && row / a.rows_per_gate != gate_row) {
                gate_row = row / a.rows_per_gate;
                if constexpr (kKeep)
#pragma unroll
                    for (int q = 0; q < NV; ++q) param(a.p.gate, gate_row, 1.f, q, gate[q]);
            }
            if (a.drop) {
#pragma unroll
                for (int q = 0; q < NV; ++q) {
                    const int c = c0 + q * 8 * TPR;
                    keep[q] = c < n ? keep_bits(philox(a.d.seed, offset, (uint64_t)(row * a.octets + (c >> 3))), a.d.thr) : 0;
                }
            }
            const float2 ps = cur.ps;
            // y of eight columns, normed where there is a post norm, without and with its weights
            const auto unit_y = [&](int q, float (&z)[8]) __attribute__((always_inline)) {
                unpack8(cur.y[q], z);
                if (FULL && a.p.post != kNormNone) {
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        z[e] = c0 + q * 8 * TPR + (RAG ? e : 0) < n ? (z[e] - ps.x) * ps.y : 0.f;
                }
            };
            const auto post_y = [&](int q, float (&z)[8]) __attribute__((always_inline)) {
                unit_y(q, z);
                if constexpr (FULL) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        if constexpr (kKeep) z[e] = fmaf(z[e], pw[q][e], pb[q][e]);
                    }
                    if constexpr (!kKeep) {
                        float s[8], t[8];
                        param(a.p.pw, 0, 1.f, q, s);
                        param(a.p.pb, 0, 0.f, q, t);
#pragma unroll
                        for (int e = 0; e < 8; ++e) z[e] = fmaf(z[e], s[e], t[e]);
                    }
                }
            };
            if (a.p.dout) {
#pragma unroll
                for (int q = 0; q < NV; ++q) {
                    unpack8(cur.h[q], u[q]);
                    unpack8(cur.g[q], g[q]);
                }
            }
            if (a.p.dout) {
                const float2 st = cur.st;
#pragma unroll
                for (int q = 0; q < NV; ++q) {
                    if (again) {
#pragma unroll
                        for (int e = 0; e < 8; ++e) u[q][e] *= a.p.x_scale;
                        if (a.p.y) {
                            float z[8];
                            post_y(q, z);
                            if (a.drop) apply_drop(z, keep[q], a.d.scale);
                            times(z, a.p.gate, gate_row, q, gate);
#pragma unroll
                            for (int e = 0; e < 8; ++e) u[q][e] = fmaf(z[e], a.p.y_scale, u[q][e]);
                        }
                    }
#pragma unroll
                    for (int e = 0; e < 8; ++e) u[q][e] = (u[q][e] - st.x) * st.y;
                    float t[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) t[e] = g[q][e] * u[q][e];
                    add(0, dw[kLdsSums ? 0 : q], t);
                    add(1, db[kLdsSums ? 0 : q], g[q]);
                    times(g[q], a.p.w, 0, q, w);
                }
                norm_grad<TPR, NV>(g, u, st.y, a.p.norm, n, sum);
                if (a.p.dh) {
#pragma unroll
                    for (int q = 0; q < NV; ++q) {
                        float t[8];
                        unpack8(cur.dh[q], t);
#pragma unroll
                        for (int e = 0; e < 8; ++e) g[q][e] += t[e];
                    }
                }
            } else {
#pragma unroll
                for (int q = 0; q < NV; ++q) unpack8(cur.dh[q], g[q]);   // zero where there is none
            }
            if (a.p.dx) {
                TS *dx = static_cast<TS *>(a.p.dx) + row * n;
#pragma unroll
                for (int q = 0; q < NV; ++q) {
                    float t[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) t[e] = g[q][e] * a.p.x_scale;
                    store_cols<RAG>(dx, c0 + q * 8 * TPR, n, t);
                }
            }
            if (!FULL && !a.p.dy) continue;   // (only rows loaded ahead)
#pragma unroll
            for (int q = 0; q < NV; ++q) {
                const int c = c0 + q * 8 * TPR;
#pragma unroll
                for (int e = 0; e < 8; ++e) g[q][e] = c + (RAG ? e : 0) < n ? g[q][e] * a.p.y_scale : 0.f;
                if (a.drop) apply_drop(g[q], keep[q], a.d.scale);
                if constexpr (FULL) {
                    if (a.gpart) {
                        float z[8];
                        post_y(q, z);
                        // what is dropped counts for nothing, whatever it was
#pragma unroll
                        for (int e = 0; e < 8; ++e) dgate[q][e] += g[q][e] != 0.f ? g[q][e] * z[e] : 0.f;
                    }
                }
                times(g[q], a.p.gate, gate_row, q, gate);
                if constexpr (FULL) {
                    if (a.p.post != kNormNone) {
                        unit_y(q, u[q]);           // the stream's u has had its turn
                        float t[8];
#pragma unroll
                        for (int e = 0; e < 8; ++e) t[e] = g[q][e] * u[q][e];
                        add(2, dpw[kLdsSums ? 0 : q], t);
                        add(3, dpb[kLdsSums ? 0 : q], g[q]);
                        times(g[q], a.p.pw, 0, q, pw);
                    }
                }
            }
            if (FULL && a.p.post != kNormNone) norm_grad<TPR, NV>(g, u, ps.y, a.p.post, n, sum);
            if (a.p.dy) {
                TB *dy = static_cast<TB *>(a.p.dy) + row * n;
#pragma unroll
                for (int q = 0; q < NV; ++q) store_cols<RAG>(dy, c0 + q * 8 * TPR, n, g[q]);
            }
            if constexpr (!kAhead)
                if (row + teams_of(TPR) < last) next = fetch(row + teams_of(TPR));
        }
        if constexpr (FULL)
            if (a.gpart) flush<TPR, NV>(dgate, a.gpart + unit * a.npad, a.npad, buf);
    }
    if constexpr (kLdsSums) {
        const auto back = [&](int k, float (&acc)[8]) {
#pragma unroll
            for (int e = 0; e < 8; ++e) acc[e] = lsum[(2 * k + e / 4) * TPR + lane][e % 4];
        };
        back(0, dw[0]);
        back(1, db[0]);
        back(2, dpw[0]);
        back(3, dpb[0]);
    }
    if (a.part[0]) flush<TPR, NV>(dw, a.part[0] + (int64_t)blockIdx.x * a.npad, a.npad, buf);
    if (a.part[1]) flush<TPR, NV>(db, a.part[1] + (int64_t)blockIdx.x * a.npad, a.npad, buf);
    if constexpr (FULL) {
        if (a.part[2]) flush<TPR, NV>(dpw, a.part[2] + (int64_t)blockIdx.x * a.npad, a.npad, buf);
        if (a.part[3]) flush<TPR, NV>(dpb, a.part[3] + (int64_t)blockIdx.x * a.npad, a.npad, buf);
    }
}

// Sums over the partials of each vector, in a fixed order: 32 columns by 32 ranges of them.
struct Sums {
    const float *part[5];
    void *out[5];
    int64_t count[5], batch[5];   // partials of an output row; output rows
    int n, npad;
    bool f32;
};

__global__ void __launch_bounds__(1024) add_norm_sum_kernel(Sums s) {
    __shared__ float buf[32][33];
    const int k = blockIdx.z, col = threadIdx.x & 31, range = threadIdx.x >> 5;
    const int c = blockIdx.x * 32 + col;
    for (int64_t row = blockIdx.y; row < s.batch[k]; row += gridDim.y) {
        float t = 0.f;
        if (c < s.n)
#pragma unroll 8
            for (int64_t i = range; i < s.count[k]; i += 32) t += s.part[k][(row * s.count[k] + i) * s.npad + c];
        buf[range][col] = t;
        __syncthreads();
        if (range == 0 && c < s.n) {
            t = 0.f;
#pragma unroll
            for (int r = 0; r < 32; ++r) t += buf[r][col];
            if (s.f32) static_cast<float *>(s.out[k])[row * s.n + c] = t;
            else static_cast<uint16_t *>(s.out[k])[row * s.n + c] = f32_to_bf16(t);
        }
        __syncthreads();
    }
}

// Threads and vectors of a row.  Forward: a wave as far as 16 columns a thread go, then more
// waves.  In the backward pass the sums over rows share the registers with a row's operands, and
// a thread takes 8 columns.
struct Shape {
    int tpr, nv;
};
Shape shape_of(int64_t n, bool backward) {
    const int64_t per = backward ? 8 : 16;
    int tpr = 64;
    while (tpr < 1024 && tpr * per < n) tpr *= 2;
    return {tpr, tpr * 8 < n ? 2 : 1};
}

struct Plan {
    int64_t grid, units, per_group, unit_rows, npad;
    bool gate, full;
};

Plan plan_of(const AddNormPass &p) {
    Plan l;
    l.npad = (p.n + 7) / 8 * 8;
    l.gate = p.y && p.gate && p.dgate;
    l.full = p.y && (p.post != kNormNone || l.gate);
    const Shape sh = shape_of(p.n, true);
    const int64_t teams = teams_of(sh.tpr);
    // two rows a team at least, and no more workgroups than the GPU holds at once: 3 waves a
    // SIMD, or 2 with the sums of a post norm (rows loaded ahead, so more would not help; with
    // eight rows a team 3997 rows of 1001 took 93 us in place of 60)
    int64_t most = 1024 * (l.full ? 2 : 3) / (threads_of(sh.tpr) / 64);
    if (most < 256) most = 256;
    int64_t want = (p.M + 2 * teams - 1) / (2 * teams);
    if (want > most) want = most;
    if (want < 1) want = 1;
    const int64_t groups = l.gate ? p.groups : 1;
    l.unit_rows = p.M / groups;
    l.per_group = (want + groups - 1) / groups;
    if (l.per_group > l.unit_rows) l.per_group = l.unit_rows > 0 ? l.unit_rows : 1;
    l.units = groups * l.per_group;
    l.grid = l.units < want ? l.units : want;
    return l;
}

template <class TS, class TB, int TPR, int NV, bool RAG>
void run_fwd(const Norm &a, hipStream_t s) {
    const int64_t blocks = (a.p.M + teams_of(TPR) - 1) / teams_of(TPR);
    const unsigned grid = (unsigned)(blocks < 4096 ? blocks : 4096);
    add_norm_kernel<TS, TB, TPR, NV, RAG><<<grid, threads_of(TPR), 0, s>>>(a);
}

template <class TS, class TB, int TPR, int NV, bool RAG>
void run_bwd(const Norm &a, const Plan &l, hipStream_t s) {
    if (l.full) add_norm_grad_kernel<TS, TB, TPR, NV, true, RAG><<<(unsigned)l.grid, threads_of(TPR), 0, s>>>(a);
    else add_norm_grad_kernel<TS, TB, TPR, NV, false, RAG><<<(unsigned)l.grid, threads_of(TPR), 0, s>>>(a);
}

template <class TS, class TB, bool RAG>
hipError_t run(const Norm &a, const Plan *l, hipStream_t s) {
    const Shape sh = shape_of(a.n, l != nullptr);
    if (l) {
        switch (sh.tpr * sh.nv) {
        case 64: run_bwd<TS, TB, 64, 1, RAG>(a, *l, s); break;
        case 128: run_bwd<TS, TB, 128, 1, RAG>(a, *l, s); break;
        case 256: run_bwd<TS, TB, 256, 1, RAG>(a, *l, s); break;
        case 512: run_bwd<TS, TB, 512, 1, RAG>(a, *l, s); break;
        case 1024: run_bwd<TS, TB, 1024, 1, RAG>(a, *l, s); break;
        default: run_bwd<TS, TB, 1024, 2, RAG>(a, *l, s);
        }
    } else {
        switch (sh.tpr * sh.nv) {
        case 64: run_fwd<TS, TB, 64, 1, RAG>(a, s); break;
        case 128: run_fwd<TS, TB, 64, 2, RAG>(a, s); break;
        case 256: run_fwd<TS, TB, 128, 2, RAG>(a, s); break;
        case 512: run_fwd<TS, TB, 256, 2, RAG>(a, s); break;
        case 1024: run_fwd<TS, TB, 512, 2, RAG>(a, s); break;
        default: run_fwd<TS, TB, 1024, 2, RAG>(a, s);
        }
    }
    return hipGetLastError();
}

hipError_t run_types(const Norm &a, const Plan *l, hipStream_t s) {
    const bool rag = a.n % 8 != 0;
    if (a.p.stream_dtype == kBF16) return rag ? run<uint16_t, uint16_t, true>(a, l, s) : run<uint16_t, uint16_t, false>(a, l, s);
    if (a.p.dtype == kBF16) return rag ? run<float, uint16_t, true>(a, l, s) : run<float, uint16_t, false>(a, l, s);
    return rag ? run<float, float, true>(a, l, s) : run<float, float, false>(a, l, s);
}

Norm norm_of(const AddNormPass &p, const DropArgs &d) {
    Norm a{};
    a.p = p;
    a.d = d;
    a.n = (int)p.n;
    a.octets = (int)((p.n + 7) / 8);
    a.npad = a.octets * 8;
    a.rows_per_gate = p.M / p.groups;
    a.drop = p.y && d.thr > 0;
    return a;
}

}  // namespace

hipError_t launch_add_norm(const AddNormPass &p, const DropArgs &d, hipStream_t s) {
    return run_types(norm_of(p, d), nullptr, s);
}

// Partials of dw, db, dpw, dpb, then of the gate's gradient.
size_t add_norm_workspace(const AddNormPass &p) {
    const Plan l = plan_of(p);
    const int64_t vectors = (p.dw != nullptr) + (p.db != nullptr) + (p.dpw != nullptr) + (p.dpb != nullptr);
    return (size_t)((vectors * l.grid + (l.gate ? l.units : 0)) * l.npad) * sizeof(float);
}

hipError_t launch_add_norm_grad(const AddNormPass &p, const DropArgs &d, hipStream_t s) {
    const Plan l = plan_of(p);
    Norm a = norm_of(p, d);
    a.units = l.units;
    a.per_group = l.per_group;
    a.unit_rows = l.unit_rows;
    void *const out[5] = {p.dw, p.db, p.dpw, p.dpb, l.gate ? p.dgate : nullptr};
    Sums t{};
    t.n = a.n;
    t.npad = a.npad;
    t.f32 = p.param_dtype == kF32;
    int count = 0;
    int64_t rows = 1;
    float *at = static_cast<float *>(p.ws);
    for (int k = 0; k < 5; ++k) {
        if (!out[k]) continue;
        const bool gate = k == 4;
        (gate ? a.gpart : a.part[k]) = at;
        t.part[count] = at;
        t.out[count] = out[k];
        t.count[count] = gate ? l.per_group : l.grid;
        t.batch[count] = gate ? p.groups : 1;
        if (t.batch[count] > rows) rows = t.batch[count];
        at += (gate ? l.units : l.grid) * a.npad;
        ++count;
    }
    hipError_t e = run_types(a, &l, s);
    if (e != hipSuccess || count == 0) return e;
    if (rows > 4096) rows = 4096;
    add_norm_sum_kernel<<<dim3((unsigned)((a.n + 31) / 32), (unsigned)rows, (unsigned)count), 1024, 0, s>>>(t);
    return hipGetLastError();
}

}  // namespace dyad
