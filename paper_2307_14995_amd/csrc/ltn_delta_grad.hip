// Gated delta rule: the gradients of a chunk of 64 tokens and a head of keys (ltn_delta.h has the formulas), from Z, dY and
// the states that the sweeps left.  The value heads that share the keys follow one another in one workgroup: their dq and
// dk are summed in registers, in a fixed order.  Wave w owns tokens 16 w .. +15; the value features come in slabs of VS.
// Scales of rows and columns (decays, beta) are applied to products' fp32 results, never to an operand.
#include "ltn_delta.h"

namespace ltn {
namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ float sum16(float x) {          // over the 16 lanes of a row of results
#pragma unroll
    for (int d = 1; d < 16; d *= 2) x += __shfl_xor(x, d, 64);
    return x;
}
template <class T> __device__ __forceinline__ float dot8(const typename El<T>::F& a, const typename El<T>::F& b) {
    f32x4 a0, a1, b0, b1;
    values_of(a, a0, a1);
    values_of(b, b0, b1);
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) s = fmaf(a0[i], b0[i], fmaf(a1[i], b1[i], s));
    return s;
}

template <class T, int DK, int VS>
struct GradLds {
    static constexpr int LD = DK + El<T>::PAD, LT = kChunk + El<T>::PAD, LV = VS + El<T>::PAD;
    T K[kChunk * LD], Q[kChunk * LD];
    union {
        struct { T G[kChunk * LV], Z[VS * LT], Y[VS * LT], S[VS * LD], D[VS * LD]; } slab;
        struct { T dP[kChunk * LT], E[kChunk * LT]; } chunk;
    };
    double Gs[kChunk];
    float gam[kChunk], end[kChunk], beta[kChunk], row[kChunk], col[4][kChunk], part[4];
};

// rows (at most 64 of them hold data) of COLS elements, contiguous in memory
template <class T, int LD, int ROWS, int COLS>
__device__ __forceinline__ void load_rows(T* tile, const T* src, int tid) {
    constexpr int V = 16 / sizeof(T), PER = COLS / V;
    for (int i = tid; i < ROWS * PER; i += kThreads) {
        const int r = i / PER, c = i % PER * V;
        *(u32x4*)(tile + r * LD + c) = *(const u32x4*)(src + (size_t)r * COLS + c);
    }
}

template <class T, int DK, int VS>
__global__ __launch_bounds__(kThreads)
void delta_grad_kernel(DeltaArgs a, int Dv) {
    typedef GradLds<T, DK, VS> Lds;
    typedef typename El<T>::F F;
    constexpr int LD = Lds::LD, LT = Lds::LT, LV = Lds::LV, NT = DK / 16;
    __shared__ __attribute__((aligned(16))) char raw[sizeof(Lds)];
    Lds& l = *(Lds*)raw;
    const int hk = blockIdx.x % a.Hk, slot = blockIdx.x / a.Hk, group = a.H / a.Hk;
    DeltaSeq s;
    int chunk;
    if (!delta_find(a, slot, s, chunk)) return;
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, m = lane & 15, grp = lane >> 4;
    const int t0 = chunk * kChunk, rows = s.len - t0 < kChunk ? s.len - t0 : kChunk;
    const size_t key_row = ((size_t)s.row * a.Hk + hk) * a.N + s.first + t0;
    const f32x4 zero = {0.f, 0.f, 0.f, 0.f};

    load_tile<T, LD, DK, kThreads>(l.K, (const T*)a.k + key_row * DK, DK, rows, tid);
    load_tile<T, LD, DK, kThreads>(l.Q, (const T*)a.q + key_row * DK, DK, rows, tid);
    f32x4 dq[NT], dk[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) dq[t] = dk[t] = zero;

    for (int j = 0; j < group; ++j) {
        const int h = hk * group + j;
        const size_t val_row = ((size_t)s.row * a.H + h) * a.N + s.first + t0, at = (size_t)slot * a.H + h;
        if (w == 0) {
            double x = 0.0;
            if (lane < rows) {
                const float gl = a.g[val_row + lane];
                x = gl < -200.f ? -200.0 : (double)gl;                   // (as for T' and P)
            }
#pragma unroll
            for (int d = 1; d < 64; d *= 2) {
                const double y = __shfl_up(x, d, 64);
                if (lane >= d) x += y;
            }
            l.Gs[lane] = x;
            l.beta[lane] = lane < rows ? a.beta[val_row + lane] : 0.f;
            l.gam[lane] = a.vec[at * 3 * kChunk + lane];
            l.end[lane] = a.vec[at * 3 * kChunk + kChunk + lane];
        }
        f32x4 dP[4], E[4], qs[NT], ks[NT], ke[NT];
#pragma unroll
        for (int ct = 0; ct < 4; ++ct) dP[ct] = E[ct] = zero;
#pragma unroll
        for (int t = 0; t < NT; ++t) qs[t] = ks[t] = ke[t] = zero;
        float sdot = 0.f, db = 0.f;
        for (int v0 = 0; v0 < Dv; v0 += VS) {
            __syncthreads();               // (the tiles' last readers are done; the first time: K, Q and the gates are there)
            load_tile<T, LV, VS, kThreads>(l.slab.G, (const T*)a.d_o + val_row * Dv + v0, Dv, rows, tid);
            load_rows<T, LT, VS, kChunk>(l.slab.Z, (const T*)a.z + (at * Dv + v0) * kChunk, tid);
            load_rows<T, LT, VS, kChunk>(l.slab.Y, (const T*)a.dy + (at * Dv + v0) * kChunk, tid);
            load_rows<T, LD, VS, DK>(l.slab.S, (const T*)a.s0 + (at * Dv + v0) * DK, tid);
            load_rows<T, LD, VS, DK>(l.slab.D, (const T*)a.ds + (at * Dv + v0) * DK, tid);
            __syncthreads();
            for (int i = tid; i < VS * DK / 8; i += kThreads) {
                const int o = i / (DK / 8) * LD + i % (DK / 8) * 8;
                sdot += dot8<T>(*(const F*)(l.slab.S + o), *(const F*)(l.slab.D + o));
            }
#pragma unroll
            for (int kb = 0; kb < VS / 32; ++kb) {
                const F g = row_frag_p<T, LV>(l.slab.G, 16 * w + m, kb, lane);
                const F y = col_frag_p<LT>(l.slab.Y, kb, w, lane);
                const F z = col_frag_p<LT>(l.slab.Z, kb, w, lane);
                db += dot8<T>(y, z);
                if (16 * w + m < rows) {
                    f32x4 y0, y1;
                    values_of(y, y0, y1);
                    const float b = l.beta[16 * w + m];
                    *(F*)((T*)a.dv + (val_row + 16 * w + m) * Dv + v0 + 32 * kb + 8 * grp) = frag_of<T>(b * y0, b * y1);
                }
#pragma unroll
                for (int ct = 0; ct < 4; ++ct) {
                    if (ct > w) continue;
                    const F b = col_frag_p<LT>(l.slab.Z, kb, ct, lane);
                    dP[ct] = mma(g, b, dP[ct]);
                    E[ct] = mma(y, b, E[ct]);
                }
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    const F b = col_frag_p<LD>(l.slab.S, kb, t, lane), d = col_frag_p<LD>(l.slab.D, kb, t, lane);
                    qs[t] = mma(g, b, qs[t]);
                    ks[t] = mma(y, b, ks[t]);
                    ke[t] = mma(z, d, ke[t]);
                }
            }
        }
        db += __shfl_xor(db, 16, 64);
        db += __shfl_xor(db, 32, 64);
        if (grp == 0 && 16 * w + m < rows) ((T*)a.dbeta)[val_row + 16 * w + m] = (T)db;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) sdot += __shfl_xor(sdot, d, 64);
        if (lane == 0) l.part[w] = sdot;
        __syncthreads();                   // the slab is read: dP and E take its place

        const f32x4 gam = *(const f32x4*)(l.gam + 16 * w + 4 * grp), end = *(const f32x4*)(l.end + 16 * w + 4 * grp),
                    beta = *(const f32x4*)(l.beta + 16 * w + 4 * grp);
        f32x4 sum = zero, ends = zero;     // of the lane's four rows
#pragma unroll
        for (int ct = 0; ct < 4; ++ct) {
            const int c = 16 * ct + m;
            f32x4 kk = zero, qk = zero;
            if (ct <= w) {
#pragma unroll
                for (int kb = 0; kb < DK / 32; ++kb) {
                    const F b = row_frag_p<T, LD>(l.K, c, kb, lane);
                    kk = mma(row_frag_p<T, LD>(l.K, 16 * w + m, kb, lane), b, kk);
                    qk = mma(row_frag_p<T, LD>(l.Q, 16 * w + m, kb, lane), b, qk);
                }
            }
            const double gc = l.Gs[c];
            const float bc = l.beta[c];
            float down = 0.f;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int r = 16 * w + 4 * grp + i;
                const float ratio = expf((float)(l.Gs[r] - gc)) * bc;
                const float p = r >= c ? a.scale * ratio * dP[ct][i] : 0.f, e = r > c ? -ratio * beta[i] * E[ct][i] : 0.f;
                const float both = (r >= c ? p * qk[i] : 0.f) + (r > c ? e * kk[i] : 0.f);
                sum[i] += both;
                down += both;
                l.chunk.dP[r * LT + c] = (T)p;
                l.chunk.E[r * LT + c] = (T)e;
            }
            down += __shfl_xor(down, 16, 64);
            down += __shfl_xor(down, 32, 64);
            if (grp == 0) l.col[w][c] = down;
        }
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            qs[t] *= a.scale * gam;
            ks[t] *= -gam * beta;
            ke[t] *= end * beta;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int o = (16 * w + 4 * grp + i) * LD + 16 * t + m;
                const float kv = (float)l.K[o], e = kv * ke[t][i];
                sum[i] += (float)l.Q[o] * qs[t][i] + kv * ks[t][i] - e;
                ends[i] += e;
            }
        }
        float last = ends[0] + ends[1] + ends[2] + ends[3];
#pragma unroll
        for (int d = 1; d < 64; d *= 2) last += __shfl_xor(last, d, 64);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float x = sum16(sum[i]);
            if (m == 0) l.row[16 * w + 4 * grp + i] = x;
        }
        if (lane == 0) l.part[w] = l.gam[kChunk - 1] * l.part[w] + last;
        __syncthreads();
        if (w == 0) {
            float x = l.row[lane] - (l.col[0][lane] + l.col[1][lane] + l.col[2][lane] + l.col[3][lane]);
            if (lane == 63) x += l.part[0] + l.part[1] + l.part[2] + l.part[3];
#pragma unroll
            for (int d = 1; d < 64; d *= 2) {
                const float y = __shfl_down(x, d, 64);
                if (lane + d < 64) x += y;
            }
            if (lane < rows) ((T*)a.dg)[val_row + lane] = (T)x;
        }
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            f32x4 x = dq[t] + qs[t], y = dk[t] + ks[t] + ke[t];
#pragma unroll
            for (int kb = 0; kb < 2; ++kb) {
                const F kf = col_frag_p<LD>(l.K, kb, t, lane);
                if (kb <= w / 2) {
                    x = mma(row_frag_p<T, LT>(l.chunk.dP, 16 * w + m, kb, lane), kf, x);
                    y = mma(row_frag_p<T, LT>(l.chunk.E, 16 * w + m, kb, lane), kf, y);
                }
                if (kb >= w / 2) {
                    y = mma(col_frag_p<LT>(l.chunk.dP, kb, w, lane), col_frag_p<LD>(l.Q, kb, t, lane), y);
                    y = mma(col_frag_p<LT>(l.chunk.E, kb, w, lane), kf, y);
                }
            }
            dq[t] = x;
            dk[t] = y;
        }
        __syncthreads();                   // dP, E and the sums are read: the next head's take their place
    }
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = 16 * w + 4 * grp + i;
            if (r < rows) {
                ((T*)a.dq)[(key_row + r) * DK + 16 * t + m] = (T)dq[t][i];
                ((T*)a.dk)[(key_row + r) * DK + 16 * t + m] = (T)dk[t][i];
            }
        }
}

template <class T, int DK, int VS>
hipError_t launch_t(const DeltaArgs& a, int Dv, hipStream_t stream) {
    static_assert(sizeof(GradLds<T, DK, VS>) <= 160 * 1024, "LDS");
    hipLaunchKernelGGL((delta_grad_kernel<T, DK, VS>), dim3((unsigned)((long long)a.slots * a.Hk)), dim3(kThreads), 0, stream, a, Dv);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_delta_grad(const DeltaArgs& a, int Dk, int Dv, int is_bf16, hipStream_t stream) {
    if (Dk == 64) return is_bf16 ? launch_t<__bf16, 64, 64>(a, Dv, stream) : launch_t<float, 64, 32>(a, Dv, stream);
    return is_bf16 ? launch_t<__bf16, 128, 64>(a, Dv, stream) : launch_t<float, 128, 32>(a, Dv, stream);
}

}  // namespace ltn
