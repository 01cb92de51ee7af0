// The norm behind a block, its gate, the residual scale and sum, and the norm before the next block, on rows of C features
// (arXiv 2307.14995, Sec. 3.1.3: SimpleRMSNorm; with weights where given):
//
//     n = y / sqrt(mean(y^2) + eps)      z = n (.) w_after      x' = x + s gate (.) z
//     m = x' / sqrt(mean(x'^2) + eps)    h = m (.) w_before
//
// and its derivative, with dx', dh coming in (x' is formed again: the backward needs x and y, nothing that was saved):
//
//     dm = dh (.) w_before      dx = dx' + (dm - m mean(dm (.) m)) / sqrt(mean(x'^2) + eps)
//     dn = s gate (.) dx (.) w_after      dy = (dn - n mean(dn (.) n)) / sqrt(mean(y^2) + eps)
//     dgate = s dx (.) z      dw_after = sum over rows of s gate (.) dx (.) n      dw_before = sum over rows of dh (.) m
//
// Streaming kernels, bound by memory: a row is read once into the registers of one to eight waves, EL features a lane,
// in pieces of 16 bytes; the means meet by lane swaps and, where a row has several waves, through LDS.  A team of waves
// takes consecutive rows (its "strip") and keeps the weights, and the sums of their derivatives, in registers.  The
// strips' sums go through memory and are added in a fixed order by a second kernel: no atomics, the same bits every run.
// The next row is on its way while one is worked on.  32768 rows of 4096, bf16, with both weights: forward 204 us, backward 320
// (5.26 and 5.03 TB/s of their tensors) and 5 for the sums.
#include "ltn_bf16_tiles.h"

namespace ltn {
namespace {

template <class T> struct Piece;           // 16 bytes as fp32
template <> struct Piece<__bf16> {
    static constexpr int N = 8;
    static __device__ __forceinline__ void load(const __bf16* p, float* v) {
        const f32x8 f = __builtin_convertvector(*(const bf16x8*)p, f32x8);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = f[i];
    }
    static __device__ __forceinline__ void store(__bf16* p, const float* v) {
        f32x8 f;
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = v[i];
        *(bf16x8*)p = __builtin_convertvector(f, bf16x8);
    }
};
template <> struct Piece<float> {
    static constexpr int N = 4;
    static __device__ __forceinline__ void load(const float* p, float* v) {
        const f32x4 f = *(const f32x4*)p;
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = f[i];
    }
    static __device__ __forceinline__ void store(float* p, const float* v) { *(f32x4*)p = f32x4{v[0], v[1], v[2], v[3]}; }
};

enum { kNoGate = 0, kElementGate = 1, kSharedGate = 2 };

// A row's pieces of a lane as they come from memory, and as fp32.
template <class T, int NP> struct Raw { u32x4 v[NP]; };
template <class T, int NP> __device__ __forceinline__ void widen(const Raw<T, NP>& r, float* v) {
#pragma unroll
    for (int i = 0; i < NP; ++i) {
        if constexpr (sizeof(T) == 2) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                v[8 * i + 2 * j] = __uint_as_float(r.v[i][j] << 16);
                v[8 * i + 2 * j + 1] = __uint_as_float(r.v[i][j] & 0xffff0000u);
            }
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) v[4 * i + j] = __uint_as_float(r.v[i][j]);
        }
    }
}

// One team of WPR waves per row.  The lane's piece i of a row begins at column at(i); live(i): it is within the row.
template <class T, int EL, int WPR, int GATE>
struct Row {
    static constexpr int N = Piece<T>::N, NP = EL / N, TEAM = 64 * WPR;
    int pos, C;
    __device__ __forceinline__ int at(int i) const { return (i * TEAM + pos) * N; }
    __device__ __forceinline__ bool live(int i) const { return at(i) < C; }
    template <class U> __device__ __forceinline__ void load(const U* p, float* v, float other) const {
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            if (live(i)) {
                if constexpr (sizeof(U) == sizeof(T)) {
                    Piece<U>::load(p + at(i), v + i * N);
                } else {
#pragma unroll
                    for (int j = 0; j < N; j += 4) Piece<U>::load(p + at(i) + j, v + i * N + j);
                }
            } else {
#pragma unroll
                for (int j = 0; j < N; ++j) v[i * N + j] = other;
            }
        }
    }
    __device__ __forceinline__ void fetch(const T* p, Raw<T, NP>& r) const {               // (zeros behind the row)
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            r.v[i] = u32x4{0, 0, 0, 0};
            if (live(i)) r.v[i] = *(const u32x4*)(p + at(i));
        }
    }
    template <class U> __device__ __forceinline__ void store(U* p, const float* v) const {
#pragma unroll
        for (int i = 0; i < NP; ++i)
            if (live(i)) {
                if constexpr (sizeof(U) == sizeof(T)) {
                    Piece<U>::store(p + at(i), v + i * N);
                } else {
#pragma unroll
                    for (int j = 0; j < N; j += 4) Piece<U>::store(p + at(i) + j, v + i * N + j);
                }
            }
    }
};

// Sums of K values over a team.  `meet`: LDS of the workgroup's teams; a call's and the next one's halves alternate, so one
// barrier a call is enough.
template <int K, int WPR>
__device__ __forceinline__ void team_sum(float (&x)[K], float* meet, int& turn, int wave) {
#pragma unroll
    for (int d = 1; d < 64; d *= 2)
#pragma unroll
        for (int i = 0; i < K; ++i) x[i] += __shfl_xor(x[i], d, 64);
    if constexpr (WPR > 1) {
        float* const at = meet + turn * 16;
        turn ^= 1;
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int i = 0; i < K; ++i) at[wave * 2 + i] = x[i];
        __syncthreads();
        const int first = wave / WPR * WPR;
#pragma unroll
        for (int i = 0; i < K; ++i) {
            x[i] = 0.f;
#pragma unroll
            for (int j = 0; j < WPR; ++j) x[i] += at[(first + j) * 2 + i];
        }
    }
}

struct NormArgs {
    const void *x, *y, *gate, *d_x_out, *d_h;
    const float *w_after, *w_before;
    void *x_out, *h, *d_x, *d_y, *d_gate;
    float scale, eps;
    int after, C;
    long long rows, strip, per_gate;       // rows of a strip; rows that share a gate
    float* part;                           // [workgroups][dw_after, dw_before][C]
    float* gate_part;                      // [strips][a gate that began before, one that goes on after][C]
};

constexpr int kThreads(int wpr) { return wpr == 8 ? 512 : 256; }

template <class T, int EL, int WPR, int GATE, bool BWD>
__global__ __launch_bounds__(kThreads(WPR))
void block_norm_kernel(NormArgs a) {
    typedef Row<T, EL, WPR, GATE> R;
    constexpr int TEAMS = kThreads(WPR) / R::TEAM;
    __shared__ float meet[32];
    int turn = 0;
    const int wave = threadIdx.x / 64, team = threadIdx.x / R::TEAM;
    const R r = {(int)threadIdx.x % R::TEAM, a.C};
    const long long strip = (long long)blockIdx.x * TEAMS + team, first = strip * a.strip;
    const float inv = 1.f / a.C;
    float wa[EL], wb[EL];
#pragma unroll
    for (int i = 0; i < EL; ++i) wa[i] = wb[i] = 1.f;
    if (a.w_after) r.load(a.w_after, wa, 1.f);
    if (a.w_before) r.load(a.w_before, wb, 1.f);
    float da[BWD ? EL : 1], db[BWD ? EL : 1], dg[BWD && GATE == kSharedGate ? EL : 1];
    if constexpr (BWD) {
#pragma unroll
        for (int i = 0; i < EL; ++i) da[i] = db[i] = 0.f;
        if constexpr (GATE == kSharedGate)
#pragma unroll
            for (int i = 0; i < EL; ++i) dg[i] = 0.f;
    }
    // every team of the workgroup runs the same number of rows: those past the end are not there, but meet at the barriers.
    // The next row is fetched while one is worked on: two waves a SIMD, all that the sums' registers leave, would else
    // have nothing under way half of the time (norm of 32768 x 4096 backward 516 us without).
    const long long wg_first = (long long)blockIdx.x * TEAMS * a.strip;
    const long long steps = a.rows - wg_first < a.strip ? a.rows - wg_first : a.strip;
    Raw<T, R::NP> rx, ry_, rg, rdx, rdh;
    auto fetch = [&](long long n) {
        const long long row = first + n < a.rows ? first + n : a.rows - 1;
        const size_t off = (size_t)row * a.C;
        r.fetch((const T*)a.x + off, rx);
        r.fetch((const T*)a.y + off, ry_);
        if constexpr (GATE == kElementGate) r.fetch((const T*)a.gate + off, rg);
        if constexpr (GATE == kSharedGate) r.fetch((const T*)a.gate + (size_t)(row / a.per_gate) * a.C, rg);
        if constexpr (BWD) {
            if (a.d_x_out) r.fetch((const T*)a.d_x_out + off, rdx);
            r.fetch((const T*)a.d_h + off, rdh);
        }
    };
    if constexpr (BWD)
        if (!a.d_x_out)
#pragma unroll
            for (int i = 0; i < R::NP; ++i) rdx.v[i] = u32x4{0, 0, 0, 0};
    if (steps > 0) fetch(0);
    for (long long n = 0; n < steps; ++n) {
        const long long row = first + n;
        const bool there = row < a.rows;
        const size_t off = (size_t)(there ? row : a.rows - 1) * a.C;
        float x[EL], y[EL], g[GATE ? EL : 1];
        widen(rx, x);
        widen(ry_, y);
        if constexpr (GATE) widen(rg, g);
        float dxo[BWD ? EL : 1], dh[BWD ? EL : 1];
        if constexpr (BWD) {
            widen(rdx, dxo);
            widen(rdh, dh);
        }
        if (n + 1 < steps) fetch(n + 1);
        float ry = 1.f;
        if (a.after) {
            float ss[1] = {0.f};
#pragma unroll
            for (int i = 0; i < EL; ++i) ss[0] = fmaf(y[i], y[i], ss[0]);
            team_sum<1, WPR>(ss, meet, turn, wave);
            ry = 1.f / sqrtf(ss[0] * inv + a.eps);
        }
        float s2[2] = {0.f, 0.f};
#pragma unroll
        for (int i = 0; i < EL; ++i) {
            y[i] *= ry;                                                  // n
            x[i] = fmaf(a.scale * (GATE ? g[i] : 1.f), y[i] * wa[i], x[i]);
            s2[0] = fmaf(x[i], x[i], s2[0]);
            if constexpr (BWD) s2[1] = fmaf(dh[i] * wb[i], x[i], s2[1]);
        }
        team_sum<BWD ? 2 : 1, WPR>(*(float(*)[BWD ? 2 : 1])s2, meet, turn, wave);
        const float rs = 1.f / sqrtf(s2[0] * inv + a.eps);
        if constexpr (!BWD) {
            if (there) {
                r.store((T*)a.x_out + off, x);
#pragma unroll
                for (int i = 0; i < EL; ++i) x[i] *= rs * wb[i];
                r.store((T*)a.h + off, x);
            }
        } else {
            const float c1 = s2[1] * rs * inv;
            float s3[1] = {0.f};
#pragma unroll
            for (int i = 0; i < EL; ++i) {
                const float mi = x[i] * rs;
                if (there) db[i] = fmaf(dh[i], mi, db[i]);
                x[i] = dxo[i] + (dh[i] * wb[i] - mi * c1) * rs;          // dx
                const float dz = a.scale * (GATE ? g[i] : 1.f) * x[i];
                if (there) da[i] = fmaf(dz, y[i], da[i]);
                if constexpr (GATE) g[i] = a.scale * x[i] * y[i] * wa[i];                // dgate
                dh[i] = dz * wa[i];                                      // dn
                s3[0] = fmaf(dh[i], y[i], s3[0]);
            }
            if (there) r.store((T*)a.d_x + off, x);
            if (a.after) {
                team_sum<1, WPR>(s3, meet, turn, wave);
                const float c2 = s3[0] * inv;
#pragma unroll
                for (int i = 0; i < EL; ++i) dh[i] = (dh[i] - y[i] * c2) * ry;
            }
            if (there) {
                r.store((T*)a.d_y + off, dh);
                if constexpr (GATE == kElementGate) r.store((T*)a.d_gate + off, g);
            }
            if constexpr (GATE == kSharedGate) {
                if (there) {
#pragma unroll
                    for (int i = 0; i < EL; ++i) dg[i] += g[i];
                    const long long gate = row / a.per_gate, begin = gate * a.per_gate, end = begin + a.per_gate;
                    const bool last = row + 1 == end;
                    if (last || n + 1 == a.strip) {                      // the gate's rows in this strip are done
                        if (begin >= first && last) r.store((T*)a.d_gate + (size_t)gate * a.C, dg);
                        else r.store(a.gate_part + ((size_t)strip * 2 + (begin < first ? 0 : 1)) * a.C, dg);
#pragma unroll
                        for (int i = 0; i < EL; ++i) dg[i] = 0.f;
                    }
                }
            }
        }
    }
    if constexpr (BWD) {                   // the teams' sums of the weights, added in LDS: one row of them a workgroup
        float* const part = a.part + (size_t)blockIdx.x * 2 * a.C;
        if constexpr (TEAMS == 1) {
            if (a.w_after) r.store(part, da);
            if (a.w_before) r.store(part + a.C, db);
        } else {
            __shared__ __attribute__((aligned(16))) float sums[TEAMS][EL * R::TEAM];
#pragma unroll
            for (int which = 0; which < 2; ++which) {
                if (which == 0 ? !a.w_after : !a.w_before) continue;
                __syncthreads();
                r.store(sums[team], which == 0 ? da : db);
                __syncthreads();
                for (int c = threadIdx.x; c < a.C; c += kThreads(WPR)) {
                    float sum = sums[0][c];
#pragma unroll
                    for (int t = 1; t < TEAMS; ++t) sum += sums[t][c];
                    part[(size_t)which * a.C + c] = sum;
                }
            }
        }
    }
}

// What workgroups and strips left, summed: blockIdx.y 0 and 1 the weights (if wanted), from 2 on the gates that no strip
// holds whole.  32 columns a workgroup, 32 threads a column, each taking every 32nd row of sums; then in the threads' order.
template <class T>
__global__ __launch_bounds__(1024)
void block_norm_sum_kernel(const float* __restrict__ part, const float* __restrict__ gate_part, float* __restrict__ dwa,
                           float* __restrict__ dwb, T* __restrict__ d_gate, long long rows, long long strip, long long per_gate,
                           long long wgs, int C) {
    __shared__ float sums[32][33];
    const int cx = threadIdx.x & 31, sy = threadIdx.x >> 5, c = blockIdx.x * 32 + cx;
    for (long long which = blockIdx.y; which < 2 + (d_gate ? rows / per_gate : 0); which += gridDim.y) {
        long long s0 = 0, s1 = wgs, begin = 0;
        if (which >= 2) {
            begin = (which - 2) * per_gate;
            s0 = begin / strip;
            s1 = (begin + per_gate - 1) / strip + 1;
            if (s1 == s0 + 1) continue;    // (written by its strip)
        } else if (which == 0 ? !dwa : !dwb) {
            continue;
        }
        float sum = 0.f;
        if (c < C)
#pragma unroll 4
            for (long long s = s0 + sy; s < s1; s += 32)
                sum += which < 2 ? part[((size_t)s * 2 + which) * C + c] : gate_part[((size_t)s * 2 + (begin < s * strip ? 0 : 1)) * C + c];
        sums[sy][cx] = sum;
        __syncthreads();
        if (sy == 0 && c < C) {
#pragma unroll
            for (int i = 1; i < 32; ++i) sum += sums[i][cx];
            if (which >= 2) d_gate[(size_t)(which - 2) * C + c] = (T)sum;
            else (which == 0 ? dwa : dwb)[c] = sum;
        }
        __syncthreads();
    }
}

// Waves of a row: the fewest that hold it at 16 features a lane (8 up to 512 columns, which leaves no lane idle: 65536 rows of
// 512, bf16, 45 us forward and 85 backward, at 16 a lane 47 and 101).  At 8 a lane and twice the waves: 32768 rows of 4096
// 221 us forward for 216, 317 backward for 327; 16384 of 2048 42.5 for 42.4 and 87 for 84.
int waves_of(int C) { return C <= 1024 ? 1 : C <= 2048 ? 2 : C <= 4096 ? 4 : 8; }

template <class T, int EL, int WPR, int GATE>
hipError_t launch_t(const NormArgs& a, bool bwd, hipStream_t stream) {
    constexpr int TEAMS = kThreads(WPR) / (64 * WPR);
    const long long strips = (a.rows + a.strip - 1) / a.strip, wgs = (strips + TEAMS - 1) / TEAMS;
    if (bwd) hipLaunchKernelGGL((block_norm_kernel<T, EL, WPR, GATE, true>), dim3((unsigned)wgs), dim3(kThreads(WPR)), 0, stream, a);
    else hipLaunchKernelGGL((block_norm_kernel<T, EL, WPR, GATE, false>), dim3((unsigned)wgs), dim3(kThreads(WPR)), 0, stream, a);
    return hipGetLastError();
}
template <class T, int GATE>
hipError_t launch_c(const NormArgs& a, bool bwd, hipStream_t stream) {
    if (a.C <= 512) return launch_t<T, 8, 1, GATE>(a, bwd, stream);
    switch (waves_of(a.C)) {
        case 1: return launch_t<T, 16, 1, GATE>(a, bwd, stream);
        case 2: return launch_t<T, 16, 2, GATE>(a, bwd, stream);
        case 4: return launch_t<T, 16, 4, GATE>(a, bwd, stream);
        default: return launch_t<T, 16, 8, GATE>(a, bwd, stream);
    }
}

// Rows of a strip, and what the strips leave.  Forward: up to 4096 workgroups, a strip only to read the weights once (40000
// rows of 2048, bf16: 131 us with 512, 135 with 1024, 127; 16384 of 8192: 211, 212, 201).  Backward: each workgroup leaves
// a row of sums, and two a unit are all that the registers allow: 512 (16384 rows of 1152: 52 us, with 256 79, with 1024
// 56), but 256 for rows of eight waves (3000 of 8192: 61 us, 73 with 512) and for many of four (16384 of 4096: 165 us, 171
// with 512; 3000: 37 and 33).
int teams_of(int C) { return waves_of(C) == 8 ? 1 : 4 / waves_of(C); }
long long strip_rows(long long rows, int C, bool bwd) {
    const bool few = waves_of(C) == 8 || (waves_of(C) == 4 && rows >= 16384);
    const long long most = (bwd ? (few ? 256 : 512) : 4096) * teams_of(C), strip = (rows + most - 1) / most;
    return strip ? strip : 1;
}
long long workgroups(long long rows, int C, bool bwd) {
    const long long strip = strip_rows(rows, C, bwd), strips = (rows + strip - 1) / strip;
    return (strips + teams_of(C) - 1) / teams_of(C);
}

}  // namespace

size_t block_norm_part_floats(long long rows, int C) {
    const long long wgs = workgroups(rows, C, true);
    return (size_t)wgs * (2 + 2 * teams_of(C)) * C;
}

hipError_t launch_block_norm(const void* x, const void* y, const void* gate, const float* w_after, const float* w_before,
                             const void* d_x_out, const void* d_h, void* o0, void* o1, void* d_gate, float* dwa, float* dwb,
                             float* part, float scale, float eps, int after, long long rows, long long gates, int C,
                             int is_bf16, int is_bwd, hipStream_t stream) {
    if (rows <= 0) {                       // sums over no rows
        if (!is_bwd) return hipSuccess;
        hipError_t e = hipSuccess;
        for (float* w : {dwa, dwb})
            if (w && e == hipSuccess) e = launch_state_copy(nullptr, w, C, stream);
        if (d_gate && e == hipSuccess) e = launch_state_copy(nullptr, (float*)d_gate, (size_t)gates * C / (is_bf16 ? 2 : 1), stream);
        return e;
    }
    NormArgs a = {};
    a.x = x;
    a.y = y;
    a.gate = gate;
    a.w_after = after ? w_after : nullptr;
    a.w_before = w_before;
    a.d_x_out = d_x_out;
    a.d_h = d_h;
    a.x_out = a.d_x = o0;
    a.h = a.d_y = o1;
    a.d_gate = d_gate;
    a.scale = scale;
    a.eps = eps;
    a.after = after;
    a.C = C;
    a.rows = rows;
    a.strip = strip_rows(rows, C, is_bwd);
    a.per_gate = gate ? rows / gates : 1;
    const long long wgs = workgroups(rows, C, true);
    a.part = part;
    a.gate_part = part ? part + (size_t)wgs * 2 * C : nullptr;
    const int kind = !gate ? kNoGate : (gates == rows ? kElementGate : kSharedGate);
    auto go = [&](auto* t) {
        typedef std::remove_pointer_t<decltype(t)> T;
        return kind == kNoGate ? launch_c<T, kNoGate>(a, is_bwd, stream)
                               : (kind == kElementGate ? launch_c<T, kElementGate>(a, is_bwd, stream) : launch_c<T, kSharedGate>(a, is_bwd, stream));
    };
    hipError_t e = is_bf16 ? go((__bf16*)nullptr) : go((float*)nullptr);
    if (e != hipSuccess || !is_bwd) return e;
    const bool shared = kind == kSharedGate;
    if (!a.w_after) dwa = nullptr;
    if (!a.w_before) dwb = nullptr;
    if (!dwa && !dwb && !shared) return hipSuccess;
    const long long lists = 2 + (shared ? gates : 0);
    const dim3 grid((C + 31) / 32, (unsigned)(lists < 4096 ? lists : 4096));
    if (is_bf16) hipLaunchKernelGGL(block_norm_sum_kernel<__bf16>, grid, dim3(1024), 0, stream, a.part, a.gate_part, dwa, dwb, shared ? (__bf16*)d_gate : nullptr, rows, a.strip, a.per_gate, wgs, C);
    else hipLaunchKernelGGL(block_norm_sum_kernel<float>, grid, dim3(1024), 0, stream, a.part, a.gate_part, dwa, dwb, shared ? (float*)d_gate : nullptr, rows, a.strip, a.per_gate, wgs, C);
    return hipGetLastError();
}

}  // namespace ltn
