// Gated delta rule: what its kernels and the C-ABI layer share.  Internal; the public boundary is include/ltn_attn.h.
//
// One head, one sequence, state S [Dk x Dv] (fp32, row = key feature, column = value feature):
//
//     S_t = a_t S_{t-1} + k_t u_t^T,   u_t = beta_t z_t,   z_t = v_t - a_t S_{t-1}^T k_t,   o_t = scale S_t^T q_t,   a_t = exp(g_t)
//
// In chunks of 64 tokens, with S0 the state before a chunk, G the log decays summed from its first token on,
// gam = exp(G), end = exp(G_last - G) and R[r,i] = exp(G_r - G_i) for r >= i, else 0 (only exponents of sums of log
// decays between two tokens are formed, never a quotient of products):
//
//     L = strict lower triangle of R (.) K K^T      T' = (I + L diag(beta))^-1      P = scale R (.) Q K^T
//     X = V - diag(gam) K S0      Z = T' X      U = diag(beta) Z
//     O = scale diag(gam) Q S0 + P U      S1 = gam_last S0 + K^T diag(end) U
//
// and, with dS the derivative by S1,
//
//     dU = P^T dO + diag(end) K dS      dV = T'^T diag(beta) dU
//     dS0 = gam_last dS + Q^T diag(scale gam) dO - K^T diag(gam) dV
//     dP = scale R (.) dO Z^T      E = -R (.) dV Z^T below the diagonal      C = diag(end) Z dS^T
//     dQ = scale diag(gam) dO S0^T + dP diag(beta) K
//     dK = -diag(gam) dV S0^T + E diag(beta) K + diag(beta) (C + dP^T Q + E^T K)
//     dbeta_r = k_r . C_r + column r's sum of dP (.) Q K^T + E (.) K K^T
//     dg_t = sum over r >= t in the chunk of dG_r,
//     dG_r = q_r . (dQ's first term)_r + k_r . (dK's first term)_r - beta_r dbeta_r + row r's sum of (dP (.) Q K^T + E (.) K K^T) diag(beta),
//     and dG_last has, besides, gam_last <S0, dS> and the sum of beta_r k_r . C_r
//
// (dbeta and dg are sums over a token of what its factor, or its exponent, multiplies; T with beta on its other side, and
// the derivative by U that goes with it, are never formed.)
//
// Three kinds of kernels: "prepare" (per chunk: T', P and the decays; no chunk needs another), "sweeps" (per chain,
// chunk after chunk: the state and what needs it; the columns of S are independent of each other, so value columns are
// split over waves and workgroups) and "grad" (per chunk, from the states that two sweeps left).
#pragma once
#include "ltn_bf16_tiles.h"

namespace ltn {

constexpr int kChunk = 64;
constexpr int kVec = 5 * kChunk;          // per chunk: gam, end, beta and G in two parts (G = hi + lo)

struct DeltaArgs {
    const void *q, *k, *v, *d_o;          // [Bt, Hk, N, Dk] twice, [Bt, H, N, Dv] twice
    void* o;                              // [Bt, H, N, Dv]
    void *dq, *dk, *dv, *dg, *dbeta;      // as q, k, v; [Bt, H, N] in the tensors' type
    const float *g, *beta;                // [Bt, H, N]
    const float* kv_in;                   // [seqs, H, Dk, Dv] or nullptr (zero)
    float* kv_out;                        // the same, or nullptr
    const int* cu;                        // packed sequences: their seqs + 1 ends in the one row of N tokens; nullptr: rows are sequences
    int Hk, H, seqs;                      // seqs = Bt without cu
    long long N;
    float scale;
    // scratch, per (chunk slot, value head): see delta_scratch()
    char *tq, *tl, *p, *z, *s0, *ds;
    float* vec;
    int slots;                            // chunk slots of all sequences
};

// Chunks of a packed sequence are numbered from cu[i] / 64 + i on: no two sequences' overlap, whatever their lengths,
// and no sum over sequences is needed.
inline long long delta_slots(long long rows, long long N, bool packed) {
    return packed ? N / kChunk + rows : rows * ((N + kChunk - 1) / kChunk);
}

// bytes per (chunk slot, value head) of each scratch array, and all of them for the forward or the backward
struct DeltaScratch {
    size_t tile, z, state;                // a 64 x 64 tile, [Dv, 64], [Dv, Dk], in the tensors' type
    size_t vec;
};
inline DeltaScratch delta_scratch(int Dk, int Dv, bool bf16) {
    const size_t e = bf16 ? 2 : 4;
    return {kChunk * kChunk * e, Dv * (size_t)kChunk * e, (size_t)Dk * Dv * e, kVec * sizeof(float)};
}
inline size_t delta_bytes(int Dk, int Dv, bool bf16, bool bwd) {
    const DeltaScratch s = delta_scratch(Dk, Dv, bf16);
    // T' (bf16: in two parts, for the fp32 state handed out; the gradients take the first), P and decays; for the gradients
    // Z, the states before chunks and their derivatives behind them
    return (bf16 && !bwd ? 3 : 2) * s.tile + s.vec + (bwd ? s.z + 2 * s.state : 0);
}

hipError_t launch_delta_fwd(const DeltaArgs& a, int Dk, int Dv, int is_bf16, hipStream_t stream);
hipError_t launch_delta_bwd(const DeltaArgs& a, int Dk, int Dv, int is_bf16, hipStream_t stream);
hipError_t launch_delta_prepare(const DeltaArgs& a, int Dk, int is_bf16, hipStream_t stream);
hipError_t launch_delta_grad(const DeltaArgs& a, int Dk, int Dv, int is_bf16, hipStream_t stream);
// q, k: [chains of Hk, steps, Dk]; v, o: [chains, steps, Dv]; g, beta: [chains, steps]; kv: [chains, Dk, Dv]
hipError_t launch_delta_decode(const void* q, const void* k, const void* v, void* o, float* kv, const float* g,
                               const float* beta, float scale, int Bt, int Hk, int H, int steps, int Dk, int Dv, int is_bf16,
                               hipStream_t stream);

namespace {

// Where sequence `seq` lies: its first token in its row of N tokens, the row's index among the batch, its length and
// the slot of its first chunk.  Ends that are out of order or out of the row are drawn into it, so that no access leaves it.
struct DeltaSeq { long long row, first; int len, slot; };
__device__ __forceinline__ DeltaSeq delta_seq(const DeltaArgs& a, int seq) {
    if (!a.cu) return {seq, 0, (int)a.N, seq * (int)((a.N + kChunk - 1) / kChunk)};
    const int N = (int)a.N, c0 = a.cu[seq], c1 = a.cu[seq + 1];
    const int first = c0 < 0 ? 0 : (c0 > N ? N : c0), end = c1 < first ? first : (c1 > N ? N : c1);
    return {0, first, end - first, first / kChunk + seq};
}
// The sequence that chunk slot `slot` belongs to, and which of its chunks; false: the slot holds none.
__device__ __forceinline__ bool delta_find(const DeltaArgs& a, int slot, DeltaSeq& s, int& chunk) {
    int seq = 0;
    if (!a.cu) {
        seq = slot / (int)((a.N + kChunk - 1) / kChunk);
    } else {
        int lo = 0, hi = a.seqs - 1;      // the last sequence whose first slot is not behind this one
        while (lo < hi) {
            const int mid = (lo + hi + 1) / 2;
            if (delta_seq(a, mid).slot <= slot) lo = mid;
            else hi = mid - 1;
        }
        seq = lo;
    }
    s = delta_seq(a, seq);
    chunk = slot - s.slot;
    return chunk >= 0 && (long long)chunk * kChunk < s.len;
}

// ---- operands of 16 x 16 x 32 products in either type: a lane holds eight consecutive elements of the summed index, from
// 8 (lane / 16) on.  fp32: eight products of 16 x 16 x 4, each taking one of them from every lane.
template <class T> struct El;
template <> struct El<__bf16> {
    typedef bf16x8 F;
};
struct F32Frag { f32x4 a, b; };
template <> struct El<float> {
    typedef F32Frag F;
};

__device__ __forceinline__ f32x4 mma(const bf16x8& a, const bf16x8& b, const f32x4& c) { return mfma16(a, b, c); }
__device__ __forceinline__ f32x4 mma(const F32Frag& a, const F32Frag& b, f32x4 c) {
#pragma unroll
    for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a.a[j], b.a[j], c, 0, 0, 0);
#pragma unroll
    for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a.b[j], b.b[j], c, 0, 0, 0);
    return c;
}
// eight fp32 values (two tiles' results) as an operand
template <class T> __device__ __forceinline__ typename El<T>::F frag_of(const f32x4& x, const f32x4& y);
template <> __device__ __forceinline__ bf16x8 frag_of<__bf16>(const f32x4& x, const f32x4& y) {
    return __builtin_convertvector(__builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7), bf16x8);
}
template <> __device__ __forceinline__ F32Frag frag_of<float>(const f32x4& x, const f32x4& y) { return {x, y}; }
__device__ __forceinline__ void values_of(const bf16x8& f, f32x4& x, f32x4& y) {
    const f32x8 v = __builtin_convertvector(f, f32x8);
    x = __builtin_shufflevector(v, v, 0, 1, 2, 3);
    y = __builtin_shufflevector(v, v, 4, 5, 6, 7);
}
__device__ __forceinline__ void values_of(const F32Frag& f, f32x4& x, f32x4& y) { x = f.a; y = f.b; }
// what rounding to the operand's type loses of x, y, as an operand (bf16: 16 bits of the significand together)
__device__ __forceinline__ bf16x8 rest_of(const bf16x8& f, const f32x4& x, const f32x4& y) {
    Frag h;
    h.v = f;
    f32x4 a, b;
#pragma unroll
    for (int i = 0; i < 4; ++i) {          // (from the packed words: the compiler would convert each value again)
        f32x4& r = i < 2 ? a : b;
        asm("v_lshlrev_b32 %0, 16, %1" : "=v"(r[2 * (i & 1)]) : "v"(h.u[i]));
        asm("v_and_b32 %0, 0xffff0000, %1" : "=v"(r[2 * (i & 1) + 1]) : "v"(h.u[i]));
    }
    return frag_of<__bf16>(x - a, y - b);
}

// ---- LDS tiles of 64 rows (tokens, or columns of a state) and COLS columns.  bf16: as Swz has it (16-byte chunks swizzled
// with the row, no padding), filled by direct loads.  fp32: rows padded by 16 bytes, filled through registers.
template <class T, int COLS> struct Tile;
template <int COLS> struct Tile<__bf16, COLS> {
    static constexpr int RB = Swz<COLS>::RB, BYTES = Swz<COLS>::BYTES;
    static __device__ __forceinline__ int chunk(int r, int c) { return Swz<COLS>::off(r, c); }    // of 16 bytes
    static __device__ __forceinline__ int at(int r, int c) { return chunk(r, c >> 3) + (c & 7) * 2; }
};
template <int COLS> struct Tile<float, COLS> {
    static constexpr int RB = COLS * 4 + 16, BYTES = kChunk * RB;
    static __device__ __forceinline__ int chunk(int r, int c) { return r * RB + c * 16; }
    static __device__ __forceinline__ int at(int r, int c) { return r * RB + c * 4; }
};

// Rows (or columns) of a 16-wide tile whose results, with those of the next tile, are eight consecutive ones in a lane:
// row m of tile t is 32 (t / 2) + 4 (t % 2) + 8 (m / 4) + m % 4; the lane then holds 32 (t / 2) + 8 (lane / 16) + 4 (t % 2) .. +3.
__device__ __forceinline__ int paired(int t, int m) { return 32 * (t >> 1) + 4 * (t & 1) + 8 * (m >> 2) + (m & 3); }

// Operands from tiles, by LDS byte address.  A reader holds a lane's address in a tile at `lds` and serves every tile of its
// width that begins a multiple of 1 KB behind: `tile` (a constant) goes into the instruction, and columns into an exclusive
// or, as the swizzle is one.  hide() keeps the compiler from forming all those addresses ahead of a loop, in registers.
#ifdef __HIP_DEVICE_COMPILE__
template <class U> __device__ __forceinline__ U lds_read(unsigned at) { return *(const __attribute__((address_space(3))) U*)at; }
template <class U> __device__ __forceinline__ void lds_write(unsigned at, const U& x) { *(__attribute__((address_space(3))) U*)at = x; }
__device__ __forceinline__ s16x4 lds_read_tr(unsigned at) {
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 __attribute__((address_space(3)))*)at);
}
#else                                      // (host code has no such addresses)
template <class U> __device__ U lds_read(unsigned);
template <class U> __device__ void lds_write(unsigned, const U&);
__device__ s16x4 lds_read_tr(unsigned);
#endif
template <class T> __device__ __forceinline__ typename El<T>::F lds_frag(unsigned at) {
    if constexpr (sizeof(T) == 2) return lds_read<bf16x8>(at);
    else return F32Frag{lds_read<f32x4>(at), lds_read<f32x4>(at + 16)};
}
// (element by element: a vector of four equal factors would be kept in registers of its own)
__device__ __forceinline__ f32x4 times(const f32x4& x, float s) { return f32x4{x[0] * s, x[1] * s, x[2] * s, x[3] * s}; }
__device__ __forceinline__ unsigned hide(unsigned x) {
    asm("" : "+v"(x));
    return x;
}

// A reader's address 32 kb columns on, kb a multiple of the power of two that the columns it then reads are fewer than.
template <class T> __device__ __forceinline__ unsigned skip_columns(unsigned at, int kb) { return sizeof(T) == 2 ? at ^ (kb << 6) : at + kb * 128; }

// Eight elements of one row, from column 32 kb + 8 (lane / 16) on.
template <class T, int COLS> struct RowReader {
    unsigned b;
    __device__ __forceinline__ RowReader(unsigned lds, int row, int lane)
        : b(lds + Tile<T, COLS>::chunk(row, (sizeof(T) == 2 ? 1 : 2) * (lane >> 4))) {}
    __device__ __forceinline__ void move(int by) { b += by; }
    __device__ __forceinline__ void skip(int kb) { b = skip_columns<T>(b, kb); }
    __device__ __forceinline__ typename El<T>::F frag(int tile, int kb) const {
        return lds_frag<T>(sizeof(T) == 2 ? (b ^ (kb << 6)) + tile : b + tile + kb * 128);
    }
};
// The same of rows paired(rt, lane % 16)
template <class T, int COLS> struct PairedRowReader {
    unsigned even, odd;
    __device__ __forceinline__ PairedRowReader(unsigned lds, int lane)
        : even(RowReader<T, COLS>(lds, paired(0, lane & 15), lane).b), odd(RowReader<T, COLS>(lds, paired(1, lane & 15), lane).b) {}
    __device__ __forceinline__ void move(int by) {
        even += by;
        odd += by;
    }
    __device__ __forceinline__ void skip(int kb) {
        even = skip_columns<T>(even, kb);
        odd = skip_columns<T>(odd, kb);
    }
    __device__ __forceinline__ typename El<T>::F frag(int tile, int rt, int kb) const {
        RowReader<T, COLS> r = {0, 0, 0};
        r.b = rt & 1 ? odd : even;
        return r.frag(tile + (rt >> 1) * 32 * Tile<T, COLS>::RB, kb);
    }
};
// Rows 32 kb + 8 (lane / 16) .. +7 of one column: of column 16 t + lane % 16, or of column paired(t, lane % 16).
template <class T, int COLS, bool PAIRED> struct ColReader {
    unsigned lo, hi;                       // bf16: rows of either half
    __device__ __forceinline__ ColReader(unsigned lds, int lane) {
        const int row = 8 * (lane >> 4), s = lane & 15;
        if constexpr (sizeof(T) == 2) {
            const int c = (PAIRED ? 8 : 4) * (s & 3);
            lo = lds + Tile<T, COLS>::at(row + (s >> 2), c);
            hi = lds + Tile<T, COLS>::at(row + 4 + (s >> 2), c);
        } else {
            lo = hi = lds + Tile<T, COLS>::at(row, PAIRED ? paired(0, s) : s);
        }
    }
    __device__ __forceinline__ void move(int by) {                       // by a multiple of 1 KB
        lo += by;
        hi += by;
    }
    __device__ __forceinline__ void skip(int kb) {
        lo = skip_columns<T>(lo, kb);
        hi = skip_columns<T>(hi, kb);
    }
    __device__ __forceinline__ void hide_all() {
        lo = hide(lo);
        if constexpr (sizeof(T) == 2) hi = hide(hi);
    }
    __device__ __forceinline__ typename El<T>::F frag(int tile, int kb, int t) const {
        const int at = tile + kb * 32 * Tile<T, COLS>::RB;
        if constexpr (sizeof(T) == 2) {
            const int x = PAIRED ? (t >> 1) << 6 : t << 5, y = PAIRED ? (t & 1) * 8 : 0;
            Frag f;
            f.h[0] = lds_read_tr((lo ^ x) + at + y);
            f.h[1] = lds_read_tr((hi ^ x) + at + y);
            return f.v;
        } else {
            const int y = at + 4 * (PAIRED ? 32 * (t >> 1) + 4 * (t & 1) : 16 * t);
            F32Frag f;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                f.a[j] = lds_read<float>(lo + y + j * Tile<T, COLS>::RB);
                f.b[j] = lds_read<float>(lo + y + (4 + j) * Tile<T, COLS>::RB);
            }
            return f;
        }
    }
    // rows 32 (rt / 2) + 8 (lane / 16) + 4 (rt % 2) .. +3 of column 16 t + lane % 16, as fp32 (not paired)
    __device__ __forceinline__ f32x4 values(int tile, int rt, int t) const {
        const int at = tile + (rt >> 1) * 32 * Tile<T, COLS>::RB;
        if constexpr (sizeof(T) == 2) {
            Frag f;
            f.h[0] = lds_read_tr(((rt & 1 ? hi : lo) ^ (t << 5)) + at);
            return __builtin_convertvector(f.b[0], f32x4);
        } else {
            f32x4 x;
#pragma unroll
            for (int j = 0; j < 4; ++j) x[j] = lds_read<float>(lo + at + 64 * t + (4 * (rt & 1) + j) * Tile<T, COLS>::RB);
            return x;
        }
    }
};

// A tile from global memory, rows `pitch` bytes apart, by W waves; rows from `valid` on become zero.  bf16: fetch() issues
// direct loads to LDS and the data is there once they have been waited for.  fp32: fetch() loads registers, put() stores them.
template <class T, int COLS, int W, int ROWS = kChunk, bool KEEP = false> struct TileFetch;
template <int COLS, int W, int ROWS, bool KEEP> struct TileFetch<__bf16, COLS, W, ROWS, KEEP> {
    typedef Swz<COLS> S;
    static constexpr int NV = S::CPR / 4, NI = S::NI * ROWS / kChunk, PER = NI / W;      // loads of a tile and of a wave
    static_assert(NI % W == 0 && NV >= 1, "every wave issues the same number of loads");
    // src: wave-uniform
    __device__ __forceinline__ void fetch(const char* src, unsigned pitch, int valid, unsigned lds, int w, int lane) {
        // KEEP: the lane's offsets are formed once, in registers; else at each fetch (where waves that fetch compute too, registers are dearer)
        const int own = KEEP ? lane : (int)hide((unsigned)lane);
        if (valid >= ROWS) {               // a scalar base and the lane's offset, the same for each load where its rows are 16 n apart
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                constexpr int STEP = W * 64 / S::CPR, APART = STEP % 16 ? 16 / STEP : 1;
                const int j = w + W * (i % APART), slot = 64 * j + own, r = slot / S::CPR, c = (slot % S::CPR) ^ S::key(r);
                dma16s<false>(lds + 1024u * (unsigned)(w + W * i), src + (size_t)(i / APART * APART * STEP) * pitch, r * pitch + c * 16);
            }
            return;
        }
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int j = w + W * i, slot = 64 * j + own, r = slot / S::CPR, c = (slot % S::CPR) ^ S::key(r);
            const char* g = src + (size_t)r * pitch + c * 16;
            dma16(lds + 1024u * (unsigned)j, r < valid ? g : (const char*)kZeros);
        }
    }
    __device__ __forceinline__ void put(unsigned, int, int) const {}
};
template <int COLS, int W, int ROWS, bool KEEP> struct TileFetch<float, COLS, W, ROWS, KEEP> {
    static constexpr int CPR = COLS / 4, PER = ROWS * CPR / (64 * W);
    u32x4 v[PER];
    __device__ __forceinline__ void fetch(const char* src, unsigned pitch, int valid, unsigned, int w, int lane) {
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int j = 64 * (w + W * i) + lane, r = j / CPR;
            v[i] = u32x4{0, 0, 0, 0};
            if (r < valid) v[i] = *(const u32x4*)(src + (size_t)r * pitch + j % CPR * 16);
        }
    }
    __device__ __forceinline__ void put(unsigned lds, int w, int lane) const {
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int j = 64 * (w + W * i) + lane;
            lds_write(lds + Tile<float, COLS>::chunk(j / CPR, j % CPR), v[i]);
        }
    }
};

}  // namespace
}  // namespace ltn
