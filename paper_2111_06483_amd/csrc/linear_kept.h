// Many rows times one small operand that a compute unit keeps whole (linear_act.hip).
//
// The operand's columns are dealt to workgroups in blocks of 128 whose pieces (k_typed_lay) fit LDS beside the rows'; a workgroup copies its block once and its
// eight wavefronts then go their own ways, with no barrier: each takes every so-manyth 32 rows, brings them by whole lines, all of the next ones while it
// multiplies these, hands them to the lanes that multiply them through LDS of its own, and finishes and stores its results while the others multiply.
// Why: with the operand passing through LDS for every 128 rows (linear_typed_rows.h) its copies, which a barrier waits for, take as long as the products, and the
// rows' own way from memory is waited for at each.  867187 x 256 -> 256, bf16, GELU, residual, argument kept, 1.78 GB: that way 576 us; so, a chunk of rows ahead 564; the next
// rows and residuals whole, under way without a branch, 433; stores without a branch 428.  (Two passes over the rows for 256 columns: both at about the same time on
// one XCD, the second from its L2.)  Bf16 rows of dA in two pieces are a third product and twice the bytes: 256 -> 256, the same rows, traced, 287 us of one, 394 of two.
#pragma once

#include "linear_typed_rows.h"

namespace sar {

namespace {

constexpr int kKeptWaves = 8, kKeptThreads = kKeptWaves * 64;
constexpr size_t kKeptLds = 160 * 1024;

template <typename E, typename Q>
struct KeptArgs {
    RowsArgs<E> rows;
    int64_t n;
    Q prologue;
};

// The residuals of step s as fetch_residual has them, without a branch: what lies behind the last column or row is read from them.
template <typename T, typename SH>
__device__ SAR_INLINE inline void residual_of(const Epilogue& e, const Place<SH>& at, int s, Neighbours<T, SH::IL> (&out)[4])
{
    const T* from = static_cast<const T*>(e.res) + at.tile();
    const uint32_t n = (uint32_t)min(at.column(s / 4), at.N - SH::IL);
#pragma unroll
    for (int k = 0; k < 4; ++k)
        out[k] = *within_tile<const Neighbours<T, SH::IL>>(from, ((uint32_t)min(at.row(4 * (s % 4) + k), at.rows - 1) * (uint32_t)at.N + n) * (uint32_t)sizeof(T));
}

// A wavefront's results, from the sums to memory.  Loads and stores are waited for in the order in which they were sent, by counting those sent since, and
// what a branch may have sent does not count: so that the next rows, which are under way, need not be waited for behind these results' stores, these are
// sent without a branch, what lies behind the last row or column to a place outside of the tile's buffer, where the memory unit drops it.  (A guard around
// each where a tile is not whole, and a wait behind them: 400000 x 100 -> 172, bf16, 226 us, so 153; 200 -> 400 514 and 348.)
template <typename T, typename SH, bool RES, typename E, int NW, int KNOWN>
__device__ SAR_INLINE inline void finish_kept(const E& e, void* out, const Place<SH>& at, const float (&bias)[NW], float16_t (&acc)[NW],
                                              const Neighbours<T, SH::IL> (&res)[KNOWN][4])
{
    constexpr int IL = SH::IL, kSteps = NW / IL * 4, kWords = IL * (int)sizeof(T) / 4;
    const int64_t tile = at.tile();
    auto store = [&](void* to, int s, const float (&v)[4][IL]) SAR_INLINE {
        const int n = at.column(s / 4);
        const auto buffer = __builtin_amdgcn_make_buffer_rsrc(static_cast<T*>(to) + tile, 0, 32 * at.N * (int)sizeof(T), 0x00020000);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int i = at.row(4 * (s % 4) + k);
            const uint32_t place = ((uint32_t)i * (uint32_t)at.N + (uint32_t)n) * (uint32_t)sizeof(T);
            const int where = i < at.rows && n < at.N ? (int)place : -1;
            Neighbours<T, IL> w;
            w.set(v[k]);
            typedef uint32_t Words __attribute__((ext_vector_type(kWords)));
            Words x;
#pragma unroll
            for (int j = 0; j < kWords; ++j) x[j] = w.x[j];
            if constexpr (kWords == 4) __builtin_amdgcn_raw_buffer_store_b128(x, buffer, where, 0, 0);
            else __builtin_amdgcn_raw_buffer_store_b64(x, buffer, where, 0, 0);
        }
    };
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
        float v[4][IL];
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
            for (int j = 0; j < IL; ++j) v[k][j] = acc[s / 4 * IL + j][4 * (s % 4) + k];
        if constexpr (E::kAny) {
            auto add_residual = [&]() SAR_INLINE {
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    float r[IL];
                    res[s][k].values(r);
#pragma unroll
                    for (int j = 0; j < IL; ++j) v[k][j] += r[j];
                }
            };
#pragma unroll
            for (int k = 0; k < 4; ++k)
#pragma unroll
                for (int j = 0; j < IL; ++j) v[k][j] += bias[s / 4 * IL + j];
            if constexpr (RES) {
                if (!e.after) add_residual();
            }
            if (e.pre) store(e.pre, s, v);
            with_act(e.act, [&](auto act) SAR_INLINE {
#pragma unroll
                for (int k = 0; k < 4; ++k)
#pragma unroll
                    for (int j = 0; j < IL; ++j) v[k][j] = act_of<decltype(act)::value>(v[k][j]);
            });
            if constexpr (RES) {
                if (e.after) add_residual();
            }
        }
        store(out, s, v);
        __builtin_amdgcn_sched_barrier(0);
    }
}

// CHUNKS: of the contraction; RES: a residual; Q: rows as they are, or (bf16) in two pieces, read or formed here, whose second ones meet the operand's first.
template <typename T, int NT, int CHUNKS, bool TRANS, bool RES, typename E, typename Q>
__global__ __launch_bounds__(kKeptThreads, 2) void k_rows_kept(KeptArgs<E, Q> g)
{
    constexpr bool kLow = Q::kAny;
    static_assert(!kLow || sizeof(T) == 2, "two pieces of bf16");
    using Sh = WholeShare<T, NT>;
    const RowsArgs<E>& a = g.rows;
    constexpr int PC = Mode<T>::kPieces, S = Mode<T>::kSteps, CH = kChunk<T>, N = Cols<T>::N, SB = Mode<T>::kStage, kSP = PC == 3 ? 3 : 1;
    constexpr int kRaw = 4, kFrags = kStageFrags<T, NT>, kStages = CHUNKS * (S / SB);      // kRaw: 16-byte pieces of 32 rows' chunk that a lane brings
    extern __shared__ __attribute__((aligned(16))) uint4 lds[];          // [kStages][kFrags][64] of B, [kKeptWaves][32][8] of rows
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5;
    // workgroups of the same rows and other columns are neighbours on one XCD
    const int turn = blockIdx.x / 8, block = turn % a.blocks, group = turn / a.blocks * 8 + blockIdx.x % 8, groups = gridDim.x / a.blocks;
    const int n0 = block * (32 * NT);
    const uint4* from = a.B + (int64_t)block * kStages * (kFrags * 64);
    for (int f = wave; f < kStages * kFrags; f += kKeptWaves)
        __builtin_amdgcn_global_load_lds((GlobalSrc*)(from + f * 64 + lane), (LdsPtr*)(lds + f * 64), 16, 0, 0);
    float bias[NT] = {};
    if constexpr (E::kAny) {
#pragma unroll
        for (int i = 0; i < NT; ++i) {
            const int n = n0 + Sh::column_of(i, lane & 31);
            if (a.epilogue.bias && n < a.N) bias[i] = a.epilogue.bias[n];
        }
    }

    const int tiles = (int)((g.n + 31) / 32), step = groups * kKeptWaves;
    uint4 raw[CHUNKS][kRaw], low[kLow ? CHUNKS : 1][kRaw];
    auto fetch = [&](const void* from, uint4 (&to)[kRaw], int tile, int chunk) SAR_INLINE {
        int own = lane;
        asm volatile("" : "+v"(own));
        const int c = chunk * CH + (own & 7) * N;
        const int64_t r0 = (int64_t)tile * 32;
        const uint32_t most = (uint32_t)min(g.n - 1 - r0, (int64_t)31);
#pragma unroll
        for (int k = 0; k < kRaw; ++k) {
            const uint32_t row = min((uint32_t)(8 * k + (own >> 3)), most) * (uint32_t)a.C;
            const T* rows = static_cast<const T*>(from) + r0 * a.C;
            // (rows of less than a piece: one chunk, value by value)
            to[k] = CHUNKS > 1 || a.C >= N ? load16(within_tile<const T>(rows, (row + (uint32_t)min(c, a.C - N)) * (uint32_t)sizeof(T)))
                                                   : Cols<T>::load(rows + row, c, a.C, a.C);
        }
    };
    auto fetch_chunk = [&](int tile, int chunk) SAR_INLINE {
        fetch(a.A, raw[chunk], tile, chunk);
        if constexpr (Q::kForms) fetch(g.prologue.pre, low[chunk], tile, chunk);
        else if constexpr (kLow) fetch(g.prologue.low, low[chunk], tile, chunk);
    };
    uint4* const rows = lds + kStages * kFrags * 64 + wave * 256;
    // A chunk, from the lanes that brought it to those that multiply it.  The lanes meet before what others wrote is read, and before it is written again: no
    // instruction, but without it lanes that a branch parts from the others (a row's last piece) may be sent through all of this ahead of them.
    auto meet = []() SAR_INLINE {
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    };
    auto hand_over = [&](int chunk, uint4 (&v)[kRaw], uint4 (&x)[kRaw]) SAR_INLINE {
        const int c = chunk * CH + (lane & 7) * N;
        if (chunk == CHUNKS - 1 && c + N > a.C) {
#pragma unroll
            for (int k = 0; k < kRaw; ++k) {
                if (c >= a.C) v[k] = make_uint4(0u, 0u, 0u, 0u);
                else if (a.C >= N) v[k] = front_of_piece<T>(v[k], a.C - c);
            }
        }
#pragma unroll
        for (int k = 0; k < kRaw; ++k) rows[(8 * k + (lane >> 3)) * 8 + ((lane & 7) ^ (lane >> 3))] = v[k];
        meet();
#pragma unroll
        for (int k = 0; k < kRaw; ++k) x[k] = rows[(lane & 31) * 8 + ((h * kRaw + k) ^ (lane & 7))];
        meet();
    };

    int tile = group * kKeptWaves + wave;
    if (tile < tiles) {
#pragma unroll
        for (int chunk = 0; chunk < CHUNKS; ++chunk) fetch_chunk(tile, chunk);
    }
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
    // residuals read with the rows, and those that wait until there are registers for them
    constexpr int kSteps = NT / Sh::IL * 4, kEarly = sizeof(T) == 2 ? kSteps : kSteps / 2;
    for (; tile < tiles; tile += step) {
        float16_t acc[NT];
#pragma unroll
        for (int i = 0; i < NT; ++i) acc[i] = float16_t{};
        const int64_t r0 = (int64_t)tile * 32;
        // (places are worked out where they are used: carried through the loop they are dozens of registers)
        auto place = [&]() SAR_INLINE {
            int own = lane;
            asm volatile("" : "+v"(own));
            return Place<Sh>(r0, g.n, a.N, n0, 0, own);
        };
        Neighbours<T, Sh::IL> res[kSteps][4];
        float sign = kDown * kDown;
#pragma unroll
        for (int chunk = 0; chunk < CHUNKS; ++chunk) {
            uint4 p[S / SB][1][SB][kSP], x[kRaw], y[kRaw];
            if constexpr (Q::kForms) {
#pragma unroll
                for (int k = 0; k < kRaw; ++k) form_piece<T>(g.prologue.act, raw[chunk][k], low[chunk][k], low[chunk][k]);
            }
            hand_over(chunk, raw[chunk], x);
            if constexpr (kLow) hand_over(chunk, low[chunk], y);
            if constexpr (Q::kForms) {
                if (g.prologue.formed && block == 0) {
#pragma unroll
                    for (int k = 0; k < kRaw; ++k) {
                        const int64_t i = r0 + 8 * k + (lane >> 3);
                        float v[N];
                        Cols<T>::unpack(raw[chunk][k], v);
                        if (i < g.n) Cols<T>::store(static_cast<T*>(g.prologue.formed) + i * a.C, chunk * CH + (lane & 7) * N, a.C, v);
                    }
                }
            }
#pragma unroll
            for (int s = 0; s < S; ++s) {
                if constexpr (PC == 3) {
                    float v[8] = {__uint_as_float(x[2 * s].x), __uint_as_float(x[2 * s].y), __uint_as_float(x[2 * s].z), __uint_as_float(x[2 * s].w),
                                  __uint_as_float(x[2 * s + 1].x), __uint_as_float(x[2 * s + 1].y), __uint_as_float(x[2 * s + 1].z),
                                  __uint_as_float(x[2 * s + 1].w)};
#pragma unroll
                    for (int j = 0; j < 8; ++j) v[j] *= kUp;
                    split8(v, p[s / SB][0][s % SB]);
                } else {
                    p[s / SB][0][s % SB][0] = x[s];
                }
            }
            if constexpr (RES) {
                if (chunk == 0) {
                    const Place<Sh> at = place();
#pragma unroll
                    for (int s = 0; s < kEarly; ++s) residual_of<T, Sh>(a.epilogue, at, s, res[s]);
                }
            }
            fetch_chunk(min(tile + step, tiles - 1), chunk);         // (the last one's are not looked at)
#pragma unroll
            for (int part = 0; part < S / SB; ++part) {
                const uint4* const b = lds + (chunk * (S / SB) + part) * (kFrags * 64) + lane;
                float16_t(&sums)[1][NT] = reinterpret_cast<float16_t(&)[1][NT]>(acc);
                if constexpr (kLow) {
                    auto add = [&](int i, const uint4& v, const uint4& w) SAR_INLINE {
                        acc[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, v), __builtin_bit_cast(bf16x8_t, w), acc[i], 0, 0, 0);
                    };
#pragma unroll
                    for (int s = 0; s < SB; ++s)
#pragma unroll
                        for (int i = 0; i < NT; ++i) {
                            const uint4 w0 = b[s * PC * NT * 64 + i * 64], w1 = b[(s * PC + 1) * NT * 64 + i * 64];
                            add(i, x[part * SB + s], w1);
                            add(i, y[part * SB + s], w0);
                            add(i, x[part * SB + s], w0);
                        }
                } else {
                    multiply_stage<T, NT, 1, NT>(b, p[part], sign, sums);
                }
            }
            sign = -sign;
        }
        bool odd = false;
#pragma unroll
        for (int i = 0; i < NT; ++i) odd |= not_finite(acc[i]);
        if (__any(odd)) exact_tiles<T, Sh, TRANS>(a, g.prologue, 0, min(r0 + (lane & 31), g.n - 1), n0, 0, acc);
        const Place<Sh> at = place();
        if constexpr (RES) {
#pragma unroll
            for (int s = kEarly; s < kSteps; ++s) residual_of<T, Sh>(a.epilogue, at, s, res[s]);
        }
        finish_kept<T, Sh, RES>(a.epilogue, a.out, at, bias, acc, res);
    }
}

// Four column tiles, eight wavefronts' rows: the chunks of a contraction that fit beside them (bf16), or that a lane's registers take (fp32).
constexpr int kKeptTiles = 4, kMostKeptChunks = 4;
// Whether they do, columns are whole groups of a lane's neighbours, and more than what half a block leaves empty.
template <typename T>
bool fits_kept(int C, int N)
{
    static_assert((kMostKeptChunks * Mode<T>::kSteps * Mode<T>::kPieces * kKeptTiles + kKeptWaves * 4) * 1024 <= kKeptLds, "LDS of a compute unit");
    return (C + kChunk<T> - 1) / kChunk<T> <= kMostKeptChunks && N % WholeShare<T, kKeptTiles>::IL == 0 && N > 16 * kKeptTiles;
}

// out [n, N] = A [n, C] B; TRANS: B = W^T.  work: lay_bytes.
template <typename T, int CHUNKS, bool TRANS, typename E, typename Q>
int run_kept_chunks(const void* A, const float* W, int64_t n, void* out, int K, int F, void* work, hipStream_t st, const E& e, const Q& q)
{
    constexpr int NT = kKeptTiles;
    const int C = TRANS ? F : K, N = TRANS ? K : F, blocks = (N + 32 * NT - 1) / (32 * NT);
    uint4* const pieces = static_cast<uint4*>(work);
    const int64_t units = (int64_t)blocks * CHUNKS * Mode<T>::kSteps * NT * 64, lay = (units + 255) / 256;
    const LayArgs l{W, pieces, 1, K, F, C, N, CHUNKS, blocks, Types{nullptr, 1, n}, nullptr, 0, (unsigned)lay};
    k_typed_lay<T, NT, TRANS, WholeShare<T, NT>><<<(unsigned)lay, 256, 0, st>>>(l);
    SAR_LAUNCH_CHECK();
    const KeptArgs<E, Q> a{{A, pieces, W, out, nullptr, C, N, CHUNKS, blocks, K, F, e}, n, q};
    constexpr size_t shared = ((size_t)CHUNKS * Mode<T>::kSteps * Mode<T>::kPieces * NT + kKeptWaves * 4) * 1024;
    const int turns = std::max(1, (shared > kKeptLds / 2 ? 32 : 64) / blocks);
    auto launch = [&](auto* fn) {
        SAR_HIP(hipFuncSetAttribute(reinterpret_cast<const void*>(fn), hipFuncAttributeMaxDynamicSharedMemorySize, (int)shared));
        fn<<<(unsigned)(8 * blocks * turns), kKeptThreads, shared, st>>>(a);
        SAR_LAUNCH_CHECK();
        return (int)SAR_OK;
    };
    if constexpr (E::kAny) {
        if (e.res) return launch(k_rows_kept<T, NT, CHUNKS, TRANS, true, E, Q>);
    }
    return launch(k_rows_kept<T, NT, CHUNKS, TRANS, false, E, Q>);
}

template <typename T, bool TRANS, typename E, typename Q = NoPrologue>
int run_kept(const void* A, const float* W, int64_t n, void* out, int K, int F, void* work, hipStream_t st, const E& e, const Q& q = {})
{
    switch (((TRANS ? F : K) + kChunk<T> - 1) / kChunk<T>) {
    case 1: return run_kept_chunks<T, 1, TRANS>(A, W, n, out, K, F, work, st, e, q);
    case 2: return run_kept_chunks<T, 2, TRANS>(A, W, n, out, K, F, work, st, e, q);
    case 3: return run_kept_chunks<T, 3, TRANS>(A, W, n, out, K, F, work, st, e, q);
    default: return run_kept_chunks<T, 4, TRANS>(A, W, n, out, K, F, work, st, e, q);
    }
}

}  // namespace
}  // namespace sar
