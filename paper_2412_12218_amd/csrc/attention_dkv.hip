// Attention between all nodes of a graph: the kernel of dK and dV.  See attention_common.hpp.
//
// A wave has 32 keys and walks over the virtual rows of their graph's queries, its K and V in registers.  Where these, dK and dV
// would leave a SIMD one wave (16 bits, D above 64), K and V of the workgroup's keys are in LDS instead and a second set of waves has the
// same keys and every second 32 rows; the two sums are added at the end.
//
// Measured as the forward kernel: D = 64 93 us, 418 TFLOP/s; D = 128 1900 us, 683 TFLOP/s (four products).  There a CU's four waves read 192 KB of LDS, 1500 cycles, for
// every 1024 cycles of matrix instructions; K and V in registers, one wave a SIMD, took 2951 us.
#include "attention_common.hpp"

namespace ftc {

template <class T, int NW>
constexpr int query_rows() { return T::BYTES == 2 && NW > 1 ? 64 : 32; }

// Sets of waves that share the keys.
template <class T, int DP, int NW>
constexpr int wave_sets() { return T::BYTES == 2 && DP == 128 && NW == 4 ? 2 : 1; }

template <class T, int DP, int NW, bool WHOLE>
__global__ __launch_bounds__(64 * NW * (wave_sets<T, DP, NW>()), DP == 128 && (wave_sets<T, DP, NW>()) == 1 ? 1 : 2) void attention_dkv_kernel(AttnArgs a)
{
    constexpr int SETS = wave_sets<T, DP, NW>(), THREADS = 64 * NW * SETS;
    constexpr int TK = 32 * NW, TQ = query_rows<T, NW>(), SUB = TQ / 32 / SETS, KS = DP / 16, DT = DP / 32, BUFFERS = tile_buffers<NW>();
    constexpr float P_BACK = 1.f / (1 << p_bits<T>());
    typedef LdsTile<T, DP> L;
    typedef Rows<T, DP, TQ, THREADS, WHOLE> R;
    typedef Rows<T, DP, TK, THREADS, WHOLE> KeyRows;
    __shared__ __align__(16) char Qs[BUFFERS][R::BYTES], Gs[BUFFERS][R::BYTES], Ks[SETS == 2 ? KeyRows::BYTES : 16], Vs[SETS == 2 ? KeyRows::BYTES : 16];
    __shared__ __align__(16) float lses[BUFFERS][TQ], deltas[BUFFERS][TQ];
    const int lane = threadIdx.x & 63, wave = (threadIdx.x >> 6) % NW, set = (threadIdx.x >> 6) / NW, col = lane & 31, half = lane >> 5;
    const Place here = place_of(a);
    const Tile tile = find_tile<TK>(a.kv_ptr, a.graphs, a.n_kv, 1, here.tile, a.tiles);
    if (tile.graph < 0) return;
    const int k0 = tile.begin, k1 = tile.end;
    if (k1 <= k0 || static_cast<int64_t>(tile.index) * TK >= k1 - k0) return;
    const bool same = a.kv_ptr == a.q_ptr && a.n_kv == a.n_q;  // uniform
    const int q0 = same ? k0 : clamped(a.q_ptr, tile.graph, a.n_q), q1 = same ? k1 : clamped(a.q_ptr, tile.graph + 1, a.n_q);
    const int rows = max(q1 - q0, 0) * a.group, tiles = (rows + TQ - 1) / TQ;
    const int each = (tiles + a.splits - 1) / a.splits, first = here.part * each, last = min(tiles, first + each);

    const int key = k0 + tile.index * TK + wave * 32 + col;
    const bool there = key < k1, seen = there && (!a.mask || a.mask[key]);
    R qs, gs;
    float my_lse, my_delta;
    auto get = [&](int t, char *Q, char *G) {
        if (t >= last) return;
        // rows from the query of the tile's first virtual row on
        int q_first, h_first;
        split_row(a, t * TQ, q_first, h_first);
        q_first = __builtin_amdgcn_readfirstlane(q_first);
        const char *qp = head_of<T>(a.Q, q0 + q_first, a.ldq, here.share * a.group * a.D), *gp = head_of<T>(a.dO, q0 + q_first, a.lddo, here.share * a.group * a.D);
        const typename R::Offset ldq = a.ldq, ldg = a.lddo;
        const bool full = (t + 1) * TQ <= rows;
#pragma unroll
        for (int e = 0; e < R::EACH; ++e) {
            uint32_t q = R::row(e), c = R::col(e);
            if (a.group > 1) {
                int query, head;
                split_row(a, t * TQ + R::row(e), query, head);
                q = query - q_first;
                c += head * a.D;
            }
            if (full || t * TQ + R::row(e) < rows) {
                qs.get(Q, e, qp, q * ldq + c, a.D);
                gs.get(G, e, gp, q * ldg + c, a.D);
            } else {
                qs.get_zeros(Q, e);
                gs.get_zeros(G, e);
            }
        }
        if (static_cast<int>(threadIdx.x) < TQ) {
            const int r = t * TQ + threadIdx.x;
            my_lse = -INFINITY;  // no probabilities behind the last row
            my_delta = 0.f;
            if (r < rows) {
                int query, head;
                split_row(a, r, query, head);
                const int64_t at = static_cast<int64_t>(q0 + query) * a.heads + here.share * a.group + head;
                const float lse = a.lse[at];
                my_lse = lse == -INFINITY ? -INFINITY : fmaf(-lse, LOG2E, p_bits<T>());
                my_delta = a.delta[at] * P_BACK;
            }
        }
    };
    auto put = [&](int t, char *Q, char *G, float *row_lse, float *row_delta) {
        if (t < last) {
            qs.put(Q, a.D);
            gs.put(G, a.D);
            if (static_cast<int>(threadIdx.x) < TQ) {
                row_lse[threadIdx.x] = my_lse;
                row_delta[threadIdx.x] = my_delta;
            }
        }
        if constexpr (WHOLE) wait_for_lds_loads();
        __syncthreads();
    };
    for (int b = 0; b < BUFFERS; ++b) {
        R::clear(Qs[b], a.D);
        R::clear(Gs[b], a.D);
    }
    if (WHOLE && a.D < DP) __syncthreads();
    get(first, Qs[0], Gs[0]);
    Frag<T> k[SETS == 2 ? 1 : KS], v[SETS == 2 ? 1 : KS];
    if constexpr (SETS == 2) {
        const int first_key = k0 + tile.index * TK;
        const char *kp = head_of<T>(a.K, first_key, a.ldk, here.share * a.D), *vp = head_of<T>(a.V, first_key, a.ldv, here.share * a.D);
        const typename R::Offset ldk = a.ldk, ldv = a.ldv;
        KeyRows kr, vr;
        KeyRows::clear(Ks, a.D);
        KeyRows::clear(Vs, a.D);
        if (WHOLE && a.D < DP) __syncthreads();
#pragma unroll
        for (int e = 0; e < KeyRows::EACH; ++e) {
            const int j = first_key + KeyRows::row(e);
            if (j < k1 && (!a.mask || a.mask[j])) {
                kr.get(Ks, e, kp, KeyRows::row(e) * ldk + KeyRows::col(e), a.D);
                vr.get(Vs, e, vp, KeyRows::row(e) * ldv + KeyRows::col(e), a.D);
            } else {
                kr.get_zeros(Ks, e);
                vr.get_zeros(Vs, e);
            }
        }
        kr.put(Ks, a.D);
        vr.put(Vs, a.D);
    } else {
        const char *k_row = head_of<T>(a.K, seen ? key : k0, a.ldk, here.share * a.D), *v_row = head_of<T>(a.V, seen ? key : k0, a.ldv, here.share * a.D);
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            const int c = 16 * s + 8 * half;
            k[s] = operand_at<T, WHOLE>(k_row, c, a.D, seen);
            v[s] = operand_at<T, WHOLE>(v_row, c, a.D, seen);
        }
    }
    auto key_operand = [&](int s) {
        if constexpr (SETS == 2) return L::along_row(Ks + 32 * wave * L::ROW, col, 2 * s + half);
        else return k[s];
    };
    auto value_operand = [&](int s) {
        if constexpr (SETS == 2) return L::along_row(Vs + 32 * wave * L::ROW, col, 2 * s + half);
        else return v[s];
    };
    const float scale2 = a.scale * LOG2E;
    const bool busy = k0 + tile.index * TK + wave * 32 < k1;  // uniform in the wave, which has keys
    f32x16 dk[DT], dv[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d) { dk[d] = zero16(); dv[d] = zero16(); }

    // products of 32 rows with the keys: <q, k> and <dO, v>
    auto scores = [&](const char *Q, const char *G, int u, f32x16 &p, f32x16 &ds) {
        p = zero16();
        ds = zero16();
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            mma<T>(p, L::along_row(Q + 32 * u * L::ROW, col, 2 * s + half), key_operand(s));
            mma<T>(ds, L::along_row(G + 32 * u * L::ROW, col, 2 * s + half), value_operand(s));
        }
    };
    // 2^p_bits p and ds from them
    auto weights = [&](const float *row_lse, const float *row_delta, int u, f32x16 &p, f32x16 &ds) {
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            const ftc_f32x4 w = *reinterpret_cast<const ftc_f32x4 *>(&row_lse[32 * u + 8 * b + 4 * half]);
            const ftc_f32x4 x = *reinterpret_cast<const ftc_f32x4 *>(&row_delta[32 * u + 8 * b + 4 * half]);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                p[4 * b + i] = __builtin_amdgcn_exp2f(fmaf(p[4 * b + i], scale2, w[i]));
                ds[4 * b + i] = p[4 * b + i] * fmaf(ds[4 * b + i], P_BACK, -x[i]);
            }
        }
    };
    auto gather = [&](const char *Q, const char *G, int u, const f32x16 &p, const f32x16 &ds) {
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const Frag<T> pf = operand_of<T>(p, s), df = operand_of<T>(ds, s);
            Frag<T> low;
            const bool two = ds_in_two<T, DP>() || (T::BYTES == 2 && NW == 1 && tiles == 1);
            if (two) low = rest_of<T>(ds, s, df);
            const int r0 = (32 * u + 16 * s) * L::ROW;
#pragma unroll
            for (int d = 0; d < DT; ++d) {
                mma<T>(dv[d], L::along_column(G + r0, 4 * half, 4 * half + 8, 32 * d), pf);
                const Frag<T> qf = L::along_column(Q + r0, 4 * half, 4 * half + 8, 32 * d);
                mma<T>(dk[d], qf, df);
                if (two) mma<T>(dk[d], qf, low);
            }
        }
    };
    // The products of one 32 rows run beside the exponentials of the other (a wave's matrix instructions take 32 cycles, 4 to issue).
    auto attend = [&](const char *Q, const char *G, const float *row_lse, const float *row_delta) {
        if (!busy) return;
        f32x16 p0, ds0, p1, ds1;
        const int u0 = SETS == 2 ? set : 0;
        scores(Q, G, u0, p0, ds0);
        if constexpr (SUB == 2) {
            __builtin_amdgcn_sched_barrier(0);
            scores(Q, G, 1, p1, ds1);
            weights(row_lse, row_delta, 0, p0, ds0);
            __builtin_amdgcn_sched_barrier(0);
            gather(Q, G, 0, p0, ds0);
            weights(row_lse, row_delta, 1, p1, ds1);
            __builtin_amdgcn_sched_barrier(0);
            gather(Q, G, 1, p1, ds1);
        } else {
            weights(row_lse, row_delta, u0, p0, ds0);
            gather(Q, G, u0, p0, ds0);
        }
    };
    if constexpr (BUFFERS == 1) {
        for (int t = first; t < last; ++t) {
            if (t > first) get(t, Qs[0], Gs[0]);
            put(t, Qs[0], Gs[0], lses[0], deltas[0]);
            attend(Qs[0], Gs[0], lses[0], deltas[0]);
            __syncthreads();
        }
    } else {
        // one buffer is read while the next tile is on its way to the other (restrict: its arrival need not be waited for before)
        auto turn = [&](int t, const char *__restrict__ Q, const char *__restrict__ G, const float *__restrict__ row_lse,
                        const float *__restrict__ row_delta, char *__restrict__ Qn, char *__restrict__ Gn, float *__restrict__ lse_n,
                        float *__restrict__ delta_n) {
            get(t + 1, Qn, Gn);
            attend(Q, G, row_lse, row_delta);
            put(t + 1, Qn, Gn, lse_n, delta_n);
        };
        put(first, Qs[0], Gs[0], lses[0], deltas[0]);
        for (int t = first, b = 0; t < last; ++t, b ^= 1) turn(t, Qs[b], Gs[b], lses[b], deltas[b], Qs[b ^ 1], Gs[b ^ 1], lses[b ^ 1], deltas[b ^ 1]);
    }
    if constexpr (SETS == 2) {  // dK, then dV of the second set, where the queries were
        static_assert(sizeof(Qs) + sizeof(Gs) >= NW * DT * 4 * 1024, "room for a sum of every wave");
        auto add = [&](f32x16(&sum)[DT]) {
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int b = 0; b < 4; ++b) {
                    const int at = (wave * DT + d) * 4 + b;
                    ftc_f32x4 *to = reinterpret_cast<ftc_f32x4 *>(at < static_cast<int>(sizeof(Qs) / 1024) ? &Qs[0][0] + at * 1024 : &Gs[0][0] + at * 1024 - sizeof(Qs)) + lane;
                    if (set == 1) {
                        *to = ftc_f32x4{sum[d][4 * b], sum[d][4 * b + 1], sum[d][4 * b + 2], sum[d][4 * b + 3]};
                    }
                }
            __syncthreads();
            if (set == 0) {
#pragma unroll
                for (int d = 0; d < DT; ++d)
#pragma unroll
                    for (int b = 0; b < 4; ++b) {
                        const int at = (wave * DT + d) * 4 + b;
                        const ftc_f32x4 x = reinterpret_cast<const ftc_f32x4 *>(at < static_cast<int>(sizeof(Qs) / 1024) ? &Qs[0][0] + at * 1024 : &Gs[0][0] + at * 1024 - sizeof(Qs))[lane];
#pragma unroll
                        for (int i = 0; i < 4; ++i) sum[d][4 * b + i] += x[i];
                    }
            }
            __syncthreads();
        };
        add(dk);
        add(dv);
        if (set == 1) return;
    }
    if (!there) return;
    const int64_t all = static_cast<int64_t>(a.n_kv) * a.kv_heads;
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            const int c = 32 * d + 8 * b + 4 * half;
            float x[4], y[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {  // a key that is not seen was a column of zeros like any other so far
                x[i] = seen ? dk[d][4 * b + i] * a.scale : 0.f;
                y[i] = seen ? dv[d][4 * b + i] * P_BACK : 0.f;
            }
            if (a.splits > 1) {
                const int64_t row = (static_cast<int64_t>(here.part) * 2 * a.n_kv + key) * a.kv_heads + here.share;
                store_four<F32>(a.part, row * a.D + c, a.D - c, x);
                store_four<F32>(a.part, (row + all) * a.D + c, a.D - c, y);
            } else {
                store_four<T>(a.dK, key * a.lddk + here.share * a.D + c, a.D - c, x);
                store_four<T>(a.dV, key * a.lddv + here.share * a.D + c, a.D - c, y);
            }
        }
}

template <class T, int DP, int NW>
constexpr int attention_dkv_kernel_threads() { return 64 * NW * wave_sets<T, DP, NW>(); }

void launch_attention_dkv(const AttnArgs &a, int dtype, int nw, bool whole, unsigned grid, hipStream_t s) { FTC_ATTN_TYPES(attention_dkv_kernel); }

}  // namespace ftc
