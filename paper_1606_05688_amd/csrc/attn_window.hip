// attn_window.hip -- attention with a sliding window and first tokens that stay visible, over sequences of any lengths.
//
// A workgroup has 128 rows of one key and value head (64 or 32, where there are few): tokens times the query heads that share it, so that
// keys and values are read once for all of them; a wave has 32 rows.  It walks the key tiles that any row sees (sinks, then the
// window), two to four of them in LDS, loads going from memory to LDS without registers in between.  Per tile, on 32x32 products:
//   scores^T [keys][32 rows] = K Q^T: a lane has one row, half of its scores; maximum and weights are lane-local but for one
//   exchange; the weights as they stand are the right operand of  out^T [D][32 rows] += V^T W^T.
// V^T's operand: 16-bit types by transposing LDS reads, fp32 (products of fp32) by plain ones, keys permuted to match.
// Rows in LDS are permuted by 16-byte chunks so that neither kind of read meets a bank twice.
// Rounded: 16-bit weights to their type before the second product (at most 2^8 times a row's largest then; two values of the type where a
// sequence has few rows), sums stay fp32.
//
// bf16, 16384 tokens, window of 4096, heads 16 of 4 x 128: 484 to 503 us by card, 960 to 997 TFLOP/s, against 1090 of a large bf16 product.  Bound
// by the LDS reads of a wave (32 KB a tile, each used for 32 rows), the weights' instructions between the products, and the clock, which falls to
// 2.2 GHz.  fp32, 2744 tokens, heads 5 x 40: 40 us and 4 for the join, matrix units busy for a third.  16-bit calls of few rows: one
// wave's chain of a tile, 1.1 us.  Values that are not finite cost two more walks: that volume with one infinity 636 us, all NaN 2030.
#include <type_traits>

#include "attn_join.h"
#include "attn_tile.h"

namespace znni {

constexpr int BM = 128, ATTN_THREADS = 256;

// What a score is multiplied by to count powers of two (queries have the sign).  Of a scale of 0: the least there is, with which scores of
// 2^128 are 2^-21 and what is masked stays so.
__host__ __device__ inline float powers_of(float scale) { return scale == 0.f ? 0x1p-149f : fabsf(scale) * 1.44269504088896340736f; }

// The x lowest bits.
__device__ inline unsigned lowest(int x) { return x <= 0 ? 0u : ~0u >> (32 - min(x, 32)); }

// SHARE waves share 32 rows, 128 / SHARE rows a workgroup.  Two: each has half of a tile's keys, their sums are joined at the end.  Four (fp32, whose
// tile has no more keys than a product): each has a quarter of the head's elements, in the scores, whose parts are added through LDS, and
// in the results; softmax statistics are the same in all four.
// TWICE (16-bit types): weights as two values of the type, for few rows.
template <typename T, int NC, int SHARE, bool TWICE>
__global__ __launch_bounds__(ATTN_THREADS, 2) void k_attn(AttnArgs a, Heads<const T> q, Heads<const T> k, Heads<const T> v, Heads<T> out)
{
    using G = AttnTile<T, NC, ATTN_THREADS>;
    using M = Mfma<T>;
    constexpr bool F32 = G::F32;
    constexpr bool BY_D = F32 && SHARE == 4;
    constexpr int BN = G::BN, EC = G::EC, RS = G::RS, CR = G::CR, PER = G::PER;
    constexpr int ROWS = BM / SHARE, KT = BY_D ? 1 : BN / 32 / SHARE, NA = BY_D ? 1 : NC;
    constexpr int STAGES = G::STAGES, ONE = STAGES > 2 ? 2 * PER : 0, TWO = STAGES > 3 ? 4 * PER : 0;      // loads of tiles behind the present one
    __shared__ __align__(1024) T ks[STAGES][BN * RS];
    __shared__ __align__(1024) T vs[STAGES][BN * RS];
    __shared__ float4 partial[BY_D ? 4 * 4 * 64 : 1];          // scores of a wave's elements; a flag

    const long long group = group_id();
    if (group >= a.groups) return;
    // whether x holds anywhere in the workgroup
    auto any_of_all = [&](bool x) {
        int* const flag = (int*)partial;
        __syncthreads();
        if (threadIdx.x == 0) *flag = 0;
        __syncthreads();
        if (__any(x) && (threadIdx.x & 63) == 0) *flag = 1;
        __syncthreads();
        const int y = __builtin_amdgcn_readfirstlane(*flag);
        __syncthreads();
        return y;
    };
    int id = in_runs((int)group, a.groups);
    const int split = id % a.splits; id /= a.splits;
    const int tile = a.tiles - 1 - id % a.tiles; id /= a.tiles;
    const int hk = id % a.Hk, b = id / a.Hk;
    const int q0 = a.cu_q[b], nq = a.cu_q[b + 1] - q0, k0 = a.cu_k[b], nk = a.cu_k[b + 1] - k0;
    const int shared = a.Hq / a.Hk;
    const long long rows = (long long)min(nq, a.max_q) * shared, row0 = (long long)tile * ROWS;
    if (row0 >= rows) return;
    const int t = threadIdx.x, l = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6), c32 = l & 31, h = l >> 5;
    const long long base = (long long)nk - nq, last = min(row0 + ROWS, rows) - 1;
    const int part = wave % SHARE, wrow = wave / SHARE * 32, key_part = BY_D ? 0 : part * KT * 32;
    const long long wrow0 = row0 + wrow;
    const Sight all_rows(base + row0 / shared, base + last / shared, nk, a.w);
    const Sight wave_rows(base + wrow0 / shared, base + (wrow0 < rows ? min(wrow0 + 31, last) / shared : wrow0 / shared - 1), nk, a.w);
    const long long row = min(wrow0 + c32, rows - 1);
    const long long pos = base + row / shared;                                         // of the lane
    int lo, hi;
    window_of(pos, nk, a.w, &lo, &hi);
    const int qh = hk * shared + (int)(row % shared);

    const KeyTiles<BN> tiles(all_rows);
    const int per = (tiles.n + a.splits - 1) / a.splits, begin = split * per, end = min(tiles.n, begin + per);

    // what this thread brings of a tile: PER chunks of keys and of values, 64 consecutive ones a wave
    const T* kp = k.row(k0, hk);
    const T* vp = v.row(k0, hk);
    const bool near = k.token >= 0 && v.token >= 0 && k.token < (1 << 22) && v.token < (1 << 22);
    constexpr unsigned TILE = BN * RS * sizeof(T);
    const unsigned k_lds = lds_address(ks) + wave * 1024, v_lds = lds_address(vs) + wave * 1024;
    unsigned ko[PER], vo[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int slot = (i * 4 + wave) * 64 + l, j = slot / CR, c = slot % CR;
        ko[i] = ((unsigned)j * (unsigned)k.token + (c ^ G::swizzle_k(j)) * EC) * (unsigned)sizeof(T);
        vo[i] = ((unsigned)j * (unsigned)v.token + (c ^ G::swizzle_v(j)) * EC) * (unsigned)sizeof(T);
    }
    // (every wave has 2 PER loads a tile in flight, whichever way: some of its lanes have a chunk of the head)
    auto bring = [&](int it) {
        const int buf = (it - begin) % STAGES, j0 = tiles.base(it);
        if (near && a.D == RS && j0 + BN <= nk) {
            const char* kt = (const char*)(kp + j0 * k.token);
            const char* vt = (const char*)(vp + j0 * v.token);
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                to_lds(kt, ko[i], k_lds + buf * TILE + i * 4096);
                to_lds(vt, vo[i], v_lds + buf * TILE + i * 4096);
            }
            return;
        }
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int slot = (i * 4 + wave) * 64 + l, j = slot / CR, ck = slot % CR ^ G::swizzle_k(j), cv = slot % CR ^ G::swizzle_v(j);
            const long long jj = min(j0 + j, nk - 1);
            if (ck * EC < a.D) to_lds(kp + jj * k.token + ck * EC, k_lds + buf * TILE + i * 4096);
            if (cv * EC < a.D) to_lds(vp + jj * v.token + cv * EC, v_lds + buf * TILE + i * 4096);
        }
    };
    // chunks past a head's end are never brought: zero
    if (a.D < RS)
        for (int i = t; i < STAGES * BN * CR; i += ATTN_THREADS) {
            const int slot = i % (BN * CR), j = slot / CR;
            if ((slot % CR ^ G::swizzle_k(j)) * EC >= a.D) *(uint4*)&ks[i / (BN * CR)][slot * EC] = make_uint4(0, 0, 0, 0);
            if ((slot % CR ^ G::swizzle_v(j)) * EC >= a.D) *(uint4*)&vs[i / (BN * CR)][slot * EC] = make_uint4(0, 0, 0, 0);
        }

    auto bring_first = [&] {
#pragma unroll
        for (int i = 0; i < STAGES - 1; ++i)
            if (begin + i < end) bring(begin + i);
    };
    bring_first();

    // queries: the right operand of the scores
    constexpr int QS = BY_D ? RS / 32 : F32 ? 4 * NC : 2 * NC;       // steps of 8 (4 a lane, in fp32) or 16 elements (8 a lane)
    const int q_part = BY_D ? part * QS : 0, d_part = BY_D ? part * 32 : 0;       // the wave's first step, its first element of results
    typename M::V qf[QS];
    {
        const T* p = q.row(q0 + row / shared, qh);
#pragma unroll
        for (int c = 0; c < QS; ++c) {
            const int d = (2 * (q_part + c) + h) * EC;
            if (d < a.D) qf[c] = *(const typename M::V*)(p + d);
            else
#pragma unroll
                for (int e = 0; e < EC; ++e) qf[c][e] = (T)0.f;
            // a negative scale turns the queries, so that the largest product is the largest score
            if (a.scale < 0.f)
#pragma unroll
                for (int e = 0; e < EC; ++e) qf[c][e] = -qf[c][e];
        }
    }

    const float by = powers_of(a.scale);
    const float ahead = fminf(8.f / by, 3.402823466e38f);          // (finite: minus infinity and this is minus infinity)
    // where this lane reads: keys row c32 (and 32 on), chunk h ^ ... of step 0, other steps by exclusive or; values likewise
    const int r4 = l >> 2 & 3, c4 = l & 3, g16 = l >> 4 & 1;
    int k_at = (((key_part + c32) * RS + (h ^ G::swizzle_k(c32)) * EC) * (int)sizeof(T)) ^ q_part * 32;
    int v_at = F32 ? (((key_part + 4 * h) * RS + (c32 ^ G::swizzle_v(4 * h) * EC)) * (int)sizeof(T)) ^ d_part * 4
                   : ((key_part + 4 * h + r4) * RS + ((2 * g16 + (c4 >> 1)) ^ G::swizzle_v(4 * h + r4)) * EC + (c4 & 1) * 4) * (int)sizeof(T);

    f32x16 acc[NA];
    float top, sum, off;            // sums stand for weights of 2^(by (s - top) + off)
    // one bit for each of 32 keys: whether the lane's row sees them
    auto sight = [&](int j) { return lowest(hi + 1 - j) & (~lowest(lo - j) | lowest(a.w.sinks - j)); };
    // adds 32 elements of the head (from 32 x on) of values of 32 keys (32 n on), times weights of this lane's row: 16 of those keys
    auto add_values = [&](f32x16& to, const char* from, int x, int n, auto weight) {
        if constexpr (F32) {
#pragma unroll
            for (int i = 0; i < 16; ++i)
                to = M::mul(*(const T*)(from + (v_at ^ x * 128) + (8 * (i / 4) + i % 4) * RS * (int)sizeof(T)), weight(i), to);
        } else {
#pragma unroll
            for (int m = 0; m < 2; ++m) {
                typename M::V w;
#pragma unroll
                for (int e = 0; e < 8; ++e) w[e] = (T)weight(8 * m + e);
                const char* p = from + (v_at ^ x * 64) + 16 * (2 * n + m) * RS * (int)sizeof(T);
                const typename M::V4 y0 = transposed<typename M::V4>(p), y1 = transposed<typename M::V4>(p + 8 * RS * (int)sizeof(T));
                to = M::mul(__builtin_shufflevector(y0, y1, 0, 1, 2, 3, 4, 5, 6, 7), w, to);
            }
        }
    };

    // values of a tile, each thread its own chunks
    auto change = [&](T* tile, auto to) {
        typedef T Chunk __attribute__((ext_vector_type(EC)));
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            Chunk* const at = (Chunk*)(tile + (i * ATTN_THREADS + t) * EC);
            Chunk y = *at;
#pragma unroll
            for (int e = 0; e < EC; ++e) y[e] = to(y[e]);
            *at = y;
        }
    };

    // Values that are not finite leave their mark on rows that do not see them (their weight is zero, and zero times those is NaN), and
    // infinities under weights that round to zero become NaN.  So the walk over the keys takes place without a thought for them, and where a result
    // is not finite twice more: products of the values' kinds with zeros and ones say which kinds a row sees; then such values are taken out of
    // the tiles, and the row gets what it sees at the end, whatever the weight.  The maximum is followed at once there, so that sums of values next
    // to the largest do not pass it before they are rescaled.
    auto walk = [&](auto carefully) {
        constexpr bool careful = decltype(carefully)::value;
#pragma unroll
        for (int x = 0; x < NA; ++x)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[x][i] = 0.f;
        top = -INFINITY;
        sum = 0.f;
        float shift = 0.f;
        bool wild = false;
        if constexpr (careful) bring_first();
        for (int it = begin; it < end; ++it) {
            const int buf = (it - begin) % STAGES, j0 = tiles.base(it);
            // this tile is there, the ones behind it may be on their way
            if (STAGES > 3 && it + 2 < end) wait_but_and_meet<TWO>();
            else if (STAGES > 2 && it + 1 < end) wait_but_and_meet<ONE>();
            else wait_but_and_meet<0>();
            if (it + STAGES - 1 < end) bring(it + STAGES - 1);
            if constexpr (careful) {
                change(vs[buf], [](T y) { return kind_of((float)y) == 0.f ? y : (T)0.f; });
                __syncthreads();
            }
            const int wj0 = j0 + key_part;                   // of the wave
            if (!wave_rows.any(wj0, 32 * KT)) continue;

            // (worked out again for every tile: kept, the addresses of all steps would take the registers)
            asm volatile("" : "+v"(k_at), "+v"(v_at));
            const char* kb = (const char*)ks[buf];
            const char* vb = (const char*)vs[buf];
            f32x16 s[KT];
#pragma unroll
            for (int n = 0; n < KT; ++n)
#pragma unroll
                for (int i = 0; i < 16; ++i) s[n][i] = 0.f;
#pragma unroll
            for (int c = 0; c < QS; ++c) {
                if (F32 && 8 * (q_part + c) >= a.D) continue;           // (256 cycles a step; in 16-bit types 32, which a branch would cost)
#pragma unroll
                for (int n = 0; n < KT; ++n) {
                    const typename M::V x = *(const typename M::V*)(kb + (k_at ^ c * 32) + n * 32 * RS * (int)sizeof(T));
                    if constexpr (F32) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) s[n] = M::mul(x[e], qf[c][e], s[n]);
                    } else {
                        s[n] = M::mul(x, qf[c], s[n]);
                    }
                }
            }
            // reads run four ahead of the products (left alone, the compiler waits for each)
            if constexpr (!F32) {
                __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
#pragma unroll
                for (int n = 0; n < QS * KT; ++n) {
                    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                    __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
                }
            }
            if constexpr (BY_D) {
                // so far of this wave's elements of the head
                float4* const mine = partial + part * 256 + l;
#pragma unroll
                for (int i = 0; i < 4; ++i) mine[i * 64] = make_float4(s[0][4 * i], s[0][4 * i + 1], s[0][4 * i + 2], s[0][4 * i + 3]);
                wait_and_meet();
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float4* const p = partial + i * 64 + l;
                    const float4 y0 = p[0], y1 = p[256], y2 = p[512], y3 = p[768];
                    s[0][4 * i] = (y0.x + y1.x) + (y2.x + y3.x);
                    s[0][4 * i + 1] = (y0.y + y1.y) + (y2.y + y3.y);
                    s[0][4 * i + 2] = (y0.z + y1.z) + (y2.z + y3.z);
                    s[0][4 * i + 3] = (y0.w + y1.w) + (y2.w + y3.w);
                }
                if (d_part >= a.D) continue;
            }
            if (!wave_rows.all(wj0, 32 * KT)) {
#pragma unroll
                for (int n = 0; n < KT; ++n) {
                    const unsigned mine = sight(wj0 + n * 32) >> 4 * h;       // two instructions a score
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const int m = (int)(mine << (31 - 8 * (i / 4) - i % 4)) >> 31;
                        s[n][i] = __int_as_float((__float_as_int(s[n][i]) & m) | (0xff800000 & ~m));
                    }
                }
            }
            float mx[4];
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                mx[x] = s[0][x];
#pragma unroll
                for (int i = 1; i < 4 * KT; ++i) mx[x] = __builtin_elementwise_maximum(mx[x], s[i / 4][4 * (i % 4) + x]);
            }
            float most = __builtin_elementwise_maximum(__builtin_elementwise_maximum(mx[0], mx[1]), __builtin_elementwise_maximum(mx[2], mx[3]));
            // Weights are 2^(by (s - top)), as one multiply-add of `shift` = -by top.  `top` follows the maximum when that is 2^8 ahead:
            // weights stay in the range of every type, and most tiles have nothing to rescale.  What the rounding of by * top leaves, by * top +
            // shift, is in all weights of a row until `top` moves, and is made good there and where sums are joined.  It may be so large that
            // weights would leave the range of the type: then the difference comes first, which leaves nothing.
            float offset = shift;
            if (wild || __any(most > top + (careful ? 0.f : ahead))) {
                most = fmaxf(fmaxf(most, __shfl_xor(most, 32)), top);
                const float zero = most == -INFINITY ? 0.f : most, now = -zero * by;
                const bool far = __any(!(fabsf(now) < 0x1p26f));
                const float was = wild ? 0.f : fmaf(top, by, shift), is = far ? 0.f : fmaf(zero, by, now);
                const float old = top == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((top - zero) * by + (is - was));
                sum *= old;
#pragma unroll
                for (int x = 0; x < NA; ++x) acc[x] *= old;
                top = most;
                wild = far;
                offset = shift = now;
                if (wild) {
#pragma unroll
                    for (int n = 0; n < KT; ++n) s[n] -= zero;
                    offset = 0.f;
                }
            }
            float part[2] = {0.f, 0.f};
            if constexpr (F32) {
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const float w = __builtin_amdgcn_exp2f(fmaf(s[0][i], by, offset));
                    part[i & 1] += w;
#pragma unroll
                    for (int x = 0; x < NA; ++x)
                        acc[x] = M::mul(*(const T*)(vb + (v_at ^ x * 128) + (8 * (i / 4) + i % 4) * RS * (int)sizeof(T)), w, acc[x]);
                }
                __builtin_amdgcn_sched_group_barrier(0x100, 8, 0);
#pragma unroll
                for (int n = 0; n < 16 * NA; ++n) {
                    __builtin_amdgcn_sched_group_barrier(0x002, 4, 0);
                    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                    __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
                }
            } else {
#pragma unroll
                for (int n = 0; n < 2 * KT; ++n) {
                    typename M::V w, rest;
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float p = __builtin_amdgcn_exp2f(fmaf(s[n / 2][8 * (n & 1) + e], by, offset));
                        part[e & 1] += p;
                        w[e] = (T)p;
                        if constexpr (TWICE) rest[e] = (T)(p - (float)w[e]);
                    }
#pragma unroll
                    for (int x = 0; x < NA; ++x) {
                        const char* from = vb + (v_at ^ x * 64) + 16 * n * RS * (int)sizeof(T);
                        const typename M::V4 y0 = transposed<typename M::V4>(from), y1 = transposed<typename M::V4>(from + 8 * RS * (int)sizeof(T));
                        const typename M::V y = __builtin_shufflevector(y0, y1, 0, 1, 2, 3, 4, 5, 6, 7);
                        acc[x] = M::mul(y, w, acc[x]);
                        if constexpr (TWICE) acc[x] = M::mul(y, rest, acc[x]);
                    }
                }
            }
            sum += part[0] + part[1];
        }
        off = wild || top == -INFINITY ? 0.f : fmaf(top, by, shift);
    };
    walk(std::false_type());
    bool fine = true;
#pragma unroll
    for (int x = 0; x < NA; ++x)
#pragma unroll
        for (int i = 0; i < 16; ++i) fine = fine && fabsf(acc[x][i]) <= 3.402823466e38f;
    const int odd_sums = any_of_all(!fine && d_part < a.D);
    if (__builtin_expect(odd_sums, 0)) {
        unsigned met[NA] = {};                   // for each element of a result whether infinity (16 bits), minus infinity (16 more) are seen
        bring_first();
        for (int it = begin; it < end; ++it) {
            const int buf = (it - begin) % STAGES, j0 = tiles.base(it) + key_part;
            wait_but_and_meet<0>();
            if (it + STAGES - 1 < end) bring(it + STAGES - 1);
            change(vs[buf], [](T y) { return (T)kind_of((float)y); });
            wait_and_meet();
            if (!wave_rows.any(j0, 32 * KT) || d_part >= a.D) continue;
#pragma unroll
            for (int x = 0; x < NA; ++x) {
                f32x16 seen;
#pragma unroll
                for (int i = 0; i < 16; ++i) seen[i] = 0.f;
#pragma unroll
                for (int n = 0; n < KT; ++n) {
                    const unsigned mine = sight(j0 + n * 32) >> 4 * h;
                    add_values(seen, (const char*)vs[buf], x, n, [&](int i) { return (float)(mine >> (8 * (i / 4) + i % 4) & 1); });
                }
#pragma unroll
                for (int i = 0; i < 16; ++i) met[x] |= ((int)seen[i] & 127 ? 1u << i : 0u) | ((int)seen[i] >= 128 ? 0x10000u << i : 0u);
            }
        }
        __syncthreads();
        walk(std::true_type());
#pragma unroll
        for (int x = 0; x < NA; ++x)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[x][i] += (met[x] >> i & 1 ? INFINITY : 0.f) - (met[x] >> (16 + i) & 1 ? INFINITY : 0.f);
    }
    sum += __shfl_xor(sum, 32);
    if constexpr (SHARE == 2) {
        // the second wave's sums by way of the tiles' memory
        float4* const sums = (float4*)&ks[0][0] + wrow / 32 * NC * 256;
        float3* const stat = (float3*)&vs[0][0] + wrow / 32 * 64;
        __syncthreads();
        if (part) {
            stat[l] = make_float3(top, sum, off);
#pragma unroll
            for (int x = 0; x < NA; ++x)
#pragma unroll
                for (int i = 0; i < 16; i += 4) sums[(x * 4 + i / 4) * 64 + l] = make_float4(acc[x][i], acc[x][i + 1], acc[x][i + 2], acc[x][i + 3]);
        }
        __syncthreads();
        if (part) return;
        const float3 theirs = stat[l];
        const float most = fmaxf(top, theirs.x), zero = most == -INFINITY ? 0.f : most;
        const float f0 = __builtin_amdgcn_exp2f((top - zero) * by - off), f1 = __builtin_amdgcn_exp2f((theirs.x - zero) * by - theirs.z);
        top = most;
        off = 0.f;
        sum = f0 * sum + f1 * theirs.y;
        auto join = [&](auto share) {
#pragma unroll
            for (int x = 0; x < NA; ++x)
#pragma unroll
                for (int i = 0; i < 16; i += 4) {
                    const float4 y = sums[(x * 4 + i / 4) * 64 + l];
                    acc[x][i] = share(f0, acc[x][i]) + share(f1, y.x);
                    acc[x][i + 1] = share(f0, acc[x][i + 1]) + share(f1, y.y);
                    acc[x][i + 2] = share(f0, acc[x][i + 2]) + share(f1, y.z);
                    acc[x][i + 3] = share(f0, acc[x][i + 3]) + share(f1, y.w);
                }
        };
        if (__builtin_expect(odd_sums, 0)) join(share_of);
        else join([](float f, float x) { return f * x; });
    }
    if (wrow0 + c32 >= rows) return;
    if (a.splits == 1) {
        T* y = out.row(q0 + row / shared, qh);
        const float inv = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
        for (int x = 0; x < NA; ++x)
#pragma unroll
            for (int i = 0; i < 16; i += 4) {
                const int d = d_part + 32 * x + 2 * i + 4 * h;
                if (d < a.D) {
                    typedef T T4 __attribute__((ext_vector_type(4)));
                    T4 o;
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[e] = (T)(sum == 0.f ? 0.f : acc[x][i + e] * inv);
                    *(T4*)(y + d) = o;
                }
            }
    } else {
        const long long at = ((((long long)b * a.Hk + hk) * a.tiles + tile) * a.splits + split) * a.tile_rows + wrow + c32;
        const float even = __builtin_amdgcn_exp2f(-off);
        if (h == 0 && d_part == 0) a.stats[at] = make_float2(top, even * sum);
        float* y = a.parts + at * a.D;
#pragma unroll
        for (int x = 0; x < NA; ++x)
#pragma unroll
            for (int i = 0; i < 16; i += 4) {
                const int d = d_part + 32 * x + 2 * i + 4 * h;
                if (d < a.D) *(float4*)(y + d) = make_float4(even * acc[x][i], even * acc[x][i + 1], even * acc[x][i + 2], even * acc[x][i + 3]);
            }
    }
}

struct AttnPlan {
    int share, tiles, splits, tile_rows;
    bool twice;                        // weights as two values of a 16-bit type
    long long groups;                  // workgroups without splitting
    size_t rows;                       // rows of parts
};

// Few row tiles over many keys: workgroups share the keys of a tile until the chip has two for every compute unit, each with four
// tiles at least.
static AttnPlan attn_plan(int share, int type, int B, int Hq, int Hk, int max_q, int max_k, int left, int right, int sinks)
{
    AttnPlan p;
    const int bm = BM / share;
    p.share = share;
    p.twice = false;
    const long long rows = (long long)max_q * (Hq / Hk);
    const long long tiles = (rows + bm - 1) / bm;
    p.tiles = (int)(tiles < INT_MAX ? tiles : INT_MAX);
    p.groups = tiles * Hk * B;
    p.tile_rows = (int)(rows < bm ? rows : bm);
    const int bn = type == ZNNI_F32 ? 32 : 64;
    const long long tokens = (rows < bm ? max_q : bm / (Hq / Hk) + 2);
    long long seen = (long long)left + right + tokens + (sinks < max_k ? sinks : max_k);
    if (seen > max_k) seen = max_k;
    const long long most = (seen + bn - 1) / bn / 4;
    long long n = p.groups > 0 && p.groups < 512 ? 512 / p.groups : 1;
    if (n > most) n = most;
    p.splits = n < 1 ? 1 : (int)n;
    p.rows = p.splits == 1 ? 0 : (size_t)p.groups * p.splits * p.tile_rows;
    return p;
}

// 16-bit types: with up to three workgroups for two compute units a wave has a SIMD nearly to itself and waits for its own
// instructions: two share the rows.  fp16, heads 8 x 64, 300 queries, window of 100, with 128 and with 64 rows a workgroup: 24 workgroups
// 10.8 and 9.4 us, 288: 13.8 and 11.9, 384: 14.1 and 13.3, 480: 14.6 and 17.7, 768: 18.2 and 23.0; bf16, heads 16 of 4 x 128, 2048
// queries, 256 workgroups: 61.6 and 54.7 us.
// A sequence whose rows fit one such tile (single tokens) is bound by its keys and values, so weights keep the bits that a second value of
// the type holds: error 0.0017 of the result in bf16 as with an fp32 softmax rounded once, 0.0023 with one value.  bf16, heads 16 of 4 x 128, one
// query: 8 sequences of 8192 keys 29.0 us with one value, 29.7 with two, 32 of 500 13.3 and 13.9, one of 16384 18.6 and 19.3.  More rows are bound by
// products: 2048 queries 45.5 and 55.2, 16384 with a window of 4096 495 and 681, fp16, heads 8 x 64, 300 ragged queries 10.7 and 11.6.
// fp32: where one wave's rows are all, the other three would wait for its products (heads 16 of 4 x 128, one query, 8 sequences of 8192
// keys: 89 us with one wave at work, 60 with four; of 500: 27 and 16); and where workgroups are very few (heads 5 x 40, 200 queries: 20.9
// and 16.8, 400: 19.5 and 16.2, 700, 30 workgroups: 21.1 and 24.0; 16 of 4 x 128, 100 queries: 24.6 and 13.0, 256 of 4000 keys: 89 and 105).
static AttnPlan attn_plan(int type, int B, int Hq, int Hk, int max_q, int max_k, int left, int right, int sinks)
{
    AttnPlan p = attn_plan(1, type, B, Hq, Hk, max_q, max_k, left, right, sinks);
    const long long rows = (long long)max_q * (Hq / Hk);
    const bool twice = type != ZNNI_F32 && rows <= BM / 2;
    const int share = type != ZNNI_F32 ? (twice || p.groups <= 384 ? 2 : 1) : p.groups <= 20 || rows <= 32 ? 4 : 1;
    if (share != 1) p = attn_plan(share, type, B, Hq, Hk, max_q, max_k, left, right, sinks);
    p.twice = twice;
    return p;
}

template <typename T>
static znni_status launch_attn(const AttnArgs& a, int B, int max_q, const AttnPlan& p, const znni_heads* q, const znni_heads* k, const znni_heads* v,
                               const znni_heads* out, hipStream_t st)
{
    const dim3 grid = launch_of(a.groups), block(ATTN_THREADS);
    const Heads<const T> qi = heads_of<const T>(q), ki = heads_of<const T>(k), vi = heads_of<const T>(v);
    const Heads<T> o = heads_of<T>(out);
    auto launch = [&](auto share, auto twice) {
        constexpr int SHARE = decltype(share)::value;
        constexpr bool TWICE = decltype(twice)::value;
        switch ((a.D + 31) / 32) {
            case 1: k_attn<T, 1, SHARE, TWICE><<<grid, block, 0, st>>>(a, qi, ki, vi, o); break;
            case 2: k_attn<T, 2, SHARE, TWICE><<<grid, block, 0, st>>>(a, qi, ki, vi, o); break;
            case 3: k_attn<T, 3, SHARE, TWICE><<<grid, block, 0, st>>>(a, qi, ki, vi, o); break;
            default: k_attn<T, 4, SHARE, TWICE><<<grid, block, 0, st>>>(a, qi, ki, vi, o); break;
        }
    };
    if constexpr (sizeof(T) == 2) {
        if (p.twice) launch(std::integral_constant<int, 2>(), std::true_type());
        else if (p.share == 2) launch(std::integral_constant<int, 2>(), std::false_type());
        else launch(std::integral_constant<int, 1>(), std::false_type());
    } else {
        if (p.share == 4) launch(std::integral_constant<int, 4>(), std::false_type());
        else launch(std::integral_constant<int, 1>(), std::false_type());
    }
    if (hipGetLastError() != hipSuccess) return ZNNI_ERR_HIP;
    if (p.splits == 1) return ZNNI_OK;
    const JoinArgs j = {a.Hq, a.Hk, a.D, p.splits, p.tiles, p.tile_rows, max_q * (a.Hq / a.Hk), a.cu_q, 0, powers_of(a.scale), a.parts, a.stats};
    return launch_join<T>(j, B, o, st);
}

static znni_status attn_shape(int type, int B, int Hq, int Hk, int D, int max_q, int max_k, int left, int right, int sinks)
{
    if (!type_ok(type)) return ZNNI_ERR_TYPE;
    if (B < 0 || B > 65535 || max_q < 0 || max_k < 0 || left < 0 || right < 0 || sinks < 0) return ZNNI_ERR_SHAPE;
    const znni_status rc = heads_shape(Hq, Hk, D);
    if (rc) return rc;
    // a workgroup for every row tile and key head
    const long long rows = (long long)max_q * (Hq / Hk), tiles = (rows + BM - 1) / BM;
    return rows > INT_MAX || tiles * Hk > INT_MAX / (B ? B : 1) ? ZNNI_ERR_SHAPE : ZNNI_OK;
}

}  // namespace znni

using namespace znni;

extern "C" {

znni_status znni_attn_window_workspace(int type, int B, int Hq, int Hk, int D, int max_q, int max_k, int left, int right, int sinks,
                                       size_t* bytes)
{
    if (!bytes) return ZNNI_ERR_NULL;
    const znni_status rc = attn_shape(type, B, Hq, Hk, D, max_q, max_k, left, right, sinks);
    if (rc) return rc;
    const AttnPlan p = attn_plan(type, B, Hq, Hk, max_q, max_k, left, right, sinks);
    *bytes = p.rows * (D + 2) * sizeof(float);
    return ZNNI_OK;
}

znni_status znni_attn_window(int type, int B, int Hq, int Hk, int D, const znni_heads* q, const znni_heads* k, const znni_heads* v,
                             const int* cu_q, const int* cu_k, int max_q, int max_k, int left, int right, int sinks, float scale,
                             const znni_heads* out, void* workspace, size_t workspace_bytes, void* stream)
{
    if (!q || !k || !v || !out) return ZNNI_ERR_NULL;
    size_t need = 0;
    const znni_status rc = znni_attn_window_workspace(type, B, Hq, Hk, D, max_q, max_k, left, right, sinks, &need);
    if (rc) return rc;
    if (B == 0 || max_q == 0) return ZNNI_OK;
    if (!q->data || !out->data || (max_k > 0 && (!k->data || !v->data)) || !cu_q || !cu_k || (need && !workspace)) return ZNNI_ERR_NULL;
    if (workspace_bytes < need) return ZNNI_ERR_WORKSPACE;
    if (((uintptr_t)cu_q | (uintptr_t)cu_k) & 3u || (need && ((uintptr_t)workspace & 255u))) return ZNNI_ERR_ALIGN;
    for (const znni_heads* h : {q, k, v, out})
        if (!heads_aligned(h, type)) return ZNNI_ERR_ALIGN;
    const AttnPlan p = attn_plan(type, B, Hq, Hk, max_q, max_k, left, right, sinks);
    float* parts = (float*)workspace;
    const AttnArgs a = {Hq, Hk, D, cu_q, cu_k, {left, right, sinks}, scale, (int)(p.groups * p.splits), max_q, p.tiles, p.splits, p.tile_rows, parts,
                        (float2*)(parts + p.rows * D)};
    const hipStream_t st = (hipStream_t)stream;
    switch (type) {
        case ZNNI_F32: return launch_attn<float>(a, B, max_q, p, q, k, v, out, st);
        case ZNNI_BF16: return launch_attn<bf16>(a, B, max_q, p, q, k, v, out, st);
        default: return launch_attn<f16>(a, B, max_q, p, q, k, v, out, st);
    }
}

}  // extern "C"
