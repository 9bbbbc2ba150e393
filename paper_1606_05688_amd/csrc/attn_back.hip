// attn_back.hip -- gradients of windowed attention: the weights are worked out again from the scores and each row's statistics.
//
//   P = exp(scale q.k - lse),  dP = dout.v,  delta = sum over d of dout out,  dS = P (dP - delta)
//   dv = P^T dout,  dk = scale dS^T q  (sums over the rows, of all query heads that share the key head),  dq = scale dS k
//
// Two kernels of one pattern: a workgroup holds 128 keys (or rows) as operands in registers, 32 a wave, and walks the rows (or keys) that
// see them (or that they see) in tiles through LDS, so that every sum has one owner and one order.  Per 32 x 32 pairs, `loop` the walked side:
//   S [loop][lane] = A a,  dP [loop][lane] = B b     (A, B: q and dout, or k and v, from LDS; a, b: k and v, or q and dout)
//   dA^T [D][lane] += A^T dS,  for keys also dB^T [D][lane] += B^T P     (P and dS as they stand are right operands; A^T, B^T by transposing reads)
// What is taken from a row's scores and its dP is there before the first product, after it, or at the end, as costs least.
//
// bf16, 16384 tokens, window of 4096, heads 16 of 4 x 128: 2100 us in all, 576 TFLOP/s of the five products that it takes, 920 of the eight that run
// (scores twice for wide heads' dk and dv, and again for dq).  Bound by LDS reads, products and exponentials of two waves a SIMD that take turns but for
// the meetings at each tile (matrix units 41 % busy, vector units 35 %), no bank conflicts.  fp16, ragged 300 tokens: 37 us, the chain of three launches.  fp32, 2744
// tokens: 151 us, matrix units of one or two workgroups a unit, 40 of 64 columns useful.  Registers run out in fp32 for heads of 97 to 128 (196 bytes of
// scratch a lane) and where weights are two values for heads of 33 to 64 (bf16 8 bytes, fp16 48) and of 97 to 128 (40 and 56).
#include <initializer_list>
#include <type_traits>

#include "attn_tile.h"
#include "back_parts.h"

namespace znni {

constexpr int BACK_THREADS = 256;

struct BackArgs : BackParts {
    int Hq, Hk, D;
    const int* cu_q;
    const int* cu_k;
    Window w;
    float scale;
    int max_q, max_k;
    int cycle;                        // tiles that a workgroup walks, or 0: they start with their first
    int heads;                        // B * Hk
    long long groups;                 // of the launch
    long long pitch;                  // rows of a sequence and key head in `rows`
    const char* rows;                 // [2][B * Hk][pitch]: what is taken from a row's scores and its dP, as fp32 or in pieces
    long long all_rows;               // B * Hk * pitch
    float* parts;
};

// fp16 has no room for weights of long rows (2^-14 is its least normal number) nor for gradients of any size: P goes into its product times 2^15, dS
// times a power of two of the lane's own (a row's, or a key's), which its sums are divided by at the end.  The power falls when a value of the lane would
// pass 2^15, to one that takes that value to 2^11, and the sums with it: so what is rounded has all its bits down to 2^-25 of the lane's largest, whatever
// sizes other rows, keys, heads and sequences have, and a lane's results do not depend on them.
constexpr int WEIGHT_POWER = 15, SLOPE_POWER = 11;
constexpr float SLOPE_MOST = 0x1p15f, SLOPE_START = 0x1p100f;       // (what would need a larger factor than that leaves nothing in fp16)
// The factor that takes x to 2^SLOPE_POWER .. 2^(SLOPE_POWER + 1).  (Infinities and what is next to them: 2^-117.)
__device__ inline float slope_factor(float x)
{
    const int power = (int)(__float_as_uint(x) >> 23) - 127;
    return __uint_as_float((unsigned)(127 + SLOPE_POWER - power) << 23);
}

// What a score is multiplied by to count powers of two.
// (At least 2^-120, so that the logarithm of a sum counts as a score: scales below that are 2^-120 for scores below 2^100.)
__host__ __device__ inline float back_powers(float scale) { return fmaxf(fabsf(scale) * 1.44269504088896340736f, 0x1p-120f); }

__device__ inline unsigned low_bits(int x) { return x <= 0 ? 0u : ~0u >> (32 - min(x, 32)); }

// ---- of every row: delta and its statistics --------------------------------------------------------------------------

// What is taken from a row's scores (its reference and, counted as a score, the logarithm of its sum) and from its dP (delta) is there
// before the first product.  Where lanes are keys each of a lane's 16 sums has a row of its own: as fp32 numbers these would be as many reads from
// LDS as the operands'.  So 16-bit types take them as a product: three bf16 numbers that add up to one, times -1, a row's 16 bytes.  fp32
// (with products eight times as long) takes the scores' number, in powers of two, after the product, whose partial sums it would make coarser.
typedef bf16 Pieces __attribute__((ext_vector_type(8)));
__device__ inline Pieces pieces_of(float x)
{
    Pieces y = {(bf16)x};
    if (fabsf(x) < 0x1p127f) {
        const float r = x - (float)y[0];
        y[1] = (bf16)r;
        y[2] = (bf16)(r - (float)y[1]);
    }
    return y;
}
template <typename T>
struct RowNumber {
    typedef std::conditional_t<sizeof(T) == 4, float, Pieces> type;
    __device__ static type of(float x)
    {
        if constexpr (sizeof(T) == 4) return x;
        else return pieces_of(x);
    }
    __device__ static float value(const type& x)
    {
        if constexpr (sizeof(T) == 4) return x;
        else return ((float)x[0] + (float)x[1]) + (float)x[2];
    }
};

// Sixteen lanes a row, 16 bytes a lane at a time.
template <typename T>
__global__ __launch_bounds__(256) void k_back_rows(BackArgs a, Heads<const T> dout, Heads<const T> out, const float2* __restrict__ stats,
                                                   typename RowNumber<T>::type* __restrict__ rows)
{
    constexpr bool F16 = std::is_same<T, f16>::value;
    constexpr int EC = 16 / sizeof(T);
    typedef T V __attribute__((ext_vector_type(EC)));
    const int G = a.Hq / a.Hk, l = threadIdx.x & 15;
    const long long id = group_id() * 16 + (threadIdx.x >> 4);
    if (id >= a.all_rows) return;
    const int bh = (int)(id / a.pitch), r = (int)(id - bh * a.pitch), b = bh / a.Hk, hk = bh - b * a.Hk;
    const int q0 = a.cu_q[b], nq = min(a.cu_q[b + 1] - q0, a.max_q);
    if (r >= nq * G) return;                             // (fits: checked by the host)
    const int i = r / G, head = hk * G + r - i * G;
    const long long token = q0 + i;
    float s = 0.f;
    for (int d = l * EC; d < a.D; d += 16 * EC) {
        const V x = *(const V*)(dout.row(token, head) + d), y = *(const V*)(out.row(token, head) + d);
#pragma unroll
        for (int e = 0; e < EC; ++e) s += (float)x[e] * (float)y[e];
    }
#pragma unroll
    for (int o = 8; o; o >>= 1) s += __shfl_xor(s, o, 16);
    if (l == 0) {
        const float2 st = stats[token * a.Hq + head];
        // (a row without weights: none whatever the scores)
        const float by = back_powers(a.scale), power = log2f(st.y) - (F16 ? WEIGHT_POWER : 0);
        rows[id] = RowNumber<T>::of(st.y == 0.f ? INFINITY : sizeof(T) == 4 ? fmaf(st.x, by, power) : st.x + power / by);
        rows[a.all_rows + id] = RowNumber<T>::of(s);
    }
}

// ---- tiles of the walk ------------------------------------------------------------------------------------------------

template <typename T, int NC>
struct BackTile {
    static constexpr bool F32 = sizeof(T) == 4;
    static constexpr int RT = F32 ? 32 : 64;                       // rows (or keys)
    static constexpr int EC = 16 / sizeof(T);
    static constexpr int RS = NC == 3 ? 128 : 32 * NC;             // elements of a row in LDS
    static constexpr int CR = RS / EC;
    static constexpr int PER = RT * CR / BACK_THREADS;             // chunks a thread brings of a tensor
    static constexpr int BYTES = RT * RS * sizeof(T);
    // Chunk c of row j lies at c ^ swizzle(j).  Every tile is read both ways: one chunk of 32 rows (16 consecutive rows get different
    // places), and transposed, 16-bit: four rows, 64 bytes each, fp32: two rows four apart, 128 bytes each.
    __device__ static constexpr int swizzle(int j)
    {
        if (F32) return CR >= 16 ? (j >> 2 & 1) << 3 | (j >> 3 & 1) << 2 | (j & 3) : j >> 1 & 7;
        return CR == 16 ? (j & 3) << 2 | (j >> 2 & 3) : CR == 8 ? (j >> 1 & 1) << 2 | (j >> 2 & 3) : j >> 2 & 3;
    }
};

template <typename T>
__device__ inline bool finite_of(T x)
{
    if constexpr (sizeof(T) == 4) return fabsf(x) <= 3.402823466e38f;
    else {
        const unsigned short all = std::is_same<T, bf16>::value ? 0x7f80 : 0x7c00;
        return (__builtin_bit_cast(unsigned short, x) & all) != all;
    }
}

// What a kernel makes.  Rows: dq.  Keys: dk and dv at once, or one of them.
enum { BACK_DQ = 0, BACK_DK = 1, BACK_DV = 2 };

// WHAT & (BACK_DK | BACK_DV): lanes are keys, the walk is over rows; else lanes are rows, the walk is over keys.
template <typename T, int NC>
struct BackMemory {
    typedef typename RowNumber<T>::type Number;
    static constexpr int RT = BackTile<T, NC>::RT;
    __align__(1024) char as[2][BackTile<T, NC>::BYTES];
    __align__(1024) char bs[2][BackTile<T, NC>::BYTES];
    __align__(16) Number rc[2][2 * RT + 4];                          // of the rows walked; then zeros
    __align__(16) int odds[4];
};

// TWICE (16-bit types): weights and their gradients as two values of the type.
template <typename T, int NC, int WHAT, bool TWICE>
__device__ __forceinline__ void back_walk(const BackArgs& a, const int group, BackMemory<T, NC>& memory, Heads<const T> q, Heads<const T> k,
                                          Heads<const T> v, Heads<const T> dout, Heads<T> da, Heads<T> db)
{
    constexpr bool KEYS = WHAT != BACK_DQ, SUM_A = WHAT != BACK_DV, SUM_B = WHAT & BACK_DV;
    using G = BackTile<T, NC>;
    using M = Mfma<T>;
    constexpr bool F32 = G::F32;
    constexpr int RT = G::RT, EC = G::EC, RS = G::RS, CR = G::CR, PER = G::PER, QS = F32 ? 4 * NC : 2 * NC;
    using N = RowNumber<T>;
    typedef typename N::type Number;
    auto& as = memory.as;
    auto& bs = memory.bs;
    auto& odds = memory.odds;
    auto& rc = memory.rc;

    const int t = threadIdx.x, l = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6), c32 = l & 31, h = l >> 5;
    // far workgroups of all heads first: others have the chip to the end
    const int shared = a.Hq / a.Hk, fars = a.far_tiles * a.far, per_head = a.tiles * a.splits, heads = a.heads;
    const bool far = KEYS && group < fars * heads;
    const int slot = far ? group : in_runs(group - fars * heads, per_head * heads), bh = far ? slot / fars : slot / per_head, rest = far ? slot % fars : slot % per_head;
    const int b = bh / a.Hk, hk = bh - b * a.Hk, splits = far ? a.far : a.splits;
    const int tile = far ? rest / splits : KEYS ? rest / splits : a.tiles - 1 - rest / splits, split = rest % splits;
    const int q0 = a.cu_q[b], nq = min(a.cu_q[b + 1] - q0, a.max_q), all_q = a.cu_q[b + 1] - q0, k0 = a.cu_k[b], nk = a.cu_k[b + 1] - k0;
    const long long base = (long long)nk - all_q;                   // position of the first row's token
    const int rows = nq * shared;                                    // (fits: checked by the host)
    // of keys (or rows).  Far workgroups: all four waves have the same 32 keys, and take turns in the rows
    const int x0 = far ? tile * 32 : tile * BACK_LANES, count = KEYS ? min(nk, a.max_k) : rows;
    if (x0 >= count) return;
    const int wx0 = far ? x0 : x0 + 32 * wave, mine = min(wx0 + c32, count - 1), wlast = min(wx0 + 32, count) - 1;
    const int last = min(x0 / BACK_LANES * BACK_LANES + BACK_LANES, count) - 1;

    // rows that see key j: from, up to (the window's, or all if it is one of the first)
    auto row_of = [&](long long p) {                                 // the first row at position p or behind it
        const long long y = (p - base) * shared;
        return y < 0 ? 0 : y > rows ? rows : (int)y;
    };
    auto from_row = [&](int j) { return row_of((long long)j - a.w.right); };
    auto window_end = [&](int j) { return row_of((long long)j + a.w.left + 1); };
    auto to_row = [&](int j) { return j < a.w.sinks ? rows : window_end(j); };
    int lo = 0, hi = 0;                                              // of the lane: rows lo .. hi - 1, or keys lo .. hi
    const long long pos = base + mine / shared;
    if (KEYS) {
        lo = from_row(mine);
        hi = to_row(mine);
    } else {
        window_of(pos, nk, a.w, &lo, &hi);
    }
    const Sight all_rows(base + x0 / shared, base + last / shared, nk, a.w);
    const Sight wave_rows(base + wx0 / shared, base + (wx0 < count ? wlast / shared : wx0 / shared - 1), nk, a.w);
    // of the wave, where lanes are keys: some key is seen by rows any0 .. any1 - 1, all are by all0 .. all1 - 1
    int any0 = 0, any1 = 0, all0 = 0, all1 = 0;
    if (KEYS && wx0 < count) {
        any0 = from_row(wx0);
        any1 = wx0 < a.w.sinks ? rows : window_end(wlast);
        all0 = from_row(wlast);
        all1 = wlast < a.w.sinks ? rows : window_end(max(wx0, a.w.sinks));
    }
    const int tile0 = KEYS ? from_row(last) : 0, tile1 = !KEYS ? 0 : last < a.w.sinks ? rows : window_end(max(x0, a.w.sinks));   // likewise of the workgroup
    auto any = [&](int i) { return KEYS ? i < any1 && i + 32 > any0 : wave_rows.any(i, 32); };
    auto all = [&](int i) { return KEYS ? i >= all0 && i + 32 <= all1 : wave_rows.all(i, 32); };
    // bits of the 32 walked from i on that the lane's pair sees
    auto sight = [&](int i) {
        return KEYS ? low_bits(hi - i) & ~low_bits(lo - i) : low_bits(hi + 1 - i) & (~low_bits(lo - i) | low_bits(a.w.sinks - i));
    };

    // tiles of the walk
    const KeyTiles<RT> keys(all_rows);
    int first = 0, n = keys.n;
    if (KEYS) {
        const int r1 = window_end(last), r0 = far ? r1 : from_row(x0), end = far ? rows : r1;
        first = r0 / RT;
        // (a far walk begins in the tile in which the window's has ended, and the rows that the window had are masked)
        n = end > r0 ? (end + RT - 1) / RT - first : 0;
        if (far) lo = max(lo, r1), any0 = max(any0, r1), all0 = max(all0, r1);
        else hi = min(hi, r1), any1 = min(any1, r1), all1 = min(all1, r1);
    }
    const int per = (n + splits - 1) / splits, begin = split * per, stop = min(n, begin + per);
    // Workgroups of an XCD that walk nearly the same tiles should be at the same ones at the same time, when these are in its L2: each starts
    // with the first of its tiles whose number is a multiple of what one walks, and takes those before it at the end.
    int turn = 0;
    if (a.cycle && !far) {
        const int head = KEYS ? first : keys.first / RT, past = (a.cycle - head % a.cycle) % a.cycle + (KEYS ? 0 : keys.sink_tiles);
        turn = past < n ? past : 0;
    }
    auto at = [&](int it) {
        const int i = it + turn < n ? it + turn : it + turn - n;
        return KEYS ? (first + i) * RT : keys.base(i);
    };
    const int walked = KEYS ? rows : nk;

    const Heads<const T> A = KEYS ? q : k, B = KEYS ? dout : v;
    const T* const ap = KEYS ? A.row(q0, hk * shared) : A.row(k0, hk);
    const T* const bp = KEYS ? B.row(q0, hk * shared) : B.row(k0, hk);
    const Number* const rows_at = (const Number*)a.rows + a.pitch * bh;
    auto element = [&](const Heads<const T>& x, int r) { return KEYS ? r / shared * x.token + r % shared * x.head : r * x.token; };
    // offsets of 32 bits from a tile's first row on
    auto near = [&](const Heads<const T>& x) { return x.token >= 0 && x.token < 1 << 22 && (!KEYS || (x.head >= 0 && x.head < 1 << 22)); };
    // chunks that a thread brings lie STEP rows apart; the swizzle has a period of 16 rows, so they have KINDS places in a row
    constexpr int STEP = BACK_THREADS / CR, KINDS = STEP % 16 ? 2 : 1;
    const bool plain = near(A) && near(B) && a.D == RS && (!KEYS || STEP % shared == 0);
    const int slot0 = t / CR;
    int chunk[KINDS];
    unsigned ao[KINDS], bo[KINDS];
#pragma unroll
    for (int i = 0; i < KINDS; ++i) {
        chunk[i] = (t % CR ^ G::swizzle(slot0 + i * STEP)) * EC;
        ao[i] = (unsigned)(element(A, slot0) + chunk[i]) * (unsigned)sizeof(T);
        bo[i] = (unsigned)(element(B, slot0) + chunk[i]) * (unsigned)sizeof(T);
    }
    const unsigned a_tile = (unsigned)element(A, RT) * (unsigned)sizeof(T), b_tile = (unsigned)element(B, RT) * (unsigned)sizeof(T);   // bytes, if plain
    const unsigned a_lds = lds_address(as), b_lds = lds_address(bs);
    auto bring = [&](int it) {
        const int buf = (it - begin) & 1, i0 = at(it);
        if (KEYS) {
            // both numbers of the tile's rows: a wave each, 16 bytes a lane
            constexpr int LANES = RT * sizeof(Number) / 16;
            if (wave < 2 && l < LANES)
                to_lds((const char*)(rows_at + wave * a.all_rows + i0) + l * 16, lds_address(rc[buf]) + wave * LANES * 16);
        }
        if (plain && i0 + RT <= walked) {
            // (rows i0 + i STEP begin with a new token, or all heads share a key head of their own)
            const char* a0 = (const char*)ap + (unsigned long long)((unsigned)i0 / RT) * a_tile;
            const char* b0 = (const char*)bp + (unsigned long long)((unsigned)i0 / RT) * b_tile;
            const unsigned lds = wave * 1024 + buf * G::BYTES;
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                to_lds(a0, ao[i % KINDS], a_lds + lds + i * 4096);
                to_lds(b0, bo[i % KINDS], b_lds + lds + i * 4096);
                a0 += a_tile / PER;
                b0 += b_tile / PER;
            }
            return;
        }
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int r = min(i0 + i * STEP + slot0, walked - 1);
            if (chunk[i % KINDS] < a.D) {
                to_lds(ap + element(A, r) + chunk[i % KINDS], a_lds + wave * 1024 + buf * G::BYTES + i * 4096);
                to_lds(bp + element(B, r) + chunk[i % KINDS], b_lds + wave * 1024 + buf * G::BYTES + i * 4096);
            }
        }
    };
    // chunks past a head's end are never brought: zero
    if (a.D < RS)
        for (int i = t; i < 2 * RT * CR; i += BACK_THREADS) {
            const int s = i % (RT * CR), j = s / CR;
            if ((s % CR ^ G::swizzle(j)) * EC >= a.D) {
                *(uint4*)(as[i / (RT * CR)] + s * 16) = make_uint4(0, 0, 0, 0);
                *(uint4*)(bs[i / (RT * CR)] + s * 16) = make_uint4(0, 0, 0, 0);
            }
        }
    if (KEYS && t < 8) ((uint4*)&rc[t / 4][2 * RT])[sizeof(T) == 4 ? 0 : t % 4] = make_uint4(0, 0, 0, 0);
    if (begin < stop) bring(begin);

    // the lanes' own operands
    typename M::V af[QS], bf[QS];
    {
        const T* const x = KEYS ? k.row(k0 + mine, hk) : q.row(q0 + mine / shared, hk * shared + mine % shared);
        const T* const y = KEYS ? v.row(k0 + mine, hk) : dout.row(q0 + mine / shared, hk * shared + mine % shared);
#pragma unroll
        for (int c = 0; c < QS; ++c) {
            const int d = (2 * c + h) * EC;
            if (d < a.D) {
                af[c] = *(const typename M::V*)(x + d);
                bf[c] = *(const typename M::V*)(y + d);
            } else {
#pragma unroll
                for (int e = 0; e < EC; ++e) af[c][e] = bf[c][e] = (T)0.f;
            }
            // a negative scale turns the scores, as in the forward kernel
            if (a.scale < 0.f)
#pragma unroll
                for (int e = 0; e < EC; ++e) af[c][e] = -af[c][e];
        }
    }
    const float by = back_powers(a.scale);
    float own0 = 0.f, own1 = 0.f;                    // minus what is taken, from scores in powers of two
    if (!KEYS) {
        own0 = -N::value(rows_at[mine]) * (F32 ? 1.f : by);
        own1 = -N::value(rows_at[a.all_rows + mine]);
    }
    constexpr bool F16 = std::is_same<T, f16>::value;
    float slope = SLOPE_START;                        // fp16: what the lane's gradients of weights, 2^WEIGHT_POWER dS, are multiplied by

    const int r4 = l >> 2 & 3, c4 = l & 3, g16 = l >> 4 & 1;
    int k_at = (c32 * RS + (h ^ G::swizzle(c32)) * EC) * (int)sizeof(T);
    int v_at = F32 ? (4 * h * RS + ((c32 >> 2) ^ G::swizzle(4 * h)) * EC + (c32 & 3)) * (int)sizeof(T)
                         : ((4 * h + r4) * RS + ((2 * g16 + (c4 >> 1)) ^ G::swizzle(4 * h + r4)) * EC + (c4 & 1) * 4) * (int)sizeof(T);
    // 32 elements of the head (from 32 x on) of the walked rows 16 m .. 16 m + 15 (fp32: row 8 (i / 4) + 4 h + i % 4 of element i)
    auto turned = [&](const char* from, int x, int m) {
        const char* const p = from + (v_at ^ x * 64) + 16 * m * RS * (int)sizeof(T);
        const char* const p8 = from + (v_at ^ x * 64 ^ 32) + (16 * m + 8) * RS * (int)sizeof(T);
        if constexpr (!F32) {
            const typename M::V4 y0 = transposed<typename M::V4>(p), y1 = transposed<typename M::V4>(p8);
            return __builtin_shufflevector(y0, y1, 0, 1, 2, 3, 4, 5, 6, 7);
        } else {
            return (typename M::V){};
        }
    };
    auto single = [&](const char* from, int x, int i) {
        return *(const T*)(from + (v_at ^ x * 128 ^ G::swizzle(8 * (i / 4) + i % 4) * 16) + (8 * (i / 4) + i % 4) * RS * (int)sizeof(T));
    };

    f32x16 acc_a[NC], acc_b[NC];
#pragma unroll
    for (int x = 0; x < NC; ++x)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc_a[x][i] = acc_b[x][i] = 0.f;
    unsigned met[NC] = {};                             // elements of results that something that is not finite enters (dA 16 bits, dB 16 more)

    for (int it = begin; it < stop; ++it) {
        const int buf = (it - begin) & 1, i0 = at(it);
        wait_but_and_meet<0>();
        if (it + 1 < stop) bring(it + 1);
        // Pairs that do not see each other have weights of zero, and zero times what is not finite is NaN: where there are such pairs and such
        // values, these count as zero, and mark the results of those that do see them.
        bool odd = false;
        if (!(KEYS ? i0 >= tile0 && i0 + RT <= tile1 : all_rows.all(i0, RT))) {
            typedef T Chunk __attribute__((ext_vector_type(EC)));
#pragma unroll
            for (int i = 0; i < 2 * PER; ++i) {
                const Chunk y = *(const Chunk*)((i < PER ? as[buf] : bs[buf]) + (i % PER * BACK_THREADS + t) * 16);
#pragma unroll
                for (int e = 0; e < EC; ++e) odd = odd || !finite_of((T)y[e]);
            }
            if (l == 0) odds[wave] = 0;
            if (__any(odd) && l == 0) odds[wave] = 1;
            wait_and_meet();
            const int4 y = *(const int4*)odds;
            odd = __builtin_amdgcn_readfirstlane(y.x | y.y | y.z | y.w);
        }
#pragma unroll
        for (int u = 0; u < RT / 32; ++u) {
            const int i = i0 + 32 * u;
            if (!any(i) || (far && ((it - begin) * (RT / 32) + u) % 4 != wave)) continue;
            // (worked out again for every tile: kept, the addresses of all steps would take the registers)
            asm volatile("" : "+v"(k_at), "+v"(v_at));
            const char* const ab = as[buf] + 32 * u * RS * sizeof(T);
            const char* const bb = bs[buf] + 32 * u * RS * sizeof(T);
            f32x16 s, dp;
            // minus what is taken from the rows' scores (0) or dP (1)
            auto start = [&](f32x16& y, int which) {
                if constexpr (!KEYS) {
                    // (one number for all of a lane's sums: taken at the end, where it costs no registers)
#pragma unroll
                    for (int e = 0; e < 16; ++e) y[e] = 0.f;
                } else if (F32 && which == 0) {
#pragma unroll
                    for (int e = 0; e < 16; ++e) y[e] = 0.f;
                } else if constexpr (F32) {
#pragma unroll
                    for (int e = 0; e < 16; e += 4) {
                        const float4 z = *(const float4*)(rc[buf] + which * RT + 32 * u + 2 * e + 4 * h);
                        y[e] = -z.x; y[e + 1] = -z.y; y[e + 2] = -z.z; y[e + 3] = -z.w;
                    }
                } else {
                    const Pieces minus = {(bf16)-1.f, (bf16)-1.f, (bf16)-1.f, (bf16)0.f, (bf16)0.f, (bf16)0.f, (bf16)0.f, (bf16)0.f};
#pragma unroll
                    for (int e = 0; e < 16; ++e) y[e] = 0.f;
                    y = Mfma<bf16>::mul(rc[buf][h ? 2 * RT : which * RT + 32 * u + c32], minus, y);
                }
            };
            start(s, 0);
#pragma unroll
            for (int c = 0; c < QS; ++c) {
                const typename M::V x = *(const typename M::V*)(ab + (k_at ^ c * 32));
                if (F32 && 8 * c >= a.D) continue;              // (256 cycles a step; in 16-bit types 32, which a branch would cost)
                if constexpr (F32) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) s = M::mul(x[e], af[c][e], s);
                } else {
                    s = M::mul(x, af[c], s);
                }
            }
            if constexpr (SUM_A) {
                start(dp, 1);
#pragma unroll
                for (int c = 0; c < QS; ++c) {
                    const typename M::V y = *(const typename M::V*)(bb + (k_at ^ c * 32));
                    if (F32 && 8 * c >= a.D) continue;
                    if constexpr (F32) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) dp = M::mul(y[e], bf[c][e], dp);
                    } else {
                        dp = M::mul(y, bf[c], dp);
                    }
                }
            }
            if constexpr (KEYS && F32) {
#pragma unroll
                for (int e = 0; e < 16; e += 4) {
                    const float4 z = *(const float4*)(rc[buf] + 32 * u + 2 * e + 4 * h);
                    s[e] = __builtin_amdgcn_exp2f(fmaf(s[e], by, -z.x));
                    s[e + 1] = __builtin_amdgcn_exp2f(fmaf(s[e + 1], by, -z.y));
                    s[e + 2] = __builtin_amdgcn_exp2f(fmaf(s[e + 2], by, -z.z));
                    s[e + 3] = __builtin_amdgcn_exp2f(fmaf(s[e + 3], by, -z.w));
                }
            } else {
#pragma unroll
                for (int e = 0; e < 16; ++e) s[e] = __builtin_amdgcn_exp2f(KEYS ? s[e] * by : fmaf(s[e], by, own0));
            }
            if constexpr (SUM_A)
#pragma unroll
                for (int e = 0; e < 16; ++e) dp[e] = (KEYS ? dp[e] : dp[e] + own1) * s[e];
            const bool whole = all(i);
            unsigned seen = ~0u;
            if (!whole) {
                seen = sight(i) >> 4 * h;
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int m = (int)(seen << (31 - 8 * (e / 4) - e % 4)) >> 31;
                    if constexpr (SUM_B) s[e] = __int_as_float(__float_as_int(s[e]) & m);
                    if constexpr (SUM_A) dp[e] = __int_as_float(__float_as_int(dp[e]) & m);
                }
            }
            if constexpr (F16 && SUM_A) {
                float most = 0.f;
#pragma unroll
                for (int e = 0; e < 16; ++e) most = fmaxf(most, fabsf(dp[e]));
                if (__any(most * slope > SLOPE_MOST)) {
                    // (both halves of the wave hold parts of a lane's sums)
                    most = fmaxf(most, __shfl_xor(most, 32));
                    const float now = most * slope > SLOPE_MOST ? slope_factor(most) : slope, less = now / slope;
                    products_done<T>();
#pragma unroll
                    for (int x = 0; x < NC; ++x)
#pragma unroll
                        for (int e = 0; e < 16; ++e) acc_a[x][e] *= less;
                    slope = now;
                }
#pragma unroll
                for (int e = 0; e < 16; ++e) dp[e] *= slope;
            }
            auto add = [&](auto carefully, f32x16* acc, const char* from, const f32x16& weight, int bit) {
                constexpr bool careful = decltype(carefully)::value;
                if constexpr (F32) {
#pragma unroll
                    for (int e = 0; e < 16; ++e)
#pragma unroll
                        for (int x = 0; x < NC; ++x) {
                            T y = single(from, x, e);
                            if (careful && !finite_of(y)) y = 0.f;
                            acc[x] = M::mul(y, weight[e], acc[x]);
                        }
                } else {
#pragma unroll
                    for (int m = 0; m < 2; ++m) {
                        typename M::V w, rest;
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            w[e] = (T)weight[8 * m + e];
                            if constexpr (TWICE) rest[e] = (T)(weight[8 * m + e] - (float)w[e]);
                        }
#pragma unroll
                        for (int x = 0; x < NC; ++x) {
                            typename M::V y = turned(from, x, m);
                            if constexpr (careful)
#pragma unroll
                                for (int e = 0; e < 8; ++e)
                                    if (!finite_of((T)y[e])) y[e] = (T)0.f;
                            acc[x] = M::mul(y, w, acc[x]);
                            if constexpr (TWICE) acc[x] = M::mul(y, rest, acc[x]);
                        }
                    }
                }
                if constexpr (careful) {
#pragma unroll
                    for (int x = 0; x < NC; ++x) {
                        asm volatile("" : "+v"(v_at));             // (one at a time)
                        f32x16 kinds;
#pragma unroll
                        for (int e = 0; e < 16; ++e) kinds[e] = 0.f;
                        if constexpr (F32) {
#pragma unroll
                            for (int e = 0; e < 16; ++e)
                                kinds = M::mul(finite_of(single(from, x, e)) ? 0.f : 1.f, (float)(seen >> (8 * (e / 4) + e % 4) & 1), kinds);
                        } else {
#pragma unroll
                            for (int m = 0; m < 2; ++m) {
                                typename M::V y = turned(from, x, m), w;
#pragma unroll
                                for (int e = 0; e < 8; ++e) {
                                    const int i8 = 8 * m + e;
                                    y[e] = finite_of((T)y[e]) ? (T)0.f : (T)1.f;
                                    w[e] = (T)(float)(seen >> (8 * (i8 / 4) + i8 % 4) & 1);
                                }
                                kinds = M::mul(y, w, kinds);
                            }
                        }
#pragma unroll
                        for (int e = 0; e < 16; ++e) met[x] |= kinds[e] != 0.f ? 1u << (bit + e) : 0u;
                    }
                }
            };
            if (__builtin_expect(odd && !whole, 0)) {
                if constexpr (SUM_B) add(std::true_type(), acc_b, bb, s, 16);
                if constexpr (SUM_A) add(std::true_type(), acc_a, ab, dp, 0);
            } else {
                if constexpr (SUM_B) add(std::false_type(), acc_b, bb, s, 16);
                if constexpr (SUM_A) add(std::false_type(), acc_a, ab, dp, 0);
            }
            if constexpr (F32) products_done<T>();
        }
    }
    // (the lane's place once more: kept, it would take registers from the walk)
    int lane = threadIdx.x & 63;
    asm volatile("" : "+v"(lane));
    const int to = wx0 + (lane & 31), half = lane >> 5, token = KEYS ? to : to / shared;
    // far workgroups: the waves' sums of the same keys, through LDS, in two steps
    auto together = [&](f32x16* acc) {
        float4* const sums = (float4*)as[0] + lane;
#pragma unroll
        for (int step = 2; step; step >>= 1) {
            __syncthreads();
            if (wave >= step && wave < 2 * step)
#pragma unroll
                for (int x = 0; x < NC; ++x)
#pragma unroll
                    for (int e = 0; e < 16; e += 4)
                        sums[(((wave - step) * NC + x) * 4 + e / 4) * 64] = make_float4(acc[x][e], acc[x][e + 1], acc[x][e + 2], acc[x][e + 3]);
            __syncthreads();
            if (wave < step)
#pragma unroll
                for (int x = 0; x < NC; ++x)
#pragma unroll
                    for (int e = 0; e < 16; e += 4) {
                        const float4 y = sums[((wave * NC + x) * 4 + e / 4) * 64];
                        acc[x][e] += y.x; acc[x][e + 1] += y.y; acc[x][e + 2] += y.z; acc[x][e + 3] += y.w;
                    }
        }
    };
    auto put = [&](const Heads<T>& out, f32x16* acc, float scale, int which) {
#pragma unroll
        for (int x = 0; x < NC; ++x)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                if (met[x] >> (16 * which + e) & 1) acc[x][e] = NAN;
                else acc[x][e] *= scale;
            }
        if (KEYS && far) {
            together(acc);
            if (wave) return;
        }
        if (to >= count) return;
        const bool parts = far || a.splits > 1 || (KEYS && tile < a.first_tiles);
        T* const y = KEYS ? out.row(k0 + to, hk) : out.row(q0 + token, hk * shared + to - token * shared);
        const long long row = (far ? a.far_part(bh, tile, split) : a.own_part(bh, tile, split)) + (to - x0);
        float* const z = a.parts + (row * (KEYS ? 2 : 1) + which) * a.D;
#pragma unroll
        for (int x = 0; x < NC; ++x)
#pragma unroll
            for (int e = 0; e < 16; e += 4) {
                const int d = 32 * x + 2 * e + 4 * half;
                if (d >= a.D) continue;
                if (parts) {
                    *(float4*)(z + d) = make_float4(acc[x][e], acc[x][e + 1], acc[x][e + 2], acc[x][e + 3]);
                } else {
                    typedef T T4 __attribute__((ext_vector_type(4)));
                    T4 o;
#pragma unroll
                    for (int f = 0; f < 4; ++f) o[f] = (T)acc[x][e + f];
                    *(T4*)(y + d) = o;
                }
            }
    };
    if constexpr (SUM_A) put(da, acc_a, F16 ? a.scale * (1.f / (1 << WEIGHT_POWER)) / slope : a.scale, 0);
    if constexpr (SUM_B) put(db, acc_b, F16 ? 1.f / (1 << WEIGHT_POWER) : 1.f, 1);
}

// All walks of a call at once, since none waits for another: keys' (dk and dv together, or one after the other), then rows'.  16-bit types, wide heads:
// sums of both gradients would leave a SIMD one wave (bf16, 16384 tokens, window of 4096, heads 16 of 4 x 128: 2700 us at once, 850 and 660 apart, the
// scores twice).
template <typename T, int NC, bool TWICE>
__global__ __launch_bounds__(BACK_THREADS, sizeof(T) == 4 ? 1 : 2) void k_back(BackArgs ak, BackArgs aq, Heads<const T> q, Heads<const T> k, Heads<const T> v,
                                                                              Heads<const T> dout, Heads<T> dq, Heads<T> dk, Heads<T> dv)
{
    __shared__ BackMemory<T, NC> memory;
    const long long group = group_id();
    constexpr bool APART = sizeof(T) == 2 && NC > 2;
    const long long keys = APART ? 2 * ak.groups : ak.groups;
    if (group >= keys + aq.groups) return;
    if (group >= keys) back_walk<T, NC, BACK_DQ, TWICE>(aq, (int)(group - keys), memory, q, k, v, dout, dq, dq);
    else if constexpr (!APART) back_walk<T, NC, BACK_DK | BACK_DV, TWICE>(ak, (int)group, memory, q, k, v, dout, dk, dv);
    else if (group < ak.groups) back_walk<T, NC, BACK_DK, TWICE>(ak, (int)group, memory, q, k, v, dout, dk, dv);
    else back_walk<T, NC, BACK_DV, TWICE>(ak, (int)(group - ak.groups), memory, q, k, v, dout, dk, dv);
}

// Sums of the parts of a tile: 32 lanes a key (or row), four elements a lane.
template <typename T, bool KEYS>
__device__ __forceinline__ void back_join(const BackArgs& a, const int id, int tiles, Heads<T> da, Heads<T> db)
{
    const int d = (threadIdx.x & 31) * 4, shared = a.Hq / a.Hk, across = tiles * (BACK_LANES / 8);
    const int bh = id / across, b = bh / a.Hk, hk = bh - b * a.Hk, x = (id - bh * across) * 8 + (threadIdx.x >> 5);
    if (d >= a.D) return;
    const int x0 = KEYS ? a.cu_k[b] : a.cu_q[b];
    const int count = KEYS ? min(a.cu_k[b + 1] - x0, a.max_k) : min(a.cu_q[b + 1] - x0, a.max_q) * shared;
    if (x >= count) return;
    const int far = KEYS && x / FAR_LANES < a.far_tiles ? a.far : 0;
    constexpr int N = KEYS ? 2 : 1;
    const float* const own = a.parts + (a.own_part(bh, x / BACK_LANES, 0) + x % BACK_LANES) * N * a.D + d;
    const float* const others = a.parts + (a.far_part(bh, x / FAR_LANES, 0) + x % FAR_LANES) * N * a.D + d;
#pragma unroll
    for (int which = 0; which < N; ++which) {
        float4 s = {0.f, 0.f, 0.f, 0.f};
        // (eight parts on their way at once)
        auto add = [&](const float* from, int n, int step) {
            for (int i = 0; i < n; i += 8) {
                float4 p[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) p[j] = *(const float4*)(from + (long long)min(i + j, n - 1) * step);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    s.x += i + j < n ? p[j].x : 0.f; s.y += i + j < n ? p[j].y : 0.f; s.z += i + j < n ? p[j].z : 0.f; s.w += i + j < n ? p[j].w : 0.f;
                }
            }
        };
        add(own + which * a.D, a.splits, BACK_LANES * N * a.D);
        add(others + which * a.D, far, FAR_LANES * N * a.D);
        const Heads<T>& to = which ? db : da;
        typedef T T4 __attribute__((ext_vector_type(4)));
        T* const y = KEYS ? to.row(x0 + x, hk) : to.row(x0 + x / shared, hk * shared + x % shared);
        *(T4*)(y + d) = T4{(T)s.x, (T)s.y, (T)s.z, (T)s.w};
    }
}

// Tiles of keys and of rows whose sums are in parts.
template <typename T>
__global__ __launch_bounds__(256) void k_back_join(BackArgs ak, BackArgs aq, int tiles_k, int tiles_q, Heads<T> dq, Heads<T> dk, Heads<T> dv)
{
    const long long id = group_id(), keys = (long long)tiles_k * (BACK_LANES / 8) * ak.heads, all = keys + (long long)tiles_q * (BACK_LANES / 8) * aq.heads;
    if (id >= all) return;
    if (id < keys) back_join<T, true>(ak, (int)id, tiles_k, dk, dv);
    else back_join<T, false>(aq, (int)(id - keys), tiles_q, dq, dq);
}

constexpr int BACK_TWICE = 512;            // keys that a row sees at most for weights to be two values

struct BackPlan : BackParts {
    int cycle;
    bool twice;
    long long groups;
    size_t parts;                          // elements
};

// Few tiles: workgroups share the walk until there are two for every compute unit, each with four tiles at least.
static int back_splits(long long groups, long long walk, int rt)
{
    long long n = groups > 0 && groups < 512 ? 512 / groups : 1;
    const long long most = (walk + rt - 1) / rt / 4;
    if (n > most) n = most;
    return n < 1 ? 1 : n > 64 ? 64 : (int)n;
}

static BackPlan back_plan(bool keys, int type, int B, int Hq, int Hk, int D, int max_q, int max_k, int left, int right, int sinks)
{
    BackPlan p = {};
    const int G = Hq / Hk, rt = type == ZNNI_F32 ? 32 : 64;
    const long long count = keys ? max_k : (long long)max_q * G;
    p.tiles = (int)((count + BACK_LANES - 1) / BACK_LANES);
    const long long groups = (long long)p.tiles * Hk * B;
    p.twice = (long long)left + right + (sinks < max_k ? sinks : max_k) < BACK_TWICE || max_k <= BACK_TWICE;
    // what a tile walks at most, first tokens (seen by all rows that follow) apart
    const long long wide = (long long)left + right + (keys ? BACK_LANES : BACK_LANES / G + 2);
    long long walk;
    if (keys) {
        walk = (wide < max_q ? wide : max_q) * G;
        const int lanes = sinks < max_k ? sinks : max_k;
        // rows past the window of first tokens: so many workgroups that each is done in a small part of the others' time
        if (lanes > 0 && (long long)left + 1 < max_k) {
            p.first_tiles = (lanes + BACK_LANES - 1) / BACK_LANES;
            p.far_tiles = (lanes + FAR_LANES - 1) / FAR_LANES;
            // (each eight tiles at least)
            long long n = 8 * ((long long)max_q + wide - 1) / wide;
            if (n > (long long)max_q * G / (8 * rt)) n = (long long)max_q * G / (8 * rt);
            p.far = n < 1 ? 1 : n > 64 ? 64 : (int)n;
        }
    } else {
        walk = wide + sinks < max_k ? wide + sinks : max_k;
    }
    p.splits = back_splits(groups, walk, rt);
    p.cycle = p.splits == 1 ? (int)((walk + rt - 1) / rt) : 0;
    const long long per_head = (long long)p.tiles * p.splits + (long long)p.far_tiles * p.far;
    p.groups = per_head * Hk * B;
    p.parts = (size_t)p.per_head() * Hk * B * (keys ? 2 : 1) * D;
    return p;
}

struct BackSizes {
    size_t rows, parts;                    // bytes
    long long pitch;
};

static BackSizes back_sizes(int type, int B, int Hq, int Hk, int D, int max_q, int max_k, int left, int right, int sinks)
{
    BackSizes s = {};
    s.pitch = ((long long)max_q * (Hq / Hk) + 63) / 64 * 64;
    s.rows = ((size_t)2 * B * Hk * s.pitch * (type == ZNNI_F32 ? sizeof(float) : sizeof(Pieces)) + 255) & ~(size_t)255;
    const size_t p0 = back_plan(true, type, B, Hq, Hk, D, max_q, max_k, left, right, sinks).parts;
    const size_t p1 = back_plan(false, type, B, Hq, Hk, D, max_q, max_k, left, right, sinks).parts;
    s.parts = (p0 + p1) * sizeof(float);
    return s;
}

static BackArgs planned(BackArgs a, const BackPlan& p, float* parts)
{
    (BackParts&)a = p;
    a.cycle = p.cycle;
    a.groups = p.groups;
    a.parts = parts;
    return a;
}

template <typename T>
static znni_status launch_back(BackArgs a, int type, int B, const znni_heads* q, const znni_heads* k, const znni_heads* v, const znni_heads* dout,
                               const znni_heads* out, const float* stats, const znni_heads* dq, const znni_heads* dk, const znni_heads* dv,
                               hipStream_t st)
{
    const Heads<const T> qi = heads_of<const T>(q), ki = heads_of<const T>(k), vi = heads_of<const T>(v), gi = heads_of<const T>(dout);
    if (a.all_rows) {
        k_back_rows<T><<<launch_of((a.all_rows + 15) / 16), dim3(256), 0, st>>>(a, gi, heads_of<const T>(out), (const float2*)stats, (typename RowNumber<T>::type*)a.rows);
        if (hipGetLastError() != hipSuccess) return ZNNI_ERR_HIP;
    }
    const BackPlan pk = back_plan(true, type, B, a.Hq, a.Hk, a.D, a.max_q, a.max_k, a.w.left, a.w.right, a.w.sinks);
    const BackPlan pq = back_plan(false, type, B, a.Hq, a.Hk, a.D, a.max_q, a.max_k, a.w.left, a.w.right, a.w.sinks);
    const BackArgs ak = planned(a, pk, a.parts), aq = planned(a, pq, a.parts + pk.parts);
    const Heads<T> oq = heads_of<T>(dq), ok = heads_of<T>(dk), ov = heads_of<T>(dv);
    const int NC = (a.D + 31) / 32;
    const dim3 grid = launch_of((sizeof(T) == 2 && NC > 2 ? 2 : 1) * pk.groups + pq.groups), block(BACK_THREADS);
    // Rounding dS to 16 bits costs as much as rounding the result, and rows of few keys get as much again from `out`, whose rounding is in delta.  Where
    // rows see few keys, products are few too: dS and P as two values there.  (fp16, ragged 300 tokens, window of 100: error 0.00031 of the result
    // and 0.00022, where products in fp32 leave 0.00021; 56 us and 64.)
    auto launch = [&](auto doubled) {
        constexpr bool TWICE = decltype(doubled)::value;
        switch (NC) {
            case 1: k_back<T, 1, TWICE><<<grid, block, 0, st>>>(ak, aq, qi, ki, vi, gi, oq, ok, ov); break;
            case 2: k_back<T, 2, TWICE><<<grid, block, 0, st>>>(ak, aq, qi, ki, vi, gi, oq, ok, ov); break;
            case 3: k_back<T, 3, TWICE><<<grid, block, 0, st>>>(ak, aq, qi, ki, vi, gi, oq, ok, ov); break;
            default: k_back<T, 4, TWICE><<<grid, block, 0, st>>>(ak, aq, qi, ki, vi, gi, oq, ok, ov); break;
        }
    };
    if constexpr (sizeof(T) == 2) {
        if (pk.twice) launch(std::true_type());
        else launch(std::false_type());
    } else {
        launch(std::false_type());
    }
    if (hipGetLastError() != hipSuccess) return ZNNI_ERR_HIP;
    const int tk = pk.splits > 1 ? pk.tiles : pk.first_tiles, tq = pq.splits > 1 ? pq.tiles : 0;
    if (!tk && !tq) return ZNNI_OK;
    k_back_join<T><<<launch_of((long long)(tk + tq) * (BACK_LANES / 8) * a.heads), dim3(256), 0, st>>>(ak, aq, tk, tq, oq, ok, ov);
    return hipGetLastError() == hipSuccess ? ZNNI_OK : ZNNI_ERR_HIP;
}

static znni_status back_shape(int type, int B, int Hq, int Hk, int D, int max_q, int max_k, int left, int right, int sinks)
{
    if (!type_ok(type)) return ZNNI_ERR_TYPE;
    if (B < 0 || B > 65535 || max_q < 0 || max_k < 0 || left < 0 || right < 0 || sinks < 0) return ZNNI_ERR_SHAPE;
    const znni_status rc = heads_shape(Hq, Hk, D);
    if (rc) return rc;
    // (tiles' ends, a tile past the last, and workgroups are 32 bits)
    const long long rows = (long long)max_q * (Hq / Hk), most = INT_MAX - 2 * BACK_LANES;
    if (rows > most || max_k > most) return ZNNI_ERR_SHAPE;
    const long long tiles = ((rows > max_k ? rows : max_k) + BACK_LANES - 1) / BACK_LANES;
    if (tiles * Hk > INT_MAX / (B ? B : 1)) return ZNNI_ERR_SHAPE;
    for (const bool keys : {false, true}) {
        const BackPlan p = back_plan(keys, type, B, Hq, Hk, D, max_q, max_k, left, right, sinks);
        const long long joined = (long long)(p.splits > 1 ? p.tiles : p.first_tiles) * (BACK_LANES / 8) * Hk * B;
        if (p.groups > INT_MAX || joined > INT_MAX) return ZNNI_ERR_SHAPE;
    }
    return ZNNI_OK;
}

}  // namespace znni

using namespace znni;

extern "C" {

znni_status znni_attn_window_backward_workspace(int type, int B, int Hq, int Hk, int D, int max_q, int max_k, int left, int right, int sinks,
                                                size_t* bytes)
{
    if (!bytes) return ZNNI_ERR_NULL;
    const znni_status rc = back_shape(type, B, Hq, Hk, D, max_q, max_k, left, right, sinks);
    if (rc) return rc;
    const BackSizes s = back_sizes(type, B, Hq, Hk, D, max_q, max_k, left, right, sinks);
    *bytes = s.rows + s.parts;
    return ZNNI_OK;
}

znni_status znni_attn_window_backward(int type, int B, int Hq, int Hk, int D, const znni_heads* q, const znni_heads* k, const znni_heads* v,
                                      const znni_heads* out, const float* stats, const znni_heads* dout, const int* cu_q, const int* cu_k,
                                      int max_q, int max_k, int left, int right, int sinks, float scale, const znni_heads* dq,
                                      const znni_heads* dk, const znni_heads* dv, void* workspace, size_t workspace_bytes, void* stream)
{
    if (!q || !k || !v || !out || !dout || !dq || !dk || !dv) return ZNNI_ERR_NULL;
    size_t need = 0;
    const znni_status rc = znni_attn_window_backward_workspace(type, B, Hq, Hk, D, max_q, max_k, left, right, sinks, &need);
    if (rc) return rc;
    if (B == 0 || (max_q == 0 && max_k == 0)) return ZNNI_OK;
    if (max_q > 0 && (!q->data || !out->data || !dout->data || !dq->data || !stats)) return ZNNI_ERR_NULL;
    if (max_k > 0 && (!k->data || !v->data || !dk->data || !dv->data)) return ZNNI_ERR_NULL;
    if (!cu_q || !cu_k || (need && !workspace)) return ZNNI_ERR_NULL;
    if (workspace_bytes < need) return ZNNI_ERR_WORKSPACE;
    if (((uintptr_t)cu_q | (uintptr_t)cu_k) & 3u || (uintptr_t)stats & 7u || (need && ((uintptr_t)workspace & 255u))) return ZNNI_ERR_ALIGN;
    for (const znni_heads* x : {q, k, v, out, dout, dq, dk, dv})
        if (!heads_aligned(x, type)) return ZNNI_ERR_ALIGN;
    const BackSizes s = back_sizes(type, B, Hq, Hk, D, max_q, max_k, left, right, sinks);
    BackArgs a = {};
    a.Hq = Hq; a.Hk = Hk; a.D = D;
    a.cu_q = cu_q; a.cu_k = cu_k;
    a.w = {left, right, sinks};
    a.scale = scale;
    a.max_q = max_q; a.max_k = max_k;
    a.pitch = s.pitch;
    a.heads = B * Hk;
    a.all_rows = (long long)B * Hk * s.pitch;
    a.rows = (const char*)workspace;
    a.parts = (float*)((char*)workspace + s.rows);
    const hipStream_t st = (hipStream_t)stream;
    switch (type) {
        case ZNNI_F32: return launch_back<float>(a, type, B, q, k, v, dout, out, stats, dq, dk, dv, st);
        case ZNNI_BF16: return launch_back<bf16>(a, type, B, q, k, v, dout, out, stats, dq, dk, dv, st);
        default: return launch_back<f16>(a, type, B, q, k, v, dout, out, stats, dq, dk, dv, st);
    }
}

}  // extern "C"
