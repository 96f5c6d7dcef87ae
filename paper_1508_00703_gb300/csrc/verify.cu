// Drafted tokens verified against the target's probabilities (pdb_verify).
//
// A sequence has D drafted tokens t_d, target logits z_0 .. z_D, draft logits y_0 .. y_{D-1}; p_d = softmax(scale z_d),
// q_d = softmax(draft_scale y_d).  Position after position, while u_d q_d(t_d) < p_d(t_d), the draft is accepted; where it is not
// (or the drafts end) the token is drawn from r = max(p - q, 0) (or r = p): the smallest j with r_0 + .. + r_j > v sum r.
// The tokens are then distributed as if drawn from p one after the other (Leviathan, Kalman, Matias 2023; Chen et al. 2023).
//
// One cluster of blocks walks a sequence's positions up to the first refusal.  A position's rows take one pass of running softmax
// statistics (rows.cuh), the draw one more over the rows of its position, which L2 mostly still holds.  Of few sequences the statistics of all
// rows are formed at once before that (k_verify_rows), those behind a refusal or a sequence's last draft too.
//
// Which token comes out must not hang on how a row is split or on 32-bit rounding: of 128,000 tokens the running sums of p lie so close that
// 32-bit ones would pick a neighbour in one draw of thirty.  So acceptances are taken from the statistics only where their error cannot
// matter (2^-15.6 apart for most tokens), and draws from terms good to 2^-31.5, summed as whole numbers (FastTerm), only where those cannot matter; the others, one
// of 1300 sequences with 5 drafts of 128,000 tokens (12 of 15,360), are decided on terms good to 2^-40 (exp_two), summed as whole numbers of 2^-92 (Units).
//
// What bounds it.  256 sequences of 5 drafts, 128,000 bf16 tokens, four of five accepted: 207 us; 463 MB, 69 us at the copy rate, 115 by
// a kernel that walks only (cluster barriers between positions: 4.1 TB/s), and 100 by one that draws only (71 instructions for a token of both
// rows, at 2.1 of 4 issued a cycle).  One sequence of 4 drafts: 15 us, two launches, seven cluster barriers and four passes of latency.
#include <algorithm>
#include <cmath>

#include "rows.cuh"

using namespace pdb;
namespace cg = cooperative_groups;

namespace {

constexpr int MAX_DRAFTS = 64;
constexpr int64_t MAX_VOCAB = 1 << 21;
constexpr int PIECE = 128;              // tokens whose weights are summed together

// ------------------------------------------------------------------ exp in two floats
// e^x = 2^k 2^(i/256) e^r with 256 k + i = rint(256 x / ln 2) and |r| <= ln 2 / 512 (table-driven, after Tang 1989), x and the
// result each the sum of two floats: the table holds 2^(i/256) to 2^-48, e^r = 1 + r + r^2/2 + r^3/6 + r^4/24 leaves 2^-52, and the
// rounding of r^2/2 <= 2^-20.1 is 2^-44 of the result.
constexpr double LN2_D = 0.693147180559945309417232121458;

constexpr double exp_series(double x)
{
    double term = 1.0, sum = 1.0;
    for (int i = 1; i < 30; ++i) term = term * x / i, sum += term;
    return sum;
}
template <int STEPS>
struct Exp2Table {
    float hi[STEPS], lo[STEPS];         // 2^(i/STEPS)
    constexpr Exp2Table() : hi(), lo()
    {
        for (int i = 0; i < STEPS; ++i) {
            const double v = exp_series(LN2_D * i / STEPS);
            hi[i] = (float)v;
            lo[i] = (float)(v - (double)(float)v);
        }
    }
};
__device__ const Exp2Table<256> EXP2_TABLE;

// ln 2 / 256 in four parts, the first three of 9 bits, so that their products with n of up to 15 bits are exact
constexpr double LN2_STEP = LN2_D / 256;
constexpr float STEP_1 = (float)((double)(int64_t)(LN2_STEP * 0x1p17) * 0x1p-17);
constexpr float STEP_2 = (float)((double)(int64_t)((LN2_STEP - (double)STEP_1) * 0x1p26) * 0x1p-26);
constexpr float STEP_3 = (float)((double)(int64_t)((LN2_STEP - (double)STEP_1 - (double)STEP_2) * 0x1p35) * 0x1p-35);
constexpr float STEP_4 = (float)(LN2_STEP - (double)STEP_1 - (double)STEP_2 - (double)STEP_3);
constexpr float PER_STEP = (float)(256 / LN2_D);

struct Two {
    float hi, lo;                       // hi + lo, |lo| <= ulp(hi)
};

// exp(scale * (z - m)), z <= m; 0 below e^-63 (2^-90.9)
__device__ __forceinline__ Two exp_two(float z, float m, float scale, const float2 *table)
{
    // z - m and its product with scale, exactly but for the last 2^-48
    const float d = __fsub_rn(z, m), b = __fsub_rn(d, z);
    const float dl = __fsub_rn(__fsub_rn(z, __fsub_rn(d, b)), __fadd_rn(m, b));
    const float x = __fmul_rn(d, scale);
    const float xl = __fmaf_rn(dl, scale, __fmaf_rn(d, scale, -x));
    if (!(x >= -63.0f)) return {0.0f, 0.0f};
    const float t = __fadd_rn(__fmul_rn(x, PER_STEP), 12582912.0f);       // 1.5 * 2^23: rounds to a whole number
    const int n = __float_as_int(t) - 0x4b400000;
    const float nf = __fsub_rn(t, 12582912.0f);
    // r = x - n ln2/256: exact as far as 2^-35 goes, what that leaves out in rl, which is then less than r's last digit
    const float r2 = __fmaf_rn(-nf, STEP_2, __fmaf_rn(-nf, STEP_1, x)), r1 = __fmaf_rn(-nf, STEP_3, r2);
    const float r0 = __fadd_rn(__fmaf_rn(-nf, STEP_3, __fsub_rn(r2, r1)), __fmaf_rn(-nf, STEP_4, xl));
    const float r = __fadd_rn(r1, r0), rl = __fadd_rn(__fsub_rn(r1, r), r0);
    // e^r - 1 = r + w
    const float q = __fmaf_rn(r, __fmaf_rn(r, 1.0f / 24.0f, 1.0f / 6.0f), 0.5f);
    const float w = __fmaf_rn(__fmul_rn(r, r), q, __fmaf_rn(rl, r, rl));
    const float2 tab = table[n & 255];
    const float ph = __fmul_rn(tab.x, r), pl = __fmaf_rn(tab.x, r, -ph);
    const float low = __fadd_rn(pl, __fmaf_rn(tab.x, w, __fmaf_rn(tab.y, r, tab.y)));
    const float h = __fadd_rn(tab.x, ph), l = __fadd_rn(__fadd_rn(__fsub_rn(tab.x, h), ph), low);
    const float sum = __fadd_rn(h, l), rest = __fadd_rn(__fsub_rn(h, sum), l);
    const float power = __int_as_float(((n >> 8) + 127) << 23);
    return {__fmul_rn(sum, power), __fmul_rn(rest, power)};
}

__device__ __forceinline__ Two times(Two a, Two b)
{
    const float h = __fmul_rn(a.hi, b.hi);
    return {h, __fadd_rn(__fmaf_rn(a.hi, b.hi, -h), __fmaf_rn(a.hi, b.lo, __fmul_rn(a.lo, b.hi)))};
}
// 1 / a
__device__ __forceinline__ Two inverse_of(Two a)
{
    const float h = __fdiv_rn(1.0f, a.hi);
    return {h, __fmul_rn(h, __fmaf_rn(-a.lo, h, __fmaf_rn(-a.hi, h, 1.0f)))};
}

// a + b, exactly
__device__ __forceinline__ Two sum_of(float a, float b)
{
    const float s = __fadd_rn(a, b), c = __fsub_rn(s, a);
    return {s, __fadd_rn(__fsub_rn(a, __fsub_rn(s, c)), __fsub_rn(b, c))};
}

// A sum of numbers from 0 to 1 in units of 2^-92, so that a term of a long tail keeps its digits beside a row's largest (rounded to 2^-46 of
// it, the 128,000 equal terms of a tail 2^-29 below it would be off by up to 2^-18 of themselves all in one direction, half a token's
// weight in all).  The units of 2^-23 are taken from the lowest bits of a float that is large enough; what is left can with the second float be
// 1.5 * 2^-24 and so is more than such bits hold; and what that leaves.
struct Units {
    int high = 0, low = 0, fine = 0, finest = 0;            // units of 2^-23, 2^-46, 2^-69, 2^-92
    __device__ __forceinline__ void add(Two a)
    {
        const float h = __fmaf_rn(a.hi, 0x1p23f, 8388608.0f);
        const Two rest = sum_of(__fmaf_rn(__fsub_rn(h, 8388608.0f), -0x1p-23f, a.hi), a.lo);
        const int l = __float2int_rn(__fmul_rn(rest.hi, 0x1p46f));
        const Two more = sum_of(__fmaf_rn((float)l, -0x1p-46f, rest.hi), rest.lo);
        const int f = __float2int_rn(__fmul_rn(more.hi, 0x1p69f));
        const float last = __fadd_rn(__fmaf_rn((float)f, -0x1p-69f, more.hi), more.lo);
        high += __float_as_int(h) - 0x4b000000, low += l, fine += f;
        finest += __float2int_rn(__fmul_rn(__fmul_rn(last, 0x1p46f), 0x1p46f));
    }
    __device__ __forceinline__ int64_t whole() const { return ((int64_t)high << 23) + low; }          // of 2^-46
    __device__ __forceinline__ int64_t rest() const { return (int64_t)fine * 0x800000 + finest; }     // of 2^-92
};
// (high * 2^23 + low) * 2^-46 + rest * 2^-92
__device__ __forceinline__ Two two_of(int64_t high, int64_t low, int64_t rest = 0)
{
    high += low >> 23, low &= 0x7fffff;
    const float h = __ll2float_rn(high);
    const int64_t left = high - __float2ll_rn(h);
    const float l = __fmaf_rn(__ll2float_rn(rest), 0x1p-46f, __ll2float_rn(left * 0x800000 + low));
    return {__fmul_rn(h, 0x1p-23f), __fmul_rn(l, 0x1p-46f)};
}

// whole numbers of 2^-92
typedef __int128 Wide;
constexpr int64_t REST = ((int64_t)1 << 46) - 1;
__device__ __forceinline__ Wide wide(int64_t whole, int64_t rest) { return (Wide)whole * (REST + 1) + rest; }
__device__ __forceinline__ Two two_of(Wide x)
{
    const int64_t whole = (int64_t)(x >> 46);
    return two_of(whole >> 23, whole & 0x7fffff, (int64_t)x & REST);
}

// max(a, 0) in units of 2^-46, and the rest of 2^-92
struct Weight {
    int64_t whole, rest;
};
__device__ __forceinline__ Weight weight_of(Two a)
{
    if (!(a.hi > 0.0f)) return {0, 0};
    Units one;
    one.add(a);
    const int64_t rest = one.rest();
    return {one.whole() + (rest >> 46), rest & REST};
}
// a - b
__device__ __forceinline__ Two less_by(Two a, Two b)
{
    const Two d = sum_of(a.hi, -b.hi);
    return sum_of(d.hi, __fadd_rn(d.lo, __fsub_rn(a.lo, b.lo)));
}

// floor(v * total), total - 1 at most (v from 1 on), 0 for a v below 0 or NaN; total below 2^103
__device__ __forceinline__ Wide share_of_total(float v, Wide total)
{
    if (!(v > 0.0f)) return 0;
    if (v >= 1.0f) return total - 1;
    const uint32_t raw = __float_as_uint(v), e = raw >> 23;
    const uint32_t digits = e ? (raw & 0x7fffff) | 0x800000 : raw & 0x7fffff;          // v = digits / 2^shift
    const int shift = 150 - (int)(e ? e : 1);
    return shift < 127 ? total * digits >> shift : 0;
}

// exp(scale (z - m)) 2^-down of two tokens at once, z <= m, where |m scale| log2(e) < 2^9, to 2^-31.5: n + f = 512 (z c - m c),
// c = scale log2(e), n whole and |f| <= 1, f formed by roundings of 2^-25; with n = 512 (-k) + i, 2^(i/512) + 2^(i/512) (2^(f/512) - 1) times a
// power of two.  An error that all tokens of a row share falls out of its probabilities.  What the sums are made of are whole numbers of 2^-22 and of
// 2^-44, both in the lowest bits of a float: additions and multiplications by the pair do nearly all of it (whole numbers
// shifted into place took 2.5 times as long: half of the integer unit's instructions).
constexpr float REACH = 512.0f;
constexpr int STEPS = 512, LOG_STEPS = 9;
__device__ const Exp2Table<STEPS> FAST_TABLE;
constexpr int HIGH0 = 0x4b000000, LOW0 = 0x4b400000;       // the bits of 2^23 and 1.5 * 2^23

__device__ __forceinline__ uint64_t both(float x) { return pair(x, x); }

struct FastTerm {
    uint64_t ch, cl, from, rest;        // of the first token's row, of the second's
    float low0, low1;
    uint32_t bias0, bias1;              // of the powers of two's bits
    __device__ __forceinline__ FastTerm(float m0, float scale0, int down0, float m1, float scale1, int down1)
    {
        float c[2], d[2], f[2], r[2];
        of_row(m0, scale0, down0, c[0], d[0], f[0], r[0], low0, bias0);
        of_row(m1, scale1, down1, c[1], d[1], f[1], r[1], low1, bias1);
        ch = pair(c[0], c[1]), cl = pair(d[0], d[1]), from = pair(f[0], f[1]), rest = pair(r[0], r[1]);
    }
    static __device__ __forceinline__ void of_row(float m, float scale, int down, float &c1, float &c2, float &from, float &rest, float &low,
                                                  uint32_t &bias)
    {
        constexpr float log2e_rest = (float)(1.4426950408889634073599 - (double)LOG2E);
        const float c = __fmul_rn(scale, LOG2E), c_rest = __fmaf_rn(scale, log2e_rest, __fmaf_rn(scale, LOG2E, -c));
        c1 = __fmul_rn(c, (float)STEPS), c2 = __fmul_rn(c_rest, (float)STEPS);
        const float mc = __fmul_rn(m, c1), whole = rintf(mc);
        from = __fsub_rn(12582912.0f, whole);
        rest = -__fadd_rn(__fsub_rn(mc, whole), __fmaf_rn(m, c2, __fmaf_rn(m, c1, -mc)));
        low = __fsub_rn(m, __fdiv_rn(60.0f, c));             // nothing below 2^-60
        bias = ((uint32_t)(127 + 22 - down) << 23) - ((uint32_t)(LOW0 >> LOG_STEPS) << 23);
    }
    // value: the terms times 2^22; high - HIGH0 units of 2^-22 and lowest - LOW0 of 2^-44 (what is left is 0.625 of 2^-22 at most)
    __device__ __forceinline__ void operator()(float z0, float z1, const float2 *table, float (&value)[2], int (&high)[2],
                                               int (&lowest)[2]) const
    {
        constexpr double L = LN2_D / STEPS;
        const uint64_t z = pair(fmaxf(z0, low0), fmaxf(z1, low1));
        const uint64_t t = fma2(z, ch, from);                // n in its lowest bits
        const uint64_t f = add2(fma2(z, ch, fma2(t, both(-1.0f), from)), fma2(z, cl, rest));
        const uint64_t s = mul2(f, fma2(f, fma2(f, both((float)(L * L * L / 6)), both((float)(L * L / 2))), both((float)L)));
        float t0, t1, x0, x1;
        unpair(t, t0, t1);
        const uint32_t n0 = __float_as_uint(t0), n1 = __float_as_uint(t1);
        const float2 a = table[n0 & (STEPS - 1)], b = table[n1 & (STEPS - 1)];
        const uint64_t power = pair(__uint_as_float(((n0 >> LOG_STEPS) << 23) + bias0), __uint_as_float(((n1 >> LOG_STEPS) << 23) + bias1));
        const uint64_t main = mul2(pair(a.x, b.x), power), more = mul2(fma2(pair(a.x, b.x), s, pair(a.y, b.y)), power);
        const uint64_t sum = add2(main, more);
        unpair(sum, value[0], value[1]);
        const uint64_t h = add2(sum, both(8388608.0f));
        unpair(h, x0, x1);
        high[0] = __float_as_int(x0), high[1] = __float_as_int(x1);
        // what is left of main + more, without rounding
        const uint64_t left = add2(fma2(add2(h, both(-8388608.0f)), both(-1.0f), main), more);
        unpair(fma2(left, both(4194304.0f), both(12582912.0f)), x0, x1);
        lowest[0] = __float_as_int(x0), lowest[1] = __float_as_int(x1);
    }
};
__device__ __forceinline__ int64_t units(int high, int low) { return (int64_t)high * 0x400000 + low; }

// How far from its token's borders a draw by FastTerm must lie to be taken, in units of 2^-44: the terms' rounding to units moves the running sum
// and v times the whole one by two for each token, ratios and products round down; and their errors e = 2^-31.5 count with (1 - v) up
// to the border and with v behind it, in all (1 - v) below + v behind: with P of p's terms below, `all` of them, half of e times all for most borders.
// The ratio of the rows' sums, between 1/2 and 2, is off by 2 e of itself, by 2^-30 for its last digit and as much for its divisor's, which
// moves both sides of q's: |Q - v all|.
// P and Q are those before the token's piece, dP and dQ the piece's.
__device__ __forceinline__ int64_t rounding_margin(int cols) { return 2 * (int64_t)cols + 8; }
__device__ __forceinline__ int64_t term_margin(float v, int64_t P, int64_t dP, int64_t all_p, int64_t Q, int64_t dQ, int64_t all_q)
{
    constexpr float E = 0x1.7p-32f, RATIO = 4 * E + 0x1p-29f;        // (2^-31.5 = 0x1.6a1p-32)
    v = fminf(fmaxf(v, 0.0f), 1.0f);
    const float w = __fsub_rn(1.0f, v), p = __ll2float_rn(P + dP), q = __ll2float_rn(Q + dQ);
    const float of_p = __fmaf_rn(w, p, __fmul_rn(v, __ll2float_rn(all_p - P)));
    const float of_q = __fmaf_rn(w, q, __fmul_rn(v, __ll2float_rn(all_q - Q)));
    const float shift = __fadd_rn(fabsf(__fmaf_rn(-v, __ll2float_rn(all_q), q)), __ll2float_rn(dQ));
    const float margin = __fmaf_rn(E, __fadd_rn(of_p, __fmul_rn(2.0f, of_q)), __fmul_rn(RATIO, shift));
    return __float2ll_ru(__fmul_rn(margin, 1.001f));
}
// what counts as near p = q, and how far off the statistics may be for it to hold all that they may have on the wrong side
constexpr float NEAR = 0x1p-16f, NEAR_OFF = 0x1p-17f;

// ------------------------------------------------------------------ shared by the blocks of a sequence
struct Shared {
    float part[2][2][16];               // the warps' m, s of the target's and the draft's row
    float stat[2][2][2];                // this block's, for two positions in turn
    float z[2][2];                      // the rows' logits of the drafted token, for two positions in turn
    int drafted[MAX_DRAFTS];
    float u[MAX_DRAFTS];
    Wide warp_sum[16];
    Wide sum[2];                        // this block's sums of the two rows
    Two row_sum[2], row_inv[2];         // the rows' sums, and their reciprocals
    Wide total;                         // this block's weights
    Wide at, before;                    // the drawn place among all weights, the weights of lower blocks
    Wide below;                         // weights before the piece that holds the drawn token
    int none, piece, good, unsure;
    // a draw by FastTerm: sums of the rows' terms, and of those of the tokens that count, by warp and over the block; what lies near p = q
    int64_t fast_warp[4][16], fast[4];
    float near_warp[16], near;
    int64_t low_p, low_q, all_p, all_q; // the sums of lower blocks, of all
    int64_t fast_at;                    // the drawn place
    int64_t margin;
    uint32_t ratio;                     // of the rows' sums, in units of 2^-30
    float2 table[256], fast_table[STEPS];
    int64_t weight[1];                  // of each of the block's pieces (as many as there are), then the rests; with FastTerm p's, then q's
};

// one row of a position
template <typename T>
struct Row {
    const T *z;
    float scale, m, s;                  // its maximum, sum of exp(scale (z - m))
    __device__ __forceinline__ bool valid() const { return s > 0.0f && s < INFINITY; }
};

template <typename T, int THREADS>
struct Walk {
    Shared &sh;
    cg::cluster_group cluster;
    int rank, blocks, cols;
    int first_piece, pieces;            // the block's

    // m and s of one or two rows (row(i): where the i-th lies, c(i): its scale * log2(e)) over the cluster, to out(i, m, s) on all threads.
    // The chunks of both follow one another, each loaded while the one before is added.
    template <typename R, typename C, typename F>
    __device__ __forceinline__ void stats(int rows, R row, C c_of, int turn, F out)
    {
        constexpr int W = THREADS / 32, SPAN = THREADS * UNROLL;
        const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
        uint4 v[UNROLL];
        const T *z = row(0);
        Share s = share_of(z, cols, rank, blocks);
        bool has_edge = (int)threadIdx.x < s.edges();
        T z_edge = from_float<T>(0.0f);
        if (has_edge) z_edge = z[s.edge(threadIdx.x)];
        load_vectors<T, THREADS, 32>(v, reinterpret_cast<const uint4 *>(z + s.b0), 0, lane_start(), s.v1 - s.v0);
        Stat<false> a;
        float top = -INFINITY;
        int base = 0;
#pragma unroll 1
        for (int i = 0; i < rows;) {
            const float c = c_of(i);
            const bool ends = base + SPAN >= s.v1 - s.v0;
            const bool edge = has_edge;
            const T own_edge = z_edge;
            base = ends ? 0 : base + SPAN;
            if (ends && i + 1 < rows) {
                z = row(i + 1);
                s = share_of(z, cols, rank, blocks);
                has_edge = (int)threadIdx.x < s.edges();
                if (has_edge) z_edge = z[s.edge(threadIdx.x)];
            }
            uint4 next[UNROLL];
            load_vectors<T, THREADS, 32>(next, reinterpret_cast<const uint4 *>(z + s.b0), base, lane_start(),
                                         ends && i + 1 == rows ? 0 : s.v1 - s.v0);
            add_vectors<T, false>(a, v, c, top);
            if (ends) {
                if (edge) add_element(a, to_float(own_edge), c);
                a.rebase(fmaxf(a.m, top), c);             // to the maximum itself
                a.template warp_join<32>(c);
                if (lane == 0) sh.part[i][0][warp] = a.m, sh.part[i][1][warp] = a.s;
                a = Stat<false>();
                top = -INFINITY;
                ++i;
            }
#pragma unroll
            for (int u = 0; u < UNROLL; ++u) v[u] = next[u];
        }
        __syncthreads();
        for (int i = warp; i < rows; i += W) {
            a.m = sh.part[i][0][lane & (W - 1)], a.s = sh.part[i][1][lane & (W - 1)];
            a.template warp_join<W>(c_of(i));
            if (lane == 0) sh.stat[turn][i][0] = a.m, sh.stat[turn][i][1] = a.s;
        }
        cluster.sync();
        // every warp for itself: barriers are what a position's end costs
        for (int i = 0; i < rows; ++i) {
            a = Stat<false>();
            const int b = lane & (MAX_CLUSTER - 1);
            if (b < blocks) {
                const float *o = cluster.map_shared_rank(&sh, b)->stat[turn][i];
                a.m = o[0], a.s = o[1];
            }
            a.template warp_join<MAX_CLUSTER>(c_of(i));
            out(i, a.m, a.s);
        }
    }

    __device__ __forceinline__ void fill_table()
    {
        for (int i = threadIdx.x; i < 256; i += THREADS) sh.table[i] = {EXP2_TABLE.hi[i], EXP2_TABLE.lo[i]};
        __syncthreads();
    }

    // f(the lane's tokens of a piece: z and, where there is one, y) of the warp's pieces; a piece's are loaded before the one before is
    // worked on
    template <typename F>
    __device__ __forceinline__ void each_piece(const T *z, const T *y, F f)
    {
        constexpr int N = PIECE / 32, W = THREADS / 32;
        const int lane = threadIdx.x & 31;
        const T none = from_float<T>(-INFINITY);
        T a[N], b[N];
        auto load = [&](int i) {
            const int j = (first_piece + i) * PIECE + lane;
            if (i < pieces && (first_piece + i + 1) * PIECE <= cols) {
#pragma unroll
                for (int u = 0; u < N; ++u) a[u] = z[j + u * 32];
                if (y)
#pragma unroll
                    for (int u = 0; u < N; ++u) b[u] = y[j + u * 32];
            } else {
#pragma unroll
                for (int u = 0; u < N; ++u) {
                    const bool on = i < pieces && j + u * 32 < cols;
                    a[u] = b[u] = none;
                    if (on) a[u] = z[j + u * 32];
                    if (on && y) b[u] = y[j + u * 32];
                }
            }
        };
        int i = threadIdx.x >> 5;
        load(i);
#pragma unroll 1
        for (; i < pieces; i += W) {
            T x[N], w[N];
#pragma unroll
            for (int u = 0; u < N; ++u) x[u] = a[u], w[u] = b[u];
            load(i + W);
            f(i, x, w);
        }
    }

    // the number of the lane `off` below, or across
    static __device__ __forceinline__ Wide of_lane(Wide x, int off, bool across)
    {
        const uint64_t low = (uint64_t)x, high = (uint64_t)(x >> 64);
        const uint64_t l = across ? __shfl_xor_sync(FULL, low, off) : __shfl_up_sync(FULL, low, off);
        const uint64_t h = across ? __shfl_xor_sync(FULL, high, off) : __shfl_up_sync(FULL, high, off);
        return (Wide)((unsigned __int128)h << 64 | l);
    }
    // the sum of the threads' numbers, on thread 0
    __device__ __forceinline__ Wide block_sum(Wide x)
    {
#pragma unroll
        for (int off = 16; off >= 1; off >>= 1) x += of_lane(x, off, true);
        __syncthreads();                 // (the last sum has been read)
        if ((threadIdx.x & 31) == 0) sh.warp_sum[threadIdx.x >> 5] = x;
        __syncthreads();
        if (threadIdx.x == 0)
            for (int w = 1; w < THREADS / 32; ++w) x += sh.warp_sum[w];
        return x;
    }

    // a row's sum lies between 2^(above - 1) and 2^above, but for the statistics' error
    static __device__ __forceinline__ int above(const Row<T> &r) { return (int)(__float_as_uint(__fmul_rn(r.s, 1.0f + 0x1p-10f)) >> 23) - 126; }

    // The rows' sums, of terms good to 2^-40, into sh.row_sum and sh.row_inv.  Whole numbers are added up: no order of warps and
    // blocks shows in them.
    __device__ __forceinline__ void sums(const Row<T> &p, const Row<T> &q)
    {
        constexpr int N = PIECE / 32;
#pragma unroll 1
        for (int which = 0; which < (q.z ? 2 : 1); ++which) {
            const float m = which ? q.m : p.m, scale = which ? q.scale : p.scale;
            int64_t whole = 0, rest = 0;
            each_piece(which ? q.z : p.z, nullptr, [&](int, const T (&x)[N], const T (&)[N]) {
                Units sum;
#pragma unroll
                for (int u = 0; u < N; ++u) sum.add(exp_two(to_float(x[u]), m, scale, sh.table));
                whole += sum.whole(), rest += sum.rest();
            });
            const Wide all = block_sum(wide(whole, rest));
            if (threadIdx.x == 0) sh.sum[which] = all;
        }
        cluster.sync();
        if (threadIdx.x < (q.z ? 2 : 1)) {
            Wide all = 0;
            for (int b = 0; b < blocks; ++b) all += cluster.map_shared_rank(&sh, b)->sum[threadIdx.x];
            sh.row_sum[threadIdx.x] = two_of(all);
            sh.row_inv[threadIdx.x] = inverse_of(sh.row_sum[threadIdx.x]);
        }
        cluster.sync();                  // the others' sums have been read
    }

    // tokens' weights in a draw
    struct Weights {
        Row<T> p, q;
        Two p_inv, q_inv;
        int without;                     // a token left out
        const float2 *table;
        __device__ __forceinline__ Weight operator()(int j, T z, T y) const
        {
            Two a = times(exp_two(to_float(z), p.m, p.scale, table), p_inv);
            if (q.z) a = less_by(a, times(exp_two(to_float(y), q.m, q.scale, table), q_inv));
            return j == without ? Weight{0, 0} : weight_of(a);
        }
    };

    // inclusive sums over the lanes
    static __device__ __forceinline__ int64_t scan(int64_t x)
    {
#pragma unroll
        for (int off = 1; off < 32; off <<= 1) {
            const int64_t y = __shfl_up_sync(FULL, x, off);
            if ((int)(threadIdx.x & 31) >= off) x += y;
        }
        return x;
    }
    static __device__ __forceinline__ Wide scan(Wide x)
    {
#pragma unroll
        for (int off = 1; off < 32; off <<= 1) {
            const Wide y = of_lane(x, off, false);
            if ((int)(threadIdx.x & 31) >= off) x += y;
        }
        return x;
    }
    // the sum of the lanes' numbers, from 0 to 2^53
    static __device__ __forceinline__ int64_t lanes_sum(int64_t x)
    {
        return ((int64_t)__reduce_add_sync(FULL, (unsigned)(x >> 27)) << 27) + __reduce_add_sync(FULL, (unsigned)x & 0x7ffffff);
    }
    // a lane's neighbouring tokens of a piece
    template <int N>
    __device__ __forceinline__ void lane_tokens(const T *z, int j0, T (&x)[N]) const
    {
#pragma unroll
        for (int u = 0; u < N; ++u) {
            x[u] = from_float<T>(-INFINITY);
            if (z && j0 + u < cols) x[u] = z[j0 + u];
        }
    }

    // The smallest token whose running sum of weights passes v times all of them, and its logit: on the thread that finds it, -1 on
    // the others.  Sets sh.none where no token has a weight.
    __device__ __forceinline__ int draw(const Weights &weight, float v, float &logit)
    {
        constexpr int N = PIECE / 32;
        const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
        Wide all = 0;                    // on lane 0
        int64_t *const rest = sh.weight + pieces;
        each_piece(weight.p.z, weight.q.z, [&](int i, const T (&z)[N], const T (&y)[N]) {
            Weight own = {0, 0};
#pragma unroll
            for (int u = 0; u < N; ++u) {
                const Weight w = weight((first_piece + i) * PIECE + u * 32 + lane, z[u], y[u]);
                own.whole += w.whole, own.rest += w.rest;
            }
            const int64_t whole = lanes_sum(own.whole), more = lanes_sum(own.rest);
            if (lane == 0) {
                sh.weight[i] = whole, rest[i] = more;
                all += wide(whole, more);
            }
        });
        all = block_sum(all);
        if (threadIdx.x == 0) sh.total = all;
        cluster.sync();
        if (threadIdx.x == 0) {
            Wide before = 0, total = 0;
            for (int b = 0; b < blocks; ++b) {
                const Wide x = cluster.map_shared_rank(&sh, b)->total;
                if (b < rank) before += x;
                total += x;
            }
            sh.none = total <= 0;
            sh.before = before;
            sh.at = share_of_total(v, total);
        }
        cluster.sync();                  // the others' totals have been read
        int found = -1;
        const Wide at = sh.at, before = sh.before;
        if (warp == 0 && !sh.none && at >= before && at < before + sh.total) {
            // a lane's run of pieces, then its pieces
            const int each = (pieces + 31) / 32, i0 = min(pieces, lane * each), i1 = min(pieces, i0 + each);
            Wide mine = 0;
            for (int i = i0; i < i1; ++i) mine += wide(sh.weight[i], rest[i]);
            Wide below = before + scan(mine) - mine;
            if (at >= below && at < below + mine) {
                int i = i0;
                for (; at >= below + wide(sh.weight[i], rest[i]); ++i) below += wide(sh.weight[i], rest[i]);
                sh.piece = first_piece + i;
                sh.below = below;
            }
            __syncwarp();
            const int j0 = sh.piece * PIECE + lane * N;
            T z[N], y[N];
            lane_tokens(weight.p.z, j0, z);
            lane_tokens(weight.q.z, j0, y);
            Wide w[N], sum = 0;
#pragma unroll
            for (int u = 0; u < N; ++u) {
                const Weight one = weight(j0 + u, z[u], y[u]);
                w[u] = wide(one.whole, one.rest), sum += w[u];
            }
            below = sh.below + scan(sum) - sum;
#pragma unroll
            for (int u = 0; u < N; ++u) {
                if (at >= below && at < below + w[u]) found = j0 + u, logit = to_float(z[u]);
                below += w[u];
            }
        }
        return found;
    }

    // The same by FastTerm in one pass, with sh.unsure set where it may not be that token.  The weights are p - (SP / SQ) q of the tokens where that is
    // positive, SP and SQ the rows' sums, which are known at the end of the pass only; so what is summed are the terms of p and those of q, over all
    // tokens and over those where p / s > q / s', s and s' the sums as the 32-bit statistics have them.  A token is taken for the wrong side only
    // where p and q differ by less than the statistics' error, and that error times the probability of the tokens near p = q (to NEAR of p) bounds
    // what it adds.
    template <bool LESS>
    __device__ __forceinline__ int fast_draw(const Row<T> &p, const Row<T> &q, int without, float v, float &logit)
    {
        constexpr int N = PIECE / 32, W = THREADS / 32;
        const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
        // the rows' sums are brought to the same size, as large as the largest term and 62 bits allow: fine units
        const int above_p = above(p), above_q = LESS ? above(q) : above_p, fine = min(min(above_p, above_q), 17);
        // two tokens of p, or one of p and q each
        const FastTerm term(p.m, p.scale, above_p - fine, LESS ? q.m : p.m, LESS ? q.scale : p.scale, above_q - fine);
        // the terms' probabilities, as the statistics have them
        const float p_inv = __fdiv_rn(__int_as_float((127 + above_p - fine - 22) << 23), p.s);
        const float q_inv = LESS ? __fdiv_rn(__int_as_float((127 + above_q - fine - 22) << 23), q.s) : 0.0f;
        int64_t *const weight_q = sh.weight + pieces;
        int64_t sum_p = 0, sum_q = 0, in_p = 0, in_q = 0;
        float near = 0.0f;
        each_piece(p.z, LESS ? q.z : nullptr, [&](int i, const T (&raw_z)[N], const T (&raw_y)[N]) {
            float z[N], y[N];
#pragma unroll
            for (int u = 0; u < N; ++u) z[u] = to_float(raw_z[u]), y[u] = to_float(raw_y[u]);
            uint32_t ph = 0u - (uint32_t)N * HIGH0, pl = 0u - (uint32_t)N * LOW0, qh = ph, ql = pl;      // all tokens (LESS)
            int aph = 0, apl = 0, aqh = 0, aql = 0;                    // those that count
            if constexpr (LESS) {
#pragma unroll
                for (int u = 0; u < N; ++u) {
                    float c[2];
                    int h[2], l[2];
                    term(z[u], y[u], sh.fast_table, c, h, l);
                    ph += h[0], pl += l[0], qh += h[1], ql += l[1];
                    const float a = __fmul_rn(c[0], p_inv), over = __fmaf_rn(-c[1], q_inv, a);
                    if (fabsf(over) <= __fmul_rn(a, NEAR)) near = __fadd_rn(near, a);
                    if (over > 0.0f) aph += h[0] - HIGH0, apl += l[0] - LOW0, aqh += h[1] - HIGH0, aql += l[1] - LOW0;
                }
            } else {
                const int skip = without >= 0 ? without - (first_piece + i) * PIECE - lane : -1;
#pragma unroll
                for (int u = 0; u < N; u += 2) {
                    float c[2];
                    int h[2], l[2];
                    term(z[u], z[u + 1], sh.fast_table, c, h, l);
#pragma unroll
                    for (int x = 0; x < 2; ++x)
                        if (skip != (u + x) * 32) aph += h[x] - HIGH0, apl += l[x] - LOW0;
                }
            }
            if (LESS) sum_p += units((int)ph, (int)pl), sum_q += units((int)qh, (int)ql);
            aph = __reduce_add_sync(FULL, aph), apl = __reduce_add_sync(FULL, apl);
            if (LESS) aqh = __reduce_add_sync(FULL, aqh), aql = __reduce_add_sync(FULL, aql);
            if (lane == 0) {
                sh.weight[i] = units(aph, apl);
                in_p += units(aph, apl);
                if (LESS) weight_q[i] = units(aqh, aql), in_q += units(aqh, aql);
            }
        });
        const int64_t own[4] = {in_p, in_q, sum_p, sum_q};
#pragma unroll
        for (int k = 0; k < (LESS ? 4 : 1); ++k) {
            int64_t x = own[k];
            if (k >= 2)
#pragma unroll
                for (int off = 16; off >= 1; off >>= 1) x += __shfl_xor_sync(FULL, x, off);
            if (lane == 0) sh.fast_warp[k][warp] = x;
        }
        if (LESS) {
#pragma unroll
            for (int off = 16; off >= 1; off >>= 1) near = __fadd_rn(near, __shfl_xor_sync(FULL, near, off));
            if (lane == 0) sh.near_warp[warp] = near;
        }
        __syncthreads();
        if (threadIdx.x < 4) {
            int64_t x = 0;
            for (int w = 0; w < (LESS || threadIdx.x == 0 ? W : 0); ++w) x += sh.fast_warp[threadIdx.x][w];
            sh.fast[threadIdx.x] = x;
        } else if (threadIdx.x == 32) {
            float x = 0.0f;
            for (int w = 0; w < (LESS ? W : 0); ++w) x = __fadd_rn(x, sh.near_warp[w]);
            sh.near = x;
        }
        cluster.sync();
        if (threadIdx.x == 0) {
            int64_t all[4] = {0, 0, 0, 0}, low_p = 0, low_q = 0;
            float close = 0.0f;
            for (int b = 0; b < blocks; ++b) {
                const Shared *o = cluster.map_shared_rank(&sh, b);
#pragma unroll
                for (int k = 0; k < (LESS ? 4 : 1); ++k) all[k] += o->fast[k];
                close = __fadd_rn(close, o->near);
                if (b < rank) low_p += o->fast[0], low_q += o->fast[1];
            }
            sh.low_p = low_p, sh.low_q = low_q, sh.all_p = all[0], sh.all_q = all[1];
            sh.ratio = 0, sh.margin = rounding_margin(cols), sh.unsure = false;
            if (LESS) {
                sh.ratio = (uint32_t)(((uint64_t)(all[2] >> fine) << 18) / (uint64_t)max((long long)(all[3] >> fine >> 12), 1ll));
                // the statistics' error, from what the sums have come to
                const float x = __fmul_rn(__fdiv_rn(__ll2float_rn(all[2]), __ll2float_rn(all[3])), __fdiv_rn(p_inv, q_inv));
                const float off = __fadd_rn(fabsf(__fsub_rn(x, 1.0f)), 0x1p-20f);
                sh.unsure = !(off < NEAR_OFF);
                sh.margin += __float2ll_rn(__fmul_rn(__fmul_rn(off, __fmul_rn(close, 1.01f)), __int_as_float((127 + 44 + fine) << 23)));
            }
            const int64_t total = all[0] - less(all[1], sh.ratio);
            if (total <= 2 * sh.margin) sh.unsure = true;
            sh.fast_at = (int64_t)share_of_total(v, max((long long)total, 1ll));
        }
        cluster.sync();                  // the others' sums have been read
        int found = -1;
        const int64_t at = sh.fast_at;
        const uint32_t ratio = sh.ratio;
        int64_t P = sh.low_p, Q = sh.low_q;
        if (warp == 0 && !sh.unsure && at >= P - less(Q, ratio) && at < P + sh.fast[0] - less(Q + sh.fast[1], ratio)) {
            const int each = (pieces + 31) / 32, i0 = min(pieces, lane * each), i1 = min(pieces, i0 + each);
            int64_t mine_p = 0, mine_q = 0;
            for (int i = i0; i < i1; ++i) {
                mine_p += sh.weight[i];
                if (LESS) mine_q += weight_q[i];
            }
            int64_t to_p = P + scan(mine_p), to_q = LESS ? Q + scan(mine_q) : 0;
            const bool here = i1 > i0 && at >= to_p - mine_p - less(to_q - mine_q, ratio) && at < to_p - less(to_q, ratio);
            const unsigned lanes = __ballot_sync(FULL, here);
            bool sure = false;
            if (lanes) {
                if (lane == __ffs(lanes) - 1) {
                    P = to_p - mine_p, Q = to_q - mine_q;
                    int i = i0;
                    for (; i < i1 - 1; ++i) {
                        const int64_t next_p = P + sh.weight[i], next_q = Q + (LESS ? weight_q[i] : 0);
                        if (at < next_p - less(next_q, ratio)) break;
                        P = next_p, Q = next_q;
                    }
                    sh.piece = first_piece + i;
                    sh.low_p = P, sh.low_q = Q;
                }
                __syncwarp();
                const int j0 = sh.piece * PIECE + lane * N;
                T z[N], y[N];
                lane_tokens(p.z, j0, z);
                lane_tokens(LESS ? q.z : nullptr, j0, y);
                int64_t wp[N], wq[N], sum_p = 0, sum_q = 0;
#pragma unroll
                for (int u = 0; u < N; ++u) {
                    float c[2];
                    int h[2], l[2];
                    term(to_float(z[u]), to_float(LESS ? y[u] : z[u]), sh.fast_table, c, h, l);
                    const bool counts = LESS ? __fmaf_rn(-c[1], q_inv, __fmul_rn(c[0], p_inv)) > 0.0f : j0 + u != without;
                    wp[u] = counts ? units(h[0] - HIGH0, l[0] - LOW0) : 0;
                    wq[u] = LESS && counts ? units(h[1] - HIGH0, l[1] - LOW0) : 0;
                    sum_p += wp[u], sum_q += wq[u];
                }
                const int64_t to_lane_p = scan(sum_p), to_lane_q = LESS ? scan(sum_q) : 0;
                const int64_t margin = sh.margin + term_margin(v, sh.low_p, __shfl_sync(FULL, to_lane_p, 31), sh.all_p, LESS ? sh.low_q : 0,
                                                               __shfl_sync(FULL, to_lane_q, 31), LESS ? sh.all_q : 0);
                P = sh.low_p + to_lane_p - sum_p, Q = LESS ? sh.low_q + to_lane_q - sum_q : 0;
#pragma unroll
                for (int u = 0; u < N; ++u) {
                    const int64_t from = P - less(Q, ratio);
                    P += wp[u], Q += wq[u];
                    if (at >= from + margin && at < P - less(Q, ratio) - margin) found = j0 + u, logit = to_float(z[u]), sure = true;
                }
                sure = __any_sync(FULL, sure);
            }
            if (!sure && lane < blocks) cluster.map_shared_rank(&sh, lane)->unsure = true;
        }
        cluster.sync();                  // every block knows
        return found;
    }
    // x * ratio / 2^30
    static __device__ __forceinline__ int64_t less(int64_t x, uint32_t ratio)
    {
        return (int64_t)(__umul64hi((uint64_t)x, (uint64_t)ratio) << 34 | (uint64_t)x * ratio >> 30);
    }
};

struct VerifyOut {
    int32_t *tokens, *accepted;
    float *logp;
};

// How far the two sides of an acceptance must lie apart for the statistics in 32 bits to decide it, in units of 2^-24 of the larger.
// An exponential's argument x (in powers of two) is off by 3.2 |x| units (the difference, its product, scale log2(e)), the power by
// 2.25 |x| + 4.  A row's sum has that by the mean over its mass, where |x| is at most log2(cols) (the entropy) and the references differ by 16: 2.25 * 37
// for 2^21 tokens; five powers' roundings, 25; the additions within a chunk and of joins, 27; and one for each chunk that a thread adds (they can
// all go one way: 2^21 fp32 tokens in one block of 512, 256 chunks, 520 units between two such rows).  Both rows 271, with divisions and u
// 284, and twice the chunks.
constexpr float SURE_X = 2.25f;
inline float sure_rows(int64_t vectors, int blocks, int threads)
{
    return 304.0f + 2.0f * (float)(vectors / blocks / (threads * UNROLL) + 1);
}

// a row's m, s and its logit of the drafted token, from k_verify_rows
struct Given {
    float m, s, z, unused;
};

// what is to be done at a position: a draw from p - q; from p; nothing (a target row without a distribution); what only exact numbers tell
enum { DRAW_REST = 0, DRAW_TARGET = 1, NOTHING = 2, EXACTLY = 3 };

// whether u q < p, where the statistics can tell it (sure)
template <typename T>
__device__ __forceinline__ bool accepts(const Row<T> &p, const Row<T> &q, float z, float zq, float u, float sure_rows, bool &sure)
{
    const float x = __fmul_rn(__fsub_rn(z, p.m), __fmul_rn(p.scale, LOG2E)), right = __fdiv_rn(ex2(x), p.s);
    float left = u, y = 0.0f;
    if (q.z) {
        y = __fmul_rn(__fsub_rn(zq, q.m), __fmul_rn(q.scale, LOG2E));
        left = __fmul_rn(u, __fdiv_rn(ex2(y), q.s));
    }
    // a power below the normal numbers is 0, however far
    const float margin = __fmaf_rn(SURE_X, fminf(-x, 150.0f) + fminf(-y, 150.0f), sure_rows);
    const float more = fmaxf(left, right);
    sure = fabsf(left - right) > 0x1p-24f * margin * more && more > 1e-30f;
    return left < right;
}

// what a position with its statistics comes to; -1 where its draft is surely accepted
template <typename T>
__device__ __forceinline__ int decide(const Row<T> &p, const Row<T> &q, int t, float z, float zq, float u, float sure_rows)
{
    if (!p.valid()) return NOTHING;
    if (t < 0 || (q.z && !q.valid())) return DRAW_TARGET;            // the drafts end here
    bool sure;
    const bool good = accepts(p, q, z, zq, u, sure_rows, sure);
    return !sure ? EXACTLY : good ? -1 : DRAW_REST;
}

// a sequence's drafted tokens (-1 from the end on) and random numbers; an id out of range is recorded where no id before it ends the drafts
template <int THREADS>
__device__ __forceinline__ void load_drafts(Shared &sh, Ids ids, int64_t s, int D, int cols, const float *accept_u, bool records, int *status)
{
    for (int d = threadIdx.x; d < D; d += THREADS) {
        const int64_t t = load_id(ids, s, d);
        sh.drafted[d] = t >= 0 && t < cols ? (int)t : -1;
        sh.u[d] = accept_u[s * D + d];
        if (t >= cols && records) {
            bool seen = true;
            for (int e = 0; e < d; ++e) {
                const int64_t before = load_id(ids, s, e);
                seen &= before >= 0 && before < cols;
            }
            if (seen) set_status(status, PDB_ERANGE);
        }
    }
}

// where a call's matrices and vectors lie
template <typename T>
struct Verify {
    const T *target, *draft;
    int64_t t_stride, d_stride;
    int cols, D;
    Ids ids;
    int64_t n;
    float scale, draft_scale, sure_rows;
    const float *accept_u, *draw_u;
    VerifyOut out;
    const Given *given;                 // of all rows, where k_verify_rows has been there
    int *status;
    __device__ __forceinline__ const T *target_row(int64_t s, int a) const { return target + (s * (D + 1) + a) * t_stride; }
    __device__ __forceinline__ const T *draft_row(int64_t s, int a) const { return draft + (s * D + a) * d_stride; }
    __device__ __forceinline__ void accept(int64_t s, int a, int t, float z, const Row<T> &p) const
    {
        out.tokens[s * (D + 1) + a] = t;
        if (out.logp) out.logp[s * (D + 1) + a] = __fmaf_rn(__fsub_rn(z, p.m), scale, -logf(p.s));
    }
    // a sequence's outputs behind its accepted drafts, but for the drawn token
    __device__ __forceinline__ void finish(int64_t s, int a, bool drawn) const
    {
        if (out.accepted) out.accepted[s] = a;
        for (int d = drawn ? a + 1 : a; d <= D; ++d) {
            out.tokens[s * (D + 1) + d] = -1;
            if (out.logp) out.logp[s * (D + 1) + d] = 0.0f;
        }
    }
    // a position's statistics as k_verify_rows left them
    __device__ __forceinline__ void look_up(int64_t s, int a, Row<T> &p, Row<T> &q, float &z, float &zq) const
    {
        const Given g = given[s * (D + 1) + a];
        p.m = g.m, p.s = g.s, z = g.z;
        if (q.z) {
            const Given h = given[n * (D + 1) + s * D + a];
            q.m = h.m, q.s = h.s, zq = h.z;
        }
    }
};

// Few sequences: the statistics of all their rows at once, a cluster for each.
template <typename T, int THREADS>
__global__ __launch_bounds__(THREADS, 1024 / THREADS) void k_verify_rows(Verify<T> v, Given *__restrict__ given)
{
    after_previous();
    let_next_start();
    __shared__ Shared sh;
    cg::cluster_group cluster = cg::this_cluster();
    const int blocks = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
    const int64_t r = blockIdx.x / (unsigned)blocks, targets = v.n * (v.D + 1);
    const bool drafts = r >= targets;
    const int each = drafts ? v.D : v.D + 1;
    const int64_t i = drafts ? r - targets : r, s = i / each;
    const int d = (int)(i - s * each);
    const T *row = drafts ? v.draft_row(s, d) : v.target_row(s, d);
    const bool writes = rank == 0 && threadIdx.x == 0;
    float z = 0.0f;
    if (writes && d < v.D) {
        const int64_t t = load_id(v.ids, s, d);
        if (t >= 0 && t < v.cols) z = to_float(row[t]);
    }
    Walk<T, THREADS> walk{sh, cluster, rank, blocks, v.cols, 0, 0};
    Row<T> of_row{};
    walk.stats(1, [&](int) { return row; }, [&](int) { return __fmul_rn(drafts ? v.draft_scale : v.scale, LOG2E); }, 0,
               [&](int, float m, float sum) { of_row.m = m, of_row.s = sum; });
    cluster.sync();                      // the others have read this block's statistics
    if (writes) given[r] = {of_row.m, of_row.s, z, 0.0f};
}

// |m scale| log2(e) within what FastTerm takes
template <typename T>
__device__ __forceinline__ bool in_reach(const Row<T> &r)
{
    return r.scale > 1e-30f && r.scale < 1e30f && fabsf(__fmul_rn(r.m, __fmul_rn(r.scale, LOG2E))) < REACH;
}

// A cluster for each sequence: its walk (bound by memory) up to the first position that is not accepted, and its draw (bound by instructions).
// On an SM some sequences walk while others draw; in a kernel each they take as long (256 x 5 drafts x 128,000 bf16: 115 us and 100), and the
// few that have to be exact are not hidden then.  An exact draw takes three passes more by the cluster that has the sequence: 38 us by eight blocks
// of 512; at the end of the launch up to 52 us of 159 (152 sequences, eight blocks of 256), 75 of 207 (256, four), 155 of 396 (608, two), 285 of
// 559 (912, one), in its middle 4, 15, 31 and 194.
constexpr int MANY_THREADS = 256, FEW_THREADS = 512, MANY_PER_SM = 3;

template <typename T, int THREADS>
__global__ __launch_bounds__(THREADS, THREADS == FEW_THREADS ? 1 : MANY_PER_SM) void k_verify(Verify<T> v)
{
    after_previous();
    extern __shared__ __align__(16) unsigned char s_raw[];
    Shared &sh = *reinterpret_cast<Shared *>(s_raw);
    cg::cluster_group cluster = cg::this_cluster();
    const int blocks = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
    const int64_t s = blockIdx.x / (unsigned)blocks;
    const int all = (v.cols + PIECE - 1) / PIECE;
    const int p0 = (int)((int64_t)all * rank / blocks), p1 = (int)((int64_t)all * (rank + 1) / blocks);
    Walk<T, THREADS> walk{sh, cluster, rank, blocks, v.cols, p0, p1 - p0};
    const bool writes = rank == 0 && threadIdx.x == 0;
    const float c = __fmul_rn(v.scale, LOG2E), cq = __fmul_rn(v.draft_scale, LOG2E);
    load_drafts<THREADS>(sh, v.ids, s, v.D, v.cols, v.accept_u, rank == 0, v.status);
    for (int i = threadIdx.x; i < STEPS; i += THREADS) sh.fast_table[i] = {FAST_TABLE.hi[i], FAST_TABLE.lo[i]};
    const float draw_u = v.draw_u[s];
    __syncthreads();
    Row<T> p{}, q{};
    p.scale = v.scale, q.scale = v.draft_scale;
    int a = 0, t = -1;                   // the position, its drafted token
    bool refused = false, exact = false; // exact: their table is there
#pragma unroll 1
    for (;; ++a) {
        t = a < v.D ? sh.drafted[a] : -1;
        p.z = v.target_row(s, a);
        q.z = t >= 0 && v.draft ? v.draft_row(s, a) : nullptr;
        float z = 0.0f, zq = 0.0f;
        if (v.given) {
            v.look_up(s, a, p, q, z, zq);
        } else {
            const int turn = a & 1;
            if (t >= 0 && threadIdx.x < (q.z ? 2 : 1)) sh.z[turn][threadIdx.x] = to_float((threadIdx.x ? q.z : p.z)[t]);
            walk.stats(q.z ? 2 : 1, [&](int i) { return i ? q.z : p.z; }, [&](int i) { return i ? cq : c; }, turn, [&](int i, float m, float sum) {
                (i ? q.m : p.m) = m, (i ? q.s : p.s) = sum;
            });
            z = sh.z[turn][0], zq = sh.z[turn][1];
        }
        const float u = t >= 0 ? sh.u[a] : 0.0f;
        int what = decide(p, q, t, z, zq, u, v.sure_rows);
        if (what == EXACTLY) {
            if (!exact) walk.fill_table();
            exact = true;
            walk.sums(p, q);
            if (threadIdx.x == 0) {
                const auto in_64 = [](float scale, float z, const Row<T> &r, Two sum) {
                    return exp((double)scale * ((double)z - (double)r.m)) / ((double)sum.hi + (double)sum.lo);
                };
                const double pe = in_64(v.scale, z, p, sh.row_sum[0]);
                const double qe = q.z ? in_64(v.draft_scale, zq, q, sh.row_sum[1]) : 1.0;
                sh.good = (double)u * qe < pe;
            }
            __syncthreads();
            what = sh.good ? -1 : DRAW_REST;
        }
        if (what >= 0) {
            refused = what == DRAW_REST;
            break;
        }
        if (writes) v.accept(s, a, t, z, p);
    }
    bool none = true;
    if (p.valid()) {
        if (!refused) q.z = nullptr;
        int without = refused && !q.z ? t : -1;
        bool fast = in_reach(p) && (!q.z || in_reach(q));
#pragma unroll 1
        for (;;) {
            float z = 0.0f;
            int drawn;
            if (fast) {
                drawn = q.z ? walk.template fast_draw<true>(p, q, -1, draw_u, z) : walk.template fast_draw<false>(p, q, without, draw_u, z);
            } else {
                if (!exact) walk.fill_table();
                exact = true;
                if (q.z) walk.sums(p, q);
                // one row's weights need no more than a common factor, a power of two
                const Two unit = {__int_as_float((127 - walk.above(p)) << 23), 0.0f};
                drawn = walk.draw({p, q, q.z ? sh.row_inv[0] : unit, sh.row_inv[1], without, sh.table}, draw_u, z);
            }
            const bool unsure = fast && sh.unsure;
            none = !fast && sh.none;
            if (drawn >= 0) v.accept(s, a, drawn, z, p);
            if (!unsure && (!none || !refused)) break;
            // once more, exactly; or, with nothing of p - q that 2^-92 could tell, from p
            if (!unsure) refused = false, q.z = nullptr, without = -1;
            fast = false;
            __syncthreads();
        }
    } else {
        cluster.sync();                  // the others have read this block's statistics
    }
    if (writes) v.finish(s, a, !none);
}

// What a block's pieces may take: MANY_PER_SM blocks find room on an SM.  A cluster gets more blocks until they do, whatever its number of
// sequences gives it.  bf16, draws alone, 1, 2, 4 and 8 blocks: 700 sequences of 500,000 tokens 710 us, 689, 673, 760, of 700,000 1586, 971, 906,
// 1007, of 1,500,000 4919, 2724, 1953, 1986; of 2^21 one block has no room at all, 5871, 2544, 2702; 400 of 1,000,000 2754, 1310, 982, 923.
constexpr size_t DRAW_SMEM = block_smem(MANY_PER_SM);

size_t verify_smem(int64_t cols, int blocks)
{
    return sizeof(Shared) + 2 * sizeof(int64_t) * (((cols + PIECE - 1) / PIECE + blocks - 1) / blocks + 1);
}

}  // namespace

extern "C" {

int pdb_verify(pdb_tokens *t, const pdb_mat *target, const pdb_ids *draft_ids, int64_t n_drafts, const pdb_mat *draft,
               float scale, float draft_scale, const float *accept_u, const float *draw_u, int32_t *tokens, int32_t *accepted,
               float *logp, void *stream)
{
    ApiScope scope("pdb_verify", nullptr, nullptr, nullptr, nullptr, false);
    if (!t || n_drafts < 0) return PDB_EINVAL;
    int rc = check_mat(target);
    if (rc == PDB_OK && draft) rc = check_mat(draft);
    if (rc != PDB_OK) return rc;
    if (n_drafts > MAX_DRAFTS || target->cols > MAX_VOCAB) return PDB_ETOOBIG;
    if (target->rows % (n_drafts + 1) != 0 || target->cols < 1 || !usable_scale(scale)) return PDB_EINVAL;
    const int64_t n = target->rows / (n_drafts + 1), drafts = n * n_drafts;
    if (n_drafts > 0) rc = check_ids(draft_ids, n, n_drafts);
    if (rc != PDB_OK) return rc;
    if (draft && (draft->rows != drafts || draft->cols != target->cols || draft->type != target->type ||
                  !usable_scale(draft_scale)))
        return PDB_EINVAL;
    const auto words = [](const void *p, int64_t k, bool optional) { return k == 0 || (p ? (uintptr_t)p % 4 == 0 : optional); };
    if (!words(accept_u, drafts, false) || !words(draw_u, n, false) || !words(tokens, n, false) || !words(accepted, n, true) ||
        !words(logp, n, true))
        return PDB_EINVAL;
    if (n == 0) return PDB_OK;
    if ((rc = check_device(t)) != PDB_OK) return rc;
    cudaStream_t s = (cudaStream_t)stream;
    TokensUse use{t, s};
    return with_type(target->type, [&](auto *a) {
        using T = std::remove_pointer_t<decltype(a)>;
        const int64_t nv = target->cols / Vec<T>::E + 1;
        const auto shaped = [&](int64_t clusters, int threads, int per_sm, bool draws) {
            Shape shape = {};
            shape.threads = threads;
            shape.blocks = cluster_of(clusters, nv, threads, [&](int blocks) { return (int64_t)t->sms * per_sm / blocks; });
            while (draws && verify_smem(target->cols, shape.blocks) > DRAW_SMEM && shape.blocks < MAX_CLUSTER) shape.blocks *= 2;
            shape.clusters = clusters;
            shape.smem = draws ? verify_smem(target->cols, shape.blocks) : 0;
            return shape;
        };
        Verify<T> v = {};
        v.target = (const T *)target->data, v.t_stride = stride_of(target);
        if (draft) v.draft = (const T *)draft->data, v.d_stride = stride_of(draft);
        v.cols = (int)target->cols, v.D = (int)n_drafts, v.n = n;
        if (n_drafts > 0) v.ids = ids_of(draft_ids);
        v.scale = scale, v.draft_scale = draft_scale, v.accept_u = accept_u, v.draw_u = draw_u;
        v.out = {tokens, accepted, logp}, v.status = t->status;
        // the statistics of all rows at once where the SMs would not be busy with a position of each sequence: a launch more, fewer rounds
        const int64_t rows = target->rows + (draft ? drafts : 0);
        if (n_drafts > 0 && n * 2 <= t->sms && rows <= VERIFY_ROWS) {
            const Shape shape = shaped(rows, 512, 2, false);
            v.given = (const Given *)t->given;
            v.sure_rows = sure_rows(nv, shape.blocks, shape.threads);
            const int rc = launch_rows(k_verify_rows<T, 512>, shape, s, v, (Given *)t->given);
            if (rc != PDB_OK) return rc;
        }
        const bool few = n * MAX_CLUSTER <= t->sms;
        const Shape shape = few ? shaped(n, FEW_THREADS, 2, true) : shaped(n, MANY_THREADS, 8, true);
        if (!v.given) v.sure_rows = sure_rows(nv, shape.blocks, shape.threads);
        return few ? launch_rows(k_verify<T, FEW_THREADS>, shape, s, v) : launch_rows(k_verify<T, MANY_THREADS>, shape, s, v);
    });
}

}  // extern "C"
