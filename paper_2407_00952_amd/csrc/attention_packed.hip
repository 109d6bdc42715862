// Softmax attention over packed records of any lengths, forward and backward; head size 64 or 128, key/value heads shared by
// groups of query heads, all keys of the record or only those up to the query, of these all or the last `window`.
//
//   P = softmax(scale q k^T), o = P v, lse = log of the row's sum of exponentials
//   dv = P^T do, dP = do v^T, dS = P (dP - delta), delta = rowsum(do o), dq = scale dS k, dk = scale dS^T q
//
// bf16 MFMA with fp32 sums, softmax arithmetic in fp32.  P is rounded to bf16 before P v and P^T do, dS before dS k and dS^T q: that is what
// the MFMA takes, fp32 operands have a sixteenth of its rate and the tensors are bf16 themselves.  Scores, the softmax's maximum and sum,
// lse, delta and every accumulator are fp32; the row's sum is that of the unrounded P.  Against 64 bits the results of a step together are
// off by 2.4e-3 of their 2-norm, by 1.7e-3 if nothing but the results is rounded; o alone by 1.7e-3 and 1.6e-3.
// The backward forms P again from lse, once in the kernel that owns queries (dq)
// and once in the one that owns keys (dk, dv; its sums run over the query heads of a group as well), so no sum needs atomics
// and results are bit-reproducible.  4 wavefronts a block, each owning 32 rows (queries or keys) against tiles of 64 of the other
// side, staged in LDS by asynchronous copies, double buffered.  A lane owns one of the wave's rows, which makes the softmax
// statistics per-lane scalars and lets the probabilities feed the next MFMA from registers; operands needed along the token axis come
// from the same row-major tiles through the LDS transpose read.
//
// Which tile of 128 rows a block works on is found from seq_start on the device: T rows divided into records have at most
// T / 128 + n_seq tiles (ceil(n / 128) <= n / 128 + 1), so that many tiles are launched whatever the division and the host needs to
// know no lengths.
// Rows of a tile past the end of its record are copies of its last row, so that nothing outside a record is read.
#include "../../include/slora.h"
#include "common.h"
#include "gemm_copy.h"

namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr int BQ = 128;                  // rows of a block
constexpr float kNoMax = -3.0e38f;       // start of a running maximum: finite, so that a row that has seen no key stays 0
constexpr float kFarMax = 67108864.0f;   // 2^26: from here on scores are rounded before a maximum is taken from them

typedef short v4s __attribute__((ext_vector_type(4)));

#define AP_WAIT_VM0() __builtin_amdgcn_s_waitcnt(0x0F70)

struct PackedArgs {
    const bf16 *q, *k, *v; long long ldq, ldk, ldv;
    const int *start; int n_seq, T, H, Hk;
    int causal, window; float scale;
    int slots;                           // tiles in the grid: T / 128 + n_seq
    int by_level;                        // how up to 64 records number them (find_tile)
};

// A probability that is formed from the stored lse: its exponent is off by the rounding of lse, by as much as 2^-21.7 |lse|, so it
// could be anything above 1 where lse is large.  (The bound is the exponential's own output modifier: no instruction.)
__device__ __forceinline__ float prob(float exponent) { return __builtin_amdgcn_fmed3f(__builtin_amdgcn_exp2f(exponent), 0.f, 1.f); }

__device__ __forceinline__ f32x16 zero16()
{
    f32x16 z;
#pragma unroll
    for (int e = 0; e < 16; ++e) z[e] = 0.f;
    return z;
}

template <int D> struct Dim {
    static constexpr int RB = 2 * D;                     // bytes of a row
    static constexpr int TILE = 64 * RB;                 // a tile of 64 rows
    static constexpr int KS = D / 16, DT = D / 32;       // k-steps over the head, 32-wide pieces of it
    static constexpr int LPR = RB / 16;                  // lanes that copy a row
    static constexpr int RPP = 64 / LPR;                 // rows of a 1 KB piece
    static constexpr int PITCH = RB + 16;                // a staged output row
};

// XOR mask of a tile row for the 16-byte chunks of its LDS row: chunk c of row r lies at r * RB + ((c ^ swizzle(r)) << 4).  LDS serves 256
// bytes a cycle (64 banks): 16 lanes of a row-major read, which are 16 rows and one chunk, or 32 lanes of a transpose read, which are 4
// rows and 4 neighbouring chunks.  With rows of 128 bytes two rows cover the banks, so the parity of the row is part of the place; with
// rows of 256 the mask has to tell all 16 rows apart, and its upper two bits any 4 neighbouring ones.  (Masks of three bits made two of five
// LDS cycles conflicts.)
template <int D>
__device__ __forceinline__ int swizzle(int row)
{
    const int b0 = row & 1, b1 = (row >> 1) & 1, b2 = (row >> 2) & 1, b3 = (row >> 3) & 1;
    return D == 64 ? (b1 << 2 | (b0 ^ b3) << 1 | b2) : ((b1 ^ b3) << 3 | b0 << 2 | b1 << 1 | b2);
}

// Asynchronous copy of rows 0 .. 63 (those past `rows` - 1 as copies of that one) into a swizzled row-major LDS tile
template <int D>
__device__ __forceinline__ void tile_copy(unsigned char *dst, const bf16 *src, unsigned ldb, int rows, int wave, int lane)
{
    typedef Dim<D> K;
    const int lrow = lane / K::LPR, lch = lane % K::LPR;
#pragma unroll
    for (int p = 0; p < D / 32; ++p) {
        const int piece = wave * (D / 32) + p, r = piece * K::RPP + lrow;
        const unsigned off = (unsigned)min(r, rows - 1) * ldb + (unsigned)((lch ^ swizzle<D>(r)) << 4);
        glds_soff(src, off, lds_addr(dst + piece * 1024));
    }
}

// One wave's copy of 32 rows (those past `rows` - 1 as copies of that one) into a piece of a tile of its own.  A wave's fragments read
// straight from memory are 64 places of 32 bytes to an instruction: the prologue of the dq kernel, four tensors, took 10700 of the 28000
// cycles that a block of short records lives.
template <int D>
__device__ __forceinline__ void rows32_copy(unsigned char *dst, const bf16 *src, unsigned ldb, int rows, int lane)
{
    typedef Dim<D> K;
    const int lrow = lane / K::LPR, lch = lane % K::LPR;
#pragma unroll
    for (int p = 0; p < D / 16; ++p) {
        const int r = p * K::RPP + lrow;
        const unsigned off = (unsigned)min(r, rows - 1) * ldb + (unsigned)((lch ^ swizzle<D>(r)) << 4);
        glds_soff(src, off, lds_addr(dst + p * 1024));
    }
}
#define AP_LANDED() do { AP_WAIT_VM0(); asm volatile("" ::: "memory"); } while (0)
#define AP_READ_OUT() asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory")

// The lane's byte offsets of both kinds of MFMA operand inside a 32-row piece of a tile.  Row-major: row lane % 32, columns of k-step ks.
// Transposed: column 32 dt + lane % 32 at rows 16 h + {0, 8} + 4 (lane / 32) + 0 .. 3, two reads of 4 rows.  One offset of each kind is
// held, that of ks = 0 and of dt = 0 and the first 4 rows: ks, dt and the rows 8 further on are bits of the chunk or of its mask, which an
// exclusive or sets.
template <int D> struct Frags { unsigned rm, tr; };
template <int D>
__device__ __forceinline__ void frag_offsets(int lane, Frags<D> &f)
{
    typedef Dim<D> K;
    const int r32 = lane & 31, g = lane >> 5, q = lane & 3, e = (lane >> 2) & 3, half = (lane >> 4) & 1;
    f.rm = r32 * K::RB + ((g ^ swizzle<D>(r32)) << 4);
    const int row = 4 * g + e;
    f.tr = row * K::RB + (((2 * half + (q >> 1)) ^ swizzle<D>(row)) << 4) + (q & 1) * 8;
}
template <int D>
__device__ __forceinline__ bf16x8 read_rm(const unsigned char *t, const Frags<D> &f, int ks)
{
    return *(const bf16x8 *)(t + (f.rm ^ (unsigned)(ks << 5)));
}
template <int D>
__device__ __forceinline__ bf16x8 read_tr(const unsigned char *t, const Frags<D> &f, int dt, int h)
{
    union { v4s s[2]; bf16x8 v; } u;
    const unsigned a0 = f.tr ^ (unsigned)(dt << 6), a1 = f.tr ^ (unsigned)((dt << 6) ^ (D == 64 ? 32 : 128));
    u.s[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s *)(t + a0 + 16 * h * Dim<D>::RB));
    u.s[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s *)(t + a1 + (16 * h + 8) * Dim<D>::RB));
    return u.v;
}

// A wave's 32 rows x D columns, held as MFMA accumulators (a lane has 4 neighbouring columns of row lane % 32 per register group), leave
// through its staging area as whole lines; rows from `rows` on stay.  what: 0 the rounded value, 1 what rounding took.
template <int D>
__device__ __forceinline__ void store_rows32(unsigned char *stg, const f32x16 (&acc)[D / 32], float scale, int what, bf16 *dst,
                                             long long ld, int rows, int lane)
{
    typedef Dim<D> K;
    const int r32 = lane & 31, g = lane >> 5, orow = lane / K::LPR, och = lane % K::LPR;
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
        for (int e4 = 0; e4 < 4; ++e4) {
            bf16x4 w;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float v = acc[dt][4 * e4 + i] * scale;
                const bf16 hi = f2bf(v);
                w[i] = what ? f2bf(v - bf2f(hi)) : hi;
            }
            *(bf16x4 *)(stg + r32 * K::PITCH + (32 * dt + 8 * e4 + 4 * g) * 2) = w;
        }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    bf16x8 t[32 / K::RPP];
#pragma unroll
    for (int it = 0; it < 32 / K::RPP; ++it) t[it] = *(const bf16x8 *)(stg + (K::RPP * it + orow) * K::PITCH + och * 16);
#pragma unroll
    for (int it = 0; it < 32 / K::RPP; ++it)
        if (K::RPP * it + orow < rows) *(bf16x8 *)(dst + (K::RPP * it + orow) * ld + och * 8) = t[it];
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// Sum over the wave, of values that are not negative their maximum: in the lanes' own data paths, a shuffle through LDS takes ten times as long
template <bool MAX>
__device__ __forceinline__ int wave_total(int v)
{
#define AP_STEP(CTRL, ROWS) { const int o = __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xf, true); v = MAX ? max(v, o) : v + o; }
    AP_STEP(0x111, 0xf) AP_STEP(0x112, 0xf) AP_STEP(0x114, 0xf) AP_STEP(0x118, 0xf)      // 1, 2, 4, 8 lanes up in rows of 16
    AP_STEP(0x142, 0xa) AP_STEP(0x143, 0xc)              // lane 15 to the next row, lane 31 to the last two
#undef AP_STEP
    return __builtin_amdgcn_readlane(v, 63);
}

// The tile with number `slot`: its record's first row and length, and which of the record's `tiles` it is, counted from the one with
// the least work in a causal launch (level 0: the first queries, the last keys); false for a number that no record uses.
//
// Blocks start in the order of their numbers, and long ones that start last run on when the others are done.  Up to 64 records are numbered
// by falling work, a lane for each record's tiles.  Long records: by the tile's level over all records, f(l) = the tiles of level l or more,
// the level of tile i being the largest one with f > i.  Short records, whose tiles share keys in the caches if they run
// together: record by record, those of many tiles first, f(l) = the tiles of records that have l or more.  Long: 1024 tokens a record or more
// on average.  Both directions, by level / by record / in the records' order, us:
//   7 records of 2341 on average, 32 heads of 128 on 8: 2085 / 2247 / 2450      64 of 257, 16 heads of 64: 169 / 161 / 166
//   16 of 1928: 16 heads of 64: 828 / 815 / 816, 32 of 128 on 8: 2953 / 2993 / 3098
//   16 of 957: 245 / 262 / 284, 934 / 952 / 1008; 4 of 1578: 159 / 164 / 158, 482 / 492 / 496; 48 of 874: 669 / 646 / 650, 2270 / 2252 / 2305
// More than 64 records are numbered one after the other, the tiles of record i from seq_start[i] / 128 + i on, which leaves each
// of them enough (records of 16 to 512 tokens, 16 heads of 64: 64 of them 148 us, 65 159, 128 355, 256 665).
// seq_start is the caller's data: whatever it holds, the rows lie within 0..T.
__device__ __forceinline__ bool find_tile(const PackedArgs &a, int slot, int lane, int &s0, int &n, int &level, int &tiles)
{
    int i, b, e;
    if (a.n_seq <= 64) {
        const int at = min(lane, a.n_seq - 1);
        b = min(max(a.start[at], 0), a.T);
        e = min(max(a.start[at + 1], b), a.T);
        const int nt = lane < a.n_seq ? (e - b + BQ - 1) / BQ : 0;
        int lo = 0, hi = wave_total<true>(nt) + 1, above = 0;                            // f(lo) > slot (if at all) >= f(hi) = above
        bool some = false;
        while (lo < hi) {
            const int mid = (lo + hi) >> 1;
            const int f = wave_total<false>(a.by_level ? max(nt - mid, 0) : nt >= mid ? nt : 0);
            if (f > slot) {
                some = true;
                if (lo == mid) break;
                lo = mid;
            } else {
                above = f;
                hi = mid;
            }
        }
        if (!some) return false;
        const bool of = a.by_level ? nt > lo : nt == lo;
        const int rank = __popcll(__ballot(of) & ((1ull << lane) - 1));
        const int mine = slot - above - (a.by_level ? rank : rank * lo);                 // (by record: which of its tiles)
        i = __ffsll((unsigned long long)__ballot(of && mine >= 0 && mine < (a.by_level ? 1 : lo))) - 1;
        if (i < 0) return false;
        b = __builtin_amdgcn_readlane(b, i);
        e = __builtin_amdgcn_readlane(e, i);
        level = __builtin_amdgcn_readfirstlane(a.by_level ? lo : lo - 1 - __builtin_amdgcn_readlane(mine, i));
    } else {
        int lo = 0, hi = a.n_seq;                        // how many records start at or before the slot: 64 probes a step
        while (lo < hi) {
            const int step = (hi - lo + 63) >> 6, at = lo + lane * step;
            const int s = min(max(a.start[min(at, a.n_seq)], 0), a.T);
            const int c = __popcll(__ballot(at < hi && (s >> 7) + at <= slot));
            if (c == 0) break;
            hi = min(hi, lo + c * step);
            lo = lo + (c - 1) * step + 1;
        }
        if (lo == 0) return false;
        i = lo - 1;
        b = min(max(a.start[i], 0), a.T);
        e = min(max(a.start[i + 1], b), a.T);
        level = __builtin_amdgcn_readfirstlane((e - b + BQ - 1) / BQ - 1 - (slot - (b >> 7) - i));
    }
    s0 = __builtin_amdgcn_readfirstlane(b);
    n = __builtin_amdgcn_readfirstlane(e - b);
    tiles = (n + BQ - 1) / BQ;
    return level >= 0 && level < tiles;
}

// Block -> (tile, key/value head, one of `w` blocks of that pair).  Workgroups go to the 8 XCDs round-robin; a key/value head keeps to one
// XCD, whose L2 then holds its keys and values, as far as the heads divide by 8; the tiles of the heads left over are dealt to all.
// On an XCD the long tiles of all its heads come first.
struct BlockPlan { int whole, rest, per; };              // heads of an XCD, heads left over, blocks of an XCD
__host__ __device__ inline BlockPlan block_plan(int slots, int heads, int w)
{
    BlockPlan p;
    p.whole = heads / 8;
    p.rest = heads % 8;
    p.per = p.whole * slots * w + (p.rest * slots * w + 7) / 8;
    return p;
}
__device__ __forceinline__ bool map_block(const PackedArgs &a, int w, int &slot, int &kvh, int &sub)
{
    const BlockPlan p = block_plan(a.slots, a.Hk, w);
    const int xcd = blockIdx.x & 7, i = blockIdx.x >> 3, own = p.whole * a.slots * w;
    if (i < own) {
        slot = i / (p.whole * w);
        const int k = i % (p.whole * w);
        kvh = xcd + 8 * (k / w);
        sub = k % w;
        return true;
    }
    const int j = (i - own) * 8 + xcd;
    if (j >= p.rest * a.slots * w) return false;
    slot = j / (p.rest * w);
    const int k = j % (p.rest * w);
    kvh = 8 * p.whole + k / w;
    sub = k % w;
    return true;
}

// ---- forward ------------------------------------------------------------------------------------
// Bound by the vector work at heads of 64: by counters, one record of 16384 tokens and 16 heads, a SIMD has 1049 cycles for 64 keys of a
// wave, its vector unit works in 845 of them (81 %), its matrix unit in 512 (49 %), and 8 % of a CU's time there is no block left.  The clock is
// 1.8 GHz meanwhile.  At heads of 128, 7 records on 32 heads, it is the alternation: matrix unit 45 %, vector unit 47 % of the cycles, by turns
// with two waves on a SIMD, CUs without a block 6 %.  (Copies put between the MFMAs spill; a raised wave priority around the MFMAs changes
// nothing.)  Four waves a SIMD at heads of 64: 604 -> 587 us for that record, 937 TFLOP/s.
template <int D>
__global__ __launch_bounds__(256, D == 64 ? 4 : 2) void packed_fwd_kernel(PackedArgs a, bf16 *__restrict__ o, bf16 *__restrict__ o_lo,
                                                                          long long ldo, float *__restrict__ lse)
{
    typedef Dim<D> K;
    __shared__ __attribute__((aligned(1024))) unsigned char KV[2][2 * K::TILE];
    const int tid = threadIdx.x, lane = tid & 63, r32 = lane & 31, g = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int G = a.H / a.Hk;
    int slot, kvh, sub, s0, n, tile, tiles;
    if (!map_block(a, G, slot, kvh, sub) || !find_tile(a, slot, lane, s0, n, tile, tiles)) return;
    const int head = kvh * G + sub, q0 = tile * BQ, qb = q0 + wave * 32, q = qb + r32;
    const bool active = qb < n;
    const int last = a.causal ? min(n, q0 + BQ) : n;     // keys of the block: from `first` (a tile's start) to last - 1
    const int first = a.window ? max(0, q0 - a.window + 1) >> 6 : 0;
    const int nt = ((last + 63) >> 6) - first;
    const bf16 *kg = a.k + (s0 + first * 64) * a.ldk + kvh * D, *vg = a.v + (s0 + first * 64) * a.ldv + kvh * D;
    const unsigned kb = (unsigned)a.ldk * 2u, vb = (unsigned)a.ldv * 2u;
    Frags<D> fr;
    frag_offsets<D>(lane, fr);

    tile_copy<D>(KV[0], kg, kb, n - first * 64, wave, lane);
    tile_copy<D>(KV[0] + K::TILE, vg, vb, n - first * 64, wave, lane);
    bf16x8 qf[K::KS];
    if (active) {                                        // the wave's queries, by way of the second buffer
        unsigned char *own = KV[1] + wave * 32 * K::RB;
        rows32_copy<D>(own, a.q + (s0 + qb) * a.ldq + head * D, (unsigned)a.ldq * 2u, n - qb, lane);
        AP_LANDED();
#pragma unroll
        for (int ks = 0; ks < K::KS; ++ks) qf[ks] = read_rm<D>(own, fr, ks);
        AP_READ_OUT();
    }
    f32x16 oacc[K::DT];
#pragma unroll
    for (int dt = 0; dt < K::DT; ++dt) oacc[dt] = zero16();
    float m = kNoMax, lsum = 0.f;
    bool far = false;                                    // (wave-uniform) some row's maximum is beyond kFarMax
    const float c = a.scale * kLog2e;
    // the keys a query sees: from lo_k to hi_k
    const int hi_k = a.causal ? min(q, n - 1) : n - 1, lo_k = a.window ? q - a.window + 1 : 0;

    for (int j = 0; j < nt; ++j) {
        AP_WAIT_VM0();
        __syncthreads();                                 // tile j has landed and nobody reads the other buffer any more
        const int k0 = (first + j) * 64;
        if (j + 1 < nt) {
            tile_copy<D>(KV[(j + 1) & 1], kg + (j + 1) * 64 * a.ldk, kb, n - k0 - 64, wave, lane);
            tile_copy<D>(KV[(j + 1) & 1] + K::TILE, vg + (j + 1) * 64 * a.ldv, vb, n - k0 - 64, wave, lane);
        }
        // (wave-uniform) nothing of the tile is visible to these 32 queries
        if (!active || (a.causal && k0 > qb + 31) || (a.window && k0 + 63 < qb - a.window + 1)) continue;
        const unsigned char *kt = KV[j & 1], *vt = kt + K::TILE;
        // all operand reads of a product go out before its first MFMA (left inline, every one is waited for in turn)
        bf16x8 kf[2][K::KS];
#pragma unroll
        for (int ks = 0; ks < K::KS; ++ks)
#pragma unroll
            for (int mt = 0; mt < 2; ++mt) kf[mt][ks] = read_rm<D>(kt + mt * 32 * K::RB, fr, ks);
        __builtin_amdgcn_sched_barrier(0);
        f32x16 sacc[2] = {zero16(), zero16()};
#pragma unroll
        for (int ks = 0; ks < K::KS; ++ks)
#pragma unroll
            for (int mt = 0; mt < 2; ++mt)
                sacc[mt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[mt][ks], qf[ks], sacc[mt], 0, 0, 0);
        if (k0 + 63 >= n || (a.causal && k0 + 63 > qb) || (a.window && k0 < qb + 31 - a.window + 1)) {
#pragma unroll
            for (int mt = 0; mt < 2; ++mt)
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int key = k0 + 32 * mt + 8 * (e >> 2) + 4 * g + (e & 3);
                    if (key > hi_k || key < lo_k) sacc[mt][e] = -INFINITY;
                }
        }
        float tmax = sacc[0][0];
#pragma unroll
        for (int mt = 0; mt < 2; ++mt)
#pragma unroll
            for (int e = 0; e < 16; ++e) tmax = fmaxf(tmax, sacc[mt][e]);
        tmax = fmaxf(tmax, __shfl_xor(tmax, 32, 64)) * c;
        // the maximum is only raised when a tile exceeds it by more than 8 (in log2 units): p <= 2^8 meanwhile
        if (__builtin_amdgcn_ballot_w64(tmax > m + 8.0f) != 0) {
            const float m_new = fmaxf(m, tmax), alpha = __builtin_amdgcn_exp2f(m - m_new);
            m = m_new;
            lsum *= alpha;
#pragma unroll
            for (int dt = 0; dt < K::DT; ++dt)
#pragma unroll
                for (int e = 0; e < 16; ++e) oacc[dt][e] *= alpha;
            far = __builtin_amdgcn_ballot_w64(fabsf(m) > kFarMax && m > kNoMax) != 0;
        }
        // s c - m subtracts the maximum, a rounded product, from an exact one: all exponents of a row are off by the same rounding, which
        // the division by their sum takes out again.  It is half a step of m: at maxima of 2^26 up to 4, at 2^31 enough for infinities.
        // So large scores are multiplied first and rounded as the maximum was.
        float cs = c;
        if (far) {
#pragma unroll
            for (int mt = 0; mt < 2; ++mt)
#pragma unroll
                for (int e = 0; e < 16; ++e) sacc[mt][e] *= c;
            cs = 1.0f;
        }
#pragma unroll
        for (int mt = 0; mt < 2; ++mt) {
            bf16x8 vf[2][K::DT];                         // this half's V fragments, under way during its exponentials
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int dt = 0; dt < K::DT; ++dt) vf[h][dt] = read_tr<D>(vt + mt * 32 * K::RB, fr, dt, h);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                // (the row's sum is that of the probabilities before they are rounded for the product: lse is exact to fp32)
                bf16x8 pb;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float p = __builtin_amdgcn_exp2f(fmaf(sacc[mt][8 * h + i], cs, -m));
                    lsum += p;
                    pb[i] = f2bf(p);
                }
#pragma unroll
                for (int dt = 0; dt < K::DT; ++dt)
                    oacc[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[h][dt], pb, oacc[dt], 0, 0, 0);
            }
        }
    }
    __syncthreads();                                     // the tiles' memory becomes the staging area
    if (!active) return;
    unsigned char *stg = &KV[0][0] + wave * 32 * K::PITCH;
    const float l = lsum + __shfl_xor(lsum, 32, 64), inv = 1.0f / l;
    bf16 *od = o + (s0 + qb) * ldo + head * D;
    store_rows32<D>(stg, oacc, inv, 0, od, ldo, n - qb, lane);
    if (o_lo) store_rows32<D>(stg, oacc, inv, 1, o_lo + (s0 + qb) * ldo + head * D, ldo, n - qb, lane);
    if (g == 0 && q < n) lse[(size_t)head * a.T + s0 + q] = (m + __builtin_amdgcn_logf(l)) * kLn2;
}

// ---- dq (and delta, which the dk/dv kernel reads) -------------------------------------------------
// 7 records of 16384 tokens, 32 heads of 128 on 8: 0.68 ms (three products: 1020 TFLOP/s), the matrix unit in 51 % of the cycles, the
// vector unit in 40 %.  64 records of 16461 tokens, 16 heads of 64: 65 us with fragments read straight from memory, 54 by way of LDS, 51 with
// operand reads right before their MFMA, which needs 128 registers: four waves a SIMD.
template <int D>
__global__ __launch_bounds__(256, D == 64 ? 4 : 2) void packed_dq_kernel(PackedArgs a, const bf16 *__restrict__ o, const bf16 *__restrict__ o_lo,
                                                           long long ldo, const float *__restrict__ lse, const bf16 *__restrict__ dout,
                                                           long long lddo, bf16 *__restrict__ dq, long long lddq,
                                                           float *__restrict__ delta)
{
    typedef Dim<D> K;
    __shared__ __attribute__((aligned(1024))) unsigned char KV[2][2 * K::TILE];
    const int tid = threadIdx.x, lane = tid & 63, r32 = lane & 31, g = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int G = a.H / a.Hk;
    int slot, kvh, sub, s0, n, tile, tiles;
    if (!map_block(a, G, slot, kvh, sub) || !find_tile(a, slot, lane, s0, n, tile, tiles)) return;
    const int head = kvh * G + sub, q0 = tile * BQ, qb = q0 + wave * 32, q = qb + r32;
    const bool active = qb < n;
    const int last = a.causal ? min(n, q0 + BQ) : n;
    const int first = a.window ? max(0, q0 - a.window + 1) >> 6 : 0;
    const int nt = ((last + 63) >> 6) - first;
    const bf16 *kg = a.k + (s0 + first * 64) * a.ldk + kvh * D, *vg = a.v + (s0 + first * 64) * a.ldv + kvh * D;
    const unsigned kb = (unsigned)a.ldk * 2u, vb = (unsigned)a.ldv * 2u;
    Frags<D> fr;
    frag_offsets<D>(lane, fr);

    tile_copy<D>(KV[0], kg, kb, n - first * 64, wave, lane);
    tile_copy<D>(KV[0] + K::TILE, vg, vb, n - first * 64, wave, lane);
    bf16x8 qf[K::KS], dof[K::KS];
    const int row = s0 + min(q, n - 1);
    float dl = 0.f;
    if (active) {
        // the wave's queries and rows of do, by way of the second buffer, one after the other; o beside them in whole lines, LPR lanes a row
        unsigned char *own = KV[1] + wave * 32 * K::RB;
        constexpr int PASSES = 32 / K::RPP;
        const int lrow = lane / K::LPR, lch = lane % K::LPR;
        rows32_copy<D>(own, a.q + (s0 + qb) * a.ldq + head * D, (unsigned)a.ldq * 2u, n - qb, lane);
        AP_LANDED();
#pragma unroll
        for (int ks = 0; ks < K::KS; ++ks) qf[ks] = read_rm<D>(own, fr, ks);
        AP_READ_OUT();
        rows32_copy<D>(own, dout + (s0 + qb) * lddo + head * D, (unsigned)lddo * 2u, n - qb, lane);
        bf16x8 ov[PASSES], lv[PASSES];
#pragma unroll
        for (int p = 0; p < PASSES; ++p) {
            const long long at = (s0 + qb + min(K::RPP * p + lrow, n - qb - 1)) * ldo + head * D + lch * 8;
            ov[p] = *(const bf16x8 *)(o + at);
            if (o_lo) lv[p] = *(const bf16x8 *)(o_lo + at);
        }
        AP_LANDED();
#pragma unroll
        for (int p = 0; p < PASSES; ++p) {
            const int r = K::RPP * p + lrow;
            const bf16x8 dv = *(const bf16x8 *)(own + r * K::RB + ((lch ^ swizzle<D>(r)) << 4));
            float t = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) t = fmaf(bf2f(dv[i]), bf2f(ov[p][i]), t);
            if (o_lo) {
#pragma unroll
                for (int i = 0; i < 8; ++i) t = fmaf(bf2f(dv[i]), bf2f(lv[p][i]), t);
            }
#pragma unroll
            for (int k = 1; k < K::LPR; k <<= 1) t += __shfl_xor(t, k, 64);
            const float v = __shfl(t, (r32 % K::RPP) * K::LPR, 64);
            if (r32 / K::RPP == p) dl = v;
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int ks = 0; ks < K::KS; ++ks) dof[ks] = read_rm<D>(own, fr, ks);
        AP_READ_OUT();
    }
    const float lse_q = lse[(size_t)head * a.T + row] * kLog2e;
    if (g == 0 && q < n) delta[(size_t)head * a.T + row] = dl;
    f32x16 acc[K::DT];
#pragma unroll
    for (int dt = 0; dt < K::DT; ++dt) acc[dt] = zero16();
    const float c = a.scale * kLog2e;
    const int hi_k = a.causal ? min(q, n - 1) : n - 1, lo_k = a.window ? q - a.window + 1 : 0;

    for (int j = 0; j < nt; ++j) {
        AP_WAIT_VM0();
        __syncthreads();
        const int k0 = (first + j) * 64;
        if (j + 1 < nt) {
            tile_copy<D>(KV[(j + 1) & 1], kg + (j + 1) * 64 * a.ldk, kb, n - k0 - 64, wave, lane);
            tile_copy<D>(KV[(j + 1) & 1] + K::TILE, vg + (j + 1) * 64 * a.ldv, vb, n - k0 - 64, wave, lane);
        }
        if (!active) continue;
#pragma clang loop unroll(disable)
        for (int mt = 0; mt < 2; ++mt) {
            const int kk = k0 + 32 * mt;
            if (kk >= n || (a.causal && kk > qb + 31) || (a.window && kk + 31 < qb - a.window + 1)) continue;
            const unsigned char *kt = KV[j & 1] + mt * 32 * K::RB, *vt = kt + K::TILE;
            // -delta as the addend of the dP product: dP - delta leaves the matrix cores ready (opaque: else it is written
            // out ahead of the loop and held)
            float nd = -dl;
            asm volatile("" : "+v"(nd));
            f32x16 sacc = zero16(), dpacc;
#pragma unroll
            for (int e = 0; e < 16; ++e) dpacc[e] = nd;
#pragma unroll
            for (int ks = 0; ks < K::KS; ++ks) {
                sacc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(read_rm<D>(kt, fr, ks), qf[ks], sacc, 0, 0, 0);
                dpacc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(read_rm<D>(vt, fr, ks), dof[ks], dpacc, 0, 0, 0);
            }
            if (kk + 31 >= n || (a.causal && kk + 31 > qb) || (a.window && kk < qb + 31 - a.window + 1)) {
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int key = kk + 8 * (e >> 2) + 4 * g + (e & 3);
                    if (key > hi_k || key < lo_k) sacc[e] = -INFINITY;
                }
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                bf16x8 ds;
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    ds[i] = f2bf(prob(fmaf(sacc[8 * h + i], c, -lse_q)) * dpacc[8 * h + i]);
#pragma unroll
                for (int dt = 0; dt < K::DT; ++dt)
                    acc[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(read_tr<D>(kt, fr, dt, h), ds, acc[dt], 0, 0, 0);
            }
        }
    }
    __syncthreads();
    if (active)
        store_rows32<D>(&KV[0][0] + wave * 32 * K::PITCH, acc, a.scale, 0, dq + (s0 + qb) * lddq + head * D, lddq, n - qb, lane);
}

// ---- dk, dv ----------------------------------------------------------------------------------------
// A block owns 128 keys of one key/value head and walks, head after head, the query tiles that see them.  parts > 1: the heads of a
// group are dealt over so many blocks, whose sums go to fp32 memory (part [2][parts][T][Hk][D]) and are added in order afterwards.
// With heads of 128 the accumulators and the wave's K and V fill 192 of the 256 registers that two waves a SIMD have each; operand reads
// stand right before their MFMA and nothing per lane is held that can be formed anew.  (One wave a SIMD with 512 registers, the halves of
// a tile interleaved by hand, takes 1.19 ms where this took 1.01 then and takes 0.94 now: four products, 990 TFLOP/s, the matrix unit in
// 48 % of the cycles, the vector unit in 33 %; registers that spill cost most, since every reload waits for the copies in flight: 1.45 ms.)
template <int D>
__global__ __launch_bounds__(256, 2) void packed_dkv_kernel(PackedArgs a, const float *__restrict__ lse, const float *__restrict__ delta,
                                                            const bf16 *__restrict__ dout, long long lddo, bf16 *__restrict__ dk,
                                                            long long lddk, bf16 *__restrict__ dv, long long lddv, int parts,
                                                            float *__restrict__ part)
{
    typedef Dim<D> K;
    __shared__ __attribute__((aligned(1024))) unsigned char QD[2][2 * K::TILE];
    __shared__ __align__(16) float st[2][128];           // lse (log2 units) | -delta of a tile's 64 queries
    const int tid = threadIdx.x, lane = tid & 63, r32 = lane & 31, g = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    int slot, kvh, pt, s0, n, level, tiles;
    if (!map_block(a, parts, slot, kvh, pt) || !find_tile(a, slot, lane, s0, n, level, tiles)) return;
    const int tile = tiles - 1 - level;                  // (the first keys are seen by the most queries)
    const int G = a.H / a.Hk, per = (G + parts - 1) / parts;
    const int h0 = kvh * G + pt * per, h1 = kvh * G + min(G, pt * per + per);      // query heads of this block (none: zeros)
    const int kt0 = tile * BQ, kb = kt0 + wave * 32, key = kb + r32;
    const bool active = kb < n;
    const int q_first = a.causal ? kt0 : 0;
    const int q_last = a.window ? min(n, kt0 + BQ - 1 + a.window) : n;
    const int ntile = (q_last - q_first + 63) >> 6;
    const int total_t = max(h1 - h0, 0) * ntile;
    const unsigned qbts = (unsigned)a.ldq * 2u, dbts = (unsigned)lddo * 2u;

    // per-query statistics travel through a register, so that their LDS store stands behind the work on the current tile
    float stat = 0.f;
    auto issue = [&](int buf, int h, int j) {
        const int q0 = q_first + j * 64;
        tile_copy<D>(QD[buf], a.q + (s0 + q0) * a.ldq + h * D, qbts, n - q0, wave, lane);
        tile_copy<D>(QD[buf] + K::TILE, dout + (s0 + q0) * lddo + h * D, dbts, n - q0, wave, lane);
        if (tid < 128) {
            const int qq = q0 + (tid & 63);
            const float *src = tid < 64 ? lse : delta;
            stat = src[(size_t)h * a.T + s0 + min(qq, n - 1)];
            if (qq >= n) stat = tid < 64 ? INFINITY : 0.f;     // a query past the end: p = 2^-inf
        }
    };
    auto put_stat = [&](int buf) {
        if (tid < 128) st[buf][tid] = tid < 64 ? stat * kLog2e : -stat;
    };
    if (total_t > 0) issue(0, h0, 0);
    bf16x8 kf[K::KS], vf[K::KS];
    if (active) {                                        // the wave's keys and values, by way of the second buffer
        Frags<D> fr;
        frag_offsets<D>(lane, fr);
        unsigned char *own = QD[1] + wave * 32 * K::RB;
        rows32_copy<D>(own, a.k + (s0 + kb) * a.ldk + kvh * D, (unsigned)a.ldk * 2u, n - kb, lane);
        AP_LANDED();
#pragma unroll
        for (int ks = 0; ks < K::KS; ++ks) kf[ks] = read_rm<D>(own, fr, ks);
        AP_READ_OUT();
        rows32_copy<D>(own, a.v + (s0 + kb) * a.ldv + kvh * D, (unsigned)a.ldv * 2u, n - kb, lane);
        AP_LANDED();
#pragma unroll
        for (int ks = 0; ks < K::KS; ++ks) vf[ks] = read_rm<D>(own, fr, ks);
        AP_READ_OUT();
    }
    f32x16 dkacc[K::DT], dvacc[K::DT];
#pragma unroll
    for (int dt = 0; dt < K::DT; ++dt) dkacc[dt] = dvacc[dt] = zero16();
    const float c = a.scale * kLog2e;
    if (total_t > 0) put_stat(0);
    int h = h0, j = 0;                                   // head and query tile of step t
    for (int t = 0; t < total_t; ++t) {
        AP_WAIT_VM0();
        __syncthreads();
        const int q0 = q_first + j * 64;
        const bool wrap = j + 1 == ntile;
        const int nh = wrap ? h + 1 : h, nj = wrap ? 0 : j + 1;
        if (t + 1 < total_t) issue((t + 1) & 1, nh, nj);
#pragma clang loop unroll(disable)
        for (int hf = 0; hf < 2; ++hf) {
            const int qh = q0 + 32 * hf;
            if (!active || qh >= n || (a.causal && qh + 31 < kb) || (a.window && qh > kb + 31 + a.window - 1)) continue;
            // (formed anew for each half: two registers less, of which the loop has none to spare)
            int ln = threadIdx.x & 63;
            asm volatile("" : "+v"(ln));
            Frags<D> fr;
            frag_offsets<D>(ln, fr);
            const int g = ln >> 5, key = kb + (ln & 31);
            const unsigned char *qt = QD[t & 1] + hf * 32 * K::RB, *dt_ = qt + K::TILE;
            const float *sl = st[t & 1] + 32 * hf + 4 * g;
            f32x16 sacc = zero16(), dpacc;
#pragma unroll
            for (int e4 = 0; e4 < 4; ++e4) {
                const f32x4 dd = *(const f32x4 *)(sl + 64 + 8 * e4);
#pragma unroll
                for (int i = 0; i < 4; ++i) dpacc[4 * e4 + i] = dd[i];
            }
#pragma unroll
            for (int ks = 0; ks < K::KS; ++ks) {
                sacc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(read_rm<D>(qt, fr, ks), kf[ks], sacc, 0, 0, 0);
                dpacc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(read_rm<D>(dt_, fr, ks), vf[ks], dpacc, 0, 0, 0);
            }
            if ((a.causal && qh < kb + 31) || (a.window && qh + 31 - kb >= a.window)) {
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int qq = qh + 8 * (e >> 2) + 4 * g + (e & 3);
                    if ((a.causal && key > qq) || (a.window && qq - key >= a.window)) sacc[e] = -INFINITY;
                }
            }
#pragma unroll
            for (int hh = 0; hh < 2; ++hh) {
                bf16x8 pb, ds;
#pragma unroll
                for (int e4 = 0; e4 < 2; ++e4) {
                    const f32x4 ls = *(const f32x4 *)(sl + 8 * (2 * hh + e4));
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int e = 8 * hh + 4 * e4 + i;
                        const float p = prob(fmaf(sacc[e], c, -ls[i]));
                        pb[4 * e4 + i] = f2bf(p);
                        ds[4 * e4 + i] = f2bf(p * dpacc[e]);
                    }
                }
#pragma unroll
                for (int dt = 0; dt < K::DT; ++dt) {
                    dvacc[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(read_tr<D>(dt_, fr, dt, hh), pb, dvacc[dt], 0, 0, 0);
                    dkacc[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(read_tr<D>(qt, fr, dt, hh), ds, dkacc[dt], 0, 0, 0);
                }
            }
        }
        if (t + 1 < total_t) put_stat((t + 1) & 1);
        h = nh;
        j = nj;
    }
    __syncthreads();
    if (!active) return;
    if (parts > 1) {
        if (key >= n) return;
        float *p = part + (((size_t)pt * a.T + s0 + key) * a.Hk + kvh) * D + 4 * g;
        const size_t other = (size_t)parts * a.T * a.Hk * D;
#pragma unroll
        for (int dt = 0; dt < K::DT; ++dt)
#pragma unroll
            for (int e4 = 0; e4 < 4; ++e4) {
                f32x4 x, y;
#pragma unroll
                for (int i = 0; i < 4; ++i) { x[i] = dkacc[dt][4 * e4 + i]; y[i] = dvacc[dt][4 * e4 + i]; }
                *(f32x4 *)(p + 32 * dt + 8 * e4) = x;
                *(f32x4 *)(p + other + 32 * dt + 8 * e4) = y;
            }
        return;
    }
    unsigned char *stg = &QD[0][0] + wave * 32 * K::PITCH;
    store_rows32<D>(stg, dkacc, a.scale, 0, dk + (s0 + kb) * lddk + kvh * D, lddk, n - kb, lane);
    store_rows32<D>(stg, dvacc, 1.0f, 0, dv + (s0 + kb) * lddv + kvh * D, lddv, n - kb, lane);
}

// the parts' sums, in order; one thread for 4 columns.  Rows outside every record hold no sums and stay.
__global__ __launch_bounds__(256) void packed_dkv_reduce_kernel(PackedArgs a, int D, int parts, const float *__restrict__ part,
                                                                bf16 *__restrict__ dk, long long lddk, bf16 *__restrict__ dv,
                                                                long long lddv)
{
    const int width = a.Hk * D / 4;
    const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
    const int row = (int)(i / width), col = (int)(i % width) * 4;
    const int lo = min(max(a.start[0], 0), a.T), hi = min(a.start[a.n_seq], a.T);
    if (row < lo || row >= hi) return;
    const size_t step = (size_t)a.T * a.Hk * D;
    const float *p = part + (size_t)row * a.Hk * D + col;
    f32x4 x = *(const f32x4 *)p, y = *(const f32x4 *)(p + parts * step);
    for (int k = 1; k < parts; ++k) {
        x += *(const f32x4 *)(p + k * step);
        y += *(const f32x4 *)(p + (parts + k) * step);
    }
    bf16x4 u, w;
#pragma unroll
    for (int e = 0; e < 4; ++e) { u[e] = f2bf(x[e] * a.scale); w[e] = f2bf(y[e]); }
    *(bf16x4 *)(dk + row * lddk + col) = u;
    *(bf16x4 *)(dv + row * lddv + col) = w;
}

// Over how many blocks the query heads of a key/value head are dealt: with few key tiles one block each would leave most of the chip idle,
// and a causal record's first keys have the most work.  One block each / until there are 256 / 512 (as here) / 1024 blocks, both directions, us:
//   16 heads of 64 on 2: 2500 tokens 652 / 180 / 180 / 179, 4096 1046 / 377 / 278 / 278, 8192 2257 / 1268 / 835 / 683
//   32 heads of 128 on 8: 2500 578 / 391 / 308 / 309, 4096 1058 / 1059 / 744 / 640, 8192 2794 / 2760 / 2783 / 2240, 16384 8963 / 8964 / 9046 / 9161
// More parts take more scratch: 8 parts T Hk D bytes, written and read.
inline int dkv_parts(int T, int H, int Hk)
{
    const int G = H / Hk, blocks = ((T + BQ - 1) / BQ) * Hk;
    int parts = 1;
    while (parts < G && blocks * parts < 512) parts *= 2;
    return parts < G ? parts : G;
}

inline size_t al256(size_t v) { return (v + 255) & ~(size_t)255; }
inline bool aligned(const void *p, unsigned n) { return ((uintptr_t)p & (n - 1)) == 0; }
inline bool stride_ok(int64_t ld, int64_t width) { return ld >= width && ld % 8 == 0 && ld < (1 << 24); }
inline bool sizes_ok(int T, int H, int Hk, int D)
{
    return T >= 0 && T <= (1 << 24) && H > 0 && H <= 1024 && Hk > 0 && H % Hk == 0 && (D == 64 || D == 128);
}
// delta, and room for the parts' sums of T rows or fewer: dkv_parts falls with the rows, so the most that a number of parts needs is at the
// last row count that has it
inline size_t bwd_ws(int T, int H, int Hk, int D)
{
    const int G = H / Hk;
    size_t sums = 0;
    for (int parts = G; parts > 1; parts = (parts & (parts - 1)) ? 1 << (31 - __builtin_clz(parts)) : parts / 2) {
        int lo = 0, hi = T;                              // the last row count up to T with at least so many parts
        while (lo < hi) {
            const int mid = lo + (hi - lo + 1) / 2;
            if (dkv_parts(mid, H, Hk) >= parts) lo = mid;
            else hi = mid - 1;
        }
        const size_t n = 8 * (size_t)parts * lo * Hk * D;
        sums = sums < n ? n : sums;
    }
    return al256(4 * (size_t)H * (T < 1 ? 1 : T)) + al256(sums);
}

bool numbers_ok(int n_seq, int T, int H, int Hk, int D, float scale, int causal, int window)
{
    if (n_seq < 0 || n_seq > (1 << 24) || !sizes_ok(T, H, Hk, D)) return false;
    if (!(scale > 0.f) || !(scale <= 1e30f) || (causal & ~1) || window < 0 || (window && !causal)) return false;
    // a grid has fewer than 2^32 threads
    return ((int64_t)T / BQ + n_seq) * H < (1 << 24) - 64;
}

int check_common(int H, int Hk, int D, const void *q, int64_t ldq, const void *k, int64_t ldk, const void *v, int64_t ldv, const int *start)
{
    if (!q || !k || !v || !start || !aligned(q, 16) || !aligned(k, 16) || !aligned(v, 16) || !aligned(start, 4)) return SLORA_EINVAL;
    if (!stride_ok(ldq, (int64_t)H * D) || !stride_ok(ldk, (int64_t)Hk * D) || !stride_ok(ldv, (int64_t)Hk * D)) return SLORA_EINVAL;
    return SLORA_OK;
}

PackedArgs pack_args(int n_seq, int T, int H, int Hk, float scale, int causal, int window, const void *q, int64_t ldq, const void *k,
                     int64_t ldk, const void *v, int64_t ldv, const int *start)
{
    return {(const bf16 *)q, (const bf16 *)k, (const bf16 *)v, ldq, ldk, ldv, start, n_seq, T, H, Hk, causal,
            window >= T ? 0 : window, scale, T / BQ + n_seq, T / 1024 >= n_seq};
}

inline dim3 xcd_grid(const PackedArgs &a, int w) { return dim3((unsigned)block_plan(a.slots, a.Hk, w).per * 8u); }

}  // namespace

extern "C" {

int slora_attention_fwd(int32_t n_seq, int32_t T, int32_t n_head, int32_t n_kv_head, int32_t head_dim, float scale,
                        int32_t causal, int32_t window, const void *q, int64_t ldq, const void *k, int64_t ldk,
                        const void *v, int64_t ldv, const int32_t *seq_start, void *o, void *o_lo, int64_t ldo,
                        float *lse, void *stream)
{
    if (!numbers_ok(n_seq, T, n_head, n_kv_head, head_dim, scale, causal, window)) return SLORA_EINVAL;
    if (n_seq == 0 || T == 0) return SLORA_OK;           // (an empty tensor has no address)
    const int rc = check_common(n_head, n_kv_head, head_dim, q, ldq, k, ldk, v, ldv, seq_start);
    if (rc) return rc;
    if (!o || !lse || !aligned(o, 16) || !aligned(o_lo, 16) || !aligned(lse, 4) || !stride_ok(ldo, (int64_t)n_head * head_dim))
        return SLORA_EINVAL;
    const PackedArgs a = pack_args(n_seq, T, n_head, n_kv_head, scale, causal, window, q, ldq, k, ldk, v, ldv, seq_start);
    const hipStream_t st = (hipStream_t)stream;
    if (head_dim == 64)
        hipLaunchKernelGGL(packed_fwd_kernel<64>, xcd_grid(a, a.H / a.Hk), dim3(256), 0, st, a, (bf16 *)o, (bf16 *)o_lo, ldo, lse);
    else
        hipLaunchKernelGGL(packed_fwd_kernel<128>, xcd_grid(a, a.H / a.Hk), dim3(256), 0, st, a, (bf16 *)o, (bf16 *)o_lo, ldo, lse);
    SL_CHECK_LAUNCH("packed_fwd");
    return SLORA_OK;
}

size_t slora_attention_bwd_ws_bytes(int32_t T, int32_t n_head, int32_t n_kv_head, int32_t head_dim)
{
    return sizes_ok(T, n_head, n_kv_head, head_dim) ? bwd_ws(T, n_head, n_kv_head, head_dim) : 0;
}

int slora_attention_bwd(int32_t n_seq, int32_t T, int32_t n_head, int32_t n_kv_head, int32_t head_dim, float scale,
                        int32_t causal, int32_t window, const void *q, int64_t ldq, const void *k, int64_t ldk,
                        const void *v, int64_t ldv, const int32_t *seq_start, const void *o, const void *o_lo,
                        int64_t ldo, const float *lse, const void *dout, int64_t lddo, void *dq, int64_t lddq,
                        void *dk, int64_t lddk, void *dv, int64_t lddv, void *ws, size_t ws_bytes, void *stream)
{
    if (!numbers_ok(n_seq, T, n_head, n_kv_head, head_dim, scale, causal, window)) return SLORA_EINVAL;
    if (n_seq == 0 || T == 0) return SLORA_OK;           // (an empty tensor has no address)
    const int rc = check_common(n_head, n_kv_head, head_dim, q, ldq, k, ldk, v, ldv, seq_start);
    if (rc) return rc;
    const int64_t wq = (int64_t)n_head * head_dim, wk = (int64_t)n_kv_head * head_dim;
    if (!o || !lse || !dout || !dq || !dk || !dv || !ws) return SLORA_EINVAL;
    if (!aligned(o, 16) || !aligned(o_lo, 16) || !aligned(lse, 4) || !aligned(dout, 16) || !aligned(dq, 16) || !aligned(dk, 16) ||
        !aligned(dv, 16) || !aligned(ws, 256))
        return SLORA_EINVAL;
    if (!stride_ok(ldo, wq) || !stride_ok(lddo, wq) || !stride_ok(lddq, wq) || !stride_ok(lddk, wk) || !stride_ok(lddv, wk))
        return SLORA_EINVAL;
    if (ws_bytes < bwd_ws(T, n_head, n_kv_head, head_dim)) return SLORA_ENOSPC;
    const PackedArgs a = pack_args(n_seq, T, n_head, n_kv_head, scale, causal, window, q, ldq, k, ldk, v, ldv, seq_start);
    const hipStream_t st = (hipStream_t)stream;
    float *delta = (float *)ws, *part = (float *)((char *)ws + al256(4 * (size_t)n_head * T));
    const int parts = dkv_parts(T, n_head, n_kv_head);
    const dim3 gq = xcd_grid(a, a.H / a.Hk), gk = xcd_grid(a, parts);
#define AP_BWD(D)                                                                                                                    \
    hipLaunchKernelGGL(packed_dq_kernel<D>, gq, dim3(256), 0, st, a, (const bf16 *)o, (const bf16 *)o_lo, ldo, lse,                   \
                       (const bf16 *)dout, lddo, (bf16 *)dq, lddq, delta);                                                           \
    hipLaunchKernelGGL(packed_dkv_kernel<D>, gk, dim3(256), 0, st, a, lse, delta, (const bf16 *)dout, lddo, (bf16 *)dk, lddk,         \
                       (bf16 *)dv, lddv, parts, part);
    if (head_dim == 64) { AP_BWD(64) } else { AP_BWD(128) }
#undef AP_BWD
    SL_CHECK_LAUNCH("packed_bwd");
    if (parts > 1) {
        const long long threads = (long long)T * a.Hk * head_dim / 4;
        hipLaunchKernelGGL(packed_dkv_reduce_kernel, dim3((unsigned)((threads + 255) / 256)), dim3(256), 0, st, a, head_dim, parts, part,
                           (bf16 *)dk, lddk, (bf16 *)dv, lddv);
        SL_CHECK_LAUNCH("packed_dkv_reduce");
    }
    return SLORA_OK;
}

}  // extern "C"
