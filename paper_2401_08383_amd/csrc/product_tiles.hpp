// The experts' products in tiles, a workgroup of four wavefronts a tile (product_forward.hip, product_rows_gradient.hip,
// product_weight_gradient.hip, product_mx4_tiles.hip instantiate it).
//
// As in ffn_tiles.hpp, whose row tiles and whose map from workgroups to them are used: H x NT outputs in 16x16 accumulators in the accumulator
// half of the registers, operands by direct-to-LDS loads into a ring of stages, one workgroup barrier a stage.  What differs:
//   - an operand whose reduction lies across memory (the weights of the rows' gradient, both operands of the weights'
//     gradient) is staged as it comes, [reduction][row], and turned on the way from LDS to registers: ds_read_b64_tr_b16 gives a lane
//     four reduction elements of one row out of 4 x 16 elements of 16 lanes.  Two of them are an operand fetch.
//   - operands in 4 bits: a fetch of 16 bytes is a block of 32 elements instead of 8 bf16, a stage 256 reduction elements, and a
//     row's 8 scale bytes of a stage are staged with it.  A matrix instruction takes as long as the bf16 one.
//   - reductions of any length: what a stage has beyond the end is fetched from outside the buffer the loads are told of, and
//     such loads deliver zeros without asking memory.  Stages behind the last one are loaded the same way, so that every stage is
//     in the steady state, the first and the last ones too: one copy of the loop's body, and no branch in it.
#pragma once

#include "ffn_tiles.hpp"
#include "product.hpp"

namespace exf {

enum ProductKind {
    kForward,         // rows [.,K] and weights [N,K]: both along the reduction
    kRowsGradient,    // rows [.,K] along, weights [K,N] across
    kWeightGradient,  // both across
    kMx4,             // as kForward, in 4 bits with scales
};

constexpr int kProductWaves = 4;
typedef __attribute__((__vector_size__(4 * sizeof(__bf16)))) __bf16 bf16x4_t;

// One wavefront-wide direct-to-LDS load of 16 bytes a lane from buffer `rsrc` (a base and how far it reaches); STREAM: past the caches.
template <bool STREAM>
__device__ __forceinline__ void lds_buffer_16B(u32x4_v rsrc, uint32_t voff, uint32_t lds_addr)
{
#if defined(__HIP_DEVICE_COMPILE__)
    if constexpr (STREAM)
        asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, 0 offen nt lds\n" : : "v"(voff), "s"(rsrc), "s"(lds_addr) : "memory");
    else
        asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds\n" : : "v"(voff), "s"(rsrc), "s"(lds_addr) : "memory");
#else
    (void)rsrc; (void)voff; (void)lds_addr;
#endif
}
constexpr uint32_t kBufferReach = 0x80000000u;  // offsets from here on deliver zeros
static_assert(static_cast<uint64_t>(kTallestTile) * EXF_MAX_PRODUCT_WIDTH * 2 < kBufferReach, "all offsets of a tile lie below");

template <typename T>
__device__ __forceinline__ T lds_fetch(uint32_t addr)
{
#if defined(__HIP_DEVICE_COMPILE__)
    return *reinterpret_cast<const __attribute__((address_space(3))) T*>(addr);
#else
    return T{};
#endif
}

// ---------------------------------------------------------------------------- operands
// One operand of a tile: ROWS output rows (or columns) by 64 (4 bits: 256) reduction elements a stage, 128 bytes of each row.
//   along : row r at base + r * ld.  One load covers 8 rows: lane -> row lane/8 and the 16-byte piece (lane%8) ^ (row/2 % 8).
//   across: reduction element r at base + r * ld, the rows side by side.  One load covers 1024 bytes of [reduction][ROWS]; the
//           32-byte granules (16 rows) of a reduction element are exchanged so that the eight of them that 32 lanes read
//           together lie in different banks.
//   STEPS: K steps of 32 bf16 a stage.
template <int ROWS, bool ACROSS, bool STREAM = false, int STEPS = 2>
struct StagedOperand {
    static constexpr int GROUPS = ROWS * STEPS / 16, LOADS = (GROUPS + kProductWaves - 1) / kProductWaves;  // 1 KiB each; of a wavefront
    static constexpr int UNITS = ACROSS ? 32 * STEPS : 8;  // of the reduction in a stage: elements, 16-byte pieces
    static constexpr int BYTES = ROWS * 64 * STEPS;
    static_assert(STEPS == 2 || ACROSS, "a row of a stage along the reduction is 128 bytes");
    static constexpr int PITCH = ROWS * 2;         // across: bytes of a reduction element in LDS
    static_assert(GROUPS >= kProductWaves && GROUPS % 2 == 0, "every wavefront has a group of its own parity");
    static_assert(!ACROSS || (ROWS & (ROWS - 1)) == 0, "rows across are a power of two");

    uint32_t off[LOADS];
    uint64_t base;    // of the stage that is loaded
    int64_t step, back;
    int left, total;  // units from there to the end, and in all (none behind the last stage)
    int todo;         // stages to load, with this one
    int place;        // along: the piece this lane loads; across: its reduction element in the first group

    // (a wavefront without a group in the last round loads its first one again: every one then has the same number in flight)
    static __device__ __forceinline__ int group(int i, int wave)
    {
        const int g = i * kProductWaves + wave;
        return GROUPS % kProductWaves == 0 || g < GROUPS ? g : wave;
    }
    static __device__ __forceinline__ int exchange(int r)
    {
        return ROWS >= 128 ? (r & 3) | ((r >> 3) & 1) << 2 : (ROWS == 64 ? ((r >> 1) & 1) | ((r >> 3) & 1) << 1 : (r >> 3) & 1);
    }

    // rows: how many there are (the last one stands in for others); units: of the reduction, k0 stages of which come last
    __device__ __forceinline__ void begin(const void* at, int64_t ld, int rows, int units, int k0, int wave)
    {
        const int lane = lane_id();
        place = ACROSS ? lane / (ROWS / 8) + wave * (512 / ROWS) : (lane & 7) ^ ((wave & 1) * 4 + (lane >> 4));
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int g = group(i, wave);
            if constexpr (ACROSS) {
                const int at_lane = g * kWave + lane, r = at_lane / (ROWS / 8), piece = (at_lane % (ROWS / 8)) ^ (exchange(r) * 2);
                off[i] = static_cast<uint32_t>(r) * static_cast<uint32_t>(ld) + static_cast<uint32_t>(min(piece, rows / 8 - 1)) * 16u;
            } else {
                off[i] = static_cast<uint32_t>(min(g * 8 + (lane >> 3), rows - 1)) * static_cast<uint32_t>(ld) + static_cast<uint32_t>(place) * 16u;
            }
        }
        step = ACROSS ? UNITS * ld : 128;
        total = units;
        left = units - k0 * UNITS;
        todo = (units + UNITS - 1) / UNITS;
        back = -step * (todo - 1);
        base = reinterpret_cast<uint64_t>(uniform_ptr(static_cast<const unsigned char*>(at))) + static_cast<uint64_t>(k0 * step);
    }
    __device__ __forceinline__ void nothing() { todo = left = total = 0; }  // from here on all loads deliver zeros
    __device__ __forceinline__ void advance()  // to the next stage; behind the end of the reduction follows its begin
    {
        const bool wrap = left <= UNITS;
        todo -= 1;
        total = todo > 0 ? total : 0;
        left = wrap || todo <= 0 ? total : left - UNITS;
        base += static_cast<uint64_t>(wrap ? back : step);
    }
    __device__ __forceinline__ void load(int i, uint32_t lds_addr, int wave)
    {
        const u32x4_v rsrc = {static_cast<uint32_t>(base), static_cast<uint32_t>(base >> 32), kBufferReach, 0x00020000u};
        // (the sign of what is left behind this lane's unit)
        const int spare = left - 1 - place - (ACROSS ? (group(i, wave) - wave) * (512 / ROWS) : 0);
        lds_buffer_16B<STREAM>(rsrc, off[i] | (static_cast<uint32_t>(spare) & kBufferReach), lds_addr + group(i, wave) * 1024);
    }

    // ---- operand fetches: 16 rows from row0 + 16 b on, reduction elements 32 ks + 8 (lane/16) .. +7
    __device__ __forceinline__ static uint32_t fetch_base(int row0, int ks)
    {
        const int in16 = lane_id() & 15, quad = lane_id() >> 4;
        if constexpr (ACROSS) {
            const int r = quad * 8 + (in16 >> 2);
            return static_cast<uint32_t>((ks * 32 + r) * PITCH + ((row0 / 16) ^ exchange(r)) * 32 + (in16 & 3) * 8);
        } else {
            return static_cast<uint32_t>((row0 + in16) * 128 + ((4 * ks + quad) ^ (in16 >> 1)) * 16);
        }
    }
    __device__ __forceinline__ static bf16x8_t fetch(uint32_t stage, uint32_t from, int b)
    {
        if constexpr (ACROSS) {
#if defined(__HIP_DEVICE_COMPILE__)
            typedef __attribute__((address_space(3))) bf16x4_t* lds_ptr;
            const uint32_t at = stage + (from ^ static_cast<uint32_t>(b * 32));
            const bf16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16(reinterpret_cast<lds_ptr>(at));
            const bf16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16(reinterpret_cast<lds_ptr>(at + 4 * PITCH));
            return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
#else
            return bf16x8_t{};
#endif
        } else {
            return lds_fetch<bf16x8_t>(stage + from + static_cast<uint32_t>(b * 2048));
        }
    }
};

// Scale bytes of an operand in 4 bits: a stage is 8 bytes of every row, consecutive in memory.
template <int ROWS>
struct StagedScales {
    static constexpr int GROUPS = ROWS / 32, LOADS = (GROUPS + kProductWaves - 1) / kProductWaves;  // 64 words each
    static constexpr int BYTES = ROWS * 8;
    uint32_t off[LOADS];
    const unsigned char* base;
    int64_t step, back;
    int left, todo;
    static __device__ __forceinline__ int group(int i, int wave) { return min(i * kProductWaves + wave, GROUPS - 1); }
    __device__ __forceinline__ void begin(const uint8_t* scale, int64_t all_rows, int rows, int nk, int k0, int wave)
    {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int word = group(i, wave) * kWave + lane_id();
            off[i] = static_cast<uint32_t>(min(word / 2, rows - 1) * 8 + (word & 1) * 4);
        }
        step = all_rows * 8;
        back = -step * (nk - 1);
        todo = nk;
        left = nk - k0;
        base = uniform_ptr(scale + k0 * step);
    }
    __device__ __forceinline__ void advance()
    {
        todo -= 1;
        if (todo > 0) base += left == 1 ? back : step;  // (behind the last stage it is loaded again: nobody reads it)
        left -= 1;
    }
    __device__ __forceinline__ void load(int i, uint32_t lds_addr, int wave) { lds_dma_4B<false>(base, off[i], lds_addr + group(i, wave) * 256); }
    __device__ __forceinline__ static uint32_t fetch_base(int row0) { return static_cast<uint32_t>((row0 + (lane_id() & 15)) * 8 + (lane_id() >> 4)); }
    __device__ __forceinline__ static int fetch(uint32_t stage, uint32_t from, int b, int ks) { return lds_fetch<uint8_t>(stage + from + static_cast<uint32_t>(b * 128 + ks * 4)); }
};

// ---------------------------------------------------------------------------- tile
template <bool ACC_HALF>
__device__ __forceinline__ void mfma_mx4(bf16x8_t a, bf16x8_t b, f32x4_t& c, int scale_a, int scale_b)
{
#if defined(__HIP_DEVICE_COMPILE__)
    if constexpr (!ACC_HALF)
        asm volatile("v_mfma_scale_f32_16x16x128_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel_hi:[0,0,0] cbsz:4 blgp:4" : "+v"(c) : "v"(a), "v"(b), "v"(scale_a), "v"(scale_b));
    else
    asm volatile("v_mfma_scale_f32_16x16x128_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel_hi:[0,0,0] cbsz:4 blgp:4" : "+a"(c) : "v"(a), "v"(b), "v"(scale_a), "v"(scale_b));
#else
    (void)a; (void)b; (void)c; (void)scale_a; (void)scale_b;
#endif
}

// Ring depths as in ffn_tiles.hpp, with the scales.
constexpr int stage_row_bytes(ProductKind kind) { return kind == kMx4 ? 136 : 128; }
__host__ __device__ constexpr bool product_ring_fits(int H, int NT, int sa, int sb, int row) { return (sa * H + sb * NT) * row <= kLdsBytes; }
__host__ __device__ constexpr int product_stages(int H, int NT, int row, int most = 8)
{
    int s = most;
    while (!product_ring_fits(H, NT, s, s, row)) --s;
    return s;
}
__host__ __device__ constexpr int product_row_stages(int H, int NT, int row, int most = 8)
{
    return most > 2 && product_stages(H, NT, row) == 2 && product_ring_fits(H, NT, 3, 2, row) ? 3 : product_stages(H, NT, row, most);
}
__host__ __device__ constexpr int product_ring_bytes(int H, int NT, int row, int most = 8)
{
    return (product_row_stages(H, NT, row, most) * H + product_stages(H, NT, row, most) * NT) * row;
}

struct NoScales {
    static constexpr int LOADS = 0, BYTES = 0;
};

// ONCE: the weights are loaded with the streaming hint (see rows_tile).
template <int H, int NT, ProductKind KIND, bool ONCE = false, int STAGES = 8, int STEPS = 2>
struct ProductTile {
    static constexpr bool MX = KIND == kMx4;
    static constexpr int WAVES = kProductWaves;
    static constexpr int WN = wave_columns(H, NT, WAVES), WM = WAVES / WN;
    static constexpr int ROW = stage_row_bytes(KIND) * STEPS / 2;
    static constexpr int SA = product_row_stages(H, NT, ROW, STAGES), SB = product_stages(H, NT, ROW, STAGES);
    static constexpr int WTM = H / WM, WTN = NT / WN, TM = WTM / 16, TN = WTN / 16;  // outputs of a wavefront
    static constexpr int SLOTS = TM * TN, HALF = SLOTS / 2;  // matrix instructions of a K step (two a stage); of the last one in front of the hand-over
    typedef StagedOperand<H, KIND == kWeightGradient, false, STEPS> OpA;
    typedef StagedOperand<NT, KIND == kRowsGradient || KIND == kWeightGradient, ONCE, STEPS> OpW;
    typedef typename std::conditional<MX, StagedScales<H>, NoScales>::type ScA;
    typedef typename std::conditional<MX, StagedScales<NT>, NoScales>::type ScW;
    static constexpr int A_BYTES = OpA::BYTES + ScA::BYTES, W_BYTES = OpW::BYTES + ScW::BYTES;
    static constexpr int LA = OpA::LOADS + ScA::LOADS, LW = OpW::LOADS + ScW::LOADS, LPW = LA + LW;  // loads of a wavefront a stage
    static constexpr int IN_FLIGHT = (SA > SB ? LA : 0) + (SB - 2) * LPW;  // behind the next stage at a hand-over
    // (Few accumulators are ordinary registers: moves from and to the accumulator half are a good part of a short reduction's time.)
    static constexpr int ACC_HALF = KIND == kWeightGradient && SLOTS <= 16 ? 0 : 256 / WAVES;
    template <typename TO>
    static constexpr int stores() { return TM * TN / (sizeof(TO) == 4 ? 1 : 2); }  // of a lane, by store()
    static_assert(TN % 2 == 0 && TM * 16 * WM == H && TN * 16 * WN == NT, "outputs of a wavefront");
    static_assert(SA >= SB && SA - SB <= 1 && SB >= 2 && IN_FLIGHT < 64, "ring");
    static_assert(product_ring_bytes(H, NT, ROW, STAGES) <= kLdsBytes, "LDS of a compute unit");

    f32x4_t acc[TM][TN];
    bf16x8_t fw[STEPS][TN], fa[TM];
    int sw[STEPS][TN], sa[TM];  // scales (4 bits)
    f32x4_t sum[TM];        // of the rows over the reduction, where asked for: multiplied by ones
    bf16x8_t ones;
    OpA a;
    OpW w;
    ScA as;
    ScW ws;
    uint32_t from_a[STEPS], from_w[STEPS], from_as, from_ws;
    uint32_t smem_addr;
    int wave;

    __device__ __forceinline__ void issue_a(uint32_t st, int i)
    {
        if (i < OpA::LOADS) a.load(i < OpA::LOADS ? i : 0, smem_addr + st, wave);
        else if constexpr (MX) as.load(i - OpA::LOADS, smem_addr + st + OpA::BYTES, wave);
    }
    __device__ __forceinline__ void issue_w(uint32_t st, int i)
    {
        if (i < OpW::LOADS) w.load(i < OpW::LOADS ? i : 0, smem_addr + SA * A_BYTES + st, wave);
        else if constexpr (MX) ws.load(i - OpW::LOADS, smem_addr + SA * A_BYTES + st + OpW::BYTES, wave);
    }
    __device__ __forceinline__ void step_a()
    {
        a.advance();
        if constexpr (MX) as.advance();
    }
    __device__ __forceinline__ void step_w()
    {
        w.advance();
        if constexpr (MX) ws.advance();
    }
    __device__ __forceinline__ void fetch_a(uint32_t st, int b, int ks)
    {
        fa[b] = OpA::fetch(smem_addr + st, from_a[ks], b);
        if constexpr (MX) sa[b] = ScA::fetch(smem_addr + st + OpA::BYTES, from_as, b, ks);
    }
    __device__ __forceinline__ void fetch_w(uint32_t st, int r, int ks)
    {
        const uint32_t at = smem_addr + SA * A_BYTES + st;
        fw[ks][r] = OpW::fetch(at, from_w[ks], r);
        if constexpr (MX) sw[ks][r] = ScW::fetch(at + OpW::BYTES, from_ws, r, ks);
    }
    __device__ __forceinline__ void multiply(int b, int r, int ks)
    {
        const bool half = b * TN + r < ACC_HALF;
        if constexpr (MX) {
            if (half) mfma_mx4<true>(fw[ks][r], fa[b], acc[b][r], sw[ks][r], sa[b]);
            else mfma_mx4<false>(fw[ks][r], fa[b], acc[b][r], sw[ks][r], sa[b]);
        } else {
            if (half) mfma_16x16x32<true>(fw[ks][r], fa[b], acc[b][r]);
            else mfma_16x16x32<false>(fw[ks][r], fa[b], acc[b][r]);
        }
    }

    struct Stages {  // of one operand's ring: the one read now, the next one, the one whose refill is being completed
        uint32_t cur, nxt, prev;
        __device__ __forceinline__ void advance(uint32_t bytes, uint32_t ring)
        {
            prev = cur;
            cur = nxt;
            nxt = nxt + bytes == ring ? 0 : nxt + bytes;
        }
    };
    Stages ra, rw;

    // Slot of load i of a refill, behind the hand-over; STREAM: all in front of the next stage.
    template <bool STREAM>
    static constexpr int slot_of(int i)
    {
        return i * (STREAM ? SLOTS - HALF : SLOTS) / LPW;
    }
    template <bool STREAM>
    static constexpr int early_loads()  // loads of a refill in front of the next stage
    {
        int n = 0;
        while (n < LPW && slot_of<STREAM>(n) < SLOTS - HALF) ++n;
        return n;
    }

    // At a hand-over the next stage has landed when only what was asked for later is in flight: refills, and the stores of those of the last SB - 1
    // stages that `ends` (a bit each) names as a whole tile's last (loads and stores are counted in the order of their issue).
    template <int STORES>
    __device__ __forceinline__ void wait_for_next(unsigned ends)
    {
        constexpr int most = 63;  // the counter has six bits
        constexpr int one = IN_FLIGHT + STORES < most ? IN_FLIGHT + STORES : most, two = IN_FLIGHT + 2 * STORES < most ? IN_FLIGHT + 2 * STORES : most;
        const int n = STORES > 0 ? __builtin_popcount(ends & ((1u << (SB - 1)) - 1u)) : 0;
        if (n == 0) wait_vmcnt<IN_FLIGHT>();
        else if (n == 1) wait_vmcnt<one>();
        else wait_vmcnt<two>();
    }

    // Matrix instructions of one stage.  Operand fetches run one K step ahead: the weights' registers are double, a row fragment is
    // fetched into the register its last instruction has just read.  At the hand-over (everyone's share of the next stage
    // has landed, everyone is done reading this one) in the middle of the last K step this stage is free: its refill, weights
    // first, is spread up to the middle of the next stage's first K step.
    //   feed: steps both operands on to the stage that is loaded next.
    //   STREAM: tiles in one stream, STORES of a lane behind each.  A refill is complete in front of the next stage, because behind the last
    //   stage of a tile come its stores, which a load behind them would have to wait for.
    template <bool NEXT, bool STREAM, int STORES, bool SUMS, typename Feed>
    __device__ __forceinline__ void stage(unsigned ends, bool sums, Feed&& feed)
    {
        static_assert(STEPS == 2 || STREAM, "a refill is spread over two K steps");
#pragma unroll
        for (int ks = 0; ks < STEPS; ++ks) {
            const bool last = ks == STEPS - 1;
#pragma unroll
            for (int m = 0; m < SLOTS; ++m) {
                const int r = m % TN, b = m / TN;
                if (NEXT && last && m == HALF) {
                    wait_for_next<STORES>(ends);
                    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // my operand fetches from this stage are complete
                    __builtin_amdgcn_s_barrier();
                    asm volatile("" ::: "memory");
                    feed(*this);
                }
                multiply(b, r, ks);
                if (KIND == kWeightGradient && SUMS && sums && r == TN - 1) mfma_16x16x32<false>(ones, fa[b], sum[b]);
                __builtin_amdgcn_sched_barrier(0);
                if constexpr (STEPS == 2) if (!last) {
                    if (r == TN - 1) fetch_a(ra.cur, b, 1);
#pragma unroll
                    for (int q = 0; q < TN; ++q)
                        if (m == (q * SLOTS / TN + 1 < SLOTS ? q * SLOTS / TN + 1 : SLOTS - 1)) fetch_w(rw.cur, q, 1);
                }
                if (last && NEXT) {
#pragma unroll
                    for (int q = 0; q < TN; ++q) {
                        const int free = STEPS > 1 ? 0 : (TM - 1) * TN + q;  // (one K step a stage: these registers, too, are in use till then)
                        const int want = HALF + 2 * q > free ? HALF + 2 * q : free;
                        const int p = want < SLOTS ? want : SLOTS - 1;
                        if (m == p) fetch_w(rw.nxt, q, 0);
                    }
#pragma unroll
                    for (int q = 0; q < TM; ++q) {
                        const int free = q * TN + TN - 1;  // its last instruction of this stage
                        const int want = HALF + 2 * q + 1 > free ? HALF + 2 * q + 1 : free;
                        const int p = want < SLOTS ? want : SLOTS - 1;
                        if (m == p) fetch_a(ra.nxt, q, 0);
                    }
                }
                const bool begun = last && m >= HALF;
                if (NEXT) {
#pragma unroll
                    for (int i = 0; i < LPW; ++i)
                        if (slot_of<STREAM>(i) == (begun ? m - HALF : SLOTS - HALF + ks * SLOTS + m)) {
                            if (i < LW) issue_w(begun ? rw.cur : rw.prev, i < LW ? i : 0);
                            else issue_a(begun ? ra.cur : ra.prev, i >= LW ? i - LW : 0);
                        }
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        }
    }

    // The accumulators begin with the bias of their columns, or with zeros.  The bias comes on the scalar path: a load to vector registers would be awaited
    // together with all stages of the ring.
    __device__ __forceinline__ void begin_sums(const bf16_t* bias, int cols)
    {
#pragma unroll
        for (int r = 0; r < TN; ++r) {
            f32x4_t v = {0.f, 0.f, 0.f, 0.f};
#if defined(__HIP_DEVICE_COMPILE__)
            const int quad = lane_id() >> 4;
            if (bias != nullptr) {
                uint32_t pair[2][2];  // of this lane's columns, if they lie in the lower or in the upper eight of 16
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int col = __builtin_amdgcn_readfirstlane(min(wave % WN * WTN + r * 16 + h * 8, cols - 8));
                    const auto* at = (const __attribute__((address_space(4))) uint32_t*)uniform_ptr(reinterpret_cast<const unsigned char*>(bias + col));
                    uint32_t d[4] = {at[0], at[1], at[2], at[3]};
                    asm volatile("" : "+s"(d[0]), "+s"(d[1]), "+s"(d[2]), "+s"(d[3]));
                    pair[h][0] = (quad & 1) != 0 ? d[2] : d[0];
                    pair[h][1] = (quad & 1) != 0 ? d[3] : d[1];
                }
                const uint32_t x = quad > 1 ? pair[1][0] : pair[0][0], y = quad > 1 ? pair[1][1] : pair[0][1];
                v = f32x4_t{__uint_as_float(x << 16), __uint_as_float(x & 0xffff0000u), __uint_as_float(y << 16), __uint_as_float(y & 0xffff0000u)};
            }
#endif
#pragma unroll
            for (int b = 0; b < TM; ++b) acc[b][r] = v;
        }
        if constexpr (KIND == kWeightGradient) {
#pragma unroll
            for (int b = 0; b < TM; ++b) sum[b] = f32x4_t{0.f, 0.f, 0.f, 0.f};
            ones = __builtin_bit_cast(bf16x8_t, u32x4_v{0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u});
            asm volatile("" : "+v"(ones));  // (in its registers from here on: a matrix instruction must not follow its operand's write at once)
        }
        pin_registers();
    }
    __device__ __forceinline__ void clear()
    {
        begin_sums(nullptr, 0);
        pin_accumulators();
    }

    __device__ __forceinline__ void next_stage()
    {
        ra.advance(A_BYTES, SA * A_BYTES);
        rw.advance(W_BYTES, SB * W_BYTES);
    }
    // The ring is filled as if the stage before the first one had handed over (all but the late loads of its last stage), and the first operands
    // are fetched.
    //   meanwhile: what is done while the first loads are on their way.
    template <bool STREAM, typename FeedA, typename FeedW, typename Meanwhile>
    __device__ __forceinline__ void begin_ring(FeedA&& feed_a, FeedW&& feed_w, Meanwhile&& meanwhile)
    {
        const int wm = wave / WN, wn = wave % WN;
#pragma unroll
        for (int ks = 0; ks < STEPS; ++ks) {
            from_a[ks] = OpA::fetch_base(wm * WTM, ks);
            from_w[ks] = OpW::fetch_base(wn * WTN, ks);
        }
        if constexpr (MX) {
            from_as = ScA::fetch_base(wm * WTM);
            from_ws = ScW::fetch_base(wn * WTN);
        }
        constexpr int EARLY = early_loads<STREAM>();
#pragma unroll
        for (int s = 0; s < SA; ++s) {
            if (s > 0 && s < SB) feed_w(*this);
            if (s > 0) feed_a(*this);
#pragma unroll
            for (int i = 0; i < LPW; ++i) {
                if (i < LW && s < SB && (s < SB - 1 || i < EARLY)) issue_w(static_cast<uint32_t>(s * W_BYTES), i < LW ? i : 0);
                if (i >= LW && (s < SA - 1 || i < EARLY)) issue_a(static_cast<uint32_t>(s * A_BYTES), i >= LW ? i - LW : 0);
            }
        }
        meanwhile();
        wait_vmcnt<(SB - 2) * LW + (SA - 2) * LA + EARLY>();  // the first stage is complete when only what follows it is in flight
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
#pragma unroll
        for (int r = 0; r < TN; ++r) fetch_w(0u, r, 0);
#pragma unroll
        for (int b = 0; b < TM; ++b) fetch_a(0u, b, 0);
        ra = Stages{0u, static_cast<uint32_t>(A_BYTES), static_cast<uint32_t>((SA - 1) * A_BYTES)};
        rw = Stages{0u, static_cast<uint32_t>(W_BYTES), static_cast<uint32_t>((SB - 1) * W_BYTES)};
    }

    // All of a reduction of nk stages, at least one.  Behind it the accumulators hold the sums.
    __device__ __forceinline__ void reduce(int nk, bool sums = false, const bf16_t* bias = nullptr, int cols = 0)
    {
        begin_ring<false>([](ProductTile& t) { t.step_a(); }, [](ProductTile& t) { t.step_w(); }, [&]() { begin_sums(bias, cols); });
        pin_accumulators();
        auto on = [](ProductTile& t) {
            t.step_a();
            t.step_w();
        };
        for (int kt = 1; kt < nk; ++kt) {
            stage<true, false, 0, true>(0u, sums, on);
            next_stage();
        }
        stage<false, false, 0, true>(0u, sums, on);
        wait_vmcnt<0>();  // (loads into LDS that nobody waited for)
        pin_accumulators();
    }

    // (the compiler sees neither that the matrix instructions read the accumulators nor that they write them)
    __device__ __forceinline__ void pin_registers()
    {
#if defined(__HIP_DEVICE_COMPILE__)
#pragma unroll
        for (int b = 0; b < TM; ++b)
#pragma unroll
            for (int r = 0; r < TN; ++r) {
                if (b * TN + r < ACC_HALF) asm volatile("" : "+a"(acc[b][r]));
                else asm volatile("" : "+v"(acc[b][r]));
            }
        if constexpr (KIND == kWeightGradient) {
#pragma unroll
            for (int b = 0; b < TM; ++b) asm volatile("" : "+v"(sum[b]));
        }
#endif
    }
    // The accumulators are there before an instruction reads them, and the last one is done before they are read.
    __device__ __forceinline__ void pin_accumulators()
    {
#if defined(__HIP_DEVICE_COMPILE__)
        asm volatile("s_nop 15\n\ts_nop 15" ::: "memory");
        pin_registers();
        asm volatile("s_nop 15\n\ts_nop 15" ::: "memory");
#endif
    }

    // 16-byte pieces of row in16 (of 16) and of unit 0 / unit 1, 64 bytes of a row each: lanes 8 to 15 trade with lanes 0 to 7, and `lo` is rows 0 to 7, `hi`
    // rows 8 to 15, of unit in16 / 8.  A store then covers 128 bytes of a row, a whole line.
    static __device__ __forceinline__ void trade(const uint32_t (&u0)[4], const uint32_t (&u1)[4], uint4& lo, uint4& hi)
    {
        uint32_t l[4], h[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            l[i] = __builtin_amdgcn_update_dpp(u0[i], u1[i], 0x128, 0xf, 0xc, false);  // row_ror:8 into the upper half
            h[i] = __builtin_amdgcn_update_dpp(u1[i], u0[i], 0x128, 0xf, 0x3, false);  // into the lower half
        }
        lo = make_uint4(l[0], l[1], l[2], l[3]);
        hi = make_uint4(h[0], h[1], h[2], h[3]);
    }

    // out[row][col] of the tile's rows and columns that there are, leading dimension ldo.  A lane holds, of the 16 x 16 block
    // (b, r), row lane%16 and columns 4 (lane/16) .. +3: in fp32 16 bytes, 64 of the row with the other lanes.  bf16: of two
    // blocks side by side the odd rows of 16 lanes of the first trade with the even ones of the second, and every lane has
    // eight consecutive columns of one block.
    //   A whole tile's stores have no condition: where a wavefront is alone on its SIMD every instruction here is time.
    template <typename TO>
    __device__ __forceinline__ void store(TO* out, int64_t ldo, int rows, int cols) const
    {
        if (rows == H && cols == NT) store_as<TO, true>(out, ldo, rows, cols);
        else store_as<TO, false>(out, ldo, rows, cols);
    }
    template <typename TO, bool WHOLE>
    __device__ __forceinline__ void store_as(TO* out, int64_t ldo, int rows, int cols) const
    {
        constexpr int BLOCKS = sizeof(TO) == 4 ? 1 : 2;                // of a unit
        constexpr bool PAIRS = TN % (2 * BLOCKS) == 0;
        constexpr int PER = PAIRS ? 2 : 1;                              // units of a store
        const int quad = lane_id() >> 4, in16 = lane_id() & 15, wm = wave / WN, wn = wave % WN;
        const int in_unit = BLOCKS == 1 ? quad * 4 : (quad & 1) * 16 + (quad >> 1) * 8;
        // (row by row: rows are often a power of two bytes apart, and column by column all compute units would write to few memory channels at a time)
#pragma unroll
        for (int b = 0; b < TM; ++b) {
#pragma unroll
            for (int r = 0; r < TN; r += BLOCKS * PER) {
                uint32_t u[PER][4];
#pragma unroll
                for (int i = 0; i < PER; ++i) {
                    if constexpr (BLOCKS == 1) {
#pragma unroll
                        for (int v = 0; v < 4; ++v) u[i][v] = __float_as_uint(acc[b][r + i][v]);
                    } else {
                        uint32_t p[2][2];
#pragma unroll
                        for (int q = 0; q < 2; ++q)
#pragma unroll
                            for (int v = 0; v < 2; ++v) {
                                const int c = r + 2 * i + q;
                                p[q][v] = pack_bf16x2(acc[b][c][2 * v], acc[b][c][2 * v + 1]);
                            }
                        const auto s0 = __builtin_amdgcn_permlane16_swap(p[0][0], p[1][0], false, false);
                        const auto s1 = __builtin_amdgcn_permlane16_swap(p[0][1], p[1][1], false, false);
                        u[i][0] = s0[0], u[i][1] = s1[0], u[i][2] = s0[1], u[i][3] = s1[1];
                    }
                }
                const int row = wm * WTM + b * 16, col = wn * WTN + r * 16 + in_unit;
                // Rows that begin anywhere in a line leave lines in part to the next tile: those stay in the L2 until they are whole (weight gradients, us with the
                // streaming hint and without: fp32, 235 rows, 8 experts of 1240 x 11752 229 and 113, bf16, 291 rows, 15 of 1432 x 2264 44 and 40; of whole
                // lines, fp32, 16384 rows, 32 of 8192 x 2048 837 and 882).
                const bool plain = ldo * static_cast<int>(sizeof(TO)) % 128 != 0;
                auto put = [&](TO* at, uint4 v) {
                    if (plain) *reinterpret_cast<uint4*>(at) = v;
                    else store_stream16(reinterpret_cast<uint4*>(at), v);
                };
                if constexpr (PAIRS) {
                    uint4 lo, hi;
                    trade(u[0], u[PER - 1], lo, hi);
                    const int row_lo = row + (in16 & 7), col_of = col + (in16 >> 3) * BLOCKS * 16;
                    TO* to = out + row_lo * ldo + col_of;
                    if (WHOLE || (row_lo < rows && col_of < cols)) put(to, lo);
                    if (WHOLE || (row_lo + 8 < rows && col_of < cols)) put(to + 8 * ldo, hi);
                } else if (WHOLE || (row + in16 < rows && col < cols)) {
                    put(out + (row + in16) * ldo + col, make_uint4(u[0][0], u[0][1], u[0][2], u[0][3]));
                }
            }
        }
    }
    // The sums over the reduction of the tile's rows.
    template <typename TO>
    __device__ __forceinline__ void store_sums(TO* out, int rows) const
    {
        const int wm = wave / WN;
        if (wave % WN != 0 || lane_id() >= 16) return;
#pragma unroll
        for (int b = 0; b < TM; ++b) {
            const int row = wm * WTM + b * 16 + lane_id();
            if (row < rows) {
                if constexpr (sizeof(TO) == 4) out[row] = sum[b][0];
                else out[row] = f32_to_bf16(sum[b][0]);
            }
        }
    }
};

template <typename T>
__device__ __forceinline__ void begin_tile(T& t, unsigned char* smem)
{
    t.wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    t.smem_addr = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) unsigned char*)smem));
}

// ---------------------------------------------------------------------------- an output row a sorted row
struct RowsTiles {
    const void* rows;         // [A,K]
    const int32_t* offsets;
    const void* weight;       // [E_local,N,K], rows' gradient [E_local,K,N]
    const bf16_t* bias;       // [E_local,N] or null
    bf16_t* out;              // [A,N]
    const uint8_t *row_scale, *weight_scale;
    int max_rows, K, N, E_local;
};

template <int H, int NT, ProductKind KIND, bool ONCE>
__device__ __forceinline__ void rows_tile(const RowsTiles& p, const Tile2D& tile, unsigned char* smem)
{
    typedef ProductTile<H, NT, KIND, ONCE> T;
    T t;
    begin_tile(t, smem);
    const int64_t row_bytes = KIND == kMx4 ? p.K / 2 : static_cast<int64_t>(p.K) * 2, K = p.K, N = p.N;
    const int rows = tile.row_end - tile.row_begin, cols = min(NT, p.N - tile.n0);
    const int per_stage = KIND == kMx4 ? 256 : 64, nk = (p.K + per_stage - 1) / per_stage;
    const int k0 = static_cast<int>(static_cast<unsigned>(tile.turn) * static_cast<unsigned>(nk) / kComputeUnits);
    const int pieces = static_cast<int>(row_bytes / 16);
    t.a.begin(static_cast<const unsigned char*>(p.rows) + tile.row_begin * row_bytes, row_bytes, rows, pieces, k0, t.wave);
    if constexpr (KIND == kRowsGradient)
        t.w.begin(static_cast<const bf16_t*>(p.weight) + tile.expert * K * N + tile.n0, N * 2, cols, p.K, k0, t.wave);
    else
        t.w.begin(static_cast<const unsigned char*>(p.weight) + (tile.expert * N + tile.n0) * row_bytes, row_bytes, cols, pieces, k0, t.wave);
    if constexpr (KIND == kMx4) {
        t.as.begin(p.row_scale + static_cast<int64_t>(tile.row_begin) * 8, p.max_rows, rows, nk, k0, t.wave);
        t.ws.begin(p.weight_scale + (tile.expert * N + tile.n0) * 8, p.E_local * N, cols, nk, k0, t.wave);
    }
    t.reduce(nk, false, p.bias != nullptr ? p.bias + tile.expert * N + tile.n0 : nullptr, cols);
    t.store(p.out + tile.row_begin * N + tile.n0, N, rows, cols);
}

// A whole tile of 320 rows and 256 columns in 4 bits has no registers left for the scales (it would spill 44 of them): there tiles take one
// quantum at most.
constexpr int most_quanta(ProductKind kind) { return kind == kMx4 ? 1 : 2; }
constexpr bool has_product_instance(ProductKind kind, int NT, int height, int cut)
{
    return has_instance(NT, height, cut) && !(cut == 0 && height > kTileRows + most_quanta(kind) * kQuantum);
}

// STREAMS: tiles whose weights nobody else reads load them with the streaming hint, and the column tiles of experts of few rows begin the reduction
// at different places (see locate_tile and streams_weights).
template <int NT, ProductKind KIND, bool STREAMS>
__global__ __launch_bounds__(kProductWaves * kWave, 1) void rows_tiles_kernel(const RowsTiles p)
{
    extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
    const RowRange range = row_range(p.offsets, p.E_local, p.max_rows);
    Tile2D tile;
    if (!locate_tile<STREAMS, most_quanta(KIND)>(range, NT, p.N, static_cast<int>(blockIdx.x), RowMap{}, tile)) return;
#define EXF_CASE(H, CUT, ONCE)            \
    case (CUT) * 16 + (H) / kQuantum: \
        if constexpr (has_product_instance(KIND, NT, H, CUT) && (!(ONCE) || H <= kTileRows)) rows_tile<H, (NT >> CUT), KIND, ONCE>(p, tile, smem); \
        break
#define EXF_CASES(CUT, ONCE)  \
    EXF_CASE(64, CUT, ONCE);  \
    EXF_CASE(96, CUT, ONCE);  \
    EXF_CASE(128, CUT, ONCE); \
    EXF_CASE(160, CUT, ONCE); \
    EXF_CASE(192, CUT, ONCE); \
    EXF_CASE(224, CUT, ONCE); \
    EXF_CASE(256, CUT, ONCE); \
    EXF_CASE(288, CUT, ONCE); \
    EXF_CASE(320, CUT, ONCE)
    const int instance = tile.cut * 16 + tile.height / kQuantum;
    if (STREAMS && tile.once) {
        switch (instance) {
            EXF_CASES(0, STREAMS);
            EXF_CASES(1, STREAMS);
            EXF_CASES(2, STREAMS);
        }
    } else {
        switch (instance) {
            EXF_CASES(0, false);
            EXF_CASES(1, false);
            EXF_CASES(2, false);
        }
    }
#undef EXF_CASES
#undef EXF_CASE
}

template <int NT, ProductKind KIND>
constexpr int rows_tiles_lds()
{
    constexpr int row = stage_row_bytes(KIND);
    int most = 0;
    const int heights[] = {64, 96, 128, 160, 192, 224, 256, 288, 320};
    for (int h : heights)
        for (int cut = 0; cut <= 2; ++cut)
            if (has_product_instance(KIND, NT, h, cut) && product_ring_bytes(h, NT >> cut, row) > most) most = product_ring_bytes(h, NT >> cut, row);
    return most;
}

template <int NT, ProductKind KIND, bool STREAMS>
static int launch_rows_tiles_as(const RowsTiles& p, hipStream_t stream, const char* fn)
{
    constexpr size_t lds = rows_tiles_lds<NT, KIND>();
    const int64_t grid = tile_grid(p.max_rows, p.N, NT, p.E_local);
    if (grid >= (1ll << 31)) return fail(EXF_ERR_BAD_SHAPE, "%s: too many tiles", fn);
    auto kern = rows_tiles_kernel<NT, KIND, STREAMS>;
    static std::atomic<uint64_t> allowed{0};
    if (int rc = allow_lds(reinterpret_cast<const void*>(kern), lds, allowed, fn)) return rc;
    hipLaunchKernelGGL(kern, dim3(static_cast<unsigned>(grid)), dim3(kProductWaves * kWave), lds, stream, p);
    return EXF_OK;
}

// Weights too many to stay in the memory-side cache of 256 MB from call to call, and so few rows that many experts have one row tile (the lines of
// ffn.hip).  512 rows, 64 experts of 16384 x 4096 as tiles 1481 us without and 1367 with; in 4 bits 384 and 361.
//   Not where weight rows begin off the lines: two loads share a line then, and the second one has to find it in the L2 (501 rows, 7 experts of 6664 x 11816
// 320 us without and 365 with; 2864 in 4 bits, 36 of 6032 x 4288 150 and 177).
inline bool streams_weights(const RowsTiles& p, ProductKind kind)
{
    const int64_t row = static_cast<int64_t>(kind == kRowsGradient ? p.N : p.K) * (kind == kMx4 ? 1 : 4) / 2;
    const int64_t bytes = row * p.E_local * (kind == kRowsGradient ? p.K : p.N);
    return row % 128 == 0 && p.max_rows <= 1024ll * p.E_local && bytes >= 128ll << 20;
}
template <int NT, ProductKind KIND>
static int launch_rows_tiles(const RowsTiles& p, hipStream_t stream, const char* fn)
{
    return streams_weights(p, KIND) ? launch_rows_tiles_as<NT, KIND, true>(p, stream, fn) : launch_rows_tiles_as<NT, KIND, false>(p, stream, fn);
}

int launch_forward_tiles(const RowsTiles& p, hipStream_t stream);
int launch_rows_gradient_tiles(const RowsTiles& p, hipStream_t stream);
int launch_mx4_tiles(const RowsTiles& p, hipStream_t stream);
// bf16; the workspace holds partial sums where weight_gradient_splits() is more than one.
int weight_gradient_splits(int64_t A, int n, int k, int E_local);
int launch_weight_gradient_tiles(const WeightGradient& p, int grad_dt, hipStream_t stream);

}  // namespace exf
