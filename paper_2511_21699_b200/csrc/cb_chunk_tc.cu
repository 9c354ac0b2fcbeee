// Attention of chunks of new tokens over the paged cache on the 5th-generation tensor cores (tcgen05) with TMA-staged keys and values.
//
// Persistent kernel, one CTA per SM, built like tree attention (cb_attn_tc.cu, which explains the chains and their costs): a CTA holds up
// to two 128-row query tiles of a unit (128 / G tokens times the G query heads of a kv head) and streams the unit's 128-key tiles through a
// ring of shared-memory slots; two chains S = Q K^T -> softmax -> O += P V run side by side, each with a row tile of its own, or, in a unit
// with one row tile (single tokens, the end of a chunk), with every second key tile, or with the unit of a head of its own.  The split over the CTAs is in cb_chunk_sched.cuh; the
// CTAs of a shared unit put their unnormalised parts together through memory, the last one to come writes the rows.
//
// Warp roles (640 threads): warp 0 copies K tiles, warp 3 V tiles, warp 1 issues the products, warp 2 walks the units, publishes them to all
// others and loads their query tiles, warps 4..19 are the softmax warpgroups (4..11 chain 0, 12..19 chain 1; a row's 128 scores over
// two threads).  All waits are bounded; one that runs out records CB_ERR_TIMEOUT and the CTA drains and exits.
//
// Causality: a row sees the keys up to its own token.  Tiles below a row tile's first token need no mask; the first row tile of a unit leaves
// out a last tile that only the second one sees.  Slots of the last page behind the sequence's last token may hold anything: their scores are
// masked, and their values are overwritten with zeros in shared memory before the product reads them (0 x NaN would reach the output).
//
// Measured: a prompt of 8 k, 64 query heads over 8, D = 128: 1.01 ms in short runs, 1.11 under the power cap, 1.0 to 1.1 PFLOP/s of the visible scores, the tensor pipe 54% busy;
// a pair of tiles takes 3.3 k to 3.5 k cycles of which 2.05 k are products, the rest hand-overs between the softmax and the products.  64 single tokens over 1.09 GB
// of keys and values: 188 to 207 us, 5.3 to 5.8 TB/s.  One token over 4 k, 32 heads: 23.8 us, nearly all of it before the first tile and behind the last.
// Of the spills (124 to 132 bytes a thread) three to four loads and one store a tile and softmax warp lie in the tile loop, beside some 450 instructions; the others
// are a unit's, some ten (counted over prompts of 1 k to 4 k).
#include <cuda.h>

#include <mutex>
#include <type_traits>

#include "cb_chunk_sched.cuh"
#include "cb_tc_dev.cuh"

namespace {

constexpr int kTwoHeads = 3;                                  // the whole units of heads kh and kh + 1, of one row tile, a chain each

// A unit as its roles see it (nrt: row tiles, or kTwoHeads; 0: no more units).
struct ChunkUnit {
    int b, kh, rg, t0, t1, tiles, nrt;
    int row0, n, ctx, end;    // first packed row, new and cached tokens of the sequence, keys that the unit sees
    int seq0;                 // copies made before it
    int skip;                 // two row tiles: 1 if the first one sees nothing of the last tile and leaves it out
    int dirty;                // slots of the last page behind the sequence's last token
    int cf, np, xpos, wt, ticket;   // shared units: the CTA that holds the first tile, CTAs that hold one, see below
};
constexpr int kUnitRing = 4;                                  // published ahead of the slowest role: at most two

template <int D>
struct Cfg {
    static constexpr int DB = D / 64;                         // 64-element (128-byte) column blocks per row
    static constexpr int NSLOT = (D == 128) ? 5 : 8;          // ring slots, each one K or one V tile
    static constexpr uint32_t TILE_BYTES = CB_KT * D * 2;
    static constexpr uint32_t Q_BYTES = CB_MT * D * 2;
    static constexpr uint32_t OFF_Q = 0;                      // two row tiles
    static constexpr uint32_t OFF_RING = 2 * Q_BYTES;
    static constexpr uint32_t OFF_BAR = OFF_RING + NSLOT * TILE_BYTES;
    // slot_full[NSLOT], slot_free[NSLOT], q_full[2], q_free[2], s_full[3], p_ready[3], pv_done[3], o_done[2], o_done_both, o_free[2], sums, unit_full[kUnitRing]
    static constexpr int NBAR = 2 * NSLOT + 19 + kUnitRing;
    static constexpr uint32_t OFF_UNITS = OFF_BAR + NBAR * 8;
    static constexpr uint32_t OFF_X = (OFF_UNITS + kUnitRing * sizeof(ChunkUnit) + 15) / 16 * 16;   // [2 chains][2][128 rows]
    static constexpr uint32_t OFF_MISC = OFF_X + 2 * 2 * CB_MT * 4;                  // positions of all units, tmem base, abort flag, pair counters
    static constexpr uint32_t SMEM = OFF_MISC + 16 + 64;
    static_assert(SMEM <= 227 * 1024, "shared memory of one CTA");
    // TMEM columns: the S buffers 128 apart from 0, O0 and O1 behind them.  With head_dim 128 a chain has one S buffer, and its next S
    // follows the product that reads the P over the last one.  With 64 there is room for a third, and the turns of both chains take the three in turn:
    // the next S of a chain is there before its softmax is done with the one before, and the product comes behind it.
    static constexpr int NSB = (D == 128) ? 2 : 3;
    static constexpr uint32_t O_COL = NSB * 128;
    static_assert(O_COL + 2 * D <= kTmemCols, "tensor memory of an SM");
};

struct ChunkMaps { CUtensorMap k, v, q; };

template <int D>
__global__ void __launch_bounds__(kThreads, 1) cb_chunk_tc_kernel(const CbChunkParams p, const __grid_constant__ ChunkMaps maps) {
    using C = Cfg<D>;
    extern __shared__ __align__(1024) uint8_t chunk_smem[];
    uint8_t* const sgen = chunk_smem;
    const uint32_t sbase = smem_u32(chunk_smem);
    if (sbase & 1023u) {                                      // the swizzled tiles need it; every thread sees the same address
        if (threadIdx.x == 0) atomicCAS(p.status, 0u, (uint32_t)CB_ERR_UNSUPPORTED);
        return;
    }
    const uint32_t bar0 = sbase + C::OFF_BAR;
    auto bar_full = [&](uint32_t s) { return bar0 + 8u * s; };
    auto bar_free = [&](uint32_t s) { return bar0 + 8u * (C::NSLOT + s); };
    auto slot_base = [&](uint32_t s) { return sbase + C::OFF_RING + s * C::TILE_BYTES; };
    constexpr uint32_t B1 = 2 * C::NSLOT;
    auto bar_qfull = [&](int k) { return bar0 + 8u * (B1 + k); };
    auto bar_qfree = [&](int k) { return bar0 + 8u * (B1 + 2 + k); };
    auto bar_sfull = [&](int k) { return bar0 + 8u * (B1 + 4 + k); };      // by S buffer, as the next two
    auto bar_pready = [&](int k) { return bar0 + 8u * (B1 + 7 + k); };
    auto bar_pvdone = [&](int k) { return bar0 + 8u * (B1 + 10 + k); };    // three buffers only
    auto bar_odone = [&](int l) { return bar0 + 8u * (B1 + 13 + l); };
    const uint32_t bar_odone_both = bar0 + 8u * (B1 + 15);
    auto bar_ofree = [&](int l) { return bar0 + 8u * (B1 + 16 + l); };
    const uint32_t bar_sums = bar0 + 8u * (B1 + 18);
    auto bar_ufull = [&](uint32_t k) { return bar0 + 8u * (B1 + 19 + k); };
    constexpr uint32_t kSoftWarps = 16;                       // a warp arrives once, behind a __syncwarp
    ChunkUnit* s_units = reinterpret_cast<ChunkUnit*>(sgen + C::OFF_UNITS);
    volatile float* s_x = reinterpret_cast<volatile float*>(sgen + C::OFF_X);
    volatile long long* s_tot = reinterpret_cast<volatile long long*>(sgen + C::OFF_MISC);
    uint32_t* s_tmem = reinterpret_cast<uint32_t*>(sgen + C::OFF_MISC + 8);
    volatile int* s_abort = reinterpret_cast<volatile int*>(sgen + C::OFF_MISC + 12);
    volatile int* s_pair = reinterpret_cast<volatile int*>(sgen + C::OFF_MISC + 16);   // [16 softmax warps]: last pair barrier entered, -1 = left

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int cta = blockIdx.x;
    const int RT = p.NPT * p.G;                               // rows of a row tile that exist
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(s_tmem)), "r"(kTmemCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    } else if (warp == 2) {
        if (lane == 0) {
            for (int s = 0; s < C::NSLOT; ++s) { mbar_init(bar_full(s), 1); mbar_init(bar_free(s), 1); }
            for (int l = 0; l < 2; ++l) {
                mbar_init(bar_qfull(l), 1); mbar_init(bar_qfree(l), 1);
                mbar_init(bar_odone(l), 1); mbar_init(bar_ofree(l), kSoftWarps);
            }
            for (int k = 0; k < C::NSB; ++k) { mbar_init(bar_sfull(k), 1); mbar_init(bar_pready(k), kSoftWarps / 2); mbar_init(bar_pvdone(k), 1); }
            mbar_init(bar_odone_both, 1); mbar_init(bar_sums, kSoftWarps);
            for (int k = 0; k < kUnitRing; ++k) mbar_init(bar_ufull(k), 1);
            *s_abort = 0;
            asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
            tma_prefetch_desc(&maps.k); tma_prefetch_desc(&maps.v); tma_prefetch_desc(&maps.q);
        }
        if (lane < 16) s_pair[lane] = 0;
    }
    CB_PDL_ENTRY();
    // What the first copy waits for is asked for before the barrier and lies in L1 when it is wanted: the lengths that the schedule reads first, and,
    // where a unit's CTAs are known, the block table's entries of this CTA's first tile if the sequence is as long as the caller's bound.
    const int unit = p.cs == 0 ? 0 : (p.cs == 1 ? cta : (int)__umulhi((uint32_t)cta, p.cs_inv)), seq_b = p.Hkv == 1 ? unit : (int)__umulhi((uint32_t)unit, p.hkv_inv);
    if (warp == 2) {
        const int b = p.cs > 0 ? seq_b : lane;
        if (b < p.B) {
            uint32_t x;
            asm volatile("ld.global.ca.u32 %0, [%1];" : "=r"(x) : "l"(p.q_start + b) : "memory");
            asm volatile("ld.global.ca.u32 %0, [%1];" : "=r"(x) : "l"(p.q_start + b + 1) : "memory");
            asm volatile("ld.global.ca.u32 %0, [%1];" : "=r"(x) : "l"(p.ctx_len + b) : "memory");
        }
    } else if ((warp == 0 || warp == 3) && p.cs > 0 && lane == 0) {
        const int tiles = (p.max_keys + CB_KT - 1) / CB_KT, n = min(p.cs, tiles);
        const long long at = cb_quot((long long)(tiles * min(cta - unit * p.cs, n - 1)), n) * (CB_KT / 16);
        if (at < p.max_pages) {
            uint32_t x;
            asm volatile("ld.global.ca.u32 %0, [%1];" : "=r"(x) : "l"(p.block_table + (size_t)seq_b * p.max_pages + at) : "memory");
        }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *s_tmem;
    constexpr uint32_t ns = (uint32_t)C::NSLOT;

    if (warp < 4) {
        reg_dealloc<64>();
        bool ok = true;
        if (warp == 0 || warp == 3) {
            // ------------------------------------------------------------------ K/V producers
            // A page's 16 keys of a head are one box, laid out as groups of 8 keys with a group's 64-dim column blocks behind one another;
            // a tile is eight copies, one per lane.  K and V tiles alternate in the ring.
            const bool isV = warp == 3;
            constexpr uint32_t GROUP = 1024 * C::DB;          // bytes of 8 keys
            const bool active = lane < 8;
            if (isV) {
                // The block table into L2, a slice per CTA, while the units are worked out: the first copies' addresses come from it.
                const long long lines = ((long long)p.B * p.max_pages * 4 + 127) / 128;
                for (long long k = (long long)cta * 32 + lane, n = 0; k < lines && n < 4; k += (long long)gridDim.x * 32, ++n)
                    asm volatile("prefetch.global.L2 [%0];" ::"l"(reinterpret_cast<const char*>(p.block_table) + k * 128));
            }
            for (uint32_t uq = 0; (ok = mbar_wait(bar_ufull(uq % kUnitRing), (uq / kUnitRing) & 1, s_abort, p.status)); ++uq) {
                const volatile ChunkUnit* u = &s_units[uq % kUnitRing];
                if (u->nrt == 0) break;
                const int t0 = u->t0, t1 = u->t1, kh = u->kh, npages = (u->end + 15) / 16, heads = u->nrt == kTwoHeads ? 2 : 1;   // their tiles come in turn
                const int32_t* bt = p.block_table + (size_t)u->b * p.max_pages;
                uint32_t seq = (uint32_t)u->seq0 + (isV ? 1u : 0u);
                // the page number is fetched one tile ahead of the copy that depends on it; out of the pool, the copy fills zeros
                auto page_of = [&](int i) {
                    const int pidx = i * (CB_KT / 16) + lane;
                    const int page = active && pidx < npages ? bt[pidx] : p.num_pages;
                    return (uint32_t)page < (uint32_t)p.num_pages ? page : p.num_pages;
                };
                int page_next = page_of(t0);
                for (int i = t0; i < t1 && ok; ++i) {
                    const int page = page_next;
                    if (i + 1 < t1) page_next = page_of(i + 1);
                    for (int hd = 0; hd < heads; ++hd, seq += 2) {
                        const uint32_t sl = seq % ns;
                        if (seq >= ns && !(ok = mbar_wait(bar_free(sl), (seq / ns - 1) & 1, s_abort, p.status))) break;
                        if (lane == 0) mbar_expect_tx(bar_full(sl), C::TILE_BYTES);
                        __syncwarp();
                        if (active) tma_load_5d(slot_base(sl) + lane * 2 * GROUP, isV ? &maps.v : &maps.k, bar_full(sl), 0, 0, 0, page * 2, kh + hd);
                    }
                }
                if (!ok) break;
            }
        } else if (warp == 1) {
            // ------------------------------------------------------------------ MMA issuer
            if (elect_one()) {
                constexpr uint32_t idesc_s = make_idesc(128, CB_KT, false);
                constexpr uint32_t idesc_o = make_idesc(128, D, true);
                uint32_t uq = 0, turn0 = 0, c_p[2] = {0u, 0u}, c_q1 = 0;     // (every unit has a first query tile, some a second one)
                while ((ok = mbar_wait(bar_ufull(uq % kUnitRing), (uq / kUnitRing) & 1, s_abort, p.status))) {
                    const volatile ChunkUnit* u = &s_units[uq % kUnitRing];
                    const int nrt = u->nrt;
                    if (nrt == 0) break;
                    const bool two = nrt == 2, heads = nrt == kTwoHeads;
                    const int nt = heads ? 2 * u->tiles : u->t1 - u->t0;          // key tiles that come through the ring
                    const uint32_t seq0 = (uint32_t)u->seq0;
                    const int nt0 = nt - u->skip;             // tiles of the first chain
                    if (!(ok = mbar_wait(bar_qfull(0), uq & 1, s_abort, p.status))) break;
                    // Turn e is tile e / 2 for chain e & 1 with two row tiles, else the e-th tile for chain e & 1.  Its S goes out behind the P V of NSB turns before,
                    // whose buffer it takes.  A tile that the first chain leaves out is a turn of nobody's; with three buffers, which
                    // go by the count of turns, it is none, and the last turn is the second chain's whatever its number.
                    const int skip = nt - nt0, turns = two ? 2 * nt - (C::NSB == 3 ? skip : 0) : nt;
                    auto chain_of = [&](int e) { return C::NSB == 3 && skip && e == turns - 1 ? 1 : e & 1; };
                    auto tile_of = [&](int e) { return two ? (C::NSB == 3 && skip && e == turns - 1 ? nt - 1 : e >> 1) : e; };
                    for (int e = 0; e < turns + C::NSB; ++e) {
                        const int ev = e - C::NSB;
                        if (ev >= 0) {
                            const int l = chain_of(ev), iv = tile_of(ev);
                            if (!two || l == 1 || iv < nt0) {
                                const uint32_t vseq = seq0 + 2u * (uint32_t)iv + 1u, vs = vseq % ns;
                                if ((!two || l == 0 || iv >= nt0) && !(ok = mbar_wait(bar_full(vs), (vseq / ns) & 1, s_abort, p.status))) break;
                                // the unit before is done with this chain's accumulator; a chain without a tile of this unit takes its turn
                                // on the barrier here too
                                if (ev < 2 && uq > 0 && !(ok = mbar_wait(bar_ofree(l), (uq - 1) & 1, s_abort, p.status))) break;
                                if (turns < 2 && uq > 0 && !(ok = mbar_wait(bar_ofree(1), (uq - 1) & 1, s_abort, p.status))) break;
                                const int k = C::NSB == 3 ? (int)((turn0 + (uint32_t)ev) % 3u) : l;
                                const uint32_t parity = C::NSB == 3 ? ((turn0 + (uint32_t)ev) / 3u) & 1u : c_p[l]++ & 1u;
                                const uint32_t vdesc = desc_lo(slot_base(vs), 1024), o_at = tmem + C::O_COL + l * D, p_at = tmem + k * 128;
                                if (!(ok = mbar_wait(bar_pready(k), parity, s_abort, p.status))) break;
                                tc_fence_after();
                                mma_pv_halves_block<D>(o_at, p_at, vdesc, idesc_o, ev < 2 ? 0u : 1u);
                                if (!two || l == 1) tc_commit(bar_free(vs));
                                if (C::NSB == 3) tc_commit(bar_pvdone(k));
                                if (iv >= (two && l == 0 ? nt0 : nt) - (heads ? 2 : 1)) tc_commit(two || heads ? bar_odone(l) : bar_odone_both);
                            }
                        }
                        if (e < turns) {
                            const int l = chain_of(e), ik = tile_of(e);
                            if (!two || l == 1 || ik < nt0) {
                                const uint32_t kseq = seq0 + 2u * (uint32_t)ik, ks = kseq % ns;
                                if (!two || l == 0 || ik >= nt0) {
                                    if (!(ok = mbar_wait(bar_full(ks), (kseq / ns) & 1, s_abort, p.status))) break;
                                    tc_fence_after();
                                }
                                if (nrt > 1 && e == 1) {
                                    if (!(ok = mbar_wait(bar_qfull(1), c_q1++ & 1, s_abort, p.status))) break;
                                    tc_fence_after();
                                }
                                const int k = C::NSB == 3 ? (int)((turn0 + (uint32_t)e) % 3u) : l;
                                mma_s_grouped_block<D>(tmem + k * 128, desc_lo(sbase + C::OFF_Q + (nrt > 1 ? l : 0) * C::Q_BYTES, 16), desc_lo(slot_base(ks), 16), idesc_s);
                                tc_commit(bar_sfull(k));
                                if (!two || l == 1) tc_commit(bar_free(ks));
                                if (ik >= (two && l == 0 ? nt0 : nt) - (heads ? 2 : 1)) tc_commit(bar_qfree(nrt > 1 ? l : 0));
                            }
                        }
                    }
                    turn0 += (uint32_t)turns;
                    if (!ok) break;
                    ++uq;
                }
            }
        } else {
            // ------------------------------------------------------------------ units for all roles, query tiles
            // The set of tickets that this launch counts in; the other one is cleared below, for the next launch (see cb_attn_tc.cu).
            uint32_t turn;
            asm volatile("ld.volatile.global.u32 %0, [%1];" : "=r"(turn) : "l"(p.part_turn));
            const int ticket_set = (int)(turn & 1u) * CB_ATTN_TICKETS;
            int error = 0, seq = 0;
            uint32_t uq = 0;
            // What all roles need of a unit; a shared one's holder of the first tile and number of CTAs are set before.
            auto publish = [&](const CbChunkUnit& x, const CbChunkShape& s, bool heads) {
                volatile ChunkUnit* u = &s_units[uq % kUnitRing];
                const int tiles = s.tiles(x.rg), nrt = s.two_rows(x.rg) ? 2 : (heads ? kTwoHeads : 1);
                u->b = x.b; u->kh = x.kh; u->rg = x.rg; u->t0 = x.t0; u->t1 = x.t1; u->tiles = tiles; u->nrt = nrt;
                u->row0 = s.row0; u->n = s.n; u->ctx = s.ctx; u->end = s.end(x.rg);
                u->seq0 = seq;
                u->skip = nrt == 2 && x.t1 == tiles && x.t1 - x.t0 > 1 && (tiles - 1) * CB_KT >= s.ctx + (2 * x.rg + 1) * p.NPT;
                u->dirty = max((s.end(x.rg) + 15) / 16 * 16 - (s.ctx + s.n), 0);
                seq += (heads ? 4 : 2) * (x.t1 - x.t0);
                mbar_arrive(bar_ufull(uq % kUnitRing));
            };
            // A unit's query tiles, each when the one before it there has been read; the next unit's are asked into L2 as soon as it is known.
            uint32_t n_q1 = 0;
            auto query_box = [&](const CbChunkUnit& x, const CbChunkShape& s, bool heads, int k, int db, bool ahead) {
                const int c0 = db * 64, c1 = (x.kh + (heads ? k : 0)) * p.G, c2 = s.row0 + (2 * x.rg + (heads ? 0 : k)) * p.NPT;
                if (ahead) asm volatile("cp.async.bulk.prefetch.tensor.4d.L2.global.tile [%0, {%1, %2, %3, %4}];" ::"l"(&maps.q), "r"(c0), "r"(c1), "r"(c2), "r"(0) : "memory");
                else tma_load_4d(sbase + C::OFF_Q + k * C::Q_BYTES + db * (CB_MT * 128), &maps.q, bar_qfull(k), c0, c1, c2, 0);
            };
            auto load_queries = [&](const CbChunkUnit& x, const CbChunkShape& s, bool heads) {
                const int nrt = s.two_rows(x.rg) || heads ? 2 : 1;
                if (uq > 0)
                    for (int k = 0; k < nrt; ++k)
                        for (int db = 0; db < C::DB; ++db) query_box(x, s, heads, k, db, true);
                for (int k = 0; k < nrt; ++k) {
                    const uint32_t before = k == 0 ? uq : n_q1;
                    if (before > 0 && !(ok = mbar_wait(bar_qfree(k), (before - 1) & 1, s_abort, p.status))) return;
                    mbar_expect_tx(bar_qfull(k), (uint32_t)(C::DB * RT * 128));
                    for (int db = 0; db < C::DB; ++db) query_box(x, s, heads, k, db, false);
                    if (k == 1) ++n_q1;
                }
            };
            CbChunkUnit x;
            if (p.cs > 0) {
                CbChunkShape s;
                int np = 0;
                const int cf = unit * p.cs;
                const bool has = cb_chunk_share(p, seq_b, unit - seq_b * p.Hkv, cta - cf, &x, &s, &np);
                error = s.error;
                if (lane == 0 && has) {
                    volatile ChunkUnit* u = &s_units[0];
                    u->cf = cf; u->np = np; u->xpos = -1; u->ticket = ticket_set + cf * 16;
                    publish(x, s, false);
                    load_queries(x, s, false);
                    ++uq;
                }
            } else {
                CbChunkWalker wk;
                CbChunkCuts cuts;
                cb_chunk_range(p, cta, lane, &wk, &cuts, &error);
                if (cta > 0) error = 0;
                if (lane == 0) {
                    *s_tot = cuts.total;
                    bool heads = false;
                    while (ok && wk.next_pair(p, &x, &heads)) {
                        const CbChunkShape& s = wk.s;         // of the unit's sequence: the walker goes on when it is asked again
                        const int tiles = s.tiles(x.rg), wt = s.wt(x.rg);
                        if (!(x.t0 == 0 && x.t1 == tiles)) {
                            // Shared with other CTAs: who holds its first tile, and how many there are (with ranges of at least one tile's positions the
                            // CTAs from the first tile's to the last one's; shorter ranges hold the deciding position of one tile at most).
                            volatile ChunkUnit* u = &s_units[uq % kUnitRing];
                            const int cf = cuts.of(x.first);
                            const bool wide = cuts.total >= (long long)p.nc * wt;
                            u->cf = cf;
                            u->np = wide ? cuts.of(x.first + (long long)(tiles - 1) * wt) - cf + 1 : tiles;
                            u->xpos = wide ? -1 : (int)x.first;
                            u->wt = wt;
                            u->ticket = ticket_set + cf * 16;
                        }
                        publish(x, s, heads);
                        load_queries(x, s, heads);
                        if (!ok) break;
                        ++uq;
                    }
                }
            }
            if (lane == 0 && ok) {
                s_units[uq % kUnitRing].nrt = 0;
                mbar_arrive(bar_ufull(uq % kUnitRing));
            }
            __syncwarp();
            for (int k = cta; k < p.nc; k += gridDim.x)       // a grid of few CTAs clears the others' too
                if (lane < 16) p.part_ticket[CB_ATTN_TICKETS - ticket_set + k * 16 + lane] = 0u;
            if (error) atomicCAS(p.status, 0u, (uint32_t)error);
        }
        __syncwarp();
    } else {
        // ---------------------------------------------------------------------- softmax / correction / epilogue
        reg_alloc<104>();
        const int sw = warp - 4, l = sw >> 3, hf = (sw >> 2) & 1;   // chain, half of the tile's keys
        const int wq = warp & 3;                              // TMEM lane quarter this warp may access
        const int row = wq * 32 + lane;
        auto token_of = [&](int r) { return (int)((uint32_t)r * p.g_inv >> 16); };   // r / G: a row is token * G + head of the group
        const uint32_t lane_addr = (uint32_t)(wq * 32) << 16;
        const int pair_id = 1 + l * 4 + wq;                   // named barrier of the two warps that share these rows
        constexpr int CW = D / 4;                             // accumulator columns handled at a time
        const bool out32 = (reinterpret_cast<uintptr_t>(p.out) & 31u) == 0;
        uint32_t c_s = 0, c_od = 0, c_ob = 0, uq = 0;         // completions consumed: S of this chain, o_done of this chain, o_done_both
        int turn0 = 0;                                        // three S buffers: turns of both chains in the units before, modulo 6
        // The pair's barrier; k numbers the barriers between two tiles, so that what a warp notes before it waits only grows.
        auto pair_sync = [&](bool v, uint32_t k) {
            if (lane == 0) s_pair[sw] = (int)(4u * (c_s + uq) + k);
            return pair_or(pair_id, v);
        };
        bool ok = true;
        for (; ok; ++uq) {
            if (!(ok = mbar_wait(bar_ufull(uq % kUnitRing), (uq / kUnitRing) & 1, s_abort, p.status))) break;
            const volatile ChunkUnit* u = &s_units[uq % kUnitRing];   // read again where it is needed: registers are short
            if (u->nrt == 0) break;
            const bool two = u->nrt > 1;                      // a chain has rows of its own: a row tile, or a head's only one
            const int first = (2 * u->rg + (u->nrt == 2 ? l : 0)) * p.NPT;   // its first token
            const int step = two ? 1 : 2, tfirst = u->t0 + (two ? 0 : l);
            const int t1 = u->t1 - (l == 0 ? u->skip : 0);
            const int nfull = (u->ctx + first + 1) / CB_KT;   // tiles that all its rows see whole
            const int token = first + token_of(row);
            const bool row_valid = row < RT && token < u->n;
            const bool warp_active = (wq * 32) < RT && first + token_of(wq * 32) < u->n;   // row 0 of the warp is valid
            const int limit = u->ctx + token + 1;             // keys that this row sees
            const uint32_t tm_O = tmem + C::O_COL + l * D + lane_addr;
            // the tile in whose last page there are slots behind the sequence's last token, for the warp that clears them
            const int unclean = u->dirty && hf == 0 && wq == 0 && (u->nrt != 2 || l == u->skip) ? u->tiles - 1 : -1;
            int sb = turn0 + l;                               // the chain's next turn, every second one, modulo 6: buffer and phase
            if (sb >= 6) sb -= 6;
            const int last_out = two && l == 1 && u->skip ? t1 - 1 : -1;   // but for a last tile that the first chain leaves out
            float m_used = -INFINITY, lsum = 0.f;
            for (int i = tfirst; i < t1; i += step) {
                // this turn's S buffer, by the issuer's count of turns
                int k = l;
                uint32_t parity = c_s & 1;
                if constexpr (C::NSB == 3) {
                    if (i == last_out) sb = sb == 0 ? 5 : sb - 1;
                    k = sb >= 3 ? sb - 3 : sb;
                    parity = sb >= 3;
                    sb = sb >= 4 ? sb - 4 : sb + 2;           // the chain's next turn
                }
                const uint32_t ts = tmem + k * 128 + lane_addr, tsh = ts + 64 * hf;
                if (!(ok = mbar_wait(bar_sfull(k), parity, s_abort, p.status))) break;
                ++c_s;
                if (warp_active) {
                    tc_fence_after();
                    const bool all_vis = i < nfull;
                    uint32_t vm[2] = {0xFFFFFFFFu, 0xFFFFFFFFu}, vref = 0xFFFFFFFFu;
                    auto below = [&](int lo) { return lo >= 32 ? 0xFFFFFFFFu : (lo <= 0 ? 0u : ((1u << lo) - 1u)); };
                    if (!all_vis) {
                        const int kv = row_valid ? limit - i * CB_KT : 0;
                        vm[0] = below(kv - 64 * hf); vm[1] = below(kv - 64 * hf - 32); vref = below(kv);
                    }
                    // Single pass, tried first on every tile: P against the reference maximum in use, no row maximum taken.  While the half
                    // row's sum stays below 2^20 no score is more than 20 above the reference and the tile stands; above that (or not finite)
                    // in either half, the two passes below move the reference.  A share's first tile takes the largest of the row's first 32
                    // scores.
                    if (i == tfirst) {
                        uint32_t rf[32];
                        CB_TMEM_LD32(rf, 0, ts);
                        CB_TMEM_WAIT_LD32(rf);
                        if (!all_vis) {
#pragma unroll
                            for (int jx = 0; jx < 32; ++jx)
                                if (!((vref >> jx) & 1u)) rf[jx] = 0xFF800000u;
                        }
                        float c0 = -INFINITY, c1 = -INFINITY;
#pragma unroll
                        for (int jx = 0; jx < 32; jx += 4) {
                            c0 = fmax3(c0, __uint_as_float(rf[jx]), __uint_as_float(rf[jx + 1]));
                            c1 = fmax3(c1, __uint_as_float(rf[jx + 2]), __uint_as_float(rf[jx + 3]));
                        }
                        m_used = fmaxf(c0, c1) * p.scale_log2;   // -inf if the row sees none of them
                    }
                    uint32_t pk[32];
                    // P of this thread's 64 scores (packed into pk) against reference mu; returns their sum.  P is rounded to bf16, the type that its product with
                    // bf16 values takes on the tensor cores (half a step, 2^-8 of each at most, as in tree attention; as two bf16 terms it would double that product): the
                    // output's error against 64 bits is 2.1e-3 to 2.4e-3 instead of the 1.6e-3 that its own rounding makes.  The sum is of the unrounded fp32 values,
                    // so that lse keeps their accuracy.
                    auto make_p_of = [&](float mu, auto masked) {
                        constexpr bool MASKED = decltype(masked)::value;
                        const uint64_t scale2 = f2_pack(p.scale_log2, p.scale_log2), negmu2 = f2_pack(-mu, -mu);
                        uint64_t lsa = f2_pack(0.f, 0.f), lsb = f2_pack(0.f, 0.f);
                        uint32_t sa[32];
#pragma unroll
                        for (int c = 0; c < 4; ++c) {
                            uint32_t* cur = sa + 16 * (c & 1);
                            if ((c & 1) == 0) { CB_TMEM_LD32(sa, 0, tsh + 16 * c); CB_TMEM_WAIT_LD32(sa); }
                            if (MASKED) {
#pragma unroll
                                for (int jx = 0; jx < 16; ++jx)
                                    if (!((vm[c >> 1] >> ((c & 1) * 16 + jx)) & 1u)) cur[jx] = 0xFF800000u;
                            }
#pragma unroll
                            for (int q = 0; q < 8; ++q) {
                                const uint64_t x = f2_fma(f2_pack(__uint_as_float(cur[2 * q]), __uint_as_float(cur[2 * q + 1])), scale2, negmu2);
                                // (All by the exponential unit: with a share of them as polynomials on the FMA pipe, as tree attention has it, prompts of
                                // 64 dims took 8 to 10% longer, of 128 dims 0 to 1%.)
                                float p0, p1;
                                f2_unpack(x, p0, p1);
                                p0 = ex2(p0); p1 = ex2(p1);
                                if (q & 1) lsb = f2_add(lsb, f2_pack(p0, p1));
                                else lsa = f2_add(lsa, f2_pack(p0, p1));
                                pk[c * 8 + q] = pack_bf16(p0, p1);
                            }
                        }
                        float l0, l1, l2, l3;
                        f2_unpack(lsa, l0, l1);
                        f2_unpack(lsb, l2, l3);
                        return (l0 + l1) + (l2 + l3);
                    };
                    auto make_p = [&](float mu) {
                        return all_vis ? make_p_of(mu, std::false_type{}) : make_p_of(mu, std::true_type{});
                    };
                    float lt = make_p(m_used == -INFINITY ? 0.f : m_used);
                    if (pair_sync(row_valid && !(lt <= kRowSumLimit), 0)) {          // rows that do not exist hold anything: they never ask
                        // pass 1: the row's maximum over all its visible scores (both threads of the row take it)
                        const int kv = all_vis ? CB_KT : (row_valid ? limit - i * CB_KT : 0);
                        float mx = -INFINITY;
#pragma unroll 1
                        for (int c = 0; c < 4; ++c) {
                            uint32_t rf[32];
                            CB_TMEM_LD32(rf, 0, ts + 32 * c);
                            CB_TMEM_WAIT_LD32(rf);
                            const uint32_t va = below(kv - 32 * c);
#pragma unroll
                            for (int jx = 0; jx < 32; ++jx) mx = fmaxf(mx, ((va >> jx) & 1u) ? __uint_as_float(rf[jx]) : -INFINITY);
                        }
                        pair_sync(false, 1);                  // both have read S: either may write P over it now
                        const float mloc = mx * p.scale_log2;
                        // the reference stays until the maximum exceeds it by 2^8
                        const bool need = mloc > m_used + 8.0f;
                        const float alpha = need ? ex2(m_used - mloc) : 1.0f;
                        if (need) m_used = mloc;
                        if (i > tfirst && __any_sync(CB_FULL, need)) {
                            // O is complete up to the chain's previous tile, whose product went out before this S, or, with three buffers, behind it;
                            // each of the two threads rescales half of the columns
                            if constexpr (C::NSB == 3) {
                                const int prev = (sb + (i == last_out ? 3 : 2)) % 6;   // the chain's turn before, four before the next one in sb (three, out of step)
                                if (!(ok = mbar_wait(bar_pvdone(prev % 3), (uint32_t)(prev / 3), s_abort, p.status))) break;
                                tc_fence_after();
                            }
#pragma unroll 1
                            for (int c = 0; c < 2; ++c) {
                                uint32_t o[CW];
                                const uint32_t ta = tm_O + hf * (D / 2) + c * CW;
                                tmem_ld_w<CW>(o, ta);
#pragma unroll
                                for (int jx = 0; jx < CW; ++jx) o[jx] = __float_as_uint(__uint_as_float(o[jx]) * alpha);
                                tmem_st_w<CW>(o, ta);
                            }
                            tmem_wait_st();
                        }
                        lsum *= alpha;
                        lt = make_p(m_used == -INFINITY ? 0.f : m_used);          // pass 2
                    }
                    CB_TMEM_ST32(pk, 0, tsh);                 // the 64 scores become 32 columns of packed P at their start
                    lsum += lt;
                    tmem_wait_st();
                }
                if (i == unclean) {
                    // Zeros there before any product reads the tile; with two row tiles by the chain whose product comes first.
                    const uint32_t vseq = (uint32_t)u->seq0 + 2u * (uint32_t)(u->nrt == kTwoHeads ? 2 * i + l : i - u->t0) + 1u, vs = vseq % ns;
                    if (!(ok = mbar_wait(bar_full(vs), (vseq / ns) & 1, s_abort, p.status))) break;
                    const int r0 = u->ctx + u->n - i * CB_KT, pieces = u->dirty * (D / 8);
                    for (int k = lane; k < pieces; k += 32) {
                        const int r = r0 + k / (D / 8), c = k % (D / 8);
                        const uint32_t at = slot_base(vs) + (r >> 3) * (1024 * C::DB) + (c >> 3) * 1024 + (r & 7) * 128 + (c & 7) * 16;
                        asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(at), "r"(0) : "memory");
                    }
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar_pready(k));
            }
            if (!ok) break;
            // ---- epilogue of this unit's share
            const int t0 = u->t0, h = (u->kh + (u->nrt == kTwoHeads ? l : 0)) * p.G + row - token_of(row) * p.G;
            const bool whole = t0 == 0 && u->t1 == u->tiles;
            const size_t at_row = (size_t)(u->row0 + (row_valid ? token : 0)) * p.Hq + h;
            // this thread's columns of the output row, 16 at a time: half a row with two row tiles, a quarter with one
            int npc, c0;
            // a shared unit: how many parts of it are in memory already; the look overlaps the wait for the last product (launches of few units
            // count CTAs, below, not warps)
            const int np = whole ? 1 : u->np;
            uint32_t* const ticket = p.part_ticket + (np > 1 ? u->ticket : 0) + sw;
            uint32_t arrived = 0;
            if (np > 1 && p.cs == 0 && lane == 0) arrived = ld_acquire(ticket);
            float x_m, x_l, x_w0 = 1.f, x_w1 = 1.f;           // reference and sum; one row tile: weights of O0 and O1
            if (two) {
                if (!(ok = mbar_wait(bar_odone(l), c_od & 1, s_abort, p.status))) break;
                ++c_od;
                s_x[(l * 2 + hf) * CB_MT + row] = lsum;
                pair_sync(false, 2);
                x_l = lsum + s_x[(l * 2 + 1 - hf) * CB_MT + row];
                x_m = m_used;
                npc = CW / 8; c0 = hf * 2 * CW;
            } else {
                if (!(ok = mbar_wait(bar_odone_both, c_ob & 1, s_abort, p.status))) break;
                ++c_ob;
                s_x[(l * 2 + hf) * CB_MT + row] = lsum;
                pair_sync(false, 2);
                const float lrow = lsum + s_x[(l * 2 + 1 - hf) * CB_MT + row];
                pair_sync(false, 3);
                s_x[(l * 2 + hf) * CB_MT + row] = hf ? lrow : m_used;
                __syncwarp();
                if (lane == 0) mbar_arrive(bar_sums);
                if (!(ok = mbar_wait(bar_sums, (c_ob - 1) & 1, s_abort, p.status))) break;
                const float m0 = s_x[row], l0 = s_x[CB_MT + row], m1 = s_x[2 * CB_MT + row], l1 = s_x[3 * CB_MT + row];
                x_m = fmaxf(m0, m1);
                x_w0 = m0 == -INFINITY ? 0.f : ex2(m0 - x_m);
                x_w1 = m1 == -INFINITY ? 0.f : ex2(m1 - x_m);
                x_l = l0 * x_w0 + l1 * x_w1;
                npc = CW / 16; c0 = (l * 2 + hf) * CW;
            }
            tc_fence_after();
            if (warp_active) {
                __nv_bfloat16* op = p.out + at_row * D;
                const bool both = !two && u->t1 - t0 > 1;     // the second chain has an accumulator too
                // 16 of this thread's accumulator columns, relative to reference x_m; with one row tile both accumulators put together
                auto load_o = [&](float* o, int col) {
                    uint32_t* r = reinterpret_cast<uint32_t*>(o);
                    tmem_ld_w<16>(r, tmem + C::O_COL + (two ? l * D : 0) + lane_addr + col);
                    if (two) return;
#pragma unroll
                    for (int k = 0; k < 16; ++k) o[k] *= x_w0;
                    if (both) {
                        uint32_t o1[16];
                        tmem_ld_w<16>(o1, tmem + C::O_COL + D + lane_addr + col);
#pragma unroll
                        for (int k = 0; k < 16; ++k) o[k] = fmaf(__uint_as_float(o1[k]), x_w1, o[k]);
                    }
                };
                auto store_out = [&](const float* o, int col, float inv) {
                    if (!row_valid) return;
                    uint32_t w[8];
#pragma unroll
                    for (int k = 0; k < 8; ++k) w[k] = pack_bf16(o[2 * k] * inv, o[2 * k + 1] * inv);
                    if (out32) {
                        st_global_v8(op + col, w[0], w[1], w[2], w[3], w[4], w[5], w[6], w[7]);
                    } else {
                        *reinterpret_cast<uint4*>(op + col) = make_uint4(w[0], w[1], w[2], w[3]);
                        *reinterpret_cast<uint4*>(op + col + 8) = make_uint4(w[4], w[5], w[6], w[7]);
                    }
                };
                auto store_lse = [&](float mx, float sum) {
                    if (row_valid && c0 == 0 && p.lse) p.lse[at_row] = (mx + log2f(sum)) * 0.6931471805599453f;
                };
                if (!whole && p.cs > 0) {
                    // left in memory by rows, for all threads of the last CTA to put together (below)
                    float* const own = p.part + (size_t)cta * (CB_MT * (D + 4));
#pragma unroll 1
                    for (int e = 0; e < npc; ++e) {
                        float o[16];
                        load_o(o, c0 + 16 * e);
                        if (row_valid) {
#pragma unroll
                            for (int q = 0; q < 4; ++q)
                                *reinterpret_cast<float4*>(own + row * D + c0 + 16 * e + q * 4) = make_float4(o[q * 4], o[q * 4 + 1], o[q * 4 + 2], o[q * 4 + 3]);
                        }
                    }
                    if (row_valid && c0 == 0) *reinterpret_cast<float2*>(own + CB_MT * D + row * 2) = make_float2(x_m, x_l);
                } else if (whole) {
                    const float inv = x_l > 0.f ? 1.0f / x_l : 0.f;
#pragma unroll 1
                    for (int e = 0; e < npc; ++e) {
                        float o[16];
                        load_o(o, c0 + 16 * e);
                        store_out(o, c0 + 16 * e, inv);
                    }
                    store_lse(x_m, x_l);
                } else {
                    // A unit shared with other CTAs: the same warp of each has the same rows and columns.  All but the last to come leave
                    // their partial (unnormalised columns, reference and sum) in memory and count themselves; the last one reads the others', in
                    // the order of the CTAs whoever is last, and writes the output.  Nobody waits.
                    const int xpos = u->xpos, cf = u->cf;
                    auto slot_of = [&](int cc, bool start) { return p.part + (size_t)(2 * cc + (start ? 1 : 0)) * (2 * CB_MT * (D + 4)); };
                    auto part_of = [&](int k) { return slot_of(xpos < 0 ? cf + k : cb_cta_of(*s_tot, p.nc, (long long)xpos + k * u->wt), k == 0); };
                    const int wofs = sw * (2 * CW * 32) + lane * 4, mlofs = 2 * CB_MT * D + (sw * 32 + lane) * 2;
                    float* const own = slot_of(cta, t0 == 0);
                    auto load_part = [&](float4* v, const float* pp, int e) {
#pragma unroll
                        for (int q = 0; q < 4; ++q)
                            v[q] = row_valid ? __ldcg(reinterpret_cast<const float4*>(pp + wofs + (e * 4 + q) * 128)) : make_float4(0.f, 0.f, 0.f, 0.f);
                    };
                    auto load_ml = [&](const float* pp) { return row_valid ? __ldcg(reinterpret_cast<const float2*>(pp + mlofs)) : make_float2(-INFINITY, 0.f); };
                    auto weight = [](float m, float mx) { return m == -INFINITY ? 0.f : ex2(m - mx); };
                    bool last = __shfl_sync(CB_FULL, arrived, 0) == (uint32_t)(np - 1);
                    if (!last) {
#pragma unroll 1
                        for (int e = 0; e < npc; ++e) {
                            float o[16];
                            load_o(o, c0 + 16 * e);
                            if (row_valid) {                  // (a single token's unit has G rows of 128)
#pragma unroll
                                for (int q = 0; q < 4; ++q)
                                    *reinterpret_cast<float4*>(own + wofs + (e * 4 + q) * 128) = make_float4(o[q * 4], o[q * 4 + 1], o[q * 4 + 2], o[q * 4 + 3]);
                            }
                        }
                        if (row_valid) *reinterpret_cast<float2*>(own + mlofs) = make_float2(x_m, x_l);
                        __syncwarp();
                        if (lane == 0) arrived = atom_add_acq_rel(ticket, 1u);   // releases the whole warp's stores
                        last = __shfl_sync(CB_FULL, arrived, 0) == (uint32_t)(np - 1);
                    }
                    if (last) {
                        __syncwarp();
                        float mx = -INFINITY, sum = 0.f;
                        if (np == 2) {
                            // the usual case: one other part, its columns fetched a group ahead
                            const bool begins = t0 == 0;
                            const float* const po = part_of(begins ? 1 : 0);
                            float4 v[4], vn[4];
                            load_part(v, po, 0);
                            const float2 ml = load_ml(po);
                            mx = fmaxf(x_m, ml.x);
                            const float wo = weight(x_m, mx), wp = weight(ml.x, mx);
                            sum = begins ? fmaf(wp, ml.y, wo * x_l) : fmaf(wo, x_l, wp * ml.y);
                            const float inv = sum > 0.f ? 1.0f / sum : 0.f;
#pragma unroll 1
                            for (int e = 0; e < npc; ++e) {
                                float o[16];
                                if (e + 1 < npc) load_part(vn, po, e + 1);
                                load_o(o, c0 + 16 * e);
                                const float* vf = reinterpret_cast<const float*>(v);
#pragma unroll
                                for (int k = 0; k < 16; ++k) o[k] = begins ? fmaf(wp, vf[k], wo * o[k]) : fmaf(wo, o[k], wp * vf[k]);
                                store_out(o, c0 + 16 * e, inv);
#pragma unroll
                                for (int q = 0; q < 4; ++q) v[q] = vn[q];
                            }
                        } else {
                            // Many parts: two at a time are fetched, with their references, before either is used (one after the other, the last
                            // to come of six spent 14 k cycles here).
                            auto part2 = [&](int k, const float* pp, float2* ml) { *ml = k >= np ? make_float2(-INFINITY, 0.f) : (pp == own ? make_float2(x_m, x_l) : load_ml(pp)); };
#pragma unroll 1
                            for (int k = 0; k < np; k += 4) {
                                float2 ml[4];
#pragma unroll
                                for (int t = 0; t < 4; ++t) part2(k + t, part_of(min(k + t, np - 1)), &ml[t]);
#pragma unroll
                                for (int t = 0; t < 4; ++t) {
                                    const float mn = fmaxf(mx, ml[t].x);
                                    sum = fmaf(weight(ml[t].x, mn), ml[t].y, sum * weight(mx, mn));
                                    mx = mn;
                                }
                            }
                            const float inv = sum > 0.f ? 1.0f / sum : 0.f;
#pragma unroll 1
                            for (int e = 0; e < npc; ++e) {
                                float acc[16];
#pragma unroll
                                for (int k = 0; k < 16; ++k) acc[k] = 0.f;
#pragma unroll 1
                                for (int k = 0; k < np; k += 2) {
                                    const float* const pp[2] = {part_of(k), part_of(min(k + 1, np - 1))};
                                    float4 v[2][4];
                                    float2 ml[2];
#pragma unroll
                                    for (int t = 0; t < 2; ++t) {
                                        part2(k + t, pp[t], &ml[t]);
                                        if (pp[t] == own) load_o(reinterpret_cast<float*>(v[t]), c0 + 16 * e);
                                        else load_part(v[t], pp[t], e);
                                    }
#pragma unroll
                                    for (int t = 0; t < 2; ++t) {
                                        const float w = weight(ml[t].x, mx);
                                        const float* vf = reinterpret_cast<const float*>(v[t]);
#pragma unroll
                                        for (int q = 0; q < 16; ++q) acc[q] = fmaf(w, vf[q], acc[q]);
                                    }
                                }
                                store_out(acc, c0 + 16 * e, inv);
                            }
                        }
                        store_lse(mx, sum);
                    }
                }
            }
            if (!whole && p.cs > 0) {
                // The CTA's only unit, shared: all its rows are in memory (row sums' barrier, next phase), one thread counts the CTA in, and
                // the threads of the last CTA to come put the parts together, an output quad each, with all parts' loads under way at once.
                // Nobody waits for another CTA.  (A warp's columns by that warp, part after part, took the last CTA 13 k cycles at batch 1.)
                __syncwarp();
                if (lane == 0) mbar_arrive(bar_sums);
                if (!(ok = mbar_wait(bar_sums, 1, s_abort, p.status))) break;
                volatile int* const s_last = reinterpret_cast<volatile int*>(sgen + C::OFF_X);
                if (sw == 0 && lane == 0) *s_last = atom_add_acq_rel(p.part_ticket + u->ticket, 1u) == (uint32_t)(np - 1);   // releases what it saw stored
                if (lane == 0) mbar_arrive(bar_ofree(0));     // (nobody waits there for the accumulator of an only unit)
                if (!(ok = mbar_wait(bar_ofree(0), 0, s_abort, p.status))) break;
                if (*s_last) {
                    const float* const parts = p.part + (size_t)u->cf * (CB_MT * (D + 4));
                    const int quads = u->n * p.G * (D / 4);
                    for (int k = sw * 32 + lane; k < quads; k += 512) {
                        const int r = k / (D / 4), c = k % (D / 4) * 4, tk = token_of(r);
                        float mx = -INFINITY, sum = 0.f;
                        float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 1
                        for (int j0 = 0; j0 < np; j0 += 4) {
                            float2 ml[4];
                            float4 v[4];
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                const float* pp = parts + (size_t)min(j0 + j, np - 1) * (CB_MT * (D + 4));
                                ml[j] = __ldcg(reinterpret_cast<const float2*>(pp + CB_MT * D + r * 2));
                                v[j] = __ldcg(reinterpret_cast<const float4*>(pp + r * D + c));
                            }
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                if (j0 + j >= np) break;
                                const float mn = fmaxf(mx, ml[j].x);
                                const float wo = mx == -INFINITY ? 0.f : ex2(mx - mn), wp = ml[j].x == -INFINITY ? 0.f : ex2(ml[j].x - mn);
                                mx = mn;
                                sum = fmaf(wp, ml[j].y, wo * sum);
                                acc.x = fmaf(wp, v[j].x, wo * acc.x); acc.y = fmaf(wp, v[j].y, wo * acc.y);
                                acc.z = fmaf(wp, v[j].z, wo * acc.z); acc.w = fmaf(wp, v[j].w, wo * acc.w);
                            }
                        }
                        const float inv = sum > 0.f ? 1.0f / sum : 0.f;
                        const size_t at = (size_t)(u->row0 + tk) * p.Hq + u->kh * p.G + r - tk * p.G;
                        *reinterpret_cast<uint2*>(p.out + at * D + c) = make_uint2(pack_bf16(acc.x * inv, acc.y * inv), pack_bf16(acc.z * inv, acc.w * inv));
                        if (c == 0 && p.lse) p.lse[at] = (mx + log2f(sum)) * 0.6931471805599453f;
                    }
                }
                break;
            }
            if constexpr (C::NSB == 3) turn0 = (turn0 + (two ? 2 * (u->t1 - t0) - u->skip : u->t1 - t0)) % 6;
            tc_fence_before();
            __syncwarp();
            if (lane == 0) {                                  // 16 arrivals per unit either way
                if (two) mbar_arrive_n(bar_ofree(l), 2u);
                else { mbar_arrive(bar_ofree(0)); mbar_arrive(bar_ofree(1)); }
            }
        }
        if (!ok) {
            // The other warp of the pair may have entered a pair barrier that this one will not: answer for it until it has left too.
            // Its own waits end as well, so this does; the loop is bounded all the same.
            __syncwarp();
            int seen = __shfl_sync(CB_FULL, lane == 0 ? s_pair[sw] : 0, 0);
            if (lane == 0) { __threadfence_block(); s_pair[sw] = -1; }
            for (int k = 0; k < 1 << 16; ++k) {
                const int other = __shfl_sync(CB_FULL, lane == 0 ? s_pair[sw ^ 4] : 0, 0);
                if (other < 0) break;
                if (other > seen) { seen = other; pair_arrive(pair_id); }
                __nanosleep(200);
            }
        }
        __syncwarp();
    }

    // ---------------------------------------------------------------------- teardown
    if (*s_abort) {
        // give copies that are still in flight time to land before the shared memory is released
        for (int k = 0; k < 64; ++k) __nanosleep(1000);
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 1) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols) : "memory");
        // the last CTA to leave hands the turn on: nobody looks at this launch's tickets any more
        if (elect_one() && atomicInc(&p.part_turn[1], gridDim.x - 1u) == gridDim.x - 1u) atomicAdd(&p.part_turn[0], 1u);
    }
}

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                  const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiledFn get_encode() {
    static const EncodeTiledFn fn = [] {
        void* ptr = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &ptr, cudaEnableDefault, &q) != cudaSuccess || q != cudaDriverEntryPointSuccess) ptr = nullptr;
        return (EncodeTiledFn)ptr;
    }();
    return fn;
}

bool encode(CUtensorMap* m, const void* base, int rank, const cuuint64_t* dims, const cuuint64_t* strides, const cuuint32_t* box, int D) {
    const EncodeTiledFn enc = get_encode();
    if (!enc) { fprintf(stderr, "cacheback: cuTensorMapEncodeTiled entry point not found\n"); return false; }
    const cuuint32_t one[5] = {1, 1, 1, 1, 1};
    const CUresult r = enc(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, (cuuint32_t)rank, const_cast<void*>(base), dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
                           CU_TENSOR_MAP_SWIZZLE_128B, D >= 128 ? CU_TENSOR_MAP_L2_PROMOTION_L2_256B : CU_TENSOR_MAP_L2_PROMOTION_L2_128B,
                           CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) fprintf(stderr, "cacheback: tensor map encode failed (%d): rank %d, D %d, base %p\n", (int)r, rank, D, base);
    return r == CUDA_SUCCESS;
}
// The pool in the order (64 dims, row of 8, column block, group of 8 rows, head); a box is a page of a head.
bool encode_pool(CUtensorMap* m, const void* base, const CbChunkParams& p) {
    const cuuint64_t row = (cuuint64_t)p.Hkv * p.D * 2;       // bytes
    const cuuint64_t dims[5] = {64, 8, (cuuint64_t)(p.D / 64), (cuuint64_t)p.num_pages * 2, (cuuint64_t)p.Hkv}, strides[4] = {row, 128, 8 * row, (cuuint64_t)p.D * 2};
    const cuuint32_t box[5] = {64, 8, (cuuint32_t)(p.D / 64), 2, 1};
    return encode(m, base, 5, dims, strides, box, p.D);
}
// Queries [rows, heads, D] as (dim, head, row, 1); a box is 64 dims of a row tile: G heads of NPT tokens.
bool encode_queries(CUtensorMap* m, const CbChunkParams& p) {
    const cuuint64_t row = (cuuint64_t)p.Hq * p.D * 2;
    const cuuint64_t dims[4] = {(cuuint64_t)p.D, (cuuint64_t)p.Hq, (cuuint64_t)p.n_rows, 1}, strides[3] = {(cuuint64_t)p.D * 2, row, row * p.n_rows};
    const cuuint32_t box[4] = {64, (cuuint32_t)p.G, (cuuint32_t)p.NPT, 1};
    return encode(m, p.q, 4, dims, strides, box, p.D);
}

constexpr int kMaxDevices = 64;
std::mutex g_mutex;
bool g_smem_set[2][kMaxDevices];

template <int D>
cb_status launch(const CbChunkParams& p, const ChunkMaps& maps, cudaStream_t st, int device) {
    {
        // the opt-in to large dynamic shared memory is a function attribute of each device
        std::lock_guard<std::mutex> lock(g_mutex);
        const bool known = device >= 0 && device < kMaxDevices;
        if (!known || !g_smem_set[D == 128][device]) {
            CB_CUDA(cudaFuncSetAttribute(cb_chunk_tc_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)Cfg<D>::SMEM));
            if (known) g_smem_set[D == 128][device] = true;
        }
    }
    CB_CUDA(cb_launch_pdl(cb_chunk_tc_kernel<D>, dim3(p.cs > 0 ? p.B * p.Hkv * p.cs : p.nc), dim3(kThreads), Cfg<D>::SMEM, st, p, maps));
    cb_count_launch(1);
    return CB_OK;
}

}  // namespace

cb_status cb_chunk_launch_tensor(cb_ctx* ctx, const CbChunkParams& given, cudaStream_t st) {
    CbChunkParams p = given;
    if (p.P != 16 || p.num_pages >= 1 << 29) return CB_ERR_UNSUPPORTED;   // (a page's coordinate is twice its number)
    p.NPT = CB_MT / p.G;
    p.g_inv = 65536u / (uint32_t)p.G + 1u;
    p.one = p.max_chunk <= p.NPT;
    p.nc = ctx->num_sms < CB_ATTN_MAX_CTAS ? ctx->num_sms : CB_ATTN_MAX_CTAS;
    CbAttnParams w = {};
    w.D = p.D;
    cb_attn_weights(w);
    p.w1 = w.w1; p.w2 = w.w2; p.d1 = w.d1; p.d2 = w.d2;
    p.cs = p.one ? cb_chunk_pick_share((long long)p.B * p.Hkv, ((long long)p.max_keys + CB_KT - 1) / CB_KT, p.nc) : 0;
    p.cs_inv = p.cs > 1 ? 0xFFFFFFFFu / (uint32_t)p.cs + 1u : 0u;      // exact for numerators below 2^16 (__umulhi); a divisor of 1 is set aside
    p.hkv_inv = p.Hkv > 1 ? 0xFFFFFFFFu / (uint32_t)p.Hkv + 1u : 0u;
    p.part = ctx->d_attn_part; p.part_ticket = ctx->d_attn_ticket; p.part_turn = ctx->d_attn_turn;
    ChunkMaps maps;
    if (!encode_pool(&maps.k, p.k_pool, p) || !encode_pool(&maps.v, p.v_pool, p) || !encode_queries(&maps.q, p)) return CB_ERR_CUDA;
    return p.D == 128 ? launch<128>(p, maps, st, ctx->device) : launch<64>(p, maps, st, ctx->device);
}
