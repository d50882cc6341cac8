// Attention of chunks of new tokens over the paged 16-bit cache (include/eas_paged.h): sequences with many rows, a row
// being one query of one head.
//
// A workgroup owns 128 or 256 rows of one (sequence, key / value head), a wave 32 of them: queries and the heads of
// their group side by side, so that a chunk of few tokens fills a wave, and tokens that stand in LDS serve the whole
// group.  The walk over the tokens is prompt attention's (attention_tiles.h); what differs is where a tile comes from:
// its 64 tokens lie in one to four pages.  A DMA instruction moves 4 or 8 tokens, which no page's border parts, so its
// page is one scalar; the page numbers of a tile are one load, a tile ahead of the DMA that goes by them, and their
// addresses one vector computation (each by itself in scalars: 4,096 tokens over 32,768 2,105 us, so 1,982).  Tokens of
// pages that are not held are masked like those behind a query's own; their DMA reads zeros, as a weight of 0 does not hide
// an infinity or a NaN, and a page of the cache would be another sequence's.
//
// Bound by the matrix units, 4 * head_dim flops for each visible (row, token) pair: 4,096 tokens of 28 heads over 4 behind
// 32,768, 2,044 GFLOP, take 1,830 - 1,920 us, 1,064 - 1,117 TFLOP/s (prompt attention over the same rows 1,914), the units
// 51% busy at 2.0 GHz: 448 workgroups on 256 CUs leave an eighth of the time to half of them.  Chunks of 512 to 1,024
// tokens over up to 6,001 beside single tokens, 88 GFLOP, 132 us: the longest walk, 48 tiles, and the join.
#pragma once

#include "attention_tiles.h"
#include "paged_ops.h"

namespace eas {

// One workgroup's work, number `block` of tile_workgroups(a.items, kv_heads, kv_heads); smem: keys x 2, values x 2
template <class T, int HD, int NW>
__device__ __forceinline__ void many_rows(const Kv16AttnArgs& a, int block, char* smem) {
  using C = Cfg<HD, NW>;
  typedef typename Mfma<T>::x8 x8;
  const unsigned lds0 = (unsigned)(size_t)(__attribute__((address_space(3))) char*)smem;

  const int group = a.heads / a.c.kv_heads;
  int kvh, item;
  place(block, a.c.kv_heads, a.c.kv_heads, &kvh, &item);
  if (item >= a.items) return;
  const auto count = [&](const Seq& s) {
    const long rows = (long)s.nq * group;
    return takes_few(a, s) ? 0 : (int)((rows + C::QT - 1) / C::QT) * many_runs(s.len, rows, a.c.kv_heads);
  };
  Items<decltype(count)> items(a, count);
  if (item >= items.all()) return;
  Seq s;
  const int r = items.find(&item, &s);
  const int rows = s.nq * group;
  const int runs = many_runs(s.len, rows, a.c.kv_heads), run = item % runs;
  const int tile = (rows + C::QT - 1) / C::QT - 1 - item / runs;   // the last rows, which see most, first
  const int tid = threadIdx.x, lane = tid & 63, g = lane >> 5, l32 = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int rw = tile * C::QT + wave * 32;

  // this lane's row, and tokens that rows see: the lane's, the wave's fewest and most, the workgroup's most
  const auto query = [&](int row) { return (int)((unsigned)min(row, rows - 1) / (unsigned)group); };
  const auto head_of = [&](int row, int i) { return kvh * group + min(row, rows - 1) - i * group; };
  const int sees = seen_by(a, s, query(rw + l32)), fewest = seen_by(a, s, query(rw));
  const int most = rw < rows ? seen_by(a, s, query(rw + 31)) : 0;
  // token tiles of the workgroup, from tb on those of the run, and of these the wave's
  const int all = (seen_by(a, s, query((tile + 1) * C::QT - 1)) + KT - 1) / KT, each = many_run_tiles(s.len, runs);
  const int tb = run * each;
  const int nt = max(0, min(each, all - tb)), nt_w = max(0, min(nt, (most + KT - 1) / KT - tb));

  x8 qf[C::KS];
  {
    const int i = query(rw + l32);
    const T* qp = static_cast<const T*>(a.q) + (s.row0 + i) * a.qs.row + head_of(rw + l32, i) * a.qs.head;
#pragma unroll
    for (int ks = 0; ks < C::KS; ++ks) qf[ks] = *reinterpret_cast<const x8*>(qp + ks * 16 + g * 8);
  }

  // A tile's DMA: instruction n = wave + NW j fills LDS slots 64 n + lane; slot i is chunk i % R of row i / R.  Its rows
  // lie in one part of 16 tokens, part part0 + j * PARTS, from row part_row on.
  constexpr int ROWS = 64 / C::R, PARTS = NW * ROWS / 16;
  const int part0 = wave * ROWS / 16, part_row = wave * ROWS % 16 + lane / C::R;
  const int dcol = C::logical(wave * ROWS + lane / C::R, lane % C::R) * 16;   // of all j: it goes by row % 16
  const int last = s.len - 1;
  const int* table = a.pages + (long)r * a.max_pages;
  // lane p has part p % 4 of a tile: its first token -- the last one where it lies behind it -- and that one's page
  const auto token_of = [&](int t) { return min((tb + t) * KT + 16 * (lane & 3), last); };
  const auto pages_of = [&](int t) { return table[token_of(t) >> a.c.page_shift]; };
  const auto held_parts = [&](int pages) { return (int)(__ballot(held_page(a, pages)) & 15); };
  // bytes before the part's first token in the cache
  const auto offset_of = [&](int t, int pages) { return token_offset(a, pages, kvh, token_of(t), HD) * 2; };
  const auto fetch = [&](const void* base, int t, long offset, int held, int lds_off) {
    const uint64_t from = (uint64_t)(uintptr_t)base + offset;
    const int lo = (int)from, hi = (int)(from >> 32);
    const auto go = [&](int j, unsigned voff, auto whole) {
      const int part = part0 + j * PARTS;
      const uint32_t at[2] = {(uint32_t)__builtin_amdgcn_readlane(lo, part), (uint32_t)__builtin_amdgcn_readlane(hi, part)};
      const void* tokens = (const void*)(uintptr_t)(at[0] | (uint64_t)at[1] << 32);
      if (!decltype(whole)::value && !(held >> part & 1)) tokens = absent_tokens;
      dma16<true>(lds0 + lds_off + (wave + NW * j) * 1024, voff, tokens);
    };
    if ((tb + t + 1) * KT <= s.len && held == 15) {
#pragma unroll
      for (int j = 0; j < C::NDMA; ++j) go(j, part_row * (HD * 2) + dcol, std::integral_constant<bool, true>{});
    } else {   // rows behind the last token read it again
#pragma unroll
      for (int j = 0; j < C::NDMA; ++j)
        go(j, min(part_row, max(last - ((tb + t) * KT + 16 * (part0 + j * PARTS)), 0)) * (HD * 2) + dcol,
           std::integral_constant<bool, false>{});
    }
  };
  const auto fetch_k = [&](int t, long offset, int held) { fetch(a.c.k, t, offset, held, (t & 1) * C::TILE); };
  const auto fetch_v = [&](int t, long offset, int held) { fetch(a.c.v, t, offset, held, (2 + (t & 1)) * C::TILE); };

  TileWalk<T, HD, NW> walk(smem, qf, a.scale_log2);
  constexpr std::integral_constant<bool, true> yes{};
  constexpr std::integral_constant<bool, false> no{};
  // Waits until the wave's own DMA has landed and its LDS reads are done, and for the other waves to be as far.  One
  // asm: no read may move up between the wait and the barrier.  Every wave passes it once a tile, from whichever of
  // the loops below it is in.
  const auto meet = [] { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory"); };
  int pages = 0;                           // of tile t + 2
  long offset = 0;                         // of tile t + 1
  int parts = 0, parts1 = 0, parts2 = 0;   // which of the parts of tiles t, t + 1 and t + 2 are held
  const auto arrive = [&](int t) {
    meet();   // keys t + 1 and values t are there, keys t and values t - 1 read by all
    asm volatile("" : "+v"(pages));   // so are the page numbers: taken here, as a wait behind the DMA would be for it, too
    const long next = offset_of(t + 2, pages);
    parts = parts1, parts1 = parts2, parts2 = held_parts(pages);
    if (t + 1 < nt) fetch_v(t + 1, offset, parts1);
    if (t + 2 < nt) fetch_k(t + 2, next, parts2);
    offset = next;
    pages = pages_of(t + 3);
  };
  const auto hidden = [&](int t) {   // of tile t's weights
    int upto[4];
#pragma unroll
    for (int p = 0; p < 4; ++p) upto[p] = (parts >> p & 1 ? sees : 0) - (tb + t) * KT;
    return [=](int v) { return key_of(v, g) >= upto[(v >> 4) * 2 + (v & 15) / 8]; };
  };
  if (nt > 0) {
    f32x16 sa[2], sb[2];
    const int pages0 = pages_of(0), pages1 = pages_of(1);
    pages = pages_of(2);
    parts1 = held_parts(pages0), parts2 = held_parts(pages1);   // of tiles 0 and 1
    const long offset0 = offset_of(0, pages0);
    offset = offset_of(1, pages1);
    fetch_k(0, offset0, parts1);
    fetch_v(0, offset0, parts1);
    if (nt > 1) fetch_k(1, offset, parts2);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    // the queries are taken here, so that no wait for them is left to the loop, where it would wait for a tile
#pragma unroll
    for (int ks = 0; ks < C::KS; ++ks) asm volatile("" ::"v"(qf[ks]));
    meet();
    int t = 0;
    if (nt_w > 0) {
      walk.scores(0, sa);
      // tiles that all the wave's queries see whole, in pairs, up to a page that is not held; those at the border, or
      // from that page on; the last one
      for (const int whole = min(fewest / KT - tb, nt_w - 1); t + 2 <= whole && (parts1 & parts2) == 15; t += 2) {
        arrive(t);
        walk.step(t, sa, sb, hidden(t), no, yes);
        arrive(t + 1);
        walk.step(t + 1, sb, sa, hidden(t + 1), no, yes);
      }
      for (; t + 1 < nt_w; ++t) {
        arrive(t);
        walk.step(t, sa, sb, hidden(t), yes, yes);
        sa[0] = sb[0];
        sa[1] = sb[1];
      }
      arrive(t);
      walk.step(t, sa, sb, hidden(t), yes, no);
      ++t;
    }
    for (; t < nt; ++t) arrive(t);
  }

  // every wave is past its last read
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __syncthreads();
  int row0 = rw;
  asm("" : "+s"(row0));   // rows' queries and heads are taken anew: no register holds them over the walk
  if (row0 >= rows) return;
  const int ri = row0 + l32, qi = query(ri);
  char* stage = smem + wave * 32 * HD * 2;
  f32x16* o = walk.o;
  float m = walk.m, l = walk.l, lift = 1.0f;
  if (any_not_finite<C::HB>(o)) {
    lift = careful_lift<T>;
    const auto page_of = [&](int i) { return table[i >> a.c.page_shift]; };
    careful_rows<T, HD>(
        qf, [&](long i) { return static_cast<const T*>(a.c.k) + token_offset(a, page_of((int)i), kvh, (int)i, HD); },
        [&](long i) { return static_cast<const T*>(a.c.v) + token_offset(a, page_of((int)i), kvh, (int)i, HD); },
        [&](int i) { return i >= sees || !held_page(a, page_of(i)); },
        [&](int t) {
          bool whole = (t + 1) * KT <= fewest;
          for (int p = 0; p < 4; ++p) whole = whole && held_page(a, page_of(t * KT + 16 * p));
          return whole;
        },
        s.len, tb, tb + nt_w, a.scale_log2, stage, o, &m, &l);
  }
  l += __shfl_xor(l, 32, 64);
  const float inv = l == 0.0f ? 0.0f : 1.0f / l, lse2 = l == 0.0f ? -INFINITY : m + __log2f(l * lift);
  if (runs > 1) {
    const long slot = first_slot(a, s, r) + ((long)run * a.c.kv_heads + kvh) * rows + ri;   // a wave's are consecutive
    if (ri < rows) {
#pragma unroll
      for (int hb = 0; hb < C::HB; ++hb)
#pragma unroll
        for (int e = 0; e < 16; e += 4)
          *reinterpret_cast<float4*>(a.part + slot * HD + hb * 32 + e * 2 + g * 4) =
              make_float4(o[hb][e] * inv, o[hb][e + 1] * inv, o[hb][e + 2] * inv, o[hb][e + 3] * inv);
      if (g == 0) a.part_lse[slot] = lse2;
    }
    return;
  }
  if (a.lse && g == 0 && ri < rows) a.lse[(s.row0 + qi) * a.heads + head_of(ri, qi)] = lse2 * kLn2;
  // the tiles' memory stages each wave's 32 x HD results, chunks of row r rotated by r, so that the stores are of
  // whole rows
#pragma unroll
  for (int hb = 0; hb < C::HB; ++hb)
#pragma unroll
    for (int e4 = 0; e4 < 4; ++e4) {
      union { uint2 u; T e[4]; } st;
#pragma unroll
      for (int e = 0; e < 4; ++e) st.e[e] = (T)(o[hb][e4 * 4 + e] * inv);
      *reinterpret_cast<uint2*>(stage + l32 * HD * 2 + (hb * 4 + e4 + l32) % C::R * 16 + g * 8) = st.u;
    }
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
  for (int k = 0; k < C::R / 2; ++k) {
    const int c = lane + 64 * k, row = c / C::R, ch = c % C::R, i = query(row0 + row);
    const uint4 x = *reinterpret_cast<const uint4*>(stage + row * HD * 2 + (ch + row) % C::R * 16);
    if (row0 + row < rows)
      *reinterpret_cast<uint4*>(static_cast<T*>(a.out) + (s.row0 + i) * a.os.row + head_of(row0 + row, i) * a.os.head +
                                ch * 8) = x;
  }
}

// Row tiles of all sequences, and their runs: a bound of what many_rows() has to do.  A sequence that comes here has more
// than FEW_ROWS rows, but for one that the rows' beginning cuts, and one that their end does; one that is split has at most
// MANY_FILL workgroups, whatever its heads.
template <int HD, int NW>
inline int64_t many_items(const Kv16AttnArgs& a) {
  constexpr int QT = Cfg<HD, NW>::QT;
  const int64_t rows = (int64_t)a.n_rows * (a.heads / a.c.kv_heads), by_rows = rows / (FEW_ROWS + 1) + 2;
  const int64_t some = a.n_seqs < a.n_rows ? a.n_seqs : a.n_rows, seqs = some < by_rows ? some : by_rows;
  const int64_t tiles = (rows + QT - 1) / QT + seqs, runs = many_runs(a.max_len, 1, a.c.kv_heads);
  const int64_t split = tiles + seqs * (MANY_FILL / a.c.kv_heads);
  return runs == 1 ? tiles : tiles * runs < split ? tiles * runs : split;
}

}  // namespace eas
