// Host-side plan of a dilated-attention forward call (see plan.h).
#include "plan.h"

#include <algorithm>
#include <cmath>
#include <cstring>

namespace da {

FastDiv make_fastdiv(uint32_t d) {
  FastDiv f;
  f.d = d;
  uint32_t l = 0;
  while ((uint64_t{1} << l) < d) ++l;           // l = ceil(log2 d)
  f.shift = 31 + l;
  const uint64_t num = uint64_t{1} << f.shift;  // 2^(31+l) <= 2^62
  f.mul = static_cast<uint32_t>((num + d - 1) / d);
  return f;
}

int block_m_for(int dtype) { return dtype == DA_BF16 ? 128 : 64; }

namespace {

constexpr uint64_t kAlign = 256;

uint64_t align_up(uint64_t x) { return (x + kAlign - 1) / kAlign * kAlign; }

}  // namespace

int make_plan(int64_t B, int64_t N, int64_t H, int64_t D, const da_pattern_t* patterns,
              int64_t num_patterns, int64_t causal, int64_t dtype, float softmax_scale,
              Plan* out) {
  if (!patterns || !out) return DA_EINVAL;
  if (B < 1 || N < 1 || H < 1 || D < 1) return DA_EINVAL;
  if (N + H >= (int64_t{1} << 31) || H >= (int64_t{1} << 16) || B >= (int64_t{1} << 31))
    return DA_EINVAL;
  if (num_patterns < 1 || num_patterns > DA_MAX_PATTERNS) return DA_EINVAL;
  if (!(softmax_scale >= 0.0f) || std::isinf(softmax_scale)) return DA_EINVAL;
  if (causal != 0 && causal != 1) return DA_EINVAL;
  for (int64_t i = 0; i < num_patterns; ++i) {
    const int64_t w = patterns[i].w, r = patterns[i].r;
    if (w < 1 || r < 1 || r > w) return DA_EINVAL;
  }
  if (dtype != DA_F32 && dtype != DA_BF16) return DA_EUNSUPPORTED;
  if (D != 32 && D != 64 && D != 128) return DA_EUNSUPPORTED;
  // every row offset ((b*N + p)*H + h) must fit in 63 bits with room to spare
  if (static_cast<double>(B) * N * H * D > 4.0e18) return DA_EINVAL;

  Plan p;
  std::memset(&p, 0, sizeof(p));
  p.B = B;
  p.N = N;
  p.H = H;
  p.D = D;
  p.causal = static_cast<int>(causal);
  p.dtype = static_cast<int>(dtype);
  p.scale = softmax_scale > 0.0f ? softmax_scale : static_cast<float>(1.0 / std::sqrt(double(D)));
  p.npat = static_cast<int>(num_patterns);
  p.block_m = block_m_for(p.dtype);
  const int64_t esize = dtype == DA_BF16 ? 2 : 4;
  // Per-pattern output rows are kept as fp16 for bf16 inputs, each row divided
  // by a power of two that brings its largest magnitude into [2^14, 2^15)
  // (fp16's eleven significant bits with bf16's exponent range), and as fp32
  // for fp32 inputs.  Each row has an 8-byte record: its lse and its scale.
  const int64_t ws_esize = dtype == DA_BF16 ? 2 : 4;
  constexpr int64_t kRecBytes = 8;

  uint64_t ws = 0;
  int64_t items = 0;
  long double pairs = 0.0L;
  int64_t covered = 0;
  for (int i = 0; i < p.npat; ++i) {
    PatternPlan& pp = p.pat[i];
    pp.w = patterns[i].w < N ? patterns[i].w : N;
    // A dilation beyond N + H keeps exactly the rows it would keep at N + H:
    // every head's offset is its own index and each segment keeps one row.
    pp.r = patterns[i].r < N + H ? patterns[i].r : N + H;
    pp.nseg = (N + pp.w - 1) / pp.w;
    pp.lmax = (pp.w + pp.r - 1) / pp.r;
    pp.ntiles = (pp.lmax + p.block_m - 1) / p.block_m;
    pp.units = B * H * pp.nseg;
    pp.item_begin = items;
    items += pp.units * pp.ntiles;
    const uint64_t rows = static_cast<uint64_t>(pp.units) * static_cast<uint64_t>(pp.lmax);
    pp.o_off = ws;
    ws = align_up(ws + rows * static_cast<uint64_t>(D) * ws_esize);
    pp.lse_off = ws;
    ws = align_up(ws + rows * kRecBytes);

    // exact kept rows and unmasked pairs: full segments, then the short tail
    const int64_t nfull = N / pp.w;
    const int64_t tail = N - nfull * pp.w;
    const int64_t nres = pp.r < H ? pp.r : H;  // offsets actually used by heads
    for (int64_t s = 0; s < nres; ++s) {
      const int64_t heads = H / pp.r + (s < H % pp.r ? 1 : 0);  // heads with h mod r == s
      const int64_t Lf = kept_rows(pp.w, s, pp.r);
      const int64_t Lt = tail > 0 ? kept_rows(tail, s, pp.r) : 0;
      covered += B * heads * (nfull * Lf + Lt);
      const long double pf = causal ? 0.5L * Lf * (Lf + 1) : (long double)Lf * Lf;
      const long double pt = causal ? 0.5L * Lt * (Lt + 1) : (long double)Lt * Lt;
      pairs += (long double)B * heads * (nfull * pf + pt);
    }
  }
  int64_t launch = 0;
  for (int i = 0; i < p.npat; ++i) launch += (p.pat[i].units + 7) / 8 * p.pat[i].ntiles;
  launch *= 8;
  if (items >= (int64_t{1} << 31) || launch >= (int64_t{1} << 31)) return DA_EINVAL;
  p.launch_items = launch;
  // A key tile of the attention kernel spans at most 128 kept rows, each r*H*D
  // elements after the previous one; 32-bit byte offsets inside a tile (plus
  // one row) must stay below 2^31.
  p.offsets32 = true;
  for (int i = 0; i < p.npat; ++i)
    if (static_cast<double>(p.pat[i].r) * H * D * esize * 129.0 >= 2147483648.0) p.offsets32 = false;
  // the combine stage launches one workgroup per 8..32 positions of each (b, h)
  if ((N + 7) / 8 * B * H >= (int64_t{1} << 31)) return DA_EINVAL;
  p.total_items = items;
  p.workspace_bytes = ws;
  p.covered_rows = covered;
  p.sparse_flops = static_cast<double>(4.0L * D * pairs);
  p.bytes_attn = static_cast<double>(covered) * (3.0 * D * esize + D * ws_esize + kRecBytes);
  p.bytes_combine = static_cast<double>(covered) * (D * ws_esize + kRecBytes) +
                    static_cast<double>(B) * N * H * (D * esize + 4.0);
  *out = p;
  return DA_OK;
}

int make_bwd_layout(const Plan& p, BwdLayout* out) {
  if (!out) return DA_EINVAL;
  if (p.dtype != DA_BF16) return DA_EUNSUPPORTED;
  // 32-bit offsets inside a tile of 64 kept rows (rows r*H*D elements apart,
  // and the rows' per-row scalars r floats apart)
  if (!p.offsets32) return DA_EUNSUPPORTED;
  for (int i = 0; i < p.npat; ++i)
    if (static_cast<double>(p.pat[i].r) * 4.0 * 65.0 >= 2147483648.0) return DA_EUNSUPPORTED;
  BwdLayout l;
  std::memset(&l, 0, sizeof(l));
  const uint64_t rows_all = static_cast<uint64_t>(p.B) * p.N * p.H;
  uint64_t ws = 0;
  l.nl2_off = ws;
  ws = align_up(ws + rows_all * 4);
  l.nd_off = ws;
  ws = align_up(ws + rows_all * 4);
  const uint64_t chunks = static_cast<uint64_t>(grad_chunks(p.D));
  for (int i = 0; i < p.npat; ++i) {
    const uint64_t rows = static_cast<uint64_t>(p.pat[i].units) * static_cast<uint64_t>(p.pat[i].lmax);
    const uint64_t bytes = rows * static_cast<uint64_t>(p.D) * 2;  // fp16 rows
    const uint64_t rec = rows * chunks * 4;                           // float scales
    l.dq_off[i] = ws;
    ws = align_up(ws + bytes);
    l.dk_off[i] = ws;
    ws = align_up(ws + bytes);
    l.dv_off[i] = ws;
    ws = align_up(ws + bytes);
    l.dq_rec_off[i] = ws;
    ws = align_up(ws + rec);
    l.dk_rec_off[i] = ws;
    ws = align_up(ws + rec);
    l.dv_rec_off[i] = ws;
    ws = align_up(ws + rec);
  }
  l.workspace_bytes = ws;
  const double D = static_cast<double>(p.D), es = 2.0, cov = static_cast<double>(p.covered_rows);
  const double grad_row = D * 2.0 + 4.0 * static_cast<double>(chunks);  // a compact row and its scales
  l.flops = 2.5 * p.sparse_flops;
  l.delta_pass = true;
  for (int i = 0; i < p.npat; ++i)
    if (p.pat[i].r == 1) l.delta_pass = false;
  // each gradient kernel reads the kept q, k, v, dout rows once and the two
  // per-row scalars; dq writes one compact row, dk/dv two.  Without a delta
  // pass dq reads the kept out rows and lse in place of the scalars, and
  // writes these once for every row.
  l.bytes_grad = cov * (2.0 * (4.0 * D * es + 8.0) + 3.0 * grad_row);
  if (!l.delta_pass) l.bytes_grad += cov * (D * es + 4.0 - 8.0) + static_cast<double>(rows_all) * 8.0;
  // sum: the compact gradients read, dq, dk, dv written; delta: out, dout and
  // lse of every row read, two scalars written
  l.bytes_combine = static_cast<double>(rows_all) * 3.0 * D * es + cov * 3.0 * grad_row;
  if (l.delta_pass) l.bytes_combine += static_cast<double>(rows_all) * (2.0 * D * es + 4.0 + 8.0);
  *out = l;
  return DA_OK;
}

int make_paged_plan(int64_t T, int64_t B, int64_t H, int64_t Hkv, int64_t D, int64_t num_pages, int64_t page,
                    int64_t max_pages, int64_t max_new, const da_pattern_t* patterns, int64_t num_patterns,
                    int64_t dtype, float softmax_scale, PagedPlan* out) {
  constexpr int64_t kMost = int64_t{1} << 31;
  if (!patterns || !out) return DA_EINVAL;
  if (T < 0 || T >= kMost || B < 1 || B > kPagedMost || H < 1 || H >= (int64_t{1} << 16) || Hkv < 1 || H % Hkv)
    return DA_EINVAL;
  if (page < 1 || page > (int64_t{1} << 16) || (page & (page - 1)) || max_pages < 1 || max_pages > kPagedMost / page ||
      num_pages < 1 || num_pages > (int64_t{1} << 32) / page / Hkv || num_pages >= kMost || max_new < 0)
    return DA_EINVAL;
  if (num_patterns < 1 || num_patterns > DA_MAX_PATTERNS) return DA_EINVAL;
  if (!(softmax_scale >= 0.0f) || std::isinf(softmax_scale)) return DA_EINVAL;
  for (int64_t i = 0; i < num_patterns; ++i)
    if (patterns[i].w < 1 || patterns[i].r < 1 || patterns[i].r > patterns[i].w) return DA_EINVAL;
  if (dtype != DA_F32 && dtype != DA_BF16) return DA_EUNSUPPORTED;
  if (D != 32 && D != 64 && D != 128) return DA_EUNSUPPORTED;

  PagedPlan p;
  std::memset(&p, 0, sizeof(p));
  p.T = T; p.B = B; p.H = H; p.Hkv = Hkv; p.D = D;
  p.num_pages = num_pages; p.page = page; p.max_pages = max_pages;
  p.dtype = static_cast<int>(dtype);
  while ((int64_t{1} << p.page_log2) < page) ++p.page_log2;
  p.npat = static_cast<int>(num_patterns);
  p.full = -1;
  p.scale = softmax_scale > 0.0f ? softmax_scale : static_cast<float>(1.0 / std::sqrt(double(D)));
  const int64_t reach = max_pages * page;  // positions that the table holds
  // The patterns whose rows see the most keys come first, of equal ones those of
  // longer segments (more of whose rows are far from their segment's begin): the
  // launch begins with its longest items.
  da_pattern_t sorted[DA_MAX_PATTERNS];
  std::copy(patterns, patterns + num_patterns, sorted);
  std::stable_sort(sorted, sorted + num_patterns, [reach](const da_pattern_t& x, const da_pattern_t& y) {
    const int64_t wx = std::min(x.w, reach), wy = std::min(y.w, reach);
    const int64_t kx = (wx - 1) / x.r, ky = (wy - 1) / y.r;
    return kx != ky ? kx > ky : wx > wy;
  });
  patterns = sorted;
  p.all_few = dtype == DA_F32 || std::min(max_new, T) <= kPagedFew;
  p.few = p.all_few ? T : B == 1 ? 0 : kPagedFew;
  p.singles = std::min(T, p.all_few ? T : B * p.few);
  // A single token's workgroups for one split: key heads with a kept query head,
  // in blocks of kPagedGroupRows query heads (float32: query heads).  A token
  // belongs to the heads of one residue mod r.
  const int64_t G = dtype == DA_F32 ? 1 : H / Hkv, key_heads = H / G;
  auto one_heads = [&](int64_t r) {
    if (r >= G) return std::min(key_heads, (H + r - 1) / r);
    return key_heads * (((G + r - 1) / r + kPagedGroupRows - 1) / kPagedGroupRows);
  };
  // Workgroups with work, of the tokens by themselves and of the tiles.  Beside
  // tiles the tokens are taken to be one of each sequence.
  const int64_t tokens = p.all_few ? p.singles : std::min(T, B);
  double one_busy = 0.0, tile_busy = 0.0;
  for (int i = 0; i < p.npat; ++i) {
    one_busy += static_cast<double>(tokens) * one_heads(patterns[i].r);
    tile_busy += H * std::ceil(double(T) / patterns[i].r / kPagedRows);
  }
  // Splits of a token's keys: until there are about four workgroups for each
  // place on the chip (768), half as many beside tiles.  More cost a start-up each
  // (64 tokens of 1000 to 32767 cached: 72 us at 2 splits, 83 at 4), fewer leave
  // the longest ones alone at the end (32 tokens of up to 30000, heads of 128: 102
  // us at 24, 113 at 12).
  const double one_target = p.all_few ? 3072.0 : 1536.0;
  // A tile's keys are split until there are 2048 workgroups, and not below this
  // many of the pattern's longest rows: an item's start-up is as long as ten key
  // tiles.  (At 512, 768, 1024: 1000 new tokens among 15 single ones 38, 34.9, 33
  // us, 1024 at 20000 35.3, 33.8, 32.7, 512 at 31500 28.2, 28.1, 28.9; 128 at 32000,
  // whose launch leaves most of the chip idle, 21.0, 22.3, 25.6.)
  const int64_t tile_least = tile_busy < 64.0 ? 512 : 768;
  int64_t one_items = 0, expected = 0;
  int64_t items = 0;
  for (int i = 0; i < p.npat; ++i) {
    PagedPattern& t = p.pat[i];
    t.w = static_cast<int32_t>(std::min(patterns[i].w, reach));
    // a dilation beyond the table's reach keeps one row of a segment, whatever it is
    t.r = static_cast<int32_t>(std::min(patterns[i].r, kMost - 1));
    t.fw = make_fastdiv(static_cast<uint32_t>(t.w));
    t.fr = make_fastdiv(static_cast<uint32_t>(t.r));
    if (t.r == 1 && (p.full < 0 || t.w > p.pat[p.full].w)) p.full = i;
    const int64_t keys = (t.w + int64_t{t.r} - 1) / t.r;  // of a row, at most
    const int64_t one = std::max<int64_t>(
        1, std::min({static_cast<int64_t>(one_target / std::max(1.0, one_busy) + 0.5), (keys + 255) / 256, int64_t{64}}));
    t.one_split = make_fastdiv(static_cast<uint32_t>(one));
    t.one_slot = static_cast<int32_t>(p.one_slots);
    p.one_slots += one;
    t.one_heads = make_fastdiv(static_cast<uint32_t>(one_heads(patterns[i].r)));
    if (one_items >= kMost) return DA_EINVAL;
    t.one_begin = static_cast<int32_t>(one_items);
    one_items += (p.singles * one_heads(patterns[i].r) + 7) / 8 * 8 * one;  // units XCD by XCD
    if (p.all_few) continue;
    const int64_t ts = std::max<int64_t>(
        1, std::min({static_cast<int64_t>(2048.0 / std::max(1.0, tile_busy)), (keys + tile_least - 1) / tile_least, int64_t{16}}));
    t.tile_split = make_fastdiv(static_cast<uint32_t>(ts));
    t.tile_slot = static_cast<int32_t>(p.tile_slots);
    p.tile_slots += ts;
    // A sequence of n tokens touches at most (n - 1) / w + 2 segments, and m
    // positions of one fill m / (128 r) tiles, rounded up.  (One sequence of 512
    // tokens, the paper's patterns: 14 tiles a head where 9 are there; with 27
    // the workgroups without work held up the others.)  Units are dealt to the
    // XCDs: up to 16 tiles, fewer where there would not be eight units each.  (At most
    // 1, 4, 16, 64 tiles: 2048 tokens at 30000, dense, 253, 251, 248, 250 us, 4096 at
    // 28672 64.5, 64.6, 65.6, 65.6, 8192 dense 141, 141, 147, 148.  Two units each, eight,
    // 32: 270, 248, 256 us; 68.8, 65.6, 64.7; 146, 147, 140.)
    const int64_t some = std::min(B, T), segments = (T - some) / t.w + 2 * some, fill = int64_t{t.r} * kPagedRows;
    const int64_t tiles = std::min(T, segments + (T - segments) / fill);
    if (tiles >= kMost / H / ts) return DA_EINVAL;
    const int64_t run = std::max<int64_t>(1, std::min<int64_t>(16, tiles * H / 64));
    if (items >= kMost) return DA_EINVAL;
    t.tiles = static_cast<int32_t>(tiles);
    t.run = static_cast<int32_t>(run);
    t.tile_begin = static_cast<int32_t>(items);
    items += ((tiles + run - 1) / run * H + 7) / 8 * 8 * run * ts;
    expected += (T / (int64_t{t.r} * kPagedRows) + 2) * H * ts + std::min(T, B) * one_heads(patterns[i].r) * one;
  }
  // (the device's own count of a launch that steps rounds its units of fewer tiles up by less than 16 each)
  if (one_items >= kMost || one_items + items + 16 * H * p.tile_slots >= kMost || (T + 1) * H >= kMost) return DA_EINVAL;
  p.one_items = one_items;
  p.tile_items = items;
  // Where the sizes allow more than one and a half times as many items as they let
  // expect, the launch is as large as the latter.  (Every item that the sizes allow
  // against that, at 1.5 times as many: two prompts of 8192 160 us, 167; 1.7: four
  // chunks of 4096 162, 166; 2.3: two chunks of 300 30.4, 29.0, three of 2000 85.5, 86.7;
  // 4.7: 16 sequences with 1000 new tokens of one 43.5, 33.1; 10: 64 with 2048 127, 87.)
  const int64_t likely = std::max<int64_t>(1024, expected);
  p.steps = !p.all_few && 2 * (one_items + items) > 3 * likely;
  p.grid = p.steps ? (likely + 7) / 8 * 8 : one_items + items;
  uint64_t off = 0;
  auto take = [&off](uint64_t bytes) {
    const uint64_t at = off;
    off = align_up(off + bytes);
    return at;
  };
  const uint64_t one_rows = static_cast<uint64_t>(p.singles * H * p.one_slots);
  const uint64_t tile_rows = static_cast<uint64_t>(p.T * H * p.tile_slots);
  p.one_rec_off = take(one_rows * 4);
  p.one_row_off = take(one_rows * D * 4);
  p.tile_rec_off = take(tile_rows * 8);
  p.tile_row_off = take(tile_rows * D * 2);
  p.workspace_bytes = off;
  *out = p;
  return DA_OK;
}

int make_weight_plan(int64_t T, int64_t B, int64_t H, int64_t Hkv, int64_t D, int64_t num_pages, int64_t page,
                     int64_t max_pages, int64_t max_new, const da_pattern_t* patterns, int64_t num_patterns,
                     int64_t dtype, float softmax_scale, WeightPlan* out) {
  constexpr int64_t kMost = int64_t{1} << 31;
  if (!out || max_new < 0) return DA_EINVAL;
  PagedPlan base;  // the same sizes and patterns are valid
  if (const int rc = make_paged_plan(T, B, H, Hkv, D, num_pages, page, max_pages, 1, patterns, num_patterns, dtype,
                                     softmax_scale, &base);
      rc != DA_OK)
    return rc;
  if ((T + 32) * H >= kMost) return DA_EINVAL;  // a unit's columns are counted in blocks of 16 tokens
  WeightPlan p;
  std::memset(&p, 0, sizeof(p));
  p.T = T; p.B = B; p.H = H; p.Hkv = Hkv; p.D = D;
  p.num_pages = num_pages; p.page = page; p.max_pages = max_pages;
  p.dtype = base.dtype;
  p.page_log2 = base.page_log2;
  p.npat = base.npat;
  p.scale = base.scale;
  // A token by itself reads its keys again: fine where most sequences have one, which is
  // taken for granted of as many tokens as sequences, unless the caller knows of more.
  // (64 new tokens of one sequence of 20000 among 63 without: 48 us as a sequence's,
  // 225 as tokens; four 44 and 23.)
  p.lone = T <= B && max_new <= kPagedFew;
  p.rows = p.lone ? T : B;
  const int64_t G = H / Hkv, reach = max_pages * page;
  auto units = [&](int64_t r) {
    if (!p.lone) return Hkv * std::min(G, r);
    return r >= G ? std::min(Hkv, (H + r - 1) / r) : Hkv;
  };
  // A sequence's columns are dealt out until a wave has about eight times sixteen.
  // (512 tokens at 31500, 16 heads over four: 33 us; four times sixteen 39, sixteen
  // times 35.)
  auto columns = [&](int64_t r) { return T / r * ((G + std::min(G, r) - 1) / std::min(G, r)); };
  auto shares = [&](int64_t r) {
    return p.lone ? 1 : std::max<int64_t>(1, std::min<int64_t>(8, columns(r) / 512));
  };
  int64_t sums = 0;  // in lines of kWeightAlign
  double busy = 0.0;
  for (int i = 0; i < p.npat; ++i)
    busy += static_cast<double>(p.rows) * units(base.pat[i].r) * shares(base.pat[i].r);
  for (int i = 0; i < p.npat; ++i) {
    PagedPattern& t = p.pat[i];
    t = base.pat[i];
    t.tile_split = make_fastdiv(static_cast<uint32_t>(shares(t.r)));
    const int64_t n = units(t.r) * shares(t.r);
    // the positions that a row's keys can lie in, and their pages
    const int64_t span = std::min(reach, p.lone ? int64_t{t.w} : t.w + T);
    const int64_t pages = std::min(max_pages, span / page + 2);
    const int64_t keys = (span + t.r - 1) / t.r;
    const int64_t least = (pages + kWeightPages - 1) / kWeightPages;
    // A round of keys an item: 64 a wave, or 64 that the waves share.  (64 tokens at 1K
    // to 32K: 33.0 us with 2048 workgroups or 1024, 34.3 with 4096 of 128 keys; the 512
    // tokens 33 with 4096 or 2048, and with keys of their own for up to 128, 256, 512
    // columns 33.2, 32.5, 41.7.)
    const int64_t round = p.lone || columns(t.r) <= kWeightApart ? 256 : 64;
    const int64_t some = static_cast<int64_t>((p.lone ? 2048.0 : 4096.0) / std::max(1.0, busy) + 0.5);
    const int64_t splits = std::max({least, int64_t{1}, std::min({some, (keys + round - 1) / round, pages})});
    if (splits >= kMost || p.rows * n >= kMost - 8) return DA_EINVAL;
    t.one_split = make_fastdiv(static_cast<uint32_t>(splits));
    t.one_heads = make_fastdiv(static_cast<uint32_t>(n));
    t.one_begin = static_cast<int32_t>(p.items);
    // in lines: of a row that begins within one, no more than those of the table
    const int64_t lines = std::min((pages - 1) / kWeightAlign + 2, (max_pages - 1) / kWeightAlign + 1);
    if (sums >= kMost || lines > (int64_t{1} << 56) / std::max<int64_t>(1, p.rows * n)) return DA_EINVAL;
    t.one_slot = static_cast<int32_t>(sums);
    t.tiles = static_cast<int32_t>(lines * kWeightAlign);
    sums += p.rows * n * lines;
    const int64_t padded = (p.rows * n + 7) / 8 * 8;  // units XCD by XCD
    if (padded > 0 && splits > (kMost - 1 - p.items) / padded) return DA_EINVAL;
    p.items += padded * splits;
  }
  p.workspace_bytes = static_cast<uint64_t>(sums) * kWeightAlign * 4;
  *out = p;
  return DA_OK;
}

}  // namespace da
