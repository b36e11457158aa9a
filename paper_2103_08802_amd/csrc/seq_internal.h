// Internal declarations of the sequence operators (pnn_seq.h): launchers called by the entry points
// (seq.hip) once the arguments are checked, and the sizes both sides use.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "pnn_seq.h"

namespace pnn {

inline int64_t cdiv64(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline int64_t round256(int64_t v) { return (v + 255) / 256 * 256; }

// ---- embedding ----
constexpr int EMB_DIGIT = 9;           // bits of a radix pass
constexpr int EMB_BINS = 1 << EMB_DIGIT;
constexpr int EMB_ITEMS = 2048;        // tokens of a sorting workgroup
constexpr int EMB_DIRECT = 64;         // sorting workgroups up to which each sums the others' histograms itself
constexpr int64_t EMB_CLEAR = 32 << 20;  // bytes of the gradient a launch of the sort clears on the side
// Sorted positions of a summing tile: 32, fewer while the tiles (of up to 256 pieces of 8 columns) are under 1024
// workgroups.
inline int embed_run(int64_t n, int64_t width) {
  int run = 32;
  while (run > 8 && cdiv64(n, run) * cdiv64(width, 2048) < 1024) run /= 2;
  return run;
}
// tokens outside the table sort as key = vocab, behind all others
inline int embed_passes(int64_t vocab) {
  int bits = 0;
  while (bits < 32 && (vocab >> bits) != 0) ++bits;
  return (bits + EMB_DIGIT - 1) / EMB_DIGIT;
}
// Workspace of the gradient: keys and positions twice (the radix passes go from one to the other),
// a pass's histogram [workgroup][bin] and its sums over the workgroups, a bit for every table row, and the partial rows [tile][2][width] of runs that
// cross tiles.
struct EmbedWs {
  int64_t key[2], pos[2], hist, total, present, part, bytes;
  int64_t blocks, tiles, words;
  int passes, run;
};
inline EmbedWs embed_ws(const pnn_embed_desc& d) {
  EmbedWs w;
  w.blocks = cdiv64(d.n, EMB_ITEMS);
  w.run = embed_run(d.n, d.width);
  w.tiles = cdiv64(d.n, w.run);
  w.words = cdiv64(d.vocab, 32);
  w.passes = embed_passes(d.vocab);
  int64_t o = 0;
  for (int i = 0; i < 2; ++i) {
    w.key[i] = o;
    o += round256(d.n * 4);
    w.pos[i] = o;
    o += round256(d.n * 4);
  }
  w.hist = o;
  o += round256(w.blocks * EMB_BINS * 4);
  w.total = o;
  o += EMB_BINS * 4;
  w.present = o;
  o += round256(w.words * 4);
  w.part = o;
  o += round256(w.tiles * 2 * d.width * 4);
  w.bytes = o;
  return w;
}
int launch_embed_fwd(const pnn_embed_desc& d, const void* table, const void* tokens, void* out, hipStream_t s);
int launch_embed_bwd(const pnn_embed_desc& d, const void* dout, const void* tokens, float* dtable, int accumulate,
                     void* ws, hipStream_t s);

// ---- recurrence ----
constexpr int SCAN_FS = 16, SCAN_BS = 8;   // steps of a wave in a tile, forward and backward
constexpr int SCAN_NW = 16;                // waves of a tile of a long sequence
constexpr int SCAN_CHUNK = 8 * SCAN_BS;         // steps from one kept state to the next: the shorter tiles of the backward
constexpr int64_t SCAN_WGS = 256;          // workgroups that fill the device (one of 16 waves a CU)
struct ScanArgs {
  const void *x, *gate;
  const int32_t* lengths;
  const float* h0;
  void* h;
  float* hT;
  float* states;       // [batch][chunks][channels]: the state each chunk starts from
  const void* dh;
  const float* dhT;
  void *dx, *dgate;
  float* dh0;
  void* ws;
};
inline int64_t scan_chunks(const pnn_scan_desc& d) { return cdiv64(d.length, SCAN_CHUNK); }
// Waves of a tile: as many as the sequence has work for; 8, of which a CU holds two workgroups, where there are two
// workgroups a CU.
inline int scan_waves(int64_t chains, int64_t length, int steps) {
  if (length <= steps) return 1;
  if (length <= 4 * steps) return 4;
  return length <= 8 * steps || chains >= 2 * SCAN_WGS ? 8 : SCAN_NW;
}
// Workgroups a sequence's tiles are dealt to, given the channel groups of the whole batch: as many as fill the device.
// Two tiles already pay (4 x 512 steps of 512 channels, backward: 12 us against 21 by one workgroup after the other).
inline int scan_dealt(int64_t chains, int64_t tiles) {
  const int64_t w = chains > 0 ? SCAN_WGS / chains : 1;
  return (int)(w < 2 || tiles < 2 ? 1 : w < tiles ? w : tiles);
}
// Whether a lane takes two neighbouring bf16 channels: where that still fills the device.  Otherwise one, which makes
// twice the workgroups, unless even those are too few: the forward, whose dealt tiles cost more than its bytes, then
// takes pairs again (65536 steps of 1024 channels: 104 us against 119; backward 253 against 202).
inline bool scan_pairs(const pnn_scan_desc& d, bool backward) {
  if (d.dtype != PNN_BF16 || d.channels <= 64) return false;
  return d.batch * cdiv64(d.channels, 128) >= SCAN_WGS || (!backward && d.batch * cdiv64(d.channels, 64) < SCAN_WGS);
}
// Channels [first, end) of a channel group, 64 lanes of vec channels.  Groups share none, so that a state may stand in
// place (hT = h0, dh0 = dhT): one group's workgroups may end before the next one's read theirs.  Of an odd number of
// channels the last two lanes' pairs meet in a channel, so where the last group had only one, it takes the pair before
// from its neighbour too (vec = 2 has more than 64 channels, hence two groups there).
struct ScanGroup {
  int first, end;
};
__host__ __device__ inline ScanGroup scan_group(int channels, int group, int vec) {
  const int size = 64 * vec, full = (group + 1) * size;
  ScanGroup r = {group * size, full < channels ? full : channels};
  if (vec == 2 && channels % size == 1) {
    if (r.end == channels) r.first -= 2;
    else if (full == channels - 1) r.end -= 2;
  }
  return r;
}
// Workspace of dealt tiles: tickets, first states, the tiles' (A, B) (64 vec pairs each)
struct ScanWs {
  int64_t tickets, first, sum, bytes;
};
inline ScanWs scan_ws(int64_t states, int64_t chains, int64_t tiles, int vec) {
  ScanWs w;
  w.tickets = 0;
  w.first = round256(chains * 4);
  w.sum = w.first + round256(states * 4);
  w.bytes = w.sum + round256(chains * tiles * 64 * vec * 8);
  return w;
}
// enough for both directions and both widths of a channel group; 0 when no sequence is dealt
inline int64_t scan_ws_bytes(const pnn_scan_desc& d) {
  int64_t most = 0;
  for (int vec = 1; vec <= 2; ++vec)
    for (int steps = SCAN_BS; steps <= SCAN_FS; steps += SCAN_FS - SCAN_BS) {
      const int64_t chains = d.batch * cdiv64(d.channels, 64 * vec), tiles = cdiv64(d.length, SCAN_NW * steps);
      if (scan_dealt(chains, tiles) < 2) continue;
      const int64_t bytes = scan_ws(d.batch * d.channels, chains, tiles, vec).bytes;
      if (bytes > most) most = bytes;
    }
  return most;
}
int launch_scan_fwd(const pnn_scan_desc& d, const ScanArgs& a, hipStream_t s);
int launch_scan_bwd(const pnn_scan_desc& d, const ScanArgs& a, hipStream_t s);

// ---- distillation ----
int launch_distill(const pnn_distill_desc& d, const void* logits, const int32_t* index, const void* teacher,
                   const int32_t* labels, const float* weight, float* loss, void* dlogits, hipStream_t s);

// ---- linear attention ----
constexpr int LIN_MAX_WIDTH = PNN_LINATTN_MAX_WIDTH;
constexpr int LIN_CHUNK = 32;              // steps of a chunk
constexpr int64_t LIN_FEW = 256, LIN_MANY = 512;  // workgroups below which sequences are cut, and to how many
// How the sums of a direction run: widths summed over padded to `pad`, workgroups of as many waves with 16 value columns
// each, segments of a sequence (of four chunks at least; the two launches before the last cost a third of it).  One
// shape for all three sums of the backward, which run side by side in a launch.  Measured, us: 128 heads x 2048 steps
// (128 and 384 workgroups) 296, with 512 in the place of 256 350, of 128 336, with 384 or 768 in the place of 512 310;
// 30 heads x 777 steps with eight chunks to a segment 140, with four 111.  Four waves to a workgroup: 128 heads x 2048
// steps 273, with eight 294.
struct LinShape {
  int pad, waves, tiny, segments, seg_chunks;
};
// Where a lane's first 16-byte piece of a tile of rows is: `pieces` to a row, `ve` elements each, `width` elements of a row
// from the tile's first column to the row's end, which may be behind the tile's.  The piece that the row's end cuts is
// moved back to end there, in front of the tile's columns if need be: a row is at least a piece long.  Lanes with nothing
// to load (behind the row's end; behind the tile's `rows`) load the row's first piece, likewise, and store it behind
// the tile's columns.
struct LinPiece {
  int row, from, to;                       // row, first element in memory and in LDS
};
__host__ __device__ constexpr LinPiece lin_piece(int lane, int rows, int pieces, int ve, int width) {
  const bool there = lane < rows * pieces;
  const int col = lane % pieces * ve, last = width - ve, first = last < 0 ? last : 0;
  const bool on = there && col < width;
  const int at = col < last ? col : last;
  return LinPiece{there ? lane / pieces : 0, on ? at : first, on ? at : pieces * ve};
}
inline int lin_blocks(const LinShape& p, int64_t value) { return (int)cdiv64(value, 16 * p.waves); }
inline LinShape lin_shape(const pnn_linattn_desc& d, bool backward) {
  LinShape p;
  const int64_t K = d.key_width, V = d.value_width, most = K > V ? K : V;
  const int64_t inner = backward ? most : K, value = backward ? most : V;
  p.pad = inner <= 64 ? 64 : inner <= 128 ? 128 : 256;
  p.tiny = (K < V ? K : V) * (d.dtype == PNN_F32 ? 4 : 2) < 16;      // rows shorter than a piece: one shape for all
  if (p.tiny) p.pad = 256;
  const int64_t chunks = cdiv64(d.length, LIN_CHUNK);
  auto count = [&](int waves) {
    p.waves = waves;
    return d.batch * d.heads * (lin_blocks(p, V) + (backward ? 2 * lin_blocks(p, K) : 0));
  };
  // four waves where eight would have idle ones, or where twice the workgroups fill the device more evenly, uncut
  const int64_t narrow = count(4), wide = count(8);
  const bool four = !p.tiny && (value <= 64 || (wide < LIN_MANY && narrow >= LIN_FEW));
  const int64_t wgs = count(four ? 4 : 8);
  int64_t seg = 1;
  if (wgs > 0 && wgs < LIN_FEW) {
    seg = cdiv64(LIN_MANY, wgs);
    if (seg > chunks / 4) seg = chunks / 4;
    if (seg < 1) seg = 1;
  }
  p.seg_chunks = (int)(chunks > 0 ? cdiv64(chunks, seg) : 1);
  p.segments = (int)(chunks > 0 ? cdiv64(chunks, p.seg_chunks) : 1);
  return p;
}
// bytes of the segments' states of a sum over values of `value` columns
inline int64_t lin_seg_bytes(const pnn_linattn_desc& d, const LinShape& p, int64_t value) {
  return p.segments > 1 ? d.batch * d.heads * p.segments * lin_blocks(p, value) * p.pad * 16 * p.waves * 4 : 0;
}
inline int64_t lin_fwd_bytes(const pnn_linattn_desc& d) {
  return d.length == 1 ? 0 : lin_seg_bytes(d, lin_shape(d, false), d.value_width);
}
inline pnn_head_stride lin_dense(const pnn_linattn_desc& d, int64_t width) {
  return pnn_head_stride{d.length * d.heads * width, d.heads * width, width};
}
// Workspace of the backward: the three sums' segments; gradients of single heads where keys and values are shared
struct LinBwd {
  LinShape shape;
  int64_t seg_q, seg_k, seg_v, part_k, part_v, bytes;
};
inline LinBwd lin_bwd(const pnn_linattn_desc& d) {
  LinBwd w;
  w.shape = lin_shape(d, true);
  int64_t o = 0;
  auto take = [&](int64_t bytes) {
    const int64_t at = o;
    o += round256(bytes);
    return at;
  };
  w.seg_q = take(lin_seg_bytes(d, w.shape, d.key_width));
  w.seg_k = take(lin_seg_bytes(d, w.shape, d.key_width));
  w.seg_v = take(lin_seg_bytes(d, w.shape, d.value_width));
  const int64_t steps = d.heads > d.kv_heads ? d.batch * d.length * d.heads * 4 : 0;
  w.part_k = take(steps * d.key_width);
  w.part_v = take(steps * d.value_width);
  w.bytes = o;
  return w;
}
// threads of the kernel that adds up what heads share: four elements each
inline int64_t lin_head_threads(const pnn_linattn_desc& d) {
  const int64_t wide = d.key_width > d.value_width ? d.key_width : d.value_width;
  return d.heads > d.kv_heads ? d.batch * d.length * d.kv_heads * cdiv64(wide, 4) : 0;
}
int launch_linattn_fwd(const pnn_linattn_desc& d, const void* q, const void* k, const void* v, const float* decay,
                       const int32_t* lengths, const float* s0, void* o, float* sT, void* ws, hipStream_t s);
int launch_linattn_bwd(const pnn_linattn_desc& d, const void* q, const void* k, const void* v, const float* decay,
                       const int32_t* lengths, const float* s0, const void* dout, const float* dsT, void* dq, void* dk,
                       void* dv, float* ds0, void* ws, hipStream_t s);

// ---- norms ----
// How rows run: lanes and 16-byte pieces a lane of one, whether their end cuts a piece, workgroups of the forward and
// the backward
struct NormShape {
  int lanes, pieces, tail, forward, backward;
};
// waves of the backward that registers leave room for on a SIMD, with as many elements a lane
constexpr int norm_waves(int lanes, int elements, bool tail) {
  return lanes == 1024 ? 4 : elements <= 4 ? 7 - tail : elements <= 8 ? 5 - tail : 3 - tail;
}
inline NormShape norm_shape(const pnn_norm_desc& d) {
  NormShape p;
  const int ve = d.dtype == PNN_F32 ? 4 : 8;
  const int64_t n = cdiv64(d.width, ve), rows = d.rows * d.heads;
  p.lanes = n <= 32 ? 16 : n <= 128 ? 64 : n <= 512 ? 256 : 1024;
  p.pieces = n <= p.lanes ? 1 : n <= 2 * p.lanes ? 2 : 4;
  p.tail = d.width % ve != 0;
  const int64_t teams = p.lanes < 256 ? 256 / p.lanes : 1, wgs = cdiv64(rows, teams);
  // As many workgroups as run at a time: 16384 x 2048 backward with 1280 (five a CU) 86 us, with 1536 113.  The forward
  // likes fewer than that: 50 us with 1024, 57 with 2048; 16-lane rows 37 with 1536, 39 with 1024.
  const int64_t most_f = p.lanes == 1024 ? 512 : p.lanes == 256 ? 1024 : 1536;
  const int64_t most_b = p.lanes == 1024 ? 256 : 256 * norm_waves(p.lanes, p.pieces * ve, p.tail);
  p.forward = (int)(wgs < most_f ? wgs : most_f);
  p.backward = (int)(wgs < most_b ? wgs : most_b);
  return p;
}
inline int64_t norm_ws_bytes(const pnn_norm_desc& d) { return (int64_t)norm_shape(d).backward * 2 * d.width * 4; }
int launch_norm_fwd(const pnn_norm_desc& d, const void* x, const float* w_post, const void* gate, const void* res,
                    const float* w_pre, void* h, void* y, hipStream_t s);
int launch_norm_bwd(const pnn_norm_desc& d, const void* x, const float* w_post, const void* gate, const void* res,
                    const float* w_pre, const void* dy, const void* dh, void* dx, void* dgate, void* dres,
                    float* dw_post, float* dw_pre, int accumulate, void* ws, hipStream_t s);

// ---- policy loss ----
int launch_policy(const pnn_policy_desc& d, const void* logits, const int32_t* tokens, const float* advantage,
                  const float* old, const float* ref, const float* weight, float* loss, float* logp, void* dlogits,
                  hipStream_t s);

}  // namespace pnn
