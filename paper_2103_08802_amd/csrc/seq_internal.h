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

}  // namespace pnn
