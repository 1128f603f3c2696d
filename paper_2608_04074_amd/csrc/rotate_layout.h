// Which coordinates of a head a lane of the norm and rotation holds, and how it
// stores their 4-bit codes (rotate.hip). Plain arithmetic, the same on the host.
#pragma once

namespace novakv {
namespace rotate {

// D / 8 lanes hold a head, two chunks of four coordinates each, from c0 and from c1: the
// two ends of rotated pairs, or eight that follow each other.
struct LaneChunks {
  bool turns;
  int c0, c1;
};
constexpr LaneChunks lane_chunks(const int lane, const int rotary_dim, const bool interleaved) {
  const bool turns = lane < rotary_dim / 8, halves = turns && !interleaved;
  const int c0 = halves ? 4 * lane : 8 * lane;
  return {turns, c0, halves ? c0 + rotary_dim / 2 : c0 + 4};
}

// Codes take half a byte each, so a chunk two bytes.
enum class CodeStore {
  kBoth,      // four bytes: the chunks follow each other
  kExchange,  // four bytes: two neighbours exchange a chunk, the even lane stores both lower ones, the odd one both upper ones
  kApart,     // two bytes twice
};
// The upper half of the pairs starts at byte rotary_dim / 4: a multiple of four, so that words may
// be stored there, for an even number of rotated chunks only.
constexpr CodeStore code_store(const LaneChunks &l, const int rotary_dim, const bool interleaved) {
  if (interleaved || !l.turns) return CodeStore::kBoth;
  return rotary_dim % 16 == 0 ? CodeStore::kExchange : CodeStore::kApart;
}
// Byte of the row where a lane's word goes.
constexpr int word_at(const LaneChunks &l, const CodeStore how, const int lane) {
  return how == CodeStore::kExchange && (lane & 1) ? (l.c1 - 4) / 2 : l.c0 / 2;
}

}  // namespace rotate
}  // namespace novakv
