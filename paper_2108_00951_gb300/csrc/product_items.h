// product_items.h — the numbering of a products launch (host only): each phase's
// work items, and the scratch tiles and arrival counters of products whose K
// parts are joined.
#pragma once

#include <cstddef>
#include <cstdint>

namespace efs {

constexpr uint32_t kTileM = 128;    // rows of a CTA's tile: lanes of tensor memory

// Numbers the items of each phase's problems and the scratch tiles of split
// ones; returns the scratch tiles' bytes. A phase whose parts would take more
// than `counters` arrival counters is not split.
template <class Args>
size_t number_items(Args& args, bool pair, uint32_t counters) {
  uint64_t most = 0;
  uint32_t chunks = 0;
  for (uint32_t ph = 0; ph < args.phases; ++ph) {
    const uint32_t first = args.first[ph], end = first + args.problems[ph];
    auto parts_of = [&](uint32_t i) -> uint64_t {
      const auto& p = args.shape[i];
      if (p.splits <= 1 || !p.join) return 0;
      return static_cast<uint64_t>(p.tiles) * p.batch * p.splits * (pair ? 2 : 1);
    };
    uint64_t parts = 0;
    for (uint32_t i = first; i < end; ++i) parts += parts_of(i);
    uint32_t items = 0, part = 0;
    for (uint32_t i = first; i < end; ++i) {
      auto& p = args.shape[i];
      if (parts > counters && p.join) p.splits = 1;
      p.item0 = items;
      p.part0 = part;
      items += p.tiles * p.batch * p.splits;
      part += static_cast<uint32_t>(parts_of(i));
      if (parts_of(i) && p.bn / 32 > chunks) chunks = p.bn / 32;
    }
    args.items[ph] = items;
    if (part > most) most = part;
    if (end > args.entries) args.entries = end;
  }
  args.part_chunks = chunks;
  return static_cast<size_t>(most) * chunks * 32 * kTileM * 4;
}

}  // namespace efs
