// How kv_attn deals keys out to work-groups.  A unit is kUnitKeys keys of one row tile; a sequence's tiles have as many units as its longest
// row sees (one at least, so that rows which see nothing are written too).  All units stand in one line,
//     KV head, sequence, row tile, unit,
// of which every work-group takes the same number, the first ones one more: sequences of any lengths keep all work-groups busy until
// the end, and nothing of it has to be known to the host.  A tile that lies in one work-group's stretch is finished there.  One that
// several share is left in shares, which a second kernel joins: a work-group has two places for them, one for the tile that its
// stretch begins inside of, one for the tile that it ends inside of.
// The same code on the host, where it is compared with a list of all units.
#pragma once

namespace aa {

constexpr int kUnitKeys = 128;

#ifdef __HIPCC__
#define AA_DEAL __host__ __device__ __forceinline__
#else
#define AA_DEAL inline
#endif

// Units of a row tile whose last row sees `see` keys (of a sequence without rows: 0).
AA_DEAL int deal_units(int see, int new_tokens) { return new_tokens <= 0 ? 0 : see <= kUnitKeys ? 1 : (see + kUnitKeys - 1) / kUnitKeys; }

// each: units of a work-group (total / groups); more: how many work-groups have one more.
struct Deal { unsigned each, more; };
AA_DEAL unsigned deal_start(const Deal& d, unsigned group) { return group * d.each + (group < d.more ? group : d.more); }
AA_DEAL unsigned deal_group(const Deal& d, unsigned unit) {
    const unsigned first = d.more * (d.each + 1);
    return unit < first ? unit / (d.each + 1) : d.more + (unit - first) / d.each;
}

// Place of the share that work-group `group` leaves of a tile that it enters at unit t of the tile.
AA_DEAL int deal_place(int group, int t) { return 2 * group + (t == 0); }

}  // namespace aa
