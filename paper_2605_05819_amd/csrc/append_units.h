// Which head of K or V each wave of an append to an 8-bit cache works on, and where
// its rows begin: plain C++, so that a host program can check every address.
#pragma once

namespace cl {

// Wave `unit` of a token's 2 heads units: K's heads, then V's.  The last
// workgroup's waves beyond them (an odd number of key heads leaves two) hold no
// head: they take part in the workgroup's barriers and read nothing.
struct KvUnit {
    bool is_v, live;
    int head;                      // 0 where there is none, so that it is an address' part anywhere
};

constexpr KvUnit kv_unit(int unit, int heads) {
    return unit < heads ? KvUnit{false, true, unit} : unit < 2 * heads ? KvUnit{true, true, unit - heads} : KvUnit{true, false, 0};
}

// Of `rows` new rows of a block, those that the wave loads.
constexpr int loaded_rows(const KvUnit& u, int rows) { return u.live ? rows : 0; }

// The wave's first element of token t, from the start of k or v.
constexpr long long row_offset(const KvUnit& u, long long stride, int dim, int t) {
    return t * stride + static_cast<long long>(u.head) * dim;
}

}  // namespace cl
