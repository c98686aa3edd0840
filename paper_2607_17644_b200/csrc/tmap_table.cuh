// A bounded table of values that are pure functions of their keys, for the library's tensor maps.  Plain C++ (no CUDA), so that a test
// can compile it alone.
#pragma once
#include <cstddef>
#include <cstdint>
#include <mutex>

namespace laga {

// kSets sets of kWays entries; a key's set comes from its hash, a full set replaces its entries in turn.  So a lookup looks at kWays
// keys whatever the table holds, and keys push one another out only within a set.
// Key: operator== and a member `uint64_t hash() const`.
template <class Key, class Value, size_t kSets, size_t kWays>
class MapTable {
public:
    // *value is the key's: the one kept, or made now by make(Value*) -> bool; false if that fails (nothing is kept then).
    template <class Make>
    bool get(const Key& key, Value* value, Make make) {
        Set& set = sets_[key.hash() % kSets];
        std::lock_guard<std::mutex> lock(mutex_);
        for (size_t i = 0; i < set.used; ++i)
            if (set.keys[i] == key) { *value = set.values[i]; return true; }
        if (!make(value)) return false;
        size_t at = set.used;
        if (at < kWays) ++set.used;
        else { at = set.next; set.next = (at + 1) % kWays; }
        set.keys[at] = key;
        set.values[at] = *value;
        return true;
    }

private:
    struct Set {
        size_t used = 0, next = 0;
        Key keys[kWays] = {};
        Value values[kWays];
    };
    Set sets_[kSets];
    std::mutex mutex_;
};

// Mixes one more word into a hash (multiplication by an odd constant near 2^64 / golden ratio, high bits folded down).
inline uint64_t hash_add(uint64_t h, uint64_t word) {
    h = (h ^ word) * 0x9e3779b97f4a7c15ull;
    return h ^ (h >> 29);
}

}  // namespace laga
