// Device memory that several calls of a context share one after the other and that grows with what they need.  Host code only, without HIP's headers.
#pragma once

#include <cstdint>
#include <vector>

namespace mqg {

// A launch that was recorded into a HIP graph has the memory's address in it and may be replayed as long as the context lives: what such a launch
// was given stays allocated until then, whatever takes its place.
struct Arena {
    char *data = nullptr;
    int64_t bytes = 0;
    bool recorded = false;               // a recorded launch has `data`
    std::vector<char *> kept;            // outgrown, but recorded

    // alloc(bytes) returns the new memory, null if there is none; then the arena is left empty
    template <typename Alloc, typename Release>
    bool grow(int64_t wanted, Alloc alloc, Release release) {
        if (recorded) kept.push_back(data);                // (first: it may throw)
        else if (data) release(data);
        data = nullptr;
        bytes = 0;
        recorded = false;
        data = alloc(wanted);
        if (data) bytes = wanted;
        return data != nullptr;
    }
    template <typename Release>
    void end(Release release) {
        if (data) release(data);
        for (char *p : kept) release(p);
        *this = Arena();
    }
};

}  // namespace mqg
