// Whether what a step of a list of tensors writes shares memory with anything else that it reads or writes.  Host code only, without HIP's headers.
#pragma once

#include <algorithm>
#include <cstdint>
#include <initializer_list>
#include <utility>
#include <vector>

#include "mqg.h"

namespace mqg {

struct MemoryRange {
    uintptr_t begin, end;
    bool written;
    bool operator<(const MemoryRange &o) const { return begin < o.begin; }
};

// scalars: numbers that the step reads on the device, with their sizes; null ones are not there.  Two ranges that are only read may share memory (tensors with one gradient).
inline bool step_shares_memory(const mqg_param *params, int32_t num, std::initializer_list<std::pair<const void *, int64_t>> scalars) {
    std::vector<MemoryRange> all;
    all.reserve(static_cast<size_t>(num) * 7 + scalars.size());
    auto bytes = [](int32_t dtype) { return dtype == MQG_F32 ? 4 : 2; };
    auto add = [&](const void *p, uint64_t size, bool written) {
        const uintptr_t at = reinterpret_cast<uintptr_t>(p);
        if (p) all.push_back({at, at + size, written});
    };
    for (const auto &s : scalars) add(s.first, static_cast<uint64_t>(s.second), false);
    std::sort(all.begin(), all.end());
    // A kind of buffer at a time: those of a list mostly lie in its order, and all of a kind beside those of the others, so that little is left to sort.
    auto kind = [&](auto add_one) {
        const auto middle = static_cast<std::ptrdiff_t>(all.size());
        for (int32_t i = 0; i < num; ++i)
            if (params[i].grad && params[i].numel > 0) add_one(params[i], static_cast<uint64_t>(params[i].numel));
        const auto from = all.begin() + middle;
        if (!std::is_sorted(from, all.end())) std::sort(from, all.end());
        if (middle > 0 && from != all.end() && *from < *(from - 1)) std::inplace_merge(all.begin(), from, all.end());
    };
    kind([&](const mqg_param &p, uint64_t n) { add(p.weight, n * bytes(p.weight_type), true); });
    kind([&](const mqg_param &p, uint64_t n) { add(p.grad, n * bytes(p.grad_type), false); });
    kind([&](const mqg_param &p, uint64_t n) { if (p.copy) add(p.copy, n * bytes(p.copy_type), true); });
    kind([&](const mqg_param &p, uint64_t n) { add(p.m, n * (p.state_type == MQG_STATE_E4M3 ? 1 : 4), true); });
    kind([&](const mqg_param &p, uint64_t n) { add(p.v, n * (p.state_type == MQG_STATE_E4M3 ? 1 : 4), true); });
    auto scales = [](uint64_t n) { return (n + MQG_ADAMW_BLOCK - 1) / MQG_ADAMW_BLOCK * 4; };
    kind([&](const mqg_param &p, uint64_t n) { if (p.state_type == MQG_STATE_E4M3) add(p.m_scale, scales(n), true); });
    kind([&](const mqg_param &p, uint64_t n) { if (p.state_type == MQG_STATE_E4M3) add(p.v_scale, scales(n), true); });
    uintptr_t written_to = 0, read_to = 0;                 // the ends of what lies before
    for (const MemoryRange &r : all) {
        if (r.begin < written_to || (r.written && r.begin < read_to)) return true;
        (r.written ? written_to : read_to) = std::max(r.written ? written_to : read_to, r.end);
    }
    return false;
}

}  // namespace mqg
