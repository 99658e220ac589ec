// Bytes that a call's operands take, and whether an output's are another operand's.
// Host arithmetic alone.
#pragma once

#include <algorithm>
#include <cstdint>
#include <functional>
#include <iterator>
#include <map>
#include <queue>
#include <utility>
#include <vector>

namespace wfd {

struct Range {
    uintptr_t lo, hi;        // bytes [lo, hi); empty where there is nothing
    uintptr_t stride = 0;    // of a matrix of several rows: bytes [lo + i stride, lo + i stride + width) of them
    uintptr_t width = 0;
};

// No byte of one is a byte of the other.  Matrices with the same stride are compared by
// their columns (slices of one buffer), others by their whole spans.
inline bool disjoint(const Range &a, const Range &b)
{
    if (!(a.lo < b.hi && b.lo < a.hi)) return true;
    if (!a.stride || a.stride != b.stride) return false;
    const uintptr_t off = b.lo >= a.lo ? (b.lo - a.lo) % a.stride : (a.stride - (a.lo - b.lo) % a.stride) % a.stride;
    return off >= a.width && off + b.width <= a.stride;
}

// Ranges of one stride that are apart from one another, although as whole spans each of
// them reaches the place that the last call of reach() named: slices of one buffer.  In
// the order of their columns a slice can only meet its neighbours.
class Slices {
public:
    // Ranges that end at lo or before it leave; lo never falls.
    void reach(uintptr_t lo)
    {
        while (!ends.empty() && ends.top().first <= lo) {
            const auto at = held.find(ends.top().second);
            if (at != held.end() && at->second.hi <= lo) held.erase(at);
            ends.pop();
        }
    }
    // one that r (from the last reach's place on) is not apart from, or NULL
    Range *meets(const Range &r)
    {
        if (held.empty()) return nullptr;
        Range &any = held.begin()->second;
        if (!r.stride || r.stride != any.stride) return &any;
        const auto next = held.lower_bound(column(r));
        Range &after = next == held.end() ? any : next->second;
        if (!disjoint(after, r)) return &after;
        Range &before = next == held.begin() ? held.rbegin()->second : std::prev(next)->second;
        return disjoint(before, r) ? nullptr : &before;
    }
    // r, which meets none of them
    void put(const Range &r)
    {
        if (held.empty()) base = r.lo;
        const uintptr_t at = column(r);
        held.emplace(at, r);
        ends.emplace(r.hi, at);
    }
    // one of them reaches as far as r, which has the same columns
    void extend(Range &one, const Range &r)
    {
        if (r.hi <= one.hi) return;
        one.hi = r.hi;
        ends.emplace(r.hi, column(one));
    }

private:
    uintptr_t column(const Range &r) const { return r.stride ? (r.lo - base) % r.stride : 0; }

    using End = std::pair<uintptr_t, uintptr_t>;   // of a range, and its column
    std::map<uintptr_t, Range> held;
    std::priority_queue<End, std::vector<End>, std::greater<End>> ends;
    uintptr_t base = 0;
};

inline bool same_columns(const Range &a, const Range &b)   // b begins at a's begin or behind it
{
    return a.stride == b.stride && a.width == b.width && (a.stride ? (b.lo - a.lo) % a.stride == 0 : b.lo == a.lo);
}

struct Span {
    Range r;
    bool written;
};

// Spans that are written lie apart from one another and from those that are read.
// They are gone through in the order of their first bytes (a sort, where each has a
// place of its own) with those that reach as far as the present one: the written ones,
// and the read ones, of which the same columns count once.  Only read ones that overlap
// others in part are gone through one by one.
inline bool spans_apart(std::vector<Span> &spans)
{
    std::erase_if(spans, [](const Span &s) { return s.r.lo == s.r.hi; });
    std::sort(spans.begin(), spans.end(), [](const Span &a, const Span &b) { return a.r.lo < b.r.lo; });
    uintptr_t end = 0;
    bool own = true;
    for (const Span &s : spans) own = own && s.r.lo >= end, end = std::max(end, s.r.hi);
    if (own) return true;
    Slices outs, ins;
    std::vector<Range> more_ins;
    for (const Span &s : spans) {
        outs.reach(s.r.lo);
        if (outs.meets(s.r)) return false;
        ins.reach(s.r.lo);
        Range *in = ins.meets(s.r);
        if (s.written) {
            if (in) return false;
            std::erase_if(more_ins, [&](const Range &r) { return r.hi <= s.r.lo; });
            for (const Range &r : more_ins)
                if (!disjoint(r, s.r)) return false;
            outs.put(s.r);
        } else if (!in) {
            ins.put(s.r);
        } else if (same_columns(*in, s.r)) {
            ins.extend(*in, s.r);
        } else {
            std::erase_if(more_ins, [&](const Range &r) { return r.hi <= s.r.lo; });
            const auto same = std::find_if(more_ins.begin(), more_ins.end(), [&](const Range &r) { return same_columns(r, s.r); });
            if (same == more_ins.end()) more_ins.push_back(s.r);
            else same->hi = std::max(same->hi, s.r.hi);
        }
    }
    return true;
}

}  // namespace wfd
