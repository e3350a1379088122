// A search among ascending places that looks at 64 of them at a time.  Plain C++, for the kernels and for the host, where it is tested.
#pragma once

namespace laq {

// What is left of the places 0 .. n - 1: `n` from `lo` on, the first of which lies before what is looked for if any does.
struct Find {
  int lo, n;
  constexpr int step() const { return n / 64 + (n % 64 != 0); }              // lane l looks at lo + l * step()
  constexpr bool looks(int lane) const { return (long long)lane * step() < n; }
  // `before`: how many of the lanes that look find that their place lies before.  Places in no order are searched too: whichever lanes those are, none or all of them among
  // them, what is left lies among what there was.  (Signed: a count of lanes is unsigned, and 0 - 1 of it is no place.)
  constexpr void narrow(int before) {
    const int s = step(), last = before > 1 ? before - 1 : 0;
    lo += last * s;
    n = n - last * s < s ? n - last * s : s;
  }
};

}  // namespace laq
