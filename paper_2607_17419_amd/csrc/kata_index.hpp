// kata_index.hpp -- places of a launch's threads in plain C++ (constexpr: host and
// device), so that their arithmetic can be checked on the CPU at sizes that no test
// allocates.
#pragma once

namespace kata {

// A thread's sequence, run of tokens and channel group in the convolution's forward.  A
// launch has up to 2^32 - 512 threads, all of one sequence perhaps.
struct ConvPlace {
  int b, run, group;
};
constexpr ConvPlace conv_place(long long id, int groups, int runs) {
  const long long per = static_cast<long long>(groups) * runs, b = id / per;
  const unsigned rest = static_cast<unsigned>(id - b * per), run = rest / static_cast<unsigned>(groups);
  return {static_cast<int>(b), static_cast<int>(run),
          static_cast<int>(rest - run * static_cast<unsigned>(groups))};
}

}  // namespace kata
