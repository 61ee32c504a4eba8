// How work that lies in a row, `total` tiles of it, is shared out among `units`: each takes what lies between two of
// units + 1 marks.  Plain arithmetic that the kernels and the CPU's tests share.
//
// total below 2^31, units up to 2^16: the products are exact in binary64, and a quotient that is no whole number is at least
// 1 / 2^31 away from one, far more than its rounding.
#pragma once

namespace hp {

// The first tile of unit u (of u = units: the end).
constexpr int first_of(int total, int u, int units) { return (int)((double)total * u / units); }
// The unit that tile t, below total, belongs to.
constexpr int unit_of(int total, int t, int units) { return (int)((((double)t + 1.0) * units - 1.0) / total); }

}  // namespace hp
