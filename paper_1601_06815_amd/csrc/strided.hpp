// Where the elements of a strided tensor lie. Plain host code.
#pragma once

namespace oaa {

// Element (b, s, c), b < images, s < rows, c < columns (each 1 or more), at b image
// + s row + c.
struct Strided {
  long long images, image, rows, row, columns;
};

// Whether no two elements of t are one: each image ends before the next begins, and
// each of its rows does; or each row, which holds that row of all images, does.
inline bool images_apart(const Strided& t) {
  return (t.rows == 1 || t.row >= t.columns) &&
         (t.images == 1 || t.image >= (t.rows - 1) * t.row + t.columns);
}

inline bool rows_apart(const Strided& t) {
  return (t.images == 1 || t.image >= t.columns) &&
         (t.rows == 1 || t.row >= (t.images - 1) * t.image + t.columns);
}

namespace strided_detail {

inline long long floor_div(long long a, long long b) { return a / b - (a % b < 0); }

// Whether k step + rest = at for some |k| < count and a rest that `within` takes,
// where two multiples of step are no further than step apart from any rest.
template <typename Fn>
bool reaches(long long at, long long count, long long step, Fn&& within) {
  if (count == 1) return within(at);
  for (long long k = floor_div(at, step), i = 0; i < 2; ++i, ++k)
    if (k > -count && k < count && within(at - k * step)) return true;
  return false;
}

}  // namespace strided_detail

// Whether t, no two of whose elements are one, and the same tensor `at` elements
// further on have an element in common.
inline bool shifted_overlap(const Strided& t, long long at) {
  using strided_detail::reaches;
  auto column = [&](long long d) { return d > -t.columns && d < t.columns; };
  if (images_apart(t))
    return reaches(at, t.images, t.image, [&](long long d) { return reaches(d, t.rows, t.row, column); });
  return reaches(at, t.rows, t.row, [&](long long d) { return reaches(d, t.images, t.image, column); });
}

// Elements from the first to the last.
inline long long extent(const Strided& t) {
  return (t.images - 1) * t.image + (t.rows - 1) * t.row + t.columns;
}

// Whether `written`, no two of whose elements are one, and `read`, of the same sizes
// and `at` elements further on, surely have an element in common: exactly where their
// strides are equal, otherwise where one fills its memory and the other begins or
// ends in it.
inline bool overlap(const Strided& written, const Strided& read, long long at) {
  const bool images = written.images == 1 || written.image == read.image;
  if (images && (written.rows == 1 || written.row == read.row)) return shifted_overlap(written, at);
  auto fills = [](const Strided& t) { return extent(t) == t.images * t.rows * t.columns; };
  auto holds = [](long long begin, long long end, long long e) { return e >= begin && e < end; };
  const long long w = extent(written), r = extent(read);
  return (fills(written) && (images_apart(written) || rows_apart(written)) &&
          (holds(0, w, at) || holds(0, w, at + r - 1))) ||
         (fills(read) && (images_apart(read) || rows_apart(read)) && (holds(at, at + r, 0) || holds(at, at + r, w - 1)));
}

}  // namespace oaa
