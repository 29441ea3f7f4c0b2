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

}  // namespace oaa
