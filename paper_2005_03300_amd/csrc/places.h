// Host-only helper, free of HIP so that it can be tested by itself.
#pragma once
#include <cstddef>
#include <cstdint>

namespace gcn {

// The bytes of a matrix: `rows` rows of `cols` elements of `bytes` each, `ld` elements apart (ld >= cols).  What lies between the rows is not the matrix's, and may be
// another one's: halves of one buffer do not meet.
class Span {
public:
    Span(const void* p, int64_t rows, int64_t cols, int64_t ld, size_t bytes) {
        if (!p || rows <= 0) return;
        from_ = (uintptr_t)p;
        rows_ = rows;
        width_ = (size_t)cols * bytes;
        pitch_ = (size_t)ld * bytes;
        if (rows > 1 && ld == cols) {                              // one range
            width_ *= (size_t)rows;
            rows_ = 1;
        }
    }
    // whether the two have a byte in common
    bool meets(const Span& o) const {
        if (!rows_ || !o.rows_ || from_ >= o.to() || o.from_ >= to()) return false;
        // at the same pitch, where rows meet, the first row of one of the two meets a row of the other
        if (rows_ == 1 || o.rows_ == 1 || pitch_ == o.pitch_) return o.has(from_, from_ + width_) || has(o.from_, o.from_ + o.width_);
        const Span &few = rows_ < o.rows_ ? *this : o, &other = rows_ < o.rows_ ? o : *this;
        for (int64_t i = 0; i < few.rows_; ++i) {
            const uintptr_t a = few.from_ + (size_t)i * few.pitch_;
            if (other.has(a, a + few.width_)) return true;
        }
        return false;
    }
    // whether the two are the same elements in the same order, for matrices of as many rows
    bool is(const Span& o) const { return from_ == o.from_ && rows_ == o.rows_ && width_ == o.width_ && (rows_ == 1 || pitch_ == o.pitch_); }

private:
    uintptr_t to() const { return from_ + (size_t)(rows_ - 1) * pitch_ + width_; }
    // whether a row has a byte of [a, b): the first row that ends behind a begins before b
    bool has(uintptr_t a, uintptr_t b) const {
        const int64_t i = a < from_ + width_ ? 0 : (int64_t)((a - from_ - width_) / pitch_) + 1;
        return i < rows_ && from_ + (size_t)i * pitch_ < b;
    }
    uintptr_t from_ = 0;
    int64_t rows_ = 0;
    size_t width_ = 0, pitch_ = 0;
};

}  // namespace gcn
