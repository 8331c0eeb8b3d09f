// What the validation layers of the 8-bit path share (q8_api.cpp, q8_xent_api.cpp):
// limits, and the checks of a call's buffers.
#pragma once
#include <cstdint>

#include "cpdp_q8.h"
#include "q8_launch.h"

namespace {

using cpdp::q8::Act;
using cpdp::q8::Held;
using cpdp::q8::Mat;

// Most rows (a grid holds at most 2^31 - 1 blocks) and the largest inner size.
constexpr int64_t kMaxRows = 0x7FFFFFFF - 8;
constexpr int64_t kMaxCols = (int64_t)1 << 30;
// Largest row stride: byte sizes of whole matrices stay below 2^62.
constexpr int64_t kMaxLd = (int64_t)1 << 28;
// Largest row, in bytes, of a matrix that a product reads: a tile's rows are
// addressed with 32-bit offsets from the first of them.
constexpr int64_t kMaxTileLd = ((int64_t)1 << 23) - 16;

inline bool is_dtype(int dt) { return dt == CPDP_F32 || dt == CPDP_BF16; }
inline int64_t esize(bool bf16) { return bf16 ? 2 : 4; }
inline int hip_status(int err) { return err == 0 ? CPDP_OK : CPDP_ERR_HIP; }

// Collects the buffers of a call: first whether all are there and described
// rightly, then whether one that is written overlaps another.
class Buffers {
  public:
    // rows x cols elements of `es` bytes with row stride ld
    void in(const void* p, int64_t ld, int64_t rows, int64_t cols, int64_t es) {
        if (ld < cols || ld > kMaxLd) {
            if (status_ == CPDP_OK) status_ = CPDP_ERR_INVALID_ARG;
            return;
        }
        const int64_t bytes = rows == 0 || cols == 0 ? 0 : ((rows - 1) * ld + cols) * es;
        add(p, bytes, 16, ld * es, cols * es);
    }
    void in(const void* p, int64_t n, int64_t es, int64_t align) { add(p, n * es, align, 0, 0); }
    void out(const void* p, int64_t ld, int64_t rows, int64_t cols, int64_t es) {
        const int before = n_;
        in(p, ld, rows, cols, es);
        if (n_ > before) b_[before].written = true;
    }
    void out(const void* p, int64_t n, int64_t es, int64_t align) {
        in(p, n, es, align);
        b_[n_ - 1].written = true;
    }
    // the last matrix may be the very same rows as buffer k
    void may_be(int k) {
        if (n_ > 0 && k >= 0 && b_[n_ - 1].lo == b_[k].lo && b_[n_ - 1].ld == b_[k].ld)
            b_[n_ - 1].twin[k] = true;
    }
    int last() const { return n_ - 1; }
    int status() const {
        if (status_ != CPDP_OK) return status_;
        for (int i = 0; i < n_; ++i)
            if (b_[i].lo == 0 && b_[i].bytes > 0) return CPDP_ERR_NULL;
        for (int i = 0; i < n_; ++i)
            if (b_[i].lo + (uintptr_t)b_[i].bytes < b_[i].lo) return CPDP_ERR_INVALID_ARG;
        for (int i = 0; i < n_; ++i)
            if (b_[i].lo % (uintptr_t)b_[i].align != 0 || b_[i].ld % 16 != 0)
                return CPDP_ERR_MISALIGNED;
        for (int i = 0; i < n_; ++i)
            for (int j = 0; j < i; ++j)
                if ((b_[i].written || b_[j].written) && !b_[i].twin[j] && overlap(b_[i], b_[j]))
                    return CPDP_ERR_OVERLAP;
        return CPDP_OK;
    }

  private:
    static constexpr int kMost = 12;
    struct Buffer {
        uintptr_t lo;
        int64_t bytes, align, ld, row;  // ld, row: bytes from row to row and in a row; 0: a vector
        bool written, twin[kMost];
    };
    static bool overlap(const Buffer& a, const Buffer& b) {
        if (a.bytes == 0 || b.bytes == 0 || a.lo >= b.lo + (uintptr_t)b.bytes ||
            b.lo >= a.lo + (uintptr_t)a.bytes)
            return false;
        if (a.ld == 0 || a.ld != b.ld) return true;
        // two column ranges of one matrix, as the halves of a fused product are
        const int64_t d = a.lo >= b.lo ? (int64_t)((a.lo - b.lo) % (uintptr_t)a.ld)
                                       : a.ld - (int64_t)((b.lo - a.lo) % (uintptr_t)a.ld);
        return !(d >= b.row && d + a.row <= a.ld);
    }
    void add(const void* p, int64_t bytes, int64_t align, int64_t ld, int64_t row) {
        b_[n_++] = Buffer{reinterpret_cast<uintptr_t>(p), bytes, align, ld, row, false, {}};
    }
    Buffer b_[kMost];
    int n_ = 0, status_ = CPDP_OK;
};

inline bool rows_ok(int64_t T, int64_t D) {
    return T >= 0 && T <= kMaxRows && D >= 1 && D <= kMaxCols;
}

inline Mat mat(const void* p, int64_t ld, int dt) {
    return {const_cast<void*>(p), ld, dt == CPDP_BF16};
}
inline Held held(const int8_t* q, int64_t ld, const float* scale) {
    return {const_cast<int8_t*>(q), ld, const_cast<float*>(scale)};
}

}  // namespace
