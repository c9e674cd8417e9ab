// The checks of arguments that layer_api.cpp and linear_api.cpp share.
#pragma once

#include <cstddef>
#include <cstdint>

#include "../../include/mics.h"
#include "internal.h"
#include "layer_internal.h"

namespace mics {
namespace {

inline uintptr_t addr(const void* p) { return reinterpret_cast<uintptr_t>(p); }

inline int hip_fail(const char* fn, int err)
{
    return fail(MICS_ERR_HIP, "%s: HIP error %d (%s)", fn, err, hip_error_text(err));
}

inline bool known(int dtype) { return dtype == MICS_DTYPE_BF16 || dtype == MICS_DTYPE_F16 || dtype == MICS_DTYPE_F32; }
inline size_t width(int dtype) { return dtype == MICS_DTYPE_F32 ? 4 : 2; }

// The arguments of one call: a matrix or vector is added with its name, then all of them are checked.
class Checked {
  public:
    Checked(const char* fn, size_t rows, size_t cols) : fn_(fn), rows_(rows), cols_(cols) {}

    int sizes(const char* cols_name) const
    {
        if (cols_ < 1) return fail(MICS_ERR_INVALID_ARG, "%s: %s = 0", fn_, cols_name);
        if (cols_ > kMostCols)
            return fail(MICS_ERR_UNSUPPORTED, "%s: %s = %zu exceeds %zu", fn_, cols_name, cols_, kMostCols);
        if (rows_ > SIZE_MAX / 32 / cols_) return fail(MICS_ERR_INVALID_ARG, "%s: rows * %s overflows", fn_, cols_name);
        return MICS_OK;
    }
    int dtype(const char* name, int value) const
    {
        return known(value) ? MICS_OK : fail(MICS_ERR_UNSUPPORTED, "%s: %s = %d is not bf16, f16 or f32", fn_, name, value);
    }
    // Matrix i of the strides: `stride` elements from row to row.
    size_t stride(const size_t* strides, int i) const { return strides ? strides[i] : cols_; }
    void matrix(const char* name, const void* p, size_t stride, size_t elem, bool out, bool optional = false)
    {
        shaped(name, p, rows_, cols_, stride, elem, out, optional, false);
    }
    // A matrix of its own shape.  `whole`: an input that is read after the first result is stored, so none may take its place.
    void shaped(const char* name, const void* p, size_t rows, size_t cols, size_t stride, size_t elem, bool out, bool optional,
                bool whole)
    {
        add({name, p, rows ? ((rows - 1) * stride + cols) * elem : 0, elem, stride * elem, cols * elem, out, optional || rows == 0, whole});
        if (stride < cols && (p || !optional) && !short_) short_ = name;
        if (rows && stride > (SIZE_MAX / 8 - cols) / rows && !long_) long_ = name;
    }
    void vector(const char* name, const void* p, size_t n, size_t elem, bool out, bool optional = false)
    {
        add({name, p, n * elem, elem, 0, 0, out, optional || n == 0, false});
    }
    int check() const
    {
        if (short_) return fail(MICS_ERR_INVALID_ARG, "%s: the row stride of %s is less than its columns", fn_, short_);
        if (long_) return fail(MICS_ERR_INVALID_ARG, "%s: rows times the row stride of %s overflows", fn_, long_);
        for (int i = 0; i < n_; ++i) {
            const Region& r = region_[i];
            if (!r.p) {
                if (r.optional) continue;
                return fail(MICS_ERR_INVALID_ARG, "%s: %s is NULL", fn_, r.name);
            }
            if (addr(r.p) % r.elem)
                return fail(MICS_ERR_ALIGNMENT, "%s: %s not aligned to %zu bytes", fn_, r.name, r.elem);
        }
        for (int i = 0; i < n_; ++i)
            for (int j = 0; j < n_; ++j) {
                const Region &out = region_[i], &other = region_[j];
                if (i == j || !out.out || (other.out && j < i)) continue;
                if (clash(out, other))
                    return fail(MICS_ERR_INVALID_ARG, "%s: %s overlaps %s", fn_, out.name, other.name);
            }
        return MICS_OK;
    }

  private:
    struct Region {
        const char* name;
        const void* p;
        size_t bytes, elem;
        size_t stride, row;          // bytes; 0: a vector
        bool out, optional, whole;
    };
    static constexpr int kMost = 16;
    const char* fn_;
    size_t rows_, cols_;
    Region region_[kMost];
    int n_ = 0;
    const char *short_ = nullptr, *long_ = nullptr;

    void add(const Region& r) { region_[n_++] = r; }
    static bool clash(const Region& out, const Region& other)
    {
        if (!out.p || !other.p || !out.bytes || !other.bytes) return false;
        const uintptr_t a = addr(out.p), b = addr(other.p);
        if (a >= b + other.bytes || b >= a + out.bytes) return false;
        if (!out.stride || out.stride != other.stride) return true;
        // a result may replace an input of the same place and stride; rows of one stride may lie between each other
        if (a == b && !other.out && !other.whole && other.row == out.row) return false;
        const size_t shift = (a > b ? a - b : b - a) % out.stride;      // of the later matrix behind a row of the earlier
        const size_t earlier = a > b ? other.row : out.row, later = a > b ? out.row : other.row;
        return shift < earlier || shift + later > out.stride;
    }
};

inline int workspace(const char* fn, const void* p, size_t bytes, size_t needed)
{
    if (bytes < needed)
        return fail(MICS_ERR_INVALID_ARG, "%s: workspace_bytes = %zu, needs %zu", fn, bytes, needed);
    if (needed && !p) return fail(MICS_ERR_INVALID_ARG, "%s: workspace is NULL", fn);
    if (addr(p) % 8) return fail(MICS_ERR_ALIGNMENT, "%s: workspace not aligned to 8 bytes", fn);
    return MICS_OK;
}

inline bool column_sizes(size_t rows, size_t cols)
{
    return cols >= 1 && cols <= kMostCols && rows <= SIZE_MAX / 32 / cols;
}

}  // namespace
}  // namespace mics

#define MICS_TRY(call) do { if (int rc_ = (call)) return rc_; } while (0)
