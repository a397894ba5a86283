// Rows of any element type by pieces of 16 bytes (routing and 4-bit kernels).
#pragma once

#include <hip/hip_runtime.h>

#include "ftk_internal.h"

namespace ftk {

// Arithmetic type of sums over elements of a type: 32 bits, 64 for doubles.
template <typename T>
struct RowType {
    using Acc = float;
};
template <>
struct RowType<double> {
    using Acc = double;
};

// 16 bytes of a row, read and written at element alignment (global memory takes unaligned vectors).
template <typename T>
constexpr int PIECE = 16 / sizeof(T);
template <typename T>
using PieceOf = T __attribute__((ext_vector_type(PIECE<T>), aligned(sizeof(T))));

template <typename T>
__device__ __forceinline__ PieceOf<T> row_piece(const T *p)
{
    return *reinterpret_cast<const PieceOf<T> *>(p);
}
// STREAM_STORE(to, value, stream): *to = value; where `stream`, past the caches (see streams_out).  A macro, because a function would
// lose the alignment of what `to` points to; the empty statements keep the branch, of whose two stores the
// compiler would make an ordinary one.
#define STREAM_STORE(to, value, stream)                    \
    do {                                                   \
        if (stream) {                                      \
            asm volatile("");                              \
            __builtin_nontemporal_store((value), (to));    \
            asm volatile("");                              \
        } else {                                           \
            *(to) = (value);                               \
        }                                                  \
    } while (0)
template <typename T>
__device__ __forceinline__ void put_piece(T *p, PieceOf<T> v, bool stream = false)
{
    STREAM_STORE(reinterpret_cast<PieceOf<T> *>(p), v, stream);
}

// Results of more than a quarter of the memory-side cache's 256 MB go past the caches: whoever reads them next finds little of
// them there, and the operands stay.  (With and without, in turn with other operands: weighted sum back, 65536 x 2 slots x 1024 bf16
// 70 / 76 us; both gradients 205 / 215; 65536 x 2048 bf16 to 4 bits and back 105 / 142; but 40 MB from 4 bits 15 / 11, and rows to
// their places, 60000 x 1024 fp32, 125 / 124 among others and 149 / 140 alone: those are written as usual.)
static inline bool streams_out(double bytes) { return bytes > 64e6; }

// Rows are read by whole pieces; the last one is moved back into the row where the row is no multiple of a
// piece, so that two pieces may share elements.  Rows shorter than a piece go by elements (one "piece" each).
template <typename T>
__host__ __device__ constexpr int row_pieces(int D)
{
    return D < PIECE<T> ? D : (D + PIECE<T> - 1) / PIECE<T>;
}

// calls f(tag of the element type) for a dtype
template <typename T>
struct TypeTag {
    using type = T;
};
template <typename F>
ftk_status with_type(ftk_dtype dtype, F &&f)
{
    switch (dtype) {
    case FTK_F32: return f(TypeTag<float>{});
    case FTK_F64: return f(TypeTag<double>{});
    case FTK_BF16: return f(TypeTag<__bf16>{});
    case FTK_F16: return f(TypeTag<_Float16>{});
    }
    set_error("unknown dtype %d", (int)dtype);
    return FTK_EINVAL;
}
static inline size_t dtype_size(ftk_dtype dtype) { return dtype == FTK_F64 ? 8 : dtype == FTK_F32 ? 4 : 2; }
static inline bool known_dtype(ftk_dtype d) { return d == FTK_F32 || d == FTK_F64 || d == FTK_BF16 || d == FTK_F16; }

}  // namespace ftk
