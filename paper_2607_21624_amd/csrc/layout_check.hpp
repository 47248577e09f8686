// layout_check.hpp -- checks of tensors given by a layout descriptor, shared by the
// entry points (host).
#pragma once

#include <cstdint>

#include "../../include/fbl.h"
#include "tokmap.hpp"

namespace fbl {

inline int64_t elem_size(int32_t dt) { return dt == FBL_BF16 ? 2 : (dt == FBL_F32 ? 4 : 0); }

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// Tile-legality of one descriptor (paper section 4.3.1 checks): intra-tile
// continuity (sd == 1), tile boundary preservation (tile_d divides D), rows
// that hold whole heads, and 16-byte aligned rows.
inline fbl_status check_layout(const fbl_layout* l) {
    if (!l) return FBL_ERR_NULL;
    const int64_t es = elem_size(l->dtype);
    if (es == 0) return FBL_ERR_DTYPE;
    if (l->B <= 0 || l->S <= 0 || l->H <= 0 || l->D <= 0) return FBL_ERR_SHAPE;
    if (l->B > INT32_MAX || l->S > (1 << 30) || l->H > 65535) return FBL_ERR_SHAPE;
    if (l->sd != 1) return FBL_ERR_LAYOUT;
    if (l->tile_d <= 0 || l->D % l->tile_d != 0 || (l->tile_d * es) % 16 != 0) return FBL_ERR_LAYOUT;
    if (l->sh < l->D) return FBL_ERR_LAYOUT;
    if (l->ss < (l->H - 1) * l->sh + l->D) return FBL_ERR_LAYOUT;
    if (l->B > 1 && l->sb < (l->S - 1) * l->ss + (l->H - 1) * l->sh + l->D) return FBL_ERR_LAYOUT;
    if (l->sb < 0) return FBL_ERR_LAYOUT;
    if ((l->ss * es) % 16 != 0 || (l->sh * es) % 16 != 0 || (l->sb * es) % 16 != 0) return FBL_ERR_ALIGN;
    return FBL_OK;
}

inline bool same_extents(const fbl_layout* a, const fbl_layout* b) {
    return a->B == b->B && a->S == b->S && a->H == b->H && a->D == b->D && a->dtype == b->dtype;
}

// Bytes spanned by a tensor from its base pointer (last element + 1).
inline int64_t span_bytes(const fbl_layout* l) {
    const int64_t last = (l->B - 1) * l->sb + (l->S - 1) * l->ss + (l->H - 1) * l->sh + (l->D - 1);
    return (last + 1) * elem_size(l->dtype);
}

// The attention kernels address a tensor from each (batch, head) base with
// 32-bit byte offsets, and their tiles run up to 128 rows past the last token
// (those rows read as zeros and are never stored): every such offset must stay
// below 2^31, the largest range of a buffer resource.
constexpr int64_t kTileRowPad = 128;
inline bool rows_fit(const fbl_layout* l) {
    return (l->S + kTileRowPad) * l->ss * elem_size(l->dtype) <= ((int64_t)1 << 31);
}

inline bool overlaps(const void* a, int64_t na, const void* b, int64_t nb) {
    const uintptr_t pa = reinterpret_cast<uintptr_t>(a), pb = reinterpret_cast<uintptr_t>(b);
    return pa < pb + (uintptr_t)nb && pb < pa + (uintptr_t)na;
}

// Whether two described tensors share any byte.  Exact for the common case of
// column views into one packed projection output (same row and batch strides,
// rows of one view falling between the columns of the other); otherwise the
// byte ranges decide (conservative).
inline bool views_overlap(const void* pa, const fbl_layout* la, const void* pb, const fbl_layout* lb) {
    const int64_t na = span_bytes(la), nb = span_bytes(lb);
    if (!overlaps(pa, na, pb, nb)) return false;
    const int64_t es = elem_size(la->dtype);
    if (es != elem_size(lb->dtype) || la->ss != lb->ss || la->B != lb->B || la->S != lb->S) return true;
    if (la->B > 1 && (la->sb != lb->sb || la->sb % la->ss != 0)) return true;
    const int64_t dbytes = (int64_t)(reinterpret_cast<uintptr_t>(pb) - reinterpret_cast<uintptr_t>(pa));
    if (dbytes % es != 0) return true;
    const int64_t delta = dbytes / es;
    const int64_t wa = (la->H - 1) * la->sh + la->D;  // columns a row of each view covers
    const int64_t wb = (lb->H - 1) * lb->sh + lb->D;
    if (delta >= 0) return !(delta >= wa && delta + wb <= la->ss);
    return !(-delta >= wb && -delta + wa <= la->ss);
}

inline TokMap tokmap(const fbl_layout* l) { return TokMap{l->sb, l->ss, l->sh}; }

}  // namespace fbl
