// What the decode, normalising and 4-bit entry points share (host side).
#pragma once
#include <string>

#include "tessera.h"

namespace tessera {

constexpr int kDecodeUnit = 16;      // keys of the tile in which a decode step's work is handed out

// Shapes, ranges and pointers of a decode call; on failure `err` holds the reason.
int32_t check_decode(const tessera_model_cfg *cfg, const tessera_decode_desc *desc, std::string *err);

// Nothing throws through a C entry point (a text for the error may find no memory).
template <class F>
int32_t guarded(F f) noexcept {
    try {
        return f();
    } catch (...) {
        return TESSERA_INVALID_ARG;
    }
}

}  // namespace tessera
