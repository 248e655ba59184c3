// Body of a C entry that may run out of host memory while it puts a message
// together: no exception leaves it.
#pragma once

#include "../../include/sangam_attn.h"

namespace sangam {

template <typename Body>
sangam_status entry(Body&& body) noexcept {
    try {
        return body();
    } catch (...) {
        return SANGAM_ERR_BUFFER;
    }
}

}  // namespace sangam
