// What the host sides of several translation units ask of arguments.
#pragma once

#include <cstdint>

#include "vlut.h"

namespace {

bool type_ok(int type) { return type == VLUT_TYPE_F32 || type == VLUT_TYPE_BF16 || type == VLUT_TYPE_F16; }
int type_bytes(int type) { return type == VLUT_TYPE_F32 ? 4 : 2; }
bool power_of_two(int64_t v) { return v > 0 && (v & (v - 1)) == 0; }

// Vectors of 4, 2 or 1: the widest that divides the pairs and whose loads and stores are aligned everywhere.
struct Alignment {
    int vec = 4;
    void pointer(const void* p, int bytes) {
        while (vec > 1 && (uintptr_t)p % (uintptr_t)(vec * bytes)) vec /= 2;
    }
    void stride(int64_t s) {
        while (vec > 1 && s % vec) vec /= 2;
    }
};

}  // namespace
