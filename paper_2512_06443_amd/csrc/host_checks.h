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

int check_cache(const vlut_cache* c) {
    if (!c || !c->k || !c->v) return VLUT_ERR_NULL;
    if (c->type != VLUT_TYPE_BF16 && c->type != VLUT_TYPE_F16) return VLUT_ERR_UNSUPPORTED;
    if (c->heads < 1 || c->heads >= (1 << 16) || c->pages < 1 || c->page_size < 1) return VLUT_ERR_SHAPE;
    if (!power_of_two(c->page_size) || c->page_size > 65536) return VLUT_ERR_UNSUPPORTED;
    return VLUT_OK;
}

// Rows that start at a dword.
bool at_dwords(const void* p, int64_t s0, int64_t s1, int64_t s2, int bytes) {
    return (uintptr_t)p % 4 == 0 && (bytes == 4 || (s0 % 2 == 0 && s1 % 2 == 0 && s2 % 2 == 0));
}

}  // namespace
