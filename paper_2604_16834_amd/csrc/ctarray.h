// Checks of a vector of ciphertexts at equal distances (he_ct_array), host only and without the context, so that they can be tested without a GPU.
#pragma once
#include <stddef.h>
#include <stdint.h>

#include "../../include/ckks.h"

// What is wrong with a vector of n ciphertexts of which `limbs` limbs of n_comp components are read, or null: what the kernels' 16-byte loads and indexes
// assume.  Kernels and entry points multiply strides by counts of ciphertexts up to n in 64 bits: no stride passes 2^40
// words, and none times n 2^59.
inline const char* ct_array_fault(const he_ct_array* a, uint64_t n, uint32_t limbs, uint32_t n_comp, uint32_t N) {
    if (!a || !a->d) return "null ciphertext array";
    const uint64_t one = (uint64_t)limbs * N, most = (uint64_t)1 << 40, all = (uint64_t)1 << 59;
    if (((uintptr_t)a->d & 15) || (a->ct_stride & 1) || (n_comp > 1 && (a->comp_stride & 1)))
        return "ciphertext array: not aligned to 16 bytes, or an odd stride";
    if (a->ct_stride > most || (n > 1 && a->ct_stride > all / n) || (n_comp > 1 && a->comp_stride > most)) return "ciphertext array: stride out of range";
    if (n_comp > 1 && a->comp_stride < one) return "ciphertext array: components overlap";
    if (n > 1 && a->ct_stride != 0 && a->ct_stride < (n_comp > 1 ? a->comp_stride : 0) + one) return "ciphertext array: ciphertexts overlap";
    return nullptr;
}
