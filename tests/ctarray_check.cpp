// Host check of the vectors that ct_array_fault lets through: with exact (128-bit) arithmetic, no offset that a kernel or an entry point forms from a stride and a
// count of ciphertexts passes 64 bits, and the layouts that a program has are accepted.  Prints what fails and returns 1.
#include <cstdio>

#include "../paper_2604_16834_amd/csrc/ctarray.h"

static int bad = 0;
static void expect(bool ok, const char* what, uint64_t ct, uint64_t comp, uint64_t n) {
    if (ok) return;
    printf("%s: ct_stride %llu comp_stride %llu n %llu\n", what, (unsigned long long)ct, (unsigned long long)comp, (unsigned long long)n);
    bad = 1;
}

int main() {
    alignas(16) static uint64_t words[4];
    const uint64_t counts[] = {1, 2, 3, 64, 65536, (uint64_t)1 << 24, ((uint64_t)1 << 40) - 1, (uint64_t)1 << 40};
    const uint32_t limbs = 2, N = 16;
    unsigned accepted = 0;
    for (uint64_t n : counts)
        for (uint32_t comps = 1; comps <= 2; comps++)
            for (int cs = 0; cs < 64; cs++)
                for (int ps = 0; ps < 64; ps++)
                    for (uint64_t less = 0; less <= 2; less += 2) {
                        const he_ct_array a = {words, ((uint64_t)1 << cs) - (cs > 1 ? less : 0), ((uint64_t)1 << ps) - (ps > 1 ? less : 0)};
                        if (ct_array_fault(&a, n, limbs, comps, N)) continue;
                        accepted++;
                        // one past the last word that is read, and a step past the last row of a loop over rows: all in bytes
                        const unsigned __int128 words_in_all = (unsigned __int128)a.ct_stride * n + (comps > 1 ? a.comp_stride : 0) + limbs * N;
                        expect(words_in_all * 8 < (unsigned __int128)1 << 64, "offset passes 64 bits", a.ct_stride, a.comp_stride, n);
                    }
    expect(accepted > 1000, "hardly anything accepted", 0, 0, accepted);
    // what programs have: compact vectors of the largest ciphertexts, one ciphertext in the place of all, 2^40 of them
    const uint64_t comp = (uint64_t)64 << 17, ct = 2 * comp;
    const he_ct_array compact = {words, ct, comp}, same = {words, 0, comp};
    for (uint64_t n : counts) {
        expect(n > ((uint64_t)1 << 34) || !ct_array_fault(&compact, n, 64, 2, 1 << 17), "compact vector refused", ct, comp, n);
        expect(!ct_array_fault(&same, n, 64, 2, 1 << 17), "repeated ciphertext refused", 0, comp, n);
    }
    // and what is refused
    const he_ct_array close = {words, comp, comp}, odd = {words, ct + 1, comp}, overlap = {words, ct, comp - 2}, wide = {words, (uint64_t)1 << 40, comp};
    expect(ct_array_fault(&close, 2, 64, 2, 1 << 17) != nullptr, "overlapping ciphertexts", comp, comp, 2);
    expect(ct_array_fault(&odd, 2, 64, 2, 1 << 17) != nullptr, "odd stride", ct + 1, comp, 2);
    expect(ct_array_fault(&overlap, 2, 64, 2, 1 << 17) != nullptr, "overlapping components", ct, comp - 2, 2);
    expect(ct_array_fault(&wide, (uint64_t)1 << 40, 64, 2, 1 << 17) != nullptr, "2^80 words", wide.ct_stride, comp, (uint64_t)1 << 40);
    const he_ct_array null_words = {nullptr, ct, comp};
    expect(ct_array_fault(&null_words, 1, 64, 2, 1 << 17) != nullptr && ct_array_fault(nullptr, 1, 64, 2, 1 << 17) != nullptr, "null", 0, 0, 1);
    return bad;
}
