// The K-th largest of a row's ranked keys by bisection over their bits: the control flow of the exact search of ulorl_token_topk.
// No device code: the tests compile it by itself.
#ifndef ULORL_KTH_KEY_HPP
#define ULORL_KTH_KEY_HPP

#include <stdint.h>

namespace ulorl_detail {

// A ranked key has the order of the logit in its upper half and 0xffffffff - id in its lower one; 0: masked.  Returns a key that exactly
// K of the keys reach, all of them where there are fewer; ids are below n.  Of the lower half only the bits that ids differ in are looked
// for.
//
// count(c, turn): how many keys reach c, the same in every thread.  turn is 0, 1, 2, ... over the calls that are made, whatever bits
// are left out between them: threads that count through two buffers by turns, with one barrier a call, need every call to
// take the other buffer than the last one, which a slow wave may still be reading.
template <class Count>
constexpr uint64_t kth_key(uint32_t K, uint32_t n, const Count& count)
{
    const int id_bits = 32 - __builtin_clz(n);
    uint64_t t = 0;
    int turn = 0;
    for (int bit = 63; bit >= 0; --bit) {
        if (bit < 32 && bit >= id_bits) {
            t |= 1ull << bit;
            continue;
        }
        const uint64_t c = t | (1ull << bit);
        const uint32_t reach = count(c, turn++);
        if (reach >= K) t = c;
        if (reach == K) break;
    }
    return t;
}

}  // namespace ulorl_detail

#endif
