// tree_attn.hip -- the kernels of cola_tree_attn: those of prefix_attn.hpp, where a
// request's new tokens see each other by their masks.
#include "prefix_attn.hpp"

namespace cola {
namespace {

template <int HD>
hipError_t go(const PrefixAttnPlan& p, const Args& a, unsigned grid, hipStream_t s) {
#define COLA_GO(P, S, C)                                      \
    if (p.kind_p == P && p.kind_s == S && (a.slots > 0) == C) \
    prefix_attn_kernel<HD, P, S, SEE_TREE, C><<<grid, NTHR, 0, s>>>(a)
    COLA_GO(ALONG, ONE, false);
    else COLA_GO(ALONG, TWO, false);
    else COLA_GO(ALONG, WIDE, false);
    else COLA_GO(ONE, ONE, false);
    else COLA_GO(TWO, ONE, false);
    else COLA_GO(TWO, TWO, false);
    else COLA_GO(WIDE, ONE, false);
    else COLA_GO(WIDE, TWO, false);
    else COLA_GO(WIDE, WIDE, false);
    else COLA_GO(WIDE, WIDE, true);
    else if constexpr (HD == 64) {
        COLA_GO(ALONG, FOUR, false);
        else COLA_GO(FOUR, FOUR, false);
        else return hipErrorInvalidValue;
    } else return hipErrorInvalidValue;
#undef COLA_GO
    return hipGetLastError();
}

}  // namespace

hipError_t start_tree_attn(int hd, const PrefixAttnPlan& p, const void* args, unsigned grid, hipStream_t s) {
    const Args& a = *static_cast<const Args*>(args);
    return hd == 64 ? go<64>(p, a, grid, s) : go<128>(p, a, grid, s);
}

}  // namespace cola
