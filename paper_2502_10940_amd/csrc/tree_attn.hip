// tree_attn.hip -- the kernels of cola_tree_attn: those of prefix_attn.hpp, where a
// request's new tokens see each other by their masks.
#include "prefix_attn.hpp"

namespace cola {
namespace {

template <int HD>
hipError_t go(const PrefixAttnPlan& p, const Args& a, unsigned grid, hipStream_t s) {
#define COLA_GO(P, S) \
    if (p.kind_p == P && p.kind_s == S) prefix_attn_kernel<HD, P, S, SEE_TREE><<<grid, NTHR, 0, s>>>(a)
    COLA_GO(ALONG, ONE);
    else COLA_GO(ALONG, TWO);
    else COLA_GO(ALONG, WIDE);
    else COLA_GO(ONE, ONE);
    else COLA_GO(TWO, ONE);
    else COLA_GO(TWO, TWO);
    else COLA_GO(WIDE, ONE);
    else COLA_GO(WIDE, TWO);
    else COLA_GO(WIDE, WIDE);
    else return hipErrorInvalidValue;
#undef COLA_GO
    return hipGetLastError();
}

}  // namespace

hipError_t start_tree_attn(int hd, const PrefixAttnPlan& p, const void* args, unsigned grid, hipStream_t s) {
    const Args& a = *static_cast<const Args*>(args);
    return hd == 64 ? go<64>(p, a, grid, s) : go<128>(p, a, grid, s);
}

}  // namespace cola
