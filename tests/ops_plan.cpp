// Prints norm_grad_streams (forge_ops_internal.h) for lines of "T d h_bf16 dres" on stdin.
#include <cstdio>

#include "forge_ops_internal.h"

int main()
{
    long long T, d;
    int h_bf16, dres;
    while (std::scanf("%lld %lld %d %d", &T, &d, &h_bf16, &dres) == 4)
        std::printf("%d\n", forge_impl::norm_grad_streams(T, d, h_bf16, dres));
    return 0;
}
