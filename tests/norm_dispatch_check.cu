// Prints, for (rows, columns, whether dgamma or dbeta is wanted) from standard input, how many owners the backward pass of the layer norm has
// and whether their sums are joined in a cluster (no GPU needed).
#include <cstdio>

#include "rocket_norm_backward.cuh"

int main() {
    int N, P, weights;
    while (std::scanf("%d %d %d", &N, &P, &weights) == 3)
        std::printf("%d %d\n", rocket::norm::owners_of(N, P, weights != 0), weights && rocket::norm::is_joined(N, P) ? 1 : 0);
    return 0;
}
