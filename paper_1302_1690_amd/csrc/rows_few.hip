// Instances of the class layer's kernels on few rows of features, one per number of rows.
#include "kernels_rows_few.hpp"

namespace mpcnn {

template <typename T>
void launch_rows_few_scores(const FewArgs& a, unsigned groups, hipStream_t st)
{
    static_assert(kFewScoreRows == 12, "a case each");
    switch (a.N) {
#define CASE(n) case n: rows_few_scores_kernel<T, n><<<groups, kFewThreads, 0, st>>>(a); break;
        CASE(1) CASE(2) CASE(3) CASE(4) CASE(5) CASE(6) CASE(7) CASE(8) CASE(9) CASE(10) CASE(11) CASE(12)
#undef CASE
    }
}
template <typename T>
void launch_rows_few_grads(const FewArgs& a, dim3 grid, hipStream_t st)
{
    static_assert(kFewRows == 16, "a case each");
    switch (a.N) {
#define CASE(n) case n: rows_few_grads_kernel<T, n><<<grid, kFewThreads, 0, st>>>(a); break;
        CASE(1) CASE(2) CASE(3) CASE(4) CASE(5) CASE(6) CASE(7) CASE(8) CASE(9) CASE(10) CASE(11) CASE(12) CASE(13) CASE(14) CASE(15) CASE(16)
#undef CASE
    }
}
template <typename T>
void launch_rows_few_sum(const FewArgs& a, unsigned groups, hipStream_t st)
{
    rows_few_sum_kernel<T><<<groups, 1024, 0, st>>>(a);
}
template void launch_rows_few_scores<float>(const FewArgs&, unsigned, hipStream_t);
template void launch_rows_few_scores<bf16>(const FewArgs&, unsigned, hipStream_t);
template void launch_rows_few_grads<float>(const FewArgs&, dim3, hipStream_t);
template void launch_rows_few_grads<bf16>(const FewArgs&, dim3, hipStream_t);
template void launch_rows_few_sum<float>(const FewArgs&, unsigned, hipStream_t);
template void launch_rows_few_sum<bf16>(const FewArgs&, unsigned, hipStream_t);

}  // namespace mpcnn
