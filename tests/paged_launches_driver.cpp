// Driver for tests/test_paged_launches.py: the largest calls of the paged cache that pd.h allows, on the stand-in for the HIP runtime of
// host_launches_driver.cpp, which refuses a launch where the GPU would refuse its grid.  No pointer is read.
#define main layer_calls
#include "host_launches_driver.cpp"
#undef main

int main()
{
    char *some = (char *)0x100000;          // aligned, and never touched
    struct Kind { pd_dtype dtype; int e4m3; } kinds[] = {{PD_BF16, 0}, {PD_F32, 0}, {PD_BF16, 1}};
    struct Size { int rows, seqs, hq, hkv; } sizes[] = {{1 << 24, 1, 32, 32},   {1 << 24, 4096, 64, 8},  {1 << 24, 4096, 0, 1024}, {7500000, 64, 32, 32},
                                                        {(1 << 21) - 1, 4096, 1024, 1024}, {(1 << 21) - 1, 1, 1024, 1}, {4096, 4096, 1024, 1024}, {1, 1, 1, 1}};
    int calls = 0;
    for (const Kind &k : kinds)
        for (const Size &z : sizes)
            for (int starts = 0; starts < 2; ++starts)
                for (int ps = 16; ps <= 128; ps *= 8)
                    for (int hd = 64; hd <= 128; hd += 64) {
                        if (z.hq > 0 && (int64_t)z.rows * z.hq >= 1ll << 31) continue;
                        pd_paged_kv kv = {some, some, (float *)some, (float *)some, 1 << 20, ps, z.hkv, hd, k.dtype, k.e4m3};
                        pd_paged_seqs seqs = {z.seqs, z.rows, starts ? (const int32_t *)some : nullptr, (const int32_t *)some, (const int32_t *)some, (1 << 30) / ps};
                        pd_paged_rows rows = {some, some, z.hq ? some : nullptr, z.hq ? some : nullptr, (int64_t)z.hkv * hd, (int64_t)z.hkv * hd, (int64_t)z.hq * hd,
                                              (int64_t)z.hq * hd, z.hq, 1e4f};
                        CHECK(pd_paged_append(&kv, &seqs, &rows, nullptr) == PD_OK && !g_refused, "append of %d rows, %d sequences, %d heads on %d: %s", z.rows, z.seqs,
                              z.hq, z.hkv, pd_last_error());
                        ++calls;
                        if (!z.hq) continue;
                        int64_t bytes = -1;
                        CHECK(pd_paged_attention_workspace(&kv, &seqs, z.hq, &bytes) == PD_OK && bytes >= 0 && bytes < 256ll << 20, "workspace %lld", (long long)bytes);
                        CHECK(pd_paged_attention(&kv, &seqs, some, (int64_t)z.hq * hd, z.hq, 0.1f, some, some, bytes, nullptr) == PD_OK && !g_refused,
                              "attention of %d rows, %d sequences, %d heads on %d: %s", z.rows, z.seqs, z.hq, z.hkv, pd_last_error());
                        ++calls;
                    }
    printf("ok %d calls, %ld launches\n", calls, g_launches);
    return 0;
}
