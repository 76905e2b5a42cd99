// The launches of attention_launch_driver.cpp at the largest numbers of each type that calls take.
#define main launch_driver
#include "attention_launch_driver.cpp"
#undef main

int main()
{
    for (grawa_dtype_t dt : {GRAWA_F32, GRAWA_BF16})
        for (int D : {8, 128})
            for (int buckets : {0, 256}) {
                call(1024, 1024, 1024, 1024, 1, 1, D, dt, 0, 0, buckets, 0, 0);
                call(1, 1, 1 << 28, 1 << 28, 4, 1, D, dt, 4096, 5, buckets, 0, 0);
                call(1, 1, 1 << 28, 1 << 28, 4, 4, D, dt, 0, 0, buckets, 0, 0);
                call(1, 65, 1 << 17, 1 << 17, 126, 1, D, dt, 9, 0, buckets, 8, 1);  // groups that eight does not divide
                call(1, 1, 1 << 16, 1 << 16, 1 << 14, 1, D, dt, 7, 0, buckets, 0, 0);
                call(3, 349525, 1023, 1023, 1, 1, D, dt, 7, 3, buckets, 0, 0);
                call(1, 1 << 20, 1, 1024, 1, 1, D, dt, 0, 0, buckets, 0, 0);
            }
    what = "";
    expect(launches > 100, "calls that launch");
    if (failures) {
        std::printf("%d failures\n", failures);
        return 1;
    }
    std::printf("ok\n");
    return 0;
}
