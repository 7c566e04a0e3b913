// Where things lie in LDS, for the kernels and for a host compiler.
#pragma once

#if defined(__HIPCC__)
#define MEM_HD __host__ __device__
#else
#define MEM_HD
#endif

// A wave of the single step: the convolved values of its `each` channels, then B, then C, as floats from the wave's start; every part begins
// at sixteen bytes, whatever the sizes, for B and C are read as whole pieces where the state is a multiple of four.
struct StepLayout {
    int each, b, c, wave;  // channels of a wave; where B and C begin; floats of a wave
};
MEM_HD inline int up4(int n) { return (n + 3) / 4 * 4; }
MEM_HD inline StepLayout step_layout(int head_dim, int state, int parts) {
    StepLayout l;
    l.each = (head_dim + parts - 1) / parts;
    l.b = up4(l.each);
    l.c = l.b + up4(state);
    l.wave = l.c + up4(state);
    return l;
}
