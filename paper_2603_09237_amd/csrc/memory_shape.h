// Where things lie in LDS, for the kernels and for a host compiler.
#pragma once

#if defined(__HIPCC__)
#define MEM_HD __host__ __device__
#else
#define MEM_HD
#endif

// A wave of the single step: the convolved values of its channels (`each`, or fewer), then B, then C, one run of floats that is laid so that B
// begins at sixteen bytes, and with it C where the state is a multiple of four: then both are read as whole pieces.
struct StepLayout {
    int each, b, wave;  // channels of a wave; where B begins; floats of a wave
};
MEM_HD inline StepLayout step_layout(int head_dim, int state, int parts) {
    StepLayout l;
    l.each = (head_dim + parts - 1) / parts;
    l.b = (l.each + 3) / 4 * 4;
    l.wave = (l.b + 2 * state + 3) / 4 * 4;
    return l;
}
