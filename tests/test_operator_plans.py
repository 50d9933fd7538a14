"""What the operators' kernels are told to touch, decided in code that runs on the host as well: compiled into a small program and looked over without a device."""
import subprocess


def _run(tmp_path, header, body):
    """Compile `body` (the inside of main, with a header of the library) and return what it prints."""
    from paper_2510_23498_b200 import build
    src = tmp_path / "t.cu"
    src.write_text('#include <stdio.h>\n#include "%s"\nusing namespace mpode;\nint main() {\n%s\nreturn 0; }\n' % (header, body))
    exe = str(tmp_path / "t")
    subprocess.run([build._nvcc(), "-gencode", "arch=compute_100a,code=sm_100a", "-std=c++17", "-I", build.CSRC, str(src), "-o", exe], check=True)
    return subprocess.run([exe], check=True, capture_output=True, text=True, timeout=60).stdout.split()


def test_the_recurrence_copies_no_row_behind_a_sequences_length(tmp_path):
    # Every tile of every warp in every round: a tile that is copied holds no row behind the length (rows below 0 and from n_steps on are clipped by the tensor), and
    # without a length all tiles that hold a row are copied.  Backward also for the tile of the states in front, one row earlier.
    out = _run(tmp_path, "recurrence_tiles.h", """
    long long beyond = 0, left = 0, copies = 0, late = 0;
    for (unsigned steps : {4u, 8u, 16u})
        for (unsigned slots : {1u, 3u})
            for (unsigned n_steps = 1; n_steps <= 70; ++n_steps)
                for (unsigned len = 0; len <= n_steps; ++len)
                    for (unsigned slot = 0; slot < slots; ++slot) {
                        const unsigned stride = slots * steps, skipped = n_steps - len;
                        for (unsigned base = 0; base < len; base += stride) {                          // forward
                            const bool copied = base < copied_below(slot * steps, steps, len, n_steps);
                            const long long t0 = base + slot * steps;
                            for (long long t = t0; t < t0 + steps; ++t) beyond += copied && t < n_steps && t >= len;
                            left += !copied && (len == n_steps || t0 + steps <= len);
                            copies += copied;
                        }
                        const unsigned begin = skipped / stride * stride;
                        for (unsigned base = begin; base < n_steps; base += stride) {                  // backward
                            const bool copied = copied_back(base + slot * steps, skipped);
                            const long long t0 = (long long)n_steps - base - slot * steps - steps;
                            for (long long t = t0 - 1; t < t0 + steps; ++t) beyond += copied && t >= 0 && t < n_steps && t >= len;
                            left += !copied && len == n_steps;
                            late += !copied && base != begin;                                          // (the kernel asks in the first round alone)
                            copies += copied;
                        }
                    }
    printf("%lld %lld %lld %d %u\\n", beyond, left, late, copies > 10000, copied_below(0u, 16u, 0x7ffffffeu, 0x7fffffffu) == 0x7fffffefu);""")
    assert out == ["0", "0", "0", "1", "1"]
