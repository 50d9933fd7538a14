"""What the operators' entry points do with a launch: its status and its size."""
from _fake_cuda import run


def test_a_call_answers_for_its_own_launch_alone(tmp_path):
    # An error that an earlier call of this thread has left is not this call's: its kernel is queued.  A launch that is refused is.
    out = run(tmp_path, """
    for (int refused = 0; refused < 2; ++refused) {
        auto begin = [&] { stale = refused ? cudaSuccess : cudaErrorInvalidDevice; refuse = refused ? cudaErrorInvalidConfiguration : cudaSuccess; launches = 0; };
        auto say = [&](mpode_status s) { printf("%d:%lld ", (int)s, launches); };
        begin(); say(mpode_dropout(MPODE_BF16, nullptr, 64, 64, at(0), 0, to(1), 0, 0.5f, at(2), 0, nullptr));
        begin(); say(mpode_dropout(MPODE_F16, nullptr, 64, 13, at(0), 0, to(1), 0, 0.5f, at(2), 0, nullptr));
        for (int steps : {1, 40}) {
            mpode_recurrence_desc d{MPODE_BF16, 2, steps, 64, 1, 0, 0, 0, 0, 0};
            begin(); say(mpode_recurrence_forward(&d, nullptr, at(0), at(1), nullptr, nullptr, to(2), nullptr));
        }
        mpode_residual_desc r{MPODE_BF16, 64, MPODE_NORM_RMS, MPODE_NORM_RMS, 1e-5f, 1.f, 0.f, 0, 0, 0, 0, 0};
        begin(); say(mpode_residual_forward(&r, nullptr, 8, (const float*)at(0), at(1), nullptr, nullptr, nullptr, nullptr, nullptr, (float*)to(2), to(3), nullptr));
    }""")
    assert out == ["0:1"] * 5 + ["4:1"] * 5


def test_the_largest_sizes_have_grids(tmp_path):
    # 2^31 - 1 columns or rows: rounding up to whole groups once left 32 bits, and the launch was refused
    out = run(tmp_path, """
    for (int width : {0x7fffffff, 0x7ffffff9, 0x7ffffff8}) {
        launches = 0; grid = dim3(0);
        const mpode_status s = mpode_dropout(MPODE_BF16, nullptr, 1, width, at(0), 0, to(1), 0, 0.5f, at(2), 0, nullptr);
        printf("%d:%lld:%u ", (int)s, launches, grid.x);
    }
    for (int rows : {0x7fffffff, 0x7ffffff9, 0x7ffffff8}) {
        launches = 0; grid = dim3(0);
        mpode_residual_desc r{MPODE_BF16, 8, MPODE_NORM_RMS, MPODE_NORM_RMS, 1e-5f, 1.f, 0.f, 0, 0, 0, 0, 0};
        const mpode_status s = mpode_residual_forward(&r, nullptr, rows, (const float*)at(0), at(1), nullptr, nullptr, nullptr, nullptr, nullptr, (float*)to(2), to(3), nullptr);
        const size_t n = mpode_residual_workspace_bytes(&r, rows);
        printf("%d:%lld:%d:%d ", (int)s, launches, grid.x >= 1 && grid.x <= 65536, n >= 64 && n <= (1u << 30));
    }""")
    assert out == ["0:1:2368"] * 3 + ["0:1:1:1"] * 3


def test_weight_gradients_in_one_buffer_are_added_one_after_another(tmp_path):
    # One kernel that writes them all would race where two of them lie over one another.  Overwriting one another has no meaning and is refused.
    out = run(tmp_path, """
    mpode_residual_desc r{MPODE_BF16, 64, MPODE_NORM_RMS, MPODE_NORM_RMS, 1e-5f, 1.f, 0.f, 0, 0, 0, 0, 0};
    auto call = [&](int post, int scale, int pre, int off, int accumulate) {
        launches = 0;
        auto grad = [&](int i) { return i ? (float*)to(i) : nullptr; };
        const mpode_status s = mpode_residual_backward(&r, nullptr, 8, (const float*)at(0), at(1), at(2), (const float*)at(3), (const float*)at(4), (const float*)at(5), nullptr,
            (const float*)at(6), (const float*)at(7), at(8), 0, (float*)to(9), to(10), to(11), grad(post), grad(scale), pre ? grad(pre) + off : nullptr, accumulate, nullptr, to(20), 1 << 24);
        printf("%d:%lld ", (int)s, launches);
    };
    for (int accumulate : {0, 1}) {
        call(12, 13, 14, 0, accumulate);
        call(12, 13, 12, 0, accumulate);
        call(12, 12, 12, 0, accumulate);
        call(0, 12, 12, 0, accumulate);
        call(12, 0, 12, 63, accumulate);
        call(12, 0, 12, 64, accumulate);
        call(0, 0, 12, 0, accumulate);
    }""")
    assert out == ["0:2", "1:0", "1:0", "1:0", "1:0", "0:2", "0:2"] + ["0:2", "0:4", "0:4", "0:3", "0:3", "0:2", "0:2"]


def test_a_question_that_failed_is_asked_again(tmp_path):
    # How many clusters the device holds: one call's failure to tell must not decide every later call's shape
    out = run(tmp_path, """
    mpode_recurrence_desc d{MPODE_BF16, 1, 5000, 64, 1, 0, 0, 0, 0, 0};
    mpode_residual_desc r{MPODE_BF16, 8192, MPODE_NORM_RMS, MPODE_NORM_RMS, 1e-5f, 1.f, 0.f, 0, 0, 0, 0, 0};
    for (int k = 0; k < 3; ++k) {
        occupancy = k == 0 ? cudaErrorMemoryAllocation : cudaSuccess;
        mpode_recurrence_forward(&d, nullptr, at(0), at(1), nullptr, nullptr, to(2), nullptr);
        printf("%u ", grid.x);
        mpode_residual_forward(&r, nullptr, 1000, (const float*)at(0), at(1), nullptr, nullptr, nullptr, nullptr, nullptr, (float*)to(2), to(3), nullptr);
        printf("%u ", grid.x);
    }""")
    # one sequence of 64 channels: a block, or a cluster of 16; rows of four blocks: as many as the grid's limit holds, or the 8 clusters that fit
    assert out == ["1", "592", "16", "32", "16", "32"]
