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
