"""The sizes that the GPU tests of the norm and the update run reach every way in which a call takes its tensors."""
import update_rules as R


def test_gpu_tests_reach_every_form():
    import test_gpu_update as S
    import test_gpu_update_large as G
    sets = S.SETS + G.LARGE_SETS
    clip = {R.clip_form(s) for s in sets}
    assert ("one workgroup",) in clip
    several = [f for f in clip if f[0] == "launches"]
    assert {f[1] for f in several} == {1024, 2048, 4096, 8192}                 # chunks of the norm,
    assert {f[2] for f in several} == {1024, 2048, 4096}                       # and of clipping
    for k in (3, 4, 5):                                                         # slots, launches of the norm and of clipping
        assert len({f[k] for f in several}) == 2, k
    assert any(f[3:5] == ("one slot", "several") for f in several)              # a norm added up over launches, read from one slot
    for clipped in (False, True):
        update = {R.adamw_form(s, clipped) for s in sets}
        assert {f[:2] for f in update} == {("small", 1024), ("small", 2048), ("large", 2048)}
        if clipped:
            assert any(f[2] == "norm here" for f in update)
            assert {(f[0], f[2]) for f in update} >= {("small", "slots"), ("small", "one slot"), ("large", "one slot")}
            assert any(f[2:4] == ("one slot", "several") and f[0] == "large" for f in update)
        assert {f[-1] for f in update if f[2] != "norm here"} == {"one", "several"}


def test_borders_of_the_update():
    bar = 16 << 20
    assert R.adamw_form([bar], True)[0] == "small" and R.adamw_form([bar + 1], True)[0] == "large"
    adamw = R.tensors_of_a_launch()[2]
    assert R.adamw_form([1] * adamw, True)[2] == "norm here" != R.adamw_form([1] * (adamw + 1), True)[2]


def test_one_workgroup_clips_few_chunks():
    """Its waves go round once for sixteen chunks, and every tensor is one at least: 144 tensors of 50 elements took it 26 us, launches 10."""
    for sizes in ([32768], [20480] + [50] * 16, [64 * 64, 64 * 64, 64, 64 * 16, 64 * 16, 16], [50] * 40, [0] * 500 + [7]):
        assert R.clip_form(sizes) == ("one workgroup",), sizes
    for sizes in ([32769], [50] * 70, [50] * 144, [1] * 60, [20480] + [50] * 60):
        assert R.clip_form(sizes) != ("one workgroup",), sizes
