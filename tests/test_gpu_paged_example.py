"""The example: captured steps whose groups change, and its command line."""
import pytest
import torch

from test_gpu_paged import status
from test_gpu_paged_stack import hidden, mod, near  # noqa: F401
from test_gpu_paged_together import shared_and_alone

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("weights", [False, True])
def test_a_captured_step_follows_places_that_begin_anew(mod, weights):  # noqa: F811
    """Steps captured while places 0 to 4 share a prompt, replayed after one of them has become another
    sequence, after others share again, and after all have shed: as steps without groups."""
    st, alone = shared_and_alone(mod, weights)
    for t in (st, alone):
        t.table.grow(3)
    x = hidden(6, 80)
    y = st.capture(x)

    def steps(seed):
        for i in range(3):
            x.copy_(hidden(6, seed + i))
            st.replay()
            want = alone.step(x)
            assert near(y[:5], want[:5])
            assert torch.isfinite(y).all()
    steps(81)
    held = st._captured
    other = hidden(150, 90)
    for t in (st, alone):
        t.table.close(2)
        t.table.open(2)
        t.chunk(other, [0, 0, 150, 0, 0, 0])
    steps(91)
    torch.cuda.empty_cache()
    waste = [torch.full((n,), 2 ** 30, dtype=torch.int32, device="cuda") for n in (1, 2, 3, 4, 5, 6, 7) for _ in range(50)]
    st.share(2, [3], 100)                              # (96 tokens of the new sequence)
    alone.table.close(3)
    alone.table.open(3)
    alone.chunk(other[:96], [0, 0, 0, 96, 0, 0])
    steps(101)
    assert st._captured is held and all((w == 2 ** 30).all() for w in waste)
    if weights:                                        # (what the two keep need not be the same positions)
        st.shed(80, sinks=4, window=16)
        before = st.table.lens.clone()
        for i in range(3):
            st.replay()
        assert torch.isfinite(y).all() and torch.equal(st.table.lens, torch.where(before < 0, before, before + 3))
    st.check()
    alone.check()
    assert status()[0] == 0


@pytest.mark.parametrize("argv", [["--keep", "128"], ["--keep", "40"], ["--shared", "200"], ["--shared", "200", "--batch", "1"],
                                  ["--shared", "130", "--keep", "100"], []])
def test_the_command_line(mod, monkeypatch, capsys, argv):  # noqa: F811
    monkeypatch.setattr("sys.argv", ["paged_stack.py", "--layers", "2", "--batch", "5", "--hidden", "256", "--kv-heads", "2",
                                     "--q-per-kv", "2", "--head-dim", "64", "--prompt", "300", "--chunk", "128",
                                     "--steps", "5"] + argv)
    mod.main()
    assert "tokens/s" in capsys.readouterr().out
    assert status()[0] == 0
