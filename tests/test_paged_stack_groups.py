"""The example's stack: groups of sequences that share prompts, as places come and go (no GPU)."""
from test_paged_stack_room import full, stack


def test_sharing_with_nobody():
    st = stack(batch=1)
    full(st, [200])
    assert st.share(0, [], 100) == 0 and st.groups == (None, None)
