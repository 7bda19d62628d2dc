"""The example's stack: groups of sequences that share prompts, as places come and go (no GPU)."""
from test_paged_stack_room import full, stack


def test_sharing_with_nobody():
    st = stack(batch=1)
    full(st, [200])
    assert st.share(0, [], 100) == 0 and st.groups == (None, None)


def test_changes_of_a_table():
    st = stack(batch=4)
    t, seen = st.table, []

    def count(call):
        call()
        seen.append(t.changes)
    for call in (lambda: t.open(0), lambda: t.grow([300, 0, 0, 0]), lambda: t.advance([300, 0, 0, 0]),
                 lambda: t.share(0, 1, 256), lambda: t.close(1), lambda: t.open(1), lambda: t.grow(1),
                 lambda: t.advance_held(1), lambda: t.close(0)):
        count(call)
    assert seen == [1, 1, 1, 2, 2, 3, 3, 3, 3]
    t.shrink(10)
    assert t.changes == 3
    t.shrunk()
    assert t.changes == 4


def test_groups_of_a_captured_step_follow_the_table():
    """They keep their memory, and are the table's, or fewer: never of a sequence that is no longer there."""
    st = stack(batch=6)
    t = st.table
    full(st, [200] + [0] * 5)
    st.share(0, [1, 2], 200)
    t.open(3)
    t.grow([0, 0, 0, 130, 0, 0])
    t.advance([0, 0, 0, 130, 0, 0])
    assert st.groups[0].tolist() == [0, 3, 6] and st.groups[1].tolist() == [192, 0]
    st._captured = st.groups                            # as capture does
    first, prefix = st._captured
    t.open(1)                                           # another sequence in the group's midst
    st.regroup()
    assert st._captured[0] is first and st._captured[1] is prefix
    assert st.groups[0] is None and prefix.tolist() == [0, 0] and first.tolist() == [0, 3, 6]
    st.share(3, [4], 130)
    assert st.groups[0].tolist() == [0, 3, 5, 6] and st.groups[1].tolist() == [0, 128, 0]
    assert first.tolist() == [0, 3, 5] and prefix.tolist() == [0, 128]
    st.share(0, [1], 200)                               # three groups, and room for two
    st.share(3, [5], 130)
    assert first.tolist() == [0, 3, 6] and prefix.tolist() == [192, 128]
    t.open(0)
    t.open(1)
    st.regroup()
    assert first.tolist() == [0, 3, 6] and prefix.tolist() == [0, 128]
