"""The runner of searches, its calls' plain statements in their place: no kernel is launched by anything in this file."""
import math

import beam_story


def test_a_group_that_waits_for_pages_goes_on_as_it_was(monkeypatch):
    """With `hold`, a group that a fork refuses has the scores and ends that belong to the rows that it has, and its next steps are those of a search that never waited."""
    beam_story.plain_calls(monkeypatch)
    assert beam_story.waits_and_goes_on(lambda n: beam_story.runner(4, 3, n, "cpu", hold=True), lambda r: r.step) > 3


def test_a_prompt_that_found_no_room_starts_no_search(monkeypatch):
    """A group whose prompt the pool had no pages for has no tokens to search from: `spread` leaves it as it was, whatever it is told, and a later admission starts it."""
    beam_story.plain_calls(monkeypatch)
    for hold in (False, True):
        s = beam_story.Story(beam_story.runner(4, 3, 8, "cpu", hold=hold), [30, 45, 100])        # 2 and 3 pages of 8, and 7 that there are not
        assert s.r.lens.tolist() == [30] * 4 + [45] * 4 + [0] * 4
        scores = s.r.scores.view(3, 4).tolist()
        assert scores == [[0.0] + [-math.inf] * 3] * 2 + [[-math.inf] * 4]
        s.step(s.r.step)
        assert s.r.lens.tolist()[8:] == [0] * 4 and s.r.parents.tolist()[8:] == [-1] * 4 and s.r.scores.tolist()[8:] == [-math.inf] * 4
        s.r.finish(beam_story.i32([1, 1, 0]))
        s.admit([0, 0, 100])
        assert s.r.lens.tolist() == [0] * 8 + [100] * 4 and s.r.scores.tolist()[8:] == [0.0] + [-math.inf] * 3
