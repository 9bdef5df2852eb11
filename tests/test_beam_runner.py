"""The runner of searches, its calls' plain statements in their place: no kernel is launched by anything in this file."""
import beam_story


def test_a_group_that_waits_for_pages_goes_on_as_it_was(monkeypatch):
    """With `hold`, a group that a fork refuses has the scores and ends that belong to the rows that it has, and its next steps are those of a search that never waited."""
    beam_story.plain_calls(monkeypatch)
    assert beam_story.waits_and_goes_on(lambda n: beam_story.runner(4, 3, n, "cpu", hold=True), lambda r: r.step) > 3
