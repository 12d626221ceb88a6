"""Profiles with prompts: what is refused before anything is measured."""
import pytest


def test_a_prompt_that_its_cache_would_cut_is_refused():
    from paper_2302_11665_amd import served
    shape = served.Shape(layers=2, hidden=64, heads=2, kv_heads=1, dim=64, inner=128, budget=96, slack=32)
    for prompt, tokens in ((119, 10), (128, 1), (5000, 10), (-1, 10)):
        with pytest.raises(ValueError, match="prompt"):
            served.measure(shape, tokens=tokens, prompt=prompt)


def test_what_is_counted_holds_a_request_with_its_prompt(monkeypatch):
    """The longest prompt that is taken: its pages and its tokens' are within the bytes of a request's cache."""
    from paper_2302_11665_amd import served
    shape = served.Shape(layers=3, hidden=64, heads=2, kv_heads=1, dim=64, inner=128, budget=97, slack=32, page=32)
    seen, per_page = [], 10_000_000

    class Block:
        nbytes = 0

        def __init__(self, shape, device):
            self.shape = shape

    class Caches:
        def __init__(self, shape, n_seqs, device):
            self.pages = 2 * -(-(shape.budget + shape.slack) // shape.page)

        def bytes_per_sequence(self):
            return self.pages * per_page

    monkeypatch.setattr(served, "Block", Block)
    monkeypatch.setattr(served, "Caches", Caches)
    monkeypatch.setattr(served, "step_seconds", lambda block, n: 1.0)
    monkeypatch.setattr(served, "prompt_seconds", lambda block, lengths: seen.append(lengths) or 0.5)
    p = served.measure(shape, tokens=29, requests=1, batch=2, prompt=100)
    assert seen == [[100], [100, 100]] and p.latency == pytest.approx(3 * 29.5)
    assert p.weight_mib * (1 << 20) >= 3 * -(-129 // shape.page) * per_page


def test_the_command_refuses_it_too(capsys):
    from paper_2302_11665_amd import served
    for argv in (["--prompt", "961"], ["--prompt", "100000"], ["--prompt", "-1"]):
        with pytest.raises(SystemExit) as e:
            served.main(argv)
        assert e.value.code == 2 and "960" in capsys.readouterr().err
