"""The ends of what the serving layer of serve_layer.py takes."""
import pytest

torch = pytest.importorskip("torch")

from paper_2411_00915_amd import serve_layer


def quiet(monkeypatch):
    """The layer on the CPU, its calls without effect: the names of those that were made"""
    made = []
    monkeypatch.setattr(serve_layer, "DEV", "cpu")
    monkeypatch.setattr(serve_layer.Projection, "__call__", lambda self, x, lengths, adapters: torch.zeros((len(x), self.n), dtype=torch.bfloat16))
    for name in ("lora_attention", "lora_pages_resize", "lora_cache_copy", "lora_cache_append", "lora_cache_digest", "lora_cache_choose", "lora_cache_attention_chosen",
                 "lora_cache_attention", "lora_base_gemm", "lora_beam_select", "lora_pages_fork"):
        monkeypatch.setattr(serve_layer.B, name, lambda *a, name=name, **k: made.append(name))
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: type("none", (), {"synchronize": staticmethod(lambda: None)}))
    return made


def layer(requests, beams, limit, chosen=0):
    return serve_layer.BeamLayer(64, 2, 1, 32, [8], requests, beams, limit, 50, page=32, chosen=chosen)


@pytest.mark.parametrize("chosen", [0, 2])
def test_no_step_beyond_the_limit(monkeypatch, chosen):
    """The longest request's beams are at the limit after three steps; the next is refused before anything is enqueued"""
    made = quiet(monkeypatch)
    search = layer(3, 2, 40, chosen)
    for again in range(2):                                      # (prompts of their own begin anew)
        search.prompts(torch.zeros((60, 64)), [20, 37, 3], [0, 0, 0])
        for _ in range(3):
            search.step()
        del made[:]
        with pytest.raises(ValueError, match="limit"):
            search.step()
        assert made == []


@pytest.mark.parametrize("rows,lengths,adapters", [(23, [20, 0, 3], [0, 0, 0]), (20, [20], [0, 0, 0]), (20, [20], [0]), (24, [20, 4], [0, 0]), (60, [20, 37, 3], [0, 0]),
                                                   (59, [20, 37, 3], [0, 0, 0]), (61, [20, 37, 3], [0, 0, 0]), (61, [20, 41, 0], [0, 0, 0])])
def test_prompts_that_do_not_fit_the_requests(monkeypatch, rows, lengths, adapters):
    """An empty prompt has no last row (its neighbour's would be taken); one length would be every request's"""
    made = quiet(monkeypatch)
    search = layer(3, 2, 60)
    with pytest.raises(ValueError, match="request"):
        search.prompts(torch.zeros((rows, 64)), lengths, adapters)
    assert made == []


@pytest.mark.gpu
def test_steps_up_to_the_limit():
    """Prompts of unequal lengths: every beam gets all of its tokens, and tables and lengths are as they were behind the refusal"""
    search = layer(3, 2, 40)
    search.prompts(torch.randn((60, 64), device=serve_layer.DEV).bfloat16(), [20, 37, 3], [0, 0, 0])
    for i in range(3):
        search.step()
        assert search.granted.all()
    held = [x.clone() for x in (search.length, search.table, search.users, search.token, search.score)]
    assert sorted(set(held[0].tolist())) == [6, 23, 40]
    with pytest.raises(ValueError, match="limit"):
        search.step()
    assert all(torch.equal(a, b) for a, b in zip(held, (search.length, search.table, search.users, search.token, search.score)))
