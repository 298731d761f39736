"""A handler of the operators' warnings that changes the lists which were passed: the call takes what they hold then, or refuses."""
import warnings

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    from paper_2207_09682_b200 import binding
    c = binding.Context(binding.make_params())
    yield c
    c.close()


def told(monkeypatch, do):
    """Warnings are shown by `do`; their number."""
    count = []

    def show(*args, **kwargs):
        count.append(str(args[0]))
        do()
    monkeypatch.setattr(warnings, "showwarning", show)
    return count


def ones(n, k=3):
    return [torch.ones(n, device="cuda") for _ in range(k)]


def test_adamw(ctx, monkeypatch):
    from paper_2207_09682_b200 import binding
    for replaced in (False, True):
        p, m, v, copies = ones(300), ones(300), ones(300), ones(300)
        g = [t.requires_grad_() for t in ones(300)]
        old = (p[1], m[1], v[1], copies[2])

        def change():
            if replaced:
                p[1], m[1], v[1], copies[2] = *ones(300), None
            else:
                g.clear()
        with warnings.catch_warnings():
            warnings.simplefilter("always")
            count = told(monkeypatch, change)
            if replaced:
                ctx.adamw(p, g, m, v, 1, 0.1, copies=copies)
                assert all(bool((t == 1).all()) for t in old) and all(bool((t != 1).all()) for t in (*p, *copies[:2]))
            else:
                with pytest.raises(binding.QgbdtError):
                    ctx.adamw(p, g, m, v, 1, 0.1, copies=copies)
                assert all(bool((t == 1).all()) for t in (*p, *m, *v, *copies))
        assert len(count) == 1


def test_clip_grad_norm(ctx, monkeypatch):
    g = [t.requires_grad_() for t in ones(300)]
    with warnings.catch_warnings():
        warnings.simplefilter("always")
        count = told(monkeypatch, lambda: g.__setitem__(slice(None), ones(400, 2)))
        assert abs(float(ctx.clip_grad_norm(g, float("inf"))) - 800 ** 0.5) < 1e-4 and len(count) == 1
        # a generator gives its tensors once
        count = told(monkeypatch, lambda: None)
        g = [t.requires_grad_() for t in ones(300)]
        out = [torch.zeros(300, device="cuda") for _ in g]
        norm = ctx.clip_grad_norm((t for t in g), 1.0, out=(t for t in out))
        assert abs(float(norm) - 30.0) < 1e-4 and len(count) == 1 and all(bool(((t - 1 / 30).abs() < 1e-6).all()) for t in out)
