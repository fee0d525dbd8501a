"""PagedPath with several beams per prompt: a step that gets no pages, and attention to states in some of the layers only."""
import pytest
import torch

import beam_reference as R
import paper_2412_03409_amd as P
from paper_2412_03409_amd.pipeline import PagedPath
from test_gpu_beam import select_inputs
from test_gpu_serving import BF16, DEV, close, f64, gen, i32, offsets, projected

pytestmark = pytest.mark.gpu
L, H, HKV, D, PS, BEAMS, G, V, END = 2, 2, 1, 64, 16, 2, 2, 101, 7


def path_of(num_pages):
    return PagedPath(G * BEAMS, L, H, HKV, D, torch.tensor([0.2, 0.1]).to(DEV), P.rope_plan(D, device=DEV), num_pages=num_pages,
                     max_pages=4, page_size=PS, device=DEV, beams=BEAMS)


def rows(T, seed):
    return (*projected(gen(seed), L, H, HKV, T, D, BF16), torch.arange(T, dtype=torch.int32, device=DEV)[None])


@pytest.mark.parametrize("with_end", [False, True])
def test_a_step_that_gets_no_pages_has_no_continuations(with_end):
    """24 entries a layer are two pages each, and two beams that continue them need a page more in both: with one free nothing may look
    as if it had been chosen, not even behind a later call that sets `status` anew."""
    path = path_of(2 * L + 1)
    path.prefill([0], [24], *rows(24, 1), [24 * L])
    assert int(path.status) == 0 and path.cache.lens.tolist() == [[24, 24]] + [[0, 0]] * 3
    x, _, _ = select_inputs(2, G, BEAMS, V, BF16)
    x, kw = x.to(DEV), dict(end_token=END) if with_end else {}
    scores = torch.tensor([[0.0, float("-inf")]] * G, device=DEV)
    before = [t.clone() for t in (path.cache.table, path.cache.lens, path.cache.ring, path.cache.state, scores)]
    got = path.advance(x, scores, **kw)
    assert int(path.status) == 1
    assert bool((got[0] == -1).all()) and bool((got[1] == -1).all()) and bool(torch.isneginf(got[2]).all())
    assert not bool(got[3].any()) if with_end else got[3] is None
    for a, b in zip((path.cache.table, path.cache.lens, path.cache.ring, path.cache.state, scores), before):
        assert torch.equal(a, b)
    # the same step with a prompt fewer: what the first call was given is still there
    again = scores.clone()
    again[0] = float("-inf")
    path.advance(x, again, **kw)
    assert int(path.status) == 0 and int(path.cache.lens.sum()) == 0
    # a caller that goes on all the same finds no beam
    path.extend([0] * 4, *rows(1, 3))
    assert int(path.status) == 0
    got = path.advance(x, got[2], **kw)
    assert int(path.status) == 0 and bool((got[1] == -1).all()) and bool(torch.isneginf(got[2]).all())


def test_a_step_that_gets_its_pages_is_the_choice():
    path = path_of(4 * L)
    path.prefill([0], [24], *rows(24, 1), [24 * L])
    x, scores, ended = select_inputs(5, G, BEAMS, V, BF16, END)
    x, scores, ended = x.to(DEV), scores.to(DEV), ended.to(DEV)
    want = P.prefixkv_beam_select(x, scores, ended=ended, end_token=END)
    got = path.advance(x, scores, ended=ended, end_token=END)
    assert int(path.status) == 0 and all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("layers", [[0], [1], [1, 0, 1]])
def test_attention_to_states_in_other_layers_than_the_paths(layers):
    """A model may attend to its encoder's states in some of its layers, all at once or one after the other, and with a scale of its own."""
    path, g = path_of(8), gen(len(layers))
    lengths, m = [1, 3, 0, 2], [40, 70]
    q, _, _ = projected(g, len(layers), H, HKV, sum(lengths), D, BF16)
    kv = torch.randn((len(layers), 2 * HKV, sum(m), D), generator=g).to(BF16).to(DEV)
    k, v, to = kv[:, :HKV], kv[:, HKV:], offsets(m)
    for scale in (path.scale[layers], torch.full((len(layers),), -0.3, device=DEV)):
        out = path.cross(lengths, q, k, v, i32(to), scale=scale)
        want, mag = R.cross(f64(q), offsets([4, 2]), f64(k), f64(v), to, scale.double().cpu().numpy())
        close(out, want, mag, BF16)
    if len(layers) != L:
        with pytest.raises(ValueError, match="scale"):
            path.cross(lengths, q, k, v, i32(to))
