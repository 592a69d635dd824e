"""CPU test of where the binding's calls allocate: with `stream`, every output and workspace that a call makes is that
stream's memory. The caching allocator orders reuse with the stream of the allocation only, so a workspace of another
stream's memory would be handed out again while the call's kernels run."""
import contextlib

import pytest

torch = pytest.importorskip("torch")


class DeviceTensor(torch.Tensor):
    """A host tensor that passes for a device tensor; no kernel runs here."""
    is_cuda = property(lambda self: True)


def T(shape, dtype=torch.float32):
    return torch.zeros(shape, dtype=dtype).as_subclass(DeviceTensor)


class Library:
    """Every entry point succeeds without doing anything."""
    def __getattr__(self, name):
        return lambda *args: 0


class SideStream:
    cuda_stream = 0x7777


def calls(pace):
    i32, i64, f64, u8, i8 = torch.int32, torch.int64, torch.float64, torch.uint8, torch.int8
    tags, off, comp, score, keep, goff = T(10, i32), T(4, i64), T(3, i32), T(3, f64), T(3, u8), T(3, i64)
    z, ids = T((3, 8)), T(3, i32)
    return {
        "score": lambda **s: pace.pace_score(tags, off, comp, 1, **s),
        "select": lambda **s: pace.pace_select(score, 1, **s),
        "compact": lambda **s: pace.pace_compact(off, keep, [tags], **s),
        "validate": lambda **s: pace.pace_validate(tags, off, comp, 1, **s),
        "filter_step": lambda **s: pace.pace_filter_step(tags, off, comp, 1, 3, 2, [tags], **s),
        "group_score": lambda **s: pace.pace_group_score(score, goff, **s),
        "group_expand": lambda **s: pace.pace_group_expand(goff, T(2, u8), 3, **s),
        "validate_groups": lambda **s: pace.pace_validate_groups(goff, 3, **s),
        "group_filter_step": lambda **s: pace.pace_group_filter_step(tags, off, comp, 1, goff, 2, 1, [tags], **s),
        "stream_admit": lambda **s: pace.pace_stream_admit(score, 0.5, pace.StreamWindow(8, "cpu"), 2, **s),
        "stream_step": lambda **s: pace.pace_stream_step(tags, off, comp, 1, 3, 2, [tags], pace.StreamWindow(8, "cpu"), 2, **s),
        "prefix_score": lambda **s: pace.pace_prefix_score(T(10), T(10), off, **s),
        "stale_k": lambda **s: pace.pace_stale_k(T(3, i64), T(3, i64), comp, 1, 2, **s),
        "diagnostics": lambda **s: pace.pace_diagnostics(score, T(3, i64), T(3, i64), comp, 1, keep, T((3, 5), f64), **s),
        "token_logprob": lambda **s: pace.pace_token_logprob(z, ids, top_k=2, **s),
        "token_logprob_backward": lambda **s: pace.pace_token_logprob_backward(z, ids, T((3, 2)), T(3), **s),
        "policy_loss": lambda **s: pace.pace_policy_loss(T(10), T(10), off, T(3), **s),
        "quantize_rows": lambda **s: pace.pace_quantize_rows(z, **s),
        "matmul_i8": lambda **s: pace.pace_matmul_i8(T((3, 8), i8), T(3), T((5, 8), i8), T(5), **s),
        "orthogonalize": lambda **s: pace.pace_orthogonalize(z, **s),
    }


@pytest.mark.parametrize("name", sorted(calls(None)))
def test_a_call_allocates_in_its_streams_memory(monkeypatch, name):
    import paper_2609_36830_amd as pace
    inside, made = [], []
    empty, empty_like = torch.empty, torch.empty_like

    @contextlib.contextmanager
    def under(stream):
        inside.append(stream)
        yield
        inside.pop()

    def record(make):
        def f(*args, **kw):
            made.append(inside[-1] if inside else None)
            t = make(*args, **kw)
            return t.as_subclass(DeviceTensor)
        return f

    monkeypatch.setattr(pace, "lib", Library)
    monkeypatch.setattr(pace, "_stream", lambda device, stream=None: 0)
    monkeypatch.setattr(torch.cuda, "stream", under)
    monkeypatch.setattr(torch.cuda, "Stream", SideStream)
    monkeypatch.setattr(torch, "empty", record(empty))
    monkeypatch.setattr(torch, "empty_like", record(empty_like))
    call, side = calls(pace)[name], SideStream()
    call()
    assert made and not any(made)
    plain = len(made)
    call(stream=side)
    assert len(made) == 2 * plain and all(s is side for s in made[plain:])
