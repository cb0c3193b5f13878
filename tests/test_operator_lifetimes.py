"""Lifetimes around AdamW lists, without a GPU: a stand-in library that knows which handles are alive, behind the
binding's own classes."""
import ctypes as C
import gc
import weakref

import pytest
import torch

from paper_2505_23725_b200 import binding


class Library:
    """Counts handles; a call with one that is gone fails the test instead of reading freed memory."""

    def __init__(self):
        self.contexts, self.lists, self.steps, self.freed = {1}, {}, 0, 0

    def muloco_adamw_create(self, ctx, cfg, table, n, out):
        assert ctx.value in self.contexts
        handle = 100 + len(self.lists)
        self.lists[handle] = ctx.value
        out._obj.value = handle
        return binding.OK

    def _alive(self, opt):
        assert opt is not None and self.lists.get(opt.value) in self.contexts, "a handle that is gone"

    def muloco_adamw_step(self, opt, table, step, scale):
        self._alive(opt)
        self.steps += 1
        return binding.OK

    def muloco_adamw_moments(self, opt, m, v):
        self._alive(opt)
        return binding.OK

    def muloco_adamw_destroy(self, opt):
        self._alive(opt)
        del self.lists[opt.value]
        self.freed += 1

    def muloco_destroy(self, ctx):
        assert ctx.value in self.contexts and not self.lists, "lists outlive their context"
        self.contexts.discard(ctx.value)

    def muloco_last_error(self, ctx):
        return b""


class Owner(binding.Context):
    def __init__(self):
        self.torch, self.lib, self.device, self._dev = torch, Library(), torch.device("cpu"), -1
        self.ctx = C.c_void_p(1)
        self.stream = None
        self._fast, self._handle, self._raw_stream = {}, 7, lambda dev: 7
        self._bf16, self._f32, self._i64 = torch.bfloat16, torch.float32, torch.int64
        self._lists = weakref.WeakSet()


@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("own", [False, True], ids=["context closed", "list closed"])
def test_a_closed_list_refuses(bits, own):
    o = Owner()
    p, g = torch.ones(300), torch.ones(300)
    opt = binding.AdamW(o, [p], grads=[g], state_bits=bits)
    opt.step()
    (opt if own else o).close()
    for call in (opt.step, lambda: opt.step([g]), *([opt.moments] if bits == 8 else [])):
        with pytest.raises(RuntimeError, match="closed"):
            call()
    assert o.lib.steps == 1 and opt.steps == 1 and o.lib.freed == 1
    if bits == 32:
        assert opt.moments()[0] is opt.state1          # the states are the caller's tensors
    opt.close()                                    # once more is nothing
    o.close()
    assert o.lib.freed == 1 and not o.lib.contexts


def test_a_context_closes_its_lists_first():
    o = Owner()
    lists = [binding.AdamW(o, [torch.ones(5)]) for _ in range(3)]
    lists[1].close()
    o.close()
    assert o.lib.freed == 3 and not o.lib.contexts
    del lists
    gc.collect()
    assert o.lib.freed == 3


def test_a_closed_context_refuses_operators():
    o = Owner()
    o._fast = {"qk_norm_rope": (None, 0), "gated_ffn": (None, 0)}
    o.close()
    x = torch.ones(8, 8, dtype=torch.bfloat16)
    with pytest.raises(RuntimeError, match="closed"):
        o.gated_ffn(x, x, x, x)
    with pytest.raises(RuntimeError, match="closed"):
        o.qk_norm_rope(torch.ones(1, 1, 8), None, torch.ones(1, 4), torch.zeros(1, 4))


def test_tensors_named_at_construction_stay_alive():
    """The library's table holds their addresses: what the caller does to its own lists afterwards must not free them."""
    o = Owner()
    params, grads, copies = [torch.ones(300)], [torch.ones(300)], [torch.ones(300, dtype=torch.bfloat16)]
    opt = binding.AdamW(o, params, grads=grads, copies=copies)
    refs = [weakref.ref(l[0]) for l in (params, grads, copies)]
    for l in (params, grads, copies):
        l[0] = None
    gc.collect()
    assert all(r() is not None for r in refs)
    opt.step()
    opt.close()


@pytest.mark.parametrize("bits", [8, 32])
def test_states_made_on_another_stream_are_handed_over(bits):
    """The zeros of the states are written on the caller's current stream: the context's has to wait for it."""
    o, calls = Owner(), []
    o._other_stream = lambda: "caller's"
    o._enter = lambda cur, tensors: calls.append((cur, {t.data_ptr() for t in tensors if t is not None}))
    opt = binding.AdamW(o, [torch.ones(300)], state_bits=bits)
    states = [t for t in (opt.state1, opt.state2, opt.scale1, opt.scale2) if t is not None]
    assert len(calls) == 1 and calls[0][0] == "caller's" and {t.data_ptr() for t in states} <= calls[0][1]
    opt.close()
