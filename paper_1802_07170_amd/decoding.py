"""Decoding in small numbers, on torch tensors: products with 4-bit weights, attention over source rows held in 8 bits, and a
beam search's choice with the states that follow it.  What the functions compute is defined in include/cytonmt_hip.h; this module checks
its arguments, makes the tensors that are returned, and calls the library.

Calls are enqueued on torch's current stream of the tensors' device and may be captured into a graph.  Nothing here is differentiable:
a tensor that wants a gradient is refused.  There is no CPU fallback."""
from __future__ import annotations

import ctypes as C
import functools
import struct

import numpy as np
import torch

from . import binding
from .binding import CMT_OK, CmtCacheConfig, CmtCacheRows, CmtError

_TYPES = {torch.float32: 0, torch.bfloat16: 1}


def _check(rc):
    if rc != CMT_OK:
        raise CmtError(rc, binding.load_library().cmt_operator_error().decode())


def _tensor(t, name, dims, dtypes, device=None):
    """Refuses what the kernels do not take: the last dimension's elements lie side by side, the other strides are free."""
    if not isinstance(t, torch.Tensor) or t.dim() not in dims:
        raise ValueError(f"{name} must be a tensor of {' or '.join(map(str, dims))} dimensions")
    if t.dtype not in dtypes:
        raise ValueError(f"{name} must be of {' or '.join(str(d) for d in dtypes)}, not {t.dtype}")
    if not t.is_cuda:
        raise ValueError(f"{name} must be on a GPU, not on {t.device}")
    if device is not None and t.device != device:
        raise ValueError(f"{name} is on {t.device}, the other tensors on {device}")
    if t.stride(-1) != 1 and t.shape[-1] > 1:
        raise ValueError(f"{name}: the elements of the last dimension must lie side by side")
    if t.requires_grad and torch.is_grad_enabled():
        raise ValueError(f"{name} wants a gradient: these operators have none (use torch.no_grad())")


def _pitch(t):
    """Elements from one row of a matrix to the next."""
    return t.stride(0) if t.shape[0] > 1 else t.shape[1]


def _call(f, device, *args):
    """f(*args, stream) with the tensors' device as the current one and its current stream.  (torch's own way to the
    stream's handle builds a Stream object for it: 1.9 us of the 4 that a launch takes.)"""
    if device.index == torch._C._cuda_getDevice():
        rc = f(*args, torch._C._cuda_getCurrentRawStream(device.index))
    else:
        with torch.cuda.device(device):
            rc = f(*args, torch._C._cuda_getCurrentRawStream(device.index))
    if rc != CMT_OK:
        _check(rc)


class QuantWeight:
    """A weight [outputs, inputs] in 4 bits, with a bf16 scale for every `group` (32, 64 or 128) inputs of a row."""

    def __init__(self, outputs, inputs, group, device):
        size = C.c_size_t()
        _check(binding.load_library().cmt_quant_weight_bytes(outputs, inputs, group, C.byref(size)))
        self.outputs, self.inputs, self.group = outputs, inputs, group
        self.packed = torch.empty(size.value, dtype=torch.uint8, device=device)

    @property
    def device(self):
        return self.packed.device

    @classmethod
    def pack(cls, weight, group=64):
        """From a weight [outputs, inputs] in fp32 or bf16: scale = bf16(max|w| / 6) and the nearest codes."""
        _tensor(weight, "weight", (2,), _TYPES)
        w = cls(*weight.shape, group, weight.device)
        _call(binding.load_library().cmt_quant_weight_pack, w.device, weight.data_ptr(), _TYPES[weight.dtype], _pitch(weight), w.outputs, w.inputs,
              group, w.packed.data_ptr())
        return w

    @classmethod
    def from_codes(cls, codes, scales, group):
        """From e2m1 codes [outputs, inputs] (uint8, one to a byte) and bf16 scales [outputs, ceil(inputs / group)]."""
        _tensor(codes, "codes", (2,), (torch.uint8,))
        _tensor(scales, "scales", (2,), (torch.bfloat16,), codes.device)
        w = cls(*codes.shape, group, codes.device)
        if tuple(scales.shape) != (w.outputs, -(-w.inputs // group)):
            raise ValueError(f"scales must be {(w.outputs, -(-w.inputs // group))}, not {tuple(scales.shape)}")
        if not codes.is_contiguous() or not scales.is_contiguous():
            raise ValueError("codes and scales must be contiguous")
        _call(binding.load_library().cmt_quant_weight_encode, w.device, codes.data_ptr(), scales.data_ptr(), w.outputs, w.inputs, group,
              w.packed.data_ptr())
        return w

    def values(self):
        """The weight that the codes stand for, fp32 [outputs, inputs]."""
        out = torch.empty(self.outputs, self.inputs, dtype=torch.float32, device=self.device)
        _call(binding.load_library().cmt_quant_weight_values, self.device, self.packed.data_ptr(), self.outputs, self.inputs, self.group, out.data_ptr())
        return out


def quant_product(x, weight, bias=None, tanh=False, out_dtype=None, out=None):
    """x [rows, inputs] (fp32 or bf16) times the 4-bit weight's transpose, plus an fp32 bias [outputs], through tanh if asked for:
    [rows, outputs] in `out_dtype` (x's type if None), or in `out`."""
    packed, outputs, inputs = weight.packed, weight.outputs, weight.inputs
    device = packed.device
    _tensor(x, "x", (2,), _TYPES, device)
    rows, columns = x.shape
    if columns != inputs:
        raise ValueError(f"x has {columns} columns, the weight {inputs} inputs")
    if bias is not None:
        _tensor(bias, "bias", (1,), (torch.float32,), device)
        if len(bias) != outputs:
            raise ValueError(f"bias has {len(bias)} elements, the weight {outputs} outputs")
    if out is None:
        dtype = x.dtype if out_dtype is None else out_dtype
        if dtype not in _TYPES:
            raise ValueError(f"out_dtype must be torch.float32 or torch.bfloat16, not {dtype}")
        out, pitch = x.new_empty((rows, outputs), dtype=dtype), outputs
    else:
        _tensor(out, "out", (2,), _TYPES if out_dtype is None else (out_dtype,), device)
        if tuple(out.shape) != (rows, outputs):
            raise ValueError(f"out must be {(rows, outputs)}, not {tuple(out.shape)}")
        _apart(out, "out", x, "x")
        dtype, pitch = out.dtype, _pitch(out)
    _call(binding.load_library().cmt_quant_product, device, x.data_ptr(), _TYPES[x.dtype], x.stride(0) if rows > 1 else inputs, rows, packed.data_ptr(),
          outputs, inputs, weight.group, None if bias is None else bias.data_ptr(), bool(tanh), out.data_ptr(), _TYPES[dtype], pitch)
    return out


def _apart(a, name, b, other):
    """Refuses two tensors of rows (first dimension; the others side by side) that share memory.  Columns of one matrix may lie beside each other."""
    (a0, ap, an, al), (b0, bp, bn, bl) = ((t.data_ptr(), t.stride(0) * t.element_size(), t.shape[0], t[0].numel() * t.element_size() if len(t) else 0)
                                          for t in (a, b))
    if not (an and bn and al and bl) or a0 >= b0 + (bn - 1) * bp + bl or b0 >= a0 + (an - 1) * ap + al:
        return
    ahead = (b0 - a0) % ap if ap > 0 else 0
    if ap != bp or an == 1 or bn == 1 or ahead < al or ahead + bl > ap:
        raise ValueError(f"{name} overlaps {other}")


class SourceCache:
    """Keys and values of up to `max_tokens` tokens of each sequence in 8 bits, a scale for every 32 tokens and head."""

    def __init__(self, sequences, heads, head_dim, max_tokens, device="cuda"):
        self.config = CmtCacheConfig(sequences, heads, head_dim, max_tokens)
        size = C.c_size_t()
        _check(binding.load_library().cmt_cache_bytes(C.byref(self.config), C.byref(size)))
        self.sequences, self.heads, self.head_dim, self.max_tokens = sequences, heads, head_dim, max_tokens
        self.data = torch.empty(size.value, dtype=torch.uint8, device=device)
        self.tokens = 0                                    # bound of the lengths, from the last fill
        self._needs = {}                                   # bytes of workspace by (tokens, rows per sequence, query heads)

    @property
    def device(self):
        return self.data.device

    def fill(self, keys, values, lengths):
        """Writes tokens [0, lengths[s]) of every sequence: keys, values [sequences, tokens, heads, head_dim] in fp32 or bf16, lengths int32
        [sequences] on the device (clamped to [0, tokens])."""
        _tensor(keys, "keys", (4,), _TYPES, self.device)
        _tensor(values, "values", (4,), (keys.dtype,), self.device)
        _tensor(lengths, "lengths", (1,), (torch.int32,), self.device)
        want = (self.sequences, keys.shape[1], self.heads, self.head_dim)
        if tuple(keys.shape) != want or tuple(values.shape) != want or not 1 <= want[1] <= self.max_tokens:
            raise ValueError(f"keys and values must be ({self.sequences}, 1..{self.max_tokens}, {self.heads}, {self.head_dim}), not "
                             f"{tuple(keys.shape)} and {tuple(values.shape)}")
        if lengths.shape[0] != self.sequences:
            raise ValueError(f"lengths must have {self.sequences} elements, not {lengths.shape[0]}")
        rows = [CmtCacheRows(t.data_ptr(), *t.stride()[:3]) for t in (keys, values)]
        _call(binding.load_library().cmt_cache_fill, self.device, self.config, self.data.data_ptr(), *rows, _TYPES[keys.dtype], lengths.data_ptr(), want[1])
        self.tokens = want[1]
        return self

    def read(self):
        """The keys and values that the cache stands for: fp32 [sequences, tokens of the last fill, heads, head_dim], 0 behind a length."""
        self._filled()
        keys = torch.empty(self.sequences, self.tokens, self.heads, self.head_dim, dtype=torch.float32, device=self.device)
        values = torch.empty_like(keys)
        _call(binding.load_library().cmt_cache_read, self.device, self.config, self.data.data_ptr(), self.tokens, keys.data_ptr(), values.data_ptr())
        return keys, values

    def attend(self, query, scale=1.0, out=None):
        """Attention of query [rows, query heads, head_dim] (fp32 or bf16): rows a multiple of the sequences, row r belonging to sequence
        r // (rows / sequences); query heads a multiple of the heads, in order.  Returns the same shape and type (0 for a sequence of
        length 0)."""
        self._filled()
        data = self.data
        device = data.device
        _tensor(query, "query", (3,), _TYPES, device)
        rows, heads, dim = query.shape
        if rows == 0 or rows % self.sequences or heads == 0 or heads % self.heads or dim != self.head_dim:
            raise ValueError(f"query must be (a multiple of {self.sequences}, a multiple of {self.heads}, {self.head_dim}), not {tuple(query.shape)}")
        if out is None:
            out = query.new_empty((rows, heads, dim))
        else:
            _tensor(out, "out", (3,), (query.dtype,), device)
            if out.shape != query.shape:
                raise ValueError(f"out must be {tuple(query.shape)}, not {tuple(out.shape)}")
            _apart(out, "out", query, "query")
        q_pitch, o_pitch = query.stride(), out.stride()
        if heads > 1 and (q_pitch[1] != dim or o_pitch[1] != dim):
            raise ValueError(f"{'query' if q_pitch[1] != dim else 'out'}: the heads of a row must lie side by side")
        lib, per = binding.load_library(), rows // self.sequences
        key = (self.tokens, per, heads)
        need = self._needs.get(key)
        if need is None:
            size = C.c_size_t()
            _check(lib.cmt_cache_attend_workspace(C.byref(self.config), per, heads, self.tokens, C.byref(size)))
            need = self._needs[key] = size.value
        work = data.new_empty(need) if need else None
        _call(lib.cmt_cache_attend, device, self.config, data.data_ptr(), query.data_ptr(), _TYPES[query.dtype],
              q_pitch[0] if rows > 1 else heads * dim, per, heads, self.tokens, scale, out.data_ptr(), o_pitch[0] if rows > 1 else heads * dim,
              None if work is None else work.data_ptr(), need)
        return out

    def _filled(self):
        if not self.tokens:
            raise ValueError("the cache has not been filled")


@functools.lru_cache(maxsize=256)
def _select_workspace(sentences, beam, vocab):
    size = C.c_size_t()
    _check(binding.load_library().cmt_beam_select_workspace(sentences, beam, vocab, C.byref(size)))
    return size.value


def beam_select(logits, scores, n=None):
    """The n (the beam if None) best one-token extensions of each sentence's hypotheses: logits [sentences * beam, vocab] (fp32 or bf16), scores
    fp32 [sentences, beam], -inf for a place without a hypothesis.  Returns scores fp32, rows int32 (b * beam + s, the
    hypothesis that is extended) and tokens int32, [sentences, n] each: best first, of equal ones the lower (row, token), and -inf, -1, -1 where
    there are fewer."""
    _tensor(logits, "logits", (2,), _TYPES)
    _tensor(scores, "scores", (2,), (torch.float32,), logits.device)
    (sentences, beam), (rows, vocab) = scores.shape, logits.shape
    if rows != sentences * beam:
        raise ValueError(f"logits have {rows} rows, scores {sentences} x {beam} places")
    if not scores.is_contiguous():
        raise ValueError("scores must be contiguous")
    n, device, pitch = beam if n is None else n, logits.device, logits.stride(0) if rows > 1 else vocab
    need = _select_workspace(sentences, beam, vocab)
    if not isinstance(n, int) or n < 1:
        raise ValueError(f"n must be a positive number, not {n!r}")
    new = scores.new_empty((sentences, n))
    rows, tokens = scores.new_empty((2, sentences, n), dtype=torch.int32).unbind(0)
    work = scores.new_empty(need // 4)
    _call(binding.load_library().cmt_beam_select, device, logits.data_ptr(), _TYPES[logits.dtype], pitch, scores.data_ptr(), sentences, beam,
          vocab, n, new.data_ptr(), rows.data_ptr(), tokens.data_ptr(), work.data_ptr(), need)
    return new, rows, tokens


def beam_reorder(rows, sources, targets):
    """targets[i][r] = sources[i][rows[r]] for all tensors in one launch per 32: rows int32 of any shape (as beam_select returns them), the
    tensors' first dimension counting rows, the others contiguous.  Target rows whose number is outside the source stay as they were."""
    if not isinstance(rows, torch.Tensor) or rows.dtype != torch.int32 or not rows.is_contiguous() or not rows.is_cuda:
        raise ValueError("rows must be a contiguous int32 tensor on a GPU")
    if len(sources) != len(targets):
        raise ValueError(f"{len(sources)} sources and {len(targets)} targets")
    if not sources:
        return
    count, source_rows, device, grad = rows.numel(), sources[0].shape[:1], rows.device, torch.is_grad_enabled()
    source_rows = source_rows[0] if source_rows else -1
    fields = []                                            # of a CmtReorderTensor each: five numbers of 64 bits
    for i, (a, b) in enumerate(zip(sources, targets)):
        sa, sb = a.shape, b.shape
        if not sa or not sb or sa[0] != source_rows or sb[0] != count or (sa != sb if count == source_rows else sa[1:] != sb[1:]):
            raise ValueError(f"tensors {i} must have {source_rows} and {count} rows alike, not {tuple(sa)} and {tuple(sb)}")
        if a.dtype != b.dtype or a.device != device or b.device != device:
            raise ValueError(f"tensors {i} must be of one type and on the device of rows")
        if grad and (a.requires_grad or b.requires_grad):
            raise ValueError(f"tensors {i} want a gradient: these operators have none (use torch.no_grad())")
        width = a.nbytes // source_rows if source_rows else 0
        if width:
            fields += (a.data_ptr(), b.data_ptr(), width if a.is_contiguous() else _row_pitch(a, i),
                       width if b.is_contiguous() else _row_pitch(b, i), width)
    if not fields or not count:
        return
    _call(binding.load_library().cmt_beam_reorder, device, rows.data_ptr(), count, source_rows, struct.pack(f"{len(fields)}q", *fields), len(fields) // 5)


def _row_pitch(t, i):
    """Bytes from one row (first dimension) to the next, whose own elements lie side by side."""
    side = 1
    for d in range(t.dim() - 1, 0, -1):
        if t.shape[d] > 1 and t.stride(d) != side:
            raise ValueError(f"tensors {i}: the elements of a row must lie side by side")
        side *= t.shape[d]
    return (t.stride(0) if t.shape[0] > 1 else side) * t.element_size()


class QuantDecoder:
    """A trainer's decoder in small numbers: its weights, W_c and the output layer in 4 bits, the source rows in 8.  The weights are those that the
    trainer has when this is made; `pack` renews them."""

    def __init__(self, trainer, group=64):
        weights, workspace = C.c_size_t(), C.c_size_t()
        if trainer.lib.cmt_quant_decoder_bytes(C.byref(trainer.ccfg), group, C.byref(weights), C.byref(workspace)) != CMT_OK:
            raise CmtError(binding.CMT_EINVAL, "group must be 32, 64 or 128")
        self.trainer, self.group = trainer, group
        with torch.cuda.stream(trainer.stream):
            self.weights = torch.empty(weights.value, dtype=torch.uint8, device=trainer.device)
            self.workspace = torch.empty(workspace.value, dtype=torch.uint8, device=trainer.device)
        self.pack()

    def pack(self):
        """Writes the packed weights from the trainer's parameters."""
        tr = self.trainer
        tr._check(tr.lib.cmt_quant_decoder_pack(tr.h, self.group, self.weights.data_ptr()))

    def beam_decode(self, src_ids, src_len, max_len, beam=10, length_penalty=0.6, eos_id=3):
        """As Trainer.beam_decode: ids [B, max_len], lengths [B], normalised scores [B] (numpy)."""
        tr = self.trainer
        src, lens = (torch.from_numpy(np.ascontiguousarray(a, np.int32)).to(tr.device) for a in (src_ids, src_len))
        if src.dim() != 2 or tuple(lens.shape) != src.shape[:1]:
            raise ValueError(f"src_ids must be [B, S] and src_len [B], not {tuple(src.shape)} and {tuple(lens.shape)}")
        B, S = src.shape
        out = torch.empty((B, max_len), dtype=torch.int32, device=tr.device)
        length = torch.empty((B,), dtype=torch.int32, device=tr.device)
        score = torch.empty((B,), dtype=torch.float32, device=tr.device)
        torch.cuda.synchronize(tr.device)
        tr._check(tr.lib.cmt_quant_beam_decode(tr.h, self.group, self.weights.data_ptr(), self.workspace.data_ptr(), src.data_ptr(), lens.data_ptr(),
                                               B, S, max_len, beam, length_penalty, eos_id, out.data_ptr(), length.data_ptr(), score.data_ptr()))
        return out.cpu().numpy(), length.cpu().numpy(), score.cpu().numpy()

    def greedy_decode(self, src_ids, src_len, max_len, eos_id=3):
        """As Trainer.greedy_decode: ids [B, max_len], lengths [B]."""
        return self.beam_decode(src_ids, src_len, max_len, beam=1, length_penalty=0.0, eos_id=eos_id)[:2]
