"""A whole quantized network on the GPU: the CIFAR-10-shaped QNN of the
paper's end-to-end evaluation (Sec. V-E): three 5x5 convolutions with
requantization + ReLU clip, each followed by 2x2 max-pooling, then a fully
connected classifier with int32 logits.  Every layer is one library call on
one stream; activations stay in device memory between calls.

And the step of a language model that checks a tree of drafted tokens, over
packed weights and packed caches (lm.py): decoder_block, tree_step and
accept_path.
"""
from . import qnn


def cifar_forward(x, n, bits, cin, convs, fc, clip, stream=None, keep=False, fused=True):
    """Run the network on packed NHWC input `x` (n x 32 x 32 x cin codes).

    convs: list of dicts with device tensors "w", "bias", "mult", "shift" and
    ints "m", "k", "pad"; fc: dict with "w", "bias", "m".  Each convolution
    runs fused with its 2x2 max-pooling (qnn_conv2d_maxpool), or, with
    fused=False, as a convolution followed by a separate pooling.  Returns
    the int32 logits [n, 1, 1, m] (and the list of intermediate activations
    if keep: pooled outputs, preceded by the convolution outputs when not
    fused).
    """
    h = w = 32
    c = cin
    acts = []
    for cv in convs:
        args = (bits, cv["w"], cv["m"], cv["k"], cv["k"], (1, 1), (cv["pad"], cv["pad"]), "requant")
        kw = dict(bias=cv["bias"], mult=cv["mult"], shift=cv["shift"], clip=clip, stream=stream)
        ho = (h + 2 * cv["pad"] - cv["k"]) + 1
        wo = (w + 2 * cv["pad"] - cv["k"]) + 1
        if fused:
            x = qnn.conv2d_maxpool(x, (n, h, w, c), *args, **kw)
            if keep:
                acts.append(x)
        else:
            y = qnn.conv2d(x, (n, h, w, c), *args, **kw)
            x = qnn.maxpool2d(y, (n, ho, wo, cv["m"]), bits, 2, 2, 2, 2, stream=stream)
            if keep:
                acts += [y, x]
        h, w, c = ho // 2, wo // 2, cv["m"]
    logits = qnn.linear(x, (n, h, w, c), bits, fc["w"], fc["m"], "raw32", bias=fc["bias"],
                        stream=stream)
    return (logits, acts) if keep else logits


def _layer(x, layer, stream, **epilogue):
    from . import lm
    return lm.matmul(x, layer["w"], layer["bits"], scale=layer.get("scale"), bias=layer.get("bias"), stream=stream,
                     **epilogue)


def decoder_block(h, x, block, cache, table, lens, mask=None, counts=None, stream=None):
    """One decoder block over the drafted tokens of a batch: attention over the
    packed cache, then a gated feed-forward layer, each between two norms.

    h, x: [b, t, d], the residual stream (x's type or float32) and its norm.
    block: a dict with
      "heads", "kv_heads", "dim"       numbers of heads and channels of a head
      "qkv", "out", "up", "down"       layers: dicts of "w", "bits" and, as lm.matmul
                                       takes them, "scale" and "bias"; "up" holds the
                                       gate's rows first
      "act"                            the gate's activation
      "norm", "eps"                    as lm.norm_residual takes them
      "attn_norm", "mlp_norm"          weights [d] of the norms after the two halves, or None
      "mid_norm", "next_norm"          of the norms before the feed-forward layer and the next block
      "alpha", "beta"                  scales of the residual stream and of a half's result
    cache: a lm.Cache; table, lens, mask, counts: as lm.tree_attention takes them.
    The block does not turn queries and keys by their positions: these are to be
    part of the embedding.  Writes the drafts' keys and values behind lens and
    returns (h, x) for the next block."""
    from . import lm
    b, t, d = x.shape
    heads, kv, dim = block["heads"], block["kv_heads"], block["dim"]
    qkv = _layer(x, block["qkv"], stream).view(b, t, heads + 2 * kv, dim)
    lm.cache_append(qkv[:, :, heads:heads + kv], qkv[:, :, heads + kv:], cache, table, lens, counts=counts, stream=stream)
    o = lm.tree_attention(qkv[:, :, :heads], cache, table, lens, mask=mask, counts=counts, stream=stream)
    norms = dict(norm=block["norm"], eps=block["eps"], alpha=block["alpha"], beta=block["beta"], stream=stream)
    h, x = lm.norm_residual(h, _layer(o.view(b, t, heads * dim), block["out"], stream),
                            post=block["attn_norm"] is not None, post_weight=block["attn_norm"],
                            pre_weight=block["mid_norm"], **norms)
    u = _layer(x, block["up"], stream, act=block["act"], gated=True)
    return lm.norm_residual(h, _layer(u, block["down"], stream), post=block["mlp_norm"] is not None,
                            post_weight=block["mlp_norm"], pre_weight=block["next_norm"], **norms)


def tree_step(h, first_norm, blocks, caches, table, lens, mask=None, counts=None, dtype=None, stream=None):
    """Every block over the drafted tokens: h [b, t, d] embedded drafts -> (h, x),
    x being the last norm's result, for the model's logits.  caches: one
    lm.Cache a block; dtype: of the activations, if h is float32."""
    from . import lm
    _, x = lm.norm_residual(h, norm=blocks[0]["norm"], eps=blocks[0]["eps"], pre_weight=first_norm, dtype=dtype,
                            stream=stream)
    for block, cache in zip(blocks, caches):
        h, x = decoder_block(h, x, block, cache, table, lens, mask=mask, counts=counts, stream=stream)
    return h, x


def accept_path(caches, table, lens, path, kept, stream=None):
    """After the drafts of a step have been judged: the accepted ones (path, kept
    as lm.cache_keep takes them) become the tokens behind lens in every block's
    cache.  Returns the new lens, like them computed on `stream`."""
    from . import lm
    if stream is not None:
        with lm._on(stream, *caches, table, lens, path, kept):
            return accept_path(caches, table, lens, path, kept)
    for cache in caches:
        lm.cache_keep(cache, table, lens, path, kept)
    return lens + kept
